"""What the norm of Q and K refuses, and the layout of its parameter blocks (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2205_14135_amd import binding
from paper_2205_14135_amd.autograd import flash_attention, norm_rotary_embedding
from paper_2205_14135_amd.rotary import HeadNorm, Rotary, rotary_frequencies

A, B, C, D, E, F = (ctypes.c_void_p(0x100000 * (i + 1)) for i in range(6))


@pytest.fixture(scope="module")
def lib():
    return binding.load()


def _rotary_params(**kw):
    p = binding.RotaryParams()
    p.B, p.N, p.d, p.dtype = 2, 8, 64, 1
    p.rotary.frequencies, p.rotary.rotary_dim, p.rotary.magnitude = 0x30000, 64, 1.0
    for k, v in kw.items():
        setattr(p.rotary if k in ("frequencies", "rotary_dim", "magnitude") else p, k, v)
    return p


def _norm(**kw):
    n = binding.NormSpec(0x40000, 0x50000, 1, 1e-6)
    for k, v in kw.items():
        setattr(n, k, v)
    return n


def _forward(lib, n=2, norm=None, params=None, tensor=None):
    t = (binding.RotaryTensor * 2)()
    for i in range(2):
        t[i].x, t[i].y, t[i].H = 0x100000 * (1 + 2 * i), 0x100000 * (2 + 2 * i), 4
        for a in "xy":
            for axis, s in zip("bhn", (4 * 8 * 64, 8 * 64, 64)):
                setattr(t[i], f"{a}_stride_{axis}", s)
    for k, v in (tensor or {}).items():
        setattr(t[0], k, v)
    return lib.attn_norm_rotary(ctypes.byref(_rotary_params(**(params or {}))), None if norm == "none" else ctypes.byref(_norm(**(norm or {}))), t, n)


BAD = [
    (dict(params=dict(B=0)), -2), (dict(params=dict(N=-1)), -2), (dict(params=dict(B=1 << 20, N=1 << 20)), -2), (dict(params=dict(dtype=2)), -3), (dict(params=dict(d=48)), -4),
    (dict(params=dict(rotary_dim=7)), -11), (dict(params=dict(frequencies=None)), -11), (dict(params=dict(rotary_dim=0)), -11), (dict(params=dict(magnitude=float("nan"))), -11),
    (dict(params=dict(inverse=1)), -11), (dict(params=dict(positions=0x30002)), -2), (dict(n=0), -2), (dict(n=3), -2),
    (dict(norm="none"), -1), (dict(norm=dict(q_weight=None)), -12), (dict(norm=dict(k_weight=None)), -12), (dict(norm=dict(q_weight=0x40002)), -12),
    (dict(norm=dict(k_weight=0x50001, weights_fp32=0)), -12), (dict(norm=dict(eps=0.0)), -12), (dict(norm=dict(eps=-1.0)), -12), (dict(norm=dict(eps=float("inf"))), -12),
    (dict(norm=dict(eps=float("nan"))), -12), (dict(norm=dict(eps=1e-40)), -12),
    (dict(tensor=dict(H=0)), -2), (dict(tensor=dict(x=None)), -1), (dict(tensor=dict(x=0x100008)), -2), (dict(tensor=dict(x_stride_n=60)), -2),
]


@pytest.mark.parametrize("kw,status", BAD + [(dict(tensor=dict(y=None)), -1), (dict(tensor=dict(y_stride_n=32)), -2), (dict(tensor=dict(y=0x300000)), -2), (dict(tensor=dict(y=0x400000)), -2)])
def test_forward_refuses(lib, kw, status):
    assert _forward(lib, **kw) == status


def _backward(lib, n=2, norm=None, params=None, tensor=None, ws=0x900000, ws_bytes=1 << 30):
    t = (binding.NormGrad * 2)()
    for i in range(2):
        t[i].x, t[i].dy, t[i].dx, t[i].dw = (0x100000 * (1 + 4 * i + j) for j in range(4))
        t[i].H = 4
        for a in ("x", "dy", "dx"):
            for axis, s in zip("bhn", (4 * 8 * 64, 8 * 64, 64)):
                setattr(t[i], f"{a}_stride_{axis}", s)
    for k, v in (tensor or {}).items():
        setattr(t[0], k, v)
    return lib.attn_norm_rotary_bwd(ctypes.byref(_rotary_params(**(params or {}))), None if norm == "none" else ctypes.byref(_norm(**(norm or {}))), t, n, ctypes.c_void_p(ws), ws_bytes)


@pytest.mark.parametrize("kw,status", BAD + [
    (dict(tensor=dict(dy=None)), -1), (dict(tensor=dict(dx=None)), -1), (dict(tensor=dict(dx_stride_n=32)), -2), (dict(tensor=dict(dw=0x400002)), -12),
    (dict(tensor=dict(dx=0x100000)), -2), (dict(tensor=dict(dx=0x200000)), -2), (dict(tensor=dict(dx=0x500000)), -2), (dict(tensor=dict(dx=0x700000)), -2), (dict(tensor=dict(dw=0x800000)), -2),
    (dict(ws=0), -7), (dict(ws=0x900010), -7), (dict(ws_bytes=1000), -7)])
def test_backward_refuses(lib, kw, status):
    assert _backward(lib, **kw) == status


def test_layout_workspace_and_texts(lib):
    assert ctypes.sizeof(binding.NormSpec) == 24 and ctypes.sizeof(binding.NormGrad) == 112
    assert binding.attn_norm_rotary_bwd_workspace_bytes(64) > 0 and binding.attn_norm_rotary_bwd_workspace_bytes(48) == 0
    assert "eps" in binding.strerror(-12) and "window" in binding.strerror(-13)
    assert lib.attn_norm_rotary(None, ctypes.byref(_norm()), (binding.RotaryTensor * 2)(), 1) == -1
    assert lib.attn_norm_rotary_bwd(None, ctypes.byref(_norm()), (binding.NormGrad * 2)(), 1, A, 1 << 30) == -1


@pytest.mark.parametrize("norm,rotary,pointers,status", [
    ("none", True, (A, B, C, D, E, F), -1), (dict(eps=0.0), True, (A, B, C, D, E, F), -12), (dict(q_weight=None), True, (A, B, C, D, E, F), -12),
    (dict(k_weight=None), True, (A, B, C, D, None, None), -12), ({}, True, (A, B, C, C, E, F), -2), ({}, False, (A, B, C, D, E, A), -2), ({}, True, (None, B, C, D, E, F), -1)])
def test_append_refuses(lib, norm, rotary, pointers, status):
    p = binding.PagedParams()
    p.B, p.T, p.Hq, p.Hk, p.d, p.dtype, p.pages, p.page_size, p.table_width = 2, 2, 8, 2, 64, 1, 10, 16, 4
    p.page_stride, p.head_stride, p.row_stride, p.table_stride = 2 * 16 * 64, 16 * 64, 64, 4
    p.q_stride_t = p.o_stride_t = 512
    p.q_stride_h = p.o_stride_h = 64
    p.k_stride_t = p.v_stride_t = 128
    p.k_stride_h = p.v_stride_h = 64
    p.block_table, p.lengths = 0x30000, 0x40000
    spec = binding.RotarySpec(0x50000, 64, 0, 1.0)
    assert lib.attn_paged_norm_append(ctypes.byref(p), ctypes.byref(spec) if rotary else None, None if norm == "none" else ctypes.byref(_norm(**norm)), *pointers) == status


def test_objects_refuse():
    w = torch.ones(64)
    for bad in (w.view(8, 8), w[::2], w[:0]):
        with pytest.raises(ValueError):
            HeadNorm(bad)
    with pytest.raises(TypeError):
        HeadNorm(w.double())
    with pytest.raises(TypeError):
        HeadNorm(w, w.half())
    with pytest.raises(ValueError):
        HeadNorm(w, w[:32])
    for eps in (0.0, -1.0, float("nan"), float("inf"), 1e-45):
        with pytest.raises(ValueError):
            HeadNorm(w, eps=eps)


def test_marshalling_refuses(lib):
    w = torch.ones(64)
    q, k = torch.zeros(1, 4, 8, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 8, 64, dtype=torch.bfloat16)
    rotary = Rotary(rotary_frequencies(64)[0])
    good = HeadNorm(w, w)
    for call in (binding.attn_norm_rotary, norm_rotary_embedding, lambda q, k, *a, **kw: binding.attn_norm_rotary_bwd(q, k, q, k, *a, **kw)):
        with pytest.raises(RuntimeError, match="GPU only"):
            call(q, k, good, rotary)
        with pytest.raises(RuntimeError, match="GPU only"):
            call(q, k, good)
        with pytest.raises((ValueError, RuntimeError)):
            call(q, k, HeadNorm(w), rotary)
        for bad in (k[:, :, :5], k.half(), k[0], k[..., :32]):
            with pytest.raises(ValueError):
                call(q, bad, good, rotary)
        with pytest.raises(TypeError):
            call(q, k, good, rotary, positions=torch.zeros(8))
        with pytest.raises(TypeError):
            call(q.float(), k.float(), good, rotary)
    with pytest.raises(ValueError):
        binding.attn_norm_rotary(q, None, good, rotary, out=(None, k))
    with pytest.raises(ValueError):
        binding.attn_norm_rotary(q, k, good, rotary, out=(k, None))
    with pytest.raises(ValueError):
        binding.attn_norm_rotary_bwd(q, k, q, None, good, rotary)
    with pytest.raises(ValueError):
        binding.attn_norm_rotary_bwd(q, k, k, k, good, rotary)
    f = rotary_frequencies(64)[0].requires_grad_(True)
    with pytest.raises(ValueError, match="frequencies require"):
        norm_rotary_embedding(q, k, good, Rotary(f))
    with pytest.raises((ValueError, RuntimeError)):
        flash_attention(q, q, q, norm=good, positions=torch.zeros(8, dtype=torch.int32))
    kv, c = torch.zeros(2, 2, 64, dtype=torch.bfloat16), torch.zeros(10, 2, 16, 64, dtype=torch.bfloat16)
    t, n = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises((ValueError, RuntimeError)):
        binding.attn_paged_append(kv, kv, c, c, t, n, norm=HeadNorm(torch.ones(32), torch.ones(32)))
    with pytest.raises((ValueError, RuntimeError)):
        binding.attn_paged_append(kv, kv, c, c, t, n, norm=HeadNorm(w))
