"""What the rotary positions and the paged cache refuse, and the layout of their parameter blocks (no GPU needed)."""
import ctypes
import os

import pytest
import torch

from paper_2205_14135_amd import binding
from paper_2205_14135_amd.autograd import flash_attention, rotary_embedding
from paper_2205_14135_amd.rotary import Rotary, rotary_frequencies

OK_PTR = ctypes.c_void_p(0x10000)
ODD = ctypes.c_void_p(0x10008)
NULL = ctypes.c_void_p(0)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2205_14135_amd import build
        build.build()
    return binding.load()


def test_layout_matches_c():
    """(the library asserts the same sizes)"""
    assert [ctypes.sizeof(t) for t in (binding.RotarySpec, binding.RotaryTensor, binding.RotaryParams, binding.PagedParams, binding.PagedCopyParams)] == [24, 72, 72, 176, 64]
    assert binding.PagedParams.page_stride.offset == 48 and binding.PagedParams.block_table.offset == 144


def test_texts(lib):
    assert "power of two" in binding.strerror(-10) and "rotary_dim" in binding.strerror(-11)


# ---- rotary

def _rotary(lib, spec=None, tensor=None, n=1, x=0x10000, y=0x20000, **kw):
    p = binding.RotaryParams()
    p.B, p.N, p.d, p.dtype = 2, 8, 64, 1
    p.rotary.frequencies, p.rotary.rotary_dim, p.rotary.magnitude = 0x30000, 64, 1.0
    for k, v in (spec or {}).items():
        setattr(p.rotary, k, v)
    for k, v in kw.items():
        setattr(p, k, v)
    t = (binding.RotaryTensor * 2)()
    for i in range(2):
        t[i].x, t[i].y, t[i].H = x, y, 4
        for a in "xy":
            for axis, s in zip("bhn", (4 * 8 * 64, 8 * 64, 64)):
                setattr(t[i], f"{a}_stride_{axis}", s)
    for k, v in (tensor or {}).items():
        setattr(t[0], k, v)
    return lib.attn_rotary(ctypes.byref(p), t, n)


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), -2), (dict(N=0), -2), (dict(N=-1), -2), (dict(B=1 << 20, N=1 << 20), -2), (dict(dtype=2), -3), (dict(d=48), -4), (dict(d=256), -4),
    (dict(positions=0x30002), -2), (dict(positions=0x30000, position_stride_b=-8), -2),
    (dict(spec=dict(rotary_dim=0)), -11), (dict(spec=dict(rotary_dim=7)), -11), (dict(spec=dict(rotary_dim=66)), -11), (dict(spec=dict(rotary_dim=-2)), -11),
    (dict(spec=dict(frequencies=None)), -11), (dict(spec=dict(frequencies=0x30004)), -11),
    (dict(spec=dict(magnitude=float("nan"))), -11), (dict(spec=dict(magnitude=float("inf"))), -11),
    (dict(n=0), -2), (dict(n=3), -2), (dict(x=None), -1), (dict(y=None), -1), (dict(x=0x10008), -2), (dict(y=0x10008), -2),
    (dict(tensor=dict(H=0)), -2), (dict(tensor=dict(x_stride_n=60)), -2), (dict(tensor=dict(x_stride_h=-512)), -2),
    (dict(tensor=dict(y_stride_n=32)), -2), (dict(tensor=dict(y_stride_b=0)), -2), (dict(tensor=dict(y_stride_h=64)), -2),    # output rows that share elements
    (dict(x=0x10000, y=0x10000, tensor=dict(x_stride_b=0)), -2),                                                            # in place with other strides
])
def test_rotary_refuses(lib, kw, status):
    assert _rotary(lib, **kw) == status


def test_rotary_needs_its_blocks(lib):
    assert lib.attn_rotary(None, (binding.RotaryTensor * 2)(), 1) == -1
    assert lib.attn_rotary(ctypes.byref(binding.RotaryParams()), None, 1) == -1


# ---- paged

def _paged(**kw):
    p = binding.PagedParams()
    p.B, p.T, p.Hq, p.Hk, p.d, p.dtype, p.pages, p.page_size, p.table_width, p.softmax_scale = 2, 2, 8, 2, 64, 1, 10, 16, 4, 0.125
    p.page_stride, p.head_stride, p.row_stride, p.table_stride = 2 * 16 * 64, 16 * 64, 64, 4
    p.q_stride_t = p.o_stride_t = 512
    p.q_stride_h = p.o_stride_h = 64
    p.k_stride_t = p.v_stride_t = 128
    p.k_stride_h = p.v_stride_h = 64
    p.block_table, p.lengths = 0x30000, 0x40000
    for k, v in kw.items():
        setattr(p, k, v)
    return p


BAD_BATCH = [
    (dict(B=0), -2), (dict(T=0), -2), (dict(T=1), -2), (dict(Hq=0), -2), (dict(Hk=0), -2), (dict(Hq=9), -2), (dict(B=1 << 25, T=1 << 25), -2), (dict(T=1 << 29), -2),
    (dict(table_width=0), -2), (dict(table_width=1 << 27), -2), (dict(pages=0), -2), (dict(dtype=5), -3), (dict(d=40), -4),
    (dict(page_size=8), -10), (dict(page_size=48), -10), (dict(page_size=0), -10), (dict(page_size=8192), -10),
    (dict(row_stride=60), -2), (dict(row_stride=1 << 24, head_stride=1 << 30, page_stride=1 << 34), -2), (dict(page_stride=0), -2), (dict(head_stride=64), -2), (dict(page_stride=-2048), -2),
    (dict(table_stride=-1), -2),
]


@pytest.mark.parametrize("kw,status", BAD_BATCH + [(dict(softmax_scale=0.0), -6), (dict(softmax_scale=float("nan")), -6), (dict(q_stride_t=511), -2),
                                                   (dict(o_stride_t=256), -2), (dict(o_stride_h=0), -2), (dict(lengths=0x40002), -2), (dict(block_table=None), -1),
                                                   (dict(lengths=None), -1)])
def test_paged_fwd_refuses(lib, kw, status):
    p = _paged(**kw)
    assert lib.attn_paged_fwd(ctypes.byref(p), OK_PTR, OK_PTR, OK_PTR, OK_PTR, OK_PTR, OK_PTR, 1 << 30) == status
    pointers = "lengths" in kw or "block_table" in kw
    assert (lib.attn_paged_workspace_bytes(ctypes.byref(p)) == 0) != pointers


@pytest.mark.parametrize("kw,ok", [
    (dict(page_stride=(1 << 31) - 8), True), (dict(page_stride=1 << 31), False),                                     # bytes from page to page: 32 bits
    (dict(page_size=4096, row_stride=(1 << 19) - 8, head_stride=64, page_stride=(1 << 31) - 8), True),
    (dict(page_size=4096, row_stride=1 << 19, head_stride=64, page_stride=(1 << 31) - 8), False),                    # and inside a page
    (dict(Hq=1 << 16, Hk=1 << 16, d=128, page_size=1024, row_stride=128, page_stride=1 << 17, head_stride=10 << 17, q_stride_h=128, o_stride_h=128, q_stride_t=1 << 23, o_stride_t=1 << 23), True),
    (dict(Hq=1 << 16, Hk=1 << 16, d=128, page_size=2048, row_stride=128, page_stride=1 << 18, head_stride=10 << 18, q_stride_h=128, o_stride_h=128, q_stride_t=1 << 23, o_stride_t=1 << 23), False),
    (dict(B=1 << 20, T=1 << 20), True), (dict(B=(1 << 20) + 1, T=(1 << 20) + 1), False)])
def test_paged_limits(lib, kw, ok):
    p = _paged(**kw)
    assert (lib.attn_paged_workspace_bytes(ctypes.byref(p)) != 0) == ok
    if not ok:
        assert lib.attn_paged_fwd(ctypes.byref(p), OK_PTR, OK_PTR, OK_PTR, OK_PTR, OK_PTR, OK_PTR, 1 << 30) == -2


def test_paged_fwd_pointers_and_workspace(lib):
    p = _paged()
    need = lib.attn_paged_workspace_bytes(ctypes.byref(p))
    assert need > 0
    for slot in range(5):
        args = [OK_PTR] * 5
        args[slot] = NULL
        assert lib.attn_paged_fwd(ctypes.byref(p), *args, OK_PTR, need) == -1
        args[slot] = ctypes.c_void_p(0x10002) if slot == 4 else ODD
        assert lib.attn_paged_fwd(ctypes.byref(p), *args, OK_PTR, need) == -2
    assert lib.attn_paged_fwd(ctypes.byref(p), *[OK_PTR] * 5, NULL, need) == -7
    assert lib.attn_paged_fwd(ctypes.byref(p), *[OK_PTR] * 5, ctypes.c_void_p(0x10010), need) == -7
    assert lib.attn_paged_fwd(ctypes.byref(p), *[OK_PTR] * 5, OK_PTR, need - 1) == -7
    assert lib.attn_paged_fwd(None, *[OK_PTR] * 5, OK_PTR, need) == -1
    # one serves every call at its head dimension
    assert lib.attn_paged_workspace_bytes(ctypes.byref(_paged(T=1000, query_starts=0x50000))) == need
    assert lib.attn_paged_workspace_bytes(ctypes.byref(_paged(B=60, T=60, Hq=4, causal=1))) == need


def _append(lib, p, rotary=True, spec=None, args=None):
    s = binding.RotarySpec(0x30000, 64, 0, 1.0)
    for k, v in (spec or {}).items():
        setattr(s, k, v)
    a = [OK_PTR] * 6 if args is None else args
    return lib.attn_paged_append(ctypes.byref(p), ctypes.byref(s) if rotary else None, *a)


@pytest.mark.parametrize("kw,status", BAD_BATCH + [(dict(k_stride_t=4), -2), (dict(v_stride_h=-64), -2), (dict(o_stride_t=256), -2), (dict(lengths=None), -1)])
def test_append_refuses(lib, kw, status):
    assert _append(lib, _paged(**kw)) == status


def test_append_pointers_and_rotation(lib):
    for slot in range(6):
        args = [OK_PTR] * 6
        args[slot] = NULL
        assert _append(lib, _paged(), args=args) == -1
        args[slot] = ODD
        assert _append(lib, _paged(), args=args) == -2
    assert _append(lib, _paged(), rotary=False) == -11                       # Q without a rotation
    assert _append(lib, _paged(), spec=dict(rotary_dim=128)) == -11
    assert _append(lib, _paged(o_stride_t=1024)) == -2                       # in place (Q == Qout) with other strides


def _copy(lib, pairs, k=OK_PTR, v=OK_PTR, **kw):
    p = binding.PagedCopyParams()
    p.layers, p.pages, p.Hk, p.page_size, p.d, p.dtype = 2, 10, 2, 16, 64, 1
    p.layer_stride, p.page_stride, p.head_stride, p.row_stride = 10 * 2048, 2048, 1024, 64
    for key, value in kw.items():
        setattr(p, key, value)
    flat = [x for pair in pairs for x in pair]
    return lib.attn_paged_copy(ctypes.byref(p), k, v, (ctypes.c_int32 * max(1, len(flat)))(*flat), len(pairs))


@pytest.mark.parametrize("pairs", [[(0, 10)], [(10, 0)], [(-1, 0)], [(0, -1)], [(3, 3)], [(0, 1), (2, 1)], [(0, 1), (1, 2)], [(1, 2), (0, 1)], [(0, 1), (0, 1)]])
def test_copy_refuses_lists(lib, pairs):
    assert _copy(lib, pairs) == -10


@pytest.mark.parametrize("kw,status", [(dict(layers=0), -2), (dict(layers=1 << 15), -2), (dict(pages=0), -2), (dict(page_size=24), -10), (dict(d=8), -4), (dict(dtype=9), -3),
                                       (dict(layer_stride=2048), -2), (dict(page_stride=1024), -2), (dict(k=NULL), -1), (dict(v=ODD), -2)])
def test_copy_refuses(lib, kw, status):
    assert _copy(lib, [(0, 1)], **kw) == status
    assert _copy(lib, [(i, 0) for i in range(11)]) == -2                     # more copies than pages
    assert _copy(lib, []) == 0


# ---- the binding's marshalling, on CPU tensors

def _call(**kw):
    a = dict(Q=torch.zeros(2, 8, 64, dtype=torch.bfloat16), k_cache=torch.zeros(10, 2, 16, 64, dtype=torch.bfloat16), v_cache=torch.zeros(10, 2, 16, 64, dtype=torch.bfloat16),
             block_table=torch.zeros(2, 4, dtype=torch.int32), lengths=torch.zeros(2, dtype=torch.int32), query_starts=None)
    opts = {k: kw.pop(k) for k in list(kw) if k not in a}
    a.update(kw)
    return binding.attn_paged_fwd(*a.values(), softmax_scale=0.1, **opts)


@pytest.mark.parametrize("kw,error", [
    (dict(Q=torch.zeros(2, 8, 64)), ValueError), (dict(Q=torch.zeros(2, 64, dtype=torch.bfloat16)), ValueError),
    (dict(Q=torch.zeros(2, 64, 8, dtype=torch.bfloat16).transpose(1, 2)), ValueError), (dict(Q=torch.zeros(2, 8, 32, dtype=torch.bfloat16)), ValueError),
    (dict(k_cache=torch.zeros(10, 2, 16, 64)), ValueError), (dict(k_cache=torch.zeros(9, 2, 16, 64, dtype=torch.bfloat16)), ValueError),
    (dict(k_cache=torch.zeros(10, 16, 2, 64, dtype=torch.bfloat16).transpose(1, 2)), ValueError),
    (dict(lengths=torch.zeros(2, dtype=torch.int64)), TypeError), (dict(lengths=torch.zeros(4, dtype=torch.int32)[::2]), TypeError), (dict(lengths=torch.zeros(3, dtype=torch.int32)), TypeError),
    (dict(block_table=torch.zeros(2, 4, dtype=torch.int64)), TypeError), (dict(block_table=torch.zeros(4, 2, dtype=torch.int32).t()), TypeError),
    (dict(query_starts=torch.zeros(2, dtype=torch.int32)), TypeError), (dict(query_starts=torch.zeros(3)), TypeError),
    (dict(out=torch.zeros(2, 8, 64)), ValueError), (dict(), RuntimeError), (dict(Q="x"), TypeError),
])
def test_paged_marshalling_refuses(lib, kw, error):
    with pytest.raises(error):
        _call(**kw)


def test_rotary_marshalling_refuses(lib):
    f, _ = rotary_frequencies(64)
    q, k = torch.zeros(1, 4, 8, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 8, 64, dtype=torch.bfloat16)
    good = Rotary(f)
    for call in (lambda *a, **kw: binding.attn_rotary(*a, **kw), lambda q, k, r, **kw: rotary_embedding(q, k, r, **kw)):
        with pytest.raises(RuntimeError, match="GPU only"):
            call(q, k, good)
        for bad in (k[:, :, :5], k.half(), k[0], k[..., :32]):
            with pytest.raises(ValueError):
                call(q, bad, good)
        for bad in (torch.zeros(8), torch.zeros(7, dtype=torch.int32), torch.zeros(2, 8, dtype=torch.int32), torch.zeros(16, dtype=torch.int32)[::2]):
            with pytest.raises(TypeError):
                call(q, k, good, positions=bad)
        with pytest.raises(TypeError):
            call(q.float(), k.float(), good)
    with pytest.raises(ValueError):
        binding.attn_rotary(q, None, good, out=(None, k))
    with pytest.raises(ValueError):
        binding.attn_rotary(q, k, good, out=(k, None))
    with pytest.raises((ValueError, RuntimeError)):
        flash_attention(q, q, q, positions=torch.zeros(8, dtype=torch.int32))


def test_append_and_copy_marshalling_refuse(lib):
    f, _ = rotary_frequencies(64)
    kv = torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    c = torch.zeros(10, 2, 16, 64, dtype=torch.bfloat16)
    t, n = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    q = torch.zeros(2, 8, 64, dtype=torch.bfloat16)
    with pytest.raises(RuntimeError, match="GPU only"):
        binding.attn_paged_append(kv, kv, c, c, t, n)
    with pytest.raises(ValueError):
        binding.attn_paged_append(q, q, c, c, t, n)                       # other heads than the caches'
    with pytest.raises(ValueError):
        binding.attn_paged_append(kv, kv[:1], c, c, t, n)
    with pytest.raises((ValueError, RuntimeError)):
        binding.attn_paged_append(kv, kv, c, c, t, n, Q=q)                # Q without a rotation
    with pytest.raises((ValueError, RuntimeError)):
        binding.attn_paged_append(kv, kv, c, c, t, n, out=q)
    with pytest.raises(RuntimeError, match="GPU only"):
        binding.attn_paged_copy(c, c, [(0, 1)])
    for bad in (torch.zeros(1, 2, dtype=torch.int64), torch.zeros(1, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(2, 4, dtype=torch.int32)[:, ::2]):
        with pytest.raises(TypeError):
            binding.attn_paged_copy(c, c, bad)
    with pytest.raises(ValueError):
        binding.attn_paged_copy(c, c[:9], [(0, 1)])
    with pytest.raises(ValueError):
        binding.attn_paged_workspace(q, torch.zeros(10, 3, 16, 64, dtype=torch.bfloat16), 2)


# ---- frequencies

def test_frequencies():
    f, m = rotary_frequencies(64)
    assert f.dtype == torch.float64 and f.shape == (32,) and m == 1.0 and f[0] == 1.0 and f[-1].item() == pytest.approx(10000.0 ** (-62 / 64), rel=1e-14)
    g, m = rotary_frequencies(64, scaling="linear", factor=4.0)
    assert torch.equal(g, f / 4) and m == 1.0
    g, m = rotary_frequencies(64, scaling="base", factor=4.0)
    assert g[0] == 1.0 and g[-1].item() == pytest.approx(f[-1].item() / 4, rel=1e-13) and m == 1.0
    g, m = rotary_frequencies(64, scaling="parts", factor=4.0, original_length=4096)
    turns = f * 4096 / (2 * 3.141592653589793)
    assert torch.equal(g[turns >= 32], f[turns >= 32]) and torch.allclose(g[turns <= 1], f[turns <= 1] / 4, rtol=1e-15) and m == pytest.approx(1.1386294361119890)
    assert (g <= f).all() and (g >= f / 4).all()
    assert torch.equal(rotary_frequencies(2, scaling="base", factor=4.0)[0], torch.ones(1, dtype=torch.float64))


@pytest.mark.parametrize("args,kw", [((0,), {}), ((7,), {}), ((64, 1.0), {}), ((64, float("nan")), {}), ((64,), dict(scaling="other")), ((64,), dict(factor=2.0)),
                                     ((64,), dict(scaling="linear", factor=0.5)), ((64,), dict(scaling="parts", factor=2.0, original_length=0)),
                                     ((64,), dict(scaling="parts", factor=2.0, slow_turns=32.0, fast_turns=1.0))])
def test_frequencies_refuse(args, kw):
    with pytest.raises(ValueError):
        rotary_frequencies(*args, **kw)


def test_rotary_object_refuses():
    f, _ = rotary_frequencies(8)
    for bad in (f.float(), f.view(2, 2), f[::2], f[:0]):
        with pytest.raises(TypeError):
            Rotary(bad)
    with pytest.raises(ValueError):
        Rotary(f, magnitude=float("inf"))
