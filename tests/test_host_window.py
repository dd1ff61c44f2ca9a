"""What attention with a sliding window refuses (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2205_14135_amd import binding
from paper_2205_14135_amd.autograd import flash_attention

PTR = ctypes.c_void_p(0x10000)


@pytest.fixture(scope="module")
def lib():
    return binding.load()


def _params(**kw):
    p = binding.AttnParams()
    p.B, p.H, p.N, p.d, p.dtype, p.softmax_scale, p.causal = 2, 4, 512, 64, binding.ATTN_BF16, 0.125, 1
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def _fwd(lib, p, window=64, sinks=4, args=None):
    return lib.attn_window_fwd(ctypes.byref(p), window, sinks, *([PTR] * 5 if args is None else args))


def _bwd(lib, p, window=64, sinks=4, args=None, ws=PTR, ws_bytes=1 << 40):
    return lib.attn_window_bwd(ctypes.byref(p), window, sinks, *([PTR] * 9 if args is None else args), ws, ws_bytes)


@pytest.mark.parametrize("kw,window,sinks,status", [
    (dict(causal=0), 64, 4, -13), ({}, 0, 4, -13), ({}, -5, 4, -13), ({}, 64, -1, -13), (dict(causal=0), 1000, 0, -13), (dict(dtype=3), 64, 4, -3), (dict(d=48), 64, 4, -4),
    (dict(N=0), 64, 4, -2), (dict(dropout_p=1.0), 64, 4, -5), (dict(softmax_scale=0.0), 64, 4, -6), (dict(stride_b=1, stride_h=1, stride_n=60), 64, 4, -2)])
def test_params(lib, kw, window, sinks, status):
    p = _params(**kw)
    assert _fwd(lib, p, window, sinks) == status and _bwd(lib, p, window, sinks) == status
    assert lib.attn_window_bwd_workspace_bytes(ctypes.byref(p), window, sinks) == 0


@pytest.mark.parametrize("window", [64, 512])
def test_pointers(lib, window):
    p = _params()
    need = lib.attn_window_bwd_workspace_bytes(ctypes.byref(p), window, 4)
    assert need > 0
    for n, call in ((5, _fwd), (9, _bwd)):
        for i in range(n):
            args = [PTR] * n
            args[i] = None
            assert call(lib, p, window, args=args) == -1
            args[i] = ctypes.c_void_p(0x10002)
            assert call(lib, p, window, args=args) == -2
    assert _bwd(lib, p, window, ws=None) == -7 and _bwd(lib, p, window, ws=ctypes.c_void_p(0x10010)) == -7 and _bwd(lib, p, window, ws_bytes=need // 2) == -7
    assert lib.attn_window_fwd(None, 64, 4, *[PTR] * 5) == -1


def test_workspace_is_linear(lib):
    """Two floats a row, and pieces for the sinks: no more than 32 keys' gradients in 32 bits for each 32 sinks and stretch of queries."""
    for N in (1000, 10 ** 5, 10 ** 6):
        p = _params(N=N)
        rows = 2 * 4 * 2 * 4 * ((N + 127) // 128 * 128)
        none = lib.attn_window_bwd_workspace_bytes(ctypes.byref(p), 256, 0)
        assert rows <= none < rows + 256
        few = lib.attn_window_bwd_workspace_bytes(ctypes.byref(p), 256, 4) - none
        assert few % (8 * 2 * 32 * 64 * 4) == 0 and few <= 8 * 2 * 32 * 64 * 4 * (2 + N // 256)
        many = lib.attn_window_bwd_workspace_bytes(ctypes.byref(p), 256, N // 2) - none
        assert many <= 8 * 2 * 64 * 4 * (N // 2 + 32) * 3 + 8 * 2 * 32 * 64 * 4 * 8 * 256


def test_marshalling(lib):
    x = torch.zeros(1, 2, 100, 64, dtype=torch.bfloat16)
    for kw in (dict(causal=False, window=8), dict(causal=True, window=0), dict(causal=True, window=-1), dict(causal=True, window=8, sinks=-1), dict(causal=True, sinks=4),
               dict(causal=True, window=8, block_mask=torch.ones(1, 1, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            flash_attention(x, x, x, **kw)
    with pytest.raises(RuntimeError, match="GPU only"):
        flash_attention(x, x, x, causal=True, window=8)
    for window, sinks, error in ((0, 0, ValueError), (-10 ** 12, 0, ValueError), (5, -1, ValueError), (2.5, 0, TypeError), ("x", 0, TypeError), (5, None, TypeError)):
        with pytest.raises(error):
            binding.attn_window_fwd(x, x, x, window=window, sinks=sinks, softmax_scale=0.1)
        with pytest.raises(error):
            binding.attn_window_bwd(x, x, x, x, x, torch.zeros(1, 2, 100), window=window, sinks=sinks, softmax_scale=0.1)
    with pytest.raises(ValueError):
        binding.attn_window_fwd(x, x[:, :1], x, window=8, softmax_scale=0.1)
    with pytest.raises(RuntimeError, match="GPU only"):
        binding.attn_window_fwd(x, x, x, window=8, softmax_scale=0.1)
    with pytest.raises(RuntimeError, match="GPU only"):
        binding.attn_window_bwd(x, x, x, x, x, torch.zeros(1, 2, 100), window=8, softmax_scale=0.1)


def _paged(**kw):
    p = binding.PagedParams()
    p.B, p.T, p.Hq, p.Hk, p.d, p.dtype, p.pages, p.page_size, p.table_width, p.softmax_scale, p.causal = 2, 2, 8, 2, 64, 1, 10, 16, 4, 0.125, 1
    p.page_stride, p.head_stride, p.row_stride, p.table_stride = 2 * 16 * 64, 16 * 64, 64, 4
    p.q_stride_t = p.o_stride_t = 512
    p.q_stride_h = p.o_stride_h = 64
    p.block_table, p.lengths = 0x30000, 0x40000
    for k, v in kw.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("kw,window,sinks,status", [(dict(causal=0), 8, 0, -13), ({}, 0, 0, -13), ({}, -1, 0, -13), ({}, 8, -1, -13), (dict(B=0), 8, 0, -2), (dict(d=48), 8, 0, -4),
                                                    (dict(page_size=8), 8, 0, -10), (dict(lengths=None), 8, 0, -1), (dict(softmax_scale=0.0), 8, 0, -6)])
def test_paged_params(lib, kw, window, sinks, status):
    assert lib.attn_paged_window_fwd(ctypes.byref(_paged(**kw)), window, sinks, *[PTR] * 5, PTR, 1 << 40) == status


def test_paged_pointers(lib):
    p = _paged()
    need = lib.attn_paged_workspace_bytes(ctypes.byref(p))
    for i in range(5):
        args = [PTR] * 5
        args[i] = None
        assert lib.attn_paged_window_fwd(ctypes.byref(p), 8, 1, *args, PTR, need) == -1
    assert lib.attn_paged_window_fwd(ctypes.byref(p), 8, 1, *[PTR] * 5, PTR, need - 1) == -7
    assert lib.attn_paged_window_fwd(None, 8, 1, *[PTR] * 5, PTR, need) == -1


def test_paged_marshalling(lib):
    q, c = torch.zeros(2, 8, 64, dtype=torch.bfloat16), torch.zeros(10, 2, 16, 64, dtype=torch.bfloat16)
    t, n = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for kw, error in ((dict(window=0), ValueError), (dict(window=-3), ValueError), (dict(window=4, sinks=-1), ValueError), (dict(window=4, causal=False), ValueError),
                      (dict(sinks=3), ValueError), (dict(window=1.5), TypeError), (dict(window=4), RuntimeError)):
        with pytest.raises(error):
            binding.attn_paged_fwd(q, c, c, t, n, softmax_scale=0.1, **kw)


def test_workspace_of_windows_beyond_32_bits(lib):
    """(as the calls take them: kept within 32 bits, not cut to their low ones)"""
    p = _params()
    nbytes = binding.attn_window_bwd_workspace_bytes
    all_keys, few = nbytes(p, 512, 0), nbytes(p, 64, 4)
    assert all_keys > 0 and few > 0
    for window in (2 ** 31 - 1, 2 ** 31, 2 ** 32 + 1, 10 ** 12):
        assert nbytes(p, window, 0) == all_keys
        assert nbytes(p, 64, window) == all_keys
        assert nbytes(p, -window, 0) == 0 and nbytes(p, 64, -window) == 0
