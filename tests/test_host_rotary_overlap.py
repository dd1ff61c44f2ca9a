"""Calls whose outputs are another tensor of the same call (no GPU needed): two groups of threads would read and write the same rows."""
import ctypes

import pytest

from paper_2205_14135_amd import binding

A, B, C, D, E, F = (0x100000 * (i + 1) for i in range(6))


@pytest.mark.parametrize("q,q_out,k,k_out", [(A, A, A, A), (A, C, B, C), (A, B, B, C), (A, C, B, A), (A, B, B, A)])
def test_rotary(q, q_out, k, k_out):
    lib = binding.load()
    p = binding.RotaryParams()
    p.B, p.N, p.d, p.dtype = 2, 8, 64, 1
    p.rotary.frequencies, p.rotary.rotary_dim, p.rotary.magnitude = F, 64, 1.0
    t = (binding.RotaryTensor * 2)()
    for i, (x, y) in enumerate(((q, q_out), (k, k_out))):
        t[i].x, t[i].y, t[i].H = x, y, 4
        for a in "xy":
            for axis, s in zip("bhn", (4 * 8 * 64, 8 * 64, 64)):
                setattr(t[i], f"{a}_stride_{axis}", s)
    assert lib.attn_rotary(ctypes.byref(p), t, 2) == -2


# K, V, K cache, V cache, Q, Q'
@pytest.mark.parametrize("pointers", [(A, B, C, C, E, F), (A, B, C, D, E, A), (A, B, C, D, E, B), (A, B, C, D, E, C), (A, B, C, D, E, D), (A, B, C, C, None, None)])
def test_append(pointers):
    lib = binding.load()
    p = binding.PagedParams()
    p.B, p.T, p.Hq, p.Hk, p.d, p.dtype, p.pages, p.page_size, p.table_width = 2, 2, 8, 2, 64, 1, 10, 16, 4
    p.page_stride, p.head_stride, p.row_stride, p.table_stride = 2 * 16 * 64, 16 * 64, 64, 4
    p.q_stride_t = p.o_stride_t = 512
    p.q_stride_h = p.o_stride_h = 64
    p.k_stride_t = p.v_stride_t = 128
    p.k_stride_h = p.v_stride_h = 64
    p.block_table, p.lengths = 0x30000, 0x40000
    spec = binding.RotarySpec(0x50000, 64, 0, 1.0)
    assert lib.attn_paged_append(ctypes.byref(p), ctypes.byref(spec) if pointers[4] else None, *pointers) == -2
