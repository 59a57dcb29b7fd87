"""Calls so large that a launch could not have a thread for every part of them: refused, or divided otherwise.  CPU only: nothing is launched."""
import ctypes

import pytest

from test_serve_host import FAKE, _cache, _rotary, _tensor, lib  # noqa: F401


@pytest.mark.parametrize("dtype,dim", [(0, 32), (0, 128), (1, 32), (1, 128)])
def test_rows_of_a_rotation_and_an_append(lib, dtype, dim):  # noqa: F811
    """rows * head_dim below 2^36 (fp32 2^35), less 2^15: one more row than that is refused before any launch."""
    most = ((1 << (36 - dtype)) - (1 << 15)) // dim
    if most >= 1 << 31:
        most = (1 << 31) - 1
    t = _tensor(heads=1, dim=dim, ss=dim, ds=dim)

    def rotary(rows, src=FAKE):
        t.src = src
        return lib.hstu_rotary(ctypes.byref(_rotary()), 0, dtype, 2, rows, 1, ctypes.byref(t), None, FAKE, None)
    assert rotary(most + (1 << 15), FAKE + 8) == -2
    assert rotary(most, FAKE + 8) == -7          # (as far as the pointers, which a call within the limit gets to)
    c = _cache(dtype=dtype, d_qk=32, d_v=dim, num_kv_heads=1, k_page_stride=512, v_page_stride=16 * dim)
    append = lambda rows: lib.hstu_cache_append(ctypes.byref(c), None, rows, None, FAKE + 8, 32, FAKE, dim, None, FAKE, None)
    assert append(most + (1 << 15)) == -2 and append(most) == -7


def test_attention_of_more_tiles_than_workgroups(lib):  # noqa: F811
    from paper_2508_04711_amd import binding

    def need(batch, rows, heads, dtype=0, max_kv=0, pages=1 << 10):
        c = _cache(batch=batch, num_kv_heads=heads, d_qk=32, d_v=32, dtype=dtype, pages_per_seq=pages, table_stride=pages,
                   k_page_stride=heads * 512, v_page_stride=heads * 512)
        p = binding._PagedParams(heads, 16, 0.1, 1, 1, max_kv, rows)
        return lib.hstu_paged_attn_workspace_bytes(ctypes.byref(p), ctypes.byref(c))
    # tiles of 128 pairs, 256 threads each: 2^24 of them are too many for a launch, so tiles of 16 share a line of workers
    tiles128, tiles16 = 2 * 768 * 128 * 32 * 4, 2 * 1024 * 16 * 32 * 4
    assert need(100000, 900001, 128) >= tiles128
    assert tiles16 <= need(150000, 1350001, 128) < tiles128
    # tiles of 16 pairs, uncut, a wave each: 2^26 are too many
    assert need(1, 1 << 29, 1, dtype=1, max_kv=100, pages=16) == 256
    assert need(1, (1 << 30) + 64, 1, dtype=1, max_kv=100, pages=16) >= tiles16
