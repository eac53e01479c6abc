"""Refusals of the 8-bit serving operators (FP8 quantiser and product, cache tables, append and
attention): every bad argument is refused on the host, before any device call, with EP_ERR_ARG
and a message; calls over nothing do nothing.  No device pointer below is ever dereferenced."""
import ctypes

import pytest

A, B, D, F, G, H = (i << 20 for i in range(1, 7))   # aligned addresses


@pytest.fixture(scope="module")
def E():
    import os
    from paper_2609_34185_amd import entropack
    if not os.path.exists(entropack.LIB_PATH):
        from paper_2609_34185_amd import build
        build.build()
    return entropack


def refused(E, call, *a, **kw):
    with pytest.raises(E.EntroPackError) as e:
        call(*a, **kw)
    assert e.value.code == E.ERR_ARG and str(e.value)


def test_struct_sizes_match_the_header(E):
    """The binding's structs, field by field, as the C declarations lay them out."""
    assert ctypes.sizeof(E.Kv8Cache) == 4 * 8 + 8 + 4 * 4
    assert ctypes.sizeof(E.Kv8Attn) == 6 * 8 + 5 * 8 + 6 * 4 + 4 + 4


def test_quant_refusals(E):
    ok = dict(x_dtype=E.BF16, m=4, k=256, d_q=B, d_scale=D)
    for bad in (dict(m=-1), dict(k=0), dict(k=24), dict(x_row=128), dict(x_row=260), dict(block_rows=2),
                dict(block_rows=0), dict(x_dtype=E.INT8), dict(d_q=0), dict(d_scale=0), dict(d_q=B + 8),
                dict(m=1 << 32)):
        refused(E, E.quant_fp8_block, A, **{**ok, **bad})
    refused(E, E.quant_fp8_block, 0, **ok)
    refused(E, E.quant_fp8_block, A + 2, **ok)
    refused(E, E.quant_fp8_block, A, **{**ok, "x_dtype": E.FP32, "x_row": 258})
    E.quant_fp8_block(0, E.BF16, 0, 256, 0, 0)            # no rows: nothing to do


def test_product_refusals(E):
    ok = dict(m=4, n=8, k=256)
    for bad in (dict(m=-1), dict(n=0), dict(k=0), dict(k=24), dict(k=1 << 25), dict(n=1 << 25), dict(m=1 << 25),
                dict(w_dtype=E.INT8), dict(w_scales=0), dict(w_scales=4), dict(y_dtype=E.INT8)):
        refused(E, E.gemm_fp8_block, A, B, D, F, G, **{**ok, **bad})
    for i in range(5):
        p = [A, B, D, F, G]
        p[i] = 0
        refused(E, E.gemm_fp8_block, *p, **ok)
    refused(E, E.gemm_fp8_block, A + 8, B, D, F, G, **ok)
    refused(E, E.gemm_fp8_block, A, B, D + 4, F, G, **ok)
    E.gemm_fp8_block(0, 0, D, F, 0, 0, 8, 256)


def test_slots_refusals(E):
    ok = [A, B, 3, 64, D, F, G, 8, H, A, B, 100, D]
    for i, bad in ((0, 0), (1, 0), (2, 0), (2, -1), (3, 0), (3, 24), (3, 512), (4, 0), (5, 0), (6, 0), (7, 0),
                   (8, 0), (9, 0), (10, 0), (11, -1), (11, 1 << 31), (12, 0)):
        a = list(ok)
        a[i] = bad
        refused(E, E.kv8_slots, *a)


def bad_caches(E):
    ok = [A, B, D, F, 10, 8, 64, 128, E.FP8_E4M3]
    for i, bad in ((0, 0), (1, 0), (2, 0), (3, 0), (0, A + 8), (1, B + 4), (4, 0), (4, 1 << 31), (5, 0), (5, -1),
                   (6, 0), (6, 48), (6, 8), (7, 96), (7, 0), (8, E.BF16), (8, E.FP8_E5M2)):
        c = list(ok)
        c[i] = bad
        yield E.kv8_cache(*c)


def good_cache(E):
    return E.kv8_cache(A, B, D, F, 10, 8, 64, 128, E.FP8_E4M3)


def test_append_refusals(E):
    ok = [G, H, E.BF16, 1024, 1024, A, 5]
    for c in bad_caches(E):
        refused(E, E.kv8_append, c, *ok)
    for i, bad in ((0, 0), (1, 0), (0, G + 8), (1, H + 2), (2, E.FP8_E4M3), (3, 1016), (4, 1016), (3, 1028),
                   (4, 1030), (5, 0), (6, -1), (6, 1 << 31)):
        a = list(ok)
        a[i] = bad
        refused(E, E.kv8_append, good_cache(E), *a)
    E.kv8_append(good_cache(E), 0, 0, E.BF16, 1024, 1024, 0, 0)


def test_attention_refusals(E):
    base = dict(d_q=A, d_out=B, d_cu_q=D, d_len=F, d_table=G, table_ld=4, n_req=2, total_q=2, q_heads=16,
                dtype=E.BF16, scale=0.1, max_q=1, max_len=100)

    def call(**kw):
        return E.kv8_attention_args(**{**base, **kw})

    for c in bad_caches(E):
        refused(E, E.kv8_attention, c, call(), H, 1 << 30)
        assert E.kv8_attention_workspace(c, call()) == 0
    for bad in (dict(d_q=0), dict(d_out=0), dict(d_cu_q=0), dict(d_len=0), dict(d_table=0), dict(d_q=A + 8),
                dict(d_out=B + 2), dict(table_ld=0), dict(n_req=0), dict(n_req=1 << 24), dict(total_q=-1),
                dict(q_heads=0), dict(q_heads=12), dict(dtype=E.FP32), dict(window=-1), dict(window=4, causal=False),
                dict(max_q=0), dict(max_len=-1), dict(q_row=1024), dict(out_row=2044)):
        refused(E, E.kv8_attention, good_cache(E), call(**bad), H, 1 << 30)
        assert E.kv8_attention_workspace(good_cache(E), call(**bad)) == 0
    long = call(max_len=100000)
    need = E.kv8_attention_workspace(good_cache(E), long)
    assert need > 0
    refused(E, E.kv8_attention, good_cache(E), long, H, need - 1)
    refused(E, E.kv8_attention, good_cache(E), long, 0, need)
    refused(E, E.kv8_attention, good_cache(E), long, H + 4, need)
    E.kv8_attention(good_cache(E), call(total_q=0, d_q=0, d_out=0), 0, 0)


def test_attention_workgroups_fit_a_grid_beyond_max_q(E):
    """A call whose queries are far more than max_q says: tiles of 16 rows times splits stay below the
    2^24 workgroups of a grid's row.  The splits show in the workspace."""
    cache = E.kv8_cache(A, B, D, F, 1 << 20, 1, 256, 64, E.FP8_E4M3)
    for total_q, q_heads, max_len in ((100, 8, 1 << 20), (1 << 18, 16, 1 << 20), (1 << 20, 8, 1 << 20), (1 << 22, 1, 1 << 18),
                                      (1 << 24, 15, 1 << 20)):
        call = E.kv8_attention_args(A, B, D, F, G, 1 << 13, 1, total_q, q_heads, E.BF16, scale=0.1, max_q=1, max_len=max_len)
        splits = max(1, E.kv8_attention_workspace(cache, call) // (total_q * q_heads * 65 * 4))
        assert splits * (total_q * q_heads // 16 + 1) < 1 << 24
