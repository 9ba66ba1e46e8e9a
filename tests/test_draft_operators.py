"""Host side of the operators that verify drafted tokens, without a GPU: what the calls refuse (before anything is queued), workspace sizes, calls with nothing to do."""
import math

import pytest

from tests.test_operators import A, refused, sts  # noqa: F401

ROWS = dict(dtype=1, rows=3, n_q=4, n_kv=2, d=64, pool_pages=7, q=A, q_stride=256, q_out=2 * A, q_out_stride=256, k=3 * A, k_stride=128, v=4 * A, v_stride=128, pool=5 * A,
            positions=6 * A, places=7 * A)


def test_norm_rope_refuses(sts):  # noqa: F811
    rope = sts.Rope(rotary_dim=64, theta=1e4)
    good = dict(dtype=1, offset_one=0, eps=1e-6, q_gain=8 * A, k_gain=9 * A)
    for change in [dict(dtype=-1), dict(dtype=3), dict(offset_one=2), dict(offset_one=-1), dict(eps=-1e-6), dict(eps=math.nan), dict(eps=math.inf), dict(q_gain=8 * A + 1), dict(k_gain=9 * A + 1),
                   dict(dtype=0, q_gain=8 * A + 2)]:
        refused(sts, lambda n: sts.op_norm_rope(n, rope, sts.RopeRows(**ROWS)), sts.HeadNorm, good, **change)
    norm = sts.HeadNorm(**good)
    call = lambda a: sts.op_norm_rope(norm, rope, a)  # noqa: E731
    for change in [dict(rows=-1), dict(d=62), dict(q=None), dict(q_stride=255), dict(pool_pages=-1), dict(places=None), dict(positions=None), dict(q=A + 1)]:
        refused(sts, call, sts.RopeRows, ROWS, **change)
    wide = dict(ROWS, pool=None, k_out=10 * A, k_out_stride=4096, q_stride=4096, q_out_stride=4096, k_stride=4096)
    refused(sts, call, sts.RopeRows, wide, d=514)
    refused(sts, lambda r: sts.op_norm_rope(norm, r, sts.RopeRows(**ROWS)), sts.Rope, dict(rotary_dim=64, theta=1e4), rotary_dim=63)
    for args in [(None, rope, ROWS), (norm, None, ROWS), (norm, rope, None)]:
        p = [None if x is None else sts.C.byref(sts.RopeRows(**x) if isinstance(x, dict) else x) for x in args]
        assert sts.lib().sts_op_norm_rope(*p, None) == sts.EINVAL
    sts.op_norm_rope(norm, rope, sts.RopeRows(**{**ROWS, "rows": 0}))
    sts.op_norm_rope(sts.HeadNorm(), rope, sts.RopeRows(**{**ROWS, "rows": 0}))


def test_norm_rope_looks_at_no_gains_of_heads_that_are_none(sts):  # noqa: F811
    """Wherever their pointer leads."""
    rope, odd = sts.Rope(rotary_dim=64, theta=1e4), 8 * A + 1
    call = lambda a, **g: sts.op_norm_rope(sts.HeadNorm(dtype=1, eps=1e-6, **g), rope, sts.RopeRows(**{**ROWS, "rows": 0, "pool": None, "k_out": 10 * A, "k_out_stride": 128, **a}))  # noqa: E731
    call(dict(n_q=0), q_gain=odd)
    call(dict(n_kv=0), k_gain=odd)
    for heads, gain in (("n_kv", "q_gain"), ("n_q", "k_gain")):
        with pytest.raises(sts.StsError):
            call({heads: 0}, **{gain: odd})


def test_tree_attention_refuses(sts):  # noqa: F811
    size = sts.attn_tree_workspace(6, 40, 8, 2, 64)
    good = dict(dtype=1, n_requests=6, max_rows=40, n_q=8, n_kv=2, d=64, pool_pages=9, max_pages=5, table_stride=5, tables=A, cached=2 * A, row_starts=3 * A, parents=4 * A,
                positions=6 * A, workspace=5 * A, workspace_bytes=size)
    layer = lambda b, q=A, qs=512, pool=A, out=A, os_=512, scale=0.0: sts.op_attn_tree(b, q, qs, pool, out, os_, None, scale)  # noqa: E731
    for change in [dict(dtype=0), dict(dtype=3), dict(n_requests=-1), dict(n_requests=4097), dict(max_rows=-1), dict(max_rows=65537), dict(n_q=7), dict(n_q=0), dict(n_kv=0), dict(n_q=66),
                   dict(d=32), dict(d=96), dict(pool_pages=-1), dict(max_pages=-1), dict(table_stride=4), dict(tables=None), dict(cached=None), dict(row_starts=None), dict(parents=None),
                   dict(workspace=None), dict(workspace=5 * A + 16), dict(workspace_bytes=size - 1), dict(n_kv=257, n_q=257), dict(max_pages=(1 << 26) + 1, table_stride=1 << 27),
                   dict(max_pages=1 << 28, table_stride=1 << 28), dict(max_rows=41), dict(n_requests=4096), dict(positions=4 * A), dict(positions=2 * A), dict(positions=3 * A)]:
        refused(sts, sts.op_attn_tree_plan, sts.TreeBatch, good, **change)
        refused(sts, layer, sts.TreeBatch, good, **change)
    # lines beyond 32 bits: 7 segments of 2^26 pages fit, 17 do not
    refused(sts, sts.op_attn_tree_plan, sts.TreeBatch, dict(good, workspace_bytes=1 << 40), n_requests=16, max_pages=1 << 26, table_stride=1 << 26)
    refused(sts, layer, sts.TreeBatch, good, pool_pages=0)
    for bad in [dict(q=None), dict(q=A + 1), dict(pool=None), dict(pool=A + 8), dict(out=None), dict(out=A + 1), dict(qs=511), dict(os_=511), dict(scale=-1.0), dict(scale=math.nan),
                dict(scale=math.inf)]:
        refused(sts, lambda b: layer(b, **bad), sts.TreeBatch, good)
    for none in (dict(n_requests=0), dict(max_rows=0)):
        b = sts.TreeBatch(**{**good, **none})
        sts.op_attn_tree_plan(b)
        layer(b)


def test_tree_attention_workspace(sts):  # noqa: F811
    for bad in [(-1, 4, 8, 2, 64), (4097, 4, 8, 2, 64), (4, -1, 8, 2, 64), (4, 65537, 8, 2, 64), (4, 4, 7, 2, 64), (4, 4, 66, 2, 64), (4, 4, 8, 2, 80), (4, 4, 0, 0, 64)]:
        assert sts.attn_tree_workspace(*bad) == -1
    sizes = [sts.attn_tree_workspace(n, n * 26, 32, 8, 128) for n in (1, 2, 64, 256)]
    assert sizes == sorted(sizes) and sizes[2] <= 128 << 20 and all(s % 256 == 0 for s in sizes)


ADJUST = dict(dtype=0, rows=3, vocab=1000, n_requests=3, row_stride=1000, out_stride=1000, logits=A, out=2 * A, requests=3 * A, n_biases=5, n_masks=2, token_stride=100, mask_stride=32,
              tokens=4 * A, lens=5 * A, prompt_lens=6 * A, repetition=7 * A, frequency=8 * A, presence=9 * A, row_starts=10 * A, parents=11 * A, drafted=12 * A, bias_starts=13 * A,
              bias_tokens=14 * A, bias_values=15 * A, masks=16 * A, mask_rows=17 * A)


@pytest.mark.parametrize("change", [dict(dtype=-1), dict(dtype=3), dict(rows=-1), dict(rows=65536), dict(vocab=0), dict(vocab=(1 << 30) + 1, row_stride=1 << 31, out_stride=1 << 31, mask_stride=1 << 26),
                                    dict(n_requests=-1), dict(row_stride=999), dict(out_stride=999), dict(logits=None), dict(out=None), dict(logits=A + 2), dict(out=2 * A + 1),
                                    dict(out=A, out_stride=1004), dict(requests=None, n_requests=2), dict(lens=None), dict(token_stride=-1), dict(row_starts=None), dict(parents=None),
                                    dict(tokens=None, drafted=None), dict(bias_starts=None), dict(bias_values=None), dict(bias_tokens=None), dict(n_biases=-1), dict(n_masks=-1),
                                    dict(mask_rows=None), dict(mask_stride=31), dict(masks=None)])
def test_adjust_logits_refuses(sts, change):  # noqa: F811
    refused(sts, sts.op_adjust_logits, sts.AdjustLogits, ADJUST, **change)


def test_adjust_logits_of_no_rows(sts):  # noqa: F811
    sts.op_adjust_logits(sts.AdjustLogits(**{**ADJUST, "rows": 0}))
    assert sts.lib().sts_op_adjust_logits(None, None) == sts.EINVAL


def test_tree_accept_refuses(sts):  # noqa: F811
    good = dict(n_requests=3, max_rows=20, cached=A, row_starts=2 * A, parents=3 * A, tokens=4 * A, chosen=5 * A, lens=6 * A, counts=7 * A, path=8 * A, next_token=9 * A)
    for change in [dict(n_requests=-1), dict(n_requests=4097), dict(max_rows=-1)] + [{k: None} for k in good if k not in ("n_requests", "max_rows")]:
        refused(sts, sts.op_tree_accept, sts.TreeAccept, good, **change)
    pages = dict(good, max_pages=4, free_capacity=9, table_stride=4, tables=10 * A, free_pages=11 * A, n_free=12 * A)
    for change in [dict(free_pages=None), dict(n_free=None), dict(max_pages=-1), dict(max_pages=(1 << 26) + 1, table_stride=1 << 27), dict(free_capacity=-1), dict(table_stride=3)]:
        refused(sts, sts.op_tree_accept, sts.TreeAccept, pages, **change)
    sts.op_tree_accept(sts.TreeAccept(**{**good, "n_requests": 0}))
    assert sts.lib().sts_op_tree_accept(None, None) == sts.EINVAL


def test_tree_accept_refuses_more_rows_than_block_tables_make(sts):  # noqa: F811
    """Beyond 2^30 a step of 64 rows of a path would leave 32 bits near 2^31."""
    good = dict(n_requests=0, max_rows=1 << 30, cached=A, row_starts=2 * A, parents=3 * A, tokens=4 * A, chosen=5 * A, lens=6 * A, counts=7 * A, path=8 * A, next_token=9 * A)
    sts.op_tree_accept(sts.TreeAccept(**good))
    for rows in ((1 << 30) + 1, (1 << 31) - 1):
        refused(sts, sts.op_tree_accept, sts.TreeAccept, good, max_rows=rows)


def test_tree_accept_refuses_outputs_in_each_others_place(sts):  # noqa: F811
    """Or in that of what is read: all but lens = cached, whose test runs on the GPU."""
    good = dict(n_requests=3, max_rows=20, cached=A, row_starts=2 * A, parents=3 * A, tokens=4 * A, chosen=5 * A, lens=6 * A, counts=7 * A, path=8 * A, next_token=9 * A, max_pages=4,
                free_capacity=9, table_stride=4, tables=10 * A, free_pages=11 * A, n_free=12 * A)
    written, read = ("lens", "counts", "next_token", "path", "free_pages", "n_free"), ("row_starts", "cached", "tables", "parents", "tokens", "chosen")
    for i, w in enumerate(written):
        for other in written[i + 1:] + read:
            if (w, other) != ("lens", "cached") and not (w == "path" and other in ("parents", "tokens", "chosen")):
                refused(sts, sts.op_tree_accept, sts.TreeAccept, good, **{w: good[other]})


def test_tree_compact_refuses(sts):  # noqa: F811
    good = dict(n_requests=3, max_rows=20, n_kv=2, d=64, pool_pages=9, max_pages=5, table_stride=5, tables=A, cached=2 * A, row_starts=3 * A, counts=4 * A, path=5 * A)
    call = lambda a: sts.op_tree_compact(a, [6 * A, 7 * A])  # noqa: E731
    for change in [dict(n_requests=-1), dict(n_requests=4097), dict(max_rows=-1), dict(n_kv=0), dict(n_kv=257), dict(d=96), dict(pool_pages=-1), dict(max_pages=-1),
                   dict(max_pages=(1 << 26) + 1, table_stride=1 << 27), dict(table_stride=4), dict(tables=None), dict(cached=None), dict(row_starts=None), dict(counts=None), dict(path=None)]:
        refused(sts, call, sts.TreeCompact, good, **change)
    for pools in ([6 * A, None], [6 * A + 8], [6 * A] * 257):
        refused(sts, lambda a: sts.op_tree_compact(a, pools), sts.TreeCompact, good)
    assert sts.lib().sts_op_tree_compact(sts.C.byref(sts.TreeCompact(**good)), None, 1, None) == sts.EINVAL
    assert sts.lib().sts_op_tree_compact(sts.C.byref(sts.TreeCompact(**good)), None, -1, None) == sts.EINVAL
    sts.op_tree_compact(sts.TreeCompact(**good), [])
    for none in (dict(n_requests=0), dict(max_rows=0)):
        call(sts.TreeCompact(**{**good, **none}))
