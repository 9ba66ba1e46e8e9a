"""Host side of the operators on device data, without a GPU: what the calls refuse (before anything is queued), the frequencies of the rotary positions, workspace sizes."""
import math
import os

import numpy as np
import pytest


@pytest.fixture(scope="module")
def sts():
    from paper_2504_19516_amd import sts as m
    if not os.path.exists(m.LIB_PATH):
        from paper_2504_19516_amd import build
        build.build()
    m.lib()
    return m


def refused(sts, call, make, good, **change):
    """`call` of a description that is good but for `change`: STS_EINVAL. The addresses are never followed."""
    with pytest.raises(sts.StsError) as e:
        call(make(**{**good, **change}))
    assert e.value.code == sts.EINVAL, change


A = 1 << 20            # an address


def test_block_tables_refuses(sts):
    good = dict(n_requests=4, max_pages=8, max_rows=10, free_capacity=5, table_stride=8, cached=A, added=2 * A, free_pages=3 * A, n_free=4 * A, tables=5 * A, lens=6 * A,
                row_starts=7 * A, requests=8 * A, positions=9 * A, places=10 * A, n_free_left=11 * A, status=12 * A)
    for change in [dict(n_requests=-1), dict(n_requests=4097), dict(max_pages=-1), dict(max_rows=-1), dict(max_rows=(1 << 30) + 1), dict(free_capacity=-1), dict(table_stride=7), dict(n_free_left=4 * A),
                   dict(lens=A), dict(lens=2 * A)] + [{k: None} for k in good if k not in ("n_requests", "max_pages", "max_rows", "free_capacity", "table_stride")]:
        refused(sts, sts.op_block_tables, sts.BlockTables, good, **change)
    with pytest.raises(sts.StsError):
        sts._ck(sts.lib().sts_op_block_tables(None, None), "null")


def test_rope_refuses(sts):
    plain = sts.Rope(rotary_dim=64, theta=1e4)
    good = dict(dtype=1, rows=3, n_q=4, n_kv=2, d=64, pool_pages=7, q=A, q_stride=256, q_out=2 * A, q_out_stride=256, k=3 * A, k_stride=128, v=4 * A, v_stride=128, pool=5 * A,
                positions=6 * A, places=7 * A)
    call = lambda a: sts.op_rope(plain, a)  # noqa: E731
    for change in [dict(dtype=-1), dict(dtype=3), dict(dtype=0), dict(rows=-1), dict(n_q=-1), dict(n_kv=-1), dict(d=62), dict(d=96), dict(q=None), dict(q_out=None), dict(k=None), dict(v=None),
                   dict(pool=None), dict(positions=None), dict(places=None), dict(q_stride=255), dict(q_out_stride=0), dict(k_stride=127), dict(v_stride=127), dict(pool_pages=-1),
                   dict(k_out=8 * A, k_out_stride=100), dict(q_out=A, q_out_stride=300), dict(k_out=3 * A, k_out_stride=136), dict(n_kv=0),
                   dict(rows=(1 << 27) + 1), dict(q=A + 1), dict(q_out=2 * A + 1), dict(k=3 * A + 1), dict(k_out=8 * A + 1, k_out_stride=128), dict(v=4 * A + 1), dict(pool=5 * A + 1)]:
        refused(sts, call, sts.RopeRows, good, **change)
    ok = dict(rotary_dim=64, theta=1e4, factor=2.0, low=1.0, high=4.0, original_len=4096, scaling=3)
    bad = [dict(rotary_dim=0), dict(rotary_dim=63), dict(rotary_dim=258), dict(theta=0.0), dict(theta=math.nan), dict(theta=math.inf), dict(scaling=5), dict(scaling=-1), dict(factor=0.0),
           dict(factor=-1.0), dict(low=0.0), dict(high=1.0), dict(original_len=0), dict(interleaved=2), dict(magnitude=-1.0), dict(magnitude=math.inf), dict(scaling=4, theta=1.0),
           dict(scaling=4, high=0.5), dict(scaling=2, rotary_dim=2)]
    for change in bad:
        refused(sts, lambda r: sts.op_rope(r, sts.RopeRows(**good)), sts.Rope, ok, **change)
        refused(sts, sts.rope_frequencies, sts.Rope, ok, **change)
    # nothing to do
    sts.op_rope(plain, sts.RopeRows(**{**good, "rows": 0}))


def test_attention_refuses(sts):
    size = sts.attn_shared_workspace(6, 8, 2, 64)
    good = dict(dtype=1, n_requests=6, n_groups=2, n_q=8, n_kv=2, d=64, pool_pages=9, max_pages=5, table_stride=5, tables=A, lens=2 * A, group_starts=3 * A, shared_lens=4 * A,
                workspace=5 * A, workspace_bytes=size)
    batch = [dict(dtype=0), dict(dtype=3), dict(n_requests=-1), dict(n_requests=4097), dict(n_groups=-1), dict(n_groups=7), dict(n_q=7), dict(n_q=0), dict(n_kv=0), dict(n_q=66),
             dict(d=32), dict(d=96), dict(pool_pages=-1), dict(max_pages=-1), dict(max_pages=1 << 26, table_stride=1 << 26), dict(table_stride=4), dict(tables=None), dict(lens=None), dict(group_starts=None), dict(shared_lens=None),
             dict(workspace=None), dict(workspace=5 * A + 16), dict(workspace_bytes=size - 1), dict(n_kv=257, n_q=257), dict(n_requests=1, n_groups=1, max_pages=(1 << 26) + 1, table_stride=1 << 27)]
    layer = lambda b, q=A, qs=512, pool=A, out=A, os_=512, scale=0.0: sts.op_attn_shared(b, q, qs, pool, out, os_, None, scale)  # noqa: E731
    for change in batch:
        refused(sts, sts.op_attn_shared_plan, sts.AttnBatch, good, **change)
        refused(sts, layer, sts.AttnBatch, good, **change)
    refused(sts, layer, sts.AttnBatch, good, pool_pages=0)
    for bad in [dict(q=None), dict(q=A + 1), dict(pool=None), dict(pool=A + 8), dict(out=None), dict(out=A + 1), dict(qs=511), dict(os_=511), dict(scale=-1.0), dict(scale=math.nan),
                dict(scale=math.inf)]:
        refused(sts, lambda b: layer(b, **bad), sts.AttnBatch, good)
    none = sts.AttnBatch(**{**good, "n_requests": 0, "n_groups": 0})
    sts.op_attn_shared_plan(none)
    layer(none)


def test_attention_workspace(sts):
    for bad in [(-1, 8, 2, 64), (4097, 8, 2, 64), (4, 7, 2, 64), (4, 66, 2, 64), (4, 8, 2, 80), (4, 0, 0, 64)]:
        assert sts.attn_shared_workspace(*bad) == -1
    sizes = [sts.attn_shared_workspace(n, 32, 8, 128) for n in (1, 2, 64, 256, 4096)]
    assert sizes == sorted(sizes) and sizes[3] <= 256 << 20 and all(s % 256 == 0 for s in sizes)


def test_logprobs_refuses(sts):
    size = sts.op_logprobs_workspace(0, 2, 100000, 5)
    good = dict(dtype=0, rows=2, vocab=100000, top_k=5, row_stride=100000, logits=A, tokens=2 * A, logprob=3 * A, entropy=4 * A, lse=5 * A, rank=6 * A, top_logprob=7 * A, top_token=8 * A,
                workspace=9 * A, workspace_bytes=size)
    assert size > 0
    for change in [dict(dtype=-1), dict(dtype=3), dict(rows=-1), dict(rows=65536), dict(vocab=0), dict(vocab=1 << 31 - 1), dict(top_k=-1), dict(top_k=33), dict(vocab=4), dict(row_stride=99999),
                   dict(logits=None), dict(logits=A + 2), dict(tokens=None), dict(top_k=0), dict(workspace=None), dict(workspace=9 * A + 8), dict(workspace_bytes=size - 1)]:
        refused(sts, sts.op_logprobs, sts.Logprobs, good, **change)
    sts.op_logprobs(sts.Logprobs(**{**good, "rows": 0}))
    for bad in [(3, 2, 10, 1), (0, -1, 10, 1), (0, 2, 0, 1), (0, 2, 10, 33), (0, 2, 10, -1), (0, 65536, 10, 1), (0, 2, (1 << 31) - 1, 1)]:
        assert sts.op_logprobs_workspace(*bad) == -1
    assert sts.op_logprobs_workspace(1, 4000, 128256, 20) == 0


@pytest.mark.parametrize("length,low,high,theta,rotary", [(4, 1.0, 32.0, 1e4, 64), (6, 1.0, 1.0, 1e4, 64), (1, 1.0, 32.0, 1e4, 64), (1 << 30, 1.0, 2.0, 1.5, 8), (4096, 1.0, 1.0, 1e4, 64),
                                                           (1 << 30, 2.0 ** -10, 1.0, 1.125, 8)])
def test_rope_ramp_that_ends_outside_the_pairs(sts, length, low, high, theta, rotary):
    """Its ends are kept within 0 and rotary_dim - 1, and the pairs up to the first end come first."""
    i, theta = np.arange(rotary // 2), np.float64(np.float32(theta))
    w = theta ** (-2.0 * i / rotary)
    pair = lambda turns: rotary * math.log(length / (turns * 2 * math.pi)) / (2 * math.log(theta))  # noqa: E731
    a, b = max(math.floor(pair(high)), 0), min(math.ceil(pair(low)), rotary - 1)
    want = np.where(i <= a, w, np.where(i >= b, w / 16, w + (w / 16 - w) * (i - a) / max(b - a, 1)))
    got = sts.rope_frequencies(sts.Rope(rotary_dim=rotary, theta=theta, scaling=sts.ROPE_SCALINGS["ramp"], factor=16.0, low=low, high=high, original_len=length))
    np.testing.assert_allclose(got, want, rtol=1e-13)


def test_logprobs_refuses_vocabularies_above_the_most(sts):
    """Of a description that nothing else is wrong with."""
    good = dict(dtype=0, rows=2, vocab=1 << 30, top_k=5, row_stride=1 << 31, logits=A, tokens=2 * A, logprob=3 * A, workspace=9 * A, workspace_bytes=1 << 40)
    assert sts.op_logprobs_workspace(0, 2, 1 << 30, 5) > 0 and sts.op_logprobs_workspace(0, 2, (1 << 30) + 1, 5) == -1
    refused(sts, sts.op_logprobs, sts.Logprobs, good, vocab=(1 << 30) + 1)


@pytest.mark.parametrize("rotary,theta", [(128, 5e5), (64, 1e4), (40, 1e6), (2, 100.0)])
def test_rope_frequencies(sts, rotary, theta):
    i = np.arange(rotary // 2)
    w = np.float64(np.float32(theta)) ** (-2.0 * i / rotary)
    get = lambda **k: sts.rope_frequencies(sts.Rope(rotary_dim=rotary, theta=theta, **k))  # noqa: E731
    near = lambda a, b: np.testing.assert_allclose(a, b, rtol=1e-13)  # noqa: E731
    near(get(), w)
    near(get(scaling=sts.ROPE_SCALINGS["linear"], factor=4.0), w / 4)
    if rotary > 2:
        base = get(scaling=sts.ROPE_SCALINGS["base"], factor=8.0)
        near(base[0], 1.0)
        near(base[-1], w[-1] / 8)                                          # the slowest pair is slowed by the whole factor
    bands = get(scaling=sts.ROPE_SCALINGS["bands"], factor=8.0, low=1.0, high=4.0, original_len=8192)
    for f, x in zip(bands, w):
        wavelength = 2 * math.pi / x
        if wavelength < 8192 / 4:
            near(f, x)
        elif wavelength > 8192:
            near(f, x / 8)
        else:
            s = (8192 / wavelength - 1.0) / 3.0
            near(f, (1 - s) * x / 8 + s * x)
    ramp = get(scaling=sts.ROPE_SCALINGS["ramp"], factor=16.0, low=1.0, high=32.0, original_len=4096)
    pair = lambda turns: rotary * math.log(4096 / (turns * 2 * math.pi)) / (2 * math.log(np.float64(np.float32(theta))))  # noqa: E731
    a, b = max(math.floor(pair(32.0)), 0), min(math.ceil(pair(1.0)), rotary - 1)
    for j, (f, x) in enumerate(zip(ramp, w)):
        s = min(max((j - a) / max(b - a, 0.001), 0.0), 1.0)
        near(f, x / 16 * s + x * (1 - s))
