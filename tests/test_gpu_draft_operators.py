"""Operators of a step that verifies drafted tokens (norms of heads with rotary positions, attention for trees of drafted tokens, penalties and masks on logits, the accepted
path) against plain implementations in 64 bits, on the same rounded inputs.

Tolerances. u is half a step of the output's type (bf16 2^-8, fp16 2^-11, fp32 2^-24), relative to the value. Each test states its bound from the
roundings that the kernels make; nothing is measured first."""
import ctypes as C

import numpy as np
import pytest

from tests.device import Device, pool_of, rounded, stored, widened
from tests.test_gpu_operators import HALF, ROPES, near, rope_of, rope_reference, sts  # noqa: F401

pytestmark = pytest.mark.gpu
assert ROPES


# ------------------------------------------------------------------------------------------ norms of heads with rotary positions
def norm_reference(x, gain, eps, offset):
    """x [rows, heads, d] float64."""
    g = 1.0 if gain is None else gain.astype(np.float64) + offset
    return x / np.sqrt((x * x).mean(axis=2, keepdims=True) + eps) * g


# One rounding to the type. Behind it: up to 24 additions of squares (a lane's 16, then between lanes) and the mean, 2^-19.4 in all and half of that in the root; the
# root's approximation 2^-23, two products 2^-23, so within 2^-19 of x / root * gain; then the rotation's 2^-21. 2^-18 holds all of it; behind the pairs, size is |y|.
def norm_rope_bound(y, size, dtype):
    return HALF[dtype] * np.abs(y) + size * 2.0 ** -18 + 1e-7 * (dtype == "f16") + 1e-30


def norm_rope_reference(sts, rope, x, gain, eps, offset, positions):  # noqa: F811
    z = norm_reference(x, gain, eps, offset)
    y, size = rope_reference(sts, rope, z, positions)
    return y, np.maximum(size, np.abs(z))


def gains_of(rng, d, dtype, offset):
    return [rounded((0.0 if offset else 1.0) + 0.4 * rng.standard_normal(d), dtype) for _ in range(2)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("name,rotary,interleaved,d,gain", [("plain", 128, 0, 128, "f32"), ("linear", 64, 0, 64, "bf16"), ("base", 32, 1, 64, "f16"), ("bands", 128, 1, 128, "bf16"),
                                                            ("ramp", 104, 0, 128, "f16"), ("ramp", 40, 1, 64, None), ("plain", 2, 0, 6, "f32"), ("bands", 250, 1, 257, "f32"),
                                                            ("linear", 256, 0, 512, "bf16"), ("plain", 40, 0, 64, "f32"), ("plain", 80, 0, 80, "bf16"), ("plain", 8, 1, 96, "f16")])
def test_norm_rope_turns_rows(sts, dtype, name, rotary, interleaved, d, gain):  # noqa: F811
    """Q out of place from a strided buffer and K in place; gains of any type, whole or less 1, or none; rows of zeros, of one element, of large and small ones."""
    rng = np.random.default_rng(rotary + d)
    rows, n_q, n_kv, eps, offset = 37, 5, 2, 1e-6, int(gain == "f16")
    rope = rope_of(sts, name, rotary, interleaved)
    positions = np.concatenate([[0, 1, 2 ** 31 - 1, -1, -70000], rng.integers(0, 2 ** 20, rows - 5)]).astype(np.int32)
    q, k = (rounded(rng.standard_normal((rows, h, d)), dtype) for h in (n_q, n_kv))
    q[3], q[4] = 0.0, 0.0
    q[4, :, d // 2] = -3.0
    q[5:7] = rounded(q[5:7] * 200.0, dtype)
    k[3] = rounded(k[3] * 2.0 ** -9, dtype)
    ld = (n_q + n_kv) * d + 3
    both = np.full((rows, ld), 5.0, np.float32)
    both[:, :n_q * d], both[:, n_q * d:-3] = q.reshape(rows, -1), k.reshape(rows, -1)
    size = 4 if dtype == "f32" else 2
    gains = gains_of(rng, d, gain or "f32", offset) if gain else [None, None]
    if gain == "bf16":
        gains[1] = None                                                    # one of them alone
    with Device() as dev:
        for aligned in (False, True):
            pad = ld if not aligned else -(-ld // 8) * 8
            rows_in = np.full((rows, pad), 5.0, np.float32)
            rows_in[:, :ld] = both
            buf, out = dev.put(rows_in, dtype), dev.alloc(rows * n_q * d * size)
            norm = sts.HeadNorm(dtype=sts.DTYPES[gain or "f32"], offset_one=offset, eps=eps, q_gain=None if gains[0] is None else dev.put(gains[0], gain),
                                k_gain=None if gains[1] is None else dev.put(gains[1], gain))
            sts.op_norm_rope(norm, rope, sts.RopeRows(dtype=sts.DTYPES[dtype], rows=rows, n_q=n_q, n_kv=n_kv, d=d, q=buf, q_stride=pad, q_out=out, q_out_stride=n_q * d, k=buf + n_q * d * size,
                                                      k_stride=pad, k_out=buf + n_q * d * size, k_out_stride=pad, positions=dev.ints(positions)))
            dev.sync()
            got_q, got = dev.get(out, (rows, n_q, d), dtype), dev.get(buf, (rows, pad), dtype)
            for y, x, g in ((got_q, q, gains[0]), (got[:, n_q * d:ld - 3].reshape(rows, n_kv, d), k, gains[1])):
                want, s = norm_rope_reference(sts, rope, x.astype(np.float64), g, np.float64(np.float32(eps)), offset, positions)
                near(y, want, norm_rope_bound(want, s, dtype))
            assert np.array_equal(got[:, :n_q * d], rows_in[:, :n_q * d]) and (got[:, ld - 3:] == 5.0).all()        # what is not K is left as it was


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows,n_q,n_kv,d,rotary,interleaved,offset", [(1, 4, 4, 64, 64, 0, 0), (3, 32, 8, 128, 128, 0, 0), (33, 8, 1, 128, 64, 1, 0), (70, 6, 2, 64, 24, 0, 2),
                                                                      (500, 32, 8, 128, 128, 0, 0), (513, 4, 4, 64, 32, 1, 0), (517, 8, 2, 128, 104, 0, 2), (4507, 32, 8, 128, 128, 0, 0),
                                                                      (2049, 32, 8, 128, 104, 0, 0), (9001, 6, 3, 64, 40, 1, 0), (600, 0, 5, 128, 128, 0, 0)])
def test_norm_rope_appends_to_pages(sts, dtype, rows, n_q, n_kv, d, rotary, interleaved, offset):  # noqa: F811
    """K's rows in the pool are those of k_out, V's the inputs'; rows without a place are not appended, what no row fills is left as it was."""
    rng = np.random.default_rng(rows)
    rope = rope_of(sts, "bands", rotary, interleaved)
    pages, eps = rows // 4 + 9, 1e-5
    order, positions, places, used = rng.permutation(pages), [], [], 0
    while len(positions) < rows:
        start, m = int(rng.integers(0, 40)), min(int(rng.integers(1, 60)), rows - len(positions))
        first, need = start // 16, (start + m - 1) // 16 - start // 16 + 1
        fits = used + need <= pages
        places += [int(order[used + (start + t) // 16 - first]) * 16 + (start + t) % 16 if fits else -1 for t in range(m)]
        positions += range(start + 50000, start + 50000 + m)
        used += need if fits else 0
    places = np.asarray(places, np.int32)
    if rows > 3:
        places[1], places[-1] = -1, pages * 16
    qkv = rounded(1.5 * rng.standard_normal((rows, (n_q + 2 * n_kv) * d)), dtype)
    old = rounded(rng.standard_normal((pages, n_kv, 32 * d)), dtype)
    gains, ld = gains_of(rng, d, dtype, 0), qkv.shape[1]
    with Device() as dev:
        base, pool, out, kout = dev.put(qkv, dtype, offset), dev.put(old, dtype), dev.alloc(rows * n_q * d * 2), dev.alloc(rows * n_kv * d * 2)
        norm = sts.HeadNorm(dtype=sts.DTYPES[dtype], eps=eps, q_gain=dev.put(gains[0], dtype), k_gain=dev.put(gains[1], dtype))
        sts.op_norm_rope(norm, rope, sts.RopeRows(dtype=sts.DTYPES[dtype], rows=rows, n_q=n_q, n_kv=n_kv, d=d, pool_pages=pages, q=base, q_stride=ld, q_out=out, q_out_stride=n_q * d,
                                                  k=base + n_q * d * 2, k_stride=ld, k_out=kout, k_out_stride=n_kv * d, v=base + (n_q + n_kv) * d * 2, v_stride=ld, pool=pool,
                                                  positions=dev.ints(positions), places=dev.put(places)))
        dev.sync()
        got_q, got_k = dev.get(out, (rows, n_q, d), dtype), dev.get(kout, (rows, n_kv, d), dtype)
        got = dev.get(pool, old.shape, dtype)
    x = qkv.reshape(rows, n_q + 2 * n_kv, d).astype(np.float64)
    for y, part, g in ((got_q, x[:, :n_q], gains[0]), (got_k, x[:, n_q:n_q + n_kv], gains[1])):
        want, s = norm_rope_reference(sts, rope, part, g, np.float64(np.float32(eps)), 0, positions)
        near(y, want, norm_rope_bound(want, s, dtype))
    kp, vp = old[:, :, :16 * d].reshape(pages, n_kv, 16, d).copy(), old[:, :, 16 * d:].reshape(pages, n_kv, d, 16).copy()
    for r, p in enumerate(places):
        if 0 <= p < pages * 16:
            kp[p // 16, :, p % 16], vp[p // 16, :, :, p % 16] = got_k[r], x[r, n_q + n_kv:]
    assert np.array_equal(got[:, :, :16 * d], kp.reshape(pages, n_kv, -1)) and np.array_equal(got[:, :, 16 * d:], vp.reshape(pages, n_kv, -1))


def test_norm_rope_of_zeros_infinities_and_nan(sts):  # noqa: F811
    """By the formula: zeros stay zeros with an eps above 0 and are NaN without one; an infinity makes its head's other elements 0 and itself NaN; other heads do not see it."""
    rope, rows, n_q, d = sts.Rope(rotary_dim=2, theta=1e4), 3, 3, 64
    x = rounded(np.random.default_rng(1).standard_normal((rows, n_q, d)), "bf16")
    x[0, 0] = 0.0
    x[1, 1, 40], x[2, 2, 5] = np.inf, np.nan
    with Device() as dev:
        for eps in (1e-6, 0.0):
            q, out = dev.put(x, "bf16"), dev.alloc(x.size * 2)
            sts.op_norm_rope(sts.HeadNorm(eps=eps), rope, sts.RopeRows(dtype=1, rows=rows, n_q=n_q, d=d, q=q, q_stride=n_q * d, q_out=out, q_out_stride=n_q * d, positions=dev.ints([0, 5, 9])))
            dev.sync()
            got = dev.get(out, x.shape, "bf16")
            assert (got[0, 0] == 0.0).all() if eps else np.isnan(got[0, 0]).all()
            assert np.isnan(got[1, 1, 40]) and (np.delete(got[1, 1], 40) == 0.0).all() and np.isnan(got[2, 2]).all()
            for r, h in ((0, 1), (0, 2), (1, 0), (1, 2), (2, 0), (2, 1)):
                assert np.isfinite(got[r, h]).all()


@pytest.mark.parametrize("rows", [3, 700])
def test_norm_rope_of_one_kind_of_heads(sts, rows):  # noqa: F811
    """Q without K, or K without Q: the other's pointers, its gains among them, are not followed."""
    rng = np.random.default_rng(rows)
    heads, d, eps = 3, 128, 1e-6
    rope, positions = rope_of(sts, "plain", d, 0), np.arange(rows) % 40
    x, gain = rounded(rng.standard_normal((rows, heads, d)), "bf16"), gains_of(rng, d, "bf16", 0)[0]
    want, size = norm_rope_reference(sts, rope, x.astype(np.float64), gain, np.float64(np.float32(eps)), 0, positions)
    with Device() as dev:
        for kind, other in (("q", "k"), ("k", "q")):
            buf, out, g, nowhere = dev.put(x, "bf16"), dev.alloc(x.size * 2), dev.put(gain, "bf16"), 1 << 20
            a = {kind: buf, kind + "_stride": heads * d, kind + "_out": out, kind + "_out_stride": heads * d, "n_q" if kind == "q" else "n_kv": heads, other: nowhere, other + "_out": nowhere}
            sts.op_norm_rope(sts.HeadNorm(dtype=1, eps=eps, **{kind + "_gain": g, other + "_gain": nowhere}), rope, sts.RopeRows(dtype=1, rows=rows, d=d, positions=dev.ints(positions), **a))
            dev.sync()
            near(dev.get(out, x.shape, "bf16"), want, norm_rope_bound(want, size, "bf16"))


# ------------------------------------------------------------------------------------------ attention of drafted trees
def chain(m):
    return list(range(-1, m - 1))


def random_tree(rng, m, roots=1):
    return [-1 if j < roots else int(rng.integers(0, j)) for j in range(m)]


def star(m):
    return [-1] + [0] * (m - 1)


def ancestors(parents):
    """Of each node: the numbers of its ancestors and its own, or None if it is none."""
    out = []
    for j, p in enumerate(parents):
        up = [] if p == -1 else out[p] if 0 <= p < j else None
        out.append(None if up is None else up + [j])
    return out


def tree_case(rng, cached, trees, n_kv, d, spare=3):
    """k, v by request (cached tokens and nodes), tables, pages."""
    lens = [c + len(t) for c, t in zip(cached, trees)]
    k, v = ([rng.standard_normal((m, n_kv, d)) for m in lens] for _ in range(2))
    need = [-(-m // 16) for m in lens]
    tables = np.full((len(lens), max(need) + 2), -9, np.int32)
    order, used = rng.permutation(sum(need) + spare), 0
    for r, m in enumerate(need):
        tables[r, :m] = order[used:used + m]
        used += m
    return k, v, tables, sum(need) + spare


def tree_reference(q, k, v, cached, trees, heads, scale, dtype):
    """Output, its bound, lse and its bound, of all rows; NaN-free. Bounds as for the attention over shared prefixes: a probability in two numbers of the type is off by less than
    one rounding of it, u; a score of d products in fp32 by d 2^-24 of the sum of their sizes, which is relative in the probability; the output is rounded once."""
    n, n_q, d = q.shape
    out, bound, lse, lb, u = np.zeros((n, n_q, d)), np.zeros((n, n_q, d)), np.full((n, n_q), -np.inf), np.zeros((n, n_q)), HALF[dtype]
    row = 0
    for r, (c, tree) in enumerate(zip(cached, trees)):
        for up in ancestors(tree):
            if up is not None:
                seen = list(range(c)) + [c + j for j in up]
                for h in range(n_q):
                    kh, vh = k[r][seen, h // heads].astype(np.float64), v[r][seen, h // heads].astype(np.float64)
                    x = kh @ q[row, h].astype(np.float64) * scale
                    m = x.max()
                    p = np.exp(x - m)
                    p, z = p / p.sum(), p.sum()
                    some = ~np.isneginf(x)                                 # a score of -inf is exact, and its weight is 0
                    delta = 2.0 ** -24 * d * (np.abs(kh[some]) @ np.abs(q[row, h]).astype(np.float64) * scale).max() + 2.0 ** -21 * (1 + np.abs(x - m)[some].max() * 2.0 ** -3)
                    out[row, h], lse[row, h], size = p @ vh, m + np.log(z), p @ np.abs(vh)
                    bound[row, h] = u * (np.abs(out[row, h]) + size) + 2 * delta * size + (2.0 ** -25 * np.abs(vh).sum(0) + 2.0 ** -24 if dtype == "f16" else 0.0) + 1e-30
                    lb[row, h] = delta + 2.0 ** -22 * (abs(lse[row, h]) + np.abs(x).max() + 8)
            row += 1
    return out, bound, lse, lb


def starts_of(trees):
    return np.concatenate([[0], np.cumsum([len(t) for t in trees])]).astype(np.int32)


def run_tree(sts, dev, dtype, q, pool, tables, cached, trees, heads, scale=0.0, stream=None, starts=None, spare_rows=0, q_pad=0, out_pad=0, q_offset=0, pool_pages=None, want_lse=True,
             want_positions=True):
    """Rows behind the last are of garbage and must stay as they were."""
    n, n_q, d = q.shape
    n_kv, rows = n_q // heads, n + spare_rows
    size = sts.attn_tree_workspace(len(cached), rows, n_q, n_kv, d)
    qs = np.full((rows, n_q * d + q_pad), np.nan, np.float32)
    qs[:n, :n_q * d] = q.reshape(n, -1)
    parents = np.full(rows, 12345, np.int32)
    parents[:n] = [p for t in trees for p in t]
    out = dev.put(np.full((rows, n_q * d + out_pad), 7.0), dtype)
    lse, positions = dev.put(np.full((rows, n_q), 7.0, np.float32)), dev.ints([777] * rows)
    batch = sts.TreeBatch(dtype=sts.DTYPES[dtype], n_requests=len(cached), max_rows=rows, n_q=n_q, n_kv=n_kv, d=d, pool_pages=pool.shape[0] if pool_pages is None else pool_pages,
                          max_pages=tables.shape[1], table_stride=tables.shape[1], tables=dev.ints(tables), cached=dev.ints(cached),
                          row_starts=dev.ints(starts_of(trees) if starts is None else starts), parents=dev.ints(parents), positions=positions if want_positions else None,
                          workspace=dev.put(np.full(size, 0xAB, np.uint8)), workspace_bytes=size)
    args = (batch, dev.put(qs, dtype, q_offset), n_q * d + q_pad, dev.put(pool, dtype), out, n_q * d + out_pad, lse if want_lse else None, scale, stream)

    def call():
        sts.op_attn_tree_plan(batch, stream)
        sts.op_attn_tree(*args)
    call()
    dev.sync()
    got, got_lse, pos = dev.get(out, (rows, n_q * d + out_pad), dtype), dev.get(lse, (rows, n_q), "f32"), dev.get(positions, rows, "i32")
    assert (got[:, n_q * d:] == 7.0).all()
    if starts is None:
        assert (got[n:] == 7.0).all() and (got_lse[n:] == 7.0).all() and (pos[n:] == 777).all()
    return got[:n, :n_q * d].reshape(n, n_q, d), got_lse[:n], pos[:n], call, (out, lse, positions)


def check_tree(got, lse, want, cached=None, trees=None, positions=None):
    out, bound, want_lse, lb = want
    near(got, out, bound)
    some = np.isfinite(want_lse)
    near(lse[some], want_lse[some], lb[some])
    assert np.isneginf(lse[~some]).all() and (got[~some] == 0.0).all()
    if positions is not None:
        assert positions.tolist() == [-1 if up is None else c + len(up) - 1 for c, t in zip(cached, trees) for up in ancestors(t)]


TREES = [
    # (query heads, kv heads, d, [(cached, kind, nodes)])
    (4, 4, 64, [(0, "chain", 1)]),
    (4, 1, 64, [(33, "tree", 5)]),
    (32, 8, 128, [(1500, "tree", 26)]),
    (32, 8, 128, [(70, "chain", 5), (16, "chain", 5), (333, "chain", 5), (1, "chain", 5), (15, "chain", 4)]),
    (8, 8, 128, [(100, "tree", 33), (0, "star", 32), (64, "tree", 31)]),
    (32, 8, 128, [(900, "tree", 64), (31, "star", 64), (48, "chain", 64), (4, "forest", 40)]),
    (64, 8, 128, [(300, "tree", 13), (0, "chain", 1), (77, "tree", 4), (512, "forest", 3), (2000, "tree", 16), (9, "tree", 0)]),
    (10, 2, 64, [(201, "tree", 7), (31, "tree", 20), (6, "chain", 3)]),
    (32, 1, 64, [(64, "tree", 3), (33, "star", 9)]),
    (16, 16, 64, [(48, "tree", 70), (0, "chain", 256), (17, "tree", 256), (5, "star", 129)]),
    (28, 4, 128, [(1600, "tree", 37), (11, "chain", 17)]),
    (4, 2, 128, [(9000, "chain", 2)]),
    (8, 1, 64, [(30000, "tree", 12), (1, "tree", 2)]),
    (6, 3, 64, [(25, "tree", 100), (160, "tree", 15), (33, "chain", 40), (0, "forest", 9)]),
    (256, 256, 64, [(32, "tree", 3), (5, "chain", 2)]),
    (32, 8, 128, [(3, "tree", 255), (2047, "tree", 200)]),
    (2, 2, 64, [(1 + i % 37, "tree" if i % 3 else "chain", 1 + i % 5) for i in range(1000)]),
    (58, 2, 64, [(30, "tree", 256), (5, "chain", 200), (77, "tree", 1), (0, "star", 5)]),
    (14, 2, 128, [(300, "tree", 256), (17, "tree", 19)]),
]
KINDS = {"chain": lambda rng, m: chain(m), "tree": random_tree, "star": lambda rng, m: star(m), "forest": lambda rng, m: random_tree(rng, m, min(m, 3))}


def tree_inputs(rng, dtype, requests, n_q, n_kv, d, behind=np.nan, scale=2.0):
    cached, trees = [c for c, _, _ in requests], [KINDS[kind](rng, m) if m else [] for _, kind, m in requests]
    k, v, tables, pages = tree_case(rng, cached, trees, n_kv, d)
    k, v = [rounded(x, dtype) for x in k], [rounded(x, dtype) for x in v]
    q = rounded(scale * rng.standard_normal((sum(map(len, trees)), n_q, d)), dtype)
    return q, k, v, tables, pages, cached, trees


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("case", range(len(TREES)))
def test_tree_attention(sts, dtype, case):  # noqa: F811
    n_q, n_kv, d, requests = TREES[case]
    rng = np.random.default_rng(200 + case)
    q, k, v, tables, pages, cached, trees = tree_inputs(rng, dtype, requests, n_q, n_kv, d)
    pool = pool_of(k, v, tables, [c + len(t) for c, t in zip(cached, trees)], pages, dtype, behind=np.nan)       # whatever lies behind the nodes must not matter
    want = tree_reference(q, k, v, cached, trees, n_q // n_kv, d ** -0.5, dtype)
    with Device() as dev:
        got, lse, positions, _, _ = run_tree(sts, dev, dtype, q, pool, tables, cached, trees, n_q // n_kv, spare_rows=case % 3)
    check_tree(got, lse, want, cached, trees, positions)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n_q,n_kv,d,cached,nodes", [(8, 2, 64, 320, 5), (8, 2, 64, 320, 21), (4, 1, 128, 300, 1), (8, 1, 128, 640, 30), (4, 2, 64, 90, 25)])
def test_tree_attention_rounds_its_outputs_once(sts, dtype, n_q, n_kv, d, cached, nodes):  # noqa: F811
    """Scores that 32 bits hold exactly (q and k of small whole numbers), so that the bound is narrow: the output's own rounding, and of the sum of |p v|
    2 u (2 u + 2^-9) for the probabilities' two numbers of the type, the first cut off (2 u of p), the second of what is left and of 2^-9 p; 2^-22 and 2^-23 |x - m| for an
    exponential and its argument, in numerator and denominator, and a rounding for each of the sums' tokens; fp16 holds probabilities to 2^-24 of the largest."""
    rng = np.random.default_rng(nodes + d)
    heads, u, trees = n_q // n_kv, HALF[dtype], [random_tree(rng, nodes)]
    k, v, tables, pages = tree_case(rng, [cached], trees, n_kv, d)
    k, v = [rng.integers(-2, 3, x.shape).astype(np.float32) for x in k], [rounded(x, dtype) for x in v]
    q = rng.integers(-2, 3, (nodes, n_q, d)).astype(np.float32)
    pool = pool_of(k, v, tables, [cached + nodes], pages, dtype, behind=np.nan)
    with Device() as dev:
        got, _, _, _, _ = run_tree(sts, dev, dtype, q, pool, tables, [cached], trees, heads, scale=0.0625)
    for r, up in enumerate(ancestors(trees[0])):
        seen = list(range(cached)) + [cached + j for j in up]
        for h in range(n_q):
            x = k[0][seen, h // heads].astype(np.float64) @ q[r, h] / 16
            w, vh = np.exp(x - x.max()), v[0][seen, h // heads].astype(np.float64)
            out, size = w @ vh / w.sum(), w @ np.abs(vh) / w.sum()
            extra = (2 * u * (2 * u + 2.0 ** -9) + 2 * (2.0 ** -22 + 2.0 ** -23 * np.abs(x - x.max()).max()) + 2 * 2.0 ** -24 * len(x)) * size
            near(got[r, h], out, u * np.abs(out) + extra + (2.0 ** -24 * np.abs(vh).sum(0) / w.sum() + 2.0 ** -25 if dtype == "f16" else 0.0))


SMALL = [(40, "tree", 9), (0, "chain", 3), (35, "tree", 40), (16, "star", 5), (33, "forest", 8), (64, "tree", 1)]


def test_tree_attention_rows_that_are_no_nodes(sts):  # noqa: F811
    """Parents of padding (-2, the row itself, a later row, far out): zeros, nobody sees them or what lies in their places, and what hangs below them is none either."""
    rng = np.random.default_rng(3)
    q, k, v, tables, pages, cached, trees = tree_inputs(rng, "bf16", SMALL, 8, 2, 64)
    trees[0][3], trees[0][7], trees[2][1], trees[2][20], trees[3][4], trees[5][0] = -2, 8, 1, 2 ** 31 - 1, 99, -2 ** 31
    trees[1] = [-2, -2, -2]                                                # a request of padding alone, without a context
    for r, tree in enumerate(trees):
        for j, up in enumerate(ancestors(tree)):
            if up is None:
                k[r][cached[r] + j] = v[r][cached[r] + j] = np.nan
    pool = pool_of(k, v, tables, [c + len(t) for c, t in zip(cached, trees)], pages, "bf16", behind=np.inf)
    want = tree_reference(q, k, v, cached, trees, 4, 0.125, "bf16")
    with Device() as dev:
        got, lse, positions, _, _ = run_tree(sts, dev, "bf16", q, pool, tables, cached, trees, 4, spare_rows=5)
    check_tree(got, lse, want, cached, trees, positions)


def test_tree_attention_strides_scale_and_outputs_that_are_not_wanted(sts):  # noqa: F811
    rng = np.random.default_rng(6)
    q, k, v, tables, pages, cached, trees = tree_inputs(rng, "f16", SMALL, 8, 2, 64, scale=3.0)
    pool = pool_of(k, v, tables, [c + len(t) for c, t in zip(cached, trees)], pages, "f16", behind="noise", rng=rng)
    want = tree_reference(q, k, v, cached, trees, 4, 0.3, "f16")
    with Device() as dev:
        for q_pad, out_pad, offset in ((8, 0, 0), (3, 5, 0), (0, 1, 2), (8, 8, 2)):
            got, lse, positions, _, _ = run_tree(sts, dev, "f16", q, pool, tables, cached, trees, 4, scale=0.3, q_pad=q_pad, out_pad=out_pad, q_offset=offset, want_lse=q_pad != 3,
                                                 want_positions=q_pad != 3)
            near(got, want[0], want[1])
            assert (lse == 7.0).all() and (positions == 777).all() if q_pad == 3 else np.isfinite(lse).all() and (positions >= 0).all()


def test_tree_attention_pages_and_lengths_out_of_range_are_nan(sts):  # noqa: F811
    """Only the requests that have them."""
    rng = np.random.default_rng(8)
    q, k, v, tables, pages, cached, trees = tree_inputs(rng, "bf16", SMALL, 8, 2, 64)
    pool = pool_of(k, v, tables, [c + len(t) for c, t in zip(cached, trees)], pages, "bf16")
    want, starts = tree_reference(q, k, v, cached, trees, 4, 0.125, "bf16"), starts_of(trees)

    def check(hit, **change):
        with Device() as dev:
            got, lse, positions, _, _ = run_tree(sts, dev, "bf16", q, pool, **{**dict(tables=tables, cached=cached), **change}, trees=trees, heads=4)
        rows = np.zeros(len(q), bool)
        rows[starts[hit]:starts[hit + 1]] = True
        assert np.isnan(got[rows]).all() and np.isnan(lse[rows]).all()
        near(got[~rows], want[0][~rows], want[1][~rows])
        return positions[rows]
    for where, value in (((0, 2), pages), ((2, 3), -1), ((4, 0), 2 ** 31 - 1)):
        t = tables.copy()
        t[where] = value
        check(where[0], tables=t)
    for bad in (-3, tables.shape[1] * 16 - 8, 2 ** 31 - 1, -2 ** 31):
        c = list(cached)
        c[0] = bad
        assert (check(0, cached=c) == -1).all()


def test_tree_attention_padding_of_a_request_with_a_bad_page_gives_zeros(sts):  # noqa: F811
    """Its nodes NaN, its padding zeros and an lse of -inf as everywhere."""
    rng = np.random.default_rng(14)
    q, k, v, tables, pages, cached, trees = tree_inputs(rng, "bf16", SMALL, 8, 2, 64)
    trees[0][3], trees[2][1], trees[2][20] = -2, 1, 99
    pool = pool_of(k, v, tables, [c + len(t) for c, t in zip(cached, trees)], pages, "bf16")
    want, starts = tree_reference(q, k, v, cached, trees, 4, 0.125, "bf16"), starts_of(trees)
    node = np.array([up is not None for t in trees for up in ancestors(t)])
    for hit, at in ((0, 1), (2, 0), (2, 4)):
        t = tables.copy()
        t[hit, at] = pages
        with Device() as dev:
            got, lse, positions, _, _ = run_tree(sts, dev, "bf16", q, pool, t, cached, trees, 4)
        bad = np.zeros(len(q), bool)
        bad[starts[hit]:starts[hit + 1]] = True
        assert np.isnan(got[bad & node]).all() and np.isnan(lse[bad & node]).all()
        assert (got[~node] == 0.0).all() and np.isneginf(lse[~node]).all() and (positions[~node] == -1).all()
        near(got[~bad & node], want[0][~bad & node], want[1][~bad & node])


def test_tree_attention_of_more_nodes_than_a_request_may_have_is_nan(sts):  # noqa: F811
    rng = np.random.default_rng(9)
    q, k, v, tables, pages, cached, trees = tree_inputs(rng, "bf16", [(20, "chain", 7), (5, "chain", 257), (31, "tree", 12)], 4, 2, 64)
    pool = pool_of(k, v, tables, [c + len(t) for c, t in zip(cached, trees)], pages, "bf16")
    fine = np.r_[0:7, 264:276]
    want = tree_reference(q[fine], [k[0], k[2]], [v[0], v[2]], [20, 31], [trees[0], trees[2]], 2, 0.125, "bf16")
    with Device() as dev:
        got, lse, positions, _, _ = run_tree(sts, dev, "bf16", q, pool, tables, cached, trees, 2)
    near(got[fine], want[0], want[1])
    assert np.isnan(got[7:264]).all() and np.isnan(lse[7:264]).all() and (positions[7:264] == -1).all()


@pytest.mark.parametrize("starts", [[0, 9, 12, 52, 57, 65, 67], [1, 9, 12, 52, 57, 65, 66], [0, 9, 12, 57, 52, 65, 66], [0, -9, 12, 52, 57, 65, 66], [0, 9, 12, 52, 57, 2 ** 31 - 1, 66]])
def test_tree_attention_row_starts_out_of_order_are_nan(sts, starts):  # noqa: F811
    rng = np.random.default_rng(7)
    q, k, v, tables, pages, cached, trees = tree_inputs(rng, "bf16", SMALL, 8, 2, 64)
    pool = pool_of(k, v, tables, [c + len(t) for c, t in zip(cached, trees)], pages, "bf16")
    assert starts_of(trees).tolist() == [0, 9, 12, 52, 57, 65, 66]
    with Device() as dev:
        got, lse, _, _, _ = run_tree(sts, dev, "bf16", q, pool, tables, cached, trees, 4, starts=starts)
    assert np.isnan(got).all() and np.isnan(lse).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("nodes", [6, 40])
def test_tree_attention_infinities_stay_with_those_who_see_them(sts, dtype, nodes):  # noqa: F811
    """A node's K or V of infinities or NaN reaches the rows below it alone; one in the context reaches all."""
    rng = np.random.default_rng(10)
    for cached in (64, 45, 0):
        tree = random_tree(rng, nodes, roots=2)
        tree[2], tree[3], tree[4] = 0, 1, 0
        q, k, v, tables, pages, _, _ = tree_inputs(rng, dtype, [(cached, "chain", nodes)], 8, 2, 64)
        q = widened(stored(np.abs(q) + 0.25, dtype), dtype)                # as it lies in memory
        up = ancestors(tree)
        big = np.finfo(np.float32).max if dtype == "bf16" else 65504.0
        for what in ("v", "nan v", "k", "-k", "context") if cached else ("v", "nan v", "k", "-k"):
            kk, vv = k[0].copy(), v[0].copy()
            if what == "v":
                vv[cached + 3, 0, 7], vv[cached + 4, 1, 60] = np.inf, -np.inf
            if what == "nan v":
                vv[cached + 3, 0, 7] = np.nan
            if what == "k":
                kk[cached + 4, 1, 5] = np.nan
            if what == "-k":
                kk[cached + 4] = -np.inf                                  # scores of -inf: no weight
            if what == "context":
                vv[cached - 1, 0, 3], vv[0, 1, 9] = np.inf, np.nan
            pool = pool_of([kk], [vv], tables, [cached + nodes], pages, dtype, behind=np.nan)
            with Device() as dev:
                got, lse, _, _, _ = run_tree(sts, dev, dtype, q, pool, tables, [cached], [tree], 4)
            with np.errstate(all="ignore"):
                out, bound, want_lse, lb = tree_reference(q, [kk], [vv], [cached], [tree], 4, 0.125, dtype)
            odd = ~np.isfinite(out)
            assert odd.any() == (what != "-k"), what
            near(got[~odd], out[~odd], np.where(np.isfinite(bound), bound, 0.0)[~odd])
            if what in ("v", "context"):
                assert np.array_equal(got[odd], out[odd], equal_nan=True), what
            else:
                assert np.isnan(got[odd]).all(), what
            assert big > 0 and all((3 in u) <= odd[r].any() for r, u in enumerate(up) if what in ("v", "nan v"))


def test_tree_attention_same_bits_again_in_a_graph_and_without_a_plan(sts):  # noqa: F811
    """Nothing depends on the order in which workgroups end: the same inputs give the same bits, eagerly, on another stream and replayed; a workspace without a plan gives NaN."""
    rng = np.random.default_rng(11)
    q, k, v, tables, pages, cached, trees = tree_inputs(rng, "bf16", [(300 + 7 * i, "tree", 1 + (5 * i) % 60) for i in range(40)], 8, 2, 64)
    pool = pool_of(k, v, tables, [c + len(t) for c, t in zip(cached, trees)], pages, "bf16")
    with Device() as dev:
        first, lse0, pos0, _, _ = run_tree(sts, dev, "bf16", q, pool, tables, cached, trees, 4)
        s = dev.stream()
        again, lse1, _, call, (out, lse, positions) = run_tree(sts, dev, "bf16", q, pool, tables, cached, trees, 4, stream=s)
        assert np.array_equal(first, again) and np.array_equal(lse0, lse1)
        replay = dev.graph(s, call)
        for _ in range(4):
            dev.write(out, np.full(again.size, 0x7FC0, np.uint16))
            dev.write(lse, np.full(lse0.size, np.nan, np.float32))
            dev.write(positions, np.zeros(len(pos0), np.int32))
            replay()
            dev.sync()
            assert np.array_equal(dev.get(out, first.shape, "bf16"), first) and np.array_equal(dev.get(lse, lse0.shape, "f32"), lse0) and np.array_equal(dev.get(positions, len(pos0), "i32"), pos0)


def test_tree_attention_without_a_plan_of_its_sizes_is_nan(sts):  # noqa: F811
    """A workspace that holds none, or one of other requests, rows, heads or tables: nothing in it is followed."""
    rng = np.random.default_rng(22)
    n, rows, heads, n_kv, d, pages = 20, 70, 4, 2, 64, 40
    width = heads * n_kv * d
    with Device() as dev:
        size = max(sts.attn_tree_workspace(n, rows, *x) for x in ((heads * n_kv, n_kv, d), (heads, 1, 2 * d), (n_kv, n_kv, d)))
        q, pool = dev.put(rng.standard_normal((rows, width)), "bf16"), dev.put(rng.standard_normal((pages, n_kv, 2 * 16 * d)), "bf16")
        starts = np.concatenate([[0], np.sort(rng.integers(0, 61, n - 1)), [60]]).astype(np.int32)
        fields = dict(tables=dev.ints(rng.integers(0, pages, (n, 6))), cached=dev.ints(rng.integers(10, 30, n)), row_starts=dev.ints(starts), parents=dev.ints([-1] * rows),
                      workspace=dev.put(np.zeros(size, np.uint8)), workspace_bytes=size)

        def batch(**change):
            return sts.TreeBatch(**{**dict(dtype=1, n_requests=n, max_rows=rows, n_q=heads * n_kv, n_kv=n_kv, d=d, pool_pages=pages, max_pages=6, table_stride=6, **fields), **change})

        def layer(b):
            out = dev.put(np.full((rows, width), 7.0), "bf16")
            sts.op_attn_tree(b, q, width, pool, out, width)
            dev.sync()
            got = dev.get(out, (rows, width), "bf16")
            assert (got[b.max_rows:] == 7.0).all() and (got[:, b.n_q * b.d:] == 7.0).all()
            return got[:b.max_rows, :b.n_q * b.d]
        assert np.isnan(layer(batch())).all()
        sts.op_attn_tree_plan(batch())
        assert np.isfinite(layer(batch())).all()
        for change in (dict(n_requests=n - 1), dict(max_rows=rows - 1), dict(n_q=n_kv), dict(n_q=heads, n_kv=1), dict(n_q=heads, n_kv=1, d=2 * d), dict(max_pages=5)):
            assert np.isnan(layer(batch(**change))).all(), change
        assert np.isfinite(layer(batch())[:60]).all() and (layer(batch())[60:] == 7.0).all()


def test_tree_attention_of_the_most_rows_and_many_heads(sts):  # noqa: F811
    """65536 rows of 2048 query heads: 2^27 rows of heads to join, 137 GB of workspace. Few of the rows are there; the others stay as they are."""
    rng = np.random.default_rng(61)
    n_q, n_kv, d, rows = 2048, 256, 128, 65536
    q, k, v, tables, pages, cached, trees = tree_inputs(rng, "bf16", [(35, "tree", 3), (0, "chain", 2), (7, "tree", 5)], n_q, n_kv, d)
    pool = pool_of(k, v, tables, [c + len(t) for c, t in zip(cached, trees)], pages, "bf16")
    want, n, size = tree_reference(q, k, v, cached, trees, n_q // n_kv, d ** -0.5, "bf16"), len(q), sts.attn_tree_workspace(3, rows, n_q, n_kv, d)
    assert size > 1 << 37
    with Device() as dev:
        fields = dict(tables=dev.ints(tables), cached=dev.ints(cached), row_starts=dev.ints(starts_of(trees)), parents=dev.ints([p for t in trees for p in t] + [-1] * (rows - n)),
                      positions=dev.ints([777] * rows), workspace=dev.alloc(size), workspace_bytes=size)
        batch = sts.TreeBatch(dtype=1, n_requests=3, max_rows=rows, n_q=n_q, n_kv=n_kv, d=d, pool_pages=pages, max_pages=tables.shape[1], table_stride=tables.shape[1], **fields)
        dev_q, out, lse = dev.alloc(rows * n_q * d * 2), dev.alloc(rows * n_q * d * 2), dev.alloc(rows * n_q * 4)
        dev.write(dev_q, stored(q.reshape(n, -1), "bf16"))
        for row in (n, rows - 1):
            dev.write(out + row * n_q * d * 2, np.full(n_q * d, 0x7FC0, np.uint16))
        sts.op_attn_tree_plan(batch)
        sts.op_attn_tree(batch, dev_q, n_q * d, dev.put(pool, "bf16"), out, n_q * d, lse)
        dev.sync()
        check_tree(dev.get(out, (n, n_q, d), "bf16"), dev.get(lse, (n, n_q), "f32"), want, cached, trees, dev.get(fields["positions"], rows, "i32")[:n])
        for row in (n, rows - 1):
            assert np.isnan(dev.get(out + row * n_q * d * 2, n_q * d, "bf16")).all()


def test_tree_attention_of_two_streams_at_once(sts):  # noqa: F811
    """Workspaces of their own: calls under way together do not see each other."""
    rng = np.random.default_rng(21)
    cases = [tree_inputs(rng, "bf16", [(600 + 5 * i, "tree", 3 + i) for i in range(30)], 8, 2, 64), tree_inputs(rng, "bf16", [(90 + 11 * i, "chain", 4) for i in range(70)], 8, 2, 64)]
    with Device() as dev:
        runs, want = [], []
        for q, k, v, tables, pages, cached, trees in cases:
            pool, s = pool_of(k, v, tables, [c + len(t) for c, t in zip(cached, trees)], pages, "bf16"), dev.stream()
            out, _, _, call, at = run_tree(sts, dev, "bf16", q, pool, tables, cached, trees, 4, stream=s)
            runs.append((call, at, out.shape))
            want.append(out)
        for _ in range(20):
            for call, _, _ in runs:
                call()
        dev.sync()
        for (_, at, shape), w in zip(runs, want):
            assert np.array_equal(dev.get(at[0], shape, "bf16"), w)


@pytest.mark.parametrize("dtype,n_q,n_kv,requests", [("bf16", 4, 2, 4096), ("f16", 32, 1, 4096)])
def test_tree_attention_of_the_most_requests(sts, dtype, n_q, n_kv, requests):  # noqa: F811
    """4096 requests, most of few rows, some of wide tiles and some without rows; a sample of rows against 64 bits."""
    rng = np.random.default_rng(31)
    shape = [(int(rng.integers(0, 40)), "tree", int(rng.choice([0, 1, 1, 2, 3, 9]))) for _ in range(requests)]
    q, k, v, tables, pages, cached, trees = tree_inputs(rng, dtype, shape, n_q, n_kv, 64)
    pool = pool_of(k, v, tables, [c + len(t) for c, t in zip(cached, trees)], pages, dtype)
    with Device() as dev:
        got, lse, positions, _, _ = run_tree(sts, dev, dtype, q, pool, tables, cached, trees, n_q // n_kv)
    starts = starts_of(trees)
    for r in list(range(0, requests, 97)) + [requests - 1]:
        a, b = starts[r], starts[r + 1]
        if a < b:
            check_tree(got[a:b], lse[a:b], tree_reference(q[a:b], [k[r]], [v[r]], [cached[r]], [trees[r]], n_q // n_kv, 0.125, dtype), [cached[r]], [trees[r]], positions[a:b])
    assert np.isfinite(got).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n_q,n_kv,d,nodes,requests", [(32, 1, 64, 17, 150), (32, 1, 64, 13, 200), (64, 8, 128, 241, 6)])
def test_tree_attention_of_last_tiles_with_few_rows(sts, dtype, n_q, n_kv, d, nodes, requests):  # noqa: F811
    """Trees whose last tile has 8 or 32 rows, in workgroups that have another tile behind it: more tiles than there are workgroups for a head."""
    rng = np.random.default_rng(41)
    q, k, v, tables, pages, cached, trees = tree_inputs(rng, dtype, [(int(rng.integers(0, 90)), "tree", nodes) for _ in range(requests)], n_q, n_kv, d)
    pool = pool_of(k, v, tables, [c + len(t) for c, t in zip(cached, trees)], pages, dtype)
    with Device() as dev:
        got, lse, positions, call, at = run_tree(sts, dev, dtype, q, pool, tables, cached, trees, n_q // n_kv)
        for _ in range(20):
            call()
        dev.sync()
        assert np.array_equal(dev.get(at[0], got.shape, dtype), got)
    for r in range(0, requests, 5):
        a, b = r * nodes, (r + 1) * nodes
        check_tree(got[a:b], lse[a:b], tree_reference(q[a:b], [k[r]], [v[r]], [cached[r]], [trees[r]], n_q // n_kv, d ** -0.5, dtype), [cached[r]], [trees[r]], positions[a:b])
    assert np.isfinite(got).all()


# ------------------------------------------------------------------------------------------ logits
def adjust_reference(x, requests, tokens, lens, prompts, penalties, trees, drafted, biases, masks, mask_rows):
    """x [rows, vocab] float64; biases: by request a list of (token, value)."""
    y, (rows, vocab) = x.copy(), x.shape
    n_requests = len(lens) if lens is not None else len(biases) if biases is not None else 0
    paths = [up for t in trees for up in ancestors(t)] if trees is not None else None
    starts = starts_of(trees) if trees is not None else None
    for r in range(rows):
        i = requests[r]
        if 0 <= i < n_requests:
            n, said = np.zeros(vocab, np.int64), np.zeros(vocab, bool)
            if tokens is not None:
                t = tokens[i, :max(0, min(lens[i], tokens.shape[1]))]
                ok = (t >= 0) & (t < vocab)
                out = np.arange(len(t)) >= prompts[i]
                np.add.at(n, t[ok & out], 1)
                said[t[ok]] = True
            if trees is not None and starts[i] <= r < starts[i + 1]:
                t = drafted[[starts[i] + j for j in paths[r]]]
                t = t[(t >= 0) & (t < vocab)]
                np.add.at(n, t, 1)
                said[t] = True
            rep, freq, pres = (np.float64(p[i]) for p in penalties)
            at = np.flatnonzero(said)
            with np.errstate(all="ignore"):
                z = np.where(x[r, at] > 0, x[r, at] / rep, x[r, at] * rep)
            y[r, at] = np.where(n[at] > 0, z - (freq * n[at] + pres), z)
            for t, b in dict(biases[i]).items() if biases is not None else ():
                if 0 <= t < vocab:
                    y[r, t] += np.float64(b)
        if masks is not None and 0 <= mask_rows[r] < len(masks):
            y[r, ~masks[mask_rows[r], :vocab]] = -np.inf
    return y


def words_of(masks):
    """[n, 32 w] bools as 32-bit words."""
    return (masks.reshape(len(masks), -1, 32).astype(np.uint64) << np.arange(32, dtype=np.uint64)).sum(2).astype(np.uint32).view(np.int32)


def adjust_case(rng, dtype, vocab, trees, history, n_biases, grammar):
    n, rows = len(trees), sum(map(len, trees))
    x = rounded(3.0 * rng.standard_normal((rows, vocab)), dtype)
    requests = np.repeat(np.arange(n), [len(t) for t in trees]).astype(np.int32)
    tokens = (vocab * rng.random((n, max(history, 1))) ** 3).astype(np.int32)
    lens = rng.integers(0, history + 1, n).astype(np.int32)
    prompts = np.array([rng.integers(0, m + 1) for m in lens], np.int32)
    penalties = [(1.0 + rng.random(n)).astype(np.float32), (0.4 * rng.random(n)).astype(np.float32), rng.random(n).astype(np.float32)]
    drafted = (vocab * rng.random(rows) ** 3).astype(np.int32)
    biases = [[(int(rng.integers(0, vocab)), float(np.float32(5 * rng.standard_normal()))) for _ in range(rng.integers(0, n_biases + 1))] for _ in range(n)]
    width = -(-vocab // 32) * 32 + 64
    masks = rng.random((3, width)) < np.array([0.5, 0.01, 0.999])[:, None]
    mask_rows = np.where(rng.random(rows) < grammar, rng.integers(0, 3, rows), -1).astype(np.int32)
    return dict(x=x, requests=requests, tokens=tokens, lens=lens, prompts=prompts, penalties=penalties, trees=trees, drafted=drafted, biases=biases, masks=masks, mask_rows=mask_rows)


def adjust_description(sts, dev, dtype, c, in_place=False, pad=0, offset=0, stream=None):
    """The description, and where its output is."""
    rows, vocab = c["x"].shape
    x = np.full((rows, vocab + pad), 11.0, np.float32)
    x[:, :vocab] = c["x"]
    logits = dev.put(x, dtype, offset)
    out = logits if in_place else dev.put(np.full((rows, vocab + pad), 7.0, np.float32), dtype, offset)
    p = c["penalties"]
    a = dict(dtype=sts.DTYPES[dtype], rows=rows, vocab=vocab, row_stride=vocab + pad, out_stride=vocab + pad, logits=logits, out=out, requests=dev.ints(c["requests"]))
    if c["lens"] is not None or c["biases"] is not None:
        a.update(n_requests=len(c["lens"] if c["lens"] is not None else c["biases"]))
    if c["tokens"] is not None:
        a.update(tokens=dev.ints(c["tokens"]), token_stride=c["tokens"].shape[1], lens=dev.ints(c["lens"]), prompt_lens=dev.ints(c["prompts"]), repetition=dev.put(p[0]), frequency=dev.put(p[1]),
                 presence=dev.put(p[2]))
    if c["trees"] is not None:
        a.update(row_starts=dev.ints(starts_of(c["trees"])), parents=dev.ints([q for t in c["trees"] for q in t]), drafted=dev.ints(c["drafted"]))
    if c["biases"] is not None:
        flat = [e for b in c["biases"] for e in b]
        a.update(bias_starts=dev.ints(starts_of(c["biases"])), bias_tokens=dev.ints([t for t, _ in flat]), bias_values=dev.put(np.array([b for _, b in flat], np.float32)), n_biases=len(flat))
    if c["masks"] is not None:
        w = words_of(c["masks"])
        a.update(masks=dev.ints(w), n_masks=len(w), mask_stride=w.shape[1], mask_rows=dev.ints(c["mask_rows"]))
    return sts.AdjustLogits(**a), out


def check_adjusted(got, c, dtype):
    """In 64 bits, rounded to 32 and then to the type: a step of 32 bits beside half a step of the type. What nothing applies to keeps its value."""
    x = c["x"].astype(np.float64)
    want = adjust_reference(x, c["requests"], c["tokens"], c["lens"], c["prompts"], c["penalties"], c["trees"], c["drafted"], c["biases"], c["masks"], c["mask_rows"])
    same = (want == x) | ~np.isfinite(want)
    assert np.array_equal(got[same], want[same], equal_nan=True)
    bound = np.abs(want[~same]) * (HALF[dtype] + 2.0 ** -24) + (2.0 ** -25 if dtype == "f16" else 1e-38)
    near(got[~same], want[~same], bound)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab,sizes,history,n_biases,grammar,pad,offset", [
    (1, [1], 3, 1, 0.0, 0, 0), (5, [1, 1], 0, 2, 0.5, 0, 0), (1000, [1], 50, 0, 0.0, 0, 0), (1003, [3, 1, 9], 700, 20, 0.5, 0, 0), (4096, [26], 300, 5, 0.2, 8, 0), (8192, [1, 5], 40, 300, 1.0, 0, 0),
    (8193, [4, 4, 4], 5000, 3, 0.4, 0, 0), (32001, [8, 3], 1000, 10, 0.3, 7, 0), (40000, [64], 100, 2, 0.3, 0, 4), (128256, [1], 2000, 20, 0.0, 0, 0), (128256, [5, 5, 5], 300, 8, 0.5, 0, 0),
    (50000, [256, 2], 20, 1, 0.1, 0, 0)])
def test_adjust_logits(sts, dtype, vocab, sizes, history, n_biases, grammar, pad, offset):  # noqa: F811
    rng = np.random.default_rng(vocab + len(sizes))
    c = adjust_case(rng, dtype, vocab, [random_tree(rng, m) for m in sizes], history, n_biases, grammar)
    with Device() as dev:
        for in_place in (False, True):
            a, out = adjust_description(sts, dev, dtype, c, in_place, pad, offset)
            sts.op_adjust_logits(a)
            dev.sync()
            got = dev.get(out, (len(c["x"]), vocab + pad), dtype)
            assert (got[:, vocab:] == (11.0 if in_place else 7.0)).all()
            check_adjusted(got[:, :vocab], c, dtype)


@pytest.mark.parametrize("leave", ["tokens", "trees", "biases", "masks", "tokens trees", "tokens trees biases", "biases masks", "tokens trees biases masks"])
def test_adjust_logits_of_parts(sts, leave):  # noqa: F811
    """Any of history, drafts, biases and masks may be missing."""
    rng = np.random.default_rng(len(leave))
    c = adjust_case(rng, "bf16", 9000, [random_tree(rng, m) for m in (4, 1, 6)], 200, 6, 0.5)
    for what in leave.split():
        c[what] = None
    if c["tokens"] is None:
        c["penalties"] = [np.ones(3, np.float32), np.zeros(3, np.float32), np.zeros(3, np.float32)]
    with Device() as dev:
        for in_place in (False, True):
            a, out = adjust_description(sts, dev, "bf16", c, in_place)
            sts.op_adjust_logits(a)
            dev.sync()
            check_adjusted(dev.get(out, c["x"].shape, "bf16"), c, "bf16")


def test_adjust_logits_without_requests_or_prompts(sts):  # noqa: F811
    """Row i is request i, and all of the history is output."""
    rng = np.random.default_rng(4)
    c = adjust_case(rng, "f32", 5000, [[-1]] * 6, 300, 0, 0.0)
    c.update(trees=None, biases=None, masks=None, prompts=np.zeros(6, np.int32))
    with Device() as dev:
        a, out = adjust_description(sts, dev, "f32", c)
        a.requests = a.prompt_lens = None
        sts.op_adjust_logits(a)
        dev.sync()
        check_adjusted(dev.get(out, c["x"].shape, "f32"), c, "f32")


def test_adjust_logits_paths_of_rows_that_are_no_nodes(sts):  # noqa: F811
    """Such a row's path ends where a parent is no earlier row."""
    rng = np.random.default_rng(15)
    c = adjust_case(rng, "f32", 3000, [random_tree(rng, 9), random_tree(rng, 4)], 30, 2, 0.3)
    odd = {2: -2, 4: 4, 5: 2, 6: 2 ** 31 - 1, 8: 6}
    first = list(c["trees"][0])
    c["trees"][0] = [-1 if odd.get(j, p) < -1 or odd.get(j, p) >= j else odd.get(j, p) for j, p in enumerate(first)]
    with Device() as dev:
        for in_place in (False, True):
            a, out = adjust_description(sts, dev, "f32", c, in_place)
            a.parents = dev.ints([odd.get(j, p) for j, p in enumerate(first)] + c["trees"][1])
            sts.op_adjust_logits(a)
            dev.sync()
            check_adjusted(dev.get(out, c["x"].shape, "f32"), c, "f32")


def test_adjust_logits_of_odd_values_and_numbers(sts):  # noqa: F811
    """Infinities and NaN go by the formula; tokens, requests, masks and lengths out of range count for nothing; a token twice among the biases has the last one; a bias of
    -inf bans; a mask that leaves nothing leaves -inf."""
    rng = np.random.default_rng(5)
    vocab = 9001
    c = adjust_case(rng, "f32", vocab, [random_tree(rng, m) for m in (3, 1, 2, 4)], 60, 0, 0.0)
    x = c["x"]
    x[:, 7], x[:, 8], x[:, 9], x[:, 10] = np.inf, -np.inf, np.nan, -0.0
    c["tokens"][:, :6] = [7, 8, 9, 10, -1, vocab]
    c["tokens"][:, 6:9] = [-2 ** 31, 2 ** 31 - 1, vocab - 1]
    c["lens"][:] = [60, 5, 1 << 30, -4]
    c["prompts"][:] = [3, 1 << 30, -7, 0]
    c["drafted"][:3] = [-5, vocab, 8]
    c["requests"] = c["requests"].copy()
    c["requests"][4], c["requests"][5] = -1, 4                            # the third request's rows belong to none
    c["biases"] = [[(20, 1.5), (20, -2.5), (21, -np.inf), (-3, 4.0), (vocab, 4.0), (8, 1.0)], [], [], [(vocab - 1, np.inf), (0, np.nan)]]
    c["mask_rows"][:] = [-1, 0, 1, 2, 3, -9, 2, 2 ** 31 - 1, -1, 1]
    c["masks"][1] = False
    with Device() as dev:
        for in_place in (False, True):
            a, out = adjust_description(sts, dev, "f32", c, in_place)
            sts.op_adjust_logits(a)
            dev.sync()
            got = dev.get(out, x.shape, "f32")
            with np.errstate(all="ignore"):
                check_adjusted(got, c, "f32")
            assert np.isneginf(got[2]).all() and np.isneginf(got[9]).all()


@pytest.mark.parametrize("starts", [[0, 2 ** 31 - 1, 3, 6], [2 ** 31 - 300, 2 ** 31 - 1, 2, 6], [-2 ** 31, 2, 2 ** 31 - 511, 2 ** 31 - 1], [6, 2, 5, 1], [-5, -1, 4, 2000], [2 ** 31 - 1, 2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1],
                                    [7, 4001, 4002, 4003]])
def test_adjust_logits_bias_starts_out_of_range(sts, starts):  # noqa: F811
    """Of a request's entries, bias_starts[i] to bias_starts[i + 1], those that the list has count, whatever the numbers; the list may be longer than a workgroup."""
    rng = np.random.default_rng(51)
    c = adjust_case(rng, "f32", 5000, [random_tree(rng, m) for m in (2, 3, 1)], 20, 0, 0.0)
    for n in (6, 3000):
        flat = list(zip(rng.integers(0, 5000, n).tolist(), np.float32(5 * rng.standard_normal(n)).tolist()))
        c["biases"] = [flat[max(a, 0):max(b, 0)] for a, b in zip(starts, starts[1:])]
        with Device() as dev:
            for in_place in (False, True):
                a, out = adjust_description(sts, dev, "f32", c, in_place)
                a.bias_starts, a.bias_tokens, a.bias_values, a.n_biases = dev.ints(starts), dev.ints([t for t, _ in flat]), dev.put(np.array([b for _, b in flat], np.float32)), n
                sts.op_adjust_logits(a)
                dev.sync()
                check_adjusted(dev.get(out, c["x"].shape, "f32"), c, "f32")


def to_type(y, dtype):
    """y (float64) in the type, as float64: one rounding, to the nearest, ties to even."""
    bits, least, most = (8, -133, float(np.uint32(0x7F7F0000).view(np.float32))) if dtype == "bf16" else (11, -24, 65504.0)
    step = np.exp2(np.maximum(np.frexp(y)[1] - bits, least).astype(np.float64))
    z = np.rint(y / step) * step
    return np.where(np.abs(z) > most, np.copysign(np.inf, y), z)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_adjust_logits_rounds_once(sts, dtype):  # noqa: F811
    """Sums that lie 2^-20 of half a step of the type beside the middle between two of its numbers, where 32 bits would round them onto the middle, at both ends of the type's range and in
    between: they are exact in 64 bits, so the outputs are known to the bit."""
    bits, least = (8, -126) if dtype == "bf16" else (11, -14)
    top = 127 if dtype == "bf16" else 15
    x, b = [], []
    for e in (least, -3, 0, 1, 6, top - 1, top):
        for m in list(range(2 ** (bits - 1), 2 ** (bits - 1) + 6)) + [2 ** bits - 3, 2 ** bits - 2, 2 ** bits - 1]:
            for side in (-1, 0, 1):
                for sign in (-1.0, 1.0):
                    x.append(sign * np.ldexp(float(m), e + 1 - bits))
                    b.append(sign * np.ldexp(1.0 + side * 2.0 ** -20, e - bits))
    for m in (0, 1, 2, 3, 7):                                               # numbers below the smallest with all its digits
        for side in (-1, 0, 1):
            x.append(np.ldexp(float(m), least + 1 - bits))
            b.append(np.ldexp(1.0 + side * 2.0 ** -20, least - bits))
    x, b = np.array(x), np.array(b)
    b32 = b.astype(np.float32)
    vocab = len(x)
    assert np.array_equal(rounded(x, dtype), x)
    y = x + b32.astype(np.float64)
    want = to_type(y, dtype)
    with np.errstate(over="ignore"):
        twice = rounded(y.astype(np.float32), dtype)
    assert (twice != want).sum() > 20
    with Device() as dev:
        for in_place in (False, True):
            logits = dev.put(x[None], dtype)
            out = logits if in_place else dev.alloc(2 * vocab)
            sts.op_adjust_logits(sts.AdjustLogits(dtype=sts.DTYPES[dtype], rows=1, vocab=vocab, n_requests=1, row_stride=vocab, out_stride=vocab, logits=logits, out=out, n_biases=vocab,
                                                  bias_starts=dev.ints([0, vocab]), bias_tokens=dev.ints(np.arange(vocab)), bias_values=dev.put(b32)))
            dev.sync()
            got = dev.get(out, vocab, dtype).astype(np.float64)
            bad = got != want
            assert not bad.any(), (bad.sum(), x[bad][:5], b[bad][:5], got[bad][:5], want[bad][:5])


@pytest.mark.parametrize("stride", [2 ** 31, 2 ** 31 - 1])
def test_adjust_logits_of_the_longest_history(sts, stride):  # noqa: F811
    """2^31 - 1 tokens, of which the first and last few are of the vocabulary: the last loads in vectors and one by one, with an index beside 2^31."""
    n, vocab = 2 ** 31 - 1, 6
    x = rounded(np.arange(1.0, 7.0)[None], "f32")
    ends = np.full(600, -1, np.int32)
    ends[:3] = [0, 1, 1]                                                   # of the prompt, but for the last of them
    ends[-2:] = [3, 4]
    with Device() as dev:
        tokens = dev.alloc(4 * stride)
        dev.ck(dev.rt.hipMemset(C.c_void_p(tokens), 0xFF, C.c_size_t(4 * stride)), "hipMemset")
        dev.write(tokens, ends[:300])
        dev.write(tokens + 4 * (n - 300), ends[300:])
        logits, out = dev.put(x, "f32"), dev.put(np.zeros((1, vocab), np.float32))
        sts.op_adjust_logits(sts.AdjustLogits(dtype=0, rows=1, vocab=vocab, n_requests=1, row_stride=vocab, out_stride=vocab, logits=logits, out=out, tokens=tokens, token_stride=stride, lens=dev.ints([n]),
                                              prompt_lens=dev.ints([2]), repetition=dev.put(np.float32([2.0])), frequency=dev.put(np.float32([0.25])), presence=dev.put(np.float32([0.5]))))
        dev.sync()
        got = dev.get(out, vocab, "f32")
    assert got.tolist() == [0.5, 1.0 - 0.75, 3.0, 2.0 - 0.75, 2.5 - 0.75, 6.0]


def test_adjust_logits_same_bits_again_and_in_a_graph(sts):  # noqa: F811
    rng = np.random.default_rng(6)
    c = adjust_case(rng, "bf16", 33000, [random_tree(rng, m) for m in (8, 30, 1)], 900, 9, 0.3)
    with Device() as dev:
        s = dev.stream()
        a, out = adjust_description(sts, dev, "bf16", c)
        sts.op_adjust_logits(a)
        dev.sync()
        first = dev.get(out, c["x"].shape, "bf16")
        check_adjusted(first, c, "bf16")
        replay = dev.graph(s, lambda: sts.op_adjust_logits(a, s))
        for _ in range(4):
            dev.write(out, np.full(first.size, 0x7FC0, np.uint16))
            replay()
            dev.sync()
            assert np.array_equal(dev.get(out, first.shape, "bf16"), first)


# ------------------------------------------------------------------------------------------ the accepted path
def accept_reference(tree, tokens, chosen):
    if not tree or tree[0] != -1 or len(tree) > 256:
        return [], -1
    path = [0]
    while True:
        fit = [j for j, p in enumerate(tree) if p == path[-1] and j > path[-1] and tokens[j] == chosen[path[-1]]]
        if not fit:
            return path, chosen[path[-1]]
        path.append(fit[0])


def run_accept(sts, dev, cached, trees, tokens, chosen, spare=0, starts=None, stream=None):
    n, rows = len(cached), sum(map(len, trees)) + spare
    flat = lambda lists: dev.ints([x for y in lists for x in y] + [0] * (spare + (rows == 0)))  # noqa: E731
    d = dict(cached=dev.ints(cached), row_starts=dev.ints(starts_of(trees) if starts is None else starts), parents=flat(trees), tokens=flat(tokens), chosen=flat(chosen), lens=dev.ints([777] * n),
             counts=dev.ints([777] * n), path=dev.ints([777] * max(rows, 1)), next_token=dev.ints([777] * n))
    a = sts.TreeAccept(n_requests=n, max_rows=rows, **d)
    sts.op_tree_accept(a, stream)
    dev.sync()
    return {k: dev.get(d[k], rows if k == "path" else n, "i32").tolist() for k in ("lens", "counts", "path", "next_token")}, d, a


@pytest.mark.parametrize("sizes", [[1], [0], [0, 5, 0], [26], [64, 65, 63, 1, 2], [256, 255, 129], list(range(1, 90)), [4] * 4096])
@pytest.mark.parametrize("agree", [0.0, 0.6, 1.0])
def test_tree_accept(sts, sizes, agree):  # noqa: F811
    """Trees in which several children may bear the same token, targets that agree in part, always, or never."""
    rng = np.random.default_rng(sum(sizes) + int(10 * agree))
    trees = [(chain if i % 4 == 1 else lambda m: random_tree(rng, m, 1 + (i % 4 == 2)))(m) if m else [] for i, m in enumerate(sizes)]
    tokens = [rng.integers(0, 6, m).tolist() for m in sizes]
    chosen = []
    for tree, tok in zip(trees, tokens):
        kids = {p: [tok[j] for j in range(len(tree)) if tree[j] == p] for p in range(len(tree))}
        chosen.append([int(rng.choice(kids[j])) if kids[j] and rng.random() < agree else 100 + j for j in range(len(tree))])
    cached = rng.integers(0, 10 ** 6, len(sizes)).tolist()
    with Device() as dev:
        got, _, _ = run_accept(sts, dev, cached, trees, tokens, chosen, spare=3)
    want = [accept_reference(*x) for x in zip(trees, tokens, chosen)]
    assert got["counts"] == [len(p) for p, _ in want] and got["next_token"] == [t for _, t in want]
    assert got["lens"] == [c + len(p) for c, (p, _) in zip(cached, want)]
    assert got["path"] == [x for t, (p, _) in zip(trees, want) for x in p + [-1] * (len(t) - len(p))] + [777] * 3


def test_tree_accept_of_rows_that_are_no_nodes(sts):  # noqa: F811
    """Padding and requests out of range accept nothing; a node that names itself or a later one as its parent is nobody's child."""
    trees = [[-2, 0, 0], [-1, 1, 2, 0], [-1] + [0] * 299, [-1, 0, -2, 2], [0, 0]]
    tokens = [[5] * len(t) for t in trees]
    chosen = [[5] * len(t) for t in trees]
    with Device() as dev:
        got, _, _ = run_accept(sts, dev, [10, 20, 30, 40, 50], trees, tokens, chosen)
        assert got["counts"] == [0, 2, 0, 2, 0] and got["next_token"] == [-1, 5, -1, 5, -1] and got["lens"] == [10, 22, 30, 42, 50]
        assert got["path"][:7] == [-1, -1, -1, 0, 3, -1, -1] and got["path"][7:307] == [-1] * 300 and got["path"][307:] == [0, 1, -1, -1, -1, -1]
        # row_starts out of range: those requests accept nothing and leave the path's rows as they were
        got, _, _ = run_accept(sts, dev, [1, 2, 3], [[-1], [-1], [-1]], [[5]] * 3, [[6]] * 3, starts=[0, 1, 4, 2])
        assert got["counts"] == [1, 0, 0] and got["path"] == [0, 777, 777]


@pytest.mark.parametrize("sizes", [[40], [40, 0, 1, 200, 16, 256], [3] * 700])
def test_tree_accept_gives_pages_back(sts, sizes):  # noqa: F811
    """The pages behind the paths, in the requests' order; where they do not fit, or the number of free ones is out of range, none."""
    rng = np.random.default_rng(len(sizes))
    trees, n = [random_tree(rng, m) for m in sizes], len(sizes)
    tokens = [rng.integers(0, 3, m).tolist() for m in sizes]
    chosen = [rng.integers(0, 3, m).tolist() for m in sizes]
    cached = rng.integers(0, 100, n).tolist()
    width = max(-(-(c + m) // 16) for c, m in zip(cached, sizes))
    tables = np.arange(n * width, dtype=np.int32).reshape(n, width) + 1000
    counts = [len(accept_reference(*x)[0]) for x in zip(trees, tokens, chosen)]
    back = [int(p) for c, m, k, row in zip(cached, sizes, counts, tables) for p in row[-(-(c + k) // 16):-(-(c + m) // 16)]]
    assert back
    old = list(range(5))
    for free, capacity, given in ((5, 5 + len(back), back), (0, 900 + len(back), back), (5, 4 + len(back), []), (-1, 900 + len(back), []), (901, 900, [])):
        with Device() as dev:
            _, d, a = run_accept(sts, dev, cached, trees, tokens, chosen)
            stack, number = dev.ints(old[:max(free, 0)] + [-7] * (capacity - min(max(free, 0), 5))), dev.ints([free])
            a.max_pages, a.table_stride, a.tables, a.free_pages, a.free_capacity, a.n_free = width, width, dev.ints(tables), stack, capacity, number
            sts.op_tree_accept(a)
            dev.sync()
            got = dev.get(stack, capacity, "i32").tolist()
            assert dev.get(number, 1, "i32")[0] == free + len(given)
            if given:
                assert got == old[:free] + back + [-7] * (capacity - free - len(back))
            else:
                assert back[0] not in got
            assert dev.get(d["counts"], n, "i32").tolist() == counts


def test_tree_accept_takes_lengths_in_place(sts):  # noqa: F811
    """lens = cached: the pages behind the paths are those of the lengths before."""
    rng = np.random.default_rng(12)
    sizes = [18, 40, 0, 1, 200, 16, 256, 300] + [3] * 100
    cached = [30] + rng.integers(0, 100, len(sizes) - 1).tolist()
    trees, n = [chain(m) for m in sizes], len(sizes)
    tokens = [list(range(m)) for m in sizes]
    chosen = [[j + 1 if j < m // 6 else -9 for j in range(m)] for m in sizes]        # the first request's path has four nodes
    width = max(-(-(c + m) // 16) for c, m in zip(cached, sizes))
    tables = np.arange(n * width, dtype=np.int32).reshape(n, width) + 1000
    counts = [len(accept_reference(*x)[0]) for x in zip(trees, tokens, chosen)]
    back = [int(p) for c, m, k, row in zip(cached, sizes, counts, tables) for p in row[-(-(c + k) // 16):-(-(c + m) // 16)]]
    with Device() as dev:
        for in_place in (False, True):
            _, d, a = run_accept(sts, dev, cached, trees, tokens, chosen)
            stack, number = dev.ints([-7] * (len(back) + 9)), dev.ints([0])
            a.max_pages, a.table_stride, a.tables, a.free_pages, a.free_capacity, a.n_free = width, width, dev.ints(tables), stack, len(back) + 9, number
            if in_place:
                a.lens = d["cached"]
            sts.op_tree_accept(a)
            dev.sync()
            assert dev.get(a.lens, n, "i32").tolist() == [c + k for c, k in zip(cached, counts)] and dev.get(d["counts"], n, "i32").tolist() == counts
            assert dev.get(number, 1, "i32")[0] == len(back) and dev.get(stack, len(back) + 9, "i32").tolist() == back + [-7] * 9


def test_tree_accept_of_rows_in_many_requests(sts):  # noqa: F811
    """row_starts up and down between 0 and 2^24: 2^31 pages seem to lie behind the paths, and none is given back."""
    n, rows, width = 4096, 1 << 24, 1 << 20
    with Device() as dev:
        stack, number, counts, lens = dev.ints([-7] * 100), dev.ints([5]), dev.ints([777] * n), dev.ints([777] * n)
        sts.op_tree_accept(sts.TreeAccept(n_requests=n, max_rows=rows, cached=dev.ints([0] * n), row_starts=dev.ints([0, rows] * (n // 2) + [0]), parents=dev.alloc(4 * rows), tokens=dev.alloc(4 * rows),
                                          chosen=dev.alloc(4 * rows), lens=lens, counts=counts, path=dev.alloc(4 * rows), next_token=dev.alloc(4 * n), max_pages=width, free_capacity=50,
                                          table_stride=width, tables=dev.alloc(4 * n * width), free_pages=stack + 100, n_free=number))
        dev.sync()
        assert dev.get(stack, 100, "i32").tolist() == [-7] * 100 and dev.get(number, 1, "i32")[0] == 5
        assert dev.get(counts, n, "i32").tolist() == [0] * n and dev.get(lens, n, "i32").tolist() == [0] * n


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n_kv,d,sizes,layers", [(8, 128, [26], 3), (2, 64, [5, 1, 0, 64, 40], 2), (4, 64, [256, 200], 1), (1, 128, [9] * 70, 2), (3, 64, [30] * 5, 4)])
def test_tree_compact(sts, dtype, n_kv, d, sizes, layers):  # noqa: F811
    """Any ascending paths, those that read where an earlier row of theirs was put among them; every other byte of the pools stays as it was."""
    rng = np.random.default_rng(sum(sizes) + d)
    cached = [int(rng.integers(0, 70)) for _ in sizes]
    trees = [chain(m) for m in sizes]
    _, _, tables, pages = tree_case(rng, cached, trees, 1, 1)
    paths = [sorted(rng.choice(np.arange(1, m), rng.integers(0, m), replace=False).tolist()) if m > 1 else [] for m in sizes]
    paths = [[0] + p if m else [] for p, m in zip(paths, sizes)]
    old = [rounded(rng.standard_normal((pages, n_kv, 32 * d)), dtype) for _ in range(layers)]
    flat = [x for p, m in zip(paths, sizes) for x in p + [-1] * (m - len(p))]
    with Device() as dev:
        pools = [dev.put(x, dtype) for x in old]
        a = sts.TreeCompact(n_requests=len(sizes), max_rows=sum(sizes), n_kv=n_kv, d=d, pool_pages=pages, max_pages=tables.shape[1], table_stride=tables.shape[1], tables=dev.ints(tables),
                            cached=dev.ints(cached), row_starts=dev.ints(starts_of(trees)), counts=dev.ints([len(p) for p in paths]), path=dev.ints(flat))
        sts.op_tree_compact(a, pools)
        dev.sync()
        got = [dev.get(p, old[0].shape, dtype) for p in pools]
    for new, before in zip(got, old):
        kp, vp = before[:, :, :16 * d].reshape(pages, n_kv, 16, d), before[:, :, 16 * d:].reshape(pages, n_kv, d, 16)
        k, v = kp.copy(), vp.copy()
        for r, (c, path) in enumerate(zip(cached, paths)):
            for j, node in enumerate(path):
                s, t = c + node, c + j
                k[tables[r, t // 16], :, t % 16], v[tables[r, t // 16], :, :, t % 16] = kp[tables[r, s // 16], :, s % 16], vp[tables[r, s // 16], :, :, s % 16]
        assert np.array_equal(new[:, :, :16 * d], k.reshape(pages, n_kv, -1)) and np.array_equal(new[:, :, 16 * d:], v.reshape(pages, n_kv, -1))


def test_tree_compact_moves_nothing_out_of_range(sts):  # noqa: F811
    """Pages outside the pool, places behind the table, counts and nodes out of range, negative lengths: those rows stay."""
    rng = np.random.default_rng(2)
    pages, n_kv, d = 12, 2, 64
    old = rounded(rng.standard_normal((pages, n_kv, 32 * d)), "bf16")
    good = dict(cached=[14, 20], tables=[[0, 1, 2], [3, 4, 5]], starts=[0, 8, 16], counts=[2, 3], path=[0, 5] + [-1] * 6 + [0, 4, 7] + [-1] * 5)
    moved = {}
    for name, change in (("none", {}), ("page of the source", dict(tables=[[0, pages, 2], [3, 4, 5]])), ("page of the target", dict(tables=[[-1, 1, 2], [3, 4, 5]])),
                         ("behind the table", dict(cached=[46, 20])), ("negative", dict(cached=[-1, 20])), ("node", dict(path=[0, 8] + [-1] * 6 + [0, 4, 7] + [-1] * 5)),
                         ("far", dict(cached=[2 ** 31 - 1, 20])), ("negative node", dict(path=[0, -7] + [-1] * 6 + [0, 4, 7] + [-1] * 5)), ("starts", dict(starts=[-1, 8, 16])), ("count", dict(counts=[-5, 3])),
                         ("starts behind", dict(starts=[0, 8, 17], counts=[2, 3]))):
        x = {**good, **change}
        with Device() as dev:
            pool = dev.put(old, "bf16")
            sts.op_tree_compact(sts.TreeCompact(n_requests=2, max_rows=16, n_kv=n_kv, d=d, pool_pages=pages, max_pages=3, table_stride=3, tables=dev.ints(x["tables"]), cached=dev.ints(x["cached"]),
                                                row_starts=dev.ints(x["starts"]), counts=dev.ints(x["counts"]), path=dev.ints(x["path"])), [pool])
            dev.sync()
            moved[name] = np.unique(np.argwhere(dev.get(pool, old.shape, "bf16") != old)[:, 0]).tolist()
    assert moved.pop("none") == [0, 4] and moved.pop("starts behind") == [0]
    assert all(m == [4] for m in moved.values()), moved


# ------------------------------------------------------------------------------------------ all together
def test_steps_that_verify_drafts_eager_and_replayed(sts):  # noqa: F811
    """Four requests whose trees of drafted tokens are verified step by step -- pages and places, positions, head norms with rotation and append, attention, logits (the library's GEMM),
    penalties, biases and a mask, the target's choice, the accepted path with its pages, the cache rows -- eagerly and as a graph of two steps that hand lengths, tables, free
    pages and the cache to each other on the device. Everything is checked behind every step against 64 bits and against a host's model of the cache."""
    rng = np.random.default_rng(88)
    n_q, n_kv, d, vocab, dtype, layers = 8, 2, 64, 256, "bf16", 2
    heads, ld, width, pages, eps = n_q // n_kv, (n_q + 2 * n_kv) * d, 14, 80, 1e-6
    trees = [random_tree(rng, 7), chain(4), [-1, 0, 0, 1, 1, -2, 2], star(5)]
    n, rows, starts = len(trees), sum(map(len, trees)), starts_of(trees)
    rope = rope_of(sts, "bands", d, 0)
    gains = gains_of(rng, d, dtype, 0)
    w = rounded(rng.standard_normal((vocab, n_q * d)) / 8, dtype)
    history = rng.integers(0, vocab, (n, 32)).astype(np.int32)
    held, prompts = np.array([32, 7, 0, 20], np.int32), np.array([10, 7, 0, 0], np.int32)
    penalties = [np.float32([1.2, 1.0, 1.5, 2.0]), np.float32([0.1, 0.0, 0.3, 0.2]), np.float32([0.5, 0.2, 0.0, 0.1])]
    biases = [[(t, 30.0 + t) for t in range(3)] + [(200, -5.0)]] * n           # some few tokens are likely: drafts are right now and then
    masks, mask_rows = rng.random((1, vocab)) < 0.9, np.where(np.arange(rows) % 5 == 1, 0, -1).astype(np.int32)
    masks[0, :3] = True
    with Device() as dev:
        s = dev.stream()
        free = rng.permutation(pages).astype(np.int32)
        free_dev, count = dev.put(free), [dev.ints([pages]), dev.ints([0])]
        lens, tables = [dev.ints([0] * n), dev.ints([0] * n)], dev.ints(np.full((n, width), -1))
        pools = [dev.put(np.zeros((pages, n_kv, 32 * d), np.uint16)) for _ in range(layers)]
        counts_of_rows, parents = dev.ints([len(t) for t in trees]), dev.ints([p for t in trees for p in t])
        norm = sts.HeadNorm(dtype=1, eps=eps, q_gain=dev.put(gains[0], dtype), k_gain=dev.put(gains[1], dtype))
        size = sts.attn_tree_workspace(n, rows, n_q, n_kv, d)
        ws, w_dev, lp_ws = dev.alloc(size), dev.put(w, dtype), dev.alloc(max(sts.op_logprobs_workspace(0, rows, vocab, 1), 16))
        flat = [e for b in biases for e in b]
        fixed = dict(tokens=dev.ints(history), token_stride=32, lens=dev.ints(held), prompt_lens=dev.ints(prompts), repetition=dev.put(penalties[0]), frequency=dev.put(penalties[1]),
                     presence=dev.put(penalties[2]), bias_starts=dev.ints(starts_of(biases)), bias_tokens=dev.ints([t for t, _ in flat]), bias_values=dev.put(np.float32([b for _, b in flat])),
                     n_biases=len(flat), masks=dev.ints(words_of(masks)), n_masks=1, mask_stride=vocab // 32, mask_rows=dev.ints(mask_rows))
        halves = []
        for _ in range(2):                                                     # each of a graph's two steps has buffers of its own
            b = {k: dev.ints([0] * rows) for k in ("requests", "places", "positions", "drafted", "chosen", "path", "behind")}
            b.update({k: dev.ints([9] * n) for k in ("full", "counts", "next")}, starts=dev.ints([0] * (n + 1)), status=dev.ints([9]),
                     qkv=[dev.alloc(rows * ld * 2) for _ in range(layers)], q=[dev.alloc(rows * n_q * d * 2) for _ in range(layers)],
                     k=[dev.alloc(rows * n_kv * d * 2) for _ in range(layers)], out=[dev.alloc(rows * n_q * d * 2) for _ in range(layers)], logits=dev.alloc(rows * vocab * 4),
                     adjusted=dev.alloc(rows * vocab * 4), chance=dev.alloc(rows * 4))
            halves.append(b)

        def step(a):
            b, x = 1 - a, halves[a]
            sts.op_block_tables(sts.BlockTables(n_requests=n, max_pages=width, max_rows=rows, free_capacity=pages, table_stride=width, cached=lens[a], added=counts_of_rows, free_pages=free_dev,
                                                n_free=count[a], tables=tables, lens=x["full"], row_starts=x["starts"], requests=x["requests"], positions=x["behind"], places=x["places"],
                                                n_free_left=count[b], status=x["status"]), s)
            batch = sts.TreeBatch(dtype=1, n_requests=n, max_rows=rows, n_q=n_q, n_kv=n_kv, d=d, pool_pages=pages, max_pages=width, table_stride=width, tables=tables, cached=lens[a],
                                  row_starts=x["starts"], parents=parents, positions=x["positions"], workspace=ws, workspace_bytes=size)
            sts.op_attn_tree_plan(batch, s)
            for i in range(layers):
                sts.op_norm_rope(norm, rope, sts.RopeRows(dtype=1, rows=rows, n_q=n_q, n_kv=n_kv, d=d, pool_pages=pages, q=x["qkv"][i], q_stride=ld, q_out=x["q"][i], q_out_stride=n_q * d,
                                                          k=x["qkv"][i] + n_q * d * 2, k_stride=ld, k_out=x["k"][i], k_out_stride=n_kv * d, v=x["qkv"][i] + (n_q + n_kv) * d * 2, v_stride=ld,
                                                          pool=pools[i], positions=x["positions"], places=x["places"]), s)
                sts.op_attn_tree(batch, x["q"][i], n_q * d, pools[i], x["out"][i], n_q * d, None, 0.0, s)
            sts.op_gemm_noalloc(x["out"][-1], w_dev, x["logits"], rows, vocab, n_q * d, "64x128", 1, 0, s)
            sts.op_adjust_logits(sts.AdjustLogits(dtype=0, rows=rows, vocab=vocab, n_requests=n, row_stride=vocab, out_stride=vocab, logits=x["logits"], out=x["adjusted"],
                                                  requests=x["requests"], row_starts=x["starts"], parents=parents, drafted=x["drafted"], **fixed), s)
            sts.op_logprobs(sts.Logprobs(dtype=0, rows=rows, vocab=vocab, top_k=1, row_stride=vocab, logits=x["adjusted"], top_logprob=x["chance"], top_token=x["chosen"], workspace=lp_ws,
                                         workspace_bytes=max(sts.op_logprobs_workspace(0, rows, vocab, 1), 16)), s)
            sts.op_tree_accept(sts.TreeAccept(n_requests=n, max_rows=rows, cached=lens[a], row_starts=x["starts"], parents=parents, tokens=x["drafted"], chosen=x["chosen"], lens=lens[b],
                                              counts=x["counts"], path=x["path"], next_token=x["next"], max_pages=width, free_capacity=pages, table_stride=width, tables=tables,
                                              free_pages=free_dev, n_free=count[b]), s)
            sts.op_tree_compact(sts.TreeCompact(n_requests=n, max_rows=rows, n_kv=n_kv, d=d, pool_pages=pages, max_pages=width, table_stride=width, tables=tables, cached=lens[a],
                                                row_starts=x["starts"], counts=x["counts"], path=x["path"]), pools, s)

        kv = [[[np.zeros((0, n_kv, d), np.float32)] * 2 for _ in range(n)] for _ in range(layers)]       # the host's cache: by layer and request K and V
        accepted = []

        def fill(a):
            x, qkv = halves[a], [rounded(rng.standard_normal((rows, ld)), dtype) for _ in range(layers)]
            drafted = rng.integers(0, 3, rows).astype(np.int32)
            for p, y in zip(x["qkv"], qkv):
                dev.write(p, stored(y, dtype))
            dev.write(x["drafted"], drafted)
            return qkv, drafted

        def check(a, qkv, drafted, last):
            """Step a's buffers against the cache before it, which then takes the path in; `last`: nothing ran behind it."""
            x, cached = halves[a], [len(kv[0][r][0]) for r in range(n)]
            assert dev.get(x["status"], 1, "i32")[0] == 0 and dev.get(x["starts"], n + 1, "i32").tolist() == starts.tolist()
            positions = dev.get(x["positions"], rows, "i32")
            ups = [up for t in trees for up in ancestors(t)]
            owner = np.repeat(np.arange(n), [len(t) for t in trees])
            assert positions.tolist() == [-1 if up is None else cached[r] + len(up) - 1 for r, up in zip(owner, ups)]
            for i in range(layers):
                y = qkv[i].reshape(rows, n_q + 2 * n_kv, d).astype(np.float64)
                got_q, got_k = dev.get(x["q"][i], (rows, n_q, d), dtype), dev.get(x["k"][i], (rows, n_kv, d), dtype)
                for got, part, g in ((got_q, y[:, :n_q], gains[0]), (got_k, y[:, n_q:n_q + n_kv], gains[1])):
                    want, sz = norm_rope_reference(sts, rope, part, g, np.float64(np.float32(eps)), 0, positions)
                    near(got, want, norm_rope_bound(want, sz, dtype))
                at = [slice(starts[r], starts[r + 1]) for r in range(n)]
                new = [[np.concatenate([kv[i][r][0], got_k[at[r]]]), np.concatenate([kv[i][r][1], qkv[i].reshape(rows, -1, d)[at[r], n_q + n_kv:]])] for r in range(n)]
                got = dev.get(x["out"][i], (rows, n_q, d), dtype)
                want, bound, _, _ = tree_reference(got_q, [m[0] for m in new], [m[1] for m in new], cached, trees, heads, d ** -0.5, dtype)
                near(got, want, bound)
                kv[i] = new
            logits = dev.get(x["logits"], (rows, vocab), "f32")
            wide = got.reshape(rows, -1).astype(np.float64)
            near(logits, wide @ w.T, n_q * d * 2.0 ** -23 * np.abs(wide) @ np.abs(w.T) + 1e-6)
            adjusted, chosen = dev.get(x["adjusted"], (rows, vocab), "f32"), dev.get(x["chosen"], rows, "i32")
            real = [r for r, up in enumerate(ups) if up is not None]
            padded = [t if None not in ancestors(t) else [p if p >= -1 else -1 for p in t] for t in trees]       # rows that are no nodes: looked at by nobody
            c = dict(x=logits, requests=owner, tokens=history, lens=held, prompts=prompts, penalties=penalties, trees=padded, drafted=drafted, biases=biases, masks=masks, mask_rows=mask_rows)
            want = adjust_reference(logits.astype(np.float64), *[c[k] for k in ("requests", "tokens", "lens", "prompts", "penalties", "trees", "drafted", "biases", "masks", "mask_rows")])[real]
            fine = np.isfinite(want)
            assert np.array_equal(adjusted[real][~fine], want[~fine])
            near(adjusted[real][fine], want[fine], np.abs(want[fine]) * 2.0 ** -23 + 1e-38)
            assert np.array_equal(chosen, adjusted.argmax(1))
            counts, path = dev.get(x["counts"], n, "i32"), dev.get(x["path"], rows, "i32")
            for r in range(n):
                want, token = accept_reference(trees[r], drafted[starts[r]:starts[r + 1]], chosen[starts[r]:starts[r + 1]])
                assert counts[r] == len(want) and path[starts[r]:starts[r + 1]].tolist() == want + [-1] * (len(trees[r]) - len(want)) and dev.get(x["next"], n, "i32")[r] == token
                keep = list(range(cached[r])) + [cached[r] + j for j in want]
                for i in range(layers):
                    kv[i][r] = [m[keep] for m in kv[i][r]]
                accepted.append(len(want))
            if last:
                length, t = [len(kv[0][r][0]) for r in range(n)], dev.get(tables, (n, width), "i32")
                own = [p for r in range(n) for p in t[r, :-(-length[r] // 16)]]
                left = dev.get(count[1 - a], 1, "i32")[0]
                assert dev.get(lens[1 - a], n, "i32").tolist() == length and left == pages - len(own)
                assert sorted(own + dev.get(free_dev, pages, "i32")[:left].tolist()) == list(range(pages))       # no page is lost or held twice
                for i in range(layers):
                    p = dev.get(pools[i], (pages, n_kv, 32 * d), dtype)
                    for r in range(n):
                        q = p[t[r, :-(-length[r] // 16)]]
                        assert np.array_equal(q[..., :16 * d].reshape(-1, n_kv, 16, d).transpose(0, 2, 1, 3).reshape(-1, n_kv, d)[:length[r]], kv[i][r][0])
                        assert np.array_equal(q[..., 16 * d:].reshape(-1, n_kv, d, 16).transpose(0, 3, 1, 2).reshape(-1, n_kv, d)[:length[r]], kv[i][r][1])

        for a in range(2):
            inputs = fill(a)
            step(a)
            dev.sync()
            check(a, *inputs, last=True)
        replay = dev.graph(s, lambda: (step(0), step(1)))
        for _ in range(8):
            inputs = [fill(0), fill(1)]
            replay()
            dev.sync()
            check(0, *inputs[0], last=False)
            check(1, *inputs[1], last=True)
        assert max(accepted) >= 3 and min(accepted) == 1 and max(len(x[0]) for x in kv[0]) > 32


def test_drafts_behind_32_bits(sts):  # noqa: F811
    """A pool of more than 2^31 elements and 2^32 bytes: its last pages are written by the append, read by the attention, and their rows moved."""
    rng = np.random.default_rng(23)
    n_kv, heads, d, pages = 16, 2, 128, 34000
    n_q, cached, trees = heads * n_kv, [17, 40, 3], [random_tree(rng, 20), chain(9), random_tree(rng, 40)]
    lens, width = [c + len(t) for c, t in zip(cached, trees)], 4
    tables = np.array([[pages - 1, 5, pages - 2, 9], [pages - 3, pages - 4, 0, pages - 7], [1, pages - 5, pages - 6, 4]], np.int32)
    assert pages * n_kv * 32 * d > 2 ** 31
    everything = sum(lens)
    qkv = rounded(rng.standard_normal((everything, (n_q + 2 * n_kv) * d)), "bf16")
    places = np.array([tables[r, t // 16] * 16 + t % 16 for r in range(3) for t in range(lens[r])], np.int32)
    rope, ld, starts = sts.Rope(rotary_dim=2, theta=1e4), qkv.shape[1], starts_of(trees)
    with Device() as dev:
        pool, base = dev.alloc(pages * n_kv * 32 * d * 2), dev.put(qkv, "bf16")
        k_out, q_out = dev.alloc(everything * n_kv * d * 2), dev.alloc(everything * n_q * d * 2)
        sts.op_norm_rope(sts.HeadNorm(eps=1e-6), rope, sts.RopeRows(dtype=1, rows=everything, n_q=n_q, n_kv=n_kv, d=d, pool_pages=pages, q=base, q_stride=ld, q_out=q_out, q_out_stride=n_q * d,
                                                                    k=base + n_q * d * 2, k_stride=ld, k_out=k_out, k_out_stride=n_kv * d, v=base + (n_q + n_kv) * d * 2, v_stride=ld,
                                                                    pool=pool, positions=dev.ints([0] * everything), places=dev.put(places)))
        rows, size = int(starts[-1]), sts.attn_tree_workspace(3, int(starts[-1]), n_q, n_kv, d)
        q = rounded(rng.standard_normal((rows, n_q, d)), "bf16")
        out, table = dev.alloc(rows * n_q * d * 2), dev.ints(tables)
        common = dict(n_requests=3, max_rows=rows, n_kv=n_kv, d=d, pool_pages=pages, max_pages=width, table_stride=width, tables=table, cached=dev.ints(cached), row_starts=dev.ints(starts))
        batch = sts.TreeBatch(dtype=1, n_q=n_q, parents=dev.ints([p for t in trees for p in t]), workspace=dev.alloc(size), workspace_bytes=size, **common)
        sts.op_attn_tree_plan(batch)
        sts.op_attn_tree(batch, dev.put(q, "bf16"), n_q * d, pool, out, n_q * d)
        paths = [[0, 3, 19], [0, 8], [0, 1, 2, 30, 39]]
        path = [x for p, t in zip(paths, trees) for x in p + [-1] * (len(t) - len(p))]
        sts.op_tree_compact(sts.TreeCompact(counts=dev.ints([3, 2, 5]), path=dev.ints(path), **common), [pool])
        dev.sync()
        got, got_k = dev.get(out, (rows, n_q, d), "bf16"), dev.get(k_out, (everything, n_kv, d), "bf16")
        page = np.stack([[dev.get(pool + int(p) * n_kv * 32 * d * 2, (n_kv, 32 * d), "bf16") for p in row] for row in tables])
    first = np.concatenate([[0], np.cumsum(lens)])
    k = [got_k[first[r]:first[r + 1]] for r in range(3)]
    v = [qkv.reshape(everything, -1, d)[first[r]:first[r + 1], n_q + n_kv:] for r in range(3)]
    want, bound, _, _ = tree_reference(q, k, v, cached, trees, heads, d ** -0.5, "bf16")
    near(got, want, bound)
    for r in range(3):
        keep = list(range(cached[r])) + [cached[r] + j for j in paths[r]]
        pk = page[r, :, :, :16 * d].reshape(width, n_kv, 16, d).transpose(0, 2, 1, 3).reshape(-1, n_kv, d)[:len(keep)]
        pv = page[r, :, :, 16 * d:].reshape(width, n_kv, d, 16).transpose(0, 3, 1, 2).reshape(-1, n_kv, d)[:len(keep)]
        assert np.array_equal(pk, k[r][keep]) and np.array_equal(pv, v[r][keep])


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_adjust_logits_behind_32_bits(sts, dtype):  # noqa: F811
    """Rows, histories and masks whose offsets pass 32 bits, out of place and in place."""
    rng = np.random.default_rng(9)
    vocab, rows, stride = 5003, 3, (1 << 31) // 2 + 7                     # the last row begins behind 2^31 elements
    c = adjust_case(rng, dtype, vocab, [[-1]] * rows, 40, 3, 1.0)
    c.update(trees=None, mask_rows=np.int32([2, 0, 1]))
    size = 4 if dtype == "f32" else 2
    with Device() as dev:
        far = dev.alloc(2 * stride * size + vocab * size)
        tokens, token_stride = dev.alloc(((2 << 30) + 40) * 4), 1 << 30
        words = words_of(c["masks"])
        masks, mask_stride = dev.alloc(((2 << 30) + words.shape[1]) * 4), 1 << 30
        for r in range(rows):
            dev.write(far + r * stride * size, stored(c["x"][r], dtype))
            dev.write(tokens + r * token_stride * 4, c["tokens"][r])
            dev.write(masks + r * mask_stride * 4, words[r])
        a, out = adjust_description(sts, dev, dtype, c)
        a.logits, a.row_stride, a.tokens, a.token_stride, a.masks, a.mask_stride = far, stride, tokens, token_stride, masks, mask_stride
        sts.op_adjust_logits(a)
        dev.sync()
        check_adjusted(dev.get(out, (rows, vocab), dtype), c, dtype)
        a.out, a.out_stride = far, stride
        sts.op_adjust_logits(a)
        dev.sync()
        check_adjusted(np.stack([dev.get(far + r * stride * size, vocab, dtype) for r in range(rows)]), c, dtype)
