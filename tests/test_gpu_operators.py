"""Operators on device data (block tables, rotary positions with append, attention over shared prefixes, log probabilities) against plain
implementations in 64 bits, on the same rounded inputs.

Tolerances. u is half a step of the output's type (bf16 2^-8, fp16 2^-11, fp32 2^-24), relative to the value. Each test states its bound from the
roundings that the kernels make; nothing is measured first."""
import numpy as np
import pytest

from tests.device import Device, pool_of, rounded

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}


@pytest.fixture(scope="module")
def sts():
    from paper_2504_19516_amd import sts as m
    m.lib()
    return m


# ------------------------------------------------------------------------------------------ block tables
def tables_reference(cached, added, free, tables, max_pages, max_rows):
    n, out = len(cached), tables.copy()
    pages = lambda t: -(-t // 16)  # noqa: E731
    need = [pages(c + a) - pages(c) for c, a in zip(cached, added)]
    status = 0
    if any(x < 0 for x in cached + added):
        status = -1
    elif sum(need) > len(free) or sum(added) > max_rows or any(a > 0 and pages(c + a) > max_pages for c, a in zip(cached, added)):
        status = -2
    if status:
        return dict(status=status, starts=[0] * (n + 1), lens=cached, left=len(free), tables=out, rows=[])
    top, rows = len(free) - sum(need), []
    for i, (c, a) in enumerate(zip(cached, added)):
        for e in range(need[i]):
            out[i, pages(c) + e] = free[top + sum(need[:i]) + e]
        rows += [(i, c + t, out[i, (c + t) // 16] * 16 + (c + t) % 16) for t in range(a)]
    return dict(status=0, starts=np.concatenate([[0], np.cumsum(added)]), lens=np.add(cached, added), left=top, tables=out, rows=rows)


def run_tables(sts, dev, cached, added, free, tables, max_pages, max_rows, stream=None):
    n = len(cached)
    fill = np.full(max_rows, 777, np.int32)
    a = dict(cached=dev.ints(cached), added=dev.ints(added), free_pages=dev.ints(free), n_free=dev.ints([len(free)]), tables=dev.ints(tables), lens=dev.ints([777] * n),
             row_starts=dev.ints([777] * (n + 1)), requests=dev.put(fill), positions=dev.put(fill), places=dev.put(fill), n_free_left=dev.ints([777]), status=dev.ints([777]))
    sts.op_block_tables(sts.BlockTables(n_requests=n, max_pages=max_pages, max_rows=max_rows, free_capacity=len(free), table_stride=tables.shape[1], **a), stream)
    dev.sync()
    size = dict(lens=n, row_starts=n + 1, requests=max_rows, positions=max_rows, places=max_rows, n_free_left=1, status=1)
    got = {k: dev.get(a[k], s, "i32") for k, s in size.items()}
    got["tables"] = dev.get(a["tables"], tables.shape, "i32")
    return got


def check_tables(got, want, max_rows):
    assert got["status"][0] == want["status"] and got["n_free_left"][0] == want["left"]
    assert np.array_equal(got["row_starts"], want["starts"]) and np.array_equal(got["lens"], want["lens"])
    assert np.array_equal(got["tables"], want["tables"])
    k = len(want["rows"])
    for j, name in enumerate(("requests", "positions", "places")):
        assert np.array_equal(got[name][:k], [r[j] for r in want["rows"]]), name
        assert (got[name][k:] == (-1 if name == "places" else 777)).all(), name


def tables_case(rng, cached, added, width, spare=5):
    n = len(cached)
    held = [-(-c // 16) for c in cached]
    ids = rng.permutation(sum(held) + sum(-(-(c + a) // 16) for c, a in zip(cached, added)) + spare).astype(np.int32)
    tables = np.full((n, width), -7, np.int32)
    for i, h in enumerate(held):
        tables[i, :h], ids = ids[:h], ids[h:]
    need = sum(-(-(c + a) // 16) - -(-c // 16) for c, a in zip(cached, added))
    return tables, ids[:need + spare]


@pytest.mark.parametrize("n", [1, 2, 63, 257, 1500, 4096])
def test_block_tables(sts, n):
    rng = np.random.default_rng(n)
    cached = rng.integers(0, 70, n).tolist()
    added = np.where(rng.random(n) < 0.7, 1, rng.integers(0, 40, n)).tolist()
    for edge, c, a in [(0, 16, 1), (n // 2, 0, 0), (n - 1, 15, 17)]:
        cached[edge], added[edge] = c, a
    width = 9                                              # entries of a row that may be used, and two more
    tables, free = tables_case(rng, cached, added, width + 2)
    rows = sum(added) + 13
    with Device() as dev:
        check_tables(run_tables(sts, dev, cached, added, free, tables, width, rows), tables_reference(cached, added, free, tables, width, rows), rows)


@pytest.mark.parametrize("cached,added", [([], []), ([0], [0]), ([0], [1]), ([5000], [9000]), ([0, 0, 0], [4097, 1, 2500]), ([31, 32, 33], [0, 0, 0])])
def test_block_tables_edges(sts, cached, added):
    tables, free = tables_case(np.random.default_rng(3), cached, added, 900)
    rows = sum(added) + 3
    with Device() as dev:
        check_tables(run_tables(sts, dev, cached, added, free, tables, 900, rows), tables_reference(cached, added, free, tables, 900, rows), rows)


@pytest.mark.parametrize("what", ["pages", "rows", "table", "negative", "negative cached", "free count"])
def test_block_tables_that_cannot_be_had_change_nothing(sts, what):
    rng = np.random.default_rng(9)
    cached, added = [3, 40, 16, 0], [14, 1, 1, 1300]
    width, rows = 90, 1400
    if what == "rows":
        rows = sum(added) - 1
    if what == "table":
        width = 81                                         # the last request needs 82 pages
    if what == "negative":
        added[1] = -1
    tables, free = tables_case(rng, [max(c, 0) for c in cached], [max(a, 0) for a in added], 95, spare=0)
    if what == "negative cached":
        cached[2] = -5
    if what == "pages":
        free = free[:-1]
    want = tables_reference(cached, added, free, tables, width, rows)
    with Device() as dev:
        if what == "free count":                           # more free pages than the array holds
            fill = np.full(rows, 777, np.int32)
            status, left, starts = dev.ints([7]), dev.ints([7]), dev.ints([7] * 5)
            t = dev.ints(tables)
            places = dev.put(fill)
            sts.op_block_tables(sts.BlockTables(n_requests=4, max_pages=width, max_rows=rows, free_capacity=len(free), table_stride=95, cached=dev.ints(cached), added=dev.ints(added),
                                                free_pages=dev.ints(free), n_free=dev.ints([len(free) + 1]), tables=t, lens=dev.ints([7] * 4), row_starts=starts, requests=dev.put(fill),
                                                positions=dev.put(fill), places=places, n_free_left=left, status=status))
            dev.sync()
            assert dev.get(status, 1, "i32")[0] == -1 and dev.get(left, 1, "i32")[0] == len(free) + 1
            assert not dev.get(starts, 5, "i32").any() and (dev.get(places, rows, "i32") == -1).all() and np.array_equal(dev.get(t, tables.shape, "i32"), tables)
            return
        assert want["status"] != 0
        check_tables(run_tables(sts, dev, cached, added, free, tables, width, rows), want, rows)


# ------------------------------------------------------------------------------------------ rotary positions
ROPES = {
    "plain": dict(scaling=0, theta=1e4),
    "linear": dict(scaling=1, theta=5e5, factor=4.0),
    "base": dict(scaling=2, theta=1e4, factor=8.0),
    "bands": dict(scaling=3, theta=5e5, factor=8.0, low=1.0, high=4.0, original_len=8192),
    "ramp": dict(scaling=4, theta=1e4, factor=16.0, low=1.0, high=32.0, original_len=4096, magnitude=1.2772588),
}


def rope_of(sts, name, rotary, interleaved):
    return sts.Rope(rotary_dim=rotary, interleaved=interleaved, **ROPES[name])


def rope_reference(sts, rope, x, positions):
    """x [rows, heads, d] float64."""
    R = rope.rotary_dim
    a = np.asarray(positions, np.float64)[:, None] * sts.rope_frequencies(rope)[None]
    mag = np.float64(np.float32(rope.magnitude)) or 1.0
    c, s = (mag * np.cos(a))[:, None], (mag * np.sin(a))[:, None]
    i, j = (np.arange(0, R, 2), np.arange(1, R, 2)) if rope.interleaved else (np.arange(R // 2), np.arange(R // 2, R))
    y = x.copy()
    y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., j] * c + x[..., i] * s
    size = np.zeros_like(x)                                # |a| + |b| of each element's pair: what the error of an angle is relative to
    size[..., i] = size[..., j] = (np.abs(x[..., i]) + np.abs(x[..., j])) * mag
    return y, size


# One rounding to the type; cosine and sine are off by the rounding of the angle (2^-25 half turns, 9.4e-8) and a few of fp32's: 2^-21 of |a| + |b|
def rope_bound(y, size, dtype):
    return HALF[dtype] * np.abs(y) + size * 2.0 ** -21 + 1e-7 * (dtype == "f16")


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("name,rotary,interleaved,d", [("plain", 128, 0, 128), ("linear", 64, 0, 64), ("base", 32, 1, 64), ("bands", 128, 1, 128), ("ramp", 104, 0, 128),
                                                       ("ramp", 40, 1, 64), ("plain", 2, 0, 6), ("bands", 250, 1, 257), ("linear", 256, 0, 256)])
def test_rope_turns_rows(sts, dtype, name, rotary, interleaved, d):
    """Q out of place from a strided buffer and K in place, positions from 0 to the last of 31 bits and negative ones."""
    rng = np.random.default_rng(rotary + d)
    rows, n_q, n_kv = 37, 5, 2
    rope = rope_of(sts, name, rotary, interleaved)
    positions = np.concatenate([[0, 1, 2 ** 31 - 1, -1, -70000], rng.integers(0, 2 ** 20, rows - 5)]).astype(np.int32)
    q, k = (rounded(rng.standard_normal((rows, h, d)), dtype) for h in (n_q, n_kv))
    ld = (n_q + n_kv) * d + 3
    both = np.full((rows, ld), 5.0, np.float32)
    both[:, :n_q * d], both[:, n_q * d:-3] = q.reshape(rows, -1), k.reshape(rows, -1)
    size = 4 if dtype == "f32" else 2
    with Device() as dev:
        buf, out = dev.put(both, dtype), dev.alloc(rows * n_q * d * size)
        sts.op_rope(rope, sts.RopeRows(dtype=sts.DTYPES[dtype], rows=rows, n_q=n_q, n_kv=n_kv, d=d, q=buf, q_stride=ld, q_out=out, q_out_stride=n_q * d, k=buf + n_q * d * size,
                                       k_stride=ld, k_out=buf + n_q * d * size, k_out_stride=ld, positions=dev.ints(positions)))
        dev.sync()
        got_q, got = dev.get(out, (rows, n_q, d), dtype), dev.get(buf, (rows, ld), dtype)
    for y, x in ((got_q, q), (got[:, n_q * d:-3].reshape(rows, n_kv, d), k)):
        want, s = rope_reference(sts, rope, x.astype(np.float64), positions)
        assert (np.abs(y - want) <= rope_bound(want, s, dtype)).all()
        assert np.array_equal(y[..., rotary:], x[..., rotary:])
    assert np.array_equal(got[:, :n_q * d], both[:, :n_q * d]) and (got[:, -3:] == 5.0).all()        # what is not K is left as it was


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows,n_q,n_kv,d,rotary,interleaved,offset", [(1, 4, 4, 64, 64, 0, 0), (3, 32, 8, 128, 128, 0, 0), (33, 8, 1, 128, 64, 1, 0), (70, 6, 2, 64, 24, 0, 2),
                                                                      (500, 32, 8, 128, 128, 0, 0), (513, 4, 4, 64, 32, 1, 0), (517, 8, 2, 128, 104, 0, 2)])
def test_rope_appends_to_pages(sts, dtype, rows, n_q, n_kv, d, rotary, interleaved, offset):
    """Ragged runs of positions, in pages in any order, from aligned rows and from rows two bytes off; rows without a place, or with one behind the pool, are not
    appended, and what no row fills is left as it was."""
    rng = np.random.default_rng(rows)
    rope = rope_of(sts, "bands", rotary, interleaved)
    pages = rows // 4 + 9
    order, positions, places, used = rng.permutation(pages), [], [], 0
    while len(positions) < rows:
        start, m = int(rng.integers(0, 40)), min(int(rng.integers(1, 60)), rows - len(positions))
        first = start // 16
        if used + (start + m - 1) // 16 - first + 1 > pages:
            places += [-1] * (rows - len(positions))
            positions += range(rows - len(positions))
            break
        places += [int(order[used + (start + t) // 16 - first]) * 16 + (start + t) % 16 for t in range(m)]
        positions += range(start + 50000, start + 50000 + m)
        used += (start + m - 1) // 16 - first + 1
    places = np.asarray(places, np.int32)
    if rows > 3:
        places[1], places[-1] = -1, pages * 16
    qkv = rounded(rng.standard_normal((rows, (n_q + 2 * n_kv) * d)), dtype)
    old = rounded(rng.standard_normal((pages, n_kv, 32 * d)), dtype)
    ld = qkv.shape[1]
    with Device() as dev:
        base, pool, out, kout = dev.put(qkv, dtype, offset), dev.put(old, dtype), dev.alloc(rows * n_q * d * 2), dev.alloc(rows * n_kv * d * 2)
        sts.op_rope(rope, sts.RopeRows(dtype=sts.DTYPES[dtype], rows=rows, n_q=n_q, n_kv=n_kv, d=d, pool_pages=pages, q=base, q_stride=ld, q_out=out, q_out_stride=n_q * d,
                                       k=base + n_q * d * 2, k_stride=ld, k_out=kout, k_out_stride=n_kv * d, v=base + (n_q + n_kv) * d * 2, v_stride=ld, pool=pool,
                                       positions=dev.ints(positions), places=dev.put(places)))
        dev.sync()
        got_q, got_k = dev.get(out, (rows, n_q, d), dtype), dev.get(kout, (rows, n_kv, d), dtype)
        got = dev.get(pool, old.shape, dtype)
    x = qkv.reshape(rows, n_q + 2 * n_kv, d).astype(np.float64)
    for y, part in ((got_q, x[:, :n_q]), (got_k, x[:, n_q:n_q + n_kv])):
        want, s = rope_reference(sts, rope, part, positions)
        assert (np.abs(y - want) <= rope_bound(want, s, dtype)).all()
    want = old.copy()
    kp, vp = want[:, :, :16 * d].reshape(pages, n_kv, 16, d), want[:, :, 16 * d:].reshape(pages, n_kv, d, 16)      # views: want's last axis is contiguous
    kp, vp = kp.copy(), vp.copy()
    for r, p in enumerate(places):
        if 0 <= p < pages * 16:
            kp[p // 16, :, p % 16], vp[p // 16, :, :, p % 16] = got_k[r], x[r, n_q + n_kv:]
    assert np.array_equal(got[:, :, :16 * d], kp.reshape(pages, n_kv, -1)) and np.array_equal(got[:, :, 16 * d:], vp.reshape(pages, n_kv, -1))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows,n_q,n_kv,d,rotary,interleaved,offset", [(4500, 32, 8, 128, 128, 0, 0), (4507, 32, 8, 128, 128, 1, 0), (2049, 32, 8, 128, 104, 0, 0), (17003, 8, 8, 64, 64, 0, 0),
                                                                      (3001, 8, 8, 64, 36, 1, 0), (9001, 6, 3, 64, 40, 0, 0), (5000, 4, 3, 64, 64, 0, 2), (8200, 8, 8, 128, 64, 0, 0)])
def test_rope_appends_long_prefills(sts, dtype, rows, n_q, n_kv, d, rotary, interleaved, offset):
    """Workgroups of 16 rows that go over their rotations and their heads of V more than once; vectors of eight and of four elements, and single ones; a last workgroup of a few rows."""
    test_rope_appends_to_pages(sts, dtype, rows, n_q, n_kv, d, rotary, interleaved, offset)


# ------------------------------------------------------------------------------------------ attention
def attention_reference(q, k, v, lens, heads, scale, dtype):
    """Output, its bound, lse and its bound. Probabilities are rounded to the type before the product (u each, fp16's smallest ones by 2^-25), the output once; a score of
    d products in fp32 is off by at most d 2^-24 of the sum of their sizes, which is relative in the probability."""
    n, n_q, d = q.shape
    out, bound, lse, lb, u = np.zeros((n, n_q, d)), np.zeros((n, n_q, d)), np.full((n, n_q), -np.inf), np.zeros((n, n_q)), HALF[dtype]
    for r, c in enumerate(lens):
        for h in range(n_q if c > 0 else 0):
            kh, vh = k[r][:c, h // heads].astype(np.float64), v[r][:c, h // heads].astype(np.float64)
            x = kh @ q[r, h].astype(np.float64) * scale
            m = x.max()
            p = np.exp(x - m)
            p, z = p / p.sum(), p.sum()
            delta = 2.0 ** -24 * d * (np.abs(kh) @ np.abs(q[r, h]).astype(np.float64) * scale).max() + 2.0 ** -21 * (1 + np.abs(x - m).max() * 2.0 ** -3)
            out[r, h], lse[r, h], size = p @ vh, m + np.log(z), p @ np.abs(vh)
            bound[r, h] = u * (np.abs(out[r, h]) + size) + 2 * delta * size + (2.0 ** -25 * np.abs(vh).sum(0) + 2.0 ** -24 if dtype == "f16" else 0.0) + 1e-30
            lb[r, h] = delta + 2.0 ** -22 * (abs(lse[r, h]) + np.abs(x).max() + 8)
    return out, bound, lse, lb


def attention_case(rng, groups, lens, n_kv, d, spare=3):
    """Requests of a group agree in the first `shared` tokens (whole pages). groups: [(members, shared)]. Returns k, v by request, tables, pages."""
    n, k, v, rows, used = len(lens), [], [], [], 0
    tables = np.full((n, max([-(-c // 16) for c in lens] + [1]) + 2), -9, np.int64)
    r = 0
    for members, shared in groups:
        s = shared // 16 * 16
        ks, vs = rng.standard_normal((2, s, n_kv, d))
        common = list(range(used, used + s // 16))
        used += s // 16
        for _ in range(members):
            own = max(0, lens[r] - s)
            m = -(-own // 16)
            row = common + list(range(used, used + m))
            used += m
            tables[r, :min(len(row), -(-lens[r] // 16))] = row[:-(-lens[r] // 16)]
            k.append(np.concatenate([ks, rng.standard_normal((own, n_kv, d))])[:max(lens[r], 0)])
            v.append(np.concatenate([vs, rng.standard_normal((own, n_kv, d))])[:max(lens[r], 0)])
            r += 1
    order = rng.permutation(used + spare)
    return k, v, np.where(tables >= 0, order[np.maximum(tables, 0)], tables).astype(np.int32), used + spare


def run_attention(sts, dev, dtype, q, pool, tables, lens, groups, heads, scale=0.0, stream=None, starts=None, q_pad=0, out_pad=0, q_offset=0, pool_pages=None, want_lse=True):
    n, n_q, d = q.shape
    n_kv = n_q // heads
    starts = np.concatenate([[0], np.cumsum([m for m, _ in groups])]) if starts is None else starts
    size = sts.attn_shared_workspace(n, n_q, n_kv, d)
    qs = np.full((n, n_q * d + q_pad), 3.0, np.float32)
    qs[:, :n_q * d] = q.reshape(n, -1)
    out = dev.put(np.full((n, n_q * d + out_pad), 7.0), dtype)
    lse = dev.put(np.full((n, n_q), 7.0, np.float32))
    batch = sts.AttnBatch(dtype=sts.DTYPES[dtype], n_requests=n, n_groups=len(groups), n_q=n_q, n_kv=n_kv, d=d, pool_pages=pool.shape[0] if pool_pages is None else pool_pages,
                          max_pages=tables.shape[1], table_stride=tables.shape[1], tables=dev.ints(tables), lens=dev.ints(lens), group_starts=dev.ints(starts) if groups else None,
                          shared_lens=dev.ints([s for _, s in groups]) if groups else None, workspace=dev.alloc(size), workspace_bytes=size)
    args = (batch, dev.put(qs, dtype, q_offset), n_q * d + q_pad, dev.put(pool, dtype), out, n_q * d + out_pad, lse if want_lse else None, scale, stream)

    def call():
        sts.op_attn_shared_plan(batch, stream)
        sts.op_attn_shared(*args)
    call()
    dev.sync()
    got = dev.get(out, (n, n_q * d + out_pad), dtype)
    assert (got[:, n_q * d:] == 7.0).all()
    return got[:, :n_q * d].reshape(n, n_q, d), dev.get(lse, (n, n_q), "f32"), call, (out, lse)


def near(got, want, bound):
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(), float(np.nanmax(np.abs(got - want) / bound)))


CASES = [
    # (query heads, kv heads, d, [(members, shared tokens)], own tokens of each request in turn)
    (4, 4, 64, [(1, 0)], [1]),
    (4, 1, 64, [(1, 0)], [33]),
    (32, 8, 128, [(8, 1031)], [7, 1, 16, 17, 60, 100, 33, 2]),
    (8, 8, 128, [(40, 160)], [5, 31, 64]),
    (32, 8, 128, [(64, 512)], [9, 40, 75]),
    (64, 8, 128, [(9, 300), (1, 0), (4, 77), (3, 512), (7, 150)], [20, 3, 48]),
    (10, 2, 64, [(13, 96), (2, 16), (6, 0)], [1, 200, 31]),
    (32, 1, 64, [(5, 64), (3, 33)], [17, 2]),
    (16, 16, 64, [(70, 48)], [0, 1, 16]),
    (28, 4, 128, [(37, 1600)], [11, 90]),
    (8, 2, 64, [(150, 700), (3, 32)], [6]),
    (4, 2, 128, [(1, 0)], [5000]),
    (8, 1, 64, [(2, 20000)], [3000, 1]),
    (6, 3, 64, [(25, 33), (20, 100)], [1, 15, 40]),
    (256, 256, 64, [(3, 32)], [5, 20]),
    (2, 2, 64, [(1000, 16), (24, 0)], [1, 2, 3, 20]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_shared_attention(sts, dtype, case):
    n_q, n_kv, d, groups, own = CASES[case]
    rng = np.random.default_rng(100 + case)
    lens = []
    for members, shared in groups:
        lens += [shared // 16 * 16 + own[(len(lens) + i) % len(own)] for i in range(members)]
    k, v, tables, pages = attention_case(rng, groups, lens, n_kv, d)
    k, v = [rounded(x, dtype) for x in k], [rounded(x, dtype) for x in v]
    q = rounded(2.0 * rng.standard_normal((len(lens), n_q, d)), dtype)
    pool = pool_of(k, v, tables, lens, pages, dtype, behind=np.nan)       # whatever lies behind a context must not matter
    out, bound, lse, lb = attention_reference(q, k, v, lens, n_q // n_kv, d ** -0.5, dtype)
    with Device() as dev:
        got, got_lse, _, _ = run_attention(sts, dev, dtype, q, pool, tables, lens, groups, n_q // n_kv)
        near(got, out, bound)
        near(got_lse[np.asarray(lens) > 0], lse[np.asarray(lens) > 0], lb[np.asarray(lens) > 0])
        alone, alone_lse, _, _ = run_attention(sts, dev, dtype, q, pool, tables, lens, [], n_q // n_kv)       # nothing said to be shared: the same result
        near(alone, out, bound)
        near(alone_lse[np.asarray(lens) > 0], lse[np.asarray(lens) > 0], lb[np.asarray(lens) > 0])


def small_case(rng, dtype, lens=(40, 0, 35, 16, 33, 64), groups=((3, 32), (3, 16)), n_q=8, n_kv=2, d=64, scale=1.0):
    groups = list(groups)
    k, v, tables, pages = attention_case(rng, groups, list(lens), n_kv, d)
    k, v = [rounded(x, dtype) for x in k], [rounded(x, dtype) for x in v]
    q = rounded(scale * rng.standard_normal((len(lens), n_q, d)), dtype)
    return q, k, v, tables, pages, list(lens), groups


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n_q,n_kv,d,members,shared,own", [(8, 2, 64, 6, 320, 37), (8, 2, 64, 40, 320, 21), (4, 1, 128, 1, 0, 300), (8, 1, 128, 30, 640, 5)])
def test_shared_attention_rounds_its_outputs_once(sts, dtype, n_q, n_kv, d, members, shared, own):
    """Scores that 32 bits hold exactly (q and k of small whole numbers), so that the bound is narrow: the output's own rounding, and of the sum of |p v|
    2 u (2 u + 2^-9) for the probabilities' two numbers of the type, the first cut off (2 u of p), the second of what is left and of 2^-9 p; 2^-22 and 2^-23 |x - m| for an
    exponential and its argument, in numerator and denominator, and a rounding for each of the sums' tokens; fp16 holds probabilities to 2^-24 of the largest.
    Probabilities of one number of the type would be off by u each."""
    rng = np.random.default_rng(members + d)
    heads, lens, groups, u = n_q // n_kv, [shared + own] * members, [(members, shared)], HALF[dtype]
    k, v, tables, pages = attention_case(rng, groups, lens, n_kv, d)
    v = [rounded(x, dtype) for x in v]
    first, rest = rng.integers(-2, 3, (shared, n_kv, d)), rng.integers(-2, 3, (members, own, n_kv, d))
    k = [np.concatenate([first, r]).astype(np.float32) for r in rest]
    q = rng.integers(-2, 3, (members, n_q, d)).astype(np.float32)
    pool = pool_of(k, v, tables, lens, pages, dtype, behind=np.nan)
    with Device() as dev:
        got, _, _, _ = run_attention(sts, dev, dtype, q, pool, tables, lens, groups, heads, scale=0.0625)
    for r in range(members):
        for h in range(n_q):
            x = k[r][:, h // heads].astype(np.float64) @ q[r, h] / 16
            w, vh = np.exp(x - x.max()), v[r][:, h // heads].astype(np.float64)
            out, size = w @ vh / w.sum(), w @ np.abs(vh) / w.sum()
            extra = (2 * u * (2 * u + 2.0 ** -9) + 2 * (2.0 ** -22 + 2.0 ** -23 * np.abs(x - x.max()).max()) + 2 * 2.0 ** -24 * len(x)) * size
            near(got[r, h], out, u * np.abs(out) + extra + (2.0 ** -24 * np.abs(vh).sum(0) / w.sum() + 2.0 ** -25 if dtype == "f16" else 0.0))


def test_shared_attention_empty_and_short_contexts(sts):
    """A context of length 0 gives zeros; a group shares what its shortest member holds."""
    rng = np.random.default_rng(5)
    for lens, groups in (((40, 0, 35, 16, 33, 64), ((3, 32), (3, 16))), ((0, 0), ((2, 64),)), ((47, 20, 15), ((3, 32),)), ((100, 48), ((2, 1000),))):
        q, k, v, tables, pages, lens, groups = small_case(rng, "bf16", lens, groups)
        pool = pool_of(k, v, tables, lens, pages, "bf16", behind=np.inf)
        out, bound, lse, lb = attention_reference(q, k, v, lens, 4, 0.125, "bf16")
        with Device() as dev:
            got, got_lse, _, _ = run_attention(sts, dev, "bf16", q, pool, tables, lens, groups, 4)
        near(got, out, bound)
        some = np.asarray(lens) > 0
        near(got_lse[some], lse[some], lb[some])
        assert (got[~some] == 0).all() and np.isneginf(got_lse[~some]).all()


def test_shared_attention_strides_scale_and_no_lse(sts):
    rng = np.random.default_rng(6)
    q, k, v, tables, pages, lens, groups = small_case(rng, "f16", scale=3.0)
    pool = pool_of(k, v, tables, lens, pages, "f16", behind="noise", rng=rng)
    out, bound, lse, lb = attention_reference(q, k, v, lens, 4, 0.3, "f16")
    with Device() as dev:
        for q_pad, out_pad, offset in ((8, 0, 0), (3, 5, 0), (0, 1, 2), (8, 8, 2)):
            got, got_lse, _, _ = run_attention(sts, dev, "f16", q, pool, tables, lens, groups, 4, scale=0.3, q_pad=q_pad, out_pad=out_pad, q_offset=offset, want_lse=q_pad != 3)
            near(got, out, bound)
            assert (got_lse == 7.0).all() if q_pad == 3 else np.isneginf(got_lse[1]).all()


@pytest.mark.parametrize("starts", [[0, 3, 5], [1, 3, 6], [0, 7, 6], [0, -1, 6], [0, 4, 2]])
def test_shared_attention_groups_out_of_order_share_nothing(sts, starts):
    rng = np.random.default_rng(7)
    q, k, v, tables, pages, lens, groups = small_case(rng, "bf16")
    pool = pool_of(k, v, tables, lens, pages, "bf16")
    out, bound, _, _ = attention_reference(q, k, v, lens, 4, 0.125, "bf16")
    with Device() as dev:
        got, _, _, _ = run_attention(sts, dev, "bf16", q, pool, tables, lens, groups, 4, starts=starts)
    near(got, out, bound)


def test_shared_attention_pages_and_lengths_out_of_range_are_nan(sts):
    """Only the requests that read them: a bad page of a shared part is its whole group's."""
    rng = np.random.default_rng(8)
    q, k, v, tables, pages, lens, groups = small_case(rng, "bf16", (40, 48, 35, 16, 33, 64))
    pool = pool_of(k, v, tables, lens, pages, "bf16")
    out, bound, _, _ = attention_reference(q, k, v, lens, 4, 0.125, "bf16")
    for name, where, value, hit in (("own", (1, 2), pages, [1]), ("own", (5, 3), -1, [5]), ("shared", (0, 1), 2 ** 31 - 1, [0, 1, 2])):
        t = tables.copy()
        t[where] = value
        with Device() as dev:
            got, lse, _, _ = run_attention(sts, dev, "bf16", q, pool, t, lens, groups, 4)
        fine = [r for r in range(6) if r not in hit]
        assert np.isnan(got[hit]).all() and np.isnan(lse[hit]).all(), name
        near(got[fine], out[fine], bound[fine])
    for bad in (-3, tables.shape[1] * 16 + 1):
        ls = list(lens)
        ls[4] = bad
        with Device() as dev:
            got, lse, _, _ = run_attention(sts, dev, "bf16", q, pool, tables, ls, groups, 4)
        fine = [0, 1, 2, 3, 5]
        assert np.isnan(got[4]).all() and np.isnan(lse[4]).all()
        near(got[fine], out[fine], bound[fine])


def test_shared_attention_infinities_stay_with_their_tokens(sts):
    """Scores of -inf weigh nothing, a V of inf reaches the output of the rows that attend to it alone."""
    rng = np.random.default_rng(10)
    q, k, v, tables, pages, lens, groups = small_case(rng, "bf16", (40, 48, 35, 16, 33, 64))
    q[:] = np.abs(q) + 0.25
    k[0][3] = k[1][3] = k[2][3] = -3e38                    # in the shared part: every score of it overflows to -inf
    v[5][60, 0, 7] = np.inf
    pool = pool_of(k, v, tables, lens, pages, "bf16")
    with np.errstate(all="ignore"):
        out, bound, _, _ = attention_reference(q, k, v, lens, 4, 0.125, "bf16")
    with Device() as dev:
        got, _, _, _ = run_attention(sts, dev, "bf16", q, pool, tables, lens, groups, 4)
    # the references of the first group without token 3
    for r in range(3):
        keep = [t for t in range(lens[r]) if t != 3]
        o, b, _, _ = attention_reference(q[r:r + 1], [k[r][keep]], [v[r][keep]], [len(keep)], 4, 0.125, "bf16")
        near(got[r:r + 1], o, b)
    near(got[3:5], out[3:5], bound[3:5])
    assert np.isposinf(got[5, :4, 7]).all()
    rest = np.ones((8, 64), bool)
    rest[:4, 7] = False
    o, b, _, _ = attention_reference(q[5:], [k[5]], [np.where(np.isinf(v[5]), 0, v[5])], [64], 4, 0.125, "bf16")
    near(got[5][rest], o[0][rest], b[0][rest])


# 43 requests of four heads on 11 shared pages: tiles of 128 and of 44 rows, the second of which leaves two waves without rows; the last pages are a part of a tile
WIDE = dict(lens=tuple(176 + 1 + 5 * i % 37 for i in range(43)), groups=((43, 176),))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_shared_attention_wide_pages_out_of_range_are_nan(sts, dtype):
    """A bad page of the shared part, whichever wave fetches it, is the whole group's; one of a request's own its alone."""
    q, k, v, tables, pages, lens, groups = small_case(np.random.default_rng(21), dtype, **WIDE)
    pool = pool_of(k, v, tables, lens, pages, dtype)
    out, bound, _, _ = attention_reference(q, k, v, lens, 4, 0.125, dtype)
    for at, value in ((0, pages), (1, -1), (2, 2 ** 31 - 1), (3, -2 ** 31), (6, pages + 3), (8, -5), (10, pages)):
        t = tables.copy()
        t[0, at] = value
        with Device() as dev:
            got, lse, _, _ = run_attention(sts, dev, dtype, q, pool, t, lens, groups, 4)
        assert np.isnan(got).all() and np.isnan(lse).all(), at
    t = tables.copy()
    t[17, 11], t[5, :11] = pages, pages                    # the shared pages are read through the first request's table
    with Device() as dev:
        got, lse, _, _ = run_attention(sts, dev, dtype, q, pool, t, lens, groups, 4)
    fine = [r for r in range(43) if r != 17]
    assert np.isnan(got[17]).all() and np.isnan(lse[17]).all()
    near(got[fine], out[fine], bound[fine])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("q_pad,out_pad,offset", [(0, 0, 2), (3, 5, 0), (8, 1, 0), (1, 0, 2)])
def test_shared_attention_wide_rows_at_any_element(sts, dtype, q_pad, out_pad, offset):
    q, k, v, tables, pages, lens, groups = small_case(np.random.default_rng(22), dtype, scale=3.0, **WIDE)
    pool = pool_of(k, v, tables, lens, pages, dtype, behind=np.nan)
    out, bound, lse, lb = attention_reference(q, k, v, lens, 4, 0.3, dtype)
    with Device() as dev:
        got, got_lse, _, _ = run_attention(sts, dev, dtype, q, pool, tables, lens, groups, 4, scale=0.3, q_pad=q_pad, out_pad=out_pad, q_offset=offset)
    near(got, out, bound)
    near(got_lse, lse, lb)


def test_shared_attention_wide_infinities(sts):
    """In the shared part: scores of -inf weigh nothing, ahead of every other one and in between; a V of inf reaches every output; a score of inf or NaN is NaN for the rows that it is one of."""
    q, k, v, tables, pages, lens, groups = small_case(np.random.default_rng(23), "bf16", **WIDE)
    q[:] = np.abs(q) + 0.25
    q[7, 2, 5] = np.nan
    low = [*range(64), 70, 175]                            # the first four pages, and some
    for r in range(43):
        k[r][low] = -3e38
        v[r][100, 1, 9], v[r][101, 1, 9], v[r][3, 0, 11], v[r][120, 1, 30] = np.inf, np.inf, 3e38, -np.inf
    pool = pool_of(k, v, tables, lens, pages, "bf16")
    with Device() as dev:
        got, lse, _, _ = run_attention(sts, dev, "bf16", q, pool, tables, lens, groups, 4)
        k_hot = [x.copy() for x in k]
        for x in k_hot:
            x[90, 1] = 3e38
        hot, _, _, _ = run_attention(sts, dev, "bf16", q, pool_of(k_hot, v, tables, lens, pages, "bf16"), tables, lens, groups, 4)
    assert np.isnan(got[7, 2]).all() and np.isnan(lse[7, 2])
    nan = np.zeros((43, 8), bool)
    nan[7, 2] = True
    assert np.isposinf(got[:, 4:, 9][~nan[:, 4:]]).all() and np.isneginf(got[:, 4:, 30][~nan[:, 4:]]).all()
    for r in range(43):
        keep = [t for t in range(lens[r]) if t not in low]
        o, b, _, _ = attention_reference(q[r:r + 1], [k[r][keep]], [np.where(np.isinf(v[r][keep]), 0, v[r][keep])], [len(keep)], 4, 0.125, "bf16")
        check = np.broadcast_to(~nan[r][:, None], (8, 64)).copy()
        check[4:, [9, 30]] = False
        near(got[r][check], o[0][check], b[0][check])
    assert np.isnan(hot[:, 4:]).all() and np.array_equal(np.isnan(hot[:, :4]).all(2), nan[:, :4])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("groups", [((43, 176),), ((3, 32), (4, 64))])
@pytest.mark.parametrize("power", [10, 18, 21])
def test_shared_attention_small_weights(sts, dtype, groups, power):
    """Tokens of 2^-power of the others' weight. They count, many of them for one other, and an infinite V of one reaches the output, wide and narrow."""
    lens = tuple(s + 40 for m, s in groups for _ in range(m))
    q, k, v, tables, pages, lens, groups = small_case(np.random.default_rng(24), dtype, lens, groups)
    small = rounded(-power * np.log(2.0) * 8 / 4, dtype)   # 4 k / 8: the score
    q[:] = 0
    q[:, :, 0] = 4
    for r in range(len(lens)):
        k[r][:, :, 0] = 0
        k[r][:, 0, 0] = small                              # of the first KV head all but the last token
        k[r][-1, 0, 0] = 0
        k[r][5, 1, 0] = small
        v[r][:-1, 0], v[r][-1, 0] = rounded(1024.0 + np.abs(v[r][:-1, 0]), dtype), 0
        v[r][5, 1, 9] = np.inf
    pool = pool_of(k, v, tables, lens, pages, dtype)
    with Device() as dev:
        got, lse, _, _ = run_attention(sts, dev, dtype, q, pool, tables, lens, groups, 4)
    assert np.isposinf(got[:, 4:, 9]).all() and np.isfinite(got[:, 4:, :9]).all() and np.isfinite(lse).all()
    # u for the output, of the weights 2 u (2 u + 2^-9), 2^-31 for fp16's last place, 2^-17 for exponentials of up to 22 and the sums
    u = HALF[dtype]
    for r in range(len(lens)):
        w = np.exp(k[r][:, 0, 0].astype(np.float64) * 0.5)
        out, size = w @ v[r][:, 0].astype(np.float64) / w.sum(), np.abs(v[r][:, 0]).astype(np.float64).sum(0)
        near(got[r, :4], np.tile(out, (4, 1)), np.tile((u + 2 * u * (2 * u + 2.0 ** -9) + 2.0 ** -17) * out + (2.0 ** -31 * size + 2.0 ** -25 if dtype == "f16" else 0.0), (4, 1)))


@pytest.mark.parametrize("dtype,n_q,n_kv,groups", [("bf16", 4, 2, [(2, 16)] * 2048), ("f16", 8, 1, [(4096, 48)]), ("bf16", 8, 1, [(9, 32)] * 455 + [(1, 0)]), ("f16", 2, 2, [(1, 0)] * 4096)])
def test_shared_attention_of_the_most_requests(sts, dtype, n_q, n_kv, groups):
    rng = np.random.default_rng(len(groups))
    lens = [int(x) for m, s in groups for x in s + rng.choice([0, 1, 1, 2, 15, 16, 17, 33], m)]
    assert len(lens) == 4096
    k, v, tables, pages = attention_case(rng, groups, lens, n_kv, 64)
    k, v = [rounded(x, dtype) for x in k], [rounded(x, dtype) for x in v]
    q = rounded(rng.standard_normal((4096, n_q, 64)), dtype)
    pool = pool_of(k, v, tables, lens, pages, dtype, behind=np.nan)
    out, bound, lse, lb = attention_reference(q, k, v, lens, n_q // n_kv, 0.125, dtype)
    with Device() as dev:
        got, got_lse, _, _ = run_attention(sts, dev, dtype, q, pool, tables, lens, groups, n_q // n_kv)
    some = np.asarray(lens) > 0
    near(got, out, bound)
    near(got_lse[some], lse[some], lb[some])
    assert np.isneginf(got_lse[~some]).all()


def test_shared_attention_same_bits_again_and_in_a_graph(sts):
    """Nothing depends on the order in which workgroups end: the same inputs give the same bits, eagerly, on another stream and replayed."""
    rng = np.random.default_rng(11)
    q, k, v, tables, pages, lens, groups = small_case(rng, "bf16", [300 + 7 * i for i in range(40)], [(25, 288), (15, 200)])
    pool = pool_of(k, v, tables, lens, pages, "bf16")
    with Device() as dev:
        first, lse0, _, _ = run_attention(sts, dev, "bf16", q, pool, tables, lens, groups, 4)
        s = dev.stream()
        again, lse1, call, (out, lse) = run_attention(sts, dev, "bf16", q, pool, tables, lens, groups, 4, stream=s)
        assert np.array_equal(first, again) and np.array_equal(lse0, lse1)
        replay = dev.graph(s, call)
        for _ in range(4):
            dev.write(out, np.full(again.size, 0x7FC0, np.uint16))
            dev.write(lse, np.full(lse0.size, np.nan, np.float32))
            replay()
            dev.sync()
            assert np.array_equal(dev.get(out, first.shape, "bf16"), first) and np.array_equal(dev.get(lse, lse0.shape, "f32"), lse0)


def test_shared_attention_without_a_plan_of_its_sizes_is_nan(sts):
    """A workspace that holds none, or one of other requests, heads or tables: nothing in it is followed."""
    rng = np.random.default_rng(22)
    n, heads, n_kv, d, pages = 70, 4, 2, 64, 40
    q = rng.standard_normal((n, heads * n_kv * d))
    with Device() as dev:
        size = sts.attn_shared_workspace(n, heads, 1, 2 * d)                 # the largest of those below
        dev_q, pool = dev.put(q, "bf16"), dev.put(rng.standard_normal((pages, n_kv, 2 * 16 * d)), "bf16")
        tables, lens = dev.ints(rng.integers(0, pages, (n, 6))), dev.ints(rng.integers(60, 90, n))
        starts, shared = dev.ints([0, n]), dev.ints([48])
        ws = dev.put(np.zeros(size, np.uint8))

        def batch(**change):
            good = dict(dtype=sts.DTYPES["bf16"], n_requests=n, n_groups=1, n_q=heads * n_kv, n_kv=n_kv, d=d, pool_pages=pages, max_pages=6, table_stride=6, tables=tables, lens=lens,
                        group_starts=starts, shared_lens=shared, workspace=ws, workspace_bytes=size)
            return sts.AttnBatch(**{**good, **change})

        width = heads * n_kv * d                             # elements of a row of q and out, whatever of them a batch has

        def layer(b):
            out, lse = dev.put(np.full((n, width), 7.0), "bf16"), dev.put(np.full((n, width // d), 7.0, np.float32))
            sts.op_attn_shared(b, dev_q, width, pool, out, width, lse)
            dev.sync()
            got = dev.get(out, (n, width), "bf16")
            assert (got[b.n_requests:] == 7.0).all() and (got[:, b.n_q * b.d:] == 7.0).all()
            return got[:b.n_requests, :b.n_q * b.d], dev.get(lse, n * width // d, "f32")[:b.n_requests * b.n_q]

        out, lse = layer(batch())
        assert np.isnan(out).all() and np.isnan(lse).all()
        sts.op_attn_shared_plan(batch())
        assert np.isfinite(layer(batch())[0]).all()
        other = dict(n_groups=0)
        for change in (dict(n_requests=n - 1, **other), dict(n_q=n_kv), dict(n_q=heads, n_kv=1), dict(n_q=heads, n_kv=1, d=2 * d), dict(max_pages=5)):
            out, lse = layer(batch(**change))
            assert np.isnan(out).all() and np.isnan(lse).all(), change
        assert np.isfinite(layer(batch())[0]).all()


def test_shared_attention_of_two_streams_at_once(sts):
    """Workspaces of their own: calls under way together do not see each other."""
    rng = np.random.default_rng(21)
    cases = [small_case(rng, "bf16", [600 + 5 * i for i in range(50)], [(30, 560), (20, 100)]), small_case(rng, "bf16", [90 + 11 * i for i in range(70)], [(70, 80)])]
    with Device() as dev:
        runs, want = [], []
        for q, k, v, tables, pages, lens, groups in cases:
            pool, s = pool_of(k, v, tables, lens, pages, "bf16"), dev.stream()
            out, lse, call, at = run_attention(sts, dev, "bf16", q, pool, tables, lens, groups, 4, stream=s)
            runs.append((call, at, out.shape))
            want.append(out)
        for _ in range(20):
            for call, _, _ in runs:
                call()
        dev.sync()
        for (_, (out, _), shape), w in zip(runs, want):
            assert np.array_equal(dev.get(out, shape, "bf16"), w)


def test_append_and_attention_behind_32_bits(sts):
    """A pool of more than 2^31 elements and 2^32 bytes: its last pages are written and read."""
    rng = np.random.default_rng(22)
    n_q, n_kv, d, pages, n, ctx = 16, 16, 128, 34000, 3, 40
    rope = sts.Rope(rotary_dim=d, theta=1e4)
    tables = np.array([[pages - 1, 5, pages - 2], [pages - 3, pages - 4, 0], [1, pages - 5, pages - 6]], np.int32)
    qkv = rounded(rng.standard_normal((n * ctx, 3 * n_q * d)), "bf16")
    positions = np.tile(np.arange(ctx), n)
    places = np.array([tables[r, t // 16] * 16 + t % 16 for r in range(n) for t in range(ctx)], np.int32)
    with Device() as dev:
        assert pages * n_kv * 32 * d > 2 ** 31
        pool, base, ld = dev.alloc(pages * n_kv * 32 * d * 2), dev.put(qkv, "bf16"), 3 * n_q * d
        q, out, lse, size = dev.alloc(n * ctx * n_q * d * 2), dev.alloc(n * n_q * d * 2), dev.alloc(n * n_q * 4), sts.attn_shared_workspace(n, n_q, n_kv, d)
        sts.op_rope(rope, sts.RopeRows(dtype=1, rows=n * ctx, n_q=n_q, n_kv=n_kv, d=d, pool_pages=pages, q=base, q_stride=ld, q_out=q, q_out_stride=n_q * d, k=base + n_q * d * 2, k_stride=ld,
                                       v=base + 2 * n_q * d * 2, v_stride=ld, pool=pool, positions=dev.ints(positions), places=dev.put(places)))
        batch = sts.AttnBatch(dtype=1, n_requests=n, n_q=n_q, n_kv=n_kv, d=d, pool_pages=pages, max_pages=3, table_stride=3, tables=dev.ints(tables), lens=dev.ints([ctx] * n),
                              workspace=dev.alloc(size), workspace_bytes=size)
        sts.op_attn_shared_plan(batch)
        sts.op_attn_shared(batch, q + (ctx - 1) * n_q * d * 2, ctx * n_q * d, pool, out, n_q * d, lse)
        dev.sync()
        got_q, got = dev.get(q, (n, ctx, n_q, d), "bf16")[:, -1], dev.get(out, (n, n_q, d), "bf16")
        page = np.stack([[dev.get(pool + int(p) * n_kv * 32 * d * 2, (n_kv, 32 * d), "bf16") for p in row] for row in tables])
    x = qkv.reshape(n, ctx, 3 * n_q, d)
    k = page[..., :16 * d].reshape(n, 3, n_kv, 16, d).transpose(0, 1, 3, 2, 4).reshape(n, 48, n_kv, d)[:, :ctx]
    v = page[..., 16 * d:].reshape(n, 3, n_kv, d, 16).transpose(0, 1, 4, 2, 3).reshape(n, 48, n_kv, d)[:, :ctx]
    assert np.array_equal(v, x[:, :, 2 * n_q:])
    for r in range(n):
        want, size = rope_reference(sts, rope, x[r, :, n_q:2 * n_q].astype(np.float64), positions[:ctx])
        near(k[r], want, rope_bound(want, size, "bf16"))
    want, bound, _, _ = attention_reference(got_q, k, v, [ctx] * n, 1, d ** -0.5, "bf16")
    near(got, want, bound)


# ------------------------------------------------------------------------------------------ log probabilities
def logprobs_reference(x, tokens, k):
    """x [rows, vocab] float64 of values in the type."""
    with np.errstate(all="ignore"):
        rows, vocab = x.shape
        whole = np.where(np.isnan(x) | np.isposinf(x), True, False).any(1)
        none = np.isneginf(x).all(1)
        m = np.where(none | whole, 0.0, np.where(whole[:, None], 0.0, x).max(1))
        p = np.exp(x - m[:, None])
        z = p.sum(1)
        ref = m + np.log(z)
        entropy = np.log(z) - np.where(p > 0, p * (x - m[:, None]), 0.0).sum(1) / z
        order = np.where(np.isnan(x), -np.inf, x)
        top = np.stack([np.lexsort((np.arange(vocab), -row))[:k] for row in order]) if k else np.zeros((rows, 0), int)
        ok = (tokens >= 0) & (tokens < vocab)
        t = np.where(ok, tokens, 0)
        xt = x[np.arange(rows), t]
        lp = (xt - m) - np.log(z)
        tlp = (np.take_along_axis(x, top, 1) - m[:, None]) - np.log(z)[:, None]
        rank = np.array([(order[r] > xt[r]).sum() + ((order[r] == xt[r]) & (np.arange(vocab) < t[r])).sum() for r in range(rows)])
        rank = np.where(ok & ~np.isnan(xt), rank, -1)
        lp, tlp, ref, entropy = np.where(none, -np.inf, lp), np.where(none[:, None], -np.inf, tlp), np.where(none, -np.inf, ref), np.where(none, 0.0, entropy)
        lp, ref, entropy = (np.where(whole, np.nan, y) for y in (lp, ref, entropy))
        tlp = np.where(whole[:, None], np.nan, tlp)
        return dict(logprob=np.where(ok, lp, np.nan), entropy=entropy, lse=ref, rank=rank, top_logprob=tlp, top_token=top)


def run_logprobs(sts, dev, dtype, x, tokens, k, pad=0, offset=0, stream=None):
    rows, vocab = x.shape
    wide = np.full((rows, vocab + pad), 1e4 if dtype == "f16" else 1e30, np.float32)       # what lies behind a row must not matter
    wide[:, :vocab] = x
    buf = dev.put(np.concatenate([np.full(8, 1e4, np.float32), wide.reshape(-1), np.full(8, 1e4, np.float32)]), dtype, offset)
    size = sts.op_logprobs_workspace(sts.DTYPES[dtype], rows, vocab, k)
    o = dict(logprob=(rows,), entropy=(rows,), lse=(rows,), rank=(rows,), top_logprob=(rows, k), top_token=(rows, k))
    kind = dict(rank="i32", top_token="i32")
    p = {n: dev.put(np.full(s, 777, np.int32 if n in kind else np.float32)) for n, s in o.items()}
    item = 4 if dtype == "f32" else 2
    a = sts.Logprobs(dtype=sts.DTYPES[dtype], rows=rows, vocab=vocab, top_k=k, row_stride=vocab + pad, logits=buf + 8 * item, tokens=dev.ints(tokens), workspace=dev.alloc(size),
                     workspace_bytes=size, **{n: v for n, v in p.items() if k or not n.startswith("top")})
    call = lambda: sts.op_logprobs(a, stream)  # noqa: E731
    call()
    dev.sync()
    read = lambda: {n: dev.get(p[n], s, kind.get(n, "f32")) for n, s in o.items()}  # noqa: E731
    return read(), call, read, p


def check_logprobs(got, want, vocab):
    """fp32 sums of a lane's share of the row (at most vocab / 256 + 64 elements) and some 40 roundings of the exponents and joins: relative in Z, absolute in its logarithm. The
    entropy's weighted sum is off by as much of itself (at most entropy + 1, in nats) again."""
    e = (vocab / 256 + 104) * 2.0 ** -24
    assert np.array_equal(got["rank"], want["rank"]) and np.array_equal(got["top_token"], want["top_token"])
    for n in ("logprob", "lse", "top_logprob", "entropy"):
        g, w = got[n].astype(np.float64), want[n]
        assert np.array_equal(np.isnan(g), np.isnan(w)), n
        fine = np.isfinite(w)
        assert np.array_equal(g[~fine & ~np.isnan(w)], w[~fine & ~np.isnan(w)]), n
        bound = e * (3 + 2 * np.abs(w)) if n == "entropy" else e + 2.0 ** -23 * np.abs(w)
        near(g[fine], w[fine], bound[fine])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab,k,pad,offset", [(1, 1, 1, 0, 0), (3, 5, 5, 0, 0), (2, 64, 32, 1, 0), (7, 1000, 20, 0, 0), (5, 4097, 8, 3, 4), (2, 32001, 32, 0, 0), (1, 128256, 20, 0, 0),
                                                     (33, 50257, 5, 0, 12), (300, 1024, 1, 0, 0), (1100, 777, 0, 0, 0), (1500, 4100, 3, 0, 0), (4, 300000, 32, 1, 0)])
def test_logprobs(sts, dtype, rows, vocab, k, pad, offset):
    rng = np.random.default_rng(vocab + rows)
    x = rounded(3.0 * rng.standard_normal((rows, vocab)), dtype)
    tokens = rng.integers(0, vocab, rows)
    tokens[::3] = x[::3].argmax(1)
    if rows > 2:
        tokens[1], tokens[2] = -1, vocab
    with Device() as dev:
        got, _, _, _ = run_logprobs(sts, dev, dtype, x, tokens, k, pad, offset)
    check_logprobs(got, logprobs_reference(x.astype(np.float64), tokens, k), vocab)


def masks(rng, vocab, dtype):
    """Rows that a mask or a broken model leaves: name, logits, token."""
    lowest = {"f32": -3.4028234663852886e38, "bf16": -3.3895313892515355e38, "f16": -65504.0}[dtype]
    x = rounded(3.0 * rng.standard_normal(vocab), dtype)
    half, inf = rng.random(vocab) < 0.5, np.float32(np.inf)
    one = np.full(vocab, -inf, np.float32)
    one[vocab // 2] = 2.5
    yield "half -inf", np.where(half, -inf, x), int(np.flatnonzero(~half)[0])
    yield "a token of -inf", np.where(half, -inf, x), int(np.flatnonzero(half)[-1])
    yield "half the lowest value", np.where(half, np.float32(lowest), x), int(np.flatnonzero(half)[3])
    yield "one token left", one, vocab // 2
    yield "one token left, another given", one, vocab - 1
    yield "nothing left", np.full(vocab, -inf, np.float32), 3
    yield "all the lowest value", np.full(vocab, lowest, np.float32), 5
    yield "the lowest value, then logits", np.where(np.arange(vocab) < vocab - vocab // 3, np.float32(lowest), x), vocab - 2
    yield "logits, then the lowest value", np.where(np.arange(vocab) > vocab // 3, np.float32(lowest), x), 2
    yield "-inf, then logits", np.where(np.arange(vocab) < vocab - vocab // 3, -inf, x), vocab - 2
    yield "lowest and -inf", np.where(half, -inf, np.float32(lowest)), int(np.flatnonzero(~half)[1])
    yield "all equal", np.full(vocab, 1.5, np.float32), vocab - 1
    yield "zeros of both signs", np.where(half, np.float32(0.0), np.float32(-0.0)), vocab // 3
    yield "ascending", np.sort(x), vocab // 4
    yield "descending", np.sort(x)[::-1].copy(), vocab // 4
    yield "few values", np.round(x), int(np.round(x).argmax())
    nan, pos = x.copy(), x.copy()
    nan[[4, vocab - 2]] = np.nan
    pos[7] = inf
    yield "NaN", nan, 9
    yield "the token NaN", nan, 4
    yield "inf", pos, 9
    yield "large", rounded(x * {"f32": 1e36, "bf16": 1e36, "f16": 5000.0}[dtype], dtype), 11


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab,k,rows", [(1003, 32, 1), (40001, 20, 1), (9001, 5, 90)])
def test_logprobs_of_masked_and_odd_rows(sts, dtype, vocab, k, rows):
    """rows: copies of each, so that rows come whole to one workgroup or in parts."""
    names, x, tokens = zip(*masks(np.random.default_rng(vocab), vocab, dtype))
    x, tokens = np.repeat(np.stack(x), rows, 0), np.repeat(np.asarray(tokens), rows)
    with Device() as dev:
        got, _, _, _ = run_logprobs(sts, dev, dtype, x, tokens, k)
    first = logprobs_reference(x[::rows].astype(np.float64), tokens[::rows], k)
    for i, name in enumerate(names):
        want = {n: np.repeat(v[i:i + 1], rows, 0) for n, v in first.items()}
        try:
            check_logprobs({n: v[i * rows:(i + 1) * rows] for n, v in got.items()}, want, vocab)
        except AssertionError as e:
            raise AssertionError(name) from e


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab,k,pad,offset", [(1, 1100003, 32, 0, 0), (2, 1700001, 1, 1, 4), (1, 2300000, 20, 0, 0), (3, 1200007, 0, 0, 0), (1, 4400001, 5, 0, 12)])
def test_logprobs_of_long_parts(sts, dtype, rows, vocab, k, pad, offset):
    """Parts of a row above 65536 elements: a lane's groups hold several batches, the last one fewer."""
    test_logprobs(sts, dtype, rows, vocab, k, pad, offset)


@pytest.mark.parametrize("dtype,vocab,k,rows", [("bf16", 70001, 32, 52), ("f32", 70001, 1, 52), ("bf16", 128256, 1, 52), ("f16", 128256, 32, 52), ("f32", 1100001, 20, 1), ("bf16", 1500001, 32, 1)])
def test_logprobs_of_masked_and_odd_long_rows(sts, dtype, vocab, k, rows):
    """The same of masked rows, in parts and (1040 rows) whole."""
    test_logprobs_of_masked_and_odd_rows(sts, dtype, vocab, k, rows)


def test_logprobs_same_bits_again_and_in_a_graph(sts):
    rng = np.random.default_rng(1)
    x = rounded(3.0 * rng.standard_normal((5, 70001)), "bf16")
    tokens = rng.integers(0, 70001, 5)
    with Device() as dev:
        first, _, _, _ = run_logprobs(sts, dev, "bf16", x, tokens, 20)
        s = dev.stream()
        again, call, read, p = run_logprobs(sts, dev, "bf16", x, tokens, 20, stream=s)
        replay = dev.graph(s, call)
        for n in first:
            assert np.array_equal(first[n], again[n])
        for _ in range(4):
            for n, v in first.items():
                dev.write(p[n], np.zeros_like(v))
            replay()
            dev.sync()
            got = read()
            for n in first:
                assert np.array_equal(first[n], got[n]), n


# ------------------------------------------------------------------------------------------ together
def test_a_step_of_all_operators_eager_and_replayed(sts):
    """Three prompts, sampled five, one and three ways: prompts placed and appended, then steps of one token each -- places, rotation and append, attention over the
    shared prompts, logits (the library's GEMM), log probabilities -- eagerly and as a graph of two steps that hand lengths and free pages to each other on the device."""
    rng = np.random.default_rng(77)
    n_q, n_kv, d, vocab, dtype = 8, 2, 64, 512, "bf16"
    members, prompts = [5, 1, 3], [70, 33, 100]
    n, width, pages, heads, ld = sum(members), 12, 90, n_q // n_kv, (n_q + 2 * n_kv) * d
    owner = np.repeat(np.arange(3), members)
    shared = [p // 16 * 16 for p in prompts]
    rope = sts.Rope(rotary_dim=d, scaling=sts.ROPE_SCALINGS["bands"], theta=1e4, factor=4.0, low=1.0, high=4.0, original_len=64)
    with Device() as dev:
        s = dev.stream()
        pool, tables = dev.put(np.zeros((pages, n_kv, 32 * d), np.uint16)), dev.ints(np.full((n, width), -1))
        free = rng.permutation(pages).astype(np.int32)
        w = rounded(rng.standard_normal((vocab, n_q * d)) / 8, dtype)
        free_dev, w_dev = dev.put(free), dev.put(w, dtype)
        count, lens, starts, status = [dev.ints([pages]), dev.ints([0])], [dev.ints([0] * n), dev.ints([0] * n)], dev.ints([0] * (n + 1)), dev.ints([9])
        rows_max = sum(p for p in prompts) + n * 100
        requests, positions, places = (dev.ints([0] * rows_max) for _ in range(3))

        def place(added, rows, a, b):
            sts.op_block_tables(sts.BlockTables(n_requests=n, max_pages=width, max_rows=rows, free_capacity=pages, table_stride=width, cached=lens[a], added=added, free_pages=free_dev,
                                                n_free=count[a], tables=tables, lens=lens[b], row_starts=starts, requests=requests, positions=positions, places=places,
                                                n_free_left=count[b], status=status), s)

        def append(qkv, rows, q_out):
            sts.op_rope(rope, sts.RopeRows(dtype=1, rows=rows, n_q=n_q, n_kv=n_kv, d=d, pool_pages=pages, q=qkv, q_stride=ld, q_out=q_out, q_out_stride=n_q * d, k=qkv + n_q * d * 2,
                                           k_stride=ld, v=qkv + (n_q + n_kv) * d * 2, v_stride=ld, pool=pool, positions=positions, places=places), s)

        # the prompts, by the first of each group; the whole pages go to the others' tables, which then get their own copy of the rest
        first = [int(np.argmax(owner == g)) for g in range(3)]
        added = np.zeros(n, np.int32)
        added[first] = prompts
        qkv_prompt = rounded(rng.standard_normal((sum(prompts), ld)), dtype)
        place(dev.ints(added), sum(prompts), 0, 1)
        append(dev.put(qkv_prompt, dtype), sum(prompts), dev.alloc(sum(prompts) * n_q * d * 2))
        dev.sync()
        assert dev.get(status, 1, "i32")[0] == 0
        t = dev.get(tables, (n, width), "i32")
        for r in range(n):
            t[r, :shared[owner[r]] // 16] = t[first[owner[r]], :shared[owner[r]] // 16]
        rest = np.array([0 if r in first else prompts[owner[r]] - shared[owner[r]] for r in range(n)], np.int32)
        offsets = np.concatenate([[0], np.cumsum(prompts)])
        qkv_rest = np.concatenate([qkv_prompt[offsets[owner[r]] + shared[owner[r]]:offsets[owner[r] + 1]] for r in range(n) if rest[r]])
        dev.write(tables, t)
        dev.write(lens[1], np.array([prompts[owner[r]] - rest[r] for r in range(n)], np.int32))
        place(dev.ints(rest), len(qkv_rest), 1, 0)
        append(dev.put(qkv_rest, dtype), len(qkv_rest), dev.alloc(len(qkv_rest) * n_q * d * 2))
        dev.sync()
        assert dev.get(status, 1, "i32")[0] == 0
        assert np.array_equal(dev.get(lens[0], n, "i32"), [prompts[g] for g in owner])

        # steps
        size = sts.attn_shared_workspace(n, n_q, n_kv, d)
        ones, qkv, q, out, lse = dev.ints([1] * n), dev.alloc(n * ld * 2), dev.alloc(n * n_q * d * 2), dev.alloc(n * n_q * d * 2), dev.alloc(n * n_q * 4)
        groups, shared_dev, ws, logits = dev.ints(np.concatenate([[0], np.cumsum(members)])), dev.ints(shared), dev.alloc(size), dev.alloc(n * vocab * 4)
        tokens = dev.ints(rng.integers(0, vocab, n))
        o = {k: dev.alloc(n * 4 * m) for k, m in (("logprob", 1), ("entropy", 1), ("lse", 1), ("rank", 1), ("top_logprob", 4), ("top_token", 4))}

        def step(a, b):
            place(ones, n, a, b)
            append(qkv, n, q)
            batch = sts.AttnBatch(dtype=1, n_requests=n, n_groups=3, n_q=n_q, n_kv=n_kv, d=d, pool_pages=pages, max_pages=width, table_stride=width, tables=tables, lens=lens[b],
                                  group_starts=groups, shared_lens=shared_dev, workspace=ws, workspace_bytes=size)
            sts.op_attn_shared_plan(batch, s)
            sts.op_attn_shared(batch, q, n_q * d, pool, out, n_q * d, lse, 0.0, s)
            sts.op_gemm_noalloc(out, w_dev, logits, n, vocab, n_q * d, "64x128", 1, 0, s)
            sts.op_logprobs(sts.Logprobs(dtype=0, rows=n, vocab=vocab, top_k=4, row_stride=vocab, logits=logits, tokens=tokens, **o), s)

        def check(done, x):
            length = [prompts[g] + done for g in owner]
            assert dev.get(status, 1, "i32")[0] == 0 and np.array_equal(dev.get(lens[done % 2], n, "i32"), length)
            p, t = dev.get(pool, (pages, n_kv, 32 * d), dtype), dev.get(tables, (n, width), "i32")
            own = [x for r in range(n) for x in t[r, shared[owner[r]] // 16:-(-length[r] // 16)]]
            assert len(set(own)) == len(own) and dev.get(count[done % 2], 1, "i32")[0] == pages - len(own) - sum(shared) // 16
            k = [p[t[r, :-(-length[r] // 16)], :, :16 * d].reshape(-1, n_kv, 16, d).transpose(0, 2, 1, 3).reshape(-1, n_kv, d)[:length[r]] for r in range(n)]
            v = [p[t[r, :-(-length[r] // 16)], :, 16 * d:].reshape(-1, n_kv, d, 16).transpose(0, 3, 1, 2).reshape(-1, n_kv, d)[:length[r]] for r in range(n)]
            rows = x.reshape(n, n_q + 2 * n_kv, d).astype(np.float64)
            got_q = dev.get(q, (n, n_q, d), dtype)
            for y, part in ((got_q, rows[:, :n_q]), (np.stack([kr[-1] for kr in k]), rows[:, n_q:n_q + n_kv])):
                want, sz = rope_reference(sts, rope, part, np.array(length) - 1)
                near(y, want, rope_bound(want, sz, dtype))
            assert np.array_equal(np.stack([vr[-1] for vr in v]), rows[:, n_q + n_kv:])
            want, bound, want_lse, lb = attention_reference(got_q, k, v, length, heads, d ** -0.5, dtype)
            got = dev.get(out, (n, n_q, d), dtype)
            near(got, want, bound)
            near(dev.get(lse, (n, n_q), "f32"), want_lse, lb)
            z = dev.get(logits, (n, vocab), "f32")
            near(z, got.reshape(n, -1).astype(np.float64) @ w.T, n_q * d * 2.0 ** -23 * np.abs(got.reshape(n, -1)) @ np.abs(w.T) + 1e-6)
            kinds = dict(rank="i32", top_token="i32")
            shape = {k_: (n, 4) if k_.startswith("top") else (n,) for k_ in o}
            check_logprobs({k_: dev.get(o[k_], shape[k_], kinds.get(k_, "f32")) for k_ in o}, logprobs_reference(z.astype(np.float64), dev.get(tokens, n, "i32"), 4), vocab)

        x = rounded(rng.standard_normal((n, ld)), dtype)
        for i in range(2):
            x = rounded(rng.standard_normal((n, ld)), dtype)
            dev.write(qkv, stored_bf16(x))
            step(i, 1 - i)
            dev.sync()
            check(i + 1, x)
        replay = dev.graph(s, lambda: (step(0, 1), step(1, 0)))
        for i in range(9):                                 # over several page borders; both steps of a replay append the same rows
            x = rounded(rng.standard_normal((n, ld)), dtype)
            dev.write(qkv, stored_bf16(x))
            replay()
            dev.sync()
            check(2 * i + 4, x)


def stored_bf16(x):
    return (np.asarray(x, np.float32).view(np.uint32) >> 16).astype(np.uint16)


# ------------------------------------------------------------------------------------------ in the engine
@pytest.fixture(scope="module")
def engine(sts):
    from paper_2504_19516_amd import synth
    desc = synth.tiny_model("fp32")
    e = sts.Engine(desc, weight_seed=5, kv_pool_pages=300, max_prefill_tokens=256, max_prefill_seqs=4, max_decode_batch=40, max_seqs=48, max_pages_per_seq=20)
    yield e, desc
    e.close()


def test_engine_reads_log_probabilities_of_its_last_call(sts, engine):
    """Of logits that the call returned, of logits that only made tokens, of a prefill's; a call that made none leaves none."""
    from paper_2504_19516_amd import synth
    e, desc = engine
    seqs = [e.seq_create() for _ in range(33)]
    prompts = [synth.tokens(40 + i, 5 + 3 * i, desc.vocab) for i in range(3)]
    rng = np.random.default_rng(3)

    def check(phase, logits, tokens, k):
        got = e.read_logprobs(phase, tokens, k)
        want = logprobs_reference(logits.astype(np.float64), np.asarray(tokens), k)
        check_logprobs(dict(got, lse=want["lse"].astype(np.float32)), want, desc.vocab)

    logits = e.prefill_batch(seqs[:3], prompts)
    check(0, logits, [7, desc.vocab - 1, -1], 5)
    check(0, logits[:2], [1, 2], 32)                       # the first rows
    for s in seqs[3:]:
        e.prefill_append(s, prompts[0], want_logits=False)
    for code, call in ((sts.EINVAL, lambda: e.read_logprobs(0, [1])), (sts.EINVAL, lambda: e.read_logprobs(1, [1]))):      # that call made none; no decode step yet
        with pytest.raises(sts.StsError) as x:
            call()
        assert x.value.code == code
    tokens = rng.integers(0, desc.vocab, 33)
    for n, with_logits, with_next in ((33, True, True), (33, True, False), (1, True, True)):
        logits, nxt = e.decode_step(seqs[:n], tokens[:n], want_logits=with_logits, want_next=with_next)
        check(1, logits, rng.integers(0, desc.vocab, n), 8)
    _, nxt = e.decode_step(seqs, tokens, want_logits=False)
    got = e.read_logprobs(1, nxt, 1)
    assert (got["rank"] == 0).all() and np.array_equal(got["top_token"][:, 0], nxt) and np.array_equal(got["top_logprob"][:, 0], got["logprob"])
    for bad in (dict(phase=2, tokens=[1]), dict(phase=1, tokens=[1] * 34), dict(phase=1, tokens=[]), dict(phase=1, tokens=[1], top_k=33), dict(phase=1, tokens=[1], top_k=-1)):
        with pytest.raises((sts.StsError, ValueError)) as x:
            e.read_logprobs(**bad)
        assert getattr(x.value, "code", sts.EINVAL) == sts.EINVAL
    e.decode_launch(seqs[:4], tokens[:4])
    with pytest.raises(sts.StsError) as x:
        e.read_logprobs(1, [1])
    assert x.value.code == sts.ESTATE
    e.decode_finish(4)
    e.decode_step(seqs, tokens, want_logits=False, want_next=False)
    with pytest.raises(sts.StsError) as x:
        e.read_logprobs(1, [1])
    assert x.value.code == sts.EINVAL
    for s in seqs:
        e.seq_free(s)


def test_engine_reads_log_probabilities_of_both_phases_of_a_step(sts, engine):
    """Each phase's own, before and after the partition changes."""
    from paper_2504_19516_amd import synth
    e, desc = engine
    seqs = [e.seq_create() for _ in range(7)]
    prompts = [synth.tokens(60 + i, 9 + 2 * i, desc.vocab) for i in range(7)]
    e.prefill_batch(seqs[2:6], prompts[2:6])
    e.prefill_append(seqs[6], prompts[6])
    try:
        e.set_partition(128, 128)
        plog, dlog, _ = e.step_concurrent(seqs[:2], prompts[:2], 0, desc.n_layers, seqs[2:], [3, 4, 5, 6, 7])
        for split in (None, (192, 64)):
            if split:
                e.set_partition(*split)
            for phase, logits in ((0, plog), (1, dlog)):
                tokens = np.arange(len(logits)) * 11 + 1
                got, want = e.read_logprobs(phase, tokens, 3), logprobs_reference(logits.astype(np.float64), tokens, 3)
                check_logprobs(dict(got, lse=want["lse"].astype(np.float32)), want, desc.vocab)
    finally:
        e.set_partition(256, 256)
    for s in seqs:
        e.seq_free(s)


@pytest.mark.parametrize("phase,after", [(1, 0), (1, 9), (0, 0), (0, 9)])
def test_engine_has_no_log_probabilities_of_a_failed_step(sts, engine, phase, after):
    """A launch of either phase fails: neither phase has logits then, though the other one's may be queued to its end; the next step's are read as ever. A refused call
    changes nothing."""
    from paper_2504_19516_amd import synth
    e, desc = engine
    seqs = [e.seq_create() for _ in range(5)]
    prompts = [synth.tokens(80 + i, 7 + i, desc.vocab) for i in range(5)]

    def check(p, logits):
        tokens = np.arange(len(logits)) * 7 + 3
        got, want = e.read_logprobs(p, tokens, 3), logprobs_reference(logits.astype(np.float64), tokens, 3)
        check_logprobs(dict(got, lse=want["lse"].astype(np.float32)), want, desc.vocab)

    def none(p):
        with pytest.raises(sts.StsError) as x:
            e.read_logprobs(p, [1])
        assert x.value.code == sts.EINVAL
    check(0, e.prefill_batch(seqs[2:], prompts[2:]))
    first = e.decode_step(seqs[2:], [3, 4, 5])[0]
    check(1, first)
    step = lambda: e.step_concurrent(seqs[:2], prompts[:2], 0, desc.n_layers, seqs[2:], [6, 7, 8])  # noqa: E731
    e.fail_launch(phase, after)
    with pytest.raises(sts.StsError) as x:
        step()
    assert x.value.code == sts.EHIP
    none(0), none(1)
    plog, dlog, _ = step()
    check(0, plog), check(1, dlog)
    # a phase by itself: the other keeps its own
    e.fail_launch(phase, 2)
    with pytest.raises(sts.StsError):
        e.prefill_append(seqs[0], prompts[0]) if phase == 0 else e.decode_step(seqs[2:], [1, 2, 3])
    none(phase)
    check(1 - phase, dlog if phase == 0 else plog)
    # launched and finished; logits only once it is finished; a call that is refused leaves them
    if phase == 0:
        e.prefill_launch(seqs[:1], prompts[:1], 0, desc.n_layers, True)
        logits = e.prefill_finish(1, True)
    else:
        e.decode_launch(seqs[2:], [1, 2, 3], want_logits=True)
        logits, _ = e.decode_finish(3, True)
    check(phase, logits)
    with pytest.raises(sts.StsError):
        e.prefill_append(seqs[0], [desc.vocab]) if phase == 0 else e.decode_step(seqs[2:], [1, 2, desc.vocab])
    check(phase, logits)
    for s in seqs:
        e.seq_free(s)


def test_engine_reads_log_probabilities_without_allocating(sts, engine):
    """Everything is allocated by sts_init: a ctx's first call of either phase maps no memory of the GPU driver's (pinned host memory is such a mapping), though
    it is one of as many rows and alternatives as there can be."""
    from paper_2504_19516_amd import synth
    first, desc = engine
    s = first.seq_create()
    first.prefill_append(s, [1, 2, 3])
    first.read_logprobs(0, [1], 32)                        # the kernels' code has been loaded
    first.seq_free(s)

    def mapped():
        return sorted(x.split()[0] for x in open("/proc/self/maps") if "/dev/dri" in x or "/dev/kfd" in x)
    e = sts.Engine(desc, weight_seed=5, kv_pool_pages=300, max_prefill_tokens=256, max_prefill_seqs=40, max_decode_batch=300, max_seqs=300, max_pages_per_seq=4)
    seqs = [e.seq_create() for _ in range(300)]
    assert mapped()
    for i in range(0, 300, 40):
        part = seqs[i:i + 40]
        logits = e.prefill_batch(part, [synth.tokens(i + j, 3, desc.vocab) for j in range(len(part))])
        if i == 0:
            before = mapped()
            got = e.read_logprobs(0, logits.argmax(1), 32)
            assert mapped() == before and (got["rank"] == 0).all()
    _, nxt = e.decode_step(seqs, np.arange(300), want_logits=False)
    before = mapped()
    got = e.read_logprobs(1, nxt, 32)
    assert mapped() == before and (got["rank"] == 0).all()
    e.close()


def test_engine_takes_scaled_rotations(sts, engine):
    """K of a prompt as the engine caches it: the plain rotation's bits come back with the plain description; scaled ones are the plain K turned on by the difference of the
    angles (both rounded to bf16 once: 2 half steps of the size of the pair)."""
    from paper_2504_19516_amd import synth
    e, desc = engine
    prompt, d = synth.tokens(9, 200, desc.vocab), desc.head_dim
    plain = sts.Rope(rotary_dim=d, theta=desc.rope_theta)

    def keys():
        s = e.seq_create()
        logits = e.prefill_append(s, prompt)
        k, _ = e.kv_read(0, s, 0, 200)
        e.seq_free(s)
        return k.astype(np.float64), logits

    before, first = keys()
    for change in (dict(scaling=1, factor=4.0), dict(scaling=2, factor=8.0), dict(scaling=3, factor=8.0, low=1.0, high=4.0, original_len=256), dict(scaling=4, factor=8.0, low=1.0, high=32.0,
                                                                                                                                                    original_len=256)):
        rope = sts.Rope(rotary_dim=d, theta=desc.rope_theta, **change)
        e.set_rope(rope)
        got, logits = keys()
        a = np.arange(200)[:, None, None] * (sts.rope_frequencies(rope) - sts.rope_frequencies(plain))
        p, q = before[..., :d // 2], before[..., d // 2:]
        want = np.concatenate([p * np.cos(a) - q * np.sin(a), q * np.cos(a) + p * np.sin(a)], axis=-1)
        size = np.tile(np.abs(p) + np.abs(q), 2)
        near(got, want, 2.0 ** -8 * (size + np.abs(want)) + 1e-6)
        assert np.abs(got - before).max() > 0.1 and not np.array_equal(logits, first)
    e.set_rope(plain)
    after, last = keys()
    assert np.array_equal(after, before) and np.array_equal(last, first)
    for bad in (dict(rotary_dim=d // 2), dict(interleaved=1), dict(magnitude=1.3), dict(theta=0.0), dict(scaling=9)):
        with pytest.raises(sts.StsError) as x:
            e.set_rope(sts.Rope(**{**dict(rotary_dim=d, theta=1e4), **bad}))
        assert x.value.code == sts.EINVAL
    s = e.seq_create()
    e.prefill_append(s, prompt, 0, 1, want_logits=False)
    with pytest.raises(sts.StsError) as x:
        e.set_rope(plain)
    assert x.value.code == sts.ESTATE
    e.prefill_abort()
    e.seq_free(s)
