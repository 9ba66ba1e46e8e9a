"""Operators of a decode step that answers one prompt many times, as cases to measure: block tables and places of new rows
from request lengths, rotary positions with the append of K and V to their pages, attention over a prefix that requests share,
and log probabilities of given tokens with their alternatives. They work on device data, through
`paper_2504_19516_amd.sts` (the plain forms below need torch alone).

The KV cache is the library's: one layer's pool is [page][kv head][K: 16 tokens x d | V^T: d x 16 tokens], a request's tokens
16 t .. 16 t + 15 lie in page table[t]. Shapes: the model shapes of `paper_2504_19516_amd.synth` (heads 32/8 and 64/8 of 128
elements, 4/4 of 64, vocabulary 128256).
"""
import math
import random

import torch

own = False

PAGE = 16
SHAPES = {"tiny": (4, 4, 64, 1.0e4), "8b": (32, 8, 128, 5.0e5), "70b": (64, 8, 128, 5.0e5)}      # query heads, kv heads, head size, rope base
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
KINDS = {"plain": 0, "linear": 1, "base": 2, "bands": 3, "ramp": 4}                             # how the angles are scaled for long contexts


# ------------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # ---- block tables: a decode step of a conversational batch, one token each, every 16th needs a page
        dict(name="tables_decode_256", op="tables", prompts=0, tokens=0, decodes=256, ctx=700),
        # a mixed step: waiting prompts of 8192 tokens in all beside 200 decodes
        dict(name="tables_mixed", op="tables", prompts=7, tokens=8192, decodes=201, ctx=1100),
        # ---- rotary positions and append: the new tokens of a decode batch
        dict(name="rope_decode_64", op="rope", shape="8b", dtype="bf16", rows=64, prompts=0, interleaved=False, rotary=128, scaling="plain", far=4096),
        # a prefill batch of ragged prompts, far positions of a context stretched by wavelength
        dict(name="rope_prefill_8192", op="rope", shape="8b", dtype="bf16", rows=8192, prompts=6, interleaved=False, rotary=128, scaling="bands", far=120000),
        # an odd chunk of a model that turns half of each head in neighbouring pairs, 16-bit floats
        dict(name="rope_partial_1201", op="rope", shape="tiny", dtype="f16", rows=1201, prompts=3, interleaved=True, rotary=32, scaling="ramp", far=30000),
        # ---- attention: eight samples of one prompt, their own tokens just begun
        dict(name="attn_8_samples", op="attention", shape="8b", dtype="bf16", groups="8", shared="1031", suffix=60, spread=0.8, layers=4),
        # 64 users behind one system prompt
        dict(name="attn_64_users", op="attention", shape="8b", dtype="bf16", groups="64", shared="2048", suffix=300, spread=0.8, layers=4),
        # 256 questions on one long document
        dict(name="attn_256_document", op="attention", shape="8b", dtype="bf16", groups="256", shared="8192", suffix=120, spread=0.5, layers=2),
        # several prompts with different numbers of samples, one alone, on the larger shape
        dict(name="attn_groups_70b", op="attention", shape="70b", dtype="f16", groups="9,1,4,3,7", shared="3001,0,777,5120,1500", suffix=200, spread=0.8, layers=2),
        # ---- log probabilities: one user's token with its alternatives
        dict(name="logprobs_1", op="logprobs", dtype="f32", rows=1, vocab=128256, top=20, masked=0.0),
        # a decode batch, as the LM head leaves it
        dict(name="logprobs_64", op="logprobs", dtype="f32", rows=64, vocab=128256, top=5, masked=0.0),
        # scoring a document's tokens; part of the rows under a grammar that rules tokens out
        dict(name="logprobs_2048", op="logprobs", dtype="bf16", rows=2048, vocab=128256, top=1, masked=0.1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tables", "rope", "rope", "attention", "attention", "attention", "logprobs", "logprobs"])
    if op == "tables":
        prompts = rng.choice([0, 0, rng.randint(1, 16)])
        return dict(op=op, prompts=prompts, tokens=_log_int(rng, 64, 32768) if prompts else 0, decodes=_log_int(rng, 1, 2000), ctx=_log_int(rng, 16, 8000))
    if op == "rope":
        shape = rng.choice(["tiny", "8b", "8b", "70b"])
        d = SHAPES[shape][2]
        rows = _log_int(rng, 1, 8192 if shape != "70b" else 4096)
        return dict(op=op, shape=shape, dtype=rng.choice(["bf16", "bf16", "f16"]), rows=rows, prompts=rng.choice([0, 1, rng.randint(1, 9)]) if rows >= 16 else 0,
                    interleaved=rng.random() < 0.4, rotary=rng.choice([d, d, d // 2, d // 4, d - 24]), scaling=rng.choice(sorted(KINDS)), far=_log_int(rng, 64, 1000000))
    if op == "attention":
        shape = rng.choice(["tiny", "8b", "8b", "70b"])
        n = _log_int(rng, 1, 256 if shape != "70b" else 96)
        cuts = sorted(rng.sample(range(1, n), min(n - 1, rng.choice([0, 0, 1, 3, 6])))) if n > 1 else []
        groups = [b - a for a, b in zip([0] + cuts, cuts + [n])]
        shared = [rng.choice([0] + [_log_int(rng, 16, min(8192, 16384 // len(groups)))] * 5) for _ in groups]
        return dict(op=op, shape=shape, dtype=rng.choice(["bf16", "bf16", "f16"]), groups=",".join(map(str, groups)), shared=",".join(map(str, shared)),
                    suffix=_log_int(rng, 1, min(2000, 20000 // n)), spread=rng.choice([0.0, 0.5, 0.9]), layers=rng.choice([1, 2]))
    dtype = rng.choice(["f32", "f32", "bf16", "f16"])
    vocab = _log_int(rng, 1000, 128256)
    return dict(op=op, dtype=dtype, rows=_log_int(rng, 1, min(2048, (65000000 if dtype == "f32" else 130000000) // vocab)), vocab=vocab, top=rng.choice([0, 1, 5, 8, 20, 32]),
                masked=rng.choice([0.0, 0.0, 0.3]))


# ------------------------------------------------------------------------------------------ inputs
def _ints(text):
    return [int(x) for x in text.split(",")]


def _rng(case):
    """Lengths are a case's own, whatever the seed: every seed is then the same amount of work."""
    return random.Random("|".join("%s=%s" % (k, case[k]) for k in sorted(case) if k != "name"))


def _cuts(rng, total, parts):
    at = sorted(rng.sample(range(1, total), parts - 1))
    return [b - a for a, b in zip([0] + at, at + [total])]


def _lengths(case):
    """Cached and new tokens of each request of a `tables` case: prompts first, then decodes."""
    rng = _rng(case)
    added = (_cuts(rng, case["tokens"], case["prompts"]) if case["prompts"] else []) + [1] * case["decodes"]
    cached = [rng.choice([0, 0, rng.randint(1, case["ctx"])]) for _ in range(case["prompts"])]
    cached += [max(1, int(case["ctx"] * math.exp(rng.gauss(0.0, 0.7)))) for _ in range(case["decodes"])]
    return cached, added


def _pages(tokens):
    return -(-tokens // PAGE)


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _prepare_tables(case, g):
    cached, added = _lengths(case)
    n, rows = len(cached), sum(added)
    width = max(_pages(c + a) for c, a in zip(cached, added))
    held = sum(_pages(c) for c in cached)
    need = sum(_pages(c + a) - _pages(c) for c, a in zip(cached, added))
    ids = torch.randperm(held + need + 64, generator=g, device="cuda").to(torch.int32)
    tables = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
    have = torch.arange(width, device="cuda")[None, :] < torch.tensor([_pages(c) for c in cached], device="cuda")[:, None]
    tables[have] = ids[:held]
    new = lambda k: torch.zeros(k, dtype=torch.int32, device="cuda")  # noqa: E731
    return dict(n=n, rows=rows, width=width, cached=_i32(cached), added=_i32(added), free=ids[held:].clone(), n_free=_i32([need + 64]), tables=tables, lens=new(n),
                starts=new(n + 1), requests=new(rows), positions=new(rows), places=new(rows), left=new(1), status=new(1))


def _rope_rows(case):
    """Positions of the rows, and the page number and slot of each in its own run of pages: ragged prompts, or one token each of a decode batch."""
    rng, rows = _rng(case), case["rows"]
    lens = _cuts(rng, rows, case["prompts"]) if case["prompts"] else [1] * rows
    first = [rng.randint(0, max(0, case["far"] - m)) for m in lens]
    positions, pages, used = [], [], 0
    for p, m in zip(first, lens):
        positions += range(p, p + m)
        pages += [used + (p % PAGE + t) // PAGE for t in range(m)]
        used += (p % PAGE + m - 1) // PAGE + 1
    return positions, pages, used


def _prepare_rope(case, g):
    n_q, n_kv, d, _ = SHAPES[case["shape"]]
    t, rows = TYPES[case["dtype"]], case["rows"]
    positions, pages, used = _rope_rows(case)
    order = torch.randperm(used + 8, generator=g, device="cuda").to(torch.int32)
    pos = _i32(positions)
    qkv = torch.randn(rows, (n_q + 2 * n_kv) * d, generator=g, device="cuda").to(t)
    pool = torch.randn(used + 8, n_kv, 2 * PAGE * d, generator=g, device="cuda").to(t)
    return dict(qkv=qkv, pool=pool, positions=pos, places=(order[torch.tensor(pages, device="cuda")] * PAGE + pos % PAGE).to(torch.int32),
                q_out=torch.empty(rows, n_q * d, dtype=t, device="cuda"))


def _contexts(case):
    """Lengths of the groups' shared parts in whole pages, and of every request's context."""
    rng, lens, shared = _rng(case), [], []
    for n, s in zip(_ints(case["groups"]), _ints(case["shared"])):
        shared.append(s // PAGE * PAGE)
        lens += [s // PAGE * PAGE + max(1, int(case["suffix"] * math.exp(rng.gauss(0.0, case["spread"])))) for _ in range(n)]
    return shared, lens


def _prepare_attention(case, g):
    n_q, n_kv, d, _ = SHAPES[case["shape"]]
    t, (shared, lens), sizes = TYPES[case["dtype"]], _contexts(case), _ints(case["groups"])
    n, width = len(lens), max(map(_pages, lens))
    starts = [sum(sizes[:i]) for i in range(len(sizes) + 1)]
    total = sum(s // PAGE for s in shared) + sum(_pages(c) - s // PAGE for s, a, b in zip(shared, starts, starts[1:]) for c in lens[a:b])
    ids = torch.randperm(total + 16, generator=g, device="cuda").to(torch.int32)
    tables, used = torch.zeros(n, width, dtype=torch.int32, device="cuda"), 0
    for s, a, b in zip(shared, starts, starts[1:]):
        common, used = ids[used:used + s // PAGE], used + s // PAGE
        for r in range(a, b):
            m = _pages(lens[r]) - s // PAGE
            tables[r, :s // PAGE + m] = torch.cat([common, ids[used:used + m]])
            used += m
    x = dict(n=n, tables=tables, lens=_i32(lens), starts=_i32(starts), shared=_i32(shared), groups=len(sizes))
    # scores with a standard deviation of 2: a softmax that has favourites
    x["q"] = [(2.0 * torch.randn(n, n_q * d, generator=g, device="cuda")).to(t) for _ in range(case["layers"])]
    x["pool"] = [torch.randn(total + 16, n_kv, 2 * PAGE * d, generator=g, device="cuda").to(t) for _ in range(case["layers"])]
    x["out"] = [torch.empty(n, n_q * d, dtype=t, device="cuda") for _ in range(case["layers"])]
    x["lse"] = [torch.empty(n, n_q, device="cuda") for _ in range(case["layers"])]
    return x


def _prepare_logprobs(case, g):
    rows, vocab, top, t = case["rows"], case["vocab"], case["top"], TYPES[case["dtype"]]
    x = 2.5 * torch.randn(rows, vocab, generator=g, device="cuda")
    x[torch.arange(rows, device="cuda"), torch.randint(0, vocab, (rows,), generator=g, device="cuda")] += 9.0      # most tokens of a text are likely ones
    tokens = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    tokens = torch.where(torch.rand(rows, generator=g, device="cuda") < 0.6, x.argmax(1), tokens).to(torch.int32)
    if case["masked"]:
        ruled = torch.rand(rows, generator=g, device="cuda") < case["masked"]
        out = (torch.rand(vocab, generator=g, device="cuda") < 0.7)[None, :] & ruled[:, None]
        x = x.masked_fill(out, -math.inf)
        x[torch.arange(rows, device="cuda"), tokens.long()] = 1.0          # a grammar rules out no token that was taken
    new = lambda *s: torch.empty(*s, device="cuda")  # noqa: E731
    return dict(logits=x.to(t), tokens=tokens, logprob=new(rows), entropy=new(rows), lse=new(rows), rank=torch.empty(rows, dtype=torch.int32, device="cuda"),
                top_logprob=new(rows, top), top_token=torch.empty(rows, top, dtype=torch.int32, device="cuda"))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    x = {"tables": _prepare_tables, "rope": _prepare_rope, "attention": _prepare_attention, "logprobs": _prepare_logprobs}[case["op"]](case, g)
    if case["op"] == "attention":                                         # workspaces that a serving program keeps
        x["workspace"] = torch.empty(64 << 20 if case["shape"] == "tiny" else 256 << 20, dtype=torch.uint8, device="cuda")
    if case["op"] == "logprobs":
        x["workspace"] = torch.empty(16 << 20, dtype=torch.uint8, device="cuda")
    return dict(x, case=case)


# ------------------------------------------------------------------------------------------ plain forms
def _plain_tables(case, s):
    cached, added, f = s["cached"].long(), s["added"].long(), s["n_free"].long()
    held = (cached + PAGE - 1) // PAGE
    need = (cached + added + PAGE - 1) // PAGE - held
    starts = torch.cat([torch.zeros(1, dtype=torch.long, device="cuda"), added.cumsum(0)])
    before = need.cumsum(0) - need
    col = torch.arange(s["width"], device="cuda")[None, :] - held[:, None]
    new = (col >= 0) & (col < need[:, None])
    at = (f - need.sum() + before[:, None] + col).clamp(0, s["free"].numel() - 1)
    tables = torch.where(new, s["free"][at], s["tables"])
    request = torch.repeat_interleave(torch.arange(s["n"], device="cuda"), added, output_size=s["rows"])
    position = torch.arange(s["rows"], device="cuda") - starts[request] + cached[request]
    place = tables[request, position // PAGE] * PAGE + position % PAGE
    i = torch.int32
    return dict(tables=tables, lens=(cached + added).to(i), starts=starts.to(i), requests=request.to(i), positions=position.to(i), places=place.to(i),
                left=(f - need.sum()).to(i), status=torch.zeros(1, dtype=i, device="cuda"))


def _angles_of(case, i, rotary, theta):
    """Radians a token of pair i (64 bits), and the factor of cosine and sine."""
    kind, f = case["scaling"], theta ** (-2.0 * i / rotary)
    factor, low, high, length = 8.0, 1.0, {"bands": 4.0, "ramp": 32.0}.get(kind, 0.0), 8192.0
    if kind == "linear":
        return f / factor, 1.0
    if kind == "base":
        return (theta * factor ** (rotary / (rotary - 2.0))) ** (-2.0 * i / rotary), 1.0
    if kind == "bands":                                                    # by wavelength against the length the model was trained on
        turns = length * f / (2.0 * math.pi)
        return f / factor + (f - f / factor) * ((turns - low) / (high - low)).clamp(0.0, 1.0), 1.0
    if kind == "ramp":                                                     # by the pair's number
        pair = lambda beta: rotary * math.log(length / (beta * 2.0 * math.pi)) / (2.0 * math.log(theta))  # noqa: E731
        a, b = max(math.floor(pair(high)), 0), min(math.ceil(pair(low)), rotary - 1)
        share = ((i - a) / max(b - a, 0.001)).clamp(0.0, 1.0)
        mag = torch.tensor(0.1 * math.log(factor) + 1.0, dtype=torch.float32).item()
        return f / factor * share + f * (1.0 - share), mag
    return f, 1.0


def _turned(case, x, heads, positions, wide):
    """Rotated rows [rows, heads, d] in the type `wide`; the angles in 64 bits."""
    _, _, d, theta = SHAPES[case["shape"]]
    R, x = case["rotary"], x.reshape(x.shape[0], heads, d).to(wide)
    w, mag = _angles_of(case, torch.arange(R // 2, dtype=torch.float64, device="cuda"), R, theta)
    a = positions.to(torch.float64)[:, None] * w[None, :]
    c, s = ((mag * f).to(wide)[:, None, :] for f in (torch.cos(a), torch.sin(a)))
    p, q = (x[:, :, 0:R:2], x[:, :, 1:R:2]) if case["interleaved"] else (x[:, :, :R // 2], x[:, :, R // 2:R])
    u, v = p * c - q * s, q * c + p * s
    turned = torch.stack([u, v], dim=3).reshape(x.shape[0], heads, R) if case["interleaved"] else torch.cat([u, v], dim=2)
    return torch.cat([turned, x[:, :, R:]], dim=2)


def _append(pool, places, k, v):
    """Rows' K and V [rows, n_kv, d] into their pages (in place)."""
    pages, n_kv, e = pool.shape
    d, page, slot = e // (2 * PAGE), places.long() // PAGE, places.long() % PAGE
    pool[:, :, :PAGE * d].view(pages, n_kv, PAGE, d)[page, :, slot] = k.to(pool.dtype)
    pool[:, :, PAGE * d:].view(pages, n_kv, d, PAGE)[page, :, :, slot] = v.to(pool.dtype)


def _plain_rope(case, s):
    n_q, n_kv, d, _ = SHAPES[case["shape"]]
    q, k, v = s["qkv"].split([n_q * d, n_kv * d, n_kv * d], dim=1)
    t = q.dtype
    out = _turned(case, q, n_q, s["positions"], torch.float32).to(t).reshape(q.shape)
    _append(s["pool"], s["places"], _turned(case, k, n_kv, s["positions"], torch.float32).to(t), v.reshape(-1, n_kv, d))
    return dict(q=out, pool=s["pool"])


def _plain_attention(s, q, pool, n_q, d):
    pages, n_kv, _ = pool.shape
    n, width, g = s["n"], s["tables"].shape[1], n_q // n_kv
    got = pool[s["tables"].long()]                                        # [n, width, n_kv, K | V^T]
    k = got[..., :PAGE * d].view(n, width, n_kv, PAGE, d).permute(0, 2, 1, 3, 4).reshape(n, n_kv, width * PAGE, d).float()
    v = got[..., PAGE * d:].view(n, width, n_kv, d, PAGE).permute(0, 2, 1, 4, 3).reshape(n, n_kv, width * PAGE, d).float()
    sc = torch.matmul(q.view(n, n_kv, g, d).float(), k.transpose(2, 3).contiguous()) / math.sqrt(d)
    there = torch.arange(width * PAGE, device="cuda")[None, :] < s["lens"][:, None]
    sc = sc.masked_fill(~there[:, None, None, :], -math.inf)
    m = sc.max(dim=3, keepdim=True).values
    p = torch.exp(sc - m)
    z = p.sum(dim=3, keepdim=True)
    v = v.masked_fill(~there[:, None, :, None], 0.0)
    return (torch.matmul(p, v) / z).reshape(n, n_q * d).to(q.dtype), (m + torch.log(z)).reshape(n, n_q)


def _in_order(x):
    """Keys whose largest are the largest values, the lowest index first among equals."""
    bits = torch.where(x == 0.0, torch.zeros_like(x), x).view(torch.int32).long()
    bits = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
    return bits * (1 << 24) + ((1 << 24) - 1 - torch.arange(x.shape[1], device="cuda"))[None, :]


def _plain_logprobs(case, s):
    x, tok = s["logits"].float(), s["tokens"].long()[:, None]
    m = x.max(dim=1, keepdim=True).values
    e = torch.exp(x - m)
    z = e.sum(dim=1, keepdim=True, dtype=torch.float64)
    lse = m.double() + torch.log(z)
    w = torch.where(e > 0.0, e * (x - m), torch.zeros_like(e)).sum(dim=1, keepdim=True, dtype=torch.float64)
    xt = x.gather(1, tok)
    rank = (x > xt).sum(dim=1) + ((x == xt) & (torch.arange(x.shape[1], device="cuda")[None, :] < tok)).sum(dim=1)
    out = dict(logprob=(xt - lse).float()[:, 0], entropy=(torch.log(z) - w / z).float()[:, 0], lse=lse.float()[:, 0], rank=rank.to(torch.int32))
    if case["top"]:
        best = torch.topk(_in_order(x), case["top"], dim=1).indices
        out.update(top_logprob=(x.gather(1, best) - lse).float(), top_token=best.to(torch.int32))
    return out


# ------------------------------------------------------------------------------------------ the library's calls
def _own_tables(case, s):
    from paper_2504_19516_amd import sts
    p = torch.Tensor.data_ptr
    sts.op_block_tables(sts.BlockTables(
        n_requests=s["n"], max_pages=s["width"], max_rows=s["rows"], free_capacity=s["free"].numel(), table_stride=s["width"], cached=p(s["cached"]), added=p(s["added"]),
        free_pages=p(s["free"]), n_free=p(s["n_free"]), tables=p(s["tables"]), lens=p(s["lens"]), row_starts=p(s["starts"]), requests=p(s["requests"]),
        positions=p(s["positions"]), places=p(s["places"]), n_free_left=p(s["left"]), status=p(s["status"])), torch.cuda.current_stream().cuda_stream)
    return {k: s[k] for k in ("tables", "lens", "starts", "requests", "positions", "places", "left", "status")}


def _own_rope(case, s):
    from paper_2504_19516_amd import sts
    n_q, n_kv, d, theta = SHAPES[case["shape"]]
    kind, size, base = case["scaling"], s["qkv"].element_size(), s["qkv"].data_ptr()
    ld = s["qkv"].stride(0)
    rope = sts.Rope(rotary_dim=case["rotary"], interleaved=case["interleaved"], scaling=KINDS[kind], original_len=8192, theta=theta, factor=8.0, low=1.0,
                    high=4.0 if kind == "bands" else 32.0, magnitude=0.1 * math.log(8.0) + 1.0 if kind == "ramp" else 1.0)
    sts.op_rope(rope, sts.RopeRows(
        dtype=sts.DTYPES[case["dtype"]], rows=case["rows"], n_q=n_q, n_kv=n_kv, d=d, pool_pages=s["pool"].shape[0], q=base, q_stride=ld, q_out=s["q_out"].data_ptr(),
        q_out_stride=n_q * d, k=base + n_q * d * size, k_stride=ld, v=base + (n_q + n_kv) * d * size, v_stride=ld, pool=s["pool"].data_ptr(),
        positions=s["positions"].data_ptr(), places=s["places"].data_ptr()), torch.cuda.current_stream().cuda_stream)
    return dict(q=s["q_out"], pool=s["pool"])


def _own_attention(case, s):
    from paper_2504_19516_amd import sts
    n_q, n_kv, d, _ = SHAPES[case["shape"]]
    stream = torch.cuda.current_stream().cuda_stream
    batch = sts.AttnBatch(dtype=sts.DTYPES[case["dtype"]], n_requests=s["n"], n_groups=s["groups"], n_q=n_q, n_kv=n_kv, d=d, pool_pages=s["pool"][0].shape[0],
                          max_pages=s["tables"].shape[1], table_stride=s["tables"].stride(0), tables=s["tables"].data_ptr(), lens=s["lens"].data_ptr(),
                          group_starts=s["starts"].data_ptr(), shared_lens=s["shared"].data_ptr(), workspace=s["workspace"].data_ptr(),
                          workspace_bytes=s["workspace"].numel())
    sts.op_attn_shared_plan(batch, stream)                                # once a step, for all its layers
    for q, pool, out, lse in zip(s["q"], s["pool"], s["out"], s["lse"]):
        sts.op_attn_shared(batch, q.data_ptr(), n_q * d, pool.data_ptr(), out.data_ptr(), n_q * d, lse.data_ptr(), 0.0, stream)
    return dict(out=s["out"], lse=s["lse"])


def _own_logprobs(case, s):
    from paper_2504_19516_amd import sts
    p = torch.Tensor.data_ptr
    sts.op_logprobs(sts.Logprobs(
        dtype=sts.DTYPES[case["dtype"]], rows=case["rows"], vocab=case["vocab"], top_k=case["top"], row_stride=case["vocab"], logits=p(s["logits"]), tokens=p(s["tokens"]),
        logprob=p(s["logprob"]), entropy=p(s["entropy"]), lse=p(s["lse"]), rank=p(s["rank"]), top_logprob=p(s["top_logprob"]), top_token=p(s["top_token"]),
        workspace=p(s["workspace"]), workspace_bytes=s["workspace"].numel()), torch.cuda.current_stream().cuda_stream)
    return {k: s[k] for k in ("logprob", "entropy", "lse", "rank") + (("top_logprob", "top_token") if case["top"] else ())}


def run(state):
    case = state["case"]
    if own:
        return {"tables": _own_tables, "rope": _own_rope, "attention": _own_attention, "logprobs": _own_logprobs}[case["op"]](case, state)
    if case["op"] == "attention":
        n_q, _, d, _ = SHAPES[case["shape"]]
        done = [_plain_attention(state, q, pool, n_q, d) for q, pool in zip(state["q"], state["pool"])]
        return dict(out=[o for o, _ in done], lse=[z for _, z in done])
    return {"tables": _plain_tables, "rope": _plain_rope, "logprobs": _plain_logprobs}[case["op"]](case, state)


# ------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    op = case["op"]
    if op == "tables":
        cached, added = _lengths(case)
        rows, n, need = sum(added), len(cached), sum(_pages(c + a) - _pages(c) for c, a in zip(cached, added))
        return {"bytes": 8.0 * n + 4.0 * need + 12.0 * rows + 8.0 * n + 4.0 * need, "flops": 4.0 * rows}
    if op == "rope":
        n_q, n_kv, d, _ = SHAPES[case["shape"]]
        return {"bytes": case["rows"] * (2.0 * 2 * (n_q + 2 * n_kv) * d + 8), "flops": 3.0 * case["rows"] * (n_q + n_kv) * case["rotary"]}
    if op == "attention":
        n_q, n_kv, d, _ = SHAPES[case["shape"]]
        (shared, lens), sizes = _contexts(case), _ints(case["groups"])
        tokens = sum(shared) + sum(lens) - sum(s * m for s, m in zip(shared, sizes))       # a group's prefix is read once
        return {"bytes": case["layers"] * (4.0 * n_kv * d * tokens + 4.0 * len(lens) * n_q * d), "flops": case["layers"] * 4.0 * n_q * d * sum(lens)}
    size = {"f32": 4, "bf16": 2, "f16": 2}[case["dtype"]]
    return {"bytes": float(size) * case["rows"] * case["vocab"] + case["rows"] * (20.0 + 8 * case["top"]), "flops": 6.0 * case["rows"] * case["vocab"]}


# ------------------------------------------------------------------------------------------ the same in 64 bits, from the definitions
def _exact_rope(case, s):
    n_q, n_kv, d, theta = SHAPES[case["shape"]]
    R, rows = case["rotary"], case["rows"]
    x = s["qkv"].double().view(rows, n_q + 2 * n_kv, d)
    w, mag = _angles_of(case, torch.arange(R // 2, dtype=torch.float64, device="cuda"), R, theta)
    turn = torch.polar(torch.full((rows, R // 2), mag, dtype=torch.float64, device="cuda"), s["positions"].double()[:, None] * w[None, :])
    pairs = torch.arange(R, device="cuda").view(R // 2, 2) if case["interleaved"] else torch.arange(R, device="cuda").view(2, R // 2).t()
    z = torch.view_as_complex(x[:, :n_q + n_kv][:, :, pairs].contiguous()) * turn[:, None, :]          # a pair is a complex number
    y = x.clone()
    y[:, :n_q + n_kv, pairs.reshape(-1)] = torch.view_as_real(z).flatten(2)
    pool = s["pool"].double()
    k_part, v_part = pool[:, :, :PAGE * d].view(-1, n_kv, PAGE, d), pool[:, :, PAGE * d:].view(-1, n_kv, d, PAGE)
    for slot in range(PAGE):
        at = (s["places"] % PAGE == slot).nonzero()[:, 0]
        page = s["places"][at].long() // PAGE
        k_part[page, :, slot, :] = y[at, n_q:n_q + n_kv]
        v_part[page, :, :, slot] = y[at, n_q + n_kv:]
    return dict(q=y[:, :n_q].reshape(rows, n_q * d), pool=pool)


def _exact_attention(case, s):
    n_q, n_kv, d, _ = SHAPES[case["shape"]]
    lens, outs, sums = s["lens"].tolist(), [], []
    for q, pool in zip(s["q"], s["pool"]):
        out, lse = torch.zeros(s["n"], n_q, d, dtype=torch.float64, device="cuda"), torch.zeros(s["n"], n_q, dtype=torch.float64, device="cuda")
        for r, c in enumerate(lens):
            got = pool[s["tables"][r, :_pages(c)].long()]
            for h in range(n_kv):
                k = got[:, h, :PAGE * d].reshape(-1, d)[:c].double()
                v = got[:, h, PAGE * d:].reshape(-1, d, PAGE).transpose(1, 2).reshape(-1, d)[:c].double()
                heads = slice(h * (n_q // n_kv), (h + 1) * (n_q // n_kv))
                a = q[r].view(n_q, d)[heads].double() @ k.t().contiguous() * d ** -0.5
                lse[r, heads] = torch.logsumexp(a, 1)
                out[r, heads] = torch.softmax(a, 1) @ v
        outs.append(out.view(s["n"], n_q * d))
        sums.append(lse)
    return dict(out=outs, lse=sums)


def _exact_logprobs(case, s):
    parts = []
    for a in range(0, case["rows"], 256):                                 # in blocks of rows, to bound the memory
        x, tok = s["logits"][a:a + 256].double(), s["tokens"][a:a + 256].long()
        lp = torch.log_softmax(x, 1)
        p = torch.exp(lp)
        part = [lp[torch.arange(len(tok), device="cuda"), tok], -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(1), torch.logsumexp(x, 1)]
        parts.append(part + ([torch.sort(lp, dim=1, descending=True).values[:, :case["top"]]] if case["top"] else []))
    got = [torch.cat(x) for x in zip(*parts)]
    out = dict(logprob=got[0], entropy=got[1], lse=got[2], rank=None)
    return dict(out, top_logprob=got[3], top_token=None) if case["top"] else out


def exact(case, seed):
    if case["op"] == "tables":                                            # whole numbers only
        return None
    return {"rope": _exact_rope, "attention": _exact_attention, "logprobs": _exact_logprobs}[case["op"]](case, prepare(case, seed))
