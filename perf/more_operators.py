"""Operators of a decode step that verifies drafted tokens, as cases to measure: norms of the heads with rotary positions and the
append to the pages, attention for trees of drafted tokens over a paged cache, penalties, biases and grammar masks on logits, and the
accepted path with its cache rows moved to where the next step expects them. They work on device data, through
`paper_2504_19516_amd.sts` (the plain forms below need torch alone).

The KV cache is the library's: one layer's pool is [page][kv head][K: 16 tokens x d | V^T: d x 16 tokens], a request's tokens
16 t .. 16 t + 15 lie in page table[t]. A request's drafted tokens are its nodes: node i lies at token cached + i and knows its parent by
number (-1: it follows the context). Shapes: the model shapes of `paper_2504_19516_amd.synth` (heads 32/8 and 64/8 of 128 elements, 4/4
of 64, vocabulary 128256).
"""
import math
import random

import torch

own = False

PAGE = 16
SHAPES = {"tiny": (4, 4, 64, 1.0e4), "8b": (32, 8, 128, 5.0e5), "70b": (64, 8, 128, 5.0e5)}      # query heads, kv heads, head size, rope base
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1.0e-6


# ------------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # ---- head norms, rotary positions and append: the drafted tokens of five requests
        dict(name="norm_rope_drafts_130", op="norm_rope", shape="8b", dtype="bf16", rows=130, runs=5, interleaved=False, rotary=128, offset=False, far=4096),
        # a prefill batch of ragged prompts
        dict(name="norm_rope_prefill_8192", op="norm_rope", shape="8b", dtype="bf16", rows=8192, runs=6, interleaved=False, rotary=128, offset=False, far=30000),
        # an odd chunk of a model that turns half of each head in neighbouring pairs and stores its gains less 1, 16-bit floats
        dict(name="norm_rope_partial_1201", op="norm_rope", shape="tiny", dtype="f16", rows=1201, runs=3, interleaved=True, rotary=32, offset=True, far=30000),
        # ---- attention: one user's tree of 26 drafted tokens
        dict(name="attn_tree_1_user", op="tree", shape="8b", dtype="bf16", requests=1, levels="1,4,8,8,5", ragged=False, ctx=1500, spread=0.0, layers=4),
        # chains of four drafted tokens behind the last one, a conversational batch
        dict(name="attn_chains_64", op="tree", shape="8b", dtype="bf16", requests=64, levels="1,1,1,1,1", ragged=False, ctx=1100, spread=0.7, layers=4),
        # wide trees over longer contexts
        dict(name="attn_trees_16", op="tree", shape="8b", dtype="bf16", requests=16, levels="1,8,16,20,19", ragged=False, ctx=4096, spread=0.4, layers=2),
        # a few long contexts with trees of different sizes, on the larger shape
        dict(name="attn_trees_70b", op="tree", shape="70b", dtype="f16", requests=6, levels="1,4,8,12,8", ragged=True, ctx=14000, spread=0.5, layers=2),
        # ---- logits: one user's token, penalties over a conversation
        dict(name="adjust_1", op="adjust", dtype="f32", requests=1, levels="1", vocab=128256, history=1500, penalties=True, biases=20, masked=0.0, in_place=False),
        # the drafted chains of a batch, each node with its own path, some rows under a grammar
        dict(name="adjust_drafts_320", op="adjust", dtype="f32", requests=64, levels="1,1,1,1,1", vocab=128256, history=2000, penalties=True, biases=8, masked=0.1, in_place=False),
        # a batch whose rows are half under grammars that rule nearly everything out, in place
        dict(name="adjust_grammar_256", op="adjust", dtype="bf16", requests=256, levels="1", vocab=128256, history=0, penalties=False, biases=0, masked=0.5, in_place=True),
        # ---- the accepted path and its cache rows: one user, all layers
        dict(name="follow_1", op="follow", shape="8b", dtype="bf16", requests=1, levels="1,4,8,8,5", ctx=200, layers=32),
        # a batch
        dict(name="follow_64", op="follow", shape="8b", dtype="bf16", requests=64, levels="1,8,16,20,19", ctx=100, layers=8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_levels(rng, most):
    """Nodes of each level of a tree of up to `most` nodes: chains as often as trees."""
    total = _log_int(rng, 1, most)
    if rng.random() < 0.5:
        return ",".join(["1"] * min(total, 16))
    levels, left = [1], total - 1
    while left > 0:
        levels.append(min(left, rng.randint(1, 20)))
        left -= levels[-1]
    return ",".join(map(str, levels))


def draw(rng):
    op = rng.choice(["norm_rope", "norm_rope", "tree", "tree", "tree", "tree", "adjust", "adjust", "adjust", "follow"])
    if op == "norm_rope":
        shape = rng.choice(["tiny", "8b", "8b", "70b"])
        d = SHAPES[shape][2]
        rows = _log_int(rng, 1, 8192 if shape != "70b" else 4096)
        return dict(op=op, shape=shape, dtype=rng.choice(["bf16", "bf16", "f16"]), rows=rows, runs=rng.randint(1, min(rows, 9)), interleaved=rng.random() < 0.4,
                    rotary=rng.choice([d, d, d // 2, d // 4, d - 24]), offset=rng.random() < 0.3, far=_log_int(rng, 64, 1000000))
    if op == "tree":
        shape = rng.choice(["tiny", "8b", "8b", "70b"])
        requests = _log_int(rng, 1, 64 if shape != "70b" else 24)
        most = max(1, min(100, (1024 if shape != "70b" else 400) // requests))
        return dict(op=op, shape=shape, dtype=rng.choice(["bf16", "bf16", "f16"]), requests=requests, levels=_draw_levels(rng, most), ragged=rng.random() < 0.5,
                    ctx=_log_int(rng, 1, min(16000, 60000 // requests)), spread=rng.choice([0.0, 0.4, 0.7]), layers=rng.choice([1, 2]))
    if op == "adjust":
        dtype, vocab = rng.choice(["f32", "f32", "bf16", "f16"]), _log_int(rng, 1000, 128256)
        penalties = rng.random() < 0.7
        rows = _log_int(rng, 1, min(1000, 40000000 // vocab))
        levels = _draw_levels(rng, min(rows, 40))
        return dict(op=op, dtype=dtype, requests=max(1, rows // sum(map(int, levels.split(",")))), levels=levels, vocab=vocab, history=_log_int(rng, 1, 8000) if penalties else 0, penalties=penalties,
                    biases=rng.choice([0, 3, 100]) if penalties else 0, masked=rng.choice([0.0, 0.2, 1.0]) if penalties else rng.choice([0.3, 1.0]), in_place=not penalties)
    shape = rng.choice(["tiny", "8b", "70b"])
    requests = _log_int(rng, 1, 64)
    return dict(op=op, shape=shape, dtype=rng.choice(["bf16", "f16"]), requests=requests, levels=_draw_levels(rng, 64), ctx=_log_int(rng, 1, 100), layers=rng.randint(1, 8))


# ------------------------------------------------------------------------------------------ inputs
def _ints(text):
    return [int(x) for x in text.split(",")]


def _rng(case):
    """Lengths and trees are a case's own, whatever the seed: every seed is then the same amount of work."""
    return random.Random("|".join("%s=%s" % (k, case[k]) for k in sorted(case) if k != "name"))


def _cuts(rng, total, parts):
    at = sorted(rng.sample(range(1, total), parts - 1))
    return [b - a for a, b in zip([0] + at, at + [total])]


def _pages(tokens):
    return -(-tokens // PAGE)


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _tree(rng, levels):
    """Parents of the nodes, level behind level; every node of a level hangs on one of the level before."""
    parents, before = [], [-1]
    for m in levels:
        here = list(range(len(parents), len(parents) + m))
        parents += sorted(rng.choice(before) for _ in here)
        before = here
    return parents


def _trees(case):
    """Cached tokens of each request, and the parents of its nodes. Ragged: the first nodes of a tree, which are one too."""
    rng = _rng(case)
    cached = [max(1, int(case["ctx"] * math.exp(rng.gauss(0.0, case.get("spread", 0.5))))) for _ in range(case["requests"])]
    trees = [_tree(rng, _ints(case["levels"])) for _ in cached]
    return cached, [t[:rng.randint(1, len(t))] if case.get("ragged") else t for t in trees]


def _starts(lists):
    out = [0]
    for x in lists:
        out.append(out[-1] + len(x))
    return out


def _paged(cached, trees, g):
    """Block tables of the requests, their pages in any order, and the pool's pages."""
    need = [_pages(c + len(t)) for c, t in zip(cached, trees)]
    ids = torch.randperm(sum(need) + 16, generator=g, device="cuda").to(torch.int32)
    tables, used = torch.zeros(len(need), max(need), dtype=torch.int32, device="cuda"), 0
    for r, m in enumerate(need):
        tables[r, :m] = ids[used:used + m]
        used += m
    return tables, ids.numel()


def _prepare_norm_rope(case, g):
    n_q, n_kv, d, _ = SHAPES[case["shape"]]
    rng, t, rows = _rng(case), TYPES[case["dtype"]], case["rows"]
    positions, pages, used = [], [], 0
    for m in _cuts(rng, rows, case["runs"]):
        p = rng.randint(0, max(0, case["far"] - m))
        positions += range(p, p + m)
        pages += [used + (p % PAGE + i) // PAGE for i in range(m)]
        used += (p % PAGE + m - 1) // PAGE + 1
    order = torch.randperm(used + 8, generator=g, device="cuda").to(torch.int32)
    pos = _i32(positions)
    qkv = (1.7 * torch.randn(rows, (n_q + 2 * n_kv) * d, generator=g, device="cuda")).to(t)
    gains = [((0.0 if case["offset"] else 1.0) + 0.3 * torch.randn(d, generator=g, device="cuda")).to(t) for _ in range(2)]
    pool = torch.randn(used + 8, n_kv, 2 * PAGE * d, generator=g, device="cuda").to(t)
    return dict(qkv=qkv, q_gain=gains[0], k_gain=gains[1], pool=pool, positions=pos, places=(order[torch.tensor(pages, device="cuda")] * PAGE + pos % PAGE).to(torch.int32),
                q_out=torch.empty(rows, n_q * d, dtype=t, device="cuda"))


def _prepare_tree(case, g):
    n_q, n_kv, d, _ = SHAPES[case["shape"]]
    t, (cached, trees) = TYPES[case["dtype"]], _trees(case)
    tables, pages = _paged(cached, trees, g)
    rows = sum(map(len, trees))
    x = dict(tables=tables, cached=_i32(cached), starts=_i32(_starts(trees)), parents=_i32(sum(trees, [])), positions=torch.zeros(rows, dtype=torch.int32, device="cuda"), rows=rows,
             most=max(map(len, trees)))
    # scores with a standard deviation of 2: a softmax that has favourites
    x["q"] = [(2.0 * torch.randn(rows, n_q * d, generator=g, device="cuda")).to(t) for _ in range(case["layers"])]
    x["pool"] = [torch.randn(pages, n_kv, 2 * PAGE * d, generator=g, device="cuda").to(t) for _ in range(case["layers"])]
    x["out"] = [torch.empty(rows, n_q * d, dtype=t, device="cuda") for _ in range(case["layers"])]
    x["lse"] = [torch.empty(rows, n_q, device="cuda") for _ in range(case["layers"])]
    if own:                                                               # a workspace that a serving program keeps
        from paper_2504_19516_amd import sts
        x["workspace"] = torch.empty(sts.attn_tree_workspace(len(cached), rows, n_q, n_kv, d), dtype=torch.uint8, device="cuda")
    return x


def _token_mix(shape, vocab, g):
    """Tokens of a text: low numbers come again and again."""
    return (vocab * torch.rand(shape, generator=g, device="cuda") ** 4).to(torch.int32).clamp(0, vocab - 1)


def _prepare_adjust(case, g):
    vocab, n = case["vocab"], case["requests"]
    rng = _rng(case)
    trees = [_tree(rng, _ints(case["levels"])) for _ in range(n)]
    rows = sum(map(len, trees))
    lens = [rng.randint(case["history"] // 2, case["history"]) for _ in range(n)]
    prompts = [rng.randint(0, m) for m in lens]
    x = dict(logits=(2.5 * torch.randn(rows, vocab, generator=g, device="cuda")).to(TYPES[case["dtype"]]), rows=rows, most=max(map(len, trees)), starts=_i32(_starts(trees)), parents=_i32(sum(trees, [])),
             requests=_i32([i for i, t in enumerate(trees) for _ in t]), drafted=_token_mix((rows,), vocab, g))
    x["out"] = x["logits"] if case["in_place"] else torch.empty_like(x["logits"])
    if case["penalties"]:
        x.update(tokens=_token_mix((n, case["history"]), vocab, g), lens=_i32(lens), prompts=_i32(prompts), repetition=1.0 + 0.4 * torch.rand(n, generator=g, device="cuda"),
                 frequency=0.3 * torch.rand(n, generator=g, device="cuda"), presence=0.5 * torch.rand(n, generator=g, device="cuda"))
    if case["biases"]:
        picks = torch.stack([torch.randperm(vocab, generator=g, device="cuda")[:case["biases"]] for _ in range(n)]).to(torch.int32)
        x.update(bias_starts=_i32([i * case["biases"] for i in range(n + 1)]), bias_tokens=picks.reshape(-1), bias_values=4.0 * torch.randn(picks.numel(), generator=g, device="cuda"))
    if case["masked"]:
        words = -(-vocab // 32)
        few = torch.rand(4, words * 32, generator=g, device="cuda") < torch.tensor([[0.02], [0.001], [0.3], [0.02]], device="cuda")
        bits = few.view(4, words, 32).long() << torch.arange(32, device="cuda")
        masks = bits.sum(dim=2)
        which = torch.randint(0, 4, (rows,), generator=g, device="cuda").to(torch.int32)
        free = torch.tensor([rng.random() >= case["masked"] for _ in range(rows)], device="cuda")
        x.update(masks=torch.where(masks >= 1 << 31, masks - (1 << 32), masks).to(torch.int32), mask_rows=torch.where(free, torch.full_like(which, -1), which))
    return x


def _prepare_follow(case, g):
    """A target that agrees with the draft along one path of each tree. The path's nodes are their own number or lie behind all its places, so that a pass over a
    cache that was moved already moves the same rows again."""
    n_q, n_kv, d, _ = SHAPES[case["shape"]]
    t, rng, (cached, trees) = TYPES[case["dtype"]], _rng(case), _trees(case)
    tables, pages = _paged(cached, trees, g)
    starts, tokens, chosen = _starts(trees), [], []
    for tree in trees:
        children = {}
        for j, p in enumerate(tree):
            children.setdefault(p, []).append(j)
        longest = rng.randint(1, 6)
        path = [0]
        while len(path) < longest:
            fit = [j for j in children.get(path[-1], []) if j == len(path) or j >= longest]
            if not fit:
                break
            path.append(rng.choice(fit))
        tok = [1000 * rng.randint(0, 9) + j for j in range(len(tree))]                 # all different
        want = [100000 + j for j in range(len(tree))]                                  # no node's
        for a, b in zip(path, path[1:]):
            want[a] = tok[b]
        tokens += tok
        chosen += want
    rows = starts[-1]
    shift = int(torch.randint(0, 1000, (1,), generator=g, device="cuda"))              # other tokens with another seed, the same paths
    new = lambda m: torch.zeros(m, dtype=torch.int32, device="cuda")  # noqa: E731
    return dict(tables=tables, cached=_i32(cached), starts=_i32(starts), parents=_i32(sum(trees, [])), tokens=_i32(tokens) + shift, chosen=_i32(chosen) + shift, rows=rows,
                most=max(map(len, trees)), pool=[torch.randn(pages, n_kv, 2 * PAGE * d, generator=g, device="cuda").to(t) for _ in range(case["layers"])],
                lens=new(len(cached)), counts=new(len(cached)), path=new(rows), next_token=new(len(cached)))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    return dict({"norm_rope": _prepare_norm_rope, "tree": _prepare_tree, "adjust": _prepare_adjust, "follow": _prepare_follow}[case["op"]](case, g), case=case)


# ------------------------------------------------------------------------------------------ plain forms
def _normed(case, x, gain):
    """x [rows, heads, d] in 32 bits, each head divided by its root mean square and scaled."""
    x = x.float()
    return x / torch.sqrt((x * x).mean(dim=2, keepdim=True) + EPS) * (gain.float() + (1.0 if case["offset"] else 0.0))


def _turned(case, x, positions):
    """The first elements of each head turned; the angles in 64 bits."""
    _, _, _, theta = SHAPES[case["shape"]]
    R = case["rotary"]
    w = theta ** (-2.0 * torch.arange(R // 2, dtype=torch.float64, device="cuda") / R)
    a = positions.to(torch.float64)[:, None] * w[None, :]
    c, s = torch.cos(a).float()[:, None, :], torch.sin(a).float()[:, None, :]
    p, q = (x[:, :, 0:R:2], x[:, :, 1:R:2]) if case["interleaved"] else (x[:, :, :R // 2], x[:, :, R // 2:R])
    u, v = p * c - q * s, q * c + p * s
    turned = torch.stack([u, v], dim=3).reshape(x.shape[0], x.shape[1], R) if case["interleaved"] else torch.cat([u, v], dim=2)
    return torch.cat([turned, x[:, :, R:]], dim=2)


def _append(pool, places, k, v):
    """Rows' K and V [rows, n_kv, d] into their pages (in place)."""
    pages, n_kv, e = pool.shape
    d, page, slot = e // (2 * PAGE), places.long() // PAGE, places.long() % PAGE
    pool[:, :, :PAGE * d].view(pages, n_kv, PAGE, d)[page, :, slot] = k.to(pool.dtype)
    pool[:, :, PAGE * d:].view(pages, n_kv, d, PAGE)[page, :, :, slot] = v.to(pool.dtype)


def _plain_norm_rope(case, s):
    n_q, n_kv, d, _ = SHAPES[case["shape"]]
    x = s["qkv"].view(case["rows"], n_q + 2 * n_kv, d)
    q = _turned(case, _normed(case, x[:, :n_q], s["q_gain"]), s["positions"]).to(x.dtype).reshape(case["rows"], n_q * d)
    k = _turned(case, _normed(case, x[:, n_q:n_q + n_kv], s["k_gain"]), s["positions"])
    _append(s["pool"], s["places"], k, x[:, n_q + n_kv:])
    return dict(q=q, pool=s["pool"])


def _padded_trees(s):
    """The ragged nodes as [requests, most nodes]: rows of each, which there are, who is an ancestor of whom (or the node itself), and each row's place in there."""
    starts, most = s["starts"].long(), s["most"]
    n, counts = starts.numel() - 1, starts[1:] - starts[:-1]
    node = torch.arange(most, device="cuda")
    there = node[None, :] < counts[:, None]
    rows = torch.where(there, starts[:-1, None] + node[None, :], torch.zeros_like(starts[:1, None]))
    parents = torch.where(there, s["parents"].long()[rows], torch.full_like(rows, -1))
    up = (parents[:, :, None] == node[None, None, :]).float() + torch.eye(most, device="cuda")[None]
    for _ in range(max(1, (most - 1).bit_length())):                      # reaches twice as far each time
        up = (torch.matmul(up, up.contiguous()) > 0.0).float()
    owner = torch.repeat_interleave(torch.arange(n, device="cuda"), counts, output_size=s["rows"])
    return rows, there, up > 0.0, (owner, torch.arange(s["rows"], device="cuda") - starts[owner])


def _plain_tree(case, s):
    n_q, n_kv, d, _ = SHAPES[case["shape"]]
    rows, there, up, place = _padded_trees(s)
    n, most, width = rows.shape[0], rows.shape[1], s["tables"].shape[1]
    g, counts, cached = n_q // n_kv, there.sum(dim=1), s["cached"].long()
    positions = (cached[:, None] + up.sum(dim=2) - 1)[place].to(torch.int32)
    token = torch.arange(width * PAGE, device="cuda")[None, :]
    node = token - cached[:, None]
    held = token < (cached + counts)[:, None]
    seen = (node < 0)[:, None, :] | (up.gather(2, node.clamp(0, most - 1)[:, None, :].expand(n, most, -1)) & (node >= 0)[:, None, :])
    seen = seen & held[:, None, :]
    outs, sums = [], []
    for q, pool in zip(s["q"], s["pool"]):
        got = pool[s["tables"].long()]                                    # [n, width, n_kv, K | V^T]
        k = got[..., :PAGE * d].view(n, width, n_kv, PAGE, d).permute(0, 2, 1, 3, 4).reshape(n, n_kv, width * PAGE, d).float()
        v = got[..., PAGE * d:].view(n, width, n_kv, d, PAGE).permute(0, 2, 1, 4, 3).reshape(n, n_kv, width * PAGE, d).float()
        qf = q[rows].view(n, most, n_kv, g, d).permute(0, 2, 1, 3, 4).reshape(n, n_kv, most * g, d).float()
        sc = torch.matmul(qf, k.transpose(2, 3).contiguous()) / math.sqrt(d)
        sc = sc.masked_fill(~seen[:, None, :, None, :].expand(-1, -1, -1, g, -1).reshape(n, 1, most * g, -1), -math.inf)
        m = sc.max(dim=3, keepdim=True).values
        p = torch.exp(sc - m)
        z = p.sum(dim=3, keepdim=True)
        o = torch.matmul(p, v.masked_fill(~held[:, None, :, None], 0.0)) / z
        back = lambda x: x.view(n, n_kv, most, g, -1).permute(0, 2, 1, 3, 4)[place].reshape(s["rows"], -1)  # noqa: E731
        outs.append(back(o).to(q.dtype))
        sums.append(back(m + torch.log(z)))
    return dict(out=outs, lse=sums, positions=positions)


def _plain_adjust(case, s):
    x, req, vocab = s["logits"].float(), s["requests"].long(), case["vocab"]
    if case["penalties"]:
        rows, _, up, place = _padded_trees(s)
        n, at = rows.shape[0], torch.arange(case["history"], device="cuda")[None, :]
        tokens = s["tokens"].long()
        zeros = torch.zeros(n, vocab, device="cuda")
        prompt = zeros.scatter_add(1, tokens, (at < s["prompts"].long()[:, None]).float())
        output = zeros.scatter_add(1, tokens, ((at >= s["prompts"].long()[:, None]) & (at < s["lens"].long()[:, None])).float())
        path = up.float()[place]                                          # [rows, most nodes], in the rows' order
        count = output[req].scatter_add(1, s["drafted"].long()[rows][req], path)
        seen = (prompt[req] > 0.0) | (count > 0.0)
        r = s["repetition"][req][:, None]
        x = torch.where(seen, torch.where(x > 0.0, x / r, x * r), x)
        x = x - count * s["frequency"][req][:, None] - (count > 0.0).float() * s["presence"][req][:, None]
    if case["biases"]:
        owner = torch.arange(case["requests"], device="cuda").repeat_interleave(case["biases"])
        bias = torch.zeros(case["requests"], vocab, device="cuda")
        bias[owner, s["bias_tokens"].long()] = s["bias_values"]
        x = x + bias[req]
    if case["masked"]:
        bits = (s["masks"].long()[:, :, None] >> torch.arange(32, device="cuda")) & 1
        allowed = bits.view(bits.shape[0], -1)[:, :vocab] > 0
        which = s["mask_rows"].long()
        x = torch.where(allowed[which.clamp(min=0)] | (which < 0)[:, None], x, torch.full_like(x, -math.inf))
    if case["in_place"]:
        s["out"].copy_(x)
        return s["out"]
    return x.to(s["logits"].dtype)


def _plain_follow(case, s):
    n_q, n_kv, d, _ = SHAPES[case["shape"]]
    starts, cached = s["starts"].long(), s["cached"].long()
    n, most, rows = starts.numel() - 1, s["most"], s["rows"]
    node = torch.arange(most, device="cuda")
    there = node[None, :] < (starts[1:] - starts[:-1])[:, None]
    at = torch.where(there, starts[:-1, None] + node[None, :], torch.zeros_like(starts[:1, None]))
    parents, tokens, chosen = (s[k].long()[at] for k in ("parents", "tokens", "chosen"))
    last, count = torch.zeros(n, dtype=torch.long, device="cuda"), torch.ones(n, dtype=torch.long, device="cuda")
    path = torch.full((n, most), -1, dtype=torch.long, device="cuda")
    path[:, 0] = 0
    for step in range(1, len(_ints(case["levels"]))):
        fit = there & (parents == last[:, None]) & (tokens == chosen.gather(1, last[:, None]))
        on = fit.any(dim=1) & (count == step)
        last = torch.where(on, fit.float().argmax(dim=1), last)
        path[:, step] = torch.where(on, last, path[:, step])
        count = count + on.long()
    owner = torch.repeat_interleave(torch.arange(n, device="cuda"), starts[1:] - starts[:-1], output_size=rows)
    mine = torch.arange(rows, device="cuda") - starts[owner]
    out = path[owner, mine].to(torch.int32)
    src, dst = cached[owner] + torch.where(out >= 0, out.long(), mine), cached[owner] + mine      # what was not accepted stays where it is
    tables = s["tables"].long()
    sp, dp = tables[owner, src // PAGE], tables[owner, dst // PAGE]
    for pool in s["pool"]:
        k, v = pool[:, :, :PAGE * d].view(-1, n_kv, PAGE, d), pool[:, :, PAGE * d:].view(-1, n_kv, d, PAGE)
        rows_k, rows_v = k[sp, :, src % PAGE].clone(), v[sp, :, :, src % PAGE].clone()
        k[dp, :, dst % PAGE] = rows_k
        v[dp, :, :, dst % PAGE] = rows_v
    i = torch.int32
    return dict(lens=(cached + count).to(i), counts=count.to(i), path=out, next_token=chosen.gather(1, last[:, None])[:, 0].to(i), pool=s["pool"])


# ------------------------------------------------------------------------------------------ the library's calls
_p = torch.Tensor.data_ptr


def _own_norm_rope(case, s):
    from paper_2504_19516_amd import sts
    n_q, n_kv, d, theta = SHAPES[case["shape"]]
    size, base, ld = s["qkv"].element_size(), s["qkv"].data_ptr(), s["qkv"].stride(0)
    norm = sts.HeadNorm(dtype=sts.DTYPES[case["dtype"]], offset_one=case["offset"], eps=EPS, q_gain=_p(s["q_gain"]), k_gain=_p(s["k_gain"]))
    sts.op_norm_rope(norm, sts.Rope(rotary_dim=case["rotary"], interleaved=case["interleaved"], theta=theta), sts.RopeRows(
        dtype=sts.DTYPES[case["dtype"]], rows=case["rows"], n_q=n_q, n_kv=n_kv, d=d, pool_pages=s["pool"].shape[0], q=base, q_stride=ld, q_out=_p(s["q_out"]),
        q_out_stride=n_q * d, k=base + n_q * d * size, k_stride=ld, v=base + (n_q + n_kv) * d * size, v_stride=ld, pool=_p(s["pool"]),
        positions=_p(s["positions"]), places=_p(s["places"])), torch.cuda.current_stream().cuda_stream)
    return dict(q=s["q_out"], pool=s["pool"])


def _own_tree(case, s):
    from paper_2504_19516_amd import sts
    n_q, n_kv, d, _ = SHAPES[case["shape"]]
    stream = torch.cuda.current_stream().cuda_stream
    batch = sts.TreeBatch(dtype=sts.DTYPES[case["dtype"]], n_requests=case["requests"], max_rows=s["rows"], n_q=n_q, n_kv=n_kv, d=d, pool_pages=s["pool"][0].shape[0],
                          max_pages=s["tables"].shape[1], table_stride=s["tables"].stride(0), tables=_p(s["tables"]), cached=_p(s["cached"]), row_starts=_p(s["starts"]),
                          parents=_p(s["parents"]), positions=_p(s["positions"]), workspace=_p(s["workspace"]), workspace_bytes=s["workspace"].numel())
    sts.op_attn_tree_plan(batch, stream)                                  # once a step, for all its layers
    for q, pool, out, lse in zip(s["q"], s["pool"], s["out"], s["lse"]):
        sts.op_attn_tree(batch, q.data_ptr(), n_q * d, pool.data_ptr(), out.data_ptr(), n_q * d, lse.data_ptr(), 0.0, stream)
    return dict(out=s["out"], lse=s["lse"], positions=s["positions"])


def _own_adjust(case, s):
    from paper_2504_19516_amd import sts
    vocab = case["vocab"]
    a = sts.AdjustLogits(dtype=sts.DTYPES[case["dtype"]], rows=s["rows"], vocab=vocab, n_requests=case["requests"], row_stride=vocab, out_stride=vocab, logits=_p(s["logits"]),
                         out=_p(s["out"]), requests=_p(s["requests"]))
    if case["penalties"]:
        a.tokens, a.token_stride, a.lens, a.prompt_lens = _p(s["tokens"]), case["history"], _p(s["lens"]), _p(s["prompts"])
        a.repetition, a.frequency, a.presence = _p(s["repetition"]), _p(s["frequency"]), _p(s["presence"])
        a.row_starts, a.parents, a.drafted = _p(s["starts"]), _p(s["parents"]), _p(s["drafted"])
    if case["biases"]:
        a.bias_starts, a.bias_tokens, a.bias_values = _p(s["bias_starts"]), _p(s["bias_tokens"]), _p(s["bias_values"])
        a.n_biases = s["bias_tokens"].numel()
    if case["masked"]:
        a.masks, a.n_masks, a.mask_stride, a.mask_rows = _p(s["masks"]), s["masks"].shape[0], s["masks"].shape[1], _p(s["mask_rows"])
    sts.op_adjust_logits(a, torch.cuda.current_stream().cuda_stream)
    return s["out"]


def _own_follow(case, s):
    from paper_2504_19516_amd import sts
    n_q, n_kv, d, _ = SHAPES[case["shape"]]
    stream = torch.cuda.current_stream().cuda_stream
    sts.op_tree_accept(sts.TreeAccept(n_requests=case["requests"], max_rows=s["rows"], cached=_p(s["cached"]), row_starts=_p(s["starts"]), parents=_p(s["parents"]), tokens=_p(s["tokens"]),
                                      chosen=_p(s["chosen"]), lens=_p(s["lens"]), counts=_p(s["counts"]), path=_p(s["path"]), next_token=_p(s["next_token"])), stream)
    move = sts.TreeCompact(n_requests=case["requests"], max_rows=s["rows"], n_kv=n_kv, d=d, pool_pages=s["pool"][0].shape[0], max_pages=s["tables"].shape[1], table_stride=s["tables"].stride(0),
                           tables=_p(s["tables"]), cached=_p(s["cached"]), row_starts=_p(s["starts"]), counts=_p(s["counts"]), path=_p(s["path"]))
    sts.op_tree_compact(move, [_p(pool) for pool in s["pool"]], stream)
    return {k: s[k] for k in ("lens", "counts", "path", "next_token", "pool")}


def run(state):
    case = state["case"]
    if own:
        return {"norm_rope": _own_norm_rope, "tree": _own_tree, "adjust": _own_adjust, "follow": _own_follow}[case["op"]](case, state)
    return {"norm_rope": _plain_norm_rope, "tree": _plain_tree, "adjust": _plain_adjust, "follow": _plain_follow}[case["op"]](case, state)


# ------------------------------------------------------------------------------------------ what a pass cannot do without
def _depths(parents):
    out = []
    for p in parents:
        out.append(0 if p < 0 else out[p] + 1)
    return out


def work(case):
    op = case["op"]
    if op == "norm_rope":
        n_q, n_kv, d, _ = SHAPES[case["shape"]]
        return {"bytes": case["rows"] * (2.0 * 2 * (n_q + 2 * n_kv) * d + 8) + 4.0 * d, "flops": case["rows"] * (n_q + n_kv) * (4.0 * d + 3.0 * case["rotary"])}
    if op == "tree":
        n_q, n_kv, d, _ = SHAPES[case["shape"]]
        cached, trees = _trees(case)
        rows = sum(map(len, trees))
        tokens = sum(c + len(t) for c, t in zip(cached, trees))
        pairs = sum(c * len(t) + sum(_depths(t)) + len(t) for c, t in zip(cached, trees))
        return {"bytes": case["layers"] * (4.0 * n_kv * d * tokens + 4.0 * rows * n_q * d + 4.0 * rows * n_q) + 8.0 * rows, "flops": case["layers"] * 4.0 * n_q * d * pairs}
    if op == "adjust":
        size, rows = {"f32": 4, "bf16": 2, "f16": 2}[case["dtype"]], case["requests"] * sum(_ints(case["levels"]))
        vocab, under = case["vocab"], case["masked"] * rows
        words = vocab / 8.0 * min(4.0, under)
        if case["in_place"]:                                              # what is ruled out is written, nothing else changes
            return {"bytes": words + under * vocab * size * 0.9 + 8.0 * rows, "flops": under * vocab}
        return {"bytes": 2.0 * size * rows * vocab + words + case["requests"] * (4.0 * case["history"] + 8.0 * case["biases"]) + 16.0 * rows, "flops": 1.0 * rows * vocab}
    n_q, n_kv, d, _ = SHAPES[case["shape"]]
    rows = case["requests"] * sum(_ints(case["levels"]))
    return {"bytes": 16.0 * rows + case["layers"] * case["requests"] * 2.0 * 4.0 * n_kv * d, "flops": 1.0 * rows}      # a row moved for each request


# ------------------------------------------------------------------------------------------ the same in 64 bits, from the definitions
def _paths(trees):
    """Node numbers from the root to each node, request after request."""
    out = []
    for tree in trees:
        paths = []
        for j, p in enumerate(tree):
            paths.append((paths[p] if p >= 0 else []) + [j])
        out.append(paths)
    return out


def _exact_norm_rope(case, s):
    n_q, n_kv, d, theta = SHAPES[case["shape"]]
    R, rows = case["rotary"], case["rows"]
    y = s["qkv"].double().view(rows, n_q + 2 * n_kv, d).clone()
    for part, gain in ((slice(0, n_q), s["q_gain"]), (slice(n_q, n_q + n_kv), s["k_gain"])):
        scale = gain.double() + float(case["offset"])
        y[:, part] *= scale * torch.rsqrt(y[:, part].square().sum(dim=2, keepdim=True) / d + EPS)
    pairs = torch.arange(R, device="cuda").view(R // 2, 2) if case["interleaved"] else torch.arange(R, device="cuda").view(2, R // 2).t()
    w = theta ** (-torch.arange(0, R, 2, dtype=torch.float64, device="cuda") / R)
    turn = torch.polar(torch.ones(rows, R // 2, dtype=torch.float64, device="cuda"), s["positions"].double()[:, None] * w)
    z = torch.view_as_complex(y[:, :n_q + n_kv][:, :, pairs].contiguous()) * turn[:, None, :]          # a pair is a complex number
    y[:, :n_q + n_kv, pairs.reshape(-1)] = torch.view_as_real(z).flatten(2)
    pool = s["pool"].double()
    k_part, v_part = pool[:, :, :PAGE * d].view(-1, n_kv, PAGE, d), pool[:, :, PAGE * d:].view(-1, n_kv, d, PAGE)
    for slot in range(PAGE):
        at = (s["places"] % PAGE == slot).nonzero()[:, 0]
        page = s["places"][at].long() // PAGE
        k_part[page, :, slot, :] = y[at, n_q:n_q + n_kv]
        v_part[page, :, :, slot] = y[at, n_q + n_kv:]
    return dict(q=y[:, :n_q].reshape(rows, n_q * d), pool=pool)


def _exact_tree(case, s):
    n_q, n_kv, d, _ = SHAPES[case["shape"]]
    cached, trees = _trees(case)
    g, starts, outs, sums = n_q // n_kv, _starts(trees), [], []
    masks = []
    for tree, paths in zip(trees, _paths(trees)):
        m = torch.zeros(len(tree), len(tree), dtype=torch.bool)
        for j, path in enumerate(paths):
            m[j, path] = True
        masks.append(m.cuda())
    for q, pool in zip(s["q"], s["pool"]):
        out, lse = torch.zeros(s["rows"], n_q, d, dtype=torch.float64, device="cuda"), torch.zeros(s["rows"], n_q, dtype=torch.float64, device="cuda")
        for r, (c, mask) in enumerate(zip(cached, masks)):
            m = mask.shape[0]
            got = pool[s["tables"][r, :_pages(c + m)].long()]
            keep = torch.cat([torch.ones(m, c, dtype=torch.bool, device="cuda"), mask], dim=1)
            here = slice(starts[r], starts[r + 1])
            for h in range(n_q):
                page = got[:, h // g]
                k = page[:, :PAGE * d].reshape(-1, d)[:c + m].double()
                v = page[:, PAGE * d:].reshape(-1, d, PAGE).transpose(1, 2).reshape(-1, d)[:c + m].double()
                a = (q[here].view(m, n_q, d)[:, h].double() @ k.t().contiguous() * d ** -0.5).masked_fill(~keep, -math.inf)
                lse[here, h] = torch.logsumexp(a, 1)
                out[here, h] = torch.softmax(a, 1) @ v
        outs.append(out.view(s["rows"], n_q * d))
        sums.append(lse)
    return dict(out=outs, lse=sums, positions=None)


def _exact_adjust(case, s):
    vocab, y = case["vocab"], s["logits"].double()
    rng = _rng(case)
    trees = [_tree(rng, _ints(case["levels"])) for _ in range(case["requests"])]
    if case["penalties"]:
        first = 0
        for i, paths in enumerate(_paths(trees)):
            p, m = int(s["prompts"][i]), int(s["lens"][i])
            told = torch.bincount(s["tokens"][i, p:m], minlength=vocab)
            asked = torch.bincount(s["tokens"][i, :p], minlength=vocab) > 0
            f, w, rep = (s[k][i].double() for k in ("frequency", "presence", "repetition"))
            for path in paths:
                n = told + torch.bincount(s["drafted"][[first + j for j in path]], minlength=vocab)
                at = (asked | (n > 0)).nonzero()[:, 0]
                row = first + path[-1]
                x = y[row, at]
                y[row, at] = torch.where(x > 0, x / rep, x * rep) - n[at] * f - w * (n[at] > 0)
            first += len(paths)
    if case["biases"]:
        for row, i in enumerate(s["requests"].tolist()):
            at = slice(i * case["biases"], (i + 1) * case["biases"])
            y[row, s["bias_tokens"][at].long()] += s["bias_values"][at].double()
    if case["masked"]:
        tokens = torch.arange(vocab, device="cuda")
        banned = [(m[tokens // 32].long() >> (tokens % 32)) % 2 == 0 for m in s["masks"]]
        for row, i in enumerate(s["mask_rows"].tolist()):
            if i >= 0:
                y[row, banned[i]] = -math.inf
    return y


def _exact_follow(case, s):
    """Rows are moved, not computed: the pools alone have values, and these are the old ones in other places."""
    n_q, n_kv, d, _ = SHAPES[case["shape"]]
    cached, trees = _trees(case)
    starts, tokens, chosen, tables = _starts(trees), s["tokens"].tolist(), s["chosen"].tolist(), s["tables"].tolist()
    moves = []
    for r, (c, tree) in enumerate(zip(cached, trees)):
        path, base = [0], starts[r]
        while True:
            nxt = [j for j, p in enumerate(tree) if p == path[-1] and tokens[base + j] == chosen[base + path[-1]]]
            if not nxt:
                break
            path.append(nxt[0])
        moves += [(tables[r][(c + a) // PAGE], (c + a) % PAGE, tables[r][(c + b) // PAGE], (c + b) % PAGE) for b, a in enumerate(path)]
    pools = []
    for pool in s["pool"]:
        old, new = pool.double().view(-1, n_kv, 2 * PAGE * d), pool.double().view(-1, n_kv, 2 * PAGE * d).clone()
        for sp, ss, dp, ds in moves:
            new[dp, :, ds * d:(ds + 1) * d] = old[sp, :, ss * d:(ss + 1) * d]
            new[dp, :, PAGE * d + ds::PAGE] = old[sp, :, PAGE * d + ss::PAGE]
        pools.append(new)
    return dict(lens=None, counts=None, path=None, next_token=None, pool=pools)


def exact(case, seed):
    return {"norm_rope": _exact_norm_rope, "tree": _exact_tree, "adjust": _exact_adjust, "follow": _exact_follow}[case["op"]](case, prepare(case, seed))
