"""Several continuations of one prompt, as cases that can be timed and compared: attention over a prefix that requests share, sampling of
tokens under temperature, top-k, top-p and min-p, and acceptance of a draft tree under the same cuts.

A case is one call through the public entry points of `paper_2507_02620_amd.flowspec`, or (`own` false) the same mathematics in elementary
torch operations.  Three kinds:

* sample: one token per row of logits, from a uniform number per row;
* accept: a draft tree's verified rows of logits, accepted along the tree, from a counter-based generator;
* shared: rows of draft-tree segments (a single token is the smallest) of groups of requests whose contexts begin alike.

Shapes are those of the repository's workloads (the tiny f32 stage, a small grouped-query one, the 7B and the grouped-query 7B shapes with
their vocabularies).

The distribution that is drawn from.  Scores z = logit * (1 / temperature) in 32 bits; weights are whole numbers, the ones acceptance at a
temperature uses: E = trunc(2^32 * e), e = 2^((z - max z) * log2 e) by a fixed polynomial in 32 bits with fused steps, E = 0 below 2^-64 and
for what is not a number.  Order: z descending, then index ascending.  top-k keeps the first k of it; top-p the shortest part of
those whose weights reach ceil(P * sum / 2^30), P = floor(p * 2^30); min-p what weighs at least ceil(min_p * 2^32).  The token is the first kept one by
index whose running sum exceeds floor(U * sum / 2^48), U = floor(u * 2^48).  Temperature 0 keeps the first of the order alone.  Sums are whole
numbers, so that every form draws the same tokens.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

PAGE = 64
#: query heads, KV heads, head dim, element type, vocabulary
SHAPES = {
    "tiny": (4, 4, 64, "f32", 1024),
    "small": (16, 8, 64, "bf16", 32000),
    "7b": (32, 32, 128, "bf16", 32000),
    "gqa": (28, 4, 128, "bf16", 152064),
}
E4M3 = torch.float8_e4m3fn
#: temperature, top-k, top-p, min-p of whole batches
SETTINGS = {
    "plain": (1.0, 0, 1.0, 0.0),
    "top_k": (0.8, 50, 1.0, 0.0),
    "top_p": (1.0, 0, 0.9, 0.0),
    "both": (0.7, 50, 0.95, 0.0),
    "min_p": (1.2, 0, 1.0, 0.05),
    "all": (0.9, 200, 0.95, 0.02),
    "wide": (1.5, 5000, 0.99, 0.0),
}


def listed():
    return [
        # one request of the tiny stage: launches are all there is to it
        dict(name="sample_tiny", kind="sample", rows=1, vocab=1024, dtype="f32", how="top_k"),
        # a serving batch of 7B requests, each with settings of its own
        dict(name="sample_7b_32", kind="sample", rows=32, vocab=32000, dtype="f32", how="mixed"),
        # one request with a large vocabulary: the latency of a decoding step
        dict(name="sample_gqa_1", kind="sample", rows=1, vocab=152064, dtype="f32", how="both"),
        # the first tokens of many samples of a prompt, large vocabulary, settings of all sorts
        dict(name="sample_gqa_64", kind="sample", rows=64, vocab=152064, dtype="f32", how="mixed"),
        # offline generation from 16-bit logits: many equal values, nucleus sampling alone
        dict(name="sample_7b_bf16_200", kind="sample", rows=200, vocab=32000, dtype="bf16", how="top_p"),
        # a 7B request's tree of 64 nodes, all of it verified
        dict(name="accept_7b_64", kind="accept", shape="7b", tree=64, n_ver=64, how="both"),
        # a grouped-query request's tree of 96 nodes, 80 of them verified
        dict(name="accept_gqa_96", kind="accept", shape="gqa", tree=96, n_ver=80, how="top_p"),
        # the tiny f32 stage: three samples of a short prompt
        dict(name="shared_tiny_f32", kind="shared", shape="tiny", groups="3:128", rows=1, own=40, ragged=True),
        # a batch of 32 chats behind one system prompt, a token each
        dict(name="shared_7b_32_tokens", kind="shared", shape="7b", groups="32:2048", rows=1, own=300, ragged=True),
        # sixteen samples of a prompt, a draft segment each, grouped heads
        dict(name="shared_gqa_16_trees", kind="shared", shape="gqa", groups="16:4096", rows=16, own=512, ragged=True),
        # two prompts with samples of each and a request that shares nothing
        dict(name="shared_7b_two_prompts", kind="shared", shape="7b", groups="9:1536,1:0,6:704", rows=24, own=200, ragged=True),
        # eight candidates behind a document, trees of 32 rows: the most work of all
        dict(name="shared_7b_8_trees_16k", kind="shared", shape="7b", groups="8:16384", rows=32, own=128, ragged=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    kind = rng.choice(["sample", "sample", "accept", "shared", "shared", "shared"])
    if kind == "sample":
        vocab = rng.choice([1024, 32000, 152064, _log_int(rng, 100, 152064), _log_int(rng, 100, 152064)])
        rows = _log_int(rng, 1, min(256, 64 * 152064 // vocab))
        return dict(kind=kind, rows=rows, vocab=vocab, dtype=rng.choice(["f32", "f32", "bf16"]), how=rng.choice(["mixed", "mixed", *SETTINGS]))
    if kind == "accept":
        shape = rng.choice(["tiny", "7b", "gqa"])
        tree = _log_int(rng, 4, {"tiny": 512, "7b": 256, "gqa": 64}[shape])
        return dict(kind=kind, shape=shape, tree=tree, n_ver=rng.randint(max(1, tree // 2), tree), how=rng.choice(list(SETTINGS)))
    shape = rng.choice(["tiny", "small", "7b", "7b", "gqa", "gqa"])
    n = rng.choice([1, 1, 1, 2, 3])
    items = [_log_int(rng, 1, 32 // n) for _ in range(n)]
    most = 2048 if shape == "tiny" else 4096 if sum(items) > 8 else 8192
    rows = _log_int(rng, 1, 32 if sum(items) <= 8 else 16)
    groups = [(k, PAGE * (0 if rng.random() < 0.1 else _log_int(rng, 1, most // PAGE // n))) for k in items]
    return dict(kind=kind, shape=shape, groups=",".join("%d:%d" % g for g in groups), rows=rows, own=_log_int(rng, 1, 400), ragged=rng.random() < 0.7)


# ---- what a case's name stands for ---------------------------------------------------------------------------------------

def _groups(case):
    """(items, shared tokens) of each group."""
    return [tuple(int(v) for v in g.split(":")) for g in case["groups"].split(",")]


def _up(n):
    return -(-n // PAGE)


def _requests(case):
    """(l_glo, n_paged, seg_off, rows, group) of each request.  Mostly the whole pages of the context are settled and the rest waits in the
    cache; a quarter has its last, partial page settled too."""
    r = np.random.default_rng([case["rows"], case["own"], sum(n * s for n, s in _groups(case)), 6])
    out = []
    for g, (n, shared) in enumerate(_groups(case)):
        for _ in range(n):
            l = shared + (int(r.integers(0, case["own"] + 1)) if case["ragged"] else case["own"])
            rows = int(r.integers(1, case["rows"] + 1)) if case["ragged"] else case["rows"]
            whole = r.random() < 0.25
            out.append((l, l if whole else l // PAGE * PAGE, int(r.integers(0, 17)) if case["rows"] > 1 else 0, rows, g))
    return out


def _tree(r, n, max_depth=10, max_branch=4):
    """Random parents, each before its children, depth and branching limited."""
    par = np.full(n, -1, dtype=np.int64)
    depth, kids = np.zeros(n, dtype=np.int64), np.zeros(n, dtype=np.int64)
    for i in range(1, n):
        open_ = np.nonzero((depth[:i] < max_depth) & (kids[:i] < max_branch))[0]
        p = int(open_[int(r.integers(0, len(open_)))]) if len(open_) else 0
        par[i], depth[i] = p, depth[p] + 1
        kids[p] += 1
    return par


# ---- inputs ---------------------------------------------------------------------------------------------------------------

def _normal(g, shape, dtype):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, 1.0, generator=g).to(dtype)


def _logits(g, rows, vocab):
    """Rows as a language model's: a broad bulk, some tokens that stand out by more or less, and in one row of eight all but a few hundred
    tokens ruled out by a grammar."""
    x = torch.empty((rows, vocab), dtype=torch.float32, device="cuda").normal_(0.0, 2.0, generator=g)
    k = min(24, vocab)
    at = torch.randint(0, vocab, (rows, k), device="cuda", generator=g)
    peak = torch.rand((rows, 1), device="cuda", generator=g) * 14.0
    x.scatter_add_(1, at, peak / torch.arange(1, k + 1, device="cuda").sqrt())
    ruled = torch.rand((rows, vocab), device="cuda", generator=g) >= min(0.5, 300.0 / vocab)
    some = (torch.arange(rows, device="cuda") % 8 == 5)[:, None]
    return x.masked_fill_(some & ruled, float("-inf"))


def _quantise(rows):
    """[..., 2, heads, 64 tokens, hd] in 32 bits -> (codes [..., 2, heads, 64 * hd] as a page holds them, scales [..., 2, heads])."""
    hd = rows.shape[-1]
    m, e = torch.frexp(rows.abs().amax(dim=(-1, -2)))  # the smallest 2^e with the largest magnitude within 448 * 2^e
    e = e - 9 + (m > 0.875).int()
    c = torch.ldexp(rows, -e[..., None, None]).to(E4M3).view(torch.uint8)
    lead = rows.shape[:-4]
    k, v = c.unbind(dim=len(lead))
    k = k.unflatten(-1, (hd // 64, 64)).transpose(-2, -3)  # [hd / 64][token][64]
    v = v.unflatten(-2, (4, 4, 4)).transpose(-3, -4).flatten(-4, -2).transpose(-1, -2)  # [hd][token's place]
    return torch.stack([k.flatten(-3), v.flatten(-2)], dim=len(lead)), torch.ldexp(torch.ones_like(e, dtype=torch.float32), e)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 2 + 1)
    r = np.random.default_rng([int(seed) & 0x7FFFFFFF, 79])
    x = {"case": case}
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    if case["kind"] == "sample":
        rows = case["rows"]
        x["logits"] = _logits(g, rows, case["vocab"]).to(torch.float32 if case["dtype"] == "f32" else torch.bfloat16)
        x["u"] = torch.rand(rows, dtype=torch.float64, device="cuda", generator=g)
        if case["how"] == "mixed":  # every request has its own settings, in device memory
            x["how"] = (dev(r.choice([0.0, 0.6, 0.7, 0.8, 1.0, 1.0, 1.3], rows).astype(np.float32)), dev(r.choice([0, 0, 20, 50, 1000], rows).astype(np.int32)),
                        dev(r.choice([1.0, 0.95, 0.9, 0.5], rows).astype(np.float32)), dev(r.choice([0.0, 0.0, 0.05, 0.1], rows).astype(np.float32)))
        else:
            x["how"] = SETTINGS[case["how"]]
        return x
    hq, hkv, hd, dt, vocab = SHAPES[case["shape"]]
    if case["kind"] == "accept":
        T, n_ver = case["tree"], case["n_ver"]
        par = _tree(r, T)
        x["logits"] = _logits(g, n_ver, vocab)
        # a draft model's tokens: what stands out in the parent's row, or not
        tok = r.integers(0, vocab, T)
        for i in range(1, T):
            while tok[i] in tok[1:i][par[1:i] == par[i]]:
                tok[i] = int(r.integers(0, vocab))
        kids = np.nonzero((par >= 0) & (par < n_ver))[0]
        x["logits"][dev(par[kids]), dev(tok[kids])] = dev(r.uniform(8.0, 20.0, len(kids)).astype(np.float32))
        x["token"], x["parent"], x["depth"] = dev(tok.astype(np.int32)), dev(par.astype(np.int32)), _depth(par)
        x["seed"], x["step"] = int(r.integers(0, 1 << 62)), int(r.integers(0, 1 << 20))
        x["how"] = SETTINGS[case["how"]]
        x["res"] = torch.zeros(6, dtype=torch.int32, device="cuda")
        x["retain"] = torch.full((T,), -1, dtype=torch.int32, device="cuda")
        return x
    dt = torch.float32 if dt == "f32" else torch.bfloat16
    reqs, groups = _requests(case), _groups(case)
    P = max(1, max(_up(p) for _, p, _, _, _ in reqs))
    n = sum(s // PAGE for _, s in groups) + sum(_up(p) - groups[i][1] // PAGE for _, p, _, _, i in reqs)
    order, at = r.permutation(max(n, 1)), 0
    table, first = np.full((len(reqs), P), -1, np.int32), []
    for i, (_, p, _, _, gi) in enumerate(reqs):
        s = groups[gi][1] // PAGE
        if gi == len(first):  # the group's first request: the pages that all of it share
            first.append(order[at:at + s])
            at += s
        table[i, :s] = first[gi]
        table[i, s:_up(p)] = order[at:at + _up(p) - s]
        at += _up(p) - s
    n = max(n, 1)
    x["codes"] = torch.empty((n, 1, 2, hkv, PAGE * hd), dtype=torch.uint8, device="cuda")
    x["scales"] = torch.empty((n, 1, 2, hkv), dtype=torch.float32, device="cuda")
    for a in range(0, n, 64):
        b = min(n, a + 64)
        x["codes"][a:b], x["scales"][a:b] = _quantise(_normal(g, (b - a, 1, 2, hkv, PAGE, hd), torch.float32))
    x["table"] = dev(table)
    x["length"] = dev(np.array([p for _, p, _, _, _ in reqs], np.int32))
    x["ref"] = dev(np.bincount(table[table >= 0], minlength=n).astype(np.int32))
    cap = max(l - p + o + m for l, p, o, m, _ in reqs)
    x["tail"] = _normal(g, (len(reqs), 1, 2, hkv, cap, hd), dt)
    rows = sum(m for _, _, _, m, _ in reqs)
    x["q"] = _normal(g, (rows, hq, hd), dt)
    anc, at = np.zeros((rows, 1024), dtype=bool), 0
    for _, _, o, m, _ in reqs:
        par, seen = _tree(r, o + m), np.zeros((o + m, o + m), dtype=bool)
        for j in range(o + m):
            if par[j] >= 0:
                seen[j] = seen[par[j]]
            seen[j, j] = True
        anc[at:at + m, :o + m] = seen[o:]
        at += m
    x["anc"] = dev(np.packbits(anc, axis=1, bitorder="little").view(np.int64))
    x["reqs"], x["groups"] = reqs, groups
    # for the padded form: request and row in it of every stacked row; lengths; the request whose pages hold what is shared
    M = max(m for _, _, _, m, _ in reqs)
    start = np.cumsum([0] + [m for _, _, _, m, _ in reqs])
    x["row"] = dev(np.array([[start[i] + min(j, m - 1) for j in range(M)] for i, (_, _, _, m, _) in enumerate(reqs)], np.int64))
    x["back"] = dev(np.array([i * M + j for i, (_, _, _, m, _) in enumerate(reqs) for j in range(m)], np.int64))
    x["lens"] = dev(np.array([q[:4] for q in reqs], np.int64))
    lead = np.cumsum([0] + [k for k, _ in groups])
    x["lead"] = dev(np.array([lead[q[4]] for q in reqs], np.int64))
    x["prefix"] = dev(np.array([groups[q[4]][1] // PAGE for q in reqs], np.int64))
    return x


def _depth(par):
    d = np.zeros(len(par), dtype=np.int64)
    for i in range(1, len(par)):
        d[i] = d[par[i]] + 1
    return int(d.max()) + 1


# ---- one pass ------------------------------------------------------------------------------------------------------------------

def run(state):
    if own:
        return _run_own(state)
    return {"sample": _plain_sample, "accept": _plain_accept, "shared": _plain_shared}[state["case"]["kind"]](state)


def _run_own(x):
    from paper_2507_02620_amd import flowspec as fs
    kind = x["case"]["kind"]
    if kind == "sample":
        if "work" not in x:  # scratch that a program keeps
            x["work"] = fs.sample_workspace(x["logits"].shape[0], x["logits"].shape[1])
        token, logprob, kept = fs.sample_tokens(x["logits"], x["u"], *x["how"], workspace=x["work"])
        return {"token": token, "logprob": logprob, "kept": kept}
    if kind == "accept":
        if "work" not in x:
            x["work"] = fs.sample_workspace(x["logits"].shape[0], x["logits"].shape[1])
        fs.tree_accept_filtered(x["logits"], *x["how"], x["token"], x["parent"], x["case"]["n_ver"], x["seed"], x["step"], x["res"], x["retain"],
                                workspace=x["work"])
        return {"result": x["res"], "retain": x["retain"]}
    if "pool" not in x:  # the handle over the pool's tensors, which a program keeps; items, groups and scratch serve every layer of a step
        x["pool"] = fs.PagePool.of(x["codes"], x["scales"], x["ref"], x["table"], x["length"])
        x["items"] = fs.paged_items([(i, p, x["tail"][i], l, o, m) for i, (l, p, o, m, _) in enumerate(x["reqs"])])
        x["prefixes"] = fs.prefix_groups(x["groups"])
        x["work"] = fs.shared_attention_workspace(x["pool"], x["q"].shape[1], x["q"].shape[0])
    return fs.shared_attention(x["pool"], 0, x["q"], x["items"], x["prefixes"], anc=x["anc"], workspace=x["work"])


# ---- the plain forms -------------------------------------------------------------------------------------------------------

#: 2^f on [0, 1], Horner from the highest power on, each step fused: p * f + c rounded once
POLY = (1.52527338e-5, 1.54035304e-4, 1.33335581e-3, 9.61812911e-3, 5.55041087e-2, 2.40226507e-1, 6.93147181e-1, 1.0)


def _weights(z):
    """Whole-number weights of scores [rows, vocab] in 32 bits; all 0 in a row without a score above -inf."""
    z = torch.where(torch.isnan(z), float("-inf"), z)
    m = z.amax(dim=-1, keepdim=True)
    t = torch.where(z == m, 0.0, (z - m) * torch.tensor(1.44269504088896341, dtype=torch.float32, device=z.device))
    n = torch.floor(t)
    f = (t - n).double()
    p = torch.full_like(t, POLY[0])
    for c in POLY[1:]:  # the product is exact in 64 bits, so one rounding to 64 and one to 32 bits stand for the fused one's
        p = (p.double() * f + float(np.float32(c))).float()
    e = torch.floor(torch.ldexp(p.double(), (n + 32.0).clamp_min(-40.0))).long()
    return torch.where((t >= -64.0) & (m > float("-inf")), e, 0)


def _part(a, bits, s):
    """floor(a * s / 2^bits), a < 2^bits, s < 2^52, without leaving 64 bits: bits is 30 or 48."""
    if bits == 30:
        return a * (s >> 30) + ((a * (s & 0x3FFFFFFF)) >> 30)
    ah, al, sh, sl = a >> 24, a & 0xFFFFFF, s >> 25, s & 0x1FFFFFF
    return 2 * ah * sh + ((ah * sl + 2 * al * sh + ((al * sl) >> 24)) >> 24)


def _column(v, rows, dtype, device):
    return (v.to(dtype) if isinstance(v, torch.Tensor) else torch.full((rows,), v, dtype=dtype, device=device))[:, None]


def _cut(logits, how):
    """(weights [rows, vocab] of what is kept, 0 elsewhere, in index order)."""
    rows, vocab = logits.shape
    temp, k, p, mp = (_column(v, rows, dt, logits.device) for v, dt in zip(how, (torch.float32, torch.int64, torch.float32, torch.float32)))
    greedy = temp == 0
    z = logits.float() * torch.where(greedy, 1.0, 1.0 / torch.where(greedy, 1.0, temp))
    w = _weights(z)
    k = torch.where(greedy, 1, torch.where(k > 0, k, vocab))
    order = torch.sort(torch.where(torch.isnan(z), float("-inf"), z), dim=1, descending=True, stable=True).indices
    ranked = torch.where(torch.arange(vocab, device=z.device)[None, :] < k, w.gather(1, order), 0)
    upto = torch.cumsum(ranked, dim=1)
    P = torch.floor(p.double().clamp(0.0, 1.0) * 2.0 ** 30).long()
    need = torch.where(P < (1 << 30), upto[:, -1:] - _part((1 << 30) - P, 30, upto[:, -1:]), upto[:, -1:])  # ceil(P S / 2^30)
    ranked = torch.where(upto - ranked < need.clamp_min(1), ranked, 0)
    ranked = torch.where(ranked >= torch.ceil(mp.double().clamp(0.0, 1.0) * 2.0 ** 32).long(), ranked, 0)
    return torch.zeros_like(w).scatter_(1, order, ranked)


def _plain_sample(x):
    w = _cut(x["logits"], x["how"])
    upto = torch.cumsum(w, dim=1)
    total = upto[:, -1:]
    U = torch.floor(x["u"] * 2.0 ** 48).long()[:, None]
    token = torch.searchsorted(upto, _part(U, 48, total), right=True)
    at = token.clamp_max(w.shape[1] - 1)
    any_ = total > 0
    logprob = torch.log(w.gather(1, at).double() / total.double().clamp_min(1.0))
    return {"token": torch.where(any_, token, -1).int()[:, 0], "logprob": torch.where(any_, logprob, float("-inf")).float()[:, 0],
            "kept": (w > 0).sum(dim=1).int()}


def _wrap(v):
    """A constant of 64 bits as torch's signed numbers hold it."""
    return v - (1 << 64) if v >= 1 << 63 else v


def _random24(seed, step, draws):
    """The generator's upper 24 bits for the draws numbered `draws` (64-bit products wrap; shifts bring zeros in)."""
    down = lambda z, k: (z >> k) & ((1 << (64 - k)) - 1)
    z = draws * _wrap(0xBF58476D1CE4E5B9)
    z = z ^ _wrap((seed ^ (step * 0x9E3779B97F4A7C15)) & ((1 << 64) - 1))
    z = (z ^ down(z, 30)) * _wrap(0xBF58476D1CE4E5B9)
    z = (z ^ down(z, 27)) * _wrap(0x94D049BB133111EB)
    return down(z ^ down(z, 31), 40)


def _plain_accept(x):
    case, token, parent = x["case"], x["token"].long(), x["parent"].long()
    T, n_ver = case["tree"], case["n_ver"]
    w = _cut(x["logits"], x["how"])
    total = w.sum(dim=1)
    nodes = torch.arange(T, device=token.device)
    under = (parent >= 0) & (parent < n_ver)
    mine = torch.where(under, w[parent.clamp(0, n_ver - 1), token], 0)
    u, draws, alive = torch.zeros_like(nodes[0]), torch.zeros_like(nodes[0]), torch.ones_like(nodes[0]).bool()
    path = nodes == 0
    n_new, last = torch.full_like(u, -1), u
    struck = torch.zeros(w.shape[1], dtype=torch.int32, device=w.device)
    for _ in range(x["depth"]):  # a step down the tree per turn; siblings carry different tokens
        kid = (parent == u) & alive
        rank = torch.cumsum(kid, 0) - 1
        left = total[u] - torch.cumsum(torch.where(kid, mine, 0), 0) + mine
        r24 = _random24(x["seed"], x["step"], draws + rank)
        took = kid & (r24 * (left >> 24) + ((r24 * (left & 0xFFFFFF)) >> 24) < mine)
        first = torch.where(took, nodes, T).amin()
        down = alive & (first < n_ver)
        ends = alive & (first >= n_ver)
        n_new = torch.where(ends & (first < T), first, n_new)
        struck = struck.index_add(0, token, (kid & ends).int())
        draws = draws + torch.where(took.any(), rank[first.clamp_max(T - 1)] + 1, kid.sum())
        last = torch.where(ends, u, last)
        path = path | (down & (nodes == first))
        u = torch.where(down, first, u)
        alive = down
    # the draw from what is left under the last accepted node
    rest = torch.where(struck > 0, 0, w[last])
    upto = torch.cumsum(rest, 0)
    U = (_random24(x["seed"], x["step"], draws) << 24) | _random24(x["seed"], x["step"], draws + 1)
    drawn = torch.searchsorted(upto, _part(U, 48, upto[-1])[None], right=True)[0].clamp_max(w.shape[1] - 1)
    goes_on = n_new >= 0
    x_new = torch.where(goes_on, token[n_new.clamp_min(0)], drawn)
    below = (nodes == n_new) & goes_on
    for _ in range(x["depth"]):
        below = below | (below[parent.clamp_min(0)] & (parent >= 0))
    keep = path | below
    res = torch.stack([path.sum(), x_new, n_new, goes_on.long(), keep.sum(), (below & (nodes < n_ver)).sum()]).int()
    held = torch.sort((~keep).int(), stable=True).indices
    return {"result": res, "retain": torch.where(nodes < keep.sum(), held, -1).int()}


def _values(codes, scales, hd):
    """Pages [..., 2, heads, 64 * hd] -> (K, V) [..., heads, 64 tokens, hd] in 32 bits."""
    w = codes.view(E4M3).float() * scales[..., None]
    k, v = w.unbind(dim=-3)
    k = k.unflatten(-1, (hd // 64, PAGE, 64)).transpose(-2, -3).flatten(-2)
    v = v.unflatten(-1, (hd, 4, 4, 4)).transpose(-2, -3).flatten(-3).transpose(-1, -2)
    return k, v


def _plain_shared(x):
    q, tail, lens = x["q"], x["tail"], x["lens"]
    n, _, _, hkv, cap, hd = tail.shape
    rows, hq, _ = q.shape
    l, paged, off, m = (lens[:, i] for i in range(4))
    held = torch.arange(x["table"].shape[1], device=q.device)[None, :] < x["prefix"][:, None]
    pages = torch.where(held, x["table"][x["lead"]], x["table"]).long().clamp_min(0)
    k, v = _values(x["codes"][pages, 0], x["scales"][pages, 0], hd)  # [n, P, hkv, 64, hd]
    k, v = (torch.cat([w.transpose(1, 2).flatten(2, 3), t.float()], dim=2) for w, t in ((k, tail[:, 0, 0]), (v, tail[:, 0, 1])))
    settled = torch.arange(pages.shape[1] * PAGE, device=q.device)[None, :] < paged[:, None]
    slot = torch.arange(cap, device=q.device)[None, :] + paged[:, None]
    bits = ((x["anc"][:, :, None] >> torch.arange(64, device=q.device)) & 1).flatten(1).bool()[x["row"]]  # [n, M, 1024]
    M = bits.shape[1]
    draft = (slot - l[:, None]).clamp(0, 1023)[:, None, :].expand(n, M, cap)
    newest = (slot < (l + off + m)[:, None])[:, None, :]
    seen = newest & ((slot < l[:, None])[:, None, :] | bits.gather(2, draft))
    seen = torch.cat([settled[:, None, :].expand(n, M, settled.shape[1]), seen], dim=2)
    G = hq // hkv
    qs = q.float()[x["row"]].view(n, M, hkv, G, hd).permute(0, 2, 3, 1, 4).reshape(n, hkv, G * M, hd)
    s = torch.matmul(qs, k.transpose(-1, -2)) / math.sqrt(hd)
    s = torch.where(seen[:, None, None].expand(n, hkv, G, M, seen.shape[2]).reshape(n, hkv, G * M, -1), s, float("-inf"))
    p = torch.exp(s - s.amax(dim=-1, keepdim=True))  # (every row sees itself)
    o = torch.matmul(p / p.sum(dim=-1, keepdim=True), v)
    o = o.view(n, hkv, G, M, hd).permute(0, 3, 1, 2, 4).reshape(n * M, hq, hd)
    return o[x["back"]].to(q.dtype)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------------------

def work(case):
    if case["kind"] == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * (4 if case["dtype"] == "f32" else 2) + case["rows"] * 36, "flops": 20 * n}
    hq, hkv, hd, dt, vocab = SHAPES[case["shape"]]
    if case["kind"] == "accept":
        return {"bytes": case["n_ver"] * vocab * 4 + case["tree"] * 12 + 24, "flops": 20 * case["n_ver"] * vocab}
    e = 4 if dt == "f32" else 2
    reqs, groups = _requests(case), _groups(case)
    page = 2 * hkv * (PAGE * hd + 4)
    byt = sum(s // PAGE for _, s in groups) * page
    flops = 0
    for l, p, o, m, g in reqs:
        byt += (_up(p) - groups[g][1] // PAGE) * page + 2 * hkv * (l - p + o + m) * hd * e + 2 * m * hq * hd * e
        flops += 4 * hd * hq * m * (l + (o + m) // 2)
    return {"bytes": byt, "flops": flops}


# ---- the same from the definitions, on the host in whole numbers or in 64 bits -------------------------------------------------------

def _weigh64(z):
    """Weights of one row of scores (numpy, 32 bits), whole numbers; sums of a fused step are formed in extended precision and rounded once."""
    fine = z[~np.isnan(z)]
    m = fine.max() if fine.size else np.float32(-np.inf)
    w = np.zeros(z.shape, dtype=np.int64)
    if m == -np.inf:
        return w
    with np.errstate(invalid="ignore", over="ignore"):
        t = ((z - m).astype(np.float32) * np.float32(1.44269504088896341)).astype(np.float32)
    t[z == m] = 0
    ok = t >= -64.0
    t = t[ok]
    n = np.floor(t)
    f = (t - n).astype(np.longdouble)
    p = np.full(t.shape, np.float32(POLY[0]))
    for c in POLY[1:]:
        p = (p.astype(np.longdouble) * f + np.longdouble(np.float32(c))).astype(np.float32)
    mant, ex = np.frexp(p)
    sig, sh = (mant * 2.0 ** 24).astype(np.int64), (ex - 24 + 32 + n.astype(np.int64)).astype(np.int64)  # E = sig * 2^sh, cut
    w[ok] = np.where(sh >= 0, sig << sh.clip(0), sig >> (-sh).clip(0, 62))
    return w


def _cut64(row, how):
    """What is kept of one row, in whole numbers of any size."""
    temp, k, p, mp = how
    z = row if temp == 0 else row * (np.float32(1.0) / np.float32(temp))
    w = _weigh64(z.astype(np.float32))
    order = np.lexsort((np.arange(len(z)), -np.where(np.isnan(z), -np.inf, z)))
    if temp == 0 or k > 0:
        order = order[:1 if temp == 0 else k]
    run = np.cumsum(w[order])
    P = int(math.floor(min(max(float(np.float32(p)), 0.0), 1.0) * 2 ** 30))
    need = max(1, -((-P * int(run[-1])) >> 30))
    order = order[:int(np.searchsorted(run, need, side="left")) + 1]
    least = math.ceil(min(max(float(np.float32(mp)), 0.0), 1.0) * 2 ** 32)
    out = np.zeros_like(w)
    out[order] = np.where(w[order] >= least, w[order], 0)
    return out


def _draw64(w, U):
    run = np.cumsum(w)
    return min(int(np.searchsorted(run, (U * int(run[-1])) >> 48, side="right")), len(w) - 1)


def _mix64(seed, step, k):
    full = (1 << 64) - 1
    z = (seed ^ (step * 0x9E3779B97F4A7C15) ^ (k * 0xBF58476D1CE4E5B9)) & full
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & full
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & full
    return (z ^ (z >> 31)) >> 40


def exact(case, seed):
    x = prepare(case, seed)
    if case["kind"] == "sample":
        rows, u = x["logits"].float().cpu().numpy(), x["u"].cpu().numpy()
        how = [v.cpu().numpy() if isinstance(v, torch.Tensor) else np.full(len(u), v) for v in x["how"]]
        token, logprob, kept = [], [], []
        for i, row in enumerate(rows):
            w = _cut64(row, [v[i] for v in how])
            total = int(w.sum())
            token.append(_draw64(w, int(math.floor(u[i] * 2 ** 48))) if total else -1)
            logprob.append(math.log(int(w[token[-1]]) / total) if total else -math.inf)
            kept.append(int((w > 0).sum()))
        return {"token": np.array(token, np.int32), "logprob": np.array(logprob), "kept": np.array(kept, np.int32)}
    if case["kind"] == "accept":
        lg, tok, par = x["logits"].cpu().numpy(), x["token"].cpu().numpy(), x["parent"].cpu().numpy()
        T, n_ver, u, acc, n_new, draws = case["tree"], case["n_ver"], 0, [0], -1, 0
        while True:
            w = _cut64(lg[u], x["how"])
            left, nxt = int(w.sum()), -1
            for c in np.nonzero(par == u)[0]:
                r, draws = _mix64(x["seed"], x["step"], draws), draws + 1
                if r * left < int(w[tok[c]]) << 24:
                    nxt = int(c)
                    break
                left -= int(w[tok[c]])
                w[tok[c]] = 0
            if nxt < 0:
                x_new = _draw64(w, (_mix64(x["seed"], x["step"], draws) << 24) | _mix64(x["seed"], x["step"], draws + 1))
                break
            if nxt >= n_ver:
                x_new, n_new = int(tok[nxt]), nxt
                break
            u = nxt
            acc.append(u)
        below = []
        for i in range(T):
            if n_new >= 0 and (i == n_new or par[i] in below):
                below.append(i)
        held = sorted(acc + below)
        res = [len(acc), x_new, n_new, int(n_new >= 0), len(held), sum(i < n_ver for i in below)]
        return {"result": np.array(res, np.int32), "retain": np.array(held + [-1] * (T - len(held)), np.int32)}
    hd, hkv = x["q"].shape[2], x["tail"].shape[3]
    group = x["q"].shape[1] // hkv
    place = torch.tensor([16 * ((t >> 2) & 3) + 4 * (t >> 4) + (t & 3) for t in range(PAGE)], device="cuda")
    table, out, at = x["table"].cpu().numpy(), [], 0
    bits = np.unpackbits(x["anc"].cpu().numpy().view(np.uint8), axis=1, bitorder="little").astype(bool)

    def rows_of(ids):
        """(K, V) [heads, 64 * pages, hd]"""
        ids = torch.from_numpy(np.asarray(ids, dtype=np.int64)).cuda()
        w = x["codes"][ids, 0].view(E4M3).double() * x["scales"][ids, 0].double()[..., None]
        k = torch.cat([w[:, 0].view(len(ids), hkv, hd // 64, PAGE, 64)[:, :, a] for a in range(hd // 64)], dim=3)
        v = w[:, 1].view(len(ids), hkv, hd, PAGE)[..., place].transpose(2, 3)
        return (t.transpose(0, 1).reshape(hkv, len(ids) * PAGE, hd) for t in (k, v))

    lead = np.cumsum([0] + [n for n, _ in x["groups"]])
    common = None
    for i, (l, p, o, m, g) in enumerate(x["reqs"]):
        shared = x["groups"][g][1]
        if i == lead[g]:
            common = tuple(rows_of(table[i, :shared // PAGE]))
        mine = tuple(t[:, :p - shared] for t in rows_of(table[i, shared // PAGE:_up(p)]))
        L = l + o + m
        seen = np.ones((m, L - shared), dtype=bool)
        seen[:, l - shared:] = bits[at:at + m, :o + m]
        seen = torch.from_numpy(seen).cuda()
        ks, vs = (torch.cat([mine[j], x["tail"][i, 0, j, :, :L - p].double()], dim=1) for j in (0, 1))
        q = x["q"][at:at + m].double().view(m, hkv, group, hd).permute(1, 2, 0, 3).reshape(hkv, group * m, hd)
        far = torch.exp(torch.bmm(q, common[0].transpose(1, 2).contiguous()) / math.sqrt(hd))  # (scores are moderate: no maximum needed in 64 bits)
        near = torch.exp(torch.bmm(q, ks.transpose(1, 2).contiguous()) / math.sqrt(hd)) * seen.repeat(group, 1)
        got = (torch.bmm(far, common[1].contiguous()) + torch.bmm(near, vs.contiguous())) / (far.sum(dim=2, keepdim=True) + near.sum(dim=2, keepdim=True))
        out.append(got.view(hkv, group, m, hd).permute(2, 0, 1, 3).reshape(m, hkv * group, hd))
        at += m
    return torch.cat(out)
