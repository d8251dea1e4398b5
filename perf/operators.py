"""The operators over prompts and over a cache of 8-bit pages, as cases that can be timed and compared.

A case is one call sequence through the public entry points of `paper_2507_02620_amd.flowspec`, or (`own` false) the same mathematics
in elementary torch operations.  Four kinds:

* prompt: causal attention over whole prompts packed behind one another, grouped heads;
* store: token rows of the 16- or 32-bit cache into pages of 64 tokens, e4m3 with a power-of-two scale per page, layer, K or V, head;
* paged: rows of draft-tree segments (a single token is the smallest) against a context in such pages, its newest slots in the cache;
* pages: forking, freeing and compacting of the sequences that share a pool of pages.

Shapes are those of the repository's workloads (the tiny f32 stage, a small grouped-query one, the 7B and the grouped-query 7B
shapes).  Inputs stand in for real ones the way `synth.py` does: queries, keys and values N(0, 1).

A page holds, per layer, K as [hd / 64][64 tokens][64 columns] and V as [hd][64 tokens], V's tokens t = 16 a + 4 b + c at place
16 b + 4 a + c of a row.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

PAGE = 64
#: query heads, KV heads, head dim, element type
SHAPES = {
    "tiny": (4, 4, 64, "f32"),
    "small": (16, 8, 64, "bf16"),
    "7b": (32, 32, 128, "bf16"),
    "gqa": (28, 4, 128, "bf16"),
}
E4M3 = torch.float8_e4m3fn


def listed():
    return [
        # the smallest prompts of the f32 parity stage, one of a single token: launches are all there is to it
        dict(name="prompt_tiny_f32", kind="prompt", shape="tiny", lens="1,17,160"),
        # short chat turns packed together, grouped heads of 64
        dict(name="prompt_small_packed", kind="prompt", shape="small", lens="5,129,300,64,1,210"),
        # ragged prompts of a 7B model in one call
        dict(name="prompt_7b_packed", kind="prompt", shape="7b", lens="389,1,1024,77,555"),
        # two long prompts, seven query heads to a KV head
        dict(name="prompt_gqa_4k", kind="prompt", shape="gqa", lens="2600,1496"),
        # one document-length prompt, the most work of all
        dict(name="prompt_7b_8k", kind="prompt", shape="7b", lens="8192"),
        # the page that a request has just completed and a partial one, a shallow stage
        dict(name="store_small_2", kind="store", shape="small", layers=2, tokens="64,29"),
        # a prompt moves into pages once its prefill is done
        dict(name="store_7b_1500", kind="store", shape="7b", layers=4, tokens="1500"),
        # one token of one request behind a context of about a thousand: the latency of a serving step
        dict(name="paged_7b_one_token", kind="paged", shape="7b", reqs=1, rows=1, l_glo=1000, ragged=False),
        # a serving batch: one token for each of 32 requests with contexts of all lengths up to 4096
        dict(name="paged_gqa_32_tokens", kind="paged", shape="gqa", reqs=32, rows=1, l_glo=4096, ragged=True),
        # a draft tree of 64 nodes behind a long context: attention carries weight
        dict(name="paged_7b_tree_16k", kind="paged", shape="7b", reqs=1, rows=64, l_glo=16384, ragged=False),
        # candidates of a search: 16 children dropped and forked anew from their parents
        dict(name="fork_7b_16", kind="fork", shape="7b", layers=4, pages=256, parents=4, children=16, tokens=900),
        # a fragmented pool made dense again
        dict(name="compact_gqa_1024", kind="compact", shape="gqa", layers=7, pages=1024, seqs=24, tokens=1800),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "prompt", "paged", "paged", "paged", "store", "fork", "compact"])
    shape = rng.choice(["tiny", "small", "7b", "7b", "gqa", "gqa"])
    if kind == "prompt":
        total = _log_int(rng, 1, 1024 if shape == "tiny" else 6000)
        n = rng.randint(1, max(1, min(9, total)))
        cuts = sorted(rng.sample(range(1, total), n - 1)) if n > 1 else []
        lens = [b - a for a, b in zip([0] + cuts, cuts + [total])]
        return dict(kind=kind, shape=shape, lens=",".join(map(str, lens)))
    if kind == "store":
        n = rng.randint(1, 4)
        return dict(kind=kind, shape=shape, layers=rng.randint(1, 4), tokens=",".join(str(_log_int(rng, 1, 1500 // n)) for _ in range(n)))
    if kind == "paged":
        reqs = rng.choice([1, 1, 2, rng.randint(2, 32)])
        rows = _log_int(rng, 1, 64 if reqs <= 2 else 16)
        most = 8192 if reqs <= 2 else 4096 if SHAPES[shape][1] <= 8 else 512
        return dict(kind=kind, shape=shape, reqs=reqs, rows=rows, l_glo=_log_int(rng, 1, most), ragged=rng.random() < 0.7)
    if kind == "fork":
        return dict(kind=kind, shape=shape, layers=rng.randint(1, 4), pages=rng.randint(200, 256), parents=rng.randint(1, 6),
                    children=rng.randint(1, 16), tokens=_log_int(rng, 1, 1000))
    seqs = rng.randint(1, 20)
    return dict(kind=kind, shape=shape, layers=rng.randint(1, 3), pages=rng.randint(400, 700), seqs=seqs, tokens=_log_int(rng, 64, 1800))


# ---- what a case's name stands for ---------------------------------------------------------------------------------------

def _dtype(case):
    return torch.float32 if SHAPES[case["shape"]][3] == "f32" else torch.bfloat16


def _ints(text):
    return [int(v) for v in text.split(",")]


def _up(n):
    return -(-n // PAGE)


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


def _requests(case):
    """(l_glo, n_paged, seg_off, rows) of each request.  Mostly the whole pages of the context are settled and the rest waits in the
    cache; a quarter has its last, partial page settled too."""
    r = np.random.default_rng([case["reqs"], case["rows"], case["l_glo"], 5])
    out = []
    for _ in range(case["reqs"]):
        l = int(r.integers(max(1, case["l_glo"] // 8), case["l_glo"] + 1)) if case["ragged"] else case["l_glo"]
        rows = int(r.integers(1, case["rows"] + 1)) if case["ragged"] else case["rows"]
        whole = case["reqs"] > 1 and r.random() < 0.25
        out.append((l, l if whole else l // PAGE * PAGE, int(r.integers(0, 33)) if case["rows"] > 1 else 0, rows))
    return out


def _pool_plan(case):
    """Tables, lengths and reference counts of the page cases, and the lists of their calls, on the host."""
    n = case["pages"]
    r = np.random.default_rng([n, case["layers"], case["tokens"], 9])
    order = r.permutation(n)
    if case["kind"] == "fork":
        seqs, width = case["parents"] + case["children"], _up(case["tokens"]) + 1
        table, length, ref, at = np.full((seqs, width), -1, np.int32), np.zeros(seqs, np.int32), np.zeros(n, np.int32), 0
        for s in range(case["parents"]):
            length[s] = int(r.integers(max(1, case["tokens"] // 2), case["tokens"] + 1))
            k = _up(int(length[s]))
            table[s, :k] = order[at:at + k]
            ref[table[s, :k]] = 1
            at += k
        was = r.integers(0, case["parents"], case["children"])  # what the children were forked from before
        for i, p in enumerate(was):
            s, k, full = case["parents"] + i, _up(int(length[p])), int(length[p]) // PAGE
            table[s, :full] = table[p, :full]
            ref[table[s, :full]] += 1
            if k > full:
                table[s, full] = order[at]
                ref[order[at]] = 1
                at += 1
            length[s] = length[p]
        src = r.integers(0, case["parents"], case["children"]).astype(np.int32)
        dst = (case["parents"] + np.arange(case["children"])).astype(np.int32)
        return table, length, ref, src, dst
    seqs, width = case["seqs"], _up(case["tokens"])
    table, length, ref, at = np.full((seqs, width), -1, np.int32), np.zeros(seqs, np.int32), np.zeros(n, np.int32), 0
    for s in range(seqs):
        k = min(_up(int(r.integers(max(1, case["tokens"] // 2), case["tokens"] + 1))), n - at)
        table[s, :k] = order[at:at + k]
        ref[order[at:at + k]] = 1
        length[s] = k * PAGE - int(r.integers(0, PAGE)) if k else 0
        at += k
    # the second half of the sequences shares the first pages of its neighbour in the first half
    for s in range(seqs // 2, seqs):
        k = min(int(length[s]) // PAGE, int(length[s - seqs // 2]) // PAGE) // 2
        ref[table[s, :k]] -= 1
        table[s, :k] = table[s - seqs // 2, :k]
        ref[table[s, :k]] += 1
    return table, length, ref, None, None


# ---- inputs ---------------------------------------------------------------------------------------------------------------

def _normal(g, shape, dtype):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, 1.0, generator=g).to(dtype)


def _codes(g, shape):
    """Finite e4m3 codes of both signs."""
    c = torch.randint(0, 254, shape, dtype=torch.uint8, device="cuda", generator=g)
    return torch.where(c >= 127, c + 1, c)


def prepare(case, seed):
    hq, hkv, hd, _ = SHAPES[case["shape"]]
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 2 + 1)
    r = np.random.default_rng([int(seed) & 0x7FFFFFFF, 78])
    dt, kind = _dtype(case), case["kind"]
    x = {"case": case}
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    if kind == "prompt":
        lens = _ints(case["lens"])
        n = sum(lens)
        x["q"], x["k"], x["v"] = _normal(g, (n, hq, hd), dt), _normal(g, (n, hkv, hd), dt), _normal(g, (n, hkv, hd), dt)
        x["cu"] = np.cumsum([0] + lens).astype(np.int32)
        x["seq"] = dev(np.repeat(np.arange(len(lens)), lens))
        return x
    if kind == "store":
        toks = _ints(case["tokens"])
        n = sum(_up(t) for t in toks)
        x["kv"] = _normal(g, (len(toks), case["layers"], 2, hkv, max(toks), hd), dt)
        layers = case["layers"]
        table = np.full((len(toks), max(_up(t) for t in toks)), -1, np.int32)
        order = r.permutation(n)
        at = 0
        for s, t in enumerate(toks):
            table[s, :_up(t)] = order[at:at + _up(t)]
            at += _up(t)
        length, ref = np.array(toks, np.int32), np.ones(n, np.int32)
        x["table"], x["length"], x["ref"] = dev(table), dev(length), dev(ref)
        x["codes"] = torch.zeros((n, layers, 2, hkv, PAGE * hd), dtype=torch.uint8, device="cuda")
        x["scales"] = torch.zeros((n, layers, 2, hkv), dtype=torch.float32, device="cuda")
        # (sequence, page of it) of every stored page, and which of the padded token rows exist
        x["page_of"] = dev(np.array([p for s, t in enumerate(toks) for p in table[s, :_up(t)]], np.int64))
        x["at"] = dev(np.array([(s, i) for s, t in enumerate(toks) for i in range(_up(t))], np.int64))
        return x
    if kind == "paged":
        reqs = _requests(case)
        P = max(1, max(_up(p) for _, p, _, _ in reqs))
        n = max(1, sum(_up(p) for _, p, _, _ in reqs))
        order = r.permutation(n)
        table, at = np.full((len(reqs), P), -1, np.int32), 0
        for i, (_, p, _, _) in enumerate(reqs):
            table[i, :_up(p)] = order[at:at + _up(p)]
            at += _up(p)
        # contents: N(0, 1) values quantised the way the store does, 1 layer
        x["codes"] = torch.empty((n, 1, 2, hkv, PAGE * hd), dtype=torch.uint8, device="cuda")
        x["scales"] = torch.empty((n, 1, 2, hkv), dtype=torch.float32, device="cuda")
        for a in range(0, n, 64):
            b = min(n, a + 64)
            c, sc = _quantise(_normal(g, (b - a, 1, 2, hkv, PAGE, hd), torch.float32))
            x["codes"][a:b], x["scales"][a:b] = c, sc
        x["table"] = dev(table)
        x["length"] = dev(np.array([p for _, p, _, _ in reqs], np.int32))
        ref = np.zeros(n, np.int32)
        ref[table[table >= 0]] = 1
        x["ref"] = dev(ref)
        cap = max(l - p + o + m for l, p, o, m in reqs)
        x["tail"] = _normal(g, (len(reqs), 1, 2, hkv, cap, hd), dt)
        rows = sum(m for _, _, _, m in reqs)
        x["q"] = _normal(g, (rows, hq, hd), dt)
        anc = np.zeros((rows, 1024), dtype=bool)
        at = 0
        for l, p, o, m in reqs:
            par, seen = _tree(r, o + m), np.zeros((o + m, o + m), dtype=bool)
            for j in range(o + m):
                if par[j] >= 0:
                    seen[j] = seen[par[j]]
                seen[j, j] = True
            anc[at:at + m, :o + m] = seen[o:]
            at += m
        x["anc"] = dev(np.packbits(anc, axis=1, bitorder="little").view(np.int64))
        x["reqs"] = reqs
        # for the padded form: request and row in it of every stacked row; lengths
        M = max(m for _, _, _, m in reqs)
        first = np.cumsum([0] + [m for _, _, _, m in reqs])
        x["row"] = dev(np.array([[first[i] + min(j, m - 1) for j in range(M)] for i, (_, _, _, m) in enumerate(reqs)], np.int64))
        x["back"] = dev(np.array([i * M + j for i, (_, _, _, m) in enumerate(reqs) for j in range(m)], np.int64))
        x["lens"] = dev(np.array(reqs, np.int64))
        return x
    table, length, ref, src, dst = _pool_plan(case)
    x["table"], x["length"], x["ref"] = dev(table), dev(length), dev(ref)
    x["codes"] = _codes(g, (case["pages"], case["layers"], 2, hkv, PAGE * hd))
    x["scales"] = torch.exp2(torch.randint(-9, -4, (case["pages"], case["layers"], 2, hkv), device="cuda", generator=g).float())
    x["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    if kind == "fork":
        x["src"], x["dst"] = src, dst
        x["src_at"], x["dst_at"] = dev(src.astype(np.int64)), dev(dst.astype(np.int64))
    else:
        x["was"] = (x["table"].clone(), x["length"].clone(), x["ref"].clone())
    return x


# ---- one pass ------------------------------------------------------------------------------------------------------------------

def run(state):
    if own:
        return _run_own(state)
    return {"prompt": _plain_prompt, "store": _plain_store, "paged": _plain_paged, "fork": _plain_fork, "compact": _plain_compact}[
        state["case"]["kind"]](state)


def _run_own(x):
    from paper_2507_02620_amd import flowspec as fs
    kind = x["case"]["kind"]
    if kind == "prompt":
        return fs.prompt_attention(x["q"], x["k"], x["v"], x["cu"])
    if "pool" not in x:  # the handle over the pool's tensors, which a program keeps
        x["pool"] = fs.PagePool.of(x["codes"], x["scales"], x["ref"], x["table"], x["length"])
    pool = x["pool"]
    if kind == "store":
        if "items" not in x:
            x["items"] = fs.store_items([(s, 0, x["kv"][s], 0, t) for s, t in enumerate(_ints(x["case"]["tokens"]))])
        fs.paged_store(pool, x["items"])
        return {"codes": x["codes"].view(E4M3), "scales": x["scales"]}
    if kind == "paged":
        if "items" not in x:  # built once per step and used by every layer; so is the scratch
            x["items"] = fs.paged_items([(i, p, x["tail"][i], l, o, m) for i, (l, p, o, m) in enumerate(x["reqs"])])
            x["work"] = fs.paged_attention_workspace(pool, x["q"].shape[1], x["q"].shape[0])
        return fs.paged_attention(pool, 0, x["q"], x["items"], anc=x["anc"], workspace=x["work"])
    if kind == "fork":
        fs.page_free(pool, x["dst"])
        fs.page_fork(pool, x["src"], x["dst"], x["status"])
    else:
        x["table"].copy_(x["was"][0])
        x["length"].copy_(x["was"][1])
        x["ref"].copy_(x["was"][2])
        fs.page_compact(pool, x["status"])
    return _pool_out(x)


def _pool_out(x):
    return {"codes": x["codes"].view(E4M3), "scales": x["scales"], "ref": x["ref"], "table": x["table"], "length": x["length"],
            "status": x["status"]}


# ---- the plain forms -------------------------------------------------------------------------------------------------------

def _attend(q, k, v, seen):
    """q [..., R, hd], k / v [..., S, hd], seen [..., R, S]: rows' sums in 32 bits; a row that sees nothing is zero."""
    s = torch.matmul(q, k.transpose(-1, -2)) / math.sqrt(q.shape[-1])
    s = torch.where(seen, s, float("-inf"))
    top = s.amax(dim=-1, keepdim=True)
    p = torch.exp(s - torch.where(torch.isinf(top), 0.0, top))
    p = p / p.sum(dim=-1, keepdim=True)
    return torch.where(seen.any(dim=-1, keepdim=True), torch.matmul(p, v), 0.0)


def _plain_prompt(x):
    q, k, v, seq = x["q"], x["k"], x["v"], x["seq"]
    n, hq, hd = q.shape
    hkv = k.shape[1]
    at = torch.arange(n, device=q.device)
    seen = (seq[:, None] == seq[None, :]) & (at[:, None] >= at[None, :])
    qs = q.float().view(n, hkv, hq // hkv, hd).permute(1, 2, 0, 3).contiguous()
    o = _attend(qs, k.float().transpose(0, 1).contiguous()[:, None], v.float().transpose(0, 1).contiguous()[:, None], seen)
    return o.permute(2, 0, 1, 3).reshape(n, hq, hd).to(q.dtype)


def _exponent(top):
    """The smallest e with top <= 448 * 2^e, at least -117."""
    m, e = torch.frexp(top)  # top = m * 2^e, m in [1/2, 1)
    return torch.where(top > 0, e - 9 + (m > 0.875).int(), -117).clamp_min(-117)


def _quantise(rows):
    """[..., 2, heads, 64 tokens, hd] in 32 bits -> (codes [..., 2, heads, 64 * hd] as a page holds them, scales [..., 2, heads])."""
    hd = rows.shape[-1]
    fine = torch.isfinite(rows)
    e = _exponent(torch.where(fine, rows, 0.0).abs().amax(dim=(-1, -2)))
    c = torch.ldexp(torch.where(fine, rows, float("nan")), -e[..., None, None]).to(E4M3).view(torch.uint8)
    lead = rows.shape[:-4]
    k, v = c.unbind(dim=len(lead))
    k = k.unflatten(-1, (hd // 64, 64)).transpose(-2, -3)  # [hd / 64][token][64]
    v = v.unflatten(-2, (4, 4, 4)).transpose(-3, -4).flatten(-4, -2).transpose(-1, -2)  # [hd][token's place]
    return torch.stack([k.flatten(-3), v.flatten(-2)], dim=len(lead)), torch.ldexp(torch.ones_like(e, dtype=torch.float32), e)


def _values(codes, scales, hd):
    """Pages [..., 2, heads, 64 * hd] -> (K, V) [..., heads, 64 tokens, hd] in 32 bits."""
    w = codes.view(E4M3).float() * scales[..., None]
    k, v = w.unbind(dim=-3)
    k = k.unflatten(-1, (hd // 64, PAGE, 64)).transpose(-2, -3).flatten(-2)
    v = v.unflatten(-1, (hd, 4, 4, 4)).transpose(-2, -3).flatten(-3).transpose(-1, -2)
    return k, v


def _plain_store(x):
    kv = x["kv"]
    n, layers, _, hkv, cap, hd = kv.shape
    pages = _up(cap)
    rows = torch.zeros((n, layers, 2, hkv, pages * PAGE, hd), dtype=torch.float32, device=kv.device)
    rows[..., :cap, :] = kv
    there = torch.arange(pages * PAGE, device=kv.device)[None, :] < x["length"][:, None]
    rows = torch.where(there[:, None, None, None, :, None], rows, 0.0)
    rows = rows.unflatten(4, (pages, PAGE)).permute(0, 4, 1, 2, 3, 5, 6)[x["at"][:, 0], x["at"][:, 1]]
    c, s = _quantise(rows)
    x["codes"][x["page_of"]] = c
    x["scales"][x["page_of"]] = s
    return {"codes": x["codes"].view(E4M3), "scales": x["scales"]}


def _plain_paged(x):
    q, tail, lens = x["q"], x["tail"], x["lens"]
    n, _, _, hkv, cap, hd = tail.shape
    rows, hq, _ = q.shape
    l, paged, off, m = (lens[:, i] for i in range(4))
    pages = x["table"].long().clamp_min(0)
    k, v = _values(x["codes"][pages, 0], x["scales"][pages, 0], hd)  # [n, P, hkv, 64, hd]
    k, v = (torch.cat([w.transpose(1, 2).flatten(2, 3), t.float()], dim=2) for w, t in ((k, tail[:, 0, 0]), (v, tail[:, 0, 1])))
    settled = torch.arange(pages.shape[1] * PAGE, device=q.device)[None, :] < paged[:, None]
    slot = torch.arange(cap, device=q.device)[None, :] + paged[:, None]
    bits = ((x["anc"][:, :, None] >> torch.arange(64, device=q.device)) & 1).flatten(1).bool()  # [rows, 1024]
    bits = bits[x["row"]]  # [n, M, 1024]
    M = bits.shape[1]
    draft = (slot - l[:, None]).clamp(0, 1023)[:, None, :].expand(n, M, cap)
    newest = (slot < (l + off + m)[:, None])[:, None, :]
    seen = newest & ((slot < l[:, None])[:, None, :] | bits.gather(2, draft))
    seen = torch.cat([settled[:, None, :].expand(n, M, settled.shape[1]), seen], dim=2)
    # masked slots count for nothing whatever they hold
    gone = ~seen.any(dim=1)[:, None, :, None]
    k, v = torch.where(gone, 0.0, k), torch.where(gone, 0.0, v)
    G = hq // hkv
    qs = q.float()[x["row"]].view(n, M, hkv, G, hd).permute(0, 2, 3, 1, 4).reshape(n, hkv, G * M, hd)
    o = _attend(qs, k, v, seen[:, None, None].expand(n, hkv, G, M, seen.shape[2]).reshape(n, hkv, G * M, -1))
    o = o.view(n, hkv, G, M, hd).permute(0, 3, 1, 2, 4).reshape(n * M, hq, hd)
    return o[x["back"]].to(q.dtype)


def _drop(x, seqs):
    """Frees sequences: their pages lose a reference, their table rows empty."""
    rows = x["table"][seqs]
    x["ref"].index_add_(0, rows.clamp_min(0).flatten().long(), -(rows >= 0).int().flatten())
    x["table"][seqs] = -1
    x["length"][seqs] = 0


def _plain_fork(x):
    src, dst, table, length, ref = x["src_at"], x["dst_at"], x["table"], x["length"], x["ref"]
    _drop(x, dst)
    ln = length[src]
    full, part = ln // PAGE, ln % PAGE > 0
    rows, cols = table[src], torch.arange(table.shape[1], device=table.device)[None, :]
    free = torch.argsort((ref > 0).int(), stable=True)  # free pages first, the lowest first
    new = free[(torch.cumsum(part, 0) - 1).clamp_min(0)]
    old = rows.gather(1, torch.where(part, full, 0).long()[:, None])[:, 0].long()
    shared = cols < full[:, None]
    ref.index_add_(0, rows.clamp_min(0).flatten().long(), shared.int().flatten())
    ref.index_add_(0, new, part.int())
    rows = torch.where(shared, rows, torch.where((cols == full[:, None]) & part[:, None], new[:, None].int(), -1))
    table[dst], length[dst] = rows, ln
    to = torch.where(part, new, old)  # (a child without a partial page writes its parent's first one back onto itself)
    x["codes"][to], x["scales"][to] = x["codes"][old], x["scales"][old]
    x["status"].copy_(part.sum()[None])
    return _pool_out(x)


def _plain_compact(x):
    x["table"].copy_(x["was"][0])
    x["length"].copy_(x["was"][1])
    x["ref"].copy_(x["was"][2])
    table, ref = x["table"], x["ref"]
    live = ref > 0
    count = live.sum()
    at = torch.arange(ref.shape[0], device=ref.device)
    src, dst = torch.nonzero(live & (at >= count))[:, 0], torch.nonzero(~live & (at < count))[:, 0]
    to = at.clone()
    to[src] = dst
    x["codes"][dst], x["scales"][dst] = x["codes"][src], x["scales"][src]
    ref[dst] = ref[src]
    ref[src] = 0
    table.copy_(torch.where(table >= 0, to[table.clamp_min(0).long()].int(), -1))
    x["status"].fill_(src.shape[0])
    return _pool_out(x)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------------------

def work(case):
    hq, hkv, hd, _ = SHAPES[case["shape"]]
    e = 4 if _dtype(case) == torch.float32 else 2
    kind = case["kind"]
    if kind == "prompt":
        lens = _ints(case["lens"])
        return {"bytes": (2 * hq + 2 * hkv) * hd * e * sum(lens), "flops": 4 * hd * hq * sum(n * (n + 1) // 2 for n in lens)}
    if kind == "store":
        toks = _ints(case["tokens"])
        per = case["layers"] * 2 * hkv
        return {"bytes": per * (hd * e * sum(toks) + (PAGE * hd + 4) * sum(_up(t) for t in toks)), "flops": 2 * per * hd * sum(toks)}
    if kind == "paged":
        reqs = _requests(case)
        rows = sum(m for _, _, _, m in reqs)
        byt = 2 * rows * hq * hd * e
        flops = 0
        for l, p, o, m in reqs:
            byt += 2 * hkv * (_up(p) * (PAGE * hd + 4) + (l - p + o + m) * hd * e)
            flops += 4 * hd * hq * m * (l + (o + m) // 2)
        return {"bytes": byt, "flops": flops}
    table, length, ref, src, dst = _pool_plan(case)
    page = case["layers"] * 2 * hkv * (PAGE * hd + 4)
    if kind == "fork":
        moved = int(sum(1 for s in src if length[s] % PAGE))
        ints = 4 * 2 * (len(dst) * table.shape[1] + ref.size)
    else:
        live = int((ref > 0).sum())
        moved = int((ref[live:] > 0).sum())
        ints = 4 * 2 * 2 * (table.size + ref.size + length.size)
    return {"bytes": 2 * page * moved + ints, "flops": moved + 1}


# ---- the same from the definitions, in 64 bits -----------------------------------------------------------------------------------

def _nearest_e4m3(y):
    """y in 64 bits to the nearest of 0, +-2^-9 * {1 .. 7}, +-2^k * {8 .. 15} / 8 for k = -6 .. 8 (up to 448), ties to the even one."""
    a = y.abs().clamp_max(448.0)
    step = torch.exp2(torch.floor(torch.log2(a.clamp_min(2.0 ** -6))) - 3)
    # (log2 of a number right below a power of two may round up to it; the step is then too large by one)
    step = torch.where(a < step * 8, step / 2, step).clamp_min(2.0 ** -9)
    return torch.sign(y) * torch.round(a / step) * step


def exact(case, seed):
    x = prepare(case, seed)
    kind = case["kind"]
    if kind == "prompt":
        cu, out = x["cu"], torch.empty(x["q"].shape, dtype=torch.float64, device="cuda")
        group = x["q"].shape[1] // x["k"].shape[1]
        for a, b in zip(cu[:-1], cu[1:]):
            for h in range(x["q"].shape[1]):
                q, k, v = x["q"][a:b, h].double(), x["k"][a:b, h // group].double(), x["v"][a:b, h // group].double()
                w = torch.tril(torch.exp(q @ k.T.contiguous() / math.sqrt(q.shape[1])))  # (scores are moderate: no maximum needed in 64 bits)
                out[a:b, h] = (w @ v) / w.sum(dim=1, keepdim=True)
        return out
    if kind == "store":
        kv, table = x["kv"].double(), x["table"].cpu().numpy()
        n, layers, _, hkv, _, hd = kv.shape
        codes = torch.zeros((x["codes"].shape[0], layers, 2, hkv, PAGE * hd), dtype=torch.float64, device="cuda")
        scales = torch.zeros(x["scales"].shape, dtype=torch.float64, device="cuda")
        place = torch.tensor([16 * ((t >> 2) & 3) + 4 * (t >> 4) + (t & 3) for t in range(PAGE)], device="cuda")
        for s, t in enumerate(_ints(case["tokens"])):
            for i in range(_up(t)):
                rows = torch.zeros((layers, 2, hkv, PAGE, hd), dtype=torch.float64, device="cuda")
                m = min(PAGE, t - i * PAGE)
                rows[:, :, :, :m] = kv[s, :, :, :, i * PAGE:i * PAGE + m]
                top = rows.abs().amax(dim=(3, 4))
                e = torch.ceil(torch.log2(top / 448.0)).clamp_min(-117.0)
                e = torch.where(top > 448.0 * torch.exp2(e), e + 1, torch.where((top <= 224.0 * torch.exp2(e)) & (e > -117), e - 1, e))
                c = _nearest_e4m3(rows / torch.exp2(e)[..., None, None])
                kk = torch.empty((layers, hkv, hd // 64, PAGE, 64), dtype=torch.float64, device="cuda")
                for a in range(hd // 64):
                    kk[:, :, a] = c[:, 0, :, :, 64 * a:64 * a + 64]
                vv = torch.empty((layers, hkv, hd, PAGE), dtype=torch.float64, device="cuda")
                vv[..., place] = c[:, 1].transpose(2, 3)
                p = int(table[s, i])
                codes[p, :, 0], codes[p, :, 1] = kk.flatten(2), vv.flatten(2)
                scales[p] = torch.exp2(e)
        return {"codes": codes, "scales": scales}
    if kind == "paged":
        hd, hkv = x["q"].shape[2], x["tail"].shape[3]
        group = x["q"].shape[1] // hkv
        place = torch.tensor([16 * ((t >> 2) & 3) + 4 * (t >> 4) + (t & 3) for t in range(PAGE)], device="cuda")
        table, out, at = x["table"].cpu().numpy(), [], 0
        bits = np.unpackbits(x["anc"].cpu().numpy().view(np.uint8), axis=1, bitorder="little").astype(bool)
        for i, (l, p, o, m) in enumerate(x["reqs"]):
            L, np_ = l + o + m, _up(p)
            k, v = (torch.empty((hkv, L, hd), dtype=torch.float64, device="cuda") for _ in range(2))
            ids = torch.from_numpy(table[i, :np_].astype(np.int64)).cuda()
            if np_:
                w = x["codes"][ids, 0].view(E4M3).double() * x["scales"][ids, 0].double()[..., None]
                kp = torch.cat([w[:, 0].view(np_, hkv, hd // 64, PAGE, 64)[:, :, a] for a in range(hd // 64)], dim=3)
                vp = w[:, 1].view(np_, hkv, hd, PAGE)[..., place].transpose(2, 3)
                k[:, :p] = kp.transpose(0, 1).reshape(hkv, np_ * PAGE, hd)[:, :p]
                v[:, :p] = vp.transpose(0, 1).reshape(hkv, np_ * PAGE, hd)[:, :p]
            k[:, p:], v[:, p:] = x["tail"][i, 0, 0, :, :L - p].double(), x["tail"][i, 0, 1, :, :L - p].double()
            seen = np.ones((m, L), dtype=bool)
            seen[:, l:] = bits[at:at + m, :o + m]
            seen = torch.from_numpy(seen).cuda()
            got = torch.empty((m, hkv * group, hd), dtype=torch.float64, device="cuda")
            for h in range(hkv * group):
                w = torch.exp(x["q"][at:at + m, h].double() @ k[h // group].T.contiguous() / math.sqrt(hd)) * seen
                got[:, h] = (w @ v[h // group]) / w.sum(dim=1, keepdim=True)
            out.append(got)
            at += m
        return torch.cat(out)
    # pages: bookkeeping step by step on the host, contents moved page by page
    table, length, ref = (x[k].cpu().numpy().copy() for k in ("table", "length", "ref"))
    moves = []
    if kind == "fork":
        for s in x["dst"]:
            for p in table[s][table[s] >= 0]:
                ref[p] -= 1
            table[s], length[s] = -1, 0
        for s, d in zip(x["src"], x["dst"]):
            n = int(length[s])
            for i in range(_up(n)):
                p = int(table[s, i])
                if (i + 1) * PAGE > n:
                    new = int(np.nonzero(ref == 0)[0][0])
                    moves.append((p, new))
                    p = new
                ref[p] += 1
                table[d, i] = p
            length[d] = n
    else:
        count = int((ref > 0).sum())
        for p in range(count, len(ref)):
            if ref[p] > 0:
                new = int(np.nonzero(ref == 0)[0][0])
                ref[new], ref[p] = ref[p], 0
                table[table == p] = new
                moves.append((p, new))
    for a, b in moves:
        x["codes"][b] = x["codes"][a]
        x["scales"][b] = x["scales"][a]
    return {"codes": x["codes"].view(E4M3), "scales": x["scales"].double(), "ref": torch.from_numpy(ref), "table": torch.from_numpy(table),
            "length": torch.from_numpy(length), "status": torch.tensor([len(moves)])}
