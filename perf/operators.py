"""The steps with which a student's rollouts are generated, as cases that a timing program can prepare,
run and check: a token's keys and values go into the paged cache, its queries attend to the cache, and
its logits give the next token.

A case is a dict of plain values.  Its ``op`` says which operator a pass calls:

  append  ``stride_kv_append``: keys (and queries) of new tokens are normalised per head and rotated to
          their positions, keys and values go to the cache's pages;
  attend  ``stride_tree_attention``: the queries of each sequence's newest tokens, one token, a chain
          or a tree of drafted ones, against its pages;
  sample  ``stride_sample``: temperature, top-k, top-p and min-p per row, the token drawn with given
          exponential random numbers.

Where ``own`` is false a pass computes the operator in elementary torch operations in 32 bits; where it
is true it makes the calls that a program makes of this package.
"""
import math
import random

import numpy as np
import torch

own = False

V_FULL = 151936
HEADS = dict(hq=16, hkv=8, d=128)  # the heads of a hidden size of 2,048
APPEND = dict(op="append", dtype="bf16", **HEADS, page=64, layout="token", seqs=8, n_lo=1, n_hi=1,
              ctx_lo=100, ctx_hi=2000, q=True, norm=True, rot=128, style="half", commit=0)
ATTEND = dict(op="attend", dtype="bf16", **HEADS, page=64, layout="token", seqs=8, n_lo=1, n_hi=1,
              ctx_lo=100, ctx_hi=2000, tree=False, share=1)
SAMPLE = dict(op="sample", dtype="bf16", rows=1, vocab=V_FULL, pad=0, mode="nucleus")


def listed():
    return [
        # Eight active rollouts each generate one token: the smallest append, where latency counts.
        dict(APPEND, name="append_step_8"),
        # After a check of 64 drafted trees of 16 tokens the accepted ones (three of sixteen here) go to
        # their final places; the others have no slot.  Pages hold one head's tokens in a row.
        dict(APPEND, name="append_commit_64x16", layout="head", seqs=64, n_lo=16, n_hi=16, ctx_hi=6000,
             q=False, commit=3),
        # The environment's answers, 16 rollouts of 384 to 1,536 tokens, enter the cache at once.
        dict(APPEND, name="append_turn_15k", seqs=16, n_lo=384, n_hi=1536, ctx_hi=4000),
        # One token for each of eight short rollouts: the smallest attention call.
        dict(ATTEND, name="attend_step_8"),
        # One token for each of 64 rollouts, the longest of 16,384 tokens: the memory's speed bounds it.
        dict(ATTEND, name="attend_step_64_long", seqs=64, ctx_lo=1000, ctx_hi=16384),
        # Trees of 9 to 24 drafted tokens over rollouts that share a task's prefix in fours.
        dict(ATTEND, name="attend_tree_32", seqs=32, n_lo=9, n_hi=24, ctx_lo=500, ctx_hi=8192, hq=32,
             tree=True, share=4),
        # The environment's answers of 129 to 1,024 tokens over what the rollouts hold already: a chain.
        dict(ATTEND, name="attend_turn_6", seqs=6, n_lo=129, n_hi=1024, ctx_lo=0, ctx_hi=6000),
        # float32, short pages, three queries to a key head, lengths from one token on.
        dict(ATTEND, name="attend_f32_odd", dtype="f32", hq=12, hkv=4, d=64, page=16, seqs=5, n_lo=1,
             n_hi=7, ctx_lo=1, ctx_hi=1500),
        # One rollout's next token with temperature 0.6, top-k 20 and top-p 0.95.
        dict(SAMPLE, name="sample_1"),
        # The full distribution, as on-policy distillation asks for: no filter, 256 rows.
        dict(SAMPLE, name="sample_plain_256", rows=256, mode="plain"),
        # 64 rows whose requests ask for different things, greedy, filtered and not.
        dict(SAMPLE, name="sample_mixed_64", rows=64, mode="mixed"),
        # float32 rows over a smaller, odd vocabulary in padded rows, top-p alone.
        dict(SAMPLE, name="sample_f32_top_p", dtype="f32", rows=24, vocab=32003, pad=13, mode="top_p"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges; none costs more than the largest listed one of its kind."""
    op = rng.choice(("append", "attend", "attend", "sample"))
    if op == "sample":
        f32 = rng.random() < 0.3
        c = dict(SAMPLE, dtype="f32" if f32 else "bf16", vocab=rng.choice((V_FULL, _log(rng, 1000, V_FULL))),
                 mode=rng.choice(("nucleus", "plain", "mixed", "top_p", "min_p", "top_k")))
        c.update(rows=_log(rng, 1, 96 if f32 else 192), pad=rng.choice((0, 0, 5, 24)))
        return c
    hkv = rng.choice((1, 2, 4, 8, 8))
    heads = dict(hkv=hkv, hq=hkv * rng.choice((1, 2, 2, 3, 4, 5, 8)), d=rng.choice((64, 96, 128, 128, 256)),
                 page=rng.choice((16, 32, 64, 64, 128)), layout=rng.choice(("token", "token", "head")),
                 dtype="f32" if rng.random() < 0.2 else "bf16")
    wide = heads["hq"] * heads["d"] * (4 if heads["dtype"] == "f32" else 2) / 4096.0
    if op == "append":
        c = dict(APPEND, **heads)
        tokens = _log(rng, 1, max(2.0, 12000 / wide))
        seqs = _log(rng, 1, max(1, min(tokens, 128)))
        per = max(1, tokens // seqs)
        rot = c["d"] if rng.random() < 0.7 else c["d"] // 2
        c.update(seqs=seqs, n_lo=max(1, per // 2), n_hi=per + per // 2, ctx_lo=0, ctx_hi=_log(rng, 10, 3000),
                 norm=rng.random() < 0.6, rot=rot, style=rng.choice(("half", "half", "pairs")),
                 q=rng.random() < 0.7)
        if 4 <= c["n_lo"] and c["n_hi"] <= 64 and rng.random() < 0.5:
            c.update(commit=rng.randint(1, 4))
        return c
    c = dict(ATTEND, **heads)
    kind = rng.choice(("step", "step", "tree", "turn"))
    narrow = 1.0 if heads["dtype"] == "bf16" else 4.0
    if kind == "turn":
        seqs = _log(rng, 1, 8)
        top = _log(rng, 40, 1024)
        c.update(seqs=seqs, n_lo=max(1, top // 8), n_hi=top, ctx_lo=0,
                 ctx_hi=_log(rng, 16, 6000 / max(1.0, wide) / narrow))
        return c
    held = hkv * heads["d"] * (2 if heads["dtype"] == "f32" else 1) / 1024.0  # of a cached token, to the listed
    seqs = _log(rng, 1, 64)
    top = _log(rng, 20, max(30.0, min(16384.0, 260000.0 / max(held, wide, 0.25) / seqs / narrow)))
    c.update(seqs=seqs, ctx_lo=rng.choice((0, 1, top // 4, top)), ctx_hi=top, share=rng.choice((1, 1, 4)))
    if kind == "tree":
        n = _log(rng, 2, 70)
        c.update(tree=True, n_lo=max(1, n // 2), n_hi=n, seqs=max(1, seqs // 2))
    return c


# ---- what a user's program has in hand ----

def _lens(case):
    """New tokens and cached tokens of each sequence: spread over the case's ranges, the same for every
    seed so that the work of a pass is the case's own."""
    g = random.Random(case["seqs"] * 7919 + case["n_hi"] * 31 + case["ctx_hi"])
    n = [g.randint(case["n_lo"], case["n_hi"]) for _ in range(case["seqs"])]
    ctx = [g.randint(case["ctx_lo"], case["ctx_hi"]) for _ in range(case["seqs"])]
    if case["seqs"] > 1:  # the longest and the shortest are always there
        ctx[0], ctx[-1] = case["ctx_hi"], case["ctx_lo"]
    return n, ctx


def _parents(case, n):
    """A drafted tree for each sequence: the parent of each of its tokens, -1 for those that follow the
    cached ones.  A tree of `commit` accepted tokens starts with that chain."""
    g = random.Random(case["seqs"] * 104729 + case["n_hi"])
    out = []
    for m in n:
        out.append([-1 if i == 0 else i - 1 if i < case.get("commit", 0) or g.random() < 0.5
                    else g.randint(-1, i - 1) for i in range(m)])
    return out


def _table(case, n, ctx, g):
    """Pages of every sequence, scattered over the cache; groups of `share` sequences have the first
    half of the shortest one's whole pages in common."""
    page, share = case["page"], case.get("share", 1)
    need = [-(-(a + b) // page) for a, b in zip(n, ctx)]
    common = [0] * len(n)
    for s in range(len(n)):
        lead = s - s % share
        if s != lead:
            common[s] = min(ctx[lead:lead + share]) // page // 2
    total = sum(a - b for a, b in zip(need, common)) + 3
    ids = torch.randperm(total, generator=g, device="cuda").to(torch.int32).cpu().numpy()
    table = np.zeros((len(n), max(need) + 1), np.int32)
    at = 0
    for s in range(len(n)):
        c = common[s]
        table[s, :c] = table[s - s % share, :c]
        table[s, c:need[s]] = ids[at:at + need[s] - c]
        at += need[s] - c
    return table, total, sum(common) * page


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _cache(case, pages, g):
    """K and V pages seen as [page, slot, head, element], whichever way they lie in memory."""
    shape = (pages, case["page"], case["hkv"], case["d"])
    if case["layout"] == "head":
        shape = (pages, case["hkv"], case["page"], case["d"])
    kv = [torch.empty(shape, device="cuda", dtype=_dtype(case)).normal_(generator=g) for _ in range(2)]
    return [x.permute(0, 2, 1, 3) for x in kv] if case["layout"] == "head" else kv


def _prepare_append(case, g):
    n, ctx = _lens(case)
    table, pages, _ = _table(case, n, ctx, g)
    seq, slot, pos = [], [], []
    for s, m in enumerate(n):
        depth = list(range(m))
        if case["commit"]:
            depth = [0] * m
            for i, p in enumerate(_parents(case, [m])[0]):
                depth[i] = 0 if p < 0 else depth[p] + 1
        seq += [s] * m
        pos += [ctx[s] + i for i in depth]
        slot += [ctx[s] + i if not case["commit"] or i < case["commit"] else -1 for i in range(m)]
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    k, v = _cache(case, pages, g)
    dt, total = _dtype(case), len(seq)
    new = lambda h: torch.empty((total, h, case["d"]), device="cuda", dtype=dt).normal_(generator=g)  # noqa: E731
    # queries, keys and values of a token side by side, as one projection leaves them
    qkv = new(case["hq"] + 2 * case["hkv"])
    s = dict(case=case, k_cache=k, v_cache=v, table=torch.from_numpy(table).cuda(), seq=dev(seq),
             slot=dev(slot), pos=dev(pos), q=qkv[:, :case["hq"]] if case["q"] else None,
             k=qkv[:, case["hq"]:case["hq"] + case["hkv"]], v=qkv[:, case["hq"] + case["hkv"]:])
    weight = lambda: (1.0 + 0.2 * torch.randn(case["d"], device="cuda", generator=g)).to(dt)  # noqa: E731
    s["q_weight"], s["k_weight"] = (weight(), weight()) if case["norm"] else (None, None)
    half = case["rot"] // 2
    inv = 1e6 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
    at = torch.arange(max(pos) + 1, dtype=torch.float64, device="cuda")[:, None] * inv
    s["rope"] = torch.cat([at.cos(), at.sin()], 1).float()
    return s


def _prepare_attend(case, g):
    n, ctx = _lens(case)
    table, pages, _ = _table(case, n, ctx, g)
    k, v = _cache(case, pages, g)
    total = sum(n)
    q = torch.empty((total, case["hq"], case["d"]), device="cuda", dtype=_dtype(case))
    q.normal_(0.0, 1.5, generator=g)
    off = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    s = dict(case=case, k_cache=k, v_cache=v, table=torch.from_numpy(table).cuda(), q=q, total=total,
             n_max=max(n), len_max=max(a + b for a, b in zip(n, ctx)), q_off=torch.from_numpy(off).cuda(),
             ctx=torch.tensor(ctx, dtype=torch.int32, device="cuda"), scale=case["d"] ** -0.5, mask=None)
    if case["tree"]:
        words = -(-max(n) // 64)
        bits = np.zeros((total, words * 64), np.uint8)
        at = 0
        for par in _parents(case, n):
            for i, p in enumerate(par):
                if p >= 0:
                    bits[at + i] = bits[at + p]
                bits[at + i, i] = 1
            at += len(par)
        s["mask"] = torch.from_numpy(np.packbits(bits, axis=1, bitorder="little").view(np.int64)).cuda()
    return s


def _prepare_sample(case, g):
    rows, vocab = case["rows"], case["vocab"]
    per = 4 if case["dtype"] == "f32" else 8
    ld = vocab + case["pad"]
    ld += -ld % per
    # logits as a language model's: a broad body and some hundred entries that stand out, by row
    z = torch.empty((rows, ld), device="cuda").normal_(0.0, 2.0, generator=g)
    at = torch.randint(0, vocab, (rows, 200), device="cuda", generator=g)
    z.scatter_add_(1, at, 3.0 + 4.0 * torch.rand(rows, 200, device="cuda", generator=g))
    best = torch.randint(0, vocab, (rows, 1), device="cuda", generator=g)
    z.scatter_add_(1, best, 9.0 + 3.0 * torch.rand(rows, 1, device="cuda", generator=g))
    s = dict(case=case, logits=z.to(_dtype(case)))
    del z
    s["noise"] = torch.empty((rows, vocab + -vocab % 4), device="cuda").exponential_(generator=g)
    # a request's parameters by its row: temperature, top-k (0: off), top-p (1: off), min-p (0: off)
    kinds = dict(plain=(1.0, 0, 1.0, 0.0), nucleus=(0.6, 20, 0.95, 0.0), top_p=(0.8, 0, 0.9, 0.0),
                 min_p=(1.0, 0, 1.0, 0.05), top_k=(0.7, 50, 1.0, 0.0), greedy=(0.0, 0, 1.0, 0.0),
                 all=(0.9, 100, 0.97, 0.02))
    order = list(kinds) if case["mode"] == "mixed" else [case["mode"]]
    par = [kinds[order[r % len(order)]] for r in range(rows)]
    for i, name in enumerate(("temperature", "top_k", "top_p", "min_p")):
        s[name] = torch.tensor([p[i] for p in par], device="cuda",
                               dtype=torch.int32 if name == "top_k" else torch.float32)
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return dict(append=_prepare_append, attend=_prepare_attend, sample=_prepare_sample)[case["op"]](case, g)


# ---- the operators in elementary operations, in 32 bits ----

def _rotated(x, weight, s):
    """x [token, head, element] normalised per head and rotated to the tokens' positions, in 32 bits."""
    case = s["case"]
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * weight.float()
    rot = case["rot"]
    half = rot // 2
    cs = s["rope"][s["pos"].long()].unsqueeze(1)
    c, sn = cs[..., :half], cs[..., half:]
    if case["style"] == "half":
        a, b = x[..., :half], x[..., half:rot]
        turned = torch.cat([a * c - b * sn, b * c + a * sn], -1)
    else:
        a, b = x[..., :rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * c - b * sn, b * c + a * sn], -1).flatten(-2)
    return torch.cat([turned, x[..., rot:]], -1)


def _plain_append(s):
    dt, page = s["k_cache"].dtype, s["case"]["page"]
    q = None if s["q"] is None else _rotated(s["q"], s["q_weight"], s).to(dt)
    k = _rotated(s["k"], s["k_weight"], s).to(dt)
    v, seq, slot = s["v"], s["seq"].long(), s["slot"].long()
    if s["case"]["commit"]:
        kept = torch.nonzero(slot >= 0).squeeze(1)
        k, v, seq, slot = k[kept], v[kept], seq[kept], slot[kept]
    at = s["table"].long()[seq, slot // page]
    s["k_cache"][at, slot % page] = k
    s["v_cache"][at, slot % page] = v
    return dict(q=q, k_cache=s["k_cache"], v_cache=s["v_cache"])


def _plain_attend(s):
    case = s["case"]
    seqs, hkv, d, page = case["seqs"], case["hkv"], case["d"], case["page"]
    grp, n_max, length = case["hq"] // hkv, s["n_max"], s["len_max"]
    off, ctx = s["q_off"].long(), s["ctx"].long()
    n = off[1:] - off[:-1]
    pages = s["table"][:, :-(-length // page)].long()

    def dense(x):  # [sequence, head, slot, element]
        x = x[pages].reshape(seqs, -1, hkv, d)[:, :length]
        return x.permute(0, 2, 1, 3).float().contiguous()

    i = torch.arange(n_max, device="cuda")
    rows = (off[:-1, None] + i).clamp(max=s["total"] - 1)
    q = s["q"].float()[rows].reshape(seqs, n_max, hkv, grp, d).permute(0, 2, 1, 3, 4)
    q = q.reshape(seqs, hkv, n_max * grp, d)
    x = torch.matmul(q, dense(s["k_cache"]).transpose(2, 3)) * s["scale"]
    new = torch.arange(length, device="cuda") - ctx[:, None]          # [sequence, slot]: which new token
    if s["mask"] is None:
        sees = new[:, None, :] <= i[:, None]
    else:
        at = new.clamp(0, s["mask"].shape[1] * 64 - 1)[:, None, :].expand(-1, n_max, -1)
        word = s["mask"][rows].gather(2, at // 64)
        sees = (new[:, None, :] < 0) | (((word >> (at % 64)) & 1) == 1)
    sees = (sees & (new < n[:, None])[:, None, :])[:, None, :, None, :].expand(-1, 1, -1, grp, -1)
    sees = sees.reshape(seqs, 1, n_max * grp, length)
    x = x.masked_fill(~sees, -math.inf)
    top = x.amax(-1, keepdim=True)
    e = (x - top.clamp(min=-3e38)).exp()
    del x
    total = e.sum(-1, keepdim=True)
    out = torch.matmul(e, dense(s["v_cache"])) / total.clamp(min=1e-38)
    lse = (top + total.log()).squeeze(-1)
    token = torch.arange(s["total"], device="cuda")
    seq = torch.searchsorted(off, token, right=True) - 1
    back = lambda y, *t: y.reshape(seqs, hkv, n_max, grp, *t).transpose(1, 2)[  # noqa: E731
        seq, token - off[seq]].reshape(s["total"], case["hq"], *t)
    return dict(out=back(out, d).to(s["q"].dtype), lse=back(lse))


def _plain_sample(s):
    case = s["case"]
    z = s["logits"][:, :case["vocab"]].float()
    temp, top_k, top_p, min_p = (s[n].unsqueeze(1) for n in ("temperature", "top_k", "top_p", "min_p"))
    top = z.amax(1, keepdim=True)
    col = torch.arange(case["vocab"], device="cuda")
    greedy = torch.where(z == top, col, case["vocab"]).amin(1)
    x, order = ((z - top) / torch.where(temp > 0, temp, 1.0)).sort(dim=1, descending=True, stable=True)
    keep = (top_k <= 0) | (col < top_k)
    w = torch.where(keep, x.exp(), 0.0)
    mass = w.cumsum(1)
    keep = keep & ((top_p >= 1) | (mass - w < top_p * mass[:, -1:])) & (x >= min_p.log())
    keep[:, 0] = True
    key = torch.where(keep, x - s["noise"].gather(1, order).log(), -math.inf)
    drawn = torch.where(key == key.amax(1, keepdim=True), order, case["vocab"]).amin(1)
    return dict(token_ids=torch.where(temp.squeeze(1) > 0, drawn, greedy).to(torch.int32))


# ---- the package's calls ----

def _own(s):
    """The handle, buffers and workspace that a program makes once and keeps."""
    import paper_2609_14636_amd as P
    case = s["case"]
    o = dict(P=P, flags=torch.zeros(1, dtype=torch.int32, device="cuda"))
    if case["op"] == "sample":
        o["ids"] = torch.empty(case["rows"], dtype=torch.int32, device="cuda")
        size = P.stride_sample_workspace_size(case["rows"], case["vocab"])
    else:
        o["cache"] = P.KVCache(s["k_cache"], s["v_cache"], s["table"])
    if case["op"] == "append":
        o["q"] = None if s["q"] is None else torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda")
        o["style"] = P.STRIDE_ROPE_HALF if case["style"] == "half" else P.STRIDE_ROPE_PAIRS
        return o
    if case["op"] == "attend":
        o["out"] = torch.empty_like(s["q"])
        o["lse"] = torch.empty(s["q"].shape[:2], device="cuda")
        size = P.stride_attention_workspace_size(o["cache"], s["total"], case["hq"])
    o["ws"] = torch.empty(max(size, 256), dtype=torch.uint8, device="cuda")
    return o


def _own_run(s):
    if "own" not in s:
        s["own"] = _own(s)
    o, case = s["own"], s["case"]
    P = o["P"]
    if case["op"] == "append":
        P.stride_kv_append(o["cache"], s["k"], s["v"], s["seq"], s["slot"], s["pos"], rope=s["rope"],
                           rope_style=o["style"], k_weight=s["k_weight"], q=s["q"],
                           q_weight=s["q_weight"] if case["q"] else None, q_out=o["q"], eps=1e-6,
                           dev_flags=o["flags"])
        return dict(q=o["q"], k_cache=s["k_cache"], v_cache=s["v_cache"])
    if case["op"] == "attend":
        P.stride_tree_attention(o["cache"], s["q"], s["q_off"], s["ctx"], s["mask"], s["scale"],
                                o["out"], o["lse"], o["flags"], o["ws"])
        return dict(out=o["out"], lse=o["lse"])
    P.stride_sample(case["vocab"], s["logits"], s["noise"], s["temperature"], s["top_k"], s["top_p"],
                    s["min_p"], o["ids"], o["flags"], o["ws"])
    return dict(token_ids=o["ids"])


def run(state):
    if own:
        return _own_run(state)
    plain = dict(append=_plain_append, attend=_plain_attend, sample=_plain_sample)
    return plain[state["case"]["op"]](state)


# ---- what a pass cannot do without ----

def work(case):
    es = 4.0 if case["dtype"] == "f32" else 2.0
    if case["op"] == "sample":
        rows, vocab = case["rows"], case["vocab"]
        total, flops = rows * (vocab * es + 4 + 16), 0.0
        kinds = ("plain", "nucleus", "top_p", "min_p", "top_k", "greedy", "all")
        for r in range(rows):  # an unfiltered row needs all its random numbers, and each entry a logarithm
            if (kinds[r % 7] if case["mode"] == "mixed" else case["mode"]) == "plain":
                total += 4.0 * vocab
                flops += 2.0 * vocab
        return dict(bytes=float(total), flops=flops)
    n, ctx = _lens(case)
    tokens, head = sum(n), case["d"] * es
    if case["op"] == "append":
        kept = case["seqs"] * min(case["commit"], min(n)) if case["commit"] else tokens
        total = 4.0 * kept * case["hkv"] * head + 12.0 * tokens
        if case["q"]:
            total += 2.0 * tokens * case["hq"] * head
        table = len({c + i for m, c in zip(n, ctx) for i in range(m)})
        total += 4.0 * case["rot"] * table
        each = (kept * case["hkv"] + (tokens * case["hq"] if case["q"] else 0)) * case["d"]
        return dict(bytes=total, flops=(3.0 * case["rot"] / case["d"] + (4 if case["norm"] else 0)) * each)
    shared = 0
    page, share = case["page"], case["share"]
    for s in range(len(n)):
        if s % share:
            lead = s - s % share
            shared += min(ctx[lead:lead + share]) // page // 2 * page
    slots = sum(n) + sum(ctx) - shared
    total = 2.0 * slots * case["hkv"] * head + tokens * case["hq"] * (2 * head + 4)
    if case["tree"]:
        pairs = 0
        for par, c in zip(_parents(case, n), ctx):
            depth = []
            for p in par:
                depth.append(1 if p < 0 else depth[p] + 1)
            pairs += c * len(par) + sum(depth)
    else:
        pairs = sum(c * m + m * (m + 1) // 2 for m, c in zip(n, ctx))
    return dict(bytes=total, flops=4.0 * pairs * case["hq"] * case["d"])


# ---- the same results in 64 bits ----

def _exact_append(s):
    case = s["case"]
    d, rot, half = case["d"], case["rot"], case["rot"] // 2
    first = torch.arange(half, device="cuda") * (1 if case["style"] == "half" else 2)
    second = first + (half if case["style"] == "half" else 1)
    pos = s["pos"].long()
    c, sn = (s["rope"][pos][:, None, a:a + half].double() for a in (0, half))

    def turn(x, w):
        x = x.double()
        if w is not None:
            x = w.double() * x / (x.pow(2).sum(-1, keepdim=True) / d + 1e-6).sqrt()
        y = x.clone()
        y[..., first] = c * x[..., first] - sn * x[..., second]
        y[..., second] = sn * x[..., first] + c * x[..., second]
        return y

    out = [s["k_cache"].double(), s["v_cache"].double()]
    new = [turn(s["k"], s["k_weight"]), s["v"].double()]
    table = s["table"].cpu().numpy()
    where = [(t, table[q, x // case["page"]], x % case["page"])
             for t, (q, x) in enumerate(zip(s["seq"].tolist(), s["slot"].tolist())) if x >= 0]
    t, pg, sl = (torch.tensor(y, dtype=torch.long, device="cuda") for y in zip(*where))
    for whole, x in zip(out, new):
        whole[pg, sl] = x[t]
    q = None if s["q"] is None else turn(s["q"], s["q_weight"])
    return dict(q=q, k_cache=out[0], v_cache=out[1])


def _exact_attend(s):
    case = s["case"]
    grp, page = case["hq"] // case["hkv"], case["page"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    off, ctx, table = s["q_off"].tolist(), s["ctx"].tolist(), s["table"].long()
    for q in range(case["seqs"]):
        a, b = off[q], off[q + 1]
        m, length = b - a, ctx[q] + b - a
        slots = torch.arange(length, device="cuda")
        pg, sl = table[q][slots // page], slots % page
        seen = torch.ones(m, length, dtype=torch.bool, device="cuda")
        if s["mask"] is None:
            seen[:, ctx[q]:] = torch.ones(m, m, dtype=torch.bool, device="cuda").tril()
        else:
            words = s["mask"][a:b].cpu().numpy().view(np.uint8)
            bits = np.unpackbits(words, axis=1, bitorder="little")[:, :m]
            seen[:, ctx[q]:] = torch.from_numpy(bits.astype(bool)).cuda()
        for h in range(case["hkv"]):
            k, v = s["k_cache"][pg, sl, h].double(), s["v_cache"][pg, sl, h].double()
            for j in range(h * grp, (h + 1) * grp):
                x = (s["q"][a:b, j].double() @ k.t() * s["scale"]).masked_fill(~seen, -math.inf)
                lse[a:b, j] = torch.logsumexp(x, 1)
                out[a:b, j] = torch.softmax(x, 1) @ v
    return dict(out=out, lse=lse)


def _exact_sample(s):
    case = s["case"]
    ids = []
    for r in range(case["rows"]):
        z = s["logits"][r, :case["vocab"]].double().cpu().numpy()
        e = s["noise"][r, :case["vocab"]].double().cpu().numpy()
        temp, k, p, low = (float(s[n][r]) for n in ("temperature", "top_k", "top_p", "min_p"))
        if temp == 0:
            ids.append(int(np.argmax(z)))
            continue
        w = np.exp((z - z.max()) / temp)
        order = np.argsort(-z, kind="stable")
        order = order[:int(k)] if k > 0 else order
        before = np.concatenate([[0.0], np.cumsum(w[order])])
        if p < 1:
            order = order[before[:-1] < p * before[-1]]
        order = np.concatenate([order[:1], order[1:][w[order[1:]] >= low]])
        with np.errstate(divide="ignore"):
            race = np.log(w[order]) - np.log(e[order])
        ids.append(int(order[np.argmax(race)]))
    return dict(token_ids=torch.tensor(ids, dtype=torch.int32))


def exact(case, seed):
    s = prepare(case, seed)
    return dict(append=_exact_append, attend=_exact_attend, sample=_exact_sample)[case["op"]](s)
