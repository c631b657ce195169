"""What a decoder block does between its linear layers, as cases that can be timed and checked.

Four operators, six kinds of case:
  attn      one new token of every sequence against its keys and values in a paged cache; `weights`: each cached token's attention weight,
            summed over the query heads that share it, comes out too, as a program that will evict by it asks for it
  append    new tokens' queries and keys rotated by their positions, keys and values stored in the cache's pages
  evict     every head of a sequence that has grown over its budget keeps the tokens of most accumulated weight
  norm      residual addition with gate and scale, the norm after a block and the norm before the next one
  norm-bwd  its gradients

A cache is [pages][kv heads][page size][head dim], fp16; token t of sequence b lies in page table[b][t // page size] at t % page size.
Where `own` is false everything is computed by elementary operations in 32 bits.
"""
import math

import torch

own = False

EPS = 1e-5
# query heads, kv heads, hidden size
MODELS = {"7b": (32, 32, 4096), "13b": (40, 40, 5120), "70b": (64, 8, 8192)}


def listed():
    return [
        # the smallest call: one short conversation
        dict(name="attn-one", kind="attn", heads=32, kv=32, d=128, page=16, seqs=1, longest=203, ragged=0.0, weights=False),
        # a batch of conversations of different lengths
        dict(name="attn-7b", kind="attn", heads=32, kv=32, d=128, page=16, seqs=8, longest=3001, ragged=0.7, weights=False),
        # one long document, eight query heads to a kv head: the largest
        dict(name="attn-70b-long", kind="attn", heads=64, kv=8, d=128, page=64, seqs=1, longest=131001, ragged=0.0, weights=False),
        # a batch whose weights are kept for eviction
        dict(name="attn-13b-weights", kind="attn", heads=40, kv=40, d=128, page=32, seqs=4, longest=2049, ragged=0.2, weights=True),
        # the next token of eight sequences
        dict(name="append-7b", kind="append", heads=32, kv=32, d=128, page=16, seqs=8, tokens=8, rot=128),
        # a prompt
        dict(name="append-70b-prompt", kind="append", heads=64, kv=8, d=128, page=64, seqs=1, tokens=4001, rot=128),
        # steady state: one token over the budget
        dict(name="evict-7b-step", kind="evict", kv=32, d=128, page=16, seqs=16, longest=2049, ragged=0.0, budget=2048, first=4, last=256),
        # a long prompt cut down before its answer begins
        dict(name="evict-70b-prompt", kind="evict", kv=8, d=128, page=64, seqs=1, longest=32768, ragged=0.0, budget=4096, first=4, last=1024),
        # between two linear layers while decoding
        dict(name="norm-7b-token", kind="norm", m=1, n=4096, f32=False, post=False, gate="none", scale=1.0),
        # fine-tuning: residual stream in 32 bits
        dict(name="norm-7b", kind="norm", m=4096, n=4096, f32=True, post=False, gate="none", scale=1.0),
        # fine-tuning at an odd length, norms on both sides of a block, a gate for every token
        dict(name="norm-bwd-13b", kind="norm-bwd", m=333, n=5120, f32=False, post=True, gate="token", scale=0.5),
        # fine-tuning, the widest rows, a gate for every channel
        dict(name="norm-bwd-70b", kind="norm-bwd", m=4096, n=8192, f32=True, post=True, gate="channel", scale=0.25),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("attn", "attn", "attn", "append", "evict", "norm", "norm-bwd"))
    if kind.startswith("norm"):
        n = rng.choice((MODELS[rng.choice(("7b", "13b", "70b"))][2], 8 * _log(rng, 8, 2048)))
        m = _log(rng, 1, max(2, min(8192, 32_000_000 // n)))
        return dict(kind=kind, m=m, n=n, f32=rng.random() < 0.5, post=rng.random() < 0.4, gate=rng.choice(("none", "channel", "token")),
                    scale=rng.choice((1.0, 0.5, round(rng.uniform(0.1, 2.0), 3))))
    heads, kv = rng.choice((MODELS["7b"][:2], MODELS["13b"][:2], MODELS["70b"][:2], (8, 8), (16, 4), (12, 2), (32, 1)))
    d = rng.choice((128, 128, 128, 64, 96, 80, 256))
    page = rng.choice((8, 16, 16, 32, 64, 64, 128, 256))
    if kind == "append":
        tokens = _log(rng, 1, max(2, min(8192, (1 << 25) // (heads * d))))
        return dict(kind=kind, heads=heads, kv=kv, d=d, page=page, seqs=rng.randint(1, min(tokens, 32)), tokens=tokens, rot=rng.choice((d, d, d // 2, 0)))
    most = (1 << 27) // (kv * d)          # tokens in the cache: as many bytes as the largest listed case
    ragged = rng.choice((0.0, round(rng.uniform(0.05, 0.95), 2)))
    if kind == "attn":
        longest = _log(rng, 1, min(131072, most))
        return dict(kind=kind, heads=heads, kv=kv, d=d, page=page, seqs=_log(rng, 1, max(1, min(64, most // longest))), longest=longest, ragged=ragged,
                    weights=rng.random() < 0.35)
    longest = _log(rng, 64, min(65536, most // 2))
    budget = rng.choice((longest - 1, max(8, int(longest * rng.uniform(0.1, 0.95)))))
    return dict(kind=kind, kv=kv, d=d, page=page, seqs=_log(rng, 1, max(1, min(32, most // 2 // longest))), longest=longest, ragged=ragged, budget=budget,
                first=rng.choice((0, min(4, budget // 4))), last=rng.choice((0, budget // 8, budget // 2)))


# ---- inputs --------------------------------------------------------------------------------------------------------


def _gen(seed, what):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 1013 + what)


def _normal(gen, *shape, std=1.0, dtype=torch.float16):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).mul_(std).to(dtype)


def _lengths(case, seed):
    """Host list: the longest, and others between (1 - ragged) of it and it."""
    g = torch.Generator().manual_seed(int(seed) * 1013 + 7)
    u = torch.rand(case["seqs"], generator=g, dtype=torch.float64)
    u[0] = 0.0
    return [max(1, int(case["longest"] * (1.0 - case["ragged"] * float(v)))) for v in u]


def _table(seed, seqs, pages):
    """Every sequence's pages, scattered over the pool."""
    return torch.randperm(seqs * pages, generator=_gen(seed, 11), device="cuda").int().view(seqs, pages)


def _pool(gen, pages, kv, page, d):
    x = torch.empty((pages, kv, page, d), dtype=torch.float16, device="cuda")
    return x.normal_(generator=gen)


def _rotation(rot, positions):
    """[position][cos of rot / 2 frequencies, sin of them], angles in 64 bits."""
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    a = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float()


def _norm_inputs(case, seed):
    m, n = case["m"], case["n"]
    t = torch.float32 if case["f32"] else torch.float16
    st = dict(y=_normal(_gen(seed, 1), m, n, std=0.5), r=_normal(_gen(seed, 2), m, n, std=2.0, dtype=t), w_pre=1 + _normal(_gen(seed, 3), n, std=0.2),
              w_post=1 + _normal(_gen(seed, 4), n, std=0.2) if case["post"] else None, gate=None)
    st["r"][:, :: max(1, n // 7)] *= 8               # a residual stream has a few large channels
    if case["gate"] != "none":
        st["gate"] = torch.sigmoid(_normal(_gen(seed, 5), *((m, n) if case["gate"] == "token" else (n,)), dtype=torch.float32)).half()
    if case["kind"] == "norm-bwd":
        st["h"] = st.pop("r")
        st["dx"], st["dh"] = _normal(_gen(seed, 6), m, n, std=0.01), _normal(_gen(seed, 8), m, n, std=0.02, dtype=t)
    return st


def prepare(case, seed):
    st = dict(case=case)
    if case["kind"].startswith("norm"):
        st.update(_norm_inputs(case, seed))
        return st
    kv, d, page, seqs = case["kv"], case["d"], case["page"], case["seqs"]
    if case["kind"] == "append":
        tokens = case["tokens"]
        each = -(-tokens // seqs)
        # tokens of all sequences in one batch: sequence b has its share, after 100 + 17 b tokens that are there already
        seq = torch.arange(tokens, device="cuda") // each
        index = torch.arange(tokens, device="cuda") % each + 100 + 17 * seq
        pages = -(-(each + 100 + 17 * seqs) // page)
        st.update(seq=seq.int(), index=index.int(), pos=index.int(), table=_table(seed, seqs, pages), rot=_rotation(case["rot"], each + 100 + 17 * seqs) if case["rot"] else None,
                  q=_normal(_gen(seed, 1), tokens, case["heads"] * d), k=_normal(_gen(seed, 2), tokens, kv * d), v=_normal(_gen(seed, 3), tokens, kv * d),
                  K=_pool(_gen(seed, 4), seqs * pages, kv, page, d), V=_pool(_gen(seed, 5), seqs * pages, kv, page, d))
        return st
    lens = _lengths(case, seed)
    pages = -(-max(lens) // page)
    st.update(lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), longest=max(lens), table=_table(seed, seqs, pages),
              K=_pool(_gen(seed, 4), seqs * pages, kv, page, d), V=_pool(_gen(seed, 5), seqs * pages, kv, page, d))
    if case["kind"] == "attn":
        st["K"][..., :: max(1, d // 4)] *= 3                    # a few channels of the keys are large
        st["q"] = _normal(_gen(seed, 1), seqs, case["heads"] * d, std=1.5)
        # what lies in a page behind a sequence's end was never written
        t = torch.arange(pages * page, device="cuda").view(pages, page)
        for b in range(seqs):
            if lens[b] < pages * page:
                last = lens[b] // page
                unused = (t[last:] >= lens[b])[:, None, :, None]
                for pool in (st["K"], st["V"]):
                    rows = st["table"][b, last:].long()
                    pool[rows] = pool[rows].masked_fill(unused, float("nan"))
        return st
    # accumulated weights: a few tokens hold most of it, and many have the same little
    at = (seqs, kv, pages * page)
    score = torch.rand(at, generator=_gen(seed, 6), device="cuda").pow_(8).mul_(64).round_().div_(64)
    score[..., ::3] += torch.rand((seqs, kv, -(-at[2] // 3)), generator=_gen(seed, 9), device="cuda")
    # earlier evictions have left every head's tokens in another order
    pos = torch.rand(at, generator=_gen(seed, 10), device="cuda").mul_(0.3).add_(torch.linspace(0, 1, at[2], device="cuda"))
    beyond = torch.arange(at[2], device="cuda") >= st["lens"][:, None, None]
    pos = pos.masked_fill_(beyond, 9.0).argsort(-1).argsort(-1).int()
    st.update(score=score, pos=pos, seen=st["lens"].clone(), score_out=torch.zeros_like(score), pos_out=torch.zeros_like(pos),
              lens_out=torch.zeros_like(st["lens"]))
    return st


# ---- the framework's operators -------------------------------------------------------------------------------------


def _kept(st, name, make):
    """What a program makes once and keeps: descriptions, workspaces, the cache's object."""
    if name not in st:
        st[name] = make()
    return st[name]


def _bytes(n):
    return torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")


def _run_own(st):
    from paper_2410_08661_amd import binding as B
    c = st["case"]
    kind = c["kind"]
    if kind.startswith("norm"):
        code = {"none": B.QEFT_GATE_NONE, "channel": B.QEFT_GATE_CHANNEL, "token": B.QEFT_GATE_TOKEN}[c["gate"]]
        desc = _kept(st, "desc", lambda: B.make_norm_desc(c["n"], torch.float32 if c["f32"] else torch.float16, code, c["scale"], EPS))
        if kind == "norm":
            h, x = _kept(st, "out", lambda: (torch.empty_like(st["r"]), torch.empty_like(st["y"])))
            B.qeft_norm_fwd(desc, st["r"], st["w_pre"], y=st["y"], w_post=st["w_post"], gate=st["gate"], h=h, x=x)
            return {"h": h, "x": x}
        out = _kept(st, "out", lambda: dict(dr=torch.empty_like(st["h"]), dy=torch.empty_like(st["y"]), dw_pre=torch.empty(c["n"], device="cuda"),
                                            dw_post=torch.empty(c["n"], device="cuda") if c["post"] else None,
                                            dgate=None if st["gate"] is None else torch.empty_like(st["gate"], dtype=torch.float32 if c["gate"] == "channel" else torch.float16)))
        ws = _kept(st, "ws", lambda: _bytes(B.qeft_norm_workspace(desc, c["m"])))
        B.qeft_norm_bwd(desc, st["dx"], st["h"], st["w_pre"], dh=st["dh"], y=st["y"], w_post=st["w_post"], gate=st["gate"], ws=ws, **out)
        return out
    cache = _kept(st, "cache", lambda: B.Cache(B.make_cache_desc(st["K"].shape[0], c["page"], c["kv"], c["d"]), k=st["K"], v=st["V"]))
    if kind == "append":
        out = _kept(st, "out", lambda: torch.empty_like(st["q"]))
        B.qeft_cache_append(cache, st["table"], st["k"], st["v"], st["index"], seq=st["seq"], q=st["q"], q_out=out, rot=st["rot"], pos=st["pos"])
        return {"q": out, "k": st["K"], "v": st["V"]}
    if kind == "attn":
        out = _kept(st, "out", lambda: torch.empty_like(st["q"]))
        weights = _kept(st, "weights", lambda: torch.zeros((c["seqs"], c["kv"], st["table"].shape[1] * c["page"]), device="cuda") if c["weights"] else None)
        ws = _kept(st, "ws", lambda: _bytes(B.qeft_attn_workspace(cache.desc, c["seqs"], c["heads"], st["longest"], c["weights"])))
        B.qeft_attn_decode(cache, st["table"], st["lens"], st["longest"], st["q"], out=out, score=weights, ws=ws)
        return {"out": out, "weights": weights}
    ws = _kept(st, "ws", lambda: _bytes(B.qeft_evict_workspace(cache.desc, c["seqs"], st["longest"], c["budget"])))
    B.qeft_cache_evict(cache, st["table"], st["lens"], st["longest"], c["budget"], st["score"], st["pos"], st["seen"], keep_first=c["first"], keep_last=c["last"],
                       score_out=st["score_out"], pos_out=st["pos_out"], lens_out=st["lens_out"], ws=ws)
    return {"k": st["K"], "v": st["V"], "score": st["score_out"], "pos": st["pos_out"], "lens": st["lens_out"]}


# ---- their plain forms ---------------------------------------------------------------------------------------------


def _rows(st, tokens):
    """Page and slot of the first `tokens` tokens of every sequence, [seqs][tokens] each."""
    t = torch.arange(tokens, device="cuda")
    page = st["case"]["page"]
    return st["table"].long()[:, t // page], (t % page).expand(st["table"].shape[0], -1)


def _rotate(x, heads, st):
    """Rows of heads of d, each head's first `rot` values rotated in pairs half of them apart; 32 bits."""
    x = x.float().view(x.shape[0], heads, -1)
    half = st["case"]["rot"] // 2
    if not half:
        return x
    cs = st["rot"][st["pos"].long()][:, None]
    c, s = cs[..., :half], cs[..., half:]
    a, b = x[..., :half], x[..., half: 2 * half]
    return torch.cat([a * c - b * s, b * c + a * s, x[..., 2 * half:]], -1)


def _plain_attn(st):
    c = st["case"]
    heads, kv, d = c["heads"], c["kv"], c["d"]
    g, n, seqs = heads // kv, st["longest"], c["seqs"]
    page, slot = _rows(st, n)
    seen = (torch.arange(n, device="cuda") < st["lens"][:, None])                        # [seqs][n]
    k = st["K"][page, :, slot].float().permute(0, 2, 1, 3).contiguous()                  # [seqs][kv][n][d]
    k = torch.where(seen[:, None, :, None], k, 0.0)
    q = st["q"].float().view(seqs * kv, g, d)
    s = torch.bmm(k.view(seqs * kv, n, d), q.transpose(1, 2).contiguous()).view(seqs, kv, n, g) / math.sqrt(d)
    del k
    s = torch.where(seen[:, None, :, None], s, float("-inf"))
    p = torch.exp(s - s.amax(2, keepdim=True))
    p = p / p.sum(2, keepdim=True)
    v = st["V"][page, :, slot].float().permute(0, 2, 1, 3).contiguous()
    v = torch.where(seen[:, None, :, None], v, 0.0)
    o = torch.bmm(p.permute(0, 1, 3, 2).reshape(seqs * kv, g, n).contiguous(), v.view(seqs * kv, n, d)).view(seqs, heads * d).half()
    weights = None
    if c["weights"]:
        weights = torch.zeros((seqs, kv, st["table"].shape[1] * c["page"]), device="cuda")
        weights[..., :n] = torch.where(seen[:, None], p.sum(3), 0.0)
    return {"out": o, "weights": weights}


def _plain_append(st):
    c = st["case"]
    kv, d = c["kv"], c["d"]
    q, k = _rotate(st["q"], c["heads"], st), _rotate(st["k"], kv, st)
    page = st["table"].long()[st["seq"].long(), st["index"].long() // c["page"]]
    slot = st["index"].long() % c["page"]
    st["K"][page, :, slot] = k.half()
    st["V"][page, :, slot] = st["v"].view(-1, kv, d)
    return {"q": q.half().view(-1, c["heads"] * d), "k": st["K"], "v": st["V"]}


def _plain_evict(st):
    c = st["case"]
    budget, n = c["budget"], st["longest"]
    lens, t = st["lens"].long()[:, None, None], torch.arange(n, device="cuda")
    pos, score = st["pos"][..., :n], st["score"][..., :n]
    sure = (pos < c["first"]) | (pos >= st["seen"][:, None, None] - c["last"])
    rank = torch.where(t < lens, torch.where(sure, float("inf"), score), float("-inf"))
    order = torch.sort(rank, dim=-1, descending=True, stable=True).indices
    keep = torch.zeros_like(rank, dtype=torch.bool).scatter_(-1, order[..., :budget], True)
    keep &= t < lens
    over = lens > budget
    hole, mover = over & ~keep & (t < budget), over & keep & (t >= budget)
    # the i-th mover goes where the i-th hole is; both are listed in order of sequence, head, index
    (b, h, src), dst = mover.nonzero(as_tuple=True), hole.nonzero(as_tuple=True)[2]
    table, page = st["table"].long(), c["page"]
    for_k, for_v = (p[table[b, src // page], h, src % page] for p in (st["K"], st["V"]))
    st["K"][table[b, dst // page], h, dst % page] = for_k
    st["V"][table[b, dst // page], h, dst % page] = for_v
    left = torch.minimum(lens, torch.full_like(lens, budget))
    stay = t < left
    for_score, for_pos = score[b, h, src], pos[b, h, src]
    st["score_out"][..., :n] = torch.where(stay, score, st["score_out"][..., :n])
    st["pos_out"][..., :n] = torch.where(stay, pos, st["pos_out"][..., :n])
    st["score_out"][b, h, dst], st["pos_out"][b, h, dst] = for_score, for_pos
    st["lens_out"].copy_(left.view(-1))
    return {"k": st["K"], "v": st["V"], "score": st["score_out"], "pos": st["pos_out"], "lens": st["lens_out"]}


def _plain_norm(st):
    c = st["case"]
    u = st["y"].float()
    if c["post"]:
        u = u * torch.rsqrt(u.square().mean(1, keepdim=True) + EPS) * st["w_post"].float()
    if st["gate"] is not None:
        u = u * st["gate"].float()
    h = (st["r"].float() + c["scale"] * u).to(st["r"].dtype)
    f = h.float()
    return {"h": h, "x": (f * torch.rsqrt(f.square().mean(1, keepdim=True) + EPS) * st["w_pre"].float()).half()}


def _plain_norm_bwd(st):
    c = st["case"]
    h, y, dx = st["h"].float(), st["y"].float(), st["dx"].float()
    rs = torch.rsqrt(h.square().mean(1, keepdim=True) + EPS)
    hh, a = h * rs, dx * st["w_pre"].float()
    t = st["dh"].float() + rs * (a - hh * (a * hh).mean(1, keepdim=True))
    du = c["scale"] * t * (1.0 if st["gate"] is None else st["gate"].float())
    out = {"dr": t.to(st["h"].dtype), "dw_pre": (dx * hh).sum(0), "dw_post": None, "dgate": None}
    u = y
    dy = du
    if c["post"]:
        rs = torch.rsqrt(y.square().mean(1, keepdim=True) + EPS)
        yh, a = y * rs, du * st["w_post"].float()
        u = yh * st["w_post"].float()
        dy = rs * (a - yh * (a * yh).mean(1, keepdim=True))
        out["dw_post"] = (du * yh).sum(0)
    if st["gate"] is not None:
        out["dgate"] = (c["scale"] * u * t).sum(0) if c["gate"] == "channel" else (c["scale"] * u * t).half()
    return {**out, "dy": dy.half()}


PLAIN = {"attn": _plain_attn, "append": _plain_append, "evict": _plain_evict, "norm": _plain_norm, "norm-bwd": _plain_norm_bwd}


def run(st):
    if own:
        return _run_own(st)
    return PLAIN[st["case"]["kind"]](st)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------


def work(case):
    kind = case["kind"]
    if kind.startswith("norm"):
        m, n = case["m"], case["n"]
        e = m * n
        res = 4 if case["f32"] else 2
        gate = {"none": 0, "channel": 2 * n, "token": 2 * e}[case["gate"]]
        if kind == "norm":       # y, r, gate and weights in; h and x out
            return {"bytes": e * (4 + 2 * res) + gate + 2 * n * (1 + case["post"]), "flops": e * (7 + 5 * case["post"])}
        # dx, dh, h, y, gate in; dr, dy, dgate and the weights' sums out
        out = {"none": 0, "channel": 4 * n, "token": 2 * e}[case["gate"]]
        return {"bytes": e * (6 + 3 * res) + gate + out + 6 * n * (1 + case["post"]), "flops": e * (16 + 12 * case["post"])}
    kv, d = case["kv"], case["d"]
    if kind == "append":
        t, heads = case["tokens"], case["heads"]
        return {"bytes": 4 * t * d * (heads + 2 * kv) + t * (12 + 4 * case["rot"]), "flops": 3 * t * case["rot"] * (heads + kv)}
    tokens = sum(_lengths(case, 0))
    if kind == "attn":
        return {"bytes": tokens * kv * (4 * d + (4 if case["weights"] else 0)) + 4 * case["seqs"] * case["heads"] * d, "flops": 4 * tokens * case["heads"] * d}
    # accumulated weights and positions of all tokens, those of the kept ones written; the kept ones that lie behind the budget moved
    kept = [(n, min(n, case["budget"])) for n in _lengths(case, 0)]
    moved = sum(k * (n - k) / n for n, k in kept)
    return {"bytes": kv * (8 * sum(n + k for n, k in kept) + moved * 8 * d), "flops": kv * tokens}


# ---- the definition in 64 bits -------------------------------------------------------------------------------------


def _exact_attn(case, st):
    seqs, heads, kv, d = case["seqs"], case["heads"], case["kv"], case["d"]
    out = torch.zeros((seqs, heads, d), dtype=torch.float64, device="cuda")
    weights = torch.zeros((seqs, kv, st["table"].shape[1] * case["page"]), dtype=torch.float64, device="cuda")
    q = st["q"].double().view(seqs, kv, heads // kv, d)
    for b, n in enumerate(st["lens"].tolist()):
        rows = st["table"][b].long()
        for h in range(kv):
            k = st["K"][rows, h].reshape(-1, d)[:n].double()
            p = torch.softmax(q[b, h] @ k.t() / d ** 0.5, 1)
            out[b, h * (heads // kv): (h + 1) * (heads // kv)] = p @ st["V"][rows, h].reshape(-1, d)[:n].double()
            weights[b, h, :n] = p.sum(0)
    return {"out": out.view(seqs, heads * d), "weights": weights if case["weights"] else None}


def _exact_append(case, st):
    d, half = case["d"], case["rot"] // 2
    t = torch.arange(case["tokens"], device="cuda")
    turned = []
    for name, heads in (("q", case["heads"]), ("k", case["kv"])):
        x = st[name].double().view(-1, heads, d).clone()
        if half:
            angle = torch.complex(*(st["rot"].double()[st["pos"].long()][:, i * half: (i + 1) * half] for i in (0, 1)))
            z = torch.complex(x[..., :half], x[..., half: 2 * half]) * angle[:, None]
            x[..., :half], x[..., half: 2 * half] = z.real, z.imag
        turned.append(x)
    K, V = st["K"].double(), st["V"].double()
    where, at = st["table"][st["seq"].long()].gather(1, (st["index"].long() // case["page"])[:, None])[:, 0].long(), st["index"].long() % case["page"]
    for h in range(case["kv"]):
        K[where, h, at] = turned[1][t, h]
        V[where, h, at] = st["v"].double()[t, h * d: (h + 1) * d]
    return {"q": turned[0].view(-1, case["heads"] * d), "k": K, "v": V}


def _exact_evict(case, st):
    if case["seqs"] * case["kv"] > 600:
        return None
    budget, page = case["budget"], case["page"]
    K, V = st["K"].double(), st["V"].double()
    score, pos, left = torch.zeros_like(st["score"], dtype=torch.float64), torch.zeros_like(st["pos"]), []
    for b, n in enumerate(st["lens"].tolist()):
        left.append(min(n, budget))
        for h in range(case["kv"]):
            s, p = st["score"][b, h, :n].tolist(), st["pos"][b, h, :n].tolist()
            to = list(range(left[b]))
            if n > budget:
                sure = [x < case["first"] or x >= n - case["last"] for x in p]
                kept = set(sorted(range(n), key=lambda i: (not sure[i], 0.0 if sure[i] else -s[i], i))[:budget])
                movers = iter(sorted(i for i in kept if i >= budget))
                to = [i if i in kept else next(movers) for i in range(budget)]
                src = torch.tensor([i for j, i in enumerate(to) if i != j], dtype=torch.long, device="cuda")
                dst = torch.tensor([j for j, i in enumerate(to) if i != j], dtype=torch.long, device="cuda")
                rows = st["table"][b].long()
                for pool in (K, V):
                    pool[rows[dst // page], h, dst % page] = pool[rows[src // page], h, src % page]
            score[b, h, :left[b]] = torch.tensor([s[i] for i in to], dtype=torch.float64)
            pos[b, h, :left[b]] = torch.tensor([p[i] for i in to], dtype=torch.int32)
    return {"k": K, "v": V, "score": score, "pos": pos, "lens": torch.tensor(left, dtype=torch.int32)}


def _exact_norm(case, st):
    def unit(z):
        return z / (z.pow(2).sum(1, keepdim=True) / case["n"] + EPS).sqrt()

    one = torch.ones((), dtype=torch.float64, device="cuda")
    wide = {k: v.double() for k, v in st.items() if isinstance(v, torch.Tensor)}
    y, gate, post = wide["y"], wide.get("gate", one), wide.get("w_post", one)
    if case["kind"] == "norm":
        h = wide["r"] + case["scale"] * gate * ((unit(y) * post) if case["post"] else y)
        return {"h": h, "x": unit(h) * wide["w_pre"]}
    # through the definition by automatic differentiation: dr is the gradient of r = h - what was added
    leaves = [t.detach().clone().requires_grad_() for t in (wide["h"] * 0, y, gate, post, wide["w_pre"])]
    dr, y, gate, post, pre = leaves
    added = case["scale"] * gate * ((unit(y) * post) if case["post"] else y)
    h = wide["h"] + dr + added - added.detach()
    loss = (unit(h) * pre * wide["dx"]).sum() + (h * wide["dh"]).sum()
    g = torch.autograd.grad(loss, leaves, allow_unused=True)
    return {"dr": g[0], "dy": g[1], "dgate": g[2] if case["gate"] != "none" else None, "dw_post": g[3] if case["post"] else None, "dw_pre": g[4]}


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"].startswith("norm"):
        return _exact_norm(case, st)
    return {"attn": _exact_attn, "append": _exact_append, "evict": _exact_evict}[case["kind"]](case, st)
