"""What a decoder has to do at the ends of its blocks' linear layers, as cases that can be timed and checked.

Three operators, eight kinds of case:
  logp       log probabilities of given tokens, the distributions' entropies and their `top` likeliest tokens, from rows of logits
  logp-bwd   the same without alternatives, then the gradient of the logits from those of log probability and entropy
  loss       log probabilities and, the gradient's weights being known before, the gradient of the logits, in one call
  qk         norms of each head of queries and keys and their rotation by position
  qk-bwd     its gradients
  qk-append  the same for new tokens, whose keys and values enter a paged cache
  adamw      an optimizer's step over many tensors; `clip`: the norm of all gradients before it; states in 32 bits or in 8
  norm       the norm of all gradients alone

The tensors of a step lie in flat buffers, each begins at a multiple of 128 values; what lies between them is zero and stays so.  8-bit states are e4m3 (first
moment) and e5m2 (second) with a power of two for every 128 values, rounded up or down at random by a number that is made from seed, step and place.
Where `own` is false everything is computed by elementary operations in 32 bits.
"""
import math

import torch

own = False

EPS = 1e-6
BLOCK = 128
BETA1, BETA2, ADAM_EPS = 0.9, 0.999, 1e-8
# hidden size, inner size, kv heads' width, blocks, weak columns of every layer
MODELS = {"small": (512, 1408, 128, 1, 8), "7b": (4096, 11008, 4096, 32, 128), "13b": (5120, 13824, 5120, 40, 128)}


def listed():
    return [
        # the smallest call: one token has been made, and its alternatives are shown
        dict(name="logp-token", kind="logp", m=1, n=32000, f32=False, top=5, scale=1.0, given=1.0, banned=0.0, entropy=True),
        # a batch of requests with a large vocabulary, sampled at a temperature, most of them with alternatives
        dict(name="logp-batch", kind="logp", m=57, n=130001, f32=False, top=20, scale=1.25, given=1.0, banned=0.0, entropy=True),
        # a prompt's own log probabilities; part of the vocabulary is ruled out; logits in 32 bits, an odd vocabulary
        dict(name="logp-prompt", kind="logp", m=2003, n=32003, f32=True, top=0, scale=1.0, given=1.0, banned=0.3, entropy=False),
        # a policy's gradient with an entropy term
        dict(name="logp-bwd", kind="logp-bwd", m=777, n=64007, f32=False, top=0, scale=1.0, given=0.9, banned=0.0, entropy=True),
        # fine-tuning: a batch's mean loss, prompts left out
        dict(name="loss-tune", kind="loss", m=4096, n=32000, f32=False, top=0, scale=1.0, given=0.7, banned=0.0, entropy=False),
        # the next token of eight sequences
        dict(name="qk-token", kind="qk-append", heads=32, kv=32, d=128, rot=128, m=8, page=16, norm=True),
        # fine-tuning, one sequence
        dict(name="qk-tune", kind="qk", heads=40, kv=40, d=128, rot=128, m=4096, norm=True),
        # the same backward, eight query heads to a kv head, an odd length
        dict(name="qk-bwd", kind="qk-bwd", heads=64, kv=8, d=128, rot=128, m=4001, norm=True),
        # one small block's weak columns and norms: a step is a few launches
        dict(name="adamw-block", kind="adamw", model="small", odd=0, bits=32, half=False, master=True, random=False, clip=True),
        # all weak columns, 32-bit states beside 32-bit weights, clipped
        dict(name="adamw-7b", kind="adamw", model="7b", odd=0, bits=32, half=False, master=True, random=False, clip=True),
        # all weak columns, 8-bit states, no second copy of the weights
        dict(name="adamw-13b-8bit", kind="adamw", model="13b", odd=0, bits=8, half=True, master=False, random=True, clip=False),
        # the norm alone
        dict(name="norm-7b", kind="norm", model="7b", odd=0, bits=32, half=True, master=False, random=False, clip=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("logp", "logp", "logp-bwd", "loss", "qk", "qk-bwd", "qk-append", "adamw", "adamw", "norm"))
    if kind in ("logp", "logp-bwd", "loss"):
        n = rng.choice((32000, _log(rng, 33, 262144), _log(rng, 20000, 160000)))
        return dict(kind=kind, m=_log(rng, 1, max(2, min(8192, (1 << 26) // n))), n=n, f32=rng.random() < 0.3,
                    top=rng.choice((0, 1, 5, rng.randint(2, 32))) if kind == "logp" else 0, scale=rng.choice((1.0, round(rng.uniform(0.5, 2.0), 3))),
                    given=rng.choice((1.0, round(rng.uniform(0.2, 1.0), 2))), banned=rng.choice((0.0, 0.0, round(rng.uniform(0.05, 0.95), 2))),
                    entropy=rng.random() < 0.5)
    if kind.startswith("qk"):
        heads, kv = rng.choice(((32, 32), (40, 40), (64, 8), (8, 8), (16, 4), (12, 2), (32, 1), (3, 3)))
        d = rng.choice((128, 128, 128, 64, 96, 80, 256, 40))
        rot = rng.choice((d, d, d // 2, 0))
        c = dict(kind=kind, heads=heads, kv=kv, d=d, rot=rot, m=_log(rng, 1, max(2, min(16384, (1 << 25) // ((heads + kv) * d)))), norm=rot == 0 or rng.random() < 0.7)
        if kind == "qk-append":
            c["page"] = rng.choice((8, 16, 16, 32, 64, 128))
        return c
    bits = rng.choice((32, 8))
    model = rng.choice(("small", "small", "7b", "13b" if bits == 8 else "7b"))
    return dict(kind=kind, model=model, odd=rng.choice((0, rng.randint(1, 200))), bits=bits, half=rng.random() < 0.5, master=rng.random() < 0.5,
                random=rng.random() < 0.5, clip=rng.random() < 0.5)


# ---- inputs --------------------------------------------------------------------------------------------------------


def _gen(seed, what):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 1013 + what)


def _normal(gen, *shape, std=1.0, dtype=torch.float16):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).mul_(std).to(dtype)


def _pitched(t):
    """The same values with rows that begin on 16 bytes."""
    m, n = t.shape
    if n % 8 == 0:
        return t
    out = torch.empty((m, (n + 7) // 8 * 8), dtype=t.dtype, device=t.device)[:, :n]
    return out.copy_(t)


def _sizes(case):
    """Host list: how many values each tensor has."""
    hidden, inner, kv, blocks, k = MODELS[case["model"]]
    out = [hidden * k, kv * k, kv * k, hidden * k, inner * k, inner * k, hidden * k, hidden, hidden] * blocks
    if case["odd"]:      # other ranks, and tensors of one value
        out = [max(1, n - (case["odd"] * (i + 3)) % n) if i % 3 else 1 + (case["odd"] * i) % (2 * BLOCK) for i, n in enumerate(out)]
    return out


def _starts(sizes):
    at, out = 0, []
    for n in sizes:
        out.append(at)
        at += -(-n // BLOCK) * BLOCK
    return out, at


def _logits(case, seed):
    m, n = case["m"], case["n"]
    t = torch.float32 if case["f32"] else torch.float16
    z = torch.randn((m, n), generator=_gen(seed, 1), device="cuda").mul_(2.0)
    z += torch.randn(n, generator=_gen(seed, 2), device="cuda") * 1.5 - 4          # some tokens are rare everywhere
    likely = torch.randint(0, n, (m, 4), generator=_gen(seed, 3), device="cuda")
    z.scatter_add_(1, likely, torch.rand((m, 4), generator=_gen(seed, 4), device="cuda") * 16)
    if case["banned"]:
        out = torch.rand(n, generator=_gen(seed, 5), device="cuda") < case["banned"]
        out[0] = False
        z.masked_fill_(out, float("-inf"))
    token = torch.where(torch.rand(m, generator=_gen(seed, 6), device="cuda") < 0.7, likely[:, 0], torch.randint(0, n, (m,), generator=_gen(seed, 7), device="cuda"))
    given = torch.rand(m, generator=_gen(seed, 8), device="cuda") <= case["given"]
    given[0] = True
    token = torch.where(given, token, -1)
    return _pitched(z.to(t)), token.int()


def _rotation(rot, positions):
    """[position][cos of rot / 2 frequencies, sin of them], angles in 64 bits."""
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    a = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float()


def _head_inputs(case, seed):
    heads, kv, d, m = case["heads"], case["kv"], case["d"], case["m"]
    st = dict(q=_normal(_gen(seed, 1), m, heads * d, std=3.0), k=_normal(_gen(seed, 2), m, kv * d, std=2.0), w_q=None, w_k=None)
    if case["norm"]:
        st.update(w_q=1 + _normal(_gen(seed, 3), d, std=0.2), w_k=1 + _normal(_gen(seed, 4), d, std=0.2))
    if case["kind"] == "qk-append":
        each = -(-m // min(m, 8))
        seqs = -(-m // each)
        # tokens of all sequences in one batch: sequence b has its share, after 100 + 17 b tokens that are there already
        seq = torch.arange(m, device="cuda") // each
        index = torch.arange(m, device="cuda") % each + 100 + 17 * seq
        most = each + 100 + 17 * seqs
        pages = -(-most // case["page"])
        table = torch.randperm(seqs * pages, generator=_gen(seed, 11), device="cuda").int().view(seqs, pages)
        K, V = (torch.empty((seqs * pages, kv, case["page"], d), dtype=torch.float16, device="cuda").normal_(generator=_gen(seed, s)) for s in (5, 6))
        st.update(seq=seq.int(), index=index.int(), pos=index.int(), table=table, K=K, V=V, v=_normal(_gen(seed, 7), m, kv * d))
    else:
        most = m + 37
        # sequences of a packed batch begin again at position 0
        st["pos"] = (torch.arange(m, device="cuda") % max(1, m // 3 + 1) + torch.randint(0, 37, (1,), generator=_gen(seed, 8), device="cuda")).int()
    if case["kind"] == "qk-bwd":
        st.update(gq=_normal(_gen(seed, 9), m, heads * d, std=0.1), gk=_normal(_gen(seed, 10), m, kv * d, std=0.1))
    st["rot"] = _rotation(case["rot"], most) if case["rot"] else None
    return st


def _tensor_inputs(case, seed):
    sizes = _sizes(case)
    starts, total = _starts(sizes)
    alive = torch.ones(total, dtype=torch.bool, device="cuda")
    for a, n in zip(starts, sizes):
        alive[a + n: a - (-n // BLOCK) * BLOCK] = False
    size = torch.exp(torch.randn(total // 4, generator=_gen(seed, 1), device="cuda") * 1.5).repeat_interleave(4)      # gradients of channels differ in size
    grad = (torch.randn(total, generator=_gen(seed, 2), device="cuda") * 1e-3 * size).masked_fill_(~alive, 0.0)
    st = dict(sizes=sizes, starts=starts, total=total, grad=grad.half() if case["half"] else grad)
    if case["kind"] == "norm":
        return st
    w = (torch.randn(total, generator=_gen(seed, 3), device="cuda") * 0.02).masked_fill_(~alive, 0.0)
    m = (torch.randn(total, generator=_gen(seed, 4), device="cuda") * 3e-4 * size).masked_fill_(~alive, 0.0)
    v = (torch.rand(total, generator=_gen(seed, 5), device="cuda") * size.square_() * 1.5e-6).masked_fill_(~alive, 0.0)
    st.update(weight=w.half(), master=w if case["master"] else None, step=37, seed=int(seed) + 5, lr=1e-4, decay=0.1)
    if case["bits"] == 32:
        st.update(m=m, v=v)
        return st
    for name, x, kind, top in (("m", m, torch.float8_e4m3fn, 7), ("v", v, torch.float8_e5m2, 14)):
        x = x.view(-1, BLOCK)
        e = (torch.frexp(x.abs().amax(1)).exponent - 1 - top).clamp_(-110, 127)
        e[x.abs().amax(1) == 0] = -127
        st[name + "_scale"] = (e + 127).to(torch.uint8)
        st[name] = torch.ldexp(x, -e[:, None]).to(kind).view(torch.uint8).view(-1)
    return st


def prepare(case, seed):
    st = dict(case=case)
    if case["kind"].startswith("qk"):
        st.update(_head_inputs(case, seed))
    elif case["kind"] in ("adamw", "norm"):
        st.update(_tensor_inputs(case, seed))
    else:
        z, token = _logits(case, seed)
        st.update(z=z, token=token)
        if case["kind"] == "loss":           # a mean over the tokens that count, times the scale that keeps fp16 gradients from vanishing
            st["dlogp"] = torch.full((case["m"],), -8192.0 / max(1.0, case["m"] * case["given"]), device="cuda")
        elif case["kind"] == "logp-bwd":     # advantages, and the entropy's weight
            st["dlogp"] = torch.randn(case["m"], generator=_gen(seed, 9), device="cuda") * 4
            st["dentropy"] = torch.full((case["m"],), -0.05, device="cuda")
    return st


# ---- the framework's operators -------------------------------------------------------------------------------------


def _kept(st, name, make):
    """What a program makes once and keeps: descriptions, workspaces, the plan of an optimizer's step, outputs."""
    if name not in st:
        st[name] = make()
    return st[name]


def _bytes(n):
    return torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")


def _f32(n):
    return torch.empty(n, dtype=torch.float32, device="cuda")


def _own_logits(st):
    from paper_2410_08661_amd import binding as B
    c = st["case"]
    m, z = c["m"], st["z"]
    desc = _kept(st, "desc", lambda: B.make_logprob_desc(c["n"], z.dtype, c["scale"]))
    o = _kept(st, "out", lambda: dict(logp=_f32(m), lse=_f32(m), entropy=_f32(m) if c["entropy"] else None, top_logp=_f32((m, c["top"])) if c["top"] else None,
                                      top_index=torch.empty((m, c["top"]), dtype=torch.int32, device="cuda") if c["top"] else None))
    ws = _kept(st, "ws", lambda: _bytes(B.qeft_logprob_workspace(desc, m, c["top"])))
    entropy = o["entropy"] if c["entropy"] else False
    if c["kind"] == "logp":
        B.qeft_logprob_fwd(desc, z, st["token"], top=c["top"], logp=o["logp"], lse=o["lse"], entropy=entropy, top_logp=o["top_logp"], top_index=o["top_index"], ws=ws)
        return dict(o)
    dz = _kept(st, "dz", lambda: torch.empty_strided(z.shape, z.stride(), dtype=z.dtype, device="cuda"))
    if c["kind"] == "loss":
        B.qeft_logprob_fwd_bwd(desc, z, st["token"], st["dlogp"], dz=dz, logp=o["logp"], lse=o["lse"], entropy=entropy, ws=ws)
    else:
        B.qeft_logprob_fwd(desc, z, st["token"], logp=o["logp"], lse=o["lse"], entropy=entropy, ws=ws)
        B.qeft_logprob_bwd(desc, z, o["lse"], token=st["token"], dlogp=st["dlogp"], entropy=o["entropy"], dentropy=st["dentropy"] if c["entropy"] else None, dz=dz)
    return {**o, "dz": dz}


def _own_heads(st):
    from paper_2410_08661_amd import binding as B
    c = st["case"]
    q, k = st["q"], st["k"]
    if c["kind"] == "qk-append":
        cache = _kept(st, "cache", lambda: B.Cache(B.make_cache_desc(st["K"].shape[0], c["page"], c["kv"], c["d"]), k=st["K"], v=st["V"]))
        out = _kept(st, "out", lambda: torch.empty_like(q))
        B.qeft_cache_append_norm(cache, st["table"], k, st["v"], st["index"], seq=st["seq"], q=q, q_out=out, rot=st["rot"], pos=st["pos"], w_q=st["w_q"], w_k=st["w_k"], eps=EPS)
        return {"q": out, "k": st["K"], "v": st["V"]}
    desc = _kept(st, "desc", lambda: B.make_qk_desc(c["d"], c["heads"], c["kv"], c["rot"], EPS))
    out = _kept(st, "out", lambda: (torch.empty_like(q), torch.empty_like(k)))
    if c["kind"] == "qk":
        B.qeft_qk_norm_fwd(desc, q, k, w_q=st["w_q"], w_k=st["w_k"], rot=st["rot"], pos=st["pos"], q_out=out[0], k_out=out[1])
        return {"q": out[0], "k": out[1]}
    sums = _kept(st, "sums", lambda: [_f32(c["d"]) if c["norm"] else None for _ in range(2)])
    ws = _kept(st, "ws", lambda: _bytes(B.qeft_qk_norm_workspace(desc, c["m"])))
    B.qeft_qk_norm_bwd(desc, st["gq"], st["gk"], q=q, k=k, w_q=st["w_q"], w_k=st["w_k"], rot=st["rot"], pos=st["pos"], dq=out[0], dk=out[1], dw_q=sums[0], dw_k=sums[1], ws=ws)
    return {"dq": out[0], "dk": out[1], "dw_q": sums[0], "dw_k": sums[1]}


def _own_tensors(st):
    from paper_2410_08661_amd import binding as B
    c = st["case"]

    def plan():
        at = list(zip(st["starts"], st["sizes"]))
        part = lambda t: None if t is None else [t[a: a + n] for a, n in at]  # noqa: E731
        if c["kind"] == "norm":
            return B.TensorList(grads=part(st["grad"]))
        scales = lambda t: None if c["bits"] == 32 else [t[a // BLOCK: a // BLOCK - (-n // BLOCK)] for a, n in at]  # noqa: E731
        return B.TensorList(grads=part(st["grad"]), weights=part(st["weight"]), masters=part(st["master"]), m=part(st["m"]), v=part(st["v"]),
                            m_scales=scales(st.get("m_scale")), v_scales=scales(st.get("v_scale")), decay=st["decay"])

    tensors = _kept(st, "plan", plan)
    norm = None
    if c["clip"] or c["kind"] == "norm":
        norm = _kept(st, "norm", lambda: _f32(2))
        ws = _kept(st, "ws", lambda: _bytes(B.qeft_grad_norm_workspace(tensors)))
        B.qeft_grad_norm(tensors, max_norm=1.0, scale=0.5, out=norm, ws=ws)
        if c["kind"] == "norm":
            return {"norm": norm}
    B.qeft_adamw_step(tensors, lr=st["lr"], step=st["step"], beta1=BETA1, beta2=BETA2, eps=ADAM_EPS, factor=None if norm is None else norm[1:], stochastic=c["random"], seed=st["seed"])
    return _state(st, norm)


def _state(st, norm):
    """The step's results; 8-bit states by the values that their bytes are, in the types that have them."""
    out = dict(norm=norm, weight=st["weight"], master=st["master"], m=st["m"], v=st["v"])
    if st["case"]["bits"] == 8:
        out.update(m=st["m"].view(torch.float8_e4m3fn), v=st["v"].view(torch.float8_e5m2), m_scale=st["m_scale"].view(torch.float8_e8m0fnu),
                   v_scale=st["v_scale"].view(torch.float8_e8m0fnu))
    return out


# ---- their plain forms ---------------------------------------------------------------------------------------------


def _statistics(c, z):
    """Scaled logits, their log-sum-exp and probabilities."""
    x = z.float() * c["scale"]
    top = x.amax(1, keepdim=True)
    e = torch.exp(x - top)
    s = e.sum(1, keepdim=True)
    return x, (top + torch.log(s))[:, 0], e.div_(s)


def _chosen(x, lse, token):
    """Log probabilities of the given tokens; rows without one have 0 everywhere."""
    has = token >= 0
    at = token.clamp(min=0).long()[:, None]
    return torch.where(has, x.gather(1, at)[:, 0] - lse, 0.0), has, at


def _entropy(x, lse, p):
    return -torch.where(p > 0, p * (x - lse[:, None]), 0.0).sum(1)


def _plain_logits(st):
    c = st["case"]
    x, lse, p = _statistics(c, st["z"])
    logp, has, at = _chosen(x, lse, st["token"])
    out = dict(logp=logp, lse=torch.where(has, lse, 0.0), entropy=None, top_logp=None, top_index=None)
    h = _entropy(x, lse, p) if c["entropy"] else None
    if c["entropy"]:
        out["entropy"] = torch.where(has, h, 0.0)
    if c["top"]:
        best, index = torch.sort(st["z"], dim=1, descending=True, stable=True)
        best, index = best[:, : c["top"]].float(), index[:, : c["top"]]
        pad = c["top"] - best.shape[1]
        best, index = torch.nn.functional.pad(best, (0, pad), value=float("-inf")), torch.nn.functional.pad(index, (0, pad))
        there = has[:, None] & (best > float("-inf"))
        out.update(top_logp=torch.where(there, best * c["scale"] - lse[:, None], float("-inf")), top_index=torch.where(there, index, -1).int())
    if c["kind"] == "logp":
        return out
    g = st["dlogp"][:, None]
    dz = p * -g
    if c["kind"] == "logp-bwd" and c["entropy"]:
        dz -= st["dentropy"][:, None] * torch.where(p > 0, p * (x - lse[:, None] + h[:, None]), 0.0)
    dz.scatter_add_(1, at, g)
    dz = torch.where(has[:, None], dz * c["scale"], 0.0)
    return {**out, "dz": dz.to(st["z"].dtype)}


def _turned(x, st, sign):
    """Heads' first `rot` values rotated in pairs half of them apart, there (+1) or back (-1); 32 bits."""
    half = st["case"]["rot"] // 2
    if not half:
        return x
    cs = st["rot"][st["pos"].long()][:, None]
    c, s = cs[..., :half], cs[..., half:] * sign
    a, b = x[..., :half], x[..., half: 2 * half]
    return torch.cat([a * c - b * s, b * c + a * s, x[..., 2 * half:]], -1)


def _normed(st, name, heads):
    x = st[name].float().view(-1, heads, st["case"]["d"])
    w = st["w_" + name]
    return x if w is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.float()


def _plain_heads(st):
    c = st["case"]
    q, k = (_turned(_normed(st, name, heads), st, 1).half() for name, heads in (("q", c["heads"]), ("k", c["kv"])))
    if c["kind"] == "qk":
        return {"q": q.view(c["m"], -1), "k": k.view(c["m"], -1)}
    page = st["table"].long()[st["seq"].long(), st["index"].long() // c["page"]]
    slot = st["index"].long() % c["page"]
    st["K"][page, :, slot] = k
    st["V"][page, :, slot] = st["v"].view(-1, c["kv"], c["d"])
    return {"q": q.view(c["m"], -1), "k": st["K"], "v": st["V"]}


def _head_grad(st, name, heads):
    x = st[name].float().view(-1, heads, st["case"]["d"])
    g = _turned(st["g" + name].float().view(x.shape), st, -1)
    w = st["w_" + name]
    if w is None:
        return g, None
    rs = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    unit, a = x * rs, g * w.float()
    return rs * (a - unit * (a * unit).mean(-1, keepdim=True)), (g * unit).double().sum((0, 1)).float()


def _plain_heads_bwd(st):
    c = st["case"]
    (dq, dw_q), (dk, dw_k) = _head_grad(st, "q", c["heads"]), _head_grad(st, "k", c["kv"])
    return {"dq": dq.half().view(c["m"], -1), "dk": dk.half().view(c["m"], -1), "dw_q": dw_q, "dw_k": dw_k}


MASK = 0xFFFFFFFF


def _mix(x):
    """A whole number's 32 bits stirred: two products with odd constants between shifts.  x: 64-bit tensors or Python numbers."""
    x = x & MASK
    x = x ^ (x >> 16)
    x = (x * 0x5C3C9CCD) & MASK
    x = x ^ (x >> 15)
    x = (x * 0xFA1B1BF1) & MASK
    return x ^ (x >> 16)


def _random(st):
    """32 random bits for every place of the flat buffers."""
    key = _mix(st["step"] + _mix((st["seed"] & MASK) + _mix(st["seed"] >> 32)))
    at = torch.arange(st["total"], device="cuda")
    return _mix((at & MASK) + _mix((at >> 32) + key))


def _cut(a, r, bits, bias, size):
    """Code of a >= 0 in a format of `bits` mantissa bits and this exponent bias: the float's low bits rounded up or down by r, of `size` bits."""
    drop = 23 - bits
    r = (r << (drop - size)).int()
    least = 2.0 ** (1 - bias)
    normal = ((a.view(torch.int32) + r) >> drop) - ((127 - bias) << bits)
    return torch.where(a >= least, normal, ((torch.clamp(a, max=least) * 2.0 ** (bias - 1 + 23)).int() + r) >> drop)


def _coded(x, r, bits, bias, top, floor):
    """8-bit codes of x with a power of two for every 128 of them, of which the largest lies in [2^top, 2^(top + 1)); and the powers."""
    x = x.view(-1, BLOCK)
    most = x.abs().amax(1)
    e = (torch.frexp(most).exponent - 1 - top).clamp(-110, 127)
    e = torch.where(most == 0, -127, e)
    a = torch.ldexp(x.abs(), -e[:, None])
    code = _cut(a, r.view(-1, BLOCK), bits, bias, 16)
    if floor:
        code = torch.where((code == 0) & (a > 0), 1, code)
    return (code | torch.where(x < 0, 128, 0)).to(torch.uint8).view(-1), (e + 127).to(torch.uint8)


def _decoded(code, scale, kind):
    return torch.ldexp(code.view(kind).float().view(-1, BLOCK), scale.int()[:, None] - 127).view(-1)


def _plain_norm(st):
    norm = 0.5 * st["grad"].double().square().sum().sqrt()
    return torch.stack([norm, 0.5 * torch.clamp(1.0 / norm, max=1.0)]).float()


def _plain_tensors(st):
    c = st["case"]
    norm = _plain_norm(st) if c["clip"] or c["kind"] == "norm" else None
    if c["kind"] == "norm":
        return {"norm": norm}
    g = st["grad"].float()
    if norm is not None:
        g = g * norm[1]
    m, v = st["m"], st["v"]
    if c["bits"] == 8:
        m, v = _decoded(m, st["m_scale"], torch.float8_e4m3fn), _decoded(v, st["v_scale"], torch.float8_e5m2)
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + (g * g) * (1 - BETA2)
    c1, c2 = 1 - BETA1 ** st["step"], 1 - BETA2 ** st["step"]
    w = st["weight"].float() if st["master"] is None else st["master"]
    w = w - (st["lr"] * st["decay"]) * w - (st["lr"] / c1 * math.sqrt(c2)) * (m / (v.sqrt() + ADAM_EPS * math.sqrt(c2)))
    r = _random(st) if c["bits"] == 8 or (c["random"] and not c["master"]) else None
    if c["master"]:
        st["master"].copy_(w)
    if c["random"] and not c["master"]:
        code = _cut(w.abs(), ((r * 0x5C3C9CCD) & MASK) >> 19, 10, 15, 13)
        st["weight"].copy_(torch.where(w < 0, code - 32768, code).to(torch.int16).view(torch.float16))
    else:
        st["weight"].copy_(w)
    if c["bits"] == 32:
        st["m"].copy_(m)
        st["v"].copy_(v)
    else:
        for name, got in (("m", _coded(m, r >> 16, 3, 7, 7, False)), ("v", _coded(v, r & 0xFFFF, 2, 15, 14, True))):
            st[name].copy_(got[0])
            st[name + "_scale"].copy_(got[1])
    return _state(st, norm)


def run(st):
    kind = st["case"]["kind"]
    if kind.startswith("qk"):
        return _own_heads(st) if own else _plain_heads_bwd(st) if kind == "qk-bwd" else _plain_heads(st)
    if kind in ("adamw", "norm"):
        return _own_tensors(st) if own else _plain_tensors(st)
    return _own_logits(st) if own else _plain_logits(st)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------


def work(case):
    kind = case["kind"]
    if kind in ("adamw", "norm"):
        n, e = sum(_sizes(case)), 2 if case["half"] else 4
        if kind == "norm":
            return {"bytes": n * e, "flops": 2 * n}
        # gradients read, states read and written, the 32-bit weights too or else the 16-bit ones, which are written in any case
        state = 16 if case["bits"] == 32 else 4 + 4 / BLOCK
        return {"bytes": n * (e + state + (10 if case["master"] else 4)), "flops": n * (14 + 2 * case["clip"])}
    m = case["m"]
    if kind.startswith("qk"):
        heads, kv, d = case["heads"], case["kv"], case["d"]
        x, turn = 2 * m * (heads + kv) * d, m * (4 * case["rot"] + 4)
        flops = m * (heads + kv) * (3 * case["rot"] + (4 * d if case["norm"] else 0))
        if kind == "qk-append":
            return {"bytes": 2 * x + 4 * m * kv * d + turn + 8 * m, "flops": flops}
        if kind == "qk":
            return {"bytes": 2 * x + turn, "flops": flops}
        return {"bytes": (3 if case["norm"] else 2) * x + turn, "flops": 3 * flops}
    # rows without a token need not be read, their gradient is zeros
    e, n, read = 4 if case["f32"] else 2, case["n"], m * case["given"]
    flops = read * n * (4 + 2 * case["entropy"])
    if kind == "logp":
        return {"bytes": read * n * e + m * (12 + 4 * case["entropy"] + 8 * case["top"]), "flops": flops}
    return {"bytes": (read + m) * n * e + m * 20, "flops": flops + 3 * read * n}


# ---- the definition in 64 bits -------------------------------------------------------------------------------------


def _exact_logits(case, st):
    m, n, s = case["m"], case["n"], case["scale"]
    z, token = st["z"], st["token"].tolist()
    out = {k: torch.zeros(m, dtype=torch.float64, device="cuda") for k in ("logp", "lse", "entropy")}
    out["top_logp"] = torch.full((m, case["top"]), -math.inf, dtype=torch.float64, device="cuda")
    out["top_index"] = torch.full((m, case["top"]), -1, dtype=torch.int32, device="cuda")
    dz = torch.zeros((m, n), dtype=torch.float64, device="cuda") if case["kind"] != "logp" else None
    order = torch.arange(n, device="cuda")
    for a in range(0, m, 64):
        rows = torch.arange(a, min(a + 64, m), device="cuda")
        rows = rows[st["token"][rows] >= 0]
        if not len(rows):
            continue
        x = z[rows].double() * s
        lse = torch.logsumexp(x, 1)
        logs = x - lse[:, None]
        p = logs.exp()
        t = st["token"][rows].long()
        plogs = torch.special.entr(p).sum(1)
        out["lse"][rows], out["entropy"][rows], out["logp"][rows] = lse, plogs, logs[torch.arange(len(rows), device="cuda"), t]
        left = z[rows].double()
        for j in range(case["top"]):
            best = left.amax(1, keepdim=True)
            at = torch.where(left == best, order, n).amin(1)
            there = (best[:, 0] > -math.inf) & (at < n)
            out["top_index"][rows, j] = torch.where(there, at, -1).int()
            out["top_logp"][rows, j] = torch.where(there, best[:, 0] * s - lse, -math.inf)
            left[torch.arange(len(rows), device="cuda"), at.clamp(max=n - 1)] = -math.inf
        if dz is not None:
            one = torch.nn.functional.one_hot(t, n).double()
            d = st["dlogp"].double()[rows, None] * (one - p)
            if case["kind"] == "logp-bwd" and case["entropy"]:
                d += st["dentropy"].double()[rows, None] * (torch.special.entr(p) - p * plogs[:, None])
            dz[rows] = s * d
    if not case["entropy"]:
        out["entropy"] = None
    if not case["top"]:
        out["top_logp"] = out["top_index"] = None
    return {**out, "dz": dz} if dz is not None else out


def _exact_heads(case, st):
    m, d, half = case["m"], case["d"], case["rot"] // 2

    def of(x, w, heads):
        x = x.view(m, heads, d)
        if w is not None:
            x = x / (x.pow(2).sum(-1, keepdim=True) / d + EPS).sqrt() * w
        if half:
            turn = torch.complex(*(st["rot"].double()[st["pos"].long()][:, i * half: (i + 1) * half] for i in (0, 1)))
            y = torch.complex(x[..., :half], x[..., half: 2 * half]) * turn[:, None]
            x = torch.cat([y.real, y.imag, x[..., 2 * half:]], -1)
        return x

    if case["kind"] == "qk-bwd":      # by automatic differentiation
        out = {}
        for name, heads in (("q", case["heads"]), ("k", case["kv"])):
            w = st["w_" + name]
            leaves = [st[name].double().requires_grad_()] + ([w.double().requires_grad_()] if w is not None else [])
            y = of(leaves[0], leaves[1] if w is not None else None, heads)
            g = torch.autograd.grad((y * st["g" + name].double().view(y.shape)).sum(), leaves)
            out["d" + name], out["dw_" + name] = g[0], g[1] if w is not None else None
        return out
    q, k = (of(st[n].double(), None if st["w_" + n] is None else st["w_" + n].double(), h) for n, h in (("q", case["heads"]), ("k", case["kv"])))
    if case["kind"] == "qk":
        return {"q": q.reshape(m, -1), "k": k.reshape(m, -1)}
    K, V = st["K"].double(), st["V"].double()
    t = torch.arange(m, device="cuda")
    where, at = st["table"][st["seq"].long()].gather(1, (st["index"].long() // case["page"])[:, None])[:, 0].long(), st["index"].long() % case["page"]
    for h in range(case["kv"]):
        K[where, h, at] = k[t, h]
        V[where, h, at] = st["v"].double()[t, h * d: (h + 1) * d]
    return {"q": q.reshape(m, -1), "k": K, "v": V}


def _exact_tensors(case, st):
    """Moments and weights from the formulas; what is kept in few bits lies on their grid, the lower or the upper neighbour as the place's random number says."""
    total = st["total"]
    g = st["grad"].double()
    norm = None
    if case["clip"] or case["kind"] == "norm":
        length = torch.linalg.vector_norm(g) * 0.5
        norm = torch.stack([length, 0.5 / length if length > 1 else torch.full_like(length, 0.5)])
        if case["kind"] == "norm":
            return {"norm": norm}
        g *= norm[1]
    out = dict(norm=norm, master=None)
    dice = None
    if case["bits"] == 8 or (case["random"] and not case["master"]):
        def stir(x):
            for shift, factor in ((16, 0x5C3C9CCD), (15, 0xFA1B1BF1), (16, 1)):
                x = ((x ^ (x >> shift)) * factor) % (1 << 32)
            return x
        top, low = divmod(st["seed"], 1 << 32)
        key = stir((st["step"] + stir((low + stir(top)) % (1 << 32))) % (1 << 32))
        dice = stir((torch.arange(total, device="cuda") + stir(key)) % (1 << 32))      # (fewer than 2^32 places)

    def grid(x, u, bits, least):
        """x >= 0 to a multiple of its binade's step, or of the smallest binade's: up where the rest and u in [0, 1) make a whole step."""
        step = torch.exp2(torch.floor(torch.log2(x.clamp(min=least))) - bits)
        return torch.floor(x / step + u) * step

    new = {}
    for name, kind, beta, add in (("m", torch.float8_e4m3fn, BETA1, g), ("v", torch.float8_e5m2, BETA2, g * g)):
        old = st[name].double() if case["bits"] == 32 else (st[name].view(kind).double().view(-1, BLOCK) * torch.exp2(st[name + "_scale"].double() - 127)[:, None]).view(-1)
        new[name] = old.mul_(beta).add_(add, alpha=1 - beta)
    del g
    c1, c2 = 1 - BETA1 ** st["step"], 1 - BETA2 ** st["step"]
    w = st["weight"].double() if st["master"] is None else st["master"].double()
    w = w * (1 - st["lr"] * st["decay"]) - st["lr"] * (new["m"] / c1) / ((new["v"] / c2).sqrt() + ADAM_EPS)
    if case["master"]:
        out["master"] = w
    if case["random"] and not case["master"]:
        w = grid(w.abs(), ((dice * 0x5C3C9CCD) % (1 << 32) >> 19).double() / 8192, 10, 2.0 ** -14) * w.sign()
    out["weight"] = w
    if case["bits"] == 32:
        return {**out, **new}
    for name, bits, least, top, u in (("m", 3, 2.0 ** -6, 7, dice >> 16), ("v", 2, 2.0 ** -14, 14, dice % 65536)):
        x = new.pop(name).view(-1, BLOCK)
        most = x.abs().amax(1)
        e = torch.where(most > 0, torch.floor(torch.log2(most.clamp(min=1e-300))) - top, -17.0).clamp(-110, 127)
        e[most == 0] = -127.0
        a = x.abs() / torch.exp2(e)[:, None]
        c = grid(a, u.double().view(-1, BLOCK) / 65536, bits, least)
        if name == "v":
            c = torch.where((c == 0) & (a > 0), 2.0 ** -16, c)
        out[name], out[name + "_scale"] = (c * x.sign()).view(-1), torch.exp2(e)
    return out


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"].startswith("qk"):
        return _exact_heads(case, st)
    return _exact_tensors(case, st) if case["kind"] in ("adamw", "norm") else _exact_logits(case, st)
