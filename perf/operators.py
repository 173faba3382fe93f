"""The operators of a beam-decode step, measured: their inputs, a plain form of
each, the work it cannot do without and a 64-bit reference.

A decode step of B requests with K beams each runs B*K tokens: every beam's
token attends to the prompt that its request's beams share and to the beam's
own suffix (prefix_attention), passes the MoE layers (layer_decode), the best
continuations of each request are chosen over its beams and the vocabulary
(beam_select), and the suffix caches follow their parents (beam_reorder).

A case is a dict of plain values; its "kind" names the operator. Where `own` is
false a pass runs elementary torch operations in 32 bits (64 for logits whose
order decides), where it is true the package's entry points. Layer shapes are
those of synth.WORKLOADS; the attention and the vocabularies are generic.
"""
import math

import torch

own = False

DEV = "cuda:0"

FAMILIES = {
    "mixtral": dict(dtype="bf16", H=4096, E=8, F=14336, k=2, shared=0, zipf=0.0, renorm=True),
    "qwen": dict(dtype="bf16", H=2048, E=60, F=1408, k=4, shared=4, zipf=1.2, renorm=False),
    "deepseek": dict(dtype="bf16", H=2048, E=64, F=1408, k=6, shared=2, zipf=1.0, renorm=False),
    "tiny": dict(dtype="f32", H=128, E=8, F=256, k=2, shared=0, zipf=0.0, renorm=True),
}


def _layer(family, T, resident=None, name=None, **over):
    c = dict(FAMILIES[family], kind="layer", T=T)
    c.update(over)
    c["S"] = c["E"] if resident is None else resident
    if name:
        c["name"] = name
    return c


def _attn(G, K, P, S, Hq, Hkv, D, dtype="bf16", ragged=False, name=None):
    """G groups of K rows (ragged: 1 to 2K - 1 of them) over prefixes of up to P
    and suffixes of up to S keys."""
    c = dict(kind="attn", G=G, K=K, P=P, S=S, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, ragged=ragged)
    if name:
        c["name"] = name
    return c


def _select(B, K, V, n, dtype="bf16", done=0, name=None):
    """done: every done-th beam has finished (0: none)."""
    c = dict(kind="select", B=B, K=K, V=V, n=n, dtype=dtype, done=done)
    if name:
        c["name"] = name
    return c


def _reorder(L, B, K, S, unit, moved, name=None):
    """moved of a request's K beams take over another beam's states."""
    c = dict(kind="reorder", L=L, B=B, K=K, S=S, unit=unit, moved=moved)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # a step of one request with eight beams through the tiny float32 layer:
        # launches and nothing else
        _layer("tiny", 8, name="layer_tiny_f32_t8"),
        # one token of one sequence over many small experts and shared ones
        _layer("qwen", 1, name="layer_qwen_t1"),
        # an odd number of sequences, 40 of 64 experts resident, some choices missed
        _layer("deepseek", 13, resident=40, name="layer_deepseek_t13"),
        # four requests of eight beams over few large experts: the weight stream
        _layer("mixtral", 32, name="layer_mixtral_t32"),
        # float32 heads of 64, one short prompt, four beams
        _attn(1, 4, 100, 7, 8, 2, 64, dtype="f32", name="attn_f32_p100"),
        # one request, four beams, a prompt of some hundred tokens
        _attn(1, 4, 777, 33, 32, 8, 128, name="attn_k4_p777"),
        # sixteen requests of about eight beams, prompts of different lengths,
        # one query head per key head
        _attn(16, 8, 4096, 160, 16, 16, 128, ragged=True, name="attn_b16_k8_p4096"),
        # a decode batch of 64 sequences behind one long shared prompt
        _attn(1, 64, 65536, 500, 32, 8, 128, name="attn_r64_p65536"),
        # one request, four beams, a vocabulary of 32000, float32 logits
        _select(1, 4, 32000, 4, dtype="f32", name="select_k4_v32000"),
        # 64 requests of eight beams, a large vocabulary, twice as many
        # candidates as beams, some beams finished
        _select(64, 8, 128000, 16, done=11, name="select_b64_k8_v128000"),
        # one request's suffixes, one beam of four replaced
        _reorder(24, 1, 4, 40, 4096, 1, name="reorder_k4_s40"),
        # sixteen requests of eight beams with long suffixes, three replaced
        _reorder(32, 16, 8, 500, 2048, 3, name="reorder_b16_k8_s500"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["mixtral", "qwen", "deepseek", "generic", "tiny", "attn", "attn", "shared",
                       "attn_f32", "select", "select", "reorder", "reorder"])
    if kind == "mixtral":
        return _layer("mixtral", _log_int(rng, 1, 32), resident=rng.choice([8, 8, 4]))
    if kind == "qwen":
        return _layer("qwen", _log_int(rng, 1, 64))
    if kind == "deepseek":
        return _layer("deepseek", _log_int(rng, 1, 64), resident=rng.randint(24, 64))
    if kind == "generic":
        E = rng.choice([2, 4, 16, 33, 128])
        return _layer("mixtral", _log_int(rng, 1, 64), H=8 * _log_int(rng, 16, 320),
                      F=8 * _log_int(rng, 16, 320), E=E, k=rng.choice([1, 2]), resident=E,
                      shared=rng.choice([0, 1, 2]), renorm=rng.choice([True, False]))
    if kind == "tiny":
        E = rng.choice([4, 8, 16])
        return _layer("tiny", _log_int(rng, 1, 64), H=4 * _log_int(rng, 16, 128),
                      F=4 * _log_int(rng, 32, 256), E=E, k=rng.choice([1, 2]), resident=E)
    if kind == "attn":
        Hkv, q = rng.choice([(8, 4), (16, 1), (2, 8), (4, 7), (1, 16)])
        return _attn(_log_int(rng, 1, 16), rng.choice([1, 2, 4, 5, 8]), _log_int(rng, 1, 4096),
                     _log_int(rng, 1, 256), Hkv * q, Hkv, rng.choice([64, 80, 128, 128]),
                     ragged=rng.choice([True, False]))
    if kind == "shared":
        Hkv, q = rng.choice([(8, 4), (4, 8), (16, 1)])
        return _attn(1, _log_int(rng, 4, 64), _log_int(rng, 1024, 32768), _log_int(rng, 1, 512),
                     Hkv * q, Hkv, 128)
    if kind == "attn_f32":
        Hkv, q = rng.choice([(2, 4), (4, 1), (3, 2)])
        return _attn(rng.randint(1, 4), rng.randint(1, 6), _log_int(rng, 1, 1024),
                     _log_int(rng, 1, 128), Hkv * q, Hkv, rng.choice([32, 64, 128]), dtype="f32",
                     ragged=rng.choice([True, False]))
    if kind == "select":
        K = rng.choice([1, 2, 3, 4, 5, 8])
        return _select(_log_int(rng, 1, 64), K, _log_int(rng, 500, 128000), rng.choice([K, 2 * K]),
                       dtype=rng.choice(["bf16", "f32"]) if K <= 4 else "bf16",
                       done=rng.choice([0, 0, 7]))
    K = rng.choice([2, 3, 4, 8])
    return _reorder(rng.choice([2, 24, 32]), _log_int(rng, 1, 16), K, _log_int(rng, 1, 400),
                    rng.choice([512, 1000, 1024, 2048]), rng.randint(1, K - 1))


# ---------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _normal(g, shape, std, dtype):
    out = torch.empty(shape, dtype=dtype, device=DEV)
    return out.normal_(0.0, std, generator=g)


def _prepare_layer(case, seed):
    """Hidden states N(0,1), weights N(0, 0.02), Zipf-skewed routers where the
    model has them; the S experts the bias favours are resident."""
    g = _gen(seed)
    T, H, E, F, S = (case[n] for n in ("T", "H", "E", "F", "S"))
    dt = _type(case)
    s = dict(case=case, x=_normal(g, (T, H), 1.0, dt), w_router=_normal(g, (E, H), 0.02, dt),
             bias=None, slot=None, shared=None)
    order = torch.randperm(E, generator=g, device=DEV)
    if case["zipf"]:
        mass = torch.arange(1, E + 1, dtype=torch.float64, device=DEV) ** -case["zipf"]
        b = torch.empty(E, dtype=torch.float64, device=DEV)
        b[order] = torch.log(mass / mass.sum())
        s["bias"] = b.float()
    if S < E:
        slot = torch.full((E,), -1, dtype=torch.int32, device=DEV)
        slot[order[:S].sort().values] = torch.arange(S, dtype=torch.int32, device=DEV)
        s["slot"] = slot
    s["w_gate"] = _normal(g, (S, F, H), 0.02, dt)
    s["w_up"] = _normal(g, (S, F, H), 0.02, dt)
    s["w_down"] = _normal(g, (S, H, F), 0.02, dt)
    if case["shared"]:
        Fs = case["shared"] * F
        s["shared"] = (_normal(g, (Fs, H), 0.02, dt), _normal(g, (Fs, H), 0.02, dt),
                       _normal(g, (H, Fs), 0.02, dt))
    if own:
        from paper_2410_17954_amd import ops
        s["y"] = torch.empty((T, H), dtype=dt, device=DEV)
        s["idx"] = torch.empty((T, case["k"]), dtype=torch.int32, device=DEV)
        s["gates"] = torch.empty((T, case["k"]), dtype=torch.float32, device=DEV)
        s["inc"] = torch.empty(T, dtype=torch.int32, device=DEV)
        s["ws"] = ops.workspace_tensor(
            ops.layer_decode_workspace(T, H, F, E, case["k"], case["shared"] * F,
                                       ops.MOE_F32 if case["dtype"] == "f32" else ops.MOE_BF16),
            DEV)
    return s


def _group_sizes(case):
    K = case["K"]
    return [1 + (5 * g + K - 1) % (2 * K - 1) if case["ragged"] else K for g in range(case["G"])]


def _lengths(case):
    """Keys of every group's prefix and of every row's suffix: the longest first
    for each, then between half of it and all (at least one)."""
    P, S = case["P"], case["S"]
    pl = [P - (g * 1237) % (P // 2 + 1) for g in range(case["G"])]
    sl = [S - (r * 29) % (S // 2 + 1) for r in range(sum(_group_sizes(case)))]
    return pl, sl


def _prepare_attn(case, seed):
    """Queries and keys whose scores have a standard deviation of about two, a
    first key that every query favours, as trained heads have it."""
    g = _gen(seed)
    G, P, S, Hq, Hkv, D = (case[n] for n in ("G", "P", "S", "Hq", "Hkv", "D"))
    dt = _type(case)
    sizes = _group_sizes(case)
    R = sum(sizes)
    pl, sl = _lengths(case)
    q = torch.empty((R, Hq, D), device=DEV).normal_(0.0, 2.0, generator=g)
    k_prefix = _normal(g, (G, P, Hkv, D), 1.0, dt)
    k_prefix[:, 0] += (0.5 * q.view(R, Hkv, Hq // Hkv, D).mean((0, 2))).to(dt)
    offs = [0]
    for n in sizes:
        offs.append(offs[-1] + n)
    s = dict(case=case, offs=offs, q=q.to(dt), k_prefix=k_prefix,
             v_prefix=_normal(g, (G, P, Hkv, D), 1.0, dt),
             k_suffix=_normal(g, (R, S, Hkv, D), 1.0, dt),
             v_suffix=_normal(g, (R, S, Hkv, D), 1.0, dt), scale=D ** -0.5,
             prefix_len=torch.tensor(pl, dtype=torch.int32, device=DEV),
             suffix_len=torch.tensor(sl, dtype=torch.int32, device=DEV),
             group_offsets=torch.tensor(offs, dtype=torch.int32, device=DEV))
    if own:
        from paper_2410_17954_amd import ops
        s["out"] = torch.empty((R, Hq, D), dtype=dt, device=DEV)
        s["lse"] = torch.empty((R, Hq), dtype=torch.float32, device=DEV)
        s["ws"] = ops.workspace_tensor(
            ops.prefix_attention_workspace(R, G, Hq, Hkv, D, P, S,
                                           ops.MOE_F32 if case["dtype"] == "f32" else ops.MOE_BF16),
            DEV)
    return s


def _prepare_select(case, seed):
    """Logits N(0, 2.5) with a few clear favourites a row; a request's beams lie
    a few units apart."""
    g = _gen(seed)
    B, K, V = case["B"], case["K"], case["V"]
    z = torch.empty((B, K, V), device=DEV).normal_(0.0, 2.5, generator=g)
    top = torch.randint(0, V, (B, K, 3), device=DEV, generator=g)
    z.scatter_add_(2, top, torch.rand((B, K, 3), device=DEV, generator=g) * 6.0 + 6.0)
    scores = -20.0 * torch.rand((B, 1), device=DEV, generator=g) \
        - 3.0 * torch.rand((B, K), device=DEV, generator=g)
    s = dict(case=case, logits=z.to(_type(case)), scores=scores, finished=None, eos=2)
    if case["done"]:
        rows = torch.arange(B * K, device=DEV).view(B, K)
        s["finished"] = (rows % case["done"] == case["done"] - 1).int()
    if own:
        from paper_2410_17954_amd import ops
        n = case["n"]
        for name in ("parent", "token", "flags"):
            s[name] = torch.empty((B, n), dtype=torch.int32, device=DEV)
        s["best"] = torch.empty((B, n), dtype=torch.float32, device=DEV)
        s["ws"] = ops.workspace_tensor(ops.beam_select_workspace(B, K, V, n), DEV)
    return s


def _prepare_reorder(case, seed):
    """Keys and values of the beams' suffixes as bytes. Of a request's beams
    `moved` die; the beams that live on keep their rows, and the dead ones' rows
    take over copies of them in turn."""
    g = _gen(seed)
    L, B, K, S, unit, m = (case[n] for n in ("L", "B", "K", "S", "unit", "moved"))
    caches = []
    for _ in range(2):
        c = torch.empty((L, B * K, S, unit), dtype=torch.uint8, device=DEV)
        c.random_(0, 256, generator=g)
        caches.append(c)
    order = torch.rand((B, K), device=DEV, generator=g).argsort(1)
    kept, dead = order[:, m:], order[:, :m]
    parent = torch.arange(K, device=DEV).expand(B, K).clone()
    parent.scatter_(1, dead, kept[:, torch.arange(m, device=DEV) % (K - m)])
    parent += K * torch.arange(B, device=DEV)[:, None]
    lens = (S - (torch.arange(B, device=DEV) * 7) % (S // 2 + 1)).repeat_interleave(K).int()
    return dict(case=case, caches=caches, parent=parent.int(), lens=lens,
                new_lens=torch.empty_like(lens),
                err=torch.zeros(1, dtype=torch.int32, device=DEV))


def prepare(case, seed):
    return _PREPARE[case["kind"]](case, seed)


# ------------------------------------------------------------ plain forms
def _plain_layer(s):
    c = s["case"]
    x = s["x"].float()
    z = s["x"].double() @ s["w_router"].double().T
    if s["bias"] is not None:
        z = z + s["bias"].double()
    idx = z.sort(dim=1, descending=True, stable=True).indices[:, :c["k"]]
    p = torch.exp((z - z.max(1, keepdim=True).values).float())
    w = p.gather(1, idx)
    w = w / (w if c["renorm"] else p).sum(1, keepdim=True)

    def ffn(v, wg, wu, wd):
        a = v @ wg.float().T
        a = a / (1.0 + torch.exp(-a)) * (v @ wu.float().T)
        return a @ wd.float().T

    y = torch.zeros_like(x)
    slot = list(range(c["E"])) if s["slot"] is None else s["slot"].tolist()
    for e, sl in enumerate(slot):
        if sl < 0:
            continue
        t, j = (idx == e).nonzero(as_tuple=True)
        if t.numel():
            y.index_add_(0, t, w[t, j, None] * ffn(x[t], s["w_gate"][sl], s["w_up"][sl],
                                                   s["w_down"][sl]))
    if s["shared"] is not None:
        y += ffn(x, *s["shared"])
    missed = torch.zeros(c["T"], dtype=torch.int32, device=DEV)
    if s["slot"] is not None:
        missed = (s["slot"][idx] < 0).any(1).int()
    return dict(y=y.to(s["x"].dtype), idx=idx.int(), gates=w, incomplete=missed)


def _plain_attn(s):
    c = s["case"]
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    n_q = Hq // Hkv
    out, lse = [], []
    pos_p, pos_s = (torch.arange(c[n], device=DEV) for n in ("P", "S"))
    for g in range(c["G"]):
        lo, hi = s["offs"][g], s["offs"][g + 1]
        n = hi - lo
        q = s["q"][lo:hi].float().view(n, Hkv, n_q, D) * s["scale"]
        # the prefix: all rows of the group against the same keys, head by head
        qh = q.permute(1, 0, 2, 3).reshape(Hkv, n * n_q, D)
        kp = s["k_prefix"][g].float().permute(1, 2, 0).contiguous()
        sp = (qh @ kp).masked_fill(pos_p >= s["prefix_len"][g], -math.inf)
        sp = sp.view(Hkv, n, n_q, c["P"])
        # the suffixes: every row against its own
        ks = s["k_suffix"][lo:hi].float().permute(2, 0, 3, 1).contiguous()
        ss = q.permute(1, 0, 2, 3) @ ks
        ss = ss.masked_fill((pos_s >= s["suffix_len"][lo:hi, None])[:, None, :], -math.inf)
        m = torch.maximum(sp.amax(-1), ss.amax(-1))
        ep, es = torch.exp(sp - m[..., None]), torch.exp(ss - m[..., None])
        den = ep.sum(-1) + es.sum(-1)
        vp = s["v_prefix"][g].float().permute(1, 0, 2).contiguous()
        vs = s["v_suffix"][lo:hi].float().permute(2, 0, 1, 3).contiguous()
        o = (ep.reshape(Hkv, n * n_q, c["P"]) @ vp).view(Hkv, n, n_q, D) + es @ vs
        o = o / den[..., None]
        out.append(o.permute(1, 0, 2, 3).reshape(n, Hq, D))
        lse.append((m + torch.log(den)).permute(1, 0, 2).reshape(n, Hq))
    return dict(out=torch.cat(out).to(s["q"].dtype), lse=torch.cat(lse))


def _plain_select(s):
    c = s["case"]
    B, K, V, n = (c[x] for x in ("B", "K", "V", "n"))
    z = s["logits"].double()
    m = z.amax(-1, keepdim=True)
    cand = z - (m + torch.log(torch.exp(z - m).sum(-1, keepdim=True)))
    cand += s["scores"].double()[..., None]
    if s["finished"] is not None:
        done = s["finished"] != 0
        stay = torch.full_like(cand[0, 0], -math.inf)
        stay[s["eos"]] = 0.0
        cand = torch.where(done[..., None], s["scores"].double()[..., None] + stay, cand)
    best = cand.view(B, K * V).sort(dim=1, descending=True, stable=True)
    pos = best.indices[:, :n]
    beam, token = pos // V, pos % V
    row = beam + K * torch.arange(B, device=DEV)[:, None]
    flags = token == s["eos"]
    if s["finished"] is not None:
        flags = flags | done.gather(1, beam)
    return dict(parent=row.int(), token=token.int(), score=best.values[:, :n].float(),
                finished=flags.int())


def _plain_reorder(s):
    c = s["case"]
    src = s["parent"].reshape(-1).long()
    rows = torch.arange(src.numel(), device=DEV)
    keep = (torch.arange(c["S"], device=DEV) < s["lens"][src][:, None]) & (src != rows)[:, None]
    for cache in s["caches"]:
        for layer in cache:
            layer.copy_(torch.where(keep[..., None], layer[src], layer))
    return dict(caches=list(s["caches"]), lens=s["lens"][src], err=s["err"])


# ----------------------------------------------------------- entry points
def _own_layer(s):
    from paper_2410_17954_amd import ops
    c = s["case"]
    y, idx, w, inc = ops.layer_decode(
        s["x"], s["w_router"], s["w_gate"], s["w_up"], s["w_down"], c["k"], bias=s["bias"],
        renormalize=c["renorm"], slot_of_expert=s["slot"], shared=s["shared"], y=s["y"],
        topk_idx=s["idx"], topk_w=s["gates"], incomplete=s["inc"], workspace=s["ws"])
    return dict(y=y, idx=idx, gates=w, incomplete=inc)


def _own_attn(s):
    from paper_2410_17954_amd import ops
    out, lse = ops.prefix_attention(
        s["q"], s["k_prefix"], s["v_prefix"], s["k_suffix"], s["v_suffix"],
        prefix_len=s["prefix_len"], suffix_len=s["suffix_len"],
        group_offsets=s["group_offsets"], scale=s["scale"], out=s["out"], lse=s["lse"],
        workspace=s["ws"])
    return dict(out=out, lse=lse)


def _own_select(s):
    from paper_2410_17954_amd import ops
    parent, token, score, flags = ops.beam_select(
        s["logits"], s["scores"], s["case"]["n"], finished=s["finished"], eos=s["eos"],
        parent=s["parent"], token=s["token"], out_scores=s["best"], out_finished=s["flags"],
        workspace=s["ws"])
    return dict(parent=parent, token=token, score=score, finished=flags)


def _own_reorder(s):
    from paper_2410_17954_amd import ops
    lens, err = ops.beam_reorder(s["caches"], s["parent"], lens=s["lens"], new_lens=s["new_lens"],
                                 err=s["err"])
    return dict(caches=list(s["caches"]), lens=lens, err=err)


def run(state):
    kind = state["case"]["kind"]
    return (_OWN if own else _PLAIN)[kind](state)


# ------------------------------------------------------------------ work
def _elt(case):
    return 4 if case["dtype"] == "f32" else 2


def _work_layer(c):
    """Weights of the experts that T tokens of k choices are expected to reach
    (as if drawn by the router's bias), once each; missed choices are not
    computed."""
    T, H, E, F, k, S = (c[n] for n in ("T", "H", "E", "F", "k", "S"))
    mass = [(i + 1.0) ** -c["zipf"] for i in range(E)]
    rate = [0.0] * E                   # chance that a token chooses expert i
    total = sum(mass)
    lo, hi = 0.0, 1e9                  # sum_i 1 - exp(-u mass_i) = k
    for _ in range(100):
        u = (lo + hi) / 2
        rate = [1.0 - math.exp(-u * m / total) for m in mass]
        lo, hi = (u, hi) if sum(rate) < k else (lo, u)
    hit = sum(1.0 - (1.0 - r) ** T for r in rate[:S])
    pairs = T * sum(rate[:S])
    elt, Fs = _elt(c), c["shared"] * F
    nbytes = elt * (2 * T * H + E * H + 3 * H * (F * hit + Fs)) + 8 * T * k + 4 * T
    return {"bytes": nbytes, "flops": 2.0 * T * H * E + 6.0 * H * (F * pairs + Fs * T)}


def _work_attn(c):
    pl, sl = _lengths(c)
    sizes = _group_sizes(c)
    R, elt, D = sum(sizes), _elt(c), c["D"]
    keys = sum(n * p for n, p in zip(sizes, pl)) + sum(sl)
    nbytes = elt * (2 * c["Hkv"] * D * (sum(pl) + sum(sl)) + 2 * R * c["Hq"] * D) \
        + 4 * R * c["Hq"]
    return {"bytes": nbytes, "flops": 4.0 * D * c["Hq"] * keys}


def _work_select(c):
    rows, done = c["B"] * c["K"], c["done"]
    live = rows - (rows // done if done else 0)
    return {"bytes": live * c["V"] * _elt(c) + 4 * rows + 16 * c["B"] * c["n"],
            "flops": 4.0 * live * c["V"]}


def _work_reorder(c):
    K, S, m = c["K"], c["S"], c["moved"]
    keys = sum(S - (b * 7) % (S // 2 + 1) for b in range(c["B"]))
    rows = m + min(m, K - m)           # written, and read once
    return {"bytes": 2 * c["L"] * keys * c["unit"] * rows + 12 * c["B"] * K, "flops": 0}


def work(case):
    return _WORK[case["kind"]](case)


# ------------------------------------------------------ 64-bit reference
def _exact_layer(case, seed):
    s = _prepare_layer(case, seed)
    x = s["x"].double()
    z = torch.stack([(x * r).sum(1) for r in s["w_router"].double()], dim=1)
    if s["bias"] is not None:
        z = z + s["bias"].double()
    T, k = case["T"], case["k"]
    left = z.clone()
    idx = torch.empty((T, k), dtype=torch.int64, device=DEV)
    for j in range(k):                 # argmax gives the first of equal ones
        idx[:, j] = (left == left.amax(1, keepdim=True)).int().argmax(1)
        left.scatter_(1, idx[:, j:j + 1], -math.inf)
    gates = torch.softmax(z, 1).gather(1, idx)
    if case["renorm"]:
        gates = gates / gates.sum(1, keepdim=True)
    y = torch.zeros_like(x)
    slots = torch.arange(case["E"]) if s["slot"] is None else s["slot"].cpu()
    slots = slots.to(DEV).long()

    def expert(rows, wg, wu, wd):
        a = rows @ wg.double().t()
        return (torch.sigmoid(a) * a * (rows @ wu.double().t())) @ wd.double().t()

    for e in idx.unique().tolist():
        if int(slots[e]) < 0:
            continue
        share = torch.where(idx == e, gates, torch.zeros_like(gates)).sum(1)
        t = share.nonzero()[:, 0]
        sl = int(slots[e])
        y[t] += share[t, None] * expert(x[t], s["w_gate"][sl], s["w_up"][sl], s["w_down"][sl])
    if s["shared"] is not None:
        y = y + expert(x, *s["shared"])
    return dict(y=y, idx=idx.int(), gates=gates, incomplete=(slots[idx] < 0).any(1).int())


def _exact_attn(case, seed):
    s = _prepare_attn(case, seed)
    pl, sl = _lengths(case)
    n_q = case["Hq"] // case["Hkv"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device=DEV)
    for h in range(case["Hkv"]):
        for g in range(case["G"]):
            kp = s["k_prefix"][g, :pl[g], h].double()
            vp = s["v_prefix"][g, :pl[g], h].double()
            for r in range(s["offs"][g], s["offs"][g + 1]):
                heads = slice(h * n_q, (h + 1) * n_q)
                k = torch.cat([kp, s["k_suffix"][r, :sl[r], h].double()])
                v = torch.cat([vp, s["v_suffix"][r, :sl[r], h].double()])
                z = s["scale"] * (s["q"][r, heads].double() @ k.t())
                lse[r, heads] = torch.logsumexp(z, 1)
                out[r, heads] = torch.softmax(z, 1) @ v
    return dict(out=out, lse=lse)


def _exact_select(case, seed):
    s = _prepare_select(case, seed)
    B, K, V, n = (case[x] for x in ("B", "K", "V", "n"))
    logp = torch.log_softmax(s["logits"].double(), -1) + s["scores"].double()[..., None]
    done = torch.zeros((B, K), dtype=torch.bool, device=DEV)
    if s["finished"] is not None:
        done = s["finished"].bool()
        logp[done] = -math.inf
        logp[..., s["eos"]] = torch.where(done, s["scores"].double(), logp[..., s["eos"]])
    flat = logp.view(B, K * V)
    pos, val = [], []
    for _ in range(n):
        top = flat.amax(1, keepdim=True)
        at = (flat == top).int().argmax(1, keepdim=True)
        pos.append(at)
        val.append(top)
        flat.scatter_(1, at, -math.inf)
    pos, val = torch.cat(pos, 1), torch.cat(val, 1)
    beam, token = pos // V, pos % V
    return dict(parent=(beam + K * torch.arange(B, device=DEV)[:, None]).int(), token=token.int(),
                score=val, finished=((token == s["eos"]) | done.gather(1, beam)).int())


def _exact_reorder(case, seed):
    s = _prepare_reorder(case, seed)
    src, lens = s["parent"].view(-1).tolist(), s["lens"].tolist()
    for cache in s["caches"]:          # parents keep their own rows
        for r, p in enumerate(src):
            cache[:, r, :lens[p]] = cache[:, p, :lens[p]]
    return dict(caches=s["caches"], lens=s["lens"][s["parent"].view(-1).long()], err=s["err"])


def exact(case, seed):
    return _EXACT[case["kind"]](case, seed)


_PREPARE = dict(layer=_prepare_layer, attn=_prepare_attn, select=_prepare_select,
                reorder=_prepare_reorder)
_PLAIN = dict(layer=_plain_layer, attn=_plain_attn, select=_plain_select, reorder=_plain_reorder)
_OWN = dict(layer=_own_layer, attn=_own_attn, select=_own_select, reorder=_own_reorder)
_WORK = dict(layer=_work_layer, attn=_work_attn, select=_work_select, reorder=_work_reorder)
_EXACT = dict(layer=_exact_layer, attn=_exact_attn, select=_exact_select, reorder=_exact_reorder)
