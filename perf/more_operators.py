"""The operators around a prompt, its cache in 4 bits and its log-probabilities,
measured: their inputs, a plain form of each, the work it cannot do without and a
64-bit reference.

A prompt's tokens (or a chunk of them, behind keys that are there already) attend
to themselves (prompt_attention); their keys and values go to a cache that holds
them in 4 bits and come back from it as values for the next chunk (kv4_store,
kv4_load); later tokens attend to that cache one by one (kv4_attention); logits
become the log-probabilities of given tokens, with the entropy and the best
alternatives (token_logprobs).

A case is a dict of plain values; its "kind" names the operator. Where `own` is
false a pass runs elementary torch operations in 32 bits (64 for the sums over a
vocabulary), where it is true the package's entry points. Sizes are generic.

Blocks of the cache: 32 channels of one token and head share a power of two 2^e,
the least with max |x| <= 7 * 2^e and e in -124..125; x is held as the nearest of
0, 0.5, 1, 1.5, 2, 3, 4, 6 times 2^e (ties to the even code), with its sign.
"""
import math

import torch

own = False

DEV = "cuda:0"
BLOCK = 32
GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _prompt(B, N, P, Hq, Hkv, D, dtype="bf16", ragged=False, name=None):
    """B sequences of N new tokens behind P keys that are there already (ragged: up
    to N and up to P)."""
    c = dict(kind="prompt", B=B, N=N, P=P, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, ragged=ragged)
    if name:
        c["name"] = name
    return c


def _cache(N, slots, Hkv, D, dtype="bf16", name=None):
    """N tokens go to N of the cache's slots, in any order, and come back."""
    c = dict(kind="cache", N=N, slots=slots, Hkv=Hkv, D=D, dtype=dtype)
    if name:
        c["name"] = name
    return c


def _attn4(R, S, Hq, Hkv, D, dtype="bf16", ragged=False, name=None):
    """R rows of one token over caches of up to S keys."""
    c = dict(kind="attn4", R=R, S=S, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, ragged=ragged)
    if name:
        c["name"] = name
    return c


def _logprobs(R, V, m, n, dtype="bf16", name=None):
    """m given tokens and the n best alternatives of each of R rows."""
    c = dict(kind="logprobs", R=R, V=V, m=m, n=n, dtype=dtype)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # a short float32 prompt: launches and nothing else
        _prompt(1, 100, 0, 8, 2, 64, dtype="f32", name="prompt_f32_n100"),
        # one prompt of some hundred tokens, an odd number of them
        _prompt(1, 777, 0, 32, 8, 128, name="prompt_n777"),
        # a prefill batch: sixteen packed prompts of different lengths
        _prompt(16, 1000, 0, 32, 8, 128, ragged=True, name="prompt_b16_n1000"),
        # one long prompt
        _prompt(1, 16384, 0, 32, 8, 128, name="prompt_n16384"),
        # a chunk of a prompt behind a long history
        _prompt(1, 500, 32000, 16, 4, 128, name="prompt_n500_p32000"),
        # a decode step's new keys and values: 64 sequences, one token each
        _cache(64, 64 * 500, 8, 128, name="cache_n64"),
        # a chunk of a long prompt: streaming
        _cache(16384, 20000, 8, 128, name="cache_n16384"),
        # one sequence, some hundred keys, float32
        _attn4(1, 777, 8, 2, 64, dtype="f32", name="attn4_f32_s777"),
        # one sequence with a very long history
        _attn4(1, 131072, 32, 8, 128, name="attn4_r1_s131072"),
        # a decode batch with histories of different lengths
        _attn4(64, 8192, 32, 8, 128, ragged=True, name="attn4_r64_s8192"),
        # one token, a vocabulary of 32000, float32 logits, five alternatives
        _logprobs(1, 32000, 1, 5, dtype="f32", name="logprobs_r1_v32000"),
        # a prompt's tokens scored over a large vocabulary
        _logprobs(2000, 128000, 1, 4, name="logprobs_r2000_v128000"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "chunk", "prompt_f32", "cache", "cache", "attn4",
                       "attn4", "attn4_f32", "logprobs", "logprobs"])
    if kind == "prompt":
        Hkv, q = rng.choice([(8, 4), (16, 1), (2, 8), (4, 7), (1, 16)])
        B = _log_int(rng, 1, 16)
        return _prompt(B, _log_int(rng, 1, 8192 // B), 0, Hkv * q, Hkv,
                       rng.choice([64, 80, 128, 128, 256]), ragged=rng.choice([True, False]))
    if kind == "chunk":
        Hkv, q = rng.choice([(8, 4), (4, 8), (8, 1)])
        B = _log_int(rng, 1, 8)
        return _prompt(B, _log_int(rng, 1, 1024 // B), _log_int(rng, 1, 32768 // B), Hkv * q, Hkv,
                       rng.choice([64, 128]), ragged=rng.choice([True, False]))
    if kind == "prompt_f32":
        Hkv, q = rng.choice([(2, 4), (4, 1), (3, 2)])
        return _prompt(rng.randint(1, 4), _log_int(rng, 1, 1024), rng.choice([0, 0, 100, 333]),
                       Hkv * q, Hkv, rng.choice([32, 64, 128]), dtype="f32",
                       ragged=rng.choice([True, False]))
    if kind == "cache":
        N = _log_int(rng, 1, 16384)
        return _cache(N, N + _log_int(rng, 1, 4096), rng.choice([1, 2, 5, 8]),
                      rng.choice([32, 64, 96, 128]), dtype=rng.choice(["bf16", "bf16", "f32"]))
    if kind == "attn4":
        Hkv, q = rng.choice([(8, 4), (16, 1), (2, 8), (4, 7), (1, 16)])
        R = _log_int(rng, 1, 64)
        return _attn4(R, _log_int(rng, 1, min(262144 // R, 65536)), Hkv * q, Hkv,
                      rng.choice([64, 96, 128, 128]), ragged=rng.choice([True, False]))
    if kind == "attn4_f32":
        Hkv, q = rng.choice([(2, 4), (4, 1), (3, 2)])
        return _attn4(_log_int(rng, 1, 16), _log_int(rng, 1, 4096), Hkv * q, Hkv,
                      rng.choice([32, 64, 128]), dtype="f32", ragged=rng.choice([True, False]))
    V = _log_int(rng, 100, 152000)
    return _logprobs(_log_int(rng, 1, max(1, min(2000, 200000000 // V))), V,
                     rng.choice([1, 1, 2, 8]), rng.choice([0, 1, 5, 16, 20]),
                     dtype=rng.choice(["bf16", "f32"]))


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


def _seqs(case):
    """New tokens and all keys of every sequence: the longest first, the others
    between a quarter of it and all (at least one)."""
    N, P = case["N"], case["P"]
    n = [N] * case["B"]
    p = [P] * case["B"]
    if case["ragged"]:
        n = [max(1, N - (b * 397) % (3 * N // 4 + 1)) for b in range(case["B"])]
        p = [P - (b * 1237) % (3 * P // 4 + 1) for b in range(case["B"])]
    return n, [a + b for a, b in zip(n, p)]


def _offsets(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


def _int32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _prepare_prompt(case, seed):
    """Scores with a standard deviation of about two; the first key of a sequence
    is one that every query favours, as trained heads have it."""
    g = _gen(seed)
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    dt = _type(case)
    nq, nk = _seqs(case)
    qo, ko = _offsets(nq), _offsets(nk)
    q = torch.empty((qo[-1], Hq, D), device=DEV).normal_(0.0, 2.0, generator=g)
    k = _normal(g, (ko[-1], Hkv, D), 1.0, dt)
    lean = torch.empty((case["B"], Hkv, D), device=DEV).normal_(0.0, 0.7, generator=g)
    for b in range(case["B"]):
        k[ko[b]] = (2.0 * lean[b]).to(dt)
        q[qo[b]:qo[b + 1]] += lean[b].repeat_interleave(Hq // Hkv, 0)
    s = dict(case=case, q=q.to(dt), k=k, v=_normal(g, (ko[-1], Hkv, D), 1.0, dt), scale=D ** -0.5,
             qo=qo, ko=ko, q_offsets=_int32(qo), k_offsets=_int32(ko))
    if own:
        from paper_2410_17954_amd import ops
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((qo[-1], Hq), dtype=torch.float32, device=DEV)
        s["ws"] = ops.workspace_tensor(
            ops.prompt_attention_workspace(qo[-1], ko[-1], case["B"], Hq, Hkv, D,
                                           ops.MOE_F32 if case["dtype"] == "f32" else ops.MOE_BF16),
            DEV)
    return s


def _prepare_cache(case, seed):
    """Keys with a few channels that are larger than the others, values without."""
    g = _gen(seed)
    N, Hkv, D, n = case["N"], case["Hkv"], case["D"], case["slots"]
    k = torch.empty((N, Hkv, D), device=DEV).normal_(0.0, 1.0, generator=g)
    k *= 1.0 + 6.0 * (torch.rand((Hkv, D), device=DEV, generator=g) < 0.05).float()
    order = torch.randperm(n, generator=g, device=DEV)[:N]
    s = dict(case=case, k=k.to(_type(case)), v=_normal(g, (N, Hkv, D), 0.5, _type(case)),
             slots=order.int())
    if own:
        s["cache"] = tuple(torch.zeros((1, n, Hkv, w), dtype=torch.uint8, device=DEV)
                           for w in (D // 2, D // BLOCK) * 2)
        s["k_back"], s["v_back"] = torch.empty_like(s["k"]), torch.empty_like(s["v"])
    return s


def _encode(x):
    """Codes, two a byte (the lower channel in the lower half), and scale bytes."""
    y = x.float().unflatten(-1, (-1, BLOCK))
    e = _exponent(y.abs().amax(-1, keepdim=True))
    code = torch.bucketize(y.abs() / _power(e), _borders(), out_int32=True)
    code = code.to(torch.uint8) + 8 * torch.signbit(y).to(torch.uint8)
    code = code.flatten(-2)
    return code[..., 0::2] + 16 * code[..., 1::2], (e[..., 0] + 127).to(torch.uint8)


def _exponent(amax):
    f, x = torch.frexp(amax)
    e = x - 3 + (f > 0.875).int()
    return torch.where(amax > 0, e, torch.full_like(e, -124)).clamp(-124, 125)


def _power(e):
    """2^e as float32, exactly."""
    return ((e + 127) << 23).view(torch.float32)


def _borders():
    """A value on a border belongs to the even code: above 0.25, from 0.75 on, ..."""
    up = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=DEV)
    odd = torch.tensor([False, True, False, True, False, True, False], device=DEV)
    return torch.where(odd, torch.nextafter(up, torch.zeros_like(up)), up)


def _decode(codes, scales):
    """The values that codes and scale bytes stand for, float32."""
    grid = torch.tensor(GRID + [-x for x in GRID], device=DEV)
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    y = grid[c.long()].unflatten(-1, (-1, BLOCK))
    return (y * _power(scales.int() - 127)[..., None]).flatten(-2)


def _rows4(case):
    """Keys of every row, and the cache row it reads (the last first)."""
    R, S = case["R"], case["S"]
    n = [S] * R
    if case["ragged"]:
        n = [max(1, S - (r * 397) % (S // 2 + 1)) for r in range(R)]
    return n, list(range(R))[::-1]


def _prepare_attn4(case, seed):
    g = _gen(seed)
    R, S, Hq, Hkv, D = (case[x] for x in ("R", "S", "Hq", "Hkv", "D"))
    q = torch.empty((R, Hq, D), device=DEV).normal_(0.0, 2.0, generator=g)
    lens, rows = _rows4(case)
    cache = tuple(torch.empty((R, S, Hkv, w), dtype=torch.uint8, device=DEV)
                  for w in (D // 2, D // BLOCK) * 2)
    lean = torch.empty((R, Hkv, D), device=DEV).normal_(0.0, 0.7, generator=g)
    step = max(1, 8192 // Hkv)
    for r in range(R):
        for lo in range(0, S, step):
            n = min(step, S - lo)
            x = torch.empty((2, n, Hkv, D), device=DEV).normal_(0.0, 1.0, generator=g)
            if lo == 0:
                x[0, 0] = 2.0 * lean[rows[r]]
            for j in range(2):
                cache[2 * j][r, lo:lo + n], cache[2 * j + 1][r, lo:lo + n] = _encode(x[j])
    q += lean.repeat_interleave(Hq // Hkv, 1)
    s = dict(case=case, q=q.to(_type(case)), cache=cache, scale=D ** -0.5, n=lens, rows=rows,
             lens=_int32(lens), cache_row=_int32(rows))
    if own:
        from paper_2410_17954_amd import ops
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((R, Hq), dtype=torch.float32, device=DEV)
        s["ws"] = ops.workspace_tensor(ops.kv4_attention_workspace(R, S, Hq, Hkv, D), DEV)
    return s


def _prepare_logprobs(case, seed):
    """Logits N(0, 2.5) with a few clear favourites a row; of the given tokens the
    first is a favourite, as a model's own text is, the others are any."""
    g = _gen(seed)
    R, V, m = case["R"], case["V"], case["m"]
    z = torch.empty((R, V), device=DEV).normal_(0.0, 2.5, generator=g)
    top = torch.randint(0, V, (R, 3), device=DEV, generator=g)
    z.scatter_add_(1, top, torch.rand((R, 3), device=DEV, generator=g) * 6.0 + 6.0)
    tokens = torch.randint(0, V, (R, m), device=DEV, generator=g)
    tokens[:, 0] = top[:, 0]
    s = dict(case=case, logits=z.to(_type(case)), tokens=tokens.int())
    if own:
        from paper_2410_17954_amd import ops
        n = case["n"]
        s["logp"] = torch.empty((R, m), dtype=torch.float32, device=DEV)
        s["entropy"] = torch.empty(R, dtype=torch.float32, device=DEV)
        s["top"] = torch.empty((R, n), dtype=torch.int32, device=DEV) if n else None
        s["top_logp"] = torch.empty((R, n), dtype=torch.float32, device=DEV) if n else None
        s["ws"] = ops.workspace_tensor(ops.token_logprobs_workspace(R, V, m, n), DEV)
    return s


def prepare(case, seed):
    return _PREPARE[case["kind"]](case, seed)


# ------------------------------------------------------------ plain forms
def _plain_prompt(s):
    c = s["case"]
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    n_q = Hq // Hkv
    out = torch.empty(s["q"].shape, device=DEV)
    lse = torch.empty(s["q"].shape[:2], device=DEV)
    for b in range(c["B"]):
        q0, q1, k0, k1 = s["qo"][b], s["qo"][b + 1], s["ko"][b], s["ko"][b + 1]
        past = (k1 - k0) - (q1 - q0)
        k = s["k"][k0:k1].float().permute(1, 2, 0).contiguous()
        v = s["v"][k0:k1].float().permute(1, 0, 2).contiguous()
        for lo in range(q0, q1, 1024):                   # scores of 1024 tokens at a time
            n = min(1024, q1 - lo)
            last = past + lo - q0 + torch.arange(n, device=DEV)
            keys = past + lo - q0 + n                    # none beyond the last one's
            hide = torch.arange(keys, device=DEV) > last[:, None]
            q = (s["q"][lo:lo + n].float() * s["scale"]).view(n, Hkv, n_q, D)
            q = q.permute(1, 2, 0, 3).reshape(Hkv, n_q * n, D)
            z = (q @ k[:, :, :keys].contiguous()).view(Hkv, n_q, n, keys).masked_fill(hide, -math.inf)
            m = z.amax(-1, keepdim=True)
            p = torch.exp(z - m)
            del z
            den = p.sum(-1, keepdim=True)
            o = (p.view(Hkv, n_q * n, keys) @ v[:, :keys]).view(Hkv, n_q, n, D) / den
            out[lo:lo + n] = o.permute(2, 0, 1, 3).reshape(n, Hq, D)
            lse[lo:lo + n] = (m + torch.log(den))[..., 0].permute(2, 0, 1).reshape(n, Hq)
    return dict(out=out.to(s["q"].dtype), lse=lse)


def _plain_cache(s):
    out = {}
    for name in ("k", "v"):
        x = s[name].float().unflatten(-1, (-1, BLOCK))
        unit = _power(_exponent(x.abs().amax(-1, keepdim=True)))
        y = x.abs() / unit
        step = torch.where(y < 2.0, 0.5, torch.where(y < 4.0, 1.0, 2.0))
        y = (torch.round(y / step) * step).clamp(max=6.0) * unit
        out[name] = torch.where(x < 0, -y, y).flatten(-2).to(s[name].dtype)
    return out


def _plain_attn4(s):
    c = s["case"]
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    out, lse = [], []
    for r in range(c["R"]):
        at, n = s["rows"][r], s["n"][r]
        k, v = (_decode(s["cache"][2 * j][at, :n], s["cache"][2 * j + 1][at, :n]) for j in range(2))
        q = s["q"][r].float().view(Hkv, Hq // Hkv, D) * s["scale"]
        z = q @ k.permute(1, 2, 0).contiguous()
        m = z.amax(-1, keepdim=True)
        p = torch.exp(z - m)
        den = p.sum(-1, keepdim=True)
        out.append(((p @ v.permute(1, 0, 2).contiguous()) / den).view(Hq, D))
        lse.append((m + torch.log(den)).view(Hq))
    return dict(out=torch.stack(out).to(s["q"].dtype), lse=torch.stack(lse))


def _plain_logprobs(s):
    c = s["case"]
    out = dict(logp=[], entropy=[], top=[], top_logp=[])
    for lo in range(0, c["R"], 256):                     # 256 rows at a time
        z = s["logits"][lo:lo + 256].double()
        d = z - z.amax(1, keepdim=True)
        e = torch.exp(d)
        total = e.sum(1, keepdim=True)
        logz = torch.log(total)
        tokens = s["tokens"][lo:lo + 256].long()
        out["logp"].append((d.gather(1, tokens) - logz).float())
        out["entropy"].append((logz - (e * d).sum(1, keepdim=True) / total)[:, 0].float())
        if c["n"]:
            best = z.sort(dim=1, descending=True, stable=True).indices[:, :c["n"]]
            out["top"].append(best.int())
            out["top_logp"].append((d.gather(1, best) - logz).float())
    return {k: torch.cat(v) for k, v in out.items() if v}


# ----------------------------------------------------------- entry points
def _own_prompt(s):
    from paper_2410_17954_amd import ops
    out, lse = ops.prompt_attention(s["q"], s["k"], s["v"], q_offsets=s["q_offsets"],
                                    k_offsets=s["k_offsets"], scale=s["scale"], out=s["out"],
                                    lse=s["lse"], workspace=s["ws"])
    return dict(out=out, lse=lse)


def _own_cache(s):
    from paper_2410_17954_amd import ops
    ops.kv4_store(s["k"], s["v"], s["cache"], slots=s["slots"])
    k, v = ops.kv4_load(s["cache"], slots=s["slots"], k=s["k_back"], v=s["v_back"])
    return dict(k=k, v=v)


def _own_attn4(s):
    from paper_2410_17954_amd import ops
    out, lse = ops.kv4_attention(s["q"], s["cache"], lens=s["lens"], cache_row=s["cache_row"],
                                 scale=s["scale"], out=s["out"], lse=s["lse"], workspace=s["ws"])
    return dict(out=out, lse=lse)


def _own_logprobs(s):
    from paper_2410_17954_amd import ops
    logp, entropy, top, top_logp = ops.token_logprobs(
        s["logits"], s["tokens"], n_top=s["case"]["n"], logprobs=s["logp"], entropy=s["entropy"],
        top_tokens=s["top"], top_logprobs=s["top_logp"], workspace=s["ws"])
    out = dict(logp=logp, entropy=entropy)
    if s["case"]["n"]:
        out.update(top=top, top_logp=top_logp)
    return out


def run(state):
    kind = state["case"]["kind"]
    return (_OWN if own else _PLAIN)[kind](state)


# ------------------------------------------------------------------ work
def _elt(case):
    return 4 if case["dtype"] == "f32" else 2


def _work_prompt(c):
    nq, nk = _seqs(c)
    pairs = sum(n * (k - n) + n * (n + 1) // 2 for n, k in zip(nq, nk))
    nbytes = _elt(c) * c["D"] * (2 * c["Hq"] * sum(nq) + 2 * c["Hkv"] * sum(nk)) \
        + 4 * c["Hq"] * sum(nq)
    return {"bytes": nbytes, "flops": 4.0 * c["D"] * c["Hq"] * pairs}


def _work_cache(c):
    """Read, written as codes, those read again, written as values."""
    n = 2 * c["N"] * c["Hkv"] * c["D"]
    return {"bytes": 2 * n * _elt(c) + 2 * n * 17 / 32 + 4 * c["N"], "flops": 4.0 * n}


def _work_attn4(c):
    keys = sum(_rows4(c)[0])
    nbytes = keys * 2 * c["Hkv"] * c["D"] * 17 / 32 \
        + c["R"] * c["Hq"] * (2 * c["D"] * _elt(c) + 4)
    return {"bytes": nbytes, "flops": 4.0 * c["D"] * c["Hq"] * keys}


def _work_logprobs(c):
    return {"bytes": c["R"] * (c["V"] * _elt(c) + 8 * c["m"] + 8 * c["n"] + 4),
            "flops": 6.0 * c["R"] * c["V"]}


def work(case):
    return _WORK[case["kind"]](case)


# ------------------------------------------------------ 64-bit reference
def _exact_prompt(case, seed):
    s = _prepare_prompt(case, seed)
    n_q = case["Hq"] // case["Hkv"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device=DEV)
    for b in range(case["B"]):
        q0, q1, k0, k1 = s["qo"][b], s["qo"][b + 1], s["ko"][b], s["ko"][b + 1]
        first = (k1 - k0) - (q1 - q0)                    # the first query's last key
        for h in range(case["Hq"]):
            k, v = s["k"][k0:k1, h // n_q].double(), s["v"][k0:k1, h // n_q].double()
            for lo in range(q0, q1, 4096):
                hi = min(lo + 4096, q1)
                z = s["scale"] * (s["q"][lo:hi, h].double() @ k.t())
                see = torch.ones_like(z, dtype=torch.bool).tril(first + lo - q0)
                z = torch.where(see, z, torch.full_like(z, -math.inf))
                lse[lo:hi, h] = torch.logsumexp(z, 1)
                out[lo:hi, h] = torch.softmax(z, 1) @ v
    return dict(out=out, lse=lse)


def _exact_cache(case, seed):
    """The nearest of the values that a block can hold, by distance."""
    s = _prepare_cache(case, seed)
    grid = torch.tensor(GRID, dtype=torch.float64, device=DEV)
    out = {}
    for name in ("k", "v"):
        x = s[name].double().unflatten(-1, (-1, BLOCK))
        top = x.abs().amax(-1, keepdim=True)
        unit = torch.full_like(top, 2.0 ** -124)
        for p in range(-123, 126):
            unit = torch.where(top > 7.0 * 2.0 ** (p - 1), 2.0 ** p, unit)
        y = x.abs() / unit
        best, dist = torch.zeros_like(y), y.clone()
        for i in range(1, 8):
            d = (y - grid[i]).abs()
            nearer = (d < dist) | ((d == dist) & (i % 2 == 0))
            best, dist = torch.where(nearer, grid[i], best), torch.where(nearer, d, dist)
        out[name] = (torch.sign(x) * best * unit).flatten(-2)
    return out


def _exact_attn4(case, seed):
    s = _prepare_attn4(case, seed)
    R, Hq, Hkv, D = (case[x] for x in ("R", "Hq", "Hkv", "D"))
    grid = torch.tensor(GRID + [-x for x in GRID], dtype=torch.float64, device=DEV)
    out = torch.empty((R, Hq, D), dtype=torch.float64, device=DEV)
    lse = torch.empty((R, Hq), dtype=torch.float64, device=DEV)

    def values(codes, scales):
        y = torch.empty(codes.shape[:-1] + (D,), dtype=torch.float64, device=DEV)
        y[..., 0::2], y[..., 1::2] = grid[(codes % 16).long()], grid[(codes // 16).long()]
        unit = torch.tensor([2.0 ** (i - 127) for i in range(255)], dtype=torch.float64, device=DEV)
        return y * unit[scales.long()].repeat_interleave(BLOCK, -1)

    for r in range(R):
        at, n = s["rows"][r], s["n"][r]
        for h in range(Hkv):
            heads = slice(h * (Hq // Hkv), (h + 1) * (Hq // Hkv))
            kc, ksc, vc, vsc = (t[at, :n, h] for t in s["cache"])
            z = s["scale"] * (s["q"][r, heads].double() @ values(kc, ksc).t())
            lse[r, heads] = torch.logsumexp(z, 1)
            out[r, heads] = torch.softmax(z, 1) @ values(vc, vsc)
    return dict(out=out, lse=lse)


def _exact_logprobs(case, seed):
    s = _prepare_logprobs(case, seed)
    R, n = case["R"], case["n"]
    out = dict(logp=[], entropy=[], top=[], top_logp=[])
    for lo in range(0, R, 200):
        logp = torch.log_softmax(s["logits"][lo:lo + 200].double(), 1)
        out["logp"].append(logp.gather(1, s["tokens"][lo:lo + 200].long()))
        out["entropy"].append(-(torch.exp(logp) * logp).sum(1))
        left = s["logits"][lo:lo + 200].double()
        for j in range(n):                               # argmax of the flags: the first one
            at = (left == left.amax(1, keepdim=True)).int().argmax(1, keepdim=True)
            out["top"].append((lo, j, at))
            out["top_logp"].append((lo, j, logp.gather(1, at)))
            left.scatter_(1, at, -math.inf)
    res = dict(logp=torch.cat(out["logp"]), entropy=torch.cat(out["entropy"]))
    if n:
        res["top"] = torch.empty((R, n), dtype=torch.int32, device=DEV)
        res["top_logp"] = torch.empty((R, n), dtype=torch.float64, device=DEV)
        for name in ("top", "top_logp"):
            for lo, j, x in out[name]:
                res[name][lo:lo + 200, j:j + 1] = x.to(res[name].dtype)
    return res


def exact(case, seed):
    return _EXACT[case["kind"]](case, seed)


_PREPARE = dict(prompt=_prepare_prompt, cache=_prepare_cache, attn4=_prepare_attn4,
                logprobs=_prepare_logprobs)
_PLAIN = dict(prompt=_plain_prompt, cache=_plain_cache, attn4=_plain_attn4,
              logprobs=_plain_logprobs)
_OWN = dict(prompt=_own_prompt, cache=_own_cache, attn4=_own_attn4, logprobs=_own_logprobs)
_WORK = dict(prompt=_work_prompt, cache=_work_cache, attn4=_work_attn4, logprobs=_work_logprobs)
_EXACT = dict(prompt=_exact_prompt, cache=_exact_cache, attn4=_exact_attn4,
              logprobs=_exact_logprobs)
