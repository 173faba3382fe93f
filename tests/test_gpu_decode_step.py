"""The decode-step operators together: beams of several requests through
attention layers with a shared prompt, MoE layers, selection and reordering; and
the calls under what a serving loop does with them (captured graphs, other
streams, two calls at once)."""
import numpy as np
import pytest
import torch

import oracle
from paper_2410_17954_amd import ops
from gpu_helpers import to_host

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _rms(h):
    return h / torch.sqrt((h * h).mean(-1, keepdim=True) + 1e-6)


class Model:
    """Two pre-normalised blocks (attention, MoE) and a head, float32."""

    def __init__(self, seed, L=2, H=64, Hq=4, Hkv=2, D=16, E=6, k=2, F=32, Fs=16, V=53):
        g = torch.Generator(device=DEV).manual_seed(seed)
        n = lambda *s, std=0.15: torch.randn(s, device=DEV, generator=g) * std
        self.L, self.H, self.Hq, self.Hkv, self.D, self.E, self.k, self.V = L, H, Hq, Hkv, D, E, k, V
        self.emb, self.head = n(V, H, std=1.0), n(V, H, std=0.4)
        self.layers = [dict(q=n(Hq * D, H), k=n(Hkv * D, H), v=n(Hkv * D, H), o=n(H, Hq * D),
                            router=n(E, H), wg=n(E, F, H), wu=n(E, F, H), wd=n(E, H, F),
                            sh=(n(Fs, H), n(Fs, H), n(H, Fs))) for _ in range(L)]

    def prompt(self, ids):
        """Keys and values [L, n, Hkv, D] of a prompt, token by token (no attention
        between prompt tokens is needed for what is tested: they are the cache)."""
        h = self.emb[ids]
        x = _rms(h)
        ks = [(x @ w["k"].T).view(-1, self.Hkv, self.D) for w in self.layers]
        vs = [(x @ w["v"].T).view(-1, self.Hkv, self.D) for w in self.layers]
        return torch.stack(ks), torch.stack(vs)

    def reference(self, kp, vp, ids):
        """Float64 scores of the continuations of one sequence [n] behind a prompt:
        log-probabilities [V] after the last token, nothing cached."""
        d = torch.float64
        ks = [[] for _ in range(self.L)]
        vs = [[] for _ in range(self.L)]
        for t in ids:
            h = self.emb[t].to(d)[None]
            for l, w in enumerate(self.layers):
                x = _rms(h)
                q = (x @ w["q"].to(d).T).view(1, self.Hq, self.D)
                ks[l].append((x @ w["k"].to(d).T).view(self.Hkv, self.D))
                vs[l].append((x @ w["v"].to(d).T).view(self.Hkv, self.D))
                K = torch.cat([kp[l].to(d), torch.stack(ks[l])])
                Vv = torch.cat([vp[l].to(d), torch.stack(vs[l])])
                rep = self.Hq // self.Hkv
                s = torch.stack([K[:, i // rep] @ q[0, i] for i in range(self.Hq)]) * self.D ** -0.5
                p = torch.softmax(s, -1)
                a = torch.stack([p[i] @ Vv[:, i // rep] for i in range(self.Hq)]).reshape(1, -1)
                h = h + a @ w["o"].to(d).T
                x = _rms(h)
                out = oracle.moe_layer(x.cpu().numpy(), w["router"].double().cpu().numpy(), self.k,
                                       *(w[n].double().cpu().numpy() for n in ("wg", "wu", "wd")),
                                       shared=tuple(m.double().cpu().numpy() for m in w["sh"]))
                h = h + torch.from_numpy(out["y"]).to(h)
        return torch.log_softmax(_rms(h)[0] @ self.head.to(d).T, -1)


def _step(m, ids, kp, vp, plen, ks, vs, slen):
    """One decode step of every row: logits [R, V]. ks, vs [L, R, S, Hkv, D] are
    written at position slen - 1."""
    h = m.emb[ids]
    R = h.shape[0]
    at = (slen - 1).long()
    rows = torch.arange(R, device=DEV)
    for l, w in enumerate(m.layers):
        x = _rms(h)
        ks[l, rows, at] = (x @ w["k"].T).view(R, m.Hkv, m.D)
        vs[l, rows, at] = (x @ w["v"].T).view(R, m.Hkv, m.D)
        q = (x @ w["q"].T).view(R, m.Hq, m.D)
        a, _ = ops.prefix_attention(q, kp[l], vp[l], ks[l], vs[l], prefix_len=plen, suffix_len=slen)
        h = h + a.view(R, -1) @ w["o"].T
        x = _rms(h)
        h, _, _, _ = ops.layer_decode(x, w["router"], w["wg"], w["wu"], w["wd"], m.k,
                                      shared=w["sh"], y=h.contiguous(), accumulate=True)
    return _rms(h) @ m.head.T


def test_beam_search_finds_what_the_definition_finds():
    """B requests of K beams, several steps: the beams kept by the cached step
    (shared prompts, suffix caches reordered in place) are those of a search that
    recomputes every sequence in float64."""
    B, K, S, steps, eos = 3, 4, 6, 5, 1
    m = Model(7)
    lens = [9, 4, 1]
    P = max(lens)
    kp = torch.full((m.L, B, P, m.Hkv, m.D), float("nan"), device=DEV)
    vp = torch.full_like(kp, float("nan"))
    g = torch.Generator(device=DEV).manual_seed(3)
    for b, n in enumerate(lens):
        ids = torch.randint(2, m.V, (n,), device=DEV, generator=g)
        kp[:, b, :n], vp[:, b, :n] = m.prompt(ids)
    plen = torch.tensor(lens, dtype=torch.int32, device=DEV)
    R = B * K
    ks = torch.full((m.L, R, S, m.Hkv, m.D), float("nan"), device=DEV)
    vs = torch.full_like(ks, float("nan"))
    slen = torch.ones(R, dtype=torch.int32, device=DEV)
    ids = torch.full((R,), 2, dtype=torch.int64, device=DEV)        # the start token
    scores = torch.full((B, K), -float("inf"), device=DEV)
    scores[:, 0] = 0.0
    done = torch.zeros((B, K), dtype=torch.int32, device=DEV)
    # the search by definition: lists of (score, tokens, finished) per request
    beams = [[(0.0, (2,), False)] for _ in range(B)]
    memo, compared = {}, 0
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    for step in range(steps):
        logits = _step(m, ids, kp, vp, plen, ks, vs, slen)
        parent, token, scores, done = ops.beam_select(
            logits.view(B, K, m.V), scores, K, finished=done, eos=eos)
        slen, _ = ops.beam_reorder([ks, vs], parent, lens=slen, err=err)
        slen = slen + 1
        ids = token.reshape(-1).long().clamp(min=0)
        for b in range(B):
            cand = []
            for sc, toks, fin in beams[b]:
                if fin:
                    cand.append((sc, toks + (eos,), True))
                    continue
                if (b, toks) not in memo:
                    n = lens[b]
                    memo[b, toks] = m.reference(kp[:, b, :n], vp[:, b, :n], toks).cpu().numpy()
                lp = memo[b, toks]
                cand += [(sc + lp[v], toks + (v,), v == eos) for v in np.argsort(-lp)[:K]]
            beams[b] = sorted(cand, key=lambda c: -c[0])[:K]
            got = to_host(scores)[b]
            want = np.array([c[0] for c in beams[b]])
            # float32 states: a product of at most 64 terms errs by 64 x 2^-24 = 4e-6
            # of its terms, some ten in a row through two blocks 4e-5, on logits of
            # up to ten 4e-4 a step; scores sum the steps
            assert np.abs(got - want).max() < 1e-3 * (step + 1)
            gaps = np.abs(np.diff(want))
            if gaps.size == 0 or gaps.min() > 4e-3 * (step + 1):
                assert to_host(token)[b].tolist() == [c[1][-1] for c in beams[b]]
                assert to_host(done)[b].tolist() == [int(c[2]) for c in beams[b]]
                compared += 1
    assert int(err) == 0
    assert compared >= B            # ties within the error are rare: most steps count


def _state(seed, T=6, H=128, F=64, E=8):
    g = torch.Generator(device=DEV).manual_seed(seed)
    n = lambda *s: torch.randn(s, device=DEV, generator=g).bfloat16()
    B, K, V, P, S = 2, 3, 700, 50, 8
    s = dict(x=n(T, H), wr=n(E, H), wg=n(E, F, H), wu=n(E, F, H), wd=n(E, H, F), q=n(T, 4, 64),
             kp=n(B, P, 2, 64), vp=n(B, P, 2, 64), ks=n(T, S, 2, 64), vs=n(T, S, 2, 64),
             logits=n(B, K, V), scores=torch.randn((B, K), device=DEV, generator=g),
             parent=torch.tensor([[0, 0, 2], [4, 3, 3]], dtype=torch.int32, device=DEV),
             cache=torch.randn((3, B * K, S, 5), device=DEV, generator=g))
    s["ws"] = [ops.workspace_tensor(ops.layer_decode_workspace(T, H, F, E, 2), DEV),
               ops.workspace_tensor(ops.prefix_attention_workspace(T, B, 4, 2, 64, P, S), DEV),
               ops.workspace_tensor(ops.beam_select_workspace(B, K, V, 4), DEV)]
    s["out"] = dict(y=torch.empty_like(s["x"]), att=torch.empty_like(s["q"]),
                    lse=torch.empty((T, 4), device=DEV),
                    idx=torch.empty((T, 2), dtype=torch.int32, device=DEV),
                    w=torch.empty((T, 2), device=DEV), inc=torch.empty(T, dtype=torch.int32, device=DEV),
                    parent=torch.empty((B, 4), dtype=torch.int32, device=DEV),
                    token=torch.empty((B, 4), dtype=torch.int32, device=DEV),
                    best=torch.empty((B, 4), device=DEV), moved=s["cache"].clone(),
                    lens=torch.empty(B * K, dtype=torch.int32, device=DEV),
                    err=torch.zeros(1, dtype=torch.int32, device=DEV))
    return s


def _calls(s, stream=None):
    o = s["out"]
    ops.layer_decode(s["x"], s["wr"], s["wg"], s["wu"], s["wd"], 2, y=o["y"], topk_idx=o["idx"],
                     topk_w=o["w"], incomplete=o["inc"], workspace=s["ws"][0], stream=stream)
    ops.prefix_attention(s["q"], s["kp"], s["vp"], s["ks"], s["vs"], out=o["att"], lse=o["lse"],
                         workspace=s["ws"][1], stream=stream)
    ops.beam_select(s["logits"], s["scores"], 4, parent=o["parent"], token=o["token"],
                    out_scores=o["best"], workspace=s["ws"][2], stream=stream)
    ops.beam_reorder([o["moved"]], s["parent"], new_lens=o["lens"], err=o["err"], stream=stream)


def _copy(o):
    return {n: t.clone() for n, t in o.items()}


def test_captured_and_replayed():
    """All four in one graph, replayed on changing inputs with eager work between."""
    s = _state(1)
    _calls(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _calls(s)
    for i in range(4):
        fresh = _state(10 + i)
        for n in ("x", "q", "kp", "logits", "scores", "ks"):
            s[n].copy_(fresh[n])
        s["out"]["moved"].copy_(fresh["cache"])
        for n, t in s["out"].items():
            if n not in ("moved", "err"):
                t.fill_(77)
        for w in s["ws"]:
            w.fill_(i * 85 % 256)
        graph.replay()
        torch.cuda.synchronize()
        got = _copy(s["out"])
        s["out"]["moved"].copy_(fresh["cache"])
        _calls(s)
        torch.cuda.synchronize()
        for n, t in s["out"].items():
            assert torch.equal(got[n], t), n
        torch.randn(1000, device=DEV).sum().item()


def test_two_graphs_of_their_own_workspaces_and_streams_at_once():
    a, b = _state(1), _state(2)
    want = []
    for s in (a, b):
        _calls(s)
        torch.cuda.synchronize()
        want.append(_copy(s["out"]))
    graphs = []
    for s in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            _calls(s)
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for s in (a, b):
            s["out"]["moved"].copy_(s["cache"])
            s["out"]["y"].zero_()
            s["out"]["att"].zero_()
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for s, w in zip((a, b), want):
            for n, t in s["out"].items():
                assert torch.equal(w[n], t), n


def test_given_stream_is_the_one_that_is_used():
    """Calls on a side stream, given and current, behind a long kernel there that
    writes their input."""
    s = _state(4)
    _calls(s)
    torch.cuda.synchronize()
    want = _copy(s["out"])
    src = {n: s[n].clone() for n in ("x", "q", "logits")}
    side = torch.cuda.Stream()
    big = torch.randn((4096, 4096), device=DEV)
    for given in (True, False):
        for n in src:
            s[n].zero_()
        s["out"]["moved"].copy_(s["cache"])
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(20):
                big = big @ big * 1e-4
            for n, t in src.items():
                s[n].copy_(t)
            if not given:
                _calls(s)
        if given:
            _calls(s, stream=side)
        torch.cuda.synchronize()
        for n, t in s["out"].items():
            assert torch.equal(want[n], t), n


def test_what_a_call_allocates_belongs_to_its_stream():
    """Outputs, fills and workspaces of a call on a given stream, while the current
    stream is far behind and reuses memory at once."""
    s = _state(5)
    off = torch.tensor([0, 3, 5], dtype=torch.int32, device=DEV)      # row 5 is in no group
    shape = (s["q"], s["kp"], s["vp"], s["ks"], s["vs"])

    def calls(stream):
        a, lse = ops.prefix_attention(*shape, group_offsets=off, stream=stream)
        y, idx, w, inc = ops.layer_decode(s["x"], s["wr"], s["wg"], s["wu"], s["wd"], 2, stream=stream)
        p, t, sc, _ = ops.beam_select(s["logits"], s["scores"], 4, stream=stream)
        n, err = ops.beam_reorder([s["out"]["moved"]], s["parent"], stream=stream)
        return [a, lse, y, idx, w, inc, p, t, sc, n, err]

    want = [t.clone() for t in calls(None)]
    assert want[1][5].isinf().all() and int(want[10]) == 0
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    big = torch.randn((4096, 4096), device=DEV)
    for _ in range(3):
        for _ in range(20):
            big = big @ big * 1e-4
        got = calls(side)
        junk = [torch.full((n,), 255, dtype=torch.uint8, device=DEV) for n in (1 << 10, 1 << 14, 1 << 18)]
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert torch.equal(g, w)
        del junk


def test_long_offsets_in_a_cache():
    """Keys that lie beyond 2^32 bytes, of rows whose caches are that far apart."""
    R, S, D = 3, 1 << 22, 128                                   # 1 GiB a row and cache
    k = torch.zeros((R, S, 1, D), dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    q = torch.zeros((R, 4, D), dtype=torch.bfloat16, device=DEV)
    q[:, :, 0] = 1.0
    at = [S - 1, S - 70, 5]
    for r in range(R):
        k[r, at[r], 0, 0] = 60.0
        v[r, at[r], 0, :] = r + 1.0
    k[2, S // 2:, 0, 1] = float("nan")                          # behind the row's length
    lens = torch.tensor([S, S, S // 2], dtype=torch.int32, device=DEV)
    out, lse = ops.prefix_attention(q, None, None, k, v, suffix_len=lens, scale=1.0)
    # exp(60) against 2^22 of exp(0): weight 1 - 4e-20
    for r in range(R):
        assert torch.equal(out[r].float(), torch.full((4, D), r + 1.0, device=DEV))
        assert (lse[r] - 60.0).abs().max() < 60 * 2 ** -22
    last = k[0, S - 1].clone()
    moved = torch.tensor([[0, 0, 1]], dtype=torch.int32, device=DEV)
    n, err = ops.beam_reorder([k[None], v[None]], moved)
    assert int(err) == 0 and n.tolist() == [S, S, S]
    assert torch.equal(k[1, S - 1], last) and float(k[2, S - 70, 0, 0]) == 60.0
    assert float(v[1, S - 1, 0, 5]) == 1.0 and float(v[2, S - 70, 0, 5]) == 2.0


@pytest.mark.parametrize("K,V,n", [(1, 1 << 25, 64), (32, 1 << 20, 64)])
def test_select_at_its_limit(K, V, n):
    g = torch.Generator(device=DEV).manual_seed(K)
    z = torch.randn((1, K, V), device=DEV, generator=g).bfloat16()
    s = torch.randn((1, K), device=DEV, generator=g)
    parent, token, score, _ = ops.beam_select(z, s, n)
    c = z.double()
    c += (s.double() - torch.logsumexp(c, -1))[..., None]
    c = c.view(-1)
    # bfloat16 logits tie: in the order of value, then beam and token
    least = torch.topk(c, n).values[-1]
    at = torch.nonzero(c >= least).view(-1)
    order = torch.sort(c[at], descending=True, stable=True).indices[:n]
    at = at[order]
    assert torch.equal(parent[0].long(), at // V) and torch.equal(token[0].long(), at % V)
    # log V + 18 steps of float32 for the sum, one for the result
    assert ((score[0] - c[at]).abs() <= 2.0 ** -24 * c[at].abs() + 40 * 2.0 ** -23).all()


@pytest.mark.parametrize("L,B,K", [(1, 9001, 2), (4100, 1, 3)])
def test_reorder_more_requests_and_layers_than_a_grid_has(L, B, K):
    g = torch.Generator(device=DEV).manual_seed(B)
    caches = [torch.randint(0, 1 << 30, (L, B * K, 2, 3), device=DEV, dtype=torch.int32, generator=g)
              for _ in range(2)]
    parent = torch.randint(0, K, (B, K), device=DEV, dtype=torch.int32, generator=g)
    parent += K * torch.arange(B, device=DEV, dtype=torch.int32)[:, None]
    want = [c[:, parent.view(-1).long()] for c in caches]
    _, err = ops.beam_reorder(caches, parent)
    assert int(err) == 0
    for c, w in zip(caches, want):
        assert torch.equal(c, w)


def test_attention_of_many_rows():
    # groups of one row: more blocks than a grid dimension of 65535 would take
    R, P, D = 70001, 3, 8
    g = torch.Generator(device=DEV).manual_seed(2)
    q, k, v = (torch.randn(s, device=DEV, generator=g) for s in ((R, 2, D), (R, P, 1, D), (R, P, 1, D)))
    out, lse = ops.prefix_attention(q, k, v, scale=1.0)
    s = (q.double()[:, :, None] * k.double().transpose(1, 2)).sum(-1)     # [R, 2, P]
    want = (torch.softmax(s, -1)[..., None] * v.double().transpose(1, 2)).sum(2)
    # scores err by 8 terms x 2^-24 of up to 40, which weigh as such in the result
    assert (out - want).abs().max() < 40 * 8 * 2.0 ** -24 * 2 * 5
    assert (lse - torch.logsumexp(s, -1)).abs().max() < 40 * 8 * 2.0 ** -24 * 2


def test_select_in_place():
    g = torch.Generator(device=DEV).manual_seed(8)
    B, K, V = 50, 4, 3001
    z = torch.randn((B, K, V), device=DEV, generator=g)
    s = torch.randn((B, K), device=DEV, generator=g)
    f = (torch.rand((B, K), device=DEV, generator=g) < 0.3).int()
    want = ops.beam_select(z, s, finished=f, eos=5)
    got = ops.beam_select(z, s, finished=f, eos=5, out_scores=s, out_finished=f)
    assert got[2] is s and got[3] is f
    for a, b in zip(got, want):
        assert torch.equal(a, b)
