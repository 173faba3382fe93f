"""The prompt operators together, as a serving loop calls them: chunks of packed
prompts attend, their keys and values go to a cache of 4 bits, later chunks and
single tokens attend to what it holds, logits become log-probabilities; and the
calls in captured graphs, on other streams, side by side."""
import numpy as np
import pytest
import torch

import oracle
from paper_2410_17954_amd import ops
from gpu_helpers import to_dev, to_host, vals
from prompt_helpers import check_row, draw, values

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompts_in_chunks_then_single_tokens(dtype):
    """Two sequences of 90 and 41 tokens: 60 and 41 of them at once, the 30 left
    behind what the cache holds, then three single tokens each. Every step against
    the oracle over the values that the cache stands for."""
    g = np.random.default_rng(1)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    Hq, Hkv, D, S, V = 8, 2, 64, 128, 300
    cache = ops.kv4_cache(3, S, Hkv, D, DEV)
    row_of, have = [2, 0], [0, 0]                    # cache rows, tokens there
    seen = [[np.zeros((0, Hkv, D))] * 2, [np.zeros((0, Hkv, D))] * 2]
    head = draw(g, "f32", V, Hq * D, std=0.05)

    def new(n):
        return draw(g, dtype, n, Hq, D, std=2.0), draw(g, dtype, n, Hkv, D), draw(g, dtype, n, Hkv, D)

    def logprobs_of(out):
        z = (out.float().reshape(len(out), -1) @ to_dev(head).T)
        tok = torch.arange(len(out), dtype=torch.int32, device=DEV)[:, None] % V
        lp, en, top, tl = ops.token_logprobs(z, tok, 3)
        ref = torch.log_softmax(z.double(), 1)
        # as the operator's own test: |d| of at most 20 times 2^-23, sums, a rounding
        assert (lp.double() - ref.gather(1, tok.long())).abs().max() <= 60 * 2.0 ** -23
        assert (en.double() + (ref.exp() * ref).sum(1)).abs().max() <= 400 * 2.0 ** -23
        assert torch.equal(top.long(), z.sort(dim=1, descending=True, stable=True).indices[:, :3])
        return top

    def store(k, v, counts):
        slots = np.concatenate([row_of[b] * S + have[b] + np.arange(n) for b, n in enumerate(counts)])
        ops.kv4_store(to_dev(k), to_dev(v), cache, slots=to_dev(slots.astype(np.int32)))
        lo = 0
        for b, n in enumerate(counts):
            for j, x in enumerate((k, v)):
                held = oracle.kv4_decode(*oracle.kv4_encode(values(x[lo:lo + n])))
                seen[b][j] = np.concatenate([seen[b][j], held])
            have[b] += n
            lo += n

    # a first chunk of each: attention over itself, unquantised
    counts = [60, 41]
    q, k, v = new(101)
    off = _i32([0, 60, 101])
    out, lse = ops.prompt_attention(to_dev(q), to_dev(k), to_dev(v), q_offsets=off)
    ro, rl = oracle.prompt_attention(values(q), values(k), values(v), [0, 60, 101], [0, 60, 101], D ** -0.5)
    for r in (0, 1, 59, 60, 100):
        lo = 0 if r < 60 else 60
        for h in range(Hq):
            check_row(vals(out)[r, h], to_host(lse)[r, h], ro[r, h], rl[r, h], values(q)[r, h],
                      values(k)[lo:r + 1, h // 4], values(v)[lo:r + 1, h // 4], D ** -0.5, dtype)
    logprobs_of(out)
    store(k, v, counts)

    # the rest of the first: its history comes back from the cache, in front of the new
    q, k, v = new(30)
    kk = torch.empty((90, Hkv, D), dtype=t, device=DEV)
    vv = torch.empty_like(kk)
    ops.kv4_load(cache, slots=_i32([row_of[0] * S + i for i in range(60)]), k=kk[:60], v=vv[:60])
    kk[60:], vv[60:] = to_dev(k), to_dev(v)
    assert np.array_equal(vals(kk[:60]), seen[0][0]) and np.array_equal(vals(vv[:60]), seen[0][1])
    out, lse = ops.prompt_attention(to_dev(q), kk, vv)
    K, Vv = vals(kk), vals(vv)
    for r in range(0, 30, 7):
        for h in range(Hq):
            ref, l = oracle.prompt.softmax_rows(D ** -0.5 * (K[:61 + r, h // 4] @ values(q)[r, h]),
                                                Vv[:61 + r, h // 4])
            check_row(vals(out)[r, h], to_host(lse)[r, h], ref, l, values(q)[r, h], K[:61 + r, h // 4],
                      Vv[:61 + r, h // 4], D ** -0.5, dtype)
    logprobs_of(out)
    store(k, v, [30, 0])

    # single tokens of both
    for _ in range(3):
        q, k, v = new(2)
        store(k, v, [1, 1])
        out, lse = ops.kv4_attention(to_dev(q), cache, lens=_i32(have), cache_row=_i32(row_of))
        for b in range(2):
            for h in range(Hq):
                K, Vv = seen[b][0][:, h // 4], seen[b][1][:, h // 4]
                ref, l = oracle.prompt.softmax_rows(D ** -0.5 * (K @ values(q)[b, h]), Vv)
                check_row(vals(out)[b, h], to_host(lse)[b, h], ref, l, values(q)[b, h], K, Vv,
                          D ** -0.5, dtype)
        logprobs_of(out)
    assert have == [93, 44]


def test_caches_of_4_bits_move_like_others():
    """beam_reorder and kv_gather on codes and scales; attention after them is that
    of the rows they came from."""
    g = torch.Generator(device=DEV).manual_seed(3)
    R, S, Hq, Hkv, D = 4, 40, 4, 2, 96
    cache = ops.kv4_cache(R, S, Hkv, D, DEV)
    ops.kv4_store(*(torch.randn((R * S, Hkv, D), device=DEV, generator=g) for _ in range(2)), cache)
    q = torch.randn((R, Hq, D), device=DEV, generator=g).bfloat16()
    lens, parent = _i32([40, 17, 33, 5]), _i32([[1, 0, 2, 1]])
    want = ops.kv4_attention(q, cache, lens=lens[parent[0].long()], cache_row=parent[0].clone())
    moved = [t.clone() for t in cache]
    for x in (0, 1):                                 # codes, scales: of equal bytes a position
        new_lens, err = ops.beam_reorder([moved[x][None], moved[2 + x][None]], parent, lens=lens)
        assert int(err) == 0
    got = ops.kv4_attention(q, moved, lens=new_lens)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    order = _i32([3, 1, 0, 2])
    gathered = [ops.kv_gather([t.view(1, R, -1)], index=order) for t in cache]
    gathered = [(x[0] if isinstance(x, tuple) else x).view(t.shape) for x, t in zip(gathered, cache)]
    a = ops.kv4_attention(q, gathered, lens=lens[order.long()])
    b = ops.kv4_attention(q, cache, lens=lens[order.long()], cache_row=order)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_joined_with_attention_over_other_keys():
    """A 4-bit history and bf16 keys since: two calls joined by their lse are attention
    over all keys."""
    g = torch.Generator(device=DEV).manual_seed(4)
    R, S, T, Hq, Hkv, D = 3, 300, 40, 4, 2, 64
    cache = ops.kv4_cache(R, S, Hkv, D, DEV)
    ops.kv4_store(*(torch.randn((R * S, Hkv, D), device=DEV, generator=g) for _ in range(2)), cache)
    ks, vs = (torch.randn((R, T, Hkv, D), device=DEV, generator=g) for _ in range(2))
    q = torch.randn((R, Hq, D), device=DEV, generator=g)
    o1, l1 = ops.kv4_attention(q, cache)
    o2, l2 = ops.prefix_attention(q, k_suffix=ks, v_suffix=vs)
    l = torch.logaddexp(l1, l2)
    out = o1 * (l1 - l).exp()[..., None] + o2 * (l2 - l).exp()[..., None]
    kk, vv = ops.kv4_load(cache, dtype=torch.float32)
    K = torch.cat([kk.view(R, S, Hkv, D), ks], 1).double().repeat_interleave(2, 2)
    V = torch.cat([vv.view(R, S, Hkv, D), vs], 1).double().repeat_interleave(2, 2)
    p = torch.softmax((q.double()[:, None] * K).sum(-1) * D ** -0.5, 1)
    ref = (p[..., None] * V).sum(1)
    # scores of at most 8 off by some 200 * 2^-24, numerators and sums likewise
    assert (out.double() - ref).abs().max() <= 2000 * 2.0 ** -24


class Step:
    """One pass over static buffers: store, prompt attention, load, attention,
    log-probabilities, each with its own workspace."""

    def __init__(self, seed, n=70, m=1500, S=700, V=4000, dtype=torch.bfloat16):
        g = torch.Generator(device=DEV).manual_seed(seed)
        r = lambda *s: torch.randn(s, device=DEV, generator=g).to(dtype)
        self.g, self.S = g, S
        self.q, self.k, self.v = r(n, 8, 64), r(m, 2, 64), r(m, 2, 64)
        self.off = _i32([0, n // 2, n]), _i32([0, m - 300, m])
        self.cache = ops.kv4_cache(3, S, 2, 64, DEV)
        self.slots = torch.randperm(3 * S, device=DEV, generator=g)[:m].int()
        self.q1, self.lens, self.rows = r(3, 8, 64), _i32([S, 500, 1]), _i32([2, 0, 1])
        self.z, self.tok = r(5, V), _i32([[1], [2], [V - 1], [0], [-1]])
        self.ws = [ops.workspace_tensor(max(256, x), DEV) for x in (
            ops.prompt_attention_workspace(n, m, 2, 8, 2, 64,
                                           ops.MOE_BF16 if dtype == torch.bfloat16 else ops.MOE_F32),
            ops.kv4_attention_workspace(3, S, 8, 2, 64), ops.token_logprobs_workspace(5, V, 1, 6))]
        self.outs = dict(a=torch.zeros_like(self.q), al=torch.zeros((n, 8), device=DEV),
                         kk=torch.zeros_like(self.k), vv=torch.zeros_like(self.v),
                         b=torch.zeros_like(self.q1), bl=torch.zeros((3, 8), device=DEV),
                         lp=torch.zeros((5, 1), device=DEV), en=torch.zeros(5, device=DEV),
                         tt=torch.zeros((5, 6), dtype=torch.int32, device=DEV),
                         tl=torch.zeros((5, 6), device=DEV))

    def fresh(self):
        for x in (self.q, self.k, self.v, self.q1, self.z):
            x.copy_(torch.randn(x.shape, device=DEV, generator=self.g))

    def run(self, stream=None):
        o = self.outs
        ops.kv4_store(self.k, self.v, self.cache, slots=self.slots, stream=stream)
        ops.prompt_attention(self.q, self.k, self.v, q_offsets=self.off[0], k_offsets=self.off[1],
                             out=o["a"], lse=o["al"], workspace=self.ws[0], stream=stream)
        ops.kv4_load(self.cache, slots=self.slots, k=o["kk"], v=o["vv"], stream=stream)
        ops.kv4_attention(self.q1, self.cache, lens=self.lens, cache_row=self.rows, out=o["b"],
                          lse=o["bl"], workspace=self.ws[1], stream=stream)
        ops.token_logprobs(self.z, self.tok, 6, logprobs=o["lp"], entropy=o["en"],
                           top_tokens=o["tt"], top_logprobs=o["tl"], workspace=self.ws[2],
                           stream=stream)

    def take(self):
        return {n: t.clone() for n, t in self.outs.items()}

    def clear(self):
        for t in self.outs.values():
            t.zero_()
        for t in self.cache:
            t.zero_()


def _equal(a, b):
    for n in a:
        assert torch.equal(a[n], b[n]), n


def _capture(step):
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step.run()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step.run()
    return graph


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_captured_and_replayed(dtype):
    step = Step(5, dtype=dtype)
    graph = _capture(step)
    for _ in range(4):
        step.fresh()
        step.clear()
        step.run()
        want = step.take()
        step.clear()
        graph.replay()
        torch.cuda.synchronize()
        _equal(step.take(), want)


def test_two_graphs_at_once_on_streams_of_their_own():
    steps = [Step(6), Step(7, n=64, m=900, S=400, V=33000)]
    graphs = [_capture(s) for s in steps]
    streams = [torch.cuda.Stream() for _ in steps]
    for _ in range(3):
        want = []
        for s in steps:
            s.fresh()
            s.clear()
            s.run()
            want.append(s.take())
            s.clear()
        torch.cuda.synchronize()
        for _ in range(5):
            for g, st in zip(graphs, streams):
                with torch.cuda.stream(st):
                    g.replay()
        torch.cuda.synchronize()
        for s, w in zip(steps, want):
            _equal(s.take(), w)


def test_given_stream_is_the_one_that_is_used():
    """Calls on a side stream, given and current, behind long kernels there that write
    their inputs."""
    step = Step(8)
    step.run()
    torch.cuda.synchronize()
    want = step.take()
    names = ("q", "k", "v", "q1", "z")
    src = {n: getattr(step, n).clone() for n in names}
    side = torch.cuda.Stream()
    big = torch.randn((4096, 4096), device=DEV)
    for given in (True, False):
        for n in names:
            getattr(step, n).zero_()
        step.clear()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(20):
                big = big @ big * 1e-4
            for n in names:
                getattr(step, n).copy_(src[n])
            if not given:
                step.run()
        if given:
            step.run(stream=side)
        torch.cuda.synchronize()
        _equal(step.take(), want)


def test_calls_of_a_shrinking_batch_on_one_workspace():
    g = torch.Generator(device=DEV).manual_seed(9)
    ws = ops.workspace_tensor(ops.kv4_attention_workspace(9, 3000, 4, 1, 64), DEV)
    cache = ops.kv4_cache(9, 3000, 1, 64, DEV)
    ops.kv4_store(*(torch.randn((9 * 3000, 1, 64), device=DEV, generator=g) for _ in range(2)), cache)
    q = torch.randn((9, 4, 64), device=DEV, generator=g).bfloat16()
    whole = ops.kv4_attention(q, cache, workspace=ws)
    for n in range(8, 0, -1):
        out, lse = ops.kv4_attention(q[:n], cache, workspace=ws)
        # other splits: of the roundings of numerators and result
        assert (out.float() - whole[0][:n].float()).abs().max() <= 2.0 ** -7
        assert (lse - whole[1][:n]).abs().max() <= 2.0 ** -12
    ws = ops.workspace_tensor(ops.prompt_attention_workspace(300, 9000, 4, 4, 1, 64), DEV)
    k, v = (torch.randn((9000, 1, 64), device=DEV, generator=g).bfloat16() for _ in range(2))
    for n in (300, 100, 7, 1):
        for m in (9000, 3000, 500):
            x = torch.randn((n, 4, 64), device=DEV, generator=g).bfloat16()
            a = ops.prompt_attention(x, k[:m], v[:m], workspace=ws)
            b = ops.prompt_attention(x, k[:m], v[:m])
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_many_rows_tokens_and_sequences():
    g = torch.Generator(device=DEV).manual_seed(10)
    # more rows than a grid dimension of 65535 would take
    R, S, D = 70001, 3, 32
    cache = ops.kv4_cache(R, S, 1, D, DEV)
    ops.kv4_store(*(torch.randn((R * S, 1, D), device=DEV, generator=g) for _ in range(2)), cache)
    q = torch.randn((R, 2, D), device=DEV, generator=g)
    out, lse = ops.kv4_attention(q, cache, scale=0.3)
    kk, vv = (x.view(R, S, 1, D).double() for x in ops.kv4_load(cache, dtype=torch.float32))
    s = 0.3 * (q.double()[:, None] * kk).sum(-1)
    p = torch.softmax(s, 1)
    # scores of at most 30 off by 100 * 2^-24 of that, weights and sums likewise
    assert (out.double() - (p[..., None] * vv).sum(1)).abs().max() <= 30 * 100 * 2.0 ** -24 * 5
    assert (lse.double() - torch.logsumexp(s, 1)).abs().max() <= 30 * 100 * 2.0 ** -24
    # sequences of one token: out is its value
    N = 70001
    x = torch.randn((N, 1, 8), device=DEV, generator=g)
    off = torch.arange(N + 1, dtype=torch.int32, device=DEV)
    out, lse = ops.prompt_attention(x, x, x, q_offsets=off)
    assert (out - x).abs().max() <= 5 * 2.0 ** -22
    # rows of logits
    z = torch.randn((70001, 37), device=DEV, generator=g)
    lp, en, top, tl = ops.token_logprobs(z, torch.zeros((70001, 1), dtype=torch.int32, device=DEV), 2)
    ref = torch.log_softmax(z.double(), 1)
    assert (lp[:, 0].double() - ref[:, 0]).abs().max() <= 60 * 2.0 ** -23
    assert torch.equal(top[:, 0].long(), z.argmax(1))
    # the largest vocabulary
    z = torch.randn((1, 1 << 24), device=DEV, generator=g)
    lp, en, top, tl = ops.token_logprobs(z, _i32([[(1 << 24) - 1]]), 64)
    ref = torch.log_softmax(z.double(), 1)
    assert abs(float(lp) - float(ref[0, -1])) <= 60 * 2.0 ** -23
    assert torch.equal(top[0].long(), z[0].sort(descending=True, stable=True).indices[:64])


def test_refusals_of_the_binding():
    q, k = torch.zeros((4, 4, 64), device=DEV), torch.zeros((4, 2, 64), device=DEV)
    for bad in (lambda: ops.prompt_attention(q, k, k.bfloat16()),
                lambda: ops.prompt_attention(q, k, k[:3]),
                lambda: ops.prompt_attention(q, k.cpu(), k),
                lambda: ops.prompt_attention(q, k, k[:, :, :32]),
                lambda: ops.prompt_attention(q.transpose(0, 1), k, k),
                lambda: ops.prompt_attention(q, k, k, q_offsets=_i32([0])),
                lambda: ops.prompt_attention(q, k[:2], k[:2], q_offsets=_i32([0, 2, 4])),
                lambda: ops.prompt_attention(q, k, k, q_offsets=_i32([0, 4]), k_offsets=_i32([0, 2, 4])),
                lambda: ops.kv4_cache(1, 4, 2, 48, DEV),
                lambda: ops.kv4_store(k, k, ops.kv4_cache(1, 4, 2, 96, DEV)),
                lambda: ops.kv4_store(k, k, ops.kv4_cache(1, 4, 2, 64, DEV), slots=_i32([0, 1])),
                lambda: ops.kv4_load(ops.kv4_cache(1, 4, 2, 64, DEV), k=k),
                lambda: ops.kv4_attention(q, ops.kv4_cache(4, 4, 2, 96, DEV)),
                lambda: ops.kv4_attention(q, ops.kv4_cache(4, 4, 2, 64, DEV), lens=_i32([1])),
                lambda: ops.token_logprobs(q[0], _i32([1])),
                lambda: ops.token_logprobs(q[0].T, _i32([[1]] * 64)),
                lambda: ops.token_logprobs(q[0], top_tokens=_i32([[1]] * 4))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        ops.prompt_attention(q.half(), k.half(), k.half())
    for bad in (lambda: ops.prompt_attention(q, k, k, out=q),
                lambda: ops.kv4_attention(q, ops.kv4_cache(2, 4, 2, 64, DEV)),
                lambda: ops.kv4_store(k, k, ops.kv4_cache(1, 3, 2, 64, DEV)),
                lambda: ops.token_logprobs(q[0], want_entropy=False)):
        with pytest.raises(ops.MoeError) as e:
            bad()
        assert e.value.status == ops.MOE_ERR_ARG
