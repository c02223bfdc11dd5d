"""The cache's operators as they are used together: a prompt's rows made, attended to, weighed and evicted, then new tokens on what is
left; a training step; captured into a graph; on another stream; by native code and by the general path."""
import math
import types

import pytest
import torch

import cache_ops_ref as ref
from paper_2512_10411_amd import binding

pytestmark = pytest.mark.gpu
HQ, HKV, D, PAGE = 8, 2, 128, 16
INV = (1e5 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)).float()


def near(got, want, tag, rel=2.0 ** -7):
    """Attention of 16-bit rows against 64 bits.  Its own roundings (P, the result) are half a step each; the rows that it reads have been
    rounded once more than the reference's: 2^-9 of each score's terms, which random signs average out; together below 2^-7 in
    the 2-norm."""
    off = ((got.cpu().double() - want).norm() / want.norm()).item()
    print(f"[chain] {tag}: {off:.2e}", flush=True)
    assert off <= rel, (tag, off)


def attention(q, k, v, seen):
    k, v = (t.double().repeat_interleave(q.shape[0] // k.shape[0], 0) for t in (k, v))
    s = (q.double() @ k.transpose(1, 2) / math.sqrt(D)).masked_fill(~seen, -math.inf)
    return torch.softmax(s, -1) @ v, torch.logsumexp(s, -1)


def test_a_conversation_on_a_bounded_cache():
    gen = torch.Generator().manual_seed(1)
    prompts, budget, n_sink, n_recent = [150, 64, 201], 80, 4, 16
    B, longest = len(prompts), max(prompts)
    cu = torch.tensor([0] + list(torch.tensor(prompts).cumsum(0)), dtype=torch.int32).cuda()
    w = [(1 + 0.2 * torch.randn(D, generator=gen)) for _ in range(2)]
    how = dict(q_weight=w[0].cuda(), k_weight=w[1].cuda(), eps=1e-6)
    per = -(-longest // PAGE)
    pages = torch.zeros(2, B * per + 2, HKV, PAGE, D, dtype=torch.bfloat16, device="cuda")
    k_cache, v_cache = pages
    table = torch.randperm(B * per + 2, generator=gen)[:B * per].to(torch.int32).view(B, per).cuda()
    held = lambda cache, b, n: cache[table[b].long()].permute(1, 0, 2, 3).flatten(1, 2)[:, :n].cpu()  # noqa: E731

    # ---- the prompts, packed, straight from a fused projection
    x = torch.randn(sum(prompts), HQ + 2 * HKV, D, generator=gen).bfloat16()
    parts = [t.permute(1, 0, 2) for t in x.split((HQ, HKV, HKV), 1)]
    on = [t.permute(1, 0, 2) for t in x.cuda().split((HQ, HKV, HKV), 1)]
    q, _, _ = binding.swaa_qk_norm_rope(on[0], on[1], INV.cuda(), v=on[2], k_out=k_cache, v_out=v_cache, cu_seqlens_q=cu, cu_seqlens_k=cu,
                                        max_seqlen_q=longest, max_seqlen_k=longest, block_table=table, **how)
    packed = dict(cu_seqlens_q=cu, cu_seqlens_k=cu, max_seqlen_q=longest, max_seqlen_k=longest, block_table=table)
    out, lse = binding.swaa_attn_fwd_ex(q, k_cache, v_cache, 10 ** 9, 0, **packed)
    weights = binding.swaa_attn_key_weights(q, k_cache, lse, 10 ** 9, 0, **packed)
    at = 0
    for b, n in enumerate(prompts):
        rows = slice(at, at + n)
        at += n
        made = [ref.norm_rope(p[:, rows], weight, torch.arange(n), INV, 1e-6, False)[0] for p, weight in zip(parts[:2], w)]
        want, _ = attention(*made, parts[2][:, rows], ref.visible(n, n, n, 0, n))
        near(out[:, rows], want, f"prompt of {n}")
        got, bound = ref.key_weights(q[:, rows].cpu(), held(k_cache, b, n), lse[:, rows].cpu(), 1 / math.sqrt(D), ref.visible(n, n, n, 0, n))
        assert ((weights[b, :, :n].cpu().double() - got).abs() <= bound).all()

    # ---- down to the budget
    before = [[held(c, b, n) for c in (k_cache, v_cache)] for b, n in enumerate(prompts)]
    old = weights.cpu()
    lens = torch.tensor(prompts, dtype=torch.int32).cuda()
    kept, lens = binding.swaa_cache_evict(k_cache, v_cache, weights, budget, n_sink, n_recent, seq_lens=lens, block_table=table,
                                          max_seqlen_k=longest)
    assert lens.tolist() == [min(n, budget) for n in prompts]
    for b, n in enumerate(prompts):
        for g in range(HKV):
            rows = ref.evict(old[b, g, :n], n, budget, n_sink, n_recent)
            assert kept[b, g, :len(rows)].tolist() == rows
            for c, was in zip((k_cache, v_cache), before[b]):
                assert torch.equal(held(c, b, len(rows))[g], was[g, rows])

    # ---- new tokens: behind the kept rows, at positions that go on
    for step in range(3):
        x = torch.randn(B, 1, HQ + 2 * HKV, D, generator=gen).bfloat16()
        new = [t.permute(0, 2, 1, 3) for t in x.cuda().split((HQ, HKV, HKV), 2)]
        pos = torch.tensor([[n + step] for n in prompts], dtype=torch.int32)
        lens = lens + 1
        room = dict(seq_lens=lens, block_table=table, max_seqlen_k=longest)
        held_before = [[held(c, b, int(lens[b]) - 1) for c in (k_cache, v_cache)] for b in range(B)]
        q, _, _ = binding.swaa_qk_norm_rope(new[0], new[1], INV.cuda(), pos.cuda(), v=new[2], k_out=k_cache, v_out=v_cache, **room, **how)
        out, lse = binding.swaa_attn_decode_ex(q, k_cache, v_cache, longest, 0, **room)
        old = weights.cpu()
        binding.swaa_attn_key_weights(q, k_cache, lse, longest, 0, weights=weights, decay=1.0, **room)
        for b in range(B):
            n = int(lens[b])
            mine = x[b].permute(1, 0, 2)
            made = [ref.norm_rope(p, weight, pos[b], INV, 1e-6, False)[0] for p, weight in zip(mine.split((HQ, HKV, HKV), 0)[:2], w)]
            k = torch.cat((held_before[b][0].double(), made[1]), 1)
            v = torch.cat((held_before[b][1].double(), mine[HQ + HKV:].double()), 1)
            want, _ = attention(made[0], k, v, ref.visible(1, n, n, 0, n))
            near(out[b], want, f"token {step} of {b}")
            added, bound = ref.key_weights(q[b].cpu(), held(k_cache, b, n), lse[b].cpu(), 1 / math.sqrt(D), ref.visible(1, n, n, 0, n))
            summed = old[b, :, :n].double() + added
            assert ((weights[b, :, :n].cpu().double() - summed).abs() <= bound + 2.0 ** -23 * (summed + added)).all()


def test_a_training_step():
    """Norms, rotation and attention, and back, against 64-bit automatic differentiation."""
    gen = torch.Generator().manual_seed(2)
    B, N, window, n_sink = 1, 150, 60, 3
    x = torch.randn(B, N, HQ + 2 * HKV, D, generator=gen).bfloat16()
    w = [(1 + 0.2 * torch.randn(D, generator=gen)) for _ in range(2)]
    dout = torch.randn(B, HQ, N, D, generator=gen).bfloat16()
    how = dict(q_weight=w[0].cuda(), k_weight=w[1].cuda())
    on = x.cuda()
    q_in, k_in, v = (t.permute(0, 2, 1, 3) for t in on.split((HQ, HKV, HKV), 2))
    v = v.contiguous()
    q, k, _ = binding.swaa_qk_norm_rope(q_in, k_in, INV.cuda(), **how)
    out, lse = binding.swaa_attn_fwd(q, k, v, window, n_sink)
    dq, dk, dv = binding.swaa_attn_bwd(q, k, v, out, lse, dout.cuda(), window, n_sink)
    got = binding.swaa_qk_norm_rope_bwd(dq, dk, q_in, k_in, INV.cuda(), **how)

    xs = [t.permute(0, 2, 1, 3).double().requires_grad_() for t in x.split((HQ, HKV, HKV), 2)]
    ws = [t.double().requires_grad_() for t in w]
    made = [ref.norm_rope(xs[i], ws[i], torch.arange(N), INV, 1e-6, False)[0] for i in range(2)]
    o = attention(made[0][0], made[1][0], xs[2][0], ref.visible(N, N, window, n_sink, N))[0]
    want = torch.autograd.grad(o, xs + ws, dout[0].double())
    # (the rows, P, dS, dq and dk are rounded to bfloat16 once each, 2^-9 on average of the 2-norm; dS is a difference of terms of the
    # size of P dP, which doubles what its rounding weighs: 2^-6 holds with a margin)
    for name, a, b in (("dq", got[0], want[0]), ("dk", got[1], want[1]), ("dv", dv, want[2]), ("dq_weight", got[2], want[3]),
                       ("dk_weight", got[3], want[4])):
        near(a, b, name, 2.0 ** -6)


class Step:
    """One new token of each sequence, weighed, and the cache cut back: everything on fixed memory."""

    def __init__(self, seed):
        gen = torch.Generator().manual_seed(seed)
        self.lens = [300, 222, 40]
        self.cache = [ref.Cache("paged", 3, HKV, 304, D, torch.bfloat16, torch.Generator().manual_seed(seed + i)) for i in range(2)]
        self.table = self.cache[0].table
        self.start = [c.gpu.clone() for c in self.cache]
        self.weights0 = torch.rand(3, HKV, 304, generator=gen).cuda()
        self.weights = self.weights0.clone()
        self.x = torch.randn(3, 1, HQ + 2 * HKV, D, generator=gen).bfloat16().cuda()
        self.seq = torch.tensor(self.lens, dtype=torch.int32).cuda()
        self.pos = torch.tensor([[5000], [77], [10 ** 6]], dtype=torch.int32).cuda()
        self.w = torch.ones(D).cuda()
        self.inv = INV.cuda()

    def __call__(self, **kw):
        for c, was in zip(self.cache, self.start):
            c.gpu.copy_(was)
        self.weights.copy_(self.weights0)
        q_in, k_in, v_in = (t.permute(0, 2, 1, 3) for t in self.x.split((HQ, HKV, HKV), 2))
        k, v = (c.view for c in self.cache)
        room = dict(seq_lens=self.seq, block_table=self.table, max_seqlen_k=304)
        q, _, _ = binding.swaa_qk_norm_rope(q_in, k_in, self.inv, self.pos, self.w, self.w, v=v_in, k_out=k, v_out=v, **room, **kw)
        out, lse = binding.swaa_attn_decode_ex(q, k, v, 304, 0, **room, **kw)
        binding.swaa_attn_key_weights(q, k, lse, 304, 0, weights=self.weights, decay=1.0, **room, **kw)
        kept, lens = binding.swaa_cache_evict(k, v, self.weights, 128, 4, 16, **room, **kw)
        return [q, out, lse, kept, lens, self.weights.clone(), self.cache[0].gpu.clone(), self.cache[1].gpu.clone()]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_two_captured_steps_replayed_among_eager_ones():
    first, second = Step(3), Step(4)
    want = [f() for f in (first, second)]
    torch.cuda.synchronize()
    graphs, outs = [], []
    side = torch.cuda.Stream()
    for f in (first, second):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            f()
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(f())
        graphs.append(graph)
    for replay in range(4):
        for i in (0, 1):
            graphs[i].replay()
        torch.cuda.synchronize()
        for i in (0, 1):
            assert same(outs[i], want[i]), (replay, i)
        assert same(first(), want[0])  # an eager step in between
        torch.cuda.synchronize()


def test_a_captured_backward():
    gen = torch.Generator(device="cuda").manual_seed(5)
    q, k, dq, dk = (torch.randn(2, H, 333, D, generator=gen, device="cuda").bfloat16() for H in (HQ, HKV, HQ, HKV))
    w, inv = torch.ones(D, device="cuda"), INV.cuda()
    call = lambda: binding.swaa_qk_norm_rope_bwd(dq, dk, q, k, inv, q_weight=w, k_weight=w)  # noqa: E731
    want = [t.clone() for t in call()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert same(got, want) and same(call(), want)


def long_calls():
    gen = torch.Generator(device="cuda").manual_seed(6)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    q, k = rand(1, HQ, 1500, D).bfloat16(), rand(1, HKV, 1500, D).bfloat16()
    w, inv = torch.ones(D, device="cuda"), INV.cuda()
    _, lse = binding.swaa_attn_fwd(q, k, k, 1500, 0)
    cache, weights = rand(1, 2, 20000, 64).half(), rand(1, 2, 20000).exp()
    return {
        "norm_rope": lambda **s: binding.swaa_qk_norm_rope(q, k, inv, q_weight=w, k_weight=w, **s)[:2],
        "norm_rope_bwd": lambda **s: binding.swaa_qk_norm_rope_bwd(q, k, q, k, inv, q_weight=w, k_weight=w, **s),
        "key_weights": lambda **s: (binding.swaa_attn_key_weights(q, k, lse, 1500, 0, **s),),
        "evict": lambda **s: binding.swaa_cache_evict(cache.clone(), cache.clone(), weights.clone(), 5000, 4, 100, **s),
    }


@pytest.mark.parametrize("call", ["norm_rope", "norm_rope_bwd", "key_weights", "evict"])
def test_what_a_call_allocates_comes_from_the_launch_streams_pool(call, monkeypatch):
    f = long_calls()[call]
    want = [t.clone() for t in f()]
    side, pools = torch.cuda.Stream(), []
    for name in ("empty", "empty_like"):
        def recording(*args, real=getattr(torch, name), **kwargs):
            pools.append(torch.cuda.current_stream().cuda_stream)
            return real(*args, **kwargs)
        monkeypatch.setattr(torch, name, recording)
    torch.cuda.synchronize()
    got = f(stream=side)
    again = f(stream=side.cuda_stream)
    torch.cuda.synchronize()
    assert len(pools) >= 4 and all(p == side.cuda_stream for p in pools)
    assert torch.cuda.current_stream() == torch.cuda.default_stream()
    assert same(got, want) and same(again, want)


NOTHING = types.SimpleNamespace(**{n: lambda *args: None for n in ("fwd", "decode", "decode_ex", "fill_fwd_ex", "norm_rope", "norm_rope_bwd",
                                                                   "key_weights", "evict")})


def forms():
    step, b = Step(7), binding
    q, k, v = (t.permute(0, 2, 1, 3) for t in torch.randn(2, 50, HQ + 2 * HKV, D, device="cuda").half().split((HQ, HKV, HKV), 2))
    w, inv, pos = torch.ones(D, device="cuda"), INV.cuda(), torch.arange(100, dtype=torch.int32, device="cuda").view(2, 50)
    packed = [t[0] for t in (q, k, v)]
    cu = torch.tensor([0, 20, 50], dtype=torch.int32, device="cuda")
    room = lambda: torch.zeros(2, HKV, 64, D, dtype=torch.float16, device="cuda")  # noqa: E731
    lens = torch.tensor([60, 50], dtype=torch.int32, device="cuda")
    lse = torch.zeros(2, HQ, 50, device="cuda")
    weights = lambda: torch.ones(2, HKV, 70, device="cuda")  # noqa: E731
    cut = dict(n_keep=20, n_sink=1, n_recent=2)
    return {  # name: (call, taken by the native way)
        "a step": (step, 4),
        "plain": (lambda: b.swaa_qk_norm_rope(q, k, inv)[:2], 1),
        "norms only": (lambda: b.swaa_qk_norm_rope(q, k, None, q_weight=w, k_weight=w, eps=1e-3)[:2], 1),
        "positions, neighbours": (lambda: b.swaa_qk_norm_rope(q, k, inv, pos, w, w, interleaved=True)[:2], 1),
        "a contiguous cache": (lambda: b.swaa_qk_norm_rope(q, k, inv, v=v, k_out=room(), v_out=room(), seq_lens=lens), 1),
        "packed": (lambda: b.swaa_qk_norm_rope(packed[0], packed[1], inv, cu_seqlens_q=cu, max_seqlen_q=30)[:2], 1),
        "results given": (lambda: b.swaa_qk_norm_rope(q, k, inv, q_out=torch.empty_like(q))[:2], 0),
        "eps below zero": (lambda: b.swaa_qk_norm_rope(q, k, inv, q_weight=w, k_weight=w, eps=-1.0), 1),
        "an int for eps": (lambda: b.swaa_qk_norm_rope(q, k, inv, q_weight=w, k_weight=w, eps=1)[:2], 0),
        "one weight": (lambda: b.swaa_qk_norm_rope(q, k, inv, q_weight=w), 0),
        "weights of bf16": (lambda: b.swaa_qk_norm_rope(q, k, inv, q_weight=w.bfloat16(), k_weight=w.bfloat16()), 0),
        "rows of another length": (lambda: b.swaa_qk_norm_rope(q, k[:, :, 1:], inv), 0),
        "a cache of another type": (lambda: b.swaa_qk_norm_rope(q, k, inv, v=v, k_out=room().bfloat16(), v_out=room().bfloat16()), 0),
        "values without a cache": (lambda: b.swaa_qk_norm_rope(q, k, inv, v=v), 0),
        "backward": (lambda: b.swaa_qk_norm_rope_bwd(q, k, q, k, inv, pos, w, w), 1),
        "backward without weights": (lambda: b.swaa_qk_norm_rope_bwd(q, k, q, k, inv)[:2], 1),
        "backward of another shape": (lambda: b.swaa_qk_norm_rope_bwd(q[:, 1:], k, q, k, inv), 0),
        "weigh": (lambda: b.swaa_attn_key_weights(q, k, lse, 10, 2, weights=weights()), 1),
        "weigh, lengths, prompts": (lambda: b.swaa_attn_key_weights(q, room(), lse, 10, 2, 30, 0.1, weights(), 0.5, seq_lens=lens, n_prompts=lens), 1),
        "weigh, new weights": (lambda: b.swaa_attn_key_weights(q, k, lse, 10, 2), 0),
        "weigh, packed": (lambda: b.swaa_attn_key_weights(packed[0], packed[1], lse[0], 10, 2, weights=weights(), cu_seqlens_q=cu, cu_seqlens_k=cu,
                                                          max_seqlen_q=30, max_seqlen_k=30), 1),
        "weights too short": (lambda: b.swaa_attn_key_weights(q, k, lse, 10, 2, weights=weights()[:, :, :40]), 0),
        "decay below zero": (lambda: b.swaa_attn_key_weights(q, k, lse, 10, 2, weights=weights(), decay=-1.0), 1),
        "lse of another shape": (lambda: b.swaa_attn_key_weights(q, k, lse[:, :, 1:], 10, 2, weights=weights()), 0),
        "evict": (lambda: b.swaa_cache_evict(room(), room(), weights(), seq_lens=lens, **cut), 1),
        "evict nothing to spare": (lambda: b.swaa_cache_evict(room(), room(), weights(), 2, 3, 4), 1),
        "evict, too long": (lambda: b.swaa_cache_evict(room(), room(), weights(), max_seqlen_k=65, **cut), 0),
        "evict, other values": (lambda: b.swaa_cache_evict(room(), room()[:, :, 1:], weights(), **cut), 0),
    }


def test_native_and_general_calls_agree(monkeypatch):
    binding._torch()
    real = binding._host
    for name, (f, taken) in forms().items():
        print(f"[case] {name}", flush=True)
        outcome, count = [], [0]

        def counted(n):
            def call(*args):
                r = getattr(real, n)(*args)
                count[0] += r is not None
                return r
            return call

        for host in (types.SimpleNamespace(**{n: counted(n) for n in vars(NOTHING)}), NOTHING):
            with monkeypatch.context() as m:
                m.setattr(binding, "_host", host)
                try:
                    r = f()
                except Exception as e:  # noqa: BLE001 (what is refused has to be refused alike)
                    r = (type(e), str(e))
            outcome.append([r] if isinstance(r, torch.Tensor) else r)
        torch.cuda.synchronize()
        assert count[0] == taken, (name, count[0])
        for x, y in zip(*outcome):
            if isinstance(y, torch.Tensor):
                assert x.dtype == y.dtype and x.stride() == y.stride() and torch.equal(x, y), name
            else:
                assert x == y, (name, x, y)
