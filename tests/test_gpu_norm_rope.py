"""swaa_qk_norm_rope and its backward against their definitions in 64 bits.

Bounds: one rounding to 16 bits, half a step, finfo.eps / 2 of the result (2^-25 where binary16 is subnormal), and the 32-bit
arithmetic in front of it.  That is a chain of some ten roundings of 2^-24 behind a sum of squares (at most 13 additions in a
row of it): below 2^-19 of the terms a result is the sum of.  Sums over rows add 2^-24 per term at most.
"""
import pytest
import torch

import cache_ops_ref as ref
from paper_2512_10411_amd import binding

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def close(got, want, size, dtype, tag):
    got, half = got.detach().cpu().double(), torch.finfo(dtype).eps / 2
    bound = half * want.abs() + 2.0 ** -19 * size * (1 + half) + (2.0 ** -25 if dtype is torch.float16 else 2.0 ** -130)
    worst = ((got - want).abs() / bound).max().item() if want.numel() else 0.0
    print(f"[norm_rope] {tag}: {worst:.3f} of the bound", flush=True)
    assert worst <= 1.0, (tag, worst)


def frequencies(R, base=1e6):
    return None if R == 0 else (base ** (-torch.arange(0, R, 2, dtype=torch.float64) / R)).float()


def weights_of(D, gen, norm):
    return [1 + 0.3 * torch.randn(D, generator=gen) for _ in range(2)] if norm else [None, None]


def gpu(t):
    return None if t is None else t.cuda()


# head dimension, rotated, norm, interleaved, Hq, Hkv, B, N
SHAPES = [(128, 128, True, False, 8, 2, 2, 37), (128, 64, True, False, 5, 5, 1, 1), (64, 64, True, True, 4, 1, 3, 65),
          (64, 0, True, False, 4, 2, 1, 130), (32, 32, True, False, 7, 1, 2, 300), (96, 48, True, True, 6, 3, 1, 77),
          (256, 256, True, False, 3, 1, 2, 19), (160, 80, False, False, 4, 4, 1, 33), (224, 16, True, True, 2, 1, 1, 50),
          (128, 128, False, True, 32, 8, 1, 1000), (192, 192, True, False, 1, 1, 1, 2)]


@pytest.mark.parametrize("fmt", ["bf16", "fp16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_prompts_of_projections(shape, fmt):
    D, R, norm, interleaved, Hq, Hkv, B, N = shape
    gen = torch.Generator().manual_seed(hash(shape) % 1000)
    dtype = DTYPES[fmt]
    print(f"[case] {shape} {fmt}", flush=True)
    qkv = (2 * torch.randn(B, N, Hq + 2 * Hkv, D, generator=gen)).to(dtype)
    q, k = qkv[:, :, :Hq].permute(0, 2, 1, 3), qkv[:, :, Hq:Hq + Hkv].permute(0, 2, 1, 3)
    on_gpu = qkv.cuda()
    gq, gk = on_gpu[:, :, :Hq].permute(0, 2, 1, 3), on_gpu[:, :, Hq:Hq + Hkv].permute(0, 2, 1, 3)
    qw, kw = weights_of(D, gen, norm)
    inv = frequencies(R)
    qo, ko, vo = binding.swaa_qk_norm_rope(gq, gk, gpu(inv), q_weight=gpu(qw), k_weight=gpu(kw), interleaved=interleaved)
    assert vo is None and qo.is_contiguous() and ko.is_contiguous() and qo.dtype is dtype
    for name, got, x, w in (("q", qo, q, qw), ("k", ko, k, kw)):
        close(got, *ref.norm_rope(x, w, torch.arange(N), inv, 1e-6, interleaved), dtype, f"{name} {shape} {fmt}")
    assert torch.equal(on_gpu.cpu(), qkv)


@pytest.mark.parametrize("N", [127, 128, 129, 1100])
@pytest.mark.parametrize("D", [32, 64, 96, 128, 256])
def test_few_tokens_and_many(D, N):
    """Two sequences: around 256 tokens, from where on every wave takes tokens of its own, and more than one workgroup's share."""
    gen = torch.Generator().manual_seed(D + N)
    print(f"[case] {D} {N}", flush=True)
    qkv = torch.randn(2, N, 9, D, generator=gen).to(torch.bfloat16)
    on_gpu = qkv.cuda()
    (q, k), (gq, gk) = ((t[:, :, :6].permute(0, 2, 1, 3), t[:, :, 6:].permute(0, 2, 1, 3)) for t in (qkv, on_gpu))
    qw, kw = weights_of(D, gen, True)
    inv = frequencies(D)
    qo, ko, _ = binding.swaa_qk_norm_rope(gq, gk, inv.cuda(), q_weight=gpu(qw), k_weight=gpu(kw))
    for name, got, x, w in (("q", qo, q, qw), ("k", ko, k, kw)):
        close(got, *ref.norm_rope(x, w, torch.arange(N), inv, 1e-6, False), torch.bfloat16, f"{name} {D} {N}")


def test_far_positions_of_every_sign():
    gen = torch.Generator().manual_seed(3)
    B, N, H, D = 1, 6, 2, 128
    q, k = (torch.randn(B, H, N, D, generator=gen).to(torch.float16) for _ in range(2))
    pos = torch.tensor([[0, 1, 131071, 2 ** 31 - 1, -1, -2 ** 31]], dtype=torch.int32)
    inv = frequencies(D, 1e4)
    qo, ko, _ = binding.swaa_qk_norm_rope(q.cuda(), k.cuda(), inv.cuda(), positions=pos.cuda())
    for got, x in ((qo, q), (ko, k)):  # 2^31 radians in 64 bits: 2^-22 of one at most, far below the bound
        close(got, *ref.norm_rope(x, None, pos[:, None], inv, 1e-6, False), torch.float16, "far")


def test_rows_of_zeros_and_tiny_and_large_ones():
    D = 128
    q = torch.zeros(1, 1, 4, D)
    q[0, 0, 1] = 1e-20
    q[0, 0, 2] = 1e15
    q[0, 0, 3, 5] = 3.0
    q = q.to(torch.bfloat16)
    w, inv = torch.ones(D), frequencies(D)
    qo, _, _ = binding.swaa_qk_norm_rope(q.cuda(), q.cuda(), inv.cuda(), q_weight=w.cuda(), k_weight=w.cuda())
    close(qo, *ref.norm_rope(q, w, torch.arange(4), inv, 1e-6, False), torch.bfloat16, "zeros")


def test_in_place():
    gen = torch.Generator().manual_seed(4)
    q, k = torch.randn(2, 8, 45, 64, generator=gen).bfloat16().cuda(), torch.randn(2, 2, 45, 64, generator=gen).bfloat16().cuda()
    w, inv = torch.ones(64).cuda(), frequencies(64).cuda()
    want = binding.swaa_qk_norm_rope(q, k, inv, q_weight=w, k_weight=w)
    got = binding.swaa_qk_norm_rope(q, k, inv, q_weight=w, k_weight=w, q_out=q, k_out=k)
    assert got[0] is q and got[1] is k
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])


@pytest.mark.parametrize("page_size", [16, 4, 7, 1])
@pytest.mark.parametrize("kind,B,Nq,Nk,lens,given", [
    ("paged", 5, 1, 90, [1, 90, 17, 33, 64], True), ("paged", 6, 4, 60, [4, 2, 77, 0, -5, 62], False), ("dense", 5, 1, 40, [40, 1, 7, 0, 41], False),
    ("rows", 2, 3, 50, None, True), ("paged", 70, 1, 20, list(range(1, 21)) * 3 + [20] * 10, True), ("dense", 1, 33, 33, None, False)])
def test_new_tokens_go_into_the_cache(kind, B, Nq, Nk, lens, given, page_size):
    if kind != "paged" and page_size != 16:
        pytest.skip("pages of paged caches only")
    gen = torch.Generator().manual_seed(Nk + page_size)
    Hq, Hkv, D = 8, 2, 128
    x = torch.randn(B, Nq, Hq + 2 * Hkv, D, generator=gen).bfloat16()
    parts = [t.permute(0, 2, 1, 3) for t in (x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:])]
    on = x.cuda()
    gq, gk, gv = (t.permute(0, 2, 1, 3) for t in (on[:, :, :Hq], on[:, :, Hq:Hq + Hkv], on[:, :, Hq + Hkv:]))
    kc, vc = (Cache_of(kind, B, Hkv, Nk, D, gen, page_size, seed) for seed in (0, 0))
    qw, kw = weights_of(D, gen, True)
    inv = frequencies(D)
    pos = torch.randint(0, 10 ** 6, (B, Nq), generator=gen, dtype=torch.int32) if given else None
    seq = None if lens is None else torch.tensor(lens, dtype=torch.int32).cuda()
    print(f"[case] {kind} B{B} Nq{Nq} Nk{Nk} pages of {page_size}", flush=True)
    qo, ko, vo = binding.swaa_qk_norm_rope(gq, gk, inv.cuda(), positions=gpu(pos), q_weight=qw.cuda(), k_weight=kw.cuda(), v=gv,
                                           k_out=kc.view, v_out=vc.view, seq_lens=seq, block_table=kc.table,
                                           max_seqlen_k=Nk if kind == "paged" else None)
    assert ko is kc.view and vo is vc.view
    want_k, want_v, size = kc.data.double(), vc.data.clone(), torch.zeros_like(kc.data, dtype=torch.float64)
    for b, n in enumerate(lens or [Nk] * B):
        rows = torch.arange(n - Nq, n)
        at = rows if pos is None else pos[b]
        close(qo[b], *ref.norm_rope(parts[0][b], qw, at, inv, 1e-6, False), torch.bfloat16, f"q of {b}")
        y, s = ref.norm_rope(parts[1][b], kw, at, inv, 1e-6, False)
        there = (rows >= 0) & (rows < Nk)  # (what the cache has no row for is not written)
        if there.any():
            first = int(rows[there][0])
            kc.put(want_k, b, first, y[:, there])
            kc.put(size, b, first, s[:, there])
            vc.put(want_v, b, first, parts[2][b][:, there])
    close(kc.gpu, want_k, size, torch.bfloat16, "cache")  # (rows of others: size 0, and what stood there)
    untouched = size.sum(-1) == 0
    assert torch.equal(kc.gpu.cpu()[untouched], kc.data[untouched])
    assert torch.equal(vc.gpu.cpu(), want_v)


def Cache_of(kind, B, H, Nk, D, gen, page_size, seed):
    return ref.Cache(kind, B, H, Nk, D, torch.bfloat16, torch.Generator().manual_seed(Nk + page_size + seed), page_size)


@pytest.mark.parametrize("stated", ["rows", "none", "fewer"])
@pytest.mark.parametrize("paged", [True, False])
def test_packed_batches(paged, stated):
    gen = torch.Generator().manual_seed(11)
    Hq, Hkv, D = 6, 3, 64
    new, lens = [3, 0, 40, 1, 0, 25, 9], [10, 0, 40, 33, 5, 20, 9]  # the sixth has more rows than keys: its first 20 count
    Nq, Nk = max(new), max(lens)
    T = sum(new)
    x = torch.randn(T, Hq + 2 * Hkv, D, generator=gen).half()
    q, k, v = (t.permute(1, 0, 2) for t in (x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]))
    on = x.cuda()
    gq, gk, gv = (t.permute(1, 0, 2) for t in (on[:, :Hq], on[:, Hq:Hq + Hkv], on[:, Hq + Hkv:]))
    cu = lambda n: torch.tensor([sum(n[:i]) for i in range(len(n) + 1)], dtype=torch.int32)  # noqa: E731
    cu_q, cu_k = cu(new), cu(lens)
    inv = frequencies(32)
    if paged:
        kc, vc = (ref.Cache("paged", len(new), Hkv, Nk, D, torch.float16, torch.Generator().manual_seed(5)) for _ in range(2))
        kd, vd, kg, vg = kc.data, vc.data, kc.view, vc.view
    else:
        kd, vd = (torch.randn(Hkv, sum(lens), D, generator=gen).half() for _ in range(2))
        kg, vg = kd.cuda(), vd.cuda()
    total = {"rows": None, "none": 0, "fewer": T - 9}[stated]
    q_start = torch.randn(Hq, T, D, generator=gen).half()
    qo = q_start.cuda()
    binding.swaa_qk_norm_rope(gq, gk, inv.cuda(), v=gv, q_out=qo, k_out=kg, v_out=vg, cu_seqlens_q=cu_q.cuda(), cu_seqlens_k=cu_k.cuda(),
                              max_seqlen_q=Nq, max_seqlen_k=Nk, block_table=kc.table if paged else None, total_rows_q=total)
    want_q, size_q, want_k, size_k, want_v = q_start.double(), torch.zeros(Hq, T, D, dtype=torch.float64), kd.double(), torch.zeros_like(kd, dtype=torch.float64), vd.clone()
    for b, (m, n) in enumerate(ref.sequences(Nq, Nk, new, lens)):
        if stated == "fewer" and b == 6:
            continue
        rows = slice(int(cu_q[b]), int(cu_q[b]) + m)
        at = torch.arange(n - m, n)
        want_q[:, rows], size_q[:, rows] = ref.norm_rope(q[:, rows], None, at, inv, 1e-6, False)
        y, s = ref.norm_rope(k[:, rows], None, at, inv, 1e-6, False)
        if paged:
            kc.put(want_k, b, n - m, y), kc.put(size_k, b, n - m, s), vc.put(want_v, b, n - m, v[:, rows])
        else:
            to = slice(int(cu_k[b]) + n - m, int(cu_k[b]) + n)
            want_k[:, to], size_k[:, to], want_v[:, to] = y, s, v[:, rows]
    close(qo, want_q, size_q, torch.float16, "packed q")
    close(kc.gpu if paged else kg, want_k, size_k, torch.float16, "packed k")
    assert torch.equal((vc.gpu if paged else vg).cpu(), want_v)


def test_rows_of_pages_outside_the_cache_are_not_written():
    gen = torch.Generator().manual_seed(2)
    kc, vc = (ref.Cache("paged", 3, 2, 32, 64, torch.bfloat16, torch.Generator().manual_seed(1)) for _ in range(2))
    pages = kc.data.shape[0]
    kc.host_table[0, 1], kc.host_table[1, 1] = pages, -1
    q, k = torch.randn(3, 4, 1, 64, generator=gen).bfloat16().cuda(), torch.randn(3, 2, 1, 64, generator=gen).bfloat16().cuda()
    binding.swaa_qk_norm_rope(q, k, v=k, k_out=kc.view, v_out=vc.view, seq_lens=torch.tensor([32, 20, 18], dtype=torch.int32).cuda(),
                              block_table=kc.host_table.cuda(), max_seqlen_k=32)
    want = kc.data.clone()
    want[int(kc.host_table[2, 1]), 1] = k[2, :, 0].cpu()
    assert torch.equal(kc.gpu.cpu(), want) and torch.equal(vc.gpu.cpu(), want)


@pytest.mark.parametrize("fmt", ["bf16", "fp16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_gradients(shape, fmt):
    D, R, norm, interleaved, Hq, Hkv, B, N = shape
    gen = torch.Generator().manual_seed(hash(shape) % 1000 + 1)
    dtype = DTYPES[fmt]
    print(f"[case] gradients {shape} {fmt}", flush=True)
    qkv = (2 * torch.randn(B, N, Hq + Hkv, D, generator=gen)).to(dtype)
    q, k = qkv[:, :, :Hq].permute(0, 2, 1, 3), qkv[:, :, Hq:].permute(0, 2, 1, 3)
    dq, dk = (torch.randn(B, H, N, D, generator=gen).to(dtype) for H in (Hq, Hkv))
    qw, kw = weights_of(D, gen, norm)
    inv = frequencies(R)
    pos = torch.randint(0, 5000, (B, N), generator=gen, dtype=torch.int32) if N % 2 else None
    at = torch.arange(N) if pos is None else pos[:, None]
    on = qkv.cuda()
    call = lambda **kw_: binding.swaa_qk_norm_rope_bwd(  # noqa: E731
        dq.cuda(), dk.cuda(), on[:, :, :Hq].permute(0, 2, 1, 3), on[:, :, Hq:].permute(0, 2, 1, 3), gpu(inv), gpu(pos), gpu(qw), gpu(kw),
        interleaved=interleaved, **kw_)
    got = call()
    for name, dx, dw, dy, x, w in (("q", got[0], got[2], dq, q, qw), ("k", got[1], got[3], dk, k, kw)):
        want, want_w, size, size_w = ref.norm_rope_bwd(dy, x, w, at, inv, 1e-6, interleaved)
        close(dx, want, size, dtype, f"d{name}")
        if norm:
            bound = (2.0 ** -19 + 2.0 ** -24 * B * N * x.shape[1]) * size_w
            assert ((dw.cpu().double() - want_w).abs() <= bound).all()
        else:
            assert dw is None
    again = call()
    assert all(a is None or torch.equal(a, b) for a, b in zip(got, again))  # bit for bit


def test_gradients_against_differences():
    gen = torch.Generator().manual_seed(8)
    B, H, N, D = 1, 2, 3, 64
    x = torch.randn(B, H, N, D, generator=gen).half()
    dy = torch.randn(B, H, N, D, generator=gen).half()
    w = 1 + 0.2 * torch.randn(D, generator=gen)
    inv, pos = frequencies(D), torch.arange(N)
    dx, _, dw, _ = binding.swaa_qk_norm_rope_bwd(dy.cuda(), dy.cuda(), x.cuda(), x.cuda(), inv.cuda(), q_weight=w.cuda(), k_weight=w.cuda())
    loss = lambda x, w: (ref.norm_rope(x, w, pos, inv, 1e-6, False)[0] * dy.double()).sum()  # noqa: E731
    h = 1e-4  # the central difference is off by h^2 / 6 of a third derivative of order 10, far below fp16's half step
    for at in ((0, 0, 0, 0), (0, 1, 2, 63), (0, 0, 1, 31), (0, 1, 0, 32)):
        e = torch.zeros_like(x, dtype=torch.float64)
        e[at] = h
        want = (loss(x.double() + e, w) - loss(x.double() - e, w)).item() / (2 * h)
        assert abs(dx[at].item() - want) <= 2.0 ** -11 * abs(want) + 1e-4
    for d in (0, 17, 63):
        e = torch.zeros(D, dtype=torch.float64)
        e[d] = h
        want = (loss(x, w.double() + e) - loss(x, w.double() - e)).item() / (2 * h)
        assert abs(dw[d].item() - want) <= 1e-4 * max(1.0, abs(want))


def test_gradients_in_place_and_in_the_projections_order():
    gen = torch.Generator().manual_seed(9)
    B, N, Hq, Hkv, D = 2, 70, 4, 2, 128
    qkv = torch.randn(B, N, Hq + 2 * Hkv, D, generator=gen).bfloat16().cuda()
    q, k = qkv[:, :, :Hq].permute(0, 2, 1, 3), qkv[:, :, Hq:Hq + Hkv].permute(0, 2, 1, 3)
    dq, dk = torch.randn(B, Hq, N, D, generator=gen).bfloat16().cuda(), torch.randn(B, Hkv, N, D, generator=gen).bfloat16().cuda()
    w, inv = torch.ones(D).cuda(), frequencies(D).cuda()
    want = binding.swaa_qk_norm_rope_bwd(dq, dk, q, k, inv, q_weight=w, k_weight=w)
    d_qkv = torch.zeros_like(qkv)
    views = d_qkv[:, :, :Hq].permute(0, 2, 1, 3), d_qkv[:, :, Hq:Hq + Hkv].permute(0, 2, 1, 3)
    got = binding.swaa_qk_norm_rope_bwd(dq, dk, q, k, inv, q_weight=w, k_weight=w, dq=views[0], dk=views[1])
    assert got[0] is views[0] and all(torch.equal(a, b) for a, b in zip(got, want))
    assert (d_qkv[:, :, Hq + Hkv:] == 0).all()
    here = binding.swaa_qk_norm_rope_bwd(dq, dk, q, k, inv, q_weight=w, k_weight=w, dq=dq, dk=dk)
    assert here[0] is dq and all(torch.equal(a, b) for a, b in zip(here, want))


def test_many_rows():
    """Past one round of workgroups, sums of weights' gradients over many of them."""
    gen = torch.Generator(device="cuda").manual_seed(10)
    B, N, Hq, Hkv, D = 1, 20011, 4, 1, 128
    q, k, dq, dk = (torch.randn(B, H, N, D, generator=gen, device="cuda").bfloat16() for H in (Hq, Hkv, Hq, Hkv))
    w, inv = torch.ones(D), frequencies(D)
    qo, ko, _ = binding.swaa_qk_norm_rope(q, k, inv.cuda(), q_weight=w.cuda(), k_weight=w.cuda())
    got = binding.swaa_qk_norm_rope_bwd(dq, dk, q, k, inv.cuda(), q_weight=w.cuda(), k_weight=w.cuda())
    for out, x, dy, dx, dw in ((qo, q, dq, got[0], got[2]), (ko, k, dk, got[1], got[3])):
        close(out, *ref.norm_rope(x.cpu(), w, torch.arange(N), inv, 1e-6, False), torch.bfloat16, "many rows")
        want, want_w, size, size_w = ref.norm_rope_bwd(dy.cpu(), x.cpu(), w, torch.arange(N), inv, 1e-6, False)
        close(dx, want, size, torch.bfloat16, "many rows' gradients")
        # (a lane adds up at most the rows of a workgroup's tiles, 16 at a time; then 64 workgroups' sums, and 16 of those)
        assert ((dw.cpu().double() - want_w).abs() <= (2.0 ** -19 + 2.0 ** -24 * 400) * size_w).all()
