"""swaa_attn_key_weights against its definition in 64 bits.  The bound of every key's weight comes with the reference
(cache_ops_ref.key_weights): fp32 scores, exponents and sums, term by term."""
import math

import pytest
import torch

import cache_ops_ref as ref
from paper_2512_10411_amd import binding

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def check(got, want, bound, tag):
    worst = ((got.cpu().double() - want).abs() / bound).max().item()
    print(f"[key_weights] {tag}: {worst:.3f} of the bound", flush=True)
    assert worst <= 1.0, (tag, worst)


# B, Hq, Hkv, Nq, Nk, D, window, n_sink, n_prompt
FIXED = [
    (1, 4, 1, 1, 1, 128, 1, 0, None), (2, 8, 2, 1, 700, 128, 10 ** 9, 0, None), (1, 5, 1, 3, 257, 128, 100, 4, None),
    (2, 4, 2, 65, 65, 128, 20, 0, None), (1, 8, 2, 300, 300, 128, 64, 10, None), (1, 8, 8, 513, 513, 128, 10 ** 9, 0, None),
    (1, 4, 2, 400, 400, 128, 30, 5, 250), (1, 2, 1, 200, 1000, 128, 90, 300, 900), (1, 2, 1, 600, 600, 128, 1, 0, 599),
    (1, 2, 1, 600, 600, 128, 17, 0, 0), (3, 7, 1, 33, 290, 64, 50, 3, None), (1, 4, 2, 100, 333, 32, 10 ** 9, 0, None),
    (1, 2, 2, 150, 150, 96, 40, 1, None), (1, 3, 1, 90, 310, 160, 10 ** 9, 0, None), (1, 2, 1, 70, 270, 192, 33, 2, 300),
    (1, 2, 1, 64, 256, 224, 10 ** 9, 0, None), (1, 4, 2, 130, 520, 256, 200, 600, None), (1, 32, 8, 16, 3000, 128, 1024, 4, None),
    (1, 16, 1, 1500, 1500, 128, 700, 4, 1400),
]


@pytest.mark.parametrize("fmt", ["bf16", "fp16"])
@pytest.mark.parametrize("shape", FIXED)
def test_sequences_of_one_length(shape, fmt):
    B, Hq, Hkv, Nq, Nk, D, window, n_sink, n_prompt = shape
    print(f"[case] {shape} {fmt}", flush=True)
    gen = torch.Generator().manual_seed(Nq + Nk + D)
    q = torch.randn(B, Nq, Hq, D, generator=gen).to(DTYPES[fmt]).permute(0, 2, 1, 3)  # (strided, as a projection leaves it)
    k = torch.randn(B, Hkv, Nk, D, generator=gen).to(DTYPES[fmt])
    scale = 1.3 / math.sqrt(D)
    seen = ref.visible(Nq, Nk, window, n_sink, 10 ** 9 if n_prompt is None else n_prompt)
    lse = torch.stack([ref.lse_of(q[b], k[b], scale, seen) for b in range(B)]).float()
    got = binding.swaa_attn_key_weights(q.cuda(), k.cuda(), lse.cuda(), window, n_sink, n_prompt, scale)
    assert got.shape == (B, Hkv, Nk)
    old = torch.rand(B, Hkv, Nk + 3, generator=gen)
    wide = old.cuda()
    binding.swaa_attn_key_weights(q.cuda(), k.cuda(), lse.cuda(), window, n_sink, n_prompt, scale, weights=wide, decay=0.75)
    for b in range(B):
        want, bound = ref.key_weights(q[b], k[b], lse[b], scale, seen)
        check(got[b], want, bound, f"{shape} {fmt}")
        summed = want + 0.75 * old[b, :, :Nk].double()
        check(wide[b, :, :Nk], summed, bound + 2.0 ** -23 * (summed + want), "summed up")
    assert torch.equal(wide[:, :, Nk:].cpu(), old[:, :, Nk:])
    # what the rows give in all: one each and head
    assert abs(got.sum().item() - B * Hq * Nq) <= 1e-3 * B * Hq * Nq


@pytest.mark.parametrize("page_size", [16, 5])
@pytest.mark.parametrize("kind,Nq,lens", [("paged", 1, [1, 300, 777, 64, 2]), ("dense", 2, [2, 900, 256, 257, 511]),
                                          ("rows", 1, [1000, 1, 1, 513, 30]), ("paged", 40, [40, 45, 600, 500, 99])])
def test_sequences_of_different_lengths(kind, Nq, lens, page_size):
    if kind != "paged" and page_size != 16:
        pytest.skip("pages of paged caches only")
    gen = torch.Generator().manual_seed(sum(lens))
    B, Hq, Hkv, D, Nk, window, n_sink = len(lens), 8, 2, 128, max(lens) + 5, 200, 3
    cache = ref.Cache(kind, B, Hkv, Nk, D, torch.float16, gen, page_size)
    q = torch.randn(B, Hq, Nq, D, generator=gen).half()
    old = torch.rand(B, Hkv, Nk, generator=gen)
    prompts = torch.tensor([n // 2 if i % 2 else 10 ** 6 for i, n in enumerate(lens)], dtype=torch.int32)
    scale, lse, wants = 1 / math.sqrt(D), torch.empty(B, Hq, Nq), []
    for b, n in enumerate(lens):
        seen = ref.visible(Nq, n, window, n_sink, int(prompts[b]))
        lse[b] = ref.lse_of(q[b], cache.rows(b, n), scale, seen)
        wants.append(ref.key_weights(q[b], cache.rows(b, n), lse[b], scale, seen))
    got = binding.swaa_attn_key_weights(q.cuda(), cache.view, lse.cuda(), window, n_sink, scale=scale, weights=old.cuda(), decay=1.0,
                                        seq_lens=torch.tensor(lens, dtype=torch.int32).cuda(), block_table=cache.table,
                                        max_seqlen_k=Nk, n_prompts=prompts.cuda())
    new = binding.swaa_attn_key_weights(q.cuda(), cache.view, lse.cuda(), window, n_sink, scale=scale,
                                        seq_lens=torch.tensor(lens, dtype=torch.int32).cuda(), block_table=cache.table,
                                        max_seqlen_k=Nk, n_prompts=prompts.cuda())
    for b, (want, bound) in enumerate(wants):
        n = lens[b]
        summed = want + old[b, :, :n].double()
        check(got[b, :, :n], summed, bound + 2.0 ** -23 * (summed + want), f"{kind} {n}")
        check(new[b, :, :n], want, bound, f"{kind} {n}, new")
        assert torch.equal(got[b, :, n:].cpu(), old[b, :, n:]) and (new[b, :, n:] == 0).all()


@pytest.mark.parametrize("paged", [False, True])
def test_packed_batches(paged):
    gen = torch.Generator().manual_seed(21)
    Hq, Hkv, D, window, n_sink, scale = 6, 2, 128, 60, 2, 0.1
    new, lens = [5, 0, 300, 1, 0, 30, 64], [600, 0, 300, 513, 9, 20, 64]  # the sixth: more rows than keys, its first 20 count
    B, Nq, Nk = len(new), max(new), max(lens)
    cu = lambda n: torch.tensor([sum(n[:i]) for i in range(len(n) + 1)], dtype=torch.int32)  # noqa: E731
    cu_q, cu_k = cu(new), cu(lens)
    q = torch.randn(Hq, sum(new), D, generator=gen).bfloat16()
    if paged:
        cache = ref.Cache("paged", B, Hkv, Nk, D, torch.bfloat16, gen)
        rows, view = cache.rows, cache.view
    else:
        k = torch.randn(Hkv, sum(lens), D, generator=gen).bfloat16()
        rows, view = (lambda b, n: k[:, int(cu_k[b]):int(cu_k[b]) + n]), k.cuda()
    lse = torch.full((Hq, sum(new)), float("nan"))  # (rows that do not count: whatever)
    old = torch.rand(B, Hkv, Nk, generator=gen)
    wants = []
    for b, (m, n) in enumerate(ref.sequences(Nq, Nk, new, lens)):
        at = slice(int(cu_q[b]), int(cu_q[b]) + m)
        seen = ref.visible(m, n, window, n_sink, 10 ** 9)
        if m:
            lse[:, at] = ref.lse_of(q[:, at], rows(b, n), scale, seen).float()
            wants.append(ref.key_weights(q[:, at], rows(b, n), lse[:, at], scale, seen))
        else:
            wants.append((torch.zeros(Hkv, n, dtype=torch.float64), torch.full((Hkv, n), 1e-30, dtype=torch.float64)))
    got = binding.swaa_attn_key_weights(q.cuda(), view, lse.cuda(), window, n_sink, scale=scale, weights=old.cuda(), decay=0.5,
                                        cu_seqlens_q=cu_q.cuda(), cu_seqlens_k=cu_k.cuda(), max_seqlen_q=Nq, max_seqlen_k=Nk,
                                        block_table=cache.table if paged else None)
    for b, (want, bound) in enumerate(wants):
        n = lens[b]
        if n:
            summed = want + 0.5 * old[b, :, :n].double()
            check(got[b, :, :n], summed, bound + 2.0 ** -23 * (summed + want), f"packed {b}")
        assert torch.equal(got[b, :, n:].cpu(), old[b, :, n:])


@pytest.mark.parametrize("Nq,window", [(1, 10 ** 9), (1, 100), (320, 50), (320, 10 ** 9)])
def test_keys_and_rows_that_do_not_see_each_other(Nq, window):
    """A key that no row sees gets nothing, whatever stands there; rows without a visible finite score give nothing."""
    gen = torch.Generator().manual_seed(31)
    Hq, Hkv, D, Nk, scale = 4, 2, 128, 320, 0.1
    q, k = torch.randn(1, Hq, Nq, D, generator=gen).bfloat16(), torch.randn(1, Hkv, Nk, D, generator=gen).bfloat16()
    seen = ref.visible(Nq, Nk, window, 0, 10 ** 9)
    lse = ref.lse_of(q[0], k[0], scale, seen)[None].float()
    lse[0, 1, Nq // 2] = -math.inf
    want, bound = ref.key_weights(q[0], k[0], lse[0], scale, seen)
    hidden = ~seen.any(0)
    k[0, :, hidden] = float("nan")
    got = binding.swaa_attn_key_weights(q.cuda(), k.cuda(), lse.cuda(), window, 0, scale=scale)[0]
    check(got, want, bound, "hidden keys")
    assert (got[:, hidden.cuda()] == 0).all()
    # an infinite key spoils no other key's weight, and a stale weight that is not a number is not read with decay 0
    seen_key = int((~hidden).nonzero()[0])
    k[0, 0, seen_key, 0] = math.inf
    stale = torch.full((1, Hkv, Nk), float("nan")).cuda()
    got = binding.swaa_attn_key_weights(q.cuda(), k.cuda(), lse.cuda(), window, 0, scale=scale, weights=stale)[0].cpu()
    others = torch.arange(Nk) != seen_key
    check(got[1], want[1], bound[1], "the other head")
    check(got[0, others], want[0, others], bound[0, others], "other keys")


def test_the_same_bits_again_and_with_a_workspace_of_the_callers():
    gen = torch.Generator(device="cuda").manual_seed(41)
    q, k = torch.randn(1, 8, 3001, 128, generator=gen, device="cuda").bfloat16(), torch.randn(1, 2, 3001, 128, generator=gen, device="cuda").bfloat16()
    _, lse = binding.swaa_attn_fwd(q, torch.clone(k), k, 3001, 0)
    need = binding.swaa_attn_key_weights_workspace_bytes(1, 8, 2, 3001, 3001, 128, 3001, 0)
    assert need > 0
    first = binding.swaa_attn_key_weights(q, k, lse, 3001, 0)
    ws = torch.full((need,), 0xff, dtype=torch.uint8, device="cuda")
    for _ in range(2):
        assert torch.equal(first, binding.swaa_attn_key_weights(q, k, lse, 3001, 0, workspace=ws))
    # the attention's own log-sum-exp: every row gives 1
    assert abs(first.sum().item() / (8 * 3001) - 1) < 1e-4


def test_against_the_64_bit_definition_on_many_rows():
    gen = torch.Generator().manual_seed(42)
    Hq, Hkv, N, D, scale, window, n_sink = 2, 1, 5000, 64, 0.125, 900, 4
    q, k = torch.randn(1, Hq, N, D, generator=gen).bfloat16(), torch.randn(1, Hkv, N, D, generator=gen).bfloat16()
    seen = ref.visible(N, N, window, n_sink, 10 ** 9)
    lse = ref.lse_of(q[0], k[0], scale, seen)[None].float()
    want, bound = ref.key_weights(q[0], k[0], lse[0], scale, seen)
    check(binding.swaa_attn_key_weights(q.cuda(), k.cuda(), lse.cuda(), window, n_sink, scale=scale)[0], want, bound, "many rows")


def test_sequences_that_pad_a_batch():
    """Lengths of 0, below the number of rows and beyond the cache: no rows, or as many keys as there are."""
    gen = torch.Generator().manual_seed(51)
    Hq, Hkv, D, Nq, Nk = 4, 2, 64, 3, 70
    lens, held = [0, 2, -4, 70, 500, 3], [0, 2, 0, 70, 70, 3]
    B = len(lens)
    q, k = torch.randn(B, Hq, Nq, D, generator=gen).half(), torch.randn(B, Hkv, Nk, D, generator=gen).half()
    lse, old = torch.full((B, Hq, Nq), float("nan")), torch.rand(B, Hkv, Nk, generator=gen)
    wants = []
    for b, n in enumerate(held):
        m = Nq if n >= Nq else 0
        seen = ref.visible(m, n, 10 ** 9, 0, 10 ** 9)
        if m:
            lse[b] = ref.lse_of(q[b], k[b, :, :n], 0.125, seen).float()
        wants.append(ref.key_weights(q[b, :, :m], k[b, :, :n], lse[b, :, :m], 0.125, seen))
    got = binding.swaa_attn_key_weights(q.cuda(), k.cuda(), lse.cuda(), 10 ** 9, 0, scale=0.125, weights=old.cuda(), decay=0.5,
                                        seq_lens=torch.tensor(lens, dtype=torch.int32).cuda())
    for b, (want, bound) in enumerate(wants):
        n = held[b]
        summed = want + 0.5 * old[b, :, :n].double()
        if n:
            check(got[b, :, :n], summed, bound + 2.0 ** -23 * (summed + want), f"length {lens[b]}")
        assert torch.equal(got[b, :, n:].cpu(), old[b, :, n:])
