"""Host-side checks of the cache's operators: refusals (nothing is launched), workspaces, and the reference's own pins.  No GPU."""
import ctypes
import math

import pytest
import torch

import cache_ops_ref as ref
from paper_2512_10411_amd import binding

P = 4096  # a non-null, 16-byte aligned fake address; never dereferenced on these paths


def filled(a, fields, changes):
    for key, val in {**fields, **changes}.items():
        if "." in key:
            t, f = key.split(".")
            setattr(getattr(a, t), f, val)
        else:
            setattr(a, key, val)
    return a


def rows(H, N, D):
    return binding.SwaaTensor(P, H * N * D, N * D, D)


def call(name, a):
    return int(getattr(binding.load_library(), name)(ctypes.byref(a)))


def norm_rope(**kw):
    q, k = rows(4, 64, 128), rows(2, 64, 128)
    return call("swaa_qk_norm_rope", filled(binding.SwaaNormRopeArgs(), dict(
        q=q, k=k, q_out=q, k_out=k, B=2, Hq=4, Hkv=2, D=128, Nq=64, Nk=64, q_weight=P, k_weight=P, eps=1e-6, inv_freq=P, rot_dim=128), kw))


@pytest.mark.parametrize("status,kw", [
    ("NULL", {"q.ptr": None}), ("NULL", {"k_out.ptr": None}), ("NULL", {"v": rows(2, 64, 128)}),  # values without a place for them
    ("NULL", {"k_weight": None}), ("NULL", {"inv_freq": None}), ("NULL", {"cu_seqlens_q": P}),
    ("SHAPE", {"B": 0}), ("SHAPE", {"Nq": 0}), ("SHAPE", {"Nq": 65}), ("SHAPE", {"Hq": 5}), ("SHAPE", {"eps": 0.0}),
    ("SHAPE", {"eps": float("nan")}), ("SHAPE", {"rot_dim": 144}), ("SHAPE", {"rot_dim": -16}), ("SHAPE", {"total_rows_q": -1}),
    ("SHAPE", {"cu_seqlens_q": P, "cu_seqlens_k": P, "seq_lens": P}), ("SHAPE", {"q.stride_n": 64}), ("SHAPE", {"k.stride_h": 4}),
    ("SHAPE", {"q_out.stride_b": 0}), ("SHAPE", {"block_table": P, "page_size": 0, "num_pages": 4, "block_table_stride": 64}),
    ("SHAPE", {"block_table": P, "page_size": 16, "num_pages": 4, "block_table_stride": 3}), ("SHAPE", {"B": 1 << 30, "Nq": 64}),
    ("UNSUPPORTED", {"D": 80}), ("UNSUPPORTED", {"D": 288}), ("UNSUPPORTED", {"rot_dim": 24}), ("UNSUPPORTED", {"dtype": 2}),
    ("ALIGN", {"q.ptr": P + 8}), ("ALIGN", {"v": binding.SwaaTensor(P + 2, 1024, 512, 128), "v_out": rows(2, 64, 128)}),
    ("ALIGN", {"positions": P + 2}), ("ALIGN", {"seq_lens": P + 1}), ("ALIGN", {"q_weight": P + 2, "k_weight": P}),
])
def test_norm_rope_refusals(status, kw):
    assert norm_rope(**kw) == getattr(binding, "SWAA_ERR_" + status)


def norm_rope_bwd(**kw):
    q, k = rows(4, 64, 128), rows(2, 64, 128)
    return call("swaa_qk_norm_rope_bwd", filled(binding.SwaaNormRopeBwdArgs(), dict(
        q=q, k=k, dq_out=q, dk_out=k, dq=q, dk=k, B=2, Hq=4, Hkv=2, D=128, N=64, q_weight=P, k_weight=P, eps=1e-6, inv_freq=P,
        rot_dim=128, dq_weight=P, dk_weight=P, workspace=P, workspace_bytes=1 << 30), kw))


@pytest.mark.parametrize("status,kw", [
    ("NULL", {"dq.ptr": None}), ("NULL", {"dk_out.ptr": None}), ("NULL", {"dk_weight": None}), ("NULL", {"q_weight": None}),
    ("SHAPE", {"N": 0}), ("SHAPE", {"Hkv": 3}), ("SHAPE", {"eps": -1.0}), ("SHAPE", {"dq.stride_n": 100}), ("UNSUPPORTED", {"D": 48}),
    ("UNSUPPORTED", {"rot_dim": 8}), ("ALIGN", {"dq_weight": P + 2}), ("ALIGN", {"dk.ptr": P + 4}), ("WORKSPACE", {"workspace": None}),
    ("WORKSPACE", {"workspace": P + 8}), ("WORKSPACE", {"workspace_bytes": 100}),
])
def test_norm_rope_bwd_refusals(status, kw):
    assert norm_rope_bwd(**kw) == getattr(binding, "SWAA_ERR_" + status)


def key_weights(**kw):
    return call("swaa_attn_key_weights", filled(binding.SwaaKeyWeightsArgs(), dict(
        q=rows(4, 64, 128), k=rows(2, 100, 128), lse=P, lse_stride_b=256, lse_stride_h=64, weights=P, weights_stride_b=200,
        weights_stride_h=100, B=2, Hq=4, Hkv=2, D=128, Nq=64, Nk=100, window=10, n_sink=0, n_prompt=1 << 30, scale=0.1, decay=0.0,
        workspace=P, workspace_bytes=1 << 30), kw))


@pytest.mark.parametrize("status,kw", [
    ("NULL", {"lse": None}), ("NULL", {"weights": None}), ("NULL", {"k.ptr": None}), ("NULL", {"cu_seqlens_k": P}),
    ("SHAPE", {"Nq": 101}), ("SHAPE", {"window": 0}), ("SHAPE", {"n_sink": -1}), ("SHAPE", {"n_prompt": -1}), ("SHAPE", {"scale": 0.0}),
    ("SHAPE", {"decay": -0.5}), ("SHAPE", {"decay": float("nan")}), ("SHAPE", {"decay": float("inf")}), ("SHAPE", {"weights_stride_h": 99}),
    ("SHAPE", {"weights_stride_b": 0}), ("SHAPE", {"lse_stride_h": -1}), ("UNSUPPORTED", {"D": 80}), ("UNSUPPORTED", {"dtype": 5}),
    ("ALIGN", {"weights": P + 2}), ("ALIGN", {"k.ptr": P + 8}), ("ALIGN", {"n_prompts": P + 3}),
])
def test_key_weights_refusals(status, kw):
    assert key_weights(**kw) == getattr(binding, "SWAA_ERR_" + status)


def test_key_weights_workspace():
    a = dict(Nq=4000, Nk=4000, window=4000, weights_stride_b=8000, weights_stride_h=4000, q=rows(4, 4000, 128), k=rows(2, 4000, 128))
    need = binding.swaa_attn_key_weights_workspace_bytes(2, 4, 2, 4000, 4000, 128, 4000, 0)
    assert need > 0
    assert key_weights(workspace_bytes=need - 1, **a) == binding.SWAA_ERR_WORKSPACE
    assert key_weights(workspace=None, **a) == binding.SWAA_ERR_WORKSPACE
    assert binding.swaa_attn_key_weights_workspace_bytes(1, 32, 8, 1, 131072, 128, 131072, 4) == 0  # a new token: nothing to share out
    for shape in ((1, 32, 8, 131072, 131072, 128), (64, 40, 8, 2048, 131072, 128), (1, 8, 8, 1 << 20, 1 << 20, 64)):
        for mask in ((1 << 30, 0), (8192, 4), (1, 0)):
            assert binding.swaa_attn_key_weights_workspace_bytes(*shape, *mask) < 16 << 20
    for bad in ((1, 3, 2, 1, 1, 128), (1, 2, 2, 2, 1, 128), (0, 2, 2, 1, 1, 128), (1, 2, 2, 1, 1, 100)):
        with pytest.raises(binding.SwaaError):
            binding.swaa_attn_key_weights_workspace_bytes(*bad, 10, 0)


def test_norm_rope_bwd_workspace():
    assert 0 < binding.swaa_qk_norm_rope_bwd_workspace_bytes(1, 32, 8, 131072, 128) <= 16 << 20  # it does not grow with the tokens
    with pytest.raises(binding.SwaaError):
        binding.swaa_qk_norm_rope_bwd_workspace_bytes(1, 32, 8, 0, 128)


def evict(**kw):
    return call("swaa_cache_evict", filled(binding.SwaaEvictArgs(), dict(
        k=rows(2, 100, 128), v=rows(2, 100, 128), weights=P, weights_stride_b=200, weights_stride_h=100, kept=P, B=2, Hkv=2, D=128, Nk=100,
        n_keep=50, n_sink=4, n_recent=10), kw))


@pytest.mark.parametrize("status,kw", [
    ("NULL", {"k.ptr": None}), ("NULL", {"kept": None}), ("NULL", {"weights": None}), ("SHAPE", {"Nk": 0}), ("SHAPE", {"n_keep": 0}),
    ("SHAPE", {"n_sink": -1}), ("SHAPE", {"n_recent": -1}), ("SHAPE", {"n_sink": 41}), ("SHAPE", {"weights_stride_h": 90}),
    ("SHAPE", {"block_table": P, "page_size": 16, "num_pages": 0, "block_table_stride": 7}),
    ("SHAPE", {"block_table": P, "page_size": 16, "num_pages": 5, "block_table_stride": 6}), ("SHAPE", {"v.stride_n": 127}),
    ("UNSUPPORTED", {"D": 72}), ("ALIGN", {"v.ptr": P + 8}), ("ALIGN", {"new_lens": P + 2}), ("ALIGN", {"kept": P + 1}),
])
def test_evict_refusals(status, kw):
    assert evict(**kw) == getattr(binding, "SWAA_ERR_" + status)


def test_evict_has_no_more_pairs_than_a_launch_can_move():
    assert binding.swaa_cache_evict_workspace_bytes(30000, 8, 64, 128) == 0
    for B, D in ((30841, 128), (1 << 24, 32)):
        assert evict(B=B, Hkv=8, D=D, Nk=64) == binding.SWAA_ERR_SHAPE


def test_evict_workspace():
    need = binding.swaa_cache_evict_workspace_bytes(2, 2, 100000, 128)
    long = dict(Nk=100000, weights_stride_b=200000, weights_stride_h=100000, k=rows(2, 100000, 128), v=rows(2, 100000, 128))
    assert need > 0 and evict(workspace=P, workspace_bytes=need - 1, **long) == binding.SWAA_ERR_WORKSPACE
    assert evict(workspace=P + 8, workspace_bytes=need, **long) == binding.SWAA_ERR_WORKSPACE
    assert binding.swaa_cache_evict_workspace_bytes(64, 8, 131072, 128) == binding.swaa_cache_evict_workspace_bytes(1, 8, 4096, 128) == 0
    for bad in ((0, 2, 100, 128), (1, 2, 0, 128), (1, 2, 100, 100), (1, 2, (1 << 28) + 1, 128)):
        with pytest.raises(binding.SwaaError):
            binding.swaa_cache_evict_workspace_bytes(*bad)


def test_a_missing_argument_block():
    for name in ("swaa_qk_norm_rope", "swaa_qk_norm_rope_bwd", "swaa_attn_key_weights", "swaa_cache_evict",
                 "swaa_qk_norm_rope_bwd_workspace_bytes", "swaa_attn_key_weights_workspace_bytes", "swaa_cache_evict_workspace_bytes"):
        assert getattr(binding.load_library(), name)(None) == binding.SWAA_ERR_NULL


def test_the_binding_refuses_tensors_of_the_cpu():
    x, f = torch.zeros(1, 2, 4, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 4)
    for bad in (lambda: binding.swaa_qk_norm_rope(x, x), lambda: binding.swaa_qk_norm_rope_bwd(x, x, x, x),
                lambda: binding.swaa_attn_key_weights(x, x, f, 4, 0), lambda: binding.swaa_cache_evict(x, x, f, 2, 0, 0)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        binding.swaa_qk_norm_rope(x.float(), x.float())


# ---- the reference, pinned by hand ----
def test_reference_rotation_by_hand():
    x = torch.tensor([[3.0, 4.0] + [0.0] * 14])
    inv = torch.tensor([0.5] + [0.0] * 7)
    y, _ = ref.norm_rope(x, None, torch.tensor([2]), inv, 1e-6, True)
    c, s = math.cos(1.0), math.sin(1.0)
    assert y[0, :2].tolist() == pytest.approx([3 * c - 4 * s, 4 * c + 3 * s])
    x = torch.zeros(1, 16)
    x[0, 0], x[0, 8] = 3.0, 4.0
    y, _ = ref.norm_rope(x, torch.full((16,), 2.0), torch.tensor([2]), inv, 0.0, False)
    n = 2 / math.sqrt(25 / 16)
    assert [y[0, 0].item(), y[0, 8].item()] == pytest.approx([n * (3 * c - 4 * s), n * (4 * c + 3 * s)])


def test_reference_gradients_by_autograd():
    gen = torch.Generator().manual_seed(1)
    x = torch.randn(2, 3, 32, generator=gen, dtype=torch.float64, requires_grad=True)
    w = torch.rand(32, generator=gen, dtype=torch.float64).requires_grad_()
    dy, inv, pos = torch.randn(2, 3, 32, generator=gen, dtype=torch.float64), torch.rand(8, generator=gen), torch.arange(3)
    for interleaved in (False, True):
        y, _ = ref.norm_rope(x, w, pos, inv, 1e-3, interleaved)
        want = torch.autograd.grad(y, (x, w), dy)
        dx, dw, _, _ = ref.norm_rope_bwd(dy, x.detach(), w.detach(), pos, inv, 1e-3, interleaved)
        assert torch.allclose(dx, want[0], rtol=1e-12, atol=1e-12) and torch.allclose(dw, want[1], rtol=1e-12, atol=1e-12)


def test_reference_weights_and_eviction_by_hand():
    seen = ref.visible(3, 3, 1, 1, 10)  # each row its own key, and key 0
    q, k = torch.zeros(1, 3, 32), torch.zeros(1, 3, 32)
    lse = ref.lse_of(q, k, 1.0, seen)
    assert ref.key_weights(q, k, lse, 1.0, seen)[0].tolist() == [pytest.approx([2.0, 0.5, 0.5])]
    w = torch.tensor([0.0, 5.0, 1.0, float("nan"), 1.0, 0.0])
    assert ref.evict(w, 6, 3, 1, 1) == [0, 3, 5] and ref.evict(w, 6, 4, 1, 1) == [0, 1, 3, 5]
    assert ref.evict(w, 6, 3, 0, 0) == [1, 2, 3] and ref.evict(w, 6, 6, 0, 0) == list(range(6))
