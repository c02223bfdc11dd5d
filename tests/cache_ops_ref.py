"""The cache's operators (norms with rotation, key weights, eviction) from their definitions in 64 bits, on the CPU."""
import math

import torch


def sequences(Nq, Nk, new, lens):
    """[(rows, keys)] of packed sequences."""
    out = []
    for m, n in zip(new, lens):
        m = max(min(m, Nq, n), 0)
        n = max(min(n, Nk), 0)
        out.append((min(m, n), n))
    return out


def pairs_of(D, R, interleaved):
    """Each dimension's frequency, partner and sign of the sine."""
    freq, partner, sign = [0] * D, list(range(D)), [0.0] * D
    for i in range(R // 2):
        a, c = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
        freq[a] = freq[c] = i
        partner[a], partner[c], sign[a], sign[c] = c, a, -1.0, 1.0
    return torch.tensor(freq), torch.tensor(partner), torch.tensor(sign, dtype=torch.float64)


def turn(pos, inv_freq, D, interleaved):
    """cos, sin * sign and partner of every dimension, for positions `pos`."""
    R = 0 if inv_freq is None else 2 * inv_freq.numel()
    freq, partner, sign = pairs_of(D, R, interleaved)
    angle = torch.zeros(*pos.shape, D, dtype=torch.float64)
    if R:
        angle = pos.double()[..., None] * inv_freq.double()[freq] * sign.abs()
    return angle.cos(), angle.sin() * sign, partner


def norm_rope(x, w, pos, inv_freq, eps, interleaved):
    """x [..., rows, D] at positions pos (shaped like its rows): result, and the magnitudes its rounding errors go by."""
    x = x.double()
    n = x if w is None else x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * w.double()
    cos, sin, partner = turn(pos, inv_freq, x.shape[-1], interleaved)
    return n * cos + n[..., partner] * sin, n.abs() + n[..., partner].abs()


def norm_rope_bwd(dy, x, w, pos, inv_freq, eps, interleaved):
    """dx, dw and the magnitudes of the terms that they are sums of."""
    dy, x = dy.double(), x.double()
    cos, sin, partner = turn(pos, inv_freq, x.shape[-1], interleaved)
    g, size = dy * cos - dy[..., partner] * sin, dy.abs() + dy[..., partner].abs()
    if w is None:
        return g, None, size, None
    s = 1.0 / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    w = w.double()
    dx = s * (w * g - x * s * s * (x * w * g).mean(-1, keepdim=True))
    size_x = s * ((w * size).abs() + x.abs() * s * s * (x * w * size).abs().mean(-1, keepdim=True))
    return dx, (g * x * s).flatten(0, -2).sum(0), size_x, (size * (x * s).abs()).flatten(0, -2).sum(0)


def visible(nq, nk, window, n_sink, n_prompt):
    """[nq, nk] truth values: does row r see key j?"""
    pos, j = torch.arange(nk - nq, nk)[:, None], torch.arange(nk)
    return (j <= pos) & ((pos >= n_prompt) | (j > pos - window) | (j < n_sink))


def lse_of(q, k, scale, seen):
    """Log-sum-exp of one sequence, q [Hq, nq, D], k [Hkv, nk, D]."""
    s = torch.matmul(q.double(), k.double().repeat_interleave(q.shape[0] // k.shape[0], 0).transpose(1, 2)) * scale
    return torch.logsumexp(s.masked_fill(~seen, -math.inf), -1)


def key_weights(q, k, lse, scale, seen):
    """Sum over the rows and the heads of a group [Hkv, nk], and a bound on its error: fp32 scores of D products (2^-23 a step, which
    holds for truncating adders, too), 32-bit exponents and exponentials, and fp32 sums."""
    Hq, nq, D = q.shape
    Hkv, nk = k.shape[:2]
    q, kk = q.double(), k.double().repeat_interleave(Hq // Hkv, 0)
    s = torch.matmul(q, kk.transpose(1, 2)) * scale
    size = torch.matmul(q.abs(), kk.abs().transpose(1, 2)) * scale
    lse = lse.double()[..., None]
    p = torch.where(seen & (lse != -math.inf), (s - lse).exp(), 0.0)
    err = torch.where(p > 0, p * 2.0 ** -23 * ((D + 2) * size + 2 * lse.abs() + 8), 0.0)
    group = lambda t: t.unflatten(0, (Hkv, Hq // Hkv)).sum((1, 2))  # noqa: E731
    terms = nq * Hq // Hkv
    return group(p), group(err) + 2.0 ** -23 * terms * group(p) + 1e-30


def evict(weights, n, n_keep, n_sink, n_recent):
    """Rows of one head that stay: weights fp32 [n]."""
    if n <= n_keep:
        return list(range(n))
    order = lambda x: math.inf if math.isnan(x) else x  # noqa: E731
    nan = [math.isnan(float(x)) for x in weights]
    middle = sorted(range(n_sink, n - n_recent), key=lambda j: (not nan[j], -order(float(weights[j])), j))
    return list(range(n_sink)) + sorted(middle[:n_keep - n_sink - n_recent]) + list(range(n - n_recent, n))


class Cache:
    """A cache on the GPU, contiguous or paged, and what it holds, [B][H, n, D]."""

    def __init__(self, kind, B, H, Nk, D, dtype, gen, page_size=16, spare=3):
        self.kind, self.B, self.page_size = kind, B, page_size
        rand = lambda *s: torch.randn(*s, generator=gen).to(dtype)  # noqa: E731
        if kind == "paged":
            per = -(-Nk // page_size)
            self.data = rand(B * per + spare, page_size, H, D)
            order = torch.randperm(B * per + spare, generator=gen)[:B * per].to(torch.int32)
            self.host_table = order.view(B, per)
            self.table = self.host_table.cuda()
            self.gpu = self.data.cuda()
            self.view = self.gpu.permute(0, 2, 1, 3)
        else:
            self.data = rand(B, H, Nk, D) if kind == "dense" else rand(B, Nk, H, D)
            self.gpu = self.data.cuda()
            self.view = self.gpu if kind == "dense" else self.gpu.permute(0, 2, 1, 3)
            self.table = None

    def rows(self, b, n, data=None):
        """[H, n, D] of sequence b, of `data` (on the CPU) or as made."""
        data = self.data if data is None else data
        if self.kind == "paged":
            t = torch.arange(n)
            return data[self.host_table[b].long()[t // self.page_size], t % self.page_size].permute(1, 0, 2)
        return (data[b] if self.kind == "dense" else data[b].permute(1, 0, 2))[:, :n]

    def put(self, data, b, at, rows):
        """Writes rows [H, n, D] to rows at, at + 1, ... of sequence b in `data`."""
        for i in range(rows.shape[1]):
            if self.kind == "paged":
                data[int(self.host_table[b, (at + i) // self.page_size]), (at + i) % self.page_size] = rows[:, i]
            elif self.kind == "dense":
                data[b, :, at + i] = rows[:, i]
            else:
                data[b, at + i] = rows[:, i]
