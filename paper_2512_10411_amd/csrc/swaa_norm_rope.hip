// RMS norms of the heads of queries and keys with the position rotation in the same pass, forward and backward (gfx950).
//
//   n = x / sqrt(mean(x^2) + eps) * w          y = n rotated in pairs (i, partner of i) by pos * inv_freq[pair]
//
// With the rotation written per element as y_j = n_j C_j + n_p S_j (p: the partner, S_j signed), a row is
// y_j = r (x_j A_j + x_p B_j) with A = w C and B = w_p S: three operations per element, and one sum of squares per row.  The
// backward pass goes through the transposed rotation, g_j = C_j dy_j + S_p dy_p with S_p = -S_j, and the norm:
// dx_j = r (w_j g_j - x_j r^2 mean(x w g)), dw_j = sum over rows of g_j x_j r.
//
// Bound by memory: every element comes in once and goes out once (backward: two in, one out).  32 + 8 heads of 128, bf16: 16384 tokens
// forward 75.6 us (4.4 TB/s; a copy of 128 MB to 2 GB: 8.6 to 4.9), backward 115.4 us (4.4 TB/s, of it 5 us for the sums of the weights'
// gradients); 16 tokens into a cache 6.2 us, a launch's time and the angles.
//   * A row is D / 8 lanes of 16 bytes (rounded up to a power of two); what a lane multiplies by depends on its token and its
//     place in the row only, so a lane keeps both through a loop over the heads: cosines, sines and weights stay in registers.
//   * The angles are taken in 64 bits (positions go beyond what 32 bits resolve), once per token and pair: a workgroup's
//     threads share them through LDS.
#include "swaa_cache_ops.h"

namespace swaa {
namespace {

constexpr int kNThreads = 256;
// Tokens from which on each wave has its own (us of the forward / backward call, 32 + 8 heads of 128, bf16: 128 tokens shared 6.2 / 11.2,
// by wave 6.6 / 11.6; 256: 7.0 / 12.2, 6.4 / 11.6; 1000: 11.2 / 19.2, 9.6 / 16.3).
constexpr int kByWaveTokens = 256;
// Units that a workgroup of those has at least: what it does for its angles has to pay.  Twice as many where there are tiles enough
// to fill the chip all the same (4 units against 8: 300 tokens 6.4 / 11.5, 7.3 / 12.4; 700: 8.1 / 14.6, 7.9 / 13.8; 2000: 15.4 / 22.4,
// 12.2 / 21.4; 1 unit against 4 at 1000: 12.0 / 18.7, 9.5 / 16.1).
constexpr int kLeastUnits = 4;
constexpr int kManyTiles = 32;
// Workgroups that a call should have: what the chip holds at once (1024 against 2048, 3000 tokens: 18.0 / 30.3, 21.2 / 32.4; 8192: 31.4 / 54.0,
// 34.5 / 54.5).
constexpr int kFillWgs = 1024;

template <bool kF16>
__device__ __forceinline__ void unpack(u32x4 raw, float (&x)[8]) {
    if constexpr (kF16) {
        const f16x8 h = __builtin_bit_cast(f16x8, raw);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = (float)h[j];
    } else {
        const bf16x8 h = __builtin_bit_cast(bf16x8, raw);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = (float)h[j];
    }
}
// (one rounding to 16 bits, to nearest even, of a result held in 32: at most half a step)
template <bool kF16>
__device__ __forceinline__ u32x4 pack(const float (&y)[8]) {
    if constexpr (kF16) {
        f16x8 h;
#pragma unroll
        for (int j = 0; j < 8; ++j) h[j] = (_Float16)y[j];
        return __builtin_bit_cast(u32x4, h);
    } else {
        bf16x8 h;
#pragma unroll
        for (int j = 0; j < 8; ++j) h[j] = (__bf16)y[j];
        return __builtin_bit_cast(u32x4, h);
    }
}

template <int kCtrl>
__device__ __forceinline__ float dpp(float x) {
    return __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), kCtrl, 0xf, 0xf, true));
}
// Sum over the kLanes lanes of a row, in all of them.
template <int kLanes>
__device__ __forceinline__ float row_sum(float x) {
    if constexpr (kLanes >= 16) {
        x += dpp<0x128>(x);  // row_ror:8
        x += dpp<0x124>(x);
        x += dpp<0x122>(x);
        x += dpp<0x121>(x);
        if constexpr (kLanes == 32) x += __shfl_xor(x, 16);
    } else {
        x += dpp<0xb1>(x);  // quad_perm [1,0,3,2]
        x += dpp<0x4e>(x);  // quad_perm [2,3,0,1]
        if constexpr (kLanes == 8) x += dpp<0x141>(x);  // row_half_mirror
    }
    return x;
}

// A lane's token.
struct Token {
    int b, row;  // batch entry to take strides of, row along the tensors' row axis
    int pos;
    int of, at;  // its sequence and row in that one's cache
    bool live, cached;  // is there such a token, and has the cache its row?
};
__device__ __forceinline__ Token find_token(const NormRopeParams &p, long long slot) {
    Token t;
    int b = 0, r = 0, nq = 0, nk = 0;
    t.live = slot < p.tokens;
    const int mine = (int)min(slot, p.tokens - 1);
    if (p.by_row) {  // the sequence that holds this row of the packed tensor: as many of the others' ends as lie at or before it
        const int lane = threadIdx.x & 63;
        for (int c0 = 0; c0 < p.seq.B; c0 += 64) {
            const int end = p.seq.cu_q[min(c0 + lane, p.seq.B - 1) + 1], n = min(64, p.seq.B - c0);
            for (int i = 0; i < n; ++i) b += (int)wave_read_lane((unsigned)end, i) <= mine;
            if ((int)wave_read_lane((unsigned)end, n - 1) > (int)wave_read_lane((unsigned)mine, 63)) break;  // (the wave's last token is found)
        }
        t.live = t.live && b < p.seq.B;
        b = min(b, p.seq.B - 1);
        r = mine - p.seq.cu_q[b];
    } else {
        b = (int)fastdiv((unsigned)mine, p.div_nq);
        r = mine - b * p.seq.Nq;
    }
    if (p.seq.seq_lens) {  // (lengths as they are: rows outside the cache -- padding, or a cache that is full -- are not written)
        nq = p.seq.Nq;
        nk = p.seq.seq_lens[b];
    } else {
        sequence(p.seq, b, nq, nk);
    }
    t.live = t.live && r >= 0 && r < nq;
    t.of = b;
    t.b = p.seq.cu_q ? 0 : b;
    t.row = r + (p.seq.cu_q ? p.seq.cu_q[b] : 0);
    t.at = (int)((unsigned)nk - (unsigned)nq + (unsigned)r);
    t.cached = t.live && t.at >= 0 && t.at < p.seq.Nk;
    t.pos = !t.live ? 0 : !p.positions ? t.at : p.positions[p.seq.cu_q ? (long long)t.row : b * (long long)p.seq.Nq + r];
    return t;
}

// The place of a lane in the work: its row slot among the workgroup's, and what that is.
template <int kLanes>
struct Place {
    int chunk, token;        // its 16 bytes of a row, its token of the tile
    int head0, heads;        // of a unit's heads the one it has, and how many those are
    int of_wave;             // its token among those in its wave, whose angles stand at `table`
    float2 *table;
    __device__ __forceinline__ Place(const NormRopeParams &p, float2 *lds) {
        const int slot = (int)threadIdx.x / kLanes, of_group = p.by_wave ? slot % (64 / kLanes) : slot;
        chunk = (int)threadIdx.x % kLanes;
        of_wave = slot & ((1 << p.wave_shift) - 1);
        head0 = of_group >> p.wave_shift;
        heads = (p.by_wave ? 64 / kLanes : kNThreads / kLanes) >> p.wave_shift;
        token = of_wave + (p.by_wave ? ((int)threadIdx.x / 64) << p.wave_shift : 0);
        table = lds + (p.by_wave ? ((int)threadIdx.x / 64) * (p.R / 2) << p.wave_shift : 0);
    }
};

// cos and sin of the tokens of a wave, [pair][token], by the wave for itself or by all four for their common ones: the angle in
// turns in 64 bits, what is left of it behind whole turns in 32.  (Token i of a wave is in the lanes of its row i.)
template <int kLanes>
__device__ __forceinline__ void find_angles(const NormRopeParams &p, int pos, float2 *table) {
    const int thread = p.by_wave ? (int)threadIdx.x % 64 : (int)threadIdx.x, threads = p.by_wave ? 64 : kNThreads;
    const int token = thread & ((1 << p.wave_shift) - 1);
    const double at = (double)__shfl(pos, token * kLanes);
    for (int pair = thread >> p.wave_shift; pair < p.R / 2; pair += threads >> p.wave_shift) {
        const double turns = at * (double)p.inv_freq[pair] * 0.15915494309189533577;
        float s, c;
        sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
        table[(pair << p.wave_shift) + token] = make_float2(c, s);
    }
}

// A lane's rotation: elements 8 chunk .. 8 chunk + 7 of its token's rows.
struct Turn {
    float c[8], s[8];  // y_j = n_j c_j + n_partner s_j
    int partner;       // lane that holds the partners (pairs of halves)
    bool swap;         // (the lanes of a row of 16 and its halves: by an operand of a vector instruction instead of the LDS crossbar)
};
__device__ __forceinline__ Turn lane_turn(const NormRopeParams &p, const float2 *table, int token, int chunk) {
    Turn t;
    const int half = p.R / 16;  // chunks of half the rotated elements
    t.partner = threadIdx.x & 63;
    t.swap = p.R == 128 && p.D == 128;
    if (8 * chunk >= p.R) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            t.c[j] = 1.f;
            t.s[j] = 0.f;
        }
        return t;
    }
    if (p.interleaved) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float2 cs = table[((4 * chunk + j / 2) << p.wave_shift) + token];
            t.c[j] = cs.x;
            t.s[j] = j % 2 ? cs.y : -cs.y;
        }
        return t;
    }
    const bool second = chunk >= half;
    t.partner += second ? -half : half;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float2 cs = table[((8 * (second ? chunk - half : chunk) + j) << p.wave_shift) + token];
        t.c[j] = cs.x;
        t.s[j] = second ? cs.y : -cs.y;
    }
    return t;
}
// The partners of a row's 8 elements, as they stand in memory.
__device__ __forceinline__ u32x4 partners(u32x4 raw, const Turn &t, bool interleaved) {
    u32x4 r;
    if (interleaved) {
#pragma unroll
        for (int j = 0; j < 4; ++j) r[j] = (raw[j] >> 16) | (raw[j] << 16);
    } else if (t.swap) {
#pragma unroll
        for (int j = 0; j < 4; ++j) r[j] = (unsigned)__builtin_amdgcn_update_dpp(0, (int)raw[j], 0x128, 0xf, 0xf, true);  // row_ror:8
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) r[j] = (unsigned)__shfl((int)raw[j], t.partner);
    }
    return r;
}
__device__ __forceinline__ void row_weights(const float *w, int chunk, bool in_row, float (&out)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) out[j] = w && in_row ? w[8 * chunk + j] : 1.f;
}
// (the partners' weights: of the same places in the other half, or the neighbours')
__device__ __forceinline__ void partner_weights(const float *w, const NormRopeParams &p, int chunk, float (&out)[8]) {
    const int half = p.R / 16;
    const bool turns = 8 * chunk < p.R;
    const int base = 8 * (!turns || p.interleaved ? chunk : chunk >= half ? chunk - half : chunk + half);
#pragma unroll
    for (int j = 0; j < 8; ++j) out[j] = w && turns ? w[base + (p.interleaved ? j ^ 1 : j)] : 1.f;
}

// A lane's way through the heads of one tensor, from unit `unit` on: the head of unit u exists while u < end.
struct Heads {
    char *at;
    long long step;  // bytes from unit to unit
    int end;
    __device__ __forceinline__ Heads(const Rows &t, long long offset, int H, int head0, int heads, int first, int unit, bool live) {
        at = t.ptr + 2 * (offset + (head0 + (long long)(unit > first ? unit - first : 0) * heads) * t.sh);
        step = 2 * (long long)heads * t.sh;
        end = live ? first + (H - head0 + heads - 1) / heads : 0;
    }
};

constexpr int kAhead = 4;  // rows of a lane on the way at a time

template <int kLanes, bool kF16>
__global__ __launch_bounds__(kNThreads, 4) void swaa_norm_rope_kernel(const NormRopeParams p) {
    fetch_args<NormRopeParams>();
    extern __shared__ float2 table[];
    const unsigned of_tile = fastdiv(blockIdx.x, p.div_wgs), part = blockIdx.x - of_tile * (unsigned)p.wgs_per_tile;
    const Place<kLanes> at(p, table);
    const int chunk = at.chunk;
    const bool in_row = 8 * chunk < p.D;
    const Token t = find_token(p, (long long)of_tile * p.tile_tokens + at.token);
    const bool live = t.live && in_row;
    const int k_first = p.q_units, v_first = k_first + p.k_units;
    const int u_begin = (int)part * p.units_per_wg, u_end = min(u_begin + p.units_per_wg, v_first + p.v_units);
    auto heads_of = [&](const Rows &x, long long offset, int H, int first, bool there) {
        return Heads(x, offset + 8 * chunk, H, at.head0, at.heads, first, u_begin, there);
    };
    // kinds of rows one behind the other: what is true of the one that unit u has
    auto load = [&](Heads &from, int u, int end, u32x4 (&raw)[kAhead]) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            raw[i] = u32x4{0, 0, 0, 0};
            if (u + i < end && u + i < from.end) raw[i] = *reinterpret_cast<const u32x4 *>(from.at);
            from.at += from.step;
        }
    };
    Heads q_in = heads_of(p.q, t.b * p.q.sb + t.row * p.q.sn, p.Hq, 0, live);
    Heads k_in = heads_of(p.k, t.b * p.k.sb + t.row * p.k.sn, p.Hkv, k_first, live);
    u32x4 raw[kAhead];
    const int q_end = min(u_end, k_first), k_begin = max(u_begin, k_first), k_end = min(u_end, v_first), v_begin = max(u_begin, v_first);
    if (u_begin < q_end)  // (the first rows are on the way while the angles are worked out)
        load(q_in, u_begin, q_end, raw);
    else if (k_begin < k_end)
        load(k_in, k_begin, k_end, raw);

    const float inv_d = 1.f / (float)p.D;
    Turn turn;
    if (u_begin < v_first) {
        find_angles<kLanes>(p, t.pos, at.table);
        __syncthreads();
        turn = lane_turn(p, at.table, at.of_wave, chunk);
    }
    auto rows = [&](Heads &from, Heads &to, int begin, int end, const float *w) {
        float a[8], b[8];  // weight times cosine, the partner's times sine
        row_weights(w, chunk, in_row, a);
        partner_weights(w, p, chunk, b);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            a[j] *= turn.c[j];
            b[j] *= turn.s[j];
        }
        for (int u = begin; u < end; u += kAhead) {
            if (u > u_begin) load(from, u, end, raw);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (u + i >= end) break;
                float x[8], xp[8], y[8];
                unpack<kF16>(raw[i], x);
                unpack<kF16>(partners(raw[i], turn, p.interleaved), xp);
                float r = 1.f;
                if (w) {
                    float ss = 0.f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) ss += x[j] * x[j];
                    r = __builtin_amdgcn_rsqf(row_sum<kLanes>(ss) * inv_d + p.eps);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = r * (x[j] * a[j] + xp[j] * b[j]);
                if (u + i < to.end) *reinterpret_cast<u32x4 *>(to.at) = pack<kF16>(y);
                to.at += to.step;
            }
        }
    };
    if (u_begin < q_end) {
        Heads q_out = heads_of(p.q_out, t.b * p.q_out.sb + t.row * p.q_out.sn, p.Hq, 0, live);
        rows(q_in, q_out, u_begin, q_end, p.q_weight);
    }
    if (u_end <= k_first) return;
    const long long row0 = p.seq.cu_k && !p.pages.block_table ? p.seq.cu_k[t.of] : 0;
    const int row = t.cached ? t.at : 0;
    bool inside;
    if (k_begin < k_end) {
        const long long k_at = cache_row(p.pages, p.k_out, t.of, row0, row, p.seq.cu_k != nullptr, inside);
        Heads k_out = heads_of(p.k_out, k_at, p.Hkv, k_first, live && t.cached && inside);
        rows(k_in, k_out, k_begin, k_end, p.k_weight);
    }
    if (v_begin >= u_end) return;
    const long long v_at = cache_row(p.pages, p.v_out, t.of, row0, row, p.seq.cu_k != nullptr, inside);
    Heads v_in = heads_of(p.v, t.b * p.v.sb + t.row * p.v.sn, p.Hkv, v_first, live), v_out = heads_of(p.v_out, v_at, p.Hkv, v_first, live && t.cached && inside);
    for (int u = v_begin; u < u_end; u += kAhead) {
        load(v_in, u, u_end, raw);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (u + i < u_end && u + i < v_out.end) *reinterpret_cast<u32x4 *>(v_out.at) = raw[i];
            v_out.at += v_out.step;
        }
    }
}

constexpr int kBwdAhead = 2;

template <int kLanes, bool kF16>
__global__ __launch_bounds__(kNThreads, 4) void swaa_norm_rope_bwd_kernel(const NormRopeParams p) {
    fetch_args<NormRopeParams>();
    __shared__ float sums[4][2][kLanes * 8];
    extern __shared__ float2 table[];
    const int tid = threadIdx.x;
    const unsigned group = fastdiv(blockIdx.x, p.div_wgs), part = blockIdx.x - group * (unsigned)p.wgs_per_tile;
    const Place<kLanes> at(p, table);
    const int chunk = at.chunk;
    const bool in_row = 8 * chunk < p.D;
    const float inv_d = 1.f / (float)p.D;
    const int k_first = p.q_units, u_begin = (int)part * p.units_per_wg, u_end = min(u_begin + p.units_per_wg, k_first + p.k_units);
    float dw[2][8];  // of q and of k
#pragma unroll
    for (int j = 0; j < 8; ++j) dw[0][j] = dw[1][j] = 0.f;

    for (long long n = 0; n < p.tiles_per_wg; ++n) {
        const long long first_token = ((long long)group * p.tiles_per_wg + n) * p.tile_tokens;
        if (first_token >= p.tokens) break;
        const Token t = find_token(p, first_token + at.token);
        const bool live = t.live && in_row;
        if (n > 0) __syncthreads();  // (the tile before's angles are done with)
        find_angles<kLanes>(p, t.pos, at.table);
        __syncthreads();
        const Turn turn = lane_turn(p, at.table, at.of_wave, chunk);
        auto rows = [&](const Rows &x_of, const Rows &dy_of, const Rows &dx_of, int H, int first, int begin, int end, const float *w, float (&sum)[8]) {
            if (begin >= end) return;
            auto heads_of = [&](const Rows &r) { return Heads(r, t.b * r.sb + t.row * r.sn + 8 * chunk, H, at.head0, at.heads, first, begin, live); };
            Heads x_in = heads_of(x_of), dy = heads_of(dy_of), dx = heads_of(dx_of);
            float wj[8];
            row_weights(w, chunk, in_row, wj);
            for (int u = begin; u < end; u += kBwdAhead) {
                u32x4 raw[kBwdAhead], grad[kBwdAhead];
#pragma unroll
                for (int i = 0; i < kBwdAhead; ++i) {
                    raw[i] = grad[i] = u32x4{0, 0, 0, 0};
                    if (u + i < end && u + i < dy.end) {
                        grad[i] = *reinterpret_cast<const u32x4 *>(dy.at);
                        if (w) raw[i] = *reinterpret_cast<const u32x4 *>(x_in.at);
                    }
                    dy.at += dy.step;
                    x_in.at += x_in.step;
                }
#pragma unroll
                for (int i = 0; i < kBwdAhead; ++i) {
                    if (u + i >= end) break;
                    float g[8], gp[8];
                    unpack<kF16>(grad[i], g);
                    unpack<kF16>(partners(grad[i], turn, p.interleaved), gp);
#pragma unroll
                    for (int j = 0; j < 8; ++j) g[j] = g[j] * turn.c[j] - gp[j] * turn.s[j];
                    if (w) {
                        float x[8], ss = 0.f, dot = 0.f;
                        unpack<kF16>(raw[i], x);
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            ss += x[j] * x[j];
                            dot += x[j] * wj[j] * g[j];
                        }
                        const float r = __builtin_amdgcn_rsqf(row_sum<kLanes>(ss) * inv_d + p.eps);
                        const float along = row_sum<kLanes>(dot) * inv_d * r * r;
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            sum[j] += g[j] * (x[j] * r);
                            g[j] = r * (wj[j] * g[j] - x[j] * along);
                        }
                    }
                    if (u + i < dx.end) *reinterpret_cast<u32x4 *>(dx.at) = pack<kF16>(g);
                    dx.at += dx.step;
                }
            }
        };
        rows(p.q, p.dq_out, p.q_out, p.Hq, 0, u_begin, min(u_end, k_first), p.q_weight, dw[0]);
        rows(p.k, p.dk_out, p.k_out, p.Hkv, k_first, max(u_begin, k_first), u_end, p.k_weight, dw[1]);
    }
    if (!p.partial) return;
    // lanes of the same place in a row, then the four waves
#pragma unroll
    for (int of_k = 0; of_k < 2; ++of_k)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float x = dw[of_k][j];
#pragma unroll
            for (int d = kLanes; d < 64; d *= 2) x += __shfl_xor(x, d);
            if ((tid & 63) < kLanes) sums[tid / 64][of_k][8 * chunk + j] = x;
        }
    __syncthreads();
    for (int i = tid; i < 2 * p.D; i += kNThreads) {
        const int of_k = i >= p.D, d = i - of_k * p.D;
        p.partial[(long long)blockIdx.x * 2 * p.D + i] = (sums[0][of_k][d] + sums[1][of_k][d]) + (sums[2][of_k][d] + sums[3][of_k][d]);
    }
}

// The workgroups' sums added up, always in the same order: 16 columns a workgroup, 64 lanes to each.
constexpr int kSumThreads = 1024;
__global__ __launch_bounds__(kSumThreads) void swaa_norm_weight_sums_kernel(const float *partial, long long n, int D, float *dq_weight, float *dk_weight) {
    __shared__ float sums[64][17];
    const int col = blockIdx.x * 16 + threadIdx.x % 16, lane = threadIdx.x / 16;  // (2 D is a multiple of 16)
    float x = 0.f;
#pragma unroll 8
    for (long long i = lane; i < n; i += 64) x += partial[i * 2 * D + col];
    sums[lane][threadIdx.x % 16] = x;
    __syncthreads();
    if (threadIdx.x < 64) {
        float part = 0.f;  // four threads to a column
        for (int i = 0; i < 16; ++i) part += sums[16 * (threadIdx.x / 16) + i][threadIdx.x % 16];
        part += __shfl_xor(part, 16);
        part += __shfl_xor(part, 32);
        if (threadIdx.x < 16) (col < D ? dq_weight : dk_weight)[col < D ? col : col - D] = part;
    }
}

int lanes_of_row(int D) { return D <= 32 ? 4 : D <= 64 ? 8 : D <= 128 ? 16 : 32; }

// Tile and units.  A wave has as many tokens as rows at a time (four of head dimension 128), fewer if there are fewer.  Few tokens: the
// four waves share them and take different heads.  Many: each wave has its own and goes through the heads by itself.  The
// units of a tile are shared out over workgroups until there are kFillWgs; a backward call has no more than those, of several tiles
// each, so that few sums are left to add up.
bool plan(NormRopeParams &p, bool backward) {
    const int wave_rows = 64 / lanes_of_row(p.D);
    p.wave_shift = 0;
    while ((2 << p.wave_shift) <= wave_rows && (1LL << p.wave_shift) < p.tokens) ++p.wave_shift;
    p.by_wave = p.tokens >= kByWaveTokens ? 1 : 0;
    p.tile_tokens = (p.by_wave ? 4 : 1) << p.wave_shift;
    const int heads = (p.by_wave ? wave_rows : 4 * wave_rows) >> p.wave_shift;
    p.q_units = (p.Hq + heads - 1) / heads;
    p.k_units = (p.Hkv + heads - 1) / heads;
    p.v_units = p.v.ptr ? p.k_units : 0;
    const int units = p.q_units + p.k_units + p.v_units;
    const long long tiles = (p.tokens + p.tile_tokens - 1) / p.tile_tokens;
    const long long parts = tiles >= kFillWgs ? 1 : (kFillWgs + tiles - 1) / tiles;
    p.units_per_wg = (int)((units + parts - 1) / parts);
    const int least = !p.by_wave ? 1 : tiles < kManyTiles ? kLeastUnits : 2 * kLeastUnits;
    if (p.units_per_wg < least) p.units_per_wg = least < units ? least : units;
    p.wgs_per_tile = (units + p.units_per_wg - 1) / p.units_per_wg;
    p.div_wgs = make_fastdiv((unsigned)p.wgs_per_tile);
    p.tiles_per_wg = backward ? (tiles + kFillWgs - 1) / kFillWgs : 1;
    p.wgs = (tiles + p.tiles_per_wg - 1) / p.tiles_per_wg * p.wgs_per_tile;
    return p.wgs <= 0x7fffffffLL;
}

template <template <int, bool> class Kernel>
hipError_t dispatch(const NormRopeParams &p, hipStream_t stream) {
    const size_t lds = sizeof(float2) * (size_t)(p.R / 2) * p.tile_tokens;
    auto go = [&](auto kernel) {
        kernel<<<dim3((unsigned)p.wgs), dim3(kNThreads), lds, stream>>>(p);
        return hipGetLastError();
    };
    switch (lanes_of_row(p.D)) {
        case 4: return p.fp16 ? go(Kernel<4, true>::fn) : go(Kernel<4, false>::fn);
        case 8: return p.fp16 ? go(Kernel<8, true>::fn) : go(Kernel<8, false>::fn);
        case 16: return p.fp16 ? go(Kernel<16, true>::fn) : go(Kernel<16, false>::fn);
        default: return p.fp16 ? go(Kernel<32, true>::fn) : go(Kernel<32, false>::fn);
    }
}
template <int kLanes, bool kF16>
struct Fwd {
    static constexpr auto fn = swaa_norm_rope_kernel<kLanes, kF16>;
};
template <int kLanes, bool kF16>
struct Bwd {
    static constexpr auto fn = swaa_norm_rope_bwd_kernel<kLanes, kF16>;
};

}  // namespace

bool plan_norm_rope(NormRopeParams &p) { return plan(p, false); }
bool plan_norm_rope_bwd(NormRopeParams &p) { return plan(p, true); }

hipError_t launch_norm_rope(const NormRopeParams &p, hipStream_t stream) { return dispatch<Fwd>(p, stream); }

hipError_t launch_norm_rope_bwd(const NormRopeParams &p, hipStream_t stream) {
    const hipError_t err = dispatch<Bwd>(p, stream);
    if (err != hipSuccess || !p.partial) return err;
    swaa_norm_weight_sums_kernel<<<dim3(2 * p.D / 16), dim3(kSumThreads), 0, stream>>>(p.partial, p.wgs, p.D, p.dq_weight, p.dk_weight);
    return hipGetLastError();
}

}  // namespace swaa
