// RMS norms of the heads of queries and keys with the position rotation in the same pass, forward and backward (gfx950).
//
//   n = x / sqrt(mean(x^2) + eps) * w          y = n rotated in pairs (i, partner of i) by pos * inv_freq[pair]
//
// With the rotation written per element as y_j = n_j C_j + n_p S_j (p: the partner, S_j signed), a row is
// y_j = r (x_j A_j + x_p B_j) with A = w C and B = w_p S: three operations per element, and one sum of squares per row.  The
// backward pass goes through the transposed rotation, g_j = C_j dy_j + S_p dy_p with S_p = -S_j, and the norm:
// dx_j = r (w_j g_j - x_j r^2 mean(x w g)), dw_j = sum over rows of g_j x_j r.
//
// Bound by memory: every element comes in once and goes out once (backward: two in, one out).
//   * A row is D / 8 lanes of 16 bytes (rounded up to a power of two); what a lane multiplies by depends on its token and its
//     place in the row only, so a lane keeps both through a loop over the heads: cosines, sines and weights stay in registers.
//   * The angles are taken in 64 bits (positions go beyond what 32 bits resolve), once per token and pair: a workgroup's
//     threads share them through LDS.
#include "swaa_cache_ops.h"

namespace swaa {
namespace {

constexpr int kNThreads = 256;

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

// What a workgroup knows about the tokens of its tile.
template <int kSlots>
struct TokenTile {
    int pos[kSlots], b[kSlots], row[kSlots];  // row: along the tensors' row axis; b: batch entry to take strides of
    long long k_at[kSlots], v_at[kSlots];     // where the token's key and value go, -1: nowhere
    int live[kSlots];
};
template <int kSlots>
__device__ __forceinline__ void find_token(const NormRopeParams &p, long long first, TokenTile<kSlots> &t) {
    const int s = threadIdx.x;
    if (s >> p.tile_shift) return;
    const long long slot = first + s;
    int b = 0, r = 0, nq = 0, nk = 0, live = slot < p.tokens;
    int axis_row = 0;
    if (live) {
        if (p.by_row) {  // the sequence that holds this row of the packed tensor
            int lo = 0, hi = p.seq.B;  // cu_q[lo] <= slot < cu_q[hi], if any holds it
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                (p.seq.cu_q[mid] <= slot ? lo : hi) = mid;
            }
            b = lo;
            r = (int)(slot - p.seq.cu_q[b]);
        } else {
            b = (int)fastdiv((unsigned)slot, p.div_nq);
            r = (int)(slot - (long long)b * p.seq.Nq);
        }
        sequence(p.seq, b, nq, nk);
        live = r >= 0 && r < nq;
        axis_row = r + (p.seq.cu_q ? p.seq.cu_q[b] : 0);
    }
    t.live[s] = live;
    t.b[s] = p.seq.cu_q ? 0 : b;
    t.row[s] = axis_row;
    const int row = nk - nq + r;
    t.pos[s] = !live ? 0 : !p.positions ? row : p.positions[p.seq.cu_q ? axis_row : b * (long long)p.seq.Nq + r];
    t.k_at[s] = t.v_at[s] = -1;
    if (live) {
        bool inside;
        const long long row0 = p.seq.cu_k && !p.pages.block_table ? p.seq.cu_k[b] : 0;
        const long long k_at = cache_row(p.pages, p.k_out, b, row0, row, p.seq.cu_k != nullptr, inside);
        if (inside) t.k_at[s] = k_at;
        const long long v_at = cache_row(p.pages, p.v_out, b, row0, row, p.seq.cu_k != nullptr, inside);
        if (inside) t.v_at[s] = v_at;
    }
}

// cos and sin of the tile's tokens, [pair][token]: the angle in turns in 64 bits, what is left of it behind whole turns in 32.
__device__ __forceinline__ void find_angles(const NormRopeParams &p, const int *pos, float2 *table) {
    const int token = threadIdx.x & ((1 << p.tile_shift) - 1);
    for (int pair = threadIdx.x >> p.tile_shift; pair < p.R / 2; pair += kNThreads >> p.tile_shift) {
        const double turns = (double)pos[token] * (double)p.inv_freq[pair] * 0.15915494309189533577;
        float s, c;
        sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
        table[(pair << p.tile_shift) + token] = make_float2(c, s);
    }
}

// A lane's rotation: elements 8 chunk .. 8 chunk + 7 of its token's rows.
struct Turn {
    float c[8], s[8];  // y_j = n_j c_j + n_partner s_j
    int partner;       // lane that holds the partners (pairs of halves)
};
__device__ __forceinline__ Turn lane_turn(const NormRopeParams &p, const float2 *table, int token, int chunk) {
    Turn t;
    const int half = p.R / 16;  // chunks of half the rotated elements
    t.partner = threadIdx.x & 63;
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
            const float2 cs = table[((4 * chunk + j / 2) << p.tile_shift) + token];
            t.c[j] = cs.x;
            t.s[j] = j % 2 ? cs.y : -cs.y;
        }
        return t;
    }
    const bool second = chunk >= half;
    t.partner += second ? -half : half;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float2 cs = table[((8 * (second ? chunk - half : chunk) + j) << p.tile_shift) + token];
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

constexpr int kAhead = 4;  // rows of a lane on the way at a time

template <int kLanes, bool kF16>
__global__ __launch_bounds__(kNThreads) void swaa_norm_rope_kernel(const NormRopeParams p) {
    constexpr int kSlots = kNThreads / kLanes;
    __shared__ TokenTile<kSlots> tile;
    extern __shared__ float2 table[];
    const int tid = threadIdx.x;
    const unsigned of_tile = blockIdx.x / (unsigned)p.wgs_per_tile, part = blockIdx.x - of_tile * (unsigned)p.wgs_per_tile;
    find_token<kSlots>(p, (long long)of_tile << p.tile_shift, tile);
    __syncthreads();
    find_angles(p, tile.pos, table);
    __syncthreads();

    const int chunk = tid % kLanes, slot = tid / kLanes;
    const int token = slot & ((1 << p.tile_shift) - 1), head0 = slot >> p.tile_shift;
    const int heads = kSlots >> p.tile_shift;  // at a time
    const bool in_row = 8 * chunk < p.D, live = tile.live[token] && in_row;
    const long long b = tile.b[token], row = tile.row[token];
    const Turn turn = lane_turn(p, table, token, chunk);

    int u = (int)part * p.units_per_wg;
    const int u_end = min(u + p.units_per_wg, p.q_units + p.k_units + p.v_units);
    const float inv_d = 1.f / (float)p.D;
    // units [u, of_part end) of one of q, k, v
    auto pass = [&](const Rows &in, const Rows &out, long long out_at, int H, int first, int units, const float *w, bool plain) {
        const int end = min(u_end, first + units);
        if (u >= end) return;
        float a[8], bq[8];
        if (!plain) {
            float wj[8], wp[8];
            row_weights(w, chunk, in_row, wj);
            partner_weights(w, p, chunk, wp);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                a[j] = wj[j] * turn.c[j];
                bq[j] = wp[j] * turn.s[j];
            }
        }
        const char *src = in.ptr + 2 * (b * in.sb + row * in.sn + 8 * chunk);
        char *dst = out.ptr + 2 * (out_at + 8 * chunk);
        for (; u < end; u += kAhead) {
            u32x4 raw[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int h = (u + i - first) * heads + head0;
                raw[i] = u32x4{0, 0, 0, 0};
                if (u + i < end && h < H && live) raw[i] = *reinterpret_cast<const u32x4 *>(src + 2 * (h * in.sh));
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (u + i >= end) break;
                const int h = (u + i - first) * heads + head0;
                if (!plain) {
                    float x[8], xp[8], y[8];
                    unpack<kF16>(raw[i], x);
                    unpack<kF16>(partners(raw[i], turn, p.interleaved), xp);
                    float r = 1.f;
                    if (w) {
                        float ss = 0.f;
#pragma unroll
                        for (int j = 0; j < 8; ++j) ss += x[j] * x[j];
                        r = 1.f / sqrtf(row_sum<kLanes>(ss) * inv_d + p.eps);
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j) y[j] = r * (x[j] * a[j] + xp[j] * bq[j]);
                    raw[i] = pack<kF16>(y);
                }
                if (h < H && live && out_at >= 0) *reinterpret_cast<u32x4 *>(dst + 2 * (h * out.sh)) = raw[i];
            }
        }
        u = end;
    };
    pass(p.q, p.q_out, b * p.q_out.sb + row * p.q_out.sn, p.Hq, 0, p.q_units, p.q_weight, false);
    pass(p.k, p.k_out, tile.k_at[token], p.Hkv, p.q_units, p.k_units, p.k_weight, false);
    pass(p.v, p.v_out, tile.v_at[token], p.Hkv, p.q_units + p.k_units, p.v_units, nullptr, true);
}

template <int kLanes, bool kF16>
__global__ __launch_bounds__(kNThreads) void swaa_norm_rope_bwd_kernel(const NormRopeParams p) {
    constexpr int kSlots = kNThreads / kLanes;
    constexpr int kBwdAhead = 2;
    __shared__ TokenTile<kSlots> tile;
    __shared__ float sums[4][2][kLanes * 8];
    extern __shared__ float2 table[];
    const int tid = threadIdx.x;
    const unsigned group = blockIdx.x / (unsigned)p.wgs_per_tile, part = blockIdx.x - group * (unsigned)p.wgs_per_tile;
    const int chunk = tid % kLanes, slot = tid / kLanes;
    const int token = slot & ((1 << p.tile_shift) - 1), head0 = slot >> p.tile_shift;
    const int heads = kSlots >> p.tile_shift;
    const bool in_row = 8 * chunk < p.D;
    const float inv_d = 1.f / (float)p.D;
    float dw[2][8];  // of q and of k
#pragma unroll
    for (int j = 0; j < 8; ++j) dw[0][j] = dw[1][j] = 0.f;

    for (long long n = 0; n < p.tiles_per_wg; ++n) {
        const long long first = ((long long)group * p.tiles_per_wg + n) << p.tile_shift;
        if (first >= p.tokens) break;
        __syncthreads();  // (the tile before is done with)
        find_token<kSlots>(p, first, tile);
        __syncthreads();
        find_angles(p, tile.pos, table);
        __syncthreads();
        const bool live = tile.live[token] && in_row;
        const long long b = tile.b[token], row = tile.row[token];
        const Turn turn = lane_turn(p, table, token, chunk);
        int u = (int)part * p.units_per_wg;
        const int u_end = min(u + p.units_per_wg, p.q_units + p.k_units);
        auto pass = [&](const Rows &in, const Rows &grad, const Rows &out, int H, int first_unit, int units, const float *w, float (&sum)[8]) {
            const int end = min(u_end, first_unit + units);
            if (u >= end) return;
            float wj[8];
            row_weights(w, chunk, in_row, wj);
            const char *src = in.ptr + 2 * (b * in.sb + row * in.sn + 8 * chunk);
            const char *gsrc = grad.ptr + 2 * (b * grad.sb + row * grad.sn + 8 * chunk);
            char *dst = out.ptr + 2 * (b * out.sb + row * out.sn + 8 * chunk);
            for (; u < end; u += kBwdAhead) {
                u32x4 raw[kBwdAhead], graw[kBwdAhead];
#pragma unroll
                for (int i = 0; i < kBwdAhead; ++i) {
                    const int h = (u + i - first_unit) * heads + head0;
                    raw[i] = graw[i] = u32x4{0, 0, 0, 0};
                    if (u + i < end && h < H && live) {
                        graw[i] = *reinterpret_cast<const u32x4 *>(gsrc + 2 * (h * grad.sh));
                        if (w) raw[i] = *reinterpret_cast<const u32x4 *>(src + 2 * (h * in.sh));
                    }
                }
#pragma unroll
                for (int i = 0; i < kBwdAhead; ++i) {
                    if (u + i >= end) break;
                    const int h = (u + i - first_unit) * heads + head0;
                    float g[8], gp[8];
                    unpack<kF16>(graw[i], g);
                    unpack<kF16>(partners(graw[i], turn, p.interleaved), gp);
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
                        const float r = 1.f / sqrtf(row_sum<kLanes>(ss) * inv_d + p.eps);
                        const float along = row_sum<kLanes>(dot) * inv_d * r * r;
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            sum[j] += g[j] * (x[j] * r);
                            g[j] = r * (wj[j] * g[j] - x[j] * along);
                        }
                    }
                    if (h < H && live) *reinterpret_cast<u32x4 *>(dst + 2 * (h * out.sh)) = pack<kF16>(g);
                }
            }
            u = end;
        };
        pass(p.q, p.dq_out, p.q_out, p.Hq, 0, p.q_units, p.q_weight, dw[0]);
        pass(p.k, p.dk_out, p.k_out, p.Hkv, p.q_units, p.k_units, p.k_weight, dw[1]);
    }
    if (!p.partial) return;
    // lanes of the same place in a row, then the four waves
#pragma unroll
    for (int part_of = 0; part_of < 2; ++part_of)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float x = dw[part_of][j];
#pragma unroll
            for (int d = kLanes; d < 64; d *= 2) x += __shfl_xor(x, d);
            if ((tid & 63) < kLanes) sums[tid / 64][part_of][8 * chunk + j] = x;
        }
    __syncthreads();
    for (int i = tid; i < 2 * p.D; i += kNThreads) {
        const int part_of = i >= p.D, d = i - part_of * p.D;
        p.partial[(long long)blockIdx.x * 2 * p.D + i] =
            (sums[0][part_of][d] + sums[1][part_of][d]) + (sums[2][part_of][d] + sums[3][part_of][d]);
    }
}

// The workgroups' sums added up, always in the same order: 16 columns a workgroup, 16 lanes to each.
__global__ __launch_bounds__(kNThreads) void swaa_norm_weight_sums_kernel(const float *partial, long long n, int D, float *dq_weight, float *dk_weight) {
    __shared__ float sums[16][17];
    const int col = blockIdx.x * 16 + threadIdx.x % 16, lane = threadIdx.x / 16;
    float x = 0.f;
    if (col < 2 * D)
        for (long long i = lane; i < n; i += 16) x += partial[i * 2 * D + col];
    sums[lane][threadIdx.x % 16] = x;
    __syncthreads();
    if (threadIdx.x < 16 && col < 2 * D) {
        float all = 0.f;
        for (int i = 0; i < 16; ++i) all += sums[i][threadIdx.x];
        (col < D ? dq_weight : dk_weight)[col < D ? col : col - D] = all;
    }
}

int lanes_of_row(int D) { return D <= 32 ? 4 : D <= 64 ? 8 : D <= 128 ? 16 : 32; }

// Tile and units: a tile of as many tokens as a workgroup takes rows at a time, fewer if there are fewer; the units of a tile are
// shared out over workgroups until there are `target`.
bool plan(NormRopeParams &p, int target, bool backward) {
    const int slots = kNThreads / lanes_of_row(p.D);
    p.tile_shift = 0;
    while ((2 << p.tile_shift) <= slots && (1LL << p.tile_shift) < p.tokens) ++p.tile_shift;
    const int heads = slots >> p.tile_shift;
    p.q_units = (p.Hq + heads - 1) / heads;
    p.k_units = (p.Hkv + heads - 1) / heads;
    p.v_units = p.v.ptr ? p.k_units : 0;
    const int units = p.q_units + p.k_units + p.v_units;
    const long long tiles = (p.tokens + (1LL << p.tile_shift) - 1) >> p.tile_shift;
    const long long parts = tiles >= target ? 1 : (target + tiles - 1) / tiles;
    p.units_per_wg = (int)((units + parts - 1) / parts);
    p.wgs_per_tile = (units + p.units_per_wg - 1) / p.units_per_wg;
    p.tiles_per_wg = backward ? (tiles + target - 1) / target : 1;
    p.wgs = (tiles + p.tiles_per_wg - 1) / p.tiles_per_wg * p.wgs_per_tile;
    return p.wgs <= 0x7fffffffLL;
}

template <template <int, bool> class Kernel>
hipError_t dispatch(const NormRopeParams &p, hipStream_t stream) {
    const size_t lds = sizeof(float2) * (size_t)(p.R / 2) << p.tile_shift;
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

bool plan_norm_rope(NormRopeParams &p) { return plan(p, 2048, false); }
bool plan_norm_rope_bwd(NormRopeParams &p) { return plan(p, 1024, true); }

hipError_t launch_norm_rope(const NormRopeParams &p, hipStream_t stream) { return dispatch<Fwd>(p, stream); }

hipError_t launch_norm_rope_bwd(const NormRopeParams &p, hipStream_t stream) {
    const hipError_t err = dispatch<Bwd>(p, stream);
    if (err != hipSuccess || !p.partial) return err;
    swaa_norm_weight_sums_kernel<<<dim3((2 * p.D + 15) / 16), dim3(kNThreads), 0, stream>>>(p.partial, p.wgs, p.D, p.dq_weight, p.dk_weight);
    return hipGetLastError();
}

}  // namespace swaa
