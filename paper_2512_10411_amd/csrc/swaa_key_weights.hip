// Attention weight that each cached key gets from the query rows of a call (gfx950): with the forward's log-sum-exp,
//
//   weight[b, g, j] = decay * weight[b, g, j] + sum over heads h of group g and rows r that see key j of exp(s_rj - lse[b, h, r])
//
// A workgroup owns 256 keys of one (sequence, KV head) pair: four waves with 64 keys each, whose K rows stay in registers as
// MFMA operands for the whole call.  Past them go the columns: the (head of the group, row) pairs whose rows see any of the 256
// keys, 64 (or 32) at a time through LDS, shared by the waves.  S = K Q^T in tiles of 16 x 16, p = exp2(s * scale - lse), and
// every lane adds up its four keys' p over its column of each tile; the 16 columns of a tile meet once, at the end.
//   * Nothing of the size rows x keys ever leaves the registers, and no sums meet in memory in an order that changes: a key's sum
//     is one workgroup's, or one sum per chunk of the columns added up by a second kernel in the chunks' order.
//   * Few rows (a decode step): the read of K is all there is.  Many: matrix and exponential work about balanced.
#include "swaa_cache_ops.h"

namespace swaa {
namespace {

constexpr int kWThreads = 256;
constexpr int kWaveKeys = 64;
constexpr int kMinChunk = 256;    // columns a workgroup goes through at least, if there are as many
constexpr int kMaxChunks = 16;    // workgroups that share a tile of keys at most
constexpr int kFillItems = 2048;  // workgroups that a call should have

typedef float f32x4 __attribute__((ext_vector_type(4)));

template <bool kF16>
__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (kF16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// The rows that see a key of [k0, k1): first those of the keys' windows, then generated rows further back.
struct SeenBy {
    int first, n, generated, n_all;  // rows first .. first + n - 1, then generated .. nq - 1: n_all in all
    __device__ __forceinline__ int row(int i) const { return i < n ? first + i : generated + (i - n); }
};
__device__ __forceinline__ SeenBy seen_by(int k0, int k1, int nq, int nk, int W, int S, int P) {
    const int off = nk - nq;  // row r stands at position off + r
    SeenBy s;
    s.first = min(max(k0 - off, 0), nq);
    const int past = k0 < S ? nk : min((long long)nk, (long long)k1 + W - 1);  // first position whose window lies behind all the keys
    const int end = min(max(past - off, s.first), nq);
    s.n = end - s.first;
    s.generated = min(max(P - off, end), nq);
    s.n_all = s.n + (nq - s.generated);
    return s;
}

struct Item {
    int b, kvh, tile, chunk;
};
__device__ __forceinline__ Item item_of(const KeyWeightsParams &p, unsigned id) {
    Item w;
    // pairs in turn, so that a die (the workgroups of one residue of 8) stays with few of them, whose rows its L2 then holds
    const unsigned rest = fastdiv(id, p.div_pairs), pair = id - rest * (unsigned)p.pairs;
    w.chunk = (int)fastdiv(rest, p.div_tiles);
    w.tile = (int)(rest - (unsigned)w.chunk * (unsigned)p.tiles);
    w.b = (int)fastdiv(pair, p.div_hkv);
    w.kvh = (int)(pair - (unsigned)w.b * (unsigned)(p.pairs / p.seq.B));
    return w;
}

// What the keys of a tile are told about a column.
struct Column {
    float lse2;   // log2 units
    int pos, lo;  // the row sees the keys up to pos that lie above lo, and the sinks; pos -1: nothing (no such column)
    int pad;
};

template <int D, bool kF16>
__global__ __launch_bounds__(kWThreads, D <= 128 ? 3 : 2) void swaa_key_weights_kernel(const KeyWeightsParams p) {
    constexpr int KS = D / 32;                   // k-steps of a product
    constexpr int kCols = D <= 128 ? 64 : 32;    // columns of a stage
    constexpr int kPitch = D * 2 + 16;           // bytes from column to column in LDS: 8 columns' chunks lie in different banks
    constexpr int kChunks = D / 8;               // of 16 bytes in a row
    constexpr int kStageChunks = kCols * kChunks;
    constexpr int kPer = (kStageChunks + kWThreads - 1) / kWThreads;  // chunks a thread brings
    __shared__ __attribute__((aligned(16))) unsigned char q_lds[2][kCols * kPitch];
    __shared__ __attribute__((aligned(16))) Column columns[2][kCols];

    const Item it = item_of(p, blockIdx.x);
    int nq, nk;
    sequence(p.seq, it.b, nq, nk);
    const int k0 = it.tile * kKeyTile;
    if (k0 >= nk) return;
    const int P = p.n_prompts ? max(p.n_prompts[it.b], 0) : p.P;
    const SeenBy seen = seen_by(k0, min(k0 + kKeyTile, nk), nq, nk, p.W, p.S, P);
    const long long all_cols = (long long)seen.n_all * p.G;
    const long long c_begin = it.chunk * p.chunk_cols;
    const long long c_end = min(all_cols, c_begin + p.chunk_cols);
    if (it.chunk > 0 && c_begin >= all_cols) return;

    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const bool packed = p.seq.cu_q != nullptr;
    const int l16 = lane & 15, quad = lane >> 4;
    const int wk0 = k0 + wave * kWaveKeys;

    // ---- K: rows wk0 + 16 m + l16, elements 32 ks + 8 quad ..; keys beyond the sequence repeat its last one
    u32x4 kf[4][KS];
    {
        const long long row0 = packed && !p.pages.block_table ? p.seq.cu_k[it.b] : 0;
        const char *src[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            bool inside;
            src[m] = p.k.ptr + 2 * (cache_row(p.pages, p.k, it.b, row0, min(wk0 + 16 * m + l16, nk - 1), packed, inside) + it.kvh * p.k.sh + 8 * quad);
        }
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) kf[m][ks] = *reinterpret_cast<const u32x4 *>(src[m] + 64 * ks);
    }

    f32x4 sum[4];
#pragma unroll
    for (int m = 0; m < 4; ++m) sum[m] = f32x4{0.f, 0.f, 0.f, 0.f};

    // ---- columns, a stage at a time: global -> registers -> LDS
    const char *q_base = p.q.ptr + 2 * ((packed ? 0 : it.b * p.q.sb) + it.kvh * (long long)p.G * p.q.sh +
                                        (packed ? p.seq.cu_q[it.b] * p.q.sn : 0));
    const float *lse_base = p.lse + (packed ? p.seq.cu_q[it.b] : it.b * p.lse_sb) + it.kvh * (long long)p.G * p.lse_sh;
    u32x4 q_next[kPer];
    Column col_next;
    auto load_stage = [&](long long c0) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int id = min(tid + i * kWThreads, kStageChunks - 1);
            const long long c = min(c0 + id / kChunks, c_end - 1);
            const unsigned h = (unsigned)c / (unsigned)seen.n_all;
            const int r = seen.row((int)((unsigned)c - h * (unsigned)seen.n_all));
            q_next[i] = *reinterpret_cast<const u32x4 *>(q_base + 2 * (h * p.q.sh + r * p.q.sn + 8 * (id % kChunks)));
        }
        if (tid < kCols) {
            const long long c = min(c0 + tid, c_end - 1);
            const unsigned h = (unsigned)c / (unsigned)seen.n_all;
            const int r = seen.row((int)((unsigned)c - h * (unsigned)seen.n_all));
            const float lse = lse_base[h * p.lse_sh + r];
            const int pos = nk - nq + r;
            // (a row whose scores are all -infinity gives no weight)
            const bool none = c0 + tid >= c_end || opaque_bits(lse) == 0xff800000u;
            col_next.lse2 = none ? 0.f : lse * 1.44269504088896340736f;
            col_next.pos = none ? -1 : pos;
            col_next.lo = pos >= P ? -1 : pos - p.W;
        }
    };
    auto store_stage = [&](int buf) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int id = tid + i * kWThreads;
            if (kStageChunks % kWThreads == 0 || id < kStageChunks) *reinterpret_cast<u32x4 *>(&q_lds[buf][id / kChunks * kPitch + id % kChunks * 16]) = q_next[i];
        }
        if (tid < kCols) columns[buf][tid] = col_next;
    };

    if (c_begin < c_end) {
        load_stage(c_begin);
        store_stage(0);
        __syncthreads();
        int buf = 0;
        for (long long c0 = c_begin; c0 < c_end; c0 += kCols, buf ^= 1) {
            const bool more = c0 + kCols < c_end;
            if (more) load_stage(c0 + kCols);
#pragma unroll
            for (int t = 0; t < kCols / 16; ++t) {
                const Column col = columns[buf][16 * t + l16];
                f32x4 s[4];
#pragma unroll
                for (int m = 0; m < 4; ++m) s[m] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    const u32x4 qf = *reinterpret_cast<const u32x4 *>(&q_lds[buf][(16 * t + l16) * kPitch + 64 * ks + 16 * quad]);
#pragma unroll
                    for (int m = 0; m < 4; ++m) s[m] = mfma16<kF16>(kf[m][ks], qf, s[m]);
                }
                // (does every column of the tile see all 64 keys?)
                const bool all = col.pos >= wk0 + kWaveKeys - 1 && (col.lo < wk0 || wk0 + kWaveKeys <= p.S);
                if (__ballot(all) == ~0ull) {
#pragma unroll
                    for (int m = 0; m < 4; ++m)
#pragma unroll
                        for (int e = 0; e < 4; ++e) sum[m][e] += __builtin_amdgcn_exp2f(s[m][e] * p.scale_log2 - col.lse2);
                } else {
#pragma unroll
                    for (int m = 0; m < 4; ++m)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int key = wk0 + 16 * m + 4 * quad + e;
                            const bool sees = key <= col.pos && (key > col.lo || key < p.S);
                            const float x = __builtin_amdgcn_exp2f(s[m][e] * p.scale_log2 - col.lse2);
                            sum[m][e] += sees ? x : 0.f;
                        }
                }
            }
            if (more) store_stage(buf ^ 1);
            __syncthreads();
        }
    }

    // ---- the 16 columns of each tile meet
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float x = sum[m][e];
            x += __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x128, 0xf, 0xf, true));
            x += __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x124, 0xf, 0xf, true));
            x += __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x122, 0xf, 0xf, true));
            x += __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x121, 0xf, 0xf, true));
            sum[m][e] = x;
        }
    // lane (l16, quad) writes key 16 (l16 / 4) + 4 quad + l16 % 4 of its wave
    float mine = 0.f;
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (l16 == 4 * m + e) mine = sum[m][e];
    const int of_tile = wave * kWaveKeys + 16 * (l16 >> 2) + 4 * quad + (l16 & 3);
    if (p.chunks > 1) {
        const long long pair = (long long)it.b * (p.pairs / p.seq.B) + it.kvh;
        p.partial[((pair * p.tiles + it.tile) * p.chunks + it.chunk) * kKeyTile + of_tile] = mine;
    } else if (k0 + of_tile < nk) {
        float *w = p.weights + it.b * p.w_sb + it.kvh * p.w_sh + k0 + of_tile;
        *w = p.decay != 0.f ? p.decay * *w + mine : mine;
    }
}

// Chunks of a tile's columns added up in their order.
__global__ __launch_bounds__(kKeyTile) void swaa_key_weights_merge_kernel(const KeyWeightsParams p) {
    const Item it = item_of(p, blockIdx.x);  // (as many workgroups as tiles: chunk 0)
    int nq, nk;
    sequence(p.seq, it.b, nq, nk);
    const int k0 = it.tile * kKeyTile, key = k0 + (int)threadIdx.x;
    if (key >= nk) return;
    const int P = p.n_prompts ? max(p.n_prompts[it.b], 0) : p.P;
    const SeenBy seen = seen_by(k0, min(k0 + kKeyTile, nk), nq, nk, p.W, p.S, P);
    const long long all_cols = (long long)seen.n_all * p.G;
    const long long pair = (long long)it.b * (p.pairs / p.seq.B) + it.kvh;
    const float *src = p.partial + (pair * p.tiles + it.tile) * p.chunks * kKeyTile + threadIdx.x;
    float x = src[0];
    for (int c = 1; c < p.chunks && c * p.chunk_cols < all_cols; ++c) x += src[(long long)c * kKeyTile];
    float *w = p.weights + it.b * p.w_sb + it.kvh * p.w_sh + key;
    *w = p.decay != 0.f ? p.decay * *w + x : x;
}

template <int D>
hipError_t launch(const KeyWeightsParams &p, hipStream_t stream) {
    const unsigned wgs = (unsigned)((long long)p.pairs * p.tiles * p.chunks);
    if (p.fp16)
        swaa_key_weights_kernel<D, true><<<dim3(wgs), dim3(kWThreads), 0, stream>>>(p);
    else
        swaa_key_weights_kernel<D, false><<<dim3(wgs), dim3(kWThreads), 0, stream>>>(p);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess || p.chunks == 1) return err;
    swaa_key_weights_merge_kernel<<<dim3((unsigned)((long long)p.pairs * p.tiles)), dim3(kKeyTile), 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace

// Columns that a tile of keys has at most, and into how many chunks they go: until the call has as many workgroups as the chip
// wants, but not below kMinChunk columns each.
bool plan_key_weights(KeyWeightsParams &p) {
    p.pairs = p.seq.B * (p.Hq / p.G);
    p.tiles = (p.seq.Nk + kKeyTile - 1) / kKeyTile;
    const long long items = (long long)p.pairs * p.tiles;
    const long long most = (long long)p.G * p.seq.Nq;
    long long chunks = (kFillItems + items - 1) / items;
    // (tiles differ: the first keys of a full-attention layer are seen by all rows, the last ones by their own)
    if (chunks < 4 && most > 16 * kMinChunk) chunks = 4;
    chunks = chunks < kMaxChunks ? chunks : kMaxChunks;
    p.chunk_cols = (most + chunks - 1) / chunks;
    if (p.chunk_cols < kMinChunk) p.chunk_cols = kMinChunk;
    p.chunk_cols = (p.chunk_cols + 63) / 64 * 64;
    p.chunks = (int)((most + p.chunk_cols - 1) / p.chunk_cols);
    if (items * p.chunks > 0x7fffffffLL || most > 0x7fffffffLL) return false;
    p.div_pairs = make_fastdiv((unsigned)p.pairs);
    p.div_tiles = make_fastdiv((unsigned)p.tiles);
    p.div_hkv = make_fastdiv((unsigned)(p.Hq / p.G));
    return true;
}

long long key_weights_workspace_bytes(const KeyWeightsParams &p) {
    return p.chunks == 1 ? 0 : (long long)p.pairs * p.tiles * p.chunks * kKeyTile * (long long)sizeof(float);
}

hipError_t launch_key_weights(const KeyWeightsParams &p, hipStream_t stream) {
    switch (p.D) {
        case 32: return launch<32>(p, stream);
        case 64: return launch<64>(p, stream);
        case 96: return launch<96>(p, stream);
        case 128: return launch<128>(p, stream);
        case 160: return launch<160>(p, stream);
        case 192: return launch<192>(p, stream);
        case 224: return launch<224>(p, stream);
        default: return launch<256>(p, stream);
    }
}

}  // namespace swaa
