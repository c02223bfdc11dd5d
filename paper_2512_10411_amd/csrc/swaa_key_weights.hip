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
constexpr int kMinChunk = 256;    // columns a workgroup goes through at least, if there are as many
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
template <typename T>
__host__ __device__ __forceinline__ T lesser(T a, T b) { return a < b ? a : b; }
__host__ __device__ __forceinline__ SeenBy seen_by(int k0, int k1, int nq, int nk, int W, int S, int P) {
    const int off = nk - nq;  // row r stands at position off + r
    SeenBy s;
    s.first = lesser(k0 > off ? k0 - off : 0, nq);
    const int past = k0 < S ? nk : (int)lesser((long long)nk, (long long)k1 + W - 1);  // first position whose window lies behind all the keys
    const int end = past - off < s.first ? s.first : lesser(past - off, nq);
    s.n = end - s.first;
    s.generated = P - off < end ? end : lesser(P - off, nq);
    s.n_all = s.n + (nq - s.generated);
    return s;
}

// Work: the tiles that hold sinks (seen by all rows that follow) have sink_chunks chunks of columns each, and come first; the others
// have `chunks`.  Pairs in turn, so that a die (the workgroups of one residue of 8) stays with few of them, whose rows its L2 then holds.
struct Item {
    int b, kvh, tile, chunk;
    bool whole;  // the tile's only chunk: its sums are the result
};
__device__ __forceinline__ Item item_of(const KeyWeightsParams &p, unsigned id) {
    Item w;
    const unsigned of_pair = fastdiv(id, p.div_pairs), pair = id - of_pair * (unsigned)p.pairs;
    if (of_pair < (unsigned)p.sink_items) {
        w.tile = (int)fastdiv(of_pair, p.div_sink_chunks);
        w.chunk = (int)(of_pair - (unsigned)w.tile * (unsigned)p.sink_chunks);
        w.whole = p.sink_chunks == 1;
    } else {
        const unsigned rest = of_pair - (unsigned)p.sink_items, others = (unsigned)(p.tiles - p.sink_tiles);
        w.chunk = (int)fastdiv(rest, p.div_others);  // (all tiles' first chunks, then all second ones: the early tiles' have more)
        w.tile = p.sink_tiles + (int)(rest - (unsigned)w.chunk * others);
        w.whole = p.chunks == 1;
    }
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

// LDS: two buffers of kCols rows of Q without padding, then two of kCols Columns.  16-byte chunk c of row r lies at chunk
// c ^ turn(r), so that eight rows' equal chunks lie in different banks; the copies apply it on the global side.
template <int D>
struct Stage {
    static constexpr int kCols = D <= 128 ? 64 : 32;
    static constexpr int kRowB = D * 2, kBufB = kCols * kRowB;
    static constexpr int kColumns = 2 * kBufB;  // byte address
    static constexpr int kBytes = kColumns + 2 * kCols * (int)sizeof(Column);
    static __device__ __forceinline__ int turn(int r) { return D % 64 == 0 ? r & 7 : (r >> 1) & 3; }
};

__device__ __forceinline__ u32x4 lds16(uint32_t addr) { return *(const u32x4 __attribute__((address_space(3))) *)(uintptr_t)addr; }

template <int D, bool kF16>
__global__ __launch_bounds__(kWThreads, D <= 128 ? 3 : 2) void swaa_key_weights_kernel(const KeyWeightsParams p) {
    using T = Stage<D>;
    constexpr int kM = 4;                       // 16-key blocks of a wave
    constexpr int kWaveKeys = 16 * kM;
    constexpr int KS = D / 32;                  // k-steps of a product
    constexpr int kCols = T::kCols, kWaveCols = kCols / 4;  // columns that a wave brings
    constexpr int kChunks = D / 8;              // of 16 bytes in a row
    constexpr int kCopies = (kWaveCols * kChunks + 63) / 64;  // wave instructions for them
    static_assert(kKeyTile == 4 * kWaveKeys, "");

    const Item it = item_of(p, blockIdx.x);
    int nq, nk;
    sequence(p.seq, it.b, nq, nk);
    const int k0 = it.tile * kKeyTile;
    if (k0 >= nk) return;
    const int P = p.n_prompts ? max(p.n_prompts[it.b], 0) : p.P;
    const SeenBy seen = seen_by(k0, min(k0 + kKeyTile, nk), nq, nk, p.W, p.S, P);
    const unsigned all_cols = (unsigned)seen.n_all * (unsigned)p.G;
    const unsigned c_begin = (unsigned)it.chunk * (unsigned)p.chunk_cols;
    if (it.chunk > 0 && c_begin >= all_cols) return;
    const unsigned c_end = min(all_cols, c_begin + (unsigned)p.chunk_cols);

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const bool packed = p.seq.cu_q != nullptr;
    const int l16 = lane & 15, quad = lane >> 4;
    const int wk0 = k0 + wave * kWaveKeys;

    // ---- K: rows wk0 + 16 m + l16, elements 32 ks + 8 quad ..; keys beyond the sequence repeat its last one
    u32x4 kf[kM][KS];
    {
        const long long row0 = packed && !p.pages.block_table ? p.seq.cu_k[it.b] : 0;
        const char *src[kM];
#pragma unroll
        for (int m = 0; m < kM; ++m) {
            bool inside;
            src[m] = p.k.ptr + 2 * (cache_row(p.pages, p.k, it.b, row0, min(wk0 + 16 * m + l16, nk - 1), packed, inside) + it.kvh * p.k.sh + 8 * quad);
        }
#pragma unroll
        for (int m = 0; m < kM; ++m)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) kf[m][ks] = *reinterpret_cast<const u32x4 *>(src[m] + 64 * ks);
    }

    f32x4 sum[kM];
#pragma unroll
    for (int m = 0; m < kM; ++m) sum[m] = f32x4{0.f, 0.f, 0.f, 0.f};

    // ---- columns, a stage at a time.  A wave brings kWaveCols of a stage's; lane l keeps track of the one at l % kWaveCols.
    const char *q_base = p.q.ptr + 2 * ((packed ? 0 : it.b * p.q.sb) + it.kvh * (long long)p.G * p.q.sh +
                                        (packed ? p.seq.cu_q[it.b] * p.q.sn : 0));
    const float *lse_base = p.lse + (packed ? p.seq.cu_q[it.b] : it.b * p.lse_sb) + it.kvh * (long long)p.G * p.lse_sh;
    const unsigned n_all = (unsigned)seen.n_all;
    unsigned col = c_begin + (unsigned)(wave * kWaveCols + lane % kWaveCols), head = 0, index = 0;  // index: of the head's rows that see the tile
    if (c_begin < c_end) {
        head = min(col, c_end - 1) / n_all;
        index = min(col, c_end - 1) - head * n_all;
    }
    float lse = 0.f;
    int row = 0;
    auto issue_stage = [&](int buf) {
        row = seen.row((int)index);
        const long long at = (long long)head * p.q.sh + (long long)row * p.q.sn;
        lse = lse_base[head * p.lse_sh + row];
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            const int id = 64 * i + lane, r = id / kChunks, c = id % kChunks;  // row of the wave's, chunk of LDS
            if (kWaveCols * kChunks % 64 != 0 && id >= kWaveCols * kChunks) break;
            const long long of_row = ((long long)__shfl((int)(at >> 32), r) << 32) | (unsigned)__shfl((int)at, r);
            const char *src = q_base + 2 * of_row + 16 * (c ^ T::turn(wave * kWaveCols + r));
            asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(src),
                         "s"((uint32_t)(buf * T::kBufB + wave * kWaveCols * T::kRowB + 1024 * i))
                         : "memory");
        }
    };
    auto put_columns = [&](int buf) {
        Column c;
        const int pos = nk - nq + row;
        // (a row whose scores are all -infinity gives no weight)
        const bool none = col >= c_end || opaque_bits(lse) == 0xff800000u;
        c.lse2 = none ? 0.f : lse * 1.44269504088896340736f;
        c.pos = none ? -1 : pos;
        c.lo = pos >= P ? -1 : pos - p.W;
        c.pad = 0;
        if (lane < kWaveCols)
            *(u32x4 __attribute__((address_space(3))) *)(uintptr_t)(uint32_t)(T::kColumns + (buf * kCols + wave * kWaveCols + lane) * (int)sizeof(Column)) =
                __builtin_bit_cast(u32x4, c);
    };
    auto next_columns = [&]() {  // kCols columns on; behind the last one, it again
        col += kCols;
        if (col >= c_end) return;
        index += kCols;
        if (index >= n_all) {
            const unsigned more = n_all >= (unsigned)kCols ? 1u : index / n_all;
            head += more;
            index -= more * n_all;
        }
    };

    const uint32_t q_lane = (uint32_t)(l16 * T::kRowB);
    if (c_begin < c_end) {
        issue_stage(0);
        put_columns(0);
    }
    int buf = 0;
    for (unsigned c0 = c_begin; c0 < c_end; c0 += kCols, buf ^= 1) {
        __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0): this wave's share of the stage has landed, and it has read the one before
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();        // everybody's; and everybody is done with the one before
        asm volatile("" ::: "memory");
        const bool more = c0 + kCols < c_end;
        if (more) {
            next_columns();
            issue_stage(buf ^ 1);
        }
        const int units = (int)min((unsigned)(kCols / 16), (c_end - c0 + 15) / 16);
        const uint32_t q_at = (uint32_t)(buf * T::kBufB) + q_lane, col_at = (uint32_t)(T::kColumns + (buf * kCols + l16) * (int)sizeof(Column));
        for (int t = 0; t < units; ++t) {
            const Column cl = __builtin_bit_cast(Column, lds16(col_at + (uint32_t)(16 * t * (int)sizeof(Column))));
            f32x4 s[kM];
#pragma unroll
            for (int m = 0; m < kM; ++m) s[m] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const u32x4 qf = lds16(q_at + (uint32_t)(16 * t * T::kRowB) + (uint32_t)(((4 * ks + quad) ^ T::turn(l16)) << 4));
#pragma unroll
                for (int m = 0; m < kM; ++m) s[m] = mfma16<kF16>(kf[m][ks], qf, s[m]);
            }
            // (does every column of the tile see all the wave's keys?)
            const bool all = cl.pos >= wk0 + kWaveKeys - 1 && (cl.lo < wk0 || wk0 + kWaveKeys <= p.S);
            if (__ballot(all) == ~0ull) {
#pragma unroll
                for (int m = 0; m < kM; ++m)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[m][e] += __builtin_amdgcn_exp2f(s[m][e] * p.scale_log2 - cl.lse2);
            } else {
#pragma unroll
                for (int m = 0; m < kM; ++m)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = wk0 + 16 * m + 4 * quad + e;
                        const bool sees = key <= cl.pos && (key > cl.lo || key < p.S);
                        const float x = __builtin_amdgcn_exp2f(s[m][e] * p.scale_log2 - cl.lse2);
                        sum[m][e] += sees ? x : 0.f;
                    }
            }
        }
        if (more) put_columns(buf ^ 1);
    }

    // ---- the 16 columns of each tile meet
#pragma unroll
    for (int m = 0; m < kM; ++m)
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
    for (int m = 0; m < kM; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (l16 == 4 * m + e) mine = sum[m][e];
    const int of_tile = wave * kWaveKeys + 16 * (l16 >> 2) + 4 * quad + (l16 & 3);
    if (!it.whole) {
        p.partial[(long long)blockIdx.x * kKeyTile + of_tile] = mine;
    } else if (k0 + of_tile < nk) {
        float *w = p.weights + it.b * p.w_sb + it.kvh * p.w_sh + k0 + of_tile;
        *w = p.decay != 0.f ? p.decay * *w + mine : mine;
    }
}

// Chunks of a tile's columns added up in their order (tiles of several chunks: those of the sinks, or all).
__global__ __launch_bounds__(kKeyTile) void swaa_key_weights_merge_kernel(const KeyWeightsParams p) {
    const unsigned tile = fastdiv(blockIdx.x, p.div_pairs), pair = blockIdx.x - tile * (unsigned)p.pairs;
    const int b = (int)fastdiv(pair, p.div_hkv), kvh = (int)(pair - (unsigned)b * (unsigned)(p.pairs / p.seq.B));
    int nq, nk;
    sequence(p.seq, b, nq, nk);
    const int k0 = (int)tile * kKeyTile, key = k0 + (int)threadIdx.x;
    if (key >= nk) return;
    const int P = p.n_prompts ? max(p.n_prompts[b], 0) : p.P;
    const SeenBy seen = seen_by(k0, min(k0 + kKeyTile, nk), nq, nk, p.W, p.S, P);
    const long long all_cols = (long long)seen.n_all * p.G;
    const bool has_sinks = (int)tile < p.sink_tiles;
    // its first chunk's place among the pair's items, and from chunk to chunk
    const long long first = has_sinks ? (long long)tile * p.sink_chunks : p.sink_items + ((long long)tile - p.sink_tiles);
    const long long step = (has_sinks ? 1LL : p.tiles - p.sink_tiles) * p.pairs * kKeyTile;
    const int chunks = has_sinks ? p.sink_chunks : p.chunks;
    const float *src = p.partial + (first * p.pairs + pair) * kKeyTile + threadIdx.x;
    float x = src[0];
    for (int c = 1; c < chunks && c * p.chunk_cols < all_cols; ++c) x += src[c * step];
    float *w = p.weights + b * p.w_sb + kvh * p.w_sh + key;
    *w = p.decay != 0.f ? p.decay * *w + x : x;
}

template <int D, bool kF16>
hipError_t launch_one(const KeyWeightsParams &p, hipStream_t stream) {
    constexpr auto kernel = swaa_key_weights_kernel<D, kF16>;
    static_assert(Stage<D>::kBytes <= 64 * 1024, "");
    kernel<<<dim3((unsigned)p.items), dim3(kWThreads), Stage<D>::kBytes, stream>>>(p);
    return hipGetLastError();
}

template <int D>
hipError_t launch(const KeyWeightsParams &p, hipStream_t stream) {
    const hipError_t err = p.fp16 ? launch_one<D, true>(p, stream) : launch_one<D, false>(p, stream);
    const int merged = p.chunks > 1 ? p.tiles : p.sink_chunks > 1 ? p.sink_tiles : 0;
    if (err != hipSuccess || merged == 0) return err;
    swaa_key_weights_merge_kernel<<<dim3((unsigned)((long long)p.pairs * merged)), dim3(kKeyTile), 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace

// The columns of all tiles, shared out in chunks of one length so that the call has as many workgroups as the chip wants.
bool plan_key_weights(KeyWeightsParams &p) {
    const int Nq = p.seq.Nq, Nk = p.seq.Nk;
    p.pairs = p.seq.B * (p.Hq / p.G);
    p.tiles = (Nk + kKeyTile - 1) / kKeyTile;
    const long long most = (long long)p.G * Nq;
    if (most > 0x7fffffffLL - 2 * kMinChunk) return false;
    // rows that see a tile without sinks: those of its window, and generated ones (of sequences with prompt lengths of their own: maybe all)
    const long long generated = p.n_prompts ? Nk : Nk - p.P;
    const long long of_window = (long long)p.W + kKeyTile - 1 + generated;
    const long long usual = (long long)p.G * (of_window < Nq ? of_window : Nq);
    p.sink_tiles = usual < most ? (p.S + kKeyTile - 1) / kKeyTile : 0;
    const bool ramp = of_window >= Nq && Nq > kKeyTile;  // (a whole prompt's rows: the last tiles see few)
    const long long all = p.pairs * ((p.tiles - p.sink_tiles) * (ramp ? usual / 2 + 1 : usual) + p.sink_tiles * most);
    long long chunk = (all + kFillItems - 1) / kFillItems;
    chunk = chunk > kMinChunk ? chunk : kMinChunk;
    p.chunk_cols = (chunk + 63) / 64 * 64;
    p.chunks = (int)((usual + p.chunk_cols - 1) / p.chunk_cols);
    p.sink_chunks = (int)((most + p.chunk_cols - 1) / p.chunk_cols);
    p.sink_items = p.sink_tiles * p.sink_chunks;
    p.items = (long long)p.pairs * (p.sink_items + (long long)(p.tiles - p.sink_tiles) * p.chunks);
    if (p.items > 0x7fffffffLL) return false;
    p.div_pairs = make_fastdiv((unsigned)p.pairs);
    p.div_hkv = make_fastdiv((unsigned)(p.Hq / p.G));
    p.div_sink_chunks = make_fastdiv((unsigned)p.sink_chunks);
    p.div_others = make_fastdiv((unsigned)(p.tiles > p.sink_tiles ? p.tiles - p.sink_tiles : 1));
    return true;
}

// (Tiles have several chunks only where the call has few of them: with chunks > 1 there are below 2 kFillItems tiles, or chunks of
// tiles of sinks, and rounding adds at most one chunk to each.  16 MiB are never reached.)
long long key_weights_workspace_bytes(const KeyWeightsParams &p) {
    const long long items = p.chunks > 1 ? p.items : p.sink_chunks > 1 ? (long long)p.pairs * p.sink_items : 0;
    return items * kKeyTile * (long long)sizeof(float);
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
