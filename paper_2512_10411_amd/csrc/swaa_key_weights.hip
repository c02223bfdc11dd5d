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
//   * Few rows (a decode step): the read of K is all there is: 131072 keys of 8 heads in 54 us, 4.9 TB/s.  Many: matrix and
//     exponential work, one beside the other (16 MFMA, 16 exponentials and 32 multiply-adds of a tile column take 406 cycles of which
//     the MFMA have 256): 1121 TFLOP/s for 16384 rows of one head on 32768 keys, where few tiles have a mask's edge in them.
#include "swaa_cache_ops.h"

namespace swaa {
namespace {

constexpr int kWThreads = 256;
// Columns a workgroup goes through at least, if there are as many (us for 256, 512, 1024; 32 heads: 2048 rows with a window of 512 37.2, 34.8,
// 49.2; 4096 with 256 57.4, 48.8, 61.3; 1024 that see 4096 keys 47.4, 44.9, 49.5).
constexpr int kMinChunk = 512;
// A wave has 32 keys instead of 64 where there are few columns and, in all pairs together, few keys, which would be workgroups for
// part of the chip only; or for a decode step's columns at any length (32 keys against 64, us: 64 rows of 32 heads on 32768 keys of 8 32.9
// and 34.2, on 131072 104 and 94; 4 x 64 rows on 4096 18.4 and 20.4; one row on 4096 4.2 and 5.6, on 131072 49.2 and 50.6).
constexpr int kFewColumns = 256, kStepColumns = 16;
constexpr long long kFewKeys = 1 << 18;
constexpr int kListedWgs = 1024;  // workgroups that go through a list of tiles (one per tile of the longest sequence instead: 47.8 -> 39.0 us, 16 of 0.2-16k)
constexpr int kFillItems = 4096;  // workgroups that a call should have (2048, 4096, 6144: 16384 rows of 32 heads with a window of 2048
                                  // 337, 328, 334 us, 8001 rows of 40 heads that see all 350, 348, 354)

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
// Sequences of different lengths whose tiles are whole (p.listed): item `id` of the list that holds every sequence's own tiles, one
// sequence behind the other; false behind its end.  Every wave reads the lengths, 64 at a time.
__device__ __forceinline__ bool listed_item(const KeyWeightsParams &p, unsigned id, int key_tile, Item &w) {
    const int lane = threadIdx.x & 63, hkv = p.pairs / p.seq.B;
    const unsigned tile = fastdiv(id, p.div_hkv);
    unsigned before = 0;
    for (int c0 = 0; c0 < p.seq.B; c0 += 64) {
        int nq, nk;
        sequence(p.seq, min(c0 + lane, p.seq.B - 1), nq, nk);
        const unsigned incl = wave_inclusive_scan(c0 + lane < p.seq.B ? (unsigned)(nk + key_tile - 1) / (unsigned)key_tile : 0u);
        const unsigned all = wave_read_lane(incl, 63);
        if (tile - before < all) {
            const int n = __popcll(__ballot(incl <= tile - before));  // sequences among these that end at or before the tile
            w.b = __builtin_amdgcn_readfirstlane(c0 + n);
            w.tile = __builtin_amdgcn_readfirstlane((int)(tile - before - (n ? wave_read_lane(incl, n - 1) : 0u)));
            w.kvh = (int)(id - tile * (unsigned)hkv);
            w.chunk = 0;
            w.whole = true;
            return true;
        }
        before += all;
    }
    return false;
}

// The columns of a tile, kCols to a stage: head by head, each one's rows from the start of a stage on, or, where a head has few, all
// heads' in a row.
template <int kCols>
struct Columns {
    bool by_head;
    int per_head, stages;
    __host__ __device__ Columns(int n_all, int G) {
        by_head = n_all >= 64;
        per_head = (n_all + kCols - 1) / kCols;
        stages = by_head ? G * per_head : (G * n_all + kCols - 1) / kCols;
    }
};

// LDS: two buffers of what the keys are told about each column -- its lse in log2 units, `pos` and `lo` (its row sees the keys up to
// pos that lie above lo, and the sinks; pos -1: nothing, no such column) -- then two of kCols rows of Q without padding.  16-byte
// chunk c of row r lies at chunk c ^ turn(r), so that the equal chunks of 16 rows lie in different banks (64 of 4 bytes); the copies
// apply it on the global side.
__host__ __device__ constexpr int stage_cols(int D) { return D <= 128 ? 64 : 32; }
template <int D>
struct Stage {
    static constexpr int kCols = stage_cols(D);
    static constexpr int kRowB = D * 2, kBufB = kCols * kRowB;
    static constexpr int kLse = 0, kPos = kLse + 2 * kCols * 4, kLo = kPos + 2 * kCols * 4;  // byte addresses
    static constexpr int kRows = kLo + 2 * kCols * 4;
    static constexpr int kBytes = kRows + 2 * kBufB, kOneStage = kRows + kBufB;  // (calls of one stage have no use for the second buffer)
    static __device__ __forceinline__ int turn(int r) { return D % 128 == 0 ? r & 15 : D % 64 == 0 ? (r >> 1) & 7 : (r >> 2) & 3; }
};

typedef char __attribute__((address_space(3))) LdsByte;
__device__ __forceinline__ LdsByte *lds_at(uint32_t addr) { return (LdsByte *)(uintptr_t)addr; }
template <typename X>
__device__ __forceinline__ X lds_word(const LdsByte *at) { return *(const X __attribute__((address_space(3))) *)at; }
template <typename X>
__device__ __forceinline__ void lds_put(LdsByte *at, X x) { *(X __attribute__((address_space(3))) *)at = x; }

// One item: kM blocks of 16 keys to a wave.
template <int D, bool kF16, int kM>
__device__ __forceinline__ void weigh_item(const KeyWeightsParams &p, const Item &it, unsigned id) {
    using T = Stage<D>;
    constexpr int kWaveKeys = 16 * kM;
    constexpr int KS = D / 32;                  // k-steps of a product
    constexpr int kCols = T::kCols, kWaveCols = kCols / 4;  // columns that a wave brings
    constexpr int kChunks = D / 8;              // of 16 bytes in a row
    constexpr int kCopies = (kWaveCols * kChunks + 63) / 64;  // wave instructions for them
    constexpr int kTile = 4 * kWaveKeys;

    int nq, nk;
    sequence(p.seq, it.b, nq, nk);
    // (the same in all lanes; the compiler has to know it for the addresses of the copies)
    nq = __builtin_amdgcn_readfirstlane(nq);
    nk = __builtin_amdgcn_readfirstlane(nk);
    const int k0 = it.tile * kTile;
    if (k0 >= nk) return;
    const int P = p.n_prompts ? __builtin_amdgcn_readfirstlane(max(p.n_prompts[it.b], 0)) : p.P;
    const int q_row0 = p.seq.cu_q ? __builtin_amdgcn_readfirstlane(p.seq.cu_q[it.b]) : 0;  // of packed sequences
    const SeenBy seen = seen_by(k0, min(k0 + kTile, nk), nq, nk, p.W, p.S, P);
    const Columns<kCols> cols(seen.n_all, p.G);
    const int s_begin = it.chunk * p.chunk_stages * (64 / kCols), s_end = min(cols.stages, s_begin + p.chunk_stages * (64 / kCols));
    if (it.chunk > 0 && s_begin >= s_end) return;

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

    // ---- columns, a stage at a time; a wave brings kWaveCols of them
    const char *q_base = p.q.ptr + 2 * ((packed ? 0 : it.b * p.q.sb) + it.kvh * (long long)p.G * p.q.sh +
                                        q_row0 * p.q.sn);
    const float *lse_base = p.lse + (packed ? q_row0 : it.b * p.lse_sb) + it.kvh * (long long)p.G * p.lse_sh;
    const int off = nk - nq;
    // (of instruction i: row 64 i + lane of kChunks chunks each of the wave's columns, chunk of LDS, and its address behind row 0's)
    uint32_t copy_at[kCopies];
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
        const int id = 64 * i + lane, c = wave * kWaveCols + id / kChunks;
        copy_at[i] = (uint32_t)(c * (int)p.q.sn * 2 + 16 * (id % kChunks ^ T::turn(c)));
    }
    int head = 0, index = 0;  // of the stage: its first column
    auto go_to = [&](int stage) {
        head = cols.by_head ? stage / cols.per_head : 0;
        index = kCols * (stage - (cols.by_head ? head * cols.per_head : 0));
    };
    // Rows of consecutive places in memory, all there: the usual stage.  row0: the first.
    int row0 = 0;
    bool straight = false;
    int valid = 0;  // columns of the stage
    float lse = 0.f;
    int pos = 0;
    auto issue_stage = [&](int buf) {
        valid = min(kCols, (cols.by_head ? seen.n_all : seen.n_all * p.G) - index);
        straight = cols.by_head && valid == kCols && (index + kCols <= seen.n || index >= seen.n);
        row0 = seen.row(index);
        const uint32_t to = (uint32_t)(T::kRows + buf * T::kBufB + wave * kWaveCols * T::kRowB);
        const int mine = wave * kWaveCols + lane % kWaveCols;
        if (straight) {
            const char *src = q_base + 2 * (head * p.q.sh + row0 * p.q.sn);
            lse = (lse_base + head * p.lse_sh + row0)[mine];
            pos = off + row0 + mine;
#pragma unroll
            for (int i = 0; i < kCopies; ++i) {
                if (kWaveCols * kChunks % 64 != 0 && 64 * i + lane >= kWaveCols * kChunks) break;
                asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(copy_at[i]), "s"(src), "s"(to + 1024 * i) : "memory");
            }
        } else {
            // column c of the stage; those behind the last one repeat it
            auto locate = [&](int c, int &h, int &r) {
                c = index + min(c, valid - 1);
                h = cols.by_head ? head : c / seen.n_all;
                r = seen.row(cols.by_head ? c : c - h * seen.n_all);
            };
            int h, r, lane_here = lane;
            asm volatile("" : "+v"(lane_here));  // (what this path needs is worked out here: kept from before the loop it would cost the other one its registers)
            locate(wave * kWaveCols + lane_here % kWaveCols, h, r);
            lse = lse_base[h * p.lse_sh + r];
            pos = mine < valid ? off + r : -1;
#pragma unroll
            for (int i = 0; i < kCopies; ++i) {
                const int id = 64 * i + lane_here, c = wave * kWaveCols + id / kChunks;
                if (kWaveCols * kChunks % 64 != 0 && id >= kWaveCols * kChunks) break;
                locate(c, h, r);
                const char *src = q_base + 2 * (h * p.q.sh + r * p.q.sn) + 16 * (id % kChunks ^ T::turn(c));
                asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(src), "s"(to + 1024 * i) : "memory");
            }
        }
    };
    auto put_columns = [&](int buf) {
        LdsByte *const at = lds_at((uint32_t)(T::kLse + 4 * (buf * kCols + wave * kWaveCols + lane)));
        // (a row whose scores are all -infinity gives no weight)
        const bool none = pos < 0 || opaque_bits(lse) == 0xff800000u;
        if (lane < kWaveCols) {
            lds_put<float>(at, none ? INFINITY : lse * 1.44269504088896340736f);
            lds_put<int>(at + (T::kPos - T::kLse), none ? -1 : pos);
            lds_put<int>(at + (T::kLo - T::kLse), pos >= P ? -1 : pos - p.W);
        }
    };

    // S of 16 columns, whose operands lie at `at`[k-step] + offset
    uint32_t q_at[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) q_at[ks] = (uint32_t)(l16 * T::kRowB + (((4 * ks + quad) ^ T::turn(l16)) << 4));
    auto products = [&](LdsByte *const (&at)[KS], int offset, f32x4 (&s)[kM]) __attribute__((always_inline)) {
#pragma unroll
        for (int m = 0; m < kM; ++m) s[m] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const u32x4 qf = lds_word<u32x4>(at[ks] + offset);
#pragma unroll
            for (int m = 0; m < kM; ++m) s[m] = mfma16<kF16>(kf[m][ks], qf, s[m]);
        }
    };
    if (s_begin < s_end) {
        go_to(s_begin);
        issue_stage(0);
        put_columns(0);
    }
    int buf = 0;
    for (int stage = s_begin; stage < s_end; ++stage, buf ^= 1) {
        __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0): this wave's share of the stage has landed, and it has read the one before
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();        // everybody's; and everybody is done with the one before
        asm volatile("" ::: "memory");
        // do all the stage's columns see all the wave's keys?
        const int pos0 = off + row0, pos1 = pos0 + kCols - 1;
        const bool all = straight && pos0 >= wk0 + kWaveKeys - 1 && (pos0 >= P || min(pos1, P - 1) - p.W < wk0 || wk0 + kWaveKeys <= p.S);
        // does any of them see any?  (Rows at the edges of the tile's window; beside the sinks, the tile's other waves.)
        const bool none = straight && (pos1 < wk0 || (pos1 < P && pos0 - p.W >= wk0 + kWaveKeys - 1 && wk0 >= p.S));
        const int units = none ? 0 : (valid + 15) / 16;
        const bool more = stage + 1 < s_end;
        if (more) {
            index += kCols;
            if (cols.by_head && index >= seen.n_all) {
                index = 0;
                ++head;
            }
            issue_stage(buf ^ 1);
        }
        LdsByte *at[KS], *const col_at = lds_at((uint32_t)(T::kLse + 4 * (buf * kCols + l16)));
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) at[ks] = lds_at(q_at[ks] + (uint32_t)(T::kRows + buf * T::kBufB));
        if (all) {
#pragma unroll
            for (int t = 0; t < kCols / 16; ++t) {
                f32x4 s[kM];
                const float lse2 = lds_word<float>(col_at + 64 * t);
                products(at, 16 * t * T::kRowB, s);
#pragma unroll
                for (int m = 0; m < kM; ++m)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[m][e] += __builtin_amdgcn_exp2f(s[m][e] * p.scale_log2 - lse2);
            }
        } else {
            for (int t = 0; t < units; ++t) {
                const float lse2 = lds_word<float>(col_at + 64 * t);
                const int cpos = lds_word<int>(col_at + 64 * t + (T::kPos - T::kLse)), clo = lds_word<int>(col_at + 64 * t + (T::kLo - T::kLse));
                f32x4 s[kM];
                products(at, 16 * t * T::kRowB, s);
                int first = wk0 + 4 * quad;
                asm volatile("" : "+v"(first));  // (as above)
#pragma unroll
                for (int m = 0; m < kM; ++m)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = first + 16 * m + e;
                        const bool sees = key <= cpos && (key > clo || key < p.S);
                        const float x = __builtin_amdgcn_exp2f(s[m][e] * p.scale_log2 - lse2);
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
    if (l16 >= 4 * kM) return;
    if (!it.whole) {
        p.partial[(long long)id * kTile + of_tile] = mine;
    } else if (k0 + of_tile < nk) {
        float *w = p.weights + it.b * p.w_sb + it.kvh * p.w_sh + k0 + of_tile;
        *w = p.decay != 0.f ? p.decay * *w + mine : mine;
    }
}

// Waves of a SIMD: what the registers allow.
constexpr int weigh_waves(int D, int kM) { return D > 128 ? 2 : kM == 2 ? 5 : 3; }
template <int D, bool kF16, int kM>
__global__ __launch_bounds__(kWThreads, weigh_waves(D, kM)) void swaa_key_weights_kernel(const KeyWeightsParams p) {
    fetch_args<KeyWeightsParams>();
    weigh_item<D, kF16, kM>(p, item_of(p, blockIdx.x), blockIdx.x);
}
template <int D, bool kF16, int kM>
__global__ __launch_bounds__(kWThreads, kM == 2 && D <= 128 ? 4 : weigh_waves(D, kM)) void swaa_key_weights_listed_kernel(const KeyWeightsParams p) {
    fetch_args<KeyWeightsParams>();
    Item it;
    for (unsigned id = blockIdx.x; listed_item(p, id, 64 * kM, it); id += gridDim.x) {
        weigh_item<D, kF16, kM>(p, it, id);
        __syncthreads();  // (the next item's columns go where this one's were)
    }
}

// Chunks of a tile's columns added up in their order (tiles of several chunks: those of the sinks, or all).
__global__ __launch_bounds__(256) void swaa_key_weights_merge_kernel(const KeyWeightsParams p) {
    const unsigned tile = fastdiv(blockIdx.x, p.div_pairs), pair = blockIdx.x - tile * (unsigned)p.pairs;
    const int b = (int)fastdiv(pair, p.div_hkv), kvh = (int)(pair - (unsigned)b * (unsigned)(p.pairs / p.seq.B));
    int nq, nk;
    sequence(p.seq, b, nq, nk);
    const int k0 = (int)tile * p.key_tile, key = k0 + (int)threadIdx.x;
    if (key >= nk) return;
    const int P = p.n_prompts ? max(p.n_prompts[b], 0) : p.P;
    const SeenBy seen = seen_by(k0, min(k0 + p.key_tile, nk), nq, nk, p.W, p.S, P);
    const bool narrow = stage_cols(p.D) == 32;
    const int stages = narrow ? Columns<32>(seen.n_all, p.G).stages : Columns<64>(seen.n_all, p.G).stages;
    const int of_chunk = p.chunk_stages * (narrow ? 2 : 1);
    const bool has_sinks = (int)tile < p.sink_tiles;
    // its first chunk's place among the pair's items, and from chunk to chunk
    const long long first = has_sinks ? (long long)tile * p.sink_chunks : p.sink_items + ((long long)tile - p.sink_tiles);
    const long long step = (has_sinks ? 1LL : p.tiles - p.sink_tiles) * p.pairs * p.key_tile;
    const int chunks = has_sinks ? p.sink_chunks : p.chunks;
    const float *src = p.partial + (first * p.pairs + pair) * p.key_tile + threadIdx.x;
    float x = src[0];
    for (int c = 1; c < chunks && c * of_chunk < stages; ++c) x += src[c * step];
    float *w = p.weights + b * p.w_sb + kvh * p.w_sh + key;
    *w = p.decay != 0.f ? p.decay * *w + x : x;
}

template <int D, bool kF16, int kM>
hipError_t launch_one(const KeyWeightsParams &p, hipStream_t stream) {
    static_assert(Stage<D>::kBytes <= 64 * 1024, "");
    const int lds = p.one_stage ? Stage<D>::kOneStage : Stage<D>::kBytes;
    if (p.listed)
        swaa_key_weights_listed_kernel<D, kF16, kM><<<dim3((unsigned)(p.items < kListedWgs ? p.items : kListedWgs)), dim3(kWThreads), lds, stream>>>(p);
    else
        swaa_key_weights_kernel<D, kF16, kM><<<dim3((unsigned)p.items), dim3(kWThreads), lds, stream>>>(p);
    return hipGetLastError();
}

template <int D>
hipError_t launch(const KeyWeightsParams &p, hipStream_t stream) {
    const hipError_t err = p.key_tile == 128 ? (p.fp16 ? launch_one<D, true, 2>(p, stream) : launch_one<D, false, 2>(p, stream))
                                             : (p.fp16 ? launch_one<D, true, 4>(p, stream) : launch_one<D, false, 4>(p, stream));
    const int merged = p.chunks > 1 ? p.tiles : p.sink_chunks > 1 ? p.sink_tiles : 0;
    if (err != hipSuccess || merged == 0) return err;
    swaa_key_weights_merge_kernel<<<dim3((unsigned)((long long)p.pairs * merged)), dim3((unsigned)p.key_tile), 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace

// The columns of all tiles, shared out in chunks of one length so that the call has as many workgroups as the chip wants.
bool plan_key_weights(KeyWeightsParams &p) {
    const int Nq = p.seq.Nq, Nk = p.seq.Nk;
    if ((long long)p.G * (Nq + 64LL) > 0x3fffffffLL) return false;
    p.pairs = p.seq.B * (p.Hq / p.G);
    const long long columns = (long long)p.G * Nq;
    p.key_tile = columns <= kStepColumns || (columns <= kFewColumns && (long long)p.pairs * Nk <= kFewKeys) ? 128 : 256;
    p.one_stage = columns <= stage_cols(p.D);
    p.tiles = (Nk + p.key_tile - 1) / p.key_tile;
    // stages (of 64 columns) of a tile seen by n rows, at most
    auto stages_of = [&](long long n) { return Columns<64>((int)(n < Nq ? n : Nq), p.G).stages; };
    const int most = stages_of(Nq);
    // rows that see a tile without sinks: those of its window, and generated ones (of sequences with prompt lengths of their own: maybe all)
    const long long generated = p.n_prompts ? Nk : Nk - p.P;
    const long long of_window = (long long)p.W + p.key_tile - 1 + generated;
    const int usual = stages_of(of_window);
    p.sink_tiles = usual < most ? (p.S + p.key_tile - 1) / p.key_tile : 0;
    const bool ramp = of_window >= Nq && Nq > p.key_tile;  // (a whole prompt's rows: the last tiles see few)
    const long long all = p.pairs * ((long long)(p.tiles - p.sink_tiles) * (ramp ? usual / 2 + 1 : usual) + (long long)p.sink_tiles * most);
    const long long chunk = (all + kFillItems - 1) / kFillItems;
    p.chunk_stages = (int)(chunk > kMinChunk / 64 ? chunk : kMinChunk / 64);
    p.chunks = (usual + p.chunk_stages - 1) / p.chunk_stages;
    p.sink_chunks = (most + p.chunk_stages - 1) / p.chunk_stages;
    p.sink_items = p.sink_tiles * p.sink_chunks;
    p.items = (long long)p.pairs * (p.sink_items + (long long)(p.tiles - p.sink_tiles) * p.chunks);
    p.listed = p.chunks == 1 && p.sink_chunks == 1 && (p.seq.seq_lens || p.seq.cu_k);
    if (p.items > 0x7fffffffLL - kListedWgs) return false;
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
    return items * p.key_tile * (long long)sizeof(float);
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
