// Eviction from a key/value cache by weight (gfx950): of the L rows of a sequence's KV head the first n_sink, the last n_recent and
// the heaviest others stay, n_keep in all, and close up in their order; equal weights: the first rows stay.
//
// Two kernels:
//   * Selection, a workgroup per (sequence, KV head): the weights as whole numbers of the same order; the least one that stays is
//     found digit by digit (11, 11 and 10 bits) from counts in LDS, then every row's place from the counts of stayers before it.
//     Writes `kept` and moves the weights.
//   * Moves of K and V in place.  A row only ever moves down, so a workgroup that goes through the kept rows from the first on,
//     reads a block of rows, waits until all its reads are done and only then writes them overwrites nothing that is still
//     wanted.  Different columns of the rows do not meet: a workgroup takes a slice of a few bytes of every row, of K or of V, of
//     one head.
// Bound by memory: each row that moves is read and written once.
#include "swaa_cache_ops.h"

namespace swaa {
namespace {

constexpr int kSThreads = 1024;
constexpr int kSWaves = kSThreads / 64;
constexpr int kSegment = 256;                             // rows of a wave's step, four to a lane
constexpr int kStep = kSWaves * kSegment;                 // rows of a workgroup's step
constexpr int kSteps = 8;                                 // steps of a round, whose weights are in registers
constexpr int kRound = kSteps * kStep;
constexpr int kBins = 2048;
constexpr int kCopies = 4;                                // of the bins: lanes of equal weights seldom meet in one

// Weights as whole numbers of the same order: -0 is 0, everything that is not a number weighs most.  (On the bits: the build does
// not honour NaNs.)
__device__ __forceinline__ unsigned order_of(unsigned bits) {
    if ((bits & 0x7fffffffu) > 0x7f800000u) return ~0u;
    if (bits == 0x80000000u) bits = 0;
    return bits & 0x80000000u ? ~bits : bits | 0x80000000u;
}

// Exclusive sum over the workgroup's threads of x; `all`: of all of them.
__device__ __forceinline__ unsigned block_exclusive(unsigned x, unsigned *scratch, unsigned &all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const unsigned incl = wave_inclusive_scan(x);
    if (lane == 63) scratch[wave] = incl;
    __syncthreads();
    unsigned before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < kSWaves; ++w) {
        const unsigned n = scratch[w];
        before += w < wave ? n : 0u;
        all += n;
    }
    __syncthreads();
    return before + incl - x;
}

__global__ __launch_bounds__(kSThreads) void swaa_evict_select_kernel(const EvictParams p) {
    __shared__ unsigned bins[kCopies][kBins];
    __shared__ unsigned scratch[kSWaves], found[2];
    __shared__ unsigned heavier[kSteps * kSWaves], equal[kSteps * kSWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const unsigned pair = blockIdx.x, b = fastdiv(pair, p.div_hkv), kvh = pair - b * (unsigned)p.Hkv;
    const int n = p.seq_lens ? max(min(p.seq_lens[b], p.Nk), 0) : p.Nk;
    int *kept = p.kept + (long long)pair * p.n_keep;
    if (n <= p.n_keep) {
        for (int i = tid; i < p.n_keep; i += kSThreads) kept[i] = i < n ? i : -1;
        return;
    }
    float *weights = p.weights + b * p.w_sb + kvh * p.w_sh;
    const unsigned *bits_of = reinterpret_cast<const unsigned *>(weights);
    const int lo = p.n_sink, hi = n - p.n_recent;                          // rows that are judged
    const unsigned wanted = (unsigned)(p.n_keep - p.n_sink - p.n_recent);  // of which stay (fewer than there are)
    const int rounds = (n + kRound - 1) / kRound;

    // element e (0 .. 3) of step s of a round: row round * kRound + s * kStep + wave * kSegment + 64 e + lane
    unsigned raw[kSteps][4];
    auto row_of = [&](int round, int s, int e) { return round * kRound + s * kStep + wave * kSegment + 64 * e + lane; };
    auto load_round = [&](int round) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = row_of(round, s, e);
                raw[s][e] = i < n ? bits_of[i] : 0u;
            }
    };
    load_round(0);

    // ---- the least weight that stays, from its highest bits down
    unsigned prefix = 0, mask = 0, left = wanted;  // `left`: how many of those with the prefix stay
    if (wanted > 0) {
        const int shifts[3] = {21, 10, 0}, widths[3] = {11, 11, 10};
        for (int d = 0; d < 3; ++d) {
            const int shift = shifts[d];
            const unsigned digits = 1u << widths[d];
            for (int i = tid; i < kCopies * kBins; i += kSThreads) bins[0][i] = 0;
            __syncthreads();
            for (int round = 0; round < rounds; ++round) {
                if (rounds > 1) load_round(round);
#pragma unroll
                for (int s = 0; s < kSteps; ++s) {
                    if (round * kRound + s * kStep >= hi) break;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int i = row_of(round, s, e);
                        const unsigned u = order_of(raw[s][e]);
                        if (i >= lo && i < hi && (u & mask) == prefix) atomicAdd(&bins[lane % kCopies][(u >> shift) & (digits - 1)], 1u);
                    }
                }
            }
            __syncthreads();
            // thread t: digits digits - 1 - 2 t and the one below, the highest first
            unsigned c[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int digit = (int)digits - 1 - 2 * tid - k;
                c[k] = 0;
                if (digit >= 0)
#pragma unroll
                    for (int copy = 0; copy < kCopies; ++copy) c[k] += bins[copy][digit];
            }
            unsigned all;
            const unsigned before = block_exclusive(c[0] + c[1], scratch, all);
            if (before < left && left <= before + c[0] + c[1]) {
                const bool first = left <= before + c[0];
                found[0] = digits - 1 - 2 * tid - (first ? 0 : 1);
                found[1] = left - before - (first ? 0 : c[0]);
            }
            __syncthreads();
            prefix |= found[0] << shift;
            mask |= (digits - 1) << shift;
            left = found[1];
            __syncthreads();
        }
    }

    // ---- places: stayers are the pinned rows, the heavier ones and the first `left` of the equal ones
    unsigned base_heavier = 0, base_equal = 0;
    for (int round = 0; round < rounds; ++round) {
        if (rounds > 1) load_round(round);
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            unsigned nh = 0, ne = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = row_of(round, s, e);
                const unsigned u = order_of(raw[s][e]);
                const bool judged = i >= lo && i < hi, pinned = i < n && !judged;
                nh += __popcll(__ballot(pinned || (wanted > 0 && judged && u > prefix)));
                ne += __popcll(__ballot(wanted > 0 && judged && u == prefix));
            }
            if (lane == 0) {
                heavier[s * kSWaves + wave] = nh;
                equal[s * kSWaves + wave] = ne;
            }
        }
        __syncthreads();
        // (the round's segments: their sums by the first threads)
        const bool has = tid < kSteps * kSWaves;
        unsigned all_heavier, all_equal;
        const unsigned eh = block_exclusive(has ? heavier[tid] : 0u, scratch, all_heavier);
        const unsigned ee = block_exclusive(has ? equal[tid] : 0u, scratch, all_equal);
        if (has) {
            heavier[tid] = eh;
            equal[tid] = ee;
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            if (round * kRound + s * kStep >= n) break;
            unsigned h = base_heavier + heavier[s * kSWaves + wave], q = base_equal + equal[s * kSWaves + wave];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = row_of(round, s, e);
                const unsigned u = order_of(raw[s][e]);
                const bool judged = i >= lo && i < hi, pinned = i < n && !judged;
                const bool is_heavier = pinned || (wanted > 0 && judged && u > prefix), is_equal = wanted > 0 && judged && u == prefix;
                const unsigned long long bh = __ballot(is_heavier), bq = __ballot(is_equal);
                const unsigned long long below = (1ull << lane) - 1ull;
                const unsigned my_h = h + __popcll(bh & below), my_q = q + __popcll(bq & below);
                if (is_heavier || (is_equal && my_q < left)) {
                    const unsigned place = my_h + min(my_q, left);
                    kept[place] = i;
                    // (a row moves down at most: in this round the weights are in registers, and earlier ones have been read)
                    weights[place] = __uint_as_float(raw[s][e]);
                }
                h += __popcll(bh);
                q += __popcll(bq);
            }
        }
        base_heavier += all_heavier;
        base_equal += all_equal;
        __syncthreads();
    }
    for (int i = p.n_keep + tid; i < n; i += kSThreads) weights[i] = 0.f;
}

constexpr int kMThreads = 256;
constexpr int kMRows = 8;  // of a thread, on the way at a time

// kLanes: lanes of 16 bytes that make a slice of a row.
template <int kLanes>
__global__ __launch_bounds__(kMThreads) void swaa_evict_move_kernel(const EvictParams p, int slices) {
    constexpr int kStride = kMThreads / kLanes;
    const int tid = threadIdx.x;
    // pairs in turn: the slices of a row share a die's L2 (where the pairs are a multiple of the dies)
    const unsigned pairs = (unsigned)(p.B * p.Hkv), pair = blockIdx.x % pairs, rest = blockIdx.x / pairs;
    const int slice = (int)(rest % (unsigned)slices), of_v = (int)(rest / (unsigned)slices);
    const unsigned b = fastdiv(pair, p.div_hkv), kvh = pair - b * (unsigned)p.Hkv;
    if (rest == 0 && kvh == 0 && tid == 0 && p.new_lens) {
        // (no other thread of this kernel reads the lengths: they may be the same array)
        const int n = p.seq_lens ? max(min(p.seq_lens[b], p.Nk), 0) : p.Nk;
        p.new_lens[b] = min(n, p.n_keep);
    }
    const Rows &t = of_v ? p.v : p.k;
    const int *kept = p.kept + (long long)pair * p.n_keep;
    const int chunk = slice * kLanes + tid % kLanes;
    const bool in_row = 8 * chunk < p.D;
    const int limit = min(p.n_keep, p.Nk);
    for (int first = p.n_sink; first < limit; first += kMRows * kStride) {
        u32x4 data[kMRows];
        char *dst[kMRows];
#pragma unroll
        for (int r = 0; r < kMRows; ++r) {
            const int i = first + r * kStride + tid / kLanes;
            const int from = i < limit && in_row ? kept[i] : -1;
            dst[r] = nullptr;
            data[r] = u32x4{0, 0, 0, 0};
            if (from > i) {
                bool inside, unused;
                const long long at = cache_row(p.pages, t, (int)b, 0, i, false, inside), src = cache_row(p.pages, t, (int)b, 0, from, false, unused);
                char *base = t.ptr + 2 * (kvh * t.sh + 8 * chunk);
                if (inside) dst[r] = base + 2 * at;
                data[r] = *reinterpret_cast<const u32x4 *>(base + 2 * src);
            }
        }
        // every read of this block of rows is done, in all waves, before the first write
#pragma unroll
        for (int r = 0; r < kMRows; ++r) asm volatile("" ::"v"(data[r]));
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kMRows; ++r)
            if (dst[r]) *reinterpret_cast<u32x4 *>(dst[r]) = data[r];
    }
}

}  // namespace

hipError_t launch_evict(const EvictParams &p, hipStream_t stream) {
    const unsigned pairs = (unsigned)(p.B * p.Hkv);
    swaa_evict_select_kernel<<<dim3(pairs), dim3(kSThreads), 0, stream>>>(p);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    const int lanes = 4, slices = (p.D / 8 + lanes - 1) / lanes;
    swaa_evict_move_kernel<4><<<dim3(pairs * 2 * (unsigned)slices), dim3(kMThreads), 0, stream>>>(p, slices);
    return hipGetLastError();
}

}  // namespace swaa
