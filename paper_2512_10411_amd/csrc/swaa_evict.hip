// Eviction from a key/value cache by weight (gfx950): of the L rows of a sequence's KV head the first n_sink, the last n_recent and
// the heaviest others stay, n_keep in all, and close up in their order; equal weights: the first rows stay.
//
//   * Selection: the weights as whole numbers of the same order; the least one that stays is found digit by digit (11, 11 and 10
//     bits) from counts in LDS, the last few candidates by ranking one against the others, then every row's place from the counts of
//     stayers before it.  A workgroup to a (sequence, KV head) pair; long sequences of few pairs are shared out, in three steps.
//   * Moves of K and V in place.  A row only ever moves down, so a workgroup that goes through the kept rows from the first on,
//     reads a block of rows, waits until all its reads are done and only then writes them overwrites nothing that is still
//     wanted.  Different columns of the rows do not meet: a workgroup takes a slice of a few bytes of every row, of K or of V, of
//     one head; the weights are one more.  Where half the rows leave or more, those that come from behind the first n_keep are left
//     to a kernel of their own behind it, in any order: nothing is written where they stand.
// Bound by memory: each row that moves is read and written once.  16 sequences of 900 to 1152 rows, 8 heads of 128, cut to 1024:
// 31 us, of it 7 for the selection; one of 65536 cut to 16384: 64 us, of it 20 for the selection, 15 for rows from near by, in order,
// and 22 for those from far (100 MB that come and go, 4.6 TB/s).
#include "swaa_cache_ops.h"

namespace swaa {
namespace {

constexpr int kSThreads = 1024;
constexpr int kSWaves = kSThreads / 64;
constexpr int kSegment = 256;              // rows of a wave's step, four to a lane
constexpr int kStep = kSWaves * kSegment;  // rows of a workgroup's step
constexpr int kBins = 2048, kDigitBits = 11;
constexpr int kCopies = 4;                 // of the bins, side by side: lanes of equal weights seldom meet in one, nor in a bank
constexpr int kMaxSteps = 8;               // of a round
constexpr int kFew = 256;                  // candidates that are ranked one against the other

// Rows as whole numbers that the heaviest ones have the largest of: a weight's bits in its order (-0 is 0, everything that is not a
// number weighs most), above them the rows that stay in any case, and 0 where there is no row.  (On the bits: the build does not
// honour NaNs.)
constexpr unsigned kPinned = ~0u, kNotANumber = ~0u - 1u;
__device__ __forceinline__ unsigned order_of(unsigned bits) {
    if ((bits & 0x7fffffffu) > 0x7f800000u) return kNotANumber;
    if (bits == 0x80000000u) bits = 0;
    return bits & 0x80000000u ? ~bits : bits | 0x80000000u;
}

// What a selecting workgroup has in LDS.
struct SelectLds {
    __attribute__((aligned(16))) unsigned bins[kBins * kCopies];  // (or candidates, when the bins are done with)
    unsigned scratch[kSWaves], scratch2[kSWaves], found[4];
    unsigned heavier[kMaxSteps * kSWaves], equal[kMaxSteps * kSWaves];
};

// Exclusive sum over the workgroup's threads of x; `all`: of all of them.  Callers have a barrier between two calls.
__device__ __forceinline__ unsigned block_exclusive(unsigned x, unsigned *scratch, unsigned &all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const unsigned incl = wave_inclusive_scan(x);
    if (lane == 63) scratch[wave] = incl;
    __syncthreads();
    const unsigned waves = wave_inclusive_scan(lane < kSWaves ? scratch[lane] : 0u);
    all = wave_read_lane(waves, kSWaves - 1);
    const unsigned before = wave ? wave_read_lane(waves, wave - 1) : 0u;
    return before + incl - x;
}

// A (sequence, KV head) pair that is longer than n_keep rows; false: one that keeps all it has (`kept` says so, if `says`).
struct Head {
    int n, lo, hi;  // rows lo .. hi - 1 are judged
    int *kept;
    __amdgpu_buffer_rsrc_t words;  // its weights (a buffer of n words: what is read behind them is 0, without a branch around the read)
};
__device__ __forceinline__ bool head_of(const EvictParams &p, unsigned pair, bool says, Head &h) {
    const unsigned b = fastdiv(pair, p.div_hkv), kvh = pair - b * (unsigned)p.Hkv;
    h.n = p.seq_lens ? max(min(p.seq_lens[b], p.Nk), 0) : p.Nk;
    h.kept = p.kept + (long long)pair * p.n_keep;
    if (h.n <= p.n_keep) {
        if (says)
            for (int i = threadIdx.x; i < p.n_keep; i += kSThreads) h.kept[i] = i < h.n ? i : -1;
        return false;
    }
    h.lo = p.n_sink;
    h.hi = h.n - p.n_recent;
    h.words = __builtin_amdgcn_make_buffer_rsrc(p.weights + b * p.w_sb + kvh * p.w_sh, 0, 4 * h.n, 0x00027000);
    return true;
}

// Orders of kSteps steps of rows from row `begin` on: element e (0 .. 3) of step s is row first_row(begin, s) + 64 e + lane.
__device__ __forceinline__ int first_row(int begin, int s) { return begin + s * kStep + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) * kSegment; }
template <int kSteps>
__device__ __forceinline__ void load_orders(const Head &h, int begin, unsigned (&order)[kSteps][4]) {
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));  // (what depends on it is worked out here: kept from one look to the next it would need the registers)
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int e = 0; e < 4; ++e) order[s][e] = __builtin_amdgcn_raw_buffer_load_b32(h.words, 4 * (first_row(begin, s) + 64 * e + lane), 0, 0);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        const int first = first_row(begin, s);
#pragma unroll
        for (int e = 0; e < 4; ++e) order[s][e] = order_of(order[s][e]);
        if (first < h.lo || first + kSegment > h.hi) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = first + 64 * e + lane;
                order[s][e] = i >= h.n ? 0u : i < h.lo || i >= h.hi ? kPinned : order[s][e];
            }
        }
    }
}

// Thread t has the counts of bins 2047 - 2 t and the one below: finds the bin that holds the left-th from above.  found: the bin,
// how many of its own stay, how many it has, 0.
__device__ __forceinline__ void find_bin(const unsigned (&c)[2], unsigned left, SelectLds &lds) {
    unsigned all;
    const unsigned before = block_exclusive(c[0] + c[1], lds.scratch, all);
    if (before < left && left <= before + c[0] + c[1]) {
        const bool first = left <= before + c[0];
        lds.found[0] = kBins - 1 - 2 * threadIdx.x - (first ? 0 : 1);
        lds.found[1] = left - before - (first ? 0 : c[0]);
        lds.found[2] = first ? c[0] : c[1];
        lds.found[3] = 0;
    }
    __syncthreads();
}
__device__ __forceinline__ void clear_bins(SelectLds &lds) {
    static_assert(kCopies == 4 && kBins == 2 * kSThreads, "");
    u32x4 *const four = reinterpret_cast<u32x4 *>(lds.bins);
    four[threadIdx.x] = four[threadIdx.x + kSThreads] = u32x4{0, 0, 0, 0};
    __syncthreads();
}
__device__ __forceinline__ unsigned bin_count(const SelectLds &lds, int bin) {
    const u32x4 copies = reinterpret_cast<const u32x4 *>(lds.bins)[bin];
    return (copies[0] + copies[1]) + (copies[2] + copies[3]);
}

// The least order that stays: `left` of those with the bits `prefix` under `mask` do, the digit at `shift` is the next to be looked at.
// look(f) calls f(order) for all of a thread's rows.  On return prefix is that order, left how many of its equals stay.
template <typename Look>
__device__ __forceinline__ void find_least(Look look, unsigned &prefix, unsigned mask, unsigned &left, int shift, SelectLds &lds) {
    const int tid = threadIdx.x;
    while (mask != ~0u) {
        clear_bins(lds);
        unsigned *const mine = lds.bins + tid % kCopies;
        if (mask == 0)
            look([&](unsigned u) { atomicAdd(&mine[(u >> (32 - kDigitBits)) * kCopies], 1u); });
        else
            look([&](unsigned u) {
                if ((u & mask) == prefix) atomicAdd(&mine[((u >> shift) & (kBins - 1)) * kCopies], 1u);  // (the last digit has ten bits: the eleventh is the prefix's)
            });
        __syncthreads();
        const unsigned c[2] = {bin_count(lds, kBins - 1 - 2 * tid), bin_count(lds, kBins - 2 - 2 * tid)};
        find_bin(c, left, lds);
        prefix |= lds.found[0] << shift;
        mask |= ((1u << kDigitBits) - 1) << shift;
        left = lds.found[1];
        const unsigned candidates = lds.found[2];
        if (candidates <= (unsigned)kFew && mask != ~0u) {
            // each of them against all others
            unsigned *const few = lds.bins;
            look([&](unsigned u) {
                if ((u & mask) == prefix) few[atomicAdd(&lds.found[3], 1u)] = u;
            });
            __syncthreads();
            if (tid < (int)candidates) {
                const unsigned u = few[tid];
                unsigned above = 0, same = 0;
                for (unsigned i = 0; i < candidates; ++i) {
                    above += few[i] > u;
                    same += few[i] == u;
                }
                if (above < left && left <= above + same) {  // (every thread that holds it says the same)
                    lds.found[0] = u;
                    lds.found[1] = left - above;
                }
            }
            __syncthreads();
            prefix = lds.found[0];
            left = lds.found[1];
            mask = ~0u;
        }
        shift = shift > kDigitBits ? shift - kDigitBits : 0;
    }
}

// Places of the rows that stay among those from row `begin` on: the heavier ones do, and the first `left` of the equal ones.  base_*: of
// the rows before them.
template <int kSteps>
__device__ __forceinline__ void put_rows(const Head &h, int begin, const unsigned (&order)[kSteps][4], unsigned prefix, unsigned left,
                                         unsigned &base_heavier, unsigned &base_equal, SelectLds &lds) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        unsigned nh = 0, ne = 0;
        if (first_row(begin, s) < h.n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                nh += __popcll(__ballot(order[s][e] > prefix));
                ne += __popcll(__ballot(order[s][e] == prefix));
            }
        if (lane == 0) {
            lds.heavier[s * kSWaves + wave] = nh;
            lds.equal[s * kSWaves + wave] = ne;
        }
    }
    __syncthreads();
    // (the segments: their sums by the first threads)
    const bool has = tid < kSteps * kSWaves;
    unsigned all_heavier, all_equal;
    const unsigned eh = block_exclusive(has ? lds.heavier[tid] : 0u, lds.scratch, all_heavier);
    const unsigned ee = block_exclusive(has ? lds.equal[tid] : 0u, lds.scratch2, all_equal);
    if (has) {
        lds.heavier[tid] = eh;
        lds.equal[tid] = ee;
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        const int first = first_row(begin, s);
        if (first >= h.n) break;
        unsigned before = base_heavier + lds.heavier[s * kSWaves + wave], q = base_equal + lds.equal[s * kSWaves + wave];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const unsigned u = order[s][e];
            const unsigned long long bh = __ballot(u > prefix), bq = __ballot(u == prefix);
            unsigned place = before + min(q, left) + __builtin_amdgcn_mbcnt_hi((unsigned)(bh >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)bh, 0u));
            bool stays = u > prefix;
            if (bq) {
                const unsigned my_q = q + __builtin_amdgcn_mbcnt_hi((unsigned)(bq >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)bq, 0u));
                place += min(my_q, left) - min(q, left);
                stays = stays || (u == prefix && my_q < left);
                q += __popcll(bq);
            }
            if (stays) h.kept[place] = first + 64 * e + lane;
            before += __popcll(bh);
        }
    }
    base_heavier += all_heavier;
    base_equal += all_equal;
}

// One workgroup to a pair.  kSteps: steps of a round, whose rows' orders are in registers; longer sequences take several rounds and
// read their weights once more for each look at them.
template <int kSteps>
__global__ __launch_bounds__(kSThreads) void swaa_evict_select_kernel(const EvictParams p) {
    static_assert(kSteps <= kMaxSteps, "");
    __shared__ SelectLds lds;
    Head h;
    if (!head_of(p, blockIdx.x, true, h)) return;
    const int rounds = (h.n + kSteps * kStep - 1) / (kSteps * kStep);
    unsigned order[kSteps][4];
    auto look = [&](auto f) __attribute__((always_inline)) {
        for (int round = 0; round < rounds; ++round) {
            if (rounds > 1) load_orders<kSteps>(h, round * kSteps * kStep, order);
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                if (first_row(round * kSteps * kStep, s) >= h.n) break;
#pragma unroll
                for (int e = 0; e < 4; ++e) f(order[s][e]);
            }
        }
    };
    load_orders<kSteps>(h, 0, order);
    unsigned prefix = 0, left = (unsigned)p.n_keep, base_heavier = 0, base_equal = 0;
    find_least(look, prefix, 0u, left, 32 - kDigitBits, lds);
    for (int round = 0; round < rounds; ++round) {
        if (rounds > 1) load_orders<kSteps>(h, round * kSteps * kStep, order);
        put_rows<kSteps>(h, round * kSteps * kStep, order, prefix, left, base_heavier, base_equal, lds);
        __syncthreads();
    }
}

// ---- long sequences of few pairs: a workgroup to every kPartRows rows of a pair.  Counts of the first digit, then the rows of the digit
// that the least one has (the candidates) one part behind the other, then its other digits from those and the part's places. ----
constexpr int kPartSteps = 2, kPartRows = kPartSteps * kStep;
struct PartSpace {
    unsigned *counts, *candidates;  // [parts][bins], [Nk]
};
__device__ __forceinline__ PartSpace part_space(const EvictParams &p, unsigned pair) {
    unsigned *const at = p.select_space + (long long)pair * ((long long)p.parts * kBins + p.Nk + p.Nk % 2);  // (pairs of counts are read at once)
    return {at, at + (long long)p.parts * kBins};
}
// The digit of the least row that stays (found[0], as find_bin leaves it) and how many rows of the parts before `part` are above it
// and in it.
__device__ __forceinline__ void first_digit(const EvictParams &p, const PartSpace &space, int part, int parts, SelectLds &lds, unsigned &above, unsigned &in) {
    const int tid = threadIdx.x;
    unsigned c[2] = {0, 0}, mine[2] = {0, 0};  // of all parts, and of those before
    for (int i = 0; i < parts; ++i) {
        const uint2 two = *reinterpret_cast<const uint2 *>(space.counts + (long long)i * kBins + kBins - 2 - 2 * tid);
        c[0] += two.y;
        c[1] += two.x;
        mine[0] += i < part ? two.y : 0u;
        mine[1] += i < part ? two.x : 0u;
    }
    find_bin(c, (unsigned)p.n_keep, lds);
    const unsigned bin = lds.found[0];
    unsigned sums[2] = {0, 0};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const unsigned of = (unsigned)(kBins - 1 - 2 * tid - k);
        sums[0] += of > bin ? mine[k] : 0u;
        sums[1] += of == bin ? mine[k] : 0u;
    }
    block_exclusive(sums[0], lds.scratch2, above);
    __syncthreads();
    block_exclusive(sums[1], lds.scratch, in);
    __syncthreads();
}
__global__ __launch_bounds__(kSThreads) void swaa_evict_count_kernel(const EvictParams p) {
    __shared__ SelectLds lds;
    const unsigned pairs = (unsigned)(p.B * p.Hkv), pair = blockIdx.x % pairs, part = blockIdx.x / pairs;
    Head h;
    if (!head_of(p, pair, part == 0, h) || (int)part * kPartRows >= h.n) return;
    unsigned order[kPartSteps][4];
    load_orders<kPartSteps>(h, (int)part * kPartRows, order);
    clear_bins(lds);
#pragma unroll
    for (int s = 0; s < kPartSteps; ++s)
#pragma unroll
        for (int e = 0; e < 4; ++e) atomicAdd(&lds.bins[(order[s][e] >> (32 - kDigitBits)) * kCopies + threadIdx.x % kCopies], 1u);
    __syncthreads();
    unsigned *const out = part_space(p, pair).counts + (long long)part * kBins;
    for (int i = threadIdx.x; i < kBins; i += kSThreads) out[i] = bin_count(lds, i);
}
__global__ __launch_bounds__(kSThreads) void swaa_evict_gather_kernel(const EvictParams p) {
    __shared__ SelectLds lds;
    const unsigned pairs = (unsigned)(p.B * p.Hkv), pair = blockIdx.x % pairs, part = blockIdx.x / pairs;
    Head h;
    if (!head_of(p, pair, false, h) || (int)part * kPartRows >= h.n) return;
    unsigned order[kPartSteps][4], above, in;
    load_orders<kPartSteps>(h, (int)part * kPartRows, order);
    const PartSpace space = part_space(p, pair);
    first_digit(p, space, (int)part, (h.n + kPartRows - 1) / kPartRows, lds, above, in);
    const unsigned bin = lds.found[0];  // (found[3] is 0: the part's candidates so far)
    unsigned *const out = space.candidates + in;
#pragma unroll
    for (int s = 0; s < kPartSteps; ++s)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (order[s][e] >> (32 - kDigitBits) == bin) out[atomicAdd(&lds.found[3], 1u)] = order[s][e];
}
__global__ __launch_bounds__(kSThreads) void swaa_evict_put_kernel(const EvictParams p) {
    __shared__ SelectLds lds;
    const unsigned pairs = (unsigned)(p.B * p.Hkv), pair = blockIdx.x % pairs, part = blockIdx.x / pairs;
    Head h;
    if (!head_of(p, pair, false, h) || (int)part * kPartRows >= h.n) return;
    unsigned order[kPartSteps][4], above, in;
    load_orders<kPartSteps>(h, (int)part * kPartRows, order);
    const PartSpace space = part_space(p, pair);
    first_digit(p, space, (int)part, (h.n + kPartRows - 1) / kPartRows, lds, above, in);
    const unsigned bin = lds.found[0], n = lds.found[2];
    unsigned prefix = bin << (32 - kDigitBits), left = lds.found[1];
    __syncthreads();  // (found is read)
    auto look = [&](auto f) {
        for (unsigned i = threadIdx.x; i < n; i += kSThreads) f(space.candidates[i]);
    };
    find_least(look, prefix, ((1u << kDigitBits) - 1) << (32 - kDigitBits), left, 32 - 2 * kDigitBits, lds);
    // candidates of the parts before this one: the heavier, the equal
    unsigned heavier = 0, equal = 0;
    for (unsigned i = threadIdx.x; i < in; i += kSThreads) {
        heavier += space.candidates[i] > prefix;
        equal += space.candidates[i] == prefix;
    }
    unsigned base_heavier, base_equal;
    __syncthreads();
    block_exclusive(heavier, lds.scratch, base_heavier);
    block_exclusive(equal, lds.scratch2, base_equal);
    base_heavier += above;
    __syncthreads();
    put_rows<kPartSteps>(h, (int)part * kPartRows, order, prefix, left, base_heavier, base_equal, lds);
}

constexpr int kMThreads = 1024;
constexpr int kMRows = 4;  // of a thread, on the way at a time; those of the next block are asked for before they are written

// Moves rows kept[i] to i for i in [begin, end), in that order as far as anyone can see: a block's rows are read, in all threads,
// before any of them is written, and the next block's come from behind those that this one writes.  Ends at the first row that comes
// from `split` or behind it (`kept` ascends).  kPerRow threads share a row; place(i) says where row i stands (elements of Data, negative: nowhere, and whether it may be written there).
template <int kPerRow, typename Data, typename Place>
__device__ __forceinline__ void move_rows(const int *kept, int begin, int end, int split, bool takes_part, Data *base, Place place) {
    constexpr int kStride = kMThreads / kPerRow, kBlock = kMRows * kStride;
    int from[kMRows];                    // of a block: the rows that come, -1 where none does,
    long long src[kMRows], dst[kMRows];  // and both ends (-1: none)
    Data data[kMRows] = {};
    auto row_of = [&](int first, int r) { return first + r * kStride + (int)threadIdx.x / kPerRow; };
    auto load_from = [&](int first) {
#pragma unroll
        for (int r = 0; r < kMRows; ++r) {
            const int i = row_of(first, r);
            from[r] = i < end && takes_part ? kept[i] : -1;
            if (from[r] >= split) from[r] = -1;
        }
    };
    auto find = [&](int first) {
#pragma unroll
        for (int r = 0; r < kMRows; ++r) {
            const int i = row_of(first, r);
            src[r] = dst[r] = -1;
            if (from[r] > i) {
                bool inside, unused;
                const long long to = place(i, inside);
                src[r] = place(from[r], unused);
                if (inside) dst[r] = to;
            }
        }
    };
    auto load_data = [&]() {
#pragma unroll
        for (int r = 0; r < kMRows; ++r)
            if (src[r] >= 0) data[r] = base[src[r]];
    };
    load_from(begin);
    find(begin);
    load_data();
    load_from(begin + kBlock);
    int comes = begin < end ? kept[begin] : 0;  // the first row of the block
    for (int first = begin; first < end && comes < split; first += kBlock) {
        comes = kept[min(first + kBlock, end - 1)];
        Data now[kMRows];
        long long to[kMRows];
#pragma unroll
        for (int r = 0; r < kMRows; ++r) {
            now[r] = data[r];
            to[r] = dst[r];
            asm volatile("" : "+v"(now[r]));  // (waits for it)
        }
        __syncthreads();
        find(first + kBlock);
        load_data();
#pragma unroll
        for (int r = 0; r < kMRows; ++r)
            if (to[r] >= 0) base[to[r]] = now[r];
        load_from(first + 2 * kBlock);
    }
}

// kLanes: lanes of 16 bytes that make a slice of a row of K or V.  One workgroup of a pair moves its weights.
// Rows that come from `split` or behind it are left to the kernel below.
template <int kLanes>
__global__ __launch_bounds__(kMThreads) void swaa_evict_move_kernel(const EvictParams p, int slices, int split) {
    const int tid = threadIdx.x;
    // pairs in turn: the slices of a row share a die's L2 (where the pairs are a multiple of the dies)
    const unsigned pairs = (unsigned)(p.B * p.Hkv), pair = blockIdx.x % pairs, part = blockIdx.x / pairs;
    const unsigned b = fastdiv(pair, p.div_hkv), kvh = pair - b * (unsigned)p.Hkv;
    const int *kept = p.kept + (long long)pair * p.n_keep;
    const int begin = p.n_sink, end = min(p.n_keep, p.Nk);
    if (part == 0) {
        float *weights = p.weights + b * p.w_sb + kvh * p.w_sh;
        move_rows<1>(kept, begin, end, p.Nk, true, weights, [](int i, bool &inside) {
            inside = true;
            return (long long)i;
        });
        __syncthreads();  // (its reads are done)
        const int n = p.seq_lens ? max(min(p.seq_lens[b], p.Nk), 0) : p.Nk;
        for (int i = p.n_keep + tid; i < n; i += kMThreads) weights[i] = 0.f;
        if (p.new_lens && kvh == 0 && tid == 0) p.new_lens[b] = min(n, p.n_keep);
        return;
    }
    const Rows &t = part > (unsigned)slices ? p.v : p.k;
    const int chunk = (int)((part - 1) % (unsigned)slices) * kLanes + tid % kLanes;
    move_rows<kLanes>(kept, begin, end, split, 8 * chunk < p.D, reinterpret_cast<u32x4 *>(t.ptr + 2 * (kvh * t.sh + 8 * chunk)), [&](int i, bool &inside) {
        return cache_row(p.pages, t, (int)b, 0, i, false, inside) / 8;  // (strides are multiples of 8 elements)
    });
}

// Rows from behind the first n_keep: nothing is written where they stand, so they move in any order.  Rows of K, then of V.
constexpr int kFThreads = 256, kFRows = 4;  // (rows of a thread)
template <int kPerRow>
__global__ __launch_bounds__(kFThreads) void swaa_evict_far_kernel(const EvictParams p, int blocks) {
    constexpr int kStride = kFThreads / kPerRow;
    const unsigned pairs = (unsigned)(p.B * p.Hkv), pair = blockIdx.x % pairs, part = blockIdx.x / pairs;
    const unsigned b = fastdiv(pair, p.div_hkv), kvh = pair - b * (unsigned)p.Hkv;
    const bool of_v = part >= (unsigned)blocks;
    const int first = (int)(of_v ? part - (unsigned)blocks : part) * kStride * kFRows + (int)threadIdx.x / kPerRow, chunk = (int)threadIdx.x % kPerRow;
    const Rows &t = of_v ? p.v : p.k;
    const int *kept = p.kept + (long long)pair * p.n_keep;
    char *const base = t.ptr + 2 * (kvh * t.sh + 8 * chunk);
    int from[kFRows];
    long long src[kFRows], dst[kFRows];
    u32x4 data[kFRows];
#pragma unroll
    for (int r = 0; r < kFRows; ++r) {
        const int i = first + r * kStride;
        from[r] = i < p.n_keep && 8 * chunk < p.D ? kept[i] : -1;
    }
#pragma unroll
    for (int r = 0; r < kFRows; ++r) {
        dst[r] = -1;
        if (from[r] >= p.n_keep) {
            bool inside, unused;
            const long long to = cache_row(p.pages, t, (int)b, 0, first + r * kStride, false, inside);
            src[r] = cache_row(p.pages, t, (int)b, 0, from[r], false, unused);
            if (inside) dst[r] = to;
        }
    }
#pragma unroll
    for (int r = 0; r < kFRows; ++r)
        if (dst[r] >= 0) data[r] = *reinterpret_cast<const u32x4 *>(base + 2 * src[r]);
#pragma unroll
    for (int r = 0; r < kFRows; ++r)
        if (dst[r] >= 0) *reinterpret_cast<u32x4 *>(base + 2 * dst[r]) = data[r];
}

// New lengths in place of the old ones: when no kernel reads those any more.
__global__ void swaa_evict_lengths_kernel(const EvictParams p) {
    const int b = (int)(blockIdx.x * blockDim.x + threadIdx.x);
    if (b < p.B) p.new_lens[b] = min(max(min(p.seq_lens[b], p.Nk), 0), p.n_keep);
}

template <int kSteps>
void select(const EvictParams &p, hipStream_t stream) {
    swaa_evict_select_kernel<kSteps><<<dim3((unsigned)(p.B * p.Hkv)), dim3(kSThreads), 0, stream>>>(p);
}
template <int kLanes>
void move(const EvictParams &p, int split, hipStream_t stream) {
    const int slices = (p.D / 8 + kLanes - 1) / kLanes;
    swaa_evict_move_kernel<kLanes><<<dim3((unsigned)(p.B * p.Hkv) * (1 + 2 * (unsigned)slices)), dim3(kMThreads), 0, stream>>>(p, slices, split);
}
template <int kPerRow>
void move_far(const EvictParams &p, hipStream_t stream) {
    constexpr int kRows = kFThreads / kPerRow * kFRows;
    const int blocks = (p.n_keep + kRows - 1) / kRows;
    swaa_evict_far_kernel<kPerRow><<<dim3((unsigned)(p.B * p.Hkv) * 2 * (unsigned)blocks), dim3(kFThreads), 0, stream>>>(p, blocks);
}

}  // namespace

// Shared out: pairs longer than one workgroup holds in a round, so few of them that a workgroup each would leave most of the chip idle
// (call with the moves, a workgroup each against shared out: 8 pairs of 65536 rows to 16384 76.2 -> 52.0 us, 64 of 40000 to 2000
// 74.0 -> 55.6, 96 of those 97.6 -> 79.8, 128 of 65536 to 16384 537 and 542; 8 of 20000 to 5000 29.8 -> 32.4).
long long plan_evict(EvictParams &p) {
    const long long pairs = (long long)p.B * p.Hkv;
    p.parts = p.Nk > kMaxSteps * kStep && pairs <= 96 ? (p.Nk + kPartRows - 1) / kPartRows : 0;
    return p.parts ? pairs * ((long long)p.parts * kBins + p.Nk + p.Nk % 2) * (long long)sizeof(unsigned) : 0;
}

hipError_t launch_evict(const EvictParams &params, hipStream_t stream) {
    EvictParams p = params;
    const bool in_place = p.new_lens && p.new_lens == p.seq_lens;
    if (in_place) p.new_lens = nullptr;
    if (p.select_space) {
        const dim3 wgs((unsigned)(p.B * p.Hkv) * (unsigned)p.parts);
        swaa_evict_count_kernel<<<wgs, dim3(kSThreads), 0, stream>>>(p);
        swaa_evict_gather_kernel<<<wgs, dim3(kSThreads), 0, stream>>>(p);
        swaa_evict_put_kernel<<<wgs, dim3(kSThreads), 0, stream>>>(p);
    } else if (p.Nk <= kStep) {
        select<1>(p, stream);
    } else if (p.Nk <= 4 * kStep) {
        select<4>(p, stream);
    } else {
        select<8>(p, stream);
    }
    hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    // Half the rows leave or more: most that stay come from behind the first n_keep, and with many of those a launch of their own pays
    // (8 pairs: 32768 rows to 8000 43.4 -> 37.3 us, 16384 to 4096 25.2 -> 24.7, 8192 to 2048 18.8 -> 20.2; 64: 20000 to 5000 102.6 -> 92.3,
    // 4096 to 2000 31.0 -> 35.6).
    const bool far = p.Nk / 2 >= p.n_keep && p.n_keep >= 4096;
    const long long halves = (long long)p.B * p.Hkv * 2;
    const int split = far ? p.n_keep : p.Nk;
    // Slices of 64 bytes where they make 256 workgroups, one for each CU, else of 32 (32 against 64 bytes, 64 pairs: 4096 rows to 3900
    // 59.6 -> 47.9 us, 128: 203 -> 131; 8: 17000 to 12000 52.5 and 59.7).
    if (halves * (p.D / 32) >= 256)
        move<4>(p, split, stream);
    else
        move<2>(p, split, stream);
    err = hipGetLastError();
    if (far && err == hipSuccess) {
        if (p.D <= 64)
            move_far<8>(p, stream);
        else if (p.D <= 128)
            move_far<16>(p, stream);
        else
            move_far<32>(p, stream);
    }
    err = hipGetLastError();
    if (err != hipSuccess || !in_place) return err;
    p.new_lens = params.new_lens;
    swaa_evict_lengths_kernel<<<dim3((unsigned)(p.B + 255) / 256), dim3(256), 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace swaa
