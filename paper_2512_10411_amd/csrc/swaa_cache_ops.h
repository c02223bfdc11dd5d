// Parameter blocks and launchers of the operators around a key/value cache: norms with rotation (swaa_norm_rope.hip),
// attention weights of the keys (swaa_key_weights.hip), eviction (swaa_evict.hip).
#ifndef SWAA_CACHE_OPS_H_
#define SWAA_CACHE_OPS_H_

#include "swaa_common.h"

namespace swaa {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// A tensor of 16-bit elements: element strides of batch entry, head and row (a paged cache: of page, head and row of a page).
struct Rows {
    char *ptr;
    long long sb, sh, sn;
};

// The sequences of a call: fixed-length (cu_q null; seq_lens or Nk keys each) or packed.
struct Sequences {
    const int *cu_q, *cu_k;   // B + 1 offsets each, or both null
    const int *seq_lens;      // B lengths, or null
    int B, Nq, Nk;
};
// Query rows and keys of sequence b: its rows are the newest nq of its nk tokens.  Lengths are clamped to [0, Nk]; a fixed-length batch's
// sequence shorter than its rows (padding) has no rows.
__device__ __forceinline__ void sequence(const Sequences &s, int b, int &nq, int &nk) {
    nq = s.Nq;
    nk = s.Nk;
    if (s.cu_q) {
        nk = s.cu_k[b + 1] - s.cu_k[b];
        nq = max(min(min(s.cu_q[b + 1] - s.cu_q[b], s.Nq), nk), 0);
        nk = max(min(nk, s.Nk), 0);
        nq = min(nq, nk);
    } else if (s.seq_lens) {
        nk = max(min(s.seq_lens[b], s.Nk), 0);
        nq = nk < s.Nq ? 0 : s.Nq;
    }
}

// A paged cache's table, or none (block_table null).
struct Pages {
    const int *block_table;
    int bt_stride, page_size, num_pages;
    FastDiv div_page;
};
// Offset in elements of row `row` of sequence b's cache, head 0; row0: of a packed cache, the sequence's first row.  With pages:
// page numbers outside the cache are clamped into it, and `inside` says whether this one was.
__device__ __forceinline__ long long cache_row(const Pages &pg, const Rows &t, int b, long long row0, int row, bool packed, bool &inside) {
    inside = true;
    if (!pg.block_table) return (packed ? 0 : b * t.sb) + (row0 + row) * t.sn;
    const int of = (int)fastdiv((unsigned)row, pg.div_page);
    const int page = pg.block_table[(long long)b * pg.bt_stride + of];
    inside = (unsigned)page < (unsigned)pg.num_pages;
    return (long long)min(max(page, 0), pg.num_pages - 1) * t.sb + (long long)(row - of * pg.page_size) * t.sn;
}

struct NormRopeParams {
    Rows q, k, v, q_out, k_out, v_out;  // v.ptr null: no values.  Backward: q, k the forward's inputs, v null, and q_out, k_out the gradients of those
    Rows dq_out, dk_out;                // backward only: gradients of the forward's outputs
    Sequences seq;
    Pages pages;
    const int *positions;  // [B, Nq], or [rows] of a packed batch; null: the row in the cache
    const float *q_weight, *k_weight;  // [D] each, or both null: no norm
    const float *inv_freq;             // [R / 2]
    float eps;
    int fp16, interleaved;
    int Hq, Hkv, D, R;
    long long tokens;  // token slots: B Nq, or the rows of the packed tensor where the caller states them (by_row)
    int by_row;
    FastDiv div_nq;
    // Work: tiles of tile_tokens tokens, 1 << wave_shift of them in a wave (its own, or with by_wave 0 the same in all four), times
    // a part of the units (as many heads as are worked on at a time): first those of q, then k, then v.
    int wave_shift, by_wave, tile_tokens;
    int q_units, k_units, v_units, units_per_wg, wgs_per_tile;
    FastDiv div_wgs;  // wgs_per_tile
    long long wgs;
    float *dq_weight, *dk_weight, *partial;  // backward: results, and [wgs][2][D] sums of the workgroups
    long long tiles_per_wg;
};
hipError_t launch_norm_rope(const NormRopeParams &p, hipStream_t stream);
hipError_t launch_norm_rope_bwd(const NormRopeParams &p, hipStream_t stream);
// Fill the work fields; false: more workgroups than a launch holds.
bool plan_norm_rope(NormRopeParams &p);
bool plan_norm_rope_bwd(NormRopeParams &p);

struct KeyWeightsParams {
    Rows q, k;
    const float *lse;
    long long lse_sb, lse_sh;
    float *weights;
    long long w_sb, w_sh;
    Sequences seq;
    Pages pages;
    const int *n_prompts;
    int fp16;
    int Hq, Hkv, G, D;
    int W, S, P;
    float scale_log2, decay;
    // Work (plan_key_weights): (sequence, KV head) pairs x (tiles of keys x chunks of the columns, heads of the group x rows that see
    // the tile).  A row sees few keys of a windowed layer, but the sinks are seen by all: their tiles have chunk counts of their own.
    int key_tile, one_stage, listed;  // keys of a workgroup; at most one stage of columns; tiles by a list of the sequences' own
    int pairs, tiles, sink_tiles, sink_items;
    int chunks, sink_chunks, chunk_stages;  // (stages of 64 columns)
    long long items;
    FastDiv div_pairs, div_hkv, div_sink_chunks, div_others;
    float *partial;  // [items][key_tile], or null: one chunk per tile
};
bool plan_key_weights(KeyWeightsParams &p);
long long key_weights_workspace_bytes(const KeyWeightsParams &p);
hipError_t launch_key_weights(const KeyWeightsParams &p, hipStream_t stream);

struct EvictParams {
    Rows k, v;
    float *weights;
    long long w_sb, w_sh;
    int *kept;      // [B, Hkv, n_keep]
    int *new_lens;  // [B] or null
    const int *seq_lens;
    Pages pages;
    int B, Hkv, D, Nk, n_keep, n_sink, n_recent;
    FastDiv div_hkv;
    int parts;               // of a pair's rows (plan_evict), 0: one workgroup selects
    unsigned *select_space;  // their counts and candidates, or null: one workgroup selects
};
long long plan_evict(EvictParams &p);  // bytes of workspace that the selection has use for
hipError_t launch_evict(const EvictParams &p, hipStream_t stream);

}  // namespace swaa

#endif  // SWAA_CACHE_OPS_H_
