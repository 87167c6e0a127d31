// Launchers of the operators of a speculative decoding step (ooco_tree.hip, ooco_spec.hip).  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace ooco {

constexpr int kMaxMaskWords = 4;   // 64-bit words of a node's mask

// ---- attention of the nodes (ooco_tree.hip)
struct TreeArgs {
    const uint16_t *q;
    const uint16_t *k_cache;
    const uint16_t *v_cache;
    const int32_t *block_tables;
    const int32_t *query_start_loc;
    const int32_t *ctx_lens;
    const uint64_t *masks;      // [total_q][words]
    uint16_t *out;
    int32_t *merges;            // [runs][5]: parts of the unit that the run continues (0: none), its first run, first row, rows, kv head
    float *part_acc;            // [2 * runs][columns of a tile][hd]  un-normalised partial outputs
    float *part_ml;             // [2 * runs][columns of a tile][2]   (reference in log2 units, sum)
    int64_t num_blocks;
    int32_t Hq, Hkv, g, hd;
    int32_t max_blocks_per_seq;
    int32_t num_seqs, total_q, words;
    int32_t runs_log2;          // runs of the line: 1 << runs_log2 workgroups
    int64_t halve_below;        // half the runs on a line of fewer steps
    int32_t tile_rows;          // rows of the widest tile
    int32_t short_line;         // up to 64 sequences, and a line of 31 bits
    float scale_log2e;          // softmax scale * log2(e)
};
// Blocks of 32 columns of the widest tile: 2 (four waves that share the tokens), 4 or 8 (a wave each).
int tree_waves(int total_q, int num_seqs, int Hkv, int g, int max_blocks_per_seq, int num_cus);
// Runs (a power of two) that a workspace of ws_bytes allows on num_cus compute units, as their logarithm; < 0: none.
int tree_runs_log2(int waves, int hd, int num_cus, size_t ws_bytes);
// a.runs_log2 runs; the workspace pointers and what follows from the waves are set here.
hipError_t launch_attn_tree(TreeArgs &a, int waves, void *ws, hipStream_t s);

// ---- masks and positions
hipError_t launch_tree_masks(const int32_t *parents, const int32_t *query_start_loc, const int32_t *ctx_lens, uint64_t *masks,
                             int32_t *positions, int words, int num_seqs, int total_q, hipStream_t s);

// ---- rotary positions and append
constexpr int kMaxRotaryPairs = 64;
struct RopeArgs {
    const uint16_t *q, *k_new, *v_new;   // rows q_stride, k_stride, v_stride elements apart
    uint16_t *q_out, *k_cache, *v_cache;
    const int32_t *positions;            // NULL: the place in the cache
    const int32_t *block_tables;
    const int32_t *query_start_loc;
    const int32_t *ctx_lens;
    int64_t q_stride, k_stride, v_stride;
    int64_t num_blocks;
    int32_t Hq, Hkv, hd;
    int32_t max_blocks_per_seq;
    int32_t num_seqs, total_q;
    int32_t pairs;                       // rotated pairs per head
    int32_t parts;                       // workgroups per (sequence, KV block)
    int32_t past_caches;                 // 16-byte stores past the caches
    float factor;                        // of cosine and sine
    double turns[kMaxRotaryPairs];       // turns per position of each pair
};
hipError_t launch_rope_append(RopeArgs &a, bool interleaved, int num_cus, hipStream_t s);

// ---- verification
struct VerifyArgs {
    const void *target, *draft;          // probabilities, rows `stride` elements apart; draft may be NULL
    const int32_t *tokens;
    const int32_t *parents;              // NULL: chains
    const float *uniforms;               // [total_q]
    const float *final_uniforms;         // [num_seqs]
    const int32_t *query_start_loc;
    int32_t *counts, *path, *out_tokens;
    double *sums;                        // [num_seqs][pieces of a row][2]: what is left, and what there was
    int32_t *arrivals;                   // of each sequence, arrivals_apart ints apart, zero between calls
    int32_t arrivals_apart;
    int64_t stride;
    int32_t vocab, max_path;
    int32_t num_seqs, total_q;
    int32_t pieces, groups;              // pieces of a row that a wave sums, and workgroups that share a row
};
constexpr int kMaxVerifyNodes = 256;
size_t verify_workspace(const VerifyArgs &a);
void verify_layout(VerifyArgs &a, bool bf16, int num_cus);
hipError_t launch_verify(const VerifyArgs &a, bool bf16, hipStream_t s);

// ---- accepted nodes to their places
constexpr int kCompactLayers = 112;      // layers per launch (their pointers travel in the kernel arguments)
struct CompactArgs {
    uint16_t *k[kCompactLayers], *v[kCompactLayers];
    const int32_t *block_tables;
    const int32_t *ctx_lens;
    const int32_t *path;
    const int32_t *counts;
    int64_t num_blocks;
    int32_t Hkv, hd, max_blocks_per_seq, max_path;
    int32_t layers, layers_each;         // and those that a workgroup has
};
hipError_t launch_kv_compact(CompactArgs &a, int num_seqs, int num_cus, hipStream_t s);

}  // namespace ooco
