// HIP kernels of libooco for gfx950: attention of a tree of drafted nodes over the paged KV cache.
//
// Row t of a sequence with n nodes on ctx cached tokens sees tokens 0 .. ctx-1 and those nodes j whose bit of its mask is set.
// As in the other attention kernels scores are computed transposed, S^T[token][query column] = K Q^T, and the output as
// O^T[dim][query column] = V^T P^T; a query column is a (row, head of the GQA group) pair, so that the K and V of a token are
// fetched once for all nodes and heads that see it.  One pass over the keys with the running maximum and sum of the softmax.
//
// Work: the columns of a sequence are cut into tiles, as few as hold them: of 32, 64 or 128 columns, a wave of the workgroup having
// 32; the waves that columns leave over share the tokens of a step.  Unit = (tile, kv head), walked in steps of 128 tokens.  The
// units of all sequences, steps end to end, form a line that is cut into equal runs, a workgroup each; where a run ends inside a
// unit, partial results meet in the merge kernel.  The lengths are read and the line is laid out on the device by every workgroup for
// itself: no plan and no host copy of lengths that the last step's verification has just decided.
//   32 columns      the four waves have 32 tokens of a step each, and load K and V from the cache to the registers of the matrix
//                   instructions: nothing is shared, so nobody waits for anybody
//   64, 128         K and V of 64 tokens at a time go through LDS, for two or four waves, by direct loads into the other of two buffers
#include "ooco_device.h"
#include "ooco_internal.h"
#include "ooco_spec.h"

#include <algorithm>

namespace ooco {

constexpr int kTreeCols = 128;        // query columns of the widest tile
constexpr int kTreeThreads = 256;
constexpr int kTreeStep = 128;        // tokens of a step
constexpr int kMergeInts = 8;
constexpr int kMinRun = 1;            // steps of a run, at least

// The largest of a lane's sixteen scores, NaN if one is.  (v_maximum3_f32, which needs no operand quieted.  Not the asm of max16:
// the waits between a matrix instruction and what reads its result are the compiler's, which does not see into asm.)
OOCO_DEV float largest(const f32x16 &s)
{
    float m = __builtin_elementwise_maximum(s[0], s[1]);
#pragma unroll
    for (int r = 2; r < 16; r += 2) m = __builtin_elementwise_maximum(__builtin_elementwise_maximum(m, s[r]), s[r + 1]);
    return m;
}

// What a sequence has on the line.
struct TreeSeq {
    int q0, n, ctx, len, steps;          // len: tokens that exist, the nodes among them
    int waves;                           // of 32 columns that a tile has: 1, 2 or 4
    int tile_rows, tiles;
    int64_t units;                       // steps of all its units
};
OOCO_DEV TreeSeq tree_seq(const TreeArgs &p, int q0, int q1, int ctx)
{
    TreeSeq s;
    s.q0 = q0;
    s.n = q1 - q0;
    if (q0 < 0 || s.n < 0 || s.n > p.total_q - q0) s.n = 0;
    const int cap = (int)min((int64_t)p.max_blocks_per_seq * kBlockSize, (int64_t)INT32_MAX - 1024);
    s.ctx = min(max(ctx, 0), cap);
    s.len = min(s.ctx + min(s.n, 64 * p.words), cap);
    // (rows of a group of heads that does not divide 32: a tile of 32 columns has fewer than 32 of them)
    s.waves = s.n <= 32 / p.g ? 1 : s.n <= 64 / p.g ? 2 : 4;
    s.tile_rows = 32 * s.waves / p.g;
    s.tiles = (s.n + s.tile_rows - 1) / s.tile_rows;
    s.steps = (s.len + kTreeStep - 1) / kTreeStep;
    s.units = (int64_t)s.tiles * p.Hkv * s.steps;
    return s;
}

// The line: its length, and the sequence that holds position `at(total)` of it, with the position of that sequence's first step.
// All threads of the workgroup call it together.
template <class At>
OOCO_DEV int64_t tree_locate(const TreeArgs &p, At at, int &seq, int64_t &start)
{
    __shared__ int64_t wave_total[kTreeThreads / 64];
    __shared__ int sh_seq;
    __shared__ int64_t sh_start;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    auto units_of = [&](int i) -> int64_t {
        return i < p.num_seqs ? tree_seq(p, p.query_start_loc[i], p.query_start_loc[i + 1], p.ctx_lens[i]).units : 0;
    };
    auto scan = [&](int64_t v, int64_t &all) -> int64_t {   // inclusive sum over the workgroup, and of all
        int64_t x = v;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int64_t o = __shfl_up(x, d);
            x += lane >= d ? o : 0;
        }
        __syncthreads();
        if (lane == 63) wave_total[wave] = x;
        __syncthreads();
        all = 0;
        int64_t before = 0;
#pragma unroll
        for (int w = 0; w < kTreeThreads / 64; ++w) {
            before += w < wave ? wave_total[w] : 0;
            all += wave_total[w];
        }
        return before + x;
    };
    int64_t total = 0, all, mine = 0, incl = 0;
    for (int base = 0; base < p.num_seqs; base += kTreeThreads) {
        mine = units_of(base + tid);
        incl = scan(mine, all);
        total += all;
    }
    const int64_t x = at(total);
    int64_t before = 0;
    for (int base = 0; base < p.num_seqs; base += kTreeThreads) {
        if (p.num_seqs > kTreeThreads) {
            mine = units_of(base + tid);
            incl = scan(mine, all);
        } else {
            all = total;
        }
        if (before + incl - mine <= x && x < before + incl) {
            sh_seq = base + tid;
            sh_start = before + incl - mine;
        }
        before += all;
        if (before > x) break;
    }
    __syncthreads();
    seq = sh_seq;
    start = sh_start;
    return total;
}

// Values that are the same in every lane, in scalar registers.
OOCO_DEV int64_t uniform(int64_t v)
{
    const uint32_t lo = __builtin_amdgcn_readfirstlane((int)(uint32_t)v), hi = __builtin_amdgcn_readfirstlane((int)(v >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}
// Lengths and block ids by scalar loads, which the waits on the vector-memory counter do not see.
typedef const __attribute__((address_space(4))) int32_t *const_i32_ptr;
OOCO_DEV const_i32_ptr scalar_ptr(const int32_t *p) { return (const_i32_ptr)(uintptr_t)p; }
OOCO_DEV TreeSeq tree_seq_at(const TreeArgs &p, int seq)
{
    const const_i32_ptr qsl = scalar_ptr(p.query_start_loc), ctx = scalar_ptr(p.ctx_lens);
    return tree_seq(p, qsl[seq], qsl[seq + 1], ctx[seq]);
}

// Runs of the line: run w = [first(w), first(w + 1)).  No run is empty but those behind `count`.
struct TreeRuns {
    int64_t total;
    int log2;
    bool split;      // the line is cut into all runs there are, else into runs of kMinRun steps
    OOCO_DEV TreeRuns(int64_t total_, int log2_) : total(total_), log2(log2_), split(total_ >= ((int64_t)kMinRun << log2_)) {}
    OOCO_DEV int64_t first(int w) const { return split ? (total * w) >> log2 : min(total, (int64_t)w * kMinRun); }
    OOCO_DEV int holding(int64_t x) const { return split ? (int)((((x + 1) << log2) - 1) / total) : (int)(x / kMinRun); }
};

// What a wave does with 32 tokens, whichever way they come: its 32 query columns' share of the softmax and of the output.
template <int HD>
struct TreeWave {
    static constexpr int KS = HD / 16;   // k-steps of QK
    static constexpr int MB = HD / 32;   // 32-dim groups of the output
    u32x4 qb[KS];
    f32x16 O[MB];
    float m, lsum;                       // reference of the column's weights in log2 units, this lane's share of their sum
    const uint64_t *mask;

    OOCO_DEV void begin(const TreeArgs &p, int64_t q_row, int head, int h)
    {
        const u32x4 *const qp = reinterpret_cast<const u32x4 *>(p.q + (q_row * p.Hq + head) * HD);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qb[ks] = qp[2 * ks + h];
        mask = p.masks + q_row * p.words;
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int r = 0; r < 16; ++r) O[mb][r] = 0.f;
        m = -1e30f;   // (finite: tokens that a column does not see weigh nothing, where -inf - -inf would make them NaN)
        lsum = 0.f;
    }
    // Bit i: the column sees token tok0 + i.  tok0 + 32 > ctx.
    OOCO_DEV uint32_t sees(int words, int tok0, int ctx, int len) const
    {
        const int j0 = tok0 - ctx;   // node that token tok0 is (negative: cached)
        uint32_t bits;
        if (j0 >= 0) {
            const int k = j0 >> 6, sh = j0 & 63;
            uint64_t b = k < words ? mask[k] >> sh : 0;
            if (sh > 32 && k + 1 < words) b |= mask[k + 1] << (64 - sh);
            bits = (uint32_t)b;
        } else {
            bits = ((uint32_t)mask[0] << -j0) | ((1u << -j0) - 1u);   // (-31 <= j0)
        }
        const int left = len - tok0;   // tokens that exist
        if (left < 32) bits &= left > 0 ? (1u << left) - 1u : 0u;
        return bits;
    }
    // Register r of S is token 16 (r / 8) + 8 h + r % 8 of the 32.
    OOCO_DEV static void hide(f32x16 &S, uint32_t bits, int h)
    {
        bits >>= 8 * h;
#pragma unroll
        for (int r = 0; r < 16; ++r) S[r] = (bits >> (16 * (r / 8) + r % 8)) & 1u ? S[r] : -INFINITY;
    }
    // Scores to weights.  The reference moves only where a score exceeds it by 2^8: weights up to 2^8 are as exact in bf16 and fp32
    // as below 1, and the division at the end takes the reference out.
    OOCO_DEV void weights(const f32x16 &S, float scale, u32x4 (&P)[2])
    {
        float x, y;
        swap32(largest(S), x, y);
        const float top = __builtin_elementwise_maximum(x, y) * scale;
        if (__any(top > m + 8.0f)) {
            const float m_new = fmaxf(m, top), alpha = fast_exp2(m - m_new);
            m = m_new;
            lsum *= alpha;
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int r = 0; r < 16; ++r) O[mb][r] *= alpha;
        }
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            float e[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                e[r] = fast_exp2(__builtin_fmaf(S[8 * b + r], scale, -m));
                lsum += e[r];
            }
            P[b] = u32x4{pack2_bf16(e[0], e[1]), pack2_bf16(e[2], e[3]), pack2_bf16(e[4], e[5]), pack2_bf16(e[6], e[7])};
        }
    }
};

// A tile of K or of V (one block, one kv head) from the cache into LDS, HD / 32 loads of 16 bytes per lane: 1 KiB each, contiguous in LDS from
// dst on.  off[n]: the lane's place in the tile for load n, less n KiB (the instruction's offset counts for both addresses).
template <int HD>
OOCO_DEV void tile_to_lds(const char *base, uint32_t dst, const uint32_t (&off)[4])
{
    uint32_t saved_m0;   // M0 is restored: the compiler may keep a value of its own there
    if constexpr (HD == 128)
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
                     "global_load_lds_dwordx4 %2, %6\n\tglobal_load_lds_dwordx4 %3, %6 offset:1024\n\t"
                     "global_load_lds_dwordx4 %4, %6 offset:2048\n\tglobal_load_lds_dwordx4 %5, %6 offset:3072\n\ts_mov_b32 m0, %0"
                     : "=&s"(saved_m0)
                     : "s"(dst), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(base)
                     : "memory");
    else
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
                     "global_load_lds_dwordx4 %2, %4\n\tglobal_load_lds_dwordx4 %3, %4 offset:1024\n\ts_mov_b32 m0, %0"
                     : "=&s"(saved_m0)
                     : "s"(dst), "v"(off[0]), "v"(off[1]), "s"(base)
                     : "memory");
}

constexpr int kStageBlocks = 4;   // KV blocks that go through LDS at a time

template <int HD>
__global__ __launch_bounds__(kTreeThreads, 2) void tree_kernel(const TreeArgs p)
{
    using Wave = TreeWave<HD>;
    constexpr int KS = Wave::KS, MB = Wave::MB;
    constexpr int ROW = HD + 4;                   // floats of a column in LDS (padded: the lanes of a wave are columns)
    constexpr int CH = 2 * HD;                    // 16-byte pieces of a tile of K or V
    constexpr int64_t kTile = (int64_t)HD * kBlockSize;
    constexpr int kSlab = 4 * 32 * ROW * 4, kStage = 2 * 2 * kStageBlocks * CH * 16;
    __shared__ __align__(16) unsigned char lds[kSlab > kStage ? kSlab : kStage];
    __shared__ float stat[4][32][2];
    float (*const slab)[32][ROW] = reinterpret_cast<float (*)[32][ROW]>(lds);           // [wave][column][dim]
    u32x4 *const ldsK = reinterpret_cast<u32x4 *>(lds), *const ldsV = ldsK + 2 * kStageBlocks * CH;   // [buffer][block][piece]

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, h = lane >> 5;
    const int g = p.g;
    const int w = blockIdx.x;

    int seq = 0;
    int64_t start = 0;
    const int64_t total = uniform(tree_locate(p, [&](int64_t t) { return TreeRuns(t, p.runs_log2).first(w); }, seq, start));
    start = uniform(start);
    const TreeRuns runs(total, p.runs_log2);
    const int64_t lo = runs.first(w), hi = runs.first(w + 1);
    int32_t *const merge = p.merges + (int64_t)w * kMergeInts;
    if (lo >= hi) {
        if (tid == 0) merge[1] = 0;
        return;
    }
    // K operand row col -> block (col >> 4) of the 32 tokens, slot with bits 2 and 3 swapped, so that register r of S^T is token
    // 16 (r / 8) + 8 h + r % 8: eight consecutive tokens of a block, as a 16-byte piece of V has them
    const int ku = col >> 4, kslot = (col & 3) | ((col & 4) << 1) | ((col & 8) >> 1);
    // Pieces of a tile in LDS: K as in the cache, V [half of the tokens][dim], so that the lanes that read together read side by side
    constexpr int kBias = 4096;   // (keeps the offsets of V positive)
    uint32_t k_off[4], v_off[4];
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        const int c = 64 * n + lane;
        k_off[n] = (uint32_t)lane * 16u;
        v_off[n] = (uint32_t)((2 * (c % HD) + c / HD) * 16 - n * 1024 + kBias);
    }
    const uint32_t ldsK_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)ldsK;
    const uint32_t ldsV_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)ldsV;

    int64_t pos = lo;
    seq = __builtin_amdgcn_readfirstlane(seq);
    TreeSeq s = tree_seq_at(p, seq);
    while (pos < hi) {
        while (pos - start >= s.units) {   // the next sequence with rows
            start += s.units;
            ++seq;
            s = tree_seq_at(p, seq);
        }
        const int unit = (int)((pos - start) / s.steps);
        const int s0 = (int)(pos - start - (int64_t)unit * s.steps);
        const int s1 = (int)min((int64_t)s.steps, s0 + (hi - pos));
        const int tile = unit / p.Hkv, kvh = unit - tile * p.Hkv;
        const int row0 = tile * s.tile_rows, rows = min(s.tile_rows, s.n - row0);

        const int cw = wave & (s.waves - 1), kw = wave / s.waves;   // this wave's columns, and its tokens of a step
        const int c = 32 * cw + col;
        // (32 columns of a tile are 32 columns of its rows end to end; columns behind the last row repeat it)
        const int c_row = min(c / g, rows - 1), c_head = c % g;

        const int nblk = (s.len + kBlockSize - 1) / kBlockSize;
        const const_i32_ptr table = scalar_ptr(p.block_tables + (int64_t)seq * p.max_blocks_per_seq);
        auto id_at = [&](int block) -> int64_t {   // of the block of the sequence; blocks past the end: the last one
            const int64_t id = table[min(block, nblk - 1)];
            return min(max(id, (int64_t)0), p.num_blocks - 1);
        };
        Wave x;
        __syncthreads();   // (LDS: the last unit's results have been read)
        if (s.waves == 1) {
            x.begin(p, (int64_t)s.q0 + row0 + c_row, kvh * g + c_head, h);
            for (int st = s0; st < s1; ++st) {
                const int tok0 = st * kTreeStep + 32 * wave;
                if (tok0 >= s.len) break;
                const int64_t t0 = (id_at(tok0 / kBlockSize) * p.Hkv + kvh) * kTile, t1 = (id_at(tok0 / kBlockSize + 1) * p.Hkv + kvh) * kTile;
                u32x4 kr[KS], vr[2][MB];
                const u32x4 *const kp = reinterpret_cast<const u32x4 *>(p.k_cache + (ku ? t1 : t0));
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) kr[ks] = kp[(2 * ks + h) * kBlockSize + kslot];
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const u32x4 *const vp = reinterpret_cast<const u32x4 *>(p.v_cache + (b ? t1 : t0));
#pragma unroll
                    for (int mb = 0; mb < MB; ++mb) vr[b][mb] = vp[2 * (32 * mb + col) + h];
                }
                f32x16 S;
#pragma unroll
                for (int r = 0; r < 16; ++r) S[r] = 0.f;
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
                    S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kr[ks]), __builtin_bit_cast(bf16x8, x.qb[ks]), S, 0, 0, 0);
                if (tok0 + 32 > s.ctx) {   // nodes among the tokens
                    Wave::hide(S, x.sees(p.words, tok0, s.ctx, s.len), h);
                    const int left = s.len - tok0;
                    if (left < 32) {
#pragma unroll
                        for (int b = 0; b < 2; ++b) {   // (slots past the end may hold anything, and 0 * NaN is NaN)
                            const int first = 16 * b + 8 * h;
                            u32x4 keep;
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                keep[i] = (first + 2 * i < left ? 0x0000FFFFu : 0u) | (first + 2 * i + 1 < left ? 0xFFFF0000u : 0u);
#pragma unroll
                            for (int mb = 0; mb < MB; ++mb) vr[b][mb] &= keep;
                        }
                    }
                }
                u32x4 P[2];
                x.weights(S, p.scale_log2e, P);
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int mb = 0; mb < MB; ++mb)
                        x.O[mb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vr[b][mb]), __builtin_bit_cast(bf16x8, P[b]),
                                                                          x.O[mb], 0, 0, 0);
            }
        } else {
            // 64 tokens at a time: wave i brings block i of the four
            const int f0 = 2 * s0, f1 = min(2 * s1, (s.len + 63) / 64);   // stages (the last step may have one)
            auto stage = [&](int f) {
                const uint64_t tile_bytes = (uint64_t)(id_at(kStageBlocks * f + wave) * p.Hkv + kvh) * (kTile * 2);
                const uint32_t at = (uint32_t)(((f & 1) * kStageBlocks + wave) * CH * 16);
                const char *const kb = reinterpret_cast<const char *>(p.k_cache) + tile_bytes;
                const char *const vb = reinterpret_cast<const char *>(p.v_cache) + tile_bytes - kBias;
                tile_to_lds<HD>(kb, ldsK_at + at, k_off);
                tile_to_lds<HD>(vb, ldsV_at + at, v_off);
            };
            stage(f0);
            x.begin(p, (int64_t)s.q0 + row0 + c_row, kvh * g + c_head, h);
            const bool used = 32 * cw < rows * g;   // (the last tile may leave waves without columns: they only bring blocks)
            for (int f = f0; f < f1; ++f) {
                asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
                __syncthreads();   // everybody's tiles have landed, and everybody is done with the other buffer
                if (f + 1 < f1) stage(f + 1);
                const u32x4 *const K = ldsK + (f & 1) * kStageBlocks * CH;
                u32x4 *const V = ldsV + (f & 1) * kStageBlocks * CH;
                if (64 * f + 64 > s.len) {   // (slots past the end may hold anything, and 0 * NaN is NaN)
                    for (int i = tid; i < kStageBlocks * CH; i += kTreeThreads) {
                        const int first = 64 * f + 16 * (i / CH) + 8 * (i % CH / HD);
                        u32x4 keep;
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            keep[k] = (first + 2 * k < s.len ? 0x0000FFFFu : 0u) | (first + 2 * k + 1 < s.len ? 0xFFFF0000u : 0u);
                        V[i] &= keep;
                    }
                    __syncthreads();
                }
                if (!used) continue;
                for (int half = s.waves == 4 ? 0 : kw; half < (s.waves == 4 ? 2 : kw + 1); ++half) {
                    const int tok0 = 64 * f + 32 * half;
                    f32x16 S;
#pragma unroll
                    for (int r = 0; r < 16; ++r) S[r] = 0.f;
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks)
                        S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, K[(2 * half + ku) * CH + (2 * ks + h) * kBlockSize + kslot]),
                                                                    __builtin_bit_cast(bf16x8, x.qb[ks]), S, 0, 0, 0);
                    if (tok0 + 32 > s.ctx) Wave::hide(S, x.sees(p.words, tok0, s.ctx, s.len), h);
                    u32x4 P[2];
                    x.weights(S, p.scale_log2e, P);
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int mb = 0; mb < MB; ++mb)
                            x.O[mb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, V[(2 * half + b) * CH + h * HD + 32 * mb + col]),
                                                                              __builtin_bit_cast(bf16x8, P[b]), x.O[mb], 0, 0, 0);
                }
            }
            __syncthreads();   // (the buffers become the slab)
        }
        float l0, l1;
        swap32(x.lsum, l0, l1);

        // ---- the waves' results meet in LDS
        if (h == 0) {
            stat[wave][col][0] = x.m;
            stat[wave][col][1] = l0 + l1;
        }
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                *reinterpret_cast<f32x4 *>(&slab[wave][col][32 * mb + 8 * k + 4 * h]) =
                    f32x4{x.O[mb][4 * k], x.O[mb][4 * k + 1], x.O[mb][4 * k + 2], x.O[mb][4 * k + 3]};
        __syncthreads();
        constexpr int PER = HD / 8;               // dims of a thread: eight threads have a column
        const bool whole = s0 == 0 && s1 == s.steps;
        const int64_t slot = 2 * (int64_t)w + (pos == lo ? 0 : 1);
        for (int i = 0; i < s.waves; ++i) {
            const int oc = 32 * i + tid / 8, od = (tid & 7) * PER;
            const int o_row = oc / g, o_head = oc - o_row * g;
            if (o_row >= rows) break;
            float M = -INFINITY;
            for (int k = i; k < 4; k += s.waves) M = fmaxf(M, stat[k][oc & 31][0]);
            float l = 0.f;
            f32x4 acc[PER / 4];
#pragma unroll
            for (int j = 0; j < PER / 4; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
            for (int k = i; k < 4; k += s.waves) {
                const float weight = fast_exp2(stat[k][oc & 31][0] - M);
                l += stat[k][oc & 31][1] * weight;
#pragma unroll
                for (int j = 0; j < PER / 4; ++j) {
                    const f32x4 o = *reinterpret_cast<const f32x4 *>(&slab[k][oc & 31][od + 4 * j]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[j][e] = __builtin_fmaf(o[e], weight, acc[j][e]);
                }
            }
            if (whole) {
                const float inv = l == 0.f ? 0.f : 1.0f / l;   // (a row that sees nothing is zero)
                u32x2 *const op = reinterpret_cast<u32x2 *>(p.out + ((int64_t)(s.q0 + row0 + o_row) * p.Hq + kvh * g + o_head) * HD + od);
#pragma unroll
                for (int j = 0; j < PER / 4; ++j)
                    op[j] = u32x2{pack2_bf16(acc[j][0] * inv, acc[j][1] * inv), pack2_bf16(acc[j][2] * inv, acc[j][3] * inv)};
            } else {
                f32x4 *const ap = reinterpret_cast<f32x4 *>(p.part_acc + (slot * kTreeCols + oc) * HD + od);
#pragma unroll
                for (int j = 0; j < PER / 4; ++j) ap[j] = acc[j];
                if ((tid & 7) == 0) {
                    p.part_ml[(slot * kTreeCols + oc) * 2] = M;
                    p.part_ml[(slot * kTreeCols + oc) * 2 + 1] = l;
                }
            }
        }
        if (pos == lo && tid == 0) {
            // the run that the second part of a unit is in says where all its parts are
            const int64_t unit_lo = pos - s0;
            int parts = 0;
            if (s0 > 0 && w > 0 && unit_lo >= runs.first(w - 1)) {
                parts = runs.holding(unit_lo + s.steps - 1) - (w - 1) + 1;
                merge[0] = unit_lo == runs.first(w - 1) ? 0 : 1;   // which part of run w - 1 it is
                merge[2] = s.q0 + row0;
                merge[3] = rows;
                merge[4] = kvh;
            }
            merge[1] = parts;
        }
        pos += s1 - s0;
    }
}

// The parts of the units that runs have cut: workgroup (run, some of the columns) merges the unit whose second part is the first
// of that run, in the order of the parts.
template <int HD>
__global__ __launch_bounds__(kTreeThreads) void tree_merge_kernel(const TreeArgs p)
{
    constexpr int COLS = 2 * kTreeThreads / HD;     // columns of a workgroup: a thread has two dims
    const int w = blockIdx.x;
    const int32_t *const merge = p.merges + (int64_t)w * kMergeInts;
    const int parts = merge[1];
    if (parts == 0) return;
    const int second = merge[0], row0 = merge[2], rows = merge[3], kvh = merge[4];
    const int col = blockIdx.y * COLS + threadIdx.x / (HD / 2), d = 2 * (threadIdx.x % (HD / 2));
    const int row = col / p.g, head = col - row * p.g;
    if (row >= rows) return;
    auto slot_of = [&](int k) -> int64_t { return (2 * (int64_t)(w - 1 + k) + (k == 0 ? second : 0)) * kTreeCols + col; };
    float M = -1e30f, l = 0.f, a0 = 0.f, a1 = 0.f;
    for (int k = 0; k < parts; ++k) {
        const int64_t slot = slot_of(k);
        const f32x2 ml = *reinterpret_cast<const f32x2 *>(p.part_ml + 2 * slot);
        const f32x2 a = *reinterpret_cast<const f32x2 *>(p.part_acc + slot * HD + d);
        const float M_new = fmaxf(M, ml[0]);
        const float w_old = fast_exp2(M - M_new), w_new = fast_exp2(ml[0] - M_new);
        M = M_new;
        l = l * w_old + ml[1] * w_new;
        a0 = a0 * w_old + a[0] * w_new;
        a1 = a1 * w_old + a[1] * w_new;
    }
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    *reinterpret_cast<uint32_t *>(p.out + ((int64_t)(row0 + row) * p.Hq + kvh * p.g + head) * HD + d) = pack2_bf16(a0 * inv, a1 * inv);
}

namespace {
size_t run_bytes(int hd) { return kMergeInts * sizeof(int32_t) + 2 * (size_t)kTreeCols * (hd + 2) * sizeof(float); }
}  // namespace

int tree_runs_log2(int hd, int num_cus, size_t ws_bytes)
{
    int log2 = 0;
    while ((2 << log2) <= 2 * num_cus) ++log2;   // two workgroups per compute unit
    while (log2 >= 0 && (run_bytes(hd) << log2) > ws_bytes) --log2;
    return log2;
}

hipError_t launch_attn_tree(TreeArgs &a, void *ws, hipStream_t s)
{
    const unsigned runs = 1u << a.runs_log2;
    a.part_acc = static_cast<float *>(ws);
    a.part_ml = a.part_acc + (size_t)2 * runs * kTreeCols * a.hd;
    a.merges = reinterpret_cast<int32_t *>(a.part_ml + (size_t)2 * runs * kTreeCols * 2);
    const dim3 merge_grid(runs, (unsigned)(kTreeCols * a.hd / (2 * kTreeThreads)));
    if (a.hd == 128) {
        hipLaunchKernelGGL(tree_kernel<128>, dim3(runs), dim3(kTreeThreads), 0, s, a);
        hipLaunchKernelGGL(tree_merge_kernel<128>, merge_grid, dim3(kTreeThreads), 0, s, a);
    } else {
        hipLaunchKernelGGL(tree_kernel<64>, dim3(runs), dim3(kTreeThreads), 0, s, a);
        hipLaunchKernelGGL(tree_merge_kernel<64>, merge_grid, dim3(kTreeThreads), 0, s, a);
    }
    return hipGetLastError();
}

}  // namespace ooco
