// HIP kernels of libooco for gfx950: attention of a tree of drafted nodes over the paged KV cache.
//
// Row t of a sequence with n nodes on ctx cached tokens sees tokens 0 .. ctx-1 and those nodes j whose bit of its mask is set.
// As in the other attention kernels scores are computed transposed, S^T[token][query column] = K Q^T, and the output as
// O^T[dim][query column] = V^T P^T; a query column is a (row, head of the GQA group) pair, so that the K and V of a token are
// fetched once for all nodes and heads that see it.  One pass over the keys with the running maximum and sum of the softmax.
//
// Work: tile = 32 / g rows of a sequence, all heads of a group (32 columns); unit = (tile, kv head); a unit walks its sequence's
// tokens in steps of 128, 32 for each of the workgroup's four waves.  The units of all sequences, steps end to end, form a line
// that is cut into equal runs, a workgroup each; where a run ends inside a unit, partial results meet in the merge kernel.  The
// lengths are read and the line is laid out on the device by every workgroup for itself: no plan and no host copy of lengths that
// the last step's verification has just decided.
#include "ooco_device.h"
#include "ooco_internal.h"
#include "ooco_spec.h"

#include <algorithm>

namespace ooco {

constexpr int kTreeCols = 32;         // query columns of a tile
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
    int q0, n, ctx, len, tiles, steps;   // len: tokens that exist, the nodes among them
    int64_t units;                       // steps of all its units
};
OOCO_DEV int tile_rows_of(int g) { return kTreeCols / g; }
OOCO_DEV TreeSeq tree_seq(const TreeArgs &p, int q0, int q1, int ctx)
{
    TreeSeq s;
    s.q0 = q0;
    s.n = q1 - q0;
    if (q0 < 0 || s.n < 0 || s.n > p.total_q - q0) s.n = 0;
    const int cap = (int)min((int64_t)p.max_blocks_per_seq * kBlockSize, (int64_t)INT32_MAX - 1024);
    s.ctx = min(max(ctx, 0), cap);
    s.len = min(s.ctx + min(s.n, 64 * p.words), cap);
    const int rows = tile_rows_of(p.g);
    s.tiles = (s.n + rows - 1) / rows;
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

// Runs of the line: run w = [first(w), first(w + 1)).  No run is empty but those behind `count`.
struct TreeRuns {
    int64_t total;
    int log2;
    bool split;      // the line is cut into all runs there are, else into runs of kMinRun steps
    OOCO_DEV TreeRuns(int64_t total_, int log2_) : total(total_), log2(log2_), split(total_ >= ((int64_t)kMinRun << log2_)) {}
    OOCO_DEV int64_t first(int w) const { return split ? (total * w) >> log2 : min(total, (int64_t)w * kMinRun); }
    OOCO_DEV int holding(int64_t x) const { return split ? (int)((((x + 1) << log2) - 1) / total) : (int)(x / kMinRun); }
};

template <int HD>
__global__ __launch_bounds__(kTreeThreads, 2) void tree_kernel(const TreeArgs p)
{
    constexpr int KS = HD / 16;                   // k-steps of QK
    constexpr int MB = HD / 32;                   // 32-dim groups of the output
    constexpr int ROW = HD + 4;                   // floats of a column in LDS (padded: the lanes of a wave are columns)
    constexpr int64_t kTile = (int64_t)HD * kBlockSize;
    __shared__ __align__(16) float slab[4][kTreeCols][ROW];
    __shared__ float stat[4][kTreeCols][2];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, h = lane >> 5;
    const int g = p.g;
    const int w = blockIdx.x;

    int seq = 0;
    int64_t start = 0;
    const int64_t total = tree_locate(p, [&](int64_t t) { return TreeRuns(t, p.runs_log2).first(w); }, seq, start);
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

    int64_t pos = lo;
    seq = __builtin_amdgcn_readfirstlane(seq);
    TreeSeq s = tree_seq(p, p.query_start_loc[seq], p.query_start_loc[seq + 1], p.ctx_lens[seq]);
    while (pos < hi) {
        while (pos - start >= s.units) {   // the next sequence with rows
            start += s.units;
            ++seq;
            s = tree_seq(p, p.query_start_loc[seq], p.query_start_loc[seq + 1], p.ctx_lens[seq]);
        }
        const int unit = (int)((pos - start) / s.steps);
        const int s0 = (int)(pos - start - (int64_t)unit * s.steps);
        const int s1 = (int)min((int64_t)s.steps, s0 + (hi - pos));
        const int tile = unit / p.Hkv, kvh = unit - tile * p.Hkv;
        const int rows_max = tile_rows_of(g);
        const int row0 = tile * rows_max, rows = min(rows_max, s.n - row0);

        // ---- this lane's query column and its mask
        const int c_row = min(col / g, rows - 1), c_head = col % g;
        const int64_t q_row = s.q0 + row0 + c_row;
        u32x4 qb[KS];
        {
            const u32x4 *qp = reinterpret_cast<const u32x4 *>(p.q + (q_row * p.Hq + kvh * g + c_head) * HD);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) qb[ks] = qp[2 * ks + h];
        }
        const uint64_t *const mask = p.masks + q_row * p.words;

        const int nblk = (s.len + kBlockSize - 1) / kBlockSize;
        const int32_t *const table = p.block_tables + (int64_t)seq * p.max_blocks_per_seq;
        auto tile_at = [&](int block) -> int64_t {   // of the block of the sequence; blocks past the end: the last one
            const int64_t id = table[min(block, nblk - 1)];
            return (min(max(id, (int64_t)0), p.num_blocks - 1) * p.Hkv + kvh) * kTile;
        };

        f32x16 O[MB];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int r = 0; r < 16; ++r) O[mb][r] = 0.f;
        float m = -1e30f, lsum = 0.f;   // (finite: tokens that a column does not see weigh nothing, where -inf - -inf would make them NaN)
        for (int st = s0; st < s1; ++st) {
            const int tok0 = st * kTreeStep + 32 * wave;
            if (tok0 >= s.len) break;
            const int64_t t0 = tile_at(tok0 / kBlockSize), t1 = tile_at(tok0 / kBlockSize + 1);
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
                S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kr[ks]), __builtin_bit_cast(bf16x8, qb[ks]), S, 0, 0, 0);
            if (tok0 + 32 > s.ctx) {   // nodes among the tokens
                const int j0 = tok0 - s.ctx;   // node that token tok0 is (negative: cached)
                uint32_t bits;
                if (j0 >= 0) {
                    const int k = j0 >> 6, sh = j0 & 63;
                    uint64_t b = k < p.words ? mask[k] >> sh : 0;
                    if (sh > 32 && k + 1 < p.words) b |= mask[k + 1] << (64 - sh);
                    bits = (uint32_t)b;
                } else {
                    bits = ((uint32_t)mask[0] << -j0) | ((1u << -j0) - 1u);   // (-31 <= j0)
                }
                const int left = s.len - tok0;   // tokens that exist
                if (left < 32) {
                    bits &= (1u << left) - 1u;
#pragma unroll
                    for (int b = 0; b < 2; ++b) {   // (slots past the end may hold anything, and 0 * NaN is NaN)
                        const int first = 16 * b + 8 * h;
                        u32x4 keep;
#pragma unroll
                        for (int x = 0; x < 4; ++x)
                            keep[x] = (first + 2 * x < left ? 0x0000FFFFu : 0u) | (first + 2 * x + 1 < left ? 0xFFFF0000u : 0u);
#pragma unroll
                        for (int mb = 0; mb < MB; ++mb) vr[b][mb] &= keep;
                    }
                }
                bits >>= 8 * h;
#pragma unroll
                for (int r = 0; r < 16; ++r) S[r] = (bits >> (16 * (r / 8) + r % 8)) & 1u ? S[r] : -INFINITY;
            }
            float x, y;
            swap32(largest(S), x, y);
            const float m_new = __builtin_elementwise_maximum(m, __builtin_elementwise_maximum(x, y) * p.scale_log2e);
            const float alpha = fast_exp2(m - m_new);
            const bool grow = m_new > m;
            m = m_new;
            float psum = 0.f;
            u32x4 P[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                float e[8];
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    e[r] = fast_exp2(__builtin_fmaf(S[8 * b + r], p.scale_log2e, -m));
                    psum += e[r];
                }
                P[b] = u32x4{pack2_bf16(e[0], e[1]), pack2_bf16(e[2], e[3]), pack2_bf16(e[4], e[5]), pack2_bf16(e[6], e[7])};
            }
            lsum = lsum * alpha + psum;
            if (__any(grow)) {
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                    for (int r = 0; r < 16; ++r) O[mb][r] *= alpha;
            }
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
                    O[mb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vr[b][mb]), __builtin_bit_cast(bf16x8, P[b]), O[mb], 0, 0, 0);
        }
        float x, y;
        swap32(lsum, x, y);
        lsum = x + y;

        // ---- the four waves' results meet in LDS
        __syncthreads();   // (the last unit's have been read)
        if (h == 0) {
            stat[wave][col][0] = m;
            stat[wave][col][1] = lsum;
        }
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                *reinterpret_cast<f32x4 *>(&slab[wave][col][32 * mb + 8 * k + 4 * h]) =
                    f32x4{O[mb][4 * k], O[mb][4 * k + 1], O[mb][4 * k + 2], O[mb][4 * k + 3]};
        __syncthreads();
        constexpr int PER = HD / 8;               // dims of a thread: eight threads have a column
        const int oc = tid / 8, od = (tid & 7) * PER;
        const int o_row = oc / g, o_head = oc - o_row * g;
        float M = stat[0][oc][0], weight[4], l = 0.f;
#pragma unroll
        for (int k = 1; k < 4; ++k) M = fmaxf(M, stat[k][oc][0]);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            weight[k] = fast_exp2(stat[k][oc][0] - M);
            l += stat[k][oc][1] * weight[k];
        }
        f32x4 acc[PER / 4];
#pragma unroll
        for (int i = 0; i < PER / 4; ++i) {
            acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const f32x4 o = *reinterpret_cast<const f32x4 *>(&slab[k][oc][od + 4 * i]);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][e] = __builtin_fmaf(o[e], weight[k], acc[i][e]);
            }
        }
        if (s0 == 0 && s1 == s.steps) {
            if (o_row < rows) {
                const float inv = l == 0.f ? 0.f : 1.0f / l;   // (a row that sees nothing is zero)
                u32x2 *const op = reinterpret_cast<u32x2 *>(p.out + ((int64_t)(s.q0 + row0 + o_row) * p.Hq + kvh * g + o_head) * HD + od);
#pragma unroll
                for (int i = 0; i < PER / 4; ++i)
                    op[i] = u32x2{pack2_bf16(acc[i][0] * inv, acc[i][1] * inv), pack2_bf16(acc[i][2] * inv, acc[i][3] * inv)};
            }
        } else {
            const int64_t slot = 2 * (int64_t)w + (pos == lo ? 0 : 1);
            f32x4 *const ap = reinterpret_cast<f32x4 *>(p.part_acc + (slot * kTreeCols + oc) * HD + od);
#pragma unroll
            for (int i = 0; i < PER / 4; ++i) ap[i] = acc[i];
            if ((tid & 7) == 0) {
                p.part_ml[(slot * kTreeCols + oc) * 2] = M;
                p.part_ml[(slot * kTreeCols + oc) * 2 + 1] = l;
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

// The parts of the units that runs have cut: workgroup (run, eighth of the columns) merges the unit whose second part is the first
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
