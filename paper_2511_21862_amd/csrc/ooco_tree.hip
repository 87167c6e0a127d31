// HIP kernels of libooco for gfx950: attention of a tree of drafted nodes over the paged KV cache.
//
// Row t of a sequence with n nodes on ctx cached tokens sees tokens 0 .. ctx-1 and those nodes j whose bit of its mask is set.
// As in the other attention kernels scores are computed transposed, S^T[token][query column] = K Q^T, and the output as
// O^T[dim][query column] = V^T P^T; a query column is a (row, head of the GQA group) pair, so that the K and V of a token are
// fetched once for all nodes and heads that see it.  One pass over the keys with the running maximum and sum of the softmax.
//
// Work: the columns of a sequence are cut into tiles of 32 for each of the NW = 4 or 8 waves of a workgroup, the last tile as wide as 32, 64,
// 128 or 256 columns have to be; the waves that columns leave over share the tokens.  Unit = (kv head, tile), walked in steps of 128
// tokens.  The units of all sequences, steps end to end, form a line that is cut into equal runs, a workgroup each, two of four waves to a
// compute unit or one of eight; where a run ends inside a unit, partial results meet in the merge kernel.  The lengths are read and the
// line is laid out on the device by every workgroup for itself: no plan and no host copy of lengths that the last step's verification has
// just decided.
//   32 columns        every wave loads K and V of its own tokens from the cache to the registers of the matrix instructions: nothing is
//                     shared, so nobody waits for anybody, and a compute unit has 128 KiB on their way
//   more              K and V of 64 tokens at a time go through LDS by direct loads into the other of two buffers
//   32 for each wave  the products of 32 tokens run beside the exponentials of 32 others (see region)
// Few sequences of up to 64 columns have a kernel of their own, in which a wave's registers hold all columns (see tree_stream_kernel).
// What bounds it, on MI355X: memory for small trees (32 sequences of 8 nodes of 32/8 heads on 4096 tokens: 88.5 us, 6.1 TB/s; a large copy
// moves 5.2); for wide ones the matrix cores and the LDS ports that feed them, each busy half of the cycles at 1.9 GHz (8 sequences of 64
// nodes of 64/8 heads on 14,000: 248 us, 945 TFLOP/s of the 1226 that a large product of matrices reaches); the chain lengths - block ids -
// tiles - merge for one small sequence (8 nodes on 700 tokens: 10.2 us).
#include "ooco_device.h"
#include "ooco_internal.h"
#include "ooco_spec.h"

#include <algorithm>
#include <type_traits>

namespace ooco {

constexpr int kTreeStep = 128;               // tokens of a step
constexpr int kMaskRow = kMaxMaskWords + 1;  // words of a mask in LDS (padded: the lanes of a wave are columns)
// Steps of the line that a unit has beyond its own, so that a run of many short units is not the last to end: the first loads, which nothing
// hides, and the end of a unit take about as long.  Not on lines of less than four steps a run, whose runs begin and end one unit anyway.
// (MI355X, us, 0 / 1 / 2 / 4 of them: 32 sequences of 5 .. 16 nodes on 512 .. 8192 tokens, 32/8 heads 113.5 / 107.7 / 103.4 / 102.7, of 64 nodes
// 194 / 184 / 181 / 179, 64 of 16 nodes 217 / 213 / 212 / 218.)
constexpr int kUnitSteps = 2;
constexpr int kMergeInts = 5;
constexpr int kMergeThreads = 256;

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
    int q0, n, ctx, len, steps;      // len: tokens that exist, the nodes among them
    int length;                      // of a unit on the line: its steps, and what its beginning and end take
    int tile_rows, tiles;            // rows of a tile but the last
    int last_waves;                  // waves that have columns of the last tile: 1, 2, 4 or 8
    int64_t units;                   // steps of all its units
};
OOCO_DEV TreeSeq tree_seq(const TreeArgs &p, int q0, int q1, int ctx, int pad)
{
    TreeSeq s;
    s.q0 = q0;
    s.n = q1 - q0;
    if (q0 < 0 || s.n < 0 || s.n > p.total_q - q0) s.n = 0;
    const int cap = (int)min((int64_t)p.max_blocks_per_seq * kBlockSize, (int64_t)INT32_MAX - 1024);
    s.ctx = min(max(ctx, 0), cap);
    s.len = (int)min((int64_t)s.ctx + min(s.n, 64 * p.words), (int64_t)cap);
    s.steps = (s.len + kTreeStep - 1) / kTreeStep;
    s.length = s.steps + pad;
    s.tile_rows = p.tile_rows;       // (a group of heads that does not divide a tile: the columns behind the last whole row are none)
    s.tiles = (s.n + s.tile_rows - 1) / s.tile_rows;
    const int last_cols = (s.n - (s.tiles - 1) * s.tile_rows) * p.g;
    s.last_waves = last_cols <= 32 ? 1 : last_cols <= 64 ? 2 : last_cols <= 128 ? 4 : 8;
    s.units = (int64_t)s.tiles * p.Hkv * s.length;
    return s;
}
// floor(a / b) of numbers below 2^53: a correctly rounded quotient does not reach the next integer.  (The compiler's 64-bit division
// is some hundred instructions, and instructions are what a small launch waits for.)
OOCO_DEV int64_t quotient(int64_t a, int64_t b) { return (int64_t)((double)a / (double)b); }

// Values that are the same in every lane, in scalar registers.
OOCO_DEV int64_t uniform(int64_t v)
{
    const uint32_t lo = __builtin_amdgcn_readfirstlane((int)(uint32_t)v), hi = __builtin_amdgcn_readfirstlane((int)(v >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}
// Lengths and block ids by scalar loads, which the waits on the vector-memory counter do not see.
typedef const __attribute__((address_space(4))) int32_t *const_i32_ptr;
OOCO_DEV const_i32_ptr scalar_ptr(const int32_t *p) { return (const_i32_ptr)(uintptr_t)p; }
OOCO_DEV TreeSeq tree_seq_at(const TreeArgs &p, int seq, int pad)
{
    const const_i32_ptr qsl = scalar_ptr(p.query_start_loc), ctx = scalar_ptr(p.ctx_lens);
    return tree_seq(p, qsl[seq], qsl[seq + 1], ctx[seq], pad);
}

// Runs of the line: run w = [first(w), first(w + 1)).  No run is empty but those behind the last.  As many as there are workgroups, or half as
// many (see launch); on a line shorter than that a run for each step, which takes the shortest time.
struct TreeRuns {
    int64_t total;
    int log2;
    bool split;      // the line is cut into 1 << log2 runs, else into runs of one step
    OOCO_DEV TreeRuns(const TreeArgs &p, int64_t total_)
        : total(total_), log2(total_ < p.halve_below ? p.runs_log2 - 1 : p.runs_log2), split(total_ >= ((int64_t)1 << log2))
    {
    }
    OOCO_DEV int64_t first(int w) const { return split ? (w >> log2 ? total : (total * w) >> log2) : min(total, (int64_t)w); }
    OOCO_DEV int holding(int64_t x) const { return split ? (int)quotient(((x + 1) << log2) - 1, total) : (int)x; }
};

// The line: its length, and the sequence that holds position at(total) of it, with the position of that sequence's first step.
// All threads of the workgroup call it together.  Up to 64 sequences on a line of 31 bits: every wave looks them up for itself, a lane
// each; the values that it needs next are then a lane away, and the next loads can go.
template <int NT, class At>
OOCO_DEV int64_t tree_locate(const TreeArgs &p, At at, int &seq, int64_t &start, TreeSeq &found)
{
    if (p.short_line) {
        const int i = threadIdx.x & 63, j = min(i, p.num_seqs - 1);
        const int q0 = p.query_start_loc[j], q1 = p.query_start_loc[j + 1], ctx = p.ctx_lens[j];
        const TreeSeq own = tree_seq(p, q0, q1, ctx, 0);
        auto scan = [&](int v) -> int {
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int o = __shfl_up(v, d);
                v += i >= d ? o : 0;
            }
            return v;
        };
        int units = i < p.num_seqs ? (int)own.units : 0, incl = scan(units), total = __builtin_amdgcn_readlane(incl, 63), pad = 0;
        if (total >= (int64_t)4 << p.runs_log2) {
            pad = kUnitSteps;
            units += i < p.num_seqs ? own.tiles * p.Hkv * pad : 0;
            incl = scan(units);
            total = __builtin_amdgcn_readlane(incl, 63);
        }
        const int64_t x = at((int64_t)total);
        seq = min(__popcll(__ballot(incl <= x)), p.num_seqs - 1);
        start = __builtin_amdgcn_readlane(incl - units, seq);
        found = tree_seq(p, __builtin_amdgcn_readlane(q0, seq), __builtin_amdgcn_readlane(q1, seq), __builtin_amdgcn_readlane(ctx, seq), pad);
        return total;
    }
    __shared__ int64_t wave_total[NT / 64];
    __shared__ int sh_seq;
    __shared__ int64_t sh_start;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int pad = 0;
    auto units_of = [&](int i) -> int64_t {
        return i < p.num_seqs ? tree_seq(p, p.query_start_loc[i], p.query_start_loc[i + 1], p.ctx_lens[i], pad).units : 0;
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
        for (int w = 0; w < NT / 64; ++w) {
            before += w < wave ? wave_total[w] : 0;
            all += wave_total[w];
        }
        return before + x;
    };
    int64_t total = 0, all, mine = 0, incl = 0;
    auto measure = [&]() {
        total = 0;
        for (int base = 0; base < p.num_seqs; base += NT) {
            mine = units_of(base + tid);
            incl = scan(mine, all);
            total += all;
        }
    };
    measure();
    if (total >= (int64_t)4 << p.runs_log2) {   // (the same in every thread)
        pad = kUnitSteps;
        measure();
    }
    const int64_t x = at(total);
    int64_t before = 0;
    for (int base = 0; base < p.num_seqs; base += NT) {
        if (p.num_seqs > NT) {
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
    if (x >= total) return uniform(total);
    seq = __builtin_amdgcn_readfirstlane(sh_seq);
    start = uniform(sh_start);
    found = tree_seq_at(p, seq, pad);
    return uniform(total);
}

// The workgroup's run, w, and the sequence that it begins in, with the position of that sequence's first step.
// Runs next to each other on the line are on one XCD (workgroup b runs on XCD b % 8): the tiles of one sequence and kv head walk the same
// tokens at about the same time, and share an L2 (512 columns on 14,000 tokens, us: 286 -> 255).  A line of runs of one step is spread over
// the XCDs.
template <int NT>
OOCO_DEV TreeRuns tree_run(const TreeArgs &p, int &w, int &seq, int64_t &start, TreeSeq &s)
{
    w = blockIdx.x;
    const int64_t total = tree_locate<NT>(
        p,
        [&](int64_t t) {
            const TreeRuns r(p, t);
            if (r.split && r.log2 >= 3 && w >> r.log2 == 0) w = (w & 7) << (r.log2 - 3) | w >> 3;
            return r.first(w);
        },
        seq, start, s);
    return TreeRuns(p, total);
}

// What a wave does with 32 tokens, whichever way they come: its 32 query columns' share of the softmax and of the output.
// KEPT: masks are read from LDS, where K and V are too.  A load from where they lie would wait for the K and V ahead of it, at every 32 nodes (20
// .. 27 nodes of 28/4 heads on 60..131K tokens, 4 sequences, us: 226 -> 208; 64 nodes of 32/8 on 4096, 64 sequences: 322 -> 307).  Small trees
// whose K and V go to registers have few such loads, and are the slower for the way through LDS (8 nodes on 300, 128 sequences, us: 41.5 /
// 46.0; 5 .. 16 on 512 .. 8192, 32 sequences: 113.5 / 115.9).
template <int HD>
struct TreeWave {
    static constexpr int KS = HD / 16;   // k-steps of QK
    static constexpr int MB = HD / 32;   // 32-dim groups of the output
    u32x4 qb[KS];
    f32x16 O[MB];
    float m, lsum;                       // reference of the column's weights in log2 units, this lane's share of their sum
    float scale;                         // of scores, to log2 units
    const uint64_t *mask;                // the column's; in LDS after keep_mask

    OOCO_DEV void begin(const TreeArgs &p, int64_t q_row, int head, int h)
    {
        const u32x4 *const qp = reinterpret_cast<const u32x4 *>(p.q + (q_row * p.Hq + head) * HD);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qb[ks] = qp[2 * ks + h];
        mask = p.masks + q_row * p.words;
        scale = p.scale_log2e;
        none();
    }
    OOCO_DEV void none()   // no tokens
    {
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int r = 0; r < 16; ++r) O[mb][r] = 0.f;
        m = -1e30f;   // (finite: tokens that a column does not see weigh nothing, where -inf - -inf would make them NaN)
        lsum = 0.f;
    }
    // The mask to LDS, for hide<true>; words behind the mask's own are zero.
    OOCO_DEV void keep_mask(uint64_t (&row)[kMaskRow], int words, int h)
    {
#pragma unroll
        for (int i = 0; i < kMaxMaskWords / 2; ++i) {
            const int k = kMaxMaskWords / 2 * h + i;
            row[k] = k < words ? mask[k] : 0;
        }
        mask = row;
    }
    // Hides the scores of tokens that the column does not see.  Register r of S is token tok0 + 16 (r / 8) + 8 h + r % 8.
    template <bool KEPT>
    OOCO_DEV void hide(f32x16 &S, int words, int tok0, int ctx, int len, int h) const
    {
        const int j0 = tok0 - ctx;   // node that token tok0 is (negative: cached)
        if (j0 <= -32) return;
        uint32_t bits;               // bit i: the column sees token tok0 + i
        if (j0 >= 0) {
            const int k = j0 >> 6, sh = j0 & 63;
            uint64_t b = k < (KEPT ? kMaxMaskWords : words) ? mask[k] >> sh : 0;
            if (sh > 32 && k + 1 < (KEPT ? kMaxMaskWords : words)) b |= mask[k + 1] << (64 - sh);
            bits = (uint32_t)b;
        } else {
            bits = ((uint32_t)mask[0] << -j0) | ((1u << -j0) - 1u);
        }
        const int left = len - tok0;   // tokens that exist
        if (left < 32) bits &= left > 0 ? (1u << left) - 1u : 0u;
        bits >>= 8 * h;
#pragma unroll
        for (int r = 0; r < 16; ++r) S[r] = (bits >> (16 * (r / 8) + r % 8)) & 1u ? S[r] : -INFINITY;
    }
    // Weights are taken against a reference that moves only where scores exceed it by 2^8: weights up to 2^8 are as exact in bf16
    // and fp32 as below 1, and the division at the end takes the reference out.
    OOCO_DEV static constexpr float slack() { return 8.0f; }
    OOCO_DEV float top(const f32x16 &S) const
    {
        float x, y;
        swap32(largest(S), x, y);
        return __builtin_elementwise_maximum(x, y) * scale;
    }
    OOCO_DEV void move(float to)
    {
        const float m_new = fmaxf(m, to), alpha = fast_exp2(m - m_new);
        m = m_new;
        lsum *= alpha;
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int r = 0; r < 16; ++r) O[mb][r] *= alpha;
    }
    // Scores to weights, and this lane's sum of them.
    OOCO_DEV float weights(const f32x16 &S, u32x4 (&P)[2]) const
    {
        float sum = 0.f;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            float e[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                e[r] = fast_exp2(__builtin_fmaf(S[8 * b + r], scale, -m));
                sum += e[r];
            }
            P[b] = u32x4{pack2_bf16(e[0], e[1]), pack2_bf16(e[2], e[3]), pack2_bf16(e[4], e[5]), pack2_bf16(e[6], e[7])};
        }
        return sum;
    }
    OOCO_DEV void add(const f32x16 &S, u32x4 (&P)[2])
    {
        const float t = top(S);
        if (__any(t > m + slack())) move(t);
        lsum += weights(S, P);
    }
};

// A column of a unit: the n waves that have it left sums and weights in LDS, `apart` rows from each other.  NT / 32 threads take it, to its
// place in the output or, of a unit that runs have cut, among the partial results.
template <int HD, int NT, int ROW>
OOCO_DEV void tree_column(const TreeArgs &p, const float (*slab)[ROW], const float (*stat)[2], int at, int apart, int n, bool whole, int64_t part,
                          int row0, int col, int kvh)
{
    constexpr int TC = NT / 32, PER = HD / TC;   // threads of a column, dims of each
    const int d = threadIdx.x % TC * PER;
    float M = -INFINITY, l = 0.f;
    for (int k = 0; k < n; ++k) M = fmaxf(M, stat[at + k * apart][0]);
    f32x4 acc[PER / 4];
#pragma unroll
    for (int j = 0; j < PER / 4; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < n; ++k) {
        const float weight = fast_exp2(stat[at + k * apart][0] - M);
        l += stat[at + k * apart][1] * weight;
#pragma unroll
        for (int j = 0; j < PER / 4; ++j) {
            const f32x4 o = *reinterpret_cast<const f32x4 *>(&slab[at + k * apart][d + 4 * j]);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[j][e] = __builtin_fmaf(o[e], weight, acc[j][e]);
        }
    }
    if (whole) {
        const float inv = l == 0.f ? 0.f : 1.0f / l;   // (a row that sees nothing is zero)
        const int row = col / p.g, head = kvh * p.g + col - row * p.g;
        u32x2 *const op = reinterpret_cast<u32x2 *>(p.out + ((int64_t)(row0 + row) * p.Hq + head) * HD + d);
#pragma unroll
        for (int j = 0; j < PER / 4; ++j)
            op[j] = u32x2{pack2_bf16(acc[j][0] * inv, acc[j][1] * inv), pack2_bf16(acc[j][2] * inv, acc[j][3] * inv)};
    } else {
        f32x4 *const ap = reinterpret_cast<f32x4 *>(p.part_acc + part * HD + d);
#pragma unroll
        for (int j = 0; j < PER / 4; ++j) ap[j] = acc[j];
        if (d == 0) *reinterpret_cast<f32x2 *>(p.part_ml + 2 * part) = f32x2{M, l};
    }
}

// A wave's share of the loads of a tile of K or of V (one block, one kv head) from the cache into LDS: NL loads of 16 bytes per lane, 1 KiB each,
// contiguous in LDS from dst on.  off[n]: the lane's place in the tile for load n, less n KiB (the instruction's offset counts for both
// addresses).  once: nobody else reads the tile, so it need not push anything out of the caches (64 sequences of 16 nodes on 4096 tokens,
// 32/8 heads, us: 197 -> 177).
template <int NL>
OOCO_DEV void tile_to_lds(const char *base, uint32_t dst, const uint32_t (&off)[NL], bool once)
{
    uint32_t saved_m0;   // M0 is restored: the compiler may keep a value of its own there
#define OOCO_ASM(loads, ...) \
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t" loads "s_mov_b32 m0, %0" : "=&s"(saved_m0) : "s"(dst), "s"(base), __VA_ARGS__ : "memory")
#define OOCO_LOAD(v, at, nt) "global_load_lds_dwordx4 " v ", %2 offset:" at nt "\n\t"
    if constexpr (NL == 4) {
        if (once)
            OOCO_ASM(OOCO_LOAD("%3", "0", " nt") OOCO_LOAD("%4", "1024", " nt") OOCO_LOAD("%5", "2048", " nt") OOCO_LOAD("%6", "3072", " nt"),
                     "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]));
        else
            OOCO_ASM(OOCO_LOAD("%3", "0", "") OOCO_LOAD("%4", "1024", "") OOCO_LOAD("%5", "2048", "") OOCO_LOAD("%6", "3072", ""),
                     "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]));
    } else if constexpr (NL == 2) {
        if (once)
            OOCO_ASM(OOCO_LOAD("%3", "0", " nt") OOCO_LOAD("%4", "1024", " nt"), "v"(off[0]), "v"(off[1]));
        else
            OOCO_ASM(OOCO_LOAD("%3", "0", "") OOCO_LOAD("%4", "1024", ""), "v"(off[0]), "v"(off[1]));
    } else {
        static_assert(NL == 1, "loads of a wave");
        if (once)
            OOCO_ASM(OOCO_LOAD("%3", "0", " nt"), "v"(off[0]));
        else
            OOCO_ASM(OOCO_LOAD("%3", "0", ""), "v"(off[0]));
    }
#undef OOCO_ASM
#undef OOCO_LOAD
}

constexpr int kStageTokens = 64;                              // tokens that go through LDS at a time
constexpr int kStageBlocks = kStageTokens / kBlockSize;       // a block for each of four waves to bring, or half a block for each of eight
static_assert(kTreeStep == 2 * kStageTokens, "stages of a step");

template <int HD, int NW>
__global__ __launch_bounds__(64 * NW, 2) void tree_kernel(const TreeArgs p)
{
    constexpr int NT = 64 * NW, COLS = 32 * NW;
    constexpr int SHARE = NW / kStageBlocks;      // waves that bring a block
    constexpr int NL = HD / 32 / SHARE;           // loads of a wave for its share of a tile
    using Wave = TreeWave<HD>;
    constexpr int KS = Wave::KS, MB = Wave::MB;
    constexpr int ROW = HD + 4;                   // floats of a column in LDS (padded: the lanes of a wave are columns)
    constexpr int CH = 2 * HD;                    // 16-byte pieces of a tile of K or V
    constexpr int STAGE = kStageBlocks * CH;
    constexpr int64_t kTile = (int64_t)HD * kBlockSize;
    constexpr int kSlab = NW * 32 * ROW * 4, kStage = 2 * 2 * STAGE * 16;
    __shared__ __align__(16) unsigned char lds[kSlab > kStage ? kSlab : kStage];
    __shared__ __align__(8) float stat[NW][32][2];
    __shared__ uint64_t masks[NW][32][kMaskRow];
    float (*const slab)[32][ROW] = reinterpret_cast<float (*)[32][ROW]>(lds);           // [wave][column][dim]
    u32x4 *const ldsK = reinterpret_cast<u32x4 *>(lds), *const ldsV = ldsK + 2 * STAGE;   // [buffer][block][piece]

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, h = lane >> 5;
    const int g = p.g;
    int w, seq = 0;
    int64_t start = 0;
    TreeSeq s = {};
    const TreeRuns runs = tree_run<NT>(p, w, seq, start, s);
    const int64_t lo = runs.first(w), hi = runs.first(w + 1);
    int32_t *const merge = p.merges + (int64_t)w * kMergeInts;
    if (lo >= hi) {
        if (tid == 0) merge[0] = 0;
        return;
    }
    // K operand row col -> block (col >> 4) of the 32 tokens, slot with bits 2 and 3 swapped, so that register r of S^T is token
    // 16 (r / 8) + 8 h + r % 8: eight consecutive tokens of a block, as a 16-byte piece of V has them
    const int ku = col >> 4, kslot = (col & 3) | ((col & 4) << 1) | ((col & 8) >> 1);
    // Pieces of a tile in LDS: K as in the cache, V [half of the tokens][dim], so that the lanes that read together read side by side.  Where
    // this wave's share of a tile comes from:
    constexpr int kBias = 4096;   // (keeps the offsets of V positive)
    const int share = (wave & (SHARE - 1)) * NL * 64;   // first piece
    uint32_t k_off[NL], v_off[NL];
#pragma unroll
    for (int n = 0; n < NL; ++n) {
        const int c = share + 64 * n + lane;
        k_off[n] = (uint32_t)(share + lane) * 16u;
        v_off[n] = (uint32_t)((2 * (c % HD) + c / HD) * 16 - n * 1024 + kBias);
    }
    const uint32_t ldsK_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)ldsK;
    const uint32_t ldsV_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)ldsV;

    int64_t pos = lo;
    int parts = 0, first_run = 0;   // of the unit that the run begins inside of
    while (pos < hi) {
        while (pos - start >= s.units) {   // the next sequence with rows
            start += s.units;
            ++seq;
            s = tree_seq_at(p, seq, s.length - s.steps);
        }
        const int unit = (int)quotient(pos - start, s.length);
        const int s0 = (int)(pos - start - (int64_t)unit * s.length);
        if (s0 >= s.steps) {
            pos += s.length - s0;
            continue;
        }
        const int s1 = (int)min((int64_t)s.steps, s0 + (hi - pos));
        const int kvh = s.tiles == 1 ? unit : unit / s.tiles, tile = unit - kvh * s.tiles;
        const int waves = tile == s.tiles - 1 ? s.last_waves : NW;
        const int row0 = tile * s.tile_rows, rows = min(s.tile_rows, s.n - row0);

        const int cw = wave & (waves - 1), kw = wave / waves;   // this wave's columns, and its share of the tokens
        // (32 columns of a tile are 32 columns of its rows end to end; columns behind the last row repeat it)
        const int c = 32 * cw + col, c_row = min(c / g, rows - 1), c_head = c % g;
        const int64_t q_row = (int64_t)s.q0 + row0 + c_row;

        const int nblk = (s.len + kBlockSize - 1) / kBlockSize;
        const const_i32_ptr table = scalar_ptr(p.block_tables + (int64_t)seq * p.max_blocks_per_seq);
        const int last_id = (int)min(p.num_blocks, (int64_t)INT32_MAX) - 1;
        auto id_at = [&](int block) -> int { return table[min(block, nblk - 1)]; };   // blocks past the end: the last one
        auto bytes_at = [&](int id) -> int64_t { return ((int64_t)min(max(id, 0), last_id) * p.Hkv + kvh) * (kTile * 2); };
        const char *const k_cache = reinterpret_cast<const char *>(p.k_cache), *const v_cache = reinterpret_cast<const char *>(p.v_cache);
        Wave x;
        __syncthreads();   // (LDS: the last unit's results have been read)
        if (waves == 1) {
            // 32 tokens, two blocks, at a time: those of the run from 32 * wave on, every 32 * NW.  Loads behind the wave's last tokens fetch
            // those again, so that every turn has the same number of loads on their way.
            const int t_end = min(4 * s1, (s.len + 31) / 32);
            int t = 4 * s0 + wave;
            x.begin(p, q_row, kvh * g + c_head, h);
            if (t < t_end) {
                const int t_last = t + (t_end - 1 - t) / NW * NW;
                int ida = id_at(2 * t), idb = id_at(2 * t + 1);
                u32x4 kr[KS], vr[2][MB];
                int64_t at0, at1;
                auto load_k = [&]() {
                    at0 = bytes_at(ida);
                    at1 = bytes_at(idb);
                    const u32x4 *const kp = reinterpret_cast<const u32x4 *>(k_cache + (ku ? at1 : at0));
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) kr[ks] = __builtin_nontemporal_load(&kp[(2 * ks + h) * kBlockSize + kslot]);
                };
                auto load_v = [&]() {
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const u32x4 *const vp = reinterpret_cast<const u32x4 *>(v_cache + (b ? at1 : at0));
#pragma unroll
                        for (int mb = 0; mb < MB; ++mb) vr[b][mb] = __builtin_nontemporal_load(&vp[2 * (32 * mb + col) + h]);
                    }
                };
                auto next_ids = [&](int next) {
                    ida = id_at(2 * min(next, t_last));
                    idb = id_at(2 * min(next, t_last) + 1);
                };
                load_k();
                __builtin_amdgcn_sched_barrier(kNoVmem);   // (the scores wait for K alone)
                load_v();
                next_ids(t + NW);
                for (; t < t_end; t += NW) {
                    const int tok0 = 32 * t, left = s.len - tok0;
                    f32x16 S;
#pragma unroll
                    for (int r = 0; r < 16; ++r) S[r] = 0.f;
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks)
                        S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kr[ks]), __builtin_bit_cast(bf16x8, x.qb[ks]), S, 0, 0, 0);
                    load_k();
                    x.template hide<false>(S, p.words, tok0, s.ctx, s.len, h);
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
                    u32x4 P[2];
                    x.add(S, P);
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int mb = 0; mb < MB; ++mb)
                            x.O[mb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vr[b][mb]), __builtin_bit_cast(bf16x8, P[b]),
                                                                              x.O[mb], 0, 0, 0);
                    load_v();
                    next_ids(t + 2 * NW);
                }
            }
        } else {
            // Stages of 64 tokens, f0 .. f1 - 1 (the sequence's last step may have one); a wave brings a block of a stage, or half of one.
            const int f0 = 2 * s0, f1 = min(2 * s1, (s.len + kStageTokens - 1) / kStageTokens);
            const bool once = s.tiles == 1;
            auto stage_id = [&](int f) -> int { return id_at(kStageBlocks * f + wave / SHARE); };
            const uint32_t to = (uint32_t)(wave / SHARE * CH + share) * 16u;
            auto stage_k = [&](int f, int id) { tile_to_lds(k_cache + bytes_at(id), ldsK_at + (uint32_t)((f & 1) * STAGE) * 16u + to, k_off, once); };
            auto stage_v = [&](int f, int id) {
                tile_to_lds(v_cache + bytes_at(id) - kBias, ldsV_at + (uint32_t)((f & 1) * STAGE) * 16u + to, v_off, once);
            };
            // Everybody's loads have landed, and everybody is done with what came before; V of stage f is used next.
            auto arrive = [&](int f) {
                asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
                __syncthreads();
                if (kStageTokens * (f + 1) > s.len) {   // (slots past the end may hold anything, and 0 * NaN is NaN)
                    u32x4 *const V = ldsV + (f & 1) * STAGE;
                    for (int i = tid; i < STAGE; i += NT) {
                        const int first = kStageTokens * f + 16 * (i / CH) + 8 * (i % CH / HD);
                        u32x4 keep;
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            keep[k] = (first + 2 * k < s.len ? 0x0000FFFFu : 0u) | (first + 2 * k + 1 < s.len ? 0xFFFF0000u : 0u);
                        V[i] &= keep;
                    }
                    __syncthreads();
                }
            };
            // operand i of the product of 32 tokens (half a stage) with K and of their weights with V
            auto k_operand = [&](int f, int half, int i) -> u32x4 { return ldsK[(f & 1) * STAGE + (2 * half + ku) * CH + (2 * i + h) * kBlockSize + kslot]; };
            auto v_operand = [&](int f, int half, int i) -> u32x4 { return ldsV[(f & 1) * STAGE + (2 * half + i / MB) * CH + h * HD + 32 * (i % MB) + col]; };
            const bool used = 32 * cw < rows * g && kw < 2;   // (waves without columns, or without tokens, only bring blocks)
            int id0 = stage_id(f0), id1 = stage_id(f0 + 1);
            stage_k(f0, id0);
            stage_v(f0, id0);
            if (waves < NW) {
                x.begin(p, q_row, kvh * g + c_head, h);
                x.keep_mask(masks[wave][col], p.words, h);
                for (int f = f0; f < f1; ++f) {   // half a stage for each of two waves that have the same columns
                    arrive(f);
                    if (f + 1 < f1) {
                        stage_k(f + 1, id1);
                        stage_v(f + 1, id1);
                        id1 = stage_id(f + 2);
                    }
                    if (!used) continue;
                    f32x16 S;
#pragma unroll
                    for (int r = 0; r < 16; ++r) S[r] = 0.f;
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks)
                        S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k_operand(f, kw, ks)), __builtin_bit_cast(bf16x8, x.qb[ks]), S, 0, 0, 0);
                    x.template hide<true>(S, p.words, kStageTokens * f + 32 * kw, s.ctx, s.len, h);
                    u32x4 P[2];
                    x.add(S, P);
#pragma unroll
                    for (int i = 0; i < KS; ++i)
                        x.O[i % MB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v_operand(f, kw, i)), __builtin_bit_cast(bf16x8, P[i / MB]),
                                                                              x.O[i % MB], 0, 0, 0);
                }
            } else {
                // Both halves of every stage, in a pipeline: a region multiplies the weights of one half by V and computes the scores
                // of the half after next while the vector ALU turns the scores of the half between them into weights.  K runs a stage ahead of V.
                if (f0 + 1 < f1) stage_k(f0 + 1, id1);
                x.begin(p, q_row, kvh * g + c_head, h);
                x.keep_mask(masks[wave][col], p.words, h);
                int id2 = stage_id(f0 + 2);
                constexpr int AHEAD = 2;   // products ahead of which an operand is asked for
                u32x4 ring[AHEAD];
                auto operand = [&](auto pv, auto qk, int i, int fv, int hv, int fk, int hk) -> u32x4 {
                    constexpr bool PV = decltype(pv)::value, QK = decltype(qk)::value;
                    const int j = PV && QK ? i / 2 : i;
                    return QK && (!PV || (i & 1) == 0) ? k_operand(fk, hk, j) : v_operand(fv, hv, j);
                };
                // PV: weights Pu by V, half hv of stage fv; NEXT: scores Ss to weights Pn; QK: scores Sq of half hk of stage fk.  Returns this lane's
                // sum of Pn.
                auto region = [&](auto pv, auto next, auto qk, const u32x4 (&Pu)[2], int fv, int hv, const f32x16 &Ss, u32x4 (&Pn)[2], f32x16 &Sq,
                                  int fk, int hk) -> float {
                    constexpr bool PV = decltype(pv)::value, NEXT = decltype(next)::value, QK = decltype(qk)::value;
                    constexpr int NM = (PV ? KS : 0) + (QK ? KS : 0);
                    float e[16], sum = 0.f;
                    auto vector_work = [&](int r) {   // of score r, one stage later per two scores
                        if (r < 16) e[r] = __builtin_fmaf(Ss[r], x.scale, -x.m);
                        const int a = r - 2;
                        if (a >= 0 && a < 16) e[a] = fast_exp2(e[a]);
                        const int y = r - 4;
                        if (y >= 0 && y < 16 && (y & 1)) {
                            Pn[y / 8][(y % 8) / 2] = pack2_bf16(e[y - 1], e[y]);
                            sum += e[y - 1] + e[y];
                        }
                    };
                    constexpr int CALLS = 20, OVER = NM - 2;   // calls of vector_work for 16 scores, products that they are spread over
#pragma unroll
                    for (int i = 0; i < AHEAD; ++i) ring[i] = operand(pv, qk, i, fv, hv, fk, hk);
#pragma unroll
                    for (int i = 0; i < NM; ++i) {
                        const int j = PV && QK ? i / 2 : i;
                        const bf16x8 op = __builtin_bit_cast(bf16x8, ring[i % AHEAD]);
                        if (QK && (!PV || (i & 1) == 0)) {
                            f32x16 z;
#pragma unroll
                            for (int r = 0; r < 16; ++r) z[r] = 0.f;
                            Sq = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op, __builtin_bit_cast(bf16x8, x.qb[j]), j == 0 ? z : Sq, 0, 0, 0);
                        } else {
                            x.O[j % MB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op, __builtin_bit_cast(bf16x8, Pu[j / MB]), x.O[j % MB], 0, 0, 0);
                        }
                        if (i + AHEAD < NM) ring[i % AHEAD] = operand(pv, qk, i + AHEAD, fv, hv, fk, hk);
                        if constexpr (NEXT) {
#pragma unroll
                            for (int r = i * CALLS / OVER; r < (i + 1) * CALLS / OVER; ++r)
                                if (r < CALLS) vector_work(r);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                    return sum;
                };
                const auto yes = std::true_type();
                const auto no = std::false_type();
                // The weights of a half were computed against a reference that was too low for some column (their sum is more than 2^8, infinite
                // or NaN): once more, against the half's maximum.
                auto settle = [&](const f32x16 &S, u32x4 (&P)[2], float sum) {
                    if (!__all(sum <= 256.0f)) {
                        x.move(x.top(S));
                        sum = x.weights(S, P);
                    }
                    x.lsum += sum;
                };
                auto hide = [&](f32x16 &S, int f, int half) { x.template hide<true>(S, p.words, kStageTokens * f + 32 * half, s.ctx, s.len, h); };
                f32x16 S0 = {}, S1 = {};
                u32x4 P0[2] = {}, P1[2] = {};
                arrive(f0);
                if (used) {
                    region(no, no, yes, P0, 0, 0, S0, P0, S0, f0, 0);
                    hide(S0, f0, 0);
                    x.m = fmaxf(x.m, x.top(S0));
                    settle(S0, P0, region(no, yes, yes, P0, 0, 0, S0, P0, S1, f0, 1));
                }
                for (int f = f0; f < f1 - 1; ++f) {
                    if (f > f0) arrive(f);
                    else __syncthreads();   // (K of stage f0 has been used)
                    if (f + 2 < f1) stage_k(f + 2, id2);
                    stage_v(f + 1, id1);
                    id1 = id2;
                    id2 = stage_id(f + 3);
                    if (!used) continue;
                    hide(S1, f, 1);
                    settle(S1, P1, region(yes, yes, yes, P0, f, 0, S1, P1, S0, f + 1, 0));
                    hide(S0, f + 1, 0);
                    settle(S0, P0, region(yes, yes, yes, P1, f, 1, S0, P0, S1, f + 1, 1));
                }
                if (f1 - 1 > f0) arrive(f1 - 1);
                if (used) {
                    hide(S1, f1 - 1, 1);
                    settle(S1, P1, region(yes, yes, no, P0, f1 - 1, 0, S1, P1, S0, 0, 0));
                    region(yes, no, no, P1, f1 - 1, 1, S0, P0, S0, 0, 0);
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
        const bool whole = s0 == 0 && s1 == s.steps;
        const int64_t slot = 2 * (int64_t)w + (s0 == 0 ? 1 : 0);   // (a run has one unit that begins before it, and one that ends behind it)
        for (int i = 0; i < waves; ++i) {
            const int oc = 32 * i + tid / (NT / 32);
            if (oc >= rows * g) break;
            tree_column<HD, NT, ROW>(p, &slab[0][0], &stat[0][0], 32 * i + (oc & 31), 32 * waves, NW / waves, whole, slot * COLS + oc, s.q0 + row0, oc, kvh);
        }
        if (s0 > 0) {   // (at most once, at the beginning of the run)
            // where all parts of the unit are: the first in the run that the unit begins in, the others at the beginnings of theirs
            first_run = runs.holding(pos - s0);
            parts = runs.holding(pos - s0 + s.steps - 1) - first_run + 1;
            if (tid == 0) {
                merge[2] = s.q0 + row0;
                merge[3] = rows;
                merge[4] = kvh;
            }
        }
        pos += s1 - s0;
    }
    if (tid == 0) {
        merge[0] = parts;
        merge[1] = first_run;
    }
}

// Tiles of up to 64 columns: every wave has all columns and a quarter of the tokens, whose K and V it loads from the cache to the registers of
// the matrix instructions.  Two blocks of 32 columns use what is there once; the waves have the registers of a whole SIMD for that, and a
// turn's loads ahead of the products, 64 KiB of a workgroup, keep the memory busy with one workgroup to a compute unit.
template <int HD>
__global__ __launch_bounds__(256, 1) void tree_stream_kernel(const TreeArgs p)
{
    constexpr int NW = 4, NT = 64 * NW, COLS = 64;
    using Wave = TreeWave<HD>;
    constexpr int KS = Wave::KS, MB = Wave::MB;
    constexpr int ROW = HD + 4;
    __shared__ __align__(16) float slab[NW * COLS][ROW];   // [wave, column][dim]
    __shared__ __align__(8) float stat[NW * COLS][2];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, h = lane >> 5;
    const int g = p.g;
    int w, seq = 0;
    int64_t start = 0;
    TreeSeq s = {};
    const TreeRuns runs = tree_run<NT>(p, w, seq, start, s);
    const int64_t lo = runs.first(w), hi = runs.first(w + 1);
    int32_t *const merge = p.merges + (int64_t)w * kMergeInts;
    if (lo >= hi) {
        if (tid == 0) merge[0] = 0;
        return;
    }
    const int ku = col >> 4, kslot = (col & 3) | ((col & 4) << 1) | ((col & 8) >> 1);   // (see tree_kernel)
    const char *const k_cache = reinterpret_cast<const char *>(p.k_cache), *const v_cache = reinterpret_cast<const char *>(p.v_cache);
    int first_run = 0, parts = 0;
    for (int64_t pos = lo; pos < hi;) {
        while (pos - start >= s.units) {
            start += s.units;
            ++seq;
            s = tree_seq_at(p, seq, s.length - s.steps);
        }
        const int unit = (int)quotient(pos - start, s.length);
        const int s0 = (int)(pos - start - (int64_t)unit * s.length);
        if (s0 >= s.steps) {
            pos += s.length - s0;
            continue;
        }
        const int s1 = (int)min((int64_t)s.steps, s0 + (hi - pos));
        const int kvh = s.tiles == 1 ? unit : unit / s.tiles, tile = unit - kvh * s.tiles;
        const int row0 = tile * s.tile_rows, rows = min(s.tile_rows, s.n - row0);
        const int nblk = (s.len + kBlockSize - 1) / kBlockSize;
        const const_i32_ptr table = scalar_ptr(p.block_tables + (int64_t)seq * p.max_blocks_per_seq);
        const int last_id = (int)min(p.num_blocks, (int64_t)INT32_MAX) - 1;
        auto id_at = [&](int block) -> int { return table[min(block, nblk - 1)]; };   // blocks past the end: the last one
        auto bytes_at = [&](int id) -> int64_t { return ((int64_t)min(max(id, 0), last_id) * p.Hkv + kvh) * (HD * 32); };
        // 32 tokens, two blocks, at a time: those of the run from 32 * wave on, every 32 * NW.  Loads behind the wave's last tokens fetch
        // those again, so that every turn has the same number of loads on their way.
        const int t_end = min(4 * s1, (s.len + 31) / 32), t0 = 4 * s0 + wave;
        auto walk = [&](auto blocks) {
            constexpr int CB = decltype(blocks)::value;   // blocks of 32 columns
            Wave x[CB];
#pragma unroll
            for (int c = 0; c < CB; ++c) {   // (columns behind the last row repeat it)
                const int at = 32 * c + col, row = min(at / g, rows - 1);
                x[c].begin(p, (int64_t)s.q0 + row0 + row, kvh * g + at % g, h);
            }
            if (t0 < t_end) {
                const int t_last = t0 + (t_end - 1 - t0) / NW * NW;
                int ida = id_at(2 * t0), idb = id_at(2 * t0 + 1);
                u32x4 kr[KS], vr[2][MB];
                int64_t at0, at1;
                auto load_k = [&]() {
                    at0 = bytes_at(ida);
                    at1 = bytes_at(idb);
                    const u32x4 *const kp = reinterpret_cast<const u32x4 *>(k_cache + (ku ? at1 : at0));
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) kr[ks] = __builtin_nontemporal_load(&kp[(2 * ks + h) * kBlockSize + kslot]);
                };
                auto load_v = [&]() {
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const u32x4 *const vp = reinterpret_cast<const u32x4 *>(v_cache + (b ? at1 : at0));
#pragma unroll
                        for (int mb = 0; mb < MB; ++mb) vr[b][mb] = __builtin_nontemporal_load(&vp[2 * (32 * mb + col) + h]);
                    }
                };
                auto next_ids = [&](int next) {
                    ida = id_at(2 * min(next, t_last));
                    idb = id_at(2 * min(next, t_last) + 1);
                };
                load_k();
                __builtin_amdgcn_sched_barrier(kNoVmem);   // (the scores wait for K alone)
                load_v();
                next_ids(t0 + NW);
                for (int t = t0; t < t_end; t += NW) {
                    const int tok0 = 32 * t, left = s.len - tok0;
                    f32x16 S[CB];
#pragma unroll
                    for (int c = 0; c < CB; ++c)
#pragma unroll
                        for (int r = 0; r < 16; ++r) S[c][r] = 0.f;
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                        for (int c = 0; c < CB; ++c)
                            S[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kr[ks]), __builtin_bit_cast(bf16x8, x[c].qb[ks]), S[c], 0, 0, 0);
                    load_k();
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
                    u32x4 P[CB][2];
#pragma unroll
                    for (int c = 0; c < CB; ++c) {
                        x[c].template hide<false>(S[c], p.words, tok0, s.ctx, s.len, h);
                        x[c].add(S[c], P[c]);
                    }
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                            for (int c = 0; c < CB; ++c)
                                x[c].O[mb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vr[b][mb]), __builtin_bit_cast(bf16x8, P[c][b]),
                                                                                    x[c].O[mb], 0, 0, 0);
                    load_v();
                    next_ids(t + 2 * NW);
                }
            }
            __syncthreads();   // (LDS: the last unit's results have been read)
#pragma unroll
            for (int c = 0; c < CB; ++c) {
                float l0, l1;
                swap32(x[c].lsum, l0, l1);
                const int at = wave * COLS + 32 * c + col;
                if (h == 0) {
                    stat[at][0] = x[c].m;
                    stat[at][1] = l0 + l1;
                }
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        *reinterpret_cast<f32x4 *>(&slab[at][32 * mb + 8 * k + 4 * h]) =
                            f32x4{x[c].O[mb][4 * k], x[c].O[mb][4 * k + 1], x[c].O[mb][4 * k + 2], x[c].O[mb][4 * k + 3]};
            }
        };
        if (rows * g <= 32)
            walk(std::integral_constant<int, 1>());
        else
            walk(std::integral_constant<int, 2>());
        __syncthreads();
        const bool whole = s0 == 0 && s1 == s.steps;
        const int64_t slot = 2 * (int64_t)w + (s0 == 0 ? 1 : 0);
        for (int oc = tid / (NT / 32); oc < rows * g; oc += 32)
            tree_column<HD, NT, ROW>(p, slab, stat, oc, COLS, NW, whole, slot * COLS + oc, s.q0 + row0, oc, kvh);
        if (s0 > 0) {   // (at most once, at the beginning of the run)
            // where all parts of the unit are: the first in the run that the unit begins in, the others at the beginnings of theirs
            first_run = runs.holding(pos - s0);
            parts = runs.holding(pos - s0 + s.steps - 1) - first_run + 1;
            if (tid == 0) {
                merge[2] = s.q0 + row0;
                merge[3] = rows;
                merge[4] = kvh;
            }
        }
        pos += s1 - s0;
    }
    if (tid == 0) {
        merge[0] = parts;
        merge[1] = first_run;
    }
}

// Slices of a run's share of the merge: 16 columns of the widest tile each, at most eight.  (Most workgroups find nothing to do, and take their
// time: 8 nodes of eight sequences on 2000 tokens, us, eight slices / four 22.9 / 22.0, of one on 300 12.4 / 12.0.)
constexpr int merge_slices(int waves) { return waves < 4 ? 2 * waves : 8; }

// The parts of the units that runs have cut.  Every run that continues a unit takes a share of its columns, so that a unit of many
// parts, which has many runs, is merged by many workgroups; merge_slices of them have the run's share.  In a workgroup HD / 4 threads
// have a column's dims, and groups of threads have every PG-th part of it; their results meet in LDS in a fixed order.
template <int HD, int NW>
__global__ __launch_bounds__(kMergeThreads) void tree_merge_kernel(const TreeArgs p)
{
    constexpr int TC = HD / 4, SLOTS = kMergeThreads / TC;   // threads of a column, columns or groups at a time
    constexpr int AHEAD = 4;                                 // parts whose loads are sent off together
    __shared__ f32x4 sh_acc[kMergeThreads];
    __shared__ f32x2 sh_ml[kMergeThreads];
    const int w = blockIdx.x;
    const int32_t *const merge = p.merges + (int64_t)w * kMergeInts;
    const int parts = merge[0], first = merge[1], row0 = merge[2], rows = merge[3], kvh = merge[4];
    if (parts == 0) return;
    const int cols = rows * p.g, shares = (parts - 1) * merge_slices(NW), share = (w - first - 1) * merge_slices(NW) + blockIdx.y;
    const int c0 = cols * share / shares, c1 = cols * (share + 1) / shares;
    const int groups = parts <= AHEAD ? 1 : parts <= 2 * AHEAD ? 2 : parts <= 4 * AHEAD ? 4 : SLOTS;
    const int slot = threadIdx.x / TC, d = 4 * (threadIdx.x % TC);
    const int group = slot & (groups - 1);
    for (int base = c0; base < c1; base += SLOTS / groups) {
        const int col = base + slot / groups;
        float M = -1e30f, l = 0.f;
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        auto fold = [&](float m2, float l2, const f32x4 &a2) {
            const float M_new = fmaxf(M, m2);
            const float w_old = fast_exp2(M - M_new), w_new = fast_exp2(m2 - M_new);
            M = M_new;
            l = l * w_old + l2 * w_new;
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] = acc[e] * w_old + a2[e] * w_new;
        };
        if (col < c1) {
            for (int k0 = group; k0 < parts; k0 += AHEAD * groups) {
                f32x2 ml[AHEAD];
                f32x4 a[AHEAD];
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) {
                    const int k = k0 + i * groups;
                    if (k < parts) {
                        const int64_t at = (2 * (int64_t)(first + k) + (k == 0 ? 1 : 0)) * (32 * NW) + col;
                        ml[i] = *reinterpret_cast<const f32x2 *>(p.part_ml + 2 * at);
                        a[i] = *reinterpret_cast<const f32x4 *>(p.part_acc + at * HD + d);
                    }
                }
#pragma unroll
                for (int i = 0; i < AHEAD; ++i)
                    if (k0 + i * groups < parts) fold(ml[i][0], ml[i][1], a[i]);
            }
        }
        __syncthreads();   // (the last columns' results have been read)
        sh_acc[threadIdx.x] = acc;
        sh_ml[threadIdx.x] = f32x2{M, l};
        __syncthreads();
        if (group == 0 && col < c1) {
            for (int k = 1; k < groups; ++k) fold(sh_ml[threadIdx.x + k * TC][0], sh_ml[threadIdx.x + k * TC][1], sh_acc[threadIdx.x + k * TC]);
            const float inv = l == 0.f ? 0.f : 1.0f / l;
            const int row = col / p.g, head = col - row * p.g;
            *reinterpret_cast<u32x2 *>(p.out + ((int64_t)(row0 + row) * p.Hq + kvh * p.g + head) * HD + d) =
                u32x2{pack2_bf16(acc[0] * inv, acc[1] * inv), pack2_bf16(acc[2] * inv, acc[3] * inv)};
        }
    }
}

namespace {
size_t run_bytes(int hd, int waves) { return kMergeInts * sizeof(int32_t) + 2 * (size_t)(32 * waves) * (hd + 2) * sizeof(float); }

template <int HD, int NW>
hipError_t launch(TreeArgs &a, void *ws, hipStream_t s)
{
    const unsigned runs = 1u << a.runs_log2;
    a.tile_rows = 32 * NW / a.g;
    // (the bound holds for sequences that overlap as well)
    const int64_t tiles = (int64_t)a.num_seqs * (a.total_q / a.tile_rows + 1), steps = (int64_t)a.max_blocks_per_seq * kBlockSize / kTreeStep + 1 + kUnitSteps;
    a.short_line = a.num_seqs <= 64 && (double)tiles * (double)a.Hkv * (double)steps < 2147483647.0;
    // One workgroup of four waves to a compute unit, and so half the runs, cuts fewer units, but waits with nothing else to do: so it is on a
    // line of less than four steps a run, unless two to a compute unit find whole units.  MI355X, us, all runs / half, 32/8 heads: 32
    // sequences of 32 nodes on 600 tokens (2.5 steps a run) 45.2 / 32.9, 16 of 24 nodes on 1000 .. 4000 (5) 55.4 / 57.9.
    const int64_t per_seq = ((int64_t)a.total_q + a.num_seqs - 1) / a.num_seqs, units = ((per_seq + a.tile_rows - 1) / a.tile_rows) * a.Hkv * a.num_seqs;
    a.halve_below = NW != 4 || runs < 2 || units >= (int64_t)runs ? 0 : (int64_t)4 << a.runs_log2;
    a.part_acc = static_cast<float *>(ws);
    a.part_ml = a.part_acc + (size_t)2 * runs * (32 * NW) * HD;
    a.merges = reinterpret_cast<int32_t *>(a.part_ml + (size_t)2 * runs * (32 * NW) * 2);
    if constexpr (NW == 2)
        hipLaunchKernelGGL((tree_stream_kernel<HD>), dim3(runs), dim3(256), 0, s, a);
    else
        hipLaunchKernelGGL((tree_kernel<HD, NW>), dim3(runs), dim3(64 * NW), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((tree_merge_kernel<HD, NW>), dim3(runs, merge_slices(NW)), dim3(kMergeThreads), 0, s, a);
    return hipGetLastError();
}
}  // namespace

// Two: the kernel for up to 64 columns, where the average sequence has no more and there are less than two units for each compute unit, so
// that two workgroups of the other kernel would have to cut them.  MI355X, us, four waves / this, 32/8 heads: 16 nodes, 32 sequences of 4096 tokens
// 101.6 / 91.3; 8 nodes, 32 of 4096 98.6 / 88.5, 8 of 2000 27.2 / 22.9; 64 of 100 .. 1000 (two units each) 46.9 / 52.3.
// Else workgroups of eight waves fetch K and V once for 256 columns where four waves fetch them twice, at about the same time if the lengths
// are equal and at different times if not; they are fewer, and their waves wait for one another.  So they are for sequences of more
// than 128 columns on average, and for work that fills them: 16 steps each, of what the block tables can hold (the lengths are on the
// device).  MI355X, us, four / eight waves, 64 nodes of 32/8 heads: 4 sequences of 1000 tokens 33 / 37, 4 of 4000 43 / 47, 32 of 4096 168 /
// 163, 64 of 4096 411 / 321; 4 x 20..27 nodes of 28/4 heads on 60..131K 308 / 226.
int tree_waves(int total_q, int num_seqs, int Hkv, int g, int max_blocks_per_seq, int num_cus)
{
    const double steps = (double)num_seqs * Hkv * ((double)max_blocks_per_seq * kBlockSize / kTreeStep);
    const int64_t tile_rows = 64 / g, per_seq = ((int64_t)total_q + num_seqs - 1) / num_seqs;
    if (per_seq * g <= 64 && (per_seq + tile_rows - 1) / tile_rows * num_seqs * Hkv < 2 * num_cus) return 2;
    return (int64_t)total_q * g > 128 * (int64_t)num_seqs && steps >= 16.0 * num_cus ? 8 : 4;
}

int tree_runs_log2(int waves, int hd, int num_cus, size_t ws_bytes)
{
    int log2 = 0;
    while ((2 << log2) <= (waves == 4 ? 2 : 1) * num_cus) ++log2;
    while (log2 >= 0 && (run_bytes(hd, waves) << log2) > ws_bytes) --log2;
    return log2;
}

hipError_t launch_attn_tree(TreeArgs &a, int waves, void *ws, hipStream_t s)
{
    if (waves == 2) return a.hd == 128 ? launch<128, 2>(a, ws, s) : launch<64, 2>(a, ws, s);
    if (a.hd == 128) return waves == 8 ? launch<128, 8>(a, ws, s) : launch<128, 4>(a, ws, s);
    return waves == 8 ? launch<64, 8>(a, ws, s) : launch<64, 4>(a, ws, s);
}

}  // namespace ooco
