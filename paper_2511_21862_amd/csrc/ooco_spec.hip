// HIP kernels of libooco for gfx950 around the attention of a speculative decoding step: masks of a tree of drafted nodes,
// rotary positions with the KV append, verification of the drafted tokens, and the accepted nodes' way to their places.
#include "ooco_device.h"
#include "ooco_internal.h"
#include "ooco_spec.h"

#include <algorithm>
#include <cfloat>
#include <climits>
#include <type_traits>

namespace ooco {

// The rows of sequence seq: the first and their number; none where the arrays contradict each other.
OOCO_DEV void rows_of(const int32_t *query_start_loc, int seq, int total_q, int &q0, int &n)
{
    q0 = query_start_loc[seq];
    n = query_start_loc[seq + 1] - q0;
    if (q0 < 0 || n < 0 || n > total_q - q0) n = 0;
}

// The sequence that owns (sequence, block) pair x, and its rows and cached tokens: sequence i owns the pairs from
// query_start_loc[i] / 16 + 2 i on.  256 sequences a memory round trip, which brings the lengths as well.  The same x in every lane.
OOCO_DEV int rows_of_pair(const int32_t *query_start_loc, const int32_t *ctx_lens, int num_seqs, int total_q, int x, int &q0, int &n, int &ctx)
{
    constexpr int LOOKS = 4;
    const int lane = threadIdx.x & 63;
    for (int base = 0;; base += 64 * LOOKS) {
        int start[LOOKS], next[LOOKS], cached[LOOKS];
#pragma unroll
        for (int k = 0; k < LOOKS; ++k) {
            const int i = min(base + 64 * k + lane, num_seqs - 1);
            start[k] = query_start_loc[i];
            next[k] = query_start_loc[i + 1];
            cached[k] = ctx_lens[i];
        }
#pragma unroll
        for (int k = 0; k < LOOKS; ++k) {
            const int i = base + 64 * k + lane;
            const int before = __popcll(__ballot(i < num_seqs && next[k] / kBlockSize + 2 * (i + 1) <= x));   // sequences that end in front of x
            if (before < 64 || base + 64 * k + 64 >= num_seqs) {
                const int at = min(before, num_seqs - 1 - (base + 64 * k));
                q0 = __builtin_amdgcn_readlane(start[k], at);
                n = __builtin_amdgcn_readlane(next[k], at) - q0;
                ctx = __builtin_amdgcn_readlane(cached[k], at);
                if (q0 < 0 || n < 0 || n > total_q - q0) n = 0;
                return base + 64 * k + at;
            }
        }
    }
}

// ------------------------------------------------------------------------------------------
// Masks and positions.  A node sees itself and its ancestors: with M_0(i) = {i} and P_0(i) = parent(i), doubling the distance
// M_k+1(i) = M_k(i) + M_k(P_k(i)), P_k+1(i) = P_k(P_k(i)) needs log2 of the depth rounds, where a walk up the tree would need the
// depth; the number of the nodes in M is the depth + 1.  One workgroup per sequence, a thread per node, the sets as bits in LDS.
// A parent has to be an earlier node: anything else is taken as none, so the walk ends whatever the array holds.  What there is to move is
// nothing; the launch and a chain of loads bound it (MI355X, 256 sequences of 20 .. 64 nodes: 3.2 us, one of 8 nodes 2.6).
template <int W>
__global__ __launch_bounds__(64 * W) void tree_masks_kernel(const int32_t *parents, const int32_t *query_start_loc, const int32_t *ctx_lens,
                                                            uint64_t *masks, int32_t *positions, int total_q)
{
    constexpr int N = 64 * W;
    __shared__ uint64_t sets[W][N];
    __shared__ int up[N];
    const int seq = blockIdx.x, t = threadIdx.x;
    int q0, n;
    rows_of(query_start_loc, seq, total_q, q0, n);
    const int ctx = ctx_lens[seq];
    const int nodes = min(n, N);
    int p = -1;
    if (t < nodes) {
        p = parents[q0 + t];
        if (p >= t) p = -1;
    }
    p = max(p, -1);
    uint64_t m[W];
#pragma unroll
    for (int w = 0; w < W; ++w) m[w] = t / 64 == w ? 1ull << (t & 63) : 0;
    while (__syncthreads_or(p >= 0)) {
#pragma unroll
        for (int w = 0; w < W; ++w) sets[w][t] = m[w];
        up[t] = p;
        __syncthreads();
        if (p >= 0) {
#pragma unroll
            for (int w = 0; w < W; ++w) m[w] |= sets[w][p];
            p = up[p];
        }
    }
    int depth = -1;
#pragma unroll
    for (int w = 0; w < W; ++w) depth += __popcll(m[w]);
    if (t < nodes) {
        uint64_t *const dst = masks + (int64_t)(q0 + t) * W;
#pragma unroll
        for (int w = 0; w < W; ++w) dst[w] = m[w];
        if (positions) positions[q0 + t] = ctx + depth;
    }
    for (int i = N + t; i < n; i += N) {   // nodes that the masks have no bits for see the cache alone
#pragma unroll
        for (int w = 0; w < W; ++w) masks[(int64_t)(q0 + i) * W + w] = 0;
        if (positions) positions[q0 + i] = ctx;
    }
}

hipError_t launch_tree_masks(const int32_t *parents, const int32_t *query_start_loc, const int32_t *ctx_lens, uint64_t *masks,
                             int32_t *positions, int words, int num_seqs, int total_q, hipStream_t s)
{
    auto *const kernel = words == 1 ? tree_masks_kernel<1> : words == 2 ? tree_masks_kernel<2> : words == 3 ? tree_masks_kernel<3> : tree_masks_kernel<4>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)num_seqs), dim3(64u * (unsigned)words), 0, s, parents, query_start_loc, ctx_lens, masks, positions, total_q);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------------
// Rotary positions and append: x'_a = x_a cos(p f) - x_b sin(p f), x'_b = x_b cos(p f) + x_a sin(p f) for the pairs (a, b) of a
// head, in fp32, rounded once to bf16; v goes to the cache as it is.  Memory bound: every element is read once and written once.
// A workgroup has two or four heads of the rows of one (sequence, KV block) pair, as the plain append does (see kv_append_kernel for the
// order of the pairs: sequence i owns the pairs from query_start_loc[i] / 16 + 2 i on), because the cache keeps 16 tokens of a dim or of a
// group of 8 dims side by side.  All heads are read the way they lie, a 16-byte piece of a row per thread, all pieces of a thread on their
// way before anything is computed; q is written the way it was read, k and v go through LDS and are written the way the cache has them.
// (MI355X, 8 x 512 rows, 32/8 heads, us: 30 with loads of k and stores of v that jump from row to row, 26 like this, 21 with stores past the
// caches: 4.9 TB/s, of the 5.2 that a large copy reaches.)
// The angles' turns p f / (2 pi) are reduced in 64 bits -- a position of 10^5 times a frequency of 1 leaves 32 bits three digits behind the
// point -- and cosine and sine are those of the hardware, which take turns (off by 2^-22.9 at most, measured over 2^22 turns); they are
// computed once per row and pair for all heads of the workgroup.
constexpr int kRopeThreads = 256;

OOCO_DEV float bf16_lo(uint32_t u) { return __builtin_bit_cast(float, u << 16); }
OOCO_DEV float bf16_hi(uint32_t u) { return __builtin_bit_cast(float, u & 0xFFFF0000u); }

template <int HD, bool INTERLEAVED, int HEADS>
__global__ __launch_bounds__(kRopeThreads) void rope_append_kernel(const RopeArgs a)
{
    constexpr int CH = HD / 8;                                    // pieces of a head
    constexpr int PITCH = HD + 8;                                 // elements of a row in LDS (padded: the lanes of a wave are rows)
    constexpr int N = kBlockSize * HEADS * CH / kRopeThreads;   // pieces of a thread
    __shared__ f32x2 turn[kBlockSize][kMaxRotaryPairs];           // (cosine, sine)
    __shared__ __align__(16) uint16_t tile[HEADS][kBlockSize][PITCH];   // by slot of the block
    const int tid = threadIdx.x;
    const int pair = blockIdx.x / a.parts, part = blockIdx.x - pair * a.parts;
    int q0, q_len, ctx;
    const int seq = rows_of_pair(a.query_start_loc, a.ctx_lens, a.num_seqs, a.total_q, pair, q0, q_len, ctx);
    if (q_len == 0 || ctx < 0) return;
    const int64_t end = (int64_t)ctx + q_len;                     // (may lie past the block table)
    const int64_t bidx = ctx / kBlockSize + (int64_t)(pair - (q0 / kBlockSize + 2 * seq));
    if (bidx < ctx / kBlockSize || bidx * kBlockSize >= end) return;   // beyond the sequence's last touched block
    const int t_lo = (int)max((int64_t)0, bidx * kBlockSize - ctx);
    const int slot0 = (int)(ctx + (int64_t)t_lo - bidx * kBlockSize);
    const int nrow = min(kBlockSize - slot0, q_len - t_lo);
    const int row0 = q0 + t_lo;

    // Heads of this part: of q, of k and of v, numbered one after the other.
    const int heads = a.Hq + 2 * a.Hkv, h0 = part * HEADS;
    const int pairs = a.pairs;
    // Piece i of the thread is piece `c` of head h0 + hs, row r.
    const int c = tid % CH, hs = tid / CH % HEADS, r_first = tid / (CH * HEADS);
    constexpr int R_STEP = kRopeThreads / (CH * HEADS);
    const int head = h0 + hs;
    const bool is_q = head < a.Hq, is_k = !is_q && head < a.Hq + a.Hkv, there = head < heads;
    const uint16_t *const src = is_q ? a.q + head * HD : is_k ? a.k_new + (head - a.Hq) * HD : a.v_new + (head - a.Hq - a.Hkv) * HD;
    const int64_t apart = is_q ? a.q_stride : is_k ? a.k_stride : a.v_stride;
    // the piece that this one turns with, and the sine's sign
    const bool rotated = (is_q || is_k) && c < pairs / 4;
    const bool second = !INTERLEAVED && c >= pairs / 8;
    const int partner = second ? c - pairs / 8 : c + pairs / 8;
    u32x4 x[N], y[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int r = r_first + i * R_STEP;
        if (there && r < nrow) {
            const u32x4 *const p = reinterpret_cast<const u32x4 *>(src + (row0 + r) * apart);
            x[i] = p[c];
            if (!INTERLEAVED && rotated) y[i] = p[partner];
        }
    }
    // (a block that the cache does not have: the queries are rotated all the same, nothing is appended)
    const int64_t blk = bidx < a.max_blocks_per_seq ? a.block_tables[(int64_t)seq * a.max_blocks_per_seq + bidx] : -1;
    const bool blk_ok = blk >= 0 && blk < a.num_blocks;

    for (int i = tid; i < nrow * pairs; i += kRopeThreads) {
        const int r = i / pairs, k = i - r * pairs;
        const int pos = a.positions ? a.positions[row0 + r] : ctx + t_lo + r;
        const float f = (float)__builtin_amdgcn_fract((double)pos * a.turns[k]);
        turn[r][k] = f32x2{__builtin_amdgcn_cosf(f) * a.factor, __builtin_amdgcn_sinf(f) * a.factor};
    }
    __syncthreads();
    auto store = [&](u32x4 *dst, const u32x4 &v) {
        if (a.past_caches)
            __builtin_nontemporal_store(v, dst);
        else
            *dst = v;
    };
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int r = r_first + i * R_STEP;
        if (!there || r >= nrow) continue;
        if (rotated) {
            if constexpr (INTERLEAVED) {
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const f32x2 t = turn[r][4 * c + w];
                    const float x0 = bf16_lo(x[i][w]), x1 = bf16_hi(x[i][w]);
                    x[i][w] = pack2_bf16(x0 * t[0] - x1 * t[1], x1 * t[0] + x0 * t[1]);
                }
            } else {
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const f32x2 t0 = turn[r][8 * (second ? partner : c) + 2 * w], t1 = turn[r][8 * (second ? partner : c) + 2 * w + 1];
                    const float s0 = second ? t0[1] : -t0[1], s1 = second ? t1[1] : -t1[1];
                    x[i][w] = pack2_bf16(bf16_lo(x[i][w]) * t0[0] + bf16_lo(y[i][w]) * s0, bf16_hi(x[i][w]) * t1[0] + bf16_hi(y[i][w]) * s1);
                }
            }
        }
        if (is_q)
            store(reinterpret_cast<u32x4 *>(a.q_out + ((int64_t)(row0 + r) * a.Hq + head) * HD + 8 * c), x[i]);
        else
            *reinterpret_cast<u32x4 *>(&tile[hs][slot0 + r][8 * c]) = x[i];
    }
    if (h0 + HEADS <= a.Hq || !blk_ok) return;   // (the whole workgroup: only heads of q, or nowhere to append)
    __syncthreads();
    const int k0 = max(h0, a.Hq), k1 = min(h0 + HEADS, a.Hq + a.Hkv), v0 = max(h0, a.Hq + a.Hkv), v1 = min(h0 + HEADS, heads);
    // K: pieces of 16 bytes, the block's slots side by side
    for (int i = tid; i < (k1 - k0) * CH * kBlockSize; i += kRopeThreads) {
        const int slot = i % kBlockSize, p = i / kBlockSize % CH, h = k0 + i / (kBlockSize * CH);
        if (slot >= slot0 && slot < slot0 + nrow)
            store(reinterpret_cast<u32x4 *>(a.k_cache) + ((blk * a.Hkv + (h - a.Hq)) * CH + p) * kBlockSize + slot,
                  *reinterpret_cast<const u32x4 *>(&tile[h - h0][slot][8 * p]));
    }
    // V: half a row of a dim, eight slots, per thread
    for (int i = tid; i < (v1 - v0) * HD * 2; i += kRopeThreads) {
        const int half = i & 1, d = i / 2 % HD, h = v0 + i / (2 * HD);
        uint32_t e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = tile[h - h0][8 * half + j][d];
        uint16_t *const dst = a.v_cache + ((blk * a.Hkv + (h - a.Hq - a.Hkv)) * HD + d) * kBlockSize + 8 * half;
        const int lo = slot0 - 8 * half, hi = slot0 + nrow - 8 * half;   // slots lo .. hi - 1 of the half are the step's
        if (lo <= 0 && hi >= 8) {
            store(reinterpret_cast<u32x4 *>(dst), u32x4{e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16});
            continue;
        }
        // quarters that the step covers whole with one store each, the ragged ends slot by slot
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (lo <= 4 * k && hi >= 4 * k + 4) {
                *reinterpret_cast<u32x2 *>(dst + 4 * k) = u32x2{e[4 * k] | e[4 * k + 1] << 16, e[4 * k + 2] | e[4 * k + 3] << 16};
            } else {
#pragma unroll
                for (int j = 4 * k; j < 4 * k + 4; ++j)
                    if (j >= lo && j < hi) dst[j] = (uint16_t)e[j];
            }
        }
    }
}

namespace {
template <int HEADS>
hipError_t launch_rope(RopeArgs &a, bool interleaved, int64_t pairs, hipStream_t s)
{
    a.parts = (a.Hq + 2 * a.Hkv + HEADS - 1) / HEADS;
    auto *const kernel = a.hd == 128 ? (interleaved ? rope_append_kernel<128, true, HEADS> : rope_append_kernel<128, false, HEADS>)
                                     : (interleaved ? rope_append_kernel<64, true, HEADS> : rope_append_kernel<64, false, HEADS>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(pairs * a.parts)), dim3(kRopeThreads), 0, s, a);
    return hipGetLastError();
}
}  // namespace

hipError_t launch_rope_append(RopeArgs &a, bool interleaved, int num_cus, hipStream_t s)
{
    const int64_t pairs = a.total_q / kBlockSize + 2 * (int64_t)a.num_seqs + 1;
    // Stores by the plain append's rule.  Alone, stores past the caches are faster (us, 8 x 512 rows 26.4 -> 20.7, 64 x 16 10.7 -> 10.1, 1 x 1000 8.8
    // -> 7.8), but with the attention that reads what they wrote the two together are level above the rule's bounds (108.1 / 108.7, 66.3 /
    // 63.8) and slower below them (1 x 300 16.0 / 16.6).
    a.past_caches = append_past_caches(a.total_q, a.num_seqs, 4 * (int64_t)a.total_q * a.Hkv * a.hd);
    // Four heads to a workgroup, or two where that leaves compute units without one (us, 8 x 12 rows 4.9 -> 4.4; 8 x 512 26 -> 31).
    const int64_t by_four = pairs * ((a.Hq + 2 * a.Hkv + 3) / 4);
    return by_four <= 2 * (int64_t)num_cus ? launch_rope<2>(a, interleaved, pairs, s) : launch_rope<4>(a, interleaved, pairs, s);
}

// ------------------------------------------------------------------------------------------
// Verification.  Child c of node v has been drafted from q_c and is looked at after its earlier siblings have been refused: it is
// accepted if u_c q_c(x_c) (1 - sum of the refused siblings' p_v) < p_v(x_c), with q = 1 for tokens that were picked and not drawn
// (draft == NULL).  The first accepted child of each node is all that the walk from the root needs, and whether a child is
// accepted does not depend on the walk: one thread per node tests its own, after one round of gathered loads.  The token behind
// the last accepted node v comes from what refusing leaves: max(p_v - q_c, 0), or p_v without the refused tokens, by the inverse
// of its running sum.  That is the work: one row (with q two) of the vocabulary per sequence is read.  A wave sums a piece of 4 KiB of it
// at a time, all loads of a piece on their way together; the workgroups of a sequence all do the walk for themselves, and the one that
// arrives last finds the token's piece by the sums and reads it once more.  All sums are held in 64 bits: the border between two tokens
// is to be found where the sum of 10^5 values has it, and the tests take products of two 32-bit values, which 64 bits hold exactly.
// MI355X, 64 chains of 5 with drafts, 128,000 tokens: 16.3 us for 65.5 MB, 4.0 TB/s; 12.6 at the rate of a large copy, the rest is the walk's
// chain of loads before and the last workgroup's after.
constexpr int kVerifyThreads = 256;
constexpr int kVerifyWaves = kVerifyThreads / 64;
constexpr int kPieceLoads = 4;                           // 16-byte loads of a lane for a piece
constexpr int kMaxPieces = 4;                            // pieces of a wave
constexpr int kMaxChunk = kMaxPieces * kVerifyWaves * kPieceLoads * 64 * 8;   // elements of a workgroup
static_assert(kMaxVerifyNodes == kVerifyThreads, "a thread per node");

template <class T>
struct RowVector;
template <>
struct RowVector<float> {
    static constexpr int N = 4;
    typedef float type __attribute__((ext_vector_type(4), aligned(4)));   // (rows of any length: their elements' alignment)
    static OOCO_DEV float get(const type &v, int i) { return v[i]; }
    static OOCO_DEV float value(float x) { return x; }
};
template <>
struct RowVector<uint16_t> {
    static constexpr int N = 8;
    typedef uint16_t type __attribute__((ext_vector_type(8), aligned(2)));
    static OOCO_DEV float get(const type &v, int i) { return bf16_lo(v[i]); }
    static OOCO_DEV float value(uint16_t x) { return bf16_lo(x); }
};
// N elements of a row from index i on; those past the row's end are 0.
template <class T>
OOCO_DEV void load_row(const T *row, int i, int size, typename RowVector<T>::type &v)
{
    using R = RowVector<T>;
    if (i + R::N <= size) {
        v = *reinterpret_cast<const typename R::type *>(row + i);
    } else {
#pragma unroll
        for (int e = 0; e < R::N; ++e) v[e] = i + e < size ? row[i + e] : (T)0;
    }
}
// Inclusive sum over the lanes of a wave, and the sum of all: four shifts within rows of 16 lanes, then the last lane of a row to the
// rows behind it, twice -- moves of the vector ALU, where a shuffle through LDS takes a hundred cycles a stage.
template <int CTRL, int ROWS>
OOCO_DEV double moved(double v)   // 0 in lanes that nothing is moved to
{
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, ROWS, 0xF, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(u >> 32), CTRL, ROWS, 0xF, false);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
OOCO_DEV double wave_prefix(double v)
{
    v += moved<0x111, 0xF>(v);   // row_shr 1, 2, 4, 8
    v += moved<0x112, 0xF>(v);
    v += moved<0x114, 0xF>(v);
    v += moved<0x118, 0xF>(v);
    v += moved<0x142, 0xA>(v);   // row_bcast 15 to rows 1 and 3, 31 to rows 2 and 3
    v += moved<0x143, 0xC>(v);
    return v;
}
OOCO_DEV double lane_of(double v, int lane)   // wave-uniform lane
{
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)u, lane), hi = __builtin_amdgcn_readlane((int)(u >> 32), lane);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
OOCO_DEV double wave_sum(double v) { return lane_of(wave_prefix(v), 63); }

template <class T, bool DRAFT>
__global__ __launch_bounds__(kVerifyThreads) void verify_kernel(const VerifyArgs a)
{
    using R = RowVector<T>;
    constexpr int VEC = R::N, PIECE = kPieceLoads * 64 * VEC;
    __shared__ double prob[kMaxVerifyNodes];
    __shared__ int tok[kMaxVerifyNodes], sibling[kMaxVerifyNodes], first_child[kMaxVerifyNodes], walk[kMaxVerifyNodes];
    __shared__ uint32_t children[DRAFT ? 1 : kMaxVerifyNodes][kMaxVerifyNodes / 32];
    __shared__ uint32_t refused[kMaxChunk / 32];   // tokens of the workgroup's elements that have been refused
    __shared__ int sh_len, sh_last;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int seq = blockIdx.x / a.groups, group = blockIdx.x - seq * a.groups;
    int q0, n;
    rows_of(a.query_start_loc, seq, a.total_q, q0, n);
    n = min(n, kMaxVerifyNodes);
    int32_t *const path = a.path + (int64_t)seq * a.max_path;
    int32_t *const out = a.out_tokens + (int64_t)seq * (a.max_path + 1);
    if (n == 0) {
        if (group == 0) {
            if (tid == 0) a.counts[seq] = 0;
            for (int i = tid; i <= a.max_path; i += kVerifyThreads) {
                if (i < a.max_path) path[i] = -1;
                out[i] = -1;
            }
        }
        return;
    }
    const T *const target = static_cast<const T *>(a.target) + (int64_t)q0 * a.stride;
    const T *const draft = static_cast<const T *>(a.draft) + (int64_t)q0 * a.stride;

    // ---- the walk
    int my_par = -1, my_tok = -1;
    double my_p = 0.0, my_q = 1.0, my_u = 0.0;
    if (tid < n) {
        my_par = a.parents ? a.parents[q0 + tid] : tid - 1;
        if (my_par >= tid || my_par < 0) my_par = -1;
        my_tok = a.tokens[q0 + tid];
        my_u = a.uniforms[q0 + tid];
        if (my_par >= 0 && my_tok >= 0 && my_tok < a.vocab) {
            my_p = R::value(target[my_par * a.stride + my_tok]);
            if (DRAFT) my_q = R::value(draft[tid * a.stride + my_tok]);
        }
    }
    tok[tid] = my_tok;
    first_child[tid] = INT_MAX;
    if (!DRAFT && a.parents) {
#pragma unroll
        for (int w = 0; w < kMaxVerifyNodes / 32; ++w) children[tid][w] = 0;
    }
    const int chunk = a.pieces * kVerifyWaves * PIECE;     // elements of the workgroup
    const int64_t c0 = (int64_t)group * chunk;
    if (!DRAFT)
        for (int i = tid; i < chunk / 32; i += kVerifyThreads) refused[i] = 0;
    __syncthreads();
    double rest = 1.0;
    if (!DRAFT && a.parents) {
        // The sibling before each node, by the children of each node as bits.
        int older = -1;
        if (my_par >= 0) atomicOr(&children[my_par][tid / 32], 1u << (tid & 31));
        __syncthreads();
        if (my_par >= 0) {
            int w = tid / 32;
            uint32_t before = children[my_par][w] & ((1u << (tid & 31)) - 1u);
            while (!before && w > 0) before = children[my_par][--w];
            if (before) older = 32 * w + 31 - __clz((int)before);
        }
        sibling[tid] = older;
        __syncthreads();
        for (int j = older; j >= 0; j = sibling[j])   // a token that a sibling has had already is not there any more
            if (tok[j] == my_tok) my_p = 0.0;
        prob[tid] = my_p;
        __syncthreads();
        for (int j = older; j >= 0; j = sibling[j]) rest -= prob[j];
    }
    if (my_par >= 0 && my_u * my_q * rest < my_p) atomicMin(&first_child[my_par], tid);
    __syncthreads();
    if (tid == 0) {
        int at = 0, len = 0;
        while (len < a.max_path) {
            const int c = first_child[at];
            if (c == INT_MAX) break;
            walk[len++] = c;
            at = c;
        }
        sh_len = len;
        sh_last = at;
    }
    __syncthreads();
    const int len = sh_len, last = sh_last;
    // (a path that ends for want of room refuses nobody)
    const bool refuses = len < a.max_path;
    auto mark = [&](int64_t first) {
        if (!DRAFT && refuses && my_par == last && my_tok >= first && my_tok < first + chunk && my_tok < a.vocab)
            atomicOr(&refused[(my_tok - first) / 32], 1u << ((my_tok - first) & 31));
    };
    mark(c0);
    __syncthreads();
    const T *const p_row = target + last * a.stride;
    const bool minus = DRAFT && refuses && last + 1 < n;
    const T *const q_row = draft + (minus ? last + 1 : 0) * a.stride;

    // The piece from element i0 on, of which the lane has elements i0 + 64 VEC j + VEC lane + e: what there was, and what is left.
    typename R::type pv[kPieceLoads], qv[kPieceLoads];
    auto load_piece = [&](int i0) {
#pragma unroll
        for (int j = 0; j < kPieceLoads; ++j) load_row(p_row, i0 + (64 * j + lane) * VEC, a.vocab, pv[j]);
        if (minus) {
#pragma unroll
            for (int j = 0; j < kPieceLoads; ++j) load_row(q_row, i0 + (64 * j + lane) * VEC, a.vocab, qv[j]);
        }
    };
    auto weights = [&](int j, int64_t bit0, float (&f)[VEC], double (&w)[VEC]) {   // of load j; bit0: place of the piece in `refused`
        const int b = (int)bit0 + (64 * j + lane) * VEC;
        const uint32_t bits = DRAFT ? 0u : refused[b / 32] >> (b & 31);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            f[e] = R::get(pv[j], e);
            f[e] = f[e] > 0.f && f[e] <= FLT_MAX ? f[e] : 0.f;
            double d = f[e];
            if (minus) d -= (double)R::get(qv[j], e);
            w[e] = d > 0.0 && !((bits >> e) & 1u) ? d : 0.0;
        }
    };
    double *const sums = a.sums + (int64_t)seq * a.groups * (a.pieces * kVerifyWaves) * 2;
    for (int k = 0; k < a.pieces; ++k) {
        const int piece = (group * a.pieces + k) * kVerifyWaves + wave;   // of the row
        const int64_t i0 = (int64_t)piece * PIECE;
        double left = 0.0, full = 0.0;
        if (i0 < a.vocab) {
            load_piece((int)i0);
#pragma unroll
            for (int j = 0; j < kPieceLoads; ++j) {
                float f[VEC];
                double w[VEC];
                weights(j, i0 - c0, f, w);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    left += w[e];
                    full += (double)f[e];
                }
            }
            left = wave_sum(left);
            full = wave_sum(full);
        }
        if (lane == 0) {
            __hip_atomic_store(sums + 2 * piece, left, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __hip_atomic_store(sums + 2 * piece + 1, full, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the sums have reached memory before the count
    __syncthreads();
    if (tid == 0) {
        const int prev = __hip_atomic_fetch_add(a.arrivals + (int64_t)seq * a.arrivals_apart, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        sh_last = prev == a.groups - 1;
    }
    __syncthreads();
    if (!sh_last) return;

    // ---- the workgroup that arrived last
    if (tid == 0) {
        a.counts[seq] = len + 1;
        __hip_atomic_store(a.arrivals + (int64_t)seq * a.arrivals_apart, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // ready for the next call
    }
    for (int i = tid; i <= a.max_path; i += kVerifyThreads) {
        if (i < a.max_path) path[i] = i < len ? walk[i] : -1;
        if (i != len) out[i] = i < len ? tok[walk[i]] : -1;
    }
    const int pieces = a.groups * a.pieces * kVerifyWaves;
    auto sum_at = [&](int i, int which) -> double {
        return i < pieces ? __hip_atomic_load(sums + 2 * i + which, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0;
    };
    // Every wave finds the piece (all the same): the first whose running sum passes the aim, or the last with a weight.
    double total[2] = {0.0, 0.0};
    for (int i = lane; i < pieces; i += 64) {
        total[0] += sum_at(i, 0);
        total[1] += sum_at(i, 1);
    }
    total[0] = wave_sum(total[0]);
    total[1] = wave_sum(total[1]);
    const bool use_full = !(total[0] > 0.0);        // (nothing left: the draw is from all there was)
    const double aim = (double)a.final_uniforms[seq] * total[use_full];
    double before = 0.0, base = 0.0;
    int found_piece = -1;
    for (int i0 = 0; i0 < pieces; i0 += 64) {
        const double v = sum_at(i0 + lane, use_full);
        const double run = before + wave_prefix(v);
        const uint64_t some = __ballot(v > 0.0), past = __ballot(v > 0.0 && run > aim);
        const int k = past ? __ffsll((unsigned long long)past) - 1 : some ? 63 - __clzll((long long)some) : -1;
        if (k >= 0) {
            found_piece = i0 + k;
            base = lane_of(run - v, k);
        }
        if (past) break;
        before = lane_of(run, 63);
    }
    int drawn = -1;
    if (found_piece >= 0) {
        const int i0 = found_piece * PIECE;
        const int64_t first = (int64_t)(found_piece / (a.pieces * kVerifyWaves)) * chunk;   // of the workgroup whose piece it is
        if (!DRAFT && first != c0) {
            __syncthreads();
            for (int i = tid; i < chunk / 32; i += kVerifyThreads) refused[i] = 0;
            __syncthreads();
            mark(first);
            __syncthreads();
        }
        if (wave != 0) return;
        load_piece(i0);
        int found = INT_MAX, any = -1;
#pragma unroll
        for (int j = 0; j < kPieceLoads; ++j) {
            float f[VEC];
            double w[VEC], own = 0.0;
            weights(j, i0 - first, f, w);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                if (use_full) w[e] = f[e];
                own += w[e];
            }
            const double incl = wave_prefix(own);
            double run = base + incl - own;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                run += w[e];
                const int i = i0 + (64 * j + lane) * VEC + e;
                any = w[e] > 0.0 ? i : any;
                found = w[e] > 0.0 && run > aim ? min(found, i) : found;
            }
            base += lane_of(incl, 63);
        }
#pragma unroll
        for (int d = 32; d; d >>= 1) {
            found = min(found, __shfl_xor(found, d));
            any = max(any, __shfl_xor(any, d));
        }
        drawn = found != INT_MAX ? found : any;
    }
    if (tid == 0) out[len] = drawn;
}

void verify_layout(VerifyArgs &a, bool bf16, int num_cus)
{
    // As many pieces for a wave, 1, 2 or 4, as leave two workgroups to a compute unit, or four that read one row and not two: all of them do
    // the walk.  MI355X, us, with up to 8 / 4 / 2 workgroups: 64 chains of 5, 128,000 tokens, with drafts 19.1 / 18.4 / 18.1, without 17.5 /
    // 15.9 / 17.3; 256 trees of three nodes, 32,000 tokens 16.8 / 15.2 / 16.2.
    const int piece = kPieceLoads * 64 * (bf16 ? 8 : 4);
    const int64_t pieces = ((int64_t)a.vocab + piece - 1) / piece, workgroups = (int64_t)num_cus * (a.draft ? 2 : 4);
    a.pieces = 1;
    while (a.pieces < kMaxPieces && pieces * a.num_seqs > workgroups * kVerifyWaves * a.pieces) a.pieces *= 2;
    a.groups = (int)((pieces + kVerifyWaves * a.pieces - 1) / (kVerifyWaves * a.pieces));
}

size_t verify_workspace(const VerifyArgs &a) { return (size_t)a.num_seqs * (size_t)a.groups * (a.pieces * kVerifyWaves) * 2 * sizeof(double); }

hipError_t launch_verify(const VerifyArgs &a, bool bf16, hipStream_t s)
{
    auto *const kernel = bf16 ? (a.draft ? verify_kernel<uint16_t, true> : verify_kernel<uint16_t, false>)
                              : (a.draft ? verify_kernel<float, true> : verify_kernel<float, false>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)((int64_t)a.num_seqs * a.groups)), dim3(kVerifyThreads), 0, s, a);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------------
// Accepted nodes to their places: the d-th node of the path goes from slot ctx + path[d] to slot ctx + 1 + d.  A path rises, so
// path[d] > d: a node moves towards the front or stays, and its place is one that no later node of the path comes from.  The nodes of
// a path go in groups of up to eight that lie next to each other in a wave: lane = (column of the cache, node), a column being a 16-byte
// piece of K or a dim of V.  All nodes of a group are loaded before one is stored, and the groups go in order, so nothing is overwritten
// before it has been read; and as the places of a group lie side by side in every column, so do its stores (64 sequences of 4.4 nodes, 32
// layers of 8 heads, us: 122 with a column's nodes one after the other in one lane, whose stores are a request to L2 each, 107 like this).
// What bounds it is the cache's layout: V keeps the 16 tokens of a block side by side, so every line of a block is touched for one token of
// it (the same batch: 73 MB to move, 327 MB of lines that miss L2, read or written in part).
constexpr int kCompactThreads = 256;
constexpr int kCompactAhead = 4;   // columns whose loads are sent off together

__global__ __launch_bounds__(kCompactThreads) void kv_compact_kernel(const CompactArgs a)
{
    __shared__ int64_t from[kCompactThreads], to[kCompactThreads];   // block * 16 + slot; from: -1 for a node that stays
    const int tid = threadIdx.x;
    const int seq = blockIdx.x;
    const int moves = min(a.counts[seq] - 1, min(a.max_path, kCompactThreads));
    if (moves <= 0) return;
    const int ctx = a.ctx_lens[seq];
    if (tid < moves) {
        auto place = [&](int64_t token) -> int64_t {
            if (token < 0 || token / kBlockSize >= a.max_blocks_per_seq) return -1;
            const int64_t blk = a.block_tables[(int64_t)seq * a.max_blocks_per_seq + token / kBlockSize];
            return blk >= 0 && blk < a.num_blocks ? blk * kBlockSize + token % kBlockSize : -1;
        };
        const int node = a.path[(int64_t)seq * a.max_path + tid];
        const bool moved = node > tid + 1 && ctx >= 0;   // (one that is in its place stays)
        const int64_t f = moved ? place((int64_t)ctx + node) : -1, t = moved ? place((int64_t)ctx + 1 + tid) : -1;
        from[tid] = t >= 0 ? f : -1;
        to[tid] = t;
    }
    __syncthreads();
    const int group_log2 = moves == 1 ? 0 : moves == 2 ? 1 : moves <= 4 ? 2 : 3;
    const int group = 1 << group_log2, columns = kCompactThreads >> group_log2;   // columns of the workgroup at a time
    const int mine = tid >> group_log2;
    const int pieces = a.Hkv * a.hd / 8, dims = a.Hkv * a.hd;
    const int64_t block = (int64_t)dims * kBlockSize;   // elements
    const int first = blockIdx.y * a.layers_each, last = min(first + a.layers_each, a.layers);
    for (int layer = first; layer < last; ++layer) {
        uint16_t *const k = a.k[layer], *const v = a.v[layer];
        for (int d0 = 0; d0 < moves; d0 += group) {
            const int d = d0 + (tid & (group - 1));
            const int64_t f = d < moves ? from[d] : -1, t = d < moves ? to[d] : -1;
            const bool moved = f >= 0;
            const u32x4 *const kf = reinterpret_cast<const u32x4 *>(k + (moved ? f / kBlockSize * block : 0)) + (moved ? f % kBlockSize : 0);
            u32x4 *const kt = reinterpret_cast<u32x4 *>(k + (moved ? t / kBlockSize * block : 0)) + (moved ? t % kBlockSize : 0);
            for (int c = blockIdx.z * columns + mine; c < pieces + mine; c += kCompactAhead * gridDim.z * columns) {
                u32x4 x[kCompactAhead];
#pragma unroll
                for (int i = 0; i < kCompactAhead; ++i) {
                    const int p = c + i * gridDim.z * columns;
                    if (moved && p < pieces) x[i] = kf[(int64_t)p * kBlockSize];
                }
#pragma unroll
                for (int i = 0; i < kCompactAhead; ++i) {
                    const int p = c + i * gridDim.z * columns;
                    if (moved && p < pieces) kt[(int64_t)p * kBlockSize] = x[i];
                }
            }
            const uint16_t *const vf = v + (moved ? f / kBlockSize * block + f % kBlockSize : 0);
            uint16_t *const vt = v + (moved ? t / kBlockSize * block + t % kBlockSize : 0);
            for (int c = blockIdx.z * columns + mine; c < dims + mine; c += 2 * kCompactAhead * gridDim.z * columns) {
                uint16_t x[2 * kCompactAhead];
#pragma unroll
                for (int i = 0; i < 2 * kCompactAhead; ++i) {
                    const int e = c + i * gridDim.z * columns;
                    if (moved && e < dims) x[i] = vf[(int64_t)e * kBlockSize];
                }
#pragma unroll
                for (int i = 0; i < 2 * kCompactAhead; ++i) {
                    const int e = c + i * gridDim.z * columns;
                    if (moved && e < dims) vt[(int64_t)e * kBlockSize] = x[i];
                }
            }
        }
    }
}

hipError_t launch_kv_compact(CompactArgs &a, int num_seqs, int num_cus, hipStream_t s)
{
    // Slices of the columns where (sequence, layer) pairs are fewer than eight workgroups to a compute unit, some layers for a workgroup where
    // they are more.
    const int64_t pairs = (int64_t)num_seqs * a.layers, want = 8 * (int64_t)num_cus;
    a.layers_each = (int)std::max<int64_t>(1, std::min<int64_t>(a.layers, pairs / want));
    const unsigned groups = (unsigned)((a.layers + a.layers_each - 1) / a.layers_each);
    const unsigned slices = (unsigned)std::max<int64_t>(1, std::min<int64_t>(8, want / std::max<int64_t>(1, pairs)));
    hipLaunchKernelGGL(kv_compact_kernel, dim3((unsigned)num_seqs, groups, slices), dim3(kCompactThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace ooco
