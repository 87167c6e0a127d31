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

// ------------------------------------------------------------------------------------------
// Masks and positions.  A node sees itself and its ancestors: with M_0(i) = {i} and P_0(i) = parent(i), doubling the distance
// M_k+1(i) = M_k(i) + M_k(P_k(i)), P_k+1(i) = P_k(P_k(i)) needs log2 of the depth rounds, where a walk up the tree would need the
// depth; the number of the nodes in M is the depth + 1.  One workgroup per sequence, a thread per node, the sets as bits in LDS.
// A parent has to be an earlier node: anything else is taken as none, so the walk ends whatever the array holds.
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
// A workgroup has the rows of one (sequence, KV block) pair, as the plain append does (see kv_append_kernel for the order of the
// pairs: sequence i owns the pairs from query_start_loc[i] / 16 + 2 i on), because the cache keeps 16 tokens of a dim or of a
// group of 8 dims side by side; `parts` workgroups share a pair's heads.  The angles' turns p f / (2 pi) are reduced in 64 bits --
// a position of 10^5 times a frequency of 1 leaves 32 bits three digits behind the point -- and cosine and sine are those of the
// hardware, which take turns; they go through LDS, once per row and pair for all heads of the workgroup.
constexpr int kRopeThreads = 256;

OOCO_DEV float bf16_lo(uint32_t u) { return __builtin_bit_cast(float, u << 16); }
OOCO_DEV float bf16_hi(uint32_t u) { return __builtin_bit_cast(float, u & 0xFFFF0000u); }

template <bool INTERLEAVED>
__global__ __launch_bounds__(kRopeThreads) void rope_append_kernel(const RopeArgs a)
{
    __shared__ f32x2 turn[kBlockSize][kMaxRotaryPairs];   // (cosine, sine)
    const int tid = threadIdx.x, lane = tid & 63;
    const int pair = blockIdx.x / a.parts, part = blockIdx.x - pair * a.parts;
    const int32_t *const qsl = a.query_start_loc;
    auto g_at = [&](int idx) -> int { return qsl[idx] / kBlockSize + 2 * idx; };
    const int seq = __builtin_amdgcn_readfirstlane(min(count_le(g_at, a.num_seqs, pair, lane), a.num_seqs - 1));
    int q0, q_len;
    rows_of(qsl, seq, a.total_q, q0, q_len);
    const int ctx = a.ctx_lens[seq];
    if (q_len == 0 || ctx < 0) return;
    const int64_t end = (int64_t)ctx + q_len;                     // (may lie past the block table)
    const int64_t bidx = ctx / kBlockSize + (int64_t)(pair - (q0 / kBlockSize + 2 * seq));
    if (bidx < ctx / kBlockSize || bidx * kBlockSize >= end) return;   // beyond the sequence's last touched block
    const int t_lo = (int)max((int64_t)0, bidx * kBlockSize - ctx);
    const int slot0 = (int)(ctx + (int64_t)t_lo - bidx * kBlockSize);
    const int nrow = min(kBlockSize - slot0, q_len - t_lo);
    const int row0 = q0 + t_lo;
    // (a block that the cache does not have: the queries are rotated all the same, nothing is appended)
    const int64_t blk = bidx < a.max_blocks_per_seq ? a.block_tables[(int64_t)seq * a.max_blocks_per_seq + bidx] : -1;
    const bool blk_ok = blk >= 0 && blk < a.num_blocks;

    const int pairs = a.pairs, hd = a.hd;
    for (int i = tid; i < nrow * pairs; i += kRopeThreads) {
        const int r = i / pairs, x = i - r * pairs;
        const int pos = a.positions ? a.positions[row0 + r] : ctx + t_lo + r;
        const float f = (float)__builtin_amdgcn_fract((double)pos * a.turns[x]);
        turn[r][x] = f32x2{__builtin_amdgcn_cosf(f) * a.factor, __builtin_amdgcn_sinf(f) * a.factor};
    }
    __syncthreads();

    // heads of this part: of q, of k and of v, numbered one after the other
    const int heads = a.Hq + 2 * a.Hkv;
    const int h0 = heads * part / a.parts, h1 = heads * (part + 1) / a.parts;
    const int qa = min(h0, a.Hq), qb = min(h1, a.Hq);
    const int ka = min(max(h0 - a.Hq, 0), a.Hkv), kb = min(max(h1 - a.Hq, 0), a.Hkv);
    const int va = max(h0 - a.Hq - a.Hkv, 0), vb = max(h1 - a.Hq - a.Hkv, 0);

    // One task: the 16-byte pieces of a head that belong together -- a piece of the first half of the rotated dims and its
    // partner of the second half, or one piece (of pairs side by side, or of dims that are not rotated).
    const int tasks = INTERLEAVED ? hd / 8 : pairs / 8 + (hd - 2 * pairs) / 8;
    auto rotate = [&](int r, int c, const u32x4 *src, u32x4 *dst, int dst_step) {   // pieces of dst are dst_step apart
        if (!INTERLEAVED && c < pairs / 8) {
            const int c2 = c + pairs / 8;
            const u32x4 x = src[c], y = src[c2];
            u32x4 ox, oy;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const f32x2 t0 = turn[r][8 * c + 2 * w], t1 = turn[r][8 * c + 2 * w + 1];
                const float x0 = bf16_lo(x[w]), x1 = bf16_hi(x[w]), y0 = bf16_lo(y[w]), y1 = bf16_hi(y[w]);
                ox[w] = pack2_bf16(x0 * t0[0] - y0 * t0[1], x1 * t1[0] - y1 * t1[1]);
                oy[w] = pack2_bf16(y0 * t0[0] + x0 * t0[1], y1 * t1[0] + x1 * t1[1]);
            }
            dst[(int64_t)c * dst_step] = ox;
            dst[(int64_t)c2 * dst_step] = oy;
            return;
        }
        if (!INTERLEAVED) c += pairs / 8;
        u32x4 x = src[c];
        if (INTERLEAVED && c < pairs / 4) {
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const f32x2 t = turn[r][4 * c + w];
                const float x0 = bf16_lo(x[w]), x1 = bf16_hi(x[w]);
                x[w] = pack2_bf16(x0 * t[0] - x1 * t[1], x1 * t[0] + x0 * t[1]);
            }
        }
        dst[(int64_t)c * dst_step] = x;
    };
    for (int i = tid; i < nrow * (qb - qa) * tasks; i += kRopeThreads) {
        const int j = i / tasks, c = i - j * tasks;
        const int r = j / (qb - qa), h = qa + j - r * (qb - qa);
        rotate(r, c, reinterpret_cast<const u32x4 *>(a.q + (row0 + r) * a.q_stride + h * hd),
               reinterpret_cast<u32x4 *>(a.q_out + ((int64_t)(row0 + r) * a.Hq + h) * hd), 1);
    }
    if (!blk_ok) return;
    // K: the rows of a piece are side by side in the cache, so they are side by side in a wave
    for (int i = tid; i < nrow * (kb - ka) * tasks; i += kRopeThreads) {
        const int j = i / nrow, r = i - j * nrow;
        const int h = ka + j / tasks, c = j - (h - ka) * tasks;
        rotate(r, c, reinterpret_cast<const u32x4 *>(a.k_new + (row0 + r) * a.k_stride + h * hd),
               reinterpret_cast<u32x4 *>(a.k_cache) + (blk * a.Hkv + h) * (hd / 8) * kBlockSize + slot0 + r, kBlockSize);
    }
    // V: a thread has two adjacent dims of all rows, which are 2 x 32 bytes of the cache
    uint16_t *const v_dst = a.v_cache + blk * a.Hkv * hd * kBlockSize;
    const uint16_t *const v_src = a.v_new + row0 * a.v_stride;
    for (int e = va * hd + 2 * tid; e < vb * hd; e += 2 * kRopeThreads) {
        uint32_t x[kBlockSize];
#pragma unroll
        for (int sl = 0; sl < kBlockSize; ++sl) {
            const int r = sl - slot0;
            x[sl] = 0;
            if (r >= 0 && r < nrow) x[sl] = *reinterpret_cast<const uint32_t *>(v_src + r * a.v_stride + e);
        }
#pragma unroll
        for (int d = 0; d < 2; ++d) {
            uint16_t *const dst = v_dst + (int64_t)(e + d) * kBlockSize;   // (32-byte aligned)
            auto at = [&](int sl) -> uint32_t { return d ? x[sl] >> 16 : x[sl] & 0xFFFFu; };
            // quarters of a cache row that the step covers whole are written with one store each, the ragged ends slot by slot
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (4 * k >= slot0 && 4 * k + 4 <= slot0 + nrow) {
                    *reinterpret_cast<u32x2 *>(dst + 4 * k) = u32x2{at(4 * k) | (at(4 * k + 1) << 16), at(4 * k + 2) | (at(4 * k + 3) << 16)};
                } else {
#pragma unroll
                    for (int sl = 4 * k; sl < 4 * k + 4; ++sl)
                        if (sl >= slot0 && sl < slot0 + nrow) dst[sl] = (uint16_t)at(sl);
                }
            }
        }
    }
}

hipError_t launch_rope_append(RopeArgs &a, bool interleaved, int num_cus, hipStream_t s)
{
    const int heads = a.Hq + 2 * a.Hkv;
    const int64_t pairs = a.total_q / kBlockSize + 2 * (int64_t)a.num_seqs + 1;
    a.parts = std::max(1, heads / 4);
    hipLaunchKernelGGL(interleaved ? rope_append_kernel<true> : rope_append_kernel<false>, dim3((unsigned)(pairs * a.parts)), dim3(kRopeThreads), 0, s, a);
    return hipGetLastError();
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
// path[d] > d: a node moves towards the front or stays, and its place is one that no later node of the path comes from.  A thread
// has one column of the cache -- a 16-byte piece of K, two dims of V -- and moves its nodes in their order, all loads of a batch
// before its stores, so nothing is overwritten before it has been read.  One workgroup per (sequence, layer, slice of columns).
constexpr int kCompactThreads = 256;

__global__ __launch_bounds__(kCompactThreads) void kv_compact_kernel(const CompactArgs a)
{
    __shared__ int64_t from[kCompactThreads], to[kCompactThreads];   // block * 16 + slot, or -1
    const int tid = threadIdx.x;
    const int seq = blockIdx.x, layer = blockIdx.y;
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
        int64_t f = node > tid + 1 && ctx >= 0 ? place((int64_t)ctx + node) : -1;   // (one that is in its place stays)
        int64_t t = f >= 0 ? place((int64_t)ctx + 1 + tid) : -1;
        from[tid] = t >= 0 ? f : -1;
        to[tid] = t;
    }
    __syncthreads();
    uint16_t *const k = a.k[layer], *const v = a.v[layer];
    const int pieces = a.Hkv * a.hd / 8, columns = pieces + a.Hkv * a.hd;
    for (int i = tid + kCompactThreads * blockIdx.z; i < columns; i += kCompactThreads * gridDim.z) {
        if (i < pieces) {   // K: piece i of a token, 16 slots of 16 bytes
            u32x4 *const col = reinterpret_cast<u32x4 *>(k) + (int64_t)i * kBlockSize;
            for (int d0 = 0; d0 < moves; d0 += 4) {
                u32x4 x[4];
#pragma unroll
                for (int d = 0; d < 4; ++d)
                    if (d0 + d < moves && from[d0 + d] >= 0)
                        x[d] = col[(from[d0 + d] / kBlockSize) * pieces * kBlockSize + from[d0 + d] % kBlockSize];
#pragma unroll
                for (int d = 0; d < 4; ++d)
                    if (d0 + d < moves && from[d0 + d] >= 0)
                        col[(to[d0 + d] / kBlockSize) * pieces * kBlockSize + to[d0 + d] % kBlockSize] = x[d];
            }
        } else {            // V: one dim, 16 slots of 2 bytes
            uint16_t *const col = v + (int64_t)(i - pieces) * kBlockSize;
            const int64_t block = (int64_t)a.Hkv * a.hd * kBlockSize;
            for (int d0 = 0; d0 < moves; d0 += 4) {
                uint16_t x[4];
#pragma unroll
                for (int d = 0; d < 4; ++d)
                    if (d0 + d < moves && from[d0 + d] >= 0) x[d] = col[(from[d0 + d] / kBlockSize) * block + from[d0 + d] % kBlockSize];
#pragma unroll
                for (int d = 0; d < 4; ++d)
                    if (d0 + d < moves && from[d0 + d] >= 0) col[(to[d0 + d] / kBlockSize) * block + to[d0 + d] % kBlockSize] = x[d];
            }
        }
    }
}

hipError_t launch_kv_compact(const CompactArgs &a, int layers, int num_seqs, hipStream_t s)
{
    const int columns = a.Hkv * a.hd / 8 + a.Hkv * a.hd;
    const unsigned slices = (unsigned)std::min(8, (columns + kCompactThreads - 1) / kCompactThreads);
    hipLaunchKernelGGL(kv_compact_kernel, dim3((unsigned)num_seqs, (unsigned)layers, slices), dim3(kCompactThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace ooco
