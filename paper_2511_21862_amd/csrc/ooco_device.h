// Device primitives that the kernels of several files share: vector types, conversions, single-instruction maxima,
// device-scope accesses, reductions over the rows of a wave, and the lookup of a work item in a cumulative array.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ooco {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

#define OOCO_DEV __device__ __forceinline__

constexpr int kNoVmem = 0x78F;   // sched_barrier mask: everything but vector-memory operations may cross

OOCO_DEV uint32_t pack2_bf16(float a, float b)
{
    bf16x2 v = {(__bf16)a, (__bf16)b};   // round to nearest even
    return __builtin_bit_cast(uint32_t, v);
}

OOCO_DEV float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// max of three without the NaN-quieting moves that fmaxf would add (one v_max3_f32)
OOCO_DEV float max3(float a, float b, float c)
{
    float d;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
    return d;
}

// max of two / with a floor of -1e30, as single instructions (no NaN-quieting moves)
OOCO_DEV float max2(float a, float b)
{
    float d;
    asm("v_max_f32_e32 %0, %1, %2" : "=v"(d) : "v"(a), "v"(b));
    return d;
}
OOCO_DEV float floor_m1e30(float a)
{
    float d;
    asm("v_max_f32_e32 %0, 0xf149f2ca, %1" : "=v"(d) : "v"(a));   // 0xf149f2ca = -1e30f
    return d;
}
// max of the 32 scores a lane holds for one step (two 16-register MFMA results), as one dependent chain of
// v_max3_f32 in two asm statements (an asm statement takes at most 30 operands)
OOCO_DEV float max32(const f32x16 &a, const f32x16 &b)
{
    float d, e;
    asm("v_max3_f32 %0, %1, %2, %3\n\t"
        "v_max3_f32 %0, %0, %4, %5\n\t"
        "v_max3_f32 %0, %0, %6, %7\n\t"
        "v_max3_f32 %0, %0, %8, %9\n\t"
        "v_max3_f32 %0, %0, %10, %11\n\t"
        "v_max3_f32 %0, %0, %12, %13\n\t"
        "v_max3_f32 %0, %0, %14, %15\n\t"
        "v_max3_f32 %0, %0, %16, %17"
        : "=&v"(d)
        : "v"(a[0]), "v"(b[0]), "v"(a[1]), "v"(b[1]), "v"(a[2]), "v"(b[2]), "v"(a[3]), "v"(b[3]), "v"(a[4]), "v"(b[4]),
          "v"(a[5]), "v"(b[5]), "v"(a[6]), "v"(b[6]), "v"(a[7]), "v"(b[7]), "v"(a[8]));
    asm("v_max3_f32 %0, %1, %2, %3\n\t"
        "v_max3_f32 %0, %0, %4, %5\n\t"
        "v_max3_f32 %0, %0, %6, %7\n\t"
        "v_max3_f32 %0, %0, %8, %9\n\t"
        "v_max3_f32 %0, %0, %10, %11\n\t"
        "v_max3_f32 %0, %0, %12, %13\n\t"
        "v_max3_f32 %0, %0, %14, %15\n\t"
        "v_max_f32_e32 %0, %0, %16"
        : "=&v"(e)
        : "v"(d), "v"(b[8]), "v"(a[9]), "v"(b[9]), "v"(a[10]), "v"(b[10]), "v"(a[11]), "v"(b[11]), "v"(a[12]), "v"(b[12]),
          "v"(a[13]), "v"(b[13]), "v"(a[14]), "v"(b[14]), "v"(a[15]), "v"(b[15]));
    return e;
}

// the same of 16 scores
OOCO_DEV float max16(const f32x16 &a)
{
    float d;
    asm("v_max3_f32 %0, %1, %2, %3\n\t"
        "v_max3_f32 %0, %0, %4, %5\n\t"
        "v_max3_f32 %0, %0, %6, %7\n\t"
        "v_max3_f32 %0, %0, %8, %9\n\t"
        "v_max3_f32 %0, %0, %10, %11\n\t"
        "v_max3_f32 %0, %0, %12, %13\n\t"
        "v_max3_f32 %0, %0, %14, %15\n\t"
        "v_max_f32_e32 %0, %0, %16"
        : "=&v"(d)
        : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "v"(a[4]), "v"(a[5]), "v"(a[6]), "v"(a[7]), "v"(a[8]), "v"(a[9]),
          "v"(a[10]), "v"(a[11]), "v"(a[12]), "v"(a[13]), "v"(a[14]), "v"(a[15]));
    return d;
}

// acc + lo + hi of a packed bf16 pair (one v_dot2c_f32_bf16 against the pair (1, 1))
OOCO_DEV float sum2_bf16(uint32_t pair, float acc)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), __builtin_bit_cast(bf16x2, 0x3F803F80u), acc,
                                           false);
}

// Device-scope (all XCDs) relaxed store / load of one float: the store writes through to memory,
// the load bypasses the non-coherent cache levels.
typedef float f32x2 __attribute__((ext_vector_type(2)));
OOCO_DEV void store_dev2(float *ptr, float a, float b)   // ptr is 8-byte aligned
{
    const f32x2 v = {a, b};
    __hip_atomic_store(reinterpret_cast<uint64_t *>(ptr), __builtin_bit_cast(uint64_t, v), __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
}
// The same cache policy for a 16-byte store (a plain vector store with the device-scope bit: the ordering
// against the arrival counter comes from s_waitcnt, 16-byte atomicity is not needed).  Far fewer memory
// operations than 8-byte atomic stores, which matters for the 64 KiB partial results of a prefill part.
// (The s_nop covers the wait states a wide store needs before its data registers may be overwritten, which
// the compiler cannot see through the asm.)
OOCO_DEV void store_dev4(float *ptr, f32x4 v)   // ptr is 16-byte aligned
{
    asm volatile("global_store_dwordx4 %0, %1, off sc1\n\ts_nop 1" ::"v"(ptr), "v"(v) : "memory");
}
OOCO_DEV f32x2 load_dev2(const float *ptr)
{
    const uint64_t u = __hip_atomic_load(reinterpret_cast<uint64_t *>(const_cast<float *>(ptr)), __ATOMIC_RELAXED,
                                         __HIP_MEMORY_SCOPE_AGENT);
    return __builtin_bit_cast(f32x2, u);
}


// ------------------------------------------------------------------------------------------
// Cross-lane reductions over the four 16-lane rows of a wave with the CDNA4 lane-swap
// instructions (VALU only, no LDS traffic): v_permlane16_swap exchanges the odd rows of its first
// operand with the even rows of the second, v_permlane32_swap the upper half of the first with
// the lower half of the second; fed with two copies of one value they return both partners of
// an xor-16 / xor-32 butterfly.  (Vector elements are copied to scalars before
// __builtin_bit_cast: a bit_cast applied directly to an element reference reads element 0.)
OOCO_DEV void swap16(float v, float &lo, float &hi)
{
    const unsigned u = __builtin_bit_cast(unsigned, v);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const unsigned a0 = a[0], a1 = a[1];
    lo = __builtin_bit_cast(float, a0);
    hi = __builtin_bit_cast(float, a1);
}
OOCO_DEV void swap32(float v, float &lo, float &hi)
{
    const unsigned u = __builtin_bit_cast(unsigned, v);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const unsigned a0 = a[0], a1 = a[1];
    lo = __builtin_bit_cast(float, a0);
    hi = __builtin_bit_cast(float, a1);
}
OOCO_DEV float rows_max(float v)
{
    float x, y;
    swap16(v, x, y);
    swap32(fmaxf(x, y), x, y);
    return fmaxf(x, y);
}
OOCO_DEV float rows_sum(float v)
{
    float x, y;
    swap16(v, x, y);
    swap32(x + y, x, y);
    return x + y;
}

// ------------------------------------------------------------------------------------------
// Work lookup shared by both kernels: cum[] is non-decreasing with cum[0] = 0; returns the number
// of entries j in [1, n] with cum[j] <= x, i.e. the index i with cum[i] <= x < cum[i+1].
// All 64 lanes of the wave must call it with the same x.
template <class CumAt>
OOCO_DEV int count_le(CumAt cum_at, int n, int x, int lane)
{
    int cnt = 0;
    for (int base = 1; base <= n; base += 64) {
        const int idx = base + lane;
        const int v = idx <= n ? cum_at(idx) : 0x7FFFFFFF;
        const int c = __popcll(__ballot(v <= x));
        cnt += c;
        if (c < 64) break;
    }
    return cnt;
}

}  // namespace ooco
