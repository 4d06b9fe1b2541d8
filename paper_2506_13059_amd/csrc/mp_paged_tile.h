// What the kernels that hold query rows in tiles of 16 share: device code of mp_paged_token.hip and mp_paged_rows.hip.
#pragma once
#include "mp_paged_plan.h"

namespace mp {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) unsigned char lds_byte;

// A part: weighted values as the lanes hold them, then maxima, then sums.
constexpr int part_floats(int groups) { return 16 * groups * kHeadDim + 2 * 16 * groups; }

__device__ __forceinline__ void load_to_lds(const void* src, uint32_t lds_off)
{
    // (the LDS address is the same in all lanes; lane i's bytes go to it + 16 i)
    auto* dst = reinterpret_cast<__attribute__((address_space(3))) uint32_t*>((uintptr_t)lds_off);
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t*)src, dst, 16, 0, 2);      // (2: non-temporal)
}
template <int N>
__device__ __forceinline__ void wait_vm()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

__device__ __forceinline__ void store_row(const PagedAttention& a, int token, int head, const f32x4& o, float m, float l, int d, int g)
{
    const bool some = l != 0.f;              // (0: no key, or none of any weight; NaN, of a logit that is NaN or +inf, stays)
    const float f = some ? 1.f / l : 0.f;
    const long long row = (long long)token * a.n_q_heads + head;
    bf16x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = (__bf16)(some ? o[e] * f : 0.f);
    *reinterpret_cast<bf16x4*>(a.out + row * kHeadDim + 16 * d + 4 * g) = w;
    if (a.lse && d == 0 && g == 0) a.lse[row] = some ? (m + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f : -INFINITY;
}

}  // namespace
}  // namespace mp
