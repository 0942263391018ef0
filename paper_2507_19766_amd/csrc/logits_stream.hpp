// What every kernel that streams rows of logits shares: how a 16-byte vector of either storage type maps to fp32 values,
// streaming loads and stores, the grid over rows, and the host's checks of a logits argument.
#ifndef ULORL_LOGITS_STREAM_HPP
#define ULORL_LOGITS_STREAM_HPP

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ulorl.h"

namespace ulorl_detail {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kEmpty = -1.0e30f;  // "no element seen yet"; finite so that 0 * kEmpty == 0
// Kernels with several workgroups per row lay the rows over grid dimensions y (up to
// kRowsPerGridY) and z (up to 65535).
constexpr int64_t kRowsPerGridY = 32768;
constexpr int64_t kMaxRows = kRowsPerGridY * 65535;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ u32x4 load_stream(const u32x4* p) { return __builtin_nontemporal_load(p); }
__device__ __forceinline__ void store_stream(u32x4* p, u32x4 v) { __builtin_nontemporal_store(v, p); }

// ---------------------------------------------------------------------------------------------
// storage traits: how a 16-byte vector maps to fp32 values
// ---------------------------------------------------------------------------------------------
struct StoreBF16 {
    using elem = uint16_t;
    static constexpr int kPerVec = 8;
    static __device__ __forceinline__ void unpack(u32x4 v, float* f)
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            f[2 * k] = __uint_as_float(v[k] << 16);
            f[2 * k + 1] = __uint_as_float(v[k] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ uint32_t pack2(float lo, float hi)
    {
        f32x2 x = {lo, hi};
        bf16x2 b = __builtin_convertvector(x, bf16x2);  // round-to-nearest-even pair convert
        return __builtin_bit_cast(uint32_t, b);
    }
    static __device__ __forceinline__ u32x4 pack(const float* f)
    {
        u32x4 v;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = pack2(f[2 * k], f[2 * k + 1]);
        return v;
    }
    static __device__ __forceinline__ float load1(const elem* p) { return __uint_as_float(((uint32_t)*p) << 16); }
    static __device__ __forceinline__ void store1(elem* p, float x) { *p = (elem)(pack2(x, 0.0f) & 0xffffu); }
    // a vector of -9.95e29 (bf16 0xF149), used as padding that contributes nothing to a row's sums
    static __device__ __forceinline__ u32x4 filler() { return u32x4{0xf149f149u, 0xf149f149u, 0xf149f149u, 0xf149f149u}; }
    static __device__ __forceinline__ u32x4 sign_bits() { return u32x4{0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u}; }
};

struct StoreF32 {
    using elem = float;
    static constexpr int kPerVec = 4;
    static __device__ __forceinline__ void unpack(u32x4 v, float* f)
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) f[k] = __uint_as_float(v[k]);
    }
    static __device__ __forceinline__ u32x4 pack(const float* f)
    {
        u32x4 v;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = __float_as_uint(f[k]);
        return v;
    }
    static __device__ __forceinline__ float load1(const elem* p) { return *p; }
    static __device__ __forceinline__ void store1(elem* p, float x) { *p = x; }
    static __device__ __forceinline__ u32x4 filler()
    {
        const uint32_t b = __float_as_uint(kEmpty);
        return u32x4{b, b, b, b};
    }
    static __device__ __forceinline__ u32x4 sign_bits() { return u32x4{0x80000000u, 0x80000000u, 0x80000000u, 0x80000000u}; }
};

inline bool shape_ok(int64_t N, int64_t V, int64_t stride)
{
    return N > 0 && N <= kMaxRows && V > 0 && V <= 0x7fffffffLL && stride >= V;
}

inline int32_t check_logits(const void* logits, int32_t dt, int64_t N, int64_t V, int64_t stride)
{
    if (!logits) return ULORL_ERR_NULL;
    if (dt != ULORL_F32 && dt != ULORL_BF16) return ULORL_ERR_DTYPE;
    if (!shape_ok(N, V, stride)) return ULORL_ERR_SHAPE;
    const size_t esz = dt == ULORL_F32 ? 4 : 2;
    if (((uintptr_t)logits & 15u) != 0 || ((size_t)stride * esz) % 16 != 0) return ULORL_ERR_ALIGN;
    return ULORL_OK;
}

inline dim3 rows_grid(unsigned x, int64_t N)
{
    return dim3(x, (unsigned)(N < kRowsPerGridY ? N : kRowsPerGridY), (unsigned)((N + kRowsPerGridY - 1) / kRowsPerGridY));
}

}  // namespace ulorl_detail

#endif
