// What the kernels of block_kernels.hip and block_attn.hip share.
#pragma once
#include "device_util.h"

#define DISPATCH_T(bf16, ...)                                        \
    do {                                                             \
        if (bf16) { typedef bf16_t T; __VA_ARGS__; }                 \
        else { typedef float T; __VA_ARGS__; }                       \
    } while (0)
#define DISPATCH_TK(bf16, kv8, ...)                                   \
    do {                                                              \
        if (kv8) { typedef fp8_t KT; DISPATCH_T(bf16, __VA_ARGS__); } \
        else if (bf16) { typedef bf16_t T; typedef bf16_t KT; __VA_ARGS__; } \
        else { typedef float T; typedef float KT; __VA_ARGS__; }      \
    } while (0)

namespace icarus {
namespace {

template <typename KT> struct Quad;  // four elements as they lie
template <> struct Quad<bf16_t> {
    typedef uint2 raw;
    static __device__ __forceinline__ void get(raw r, float (&v)[4]) {
        v[0] = __uint_as_float(r.x << 16); v[1] = __uint_as_float(r.x & 0xffff0000u);
        v[2] = __uint_as_float(r.y << 16); v[3] = __uint_as_float(r.y & 0xffff0000u);
    }
};
template <> struct Quad<float> {
    typedef float4 raw;
    static __device__ __forceinline__ void get(raw r, float (&v)[4]) { v[0] = r.x; v[1] = r.y; v[2] = r.z; v[3] = r.w; }
};
template <> struct Quad<fp8_t> {
    typedef uint32_t raw;
    static __device__ __forceinline__ void get(raw r, float (&v)[4]) {
        const f32x2_t p = __builtin_amdgcn_cvt_pk_f32_fp8(r, false), q = __builtin_amdgcn_cvt_pk_f32_fp8(r, true);
        v[0] = p[0]; v[1] = p[1]; v[2] = q[0]; v[3] = q[1];
    }
};

}  // namespace
}  // namespace icarus
