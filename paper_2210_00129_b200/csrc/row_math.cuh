// Rows as 16-byte vectors of bf16 or fp32 numbers, and sums over the threads that share a row.
#pragma once

#include "sbp_common.cuh"

namespace sbp {

template <typename T>
struct Vec;                                           // T numbers in a 16-byte vector
template <>
struct Vec<__nv_bfloat16> {
    static constexpr int N = 8;
    __device__ static __forceinline__ void unpack(const uint4& q, float* f) {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    __device__ static __forceinline__ uint4 pack(const float* f) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 v = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&v);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <>
struct Vec<float> {
    static constexpr int N = 4;
    __device__ static __forceinline__ void unpack(const uint4& q, float* f) {
        f[0] = __uint_as_float(q.x);
        f[1] = __uint_as_float(q.y);
        f[2] = __uint_as_float(q.z);
        f[3] = __uint_as_float(q.w);
    }
    __device__ static __forceinline__ uint4 pack(const float* f) {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
};

// N consecutive fp32 numbers (a multiple of four, 16-byte aligned) that no kernel writes meanwhile
template <int N>
__device__ __forceinline__ void load_f32(const float* p, float* f) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        const float4 v = __ldg(reinterpret_cast<const float4*>(p + i));
        f[i] = v.x;
        f[i + 1] = v.y;
        f[i + 2] = v.z;
        f[i + 3] = v.w;
    }
}

// a row that is read once; not through the read-only path, for the buffer may be written in place by the same thread
__device__ __forceinline__ uint4 ld_row(const uint4* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}

// Sums of V values over a row's threads: one warp, or all the warps of a block (kMulti), through shared memory.  `scratch` holds
// two halves of V floats a warp, taken in turns: a half is written again only after the barrier of the sum between, by which
// every thread has read it.  The order of additions depends on the number of threads alone.
template <int V, bool kMulti>
__device__ __forceinline__ void row_sums(float (&v)[V], float* scratch, int warps, int& turn) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    if constexpr (kMulti) {
        float* s = scratch + (turn ? 32 * V : 0);
        turn ^= 1;
        if ((threadIdx.x & 31) == 0) {
#pragma unroll
            for (int i = 0; i < V; ++i) s[(threadIdx.x >> 5) * V + i] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = 0.f;
        for (int w = 0; w < warps; ++w)
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] += s[w * V + i];
    }
}

}  // namespace sbp
