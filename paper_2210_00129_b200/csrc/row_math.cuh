// Rows as 16-byte vectors of bf16 or fp32 numbers, and sums over the threads that share a row.
#pragma once

#include "sbp_common.cuh"

namespace sbp {

// Two fp32 numbers in a register pair, for the instructions that work on both.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair(float lo, float hi) {
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 both(f32x2 v) {
    float2 f;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(v));
    return f;
}
__device__ __forceinline__ f32x2 add(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 mul(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 fma(f32x2 a, f32x2 b, f32x2 c) {
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

template <typename T>
struct Vec;                                           // T numbers in a 16-byte vector
template <>
struct Vec<__nv_bfloat16> {
    static constexpr int N = 8;
    __device__ static __forceinline__ void unpack(const uint4& q, f32x2* f) {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = pair(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
    }
    __device__ static __forceinline__ uint4 pack(const f32x2* f) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 x = both(f[i]);
            const __nv_bfloat162 v = __floats2bfloat162_rn(x.x, x.y);
            w[i] = *reinterpret_cast<const uint32_t*>(&v);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <>
struct Vec<float> {
    static constexpr int N = 4;
    __device__ static __forceinline__ void unpack(const uint4& q, f32x2* f) {
        f[0] = pair(__uint_as_float(q.x), __uint_as_float(q.y));
        f[1] = pair(__uint_as_float(q.z), __uint_as_float(q.w));
    }
    __device__ static __forceinline__ uint4 pack(const f32x2* f) {
        const float2 a = both(f[0]), b = both(f[1]);
        return make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
    }
};

// N consecutive fp32 numbers (a multiple of four, 16-byte aligned) that no kernel writes meanwhile
template <int N>
__device__ __forceinline__ void load_f32(const float* p, f32x2* f) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) Vec<float>::unpack(__ldg(reinterpret_cast<const uint4*>(p) + i), f + 2 * i);
}

// The threads that share a row: kLanes (8, 16 or 32) of a warp, or, kLanes 0, `warps` warps of a block, which meet at barrier `id`
// and add up through `scratch`: two halves of 32 float4, taken in turns - a half is written again only after the barrier of
// the sum between, by which every thread has read it.
template <int kLanes>
struct RowThreads {
    static constexpr bool kMulti = kLanes == 0;
    static constexpr int kHalf = 32;                  // float4 of half of `scratch`: 16 warps of eight values
    int t, count;                                     // this thread, of how many
    int warps, id, turn;
    float4* scratch;
    __device__ __forceinline__ int threads() const { return kMulti ? count : kLanes; }

    // Sums of V <= 8 values over those threads, in an order that depends on their number alone.  Several values over 32 lanes: the first
    // exchanges halve what a lane carries, so that 4 or 8 values take 6 or 9 of them.
    template <int V>
    __device__ __forceinline__ void sums(float (&v)[V]) {
        const int lane = threadIdx.x & 31;
        if constexpr (V == 1 || (!kMulti && kLanes < 32)) {
#pragma unroll
            for (int o = (kMulti ? 32 : kLanes) / 2; o > 0; o >>= 1)
#pragma unroll
                for (int i = 0; i < V; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
            if constexpr (!kMulti) return;
        }
        constexpr int kSlots = V > 4 ? 8 : 4, kEach = 32 / kSlots;   // lanes kEach i .. come to hold the sum of value i
        float s = v[0];
        if constexpr (V > 1) {
            float f[kSlots];
#pragma unroll
            for (int i = 0; i < kSlots; ++i) f[i] = i < V ? v[i < V ? i : 0] : 0.f;
#pragma unroll
            for (int n = kSlots / 2, o = 16; n > 0; n /= 2, o /= 2) {
                const bool upper = lane & o;
#pragma unroll
                for (int i = 0; i < n; ++i) {
                    const float send = upper ? f[i] : f[i + n], keep = upper ? f[i + n] : f[i];
                    f[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
                }
            }
            s = f[0];
#pragma unroll
            for (int o = kEach / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        }
        if constexpr (!kMulti) {
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = __shfl_sync(0xffffffffu, s, kEach * i);
        } else {
            constexpr int kQuads = kSlots / 4;
            float4* half = scratch + (turn ? kHalf : 0);
            turn ^= 1;
            if (lane % kEach == 0) reinterpret_cast<float*>(half + (t >> 5) * kQuads)[lane / kEach] = s;       // (V == 1: the sum four times)
            asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(count) : "memory");
            float4 f[kQuads];
#pragma unroll
            for (int i = 0; i < kQuads; ++i) f[i] = half[i];
            auto more = [&](int w) {
#pragma unroll
                for (int i = 0; i < kQuads; ++i) {
                    const float4 q = half[w * kQuads + i];
                    f[i].x += q.x;
                    f[i].y += q.y;
                    f[i].z += q.z;
                    f[i].w += q.w;
                }
            };
            if (warps > 1) more(1);
            if (warps > 2) more(2);
            if (warps > 3) more(3);
            for (int w = 4; w < warps; ++w) more(w);
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = i % 4 == 0 ? f[i / 4].x : i % 4 == 1 ? f[i / 4].y : i % 4 == 2 ? f[i / 4].z : f[i / 4].w;
        }
    }
};

}  // namespace sbp
