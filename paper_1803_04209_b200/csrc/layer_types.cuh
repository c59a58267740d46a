// Rows of fp32, fp16 and bf16 values as the layer operators read and write them.
//
// A thread handles packs of V consecutive values of a row: 16 bytes (V = 4 or 8) where every row of every operand starts on a
// 16-byte boundary and its length is whole packs, single values (V = 1) otherwise.  Arithmetic is in fp32; results are rounded
// once, to nearest even, when they are stored.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"

namespace cutoff {
namespace layers {

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void from_float(float& d, float v) { d = v; }
__device__ __forceinline__ void from_float(__half& d, float v) { d = __float2half_rn(v); }
__device__ __forceinline__ void from_float(__nv_bfloat16& d, float v) { d = __float2bfloat16_rn(v); }

template <typename T>
constexpr int kPack = 16 / static_cast<int>(sizeof(T));

template <typename T, int V>
struct alignas(sizeof(T) * V) Pack {
    T v[V];
};

// Values that are read once: they leave the L1 to the parameters that every row uses.
template <typename T, int V>
__device__ __forceinline__ Pack<T, V> load_pack(const T* p) {
    Pack<T, V> r;
    if constexpr (sizeof(r) == 16) {
        uint4 u;
        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "l"(p) : "memory");
        r = *reinterpret_cast<Pack<T, V>*>(&u);
    } else {
        static_assert(V == 1, "whole packs or single values");
        r.v[0] = *p;
    }
    return r;
}
template <typename T, int V>
__device__ __forceinline__ Pack<T, V> zero_pack() {
    Pack<T, V> r;
#pragma unroll
    for (int i = 0; i < V; ++i) from_float(r.v[i], 0.f);
    return r;
}

template <typename T, int V>
__device__ __forceinline__ void unpack(const Pack<T, V>& r, float (&f)[V]) {
    if constexpr (V == 1 || sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = to_float(r.v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            float2 t;
            if constexpr (std::is_same<T, __half>::value) t = __half22float2(*reinterpret_cast<const __half2*>(&r.v[i]));
            else t = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&r.v[i]));
            f[i] = t.x;
            f[i + 1] = t.y;
        }
    }
}
template <typename T, int V>
__device__ __forceinline__ void store_pack(T* p, const float (&f)[V]) {
    if constexpr (V == 1) {
        from_float(*p, f[0]);
    } else if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
    } else {
        Pack<T, V> r;
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            if constexpr (std::is_same<T, __half>::value) *reinterpret_cast<__half2*>(&r.v[i]) = __floats2half2_rn(f[i], f[i + 1]);
            else *reinterpret_cast<__nv_bfloat162*>(&r.v[i]) = __floats2bfloat162_rn(f[i], f[i + 1]);
        }
        *reinterpret_cast<uint4*>(p) = *reinterpret_cast<uint4*>(&r);
    }
}

// V parameters (fp32, used by every row) from column c on; `other` where there are none.
template <int V>
__device__ __forceinline__ void load_params(const float* p, int c, float other, float (&f)[V]) {
    if (p == nullptr) {
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = other;
    } else if constexpr (V % 4 == 0) {
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            const float4 t = __ldg(reinterpret_cast<const float4*>(p + c + i));
            f[i] = t.x; f[i + 1] = t.y; f[i + 2] = t.z; f[i + 3] = t.w;
        }
    } else {
        f[0] = __ldg(p + c);
    }
}

// The threads that share a row: SIZE lanes of a warp, or (SIZE = 0) a whole CTA.  sum() adds N values over them, in an order that
// depends on nothing but the number of threads, and every thread gets the same bits.
template <int SIZE>
struct Team {
    static constexpr int kMostSums = 2;
    static constexpr int kScratch = 2 * kMostSums * 32;
    float* scratch;                 // CTA: [2][kMostSums][32 warps], 16-byte aligned
    uint32_t parity = 0;
    __device__ __forceinline__ explicit Team(float* s) : scratch(s) {
        if constexpr (SIZE == 0) {
            for (int i = threadIdx.x; i < kScratch; i += blockDim.x) s[i] = 0.f;
            __syncthreads();
        }
    }
    __device__ __forceinline__ int size() const { return SIZE ? SIZE : blockDim.x; }
    __device__ __forceinline__ int rank() const { return SIZE ? threadIdx.x % SIZE : threadIdx.x; }

    template <int N>
    __device__ __forceinline__ void sum(float (&v)[N]) {
        static_assert(N <= kMostSums, "scratch");
        constexpr int kFirst = (SIZE ? SIZE : 32) / 2;
#pragma unroll
        for (int d = kFirst; d; d >>= 1)
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], d);
        if constexpr (SIZE == 0) {
            const int warps = blockDim.x >> 5;
            if (warps == 1) return;
            float* const s = scratch + parity * 32 * kMostSums;     // the other half may still be read: one barrier is enough
            parity ^= 1u;
            if ((threadIdx.x & 31) == 0)
#pragma unroll
                for (int i = 0; i < N; ++i) s[32 * i + (threadIdx.x >> 5)] = v[i];
            __syncthreads();
            // every thread adds all warps' sums, four at a time; what belongs to no warp is zero
#pragma unroll
            for (int i = 0; i < N; ++i) {
                float4 q = *reinterpret_cast<const float4*>(s + 32 * i);
                for (int w = 4; w < warps; w += 4) {
                    const float4 t = *reinterpret_cast<const float4*>(s + 32 * i + w);
                    q.x += t.x; q.y += t.y; q.z += t.z; q.w += t.w;
                }
                v[i] = (q.x + q.y) + (q.z + q.w);
            }
        }
    }
    // The largest of the teams' values, which are compared as unsigned integers.
    __device__ __forceinline__ uint32_t top(uint32_t v) {
        constexpr int kFirst = (SIZE ? SIZE : 32) / 2;
#pragma unroll
        for (int d = kFirst; d; d >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, d));
        if constexpr (SIZE == 0) {
            const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
            if (warps == 1) return v;
            uint32_t* const s = reinterpret_cast<uint32_t*>(scratch) + parity * 32 * kMostSums;
            parity ^= 1u;
            if (lane == 0) s[warp] = v;
            __syncthreads();
            v = __reduce_max_sync(0xffffffffu, lane < warps ? s[lane] : 0u);
        }
        return v;
    }
};

// 8-bit integers of a row whose largest magnitude has these bits (compared as an integer, so that a NaN is the largest of all): value =
// integer * scale, integer = rint(value * inverse).  A row of magnitudes below 2^-100 counts as zeros, because 127 / top would leave the range;
// one with an infinity or a NaN has a scale that is not finite either.
struct RowScale {
    float scale, inverse;
};
__device__ __forceinline__ RowScale row_scale(uint32_t top_bits) {
    const float top = __uint_as_float(top_bits);
    if (top < 7.8886090522101181e-31f) return RowScale{0.f, 0.f};
    return RowScale{__fdiv_rn(top, 127.f), __fdiv_rn(127.f, top)};
}
__device__ __forceinline__ int quantised(float v, float inverse) { return __float2int_rn(__fmul_rn(v, inverse)); }   // a NaN becomes 0
__device__ __forceinline__ uint32_t magnitude_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

template <int V>
__device__ __forceinline__ void store_quantised(int8_t* p, const float (&f)[V], float inverse) {
    if constexpr (V == 1) {
        *p = static_cast<int8_t>(quantised(f[0], inverse));
    } else {
        uint32_t w[V / 4];
#pragma unroll
        for (int i = 0; i < V; i += 4)
            w[i / 4] = (quantised(f[i], inverse) & 0xff) | (quantised(f[i + 1], inverse) & 0xff) << 8 | (quantised(f[i + 2], inverse) & 0xff) << 16 |
                       (quantised(f[i + 3], inverse) & 0xff) << 24;
        if constexpr (V == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t*>(p) = w[0];
    }
}

}  // namespace layers
}  // namespace cutoff
