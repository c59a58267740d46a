// Rows of fp32, fp16 and bf16 values as the layer operators read and write them.
//
// A thread handles packs of V consecutive values of a row: 16 bytes (V = 4 or 8) where every row of every operand starts on a
// 16-byte boundary and its length is whole packs, single values (V = 1) otherwise.  Arithmetic is in fp32; results are rounded
// once, to nearest even, when they are stored.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "async.cuh"
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

// ---- one fp32 value, or two that one instruction works on (V > 1): the kernels' arithmetic is half their instructions
struct F1 {
    float v;
};
struct F2 {
    unsigned long long v;
};
template <int V>
using Num = typename std::conditional<V == 1, F1, F2>::type;
template <int V>
constexpr int kNums = V == 1 ? 1 : V / 2;

__device__ __forceinline__ F1 mul(F1 a, F1 b) { return F1{a.v * b.v}; }
__device__ __forceinline__ F1 add(F1 a, F1 b) { return F1{a.v + b.v}; }
__device__ __forceinline__ F1 fma(F1 a, F1 b, F1 c) { return F1{fmaf(a.v, b.v, c.v)}; }
__device__ __forceinline__ float total(F1 a) { return a.v; }
__device__ __forceinline__ F2 mul(F2 a, F2 b) { return F2{mul2(a.v, b.v)}; }
__device__ __forceinline__ F2 add(F2 a, F2 b) { return F2{add2(a.v, b.v)}; }
__device__ __forceinline__ F2 fma(F2 a, F2 b, F2 c) {
    fma2(c.v, a.v, b.v);
    return c;
}
__device__ __forceinline__ float total(F2 a) {
    float x, y;
    unpack2(a.v, x, y);
    return x + y;
}
template <typename N>
__device__ __forceinline__ N splat(float x) {
    if constexpr (std::is_same<N, F1>::value) return F1{x};
    else return F2{pack2(x, x)};
}
// f applied to each value
template <typename F>
__device__ __forceinline__ F1 each(F1 a, F f) { return F1{f(a.v)}; }
template <typename F>
__device__ __forceinline__ F2 each(F2 a, F f) {
    float x, y;
    unpack2(a.v, x, y);
    return F2{pack2(f(x), f(y))};
}

template <typename T>
__device__ __forceinline__ F2 pair_of(uint32_t w) {
    if constexpr (std::is_same<T, __half>::value) {
        const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&w));
        return F2{pack2(t.x, t.y)};
    } else {
        return F2{pack2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u))};
    }
}
// V values of type T at a shared-memory address (16-byte aligned if V > 1); with CHECK zeros unless column < columns.  Predicates and not branches, here and
// in write_global, and the comparison beside them: a branch for each pack costs more than the pack's arithmetic.
template <typename T, int V, bool CHECK>
__device__ __forceinline__ void read_shared(uint32_t at, int column, int columns, Num<V> (&f)[kNums<V>]) {
    if constexpr (!CHECK) {
        static_assert(V > 1, "single values are checked");
        if constexpr (sizeof(T) == 4) {
            asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(f[0].v), "=l"(f[1].v) : "r"(at) : "memory");
        } else {
            uint32_t w[4];
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] = pair_of<T>(w[i]);
        }
    } else if constexpr (V == 1 && sizeof(T) == 4) {
        asm volatile("{\n\t.reg .pred p;\n\tsetp.lt.s32 p, %2, %3;\n\tmov.f32 %0, 0f00000000;\n\t@p ld.shared.f32 %0, [%1];\n\t}" : "=f"(f[0].v) : "r"(at), "r"(column), "r"(columns) : "memory");
    } else if constexpr (V == 1) {
        unsigned short u;
        asm volatile("{\n\t.reg .pred p;\n\tsetp.lt.s32 p, %2, %3;\n\tmov.u16 %0, 0;\n\t@p ld.shared.u16 %0, [%1];\n\t}" : "=h"(u) : "r"(at), "r"(column), "r"(columns) : "memory");
        f[0].v = to_float(*reinterpret_cast<const T*>(&u));
    } else if constexpr (sizeof(T) == 4) {
        asm volatile("{\n\t.reg .pred p;\n\tsetp.lt.s32 p, %3, %4;\n\tmov.b64 %0, 0;\n\tmov.b64 %1, 0;\n\t@p ld.shared.v2.b64 {%0, %1}, [%2];\n\t}"
                     : "=l"(f[0].v), "=l"(f[1].v) : "r"(at), "r"(column), "r"(columns) : "memory");
    } else {
        uint32_t w[4];
        asm volatile("{\n\t.reg .pred p;\n\tsetp.lt.s32 p, %5, %6;\n\tmov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\tmov.b32 %3, 0;\n\t@p ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];\n\t}"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at), "r"(column), "r"(columns) : "memory");
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = pair_of<T>(w[i]);
    }
}
// V fp32 values at a shared-memory address
template <int V>
__device__ __forceinline__ void read_shared_params(uint32_t at, Num<V> (&f)[kNums<V>]) {
    if constexpr (V == 1) {
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(f[0].v) : "r"(at) : "memory");
    } else {
#pragma unroll
        for (int i = 0; i < V / 2; i += 2) asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(f[i].v), "=l"(f[i + 1].v) : "r"(at + 8 * i) : "memory");
    }
}
// V values of type T in global memory that other rows use too
template <typename T, int V>
__device__ __forceinline__ void read_global(const T* p, Num<V> (&f)[kNums<V>]) {
    if constexpr (V == 1) {
        f[0].v = to_float(*p);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < V / 2; i += 2) {
            const ulonglong2 t = __ldg(reinterpret_cast<const ulonglong2*>(p + 2 * i));
            f[i].v = t.x;
            f[i + 1].v = t.y;
        }
    } else {
        const uint4 t = __ldg(reinterpret_cast<const uint4*>(p));
        f[0] = pair_of<T>(t.x); f[1] = pair_of<T>(t.y); f[2] = pair_of<T>(t.z); f[3] = pair_of<T>(t.w);
    }
}
// V values at p + column, if column < columns.
template <typename T, int V>
__device__ __forceinline__ void write_global(T* p, int column, int columns, const Num<V> (&n)[kNums<V>]) {
    T* const at = p + column;
    if constexpr (V == 1) {
        T v;
        from_float(v, n[0].v);
        if constexpr (sizeof(T) == 4) {
            asm volatile("{\n\t.reg .pred p;\n\tsetp.lt.s32 p, %2, %3;\n\t@p st.global.f32 [%0], %1;\n\t}" ::"l"(at), "f"(n[0].v), "r"(column), "r"(columns) : "memory");
        } else {
            asm volatile("{\n\t.reg .pred p;\n\tsetp.lt.s32 p, %2, %3;\n\t@p st.global.u16 [%0], %1;\n\t}" ::"l"(at), "h"(*reinterpret_cast<const unsigned short*>(&v)), "r"(column), "r"(columns) : "memory");
        }
    } else if constexpr (sizeof(T) == 4) {
        asm volatile("{\n\t.reg .pred p;\n\tsetp.lt.s32 p, %3, %4;\n\t@p st.global.v2.b64 [%0], {%1, %2};\n\t}" ::"l"(at), "l"(n[0].v), "l"(n[1].v), "r"(column), "r"(columns) : "memory");
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x, y;
            unpack2(n[i].v, x, y);
            if constexpr (std::is_same<T, __half>::value) {
                const __half2 h = __floats2half2_rn(x, y);
                w[i] = *reinterpret_cast<const uint32_t*>(&h);
            } else {
                const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
                w[i] = *reinterpret_cast<const uint32_t*>(&h);
            }
        }
        asm volatile("{\n\t.reg .pred p;\n\tsetp.lt.s32 p, %5, %6;\n\t@p st.global.v4.b32 [%0], {%1, %2, %3, %4};\n\t}"
                     ::"l"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(column), "r"(columns) : "memory");
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
    __device__ __forceinline__ void sync() const {
        if constexpr (SIZE == 0) __syncthreads();
        else __syncwarp();
    }
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

// ---- rows on their way to shared memory -------------------------------------------------------------------------------
// An operand whose rows are staged.
struct RowOperand {
    const char* at;
    int64_t ld;                     // bytes from one row to the next
};
constexpr int kMostOperands = 5;
struct RowOperands {
    RowOperand o[kMostOperands];
    int n;
    int row_bytes;
    int slot_bytes;                 // of shared memory for a row of an operand: a multiple of 16
    int stages;                     // rows of a team in shared memory: 2, the next one on its way, or 1
};

// The rows of a team, copied by the asynchronous copy engine: one thread asks for a whole row of each operand and no thread of the team spends
// an instruction on it.  Copies are whole 16-byte units, rounded outwards where a row does not start or end on one.  Every wait is
// bounded; a row whose copies do not arrive in time is marked by the caller.
template <typename T, int SIZE>
struct RowPipe {
    const RowOperands& r;
    uint32_t slots, bars;           // this team's
    __device__ __forceinline__ RowPipe(const RowOperands& operands, uint32_t smem, uint32_t barriers, int team)
        : r(operands), slots(smem + team * operands.stages * operands.n * operands.slot_bytes), bars(barriers + 16 * team) {}
    // One thread of the team, before the first use (and a barrier of the CTA in between).
    __device__ __forceinline__ void open() const {
        async::mbar_init(bars, r.n);
        async::mbar_init(bars + 8, r.n);
        async::fence_barrier_init();
    }
    __device__ __forceinline__ uint32_t slot(int stage, int o) const { return slots + (stage * r.n + o) * r.slot_bytes; }
    // The team's first threads, an operand each; all of the team is done with what the stage held.
    __device__ __forceinline__ void fetch(int stage, int64_t row, const Team<SIZE>& team) const {
        for (int o = team.rank(); o < r.n; o += team.size()) {
            const char* const p = r.o[o].at + row * r.o[o].ld;
            const uint32_t off = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p)) & 15u, bytes = (off + r.row_bytes + 15u) & ~15u;
            async::mbar_arrive_expect_tx(bars + 8 * stage, bytes);
            async::bulk_load_1d(slot(stage, o), p - off, bytes, bars + 8 * stage);
        }
    }
    // Turn t of the team; false if the copies have not arrived within the limit.
    __device__ __forceinline__ bool wait(int turn) const {
        const int stage = r.stages == 2 ? turn & 1 : 0;
        const uint32_t bar = bars + 8 * stage, parity = (r.stages == 2 ? turn >> 1 : turn) & 1;
        if (async::mbar_try_wait(bar, parity)) return true;
        const unsigned long long t0 = async::global_ns();
        while (!async::mbar_try_wait(bar, parity))
            if (async::global_ns() - t0 > async::kWaitLimitNs) return false;
        return true;
    }
    // After a wait that gave up: the copies in flight land before the CTA leaves (bounded again).
    __device__ __forceinline__ void drain() const {
        for (int i = 0; i < 2 * r.stages; ++i) async::mbar_wait_quiet(bars + 8 * (i >> 1), i & 1);
    }
    // Address of the row's first value (V > 1: it is aligned).
    template <int V>
    __device__ __forceinline__ uint32_t row_at(int stage, int o, int64_t row) const {
        const uint32_t s = slot(stage, o);
        if constexpr (V > 1) return s;
        else return s + (static_cast<uint32_t>(reinterpret_cast<uintptr_t>(r.o[o].at + row * r.o[o].ld)) & 15u);
    }
};
// Bytes of a slot: whole packs of all threads, so that what lies beyond the row can be zeros; single values: the row and what rounding adds.
__host__ __device__ inline int slot_bytes_of(int row_bytes, int team_threads, int per_thread, int size, bool packs) {
    return packs ? team_threads * per_thread * size : (row_bytes + 30 + 15) / 16 * 16;
}

// 8-bit integers of a row whose largest magnitude has these bits (compared as an integer, so that a NaN is the largest of all): value =
// integer * scale, integer = rint(value * inverse).  A row of magnitudes below 2^-100 counts as zeros: 127 / top leaves the range of fp32 below 2^-121 and
// top / 127 its normal numbers below 2^-119, and the border keeps some distance from both.  One with an infinity or a NaN has a scale that is not finite either, and integers of no meaning.
struct RowScale {
    float scale, inverse;
};
__device__ __forceinline__ RowScale row_scale(uint32_t top_bits) {
    const float top = __uint_as_float(top_bits);
    if (top < 7.8886090522101181e-31f) return RowScale{0.f, 0.f};
    return RowScale{__fdiv_rn(top, 127.f), __fdiv_rn(127.f, top)};
}
// The integer is in the low bits of the sum with 1.5 * 2^23, whose last place is one: two full-rate operations, each rounded as the definition says, in place
// of a conversion at a quarter of the rate.
__device__ __forceinline__ uint32_t quantised(float v, float inverse) { return __float_as_uint(__fadd_rn(__fmul_rn(v, inverse), 12582912.f)); }
__device__ __forceinline__ uint32_t magnitude_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

template <int V>
__device__ __forceinline__ void store_quantised(int8_t* p, const float (&f)[V], float inverse) {
    if constexpr (V == 1) {
        *p = static_cast<int8_t>(quantised(f[0], inverse));
    } else {
        uint32_t w[V / 4];
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            const uint32_t lo = __byte_perm(quantised(f[i], inverse), quantised(f[i + 1], inverse), 0x0040);
            const uint32_t hi = __byte_perm(quantised(f[i + 2], inverse), quantised(f[i + 3], inverse), 0x0040);
            w[i / 4] = __byte_perm(lo, hi, 0x5410);
        }
        if constexpr (V == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t*>(p) = w[0];
    }
}

}  // namespace layers
}  // namespace cutoff
