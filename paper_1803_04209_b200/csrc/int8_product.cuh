// Products of 8-bit integers with a scale per row of either operand:
//
//   y[i][j] = (sum over k of a[i][k] b[j][k]) * a_scale[i] * b_scale[j] + bias[j]
//
// The sums are exact (32-bit integers, at most 131071 products of magnitudes up to 128: 131072 would be 2^31), so no split or order of them changes a result; they are
// scaled in fp32 and rounded once when stored.
//
// k_quantize_rows brings rows of fp32, fp16 or bf16 values into that form.
#pragma once
#include "layer_types.cuh"

namespace cutoff {
namespace layers {

struct QuantizeArgs {
    const void* x;
    int8_t* q;
    float* scale;
    int64_t rows, x_ld, q_ld;
    int cols;
};
constexpr int kQuantizeWarps = 4;                 // rows of a CTA if a warp has one

// A warp (SIZE = 32) or a CTA (SIZE = 0) per row.  Rows of up to four packs per thread stay in registers; longer ones are read a second time, from the L2.
// A CTA for each of 20000 rows of 1024 bf16 values took 66 us; see the launch for the choice.
constexpr int kQuantizeKeep = 4;
template <typename T, int V, int SIZE>
__global__ void __launch_bounds__(512) k_quantize_rows(QuantizeArgs a) {
    __shared__ __align__(16) float scratch[Team<SIZE>::kScratch];
    Team<SIZE> team(scratch);
    const int64_t row = SIZE ? static_cast<int64_t>(blockIdx.x) * kQuantizeWarps + threadIdx.x / 32 : blockIdx.x;
    if (row >= a.rows) return;                    // a whole warp, or nobody
    const T* const x = static_cast<const T*>(a.x) + row * a.x_ld;
    int8_t* const q = a.q + row * a.q_ld;
    const int kStep = team.size() * V, c0 = team.rank() * V;
    dependency_wait();
    launch_dependents();
    Pack<T, V> keep[kQuantizeKeep];
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < kQuantizeKeep; ++k) keep[k] = c0 + k * kStep < a.cols ? load_pack<T, V>(x + c0 + k * kStep) : zero_pack<T, V>();
#pragma unroll
    for (int k = 0; k < kQuantizeKeep; ++k) {
        float f[V];
        unpack(keep[k], f);
#pragma unroll
        for (int i = 0; i < V; ++i) top = max(top, magnitude_bits(f[i]));
    }
#pragma unroll 4
    for (int c = c0 + kQuantizeKeep * kStep; c < a.cols; c += kStep) {
        float f[V];
        unpack(load_pack<T, V>(x + c), f);
#pragma unroll
        for (int i = 0; i < V; ++i) top = max(top, magnitude_bits(f[i]));
    }
    const RowScale s = row_scale(team.top(top));
    if (team.rank() == 0) a.scale[row] = s.scale;
#pragma unroll
    for (int k = 0; k < kQuantizeKeep; ++k) {
        float f[V];
        unpack(keep[k], f);
        if (c0 + k * kStep < a.cols) store_quantised<V>(q + c0 + k * kStep, f, s.inverse);
    }
#pragma unroll 4
    for (int c = c0 + kQuantizeKeep * kStep; c < a.cols; c += kStep) {
        float f[V];
        unpack(load_pack<T, V>(x + c), f);
        store_quantised<V>(q + c, f, s.inverse);
    }
}

struct ProductArgs {
    const int8_t *a, *b;
    const float *a_scale, *b_scale, *bias;       // bias: or null
    void* y;
    int64_t m, a_ld, b_ld, y_ld;
    int n, k;
};

// One result: the same steps in the same order in every kernel.
__device__ __forceinline__ float scaled(int total, float a_scale, float b_scale, float bias) { return fmaf(static_cast<float>(total) * a_scale, b_scale, bias); }

// One row of a: a warp per row of b, which its lanes read 16 bytes at a time.
constexpr int kDotWarps = 4;
template <typename T>
__global__ void __launch_bounds__(kDotWarps * 32) k_product_dot(ProductArgs p) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int j = blockIdx.x * kDotWarps + warp;
    dependency_wait();
    if (j >= p.n) return;
    const int8_t* const b = p.b + static_cast<int64_t>(j) * p.b_ld;
    const float a_scale = p.a_scale[0], b_scale = p.b_scale[j], bias = p.bias ? p.bias[j] : 0.f;
    int sum = 0;
    const int whole = p.k & ~15;
#pragma unroll 8                                   // loads that wait for nothing
    for (int c = lane * 16; c < whole; c += 512) {
        int4 w;
        asm volatile("ld.global.L1::no_allocate.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "l"(b + c));
        const int4 v = *reinterpret_cast<const int4*>(p.a + c);
        sum = __dp4a(v.x, w.x, __dp4a(v.y, w.y, __dp4a(v.z, w.z, __dp4a(v.w, w.w, sum))));
    }
    if (whole + lane < p.k) sum += static_cast<int>(p.a[whole + lane]) * b[whole + lane];       // at most 15 values behind the last chunk
    const int total = __reduce_add_sync(0xffffffffu, sum);
    if (lane == 0) from_float(static_cast<T*>(p.y)[j], scaled(total, a_scale, b_scale, bias));
}

}  // namespace layers
}  // namespace cutoff
