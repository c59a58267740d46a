// Products of 8-bit integers with a scale per row of either operand:
//
//   y[i][j] = (sum over k of a[i][k] b[j][k]) * a_scale[i] * b_scale[j] + bias[j]
//
// The sums are exact (32-bit integers, at most 131072 products of magnitudes up to 128), so no split or order of them changes a result; they are
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
constexpr int kQuantizeThreads = 256;

// A CTA per row.  The row is read twice; the second time it is in the L1 or L2.
template <typename T, int V>
__global__ void __launch_bounds__(kQuantizeThreads) k_quantize_rows(QuantizeArgs a) {
    __shared__ __align__(16) float scratch[Team<0>::kScratch];
    Team<0> team(scratch);
    const T* const x = static_cast<const T*>(a.x) + blockIdx.x * a.x_ld;
    int8_t* const q = a.q + blockIdx.x * a.q_ld;
    dependency_wait();
    uint32_t top = 0;
    for (int c = threadIdx.x * V; c < a.cols; c += kQuantizeThreads * V) {
        float f[V];
        unpack(load_pack<T, V>(x + c), f);
#pragma unroll
        for (int i = 0; i < V; ++i) top = max(top, magnitude_bits(f[i]));
    }
    const RowScale s = row_scale(team.top(top));
    launch_dependents();
    if (threadIdx.x == 0) a.scale[blockIdx.x] = s.scale;
    for (int c = threadIdx.x * V; c < a.cols; c += kQuantizeThreads * V) {
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

// Few rows of a: a warp per row of b, which its lanes read 16 bytes at a time, for MT rows of a.
constexpr int kDotWarps = 4;
template <typename T, int MT>
__global__ void __launch_bounds__(kDotWarps * 32) k_product_dot(ProductArgs p) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int j = blockIdx.x * kDotWarps + warp;
    const int64_t i0 = static_cast<int64_t>(blockIdx.y) * MT;
    if (j >= p.n) return;
    const int8_t* const b = p.b + static_cast<int64_t>(j) * p.b_ld;
    int sum[MT] = {};
    dependency_wait();
    for (int c = lane * 16; c < p.k; c += 512) {
        int4 w = *reinterpret_cast<const int4*>(b + c);
        const int left = p.k - c;                // bytes beyond the row count as zeros on this side
        if (left < 16) {
            int* const v = &w.x;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int bytes = min(max(left - 4 * i, 0), 4);
                v[i] = bytes == 4 ? v[i] : v[i] & ((1 << 8 * bytes) - 1);
            }
        }
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            if (i0 + t >= p.m) break;
            const int4 v = *reinterpret_cast<const int4*>(p.a + (i0 + t) * p.a_ld + c);
            sum[t] = __dp4a(v.x, w.x, __dp4a(v.y, w.y, __dp4a(v.z, w.z, __dp4a(v.w, w.w, sum[t]))));
        }
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int total = __reduce_add_sync(0xffffffffu, sum[t]);
        if (lane == 0 && i0 + t < p.m)
            from_float(static_cast<T*>(p.y)[(i0 + t) * p.y_ld + j],
                       fmaf(static_cast<float>(total) * p.a_scale[i0 + t], p.b_scale[j], p.bias ? p.bias[j] : 0.f));
    }
}

}  // namespace layers
}  // namespace cutoff
