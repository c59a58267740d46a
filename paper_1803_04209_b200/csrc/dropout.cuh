// Dropout whose mask is a function of (seed, step, stream, row, column) and is never stored:
//
//   y[i][j] = residual[i][j] + (bits(i, j) >= T ? x[i][j] * 65536 / (65536 - T) : 0),   T = round(65536 p)
//
// bits(i, j) are 16 of the 128 bits of Philox4x32-10 at counter (j / 8, row of i, stream, step): word (j % 8) / 2, its low half for
// even j.  The gradient with respect to x is the same map of the gradient of y.
//
// A thread owns eight consecutive columns, one generator call, and walks down the rows, so that what the first rounds compute from
// the column alone is computed once per thread (philox_column): the ten rounds are the longest part of the instructions, and 16 bits
// per value instead of 32 halve them.
//
// What bounds it is the memory, and next to it the issue slots (some fifteen instructions per value): 16384 x 4096 bf16 with a residual 72 us, 0.40 GB, 85 %
// of a copy's rate; 8001 x 2175 fp32, rows that are not aligned, 26 us (81 %).  Two rows of a thread at a time with bounds checks on each took 96 and 33.
#pragma once
#include "layer_types.cuh"
#include "rng.cuh"

namespace cutoff {
namespace layers {

struct DropoutArgs {
    const void* x;
    const void* residual;          // or null
    void* y;
    int64_t rows, x_ld, residual_ld, y_ld;
    int cols, tiles;               // tiles: groups of LX * 8 columns
    uint32_t first_row, stream, step;
    NoiseKey key;
    uint32_t border;               // T << 16; a half-word h is kept where h << 16 >= border
    uint32_t word_mask;            // 0 if everything is dropped (T = 65536), else all ones
    float scale;
};

constexpr int kDropoutThreads = 256;

// LX: lanes that share a row (each with eight columns), 32 / LX rows per warp.  V: values per access.  U: rows of a thread on their way at a time.
// ADD: there is a residual.
template <typename T, int V, int LX, int U, bool ADD>
__global__ void __launch_bounds__(kDropoutThreads, 3) k_dropout(DropoutArgs a) {
    constexpr int kRowsPerWarp = 32 / LX;
    const int lane = threadIdx.x & 31, l = lane % LX;
    const int64_t warp = (static_cast<int64_t>(blockIdx.x) * kDropoutThreads + threadIdx.x) >> 5, warps = static_cast<int64_t>(gridDim.x) * (kDropoutThreads / 32);
    const int tile = static_cast<int>(warp % a.tiles);
    const int64_t each = warps / a.tiles;                 // warps that share a tile of columns; those left over have nothing to do
    if (warp >= each * a.tiles) return;
    const int64_t stride = each * kRowsPerWarp;
    const int c0 = (tile * LX + l) * 8;                   // this lane's columns, as the generator counts them
    const uint4 column = philox_column(static_cast<uint32_t>(c0 >> 3), a.stream, a.step, a.key.seed_lo, a.key.seed_hi);

    // Values of this lane: with whole packs the eight columns from c0; with single values columns l, LX + l, ... of the tile, so that
    // a warp's accesses are consecutive, and the kept bits come from the lanes that drew them.
    constexpr int kPacks = V == 1 ? 8 : 8 / V;
    constexpr int kApart = V == 1 ? LX : V;
    const int first = V == 1 ? tile * LX * 8 + l : c0;
    bool has[kPacks];
#pragma unroll
    for (int k = 0; k < kPacks; ++k) has[k] = first + k * kApart < a.cols;
    const T* const x = static_cast<const T*>(a.x) + first;
    const T* const res = static_cast<const T*>(a.residual) + first;
    T* const y = static_cast<T*>(a.y) + first;

    const auto rows_from = [&](int64_t row0, auto all) {  // all: the U rows are there
        Pack<T, V> in[U][kPacks], add[ADD ? U : 1][kPacks];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t row = row0 + u * stride;
#pragma unroll
            for (int k = 0; k < kPacks; ++k) {
                const bool ok = (decltype(all)::value || row < a.rows) && has[k];
                in[u][k] = ok ? load_pack<T, V>(x + row * a.x_ld + k * kApart) : zero_pack<T, V>();
                if constexpr (ADD) add[u][k] = ok ? load_pack<T, V>(res + row * a.residual_ld + k * kApart) : zero_pack<T, V>();
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t row = row0 + u * stride;
            const Philox4 r = philox_row_column(philox_row(a.first_row + static_cast<uint32_t>(row), a.stream, a.key.seed_lo), column, a.key.seed_lo, a.key.seed_hi);
            const uint32_t w[4] = {r.x & a.word_mask, r.y & a.word_mask, r.z & a.word_mask, r.w & a.word_mask};
            bool keep[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                keep[2 * i] = (w[i] << 16) >= a.border;
                keep[2 * i + 1] = w[i] >= a.border;
            }
            if constexpr (V == 1) {
                uint32_t bits = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) bits |= keep[i] ? 1u << i : 0u;
#pragma unroll
                for (int k = 0; k < 8; ++k) keep[k] = __shfl_sync(0xffffffffu, bits, (k * LX + l) >> 3, LX) >> ((k * LX + l) & 7) & 1u;
            }
#pragma unroll
            for (int k = 0; k < kPacks; ++k) {
                float f[V], g[V];
                unpack(in[u][k], f);
                if constexpr (ADD) {
                    unpack(add[u][k], g);
#pragma unroll
                    for (int i = 0; i < V; ++i) f[i] = keep[k * V + i] ? fmaf(f[i], a.scale, g[i]) : g[i];
                } else {
#pragma unroll
                    for (int i = 0; i < V; ++i) f[i] = keep[k * V + i] ? f[i] * a.scale : 0.f;
                }
                if ((decltype(all)::value || row < a.rows) && has[k]) store_pack<T, V>(y + row * a.y_ld + k * kApart, f);
            }
        }
    };
    // the warp's first row decides for the warp: its shuffles take all lanes
    int64_t row0 = warp / a.tiles * kRowsPerWarp;
    for (; row0 + (U - 1) * stride + kRowsPerWarp <= a.rows; row0 += U * stride) rows_from(row0 + lane / LX, std::true_type{});
    for (; row0 < a.rows; row0 += U * stride) rows_from(row0 + lane / LX, std::false_type{});
}

}  // namespace layers
}  // namespace cutoff
