// The end of one residual block and the start of the next, in one pass over the rows:
//
//   r = x + scale * act(gate) * post(h),   n = pre(r)
//   post(h) = (h - mean(h)) / sqrt(var(h) + eps) * post_weight + post_bias    (layer; RMS: without the mean; none: h itself)
//
// and the gradients of all of it.  Statistics and sums are fp32, r enters the second norm unrounded; a value is rounded once, where
// it is stored.  The backward pass reads x and h, not r: the parameters' gradients are fp32 sums, and a rounded r would be seen in them.
// It forms the statistics again instead of reading them: the rows are in registers anyway.
//
// A row belongs to a team, 4 to 32 lanes of a warp (rows of up to 512 values) or a CTA.  Forward: one row per team.  Backward:
// each team walks over consecutive rows and keeps the parameters' sums of its columns in registers; k_norm_grad_finish adds the CTAs' sums
// in their order, so that results are the same on every run.
#pragma once
#include "layer_types.cuh"

namespace cutoff {
namespace layers {

enum : int { kNormNone = 0, kNormRms = 1, kNormLayer = 2 };
enum : int { kGateLinear = 0, kGateSigmoid = 1, kGateSilu = 2 };

struct NormArgs {
    const void *x, *h, *gate;                     // h: null = no block before (r = x); gate: null = 1
    const float *scale, *post_w, *post_b, *pre_w, *pre_b;
    int64_t rows, x_ld, h_ld, gate_ld, gate_rows;
    int cols, gate_kind, post, pre;
    float eps, inv_cols;
    // forward
    void *r, *n;                                  // or null
    float* n_scale;                               // not null: n is 8-bit rows with these scales
    int64_t r_ld, n_ld;
};

struct GateValue {
    float a, slope;
};
__device__ __forceinline__ GateValue gate_value(float g, int kind) {
    if (kind == kGateLinear) return GateValue{g, 1.f};
    const float s = __fdividef(1.f, 1.f + __expf(-g));           // exp of a large -g is infinite and s 0
    if (kind == kGateSigmoid) return GateValue{s, s * (1.f - s)};
    return GateValue{g * s, s * (1.f + g * (1.f - s))};
}

// The team's columns: K packs of V values per thread.
template <int SIZE, int V, int K>
struct Columns {
    int cols, at, step;
    __device__ __forceinline__ Columns(const Team<SIZE>& t, int n) : cols(n), at(t.rank() * V), step(t.size() * V) {}
    __device__ __forceinline__ int operator()(int k) const { return at + k * step; }
    __device__ __forceinline__ bool has(int k) const { return at + k * step < cols; }
};

// v becomes (v - mean) * inv, inv = 1 / sqrt(mean square + eps), over the row; values outside of the row stay 0.  Returns inv.
template <int SIZE, int V, int K>
__device__ __forceinline__ float normalise(float (&v)[K][V], Team<SIZE>& team, const Columns<SIZE, V, K>& col, int kind, float eps, float inv_cols) {
    if (kind == kNormNone) return 1.f;
    if (kind == kNormLayer) {
        float s[1] = {0.f};
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) s[0] += v[k][i];
        team.sum(s);
        const float mean = s[0] * inv_cols;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) v[k][i] = col.has(k) ? v[k][i] - mean : 0.f;
    }
    float q[1] = {0.f};
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) q[0] = fmaf(v[k][i], v[k][i], q[0]);
    team.sum(q);
    const float inv = rsqrtf(fmaf(q[0], inv_cols, eps));
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) v[k][i] *= inv;
    return inv;
}

constexpr int kNormWarpThreads = 256;            // CTA of warp teams

// Most threads of a CTA: a CTA team has up to 8192 / (K * V) threads.
template <int SIZE, int V, int K>
constexpr int kNormThreads = SIZE ? kNormWarpThreads : 8192 / (K * V);

template <typename T, int V, int K, int SIZE>
__global__ void __launch_bounds__(kNormThreads<SIZE, V, K>) k_residual_norm(NormArgs a) {
    __shared__ float scratch[2 * 32 * Team<SIZE>::kMostSums];
    Team<SIZE> team(scratch);
    const Columns<SIZE, V, K> col(team, a.cols);
    const int64_t row = SIZE ? static_cast<int64_t>(blockIdx.x) * (blockDim.x / (SIZE ? SIZE : 1)) + threadIdx.x / (SIZE ? SIZE : 1) : blockIdx.x;
    const bool mine = row < a.rows;               // a warp's last teams may have no row, but take part in its shuffles

    Pack<T, V> px[K], ph[K], pg[K];
    const T* const x = static_cast<const T*>(a.x) + row * a.x_ld;
    const T* const h = static_cast<const T*>(a.h) + row * a.h_ld;
    const T* const g = static_cast<const T*>(a.gate) + (a.gate ? row / a.gate_rows : 0) * a.gate_ld;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const bool ok = mine && col.has(k);
        if (a.h) ph[k] = ok ? load_pack<T, V>(h + col(k)) : zero_pack<T, V>();
        if (a.gate) pg[k] = ok ? load_pack<T, V>(g + col(k)) : zero_pack<T, V>();
        px[k] = ok ? load_pack<T, V>(x + col(k)) : zero_pack<T, V>();
    }
    float r[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k) unpack(px[k], r[k]);
    if (a.h) {
        float p[K][V];
#pragma unroll
        for (int k = 0; k < K; ++k) unpack(ph[k], p[k]);
        normalise(p, team, col, a.post, a.eps, a.inv_cols);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (!col.has(k)) continue;
            float w[V], b[V], s[V], t[V];
            load_params(a.post_w, col(k), 1.f, w);
            load_params(a.post_b, col(k), 0.f, b);
            load_params(a.scale, col(k), 1.f, s);
            if (a.gate) unpack(pg[k], t);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (a.gate) s[i] *= gate_value(t[i], a.gate_kind).a;
                r[k][i] = fmaf(s[i], fmaf(p[k][i], w[i], b[i]), r[k][i]);
            }
        }
        if (a.r && mine) {
            T* const out = static_cast<T*>(a.r) + row * a.r_ld;
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (col.has(k)) store_pack<T, V>(out + col(k), r[k]);
        }
    }
    if (!a.n) return;
    normalise(r, team, col, a.pre, a.eps, a.inv_cols);
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (!col.has(k)) continue;
        float w[V], b[V];
        load_params(a.pre_w, col(k), 1.f, w);
        load_params(a.pre_b, col(k), 0.f, b);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            r[k][i] = fmaf(r[k][i], w[i], b[i]);
            top = max(top, magnitude_bits(r[k][i]));
        }
        if (!a.n_scale && mine) store_pack<T, V>(static_cast<T*>(a.n) + row * a.n_ld + col(k), r[k]);
    }
    if (!a.n_scale) return;
    const RowScale q = row_scale(team.top(top));
    if (!mine) return;
    if (team.rank() == 0) a.n_scale[row] = q.scale;
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (col.has(k)) store_quantised<V>(static_cast<int8_t*>(a.n) + row * a.n_ld + col(k), r[k], q.inverse);
}

// ---- backward ----------------------------------------------------------------------------------------------------------
struct NormGradArgs {
    NormArgs f;
    const void *d_r, *d_n;                        // either may be null
    int64_t d_r_ld, d_n_ld;
    void *d_x, *d_h, *d_gate;                     // each may be null
    int64_t d_x_ld, d_h_ld, d_gate_ld;
    float* sums;                                  // [CTAs][2 or 4][cols]: sum e * hat, sum d_n * r_hat, with BIAS also sum e, sum d_n
    float* gate_sums;                             // [teams][2][cols]: of the team's first and last group, where another team has the rest
    int64_t teams;
};
// Rows of team t.
__device__ __forceinline__ int64_t first_row_of(int64_t t, int64_t teams, int64_t rows) {
    return rows / teams * t + (rows % teams * t) / teams;
}

// GROUPS: a gate for each group of rows, whose gradient is a sum over them.  BIAS: either norm has one, so that the plain sums are needed.
template <typename T, int V, int K, int SIZE, bool BIAS, bool GROUPS>
__global__ void __launch_bounds__(kNormThreads<SIZE, V, K>) k_residual_norm_grad(NormGradArgs g) {
    extern __shared__ float column_sums[];        // [cols], for CTAs of several teams
    __shared__ float scratch[2 * 32 * Team<SIZE>::kMostSums];
    const NormArgs& a = g.f;
    Team<SIZE> team(scratch);
    const Columns<SIZE, V, K> col(team, a.cols);
    const int teams_here = SIZE ? blockDim.x / (SIZE ? SIZE : 1) : 1, team_here = SIZE ? threadIdx.x / (SIZE ? SIZE : 1) : 0;
    const int64_t t = static_cast<int64_t>(blockIdx.x) * teams_here + team_here;
    const int64_t first = first_row_of(t, g.teams, a.rows), last = first_row_of(t + 1, g.teams, a.rows);
    const int64_t turns = ceil_div64(a.rows, g.teams);         // the same for all teams of a warp: its shuffles take all lanes
    constexpr int kBias = BIAS ? K : 1, kGroups = GROUPS ? K : 1;
    float e_hat[K][V] = {}, n_hat[K][V] = {}, e_sum[kBias][V] = {}, n_sum[kBias][V] = {}, gate_sum[kGroups][V] = {};

    dependency_wait();
    for (int64_t turn = 0; turn < turns; ++turn) {
        const int64_t row = first + turn;
        const bool mine = row < last;
        Pack<T, V> px[K], ph[K], pg[K], pr[K], pn[K];
        const int64_t group = a.gate && mine ? row / a.gate_rows : 0;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const bool ok = mine && col.has(k);
            ph[k] = ok && a.h ? load_pack<T, V>(static_cast<const T*>(a.h) + row * a.h_ld + col(k)) : zero_pack<T, V>();
            px[k] = ok ? load_pack<T, V>(static_cast<const T*>(a.x) + row * a.x_ld + col(k)) : zero_pack<T, V>();
            if (a.gate) pg[k] = ok ? load_pack<T, V>(static_cast<const T*>(a.gate) + group * a.gate_ld + col(k)) : zero_pack<T, V>();
            pn[k] = ok && g.d_n ? load_pack<T, V>(static_cast<const T*>(g.d_n) + row * g.d_n_ld + col(k)) : zero_pack<T, V>();
            pr[k] = ok && g.d_r ? load_pack<T, V>(static_cast<const T*>(g.d_r) + row * g.d_r_ld + col(k)) : zero_pack<T, V>();
        }
        float hat[K][V], r[K][V], d[K][V];        // d: the whole gradient at r
#pragma unroll
        for (int k = 0; k < K; ++k) unpack(ph[k], hat[k]);
        const float h_inv = a.h ? normalise(hat, team, col, a.post, a.eps, a.inv_cols) : 1.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            unpack(px[k], r[k]);
            if (!a.h || !col.has(k)) continue;
            float w[V], b[V], s[V], u[V];
            load_params(a.post_w, col(k), 1.f, w);
            load_params(a.post_b, col(k), 0.f, b);
            load_params(a.scale, col(k), 1.f, s);
            if (a.gate) unpack(pg[k], u);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (a.gate) s[i] *= gate_value(u[i], a.gate_kind).a;
                r[k][i] = fmaf(s[i], fmaf(hat[k][i], w[i], b[i]), r[k][i]);
            }
        }
        if (g.d_n) {
            const float r_inv = normalise(r, team, col, a.pre, a.eps, a.inv_cols);
            float s[2] = {0.f, 0.f};              // sums of the gradient at r_hat, and of its products with r_hat
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float w[V], dn[V];
                unpack(pn[k], dn);
                if (col.has(k)) load_params(a.pre_w, col(k), 1.f, w);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    n_hat[k][i] = fmaf(dn[i], r[k][i], n_hat[k][i]);
                    if constexpr (BIAS) n_sum[k][i] += dn[i];
                    d[k][i] = col.has(k) ? dn[i] * w[i] : 0.f;
                    s[0] += d[k][i];
                    s[1] = fmaf(d[k][i], r[k][i], s[1]);
                }
            }
            if (a.pre != kNormNone) {
                team.sum(s);
                const float mean = a.pre == kNormLayer ? s[0] * a.inv_cols : 0.f, along = s[1] * a.inv_cols;
#pragma unroll
                for (int k = 0; k < K; ++k)
#pragma unroll
                    for (int i = 0; i < V; ++i) d[k][i] = r_inv * (d[k][i] - mean - r[k][i] * along);
            }
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) d[k][i] = 0.f;
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float dr[V];
            unpack(pr[k], dr);
#pragma unroll
            for (int i = 0; i < V; ++i) d[k][i] += dr[i];
            if (g.d_x && mine && col.has(k)) store_pack<T, V>(static_cast<T*>(g.d_x) + row * g.d_x_ld + col(k), d[k]);
        }
        if (!a.h) continue;
        float s[2] = {0.f, 0.f};                  // the same two sums at hat
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (!col.has(k)) continue;
            float w[V], b[V], scale[V], u[V], dg[V];
            load_params(a.post_w, col(k), 1.f, w);
            load_params(a.post_b, col(k), 0.f, b);
            load_params(a.scale, col(k), 1.f, scale);
            if (a.gate) unpack(pg[k], u);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const GateValue gate = a.gate ? gate_value(u[i], a.gate_kind) : GateValue{1.f, 0.f};
                const float e = d[k][i] * gate.a, at_gate = d[k][i] * scale[i] * fmaf(hat[k][i], w[i], b[i]);
                e_hat[k][i] = fmaf(e, hat[k][i], e_hat[k][i]);
                if constexpr (BIAS) e_sum[k][i] += e;
                if constexpr (GROUPS) gate_sum[k][i] += at_gate;
                else dg[i] = at_gate * gate.slope;
                d[k][i] = e * scale[i] * w[i];
                s[0] += d[k][i];
                s[1] = fmaf(d[k][i], hat[k][i], s[1]);
            }
            if constexpr (!GROUPS)
                if (g.d_gate && mine) store_pack<T, V>(static_cast<T*>(g.d_gate) + row * g.d_gate_ld + col(k), dg);
        }
        if (a.post != kNormNone) {
            team.sum(s);
            const float mean = a.post == kNormLayer ? s[0] * a.inv_cols : 0.f, along = s[1] * a.inv_cols;
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) d[k][i] = h_inv * (d[k][i] - mean - hat[k][i] * along);
        }
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (g.d_h && mine && col.has(k)) store_pack<T, V>(static_cast<T*>(g.d_h) + row * g.d_h_ld + col(k), d[k]);
        if constexpr (GROUPS) {
            // the last row of a group, or of this team: the sum is the gradient, or this team's part of it
            if (mine && (row + 1 == last || (row + 1) / a.gate_rows != group)) {
                const int64_t start = group * a.gate_rows, end = min(start + a.gate_rows, a.rows);
                const bool whole = start >= first && end <= last;
                float* const part = g.gate_sums + (2 * t + (start < first ? 0 : 1)) * a.cols;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    if (col.has(k)) {
                        if (whole) {
                            float u[V];
                            unpack(pg[k], u);
#pragma unroll
                            for (int i = 0; i < V; ++i) gate_sum[k][i] *= gate_value(u[i], a.gate_kind).slope;
                            if (g.d_gate) store_pack<T, V>(static_cast<T*>(g.d_gate) + group * g.d_gate_ld + col(k), gate_sum[k]);
                        } else {
#pragma unroll
                            for (int i = 0; i < V; ++i) part[col(k) + i] = gate_sum[k][i];
                        }
                    }
#pragma unroll
                    for (int i = 0; i < V; ++i) gate_sum[k][i] = 0.f;
                }
            }
        }
    }
    // this CTA's sums
    float* const out = g.sums + static_cast<int64_t>(blockIdx.x) * (BIAS ? 4 : 2) * a.cols;
    const auto put = [&](float* to, const float (&v)[K][V]) {
        if constexpr (SIZE == 0) {
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (col.has(k))
#pragma unroll
                    for (int i = 0; i < V; ++i) to[col(k) + i] = v[k][i];
        } else {
            for (int w = 0; w < teams_here; ++w) {
                if (w == team_here)
#pragma unroll
                    for (int k = 0; k < K; ++k)
                        if (col.has(k))
#pragma unroll
                            for (int i = 0; i < V; ++i) column_sums[col(k) + i] = w ? column_sums[col(k) + i] + v[k][i] : v[k][i];
                __syncthreads();
            }
            for (int c = threadIdx.x; c < a.cols; c += blockDim.x) to[c] = column_sums[c];
            __syncthreads();
        }
    };
    put(out, e_hat);
    put(out + a.cols, n_hat);
    if constexpr (BIAS) {
        put(out + 2 * a.cols, e_sum);
        put(out + 3 * a.cols, n_sum);
    }
}

struct NormFinishArgs {
    NormGradArgs g;
    int ctas, each;                               // CTAs whose sums there are, and how many sums each has
    int column_blocks;                            // the grid's first blocks: the parameters; the others: the groups' gates
    float *d_scale, *d_post_w, *d_post_b, *d_pre_w, *d_pre_b;      // each may be null
};
constexpr int kFinishColumns = 32, kFinishSlices = 16;

// The parameters' gradients from the CTAs' sums (32 columns per block, the CTAs in 16 interleaved parts), and the gradients of gates whose rows
// several teams had.
template <typename T>
__global__ void __launch_bounds__(kFinishColumns * kFinishSlices) k_norm_grad_finish(NormFinishArgs q) {
    __shared__ float part[4][kFinishSlices][kFinishColumns];
    const NormArgs& a = q.g.f;
    dependency_wait();
    if (static_cast<int>(blockIdx.x) >= q.column_blocks) {
        // team t begins a group that it does not end: the parts of that group, in the teams' order
        for (int64_t t = static_cast<int64_t>(blockIdx.x) - q.column_blocks; t < q.g.teams; t += static_cast<int64_t>(gridDim.x) - q.column_blocks) {
            const int64_t first = first_row_of(t, q.g.teams, a.rows), last = first_row_of(t + 1, q.g.teams, a.rows);
            if (first == last) continue;
            const int64_t group = (last - 1) / a.gate_rows, start = group * a.gate_rows, end = min(start + a.gate_rows, a.rows);
            if (start < first || end <= last) continue;
            for (int c = threadIdx.x; c < a.cols; c += blockDim.x) {
                float s = q.g.gate_sums[(2 * t + 1) * a.cols + c];
                int64_t at = last;
                for (int64_t v = t + 1; at < end; ++v) {
                    const int64_t next = first_row_of(v + 1, q.g.teams, a.rows);
                    if (next > at) s += q.g.gate_sums[2 * v * a.cols + c];
                    at = next;
                }
                const float u = to_float(static_cast<const T*>(a.gate)[group * a.gate_ld + c]);
                from_float(static_cast<T*>(q.g.d_gate)[group * q.g.d_gate_ld + c], s * gate_value(u, a.gate_kind).slope);
            }
        }
        return;
    }
    const int x = threadIdx.x % kFinishColumns, slice = threadIdx.x / kFinishColumns, c = blockIdx.x * kFinishColumns + x;
    float s[4] = {};
    if (c < a.cols)
        for (int b = slice; b < q.ctas; b += kFinishSlices)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < q.each) s[i] += q.g.sums[(static_cast<int64_t>(b) * q.each + i) * a.cols + c];
#pragma unroll
    for (int i = 0; i < 4; ++i) part[i][slice][x] = s[i];
    __syncthreads();
    if (slice != 0 || c >= a.cols) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        s[i] = 0.f;
#pragma unroll
        for (int j = 0; j < kFinishSlices; ++j) s[i] += part[i][j][x];
    }
    const float w = a.post_w ? a.post_w[c] : 1.f, b = a.post_b ? a.post_b[c] : 0.f, scale = a.scale ? a.scale[c] : 1.f;
    if (q.d_scale) q.d_scale[c] = fmaf(w, s[0], b * s[2]);
    if (q.d_post_w) q.d_post_w[c] = scale * s[0];
    if (q.d_post_b) q.d_post_b[c] = scale * s[2];
    if (q.d_pre_w) q.d_pre_w[c] = s[1];
    if (q.d_pre_b) q.d_pre_b[c] = s[3];
}

// Teams of a backward pass and the CTAs that hold them.
struct GradPlan {
    int64_t ctas, teams;
};

// The launches (norm_launch.cuh), compiled once for each type.  packs: accesses of 16 bytes.
template <typename T>
void run_norm(const NormArgs& a, bool packs, cudaStream_t s);
template <typename T>
void run_norm_grad(const NormFinishArgs& q, const GradPlan& plan, bool packs, bool bias, bool groups, int finish_blocks, cudaStream_t s);

}  // namespace layers
}  // namespace cutoff
