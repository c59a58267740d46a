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
    int64_t x_ld, h_ld, gate_ld;
    int rows, gate_rows, cols, gate_kind, post, pre;
    float eps, inv_cols;
    // forward
    void *r, *n;                                  // or null
    float* n_scale;                               // not null: n is 8-bit rows with these scales
    int64_t r_ld, n_ld;
};

// 1 / (1 + exp(-g)); exp of a large -g is infinite and the result 0.  Within some units of the last place for gates of ordinary size.
__device__ __forceinline__ float logistic(float g) {
    float e, s;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(g * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s) : "f"(1.f + e));
    return s;
}
// act(g) of a pack, and with SLOPE its derivative; the kind is the same for a whole call, so that one branch serves the pack.
template <bool SLOPE, int V>
__device__ __forceinline__ void gate_values(const float (&g)[V], int kind, float (&a)[V], float (&slope)[V]) {
    if (kind == kGateLinear) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            a[i] = g[i];
            if constexpr (SLOPE) slope[i] = 1.f;
        }
    } else if (kind == kGateSigmoid) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            a[i] = logistic(g[i]);
            if constexpr (SLOPE) slope[i] = fmaf(-a[i], a[i], a[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float t = logistic(g[i]);
            a[i] = g[i] * t;
            if constexpr (SLOPE) slope[i] = fmaf(a[i], 1.f - t, t);
        }
    }
}
template <int V>
__device__ __forceinline__ void multiply(float (&s)[V], const float* p, int c) {
    if (p == nullptr) return;
    float f[V];
    load_params(p, c, 1.f, f);
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] *= f[i];
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

template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src) {
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}

// The operands of a team's rows in shared memory: one or two stages, [stage][operand][k][thread].  A thread copies what it reads itself, so that
// no barrier is needed; with two stages the next row is on its way while this one is worked on.
template <typename T, int V, int K, int SIZE>
struct Staged {
    using P = Pack<T, V>;
    P* own;
    int stage_packs;
    const Columns<SIZE, V, K>& col;
    __device__ __forceinline__ Staged(uint8_t* smem, int operands, const Columns<SIZE, V, K>& c)
        : own(reinterpret_cast<P*>(smem) + threadIdx.x), stage_packs(operands * K * static_cast<int>(blockDim.x)), col(c) {}
    __device__ __forceinline__ P& slot(int stage, int operand, int k) const { return own[stage * stage_packs + (operand * K + k) * static_cast<int>(blockDim.x)]; }
    __device__ __forceinline__ void copy(const void* base, int64_t ld, int64_t row, int stage, int operand) const {
        const T* const p = static_cast<const T*>(base) + row * ld;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (!col.has(k)) continue;
            if constexpr (sizeof(P) >= 4) copy_async<sizeof(P)>(static_cast<uint32_t>(__cvta_generic_to_shared(&slot(stage, operand, k))), p + col(k));
            else slot(stage, operand, k).v[0] = p[col(k)];
        }
    }
    __device__ __forceinline__ void get(int stage, int operand, int k, bool ok, float (&f)[V]) const { unpack(ok ? slot(stage, operand, k) : zero_pack<T, V>(), f); }
};
__device__ __forceinline__ void end_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// The copies of this row have landed; with two stages the next row's may be on their way.
__device__ __forceinline__ void wait_copies(int stages) {
    if (stages == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// A pack of the gate that a group of rows shares: it stays in the L1.
template <typename T, int V>
__device__ __forceinline__ void shared_gate(const T* p, float (&u)[V]) {
    if constexpr (V == 1) {
        u[0] = to_float(*p);
    } else {
        const uint4 raw = __ldg(reinterpret_cast<const uint4*>(p));
        unpack(*reinterpret_cast<const Pack<T, V>*>(&raw), u);
    }
}

constexpr int kNormWarpThreads = 256;            // CTA of warp teams

// Most threads of a CTA: a CTA team has up to 8192 / (K * V) threads.
template <int SIZE, int V, int K>
constexpr int kNormThreads = SIZE ? kNormWarpThreads : 8192 / (K * V);

// Operands of a row that are staged: not the gate of a group, which stays for many rows.
__host__ __device__ inline int norm_operands(const NormArgs& a) { return 1 + (a.h != nullptr) + (a.gate != nullptr && a.gate_rows == 1); }

template <typename T, int V, int K, int SIZE>
__global__ void __launch_bounds__(kNormThreads<SIZE, V, K>, 1024 / kNormThreads<SIZE, V, K>) k_residual_norm(NormArgs a, int stages) {
    extern __shared__ __align__(16) uint8_t operands[];
    __shared__ __align__(16) float scratch[Team<SIZE>::kScratch];
    Team<SIZE> team(scratch);
    const Columns<SIZE, V, K> col(team, a.cols);
    const bool gate_rows = a.gate && a.gate_rows == 1;
    const int at_h = 1, at_gate = at_h + (a.h != nullptr);
    const Staged<T, V, K, SIZE> staged(operands, at_gate + gate_rows, col);
    const int teams_here = SIZE ? blockDim.x / (SIZE ? SIZE : 1) : 1, team_here = SIZE ? threadIdx.x / (SIZE ? SIZE : 1) : 0;
    const int teams = gridDim.x * teams_here, turns = ceil_div(a.rows, teams);        // as many for all teams of a warp: its shuffles take all lanes
    const int64_t first = static_cast<int64_t>(blockIdx.x) * teams_here + team_here;
    const auto fetch = [&](int stage, int64_t row) {
        if (row < a.rows) {
            if (a.h) staged.copy(a.h, a.h_ld, row, stage, at_h);
            staged.copy(a.x, a.x_ld, row, stage, 0);
            if (gate_rows) staged.copy(a.gate, a.gate_ld, row, stage, at_gate);
        }
        end_copies();
    };
    fetch(0, first);
    for (int turn = 0; turn < turns; ++turn) {
        const int64_t row = first + static_cast<int64_t>(turn) * teams;
        const int stage = stages == 2 ? turn & 1 : 0;
        if (stages == 2) fetch(stage ^ 1, row + teams);
        wait_copies(stages);
        const bool mine = row < a.rows;           // a warp's last teams may have no row
        float r[K][V];
        if (a.h) {
#pragma unroll
            for (int k = 0; k < K; ++k) staged.get(stage, at_h, k, mine && col.has(k), r[k]);
            normalise(r, team, col, a.post, a.eps, a.inv_cols);
            const T* const group_gate =
                static_cast<const T*>(a.gate) + (a.gate && !gate_rows ? static_cast<int64_t>(static_cast<unsigned>(row) / static_cast<unsigned>(a.gate_rows)) * a.gate_ld : 0);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (!col.has(k)) continue;
                float t[V];
                multiply(r[k], a.post_w, col(k));
                if (a.post_b) {
                    load_params(a.post_b, col(k), 0.f, t);
#pragma unroll
                    for (int i = 0; i < V; ++i) r[k][i] += t[i];
                }
                multiply(r[k], a.scale, col(k));
                if (a.gate) {
                    float act[V];
                    if (gate_rows) staged.get(stage, at_gate, k, mine, t);
                    else if (mine) shared_gate(group_gate + col(k), t);
                    gate_values<false>(t, a.gate_kind, act, act);
#pragma unroll
                    for (int i = 0; i < V; ++i) r[k][i] *= act[i];
                }
                staged.get(stage, 0, k, mine, t);
#pragma unroll
                for (int i = 0; i < V; ++i) r[k][i] = mine ? r[k][i] + t[i] : 0.f;
                if (a.r && mine) store_pack<T, V>(static_cast<T*>(a.r) + row * a.r_ld + col(k), r[k]);
            }
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k) staged.get(stage, 0, k, mine && col.has(k), r[k]);
        }
        if (stages == 1) fetch(0, row + teams);   // this row's values have been used
        if (!a.n) continue;
        normalise(r, team, col, a.pre, a.eps, a.inv_cols);
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (!col.has(k)) continue;
            multiply(r[k], a.pre_w, col(k));
            if (a.pre_b) {
                float b[V];
                load_params(a.pre_b, col(k), 0.f, b);
#pragma unroll
                for (int i = 0; i < V; ++i) r[k][i] += b[i];
            }
            if (!a.n_scale) {
                if (mine) store_pack<T, V>(static_cast<T*>(a.n) + row * a.n_ld + col(k), r[k]);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) top = max(top, magnitude_bits(r[k][i]));
            }
        }
        if (!a.n_scale) continue;
        const RowScale q = row_scale(team.top(top));
        if (!mine) continue;
        if (team.rank() == 0) a.n_scale[row] = q.scale;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (col.has(k)) store_quantised<V>(static_cast<int8_t*>(a.n) + row * a.n_ld + col(k), r[k], q.inverse);
    }
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
    int teams;
    int stages;                                   // rows of a team in shared memory: 2, the next one on its way, or 1
};
// Rows of team t.
__device__ __forceinline__ int first_row_of(int t, int teams, int rows) { return static_cast<int>(static_cast<int64_t>(rows) * t / teams); }

// Operands that a row of the backward pass reads; with GROUPS the gate is not among them, it stays for many rows and is read through the L1.
template <bool GROUPS>
__host__ __device__ inline int grad_operands(const NormGradArgs& g) { return 1 + (g.f.h != nullptr) + (!GROUPS && g.f.gate) + (g.d_r != nullptr) + (g.d_n != nullptr); }

constexpr int kGradThreads = 512;                 // most threads of a CTA: 128 registers each

// GROUPS: a gate for each group of rows, whose gradient is a sum over them.  BIAS: either norm has one, so that the plain sums are needed.
// The operands of a team's next row are on their way to shared memory while this one is worked on; every thread copies what it reads itself, so that no barrier
// is needed for them.
template <typename T, int V, int K, int SIZE, bool BIAS, bool GROUPS>
__global__ void __launch_bounds__(SIZE ? kNormWarpThreads : kGradThreads, SIZE ? 2 : 1) k_residual_norm_grad(NormGradArgs g) {
    extern __shared__ __align__(16) uint8_t operands[];       // [stage][operand][k][thread]; afterwards [cols] sums
    __shared__ __align__(16) float scratch[Team<SIZE>::kScratch];
    const NormArgs& a = g.f;
    Team<SIZE> team(scratch);
    const Columns<SIZE, V, K> col(team, a.cols);
    const int teams_here = SIZE ? blockDim.x / (SIZE ? SIZE : 1) : 1, team_here = SIZE ? threadIdx.x / (SIZE ? SIZE : 1) : 0;
    const int t = blockIdx.x * teams_here + team_here;
    const int first = first_row_of(t, g.teams, a.rows), last = first_row_of(t + 1, g.teams, a.rows);
    const int turns = ceil_div(a.rows, g.teams);               // the same for all teams of a warp: its shuffles take all lanes
    constexpr int kBias = BIAS ? K : 1, kGroups = GROUPS ? K : 1;
    float e_hat[K][V] = {}, n_hat[K][V] = {}, e_sum[kBias][V] = {}, n_sum[kBias][V] = {}, gate_sum[kGroups][V] = {};

    // places of the operands in a stage
    const bool has_gate_rows = !GROUPS && a.gate != nullptr;
    const int at_h = 1, at_gate = at_h + (a.h != nullptr), at_r = at_gate + has_gate_rows, at_n = at_r + (g.d_r != nullptr), n_operands = at_n + (g.d_n != nullptr);
    const Staged<T, V, K, SIZE> staged(operands, n_operands, col);
    const auto fetch = [&](int stage, int row) {
        if (row < last) {
            if (a.h) staged.copy(a.h, a.h_ld, row, stage, at_h);
            staged.copy(a.x, a.x_ld, row, stage, 0);
            if (has_gate_rows) staged.copy(a.gate, a.gate_ld, row, stage, at_gate);
            if (g.d_n) staged.copy(g.d_n, g.d_n_ld, row, stage, at_n);
            if (g.d_r) staged.copy(g.d_r, g.d_r_ld, row, stage, at_r);
        }
        end_copies();
    };
    const auto get = [&](int stage, int operand, int k, bool ok, float (&f)[V]) { staged.get(stage, operand, k, ok, f); };

    dependency_wait();
    fetch(0, first);
    for (int turn = 0; turn < turns; ++turn) {
        const int row = first + turn, stage = g.stages == 2 ? turn & 1 : 0;
        const bool mine = row < last;
        if (g.stages == 2) fetch(stage ^ 1, row + 1);
        wait_copies(g.stages);
        const int group = GROUPS && mine ? row / a.gate_rows : 0;
        const T* const group_gate = static_cast<const T*>(a.gate) + group * a.gate_ld;
        const auto gate_of = [&](int k, float (&u)[V]) {
            if constexpr (GROUPS) {
                shared_gate(group_gate + col(k), u);
            } else {
                get(stage, at_gate, k, mine, u);
            }
        };
        float hat[K][V], r[K][V], d[K][V];        // d: the whole gradient at r
        float h_inv = 1.f;
        if (a.h) {
#pragma unroll
            for (int k = 0; k < K; ++k) get(stage, at_h, k, mine && col.has(k), hat[k]);
            h_inv = normalise(hat, team, col, a.post, a.eps, a.inv_cols);
        }
        if (g.d_n) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (a.h && col.has(k)) {
                    float u[V], act[V];
#pragma unroll
                    for (int i = 0; i < V; ++i) r[k][i] = hat[k][i];
                    multiply(r[k], a.post_w, col(k));
                    if constexpr (BIAS) {
                        load_params(a.post_b, col(k), 0.f, u);
#pragma unroll
                        for (int i = 0; i < V; ++i) r[k][i] += u[i];
                    }
                    multiply(r[k], a.scale, col(k));
                    if (a.gate) {
                        gate_of(k, u);
                        gate_values<false>(u, a.gate_kind, act, act);
#pragma unroll
                        for (int i = 0; i < V; ++i) r[k][i] *= act[i];
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < V; ++i) r[k][i] = 0.f;
                }
                float x[V];
                get(stage, 0, k, mine && col.has(k), x);
#pragma unroll
                for (int i = 0; i < V; ++i) r[k][i] += x[i];
            }
            const float r_inv = normalise(r, team, col, a.pre, a.eps, a.inv_cols);
            float s[2] = {0.f, 0.f};              // sums of the gradient at r_hat, and of its products with r_hat
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float dn[V];
                get(stage, at_n, k, mine && col.has(k), dn);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    n_hat[k][i] = fmaf(dn[i], r[k][i], n_hat[k][i]);
                    if constexpr (BIAS) n_sum[k][i] += dn[i];
                }
                if (col.has(k)) multiply(dn, a.pre_w, col(k));
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    d[k][i] = dn[i];
                    s[0] += dn[i];
                    s[1] = fmaf(dn[i], r[k][i], s[1]);
                }
            }
            if (a.pre != kNormNone) {
                team.sum(s);
                const float mean = a.pre == kNormLayer ? s[0] * a.inv_cols : 0.f, along = s[1] * a.inv_cols;
#pragma unroll
                for (int k = 0; k < K; ++k)
#pragma unroll
                    for (int i = 0; i < V; ++i) d[k][i] = r_inv * (fmaf(-along, r[k][i], d[k][i]) - mean);
            }
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) d[k][i] = 0.f;
        }
        if (g.d_r) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float dr[V];
                get(stage, at_r, k, mine && col.has(k), dr);
#pragma unroll
                for (int i = 0; i < V; ++i) d[k][i] += dr[i];
            }
        }
        if (g.d_x && mine) {
            T* const out = static_cast<T*>(g.d_x) + row * g.d_x_ld;
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (col.has(k)) store_pack<T, V>(out + col(k), d[k]);
        }
        if (a.h) {
            float s[2] = {0.f, 0.f};              // the same two sums at hat
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (!col.has(k)) continue;
                float w[V], scale[V], at_gate_value[V];
                load_params(a.post_w, col(k), 1.f, w);
                load_params(a.scale, col(k), 1.f, scale);
                if (a.gate && (GROUPS || g.d_gate)) {
                    float p[V];
#pragma unroll
                    for (int i = 0; i < V; ++i) p[i] = hat[k][i] * w[i];
                    if constexpr (BIAS) {
                        float b[V];
                        load_params(a.post_b, col(k), 0.f, b);
#pragma unroll
                        for (int i = 0; i < V; ++i) p[i] += b[i];
                    }
#pragma unroll
                    for (int i = 0; i < V; ++i) at_gate_value[i] = d[k][i] * scale[i] * p[i];
                }
                if (a.gate) {
                    float u[V], act[V], slope[V];
                    gate_of(k, u);
                    if constexpr (GROUPS) {
                        gate_values<false>(u, a.gate_kind, act, slope);
#pragma unroll
                        for (int i = 0; i < V; ++i) gate_sum[k][i] += at_gate_value[i];
                    } else if (g.d_gate) {
                        gate_values<true>(u, a.gate_kind, act, slope);
#pragma unroll
                        for (int i = 0; i < V; ++i) slope[i] *= at_gate_value[i];
                        if (mine) store_pack<T, V>(static_cast<T*>(g.d_gate) + row * g.d_gate_ld + col(k), slope);
                    } else {
                        gate_values<false>(u, a.gate_kind, act, slope);
                    }
#pragma unroll
                    for (int i = 0; i < V; ++i) d[k][i] *= act[i];
                }
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    e_hat[k][i] = fmaf(d[k][i], hat[k][i], e_hat[k][i]);
                    if constexpr (BIAS) e_sum[k][i] += d[k][i];
                    d[k][i] *= scale[i] * w[i];
                    s[0] += d[k][i];
                    s[1] = fmaf(d[k][i], hat[k][i], s[1]);
                }
            }
            if (g.d_h) {
                if (a.post != kNormNone) {
                    team.sum(s);
                    const float mean = a.post == kNormLayer ? s[0] * a.inv_cols : 0.f, along = s[1] * a.inv_cols;
#pragma unroll
                    for (int k = 0; k < K; ++k)
#pragma unroll
                        for (int i = 0; i < V; ++i) d[k][i] = h_inv * (fmaf(-along, hat[k][i], d[k][i]) - mean);
                }
                if (mine) {
                    T* const out = static_cast<T*>(g.d_h) + row * g.d_h_ld;
#pragma unroll
                    for (int k = 0; k < K; ++k)
                        if (col.has(k)) store_pack<T, V>(out + col(k), d[k]);
                }
            }
            if constexpr (GROUPS) {
                // the last row of a group, or of this team: the sum is the gradient, or this team's part of it
                if (mine && (row + 1 == last || (row + 1) / a.gate_rows != group)) {
                    const int64_t start = static_cast<int64_t>(group) * a.gate_rows, end = min(start + a.gate_rows, static_cast<int64_t>(a.rows));
                    const bool whole = start >= first && end <= last;
                    float* const part = g.gate_sums + (2 * static_cast<int64_t>(t) + (start < first ? 0 : 1)) * a.cols;
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        if (col.has(k)) {
                            if (whole) {
                                float u[V], act[V], slope[V];
                                gate_of(k, u);
                                gate_values<true>(u, a.gate_kind, act, slope);
#pragma unroll
                                for (int i = 0; i < V; ++i) slope[i] *= gate_sum[k][i];
                                if (g.d_gate) store_pack<T, V>(static_cast<T*>(g.d_gate) + group * g.d_gate_ld + col(k), slope);
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
        if (g.stages == 1) fetch(0, row + 1);     // this row's values have been used
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    // this CTA's sums
    float* const out = g.sums + static_cast<int64_t>(blockIdx.x) * (BIAS ? 4 : 2) * a.cols;
    float* const column_sums = reinterpret_cast<float*>(operands);
    if constexpr (SIZE != 0) __syncthreads();     // nobody reads operands any more
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
        for (int t = static_cast<int>(blockIdx.x) - q.column_blocks; t < q.g.teams; t += static_cast<int>(gridDim.x) - q.column_blocks) {
            const int first = first_row_of(t, q.g.teams, a.rows), last = first_row_of(t + 1, q.g.teams, a.rows);
            if (first == last) continue;
            const int64_t group = (last - 1) / a.gate_rows, start = group * a.gate_rows, end = min(start + a.gate_rows, static_cast<int64_t>(a.rows));
            if (start < first || end <= last) continue;
            for (int c = threadIdx.x; c < a.cols; c += blockDim.x) {
                float s = q.g.gate_sums[(2 * static_cast<int64_t>(t) + 1) * a.cols + c];
                int at = last;
                for (int v = t + 1; at < end; ++v) {
                    const int next = first_row_of(v + 1, q.g.teams, a.rows);
                    if (next > at) s += q.g.gate_sums[2 * static_cast<int64_t>(v) * a.cols + c];
                    at = next;
                }
                const float u[1] = {to_float(static_cast<const T*>(a.gate)[group * a.gate_ld + c])};
                float act[1], slope[1];
                gate_values<true>(u, a.gate_kind, act, slope);
                from_float(static_cast<T*>(q.g.d_gate)[group * q.g.d_gate_ld + c], s * slope[0]);
            }
        }
        return;
    }
    const int x = threadIdx.x % kFinishColumns, slice = threadIdx.x / kFinishColumns, c = blockIdx.x * kFinishColumns + x;
    float s[4] = {};
    if (c < a.cols) {
#pragma unroll 8                                   // loads that wait for nothing
        for (int b = slice; b < q.ctas; b += kFinishSlices)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < q.each) s[i] += q.g.sums[(static_cast<int64_t>(b) * q.each + i) * a.cols + c];
    }
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

// The teams of a backward pass: their threads (32 lanes or fewer, or a CTA), the values of a thread, the CTAs.  Without more sums than the two products
// a thread has room for 16 values (rows of 4096 bf16 values 719 us with eight and operands in registers, ...); with them it has eight, where a CTA can then
// hold a row at all.
struct GradPlan {
    int lanes, values, threads, per_sm, ctas, teams;
};
constexpr int kMostSms = 160, kMostTeamRows = 1024;          // a team adds at most this many rows in a row
inline GradPlan grad_plan(int rows, int cols, bool many_sums, int sms) {
    GradPlan p;
    p.lanes = cols <= 32 ? 4 : cols <= 128 ? 16 : cols <= 256 || (cols <= 512 && !many_sums) ? 32 : 0;
    p.values = p.lanes ? (cols <= 256 ? 8 : 16) : many_sums && cols <= 8 * kGradThreads ? 8 : 16;
    p.threads = p.lanes ? kNormWarpThreads : ceil_div(ceil_div(cols, p.values), 32) * 32;
    p.per_sm = kGradThreads / p.threads;                      // by the registers; shared memory may allow fewer
    const int per_cta = p.lanes ? p.threads / p.lanes : 1;
    const int few = ceil_div(rows, per_cta), many = ceil_div(few, kMostTeamRows), resident = (sms < kMostSms ? sms : kMostSms) * p.per_sm;
    p.ctas = resident < many ? many : resident;
    p.ctas = p.ctas < few ? p.ctas : few;
    p.teams = p.ctas * per_cta;
    return p;
}

// The launches (norm_launch.cuh), compiled once for each type.  packs: accesses of 16 bytes.
template <typename T>
bool run_norm(const NormArgs& a, bool packs, int sms, cudaStream_t s);
template <typename T>
bool run_norm_grad(NormFinishArgs& q, const GradPlan& plan, bool packs, bool bias, bool groups, int finish_blocks, cudaStream_t s);

}  // namespace layers
}  // namespace cutoff
