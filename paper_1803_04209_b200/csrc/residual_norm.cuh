// The end of one residual block and the start of the next, in one pass over the rows:
//
//   r = x + scale * act(gate) * post(h),   n = pre(r)
//   post(h) = (h - mean(h)) / sqrt(var(h) + eps) * post_weight + post_bias    (layer; RMS: without the mean; none: h itself)
//
// and the gradients of all of it.  Statistics and sums are fp32, r enters the second norm unrounded; a value is rounded once, where
// it is stored.  The backward pass reads x and h, not r: the parameters' gradients are fp32 sums, and a rounded r would be seen in them.
// It forms the statistics again instead of reading them: the rows are in registers anyway.
//
// A row belongs to a team, 4 to 32 lanes of a warp (rows of up to 512 values) or a CTA, that goes through many rows; the asynchronous copy engine brings
// the operands of the next row into shared memory meanwhile (RowPipe).  The backward pass keeps the parameters' sums of a thread's columns in
// registers; k_norm_grad_finish adds the CTAs' sums in a tree of fixed shape, so that results are the same on every run.
//
// What bounds it (4096 bf16 values, 16384 rows, a gate value for each): the forward pass the memory, 0.67 GB in 108 us, 95 % of a copy's rate; the
// backward pass, 1.07 GB in 225 us (73 %), its instructions, some 55 per value and as many as 16 warps of 128 registers issue between four sums
// over the CTA per row (RMS norms; layer norms take two more).  What made it so, in us: operands in registers 341 and 703; staged by cp.async 157 and 357; by bulk copies, with two values per
// instruction and parameters in registers or shared memory (in the L1, beside the operands, there is no room for them) 153 and 281; predicates beside the accesses and one branch
// on the gate's kind per row instead of one for each pack 108 and 224.  Odd rows pay for single values: 5000 rows of 2175 fp32 values with
// layer norms, biases and a gate for every 125 rows 53 us (floor 27), the gradients of 4001 x 1025 58 us (floor 15).  Not kept: consecutive rows per team
// where nothing asks for them (150 us against 106); single values in pairs a team apart, two to an instruction (no gain: latency bounds those rows).
#pragma once
#include "layer_types.cuh"

namespace cutoff {
namespace layers {

enum : int { kNormNone = 0, kNormRms = 1, kNormLayer = 2 };
enum : int { kGateLinear = 0, kGateSigmoid = 1, kGateSilu = 2 };

constexpr int kMostRows = 1 << 30;

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

// 1 / (1 + exp(-g)) and, with SLOPE, its derivative as a product, not as value - value^2, of which nothing is left where the value is close to 1.
// EXACT, for fp32: from u = exp(-|g|), which is two units of the last place off, and s = 1 / (1 + u): s or u s, within six units, and u s s, within
// eight, whatever the gate.  Otherwise, for what is rounded to 16 bits: the hardware's exponential of -g log2(e), e, at a third of the instructions:
// s = 1 / (1 + e) within 2 |g| + 10 units of 2^-24, a hundredth of its own rounding, and e s s; zero below 2^-126 (e stops at 2^127: infinity times
// zero would be NaN).  100000 x 512 fp32 values with gates, gradients: 325 us if nothing is EXACT, 345 as it is; 60000 x 333 fp16
// 139 us so and 149 with EXACT's form.
template <bool EXACT, bool SLOPE>
__device__ __forceinline__ float logistic(float g, float& slope) {
    float e, s;
    if constexpr (EXACT) {
        e = expf(-fabsf(g));
    } else {
        float t = g * -1.4426950408889634f;
        if constexpr (SLOPE) asm("min.NaN.f32 %0, %0, %1;" : "+f"(t) : "f"(127.f));
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(t));
    }
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s) : "f"(1.f + e));
    if constexpr (SLOPE) slope = e * s * s;
    return EXACT ? (g < 0.f ? e : 1.f) * s : s;
}
template <bool EXACT, bool SLOPE>
__device__ __forceinline__ F1 logistic(F1 g, F1& slope) { return F1{logistic<EXACT, SLOPE>(g.v, slope.v)}; }
template <bool EXACT, bool SLOPE>
__device__ __forceinline__ F2 logistic(F2 g, F2& slope) {
    float x, y, s = 0.f, t = 0.f;
    unpack2(g.v, x, y);
    x = logistic<EXACT, SLOPE>(x, s);
    y = logistic<EXACT, SLOPE>(y, t);
    if constexpr (SLOPE) slope.v = pack2(s, t);
    return F2{pack2(x, y)};
}
template <typename T>
constexpr bool kExactGate = sizeof(T) == 4;
// g becomes act(g), and with SLOPE slope its derivative.
template <bool EXACT, int KIND, bool SLOPE, typename N, int M>
__device__ __forceinline__ void gate_values(N (&g)[M], N (&slope)[M]) {
#pragma unroll
    for (int i = 0; i < M; ++i) {
        if constexpr (KIND == kGateLinear) {
            if constexpr (SLOPE) slope[i] = splat<N>(1.f);
        } else {
            N d;
            const N s = logistic<EXACT, SLOPE>(g[i], d);
            if constexpr (KIND == kGateSigmoid) {
                g[i] = s;
                if constexpr (SLOPE) slope[i] = d;
            } else {
                if constexpr (SLOPE) slope[i] = fma(g[i], d, s);
                g[i] = mul(g[i], s);
            }
        }
    }
}
// f(kind as a constant): the kind is the same for a whole call, and one branch serves a thread's whole row.
template <typename F>
__device__ __forceinline__ void with_gate(int kind, F f) {
    if (kind == kGateLinear) f(std::integral_constant<int, kGateLinear>{});
    else if (kind == kGateSigmoid) f(std::integral_constant<int, kGateSigmoid>{});
    else f(std::integral_constant<int, kGateSilu>{});
}

// The team's columns: K packs of V values per thread.
template <int SIZE, int V, int K>
struct Columns {
    int cols, at, step;
    __device__ __forceinline__ Columns(const Team<SIZE>& t, int n) : cols(n), at(t.rank() * V), step(t.size() * V) {}
    __device__ __forceinline__ int operator()(int k) const { return at + k * step; }
    __device__ __forceinline__ bool has(int k) const { return at + k * step < cols; }
};

// A thread's values of a row: K packs of V.
template <int V, int K>
using Values = Num<V>[K][kNums<V>];

template <int V, int K>
__device__ __forceinline__ float dot(const Values<V, K>& a, const Values<V, K>& b) {
    Num<V> s = splat<Num<V>>(0.f);
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < kNums<V>; ++i) s = fma(a[k][i], b[k][i], s);
    return total(s);
}
template <int V, int K>
__device__ __forceinline__ float sum_of(const Values<V, K>& a) {
    Num<V> s = splat<Num<V>>(0.f);
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < kNums<V>; ++i) s = add(s, a[k][i]);
    return total(s);
}

// What did not arrive in time is marked.
template <int V, int K>
__device__ __forceinline__ void mark(bool failed, Values<V, K>& v) {
    if (!failed) return;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < kNums<V>; ++i) v[k][i] = splat<Num<V>>(__int_as_float(0x7fc00000));
}

// v becomes (v - mean) * inv, inv = 1 / sqrt(mean square + eps), over the row; values outside of the row are 0 and stay so.  Returns inv.
// LAYER: the kind may be a layer norm; without it no mean is looked for.
template <bool LAYER, int SIZE, int V, int K>
__device__ __forceinline__ float normalise(Values<V, K>& v, Team<SIZE>& team, const Columns<SIZE, V, K>& col, int kind, float eps, float inv_cols) {
    if (kind == kNormNone) return 1.f;
    if constexpr (LAYER) {
        if (kind == kNormLayer) {
            float s[1] = {sum_of<V, K>(v)};
            team.sum(s);
            const Num<V> mean = splat<Num<V>>(-s[0] * inv_cols);
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < kNums<V>; ++i) v[k][i] = col.has(k) ? add(v[k][i], mean) : splat<Num<V>>(0.f);
        }
    }
    float q[1] = {dot<V, K>(v, v)};
    team.sum(q);
    const float inv = rsqrtf(fmaf(q[0], inv_cols, eps));
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < kNums<V>; ++i) v[k][i] = mul(v[k][i], splat<Num<V>>(inv));
    return inv;
}
// v becomes the gradient at what hat = (v - mean) * inv was formed of, given the one at hat.
template <bool LAYER, int SIZE, int V, int K>
__device__ __forceinline__ void through_norm(Values<V, K>& v, const Values<V, K>& hat, float inv, Team<SIZE>& team, int kind, float inv_cols) {
    using N = Num<V>;
    if (kind == kNormNone) return;
    if (LAYER && kind == kNormLayer) {
        float s[2] = {sum_of<V, K>(v), dot<V, K>(v, hat)};
        team.sum(s);
        const N mean = splat<N>(-s[0] * inv_cols * inv), along = splat<N>(-s[1] * inv_cols * inv);
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < kNums<V>; ++i) v[k][i] = fma(along, hat[k][i], fma(splat<N>(inv), v[k][i], mean));
    } else {
        float s[1] = {dot<V, K>(v, hat)};
        team.sum(s);
        const N along = splat<N>(-s[0] * inv_cols * inv);
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < kNums<V>; ++i) v[k][i] = fma(along, hat[k][i], mul(splat<N>(inv), v[k][i]));
    }
}
template <int V>
__device__ __forceinline__ void multiply(Num<V> (&s)[kNums<V>], const float* p, int c) {
    if (p == nullptr) return;
    Num<V> f[kNums<V>];
    read_global<float, V>(p + c, f);
#pragma unroll
    for (int i = 0; i < kNums<V>; ++i) s[i] = mul(s[i], f[i]);
}
template <int V>
__device__ __forceinline__ void add_to(Num<V> (&s)[kNums<V>], const float* p, int c) {
    if (p == nullptr) return;
    Num<V> f[kNums<V>];
    read_global<float, V>(p + c, f);
#pragma unroll
    for (int i = 0; i < kNums<V>; ++i) s[i] = add(s[i], f[i]);
}

// Values as fp32 at p (16-byte aligned if V > 1), or added to what is there.
template <int V>
__device__ __forceinline__ void write_floats(float* p, const Num<V> (&n)[kNums<V>], bool more) {
    if constexpr (V == 1) {
        *p = more ? *p + n[0].v : n[0].v;
    } else {
#pragma unroll
        for (int i = 0; i < V / 2; i += 2) {
            ulonglong2* const q = reinterpret_cast<ulonglong2*>(p + 2 * i);
            ulonglong2 t = make_ulonglong2(n[i].v, n[i + 1].v);
            if (more) t = make_ulonglong2(add2(q->x, t.x), add2(q->y, t.y));
            *q = t;
        }
    }
}

constexpr int kNormWarpThreads = 128;            // CTA of warp teams

// Most threads of a CTA: a CTA team has up to 8192 / (K * V) threads.
template <int SIZE, int V, int K>
constexpr int kNormThreads = SIZE ? kNormWarpThreads : 8192 / (K * V);
template <int SIZE>
constexpr int kTeamsHere = SIZE ? kNormWarpThreads / (SIZE ? SIZE : 1) : 1;

// What the kernels of both directions set up: scratch, barriers, the team, its columns, its pipe (teams of operands from `smem` on, zeros beyond the rows).
#define CUTOFF_NORM_TEAM(ARGS, OPERANDS)                                                                                          \
    extern __shared__ __align__(16) uint8_t dynamic[];                                                                           \
    __shared__ __align__(16) float scratch[Team<SIZE>::kScratch];                                                                \
    __shared__ __align__(8) uint64_t barriers[2 * kTeamsHere<SIZE>];                                                             \
    Team<SIZE> team(scratch);                                                                                                    \
    const Columns<SIZE, V, K> col(team, (ARGS).cols);                                                                            \
    const Columns<SIZE, V, GROUPS ? K : 0> gate_columns(team, (ARGS).cols);                                                      \
    const int team_here = SIZE ? threadIdx.x / (SIZE ? SIZE : 1) : 0;                                                            \
    const RowPipe<T, SIZE> pipe(OPERANDS, async::smem_u32(dynamic), async::smem_u32(barriers), team_here);                       \
    if (team.rank() == 0) pipe.open();                                                                                           \
    if constexpr (V > 1)                                                                                                         \
        for (int s = 0; s < (OPERANDS).stages * (OPERANDS).n; ++s)                                                               \
            _Pragma("unroll") for (int k = 0; k < K; ++k)                                                                        \
                if (!col.has(k)) asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(pipe.slots + s * (OPERANDS).slot_bytes + col(k) * static_cast<int>(sizeof(T))), "r"(0) : "memory"); \
    async::fence_proxy_async();                                                                                                  \
    __syncthreads();

// A pack of an operand; single values beyond the row, or of a row that the team does not have, are zeros (packs beyond the row are zeros in shared memory).
// columns: of the row, or none.
template <typename T, int V, int SIZE, int K>
__device__ __forceinline__ void take(uint32_t row_at, const Columns<SIZE, V, K>& col, int k, int columns, Num<V> (&f)[kNums<V>]) {
    read_shared<T, V, V == 1 || SIZE != 0>(row_at + col(k) * static_cast<int>(sizeof(T)), col(k), columns, f);
}

// act(gate) of a group of rows, in shared memory, formed when a team that goes through the rows in their order comes to the group: a thread
// writes and reads its own columns.  Zeros beyond the row (where an infinite gate would turn zeros into NaN).
template <typename T, int V, int K, int SIZE>
struct GroupGate {
    uint32_t at;                    // this team's [columns of all its threads] fp32
    const Columns<SIZE, V, K>& col;
    int group;
    __device__ __forceinline__ GroupGate(uint32_t smem, int team_here, const Team<SIZE>& team, const Columns<SIZE, V, K>& c)
        : at(smem + team_here * team.size() * V * K * 4), col(c), group(-1) {
        put([](int, Num<V> (&u)[kNums<V>]) {      // a team without rows has zeros
#pragma unroll
            for (int i = 0; i < kNums<V>; ++i) u[i] = splat<Num<V>>(0.f);
        });
    }
    template <typename F>
    __device__ __forceinline__ void put(F f) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            Num<V> u[kNums<V>];
            f(k, u);
            if constexpr (V == 1) {
                asm volatile("st.shared.f32 [%0], %1;" ::"r"(at + 4 * col(k)), "f"(u[0].v) : "memory");
            } else {
#pragma unroll
                for (int i = 0; i < V / 2; i += 2) asm volatile("st.shared.v2.b64 [%0], {%1, %2};" ::"r"(at + 4 * col(k) + 8 * i), "l"(u[i].v), "l"(u[i + 1].v) : "memory");
            }
        }
    }
    __device__ __forceinline__ void turn_to(int g, const NormArgs& a) {
        if (g == group) return;
        group = g;
        const T* const row = static_cast<const T*>(a.gate) + g * a.gate_ld;
        with_gate(a.gate_kind, [&](auto kind) {
            put([&](int k, Num<V> (&u)[kNums<V>]) {
                read_global<T, V>(row + (col.has(k) ? col(k) : 0), u);
                gate_values<kExactGate<T>, decltype(kind)::value, false>(u, u);
                if (!col.has(k))
#pragma unroll
                    for (int i = 0; i < kNums<V>; ++i) u[i] = splat<Num<V>>(0.f);
            });
        });
    }
    __device__ __forceinline__ void get(int k, Num<V> (&f)[kNums<V>]) const { read_shared_params<V>(at + 4 * col(k), f); }
};
// Rows of team t where the teams' rows are consecutive.
__device__ __forceinline__ int first_row_of(int t, int teams, int rows) { return rows / teams * t + min(t, rows % teams); }
// The team that has a row.
__device__ __forceinline__ int team_of(int row, int teams, int rows) {
    const int each = rows / teams, more = rows % teams;        // the first `more` teams have a row more
    return row < more * (each + 1) ? row / (each + 1) : more + (row - more * (each + 1)) / each;
}
// Rows of a team.  With groups of rows they are consecutive, so that a group's gate and its gradient stay with few teams; otherwise the teams take
// turns, so that what is read and written at a time lies together (16384 rows of 4096 bf16 values with gate: 106 us, consecutive rows 150).
template <bool GROUPS>
struct TeamRows {
    int first, last, step;
    __device__ __forceinline__ TeamRows(int t, int teams, int rows)
        : first(GROUPS ? first_row_of(t, teams, rows) : t), last(GROUPS ? first_row_of(t + 1, teams, rows) : rows), step(GROUPS ? 1 : teams) {}
    __device__ __forceinline__ int operator()(int turn) const { return first + turn * step; }     // rows are few enough (kMostRows) for the turns behind the last
    __device__ __forceinline__ bool has(int turn) const { return (*this)(turn) < last; }
};

// Registers of a forward thread: with 16 values and their parameters 80, three CTAs of 256 threads per SM.  With biases 96, and the form of odd rows with
// layer norms and groups still spills 144 bytes per thread, warp teams of 16 single values up to 308.
template <int V, int K, bool MORE>
constexpr int kNormRegisters = V * K > 8 ? (MORE ? 96 : 80) : (MORE ? 80 : 64);

// The parameters of a thread's columns stay in its registers.
template <typename T, int V, int K, int SIZE, bool LAYER, bool BIAS, bool GROUPS>
__global__ void __maxnreg__((kNormRegisters<V, K, BIAS>)) k_residual_norm(NormArgs a, const __grid_constant__ RowOperands operands, int gate_bytes, bool few) {
    using N = Num<V>;
    constexpr int M = kNums<V>, kBias = BIAS ? K : 1;
    CUTOFF_NORM_TEAM(a, operands)
    // With at most a CTA per SM (few) the successor, a product of few tokens perhaps, may set itself up meanwhile; the CTAs of a large one would crowd on some SMs.
    if (few) launch_dependents();
    const int at_h = 1, at_gate = 2;
    const int t = blockIdx.x * kTeamsHere<SIZE> + team_here, teams = gridDim.x * kTeamsHere<SIZE>;
    const TeamRows<GROUPS> rows(t, teams, a.rows);
    const int turns = ceil_div(a.rows, teams);                 // the same for all teams of a warp: its shuffles take all lanes
    bool failed = false;                          // a wait gave up: none is made after it, and nothing is asked for
    for (int s = 0; s < operands.stages; ++s)
        if (rows.has(s)) pipe.fetch(s, rows(s), team);
    GroupGate<T, V, GROUPS ? K : 0, SIZE> group_gate(async::smem_u32(dynamic) + gate_bytes, team_here, team, gate_columns);
    N post_w[K][M], pre_w[K][M], post_b[kBias][M] = {}, pre_b[kBias][M] = {};       // the block's scale is part of the first and the third
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
        for (int i = 0; i < M; ++i) post_w[k][i] = pre_w[k][i] = splat<N>(col.has(k) ? 1.f : 0.f);
        if (!col.has(k)) continue;
        multiply<V>(post_w[k], a.post_w, col(k));
        multiply<V>(post_w[k], a.scale, col(k));
        multiply<V>(pre_w[k], a.pre_w, col(k));
        if constexpr (BIAS) {
            add_to<V>(post_b[k], a.post_b, col(k));
            multiply<V>(post_b[k], a.scale, col(k));
            add_to<V>(pre_b[k], a.pre_b, col(k));
        }
    }
    for (int turn = 0; turn < turns; ++turn) {
        const int row = rows(turn);
        const int stage = operands.stages == 2 ? turn & 1 : 0;
        const bool mine = rows.has(turn);         // a warp's teams may have a row more or less
        const int columns = !SIZE || mine ? a.cols : 0;
        if (!SIZE && !mine) break;
        if constexpr (GROUPS)
            if (mine) group_gate.turn_to(row / a.gate_rows, a);
        failed = failed || (mine && !pipe.wait(turn));
        const uint32_t x_at = pipe.template row_at<V>(stage, 0, row);
        N r[K][M];
        if (a.h) {
            const uint32_t h_at = pipe.template row_at<V>(stage, at_h, row);
#pragma unroll
            for (int k = 0; k < K; ++k) take<T, V>(h_at, col, k, columns, r[k]);
            mark<V, K>(failed, r);
            normalise<LAYER, SIZE, V, K>(r, team, col, a.post, a.eps, a.inv_cols);
            T* const r_row = static_cast<T*>(a.r) + row * a.r_ld;
            const int r_columns = a.r ? columns : 0;
            const uint32_t gate_at = !GROUPS && a.gate ? pipe.template row_at<V>(stage, at_gate, row) : 0u;
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < M; ++i) r[k][i] = BIAS ? fma(r[k][i], post_w[k][i], post_b[BIAS ? k : 0][i]) : mul(r[k][i], post_w[k][i]);
            const auto add_x = [&](int k, const N (&t)[M]) {              // r = x + t r, and out it goes
                N x[M];
                take<T, V>(x_at, col, k, columns, x);
#pragma unroll
                for (int i = 0; i < M; ++i) r[k][i] = fma(r[k][i], t[i], x[i]);
                write_global<T, V>(r_row, col(k), r_columns, r[k]);
            };
            if constexpr (GROUPS) {
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    N t[M];
                    group_gate.get(k, t);
                    add_x(k, t);
                }
            } else if (a.gate) {
                with_gate(a.gate_kind, [&](auto kind) {
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        N t[M];
                        take<T, V>(gate_at, col, k, columns, t);
                        gate_values<kExactGate<T>, decltype(kind)::value, false>(t, t);
                        add_x(k, t);
                    }
                });
            } else {
                N one[M];
#pragma unroll
                for (int i = 0; i < M; ++i) one[i] = splat<N>(1.f);
#pragma unroll
                for (int k = 0; k < K; ++k) add_x(k, one);
            }
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k) take<T, V>(x_at, col, k, columns, r[k]);
            mark<V, K>(failed, r);
        }
        // this row's values have been used, by all of the team
        if (turn + operands.stages < turns) {
            team.sync();
            if (!failed && rows.has(turn + operands.stages)) pipe.fetch(stage, rows(turn + operands.stages), team);
        }
        if (!a.n) continue;
        normalise<LAYER, SIZE, V, K>(r, team, col, a.pre, a.eps, a.inv_cols);
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < M; ++i) r[k][i] = BIAS ? fma(r[k][i], pre_w[k][i], pre_b[BIAS ? k : 0][i]) : mul(r[k][i], pre_w[k][i]);
        if (!a.n_scale) {
            T* const n_row = static_cast<T*>(a.n) + row * a.n_ld;
#pragma unroll
            for (int k = 0; k < K; ++k) write_global<T, V>(n_row, col(k), columns, r[k]);
            continue;
        }
        uint32_t top = 0;                         // beyond the row everything is zero, the parameters too
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < M; ++i) each(r[k][i], [&](float v) { top = max(top, magnitude_bits(v)); return v; });
        const RowScale q = row_scale(team.top(top));
        if (!mine) continue;
        if (team.rank() == 0) a.n_scale[row] = q.scale;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (!col.has(k)) continue;
            float f[V];
            if constexpr (V == 1) f[0] = r[k][0].v;
            else
#pragma unroll
                for (int i = 0; i < M; ++i) unpack2(r[k][i].v, f[2 * i], f[2 * i + 1]);
            store_quantised<V>(static_cast<int8_t*>(a.n) + row * a.n_ld + col(k), f, q.inverse);
        }
    }
    if (failed) pipe.drain();
}

// ---- backward ----------------------------------------------------------------------------------------------------------
struct NormGradArgs {
    NormArgs f;
    const void *d_r, *d_n;                        // either may be null
    int64_t d_r_ld, d_n_ld;
    void *d_x, *d_h, *d_gate;                     // each may be null
    int64_t d_x_ld, d_h_ld, d_gate_ld;
    float* sums;                                  // [CTAs][2 or 4][cols]: sum e * hat, sum d_n * r_hat, with BIAS also sum e, sum d_n
    float* gate_sums;                             // [CTAs][2][cols]: of the CTA's first and last group, where another CTA has the rest
    int teams;
    int gate_bytes;                               // offset in shared memory of the teams' group gates
    int param_bytes;                              // offset in shared memory of the parameters: scale * post_w, pre_w, with BIAS scale * post_b
    int part_bytes;                               // offset in shared memory of [teams here][2][columns of a team's threads]: as gate_sums, of warp teams
};
constexpr int kGradThreads = 512;                 // most threads of a CTA: 128 registers each
constexpr int kGradThreadsMany = 384;             // with 16 values and many sums: 168, where the row allows it
// CTAs of warp teams per SM: 128 registers for each thread, 168 with 16 values and many sums.
template <int VALUES, bool MORE>
constexpr int kGradWarpCtas = VALUES > 8 && MORE ? 3 : 4;

// Of a group of rows and a range of them: the group of a row, where it starts and ends.
struct Group {
    int64_t start, end;
    int at;
    __device__ __forceinline__ Group(int row, const NormArgs& a)
        : start(static_cast<int64_t>(row / a.gate_rows) * a.gate_rows), end(min(start + a.gate_rows, static_cast<int64_t>(a.rows))), at(row / a.gate_rows) {}
};
// The gradient of a group's gate in column c, given the sum over the group's rows.
template <typename T>
__device__ __forceinline__ void finish_gate(const NormGradArgs& g, int group, int c, float sum) {
    const NormArgs& a = g.f;
    F1 u[1] = {F1{to_float(static_cast<const T*>(a.gate)[group * a.gate_ld + c])}}, slope[1];
    with_gate(a.gate_kind, [&](auto kind) { gate_values<kExactGate<T>, decltype(kind)::value, true>(u, slope); });
    from_float(static_cast<T*>(g.d_gate)[group * g.d_gate_ld + c], sum * slope[0].v);
}
// The parts that a CTA's warp teams have of groups that they share, in the teams' order: the gradient where the whole group is this CTA's, else this CTA's part.
// So a group of many short rows leaves a part per CTA and not one per team (200000 rows of 32 values under one gate: 18944 teams, 592 CTAs).
template <typename T>
__device__ __forceinline__ void add_parts(const NormGradArgs& g, const float* parts, int apart, int teams_here) {
    const NormArgs& a = g.f;
    const int t0 = blockIdx.x * teams_here, from = first_row_of(t0, g.teams, a.rows), to = first_row_of(t0 + teams_here, g.teams, a.rows);
    float* const mine = g.gate_sums + 2 * static_cast<int64_t>(blockIdx.x) * a.cols;
    for (int c = threadIdx.x; c < a.cols; c += blockDim.x) {
        float sum = 0.f;                          // of the group that the last team has not ended
        for (int i = 0; i < teams_here; ++i) {
            const int first = first_row_of(t0 + i, g.teams, a.rows), last = first_row_of(t0 + i + 1, g.teams, a.rows);
            if (first == last) break;             // teams without rows are all at the end
            const Group begun(first, a);
            if (begun.start < first) {
                sum += parts[2 * i * apart + c];
                if (begun.end <= last) {
                    if (begun.start >= from) finish_gate<T>(g, begun.at, c, sum);
                    else mine[c] = sum;
                }
            }
            const Group open(last - 1, a);
            if (open.start >= first && open.end > last) sum = parts[(2 * i + 1) * apart + c];
        }
        if (from == to) continue;
        const Group open(to - 1, a);
        if (open.end > to) mine[(open.start < from ? 0 : a.cols) + c] = sum;
    }
}

// GROUPS: a gate for each group of rows, whose gradient is a sum over them.  BIAS: either norm has one, so that the plain sums are needed.
// SHARED: the parameters are in shared memory (there is no room for them beside one row of five fp32 operands of 8192 values).
// THREADS: most threads of a CTA team, and so its registers.
template <typename T, int V, int K, int SIZE, bool BIAS, bool GROUPS, bool LAYER, bool SHARED, int THREADS>
__global__ void __launch_bounds__(SIZE ? kNormWarpThreads : THREADS, SIZE ? kGradWarpCtas<V * K, BIAS || GROUPS> : 1) k_residual_norm_grad(NormGradArgs g, const __grid_constant__ RowOperands operands) {
    using N = Num<V>;
    constexpr int M = kNums<V>;
    const NormArgs& a = g.f;
    CUTOFF_NORM_TEAM(a, operands)
    const int t = blockIdx.x * kTeamsHere<SIZE> + team_here;
    const TeamRows<GROUPS> rows(t, g.teams, a.rows);
    const int turns = ceil_div(a.rows, g.teams);               // the same for all teams of a warp: its shuffles take all lanes
    constexpr int kBias = BIAS ? K : 1, kGroups = GROUPS ? K : 1;
    GroupGate<T, V, GROUPS ? K : 0, SIZE> group_gate(async::smem_u32(dynamic) + g.gate_bytes, team_here, team, gate_columns);
    N e_hat[K][M] = {}, n_hat[K][M] = {}, e_sum[kBias][M] = {}, n_sum[kBias][M] = {}, gate_sum[kGroups][M] = {};

    // places of the operands in a stage
    const bool has_gate_rows = !GROUPS && a.gate != nullptr;
    const int at_h = 1, at_gate = at_h + (a.h != nullptr), at_r = at_gate + has_gate_rows, at_n = at_r + (g.d_r != nullptr);
    bool failed = false;                          // a wait gave up: none is made after it, and nothing is asked for
    for (int s = 0; s < operands.stages; ++s)
        if (rows.has(s)) pipe.fetch(s, rows(s), team);
    // the parameters: in the L1, beside the operands, there is no room for them
    const uint32_t params = async::smem_u32(dynamic) + g.param_bytes;
    const int param_cols = team.size() * V * K;               // zeros beyond the row
    const auto param_of = [&](int which, int k, N (&f)[M]) {
        if constexpr (SHARED) {
            read_shared_params<V>(params + 4 * (which * param_cols + col(k)), f);
        } else {
#pragma unroll
            for (int i = 0; i < M; ++i) f[i] = splat<N>(!col.has(k) || (which == 2 && !a.post_b) ? 0.f : 1.f);
            if (!col.has(k)) return;
            multiply<V>(f, which == 0 ? a.post_w : which == 1 ? a.pre_w : a.post_b, col(k));
            if (which != 1) multiply<V>(f, a.scale, col(k));
        }
    };
    if constexpr (SHARED) {
        if (team_here == 0) {                     // a thread of the first team writes its own columns, zeros beyond the row
            float* const p = reinterpret_cast<float*>(dynamic + g.param_bytes);
            N w[K][M], n[K][M], b[BIAS ? K : 1][M];
#pragma unroll
            for (int k = 0; k < K; ++k) {
#pragma unroll
                for (int i = 0; i < M; ++i) w[k][i] = n[k][i] = splat<N>(col.has(k) ? 1.f : 0.f);
                if constexpr (BIAS)
#pragma unroll
                    for (int i = 0; i < M; ++i) b[k][i] = splat<N>(0.f);
                if (!col.has(k)) continue;
                multiply<V>(w[k], a.post_w, col(k));
                multiply<V>(w[k], a.scale, col(k));
                multiply<V>(n[k], a.pre_w, col(k));
                if constexpr (BIAS) {
                    add_to<V>(b[k], a.post_b, col(k));
                    multiply<V>(b[k], a.scale, col(k));
                }
            }
#pragma unroll
            for (int k = 0; k < K; ++k) {
                write_floats<V>(p + col(k), w[k], false);
                write_floats<V>(p + param_cols + col(k), n[k], false);
                if constexpr (BIAS) write_floats<V>(p + 2 * param_cols + col(k), b[k], false);
            }
        }
    }
    __syncthreads();
    for (int turn = 0; turn < turns; ++turn) {
        const int row = rows(turn);
        const int stage = operands.stages == 2 ? turn & 1 : 0;
        const bool mine = rows.has(turn);
        const int columns = !SIZE || mine ? a.cols : 0;
        if (!SIZE && !mine) break;
        failed = failed || (mine && !pipe.wait(turn));
        const int group = GROUPS && mine ? row / a.gate_rows : 0;
        if constexpr (GROUPS)
            if (mine) group_gate.turn_to(group, a);
        const uint32_t gate_at = has_gate_rows ? pipe.template row_at<V>(stage, at_gate, row) : 0u;
        N hat[K][M], d[K][M];                     // d: the whole gradient at r
        float h_inv = 1.f;
        if (a.h) {
            const uint32_t h_at = pipe.template row_at<V>(stage, at_h, row);
#pragma unroll
            for (int k = 0; k < K; ++k) take<T, V>(h_at, col, k, columns, hat[k]);
            mark<V, K>(failed, hat);
            h_inv = normalise<LAYER, SIZE, V, K>(hat, team, col, a.post, a.eps, a.inv_cols);
        }
        const uint32_t d_r_at = g.d_r ? pipe.template row_at<V>(stage, at_r, row) : 0u;
        if (g.d_n) {
            N r[K][M];
            const uint32_t x_at = pipe.template row_at<V>(stage, 0, row), d_n_at = pipe.template row_at<V>(stage, at_n, row);
            if (a.h) {
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    N w[M];
                    param_of(0, k, w);
#pragma unroll
                    for (int i = 0; i < M; ++i) r[k][i] = mul(w[i], hat[k][i]);
                    if constexpr (BIAS) {
                        param_of(2, k, w);
#pragma unroll
                        for (int i = 0; i < M; ++i) r[k][i] = add(r[k][i], w[i]);
                    }
                }
                const auto add_x = [&](int k, const N (&t)[M]) {          // r = x + t r
                    N x[M];
                    take<T, V>(x_at, col, k, columns, x);
#pragma unroll
                    for (int i = 0; i < M; ++i) r[k][i] = fma(r[k][i], t[i], x[i]);
                };
                if constexpr (GROUPS) {
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        N t[M];
                        group_gate.get(k, t);
                        add_x(k, t);
                    }
                } else if (a.gate) {
                    with_gate(a.gate_kind, [&](auto kind) {
#pragma unroll
                        for (int k = 0; k < K; ++k) {
                            N t[M];
                            take<T, V>(gate_at, col, k, columns, t);
                            gate_values<false, decltype(kind)::value, false>(t, t);      // a summand of r: what counts is its absolute error, 2 u at most
                            add_x(k, t);
                        }
                    });
                } else {
                    N one[M];
#pragma unroll
                    for (int i = 0; i < M; ++i) one[i] = splat<N>(1.f);
#pragma unroll
                    for (int k = 0; k < K; ++k) add_x(k, one);
                }
            } else {
#pragma unroll
                for (int k = 0; k < K; ++k) take<T, V>(x_at, col, k, columns, r[k]);
            }
            if (SIZE != 0 && !mine)               // a bias would be left of a row that there is not
#pragma unroll
                for (int k = 0; k < K; ++k)
#pragma unroll
                    for (int i = 0; i < M; ++i) r[k][i] = splat<N>(0.f);
            const float r_inv = normalise<LAYER, SIZE, V, K>(r, team, col, a.pre, a.eps, a.inv_cols);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                take<T, V>(d_n_at, col, k, columns, d[k]);
#pragma unroll
                for (int i = 0; i < M; ++i) {
                    n_hat[k][i] = fma(d[k][i], r[k][i], n_hat[k][i]);
                    if constexpr (BIAS) n_sum[k][i] = add(n_sum[k][i], d[k][i]);
                }
                N w[M];
                param_of(1, k, w);
#pragma unroll
                for (int i = 0; i < M; ++i) d[k][i] = mul(d[k][i], w[i]);
            }
            through_norm<LAYER, SIZE, V, K>(d, r, r_inv, team, a.pre, a.inv_cols);
            if (g.d_r) {
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    N dr[M];
                    take<T, V>(d_r_at, col, k, columns, dr);
#pragma unroll
                    for (int i = 0; i < M; ++i) d[k][i] = add(d[k][i], dr[i]);
                }
            }
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k) take<T, V>(d_r_at, col, k, columns, d[k]);
        }
        mark<V, K>(failed, d);
        {
            T* const out = static_cast<T*>(g.d_x) + row * g.d_x_ld;
            const int x_columns = g.d_x ? columns : 0;
#pragma unroll
            for (int k = 0; k < K; ++k) write_global<T, V>(out, col(k), x_columns, d[k]);
        }
        if (a.h) {
            // e = d act(gate) and the gradient at the branch's hat; w is scale * post_w, zero beyond the row, whatever a layer norm's gradient left in d
            const auto at_hat = [&](int k, const N (&w)[M]) {
#pragma unroll
                for (int i = 0; i < M; ++i) {
                    e_hat[k][i] = fma(d[k][i], hat[k][i], e_hat[k][i]);
                    if constexpr (BIAS) e_sum[k][i] = add(e_sum[k][i], d[k][i]);
                    d[k][i] = mul(d[k][i], w[i]);
                }
            };
            // the branch behind its scale, scale * post(h), of which the gate's gradient is a multiple
            const auto branch_of = [&](int k, const N (&w)[M], N (&p)[M]) {
#pragma unroll
                for (int i = 0; i < M; ++i) p[i] = mul(hat[k][i], w[i]);
                if constexpr (BIAS) {
                    N b[M];
                    param_of(2, k, b);
#pragma unroll
                    for (int i = 0; i < M; ++i) p[i] = add(p[i], b[i]);
                }
            };
            if constexpr (GROUPS) {
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    N w[M], u[M], p[M];
                    param_of(0, k, w);
                    group_gate.get(k, u);
                    branch_of(k, w, p);
#pragma unroll
                    for (int i = 0; i < M; ++i) gate_sum[k][i] = fma(d[k][i], p[i], gate_sum[k][i]);
#pragma unroll
                    for (int i = 0; i < M; ++i) d[k][i] = mul(d[k][i], u[i]);
                    at_hat(k, w);
                }
            } else if (a.gate) {
                T* const gate_row = static_cast<T*>(g.d_gate) + row * g.d_gate_ld;
                const int gate_columns = g.d_gate ? columns : 0;
                with_gate(a.gate_kind, [&](auto kind) {
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        N w[M], u[M], slope[M], p[M];
                        param_of(0, k, w);
                        take<T, V>(gate_at, col, k, columns, u);
                        gate_values<kExactGate<T>, decltype(kind)::value, true>(u, slope);
                        branch_of(k, w, p);
#pragma unroll
                        for (int i = 0; i < M; ++i) slope[i] = mul(slope[i], mul(d[k][i], p[i]));
                        write_global<T, V>(gate_row, col(k), gate_columns, slope);
#pragma unroll
                        for (int i = 0; i < M; ++i) d[k][i] = mul(d[k][i], u[i]);
                        at_hat(k, w);
                    }
                });
            } else {
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    N w[M];
                    param_of(0, k, w);
                    at_hat(k, w);
                }
            }
        }
        // this row's values have been used, by all of the team
        if (turn + operands.stages < turns) {
            team.sync();
            if (!failed && rows.has(turn + operands.stages)) pipe.fetch(stage, rows(turn + operands.stages), team);
        }
        if (a.h) {
            if (g.d_h) {
                through_norm<LAYER, SIZE, V, K>(d, hat, h_inv, team, a.post, a.inv_cols);
                T* const out = static_cast<T*>(g.d_h) + row * g.d_h_ld;
#pragma unroll
                for (int k = 0; k < K; ++k) write_global<T, V>(out, col(k), columns, d[k]);
            }
            if constexpr (GROUPS) {
                // the last row of a group, or of this team: the sum is the gradient, or this team's part of it
                if (mine && (row + 1 == rows.last || (row + 1) / a.gate_rows != group)) {
                    const int64_t start = static_cast<int64_t>(group) * a.gate_rows, end = min(start + a.gate_rows, static_cast<int64_t>(a.rows));
                    const bool whole = start >= rows.first && end <= rows.last;
                    const int which = start < rows.first ? 0 : 1;
                    float* const part = SIZE ? reinterpret_cast<float*>(dynamic + g.part_bytes) + (2 * team_here + which) * param_cols
                                             : g.gate_sums + (2 * static_cast<int64_t>(blockIdx.x) + which) * a.cols;
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        if (col.has(k)) {
                            if (whole) {
                                N u[M], slope[M];
                                read_global<T, V>(static_cast<const T*>(a.gate) + group * a.gate_ld + col(k), u);
                                with_gate(a.gate_kind, [&](auto kind) { gate_values<kExactGate<T>, decltype(kind)::value, true>(u, slope); });
#pragma unroll
                                for (int i = 0; i < M; ++i) slope[i] = mul(slope[i], gate_sum[k][i]);
                                if (g.d_gate) write_global<T, V>(static_cast<T*>(g.d_gate) + group * g.d_gate_ld, col(k), a.cols, slope);
                            } else {
                                write_floats<V>(part + col(k), gate_sum[k], false);
                            }
                        }
#pragma unroll
                        for (int i = 0; i < M; ++i) gate_sum[k][i] = splat<N>(0.f);
                    }
                }
            }
        }
    }
    if (failed) pipe.drain();
    launch_dependents();                          // the kernel that adds the sums up may set itself up
    // this CTA's sums
    float* const out = g.sums + static_cast<int64_t>(blockIdx.x) * (BIAS ? 4 : 2) * a.cols;
    float* const column_sums = reinterpret_cast<float*>(dynamic);
    if constexpr (SIZE != 0) __syncthreads();     // nobody reads operands any more
    if constexpr (SIZE != 0 && GROUPS)
        if (g.d_gate) add_parts<T>(g, reinterpret_cast<const float*>(dynamic + g.part_bytes), param_cols, kTeamsHere<SIZE>);
    const auto put = [&](float* to, const N (&v)[K][M]) {
        if constexpr (SIZE == 0) {
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (col.has(k)) write_floats<V>(to + col(k), v[k], false);
        } else {
            for (int w = 0; w < kTeamsHere<SIZE>; ++w) {
                if (w == team_here)
#pragma unroll
                    for (int k = 0; k < K; ++k)
                        if (col.has(k)) write_floats<V>(column_sums + col(k), v[k], w > 0);
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
    int teams_here;                               // teams of a CTA
    int column_blocks;                            // the grid's first blocks: the parameters; the others: the groups' gates
    int groups;                                   // of rows under one gate
    int slices;                                   // of the CTAs that a group spans: a power of two up to kGateSlices
    float *d_scale, *d_post_w, *d_post_b, *d_pre_w, *d_pre_b;      // each may be null
};
constexpr int kFinishColumns = 8, kFinishSlices = 64;          // eight columns are a sector
constexpr int kFinishThreads = kFinishColumns * kFinishSlices;
constexpr int kGateSlices = 16;                   // 32 columns at a time then, four sectors
constexpr int kGateColumns = 4;                   // of a thread: a block finds out its CTAs by some ten divisions, which a block for each 512 columns paid too often (638 x 5248, 11 us)

// The parameters' gradients from the CTAs' sums (8 columns per block, the CTAs in 64 interleaved parts), and the gradients of gates whose rows
// several CTAs had.  Either is a tree of fixed shape over chains that are 1/64 and 1/16 of the CTAs long: one chain over all parts took 1.2 ms and lost
// eleven bits of a sum of 200000 rows of 32 values (18944 parts then).
template <typename T>
__global__ void __launch_bounds__(kFinishThreads) k_norm_grad_finish(NormFinishArgs q) {
    __shared__ float part[4][kFinishSlices / 4][kFinishColumns];
    __shared__ float gate_part[kGateColumns][kFinishThreads];
    const NormArgs& a = q.g.f;
    dependency_wait();
    if (static_cast<int>(blockIdx.x) >= q.column_blocks) {
        // a group, or where there are more groups than CTAs the one that a CTA has not ended, and some columns
        const int wide = kFinishThreads / q.slices, chunks = ceil_div(a.cols, kGateColumns * wide), at = static_cast<int>(blockIdx.x) - q.column_blocks;
        const int unit = at / chunks, c0 = at % chunks * kGateColumns * wide + threadIdx.x % wide, slice = threadIdx.x / wide;
        const bool by_group = q.groups <= q.ctas;
        int row, first = unit;
        if (by_group) {
            row = unit * a.gate_rows;
        } else {
            row = first_row_of((unit + 1) * q.teams_here, q.g.teams, a.rows) - 1;
            if (row < first_row_of(unit * q.teams_here, q.g.teams, a.rows)) return;       // a CTA without rows
        }
        const Group group(row, a);
        if (by_group) first = team_of(row, q.g.teams, a.rows) / q.teams_here;
        const int behind = first_row_of((first + 1) * q.teams_here, q.g.teams, a.rows);   // the CTA's last row, and one
        if (group.end <= behind || group.start < first_row_of(first * q.teams_here, q.g.teams, a.rows)) return;      // one CTA's, or begun by another
        const int last = team_of(static_cast<int>(group.end) - 1, q.g.teams, a.rows) / q.teams_here;
        float s[kGateColumns];
#pragma unroll
        for (int i = 0; i < kGateColumns; ++i) {
            const int c = c0 + i * wide;
            s[i] = slice == 0 && c < a.cols ? q.g.gate_sums[(2 * static_cast<int64_t>(first) + 1) * a.cols + c] : 0.f;
        }
#pragma unroll 2                                   // loads that wait for nothing
        for (int v = first + 1 + slice; v <= last; v += q.slices)
#pragma unroll
            for (int i = 0; i < kGateColumns; ++i)
                if (c0 + i * wide < a.cols) s[i] += q.g.gate_sums[2 * static_cast<int64_t>(v) * a.cols + c0 + i * wide];
        if (q.slices > 1) {
#pragma unroll
            for (int i = 0; i < kGateColumns; ++i) gate_part[i][threadIdx.x] = s[i];
            __syncthreads();
            if (slice != 0) return;
#pragma unroll
            for (int i = 0; i < kGateColumns; ++i)
                for (int j = 1; j < q.slices; ++j) s[i] += gate_part[i][j * wide + threadIdx.x];
        }
#pragma unroll
        for (int i = 0; i < kGateColumns; ++i)
            if (c0 + i * wide < a.cols) finish_gate<T>(q.g, group.at, c0 + i * wide, s[i]);
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
    // four slices share a warp
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        s[i] += __shfl_xor_sync(0xffffffffu, s[i], 8);
        s[i] += __shfl_xor_sync(0xffffffffu, s[i], 16);
    }
    if (slice % 4 == 0)
#pragma unroll
        for (int i = 0; i < 4; ++i) part[i][slice / 4][x] = s[i];
    __syncthreads();
    if (slice != 0 || c >= a.cols) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        s[i] = 0.f;
#pragma unroll
        for (int j = 0; j < kFinishSlices / 4; ++j) s[i] += part[i][j][x];
    }
    const float w = a.post_w ? a.post_w[c] : 1.f, b = a.post_b ? a.post_b[c] : 0.f, scale = a.scale ? a.scale[c] : 1.f;
    if (q.d_scale) q.d_scale[c] = fmaf(w, s[0], b * s[2]);
    if (q.d_post_w) q.d_post_w[c] = scale * s[0];
    if (q.d_post_b) q.d_post_b[c] = scale * s[2];
    if (q.d_pre_w) q.d_pre_w[c] = s[1];
    if (q.d_pre_b) q.d_pre_b[c] = s[3];
}

// The teams of a backward pass: their threads (32 lanes or fewer, or a CTA), the values of a thread, the CTAs.  A thread has sixteen values; its sums, two each,
// fit 128 registers, with groups or biases up to five, 168 (100000 rows of 512 fp16 values with groups: 178 us so, 217 with eight values and 128).  Rows of fp32
// values have eight, as shared memory holds few of them and 16 would leave a CTA half of its warps.
struct GradPlan {
    int lanes, values, threads, per_sm, per_cta, ctas, teams;         // per_cta: teams of a CTA
};
constexpr int kMostSms = 160, kMostTeamRows = 1024;          // a team adds at most this many rows in a row
inline GradPlan grad_plan(int rows, int cols, int type_size, bool many_sums, int sms) {
    GradPlan p;
    p.lanes = cols <= 32 ? 4 : cols <= 128 ? 16 : cols <= 512 ? 32 : 0;
    p.values = p.lanes ? (cols <= 256 ? 8 : 16) : type_size == 4 && cols <= 8 * kGradThreads ? 8 : 16;
    p.threads = p.lanes ? kNormWarpThreads : ceil_div(ceil_div(cols, p.values), 32) * 32;
    // by the registers; shared memory may allow fewer
    p.per_sm = p.lanes ? (p.values > 8 && many_sums ? kGradWarpCtas<16, true> : kGradWarpCtas<8, false>)
               : p.values > 8 && many_sums && p.threads <= kGradThreadsMany ? kGradThreadsMany / p.threads : kGradThreads / p.threads;
    p.per_cta = p.lanes ? p.threads / p.lanes : 1;
    const int few = ceil_div(rows, p.per_cta), many = ceil_div(few, kMostTeamRows), resident = (sms < kMostSms ? sms : kMostSms) * p.per_sm;
    p.ctas = resident < many ? many : resident;
    p.ctas = p.ctas < few ? p.ctas : few;
    p.teams = p.ctas * p.per_cta;
    return p;
}

// The launches (norm_launch.cuh), compiled once for each type.  packs: accesses of 16 bytes.
template <typename T>
bool run_norm(const NormArgs& a, bool packs, int sms, cudaStream_t s);
template <typename T>
bool run_norm_grad(NormFinishArgs& q, const GradPlan& plan, bool packs, bool bias, bool groups, int64_t finish_blocks, cudaStream_t s);

}  // namespace layers
}  // namespace cutoff
