// Launches of the norm kernels for one element type: the team and the number of values per access by the rows' length and alignment.
#pragma once
#include <type_traits>

#include "launch.cuh"
#include "residual_norm.cuh"

namespace cutoff {
namespace layers {

// f(values per access, accesses per thread, lanes per row or 0 for a CTA): `wide` threads have 16 values of a row, the others eight.
template <typename T, int V, typename F>
void with_team(int cols, bool wide, F f) {
    using std::integral_constant;
    constexpr integral_constant<int, V> v{};
    constexpr integral_constant<int, 8 / V> eight{};
    constexpr integral_constant<int, 16 / V> sixteen{};
    if (cols <= 32) f(v, eight, integral_constant<int, 4>{});
    else if (cols <= 128) f(v, eight, integral_constant<int, 16>{});
    else if (cols <= 256) f(v, eight, integral_constant<int, 32>{});
    else if (cols <= 512) f(v, sixteen, integral_constant<int, 32>{});
    else if (wide) f(v, sixteen, integral_constant<int, 0>{});
    else f(v, eight, integral_constant<int, 0>{});
}
inline int team_threads(int cols, int per_thread) { return ceil_div(ceil_div(cols, per_thread), 32) * 32; }

// Most bytes of shared memory that the CTAs of an SM may take together for their operands.
constexpr int kNormSmem = 228 * 1024;

constexpr int kNormFixed = 2560;                  // what the system and static arrays take of a CTA, at most
// Most dynamic shared memory that any of these kernels is ever given (rows of 8192 fp32 values take 225 KB of it).
constexpr int kNormDynamic = kNormSmem - kNormFixed;

// Allows a kernel what it may ever need.  The limit belongs to the kernel on the device, whichever host thread sets it: a call that set its own size would
// lower it between another thread's setting and launch.
template <typename Kernel>
bool allow_smem(Kernel kernel, int bytes) {
    if (bytes <= 40 * 1024) return true;          // with static arrays, what every kernel may have
    return bytes <= kNormDynamic && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kNormDynamic) == cudaSuccess;
}

// CTAs of an SM and rows of a team in shared memory: `most` CTAs by their registers; two stages unless they do not fit even one CTA.
struct Staging {
    int per_sm, stages, bytes;
};
inline Staging staging(int most, int stage_bytes, int more_bytes) {
    Staging s{most, 2, 0};
    while (s.per_sm > 1 && s.per_sm * (2 * stage_bytes + more_bytes + kNormFixed) > kNormSmem) --s.per_sm;
    if (2 * stage_bytes + more_bytes + kNormFixed > kNormSmem) s.stages = 1;
    s.bytes = s.stages * stage_bytes + more_bytes;
    return s;
}

template <typename T, int V>
bool launch_norm(const NormArgs& a, int sms, cudaStream_t s) {
    bool ok = false;
    with_team<T, V>(a.cols, a.rows > 512 || a.cols > 4096, [&](auto v, auto k, auto size) {
        constexpr int VV = decltype(v)::value, K = decltype(k)::value, SIZE = decltype(size)::value, kSize = static_cast<int>(sizeof(T));
        const bool bias = a.post_b || a.pre_b, groups = a.gate && a.gate_rows > 1;
        const bool layer = a.post == kNormLayer || a.pre == kNormLayer;
        const auto kernel = bias && groups ? k_residual_norm<T, VV, K, SIZE, true, true, true> : bias ? k_residual_norm<T, VV, K, SIZE, true, true, false>
                            : groups ? k_residual_norm<T, VV, K, SIZE, true, false, true>
                            : layer  ? k_residual_norm<T, VV, K, SIZE, true, false, false> : k_residual_norm<T, VV, K, SIZE, false, false, false>;
        const int threads = SIZE ? kNormWarpThreads : team_threads(a.cols, VV * K);
        RowOperands ops{};
        const auto use = [&](const void* p, int64_t ld) { ops.o[ops.n++] = RowOperand{static_cast<const char*>(p), ld * kSize}; };
        use(a.x, a.x_ld);
        if (a.h) use(a.h, a.h_ld);
        if (a.gate && a.gate_rows == 1) use(a.gate, a.gate_ld);
        ops.row_bytes = a.cols * kSize;
        ops.slot_bytes = slot_bytes_of(ops.row_bytes, SIZE ? SIZE : threads, VV * K, kSize, VV > 1);
        const int stage = kTeamsHere<SIZE> * ops.n * ops.slot_bytes, by_registers = 65536 / (threads * (bias ? kNormRegisters<VV, K, true> : kNormRegisters<VV, K, false>)), most = by_registers < 16 ? by_registers : 16;
        const int ctas = ceil_div(a.rows, kTeamsHere<SIZE>);
        const int gate = groups ? kTeamsHere<SIZE> * (SIZE ? SIZE : threads) * VV * K * 4 : 0;
        Staging st = staging(most, stage, gate);
        if (ctas <= sms * st.per_sm) st.stages = 1, st.bytes = stage + gate;  // a row each
        ops.stages = st.stages;
        if (!allow_smem(kernel, st.bytes)) return;
        const int grid = ctas < sms * st.per_sm ? ctas : sms * st.per_sm;
        ok = launch_plain(kernel, dim3(grid), dim3(threads), st.bytes, s, a, ops, st.stages * stage, grid <= sms) == cudaSuccess;
    });
    return ok;
}

template <typename T, int V, bool BIAS, bool GROUPS>
bool launch_grad(NormFinishArgs& q, const GradPlan& plan, cudaStream_t s) {
    NormGradArgs& g = q.g;
    bool ok = false;
    const auto run = [&](auto k, auto size) {
        constexpr int K = decltype(k)::value, SIZE = decltype(size)::value, kSize = static_cast<int>(sizeof(T));
        RowOperands ops{};
        const auto use = [&](const void* p, int64_t ld) {
            if (p) ops.o[ops.n++] = RowOperand{static_cast<const char*>(p), ld * kSize};
        };
        use(g.f.x, g.f.x_ld);
        use(g.f.h, g.f.h_ld);
        if (!GROUPS) use(g.f.gate, g.f.gate_ld);
        use(g.d_r, g.d_r_ld);
        use(g.d_n, g.d_n_ld);
        ops.row_bytes = g.f.cols * kSize;
        ops.slot_bytes = slot_bytes_of(ops.row_bytes, SIZE ? SIZE : plan.threads, V * K, kSize, V > 1);
        const int stage = kTeamsHere<SIZE> * ops.n * ops.slot_bytes,
                  columns = (SIZE ? SIZE : plan.threads) * V * K, params = (BIAS ? 3 : 2) * 4 * columns, gate = GROUPS ? kTeamsHere<SIZE> * 4 * columns : 0, parts = SIZE ? 2 * gate : 0;
        // the plan's CTAs are resident by their registers; where shared memory holds fewer, the others follow
        Staging st = staging(plan.per_sm, stage, params + gate + parts);
        const bool layer = g.f.post == kNormLayer || g.f.pre == kNormLayer;
        // 168 registers where they are needed and the row's threads leave them
        constexpr int kThreads = V * K == 16 && (BIAS || GROUPS) ? kGradThreadsMany : kGradThreads;
        auto kernel = layer ? k_residual_norm_grad<T, V, K, SIZE, BIAS, GROUPS, true, true, kThreads> : k_residual_norm_grad<T, V, K, SIZE, BIAS, GROUPS, false, true, kThreads>;
        if constexpr (SIZE == 0 && kThreads < kGradThreads)
            if (plan.threads > kThreads)
                kernel = layer ? k_residual_norm_grad<T, V, K, SIZE, BIAS, GROUPS, true, true, kGradThreads>
                               : k_residual_norm_grad<T, V, K, SIZE, BIAS, GROUPS, false, true, kGradThreads>;
        if constexpr (sizeof(T) == 4 && V * K == 16 && SIZE == 0)
            if (st.bytes > 225 * 1024) {
                st.bytes -= params;
                kernel = layer ? k_residual_norm_grad<T, V, K, SIZE, BIAS, GROUPS, true, false, kGradThreads>
                               : k_residual_norm_grad<T, V, K, SIZE, BIAS, GROUPS, false, false, kGradThreads>;
            }
        ops.stages = st.stages;
        g.gate_bytes = st.stages * stage;
        g.param_bytes = st.stages * stage + gate;
        g.part_bytes = st.stages * stage + gate + params;
        const int sums = SIZE ? g.f.cols * 4 : 0;
        if (st.bytes < sums) st.bytes = sums;
        if (!allow_smem(kernel, st.bytes)) return;
        ok = launch_plain(kernel, dim3(plan.ctas), dim3(plan.threads), st.bytes, s, g, ops) == cudaSuccess;
    };
    using std::integral_constant;
    constexpr integral_constant<int, 8 / V> eight{};
    constexpr integral_constant<int, 16 / V> sixteen{};
    if (plan.lanes == 4) run(eight, integral_constant<int, 4>{});
    else if (plan.lanes == 16) run(eight, integral_constant<int, 16>{});
    else if (plan.lanes == 32 && plan.values == 8) run(eight, integral_constant<int, 32>{});
    else if (plan.lanes == 32) run(sixteen, integral_constant<int, 32>{});
    else if (plan.values == 8) {
        if constexpr (sizeof(T) == 4) run(eight, integral_constant<int, 0>{});
    } else run(sixteen, integral_constant<int, 0>{});
    return ok;
}

template <typename T>
bool run_norm(const NormArgs& a, bool packs, int sms, cudaStream_t s) { return packs ? launch_norm<T, kPack<T>>(a, sms, s) : launch_norm<T, 1>(a, sms, s); }

template <typename T>
bool run_norm_grad(NormFinishArgs& q, const GradPlan& plan, bool packs, bool bias, bool groups, int64_t finish_blocks, cudaStream_t s) {
    bool ok = true;
    const auto run = [&](auto v) {
        constexpr int V = decltype(v)::value;
        ok = bias && groups ? launch_grad<T, V, true, true>(q, plan, s)
             : bias         ? launch_grad<T, V, true, false>(q, plan, s)
             : groups       ? launch_grad<T, V, false, true>(q, plan, s)
                            : launch_grad<T, V, false, false>(q, plan, s);
    };
    if (q.g.f.rows > 0) {
        if (packs) run(std::integral_constant<int, kPack<T>>{});
        else run(std::integral_constant<int, 1>{});
    }
    // sums that no kernel has formed are not added up
    if (!ok || finish_blocks == 0) return ok;
    return launch_dependent(k_norm_grad_finish<T>, dim3(static_cast<unsigned>(finish_blocks)), dim3(kFinishThreads), 0, s, q) == cudaSuccess;
}

}  // namespace layers
}  // namespace cutoff
