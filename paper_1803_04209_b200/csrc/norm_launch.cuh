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
constexpr int kNormSmem = 220 * 1024;

template <typename T, int V>
bool launch_norm(const NormArgs& a, int sms, cudaStream_t s) {
    bool ok = false;
    with_team<T, V>(a.cols, a.rows > 512, [&](auto v, auto k, auto size) {
        constexpr int VV = decltype(v)::value, K = decltype(k)::value, SIZE = decltype(size)::value;
        const auto kernel = k_residual_norm<T, VV, K, SIZE>;
        const int threads = SIZE ? kNormWarpThreads : team_threads(a.cols, VV * K), teams = SIZE ? kNormWarpThreads / (SIZE ? SIZE : 1) : 1;
        const int stage = norm_operands(a) * K * threads * static_cast<int>(sizeof(Pack<T, VV>));
        // as many CTAs as fit the registers (64 for each of 1024 threads), two rows of each in shared memory, or one
        int per_sm = 1024 / threads, stages = 2;
        if (per_sm > 16) per_sm = 16;
        while (per_sm > 1 && per_sm * (2 * stage + 2048) > kNormSmem) --per_sm;
        if (2 * stage + 2048 > kNormSmem) stages = 1;
        const int ctas = ceil_div(a.rows, teams), resident = sms * per_sm;
        if (ctas <= resident) stages = 1;         // a row each
        const int smem = stages * stage;
        if (smem > 40 * 1024 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return;
        kernel<<<ctas < resident ? ctas : resident, threads, smem, s>>>(a, stages);
        ok = true;
    });
    return ok;
}

template <typename T, int V, bool BIAS, bool GROUPS>
bool launch_grad(NormFinishArgs& q, const GradPlan& plan, cudaStream_t s) {
    NormGradArgs& g = q.g;
    bool ok = false;
    const auto run = [&](auto k, auto size) {
        constexpr int K = decltype(k)::value, SIZE = decltype(size)::value;
        const auto kernel = k_residual_norm_grad<T, V, K, SIZE, BIAS, GROUPS>;
        const size_t stage = static_cast<size_t>(grad_operands<GROUPS>(g)) * K * plan.threads * sizeof(Pack<T, V>);
        g.stages = 2 * stage + 2048 <= kNormSmem ? 2 : 1;
        size_t smem = g.stages * stage;
        const size_t sums = SIZE ? g.f.cols * sizeof(float) : 0;
        if (smem < sums) smem = sums;
        if (smem > 40 * 1024 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)) != cudaSuccess) return;
        kernel<<<plan.ctas, plan.threads, smem, s>>>(g);
        ok = true;
    };
    using std::integral_constant;
    constexpr integral_constant<int, 8 / V> eight{};
    constexpr integral_constant<int, 16 / V> sixteen{};
    if (plan.lanes == 4) run(eight, integral_constant<int, 4>{});
    else if (plan.lanes == 16) run(eight, integral_constant<int, 16>{});
    else if (plan.lanes == 32 && plan.values == 8) run(eight, integral_constant<int, 32>{});
    else if (plan.lanes == 32) {
        if constexpr (!BIAS && !GROUPS) run(sixteen, integral_constant<int, 32>{});       // otherwise a CTA has the row
    } else if (plan.values == 8) {
        if constexpr (BIAS || GROUPS) run(eight, integral_constant<int, 0>{});
    } else run(sixteen, integral_constant<int, 0>{});
    return ok;
}

template <typename T>
bool run_norm(const NormArgs& a, bool packs, int sms, cudaStream_t s) { return packs ? launch_norm<T, kPack<T>>(a, sms, s) : launch_norm<T, 1>(a, sms, s); }

template <typename T>
bool run_norm_grad(NormFinishArgs& q, const GradPlan& plan, bool packs, bool bias, bool groups, int finish_blocks, cudaStream_t s) {
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
    if (ok && finish_blocks > 0) launch_dependent(k_norm_grad_finish<T>, dim3(finish_blocks), dim3(kFinishColumns * kFinishSlices), 0, s, q);
    return ok;
}

}  // namespace layers
}  // namespace cutoff
