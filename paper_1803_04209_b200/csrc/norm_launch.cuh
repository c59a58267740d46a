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

template <typename T, int V>
void launch_norm(const NormArgs& a, cudaStream_t s) {
    with_team<T, V>(a.cols, a.rows > 512, [&](auto v, auto k, auto size) {
        constexpr int VV = decltype(v)::value, K = decltype(k)::value, SIZE = decltype(size)::value;
        if constexpr (SIZE) {
            constexpr int kTeams = kNormWarpThreads / SIZE;
            k_residual_norm<T, VV, K, SIZE><<<static_cast<unsigned>(ceil_div64(a.rows, kTeams)), kNormWarpThreads, 0, s>>>(a);
        } else {
            k_residual_norm<T, VV, K, 0><<<static_cast<unsigned>(a.rows), team_threads(a.cols, VV * K), 0, s>>>(a);
        }
    });
}

template <typename T, int V, bool BIAS, bool GROUPS>
void launch_grad(const NormGradArgs& g, const GradPlan& plan, cudaStream_t s) {
    with_team<T, V>(g.f.cols, false, [&](auto v, auto k, auto size) {
        constexpr int VV = decltype(v)::value, K = decltype(k)::value, SIZE = decltype(size)::value;
        const int threads = SIZE ? kNormWarpThreads : team_threads(g.f.cols, VV * K);
        k_residual_norm_grad<T, VV, K, SIZE, BIAS, GROUPS><<<static_cast<unsigned>(plan.ctas), threads, SIZE ? g.f.cols * sizeof(float) : 0, s>>>(g);
    });
}

template <typename T>
void run_norm(const NormArgs& a, bool packs, cudaStream_t s) {
    if (packs) launch_norm<T, kPack<T>>(a, s);
    else launch_norm<T, 1>(a, s);
}

template <typename T>
void run_norm_grad(const NormFinishArgs& q, const GradPlan& plan, bool packs, bool bias, bool groups, int finish_blocks, cudaStream_t s) {
    const NormGradArgs& g = q.g;
    const auto run = [&](auto v) {
        constexpr int V = decltype(v)::value;
        if (bias && groups) launch_grad<T, V, true, true>(g, plan, s);
        else if (bias) launch_grad<T, V, true, false>(g, plan, s);
        else if (groups) launch_grad<T, V, false, true>(g, plan, s);
        else launch_grad<T, V, false, false>(g, plan, s);
    };
    if (g.f.rows > 0) {
        if (packs) run(std::integral_constant<int, kPack<T>>{});
        else run(std::integral_constant<int, 1>{});
    }
    if (finish_blocks > 0) launch_dependent(k_norm_grad_finish<T>, dim3(finish_blocks), dim3(kFinishColumns * kFinishSlices), 0, s, q);
}

}  // namespace layers
}  // namespace cutoff
