// Products of 8-bit integers on the tensor cores (tcgen05, kind::i8): exact 32-bit sums in tensor memory, scaled in the epilogue.
//
// Rows of b (the weights' output channels) are the M side of the instruction and so the lanes of tensor memory, rows of a (tokens) its N side: a warp's
// 32 lanes hold 32 neighbouring outputs of one token, and its stores are consecutive whatever the alignment of y.  Operands come by TMA as
// 128-byte-swizzled K-major blocks of 128 values; what lies beyond k or the last row reads as zeros.
//
// k_product_tile: one tile of 128 channels x BN tokens per CTA, for few tokens or outputs.  Then the weights' bytes bound it, and what
// counts is that all SMs stream: the K blocks of a tile are split over the CTAs of a cluster, which send their partial sums to one another's
// shared memory (integers: in any order the same) as bulk copies, each finishing its share of the tokens.  Measured, one token, 4096 x 4096 weights: split
// in four 8.5 us, whole 12.1; 48 tokens, 8192 x 8192: 19.7 and 28.9.  Tiles of 128 tokens are never split: the exchange costs more than it gives
// (256 tokens, 4096 x 4096: 18.8 us in two, 14.9 whole).
//
// k_product_pair: for many tokens and outputs.  A cluster of two CTAs works on tiles of 256 channels x 256 tokens with instructions that span both SMs
// (cta_group::2): each CTA brings in its own 128 channels and half of the tokens, 32 KB for each 128 values of k instead of 48, and keeps the
// sums of its own channels, twice 256 columns of tensor memory, so that one tile's epilogue runs under the next tile's products.
// Persistent; tiles are taken in blocks of kPairGroup rows of tiles, so that what runs at a time shares operands in the L2.  The tensor pipe bounds it:
// 8192 x 8192 x 8192 303 us, 3.6e15 operations a second, twice the bf16 rate of the library's products and a little more (one-SM tiles of 128 x 256, which
// stream half as much again, 431); back to back, under the power limit, 420.
//
// Every wait on an mbarrier is bounded as in the emission kernels.  The call has no status to write to: a tile whose wait gave up is NaN.
#pragma once
#include "int8_product.cuh"
#include "tcgen05.cuh"

namespace cutoff {
namespace layers {

using namespace cutoff::async;
using tc::elect_one;

constexpr int kProdM = 128;                       // channels per tile: lanes of tensor memory
constexpr int kProdK = 128;                       // values per K block: one 128-byte swizzle row
constexpr int kProdABytes = kProdM * kProdK;

// instruction descriptor: D = s32, A = B = s8, both K-major, N columns, M rows
__host__ __device__ constexpr uint32_t instr_desc_s8(uint32_t n, uint32_t m) { return (2u << 4) | (1u << 7) | (1u << 10) | ((n >> 3) << 17) | ((m >> 4) << 24); }

__device__ __forceinline__ void umma_s8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}

template <int BN>
struct ProductTile {
    static constexpr int kStageBytes = kProdABytes + BN * kProdK;
    // Two CTAs per SM for few tokens, so that one streams while the other starts or ends.
    static constexpr int kStages = BN <= 16 ? 5 : BN <= 32 ? 4 : BN <= 64 ? 3 : 6;
    static constexpr bool kSplits = BN <= 64;
    static constexpr int kColumns = BN < 32 ? 32 : BN;                       // tensor memory comes in powers of two from 32
    static constexpr int kThreads = 192;
    static constexpr int kExchangeBytes = kSplits ? kProdM * BN * 4 : 0;     // a tile's sums: they leave through the ring, which is empty by then, and arrive beside it
    static constexpr int kTailBytes = 256 + BN * 4;                          // barriers, flags; the tokens' scales
    static_assert(kExchangeBytes <= kStages * kStageBytes, "exchange");
    static constexpr size_t kSmemBytes = 1024 + kStages * kStageBytes + kExchangeBytes + kTailBytes;
};
constexpr int kMostSplits = 4;                    // a CTA's share is at least four tokens

// Barrier of the four epilogue warps; it takes whole warps, so their lanes meet first.
__device__ __forceinline__ void epilogue_sync() {
    __syncwarp();
    asm volatile("bar.sync 1, 128;" ::: "memory");
}

// Bulk copy from this CTA's shared memory to another's, counted on a barrier there.
__device__ __forceinline__ void bulk_to_cta(uint32_t cluster_dst, uint32_t src, uint32_t bytes, uint32_t cluster_bar) {
    asm volatile("cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(cluster_dst), "r"(src), "r"(bytes), "r"(cluster_bar) : "memory");
}

// Grid: channel tiles x token tiles x splits, a cluster of `splits` CTAs per tile.
template <typename T, int BN>
__global__ void __launch_bounds__(192) k_product_tile(const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_a, ProductArgs p,
                                                      int token_tiles, int splits) {
    using Tile = ProductTile<BN>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw), ring = (raw + 1023u) & ~1023u;
    uint8_t* const base = smem_raw + (ring - raw);
    int* const outbox = reinterpret_cast<int*>(base);
    int* const inbox = reinterpret_cast<int*>(base + Tile::kStages * Tile::kStageBytes);
    uint8_t* const tail = base + Tile::kStages * Tile::kStageBytes + Tile::kExchangeBytes;
    float* const token_scale = reinterpret_cast<float*>(tail + 256);
    const uint32_t bars = smem_u32(tail);
    const auto full = [&](int s) { return bars + 8 * s; };
    const auto empty = [&](int s) { return bars + 8 * (Tile::kStages + s); };
    const uint32_t acc_full = bars + 16 * Tile::kStages, arrived = acc_full + 8;
    volatile uint32_t* const tmem_slot = reinterpret_cast<volatile uint32_t*>(tail + 16 * Tile::kStages + 16);
    volatile int* const abort_flag = reinterpret_cast<volatile int*>(tail + 16 * Tile::kStages + 24);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int split = static_cast<int>(blockIdx.x) % splits, tile = static_cast<int>(blockIdx.x) / splits;
    const int n0 = tile / token_tiles * kProdM;
    const int64_t m0 = static_cast<int64_t>(tile % token_tiles) * BN;
    const int blocks = ceil_div(p.k, kProdK);
    const int first = static_cast<int>(static_cast<int64_t>(blocks) * split / splits), last = static_cast<int>(static_cast<int64_t>(blocks) * (split + 1) / splits);
    DevState* const none = nullptr;

    if (threadIdx.x == 0) {
        for (int s = 0; s < Tile::kStages; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        mbar_init(acc_full, 1);
        mbar_init(arrived, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        if (splits > 1) mbar_arrive_expect_tx(arrived, (splits - 1) * (Tile::kExchangeBytes / splits));      // the other CTAs' part of this one's share
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32(const_cast<uint32_t*>(tmem_slot))), "r"(Tile::kColumns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc::tc_fence_before();
    __syncthreads();
    if (splits > 1) tc::cluster_sync_all();       // the others' barriers are set up before anything reaches across
    tc::tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    dependency_wait();                            // a is an earlier kernel's, perhaps

    bool ok = true;
    if (warp == 0) {
        int s = 0;
        uint32_t phase = 0;
        int armed = 0;
        for (int kb = first; ok && kb < last; ++kb) {
            ok = mbar_wait(empty(s), phase ^ 1u, abort_flag, none);
            if (!ok) break;
            if (lane == 0) {
                const uint32_t dst = ring + s * Tile::kStageBytes;
                mbar_arrive_expect_tx(full(s), Tile::kStageBytes);
                tc::tma_load_2d(dst, &map_b, kb * kProdK, n0, full(s));
                tc::tma_load_2d(dst + kProdABytes, &map_a, kb * kProdK, static_cast<int>(m0), full(s));
            }
            __syncwarp();
            armed = kb - first + 1;
            if (++s == Tile::kStages) { s = 0; phase ^= 1u; }
        }
        // every copy has landed before the CTA leaves or its ring takes partial sums (if the products ran, all but the unread ones have)
        if (!ok)
            for (int b = armed > Tile::kStages ? armed - Tile::kStages : 0; b < armed; ++b) mbar_wait_quiet(full(b % Tile::kStages), (b / Tile::kStages) & 1u);
    } else if (warp == 1) {
        int s = 0;
        uint32_t phase = 0;
        for (int kb = first; ok && kb < last; ++kb) {
            ok = mbar_wait(full(s), phase, abort_flag, none);
            if (!ok) break;
            tc::tc_fence_after();
            if (elect_one()) {
                const uint32_t at = ring + s * Tile::kStageBytes;
                const uint64_t a_desc = tc::make_smem_desc(at), b_desc = tc::make_smem_desc(at + kProdABytes);
#pragma unroll
                for (int k = 0; k < kProdK / 32; ++k) umma_s8(tmem, a_desc + 2 * k, b_desc + 2 * k, instr_desc_s8(BN, kProdM), (kb - first) | k);
                tc::umma_commit(empty(s));
                if (kb == last - 1) tc::umma_commit(acc_full);
            }
            __syncwarp();
            if (++s == Tile::kStages) { s = 0; phase ^= 1u; }
        }
        if (!ok) {
            // no product is running when tensor memory is released (bounded)
            if (elect_one()) tc::umma_commit(acc_full);
            __syncwarp();
            mbar_wait_quiet(acc_full, 0u);
        }
        __syncwarp();
    } else {
        for (int c = threadIdx.x - 64; c < BN; c += 128) token_scale[c] = m0 + c < p.m ? p.a_scale[m0 + c] : 0.f;
        epilogue_sync();
        ok = mbar_wait(acc_full, 0u, abort_flag, none);
        tc::tc_fence_after();
    }
    const int quarter = warp & 3, channel = n0 + quarter * 32 + lane;
    const bool epilogue = warp >= 2, has_channel = epilogue && channel < p.n;
    const float b_scale = has_channel ? p.b_scale[channel] : 0.f, bias = has_channel && p.bias ? p.bias[channel] : 0.f;
    const uint32_t lanes = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
    const auto put = [&](int c, float v) {
        if (has_channel && m0 + c < p.m) from_float(static_cast<T*>(p.y)[(m0 + c) * p.y_ld + channel], v);
    };
    if (!Tile::kSplits || splits == 1) {
        if (epilogue) {
            const bool bad = !ok || *abort_flag;
#pragma unroll 2
            for (int c0 = 0; c0 < BN; c0 += 16) {
                uint32_t r[16];
                __syncwarp();                     // lanes without a channel went on earlier
                tc::tmem_ld16(lanes + c0, r);
                tc::tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 16; ++i) put(c0 + i, bad ? __int_as_float(0x7fc00000) : scaled(static_cast<int>(r[i]), token_scale[c0 + i], b_scale, bias));
            }
        }
    } else {
        // Token c of the tile belongs to CTA c / share.  Sums lie as [four tokens][channel][token], so that a lane writes and reads 16 bytes beside
        // its neighbour's and a share is one piece.
        const int share = BN / splits, piece = share * kProdM;
        if (epilogue) {
            const int lane_at = (quarter * 32 + lane) * 4;
            const bool good = !__any_sync(0xffffffffu, !ok || *abort_flag);      // one answer for the warp: reading tensor memory takes all lanes
            if (good) {
#pragma unroll 2
                for (int c0 = 0; c0 < BN; c0 += 16) {
                    uint32_t r[16];
                    tc::tmem_ld16(lanes + c0, r);
                    tc::tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 16; i += 4)
                        *reinterpret_cast<uint4*>(outbox + (c0 + i) * kProdM + lane_at) = make_uint4(r[i], r[i + 1], r[i + 2], r[i + 3]);
                }
                fence_proxy_async();
            }
            epilogue_sync();
            const bool sent = !__any_sync(0xffffffffu, !good || *abort_flag);    // all four warps' sums are in the outbox: one that gave up has set the flag
            const int to = threadIdx.x - 64;      // one thread per receiver; a CTA that gave up sends nothing, and the others' waits will too
            if (sent && to < splits && to != split)
                bulk_to_cta(tc::map_to_cta(smem_u32(inbox + split * piece), to), smem_u32(outbox + to * piece), piece * 4, tc::map_to_cta(arrived, to));
            const bool all = mbar_wait(arrived, 0u, abort_flag, none) && sent;
            for (int c = 0; c < share; c += 4) {
                int4 total = *reinterpret_cast<const int4*>(outbox + split * piece + c * kProdM + lane_at);
                for (int r = 0; r < splits; ++r) {
                    if (r == split) continue;
                    const int4 t = *reinterpret_cast<const int4*>(inbox + r * piece + c * kProdM + lane_at);
                    total.x += t.x; total.y += t.y; total.z += t.z; total.w += t.w;
                }
                const int v[4] = {total.x, total.y, total.z, total.w};
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    put(split * share + c + i, all ? scaled(v[i], token_scale[split * share + c + i], b_scale, bias) : __int_as_float(0x7fc00000));
            }
        }
        tc::cluster_sync_all();                   // nobody leaves while its sums are on their way
    }
    tc::tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc::tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(Tile::kColumns) : "memory");
    }
}

// ---- pairs of SMs ------------------------------------------------------------------------------------------------------
constexpr int kPairTokens = 256;                  // tokens per tile; each CTA brings in half of them
constexpr int kPairStageBytes = kProdABytes + kPairTokens / 2 * kProdK;
constexpr int kPairStages = 6;
constexpr int kPairEpiWarps = 8;
constexpr int kPairThreads = (2 + kPairEpiWarps) * 32;
constexpr int kPairGroup = 8;
constexpr int kPairTail = 256 + kPairEpiWarps * 128 * 4;                    // barriers, flags; the tokens' scales of each epilogue warp
constexpr size_t kPairSmem = 1024 + kPairStages * kPairStageBytes + kPairTail;

__device__ __forceinline__ void umma_s8_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}

// Tile t of the order: blocks of kPairGroup channel tiles, within a block token tile by token tile.
struct PairTile {
    int channels, tokens;
};
__device__ __forceinline__ PairTile pair_tile(int t, int channel_tiles, int token_tiles) {
    const int block = t / (kPairGroup * token_tiles), first = block * kPairGroup, rows = min(kPairGroup, channel_tiles - first);
    const int in = t - first * token_tiles;
    return PairTile{first + in % rows, in / rows};
}

template <typename T>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
k_product_pair(const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_a, ProductArgs p, int channel_tiles, int token_tiles) {
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw), ring = (raw + 1023u) & ~1023u;
    uint8_t* const tail = smem_raw + (ring - raw) + kPairStages * kPairStageBytes;
    const uint32_t bars = smem_u32(tail);
    const auto full = [&](int s) { return bars + 8 * s; };                              // the leader's is the one used
    const auto empty = [&](int s) { return bars + 8 * (kPairStages + s); };
    const auto acc_full = [&](int b) { return bars + 8 * (2 * kPairStages + b); };
    const auto acc_empty = [&](int b) { return bars + 8 * (2 * kPairStages + 2 + b); };
    const auto peer_free = [&](int b) { return bars + 8 * (2 * kPairStages + 4 + b); }; // the leader's: the peer's epilogue has emptied accumulator b
    const uint32_t drain = bars + 8 * (2 * kPairStages + 6);
    volatile uint32_t* const tmem_slot = reinterpret_cast<volatile uint32_t*>(tail + 8 * (2 * kPairStages + 7));
    volatile int* const abort_flag = reinterpret_cast<volatile int*>(tail + 8 * (2 * kPairStages + 7) + 8);
    static_assert(8 * (2 * kPairStages + 7) + 16 <= 256, "barriers, tensor-memory address and abort flag");
    float* const scales = reinterpret_cast<float*>(tail + 256);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = tc::cluster_ctarank();
    const int cluster = blockIdx.x >> 1, clusters = gridDim.x >> 1, total = channel_tiles * token_tiles, blocks = ceil_div(p.k, kProdK);
    DevState* const none = nullptr;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kPairStages; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(acc_full(b), 1);
            mbar_init(acc_empty(b), kPairEpiWarps);
            mbar_init(peer_free(b), 1);
        }
        mbar_init(drain, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        tc::tmem_alloc_pair(smem_u32(const_cast<uint32_t*>(tmem_slot)), 512);
    }
    tc::tc_fence_before();
    __syncthreads();
    tc::cluster_sync_all();               // the peer's barriers and tensor memory exist before anything reaches across
    tc::tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    dependency_wait();

    if (warp == 0) {
        // both CTAs: their own 128 channels, their half of the tokens
        int s = 0;
        uint32_t phase = 0;
        const uint32_t leader_full = tc::map_to_cta(bars, 0u);
        bool ok = true;
        for (int t = cluster; ok && t < total; t += clusters) {
            const PairTile tile = pair_tile(t, channel_tiles, token_tiles);
            const int n0 = tile.channels * 2 * kProdM + static_cast<int>(rank) * kProdM, m0 = tile.tokens * kPairTokens + static_cast<int>(rank) * (kPairTokens / 2);
            for (int kb = 0; kb < blocks; ++kb) {
                ok = mbar_wait(empty(s), phase ^ 1u, abort_flag, none);
                if (!ok) break;
                if (lane == 0) {
                    const uint32_t dst = ring + s * kPairStageBytes, bar = leader_full + 8 * s;
                    // The leader expects the bytes of both CTAs; the peer's copies are counted there, if need be before they are expected.  (An
                    // arrival from the peer, a release across the cluster, takes its producer 0.8 us for each stage: 8192 x 8192 x 8192 718 us.)
                    if (rank == 0) mbar_arrive_expect_tx(full(s), 2 * kPairStageBytes);
                    tc::tma_load_2d_pair(dst, &map_b, kb * kProdK, n0, bar);
                    tc::tma_load_2d_pair(dst + kProdABytes, &map_a, kb * kProdK, m0, bar);
                }
                __syncwarp();
                if (++s == kPairStages) { s = 0; phase ^= 1u; }
            }
        }
        if (!ok) {
            // the copies still in flight land within microseconds; they get a bounded while
            const unsigned long long t0 = global_ns();
            while (global_ns() - t0 < 200000ull) {}
        }
    } else if (warp == 1 && rank != 0) {
        // the peer: tells the leader when its epilogue has emptied an accumulator
        int acc = 0;
        uint32_t phase = 0;
        bool ok = true;
        const uint32_t leader = tc::map_to_cta(peer_free(0), 0u);
        for (int t = cluster; ok && t < total; t += clusters) {
            ok = mbar_wait(acc_empty(acc), phase, abort_flag, none);
            if (!ok) break;
            if (lane == 0) mbar_arrive_cluster(leader + 8 * acc);
            __syncwarp();
            if (++acc == 2) { acc = 0; phase ^= 1u; }
        }
    } else if (warp == 1) {
        // the leader: issues the products of the pair
        int s = 0, acc = 0;
        uint32_t phase = 0, acc_phase = 0;
        bool ok = true;
        for (int t = cluster; ok && t < total; t += clusters) {
            ok = mbar_wait(acc_empty(acc), acc_phase ^ 1u, abort_flag, none) && mbar_wait(peer_free(acc), acc_phase ^ 1u, abort_flag, none);
            if (!ok) break;
            tc::tc_fence_after();
            const uint32_t d = tmem + acc * kPairTokens;
            for (int kb = 0; kb < blocks; ++kb) {
                ok = mbar_wait(full(s), phase, abort_flag, none);
                if (!ok) break;
                tc::tc_fence_after();
                if (elect_one()) {
                    const uint32_t at = ring + s * kPairStageBytes;
                    const uint64_t a_desc = tc::make_smem_desc(at), b_desc = tc::make_smem_desc(at + kProdABytes);
#pragma unroll
                    for (int k = 0; k < kProdK / 32; ++k) umma_s8_pair(d, a_desc + 2 * k, b_desc + 2 * k, instr_desc_s8(kPairTokens, 2 * kProdM), kb | k);
                    tc::umma_commit_pair(empty(s));
                    if (kb == blocks - 1) tc::umma_commit_pair(acc_full(acc));
                }
                __syncwarp();
                if (++s == kPairStages) { s = 0; phase ^= 1u; }
            }
            if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
        }
        if (!ok) {
            if (elect_one()) tc::umma_commit_pair(drain, 1);
            __syncwarp();
            mbar_wait_quiet(drain, 0u);
        }
        __syncwarp();
    } else {
        // both CTAs: a warp has 32 channels x 128 tokens
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        float* const scale = scales + (warp - 2) * 128;
        int acc = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (int t = cluster; t < total; t += clusters) {
            const PairTile tile = pair_tile(t, channel_tiles, token_tiles);
            const int channel = tile.channels * 2 * kProdM + static_cast<int>(rank) * kProdM + quarter * 32 + lane;
            const int64_t m0 = static_cast<int64_t>(tile.tokens) * kPairTokens + half * 128;
            const int here = static_cast<int>(p.m - m0 < 128 ? p.m - m0 : 128);          // tokens of this warp, none if it is <= 0
            const bool has = channel < p.n;
            __syncwarp();
            for (int i = lane; i < here; i += 32) scale[i] = p.a_scale[m0 + i];
            __syncwarp();
            const float b_scale = has ? p.b_scale[channel] : 0.f, bias = has && p.bias ? p.bias[channel] : 0.f;
            // after a wait that gave up the tiles that are left are marked, without another wait
            ok = ok && mbar_wait(acc_full(acc), phase, abort_flag, none);
            tc::tc_fence_after();
            const uint32_t lanes = tmem + (static_cast<uint32_t>(quarter * 32) << 16) + acc * kPairTokens + half * 128;
            T* const y = static_cast<T*>(p.y) + m0 * p.y_ld + channel;
#pragma unroll 1
            for (int c0 = 0; c0 < 128; c0 += 16) {
                uint32_t r[16];
                __syncwarp();                     // lanes without a channel went on earlier
                tc::tmem_ld16(lanes + c0, r);
                tc::tmem_ld_wait();
                if (c0 == 112 && ok) {
                    tc::tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(acc_empty(acc));
                }
                if (c0 >= here || !has) continue;
                float v[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] = ok ? scaled(static_cast<int>(r[i]), scale[c0 + i], b_scale, bias) : __int_as_float(0x7fc00000);
                if (c0 + 16 <= here) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) from_float(y[(c0 + i) * p.y_ld], v[i]);
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (c0 + i < here) from_float(y[(c0 + i) * p.y_ld], v[i]);
                }
            }
            if (++acc == 2) { acc = 0; phase ^= 1u; }
        }
    }
    tc::tc_fence_before();
    __syncthreads();
    tc::cluster_sync_all();               // neither CTA frees its tensor memory or leaves while the other may still reach it
    if (warp == 1) {
        tc::tc_fence_after();
        tc::tmem_free_pair(tmem, 512);
    }
}

}  // namespace layers
}  // namespace cutoff
