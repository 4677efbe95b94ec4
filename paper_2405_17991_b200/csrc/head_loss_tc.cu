// The logits of a linear head on CTA pairs, used up where they come out of the tensor cores:
//   HEAD_STATS     per row and 128 columns the maximum and the sum of exponentials relative to it, and the target's logit
//   HEAD_GRADIENT  G[n, v] = g[n] (exp(l[n, v] - lse[n]) - [v = t[n]]) in bf16
//   DISTILL_STATS, DISTILL_GRADIENT  the same of logits over a temperature, with a list of columns and probabilities for a target (distill.cu)
// l = X W^T, bf16 operands K-major, 256 x 256 logits a pair (tcgen05 cta_group::2; the pipeline is that of gemm_tc2.cu).
//
// The tensor cores add with truncation, 16 products at a time: over D = 4096 that shrinks a logit by some 5e-6 of itself.  So a tile's
// contraction is cut into segments of 512 (kHeadSegment), each into an accumulator of its own (two, alternating), and the epilogue adds the segments
// up in registers, rounded to nearest: eight warps with 128 sums a thread.  The next segment's products run meanwhile.  Error of the loss
// in norm, 8192 x 4096 of 32000 columns: 7.1e-8 (segments of 1024: 1.3e-7).  Both passes do it: G = g (exp(l - lse) - 1) of a target whose share is
// near one has what its l and the l in lse differ by divided by 1 - p (one accumulator in the backward pass alone, D = 4096: rows of dX off by 1.4e-2 in
// the median at a loss of 1e-3 to 1e-2, by 0.3 below; now 1.9e-3 and 3.7e-3, the latter by lse's rounding to fp32).  8192 x 4096 of 32000, forward and
// backward: 1470 to 1520 + 5130 to 5310 us, 1420 to 1470 + 5040 to 5230 with segments of 1024 and one accumulator.
//
// Bound by the power limit and by what the operands' way from L2 costs of it: the statistics of 8192 x 4096 of 32000 (with segments of
// 1024) in bands of 4 row blocks 1728 us, 8: 1643, 16: 1615 (W crosses HBM twice, X stays in L2), 32: 1689.
//
// Roles per CTA (320 threads): warp 0 lane 0 TMA producer, warp 1 lane 0 MMA issuer (leader only), warps 2..9 epilogue: TMEM lanes
// 32 * (w % 4) .., columns 128 * (w >= 6) ...  Barriers as in gemm_tc2.cu.  Every wait is bounded; both CTAs reach the closing
// cluster barrier.
#include <cooperative_groups.h>

#include "gemm_store.cuh"
#include "gemm_tc.cuh"
#include "head_loss.cuh"
#include "tc_pair.cuh"

namespace velora {

using namespace tc;

namespace {

constexpr int H_BM = 128;                  // rows per CTA (256 per pair)
constexpr int H_BN = 256;                  // columns per pair; half of them staged by each CTA
constexpr int H_BK = 64;
constexpr int H_BAND = 16;                 // row blocks that are walked together
constexpr int H_STAGES = 6;
constexpr int H_A_BYTES = H_BM * H_BK * 2;
constexpr int H_STAGE_BYTES = H_A_BYTES + (H_BN / 2) * H_BK * 2;
constexpr int H_EPILOGUE_WARPS = 8;
constexpr int H_THREADS = 64 + 32 * H_EPILOGUE_WARPS;
constexpr int H_STAGING_BYTES = H_EPILOGUE_WARPS * kStoreBytes;
constexpr int H_BARRIER_BYTES = 256;
constexpr size_t H_SMEM = 1024 + static_cast<size_t>(H_STAGES) * H_STAGE_BYTES + H_STAGING_BYTES + H_BARRIER_BYTES;

enum HeadRole { HEAD_STATS = 0, HEAD_GRADIENT = 1, DISTILL_STATS = 2, DISTILL_GRADIENT = 3 };

// 32 values of a lane to and from 128 bytes of shared memory.
__device__ __forceinline__ void put_values(uint32_t turn, uint32_t swap, const uint32_t (&l)[32])
{
#pragma unroll
    for (int k = 0; k < 8; ++k)
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(turn + (16 * k ^ swap)), "r"(l[4 * k]), "r"(l[4 * k + 1]), "r"(l[4 * k + 2]), "r"(l[4 * k + 3]) : "memory");
}
__device__ __forceinline__ void get_values(uint32_t turn, uint32_t swap, uint32_t (&l)[32])
{
#pragma unroll
    for (int k = 0; k < 8; ++k)
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(l[4 * k]), "=r"(l[4 * k + 1]), "=r"(l[4 * k + 2]), "=r"(l[4 * k + 3]) : "r"(turn + (16 * k ^ swap)) : "memory");
}
__device__ __forceinline__ float ld_shared(uint32_t at)
{
    float x;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(at) : "memory");
    return x;
}
__device__ __forceinline__ void st_shared(uint32_t at, float x) { asm volatile("st.shared.f32 [%0], %1;" ::"r"(at), "f"(x) : "memory"); }

template <int ROLE>
__global__ void __launch_bounds__(H_THREADS, 1)
head_pair_kernel(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmG,
                 const HeadTile h, int* __restrict__ status)
{
    constexpr bool STORES = ROLE == HEAD_GRADIENT || ROLE == DISTILL_GRADIENT, LISTS = ROLE == DISTILL_STATS || ROLE == DISTILL_GRADIENT;
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    const uint32_t rank = cluster.block_rank();              // 0 = leader
    const int pair = blockIdx.x >> 1;
    const int num_pairs = gridDim.x >> 1;

    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    uint8_t* tail = smem_raw + (base - raw) + H_STAGES * H_STAGE_BYTES + H_STAGING_BYTES;
    const uint32_t staging = base + H_STAGES * H_STAGE_BYTES;
    const uint32_t full = staging + H_STAGING_BYTES, empty = full + 8 * H_STAGES;
    const uint32_t tfull = full + 16 * H_STAGES, tempty = tfull + 16;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(tail + 16 * H_STAGES + 48);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tail + 16 * H_STAGES + 56);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int kblocks = (h.D + H_BK - 1) / H_BK;
    const int live = *h.live;
    const int tiles_m = (live + 2 * H_BM - 1) / (2 * H_BM);          // rows without a target are not computed
    const int tiles_n = (h.cols + H_BN - 1) / H_BN;
    const int num_tiles = tiles_m * tiles_n;

    if (threadIdx.x == 0) {
        for (int s = 0; s < H_STAGES; ++s) {
            mbar_init(full + 8 * s, 1);                      // the leader's expect_tx arrival
            mbar_init(empty + 8 * s, 1);                     // the leader's commit
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(tfull + 8 * a, 1);
            mbar_init(tempty + 8 * a, 2 * H_EPILOGUE_WARPS); // the epilogue warps of both CTAs
        }
        *abort_flag = 0;
        fence_mbar_init();
        prefetch_tensormap(&tmX);
        prefetch_tensormap(&tmW);
        if (STORES) prefetch_tensormap(&tmG);
    }
    if (warp == 1) {
        tmem_alloc_pair(smem_u32(tmem_slot), 2 * H_BN);
        tmem_relinquish_pair();
    }
    tc_fence_before_sync();
    __syncthreads();
    cluster.sync();                                          // both CTAs' barriers exist before anyone signals them
    tc_fence_after_sync();
    const uint32_t tmem_base = *tmem_slot;

    bool failed = false;
    if (warp == 0) {
        // ------------------------------------------------ TMA producer: this CTA's rows of X, its half of W's
        if (lane == 0) {
            uint32_t it = 0;
            for (int tile = pair; tile < num_tiles && !failed; tile += num_pairs) {
                const PairTile t0 = pair_tile(tile, tiles_m, tiles_n, 2 * H_BM, H_BN, H_BAND);
                const int m0 = t0.m0 + static_cast<int>(rank) * H_BM;
                const int n0 = t0.n0 + static_cast<int>(rank) * (H_BN / 2);
                for (int kb = 0; kb < kblocks; ++kb, ++it) {
                    const uint32_t s = it % H_STAGES, ph = (it / H_STAGES) & 1u;
                    if (!mbar_wait(empty + 8 * s, ph ^ 1u, abort_flag)) { failed = true; break; }
                    const uint32_t lead_full = map_to_cta(full + 8 * s, 0);
                    if (rank == 0) mbar_arrive_expect_tx(full + 8 * s, 2 * H_STAGE_BYTES);
                    const uint32_t dst = base + s * H_STAGE_BYTES;
                    tma_load_2d_pair(dst, &tmX, lead_full, kb * H_BK, m0);
                    tma_load_2d_pair(dst + H_A_BYTES, &tmW, lead_full, kb * H_BK, n0);
                }
            }
            if (failed) {
                *abort_flag = 1;
                // Copies in flight land before shared memory is given up: the leader watches its barriers (each phase needs both
                // CTAs' bytes), the peer allows them 50 us.
                const unsigned long long t0 = globaltimer_ns();
                if (rank == 0) {
                    const uint32_t back = it < H_STAGES ? it : H_STAGES;
                    for (uint32_t j = 1; j <= back; ++j) {
                        const uint32_t jt = it - j;
                        while (!mbar_try_wait(full + 8 * (jt % H_STAGES), (jt / H_STAGES) & 1u))
                            if (globaltimer_ns() - t0 > kWaitLimitNs) break;
                    }
                } else {
                    while (globaltimer_ns() - t0 < 50000ull) __nanosleep(1000);
                }
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------ MMA issuer: the leader's lane 0 drives both tensor cores
        if (lane == 0 && rank == 0) {
            constexpr uint32_t idesc = umma_idesc_bf16(2 * H_BM, H_BN, false, false);
            uint32_t it = 0, seg = 0;
            for (int tile = pair; tile < num_tiles && !failed; tile += num_pairs) {
                for (int k0 = 0; k0 < kblocks && !failed; k0 += kHeadSegment, ++seg) {
                    const uint32_t acc = seg & 1u, aph = (seg >> 1) & 1u;
                    if (!mbar_wait(tempty + 8 * acc, aph ^ 1u, abort_flag)) { failed = true; break; }
                    tc_fence_after_sync();
                    const uint32_t d_tmem = tmem_base + acc * H_BN;
                    const int k1 = min(kblocks, k0 + kHeadSegment);
                    for (int kb = k0; kb < k1; ++kb, ++it) {
                        const uint32_t s = it % H_STAGES, ph = (it / H_STAGES) & 1u;
                        if (!mbar_wait(full + 8 * s, ph, abort_flag)) { failed = true; break; }
                        tc_fence_after_sync();
                        const uint32_t a_addr = base + s * H_STAGE_BYTES, b_addr = a_addr + H_A_BYTES;
#pragma unroll
                        for (int j = 0; j < H_BK / 16; ++j)
                            umma_bf16_pair(d_tmem, umma_smem_desc(a_addr + j * 32, 16, 1024), umma_smem_desc(b_addr + j * 32, 16, 1024), idesc,
                                           ((kb - k0) | j) != 0);
                        umma_commit_pair(empty + 8 * s);      // both CTAs may refill the stage
                    }
                    if (!failed) umma_commit_pair(tfull + 8 * acc);
                }
            }
            if (failed) *abort_flag = 1;
        }
    } else {
        // ------------------------------------------------ epilogue
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        const uint32_t lead_tempty = map_to_cta(tempty, 0);
        const uint32_t block = staging + (warp - 2) * kStoreBytes;
        uint32_t seg = 0;
        EntryPlace ahead;                                    // of the tile that comes next
        if (LISTS && pair < num_tiles) {
            const PairTile t0 = pair_tile(pair, tiles_m, tiles_n, 2 * H_BM, H_BN, H_BAND);
            const int row = t0.m0 + static_cast<int>(rank) * H_BM + quarter * 32 + lane, col0 = t0.n0 + half * 128;
            ahead.find_token(h.e, h.target, row, row < h.N && col0 < h.cols);
            ahead.find_entries(h.e, h.v0 + col0);
        }
        for (int tile = pair; tile < num_tiles && !failed; tile += num_pairs) {
            const PairTile t0 = pair_tile(tile, tiles_m, tiles_n, 2 * H_BM, H_BN, H_BAND);
            const int row0 = t0.m0 + static_cast<int>(rank) * H_BM + quarter * 32, row = row0 + lane;
            const int col0 = t0.n0 + half * 128, valid = h.cols - col0;
            uint32_t l[4][32];                               // fp32 bits
            EntryWalk walk;                                  // its first entries are on their way while the products run
            int col_ahead = 0;
            const bool part = LISTS && ahead.token >= 0;     // whether this row has any
            float g_row = 0.f, lse_row = 0.f, mass = 1.f;    // loaded before the products are waited for, with a list; without one behind them
            if (LISTS) {
                walk.none();
                if (part) {
                    walk.begin(h.e, ahead.token, ahead.j, ahead.end, h.v0 + col0);
                    if (STORES) {
                        g_row = h.scale[row];
                        lse_row = h.lse[row];
                        mass = h.e.mass[ahead.token];
                    }
                }
                if (tile + num_pairs < num_tiles) {
                    const PairTile t1 = pair_tile(tile + num_pairs, tiles_m, tiles_n, 2 * H_BM, H_BN, H_BAND);
                    const int row1 = t1.m0 + static_cast<int>(rank) * H_BM + quarter * 32 + lane;
                    col_ahead = t1.n0 + half * 128;
                    ahead.find_token(h.e, h.target, row1, row1 < h.N && col_ahead < h.cols);
                }
            }
            for (int k0 = 0; k0 < kblocks; k0 += kHeadSegment, ++seg) {
                const uint32_t acc = seg & 1u, aph = (seg >> 1) & 1u;
                if (!mbar_wait_warp(tfull + 8 * acc, aph, abort_flag, 256)) { failed = true; break; }
                tc_fence_after_sync();
                const uint32_t taddr = tmem_base + acc * H_BN + half * 128 + (static_cast<uint32_t>(quarter * 32) << 16);
                if (k0 > 0) {                                // 16 columns a step: the sums leave few registers
#pragma unroll
                    for (int c = 0; c < 16; c += 2) {
                        uint32_t r[2][8];
                        tmem_ld_32x8(taddr + c * 8, r[0]);
                        tmem_ld_32x8(taddr + c * 8 + 8, r[1]);
                        tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            uint32_t& y = l[c / 4][c % 4 * 8 + i];
                            y = __float_as_uint(__uint_as_float(y) + __uint_as_float(r[i / 8][i % 8]));
                        }
                    }
                } else {
#pragma unroll
                    for (int c = 0; c < 4; ++c) tmem_ld_32x32(taddr + c * 32, l[c]);
                    tmem_ld_wait();
                }
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(lead_tempty + 8 * acc);
            }
            if (LISTS) ahead.find_entries(h.e, h.v0 + col_ahead);
            if (failed || valid <= 0) continue;
            const bool in = row < h.N;
            // Logits are divided by the temperature where they go into an exponent.  What log2 e / T has lost by its rounding, and a maximum over T by its own, would
            // move a row's logits against its lse; sums and gradients make up for both (one column, l / T up to 3000, T = 1.1: G off by 1.4 times what
            // lse's rounding accounts for).
            const float log2e = LISTS ? kHeadLog2e * h.e.inverse_t : kHeadLog2e;
            // Entries: 32 of this lane's values through its 128 bytes of the warp's block of shared memory, 16 at a time in an order that keeps the lanes apart.
            const uint32_t turn = block + lane * 128, swap = (lane & 7) << 4;
            auto value = [&](int column) { return turn + ((static_cast<uint32_t>(column) << 2 & 0x70u) ^ swap) + (static_cast<uint32_t>(column) << 2 & 0xcu); };
            const int t = !LISTS && in ? h.target[row] - h.v0 - col0 : -1;                // in this warp's columns: 0 .. 127
            if (!STORES) {
                if (valid < 128) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (32 * c + i >= valid) l[c][i] = 0xff800000u;
                }
                float m = __uint_as_float(l[0][0]);
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int i = 0; i < 32; ++i) m = fmaxf(m, __uint_as_float(l[c][i]));
                if (LISTS && __any_sync(0xffffffffu, walk.column != kNoColumn)) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (__any_sync(0xffffffffu, walk.column < 32 * c + 32)) {
                            put_values(turn, swap, l[c]);
                            for (; walk.column < 32 * c + 32; walk.next()) h.e.at[walk.list - h.e.entries + walk.j] = ld_shared(value(walk.column - 32 * c)) * h.e.inverse_t;
                        }
                }
                const bool hit = !LISTS && t >= 0 && t < 128;
                if (!LISTS && __any_sync(0xffffffffu, hit)) {
                    float x = 0.f;
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (t == 32 * c + i) x = __uint_as_float(l[c][i]);
                    if (hit) h.at_target[row] = x;
                }
                // 2^(l log2 e - c) with c = m log2 e as rounded, in one multiply-add each; what c lost is put right in the sum, or, where it is
                // more than a first-order term can (m beyond 10^5), m is taken off first.
                const float ref = m == -INFINITY ? 0.f : m;
                float c2 = ref * log2e, lost = fmaf(ref, log2e, -c2);
                if (__any_sync(0xffffffffu, fabsf(lost) > kHeadLost)) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int i = 0; i < 32; ++i) l[c][i] = __float_as_uint(__uint_as_float(l[c][i]) - ref);
                    c2 = lost = 0.f;
                }
                float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int i = 0; i < 32; ++i) s[i & 3] += head_exp2(fmaf(__uint_as_float(l[c][i]), log2e, -c2));
                float back = 1.f - lost * 0.69314718f;
                if (LISTS) back += fmaf(ref, h.e.inverse_t, -__fmul_rn(ref, h.e.inverse_t));
                const float sum = ((s[0] + s[1]) + (s[2] + s[3])) * back;
                if (in) h.running[static_cast<int64_t>((t0.n0 >> 7) + half) * h.N + row] = make_float2(LISTS ? __fmul_rn(m, h.e.inverse_t) : m, sum);
            } else {
                const bool is = LISTS ? part : in && h.target[row] >= 0;
                const float g = LISTS ? g_row : (is ? h.scale[row] : 0.f), lse = LISTS ? lse_row : (is ? h.lse[row] : 0.f);
                float z = -lse * kHeadLog2e, lost = fmaf(-lse, kHeadLog2e, -z), scale = log2e;      // as for the statistics
                if (__any_sync(0xffffffffu, fabsf(lost) > kHeadLost)) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int i = 0; i < 32; ++i) l[c][i] = __float_as_uint((LISTS ? __uint_as_float(l[c][i]) * h.e.inverse_t : __uint_as_float(l[c][i])) - lse);
                    z = lost = 0.f;
                    scale = kHeadLog2e;
                } else if (LISTS) {                          // at l / T = lse, where it counts
                    lost = fmaf(-z, __fdividef(fmaf(kHeadLog2e, h.e.inverse_t, -log2e), log2e), lost);
                }
                const float gp = (LISTS ? g * mass : g) * (1.f + lost * 0.69314718f);
                if (LISTS && __any_sync(0xffffffffu, walk.column != kNoColumn)) {
                    if (lane == 0) bulk_wait_read();         // the last tile's outputs are out of the block
                    __syncwarp();
                }
#pragma unroll
                for (int c = 0; c < 4; ++c) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) l[c][i] = __float_as_uint(head_exp2(fmaf(__uint_as_float(l[c][i]), LISTS ? scale : kHeadLog2e, z)) * gp);
                    if (LISTS) {
                        if (__any_sync(0xffffffffu, walk.column < 32 * c + 32)) {
                            put_values(turn, swap, l[c]);
                            for (; walk.column < 32 * c + 32; walk.next()) {
                                const uint32_t at = value(walk.column - 32 * c);
                                st_shared(at, ld_shared(at) - g * walk.p);
                            }
                            get_values(turn, swap, l[c]);
                        }
                    } else if (__any_sync(0xffffffffu, t >= 32 * c && t < 32 * c + 32)) {
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (t == 32 * c + i) l[c][i] = __float_as_uint(__uint_as_float(l[c][i]) - g);
                    }
                    if (!__all_sync(0xffffffffu, is)) {      // rows without a target, whatever W holds
#pragma unroll
                        for (int i = 0; i < 32; ++i) l[c][i] = is ? l[c][i] : 0u;
                    }
                }
#pragma unroll
                for (int b = 0; b < 2; ++b)
                    if (row0 < h.N && valid > 64 * b)
                        store_block(&tmG, block, *reinterpret_cast<uint32_t(*)[2][32]>(&l[2 * b]), col0 + 64 * b, row0, lane);
            }
        }
        if (STORES && !failed) {
            // Zeros for the row blocks that no tile has: a block of them, stored as often as it takes.
            if (lane == 0) bulk_wait_read();
            __syncwarp();
            for (int i = lane; i < kStoreBytes / 16; i += 32)
                asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(block + 16 * i), "r"(0) : "memory");
            fence_proxy_async_smem();
            __syncwarp();
            const int blocks_n = (h.cols + 63) / 64, first = tiles_m * (2 * H_BM / 32);
            const int blocks = ((h.N + 31) / 32 - first) * blocks_n;
            if (lane == 0)
                for (int i = blockIdx.x * H_EPILOGUE_WARPS + (warp - 2); i < blocks; i += gridDim.x * H_EPILOGUE_WARPS)
                    tma_store_2d(&tmG, block, i % blocks_n * 64, (first + i / blocks_n) * 32);
        }
        if (STORES && lane == 0) bulk_wait_all();
        if (failed) *abort_flag = 1;
    }
    if (failed && status) atomicExch(status, VELORA_ERR_TIMEOUT);

    tc_fence_before_sync();
    __syncthreads();
    cluster.sync();                                          // nobody signals or reads a CTA that has left
    tc_fence_after_sync();
    if (warp == 1) {
        __syncwarp();
        tmem_dealloc_pair(tmem_base, 2 * H_BN);
    }
}

template <int ROLE>
int launch_role(const CUtensorMap& tx, const CUtensorMap& tw, const CUtensorMap& tg, const HeadTile& h, int* status, int sm_count, cudaStream_t stream)
{
    static DeviceOnce configured;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return VELORA_ERR_CUDA;
    auto kern = head_pair_kernel<ROLE>;
    if (!configured.get(dev)) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(H_SMEM)) != cudaSuccess) return VELORA_ERR_CUDA;
        configured.set(dev);
    }
    const int64_t tiles = ceil_div64(h.N, 2 * H_BM) * ceil_div64(h.cols, H_BN);
    const int64_t pairs = tiles < sm_count / 2 ? tiles : sm_count / 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(2 * pairs), 1, 1);
    cfg.blockDim = dim3(H_THREADS, 1, 1);
    cfg.dynamicSmemBytes = H_SMEM;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kern, tx, tw, tg, h, status) != cudaSuccess) {
        cudaGetLastError();
        return VELORA_ERR_CUDA;
    }
    return after_launch();
}

}  // namespace

int launch_head_tiles(const void* x, int64_t ldx, const void* W, int64_t ldw, void* G, int64_t ldg, const HeadTile& h, int* status, cudaStream_t stream)
{
    DeviceInfo di;
    int rc = device_info(&di);
    if (rc != VELORA_OK) return rc;
    CUtensorMap tx, tw, tg;
    rc = make_tmap_bf16_2d(&tx, x, h.D, h.N, ldx, H_BK, H_BM);
    if (rc != VELORA_OK) return rc;
    rc = make_tmap_bf16_2d(&tw, W, h.D, h.cols, ldw, H_BK, H_BN / 2);
    if (rc != VELORA_OK) return rc;
    tg = tx;
    if (G) {
        rc = make_tmap_bf16_2d(&tg, G, ldg, h.N, ldg, 64, 32);              // whole pitch: columns past the piece's are written as well
        if (rc != VELORA_OK) return rc;
        return h.e.entries ? launch_role<DISTILL_GRADIENT>(tx, tw, tg, h, status, di.sm_count, stream)
                           : launch_role<HEAD_GRADIENT>(tx, tw, tg, h, status, di.sm_count, stream);
    }
    return h.e.entries ? launch_role<DISTILL_STATS>(tx, tw, tg, h, status, di.sm_count, stream)
                       : launch_role<HEAD_STATS>(tx, tw, tg, h, status, di.sm_count, stream);
}

}  // namespace velora
