// The logits of a linear head for few tokens (up to 128), used up where they come out of the tensor cores; roles and results as in
// head_loss_tc.cu.  What bounds it is reading W once, so W's rows are the rows of the products: tiles of up to 128 columns of the vocabulary,
// as high as shares the vocabulary out most evenly (32000: 112, 224 columns for a CTA that has two), the tokens (rounded up to 32, 64 or
// 128) are the other side, and no tensor-core time goes into rows that are not there.  Single CTAs with 160 KB of W in flight each (128 for more than
// 32 tokens, 96 for more than 64).
//
// Per CTA: warp 0 lane 0 TMA producer, warp 1 lane 0 MMA issuer, warps 2..5 epilogue (32 columns of the vocabulary each).  A lane of the
// epilogue has one column for all tokens; 32 x 32 blocks are turned over through shared memory, and then it has one token for 32
// columns.  Contractions are cut into segments as in head_loss_tc.cu (of 128 instead of 512: 61 us).  1 x 4096 of 32000: the call 54 us, W
// alone at the copy rate 41 (87 us with the tokens as rows of 256).
#include "gemm_tc.cuh"
#include "head_loss.cuh"
#include "tc_common.cuh"

namespace velora {

using namespace tc;

namespace {

constexpr int W_BM = 128;                  // columns of the vocabulary in a tile
constexpr int W_BK = 64;
constexpr int W_THREADS = 192;
constexpr int W_PITCH = 33;
constexpr int W_STAGING_BYTES = 4 * 32 * W_PITCH * 4;
constexpr int W_PARTS_BYTES = 4 * 128 * 8;                     // (maximum, sum) of each warp and token
constexpr int W_BARRIER_BYTES = 256;

template <int NT> struct FewShape {
    static constexpr int kStageBytes = (W_BM + NT) * W_BK * 2;
    static constexpr int kStages = 200 * 1024 / kStageBytes < 10 ? 200 * 1024 / kStageBytes : 10;
    static constexpr int kTmemCols = 2 * NT;                   // a power of two, 64 or more
    static constexpr size_t kSmem = 1024 + static_cast<size_t>(kStages) * kStageBytes + W_STAGING_BYTES + W_PARTS_BYTES + W_BARRIER_BYTES;
};

// All epilogue warps; true in all of them if `p` is in one.  A warp that has given up comes here as well, so nobody waits for it.
__device__ __forceinline__ bool epilogue_any(bool p)
{
    uint32_t any;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.or.pred q, 1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(any) : "r"(static_cast<uint32_t>(p)) : "memory");
    return any != 0;
}

// Of a lane's rows 32 c + lane: the tokens (negative: the row has no part in it), where their entries in a warp's columns are, the first of those, what a
// gradient takes.
template <int C> struct FewLists {
    int token[C], j[C], end[C];
    Entry head[C];
    float scale[C], lse[C], mass[C];
    template <bool GRADIENT> __device__ __forceinline__ void find(const HeadTile& h, int lane, int v0, int valid)
    {
        if (valid <= 0) {                                    // for the warp
#pragma unroll
            for (int c = 0; c < C; ++c) token[c] = -1;
            return;
        }
        const int from = h.v0 + v0;
        bool live[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {                        // rows that are not there: the last one, no branch
            const int row = min(32 * c + lane, h.N - 1);
            live[c] = h.target[row] >= 0;
            token[c] = h.e.order[row];
            if (GRADIENT) {
                scale[c] = h.scale[row];
                lse[c] = h.lse[row];
            }
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            live[c] &= 32 * c + lane < h.N;
            const unsigned short* s = h.e.starts + static_cast<int64_t>(token[c]) * h.e.pitch;
            j[c] = s[from / kEntryColumns];                  // of a token without entries: anything
            end[c] = s[(from + valid - 1) / kEntryColumns + 1];
            if (GRADIENT) mass[c] = h.e.mass[token[c]];
        }
#pragma unroll
        for (int c = 0; c < C; ++c) head[c] = h.e.entries[static_cast<int64_t>(token[c]) * h.e.K + (live[c] ? min(j[c], h.e.K - 1) : 0)];
#pragma unroll
        for (int c = 0; c < C; ++c)
            if (!live[c]) {
                token[c] = -1;
                scale[c] = lse[c] = mass[c] = 0.f;
            }
    }
    __device__ __forceinline__ void walk(EntryWalk& w, const Entries& e, int c, int from) const
    {
        w.none();
        if (token[c] < 0) return;
        w.begin(e, token[c], j[c], end[c], from, head[c]);
        while (w.column < 0) w.next();                       // of the same 128 columns, but in front
    }
};

template <bool GRADIENT, bool LISTS, int NT>
__global__ void __launch_bounds__(W_THREADS, 1)
head_few_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX, const HeadTile h, int height, __nv_bfloat16* G, int64_t ldg,
                int twice, int* status)
{
    typedef FewShape<NT> S;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    uint8_t* smem = smem_raw + (base - raw);
    float* staging = reinterpret_cast<float*>(smem + S::kStages * S::kStageBytes);
    float2* parts = reinterpret_cast<float2*>(smem + S::kStages * S::kStageBytes + W_STAGING_BYTES);
    uint8_t* tail = smem + S::kStages * S::kStageBytes + W_STAGING_BYTES + W_PARTS_BYTES;
    const uint32_t full = smem_u32(tail), empty = full + 8 * S::kStages;
    const uint32_t tfull = full + 16 * S::kStages, tempty = tfull + 16;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(tail + 16 * S::kStages + 32);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tail + 16 * S::kStages + 40);
    static_assert(16 * S::kStages + 48 <= W_BARRIER_BYTES, "barriers");

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int num_tiles = (h.cols + height - 1) / height, kblocks = (h.D + W_BK - 1) / W_BK;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(tfull + 8 * a, 1);
            mbar_init(tempty + 8 * a, 4);
        }
        *abort_flag = 0;
        fence_mbar_init();
        prefetch_tensormap(&tmW);
        prefetch_tensormap(&tmX);
    }
    if (warp == 1) {
        tmem_alloc(smem_u32(tmem_slot), S::kTmemCols);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem_base = *tmem_slot;
    pdl_wait();                                              // nothing in global memory has been touched so far
    pdl_trigger();

    bool failed = false;
    if (warp == 0) {
        // ------------------------------------------------ TMA producer
        if (lane == 0) {
            uint32_t it = 0;
            for (int tile = blockIdx.x; tile < num_tiles && !failed; tile += gridDim.x) {
                for (int kb = 0; kb < kblocks; ++kb, ++it) {
                    const uint32_t s = it % S::kStages, ph = (it / S::kStages) & 1u;
                    if (!mbar_wait(empty + 8 * s, ph ^ 1u, abort_flag)) { failed = true; break; }
                    mbar_arrive_expect_tx(full + 8 * s, static_cast<uint32_t>((height + NT) * W_BK * 2));
                    const uint32_t dst = base + s * S::kStageBytes;
                    tma_load_2d(dst, &tmW, full + 8 * s, kb * W_BK, tile * height);                  // rows behind it: whatever was there, outputs that nobody reads
                    tma_load_2d(dst + W_BM * W_BK * 2, &tmX, full + 8 * s, kb * W_BK, 0);
                }
            }
            if (failed) {
                *abort_flag = 1;
                // Let the copies in flight land before shared memory is given up.
                const unsigned long long t0 = globaltimer_ns();
                const uint32_t back = it < S::kStages ? it : S::kStages;
                for (uint32_t j = 1; j <= back; ++j) {
                    const uint32_t jt = it - j;
                    while (!mbar_try_wait(full + 8 * (jt % S::kStages), (jt / S::kStages) & 1u))
                        if (globaltimer_ns() - t0 > kWaitLimitNs) break;
                }
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------ MMA issuer
        if (lane == 0) {
            constexpr uint32_t idesc = umma_idesc_bf16(W_BM, NT, false, false);
            uint32_t it = 0, seg = 0;
            for (int tile = blockIdx.x; tile < num_tiles && !failed; tile += gridDim.x) {
                for (int k0 = 0; k0 < kblocks && !failed; k0 += kHeadSegment, ++seg) {
                    const uint32_t acc = seg & 1u, aph = (seg >> 1) & 1u;
                    if (!mbar_wait(tempty + 8 * acc, aph ^ 1u, abort_flag)) { failed = true; break; }
                    tc_fence_after_sync();
                    const uint32_t d_tmem = tmem_base + acc * NT;
                    const int k1 = min(kblocks, k0 + kHeadSegment);
                    for (int kb = k0; kb < k1; ++kb, ++it) {
                        const uint32_t s = it % S::kStages, ph = (it / S::kStages) & 1u;
                        if (!mbar_wait(full + 8 * s, ph, abort_flag)) { failed = true; break; }
                        tc_fence_after_sync();
                        const uint32_t a_addr = base + s * S::kStageBytes, b_addr = a_addr + W_BM * W_BK * 2;
#pragma unroll
                        for (int j = 0; j < W_BK / 16; ++j)
                            umma_bf16(d_tmem, umma_smem_desc(a_addr + j * 32, 16, 1024), umma_smem_desc(b_addr + j * 32, 16, 1024), idesc, ((kb - k0) | j) != 0);
                        umma_commit(empty + 8 * s);
                    }
                    if (!failed) umma_commit(tfull + 8 * acc);
                }
            }
            if (failed) *abort_flag = 1;
        }
    } else {
        // ------------------------------------------------ epilogue
        const int quarter = warp & 3;
        float* block = staging + quarter * (32 * W_PITCH);
        uint32_t seg = 0;
        for (int tile = blockIdx.x; tile < num_tiles && !failed; tile += gridDim.x) {
            const int v0 = tile * height + quarter * 32, valid = min(min(32, height - quarter * 32), h.cols - v0);      // this warp's columns; may be none
            FewLists<LISTS ? NT / 32 : 1> lists;             // looked up while the products run: four loads, each with the address of the next
            if (LISTS) lists.template find<GRADIENT>(h, lane, v0, valid);
            uint32_t l[NT / 32][32];                         // fp32 bits
#pragma unroll
            for (int c = 0; c < NT / 32; ++c)
#pragma unroll
                for (int i = 0; i < 32; ++i) l[c][i] = 0u;
            for (int k0 = 0; k0 < kblocks; k0 += kHeadSegment, ++seg) {
                const uint32_t acc = seg & 1u, aph = (seg >> 1) & 1u;
                if (!mbar_wait_warp(tfull + 8 * acc, aph, abort_flag, 64)) { failed = true; *abort_flag = 1; break; }
                tc_fence_after_sync();
#pragma unroll
                for (int c = 0; c < NT / 32; ++c) {
                    uint32_t r[32];
                    tmem_ld_32x32(tmem_base + acc * NT + c * 32 + (static_cast<uint32_t>(quarter * 32) << 16), r);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 32; ++i) l[c][i] = __float_as_uint(__uint_as_float(l[c][i]) + __uint_as_float(r[i]));
                }
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(tempty + 8 * acc);
            }
            if (GRADIENT ? failed : (failed = epilogue_any(failed))) break;      // behind it nobody reads the last tile's parts any more
#pragma unroll
            for (int c = 0; c < NT / 32; ++c) {
                const int row = 32 * c + lane;               // this lane's token behind the turn
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 32; ++i) block[i * W_PITCH + lane] = LISTS ? __uint_as_float(l[c][i]) * h.e.inverse_t : __uint_as_float(l[c][i]);
                __syncwarp();
                if (32 * c >= h.N) break;                    // for all epilogue warps
                const int target = !LISTS && row < h.N ? h.target[row] : -1, t = target - h.v0 - v0;
                float* mine = block + lane * W_PITCH;
                EntryWalk walk;
                if (LISTS) lists.walk(walk, h.e, c, h.v0 + v0);
                if (!GRADIENT) {
                    float m = -INFINITY, s = 0.f;
                    for (int i = 0; i < valid; ++i) m = fmaxf(m, mine[i]);
                    const float ref = m == -INFINITY ? 0.f : m;
                    float off = 0.f, c2 = ref * kHeadLog2e, lost = fmaf(ref, kHeadLog2e, -c2);
                    if (fabsf(lost) > kHeadLost) {           // the maximum is taken off first, see head_loss_tc.cu
                        off = ref;
                        c2 = lost = 0.f;
                    }
#pragma unroll 8
                    for (int i = 0; i < valid; ++i) s += head_exp2(fmaf(mine[i] - off, kHeadLog2e, -c2));
                    parts[quarter * NT + row] = make_float2(m, s * (1.f - lost * 0.69314718f));
                    if (LISTS) {
                        for (; walk.column < valid; walk.next()) h.e.at[walk.list - h.e.entries + walk.j] = mine[walk.column];
                    } else if (t >= 0 && t < valid) {
                        h.at_target[row] = mine[t];
                    }
                } else if (row < h.N && valid > 0) {
                    const bool is = LISTS ? lists.token[LISTS ? c : 0] >= 0 : target >= 0;
                    const float g = LISTS ? lists.scale[LISTS ? c : 0] : (is ? h.scale[row] : 0.f);
                    const float lse = LISTS ? lists.lse[LISTS ? c : 0] : (is ? h.lse[row] : 0.f);
                    float off = 0.f, z = -lse * kHeadLog2e, lost = fmaf(-lse, kHeadLog2e, -z);
                    if (fabsf(lost) > kHeadLost) {
                        off = lse;
                        z = lost = 0.f;
                    }
                    const float gp = (LISTS ? g * lists.mass[LISTS ? c : 0] : g) * (1.f + lost * 0.69314718f);
                    if (LISTS) {                             // complete before they are rounded
                        for (int i = 0; i < valid; ++i) mine[i] = head_exp2(fmaf(mine[i] - off, kHeadLog2e, z)) * gp;
                        for (; walk.column < valid; walk.next()) mine[walk.column] -= g * walk.p;
                    }
                    // The pitch is a multiple of 256 and the height of 16: columns past the piece's are there to be written, those of the next tile
                    // are not touched.
                    uint4* dst = reinterpret_cast<uint4*>(G + row * ldg + v0);
                    uint4* rest = reinterpret_cast<uint4*>(G + (row + h.N) * ldg + v0);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t w[4], r[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const int j = 8 * i + 2 * k;
                            float x = mine[j], y = mine[j + 1];
                            if (!LISTS) {
                                x = head_exp2(fmaf(x - off, kHeadLog2e, z)) * gp;
                                y = head_exp2(fmaf(y - off, kHeadLog2e, z)) * gp;
                                if (t == j) x -= g;
                                if (t == j + 1) y -= g;
                            }
                            w[k] = is ? pack_bf16x2(x, y) : 0u;
                            r[k] = is ? pack_bf16x2(x - bf16_lo(w[k]), y - bf16_hi(w[k])) : 0u;
                        }
                        if (8 * i < valid) {
                            dst[i] = make_uint4(w[0], w[1], w[2], w[3]);
                            if (twice) rest[i] = make_uint4(r[0], r[1], r[2], r[3]);
                        }
                    }
                }
            }
            if (!GRADIENT) {
                epilogue_any(false);
                const int row = static_cast<int>(threadIdx.x) - 64;
                if (row < NT && row < h.N) {
                    float m = -INFINITY, s = 0.f;
                    bool nan = false;
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        m = fmaxf(m, parts[w * NT + row].x);
                        nan |= parts[w * NT + row].y != parts[w * NT + row].y;
                    }
                    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
                    for (int w = 0; w < 4; ++w) s += parts[w * NT + row].y * expf(parts[w * NT + row].x - ref);
                    h.running[static_cast<int64_t>(tile) * h.N + row] = make_float2(m, nan ? __int_as_float(0x7fc00000) : s);
                }
            }
        }
        if (failed) *abort_flag = 1;
    }
    if (failed && status) atomicExch(status, VELORA_ERR_TIMEOUT);

    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (warp == 1) {
        __syncwarp();
        tmem_dealloc(tmem_base, S::kTmemCols);
    }
}

template <bool GRADIENT, bool LISTS, int NT>
int launch_few(const CUtensorMap& tw, const CUtensorMap& tx, const HeadTile& h, int height, void* G, int64_t ldg, int twice, int* status, int sm_count, cudaStream_t stream)
{
    static DeviceOnce configured;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return VELORA_ERR_CUDA;
    auto kern = head_few_kernel<GRADIENT, LISTS, NT>;
    if (!configured.get(dev)) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(FewShape<NT>::kSmem)) != cudaSuccess) return VELORA_ERR_CUDA;
        configured.set(dev);
    }
    const int tiles = (h.cols + height - 1) / height;
    return launch_chained(kern, dim3(static_cast<unsigned>(tiles < sm_count ? tiles : sm_count)), W_THREADS, FewShape<NT>::kSmem, stream,
                          tw, tx, h, height, static_cast<__nv_bfloat16*>(G), ldg, twice, status);
}

}  // namespace

int head_few_height(int64_t cols)
{
    int best = W_BM;
    int64_t most = 0;                                         // columns of the CTA that has the most of them, on 148 SMs
    for (int t = W_BM; t >= kHeadFewHeight; t -= 16) {
        const int64_t share = ceil_div64(ceil_div64(cols, t), 148) * t;
        if (most == 0 || share < most) {
            best = t;
            most = share;
        }
    }
    return best;
}

int launch_head_few(const void* x, int64_t ldx, const void* W, int64_t ldw, void* G, int64_t ldg, int twice, const HeadTile& h, int* status, cudaStream_t stream)
{
    DeviceInfo di;
    int rc = device_info(&di);
    if (rc != VELORA_OK) return rc;
    const int nt = h.N <= 32 ? 32 : (h.N <= 64 ? 64 : 128);
    CUtensorMap tw, tx;
    const int height = head_few_height(h.cols);
    rc = make_tmap_bf16_2d(&tw, W, h.D, h.cols, ldw, W_BK, height);
    if (rc != VELORA_OK) return rc;
    rc = make_tmap_bf16_2d(&tx, x, h.D, h.N, ldx, W_BK, nt);
    if (rc != VELORA_OK) return rc;
#define VELORA_FEW(GRAD, LISTS)                                                                                      \
    (nt == 32 ? launch_few<GRAD, LISTS, 32>(tw, tx, h, height, G, ldg, twice, status, di.sm_count, stream)                          \
              : (nt == 64 ? launch_few<GRAD, LISTS, 64>(tw, tx, h, height, G, ldg, twice, status, di.sm_count, stream)              \
                          : launch_few<GRAD, LISTS, 128>(tw, tx, h, height, G, ldg, twice, status, di.sm_count, stream)))
    if (h.e.entries) return G ? VELORA_FEW(true, true) : VELORA_FEW(false, true);
    return G ? VELORA_FEW(true, false) : VELORA_FEW(false, false);
#undef VELORA_FEW
}

}  // namespace velora
