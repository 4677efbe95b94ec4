// Distillation into a linear head from a teacher's top logits: what it takes beside the head's own kernels.  With T the temperature, l = X W^T / T and
// lse its log sum exp, and a teacher's K columns i and logits t of a token,
//   p[n, k] = exp(t[n, k] / T - s[n]),  s[n] = log sum_k exp(t[n, k] / T)  or as given
//   loss[n] = sum_k p (log p - (l[n, i] - lse)),    G[n, v] = g[n] / T (exp(l - lse) sum_k p - sum_{k: i = v} p)
// A token's entries are put in the order of their columns once a call (distill_lists_kernel), and where every 128 columns' entries start is noted:
// the kernels that have a row of logits in registers, 128 columns of it at a time, find what belongs there with one look and turn only those
// values over through shared memory.  The logits' gradients are complete before they are rounded, so G of a student that agrees with its
// teacher is the rounded difference and not the difference of roundings.
#include "head_loss.cuh"

namespace velora {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
struct ListsArgs {
    Teacher t;
    int64_t* mark;                                         // 0: has entries; -1: has none; V: one of them is no column
    Entry* entries;
    unsigned short* starts;
    float* mass;
    int N, V, pitch, size, shift;                          // size: K rounded up to a power of two, four at least, 2^shift
    float inverse_t;
};

__device__ __forceinline__ float teacher_logit(const Teacher& t, int64_t at)
{
    return t.t_dtype == VELORA_BF16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(t.logits)[at]) : static_cast<const float*>(t.logits)[at];
}

// A warp a token: probabilities, the entries' order by (column, place in the list), where every 128 columns' entries start.  KEY holds both (32 bits where they
// fit).  Up to 64 entries are put in order by counting, for each, the smaller ones, 64 comparisons that wait for nothing (bitonic steps through shared memory
// one after the other: 8192 lists of 64 22 us instead of 16); starts by a search a lane and a walk along its share of the columns, by searches for longer lists,
// of which one lane might have them all to walk along.
template <typename KEY, bool FEW>
__global__ void __launch_bounds__(kThreads)
distill_lists_kernel(const ListsArgs a)
{
    constexpr KEY kLast = ~static_cast<KEY>(0);               // sorts behind every entry; none is as large
    extern __shared__ __align__(16) char room[];
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5, K = a.t.K;
    KEY* key = reinterpret_cast<KEY*>(room) + warp * a.size;
    float* p = reinterpret_cast<float*>(room + static_cast<size_t>(warps) * a.size * sizeof(KEY)) + warp * a.size;
    KEY* sorted = FEW ? reinterpret_cast<KEY*>(room + static_cast<size_t>(warps) * a.size * (sizeof(KEY) + 4)) + warp * a.size : key;
    for (int n = blockIdx.x * warps + warp; n < a.N; n += gridDim.x * warps) {
        bool bad = false, some = false;
        float m = -INFINITY;
        int count = 0;
        for (int k = lane; k < a.size; k += 32) {
            const int64_t i = k < K ? a.t.index[n * a.t.ldi + k] : -1;
            const bool is = i >= 0 && i < a.V;
            const float t = k < K ? teacher_logit(a.t, n * a.t.ldt + k) : 0.f;              // does not wait for the column
            const float u = is ? t * a.inverse_t : -INFINITY;
            bad |= i >= a.V;
            some |= is && u != -INFINITY;                  // a NaN is something
            m = fmaxf(m, u);
            p[k] = u;
            key[k] = is ? static_cast<KEY>(i) << a.shift | static_cast<unsigned>(k) : kLast;
            count += is;
        }
        bad = __any_sync(0xffffffffu, bad);
        some = __any_sync(0xffffffffu, some) && !bad;
        count = __reduce_add_sync(0xffffffffu, count);
        if (lane == 0) a.mark[n] = bad ? a.V : (some ? 0 : -1);
        if (!some) continue;                               // for the warp; nobody reads its entries
        float s = 0.f;
        if (a.t.lse) {
            m = a.t.lse[n];
            for (int k = lane; k < K; k += 32) s += p[k] = p[k] == -INFINITY ? 0.f : expf(p[k] - m);
        } else {
            m = warp_max(m);
            for (int k = lane; k < K; k += 32) s += p[k] = expf(p[k] - m);
            const float scale = 1.f / warp_sum(s);
            s = 0.f;
            for (int k = lane; k < K; k += 32) s += p[k] *= scale;
        }
        s = warp_sum(s);
        if (lane == 0) a.mass[n] = s;
        __syncwarp();
        Entry* out = a.entries + static_cast<int64_t>(n) * K;
        const unsigned place = (1u << a.shift) - 1u;
        if (FEW) {
            const KEY mine[2] = {lane < a.size ? key[lane] : kLast, lane + 32 < a.size ? key[lane + 32] : kLast};
            int rank[2] = {0, 0};
#pragma unroll 4
            for (int j = 0; j < a.size; j += 4) {
                const uint4 x = *reinterpret_cast<const uint4*>(key + j);
#pragma unroll
                for (int i = 0; i < 2; ++i) rank[i] += (x.x < mine[i]) + (x.y < mine[i]) + (x.z < mine[i]) + (x.w < mine[i]);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (mine[i] != kLast) {
                    sorted[rank[i]] = mine[i];
                    out[rank[i]] = Entry{static_cast<int>(mine[i] >> a.shift), p[lane + 32 * i]};
                }
        } else {
            for (int run = 2; run <= a.size; run *= 2)
                for (int step = run / 2; step > 0; step /= 2) {
                    for (int i = lane; i < a.size / 2; i += 32) {
                        const int x = 2 * i - (i & (step - 1)), y = x + step;
                        const KEY kx = key[x], ky = key[y];
                        if ((kx > ky) == ((x & run) == 0)) {
                            key[x] = ky;
                            key[y] = kx;
                        }
                    }
                    __syncwarp();
                }
            for (int j = lane; j < count; j += 32) out[j] = Entry{static_cast<int>(key[j] >> a.shift), p[static_cast<unsigned>(key[j]) & place]};
        }
        for (int j = count + lane; j < K; j += 32) out[j] = Entry{0, 0.f};                  // none
        __syncwarp();
        unsigned short* starts = a.starts + static_cast<int64_t>(n) * a.pitch;
        const int share = FEW ? (a.pitch + 31) / 32 : 1, step = FEW ? 1 : 32, first = lane * share, behind = FEW ? min(a.pitch, first + share) : a.pitch;
        int lo = 0;
        for (int b = first; b < behind; b += step) {
            const KEY from = static_cast<KEY>(b) * kEntryColumns << a.shift;
            // The last start is behind all entries: its key may not fit.
            if (b == a.pitch - 1) lo = count;
            else if (FEW && b > first) {
                while (lo < count && sorted[lo] < from) ++lo;
            } else {
                lo = 0;
                int hi = count;
                while (lo < hi) {
                    const int mid = (lo + hi) / 2;
                    if (sorted[mid] < from) lo = mid + 1; else hi = mid;
                }
            }
            starts[b] = static_cast<unsigned short>(lo);
        }
        __syncwarp();
    }
}

// fp32: a block per row takes the piece's maximum and its exponentials into what the pieces before have left, and notes the entries' logits.
__global__ void __launch_bounds__(kThreads)
distill_stats_kernel(float* logits, int64_t ld, int parts, int64_t part_stride, const HeadTile h, int first)
{
    __shared__ float part[2][kWarps];
    pdl_wait();
    pdl_trigger();
    const int row = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (row >= *h.live) return;                            // the same for the block
    float* l = logits + row * ld;
    float m = -INFINITY;
    for (int c = threadIdx.x; c < h.cols; c += kThreads) {
        const float x = sum_of_parts(l + c, parts, part_stride) * h.e.inverse_t;
        l[c] = x;                                          // read again by this thread, the entries' behind a barrier
        m = fmaxf(m, x);
    }
    m = warp_max(m);
    if (lane == 0) part[0][warp] = m;
    __syncthreads();
    for (int w = 0; w < kWarps; ++w) m = fmaxf(m, part[0][w]);
    const float2 old = first ? make_float2(-INFINITY, 0.f) : h.running[row];
    m = fmaxf(m, old.x);
    const float ref = m == -INFINITY ? 0.f : m;
    float s = 0.f;
#pragma unroll 4
    for (int c = threadIdx.x; c < h.cols; c += kThreads) s += expf(l[c] - ref);
    s = warp_sum(s);
    if (lane == 0) part[1][warp] = s;
    const int n = h.e.order[row];
    const unsigned short* starts = h.e.starts + static_cast<int64_t>(n) * h.e.pitch;
    const Entry* entries = h.e.entries + static_cast<int64_t>(n) * h.e.K;
    for (int j = starts[h.v0 / kEntryColumns] + threadIdx.x; j < starts[(h.v0 + h.cols + kEntryColumns - 1) / kEntryColumns]; j += kThreads)
        h.e.at[static_cast<int64_t>(n) * h.e.K + j] = l[entries[j].column - h.v0];
    __syncthreads();
    if (threadIdx.x == 0) {
        s = old.y * expf(old.x - ref);
        for (int w = 0; w < kWarps; ++w) s += part[1][w];
        h.running[row] = make_float2(m, s);
    }
}

// fp32: logits to their gradients, in place; a warp takes 128 columns of a row at a time.
__global__ void __launch_bounds__(kThreads)
distill_gradient_kernel(float* logits, int64_t ld, int parts, int64_t part_stride, const HeadTile h)
{
    pdl_wait();
    pdl_trigger();
    const int row = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float* l = logits + row * ld;
    const bool is = h.target[row] >= 0;
    const int n = h.e.order[row];
    const float g = h.scale[row] * h.e.inverse_t, z = h.lse[row], q = is ? g * h.e.mass[n] : 0.f;
    const unsigned short* starts = h.e.starts + static_cast<int64_t>(n) * h.e.pitch;
    const Entry* entries = h.e.entries + static_cast<int64_t>(n) * h.e.K;
    for (int c0 = (static_cast<int>(blockIdx.y) * kWarps + warp) * kEntryColumns; c0 < h.cols; c0 += static_cast<int>(gridDim.y) * kWarps * kEntryColumns) {
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = is && c0 + lane + 32 * i < h.cols ? sum_of_parts(l + c0 + lane + 32 * i, parts, part_stride) : 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = is ? q * expf(x[i] * h.e.inverse_t - z) : 0.f;
        if (is) {
            const int b = (h.v0 + c0) / kEntryColumns;
            for (int j = starts[b]; j < starts[b + 1]; ++j) {
                const Entry e = entries[j];
                const int c = e.column - h.v0 - c0 - lane;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (c == 32 * i) x[i] -= g * e.p;
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c0 + lane + 32 * i < h.cols) l[c0 + lane + 32 * i] = x[i];
    }
}

__device__ __forceinline__ float2 merged(float2 a, float2 b)          // (maximum, sum of exponentials relative to it); a NaN stays one
{
    const float m = a.x > b.x ? a.x : (a.x == a.x ? b.x : a.x), ref = m == -INFINITY ? 0.f : m;
    return make_float2(m, a.y * expf(a.x - ref) + b.y * expf(b.x - ref));
}

// A block takes up to 32 rows: its threads are shared out over rows and slices of their parts, 16 loads in flight each, a warp puts a row's slices together; then
// a warp takes two rows' entries.  Few rows have that many more slices.
constexpr int kMergeThreads = 512, kMergeWarps = kMergeThreads / 32;
__global__ void __launch_bounds__(kMergeThreads)
distill_merge_kernel(const HeadTile h, int parts, int rows, float* loss, float* lse)          // rows: a power of two
{
    __shared__ float2 slice[kMergeThreads];
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, row0 = blockIdx.x * rows, slices = kMergeThreads / rows;
    const int live = *h.live, mine = row0 + static_cast<int>(threadIdx.x) % rows;
    float2 ms = make_float2(-INFINITY, 0.f);
    if (mine < live) {
        const float2* p = h.running + mine;
        for (int p0 = static_cast<int>(threadIdx.x) / rows; p0 < parts; p0 += slices * 16) {
            float2 x[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = p0 + slices * i < parts ? p[static_cast<int64_t>(p0 + slices * i) * h.N] : make_float2(-INFINITY, 0.f);
            float m = ms.x;
#pragma unroll
            for (int i = 0; i < 16; ++i) m = x[i].x > m ? x[i].x : (x[i].x == x[i].x ? m : x[i].x);      // a NaN stays one
            const float ref = m == -INFINITY ? 0.f : m;
            float s = ms.y * expf(ms.x - ref);
#pragma unroll
            for (int i = 0; i < 16; ++i) s += x[i].y * expf(x[i].x - ref);
            ms = make_float2(m, s);
        }
    }
    slice[static_cast<int>(threadIdx.x) % rows * slices + static_cast<int>(threadIdx.x) / rows] = ms;
    // What the entries need, on its way meanwhile.
    int token[2], mark[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = warp + kMergeWarps * i;
        mark[i] = -3;
        if (r < rows && row0 + r < h.N) {
            mark[i] = h.target[row0 + r];
            token[i] = h.e.order[row0 + r];
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (mark[i] == -3) continue;                           // for the warp
        const int r = warp + kMergeWarps * i;
        float y = 0.f, z = 0.f;
        if (mark[i] >= 0) {
            const Entry* entries = h.e.entries + static_cast<int64_t>(token[i]) * h.e.K;
            const float* at = h.e.at + static_cast<int64_t>(token[i]) * h.e.K;
            Entry e[2];
            float l[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const bool is = lane + 32 * k < h.e.K;
                e[k].p = is ? entries[lane + 32 * k].p : 0.f;
                l[k] = is ? at[lane + 32 * k] : 0.f;
            }
            ms = make_float2(-INFINITY, 0.f);
            for (int k = lane; k < slices; k += 32) ms = merged(ms, slice[r * slices + k]);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) ms = merged(ms, make_float2(__shfl_xor_sync(0xffffffffu, ms.x, o), __shfl_xor_sync(0xffffffffu, ms.y, o)));
            z = ms.x + logf(ms.y);
#pragma unroll
            for (int k = 0; k < 2; ++k)
                if (e[k].p != 0.f) y += e[k].p * (logf(e[k].p) - (l[k] - z));              // p log p is 0 there, whatever the student's logit
            for (int k = lane + 64; k < h.e.K; k += 32) {
                const float p = entries[k].p;
                if (p != 0.f) y += p * (logf(p) - (at[k] - z));
            }
            y = warp_sum(y);
        }
        if (lane == 0) {
            loss[token[i]] = mark[i] == -2 ? __int_as_float(0x7fc00000) : y;
            lse[token[i]] = z;
        }
    }
}

}  // namespace

Entries distill_entries(const HeadArgs& a, const HeadLayout& l)
{
    Entries e{};
    e.entries = reinterpret_cast<const Entry*>(a.ws + l.entries);
    e.starts = reinterpret_cast<const unsigned short*>(a.ws + l.starts);
    e.mass = reinterpret_cast<const float*>(a.ws + l.mass);
    e.order = reinterpret_cast<const int*>(a.ws + l.order);
    e.at = reinterpret_cast<float*>(a.ws + l.at_entries);
    e.K = a.teacher->K;
    e.pitch = entry_pitch(a.V);
    e.inverse_t = 1.f / a.teacher->temperature;
    return e;
}

int launch_distill_lists(const HeadArgs& a, const HeadLayout& l)
{
    DeviceInfo di;
    const int rc = device_info(&di);
    if (rc != VELORA_OK) return rc;
    const Entries e = distill_entries(a, l);
    ListsArgs args{};
    args.t = *a.teacher;
    args.mark = reinterpret_cast<int64_t*>(a.ws + l.mark);
    args.entries = const_cast<Entry*>(e.entries);
    args.starts = const_cast<unsigned short*>(e.starts);
    args.mass = const_cast<float*>(e.mass);
    args.N = static_cast<int>(a.N);
    args.V = static_cast<int>(a.V);
    args.pitch = e.pitch;
    args.size = 4;                                         // keys are compared four at a time
    args.shift = 2;
    while (args.size < a.teacher->K) {
        args.size *= 2;
        ++args.shift;
    }
    args.inverse_t = e.inverse_t;
    const int warps = args.size <= 256 ? kWarps : 2;       // 24 KB of keys and probabilities at most
    const int64_t ctas = ceil_div64(a.N, warps), most = static_cast<int64_t>(di.sm_count) * 8;
    const dim3 grid(static_cast<unsigned>(ctas < most ? ctas : most));
    const size_t keys = static_cast<size_t>(warps) * args.size;
    const bool narrow = a.V <= (static_cast<int64_t>(1) << (32 - args.shift)) - 1;              // columns and places below 2^32 - 2^shift
    if (!narrow) return launch_chained(distill_lists_kernel<unsigned long long, false>, grid, 32 * warps, keys * 12, a.stream, args);
    return args.size <= 64 ? launch_chained(distill_lists_kernel<unsigned, true>, grid, 32 * warps, keys * 12, a.stream, args)
                           : launch_chained(distill_lists_kernel<unsigned, false>, grid, 32 * warps, keys * 8, a.stream, args);
}

int launch_distill_stats(float* logits, int64_t ld, int parts, int64_t part_stride, const HeadTile& h, bool first, cudaStream_t stream)
{
    return launch_chained(distill_stats_kernel, dim3(static_cast<unsigned>(h.N)), kThreads, 0, stream, logits, ld, parts, part_stride, h, first ? 1 : 0);
}

int launch_distill_gradient(float* logits, int64_t ld, int parts, int64_t part_stride, const HeadTile& h, cudaStream_t stream)
{
    const int64_t blocks = ceil_div64(h.cols, kEntryColumns * kWarps);
    return launch_chained(distill_gradient_kernel, dim3(static_cast<unsigned>(h.N), static_cast<unsigned>(blocks < 16 ? blocks : 16)), kThreads, 0,
                          stream, logits, ld, parts, part_stride, h);
}

int launch_distill_merge(const HeadTile& h, int parts, float* loss, float* lse, cudaStream_t stream)
{
    int rows = 1;
    while (rows < 32 && rows < h.N) rows *= 2;
    return launch_chained(distill_merge_kernel, dim3(static_cast<unsigned>(ceil_div64(h.N, rows))), kMergeThreads, 0, stream, h, parts, rows, loss, lse);
}

}  // namespace velora
