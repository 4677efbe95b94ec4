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
    int N, V, pitch, size, shift;                          // size: K rounded up to a power of two, 32 at least, 2^shift
    float inverse_t;
};

__device__ __forceinline__ float teacher_logit(const Teacher& t, int64_t at)
{
    return t.t_dtype == VELORA_BF16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(t.logits)[at]) : static_cast<const float*>(t.logits)[at];
}

// The row's threads: a warp (WARPS = 1, eight rows a block), or a block of WARPS warps.
template <int WARPS> __device__ __forceinline__ void row_sync()
{
    if (WARPS == 1) __syncwarp();
    else __syncthreads();
}
// Over the row's threads; `part` of WARPS values.
template <int WARPS, typename OP> __device__ __forceinline__ float row_all(float x, float* part, OP op)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x = op(x, __shfl_xor_sync(0xffffffffu, x, o));
    if (WARPS == 1) return x;
    __syncthreads();                                       // the last result has been read by all
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = x;
    __syncthreads();
    x = part[0];
#pragma unroll
    for (int w = 1; w < WARPS; ++w) x = op(x, part[w]);
    return x;
}

// The keys of 32 EACH entries in order over a warp, entry 32 i + lane in k[i]: bitonic steps, between lanes or between a lane's own.
template <typename KEY, int EACH> __device__ __forceinline__ void warp_sort(KEY (&k)[EACH])
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int run = 2; run <= 32 * EACH; run *= 2)
#pragma unroll
        for (int step = run / 2; step > 0; step /= 2) {
            if (step >= 32) {
#pragma unroll
                for (int i = 0; i < EACH; ++i) {
                    const int j = i | (step / 32);
                    if (j == i) continue;
                    const KEY lo = min(k[i], k[j]), hi = max(k[i], k[j]);
                    const bool up = ((32 * i) & run) == 0;
                    k[i] = up ? lo : hi;
                    k[j] = up ? hi : lo;
                }
            } else {
#pragma unroll
                for (int i = 0; i < EACH; ++i) {
                    const KEY other = __shfl_xor_sync(0xffffffffu, k[i], step);
                    const bool up = ((32 * i + lane) & run) == 0, low = (lane & step) == 0;
                    k[i] = up == low ? min(k[i], other) : max(k[i], other);
                }
            }
        }
}

// A row's probabilities, its entries' order by (column, place in the list), and where every 128 columns' entries start.  KEY holds column and place (32 bits
// where they fit).  Up to 256 entries a warp puts in order in its registers; more, and wide keys, a block in shared memory with a thread a pair (one warp through
// shared memory: 16 lists of 247 18 us, 8192 of 64 22 us; counting the smaller ones for each: 8904 of 125 26 us).  Starts by a search each, or, for up to 64
// entries, a search a lane and a walk along its share of the columns.
template <typename KEY, int WARPS, int EACH>               // EACH: entries a lane, with one warp
__global__ void __launch_bounds__(WARPS == 1 ? kThreads : 32 * WARPS)
distill_lists_kernel(const ListsArgs a)
{
    constexpr KEY kLast = ~static_cast<KEY>(0);            // sorts behind every entry; none is as large
    constexpr int kTeam = 32 * WARPS, kRows = WARPS == 1 ? kWarps : 1;
    extern __shared__ __align__(16) char room[];
    __shared__ float part[WARPS];
    pdl_wait();
    pdl_trigger();
    const int row = WARPS == 1 ? threadIdx.x >> 5 : 0, t = threadIdx.x % kTeam, K = a.t.K;
    KEY* key = reinterpret_cast<KEY*>(room) + row * a.size;
    float* p = reinterpret_cast<float*>(room + static_cast<size_t>(kRows) * a.size * sizeof(KEY)) + row * a.size;
    auto sum = [](float x, float y) { return x + y; };
    auto most = [](float x, float y) { return fmaxf(x, y); };
    for (int n = blockIdx.x * kRows + row; n < a.N; n += gridDim.x * kRows) {
        float m = -INFINITY, count_f = 0.f, kind = 0.f;    // kind: 1, something counts (a NaN does); 2: an entry is no column
        for (int k = t; k < a.size; k += kTeam) {
            const int64_t i = k < K ? a.t.index[n * a.t.ldi + k] : -1;
            const float x = k < K ? teacher_logit(a.t, n * a.t.ldt + k) : 0.f;              // does not wait for the column
            const bool is = i >= 0 && i < a.V;
            const float u = is ? (x == INFINITY ? __int_as_float(0x7fc00000) : x) : -INFINITY;         // over T below: a finite one stays one until then
            if (i >= a.V) kind = 2.f;
            else if (is && u != -INFINITY) kind = fmaxf(kind, 1.f);
            m = fmaxf(m, u);
            p[k] = u;
            key[k] = is ? static_cast<KEY>(i) << a.shift | static_cast<unsigned>(k) : kLast;
            count_f += is ? 1.f : 0.f;
        }
        kind = row_all<WARPS>(kind, part, most);
        const int count = static_cast<int>(row_all<WARPS>(count_f, part, sum));
        if (t == 0) a.mark[n] = kind == 2.f ? a.V : (kind == 1.f ? 0 : -1);
        if (kind != 1.f) continue;                         // for all the row's threads; nobody reads its entries
        float s = 0.f;
        if (a.t.lse) {
            m = a.t.lse[n];
            for (int k = t; k < K; k += kTeam) s += p[k] = p[k] == -INFINITY ? 0.f : expf(p[k] * a.inverse_t - m);
        } else {
            m = row_all<WARPS>(m, part, most);
            for (int k = t; k < K; k += kTeam) s += p[k] = expf((p[k] - m) * a.inverse_t);
            const float scale = 1.f / row_all<WARPS>(s, part, sum);
            s = 0.f;
            for (int k = t; k < K; k += kTeam) s += p[k] *= scale;
        }
        s = row_all<WARPS>(s, part, sum);
        if (t == 0) a.mass[n] = s;
        row_sync<WARPS>();
        Entry* out = a.entries + static_cast<int64_t>(n) * K;
        const unsigned place = (1u << a.shift) - 1u;
        if constexpr (WARPS == 1) {
            KEY mine[EACH];
#pragma unroll
            for (int i = 0; i < EACH; ++i) mine[i] = key[t + 32 * i];
            warp_sort<KEY, EACH>(mine);
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                key[t + 32 * i] = mine[i];                 // each lane's own so far
                if (mine[i] != kLast) out[t + 32 * i] = Entry{static_cast<int>(mine[i] >> a.shift), p[static_cast<unsigned>(mine[i]) & place]};
            }
        } else {
            for (int run = 2; run <= a.size; run *= 2)
                for (int step = run / 2; step > 0; step /= 2) {
                    for (int i = t; i < a.size / 2; i += kTeam) {
                        const int x = 2 * i - (i & (step - 1)), y = x + step;
                        const KEY kx = key[x], ky = key[y];
                        if ((kx > ky) == ((x & run) == 0)) {
                            key[x] = ky;
                            key[y] = kx;
                        }
                    }
                    row_sync<WARPS>();
                }
            for (int j = t; j < count; j += kTeam) out[j] = Entry{static_cast<int>(key[j] >> a.shift), p[static_cast<unsigned>(key[j]) & place]};
        }
        for (int j = count + t; j < K; j += kTeam) out[j] = Entry{0, 0.f};                  // none
        row_sync<WARPS>();
        unsigned short* starts = a.starts + static_cast<int64_t>(n) * a.pitch;
        const bool walk = WARPS == 1 && EACH <= 2;         // a lane may have all the entries to walk along
        const int share = walk ? (a.pitch + 31) / 32 : 1, step = walk ? 1 : kTeam, first = t * share, behind = walk ? min(a.pitch, first + share) : a.pitch;
        int lo = 0;
        for (int b = first; b < behind; b += step) {
            const KEY from = static_cast<KEY>(b) * kEntryColumns << a.shift;
            if (b == a.pitch - 1) {                        // behind all entries: its key may not fit
                lo = count;
            } else if (walk && b > first) {
                while (lo < count && key[lo] < from) ++lo;
            } else {
                lo = 0;
                int hi = count;
                while (lo < hi) {
                    const int mid = (lo + hi) / 2;
                    if (key[mid] < from) lo = mid + 1; else hi = mid;
                }
            }
            starts[b] = static_cast<unsigned short>(lo);
        }
        row_sync<WARPS>();
    }
}

// A logit over the temperature, rounded to the same number in both passes: contracted into the subtraction behind it, it would differ from what is in lse.
__device__ __forceinline__ float over_t(float l, const Entries& e) { return __fmul_rn(l, e.inverse_t); }

// fp32: a block takes a slice of a row's logits, 1024 columns, in registers: its maximum, its exponentials, the entries' logits.  (A block a row, three times
// over it: 1 x 24008 88 us, 8904 x 501 46 us.)
constexpr int kSliceColumns = 4 * kThreads;
__global__ void __launch_bounds__(kThreads)
distill_stats_kernel(const float* logits, int64_t ld, int parts, int64_t part_stride, const HeadTile h, int part0)
{
    __shared__ float part[2][kWarps];
    __shared__ float value[kSliceColumns];
    pdl_wait();
    pdl_trigger();
    const int row = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c0 = blockIdx.y * kSliceColumns;
    if (row >= *h.live) return;                            // the same for the block
    const int n = h.e.order[row];
    const unsigned short* starts = h.e.starts + static_cast<int64_t>(n) * h.e.pitch;
    const int from = starts[(h.v0 + c0) / kEntryColumns], to = starts[(h.v0 + min(h.cols, c0 + kSliceColumns) + kEntryColumns - 1) / kEntryColumns];
    const float* l = logits + row * ld + c0;
    float x[4], m = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = threadIdx.x + kThreads * i;
        x[i] = c0 + c < h.cols ? over_t(parts > 1 ? sum_of_parts(l + c, parts, part_stride) : l[c], h.e) : -INFINITY;
        value[c] = x[i];
        m = fmaxf(m, x[i]);
    }
    m = warp_max(m);
    if (lane == 0) part[0][warp] = m;
    __syncthreads();
    for (int w = 0; w < kWarps; ++w) m = fmaxf(m, part[0][w]);
    const float ref = m == -INFINITY ? 0.f : m;
    float s = (expf(x[0] - ref) + expf(x[1] - ref)) + (expf(x[2] - ref) + expf(x[3] - ref));          // a NaN among them stays one here
    s = warp_sum(s);
    if (lane == 0) part[1][warp] = s;
    const Entry* entries = h.e.entries + static_cast<int64_t>(n) * h.e.K;
    for (int j = from + threadIdx.x; j < to; j += kThreads) h.e.at[static_cast<int64_t>(n) * h.e.K + j] = value[entries[j].column - h.v0 - c0];
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0.f;
        for (int w = 0; w < kWarps; ++w) s += part[1][w];
        h.running[static_cast<int64_t>(part0 + blockIdx.y) * h.N + row] = make_float2(m, s);
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
    const float g = h.scale[row], z = h.lse[row], q = is ? g * h.e.mass[n] : 0.f;
    const unsigned short* starts = h.e.starts + static_cast<int64_t>(n) * h.e.pitch;
    const Entry* entries = h.e.entries + static_cast<int64_t>(n) * h.e.K;
    for (int c0 = (static_cast<int>(blockIdx.y) * kWarps + warp) * kEntryColumns; c0 < h.cols; c0 += static_cast<int>(gridDim.y) * kWarps * kEntryColumns) {
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float* at = l + c0 + lane + 32 * i;
            x[i] = is && c0 + lane + 32 * i < h.cols ? (parts > 1 ? sum_of_parts(at, parts, part_stride) : *at) : 0.f;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = is ? q * expf(over_t(x[i], h.e) - z) : 0.f;
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
// a warp takes two rows' entries.
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
            for (int i = 0; i < 16; ++i) x[i] = p[static_cast<int64_t>(min(p0 + slices * i, parts - 1)) * h.N];          // no branch: all under way
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (p0 + slices * i >= parts) x[i] = make_float2(-INFINITY, 0.f);
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
            float e[4], l[4];
            auto load = [&](int k0) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const bool is = k0 + 32 * k < h.e.K;
                    e[k] = is ? entries[k0 + 32 * k].p : 0.f;
                    l[k] = is ? at[k0 + 32 * k] : 0.f;
                }
            };
            load(lane);
            ms = make_float2(-INFINITY, 0.f);
            for (int k = lane; k < slices; k += 32) ms = merged(ms, slice[r * slices + k]);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) ms = merged(ms, make_float2(__shfl_xor_sync(0xffffffffu, ms.x, o), __shfl_xor_sync(0xffffffffu, ms.y, o)));
            z = ms.x + logf(ms.y);
            for (int k0 = lane;;) {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (e[k] != 0.f) y += e[k] * (logf(e[k]) - (l[k] - z));                // p log p is 0 there, whatever the student's logit
                k0 += 128;
                if (k0 >= h.e.K) break;
                load(k0);
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
    args.size = 32;                                        // a warp's at least
    args.shift = 5;
    while (args.size < a.teacher->K) {
        args.size *= 2;
        ++args.shift;
    }
    args.inverse_t = e.inverse_t;
    const int64_t most = static_cast<int64_t>(di.sm_count) * 8;
    const bool narrow = a.V <= (static_cast<int64_t>(1) << (32 - args.shift)) - 1;              // columns and places below 2^32 - 2^shift
    auto grid = [&](int rows) { return dim3(static_cast<unsigned>(ceil_div64(a.N, rows) < most ? ceil_div64(a.N, rows) : most)); };
    const size_t size = static_cast<size_t>(args.size);
    const size_t warps = kWarps * size * 8;
    if (narrow && size <= 32) return launch_chained(distill_lists_kernel<unsigned, 1, 1>, grid(kWarps), kThreads, warps, a.stream, args);
    if (narrow && size <= 64) return launch_chained(distill_lists_kernel<unsigned, 1, 2>, grid(kWarps), kThreads, warps, a.stream, args);
    if (narrow && size <= 128) return launch_chained(distill_lists_kernel<unsigned, 1, 4>, grid(kWarps), kThreads, warps, a.stream, args);
    if (narrow && size <= 256) return launch_chained(distill_lists_kernel<unsigned, 1, 8>, grid(kWarps), kThreads, warps, a.stream, args);
    if (size <= 256) return launch_chained(distill_lists_kernel<unsigned long long, 4, 0>, grid(1), 128, size * 12, a.stream, args);
    if (size <= 512)
        return narrow ? launch_chained(distill_lists_kernel<unsigned, 8, 0>, grid(1), 256, size * 8, a.stream, args)
                      : launch_chained(distill_lists_kernel<unsigned long long, 8, 0>, grid(1), 256, size * 12, a.stream, args);
    return narrow ? launch_chained(distill_lists_kernel<unsigned, 16, 0>, grid(1), 512, size * 8, a.stream, args)
                  : launch_chained(distill_lists_kernel<unsigned long long, 16, 0>, grid(1), 512, size * 12, a.stream, args);
}

int launch_distill_stats(const float* logits, int64_t ld, int parts, int64_t part_stride, const HeadTile& h, int* part, cudaStream_t stream)
{
    const int slices = static_cast<int>(ceil_div64(h.cols, kSliceColumns)), part0 = *part;
    *part += slices;
    return launch_chained(distill_stats_kernel, dim3(static_cast<unsigned>(h.N), static_cast<unsigned>(slices)), kThreads, 0, stream, logits, ld, parts,
                          part_stride, h, part0);
}

int launch_distill_gradient(float* logits, int64_t ld, int parts, int64_t part_stride, const HeadTile& h, cudaStream_t stream)
{
    const int64_t blocks = ceil_div64(h.cols, kEntryColumns * kWarps);
    return launch_chained(distill_gradient_kernel, dim3(static_cast<unsigned>(h.N), static_cast<unsigned>(blocks < 16 ? blocks : 16)), kThreads, 0,
                          stream, logits, ld, parts, part_stride, h);
}

int launch_distill_merge(const HeadTile& h, int parts, float* loss, float* lse, cudaStream_t stream)
{
    int rows = 1;                                          // two blocks an SM, if there are as many (64 rows of 286 parts, cold: 9 us with 32 rows a block, 5 with one)
    while (rows < 32 && h.N > 296 * rows) rows *= 2;
    return launch_chained(distill_merge_kernel, dim3(static_cast<unsigned>(ceil_div64(h.N, rows))), kMergeThreads, 0, stream, h, parts, rows, loss, lse);
}

}  // namespace velora
