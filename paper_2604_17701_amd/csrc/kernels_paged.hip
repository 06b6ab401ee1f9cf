// The paged cache: keys and values of many requests in pools of pages.
//   K pool  [page][kv head][position][feature]           V pool  [page][kv head][position / 8][feature][position % 8]
// The V pool keeps eight positions of a feature together: O^T = V^T P^T reads eight (bf16) or four (float) keys of one
// feature per lane, which is then one 16-byte load, from memory or from LDS, without turning anything over.
#include "paged.h"

namespace wisv {

// ------------------------------------------------------------------------------------------ step planning
// One launch: every workgroup scans the lengths for itself (two prefix sums over the requests, kept in LDS) and then
// writes its share of the table and of the tokens; no workgroup waits for another.  Bound by the latency of launch,
// loads and scan: 5.2 us for 16 requests of 6 tokens, 5.9 for 512 with 22171 (a launch that does nothing takes 2.3).
// A workgroup reads the lengths once, before it writes anything, so that one alone may write over them (in a graph, the 512
// requests 11.7 us instead of 5.5).
constexpr int PLAN_THREADS = 256, PLAN_THREADS_ALONE = 1024;

// exclusive prefix sum over the workgroup's threads
__device__ __forceinline__ int64_t plan_scan(int64_t v, int64_t *waves, int lane, int wave) {
    int64_t x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t y = __shfl_up(x, o, 64);
        if (lane >= o) x += y;
    }
    __syncthreads();   // whoever still reads the sums of the scan before
    if (lane == 63) waves[wave] = x;
    __syncthreads();
    for (int w = 0; w < wave; ++w) x += waves[w];
    return x - v;
}

template <int THREADS> __global__ __launch_bounds__(THREADS) void k_paged_plan(PagedPlan a) {
    __shared__ int held[PLAN_MAX_BATCH];     // its cached tokens
    __shared__ int q_end[PLAN_MAX_BATCH];    // rows up to and with the request, at most max_tokens; first its own rows
    __shared__ int first[PLAN_MAX_BATCH];    // where its pages begin in free_pages; -1 - status: it is refused
    __shared__ int64_t waves[THREADS / 64];
    __shared__ int used[THREADS / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, ps = 1 << a.page_shift;
    const int64_t room = (int64_t)a.max_pages << a.page_shift;
    const int per = (a.batch + THREADS - 1) / THREADS, b0 = min(tid * per, a.batch), b1 = min(b0 + per, a.batch);
    const bool writes = blockIdx.x == 0;

    int64_t rows = 0;
    for (int b = b0; b < b1; ++b) {
        held[b] = max(a.cached_len[b], 0);
        q_end[b] = max(a.new_len[b], 0);
        rows += q_end[b];
    }
    rows = plan_scan(rows, waves, lane, wave);   // (behind its barriers the workgroup has read all lengths)
    // rows of a request, once q_end counts up to it (not of one whose rows end behind max_tokens)
    const auto rows_of = [&](int b) { return (int64_t)q_end[b] - (b ? q_end[b - 1] : 0); };
    if (writes && tid == 0) a.q_start[0] = 0;
    int64_t pages = 0;
    for (int b = b0; b < b1; ++b) {
        const int64_t c = held[b], n = q_end[b];
        rows += n;
        const int status = (c + n > room ? 2 : 0) | (rows > a.max_tokens ? 4 : 0);
        q_end[b] = (int)min(rows, (int64_t)a.max_tokens);
        first[b] = status;
        if (!status) pages += ((c + n + ps - 1) >> a.page_shift) - ((c + ps - 1) >> a.page_shift);
        if (writes) a.q_start[b + 1] = q_end[b];
    }
    pages = plan_scan(pages, waves, lane, wave);
    int most = 0;
    for (int b = b0; b < b1; ++b) {
        const int64_t c = held[b], n = rows_of(b);
        int status = first[b];
        const int64_t need = status ? 0 : ((c + n + ps - 1) >> a.page_shift) - ((c + ps - 1) >> a.page_shift), end = pages + need;
        if (need && end > a.n_free) status |= 1;
        first[b] = status ? -1 - status : need ? (int)pages : 0;
        if (need && !status) most = (int)end;   // the ends rise from request to request
        pages = end;
        if (writes) {
            a.kv_len[b] = (int)(status ? c : c + n);
            a.status[b] = status;
        }
    }
    if (writes) {
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) most = max(most, __shfl_xor(most, o, 64));
        if (lane == 0) used[wave] = most;
    }
    __syncthreads();
    if (writes && tid == 0) {
        for (int w = 1; w < THREADS / 64; ++w) most = max(most, used[w]);
        *a.n_used = most;
    }

    // new table entries: a wave per request
    for (int b = blockIdx.x * (THREADS / 64) + wave; b < a.batch; b += gridDim.x * (THREADS / 64)) {
        const int f = first[b];
        if (f < 0) continue;
        const int64_t c = held[b], n = rows_of(b);
        const int have = (int)((c + ps - 1) >> a.page_shift), end = (int)((c + n + ps - 1) >> a.page_shift);
        for (int p = have + lane; p < end; p += 64) a.block_table[(size_t)b * a.max_pages + p] = a.free_pages[f + p - have];
    }
    // tokens: a thread each
    const int live = q_end[a.batch - 1];
    for (int64_t t = blockIdx.x * THREADS + tid; t < a.max_tokens; t += gridDim.x * THREADS) {   // (a step past the last may pass 32 bits)
        int pos = 0, slot = -1;
        if (t < live) {
            int lo = 0, hi = a.batch - 1;   // the first request that ends behind t
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (q_end[mid] > t) hi = mid; else lo = mid + 1;
            }
            const int c = held[lo], f = first[lo];
            const int64_t at = (int64_t)c + t - (lo ? q_end[lo - 1] : 0);
            pos = (int)min(at, (int64_t)INT32_MAX);
            if (f >= 0) {
                const int have = (int)(((int64_t)c + ps - 1) >> a.page_shift), p = pos >> a.page_shift;
                const int page = p < have ? a.block_table[(size_t)lo * a.max_pages + p] : a.free_pages[f + p - have];
                if (page >= 0 && page <= INT32_MAX >> a.page_shift) slot = (page << a.page_shift) + (pos & (ps - 1));
            }
        }
        a.positions[t] = pos;
        a.slots[t] = slot;
    }
}

void launch_paged_plan(const PagedPlan &a, bool over_lengths, hipStream_t stream) {
    if (over_lengths) {
        hipLaunchKernelGGL((k_paged_plan<PLAN_THREADS_ALONE>), dim3(1), dim3(PLAN_THREADS_ALONE), 0, stream, a);
        return;
    }
    const int wgs = std::min(256, std::max((a.max_tokens + PLAN_THREADS - 1) / PLAN_THREADS, (a.batch + 15) / 16));
    hipLaunchKernelGGL((k_paged_plan<PLAN_THREADS>), dim3(std::max(wgs, 1)), dim3(PLAN_THREADS), 0, stream, a);
}

// ------------------------------------------------------------------------------------------ rotate and append
// Bound by HBM: every element is read once and written once (2483 rows of 32 / 8 heads of 128 in bf16, 62 MB: 12.6 us = 4.9 TB/s, the rate of a
// large copy; four rows 3.3 us).  Two kinds of workgroups in one launch:
//   q and k   a thread owns one 16-byte piece of a head's first half and its partner in the second half, for up to
//             ROT_HEADS heads of a token whose rotary factors it reads once;
//   v         a tile of 64 tokens x one KV head goes through LDS, since the pool keeps eight positions of a feature
//             together.  The tile's tokens fall into groups of at most eight that share such a block: whole blocks leave
//             as 16-byte stores, the ends of a request's run as single elements.
constexpr int ROT_HEADS = 4, V_TILE = 64, APPEND_THREADS = 256;

template <typename T> struct Pack;   // 16 bytes
template <> struct Pack<bf16_t> {
    static constexpr int N = 8;
    uint32_t w[4];
    __device__ __forceinline__ float get(int i) const { return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16); }
    __device__ __forceinline__ void set2(int i, float x, float y) { w[i >> 1] = f32x2_to_bf16x2(x, y); }
};
template <> struct Pack<float> {
    static constexpr int N = 4;
    float w[4];
    __device__ __forceinline__ float get(int i) const { return w[i]; }
    __device__ __forceinline__ void set2(int i, float x, float y) { w[i] = x; w[i + 1] = y; }
};

template <typename T, int HD>
__global__ __launch_bounds__(APPEND_THREADS) void k_paged_append(PagedAppend a, int rot_groups, int rot_wgs) {
    constexpr int N = Pack<T>::N, PIECES = HD / 2 / N;
    __shared__ T tile[V_TILE][HD + 16 / sizeof(T)];
    __shared__ int slot_of[V_TILE];
    __shared__ int start_of[V_TILE + 1];
    const int tid = threadIdx.x;
    const int64_t n_slots = (int64_t)a.n_pages << a.page_shift;
    const int in_page = (1 << a.page_shift) - 1;

    if ((int)blockIdx.x < rot_wgs) {
        const int64_t item = (int64_t)blockIdx.x * APPEND_THREADS + tid;
        const int piece = item % PIECES, heads = a.H + a.G;
        const int64_t rest = item / PIECES;
        const int group = rest % rot_groups;
        const int64_t t = rest / rot_groups;
        if (t >= a.n_tokens) return;
        const int h0 = group * ROT_HEADS, i = piece * N;
        // all heads' pieces are requested before the first is used (heads past the last re-read it)
        Pack<T> x[ROT_HEADS], y[ROT_HEADS];
#pragma unroll
        for (int u = 0; u < ROT_HEADS; ++u) {
            const int h = min(h0 + u, heads - 1);
            const T *src = h < a.H ? (const T *)a.q + t * a.q_stride + (int64_t)h * HD : (const T *)a.k + t * a.k_stride + (int64_t)(h - a.H) * HD;
            x[u] = *reinterpret_cast<const Pack<T> *>(src + i);
            y[u] = *reinterpret_cast<const Pack<T> *>(src + i + HD / 2);
        }
        const int slot = a.slots[t];
        float c[N], s[N];
        if (a.cs) {
            const int64_t p = min(max(a.positions[t], 0), a.n_rope - 1);
#pragma unroll
            for (int e = 0; e < N; e += 4) {
                *reinterpret_cast<paged_f4 *>(c + e) = *reinterpret_cast<const paged_f4 *>(a.cs + p * (HD / 2) + i + e);
                *reinterpret_cast<paged_f4 *>(s + e) = *reinterpret_cast<const paged_f4 *>(a.sn + p * (HD / 2) + i + e);
            }
        }
#pragma unroll
        for (int u = 0; u < ROT_HEADS; ++u) {
            const int h = h0 + u;
            if (h >= heads) break;
            Pack<T> r0 = x[u], r1 = y[u];
            if (a.cs) {
#pragma unroll
                for (int e = 0; e < N; e += 2) {
                    const float x0 = x[u].get(e), x1 = x[u].get(e + 1), y0 = y[u].get(e), y1 = y[u].get(e + 1);
                    r0.set2(e, x0 * c[e] - y0 * s[e], x1 * c[e + 1] - y1 * s[e + 1]);
                    r1.set2(e, y0 * c[e] + x0 * s[e], y1 * c[e + 1] + x1 * s[e + 1]);
                }
            }
            T *dst;
            if (h < a.H) {
                dst = (T *)a.q_out + t * a.q_out_stride + (int64_t)h * HD;
            } else {
                if (slot < 0 || slot >= n_slots) break;
                dst = (T *)a.k_pages + (int64_t)(slot >> a.page_shift) * a.page_stride +
                      (((int64_t)(h - a.H) << a.page_shift) + (slot & in_page)) * HD;
            }
            *reinterpret_cast<Pack<T> *>(dst + i) = r0;
            *reinterpret_cast<Pack<T> *>(dst + i + HD / 2) = r1;
        }
        return;
    }

    // ---- v
    const int vb = blockIdx.x - rot_wgs, g = vb % a.G;
    const int64_t t0 = (int64_t)(vb / a.G) * V_TILE;
    const int n = (int)min((int64_t)V_TILE, a.n_tokens - t0);
    for (int it = tid; it < n * (HD / N); it += APPEND_THREADS) {
        const int r = it / (HD / N), c = it % (HD / N) * N;
        *reinterpret_cast<Pack<T> *>(&tile[r][c]) = *reinterpret_cast<const Pack<T> *>((const T *)a.v + (t0 + r) * a.v_stride + (int64_t)g * HD + c);
    }
    int n_groups;
    if (tid < 64) {
        // the first wave finds where groups begin: a new block of eight positions, or a slot that does not follow
        int s = tid < n ? a.slots[t0 + tid] : -1;
        if (s < 0 || s >= n_slots) s = -1;
        slot_of[tid] = s;
        const int before = __shfl_up(s, 1, 64);
        const bool begins = tid < n && (tid == 0 || s < 0 || s != before + 1 || (s & 7) == 0);
        const unsigned long long m = __ballot(begins);
        if (begins) start_of[__popcll(m & ((1ull << tid) - 1))] = tid;
        if (tid == 0) start_of[V_TILE] = __popcll(m);
    }
    __syncthreads();
    n_groups = start_of[V_TILE];
    for (int it = tid; it < n_groups * HD; it += APPEND_THREADS) {
        const int k = it / HD, d = it % HD;
        const int r0 = start_of[k], r1 = k + 1 < n_groups ? start_of[k + 1] : n, s = slot_of[r0];
        if (s < 0) continue;
        T *dst = (T *)a.v_pages + (int64_t)(s >> a.page_shift) * a.page_stride + (((int64_t)g << a.page_shift) + (s & in_page & ~7)) * HD + d * 8;
        if (r1 - r0 == 8) {   // (then s is a multiple of 8)
            Pack<T> w[8 / N];
#pragma unroll
            for (int e = 0; e < 8; ++e) reinterpret_cast<T *>(w)[e] = tile[r0 + e][d];
#pragma unroll
            for (int e = 0; e < 8 / N; ++e) *reinterpret_cast<Pack<T> *>(dst + e * N) = w[e];
        } else {
            for (int r = r0; r < r1; ++r) dst[(s & 7) + r - r0] = tile[r][d];
        }
    }
}

static int64_t append_rot_wgs(const PagedAppend &a, bool bf16, int head_dim) {
    const int64_t items = (int64_t)a.n_tokens * ((a.H + a.G + ROT_HEADS - 1) / ROT_HEADS) * (head_dim / 2 / (bf16 ? 8 : 4));
    return (items + APPEND_THREADS - 1) / APPEND_THREADS;
}
static int64_t append_v_wgs(const PagedAppend &a) { return ((int64_t)a.n_tokens + V_TILE - 1) / V_TILE * a.G; }
int64_t paged_append_threads(const PagedAppend &a, bool bf16, int head_dim) {
    return (append_rot_wgs(a, bf16, head_dim) + append_v_wgs(a)) * APPEND_THREADS;
}
template <typename T, int HD> static void launch_append_t(const PagedAppend &a, hipStream_t stream) {
    const int rot_groups = (a.H + a.G + ROT_HEADS - 1) / ROT_HEADS;
    const int rot_wgs = (int)append_rot_wgs(a, sizeof(T) == 2, HD), v_wgs = (int)append_v_wgs(a);
    hipLaunchKernelGGL((k_paged_append<T, HD>), dim3(rot_wgs + v_wgs), dim3(APPEND_THREADS), 0, stream, a, rot_groups, rot_wgs);
}
template <typename T> static void launch_append_d(const PagedAppend &a, int head_dim, hipStream_t stream) {
    switch (head_dim) {
        case 32: return launch_append_t<T, 32>(a, stream);
        case 64: return launch_append_t<T, 64>(a, stream);
        case 128: return launch_append_t<T, 128>(a, stream);
        default: return launch_append_t<T, 256>(a, stream);
    }
}
void launch_paged_append(const PagedAppend &a, bool bf16, int head_dim, hipStream_t stream) {
    return bf16 ? launch_append_d<bf16_t>(a, head_dim, stream) : launch_append_d<float>(a, head_dim, stream);
}

}  // namespace wisv
