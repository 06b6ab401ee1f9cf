// Internal declarations of the paged cache's operators: step planning, the rotating append, attention over the pages.
#pragma once

#include "wisv_internal.h"

namespace wisv {

struct PagedPlan {
    int batch, page_shift, max_pages, n_free, max_tokens;
    const int32_t *cached_len, *new_len, *free_pages;
    int32_t *block_table, *q_start, *kv_len, *positions, *slots, *n_used, *status;
};
constexpr int PLAN_MAX_BATCH = 4096;   // the plan keeps three ints per request in LDS
void launch_paged_plan(const PagedPlan &a, bool over_lengths, hipStream_t stream);   // over_lengths: the lengths lie where it writes

struct PagedAppend {
    int n_tokens, H, G, n_rope, n_pages, page_shift;
    const void *q, *k, *v;
    void *q_out, *k_pages, *v_pages;
    int64_t q_stride, k_stride, v_stride, q_out_stride, page_stride;   // elements
    const int32_t *positions, *slots;
    const float *cs, *sn;
};
int64_t paged_append_threads(const PagedAppend &a, bool bf16, int head_dim);   // of the launch, at most 2^32 - 1
void launch_paged_append(const PagedAppend &a, bool bf16, int head_dim, hipStream_t stream);

struct PagedAttn {
    int batch, n_tokens, H, G, rep, n_pages, max_pages, page_shift, window;
    int n_splits, split_steps;     // key steps of a split; the last split takes what is left
    bool tiles;                    // k_paged_rows: a workgroup per tile of rows and not per request
    float scale, softcap;
    const void *q, *k_pages, *v_pages;
    void *out;
    int64_t q_stride, out_stride, page_stride;   // elements
    const int32_t *block_table, *q_start, *kv_len, *prefix_len;
    const float *slopes;
    float *po, *pm, *pl;           // n_splits > 1: [split][n_tokens][H][head_dim], [split][n_tokens][H]; pm in units of ln 2
};
constexpr int PAGED_MAX_SPLITS = 64;
// What a call will launch, from the sizes and the hints alone
struct PagedCut {
    bool prompt;                   // k_paged_prompt, or k_paged_rows
    int n_splits, split_steps;     // split_steps: of 64 keys
    size_t workspace;              // bytes
};
PagedCut paged_cut(const PagedAttn &a, bool bf16, int head_dim, int max_new, int max_len);
// The kernel of many rows, how many of its workgroups a CU's registers and LDS have room for, and how many tiles a call has at most
constexpr int paged_prompt_wgs(bool bf16, int head_dim) { return head_dim <= 64 ? 3 : bf16 || head_dim == 128 ? 2 : 1; }
int paged_prompt_tiles(const PagedAttn &a);
// few: requests have at most PAGED_FEW_ROWS rows, by the hint
constexpr int PAGED_FEW_ROWS = 32;
const char *launch_paged_prompt(const PagedAttn &a, bool bf16, int head_dim, bool few, int device, hipStream_t stream);
// null, or why the launch failed
const char *launch_paged_attention(PagedAttn a, bool bf16, int head_dim, int max_new, int max_len, int device, hipStream_t stream);

// ------------------------------------------------------------------------------------------ shared device code

typedef __bf16 paged_bf16x8 __attribute__((ext_vector_type(8)));
typedef float paged_f4 __attribute__((ext_vector_type(4)));
typedef unsigned int paged_u4 __attribute__((ext_vector_type(4)));

// tables read through the scalar cache (a vector load's wait would be one for the loads of keys and values as well)
typedef const int32_t __attribute__((address_space(4))) *paged_ints;

// What a workgroup knows of its request.  Every number is brought into the range the buffers have, whatever the arrays hold.
struct PagedRequest {
    int row0;      // first row of q
    int n_new;     // its rows
    int pos0;      // position of the first row
    int n_keys;    // keys the cache can hold for it: positions 0 .. n_keys - 1
    int prefix;    // positions below it are seen by every row
};
__device__ __forceinline__ PagedRequest paged_request(const PagedAttn &a, int b) {
    PagedRequest r;
    const int qs = a.q_start[b], qe = a.q_start[b + 1], len = max(a.kv_len[b], 0);
    const int pre = a.prefix_len ? a.prefix_len[b] : 0;
    r.row0 = min(max(qs, 0), a.n_tokens);
    r.n_new = min(max(qe, r.row0), a.n_tokens) - r.row0;
    r.pos0 = len - r.n_new;
    r.n_keys = min((int64_t)len, (int64_t)a.max_pages << a.page_shift);
    r.prefix = min(max(pre, 0), r.n_keys);
    return r;
}

// Ragged tiles: request b owns ceil(its rows / rows) of them, one request behind the other, so that the workgroups without a tile
// are the grid's last.  (Leaving gaps costs: with every second workgroup empty the dispatch gives some CUs three of the others and
// some one, 64 requests of 128 rows over 8192 positions 533 us instead of 363.)  A wave finds the request that owns `tile`, 512
// candidates at a time.
struct PagedTile {
    int b, index;   // the request, and which of its tiles; b < 0: there is no such tile
};
__device__ __forceinline__ PagedTile paged_find(const PagedAttn &a, int tile, int rows, int lane) {
    constexpr int PER = 8;
    int left = tile;
    for (int b0 = 0; b0 < a.batch; b0 += 64 * PER) {
        int start[PER + 1], count[PER], sum = 0;
#pragma unroll
        for (int i = 0; i <= PER; ++i) start[i] = min(max(a.q_start[min(b0 + lane * PER + i, a.batch)], 0), a.n_tokens);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            count[i] = max(start[i + 1] - start[i], 0);   // (past the last request: none)
            count[i] = (int)(((int64_t)count[i] * a.rep + rows - 1) / rows);
            sum += count[i];
        }
        int upto = sum;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int y = __shfl_up(upto, o, 64);
            if (lane >= o) upto += y;
        }
        const unsigned long long beyond = __ballot(upto > left);
        if (beyond) {
            const int owner = __ffsll(beyond) - 1;
            int in = left - (upto - sum), b = b0 + lane * PER;   // (of the owner's lane)
#pragma unroll
            for (int i = 0; i < PER - 1; ++i)
                if (in >= count[i] && b == b0 + lane * PER + i) in -= count[i], ++b;
            return PagedTile{__builtin_amdgcn_readfirstlane(__shfl(b, owner, 64)), __builtin_amdgcn_readfirstlane(__shfl(in, owner, 64))};
        }
        left -= __builtin_amdgcn_readfirstlane(__shfl(upto, 63, 64));
    }
    return PagedTile{-1, 0};
}

// The key steps some row of a tile sees: the prefix's, then from the window of its first row to its last position.
// Virtual step s is step s of the cache below n_pre and step s + skip from there.
struct PagedSteps {
    int n_pre, skip, total;
};
__device__ __forceinline__ PagedSteps paged_steps(const PagedRequest &r, int pos_min, int pos_max, int window, int step) {
    PagedSteps t;
    t.n_pre = (r.prefix + step - 1) / step;
    const int lo = window ? max(pos_min - window + 1, 0) : 0;
    const int first = max(t.n_pre, lo / step);
    const int last = (min(r.n_keys, max(pos_max + 1, 0)) + step - 1) / step;
    t.skip = first - t.n_pre;
    t.total = t.n_pre + max(last - first, 0);
    return t;
}

// Whether a row at position pos sees key j of n keys; lo: the position before its window, -1 without one.  (No && or ||: a
// branch per score costs more than the comparisons.)
__device__ __forceinline__ bool paged_sees(int j, int n, int prefix, int pos, int lo) {
    return bool((int)(j < n) & ((int)(j < prefix) | ((int)(j <= pos) & (int)(j > lo))));
}

// Two bf16 values: the halves that are finite, all bits of each
__device__ __forceinline__ uint32_t finite_halves(uint32_t w) {
    return ((w & 0x7f80u) != 0x7f80u ? 0xffffu : 0u) | ((w & 0x7f800000u) != 0x7f800000u ? 0xffff0000u : 0u);
}
// the value if it is infinite or no number, else 0
template <typename T> __device__ __forceinline__ float only_not_finite(T bits) {
    const float v = Elem<T>::load(&bits);
    return (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u ? v : 0.f;
}

}  // namespace wisv
