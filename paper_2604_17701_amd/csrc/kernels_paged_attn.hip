// Attention of a chunk of new tokens over the paged cache: few rows per request (or short float prompts), the join of split keys, and the
// choice between this kernel and kernels_paged_prompt.hip's.
//
// k_paged_rows.  The rows of a request and KV head - its new tokens x the query heads that share the KV head, token by
// token - are cut into tiles of 16 NQ rows, so that every cached byte meets a whole tile.  One workgroup = (split of the keys,
// KV head, request or tile); its waves take steps of 32 (bf16) or 16 (float) keys in turn and never meet before the end: keys
// and values go from the pages straight into matrix operands.
//   S^T = K Q^T   A operand: keys.  The rows are dealt so that lane group g of 16 lanes ends up with the scores of E
//                 consecutive keys (8, or 4) of each of 16 queries;
//   O^T += V^T P^T  those E probabilities are, as they stand, the B operand, and the A operand is one 16-byte load per
//                 lane and 16 features from the V pool, which keeps eight positions of a feature together.
// The softmax keeps a running maximum and sum in float; waves are joined in LDS, splits of the keys by k_paged_join.
// bf16: probabilities enter the matrix cores as two terms p = hi + lo, |p - hi - lo| <= 2^-17 p (what bounds this kernel
// is memory, the second term is free).  float: 16x16x4 float products throughout.
// Bound by bytes: 36 GB/s into one CU, about 6 TB/s into all; by latency below 100 KB per CU (a launch that reads next to nothing
// takes 6.4 us), and float prompts by the float matrix rate.  Kernel traces: one token over 131072 positions, 32 / 8 heads of 128
// (537 MB, 32 splits) 98 us = 5.5 TB/s; 36 tokens in windows of 4096, 16 / 8 heads of 256 (376 MB, ragged) 86 us = 4.4 TB/s; four
// rows over 516 positions, 32 / 8 heads of 128 (2.2 MB) 11.6 us; 24 float requests of 40 tokens behind 4000, 32 / 8 heads of
// 64 (32 GFLOP), 338 us = 94 TFLOP/s of 153.  Keys and values of one step in the same registers, so that two waves share a SIMD at head_dim
// 256, spill (99 us -> 155).
#include "paged.h"

namespace wisv {

template <typename T> struct Step;
template <> struct Step<bf16_t> { static constexpr int KEYS = 32, E = 8; };
template <> struct Step<float> { static constexpr int KEYS = 16, E = 4; };

__device__ __forceinline__ paged_f4 mfma_bf16(paged_u4 a, paged_u4 b, paged_f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(*reinterpret_cast<paged_bf16x8 *>(&a), *reinterpret_cast<paged_bf16x8 *>(&b), c, 0, 0, 0);
}
__device__ __forceinline__ paged_f4 mfma_f32(uint32_t a, uint32_t b, paged_f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a), __uint_as_float(b), c, 0, 0, 0);
}

// the pages of one step: two runs of KEYS / 2 keys (a page holds at least 16), each in its page or in a hole of the table
struct StepPages {
    int64_t at[2];   // elements from the pool's start to the run, in either pool
    bool has[2];
};
template <typename T, int HD>
__device__ __forceinline__ StepPages step_pages(const PagedAttn &a, paged_ints row, int g, int step) {
    constexpr int KEYS = Step<T>::KEYS;
    const int key = step * KEYS, p0 = key >> a.page_shift;
    StepPages s;
    const int id0 = row[min(p0, a.max_pages - 1)], in = key & ((1 << a.page_shift) - 1);
    const bool ok0 = (unsigned)id0 < (unsigned)a.n_pages;
    s.has[0] = ok0;
    s.at[0] = (int64_t)(ok0 ? id0 : 0) * a.page_stride + (((int64_t)g << a.page_shift) + in) * HD;
    s.has[1] = ok0;
    s.at[1] = s.at[0] + KEYS / 2 * HD;
    if (KEYS > 16 && a.page_shift == 4) {
        const int id1 = row[min(p0 + 1, a.max_pages - 1)];
        const bool ok1 = (unsigned)id1 < (unsigned)a.n_pages;
        s.has[1] = ok1;
        s.at[1] = (int64_t)(ok1 ? id1 : 0) * a.page_stride + ((int64_t)g << a.page_shift) * HD;
    }
    return s;
}

// Waves of a workgroup of k_paged_rows: eight, two to a SIMD, where the registers of half a SIMD hold a wave, else four
constexpr int rows_waves(int hd, int nq) { return hd * nq <= 128 ? 8 : 4; }

constexpr int merge_tiles(int nw, int nq, int dt) {   // feature tiles of 16 joined at a time: at most 32 KB of LDS
    int d = dt;
    while (d > 1 && nw * nq * d > 32) d /= 2;
    return d;
}

template <typename T, int HD, int NQ, bool MODS>
__global__ __launch_bounds__(64 * rows_waves(HD, NQ)) void k_paged_rows(PagedAttn a) {
    constexpr int NW = rows_waves(HD, NQ);
    constexpr int KEYS = Step<T>::KEYS, E = Step<T>::E, KL = HD / 16, QL = HD * (int)sizeof(T) / 64, DT = HD / 16;
    constexpr int DP = merge_tiles(NW, NQ, DT);
    constexpr bool BF = sizeof(T) == 2;
    __shared__ float sm[NW][NQ][16], sl[NW][NQ][16];
    __shared__ paged_f4 so[NW][NQ][DP][64];
    const int tid = threadIdx.x, lane = tid & 63, bj = lane & 15, bg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = blockIdx.x % a.G, split = blockIdx.y;
    // a workgroup per request, or (tiles) per tile
    const PagedTile mine = a.tiles ? paged_find(a, blockIdx.x / a.G, 16 * NQ, lane) : PagedTile{(int)blockIdx.x / a.G, 0};
    if (mine.b < 0) return;
    const int b = mine.b;
    const paged_ints table = (paged_ints)(uintptr_t)(a.block_table + (int64_t)b * a.max_pages);
    // the pages of the step that is this wave's first unless a window or a prefix says otherwise: asked for beside the lengths
    const int guess = split * a.split_steps + wave;
    const StepPages guessed = step_pages<T, HD>(a, table, g, guess);
    const PagedRequest rq = paged_request(a, b);
    const int R = rq.n_new * a.rep;
    const T *kpool = (const T *)a.k_pages, *vpool = (const T *)a.v_pages;
    constexpr float LOG2E = 1.4426950408889634f;
    const float scale2 = a.scale * LOG2E, cap_out = a.softcap * LOG2E, cap_in = (BF ? 2.f * scale2 : a.scale) / a.softcap;   // (cap_in: only with a cap)
    // this lane's part of a step: keys of its K rows lie in run krun, those of its V operand and scores in run vrun
    constexpr int HALF = KEYS / 2;
    const int krow = BF ? 8 * ((bj >> 2) & 1) + (bj & 3) : bj & 7, krun = bj >> 3, vrun = bg >> 1;
    const int koff = krow * HD + (BF ? 8 : 4) * bg;
    const int voff = BF ? ((bg & 1) * HD + bj) * 8 : bj * 8 + (bg & 1) * 4;

    for (int rho0 = mine.index * 16 * NQ; rho0 < R; rho0 += a.tiles ? R : 16 * NQ) {
        const int rho_end = min(rho0 + 16 * NQ, R);
        const int pos_min = rq.pos0 + rho0 / a.rep, pos_max = rq.pos0 + (rho_end - 1) / a.rep;
        const PagedSteps st = paged_steps(rq, pos_min, pos_max, a.window, KEYS);
        const int s_begin = split * a.split_steps, s_end = split == a.n_splits - 1 ? st.total : min(st.total, s_begin + a.split_steps);
        int s = s_begin + wave;

        // queries: operand (nq, t) of lane (bj, bg) holds 16 bytes of row rho0 + 16 nq + bj
        paged_u4 q[NQ][QL];
        int pos[NQ];
        float slope[NQ];
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) {
            const int rho = min(rho0 + 16 * nq + bj, R - 1), tok = rho / a.rep, h = g * a.rep + rho % a.rep;
            const T *src = (const T *)a.q + (int64_t)(rq.row0 + tok) * a.q_stride + (int64_t)h * HD + (BF ? 8 : 4) * bg;
#pragma unroll
            for (int t = 0; t < QL; ++t) q[nq][t] = *reinterpret_cast<const paged_u4 *>(src + t * (BF ? 32 : 16));
            pos[nq] = rq.pos0 + tok;
            slope[nq] = MODS && a.slopes ? a.slopes[h] * LOG2E : 0.f;
        }
        float m_run[NQ], l_run[NQ];
        paged_f4 oacc[NQ][DT];
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) {
            m_run[nq] = -INFINITY;
            l_run[nq] = 0.f;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) oacc[nq][dt] = paged_f4{0.f, 0.f, 0.f, 0.f};
        }

        if (s < s_end) {
            paged_u4 ka[KL], va[DT];   // bf16: K operands of tile A, then of tile B (four keys further)
            auto load_k = [&](const StepPages &p) {
                const T *src = kpool + (krun ? p.at[1] : p.at[0]) + koff;
                if (BF) {
#pragma unroll
                    for (int t = 0; t < KL / 2; ++t) {
                        ka[t] = *reinterpret_cast<const paged_u4 *>(src + 32 * t);
                        ka[KL / 2 + t] = *reinterpret_cast<const paged_u4 *>(src + 4 * HD + 32 * t);
                    }
                } else {
#pragma unroll
                    for (int t = 0; t < KL; ++t) ka[t] = *reinterpret_cast<const paged_u4 *>(src + 16 * t);
                }
            };
            auto load_v = [&](const StepPages &p) {
                const T *src = vpool + (vrun ? p.at[1] : p.at[0]) + voff;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) va[dt] = *reinterpret_cast<const paged_u4 *>(src + dt * 128);
            };
            auto real = [&](int v) { return v < st.n_pre ? v : v + st.skip; };
            // whether every row sees every key of the step (the same for the whole wave)
            auto see_all = [&](int key0, const StepPages &p) {
                return p.has[0] && p.has[1] && key0 + KEYS <= rq.n_keys &&
                       (key0 + KEYS <= rq.prefix || (key0 + KEYS - 1 <= pos_min && (!a.window || key0 > pos_max - a.window)));
            };
            uint32_t odd = 0;   // bits of values that are not finite, of steps that not every row sees
            StepPages cur = real(s) == guess ? guessed : step_pages<T, HD>(a, table, g, real(s));
            load_k(cur);
            load_v(cur);
            StepPages nxt = step_pages<T, HD>(a, table, g, real(min(s + NW, s_end - 1)));
            for (; s < s_end; s += NW) {
                const int step = real(s), key0 = step * KEYS, kbase = key0 + E * bg;   // this lane's keys: kbase .. kbase + E - 1
                const int n_mine = (vrun ? cur.has[1] : cur.has[0]) ? rq.n_keys : 0;   // keys in a hole of the table are not there
                const bool whole = see_all(key0, cur);
                paged_u4 phi[NQ], plo[NQ];   // float: phi holds the four probabilities themselves
#pragma unroll
                for (int nq = 0; nq < NQ; ++nq) {
                    paged_f4 sa = {0.f, 0.f, 0.f, 0.f}, sb = {0.f, 0.f, 0.f, 0.f};
                    if (BF) {
#pragma unroll
                        for (int t = 0; t < KL / 2; ++t) {
                            sa = mfma_bf16(ka[t], q[nq][t], sa);
                            sb = mfma_bf16(ka[KL / 2 + t], q[nq][t], sb);
                        }
                    } else {
#pragma unroll
                        for (int t = 0; t < KL; ++t)
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                if (t & 1) sb = mfma_f32(ka[t][j], q[nq][t][j], sb);
                                else sa = mfma_f32(ka[t][j], q[nq][t][j], sa);
                            }
                        sa += sb;
                    }
                    float x[E];
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        // in units of ln 2: every exponential is one instruction
                        float v = e < 4 ? sa[e] : sb[e & 3];
                        if (MODS && a.softcap > 0.f) {
                            if (BF) v = fmaf(__builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(v * cap_in) + 1.f), -2.f * cap_out, cap_out);   // tanh = 1 - 2 / (exp(2 x) + 1)
                            else v = cap_out * tanhf(v * cap_in);
                        } else {
                            v *= scale2;
                        }
                        x[e] = MODS ? fmaf(slope[nq], (float)(kbase + e - pos[nq]), v) : v;
                    }
                    if (!whole) {
                        const int lo = a.window ? pos[nq] - a.window : -1;
#pragma unroll
                        for (int e = 0; e < E; ++e) {
                            const int j = kbase + e;
                            x[e] = paged_sees(j, n_mine, rq.prefix, pos[nq], lo) ? x[e] : -INFINITY;
                        }
                    }
                    float mx = x[0];
#pragma unroll
                    for (int e = 1; e < E; ++e) mx = fmaxf(mx, x[e]);
                    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
                    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
                    const float m_new = fmaxf(m_run[nq], mx);
                    const float m_sub = m_new == -INFINITY ? 0.f : m_new;   // a row that has seen no key yet
                    const float alpha = __builtin_amdgcn_exp2f(m_run[nq] - m_sub);
                    float p[E], sum = 0.f;
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        p[e] = __builtin_amdgcn_exp2f(x[e] - m_sub);
                        sum += p[e];
                    }
                    l_run[nq] = fmaf(l_run[nq], alpha, sum);
                    m_run[nq] = m_new;
                    if (__any(alpha != 1.f)) {   // the running maximum rarely moves after a row's first steps
#pragma unroll
                        for (int dt = 0; dt < DT; ++dt) oacc[nq][dt] *= alpha;
                    }
                    if (BF) {
#pragma unroll
                        for (int e = 0; e < E / 2; ++e) {
                            uint32_t h, l;
                            split2x2(p[2 * e], p[(2 * e + 1) % E], h, l);
                            phi[nq][e & 3] = h;
                            plo[nq][e & 3] = l;
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) phi[nq][e] = __float_as_uint(p[e]);
                    }
                }
                load_k(nxt);
                if (!whole) {
                    // values behind the end of the request, or of a page that is not there, may be anything: 0 x NaN would
                    // reach every row.  The same holds for values that only some rows see: those that are not finite are
                    // taken out here and added below.
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            uint32_t keep;
                            if (BF) keep = (kbase + 2 * e < n_mine ? 0xffffu : 0u) | (kbase + 2 * e + 1 < n_mine ? 0xffff0000u : 0u);
                            else keep = kbase + e < n_mine ? 0xffffffffu : 0u;
                            const uint32_t w = va[dt][e] & keep;
                            const uint32_t fine = BF ? finite_halves(w) : (w & 0x7f800000u) != 0x7f800000u ? 0xffffffffu : 0u;
                            odd |= w & ~fine;
                            va[dt][e] = w & fine;
                        }
                }
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                    for (int nq = 0; nq < NQ; ++nq) {
                        if (BF) {
                            oacc[nq][dt] = mfma_bf16(va[dt], phi[nq], oacc[nq][dt]);
                            oacc[nq][dt] = mfma_bf16(va[dt], plo[nq], oacc[nq][dt]);
                        } else {
#pragma unroll
                            for (int j = 0; j < 4; ++j) oacc[nq][dt] = mfma_f32(va[dt][j], phi[nq][j], oacc[nq][dt]);
                        }
                    }
                load_v(nxt);
                cur = nxt;
                nxt = step_pages<T, HD>(a, table, g, real(min(s + 2 * NW, s_end - 1)));
            }
            if (__any(odd != 0)) {
                // rare: some value of a step that not every row sees is not finite.  Each row takes those that it sees
#pragma unroll 1
                for (s = s_begin + wave; s < s_end; s += NW) {
                    const int key0 = real(s) * KEYS;
                    const StepPages sp = step_pages<T, HD>(a, table, g, real(s));
                    if (see_all(key0, sp)) continue;
#pragma unroll 1
                    for (int j = key0; j < min(key0 + KEYS, rq.n_keys); ++j) {
                        const int run = j - key0 >= HALF, in = j - key0 - run * HALF;   // (a run of keys begins a group of eight)
                        if (!sp.has[run]) continue;
                        const T *v = vpool + sp.at[run] + (in & ~7) * HD + (in & 7) + 32 * bg;
#pragma unroll
                        for (int nq = 0; nq < NQ; ++nq) {
                            if (!paged_sees(j, rq.n_keys, rq.prefix, pos[nq], a.window ? pos[nq] - a.window : -1)) continue;
#pragma unroll
                            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                                for (int r = 0; r < 4; ++r) oacc[nq][dt][r] += only_not_finite(v[(16 * dt + r) * 8]);
                        }
                    }
                }
            }
        }

        // ---- sums over the four lane groups, then over the waves, in a fixed order
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) {
            const float l1 = l_run[nq] + __shfl_xor(l_run[nq], 16, 64);
            l_run[nq] = l1 + __shfl_xor(l1, 32, 64);
        }
        __syncthreads();   // the tile before has been written out
        if (bg == 0) {
#pragma unroll
            for (int nq = 0; nq < NQ; ++nq) {
                sm[wave][nq][bj] = m_run[nq];
                sl[wave][nq][bj] = l_run[nq];
            }
        }
        __syncthreads();
        float m_all[NQ], l_all[NQ];
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) {
            float mx = -INFINITY, ls = 0.f;
            for (int w = 0; w < NW; ++w) mx = fmaxf(mx, sm[w][nq][bj]);
            const float sub = mx == -INFINITY ? 0.f : mx;
            for (int w = 0; w < NW; ++w) ls = fmaf(sl[w][nq][bj], __builtin_amdgcn_exp2f(sm[w][nq][bj] - sub), ls);
            m_all[nq] = mx;
            l_all[nq] = ls;
            m_run[nq] = __builtin_amdgcn_exp2f(m_run[nq] - sub);   // from here on: the weight of this wave's output
        }
#pragma unroll
        for (int part = 0; part < DT / DP; ++part) {
            if (part) __syncthreads();
#pragma unroll
            for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
                for (int dt = 0; dt < DP; ++dt) so[wave][nq][dt][lane] = oacc[nq][part * DP + dt] * m_run[nq];
            __syncthreads();
            for (int it = wave; it < DP * NQ; it += NW) {
                const int dl = it / NQ, nqs = it % NQ, rho = rho0 + 16 * nqs + bj;
                paged_f4 acc = so[0][nqs][dl][lane];
                for (int w = 1; w < NW; ++w) acc += so[w][nqs][dl][lane];
                float m = m_all[0], l = l_all[0];
#pragma unroll
                for (int nq = 1; nq < NQ; ++nq)
                    if (nqs == nq) { m = m_all[nq]; l = l_all[nq]; }
                if (rho >= R) continue;
                // this lane holds features d .. d + 3 of the row
                const int d = 16 * (part * DP + dl) + 4 * bg, h = g * a.rep + rho % a.rep;
                const int64_t row = rq.row0 + rho / a.rep;
                if (a.n_splits == 1) {
                    const float inv = l == 0.f ? 0.f : 1.f / l;   // a row that sees no key is 0
                    acc *= inv;
                    T *dst = (T *)a.out + row * a.out_stride + (int64_t)h * HD + d;
                    if (BF) *reinterpret_cast<uint2 *>(dst) = make_uint2(f32x2_to_bf16x2(acc[0], acc[1]), f32x2_to_bf16x2(acc[2], acc[3]));
                    else *reinterpret_cast<paged_f4 *>(dst) = acc;
                } else {
                    const int64_t at = ((int64_t)split * a.n_tokens + row) * a.H + h;
                    if (l != 0.f) *reinterpret_cast<paged_f4 *>(a.po + at * HD + d) = acc;   // (a part without keys is not read)
                    if (d == 0) {
                        a.pm[at] = m;
                        a.pl[at] = l;
                    }
                }
            }
        }
    }
}

// out = sum_s 2^(m_s - m*) o_s / sum_s 2^(m_s - m*) l_s over the splits that saw a key.  A thread owns four features of a (row,
// head) and every GROUPS-th split, four of which are on their way at a time; the groups' sums are added in order.  GROUPS 1 fills
// the chip when there are many rows, the whole workgroup on one (row, head) is for few rows of many splits (one row of 32 heads,
// 32 splits: 4.7 us; a wave per (row, head) that takes one split after the other 22.9).
template <typename T, int HD, int GROUPS>
__global__ __launch_bounds__(256) void k_paged_join(PagedAttn a) {
    constexpr int TPI = HD / 4, ITEMS = 256 / (TPI * GROUPS), AHEAD = 4;
    __shared__ float sm[GROUPS][TPI * ITEMS], sd[GROUPS][TPI * ITEMS];
    __shared__ paged_f4 sa[GROUPS][TPI * ITEMS];
    const int tid = threadIdx.x, group = tid / (TPI * ITEMS), in = tid % (TPI * ITEMS), d = in % TPI * 4;
    const int64_t item = (int64_t)blockIdx.x * ITEMS + in / TPI, row = item / a.H;
    const int h = item % a.H;
    const bool live = row >= a.q_start[0] && row < min(a.q_start[a.batch], a.n_tokens);   // other rows stay as they are
    if (GROUPS == 1 && !live) return;
    const int64_t at = (live ? row : 0) * a.H + h, step = (int64_t)a.n_tokens * a.H;
    float mx = -INFINITY, den = 0.f;
    paged_f4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = group; s0 < a.n_splits; s0 += GROUPS * AHEAD) {
        float m[AHEAD], l[AHEAD];
        paged_f4 o[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int64_t from = at + min(s0 + i * GROUPS, a.n_splits - 1) * step;   // (splits past the last re-read it and count as none)
            m[i] = a.pm[from];
            l[i] = s0 + i * GROUPS < a.n_splits ? a.pl[from] : 0.f;
            o[i] = *reinterpret_cast<const paged_f4 *>(a.po + from * HD + d);
        }
        float top = mx;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) top = fmaxf(top, l[i] != 0.f ? fmaxf(m[i], -3e38f) : -INFINITY);   // (scores that are all no numbers: -infinity)
        if (top == -INFINITY) continue;
        const float keep = __builtin_amdgcn_exp2f(mx - top);
        den *= keep;
        acc *= keep;
        mx = top;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (l[i] == 0.f) continue;   // (a split without keys has written no output)
            const float w = __builtin_amdgcn_exp2f(m[i] - top);
            den = fmaf(w, l[i], den);
            acc += o[i] * w;
        }
    }
    if (GROUPS > 1) {
        sm[group][in] = mx;
        sd[group][in] = den;
        sa[group][in] = acc;
        __syncthreads();
        if (group || !live) return;
        float top = -INFINITY;
        for (int i = 0; i < GROUPS; ++i) top = fmaxf(top, sm[i][in]);
        const float sub = top == -INFINITY ? 0.f : top;
        den = 0.f;
        acc = paged_f4{0.f, 0.f, 0.f, 0.f};
        for (int i = 0; i < GROUPS; ++i) {
            const float w = __builtin_amdgcn_exp2f(sm[i][in] - sub);
            den = fmaf(w, sd[i][in], den);
            acc += sa[i][in] * w;
        }
    }
    acc *= den == 0.f ? 0.f : 1.f / den;
    T *dst = (T *)a.out + row * a.out_stride + (int64_t)h * HD + d;
    if (sizeof(T) == 2) *reinterpret_cast<uint2 *>(dst) = make_uint2(f32x2_to_bf16x2(acc[0], acc[1]), f32x2_to_bf16x2(acc[2], acc[3]));
    else *reinterpret_cast<paged_f4 *>(dst) = acc;
}

// ------------------------------------------------------------------------------------------ launch

// Rows of a request that k_paged_rows takes: beyond them it would read the keys twice, and k_paged_prompt, which holds 128, serves
// bf16.  From head_dim 128 on, where its two query tiles do not fit the registers, that kernel is as fast or faster from 17 rows on.  us
// per call, k_paged_rows and k_paged_prompt: 64 requests of 32 rows, over 8192 positions, head_dim 128, two tiles of 16, 370 and 362; over
// 4096, 256, 441 and 355; over 512, 256, 89 and 48; over 8192, 64, 187 and 213; 256 of them over 2048, 64, 221 and 204; 64 of 16 rows over
// 4096, 256, 366 and 361; 37 of two rows over up to 4096, 256, 232 and 291.
static int row_limit(bool bf16, int head_dim) { return bf16 && head_dim >= 128 ? 16 : PAGED_FEW_ROWS; }

PagedCut paged_cut(const PagedAttn &a, bool bf16, int head_dim, int max_new, int max_len) {
    PagedCut c;
    const int64_t rows = (int64_t)a.rep * max_new;
    const bool many = rows > row_limit(bf16, head_dim);
    // Float takes k_paged_prompt's 128 rows where they fill its tiles and the chip: with half the chip's CUs or more, and tiles that a
    // request of average length fills to three quarters or more.  us per call, k_paged_rows and k_paged_prompt: two prompts of 1024
    // behind 1024, 32 / 8 heads of 128, 605 and 518; one of 2048 behind 20000, 8 / 2 of 128, 1707 and 1357; 64 of 100 behind 100, 4 / 4
    // of 64, 46 and 35; too few: one of 200 behind 900, 32 / 8 of 128, 57 and 58; 160 rows each: 24 of 40 tokens behind 4000, 32 / 8 of
    // 64, 338 and 514; head_dim 32: 30 of 500 behind 500, 8 / 2, 157 and 167
    const int64_t all_rows = (int64_t)a.n_tokens * a.rep, tiles_each = (all_rows + 128 * (int64_t)a.batch - 1) / (128 * (int64_t)a.batch);
    c.prompt = many && (bf16 || (head_dim >= 64 && all_rows / 128 * a.G >= 128 && all_rows >= 96 * tiles_each * a.batch));
    // positions that a tile's rows see at most: a window's are those of its first row and what its rows span.  (A prefix in front of the
    // window is not counted, and the last split has all that is left: one token over 12000 positions, 32 / 8 heads of 128, without a window
    // 16.5 us, with one of 512 11, and with a prefix of 8000 80.)
    const int reach = a.window ? (int)std::min<int64_t>(max_len, (int64_t)a.window + 64 + (c.prompt ? 128 / a.rep : max_new)) : max_len;
    const int64_t steps = (reach + 63) / 64;
    if (c.prompt) {
        // Splitting the keys fills a chip, or the last of its rounds, that is not full.  In steps of 64 keys, in bf16 about 2 us each: a
        // split costs six (its start, its way to the join), the join three and the parts' way through memory; float steps are as much
        // longer as its products.  us per call: six prompts of up to 777 behind 900, 28 / 4 heads of 64, with a bias 1 split 43, 2 36.7, 3
        // 36.0, 4 36.2, the rule's 35.0; one of 723 behind 20990, 56 / 8 of 64, with a cap 1 split 548, 2 (taken) 490, 3 437, 4 420: there
        // the charge for rounds that are not whole is too high; two of 2048 behind 6144, 32 / 8 of 128, 1 (taken) 482, 2 537; float, one of
        // 2048 behind 20000, 8 / 2 of 128, with a cap 3417, 2636, 1993, 4 (taken) 1518, 6 1567
        const double wgs = (double)std::max<int64_t>(((int64_t)a.n_tokens * a.rep + 127) / 128, a.batch) * a.G, slots = 256 * paged_prompt_wgs(bf16, head_dim);
        const double fixed = bf16 ? 1 : 18.0 / head_dim;
        const double part = (double)a.n_tokens * a.H * head_dim * 8 / 9e6;
        double best = 0;
        c.n_splits = 1;
        for (int s = 1; s <= 32 && (s == 1 || steps / s >= 2); ++s) {
            const double rounds = wgs * s / slots, cost = (rounds <= 1 ? 1 : rounds + (bf16 ? 0.25 : 0.5)) * ((double)steps / s + 6 * fixed) + (s > 1 ? (3 + s * part) * fixed : 0);
            if (s == 1 || cost < best) best = cost, c.n_splits = s;
        }
    } else {
        // One workgroup per CU.  In us: 64 keys of a head come into a CU at about 36 GB/s, a split costs 6 (its start and its
        // end), the join, its launch and its workspace 9 and the parts' way through memory.  us per call: 36 tokens in windows of 4096, 16 /
        // 8 heads of 256, 1 split 116, 2 96, 3 96, 4 (taken) 92, 6 102; four rows over 516, 32 / 8 of 128, 1 (taken) 12.5, 2 15.7, 4
        // 15.5, over 2004 25.7, 20.2, 16.7; 16 single tokens over 1001, 1 (taken) 18.1, 2 20.0, 4 24.6
        const int64_t wgs = (many ? std::max<int64_t>((int64_t)a.n_tokens * a.rep / (head_dim == 256 ? 16 : 32), a.batch) : a.batch) * a.G;
        const double unit = 128.0 * head_dim * (bf16 ? 2 : 4) / 36e3, part = (double)a.n_tokens * a.H * head_dim * 8 / 4e6;
        double best = 0;
        c.n_splits = 1;
        for (int s = 1; s <= PAGED_MAX_SPLITS && (s == 1 || steps / s >= 2); ++s) {
            const double cost = (double)((wgs * s + 255) / 256) * (unit * steps / s + 6) + (s > 1 ? 9 + s * part : 0);
            if (s == 1 || cost < best) best = cost, c.n_splits = s;
        }
    }
    c.split_steps = (int)((steps + c.n_splits - 1) / c.n_splits);
    c.workspace = c.n_splits == 1 ? 0 : (size_t)c.n_splits * a.n_tokens * a.H * (head_dim + 2) * 4;
    return c;
}

template <typename T, int HD, int NQ> static void launch_rows(const PagedAttn &a, hipStream_t stream) {
    const dim3 grid((a.tiles ? (unsigned)((int64_t)a.n_tokens * a.rep / (16 * NQ) + a.batch) : a.batch) * a.G, a.n_splits);
    if (a.softcap > 0.f || a.slopes) hipLaunchKernelGGL((k_paged_rows<T, HD, NQ, true>), grid, dim3(64 * rows_waves(HD, NQ)), 0, stream, a);
    else hipLaunchKernelGGL((k_paged_rows<T, HD, NQ, false>), grid, dim3(64 * rows_waves(HD, NQ)), 0, stream, a);
}
template <typename T, int HD> static void launch_rows_t(const PagedAttn &a, bool two, hipStream_t stream) {
    if constexpr (HD == 256 || (sizeof(T) == 2 && HD == 128)) return launch_rows<T, HD, 1>(a, stream);   // (bf16, head_dim 128: row_limit)
    else return two ? launch_rows<T, HD, 2>(a, stream) : launch_rows<T, HD, 1>(a, stream);
}
template <typename T> static void launch_rows_d(const PagedAttn &a, int head_dim, bool two, hipStream_t stream) {
    switch (head_dim) {
        case 32: return launch_rows_t<T, 32>(a, two, stream);
        case 64: return launch_rows_t<T, 64>(a, two, stream);
        case 128: return launch_rows_t<T, 128>(a, two, stream);
        default: return launch_rows_t<T, 256>(a, two, stream);
    }
}
template <typename T, int HD> static void launch_join_t(const PagedAttn &a, hipStream_t stream) {
    constexpr int ALL = 1024 / HD;   // groups that a workgroup has for one (row, head)
    const int64_t items = (int64_t)a.n_tokens * a.H;
    if (a.n_splits > 8 && items <= 1 << 16) hipLaunchKernelGGL((k_paged_join<T, HD, ALL>), dim3((unsigned)items), dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((k_paged_join<T, HD, 1>), dim3((unsigned)((items + ALL - 1) / ALL)), dim3(256), 0, stream, a);
}
template <typename T> static void launch_join(const PagedAttn &a, int head_dim, hipStream_t stream) {
    switch (head_dim) {
        case 32: return launch_join_t<T, 32>(a, stream);
        case 64: return launch_join_t<T, 64>(a, stream);
        case 128: return launch_join_t<T, 128>(a, stream);
        default: return launch_join_t<T, 256>(a, stream);
    }
}

const char *launch_paged_attention(PagedAttn a, bool bf16, int head_dim, int max_new, int max_len, int device, hipStream_t stream) {
    const PagedCut cut = paged_cut(a, bf16, head_dim, max_new, max_len);
    a.n_splits = cut.n_splits;
    if (cut.prompt) {
        a.split_steps = cut.split_steps;
        if (const char *why = launch_paged_prompt(a, bf16, head_dim, (int64_t)a.rep * max_new <= PAGED_FEW_ROWS, device, stream)) return why;
    } else {
        a.split_steps = cut.split_steps * (bf16 ? 2 : 4);
        const int64_t rows = (int64_t)a.rep * max_new;
        // Two query tiles per wave read the keys half as often; one where that leaves few workgroups (float, 5 requests of up to 37
        // rows, 4 KV heads: 15.8 us and 12.8) and at head_dim 256, where two do not fit the registers (float, 23 prompts of 400, one
        // KV head, when this kernel served them: 785 us and 634)
        const bool two = rows > 16 && head_dim < 256 && ((int64_t)a.n_tokens * a.rep / 32 + 1) * a.G >= 32;
        a.tiles = rows > (two ? row_limit(bf16, head_dim) : 16);
        if (bf16) launch_rows_d<bf16_t>(a, head_dim, two, stream);
        else launch_rows_d<float>(a, head_dim, two, stream);
    }
    if (a.n_splits > 1) {
        if (bf16) launch_join<bf16_t>(a, head_dim, stream);
        else launch_join<float>(a, head_dim, stream);
    }
    return nullptr;
}

}  // namespace wisv
