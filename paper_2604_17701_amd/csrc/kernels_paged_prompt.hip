// Attention of many rows over the paged cache: prompts, and blocks of more rows than k_paged_rows takes at once.
//
// A workgroup takes 128 rows of a request and KV head (its new tokens x the query heads that share the KV head), 32 per wave; keys
// and values pass through LDS in blocks of 64 positions (float, and head_dim 256: 32), one read while the next arrives straight from
// the pages (global_load_lds, 16 bytes a lane; a wave fetches the keys and the values of the same sixteen (8) positions, which lie in
// one page).  On 32x32x16 products of bf16:
//   S^T = K Q^T    the A operand's rows are dealt (bits 2 and 3 of the row swapped) so that a lane's sixteen scores of a tile are
//                  two runs of eight consecutive keys of one query ...
//   O^T += V^T P^T ... which are, rounded to bf16, the B operand as they stand; the A operand is one 16-byte LDS read from the V
//                  pool's own order.
// Keys lie in LDS with their 16-byte chunks exchanged by an XOR of the row, so that neither operand's reads meet in a bank
// (SQ_LDS_BANK_CONFLICT 0).  A query's scores lie in two lanes: a maximum costs one exchange.  The running maximum is a reference that
// moves only when a score exceeds it by 2^8 (sums and outputs are float: nothing is lost by a reference that is too low), so that
// rescaling the outputs is rare.
// Probabilities enter the product as one bf16 term, an error of at most 2^-8 relative each, in the mean like that of the output's own
// rounding: the error against 64 bits is 1.1 to 1.35 times that of a result rounded once.  Two terms cost 478 -> 600 us (below).  Where the
// hint says that requests have at most 32 rows, one wave of a tile, memory is the bound and they are two terms p = hi + lo, |p - hi - lo| <=
// 2^-17 p: 64 of 8 tokens over 8192, 32 / 8 heads of 128, 359 -> 363 us, with a cap 363 -> 390.  For 64 rows they would cost 361 -> 388.
// Float multiplies by 32x32x2 products: a lane's sixteen scores of a tile are four runs of four keys, in the order of the B operand's
// halves, and the probabilities enter as they are.
//
// bf16 is bound by the matrix cores and the vector unit, which a SIMD's two or three waves, of different workgroups, overlap (the waves
// of one workgroup run in step), and long calls by power: two prompts of 2048 behind 6144, 32 / 8 heads of 128, keep the matrix cores
// busy 52 % of the cycles of a clock that falls to 1.9 GHz.  us per call among others: these (481 GFLOP) 454 to 482 = 1.0 to 1.06
// PFLOP/s, of a library product's 1.21; the same prompts with 32 / 8 of 64 (241 GFLOP) 290, 16 / 8 of 256 (481 GFLOP) 510; 12 of 855
// behind 187 with a cap, 32 / 8 of 128 (103 GFLOP) 185: a cap is two transcendentals a score more.  With up to 32 rows per request it is
// bound by memory: 64 of 8 tokens over 8192, 32 / 8 of 128 (2.16 GB) 363 = 5.9 TB/s.  A step of 64 keys alone on its CU takes 1.1 us at
// head_dim 64, 1.4 at 128, spread over loads, products, exponentials and maxima.
// Workgroups that share a CU count for more than blocks on their way: rings of 64 KB, for two workgroups, against these two blocks, for
// three, the prompts above at head_dim 64 341 and 292, at 32 240 and 206.  At head_dim 128 three need blocks of 32 positions: 12 of 855
// behind 187 164 and 156, but the prompts above 480 and 573, whose 1024 workgroups are no whole rounds of 768, and 64 of 32 over 8192
// 403 and 440: two.  At head_dim 256 blocks of 32 leave registers for two instead of one: the prompts above 682 and 509, one workgroup
// with such blocks 828.
// Two workgroups of four waves against one of eight with the keys loaded half as often: 503 and 499 us for the prompts above, six of up
// to 777 behind 900, 28 / 4 heads of 64, with a bias 53 and 72.  Priority to the phases of products: 481 -> 460, one of 723 behind 20990,
// 56 / 8 of 64, with a cap 464 -> 436.  The next block's scores beside this block's exponentials in one wave, blocks of 32: 655 -> 735.
// Float is bound by the matrix cores, whose 64 cycles a product hide the rest: one prompt of 2048 behind 20000, 8 / 2 heads of 128 (176
// GFLOP) 1357 us = 130 TFLOP/s (k_paged_rows 1707; a library's product of 8192^3 153).
#include <atomic>

#include "paged.h"

namespace wisv {

typedef float paged_f16 __attribute__((ext_vector_type(16)));
typedef __bf16 paged_bf16x2 __attribute__((ext_vector_type(2)));
template <typename T, int HD> constexpr int BLOCK = sizeof(T) == 2 && HD < 256 ? 64 : 32;   // positions

__device__ __forceinline__ paged_f16 mfma32(paged_u4 a, paged_u4 b, paged_f16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<paged_bf16x8 *>(&a), *reinterpret_cast<paged_bf16x8 *>(&b), c, 0, 0, 0);
}
__device__ __forceinline__ paged_f16 mfma32(uint32_t a, uint32_t b, paged_f16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a), __uint_as_float(b), c, 0, 0, 0);
}
// lane l: 16 bytes from base + voff to lds_addr + 16 l
__device__ __forceinline__ void page_to_lds(uint32_t lds_addr, uint32_t voff, const void *base) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds_addr), "v"(voff), "s"(base) : "memory", "m0");
}

constexpr int PROMPT_WAVES = 4;
template <typename T, int HD> constexpr int prompt_lds() { return 4 * BLOCK<T, HD> * HD * (int)sizeof(T); }   // two blocks of keys and of values
enum { PLAIN = 0, CAP = 1, BIAS = 2 };   // what MODS adds to the scores

// TERMS: bf16 terms of a probability (float: one)
template <typename T, int HD, int MODS, int TERMS>
__global__ __launch_bounds__(64 * PROMPT_WAVES, paged_prompt_wgs(sizeof(T) == 2, HD)) void k_paged_prompt(PagedAttn a) {
    extern __shared__ __align__(16) unsigned char lds[];   // [2][K, V][BLOCK * HD]
    constexpr bool BF = sizeof(T) == 2;
    constexpr int BLOCK = wisv::BLOCK<T, HD>, RUNS = BLOCK / 16, TILES = BLOCK / 32, PER = 16 / (int)sizeof(T);   // PER: elements in 16 bytes
    constexpr int ROWS = 32 * PROMPT_WAVES, CPR = HD / PER, QT = CPR / 2, OT = HD / 32;
    constexpr float LOG2E = 1.4426950408889634f;
    constexpr int HALF = BLOCK * HD * (int)sizeof(T), BUF = 2 * HALF;   // bytes
    constexpr int OWN = BLOCK / PROMPT_WAVES, LOADS = OWN * CPR / 64;   // positions a wave fetches, in loads of 1 KB of either pool
    static_assert(LOADS * 64 == OWN * CPR, "whole loads");
    const int tid = threadIdx.x, lane = tid & 63, h2 = lane >> 5, qi = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = blockIdx.x % a.G, split = blockIdx.y;
    const PagedTile mine = paged_find(a, blockIdx.x / a.G, ROWS, lane);
    if (mine.b < 0) return;
    const int b = mine.b;
    const PagedRequest rq = paged_request(a, b);
    const int R = rq.n_new * a.rep;
    const int rho0 = ((R + ROWS - 1) / ROWS - 1 - mine.index) * ROWS;   // a request's later rows see more keys: they start first
    const PagedSteps st = paged_steps(rq, rq.pos0 + rho0 / a.rep, rq.pos0 + (min(rho0 + ROWS, R) - 1) / a.rep, a.window, BLOCK);
    const int s_begin = split * a.split_steps, s_end = split == a.n_splits - 1 ? st.total : min(st.total, s_begin + a.split_steps);
    const paged_ints table = (paged_ints)(uintptr_t)(a.block_table + (int64_t)b * a.max_pages);
    const auto real = [&](int v) { return v < st.n_pre ? v : v + st.skip; };

    const int tile_min = rq.pos0 + rho0 / a.rep, tile_max = rq.pos0 + (min(rho0 + ROWS, R) - 1) / a.rep;

    // ---- this wave's rows
    const int wrow = rho0 + 32 * wave;
    const bool busy = wrow < R;
    const int pos_min = rq.pos0 + min(wrow, R - 1) / a.rep, pos_max = rq.pos0 + min(wrow + 31, R - 1) / a.rep;
    const int rho = min(wrow + qi, R - 1), tok = rho / a.rep, head = g * a.rep + rho % a.rep, pos = rq.pos0 + tok;
    const int lo = a.window ? pos - a.window : -1;   // the position before the window
    const float slope = (MODS & BIAS) && a.slopes ? a.slopes[head] * LOG2E : 0.f;
    paged_u4 q[QT];   // lane: features PER (2 t + h2) .. of its row
    {
        const T *src = (const T *)a.q + (int64_t)(rq.row0 + tok) * a.q_stride + (int64_t)head * HD + PER * h2;
#pragma unroll
        for (int t = 0; t < QT; ++t) q[t] = *reinterpret_cast<const paged_u4 *>(src + 2 * PER * t);
    }

    // ---- holes in the part of the table that this workgroup reads: then every block is looked at
    bool hole = false;
    if (s_begin < s_end) {
        const int p0 = (real(s_begin) * BLOCK) >> a.page_shift, p1 = (min((real(s_end - 1) + 1) * BLOCK, rq.n_keys) - 1) >> a.page_shift;
        for (int p = p0 + tid; p <= p1; p += 64 * PROMPT_WAVES) hole |= (unsigned)a.block_table[(int64_t)b * a.max_pages + p] >= (unsigned)a.n_pages;
    }
    hole = __syncthreads_or(hole);

    // ---- fetching: every wave fetches OWN positions of a block, which lie in one page, of both pools.  Chunk c of key row r
    //      lies at chunk c ^ swizzle(r) in LDS, the values as they lie in the pool
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)lds + wave * OWN * HD * (int)sizeof(T);
    constexpr int SWZ_SHIFT = CPR == 4 ? 2 : CPR == 8 ? 1 : 0, SWZ_MASK = CPR >= 16 ? 15 : CPR - 1;
    uint32_t koff[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int r = i * (64 / CPR) + lane / CPR;
        koff[i] = r * CPR * 16 + ((lane % CPR) ^ (((wave * OWN + r) >> SWZ_SHIFT) & SWZ_MASK)) * 16;
    }
    const auto place = [&](int step) {   // elements from a pool's start to this wave's positions
        const int key = step * BLOCK + OWN * wave;
        const int id = table[min(key >> a.page_shift, a.max_pages - 1)];
        return (int64_t)((unsigned)id < (unsigned)a.n_pages ? id : 0) * a.page_stride + (((int64_t)g << a.page_shift) + (key & ((1 << a.page_shift) - 1))) * HD;
    };
    const auto fetch = [&](int64_t at, int stage) __attribute__((always_inline)) {
        const uint32_t to = lds0 + stage * BUF;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) page_to_lds(to + i * 1024, koff[i], (const T *)a.k_pages + at);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) page_to_lds(to + HALF + i * 1024, i * 1024 + lane * 16, (const T *)a.v_pages + at);
    };

    // ---- reading: K rows (bf16: with bits 2 and 3 swapped), chunk 2 t + h2; of V the group of eight keys 2 kc + h2 (float: half h2
    //      of a group, four keys).  Register r of tile i of the scores is then key 32 i + key_of(r) + first
    const int krow = BF ? (qi & ~12) | ((qi & 4) << 1) | ((qi & 8) >> 1) : qi;
    const uint32_t kaddr = krow * CPR * 16 + ((h2 ^ ((krow >> SWZ_SHIFT) & SWZ_MASK)) * 16);   // of chunk h2; chunk 2 t + h2 lies at kaddr ^ 32 t
    const uint32_t vaddr = HALF + (BF ? (h2 * HD + qi) * 16 : qi * 32 + h2 * 16);
    const auto key_of = [](int r) { return BF ? 16 * (r >> 3) + (r & 7) : 8 * (r >> 2) + (r & 3); };
    const int first = (BF ? 8 : 4) * h2;

    // every row from position p0 to p1 sees every key of the block
    const auto see_all = [&](int key0, int p0, int p1) {
        return !hole && key0 + BLOCK <= rq.n_keys &&
               (key0 + BLOCK <= rq.prefix || (key0 + BLOCK - 1 <= p0 && (!a.window || key0 > p1 - a.window)));
    };
    const auto see_none = [&](int key0) {   // no row of the wave sees any
        return !busy || (key0 >= rq.prefix && (key0 > pos_max || (a.window && key0 + BLOCK - 1 <= pos_min - a.window)));
    };
    const auto runs_there = [&](int key0) {   // bit i: run i of sixteen keys is in a page
        uint32_t ok = (1u << RUNS) - 1;
        if (hole) {
            ok = 0;
            for (int i = 0; i < RUNS; ++i) {
                const int key = key0 + 16 * i;
                if (key < rq.n_keys && (unsigned)table[key >> a.page_shift] < (unsigned)a.n_pages) ok |= 1u << i;
            }
        }
        return ok;
    };

    int odd = 0;   // whether a value was not finite, of the blocks that not every row of the workgroup sees
    float m_ref = -INFINITY, l_run[2] = {0.f, 0.f};
    paged_f16 o[OT];
#pragma unroll
    for (int dt = 0; dt < OT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
    const float scale2 = a.scale * LOG2E;                                                   // scores in units of ln 2
    const float cap_in = (BF ? 2.f * scale2 : a.scale) / a.softcap, cap_out = a.softcap * LOG2E;             // (CAP only)
    const paged_f16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};

    int64_t at_next = 0;   // where this wave's positions of the next block to be fetched lie
    if (s_begin < s_end) {
        fetch(place(real(s_begin)), 0);
        at_next = place(real(min(s_begin + 1, s_end - 1)));
    }
    for (int s = s_begin; s < s_end; ++s) {
        // block s has arrived, everybody's part of it, and nobody reads block s - 1 any more; its place takes block s + 1
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        const int stage = (s - s_begin) & 1, key0 = real(s) * BLOCK;
        if (s + 1 < s_end) {
            fetch(at_next, stage ^ 1);
            at_next = place(real(min(s + 2, s_end - 1)));
        }
        if (!see_all(key0, tile_min, tile_max)) {
            // values behind the end of the request, or of a page that is not there, may be anything: 0 x NaN would reach every row.
            // The same holds for values that only some rows see: those that are not finite are taken out and added at the end.
            const uint32_t ok = runs_there(key0);
            uint32_t out = 0;
            for (int i = tid; i < HALF / 16; i += 64 * PROMPT_WAVES) {
                const int key = BF ? i / HD * 8 : i / (2 * HD) * 8 + (i & 1) * 4;            // the first of the chunk's PER keys
                const int n = ok >> (key >> 4) & 1 ? rq.n_keys - (key0 + key) : 0;          // of them
                paged_u4 *to = reinterpret_cast<paged_u4 *>(lds + stage * BUF + HALF) + i;
                paged_u4 v = *to;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    v[w] &= BF ? (2 * w < n ? 0xffffu : 0u) | (2 * w + 1 < n ? 0xffff0000u : 0u) : w < n ? 0xffffffffu : 0u;
                    const uint32_t fine = BF ? finite_halves(v[w]) : (v[w] & 0x7f800000u) != 0x7f800000u ? 0xffffffffu : 0u;
                    out |= v[w] & ~fine;
                    v[w] &= fine;
                }
                *to = v;
            }
            odd |= __syncthreads_or(out != 0);
        }
        if (see_none(key0)) continue;
        // ---- scores
        paged_f16 x[TILES];
        __builtin_amdgcn_s_setprio(1);   // products first: the other workgroup's wave has its exponentials meanwhile
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
            for (int i = 0; i < TILES; ++i) {
                const paged_u4 k = *reinterpret_cast<const paged_u4 *>(lds + ((kaddr + stage * BUF) ^ (32 * t)) + i * 32 * HD * (int)sizeof(T));
                if constexpr (BF) {
                    x[i] = mfma32(k, q[t], t ? x[i] : zero);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[i] = mfma32(k[j], q[t][j], t || j ? x[i] : zero);
                }
            }
        __builtin_amdgcn_s_setprio(0);
        if (MODS != PLAIN) {   // into units of ln 2, with cap and bias (PLAIN scales them with the exponentials)
            const float near = slope * (float)(key0 + first - pos);
#pragma unroll
            for (int i = 0; i < TILES; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float bias = MODS & BIAS ? fmaf(slope, (float)(32 * i + key_of(r)), near) : 0.f;
                    if (MODS & CAP) {
                        // tanh = 1 - 2 / (exp(2 x) + 1)
                        if (BF) x[i][r] = fmaf(__builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(x[i][r] * cap_in) + 1.f), -2.f * cap_out, cap_out + bias);
                        else x[i][r] = fmaf(cap_out, tanhf(x[i][r] * cap_in), bias);
                    } else {
                        x[i][r] = fmaf(x[i][r], scale2, bias);
                    }
                }
        }
        if (!see_all(key0, pos_min, pos_max)) {
            const uint32_t ok = runs_there(key0);
#pragma unroll
            for (int i = 0; i < TILES; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int run = 2 * i + (key_of(r) >> 4), j = key0 + 32 * i + key_of(r) + first;
                    x[i][r] = paged_sees(j, ok >> run & 1 ? rq.n_keys : 0, rq.prefix, pos, lo) ? x[i][r] : -INFINITY;
                }
        }
        // (the maximum that lets NaN through is one instruction for two values; a row with one is NaN whatever the reference)
        float part[2 * TILES];
#pragma unroll
        for (int i = 0; i < 2 * TILES; ++i) {
            part[i] = x[i >> 1][8 * (i & 1)];
#pragma unroll
            for (int r = 1; r < 8; ++r) part[i] = __builtin_elementwise_maximum(part[i], x[i >> 1][8 * (i & 1) + r]);
        }
        float mx = part[0];
#pragma unroll
        for (int i = 1; i < 2 * TILES; ++i) mx = __builtin_elementwise_maximum(mx, part[i]);
        const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);   // the lower and the upper lanes', in all
        mx = __builtin_elementwise_maximum(__uint_as_float(halves[0]), __uint_as_float(halves[1]));
        if (MODS == PLAIN) mx *= scale2;
        if (__any(mx > m_ref + 8.f)) {
            const float m_new = fmaxf(m_ref, mx);
            const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_ref - m_new);
            m_ref = m_new;
            l_run[0] *= alpha;
            l_run[1] *= alpha;
#pragma unroll
            for (int dt = 0; dt < OT; ++dt) o[dt] *= alpha;
        }
        const float sub = m_ref == -INFINITY ? 0.f : m_ref;   // a row that has seen no key yet
        if constexpr (BF) {
            paged_u4 p[RUNS], rest[RUNS];   // (rest: the second terms)
            const auto probs = [&](int kc) __attribute__((always_inline)) {
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const float x0 = x[kc >> 1][8 * (kc & 1) + 2 * w], x1 = x[kc >> 1][8 * (kc & 1) + 2 * w + 1];
                    const float e0 = __builtin_amdgcn_exp2f(MODS ? x0 - sub : fmaf(x0, scale2, -sub)), e1 = __builtin_amdgcn_exp2f(MODS ? x1 - sub : fmaf(x1, scale2, -sub));
                    if constexpr (TERMS == 2) {
                        uint32_t hi, lo;
                        split2x2(e0, e1, hi, lo);
                        p[kc][w] = hi;
                        rest[kc][w] = lo;
                        l_run[w & 1] += e0 + e1;
                    } else {
                        const uint32_t both = f32x2_to_bf16x2(e0, e1);
                        p[kc][w] = both;
                        // (the sum of what the product weighs with: rounding errors that all probabilities share cancel)
                        l_run[w & 1] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(paged_bf16x2, both), __builtin_bit_cast(paged_bf16x2, 0x3f803f80u), l_run[w & 1], false);
                    }
                }
            };
            // a run of sixteen keys' products, and the next run's exponentials beside them
            probs(0);
            __builtin_amdgcn_s_setprio(1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int kc = 0; kc < RUNS; ++kc) {
#pragma unroll
                for (int dt = 0; dt < OT; ++dt) {
                    const paged_u4 v = *reinterpret_cast<const paged_u4 *>(lds + vaddr + stage * BUF + (2 * kc * HD + 32 * dt) * 16);
                    o[dt] = mfma32(v, p[kc], o[dt]);
                    if constexpr (TERMS == 2) o[dt] = mfma32(v, rest[kc], o[dt]);
                }
                if (kc < RUNS - 1) probs(kc + 1);
                __builtin_amdgcn_sched_barrier(0);
            }
            __builtin_amdgcn_s_setprio(0);
        } else {
            // (exact in float; the products are 25 times the exponentials)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                x[0][r] = __builtin_amdgcn_exp2f(MODS ? x[0][r] - sub : fmaf(x[0][r], scale2, -sub));
                l_run[r & 1] += x[0][r];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int dt = 0; dt < OT; ++dt) {
                    const paged_u4 v = *reinterpret_cast<const paged_u4 *>(lds + vaddr + stage * BUF + (i * HD + 32 * dt) * 32);
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[dt] = mfma32(v[j], __float_as_uint(x[0][4 * i + j]), o[dt]);
                }
        }
    }

    if (odd) {
        // rare: a value that is not finite has been taken out.  Each row adds those that it sees (a second time where it has: they
        // stay what they are)
#pragma unroll 1
        for (int s = s_begin; s < s_end; ++s) {
            const int key0 = real(s) * BLOCK;
#pragma unroll 1
            for (int j = key0; j < min(key0 + BLOCK, rq.n_keys); ++j) {
                const int id = table[j >> a.page_shift], in = j & ((1 << a.page_shift) - 1);
                if ((unsigned)id >= (unsigned)a.n_pages || !paged_sees(j, rq.n_keys, rq.prefix, pos, lo)) continue;
                const T *v = (const T *)a.v_pages + (int64_t)id * a.page_stride + (((int64_t)g << a.page_shift) + (in & ~7)) * HD + (in & 7) + 32 * h2;
#pragma unroll
                for (int dt = 0; dt < OT; ++dt)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[dt][r] += only_not_finite(v[(32 * dt + 8 * (r >> 2) + (r & 3)) * 8]);
            }
        }
    }

    float l = l_run[0] + l_run[1];
    l += __shfl_xor(l, 32, 64);
    if (wrow + qi >= R) return;
    const int64_t row = rq.row0 + tok;
    if (a.n_splits == 1) {
        const float inv = l == 0.f ? 0.f : 1.f / l;   // a row that sees no key is 0
        T *dst = (T *)a.out + row * a.out_stride + (int64_t)head * HD + 4 * h2;
#pragma unroll
        for (int dt = 0; dt < OT; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const paged_f4 v = paged_f4{o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]} * inv;
                if (BF) *reinterpret_cast<uint2 *>(dst + 32 * dt + 8 * i) = make_uint2(f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]));
                else *reinterpret_cast<paged_f4 *>(dst + 32 * dt + 8 * i) = v;
            }
    } else {
        const int64_t to = ((int64_t)split * a.n_tokens + row) * a.H + head;
        if (l != 0.f) {   // (a part without keys is not read)
#pragma unroll
            for (int dt = 0; dt < OT; ++dt)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *reinterpret_cast<paged_f4 *>(a.po + to * HD + 32 * dt + 8 * i + 4 * h2) = paged_f4{o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]};
        }
        if (h2 == 0) {
            a.pm[to] = m_ref;
            a.pl[to] = l;
        }
    }
}

int paged_prompt_tiles(const PagedAttn &a) { return (int)((int64_t)a.n_tokens * a.rep / (32 * PROMPT_WAVES)) + a.batch; }

template <typename T, int HD, int MODS, int TERMS> static const char *launch_t(PagedAttn a, int device, hipStream_t stream) {
    a.split_steps *= 64 / BLOCK<T, HD>;
    static std::atomic<bool> allowed[MAX_DEVICES];   // a cache of an idempotent call (of any thread), not state that results depend on
    constexpr int lds = prompt_lds<T, HD>();
    if (!(device >= 0 && device < MAX_DEVICES && allowed[device])) {
        if (hipFuncSetAttribute(reinterpret_cast<const void *>(&k_paged_prompt<T, HD, MODS, TERMS>), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess) {
            (void)hipGetLastError();
            return "the device refuses the kernel's LDS request";
        }
        if (device >= 0 && device < MAX_DEVICES) allowed[device] = true;
    }
    hipLaunchKernelGGL((k_paged_prompt<T, HD, MODS, TERMS>), dim3(paged_prompt_tiles(a) * a.G, a.n_splits), dim3(64 * PROMPT_WAVES), lds, stream, a);
    return nullptr;
}
template <typename T, int HD, int TERMS> static const char *launch_m(const PagedAttn &a, int device, hipStream_t stream) {
    const bool cap = a.softcap > 0.f;
    // (PLAIN scales the maximum in the place of the scores, which only a positive scale keeps a maximum)
    if (a.slopes || (a.scale < 0.f && !cap)) return cap ? launch_t<T, HD, CAP | BIAS, TERMS>(a, device, stream) : launch_t<T, HD, BIAS, TERMS>(a, device, stream);
    return cap ? launch_t<T, HD, CAP, TERMS>(a, device, stream) : launch_t<T, HD, PLAIN, TERMS>(a, device, stream);
}
template <int HD> static const char *launch_bf16(const PagedAttn &a, bool few, int device, hipStream_t stream) {
    if constexpr (HD >= 128)   // (smaller heads: few rows are k_paged_rows's, by paged_cut)
        if (few) return launch_m<bf16_t, HD, 2>(a, device, stream);
    return launch_m<bf16_t, HD, 1>(a, device, stream);
}
const char *launch_paged_prompt(const PagedAttn &a, bool bf16, int head_dim, bool few, int device, hipStream_t stream) {
    switch (head_dim) {
        case 32: return bf16 ? launch_bf16<32>(a, few, device, stream) : "no such kernel";   // (float, head_dim 32: k_paged_rows, by paged_cut)
        case 64: return bf16 ? launch_bf16<64>(a, few, device, stream) : launch_m<float, 64, 1>(a, device, stream);
        case 128: return bf16 ? launch_bf16<128>(a, few, device, stream) : launch_m<float, 128, 1>(a, device, stream);
        default: return bf16 ? launch_bf16<256>(a, few, device, stream) : launch_m<float, 256, 1>(a, device, stream);
    }
}

}  // namespace wisv
