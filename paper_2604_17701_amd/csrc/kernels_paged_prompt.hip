// Attention of many rows over the paged cache (bf16): prompts, and blocks of more rows than k_paged_rows takes at once.
//
// Bound by the matrix cores.  A workgroup takes 32 NW rows of a request and KV head (its new tokens x the query heads that
// share the KV head), 32 per wave; keys and values pass through LDS in blocks of 64 positions, two buffers deep, loaded
// straight from the pages (global_load_lds, 16 bytes a lane; a wave fetches the keys and the values of the same few
// positions, so that it needs one page number).  On 32x32x16 products:
//   S^T = K Q^T    the A operand's rows are dealt (bits 2 and 3 of the row swapped) so that a lane's sixteen scores of a tile are
//                  two runs of eight consecutive keys of one query ...
//   O^T += V^T P^T ... which are, rounded to bf16, the B operand as they stand; the A operand is one 16-byte LDS read from the V
//                  pool's own order.
// Keys lie in LDS with their 16-byte chunks exchanged by an XOR of the row, so that neither operand's reads meet in a bank.
// A query's scores lie in two lanes: a maximum costs one exchange.  The running maximum is a reference that moves only when a
// score exceeds it by 2^8 (sums and outputs are float: nothing is lost by a reference that is too low), so that rescaling the
// outputs is rare.
// Probabilities enter the product as one bf16 term, an error of 2^-8 relative each and of about 2^-9.3 in the mean, like that of the
// output's own rounding; a second term would cost half as many matrix instructions again.
#include "paged.h"

namespace wisv {

typedef float paged_f16 __attribute__((ext_vector_type(16)));
constexpr int BLOCK = 64;   // positions

__device__ __forceinline__ paged_f16 mfma32(paged_u4 a, paged_u4 b, paged_f16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<paged_bf16x8 *>(&a), *reinterpret_cast<paged_bf16x8 *>(&b), c, 0, 0, 0);
}
// lane l: 16 bytes from base + voff to lds_addr + 16 l
__device__ __forceinline__ void page_to_lds(uint32_t lds_addr, uint32_t voff, const void *base) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds_addr), "v"(voff), "s"(base) : "memory", "m0");
}

// waves of a workgroup, and what they leave of a SIMD's registers: two waves per SIMD overlap one's softmax with the other's
// products; head_dim 256 needs the registers of one
constexpr int prompt_waves(int hd) { return hd == 256 ? 4 : 8; }
constexpr size_t prompt_lds(int hd) { return (size_t)2 * 2 * BLOCK * hd * 2; }

template <int HD, bool MODS>
__global__ __launch_bounds__(64 * prompt_waves(HD), HD == 256 ? 1 : 2) void k_paged_prompt(PagedAttn a) {
    extern __shared__ __align__(16) unsigned char lds[];   // [2 buffers][K, V][BLOCK * HD]
    constexpr int NWV = prompt_waves(HD), ROWS = 32 * NWV, CPR = HD / 8, QT = HD / 16, OT = HD / 32;
    constexpr int HALF = BLOCK * HD * 2, BUF = 2 * HALF;                               // bytes
    constexpr int KW = BLOCK / NWV > 512 / HD ? BLOCK / NWV : 512 / HD;                // positions a wave fetches
    constexpr int PIECES = KW * HD * 2 / 1024;
    const int tid = threadIdx.x, lane = tid & 63, h2 = lane >> 5, qi = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = blockIdx.x % a.G, split = blockIdx.y;
    const int tile = gridDim.x / a.G - 1 - blockIdx.x / a.G;   // later rows see more keys: they start first

    // ---- whose tile this is: request b owns the tiles from floor(q_start[b] rep / ROWS) + b on
    int b = 0;
    for (int n = a.batch; n > 1;) {
        const int stride = (n + 63) / 64, at = lane * stride;
        const bool before = at < n && (int64_t)min(max(a.q_start[b + min(at, n - 1)], 0), a.n_tokens) * a.rep / ROWS + b + at <= tile;
        const int k = max(__popcll(__ballot(before)) - 1, 0);
        b = __builtin_amdgcn_readfirstlane(b + k * stride);
        n = __builtin_amdgcn_readfirstlane(min(stride, n - k * stride));
    }
    const PagedRequest rq = paged_request(a, b);
    const int R = rq.n_new * a.rep;
    const int64_t first = (int64_t)rq.row0 * a.rep / ROWS + b;
    if (tile < first || (tile - first) * ROWS >= R || R <= a.row_limit) return;
    const int rho0 = (int)(tile - first) * ROWS;
    const PagedSteps st = paged_steps(rq, rq.pos0 + rho0 / a.rep, rq.pos0 + (min(rho0 + ROWS, R) - 1) / a.rep, a.window, BLOCK);
    const int s_begin = split * a.split_steps, s_end = split == a.n_splits - 1 ? st.total : min(st.total, s_begin + a.split_steps);
    const int32_t *table = a.block_table + (int64_t)b * a.max_pages;

    // ---- this wave's rows
    const int wrow = rho0 + 32 * wave;
    const bool busy = wrow < R;
    const int rho = min(wrow + qi, R - 1), tok = rho / a.rep, head = g * a.rep + rho % a.rep;
    const int pos = rq.pos0 + tok, pos_min = rq.pos0 + min(wrow, R - 1) / a.rep, pos_max = rq.pos0 + min(wrow + 31, R - 1) / a.rep;
    const int lo = a.window ? pos - a.window : -1;   // keys at or below it lie outside the window
    const float slope = MODS && a.slopes ? a.slopes[head] : 0.f;
    paged_u4 q[QT];   // lane: features 16 t + 8 h2 .. + 7 of its row
    {
        const bf16_t *src = (const bf16_t *)a.q + (int64_t)(rq.row0 + tok) * a.q_stride + (int64_t)head * HD + 8 * h2;
#pragma unroll
        for (int t = 0; t < QT; ++t) q[t] = *reinterpret_cast<const paged_u4 *>(src + 16 * t);
    }

    // ---- holes in the part of the table that this workgroup reads: then every block is looked at
    const auto real = [&](int v) { return v < st.n_pre ? v : v + st.skip; };
    bool hole = false;
    if (s_begin < s_end) {
        const int p0 = (real(s_begin) * BLOCK) >> a.page_shift, p1 = (min((real(s_end - 1) + 1) * BLOCK, rq.n_keys) - 1) >> a.page_shift;
        for (int p = p0 + tid; p <= p1; p += 64 * NWV) hole |= (unsigned)table[p] >= (unsigned)a.n_pages;
    }
    hole = __syncthreads_or(hole);

    // ---- fetching: this wave's positions of a block
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)lds;
    constexpr int SWZ_SHIFT = CPR == 4 ? 2 : CPR == 8 ? 1 : 0, SWZ_MASK = CPR == 32 ? 15 : CPR - 1;
    uint32_t koff[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int r = i * (512 / HD) + lane / CPR, row = wave * KW + r;
        koff[i] = r * HD * 2 + ((lane % CPR) ^ ((row >> SWZ_SHIFT) & SWZ_MASK)) * 16;
    }
    const auto page_of = [&](int step) {   // page number and offset of this wave's positions (elements)
        const int key = step * BLOCK + wave * KW;
        const int id = table[min(key >> a.page_shift, a.max_pages - 1)];
        return (int64_t)((unsigned)id < (unsigned)a.n_pages ? id : 0) * a.page_stride + (((int64_t)g << a.page_shift) + (key & ((1 << a.page_shift) - 1))) * HD;
    };
    const auto fetch = [&](int64_t at, int buf) {
        if (KW * NWV > BLOCK && wave * KW >= BLOCK) return;
        const bf16_t *kb = (const bf16_t *)a.k_pages + at, *vb = (const bf16_t *)a.v_pages + at;
        const uint32_t dst = lds0 + buf * BUF + wave * KW * HD * 2;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) page_to_lds(dst + i * 1024, koff[i], kb);
#pragma unroll
        for (int i = 0; i < PIECES; ++i) page_to_lds(dst + HALF + i * 1024, i * 1024 + lane * 16, vb);
    };

    // ---- reading: K rows with bits 2 and 3 swapped, chunk 2 t + h2; V groups 2 kc + h2
    const int krow = (qi & ~12) | ((qi & 4) << 1) | ((qi & 8) >> 1);
    uint32_t kaddr[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) kaddr[t] = krow * HD * 2 + (((2 * t + h2) ^ ((krow >> SWZ_SHIFT) & SWZ_MASK)) * 16);
    const uint32_t vaddr = HALF + (h2 * HD + qi) * 16;

    const auto see_all = [&](int key0) {   // every row of the wave sees every key of the block
        return !hole && key0 + BLOCK <= rq.n_keys &&
               (key0 + BLOCK <= rq.prefix || (key0 + BLOCK - 1 <= pos_min && (!a.window || key0 > pos_max - a.window)));
    };
    uint32_t odd = 0;   // bits of values that are not finite, of blocks that not every row sees
    float m_ref = -INFINITY, l_run = 0.f;
    paged_f16 o[OT];
#pragma unroll
    for (int dt = 0; dt < OT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
    const float c = a.scale * 1.4426950408889634f;   // scores in units of ln 2

    int64_t next_at = 0;
    if (s_begin < s_end) {
        fetch(page_of(real(s_begin)), 0);
        next_at = page_of(real(min(s_begin + 1, s_end - 1)));
    }
    for (int s = s_begin; s < s_end; ++s) {
        const int buf = (s - s_begin) & 1;
        // this wave's part of block s has arrived, and so has everybody's; nobody reads the other buffer any more
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (s + 1 < s_end) {
            fetch(next_at, buf ^ 1);
            next_at = page_of(real(min(s + 2, s_end - 1)));
        }
        const int key0 = real(s) * BLOCK;
        const bool none = !busy || (key0 >= rq.prefix && (key0 > pos_max || (a.window && key0 + BLOCK - 1 <= pos_min - a.window)));
        if (none) continue;
        const bool whole = see_all(key0);
        const unsigned char *kb = lds + buf * BUF;
        paged_f16 x[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int r = 0; r < 16; ++r) x[i][r] = 0.f;
#pragma unroll
            for (int t = 0; t < QT; ++t) x[i] = mfma32(*reinterpret_cast<const paged_u4 *>(kb + kaddr[t] + i * 32 * HD * 2), q[t], x[i]);
        }
        // register r of tile i: key key0 + 32 i + 16 (r / 8) + 8 h2 + r % 8
        if (MODS) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    float v = x[i][r] * a.scale;
                    if (a.softcap > 0.f) v = a.softcap * paged_tanh_fast(v / a.softcap);
                    if (a.slopes) v = fmaf(slope, (float)(key0 + 32 * i + 16 * (r >> 3) + 8 * h2 + (r & 7) - pos), v);
                    x[i][r] = v * 1.4426950408889634f;
                }
        }
        uint32_t run_ok = 15;   // bit i: run i of sixteen keys is in a page
        if (!whole) {
            if (hole) {
                run_ok = 0;
                for (int i = 0; i < 4; ++i) {
                    const int key = key0 + 16 * i;
                    if (key < rq.n_keys && (unsigned)table[key >> a.page_shift] < (unsigned)a.n_pages) run_ok |= 1u << i;
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int run = 2 * i + (r >> 3), j = key0 + 16 * run + 8 * h2 + (r & 7);
                    x[i][r] = paged_sees(j, run_ok >> run & 1 ? rq.n_keys : 0, rq.prefix, pos, lo) ? x[i][r] : -INFINITY;
                }
        }
        float mx = x[0][0];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = fmaxf(mx, x[i][r]);
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        if (!MODS) mx *= c;
        if (__any(mx > m_ref + 8.f)) {
            const float m_new = fmaxf(m_ref, mx);
            const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_ref - m_new);
            m_ref = m_new;
            l_run *= alpha;
#pragma unroll
            for (int dt = 0; dt < OT; ++dt) o[dt] *= alpha;
        }
        const float sub = m_ref == -INFINITY ? 0.f : m_ref;   // a row that has seen no key yet
        float sum[2] = {0.f, 0.f};
        paged_u4 p[4];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int r = 0; r < 16; r += 2) {
                const float e0 = __builtin_amdgcn_exp2f(MODS ? x[i][r] - sub : fmaf(x[i][r], c, -sub));
                const float e1 = __builtin_amdgcn_exp2f(MODS ? x[i][r + 1] - sub : fmaf(x[i][r + 1], c, -sub));
                sum[0] += e0;
                sum[1] += e1;
                p[2 * i + (r >> 3)][(r & 7) >> 1] = f32x2_to_bf16x2(e0, e1);
            }
        l_run += sum[0] + sum[1];
        const unsigned char *vb = kb + vaddr;
        if (whole) {
#pragma unroll
            for (int kc = 0; kc < 4; ++kc)
#pragma unroll
                for (int dt = 0; dt < OT; ++dt) o[dt] = mfma32(*reinterpret_cast<const paged_u4 *>(vb + (2 * kc * HD + 32 * dt) * 16), p[kc], o[dt]);
            continue;
        }
        // values behind the end of the request, or of a page that is not there, may be anything: 0 x NaN would reach every row.
        // The same holds for values that only some rows see: those that are not finite are taken out here and added below.
#pragma unroll
        for (int kc = 0; kc < 4; ++kc) {
            const int n = run_ok >> kc & 1 ? rq.n_keys - (key0 + 16 * kc + 8 * h2) : 0;   // of this lane's eight keys
#pragma unroll
            for (int dt = 0; dt < OT; ++dt) {
                paged_u4 v = *reinterpret_cast<const paged_u4 *>(vb + (2 * kc * HD + 32 * dt) * 16);
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    v[w] &= (2 * w < n ? 0xffffu : 0u) | (2 * w + 1 < n ? 0xffff0000u : 0u);
                    const uint32_t fine = finite_halves(v[w]);
                    odd |= v[w] & ~fine;
                    v[w] &= fine;
                }
                o[dt] = mfma32(v, p[kc], o[dt]);
            }
        }
    }

    if (__any(odd != 0)) {
        // rare: some value of a block that not every row sees is not finite.  Each row takes those that it sees, by their kind
#pragma unroll 1
        for (int s = s_begin; s < s_end; ++s) {
            const int key0 = real(s) * BLOCK;
            if (see_all(key0)) continue;
#pragma unroll 1
            for (int j = key0; j < min(key0 + BLOCK, rq.n_keys); ++j) {
                const int id = table[j >> a.page_shift], in = j & ((1 << a.page_shift) - 1);
                if ((unsigned)id >= (unsigned)a.n_pages || !paged_sees(j, rq.n_keys, rq.prefix, pos, lo)) continue;
                const bf16_t *v = (const bf16_t *)a.v_pages + (int64_t)id * a.page_stride + (((int64_t)g << a.page_shift) + (in & ~7)) * HD + (in & 7) + 32 * h2;
#pragma unroll
                for (int dt = 0; dt < OT; ++dt)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[dt][r] += only_not_finite(v[(32 * dt + 8 * (r >> 2) + (r & 3)) * 8]);
            }
        }
    }
    if (wrow + qi >= R) return;
    const float l = l_run + __shfl_xor(l_run, 32, 64);
    const int64_t row = rq.row0 + tok;
    if (a.n_splits == 1) {
        const float inv = l == 0.f ? 0.f : 1.f / l;   // a row that sees no key is 0
        bf16_t *dst = (bf16_t *)a.out + row * a.out_stride + (int64_t)head * HD + 4 * h2;
#pragma unroll
        for (int dt = 0; dt < OT; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<uint2 *>(dst + 32 * dt + 8 * i) = make_uint2(f32x2_to_bf16x2(o[dt][4 * i] * inv, o[dt][4 * i + 1] * inv),
                                                                                f32x2_to_bf16x2(o[dt][4 * i + 2] * inv, o[dt][4 * i + 3] * inv));
    } else {
        const int64_t at = ((int64_t)split * a.n_tokens + row) * a.H + head;
        if (l != 0.f) {   // (a part without keys is not read)
#pragma unroll
            for (int dt = 0; dt < OT; ++dt)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *reinterpret_cast<paged_f4 *>(a.po + at * HD + 32 * dt + 8 * i + 4 * h2) = paged_f4{o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]};
        }
        if (h2 == 0) {
            a.pm[at] = m_ref;
            a.pl[at] = l;
        }
    }
}

int paged_prompt_rows(int head_dim) { return 32 * prompt_waves(head_dim); }
int paged_prompt_tiles(const PagedAttn &a, int head_dim) { return (int)((int64_t)a.n_tokens * a.rep / paged_prompt_rows(head_dim)) + a.batch; }

template <int HD, bool MODS> static const char *launch_t(const PagedAttn &a, int device, hipStream_t stream) {
    static bool allowed[MAX_DEVICES];
    const size_t lds = prompt_lds(HD);
    if (lds > 60 * 1024 && !(device >= 0 && device < MAX_DEVICES && allowed[device])) {
        if (hipFuncSetAttribute(reinterpret_cast<const void *>(&k_paged_prompt<HD, MODS>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess) {
            (void)hipGetLastError();
            return "the device refuses the kernel's LDS request";
        }
        if (device >= 0 && device < MAX_DEVICES) allowed[device] = true;
    }
    hipLaunchKernelGGL((k_paged_prompt<HD, MODS>), dim3(paged_prompt_tiles(a, HD) * a.G, a.n_splits), dim3(64 * prompt_waves(HD)), lds, stream, a);
    return nullptr;
}
const char *launch_paged_prompt(const PagedAttn &a, int head_dim, int device, hipStream_t stream) {
    // (without cap and bias the scale is applied to the maximum, which only a positive one keeps a maximum)
    const bool mods = a.softcap > 0.f || a.slopes || a.scale < 0.f;
    switch (head_dim) {
        case 32: return mods ? launch_t<32, true>(a, device, stream) : launch_t<32, false>(a, device, stream);
        case 64: return mods ? launch_t<64, true>(a, device, stream) : launch_t<64, false>(a, device, stream);
        case 128: return mods ? launch_t<128, true>(a, device, stream) : launch_t<128, false>(a, device, stream);
        default: return mods ? launch_t<256, true>(a, device, stream) : launch_t<256, false>(a, device, stream);
    }
}

}  // namespace wisv
