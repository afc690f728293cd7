// Cross attention, backward in bf16: preparation, dQ, dK/dV, sums of parts.  Arithmetic, fragments and scaling of dO are the
// self-attention backward's (hyd_bwd_bf16.h), whose dQ tile body and wide dK/dV kernel (hyd_bwd_wide.h) run here.
//
// Everything that the two tile kernels hand on is kept by packed row (hyd_cross.h): statistics [Hkv][Tq G], fp16 copies of Q and dO
// [Hkv][Tq G][d].  dK/dV then streams one run of rows for all heads of a group, whatever their number.  Where there are too few
// items for the chip, they are taken in parts of the other side's tiles, whose fp32 sums are added in order and rounded once.
#pragma once
#include "hyd_bwd_wide.h"
#include "hyd_cross.h"
#include "hyd_find.h"

namespace hyd {

// ---------------------------------------------------------------------------------------------
// Preparation, one launch: workgroups 0 and 1 build the item lists, then zero.n of them clear dK and dV behind the valid keys of
// their sequences (padded caches), n_q make one pass over O and dO (row statistics, negated, and the maxima of |dO|), the others
// copy K to fp16.  Bound by HBM, or by latency on small batches: 24 sequences, 18000 keys and 5400 queries of 20 heads, d = 64, 131 MB, 25 us.
// ---------------------------------------------------------------------------------------------
struct CrossPrepParams {
    CrossShape c;
    const uint16_t* o; const uint16_t* d_o; const float* lse; const uint16_t* k;
    uint16_t* dk; uint16_t* dv;
    BwdScratch sc;
    int tok;                              // tokens of a statistics workgroup at a time
    CrossZero zero;
    int n_q;                              // workgroups of the pass over O and dO
    CrossList lists[2];
};
constexpr int kCrossLists = 2;
inline size_t cross_prep_lds(int hq, int tok) {
    const size_t st = sizeof(float) * 2 * (size_t)(hq < kPrepRows ? hq : kPrepRows) * tok + sizeof(int) * 32;
    return st > (size_t)kCrossListLds ? st : (size_t)kCrossListLds;
}

template <int D>
__global__ void __launch_bounds__(kPrepThreads) hyd_cross_prep_bf16_kernel(CrossPrepParams p) {
    extern __shared__ float st[];                  // [2][heads][tok]: -D, the row's largest |dO| as bits
    const int tid = threadIdx.x;
    int wg = blockIdx.x;
    if (wg < kCrossLists) {
        cross_build_list(p.c, p.lists[wg], reinterpret_cast<int*>(st), kPrepThreads);
        return;
    }
    wg -= kCrossLists;
    constexpr int kLanes = D / 8, kGrps = kPrepThreads / kLanes, kU = 4;      // lanes per row, rows at a time, in flight
    const int hq = p.c.hq, hkv = p.c.hkv, G = p.c.G, tok = p.tok;
    if (wg < p.zero.n) {
        cross_clear<u32x4, 8>(p.c, p.zero, wg, kPrepThreads, (int64_t)hkv * D, p.dk, p.dv);
        return;
    }
    wg -= p.zero.n;
    const int grp = tid / kLanes, c = tid % kLanes;
    if (wg >= p.n_q) {                             // fp16 copy of K, rows [cu_kv[0], cu_kv[nseq])
        const int64_t first = (int64_t)max(p.c.cu_kv[0], 0) * hkv, last = (int64_t)min(p.c.cu_kv[p.c.nseq], p.c.Tk) * hkv;
        const int64_t step = (int64_t)(gridDim.x - kCrossLists - p.zero.n - p.n_q) * kGrps * kU;
        for (int64_t r0 = first + (int64_t)(wg - p.n_q) * kGrps * kU + grp; r0 < last; r0 += step) {
            u32x4 x[kU];
#pragma unroll
            for (int u = 0; u < kU; ++u)
                if (r0 + kGrps * u < last) x[u] = *reinterpret_cast<const u32x4*>(p.k + (r0 + kGrps * u) * D + c * 8);
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                if (r0 + kGrps * u < last) {
                    u32x4 x16;
#pragma unroll
                    for (int e = 0; e < 4; ++e) x16[e] = bf16x2_to_f16x2(x[u][e]);
                    *reinterpret_cast<u32x4*>(p.sc.k16 + (r0 + kGrps * u) * D + c * 8) = x16;
                }
            }
        }
        return;
    }
    // Rows of sequences only: what lies outside may be anything, and would enter the maximum.  Rows without keys (LSE = -inf) have no
    // part in dK and dV, and none in the maximum either.
    const int T0 = max(p.c.cu_q[0], 0), T1 = min(p.c.cu_q[p.c.nseq], p.c.Tq);
    const int64_t packed = (int64_t)p.c.Tq * G;
    uint32_t gmax = 0;
    const int heads = min(hq, kPrepRows);          // of a block; of more heads than that, one token at a time (prep_tokens)
    for (int t0 = T0 + wg * tok; t0 < T1; t0 += p.n_q * tok) {
        const int nt = min(tok, T1 - t0);
        for (int h0 = 0; h0 < hq; h0 += heads) {
            const int nh = min(heads, hq - h0), n_rows = nt * nh;
            for (int r0 = grp; r0 < n_rows; r0 += kGrps * kU) {       // row r of the block = (token t0 + r / nh, head h0 + r % nh)
                u32x4 a[kU], b[kU];
#pragma unroll
                for (int u = 0; u < kU; ++u) {
                    const int r = r0 + kGrps * u;
                    a[u] = u32x4{0u, 0u, 0u, 0u};
                    b[u] = u32x4{0u, 0u, 0u, 0u};
                    if (r < n_rows) {
                        const int64_t at = ((int64_t)t0 * hq + h0 + r) * D + c * 8;
                        a[u] = *reinterpret_cast<const u32x4*>(p.o + at);
                        b[u] = *reinterpret_cast<const u32x4*>(p.d_o + at);
                    }
                }
#pragma unroll
                for (int u = 0; u < kU; ++u) {
                    float acc = 0.f;
                    uint32_t amax = 0;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        acc += bf16_lo(a[u][e]) * bf16_lo(b[u][e]) + bf16_hi(a[u][e]) * bf16_hi(b[u][e]);
                        amax = max(amax, max(b[u][e] & 0x7fffu, (b[u][e] >> 16) & 0x7fffu));
                    }
#pragma unroll
                    for (int m = 1; m < kLanes; m <<= 1) {
                        acc += __shfl_xor(acc, m, 64);
                        amax = max(amax, (uint32_t)__shfl_xor((int)amax, m, 64));
                    }
                    const int r = r0 + kGrps * u;
                    if (c == 0 && r < n_rows) {
                        const int tl = r / nh, h = r - tl * nh;
                        st[h * tok + tl] = -acc;
                        st[(heads + h) * tok + tl] = __uint_as_float(amax);
                    }
                }
            }
            __syncthreads();
            for (int idx = tid; idx < n_rows; idx += kPrepThreads) {  // by packed row
                const int x = h0 + idx, g = x / (nt * G), i = x - g * nt * G, tl = i / G, h = g * G + i - tl * G;
                const int64_t at = g * packed + (int64_t)t0 * G + i;
                const uint32_t amax = __float_as_uint(st[(heads + h - h0) * tok + tl]);
                const float lse = p.lse[(int64_t)h * p.c.Tq + t0 + tl];
                p.sc.Dq[at] = st[(h - h0) * tok + tl];
                p.sc.kqmul[at] = pow2i(-shift_of(amax));
                p.sc.lse2[at] = -lse * kLog2e;
                if (lse != -INFINITY) gmax = max(gmax, amax);
            }
            __syncthreads();
        }
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) gmax = max(gmax, (uint32_t)__shfl_xor((int)gmax, m, 64));
    uint32_t* wmax = reinterpret_cast<uint32_t*>(st);
    if ((tid & 63) == 0) wmax[tid >> 6] = gmax;
    __syncthreads();
    if (tid == 0) p.sc.absmax[wg] = max(max(wmax[0], wmax[1]), max(wmax[2], wmax[3]));
    if (wg == p.n_q - 1 && tid > 0 && tid < 4 && (wg + tid) / 4 == wg / 4) p.sc.absmax[wg + tid] = 0;
}

// ---------------------------------------------------------------------------------------------
// dQ.  Work item = (256 packed rows of a sequence and KV head, a part of its keys); see hyd_bwd_bf16.h's dQ for the products and the
// scaling.  The first part also writes what dK/dV streams: the fp16 copies of Q and of dO * 2^kg, and -D * 2^kg, by packed row.
// 4 sequences of 1500 to 6000 queries and 4000 to 12000 keys, 32/8 heads, d = 128: 2.5 ms, 1.23 PFLOP/s in its three products (dK/dV 3.15 ms,
// 1.3 in four), the matrix pipe busy for 69 % of the clocks (72).  Short items wait: 24 sequences of up to 448 queries and 1500 keys, 20 heads, d = 64,
// 79 us at 24 % of the pipe, 41 % of the vector ALU and 2.7 TB/s (dK/dV 119 us, 22, 29 %, 2.5).  P and dS are fp16 numbers here, 2^-11 of
// themselves, an eighth of the results' own rounding.  Items of 128 rows, two workgroups to a CU, gained 20 % with 64 queries
// of a sequence and lost 5 % with 256 or 448 (d = 64, 1536 keys), so there is one form.
// ---------------------------------------------------------------------------------------------
struct CrossDqParams {
    CrossShape c;
    const uint16_t* q; const uint16_t* v; const uint16_t* d_o;
    BwdScratch sc;
    uint16_t* dq;
    float* part;                          // parts > 1: [parts][Tq][Hq][d]
    int parts;
    float scale, scale_log2;
};

template <int D>
__global__ void __launch_bounds__(kDqThreads, 1) hyd_cross_dq_bf16_kernel(CrossDqParams p, WorkList list) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    constexpr int kRowB = D * 2;
    int* slot = reinterpret_cast<int*>(smem + kDqQxOff);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, half = lane >> 5;
    const int G = p.c.G;
    const int64_t q_stride = (int64_t)p.c.hq * D, kv_stride = (int64_t)p.c.hkv * D, packed = (int64_t)p.c.Tq * G;
    const uint32_t kv_stride_b = (uint32_t)kv_stride * 2, q_stride_b = (uint32_t)q_stride * 2;
    FragAddr fa;
    fa.init(lane, smem);
    CrossRows cr;
    cr.init(G);
    const uint32_t dma_voff = dma_lane_voff<D>(4 * wave + (lane >> 4), lane, kv_stride_b);
    const uint32_t tile_bytes = kDqBN * kv_stride_b;
    const int row_stage = wave * 32 * kRowBytes;
    const uint32_t o_stage = (uint32_t)(uintptr_t)(lds_char*)smem + (uint32_t)row_stage;
    const float scale_log2 = fmaxf(fabsf(p.scale_log2), 1e-30f);
    const uint32_t sign_flip = p.scale_log2 < 0.f ? 0x80008000u : 0u;
    PartialMaxima pm;
    pm.load(p.sc, lane);

    WorkFetcher wf;
    WorkItem wi;
    bool have = wf.first(list.hm, list.hdr, list.cursors, list.items, slot, wi, blockIdx.x);
    const float up = pow2i(pm.shift());                               // 2^kg
    while (have) {
        __syncthreads();                                  // everybody has read the work slot: its bytes may be overwritten
        const int g = wi.head, R = wi.seq, rows = wi.lev & ((1 << kCrossPartShift) - 1), part = wi.lev >> kCrossPartShift, n = wi.len;
        const int t0 = R / G, rem = R - t0 * G;
        const int n_all = (n + kDqBN - 1) / kDqBN, per_part = (n_all + p.parts - 1) / p.parts;
        const int t_lo = min(part * per_part, n_all), n_kt = min(t_lo + per_part, n_all);      // key tiles (the first part has some if there are any)
        const int wrow0 = 32 * wave, row = wrow0 + l32;
        const bool active = wrow0 < rows, valid = row < rows;
        const auto q_at = [&](int r) -> int64_t {         // element offset of row r of the tile in Q, dO and dQ
            asm volatile("" : "+v"(r));                   // (formed where it is asked for)
            int token, head;
            cr.split(rem + r, token, head);
            return (int64_t)(t0 + token) * q_stride + (int64_t)(g * G + head) * D;
        };
        if (t_lo == n_kt) {                               // no keys: dQ = 0
            if (valid) {
                const int64_t at = q_at(row) + 4 * half;
#pragma unroll
                for (int i = 0; i < D / 8; ++i) {
                    if (p.parts == 1) *reinterpret_cast<u32x2*>(p.dq + at + 8 * i) = u32x2{0u, 0u};
                    else *reinterpret_cast<f32x4*>(p.part + part * packed * kv_stride + at + 8 * i) = f32x4{0.f, 0.f, 0.f, 0.f};
                }
            }
            have = wf.next(list.hm, list.cursors, list.items, slot, wi);
            continue;
        }
        const uint32_t kv_bytes = (uint32_t)(min(n, n_kt * kDqBN) - 1) * kv_stride_b + kRowB;
        const __amdgpu_buffer_rsrc_t rk = make_rsrc(p.sc.k16 + (int64_t)wi.row0 * kv_stride + (int64_t)g * D, kv_bytes);
        const __amdgpu_buffer_rsrc_t rv = make_rsrc(p.v + (int64_t)wi.row0 * kv_stride + (int64_t)g * D, kv_bytes);
        auto dma_tile = [&](int t, int stage) {
            char* dst = smem + stage * kDqStageBytes + 4 * wave * kRowBytes;
#pragma unroll
            for (int j = 0; j < 16 / kDqWaves; ++j) {
                const uint32_t soff = (uint32_t)t * tile_bytes + (uint32_t)(j * kDqWaves * 4) * kv_stride_b;
                char* d = dst + j * kDqWaves * 4 * kRowBytes;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rk, (lds_void_b*)d, 16, dma_voff, soff, 0, 0);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rv, (lds_void_b*)(d + kDqTileBytes), 16, dma_voff, soff, 0, 0);
            }
        };
        const bool short_item = n_kt - t_lo <= kShortItem;
        if (short_item) wf.claim(list.hm, list.cursors);
        dma_tile(t_lo, 0);
        {
            const uint32_t q_bytes = (uint32_t)((rem + rows - 1) / G) * q_stride_b + (uint32_t)G * kRowB;
            const int64_t off = (int64_t)t0 * q_stride + (int64_t)g * G * D;
            dma_packed_rows<kDqWaves, D>(make_rsrc(p.q + off, q_bytes), smem + kDqQxOff, [](int j) { return j * kDqTileBytes; },
                                         (rows + 63) / 64, cr, rem, rows, q_stride_b, wave, lane);
            dma_packed_rows<kDqWaves, D>(make_rsrc(p.d_o + off, q_bytes), smem + kDqStageBytes, [](int j) { return j * kDqTileBytes; },
                                         (rows + 63) / 64, cr, rem, rows, q_stride_b, wave, lane);
        }
        float lse2 = 0.f, Dq = 0.f, unshift = 1.f;
        if (valid) {
            const int64_t at = g * packed + R + row;
            lse2 = p.sc.lse2[at];
            Dq = p.sc.Dq[at];
            unshift = p.sc.kqmul[at];
            if (part == 0 && half == 0) p.sc.Dkv[at] = Dq * up;
        }
        // 2^kq, the exact reciprocal of the power of two 2^-kq; rows past the tile keep 1
        const auto reciprocal = [](float x) { return __uint_as_float((254u << 23) - __float_as_uint(x)); };
        const float shift = reciprocal(unshift);
        Dq *= shift;
        f32x16 acc[D / 32];
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[db][r] = 0.f;
        __syncthreads();                                  // tile t_lo and the Q / dO rows have landed
        bf16x8 qf[D / 16], dof[D / 16];
        {
            u32x4 a[D / 16], b[D / 16];
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                a[ks] = *(lds_u32x4*)(uintptr_t)(fa.row[ks] + (uint32_t)(kDqQxOff + row_stage));
                b[ks] = *(lds_u32x4*)(uintptr_t)(fa.row[ks] + (uint32_t)(kDqStageBytes + row_stage));
            }
            __builtin_amdgcn_s_waitcnt(0xc07f);           // lgkmcnt(0)
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                asm volatile("" : "+v"(a[ks]), "+v"(b[ks]));      // the reads stay on this side of the barrier
#pragma unroll
                for (int e = 0; e < 4; ++e) a[ks][e] = bf16x2_to_f16x2(a[ks][e]);
            }
            if (part == 0) {
                // each wave puts its 32 rows back where it took them from and sends them out in whole rows
                typedef __attribute__((address_space(3))) u32x4 lds_u32x4_w;
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    u32x4 s16;
#pragma unroll
                    for (int e = 0; e < 4; ++e) s16[e] = bf16x2_to_f16x2(b[ks][e], up);
                    *(lds_u32x4_w*)(uintptr_t)(fa.row[ks] + (uint32_t)(kDqQxOff + row_stage)) = a[ks];
                    *(lds_u32x4_w*)(uintptr_t)(fa.row[ks] + (uint32_t)(kDqStageBytes + row_stage)) = s16;
                }
                int ln = lane;
                asm volatile("" : "+v"(ln));              // (these addresses are formed here)
                const int r4 = ln >> 4, ch = ln & 15;
                const uint32_t wbase = (uint32_t)(uintptr_t)(lds_char*)smem + (uint32_t)(row_stage + r4 * kRowBytes);
                const int64_t goff = (g * packed + R + wrow0 + r4) * D + ch * 8;
#pragma unroll
                for (int which = 0; which < 2; ++which) {
                    uint16_t* dst = (which ? p.sc.do16 : p.sc.q16) + goff;
                    u32x4 x[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i)           // row r4 + 4 i of the wave: swz = (r4 << 2) | (i & 3)
                        x[i] = *(lds_u32x4*)(uintptr_t)(wbase + (uint32_t)((which ? kDqStageBytes : kDqQxOff) + 4 * i * kRowBytes + ((ch ^ ((r4 << 2) | (i & 3))) << 4)));
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (wrow0 + r4 + 4 * i < rows && (D == kHeadDim || ch < D / 8)) *reinterpret_cast<u32x4*>(dst + 4 * i * D) = x[i];
                }
            }
            __builtin_amdgcn_s_waitcnt(0xc07f);           // lgkmcnt(0): the staging areas have been read
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                qf[ks] = as_bf16x8(a[ks] ^ sign_flip);
                // the row's dO times 2^kq (exact: a power of two, and the row's largest element lands in [1, 2))
#pragma unroll
                for (int e = 0; e < 4; ++e) b[ks][e] = pack_bf16(bf16_lo(b[ks][e]) * shift, bf16_hi(b[ks][e]) * shift);
                dof[ks] = as_bf16x8(b[ks]);
            }
        }
        __builtin_amdgcn_s_barrier();                     // stages 1 and 2 may take K/V tiles now
        if (t_lo + 1 < n_kt) dma_tile(t_lo + 1, 1);

        auto step = [&](auto stage_tag, int t) {
            constexpr int ST = decltype(stage_tag)::value;
            constexpr int Kt = ST * kDqStageBytes, Vt = Kt + kDqTileBytes, ST2 = (ST + 2) % kDqStages;
            constexpr int kDmaPerTile = 2 * (16 / kDqWaves);
            const bool more2 = t + 2 < n_kt;
            if (more2) dma_tile(t + 2, ST2);
            if (active) {
                // keys behind the last one: hidden (the tile's zeros would be keys of score 0), and a block of them is skipped
                const int left = n - t * kDqBN, krel = 4 * half - (left - 1);
                dq_block<D>(Kt, Vt, fa, 0, qf, dof, acc, scale_log2, lse2, Dq, left < 32, krel);
                if (left > 32) dq_block<D>(Kt, Vt, fa, 1, qf, dof, acc, scale_log2, lse2, Dq, left < 64, krel + 32);
            }
            if (more2) __builtin_amdgcn_s_waitcnt(0x0070 | (kDmaPerTile & 15));     // vmcnt(kDmaPerTile), lgkmcnt(0)
            else __builtin_amdgcn_s_waitcnt(0x0070);                                // vmcnt(0), lgkmcnt(0)
            __builtin_amdgcn_s_barrier();
        };
        for (int t = t_lo; t < n_kt; t += 3) {
            step(std::integral_constant<int, 0>{}, t);
            if (t + 1 < n_kt) step(std::integral_constant<int, 1>{}, t + 1);
            if (t + 2 < n_kt) step(std::integral_constant<int, 2>{}, t + 2);
        }
        if (!short_item) wf.claim(list.hm, list.cursors);
        if (active) {
            const float mul = p.scale * reciprocal(shift);
            if (p.parts == 1) {
                store_packed_rows<D>([&](int r) { return p.dq + q_at(wrow0 + r); }, rows - wrow0, acc, mul, o_stage, lane);
            } else if (valid) {
                float* at = p.part + part * packed * kv_stride + q_at(row);
#pragma unroll
                for (int db = 0; db < D / 32; ++db)
#pragma unroll
                    for (int rq = 0; rq < 4; ++rq) {
                        *reinterpret_cast<f32x4*>(at + 32 * db + 8 * rq + 4 * half) =
                            f32x4{acc[db][4 * rq] * mul, acc[db][4 * rq + 1] * mul, acc[db][4 * rq + 2] * mul, acc[db][4 * rq + 3] * mul};
                    }
            }
        }
        have = wf.next(list.hm, list.cursors, list.items, slot, wi);
    }
}

// ---------------------------------------------------------------------------------------------
// Sums of parts: planes of fp32 [rows][heads][d] added in order and rounded once, for the rows of sequences; of keys, with kv_lens,
// for the valid ones only.  16 bytes of a plane per lane; bound by HBM.
// ---------------------------------------------------------------------------------------------
constexpr int kCrossSumThreads = 256;
struct CrossSum {
    const float* part; void* out[2];              // [outputs][parts] planes
    const int32_t* cu; const int32_t* lens;       // lens: NULL, or valid rows of a sequence
    int nseq, T, heads, parts;
};
template <int D, bool kF32>
__global__ void __launch_bounds__(kCrossSumThreads) hyd_cross_sum_kernel(CrossSum p) {
    const int t = blockIdx.x;
    if (t < p.cu[0] || t >= p.cu[p.nseq]) return;
    if (p.lens) {
        int s, first, end;
        if (!find_sequence(p.cu, p.nseq, t, s, first, end) || t - first >= p.lens[s]) return;
    }
    const int64_t row = (int64_t)p.heads * D, plane = (int64_t)p.T * row;
    for (int i = 4 * threadIdx.x; i < p.heads * D; i += 4 * kCrossSumThreads) {
        const float* src = p.part + blockIdx.y * (int64_t)p.parts * plane + t * row + i;
        f32x4 sum = *reinterpret_cast<const f32x4*>(src);
        for (int x = 1; x < p.parts; ++x) sum += *reinterpret_cast<const f32x4*>(src + x * plane);
        if (kF32) *reinterpret_cast<f32x4*>(static_cast<float*>(p.out[blockIdx.y]) + t * row + i) = sum;
        else *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(p.out[blockIdx.y]) + t * row + i) = u32x2{pack_bf16(sum[0], sum[1]), pack_bf16(sum[2], sum[3])};
    }
}

}  // namespace hyd
