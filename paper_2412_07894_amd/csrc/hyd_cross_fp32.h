// Cross attention in fp32 on v_mfma_f32_32x32x2_f32: forward, dQ, dK/dV.  Split of an item, LDS tiles and products are those of hyd_fp32.h; what
// differs is which rows an item holds (hyd_cross.h: packed rows of a KV head's query heads) and that nothing is masked but the
// keys behind a sequence's last one.  Hidden rows are zeros in every tile, so that 0 * x never meets a value that is not finite.
// Bound by the matrix pipe: 8 sequences of 1000 queries and 1000 keys, 16/4 heads, d = 128: dQ 0.95 ms, 103 TFLOP/s in its three products, dK/dV
// 1.39 ms, 94 in four, forward 0.68 ms, 96 in two, of 4000 queries and keys 9.6 ms, 109 (a large fp32 matrix product reaches 153); the tile that
// a product waits for is what is left.  Small batches wait for
// their longest items: parts of them cost in fetches and sums what they save in balance, so they are taken only where there are
// fewer items than CUs (7 sequences of up to 500 queries and 900 keys, 8/2 heads, d = 128: 257 us whole, 242 in parts of a few steps each;
// with all sequences alike 255 and 310 us).
#pragma once
#include "hyd_cross.h"
#include "hyd_fp32.h"

namespace hyd {

struct CrossF32Params {
    CrossShape c;
    const float* q; const float* k; const float* v; const float* o; const float* d_o; const float* lse_in;
    float* o_out; float* lse_out;
    float* dq; float* dk; float* dv;
    float* D;                             // [Hq][Tq], written by dQ, read by dK/dV
    float scale;
    const int* hdr; int* cursors; const int* items;
    HeadMap hm;
    int parts, tiles;                     // parts of an item; forward, own items: tiles of a sequence at most
    float* part_o; float* part_lse;       // forward: see CrossJoin; backward: part_o holds the planes that are summed
};

// Item lists of the backward (workgroups 0 and 1), zeros in dK and dV behind the valid keys (the others).
struct CrossF32Begin { CrossShape c; CrossList lists[2]; CrossZero zero; float* dk; float* dv; int d; };
__global__ void __launch_bounds__(kPreludeThreads) hyd_cross_begin_fp32_kernel(CrossF32Begin p) {
    extern __shared__ int lds_classes[];
    if (blockIdx.x < 2) {
        cross_build_list(p.c, p.lists[blockIdx.x], lds_classes, kPreludeThreads);
        return;
    }
    cross_clear<f32x4, 4>(p.c, p.zero, (int)blockIdx.x - 2, kPreludeThreads, (int64_t)p.c.hkv * p.d, p.dk, p.dv);
}

// LDS reads of this wave done (before a barrier after which the tile may be overwritten)
__device__ __forceinline__ void f32_wait_lds() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);
    asm volatile("" ::: "memory");
}

// Where the packed rows of an item lie in the caller's tensors.
struct CrossF32Rows {
    CrossRows cr;
    int t0, rem, head0, Tq;
    int64_t stride;
    int d;
    __device__ __forceinline__ CrossF32Rows(const CrossShape& c, int R, int g, int D) {
        cr.init(c.G);
        t0 = R / c.G; rem = R - t0 * c.G; head0 = g * c.G; Tq = c.Tq; stride = (int64_t)c.hq * D; d = D;
    }
    __device__ __forceinline__ int64_t at(int r) const {              // element of Q, O, dO, dQ
        int token, head;
        cr.split(rem + r, token, head);
        return (t0 + token) * stride + (int64_t)(head0 + head) * d;
    }
    __device__ __forceinline__ int64_t stat(int r) const {            // element of LSE and D
        int token, head;
        cr.split(rem + r, token, head);
        return (int64_t)(head0 + head) * Tq + t0 + token;
    }
};

template <int D, bool kSelf>
__global__ void __launch_bounds__(64 * kF32Waves, 1) hyd_cross_fwd_fp32_kernel(CrossF32Params p) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    constexpr int kT = f32_tile_bytes<D>(), NDB = D / 32, kL = F32Lds<D, kF32Waves>::kLoads;
    constexpr int kAcc = NDB * 64 * 64;                          // bytes of a wave's accumulators
    int* slot = reinterpret_cast<int*>(smem + 2 * kT);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rg = wave & 1, split = wave >> 1, l32 = lane & 31, half = lane >> 5;
    const uint32_t stride_b = (uint32_t)p.c.hkv * D * 4;
    F32Lds<D, kF32Waves> fl;
    fl.init(lane, wave, split, smem, stride_b);
    WorkFetcher wf;
    WorkItem wi;
    auto claim = [&]() { if (!kSelf) wf.claim(p.hm, p.cursors); };
    bool have;
    if constexpr (kSelf) {
        int b = blockIdx.x;
        wi.head = b % p.c.hkv; b /= p.c.hkv;
        const int part = b % p.parts; b /= p.parts;
        const int tile = b % p.tiles;
        const CrossSeq x = cross_seq(p.c, b / p.tiles);
        const int left = x.lq * p.c.G - tile * kF32BM;
        wi.seq = x.q0 * p.c.G + tile * kF32BM; wi.lev = min(left, kF32BM) | (part << kCrossPartShift); wi.row0 = x.k0; wi.len = x.n;
        have = left > 0;
    } else {
        have = wf.first(p.hm, p.hdr, p.cursors, p.items, slot, wi, blockIdx.x);
    }
    for (; have; have = kSelf ? false : wf.next(p.hm, p.cursors, p.items, slot, wi)) {
        const int g = wi.head, rows = wi.lev & ((1 << kCrossPartShift) - 1), part = wi.lev >> kCrossPartShift, n = wi.len;
        const CrossF32Rows at(p.c, wi.seq, g, D);
        const int wrow0 = 32 * rg, i = wrow0 + l32;
        const int n_all = (n + kF32Tile - 1) / kF32Tile;
        const int t_lo = (int)((long long)n_all * part / p.parts), n_kt = (int)((long long)n_all * (part + 1) / p.parts);
        const int64_t plane = (int64_t)part * p.c.hq * p.c.Tq;
        float* const o_out = p.parts > 1 ? p.part_o + plane * D : p.o_out;
        float* const lse_out = p.parts > 1 ? p.part_lse + plane : p.lse_out;
        const float ln2 = p.parts > 1 ? 1.44269504088896340736f : 1.f;        // (the join takes sums in base 2)
        if (t_lo == n_kt) {                                      // no keys: O = 0, LSE = -inf
            claim();
            if (split == 0 && i < rows) {
                f32x16 z[NDB];
                f32_zero(z);
                f32_store_row<D>(o_out + at.at(i), z, 0.f, half);
                if (half == 0) lse_out[at.stat(i)] = -INFINITY;
            }
            continue;
        }
        const uint32_t kv_bytes = (uint32_t)(n - 1) * stride_b + D * 4;
        const __amdgpu_buffer_rsrc_t rk = make_rsrc(p.k + ((int64_t)wi.row0 * p.c.hkv + g) * D, kv_bytes);
        const __amdgpu_buffer_rsrc_t rv = make_rsrc(p.v + ((int64_t)wi.row0 * p.c.hkv + g) * D, kv_bytes);
        fl.load(rk, smem, (uint32_t)t_lo * kF32Tile * stride_b, stride_b);
        f32x4 q[D / 8];
        f32_load_row<D>(q, p.q + at.at(min(i, rows - 1)), half);
        fl.load(rv, smem + kT, (uint32_t)t_lo * kF32Tile * stride_b, stride_b);
        f32x16 o[NDB];
        f32_zero(o);
        float m = -INFINITY, l = 0.f;
        for (int t = t_lo; t < n_kt; ++t) {
            const uint32_t nxt = (uint32_t)(t + 1) * kF32Tile * stride_b;
            const bool more = t + 1 < n_kt;
            if (t == max(n_kt - 2, t_lo)) claim();
            const int key0 = t * kF32Tile + 32 * split;
            const bool work = key0 < n && wrow0 < rows;
            f32_arrive<kL>();                                    // K tile t is there
            f32x16 s[1];
            f32_zero(s);
            if (work) f32_row_product(s[0], fl, 0, q);
            f32_release();
            if (more) fl.load(rk, smem, nxt, stride_b);
            if (work) {
                const int rel = n - 1 - key0 - 4 * half;         // register r is visible iff its key offset <= rel
#pragma unroll
                for (int r = 0; r < 16; ++r) s[0][r] *= p.scale;
                if (key0 + 32 > n) {
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (8 * (r >> 2) + (r & 3) > rel) s[0][r] = -INFINITY;
                }
                float mx = s[0][0];
#pragma unroll
                for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[0][r]);
                float lo, hi;
                both_halves(mx, lo, hi);
                const float m_new = fmaxf(m, fmaxf(lo, hi));
                const float ref = m_new == -INFINITY ? 0.f : m_new;
                const float alpha = f32_exp(m - ref);
                m = m_new;
                float sum = 0.f;
#pragma unroll
                for (int r = 0; r < 16; ++r) { s[0][r] = f32_exp(s[0][r] - ref); sum += s[0][r]; }
                l = l * alpha + sum;
                if (__any(alpha != 1.f)) {
#pragma unroll
                    for (int db = 0; db < NDB; ++db)
#pragma unroll
                        for (int r = 0; r < 16; ++r) o[db][r] *= alpha;
                }
            }
            if (more) f32_arrive<kL>(); else f32_arrive<0>();    // V tile t is there
            if (work) f32_col_product(o, fl, kT, s[0]);
            f32_release();
            if (more) fl.load(rv, smem + kT, nxt, stride_b);
        }
        {   // l is still split over the two halves of the wave
            float lo, hi;
            both_halves(l, lo, hi);
            l = lo + hi;
        }
        // The splits' results meet in LDS, as in hyd_fp32.h.
        float* ml = reinterpret_cast<float*>(smem + 2 * kT - kAcc);
        if (split) f32_put(smem + (2 * (split - 1) + rg) * kAcc, o, lane);
        ml[wave * 128 + lane] = m;
        ml[wave * 128 + 64 + lane] = l;
        __syncthreads();
        if (split == 0 && wrow0 < rows) {
            float mt = m, lt = 0.f;                              // (a split that saw no key has m = -inf and l = 0)
#pragma unroll
            for (int x = 1; x < kF32Splits; ++x) mt = fmaxf(mt, ml[(2 * x + rg) * 128 + lane]);
            float w = f32_exp(m - mt);
            lt = l * w;
#pragma unroll
            for (int x = 1; x < kF32Splits; ++x) {
                const float wx = f32_exp(ml[(2 * x + rg) * 128 + lane] - mt);
                lt += ml[(2 * x + rg) * 128 + 64 + lane] * wx;
                f32_add(o, w, smem + (2 * (x - 1) + rg) * kAcc, wx, lane);
                w = 1.f;
            }
            if (i < rows) {
                f32_store_row<D>(o_out + at.at(i), o, 1.f / lt, half);
                if (half == 0) lse_out[at.stat(i)] = (mt + logf(lt)) * ln2;
            }
        }
        if (kSelf) break;
    }
}

template <int D>
__global__ void __launch_bounds__(64 * kF32Waves, 1) hyd_cross_dq_fp32_kernel(CrossF32Params p) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    constexpr int kT = f32_tile_bytes<D>(), NDB = D / 32, kL = F32Lds<D, kF32Waves>::kLoads;
    constexpr int kAcc = NDB * 64 * 64;
    int* slot = reinterpret_cast<int*>(smem + 2 * kT);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rg = wave & 1, split = wave >> 1, l32 = lane & 31, half = lane >> 5;
    const uint32_t stride_b = (uint32_t)p.c.hkv * D * 4;
    F32Lds<D, kF32Waves> fl;
    fl.init(lane, wave, split, smem, stride_b);
    WorkFetcher wf;
    WorkItem wi;
    for (bool have = wf.first(p.hm, p.hdr, p.cursors, p.items, slot, wi, blockIdx.x); have; have = wf.next(p.hm, p.cursors, p.items, slot, wi)) {
        const int g = wi.head, rows = wi.lev & ((1 << kCrossPartShift) - 1), part = wi.lev >> kCrossPartShift, n = wi.len;
        const CrossF32Rows at(p.c, wi.seq, g, D);
        const int wrow0 = 32 * rg, i = wrow0 + l32;
        const int n_all = (n + kF32Tile - 1) / kF32Tile, per_part = (n_all + p.parts - 1) / p.parts;
        const int t_lo = min(part * per_part, n_all), n_kt = min(t_lo + per_part, n_all);      // (the first part has tiles if there are any)
        float* const out = p.parts > 1 ? p.part_o + (int64_t)part * p.c.Tq * p.c.hq * D : p.dq;
        if (t_lo == n_kt) {
            wf.claim(p.hm, p.cursors);
            if (split == 0 && i < rows) {
                f32x16 z[NDB];
                f32_zero(z);
                f32_store_row<D>(out + at.at(i), z, 0.f, half);
            }
            continue;
        }
        const uint32_t kv_bytes = (uint32_t)(n - 1) * stride_b + D * 4;
        const __amdgpu_buffer_rsrc_t rk = make_rsrc(p.k + ((int64_t)wi.row0 * p.c.hkv + g) * D, kv_bytes);
        const __amdgpu_buffer_rsrc_t rv = make_rsrc(p.v + ((int64_t)wi.row0 * p.c.hkv + g) * D, kv_bytes);
        const int64_t roff = at.at(min(i, rows - 1)), soff = at.stat(min(i, rows - 1));
        const uint32_t first = (uint32_t)t_lo * kF32Tile * stride_b;
        fl.load(rv, smem + kT, first, stride_b);
        f32x4 q[D / 8], dof[D / 8];
        f32_load_row<D>(q, p.q + roff, half);
        f32_load_row<D>(dof, p.d_o + roff, half);
        float Di = 0.f;
#pragma unroll
        for (int a = 0; a < D / 8; ++a) {
            const f32x4 x = *reinterpret_cast<const f32x4*>(p.o + roff + 8 * a + 4 * half);
#pragma unroll
            for (int e = 0; e < 4; ++e) Di = __builtin_fmaf(x[e], dof[a][e], Di);
        }
        {
            float lo, hi;
            both_halves(Di, lo, hi);
            Di = lo + hi;
        }
        if (part == 0 && split == 0 && half == 0 && i < rows) p.D[soff] = Di;
        const float lse = p.lse_in[soff];
        fl.load(rk, smem, first, stride_b);
        f32x16 acc[NDB];
        f32_zero(acc);
        for (int t = t_lo; t < n_kt; ++t) {
            const uint32_t nxt = (uint32_t)(t + 1) * kF32Tile * stride_b;
            const bool more = t + 1 < n_kt;
            if (t == max(n_kt - 2, t_lo)) wf.claim(p.hm, p.cursors);
            const int key0 = t * kF32Tile + 32 * split;
            const bool work = key0 < n && wrow0 < rows;
            f32x16 s[1], dp[1];
            f32_zero(s);
            f32_zero(dp);
            f32_arrive<kL>();                                       // V tile t is there; K was requested after it
            if (work) f32_row_product(dp[0], fl, kT, dof);
            f32_wait_lds();
            f32_arrive<0>();                                        // K tile t is there, V may be overwritten
            if (more) fl.load(rv, smem + kT, nxt, stride_b);
            if (work) f32_row_product(s[0], fl, 0, q);
            if (work) {
                const int rel = n - 1 - key0 - 4 * half;
#pragma unroll
                for (int r = 0; r < 16; ++r) s[0][r] = f32_exp(__builtin_fmaf(p.scale, s[0][r], -lse)) * (dp[0][r] - Di);
                if (key0 + 32 > n) {                             // (exp(-LSE) of a zero row need not be finite)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (8 * (r >> 2) + (r & 3) > rel) s[0][r] = 0.f;
                }
                f32_col_product(acc, fl, 0, s[0]);
            }
            f32_release();
            if (more) fl.load(rk, smem, nxt, stride_b);
        }
        if (split) f32_put(smem + (2 * (split - 1) + rg) * kAcc, acc, lane);
        __syncthreads();
        if (split == 0 && wrow0 < rows) {
#pragma unroll
            for (int x = 1; x < kF32Splits; ++x) f32_add(acc, 1.f, smem + (2 * (x - 1) + rg) * kAcc, 1.f, lane);
            if (i < rows) f32_store_row<D>(out + roff, acc, p.scale, half);
        }
    }
}

// dK/dV: 32 keys of a KV head, the query rows of its heads one after the other in tiles of 128 tokens; kParts: parts of them.  (A
// form of its own: the registers are full, and the parts' numbers cost the whole form 12 % at d = 128.)
template <int D, bool kParts>
__global__ void __launch_bounds__(64 * kF32KvWaves, 1) hyd_cross_dkdv_fp32_kernel(CrossF32Params p) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    constexpr int kT = f32_tile_bytes<D>(), NDB = D / 32;
    constexpr int kAcc = NDB * 64 * 64;
    int* slot = reinterpret_cast<int*>(smem + 2 * kT);
    const int tid = threadIdx.x, lane = tid & 63;
    const int split = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, half = lane >> 5;
    const int G = p.c.G;
    const uint32_t stride_b = (uint32_t)p.c.hq * D * 4;
    F32Lds<D, kF32KvWaves> fl;
    fl.init(lane, split, split, smem, stride_b);
    WorkFetcher wf;
    WorkItem wi;
    for (bool have = wf.first(p.hm, p.hdr, p.cursors, p.items, slot, wi, blockIdx.x); have; have = wf.next(p.hm, p.cursors, p.items, slot, wi)) {
        const int g = wi.head, keys = kParts ? wi.lev & ((1 << kCrossPartShift) - 1) : wi.lev, part = kParts ? wi.lev >> kCrossPartShift : 0;
        const int q0 = wi.row0 / G, L = wi.len / G;              // tokens of the sequence's queries
        const int64_t koff = ((int64_t)(wi.seq + min(l32, keys - 1)) * p.c.hkv + g) * D;
        int it0 = 0, n_iter = (L + kF32Tile - 1) / kF32Tile * G;      // iterations: (tile, head), heads inner
        if (kParts) {
            const int per_part = (n_iter + p.parts - 1) / p.parts;
            it0 = min(part * per_part, n_iter);
            n_iter = min(it0 + per_part, n_iter) - it0;
        }
        f32x16 acck[NDB], accv[NDB];
        f32_zero(acck);
        f32_zero(accv);
        if (n_iter == 0) wf.claim(p.hm, p.cursors);
        const uint32_t q_bytes = L > 0 ? (uint32_t)(L - 1) * stride_b + D * 4 : 0;
        int ld_i = kParts ? it0 / G * kF32Tile : 0, ld_h = kParts ? it0 % G : 0;
        auto load_q = [&]() {
            fl.load(make_rsrc(p.q + ((int64_t)q0 * p.c.hq + g * G + ld_h) * D, q_bytes), smem, (uint32_t)ld_i * stride_b, stride_b);
        };
        auto load_do = [&]() {                                   // follows load_q of the same iteration
            fl.load(make_rsrc(p.d_o + ((int64_t)q0 * p.c.hq + g * G + ld_h) * D, q_bytes), smem + kT, (uint32_t)ld_i * stride_b, stride_b);
            if (++ld_h == G) { ld_h = 0; ld_i += kF32Tile; }
        };
        if (n_iter > 0) load_q();
        f32x4 kr[D / 8], vr[D / 8];
        f32_load_row<D>(kr, p.k + koff, half);
        f32_load_row<D>(vr, p.v + koff, half);
        if (n_iter > 0) load_do();
        int ti = kParts ? it0 / G * kF32Tile : 0, hh = kParts ? it0 % G : 0;
        for (int it = 0; it < n_iter; ++it) {
            const bool more = it + 1 < n_iter;
            if (it == max(n_iter - 2, 0)) wf.claim(p.hm, p.cursors);
            const int i0 = ti + 32 * split;
            const bool work = i0 < L;
            // statistics of the block's rows (register r: row i0 + 8 (r / 4) + 4 half + r % 4); rows past the
            // sequence repeat its last one and are masked below, as exp(-LSE) need not be finite
            float nl[16], nd[16];
            if (work) {
                const int64_t at = (int64_t)(g * G + hh) * p.c.Tq + q0;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int ii = min(i0 + 8 * (r >> 2) + 4 * half + (r & 3), L - 1);
                    nl[r] = p.lse_in[at + ii];
                    nd[r] = p.D[at + ii];
                }
            }
            f32x16 s[1], dp[1];
            f32_zero(s);
            f32_zero(dp);
            f32_arrive<0>();                                     // Q and dO tiles of this iteration
            if (work) {
                f32_row_product(s[0], fl, 0, kr);
                f32_row_product(dp[0], fl, kT, vr);
                const int end = L - i0 - 4 * half;               // register r is a row of the sequence iff its offset < end
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    float pr = f32_exp(__builtin_fmaf(p.scale, s[0][r], -nl[r]));
                    float ds = pr * (dp[0][r] - nd[r]);
                    if (i0 + 32 > L) {
                        pr = 8 * (r >> 2) + (r & 3) < end ? pr : 0.f;
                        ds = 8 * (r >> 2) + (r & 3) < end ? ds : 0.f;
                    }
                    s[0][r] = pr;
                    dp[0][r] = ds;
                }
                f32_col_product(acck, fl, 0, dp[0]);
            }
            f32_release();
            if (more) load_q();                                  // under the dV product
            if (work) f32_col_product(accv, fl, kT, s[0]);
            f32_release();
            if (more) load_do();
            if (++hh == G) { hh = 0; ti += kF32Tile; }
        }
        if (split) {
            f32_put(smem + 2 * (split - 1) * kAcc, acck, lane);
            f32_put(smem + (2 * (split - 1) + 1) * kAcc, accv, lane);
        }
        __syncthreads();
        if (split == 0) {
#pragma unroll
            for (int x = 0; x < kF32Splits - 1; ++x) {
                f32_add(acck, 1.f, smem + 2 * x * kAcc, 1.f, lane);
                f32_add(accv, 1.f, smem + (2 * x + 1) * kAcc, 1.f, lane);
            }
            if (l32 < keys) {
                const int64_t plane = (int64_t)p.c.Tk * p.c.hkv * D;
                f32_store_row<D>((kParts ? p.part_o + part * plane : p.dk) + koff, acck, p.scale, half);
                f32_store_row<D>((kParts ? p.part_o + (p.parts + part) * plane : p.dv) + koff, accv, 1.f, half);
            }
        }
    }
}

}  // namespace hyd
