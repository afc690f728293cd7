// Cross attention, backward in bf16 where a sequence has few keys (at most kKeysMax), as when an image or sound model looks at a
// prompt: all three gradients in one pass over the rows.
//
// The general backward goes over Q and dO three times and writes copies of both (hyd_cross_bwd.h), which is what a call with few keys
// takes: 9 units of HBM traffic (a unit: Q once) where 4 have to be, Q, dO and O read and dQ written.  Here the keys of a (sequence, KV
// head) stay in registers, 32 for each of four waves, and tiles of 64 packed rows stream past them:
//     S = Q K^T, P = exp2(S scale - LSE2), dP = dO V^T - D, dS = P dP        (one key per lane, rows in the slots)
//     dV^T += dO^T P, dK^T += Q^T dS                                        (the wave's keys)
//     dQ^T = K^T dS^T                  (dS of all keys meets in LDS; a wave forms 32 columns of the head, for d = 64 of 32 rows)
// D = rowsum(dO * O) and LSE2 of a tile are formed one tile ahead.
//
// Arithmetic.  P and dS enter the second products as two bf16 numbers, the rounded value and the rest, 16 bits together, so that
// every product runs on the bf16 MFMA with Q, K, dO as they are: no scaling of dO, no copies, and no range but bf16's own.
//
// Bound by HBM for 64 keys and more rows.  Each tile has two barriers: the first opens the tile (and says that the stage before the
// last has been read by all), the second publishes dS.
#pragma once
#include "hyd_cross_bwd.h"

namespace hyd {

constexpr int kKeysMax = 128, kKeysWaves = 4, kKeysThreads = 64 * kKeysWaves, kKeysBM = 64, kKeysStages = 3;
constexpr int kKeysTileBytes = kKeysBM * kRowBytes, kKeysStageBytes = 2 * kKeysTileBytes;         // Q, dO
// dS: [hi, lo][key][64 rows] bf16; the 32-byte quarter of rows 16 q .. of a key lies at q ^ ds_swz(key), so that the transposing reads
// (four keys, 32 rows) meet no bank twice
constexpr int kKeysDsOff = kKeysStages * kKeysStageBytes, kKeysDsRow = kKeysBM * 2, kKeysDsBytes = kKeysMax * kKeysDsRow;
constexpr int kKeysStatOff = kKeysDsOff + 2 * kKeysDsBytes;                                        // [parity][LSE2, D][64]
constexpr int kKeysLds = kKeysStatOff + 4 * kKeysBM * 4;
constexpr int kKeysOutRow = 80;           // bytes of a row of 32 dQ columns in LDS
static_assert(kKeysMax * kRowBytes <= kKeysStageBytes && kKeysMax * kRowBytes <= 2 * kKeysDsBytes, "K and V rows while an item begins");
__device__ __forceinline__ int ds_swz(int key) { return (((key >> 1) & 1) << 1) | ((key >> 2) & 1); }

struct CrossKeysParams {
    CrossShape c;
    const uint16_t* q; const uint16_t* k; const uint16_t* v; const uint16_t* o; const uint16_t* d_o; const float* lse;
    uint16_t* dq; uint16_t* dk; uint16_t* dv;
    float* part;                          // parts > 1: [dK, dV][parts][Tk][Hkv][d]
    int parts;                            // of the rows of a (sequence, KV head)
    float scale, scale_log2;
};

// LDS stores beside direct-to-LDS loads in flight, in assembly for the reason given at lds_issue_row
__device__ __forceinline__ void lds_store(uint32_t addr, u32x2 v) { asm volatile("ds_write_b64 %0, %1" : : "v"(addr), "v"(v) : "memory"); }
__device__ __forceinline__ void lds_store(uint32_t addr, float v) { asm volatile("ds_write_b32 %0, %1" : : "v"(addr), "v"(v) : "memory"); }
// two floats as pairs of bf16: rounded values, and what they leave
__device__ __forceinline__ void split_bf16(float a, float b, uint32_t& hi, uint32_t& lo) {
    hi = pack_bf16(a, b);
    lo = pack_bf16(a - bf16_lo(hi), b - bf16_hi(hi));
}

template <int D>
__global__ void __launch_bounds__(kKeysThreads, 1) hyd_cross_bwd_keys_bf16_kernel(CrossKeysParams p) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    constexpr int kRowB = D * 2, NK = D / 16, NDB = D / 32, NV = D / 32;
    constexpr int kDma = 2 * 64 * kRowBytes / 1024 / kKeysWaves;              // loads of a tile by each wave
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, half = lane >> 5, lane16 = lane & 15;
    const int g = blockIdx.x % p.c.hkv, part = (blockIdx.x / p.c.hkv) % p.parts, seq = blockIdx.x / p.c.hkv / p.parts;
    const CrossSeq x = cross_seq(p.c, seq);
    const int G = p.c.G, n = min(x.n, kKeysMax), rows_all = x.lq * G;
    const int64_t q_stride = (int64_t)p.c.hq * D, kv_stride = (int64_t)p.c.hkv * D;
    const uint32_t kv_stride_b = (uint32_t)kv_stride * 2, q_stride_b = (uint32_t)q_stride * 2;
    const int n_all = (rows_all + kKeysBM - 1) / kKeysBM, per_part = (n_all + p.parts - 1) / p.parts;
    const int t_lo = min(part * per_part, n_all), t_hi = min(t_lo + per_part, n_all);
    const int64_t kv_at = (int64_t)x.k0 * kv_stride + (int64_t)g * D;
    CrossRows cr;
    cr.init(G);
    if (part == 0)                                        // behind the valid keys: zeros
        for (int i = n * (D / 8) + tid; i < x.rows * (D / 8); i += kKeysThreads) {
            const int64_t at = kv_at + (int64_t)(i / (D / 8)) * kv_stride + 8 * (i % (D / 8));
            *reinterpret_cast<u32x4*>(p.dk + at) = u32x4{0u, 0u, 0u, 0u};
            *reinterpret_cast<u32x4*>(p.dv + at) = u32x4{0u, 0u, 0u, 0u};
        }
    if (n == 0) {                                         // no keys: dQ = 0
        for (int i = t_lo * kKeysBM * (D / 8) + tid; i < min(t_hi * kKeysBM, rows_all) * (D / 8); i += kKeysThreads) {
            const int r = i / (D / 8), token = r / G;
            *reinterpret_cast<u32x4*>(p.dq + (x.q0 + token) * q_stride + (int64_t)(g * G + r - token * G) * D + 8 * (i % (D / 8))) = u32x4{0u, 0u, 0u, 0u};
        }
        return;
    }
    FragAddr fa;
    fa.init(lane, smem);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)smem;
    const float scale_log2 = fmaxf(fabsf(p.scale_log2), 1e-30f);
    const uint32_t sign_flip = p.scale_log2 < 0.f ? 0x80008000u : 0u;

    // ---- row tiles
    struct Rows { int t0, rem, rows; };                   // token of the first row, its head in the group, rows of the tile
    const auto tile_rows = [&](int t) -> Rows {
        const int r = t * kKeysBM, token = r / G;
        return Rows{x.q0 + token, r - token * G, min(rows_all - r, kKeysBM)};
    };
    const auto tile_rsrc = [&](const uint16_t* base, const Rows& w) {
        return make_rsrc(base + (int64_t)w.t0 * q_stride + (int64_t)g * G * D, (uint32_t)((w.rem + w.rows - 1) / G) * q_stride_b + (uint32_t)G * kRowB);
    };
    auto load_tile = [&](int t, int stage) {
        const Rows w = tile_rows(t);
        dma_packed_rows<kKeysWaves, D>(tile_rsrc(p.q, w), smem + stage * kKeysStageBytes, [](int) { return 0; }, 1, cr, w.rem, w.rows, q_stride_b, wave, lane);
        dma_packed_rows<kKeysWaves, D>(tile_rsrc(p.d_o, w), smem + stage * kKeysStageBytes + kKeysTileBytes, [](int) { return 0; }, 1, cr, w.rem, w.rows, q_stride_b, wave, lane);
    };
    // statistics: four threads to a row
    u32x4 so[NV], sd[NV];
    float sl = 0.f;
    auto load_stats = [&](int t) {
        const Rows w = tile_rows(t);
        const __amdgpu_buffer_rsrc_t ro = tile_rsrc(p.o, w), rd = tile_rsrc(p.d_o, w);
        const int r = tid >> 2;
        int token, head;
        cr.split(w.rem + r, token, head);
        const uint32_t at = r < w.rows ? (uint32_t)token * q_stride_b + (uint32_t)(head * kRowB + (tid & 3) * (kRowB / 4)) : kDmaOutOfRange;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            so[i] = __builtin_amdgcn_raw_buffer_load_b128(ro, at, 16 * i, 0);
            sd[i] = __builtin_amdgcn_raw_buffer_load_b128(rd, at, 16 * i, 0);
        }
        sl = r < w.rows ? p.lse[(int64_t)(g * G + head) * p.c.Tq + w.t0 + token] : 0.f;
        __builtin_amdgcn_sched_barrier(0);
    };
    auto put_stats = [&](int t) {                         // rows behind the last one: zeros, like their Q and dO
        float acc = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc += bf16_lo(so[i][e]) * bf16_lo(sd[i][e]) + bf16_hi(so[i][e]) * bf16_hi(sd[i][e]);
        acc += __shfl_xor(acc, 1, 64);
        acc += __shfl_xor(acc, 2, 64);
        const uint32_t at = lds0 + (uint32_t)(kKeysStatOff + (t & 1) * 2 * kKeysBM * 4 + (tid >> 2) * 4);
        if ((tid & 3) == 0) {
            lds_store(at, -sl * kLog2e);
            lds_store(at + kKeysBM * 4, -acc);
        }
    };
    if (t_lo < t_hi) load_stats(t_lo);
    // K rows to stage 2, V rows to the place of dS
    {
        const uint32_t bytes = (uint32_t)(n - 1) * kv_stride_b + kRowB;
        const uint32_t voff = dma_lane_voff<D>(4 * wave + (lane >> 4), lane, kv_stride_b);
        auto tile_at = [&](int j) { return (uint32_t)(64 * j) * kv_stride_b; };
        dma_rows<kKeysWaves>(make_rsrc(p.k + kv_at, bytes), smem + 2 * kKeysStageBytes, [](int j) { return j * 64 * kRowBytes; }, kKeysMax / 64, kv_stride_b, tile_at, wave, voff);
        dma_rows<kKeysWaves>(make_rsrc(p.v + kv_at, bytes), smem + kKeysDsOff, [](int j) { return j * 64 * kRowBytes; }, kKeysMax / 64, kv_stride_b, tile_at, wave, voff);
    }
    if (t_lo < t_hi) load_tile(t_lo, 0);
    if (t_lo + 1 < t_hi) load_tile(t_lo + 1, 1);
    f32x16 dv[NDB], dk[NDB];
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) dv[db][r] = dk[db][r] = 0.f;
    __builtin_amdgcn_s_waitcnt(0x0F70);                   // vmcnt(0)
    __syncthreads();
    // this wave's keys, and the columns of K that its dQ takes
    const bool active = 32 * wave < n;
    const int cb = D == 128 ? wave : wave & 1, rb0 = D == 128 ? 0 : wave >> 1;
    constexpr int kRb = D == 128 ? 2 : 1;                 // row blocks of a wave's dQ
    bf16x8 kf[NK], vf[NK], ktf[kKeysMax / 16];
    {
        LdsQueue lq{0};
        RowFrag f[2 * NK];
#pragma unroll
        for (int ks = 0; ks < NK; ++ks) {
            lds_issue_row(lq, f[ks], fa.row[ks] + (uint32_t)(2 * kKeysStageBytes + 32 * wave * kRowBytes), 0);
            lds_issue_row(lq, f[NK + ks], fa.row[ks] + (uint32_t)(kKeysDsOff + 32 * wave * kRowBytes), 0);
        }
#pragma unroll
        for (int ks = 0; ks < NK; ++ks) {
            lds_wait(lq, f[ks]);
            kf[ks] = as_bf16x8(f[ks].v ^ sign_flip);      // (only the scores see the sign)
            vf[ks] = lds_wait(lq, f[NK + ks]);
        }
        uint32_t c_lo = fa.col[0], c_hi = fa.col[1];
#pragma unroll
        for (int i = 1; i < NDB; ++i)
            if (cb == i) { c_lo = fa.col[2 * i]; c_hi = fa.col[2 * i + 1]; }
        ColFrag c[kKeysMax / 16];
#pragma unroll
        for (int b = 0; b < kKeysMax / 16; ++b) lds_issue_col(lq, c[b], c_lo + (uint32_t)(2 * kKeysStageBytes), c_hi + (uint32_t)(2 * kKeysStageBytes), b * 16 * kRowBytes);
#pragma unroll
        for (int b = 0; b < kKeysMax / 16; ++b) ktf[b] = lds_wait(lq, c[b]);
    }
    if (t_lo < t_hi) put_stats(t_lo);
    __builtin_amdgcn_s_waitcnt(0xc07f);                   // lgkmcnt(0)
    const float hidden = 32 * wave + l32 < n ? 0.f : -INFINITY;       // a key behind the last one: its scores begin, and stay, at -inf
    // this lane's dS: written by key, read by row
    const int my_key = 32 * wave + l32;
    const uint32_t ds_w = lds0 + (uint32_t)(kKeysDsOff + my_key * kKeysDsRow + 8 * half);
    uint32_t ds_r[kRb][2];
#pragma unroll
    for (int i = 0; i < kRb; ++i)
#pragma unroll
        for (int hi = 0; hi < 2; ++hi) {
            const int key = 4 * half + 8 * hi + (lane16 >> 2), quarter = 2 * (D == 128 ? i : rb0) + ((lane >> 4) & 1);
            ds_r[i][hi] = lds0 + (uint32_t)(kKeysDsOff + key * kKeysDsRow + ((quarter ^ ds_swz(key)) << 5) + 8 * (lane16 & 3));
        }

    for (int t = t_lo; t < t_hi; ++t) {
        const int stage = (t - t_lo) % kKeysStages, base = stage * kKeysStageBytes;
        // this tile is there: at most the next one's loads are under way (stores of dQ only make the wait stricter)
        if (t + 1 < t_hi) __builtin_amdgcn_s_waitcnt(0x0F70 | (kDma & 15));
        else __builtin_amdgcn_s_waitcnt(0x0F70);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (t + 1 < t_hi) load_stats(t + 1);
        if (t + 2 < t_hi) load_tile(t + 2, stage == 0 ? 2 : stage - 1);
        __builtin_amdgcn_sched_barrier(0);
        {   // (a wave without keys goes along: its P and dS are zeros, and a branch here costs copies of the accumulators)
            const uint32_t qt = (uint32_t)base, stat = lds0 + (uint32_t)(kKeysStatOff + (t & 1) * 2 * kKeysBM * 4 + 16 * half);
#pragma unroll
            for (int rb = 0; rb < 2; ++rb) {
                // fragments are read kAhead ahead: Q and dO rows, then dO and Q columns
                constexpr int kAhead = 4;
                LdsQueue lq{0};
                RowFrag f[kAhead], l4[4], d4[4];
                ColFrag cf[kAhead];
                f32x16 s, xd;
                uint32_t ph[8], pl[8], sh[8], sl2[8];
                auto issue_first = [&](int i) {
                    lds_issue_row(lq, f[i % kAhead], fa.row[i % NK] + qt, (i < NK ? 0 : kKeysTileBytes) + 32 * rb * kRowBytes);
                };
                auto issue_second = [&](int i) {
                    const int j = i % (2 * NDB);
                    lds_issue_col(lq, cf[i % kAhead], fa.col[2 * (j % NDB)] + qt, fa.col[2 * (j % NDB) + 1] + qt, (i < 2 * NDB ? kKeysTileBytes : 0) + (2 * rb + j / NDB) * 16 * kRowBytes);
                };
#pragma unroll
                for (int i = 0; i < kAhead; ++i) issue_first(i);
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = hidden;
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < NK; ++i) {            // S
                    s = mfma32(lds_wait(lq, f[i % kAhead]), kf[i], s);
                    issue_first(i + kAhead);
                    if (i < 4) lds_issue_row(lq, d4[i], stat, (kKeysBM + 32 * rb + 8 * i) * 4);
                    __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int rq = 0; rq < 4; ++rq) {          // dP begins at -D
                    const u32x4 v = lds_wait_raw(lq, d4[rq]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) xd[4 * rq + e] = __uint_as_float(v[e]);
                }
#pragma unroll
                for (int rq = 0; rq < 4; ++rq) lds_issue_row(lq, l4[rq], stat, (32 * rb + 8 * rq) * 4);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < NK; ++i) {            // dP
                    xd = mfma32(lds_wait(lq, f[i % kAhead]), vf[i], xd);
                    if (i + kAhead < NK) issue_first(NK + i + kAhead);
                    else issue_second(i + kAhead - NK);
                    __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int rq = 0; rq < 4; ++rq) {          // P in place of S
                    const u32x4 v = lds_wait_raw(lq, l4[rq]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[4 * rq + e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[4 * rq + e], scale_log2, __uint_as_float(v[e])));
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) split_bf16(s[2 * j], s[2 * j + 1], ph[j], pl[j]);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < 4 * NDB; ++i) {       // dV, then dK; dS is formed under the first products of dV
                    const int j = i % (2 * NDB), b2 = j / NDB, db = j % NDB;
                    const bf16x8 a = lds_wait(lq, cf[i % kAhead]);
                    const auto frag = [&](const uint32_t (&w)[8]) { return as_bf16x8(u32x4{w[4 * b2], w[4 * b2 + 1], w[4 * b2 + 2], w[4 * b2 + 3]}); };
                    if (i < 2 * NDB) {
                        dv[db] = mfma32(a, frag(ph), dv[db]);
                        dv[db] = mfma32(a, frag(pl), dv[db]);
                    } else {
                        dk[db] = mfma32(a, frag(sh), dk[db]);
                        dk[db] = mfma32(a, frag(sl2), dk[db]);
                    }
                    if (i + kAhead < 4 * NDB) issue_second(i + kAhead);
                    constexpr int kPer = 8 / (2 * NDB);   // pairs of dS formed beside a fragment of dO
#pragma unroll
                    for (int e = 0; e < kPer; ++e) {
                        const int m = kPer * i + e;
                        if (i < 2 * NDB) split_bf16(s[2 * m] * xd[2 * m], s[2 * m + 1] * xd[2 * m + 1], sh[m], sl2[m]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int rq = 0; rq < 4; ++rq) {          // rows 32 rb + 8 rq + 4 half ..: quarter 2 rb + rq / 2
                    const uint32_t at = ds_w + (uint32_t)(((2 * rb + (rq >> 1)) ^ ds_swz(my_key)) << 5) + 16 * (rq & 1);
                    lds_store(at, u32x2{sh[2 * rq], sh[2 * rq + 1]});
                    lds_store(at + kKeysDsBytes, u32x2{sl2[2 * rq], sl2[2 * rq + 1]});
                }
            }
        }
        if (t + 1 < t_hi) put_stats(t + 1);
        __builtin_amdgcn_s_waitcnt(0xc07f);               // lgkmcnt(0): dS and the statistics are written, Q and dO read
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        // dQ^T = K^T dS^T, 32 columns of the head
        f32x16 dq[kRb];
#pragma unroll
        for (int i = 0; i < kRb; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) dq[i][r] = 0.f;
        {
            constexpr int kAhead = 4, kFrags = kKeysMax / 16 * 2 * kRb;      // fragment m: 16 keys, hi or lo, row block
            LdsQueue lq{0};
            ColFrag f[kAhead];
            auto issue = [&](int m) {
                const int i = m % kRb, lo = m / kRb % 2, b = m / kRb / 2;
                lds_issue_col(lq, f[m % kAhead], ds_r[i][0], ds_r[i][1], lo * kKeysDsBytes + b * 16 * kKeysDsRow);
            };
#pragma unroll
            for (int m = 0; m < kAhead; ++m) issue(m);
#pragma unroll
            for (int m = 0; m < kFrags; ++m) {
                dq[m % kRb] = mfma32(ktf[m / kRb / 2], lds_wait(lq, f[m % kAhead]), dq[m % kRb]);
                if (m + kAhead < kFrags) issue(m + kAhead);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        // through this wave's part of the stage (its Q and dO have been read), then 64 bytes of each row
        const Rows w = tile_rows(t);
        const uint32_t out = lds0 + (uint32_t)(base + wave * kKeysBM * kKeysOutRow);
#pragma unroll
        for (int i = 0; i < kRb; ++i)
#pragma unroll
            for (int rq = 0; rq < 4; ++rq)
                lds_store(out + (uint32_t)((32 * i + l32) * kKeysOutRow + (8 * rq + 4 * half) * 2),
                          u32x2{pack_bf16(dq[i][4 * rq] * p.scale, dq[i][4 * rq + 1] * p.scale), pack_bf16(dq[i][4 * rq + 2] * p.scale, dq[i][4 * rq + 3] * p.scale)});
        __builtin_amdgcn_s_waitcnt(0xc07f);
        {
            LdsQueue lq{0};
            RowFrag f[2 * kRb];
#pragma unroll
            for (int i = 0; i < 2 * kRb; ++i) lds_issue_row(lq, f[i], out + (uint32_t)((lane >> 2) * kKeysOutRow + (lane & 3) * 16), 16 * i * kKeysOutRow);
#pragma unroll
            for (int i = 0; i < 2 * kRb; ++i) {
                const u32x4 v = lds_wait_raw(lq, f[i]);
                const int r = 32 * rb0 + 16 * i + (lane >> 2);
                int token, head;
                cr.split(w.rem + r, token, head);
                if (r < w.rows)
                    *reinterpret_cast<u32x4*>(p.dq + (int64_t)(w.t0 + token) * q_stride + (int64_t)(g * G + head) * D + 32 * cb + 8 * (lane & 3)) = v;
            }
        }
    }
    __syncthreads();                                      // every wave is done with the ring
    if (active) {
        const uint32_t o_stage = lds0 + (uint32_t)(wave * 2 * 32 * kRowBytes);
        const int64_t at = kv_at + (int64_t)(32 * wave) * kv_stride;
        if (p.parts == 1) {
            store_rows_via_lds<D>(p.dv + at, kv_stride, n - 32 * wave, dv, 1.f, o_stage, lane);
            store_rows_via_lds<D>(p.dk + at, kv_stride, n - 32 * wave, dk, p.scale, o_stage + 32 * kRowBytes, lane);
        } else {
            const int64_t plane = (int64_t)p.c.Tk * kv_stride;
            store_rows_f32_via_lds<D>(p.part + (p.parts + part) * plane + at, kv_stride, n - 32 * wave, dv, 1.f, o_stage, lane);
            store_rows_f32_via_lds<D>(p.part + part * plane + at, kv_stride, n - 32 * wave, dk, p.scale, o_stage + 32 * kRowBytes, lane);
        }
    }
}

}  // namespace hyd
