// Cross attention, backward in bf16 where a sequence has few keys (at most kKeysMax), as when an image or sound model looks at a
// prompt: all three gradients in one pass over the rows.
//
// The general backward goes over Q and dO three times and writes copies of both (hyd_cross_bwd.h): 9 units of HBM traffic (a unit:
// Q once) where 4 have to be, Q, dO and O read and dQ written.  Here the keys of a (sequence, KV head) stay in registers, 32 for each of
// four pairs of waves, and tiles of 64 packed rows stream past them (one key per lane, rows in the slots):
//     first waves:   S = Q K^T, P = exp2(S scale - LSE2), handed over through LDS, dV^T += dO^T P
//     second waves:  dP = dO V^T - D, dS = P dP, dK^T += Q^T dS
//     then all:      dQ^T = K^T dS^T, a block of 32 rows and 32 columns of the head each    (dS of all keys meets in LDS)
// D = rowsum(dO * O) and LSE2 of a tile are formed one tile ahead.  The two waves of a pair share a SIMD, so that one's vector work
// runs under the other's products.
//
// Arithmetic.  P and dS enter the second products as two bf16 numbers, the rounded value and the rest, 16 bits together, so that
// every product runs on the bf16 MFMA with Q, K, dO as they are: no scaling of dO, no copies, and no range but bf16's own.
//
// Bound by the meetings of its two waves to a SIMD: the waves wait for 47 % of their time, the matrix pipe is busy for 29 % of the clocks, vector
// ALU and LDS for 41 each.  All 128 keys are computed whatever their number.  16 sequences of 2000 queries, 8 heads, 128 keys here and
// 129 keys in the general form: d = 64 72 and 129 us, d = 128 121 and 236 us; of 1024 to 4096 queries and 8 to 77 keys, d = 64, 84 us and 5 for
// the sums (151 MB have to be moved, 177 are).
//
// A tile has three barriers: the first opens it (and says that the stage before the last has been read by all), the second hands P
// over, the third publishes dS.
#pragma once
#include "hyd_cross_bwd.h"

namespace hyd {

constexpr int kKeysMax = 128, kKeysPairs = 4, kKeysWaves = 2 * kKeysPairs, kKeysThreads = 64 * kKeysWaves;
// Tiles.  A row of a tile in LDS is 256 bytes: a row of d = 128, or rows r and r + 64 of d = 64, whose tiles have 128 rows then.
// (What a tile takes is mostly waiting for the step before, so tiles are as large as registers and LDS allow.)
template <int D> struct KeysForm {
    static constexpr int kBM = D == 64 ? 128 : 64, kBlocks = kBM / 32, kStages = D == 64 ? 2 : 3;
    static constexpr int kTileBytes = 64 * kRowBytes, kStageBytes = 2 * kTileBytes;                // Q, dO
    // dS: [hi, lo][key][row] bf16; the 32 bytes of rows 16 q .. of a key lie at q ^ swz(key), so that the transposing reads (four keys, 32
    // rows) meet no bank twice.  Before, the bytes of a pair's keys hold its P: [row block][4 slots][lane] floats.
    static constexpr int kDsOff = kStages * kStageBytes, kDsRow = kBM * 2, kDsBytes = kKeysMax * kDsRow;
    static constexpr int kStatOff = kDsOff + 2 * kDsBytes;                                         // [parity][LSE2, D][row]
    static constexpr int kLds = kStatOff + 4 * kBM * 4;
    static_assert(kKeysMax * kRowBytes <= kStageBytes && kKeysMax * kRowBytes <= 2 * kDsBytes, "K and V rows while an item begins");
    static_assert(32 * kDsRow == kBlocks / 2 * 64 * 16 * 4, "P of half the row blocks in the place of half of dS");
    __device__ __forceinline__ static int swz(int key) { return D == 64 ? ((key & 3) << 1) | ((key >> 2) & 1) : (((key >> 1) & 1) << 1) | ((key >> 2) & 1); }
    __device__ __forceinline__ static constexpr int p_off(int rb) { return rb / (kBlocks / 2) * kDsBytes + rb % (kBlocks / 2) * 4096; }
};
constexpr int kKeysOutRow = 80;           // bytes of a row of 32 dQ columns in LDS

struct CrossKeysParams {
    CrossShape c;
    const uint16_t* q; const uint16_t* k; const uint16_t* v; const uint16_t* o; const uint16_t* d_o; const float* lse;
    uint16_t* dq; uint16_t* dk; uint16_t* dv;
    float* part;                          // parts > 1: [dK, dV][parts][Tk][Hkv][d]
    int parts;                            // of the rows of a (sequence, KV head)
    float scale, scale_log2;
};

// LDS stores beside direct-to-LDS loads in flight, in assembly for the reason given at lds_issue_row
__device__ __forceinline__ void lds_store(uint32_t addr, u32x4 v, int off) { asm volatile("ds_write_b128 %0, %1 offset:%2" : : "v"(addr), "v"(v), "i"(off) : "memory"); }
__device__ __forceinline__ void lds_store(uint32_t addr, u32x2 v) { asm volatile("ds_write_b64 %0, %1" : : "v"(addr), "v"(v) : "memory"); }
__device__ __forceinline__ void lds_store(uint32_t addr, float v) { asm volatile("ds_write_b32 %0, %1" : : "v"(addr), "v"(v) : "memory"); }
// two floats as pairs of bf16: rounded values, and what they leave
__device__ __forceinline__ void split_bf16(float a, float b, uint32_t& hi, uint32_t& lo) {
    hi = pack_bf16(a, b);
    lo = pack_bf16(a - bf16_lo(hi), b - bf16_hi(hi));
}

// A wave's direct-to-LDS loads of a tile: N of them, kStep rows apart.  (D keeps the two kernels' instances apart: the compiler's host
// pass, which does not know the instruction, drops whoever calls an instance for the second time.)
template <int D, int kStep, int N>
__device__ __forceinline__ void dma_at(const __amdgpu_buffer_rsrc_t& rs, char* lds, const uint32_t (&voff)[N]) {
#pragma unroll
    for (int j = 0; j < N; ++j)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void_c*)(lds + kStep * j * kRowBytes), 16, voff[j], 0, 0, 0);
}

struct KeysRows { int t0, rem, rows; };       // a tile: token of its first row, that row's head in the group, rows

template <int D>
__global__ void __launch_bounds__(kKeysThreads, 1) hyd_cross_bwd_keys_bf16_kernel(CrossKeysParams p) {
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    using F = KeysForm<D>;
    constexpr int kRowB = D * 2, NK = D / 16, NDB = D / 32, kBM = F::kBM, kBlocks = F::kBlocks;
    constexpr int kPerRow = kKeysThreads / kBM, NV = kRowB / 16 / kPerRow;     // threads that form a row's statistics, 16-byte pieces of each
    constexpr int kDma = F::kStageBytes / 1024 / kKeysWaves;                   // loads of a tile by each wave
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), pair = wave & (kKeysPairs - 1);
    const int l32 = lane & 31, half = lane >> 5, lane16 = lane & 15;
    const int g = blockIdx.x % p.c.hkv, part = (blockIdx.x / p.c.hkv) % p.parts, seq = blockIdx.x / p.c.hkv / p.parts;
    const CrossSeq x = cross_seq(p.c, seq);
    const int G = p.c.G, n = min(x.n, kKeysMax), rows_all = x.lq * G;
    const int64_t q_stride = (int64_t)p.c.hq * D, kv_stride = (int64_t)p.c.hkv * D;
    const uint32_t kv_stride_b = (uint32_t)kv_stride * 2, q_stride_b = (uint32_t)q_stride * 2;
    const int n_all = (rows_all + kBM - 1) / kBM, per_part = (n_all + p.parts - 1) / p.parts;
    const int t_lo = min(part * per_part, n_all), t_hi = min(t_lo + per_part, n_all);
    const int64_t kv_at = (int64_t)x.k0 * kv_stride + (int64_t)g * D;
    CrossRows cr;
    cr.init(G);
    // behind the valid keys: zeros
    for (int64_t i = n * (D / 8) + part * kKeysThreads + tid; i < (int64_t)x.rows * (D / 8); i += (int64_t)p.parts * kKeysThreads) {
        const int64_t at = kv_at + i / (D / 8) * kv_stride + 8 * (i % (D / 8));
        *reinterpret_cast<u32x4*>(p.dk + at) = u32x4{0u, 0u, 0u, 0u};
        *reinterpret_cast<u32x4*>(p.dv + at) = u32x4{0u, 0u, 0u, 0u};
    }
    if (n == 0) {                                         // no keys: dQ = 0
        for (int i = t_lo * kBM * (D / 8) + tid; i < min(t_hi * kBM, rows_all) * (D / 8); i += kKeysThreads) {
            const int r = i / (D / 8), token = r / G;
            *reinterpret_cast<u32x4*>(p.dq + (x.q0 + token) * q_stride + (int64_t)(g * G + r - token * G) * D + 8 * (i % (D / 8))) = u32x4{0u, 0u, 0u, 0u};
        }
        return;
    }
    // Fragment addresses (see FragAddr): those of the contraction steps of a row fragment differ in bits 5-7 only, those of the column
    // blocks of a column fragment in bits 6-7 and its second row group in bit 5 besides 8 rows.
    uint32_t row_frag, col_frag;
    {
        FragAddr fa;
        fa.init(lane, smem);
        row_frag = fa.row[0];
        col_frag = fa.col[0];
    }
    const auto issue_column = [](LdsQueue& q, ColFrag& f, uint32_t at, int c, int off) {
        lds_issue_col(q, f, at ^ (uint32_t)(c << 6), (at + 8 * kRowBytes) ^ (uint32_t)(c << 6 | 32), off);
    };
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)smem;
    const float scale_log2 = fmaxf(fabsf(p.scale_log2), 1e-30f);
    const uint32_t sign_flip = p.scale_log2 < 0.f ? 0x80008000u : 0u;

    // ---- row tiles.  Where G divides a tile's rows holds whole tokens, and where its rows lie in it is the same for every tile; else
    // both are found by division, tile by tile.
    const bool whole = kBM % G == 0;
    const int per_tile = whole ? kBM / G : 0;         // tokens of a tile
    const auto tile_rows = [&](int t) -> KeysRows {
        const int r = t * kBM, rows = min(rows_all - r, kBM);
        if (whole) return KeysRows{x.q0 + t * per_tile, 0, rows};
        const int token = r / G;
        return KeysRows{x.q0 + token, r - token * G, rows};
    };
    const auto tile_rsrc = [&](const uint16_t* base, const KeysRows& w, bool on) {
        // (bounded by the sequence's last row: those behind it are cut here, or by their offset where tokens are not whole)
        return make_rsrc(base + (int64_t)w.t0 * q_stride + (int64_t)g * G * D, on ? (uint32_t)(min(x.q0 + x.lq - w.t0, kBM + 1) - 1) * q_stride_b + (uint32_t)G * kRowB : 0u);
    };
    constexpr int kRowLoads = kDma / 2;                   // loads of a tensor's tile by each wave
    uint32_t voff[kRowLoads], soff;                       // this lane's rows: of the tile loads, and of the statistics
    const auto find_rows = [&](int rem, int rows) {
        int ln = lane, token, head;
        asm volatile("" : "+v"(ln));
        const int row = 4 * wave + (ln >> 4), chunk = (ln & 15) ^ swz(row);
#pragma unroll
        for (int j = 0; j < kRowLoads; ++j) {
            const int r = row + 4 * kKeysWaves * j + (D == kHeadDim ? 0 : 64 * (chunk / (D / 8)));
            cr.split(rem + r, token, head);
            voff[j] = r < rows ? (uint32_t)token * q_stride_b + (uint32_t)(head * kRowB + (chunk % (D / 8) << 4)) : kDmaOutOfRange;
        }
        cr.split(rem + tid / kPerRow, token, head);
        soff = tid / kPerRow < rows ? (uint32_t)token * q_stride_b + (uint32_t)(head * kRowB + tid % kPerRow * (kRowB / kPerRow)) : kDmaOutOfRange;
    };
    if (whole) find_rows(0, kBM);
    // Tiles behind the last one are asked for too, of a resource without bytes: with the loads under a condition, the compiler does not
    // know how many are under way, and waits for all of them where it needs the statistics, whose loads are older.
    auto load_tile = [&](int t, int stage) {
        const KeysRows w = tile_rows(min(t, t_hi - 1));
        if (!whole) find_rows(w.rem, w.rows);
        const __amdgpu_buffer_rsrc_t rq = tile_rsrc(p.q, w, t < t_hi), rd = tile_rsrc(p.d_o, w, t < t_hi);
        char* d = smem + stage * F::kStageBytes + 4 * wave * kRowBytes;
        dma_at<D, 4 * kKeysWaves>(rq, d, voff);
        dma_at<D, 4 * kKeysWaves>(rd, d + F::kTileBytes, voff);
    };
    u32x4 so[NV], sd[NV];
    float sl = 0.f;
    auto load_stats = [&](int t) {
        const KeysRows w = tile_rows(min(t, t_hi - 1));
        if (!whole) find_rows(w.rem, w.rows);
        const __amdgpu_buffer_rsrc_t ro = tile_rsrc(p.o, w, t < t_hi), rd = tile_rsrc(p.d_o, w, t < t_hi);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            so[i] = __builtin_amdgcn_raw_buffer_load_b128(ro, soff, 16 * i, 0);
            sd[i] = __builtin_amdgcn_raw_buffer_load_b128(rd, soff, 16 * i, 0);
        }
        {
            int token, head;
            cr.split(w.rem + min(tid & (kBM - 1), w.rows - 1), token, head);
            sl = p.lse[(int64_t)(g * G + head) * p.c.Tq + w.t0 + token];
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto put_stats = [&](int t) {                         // rows behind the last one: zeros, like their Q and dO
        float acc = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc += bf16_lo(so[i][e]) * bf16_lo(sd[i][e]) + bf16_hi(so[i][e]) * bf16_hi(sd[i][e]);
#pragma unroll
        for (int m = 1; m < kPerRow; m <<= 1) acc += __shfl_xor(acc, m, 64);
        const uint32_t at = lds0 + (uint32_t)(F::kStatOff + (t & 1) * 2 * kBM * 4);
        if (tid < kBM) lds_store(at + 4 * tid, tid < rows_all - t * kBM ? -sl * kLog2e : 0.f);
        if (tid % kPerRow == 0) lds_store(at + (kBM + tid / kPerRow) * 4, -acc);
    };
    if (t_lo < t_hi) load_stats(t_lo);
    // K rows to the last stage, V rows to the place of dS
    {
        const uint32_t bytes = (uint32_t)(n - 1) * kv_stride_b + kRowB;
        const uint32_t voff_kv = dma_lane_voff<D>(4 * wave + (lane >> 4), lane, kv_stride_b);
        auto tile_at = [&](int j) { return (uint32_t)(64 * j) * kv_stride_b; };
        dma_rows<kKeysWaves>(make_rsrc(p.k + kv_at, bytes), smem + (F::kStages - 1) * F::kStageBytes, [](int j) { return j * 64 * kRowBytes; }, kKeysMax / 64, kv_stride_b, tile_at, wave, voff_kv);
        dma_rows<kKeysWaves>(make_rsrc(p.v + kv_at, bytes), smem + F::kDsOff, [](int j) { return j * 64 * kRowBytes; }, kKeysMax / 64, kv_stride_b, tile_at, wave, voff_kv);
    }
    if (t_lo < t_hi) {
        load_tile(t_lo, 0);
        if (F::kStages > 2) load_tile(t_lo + 1, 1);
    }
    f32x16 acc[NDB];                                      // dV^T (first waves) or dK^T
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[db][r] = 0.f;
    __builtin_amdgcn_s_waitcnt(0x0F70);                   // vmcnt(0)
    __syncthreads();
    // this wave's operand of the first product, and the columns of K that its dQ takes
    const int cb = wave % NDB, rb_dq = wave / NDB;        // block of dQ
    bf16x8 kv[NK], ktf[kKeysMax / 16];
    {
        LdsQueue lq{0};
        RowFrag f[NK];
        const uint32_t at = (uint32_t)((wave < kKeysPairs ? (F::kStages - 1) * F::kStageBytes : F::kDsOff) + 32 * pair * kRowBytes);
#pragma unroll
        for (int ks = 0; ks < NK; ++ks) lds_issue_row(lq, f[ks], (row_frag + at) ^ (uint32_t)(ks << 5), 0);
#pragma unroll
        for (int ks = 0; ks < NK; ++ks) kv[ks] = as_bf16x8(lds_wait_raw(lq, f[ks]) ^ (wave < kKeysPairs ? sign_flip : 0u));      // (only the scores see the sign)
        ColFrag c[kKeysMax / 16];
#pragma unroll
        for (int b = 0; b < kKeysMax / 16; ++b) issue_column(lq, c[b], col_frag + (uint32_t)((F::kStages - 1) * F::kStageBytes), cb, b * 16 * kRowBytes);
#pragma unroll
        for (int b = 0; b < kKeysMax / 16; ++b) ktf[b] = lds_wait(lq, c[b]);
    }
    if (t_lo < t_hi) put_stats(t_lo);
    __builtin_amdgcn_s_waitcnt(0xc07f);                   // lgkmcnt(0)
    const int my_key = 32 * pair + l32;
    const float hidden = my_key < n ? 0.f : -INFINITY;    // a key behind the last one: its scores begin, and stay, at -inf
    // this pair's P; this lane's dS, written by key and read by row
    const uint32_t p_at = lds0 + (uint32_t)(F::kDsOff + 32 * pair * F::kDsRow + 16 * lane);
    const uint32_t ds_w = lds0 + (uint32_t)(F::kDsOff + my_key * F::kDsRow + 8 * half + (F::swz(my_key) << 5));
    uint32_t ds_r[2];
#pragma unroll
    for (int hi = 0; hi < 2; ++hi) {
        const int key = 4 * half + 8 * hi + (lane16 >> 2), quarter = 2 * rb_dq + ((lane >> 4) & 1);
        ds_r[hi] = lds0 + (uint32_t)(F::kDsOff + key * F::kDsRow + ((quarter ^ F::swz(key)) << 5) + 8 * (lane16 & 3));
    }

    // (each role runs its own copy of the tile loop, so that no register has to be reconciled where their paths would join)
    auto tiles = [&](auto role_tag) {
        constexpr bool kB = decltype(role_tag)::value;
        constexpr int kAhead = 4;
        for (int t = t_lo; t < t_hi; ++t) {
            const int stage = (t - t_lo) % F::kStages, base = stage * F::kStageBytes;
            // this tile is there, and what was written behind the last barrier: at most the next one's loads are under way (stores of dQ
            // only make the wait stricter)
            __builtin_amdgcn_s_waitcnt(0x0070 | (F::kStages > 2 ? kDma & 15 : 0));
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            auto load_next = [&]() {
                load_stats(t + 1);
                load_tile(t + F::kStages - 1, stage == 0 ? F::kStages - 1 : stage - 1);
                __builtin_amdgcn_sched_barrier(0);
            };
            const uint32_t qt = (uint32_t)base, stat = lds0 + (uint32_t)(F::kStatOff + (t & 1) * 2 * kBM * 4 + 16 * half);
            f32x16 x1[kBlocks];                           // S and P, or dP
            LdsQueue lq{0};
            ColFrag cf[kAhead];
            // fragment i of the second product: (row block, 16 rows of it, column block)
            uint32_t row_at = row_frag + qt, col_at = col_frag + qt;
            auto issue_second = [&](int i) {
                const int rb = i / (2 * NDB), j = i % (2 * NDB);
                if (j == 0) asm volatile("" : "+v"(col_at));                  // (addresses of one block at a time)
                issue_column(lq, cf[i % kAhead], col_at, j % NDB + (rb >> 1) * NDB, (kB ? 0 : F::kTileBytes) + (2 * (rb & 1) + j / NDB) * 16 * kRowBytes);
            };
            {
                RowFrag f[kAhead], st[4];
                auto issue_first = [&](int i) {
                    if (i % NK == 0) asm volatile("" : "+v"(row_at));
                    lds_issue_row(lq, f[i % kAhead], row_at ^ (uint32_t)((i % NK + i / NK / 2 * NK) << 5), (kB ? F::kTileBytes : 0) + 32 * (i / NK % 2) * kRowBytes);
                };
                // statistics of a row block: -D starts dP, -LSE2 is needed when the scores are there
                auto issue_stat = [&](int rb, int rq) { lds_issue_row(lq, st[rq], stat, ((kB ? kBM : 0) + 32 * rb + 8 * rq) * 4); };
                auto form_p = [&](int rb, int rq) {
                    const u32x4 v = lds_wait_raw(lq, st[rq]);
                    u32x4 w;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x1[rb][4 * rq + e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x1[rb][4 * rq + e], scale_log2, __uint_as_float(v[e])));
                        w[e] = __float_as_uint(x1[rb][4 * rq + e]);
                    }
                    lds_store(p_at, w, F::p_off(rb) + rq * 1024);
                    ++lq.issued;
                };
#pragma unroll
                for (int rq = 0; rq < 4; ++rq) issue_stat(0, rq);
#pragma unroll
                for (int i = 0; i < kAhead; ++i) issue_first(i);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int rb = 0; rb < kBlocks; ++rb) {
                    if (kB) {
#pragma unroll
                        for (int rq = 0; rq < 4; ++rq) {
                            const u32x4 v = lds_wait_raw(lq, st[rq]);
#pragma unroll
                            for (int e = 0; e < 4; ++e) x1[rb][4 * rq + e] = __uint_as_float(v[e]);
                        }
                        if (rb + 1 < kBlocks) {
#pragma unroll
                            for (int rq = 0; rq < 4; ++rq) issue_stat(rb + 1, rq);
                        }
                    } else {
#pragma unroll
                        for (int r = 0; r < 16; ++r) x1[rb][r] = hidden;
                    }
#pragma unroll
                    for (int i = 0; i < NK; ++i) {        // (a block's probabilities are formed under the next one's scores)
                        const int m = NK * rb + i;
                        x1[rb] = mfma32(lds_wait(lq, f[m % kAhead]), kv[i], x1[rb]);
                        if (m + kAhead < kBlocks * NK) issue_first(m + kAhead);
                        __builtin_amdgcn_sched_barrier(0);
                        if (!kB && rb > 0) {
                            constexpr int kEvery = NK / 4;
                            if (i % kEvery == kEvery - 1) {
                                form_p(rb - 1, i / kEvery);
                                issue_stat(rb, i / kEvery);
                            }
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    }
                }
                if (!kB) {
#pragma unroll
                    for (int rq = 0; rq < 4; ++rq) form_p(kBlocks - 1, rq);
                }
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) issue_second(i);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_waitcnt(0xc07f | ((2 * kAhead) << 8));         // LDS operations complete in order: P is written
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            load_next();                                  // (here and not at the top: fewer registers through the first products)
            if constexpr (kB) {                           // dS in place of dP; all of P is read before dS takes its place
#pragma unroll
                for (int rb = 0; rb < kBlocks; ++rb) {
                    LdsQueue lp{0};
                    RowFrag f[4];
#pragma unroll
                    for (int rq = 0; rq < 4; ++rq) lds_issue_row(lp, f[rq], p_at, F::p_off(rb) + rq * 1024);
#pragma unroll
                    for (int rq = 0; rq < 4; ++rq) {
                        const u32x4 v = lds_wait_raw(lp, f[rq]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) x1[rb][4 * rq + e] *= __uint_as_float(v[e]);
                    }
                }
            }
            // The second product, in groups of 16 rows.  A group's operand is formed under the products of the one before it.
            uint32_t hi[2][4], lo[2][4], ds_at = ds_w;
            asm volatile("" : "+v"(ds_at));               // (the addresses that follow from it are formed here, not kept through the loop)
            auto form = [&](int q, int m) {               // pair m of group q
                const int r = 8 * (q & 1) + 2 * m;
                split_bf16(x1[q >> 1][r], x1[q >> 1][r + 1], hi[q & 1][m], lo[q & 1][m]);
                if (kB && (m & 1)) {                      // dS of rows 32 rb + 8 rq + 4 half ..
                    const int rb = q >> 1, rq = 2 * (q & 1) + (m >> 1);
                    const uint32_t at = (ds_at ^ (uint32_t)((2 * rb + (rq >> 1)) << 5)) + 16 * (rq & 1);
                    lds_store(at, u32x2{hi[q & 1][m - 1], hi[q & 1][m]});
                    lds_store(at + F::kDsBytes, u32x2{lo[q & 1][m - 1], lo[q & 1][m]});
                    lq.issued += 2;
                }
            };
            lq.issued = 2 * kAhead;                       // (the reads from before the barrier, restated; B's have been waited for)
#pragma unroll
            for (int i = 0; i < kAhead; ++i) cf[i].seq = 2 * (i + 1);
#pragma unroll
            for (int m = 0; m < 4; ++m) form(0, m);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < kBlocks * 2 * NDB; ++i) {
                const int q = i / NDB, db = i % NDB;
                const bf16x8 a = lds_wait(lq, cf[i % kAhead]);
                const uint32_t (&h)[4] = hi[q & 1], (&l)[4] = lo[q & 1];
                acc[db] = mfma32(a, as_bf16x8(u32x4{h[0], h[1], h[2], h[3]}), acc[db]);
                acc[db] = mfma32(a, as_bf16x8(u32x4{l[0], l[1], l[2], l[3]}), acc[db]);
                if (i + kAhead < kBlocks * 2 * NDB) issue_second(i + kAhead);
                constexpr int kPer = 4 / NDB;
#pragma unroll
                for (int e = 0; e < kPer; ++e)
                    if (q + 1 < 2 * kBlocks) form(q + 1, kPer * db + e);
                __builtin_amdgcn_sched_barrier(0);
            }
            __builtin_amdgcn_s_waitcnt(0xc07f);           // lgkmcnt(0): dS is written, Q and dO read
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            put_stats(t + 1);                             // (the next barrier publishes them)
            f32x16 dq;
#pragma unroll
            for (int r = 0; r < 16; ++r) dq[r] = 0.f;
            {
                constexpr int kFrags = kKeysMax / 16 * 2; // fragment m: 16 keys, hi or lo
                LdsQueue ld{0};
                ColFrag f[kAhead];
                auto issue = [&](int m) { lds_issue_col(ld, f[m % kAhead], ds_r[0], ds_r[1], (m & 1) * F::kDsBytes + (m >> 1) * 16 * F::kDsRow); };
#pragma unroll
                for (int m = 0; m < kAhead; ++m) issue(m);
#pragma unroll
                for (int m = 0; m < kFrags; ++m) {
                    dq = mfma32(ktf[m >> 1], lds_wait(ld, f[m % kAhead]), dq);
                    if (m + kAhead < kFrags) issue(m + kAhead);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            // through this wave's part of the stage (its Q and dO have been read), then 64 bytes of each row
            const KeysRows w = tile_rows(t);
            const uint32_t out = lds0 + (uint32_t)(base + wave * 32 * kKeysOutRow);
            int ln = lane;
            asm volatile("" : "+v"(ln));                  // (likewise)
#pragma unroll
            for (int rq = 0; rq < 4; ++rq)
                lds_store(out + (uint32_t)((ln & 31) * kKeysOutRow + (8 * rq + 4 * (ln >> 5)) * 2),
                          u32x2{pack_bf16(dq[4 * rq] * p.scale, dq[4 * rq + 1] * p.scale), pack_bf16(dq[4 * rq + 2] * p.scale, dq[4 * rq + 3] * p.scale)});
            __builtin_amdgcn_s_waitcnt(0xc07f);
            {
                LdsQueue ld{0};
                RowFrag f[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) lds_issue_row(ld, f[i], out + (uint32_t)((ln >> 2) * kKeysOutRow + (ln & 3) * 16), 16 * i * kKeysOutRow);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const u32x4 v = lds_wait_raw(ld, f[i]);
                    const int r = 32 * rb_dq + 16 * i + (ln >> 2);
                    int token, head;
                    cr.split(w.rem + r, token, head);
                    if (r < w.rows)
                        *reinterpret_cast<u32x4*>(p.dq + (int64_t)(w.t0 + token) * q_stride + (int64_t)(g * G + head) * D + 32 * cb + 8 * (ln & 3)) = v;
                }
            }
        }
    };
    if (wave >= kKeysPairs) tiles(std::true_type{});
    else tiles(std::false_type{});
    __syncthreads();                                      // every wave is done with the ring
    if (32 * pair < n) {
        const uint32_t o_stage = lds0 + (uint32_t)(wave * 32 * kRowBytes);
        const int64_t at = kv_at + (int64_t)(32 * pair) * kv_stride;
        const bool is_k = wave >= kKeysPairs;
        const float mul = is_k ? p.scale : 1.f;
        if (p.parts == 1) store_rows_via_lds<D>((is_k ? p.dk : p.dv) + at, kv_stride, n - 32 * pair, acc, mul, o_stage, lane);
        else store_rows_f32_via_lds<D>(p.part + ((is_k ? 0 : p.parts) + part) * (int64_t)p.c.Tk * kv_stride + at, kv_stride, n - 32 * pair, acc, mul, o_stage, lane);
    }
}

}  // namespace hyd
