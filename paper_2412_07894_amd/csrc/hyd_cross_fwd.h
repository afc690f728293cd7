// Cross attention, forward in bf16: the tile form, for long query sequences, and the form for few rows.
//
// Arithmetic, orientation and the reference of a row are the self-attention forward's (hyd_fwd_bf16.h, whose tile body this runs); O
// is divided by, and LSE taken from, the sum of the probabilities in fp32 as they are, before they are rounded for the second
// product.  Only the last key tile of a sequence is masked, behind its last key; rows behind a sequence's valid keys are never read
// (buffer loads past the last one return zeros), whatever a padded cache holds there.
#pragma once
#include "hyd_cross.h"
#include "hyd_fwd_bf16.h"

namespace hyd {

struct CrossFwdParams {
    CrossShape c;
    const uint16_t* q; const uint16_t* k; const uint16_t* v;
    uint16_t* o; float* lse;
    float scale_log2;
    const int* hdr; int* cursors; const int* items;      // the list of query tiles
    HeadMap hm;
    int parts, tiles;                 // parts of the keys; own items: query tiles of a sequence at most
    float* part_o; float* part_lse;   // parts > 1: what hyd_cross_join_kernel reads
};

// fp32 rows for the join, straight from the accumulators.
template <int D>
__device__ __forceinline__ void cross_store_part(float* row, const f32x16 (&acc)[D / 32], float mul, int half) {
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int rq = 0; rq < 4; ++rq)
            *reinterpret_cast<f32x4*>(row + 32 * db + 8 * rq + 4 * half) =
                f32x4{acc[db][4 * rq] * mul, acc[db][4 * rq + 1] * mul, acc[db][4 * rq + 2] * mul, acc[db][4 * rq + 3] * mul};
}

// Work item = (256 packed rows of a sequence and KV head, a part of its keys); 8 waves of 32 rows, K/V tiles of 64 keys through a ring
// of three stages that all waves share.  kSelf: one item per workgroup, its sequence and tile from the workgroup's number (launches
// whose items all fit on the chip, which are too short to wait for a list).
//
// P is rounded to bf16 for the second product, off by 2^-8 of itself at most: O is off by about sqrt(2) of what its own rounding
// costs (2.3e-3 of its norm).  A second bf16 number for what the rounding leaves would double the second product.
//
// Bound by the matrix pipe where rows are many: 6 sequences of 1500 to 6000 queries and 4000 to 12000 keys, 32/8 heads, d = 128, 2.22 to
// 2.3 ms, 1.15 to 1.19 PFLOP/s (a large bf16 matrix product reaches 1.37), the pipe busy for 60 % of the clocks and the vector ALU for
// 47.  Short items wait for their first tiles and for their stores: 24 sequences of up to 448 queries and 1500 keys, 20 heads, d = 64, 59 us with
// the 5 of the list in front (pipe 19 %, vector ALU 41 %, 2.9 TB/s).
//
// NW = 4: 128 rows, two stages, and two workgroups to a CU, one of which streams while the other begins or ends; for sequences that
// have no more rows.  NW = 8 and 4 with 24 sequences of 1536 keys, 20 heads: 64 queries 52 and 36 us (d = 64), 85 and 79 (128); 128 queries
// 55 and 38, 91 and 86; 256 queries 73 and 78, 117 and 132.
template <int NW>
struct CrossFwd {
    static constexpr int kBM = 32 * NW, kThreads = 64 * NW, kPerCu = 8 / NW;
    static constexpr int kStages = NW == 8 ? kFwdStages : 2;
    static constexpr int kSlotOff = NW == 8 ? kFwdSlotOff : kStages * kFwdStageBytes, kLds = kSlotOff + 128;
    // where the Q rows of a tile wait, by 64 rows: in what is not a K or V tile's yet
    __device__ __forceinline__ static constexpr int q_stage(int j) { return NW == 8 ? fwd_q_stage_off(j) : kFwdStageBytes + j * kFwdTileBytes; }
};
static_assert(CrossFwd<8>::kLds == kFwdLds && CrossFwd<8>::kBM == kFwdBM && kFwdStages == 3, "the tile form of the self-attention forward");

template <int D, bool kSelf, int NW>
__global__ void __launch_bounds__(CrossFwd<NW>::kThreads, CrossFwd<NW>::kPerCu) hyd_cross_fwd_bf16_kernel(CrossFwdParams p) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    using F = CrossFwd<NW>;
    constexpr int kRowB = D * 2, kAhead = F::kStages - 1;             // tiles under way
    int* slot = reinterpret_cast<int*>(smem + F::kSlotOff);
    volatile int* redo = slot + 16;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, half = lane >> 5;
    const int G = p.c.G;
    const int64_t q_stride = (int64_t)p.c.hq * D, kv_stride = (int64_t)p.c.hkv * D;
    const uint32_t kv_stride_b = (uint32_t)kv_stride * 2, q_stride_b = (uint32_t)q_stride * 2;
    FragAddr fa;
    fa.init(lane, smem);
    CrossRows cr;
    cr.init(G);
    const uint32_t dma_voff = dma_lane_voff<D>(4 * wave + (lane >> 4), lane, kv_stride_b);
    const uint32_t tile_bytes = kFwdBN * kv_stride_b;
    const int q_stage = F::q_stage(wave >> 1) + (wave & 1) * 32 * kRowBytes;
    const uint32_t o_stage = (uint32_t)(uintptr_t)(lds_char*)smem + (uint32_t)(wave * 32 * kRowBytes);
    const float scale_log2 = fmaxf(fabsf(p.scale_log2), 1e-30f);
    const uint32_t sign_flip = p.scale_log2 < 0.f ? 0x80008000u : 0u;

    WorkFetcher wf;
    WorkItem wi;                          // see CrossList for what its record holds
    bool have;
    if constexpr (kSelf) {
        int b = blockIdx.x;
        wi.head = b % p.c.hkv; b /= p.c.hkv;
        const int part = b % p.parts; b /= p.parts;
        const int tile = b % p.tiles;
        const CrossSeq x = cross_seq(p.c, b / p.tiles);
        const int left = x.lq * G - tile * F::kBM;
        wi.seq = x.q0 * G + tile * F::kBM; wi.lev = min(left, F::kBM) | (part << kCrossPartShift); wi.row0 = x.k0; wi.len = x.n;
        have = left > 0;
    } else {
        have = wf.first(p.hm, p.hdr, p.cursors, p.items, slot, wi, blockIdx.x);
    }
    while (have) {
        const int g = wi.head, R = wi.seq, rows = wi.lev & ((1 << kCrossPartShift) - 1), part = wi.lev >> kCrossPartShift;
        const int t0 = R / G, rem = R - t0 * G;           // token of the first row, its head in the group
        const int n_all = (wi.len + kFwdBN - 1) / kFwdBN;
        const int t_lo = (int)((long long)n_all * part / p.parts), n_kt = (int)((long long)n_all * (part + 1) / p.parts);      // key tiles
        const int n_keys = min(wi.len, n_kt * kFwdBN);
        const int wrow0 = 32 * wave, row = wrow0 + l32;
        const bool active = wrow0 < rows, valid = row < rows;
        const auto q_at = [&](int r) -> int64_t {         // element offset of row r of the tile in Q and O
            int token, head;
            cr.split(rem + r, token, head);
            return (int64_t)(t0 + token) * q_stride + (int64_t)(g * G + head) * D;
        };
        const auto lse_at = [&](int r) -> int64_t {
            int token, head;
            cr.split(rem + r, token, head);
            return (int64_t)(g * G + head) * p.c.Tq + t0 + token;
        };
        if (t_lo == n_kt) {                               // no keys: O = 0, LSE = -inf
            if (valid && half == 0) (p.parts > 1 ? p.part_lse + (int64_t)part * p.c.hq * p.c.Tq : p.lse)[lse_at(row)] = -INFINITY;
            if (valid && p.parts == 1) {
                uint16_t* op = p.o + q_at(row) + 4 * half;
#pragma unroll
                for (int i = 0; i < D / 8; ++i) *reinterpret_cast<u32x2*>(op + 8 * i) = u32x2{0u, 0u};
            }
            if constexpr (kSelf) have = false;
            else have = wf.next(p.hm, p.cursors, p.items, slot, wi);
            continue;
        }
        const uint32_t kv_bytes = (uint32_t)(n_keys - 1) * kv_stride_b + kRowB;
        const __amdgpu_buffer_rsrc_t rk = make_rsrc(p.k + (int64_t)wi.row0 * kv_stride + (int64_t)g * D, kv_bytes);
        const __amdgpu_buffer_rsrc_t rv = make_rsrc(p.v + (int64_t)wi.row0 * kv_stride + (int64_t)g * D, kv_bytes);
        auto dma_tile = [&](int t, int stage) {
            char* dst = smem + stage * kFwdStageBytes + 4 * wave * kRowBytes;
#pragma unroll
            for (int j = 0; j < 16 / NW; ++j) {
                const uint32_t soff = (uint32_t)t * tile_bytes + (uint32_t)(j * NW * 4) * kv_stride_b;
                char* d = dst + j * NW * 4 * kRowBytes;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rk, (lds_void*)d, 16, dma_voff, soff, 0, 0);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rv, (lds_void*)(d + kFwdTileBytes), 16, dma_voff, soff, 0, 0);
            }
        };
        const auto dma_first = [&]() {
            dma_tile(t_lo, 0);
            if (kAhead > 1 && t_lo + 1 < n_kt) dma_tile(t_lo + 1, 1);
        };
        dma_first();
        {
            const uint32_t q_bytes = (uint32_t)((rem + rows - 1) / G) * q_stride_b + (uint32_t)G * kRowB;
            dma_packed_rows<NW, D>(make_rsrc(p.q + (int64_t)t0 * q_stride + (int64_t)g * G * D, q_bytes), smem,
                                          [](int j) { return F::q_stage(j); }, (rows + 63) / 64, cr, rem, rows, q_stride_b, wave, lane);
        }
        if (tid == 0) *redo = 0;
        __syncthreads();                                  // the first tiles and the Q rows have landed
        bf16x8 qf[D / 16];
        {
            u32x4 qv[D / 16];
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) qv[ks] = *(lds_u32x4*)(uintptr_t)(fa.row[ks] + (uint32_t)q_stage);
            __builtin_amdgcn_s_waitcnt(0xc07f);           // lgkmcnt(0)
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                asm volatile("" : "+v"(qv[ks]));          // the reads stay on this side of the barrier
                qf[ks] = as_bf16x8(qv[ks] ^ sign_flip);
            }
        }
        __builtin_amdgcn_s_barrier();                     // the staged Q may be overwritten (the next tile goes there)
        const bool short_item = n_kt - t_lo <= kShortItem;
        if (!kSelf && short_item) wf.claim(p.hm, p.cursors);
        // the tile that is masked (see fwd_tile), in a vector register: as a scalar it has the accumulators copied in every tile
        int td = wi.len < n_kt * kFwdBN ? n_kt - 1 : INT_MAX;
        asm volatile("" : "+v"(td));
        const int koff0 = 4 * half - (wi.len - 1);

        f32x16 acc_o[D / 32];
        float m_ref, l_run;
        bool overflow = false;
        int t_find = t_lo;
        while (true) {
            m_ref = -INFINITY;
            l_run = 0.f;
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc_o[db][r] = 0.f;
            auto step = [&](auto stage_tag, int t) {
                constexpr int ST = decltype(stage_tag)::value;
                constexpr int Kt = ST * kFwdStageBytes, Vt = Kt + kFwdTileBytes, ST2 = (ST + kAhead) % F::kStages;
                constexpr int kDmaBehind = (kAhead - 1) * 2 * (16 / NW);      // loads of the tiles behind the next one
                const bool more = t + kAhead < n_kt;
                if (more) dma_tile(t + kAhead, ST2);
                if (active)
                    fwd_tile<D, true>(Kt, Vt, fa, qf, acc_o, m_ref, l_run, scale_log2, t * kFwdBN + koff0, t == td, t, t_find, overflow);
                if (more) __builtin_amdgcn_s_waitcnt(0x0070 | (kDmaBehind & 15));       // vmcnt(kDmaBehind), lgkmcnt(0)
                else __builtin_amdgcn_s_waitcnt(0x0070);                                // vmcnt(0), lgkmcnt(0)
                __builtin_amdgcn_s_barrier();
            };
            for (int t = t_lo; t < n_kt; t += F::kStages) {
                step(std::integral_constant<int, 0>{}, t);
                if (t + 1 < n_kt) step(std::integral_constant<int, 1>{}, t + 1);
                if (F::kStages > 2 && t + 2 < n_kt) step(std::integral_constant<int, 2 % F::kStages>{}, t + 2);
            }
            if (__any(l_run > kRefQuiet)) overflow |= largest_bits(acc_o) >= kInfBits;
            if (t_find == t_lo && __any(overflow)) *redo = 1;
            __syncthreads();
            if (__builtin_expect(*redo == 0, 1)) break;
            t_find = INT_MAX;
            __syncthreads();
            if (tid == 0) *redo = 0;
            dma_first();
            __syncthreads();
        }
        if (!kSelf && !short_item) wf.claim(p.hm, p.cursors);
        float l_lo, l_hi;
        both_halves(l_run, l_lo, l_hi);
        const float l_tot = l_lo + l_hi, inv = 1.f / l_tot, log2_sum = m_ref + __builtin_amdgcn_logf(l_tot);
        if (active) {
            if (p.parts == 1) {
                store_packed_rows<D>([&](int r) { return p.o + q_at(wrow0 + r); }, rows - wrow0, acc_o, inv, o_stage, lane);
                if (valid && half == 0) p.lse[lse_at(row)] = log2_sum * 0.69314718055994530942f;
            } else if (valid) {
                const int64_t plane = (int64_t)part * p.c.hq * p.c.Tq;
                cross_store_part<D>(p.part_o + plane * D + q_at(row), acc_o, inv, half);
                if (half == 0) p.part_lse[plane + lse_at(row)] = log2_sum;
            }
        }
        if constexpr (kSelf) have = false;
        else have = wf.next(p.hm, p.cursors, p.items, slot, wi);
    }
}

// ---------------------------------------------------------------------------------------------
// Few rows: at most 32 packed rows of a (sequence, KV head), as when a model writes one token after the other.  Bound by HBM: K and V
// are read once and 32 rows cost the matrix pipe the same as one.  So the keys are spread: over workgroups in parts of `chunk` keys,
// inside one over its 4 waves in turns of 32 keys, and each wave streams its own keys through its own 16 KB of LDS (K and V, 32
// rows each) without meeting the others: K of its next turn is requested as soon as the scores are formed, V as soon as
// the second product is done, so that 64 to 128 KB are under way per CU.  The waves' results meet in LDS once, the parts' by
// hyd_cross_join_kernel.  Two workgroups share a CU, so that one streams while the other begins or ends: with one of 8 waves 64 tokens
// of 32/8 heads, d = 128, against 500 to 8192 keys took 258 us, so 222 (1.13 GB, 5.1 TB/s); 16 against 30000 keys 359 us
// (5.5 TB/s).  The smallest calls, 11 us, are two launches: 4 tokens of 20 heads, d = 64, against 1500 keys 8.8 us in 240 workgroups
// (30.7 MB, 3.5 TB/s) and 3.6 us for the join.
//
// P is rounded to bf16 as in the tile form.  With what the rounding leaves as a second bf16 number, large calls take what they took, but
// small ones 5 % more (11.1 for 10.6 us, 8.8 for 8.3, 12.4 for 11.8), so it is one number here too.
// ---------------------------------------------------------------------------------------------
constexpr int kFewRows = 32, kFewKeys = 32, kFewWaves = 4, kFewThreads = 64 * kFewWaves;
constexpr int kFewTileBytes = kFewKeys * kRowBytes;                   // 8 KB
constexpr int kFewWaveBytes = 2 * kFewTileBytes;                      // K, V; later the wave's sums
constexpr int kFewMlOff = kFewWaves * kFewWaveBytes;                  // [wave][m, l][32 rows]
constexpr int kFewLds = kFewMlOff + kFewWaves * 2 * kFewRows * 4;
struct CrossFewParams {
    CrossShape c;
    const uint16_t* q; const uint16_t* k; const uint16_t* v;
    uint16_t* o; float* lse;
    float scale_log2;
    int chunk, parts;                 // keys of a part, a multiple of kFewWaves * kFewKeys unless parts = 1
    float* part_o; float* part_lse;
};

template <int D>
__global__ void __launch_bounds__(kFewThreads, 2) hyd_cross_few_bf16_kernel(CrossFewParams p) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
    constexpr int kRowB = D * 2, NK = D / 16, NDB = D / 32;
    static_assert(kFewRows * kHeadDim * 4 <= kFewWaveBytes, "a wave's sums take the place of its tiles");
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, half = lane >> 5;
    const int g = blockIdx.x % p.c.hkv, part = (blockIdx.x / p.c.hkv) % p.parts, seq = blockIdx.x / p.c.hkv / p.parts;
    const CrossSeq x = cross_seq(p.c, seq);
    const int G = p.c.G, rows = min(x.lq * G, kFewRows);
    if (rows == 0) return;
    const int64_t q_stride = (int64_t)p.c.hq * D, kv_stride = (int64_t)p.c.hkv * D;
    const uint32_t kv_stride_b = (uint32_t)kv_stride * 2, q_stride_b = (uint32_t)q_stride * 2;
    CrossRows cr;
    cr.init(G);
    const auto q_at = [&](int r) -> int64_t {
        int token, head;
        cr.split(r, token, head);
        return (int64_t)(x.q0 + token) * q_stride + (int64_t)(g * G + head) * D;
    };
    const auto lse_at = [&](int r) -> int64_t {
        int token, head;
        cr.split(r, token, head);
        return (int64_t)(g * G + head) * p.c.Tq + x.q0 + token;
    };
    const int64_t plane = (int64_t)part * p.c.hq * p.c.Tq;
    const int first = min((long long)part * p.chunk, (long long)x.n), last = min((long long)first + p.chunk, (long long)x.n);
    if (first == last && p.parts > 1) {                  // a part without keys
        if (tid < rows) p.part_lse[plane + lse_at(tid)] = -INFINITY;
        return;
    }
    FragAddr fa;
    fa.init(lane, smem + wave * kFewWaveBytes);
    const float scale_log2 = fmaxf(fabsf(p.scale_log2), 1e-30f);
    const uint32_t sign_flip = p.scale_log2 < 0.f ? 0x80008000u : 0u;

    // keys of this wave's turn t: first + (4 t + wave) * 32 + 0..31; reads past `last` return zero
    const int n_turns = max((last - first - wave * kFewKeys + kFewWaves * kFewKeys - 1) / (kFewWaves * kFewKeys), 0);
    const uint32_t kv_bytes = last > first ? (uint32_t)(last - first - 1) * kv_stride_b + kRowB : 0;
    const int64_t kv_off = (int64_t)(x.k0 + first) * kv_stride + (int64_t)g * D;
    const __amdgpu_buffer_rsrc_t rk = make_rsrc(p.k + kv_off, kv_bytes), rv = make_rsrc(p.v + kv_off, kv_bytes);
    // instruction j loads rows 4 j .. 4 j + 3; swz of a row repeats every 16 rows, so four offsets serve eight instructions
    uint32_t voff[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) voff[j] = dma_lane_voff<D>(4 * j + (lane >> 4), lane, kv_stride_b);
    char* const mine = smem + wave * kFewWaveBytes;
    auto load = [&](const __amdgpu_buffer_rsrc_t& rs, char* dst, int t) {
        const uint32_t soff = (uint32_t)((t * kFewWaves + wave) * kFewKeys) * kv_stride_b;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void*)(dst + 4 * j * kRowBytes), 16, voff[j & 3], soff + (uint32_t)(j >> 2) * 16 * kv_stride_b, 0, 0);
    };
    bf16x8 qf[NK];
    {
        const uint32_t q_bytes = (uint32_t)(x.lq - 1) * q_stride_b + (uint32_t)G * kRowB;
        const __amdgpu_buffer_rsrc_t rq = make_rsrc(p.q + (int64_t)x.q0 * q_stride + (int64_t)g * G * D, q_bytes);
        int token, head;
        cr.split(l32, token, head);
        const uint32_t at = l32 < rows ? (uint32_t)token * q_stride_b + (uint32_t)(head * kRowB + 16 * half) : kDmaOutOfRange;
        u32x4 qv[NK];
#pragma unroll
        for (int ks = 0; ks < NK; ++ks) qv[ks] = __builtin_amdgcn_raw_buffer_load_b128(rq, at, 32 * ks, 0);
#pragma unroll
        for (int ks = 0; ks < NK; ++ks) qf[ks] = as_bf16x8(qv[ks] ^ sign_flip);
    }
    if (n_turns > 0) {
        load(rk, mine, 0);
        load(rv, mine + kFewTileBytes, 0);
    }
    f32x16 acc[NDB];
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[db][r] = 0.f;
    float m = -INFINITY, l = 0.f;                         // l: this half's keys only
    for (int t = 0; t < n_turns; ++t) {
        const bool more = t + 1 < n_turns;
        // K of this turn is there once at most V's 8 loads are under way
        asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
        f32x16 s;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = 0.f;
        {
            LdsQueue lq{0};
            RowFrag kf[NK];
#pragma unroll
            for (int i = 0; i < NK; ++i) issue_row(lq, kf[i], 0, fa, 0, i);
#pragma unroll
            for (int i = 0; i < NK; ++i) s = mfma32(lds_wait(lq, kf[i]), qf[i], s);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");            // K has been read
        if (more) load(rk, mine, t + 1);
        const int key = first + (t * kFewWaves + wave) * kFewKeys + 4 * half;
        if (key - 4 * half + kFewKeys > last) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (key + 8 * (r >> 2) + (r & 3) >= last) s[r] = -INFINITY;
        }
        float mx = s[0], lo, hi;
#pragma unroll
        for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
        both_halves(mx, lo, hi);
        const float m_new = fmaxf(m, fmaxf(lo, hi) * scale_log2);
        if (__any(m_new > m)) {
            const float alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - m_new);
            l *= alpha;
#pragma unroll
            for (int db = 0; db < NDB; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[db][r] *= alpha;
            m = m_new;
        }
        u32x4 pk[2];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * j], scale_log2, -m));
            const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * j + 1], scale_log2, -m));
            l += p0 + p1;
            pk[j >> 2][j & 3] = pack_bf16(p0, p1);
        }
        if (more) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");      // V is there once at most the next K is under way
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        {
            LdsQueue lq{0};
            ColFrag vf[2 * NDB];
#pragma unroll
            for (int i = 0; i < 2 * NDB; ++i) issue_col(lq, vf[i], kFewTileBytes, fa, i / NDB, i % NDB);
#pragma unroll
            for (int i = 0; i < 2 * NDB; ++i) acc[i % NDB] = mfma32(lds_wait(lq, vf[i]), as_bf16x8(pk[i / NDB]), acc[i % NDB]);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (more) load(rv, mine + kFewTileBytes, t + 1);
    }
    {
        float lo, hi;
        both_halves(l, lo, hi);
        l = lo + hi;
    }
    // The waves' sums: (m, l) of all rows, then the accumulators times 2^(m - largest m), row r chunk c (16 bytes) at c ^ (r & 15).
    float* ml = reinterpret_cast<float*>(smem + kFewMlOff);
    if (half == 0) {
        ml[wave * 2 * kFewRows + l32] = m;
        ml[wave * 2 * kFewRows + kFewRows + l32] = l;
    }
    __syncthreads();
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) top = fmaxf(top, ml[w * 2 * kFewRows + l32]);
    const float w_mine = l == 0.f ? 0.f : __builtin_amdgcn_exp2f(m - top);      // (l = 0: no keys; m = -inf alone may be a row of nan)
    const uint32_t sums = (uint32_t)(uintptr_t)(lds_char*)smem;
    if (l32 < rows) {
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
            for (int rq = 0; rq < 4; ++rq)
                *(lds_f32x4*)(uintptr_t)(sums + (uint32_t)(wave * kFewWaveBytes + l32 * D * 4 + (((8 * db + 2 * rq + half) ^ (l32 & 15)) << 4))) =
                    f32x4{acc[db][4 * rq] * w_mine, acc[db][4 * rq + 1] * w_mine, acc[db][4 * rq + 2] * w_mine, acc[db][4 * rq + 3] * w_mine};
    }
    __syncthreads();
    constexpr int kLanes = D / 4;
    for (int e = tid; e < rows * kLanes; e += kFewThreads) {
        const int r = e / kLanes, c = e % kLanes;
        float mt = -INFINITY, lt = 0.f;
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) mt = fmaxf(mt, ml[w * 2 * kFewRows + r]);
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) {
            const float lw = ml[w * 2 * kFewRows + kFewRows + r];
            lt += lw == 0.f ? 0.f : lw * __builtin_amdgcn_exp2f(ml[w * 2 * kFewRows + r] - mt);
            sum += *(lds_f32x4*)(uintptr_t)(sums + (uint32_t)(w * kFewWaveBytes + r * D * 4 + ((c ^ (r & 15)) << 4)));
        }
        const float inv = lt == 0.f ? 0.f : 1.f / lt, log2_sum = lt == 0.f ? -INFINITY : mt + __builtin_amdgcn_logf(lt);
        sum *= inv;
        if (p.parts == 1) {
            *reinterpret_cast<u32x2*>(p.o + q_at(r) + 4 * c) = u32x2{pack_bf16(sum[0], sum[1]), pack_bf16(sum[2], sum[3])};
            if (c == 0) p.lse[lse_at(r)] = log2_sum * 0.69314718055994530942f;
        } else {
            *reinterpret_cast<f32x4*>(p.part_o + plane * D + q_at(r) + 4 * c) = sum;
            if (c == 0) p.part_lse[plane + lse_at(r)] = log2_sum;
        }
    }
}

}  // namespace hyd
