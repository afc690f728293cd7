// Cross attention of packed batches: what its kernels share.
//
// The queries of sequence s are rows of one packed buffer, its keys rows of another; every query sees all valid keys.  Without
// a mask between rows and keys the query heads of a KV head are just more rows: packed row r of (sequence, KV head g) is
// query head g G + r % G of token r / G, so that a tile of rows holds queries of all G heads, K and V are read once for
// them, and short query sequences fill tiles.  In Q, O, dO and dQ the rows of a token's group lie side by side; the backward's own
// copies are [Hkv][Tq G][d], in which packed rows simply follow each other.
#pragma once
#include "hyd_sched.h"

namespace hyd {

struct CrossShape {
    const int32_t* cu_q; const int32_t* cu_kv; const int32_t* kv_lens;      // kv_lens may be NULL
    int nseq, Tq, Tk, max_q, max_kv;
    int hq, hkv, G;
};

// A sequence: first token and number of tokens of its queries; first row, valid rows and all rows of its keys.  Whatever the arrays
// hold, the rows lie inside the buffers and within the bounds.
struct CrossSeq { int q0, lq, k0, n, rows; };
__device__ __forceinline__ CrossSeq cross_seq(const CrossShape& c, int s) {
    CrossSeq x;
    const int qa = c.cu_q[s], qb = c.cu_q[s + 1], ka = c.cu_kv[s], kb = c.cu_kv[s + 1];
    const int valid = c.kv_lens ? c.kv_lens[s] : 0x7fffffff;
    x.q0 = min(max(qa, 0), c.Tq);
    x.lq = min(max(min(qb, c.Tq) - x.q0, 0), c.max_q);
    x.k0 = min(max(ka, 0), c.Tk);
    x.rows = max(min(kb, c.Tk) - x.k0, 0);
    x.n = min(min(max(valid, 0), x.rows), c.max_kv);
    return x;
}

// ---- zeros behind the valid keys, by n workgroups of which so many share a sequence
struct CrossZero { int n, per_seq; };
inline CrossZero cross_zero(int nseq, bool padded) {
    constexpr int kZeroWg = 256;
    if (!padded) return CrossZero{0, 1};
    return nseq < kZeroWg ? CrossZero{kZeroWg / nseq * nseq, kZeroWg / nseq} : CrossZero{kZeroWg, 1};
}
// E: 16 bytes of an element type, kPer elements; row: elements of a key row
template <typename E, int kPer, typename T>
__device__ __forceinline__ void cross_clear(const CrossShape& c, const CrossZero& z, int wg, int nthreads, int64_t row, T* dk, T* dv) {
    for (int s = wg / z.per_seq; s < c.nseq; s += z.n / z.per_seq) {
        const CrossSeq x = cross_seq(c, s);
        const int64_t last = (int64_t)(x.k0 + x.rows) * row / kPer;
        for (int64_t i = (int64_t)(x.k0 + x.n) * row / kPer + (wg % z.per_seq) * nthreads + threadIdx.x; i < last; i += (int64_t)z.per_seq * nthreads) {
            *reinterpret_cast<E*>(dk + kPer * i) = E{};
            *reinterpret_cast<E*>(dv + kPer * i) = E{};
        }
    }
}

// ---- item lists (WorkFetcher hands them out).  A record names a tile by rows, so that nothing has to be looked up:
//   queries: {first packed row (over all sequences), rows | part << 16, first key row, keys}
//   keys:    {first key row, keys | part << 16, first packed row, packed rows}
// in order of decreasing cost, which is the length of the other side.
struct CrossList {
    int* hdr; int* items;
    int tile, parts, max_items;           // rows of a tile; parts of an item; records at most
    bool keys;                            // the list of key tiles
};
// Classes of cost: exact up to 255 tiles, then 32 to an octave; the largest first.
constexpr int kCrossClasses = 1024;
__device__ __forceinline__ int cross_class(int tiles) {
    if (tiles < 256) return kCrossClasses - 1 - tiles;
    const int e = 31 - __clz(tiles);
    return kCrossClasses - 1 - min(256 + (e - 8) * 32 + ((tiles >> (e - 5)) & 31), kCrossClasses - 1);
}
constexpr int kCrossListLds = sizeof(int) * kCrossClasses;
// Called by all threads of a workgroup (a multiple of 64), with kCrossListLds bytes of LDS.
__device__ __forceinline__ void cross_build_list(const CrossShape& c, const CrossList& l, int* lds, int nthreads) {
    const int tid = threadIdx.x, lane = tid & 63;
    for (int i = tid; i < kCrossClasses; i += nthreads) lds[i] = 0;
    for (int i = tid; i < kHdrTotal; i += nthreads) l.hdr[i] = 0;
    __syncthreads();
    const auto item = [&](const CrossSeq& x, int& count, int& cls) {
        const int mine = l.keys ? x.n : x.lq * c.G, other = l.keys ? x.lq * c.G : x.n;
        count = (mine + l.tile - 1) / l.tile * l.parts;
        cls = cross_class((other + 63) / 64);
    };
    for (int s = tid; s < c.nseq; s += nthreads) {
        int count, cls;
        item(cross_seq(c, s), count, cls);
        if (count > 0) atomicAdd(&lds[cls], count);
    }
    __syncthreads();
    if (tid < 64) wave_inclusive_scan(lds, kCrossClasses, lane);
    __syncthreads();
    const int n_items = min(lds[kCrossClasses - 1], l.max_items);
    __syncthreads();
    if (tid == 0) { l.hdr[0] = n_items; l.hdr[kHdrExec] = n_items; }
    // a class fills its range from the end
    for (int s0 = tid - lane; s0 < c.nseq; s0 += nthreads) {
        const int s = s0 + lane;
        CrossSeq x = {0, 0, 0, 0, 0};
        int count = 0, cls = 0, at = 0;
        if (s < c.nseq) {
            x = cross_seq(c, s);
            item(x, count, cls);
            if (count > 0) at = atomicSub(&lds[cls], count) - count;
        }
        const int first = l.keys ? x.k0 : x.q0 * c.G, mine = l.keys ? x.n : x.lq * c.G;
        const int other0 = l.keys ? x.q0 * c.G : x.k0, other = l.keys ? x.lq * c.G : x.n;
        const auto put = [&](int f, int m, int o0, int o, int a, int i) {
            const int tile = i / l.parts, part = i - tile * l.parts;
            const i32x4 rec = {f + tile * l.tile, min(m - tile * l.tile, l.tile) | (part << kCrossPartShift), o0, o};
            if ((unsigned)(a + i) < (unsigned)l.max_items) *reinterpret_cast<i32x4*>(l.items + 4 * (size_t)(a + i)) = rec;
        };
        constexpr int kFew = 4;           // sequences of more items: by the whole wave
        if (count <= kFew)
            for (int i = 0; i < count; ++i) put(first, mine, other0, other, at, i);
        for (unsigned long long big = __ballot(count > kFew); big; big &= big - 1) {
            const int src = __ffsll((long long)big) - 1;
            const int f = __shfl(first, src, 64), m = __shfl(mine, src, 64), o0 = __shfl(other0, src, 64), o = __shfl(other, src, 64);
            const int a = __shfl(at, src, 64), n = __shfl(count, src, 64);
            for (int i = lane; i < n; i += 64) put(f, m, o0, o, a, i);
        }
    }
}

__global__ void __launch_bounds__(kPreludeThreads) hyd_cross_list_kernel(CrossShape c, CrossList l) {
    extern __shared__ int lds_classes[];
    cross_build_list(c, l, lds_classes, kPreludeThreads);
}

// ---- packed rows in the caller's layout
//
// Rows `rem` + 0, 1, ... counted from head 0 of a group: token and head of the group.  Row numbers stay below 256 + G, where the
// product with 1 / G truncates to the quotient.
struct CrossRows {
    int G;
    float inv;
    __device__ __forceinline__ void init(int g) { G = g; inv = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(1.f / (float)g))); }
    __device__ __forceinline__ void split(int r, int& token, int& head) const {
        token = (int)(((float)r + 0.5f) * inv);
        head = r - token * G;
    }
};

typedef __attribute__((address_space(3))) void lds_void_c;

// Direct-to-LDS load of `n64` x 64 packed rows starting at row `rem` of the group (rows from `rows` on read as zeros), LDS tile j at
// lds + off(j), in the swizzled layout; see dma_rows.
template <int NW, int D, typename OffFn>
__device__ __forceinline__ void dma_packed_rows(const __amdgpu_buffer_rsrc_t& rs, char* lds, OffFn off, int n64, const CrossRows& cr, int rem,
                                                int rows, uint32_t token_stride_b, int wave, int lane) {
    asm volatile("" : "+v"(lane));       // addresses are formed here, not hoisted
    const int row = 4 * wave + (lane >> 4), chunk = (lane & 15) ^ swz(row);
#pragma unroll
    for (int sub = 0; sub < 4; ++sub) {
        if (sub < n64) {
#pragma unroll
            for (int j = 0; j < 16 / NW; ++j) {
                const int r = 64 * sub + 4 * NW * j + row;
                int token, head;
                cr.split(rem + r, token, head);
                const uint32_t voff = r < rows && (D == kHeadDim || chunk < D / 8) ? (uint32_t)token * token_stride_b + (uint32_t)(head * D * 2 + (chunk << 4)) : kDmaOutOfRange;
                char* d = lds + off(sub) + (4 * wave + j * NW * 4) * kRowBytes;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void_c*)d, 16, voff, 0, 0, 0);
            }
        }
    }
}

// Transposed accumulators of a wave (lane: one row) as 32 bf16 rows through 8 KB of LDS: store_rows_via_lds with an address per row.
// at(r): where row r of the wave begins; only rows below `rows` are asked for and written.
template <int D, typename AtFn>
__device__ __forceinline__ void store_packed_rows(AtFn at, int rows, const f32x16 (&acc)[D / 32], float mul, uint32_t stage, int lane) {
    asm volatile("" : "+v"(lane));
    const int l32 = lane & 31, half = lane >> 5, c16 = lane & 15, r4 = lane >> 4;
    const uint32_t wbase = stage + (uint32_t)(l32 * kRowBytes + 8 * half);
    const int wswz = swz(l32);
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
#pragma unroll
        for (int rq = 0; rq < 4; ++rq) {
            u32x2 w = {pack_bf16(acc[db][4 * rq] * mul, acc[db][4 * rq + 1] * mul),
                       pack_bf16(acc[db][4 * rq + 2] * mul, acc[db][4 * rq + 3] * mul)};
            *(lds_u32x2*)(uintptr_t)(wbase + (uint32_t)(((4 * db + rq) ^ wswz) << 4)) = w;
        }
    }
    const uint32_t rbase = stage + (uint32_t)(r4 * kRowBytes);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const u32x4 w = *(lds_u32x4*)(uintptr_t)(rbase + (uint32_t)(4 * k * kRowBytes + ((c16 ^ (((r4 & 3) << 2) | (k & 3))) << 4)));
        if (4 * k + r4 < rows && (D == kHeadDim || c16 < D / 8)) *reinterpret_cast<u32x4*>(at(4 * k + r4) + 8 * c16) = w;
    }
}

// ---- joining parts: each part of the keys has left O (fp32, divided by its own sum) and log2 of its sum, -inf where it saw none
// (such a part's O may be anything).  A group of D / 4 lanes adds parts of a row, four at a time; kWide: all groups of the
// workgroup share the parts of one row.  Bound by latency: 2 us and the launch; one token of 32 heads, d = 128, in 64 parts by single groups took 31 us.
constexpr int kCrossMaxParts = 64, kCrossJoinThreads = 256, kCrossJoinFew = 4;
struct CrossJoin {
    const float* part_o; const float* part_lse;      // [parts][Tq][Hq][d], [parts][Hq][Tq]
    void* o; float* lse;
    const int32_t* cu_q;
    int nseq, Tq, hq, parts;
};
template <int D, bool kF32, bool kWide>
__global__ void __launch_bounds__(kCrossJoinThreads) hyd_cross_join_kernel(CrossJoin p) {
    constexpr int kLanes = D / 4, kGroups = kCrossJoinThreads / kLanes;
    const int grp = threadIdx.x / kLanes, c = threadIdx.x % kLanes;
    const int64_t row = kWide ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * kGroups + grp;
    const int64_t rows = (int64_t)p.Tq * p.hq, plane = rows * D;
    if (row >= rows) return;
    const int t = (int)(row / p.hq), h = (int)(row - (int64_t)t * p.hq);
    if (t < p.cu_q[0] || t >= p.cu_q[p.nseq]) return;
    const float* pl = p.part_lse + (int64_t)h * p.Tq + t;
    const float* po = p.part_o + row * D + 4 * c;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    const auto factor = [](float x, float top) { return x == top ? 1.f : __builtin_amdgcn_exp2f(x - top); };      // (both may be -inf)
    constexpr int kStep = kWide ? kGroups : 1;
    for (int i0 = kWide ? grp : 0; i0 < p.parts; i0 += 4 * kStep) {
        float x[4], top = m;
        f32x4 v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int i = min(i0 + u * kStep, p.parts - 1);
            x[u] = pl[i * rows];
            v[u] = *reinterpret_cast<const f32x4*>(po + i * plane);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (i0 + u * kStep >= p.parts) x[u] = -INFINITY;
            top = fmaxf(top, x[u]);
        }
        const float f = factor(m, top);
        sum *= f;
        l *= f;
        m = top;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (x[u] == -INFINITY) continue;
            const float w = __builtin_amdgcn_exp2f(x[u] - m);
            l += w;
            sum += v[u] * w;
        }
    }
    if (kWide) {
        __shared__ f32x4 sums[kCrossJoinThreads];
        __shared__ float ml[2][kGroups];
        sums[threadIdx.x] = sum;
        if (c == 0) { ml[0][grp] = m; ml[1][grp] = l; }
        __syncthreads();
        if (grp) return;
        float top = -INFINITY;
#pragma unroll
        for (int g = 0; g < kGroups; ++g) top = fmaxf(top, ml[0][g]);
        sum = f32x4{0.f, 0.f, 0.f, 0.f};
        l = 0.f;
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const float f = factor(ml[0][g], top);
            l += ml[1][g] * f;
            sum += sums[g * kLanes + c] * f;
        }
        m = top;
    }
    const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);      // (a NaN stays one)
    sum *= inv;
    if (kF32) *reinterpret_cast<f32x4*>(static_cast<float*>(p.o) + row * D + 4 * c) = sum;
    else *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(p.o) + row * D + 4 * c) = u32x2{pack_bf16(sum[0], sum[1]), pack_bf16(sum[2], sum[3])};
    if (c == 0) p.lse[(int64_t)h * p.Tq + t] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f;
}

}  // namespace hyd
