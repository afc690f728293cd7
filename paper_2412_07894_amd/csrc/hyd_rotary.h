// Rotary positions in their general form: pairs that lie half the turned part apart or side by side, the first rot
// elements of a head only, any table of frequencies, positions that start anywhere, bf16 and fp32, strided tokens, Q and
// K in one launch.  (hyd_rope.h turns whole heads of 64 or 128 bf16 elements by the plain frequencies.)
//
// Pair i of a head at position m turns by the angle m f_i: (a, b) -> mag (a cos - b sin, b cos + a sin); `inverse` negates the
// angle, which is the transpose and carries gradients back.  m f_i / (2 pi) is formed in double and reduced to half a
// revolution there; sine and cosine are formed in fp32 from the rest, the products in fp32, and the result is rounded once.
//
// Bound by HBM: each element is read once and written once.  A workgroup takes `tok` packed rows of all heads: sine and cosine of
// its rows' pairs go to LDS once (their cost is shared by the heads), and the threads walk the units of its rows in memory order,
// a unit being C pairs (two loads of C elements, 16 bytes each where alignment allows) or 2 C elements behind the
// turned part, which are only copied.  The first units are requested before the table is formed.  24700 tokens of 32/8 heads of 128
// out of a fused projection, 506 MB: 104 us, 4.9 TB/s (a large copy reaches 5.07); half of 80 heads of 128, side by side, 317 MB: 60 us;
// one token for each of 16 requests: 4.4 us, of the 8 that the call takes.
#pragma once
#include "hyd_find.h"

namespace hyd {

constexpr int kRotThreads = 256, kRotTokens = 16, kRotAhead = 4;
constexpr int kRotMaxDim = 1024;          // elements of a head
constexpr int kRotGridX = 1 << 22;        // workgroups of a grid's row (a launch has fewer than 2^32 threads in one dimension)

struct RotTensor { const void* x; void* out; int64_t x_stride, out_stride; int heads; };      // strides of a token in elements
struct RotParams {
    RotTensor t[2];                       // Q, K
    const int32_t* cu; const int32_t* starts; const int32_t* positions;
    const double* freqs;
    int nseq, T, tok, head_dim, rot;
    int units, pair_units;                // of a head
    float mag;
    int inverse, in_place;                // in_place: nothing is copied
};

template <typename E, int C> struct RotVec { E v[C]; };
template <int C, typename E>
__device__ __forceinline__ void rot_load(RotVec<E, C>& r, const E* p) { __builtin_memcpy(&r, __builtin_assume_aligned(p, sizeof(E) * C), sizeof(E) * C); }
template <int C, typename E>
__device__ __forceinline__ void rot_store(E* p, const RotVec<E, C>& r) { __builtin_memcpy(__builtin_assume_aligned(p, sizeof(E) * C), &r, sizeof(E) * C); }
__device__ __forceinline__ float rot_float(uint16_t u) { return __uint_as_float((uint32_t)u << 16); }
__device__ __forceinline__ float rot_float(float f) { return f; }
__device__ __forceinline__ void rot_pair(uint16_t& a, uint16_t& b, float x, float y) {
    const uint32_t w = pack_bf16(x, y);
    a = (uint16_t)w;
    b = (uint16_t)(w >> 16);
}
__device__ __forceinline__ void rot_pair(float& a, float& b, float x, float y) { a = x; b = y; }

// E: element type (uint16_t: bf16).  C: pairs of a unit.  kSide: the elements of a pair lie side by side.
template <typename E, int C, bool kSide>
__global__ void __launch_bounds__(kRotThreads) hyd_rotary_kernel(RotParams p) {
    extern __shared__ f32x2 cs[];                        // [tok][rot / 2] cosine, sine
    __shared__ long long pos[kRotTokens];                // of the workgroup's rows; kNone: in no sequence
    constexpr long long kNone = INT64_MIN;
    const int tid = threadIdx.x, half = p.rot / 2;
    const int64_t begin = ((int64_t)blockIdx.y * kRotGridX + blockIdx.x) * p.tok;
    if (begin >= p.T) return;
    const int t0 = (int)begin, nt = min(p.tok, p.T - t0);
    const int H = p.t[0].heads + p.t[1].heads;
    const int n_units = nt * H * p.units;
    const float inv_units = 1.f / (float)p.units, inv_h = 1.f / (float)H;
    struct Unit { const E* src; E* dst; int second, row, u; };       // second: offset of the second vector
    auto unit_at = [&](int e) {
        Unit x;
        // (e + 1/2) / n truncates to the quotient as long as e < 2^21
        const int rest = (int)(((float)e + 0.5f) * inv_units);
        x.u = e - rest * p.units;
        x.row = (int)(((float)rest + 0.5f) * inv_h);
        int h = rest - x.row * H;
        const bool second_tensor = h >= p.t[0].heads;
        const RotTensor& w = p.t[second_tensor];
        if (second_tensor) h -= p.t[0].heads;
        int first;
        if (x.u < p.pair_units) { first = (kSide ? 2 * C : C) * x.u; x.second = kSide ? C : half; }
        else { first = p.rot + 2 * C * (x.u - p.pair_units); x.second = first + C < p.head_dim ? C : 0; }
        x.src = static_cast<const E*>(w.x) + (int64_t)(t0 + x.row) * w.x_stride + (int64_t)h * p.head_dim + first;
        x.dst = static_cast<E*>(w.out) + (int64_t)(t0 + x.row) * w.out_stride + (int64_t)h * p.head_dim + first;
        return x;
    };
    RotVec<E, C> a[kRotAhead], b[kRotAhead];
    Unit un[kRotAhead];
    auto load = [&](int e0) {
#pragma unroll
        for (int k = 0; k < kRotAhead; ++k) {
            const int e = e0 + k * kRotThreads;
            if (e < n_units) {
                un[k] = unit_at(e);
                rot_load<C>(a[k], un[k].src);
                rot_load<C>(b[k], un[k].src + un[k].second);
            }
        }
    };
    load(tid);
    if (p.positions) {
        if (tid < nt) pos[tid] = p.positions[t0 + tid];
    } else if (tid < 64) {
        int s = 0, first = 0, end = -1;
        bool in = false;
        for (int r = 0; r < nt; ++r) {
            const int t = t0 + r;
            if (!in || t >= end) in = find_sequence(p.cu, p.nseq, t, s, first, end);
            if (tid == 0) pos[r] = in ? (long long)(t - first) + (p.starts ? p.starts[s] : 0) : kNone;
        }
    }
    __syncthreads();
    for (int e = tid; e < nt * half; e += kRotThreads) {
        const int r = (int)(((float)e + 0.5f) * (1.f / (float)half)), i = e - r * half;
        const double rev = (double)pos[r] * (p.freqs[i] * 0.15915494309189533576888);      // kNone: never used
        float s, c;
        sincospif(2.f * (float)(rev - rint(rev)), &s, &c);
        cs[e] = f32x2{c * p.mag, (p.inverse ? -s : s) * p.mag};
    }
    __syncthreads();
    for (int e0 = tid; e0 < n_units; e0 += kRotAhead * kRotThreads) {
        if (e0 != tid) load(e0);
#pragma unroll
        for (int k = 0; k < kRotAhead; ++k) {
            if (e0 + k * kRotThreads >= n_units || pos[un[k].row] == kNone) continue;
            if (un[k].u < p.pair_units) {
                const f32x2* w = cs + un[k].row * half + C * un[k].u;
                RotVec<E, C> y, z;
#pragma unroll
                for (int j = 0; j < C; ++j) {
                    const float c = w[j][0], s = w[j][1];
                    E &pa = kSide ? (2 * j < C ? a[k].v[(2 * j) % C] : b[k].v[(2 * j) % C]) : a[k].v[j];
                    E &pb = kSide ? (2 * j + 1 < C ? a[k].v[(2 * j + 1) % C] : b[k].v[(2 * j + 1) % C]) : b[k].v[j];
                    const float x0 = rot_float(pa), x1 = rot_float(pb);
                    E r0, r1;
                    rot_pair(r0, r1, x0 * c - x1 * s, x1 * c + x0 * s);
                    if (kSide) {
                        (2 * j < C ? y.v[(2 * j) % C] : z.v[(2 * j) % C]) = r0;
                        (2 * j + 1 < C ? y.v[(2 * j + 1) % C] : z.v[(2 * j + 1) % C]) = r1;
                    } else {
                        y.v[j] = r0;
                        z.v[j] = r1;
                    }
                }
                rot_store<C>(un[k].dst, y);
                rot_store<C>(un[k].dst + un[k].second, z);
            } else if (!p.in_place) {
                rot_store<C>(un[k].dst, a[k]);
                rot_store<C>(un[k].dst + un[k].second, b[k]);      // (second = 0: the same once more)
            }
        }
    }
}

}  // namespace hyd
