// Host side of the general rotary positions (hyd_rotary.h): the frequency table, argument checks, launch.
#include <math.h>

#include "hyd_host.h"
#include "hyd_rotary.h"

namespace {

using namespace hyd;

typedef void (*RotKernel)(RotParams);
template <typename E, int C>
RotKernel rot_kernel(bool side) { return side ? hyd_rotary_kernel<E, C, true> : hyd_rotary_kernel<E, C, false>; }

// Pairs of a unit: as many as one 16-byte load holds, halved until head, turned part, strides and addresses are multiples.
int unit_pairs(const RotParams& p, int size) {
    int c = 16 / size;
    const auto fits = [&](int n) {
        if (p.head_dim % n != 0 || (p.rot / 2) % n != 0) return false;
        for (const RotTensor& t : p.t)
            if (t.heads > 0 && (t.x_stride % n != 0 || t.out_stride % n != 0 || (uintptr_t)t.x % (n * size) != 0 || (uintptr_t)t.out % (n * size) != 0)) return false;
        return true;
    };
    while (c > 1 && !fits(c)) c /= 2;
    return c;
}

}  // namespace

extern "C" {

hyd_status hyd_rope_frequencies(int rot_dim, double base, hyd_rope_scaling scaling, double factor, double original_length,
                                double low, double high, double* freqs) {
    if (rot_dim < 2 || rot_dim % 2 != 0 || rot_dim > kRotMaxDim) return HYD_ERR_HEADDIM;
    if (!(base > 1.0) || !isfinite(base)) return HYD_ERR_SHAPE;
    if (scaling != HYD_ROPE_PLAIN && scaling != HYD_ROPE_LINEAR && scaling != HYD_ROPE_PARTS) return HYD_ERR_SHAPE;
    if (scaling != HYD_ROPE_PLAIN && (!(factor > 0.0) || !isfinite(factor))) return HYD_ERR_SHAPE;
    if (scaling == HYD_ROPE_PARTS && (!(original_length > 0.0) || !isfinite(original_length) || !(low >= 0.0) || !(high > low) || !isfinite(high))) return HYD_ERR_SHAPE;
    if (!freqs) return HYD_ERR_NULL;
    for (int i = 0; i < rot_dim / 2; ++i) {
        const double f = pow(base, -2.0 * i / rot_dim);
        double keep = scaling == HYD_ROPE_PLAIN ? 1.0 : 0.0;
        if (scaling == HYD_ROPE_PARTS) {
            keep = (original_length * f / 6.283185307179586476925 - low) / (high - low);
            keep = keep < 0.0 ? 0.0 : (keep > 1.0 ? 1.0 : keep);
        }
        freqs[i] = keep == 1.0 ? f : f * keep + f / factor * (1.0 - keep);
    }
    return HYD_OK;
}

hyd_status hyd_rope_rotate(const void* q, int hq, int64_t q_stride, void* q_out, int64_t q_out_stride,
                           const void* k, int hkv, int64_t k_stride, void* k_out, int64_t k_out_stride,
                           const int32_t* cu_seqlens, const int32_t* starts, int num_seqs, const int32_t* positions,
                           int total_tokens, int head_dim, const double* freqs, int rot_dim, hyd_rope_layout layout,
                           float magnitude, int inverse, hyd_dtype dt, void* hip_stream) {
    if (dt != HYD_BF16 && dt != HYD_FP32) return HYD_ERR_DTYPE;
    if (total_tokens < 0 || num_seqs < 0) return HYD_ERR_SHAPE;
    if (layout != HYD_ROPE_HALF && layout != HYD_ROPE_INTERLEAVED) return HYD_ERR_SHAPE;
    if (hq <= 0 || hkv < 0) return HYD_ERR_HEADS;
    if (head_dim < 2 || head_dim > kRotMaxDim || rot_dim < 2 || rot_dim % 2 != 0 || rot_dim > head_dim) return HYD_ERR_HEADDIM;
    const int64_t q_row = (int64_t)hq * head_dim, k_row = (int64_t)hkv * head_dim;
    if (q_stride < q_row || q_out_stride < q_row || (hkv > 0 && (k_stride < k_row || k_out_stride < k_row))) return HYD_ERR_SHAPE;
    if ((hq + (long long)hkv) * head_dim > (1 << 20)) return HYD_ERR_HEADS;      // the kernel counts the units of its rows in 21 bits
    if (total_tokens == 0 || (num_seqs == 0 && !positions)) return HYD_OK;
    if (!q || !q_out || !freqs || (hkv > 0 && (!k || !k_out)) || (!positions && !cu_seqlens)) return HYD_ERR_NULL;
    const size_t size = dt == HYD_BF16 ? 2 : 4;
    for (const void* x : {q, (const void*)q_out, hkv > 0 ? k : q, hkv > 0 ? (const void*)k_out : q})
        if ((uintptr_t)x % size != 0) return HYD_ERR_SHAPE;
    // in place is in place for both, with the same strides
    const bool q_in = q == q_out, k_in = hkv == 0 || k == k_out;
    if ((q_in && q_stride != q_out_stride) || (hkv > 0 && k_in && k_stride != k_out_stride)) return HYD_ERR_SHAPE;

    RotParams p;
    p.t[0] = {q, q_out, q_stride, q_out_stride, hq};
    p.t[1] = {k, k_out, k_stride, k_out_stride, hkv};
    p.cu = cu_seqlens; p.starts = starts; p.positions = positions; p.freqs = freqs;
    p.nseq = num_seqs; p.T = total_tokens; p.head_dim = head_dim; p.rot = rot_dim;
    p.mag = magnitude; p.inverse = inverse != 0; p.in_place = q_in && k_in;
    const int c = unit_pairs(p, (int)size);
    p.pair_units = rot_dim / 2 / c;
    p.units = p.pair_units + (p.in_place ? 0 : (head_dim - rot_dim + 2 * c - 1) / (2 * c));
    const long long row_units = (hq + (long long)hkv) * p.units;
    int device = 0, cus = 0;
    const hyd_status ds = current_device(&device, &cus);
    if (ds != HYD_OK) return ds;
    // Rows of a workgroup: as many, up to sixteen, as leave sixteen workgroups for each CU; with few heads a row alone does not
    // fill one.  Always one row, this rule, always sixteen (32/8 heads, d = 128, bf16): 512 tokens 7.9, 8.2 and 17.4 us, 4096 tokens 18.2,
    // 18.2 and 22.9 us, 24700 tokens 109, 106 and 123 us.
    p.tok = 1;
    while (2 * p.tok <= kRotTokens && 2ll * p.tok * cus * 16 <= total_tokens && 2 * p.tok * row_units <= (1 << 20)) p.tok *= 2;
    const unsigned groups = (unsigned)((total_tokens + (long long)p.tok - 1) / p.tok);
    const dim3 grid(groups < kRotGridX ? groups : kRotGridX, (groups + kRotGridX - 1) / kRotGridX);
    const size_t lds = sizeof(float) * 2 * (size_t)p.tok * (size_t)(rot_dim / 2);
    const bool side = layout == HYD_ROPE_INTERLEAVED;
    const RotKernel kernel = dt == HYD_BF16 ? (c == 8 ? rot_kernel<uint16_t, 8>(side) : c == 4 ? rot_kernel<uint16_t, 4>(side)
                                             : c == 2 ? rot_kernel<uint16_t, 2>(side) : rot_kernel<uint16_t, 1>(side))
                                            : (c == 4 ? rot_kernel<float, 4>(side) : c == 2 ? rot_kernel<float, 2>(side) : rot_kernel<float, 1>(side));
    {
        KernelTimer kt("rotary", static_cast<hipStream_t>(hip_stream));
        hipLaunchKernelGGL(kernel, grid, dim3(kRotThreads), lds, static_cast<hipStream_t>(hip_stream), p);
    }
    return hipGetLastError() == hipSuccess ? HYD_OK : HYD_ERR_LAUNCH;
}

}  // extern "C"
