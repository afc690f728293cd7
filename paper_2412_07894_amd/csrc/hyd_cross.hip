// Host side of cross attention (include/hyd_attn.h): argument checks, workspace, choice of the form, launches.
#include <string.h>

#include <mutex>

#include "hyd_cross_fwd.h"
#include "hyd_host.h"

namespace {

using namespace hyd;

constexpr float kLog2eHost = 1.44269504088896340736f;
constexpr size_t kAlign = 256;
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
// Compute units that choices and sizes are made for (the size of a workspace follows from host arithmetic alone).
constexpr int kCus = 256;

struct Sizes { int Tq, Tk, nseq, max_q, max_kv, hq, hkv, d; hyd_dtype dt; };

hyd_status check_sizes(const Sizes& z) {
    if (z.dt != HYD_BF16 && z.dt != HYD_FP32) return HYD_ERR_DTYPE;
    if (z.Tq < 0 || z.Tk < 0 || z.nseq < 0 || z.max_q < 0 || z.max_kv < 0) return HYD_ERR_SHAPE;
    if (z.hq <= 0 || z.hkv <= 0 || z.hq % z.hkv != 0) return HYD_ERR_HEADS;
    if (z.d != 64 && z.d != 128) return HYD_ERR_HEADDIM;
    if (z.nseq == 0 && z.Tq != 0) return HYD_ERR_SHAPE;
    if (z.max_q > z.Tq || z.max_kv > z.Tk) return HYD_ERR_SHAPE;
    // packed rows are counted in 31 bits; a sequence has to fit the range of a buffer resource, of which the upper half stands for
    // "outside"
    const unsigned long long size = z.dt == HYD_BF16 ? 2 : 4;
    if ((unsigned long long)z.Tq * (z.hq / z.hkv) >= (1ull << 31) - 256) return HYD_ERR_SHAPE;
    if ((unsigned long long)z.max_q * z.hq * z.d * size >= (1ull << 31) - 256 || (unsigned long long)z.max_kv * z.hkv * z.d * size >= (1ull << 31) - 256 ||
        258ull * z.hq * z.d * size >= (1ull << 31) - 256)
        return HYD_ERR_SHAPE;
    return HYD_OK;
}

hyd_status check_lengths(const int32_t* cu, int nseq, int T, int most, bool bounded) {
    if (!cu) return HYD_OK;
    if (cu[0] < 0 || cu[nseq] > T) return HYD_ERR_SEQLENS;
    for (int s = 0; s < nseq; ++s) {
        if (cu[s + 1] < cu[s]) return HYD_ERR_SEQLENS;
        if (bounded && cu[s + 1] - cu[s] > most) return HYD_ERR_SHAPE;
    }
    return HYD_OK;
}

long long tiles(long long rows, int tile) { return (rows + tile - 1) / tile; }
// tiles of nseq sequences with `total` rows, none longer than `most`, at most
long long most_tiles(long long total, long long most, int nseq, int tile) {
    const long long a = total / tile + nseq, b = tiles(most, tile) * nseq;
    return a < b ? a : b;
}

// ---- forward
struct FwdLayout { size_t hdr, items, need, part_o, part_lse, total; long long max_items; };
constexpr size_t kPartRoomRows = 65536;   // rows (tokens times query heads, times parts) that are joined at most
FwdLayout fwd_layout(const Sizes& z) {
    FwdLayout w;
    const int G = z.hq / z.hkv;
    w.max_items = most_tiles((long long)z.Tq * G, (long long)z.max_q * G, z.nseq, kFwdBM);
    size_t at = 0;
    w.hdr = at;   at += align_up(sizeof(int) * kHdrTotal);
    w.items = at; at += align_up(16 * (size_t)(w.max_items > 0 ? w.max_items : 1));
    w.need = at;
    const size_t rows = (size_t)z.Tq * z.hq, most = kCrossMaxParts * rows < kPartRoomRows ? kCrossMaxParts * rows : kPartRoomRows;
    w.total = at + (z.dt == HYD_BF16 ? align_up(most * (size_t)z.d * 4) + align_up(most * 4) : 0);
    return w;
}

// Parts that the room behind the rest of a workspace allows (1: the keys stay whole).
int parts_in_room(const FwdLayout& w, const Sizes& z, size_t bytes, int want) {
    const size_t rows = (size_t)z.Tq * z.hq, room = bytes - w.need;
    while (want > 1 && ((size_t)want * rows > kPartRoomRows || align_up(want * rows * z.d * 4) + align_up(want * rows * 4) > room)) --want;
    return want;
}

// ---- per-device state
struct CrossDevice { bool ready = false, ok = false; };
CrossDevice g_cross[64];
std::mutex g_cross_mutex;

template <typename K>
bool allow_lds(K kernel, int lds) {
    return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds) == hipSuccess;
}
template <int D>
bool prep_kernels() {
    return allow_lds(hyd_cross_fwd_bf16_kernel<D, false>, kFwdLds) && allow_lds(hyd_cross_fwd_bf16_kernel<D, true>, kFwdLds) &&
           allow_lds(hyd_cross_few_bf16_kernel<D>, kFewLds);
}
hyd_status cross_device(int* cus) {
    int dev = 0;
    const hyd_status st = current_device(&dev, cus);
    if (st != HYD_OK) return st;
    std::lock_guard<std::mutex> lock(g_cross_mutex);
    CrossDevice& d = g_cross[dev];
    if (!d.ready) {
        d.ok = prep_kernels<64>() && prep_kernels<128>();
        d.ready = d.ok;
    }
    return d.ok ? HYD_OK : HYD_ERR_LAUNCH;
}

CrossShape shape_of(const Sizes& z, const int32_t* cu_q, const int32_t* cu_kv, const int32_t* kv_lens) {
    CrossShape c;
    c.cu_q = cu_q; c.cu_kv = cu_kv; c.kv_lens = kv_lens;
    c.nseq = z.nseq; c.Tq = z.Tq; c.Tk = z.Tk; c.max_q = z.max_q; c.max_kv = z.max_kv;
    c.hq = z.hq; c.hkv = z.hkv; c.G = z.hq / z.hkv;
    return c;
}

template <int D>
void launch_join(const CrossJoin& j, hipStream_t st) {
    constexpr int kRows = kCrossJoinThreads / (D / 4);
    KernelTimer kt("cross_join", st);
    hipLaunchKernelGGL(hyd_cross_join_kernel<D>, dim3((unsigned)tiles((long long)j.Tq * j.hq, kRows)), dim3(kCrossJoinThreads), 0, st, j);
}

template <int D>
void launch_fwd(const Sizes& z, const CrossShape& c, const void* q, const void* k, const void* v, float scale, void* o, float* lse, char* ws,
                size_t ws_bytes, int cus, hipStream_t st) {
    const FwdLayout w = fwd_layout(z);
    CrossJoin j;
    j.part_o = reinterpret_cast<float*>(ws + w.need);
    j.o = static_cast<uint16_t*>(o); j.lse = lse; j.cu_q = c.cu_q; j.nseq = z.nseq; j.Tq = z.Tq; j.hq = z.hq; j.parts = 1;
    const long long rows = (long long)z.max_q * c.G;
    const auto part_lse = [&](int parts) { return reinterpret_cast<float*>(ws + w.need + align_up((size_t)parts * z.Tq * z.hq * z.d * 4)); };
    if (rows <= kFewRows) {
        CrossFewParams p;
        p.c = c;
        p.q = static_cast<const uint16_t*>(q); p.k = static_cast<const uint16_t*>(k); p.v = static_cast<const uint16_t*>(v);
        p.o = j.o; p.lse = lse; p.scale_log2 = scale * kLog2eHost;
        const long long items = (long long)z.nseq * z.hkv;
        constexpr int kTurn = kFewWaves * kFewKeys;
        long long want = items >= kCus ? tiles(8 * kCus, items) : kCus / items;
        if (want > kCrossMaxParts) want = kCrossMaxParts;
        long long chunk = tiles(tiles(z.max_kv, want), kTurn) * kTurn;
        if (items >= kCus && chunk < 4 * kTurn) chunk = 4 * kTurn;
        j.parts = parts_in_room(w, z, ws_bytes, (int)tiles(z.max_kv, chunk));
        p.parts = j.parts;
        p.chunk = j.parts == 1 ? z.max_kv : (int)(tiles(tiles(z.max_kv, j.parts), kTurn) * kTurn);
        p.part_o = const_cast<float*>(j.part_o); p.part_lse = part_lse(j.parts);
        KernelTimer kt("cross_few", st);
        hipLaunchKernelGGL(hyd_cross_few_bf16_kernel<D>, dim3((unsigned)(items * p.parts)), dim3(kFewThreads), kFewLds, st, p);
    } else {
        CrossFwdParams p;
        p.c = c;
        p.q = static_cast<const uint16_t*>(q); p.k = static_cast<const uint16_t*>(k); p.v = static_cast<const uint16_t*>(v);
        p.o = j.o; p.lse = lse; p.scale_log2 = scale * kLog2eHost;
        p.hdr = reinterpret_cast<int*>(ws + w.hdr); p.cursors = reinterpret_cast<int*>(ws + w.hdr) + kHdrCursor; p.items = reinterpret_cast<int*>(ws + w.items);
        p.tiles = (int)tiles(rows, kFwdBM);
        const long long own = (long long)z.nseq * p.tiles * z.hkv;
        const bool self = own <= kCus;
        long long want = 1;
        if (self) {
            want = kCus / own;
            const long long most = tiles(z.max_kv, 4 * kFwdBN);
            if (want > most) want = most;
            if (want > kCrossMaxParts) want = kCrossMaxParts;
        }
        j.parts = p.parts = want > 1 ? parts_in_room(w, z, ws_bytes, (int)want) : 1;
        p.part_o = const_cast<float*>(j.part_o); p.part_lse = part_lse(j.parts);
        long long grid = self ? own * p.parts : w.max_items * z.hkv;
        if (!self && grid > cus) grid = cus;
        p.hm = head_map_kv(z.hkv, (int)grid);
        if (!self) {
            const CrossList l{reinterpret_cast<int*>(ws + w.hdr), reinterpret_cast<int*>(ws + w.items), kFwdBM, 1, (int)w.max_items, false};
            KernelTimer kt("cross_list", st);
            hipLaunchKernelGGL(hyd_cross_list_kernel, dim3(1), dim3(kPreludeThreads), kCrossListLds, st, c, l);
        }
        KernelTimer kt("cross_fwd", st);
        hipLaunchKernelGGL((self ? hyd_cross_fwd_bf16_kernel<D, true> : hyd_cross_fwd_bf16_kernel<D, false>), dim3((unsigned)grid), dim3(kFwdThreads), kFwdLds, st, p);
    }
    if (j.parts > 1) {
        j.part_lse = part_lse(j.parts);
        launch_join<D>(j, st);
    }
}

}  // namespace

extern "C" {

size_t hyd_cross_attn_workspace_bytes(int total_q, int total_kv, int num_seqs, int max_seqlen_q, int max_seqlen_kv, int hq, int hkv,
                                      int head_dim, hyd_dtype dt, int is_bwd) {
    const Sizes z{total_q, total_kv, num_seqs, max_seqlen_q, max_seqlen_kv, hq, hkv, head_dim, dt};
    if (check_sizes(z) != HYD_OK) return 0;
    (void)is_bwd;
    return fwd_layout(z).total;
}

hyd_status hyd_cross_attn_fwd(const void* q, const void* k, const void* v, const int32_t* cu_q, const int32_t* cu_kv, const int32_t* kv_lens,
                              int num_seqs, const int32_t* cu_q_host, const int32_t* cu_kv_host, int total_q, int total_kv, int max_seqlen_q,
                              int max_seqlen_kv, int hq, int hkv, int head_dim, float softmax_scale, hyd_dtype dt, void* o, float* lse,
                              void* workspace, size_t workspace_bytes, void* hip_stream) {
    const Sizes z{total_q, total_kv, num_seqs, max_seqlen_q, max_seqlen_kv, hq, hkv, head_dim, dt};
    hyd_status st = check_sizes(z);
    if (st != HYD_OK) return st;
    if (dt != HYD_BF16) return HYD_ERR_DTYPE;
    if (total_q == 0 || num_seqs == 0) return HYD_OK;
    if (max_seqlen_q == 0) return HYD_ERR_SHAPE;
    if (!cu_q || !cu_kv || !q || !o || !lse || (total_kv > 0 && (!k || !v))) return HYD_ERR_NULL;
    if ((st = check_lengths(cu_q_host, num_seqs, total_q, max_seqlen_q, true)) != HYD_OK) return st;
    if ((st = check_lengths(cu_kv_host, num_seqs, total_kv, max_seqlen_kv, kv_lens == nullptr)) != HYD_OK) return st;
    if (!workspace || (uintptr_t)workspace % kAlign != 0 || workspace_bytes < fwd_layout(z).need) return HYD_ERR_WORKSPACE;
    int cus = 0;
    if ((st = cross_device(&cus)) != HYD_OK) return st;
    const CrossShape c = shape_of(z, cu_q, cu_kv, kv_lens);
    const auto launch = head_dim == 64 ? launch_fwd<64> : launch_fwd<128>;
    launch(z, c, q, k, v, softmax_scale, o, lse, static_cast<char*>(workspace), workspace_bytes, cus, static_cast<hipStream_t>(hip_stream));
    return hipGetLastError() == hipSuccess ? HYD_OK : HYD_ERR_LAUNCH;
}

}  // extern "C"
