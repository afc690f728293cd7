// Host side of cross attention (include/hyd_attn.h): argument checks, workspace, choice of the form, launches.
#include <string.h>

#include <initializer_list>
#include <mutex>

#include "hyd_cross_bwd.h"
#include "hyd_cross_fp32.h"
#include "hyd_cross_keys.h"
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

int tile_q(hyd_dtype dt) { return dt == HYD_BF16 ? kFwdBM : kF32BM; }
int tile_kv(hyd_dtype dt) { return dt == HYD_BF16 ? kKwBN : kF32KvBN; }
long long tiles(long long rows, int tile) { return (rows + tile - 1) / tile; }
// tiles of nseq sequences with `total` rows, none longer than `most`, at most
long long most_tiles(long long total, long long most, int nseq, int tile) {
    const long long a = total / tile + nseq, b = tiles(most, tile) * nseq;
    return a < b ? a : b;
}

// ---- forward
// Sequences of at most 128 packed rows in bf16: tiles of as many, two workgroups to a CU (see CrossFwd).
bool short_rows(const Sizes& z) { return z.dt == HYD_BF16 && (long long)z.max_q * (z.hq / z.hkv) <= CrossFwd<4>::kBM; }
int fwd_rows(const Sizes& z) { return short_rows(z) ? CrossFwd<4>::kBM : tile_q(z.dt); }
struct FwdLayout { size_t hdr, items, need, total; long long max_items; };
constexpr size_t kPartRoomRows = 65536;   // rows (tokens times query heads, times parts) that are joined at most
FwdLayout fwd_layout(const Sizes& z) {
    FwdLayout w;
    const int G = z.hq / z.hkv;
    w.max_items = most_tiles((long long)z.Tq * G, (long long)z.max_q * G, z.nseq, fwd_rows(z));
    size_t at = 0;
    w.hdr = at;   at += align_up(sizeof(int) * kHdrTotal);
    w.items = at; at += align_up(16 * (size_t)(w.max_items > 0 ? w.max_items : 1));
    w.need = at;
    const size_t rows = (size_t)z.Tq * z.hq, most = kCrossMaxParts * rows < kPartRoomRows ? kCrossMaxParts * rows : kPartRoomRows;
    w.total = at + align_up(most * (size_t)z.d * 4) + align_up(most * 4);
    return w;
}

// Parts that the room behind the rest of a workspace allows (1: the keys stay whole).
int parts_in_room(const FwdLayout& w, const Sizes& z, size_t bytes, int want) {
    const size_t rows = (size_t)z.Tq * z.hq, room = bytes - w.need;
    while (want > 1 && ((size_t)want * rows > kPartRoomRows || align_up(want * rows * z.d * 4) + align_up(want * rows * 4) > room)) --want;
    return want;
}

// ---- backward
constexpr int kBwdMaxParts = 16, kDqPartRows = 65536, kKvPartRows = 131072, kBwdItems = 2 * kCus;
struct BwdLayout { size_t q_hdr, q_items, kv_hdr, kv_items, stat[4], q16, do16, k16, absmax, need, total; long long n_q, n_kv; };
BwdLayout bwd_layout(const Sizes& z) {
    BwdLayout w;
    const int G = z.hq / z.hkv;
    w.n_q = most_tiles((long long)z.Tq * G, (long long)z.max_q * G, z.nseq, tile_q(z.dt));
    w.n_kv = most_tiles(z.Tk, z.max_kv, z.nseq, tile_kv(z.dt));
    const size_t q_elems = (size_t)z.Tq * z.hq * z.d, kv_elems = (size_t)z.Tk * z.hkv * z.d;
    const auto records = [](long long n) { return align_up(16 * (size_t)(n > kBwdItems ? n : kBwdItems)); };      // (in parts: kBwdItems records at most)
    size_t at = 0;
    w.q_hdr = at;    at += align_up(sizeof(int) * kHdrTotal);
    w.q_items = at;  at += records(w.n_q);
    w.kv_hdr = at;   at += align_up(sizeof(int) * kHdrTotal);
    w.kv_items = at; at += records(w.n_kv);
    if (z.dt == HYD_FP32) {
        w.stat[0] = at; at += align_up(sizeof(float) * (size_t)z.Tq * z.hq);
    } else {
        for (size_t& s : w.stat) { s = at; at += align_up(sizeof(float) * (size_t)z.Tq * z.hq); }
        w.q16 = at;      at += align_up(2 * q_elems);
        w.do16 = at;     at += align_up(2 * q_elems);
        w.k16 = at;      at += align_up(2 * kv_elems);
        w.absmax = at;   at += align_up(sizeof(uint32_t) * kPrepMaxWg);
    }
    w.need = at;
    const size_t q_rows = (size_t)z.Tq * z.hq * kBwdMaxParts, kv_rows = (size_t)z.Tk * z.hkv * kBwdMaxParts;
    const size_t dq = (q_rows < kDqPartRows ? q_rows : kDqPartRows) * (size_t)z.d * 4, dkv = (kv_rows < kKvPartRows ? kv_rows : kKvPartRows) * (size_t)z.d * 8;
    w.total = at + align_up(dq > dkv ? dq : dkv);
    return w;
}
// Parts of an item where `items` of them leave workgroups idle: up to `target` in all, none shorter than `least` of its `steps`, and as
// many as their sums of `row_bytes` have room for (most_rows of `rows` at most).  Whole and in parts: 50 queries against 2000 keys, fp32,
// d = 128, dQ 220 and 55 us; 4000 against 77 keys, dK/dV 350 and 66 us.
int bwd_parts(long long items, int target, long long steps, int least, size_t rows, size_t most_rows, size_t row_bytes, size_t room) {
    long long n = items > 0 ? target / items : 1;
    if (n > steps / least) n = steps / least;
    if (n > kBwdMaxParts) n = kBwdMaxParts;
    while (n > 1 && ((size_t)n * rows > most_rows || (size_t)n * rows * row_bytes > room)) --n;
    return n > 1 ? (int)n : 1;
}

// ---- per-device state
struct CrossDevice { bool ready = false, ok = false; };
CrossDevice g_cross[64];
std::mutex g_cross_mutex;

// A kernel whose input another one of the call should have written is not launched where that launch was refused.
bool launched() { return hipPeekAtLastError() == hipSuccess; }

template <typename K>
bool allow_lds(K kernel, int lds) {
    return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds) == hipSuccess;
}
template <int D>
bool prep_kernels() {
    return allow_lds(hyd_cross_fwd_bf16_kernel<D, false, 8>, CrossFwd<8>::kLds) && allow_lds(hyd_cross_fwd_bf16_kernel<D, true, 8>, CrossFwd<8>::kLds) &&
           allow_lds(hyd_cross_fwd_bf16_kernel<D, false, 4>, CrossFwd<4>::kLds) && allow_lds(hyd_cross_fwd_bf16_kernel<D, true, 4>, CrossFwd<4>::kLds) &&
           allow_lds(hyd_cross_few_bf16_kernel<D>, kFewLds) && allow_lds(hyd_cross_dq_bf16_kernel<D>, kDqLds) &&
           allow_lds(hyd_cross_bwd_keys_bf16_kernel<D>, KeysForm<D>::kLds) &&
           allow_lds(hyd_bwd_dkdv_wide_bf16_kernel<D, CrossBwdParams>, kKwLds) && allow_lds(hyd_cross_fwd_fp32_kernel<D, false>, f32_lds<D>()) &&
           allow_lds(hyd_cross_fwd_fp32_kernel<D, true>, f32_lds<D>()) && allow_lds(hyd_cross_dq_fp32_kernel<D>, f32_lds<D>()) &&
           allow_lds(hyd_cross_dkdv_fp32_kernel<D, false>, f32_lds<D>()) &&
           allow_lds(hyd_cross_dkdv_fp32_kernel<D, true>, f32_lds<D>());
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

// A launch has fewer than 2^32 threads.  The forms that give a workgroup to every (sequence, KV head) leave more of them to those
// that take items from a list.
bool fits_launch(long long workgroups, int threads) { return workgroups * threads < (1ll << 32); }

template <int D, bool kF32>
void launch_join(const CrossJoin& j, hipStream_t st) {
    KernelTimer kt("cross_join", st);
    const long long rows = (long long)j.Tq * j.hq;
    if (j.parts > kCrossJoinFew) hipLaunchKernelGGL((hyd_cross_join_kernel<D, kF32, true>), dim3((unsigned)rows), dim3(kCrossJoinThreads), 0, st, j);
    else hipLaunchKernelGGL((hyd_cross_join_kernel<D, kF32, false>), dim3((unsigned)tiles(rows, kCrossJoinThreads / (D / 4))), dim3(kCrossJoinThreads), 0, st, j);
}

template <int D>
void launch_fwd(const Sizes& z, const CrossShape& c, const void* q, const void* k, const void* v, float scale, void* o, float* lse, char* ws,
                size_t ws_bytes, int cus, hipStream_t st) {
    const FwdLayout w = fwd_layout(z);
    CrossJoin j;
    j.part_o = reinterpret_cast<float*>(ws + w.need);
    j.o = o; j.lse = lse; j.cu_q = c.cu_q; j.nseq = z.nseq; j.Tq = z.Tq; j.hq = z.hq; j.parts = 1;
    const long long rows = (long long)z.max_q * c.G, items = (long long)z.nseq * z.hkv;
    const auto part_lse = [&](int parts) { return reinterpret_cast<float*>(ws + w.need + align_up((size_t)parts * z.Tq * z.hq * z.d * 4)); };
    if (z.dt == HYD_BF16 && rows <= kFewRows && fits_launch(items, kFewThreads)) {
        CrossFewParams p;
        p.c = c;
        p.q = static_cast<const uint16_t*>(q); p.k = static_cast<const uint16_t*>(k); p.v = static_cast<const uint16_t*>(v);
        p.o = static_cast<uint16_t*>(o); p.lse = lse; p.scale_log2 = scale * kLog2eHost;
        constexpr int kTurn = kFewWaves * kFewKeys;
        // Parts of the keys: two workgroups for a CU, or if there are as many items as CUs, 32, whose ends then hardly differ;
        // each of 512 keys at least (1024 where the chip is full).  Up to 1024 keys (2048) they stay whole: a second launch costs 3 us.
        // Whole and in parts: 4 tokens of 32/8 heads, d = 128, 700 keys 9.4 and 11.0 us, 1500 keys 12.7 and 10.9, 8000 keys 52 and 26;
        // 40 tokens of 8 heads, d = 64, 1 to 30000 keys 462 and 293 us.  Parts of 512 and of 256 keys at least: one token of 32/8 heads,
        // d = 128, 8000 keys 11.7 and 10.8 us, 3000 keys 11.2 and 10.7; 4 of 20 heads, d = 64, 1500 keys 11.1 and 11.0; 16 of 32/8 heads, 1500 keys
        // 21.0 and 20.6, 8000 keys 98.7 and 99.7; but 700 keys, which stay whole here, 9.5 and 10.4 us for one token, 11.8 and 14.8 for 16.
        long long want = items >= kCus ? tiles(32 * kCus, items) : 2 * kCus / items;
        if (want > kCrossMaxParts) want = kCrossMaxParts;
        long long chunk = tiles(tiles(z.max_kv, want), kTurn) * kTurn;
        const long long least = (items >= kCus ? 8 : 4) * kTurn;
        if (chunk < least) chunk = least;
        if (z.max_kv <= 2 * least) chunk = z.max_kv;
        j.parts = z.max_kv > 0 ? parts_in_room(w, z, ws_bytes, (int)tiles(z.max_kv, chunk)) : 1;
        p.parts = j.parts;
        p.chunk = j.parts == 1 ? z.max_kv : (int)(tiles(tiles(z.max_kv, j.parts), kTurn) * kTurn);
        p.part_o = const_cast<float*>(j.part_o); p.part_lse = part_lse(j.parts);
        KernelTimer kt("cross_few", st);
        hipLaunchKernelGGL(hyd_cross_few_bf16_kernel<D>, dim3((unsigned)(items * p.parts)), dim3(kFewThreads), kFewLds, st, p);
    } else {
        // items of whole tiles: own ones where they all fit on the chip, with the keys in parts where they do not fill it, else from a list
        // (2 x 200 queries of 8/2 heads against 8000 keys, d = 128: 16 parts 34 us, whole 179 us).  Parts are counted for one workgroup to a CU,
        // also in tiles of 128 rows, of which two fit.  Counted for one and for two: 100 queries of 8 heads, d = 128, 12000 keys 21.2 and 24.4 us,
        // 4 x 100 of 20 heads, 4000 keys 38 and 44; 12 x 64 of 20 heads, d = 64, 1000 keys 20 and 21, but 4000 keys 58 and 50, 12000 keys 197 and 150.
        const bool small = short_rows(z);
        const int per_cu = small ? CrossFwd<4>::kPerCu : 1;
        const int tile = fwd_rows(z), key_tile = z.dt == HYD_BF16 ? kFwdBN : kF32Tile;
        const long long per_seq = tiles(rows, tile), own = (long long)z.nseq * per_seq * z.hkv;
        const bool self = own <= per_cu * kCus;
        long long want = 1;
        if (self) {
            const long long most = tiles(z.max_kv, 4 * key_tile);
            want = kCus / own < most ? kCus / own : most;
            if (want > kCrossMaxParts) want = kCrossMaxParts;
        }
        j.parts = want > 1 ? parts_in_room(w, z, ws_bytes, (int)want) : 1;
        long long grid = self ? own * j.parts : w.max_items * z.hkv;
        if (!self && grid > per_cu * cus) grid = per_cu * cus;
        int* hdr = reinterpret_cast<int*>(ws + w.hdr); int* items = reinterpret_cast<int*>(ws + w.items);
        if (!self) {
            const CrossList l{hdr, items, tile, 1, (int)w.max_items, false};
            KernelTimer kt("cross_list", st);
            hipLaunchKernelGGL(hyd_cross_list_kernel, dim3(1), dim3(kPreludeThreads), kCrossListLds, st, c, l);
        }
        if (!launched()) return;
        const auto common = [&](auto& p) {
            p.c = c; p.hdr = hdr; p.cursors = hdr + kHdrCursor; p.items = items; p.hm = head_map_kv(z.hkv, (int)grid);
            p.parts = j.parts; p.tiles = (int)per_seq; p.part_o = const_cast<float*>(j.part_o); p.part_lse = part_lse(j.parts);
        };
        KernelTimer kt("cross_fwd", st);
        if (z.dt == HYD_BF16) {
            CrossFwdParams p;
            common(p);
            p.q = static_cast<const uint16_t*>(q); p.k = static_cast<const uint16_t*>(k); p.v = static_cast<const uint16_t*>(v);
            p.o = static_cast<uint16_t*>(o); p.lse = lse; p.scale_log2 = scale * kLog2eHost;
            if (small)
                hipLaunchKernelGGL((self ? hyd_cross_fwd_bf16_kernel<D, true, 4> : hyd_cross_fwd_bf16_kernel<D, false, 4>), dim3((unsigned)grid), dim3(CrossFwd<4>::kThreads), CrossFwd<4>::kLds, st, p);
            else
                hipLaunchKernelGGL((self ? hyd_cross_fwd_bf16_kernel<D, true, 8> : hyd_cross_fwd_bf16_kernel<D, false, 8>), dim3((unsigned)grid), dim3(CrossFwd<8>::kThreads), CrossFwd<8>::kLds, st, p);
        } else {
            CrossF32Params p;
            memset(&p, 0, sizeof(p));
            common(p);
            p.q = static_cast<const float*>(q); p.k = static_cast<const float*>(k); p.v = static_cast<const float*>(v);
            p.o_out = static_cast<float*>(o); p.lse_out = lse; p.scale = scale;
            hipLaunchKernelGGL((self ? hyd_cross_fwd_fp32_kernel<D, true> : hyd_cross_fwd_fp32_kernel<D, false>), dim3((unsigned)grid), dim3(64 * kF32Waves), f32_lds<D>(), st, p);
        }
    }
    if (j.parts > 1 && launched()) {
        j.part_lse = part_lse(j.parts);
        if (z.dt == HYD_FP32) launch_join<D, true>(j, st);
        else launch_join<D, false>(j, st);
    }
}

template <int D>
void launch_sum(const CrossSum& x, bool f32, hipStream_t st) {
    KernelTimer kt("cross_sum", st);
    hipLaunchKernelGGL((f32 ? hyd_cross_sum_kernel<D, true> : hyd_cross_sum_kernel<D, false>), dim3((unsigned)x.T, x.out[1] ? 2 : 1), dim3(kCrossSumThreads), 0, st, x);
}

struct BwdArgs { const void *q, *k, *v, *o; const float* lse; const void* d_o; void *dq, *dk, *dv; };
template <int D>
void launch_bwd(const Sizes& z, const CrossShape& c, const BwdArgs& a, float scale, char* ws, size_t ws_bytes, int cus, hipStream_t st) {
    const BwdLayout w = bwd_layout(z);
    const int G = c.G;
    BwdScratch sc;
    sc.Dq = reinterpret_cast<float*>(ws + w.stat[0]); sc.kqmul = reinterpret_cast<float*>(ws + w.stat[1]);
    sc.lse2 = reinterpret_cast<float*>(ws + w.stat[2]); sc.Dkv = reinterpret_cast<float*>(ws + w.stat[3]);
    sc.q16 = reinterpret_cast<uint16_t*>(ws + w.q16); sc.do16 = reinterpret_cast<uint16_t*>(ws + w.do16); sc.k16 = reinterpret_cast<uint16_t*>(ws + w.k16);
    sc.absmax = reinterpret_cast<uint32_t*>(ws + w.absmax);
    float* part = reinterpret_cast<float*>(ws + w.need);
    const size_t room = ws_bytes - w.need, q_rows = (size_t)z.Tq * z.hq, kv_rows = (size_t)z.Tk * z.hkv;
    const int parts_q = bwd_parts(w.n_q * z.hkv, kCus, tiles(z.max_kv, kDqBN), 8, q_rows, kDqPartRows, (size_t)D * 4, room);
    const int parts_kv = bwd_parts(w.n_kv * z.hkv, kBwdItems, tiles((long long)z.max_q * G, kKwBM), 8, kv_rows, kKvPartRows, (size_t)D * 8, room);
    const long long pairs = (long long)z.nseq * z.hkv;
    if (z.max_kv <= kKeysMax && z.max_kv > 0 && fits_launch(pairs, kKeysThreads)) {
        CrossKeysParams p;
        p.c = c;
        p.q = static_cast<const uint16_t*>(a.q); p.k = static_cast<const uint16_t*>(a.k); p.v = static_cast<const uint16_t*>(a.v);
        p.o = static_cast<const uint16_t*>(a.o); p.d_o = static_cast<const uint16_t*>(a.d_o); p.lse = a.lse;
        p.dq = static_cast<uint16_t*>(a.dq); p.dk = static_cast<uint16_t*>(a.dk); p.dv = static_cast<uint16_t*>(a.dv);
        p.parts = bwd_parts(pairs, kBwdItems, tiles((long long)z.max_q * G, KeysForm<D>::kBM), 4, kv_rows, kKvPartRows, (size_t)D * 8, room);
        p.part = part; p.scale = scale; p.scale_log2 = scale * kLog2eHost;
        {
            KernelTimer kt("cross_bwd_keys", st);
            hipLaunchKernelGGL(hyd_cross_bwd_keys_bf16_kernel<D>, dim3((unsigned)(pairs * p.parts)), dim3(kKeysThreads), KeysForm<D>::kLds, st, p);
        }
        if (p.parts > 1 && launched())
            launch_sum<D>(CrossSum{part, {p.dk, p.dv}, c.cu_kv, c.kv_lens, z.nseq, z.Tk, z.hkv, p.parts}, false, st);
        return;
    }
    int* q_hdr = reinterpret_cast<int*>(ws + w.q_hdr); int* kv_hdr = reinterpret_cast<int*>(ws + w.kv_hdr);
    int* q_items = reinterpret_cast<int*>(ws + w.q_items); int* kv_items = reinterpret_cast<int*>(ws + w.kv_items);
    const long long work_q = w.n_q * z.hkv * parts_q, work_kv = w.n_kv * z.hkv * parts_kv;
    {
        CrossPrepParams p;
        p.c = c;
        p.o = static_cast<const uint16_t*>(a.o); p.d_o = static_cast<const uint16_t*>(a.d_o); p.lse = a.lse; p.k = static_cast<const uint16_t*>(a.k);
        p.dk = static_cast<uint16_t*>(a.dk); p.dv = static_cast<uint16_t*>(a.dv);
        p.tok = prep_tokens(z.Tq, z.hq);
        p.n_q = sc.n_absmax = prep_workgroups(z.Tq, p.tok);
        p.sc = sc;
        p.zero = cross_zero(z.nseq, c.kv_lens != nullptr);
        const long long copies = tiles((long long)z.Tk * z.hkv, 4 * kPrepThreads / (D / 8));
        const int n_k = (int)(copies < kPrepTarget ? copies : kPrepTarget);
        p.lists[0] = CrossList{q_hdr, q_items, kDqBM, parts_q, (int)(w.n_q * parts_q), false};
        p.lists[1] = CrossList{kv_hdr, kv_items, kKwBN, parts_kv, (int)(w.n_kv * parts_kv), true};
        KernelTimer kt("cross_prep", st);
        hipLaunchKernelGGL(hyd_cross_prep_bf16_kernel<D>, dim3((unsigned)(kCrossLists + p.zero.n + p.n_q + n_k)), dim3(kPrepThreads), cross_prep_lds(z.hq, p.tok), st, p);
    }
    if (!launched()) return;
    const auto grid_of = [&](long long work) { return (int)(work < 1 ? 1 : (work < cus ? work : cus)); };
    {
        CrossDqParams p;
        p.c = c;
        p.q = static_cast<const uint16_t*>(a.q); p.v = static_cast<const uint16_t*>(a.v); p.d_o = static_cast<const uint16_t*>(a.d_o);
        p.sc = sc; p.dq = static_cast<uint16_t*>(a.dq);
        p.part = part; p.parts = parts_q; p.scale = scale; p.scale_log2 = scale * kLog2eHost;
        const int grid = grid_of(work_q);
        const WorkList l{q_hdr, q_hdr + kHdrCursor, q_items, head_map_kv(z.hkv, grid)};
        KernelTimer kt("cross_dq", st);
        hipLaunchKernelGGL(hyd_cross_dq_bf16_kernel<D>, dim3(grid), dim3(kDqThreads), kDqLds, st, p, l);
    }
    if (!launched()) return;
    if (parts_q > 1) launch_sum<D>(CrossSum{part, {a.dq, nullptr}, c.cu_q, nullptr, z.nseq, z.Tq, z.hq, parts_q}, false, st);
    if (z.Tk == 0 || !launched()) return;
    {
        CrossBwdParams p;
        memset(&p, 0, sizeof(p));
        p.v = static_cast<const uint16_t*>(a.v);
        p.sc = sc;
        p.dk = static_cast<uint16_t*>(a.dk); p.dv = static_cast<uint16_t*>(a.dv);
        p.T = z.Tq * G; p.hq = z.hkv; p.hkv = z.hkv;
        p.scale = scale; p.scale_log2 = scale * kLog2eHost;
        p.part = part; p.part_max = parts_kv; p.part_rows = z.Tk;
        const int grid = grid_of(work_kv);
        const WorkList l{kv_hdr, kv_hdr + kHdrCursor, kv_items, head_map_kv(z.hkv, grid)};
        KernelTimer kt("cross_dkdv", st);
        hipLaunchKernelGGL((hyd_bwd_dkdv_wide_bf16_kernel<D, CrossBwdParams>), dim3(grid), dim3(kKwThreads), kKwLds, st, p, l);
    }
    if (parts_kv > 1 && launched())
        launch_sum<D>(CrossSum{part, {a.dk, a.dv}, c.cu_kv, c.kv_lens, z.nseq, z.Tk, z.hkv, parts_kv}, false, st);
}

template <int D>
void launch_bwd_f32(const Sizes& z, const CrossShape& c, const BwdArgs& a, float scale, char* ws, size_t ws_bytes, int cus, hipStream_t st) {
    const BwdLayout w = bwd_layout(z);
    float* part = reinterpret_cast<float*>(ws + w.need);
    const size_t room = ws_bytes - w.need, q_rows = (size_t)z.Tq * z.hq, kv_rows = (size_t)z.Tk * z.hkv;
    const int parts_q = bwd_parts(w.n_q * z.hkv, kCus, tiles(z.max_kv, kF32Tile), 1, q_rows, kDqPartRows, (size_t)D * 4, room);
    const int parts_kv = bwd_parts(w.n_kv * z.hkv, kCus, tiles(z.max_q, kF32Tile) * c.G, 2, kv_rows, kKvPartRows, (size_t)D * 8, room);
    int* hdr[2] = {reinterpret_cast<int*>(ws + w.q_hdr), reinterpret_cast<int*>(ws + w.kv_hdr)};
    int* items[2] = {reinterpret_cast<int*>(ws + w.q_items), reinterpret_cast<int*>(ws + w.kv_items)};
    {
        CrossF32Begin b;
        b.c = c; b.dk = static_cast<float*>(a.dk); b.dv = static_cast<float*>(a.dv); b.d = D;
        b.lists[0] = CrossList{hdr[0], items[0], kF32BM, parts_q, (int)(w.n_q * parts_q), false};
        b.lists[1] = CrossList{hdr[1], items[1], kF32KvBN, parts_kv, (int)(w.n_kv * parts_kv), true};
        b.zero = cross_zero(z.nseq, c.kv_lens != nullptr);
        KernelTimer kt("cross_begin", st);
        hipLaunchKernelGGL(hyd_cross_begin_fp32_kernel, dim3(2 + b.zero.n), dim3(kPreludeThreads), kCrossListLds, st, b);
    }
    if (!launched()) return;
    CrossF32Params p;
    memset(&p, 0, sizeof(p));
    p.c = c; p.scale = scale; p.part_o = part;
    p.q = static_cast<const float*>(a.q); p.k = static_cast<const float*>(a.k); p.v = static_cast<const float*>(a.v);
    p.o = static_cast<const float*>(a.o); p.d_o = static_cast<const float*>(a.d_o); p.lse_in = a.lse;
    p.dq = static_cast<float*>(a.dq); p.dk = static_cast<float*>(a.dk); p.dv = static_cast<float*>(a.dv);
    p.D = reinterpret_cast<float*>(ws + w.stat[0]);
    const auto take = [&](int list, long long work) {
        const int grid = (int)(work < 1 ? 1 : (work < cus ? work : cus));
        p.hdr = hdr[list]; p.cursors = hdr[list] + kHdrCursor; p.items = items[list]; p.hm = head_map_kv(z.hkv, grid);
        return grid;
    };
    {
        const int grid = take(0, w.n_q * z.hkv * parts_q);
        p.parts = parts_q;
        KernelTimer kt("cross_dq", st);
        hipLaunchKernelGGL(hyd_cross_dq_fp32_kernel<D>, dim3(grid), dim3(64 * kF32Waves), f32_lds<D>(), st, p);
    }
    if (!launched()) return;
    if (parts_q > 1) launch_sum<D>(CrossSum{part, {a.dq, nullptr}, c.cu_q, nullptr, z.nseq, z.Tq, z.hq, parts_q}, true, st);
    const int grid = take(1, w.n_kv * z.hkv * parts_kv);
    p.parts = parts_kv;
    {
        KernelTimer kt("cross_dkdv", st);
        hipLaunchKernelGGL((parts_kv > 1 ? hyd_cross_dkdv_fp32_kernel<D, true> : hyd_cross_dkdv_fp32_kernel<D, false>), dim3(grid), dim3(64 * kF32KvWaves), f32_lds<D>(), st, p);
    }
    if (parts_kv > 1 && launched()) launch_sum<D>(CrossSum{part, {a.dk, a.dv}, c.cu_kv, c.kv_lens, z.nseq, z.Tk, z.hkv, parts_kv}, true, st);
}

// What both directions check before any HIP call; HYD_OK with *nothing set: there is nothing to do.
hyd_status check_call(const Sizes& z, const int32_t* cu_q, const int32_t* cu_kv, const int32_t* kv_lens, const int32_t* cu_q_host,
                      const int32_t* cu_kv_host, bool pointers, std::initializer_list<const void*> tensors, const void* workspace, size_t bytes, size_t need, bool* nothing) {
    *nothing = (z.Tq == 0 && z.Tk == 0) || z.nseq == 0;
    if (*nothing) return HYD_OK;
    if (z.Tq > 0 && z.max_q == 0) return HYD_ERR_SHAPE;
    if (!cu_q || !cu_kv || !pointers) return HYD_ERR_NULL;
    for (const void* t : tensors)
        if ((uintptr_t)t % 16 != 0) return HYD_ERR_SHAPE;                     // rows are moved 16 bytes at a time
    hyd_status st = check_lengths(cu_q_host, z.nseq, z.Tq, z.max_q, true);
    if (st == HYD_OK) st = check_lengths(cu_kv_host, z.nseq, z.Tk, z.max_kv, kv_lens == nullptr);
    if (st != HYD_OK) return st;
    return !workspace || (uintptr_t)workspace % kAlign != 0 || bytes < need ? HYD_ERR_WORKSPACE : HYD_OK;
}

}  // namespace

extern "C" {

size_t hyd_cross_attn_workspace_bytes(int total_q, int total_kv, int num_seqs, int max_seqlen_q, int max_seqlen_kv, int hq, int hkv,
                                      int head_dim, hyd_dtype dt, int is_bwd) {
    const Sizes z{total_q, total_kv, num_seqs, max_seqlen_q, max_seqlen_kv, hq, hkv, head_dim, dt};
    if (check_sizes(z) != HYD_OK) return 0;
    return is_bwd ? bwd_layout(z).total : fwd_layout(z).total;
}

hyd_status hyd_cross_attn_fwd(const void* q, const void* k, const void* v, const int32_t* cu_q, const int32_t* cu_kv, const int32_t* kv_lens,
                              int num_seqs, const int32_t* cu_q_host, const int32_t* cu_kv_host, int total_q, int total_kv, int max_seqlen_q,
                              int max_seqlen_kv, int hq, int hkv, int head_dim, float softmax_scale, hyd_dtype dt, void* o, float* lse,
                              void* workspace, size_t workspace_bytes, void* hip_stream) {
    const Sizes z{total_q, total_kv, num_seqs, max_seqlen_q, max_seqlen_kv, hq, hkv, head_dim, dt};
    hyd_status st = check_sizes(z);
    if (st != HYD_OK) return st;
    if (total_q == 0) return HYD_OK;
    bool nothing = false;
    st = check_call(z, cu_q, cu_kv, kv_lens, cu_q_host, cu_kv_host, q && o && lse && (total_kv == 0 || (k && v)), {q, k, v, o}, workspace,
                    workspace_bytes, fwd_layout(z).need, &nothing);
    if (st != HYD_OK || nothing) return st;
    int cus = 0;
    if ((st = cross_device(&cus)) != HYD_OK) return st;
    const CrossShape c = shape_of(z, cu_q, cu_kv, kv_lens);
    const auto launch = head_dim == 64 ? launch_fwd<64> : launch_fwd<128>;
    launch(z, c, q, k, v, softmax_scale, o, lse, static_cast<char*>(workspace), workspace_bytes, cus, static_cast<hipStream_t>(hip_stream));
    return hipGetLastError() == hipSuccess ? HYD_OK : HYD_ERR_LAUNCH;
}

hyd_status hyd_cross_attn_bwd(const void* q, const void* k, const void* v, const void* o, const float* lse, const void* d_o,
                              const int32_t* cu_q, const int32_t* cu_kv, const int32_t* kv_lens, int num_seqs, const int32_t* cu_q_host,
                              const int32_t* cu_kv_host, int total_q, int total_kv, int max_seqlen_q, int max_seqlen_kv, int hq, int hkv,
                              int head_dim, float softmax_scale, hyd_dtype dt, void* dq, void* dk, void* dv, void* workspace,
                              size_t workspace_bytes, void* hip_stream) {
    const Sizes z{total_q, total_kv, num_seqs, max_seqlen_q, max_seqlen_kv, hq, hkv, head_dim, dt};
    hyd_status st = check_sizes(z);
    if (st != HYD_OK) return st;
    bool nothing = false;
    st = check_call(z, cu_q, cu_kv, kv_lens, cu_q_host, cu_kv_host,
                    (total_q == 0 || (q && o && lse && d_o && dq)) && (total_kv == 0 || (k && v && dk && dv)),
                    {q, k, v, o, d_o, dq, dk, dv}, workspace, workspace_bytes, bwd_layout(z).need, &nothing);
    if (st != HYD_OK || nothing) return st;
    int cus = 0;
    if ((st = cross_device(&cus)) != HYD_OK) return st;
    const CrossShape c = shape_of(z, cu_q, cu_kv, kv_lens);
    const BwdArgs a{q, k, v, o, lse, d_o, dq, dk, dv};
    const auto launch = dt == HYD_FP32 ? (head_dim == 64 ? launch_bwd_f32<64> : launch_bwd_f32<128>) : (head_dim == 64 ? launch_bwd<64> : launch_bwd<128>);
    launch(z, c, a, softmax_scale, static_cast<char*>(workspace), workspace_bytes, cus, static_cast<hipStream_t>(hip_stream));
    return hipGetLastError() == hipSuccess ? HYD_OK : HYD_ERR_LAUNCH;
}

}  // extern "C"
