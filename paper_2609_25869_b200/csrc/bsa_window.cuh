// What the windowed attention kernels share: who sees whom.
#pragma once
#include <limits.h>

#include "bsa_common.h"
#include "sm100_ptx.cuh"

namespace bsa {

// The device's word that kernels set whose bounded wait expired; read by bsa_window_status.
cudaError_t window_status_word(int device, int** out);

constexpr int kWinT = 128;             // rows and keys of a tile
constexpr int kWinNoLimit = 1 << 29;   // left or right where there is no limit: beyond every position

// A call's sizes and mask.  Positions stay below 2^30, sums of two below 2^31: plain int arithmetic.
struct WindowGeom {
    int batch, heads, heads_kv, group;  // group = heads / heads_kv
    int N, N_kv;
    int left, right, sinks;
    const int32_t* q_start;
    const int32_t* kv_len;
};

struct Sequence {
    int start, len;  // position of row 0, number of keys
};
// (Ordinary loads, not those of the read-only path: a kernel in front may write the two words while this one already runs, up to its
// grid_dependency_wait, and only memory that nobody writes during a kernel's whole life may be read that way.)
__device__ __forceinline__ Sequence load_sequence(const WindowGeom& g, int b) {
    Sequence s;
    s.len = g.kv_len ? min(max(g.kv_len[b], 0), g.N_kv) : g.N_kv;
    s.start = g.q_start ? min(max(g.q_start[b], -kWinNoLimit), kWinNoLimit) : s.len - g.N;
    return s;
}

// The keys that rows [r0, r1) of a sequence see between them: [0, sink_hi) and [lo, hi), sink_hi <= lo; and, for the tiles that
// need no mask, the keys that all of them see: those below all_hi that are sinks or not below all_lo.  Rows at no position of
// the sequence are left out of both.
struct KeyRange {
    int lo, hi, sink_hi;
    int all_lo, all_hi;
};
__device__ __forceinline__ KeyRange key_range(const WindowGeom& g, const Sequence& s, int r0, int r1) {
    KeyRange k;
    const int p0 = max(s.start + r0, 0), p1 = min(s.start + min(r1, g.N), s.len) - 1;
    if (p0 > p1) {
        k.lo = k.hi = k.sink_hi = k.all_lo = k.all_hi = 0;
        return k;
    }
    k.hi = min(s.len, p1 + g.right + 1);
    k.lo = max(0, p0 - g.left);
    k.sink_hi = min(min(g.sinks, k.hi), k.lo);
    k.all_hi = min(s.len, p0 + g.right + 1);
    k.all_lo = p1 - g.left;
    return k;
}
__device__ __forceinline__ bool tile_is_full(const WindowGeom& g, const KeyRange& k, int key0) {
    return key0 + kWinT <= k.all_hi && (key0 >= k.all_lo || key0 + kWinT <= g.sinks);
}

// 128-key tiles of a range: [0, st) and [w0, w1).
struct TileSpan {
    int st, w0, w1;
    __device__ __forceinline__ int count() const { return st + (w1 - w0); }
    __device__ __forceinline__ int tile(int j) const { return j < st ? j : w0 + (j - st); }
};
__device__ __forceinline__ TileSpan tile_span(const KeyRange& k) {
    TileSpan t;
    t.w0 = k.lo / kWinT;
    t.w1 = (k.hi + kWinT - 1) / kWinT;
    t.st = min((k.sink_hi + kWinT - 1) / kWinT, t.w0);
    return t;
}
// The lowest n bits (none for n <= 0, all from 32 on).
__device__ __forceinline__ uint32_t bits_below(int n) {
    uint32_t m;
    asm("bmsk.clamp.b32 %0, 0, %1;" : "=r"(m) : "r"(max(n, 0)));
    return m;
}
// What a row sees of a tile: bounds on the tile's columns, and 32 of them as bits.
struct RowView {
    int hi, lo, sink;
    __device__ __forceinline__ RowView(const WindowGeom& g, const Sequence& s, int pos, int key0)
        : hi(((pos >= 0 && pos < s.len) ? min(s.len, pos + g.right + 1) : 0) - key0), lo(pos - g.left - key0), sink(g.sinks - key0) {}
    __device__ __forceinline__ uint32_t bits(int col) const {
        return bits_below(hi - col) & (~bits_below(lo - col) | bits_below(sink - col));
    }
};
// Hidden scores become -inf: two instructions each (a test of the two bounds branched, 7000 clk a tile).
__device__ __forceinline__ void hide(uint32_t* r, uint32_t bits) {
#pragma unroll
    for (int i = 0; i < 32; ++i) r[i] = (bits & (1u << i)) ? r[i] : 0xff800000u;
}

// Rows of a tile in shared memory that no row of the CTA sees may hold anything, and a weight of zero times NaN would not be zero:
// they become zero themselves (all their 64-column sub-tiles, whatever the swizzle).  Eight of the THREADS to a row, so that a warp's
// stores fall into different banks (with a row to a thread a window's edge tile took 2000 clk more); the caller fences.
template <int D, int THREADS>
__device__ __forceinline__ void zero_rows(uint8_t* tile, int from, int to, int thread) {
    for (int row = max(from, 0) + (thread >> 3); row < min(to, kWinT); row += THREADS / 8)
#pragma unroll
        for (int s = 0; s < D / 64; ++s)
            *reinterpret_cast<uint4*>(tile + s * (kWinT * 128) + row * 128 + (thread & 7) * 16) = make_uint4(0, 0, 0, 0);
}
__device__ __forceinline__ bool has_unseen_keys(const WindowGeom& g, const KeyRange& k, int key0) {
    return k.hi - key0 < kWinT || k.lo - key0 > max(g.sinks - key0, 0);
}
template <int D, int THREADS>
__device__ __forceinline__ void zero_unseen_keys(uint8_t* tile, const WindowGeom& g, const KeyRange& k, int key0, int thread) {
    zero_rows<D, THREADS>(tile, g.sinks - key0, k.lo - key0, thread);
    zero_rows<D, THREADS>(tile, k.hi - key0, kWinT, thread);
}

// The slot of a ring of barriers that comes next, and its phase.
struct Ring {
    int stage = 0;
    uint32_t phase = 0;
    template <int DEPTH>
    __device__ __forceinline__ void advance() {
        if (++stage == DEPTH) {
            stage = 0;
            phase ^= 1u;
        }
    }
};

// Division of non-negative ints by a constant of the call: the items of a persistent CTA are decoded on its critical path.
struct Divisor {
    uint32_t d, mul, shift;
    Divisor() = default;
    explicit Divisor(int n) : d((uint32_t)n), mul(0), shift(0) {
        while ((1ull << shift) < d) ++shift;  // n / d = (n + n * mul / 2^32) / 2^shift
        mul = (uint32_t)((((1ull << shift) - d) << 32) / d + 1);
    }
    __device__ __forceinline__ int div(int n, int& rest) const {
        const uint32_t q = (__umulhi((uint32_t)n, mul) + (uint32_t)n) >> shift;
        rest = n - (int)(q * d);
        return (int)q;
    }
};

// The order of a call's items, tile by tile of every sequence and head ("row" below): the tiles with a whole window first, neighbours of
// one row side by side, so that the CTAs at work share keys in L2 (115200 rows, 24 heads, window 8191: 10.2 ms, 12.0 the other way round);
// then the tiles at the end where the window is cut off, or all of them where there is no left limit: the longest of every row, then the
// next, so that the last items are the shortest (16384 rows, 16 heads, causal window 2048: 254 -> 241 us).
struct ItemOrder {
    Divisor whole, rows;  // tiles of a row with a whole window, rows
    int n_whole;          // items with a whole window
    int n_tiles;          // tiles of a row
    int n_items;
    ItemOrder() = default;
    ItemOrder(int tiles, int cut, int n_rows) : whole(tiles > cut ? tiles - cut : 1), rows(n_rows), n_whole((tiles > cut ? tiles - cut : 0) * n_rows), n_tiles(tiles), n_items(tiles * n_rows) {}
    // item -> row; tile counts from the end of the row where windows are whole
    __device__ __forceinline__ int row_of(int idx, int& tile) const {
        int row;
        if (idx < n_whole) {
            row = whole.div(idx, tile);
        } else {
            tile = (int)whole.d * (n_whole > 0) + rows.div(idx - n_whole, row);
        }
        return row;
    }
};
// Tiles of a sequence's rows whose window is cut off by its beginning, as far as the host knows where they stand.
inline int cut_tiles(const WindowGeom& g, int tiles, int rows = kWinT) {
    const int64_t start = g.q_start || g.kv_len ? 0 : (int64_t)g.N_kv - g.N;
    const int64_t cut = ((int64_t)g.left - start + rows - 1) / rows;
    return (int)(cut < 0 ? 0 : cut > tiles ? tiles : cut);
}

// ---- host side (bsa_window.cu) ----
struct WindowArgs {
    WindowGeom g;
    int d;
    bool f16;
    float scale;
    int device, num_sms;
};
// Checks a description and fills `a` in, all but the device; the current device becomes the call's.
bsa_status_t window_args(const bsa_window_desc_t* t, WindowArgs* a);
bsa_status_t window_device(WindowArgs* a);
// Whether every row of a view with these sizes lies on a 32-byte boundary.
bool view_is_wide(const bsa_view_t& v, int64_t batch, int64_t heads, int64_t rows);
// Whether a call has no more row tiles than the kernels count.
inline bool window_tiles_fit(const WindowArgs& a) { return (int64_t)((a.g.N + kWinT - 1) / kWinT) * a.g.batch * a.g.heads <= INT_MAX / 2; }
// `even`: the rows' windows are about equally long (else their lengths follow from the sizes).  `behind`: the kernel in front on the stream, which writes K, V,
// starts and lengths, lets its dependents start early (grid_launch_dependents) and is waited for on the device.
cudaError_t launch_window_tiles(const WindowArgs& a, const bsa_view_t& Q, const bsa_view_t& K, const bsa_view_t& V, const bsa_view_t& O,
                                float* LSE, bool even, bool behind, cudaStream_t stream);
// Forward for few rows (bsa_window_rows.cu).
cudaError_t launch_window_rows(const WindowArgs& a, const bsa_view_t& Q, const bsa_view_t& K, const bsa_view_t& V, const bsa_view_t& O,
                               float* LSE, cudaStream_t stream);

}  // namespace bsa
