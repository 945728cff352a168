// Writing the 8-bit cache and reading it back: one pass over the data, bound by memory.
//
// Written: a block of tokens of one head, of K or of V, is the work of up to 256 threads.  All of its new elements are loaded before the first is rounded (64 of
// 16 bits to a thread, in four loads under way at once; 32 in two for blocks of 16 tokens at d = 64), so that the block's largest is found without a second
// look at memory: 2 bytes read and 1 written an element.  (They are 32 of the 64 registers that 1024 threads of an SM have each; all but the shortest
// block's kernels spill 50 to 100 bytes of the rest.)  With the amplitude a = max |x| of the finite elements the scale is 2^e,
//     e = ceil(log2(a / 448)),  from the bits of a: 448 = 1.75 * 2^8, so the exponent of a, less 8, and one more where the
// mantissa is above 1.75.  code = round(x 2^-e): the product is exact, so this is the one rounding.  A block that holds tokens in front of
// the new ones keeps its scale where that is large enough; else those tokens' codes take the larger scale's (x 2^(old - new), again exact
// but for subnormals).
// Read: four times 16 codes to a thread, 32 bytes out for each.
// 115200 tokens, 24 heads, d = 128, blocks of 64 (2.1 GB each way): written in 329 us, 6.45 TB/s, read back in 311, 6.8; token-major 337 and 325; 23400 tokens of
// 12 heads 37 and 35; one token of four sequences, 8 heads 3.1 and 2.1.
#include <cuda_fp16.h>

#include "bsa_cache.cuh"

namespace bsa {

using namespace ptx;

namespace {

// CTAs that are at work together are neighbours in memory: runs of tokens of one head after the other, or, where a token's heads lie side by side, all
// heads of a run (115200 tokens, 24 heads, token-major: 373 -> 337 us written, 380 -> 322 read).
struct GridOrder {
    Divisor inner;
    int by_head;
    GridOrder() = default;
    GridOrder(const CacheGeom& c, int64_t runs) : inner((int)(c.k_head >= c.k_row || c.heads == 1 ? runs : c.heads)), by_head(c.k_head >= c.k_row || c.heads == 1) {}
    __device__ __forceinline__ void of(int i, int& h, int& run, bool& is_v) const {
        int rest;
        is_v = i & 1;
        const int q = inner.div(i >> 1, rest);
        h = by_head ? q : rest;
        run = by_head ? rest : q;
    }
};

struct WriteParams {
    CacheGeom c;
    const uint16_t *K, *V;
    long long k_batch, k_head, k_row, v_batch, v_head, v_row;
    int N;
    int wide;        // rows of K and V lie on 32-byte boundaries
    GridOrder order;
    const int32_t *start, *count;
};

// 32 bytes of global memory from a 16-byte boundary: one load where it is a 32-byte one (`wide`), else two.
__device__ __forceinline__ void ld_global_v8_or_2v4(const void* p, uint4& lo, uint4& hi, int wide) {
    asm volatile(
        "{\n\t.reg .pred w;\n\t"
        "setp.ne.s32 w, %9, 0;\n\t"
        "@w ld.global.nc.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n\t"
        "@!w ld.global.nc.v4.b32 {%0, %1, %2, %3}, [%8];\n\t"
        "@!w ld.global.nc.v4.b32 {%4, %5, %6, %7}, [%8+16];\n\t}"
        : "=r"(lo.x), "=r"(lo.y), "=r"(lo.z), "=r"(lo.w), "=r"(hi.x), "=r"(hi.y), "=r"(hi.z), "=r"(hi.w)
        : "l"(p), "r"(wide));
}

// Positions [p0, p1) of a sequence's rows that count.
__device__ __forceinline__ void rows_of(const int32_t* start, const int32_t* count, int b, int N, int N_kv, int& first, int& p0, int& p1) {
    first = start ? min(max(__ldg(start + b), -kWinNoLimit), kWinNoLimit) : 0;
    const int n = count ? min(max(__ldg(count + b), 0), N) : N;
    p0 = max(first, 0);
    p1 = min(first + n, N_kv);
}

template <bool F16>
__device__ __forceinline__ float2 to_f32x2(uint32_t v) {
    if (F16) return __half22float2(*reinterpret_cast<const __half2*>(&v));
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}

// Threads to a block of tokens: four times 16 elements each, a warp at least; a CTA has as many blocks as make 128 threads (with one to a CTA, blocks
// of 16 tokens took 356 us instead of 332 for 115200 tokens, 24 heads).
template <int D, int B>
constexpr int kBlockThreads = B * D / 64 < 32 ? 32 : B * D / 64;
template <int D, int B>
constexpr int kWriteThreads = kBlockThreads<D, B> < 128 ? 128 : kBlockThreads<D, B>;

template <int D, int B, bool F16>
__global__ void __launch_bounds__(kWriteThreads<D, B>, 1024 / kWriteThreads<D, B>) cache_write_kernel(const __grid_constant__ WriteParams p) {
    constexpr int TB = kBlockThreads<D, B>, PER = kWriteThreads<D, B> / TB, ROW = D / 16, UNITS = B * ROW, U = UNITS / TB;
    static_assert(UNITS % TB == 0, "whole units");
    __shared__ uint32_t most_of[kWriteThreads<D, B> / 32];
    const int tid = threadIdx.x % TB, b = blockIdx.y;
    int h, run, first, p0, p1;
    bool is_v;
    p.order.of(blockIdx.x, h, run, is_v);
    rows_of(p.start, p.count, b, p.N, p.c.N, first, p0, p1);
    const int block = p0 / B + run * PER + threadIdx.x / TB, base = block * B;  // (base below 2^30: block counts from p0 <= 2^29 over N <= 2^29)
    const bool mine = p0 < p1 && base < p1;
    if (PER == 1 ? !mine : !__syncthreads_or(mine)) return;
    const uint16_t* src = (is_v ? p.V + b * p.v_batch + h * p.v_head : p.K + b * p.k_batch + h * p.k_head);
    const long long src_row = is_v ? p.v_row : p.k_row, dst_row = is_v ? p.c.v_row : p.c.k_row;
    uint8_t* dst = is_v ? p.c.V + b * p.c.v_batch + h * p.c.v_head : p.c.K + b * p.c.k_batch + h * p.c.k_head;
    uint8_t* scale = (is_v ? p.c.V_scale : p.c.K_scale) + b * p.c.s_batch + h * p.c.s_head + block;
    const bool keeps = base < p0;
    const int old = keeps && mine ? *scale : 0;
    uint4 x[U][2];
    uint32_t most = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int unit = u * TB + tid, pos = base + unit / ROW;
        x[u][0] = x[u][1] = make_uint4(0, 0, 0, 0);
        if (mine && pos >= p0 && pos < p1) {
            ld_global_v8_or_2v4(src + (long long)(pos - first) * src_row + unit % ROW * 16, x[u][0], x[u][1], p.wide);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 f = to_f32x2<F16>(reinterpret_cast<const uint32_t*>(x[u])[i]);
            const uint32_t lo = __float_as_uint(f.x) & 0x7fffffffu, hi = __float_as_uint(f.y) & 0x7fffffffu;
            most = max(most, max(lo < 0x7f800000u ? lo : 0u, hi < 0x7f800000u ? hi : 0u));
        }
    most = __reduce_max_sync(0xffffffffu, most);
    if (TB > 32) {
        if ((threadIdx.x & 31) == 0) most_of[threadIdx.x >> 5] = most;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < TB / 32; ++w) most = max(most, most_of[threadIdx.x / TB * (TB / 32) + w]);
    }
    if (TB == 32) __syncwarp();  // (all lanes have read the old scale; longer blocks have the barrier above)
    if (!mine) return;
    const int need = scale_code(most);
    const int code = keeps ? max(old, need) : need;
    const float inv = code == 255 ? 0.f : scale_of(254 - code);  // (a block that held 255 stays NaN whatever is written)
    if (tid == 0) *scale = (uint8_t)code;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int unit = u * TB + tid, pos = base + unit / ROW;
        uint4* out = reinterpret_cast<uint4*>(dst + (long long)pos * dst_row + unit % ROW * 16);
        uint32_t w[4];
        if (pos >= p0 && pos < p1) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 f = to_f32x2<F16>(reinterpret_cast<const uint32_t*>(x[u])[2 * i]);
                const float2 g = to_f32x2<F16>(reinterpret_cast<const uint32_t*>(x[u])[2 * i + 1]);
                // (plus x times zero: NaN where x is infinite, which has no code)
                w[i] = f32x2_to_e4m3x2(fmaf(f.x, 0.f, f.x * inv), fmaf(f.y, 0.f, f.y * inv)) |
                       f32x2_to_e4m3x2(fmaf(g.x, 0.f, g.x * inv), fmaf(g.y, 0.f, g.y * inv)) << 16;
            }
            *out = make_uint4(w[0], w[1], w[2], w[3]);
        } else if (pos < p0 && code > old) {
            const uint4 held = *out;
            const float down = __int_as_float(max(127 - (code - old), 0) << 23);  // (zero from 2^-127 on: everything rounds to zero there)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t v = reinterpret_cast<const uint32_t*>(&held)[i];
                const float2 f = to_f32x2<true>(e4m3x2_to_f16x2(v)), g = to_f32x2<true>(e4m3x2_to_f16x2(v >> 16));
                w[i] = f32x2_to_e4m3x2(f.x * down, f.y * down) | f32x2_to_e4m3x2(g.x * down, g.y * down) << 16;
            }
            *out = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}

// Rows of the cache in 16 bits.
struct ReadParams {
    CacheGeom c;
    uint16_t *K, *V;
    long long k_batch, k_head, k_row, v_batch, v_head, v_row;
    int N;           // rows written
    int wide;        // they lie on 32-byte boundaries
    GridOrder order;
    const int32_t *start, *count;
    // what an attention needs instead (WINDOW): the rows' window, the first tokens in front of it
    WindowGeom g;
    int front;                   // rows for the first tokens: a multiple of 128
    int32_t *q_start, *kv_len;   // where the window's rows stand now
};

template <bool F16>
__device__ __forceinline__ uint32_t pack_16x2_sat(float lo, float hi) {  // beyond the type's range its largest number
    uint32_t r;
    if (F16) asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.satfinite.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

constexpr int kReadThreads = 256, kReadUnits = 4;

template <int D, bool F16, bool WINDOW>
__global__ void __launch_bounds__(kReadThreads) cache_read_kernel(const __grid_constant__ ReadParams p) {
    constexpr int ROW = D / 16;
    if (WINDOW) grid_launch_dependents();
    const int b = blockIdx.y;
    int h, run;
    bool is_v;
    p.order.of(blockIdx.x, h, run, is_v);
    int first = 0, p0, p1, sinks = 0, shift = 0;  // rows' positions, and those of them that count: [p0, p1) and [0, sinks)
    if (WINDOW) {
        const Sequence s = load_sequence(p.g, b);
        const KeyRange k = key_range(p.g, s, 0, p.g.N);
        shift = max(k.lo - p.front, 0);  // rows from `front` on stand for positions from front + shift on
        if (p.N == p.c.N) shift = 0;
        p0 = k.lo;
        p1 = k.hi;
        sinks = k.sink_hi;
        if (blockIdx.x == 0 && threadIdx.x == 0) {
            p.q_start[b] = s.start - shift;
            p.kv_len[b] = s.len - shift;
        }
    } else {
        rows_of(p.start, p.count, b, p.N, p.c.N, first, p0, p1);
    }
    const uint8_t* src = is_v ? p.c.V + b * p.c.v_batch + h * p.c.v_head : p.c.K + b * p.c.k_batch + h * p.c.k_head;
    const uint8_t* scale = (is_v ? p.c.V_scale : p.c.K_scale) + b * p.c.s_batch + h * p.c.s_head;
    const long long src_row = is_v ? p.c.v_row : p.c.k_row, dst_row = is_v ? p.v_row : p.k_row;
    uint16_t* dst = is_v ? p.V + b * p.v_batch + h * p.v_head : p.K + b * p.k_batch + h * p.k_head;
    uint4 x[kReadUnits];
    int code[kReadUnits];
    const long long unit0 = (long long)run * (kReadThreads * kReadUnits) + threadIdx.x;
#pragma unroll
    for (int u = 0; u < kReadUnits; ++u) {
        const long long unit = unit0 + u * kReadThreads;
        const int row = (int)min(unit / ROW, (long long)p.N);
        const int pos = WINDOW ? (row < p.front ? row : row + shift) : first + row;
        const bool there = row < p.N && ((pos >= p0 && pos < p1) || (WINDOW && pos < sinks));
        x[u] = make_uint4(0, 0, 0, 0);
        code[u] = there ? 0 : -1;
        if (there) {
            x[u] = __ldg(reinterpret_cast<const uint4*>(src + (long long)pos * src_row + (int)(unit % ROW) * 16));
            code[u] = __ldg(scale + (pos >> p.c.lg_block));
        }
    }
#pragma unroll
    for (int u = 0; u < kReadUnits; ++u) {
        const long long unit = unit0 + u * kReadThreads;
        const int row = (int)min(unit / ROW, (long long)p.N);
        if (row >= p.N || (WINDOW && code[u] < 0)) continue;
        const float f = code[u] < 0 ? 0.f : scale_of(code[u]);
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t v = reinterpret_cast<const uint32_t*>(&x[u])[i];
            const float2 lo = to_f32x2<true>(e4m3x2_to_f16x2(v)), hi = to_f32x2<true>(e4m3x2_to_f16x2(v >> 16));
            w[2 * i] = pack_16x2_sat<F16>(lo.x * f, lo.y * f);
            w[2 * i + 1] = pack_16x2_sat<F16>(hi.x * f, hi.y * f);
        }
        st_global_v8_or_2v4(dst + (long long)row * dst_row + (int)(unit % ROW) * 16, w, p.wide);
    }
}

// CTAs for all runs and heads of K and V; zero: more than a grid takes.
unsigned grid_of(int64_t runs, int heads) { return 2 * runs * heads <= INT_MAX ? (unsigned)(2 * runs * heads) : 0u; }

template <int D, int B>
cudaError_t launch_write(WriteParams p, bool f16, cudaStream_t stream) {
    const int64_t touched = ((int64_t)p.N + B - 2) / B + 1;  // (p0 may stand anywhere in its block)
    constexpr int PER = kWriteThreads<D, B> / kBlockThreads<D, B>;
    const int64_t runs = (touched + PER - 1) / PER;
    const dim3 grid(grid_of(runs, p.c.heads), (unsigned)p.c.batch);
    if (grid.x == 0) return cudaErrorInvalidConfiguration;
    p.order = GridOrder(p.c, runs);
    if (f16) cache_write_kernel<D, B, true><<<grid, kWriteThreads<D, B>, 0, stream>>>(p);
    else cache_write_kernel<D, B, false><<<grid, kWriteThreads<D, B>, 0, stream>>>(p);
    count_launch();
    return cudaGetLastError();
}
template <int D>
cudaError_t launch_write(const WriteParams& p, bool f16, cudaStream_t stream) {
    switch (p.c.lg_block) {
        case 4: return launch_write<D, 16>(p, f16, stream);
        case 5: return launch_write<D, 32>(p, f16, stream);
        case 6: return launch_write<D, 64>(p, f16, stream);
        default: return launch_write<D, 128>(p, f16, stream);
    }
}

template <bool WINDOW>
cudaError_t launch_read(ReadParams p, bool f16, cudaStream_t stream) {
    const int64_t units = (int64_t)p.N * (p.c.d / 16), per = kReadThreads * kReadUnits, runs = (units + per - 1) / per;
    const dim3 grid(grid_of(runs, p.c.heads), (unsigned)p.c.batch);
    if (grid.x == 0) return cudaErrorInvalidConfiguration;
    p.order = GridOrder(p.c, runs);
    if (p.c.d == 64) {
        if (f16) cache_read_kernel<64, true, WINDOW><<<grid, kReadThreads, 0, stream>>>(p);
        else cache_read_kernel<64, false, WINDOW><<<grid, kReadThreads, 0, stream>>>(p);
    } else {
        if (f16) cache_read_kernel<128, true, WINDOW><<<grid, kReadThreads, 0, stream>>>(p);
        else cache_read_kernel<128, false, WINDOW><<<grid, kReadThreads, 0, stream>>>(p);
    }
    count_launch();
    return cudaGetLastError();
}

bool codes_ok(const bsa_view_t& v, const bsa_cache_t& c) {
    if (!view_ok(&v, c.batch, c.heads, c.N)) return false;
    const int64_t n[3] = {c.batch, c.heads, c.N}, s[3] = {v.batch, v.head, v.row};
    for (int i = 0; i < 3; ++i)
        if (n[i] > 1 && (s[i] & 15)) return false;
    return true;
}
bool scales_ok(const bsa_cache_t& c) {
    return c.K_scale && c.V_scale && (c.batch == 1 || (c.scale_batch > 0 && c.scale_batch < (int64_t(1) << 38))) &&
           (c.heads == 1 || (c.scale_head > 0 && c.scale_head < (int64_t(1) << 38)));
}
// Outputs of a write: no two entries in one place, no output in another's.
bool cache_writable(const bsa_cache_t& c, const CacheGeom& g) {
    const bsa_view_t s{c.K_scale, c.scale_batch, c.scale_head, 0};
    return !view_overlaps(c.K, c.batch, c.heads, c.N, c.d) && !view_overlaps(c.V, c.batch, c.heads, c.N, c.d) &&
           !view_overlaps(s, c.batch, c.heads, 1, g.blocks) && c.K.data != c.V.data && c.K_scale != c.V_scale && c.K.data != c.K_scale &&
           c.K.data != c.V_scale && c.V.data != c.K_scale && c.V.data != c.V_scale;
}
bool rows_ok(const bsa_cache_rows_t* r) {
    return r && r->N >= 1 && (r->dtype == BSA_DTYPE_BF16 || r->dtype == BSA_DTYPE_FP16) && r->reserved == 0 &&
           !(reinterpret_cast<uintptr_t>(r->start_dev) & 3) && !(reinterpret_cast<uintptr_t>(r->count_dev) & 3);
}
bsa_status_t cuda_status(cudaError_t e, const char* where) {
    if (e == cudaSuccess) return BSA_OK;
    set_cuda_err(e, where);
    return BSA_ERR_CUDA;
}

// ---- attention: which way a call goes ----
// Few rows: the kernel that spreads the keys over the GPU (bsa_cache_rows.cu).  Rows by the tile: their keys and values in 16 bits first, then the kernel for the
// 16-bit cache; or the kernel that reads the codes (bsa_cache_tiles.cu), which takes longer over a tile, but needs no pass in front and cuts keys into
// parts where the rows leave SMs without work.  By what they would take, in us: few rows, 1.0 (d = 64: 0.7) of an SM for each 16 rows of a key head and 128 keys;
// in 16 bits, 6 bytes an element at 6.4 TB/s for the pass and, whole rounds of items over the SMs, 0.97 (0.82) for 128 rows of a query head and 128 keys;
// from the codes, cache_tiles_time.
// The constants are from calls of one sequence, bf16, head-major, without a window and with all scales equal (376 shapes: 7 of them 16 to 36 % over their best way,
// the rest closer).  Nothing stands for half's third piece of Q, nor for scales that differ, with which the kernel that reads the codes takes 12 to 20 % longer; and
// the tensors' sizes stand for the lengths, which only the device knows.
// Rows of the workspace's K and V: the first tokens (in whole tiles) and the longest window that the queries see between them, or all.
struct Unpacked {
    int64_t rows;
    int front;
};
Unpacked unpacked_rows(const WindowArgs& a) {
    const int64_t front = ((int64_t)a.g.sinks + kWinT - 1) / kWinT * kWinT, rows = front + (int64_t)a.g.left + a.g.right + a.g.N;
    if (rows >= a.g.N_kv) return {a.g.N_kv, 0};
    return {rows, (int)front};
}
int64_t up256(int64_t n) { return (n + 255) / 256 * 256; }
int64_t unpacked_bytes(const WindowArgs& a) {
    const int64_t each = (int64_t)a.g.batch * a.g.heads_kv * unpacked_rows(a).rows * a.d * 2;
    return 2 * up256(each) + up256(8ll * a.g.batch);
}
enum class Way { kRows, kTiles, kUnpacked };
Way way_of(const WindowArgs& a) {
    const int64_t rows = (int64_t)a.g.N * a.g.group;
    if (rows <= 16) return Way::kRows;
    const auto tiles_of = [&](int64_t n) {  // of 128 keys, that n rows see between them
        const int64_t window = (int64_t)a.g.left + a.g.right + a.g.sinks + n;
        return ((window < a.g.N_kv ? window : a.g.N_kv) + kWinT - 1) / kWinT;
    };
    const double per = a.d == 128 ? 0.97 : 0.82;
    const int64_t items = (int64_t)((a.g.N + kWinT - 1) / kWinT) * a.g.batch * a.g.heads;
    const double unpacked = 6.0 * a.g.batch * a.g.heads_kv * (double)unpacked_rows(a).rows * a.d / 6.4e6 + 3.0 +
                            (double)((items + a.num_sms - 1) / a.num_sms) * (tiles_of(kWinT) + 2) * per;
    const double tiles = cache_tiles_time(a);
    const int64_t blocks = (rows + 15) / 16 * a.g.batch * a.g.heads_kv;
    const double few = rows > 512 ? 1e30 : blocks * tiles_of(a.g.N) * (a.d == 128 ? 1.0 : 0.7) / a.num_sms + 8.0;
    return few <= tiles && few <= unpacked ? Way::kRows : tiles <= unpacked ? Way::kTiles : Way::kUnpacked;
}
int64_t workspace_of(const WindowArgs& a, Way way) {
    return way == Way::kRows ? cache_rows_bytes(a) : way == Way::kTiles ? cache_tiles_bytes(a) : unpacked_bytes(a);
}
bsa_status_t forward_unpacked(WindowArgs a, const CacheGeom& g, const bsa_view_t& Q, const bsa_view_t& O, float* LSE, void* workspace, cudaStream_t stream) {
    // The visible keys and values in 16 bits.  Where the window is shorter than the cache its rows move up behind the first tokens; starts and
    // lengths follow, so that who sees whom stays the same.
    const Unpacked u = unpacked_rows(a);
    const int64_t each = (int64_t)a.g.batch * a.g.heads_kv * u.rows * a.d;
    ReadParams p = {};
    p.c = g;
    p.K = static_cast<uint16_t*>(workspace);
    p.V = p.K + up256(2 * each) / 2;
    p.q_start = reinterpret_cast<int32_t*>(p.V + up256(2 * each) / 2);
    p.kv_len = p.q_start + a.g.batch;
    p.k_row = p.v_row = a.d;
    p.k_head = p.v_head = u.rows * a.d;
    p.k_batch = p.v_batch = a.g.heads_kv * p.k_head;
    p.N = (int)u.rows;
    p.wide = 1;
    p.front = u.front;
    p.g = a.g;
    const cudaError_t e = launch_read<true>(p, a.f16, stream);
    if (e != cudaSuccess) return cuda_status(e, "bsa_cache_forward");
    // (a chunk against a longer cache mostly stands at its end, where all items are about as long)
    const bool even = 2 * (int64_t)a.g.N <= a.g.N_kv;
    a.g.N_kv = p.N;
    a.g.q_start = p.q_start;
    a.g.kv_len = p.kv_len;
    const bsa_view_t k{p.K, p.k_batch, p.k_head, p.k_row}, v{p.V, p.v_batch, p.v_head, p.v_row};
    return cuda_status(launch_window_tiles(a, Q, k, v, O, LSE, even, true, stream), "bsa_cache_forward");
}

// What a description of attention and a cache have to agree in.
bsa_status_t forward_args(const bsa_window_desc_t* t, const bsa_cache_t* c, WindowArgs* a, CacheGeom* g) {
    bsa_status_t st = window_args(t, a);
    if (st == BSA_OK) st = cache_geom(c, g);
    if (st == BSA_OK && (t->batch != c->batch || t->heads_kv != c->heads || t->d != c->d || t->N_kv != c->N)) st = BSA_ERR_INVALID_ARG;
    return st;
}

}  // namespace

bsa_status_t cache_geom(const bsa_cache_t* c, CacheGeom* g) {
    if (!c || c->batch < 1 || c->heads < 1 || c->N < 1 || c->d < 1) return BSA_ERR_INVALID_ARG;
    if (c->block != 16 && c->block != 32 && c->block != 64 && c->block != 128) return BSA_ERR_INVALID_ARG;
    if (!codes_ok(c->K, *c) || !codes_ok(c->V, *c) || !scales_ok(*c)) return BSA_ERR_INVALID_ARG;
    if (c->d != 64 && c->d != 128) return BSA_ERR_UNSUPPORTED;
    if (c->N > kWinNoLimit || (int64_t)c->batch * c->heads > 65535) return BSA_ERR_UNSUPPORTED;
    const int lg = c->block == 16 ? 4 : c->block == 32 ? 5 : c->block == 64 ? 6 : 7;
    *g = CacheGeom{c->batch, c->heads, c->d, lg, (int)c->N, (int)((c->N + c->block - 1) >> lg),
                   static_cast<uint8_t*>(c->K.data), static_cast<uint8_t*>(c->V.data), c->K_scale, c->V_scale,
                   c->K.batch, c->K.head, c->K.row, c->V.batch, c->V.head, c->V.row, c->scale_batch, c->scale_head};
    return BSA_OK;
}

}  // namespace bsa

using namespace bsa;

static_assert(sizeof(bsa_cache_t) == 120 && sizeof(bsa_cache_rows_t) == 32, "layout of the C structs");

extern "C" bsa_status_t bsa_cache_write(const bsa_cache_t* c, const bsa_cache_rows_t* r, const bsa_view_t* K, const bsa_view_t* V, void* stream) {
    WriteParams p = {};
    if (!c || !rows_ok(r) || !view_ok(K, c->batch, c->heads, r->N) || !view_ok(V, c->batch, c->heads, r->N)) return BSA_ERR_INVALID_ARG;
    const bsa_status_t st = cache_geom(c, &p.c);
    if (st != BSA_OK) return st;
    for (const void* out : {c->K.data, c->V.data, (void*)c->K_scale, (void*)c->V_scale})
        if (out == K->data || out == V->data) return BSA_ERR_INVALID_ARG;
    if (!cache_writable(*c, p.c)) return BSA_ERR_INVALID_ARG;
    if (r->N > kWinNoLimit) return BSA_ERR_UNSUPPORTED;
    p.K = static_cast<const uint16_t*>(K->data);
    p.V = static_cast<const uint16_t*>(V->data);
    p.k_batch = K->batch; p.k_head = K->head; p.k_row = K->row;
    p.v_batch = V->batch; p.v_head = V->head; p.v_row = V->row;
    p.N = (int)r->N;
    p.wide = view_is_wide(*K, c->batch, c->heads, r->N) && view_is_wide(*V, c->batch, c->heads, r->N);
    p.start = r->start_dev;
    p.count = r->count_dev;
    const bool f16 = r->dtype == BSA_DTYPE_FP16;
    const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    return cuda_status(c->d == 64 ? launch_write<64>(p, f16, s) : launch_write<128>(p, f16, s), "bsa_cache_write");
}

extern "C" bsa_status_t bsa_cache_read(const bsa_cache_t* c, const bsa_cache_rows_t* r, const bsa_view_t* K, const bsa_view_t* V, void* stream) {
    ReadParams p = {};
    if (!c || !rows_ok(r) || !view_ok(K, c->batch, c->heads, r->N) || !view_ok(V, c->batch, c->heads, r->N)) return BSA_ERR_INVALID_ARG;
    const bsa_status_t st = cache_geom(c, &p.c);
    if (st != BSA_OK) return st;
    for (const void* in : {c->K.data, c->V.data, (void*)c->K_scale, (void*)c->V_scale})
        if (in == K->data || in == V->data) return BSA_ERR_INVALID_ARG;
    if (K->data == V->data || view_overlaps(*K, c->batch, c->heads, r->N, c->d) || view_overlaps(*V, c->batch, c->heads, r->N, c->d)) return BSA_ERR_INVALID_ARG;
    if (r->N > kWinNoLimit) return BSA_ERR_UNSUPPORTED;
    p.K = static_cast<uint16_t*>(K->data);
    p.V = static_cast<uint16_t*>(V->data);
    p.k_batch = K->batch; p.k_head = K->head; p.k_row = K->row;
    p.v_batch = V->batch; p.v_head = V->head; p.v_row = V->row;
    p.N = (int)r->N;
    p.wide = view_is_wide(*K, c->batch, c->heads, r->N) && view_is_wide(*V, c->batch, c->heads, r->N);
    p.start = r->start_dev;
    p.count = r->count_dev;
    return cuda_status(launch_read<false>(p, r->dtype == BSA_DTYPE_FP16, reinterpret_cast<cudaStream_t>(stream)), "bsa_cache_read");
}

extern "C" int64_t bsa_cache_workspace_bytes(const bsa_window_desc_t* t, const bsa_cache_t* c) {
    WindowArgs a;
    CacheGeom g;
    if (forward_args(t, c, &a, &g) != BSA_OK || !window_tiles_fit(a) || window_device(&a) != BSA_OK) return 0;
    return workspace_of(a, way_of(a));
}

extern "C" bsa_status_t bsa_cache_forward(const bsa_window_desc_t* t, const bsa_cache_t* c, const bsa_view_t* Q, const bsa_view_t* O, float* LSE,
                                          void* workspace, int64_t workspace_bytes, void* stream_v) {
    WindowArgs a;
    CacheGeom g;
    if (!t || !LSE || (reinterpret_cast<uintptr_t>(LSE) & 3) || !view_ok(Q, t->batch, t->heads, t->N) || !view_ok(O, t->batch, t->heads, t->N))
        return BSA_ERR_INVALID_ARG;
    bsa_status_t st = forward_args(t, c, &a, &g);
    if (st != BSA_OK) return st;
    if (view_overlaps(*O, t->batch, t->heads, t->N, t->d)) return BSA_ERR_INVALID_ARG;
    for (const void* in : {c->K.data, c->V.data, (void*)c->K_scale, (void*)c->V_scale, Q->data})
        if ((O->data == in && in != Q->data) || LSE == in || (workspace && workspace == in)) return BSA_ERR_INVALID_ARG;  // (O may take the place of Q)
    if (LSE == O->data || (workspace && (workspace == O->data || workspace == LSE))) return BSA_ERR_INVALID_ARG;
    if ((st = window_device(&a)) != BSA_OK) return st;
    const cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_v);
    if (!window_tiles_fit(a)) return BSA_ERR_UNSUPPORTED;
    const Way way = way_of(a);
    const int64_t need = workspace_of(a, way);
    if (need && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < need)) return BSA_ERR_INVALID_ARG;
    if (way == Way::kUnpacked) return forward_unpacked(a, g, *Q, *O, LSE, workspace, stream);
    return cuda_status(way == Way::kRows ? launch_cache_rows(a, g, *Q, *O, LSE, workspace, stream) : launch_cache_tiles(a, g, *Q, *O, LSE, workspace, stream),
                       "bsa_cache_forward");
}

extern "C" bsa_status_t bsa_debug_cache_way(const bsa_window_desc_t* t, const bsa_cache_t* c, int* way_out, int* parts_out) {
    WindowArgs a;
    CacheGeom g;
    if (!way_out || !parts_out) return BSA_ERR_INVALID_ARG;
    bsa_status_t st = forward_args(t, c, &a, &g);
    if (st == BSA_OK) st = window_device(&a);
    if (st != BSA_OK) return st;
    const Way way = way_of(a);
    *way_out = way == Way::kRows ? 0 : way == Way::kTiles ? 1 : 2;
    *parts_out = way == Way::kRows ? cache_rows_parts(a) : way == Way::kTiles ? cache_tiles_parts(a) : 1;
    return BSA_OK;
}
