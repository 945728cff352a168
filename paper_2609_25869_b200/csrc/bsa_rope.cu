// Rotary positions with several axes: y = R(t) x pair by pair of channels, t = pos[axis of the pair] * freq[pair].
//
// The kernel is bound by memory: every element is read and written once, 4 bytes of traffic against three operations.  A
// thread owns 8 channels (16 bytes; with paired halves 8 + 8) of one token and walks over heads with them: the pair's
// angle depends on the token alone, so its sine and cosine are computed once and serve every head of Q and K in registers.
// The loads of four heads are issued before the first is used (two: 4 % slower, eight: 1 % faster on the largest call, 5 % slower on
// paired halves).  75600 tokens, 24 + 24 heads, d = 128, token-major: 288 us, 98 % of the rate of a plain copy; one token of 40 heads 2.6 us.
//
// Angles.  A position of 10^6 times a frequency near 1 leaves no correct bit of the angle's fraction in fp32.  The host
// turns each frequency into F = freq / 2 pi in units of 2^-64 turns; pos * F in wrap-around 64-bit integers is the angle
// modulo one turn, off by pos times what F is off: 2^-65 turns of its own rounding, and the frequency's error (below; a given one
// of f radians per position: f 2^-66 turns, from the product with 1 / 2 pi).  For theta = 10^4 and 128 pairs that is pos * 2^-62.3, 2^-31.3
// turns at the last int32 position.  The upper 32 bits become a float in [-1, 1) half turns for sincospif.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include <algorithm>

#include "bsa_common.h"
#include "sm100_ptx.cuh"

namespace bsa {

using namespace ptx;

namespace {

constexpr int kRopeThreads = 256;
constexpr int kMaxPairs = 128;
constexpr int kHeadsInFlight = 4;

struct RopeParams {
    const uint16_t* x[2];  // Q, K
    uint16_t* y[2];
    long long xs_batch[2], xs_head[2], xs_row[2], ys_batch[2], ys_head[2], ys_row[2];
    int heads[2];
    int N, d, pairs;       // pairs = R / 2
    int cols;              // work columns of a token (see the kernel)
    int heads_per_block;   // of heads[0] + heads[1], counted over both tensors
    int n_axes;
    int halves, inverse;
    const int32_t* pos;
    long long pos_batch;
    long long first, grid_tokens;
    int grid[BSA_MAX_AXES], origin[BSA_MAX_AXES];
    unsigned long long freq[kMaxPairs];  // in 2^-64 turns
    unsigned char axis[kMaxPairs];
};

template <bool F16>
__device__ __forceinline__ float2 unpack_16x2(uint32_t v) {
    if (F16) return __half22float2(*reinterpret_cast<const __half2*>(&v));
    // bf16: the upper half of the fp32 pattern
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}

__device__ __forceinline__ uint4 ld_stream(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ void st_stream(void* p, uint4 v) {
    asm volatile("st.global.L1::no_allocate.v4.b32 [%0], {%1,%2,%3,%4};" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// What a thread's column of a token is:
//   interleaved: channels 8c .. 8c+7, four pairs (pairs from R/2 on are copied)
//   halves     : c < pairs/8: channels 8c .. and R/2 + 8c .., eight pairs; columns behind those copy 8 channels from R on
// VEC = false: R/2 is no multiple of 8; a column is one pair, or one channel behind R.
template <bool F16, bool HALVES, bool VEC>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const __grid_constant__ RopeParams p) {
    const int token_slots = kRopeThreads / p.cols;  // tokens of a block
    const int slot = threadIdx.x / p.cols;
    if (slot >= token_slots) return;
    const int c = threadIdx.x - slot * p.cols;
    const long long n = (long long)blockIdx.x * token_slots + slot;
    if (n >= p.N) return;
    const int b = blockIdx.z;

    constexpr int NP = !VEC ? 1 : (HALVES ? 8 : 4);
    const int pair0 = c * NP;
    const bool copies = pair0 >= p.pairs;  // nothing of this column turns
    float cs[NP], sn[NP];
    bool turns = !copies;
    if (turns) {
        int at[BSA_MAX_AXES];
        if (p.pos) {
            const int32_t* src = p.pos + (long long)b * p.pos_batch + n * p.n_axes;
#pragma unroll
            for (int a = 0; a < BSA_MAX_AXES; ++a) at[a] = a < p.n_axes ? __ldg(src + a) : 0;
        } else {
            long long t = n - p.first;
            turns = t >= 0 && t < p.grid_tokens;
            unsigned u = turns ? (unsigned)t : 0u;
#pragma unroll
            for (int a = BSA_MAX_AXES - 1; a >= 0; --a) {
                at[a] = 0;
                if (a < p.n_axes) {
                    const unsigned q = u / (unsigned)p.grid[a];
                    at[a] = (int)(u - q * (unsigned)p.grid[a]) + p.origin[a];
                    u = q;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int pr = min(pair0 + i, p.pairs - 1);
            const int a = p.axis[pr];
            const int position = a == 0 ? at[0] : a == 1 ? at[1] : a == 2 ? at[2] : at[3];
            const unsigned long long turn = (unsigned long long)(long long)position * p.freq[pr];
            sincospif((float)(int)(unsigned)(turn >> 32) * 4.6566128730773926e-10f, &sn[i], &cs[i]);  // * 2^-31 half turns
            if (p.inverse) sn[i] = -sn[i];
        }
    }
    const bool partial = !HALVES && VEC && turns && pair0 + NP > p.pairs;

    const int h0 = blockIdx.y * p.heads_per_block, h1 = min(h0 + p.heads_per_block, p.heads[0] + p.heads[1]);
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        const int base = which ? p.heads[0] : 0;
        const int lo = max(h0 - base, 0), hi = min(h1 - base, p.heads[which]);
        if (lo >= hi) continue;
        const long long xs = p.xs_head[which], ys = p.ys_head[which];
        const uint16_t* x = p.x[which] + (long long)b * p.xs_batch[which] + n * p.xs_row[which] + lo * xs;
        uint16_t* y = p.y[which] + (long long)b * p.ys_batch[which] + n * p.ys_row[which] + lo * ys;
        if constexpr (VEC) {
            const int off0 = copies && HALVES ? 2 * p.pairs + (c - p.pairs / 8) * 8 : c * 8;
            const int off1 = p.pairs + c * 8;  // HALVES: the pairs' second channels
            const bool two = HALVES && !copies;
            for (int h = lo; h < hi; h += kHeadsInFlight, x += kHeadsInFlight * xs, y += kHeadsInFlight * ys) {
                uint4 u[kHeadsInFlight], v[kHeadsInFlight];
#pragma unroll
                for (int k = 0; k < kHeadsInFlight; ++k) {
                    if (h + k >= hi) break;
                    u[k] = ld_stream(x + k * xs + off0);
                    if (two) v[k] = ld_stream(x + k * xs + off1);
                }
#pragma unroll
                for (int k = 0; k < kHeadsInFlight; ++k) {
                    if (h + k >= hi) break;
                    uint32_t* a = reinterpret_cast<uint32_t*>(&u[k]);
                    uint32_t* e = reinterpret_cast<uint32_t*>(&v[k]);
                    if (turns) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if constexpr (HALVES) {
                                const float2 f = unpack_16x2<F16>(a[i]), g = unpack_16x2<F16>(e[i]);
                                a[i] = pack_16x2<F16>(f.x * cs[2 * i] - g.x * sn[2 * i], f.y * cs[2 * i + 1] - g.y * sn[2 * i + 1]);
                                e[i] = pack_16x2<F16>(f.x * sn[2 * i] + g.x * cs[2 * i], f.y * sn[2 * i + 1] + g.y * cs[2 * i + 1]);
                            } else if (!partial || pair0 + i < p.pairs) {
                                const float2 f = unpack_16x2<F16>(a[i]);
                                a[i] = pack_16x2<F16>(f.x * cs[i] - f.y * sn[i], f.x * sn[i] + f.y * cs[i]);
                            }
                        }
                    }
                    st_stream(y + k * ys + off0, u[k]);
                    if (two) st_stream(y + k * ys + off1, v[k]);
                }
            }
        } else {
            const int off0 = copies ? 2 * p.pairs + (c - p.pairs) : c, off1 = p.pairs + c;
            for (int h = lo; h < hi; ++h, x += xs, y += ys) {
                const uint16_t u = x[off0], v = copies ? (uint16_t)0 : x[off1];
                if (turns) {
                    const float2 f = unpack_16x2<F16>((uint32_t)u | ((uint32_t)v << 16));
                    const uint32_t r = pack_16x2<F16>(f.x * cs[0] - f.y * sn[0], f.x * sn[0] + f.y * cs[0]);
                    y[off0] = (uint16_t)r;
                    y[off1] = (uint16_t)(r >> 16);
                } else {
                    y[off0] = u;
                    if (!copies) y[off1] = v;
                }
            }
        }
    }
}

}  // namespace

// A stride that the vector accesses and tensor maps can use; dimensions with one entry have none.
bool view_ok(const bsa_view_t* v, int64_t batch, int64_t heads, int64_t rows) {
    if (!v || !v->data || (reinterpret_cast<uintptr_t>(v->data) & 15)) return false;
    const int64_t n[3] = {batch, heads, rows}, s[3] = {v->batch, v->head, v->row};
    for (int i = 0; i < 3; ++i)
        if (n[i] > 1 && (s[i] <= 0 || (s[i] & 7) || s[i] >= (int64_t(1) << 38))) return false;
    return true;
}

// Whether two entries of a view (view_ok) share an element: for an output, whose entries different threads write.
bool view_overlaps(const bsa_view_t& v, int64_t batch, int64_t heads, int64_t rows, int d) {
    struct { int64_t n, s; } e[3];
    int dims = 0;
    const int64_t n[3] = {batch, heads, rows}, s[3] = {v.batch, v.head, v.row};
    for (int i = 0; i < 3; ++i)
        if (n[i] > 1) e[dims++] = {n[i], s[i]};
    std::sort(e, e + dims, [](const auto& a, const auto& b) { return a.s < b.s; });
    __int128 extent = d;  // of the dimensions so far
    bool nested = true;   // each dimension steps over all of those with smaller strides: every ordinary layout
    for (int i = 0; i < dims; ++i) {
        nested = nested && e[i].s >= extent;
        extent += (__int128)e[i].s * (e[i].n - 1);
    }
    if (nested) return false;
    // Interleaved dimensions may still keep apart.  Two entries meet if their distance i * s0 + j * s1 + k * s2 is below d; of the most
    // numerous dimension only the k nearest to it and its neighbour count, once its own stride is at least d.
    std::sort(e, e + dims, [](const auto& a, const auto& b) { return a.n < b.n; });
    while (dims < 3) {
        for (int i = dims++; i > 0; --i) e[i] = e[i - 1];
        e[0] = {1, 0};
    }
    if (e[2].s < d) return true;
    if ((__int128)e[0].n * e[1].n > (1 << 23)) return true;  // (kept apart, 2^23 to the 3/2 rows of 16 bytes would not fit a GPU)
    for (int64_t i = 0; i < e[0].n; ++i)
        for (int64_t j = i ? 1 - e[1].n : 0; j < e[1].n; ++j) {
            if (i == 0 && j == 0) continue;
            __int128 x = (__int128)i * e[0].s + (__int128)j * e[1].s;
            if (x < 0) x = -x;  // (k takes either sign)
            const __int128 k = x / e[2].s;
            if ((k < e[2].n && x - k * e[2].s < d) || (k + 1 < e[2].n && (k + 1) * e[2].s - x < d)) return true;
        }
    return false;
}

}  // namespace bsa

using namespace bsa;

// the binding packs them as bytes
static_assert(sizeof(bsa_view_t) == 32 && sizeof(bsa_rope_desc_t) == 136 && sizeof(bsa_window_desc_t) == 80, "layout of the C structs");

extern "C" bsa_status_t bsa_rope(const bsa_rope_desc_t* t, const bsa_view_t* Q, const bsa_view_t* K, const bsa_view_t* Q_out,
                                 const bsa_view_t* K_out, void* stream_v) {
    if (!t || t->batch < 1 || t->heads < 1 || t->heads_kv < 0 || t->N < 1 || t->d < 1 || t->n_axes < 1 || t->n_axes > BSA_MAX_AXES)
        return BSA_ERR_INVALID_ARG;
    if ((t->dtype != BSA_DTYPE_BF16 && t->dtype != BSA_DTYPE_FP16) || (t->pairs != BSA_PAIRS_INTERLEAVED && t->pairs != BSA_PAIRS_HALVES))
        return BSA_ERR_INVALID_ARG;
    int64_t R = 0;
    for (int a = 0; a < t->n_axes; ++a) {
        if (t->axis_dim[a] < 0 || (t->axis_dim[a] & 1)) return BSA_ERR_INVALID_ARG;
        R += t->axis_dim[a];
    }
    if (R < 2 || R > t->d) return BSA_ERR_INVALID_ARG;
    if ((t->d & 7) || t->d > 2 * kMaxPairs || t->N > (int64_t(1) << 29) || t->batch > 65535) return BSA_ERR_UNSUPPORTED;
    if (!t->freq_host && !(t->theta > 0.0 && isfinite(t->theta))) return BSA_ERR_INVALID_ARG;
    if (!view_ok(Q, t->batch, t->heads, t->N) || !view_ok(Q_out, t->batch, t->heads, t->N)) return BSA_ERR_INVALID_ARG;
    if (t->heads_kv > 0 && (!view_ok(K, t->batch, t->heads_kv, t->N) || !view_ok(K_out, t->batch, t->heads_kv, t->N)))
        return BSA_ERR_INVALID_ARG;
    if (view_overlaps(*Q_out, t->batch, t->heads, t->N, t->d) || (t->heads_kv > 0 && view_overlaps(*K_out, t->batch, t->heads_kv, t->N, t->d)))
        return BSA_ERR_INVALID_ARG;

    RopeParams p = {};
    p.heads[0] = t->heads;
    p.heads[1] = t->heads_kv;
    p.N = (int)t->N;
    p.d = t->d;
    p.pairs = (int)(R / 2);
    p.n_axes = t->n_axes;
    p.halves = t->pairs == BSA_PAIRS_HALVES;
    p.inverse = t->inverse != 0;
    const bsa_view_t* in[2] = {Q, K};
    const bsa_view_t* out[2] = {Q_out, K_out};
    for (int w = 0; w < (t->heads_kv > 0 ? 2 : 1); ++w) {
        p.x[w] = static_cast<const uint16_t*>(in[w]->data);
        p.y[w] = static_cast<uint16_t*>(out[w]->data);
        p.xs_batch[w] = in[w]->batch; p.xs_head[w] = in[w]->head; p.xs_row[w] = in[w]->row;
        p.ys_batch[w] = out[w]->batch; p.ys_head[w] = out[w]->head; p.ys_row[w] = out[w]->row;
    }
    if (t->pos_dev) {
        if (t->pos_batch < 0 || (reinterpret_cast<uintptr_t>(t->pos_dev) & 3)) return BSA_ERR_INVALID_ARG;
        p.pos = t->pos_dev;
        p.pos_batch = t->pos_batch;
    } else {
        if (t->first < 0) return BSA_ERR_INVALID_ARG;
        p.first = t->first;
        p.grid_tokens = 1;
        for (int a = 0; a < t->n_axes; ++a) {
            if (t->grid[a] < 1 || t->origin[a] > INT32_MAX - (t->grid[a] - 1)) return BSA_ERR_INVALID_ARG;
            p.grid[a] = t->grid[a];
            p.origin[a] = t->origin[a];
            p.grid_tokens *= t->grid[a];
            if (p.grid_tokens > t->N) return BSA_ERR_INVALID_ARG;
        }
        if (p.first > t->N - p.grid_tokens) return BSA_ERR_INVALID_ARG;
    }
    // theta^(-2 i / n) by repeated products in 64-bit mantissas.  The step is off by 2^-63 of itself (a power within one unit), which its
    // i-th power takes i times, and every product by 2^-64: 3 i 2^-64, below 2^-55 for the last of 128.  In turns that is largest where
    // i theta^(-2 i / n) is: 2^-62.7 at theta = 10^4 and 128 pairs, 2^-58 where all frequencies are near 1.
    // (A power for each of 64 pairs cost the host 6 us of a call.)
    int pair = 0;
    long double f = 1.0L;
    const long double step_shared = t->freq_host || !t->shared_freq ? 0.0L : powl((long double)t->theta, -2.0L / (long double)R);
    for (int a = 0; a < t->n_axes; ++a) {
        if (t->axis_dim[a] == 0) continue;
        const long double step = t->freq_host ? 0.0L : t->shared_freq ? step_shared : powl((long double)t->theta, -2.0L / (long double)t->axis_dim[a]);
        if (!t->shared_freq) f = 1.0L;
        for (int i = 0; i < t->axis_dim[a] / 2; ++i, ++pair, f *= step) {
            if (t->freq_host) f = (long double)t->freq_host[pair];
            if (!isfinite(f)) return BSA_ERR_INVALID_ARG;
            long double turns = f * 0.159154943091895335768883763372514362L;
            if (!(turns >= 0.0L && turns < 1.0L)) turns -= floorl(turns);  // whole turns change nothing at whole positions
            const long double units = turns * 18446744073709551616.0L + 0.5L;
            p.freq[pair] = units >= 18446744073709551616.0L ? 0ull : (unsigned long long)units;
            p.axis[pair] = (unsigned char)a;
        }
    }

    const bool vec = !p.halves || p.pairs % 8 == 0;
    p.cols = !vec ? p.pairs + (p.d - 2 * p.pairs) : p.halves ? p.pairs / 8 + (p.d - 2 * p.pairs) / 8 : p.d / 8;
    const int tokens = kRopeThreads / p.cols;
    const int64_t blocks_x = (t->N + tokens - 1) / tokens;
    // Sines and cosines are shared by the heads of a block; the heads are spread over blocks only as far as the GPU is
    // not filled otherwise (eight blocks of 256 threads on each of 148 SMs).
    const int heads = t->heads + t->heads_kv;
    int64_t split = (148 * 8 + blocks_x * t->batch - 1) / (blocks_x * t->batch);
    const int64_t most = (heads + kHeadsInFlight - 1) / kHeadsInFlight;
    if (split > most) split = most;
    if (split < 1) split = 1;
    p.heads_per_block = (int)((heads + split - 1) / split);
    p.heads_per_block = (p.heads_per_block + kHeadsInFlight - 1) / kHeadsInFlight * kHeadsInFlight;
    const dim3 grid((unsigned)blocks_x, (unsigned)((heads + p.heads_per_block - 1) / p.heads_per_block), (unsigned)t->batch);
    const cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_v);
    const bool f16 = t->dtype == BSA_DTYPE_FP16;
    const auto launch = [&](auto kernel) { kernel<<<grid, kRopeThreads, 0, stream>>>(p); };
    if (!p.halves) f16 ? launch(rope_kernel<true, false, true>) : launch(rope_kernel<false, false, true>);
    else if (vec) f16 ? launch(rope_kernel<true, true, true>) : launch(rope_kernel<false, true, true>);
    else f16 ? launch(rope_kernel<true, true, false>) : launch(rope_kernel<false, true, false>);
    count_launch();
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) {
        set_cuda_err(e, "bsa_rope");
        return BSA_ERR_CUDA;
    }
    return BSA_OK;
}
