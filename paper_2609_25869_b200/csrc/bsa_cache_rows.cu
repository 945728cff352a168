// Attention over a window of the 8-bit cache: forward for few rows (the next token, a handful of drafted ones, a short chunk).
//
// What bounds it is reading the visible codes once.  As for the 16-bit cache (bsa_window_rows.cu), the keys are spread over the GPU: a cluster of
// CTAs takes up to 16 rows of one key head, every warp walks its own share of the keys in steps of 4 KB (32 keys at d = 128, 64 at d = 64), copied
// by TMA into two rings private to the warp, and the warps' and CTAs' (m, l, O) are joined in shared and distributed shared memory.  Long lists of
// keys are cut into parts besides, a cluster each, whose (m, l, O) a last kernel joins: the GPU is full with one short head and a long cache, and where
// lengths differ the last clusters are short ones.
//
// Per byte there are twice as many elements to multiply as in 16 bits, and each has to be widened first, so the way from shared memory to the
// tensor instruction (mma.sync.m16n8k16 on halves) is kept short:
//   * The products are taken the other way round, S^T = K Q^T and O^T = V^T P^T: the 16 rows of an instruction are keys (channels), its eight columns query
//     rows.  With eight rows of a key head at most (the next token under grouped heads) that is half of the instructions and registers that 16
//     query rows would take (600 -> 460 instructions for 32 keys with all else; one sequence of 65536 keys, 8 key heads 61 -> 43 us); up to 16 have two such
//     columns (NB).
//   * The order of the channels inside a product is free as long as Q has it too, and so is the order of the keys and that of the output's
//     channels.  A lane takes 16 channels of one key (K Q^T) or of four keys (V^T P^T) with one 16-byte load, and two neighbouring codes are
//     one instruction away from a fragment's register: K's are neighbours in memory, V's (two keys of one channel) after a byte permutation.
//   * Which key stands behind row n of a product (key_even, kOdd) is chosen so that both kinds of load are free of bank conflicts.
//   * e4m3 widens to half exactly.  Q comes as bf16 or half; a row of bf16 is multiplied by the power of two that takes its largest element to
//     2^14 .. 2^15, and its elements down to 2^-31 of that one keep all their bits (what is lost below is at most 2^-39 of it).
//   * Scales stay out of the products: scores are multiplied by their block's power of two; V's goes into the exponent of its keys' weights,
//     relative to the largest so far of the warp's keys, which the accumulator is in units of.  P and its sum stay fp32 until P is rounded to half: 2^15 P times
//     the relative scale, off by 2^-25 at most below half's normal numbers, so by 2^-40 of 448 times the largest scale for each key.
// Eight sequences of 65536 keys, 8 key heads under 32, d = 128, one token: 178 us for 1.07 GB, 6.0 TB/s (94 % of what a copy has); six of 1111 to 115200
// keys 129 us, 5.3 TB/s (token-major; the 16-bit cache 239); four with a window of 1024 keys 7 us, latencies.
#include <cuda_fp16.h>
#include <float.h>
#include <math.h>

#include <atomic>
#include <type_traits>

#include "bsa_cache.cuh"

namespace bsa {

using namespace ptx;

namespace {

constexpr int kWarps = 6;
constexpr int kRing = 8192;  // bytes of a warp's K or V ring
constexpr int kSlot = 4096;
constexpr int kSlots = kRing / kSlot;
constexpr int kMaxC = 8;  // CTAs of a cluster (the join's loads are written out)
constexpr int kMaxParts = 16;
constexpr unsigned kAll = 0xffffffffu;
// P, at most one, is computed 2^15 times as large (half ends at 2^16), so that less of it falls below 2^-14.
constexpr float kShift = 15.0f;
// A block of V whose scale is 2^100 below the largest of the warp's adds nothing that half could hold.
constexpr int kFar = 100;

struct Params {
    WindowGeom g;
    const uint16_t* Q;
    uint16_t* O;
    float* LSE;
    long long q_batch, q_head, q_row, o_batch, o_head, o_row;
    const uint8_t *k_scale, *v_scale;
    long long s_batch, s_head;
    int lg_block, last_block;
    int parts;
    float* part_O;     // [parts][batch][heads][N][D]
    float2* part_ml;   // [parts][batch][heads][N]: maximum (log2 domain), sum
    float scale_log2;
    int n_rows;    // N * group
    int withhold;  // test hook: no copy of a warp's first tile of V
    int* status;
};

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t map_to_rank(uint32_t smem, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem), "r"(rank));
    return r;
}
// 16 (8) bytes to another CTA's shared memory; they count at a barrier there.
__device__ __forceinline__ void send(uint32_t to, const float4& v, uint32_t bar) {
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(to), "r"(__float_as_uint(v.x)),
                 "r"(__float_as_uint(v.y)), "r"(__float_as_uint(v.z)), "r"(__float_as_uint(v.w)), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void send(uint32_t to, const float2& v, uint32_t bar) {
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.b32 [%0], {%1, %2}, [%3];" ::"r"(to), "r"(__float_as_uint(v.x)),
                 "r"(__float_as_uint(v.y)), "r"(bar)
                 : "memory");
}
// (Not volatile, as loads from the ring are plain ones: the compiler may put other products and loads between those that depend on each other.
// In program order a step took 5000 clk of a warp that had its SM's quarter nearly to itself.)
__device__ __forceinline__ void mma(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// P as a product's columns has keys along the rows of 8 x 8 pieces; P^T as an operand has them along the columns.
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t v) {
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}

// The keys of eight behind rows 2t and 2t + 1 of a product.  Rows of the ring lie D bytes apart, their 16-byte chunks XORed with the row's low bits (d = 128:
// three, of 128 bytes; d = 64: bits 1 and 2, of 64 bytes, two rows to 128 bytes).  Eight lanes of a 16-byte load of K have two rows of the product, 2j and 2j + 1,
// and four chunks; of V they have the four even (odd) ones and two chunks (d = 64: sixteen lanes, four half chunks).
template <int D>
__device__ __forceinline__ int key_even(int t) { return D == 128 ? 2 * t : (t & 1) | ((t & 2) << 1); }
template <int D>
constexpr int kOdd = D == 128 ? 5 : 3;  // the odd row's key is the even one's XOR this
template <int D>
__device__ __forceinline__ uint32_t chunk_at(int row, int chunk) {
    return (uint32_t)(row * D + ((chunk ^ (D == 128 ? row & 7 : (row >> 1) & 3)) << 4));
}
// Where 16-byte piece c of a row of the partial sums lies: eight lanes write two pieces (D / 32 apart) of four even or odd rows.
template <int D>
__device__ __forceinline__ int piece_at(int row, int c) {
    return D == 128 ? c ^ ((row >> 1) & 3) : c ^ (((row >> 1) & 1) | (row & 4));
}

// NB: query rows of a cluster by eight.
template <int D, bool F16, int NB>
__global__ void __launch_bounds__(kWarps * 32, 2)
cache_rows_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ Params p) {
    constexpr int KS = kSlot / D;  // keys per step
    constexpr int G = KS / 16;     // groups of 16 keys, the shortest block
    constexpr int ROWS = 8 * NB, KS_QK = D / 16, MT_O = D / 16, HALVES = D / 64;
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ __align__(8) uint64_t bars[kWarps][2 * kSlots];  // K slots, then V slots: the copy has landed
    __shared__ float wm[kWarps][ROWS], wl[kWarps][ROWS];        // the warps' maxima (log2 domain) and sums
    // What the cluster's CTAs send to this one: their sums of this one's share of the rows, [C][ROWS * D / C], and their maxima and weights' sums.
    __shared__ __align__(16) float in_sum[ROWS * D];
    __shared__ __align__(8) float2 in_ml[kMaxC][ROWS];
    __shared__ __align__(8) uint64_t in_bar;
    __shared__ uint32_t abort_flag;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gid = lane >> 2, t = lane & 3;
    const int C = gridDim.x, rank = blockIdx.x;
    const int b = blockIdx.z / p.g.heads_kv, hk = blockIdx.z - b * p.g.heads_kv, key_part = blockIdx.y % p.parts, row0 = blockIdx.y / p.parts * ROWS;
    // Everything that does not wait for something else is on its way first: lengths, then Q (behind the copies it came 6000 clk later), then barriers.
    const Sequence seq = load_sequence(p.g, b);
    // Q^T fragments (B operand, 16 channels x 8 rows per step) of row gid of each eight: positions 2t, 2t + 1, 2t + 8, 2t + 9 of product x * 4 + y
    // are channels x * 64 + t * 16 + y * 4 .. + 3.
    uint32_t qb[NB][KS_QK][2];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int r = row0 + nb * 8 + gid;
        const int n = r / p.g.group, h = hk * p.g.group + (r - n * p.g.group);
        const uint16_t* q = p.Q + (long long)b * p.q_batch + (long long)h * p.q_head + (long long)n * p.q_row;
#pragma unroll
        for (int x = 0; x < HALVES; ++x)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const uint4 v = r < p.n_rows ? __ldg(reinterpret_cast<const uint4*>(q + x * 64 + t * 16 + y * 8)) : make_uint4(0, 0, 0, 0);
                const int ks = x * 4 + y * 2;
                qb[nb][ks][0] = v.x;
                qb[nb][ks][1] = v.y;
                qb[nb][ks + 1][0] = v.z;
                qb[nb][ks + 1][1] = v.w;
            }
    }
    const uint32_t sK = smem_u32(smem) + warp * 2 * kRing, sV = sK + kRing;
    const uint32_t bK = smem_u32(&bars[warp][0]), bV = bK + kSlots * 8;
    const int per = ROWS * D / C;  // (C divides it) this CTA's share of the outputs, in the partial sums' order
    if (threadIdx.x == 0) {
        abort_flag = 0;
        mbar_init(smem_u32(&in_bar), 1);
    }
    if (lane == 0) {
        prefetch_tensormap(&tmK);
        prefetch_tensormap(&tmV);
        for (int i = 0; i < 2 * kSlots; ++i) mbar_init(bK + i * 8, 1);
        fence_mbar_init();
    }
    if (threadIdx.x == 0) mbar_arrive_expect_tx(smem_u32(&in_bar), C * (per * 4 + ROWS * 8));
    __syncthreads();
    cluster_arrive();  // (waited for in front of the first thing sent)
    volatile uint32_t* abortp = &abort_flag;

    // Row r of the key head is query token r / group under query head hk * group + r % group.
    const int n0 = row0 / p.g.group, n1 = min((row0 + ROWS - 1) / p.g.group + 1, p.g.N);
    const KeyRange range = key_range(p.g, seq, n0, n1);
    // steps of KS keys: [0, st) and [w0, w1), as the tiles of the other kernel
    const int w0 = range.lo / KS, w1 = (range.hi + KS - 1) / KS, st = min((range.sink_hi + KS - 1) / KS, w0);
    const int steps = st + (w1 - w0);
    // The CTA's share of them is one run, its warps take turns.
    const long long share = (long long)p.parts * C, mine = (long long)key_part * C + rank;
    const int first = (int)(steps * mine / share) + warp, last = (int)(steps * (mine + 1) / share);
    auto key_of = [&](int j) { return (j < st ? j : w0 + (j - st)) * KS; };
    auto copy_in = [&](uint32_t dst, const CUtensorMap* map, uint32_t bar, int key0) {
        mbar_arrive_expect_tx(bar, kSlot);
        tma_load_4d(dst, map, bar, 0, key0, hk, b);
    };
    if (lane == 0) {
        for (int i = 0; i < kSlots && first + i * kWarps < last; ++i) {
            copy_in(sK + i * kSlot, &tmK, bK + i * 8, key_of(first + i * kWarps));
            if (!(p.withhold && i == 0)) copy_in(sV + i * kSlot, &tmV, bV + i * 8, key_of(first + i * kWarps));
        }
    }
    // A step's scales: lanes 0 .. G - 1 have K's, lanes 16 .. 16 + G - 1 V's, a step ahead.
    const uint8_t* scales = (lane < 16 ? p.k_scale : p.v_scale) + b * p.s_batch + hk * p.s_head;
    auto load_scale = [&](int j) -> int {
        return (lane & 15) < G ? (int)__ldg(scales + min((key_of(j) + (lane & 15) * 16) >> p.lg_block, p.last_block)) : 0;
    };
    int next_code = first < last ? load_scale(first) : 0;
    float c2[NB][2];  // what takes the products of rows 2t and 2t + 1 to scores (log2 domain), but for K's scale
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        float factor = p.scale_log2;
        if (!F16) {
            uint32_t most = 0;
#pragma unroll
            for (int ks = 0; ks < KS_QK; ++ks)
#pragma unroll
                for (int k = 0; k < 2; ++k) most = max(most, max((qb[nb][ks][k] >> 7) & 0xffu, (qb[nb][ks][k] >> 23) & 0xffu));
            most = max(most, __shfl_xor_sync(kAll, most, 1));
            most = max(most, __shfl_xor_sync(kAll, most, 2));
            const int field = min(268 - (int)most, 253);  // of the factor that takes exponent most - 127 to 14, and of a finite inverse
            const float up = __int_as_float(field << 23);
            factor *= __int_as_float((254 - field) << 23);
#pragma unroll
            for (int ks = 0; ks < KS_QK; ++ks)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint32_t w = qb[nb][ks][k];
                    qb[nb][ks][k] = pack_f16x2(__uint_as_float(w << 16) * up, __uint_as_float(w & 0xffff0000u) * up);
                }
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) c2[nb][e] = __shfl_sync(kAll, factor, (2 * t + e) * 4);
    }
    float o[NB][MT_O][4];
    float m[NB][2], l[NB][2];  // maxima of rows 2t, 2t + 1, this thread's share of their sums
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
        for (int i = 0; i < MT_O; ++i) o[nb][i][0] = o[nb][i][1] = o[nb][i][2] = o[nb][i][3] = 0.f;
        m[nb][0] = m[nb][1] = -INFINITY;
        l[nb][0] = l[nb][1] = 0.f;
    }
    int v_unit = 0;  // the accumulator counts in 2^(v_unit - 127): the largest scale so far
    int slot = 0;
    uint32_t phase = 0;
    bool ok = true;
    const int ke = key_even<D>(t), ko = ke ^ kOdd<D>;                                // the keys behind rows 2t and 2t + 1 of a product
    const int kg = key_even<D>((gid >> 1) & 3) ^ ((gid & 1) ? kOdd<D> : 0);  // and behind row gid
    for (int j = first; j < last; j += kWarps) {
        const int key0 = key_of(j);
        const uint32_t cK = sK + slot * kSlot, cV = sV + slot * kSlot;
        const uint8_t *gK = smem + warp * 2 * kRing + slot * kSlot, *gV = gK + kRing;
        const int code = next_code;
        if (j + kWarps < last) next_code = load_scale(j + kWarps);
        ok = mbar_wait_warp(bK + slot * 8, phase, abortp);
        if (!ok) break;
        float s[G][NB][4];  // keys kg, kg + 8 of a group x rows 2t, 2t + 1
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) s[g][nb][0] = s[g][nb][1] = s[g][nb][2] = s[g][nb][3] = 0.f;
#pragma unroll
        for (int x = 0; x < HALVES; ++x) {
            uint4 w[2 * G];
#pragma unroll
            for (int n = 0; n < 2 * G; ++n) w[n] = *reinterpret_cast<const uint4*>(gK + chunk_at<D>(n * 8 + kg, x * 4 + t));
#pragma unroll
            for (int y = 0; y < 4; ++y)
#pragma unroll
                for (int g = 0; g < G; ++g) {  // (groups inside: neighbours do not depend on each other)
                    const uint4 &u = w[2 * g], &v = w[2 * g + 1];
                    uint32_t a[4];
                    e4m3x4_to_f16x4(y == 0 ? u.x : y == 1 ? u.y : y == 2 ? u.z : u.w, a[0], a[2]);
                    e4m3x4_to_f16x4(y == 0 ? v.x : y == 1 ? v.y : y == 2 ? v.z : v.w, a[1], a[3]);
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) mma(s[g][nb], a, qb[nb][x * 4 + y][0], qb[nb][x * 4 + y][1]);
                }
        }
        __syncwarp();  // every lane has read the K slot
        if (lane == 0 && j + kSlots * kWarps < last) copy_in(cK, &tmK, bK + slot * 8, key_of(j + kSlots * kWarps));
        int vc[G];  // V's codes; of groups that nobody here sees, zero
        int v_most = v_unit;
        const bool full = key0 + KS <= range.all_hi && (key0 >= range.all_lo || key0 + KS <= p.g.sinks);
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const float f = scale_of(__shfl_sync(kAll, code, g));
            vc[g] = __shfl_sync(kAll, code, 16 + g);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float c = c2[nb][e] * f;
                    c = c > FLT_MAX ? FLT_MAX : c;  // (so that a product of zero stays a score of zero)
                    s[g][nb][e] *= c;
                    s[g][nb][2 + e] *= c;
                }
            const int k = key0 + 16 * g;
            if (!full && (k >= range.hi || (k + 16 <= range.lo && k >= range.sink_hi))) vc[g] = 0;
            v_most = max(v_most, vc[g] == 255 ? 0 : vc[g]);
        }
        ok = mbar_wait_warp(bV + slot * 8, phase, abortp);
        if (!ok) break;
        if (!full) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int r = row0 + nb * 8 + 2 * t + e;
                    const RowView view(p.g, seq, r < p.n_rows ? seq.start + r / p.g.group : -1, key0);
#pragma unroll
                    for (int w = 0; w < KS / 32; ++w) {
                        const uint32_t bits = view.bits(w * 32) >> kg;
#pragma unroll
                        for (int g = 2 * w; g < 2 * w + 2; ++g) {
                            if (!((bits >> (g & 1) * 16) & 1)) s[g][nb][e] = -INFINITY;
                            if (!((bits >> ((g & 1) * 16 + 8)) & 1)) s[g][nb][2 + e] = -INFINITY;
                        }
                    }
                }
            // V rows that no row here sees may hold anything: their weight is zero, which times NaN would not be
            for (int k = lane; k < KS; k += 32) {
                const int key = key0 + k;
                if (key >= range.hi || (key < range.lo && key >= p.g.sinks)) {
#pragma unroll
                    for (int c = 0; c < D / 16; ++c)
                        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(cV + k * D + c * 16), "r"(0) : "memory");
                }
            }
            fence_proxy_async_smem();  // before the slot's next copy
            __syncwarp();
        }
        float mx[NB][2];
        bool grows = false;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                mx[nb][e] = -INFINITY;
#pragma unroll
                for (int g = 0; g < G; ++g) mx[nb][e] = max3(mx[nb][e], s[g][nb][e], s[g][nb][2 + e]);
                grows |= mx[nb][e] > m[nb][e];
            }
        if (__any_sync(kAll, grows) || v_most > v_unit) {
            const float unit = ex2_approx((float)(v_unit - v_most));
            v_unit = v_most;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                float u[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
#pragma unroll
                    for (int x = 4; x < 32; x *= 2) mx[nb][e] = fmaxf(mx[nb][e], __shfl_xor_sync(kAll, mx[nb][e], x));
                    const float mn = fmaxf(m[nb][e], mx[nb][e]), a = (m[nb][e] == -INFINITY) ? 0.f : ex2_approx(m[nb][e] - mn);
                    m[nb][e] = mn;
                    l[nb][e] *= a;
                    u[e] = a * unit;
                }
#pragma unroll
                for (int i = 0; i < MT_O; ++i) {
                    o[nb][i][0] *= u[0];
                    o[nb][i][1] *= u[1];
                    o[nb][i][2] *= u[0];
                    o[nb][i][3] *= u[1];
                }
            }
        }
        float nm[NB][2];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int e = 0; e < 2; ++e) nm[nb][e] = (m[nb][e] == -INFINITY) ? 0.f : kShift - m[nb][e];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int dv = max(vc[g] - v_unit, -kFar);
            const float up = vc[g] == 255 ? NAN : (float)dv, down = __int_as_float((127 - dv) << 23);  // (255: dv is not used)
            uint32_t pb[NB][2];  // P^T as the B operand of V^T P^T
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const float n0 = nm[nb][0] + up, n1 = nm[nb][1] + up;
                const float p0 = ex2_approx(s[g][nb][0] + n0), p1 = ex2_approx(s[g][nb][1] + n1);
                const float p2 = ex2_approx(s[g][nb][2] + n0), p3 = ex2_approx(s[g][nb][3] + n1);
                l[nb][0] = fmaf(p0 + p2, down, l[nb][0]);
                l[nb][1] = fmaf(p1 + p3, down, l[nb][1]);
                pb[nb][0] = transpose_8x8(pack_f16x2(p0, p1));
                pb[nb][1] = transpose_8x8(pack_f16x2(p2, p3));
            }
            // V of the keys behind rows 2t, 2t + 1, 2t + 8, 2t + 9, channels gid * D / 8 ..
            uint32_t v[4][D / 32];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int key = g * 16 + (i >> 1) * 8 + ((i & 1) ? ko : ke);
                if constexpr (D == 128) {
                    const uint4 x = *reinterpret_cast<const uint4*>(gV + chunk_at<D>(key, gid));
                    v[i][0] = x.x, v[i][1] = x.y, v[i][2] = x.z, v[i][3] = x.w;
                } else {
                    const uint2 x = *reinterpret_cast<const uint2*>(gV + chunk_at<D>(key, gid >> 1) + (gid & 1) * 8);
                    v[i][0] = x.x, v[i][1] = x.y;
                }
            }
#pragma unroll
            for (int w = 0; w < D / 32; ++w) {  // four channels: rows gid and gid + 8 of two products
                uint32_t a[4], c[4];
                e4m3x4_to_f16x4(__byte_perm(v[0][w], v[1][w], 0x5140), a[0], a[1]);
                e4m3x4_to_f16x4(__byte_perm(v[2][w], v[3][w], 0x5140), a[2], a[3]);
                e4m3x4_to_f16x4(__byte_perm(v[0][w], v[1][w], 0x7362), c[0], c[1]);
                e4m3x4_to_f16x4(__byte_perm(v[2][w], v[3][w], 0x7362), c[2], c[3]);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    mma(o[nb][2 * w], a, pb[nb][0], pb[nb][1]);
                    mma(o[nb][2 * w + 1], c, pb[nb][0], pb[nb][1]);
                }
            }
        }
        __syncwarp();  // every lane has read the V slot
        if (lane == 0 && j + kSlots * kWarps < last) copy_in(cV, &tmV, bV + slot * 8, key_of(j + kSlots * kWarps));
        if (++slot == kSlots) {
            slot = 0;
            phase ^= 1u;
        }
    }
    if (!ok) let_copies_land();  // before the rings are used for anything else (a warp that came to its end has waited for all of its own)
    // ---- join the warps: weights first, then the rows, scaled, into shared memory ----
    constexpr float kBack = 1.f / 32768.f;  // 2^-kShift
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int x = 4; x < 32; x *= 2) l[nb][e] += __shfl_xor_sync(kAll, l[nb][e], x);
            if (gid == 0) {
                wm[warp][nb * 8 + 2 * t + e] = m[nb][e];
                wl[warp][nb * 8 + 2 * t + e] = l[nb][e] * kBack;
            }
        }
    __syncthreads();  // (every warp's ring is idle from here on)
    const float unit = scale_of(v_unit);
    // [warp][row][D], a lane's D / 8 consecutive channels of two rows in pieces of 16 bytes (see piece_at)
    float* part = reinterpret_cast<float*>(smem) + warp * ROWS * D;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = nb * 8 + 2 * t + e;
            float M = -INFINITY;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) M = fmaxf(M, wm[w][r]);
            const float f = m[nb][e] == -INFINITY ? 0.f : ex2_approx(m[nb][e] - M) * kBack;
#pragma unroll
            for (int i = 0; i < MT_O; i += 2) {
                const float4 x = make_float4(o[nb][i][e] * f * unit, o[nb][i][2 + e] * f * unit, o[nb][i + 1][e] * f * unit, o[nb][i + 1][2 + e] * f * unit);
                *reinterpret_cast<float4*>(part + r * D + piece_at<D>(r, gid * (D / 32) + i / 2) * 4) = x;
            }
        }
    __syncthreads();
    // ---- join the CTAs of the cluster: each sends the others their shares, and writes its own of the outputs ----
    cluster_wait();  // all have started: their barriers are there
    const uint32_t a_sum = smem_u32(in_sum), a_ml = smem_u32(in_ml), a_bar = smem_u32(&in_bar);
    for (int i = threadIdx.x * 4; i < ROWS * D; i += kWarps * 32 * 4) {
        const float* x = reinterpret_cast<const float*>(smem) + i;
        float4 a = *reinterpret_cast<const float4*>(x);
#pragma unroll
        for (int w = 1; w < kWarps; ++w) {
            const float4 y = *reinterpret_cast<const float4*>(x + w * ROWS * D);
            a.x += y.x;
            a.y += y.y;
            a.z += y.z;
            a.w += y.w;
        }
        const int q = i / per;
        send(map_to_rank(a_sum + (rank * per + i - q * per) * 4, q), a, map_to_rank(a_bar, q));
    }
    for (int i = threadIdx.x; i < C * ROWS; i += kWarps * 32) {
        const int q = i / ROWS, r = i % ROWS;
        float M = -INFINITY, L = 0.f;
        for (int w = 0; w < kWarps; ++w) M = fmaxf(M, wm[w][r]);
        // (a maximum of -inf: nothing seen, the sum is zero, or nothing but NaN, which the maximum passes over and the sum keeps)
        for (int w = 0; w < kWarps; ++w) L += wm[w][r] == -INFINITY ? wl[w][r] : wl[w][r] * ex2_approx(wm[w][r] - M);
        send(map_to_rank(a_ml + (rank * ROWS + r) * 8, q), make_float2(M, L), map_to_rank(a_bar, q));
    }
    __syncwarp();
    cluster_arrive();
    ok = mbar_wait_warp(a_bar, 0, abortp);
    for (int i = threadIdx.x * 4; ok && i < per; i += kWarps * 32 * 4) {
        const int at_all = rank * per + i, r = at_all / D, c = piece_at<D>(r, (at_all - r * D) >> 2) * 4;  // element at_all of the stored order is column c
        float M = -INFINITY, L = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int q = 0; q < kMaxC; ++q)
            if (q < C) M = fmaxf(M, in_ml[q][r].x);
#pragma unroll
        for (int q = 0; q < kMaxC; ++q) {
            if (q >= C) continue;
            const float2 ml = in_ml[q][r];
            const float4 x = *reinterpret_cast<const float4*>(in_sum + q * per + i);
            const float f = ml.x == -INFINITY ? 0.f : ex2_approx(ml.x - M);
            L = fmaf(f, ml.y, L);
            v.x = fmaf(f, x.x, v.x);
            v.y = fmaf(f, x.y, v.y);
            v.z = fmaf(f, x.z, v.z);
            v.w = fmaf(f, x.w, v.w);
        }
        const int row = row0 + r;
        if (row < p.n_rows) {
            const int n = row / p.g.group, h = hk * p.g.group + (row - n * p.g.group);
            const long long where = ((long long)b * p.g.heads + h) * p.g.N + n;
            if (p.parts > 1) {
                const long long there = (long long)key_part * p.g.batch * p.g.heads * p.g.N + where;
                *reinterpret_cast<float4*>(p.part_O + there * D + c) = v;
                if (c == 0) p.part_ml[there] = make_float2(M, L);
                continue;
            }
            const int at = seq.start + n;
            // Decided by the position alone: a row at a position sees its own key at least, and a sum that is NaN belongs to its outputs.
            // (A row at none may have a sum: steps that the rows of the sequence see whole are not masked.)
            const bool any = at >= 0 && at < seq.len;
            const float inv = any ? 1.f / L : 0.f;
            *reinterpret_cast<uint2*>(p.O + (long long)b * p.o_batch + (long long)h * p.o_head + (long long)n * p.o_row + c) =
                any ? make_uint2(pack_16x2<F16>(v.x * inv, v.y * inv), pack_16x2<F16>(v.z * inv, v.w * inv)) : make_uint2(0u, 0u);
            if (c == 0) p.LSE[where] = any ? fmaf(M, 0.6931471805599453f, logf(L)) : -INFINITY;
        }
    }
    if (!ok) let_copies_land();  // (and what is still on its way here)
    if (threadIdx.x == 0 && abort_flag) atomicExch(p.status, (int)BSA_ERR_DEVICE_TIMEOUT);
    __syncwarp();
    cluster_wait();  // all have sent: nobody leaves while it is sent something
}

// How a call is spread over the GPU, and where its workspace has what.
struct Plan {
    int C, parts, blocks;
    int64_t part_ml, bytes;  // the partial sums' offset is zero
};
Plan plan_of(const WindowArgs& a) {
    Plan w = {};
    const int64_t rows = (int64_t)a.g.N * a.g.group, width = rows <= 8 ? 8 : 16;
    w.blocks = (int)((rows + width - 1) / width);
    const int64_t clusters = (int64_t)w.blocks * a.g.batch * a.g.heads_kv, KS = kSlot / a.d;
    const int64_t longest = (int64_t)a.g.left + a.g.right + a.g.sinks + a.g.N;
    const int64_t steps = ((longest < a.g.N_kv ? longest : a.g.N_kv) + KS - 1) / KS;
    // CTAs of a cluster: until the GPU is full (two per SM), and eight where a sequence may be long; not more than there are steps for their warps.
    const auto idle = [&](int64_t n) { return n * clusters < 2 * a.num_sms; };
    w.C = w.parts = 1;
    while (w.C < kMaxC && (int64_t)w.C * kWarps < steps && (idle(w.C) || steps > (int64_t)w.C * kWarps * 64)) w.C *= 2;
    // Where a warp has more than twelve steps, clusters of four (they find places more easily) and as many parts as make the call shortest, counted in
    // steps (2.2 us of a warp with the GPU full): a CTA's start and end take two; the places share all of it, in rounds where the lengths are one,
    // else, lengths being half of the longest, with a quarter of a CTA's time behind; alone a CTA takes 0.7 of that; the join 1.5.
    // us, d = 128, CTAs x parts 8 x 1 / 8 x 4 / 4 x 4 / 4 x 8 / 4 x 16: 8 x 65536 keys, 8 key heads 185 / 191 / 178 / 187 / 219; six sequences of 1111 to 115200
    // keys 138 / 144 / 135 / 142 / 168; one of 65536 45 / 33 / 33 / 33 / 39.
    if (w.C == kMaxC && steps > kMaxC * kWarps * 12) {
        w.C = 4;
        const auto cost = [&](int parts) {
            const double each = (double)steps / (4 * kWarps * parts), ctas = 4.0 * parts * clusters / (1.8 * a.num_sms);  // (not every place suits a cluster)
            const double rest = ctas - floor(ctas), rounds = floor(ctas) + (rest > 0 ? fmax(rest, 0.7) : 0.0);
            const double all = a.g.kv_len ? fmax(ctas * (0.5 * each + 2) + 0.25 * (each + 2), 0.7 * each + 2) : rounds * (each + 2);
            return all + (parts > 1 ? 1.5 : 0.0);
        };
        for (int parts = 2; parts <= kMaxParts; ++parts)
            if (cost(parts) < cost(w.parts)) w.parts = parts;
    }
    if (w.parts > 1) {
        const int64_t all = (int64_t)w.parts * a.g.batch * a.g.heads * a.g.N;
        w.part_ml = (all * a.d * 4 + 255) / 256 * 256;
        w.bytes = w.part_ml + (all * 8 + 255) / 256 * 256;
    }
    return w;
}

template <int D, bool F16, int NB>
cudaError_t launch(const WindowArgs& a, const CacheGeom& c, const Params& p, const Plan& w, cudaStream_t stream) {
    constexpr int KS = kSlot / D, kSmem = kWarps * 2 * kRing;
    CUtensorMap tk, tv;
    if (!encode_codes_map(&tk, c.K, c.k_batch, c.k_head, c.k_row, c.N, c.heads, c.batch, D, KS) ||
        !encode_codes_map(&tv, c.V, c.v_batch, c.v_head, c.v_row, c.N, c.heads, c.batch, D, KS))
        return cudaErrorInvalidValue;
    const auto kernel = cache_rows_kernel<D, F16, NB>;
    static std::atomic<bool> allowed[kMaxDevices];
    if (!allowed[a.device].load(std::memory_order_relaxed)) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
        if (e != cudaSuccess) return e;
        allowed[a.device].store(true, std::memory_order_relaxed);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(kWarps * 32);
    cfg.dynamicSmemBytes = kSmem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cfg.gridDim = dim3((unsigned)w.C, (unsigned)(w.blocks * w.parts), (unsigned)(a.g.batch * a.g.heads_kv));
    attr[0].val.clusterDim.x = (unsigned)w.C;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, tk, tv, p);
    if (e == cudaSuccess) count_launch();
    return e;
}

}  // namespace

cudaError_t set_cache_rows_wait_limit(long long cycles) { return cudaMemcpyToSymbol(ptx::g_wait_limit_cycles, &cycles, sizeof cycles); }

int64_t cache_rows_bytes(const WindowArgs& a) { return plan_of(a).bytes; }
int cache_rows_parts(const WindowArgs& a) { return plan_of(a).parts; }

cudaError_t launch_cache_rows(const WindowArgs& a, const CacheGeom& c, const bsa_view_t& Q, const bsa_view_t& O, float* LSE, void* workspace, cudaStream_t stream) {
    const Plan w = plan_of(a);
    Params p = {};
    p.g = a.g;
    p.Q = static_cast<const uint16_t*>(Q.data);
    p.O = static_cast<uint16_t*>(O.data);
    p.LSE = LSE;
    p.q_batch = Q.batch; p.q_head = Q.head; p.q_row = Q.row;
    p.o_batch = O.batch; p.o_head = O.head; p.o_row = O.row;
    p.k_scale = c.K_scale;
    p.v_scale = c.V_scale;
    p.s_batch = c.s_batch;
    p.s_head = c.s_head;
    p.lg_block = c.lg_block;
    p.last_block = c.blocks - 1;
    p.parts = w.parts;
    p.part_O = static_cast<float*>(workspace);
    p.part_ml = reinterpret_cast<float2*>(static_cast<uint8_t*>(workspace) + w.part_ml);
    p.scale_log2 = a.scale * 1.4426950408889634f;
    p.n_rows = a.g.N * a.g.group;
    p.withhold = window_withhold();
    cudaError_t e = window_status_word(a.device, &p.status);
    if (e != cudaSuccess) return e;
    const auto of = [&](auto nb) {
        constexpr int NB = decltype(nb)::value;
        return a.d == 64 ? (a.f16 ? launch<64, true, NB>(a, c, p, w, stream) : launch<64, false, NB>(a, c, p, w, stream))
                         : (a.f16 ? launch<128, true, NB>(a, c, p, w, stream) : launch<128, false, NB>(a, c, p, w, stream));
    };
    e = p.n_rows <= 8 ? of(std::integral_constant<int, 1>{}) : of(std::integral_constant<int, 2>{});
    if (e != cudaSuccess || w.parts == 1) return e;
    return launch_cache_join(a, w.parts, p.part_O, p.part_ml, nullptr, 0.f, O, LSE, stream);
}

}  // namespace bsa
