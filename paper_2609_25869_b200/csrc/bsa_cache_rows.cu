// Attention over a window of the 8-bit cache: forward for few rows (the next token, a handful of drafted ones, a short chunk).
//
// What bounds it is reading the visible codes once.  As for the 16-bit cache (bsa_window_rows.cu), the keys are spread over the GPU: a cluster of
// CTAs takes 16 rows of one key head, every warp walks its own share of the keys in steps of 4 KB (32 keys at d = 128, 64 at d = 64), copied
// by TMA into two rings private to the warp, and the warps' and CTAs' (m, l, O) are joined in shared and distributed shared memory.
//
// Per byte there are twice as many elements to multiply as in 16 bits, and each has to be widened first, so the way from shared memory to the
// tensor instruction (mma.sync.m16n8k16 on halves) is kept short:
//   * The order of the channels inside a product is free as long as Q has it too, and so is the order of the keys and, for P V, that of the
//     output's columns.  A lane takes 16 channels of one key (Q K^T) or of four keys (P V) with one 16-byte load, and two neighbouring codes are
//     one instruction away from a fragment's register: K's are neighbours in memory, V's (two keys of one channel) after a byte permutation.
//   * Which key stands behind column n of a product (key_even, key_odd) is chosen so that both kinds of load are free of bank conflicts.
//   * e4m3 widens to half exactly.  Q comes as bf16 or half; a row of bf16 is multiplied by the power of two that takes its largest element to
//     2^14 .. 2^15, and its elements down to 2^-31 of that one keep all their bits (what is lost below is at most 2^-39 of it).
//   * Scales stay out of the products: scores are multiplied by their block's power of two; V's goes into the exponent of its keys' weights,
//     relative to the largest so far of the warp's keys, which the accumulator is in units of.  P and its sum stay fp32 until P is rounded to half.
#include <cuda_fp16.h>
#include <float.h>
#include <math.h>

#include <atomic>

#include "bsa_cache.cuh"

namespace bsa {

using namespace ptx;

namespace {

constexpr int kWarps = 6;
constexpr int kRows = 16;
constexpr int kRing = 8192;  // bytes of a warp's K or V ring
constexpr int kSlot = 4096;
constexpr int kSlots = kRing / kSlot;
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
    float scale_log2;
    int n_rows;    // N * group
    int withhold;  // test hook: no copy of a warp's first tile of V
    int* status;
};

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t map_to_rank(uint32_t smem, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem), "r"(rank));
    return r;
}
__device__ __forceinline__ float2 ld_cluster(uint32_t addr) {
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
    return v;
}
// (Not volatile, as loads from the ring are plain ones: the compiler may put other products and loads between those that depend on each other.
// In program order a step took 5000 clk of a warp that had its SM's quarter nearly to itself.)
__device__ __forceinline__ void mma(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The keys of eight behind columns 2t and 2t + 1 of a product.  Rows lie D bytes apart, their 16-byte chunks XORed with the row's low bits (d = 128:
// three, of 128 bytes; d = 64: bits 1 and 2, of 64 bytes, two rows to 128 bytes).  Eight lanes of a 16-byte load of K have two columns, 2j and 2j + 1,
// and four chunks; of V they have the four even (odd) columns and two chunks (d = 64: sixteen lanes, four half chunks).
template <int D>
__device__ __forceinline__ int key_even(int t) { return D == 128 ? 2 * t : (t & 1) | ((t & 2) << 1); }
template <int D>
constexpr int kOdd = D == 128 ? 5 : 3;  // the odd column's key is the even one's XOR this
template <int D>
__device__ __forceinline__ uint32_t chunk_at(int row, int chunk) {
    return (uint32_t)(row * D + ((chunk ^ (D == 128 ? row & 7 : (row >> 1) & 3)) << 4));
}
// Where 16-byte piece c of a row of the partial sums lies: a lane writes D / 4 consecutive columns of a row, eight lanes at a time two rows.
template <int D>
__device__ __forceinline__ int piece_at(int row, int c) {
    return D == 128 ? c ^ (((c >> 3) & 3) | ((row & 1) << 2)) : c ^ (((c >> 3) & 1) | ((row & 1) << 1));
}

// MAX_C: most CTAs of the cluster, eight or sixteen (the join's loads are written out).
template <int D, bool F16, int MAX_C>
__global__ void __launch_bounds__(kWarps * 32, 2)
cache_rows_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ Params p) {
    constexpr int KS = kSlot / D;  // keys per step
    constexpr int G = KS / 16;     // groups of 16 keys, the shortest block
    constexpr int NT_S = KS / 8, KS_QK = D / 16, NT_O = D / 8, HALVES = D / 64;
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ __align__(8) uint64_t bars[kWarps][2 * kSlots];  // K slots, then V slots: the copy has landed
    __shared__ float wm[kWarps][kRows], wl[kWarps][kRows];      // the warps' maxima (log2 domain) and sums
    __shared__ __align__(8) float2 cml[kRows];                  // the CTA's
    __shared__ uint32_t abort_flag;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gid = lane >> 2, t = lane & 3;
    const int C = gridDim.x, rank = blockIdx.x;
    const int b = blockIdx.z / p.g.heads_kv, hk = blockIdx.z - b * p.g.heads_kv, row0 = blockIdx.y * kRows;
    const uint32_t sK = smem_u32(smem) + warp * 2 * kRing, sV = sK + kRing;
    const uint32_t bK = smem_u32(&bars[warp][0]), bV = bK + kSlots * 8;
    if (threadIdx.x == 0) abort_flag = 0;
    if (lane == 0) {
        prefetch_tensormap(&tmK);
        prefetch_tensormap(&tmV);
        for (int i = 0; i < 2 * kSlots; ++i) mbar_init(bK + i * 8, 1);
        fence_mbar_init();
    }
    __syncthreads();
    volatile uint32_t* abortp = &abort_flag;

    // Row r of the key head is query token r / group under query head hk * group + r % group.
    const Sequence seq = load_sequence(p.g, b);
    const int n0 = row0 / p.g.group, n1 = min((row0 + kRows - 1) / p.g.group + 1, p.g.N);
    const KeyRange range = key_range(p.g, seq, n0, n1);
    // steps of KS keys: [0, st) and [w0, w1), as the tiles of the other kernel
    const int w0 = range.lo / KS, w1 = (range.hi + KS - 1) / KS, st = min((range.sink_hi + KS - 1) / KS, w0);
    const int steps = st + (w1 - w0);
    const long long share = (long long)C * kWarps, mine = (long long)rank * kWarps + warp;
    const int first = (int)(steps * mine / share), last = (int)(steps * (mine + 1) / share);
    auto key_of = [&](int j) { return (j < st ? j : w0 + (j - st)) * KS; };
    auto copy_in = [&](uint32_t dst, const CUtensorMap* map, uint32_t bar, int key0) {
        mbar_arrive_expect_tx(bar, kSlot);
        tma_load_4d(dst, map, bar, 0, key0, hk, b);
    };
    if (lane == 0) {
        for (int i = 0; i < kSlots && first + i < last; ++i) {
            copy_in(sK + i * kSlot, &tmK, bK + i * 8, key_of(first + i));
            if (!(p.withhold && i == 0)) copy_in(sV + i * kSlot, &tmV, bV + i * 8, key_of(first + i));
        }
    }
    // A step's scales: lanes 0 .. G - 1 have K's, lanes 16 .. 16 + G - 1 V's, a step ahead.
    const uint8_t* scales = (lane < 16 ? p.k_scale : p.v_scale) + b * p.s_batch + hk * p.s_head;
    auto load_scale = [&](int j) -> int {
        return (lane & 15) < G ? (int)__ldg(scales + min((key_of(j) + (lane & 15) * 16) >> p.lg_block, p.last_block)) : 0;
    };
    int next_code = first < last ? load_scale(first) : 0;
    // Q fragments (A operand, row-major 16 x 16 per step) of rows gid and gid + 8: positions 2t, 2t + 1, 2t + 8, 2t + 9 of product h * 4 + s
    // are channels h * 64 + t * 16 + s * 4 .. + 3.
    int pos[2];
    float c2[2];  // what takes a row's products to scores (log2 domain), but for K's scale
    uint32_t qa[KS_QK][4];
#pragma unroll
    for (int hi = 0; hi < 2; ++hi) {
        const int r = row0 + gid + 8 * hi;
        const int n = r / p.g.group, h = hk * p.g.group + (r - n * p.g.group);
        const bool ok = r < p.n_rows;
        pos[hi] = ok ? seq.start + n : -1;
        const uint16_t* q = p.Q + (long long)b * p.q_batch + (long long)h * p.q_head + (long long)n * p.q_row;
        uint32_t most = 0;
#pragma unroll
        for (int x = 0; x < HALVES; ++x) {
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const uint4 v = ok ? __ldg(reinterpret_cast<const uint4*>(q + x * 64 + t * 16 + y * 8)) : make_uint4(0, 0, 0, 0);
                const int ks = x * 4 + y * 2;
                qa[ks][hi] = v.x;
                qa[ks][2 + hi] = v.y;
                qa[ks + 1][hi] = v.z;
                qa[ks + 1][2 + hi] = v.w;
                if (!F16)
                    for (const uint32_t w : {v.x, v.y, v.z, v.w}) most = max(most, max((w >> 7) & 0xffu, (w >> 23) & 0xffu));
            }
        }
        c2[hi] = p.scale_log2;
        if (!F16) {
            most = max(most, __shfl_xor_sync(kAll, most, 1));
            most = max(most, __shfl_xor_sync(kAll, most, 2));
            const int field = min(268 - (int)most, 253);  // of the factor that takes exponent most - 127 to 14, and of a finite inverse
            const float up = __int_as_float(field << 23);
            c2[hi] *= __int_as_float((254 - field) << 23);
#pragma unroll
            for (int ks = 0; ks < KS_QK; ++ks)
#pragma unroll
                for (int k = hi; k < 4; k += 2) {
                    const uint32_t w = qa[ks][k];
                    qa[ks][k] = pack_f16x2(__uint_as_float(w << 16) * up, __uint_as_float(w & 0xffff0000u) * up);
                }
        }
    }
    float o[NT_O][4];
#pragma unroll
    for (int n = 0; n < NT_O; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
    float m_lo = -INFINITY, m_hi = -INFINITY, l_lo = 0.f, l_hi = 0.f;  // maxima of the rows, this thread's share of their sums
    int v_unit = 0;  // the accumulator counts in 2^(v_unit - 127): the largest scale so far
    int slot = 0;
    uint32_t phase = 0;
    bool ok = true;
    const int ke = key_even<D>(t), ko = ke ^ kOdd<D>;     // of this lane's two columns
    const int kg = key_even<D>((gid >> 1) & 3) ^ ((gid & 1) ? kOdd<D> : 0);  // and the key behind column gid
    for (int j = first; j < last; ++j) {
        const int key0 = key_of(j);
        const uint32_t cK = sK + slot * kSlot, cV = sV + slot * kSlot;
        const uint8_t *gK = smem + warp * 2 * kRing + slot * kSlot, *gV = gK + kRing;
        const int code = next_code;
        if (j + 1 < last) next_code = load_scale(j + 1);
        ok = mbar_wait_warp(bK + slot * 8, phase, abortp);
        if (!ok) break;
        float s[NT_S][4];
#pragma unroll
        for (int n = 0; n < NT_S; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
#pragma unroll
        for (int x = 0; x < HALVES; ++x) {
            uint4 w[NT_S];
#pragma unroll
            for (int n = 0; n < NT_S; ++n) w[n] = *reinterpret_cast<const uint4*>(gK + chunk_at<D>(n * 8 + kg, x * 4 + t));
#pragma unroll
            for (int y = 0; y < 4; ++y)
#pragma unroll
                for (int n = 0; n < NT_S; ++n) {  // (n inside: neighbours do not depend on each other)
                    const uint32_t v = y == 0 ? w[n].x : y == 1 ? w[n].y : y == 2 ? w[n].z : w[n].w;
                    uint32_t b0, b1;
                    e4m3x4_to_f16x4(v, b0, b1);
                    mma(s[n], qa[x * 4 + y], b0, b1);
                }
        }
        __syncwarp();  // every lane has read the K slot
        if (lane == 0 && j + kSlots < last) copy_in(cK, &tmK, bK + slot * 8, key_of(j + kSlots));
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int kc = __shfl_sync(kAll, code, g);
            const float f = scale_of(kc);
            float f_lo = c2[0] * f, f_hi = c2[1] * f;
            f_lo = f_lo > FLT_MAX ? FLT_MAX : f_lo;  // (so that a product of zero stays a score of zero)
            f_hi = f_hi > FLT_MAX ? FLT_MAX : f_hi;
#pragma unroll
            for (int n = 2 * g; n < 2 * g + 2; ++n) {
                s[n][0] *= f_lo;
                s[n][1] *= f_lo;
                s[n][2] *= f_hi;
                s[n][3] *= f_hi;
            }
        }
        int vc[G];  // V's codes; of groups that nobody here sees, the unit's
        int v_most = v_unit;
        const bool full = key0 + KS <= range.all_hi && (key0 >= range.all_lo || key0 + KS <= p.g.sinks);
#pragma unroll
        for (int g = 0; g < G; ++g) {
            vc[g] = __shfl_sync(kAll, code, 16 + g);
            const int k = key0 + 16 * g;
            if (!full && (k >= range.hi || (k + 16 <= range.lo && k >= range.sink_hi))) vc[g] = 0;
            v_most = max(v_most, vc[g] == 255 ? 0 : vc[g]);
        }
        ok = mbar_wait_warp(bV + slot * 8, phase, abortp);
        if (!ok) break;
        if (!full) {
            const RowView lo(p.g, seq, pos[0], key0), hi(p.g, seq, pos[1], key0);
#pragma unroll
            for (int w = 0; w < KS / 32; ++w) {
                const uint32_t lo_bits = lo.bits(w * 32), hi_bits = hi.bits(w * 32);
#pragma unroll
                for (int n = 4 * w; n < 4 * w + 4; ++n) {
                    const int c = (n & 3) * 8;
                    if (!((lo_bits >> (c + ke)) & 1)) s[n][0] = -INFINITY;
                    if (!((lo_bits >> (c + ko)) & 1)) s[n][1] = -INFINITY;
                    if (!((hi_bits >> (c + ke)) & 1)) s[n][2] = -INFINITY;
                    if (!((hi_bits >> (c + ko)) & 1)) s[n][3] = -INFINITY;
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
        float mx_lo = -INFINITY, mx_hi = -INFINITY;
#pragma unroll
        for (int n = 0; n < NT_S; ++n) {
            mx_lo = max3(mx_lo, s[n][0], s[n][1]);
            mx_hi = max3(mx_hi, s[n][2], s[n][3]);
        }
        if (__any_sync(kAll, mx_lo > m_lo || mx_hi > m_hi) || v_most > v_unit) {
            mx_lo = fmaxf(mx_lo, __shfl_xor_sync(kAll, mx_lo, 1));
            mx_hi = fmaxf(mx_hi, __shfl_xor_sync(kAll, mx_hi, 1));
            mx_lo = fmaxf(mx_lo, __shfl_xor_sync(kAll, mx_lo, 2));
            mx_hi = fmaxf(mx_hi, __shfl_xor_sync(kAll, mx_hi, 2));
            const float mn_lo = fmaxf(m_lo, mx_lo), mn_hi = fmaxf(m_hi, mx_hi);
            const float a_lo = (m_lo == -INFINITY) ? 0.f : ex2_approx(m_lo - mn_lo);
            const float a_hi = (m_hi == -INFINITY) ? 0.f : ex2_approx(m_hi - mn_hi);
            const float unit = ex2_approx((float)(v_unit - v_most));
            m_lo = mn_lo;
            m_hi = mn_hi;
            v_unit = v_most;
            l_lo *= a_lo;
            l_hi *= a_hi;
            const float u_lo = a_lo * unit, u_hi = a_hi * unit;
#pragma unroll
            for (int n = 0; n < NT_O; ++n) {
                o[n][0] *= u_lo;
                o[n][1] *= u_lo;
                o[n][2] *= u_hi;
                o[n][3] *= u_hi;
            }
        }
        const float nm_lo = (m_lo == -INFINITY) ? 0.f : kShift - m_lo, nm_hi = (m_hi == -INFINITY) ? 0.f : kShift - m_hi;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int dv = max(vc[g] - v_unit, -kFar);
            const float up = vc[g] == 255 ? NAN : (float)dv, down = __int_as_float((127 - dv) << 23);  // (255: dv is not used)
            const float g_lo = nm_lo + up, g_hi = nm_hi + up;
            uint32_t pa[4];  // P as the A operand of P V
            float sum_lo = 0.f, sum_hi = 0.f;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float* x = s[2 * g + i];
                const float p0 = ex2_approx(x[0] + g_lo), p1 = ex2_approx(x[1] + g_lo);
                const float p2 = ex2_approx(x[2] + g_hi), p3 = ex2_approx(x[3] + g_hi);
                sum_lo += p0 + p1;
                sum_hi += p2 + p3;
                pa[i * 2] = pack_f16x2(p0, p1);
                pa[i * 2 + 1] = pack_f16x2(p2, p3);
            }
            l_lo = fmaf(sum_lo, down, l_lo);
            l_hi = fmaf(sum_hi, down, l_hi);
            // V of keys 2t, 2t + 1, 2t + 8, 2t + 9 (columns of P), channels gid * D / 8 ..
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
            for (int w = 0; w < D / 32; ++w) {
                const uint32_t a01 = __byte_perm(v[0][w], v[1][w], 0x5140), a23 = __byte_perm(v[0][w], v[1][w], 0x7362);
                const uint32_t b01 = __byte_perm(v[2][w], v[3][w], 0x5140), b23 = __byte_perm(v[2][w], v[3][w], 0x7362);
                uint32_t a0, a1, a2, a3, b0, b1, b2, b3;
                e4m3x4_to_f16x4(a01, a0, a1);
                e4m3x4_to_f16x4(a23, a2, a3);
                e4m3x4_to_f16x4(b01, b0, b1);
                e4m3x4_to_f16x4(b23, b2, b3);
                mma(o[4 * w], pa, a0, b0);
                mma(o[4 * w + 1], pa, a1, b1);
                mma(o[4 * w + 2], pa, a2, b2);
                mma(o[4 * w + 3], pa, a3, b3);
            }
        }
        __syncwarp();  // every lane has read the V slot
        if (lane == 0 && j + kSlots < last) copy_in(cV, &tmV, bV + slot * 8, key_of(j + kSlots));
        if (++slot == kSlots) {
            slot = 0;
            phase ^= 1u;
        }
    }
    if (!ok) let_copies_land();  // before the rings are used for anything else (a warp that came to its end has waited for all of its own)
    // ---- join the warps: weights first, then the rows, scaled, into shared memory ----
    l_lo += __shfl_xor_sync(kAll, l_lo, 1);
    l_hi += __shfl_xor_sync(kAll, l_hi, 1);
    l_lo += __shfl_xor_sync(kAll, l_lo, 2);
    l_hi += __shfl_xor_sync(kAll, l_hi, 2);
    constexpr float kBack = 1.f / 32768.f;  // 2^-kShift
    if (t == 0) {
        wm[warp][gid] = m_lo;
        wm[warp][gid + 8] = m_hi;
        wl[warp][gid] = l_lo * kBack;
        wl[warp][gid + 8] = l_hi * kBack;
    }
    __syncthreads();  // (every warp's ring is idle from here on)
    float M_lo = -INFINITY, M_hi = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        M_lo = fmaxf(M_lo, wm[w][gid]);
        M_hi = fmaxf(M_hi, wm[w][gid + 8]);
    }
    const float unit = scale_of(v_unit);
    const float f_lo = m_lo == -INFINITY ? 0.f : ex2_approx(m_lo - M_lo) * kBack, f_hi = m_hi == -INFINITY ? 0.f : ex2_approx(m_hi - M_hi) * kBack;
    // [warp][row][D], a lane's D / 4 consecutive columns of two rows in pieces of 16 bytes (see piece_at)
    float* part = reinterpret_cast<float*>(smem) + warp * kRows * D;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
        constexpr int PER = D / 32;  // pieces of one of the lane's two columns
        const int e = i / PER, n = i % PER * 4, c = t * (D / 16) + i;
        *reinterpret_cast<float4*>(part + gid * D + piece_at<D>(gid, c) * 4) =
            make_float4(o[n][e] * f_lo * unit, o[n + 1][e] * f_lo * unit, o[n + 2][e] * f_lo * unit, o[n + 3][e] * f_lo * unit);
        *reinterpret_cast<float4*>(part + (gid + 8) * D + piece_at<D>(gid, c) * 4) =
            make_float4(o[n][2 + e] * f_hi * unit, o[n + 1][2 + e] * f_hi * unit, o[n + 2][2 + e] * f_hi * unit, o[n + 3][2 + e] * f_hi * unit);
    }
    if (threadIdx.x < kRows) {
        const int r = threadIdx.x;
        float M = -INFINITY, L = 0.f;
        for (int w = 0; w < kWarps; ++w) M = fmaxf(M, wm[w][r]);
        // (a maximum of -inf: nothing seen, the sum is zero, or nothing but NaN, which the maximum passes over and the sum keeps)
        for (int w = 0; w < kWarps; ++w) L += wm[w][r] == -INFINITY ? wl[w][r] : wl[w][r] * ex2_approx(wm[w][r] - M);
        cml[r] = make_float2(M, L);
    }
    __syncthreads();
    float* sum = reinterpret_cast<float*>(smem);  // the CTA's rows, in the place of warp 0's
    for (int i = threadIdx.x; i < kRows * D; i += kWarps * 32) {
        float a = sum[i];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) a += sum[w * kRows * D + i];
        sum[i] = a;
    }
    // ---- join the CTAs of the cluster; each writes its share of the outputs ----
    if (C > 1) cluster_sync(); else __syncthreads();
    const int per = kRows * D / C;  // (C divides it)
    const uint32_t a_sum = smem_u32(sum), a_ml = smem_u32(cml);
    for (int i = rank * per + 2 * threadIdx.x; i < (rank + 1) * per; i += 2 * kWarps * 32) {
        const int r = i / D, c = piece_at<D>(r, (i - r * D) >> 2) * 4 + (i & 3);  // element i of the stored order is column c
        float2 ml[MAX_C], v[MAX_C];
#pragma unroll
        for (int q = 0; q < MAX_C; ++q) {  // all loads on their way before the first is used (ranks beyond C: this one again)
            const uint32_t from = q < C ? q : rank;
            ml[q] = ld_cluster(map_to_rank(a_ml + r * 8, from));
            v[q] = ld_cluster(map_to_rank(a_sum + i * 4, from));
        }
        float M = -INFINITY, L = 0.f, v0 = 0.f, v1 = 0.f;
#pragma unroll
        for (int q = 0; q < MAX_C; ++q) M = fmaxf(M, ml[q].x);
#pragma unroll
        for (int q = 0; q < MAX_C; ++q) {
            const float f = ml[q].x == -INFINITY ? 0.f : ex2_approx(ml[q].x - M);
            const bool own = q < C;  // (left out, not taken times zero: an infinite sum would become NaN)
            L = own ? fmaf(f, ml[q].y, L) : L;
            v0 = own ? fmaf(f, v[q].x, v0) : v0;
            v1 = own ? fmaf(f, v[q].y, v1) : v1;
        }
        const int row = row0 + r;
        if (row < p.n_rows) {
            const int n = row / p.g.group, h = hk * p.g.group + (row - n * p.g.group);
            const int at = seq.start + n;
            // Decided by the position alone: a row at a position sees its own key at least, and a sum that is NaN belongs to its outputs.
            // (A row at none may have a sum: steps that the rows of the sequence see whole are not masked.)
            const bool any = at >= 0 && at < seq.len;
            const float inv = any ? 1.f / L : 0.f;
            *reinterpret_cast<uint32_t*>(p.O + (long long)b * p.o_batch + (long long)h * p.o_head + (long long)n * p.o_row + c) =
                any ? pack_16x2<F16>(v0 * inv, v1 * inv) : 0u;
            if (c == 0) p.LSE[((long long)b * p.g.heads + h) * p.g.N + n] = any ? fmaf(M, 0.6931471805599453f, logf(L)) : -INFINITY;
        }
    }
    if (threadIdx.x == 0 && abort_flag) atomicExch(p.status, (int)BSA_ERR_DEVICE_TIMEOUT);
    if (C > 1) cluster_sync();  // nobody leaves while its shared memory is being read
}

template <int D, bool F16>
cudaError_t launch(const WindowArgs& a, const CacheGeom& c, const Params& p, cudaStream_t stream) {
    constexpr int KS = kSlot / D, kSmem = kWarps * 2 * kRing;
    CUtensorMap tk, tv;
    if (!encode_codes_map(&tk, c.K, c.k_batch, c.k_head, c.k_row, c.N, c.heads, c.batch, D, KS) ||
        !encode_codes_map(&tv, c.V, c.v_batch, c.v_head, c.v_row, c.N, c.heads, c.batch, D, KS))
        return cudaErrorInvalidValue;
    const auto kernel = cache_rows_kernel<D, F16, 8>, wide_kernel = cache_rows_kernel<D, F16, 16>;
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(kWarps * 32);
    cfg.dynamicSmemBytes = kSmem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    static std::atomic<bool> allowed[kMaxDevices];
    static std::atomic<int> resident8[kMaxDevices], resident16[kMaxDevices];  // clusters that the GPU holds at once
    if (!allowed[a.device].load(std::memory_order_acquire)) {
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(wide_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(wide_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        int n = 0;
        cfg.gridDim = dim3(attr[0].val.clusterDim.x = 8);
        if (e == cudaSuccess) e = cudaOccupancyMaxActiveClusters(&n, kernel, &cfg);
        if (e != cudaSuccess) return e;
        resident8[a.device].store(n, std::memory_order_relaxed);
        cfg.gridDim = dim3(attr[0].val.clusterDim.x = 16);
        if (cudaOccupancyMaxActiveClusters(&n, wide_kernel, &cfg) != cudaSuccess) {  // a GPU without a place for them
            cudaGetLastError();
            n = 0;
        }
        resident16[a.device].store(n, std::memory_order_relaxed);
        allowed[a.device].store(true, std::memory_order_release);
    }
    const unsigned blocks = (unsigned)((p.n_rows + kRows - 1) / kRows), heads = (unsigned)(a.g.batch * a.g.heads_kv);
    // CTAs of a cluster, by the rule of the kernel for the 16-bit cache (bsa_window_rows.cu has the figures): until the GPU is full, and eight at once
    // where a sequence may be long; sixteen where eight leave the GPU idle and a warp has 64 steps and more.
    const int64_t longest = (int64_t)a.g.left + a.g.right + a.g.sinks + a.g.N;
    const int64_t steps = ((longest < a.g.N_kv ? longest : a.g.N_kv) + KS - 1) / KS;
    const auto idle = [&](int n) { return (int64_t)n * blocks * heads < 2 * a.num_sms; };
    const auto long_shares = [&](int n) { return steps > (int64_t)n * kWarps * 64; };
    int C = 1;
    while (C < 8 && (int64_t)C * kWarps < steps && (idle(C) || long_shares(C))) C *= 2;
    const int64_t clusters = (int64_t)blocks * heads;
    const int at_once8 = resident8[a.device].load(std::memory_order_relaxed), at_once16 = resident16[a.device].load(std::memory_order_relaxed);
    if (C == 8 && idle(8) && long_shares(8) && at_once16 > 0 && (clusters <= at_once16 || clusters > at_once8)) C = 16;
    cfg.gridDim = dim3((unsigned)C, blocks, heads);
    attr[0].val.clusterDim.x = (unsigned)C;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, C > 8 ? wide_kernel : kernel, tk, tv, p);
    if (e == cudaSuccess) count_launch();
    return e;
}

}  // namespace

cudaError_t set_cache_rows_wait_limit(long long cycles) { return cudaMemcpyToSymbol(ptx::g_wait_limit_cycles, &cycles, sizeof cycles); }

cudaError_t launch_cache_rows(const WindowArgs& a, const CacheGeom& c, const bsa_view_t& Q, const bsa_view_t& O, float* LSE, cudaStream_t stream) {
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
    p.scale_log2 = a.scale * 1.4426950408889634f;
    p.n_rows = a.g.N * a.g.group;
    p.withhold = window_withhold();
    const cudaError_t e = window_status_word(a.device, &p.status);
    if (e != cudaSuccess) return e;
    return a.d == 64 ? (a.f16 ? launch<64, true>(a, c, p, stream) : launch<64, false>(a, c, p, stream))
                     : (a.f16 ? launch<128, true>(a, c, p, stream) : launch<128, false>(a, c, p, stream));
}

}  // namespace bsa
