// Attention over a sliding window and a few first tokens: gradients.
//
//   P = exp(S - LSE),  D_i = sum dO * O,  dV = P^T dO,  dS = P * (dO V^T - D),  dQ = scale dS K,  dK = scale dS^T Q
//
// Three kernels:
//   delta  : D of every row, and LSE in the exp2 domain
//   dQ     : a CTA owns 128 query rows and walks over the key tiles that they see      (S, dO V^T, dS K: three products a tile)
//   dK, dV : a CTA owns 128 keys and walks over the query tiles, of every head that shares the keys, that see them, with the
//            scores transposed so that P^T and dS^T, where they are computed, are the products' left operands in tensor memory
//            (K Q^T, V dO^T, P^T dO, dS^T Q: four products a tile)
// Seven products instead of the five that one kernel for all three gradients needs; that one would add either dQ or dK and dV up
// in global memory, in an order that changes from run to run, or keep partial sums of one of them per tile of the other.  Here
// every gradient is summed in tensor memory by one CTA.  Only the keys of the first tokens, seen by every query, are cut into
// several shares of their queries, whose sums are added up in a fixed order by a fourth kernel.
// In both kernels eight softmax warps (thread = row of a tile), one warp that copies and one that issues the products.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include <atomic>

#include "bsa_window.cuh"

namespace bsa {

using namespace ptx;

namespace {

constexpr int kThreads = 320;  // warps 0-7: softmax, 8: copies, 9: products
constexpr uint32_t kTmemCols = 512;
constexpr int SUB = kWinT * 128;  // bytes of a [128 rows][64 columns] sub-tile

struct BwdParams {
    WindowGeom g;
    float scale, scale_log2;
    int n_pad;             // N rounded up to whole tiles
    const float* neg_lse2;   // [batch * heads][n_pad]: -LSE in the exp2 domain (-inf for rows that see nothing: their P is zero)
    const float* neg_delta;  // -D
    uint16_t* dQ;
    uint16_t* dK;
    uint16_t* dV;
    long long q_batch, q_head, q_row, k_batch, k_head, k_row, v_batch, v_head, v_row;  // strides of the gradients
    int n_qt, n_kt;        // tiles of a sequence
    int longest_first;
    int sink_tiles, sink_shares;  // key tiles in front that are cut into shares (0: none)
    float* partial;        // [batch * heads_kv][sink_tiles][sink_shares][dV, dK][128][D]
    int* status;
};

struct __align__(8) DqBarriers {
    uint64_t q_full, k_full[3], k_empty[3], v_full[2], v_empty[2];
    uint64_t s_full[2], s_free, dp_full[2], ds_ready[2], acc_full;  // (one s_full for each of its readers)
};
struct __align__(8) DkvBarriers {
    uint64_t kv_full, q_full[4], q_empty[4], o_full[4], o_empty[4];
    uint64_t s_full, dp_full, p_ready[2], ds_ready, acc_full;
};

__device__ __forceinline__ void let_copies_land() {
    const uint64_t t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 200000ull) __nanosleep(1000);
}
// 1-D copy of whole 16-byte pieces, counted in bytes on an mbarrier
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}
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
template <int R>
__device__ __forceinline__ void reg_inc() {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(R));
}

// Row `row` of a tile in shared memory becomes zero (its 64-column sub-tiles, whatever the swizzle).
template <int D>
__device__ __forceinline__ void zero_row(uint8_t* tile, int row) {
#pragma unroll
    for (int s = 0; s < D / 64; ++s)
#pragma unroll
        for (int c = 0; c < 8; ++c) reinterpret_cast<uint4*>(tile + s * SUB + row * 128)[c] = make_uint4(0, 0, 0, 0);
}

// A row of an accumulator, times `f`, to global memory in the element type.
template <int D, bool F16>
__device__ __forceinline__ void store_row(uint32_t t_acc, float f, bool zero, uint16_t* out) {
#pragma unroll 1
    for (int c = 0; c < D / 32; ++c) {
        uint32_t o[32];
        tmem_ld32(t_acc + c * 32, o);
        tc_wait_ld();
        if (!out) continue;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            uint32_t v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = zero ? 0u : pack_16x2<F16>(__uint_as_float(o[q * 8 + 2 * e]) * f, __uint_as_float(o[q * 8 + 2 * e + 1]) * f);
            *reinterpret_cast<uint4*>(out + c * 32 + q * 8) = make_uint4(v[0], v[1], v[2], v[3]);
        }
    }
}

// ------------------------------------------------------------------------------------------ delta
// Eight lanes a row.  Bound by memory: O and dO are read once.
template <int D, bool F16>
__global__ void __launch_bounds__(256) window_delta_kernel(const WindowGeom g, const uint16_t* O, const uint16_t* dO, long long o_batch,
                                                          long long o_head, long long o_row, long long d_batch, long long d_head,
                                                          long long d_row, const float* LSE, float* neg_lse2, float* neg_delta, int n_pad) {
    const int bh = blockIdx.y, b = bh / g.heads, h = bh - b * g.heads;
    const int row = blockIdx.x * 32 + (threadIdx.x >> 3), l8 = threadIdx.x & 7;
    const Sequence seq = load_sequence(g, b);
    const int pos = seq.start + row;
    const bool seen = row < g.N && pos >= 0 && pos < seq.len;
    float sum = 0.f;
    if (seen) {
        const uint16_t* o = O + (long long)b * o_batch + (long long)h * o_head + (long long)row * o_row;
        const uint16_t* d = dO + (long long)b * d_batch + (long long)h * d_head + (long long)row * d_row;
#pragma unroll
        for (int c = 0; c < D / 64; ++c) {
            const uint4 a = __ldg(reinterpret_cast<const uint4*>(o) + c * 8 + l8), e = __ldg(reinterpret_cast<const uint4*>(d) + c * 8 + l8);
            const uint32_t u[4] = {a.x, a.y, a.z, a.w}, v[4] = {e.x, e.y, e.z, e.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (F16) {
                    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[i])), w = __half22float2(*reinterpret_cast<const __half2*>(&v[i]));
                    sum = fmaf(f.x, w.x, fmaf(f.y, w.y, sum));
                } else {
                    sum = fmaf(__uint_as_float(u[i] << 16), __uint_as_float(v[i] << 16), sum);
                    sum = fmaf(__uint_as_float(u[i] & 0xffff0000u), __uint_as_float(v[i] & 0xffff0000u), sum);
                }
            }
        }
    }
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
    sum += __shfl_xor_sync(0xffffffffu, sum, 4);
    if (l8 == 0 && row < n_pad) {
        neg_delta[(long long)bh * n_pad + row] = -sum;
        neg_lse2[(long long)bh * n_pad + row] = seen ? LSE[(long long)bh * g.N + row] * -1.4426950408889634f : -INFINITY;
    }
}

// ------------------------------------------------------------------------------------------ dQ
template <int D>
struct DqCfg {
    static constexpr int kTile = kWinT * D * 2;
    static constexpr int kK = 3, kV = 2;
    static constexpr int kSmem = (2 + kK + kV) * kTile;  // Q, dO, rings of K and V
    static constexpr uint32_t kS = 0, kDP0 = 128, kDP1 = 256, kDQ = 384;
};

template <int D, bool F16>
__global__ void __launch_bounds__(kThreads, 1)
window_dq_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                 const __grid_constant__ CUtensorMap tmG, const __grid_constant__ BwdParams p) {
    using C = DqCfg<D>;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint8_t* sQ = smem;
    uint8_t* sG = sQ + C::kTile;
    uint8_t* sK = sG + C::kTile;
    uint8_t* sV = sK + C::kK * C::kTile;
    __shared__ DqBarriers bars;
    __shared__ uint32_t tmem_base_s, abort_flag;
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    if (smem_u32(smem) & 1023u) {  // never expected
        if (tid == 0) atomicExch(p.status, (int)BSA_ERR_CUDA);
        return;
    }
    int bh, qt;
    if (p.longest_first) {
        const int n_bh = p.g.batch * p.g.heads;
        qt = p.n_qt - 1 - (int)blockIdx.x / n_bh;
        bh = (int)blockIdx.x % n_bh;
    } else {
        bh = (int)blockIdx.x / p.n_qt;
        qt = (int)blockIdx.x % p.n_qt;
    }
    const int b = bh / p.g.heads, h = bh - b * p.g.heads, hk = h / p.g.group, row0 = qt * kWinT;
    const Sequence seq = load_sequence(p.g, b);
    const KeyRange range = key_range(p.g, seq, row0, row0 + kWinT);
    const TileSpan tiles = tile_span(range);
    const int n = tiles.count();
    if (n == 0) {  // nothing is seen: zero gradient
        const int row = row0 + tid;
        if (tid < kWinT && row < p.g.N) {
            uint4* o = reinterpret_cast<uint4*>(p.dQ + (long long)b * p.q_batch + (long long)h * p.q_head + (long long)row * p.q_row);
            for (int c = 0; c < D / 8; ++c) o[c] = make_uint4(0, 0, 0, 0);
        }
        return;
    }
    if (tid == 0) {
        abort_flag = 0;
        mbar_init(smem_u32(&bars.q_full), 1);
        for (int i = 0; i < C::kK; ++i) {
            mbar_init(smem_u32(&bars.k_full[i]), 1);
            mbar_init(smem_u32(&bars.k_empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&bars.v_full[i]), 1);
            mbar_init(smem_u32(&bars.v_empty[i]), 1);
            mbar_init(smem_u32(&bars.s_full[i]), 1);
            mbar_init(smem_u32(&bars.dp_full[i]), 1);
            mbar_init(smem_u32(&bars.ds_ready[i]), 128);
        }
        mbar_init(smem_u32(&bars.s_free), 128);
        mbar_init(smem_u32(&bars.acc_full), 1);
        fence_mbar_init();
    }
    if (warp == 9) {
        tmem_alloc(smem_u32(&tmem_base_s), kTmemCols);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_base_s, 0);
    volatile uint32_t* abortp = &abort_flag;

    if (warp == 8) {
        if (lane == 0) {
            Ring rk, rv;
            mbar_arrive_expect_tx(smem_u32(&bars.q_full), 2 * C::kTile);
            tma_load_rows(smem_u32(sQ), &tmQ, smem_u32(&bars.q_full), row0, h, b);
            tma_load_rows(smem_u32(sG), &tmG, smem_u32(&bars.q_full), row0, h, b);
            bool ok = true;
            for (int j = 0; j < n; ++j) {
                const int key0 = tiles.tile(j) * kWinT;
                ok = mbar_wait(smem_u32(&bars.k_empty[rk.stage]), rk.phase ^ 1, abortp);
                if (!ok) break;
                mbar_arrive_expect_tx(smem_u32(&bars.k_full[rk.stage]), C::kTile);
                tma_load_rows(smem_u32(sK) + rk.stage * C::kTile, &tmK, smem_u32(&bars.k_full[rk.stage]), key0, hk, b);
                rk.advance<C::kK>();
                ok = mbar_wait(smem_u32(&bars.v_empty[rv.stage]), rv.phase ^ 1, abortp);
                if (!ok) break;
                mbar_arrive_expect_tx(smem_u32(&bars.v_full[rv.stage]), C::kTile);
                tma_load_rows(smem_u32(sV) + rv.stage * C::kTile, &tmV, smem_u32(&bars.v_full[rv.stage]), key0, hk, b);
                rv.advance<C::kV>();
            }
            if (!ok) let_copies_land();
        }
    } else if (warp == 9) {
        // Tile i belongs to softmax warpgroup i mod 2 and has dP buffer i mod 2, where its dS goes as well; S has one buffer, free
        // as soon as it has been read.  Order: S(0), dP(0), S(1), dP(1); then for every tile i: S(i + 2), dQ(i) behind its dS, dP(i + 2).
        constexpr uint32_t idesc_s = make_idesc_f32(kWinT, kWinT, 0, 0, F16), idesc_dq = make_idesc_f32(kWinT, D, 0, 1, F16);
        const uint64_t descQ = make_smem_desc_sw128(smem_u32(sQ), 16, 1024), descG = make_smem_desc_sw128(smem_u32(sG), 16, 1024);
        const uint64_t descK = make_smem_desc_sw128(smem_u32(sK), 16, 1024), descV = make_smem_desc_sw128(smem_u32(sV), 16, 1024);
        const uint64_t descKt = make_smem_desc_sw128(smem_u32(sK), SUB, 1024);
        const bool leader = elect_one();
        Ring rs, rv, rq;  // K of the next S, V of the next dP, K of the next dQ
        bool ok = mbar_wait_warp(smem_u32(&bars.q_full), 0, abortp);
        auto product = [&](uint32_t d, uint64_t a, uint64_t b0) {
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
                const uint64_t off = (uint64_t)(((kk / 4) * SUB + (kk % 4) * 32) >> 4);
                mma_ss(d, a + off, b0 + off, idesc_s, kk > 0);
            }
        };
        auto issue_s = [&](int j) -> bool {
            if (j >= 1 && !mbar_wait_warp(smem_u32(&bars.s_free), (j - 1) & 1, abortp)) return false;
            if (!mbar_wait_warp(smem_u32(&bars.k_full[rs.stage]), rs.phase, abortp)) return false;
            tc_fence_after();
            if (leader) {
                product(tmem + C::kS, descQ, descK + (uint64_t)((rs.stage * C::kTile) >> 4));
                mma_commit(smem_u32(&bars.s_full[j & 1]));
            }
            rs.advance<C::kK>();
            return true;
        };
        auto issue_dp = [&](int j) -> bool {
            if (!mbar_wait_warp(smem_u32(&bars.v_full[rv.stage]), rv.phase, abortp)) return false;
            tc_fence_after();
            if (leader) {
                product(tmem + ((j & 1) ? C::kDP1 : C::kDP0), descG, descV + (uint64_t)((rv.stage * C::kTile) >> 4));
                mma_commit(smem_u32(&bars.dp_full[j & 1]));
                mma_commit(smem_u32(&bars.v_empty[rv.stage]));
            }
            rv.advance<C::kV>();
            return true;
        };
        ok = ok && issue_s(0) && issue_dp(0);
        if (ok && n > 1) ok = issue_s(1) && issue_dp(1);
        for (int i = 0; ok && i < n; ++i) {
            if (i + 2 < n) ok = issue_s(i + 2);
            ok = ok && mbar_wait_warp(smem_u32(&bars.ds_ready[i & 1]), (i >> 1) & 1, abortp);
            if (!ok) break;
            tc_fence_after();
            if (leader) {
                const uint64_t k0 = descKt + (uint64_t)((rq.stage * C::kTile) >> 4);
                const uint32_t a_ds = tmem + ((i & 1) ? C::kDP1 : C::kDP0);
#pragma unroll
                for (int kk = 0; kk < 8; ++kk)
                    mma_ts(tmem + C::kDQ, a_ds + kk * 8, k0 + (uint64_t)(kk * 128), idesc_dq, (i > 0 || kk > 0) ? 1u : 0u);
                mma_commit(smem_u32(&bars.k_empty[rq.stage]));
                if (i == n - 1) mma_commit(smem_u32(&bars.acc_full));
            }
            rq.advance<C::kK>();
            if (i + 2 < n) ok = issue_dp(i + 2);
        }
    } else {
        const int x = warp >> 2, tw = tid & 127;
        const uint32_t t_lane = tmem + ((uint32_t)((warp & 3) * 32) << 16), t_dp = t_lane + (x ? C::kDP1 : C::kDP0);
        const int row = row0 + tw, pos = seq.start + row;
        const float neg_lse = __ldg(p.neg_lse2 + (long long)bh * p.n_pad + row), neg_del = __ldg(p.neg_delta + (long long)bh * p.n_pad + row);
        const uint64_t c22 = pack_f32x2(p.scale_log2, p.scale_log2), nl2 = pack_f32x2(neg_lse, neg_lse), nd2 = pack_f32x2(neg_del, neg_del);
        bool ok = true;
        for (int i = x; i < n; i += 2) {
            const int key0 = tiles.tile(i) * kWinT;
            const bool full = tile_is_full(p.g, range, key0);
            ok = mbar_wait_warp(smem_u32(&bars.s_full[x]), (i >> 1) & 1, abortp);
            if (!ok) break;
            tc_fence_after();
            uint32_t r[kWinT];
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld32(t_lane + C::kS + c * 32, r + c * 32);
            tc_wait_ld();
            tc_fence_before();
            mbar_arrive(smem_u32(&bars.s_free));
#pragma unroll
            for (int c = 0; c < kWinT; c += 2) {
                float a, e;
                unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(r[c]), __uint_as_float(r[c + 1])), c22, nl2), a, e);
                r[c] = __float_as_uint(ex2_approx(a));
                r[c + 1] = __float_as_uint(ex2_approx(e));
            }
            if (!full) {
                // K rows that no row here sees may hold anything: their dS is zero, which times NaN would not be
                const int key = key0 + tw;
                if (key >= range.hi || (key < range.lo && key >= p.g.sinks)) zero_row<D>(sK + (i % C::kK) * C::kTile, tw);
                fence_proxy_async_smem();
            }
            ok = mbar_wait_warp(smem_u32(&bars.dp_full[x]), (i >> 1) & 1, abortp);
            if (!ok) break;
            tc_fence_after();
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t d[32];
                tmem_ld32(t_dp + c * 32, d);
                tc_wait_ld();
#pragma unroll
                for (int e = 0; e < 32; e += 2) {
                    float u, v;
                    unpack_f32x2(mul_f32x2(add_f32x2(pack_f32x2(__uint_as_float(d[e]), __uint_as_float(d[e + 1])), nd2),
                                           pack_f32x2(__uint_as_float(r[c * 32 + e]), __uint_as_float(r[c * 32 + e + 1]))), u, v);
                    d[e] = __float_as_uint(u);
                    d[e + 1] = __float_as_uint(v);
                }
                if (!full) {
                    const uint32_t bits = row_bits(p.g, seq, pos, key0 + c * 32);
#pragma unroll
                    for (int e = 0; e < 32; ++e) d[e] = (bits & (1u << e)) ? d[e] : 0u;
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) d[e] = pack_16x2<F16>(__uint_as_float(d[2 * e]), __uint_as_float(d[2 * e + 1]));
                tmem_st16(t_dp + c * 16, d);  // over columns that have been read
            }
            tc_wait_st();
            tc_fence_before();
            mbar_arrive(smem_u32(&bars.ds_ready[x]));
        }
        if (ok && mbar_wait_warp(smem_u32(&bars.acc_full), 0, abortp)) {
            tc_fence_after();
            if (x == 0) {
                const bool seen = pos >= 0 && pos < seq.len;
                store_row<D, F16>(t_lane + C::kDQ, p.scale, !seen,
                                  row < p.g.N ? p.dQ + (long long)b * p.q_batch + (long long)h * p.q_head + (long long)row * p.q_row : nullptr);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (tid == 0 && abort_flag) atomicExch(p.status, (int)BSA_ERR_DEVICE_TIMEOUT);
    if (warp == 9) tmem_dealloc(tmem, kTmemCols);
}

// ------------------------------------------------------------------------------------------ dK, dV
template <int D>
struct DkvCfg {
    static constexpr int kTile = kWinT * D * 2;
    static constexpr int kQ = 2;  // tiles in the rings of Q and of dO
    static constexpr int kRows = 2 * kWinT * 4;  // bytes of a Q tile's LSE and D
    static constexpr int kSmem = (2 + 2 * kQ) * kTile + kQ * kRows;
    static constexpr uint32_t kS = 0, kDP = 128, kDV = 256, kDK = 384;
};

// The query rows that see some of the keys [k0, k0 + 128) of a sequence, as tiles [t0, t1).
struct RowSpan {
    int t0, t1;
};
__device__ __forceinline__ RowSpan row_span(const WindowGeom& g, const Sequence& s, int k0) {
    RowSpan r = {0, 0};
    const int k1 = min(k0 + kWinT, s.len) - 1;
    if (k1 < k0) return r;
    const int p0 = max(max(0, k0 - g.right), s.start);
    const int p1 = min(min(s.len - 1, k0 < g.sinks ? s.len - 1 : k1 + g.left), s.start + g.N - 1);
    if (p0 > p1) return r;
    r.t0 = (p0 - s.start) / kWinT;
    r.t1 = (p1 - s.start) / kWinT + 1;
    return r;
}
// Which of the 32 query rows from row q0 on see key j.
__device__ __forceinline__ uint32_t key_bits(const WindowGeom& g, const Sequence& s, int j, int q0) {
    if (j >= s.len) return 0u;
    const int from = max(j - g.right, 0), to = min(j < g.sinks ? s.len - 1 : j + g.left, s.len - 1);  // positions
    return bits_below(to + 1 - s.start - q0) & ~bits_below(from - s.start - q0);
}

template <int D, bool F16>
__global__ void __launch_bounds__(kThreads, 1)
window_dkv_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                  const __grid_constant__ CUtensorMap tmG, const __grid_constant__ BwdParams p) {
    using C = DkvCfg<D>;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint8_t* sK = smem;
    uint8_t* sV = sK + C::kTile;
    uint8_t* sQ = sV + C::kTile;
    uint8_t* sG = sQ + C::kQ * C::kTile;
    uint8_t* sR = sG + C::kQ * C::kTile;  // [stage][LSE, D][128]
    __shared__ DkvBarriers bars;
    __shared__ uint32_t tmem_base_s, abort_flag;
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    if (smem_u32(smem) & 1023u) {  // never expected
        if (tid == 0) atomicExch(p.status, (int)BSA_ERR_CUDA);
        return;
    }
    // Items: the shares of the sinks' tiles first (the longest), then the other tiles, a sequence's neighbours side by side.
    const int n_bh = p.g.batch * p.g.heads_kv, n_shared = p.sink_tiles * p.sink_shares;
    int bh, kt, share = 0, shares = 1;
    {
        int idx = blockIdx.x;
        if (idx < n_bh * n_shared) {
            bh = idx / n_shared;
            idx -= bh * n_shared;
            kt = idx / p.sink_shares;
            share = idx - kt * p.sink_shares;
            shares = p.sink_shares;
        } else {
            idx -= n_bh * n_shared;
            const int per = p.n_kt - p.sink_tiles;
            if (p.longest_first) {  // the first keys are seen by the most rows
                kt = p.sink_tiles + idx / n_bh;
                bh = idx % n_bh;
            } else {
                bh = idx / per;
                kt = p.sink_tiles + idx % per;
            }
        }
    }
    const int b = bh / p.g.heads_kv, hk = bh - b * p.g.heads_kv, key0 = kt * kWinT;
    const Sequence seq = load_sequence(p.g, b);
    const RowSpan span = row_span(p.g, seq, key0);
    const int per_head = span.t1 - span.t0, all = per_head * p.g.group;
    const int first = (int)((long long)all * share / shares), last = (int)((long long)all * (share + 1) / shares), n = last - first;

    if (tid == 0) {
        abort_flag = 0;
        mbar_init(smem_u32(&bars.kv_full), 1);
        for (int i = 0; i < C::kQ; ++i) {
            mbar_init(smem_u32(&bars.q_full[i]), 1);
            mbar_init(smem_u32(&bars.q_empty[i]), 1);
            mbar_init(smem_u32(&bars.o_full[i]), 1);
            mbar_init(smem_u32(&bars.o_empty[i]), 1);
        }
        mbar_init(smem_u32(&bars.s_full), 1);
        mbar_init(smem_u32(&bars.dp_full), 1);
        mbar_init(smem_u32(&bars.p_ready[0]), 256);
        mbar_init(smem_u32(&bars.p_ready[1]), 256);
        mbar_init(smem_u32(&bars.ds_ready), 256);
        mbar_init(smem_u32(&bars.acc_full), 1);
        fence_mbar_init();
    }
    if (warp == 9) {
        tmem_alloc(smem_u32(&tmem_base_s), kTmemCols);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_base_s, 0);
    volatile uint32_t* abortp = &abort_flag;
    auto head_of = [&](int i) { return hk * p.g.group + (first + i) / per_head; };
    auto row_of = [&](int i) { return (span.t0 + (first + i) % per_head) * kWinT; };

    if (warp == 8) {
        if (lane == 0 && n > 0) {
            mbar_arrive_expect_tx(smem_u32(&bars.kv_full), 2 * C::kTile);
            tma_load_rows(smem_u32(sK), &tmK, smem_u32(&bars.kv_full), key0, hk, b);
            tma_load_rows(smem_u32(sV), &tmV, smem_u32(&bars.kv_full), key0, hk, b);
            Ring ring;
            bool ok = true;
            for (int i = 0; i < n; ++i, ring.advance<C::kQ>()) {
                const int h = head_of(i), row = row_of(i);
                ok = mbar_wait(smem_u32(&bars.q_empty[ring.stage]), ring.phase ^ 1, abortp);
                if (!ok) break;
                const uint32_t bar = smem_u32(&bars.q_full[ring.stage]), rows = smem_u32(sR) + ring.stage * C::kRows;
                const long long at = ((long long)b * p.g.heads + h) * p.n_pad + row;
                mbar_arrive_expect_tx(bar, C::kTile + C::kRows);
                tma_load_rows(smem_u32(sQ) + ring.stage * C::kTile, &tmQ, bar, row, h, b);
                bulk_load(rows, p.neg_lse2 + at, kWinT * 4, bar);
                bulk_load(rows + kWinT * 4, p.neg_delta + at, kWinT * 4, bar);
                ok = mbar_wait(smem_u32(&bars.o_empty[ring.stage]), ring.phase ^ 1, abortp);
                if (!ok) break;
                mbar_arrive_expect_tx(smem_u32(&bars.o_full[ring.stage]), C::kTile);
                tma_load_rows(smem_u32(sG) + ring.stage * C::kTile, &tmG, smem_u32(&bars.o_full[ring.stage]), row, h, b);
            }
            if (!ok) let_copies_land();
        }
    } else if (warp == 9) {
        // Order: S(0), dP(0); then for every tile i: dV(i) behind its P, S(i + 1) in the place of that P, dK(i) behind its dS,
        // dP(i + 1) in the place of that dS.  The softmax of S(i + 1) runs beside dK(i) and dP(i + 1), that of dP(i) beside dV(i)
        // and S(i + 1).
        constexpr uint32_t idesc_s = make_idesc_f32(kWinT, kWinT, 0, 0, F16), idesc_g = make_idesc_f32(kWinT, D, 0, 1, F16);
        const uint64_t descK = make_smem_desc_sw128(smem_u32(sK), 16, 1024), descV = make_smem_desc_sw128(smem_u32(sV), 16, 1024);
        const uint64_t descQ = make_smem_desc_sw128(smem_u32(sQ), 16, 1024), descG = make_smem_desc_sw128(smem_u32(sG), 16, 1024);
        const uint64_t descQt = make_smem_desc_sw128(smem_u32(sQ), SUB, 1024), descGt = make_smem_desc_sw128(smem_u32(sG), SUB, 1024);
        const bool leader = elect_one();
        auto product = [&](uint32_t d, uint64_t a, uint64_t b0) {
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
                const uint64_t off = (uint64_t)(((kk / 4) * SUB + (kk % 4) * 32) >> 4);
                mma_ss(d, a + off, b0 + off, idesc_s, kk > 0);
            }
        };
        auto gradient = [&](uint32_t d, uint32_t a, uint64_t b0, bool begin) {
#pragma unroll
            for (int kk = 0; kk < 8; ++kk)
                mma_ts(d, a + (kk < 4 ? kk * 8 : 64 + (kk - 4) * 8), b0 + (uint64_t)(kk * 128), idesc_g, (begin && kk == 0) ? 0u : 1u);
        };
        Ring cur, next;
        bool ok = n > 0 && mbar_wait_warp(smem_u32(&bars.kv_full), 0, abortp) && mbar_wait_warp(smem_u32(&bars.q_full[0]), 0, abortp);
        if (ok) {
            tc_fence_after();
            if (leader) {
                product(tmem + C::kS, descK, descQ);
                mma_commit(smem_u32(&bars.s_full));
            }
            ok = mbar_wait_warp(smem_u32(&bars.o_full[0]), 0, abortp);
            tc_fence_after();
            if (ok && leader) {
                product(tmem + C::kDP, descV, descG);
                mma_commit(smem_u32(&bars.dp_full));
            }
        }
        next.advance<C::kQ>();
        for (int i = 0; ok && i < n; ++i) {
            const uint64_t g0 = descGt + (uint64_t)((cur.stage * C::kTile) >> 4);
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                ok = ok && mbar_wait_warp(smem_u32(&bars.p_ready[part]), i & 1, abortp);
                if (!ok) break;
                tc_fence_after();
                if (leader) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int kk = (e >> 1) * 4 + part * 2 + (e & 1);  // 16 query rows, of either warpgroup's 64
                        mma_ts(tmem + C::kDV, tmem + C::kS + (kk < 4 ? kk * 8 : 64 + (kk - 4) * 8), g0 + (uint64_t)(kk * 128), idesc_g,
                               (i > 0 || part > 0 || e > 0) ? 1u : 0u);
                    }
                }
            }
            if (!ok) break;
            if (leader) mma_commit(smem_u32(&bars.o_empty[cur.stage]));
            if (i + 1 < n) {
                ok = mbar_wait_warp(smem_u32(&bars.q_full[next.stage]), next.phase, abortp);
                if (!ok) break;
                tc_fence_after();
                if (leader) {
                    product(tmem + C::kS, descK, descQ + (uint64_t)((next.stage * C::kTile) >> 4));
                    mma_commit(smem_u32(&bars.s_full));
                }
            }
            ok = mbar_wait_warp(smem_u32(&bars.ds_ready), i & 1, abortp);
            if (!ok) break;
            tc_fence_after();
            if (leader) {
                gradient(tmem + C::kDK, tmem + C::kDP, descQt + (uint64_t)((cur.stage * C::kTile) >> 4), i == 0);
                mma_commit(smem_u32(&bars.q_empty[cur.stage]));
                if (i == n - 1) mma_commit(smem_u32(&bars.acc_full));
            }
            if (i + 1 < n) {
                ok = mbar_wait_warp(smem_u32(&bars.o_full[next.stage]), next.phase, abortp);
                if (!ok) break;
                tc_fence_after();
                if (leader) {
                    product(tmem + C::kDP, descV, descG + (uint64_t)((next.stage * C::kTile) >> 4));
                    mma_commit(smem_u32(&bars.dp_full));
                }
            }
            cur.advance<C::kQ>();
            next.advance<C::kQ>();
        }
    } else {
        const int x = warp >> 2, tw = tid & 127, key = key0 + tw;
        const uint32_t t_lane = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t t_s = t_lane + C::kS + x * 64, t_dp = t_lane + C::kDP + x * 64;
        const float c2 = p.scale_log2;
        bool ok = true;
        Ring ring;
        for (int i = 0; i < n; ++i, ring.advance<C::kQ>()) {
            const int row0 = row_of(i), pos0 = seq.start + row0;
            const bool rows_ok = pos0 >= 0 && pos0 + kWinT <= seq.len;
            const bool full = rows_ok && key0 + kWinT <= seq.len && key0 + kWinT - 1 <= pos0 + p.g.right &&
                              (pos0 + kWinT - 1 <= key0 + p.g.left || key0 + kWinT <= p.g.sinks);
            const float4* lse = reinterpret_cast<const float4*>(sR + ring.stage * C::kRows) + x * 16;
            const float4* del = lse + kWinT / 4;  // (both negated)
            ok = mbar_wait_warp(smem_u32(&bars.q_full[ring.stage]), ring.phase, abortp) && mbar_wait_warp(smem_u32(&bars.s_full), i & 1, abortp);
            if (!ok) break;
            tc_fence_after();
            uint32_t r[64];
            tmem_ld32(t_s, r);
            tmem_ld32(t_s + 32, r + 32);
            tc_wait_ld();
            const uint64_t c22 = pack_f32x2(c2, c2);
            uint32_t bits[2] = {0xffffffffu, 0xffffffffu};
            if (!full) {
                bits[0] = key_bits(p.g, seq, key, row0 + x * 64);
                bits[1] = key_bits(p.g, seq, key, row0 + x * 64 + 32);
                if (!rows_ok) {  // rows at no position may hold anything: their weight is zero, which times NaN would not be
                    ok = mbar_wait_warp(smem_u32(&bars.o_full[ring.stage]), ring.phase, abortp);
                    if (!ok) break;
                    if (pos0 + tw < 0 || pos0 + tw >= seq.len) zero_row<D>((x ? sQ : sG) + ring.stage * C::kTile, tw);
                    fence_proxy_async_smem();
                }
            }
            // P goes out in two parts of 32 columns: the first part's products run beside the second's exponentials
#pragma unroll
            for (int part = 0; part < 2; ++part) {
#pragma unroll
                for (int c = part * 32; c < part * 32 + 32; c += 4) {
                    const float4 l = lse[c / 4];
                    float a0, a1, a2, a3;
                    unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(r[c]), __uint_as_float(r[c + 1])), c22, pack_f32x2(l.x, l.y)), a0, a1);
                    unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(r[c + 2]), __uint_as_float(r[c + 3])), c22, pack_f32x2(l.z, l.w)), a2, a3);
                    r[c] = __float_as_uint(ex2_approx(a0));
                    r[c + 1] = __float_as_uint(ex2_approx(a1));
                    r[c + 2] = __float_as_uint(ex2_approx(a2));
                    r[c + 3] = __float_as_uint(ex2_approx(a3));
                }
                if (!full) {
#pragma unroll
                    for (int c = 0; c < 32; ++c) r[part * 32 + c] = (bits[part] & (1u << c)) ? r[part * 32 + c] : 0u;
                }
                uint32_t q[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) q[e] = pack_16x2<F16>(__uint_as_float(r[part * 32 + 2 * e]), __uint_as_float(r[part * 32 + 2 * e + 1]));
                tmem_st16(t_s + part * 16, q);
                tc_wait_st();
                tc_fence_before();
                mbar_arrive(smem_u32(&bars.p_ready[part]));
            }
            ok = mbar_wait_warp(smem_u32(&bars.dp_full), i & 1, abortp);
            if (!ok) break;
            tc_fence_after();
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                uint32_t d[32];
                tmem_ld32(t_dp + c * 32, d);
                tc_wait_ld();
#pragma unroll
                for (int e = 0; e < 32; e += 4) {
                    const float4 l = del[c * 8 + e / 4];
                    float a0, a1, a2, a3;
                    unpack_f32x2(mul_f32x2(add_f32x2(pack_f32x2(__uint_as_float(d[e]), __uint_as_float(d[e + 1])), pack_f32x2(l.x, l.y)),
                                           pack_f32x2(__uint_as_float(r[c * 32 + e]), __uint_as_float(r[c * 32 + e + 1]))), a0, a1);
                    unpack_f32x2(mul_f32x2(add_f32x2(pack_f32x2(__uint_as_float(d[e + 2]), __uint_as_float(d[e + 3])), pack_f32x2(l.z, l.w)),
                                           pack_f32x2(__uint_as_float(r[c * 32 + e + 2]), __uint_as_float(r[c * 32 + e + 3]))), a2, a3);
                    d[e] = __float_as_uint(a0);
                    d[e + 1] = __float_as_uint(a1);
                    d[e + 2] = __float_as_uint(a2);
                    d[e + 3] = __float_as_uint(a3);
                }
                if (!full) {
#pragma unroll
                    for (int e = 0; e < 32; ++e) d[e] = (bits[c] & (1u << e)) ? d[e] : 0u;
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) r[c * 32 + e] = pack_16x2<F16>(__uint_as_float(d[2 * e]), __uint_as_float(d[2 * e + 1]));
            }
            tmem_st16(t_dp, r);
            tmem_st16(t_dp + 16, r + 32);
            tc_wait_st();
            tc_fence_before();
            mbar_arrive(smem_u32(&bars.ds_ready));
        }
        // Warps 0-3 write dV, warps 4-7 dK.
        if (n > 0) ok = ok && mbar_wait_warp(smem_u32(&bars.acc_full), 0, abortp);
        tc_fence_after();
        if (ok) {
            const uint32_t t_acc = t_lane + (x ? C::kDK : C::kDV);
            if (shares > 1) {
                float* out = p.partial + ((((long long)bh * p.sink_tiles + kt) * shares + share) * 2 + x) * kWinT * D + tw * D;
#pragma unroll 1
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t o[32];
                    if (n > 0) {
                        tmem_ld32(t_acc + c * 32, o);
                        tc_wait_ld();
                    }
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        reinterpret_cast<uint4*>(out + c * 32)[q] = n > 0 ? make_uint4(o[q * 4], o[q * 4 + 1], o[q * 4 + 2], o[q * 4 + 3]) : make_uint4(0, 0, 0, 0);
                }
            } else {
                uint16_t* out = x ? p.dK + (long long)b * p.k_batch + (long long)hk * p.k_head + (long long)key * p.k_row
                                  : p.dV + (long long)b * p.v_batch + (long long)hk * p.v_head + (long long)key * p.v_row;
                store_row<D, F16>(t_acc, x ? p.scale : 1.f, n == 0, key < p.g.N_kv ? out : nullptr);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (tid == 0 && abort_flag) atomicExch(p.status, (int)BSA_ERR_DEVICE_TIMEOUT);
    if (warp == 9) tmem_dealloc(tmem, kTmemCols);
}

// The shares of the sinks' tiles, added up in their order.  Eight columns a thread.
template <int D, bool F16>
__global__ void __launch_bounds__(256) window_sink_sum_kernel(const __grid_constant__ BwdParams p) {
    constexpr int PER = kWinT * D / 8;  // threads of a tile
    const int unit = blockIdx.x * 256 + threadIdx.x;
    const int which = blockIdx.z;
    const int tile = unit / PER, e = (unit - tile * PER) * 8, row = e / D, col = e - row * D;
    if (tile >= p.sink_tiles) return;
    const int bh = blockIdx.y, b = bh / p.g.heads_kv, hk = bh - b * p.g.heads_kv, key = tile * kWinT + row;
    if (key >= p.g.N_kv) return;
    float s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    const float* src = p.partial + (((long long)bh * p.sink_tiles + tile) * p.sink_shares * 2 + which) * kWinT * D + e;
    for (int k = 0; k < p.sink_shares; ++k, src += 2 * kWinT * D) {
        const float4 a = __ldg(reinterpret_cast<const float4*>(src)), c = __ldg(reinterpret_cast<const float4*>(src) + 1);
        s[0] += a.x; s[1] += a.y; s[2] += a.z; s[3] += a.w;
        s[4] += c.x; s[5] += c.y; s[6] += c.z; s[7] += c.w;
    }
    const float f = which ? p.scale : 1.f;
    uint16_t* out = which ? p.dK + (long long)b * p.k_batch + (long long)hk * p.k_head + (long long)key * p.k_row
                          : p.dV + (long long)b * p.v_batch + (long long)hk * p.v_head + (long long)key * p.v_row;
    *reinterpret_cast<uint4*>(out + col) = make_uint4(pack_16x2<F16>(s[0] * f, s[1] * f), pack_16x2<F16>(s[2] * f, s[3] * f),
                                                      pack_16x2<F16>(s[4] * f, s[5] * f), pack_16x2<F16>(s[6] * f, s[7] * f));
}

// ------------------------------------------------------------------------------------------ host side
struct Layout {
    int n_pad, n_qt, n_kt, sink_tiles, sink_shares;
    int64_t lse2, delta, partial, bytes;  // offsets in the workspace
};
Layout layout_of(const WindowArgs& a) {
    Layout l = {};
    const WindowGeom& g = a.g;
    l.n_qt = (g.N + kWinT - 1) / kWinT;
    l.n_kt = (g.N_kv + kWinT - 1) / kWinT;
    l.n_pad = l.n_qt * kWinT;
    // A sink's key is seen by every query behind it, another by those of its window.  Where that is many times fewer, the sinks'
    // tiles are cut into shares about as long as the other tiles' work, as long as no more than four items per SM come out
    // of it (their partial sums are 128 KB each at d = 128).
    const int64_t window = ((int64_t)g.left + g.right + 2 * kWinT - 1) / kWinT + 1;
    const int64_t tiles = (g.sinks + kWinT - 1) / kWinT;
    if (tiles > 0 && window * 2 <= l.n_qt) {
        l.sink_tiles = (int)(tiles < l.n_kt ? tiles : l.n_kt);
        const int64_t most = 4 * (int64_t)a.num_sms / ((int64_t)g.batch * g.heads_kv * l.sink_tiles);
        int64_t shares = (l.n_qt + window - 1) / window;
        if (shares > most) shares = most;
        l.sink_shares = (int)(shares > 1 ? shares : 1);
        if (l.sink_shares == 1) l.sink_tiles = 0;
    }
    if (l.sink_tiles == 0) l.sink_shares = 1;
    const int64_t rows = (int64_t)g.batch * g.heads * l.n_pad * 4;
    l.lse2 = 0;
    l.delta = rows;
    l.partial = (2 * rows + 255) / 256 * 256;
    l.bytes = l.partial + (l.sink_tiles ? (int64_t)g.batch * g.heads_kv * l.sink_tiles * l.sink_shares * 2 * kWinT * a.d * 4 : 0);
    return l;
}

template <int D, bool F16>
cudaError_t launch(const WindowArgs& a, const Layout& l, const bsa_view_t& Q, const bsa_view_t& K, const bsa_view_t& V, const bsa_view_t& O,
                   const bsa_view_t& G, const float* LSE, const BwdParams& p, float* lse2, float* delta, cudaStream_t stream) {
    const WindowGeom& g = a.g;
    CUtensorMap tq, tk, tv, tg;
    if (!encode_view_map(&tq, Q, g.N, g.heads, g.batch, D, kWinT, F16) || !encode_view_map(&tg, G, g.N, g.heads, g.batch, D, kWinT, F16) ||
        !encode_view_map(&tk, K, g.N_kv, g.heads_kv, g.batch, D, kWinT, F16) || !encode_view_map(&tv, V, g.N_kv, g.heads_kv, g.batch, D, kWinT, F16))
        return cudaErrorInvalidValue;
    const auto dq = window_dq_kernel<D, F16>;
    const auto dkv = window_dkv_kernel<D, F16>;
    static std::atomic<bool> allowed[kMaxDevices];
    if (!allowed[a.device].load(std::memory_order_relaxed)) {
        cudaError_t e = cudaFuncSetAttribute(dq, cudaFuncAttributeMaxDynamicSharedMemorySize, DqCfg<D>::kSmem);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(dkv, cudaFuncAttributeMaxDynamicSharedMemorySize, DkvCfg<D>::kSmem);
        if (e != cudaSuccess) return e;
        allowed[a.device].store(true, std::memory_order_relaxed);
    }
    window_delta_kernel<D, F16><<<dim3((unsigned)(l.n_pad / 32), (unsigned)(g.batch * g.heads)), 256, 0, stream>>>(
        g, static_cast<const uint16_t*>(O.data), static_cast<const uint16_t*>(G.data), O.batch, O.head, O.row, G.batch, G.head, G.row, LSE, lse2, delta, l.n_pad);
    dq<<<(unsigned)(l.n_qt * g.batch * g.heads), kThreads, DqCfg<D>::kSmem, stream>>>(tq, tk, tv, tg, p);
    const unsigned items = (unsigned)(g.batch * g.heads_kv) * (unsigned)(l.sink_tiles * l.sink_shares + (l.n_kt - l.sink_tiles));
    dkv<<<items, kThreads, DkvCfg<D>::kSmem, stream>>>(tq, tk, tv, tg, p);
    count_launch(3);
    if (l.sink_tiles) {
        window_sink_sum_kernel<D, F16><<<dim3((unsigned)(l.sink_tiles * kWinT * D / 8 / 256), (unsigned)(g.batch * g.heads_kv), 2), 256, 0, stream>>>(p);
        count_launch();
    }
    return cudaGetLastError();
}

}  // namespace
}  // namespace bsa

using namespace bsa;

extern "C" int64_t bsa_window_workspace_bytes(const bsa_window_desc_t* t) {
    WindowArgs a;
    return window_args(t, &a) == BSA_OK ? layout_of(a).bytes : 0;
}

extern "C" bsa_status_t bsa_window_backward(const bsa_window_desc_t* t, const bsa_view_t* Q, const bsa_view_t* K, const bsa_view_t* V,
                                            const bsa_view_t* O, const float* LSE, const bsa_view_t* dO, const bsa_view_t* dQ,
                                            const bsa_view_t* dK, const bsa_view_t* dV, void* workspace, int64_t workspace_bytes, void* stream_v) {
    if (!t || !LSE || (reinterpret_cast<uintptr_t>(LSE) & 3)) return BSA_ERR_INVALID_ARG;
    for (const bsa_view_t* v : {Q, O, dO, dQ})
        if (!view_ok(v, t->batch, t->heads, t->N)) return BSA_ERR_INVALID_ARG;
    for (const bsa_view_t* v : {K, V, dK, dV})
        if (!view_ok(v, t->batch, t->heads_kv, t->N_kv)) return BSA_ERR_INVALID_ARG;
    WindowArgs a;
    const bsa_status_t st = window_args(t, &a);
    if (st != BSA_OK) return st;
    const Layout l = layout_of(a);
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < l.bytes) return BSA_ERR_INVALID_ARG;
    if ((int64_t)l.n_qt * a.g.batch * a.g.heads > INT_MAX / 2 || (int64_t)(l.n_kt + 8 * a.num_sms) * a.g.batch * a.g.heads_kv > INT_MAX / 2)
        return BSA_ERR_UNSUPPORTED;
    BwdParams p = {};
    p.g = a.g;
    p.scale = a.scale;
    p.scale_log2 = a.scale * 1.4426950408889634f;
    char* ws = static_cast<char*>(workspace);
    float* lse2 = reinterpret_cast<float*>(ws + l.lse2);
    float* delta = reinterpret_cast<float*>(ws + l.delta);
    p.n_pad = l.n_pad;
    p.neg_lse2 = lse2;
    p.neg_delta = delta;
    p.partial = reinterpret_cast<float*>(ws + l.partial);
    p.dQ = static_cast<uint16_t*>(dQ->data);
    p.dK = static_cast<uint16_t*>(dK->data);
    p.dV = static_cast<uint16_t*>(dV->data);
    p.q_batch = dQ->batch; p.q_head = dQ->head; p.q_row = dQ->row;
    p.k_batch = dK->batch; p.k_head = dK->head; p.k_row = dK->row;
    p.v_batch = dV->batch; p.v_head = dV->head; p.v_row = dV->row;
    p.n_qt = l.n_qt;
    p.n_kt = l.n_kt;
    p.longest_first = a.g.left >= a.g.N_kv;
    p.sink_tiles = l.sink_tiles;
    p.sink_shares = l.sink_shares;
    cudaError_t e = window_status_word(a.device, &p.status);
    const cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_v);
    if (e == cudaSuccess)
        e = a.d == 64 ? (a.f16 ? launch<64, true>(a, l, *Q, *K, *V, *O, *dO, LSE, p, lse2, delta, stream) : launch<64, false>(a, l, *Q, *K, *V, *O, *dO, LSE, p, lse2, delta, stream))
                      : (a.f16 ? launch<128, true>(a, l, *Q, *K, *V, *O, *dO, LSE, p, lse2, delta, stream) : launch<128, false>(a, l, *Q, *K, *V, *O, *dO, LSE, p, lse2, delta, stream));
    if (e != cudaSuccess) {
        set_cuda_err(e, "bsa_window_backward");
        return BSA_ERR_CUDA;
    }
    return BSA_OK;
}
