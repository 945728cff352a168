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
// every gradient is summed in tensor memory by one CTA.  Only the keys of the first tokens, seen by every query, and the keys of calls
// that would leave the GPU idle, are cut into several shares of their queries, whose sums are added up in a fixed order by a fourth
// kernel.
// In both kernels eight softmax warps (thread = row of a tile), one warp that copies and one that issues the products.
// 16384 rows, 16 + 4 heads, d = 128, causal window 2048, 16 sinks: delta 24 us (bytes), dQ 359, dK and dV 470, the sinks' sum 5.  Per tile dQ
// takes 2230 clk where its three products are 1536: two of them read both operands from shared memory, 224 KB a tile with the copies, at
// 128 B/clk; dK and dV take 3000 for 2048 (tensor pipe 76 % busy): P, its product, the next scores and their exponentials follow each other,
// since S, dO V^T and both accumulators fill tensor memory.  An own chain for each half of the query rows: 599 us.
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
// Half: P, at most one and over a window of thousands of keys mostly below 2^-14, where half loses bits, is computed 2^14 times as large
// (half ends at 2^16); dV is scaled back at its end.  dS keeps its size: it follows dO, whose scale is the caller's.
template <bool F16>
constexpr float kShift = F16 ? 14.0f : 0.0f;
template <bool F16>
constexpr float kUnshift = F16 ? 1.0f / 16384.0f : 1.0f;

struct BwdParams {
    WindowGeom g;
    float scale, scale_log2;
    int n_pad;             // N rounded up to whole tiles
    const float* neg_lse2;   // [batch * heads][n_pad]: kShift - LSE in the exp2 domain (-inf for rows that see nothing: their P is zero)
    const float* neg_delta;  // -D * kUnshift: what is multiplied with the larger P is that much smaller
    uint16_t* dQ;
    uint16_t* dK;
    uint16_t* dV;
    long long q_batch, q_head, q_row, k_batch, k_head, k_row, v_batch, v_head, v_row;  // strides of the gradients
    ItemOrder dq, dkv;                 // query tiles from a sequence's last to its first; key tiles that are not cut into shares
    int n_shared;                      // items in front of those: shares of the sinks' tiles
    Divisor heads, heads_kv, group;    // heads; key heads; heads that share a key head
    Divisor shares, shared;            // shares of a tile, of all of a sequence's tiles
    int sink_tiles, sink_shares;            // key tiles in front that are cut into shares (0: none)
    int wide_q, wide_k, wide_v;             // gradients whose rows lie on 32-byte boundaries
    float* partial;        // [batch * heads_kv][sink_tiles][sink_shares][dV, dK][128][D]
    int* status;
    int withhold;          // test hook: no copy of the first tile of V (dQ) or of dO (dK, dV)
};

struct __align__(8) DqBarriers {
    uint64_t q_full, q_empty, k_full[4], k_empty[4], v_full, v_empty;
    uint64_t s_full[2], s_free, dp_full[2], ds_ready[2], acc_full, acc_free;  // (one s_full for each of its readers)
};
struct __align__(8) DkvBarriers {
    uint64_t kv_full, kv_empty, q_full[2], q_empty[2], o_full[2], o_empty[2];
    uint64_t s_full, dp_full, p_ready[2], ds_ready, acc_full, acc_free;
};

// 1-D copy of whole 16-byte pieces, counted in bytes on an mbarrier
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}
// The k-th item of a persistent CTA, dealt in alternating directions (the longest items come first).
__device__ __forceinline__ int item_index(int k) {
    const int G = gridDim.x;
    return k * G + ((k & 1) ? (G - 1 - (int)blockIdx.x) : (int)blockIdx.x);
}

// Columns [c0 * 32, c1 * 32) of a row of an accumulator, times `f`, to global memory in the element type; out null: nowhere.
template <bool F16>
__device__ __forceinline__ void store_row(uint32_t t_acc, int c0, int c1, float f, bool zero, uint16_t* out, int wide) {
#pragma unroll 1
    for (int c = c0; c < c1; ++c) {
        uint32_t o[32];
        tmem_ld32(t_acc + c * 32, o);
        tc_wait_ld();
        if (out) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                uint32_t v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    v[e] = zero ? 0u : pack_16x2<F16>(__uint_as_float(o[q * 16 + 2 * e]) * f, __uint_as_float(o[q * 16 + 2 * e + 1]) * f);
                st_global_v8_or_2v4(out + c * 32 + q * 16, v, wide);
            }
        }
        __syncwarp();
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
        neg_delta[(long long)bh * n_pad + row] = -sum * kUnshift<F16>;
        neg_lse2[(long long)bh * n_pad + row] = seen ? fmaf(LSE[(long long)bh * g.N + row], -1.4426950408889634f, kShift<F16>) : -INFINITY;
    }
}

// ------------------------------------------------------------------------------------------ dQ
template <int D>
struct DqCfg {
    static constexpr int kTile = kWinT * D * 2;
    static constexpr int kK = 4;                       // K tiles in the ring (a tile lives from its S to its dQ, two tiles later); V has one
    static constexpr int kSmem = (2 + kK + 1) * kTile;  // Q, dO, K, V
    static constexpr uint32_t kS = 0, kDP0 = 128, kDP1 = 256, kDQ = 384;
};

struct DqItem {
    int b, h, hk, row0;
    Sequence seq;
    KeyRange range;
    TileSpan tiles;
};
__device__ __forceinline__ bool load_item(const BwdParams& p, int k, DqItem& it) {
    const int idx = item_index(k);
    if (idx >= p.dq.n_items) return false;
    int tile;
    const int bh = p.dq.row_of(idx, tile), qt = p.dq.n_tiles - 1 - tile;
    it.b = p.heads.div(bh, it.h);
    int rest;
    it.hk = p.group.div(it.h, rest);
    it.row0 = qt * kWinT;
    it.seq = load_sequence(p.g, it.b);
    it.range = key_range(p.g, it.seq, it.row0, it.row0 + kWinT);
    it.tiles = tile_span(it.range);
    return true;
}

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
    if (tid == 0) {
        abort_flag = 0;
        mbar_init(smem_u32(&bars.q_full), 1);
        mbar_init(smem_u32(&bars.q_empty), 1);
        mbar_init(smem_u32(&bars.v_full), 1);
        mbar_init(smem_u32(&bars.v_empty), 1);
        for (int i = 0; i < C::kK; ++i) {
            mbar_init(smem_u32(&bars.k_full[i]), 1);
            mbar_init(smem_u32(&bars.k_empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&bars.s_full[i]), 1);
            mbar_init(smem_u32(&bars.dp_full[i]), 1);
            mbar_init(smem_u32(&bars.ds_ready[i]), 128);
        }
        mbar_init(smem_u32(&bars.s_free), 128);
        mbar_init(smem_u32(&bars.acc_full), 1);
        mbar_init(smem_u32(&bars.acc_free), 256);
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
    DqItem it;

    if (warp == 8) {
        if (lane == 0) {
            Ring rk;
            uint32_t n_q = 0, n_v = 0;
            bool ok = true;
            for (int k = 0; ok && load_item(p, k, it); ++k) {
                const int n = it.tiles.count();
                if (n == 0) continue;
                auto copy_k = [&](int j) -> bool {
                    if (!mbar_wait(smem_u32(&bars.k_empty[rk.stage]), rk.phase ^ 1, abortp)) return false;
                    mbar_arrive_expect_tx(smem_u32(&bars.k_full[rk.stage]), C::kTile);
                    tma_load_rows(smem_u32(sK) + rk.stage * C::kTile, &tmK, smem_u32(&bars.k_full[rk.stage]), it.tiles.tile(j) * kWinT, it.hk, it.b);
                    rk.advance<C::kK>();
                    return true;
                };
                ok = mbar_wait(smem_u32(&bars.q_empty), (n_q & 1) ^ 1, abortp);
                if (!ok) break;
                mbar_arrive_expect_tx(smem_u32(&bars.q_full), 2 * C::kTile);
                tma_load_rows(smem_u32(sQ), &tmQ, smem_u32(&bars.q_full), it.row0, it.h, it.b);
                tma_load_rows(smem_u32(sG), &tmG, smem_u32(&bars.q_full), it.row0, it.h, it.b);
                ++n_q;
                ok = copy_k(0);
                for (int j = 0; ok && j < n; ++j) {  // K a tile ahead of V
                    if (j + 1 < n) ok = copy_k(j + 1);
                    ok = ok && mbar_wait(smem_u32(&bars.v_empty), (n_v & 1) ^ 1, abortp);
                    if (!ok) break;
                    if (!(p.withhold && n_v == 0)) {
                        mbar_arrive_expect_tx(smem_u32(&bars.v_full), C::kTile);
                        tma_load_rows(smem_u32(sV), &tmV, smem_u32(&bars.v_full), it.tiles.tile(j) * kWinT, it.hk, it.b);
                    }
                    ++n_v;
                }
            }
        }
    } else if (warp == 9) {
        // Tile t (counted over the CTA's items) belongs to softmax warpgroup t mod 2 and has dP buffer t mod 2, where its dS goes as
        // well; S has one buffer, free as soon as it has been read.  Order within an item: S(0), dP(0), S(1), dP(1); then for every
        // tile i: S(i + 2), dQ(i) behind its dS, dP(i + 2).
        constexpr uint32_t idesc_s = make_idesc_f32(kWinT, kWinT, 0, 0, F16), idesc_dq = make_idesc_f32(kWinT, D, 0, 1, F16);
        const uint64_t descQ = make_smem_desc_sw128(smem_u32(sQ), 16, 1024), descG = make_smem_desc_sw128(smem_u32(sG), 16, 1024);
        const uint64_t descK = make_smem_desc_sw128(smem_u32(sK), 16, 1024), descV = make_smem_desc_sw128(smem_u32(sV), 16, 1024);
        const uint64_t descKt = make_smem_desc_sw128(smem_u32(sK), SUB, 1024);
        const bool leader = elect_one();
        Ring rs, rq;  // K of the next S and of the next dQ
        uint32_t n_it = 0, n_v = 0, g = 0;
        bool ok = true;
        auto product = [&](uint32_t d, uint64_t a, uint64_t b0) {
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
                const uint64_t off = (uint64_t)(((kk / 4) * SUB + (kk % 4) * 32) >> 4);
                mma_ss(d, a + off, b0 + off, idesc_s, kk > 0);
            }
        };
        auto issue_s = [&](uint32_t t) -> bool {
            if (t >= 1 && !mbar_wait_warp(smem_u32(&bars.s_free), (t - 1) & 1, abortp)) return false;
            if (!mbar_wait_warp(smem_u32(&bars.k_full[rs.stage]), rs.phase, abortp)) return false;
            tc_fence_after();
            if (leader) {
                product(tmem + C::kS, descQ, descK + (uint64_t)((rs.stage * C::kTile) >> 4));
                mma_commit(smem_u32(&bars.s_full[t & 1]));
            }
            rs.advance<C::kK>();
            return true;
        };
        auto issue_dp = [&](uint32_t t, bool last) -> bool {
            if (!mbar_wait_warp(smem_u32(&bars.v_full), n_v & 1, abortp)) return false;
            ++n_v;
            tc_fence_after();
            if (leader) {
                product(tmem + ((t & 1) ? C::kDP1 : C::kDP0), descG, descV);
                mma_commit(smem_u32(&bars.dp_full[t & 1]));
                mma_commit(smem_u32(&bars.v_empty));
                if (last) mma_commit(smem_u32(&bars.q_empty));  // (its S is in front of it)
            }
            return true;
        };
        for (int k = 0; ok && load_item(p, k, it); ++k) {
            const int n = it.tiles.count();
            if (n == 0) continue;
            ok = mbar_wait_warp(smem_u32(&bars.q_full), n_it & 1, abortp);
            ok = ok && issue_s(g) && issue_dp(g, n == 1);
            if (ok && n > 1) ok = issue_s(g + 1) && issue_dp(g + 1, n == 2);
            for (int i = 0; ok && i < n; ++i) {
                const uint32_t t = g + i;
                if (i + 2 < n) ok = issue_s(t + 2);
                if (ok && i == 0) ok = mbar_wait_warp(smem_u32(&bars.acc_free), (n_it & 1) ^ 1, abortp);  // the last item's gradient is out
                ok = ok && mbar_wait_warp(smem_u32(&bars.ds_ready[t & 1]), (t >> 1) & 1, abortp);
                if (!ok) break;
                tc_fence_after();
                if (leader) {
                    const uint64_t k0 = descKt + (uint64_t)((rq.stage * C::kTile) >> 4);
                    const uint32_t a_ds = tmem + ((t & 1) ? C::kDP1 : C::kDP0);
#pragma unroll
                    for (int kk = 0; kk < 8; ++kk)
                        mma_ts(tmem + C::kDQ, a_ds + kk * 8, k0 + (uint64_t)(kk * 128), idesc_dq, (i > 0 || kk > 0) ? 1u : 0u);
                    mma_commit(smem_u32(&bars.k_empty[rq.stage]));
                    if (i == n - 1) mma_commit(smem_u32(&bars.acc_full));
                }
                rq.advance<C::kK>();
                if (i + 2 < n) ok = issue_dp(t + 2, i + 3 == n);
            }
            g += (uint32_t)n;
            ++n_it;
        }
    } else {
        const int x = warp >> 2, tw = tid & 127;
        const uint32_t t_lane = tmem + ((uint32_t)((warp & 3) * 32) << 16), t_dp = t_lane + (x ? C::kDP1 : C::kDP0);
        const uint64_t c22 = pack_f32x2(p.scale_log2, p.scale_log2), unshift2 = pack_f32x2(kUnshift<F16>, kUnshift<F16>);
        uint32_t g = 0, n_it = 0;
        bool ok = true, more = load_item(p, 0, it);
        auto row_value = [&](const float* v) { return __ldg(v + ((long long)it.b * p.g.heads + it.h) * p.n_pad + it.row0 + tw); };
        float neg_lse = more ? row_value(p.neg_lse2) : 0.f, neg_del = more ? row_value(p.neg_delta) : 0.f;
        for (int k = 0; ok && more; ++k) {
            const int n = it.tiles.count();
            const int row = it.row0 + tw, pos = it.seq.start + row;
            const bool seen = pos >= 0 && pos < it.seq.len;
            uint16_t* out = row < p.g.N ? p.dQ + (long long)it.b * p.q_batch + (long long)it.h * p.q_head + (long long)row * p.q_row : nullptr;
            const uint64_t nl2 = pack_f32x2(neg_lse, neg_lse), nd2 = pack_f32x2(neg_del, neg_del);
            for (int i = ((g & 1) == (uint32_t)x) ? 0 : 1; i < n; i += 2) {
                const uint32_t t = g + i;
                const int key0 = it.tiles.tile(i) * kWinT;
                const bool full = tile_is_full(p.g, it.range, key0);
                ok = mbar_wait_warp(smem_u32(&bars.s_full[x]), (t >> 1) & 1, abortp);
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
                    zero_unseen_keys<D, 128>(sK + (t % C::kK) * C::kTile, p.g, it.range, key0, tw);
                    fence_proxy_async_smem();
                }
                ok = mbar_wait_warp(smem_u32(&bars.dp_full[x]), (t >> 1) & 1, abortp);
                if (!ok) break;
                tc_fence_after();
                const RowView view(p.g, it.seq, pos, key0);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t d[32];
                    tmem_ld32(t_dp + c * 32, d);
                    tc_wait_ld();
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        float u, v;
                        unpack_f32x2(mul_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(d[e]), __uint_as_float(d[e + 1])), unshift2, nd2),
                                               pack_f32x2(__uint_as_float(r[c * 32 + e]), __uint_as_float(r[c * 32 + e + 1]))), u, v);
                        d[e] = __float_as_uint(u);
                        d[e + 1] = __float_as_uint(v);
                    }
                    if (!full) {
                        const uint32_t bits = view.bits(c * 32);
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
            if (!ok) break;
            more = load_item(p, k + 1, it);
            if (more) {  // under way while the accumulator is waited for
                neg_lse = row_value(p.neg_lse2);
                neg_del = row_value(p.neg_delta);
            }
            if (n > 0) {
                ok = mbar_wait_warp(smem_u32(&bars.acc_full), n_it & 1, abortp);
                if (!ok) break;
                ++n_it;
                g += (uint32_t)n;
                tc_fence_after();
            }
            // either warpgroup stores half of the columns (nothing seen, n = 0: zeros)
            store_row<F16>(t_lane + C::kDQ, x * (D / 64), (x + 1) * (D / 64), p.scale, !seen || n == 0, out, p.wide_q);
            if (n > 0) {
                tc_fence_before();
                mbar_arrive(smem_u32(&bars.acc_free));
            }
        }
    }
    end_of_cta(abortp, p.status, (int)BSA_ERR_DEVICE_TIMEOUT);
    if (warp == 9) tmem_dealloc(tmem, kTmemCols);
}

// ------------------------------------------------------------------------------------------ dK, dV
template <int D>
struct DkvCfg {
    static constexpr int kTile = kWinT * D * 2;
    static constexpr int kQ = 2;                 // tiles in the rings of Q and of dO
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
// The query rows [lo, hi) that see a key, none behind the last query: positions may follow in its tile, and a key that only they would see
// may hold anything.  And 32 of them from row q0 on as bits.
struct KeyView {
    int lo, hi;
    __device__ __forceinline__ KeyView(const WindowGeom& g, const Sequence& s, int key)
        : lo(max(key - g.right, 0) - s.start), hi(key < s.len ? min(min(key < g.sinks ? s.len : key + g.left + 1, s.len) - s.start, g.N) : 0) {}
    __device__ __forceinline__ uint32_t bits(int q0) const { return bits_below(hi - q0) & ~bits_below(lo - q0); }
};

struct DkvItem {
    int b, hk, bh, kt, share, shares;
    Sequence seq;
    int key0, t0, per_head;  // query tiles t0 .. t0 + per_head - 1 of every head
    int head, tile, n;       // the first of this item's n tiles: head (of those that share the key head), tile behind t0
};
// Items: the shares of the sinks' tiles first (the longest), then the other tiles, a sequence's neighbours side by side.
__device__ __forceinline__ bool load_item(const BwdParams& p, int k, DkvItem& it) {
    int idx = item_index(k);
    if (idx >= p.n_shared + p.dkv.n_items) return false;
    if (idx < p.n_shared) {
        it.bh = p.shared.div(idx, idx);
        it.kt = p.shares.div(idx, it.share);
        it.shares = p.sink_shares;
    } else {
        it.share = 0;
        it.shares = 1;
        it.bh = p.dkv.row_of(idx - p.n_shared, it.kt);  // (the last keys are seen by the fewest rows)
        it.kt += p.sink_tiles;
    }
    it.b = p.heads_kv.div(it.bh, it.hk);
    it.seq = load_sequence(p.g, it.b);
    it.key0 = it.kt * kWinT;
    const RowSpan span = row_span(p.g, it.seq, it.key0);
    it.t0 = span.t0;
    it.per_head = span.t1 - span.t0;
    it.n = it.per_head * p.g.group;
    it.head = it.tile = 0;
    if (it.shares > 1 && it.n > 0) {
        const int all = it.n, first = (int)((long long)all * it.share / it.shares);
        it.n = (int)((long long)all * (it.share + 1) / it.shares) - first;
        it.head = first / it.per_head;
        it.tile = first - it.head * it.per_head;
    }
    return true;
}
// Walks over an item's tiles.
struct Cursor {
    int head, tile;
    __device__ __forceinline__ explicit Cursor(const DkvItem& it) : head(it.head), tile(it.tile) {}
    __device__ __forceinline__ void next(const DkvItem& it) {
        if (++tile == it.per_head) {
            tile = 0;
            ++head;
        }
    }
};

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
    uint8_t* sR = sG + C::kQ * C::kTile;  // [stage][-LSE, -D][128]
    __shared__ DkvBarriers bars;
    __shared__ uint32_t tmem_base_s, abort_flag;
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    if (smem_u32(smem) & 1023u) {  // never expected
        if (tid == 0) atomicExch(p.status, (int)BSA_ERR_CUDA);
        return;
    }
    if (tid == 0) {
        abort_flag = 0;
        mbar_init(smem_u32(&bars.kv_full), 1);
        mbar_init(smem_u32(&bars.kv_empty), 1);
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
        mbar_init(smem_u32(&bars.acc_free), 256);
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
    DkvItem it;

    if (warp == 8) {
        if (lane == 0) {
            Ring ring;
            uint32_t n_it = 0;
            bool ok = true;
            for (int k = 0; ok && load_item(p, k, it); ++k) {
                if (it.n == 0) continue;
                ok = mbar_wait(smem_u32(&bars.kv_empty), (n_it & 1) ^ 1, abortp);
                if (!ok) break;
                ++n_it;
                mbar_arrive_expect_tx(smem_u32(&bars.kv_full), 2 * C::kTile);
                tma_load_rows(smem_u32(sK), &tmK, smem_u32(&bars.kv_full), it.key0, it.hk, it.b);
                tma_load_rows(smem_u32(sV), &tmV, smem_u32(&bars.kv_full), it.key0, it.hk, it.b);
                Cursor at(it);
                for (int i = 0; i < it.n; ++i, ring.advance<C::kQ>(), at.next(it)) {
                    const int h = it.hk * p.g.group + at.head, row = (it.t0 + at.tile) * kWinT;
                    ok = mbar_wait(smem_u32(&bars.q_empty[ring.stage]), ring.phase ^ 1, abortp);
                    if (!ok) break;
                    const uint32_t bar = smem_u32(&bars.q_full[ring.stage]), rows = smem_u32(sR) + ring.stage * C::kRows;
                    const long long from = ((long long)it.b * p.g.heads + h) * p.n_pad + row;
                    mbar_arrive_expect_tx(bar, C::kTile + C::kRows);
                    tma_load_rows(smem_u32(sQ) + ring.stage * C::kTile, &tmQ, bar, row, h, it.b);
                    bulk_load(rows, p.neg_lse2 + from, kWinT * 4, bar);
                    bulk_load(rows + kWinT * 4, p.neg_delta + from, kWinT * 4, bar);
                    ok = mbar_wait(smem_u32(&bars.o_empty[ring.stage]), ring.phase ^ 1, abortp);
                    if (!ok) break;
                    if (p.withhold && n_it == 1 && i == 0) continue;
                    mbar_arrive_expect_tx(smem_u32(&bars.o_full[ring.stage]), C::kTile);
                    tma_load_rows(smem_u32(sG) + ring.stage * C::kTile, &tmG, smem_u32(&bars.o_full[ring.stage]), row, h, it.b);
                }
            }
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
        Ring cur, next;  // of the tile whose gradients, and of the one whose scores come next
        uint32_t n_it = 0, t = 0;
        bool ok = true;
        auto product = [&](uint32_t d, uint64_t a, uint64_t b0) {
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
                const uint64_t off = (uint64_t)(((kk / 4) * SUB + (kk % 4) * 32) >> 4);
                mma_ss(d, a + off, b0 + off, idesc_s, kk > 0);
            }
        };
        auto issue_s = [&]() -> bool {
            if (!mbar_wait_warp(smem_u32(&bars.q_full[next.stage]), next.phase, abortp)) return false;
            tc_fence_after();
            if (leader) {
                product(tmem + C::kS, descK, descQ + (uint64_t)((next.stage * C::kTile) >> 4));
                mma_commit(smem_u32(&bars.s_full));
            }
            return true;
        };
        auto issue_dp = [&](bool last) -> bool {
            if (!mbar_wait_warp(smem_u32(&bars.o_full[next.stage]), next.phase, abortp)) return false;
            tc_fence_after();
            if (leader) {
                product(tmem + C::kDP, descV, descG + (uint64_t)((next.stage * C::kTile) >> 4));
                mma_commit(smem_u32(&bars.dp_full));
                if (last) mma_commit(smem_u32(&bars.kv_empty));  // (its S is in front of it)
            }
            next.advance<C::kQ>();
            return true;
        };
        for (int k = 0; ok && load_item(p, k, it); ++k) {
            const int n = it.n;
            if (n == 0) continue;
            ok = mbar_wait_warp(smem_u32(&bars.kv_full), n_it & 1, abortp);
            ok = ok && issue_s() && issue_dp(n == 1);
            ok = ok && mbar_wait_warp(smem_u32(&bars.acc_free), (n_it & 1) ^ 1, abortp);  // the last item's gradients are out
            ++n_it;
            for (int i = 0; ok && i < n; ++i, ++t) {
                const uint64_t g0 = descGt + (uint64_t)((cur.stage * C::kTile) >> 4), q0 = descQt + (uint64_t)((cur.stage * C::kTile) >> 4);
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    ok = ok && mbar_wait_warp(smem_u32(&bars.p_ready[part]), t & 1, abortp);
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
                if (i + 1 < n) ok = issue_s();
                ok = ok && mbar_wait_warp(smem_u32(&bars.ds_ready), t & 1, abortp);
                if (!ok) break;
                tc_fence_after();
                if (leader) {
#pragma unroll
                    for (int kk = 0; kk < 8; ++kk)
                        mma_ts(tmem + C::kDK, tmem + C::kDP + (kk < 4 ? kk * 8 : 64 + (kk - 4) * 8), q0 + (uint64_t)(kk * 128), idesc_g,
                               (i > 0 || kk > 0) ? 1u : 0u);
                    mma_commit(smem_u32(&bars.q_empty[cur.stage]));
                    if (i == n - 1) mma_commit(smem_u32(&bars.acc_full));
                }
                if (i + 1 < n) ok = issue_dp(i + 2 == n);
                cur.advance<C::kQ>();
            }
        }
    } else {
        // A tile is shared by columns: warpgroup x takes query rows 64 x .. 64 x + 63 of it, thread = key.
        const int x = warp >> 2, tw = tid & 127;
        const uint32_t t_lane = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t t_s = t_lane + C::kS + x * 64, t_dp = t_lane + C::kDP + x * 64;
        const float c2 = p.scale_log2;
        uint32_t t = 0, n_it = 0;
        bool ok = true;
        Ring ring;
        for (int k = 0; ok && load_item(p, k, it); ++k) {
            const int n = it.n, key0 = it.key0, key = key0 + tw;
            const Sequence seq = it.seq;
            const KeyView view(p.g, seq, key);
            Cursor at(it);
            for (int i = 0; i < n; ++i, ++t, ring.advance<C::kQ>(), at.next(it)) {
                const int row0 = (it.t0 + at.tile) * kWinT, pos0 = seq.start + row0;
                const bool rows_ok = pos0 >= 0 && pos0 + kWinT <= seq.len;
                const bool full = rows_ok && key0 + kWinT <= seq.len && key0 + kWinT - 1 <= pos0 + p.g.right &&
                                  (pos0 + kWinT - 1 <= key0 + p.g.left || key0 + kWinT <= p.g.sinks);
                const float4* lse = reinterpret_cast<const float4*>(sR + ring.stage * C::kRows) + x * 16;
                const float4* del = lse + kWinT / 4;  // (both negated)
                ok = mbar_wait_warp(smem_u32(&bars.q_full[ring.stage]), ring.phase, abortp) && mbar_wait_warp(smem_u32(&bars.s_full), t & 1, abortp);
                if (!ok) break;
                tc_fence_after();
                uint32_t r[64];
                tmem_ld32(t_s, r);
                tmem_ld32(t_s + 32, r + 32);
                tc_wait_ld();
                const uint64_t c22 = pack_f32x2(c2, c2), unshift2 = pack_f32x2(kUnshift<F16>, kUnshift<F16>);
                uint32_t bits[2] = {0xffffffffu, 0xffffffffu};
                if (!full) {
                    bits[0] = view.bits(row0 + x * 64);
                    bits[1] = view.bits(row0 + x * 64 + 32);
                    if (!rows_ok) {  // rows at no position
                        ok = mbar_wait_warp(smem_u32(&bars.o_full[ring.stage]), ring.phase, abortp);
                        if (!ok) break;
                        uint8_t* rows = (x ? sQ : sG) + ring.stage * C::kTile;
                        zero_rows<D, 128>(rows, 0, -pos0, tw);
                        zero_rows<D, 128>(rows, seq.len - pos0, kWinT, tw);
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
                ok = mbar_wait_warp(smem_u32(&bars.dp_full), t & 1, abortp);
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
                        unpack_f32x2(mul_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(d[e]), __uint_as_float(d[e + 1])), unshift2, pack_f32x2(l.x, l.y)),
                                               pack_f32x2(__uint_as_float(r[c * 32 + e]), __uint_as_float(r[c * 32 + e + 1]))), a0, a1);
                        unpack_f32x2(mul_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(d[e + 2]), __uint_as_float(d[e + 3])), unshift2, pack_f32x2(l.z, l.w)),
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
            if (!ok) break;
            if (n > 0) {
                ok = mbar_wait_warp(smem_u32(&bars.acc_full), n_it & 1, abortp);
                if (!ok) break;
                ++n_it;
                tc_fence_after();
            }
            // Warps 0-3 write dV, warps 4-7 dK.
            const uint32_t t_acc = t_lane + (x ? C::kDK : C::kDV);
            if (it.shares > 1) {
                float* out = p.partial + ((((long long)it.bh * p.sink_tiles + it.kt) * it.shares + it.share) * 2 + x) * kWinT * D + tw * D;
#pragma unroll 1
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t o[32];
                    tmem_ld32(t_acc + c * 32, o);
                    tc_wait_ld();
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        uint32_t v[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] = n > 0 ? o[q * 8 + e] : 0u;
                        st_global_v8(out + c * 32 + q * 8, v);
                    }
                }
            } else {
                uint16_t* out = x ? p.dK + (long long)it.b * p.k_batch + (long long)it.hk * p.k_head + (long long)key * p.k_row
                                  : p.dV + (long long)it.b * p.v_batch + (long long)it.hk * p.v_head + (long long)key * p.v_row;
                store_row<F16>(t_acc, 0, D / 32, x ? p.scale : kUnshift<F16>, n == 0, key < p.g.N_kv ? out : nullptr, x ? p.wide_k : p.wide_v);
            }
            if (n > 0) {
                tc_fence_before();
                mbar_arrive(smem_u32(&bars.acc_free));
            }
        }
    }
    end_of_cta(abortp, p.status, (int)BSA_ERR_DEVICE_TIMEOUT);
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
    const float f = which ? p.scale : kUnshift<F16>;
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
    const int64_t tiles = (g.sinks + kWinT - 1) / kWinT, rows = (int64_t)g.batch * g.heads_kv;
    if (tiles > 0 && window * 2 <= l.n_qt) {
        l.sink_tiles = (int)(tiles < l.n_kt ? tiles : l.n_kt);
        const int64_t most = 4 * (int64_t)a.num_sms / (rows * l.sink_tiles);
        int64_t shares = (l.n_qt + window - 1) / window;
        if (shares > most) shares = most;
        l.sink_shares = (int)(shares > 1 ? shares : 1);
        if (l.sink_shares == 1) l.sink_tiles = 0;
    }
    // Where all key tiles together leave most of the GPU idle, every one is cut: into as many shares as fill it, of four query tiles at least
    // (the sum of the shares costs about 5 us, a query tile 1.6).
    const int64_t work = (window < l.n_qt ? window : l.n_qt) * g.group;
    const int64_t fill = a.num_sms / (rows * l.n_kt), each = work / 4;
    if (fill >= 2 && each >= 2) {
        l.sink_tiles = l.n_kt;
        l.sink_shares = (int)(fill < each ? fill : each);
    }
    if (l.sink_tiles == 0) l.sink_shares = 1;
    const int64_t bytes = (int64_t)g.batch * g.heads * l.n_pad * 4;
    l.lse2 = 0;
    l.delta = bytes;
    l.partial = (2 * bytes + 255) / 256 * 256;
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
    const int n_dkv = p.n_shared + p.dkv.n_items;
    dq<<<p.dq.n_items < a.num_sms ? p.dq.n_items : a.num_sms, kThreads, DqCfg<D>::kSmem, stream>>>(tq, tk, tv, tg, p);
    dkv<<<n_dkv < a.num_sms ? n_dkv : a.num_sms, kThreads, DkvCfg<D>::kSmem, stream>>>(tq, tk, tv, tg, p);
    count_launch(3);
    if (l.sink_tiles) {
        window_sink_sum_kernel<D, F16><<<dim3((unsigned)(l.sink_tiles * kWinT * D / 8 / 256), (unsigned)(g.batch * g.heads_kv), 2), 256, 0, stream>>>(p);
        count_launch();
    }
    return cudaGetLastError();
}

}  // namespace
}  // namespace bsa

cudaError_t bsa::set_window_bwd_wait_limit(long long cycles) { return cudaMemcpyToSymbol(ptx::g_wait_limit_cycles, &cycles, sizeof cycles); }

using namespace bsa;

extern "C" int64_t bsa_window_workspace_bytes(const bsa_window_desc_t* t) {
    WindowArgs a;
    return window_args(t, &a) == BSA_OK && window_device(&a) == BSA_OK ? layout_of(a).bytes : 0;
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
    bsa_status_t st = window_args(t, &a);
    if (st == BSA_OK && (view_overlaps(*dQ, t->batch, t->heads, t->N, t->d) || view_overlaps(*dK, t->batch, t->heads_kv, t->N_kv, t->d) ||
                         view_overlaps(*dV, t->batch, t->heads_kv, t->N_kv, t->d)))
        st = BSA_ERR_INVALID_ARG;
    // The kernels read Q, K, V and dO until the last: dQ is finished before K and V are read for dK and dV, and any key tile's dK and dV
    // before another's rows of Q and dO.  (O is read in front of them; a key tile's K and V before its own dK and dV.)
    const auto over = [](const bsa_view_t* x, std::initializer_list<const bsa_view_t*> others) {
        for (const bsa_view_t* y : others)
            if (x->data == y->data) return true;
        return false;
    };
    if (st == BSA_OK && (over(dQ, {Q, K, V, dO, dK, dV}) || over(dK, {Q, dO, dV}) || over(dV, {Q, dO}))) st = BSA_ERR_INVALID_ARG;
    if (st == BSA_OK) st = window_device(&a);
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
    const int cut = cut_tiles(a.g, l.n_qt), own = l.n_kt - l.sink_tiles;
    p.dq = ItemOrder(l.n_qt, cut, a.g.batch * a.g.heads);
    p.dkv = ItemOrder(own, cut < own ? cut : own, a.g.batch * a.g.heads_kv);
    p.n_shared = a.g.batch * a.g.heads_kv * l.sink_tiles * l.sink_shares;
    p.heads = Divisor(a.g.heads);
    p.heads_kv = Divisor(a.g.heads_kv);
    p.group = Divisor(a.g.group);
    p.shares = Divisor(l.sink_shares);
    p.shared = Divisor(l.sink_tiles > 0 ? l.sink_tiles * l.sink_shares : 1);
    p.wide_q = view_is_wide(*dQ, a.g.batch, a.g.heads, a.g.N);
    p.wide_k = view_is_wide(*dK, a.g.batch, a.g.heads_kv, a.g.N_kv);
    p.wide_v = view_is_wide(*dV, a.g.batch, a.g.heads_kv, a.g.N_kv);
    p.sink_tiles = l.sink_tiles;
    p.sink_shares = l.sink_shares;
    p.withhold = window_withhold();
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
