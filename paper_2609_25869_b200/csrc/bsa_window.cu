// Attention over a sliding window and a few first tokens: forward for rows by the tile (prefill, chunks of a stream).
//
//   S = scale Q K^T,  LSE = log sum exp S,  O = sum exp(S - LSE) V   over the keys that a row sees
//
// One CTA takes 256 query rows of one head as two 128-row slots that share every K and V tile of 128 keys: a 128x128x128
// product with both operands in shared memory reads them at the full 128 B/clk, and with one slot per tile the copies of K
// and V would come on top of that; with two they are half as many.  The tiles that a slot needs follow from its rows'
// positions (no list, no mask in memory): a run of tiles around the diagonal and the sinks' tiles; a tile that only one slot
// needs is left out for the other.  Bounds on the columns of a row are applied only in tiles that some row of the slot does
// not see whole.
//   warps 0-3 / 4-7 : softmax of slot 0 / 1 (thread = row)     warps 8-11 : epilogue of both slots
//   warp 12 : TMA producer    warp 13 : MMA issuer (d = 64: Q K^T)    warp 14 : d = 64: P V issuer
// Tensor memory: d = 128: S0, S1, O0, O1 take all 512 columns; P takes the place of the scores that it comes from, and a
// slot's next Q K^T is issued behind its P V (one thread issues both, in order).  While one slot's softmax runs, the other's
// two products do.  P is handed over in halves of 64 keys, so that P V starts while the second half's exponentials run.
// d = 64: P has columns of its own, so a slot's next scores are computed as soon as the last have been read.
// Work per 128-key tile and slot: 4 * 128 * 128 * d flops (1024 clk at d = 128) and 128 * 128 exponentials (1024 clk at 16 per
// clk and SM): the tensor pipe and the special-function unit bind together at d = 128, the latter alone at d = 64.
#include <cuda_bf16.h>
#include <math.h>

#include <atomic>

#include "bsa_window.cuh"

namespace bsa {

using namespace ptx;

namespace {

__device__ int g_window_status = 0;

constexpr int kThreads = 512;
constexpr uint32_t kTmemCols = 512;
constexpr float kRescale = 8.0f;  // log2 units: P stays below 2^8 between rescales
constexpr int kSlotRows = 128, kCtaRows = 256;

template <int D>
struct Cfg {
    static constexpr bool kOwnP = (D == 64);
    static constexpr int kTile = kWinT * D * 2;                 // bytes of a 128-row tile of Q, K or V
    static constexpr int kQBuffers = (D == 64) ? 2 : 1;         // of two slots each
    static constexpr int kStages = (D == 64) ? 8 : 5;           // K and V tiles in turn
    static constexpr int kSmem = (kQBuffers * 2 + kStages) * kTile;
    static constexpr uint32_t kS0 = 0, kS1 = 128, kO0 = 256, kO1 = (D == 64) ? 320 : 384;
    static constexpr uint32_t kP0 = kOwnP ? 384 : kS0, kP1 = kOwnP ? 448 : kS1;
};

struct Params {
    WindowGeom g;
    uint16_t* O;
    long long o_batch, o_head, o_row;
    float* LSE;
    float scale_log2;  // scale * log2(e)
    int n_qt;          // 256-row tiles of a sequence
    int n_items;
    int longest_first; // no left limit: later tiles are longer
};

struct __align__(8) Barriers {
    uint64_t q_full[2], q_empty[2];
    uint64_t kv_full[8], kv_empty[8];
    uint64_t s_full[2], s_free[2], p_half[2][2], pv_done[2];
    uint64_t o_full[2], o_free[2], e_ready[2], e_taken[2];
};

struct Item {
    int b, h, row0;
    Sequence seq;
    KeyRange r0, r1;
    TileSpan t0, t1, both;
};

__device__ __forceinline__ bool load_item(const Params& p, int k, Item& it) {
    const int G = gridDim.x;
    const int idx = k * G + ((k & 1) ? (G - 1 - (int)blockIdx.x) : (int)blockIdx.x);
    if (idx >= p.n_items) return false;
    int bh, qt;
    if (p.longest_first) {
        const int n_bh = p.g.batch * p.g.heads;
        qt = p.n_qt - 1 - idx / n_bh;
        bh = idx % n_bh;
    } else {
        bh = idx / p.n_qt;
        qt = idx % p.n_qt;
    }
    it.b = bh / p.g.heads;
    it.h = bh - it.b * p.g.heads;
    it.row0 = qt * kCtaRows;
    it.seq = load_sequence(p.g, it.b);
    it.r0 = key_range(p.g, it.seq, it.row0, it.row0 + kSlotRows);
    it.r1 = key_range(p.g, it.seq, it.row0 + kSlotRows, it.row0 + kCtaRows);
    it.t0 = tile_span(it.r0);
    it.t1 = tile_span(it.r1);
    it.both = join(it.t0, it.t1);
    return true;
}

template <int R>
__device__ __forceinline__ void reg_inc() {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(R));
}
template <int R>
__device__ __forceinline__ void reg_dec() {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(R));
}

// after a wait gave up: copies in flight land before the CTA's shared memory goes away
__device__ __forceinline__ void let_copies_land() {
    const uint64_t t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 200000ull) __nanosleep(1000);
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

template <int D, bool F16>
__global__ void __launch_bounds__(kThreads, 1)
window_forward_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                      const __grid_constant__ CUtensorMap tmV, const __grid_constant__ Params p) {
    using C = Cfg<D>;
    constexpr int SUB = kWinT * 128;  // bytes of a [128 rows][64 columns] sub-tile
    extern __shared__ __align__(1024) uint8_t smem[];
    uint8_t* sQ = smem;
    uint8_t* sKV = smem + C::kQBuffers * 2 * C::kTile;
    __shared__ Barriers bars;
    __shared__ float fin_m[2][kSlotRows], fin_l[2][kSlotRows];  // an item's reference maxima (log2 domain) and row sums
    __shared__ uint32_t tmem_base_s, abort_flag;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (smem_u32(smem) & 1023u) {  // never expected; fail with a status instead of corrupting tiles
        if (tid == 0) atomicExch(&g_window_status, (int)BSA_ERR_CUDA);
        return;
    }
    if (tid == 0) {
        abort_flag = 0;
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&bars.q_full[i]), 1);
            mbar_init(smem_u32(&bars.q_empty[i]), 1);
            mbar_init(smem_u32(&bars.s_full[i]), 1);
            mbar_init(smem_u32(&bars.s_free[i]), 128);
            mbar_init(smem_u32(&bars.p_half[i][0]), 128);
            mbar_init(smem_u32(&bars.p_half[i][1]), 128);
            mbar_init(smem_u32(&bars.pv_done[i]), 1);
            mbar_init(smem_u32(&bars.o_full[i]), 1);
            mbar_init(smem_u32(&bars.o_free[i]), 128);
            mbar_init(smem_u32(&bars.e_ready[i]), 128);
            mbar_init(smem_u32(&bars.e_taken[i]), 128);
        }
        for (int i = 0; i < C::kStages; ++i) {
            mbar_init(smem_u32(&bars.kv_full[i]), 1);
            mbar_init(smem_u32(&bars.kv_empty[i]), 1);
        }
        fence_mbar_init();
    }
    if (warp == 13) {
        tmem_alloc(smem_u32(&tmem_base_s), kTmemCols);
        tmem_relinquish();
    }
    if (warp == 12 && lane == 0) {
        prefetch_tensormap(&tmQ);
        prefetch_tensormap(&tmK);
        prefetch_tensormap(&tmV);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_base_s;
    volatile uint32_t* abortp = &abort_flag;
    Item it;

    if (warp >= 12) {
        reg_dec<48>();
        if (warp == 12 && lane == 0) {
            // =========================== producer ===========================
            Ring ring;
            uint32_t n_q = 0;
            bool ok = true;
            for (int k = 0; ok && load_item(p, k, it); ++k) {
                const int n = it.both.count();
                if (n == 0) continue;
                const int hk = it.h / p.g.group;
                const uint32_t qb = n_q % C::kQBuffers;
                ok = mbar_wait(smem_u32(&bars.q_empty[qb]), ((n_q / C::kQBuffers) & 1) ^ 1, abortp);
                if (!ok) break;
                const uint32_t q_bar = smem_u32(&bars.q_full[qb]), q_dst = smem_u32(sQ) + qb * 2 * C::kTile;
                const bool s0 = it.t0.w1 > 0, s1 = it.t1.w1 > 0;
                mbar_arrive_expect_tx(q_bar, (int(s0) + int(s1)) * C::kTile);
                if (s0) tma_load_rows(q_dst, &tmQ, q_bar, it.row0, it.h, it.b);
                if (s1) tma_load_rows(q_dst + C::kTile, &tmQ, q_bar, it.row0 + kSlotRows, it.h, it.b);
                ++n_q;
                for (int j = 0; j < n && ok; ++j) {
                    const int key0 = it.both.tile(j) * kWinT;
#pragma unroll
                    for (int kv = 0; kv < 2; ++kv) {
                        ok = ok && mbar_wait(smem_u32(&bars.kv_empty[ring.stage]), ring.phase ^ 1, abortp);
                        if (!ok) break;
                        const uint32_t bar = smem_u32(&bars.kv_full[ring.stage]);
                        mbar_arrive_expect_tx(bar, C::kTile);
                        tma_load_rows(smem_u32(sKV) + ring.stage * C::kTile, kv ? &tmV : &tmK, bar, key0, hk, it.b);
                        ring.advance<C::kStages>();
                    }
                }
            }
            if (!ok) let_copies_land();
        } else if (warp == 13 && lane == 0) {
            // =========================== MMA issuer (d = 64: Q K^T only) ===========================
            constexpr uint32_t idesc_qk = make_idesc_f32(kSlotRows, kWinT, 0, 0, F16);
            constexpr uint32_t idesc_pv = make_idesc_f32(kSlotRows, D, 0, 1, F16);
            const uint64_t descQ = make_smem_desc_sw128(smem_u32(sQ), 16, 1024);
            const uint64_t descK = make_smem_desc_sw128(smem_u32(sKV), 16, 1024);
            const uint64_t descV = make_smem_desc_sw128(smem_u32(sKV), SUB, 1024);
            Ring ring;                 // of the tile being looked at: K, then V
            uint32_t n_q = 0;
            uint32_t n_s[2] = {0, 0};  // score tiles issued
            uint32_t n_p[2] = {0, 0};  // P V issued
            uint32_t n_o[2] = {0, 0};  // accumulators begun
            bool ok = true;
            for (int k = 0; ok && load_item(p, k, it); ++k) {
                const int n = it.both.count();
                if (n == 0) continue;
                const uint32_t qb = n_q % C::kQBuffers;
                ok = mbar_wait(smem_u32(&bars.q_full[qb]), (n_q / C::kQBuffers) & 1, abortp);
                if (!ok) break;
                ++n_q;
                bool pend[2] = {false, false}, first[2] = {true, true};
                int v_stage = 0;
                uint32_t v_phase = 0;
                auto issue_pv = [&](int x, bool last_user, bool last_tile) -> bool {
                    const uint32_t d_o = tmem + (x ? C::kO1 : C::kO0), a_p = tmem + (x ? C::kP1 : C::kP0);
                    if (first[x]) {  // the accumulator has been drained
                        if (!mbar_wait(smem_u32(&bars.o_free[x]), (n_o[x] & 1) ^ 1, abortp)) return false;
                        ++n_o[x];
                    }
                    if (!mbar_wait(smem_u32(&bars.kv_full[v_stage]), v_phase, abortp)) return false;
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        if (!mbar_wait(smem_u32(&bars.p_half[x][half]), n_p[x] & 1, abortp)) return false;
                        tc_fence_after();
#pragma unroll
                        for (int kk = half * 4; kk < half * 4 + 4; ++kk)
                            mma_ts(d_o, a_p + kk * 8, descV + (uint64_t)((v_stage * C::kTile + kk * 2048) >> 4), idesc_pv,
                                   (!first[x] || kk > 0) ? 1u : 0u);
                    }
                    if (last_user) mma_commit(smem_u32(&bars.kv_empty[v_stage]));
                    mma_commit(smem_u32(&bars.pv_done[x]));
                    if (last_tile) mma_commit(smem_u32(&bars.o_full[x]));
                    first[x] = false;
                    ++n_p[x];
                    return true;
                };
                int left_over[2] = {it.t0.count(), it.t1.count()};  // tiles of each slot whose P V is to come
                for (int j = 0; j <= n && ok; ++j) {
                    const int tile = j < n ? it.both.tile(j) : -1;
                    const bool act[2] = {j < n && it.t0.has(tile), j < n && it.t1.has(tile)};
                    const int k_stage = ring.stage;
                    if (j < n) ok = mbar_wait(smem_u32(&bars.kv_full[k_stage]), ring.phase, abortp);
                    if (!ok) break;
                    const bool last_pv1 = pend[1];
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        if (!C::kOwnP && pend[x]) {
                            ok = ok && issue_pv(x, x == 1 || !last_pv1, --left_over[x] == 0);
                            if (!ok) break;
                            pend[x] = false;
                        }
                        if (act[x]) {
                            if (C::kOwnP && n_s[x] > 0) {  // the last scores of this slot have been read
                                ok = mbar_wait(smem_u32(&bars.s_free[x]), (n_s[x] - 1) & 1, abortp);
                                if (!ok) break;
                            }
                            tc_fence_after();
                            const uint64_t q0 = descQ + (uint64_t)(((qb * 2 + x) * C::kTile) >> 4);
                            const uint64_t k0 = descK + (uint64_t)((k_stage * C::kTile) >> 4);
                            const uint32_t d_s = tmem + (x ? C::kS1 : C::kS0);
#pragma unroll
                            for (int kk = 0; kk < D / 16; ++kk) {
                                const uint64_t off = (uint64_t)(((kk / 4) * SUB + (kk % 4) * 32) >> 4);
                                mma_ss(d_s, q0 + off, k0 + off, idesc_qk, kk > 0);
                            }
                            mma_commit(smem_u32(&bars.s_full[x]));
                            ++n_s[x];
                            pend[x] = true;
                        }
                    }
                    if (!ok || j == n) break;
                    mma_commit(smem_u32(&bars.kv_empty[k_stage]));
                    if (j == n - 1) mma_commit(smem_u32(&bars.q_empty[qb]));
                    ring.advance<C::kStages>();
                    v_stage = ring.stage;
                    v_phase = ring.phase;
                    ring.advance<C::kStages>();
                }
            }
        } else if (C::kOwnP && warp == 14 && lane == 0) {
            // =========================== P V issuer (d = 64) ===========================
            constexpr uint32_t idesc_pv = make_idesc_f32(kSlotRows, D, 0, 1, F16);
            const uint64_t descV = make_smem_desc_sw128(smem_u32(sKV), SUB, 1024);
            Ring ring;
            uint32_t n_p[2] = {0, 0}, n_o[2] = {0, 0};
            bool ok = true;
            for (int k = 0; ok && load_item(p, k, it); ++k) {
                const int n = it.both.count();
                bool first[2] = {true, true};
                int left_over[2] = {it.t0.count(), it.t1.count()};
                for (int j = 0; j < n && ok; ++j) {
                    const int tile = it.both.tile(j);
                    const bool act[2] = {it.t0.has(tile), it.t1.has(tile)};
                    ring.advance<C::kStages>();  // past K
                    ok = mbar_wait(smem_u32(&bars.kv_full[ring.stage]), ring.phase, abortp);
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        if (!ok || !act[x]) continue;
                        if (first[x]) {
                            ok = mbar_wait(smem_u32(&bars.o_free[x]), (n_o[x] & 1) ^ 1, abortp);
                            if (!ok) break;
                            ++n_o[x];
                        }
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            ok = ok && mbar_wait(smem_u32(&bars.p_half[x][half]), n_p[x] & 1, abortp);
                            if (!ok) break;
                            tc_fence_after();
#pragma unroll
                            for (int kk = half * 4; kk < half * 4 + 4; ++kk)
                                mma_ts(tmem + (x ? C::kO1 : C::kO0), tmem + (x ? C::kP1 : C::kP0) + kk * 8,
                                       descV + (uint64_t)((ring.stage * C::kTile + kk * 2048) >> 4), idesc_pv, (!first[x] || kk > 0) ? 1u : 0u);
                        }
                        if (!ok) break;
                        mma_commit(smem_u32(&bars.pv_done[x]));
                        if (--left_over[x] == 0) mma_commit(smem_u32(&bars.o_full[x]));
                        first[x] = false;
                        ++n_p[x];
                    }
                    if (!ok) break;
                    mma_commit(smem_u32(&bars.kv_empty[ring.stage]));
                    ring.advance<C::kStages>();
                }
            }
        }
    } else if (warp >= 8) {
        // =========================== epilogue ===========================
        reg_dec<80>();
        const int tw = tid & 127;
        const uint32_t t_lane = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        uint32_t n_e[2] = {0, 0};
        bool ok = true;
        for (int k = 0; ok && load_item(p, k, it); ++k) {
#pragma unroll 1
            for (int x = 0; x < 2 && ok; ++x) {
                const int row = it.row0 + x * kSlotRows + tw;
                const bool row_ok = row < p.g.N;
                const int pos = it.seq.start + row;
                const bool seen = pos >= 0 && pos < it.seq.len;
                uint16_t* orow = p.O + (long long)it.b * p.o_batch + (long long)it.h * p.o_head + (long long)row * p.o_row;
                float* lse_out = p.LSE + ((long long)it.b * p.g.heads + it.h) * p.g.N + row;
                if ((x ? it.t1.w1 : it.t0.w1) == 0) {  // no row of the slot sees anything
                    if (row_ok) {
#pragma unroll
                        for (int c = 0; c < D / 8; ++c) reinterpret_cast<uint4*>(orow)[c] = make_uint4(0, 0, 0, 0);
                        *lse_out = -INFINITY;
                    }
                    continue;
                }
                ok = mbar_wait_warp(smem_u32(&bars.e_ready[x]), n_e[x] & 1, abortp);
                if (!ok) break;
                const float l = fin_l[x][tw], m = fin_m[x][tw];
                mbar_arrive(smem_u32(&bars.e_taken[x]));
                const bool any = seen && l > 0.f;
                const float inv = any ? 1.f / l : 0.f;
                if (row_ok) *lse_out = any ? fmaf(m, 0.6931471805599453f, logf(l)) : -INFINITY;
                ok = mbar_wait_warp(smem_u32(&bars.o_full[x]), n_e[x] & 1, abortp);
                if (!ok) break;
                ++n_e[x];
                tc_fence_after();
#pragma unroll 1
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t o[32];
                    tmem_ld32(t_lane + (x ? C::kO1 : C::kO0) + c * 32, o);
                    tc_wait_ld();
                    if (c == D / 32 - 1) {
                        tc_fence_before();
                        mbar_arrive(smem_u32(&bars.o_free[x]));
                    }
                    if (row_ok) {
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            uint32_t v[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float a = __uint_as_float(o[q * 8 + 2 * e]) * inv, b = __uint_as_float(o[q * 8 + 2 * e + 1]) * inv;
                                v[e] = seen ? pack_16x2<F16>(a, b) : 0u;
                            }
                            *reinterpret_cast<uint4*>(orow + c * 32 + q * 8) = make_uint4(v[0], v[1], v[2], v[3]);
                        }
                    }
                }
            }
        }
    } else {
        // =========================== softmax of slot x ===========================
        reg_inc<192>();
        const int x = warp >> 2, tw = tid & 127;
        const uint32_t t_lane = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t t_s = t_lane + (x ? C::kS1 : C::kS0), t_p = t_lane + (x ? C::kP1 : C::kP0), t_o = t_lane + (x ? C::kO1 : C::kO0);
        const float c2 = p.scale_log2;
        uint32_t n_s = 0, n_e = 0;
        Ring ring;
        bool ok = true;
        for (int k = 0; ok && load_item(p, k, it); ++k) {
            const int n = it.both.count();
            const TileSpan own = x ? it.t1 : it.t0;
            const KeyRange rng = x ? it.r1 : it.r0;
            if (own.w1 == 0) {
                for (int j = 0; j < n; ++j) {
                    ring.advance<C::kStages>();
                    ring.advance<C::kStages>();
                }
                continue;
            }
            const int pos = it.seq.start + it.row0 + x * kSlotRows + tw;
            // keys that some row of the CTA sees: all others may hold anything
            const int any_lo = it.t0.w1 == 0 ? it.r1.lo : it.t1.w1 == 0 ? it.r0.lo : min(it.r0.lo, it.r1.lo);
            const int any_hi = max(it.r0.hi, it.r1.hi);
            float m_ref = -INFINITY, l = 0.f;
            bool first = true;
            for (int j = 0; j < n; ++j) {
                const int tile = it.both.tile(j), key0 = tile * kWinT;
                ring.advance<C::kStages>();  // past K
                const int v_stage = ring.stage;
                const uint32_t v_phase = ring.phase;
                ring.advance<C::kStages>();
                if (!own.has(tile)) continue;
                const bool full = tile_is_full(p.g, rng, key0);
                ok = mbar_wait_warp(smem_u32(&bars.s_full[x]), n_s & 1, abortp);
                if (!ok) break;
                tc_fence_after();
                uint32_t r[kWinT];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32(t_s + c * 32, &r[c * 32]);
                tc_wait_ld();
                if constexpr (C::kOwnP) {
                    tc_fence_before();
                    mbar_arrive(smem_u32(&bars.s_free[x]));
                }
                if (!full) {
                    const RowMask mk = row_mask(p.g, it.seq, pos, key0);
#pragma unroll
                    for (int i = 0; i < kWinT; ++i)
                        r[i] = (i < mk.hi && (i >= mk.lo || i < mk.sink)) ? r[i] : 0xff800000u;  // -inf
                    // V rows that nobody sees: their weight is zero, which times NaN would not be
                    const int from = any_hi - key0, below = any_lo - key0;
                    if (from < kWinT || (below > 0 && p.g.sinks - key0 < below)) {
                        ok = mbar_wait_warp(smem_u32(&bars.kv_full[v_stage]), v_phase, abortp);
                        if (!ok) break;
                        if (tw >= from || (tw < below && key0 + tw >= p.g.sinks)) {
                            uint4* v = reinterpret_cast<uint4*>(sKV + v_stage * C::kTile + tw * 128);
#pragma unroll
                            for (int s = 0; s < D / 64; ++s)
#pragma unroll
                                for (int c = 0; c < 8; ++c) v[s * (SUB / 16) + c] = make_uint4(0, 0, 0, 0);
                        }
                        fence_proxy_async_smem();
                    }
                }
                float m0 = -INFINITY, m1 = m0, m2 = m0, m3 = m0;
#pragma unroll
                for (int i = 0; i < kWinT; i += 8) {
                    m0 = max3(m0, __uint_as_float(r[i]), __uint_as_float(r[i + 1]));
                    m1 = max3(m1, __uint_as_float(r[i + 2]), __uint_as_float(r[i + 3]));
                    m2 = max3(m2, __uint_as_float(r[i + 4]), __uint_as_float(r[i + 5]));
                    m3 = max3(m3, __uint_as_float(r[i + 6]), __uint_as_float(r[i + 7]));
                }
                const float mx = fmaxf(fmaxf(m0, m1), fmaxf(m2, m3)) * c2;
                float alpha = 1.f;
                bool moved = false;
                if (mx > m_ref + kRescale) {
                    alpha = ex2_approx(m_ref - mx);  // m_ref = -inf: 0
                    moved = m_ref != -INFINITY;
                    m_ref = mx;
                }
                if (!first && __any_sync(0xffffffffu, moved)) {  // the accumulator follows the new reference
                    ok = mbar_wait_warp(smem_u32(&bars.pv_done[x]), (n_s - 1) & 1, abortp);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll 1
                    for (int c = 0; c < D / 16; ++c) {
                        uint32_t o[16];
                        tmem_ld16(t_o + c * 16, o);
                        tc_wait_ld();
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
                        tmem_st16(t_o + c * 16, o);
                    }
                }
                first = false;
                const float neg_m = (m_ref == -INFINITY) ? 0.f : -m_ref;
                const uint64_t c22 = pack_f32x2(c2, c2), nm2 = pack_f32x2(neg_m, neg_m);
                uint64_t sum01 = pack_f32x2(0.f, 0.f), sum23 = sum01;
                if constexpr (C::kOwnP) {  // the last P of this slot has been read
                    if (n_s > 0) ok = mbar_wait_warp(smem_u32(&bars.pv_done[x]), (n_s - 1) & 1, abortp);
                    if (!ok) break;
                    tc_fence_after();
                }
#pragma unroll
                for (int half = 0; half < 2; ++half) {
#pragma unroll
                    for (int i = half * 64; i < half * 64 + 64; i += 4) {
                        float x0, x1, x2, x3;
                        unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(r[i]), __uint_as_float(r[i + 1])), c22, nm2), x0, x1);
                        unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(r[i + 2]), __uint_as_float(r[i + 3])), c22, nm2), x2, x3);
                        const float p0 = ex2_approx(x0), p1 = ex2_approx(x1), p2 = ex2_approx(x2), p3 = ex2_approx(x3);
                        sum01 = add_f32x2(sum01, pack_f32x2(p0, p1));
                        sum23 = add_f32x2(sum23, pack_f32x2(p2, p3));
                        r[i / 2] = pack_16x2<F16>(p0, p1);
                        r[i / 2 + 1] = pack_16x2<F16>(p2, p3);
                    }
                    tmem_st32(t_p + half * 32, &r[half * 32]);
                    tc_wait_st();
                    tc_fence_before();
                    mbar_arrive(smem_u32(&bars.p_half[x][half]));
                }
                float s0, s1, s2, s3;
                unpack_f32x2(sum01, s0, s1);
                unpack_f32x2(sum23, s2, s3);
                l = l * alpha + ((s0 + s1) + (s2 + s3));
                ++n_s;
            }
            if (!ok) break;
            ok = mbar_wait_warp(smem_u32(&bars.e_taken[x]), (n_e & 1) ^ 1, abortp);
            if (!ok) break;
            fin_m[x][tw] = m_ref;
            fin_l[x][tw] = l;
            mbar_arrive(smem_u32(&bars.e_ready[x]));
            ++n_e;
        }
    }

    tc_fence_before();
    __syncthreads();
    if (tid == 0 && abort_flag) atomicExch(&g_window_status, (int)BSA_ERR_DEVICE_TIMEOUT);
    if (warp == 13) tmem_dealloc(tmem, kTmemCols);
}

template <int D, bool F16>
cudaError_t launch_rows(const WindowArgs& a, const bsa_view_t& Q, const bsa_view_t& K, const bsa_view_t& V, Params p, cudaStream_t stream) {
    CUtensorMap tq, tk, tv;
    if (!encode_view_map(&tq, Q, a.g.N, a.g.heads, a.g.batch, D, kSlotRows, F16) ||
        !encode_view_map(&tk, K, a.g.N_kv, a.g.heads_kv, a.g.batch, D, kWinT, F16) ||
        !encode_view_map(&tv, V, a.g.N_kv, a.g.heads_kv, a.g.batch, D, kWinT, F16))
        return cudaErrorInvalidValue;
    const auto kernel = window_forward_kernel<D, F16>;
    static std::atomic<bool> allowed[kMaxDevices];  // the attribute belongs to the device's copy of the kernel
    if (!allowed[a.device].load(std::memory_order_relaxed)) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<D>::kSmem);
        if (e != cudaSuccess) return e;
        allowed[a.device].store(true, std::memory_order_relaxed);
    }
    const int grid = a.num_sms < p.n_items ? a.num_sms : p.n_items;
    kernel<<<grid, kThreads, Cfg<D>::kSmem, stream>>>(tq, tk, tv, p);
    count_launch();
    return cudaGetLastError();
}

}  // namespace

cudaError_t window_status_word(int** out) { return cudaGetSymbolAddress(reinterpret_cast<void**>(out), g_window_status); }

bsa_status_t window_args(const bsa_window_desc_t* t, WindowArgs* a) {
    if (!t || t->batch < 1 || t->heads < 1 || t->heads_kv < 1 || t->N < 1 || t->N_kv < 1 || t->heads % t->heads_kv) return BSA_ERR_INVALID_ARG;
    if (t->left < -1 || t->right < -1 || t->sinks < 0 || (t->dtype != BSA_DTYPE_BF16 && t->dtype != BSA_DTYPE_FP16)) return BSA_ERR_INVALID_ARG;
    if (!(t->scale >= 0.f) || !isfinite(t->scale)) return BSA_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(t->q_start_dev) & 3) || (reinterpret_cast<uintptr_t>(t->kv_len_dev) & 3)) return BSA_ERR_INVALID_ARG;
    if (t->d != 64 && t->d != 128) return BSA_ERR_UNSUPPORTED;
    if (t->N > kWinNoLimit || t->N_kv > kWinNoLimit || (int64_t)t->batch * t->heads > 65535) return BSA_ERR_UNSUPPORTED;
    const auto limit = [](int64_t v) { return v < 0 || v > kWinNoLimit ? kWinNoLimit : (int)v; };
    a->g = WindowGeom{t->batch, t->heads, t->heads_kv, t->heads / t->heads_kv, (int)t->N, (int)t->N_kv,
                      limit(t->left), limit(t->right), t->sinks > kWinNoLimit ? kWinNoLimit : (int)t->sinks, t->q_start_dev, t->kv_len_dev};
    a->d = t->d;
    a->f16 = t->dtype == BSA_DTYPE_FP16;
    a->scale = t->scale > 0.f ? t->scale : 1.f / sqrtf((float)t->d);
    static std::atomic<int> sms[kMaxDevices];
    cudaError_t e = cudaGetDevice(&a->device);
    if (e == cudaSuccess && a->device >= kMaxDevices) return BSA_ERR_CUDA;
    if (e == cudaSuccess && (a->num_sms = sms[a->device].load(std::memory_order_relaxed)) == 0) {
        e = cudaDeviceGetAttribute(&a->num_sms, cudaDevAttrMultiProcessorCount, a->device);
        if (e == cudaSuccess) sms[a->device].store(a->num_sms, std::memory_order_relaxed);
    }
    if (e != cudaSuccess) {
        set_cuda_err(e, "device");
        return BSA_ERR_CUDA;
    }
    return BSA_OK;
}

}  // namespace bsa

using namespace bsa;

extern "C" bsa_status_t bsa_window_forward(const bsa_window_desc_t* t, const bsa_view_t* Q, const bsa_view_t* K,
                                           const bsa_view_t* V, const bsa_view_t* O, float* LSE, void* stream_v) {
    if (!t || !LSE || (reinterpret_cast<uintptr_t>(LSE) & 3)) return BSA_ERR_INVALID_ARG;
    if (!view_ok(Q, t->batch, t->heads, t->N) || !view_ok(O, t->batch, t->heads, t->N) ||
        !view_ok(K, t->batch, t->heads_kv, t->N_kv) || !view_ok(V, t->batch, t->heads_kv, t->N_kv))
        return BSA_ERR_INVALID_ARG;
    WindowArgs a;
    const bsa_status_t st = window_args(t, &a);
    if (st != BSA_OK) return st;
    Params p = {};
    p.g = a.g;
    p.O = static_cast<uint16_t*>(O->data);
    p.o_batch = O->batch; p.o_head = O->head; p.o_row = O->row;
    p.LSE = LSE;
    p.scale_log2 = a.scale * 1.4426950408889634f;
    p.n_qt = (a.g.N + kCtaRows - 1) / kCtaRows;
    const int64_t items = (int64_t)p.n_qt * a.g.batch * a.g.heads;
    if (items > INT_MAX / 2) return BSA_ERR_UNSUPPORTED;
    p.n_items = (int)items;
    p.longest_first = a.g.left >= a.g.N_kv;
    const cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_v);
    const cudaError_t e = a.d == 64 ? (a.f16 ? launch_rows<64, true>(a, *Q, *K, *V, p, stream) : launch_rows<64, false>(a, *Q, *K, *V, p, stream))
                                    : (a.f16 ? launch_rows<128, true>(a, *Q, *K, *V, p, stream) : launch_rows<128, false>(a, *Q, *K, *V, p, stream));
    if (e != cudaSuccess) {
        set_cuda_err(e, "bsa_window_forward");
        return BSA_ERR_CUDA;
    }
    return BSA_OK;
}

extern "C" bsa_status_t bsa_window_status(int* status_out) {
    if (!status_out) return BSA_ERR_INVALID_ARG;
    int* word = nullptr;
    int v = 0;
    cudaError_t e = window_status_word(&word);
    if (e == cudaSuccess) e = cudaMemcpy(&v, word, sizeof v, cudaMemcpyDeviceToHost);
    if (e == cudaSuccess && v != 0) e = cudaMemset(word, 0, sizeof v);
    if (e != cudaSuccess) {
        set_cuda_err(e, "bsa_window_status");
        return BSA_ERR_CUDA;
    }
    *status_out = v;
    return BSA_OK;
}
