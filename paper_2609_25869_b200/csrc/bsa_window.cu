// Attention over a sliding window and a few first tokens: forward for rows by the tile (prefill, chunks of a stream).
//
//   S = scale Q K^T,  LSE = log sum exp S,  O = sum exp(S - LSE) V   over the keys that a row sees
//
// A persistent CTA takes 128 query rows of one head at a time and walks over the 128-key tiles that they see: a run of tiles
// around the diagonal and the sinks' tiles, computed from the rows' positions (no list, no mask in memory).  Bounds on a
// row's columns are applied only in tiles that some row does not see whole.
//   warps 0-3 / 4-7 : softmax warpgroups (thread = row); tile t belongs to warpgroup t mod 2, and S and P buffer t mod 2 with it
//   warp 8 : Q and K producer   warp 9 : Q K^T issuer   warp 10 : P V issuer   warp 11 : V producer
//   warps 12-15 : references: each row's running maximum, the tiles' edges, the accumulator's rescaling, and the epilogue
// Work per tile: 4 * 128 * 128 * d flops (1024 clk at d = 128) and 128 * 128 exponentials (1024 clk at 16 per clk and SM): at
// d = 128 the tensor pipe and the special-function unit bind together, at d = 64 the latter alone.  A warpgroup takes longer
// than that over a tile (latencies), so two must run at once and neither may wait: S and P have their own columns, Q K^T runs
// two tiles ahead, and the maxima are found by a third warpgroup while the tile in front is still in the softmax.  That also
// makes one reference maximum per row for both warpgroups, and one accumulator.
// On one GPU, 25088 keys for 4736 rows, bf16, d = 128, 12 heads: 256 rows per CTA, a slot of 128 per warpgroup with P in the place of S (so
// that a slot's softmax, P V and Q K^T follow each other) 900 TFLOP/s; 128 rows, warpgroups finding the maxima themselves 1100; this form
// 1280 (4 heads, where the power cap takes less: 1380), d = 64 760.  The tensor pipe and the special-function unit are 69 % busy each
// (16384 rows, 8 heads, causal window 4096).  Short windows pay per item: edge tiles take the reference warpgroup 1400 clk instead of 550, an
// item's end 2000.
// Tensor-memory columns: S0 0, S1 128, O 256, P0 384, P1 448.  Registers (setmaxnreg): 256 * 184 + 128 * 96 + 128 * 48 = 65536, the
// launch's 512 * 128.
#include <cuda_bf16.h>
#include <math.h>

#include <atomic>
#include <mutex>

#include "bsa_window.cuh"

namespace bsa {

using namespace ptx;

namespace {

__device__ int g_window_status = 0;
__device__ int g_window_taken = 0;
// Read and cleared in one step: what a call of another thread sets meanwhile is left for the next look.
__global__ void take_window_status() { g_window_taken = atomicExch(&g_window_status, 0); }

constexpr int kThreads = 512;
constexpr uint32_t kTmemCols = 512;
constexpr float kRescale = 8.0f;  // log2 units: P stays below 2^8 between rescales
// Half: P is computed 2^7 times as large, up to 2^15 (half ends at 2^16).  A row's largest weight is at least its reference's, so what
// half loses below 2^-14 of P is below 2^-21 of it.
template <bool F16>
constexpr float kShift = F16 ? 7.0f : 0.0f;

template <int D>
struct Cfg {
    static constexpr int kTile = kWinT * D * 2;           // bytes of a 128-row tile of Q, K or V
    static constexpr int kK = (D == 64) ? 4 : 2, kV = (D == 64) ? 4 : 3;  // tiles in the rings
    static constexpr int kSmem = (2 + kK + kV) * kTile;   // two Q tiles
    static constexpr uint32_t kS0 = 0, kS1 = 128, kO = 256, kP0 = 384, kP1 = 448;
};

struct Params {
    WindowGeom g;
    uint16_t* O;
    long long o_batch, o_head, o_row;
    float* LSE;
    int o_wide;        // rows of O lie on 32-byte boundaries
    float scale_log2;  // scale * log2(e)
    int withhold;      // test hook: no copy of the first tile of V
    ItemOrder order;       // 128-row tiles, from a sequence's last to its first
    Divisor heads, group;  // heads; heads that share a key head
};

struct __align__(8) Barriers {
    uint64_t q_full[2], q_empty[2];
    uint64_t k_full[4], k_empty[4], v_full[4], v_empty[4], v_land[4];
    uint64_t s_full[2], s_free[2], ref_ready[2], p_ready[2];
    uint64_t pv_done[8];  // tile t: t mod 8 (see the reference warpgroup)
    uint64_t o_full, o_free, e_ready, e_taken;
};

struct Item {
    int b, h, hk, row0;
    Sequence seq;
    KeyRange range;
    TileSpan tiles;
};

// The CTA's k-th item, dealt in alternating directions; false past the end.
__device__ __forceinline__ bool load_item(const Params& p, int k, Item& it) {
    const int G = gridDim.x;
    const int idx = k * G + ((k & 1) ? (G - 1 - (int)blockIdx.x) : (int)blockIdx.x);
    if (idx >= p.order.n_items) return false;
    int tile, rest;
    const int bh = p.order.row_of(idx, tile), qt = p.order.n_tiles - 1 - tile;
    it.b = p.heads.div(bh, it.h);
    it.hk = p.group.div(it.h, rest);
    it.row0 = qt * kWinT;
    it.seq = load_sequence(p.g, it.b);
    it.range = key_range(p.g, it.seq, it.row0, it.row0 + kWinT);
    it.tiles = tile_span(it.range);
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

// P of 32 keys in the place of their scores: exp2(s * c2 + neg_m), rounded and packed by pairs; its unrounded sum.
template <bool F16>
__device__ __forceinline__ void exp_keys(uint32_t* r, uint64_t c22, uint64_t neg_m2, uint64_t& sum01, uint64_t& sum23) {
#pragma unroll
    for (int i = 0; i < 32; i += 4) {
        float x0, x1, x2, x3;
        unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(r[i]), __uint_as_float(r[i + 1])), c22, neg_m2), x0, x1);
        unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(r[i + 2]), __uint_as_float(r[i + 3])), c22, neg_m2), x2, x3);
        const float p0 = ex2_approx(x0), p1 = ex2_approx(x1), p2 = ex2_approx(x2), p3 = ex2_approx(x3);
        sum01 = add_f32x2(sum01, pack_f32x2(p0, p1));
        sum23 = add_f32x2(sum23, pack_f32x2(p2, p3));
        r[i / 2] = pack_16x2<F16>(p0, p1);
        r[i / 2 + 1] = pack_16x2<F16>(p2, p3);
    }
}

template <int D, bool F16>
__global__ void __launch_bounds__(kThreads, 1)
window_forward_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                      const __grid_constant__ CUtensorMap tmV, const __grid_constant__ Params p) {
    using C = Cfg<D>;
    constexpr int SUB = kWinT * 128;  // bytes of a [128 rows][64 columns] sub-tile
    extern __shared__ __align__(1024) uint8_t smem[];
    uint8_t* sQ = smem;
    uint8_t* sK = sQ + 2 * C::kTile;
    uint8_t* sV = sK + C::kK * C::kTile;
    __shared__ Barriers bars;
    __shared__ float mref[2][kWinT];               // [tile mod 2][row]: the tile's reference maximum (log2 domain)
    __shared__ float lfin[2][kWinT];  // [warpgroup][row]: an item's row sums, each in the reference of the warpgroup's last tile,
    __shared__ float mfin[kWinT];     // which is here for the warpgroup that did not have the item's last one
    __shared__ uint32_t tmem_base_s, abort_flag;

    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
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
            mbar_init(smem_u32(&bars.ref_ready[i]), 128);
            mbar_init(smem_u32(&bars.p_ready[i]), 128);
        }
        for (int i = 0; i < 4; ++i) {
            mbar_init(smem_u32(&bars.k_full[i]), 1);
            mbar_init(smem_u32(&bars.k_empty[i]), 1);
            mbar_init(smem_u32(&bars.v_full[i]), 1);
            mbar_init(smem_u32(&bars.v_empty[i]), 1);
            mbar_init(smem_u32(&bars.v_land[i]), 1);
        }
        for (int i = 0; i < 8; ++i) mbar_init(smem_u32(&bars.pv_done[i]), 1);
        mbar_init(smem_u32(&bars.o_full), 1);
        mbar_init(smem_u32(&bars.o_free), 128);
        mbar_init(smem_u32(&bars.e_ready), 256);
        mbar_init(smem_u32(&bars.e_taken), 128);
        fence_mbar_init();
    }
    if (warp == 9) {
        tmem_alloc(smem_u32(&tmem_base_s), kTmemCols);
        tmem_relinquish();
    }
    if (warp == 8 && lane == 0) {
        prefetch_tensormap(&tmQ);
        prefetch_tensormap(&tmK);
        prefetch_tensormap(&tmV);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_base_s, 0);
    volatile uint32_t* abortp = &abort_flag;
    grid_dependency_wait();  // (where a kernel in front writes K, V, starts and lengths)
    Item it;

    if (warp >= 12) {
        // =========================== references and epilogue ===========================
        reg_dec<96>();
        const int tw = tid & 127;
        const uint32_t t_lane = tmem + ((uint32_t)((warp & 3) * 32) << 16), t_o = t_lane + C::kO;
        const float c2 = p.scale_log2;
        uint32_t n_it = 0, g = 0;  // items finished (with tiles), tiles in front of the item
        // The reference of tile j of an item (running index t) follows from `m`, that of the tile before, and its scores.  Where rows do
        // not see the whole tile, this warpgroup writes the scores back with the hidden ones at -inf: the softmax warpgroups, whose loop is
        // the kernel's bottleneck, have no edges.  Returns whether any row of the warp has moved to a new reference (m_old: the one before).
        auto find = [&](const Item& w, int j, uint32_t t, float& m, float& m_old, bool& moved) -> bool {
            const uint32_t t_s = t_lane + ((t & 1) ? C::kS1 : C::kS0);
            const int key0 = w.tiles.tile(j) * kWinT;
            const bool full = tile_is_full(p.g, w.range, key0);
            if (!mbar_wait_warp(smem_u32(&bars.s_full[t & 1]), (t >> 1) & 1, abortp)) return false;
            tc_fence_after();
            float m0 = -INFINITY, m1 = m0, m2 = m0, m3 = m0;
            auto take = [&](const uint32_t* r) {  // the maximum of 32 scores
#pragma unroll
                for (int i = 0; i < 32; i += 8) {
                    m0 = max3(m0, __uint_as_float(r[i]), __uint_as_float(r[i + 1]));
                    m1 = max3(m1, __uint_as_float(r[i + 2]), __uint_as_float(r[i + 3]));
                    m2 = max3(m2, __uint_as_float(r[i + 4]), __uint_as_float(r[i + 5]));
                    m3 = max3(m3, __uint_as_float(r[i + 6]), __uint_as_float(r[i + 7]));
                }
            };
            if (full) {
#pragma unroll 1
                for (int c = 0; c < kWinT; c += 64) {  // (this way lies on every tile's path: two waits, no votes)
                    uint32_t r[64];
                    tmem_ld32(t_s + c, r);
                    tmem_ld32(t_s + c + 32, r + 32);
                    tc_wait_ld();
                    take(r);
                    take(r + 32);
                }
            } else {
                const RowView view(p.g, w.seq, w.seq.start + w.row0 + tw, key0);
#pragma unroll 1
                for (int c = 0; c < kWinT; c += 32) {
                    const uint32_t bits = view.bits(c);
                    uint32_t r[32];
                    if (!__any_sync(0xffffffffu, bits)) {  // (of an edge tile's four pieces a warp mostly has one that is hidden in part)
#pragma unroll
                        for (int i = 0; i < 32; ++i) r[i] = 0xff800000u;
                        tmem_st32(t_s + c, r);
                        continue;
                    }
                    tmem_ld32(t_s + c, r);
                    tc_wait_ld();
                    if (!__all_sync(0xffffffffu, bits == 0xffffffffu)) {
                        hide(r, bits);
                        tmem_st32(t_s + c, r);
                    }
                    take(r);
                }
                tc_wait_st();
            }
            const float mx = fmaxf(fmaxf(m0, m1), fmaxf(m2, m3)) * c2;
            m_old = m;
            if (mx > m + kRescale) m = mx;
            moved = j > 0 && __any_sync(0xffffffffu, m != m_old && m_old != -INFINITY);
            return true;
        };
        auto publish = [&](uint32_t t, float m, float m_old, bool moved) -> bool {
            // The accumulator follows, once all products before are in it.  This wait comes now and then, and a barrier's parity tells whether
            // its last phase but one or its last is over, no more: the barrier's phase before the one waited for has to be over for sure.
            // That is P V of tile t - 9: the scores of t are there, so those of t - 2 and t - 3 have been read, so the warpgroups are
            // done with t - 4 and t - 5, for which they waited until P V of t - 6 and t - 7 was over.
            if (moved) {
                if (!mbar_wait_warp(smem_u32(&bars.pv_done[(t - 1) & 7]), ((t - 1) >> 3) & 1, abortp)) return false;
                tc_fence_after();
                const float alpha = (m != m_old && m_old != -INFINITY) ? ex2_approx(m_old - m) : 1.f;
#pragma unroll 1
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t o[32];
                    tmem_ld32(t_o + c * 32, o);
                    tc_wait_ld();
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
                    tmem_st32(t_o + c * 32, o);
                }
                tc_wait_st();
            }
            mref[t & 1][tw] = m;
            tc_fence_before();
            mbar_arrive(smem_u32(&bars.ref_ready[t & 1]));
            return true;
        };
        bool more = load_item(p, 0, it), ok = true;
        int done = 0;  // of this item's tiles: references that are out
        float m = -INFINITY;
        for (int k = 0; more; ++k) {
            const Item w = it;
            const int row = w.row0 + tw;
            const bool row_ok = row < p.g.N;
            const int pos = w.seq.start + row;
            const bool seen = pos >= 0 && pos < w.seq.len;
            uint16_t* orow = p.O + (long long)w.b * p.o_batch + (long long)w.h * p.o_head + (long long)row * p.o_row;
            float* lse_out = p.LSE + ((long long)w.b * p.g.heads + w.h) * p.g.N + row;
            const int n = w.tiles.count();
            float m_old;
            bool moved;
            for (int j = done; ok && j < n; ++j) ok = find(w, j, g + j, m, m_old, moved) && publish(g + j, m, m_old, moved);
            if (!ok) break;
            g += (uint32_t)n;
            more = load_item(p, k + 1, it);
            done = 0;
            if (n == 0) {  // no row of the tile sees anything
                if (row_ok) {
#pragma unroll
                    for (int c = 0; c < D / 8; ++c) reinterpret_cast<uint4*>(orow)[c] = make_uint4(0, 0, 0, 0);
                    *lse_out = -INFINITY;
                }
                m = -INFINITY;
                continue;
            }
            // The next item's first two tiles come before this item's end, so that both warpgroups have work until the accumulator is
            // drained; the second one's reference waits until then where it moves the accumulator.
            const int n_next = more ? it.tiles.count() : 0;
            float m_next = -INFINITY;
            bool held = false;
            if (n_next > 0) {
                ok = find(it, 0, g, m_next, m_old, moved) && publish(g, m_next, m_old, moved);
                done = 1;
                if (ok && n_next > 1) {
                    ok = find(it, 1, g + 1, m_next, m_old, moved);
                    held = moved;
                    if (ok && !held) ok = publish(g + 1, m_next, m_old, false);
                    done = 2;
                }
                if (!ok) break;
            }
            if (!mbar_wait_warp(smem_u32(&bars.e_ready), n_it & 1, abortp)) break;
            // (g is the next item's first tile, of the warpgroup that did not have this one's last; -inf where it had none: its sum is zero)
            const float m_other = mfin[tw], l_other = lfin[g & 1][tw];
            const float l = lfin[(g & 1) ^ 1][tw] + (m_other == m ? l_other : l_other * ex2_approx(m_other - m));
            mbar_arrive(smem_u32(&bars.e_taken));
            // (a row at a position sees its own key at least: its sum is above zero, or NaN, which belongs to its outputs)
            const float inv = seen ? 1.f / l : 0.f;
            if (row_ok) *lse_out = seen ? fmaf(m - kShift<F16>, 0.6931471805599453f, logf(l)) : -INFINITY;
            m = m_next;
            if (!mbar_wait_warp(smem_u32(&bars.o_full), n_it & 1, abortp)) break;
            ++n_it;
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < D / 32; ++c) {
                uint32_t o[32];
                tmem_ld32(t_o + c * 32, o);
                tc_wait_ld();
                if (c == D / 32 - 1) {  // drained: the next item's first P V may overwrite it
                    tc_fence_before();
                    mbar_arrive(smem_u32(&bars.o_free));
                }
                if (row_ok) {
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        uint32_t v[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            v[e] = seen ? pack_16x2<F16>(__uint_as_float(o[q * 16 + 2 * e]) * inv, __uint_as_float(o[q * 16 + 2 * e + 1]) * inv) : 0u;
                        st_global_v8_or_2v4(orow + c * 32 + q * 16, v, p.o_wide);
                    }
                }
                __syncwarp();
            }
            if (held && !publish(g + 1, m, m_old, true)) break;
        }
    } else if (warp >= 8) {
        reg_dec<48>();
        if (warp == 8 && lane == 0) {
            // =========================== Q and K producer ===========================
            Ring ring;
            uint32_t n_q = 0;
            bool ok = true;
            for (int k = 0; ok && load_item(p, k, it); ++k) {
                const int n = it.tiles.count(), hk = it.hk;
                if (n == 0) continue;
                const uint32_t qb = n_q & 1;
                ok = mbar_wait(smem_u32(&bars.q_empty[qb]), ((n_q >> 1) & 1) ^ 1, abortp);
                if (!ok) break;
                mbar_arrive_expect_tx(smem_u32(&bars.q_full[qb]), C::kTile);
                tma_load_rows(smem_u32(sQ) + qb * C::kTile, &tmQ, smem_u32(&bars.q_full[qb]), it.row0, it.h, it.b);
                ++n_q;
                for (int j = 0; j < n; ++j, ring.advance<C::kK>()) {
                    ok = mbar_wait(smem_u32(&bars.k_empty[ring.stage]), ring.phase ^ 1, abortp);
                    if (!ok) break;
                    const uint32_t bar = smem_u32(&bars.k_full[ring.stage]);
                    mbar_arrive_expect_tx(bar, C::kTile);
                    tma_load_rows(smem_u32(sK) + ring.stage * C::kTile, &tmK, bar, it.tiles.tile(j) * kWinT, hk, it.b);
                }
            }
        } else if (warp == 11) {
            // =========================== V producer ===========================
            // A tile with keys that no row sees lands at a barrier of its own; it is handed on once they are zero, behind the next tile's copy.
            Ring ring;
            uint32_t land_phases = 0;
            int held = -1, held_key0 = 0;  // stage of the tile that is not handed on yet
            KeyRange held_range = {0, 0, 0, 0, 0};
            auto hand_on = [&]() -> bool {
                if (held < 0) return true;
                if (!mbar_wait_warp(smem_u32(&bars.v_land[held]), (land_phases >> held) & 1, abortp)) return false;
                land_phases ^= 1u << held;
                zero_unseen_keys<D, 32>(sV + held * C::kTile, p.g, held_range, held_key0, lane);
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bars.v_full[held]));
                held = -1;
                return true;
            };
            bool ok = true, first = true;
            for (int k = 0; ok && load_item(p, k, it); ++k) {
                const int n = it.tiles.count(), hk = it.hk;
                for (int j = 0; j < n; ++j, ring.advance<C::kV>()) {
                    const int key0 = it.tiles.tile(j) * kWinT;
                    // (a slot becomes free without the tile that is held: that is a later one's)
                    ok = mbar_wait_warp(smem_u32(&bars.v_empty[ring.stage]), ring.phase ^ 1, abortp);
                    if (!ok) break;
                    const bool unseen = has_unseen_keys(p.g, it.range, key0);
                    if (lane == 0 && !(p.withhold && first)) {
                        const uint32_t bar = smem_u32(unseen ? &bars.v_land[ring.stage] : &bars.v_full[ring.stage]);
                        mbar_arrive_expect_tx(bar, C::kTile);
                        tma_load_rows(smem_u32(sV) + ring.stage * C::kTile, &tmV, bar, key0, hk, it.b);
                    }
                    first = false;
                    ok = hand_on();
                    if (!ok) break;
                    if (unseen) {
                        held = ring.stage;
                        held_key0 = key0;
                        held_range = it.range;
                    }
                }
            }
            if (ok) hand_on();
        } else if (warp == 9) {
            // =========================== Q K^T issuer ===========================
            // (Here and below the whole warp walks through the loop and one elected lane issues: with uniform control flow the
            // descriptors stay in uniform registers.  From one lane's registers an instruction took about 100 clk to issue.)
            constexpr uint32_t idesc = make_idesc_f32(kWinT, kWinT, 0, 0, F16);
            const uint64_t descQ = make_smem_desc_sw128(smem_u32(sQ), 16, 1024), descK = make_smem_desc_sw128(smem_u32(sK), 16, 1024);
            const bool leader = elect_one();
            Ring ring;
            uint32_t n_q = 0, g = 0;
            bool ok = true;
            for (int k = 0; ok && load_item(p, k, it); ++k) {
                const int n = it.tiles.count();
                if (n == 0) continue;
                const uint32_t qb = n_q & 1;
                ok = mbar_wait_warp(smem_u32(&bars.q_full[qb]), (n_q >> 1) & 1, abortp);
                ++n_q;
                const uint64_t q0 = descQ + (uint64_t)((qb * C::kTile) >> 4);
                for (int j = 0; ok && j < n; ++j, ++g) {
                    if (g >= 2) ok = mbar_wait_warp(smem_u32(&bars.s_free[g & 1]), ((g >> 1) - 1) & 1, abortp);  // scores read
                    ok = ok && mbar_wait_warp(smem_u32(&bars.k_full[ring.stage]), ring.phase, abortp);
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t k0 = descK + (uint64_t)((ring.stage * C::kTile) >> 4);
                    const uint32_t d_s = tmem + ((g & 1) ? C::kS1 : C::kS0);
                    if (leader) {
#pragma unroll
                        for (int kk = 0; kk < D / 16; ++kk) {
                            const uint64_t off = (uint64_t)(((kk / 4) * SUB + (kk % 4) * 32) >> 4);
                            mma_ss(d_s, q0 + off, k0 + off, idesc, kk > 0);
                        }
                        mma_commit(smem_u32(&bars.s_full[g & 1]));
                        mma_commit(smem_u32(&bars.k_empty[ring.stage]));
                        if (j == n - 1) mma_commit(smem_u32(&bars.q_empty[qb]));
                    }
                    ring.advance<C::kK>();
                }
            }
        } else if (warp == 10) {
            // =========================== P V issuer ===========================
            constexpr uint32_t idesc = make_idesc_f32(kWinT, D, 0, 1, F16);
            const uint64_t descV = make_smem_desc_sw128(smem_u32(sV), SUB, 1024);
            const bool leader = elect_one();
            Ring ring;
            uint32_t n_it = 0, g = 0;
            bool ok = true;
            for (int k = 0; ok && load_item(p, k, it); ++k) {
                const int n = it.tiles.count();
                if (n == 0) continue;
                ok = mbar_wait_warp(smem_u32(&bars.o_free), (n_it & 1) ^ 1, abortp);  // the accumulator has been drained
                ++n_it;
                for (int j = 0; ok && j < n; ++j, ++g) {
                    ok = mbar_wait_warp(smem_u32(&bars.v_full[ring.stage]), ring.phase, abortp) &&
                         mbar_wait_warp(smem_u32(&bars.p_ready[g & 1]), (g >> 1) & 1, abortp);
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t v0 = descV + (uint64_t)((ring.stage * C::kTile) >> 4);
                    const uint32_t d_o = tmem + C::kO, a_p = tmem + ((g & 1) ? C::kP1 : C::kP0);
                    const uint32_t keep = j > 0;
                    if (leader) {
#pragma unroll
                        for (int kk = 0; kk < kWinT / 16; ++kk)
                            mma_ts(d_o, a_p + kk * 8, v0 + (uint64_t)(kk * 128), idesc, kk > 0 ? 1u : keep);
                        mma_commit(smem_u32(&bars.v_empty[ring.stage]));
                        mma_commit(smem_u32(&bars.pv_done[g & 7]));
                        if (j == n - 1) mma_commit(smem_u32(&bars.o_full));
                    }
                    ring.advance<C::kV>();
                }
            }
        }
    } else {
        // =========================== softmax warpgroup x ===========================
        reg_inc<184>();
        const int x = warp >> 2, tw = tid & 127;
        const uint32_t t_lane = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t t_s = t_lane + (x ? C::kS1 : C::kS0), t_p = t_lane + (x ? C::kP1 : C::kP0);
        const uint32_t b_ref = smem_u32(&bars.ref_ready[x]);
        const float c2 = p.scale_log2;
        const uint64_t c22 = pack_f32x2(c2, c2);
        uint32_t g = 0, n_it = 0;
        bool ok = true;
        for (int k = 0; ok && load_item(p, k, it); ++k) {
            const int n = it.tiles.count();
            if (n == 0) continue;
            float m_ref = -INFINITY, l = 0.f;  // the reference of this warpgroup's last tile, and its sum in it
            for (int j = ((g & 1) == (uint32_t)x) ? 0 : 1; j < n; j += 2) {
                const uint32_t t = g + j;
                ok = mbar_wait_warp(b_ref, (t >> 1) & 1, abortp);  // (which is behind s_full)
                if (!ok) break;
                tc_fence_after();
                const float m = mref[x][tw];
                uint32_t r[kWinT];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32(t_s + c * 32, &r[c * 32]);
                tc_wait_ld();
                tc_fence_before();
                mbar_arrive(smem_u32(&bars.s_free[x]));
                if (m_ref != m) {
                    l *= ex2_approx(m_ref - m);  // (m_ref = -inf: l is zero)
                    m_ref = m;
                }
                const float neg_m = (m == -INFINITY) ? 0.f : kShift<F16> - m;
                const uint64_t nm2 = pack_f32x2(neg_m, neg_m);
                uint64_t sum01 = pack_f32x2(0.f, 0.f), sum23 = sum01;
                if (t >= 2) {  // this warpgroup's last P has been read
                    ok = mbar_wait_warp(smem_u32(&bars.pv_done[(t - 2) & 7]), ((t - 2) >> 3) & 1, abortp);
                    if (!ok) break;
                    tc_fence_after();
                }
                // stored 32 keys at a time, beside the next keys' exponentials (all at the end: 190 -> 174 us at 4 heads, the shape above)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    exp_keys<F16>(r + c * 32, c22, nm2, sum01, sum23);
                    tmem_st16(t_p + c * 16, r + c * 32);
                }
                float s0, s1, s2, s3;
                unpack_f32x2(sum01, s0, s1);
                unpack_f32x2(sum23, s2, s3);
                l += (s0 + s1) + (s2 + s3);
                tc_wait_st();
                tc_fence_before();
                mbar_arrive(smem_u32(&bars.p_ready[x]));
            }
            if (!ok) break;
            ok = mbar_wait_warp(smem_u32(&bars.e_taken), (n_it & 1) ^ 1, abortp);
            if (!ok) break;
            g += n;
            lfin[x][tw] = l;
            if (((g - 1) & 1) != (uint32_t)x) mfin[tw] = m_ref;
            mbar_arrive(smem_u32(&bars.e_ready));
            ++n_it;
        }
    }

    end_of_cta(abortp, &g_window_status, (int)BSA_ERR_DEVICE_TIMEOUT);
    if (warp == 9) tmem_dealloc(tmem, kTmemCols);
}

template <int D, bool F16>
cudaError_t launch_rows(const WindowArgs& a, const bsa_view_t& Q, const bsa_view_t& K, const bsa_view_t& V, Params p, bool behind, cudaStream_t stream) {
    CUtensorMap tq, tk, tv;
    if (!encode_view_map(&tq, Q, a.g.N, a.g.heads, a.g.batch, D, kWinT, F16) ||
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
    const int grid = a.num_sms < p.order.n_items ? a.num_sms : p.order.n_items;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = Cfg<D>::kSmem;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = behind ? 1 : 0;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, tq, tk, tv, p);
    if (e == cudaSuccess) count_launch();
    return e;
}

}  // namespace

cudaError_t set_window_wait_limit(long long cycles) { return cudaMemcpyToSymbol(ptx::g_wait_limit_cycles, &cycles, sizeof cycles); }
static std::atomic<bool> g_withhold{false};
void set_window_withhold(bool on) { g_withhold.store(on, std::memory_order_relaxed); }
bool window_withhold() { return g_withhold.load(std::memory_order_relaxed); }

cudaError_t window_status_word(int device, int** out) {
    static std::atomic<int*> word[kMaxDevices];
    *out = word[device].load(std::memory_order_acquire);
    if (*out) return cudaSuccess;
    const cudaError_t e = cudaGetSymbolAddress(reinterpret_cast<void**>(out), g_window_status);
    if (e == cudaSuccess) word[device].store(*out, std::memory_order_release);
    return e;
}

bool view_is_wide(const bsa_view_t& v, int64_t batch, int64_t heads, int64_t rows) {
    const auto on32 = [](int64_t n, int64_t stride) { return n == 1 || stride % 16 == 0; };
    return (reinterpret_cast<uintptr_t>(v.data) & 31) == 0 && on32(batch, v.batch) && on32(heads, v.head) && on32(rows, v.row);
}

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
    return BSA_OK;
}

bsa_status_t window_device(WindowArgs* a) {
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

// Which kernel.  Per 128 keys the one for few rows takes an SM 0.77 us for each 16 rows of a key head (d = 128) and spreads the keys over the
// GPU; the one for tiles takes 0.73 us for 128 rows of a query head and gives a tile to one SM, so that it needs whole rounds of them.
// us, few rows / tiles: 65536 keys, 32 + 8 heads: 64 rows per key head, one sequence 75 / 375, eight 590 / 922; 96 rows, eight sequences
// 982 / 936; 256 rows, one 305 to 365 / 375; 512 rows, one 580 / 375; 16384 keys, 8 x 16 heads, d = 64: 16 rows 84 / 97, 48 rows 131 / 105.
// Over a short window the joins weigh more: 1024 keys, one sequence, 64 rows 10 / 19, 96 rows 18 / 14.
static bool takes_rows(const WindowArgs& a) {
    const int64_t window = (int64_t)a.g.left + a.g.right + a.g.sinks + a.g.N, most = (window < a.g.N_kv ? window : a.g.N_kv) > 4096 ? 256 : 64;
    const int64_t rows = (int64_t)a.g.N * a.g.group, blocks = (rows + 15) / 16 * a.g.batch * a.g.heads_kv;
    const int64_t tiles = (a.g.N + kWinT - 1) / kWinT, rounds = (tiles * a.g.batch * a.g.heads + a.num_sms - 1) / a.num_sms;
    return rows <= most && blocks <= rounds * a.num_sms;
}

cudaError_t launch_window_tiles(const WindowArgs& a, const bsa_view_t& Q, const bsa_view_t& K, const bsa_view_t& V, const bsa_view_t& O,
                                float* LSE, bool even, bool behind, cudaStream_t stream) {
    Params p = {};
    p.g = a.g;
    p.O = static_cast<uint16_t*>(O.data);
    p.o_batch = O.batch; p.o_head = O.head; p.o_row = O.row;
    p.LSE = LSE;
    p.o_wide = view_is_wide(O, a.g.batch, a.g.heads, a.g.N);
    p.scale_log2 = a.scale * 1.4426950408889634f;
    p.withhold = window_withhold();
    const int n_qt = (a.g.N + kWinT - 1) / kWinT;
    p.order = ItemOrder(n_qt, even ? 0 : cut_tiles(a.g, n_qt), a.g.batch * a.g.heads);
    p.heads = Divisor(a.g.heads);
    p.group = Divisor(a.g.group);
    return a.d == 64 ? (a.f16 ? launch_rows<64, true>(a, Q, K, V, p, behind, stream) : launch_rows<64, false>(a, Q, K, V, p, behind, stream))
                     : (a.f16 ? launch_rows<128, true>(a, Q, K, V, p, behind, stream) : launch_rows<128, false>(a, Q, K, V, p, behind, stream));
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
    bsa_status_t st = window_args(t, &a);
    if (st == BSA_OK && (view_overlaps(*O, t->batch, t->heads, t->N, t->d) || O->data == K->data || O->data == V->data ||
                         LSE == Q->data || LSE == K->data || LSE == V->data || LSE == O->data))
        st = BSA_ERR_INVALID_ARG;
    if (st == BSA_OK) st = window_device(&a);
    if (st != BSA_OK) return st;
    const cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_v);
    if (!window_tiles_fit(a)) return BSA_ERR_UNSUPPORTED;
    const cudaError_t e = takes_rows(a) ? launch_window_rows(a, *Q, *K, *V, *O, LSE, stream)
                                        : launch_window_tiles(a, *Q, *K, *V, *O, LSE, false, false, stream);
    if (e != cudaSuccess) {
        set_cuda_err(e, "bsa_window_forward");
        return BSA_ERR_CUDA;
    }
    return BSA_OK;
}

extern "C" bsa_status_t bsa_window_status(int* status_out) {
    if (!status_out) return BSA_ERR_INVALID_ARG;
    int v = 0;
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e == cudaSuccess && device >= kMaxDevices) return BSA_ERR_CUDA;
    static std::mutex one_look;  // of a process at a time: g_window_taken is the look's
    const std::lock_guard<std::mutex> lock(one_look);
    if (e == cudaSuccess) e = cudaDeviceSynchronize();  // (a copy alone is not ordered behind non-blocking streams)
    if (e == cudaSuccess) {
        take_window_status<<<1, 1>>>();
        e = cudaGetLastError();
    }
    if (e == cudaSuccess) e = cudaMemcpyFromSymbol(&v, g_window_taken, sizeof v);
    if (e != cudaSuccess) {
        set_cuda_err(e, "bsa_window_status");
        return BSA_ERR_CUDA;
    }
    *status_out = v;
    return BSA_OK;
}
