// Attention over a window of the 8-bit cache: forward for rows by the tile (prefill, chunks of a stream).
//
// The same mathematics and the same way through a tile as for the 16-bit cache (bsa_window.cu), with these differences:
//   * A pair of CTAs takes 256 query rows of one head, each 128 of them, and one tensor instruction works for both (cta_group::2): of a tile of 128
//     keys each CTA brings, widens and keeps half (64 keys of K, half of V's channels).  A tile's codes cross from L2 once for 256 rows, in
//     one byte an element: a quarter of the traffic of 128-row tiles of 16-bit keys.
//   * K's codes go to the tensor instruction as they are (kind::f8f6f4, twice as fast as on halves).  For that Q is cut into numbers of 8 bits
//     that add up to it: a row is multiplied by the power of two that takes its largest element to 448 at most; the first piece is the nearest e4m3
//     number, the others are the nearest e5m2 numbers to what is left, one of them for bf16, two for half.  From 2^-6 on (2^-15 of the row's largest)
//     that is exact, below it is off by 2^-21 (half: 2^-23) of the largest at most.  A pass in front cuts Q up and leaves for each row the factor that
//     takes its products to scores (log2 domain): scale, the row's power of two and K's largest scale in one.  The softmax multiplies it with the
//     blocks' scales relative to the largest.
//   * V's codes widen to half on their way through the SM: two warps read the copied codes and write the swizzled tiles that the tensor instruction takes.
//     A block's scale is applied there, relative to the largest scale of the call's window of that head: code 2^(s - s_max) is exact while a block is
//     within 2^15 of the largest (below, it is off by 2^-25 of that scale at most, half of half's smallest step).
//   * Where there are few row tiles and long windows, an item's keys are cut into parts, whose (m, l, O) a last kernel joins.
//   warps 0-3 / 4-7 : softmax warpgroups (thread = row); tile t belongs to warpgroup t mod 2, and S and P buffer t mod 2 with it
//   warp 8 : copies, K's scales   warp 9 : issuer (second CTA: tells the first what has landed)   warps 10, 11 : V converters
//   warps 12-15 : references: each row's running maximum, the tiles' edges, the accumulator's rescaling, and the epilogue
// Barriers that the issuer waits for lie in the first CTA and count the warps of both; its commits arrive in both.
// 300 rows x 65536 keys, 8 heads, d = 128: 145 us, of which the pass in front has 5 and the join 5; 466 through 16 bits.  With the GPU full 870 to 1040 TFLOP/s
// where blocks' scales differ, 1010 to 1260 where they do not (4736 x 25088, 12 heads; the power cap among the reasons), 16 bits 1120 to 1270: this kernel is for calls that do not fill it.
// Tensor pipe and special-function unit are 51 % busy, a quarter-SM issues 38 % of its time: what bounds a tile is its chain from Q K^T over the references and
// weights to P V, across two CTAs.  Tried: an issuer that polls for whichever product is ready (10 % slower: three tests of barriers take longer than
// the order costs), a warp for each product with the copies beside one of them (25 % slower), the issuer's loop unrolled by four with constant
// descriptors (spills; 40 % slower), K widened to half as V is (its converter became the bottleneck: 530 TFLOP/s), V's scales in the exponents of the weights
// instead of in V (no faster at d = 128, 5 to 10 % slower at 64 where scales differ).
// Tensor-memory columns: S0 0, S1 128, O 256, P0 384, P1 448.  Registers (setmaxnreg): 256 * 176 + 128 * 96 + 128 * 64 = 65536, the
// launch's 512 * 128.
#include <cuda_fp16.h>
#include <float.h>
#include <math.h>

#include <atomic>
#include <type_traits>

#include "bsa_cache.cuh"

namespace bsa {

using namespace ptx;

namespace {

constexpr int kThreads = 512;
constexpr int kPairRows = 2 * kWinT;
constexpr uint32_t kTmemCols = 512;
constexpr float kRescale = 8.0f;  // log2 units: P stays below 2^8 between rescales
constexpr float kShift = 7.0f;    // P is computed 2^7 times as large, up to 2^15: half ends at 2^16, and loses bits below 2^-14
constexpr int kMaxParts = 16;

template <int D, bool F16>
struct Cfg {
    static constexpr int kPieces = F16 ? 3 : 2;    // of Q
    static constexpr int kPiece = kWinT * D;       // bytes of one of a CTA's Q tile
    static constexpr int kQ = kPieces * kPiece;
    static constexpr int kHalf = kWinT * D;        // of a CTA's half of a tile of V in 16 bits
    static constexpr int kCodes = kWinT * D / 2;   // and of K or V in codes
    static constexpr int kK = 4, kC = 3, kV = 2;   // tiles in the rings: K's codes, V's codes, V
    static constexpr int kSmem = 2 * kQ + kV * kHalf + (kK + kC) * kCodes;
    static constexpr uint32_t kS0 = 0, kS1 = 128, kO = 256, kP0 = 384, kP1 = 448;
};

struct Params {
    WindowGeom g;
    uint16_t* O;
    long long o_batch, o_head, o_row;
    float* LSE;
    int o_wide;
    const float* c2;           // [batch][heads][N]
    const int32_t* refs;       // [batch][heads_kv][2]: the largest scales of K and V
    const uint8_t *k_scale, *v_scale;
    long long s_batch, s_head;
    int lg_block, last_block;
    int withhold;              // test hook: no copy of the first tile of V
    ItemOrder order;           // 256-row tiles, from a sequence's last to its first
    Divisor heads, group, items;
    int parts, n_all;          // of an item; items of all parts
    float* part_O;             // [parts][batch][heads][N][D], in the accumulator's units
    float2* part_ml;           // [parts][batch][heads][N]: maximum (log2 domain), sum
    int* status;
};

struct __align__(8) Barriers {
    uint64_t q_full[2], q_empty[2];  // (first CTA: its own copies and the second's message that its have landed)
    uint64_t k_full[4], k_empty[4];
    uint64_t v8_full[3], v8_empty[3], v_empty[2];
    uint64_t s_full[2], s_free[2], ref_ready[2], p_ready[2];
    uint64_t pv_done[8];  // tile t: t mod 8 (see the reference warpgroup)
    uint64_t o_full, o_free, e_ready, e_taken;
};

struct Item {
    int b, h, hk, row0, part;
    Sequence seq;
    KeyRange range;  // of the pair's rows
    TileSpan tiles;
    int j0, n;       // this part's tiles
};

// The pair's k-th item, dealt in alternating directions; false past the end.
__device__ __forceinline__ bool load_item(const Params& p, int k, Item& it) {
    const int G = gridDim.x >> 1, me = blockIdx.x >> 1;
    const int idx = k * G + ((k & 1) ? (G - 1 - me) : me);
    if (idx >= p.n_all) return false;
    int item, tile, rest;
    it.part = p.items.div(idx, item);
    const int bh = p.order.row_of(item, tile), qt = p.order.n_tiles - 1 - tile;
    it.b = p.heads.div(bh, it.h);
    it.hk = p.group.div(it.h, rest);
    it.row0 = qt * kPairRows;
    it.seq = load_sequence(p.g, it.b);
    it.range = key_range(p.g, it.seq, it.row0, it.row0 + kPairRows);
    it.tiles = tile_span(it.range);
    const int n = it.tiles.count();
    it.j0 = p.parts == 1 ? 0 : (int)((long long)n * it.part / p.parts);
    it.n = p.parts == 1 ? n : (int)((long long)n * (it.part + 1) / p.parts) - it.j0;
    return true;
}
__device__ __forceinline__ int item_key0(const Item& it, int j) { return it.tiles.tile(it.j0 + j) * kWinT; }

template <int R>
__device__ __forceinline__ void reg_inc() {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(R));
}
template <int R>
__device__ __forceinline__ void reg_dec() {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(R));
}

// ---- what works across the pair ----
__device__ __forceinline__ uint32_t cta_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void pair_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t in_first_cta(uint32_t smem) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(smem));
    return r;
}
// (What the first CTA's products then read lies in tensor memory, behind tcgen05.fence, or in the arriving CTA's shared memory, behind fence.proxy.async; a
// release at cluster scope besides took a quarter of the kernel's time.)
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void pair_tmem_alloc(uint32_t dst_smem, uint32_t ncols) {  // a whole warp of each CTA
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst_smem), "r"(ncols) : "memory");
}
__device__ __forceinline__ void pair_tmem_relinquish() { asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void pair_tmem_dealloc(uint32_t taddr, uint32_t ncols) {
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols) : "memory");
}
__device__ __forceinline__ void pair_mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void pair_mma_ss8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// Arrive at this barrier of both CTAs once every product issued so far has completed.
__device__ __forceinline__ void pair_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((unsigned short)3) : "memory");
}
// The same in every lane, and the compiler knows it: what the tensor instructions take from uniform registers.
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __shfl_sync(0xffffffffu, v, 0); }
__device__ __forceinline__ uint64_t uniform(uint64_t v) { return (uint64_t)uniform((uint32_t)(v >> 32)) << 32 | uniform((uint32_t)v); }
// As make_smem_desc_sw128, rows of 64 bytes with their own swizzle.
__device__ __forceinline__ uint64_t make_smem_desc_sw64(uint32_t smem_addr, uint32_t lbo_bytes, uint32_t sbo_bytes) {
    const uint64_t d = make_smem_desc_sw128(smem_addr, lbo_bytes, sbo_bytes);
    return (d & ~(7ull << 61)) | (4ull << 61);
}

// Instruction descriptor for kind::f8f6f4: A e4m3 or e5m2, B e4m3, fp32 accumulation, both with their channels contiguous.
__host__ __device__ constexpr uint32_t make_idesc_8(int M, int N, bool a_e5m2) {
    return (1u << 4) | (uint32_t(a_e5m2) << 7) | (uint32_t(N >> 3) << 17) | (uint32_t(M >> 4) << 24);
}

// Of a tile whose rows are as long as its swizzle: D bytes.
template <int D>
__device__ __forceinline__ uint64_t desc_of(const uint8_t* at) {
    return D == 128 ? make_smem_desc_sw128(smem_u32(at), 16, 1024) : make_smem_desc_sw64(smem_u32(at), 16, 512);
}

// P of 32 keys in the place of their scores: exp2(s * c2 + neg_m), rounded and packed by pairs; its unrounded sum.
__device__ __forceinline__ void exp_keys(uint32_t* r, float c_lo, float c_hi, uint64_t neg_m2, uint64_t& sum01, uint64_t& sum23) {
    const uint64_t lo = pack_f32x2(c_lo, c_lo), hi = pack_f32x2(c_hi, c_hi);  // of the first and of the last 16
#pragma unroll
    for (int i = 0; i < 32; i += 4) {
        const uint64_t c22 = i < 16 ? lo : hi;
        float x0, x1, x2, x3;
        unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(r[i]), __uint_as_float(r[i + 1])), c22, neg_m2), x0, x1);
        unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(r[i + 2]), __uint_as_float(r[i + 3])), c22, neg_m2), x2, x3);
        const float p0 = ex2_approx(x0), p1 = ex2_approx(x1), p2 = ex2_approx(x2), p3 = ex2_approx(x3);
        sum01 = add_f32x2(sum01, pack_f32x2(p0, p1));
        sum23 = add_f32x2(sum23, pack_f32x2(p2, p3));
        r[i / 2] = pack_f16x2(p0, p1);
        r[i / 2 + 1] = pack_f16x2(p2, p3);
    }
}

// 16 codes to 16 halves times m2 (PLAIN: that is one), as two 16-byte pieces.
template <bool PLAIN>
__device__ __forceinline__ void widen(const uint4& w, uint32_t m2, uint4& lo, uint4& hi) {
    const __half2 m = *reinterpret_cast<const __half2*>(&m2);
    const uint32_t in[4] = {w.x, w.y, w.z, w.w};
    uint32_t out[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t a, b;
        e4m3x4_to_f16x4(in[i], a, b);
        if (!PLAIN) {
            const __half2 x = __hmul2(*reinterpret_cast<const __half2*>(&a), m), y = __hmul2(*reinterpret_cast<const __half2*>(&b), m);
            a = *reinterpret_cast<const uint32_t*>(&x);
            b = *reinterpret_cast<const uint32_t*>(&y);
        }
        out[2 * i] = a;
        out[2 * i + 1] = b;
    }
    lo = make_uint4(out[0], out[1], out[2], out[3]);
    hi = make_uint4(out[4], out[5], out[6], out[7]);
}
// 2^(code - ref) as a pair of halves (ref: the largest, so that a larger one belongs to keys that nobody sees); NaN for 255.
__device__ __forceinline__ uint32_t block_factor(int code, int ref) {
    const int f = 15 + min(code - ref, 0);  // exponent field, below one: subnormal
    uint32_t bits = f >= 1 ? (uint32_t)f << 10 : f > -10 ? 1u << (9 + f) : 0u;
    if (code == 255) bits = 0x7e00u;
    return bits | bits << 16;
}

// FINE: blocks of 16 or 32 tokens, so that a tile of keys may have eight scales; else it has two.
template <int D, bool F16, bool FINE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
cache_tiles_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                   const __grid_constant__ CUtensorMap tmV, const __grid_constant__ Params p) {
    using C = Cfg<D, F16>;
    constexpr int NV = D / 2;             // V's channels of a CTA
    extern __shared__ __align__(1024) uint8_t smem[];
    uint8_t* sQ = smem;
    uint8_t* sK = sQ + 2 * C::kQ;
    uint8_t* sV = sK + C::kK * C::kCodes;
    uint8_t* sV8 = sV + C::kV * C::kHalf;
    __shared__ Barriers bars;
    __shared__ float mref[2][kWinT];  // [tile mod 2][row]: the tile's reference maximum (log2 domain)
    // K's scales relative to the largest, for each 16 (64) keys of tile t at t mod 8: written again when Q K^T of t + 4 is done, so the scores of t + 2 have
    // been read, by warpgroups that are done with t.
    constexpr int NF = FINE ? 8 : 2, FK = kWinT / NF;  // scales of a tile, keys of one
    __shared__ __align__(16) float kfac[8][NF];
    __shared__ float lfin[2][kWinT];  // [warpgroup][row]: an item's row sums, each in the reference of the warpgroup's last tile,
    __shared__ float mfin[kWinT];     // which is here for the warpgroup that did not have the item's last one
    __shared__ uint32_t tmem_base_s, abort_flag;

    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    const int rank = (int)cta_rank();
    const bool misplaced = (smem_u32(smem) & 1023u) != 0;  // never expected; fail with a status instead of corrupting tiles
    if (misplaced) {
        if (tid == 0) atomicExch(p.status, (int)BSA_ERR_CUDA);
        return;  // (both CTAs of the pair: the layout is the kernel's)
    }
    if (tid == 0) {
        abort_flag = 0;
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&bars.q_full[i]), rank == 0 ? 2 : 1);
            mbar_init(smem_u32(&bars.q_empty[i]), 1);
            mbar_init(smem_u32(&bars.s_full[i]), 1);
            mbar_init(smem_u32(&bars.s_free[i]), 8);
            mbar_init(smem_u32(&bars.ref_ready[i]), 128);
            mbar_init(smem_u32(&bars.p_ready[i]), 12);
            mbar_init(smem_u32(&bars.v_empty[i]), 1);
        }
        for (int i = 0; i < 4; ++i) {
            mbar_init(smem_u32(&bars.k_full[i]), rank == 0 ? 2 : 1);
            mbar_init(smem_u32(&bars.k_empty[i]), 1);
        }
        for (int i = 0; i < 3; ++i) {
            mbar_init(smem_u32(&bars.v8_full[i]), 1);
            mbar_init(smem_u32(&bars.v8_empty[i]), 2);
        }
        for (int i = 0; i < 8; ++i) mbar_init(smem_u32(&bars.pv_done[i]), 1);
        mbar_init(smem_u32(&bars.o_full), 1);
        mbar_init(smem_u32(&bars.o_free), 8);
        mbar_init(smem_u32(&bars.e_ready), 256);
        mbar_init(smem_u32(&bars.e_taken), 128);
        fence_mbar_init();
    }
    if (warp == 9) {
        pair_tmem_alloc(smem_u32(&tmem_base_s), kTmemCols);
        pair_tmem_relinquish();
    }
    if (warp == 8 && lane == 0) {
        prefetch_tensormap(&tmQ);
        prefetch_tensormap(&tmK);
        prefetch_tensormap(&tmV);
    }
    tc_fence_before();
    __syncthreads();
    pair_sync();  // the other CTA's barriers are there, too
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_base_s, 0);
    volatile uint32_t* abortp = &abort_flag;
    grid_dependency_wait();  // Q's pieces, the rows' factors and the largest scales are from the kernel in front
    Item it;

    if (warp >= 12) {
        // =========================== references and epilogue ===========================
        reg_dec<96>();
        const int tw = tid & 127;
        const uint32_t t_lane = tmem + ((uint32_t)((warp & 3) * 32) << 16), t_o = t_lane + C::kO;
        const uint32_t o_free = in_first_cta(smem_u32(&bars.o_free));
        uint32_t n_it = 0, g = 0;  // items finished (with tiles), tiles in front of the item
        KeyRange own;              // what this CTA's rows of the item at hand see
        float c2;                  // and their factor
        auto take_item = [&](const Item& w) {
            const int row0 = w.row0 + rank * kWinT, row = row0 + tw;
            own = key_range(p.g, w.seq, row0, row0 + kWinT);
            c2 = row < p.g.N ? p.c2[((long long)w.b * p.g.heads + w.h) * p.g.N + row] : 1.f;
        };
        // The reference of tile j of an item (running index t) follows from `m`, that of the tile before, and its scores.  Where rows do
        // not see the whole tile, this warpgroup writes the scores back with the hidden ones at -inf: the softmax warpgroups, whose loop is
        // the kernel's bottleneck, have no edges.  Returns whether any row of the warp has moved to a new reference (m_old: the one before).
        auto find = [&](const Item& w, int j, uint32_t t, float& m, float& m_old, bool& moved) -> bool {
            const uint32_t t_s = t_lane + ((t & 1) ? C::kS1 : C::kS0);
            const int key0 = item_key0(w, j);
            const bool full = own.hi == 0 || tile_is_full(p.g, own, key0);  // (rows that see nothing need no mask: their outputs go by their positions)
            if (!mbar_wait_warp(smem_u32(&bars.s_full[t & 1]), (t >> 1) & 1, abortp)) return false;
            tc_fence_after();
            float mx = -INFINITY;
            auto largest16 = [](const uint32_t* r) -> float {
                float m0 = max3(__uint_as_float(r[0]), __uint_as_float(r[1]), __uint_as_float(r[2]));
                float m1 = max3(__uint_as_float(r[3]), __uint_as_float(r[4]), __uint_as_float(r[5]));
                m0 = max3(m0, __uint_as_float(r[6]), __uint_as_float(r[7]));
                m1 = max3(m1, __uint_as_float(r[8]), __uint_as_float(r[9]));
                m0 = max3(m0, __uint_as_float(r[10]), __uint_as_float(r[11]));
                m1 = max3(m1, __uint_as_float(r[12]), __uint_as_float(r[13]));
                return fmaxf(max3(m0, __uint_as_float(r[14]), __uint_as_float(r[15])), m1);
            };
            const float* fac = kfac[t & 7];
            if (full) {
#pragma unroll 1
                for (int c = 0; c < kWinT; c += 64) {  // (this way lies on most tiles' path: two waits, no votes)
                    uint32_t r[64];
                    tmem_ld32(t_s + c, r);
                    tmem_ld32(t_s + c + 32, r + 32);
                    if (FINE) {
                        const float4 f = *reinterpret_cast<const float4*>(fac + c / 16);
                        tc_wait_ld();
                        mx = max3(mx, largest16(r) * f.x, largest16(r + 16) * f.y);
                        mx = max3(mx, largest16(r + 32) * f.z, largest16(r + 48) * f.w);
                    } else {
                        const float f = fac[c / 64];
                        tc_wait_ld();
                        float m0 = -INFINITY, m1 = m0, m2 = m0, m3 = m0;
#pragma unroll
                        for (int i = 0; i < 64; i += 8) {
                            m0 = max3(m0, __uint_as_float(r[i]), __uint_as_float(r[i + 1]));
                            m1 = max3(m1, __uint_as_float(r[i + 2]), __uint_as_float(r[i + 3]));
                            m2 = max3(m2, __uint_as_float(r[i + 4]), __uint_as_float(r[i + 5]));
                            m3 = max3(m3, __uint_as_float(r[i + 6]), __uint_as_float(r[i + 7]));
                        }
                        mx = fmaxf(mx, max3(m0, m1, fmaxf(m2, m3)) * f);
                    }
                }
            } else {
                const RowView view(p.g, w.seq, w.seq.start + w.row0 + rank * kWinT + tw, key0);
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
                    mx = max3(mx, largest16(r) * fac[c / FK], largest16(r + 16) * fac[(c + 16) / FK]);
                }
                tc_wait_st();
            }
            mx *= c2;
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
        if (more) take_item(it);
        for (int k = 0; more; ++k) {
            const Item w = it;
            const int row = w.row0 + rank * kWinT + tw;
            const bool row_ok = row < p.g.N;
            const int pos = w.seq.start + row;
            const bool seen = pos >= 0 && pos < w.seq.len;
            const long long at = ((long long)w.b * p.g.heads + w.h) * p.g.N + row;
            uint16_t* orow = p.O + (long long)w.b * p.o_batch + (long long)w.h * p.o_head + (long long)row * p.o_row;
            float2* ml = p.part_ml + (long long)w.part * p.g.batch * p.g.heads * p.g.N + at;
            const int n = w.n;
            float m_old;
            bool moved;
            for (int j = done; ok && j < n; ++j) ok = find(w, j, g + j, m, m_old, moved) && publish(g + j, m, m_old, moved);
            if (!ok) break;
            g += (uint32_t)n;
            more = load_item(p, k + 1, it);
            if (more) take_item(it);
            done = 0;
            if (n == 0) {  // no row of the tile sees anything here
                if (row_ok && p.parts > 1) {
                    *ml = make_float2(-INFINITY, 0.f);
                } else if (row_ok) {
#pragma unroll
                    for (int c = 0; c < D / 8; ++c) reinterpret_cast<uint4*>(orow)[c] = make_uint4(0, 0, 0, 0);
                    p.LSE[at] = -INFINITY;
                }
                m = -INFINITY;
                continue;
            }
            // The next item's first two tiles come before this item's end, so that both warpgroups have work until the accumulator is
            // drained; the second one's reference waits until then where it moves the accumulator.
            const int n_next = more ? it.n : 0;
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
            // (The sum's reciprocal first, then V's largest scale: the two in one may lie below the smallest normal number where the outputs do not.)
            const float unit = scale_of(p.refs[2 * (w.b * p.g.heads_kv + w.hk) + 1]);
            const float inv = seen ? 1.f / l : 0.f;
            if (row_ok) {
                if (p.parts > 1) *ml = make_float2(m, l);
                else p.LSE[at] = seen ? fmaf(m - kShift, 0.6931471805599453f, logf(l)) : -INFINITY;
            }
            m = m_next;
            if (!mbar_wait_warp(smem_u32(&bars.o_full), n_it & 1, abortp)) break;
            ++n_it;
            tc_fence_after();
            float* part = p.part_O + ((long long)w.part * p.g.batch * p.g.heads * p.g.N + at) * D;
#pragma unroll 1
            for (int c = 0; c < D / 32; ++c) {
                uint32_t o[32];
                tmem_ld32(t_o + c * 32, o);
                tc_wait_ld();
                if (c == D / 32 - 1) {  // drained: the next item's first P V may overwrite it
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(o_free);
                }
                if (row_ok && p.parts > 1) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) st_global_v8(part + c * 32 + q * 8, o + q * 8);
                } else if (row_ok) {
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        uint32_t v[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            v[e] = seen ? pack_16x2<F16>(__uint_as_float(o[q * 16 + 2 * e]) * inv * unit, __uint_as_float(o[q * 16 + 2 * e + 1]) * inv * unit) : 0u;
                        st_global_v8_or_2v4(orow + c * 32 + q * 16, v, p.o_wide);
                    }
                }
                __syncwarp();
            }
            if (held && !publish(g + 1, m, m_old, true)) break;
        }
    } else if (warp >= 8) {
        reg_dec<64>();
        if (warp == 8) {
            // =========================== copies, K's scales ===========================
            Ring rk, rv;
            uint32_t n_q = 0, t = 0;
            bool ok = true, first = true;
            for (int k = 0; ok && load_item(p, k, it); ++k) {
                const int n = it.n;
                if (n == 0) continue;
                const uint8_t* scales = p.k_scale + it.b * p.s_batch + it.hk * p.s_head;
                const int ref = p.refs[2 * (it.b * p.g.heads_kv + it.hk)];
                auto code_of = [&](int j) -> int { return __ldg(scales + min((item_key0(it, j) + lane % NF * FK) >> p.lg_block, p.last_block)); };
                int next = code_of(0);
                const uint32_t qb = n_q & 1;
                ok = mbar_wait_warp(smem_u32(&bars.q_empty[qb]), ((n_q >> 1) & 1) ^ 1, abortp);
                if (!ok) break;
                if (lane == 0) {
                    const uint32_t bar = smem_u32(&bars.q_full[qb]);
                    mbar_arrive_expect_tx(bar, C::kQ);
#pragma unroll
                    for (int i = 0; i < C::kPieces; ++i)
                        tma_load_4d(smem_u32(sQ) + qb * C::kQ + i * C::kPiece, &tmQ, bar, 0, it.row0 + rank * kWinT, it.h, i * p.g.batch + it.b);
                }
                ++n_q;
                for (int j = 0; j < n; ++j, ++t, rk.advance<C::kK>(), rv.advance<C::kC>()) {
                    const int key0 = item_key0(it, j), code = next;
                    if (j + 1 < n) next = code_of(j + 1);
                    ok = mbar_wait_warp(smem_u32(&bars.k_empty[rk.stage]), rk.phase ^ 1, abortp);
                    if (!ok) break;
                    // (Never so small that the row's factor times it is zero, nor NaN where nobody sees any of the keys: hidden scores of -inf have to
                    // stay that.)
                    const int key = key0 + lane % NF * FK;
                    const bool seen = key < it.range.hi && (key + FK > it.range.lo || key < it.range.sink_hi);
                    const float f = !seen ? 1.f : code == 255 ? NAN : scale_of(127 + max(min(code - ref, 0), -60));
                    if (lane < NF) kfac[t & 7][lane] = f;
                    __syncwarp();
                    if (lane == 0) {
                        const uint32_t bar = smem_u32(&bars.k_full[rk.stage]);
                        mbar_arrive_expect_tx(bar, C::kCodes);
                        tma_load_4d(smem_u32(sK) + rk.stage * C::kCodes, &tmK, bar, 0, key0 + rank * 64, it.hk, it.b);
                    }
                    ok = mbar_wait_warp(smem_u32(&bars.v8_empty[rv.stage]), rv.phase ^ 1, abortp);
                    if (!ok) break;
                    if (lane == 0 && !(p.withhold && first)) {
                        const uint32_t bar = smem_u32(&bars.v8_full[rv.stage]);
                        mbar_arrive_expect_tx(bar, C::kCodes);
                        if (D == 128) tma_load_5d(smem_u32(sV8) + rv.stage * C::kCodes, &tmV, bar, 0, key0, rank, it.hk, it.b);
                        else tma_load_5d(smem_u32(sV8) + rv.stage * C::kCodes, &tmV, bar, rank * 32, key0, 0, it.hk, it.b);
                    }
                    first = false;
                }
            }
        } else if (warp == 9 && rank == 1) {
            // =========================== tells the first CTA that this one's Q and K are there ===========================
            Ring rk;
            uint32_t n_q = 0;
            const uint32_t q_full = in_first_cta(smem_u32(&bars.q_full[0])), k_full = in_first_cta(smem_u32(&bars.k_full[0]));
            bool ok = true;
            for (int k = 0; ok && load_item(p, k, it); ++k) {
                const int n = it.n;
                if (n == 0) continue;
                ok = mbar_wait_warp(smem_u32(&bars.q_full[n_q & 1]), (n_q >> 1) & 1, abortp);
                if (ok && lane == 0) mbar_arrive_cluster(q_full + (n_q & 1) * 8);
                ++n_q;
                for (int j = 0; ok && j < n; ++j, rk.advance<C::kK>()) {
                    ok = mbar_wait_warp(smem_u32(&bars.k_full[rk.stage]), rk.phase, abortp);
                    if (ok && lane == 0) mbar_arrive_cluster(k_full + rk.stage * 8);
                }
            }
        } else if (warp == 9) {
            // =========================== issuer (first CTA) ===========================
            // (The whole warp walks through the loop and one elected lane issues; descriptors are uniform for the compiler to see.)
            constexpr uint32_t idesc = make_idesc_8(kPairRows, kWinT, false), idesc_rest = make_idesc_8(kPairRows, kWinT, true);
            constexpr uint32_t idesc_o = make_idesc_f32(kPairRows, D, 0, 1, true);
            const uint64_t descQ = desc_of<D>(sQ), descK = desc_of<D>(sK), descV = desc_of<D>(sV);
            const bool leader = elect_one();
            Ring rk;
            uint32_t n_q = 0, n_o = 0, g_s = 0, g_o = 0;
            // two cursors: the item (its tiles, the tile) that Q K^T and P V are at; no tiles: past the end
            auto next_item = [&](int& k, int& n, int& j) {
                j = 0;
                do n = load_item(p, k++, it) ? it.n : -1;
                while (n == 0);
            };
            int ks = 0, ns, js, ko = 0, no, jo;
            next_item(ks, ns, js);
            next_item(ko, no, jo);
            auto issue_s = [&]() -> bool {
                const uint32_t qb = n_q & 1;
                if (js == 0 && !mbar_wait_warp(smem_u32(&bars.q_full[qb]), (n_q >> 1) & 1, abortp)) return false;
                if (g_s >= 2 && !mbar_wait_warp(smem_u32(&bars.s_free[g_s & 1]), ((g_s >> 1) - 1) & 1, abortp)) return false;  // scores read
                if (!mbar_wait_warp(smem_u32(&bars.k_full[rk.stage]), rk.phase, abortp)) return false;
                tc_fence_after();
                const uint64_t q0 = uniform(descQ + (uint64_t)((qb * C::kQ) >> 4)), k0 = uniform(descK + (uint64_t)((rk.stage * C::kCodes) >> 4));
                const uint32_t d_s = uniform(tmem + ((g_s & 1) ? C::kS1 : C::kS0));
                if (leader) {
#pragma unroll
                    for (int i = 0; i < C::kPieces; ++i)
#pragma unroll
                        for (int kk = 0; kk < D / 32; ++kk)
                            pair_mma_ss8(d_s, q0 + (uint64_t)((i * C::kPiece + kk * 32) >> 4), k0 + (uint64_t)((kk * 32) >> 4), i ? idesc_rest : idesc, i + kk > 0);
                    pair_commit(smem_u32(&bars.s_full[g_s & 1]));
                    pair_commit(smem_u32(&bars.k_empty[rk.stage]));
                    if (js == ns - 1) pair_commit(smem_u32(&bars.q_empty[qb]));
                }
                rk.advance<C::kK>();
                ++g_s;
                if (++js == ns) {
                    ++n_q;
                    next_item(ks, ns, js);
                }
                return true;
            };
            auto issue_o = [&]() -> bool {
                if (jo == 0) {  // the accumulator has been drained
                    if (!mbar_wait_warp(smem_u32(&bars.o_free), (n_o & 1) ^ 1, abortp)) return false;
                    ++n_o;
                }
                if (!mbar_wait_warp(smem_u32(&bars.p_ready[g_o & 1]), (g_o >> 1) & 1, abortp)) return false;  // and V
                tc_fence_after();
                const uint64_t v0 = uniform(descV + (uint64_t)(((g_o & 1) * C::kHalf) >> 4));
                const uint32_t d_o = uniform(tmem + C::kO), a_p = uniform(tmem + ((g_o & 1) ? C::kP1 : C::kP0)), keep = uniform((uint32_t)(jo > 0));
                if (leader) {
#pragma unroll
                    for (int kk = 0; kk < kWinT / 16; ++kk)
                        pair_mma_ts(d_o, a_p + kk * 8, v0 + (uint64_t)((kk * 16 * NV * 2) >> 4), idesc_o, kk > 0 ? 1u : keep);
                    pair_commit(smem_u32(&bars.v_empty[g_o & 1]));
                    pair_commit(smem_u32(&bars.pv_done[g_o & 7]));
                    if (jo == no - 1) pair_commit(smem_u32(&bars.o_full));
                }
                ++g_o;
                if (++jo == no) next_item(ko, no, jo);
                return true;
            };
            bool ok = true;
            for (int i = 0; ok && i < 2 && ns > 0; ++i) ok = issue_s();
            while (ok && no > 0) {
                if (ns > 0) ok = issue_s();
                ok = ok && issue_o();
            }
        } else {
            // =========================== V converters: this CTA's half of the channels, 64 keys each ===========================
            // Keys that no row of the pair sees may hold anything, and a weight of zero times NaN would not be zero: they become zero.
            Ring r8;
            uint32_t t = 0;
            const int half = warp - 10;
            const uint32_t full = in_first_cta(smem_u32(&bars.p_ready[0]));
            constexpr int ROWS = D == 128 ? 8 : 16, STEPS = 64 / ROWS;  // of a step: 64 (32) bytes each
            // [64 keys][64 (32) bytes] -> [64 keys][128 (64) bytes], 16-byte pieces XORed with bits 0-2 (1-2) of the row: eight lanes' stores fall into
            // different banks.  (A row of the result has D bytes.)
            const int r0 = D == 128 ? lane >> 2 : lane >> 1, c = D == 128 ? (lane & 3) * 2 : (lane & 1) * 2, x = D == 128 ? r0 & 7 : (r0 >> 1) & 3;
            const uint8_t* from0 = sV8 + half * (C::kCodes / 2) + lane * 16;
            uint8_t* to0 = sV + half * (C::kHalf / 2) + r0 * D + ((c ^ x) << 4);
            const int other = ((c + 1) ^ x) > (c ^ x) ? 16 : -16;  // (c is even: its neighbour lies 16 bytes further or back)
            bool ok = true;
            for (int k = 0; ok && load_item(p, k, it); ++k) {
                const int n = it.n;
                if (n == 0) continue;
                const uint8_t* scales = p.v_scale + it.b * p.s_batch + it.hk * p.s_head;
                const int ref = p.refs[2 * (it.b * p.g.heads_kv + it.hk) + 1];
                auto code_of = [&](int j) -> int { return __ldg(scales + min((item_key0(it, j) + half * 64 + (FINE ? (lane & 3) * 16 : 0)) >> p.lg_block, p.last_block)); };
                int next = code_of(0);
                for (int j = 0; j < n; ++j, ++t, r8.advance<C::kC>()) {
                    const uint32_t m2 = block_factor(next, ref);  // (FINE: lane g mod 4: of keys g * 16 ..)
                    if (j + 1 < n) next = code_of(j + 1);
                    const int key0 = item_key0(it, j);
                    const bool unseen = has_unseen_keys(p.g, it.range, key0);
                    ok = mbar_wait_warp(smem_u32(&bars.v8_full[r8.stage]), r8.phase, abortp) && mbar_wait_warp(smem_u32(&bars.v_empty[t & 1]), ((t >> 1) & 1) ^ 1, abortp);
                    if (!ok) break;
                    const uint8_t* from = from0 + r8.stage * C::kCodes;
                    uint8_t* to = to0 + (t & 1) * C::kHalf;
                    auto convert = [&](auto plain) {
#pragma unroll
                        for (int i0 = 0; i0 < STEPS; i0 += 4) {  // four loads at a time (the compiler keeps loads behind stores)
                            uint4 w[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) w[i] = *reinterpret_cast<const uint4*>(from + (i0 + i) * 512);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                uint4 lo, hi;
                                widen<decltype(plain)::value>(w[i], !FINE || decltype(plain)::value ? m2 : __shfl_sync(0xffffffffu, m2, (i0 + i) * ROWS / 16), lo, hi);
                                *reinterpret_cast<uint4*>(to + (i0 + i) * ROWS * D) = lo;
                                *reinterpret_cast<uint4*>(to + (i0 + i) * ROWS * D + other) = hi;
                            }
                        }
                    };
                    if (__all_sync(0xffffffffu, m2 == 0x3c003c00u)) convert(std::true_type{});  // all of the largest scale
                    else convert(std::false_type{});
                    if (unseen) {
                        __syncwarp();
                        for (int i = lane; i < 64; i += 32) {
                            const int key = key0 + half * 64 + i;
                            if (key >= it.range.hi || (key < it.range.lo && key >= p.g.sinks)) {
#pragma unroll
                                for (int q = 0; q < D / 16; ++q)
                                    *reinterpret_cast<uint4*>(sV + (t & 1) * C::kHalf + (half * 64 + i) * D + q * 16) = make_uint4(0, 0, 0, 0);
                            }
                        }
                    }
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(smem_u32(&bars.v8_empty[r8.stage]));
                        mbar_arrive_cluster(full + (t & 1) * 8);
                    }
                }
            }
        }
        __syncwarp();
    } else {
        // =========================== softmax warpgroup x ===========================
        reg_inc<176>();
        const int x = warp >> 2, tw = tid & 127;
        const uint32_t t_lane = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t t_s = t_lane + (x ? C::kS1 : C::kS0), t_p = t_lane + (x ? C::kP1 : C::kP0);
        const uint32_t b_ref = smem_u32(&bars.ref_ready[x]);
        const uint32_t s_free = in_first_cta(smem_u32(&bars.s_free[x])), p_ready = in_first_cta(smem_u32(&bars.p_ready[x]));
        uint32_t g = 0, n_it = 0;
        bool ok = true;
        for (int k = 0; ok && load_item(p, k, it); ++k) {
            const int n = it.n;
            if (n == 0) continue;
            const int row = it.row0 + rank * kWinT + tw;
            const float c2 = row < p.g.N ? p.c2[((long long)it.b * p.g.heads + it.h) * p.g.N + row] : 1.f;
            float m_ref = -INFINITY, l = 0.f;  // the reference of this warpgroup's last tile, and its sum in it
            for (int j = ((g & 1) == (uint32_t)x) ? 0 : 1; j < n; j += 2) {
                const uint32_t t = g + j;
                ok = mbar_wait_warp(b_ref, (t >> 1) & 1, abortp);  // (which is behind s_full)
                if (!ok) break;
                tc_fence_after();
                const float m = mref[x][tw];
                float cf[NF];  // what takes a product to its score, for each scale
                if (FINE) {
                    const float4 f0 = *reinterpret_cast<const float4*>(kfac[t & 7]), f1 = *reinterpret_cast<const float4*>(kfac[t & 7] + NF - 4);
                    const float f[8] = {f0.x, f0.y, f0.z, f0.w, f1.x, f1.y, f1.z, f1.w};
#pragma unroll
                    for (int i = 0; i < NF; ++i) cf[i] = c2 * f[i];
                } else {
                    const float2 f = *reinterpret_cast<const float2*>(kfac[t & 7]);
                    cf[0] = c2 * f.x;
                    cf[1] = c2 * f.y;
                }
                uint32_t r[kWinT];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32(t_s + c * 32, &r[c * 32]);
                tc_wait_ld();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(s_free);
                if (m_ref != m) {
                    l *= ex2_approx(m_ref - m);  // (m_ref = -inf: l is zero)
                    m_ref = m;
                }
                const float neg_m = (m == -INFINITY) ? 0.f : kShift - m;
                const uint64_t nm2 = pack_f32x2(neg_m, neg_m);
                uint64_t sum01 = pack_f32x2(0.f, 0.f), sum23 = sum01;
                if (t >= 2) {  // this warpgroup's last P has been read
                    ok = mbar_wait_warp(smem_u32(&bars.pv_done[(t - 2) & 7]), ((t - 2) >> 3) & 1, abortp);
                    if (!ok) break;
                    tc_fence_after();
                }
                // stored 32 keys at a time, beside the next keys' exponentials
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    exp_keys(r + c * 32, cf[c * 32 / FK], cf[(c * 32 + 16) / FK], nm2, sum01, sum23);
                    tmem_st16(t_p + c * 16, r + c * 32);
                }
                float s0, s1, s2, s3;
                unpack_f32x2(sum01, s0, s1);
                unpack_f32x2(sum23, s2, s3);
                l += (s0 + s1) + (s2 + s3);
                tc_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(p_ready);
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

    // The end of the pair.  Behind the first barrier no warp of either CTA issues or arrives any more; where a wait gave up, copies and products may be in
    // flight that nobody will wait for, and the memory stays the pair's until they have ended.
    tc_fence_before();
    __syncthreads();
    pair_sync();
    if (*abortp) {
        if (tid == 0) {
            let_copies_land();
            atomicExch(p.status, (int)BSA_ERR_DEVICE_TIMEOUT);
        }
        __syncthreads();
    }
    pair_sync();
    if (warp == 9) pair_tmem_dealloc(tmem, kTmemCols);
}

// ---- in front: Q in pieces, the rows' factors, the largest scales ----
struct PrepareParams {
    WindowGeom g;
    const uint16_t* Q;
    long long q_batch, q_head, q_row;
    uint8_t* Q8;  // [pieces][batch][heads][N][D]
    float* c2;
    int32_t* refs;
    const uint8_t *k_scale, *v_scale;
    long long s_batch, s_head;
    int lg_block;
    float scale_log2;
};
constexpr int kPrepThreads = 256;

__device__ __forceinline__ uint32_t f32x2_to_e5m2x2(float lo, float hi) {
    unsigned short r;
    asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float2 f16x2_to_f32x2(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }
__device__ __forceinline__ float2 e5m2x2_to_f32x2(uint32_t two) {
    uint32_t r;
    asm("cvt.rn.f16x2.e5m2x2 %0, %1;" : "=r"(r) : "h"((unsigned short)two));
    return f16x2_to_f32x2(r);
}

// A CTA takes 32 (d = 64: 64) rows of one head.  The largest scale is looked up by each anew: a byte for each block of the
// window, a few KB out of L2.
template <int D, bool F16>
__global__ void __launch_bounds__(kPrepThreads) cache_prepare_kernel(const __grid_constant__ PrepareParams p) {
    constexpr int LANES = D / 16, ROWS = kPrepThreads / LANES;
    __shared__ int most_of[kPrepThreads / 32];
    grid_launch_dependents();
    const int tid = threadIdx.x, h = blockIdx.y, b = blockIdx.z, hk = h / p.g.group;
    const Sequence seq = load_sequence(p.g, b);
    const KeyRange range = key_range(p.g, seq, 0, p.g.N);
    const int row = blockIdx.x * ROWS + tid / LANES, c = tid % LANES * 16;
    uint4 v[2];
    v[0] = v[1] = make_uint4(0, 0, 0, 0);
    if (row < p.g.N) {
        const uint4* at = reinterpret_cast<const uint4*>(p.Q + b * p.q_batch + h * p.q_head + (long long)row * p.q_row + c);
        v[0] = __ldg(at);
        v[1] = __ldg(at + 1);
    }
    auto largest = [&](const uint8_t* scales) -> int {
        scales += b * p.s_batch + hk * p.s_head;
        int most = 0;
        const int s1 = range.sink_hi > 0 ? ((range.sink_hi - 1) >> p.lg_block) + 1 : 0;
        const int w0 = range.lo >> p.lg_block, w1 = range.hi > range.lo ? ((range.hi - 1) >> p.lg_block) + 1 : 0;
        auto look = [&](int from, int to) {
#pragma unroll 8
            for (int i = from + tid; i < to; i += kPrepThreads) {
                const int code = __ldg(scales + i);
                most = max(most, code == 255 ? 0 : code);
            }
        };
        look(0, min(s1, w0));
        look(w0, w1);
        most = __reduce_max_sync(0xffffffffu, most);
        __syncthreads();
        if ((tid & 31) == 0) most_of[tid >> 5] = most;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kPrepThreads / 32; ++w) most = max(most, most_of[w]);
        return most;
    };
    const int k_ref = largest(p.k_scale);
    if (blockIdx.x == 0 && h == hk * p.g.group) {
        const int v_ref = largest(p.v_scale);
        if (tid == 0) {
            p.refs[2 * (b * p.g.heads_kv + hk)] = k_ref;
            p.refs[2 * (b * p.g.heads_kv + hk) + 1] = v_ref;
        }
    }
    float x[16];
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t w = reinterpret_cast<const uint32_t*>(v)[i];
        const float2 f = F16 ? f16x2_to_f32x2(w) : make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
        const uint32_t lo = __float_as_uint(f.x) & 0x7fffffffu, hi = __float_as_uint(f.y) & 0x7fffffffu;
        most = max(most, max(lo < 0x7f800000u ? lo : 0u, hi < 0x7f800000u ? hi : 0u));
    }
#pragma unroll
    for (int o = 1; o < LANES; o *= 2) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
    const int code = scale_code(most);
    const float up = scale_of(254 - code);
    if (row < p.g.N) {
        uint32_t piece[3][4] = {};
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            // (plus x times zero: NaN where x is infinite, as its products would be)
            float a = fmaf(x[i], 0.f, x[i] * up), b2 = fmaf(x[i + 1], 0.f, x[i + 1] * up);
            const uint32_t p0 = f32x2_to_e4m3x2(a, b2);
            const float2 f0 = f16x2_to_f32x2(e4m3x2_to_f16x2(p0));
            a -= f0.x;
            b2 -= f0.y;
            const uint32_t p1 = f32x2_to_e5m2x2(a, b2);
            piece[0][i / 4] |= p0 << (i & 2) * 8;
            piece[1][i / 4] |= p1 << (i & 2) * 8;
            if (F16) {
                const float2 f1 = e5m2x2_to_f32x2(p1);
                piece[2][i / 4] |= f32x2_to_e5m2x2(a - f1.x, b2 - f1.y) << (i & 2) * 8;
            }
        }
#pragma unroll
        for (int i = 0; i < (F16 ? 3 : 2); ++i)
            *reinterpret_cast<uint4*>(p.Q8 + ((((long long)i * p.g.batch + b) * p.g.heads + h) * p.g.N + row) * D + c) =
                make_uint4(piece[i][0], piece[i][1], piece[i][2], piece[i][3]);
    }
    // (never so small that a block's scale times it is zero, nor infinite: a hidden score of -inf, or a product of zero, times it stays what it is.  A
    // product is 2^25 at most, so that scores are off by 2^-35 at most where the smallest factor is raised.)
    if (c == 0 && row < p.g.N)
        p.c2[((long long)b * p.g.heads + h) * p.g.N + row] = fminf(fmaxf(ldexpf(p.scale_log2 * scale_of(code), k_ref - 127), 0x1p-60f), FLT_MAX);
}

// ---- behind: the parts of cut items ----
struct JoinParams {
    WindowGeom g;
    const float* part_O;
    const float2* part_ml;
    const int32_t* refs;  // or NULL
    float shift;
    int parts;
    uint16_t* O;
    long long o_batch, o_head, o_row;
    float* LSE;
};
constexpr int kJoinThreads = 128;

template <int D, bool F16>
__global__ void __launch_bounds__(kJoinThreads) cache_join_kernel(const __grid_constant__ JoinParams p) {
    constexpr int LANES = D / 4, ROWS = kJoinThreads / LANES;  // four channels to a thread
    grid_dependency_wait();
    const long long rows = (long long)p.g.batch * p.g.heads * p.g.N, at = (long long)blockIdx.x * ROWS + threadIdx.x / LANES;
    if (at >= rows) return;
    const int c = threadIdx.x % LANES * 4, n = (int)(at % p.g.N), bh = (int)(at / p.g.N), b = bh / p.g.heads, h = bh - b * p.g.heads;
    const Sequence seq = load_sequence(p.g, b);
    const int pos = seq.start + n;
    const bool seen = pos >= 0 && pos < seq.len;
    float M = -INFINITY, L = 0.f;
    for (int s = 0; s < p.parts; ++s) M = fmaxf(M, p.part_ml[s * rows + at].x);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int s = 0; s < p.parts; ++s) {
        const float2 ml = p.part_ml[s * rows + at];
        if (ml.x == -INFINITY && ml.y == 0.f) continue;  // nothing there, or nothing that counts
        const float f = ml.x == -INFINITY ? 1.f : ex2_approx(ml.x - M);  // (nothing but NaN keeps its sum)
        const float4 x = *reinterpret_cast<const float4*>(p.part_O + (s * rows + at) * D + c);
        L = fmaf(f, ml.y, L);
        o.x = fmaf(f, x.x, o.x);
        o.y = fmaf(f, x.y, o.y);
        o.z = fmaf(f, x.z, o.z);
        o.w = fmaf(f, x.w, o.w);
    }
    const float inv = 1.f / L, unit = p.refs ? scale_of(p.refs[2 * (b * p.g.heads_kv + h / p.g.group) + 1]) : 1.f;  // (one after the other, see above)
    uint16_t* out = p.O + (long long)b * p.o_batch + (long long)h * p.o_head + (long long)n * p.o_row + c;
    *reinterpret_cast<uint2*>(out) = seen ? make_uint2(pack_16x2<F16>(o.x * inv * unit, o.y * inv * unit), pack_16x2<F16>(o.z * inv * unit, o.w * inv * unit)) : make_uint2(0u, 0u);
    if (c == 0) p.LSE[at] = seen ? fmaf(M - p.shift, 0.6931471805599453f, logf(L)) : -INFINITY;
}

// ---- host ----
int64_t up256(int64_t n) { return (n + 255) / 256 * 256; }

// How a call is cut up, and where its workspace has what.
struct Plan {
    int tiles, parts;
    double us;  // about what it takes
    int64_t rows;
    int64_t q8, c2, refs, part_ml, part_O, bytes;  // offsets
};
// Parts of an item: as many as make the call shortest.  In tile times (1.3 us; d = 64: 1.0) every pair of CTAs takes its share of whole items, and an
// item costs about four tiles for its start and end, a cut call eight for the join.  (The host knows no lengths: the tensors' sizes stand for them.)
Plan plan_of(const WindowArgs& a) {
    Plan w = {};
    w.tiles = (a.g.N + kPairRows - 1) / kPairRows;
    w.rows = (int64_t)a.g.batch * a.g.heads * a.g.N;
    const int64_t window = (int64_t)a.g.left + a.g.right + a.g.sinks + kPairRows, keys = window < a.g.N_kv ? window : a.g.N_kv;
    const int64_t items = (int64_t)w.tiles * a.g.batch * a.g.heads, pairs = a.num_sms / 2, tiles = (keys + kWinT - 1) / kWinT;
    const auto cost = [&](int64_t s) { return (items * s + pairs - 1) / pairs * ((tiles + s - 1) / s + 4) + (s > 1 ? 8 : 0); };
    w.parts = 1;
    for (int s = 2; s <= kMaxParts && s * 4 <= tiles && items * s < (1 << 24); ++s)  // (where there are more items parts bring nothing)
        if (cost(s) < cost(w.parts)) w.parts = s;
    w.us = (double)cost(w.parts) * (a.d == 128 ? 1.3 : 1.0);
    int64_t at = 0;
    const auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += up256(bytes);
        return here;
    };
    w.q8 = take(w.rows * a.d * (a.f16 ? 3 : 2));
    w.c2 = take(w.rows * 4);
    w.refs = take((int64_t)a.g.batch * a.g.heads_kv * 8);
    w.part_ml = take(w.parts > 1 ? w.parts * w.rows * 8 : 0);
    w.part_O = take(w.parts > 1 ? w.parts * w.rows * a.d * 4 : 0);
    w.bytes = at;
    return w;
}

template <int D, bool F16, bool FINE>
cudaError_t launch(const WindowArgs& a, const CacheGeom& c, const bsa_view_t& Q, const bsa_view_t& O, float* LSE, uint8_t* ws, cudaStream_t stream) {
    const Plan w = plan_of(a);
    PrepareParams q = {};
    q.g = a.g;
    q.Q = static_cast<const uint16_t*>(Q.data);
    q.q_batch = Q.batch; q.q_head = Q.head; q.q_row = Q.row;
    q.Q8 = ws + w.q8;
    q.c2 = reinterpret_cast<float*>(ws + w.c2);
    q.refs = reinterpret_cast<int32_t*>(ws + w.refs);
    q.k_scale = c.K_scale;
    q.v_scale = c.V_scale;
    q.s_batch = c.s_batch;
    q.s_head = c.s_head;
    q.lg_block = c.lg_block;
    q.scale_log2 = a.scale * 1.4426950408889634f;
    constexpr int ROWS = kPrepThreads / (D / 16);
    cache_prepare_kernel<D, F16><<<dim3((a.g.N + ROWS - 1) / ROWS, a.g.heads, a.g.batch), kPrepThreads, 0, stream>>>(q);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    count_launch();

    using C = Cfg<D, F16>;
    CUtensorMap tq, tk, tv;
    const long long head = (long long)a.g.N * D;
    if (!encode_codes_map(&tq, q.Q8, head * a.g.heads, head, D, a.g.N, a.g.heads, a.g.batch * C::kPieces, D, kWinT) ||
        !encode_codes_map(&tk, c.K, c.k_batch, c.k_head, c.k_row, c.N, c.heads, c.batch, D, 64) ||
        !encode_code_tiles_map(&tv, c.V, c.v_batch, c.v_head, c.v_row, c.N, c.heads, c.batch, D, D / 2, kWinT, 1))
        return cudaErrorInvalidValue;
    Params p = {};
    p.g = a.g;
    p.O = static_cast<uint16_t*>(O.data);
    p.o_batch = O.batch; p.o_head = O.head; p.o_row = O.row;
    p.LSE = LSE;
    p.o_wide = view_is_wide(O, a.g.batch, a.g.heads, a.g.N);
    p.c2 = q.c2;
    p.refs = q.refs;
    p.k_scale = c.K_scale;
    p.v_scale = c.V_scale;
    p.s_batch = c.s_batch;
    p.s_head = c.s_head;
    p.lg_block = c.lg_block;
    p.last_block = c.blocks - 1;
    p.withhold = window_withhold();
    // (a chunk against a longer cache mostly stands at its end, where all items are about as long: neighbours of one head side by side)
    p.order = ItemOrder(w.tiles, 2 * (int64_t)a.g.N <= a.g.N_kv ? 0 : cut_tiles(a.g, w.tiles, kPairRows), a.g.batch * a.g.heads);
    p.heads = Divisor(a.g.heads);
    p.group = Divisor(a.g.group);
    p.items = Divisor(p.order.n_items);
    p.parts = w.parts;
    p.n_all = p.order.n_items * w.parts;
    p.part_O = reinterpret_cast<float*>(ws + w.part_O);
    p.part_ml = reinterpret_cast<float2*>(ws + w.part_ml);
    if ((e = window_status_word(a.device, &p.status)) != cudaSuccess) return e;
    const auto kernel = cache_tiles_kernel<D, F16, FINE>;
    static std::atomic<int> pairs_of[kMaxDevices];  // pairs of CTAs that the GPU holds at once
    int pairs = pairs_of[a.device].load(std::memory_order_relaxed);
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = C::kSmem;
    cfg.stream = stream;
    if (pairs == 0) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem);
        cfg.gridDim = dim3(2);
        if (e == cudaSuccess) e = cudaOccupancyMaxActiveClusters(&pairs, kernel, &cfg);
        if (e != cudaSuccess) return e;
        if (pairs < 1) return cudaErrorInvalidConfiguration;
        pairs_of[a.device].store(pairs, std::memory_order_relaxed);
    }
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cfg.gridDim = dim3(2u * (unsigned)(pairs < p.n_all ? pairs : p.n_all));
    if ((e = cudaLaunchKernelEx(&cfg, kernel, tq, tk, tv, p)) != cudaSuccess) return e;
    count_launch();
    if (w.parts == 1) return cudaSuccess;

    return launch_cache_join(a, w.parts, p.part_O, p.part_ml, p.refs, kShift, O, LSE, stream);
}

}  // namespace

cudaError_t set_cache_tiles_wait_limit(long long cycles) { return cudaMemcpyToSymbol(ptx::g_wait_limit_cycles, &cycles, sizeof cycles); }

cudaError_t launch_cache_join(const WindowArgs& a, int parts, const float* part_O, const float2* part_ml, const int32_t* refs, float shift,
                              const bsa_view_t& O, float* LSE, cudaStream_t stream) {
    JoinParams j = {};
    j.g = a.g;
    j.part_O = part_O;
    j.part_ml = part_ml;
    j.refs = refs;
    j.shift = shift;
    j.parts = parts;
    j.O = static_cast<uint16_t*>(O.data);
    j.o_batch = O.batch; j.o_head = O.head; j.o_row = O.row;
    j.LSE = LSE;
    const int64_t rows = (int64_t)a.g.batch * a.g.heads * a.g.N, per = kJoinThreads / (a.d / 4);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(kJoinThreads);
    cfg.gridDim = dim3((unsigned)((rows + per - 1) / per));
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, a.d == 64 ? (a.f16 ? cache_join_kernel<64, true> : cache_join_kernel<64, false>)
                                                             : (a.f16 ? cache_join_kernel<128, true> : cache_join_kernel<128, false>), j);
    if (e == cudaSuccess) count_launch();
    return e;
}

int64_t cache_tiles_bytes(const WindowArgs& a) { return plan_of(a).bytes; }
int cache_tiles_parts(const WindowArgs& a) { return plan_of(a).parts; }
double cache_tiles_time(const WindowArgs& a) { return plan_of(a).us; }

cudaError_t launch_cache_tiles(const WindowArgs& a, const CacheGeom& c, const bsa_view_t& Q, const bsa_view_t& O, float* LSE, void* workspace, cudaStream_t stream) {
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    const auto of = [&](auto fine) {
        constexpr bool F = decltype(fine)::value;
        return a.d == 64 ? (a.f16 ? launch<64, true, F>(a, c, Q, O, LSE, ws, stream) : launch<64, false, F>(a, c, Q, O, LSE, ws, stream))
                         : (a.f16 ? launch<128, true, F>(a, c, Q, O, LSE, ws, stream) : launch<128, false, F>(a, c, Q, O, LSE, ws, stream));
    };
    return c.lg_block < 6 ? of(std::true_type{}) : of(std::false_type{});
}

}  // namespace bsa
