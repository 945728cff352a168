// Attention over a sliding window and a few first tokens: forward for few rows (the next token, a handful of drafted ones, a short chunk).
//
// The same mathematics as the kernel for tiles of rows (bsa_window.cu), but the work is to read the visible keys and values once:
// with R rows per key head (query tokens x heads that share it) there are R multiplications per element read, far below what
// the GPU offers per byte, and a 128-row tile would hold mostly nothing.  So the keys are what is spread over the GPU:
//   * a cluster of C CTAs takes 16 rows of one key head; every warp of it walks its own share of the visible keys with
//     mma.sync.m16n8k16, copies in steps of 4 KB (16 keys at d = 128, 32 at d = 64) by TMA into two rings private to the warp,
//     a slot refilled as soon as it has been read;
//   * the warps' (m, l, O) are joined in shared memory, the CTAs' through distributed shared memory, each CTA writing its
//     share of the columns: one launch, no workspace, no counters, the same bits every time.
// Two CTAs of six warps per SM: 192 KB of copies in flight, and one CTA's start and end beside the other's middle.
// Six sequences of 1111 to 115200 keys, 32 + 8 heads, d = 128, one token: 236 us for 1.37 GB, 5.8 TB/s; four sequences with a window of 1024:
// 7.7 us in a graph (clusters of two instead of eight 10.3; the joins' loads one after the other 8.4).
#include <cuda_bf16.h>
#include <math.h>

#include <atomic>

#include "bsa_window.cuh"

namespace bsa {

using namespace ptx;

namespace {

constexpr int kWarps = 6;
constexpr int kRows = 16;
constexpr int kRing = 8192;  // bytes of a warp's K or V ring
constexpr int kSlot = 4096;
constexpr int kSlots = kRing / kSlot;
constexpr unsigned kAll = 0xffffffffu;
// Half: P, at most one, is computed 2^15 times as large (half ends at 2^16), so that less of it falls below 2^-14.
template <bool F16>
constexpr float kShift = F16 ? 15.0f : 0.0f;

struct RowsParams {
    WindowGeom g;
    const uint16_t* Q;
    uint16_t* O;
    float* LSE;
    long long q_batch, q_head, q_row, o_batch, o_head, o_row;
    float scale_log2;
    int n_rows;  // N * group
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

// MAX_C: most CTAs of the cluster, eight or sixteen (the join's loads are written out).
template <int D, bool F16, int MAX_C>
__global__ void __launch_bounds__(kWarps * 32, 2)
window_rows_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ RowsParams p) {
    constexpr int KS = kSlot / (D * 2);  // keys per step
    constexpr int NT_S = KS / 8, KS_QK = D / 16, KS_PV = KS / 16, NT_O = D / 8;
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
        tma_load_rows(dst, map, bar, key0, hk, b);
    };
    if (lane == 0) {
        for (int i = 0; i < kSlots && first + i < last; ++i) {
            copy_in(sK + i * kSlot, &tmK, bK + i * 8, key_of(first + i));
            if (!(p.withhold && i == 0)) copy_in(sV + i * kSlot, &tmV, bV + i * 8, key_of(first + i));
        }
    }
    // Q fragments (A operand, row-major 16 x 16 per step) of rows gid and gid + 8
    int pos[2];
    uint32_t qa[KS_QK][4];
#pragma unroll
    for (int hi = 0; hi < 2; ++hi) {
        const int r = row0 + gid + 8 * hi;
        const int n = r / p.g.group, h = hk * p.g.group + (r - n * p.g.group);
        const bool ok = r < p.n_rows;
        pos[hi] = ok ? seq.start + n : -1;
        const uint16_t* q = p.Q + (long long)b * p.q_batch + (long long)h * p.q_head + (long long)n * p.q_row;
#pragma unroll
        for (int ks = 0; ks < KS_QK; ++ks) {
            const int c = ks * 16 + 2 * t;
            qa[ks][hi] = ok ? __ldg(reinterpret_cast<const uint32_t*>(q + c)) : 0u;
            qa[ks][2 + hi] = ok ? __ldg(reinterpret_cast<const uint32_t*>(q + c + 8)) : 0u;
        }
    }
    float o[NT_O][4];
#pragma unroll
    for (int n = 0; n < NT_O; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
    float m_lo = -INFINITY, m_hi = -INFINITY, l_lo = 0.f, l_hi = 0.f;  // maxima of the rows, this thread's share of their sums
    const float c2 = p.scale_log2;
    int slot = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int j = first; j < last; ++j) {
        const int key0 = key_of(j);
        const uint32_t cK = sK + slot * kSlot, cV = sV + slot * kSlot;
        ok = mbar_wait_warp(bK + slot * 8, phase, abortp);
        if (!ok) break;
        float s[NT_S][4];
#pragma unroll
        for (int n = 0; n < NT_S; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
#pragma unroll
        for (int np = 0; np < NT_S / 2; ++np) {
#pragma unroll
            for (int ks = 0; ks < KS_QK; ++ks) {
                const int key = np * 16 + ((lane >> 4) << 3) + (lane & 7);
                const int chunk = ks * 2 + ((lane >> 3) & 1);
                uint32_t b0, b1, b2, b3;
                ldmatrix_x4(cK + swz<KS>(key, chunk), b0, b1, b2, b3);
                mma_16816<F16>(s[2 * np], qa[ks][0], qa[ks][1], qa[ks][2], qa[ks][3], b0, b1);
                mma_16816<F16>(s[2 * np + 1], qa[ks][0], qa[ks][1], qa[ks][2], qa[ks][3], b2, b3);
            }
        }
        __syncwarp();  // every lane has read the K slot
        if (lane == 0 && j + kSlots < last) copy_in(cK, &tmK, bK + slot * 8, key_of(j + kSlots));
        const bool full = key0 + KS <= range.all_hi && (key0 >= range.all_lo || key0 + KS <= p.g.sinks);
        ok = mbar_wait_warp(bV + slot * 8, phase, abortp);
        if (!ok) break;
        if (!full) {
            const uint32_t lo_bits = RowView(p.g, seq, pos[0], key0).bits(0), hi_bits = RowView(p.g, seq, pos[1], key0).bits(0);
#pragma unroll
            for (int n = 0; n < NT_S; ++n) {
                const int c = n * 8 + 2 * t;
                if (!((lo_bits >> c) & 1)) s[n][0] = -INFINITY;
                if (!((lo_bits >> c) & 2)) s[n][1] = -INFINITY;
                if (!((hi_bits >> c) & 1)) s[n][2] = -INFINITY;
                if (!((hi_bits >> c) & 2)) s[n][3] = -INFINITY;
            }
            // V rows that no row here sees may hold anything: their weight is zero, which times NaN would not be
            for (int k = lane; k < KS; k += 32) {
                const int key = key0 + k;
                if (key >= range.hi || (key < range.lo && key >= p.g.sinks)) {
#pragma unroll
                    for (int c = 0; c < D / 8; ++c)
                        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(cV + swz<KS>(k, c)), "r"(0) : "memory");
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
        mx_lo *= c2;
        mx_hi *= c2;
        if (__any_sync(kAll, mx_lo > m_lo || mx_hi > m_hi)) {
            mx_lo = fmaxf(mx_lo, __shfl_xor_sync(kAll, mx_lo, 1));
            mx_hi = fmaxf(mx_hi, __shfl_xor_sync(kAll, mx_hi, 1));
            mx_lo = fmaxf(mx_lo, __shfl_xor_sync(kAll, mx_lo, 2));
            mx_hi = fmaxf(mx_hi, __shfl_xor_sync(kAll, mx_hi, 2));
            const float mn_lo = fmaxf(m_lo, mx_lo), mn_hi = fmaxf(m_hi, mx_hi);
            const float a_lo = (m_lo == -INFINITY) ? 0.f : ex2_approx(m_lo - mn_lo);
            const float a_hi = (m_hi == -INFINITY) ? 0.f : ex2_approx(m_hi - mn_hi);
            m_lo = mn_lo;
            m_hi = mn_hi;
            l_lo *= a_lo;
            l_hi *= a_hi;
#pragma unroll
            for (int n = 0; n < NT_O; ++n) {
                o[n][0] *= a_lo;
                o[n][1] *= a_lo;
                o[n][2] *= a_hi;
                o[n][3] *= a_hi;
            }
        }
        const float nm_lo = (m_lo == -INFINITY) ? 0.f : kShift<F16> - m_lo, nm_hi = (m_hi == -INFINITY) ? 0.f : kShift<F16> - m_hi;
        uint32_t pa[KS_PV][4];  // P as the A operand of P V
#pragma unroll
        for (int n = 0; n < NT_S; ++n) {
            const float p0 = ex2_approx(fmaf(s[n][0], c2, nm_lo)), p1 = ex2_approx(fmaf(s[n][1], c2, nm_lo));
            const float p2 = ex2_approx(fmaf(s[n][2], c2, nm_hi)), p3 = ex2_approx(fmaf(s[n][3], c2, nm_hi));
            l_lo += p0 + p1;
            l_hi += p2 + p3;
            pa[n >> 1][(n & 1) * 2 + 0] = pack_16x2<F16>(p0, p1);
            pa[n >> 1][(n & 1) * 2 + 1] = pack_16x2<F16>(p2, p3);
        }
#pragma unroll
        for (int ks = 0; ks < KS_PV; ++ks) {
#pragma unroll
            for (int nd = 0; nd < NT_O / 2; ++nd) {
                const int key = ks * 16 + (((lane >> 3) & 1) << 3) + (lane & 7);
                const int chunk = nd * 2 + (lane >> 4);
                uint32_t b0, b1, b2, b3;
                ldmatrix_x4_trans(cV + swz<KS>(key, chunk), b0, b1, b2, b3);
                mma_16816<F16>(o[2 * nd], pa[ks][0], pa[ks][1], pa[ks][2], pa[ks][3], b0, b1);
                mma_16816<F16>(o[2 * nd + 1], pa[ks][0], pa[ks][1], pa[ks][2], pa[ks][3], b2, b3);
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
    if (t == 0) {
        wm[warp][gid] = m_lo;
        wm[warp][gid + 8] = m_hi;
        wl[warp][gid] = l_lo;
        wl[warp][gid + 8] = l_hi;
    }
    __syncthreads();  // (every warp's ring is idle from here on)
    float M_lo = -INFINITY, M_hi = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        M_lo = fmaxf(M_lo, wm[w][gid]);
        M_hi = fmaxf(M_hi, wm[w][gid + 8]);
    }
    const float f_lo = m_lo == -INFINITY ? 0.f : ex2_approx(m_lo - M_lo), f_hi = m_hi == -INFINITY ? 0.f : ex2_approx(m_hi - M_hi);
    // [warp][row][D]; 16-byte pieces rotated by the row's low bits so that the eight rows of a store fall into different banks
    float* part = reinterpret_cast<float*>(smem) + warp * kRows * D;
#pragma unroll
    for (int n = 0; n < NT_O; ++n) {
        const int c = (n * 8 + 2 * t) ^ (gid << 3);
        *reinterpret_cast<float2*>(part + gid * D + c) = make_float2(o[n][0] * f_lo, o[n][1] * f_lo);
        *reinterpret_cast<float2*>(part + (gid + 8) * D + c) = make_float2(o[n][2] * f_hi, o[n][3] * f_hi);
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
        const int r = i / D, c = (i - r * D) ^ ((r & 7) << 3);  // element i of the stored order is column c
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
            if (c == 0) p.LSE[((long long)b * p.g.heads + h) * p.g.N + n] = any ? fmaf(M - kShift<F16>, 0.6931471805599453f, logf(L)) : -INFINITY;
        }
    }
    if (threadIdx.x == 0 && abort_flag) atomicExch(p.status, (int)BSA_ERR_DEVICE_TIMEOUT);
    if (C > 1) cluster_sync();  // nobody leaves while its shared memory is being read
}

template <int D, bool F16>
cudaError_t launch(const WindowArgs& a, const bsa_view_t& K, const bsa_view_t& V, const RowsParams& p, cudaStream_t stream) {
    constexpr int KS = kSlot / (D * 2), kSmem = kWarps * 2 * kRing;
    CUtensorMap tk, tv;
    if (!encode_view_map(&tk, K, a.g.N_kv, a.g.heads_kv, a.g.batch, D, KS, F16) || !encode_view_map(&tv, V, a.g.N_kv, a.g.heads_kv, a.g.batch, D, KS, F16))
        return cudaErrorInvalidValue;
    const auto kernel = window_rows_kernel<D, F16, 8>, wide_kernel = window_rows_kernel<D, F16, 16>;
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
    // CTAs of a cluster: until the GPU is full (two per SM), and eight at once where a sequence may be long: how the lengths differ
    // is not known here, and smaller shares even the SMs out.  Not more than there are steps for their warps.  Sixteen where eight leave
    // the GPU idle and a warp has 64 steps and more, if all clusters run at once, or if not all of eight would either (this B200 holds 14
    // of sixteen, 33 of eight).  us, eight / sixteen, d = 128, 65536 keys: 1 key head 56 / 31, 8: 59 / 46, 11: 63 / 60, 14: 73 / 75,
    // 16: 85 / 101, 24: 120 / 123, 33: 168 / 171, 36: 199 / 182; four sequences, window 1024, 8.3 / 19.1.  Where the tensors are long and the
    // lengths short sixteen start later (500 of 131072 keys, 9 key heads: 6.5 / 8.2); 30000 of them: 32 / 28.
    const int64_t longest = (int64_t)a.g.left + a.g.right + a.g.sinks + a.g.N;
    const int64_t steps = ((longest < a.g.N_kv ? longest : a.g.N_kv) + KS - 1) / KS;
    const auto idle = [&](int c) { return (int64_t)c * blocks * heads < 2 * a.num_sms; };
    const auto long_shares = [&](int c) { return steps > (int64_t)c * kWarps * 64; };
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

cudaError_t set_window_rows_wait_limit(long long cycles) { return cudaMemcpyToSymbol(ptx::g_wait_limit_cycles, &cycles, sizeof cycles); }

cudaError_t launch_window_rows(const WindowArgs& a, const bsa_view_t& Q, const bsa_view_t& K, const bsa_view_t& V, const bsa_view_t& O,
                               float* LSE, cudaStream_t stream) {
    RowsParams p = {};
    p.g = a.g;
    p.Q = static_cast<const uint16_t*>(Q.data);
    p.O = static_cast<uint16_t*>(O.data);
    p.LSE = LSE;
    p.q_batch = Q.batch; p.q_head = Q.head; p.q_row = Q.row;
    p.o_batch = O.batch; p.o_head = O.head; p.o_row = O.row;
    p.scale_log2 = a.scale * 1.4426950408889634f;
    p.n_rows = a.g.N * a.g.group;
    p.withhold = window_withhold();
    const cudaError_t e = window_status_word(a.device, &p.status);
    if (e != cudaSuccess) return e;
    return a.d == 64 ? (a.f16 ? launch<64, true>(a, K, V, p, stream) : launch<64, false>(a, K, V, p, stream))
                     : (a.f16 ? launch<128, true>(a, K, V, p, stream) : launch<128, false>(a, K, V, p, stream));
}

}  // namespace bsa
