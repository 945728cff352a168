// The 8-bit cache: codes, scales, and what its kernels share.
//
// An element is an e4m3 number, and the elements of a block of tokens of one head share a scale 2^(s - 127), s an unsigned byte
// (e8m0; 255: NaN).  e4m3 is a floating type, so a scale between two powers of two would gain no precision; powers of two make
// quantising one rounding, a growing scale a shift of the exponents of what is there already (exact above e4m3's subnormals), and
// reading back exact.
#pragma once
#include "bsa_window.cuh"

namespace bsa {

// Two e4m3 numbers as halves (exact).
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t two) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((unsigned short)two));
    return r;
}
// Four: the pairs of the lower and of the upper half.
__device__ __forceinline__ void e4m3x4_to_f16x4(uint32_t four, uint32_t& lo, uint32_t& hi) {
    asm("{\n\t.reg .b16 l, h;\n\t"
        "mov.b32 {l, h}, %2;\n\t"
        "cvt.rn.f16x2.e4m3x2 %0, l;\n\t"
        "cvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
        : "=r"(lo), "=r"(hi)
        : "r"(four));
}
// Nearest e4m3 numbers, ties to even; beyond 448 the largest, NaN stays NaN.
__device__ __forceinline__ uint32_t f32x2_to_e4m3x2(float lo, float hi) {
    unsigned short r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
// 2^(code - 127): an exponent field, but for 0 (2^-127 is subnormal) and 255.
__device__ __forceinline__ float scale_of(int code) {
    return __int_as_float(code == 0 ? 0x00400000 : code == 255 ? 0x7fc00000 : code << 23);
}

// The code of the smallest power of two that takes the finite magnitude with these bits to 448 = 1.75 * 2^8 at most.
__device__ __forceinline__ int scale_code(uint32_t most) { return max((int)(most >> 23) - 8 + ((most & 0x7fffffu) > 0x600000u), 0); }

struct CacheGeom {
    int batch, heads, d, lg_block;
    int N, blocks;  // tokens that fit, blocks of them
    uint8_t *K, *V, *K_scale, *V_scale;
    long long k_batch, k_head, k_row, v_batch, v_head, v_row, s_batch, s_head;
};
// Checks a cache and fills `g` in.
bsa_status_t cache_geom(const bsa_cache_t* c, CacheGeom* g);

// Rows by the tile from the codes (bsa_cache_tiles.cu), the workspace that they need, and about how many us they take.
int64_t cache_tiles_bytes(const WindowArgs& a);
int cache_tiles_parts(const WindowArgs& a);
double cache_tiles_time(const WindowArgs& a);
cudaError_t launch_cache_tiles(const WindowArgs& a, const CacheGeom& c, const bsa_view_t& Q, const bsa_view_t& O, float* LSE, void* workspace,
                               cudaStream_t stream);
// Few rows (bsa_cache_rows.cu), and the workspace that they need.
int64_t cache_rows_bytes(const WindowArgs& a);
int cache_rows_parts(const WindowArgs& a);
cudaError_t launch_cache_rows(const WindowArgs& a, const CacheGeom& c, const bsa_view_t& Q, const bsa_view_t& O, float* LSE, void* workspace,
                              cudaStream_t stream);
// Behind either, where keys were cut into parts: O and LSE from the parts' [parts][batch][heads][N][d] sums, their maxima (log2 domain) and weights' sums
// (bsa_cache_tiles.cu).  The sums count in the scale refs[..][1] of their key head, where refs is given; maxima are `shift` lower than the scores'.
cudaError_t launch_cache_join(const WindowArgs& a, int parts, const float* part_O, const float2* part_ml, const int32_t* refs, float shift,
                              const bsa_view_t& O, float* LSE, cudaStream_t stream);

}  // namespace bsa
