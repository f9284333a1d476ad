// Attention weight that each cached token receives from the last queries of a chunk.
#include "sik_chunk.h"

namespace sik {

// 16 lanes own one token: its key stays in registers while the queries pass, nothing is shared and no sum depends on an order
// of arrival.
template <int DT>
__global__ __launch_bounds__(kBlock) void mass_kernel(const uint16_t* __restrict__ q, const uint16_t* __restrict__ K,
                                                      const float* __restrict__ lse, CacheView cv, ChunkView ch, int Hq,
                                                      int R, int nblk, int n_obs, float scale_log2e,
                                                      const float* before, float* mass) {
    const int lane = threadIdx.x & 63, p = lane & 15;
    const int blk = blockIdx.x % nblk, u = blockIdx.x / nblk, h = u % cv.Hkv, b = u / cv.Hkv;
    const int j = blk * (kBlock / 16) + (threadIdx.x >> 4);
    const int past = chunk_past(ch, b, cv.Lmax), nn = chunk_new(ch, b, past, cv.Lmax);
    if (j >= past + nn) return;
    const int64_t row = cache_row(cv, b, h, j);
    const uint4 k = row < 0 ? make_uint4(0u, 0u, 0u, 0u) : reinterpret_cast<const uint4*>(K + row * kD)[p];
    float sum = 0.0f;
    for (int t = max(max(0, nn - n_obs), j - past); t < nn && row >= 0; ++t) {
        for (int r = 0; r < R; ++r) {
            const int64_t qr = (static_cast<int64_t>(b) * ch.n + t) * Hq + h * R + r;
            const uint4 x = reinterpret_cast<const uint4*>(q + qr * kD)[p];
            float dot = dot2_acc<DT>(x.x, k.x, 0.0f);
            dot = dot2_acc<DT>(x.y, k.y, dot);
            dot = dot2_acc<DT>(x.z, k.z, dot);
            dot = dot2_acc<DT>(x.w, k.w, dot);
            const float l = lse[qr];
            if (l > -1e30f) sum += fast_exp2(fmaf(row16_sum(dot), scale_log2e, -l * 1.4426950408889634f));
        }
    }
    const int64_t at = static_cast<int64_t>(u) * cv.Lmax + j;
    if (p == 0) mass[at] = (before ? before[at] : 0.0f) + sum;
}

hipError_t launch_mass(const Dims& d, const CacheView& c, const ChunkView& ch, const void* q, const void* K, float scale,
                       const float* lse, int n_obs, const float* before, float* mass, hipStream_t s) {
    const int nblk = (d.Lmax + kBlock / 16 - 1) / (kBlock / 16);
    const int64_t grid = static_cast<int64_t>(nblk) * d.units();
    if (grid > 0x7fffffff / kBlock) return hipErrorInvalidConfiguration;
    const float sl2 = (scale > 0.0f ? scale : 1.0f / sqrtf(static_cast<float>(kD))) * 1.4426950408889634f;
#define SIK_MASS(DTV)                                                                                                \
    launch_kernel(mass_kernel<DTV>, static_cast<int>(grid), kBlock, s, static_cast<const uint16_t*>(q),              \
                  static_cast<const uint16_t*>(K), lse, c, ch, d.Hq, d.R, nblk, n_obs, sl2, before, mass)
    return d.kv_dtype == kBF16 ? SIK_MASS(kBF16) : SIK_MASS(kF16);
#undef SIK_MASS
}

}  // namespace sik
