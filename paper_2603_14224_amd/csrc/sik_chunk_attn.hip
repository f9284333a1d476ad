// Attention of a chunk of new tokens over a contiguous or paged cache.
#include "sik_attn_core.h"
#include "sik_chunk.h"

namespace sik {

// A workgroup takes one token of the chunk and a block of up to four query heads of one KV head, and walks over the cache.
template <int DT, int ODT>
__global__ __launch_bounds__(kBlock) void chunk_attn_kernel(const uint16_t* __restrict__ q, const uint16_t* __restrict__ K,
                                                            const uint16_t* __restrict__ V, CacheView cv, ChunkView ch,
                                                            int Hq, int R, int nblk, float scale_log2e,
                                                            void* __restrict__ out, float* __restrict__ lse) {
    constexpr int NH = kSharedHeads;
    __shared__ MergeLds<NH> lds;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, p = lane & 15;
    const int blk = blockIdx.x % nblk, u = blockIdx.x / nblk;
    const int h = u % cv.Hkv, tok = u / cv.Hkv, b = tok / ch.n, t = tok % ch.n;
    const int past = chunk_past(ch, b, cv.Lmax);
    if (t >= chunk_new(ch, b, past, cv.Lmax)) return;
    const int nh = min(NH, R - blk * NH);
    const int64_t row0 = static_cast<int64_t>(tok) * Hq + h * R + blk * NH;
    uint4 qraw[NH];
    SoftmaxState st[NH];
#pragma unroll
    for (int x = 0; x < NH; ++x) {
        qraw[x] = x < nh ? reinterpret_cast<const uint4*>(q + (row0 + x) * kD)[p] : make_uint4(0u, 0u, 0u, 0u);
        init_state(st[x]);
    }
    for (int j0 = 0; j0 <= past + t; j0 += 16) {  // 16 tokens lie on one page
        if (((j0 >> 4) & 3) != wv) continue;
        const int64_t at = cache_row(cv, b, h, j0);
        if (at < 0) continue;
        auto fetch = [&](int j) { return j; };
        attend_list_multi<DT, NH>(fetch, min(16, past + t + 1 - j0), 0, 16,
                                  reinterpret_cast<const uint4*>(K + at * kD),
                                  reinterpret_cast<const uint4*>(V + at * kD), qraw, scale_log2e, 16, st);
    }
    workgroup_merge_multi<NH>(st, nh, lds, [&](int x, int d, float M, float l, float o) {
        store_out<ODT>(out, (row0 + x) * kD + d, l > 0.0f ? o / l : 0.0f);
        if (lse && d == 0) lse[row0 + x] = l > 0.0f ? (M + log2f(l)) * 0.6931471805599453f : -__builtin_inff();
    });
}

size_t chunk_attn_bytes(const Dims&, int) { return 0; }

hipError_t launch_chunk_attn(const Dims& d, const CacheView& c, const ChunkView& ch, const void* q, const void* K,
                             const void* V, float scale, void* out, float* lse, void*, hipStream_t s) {
    const int nblk = (d.R + kSharedHeads - 1) / kSharedHeads;
    const int64_t grid = static_cast<int64_t>(d.B) * ch.n * d.Hkv * nblk;
    if (grid > 0x7fffffff / kBlock) return hipErrorInvalidConfiguration;
    const float sl2 = (scale > 0.0f ? scale : 1.0f / sqrtf(static_cast<float>(kD))) * 1.4426950408889634f;
#define SIK_CHUNK(DTV, ODTV)                                                                                       \
    launch_kernel(chunk_attn_kernel<DTV, ODTV>, static_cast<int>(grid), kBlock, s, static_cast<const uint16_t*>(q), \
                  static_cast<const uint16_t*>(K), static_cast<const uint16_t*>(V), c, ch, d.Hq, d.R, nblk, sl2, out, lse)
    if (d.kv_dtype == kBF16) return d.out_dtype == kF32 ? SIK_CHUNK(kBF16, kF32) : SIK_CHUNK(kBF16, kBF16);
    return d.out_dtype == kF32 ? SIK_CHUNK(kF16, kF32) : SIK_CHUNK(kF16, kF16);
#undef SIK_CHUNK
}

}  // namespace sik
