// Eviction by accumulated attention weight: the tokens that stay, in ascending order, and the cache cut down to them.
#include "sik_chunk.h"

namespace sik {

constexpr int kEvictBlock = 1024;

// One workgroup per (sequence, KV head): the threshold key by four passes of 8-bit digits over the weights between the kept
// ends, then one pass in token order that places what is above it and the first ones that equal it.
__global__ __launch_bounds__(kEvictBlock) void evict_select_kernel(EvictArgs a, int Hkv, int Lmax) {
    __shared__ uint32_t hist[256];
    __shared__ uint32_t s_digit, s_need;
    __shared__ uint32_t wsum[2][kEvictBlock / kWave];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int u = blockIdx.x, b = u / Hkv;
    const int L = min(max(a.seq_len[b], 0), Lmax);
    const float* m = a.mass + static_cast<int64_t>(u) * Lmax;
    int32_t* keep = a.keep + static_cast<int64_t>(u) * a.n_keep;
    if (a.new_len && u % Hkv == 0 && tid == 0) a.new_len[b] = min(L, a.n_keep);
    if (L <= a.n_keep) {
        for (int i = tid; i < a.n_keep; i += kEvictBlock) keep[i] = i < L ? i : -1;
        return;
    }
    const int lo = a.n_sink, hi = L - a.n_recent;
    uint32_t need = a.n_keep - a.n_sink - a.n_recent, prefix = 0;
    for (int sh = 24; sh >= 0 && need > 0; sh -= 8) {
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        for (int i = lo + tid; i < hi; i += kEvictBlock) {
            const uint32_t key = float_to_key(m[i]);
            if (sh == 24 || (key >> (sh + 8)) == prefix) atomicAdd(&hist[(key >> sh) & 255], 1u);
        }
        __syncthreads();
        if (tid == 0) {
            uint32_t n = need, dg = 255;
            while (dg > 0 && hist[dg] < n) n -= hist[dg--];
            s_digit = dg;
            s_need = n;
        }
        __syncthreads();
        prefix = prefix << 8 | s_digit;
        need = s_need;
    }
    // prefix: the key at the cut (need > 0 of the tokens that equal it stay)
    const bool any = a.n_keep > a.n_sink + a.n_recent;
    uint32_t placed = 0, equal = 0;
    for (int i0 = 0; i0 < L; i0 += kEvictBlock) {
        const int i = i0 + tid;
        const bool end = i < L && (i < lo || i >= hi);
        const uint32_t key = i < L && !end && any ? float_to_key(m[i]) : 0u;
        const bool mid = i < L && !end && any;
        const bool eq = mid && key == prefix, sure = end || (mid && key > prefix);
        const uint64_t me = __ballot(eq), ms = __ballot(sure), below = (1ull << lane) - 1;
        if (lane == 0) {
            wsum[0][wv] = __popcll(me);
            wsum[1][wv] = __popcll(ms);
        }
        __syncthreads();
        uint32_t e0 = equal, s0 = 0, et = 0, st = 0;
        for (int w = 0; w < kEvictBlock / kWave; ++w) {
            if (w < wv) {
                e0 += wsum[0][w];
                s0 += wsum[1][w];
            }
            et += wsum[0][w];
            st += wsum[1][w];
        }
        const uint32_t e_rank = e0 + __popcll(me & below);
        // kept before this token: the sure ones and as many of the equal ones as still fit
        const uint32_t at = placed + s0 + __popcll(ms & below) + (min(e_rank, need) - min(equal, need));
        if (sure || (eq && e_rank < need)) keep[at] = i;
        placed += st + (min(equal + et, need) - min(equal, need));
        equal += et;
        __syncthreads();
    }
}

// 16 lanes copy one kept row of K and of V.
__global__ __launch_bounds__(kBlock) void evict_rows_kernel(EvictArgs a, CacheView cv, int nblk) {
    const int p = threadIdx.x & 15;
    const int u = blockIdx.x / nblk, b = u / cv.Hkv, h = u % cv.Hkv;
    const int i = (blockIdx.x % nblk) * (kBlock / 16) + (threadIdx.x >> 4);
    if (i >= a.n_keep) return;
    const int j = a.keep[static_cast<int64_t>(u) * a.n_keep + i];
    if (j < 0) return;
    const int64_t to = static_cast<int64_t>(u) * a.out_len + i;
    if (a.mass_out && p == 0) a.mass_out[to] = a.mass[static_cast<int64_t>(u) * cv.Lmax + j];
    if (!a.K_out) return;
    const int64_t from = cache_row(cv, b, h, j);
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
    reinterpret_cast<uint4*>(a.K_out + to * kD)[p] = from < 0 ? zero : reinterpret_cast<const uint4*>(a.K + from * kD)[p];
    reinterpret_cast<uint4*>(a.V_out + to * kD)[p] = from < 0 ? zero : reinterpret_cast<const uint4*>(a.V + from * kD)[p];
}

size_t evict_bytes(const Dims&) { return 0; }

hipError_t launch_evict(const Dims& d, const CacheView& c, const EvictArgs& a, void*, hipStream_t s) {
    hipError_t e = launch_kernel(evict_select_kernel, d.units(), kEvictBlock, s, a, d.Hkv, d.Lmax);
    if (e != hipSuccess || (!a.K_out && !a.mass_out)) return e;
    const int nblk = (a.n_keep + kBlock / 16 - 1) / (kBlock / 16);
    if (static_cast<int64_t>(nblk) * d.units() > 0x7fffffff / kBlock) return hipErrorInvalidConfiguration;
    return launch_kernel(evict_rows_kernel, nblk * d.units(), kBlock, s, a, c, nblk);
}

}  // namespace sik
