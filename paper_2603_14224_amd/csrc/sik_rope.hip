// Per-head norms of queries and keys with the position rotation in the same pass, keys and values into the cache.
//
// A wavefront takes four head rows of one token per step, 16 lanes of 8 channels to a row; the rows of a token are its query
// heads, then its key heads, then (into a cache) its value heads, which are copied.  A lane needs the channels that its own
// are paired with: the same 16 bytes of another lane, loaded a second time (from the first-level cache) rather than
// exchanged.  The angles of a token are the same for all its heads: a wavefront computes them once, in front of its steps.
//
// Bound by memory: 8192 tokens of 40 rows rotated and 8 copied, 201 MB, in 40 us where the outputs stay in the Infinity Cache
// and in 53 to 57 where they do not (3.5 TB/s; a copy reaches 4.7).  Requests one step ahead (76 us), two steps at a time
// (62), the partners exchanged between lanes (70) and streaming stores on top of these (66 to 72) were all slower there; one
// token takes 3.6 us.
#include "sik_chunk.h"

namespace sik {

// sin and cos of position * freq: the product of 31 and 24 bits is all but exact in 64 bits (exact for positions below 2^29),
// the whole turns go in 64 bits too (in 32 bits a position of a million would be off by 0.06 rad), what is left of a turn
// fits 32.
__device__ __forceinline__ void turn(int position, float freq, float& s, float& c) {
    const double rev = static_cast<double>(position) * static_cast<double>(freq) * 0.15915494309189533577;
    sincospif(2.0f * static_cast<float>(rev - rint(rev)), &s, &c);
}

template <int DT, bool PAIRS>
__global__ __launch_bounds__(kBlock) void rope_kernel(RopeArgs a, CacheView cv, ChunkView ch, int B, int Hq, int steps,
                                                      int waves) {
    const int lane = threadIdx.x & 63, slot = lane >> 4, p = lane & 15;
    const int w = blockIdx.x * (kBlock / kWave) + (threadIdx.x >> 6);  // wavefront: (sequence, token, part of the heads)
    const int part = w % waves, tok = w / waves;
    const int b = tok / ch.n, t = tok % ch.n;
    const int Hkv = cv.Hkv, n_rows = Hq + Hkv + (a.k_out ? 0 : Hkv);
    if (b >= B) return;
    const int past = chunk_past(ch, b, cv.Lmax);
    if (t >= chunk_new(ch, b, past, cv.Lmax)) return;
    const int64_t src = static_cast<int64_t>(b) * ch.n + t;  // token row of the chunk's tensors

    const int half = a.rotary_dim >> 1;
    const bool rotated = 8 * p < a.rotary_dim;
    const bool upper = !PAIRS && 8 * p >= half;                          // second channels of their pairs
    const int po = !rotated ? p : PAIRS ? p : upper ? p - half / 8 : p + half / 8;  // lane with the partners
    float sn[PAIRS ? 4 : 8], cs[PAIRS ? 4 : 8];  // (of rotated channels)
    if (rotated) {
        const int position = a.positions ? a.positions[src] : past + t;
        const float* f = a.inv_freq + (PAIRS ? 4 * p : 8 * (upper ? po : p));
#pragma unroll
        for (int e = 0; e < (PAIRS ? 4 : 8); ++e) turn(position, f[e], sn[e], cs[e]);
    }

    for (int it = 0; it < steps; ++it) {
        const int hr = (part * steps + it) * 4 + slot;
        if (hr >= n_rows) return;
        const bool is_q = hr < Hq, is_v = hr >= Hq + Hkv;
        const int h = is_q ? hr : is_v ? hr - Hq - Hkv : hr - Hq;
        const uint16_t* x = (is_q ? a.q + src * a.q_stride : is_v ? a.v + src * a.v_stride : a.k + src * a.k_stride) +
                            static_cast<int64_t>(h) * kD;
        const uint4 own = reinterpret_cast<const uint4*>(x)[p];
        const uint4 other = reinterpret_cast<const uint4*>(x)[po];
        uint16_t* y;
        if (is_q) {
            y = a.q_out + (src * Hq + h) * kD;
        } else if (a.k_out) {
            y = a.k_out + (src * Hkv + h) * kD;
        } else {
            const int64_t row = cache_row(cv, b, h, past + t);
            y = row < 0 ? nullptr : (is_v ? a.V : a.K) + row * kD;
        }
        uint4 res = own;
        if (!is_v) {
            float xo[8], xp[8];
            widen8<DT>(own, xo);
            widen8<DT>(other, xp);
            const float* wt = is_q ? a.q_weight : a.k_weight;
            if (wt) {
                float ss = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) ss = fmaf(xo[e], xo[e], ss);
                const float r = 1.0f / sqrtf(row16_sum(ss) * (1.0f / kD) + a.eps);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    xo[e] *= r * wt[8 * p + e];
                    xp[e] *= r * wt[8 * po + e];
                }
            }
            float yo[8];
            if (rotated) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if constexpr (PAIRS) {
                        const float s = (e & 1) ? sn[e >> 1] : -sn[e >> 1];
                        yo[e] = fmaf(xo[e], cs[e >> 1], xo[e ^ 1] * s);
                    } else {
                        yo[e] = fmaf(xo[e], cs[e], xp[e] * (upper ? sn[e] : -sn[e]));
                    }
                }
            } else {  // (not by a sine of zero: an infinity has to stay one, and beside its neighbour)
#pragma unroll
                for (int e = 0; e < 8; ++e) yo[e] = xo[e];
            }
            uint32_t o[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = narrow16<DT>(yo[2 * i]) | narrow16<DT>(yo[2 * i + 1]) << 16;
            res = make_uint4(o[0], o[1], o[2], o[3]);
        }
        if (y) reinterpret_cast<uint4*>(y)[p] = res;
    }
}

hipError_t launch_rope(const Dims& d, const CacheView& c, const ChunkView& ch, const RopeArgs& a, bool interleaved,
                       hipStream_t s) {
    const int64_t tokens = static_cast<int64_t>(d.B) * ch.n;
    const int rows = d.Hq + d.Hkv + (a.k_out ? 0 : d.Hkv), groups = (rows + 3) / 4;
    // steps per wavefront: one where there are few tokens (latency), more where the chip is full (the angles are shared)
    int steps = static_cast<int>(tokens * groups / 8192);
    steps = steps < 1 ? 1 : steps > groups ? groups : steps;
    const int waves = (groups + steps - 1) / steps;
    const int64_t blocks = (tokens * waves + kBlock / kWave - 1) / (kBlock / kWave);
    if (blocks > 0x7fffffff / kBlock) return hipErrorInvalidConfiguration;
#define SIK_ROPE(DTV, PV) \
    launch_kernel(rope_kernel<DTV, PV>, static_cast<int>(blocks), kBlock, s, a, c, ch, d.B, d.Hq, steps, waves)
    if (d.kv_dtype == kBF16) return interleaved ? SIK_ROPE(kBF16, true) : SIK_ROPE(kBF16, false);
    return interleaved ? SIK_ROPE(kF16, true) : SIK_ROPE(kF16, false);
#undef SIK_ROPE
}

}  // namespace sik
