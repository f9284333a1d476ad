// Attention weight that each cached token receives from the last queries of a chunk.
//
// A wavefront owns 32 tokens: their keys stay in its registers as the second operand, the queries pass by as the first, 32
// rows at a time through LDS (three tiles ahead, shared by the eight wavefronts of a workgroup).  A lane then has one token
// (column l % 32) and half of the tile's queries in its registers, so the weights are summed in the lane: no exchange, no
// atomics, one order of additions.  Rows as in chunk attention: token t of the chunk and head r of the group are row t R + r.
//
// Bounds: one query per sequence, the keys (8 x 16384 tokens of 8 KV heads, 276 MB: 50 us, 5.5 TB/s; 66 over changing tensors);
// many, products and exponentials (256 queries of 32 heads on 32768 tokens: 90 us, 760 TFLOP/s; matrix units busy a third of the
// time, vector units half).  Eight wavefronts to a workgroup, not four: a tile's load is one instruction to each of them (these
// two took 8 and 3 % longer with four; 100 queries on 8000 tokens of 4 x 8 heads with 5:1 12 %).
#include "sik_mma.h"

namespace sik {

constexpr int kMassFull = 160;   // halves of workgroups, 128 tokens each, below which four wavefronts share 32 tokens
constexpr int kMassBlock = 512, kMassKeys = kMassBlock / kWave * 32;  // threads and tokens of a workgroup
constexpr int kMassRows = 32;    // query rows of a tile
constexpr int kMassBuffers = 4;  // tiles in LDS
constexpr int kMassStage = 512;  // rows whose sums are in LDS at a time

struct MassArgs {
    const uint16_t *q, *K;
    const float* lse;
    CacheView cv;
    ChunkView ch;
    int Hq, R, blocks, n_obs;
    float scale_log2e;
    const float* before;
    float* mass;
};

template <int DT>
__global__ __launch_bounds__(kMassBlock, 4) void mass_kernel(const MassArgs a) {
    __shared__ struct {
        __align__(16) char q[kMassBuffers][kMassRows * 256];
        __align__(16) float lse[kMassStage];  // in powers of two; +infinity: the row contributes nothing
        __align__(16) int last[kMassStage];   // last token that the row attends
    } lds;
    const int lane = threadIdx.x & 63, wv = uniform(threadIdx.x >> 6);
    const int u = blockIdx.x / a.blocks, b = u / a.cv.Hkv, h = u % a.cv.Hkv;
    const int key0 = (blockIdx.x % a.blocks) * kMassKeys;
    const int past = chunk_past(a.ch, b, a.cv.Lmax), nn = chunk_new(a.ch, b, past, a.cv.Lmax);
    const int end = past + nn;
    if (key0 >= end) return;

    const int key = key0 + 32 * wv + (lane & 31);
    const int64_t krow = cache_row(a.cv, b, h, min(key, end - 1));
    u32x4 kf[8];
#pragma unroll
    for (int step = 0; step < 8; ++step)
        kf[step] = krow < 0 ? u32x4{0u, 0u, 0u, 0u}
                            : *reinterpret_cast<const u32x4*>(a.K + krow * kD + 16 * step + 8 * (lane >> 5));

    // rows of the queries that count and attend a token of this workgroup
    const int t_begin = max(max(nn - a.n_obs, 0), key0 - past);
    const int m0 = t_begin * a.R, rows = nn * a.R;
    const int tiles = t_begin < nn ? (rows - m0 + kMassRows - 1) / kMassRows : 0;
    const int64_t chunk_row = static_cast<int64_t>(b) * a.ch.n;
    // (token, head) of the next tile's first row and of this lane's row of its load; 32 rows on is a fixed step with at most one
    // carry, no division
    const int step_t = kMassRows / a.R, step_r = kMassRows % a.R, row = 4 * wv + (lane >> 4);
    const uint32_t piece = ((lane & 15) ^ key_swizzle(row)) << 4;
    int ft = t_begin, fr = 0, lt = t_begin + row / a.R, lr = row % a.R;
    auto advance = [&](int& t, int& r) {
        t += step_t;
        r += step_r;
        if (r >= a.R) {
            r -= a.R;
            ++t;
        }
    };
    // where R divides 32, the rows of every full tile lie alike behind its first one
    const int behind = lt - t_begin;
    const uint32_t alike = (static_cast<uint32_t>(behind) * a.Hq + lr) * 256u + piece;
    auto load = [&](int tile) {
        const uint16_t* base = dma_base(uniform(a.q + ((chunk_row + ft) * a.Hq + h * a.R) * kD));
        uint32_t off = alike;
        if (step_r != 0 || (tile + 1) * kMassRows > rows - m0) {
            if (step_r == 0) lt = ft + behind;
            const bool in = lt < nn;  // rows beyond the end repeat the last one
            off = (static_cast<uint32_t>((in ? lt : nn - 1) - ft) * a.Hq + (in ? lr : a.R - 1)) * 256u + piece;
            advance(lt, lr);
        }
        dma_16(base, off, uniform(static_cast<int>(lds_offset(lds.q[tile % kMassBuffers]) + 4 * wv * 256)));
        advance(ft, fr);
    };
    auto stage = [&](int tile) {  // sums and last tokens of the next kMassStage rows
        for (int i = threadIdx.x; i < kMassStage; i += kMassBlock) {
            const int m = m0 + tile * kMassRows + i, t = m / a.R;
            float l = __builtin_inff();
            if (m < rows) {
                const float x = a.lse[(chunk_row + t) * a.Hq + h * a.R + (m - t * a.R)];
                if (x > -__builtin_inff()) l = x * 1.4426950408889634f;
            }
            lds.lse[i] = l;
            lds.last[i] = past + t;
        }
    };
    float sum = 0.0f;
    int first_t = t_begin, first_r = 0;
#pragma unroll
    for (int i = 0; i < kMassBuffers - 1; ++i)
        if (i < tiles) load(i);
    arrived(kf);
    for (int tile = 0; tile < tiles; ++tile) {
        const int row0 = (tile * kMassRows) % kMassStage;
        if (row0 == 0) {
            if (tile) __syncthreads();  // the sums staged before have been read
            stage(tile);
        }
        if (tile + kMassBuffers - 1 <= tiles)  // two newer tiles are on their way, a load each
            dma_wait<kMassBuffers - 2>();
        else
            dma_wait<0>();
        lds_reads_done();
        barrier_only();
        if (tile + kMassBuffers - 1 < tiles) load(tile + kMassBuffers - 1);
        const char* qt = lds.q[tile % kMassBuffers];
        f32x16 s{};
#pragma unroll
        for (int step = 0; step < 8; ++step) s = mma32<DT>(row_fragment(qt, lane, step), kf[step], s);
        const int at = row0 + 4 * (lane >> 5);
        if (key0 + 32 * wv + 31 > past + first_t) {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int4 x = *reinterpret_cast<const int4*>(&lds.last[at + 8 * g]);
                s[4 * g] = key > x.x ? -__builtin_inff() : s[4 * g];
                s[4 * g + 1] = key > x.y ? -__builtin_inff() : s[4 * g + 1];
                s[4 * g + 2] = key > x.z ? -__builtin_inff() : s[4 * g + 2];
                s[4 * g + 3] = key > x.w ? -__builtin_inff() : s[4 * g + 3];
            }
        }
        float part = 0.0f;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const float4 x = *reinterpret_cast<const float4*>(&lds.lse[at + 8 * g]);
            part += (fast_exp2(fmaf(s[4 * g], a.scale_log2e, -x.x)) + fast_exp2(fmaf(s[4 * g + 1], a.scale_log2e, -x.y))) +
                    (fast_exp2(fmaf(s[4 * g + 2], a.scale_log2e, -x.z)) + fast_exp2(fmaf(s[4 * g + 3], a.scale_log2e, -x.w)));
        }
        sum += part;
        advance(first_t, first_r);
    }
    float lo, hi;
    both_halves(sum, lo, hi);
    sum = krow < 0 ? 0.0f : lo + hi;
    if (lane < 32 && key < end) {
        const int64_t at = static_cast<int64_t>(u) * a.cv.Lmax + key;
        a.mass[at] = (a.before ? a.before[at] : 0.0f) + sum;
    }
}

// The same where there are too few tokens for the chip: the four wavefronts of a workgroup share 32 tokens and take every
// fourth tile of queries each, through LDS of their own without a barrier; their sums are added in a fixed order at the end.
template <int DT>
__global__ __launch_bounds__(kBlock, 2) void mass_split_kernel(const MassArgs a) {
    __shared__ struct {
        __align__(16) char q[4][2][kMassRows * 256];
        __align__(16) float lse[4][kMassRows];
        __align__(16) int last[4][kMassRows];
        float sum[4][32];
    } lds;
    const int lane = threadIdx.x & 63, wv = uniform(threadIdx.x >> 6);
    const int u = blockIdx.x / a.blocks, b = u / a.cv.Hkv, h = u % a.cv.Hkv;
    const int key0 = (blockIdx.x % a.blocks) * 32;
    const int past = chunk_past(a.ch, b, a.cv.Lmax), nn = chunk_new(a.ch, b, past, a.cv.Lmax);
    const int end = past + nn;
    if (key0 >= end) return;
    const int key = key0 + (lane & 31);
    const int64_t krow = cache_row(a.cv, b, h, min(key, end - 1));
    u32x4 kf[8];
#pragma unroll
    for (int step = 0; step < 8; ++step)
        kf[step] = krow < 0 ? u32x4{0u, 0u, 0u, 0u}
                            : *reinterpret_cast<const u32x4*>(a.K + krow * kD + 16 * step + 8 * (lane >> 5));
    const int t_begin = max(max(nn - a.n_obs, 0), key0 - past);
    const int m0 = t_begin * a.R, rows = nn * a.R;
    const int tiles = t_begin < nn ? (rows - m0 + kMassRows - 1) / kMassRows : 0;
    const int64_t chunk_row = static_cast<int64_t>(b) * a.ch.n;
    auto load = [&](int tile, int buf, float& l, int& last) {
        const int first = m0 + tile * kMassRows, t_first = first / a.R;
        const uint16_t* base = dma_base(uniform(a.q + ((chunk_row + t_first) * a.Hq + h * a.R) * kD));
        if (lane < kMassRows) {
            const int m = first + lane, t = m / a.R;
            l = __builtin_inff();
            last = past + t;
            if (m < rows) {
                const float x = a.lse[(chunk_row + t) * a.Hq + h * a.R + (m - t * a.R)];
                if (x > -__builtin_inff()) l = x * 1.4426950408889634f;
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = 4 * i + (lane >> 4), m = min(first + r, rows - 1), t = m / a.R;
            const uint32_t off = (static_cast<uint32_t>(t - t_first) * a.Hq + (m - t * a.R)) * 256u;
            dma_16(base, off + (((lane & 15) ^ key_swizzle(r)) << 4),
                   uniform(static_cast<int>(lds_offset(lds.q[wv][buf]) + 4 * i * 256)));
        }
    };
    float l = 0.0f, sum = 0.0f;
    int last = 0, buf = 0;
    if (wv < tiles) load(wv, 0, l, last);
    for (int tile = wv; tile < tiles; tile += 4, buf ^= 1) {
        dma_wait<0>();
        lds_reads_done();
        if (lane < kMassRows) {
            lds.lse[wv][lane] = l;
            lds.last[wv][lane] = last;
        }
        if (tile + 4 < tiles) load(tile + 4, buf ^ 1, l, last);
        const char* qt = lds.q[wv][buf];
        f32x16 s{};
#pragma unroll
        for (int step = 0; step < 8; ++step) s = mma32<DT>(row_fragment(qt, lane, step), kf[step], s);
        const bool mask = key0 + 31 > past + (m0 + tile * kMassRows) / a.R;
        float part = 0.0f;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const float4 x = *reinterpret_cast<const float4*>(&lds.lse[wv][8 * g + 4 * (lane >> 5)]);
            float e[4] = {fmaf(s[4 * g], a.scale_log2e, -x.x), fmaf(s[4 * g + 1], a.scale_log2e, -x.y),
                          fmaf(s[4 * g + 2], a.scale_log2e, -x.z), fmaf(s[4 * g + 3], a.scale_log2e, -x.w)};
            if (mask) {
                const int4 y = *reinterpret_cast<const int4*>(&lds.last[wv][8 * g + 4 * (lane >> 5)]);
                e[0] = key > y.x ? -__builtin_inff() : e[0];
                e[1] = key > y.y ? -__builtin_inff() : e[1];
                e[2] = key > y.z ? -__builtin_inff() : e[2];
                e[3] = key > y.w ? -__builtin_inff() : e[3];
            }
            part += (fast_exp2(e[0]) + fast_exp2(e[1])) + (fast_exp2(e[2]) + fast_exp2(e[3]));
        }
        sum += part;
    }
    float lo, hi;
    both_halves(sum, lo, hi);
    if (lane < 32) lds.sum[wv][lane] = lo + hi;
    __syncthreads();
    if (wv != 0 || lane >= 32 || key >= end) return;
    sum = krow < 0 ? 0.0f : (lds.sum[0][lane] + lds.sum[1][lane]) + (lds.sum[2][lane] + lds.sum[3][lane]);
    const int64_t at = static_cast<int64_t>(u) * a.cv.Lmax + key;
    a.mass[at] = (a.before ? a.before[at] : 0.0f) + sum;
}

hipError_t launch_mass(const Dims& d, const CacheView& c, const ChunkView& ch, const void* q, const void* K, float scale,
                       const float* lse, int n_obs, const float* before, float* mass, hipStream_t s) {
    // shared tokens where workgroups of 256 tokens would leave most compute units idle and there are queries for all four
    // wavefronts.  8 KV heads with 4:1 heads, shared against not: 256 queries on 1264 tokens (80 halves of workgroups) 18 us and
    // 30, on 2264 (144) 28 and 28, on 2764 (176) 31 and 29, on 4264 (272) 42 and 31; 2048 on 2556 (160) 140 and 193, on 3056 (192)
    // 195 and 192.  One KV head, 64 queries on 16072 tokens (126) 7.9 and 11.1, on 20072 (157) 11.7 and 10.7.
    const int64_t wide = (d.Lmax + 127) / 128 * static_cast<int64_t>(d.units());
    const bool split = wide < kMassFull && static_cast<int64_t>(n_obs) * d.R > 2 * kMassRows;
    const int blocks = split ? (d.Lmax + 31) / 32 : (d.Lmax + kMassKeys - 1) / kMassKeys;
    const int64_t grid = static_cast<int64_t>(blocks) * d.units();
    if (grid > 0x7fffffff / kMassBlock || static_cast<int64_t>(ch.n) * d.R > 0x7fffffff - kMassStage)
        return hipErrorInvalidConfiguration;
    const float sl2 = (scale > 0.0f ? scale : 1.0f / sqrtf(static_cast<float>(kD))) * 1.4426950408889634f;
    const MassArgs a{static_cast<const uint16_t*>(q), static_cast<const uint16_t*>(K), lse, c, ch, d.Hq, d.R, blocks, n_obs,
                     sl2, before, mass};
#define SIK_MASS(DTV)                                                                                  \
    split ? launch_kernel(mass_split_kernel<DTV>, static_cast<int>(grid), kBlock, s, a)                 \
          : launch_kernel(mass_kernel<DTV>, static_cast<int>(grid), kMassBlock, s, a)
    return d.kv_dtype == kBF16 ? (SIK_MASS(kBF16)) : (SIK_MASS(kF16));
#undef SIK_MASS
}

}  // namespace sik
