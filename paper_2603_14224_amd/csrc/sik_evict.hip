// Eviction by accumulated attention weight: the tokens that stay, in ascending order, and the cache cut down to them.
//
// The cut is found by a radix selection on order-preserving keys of 32 bits, in digits of 11, 11 and 10 bits; what stays is
// placed from bit counts, in token order, so the list needs no sort and no atomics decide an order.  Short caches, and longer
// ones in large batches: one workgroup per (sequence, KV head) holds the weights in its registers.  Else three launches of many
// workgroups, a chunk of tokens each: `count` (first digit of every chunk), `collect` (every workgroup adds the chunks' counts
// up, finds the cut's bin and writes its tokens of that bin, a few per cent, behind those of the chunks before), `place` (the
// other two digits from those tokens alone, then the chunk's part of the list).
//
// Bounds: the list, chains of memory, counting and barriers (one row of 65536 weights in 18.5 us, 32 of them in 28; 256 rows of
// 16370 in 22); the rows, memory (2048 rows of K and V for each of 256, 537 MB: 87 us, 6.2 TB/s).
#include "sik_chunk.h"

namespace sik {

constexpr int kEvictBlock = 1024;
constexpr int kDigitBins = 2048;   // of the first two digits; the last one has 1024
constexpr int kChunkTokens = 4096; // the fewest tokens of a chunk
constexpr int kEvictChunks = 64;   // the most chunks of a row, whose counts every workgroup adds up
// Compute units.  A second round of workgroups costs more than longer chunks: 32 rows of 65544 weights in nine chunks of 8192
// take 37 us, in eight of 8256 28.
constexpr int kEvictUnits = 256;
constexpr int kEvictStep = 4096;   // tokens of a workgroup at four weights per thread

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));  // rows start at any multiple of 4 bytes

struct EvictRow {
    int L, lo, hi, need;  // tokens; those between the kept ends; how many of them stay
    __device__ __forceinline__ bool inner(int i) const { return i >= lo && i < hi; }
};
__device__ __forceinline__ EvictRow evict_row(const EvictArgs& a, int b, int Lmax) {
    EvictRow r;
    r.L = min(max(a.seq_len[b], 0), Lmax);
    r.lo = a.n_sink;
    r.hi = r.L - a.n_recent;
    r.need = a.n_keep - a.n_sink - a.n_recent;
    return r;
}

// Counts of `bin` over the lanes that are `on`.  Equal weights (vanished ones above all) would meet in one counter: the lanes
// that share the first lane's bin are counted by one addition.
__device__ __forceinline__ void count_bins(uint32_t* hist, uint32_t bin, bool on) {
    const uint64_t some = __ballot(on);
    if (some == 0) return;
    const int first = __ffsll(static_cast<unsigned long long>(some)) - 1;
    const uint32_t lead = __builtin_amdgcn_readlane(bin, first);
    const bool same = on && bin == lead;
    const uint64_t m = __ballot(same);
    if (on && !same) atomicAdd(&hist[bin], 1u);
    if (static_cast<int>(threadIdx.x & 63) == first) atomicAdd(&hist[lead], static_cast<uint32_t>(__popcll(m)));
}

__device__ __forceinline__ f32x4_any load4(const float* m, int i, int L) {
    if (i + 4 <= L) return *reinterpret_cast<const f32x4_any*>(m + i);
    f32x4_any v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int e = 0; e < 3; ++e)
        if (i + e < L) v[e] = m[i + e];
    return v;
}

// The bin, from the top, in which the need-th token lies, and how many of that bin's tokens are still needed.  Thread t of
// BLOCK holds the counts of bins NB (BLOCK - 1 - t) ..; exactly one thread finds the bin.
template <int BLOCK, int NB>
__device__ __forceinline__ void find_digit(const uint32_t (&c)[NB], uint32_t& digit, uint32_t& need, uint32_t* totals,
                                           uint32_t* found) {
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    uint32_t mine = 0;
#pragma unroll
    for (int i = 0; i < NB; ++i) mine += c[i];
    const uint32_t incl = wave_inclusive_sum(mine);
    if (lane == 63) totals[wv] = incl;
    __syncthreads();
    uint32_t before = incl - mine;
#pragma unroll
    for (int w = 0; w < BLOCK / kWave; ++w) before += w < wv ? totals[w] : 0u;
    if (before < need && need <= before + mine) {
#pragma unroll
        for (int i = NB - 1; i >= 0; --i) {
            if (before < need && need <= before + c[i]) {
                found[0] = NB * (BLOCK - 1 - tid) + i;
                found[1] = need - before;
            }
            before += c[i];
        }
    }
    __syncthreads();
    digit = found[0];
    need = found[1];
}

// Places what stays of four consecutive tokens per lane (from i): `sure` ones, and of those `equal` to the cut the first
// `need`.
// ps, pe: sure and equal tokens before this wavefront's step, advanced by it.
__device__ __forceinline__ void place4(int32_t* keep, int i, const bool (&sure)[4], const bool (&equal)[4], uint32_t need,
                                       uint32_t& ps, uint32_t& pe) {
    uint32_t cs = 0, ce = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        cs += sure[e];
        ce += equal[e];
    }
    if (__ballot((cs | ce) != 0) == 0) return;
    const uint32_t both = wave_inclusive_sum(cs | ce << 16);
    uint32_t s = ps + (both & 0xffffu) - cs, q = pe + (both >> 16) - ce;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (sure[e] || (equal[e] && q < need)) keep[s + min(q, need)] = i + e;
        s += sure[e];
        q += equal[e];
    }
    const uint32_t all = __builtin_amdgcn_readlane(both, 63);
    ps += all & 0xffffu;
    pe += all >> 16;
}

// Sums of two counts over the wavefronts before this one; tot: [waves][2] of LDS.
template <int WAVES>
__device__ __forceinline__ void before_wave(uint32_t a, uint32_t b, uint32_t (*tot)[2], uint32_t& ba, uint32_t& bb) {
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    if (lane == 0) {
        tot[wv][0] = a;
        tot[wv][1] = b;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        ba += w < wv ? tot[w][0] : 0u;
        bb += w < wv ? tot[w][1] : 0u;
    }
}

// ---- one workgroup per row ------------------------------------------------------------------------------
// NV: steps of 256 tokens that a wavefront holds, so kEvictStep NV tokens to a row at most.
template <int NV>
__global__ __launch_bounds__(kEvictBlock) void evict_select_kernel(EvictArgs a, int Hkv, int Lmax) {
    constexpr int kWaves = kEvictBlock / kWave;
    __shared__ uint32_t hist[kDigitBins];
    __shared__ uint32_t totals[kWaves], found[2], s_tot[kWaves][2];
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int u = blockIdx.x, b = u / Hkv;
    const EvictRow r = evict_row(a, b, Lmax);
    const float* m = a.mass + static_cast<int64_t>(u) * Lmax;
    int32_t* keep = a.keep + static_cast<int64_t>(u) * a.n_keep;
    if (a.new_len && u % Hkv == 0 && tid == 0) a.new_len[b] = min(r.L, a.n_keep);
    if (r.L <= a.n_keep) {
        for (int i = tid; i < a.n_keep; i += kEvictBlock) keep[i] = i < r.L ? i : -1;
        return;
    }
    f32x4_any v[NV];  // a wavefront's consecutive tokens, 256 a step
    const int at = wv * (256 * NV) + 4 * lane;
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = load4(m, at + 256 * i, r.L);
    uint32_t cut = 0, need = r.need;
    for (int digit = 0; digit < 3 && r.need > 0; ++digit) {
        const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, above = digit == 1 ? 21 : 10;
        hist[tid] = 0;
        hist[tid + kEvictBlock] = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t key = float_to_key(v[i][e]);
                count_bins(hist, (key >> shift) & (digit == 2 ? 1023u : 2047u),
                           r.inner(at + 256 * i + e) && (digit == 0 || (key >> above) == cut));
            }
        __syncthreads();
        const uint32_t c[2] = {hist[2 * (kEvictBlock - 1 - tid)], hist[2 * (kEvictBlock - 1 - tid) + 1]};
        uint32_t d;
        find_digit<kEvictBlock>(c, d, need, totals, found);
        cut = cut << (digit == 2 ? 10 : 11) | d;
    }
    auto sure_of = [&](int j, float x) { return j < r.L && (!r.inner(j) || (r.need > 0 && float_to_key(x) > cut)); };
    auto equal_of = [&](int j, float x) { return r.need > 0 && r.inner(j) && float_to_key(x) == cut; };
    uint32_t ns = 0, ne = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            ns += __popcll(__ballot(sure_of(at + 256 * i + e, v[i][e])));
            ne += __popcll(__ballot(equal_of(at + 256 * i + e, v[i][e])));
        }
    uint32_t ps = 0, pe = 0;
    before_wave<kWaves>(ns, ne, s_tot, ps, pe);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        bool sure[4], equal[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            sure[e] = sure_of(at + 256 * i + e, v[i][e]);
            equal[e] = equal_of(at + 256 * i + e, v[i][e]);
        }
        place4(keep, at + 256 * i, sure, equal, need, ps, pe);
    }
}

// ---- a workgroup per chunk of `per` tokens -----------------------------------------------------------------
struct EvictScratch {
    uint32_t* counts;  // [unit][chunk][kDigitBins]  first digits
    uint32_t* list;    // [unit][list_len]           keys of the tokens in the cut's bin, in token order
    uint32_t* heads;   // [unit][chunk][4]           of the chunk: its first entry of the list, tokens that surely stay before
                       //                            it; of the row: length of the list, how many of it stay
    uint32_t* bins;    // [unit]                     the cut's bin
    int chunks, per;
    int64_t list_len;
};

// A wavefront's consecutive part of a chunk, [first, last) in steps of 256 tokens, four per lane.  The first two steps are
// requested before anything else is known, lengths included, so that a launch waits for memory once where these are all: a
// step's weights then come from registers however often they are looked at.
struct PartWeights {
    static constexpr int kHeld = 2;
    const float* m;
    int Lmax, lane, start, len, first, last;
    f32x4_any held[kHeld];
    __device__ __forceinline__ PartWeights(const float* mass, int Lmax_, const EvictScratch& w, int c) : m(mass), Lmax(Lmax_) {
        len = w.per / (kEvictBlock / kWave);
        lane = threadIdx.x & 63;
        start = c * w.per + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * len;
#pragma unroll
        for (int k = 0; k < kHeld; ++k) held[k] = load4(m, start + 256 * k + 4 * lane, 256 * k < len ? Lmax : 0);
    }
    __device__ __forceinline__ void end_at(int L) {
        first = min(start, L);
        last = min(start + len, L);
    }
    // f(token, its weight and the three after it), every lane of the wavefront in every step
    template <class F>
    __device__ __forceinline__ void each(F f) const {
#pragma unroll
        for (int k = 0; k < kHeld; ++k)
            if (first + 256 * k < last) f(first + 256 * k + 4 * lane, held[k]);
        for (int i0 = first + 256 * kHeld; i0 < last; i0 += 256) f(i0 + 4 * lane, load4(m, i0 + 4 * lane, Lmax));
    }
};

__global__ __launch_bounds__(kEvictBlock) void evict_count_kernel(EvictArgs a, int Hkv, int Lmax, EvictScratch w) {
    __shared__ uint32_t hist[kDigitBins];
    const int u = blockIdx.x / w.chunks, c = blockIdx.x % w.chunks;
    PartWeights part(a.mass + static_cast<int64_t>(u) * Lmax, Lmax, w, c);
    const EvictRow r = evict_row(a, u / Hkv, Lmax);
    for (int i = threadIdx.x; i < kDigitBins; i += kEvictBlock) hist[i] = 0;
    if (r.L <= a.n_keep || c * w.per >= r.L) return;
    __syncthreads();
    part.end_at(r.L);
    part.each([&](int i, f32x4_any v) {
#pragma unroll
        for (int e = 0; e < 4; ++e) count_bins(hist, float_to_key(v[e]) >> 21, i + e < part.last && r.inner(i + e));
    });
    __syncthreads();
    uint2* out = reinterpret_cast<uint2*>(w.counts + static_cast<int64_t>(blockIdx.x) * kDigitBins);
    out[threadIdx.x] = reinterpret_cast<const uint2*>(hist)[threadIdx.x];
}

__global__ __launch_bounds__(kEvictBlock) void evict_collect_kernel(EvictArgs a, int Hkv, int Lmax, EvictScratch w) {
    constexpr int kWaves = kEvictBlock / kWave;
    __shared__ uint32_t totals[kWaves], found[2], s_before, s_list, s_len, s_tot[kWaves][2];
    const int tid = threadIdx.x, lane = tid & 63;
    const int u = blockIdx.x / w.chunks, c = blockIdx.x % w.chunks;
    // counts of this thread's two bins over all chunks and over those before this one (chunks without tokens have not
    // written theirs)
    const uint32_t* cp = w.counts + static_cast<int64_t>(u) * w.chunks * kDigitBins + 2 * (kEvictBlock - 1 - tid);
    constexpr int kAhead = 8;
    uint2 x[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
        x[k] = k < w.chunks ? *reinterpret_cast<const uint2*>(cp + static_cast<int64_t>(k) * kDigitBins) : make_uint2(0u, 0u);
    PartWeights part(a.mass + static_cast<int64_t>(u) * Lmax, Lmax, w, c);
    const EvictRow r = evict_row(a, u / Hkv, Lmax);
    if (r.L <= a.n_keep || c * w.per >= r.L) return;
    part.end_at(r.L);
    const int used = (r.L + w.per - 1) / w.per;
    uint32_t all[2] = {0u, 0u}, before[2] = {0u, 0u};
    auto add = [&](int k, uint2 y) {
        if (k >= used) return;
        all[0] += y.x, all[1] += y.y;
        if (k < c) before[0] += y.x, before[1] += y.y;
    };
#pragma unroll
    for (int k = 0; k < kAhead; ++k) add(k, x[k]);
#pragma unroll 4
    for (int k = kAhead; k < used; ++k) add(k, *reinterpret_cast<const uint2*>(cp + static_cast<int64_t>(k) * kDigitBins));
    if (tid == 0) s_before = 0;
    uint32_t bin, need = r.need;
    find_digit<kEvictBlock>(all, bin, need, totals, found);
    uint32_t above = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t mine = 2 * (kEvictBlock - 1 - tid) + i;
        if (mine > bin) above += before[i];
        if (mine == bin) {
            s_list = before[i];
            s_len = all[i];
        }
    }
    above = wave_sum(above);
    if (lane == 0 && above) atomicAdd(&s_before, above);
    // the tokens of that bin, in order
    auto in_bin = [&](int i, float v) { return i < part.last && r.inner(i) && float_to_key(v) >> 21 == bin; };
    uint32_t n = 0;
    part.each([&](int i, f32x4_any v) {
#pragma unroll
        for (int e = 0; e < 4; ++e) n += __popcll(__ballot(in_bin(i + e, v[e])));
    });
    uint32_t at = 0, none = 0;
    before_wave<kWaves>(n, 0u, s_tot, at, none);
    at += s_list;
    if (tid == 0) {
        const int cs = c * w.per;  // kept ends in front of the chunk stay as well
        reinterpret_cast<uint4*>(w.heads)[blockIdx.x] =
            make_uint4(s_list, s_before + min(cs, r.lo) + max(0, cs - max(r.hi, r.lo)), s_len, need);
        if (c == 0) w.bins[u] = bin;
    }
    uint32_t* list = w.list + u * w.list_len;
    part.each([&](int i, f32x4_any v) {
        bool in[4];
        uint32_t k = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            in[e] = in_bin(i + e, v[e]);
            k += in[e];
        }
        if (__ballot(k != 0) == 0) return;
        const uint32_t incl = wave_inclusive_sum(k);
        uint32_t p = at + incl - k;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (in[e]) list[p++] = float_to_key(v[e]);
        at += __builtin_amdgcn_readlane(incl, 63);
    });
}

__global__ __launch_bounds__(kEvictBlock) void evict_place_kernel(EvictArgs a, int Hkv, int Lmax, EvictScratch w) {
    constexpr int kWaves = kEvictBlock / kWave, kListed = 4;
    __shared__ uint32_t hist[kDigitBins];
    __shared__ uint32_t totals[kWaves], found[2], s_sure, s_equal, s_tot[kWaves][2];
    const int tid = threadIdx.x, lane = tid & 63;
    const int u = blockIdx.x / w.chunks, c = blockIdx.x % w.chunks, cs = c * w.per;
    const bool any = a.n_sink + a.n_recent < a.n_keep;
    // the front of the list, long enough for most rows, is requested with the weights (what lies behind its end is not used)
    const uint32_t* list = w.list + u * w.list_len;
    uint32_t listed[kListed];
#pragma unroll
    for (int k = 0; k < kListed; ++k) listed[k] = any && k * kEvictBlock + tid < w.list_len ? list[k * kEvictBlock + tid] : 0u;
    uint4 hd = make_uint4(0u, 0u, 0u, 0u);
    uint32_t cut = 0;
    if (any) {
        hd = reinterpret_cast<const uint4*>(w.heads)[blockIdx.x];
        cut = w.bins[u];
    }
    PartWeights part(a.mass + static_cast<int64_t>(u) * Lmax, Lmax, w, c);
    const EvictRow r = evict_row(a, u / Hkv, Lmax);
    int32_t* keep = a.keep + static_cast<int64_t>(u) * a.n_keep;
    if (a.new_len && u % Hkv == 0 && c == 0 && tid == 0) a.new_len[u / Hkv] = min(r.L, a.n_keep);
    if (r.L <= a.n_keep) {
        for (int i = cs + tid; i < min(a.n_keep, cs + w.per); i += kEvictBlock) keep[i] = i < r.L ? i : -1;
        return;
    }
    if (cs >= r.L) return;
    part.end_at(r.L);
    uint32_t need = hd.w, sure0 = hd.y, equal0 = 0;
    if (any) {
        const uint32_t mine = hd.x, len = hd.z;
        auto each = [&](uint32_t n, auto f) {  // f(key, place < n), every lane of the wavefront in every step
#pragma unroll
            for (uint32_t k = 0; k < kListed; ++k)
                if (k * kEvictBlock < n) f(listed[k], k * kEvictBlock + tid < n);
            for (uint32_t p = kListed * kEvictBlock; p < n; p += kEvictBlock) f(p + tid < n ? list[p + tid] : 0u, p + tid < n);
        };
        if (tid == 0) s_sure = s_equal = 0;
        for (int digit = 1; digit < 3; ++digit) {
            hist[tid] = hist[tid + kEvictBlock] = 0;
            __syncthreads();
            each(len, [&](uint32_t key, bool on) {
                count_bins(hist, digit == 1 ? (key >> 10) & 2047u : key & 1023u, on && (digit == 1 || key >> 10 == cut));
            });
            __syncthreads();
            const uint32_t x[2] = {hist[2 * (kEvictBlock - 1 - tid)], hist[2 * (kEvictBlock - 1 - tid) + 1]};
            uint32_t d;
            find_digit<kEvictBlock>(x, d, need, totals, found);
            cut = cut << (digit == 1 ? 11 : 10) | d;
        }
        uint32_t ns = 0, ne = 0;  // of the list's tokens in front of the chunk
        each(mine, [&](uint32_t key, bool on) {
            ns += on && key > cut;
            ne += on && key == cut;
        });
        ns = wave_sum(ns);
        ne = wave_sum(ne);
        if (lane == 0 && (ns | ne)) {
            atomicAdd(&s_sure, ns);
            atomicAdd(&s_equal, ne);
        }
        __syncthreads();
        sure0 += s_sure;
        equal0 = s_equal;
    } else {
        sure0 = min(cs, r.lo) + max(0, cs - max(r.hi, r.lo));
    }
    auto sure_of = [&](int i, float v) { return i < part.last && (!r.inner(i) || (any && float_to_key(v) > cut)); };
    auto equal_of = [&](int i, float v) { return any && i < part.last && r.inner(i) && float_to_key(v) == cut; };
    uint32_t ns = 0, ne = 0;
    part.each([&](int i, f32x4_any v) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            ns += __popcll(__ballot(sure_of(i + e, v[e])));
            ne += __popcll(__ballot(equal_of(i + e, v[e])));
        }
    });
    uint32_t ps = sure0, pe = equal0;
    before_wave<kWaves>(ns, ne, s_tot, ps, pe);
    part.each([&](int i, f32x4_any v) {
        bool sure[4], equal[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            sure[e] = sure_of(i + e, v[e]);
            equal[e] = equal_of(i + e, v[e]);
        }
        place4(keep, i, sure, equal, need, ps, pe);
    });
}

// 16 lanes copy a kept row of K and of V, kRowsEach of them, all requested before the first is stored.
constexpr int kRowsEach = 2;
__global__ __launch_bounds__(kBlock) void evict_rows_kernel(EvictArgs a, CacheView cv, int nblk) {
    const int p = threadIdx.x & 15;
    const int u = blockIdx.x / nblk, b = u / cv.Hkv, h = u % cv.Hkv;
    const int i0 = (blockIdx.x % nblk) * (kBlock / 16 * kRowsEach) + (threadIdx.x >> 4);
    int j[kRowsEach];
    int64_t from[kRowsEach];
    uint4 k[kRowsEach], v[kRowsEach];
#pragma unroll
    for (int x = 0; x < kRowsEach; ++x) {
        const int i = i0 + x * (kBlock / 16);
        j[x] = i < a.n_keep ? a.keep[static_cast<int64_t>(u) * a.n_keep + i] : -1;
    }
#pragma unroll
    for (int x = 0; x < kRowsEach; ++x) {
        from[x] = j[x] < 0 || !a.K_out ? -1 : cache_row(cv, b, h, j[x]);
        k[x] = v[x] = make_uint4(0u, 0u, 0u, 0u);
        if (from[x] >= 0) {
            k[x] = ld_stream(reinterpret_cast<const uint4*>(a.K + from[x] * kD) + p);
            v[x] = ld_stream(reinterpret_cast<const uint4*>(a.V + from[x] * kD) + p);
        }
    }
#pragma unroll
    for (int x = 0; x < kRowsEach; ++x) {
        if (j[x] < 0) continue;
        const int64_t to = static_cast<int64_t>(u) * a.out_len + i0 + x * (kBlock / 16);
        if (a.mass_out && p == 0) a.mass_out[to] = a.mass[static_cast<int64_t>(u) * cv.Lmax + j[x]];
        if (!a.K_out) continue;
        reinterpret_cast<uint4*>(a.K_out + to * kD)[p] = k[x];
        reinterpret_cast<uint4*>(a.V_out + to * kD)[p] = v[x];
    }
}

// One workgroup per row up to 12288 tokens, up to 32768 from as many rows on as the chip has no room to split (us against the
// three launches): 12000 tokens, 1 row 16.0 / 16.4, 256 rows 19.4 / 29.4; 16370, 1 row 19.7 / 16.6, 64 rows 21.2 / 19.3, 128
// rows 22.1 / 23.2, 256 rows 24.1 / 35.6; 20000, 64 rows 25.4 / 23.1, 128 rows 26.8 / 29.2; 24000, 64 rows 29.7 / 23.5, 128 rows
// 31.5 / 29.6, 192 rows 32.4 / 44.6; 32000, 128 rows 41.8 / 35.4, 192 rows 43.0 / 57.4.
static bool evict_direct(const Dims& d) {
    const int steps = (d.Lmax + kEvictStep - 1) / kEvictStep;
    return steps <= 3 || (steps <= 8 && d.units() >= (steps <= 5 ? 64 : steps <= 6 ? 128 : 192));
}

static EvictScratch evict_plan(const Dims& d, void* ws, size_t* bytes) {
    EvictScratch w{};
    if (!evict_direct(d)) {
        const int by_units = kEvictUnits / d.units(), by_len = (d.Lmax + kChunkTokens - 1) / kChunkTokens;
        w.chunks = by_units < 1 ? 1 : by_units < kEvictChunks ? by_units : kEvictChunks;
        if (w.chunks > by_len) w.chunks = by_len;
        w.per = ((d.Lmax + w.chunks - 1) / w.chunks + 63) / 64 * 64;  // four tokens to a lane of each of 16 wavefronts
        w.chunks = (d.Lmax + w.per - 1) / w.per;
    }
    w.list_len = d.Lmax;
    const int64_t units = d.units(), rows = units * w.chunks;
    uint32_t* p = static_cast<uint32_t*>(ws);
    w.counts = p;
    w.heads = w.counts + rows * kDigitBins;  // (16-byte entries behind a multiple of 8 KB)
    w.bins = w.heads + rows * 4;
    w.list = w.bins + units;
    *bytes = w.chunks ? static_cast<size_t>(rows * (kDigitBins + 4) + units + units * w.list_len) * 4 : 0;
    return w;
}

size_t evict_bytes(const Dims& d) {
    size_t n;
    evict_plan(d, nullptr, &n);
    return n;
}

hipError_t launch_evict(const Dims& d, const CacheView& c, const EvictArgs& a, void* ws, hipStream_t s) {
    size_t bytes;
    const EvictScratch w = evict_plan(d, ws, &bytes);
    const int nblk = (a.n_keep + kBlock / 16 * kRowsEach - 1) / (kBlock / 16 * kRowsEach);
    const bool rows = a.K_out || a.mass_out;
    const int64_t chunks = static_cast<int64_t>(w.chunks) * d.units();
    if (chunks > 0x7fffffff / kEvictBlock || d.units() > 0x7fffffff / kEvictBlock ||
        (rows && static_cast<int64_t>(nblk) * d.units() > 0x7fffffff / kBlock))
        return hipErrorInvalidConfiguration;
    hipError_t e;
    if (w.chunks == 0) {
        auto select = [&](auto kernel) { return launch_kernel(kernel, d.units(), kEvictBlock, s, a, d.Hkv, d.Lmax); };
        switch ((d.Lmax + kEvictStep - 1) / kEvictStep) {
            case 1: e = select(evict_select_kernel<1>); break;
            case 2: e = select(evict_select_kernel<2>); break;
            case 3: e = select(evict_select_kernel<3>); break;
            case 4: e = select(evict_select_kernel<4>); break;
            case 5: e = select(evict_select_kernel<5>); break;
            case 6: e = select(evict_select_kernel<6>); break;
            default: e = select(evict_select_kernel<8>);
        }
    } else {
        const int grid = static_cast<int>(chunks);
        e = hipSuccess;
        if (a.n_sink + a.n_recent < a.n_keep) {
            e = launch_kernel(evict_count_kernel, grid, kEvictBlock, s, a, d.Hkv, d.Lmax, w);
            if (e == hipSuccess) e = launch_kernel(evict_collect_kernel, grid, kEvictBlock, s, a, d.Hkv, d.Lmax, w);
        }
        if (e == hipSuccess) e = launch_kernel(evict_place_kernel, grid, kEvictBlock, s, a, d.Hkv, d.Lmax, w);
    }
    if (e != hipSuccess || !rows) return e;
    return launch_kernel(evict_rows_kernel, nblk * d.units(), kBlock, s, a, c, nblk);
}

}  // namespace sik
