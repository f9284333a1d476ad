// Attention of a chunk of new tokens over a contiguous or paged cache: one pass over the cache with the running maximum and
// sum of a softmax, both products on the matrix units.
//
// The rows that share a KV head's keys are the chunk's tokens times the R query heads of its group; row m is token m / R,
// head m % R.  A wavefront holds 32 of them.  Its logits are computed transposed, S^T = K Q^T, so that a lane has one query
// (column l % 32) and half of the tile's keys in its registers: maximum and sum of a softmax row stay in the lane but for one
// exchange with the lane 32 away, and the weights are already laid out as the second operand of O^T = V^T P^T, whose first
// one the transposing LDS reads deliver in the same order of tokens.  Nothing of the weights goes through LDS.
//
// Two forms.  `rows`: four wavefronts of a workgroup take 128 rows and share tiles of 64 tokens, loaded into LDS one tile
// ahead.  `tokens`: few rows (at most 32 per KV head, a generated token above all); each wavefront takes its own tiles of 32
// tokens, and the four states of a workgroup are joined at the end.  Either form splits the cache over several workgroups
// where there are too few to fill the chip; a second launch joins their states.
//
// Bounds: few rows, memory (one token of 32 heads on 32767 tokens, 134 MB: 23 us and 5 for the join); many, matrix and vector
// instructions in turn at a clock that falls under the load (8192-token prompt of 32 heads 533 to 550 us, 1.00 to 1.03 PFLOP/s;
// 2048 tokens behind 30720 1010 us, 1.05; a plain product of the library 1.2).
#include "sik_attn_core.h"
#include "sik_mma.h"

namespace sik {

constexpr int kRowsTile = 128;   // rows of a workgroup of the `rows` form
constexpr int kTokensTile = 32;  // of the `tokens` form
constexpr int kMaxParts = 128;   // workgroups that share one row tile's cache
// A row's weights are exp2(logit - m).  The reference m moves only when a tile's largest logit leaves a band around it, so that
// the 64 registers of the output are rescaled a few times per pass instead of once per tile.
//   bf16: m is a maximum that was, and moves up when a logit exceeds it by more than kSlack: weights stay below 2^8, and what is
//   far below keeps its 8 bits, as the type has the exponents of binary32.
//   fp16 has few exponents: below 2^-14 a weight is held to 2^-25 only, and where one token outweighs thousands of others by
//   that much (a sink), all of them would vanish from the sum of the values but not from the sum of the weights.  So m lies
//   2^kUnder below the largest logit, and moves down as well, to the largest logit of a tile that is more than 2^kDrop (binary32
//   results: kDropPrec) below: a tile's largest weight is then at least 2^(kUnder - kDrop), and what the tile's 64 tokens lose
//   at the lower end is at most 2^-14 (2^-18) of that one.  At most 2^kDepth down from the highest reference: a row of 2^22 tokens
//   of weights below 2^(15 + kDepth) and values below 2^16 stays within binary32.  The downward moves cost 1 % of a prompt's
//   time (2048 tokens behind 6144, 8/32 heads: 260 us against 257) and 4 % with binary32 results (352 against 340; 366 with
//   kDropPrec 4, 356 with 6).
// Either way the weight of the logit that m was taken from is a power of two, which 16 bits hold exactly: where one token has
// most of a row's weight, that rounds nothing.
constexpr float kSlack = 8.0f, kUnder = 7.0f, kDrop = 12.0f, kDropPrec = 8.0f, kDepth = 60.0f;

struct ChunkAttn {
    const uint16_t *q, *K, *V;
    CacheView cv;
    ChunkView ch;
    int B, Hq, R, tiles, parts;  // row tiles per unit, workgroups per row tile
    float scale_log2e;
    void* out;
    float* lse;
    float* part_o;   // [unit][tile][part] states: `tokens` form [32 rows][kD]; `rows` form [4 wavefronts] register by register
    float* part_ml;  // [unit][tile][part][rows][2]
};

// A wavefront's 32 rows: one query per lane (both halves hold the same), output registers [channel block][16].
struct RowState {
    float m, l;
    float hi;  // fp16: the highest m so far
    f32x16 o[4];
};

__device__ __forceinline__ void init_rows(RowState& st) {
    st.m = st.hi = kNegBig;
    st.l = 0.0f;
#pragma unroll
    for (int c = 0; c < 4; ++c) st.o[c] = f32x16{};
}

// One tile of 32 NK tokens: `keys` are its LDS rows, s its logits.
template <int DT, int NK>
__device__ __forceinline__ void tile_logits(const char* keys, int lane, const u32x4 (&qf)[8], f32x16 (&s)[NK]) {
#pragma unroll
    for (int t = 0; t < NK; ++t) s[t] = f32x16{};
#pragma unroll
    for (int step = 0; step < 8; ++step)
#pragma unroll
        for (int t = 0; t < NK; ++t) s[t] = mma32<DT>(row_fragment(keys + t * 32 * 256, lane, step), qf[step], s[t]);
}

// Logits of tokens beyond `last` (relative to the tile) or of 16-token groups whose bit is not in `mapped` do not count.
template <int NK>
__device__ __forceinline__ void mask_logits(f32x16 (&s)[NK], int lane, int last, uint32_t mapped) {
    const int lim = last - 4 * (lane >> 5);
#pragma unroll
    for (int t = 0; t < NK; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int at = 32 * t + 8 * (i / 4) + i % 4;
            if (at > lim || !((mapped >> (2 * t + i / 8)) & 1u)) s[t][i] = -__builtin_inff();
        }
}

// Largest logit of a tile, in powers of two.
template <int NK>
__device__ __forceinline__ float tile_top(const f32x16 (&s)[NK], float c) {
    float top = s[0][0];
#pragma unroll
    for (int t = 0; t < NK; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, s[t][i]);
    float lo, hi;
    both_halves(top, lo, hi);
    return fmaxf(lo, hi) * c;
}

// Does the row's reference have to move before a tile whose largest logit is top (-infinity: none counts)?
template <int DT, bool PREC>
__device__ __forceinline__ bool has_to_move(const RowState& st, float top) {
    if constexpr (DT != kF16) return top > st.m + kSlack;
    constexpr float low = kUnder - (PREC ? kDropPrec : kDrop);
    return top > st.m + kUnder + kSlack || (top > kNegBig && fmaxf(top, st.hi - kDepth + kUnder) < st.m + low);
}

template <int DT, bool PREC>
__device__ __forceinline__ void rescale(RowState& st, float top) {
    float m = fmaxf(st.m, top);
    if constexpr (DT == kF16) {
        m = top - kUnder;
        m = m > st.m ? m : has_to_move<DT, PREC>(st, top) ? fmaxf(m, st.hi - kDepth) : st.m;
        st.hi = fmaxf(st.hi, m);
    }
    const float f = fast_exp2(st.m - m);
    st.m = m;
    st.l *= f;
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) st.o[b][i] *= f;
}

// A tile's weights as operands, a group of 16 tokens in each.  The matrix units take both operands in the values' type, so a
// weight is rounded to 16 bits, by at most 2^-8 (bf16) or 2^-11 (fp16; below 2^-14 by 2^-25, see the references above) of itself,
// half of its step, up or down.  The sum that divides it is taken before the rounding.  PREC: what the rounding dropped is a second
// operand.  The `rows` form has it for binary32 results only: with 16-bit ones a row is off by about as much through the weights
// as through its own rounding (root mean square over prompts of random rows: bf16 2.2e-3 of the result against 1.65e-3 with
// the second operand, fp16 2.8e-4 against 2.1e-4; a single row can be off by twice as much), and the second operand takes 1.35
// times as long.  The `tokens` form always has it, beside loads that take longer: 8 tokens behind 32760 of 8/32 heads 38.3 us
// against 37.8, 32 x 4 behind 4000 of 8/64 134.2 against 132.9.
template <int NK, bool PREC>
struct Weights {
    u32x4 w[2 * NK], rest[PREC ? 2 * NK : 1];
};
template <int DT, int NK, bool PREC>
__device__ __forceinline__ void tile_weights(RowState& st, const f32x16 (&s)[NK], float c, Weights<NK, PREC>& x) {
    float sum = 0.0f;
#pragma unroll
    for (int t = 0; t < NK; ++t)
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            const float a = fast_exp2(fmaf(s[t][i], c, -st.m)), b = fast_exp2(fmaf(s[t][i + 1], c, -st.m));
            sum += a;
            sum += b;
            const uint32_t p = pack16<DT>(a, b);
            x.w[2 * t + i / 8][(i % 8) / 2] = p;
            if constexpr (PREC)
                x.rest[2 * t + i / 8][(i % 8) / 2] = pack16<DT>(a - widen16<DT>(p & 0xffffu), b - widen16<DT>(p >> 16));
        }
    st.l += sum;
}

template <int DT, int NK, bool PREC>
__device__ __forceinline__ void tile_values(RowState& st, const Weights<NK, PREC>& x, const char* values, int lane) {
#pragma unroll
    for (int g = 0; g < 2 * NK; ++g)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const u32x4 v = value_fragment(values + g * 16 * 256, lane, b);
            st.o[b] = mma32<DT>(v, x.w[g], st.o[b]);
            if constexpr (PREC) st.o[b] = mma32<DT>(v, x.rest[g], st.o[b]);
        }
}

template <int DT>
__device__ __forceinline__ void load_queries(const uint16_t* row, int lane, u32x4 (&qf)[8]) {
#pragma unroll
    for (int step = 0; step < 8; ++step)
        qf[step] = *reinterpret_cast<const u32x4*>(row + 16 * step + 8 * (lane >> 5));
}

template <int ODT>
__device__ __forceinline__ void store4(void* out, size_t at, float a, float b, float c, float d) {
    if constexpr (ODT == kF32)
        *reinterpret_cast<float4*>(static_cast<float*>(out) + at) = make_float4(a, b, c, d);
    else
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(out) + at) = make_uint2(pack16<ODT>(a, b), pack16<ODT>(c, d));
}

__device__ __forceinline__ float log_sum(float m, float l) {
    return l > 0.0f ? (m + log2f(l)) * 0.6931471805599453f : -__builtin_inff();
}

// A workgroup's place in the launch.  Workgroups go to the XCDs in turn and each XCD has a cache of its own: where the units
// divide by 8, a unit's workgroups all go to one XCD, so that its keys and values are read into one cache only.  The row
// tiles with the most tokens in front of them start first.
struct Place {
    int unit, tile, part;
};
__device__ __forceinline__ Place place_of(int idx, int units, int tiles, int parts) {
    const int per = tiles * parts;
    int u, r;
    if ((units & 7) == 0) {
        const int k = idx >> 3;
        u = (k / per) * 8 + (idx & 7);
        r = k % per;
    } else {
        u = idx % units;
        r = idx / units;
    }
    return Place{u, tiles - 1 - r / parts, r % parts};
}

// 16-token groups of a tile: address of the first row of the group that holds token j (uniform), or nullptr.
__device__ __forceinline__ const uint16_t* group_row(const uint16_t* x, int64_t row) {
    return row < 0 ? nullptr : uniform(x + row * kD);
}

template <int DT, int ODT, bool PAGED>
__global__ __launch_bounds__(kBlock, 2) void chunk_rows_kernel(const ChunkAttn a) {
    constexpr int kTile = 64, kSide = kTile * 256, kBuf = 2 * kSide;
    __shared__ struct {
        __align__(16) char tiles[2 * kBuf];  // first: the loads reach the first 64 KB
        int mapped[2][4];
    } shared;
    char* lds = shared.tiles;
    auto& s_mapped = shared.mapped;
    const int lane = threadIdx.x & 63, wv = uniform(threadIdx.x >> 6);
    const Place pl = place_of(blockIdx.x, a.B * a.cv.Hkv, a.tiles, a.parts);
    const int b = pl.unit / a.cv.Hkv, h = pl.unit % a.cv.Hkv;
    const int past = chunk_past(a.ch, b, a.cv.Lmax), nn = chunk_new(a.ch, b, past, a.cv.Lmax);
    const int rows = nn * a.R, r0 = pl.tile * kRowsTile;
    if (r0 >= rows) return;
    const int end = past + (min(r0 + kRowsTile, rows) - 1) / a.R + 1;  // tokens that the last row attends
    const int n_tiles = (end + kTile - 1) / kTile;
    const int t0 = static_cast<int>(static_cast<int64_t>(n_tiles) * pl.part / a.parts);
    const int t1 = static_cast<int>(static_cast<int64_t>(n_tiles) * (pl.part + 1) / a.parts);

    const int w0 = r0 + 32 * wv;                       // this wavefront's rows
    const int mine = min(w0 + (lane & 31), rows - 1);  // this lane's row (the last one again beyond the end)
    const int t = mine / a.R;
    const int64_t qrow = (static_cast<int64_t>(b) * a.ch.n + t) * a.Hq + h * a.R + mine % a.R;
    const int first_t = uniform(min(w0, rows - 1) / a.R), last_t = uniform(min(w0 + 31, rows - 1) / a.R);
    u32x4 qf[8];
    load_queries<DT>(a.q + qrow * kD, lane, qf);
    RowState st;
    init_rows(st);

    const RowOffsets ko = row_offsets<true>(lane, 15), vo = row_offsets<false>(lane, 15);
    GroupRows<PAGED> at(a.cv, b, h);
    auto issue = [&](const uint16_t* x, int tile, bool is_key) {
        int g = tile * kTile + 16 * wv;
        if (g >= end) g = (end - 1) & ~15;
        const int buf = (tile - t0) & 1, last = end - 1 - g;
        const uint16_t* base = group_row(x, at.row(uniform(g)));
        if constexpr (PAGED) {
            if (is_key && lane == 0) s_mapped[buf][wv] = base != nullptr;
        }
        const uint32_t to = buf * kBuf + (is_key ? 0 : kSide) + wv * 16 * 256;
        if (last >= 15)
            load_rows16(base, is_key ? ko : vo, to, lds, lane);
        else  // the group holds the last token
            load_rows16(base, is_key ? row_offsets<true>(lane, last) : row_offsets<false>(lane, last), to, lds, lane);
    };
    // Tile by tile, the logits of the next one are computed beside the weights of this one: the matrix units have work while
    // the exponentials run.  So keys are loaded two tiles ahead, values one.
    const int tw = w0 < rows ? min(t1, (past + last_t) / kTile + 1) : t0;  // tiles beyond tw: masked for all of the wavefront
    auto arrive = [&](int tile) {
        dma_wait<0>();
        lds_reads_done();
        barrier_only();
        if (tile + 2 < t1) issue(a.K, tile + 2, true);
        if (tile + 1 < t1) issue(a.V, tile + 1, false);
    };
    auto side = [&](int tile) { return lds + ((tile - t0) & 1) * kBuf; };
    float top = kNegBig;
    auto masked_top = [&](f32x16(&s)[2], int tile) {
        uint32_t mapped = 15u;
        if constexpr (PAGED) {
            const int* x = s_mapped[(tile - t0) & 1];
            mapped = uniform(x[0] | x[1] << 1 | x[2] << 2 | x[3] << 3);
        }
        if (tile * kTile + kTile - 1 > past + first_t || mapped != 15u)
            mask_logits<2>(s, lane, past + t - tile * kTile, mapped);
        top = tile_top<2>(s, a.scale_log2e);
        return __any(has_to_move<DT, ODT == kF32>(st, top)) != 0;
    };
    // one tile, whose logits are s; the next one's to n; true: the maximum has to move before they can be used
    auto step = [&](const f32x16(&s)[2], f32x16(&n)[2], int tile) {
        arrive(tile);
        Weights<2, ODT == kF32> w;
        tile_weights<DT, 2>(st, s, a.scale_log2e, w);
        tile_logits<DT, 2>(side(tile + 1), lane, qf, n);  // (after the last tile of what lies there, and not used)
        tile_values<DT, 2>(st, w, side(tile) + kSide, lane);
        return tile + 1 < tw && masked_top(n, tile + 1);
    };
    f32x16 s[2], n[2];
    if (t0 < t1) {
        issue(a.K, t0, true);
        arrived(qf);
        dma_wait<0>();
        lds_reads_done();
        barrier_only();
        issue(a.V, t0, false);
        if (t0 + 1 < t1) issue(a.K, t0 + 1, true);
    }
    int tile = t0;
    bool moved = false;
    if (tile < tw) {
        tile_logits<DT, 2>(side(tile), lane, qf, s);
        moved = masked_top(s, tile);
    }
    while (tile < tw) {
        if (moved) rescale<DT, ODT == kF32>(st, top);
        // (left only where the maximum moves: the output registers stay where they are while it does not)
        for (moved = false; tile < tw && !moved;) {
            moved = step(s, n, tile++);
            if (moved || tile >= tw) {
                s[0] = n[0], s[1] = n[1];
                break;
            }
            moved = step(n, s, tile++);
        }
    }
    for (; tile < t1; ++tile) arrive(tile);
    float lo, hi;
    both_halves(st.l, lo, hi);
    const float l = lo + hi;
    if (a.parts == 1) {
        if (w0 + (lane & 31) >= rows) return;
        const float inv = l > 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                store4<ODT>(a.out, qrow * kD + 32 * c + 2 * i + 4 * (lane >> 5), st.o[c][i] * inv, st.o[c][i + 1] * inv,
                            st.o[c][i + 2] * inv, st.o[c][i + 3] * inv);
        if (a.lse && lane < 32) a.lse[qrow] = log_sum(st.m, l);
        return;
    }
    if (w0 >= rows) return;
    // (four registers of all lanes at a time, 1 KB each: whole lines, whereas a row's 16 B would be pieces of 32 of them)
    const int64_t pr = ((static_cast<int64_t>(pl.unit) * a.tiles + pl.tile) * a.parts + pl.part) * kRowsTile + 32 * wv;
    if (lane < 32) reinterpret_cast<float2*>(a.part_ml)[pr + lane] = make_float2(st.m, l);
    if (t0 < t1) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                store4<kF32>(a.part_o, pr * kD + ((4 * c + i / 4) * 64 + lane) * 4, st.o[c][i], st.o[c][i + 1], st.o[c][i + 2],
                             st.o[c][i + 3]);
    }
}

template <int DT, int ODT, bool PAGED>
__global__ __launch_bounds__(kBlock, 2) void chunk_tokens_kernel(const ChunkAttn a) {
    constexpr int kTile = 32, kSide = kTile * 256;
    __shared__ struct {
        __align__(16) char tiles[4 * 2 * kSide];  // per wavefront keys, values; at the end the wavefronts' outputs
        float m[4][32], l[4][32];
    } shared;
    char* lds = shared.tiles;
    auto &s_m = shared.m, &s_l = shared.l;
    const int lane = threadIdx.x & 63, wv = uniform(threadIdx.x >> 6);
    const Place pl = place_of(blockIdx.x, a.B * a.cv.Hkv, a.tiles, a.parts);
    const int b = pl.unit / a.cv.Hkv, h = pl.unit % a.cv.Hkv;
    const int past = chunk_past(a.ch, b, a.cv.Lmax), nn = chunk_new(a.ch, b, past, a.cv.Lmax);
    const int rows = nn * a.R;
    if (rows == 0) return;
    const int end = past + nn, n_tiles = (end + kTile - 1) / kTile;
    const int steps = (n_tiles + 3) / 4;
    const int s0 = static_cast<int>(static_cast<int64_t>(steps) * pl.part / a.parts);
    const int s1 = static_cast<int>(static_cast<int64_t>(steps) * (pl.part + 1) / a.parts);

    const int mine = min(lane & 31, rows - 1), t = mine / a.R;
    const int64_t qrow = (static_cast<int64_t>(b) * a.ch.n + t) * a.Hq + h * a.R + mine % a.R;
    u32x4 qf[8];
    load_queries<DT>(a.q + qrow * kD, lane, qf);
    RowState st;
    init_rows(st);

    char* keys = lds + wv * 2 * kSide;
    char* values = keys + kSide;
    const RowOffsets ko = row_offsets<true>(lane, 15), vo = row_offsets<false>(lane, 15);
    uint32_t mapped = 3u;
    GroupRows<PAGED> at(a.cv, b, h);
    // the two 16-token groups of one of this wavefront's tiles, keys and values one after the other
    auto issue = [&](const uint16_t* x, int tile, bool is_key) {
        uint32_t got = 0;
#pragma unroll
        for (int g2 = 0; g2 < 2; ++g2) {
            int g = tile * kTile + 16 * g2;
            if (g >= end) g = (end - 1) & ~15;
            const uint16_t* base = group_row(x, at.row(uniform(g)));
            got |= (base != nullptr) << g2;
            const int last = min(end - 1 - g, 15);
            RowOffsets r = is_key ? ko : vo;
            if (last < 15) r = is_key ? row_offsets<true>(lane, last) : row_offsets<false>(lane, last);
            load_rows16(base, r, (is_key ? keys : values) - lds + g2 * 16 * 256, lds, lane);
        }
        return got;
    };
    int tile = 4 * s0 + wv;
    const int stop = min(4 * s1, n_tiles);
    uint32_t next = 3u;
    if (tile < stop) {
        mapped = issue(a.K, tile, true);
        issue(a.V, tile, false);
    }
    arrived(qf);
    for (; tile < stop; tile += 4) {
        const bool more = tile + 4 < stop;
        dma_wait<8>();
        if constexpr (PAGED) {
            if (mapped != 3u) dma_wait<0>();  // fewer loads than counted
        }
        f32x16 s[1];
        tile_logits<DT, 1>(keys, lane, qf, s);
        lds_reads_done();
        if (more) next = issue(a.K, tile + 4, true);
        if (tile * kTile + kTile - 1 > past || mapped != 3u) mask_logits<1>(s, lane, past + t - tile * kTile, mapped);
        if (more && (!PAGED || next == 3u))
            dma_wait<8>();
        else
            dma_wait<0>();
        const float top = tile_top<1>(s, a.scale_log2e);
        if (__any(has_to_move<DT, true>(st, top))) rescale<DT, true>(st, top);
        Weights<1, true> w;
        tile_weights<DT, 1>(st, s, a.scale_log2e, w);
        tile_values<DT, 1>(st, w, values, lane);
        lds_reads_done();
        if (more) issue(a.V, tile + 4, false);
        mapped = next;
    }
    float lo, hi;
    both_halves(st.l, lo, hi);
    st.l = lo + hi;
    __syncthreads();
    // the four wavefronts' states of each row, joined
    float* so = reinterpret_cast<float*>(lds) + wv * 32 * kD;
    if (lane < 32) {
        s_m[wv][lane] = st.m;
        s_l[wv][lane] = st.l;
    }
    if ((lane & 31) < rows) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *reinterpret_cast<float4*>(so + (lane & 31) * kD + 32 * c + 2 * i + 4 * (lane >> 5)) =
                    make_float4(st.o[c][i], st.o[c][i + 1], st.o[c][i + 2], st.o[c][i + 3]);
    }
    __syncthreads();
    const int n_rows = min(rows, 32);
    for (int e = threadIdx.x; e < n_rows * (kD / 4); e += kBlock) {
        const int r = e / (kD / 4), d = (e % (kD / 4)) * 4;
        float M = kNegBig, l = 0.0f, o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < 4; ++w) M = fmaxf(M, s_m[w][r]);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = fast_exp2(s_m[w][r] - M);
            const float4 x = *reinterpret_cast<const float4*>(reinterpret_cast<float*>(lds) + (w * 32 + r) * kD + d);
            l += s_l[w][r] * f;
            o[0] += x.x * f, o[1] += x.y * f, o[2] += x.z * f, o[3] += x.w * f;
        }
        if (a.parts == 1) {
            const int64_t at = (static_cast<int64_t>(b) * a.ch.n + r / a.R) * a.Hq + h * a.R + r % a.R;
            const float inv = l > 0.0f ? 1.0f / l : 0.0f;
            store4<ODT>(a.out, at * kD + d, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
            if (a.lse && d == 0) a.lse[at] = log_sum(M, l);
        } else {
            const int64_t pr = (static_cast<int64_t>(pl.unit) * a.parts + pl.part) * kTokensTile + r;
            store4<kF32>(a.part_o, pr * kD + d, o[0], o[1], o[2], o[3]);
            if (d == 0) reinterpret_cast<float2*>(a.part_ml)[pr] = make_float2(M, l);
        }
    }
}

// The states of a row's parts, joined in their order.  After the `tokens` form a workgroup per row: a part per lane for the
// maxima and sums, then 32 lanes of four channels and eight parts at a time for the outputs, all requested before the first
// is used.
template <int ODT>
__global__ __launch_bounds__(kBlock) void join_tokens_kernel(const ChunkAttn a) {
    constexpr int kGroups = kBlock / 32, kEach = kMaxParts / kGroups;
    __shared__ float s_f[kMaxParts];
    __shared__ float4 s_o[kGroups][32];
    const int64_t row = blockIdx.x;  // of [unit][n * R]
    const int per = a.ch.n * a.R, u = static_cast<int>(row / per), m = static_cast<int>(row % per);
    const int b = u / a.cv.Hkv, h = u % a.cv.Hkv;
    const int tid = threadIdx.x, lane = tid & 63, g = tid >> 5, c4 = tid & 31;
    const int64_t p0 = (static_cast<int64_t>(u) * a.tiles + m / kTokensTile) * a.parts;
    const int past = chunk_past(a.ch, b, a.cv.Lmax), nn = chunk_new(a.ch, b, past, a.cv.Lmax);
    if (m >= nn * a.R) return;
    // every wavefront takes the maxima and sums of all parts, two to a lane
    float2 ml[kMaxParts / 64];
    float M = kNegBig, l = 0.0f;
#pragma unroll
    for (int i = 0; i < kMaxParts / 64; ++i) {
        const int p = lane + 64 * i;
        ml[i] = p < a.parts ? reinterpret_cast<const float2*>(a.part_ml)[(p0 + p) * kTokensTile + m % kTokensTile]
                            : make_float2(kNegBig, 0.0f);
        M = fmaxf(M, ml[i].x);
    }
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) M = fmaxf(M, __shfl_xor(M, x, 64));
#pragma unroll
    for (int i = 0; i < kMaxParts / 64; ++i) {
        const float f = ml[i].y > 0.0f ? fast_exp2(ml[i].x - M) : 0.0f;  // a part without tokens gives nothing
        l += ml[i].y * f;
        if (tid < 64) s_f[lane + 64 * i] = f;
    }
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) l += __shfl_xor(l, x, 64);
    __syncthreads();
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int i0 = 0; i0 < kEach && i0 * kGroups < a.parts; i0 += 4) {
        float4 x[4];
        float f[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int p = g + kGroups * (i0 + i);
            f[i] = p < a.parts ? s_f[p] : 0.0f;
            const int64_t at = ((p0 + p) * kTokensTile + m % kTokensTile) * (kD / 4) + c4;
            x[i] = f[i] > 0.0f ? reinterpret_cast<const float4*>(a.part_o)[at] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) o.x += x[i].x * f[i], o.y += x[i].y * f[i], o.z += x[i].z * f[i], o.w += x[i].w * f[i];
    }
    s_o[g][c4] = o;
    __syncthreads();
    if (g != 0) return;
#pragma unroll
    for (int x = 1; x < kGroups; ++x) {
        const float4 y = s_o[x][c4];
        o.x += y.x, o.y += y.y, o.z += y.z, o.w += y.w;
    }
    const int64_t at = (static_cast<int64_t>(b) * a.ch.n + m / a.R) * a.Hq + h * a.R + m % a.R;
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    store4<ODT>(a.out, at * kD + 4 * c4, o.x * inv, o.y * inv, o.z * inv, o.w * inv);
    if (a.lse && c4 == 0) a.lse[at] = log_sum(M, l);
}

// After the `rows` form: a lane has a row and four of its channels, as the states lie in memory.  SPLIT: the 8 groups of 32
// lanes of a workgroup share one such block's parts (many parts, few rows), otherwise each has a block of its own.
template <int ODT, bool SPLIT>
__global__ __launch_bounds__(kBlock) void join_rows_kernel(const ChunkAttn a, int blocks) {
    constexpr int kGroups = kBlock / 32, kEach = SPLIT ? kMaxParts / kGroups : kGroups;
    __shared__ float s_m[kGroups][32], s_l[kGroups][32];
    __shared__ float4 s_o[kGroups][32];
    const int r = threadIdx.x & 31, g = threadIdx.x >> 5;
    constexpr int kPer = SPLIT ? 32 : 32 / kGroups;  // workgroups to 32 rows
    // channels 32 (x / 8) + 8 (x % 8 / 2) + 4 (x % 2) ..
    const int x = SPLIT ? blockIdx.x % kPer : blockIdx.x % kPer * kGroups + g;
    const int64_t w = blockIdx.x / kPer;  // 32 rows: [unit][block]
    const int u = static_cast<int>(w / blocks), m = static_cast<int>(w % blocks) * 32 + r;
    const int b = u / a.cv.Hkv, h = u % a.cv.Hkv;
    const int past = chunk_past(a.ch, b, a.cv.Lmax), nn = chunk_new(a.ch, b, past, a.cv.Lmax), rows = nn * a.R;
    if (m - r >= rows) return;
    const int64_t p0 = (static_cast<int64_t>(u) * a.tiles + m / kRowsTile) * a.parts;
    float2 ml[kEach];
    float M = kNegBig, l = 0.0f;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int p = SPLIT ? g + kGroups * i : i;
        ml[i] = p < a.parts ? reinterpret_cast<const float2*>(a.part_ml)[(p0 + p) * kRowsTile + m % kRowsTile]
                            : make_float2(kNegBig, 0.0f);
        if (ml[i].y > 0.0f) M = fmaxf(M, ml[i].x);
    }
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    const float4* po = reinterpret_cast<const float4*>(a.part_o) +
                       (p0 * kRowsTile + (m % kRowsTile - r)) * (kD / 4) + (x >> 1) * 64 + (x & 1) * 32 + r;
#pragma unroll
    for (int i0 = 0; i0 < kEach; i0 += 4) {
        if ((SPLIT ? kGroups * i0 : i0) >= a.parts) break;
        float4 y[4];
        float f[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int p = SPLIT ? g + kGroups * (i0 + i) : i0 + i;
            const bool on = ml[i0 + i].y > 0.0f;  // a part without tokens has not written its state
            f[i] = on ? fast_exp2(ml[i0 + i].x - M) : 0.0f;
            y[i] = on ? po[static_cast<int64_t>(p) * kRowsTile * (kD / 4)] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            l += ml[i0 + i].y * f[i];
            o.x += y[i].x * f[i], o.y += y[i].y * f[i], o.z += y[i].z * f[i], o.w += y[i].w * f[i];
        }
    }
    if constexpr (SPLIT) {
        s_m[g][r] = M;
        s_l[g][r] = l;
        s_o[g][r] = o;
        __syncthreads();
        if (g != 0) return;
#pragma unroll
        for (int k = 1; k < kGroups; ++k) M = fmaxf(M, s_m[k][r]);
        l = 0.0f;
        o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < kGroups; ++k) {
            const float f = fast_exp2(s_m[k][r] - M);
            const float4 y = s_o[k][r];
            l += s_l[k][r] * f;
            o.x += y.x * f, o.y += y.y * f, o.z += y.z * f, o.w += y.w * f;
        }
    }
    if (m >= rows) return;
    const int64_t at = (static_cast<int64_t>(b) * a.ch.n + m / a.R) * a.Hq + h * a.R + m % a.R;
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    store4<ODT>(a.out, at * kD + 32 * (x >> 3) + 8 * ((x & 7) >> 1) + 4 * (x & 1), o.x * inv, o.y * inv, o.z * inv, o.w * inv);
    if (a.lse && x == 0) a.lse[at] = log_sum(M, l);
}

// Form and split of a call.  Both forms run two workgroups to a compute unit, kSlots at a time.
constexpr int kSlots = 512, kMaxGroups = 3 * kSlots;
struct ChunkPlan {
    bool tokens;
    int tiles, parts, tile_rows;
};
// At least 256 tokens to a part; of short caches in the `tokens` form 128, a step of its four wavefronts, up to 32 parts (one
// token on 500 to 2000 tokens of 8 KV heads 9.2 to 10.2 us against 10.3 to 11.3; on 8000 63 parts take 15.7, 32 take 14.8).
static int most_parts(const Dims& d, bool tokens) {
    int most = (d.Lmax + 255) / 256;
    if (tokens && most < 32) most = (d.Lmax + 127) / 128 < 32 ? (d.Lmax + 127) / 128 : 32;
    return most < kMaxParts ? most : kMaxParts;
}
static ChunkPlan chunk_plan(const Dims& d, int n) {
    ChunkPlan p;
    const int64_t rows = static_cast<int64_t>(n) * d.R;
    p.tokens = rows <= kTokensTile;
    p.tile_rows = p.tokens ? kTokensTile : kRowsTile;
    p.tiles = static_cast<int>((rows + p.tile_rows - 1) / p.tile_rows);
    const int64_t groups = static_cast<int64_t>(d.units()) * p.tiles;
    p.parts = 1;
    const int most = most_parts(d, p.tokens);
    if (p.tokens) {
        // memory-bound: one round of workgroups (one token on 32767 tokens of 8 KV heads: 33 us in 64 parts, 38 in 96; on 1000 of
        // 32 x 8 heads 33.8 in two, 36.6 in three).  From 257 units on that is one part, which leaves up to half of the round
        // empty: a token on 1000 of 33 x 8 heads 38.2 in one, 37.3 in two, on 8000 278 and 249.
        const int64_t by_slots = kSlots / groups;
        p.parts = static_cast<int>(by_slots < 1 ? 1 : by_slots < most ? by_slots : most);
        return p;
    }
    // Cost of a split in tiles of 64 tokens, a part's state and its join counted as six (a lone part's start as two): rounds
    // of workgroups, as if all sequences were as long as the cache; in a batch, where they seldom are, plus the same with
    // lengths spread (two thirds on average, half of the last round idle).  333 tokens behind 9000 of 6 x 8 KV heads with
    // 5:1 heads: two parts 457 us against 468 of one, with unequal lengths over pages 250 against 305; 100 behind 16000 of 8 x 8
    // with 8:1, unequal: 270 against 357; 64 behind 2000 of 16 x 8 with 4:1: two parts 63, one 61, four 73.
    const float T = static_cast<float>((d.Lmax + 63) / 64);
    float best = 0.0f;
    for (int k = 1; k <= most && (k == 1 || groups * k <= kMaxGroups); ++k) {
        const float part = T / k, extra = k == 1 ? 2.0f : 6.0f, g = static_cast<float>(groups);
        float cost = static_cast<float>((groups * k + kSlots - 1) / kSlots) * (part + extra);
        if (d.B > 1) {
            const float spread = g * (0.65f * T + k * extra) / kSlots + 0.5f * (part + extra);
            cost += spread > part + extra ? spread : part + extra;
        }
        if (k == 1 || cost < best) {
            best = cost;
            p.parts = k;
        }
    }
    return p;
}

static int join_blocks(const Dims& d, int n) { return static_cast<int>((static_cast<int64_t>(n) * d.R + 31) / 32); }
static bool join_splits(const ChunkPlan& p) { return p.parts > 8; }
static int64_t join_grid(const Dims& d, const ChunkPlan& p, int n) {
    if (p.tokens) return static_cast<int64_t>(d.rows()) * n;
    return static_cast<int64_t>(d.units()) * join_blocks(d, n) * (join_splits(p) ? 32 : 4);
}

static size_t plan_rows(const Dims& d, const ChunkPlan& p) {
    return p.parts == 1 ? 0 : static_cast<size_t>(d.units()) * p.tiles * p.parts * p.tile_rows;
}

size_t chunk_attn_bytes(const Dims& d, int n) {
    // what any chunk of up to n tokens needs, whatever its plan: no split has more than kMaxGroups workgroups
    const int64_t parts = most_parts(d, true), tiles = (static_cast<int64_t>(n) * d.R + kRowsTile - 1) / kRowsTile;
    auto bound = [&](int64_t groups, int64_t cap) { return groups > cap / parts ? cap : groups * parts; };
    const int64_t r = bound(d.units() * tiles, kMaxGroups) * kRowsTile, t = bound(d.units(), kSlots) * kTokensTile;
    return parts == 1 ? 0 : static_cast<size_t>(r > t ? r : t) * (kD + 2) * 4;
}

hipError_t launch_chunk_attn(const Dims& d, const CacheView& c, const ChunkView& ch, const void* q, const void* K,
                             const void* V, float scale, void* out, float* lse, void* ws, hipStream_t s) {
    if (static_cast<int64_t>(ch.n) * d.R > 0x7fffffff - kRowsTile)
        return hipErrorInvalidConfiguration;  // rows are counted in 32 bits
    const ChunkPlan p = chunk_plan(d, ch.n);
    const int64_t grid = static_cast<int64_t>(d.units()) * p.tiles * p.parts, join = join_grid(d, p, ch.n);
    const int blocks = join_blocks(d, ch.n);
    if (grid > 0x7fffffff / kBlock || (p.parts > 1 && join > 0x7fffffff / kBlock)) return hipErrorInvalidConfiguration;
    const float sl2 = (scale > 0.0f ? scale : 1.0f / sqrtf(static_cast<float>(kD))) * 1.4426950408889634f;
    float* po = static_cast<float*>(ws);
    const ChunkAttn a{static_cast<const uint16_t*>(q), static_cast<const uint16_t*>(K), static_cast<const uint16_t*>(V),
                      c, ch, d.B, d.Hq, d.R, p.tiles, p.parts, sl2, out, lse, po, po + plan_rows(d, p) * kD};
    hipError_t e = hipErrorInvalidValue;
#define SIK_CHUNK(DTV, ODTV)                                                                                                \
    e = p.tokens ? (c.table ? launch_kernel(chunk_tokens_kernel<DTV, ODTV, true>, static_cast<int>(grid), kBlock, s, a)     \
                            : launch_kernel(chunk_tokens_kernel<DTV, ODTV, false>, static_cast<int>(grid), kBlock, s, a))   \
                 : (c.table ? launch_kernel(chunk_rows_kernel<DTV, ODTV, true>, static_cast<int>(grid), kBlock, s, a)       \
                            : launch_kernel(chunk_rows_kernel<DTV, ODTV, false>, static_cast<int>(grid), kBlock, s, a));    \
    if (e == hipSuccess && p.parts > 1)                                                                                     \
        e = p.tokens           ? launch_kernel(join_tokens_kernel<ODTV>, static_cast<int>(join), kBlock, s, a)              \
            : join_splits(p)   ? launch_kernel(join_rows_kernel<ODTV, true>, static_cast<int>(join), kBlock, s, a, blocks)  \
                               : launch_kernel(join_rows_kernel<ODTV, false>, static_cast<int>(join), kBlock, s, a, blocks)
    if (d.kv_dtype == kBF16) {
        if (d.out_dtype == kF32) {
            SIK_CHUNK(kBF16, kF32);
        } else {
            SIK_CHUNK(kBF16, kBF16);
        }
    } else if (d.out_dtype == kF32) {
        SIK_CHUNK(kF16, kF32);
    } else {
        SIK_CHUNK(kF16, kF16);
    }
#undef SIK_CHUNK
    return e;
}

}  // namespace sik
