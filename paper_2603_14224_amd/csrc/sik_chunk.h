// The prompt side's view of a cache and a chunk of new tokens, shared by the norm + rotation, chunk attention, weight and
// eviction kernels and their launchers.
#pragma once

#include "sik_device.h"
#include "sik_internal.h"

namespace sik {

// Where the rows of a contiguous or paged cache lie.  table == nullptr: contiguous.
struct CacheView {
    const int32_t* table;  // [B][per_seq]
    int per_seq, shift, n_pages;
    int Hkv, Lmax;
};

struct ChunkView {
    const int32_t* seq_len;
    const int32_t* n_new;  // nullptr: n
    int n;
};

// Row (of kD values) of token j < Lmax of head h of sequence b, or -1 where its page is unmapped.
__device__ __forceinline__ int64_t cache_row(const CacheView& c, int b, int h, int j) {
    if (c.table == nullptr) return (static_cast<int64_t>(b) * c.Hkv + h) * c.Lmax + j;
    const int page = c.table[static_cast<int64_t>(b) * c.per_seq + (j >> c.shift)];
    if (static_cast<uint32_t>(page) >= static_cast<uint32_t>(c.n_pages)) return -1;
    return ((static_cast<int64_t>(page) * c.Hkv + h) << c.shift) + (j & ((1 << c.shift) - 1));
}

// Tokens of sequence b in the cache before the chunk, and tokens of the chunk that have a place in it.
__device__ __forceinline__ int chunk_past(const ChunkView& c, int b, int Lmax) {
    return min(max(c.seq_len[b], 0), Lmax);
}
__device__ __forceinline__ int chunk_new(const ChunkView& c, int b, int past, int Lmax) {
    const int n = c.n_new ? min(max(c.n_new[b], 0), c.n) : c.n;
    return min(n, Lmax - past);
}

struct RopeArgs {
    const uint16_t *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;  // elements from token to token
    const float *q_weight, *k_weight;
    float eps;
    const float* inv_freq;
    int rotary_dim;
    const int32_t* positions;
    uint16_t *q_out, *k_out, *K, *V;
};
hipError_t launch_rope(const Dims& d, const CacheView& c, const ChunkView& ch, const RopeArgs& a, bool interleaved,
                       hipStream_t s);

size_t chunk_attn_bytes(const Dims& d, int n);
hipError_t launch_chunk_attn(const Dims& d, const CacheView& c, const ChunkView& ch, const void* q, const void* K,
                             const void* V, float scale, void* out, float* lse, void* ws, hipStream_t s);

hipError_t launch_mass(const Dims& d, const CacheView& c, const ChunkView& ch, const void* q, const void* K, float scale,
                       const float* lse, int n_obs, const float* before, float* mass, hipStream_t s);

struct EvictArgs {
    const float* mass;
    const int32_t* seq_len;
    int n_keep, n_sink, n_recent;
    int32_t *keep, *new_len;
    const uint16_t *K, *V;
    uint16_t *K_out, *V_out;
    float* mass_out;
    int out_len;
};
size_t evict_bytes(const Dims& d);
hipError_t launch_evict(const Dims& d, const CacheView& c, const EvictArgs& a, void* ws, hipStream_t s);

}  // namespace sik
