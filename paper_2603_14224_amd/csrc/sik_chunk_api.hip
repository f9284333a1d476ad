// C ABI of the prompt side of the cache: host-side validation and launches.  Contracts live in include/sik.h.
#include "sik_chunk.h"

namespace sik {

static bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

static bool overlap(const void* p, size_t np, const void* q, size_t nq) {  // false where one is NULL
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
    return a != 0 && b != 0 && a < b + nq && b < a + np;
}

static int check_pages(const Dims& d, const sik_pages* p, CacheView* c) {
    *c = CacheView{nullptr, 0, 0, 0, d.Hkv, d.Lmax};
    if (!p) return SIK_OK;
    if (!p->page_table) return SIK_ERR_NULL;
    if (p->page_len < 16 || (p->page_len & (p->page_len - 1)) != 0 || p->n_pages < 1 || p->pages_per_seq < 1)
        return SIK_ERR_SHAPE;
    if (static_cast<int64_t>(p->pages_per_seq) * p->page_len < d.Lmax) return SIK_ERR_SHAPE;
    c->table = p->page_table;
    c->per_seq = p->pages_per_seq;
    c->n_pages = p->n_pages;
    while ((1 << c->shift) < p->page_len) ++c->shift;
    return SIK_OK;
}

static int check_chunk(const Dims& d, const sik_chunk* ch, CacheView* c, ChunkView* v) {
    if (!ch) return SIK_ERR_NULL;
    if (!ch->seq_len) return SIK_ERR_NULL;
    if (ch->n < 1 || ch->n > d.Lmax) return SIK_ERR_CAPACITY;
    *v = ChunkView{ch->seq_len, ch->n_new, ch->n};
    return check_pages(d, ch->pages, c);
}

static int launched(hipError_t e) {
    if (e == hipSuccess) return SIK_OK;
    return e == hipErrorInvalidConfiguration ? SIK_ERR_SHAPE : SIK_ERR_LAUNCH;  // more workgroups than a launch can have
}

}  // namespace sik

using namespace sik;

extern "C" {

int sik_rope_append(const sik_layout* layout, const sik_chunk* chunk, const sik_rope_args* a) {
    Dims d;
    int rc = check_layout(layout, &d);
    if (rc) return rc;
    CacheView c;
    ChunkView ch;
    rc = check_chunk(d, chunk, &c, &ch);
    if (rc) return rc;
    if (!a || !a->q || !a->k || !a->q_out) return SIK_ERR_NULL;
    if (a->k_out ? (a->K || a->V || a->v) : (!a->K || !a->V || !a->v)) return SIK_ERR_NULL;
    if (a->interleaved != 0 && a->interleaved != 1) return SIK_ERR_FLAGS;
    if (a->rotary_dim < 0 || a->rotary_dim > kD || a->rotary_dim % 16 != 0) return SIK_ERR_SHAPE;
    if (a->rotary_dim > 0 && !a->inv_freq) return SIK_ERR_NULL;
    if (!(a->eps >= 0.0f)) return SIK_ERR_FLAGS;
    const int64_t qs = a->q_stride ? a->q_stride : static_cast<int64_t>(d.Hq) * kD;
    const int64_t ks = a->k_stride ? a->k_stride : static_cast<int64_t>(d.Hkv) * kD;
    const int64_t vs = a->v_stride ? a->v_stride : static_cast<int64_t>(d.Hkv) * kD;
    if (qs < static_cast<int64_t>(d.Hq) * kD || ks < static_cast<int64_t>(d.Hkv) * kD || vs < static_cast<int64_t>(d.Hkv) * kD)
        return SIK_ERR_SHAPE;
    if (((qs | ks | vs) & 7) != 0) return SIK_ERR_ALIGN;
    for (const void* p : {a->q, a->k, a->v, static_cast<const void*>(a->q_weight), static_cast<const void*>(a->k_weight),
                          static_cast<const void*>(a->q_out), static_cast<const void*>(a->k_out),
                          static_cast<const void*>(a->K), static_cast<const void*>(a->V)})
        if (misaligned(p)) return SIK_ERR_ALIGN;
    if (a->q_out == a->q || a->q_out == a->k || (a->k_out && (a->k_out == a->k || a->k_out == a->q || a->k_out == a->q_out)) ||
        (a->K && a->K == a->V))
        return SIK_ERR_FLAGS;
    const RopeArgs r{static_cast<const uint16_t*>(a->q), static_cast<const uint16_t*>(a->k),
                     static_cast<const uint16_t*>(a->v), qs, ks, vs, a->q_weight, a->k_weight, a->eps, a->inv_freq,
                     a->rotary_dim, a->positions, static_cast<uint16_t*>(a->q_out), static_cast<uint16_t*>(a->k_out),
                     static_cast<uint16_t*>(a->K), static_cast<uint16_t*>(a->V)};
    return launched(launch_rope(d, c, ch, r, a->interleaved == 1, static_cast<hipStream_t>(a->stream)));
}

size_t sik_chunk_workspace_bytes(const sik_layout* layout, int32_t n) {
    Dims d;
    if (check_layout(layout, &d) != SIK_OK || n < 1 || n > d.Lmax) return 0;
    const size_t a = chunk_attn_bytes(d, n), e = evict_bytes(d);
    const size_t most = a > e ? a : e;
    return (most + 255) / 256 * 256 + 256;  // never 0
}

static int check_chunk_ws(const sik_layout* layout, int n, const void* ws, size_t bytes) {
    if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u) != 0) return SIK_ERR_WORKSPACE;
    return bytes < sik_chunk_workspace_bytes(layout, n) ? SIK_ERR_WORKSPACE : SIK_OK;
}

int sik_chunk_attn(const sik_layout* layout, const sik_chunk* chunk, const void* q, const void* K, const void* V,
                   float softmax_scale, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    Dims d;
    int rc = check_layout(layout, &d);
    if (rc) return rc;
    CacheView c;
    ChunkView ch;
    rc = check_chunk(d, chunk, &c, &ch);
    if (rc) return rc;
    if (!q || !K || !V || !out) return SIK_ERR_NULL;
    if (misaligned(q) || misaligned(K) || misaligned(V) || misaligned(out)) return SIK_ERR_ALIGN;
    if (out == q) return SIK_ERR_FLAGS;
    rc = check_chunk_ws(layout, ch.n, workspace, workspace_bytes);
    if (rc) return rc;
    return launched(launch_chunk_attn(d, c, ch, q, K, V, softmax_scale, out, lse, workspace, static_cast<hipStream_t>(stream)));
}

int sik_attn_mass(const sik_layout* layout, const sik_chunk* chunk, const void* q, const void* K, float softmax_scale,
                  const float* lse, int32_t n_obs, const float* before, float* mass, void* stream) {
    Dims d;
    int rc = check_layout(layout, &d);
    if (rc) return rc;
    CacheView c;
    ChunkView ch;
    rc = check_chunk(d, chunk, &c, &ch);
    if (rc) return rc;
    if (!q || !K || !lse || !mass) return SIK_ERR_NULL;
    if (misaligned(q) || misaligned(K)) return SIK_ERR_ALIGN;
    if (n_obs < 1 || n_obs > ch.n) return SIK_ERR_CAPACITY;
    return launched(launch_mass(d, c, ch, q, K, softmax_scale, lse, n_obs, before, mass, static_cast<hipStream_t>(stream)));
}

int sik_evict(const sik_layout* layout, const sik_evict_args* a) {
    Dims d;
    int rc = check_layout(layout, &d);
    if (rc) return rc;
    if (!a || !a->mass || !a->seq_len || !a->keep) return SIK_ERR_NULL;
    if (a->n_keep < 1 || a->n_keep > d.Lmax) return SIK_ERR_K_RANGE;
    if (a->n_sink < 0 || a->n_recent < 0 || static_cast<int64_t>(a->n_sink) + a->n_recent > a->n_keep) return SIK_ERR_K_RANGE;
    CacheView c;
    rc = check_pages(d, a->pages, &c);
    if (rc) return rc;
    if (!a->K_out != !a->V_out) return SIK_ERR_NULL;
    if (a->K_out) {
        if (!a->K || !a->V) return SIK_ERR_NULL;
        if (a->K_out == a->K || a->V_out == a->V || a->K_out == a->V_out || a->K_out == a->V || a->V_out == a->K)
            return SIK_ERR_FLAGS;
        if (misaligned(a->K) || misaligned(a->V) || misaligned(a->K_out) || misaligned(a->V_out)) return SIK_ERR_ALIGN;
    }
    if (a->mass_out == a->mass) return SIK_ERR_FLAGS;
    if ((a->K_out || a->mass_out) && a->out_len < a->n_keep) return SIK_ERR_CAPACITY;
    rc = check_chunk_ws(layout, 1, a->workspace, a->workspace_bytes);
    if (rc) return rc;
    // workgroups read lengths and weights while others already write their part of the list
    const size_t lens = static_cast<size_t>(d.B) * 4, list = static_cast<size_t>(d.units()) * a->n_keep * 4;
    const size_t sums = static_cast<size_t>(d.units()) * d.Lmax * 4;
    if (overlap(a->new_len, lens, a->seq_len, lens) || overlap(a->new_len, lens, a->mass, sums) ||
        overlap(a->keep, list, a->seq_len, lens) || overlap(a->keep, list, a->mass, sums) ||
        overlap(a->keep, list, a->new_len, lens))
        return SIK_ERR_FLAGS;
    const EvictArgs e{a->mass, a->seq_len, a->n_keep, a->n_sink, a->n_recent, a->keep, a->new_len,
                      static_cast<const uint16_t*>(a->K), static_cast<const uint16_t*>(a->V),
                      static_cast<uint16_t*>(a->K_out), static_cast<uint16_t*>(a->V_out), a->mass_out, a->out_len};
    return launched(launch_evict(d, c, e, a->workspace, static_cast<hipStream_t>(a->stream)));
}

}  // extern "C"
