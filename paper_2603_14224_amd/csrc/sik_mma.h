// Matrix-unit building blocks of the prompt-side kernels (gfx950): 32x32x16 products of 16-bit operands with binary32 sums,
// rows of a cache brought into LDS without passing through registers, and the swizzles that keep both sides free of bank
// conflicts.
//
// Lane layouts of the 32x32x16 product (l = lane, h = l / 32): operand A holds row l % 32, B column l % 32, each the eight
// values 8 h .. 8 h + 7 of the summed axis; the result's register i holds row 8 (i / 4) + 4 h + i % 4 of column l % 32.
#pragma once

#include "sik_chunk.h"

namespace sik {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

template <int DT>
__device__ __forceinline__ f32x16 mma32(u32x4 a, u32x4 b, f32x16 c) {
    if constexpr (DT == kBF16)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Two binary32 values to a register of two 16-bit ones, to nearest even (one instruction on this target), and back.
template <int DT>
__device__ __forceinline__ uint32_t pack16(float a, float b) {
    const f32x2 x = {a, b};
    if constexpr (DT == kBF16)
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
    else
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, f16x2));
}

// x of this lane and of the lane 32 away, in either order.
__device__ __forceinline__ void both_halves(float x, float& lo, float& hi) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    lo = __uint_as_float(r[0]);
    hi = __uint_as_float(r[1]);
}

// ---- rows of a cache into LDS -------------------------------------------------------------------------------------
// A row of 256 B is 16 pieces of 16 B; LDS row r keeps piece c in place c ^ swizzle(r).  The row-wise reads of keys (16 lanes
// read one piece of 16 rows) meet all 64 banks once with r % 16, the transposing reads of values (32 lanes read 64 B of four
// rows) with 4 (r % 4).  The loads put a wavefront's 64 x 16 B one behind the other, so the swizzle is applied to the
// address that a lane reads from.
__device__ __forceinline__ int key_swizzle(int r) { return r & 15; }
__device__ __forceinline__ int value_swizzle(int r) { return (r & 3) << 2; }

__device__ __forceinline__ uint32_t lds_offset(const void* p) {
    return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const char*)(p)));
}

// 64 x 16 B from base + off (bytes, per lane) to LDS [to, to + 1 KB).  Written in assembly because the compiler would wait
// for it before every LDS read that follows; dma_wait is the wait.  A base may come from a vector instruction
// (readfirstlane), and a memory instruction may read such a scalar register only five states later: dma_base sees to that,
// which the compiler does not do for assembly.  (m0 holds nothing across instructions here: the compiler sets it right before
// a use of its own, and these kernels have none.)
template <class T>
__device__ __forceinline__ T* dma_base(T* base) {
    asm volatile("s_nop 4" : "+s"(base));
    return base;
}
__device__ __forceinline__ void dma_16(const void* base, uint32_t off, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(base) : "memory");
}
// All but the newest n loads of this wavefront have arrived.
template <int N>
__device__ __forceinline__ void dma_wait() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// Reads of LDS that were asked for have been served: what they read may be overwritten.
__device__ __forceinline__ void lds_reads_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void barrier_only() { asm volatile("s_barrier" ::: "memory"); }

// Fragments that were loaded into registers have arrived.  Without this the compiler would wait for them where a loop first
// uses them, in every pass, and with them for the loads that the loop keeps on their way.
__device__ __forceinline__ void arrived(u32x4 (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) asm volatile("" : "+v"(f[i]));
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
template <class T>
__device__ __forceinline__ T* uniform(T* p) {
    const uint64_t a = reinterpret_cast<uint64_t>(p);
    const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(a));
    const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(a >> 32));
    return reinterpret_cast<T*>(static_cast<uint64_t>(hi) << 32 | lo);
}

// Rows of the 16-token groups of one sequence and head, a group at a time (uniform over the wavefront).  Of a page table the
// wavefront holds 64 entries, one per lane, so that a group costs a register read and the table a load every 64 pages: a load
// per group would wait for all the rows that are on their way.
template <bool PAGED>
struct GroupRows {
    const CacheView& c;
    int64_t first;  // contiguous: row of token 0
    const int32_t* table;
    int h, window = -64, held = 0;
    __device__ __forceinline__ GroupRows(const CacheView& c_, int b, int h_) : c(c_), h(h_) {
        first = (static_cast<int64_t>(b) * c.Hkv + h) * c.Lmax;
        if constexpr (PAGED) table = c.table + static_cast<int64_t>(b) * c.per_seq;
    }
    // row of token j, -1 without a page
    __device__ __forceinline__ int64_t row(int j) {
        if constexpr (!PAGED) return first + j;
        const int p = j >> c.shift;
        if (p < window || p >= window + 64) {
            window = p;
            held = table[min(p + static_cast<int>(threadIdx.x & 63), c.per_seq - 1)];
        }
        const int page = __builtin_amdgcn_readlane(held, p - window);
        if (static_cast<uint32_t>(page) >= static_cast<uint32_t>(c.n_pages)) return -1;
        return ((static_cast<int64_t>(page) * c.Hkv + h) << c.shift) + (j & ((1 << c.shift) - 1));
    }
};

// What a lane reads when its wavefront loads 16 rows of 256 B in four instructions: row 4 i + l / 16, the piece that the
// swizzle puts in place l % 16.
struct RowOffsets {
    uint32_t off[4];
};
template <bool KEYS>
__device__ __forceinline__ RowOffsets row_offsets(int lane, int last) {  // rows beyond `last` repeat it
    RowOffsets r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = 4 * i + (lane >> 4);
        const int piece = (lane & 15) ^ (KEYS ? key_swizzle(row) : value_swizzle(row));
        r.off[i] = min(row, last) * 256 + piece * 16;
    }
    return r;
}

// 16 rows (all on one page) to LDS rows starting at byte `to`; base == nullptr: zeros (no page).
__device__ __forceinline__ void load_rows16(const uint16_t* base, const RowOffsets& r, uint32_t to, char* lds, int lane) {
    if (base == nullptr) {
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<u32x4*>(lds + to + i * 1024 + lane * 16) = u32x4{0u, 0u, 0u, 0u};
        return;
    }
    const uint32_t at = lds_offset(lds) + to;
    base = dma_base(base);
#pragma unroll
    for (int i = 0; i < 4; ++i) dma_16(base, r.off[i], uniform(static_cast<int>(at + i * 1024)));
}

// Operand A or B from 32 rows at `rows` (LDS, key swizzle): row lane % 32, values 16 step + 8 h ..
__device__ __forceinline__ u32x4 row_fragment(const char* rows, int lane, int step) {
    const int r = lane & 31, c = 2 * step + (lane >> 5);
    return *reinterpret_cast<const u32x4*>(rows + r * 256 + ((c ^ key_swizzle(r)) << 4));
}

// Operand A of V^T from 16 rows at `rows` (LDS, value swizzle): channels 32 block + lane % 32, and of the 16 tokens those
// that register order of a 32x32 result gives this lane's half: 4 h .. 4 h + 3, 8 + 4 h .. 8 + 4 h + 3.
__device__ __forceinline__ u32x4 value_fragment(const char* rows, int lane, int block) {
    const int h = lane >> 5, i = lane & 15, r = 4 * h + (i >> 2);
    const int c = 4 * block + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
    const uint32_t at = r * 256 + ((c ^ value_swizzle(r)) << 4) + (i & 1) * 8;
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(rows + at));
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(rows + at + 8 * 256));
    return __builtin_bit_cast(u32x4, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

}  // namespace sik
