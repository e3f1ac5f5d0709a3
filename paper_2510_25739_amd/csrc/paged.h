// What the kernels over a paged cache share: where an entry lies, which sequence a row belongs to, and values of the
// three types in 16-byte pieces.
#pragma once

#include "hawk_internal.h"

#include <algorithm>

namespace hawk {

// n / d for n below 2^31 and a d of the host's: with s = ceil(log2 d) and M = ceil(2^(31 + s) / d) < 2^32 the product n M / 2^(31 + s) is
// above n / d by less than 1 / d.
struct Divisor { unsigned magic; int shift, d; };   // shift < 0: d is one
inline Divisor divisor(int d) {
    int s = 0;
    while ((1ll << s) < d) ++s;
    return {(unsigned)(((1ull << (31 + s)) + d - 1) / d), s - 1, d};
}
__host__ __device__ inline int operator/(int n, const Divisor& d) {
    if (d.shift < 0) return n;
#if defined(__HIP_DEVICE_COMPILE__)
    return (int)(__umulhi((unsigned)n, d.magic) >> d.shift);
#else
    return (int)((((uint64_t)(unsigned)n * d.magic) >> 32) >> d.shift);
#endif
}

// One layer of a hawk_paged_cache as the kernels see it.
struct PagedView {
    char *k, *v;                 // of the layer
    int64_t page_stride, head_stride, entry_stride;   // elements
    const int32_t* table;
    int64_t table_stride;
    int n_pages, page_size, n_heads, hd, n_seq, max_pages, capacity;   // capacity: entries of a sequence's pages
    Divisor page;                // page_size
};
struct RowsView { const int32_t *row_start, *n_past; int rows; };
struct HeadsView { char* data; int64_t row_stride, head_stride; int n_heads, dtype; };

__host__ __device__ inline int page_of(const PagedView& c, int e) { return e / c.page; }
// Elements from the layer's start to entry e (head 0), given its page; -1 if there is no such page.
__host__ __device__ inline int64_t place_in(const PagedView& c, int page, int slot) {
    return page >= 0 && page < c.n_pages ? page * c.page_stride + slot * c.entry_stride : -1;
}
__host__ __device__ inline int64_t entry_at(const PagedView& c, const int32_t* table_row, int64_t e) {
    if (e < 0 || e >= c.capacity) return -1;
    const int p = page_of(c, (int)e);
    return place_in(c, table_row[p], (int)e - p * c.page_size);
}

inline bool is_type(int dtype) { return dtype == HAWK_FP32 || dtype == HAWK_BF16 || dtype == HAWK_FP16; }
inline size_t type_bytes(int dtype) { return dtype == HAWK_FP32 ? 4 : 2; }
// Whether rows a and rows b, each `rows` pieces of so many bytes that start so many bytes apart, have a byte in common.  Columns of one buffer
// lie between one another's rows and have none.
inline bool rows_meet(const void* a, int64_t a_step, int64_t a_bytes, const void* b, int64_t b_step, int64_t b_bytes, int rows) {
    const int64_t d = (int64_t)(reinterpret_cast<uintptr_t>(b) - reinterpret_cast<uintptr_t>(a)), last = rows - 1;
    if (rows < 2) a_step = b_step = 0;
    if (rows < 1 || d >= last * a_step + a_bytes || d + last * b_step + b_bytes <= 0) return false;
    // whether a step of a's, from the first to the last, starts in lo + 1 .. hi - 1
    auto starts = [&](int64_t lo, int64_t hi, int64_t first) {
        if (a_step == 0) return lo < 0 && hi > 0;
        const int64_t q = lo / a_step - (lo % a_step < 0 ? 1 : 0), k = std::max(q + 1, first);
        return k <= last && k * a_step < hi;
    };
    if (a_step == b_step) return starts(d - a_bytes, d + b_bytes, -last);
    for (int64_t i = 0; i <= last; ++i)
        if (starts(d + i * b_step - a_bytes, d + i * b_step + b_bytes, 0)) return true;
    return false;
}
bool paged_view(const hawk_paged_cache* c, int layer, PagedView* out);     // false: bad argument
bool heads_view(const hawk_heads* h, HeadsView* out);
// An output whose vectors do not overlap because of a stride alone.
inline bool room_for(const HeadsView& h, int rows, int hd) {
    return (rows < 2 || h.row_stride >= hd) && (h.n_heads < 2 || h.head_stride >= hd);
}
// No rows or no sequences: the buffers may be null.
inline bool nothing_to_do(const hawk_paged_cache* c, const hawk_paged_rows* r) { return c->n_seq == 0 || (r && r->rows == 0); }
inline bool rows_view(const hawk_paged_rows* r, RowsView* out) {
    if (!r || !r->row_start || !r->n_past || r->rows < 0) return false;
    out->row_start = r->row_start; out->n_past = r->n_past; out->rows = r->rows;
    return true;
}

int launch_rotary_table(float* table, int n_pos, int rot_dim, double theta, hipStream_t stream);
int launch_paged_append(const hawk_paged_cache* cache, int layer, const hawk_paged_rows* rows, const hawk_heads* q,
                        const hawk_heads* k, const hawk_heads* v, const float* q_gain, const float* k_gain, float eps,
                        const float* rot, int n_pos, int rot_dim, int pairs, const int32_t* pos, const hawk_heads* q_out,
                        hipStream_t stream);
int launch_paged_keep(const hawk_paged_cache* cache, const int32_t* n_past, const int32_t* path, const int32_t* n_keep,
                      int depth, hipStream_t stream);
size_t paged_pages_workspace_bytes(const hawk_paged_cache* cache);
int launch_paged_fork(const hawk_paged_cache* cache, int32_t* refs, int32_t* n_past, const int32_t* src, const int32_t* dst, int n, hipStream_t stream);
int launch_paged_take(const hawk_paged_cache* cache, int32_t* refs, const int32_t* n_past, const int32_t* n_new, int32_t* short_by, void* workspace,
                      size_t workspace_bytes, hipStream_t stream);
int launch_paged_trim(const hawk_paged_cache* cache, int32_t* refs, const int32_t* n_past, hipStream_t stream);
int launch_paged_compact(const hawk_paged_cache* cache, const int32_t* refs, int32_t* table_out, int64_t table_out_stride, int32_t* refs_out,
                         int32_t* n_used, void* workspace, size_t workspace_bytes, hipStream_t stream);
int launch_paged_copy(const hawk_paged_cache* from, const hawk_paged_cache* to, const int32_t* src, const int32_t* dst, int n, hipStream_t stream);
size_t paged_attention_workspace_bytes(const hawk_paged_cache* cache, int rows, int n_q_heads, int max_len);
int launch_paged_attention(const hawk_paged_cache* cache, int layer, const hawk_paged_rows* rows, const hawk_heads* q,
                           const uint64_t* tree, float scale, int max_len, const hawk_heads* out, void* workspace,
                           size_t workspace_bytes, hipStream_t stream);
// rules of the dispatch and of the kernels, for the tests as well
extern "C" int hawk_paged_attention_plan(int dtype, int n_seq, int rows, int n_heads, int n_q_heads, int hd, int capacity, int max_len);
extern "C" int hawk_paged_attention_row(const int32_t* row_start, int n_past, int s, int rows, int group, int capacity, int tile_log2, int tile, int r);

#if defined(__HIPCC__)
namespace {

typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef unsigned v2u __attribute__((ext_vector_type(2)));

// The last of n items whose key(i), ascending in i, is at most `at`; -1 if there is none.  One wave, the same answer in every
// lane: 64 keys are looked at in one step, so 4096 items take two dependent loads.
template <class K> __device__ __forceinline__ int last_not_above(int n, int lane, int64_t at, K key) {
    int lo = 0, len = n;
    for (;;) {
        const int step = (len + 63) >> 6, off = lane * step;
        const bool below = off < len && key(lo + off) <= at;
        const int c = __popcll(__ballot(below));
        if (c == 0) return lo == 0 ? -1 : lo - 1;   // (past the first step only where the keys do not ascend)
        lo += (c - 1) * step;
        if (step == 1) return lo;
        len = min(step, len - (c - 1) * step);
    }
}

// Eight or four consecutive values of any of the three types.
__device__ __forceinline__ float half_up(unsigned b) { return (float)__builtin_bit_cast(_Float16, (unsigned short)b); }
__device__ __forceinline__ void widen2(unsigned w, int dtype, float& a, float& b) {
    if (dtype == HAWK_BF16) {
        a = __uint_as_float(w << 16);
        b = __uint_as_float(w & 0xFFFF0000u);
    } else {
        a = half_up(w & 0xFFFFu);
        b = half_up(w >> 16);
    }
}
__device__ __forceinline__ unsigned narrow2(float a, float b, int dtype) {   // to nearest, ties to even
    typedef float f2 __attribute__((ext_vector_type(2)));
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    const f2 v = {a, b};
    return dtype == HAWK_BF16 ? __builtin_bit_cast(unsigned, __builtin_convertvector(v, b2)) : __builtin_bit_cast(unsigned, __builtin_convertvector(v, h2));
}
__device__ __forceinline__ void load4(const char* base, int64_t at, int dtype, float* x) {
    if (dtype == HAWK_FP32) {
        const float4 a = *reinterpret_cast<const float4*>(base + at * 4);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    } else {
        const v2u w = *reinterpret_cast<const v2u*>(base + at * 2);
        widen2(w[0], dtype, x[0], x[1]);
        widen2(w[1], dtype, x[2], x[3]);
    }
}
__device__ __forceinline__ void load8(const char* base, int64_t at, int dtype, float* x) {
    if (dtype == HAWK_FP32) {
        load4(base, at, dtype, x);
        load4(base, at + 4, dtype, x + 4);
    } else {
        const v4u w = *reinterpret_cast<const v4u*>(base + at * 2);
#pragma unroll
        for (int i = 0; i < 4; ++i) widen2(w[i], dtype, x[2 * i], x[2 * i + 1]);
    }
}
__device__ __forceinline__ void store4(char* base, int64_t at, int dtype, const float* x) {
    if (dtype == HAWK_FP32) *reinterpret_cast<float4*>(base + at * 4) = make_float4(x[0], x[1], x[2], x[3]);
    else *reinterpret_cast<v2u*>(base + at * 2) = (v2u){narrow2(x[0], x[1], dtype), narrow2(x[2], x[3], dtype)};
}
__device__ __forceinline__ void store8(char* base, int64_t at, int dtype, const float* x) {
    if (dtype == HAWK_FP32) {
        float4* d = reinterpret_cast<float4*>(base + at * 4);
        d[0] = make_float4(x[0], x[1], x[2], x[3]);
        d[1] = make_float4(x[4], x[5], x[6], x[7]);
    } else {
        v4u w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = narrow2(x[2 * i], x[2 * i + 1], dtype);
        *reinterpret_cast<v4u*>(base + at * 2) = w;
    }
}

}  // namespace
#endif

}  // namespace hawk
