// Low-rank adapters of many requests beside a shared projection: out[r] = base[r] + scale[a] B_a (A_a x[r]), a the adapter of row r's sequence.
//
// Rows are grouped by adapter into tiles of 16, once a step (the plan), so that an adapter that many requests use is read once for 16 of
// their rows.  One launch a projection: a workgroup has a tile and some of the columns.  Its waves share the sum over d_in - both
// operands of A x go from memory straight into the matrix units' registers, 16 bytes a lane -, their parts are added in shared memory, and
// B h is added to base on the way out.  Both products are computed transposed (h^T = A x^T, out^T = B h^T): a result lane then has neighbouring
// elements of one row.
#include "adapters.h"
#include "paged.h"

#include <algorithm>

namespace hawk {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));

constexpr int kTile = 16;            // rows of a tile
constexpr int kPlanThreads = 1024;
constexpr int kMostAdapters = 8192;

// The plan: [0] tiles in use, from kHead on for every tile its adapter (n_adapters: none) and 16 rows (-1: none), then a word pair a row
// that only its making uses.
constexpr int kHead = 4, kEntry = 1 + kTile;
__host__ __device__ inline int most_tiles(int rows, int n_adapters) { return rows / kTile + (rows < n_adapters + 1 ? rows : n_adapters + 1); }
__host__ __device__ inline size_t plan_words(int rows, int n_adapters) { return kHead + (size_t)most_tiles(rows, n_adapters) * kEntry; }

// Which rows have which adapter.  A row belongs to the last sequence that starts at or before it, if that one goes as far.  A row's number
// among its adapter's rows is whatever the counters give it: which rows share a tile has no part in any row's result.
__global__ __launch_bounds__(kPlanThreads) void adapter_plan_kernel(const int32_t* row_start, const int32_t* adapter, int n_seq, int rows, int n_adapters,
                                                                    int32_t* plan) {
    extern __shared__ int count[];   // [n_adapters + 1]: rows, then the first tile
    __shared__ int sums[kPlanThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, classes = n_adapters + 1;
    int2* place = reinterpret_cast<int2*>(plan + (plan_words(rows, n_adapters) + 1) / 2 * 2);
    for (int i = tid; i < classes; i += kPlanThreads) count[i] = 0;
    __syncthreads();
    for (int r = tid; r < rows; r += kPlanThreads) {
        int lo = 0, hi = n_seq;      // the last s with row_start[s] <= r lies in lo - 1 .. hi - 1
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (row_start[mid] <= r) lo = mid + 1;
            else hi = mid;
        }
        const int s = lo - 1;
        int which = -1, k = 0;
        if (s >= 0 && r < row_start[s + 1]) {
            which = adapter[s];
            if (which < 0 || which > n_adapters) which = n_adapters;
            // lanes of one adapter count together
            unsigned long long left = __ballot(1);
            while (left) {
                const int first = __ffsll((unsigned long long)left) - 1;
                const unsigned long long same = __ballot(which == __builtin_amdgcn_readlane(which, first)) & left;
                if ((same >> lane) & 1ull) {
                    int base = 0;
                    if (lane == first) base = atomicAdd(&count[which], __popcll(same));
                    k = __builtin_amdgcn_readlane(base, first) + __popcll(same & ((1ull << lane) - 1ull));
                }
                left &= ~same;
            }
        }
        place[r] = make_int2(which, k);
    }
    __syncthreads();
    int tiles = 0;                   // of the classes before
    for (int c0 = 0; c0 < classes; c0 += kPlanThreads) {
        const int c = c0 + tid, n = c < classes ? count[c] : 0, t = (n + kTile - 1) / kTile;
        int x = t;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int y = __shfl_up(x, d);
            if (lane >= d) x += y;
        }
        if (lane == 63) sums[wave] = x;
        __syncthreads();
        int before = tiles, all = 0;
        for (int w = 0; w < kPlanThreads / 64; ++w) {
            before += w < wave ? sums[w] : 0;
            all += sums[w];
        }
        before += x - t;
        for (int i = 0; i < t; ++i) plan[kHead + (before + i) * kEntry] = c;
        for (int i = n; i < t * kTile; ++i) plan[kHead + (before + i / kTile) * kEntry + 1 + i % kTile] = -1;
        if (c < classes) count[c] = before;
        tiles += all;
        __syncthreads();
    }
    if (tid == 0) plan[0] = tiles;
    for (int r = tid; r < rows; r += kPlanThreads) {
        const int2 p = place[r];
        if (p.x >= 0) plan[kHead + (count[p.x] + p.y / kTile) * kEntry + 1 + p.y % kTile] = r;
    }
}

struct ApplyArgs {
    const int32_t* plan;
    const char *a, *b, *x, *base;
    char* out;
    const float* scale;
    int64_t a_adapter, a_row, b_adapter, b_row, x_row, base_row, out_row;   // elements
    int n_adapters, rank, d_in, d_out, rows, tiles, out_type;
    Divisor parts;                   // workgroups of a tile
};

template <int TYPE> struct Of;
template <> struct Of<HAWK_BF16> {
    static constexpr int kBytes = 2;
    static __device__ __forceinline__ f32x4 mul(v4u a, v4u b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
    }
};
template <> struct Of<HAWK_FP16> {
    static constexpr int kBytes = 2;
    static __device__ __forceinline__ f32x4 mul(v4u a, v4u b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
    }
};
template <> struct Of<HAWK_FP32> {
    static constexpr int kBytes = 4;
    static __device__ __forceinline__ f32x4 mul(v4u a, v4u b, f32x4 c) {   // element i of a lane's piece is step i's
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[i]), __uint_as_float(b[i]), c, 0, 0, 0);
        return c;
    }
};

// h of 32 bits as a sum of P numbers of the operands' type, each what is left rounded to nearest.  bf16: 8 bits and half a step a part; two
// parts are off by 2^-16 of h, a 256th of what rounding the result to 16 bits is, three, for results of 32 bits, by 2^-24.  fp16: 11 bits a
// part, of h scaled to below 2^14 (see below).  An infinity is its own first part, and nothing is rounded to one.
template <int TYPE> __device__ __forceinline__ unsigned short cut(float& x) {
    unsigned short u;
    float y;
    if (TYPE == HAWK_BF16) {
        u = __builtin_bit_cast(unsigned short, (__bf16)x);
        if ((u & 0x7FFF) == 0x7F80) u = (unsigned short)(__float_as_uint(x) >> 16);
        y = __uint_as_float((unsigned)u << 16);
    } else {
        const _Float16 f = (_Float16)x;
        u = __builtin_bit_cast(unsigned short, f);
        y = (float)f;
    }
    x = fabsf(y) <= 3.4028235e38f ? x - y : 0.f;
    return u;
}

// NR: groups of 16 of the rank.  P: parts of h.  NW waves.
template <int TYPE, int NR, int P, int NW>
__global__ __launch_bounds__(64 * NW, NR <= 4 ? 4 : 2) void adapter_apply_kernel(ApplyArgs a) {
    using T = Of<TYPE>;
    constexpr int ES = T::kBytes, VEC = 16 / ES, STEP = 4 * VEC;               // features of a lane's piece, of a product
    constexpr int RP = 16 * NR, LD = RP + 4;                                   // the rank, rounded up
    constexpr bool PAIR = TYPE != HAWK_FP32 && NR == 1;                        // two parts of h share a product's 32 features
    constexpr int KS = TYPE == HAWK_FP32 ? NR : (NR + 1) / 2;                  // products over the rank
    constexpr int PP = PAIR ? (P + 1) / 2 : P;
    __shared__ float parts[NW][NR][kTile][16];                                 // [wave][..][row][..]
    __shared__ float h[kTile][LD];
    __shared__ float factor[kTile];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), m16 = lane & 15, g = lane >> 4;
    const int part = (int)blockIdx.x / a.tiles, tile = (int)blockIdx.x - part * a.tiles;
    if (tile >= a.plan[0]) return;
    const int32_t* entry = a.plan + kHead + tile * kEntry;
    const int who = __builtin_amdgcn_readfirstlane(entry[0]);
    int row = entry[1 + m16];
    if (row >= a.rows) row = -1;
    const bool none = who < 0 || who >= a.n_adapters;
    if (none && a.base == a.out) return;
    const int64_t at = row < 0 ? 0 : row;

    f32x4 acc[NR];
#pragma unroll
    for (int j = 0; j < NR; ++j) acc[j] = (f32x4){0.f, 0.f, 0.f, 0.f};
    if (!none) {
        const char* x = a.x + at * a.x_row * ES;
        const char* w = a.a + (who * a.a_adapter + m16 * a.a_row) * ES;
        for (int k0 = wave * STEP; k0 < a.d_in; k0 += NW * STEP) {
            const int k = k0 + g * VEC;
            v4u xv = {0u, 0u, 0u, 0u};
            const bool there = k < a.d_in;
            if (there && row >= 0) xv = *reinterpret_cast<const v4u*>(x + (int64_t)k * ES);
#pragma unroll
            for (int j = 0; j < NR; ++j) {
                v4u wv = {0u, 0u, 0u, 0u};
                if (there && j * 16 + m16 < a.rank) wv = *reinterpret_cast<const v4u*>(w + (j * 16 * a.a_row + k) * ES);
                acc[j] = T::mul(wv, xv, acc[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < NR; ++j) *reinterpret_cast<f32x4*>(&parts[wave][j][m16][4 * g]) = acc[j];
    }
    __syncthreads();
    if (!none) {
        for (int i = threadIdx.x; i < kTile * RP; i += 64 * NW) {
            const int j = i / (kTile * 16), r = (i >> 4) & 15, c = i & 15;
            float s = 0.f;
#pragma unroll
            for (int v = 0; v < NW; ++v) s += parts[v][j][r][c];
            h[r][j * 16 + c] = j * 16 + c < a.rank ? s : 0.f;   // (zero weights of an infinite x are no zeros)
        }
    }
    __syncthreads();
    // scale[a], and of fp16 the power of two that brings a row's largest h below 2^14: half a step of a part of the smallest is then
    // 2^-39 of the largest, and nothing overflows
    if (threadIdx.x < 64) {
        float top = 0.f;
        if (TYPE == HAWK_FP16 && !none)
            for (int j = g; j < RP; j += 4) {
                const float v = fabsf(h[m16][j]);
                top = fmaxf(top, v <= 3.4028235e38f ? v : 0.f);
            }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        int e = 0;
        if (TYPE == HAWK_FP16 && top > 0.f) e = max(ilogbf(top) - 13, -126);
        if (lane < kTile) factor[lane] = __uint_as_float((unsigned)(e + 127) << 23);
    }
    __syncthreads();
    v4u hv[PP][KS];
    const float up = factor[m16], s = none ? 0.f : (a.scale ? a.scale[who] * up : up), down = 1.f / up;
    if (TYPE == HAWK_FP32) {
#pragma unroll
        for (int k = 0; k < KS; ++k) hv[0][k] = *reinterpret_cast<const v4u*>(&h[m16][k * 16 + 4 * g]);
    } else {
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            unsigned short bits[4][8];   // [part]
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int j = k * 32 + 8 * (PAIR ? g & 1 : g) + i;
                float v = j < RP ? h[m16][j] * down : 0.f;
#pragma unroll
                for (int p = 0; p < 4; ++p) bits[p][i] = p < P ? cut<TYPE>(v) : 0;
            }
#pragma unroll
            for (int p = 0; p < PP; ++p)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const unsigned low = bits[PAIR ? 2 * p : p][2 * i] | (unsigned)bits[PAIR ? 2 * p : p][2 * i + 1] << 16;
                    const unsigned high = PAIR ? bits[2 * p + 1][2 * i] | (unsigned)bits[2 * p + 1][2 * i + 1] << 16 : 0u;
                    hv[p][k][i] = PAIR && g >= 2 ? high : low;
                }
        }
    }

    // 64 columns a wave: row mu of block i of the product stands for column 16 (mu / 4) + 4 i + mu % 4, so that a lane's results are 16 neighbours
    const char* wb = none ? nullptr : a.b + who * a.b_adapter * ES;
    const int od = a.out_type, groups = (a.d_out + 63) >> 6;
    for (int q = part * NW + wave; q < groups; q += a.parts.d * NW) {
        const int c0 = q * 64, mine = c0 + 16 * g;
        f32x4 o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
        if (!none) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int c = c0 + 16 * (m16 >> 2) + 4 * i + (m16 & 3);
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    const int j = PAIR ? 8 * (g & 1) : k * STEP + VEC * g;
                    v4u wv = {0u, 0u, 0u, 0u};
                    if (c < a.d_out && j < a.rank) wv = *reinterpret_cast<const v4u*>(wb + (c * a.b_row + j) * ES);
#pragma unroll
                    for (int p = 0; p < PP; ++p) o[i] = T::mul(wv, hv[p][k], o[i]);
                }
            }
        }
        if (row < 0) continue;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (mine + 8 * i >= a.d_out) continue;
            float y[8];
            if (a.base) load8(a.base, at * a.base_row + mine + 8 * i, od, y);
            else {
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = 0.f;
            }
            if (!none) {
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = fmaf(o[2 * i + (e >> 2)][e & 3], s, y[e]);
            }
            store8(a.out, at * a.out_row + mine + 8 * i, od, y);
        }
    }
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
int status() { return hipGetLastError() == hipSuccess ? HAWK_OK : HAWK_EDEVICE; }
bool matrix_ok(const hawk_matrix* m, int width) {
    return m && m->data && aligned16(m->data) && is_type(m->dtype) && !(m->row_stride & 7) && m->row_stride >= 0 && width > 0;
}

template <int TYPE, int NR, int P> void launch_of(const ApplyArgs& a, unsigned grid, hipStream_t stream) {
    adapter_apply_kernel<TYPE, NR, P, 8><<<grid, 512, 0, stream>>>(a);
}
template <int TYPE, int P> void launch_rank(const ApplyArgs& a, unsigned grid, hipStream_t stream) {
    if (a.rank <= 16) launch_of<TYPE, 1, P>(a, grid, stream);
    else if (a.rank <= 32) launch_of<TYPE, 2, P>(a, grid, stream);
    else if (a.rank <= 64) launch_of<TYPE, 4, P>(a, grid, stream);
    else launch_of<TYPE, 8, P>(a, grid, stream);
}

}  // namespace

size_t adapter_plan_bytes(int rows, int n_adapters) {
    if (rows < 0 || rows > (1 << 22) || n_adapters < 0 || n_adapters > kMostAdapters) return 0;
    return ((plan_words(rows, n_adapters) + 1) / 2 * 2 + 2 * (size_t)rows) * sizeof(int32_t);
}

int launch_adapter_plan(const int32_t* row_start, const int32_t* adapter, int n_seq, int rows, int n_adapters, void* plan, size_t plan_bytes,
                        hipStream_t stream) {
    const size_t need = adapter_plan_bytes(rows, n_adapters);
    if (need == 0 || n_seq < 0 || !plan || !aligned16(plan) || (n_seq > 0 && (!row_start || !adapter))) return HAWK_EINVAL;
    if (plan_bytes < need) return HAWK_ENOMEM;
    adapter_plan_kernel<<<1, kPlanThreads, (size_t)(n_adapters + 1) * sizeof(int), stream>>>(row_start, adapter, n_seq, rows, n_adapters, static_cast<int32_t*>(plan));
    return status();
}

int launch_adapter_apply(const hawk_adapters* w, const void* plan, size_t plan_bytes, int rows, const hawk_matrix* x, const hawk_matrix* base,
                         const hawk_matrix* out, hipStream_t stream) {
    if (!w || rows < 0 || !is_type(w->dtype) || w->n_adapters < 0 || w->rank < 8 || w->rank > 128 || w->rank % 8 || w->d_in < 8 || w->d_in % 8 ||
        w->d_out < 8 || w->d_out % 8 || w->d_in > (1 << 24) || w->d_out > (1 << 24))
        return HAWK_EINVAL;
    if ((w->a_adapter_stride | w->a_row_stride | w->b_adapter_stride | w->b_row_stride) & 7) return HAWK_EINVAL;
    if (w->a_adapter_stride < 0 || w->b_adapter_stride < 0 || w->a_row_stride < w->d_in || w->b_row_stride < w->rank) return HAWK_EINVAL;
    const size_t need = adapter_plan_bytes(rows, w->n_adapters);
    if (need == 0) return HAWK_EINVAL;
    if (rows == 0) return HAWK_OK;
    if (w->n_adapters > 0 && (!w->a || !w->b || !aligned16(w->a) || !aligned16(w->b))) return HAWK_EINVAL;
    if (!matrix_ok(x, w->d_in) || !matrix_ok(out, w->d_out) || (base && !matrix_ok(base, w->d_out))) return HAWK_EINVAL;
    if (x->dtype != w->dtype || (base && base->dtype != out->dtype) || (rows > 1 && out->row_stride < w->d_out)) return HAWK_EINVAL;
    if (base && base->data == out->data && rows > 1 && base->row_stride != out->row_stride) return HAWK_EINVAL;
    if (!plan || !aligned16(plan)) return HAWK_EINVAL;
    if (plan_bytes < need) return HAWK_ENOMEM;
    ApplyArgs a = {};
    a.plan = static_cast<const int32_t*>(plan);
    a.a = static_cast<const char*>(w->a); a.b = static_cast<const char*>(w->b); a.scale = w->scale;
    a.x = static_cast<const char*>(x->data); a.base = base ? static_cast<const char*>(base->data) : nullptr; a.out = static_cast<char*>(out->data);
    a.a_adapter = w->a_adapter_stride; a.a_row = w->a_row_stride; a.b_adapter = w->b_adapter_stride; a.b_row = w->b_row_stride;
    a.x_row = x->row_stride; a.base_row = base ? base->row_stride : 0; a.out_row = out->row_stride;
    a.n_adapters = w->n_adapters; a.rank = w->rank; a.d_in = w->d_in; a.d_out = w->d_out; a.rows = rows; a.out_type = out->dtype;
    a.tiles = most_tiles(rows, w->n_adapters);
    const int groups = (a.d_out + 63) / 64;
    const int parts = std::max(1, std::min((groups + 7) / 8, 512 / std::max(1, a.tiles)));
    a.parts = divisor(parts);
    const int64_t grid = (int64_t)a.tiles * parts;
    if (grid > (1 << 22)) return HAWK_EINVAL;
    const bool exact = out->dtype == HAWK_FP32;
    if (w->dtype == HAWK_FP32) launch_rank<HAWK_FP32, 1>(a, (unsigned)grid, stream);
    else if (w->dtype == HAWK_BF16) exact ? launch_rank<HAWK_BF16, 3>(a, (unsigned)grid, stream) : launch_rank<HAWK_BF16, 2>(a, (unsigned)grid, stream);
    else launch_rank<HAWK_FP16, 2>(a, (unsigned)grid, stream);
    return status();
}

}  // namespace hawk
