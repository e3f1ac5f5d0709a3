// Attention of a step's rows over the pages of hawk_paged_cache.
//
// With S = scale Q K^T over the entries a row sees, out = softmax(S) V in one pass over the entries: a running maximum
// m and sum l per row, results rescaled when the maximum grows.  Everything is computed transposed, S^T = K Q^T and
// out^T = V^T P^T: a result lane of the matrix unit then holds one row's scores of four entries, which is what the next
// product takes as its operand if its entries are named in that order - the weights stay in the registers they are computed
// in, and a row's maximum, sum and rescaling are one value per lane.  Query heads that share a cache head are rows of the
// same tile: row r of a tile is (row of the sequence r / group, head r % group).
#include "paged.h"

namespace hawk {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));

constexpr int kTile = 16;      // rows of a tile
constexpr int kKeys = 32;      // entries of one turn of a wave

struct AttnArgs {
    PagedView c;
    RowsView r;
    HeadsView q, out;
    const uint64_t* tree;
    float scale2;              // scale * log2(e)
    int group, tiles;          // query heads of a cache head; tiles of the launch
    int splits, split_keys;    // parts of a long axis, entries of a part (the last one has the rest)
    float *part, *part_ml;     // [split][row][head][hd], [split][row][head][2]
};

// Which entries the rows of a tile are about.
struct Span {
    int s, r0, n;              // sequence, its first row, its rows
    int past;                  // committed entries (clamped to what an entry number can be)
    int end;                   // entries behind this one are seen by no row of the tile
    int all;                   // entries before this one are seen by every row of the tile
};
__device__ __forceinline__ Span span_of(const AttnArgs& a, int s, int first) {   // first: the tile's first row * group + head
    Span t;
    t.s = s;
    const int b = min(max(a.r.row_start[s], 0), a.r.rows), e = min(max(a.r.row_start[s + 1], 0), a.r.rows);
    t.r0 = b;
    t.n = max(e - b, 0);
    t.past = min(max(a.r.n_past[s], -(1 << 30)), 1 << 30);
    const int cap = a.c.max_pages * a.c.page_size;
    const int lo = first / a.group, hi = min((first + kTile - 1) / a.group, t.n - 1);
    if (a.tree) {
        t.end = t.past + max(min(t.n, 64), hi + 1);
        t.all = t.past;
    } else {
        t.end = t.past + hi + 1;
        t.all = t.past + lo + 1;
    }
    t.end = max(min(t.end, cap), 0);
    return t;
}
// Tiles are counted so that a sequence's first tile follows from its first row alone: base(s) = row_start[s] * group / 16 + s,
// which leaves every sequence room for its tiles and at most one unused number per sequence.
__device__ __forceinline__ int tile_base(const AttnArgs& a, int s) {
    const int64_t b = min(max(a.r.row_start[s], 0), a.r.rows);
    return (int)(b * a.group / kTile) + s;
}
__device__ __forceinline__ int used_splits(const AttnArgs& a, int end) {
    return min(a.splits, max(1, (end + a.split_keys - 1) / a.split_keys));
}

__device__ __forceinline__ float swap16(float v, bool add) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    const float x = __uint_as_float(r[0]), y = __uint_as_float(r[1]);
    return add ? x + y : fmaxf(x, y);
}
__device__ __forceinline__ float swap32(float v, bool add) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    const float x = __uint_as_float(r[0]), y = __uint_as_float(r[1]);
    return add ? x + y : fmaxf(x, y);
}
__device__ __forceinline__ float row_max(float v) { return swap32(swap16(v, false), false); }   // over the four lanes of a row
__device__ __forceinline__ float row_sum(float v) { return swap32(swap16(v, true), true); }

template <int TYPE> struct Of;
template <> struct Of<HAWK_BF16> {
    static constexpr int kBytes = 2;
    static constexpr float kLift = 0.f;
    static __device__ __forceinline__ f32x4 mul(v4u a, v4u b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ unsigned short narrow(float x) { return __builtin_bit_cast(unsigned short, (__bf16)x); }
    static __device__ __forceinline__ float widen(unsigned short b) { return __uint_as_float((unsigned)b << 16); }
    static __device__ __forceinline__ bool odd(unsigned w) { return (w & 0x7F80u) == 0x7F80u || (w & 0x7F800000u) == 0x7F800000u; }
    static __device__ __forceinline__ unsigned clear(unsigned w) {
        return ((w & 0x7F80u) == 0x7F80u ? 0u : w & 0xFFFFu) | ((w & 0x7F800000u) == 0x7F800000u ? 0u : w & 0xFFFF0000u);
    }
};
template <> struct Of<HAWK_FP16> {
    static constexpr int kBytes = 2;
    static constexpr float kLift = 14.f;   // weights are 2^14 exp2(..): halves of small ones would be subnormal
    static __device__ __forceinline__ f32x4 mul(v4u a, v4u b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ unsigned short narrow(float x) { return __builtin_bit_cast(unsigned short, (_Float16)x); }
    static __device__ __forceinline__ float widen(unsigned short b) { return half_up(b); }
    static __device__ __forceinline__ bool odd(unsigned w) { return (w & 0x7C00u) == 0x7C00u || (w & 0x7C000000u) == 0x7C000000u; }
    static __device__ __forceinline__ unsigned clear(unsigned w) {
        return ((w & 0x7C00u) == 0x7C00u ? 0u : w & 0xFFFFu) | ((w & 0x7C000000u) == 0x7C000000u ? 0u : w & 0xFFFF0000u);
    }
};
template <> struct Of<HAWK_FP32> {
    static constexpr int kBytes = 4;
    static constexpr float kLift = 0.f;
    // four steps of 16 x 16 x 4: element i of a lane's piece is the step's, so the features of a step are four apart
    static __device__ __forceinline__ f32x4 mul(v4u a, v4u b, f32x4 c) {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[i]), __uint_as_float(b[i]), c, 0, 0, 0);
        return c;
    }
    static __device__ __forceinline__ bool odd(unsigned w) { return (w & 0x7F800000u) == 0x7F800000u; }
    static __device__ __forceinline__ unsigned clear(unsigned w) { return odd(w) ? 0u : w; }
};

// Tile of 16 rows, NW waves that share the entries of its part in turns of 32.  Keys and values go from the pages straight into the
// operands' registers: a lane's 16 bytes of a key are its features of one product, and its piece of eight keys' values
// - the same few features of each - become the transposed operand by pairing words of two keys.
template <int TYPE, int DP, bool PAD, int NW>
__global__ __launch_bounds__(64 * NW) void paged_rows_kernel(AttnArgs a) {
    using T = Of<TYPE>;
    constexpr int ES = T::kBytes, VEC = 16 / ES, STEP = 4 * VEC, NS = DP / STEP;   // features of a lane's piece, of a product; products
    constexpr int VD = DP / 16, VC = VD < VEC ? VD : VEC, NC = VD / VC;            // a lane's features of a value, per piece; pieces
    constexpr int VW = VC * ES / 4;                                                // words of a piece
    constexpr int COLS = 16 * VC;                                                  // features of a round of pieces
    __shared__ float lo[NW][kTile][COLS + 4];
    __shared__ float lm[NW][kTile], ll[NW][kTile];

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m16 = lane & 15, g = lane >> 4;
    const int head = blockIdx.x % a.c.n_heads, rest = blockIdx.x / a.c.n_heads;
    const int split = rest % a.splits, tile = a.tiles - 1 - rest / a.splits;   // later tiles see more: they start first
    const int s = last_not_above(a.c.n_seq, lane, tile, [&](int i) { return (int64_t)tile_base(a, i); });
    if (s < 0) return;
    const int first = (tile - tile_base(a, s)) * kTile;
    const Span t = span_of(a, s, first);
    if (first >= t.n * a.group || split >= used_splits(a, t.end)) return;
    const int k0 = split * a.split_keys, k1 = split == a.splits - 1 ? t.end : min(t.end, k0 + a.split_keys);
    const int hd = a.c.hd;

    // this lane's row: its query, and what it sees
    const int pr = first + m16, i = pr / a.group;
    const bool real = pr < t.n * a.group;
    const int row = t.r0 + (real ? i : 0), qh = head * a.group + (real ? pr - i * a.group : 0);
    const int own = t.past + i;   // the row's own entry, the last one it sees of a chain
    const unsigned long long bits = a.tree && real ? a.tree[row] : 0ull;
    v4u q[NS];
#pragma unroll
    for (int ks = 0; ks < NS; ++ks) {
        q[ks] = (v4u){0u, 0u, 0u, 0u};
        const int f = ks * STEP + g * VEC;
        if (real && (!PAD || f < hd)) q[ks] = *reinterpret_cast<const v4u*>(a.q.data + ((int64_t)row * a.q.row_stride + (int64_t)qh * a.q.head_stride + f) * ES);
    }

    f32x4 o[VD];
#pragma unroll
    for (int d = 0; d < VD; ++d) o[d] = (f32x4){0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    const int32_t* pages = a.c.table + (int64_t)t.s * a.c.table_stride;
    const char *kh = a.c.k + (int64_t)head * a.c.head_stride * ES, *vh = a.c.v + (int64_t)head * a.c.head_stride * ES;
    const bool quads = (a.c.page_size & 3) == 0;

    for (int kb = k0 + kKeys * wave; kb < k1; kb += kKeys * NW) {
        int64_t at[2], vat[2][4];   // places of the lane's keys, and of the entries whose scores and values it has
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            const int e = kb + kt * 16 + m16;
            at[kt] = e < k1 ? entry_at(a.c, pages, e) : -1;
            const int e0 = kb + kt * 16 + g * 4;
            if (quads) {   // four entries from a multiple of four on lie in one page
                const int64_t p = e0 < k1 ? entry_at(a.c, pages, e0) : -1;
#pragma unroll
                for (int r = 0; r < 4; ++r) vat[kt][r] = p >= 0 && e0 + r < k1 ? p + r * a.c.entry_stride : -1;
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r) vat[kt][r] = e0 + r < k1 ? entry_at(a.c, pages, e0 + r) : -1;
            }
        }
        const bool full = kb + kKeys <= t.all && kb + kKeys <= k1 && !__any(at[0] < 0 || at[1] < 0);
        v4u k[2][NS];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int ks = 0; ks < NS; ++ks) {   // (an entry that does not exist reads entry 0 of page 0: its score is dropped)
                const int f = ks * STEP + g * VEC;
                k[kt][ks] = (v4u){0u, 0u, 0u, 0u};
                if (!PAD || f < hd) k[kt][ks] = *reinterpret_cast<const v4u*>(kh + (max(at[kt], (int64_t)0) + f) * ES);
            }
        unsigned v[2][4][NC][VW];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    const int f = c * COLS + m16 * VC;
                    const unsigned* src = reinterpret_cast<const unsigned*>(vh + (max(vat[kt][r], (int64_t)0) + f) * ES);
                    typedef unsigned piece __attribute__((ext_vector_type(VW)));
                    piece w = {};
                    if (!PAD || f < hd) w = *reinterpret_cast<const piece*>(src);
#pragma unroll
                    for (int x = 0; x < VW; ++x) v[kt][r][c][x] = w[x];
                }
        f32x4 sc[2];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            sc[kt] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < NS; ++ks) sc[kt] = T::mul(k[kt][ks], q[ks], sc[kt]);
            sc[kt] *= a.scale2;
        }
        unsigned seen = 0xFFu;   // bit kt * 4 + r
        if (!full) {
            seen = 0u;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int e = kb + kt * 16 + g * 4 + r;
                    const bool see = real && vat[kt][r] >= 0 &&
                                     (a.tree ? e < t.past || e == own || (e - t.past < 64 && ((bits >> (e - t.past)) & 1ull)) : e <= own);
                    seen |= see ? 1u << (kt * 4 + r) : 0u;
                    if (!see) sc[kt][r] = -INFINITY;
                }
        }
        float top = m;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int r = 0; r < 4; ++r) top = fmaxf(top, sc[kt][r]);
        top = row_max(top);
        const float base = top == -INFINITY ? 0.f : top, shrink = __builtin_amdgcn_exp2f(m - base);
        m = top;
        float p[2][4], sum = 0.f;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                p[kt][r] = __builtin_amdgcn_exp2f(sc[kt][r] - base + T::kLift);
                sum += p[kt][r];
            }
        l = l * shrink + sum;
#pragma unroll
        for (int d = 0; d < VD; ++d) o[d] *= shrink;

        if (!full) {   // values of entries that do not exist are nothing, and infinities and NaN must not meet a weight of zero
            bool odd = false;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int c = 0; c < NC; ++c)
#pragma unroll
                        for (int x = 0; x < VW; ++x) {
                            if (vat[kt][r] < 0) v[kt][r][c][x] = 0u;
                            odd = odd || T::odd(v[kt][r][c][x]);
                        }
            if (__any(odd)) {   // they are added one by one to the rows that see them, and are zero in the product
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        for (int from = 0; from < 64; from += 16) {
                            const float w = __shfl(p[kt][r], from + m16);
                            const bool see = (__shfl((int)seen, from + m16) >> (kt * 4 + r)) & 1;
                            const int64_t place = __shfl((long long)vat[kt][r], from);
                            if (place < 0) continue;
#pragma unroll
                            for (int d = 0; d < VD; ++d)
#pragma unroll
                                for (int y = 0; y < 4; ++y) {
                                    const int f = (d / VC) * COLS + (g * 4 + y) * VC + d % VC;
                                    float x = 0.f;
                                    if (!PAD || f < hd) {
                                        if constexpr (TYPE == HAWK_FP32) x = *reinterpret_cast<const float*>(vh + (place + f) * ES);
                                        else x = T::widen(*reinterpret_cast<const unsigned short*>(vh + (place + f) * ES));
                                    }
                                    if (see && !(fabsf(x) <= 3.4028235e38f)) o[d][y] += w * x;
                                }
                        }
#pragma unroll
                        for (int c = 0; c < NC; ++c)
#pragma unroll
                            for (int x = 0; x < VW; ++x) v[kt][r][c][x] = T::clear(v[kt][r][c][x]);
                    }
            }
        }

        if constexpr (TYPE == HAWK_FP32) {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int d = 0; d < VD; ++d)
                        o[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[kt][r][d / VC][d % VC]), p[kt][r], o[d], 0, 0, 0);
        } else {
            // the weights as two values of the type, the second the first one's remainder: about 16 bits
            unsigned short hi[8], low[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                hi[j] = T::narrow(p[j >> 2][j & 3]);
                low[j] = T::narrow(p[j >> 2][j & 3] - T::widen(hi[j]));
            }
            v4u ph, pl;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                ph[j] = hi[2 * j] | ((unsigned)hi[2 * j + 1] << 16);
                pl[j] = low[2 * j] | ((unsigned)low[2 * j + 1] << 16);
            }
#pragma unroll
            for (int d = 0; d < VD; ++d) {
                v4u w;
#pragma unroll
                for (int j = 0; j < 4; ++j) {   // feature d of entries 2 j and 2 j + 1
                    const unsigned x = v[j >> 1][2 * j & 3][d / VC][(d % VC) >> 1], y = v[j >> 1][(2 * j & 3) + 1][d / VC][(d % VC) >> 1];
                    w[j] = __builtin_amdgcn_perm(y, x, (d & 1) ? 0x07060302u : 0x05040100u);
                }
                o[d] = T::mul(w, pl, o[d]);
                o[d] = T::mul(w, ph, o[d]);
            }
        }
    }

    // the waves' parts: maximum and sum, then the results in rounds of COLS features
    l = row_sum(l);
    if (g == 0) {
        lm[wave][m16] = m;
        ll[wave][m16] = l;
    }
    __syncthreads();
    float mt = -INFINITY, lt = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) mt = fmaxf(mt, lm[w][m16]);
    const float base = mt == -INFINITY ? 0.f : mt;
#pragma unroll
    for (int w = 0; w < NW; ++w) lt += ll[w][m16] * __builtin_amdgcn_exp2f(lm[w][m16] - base);
    const float mine = __builtin_amdgcn_exp2f(m - base);
    const bool whole = a.splits == 1;
    const float norm = whole ? (lt == 0.f ? 0.f : 1.f / lt) : 1.f;
    if (!whole && real && wave == 0 && g == 0) {
        float* ml = a.part_ml + (((int64_t)split * a.r.rows + row) * a.q.n_heads + qh) * 2;
        ml[0] = mt;
        ml[1] = lt;
    }
    for (int c = 0; c < NC; ++c) {
        if (c > 0) __syncthreads();
#pragma unroll
        for (int cc = 0; cc < NC; ++cc)
            if (cc == c) {
#pragma unroll
                for (int y = 0; y < 4; ++y)
#pragma unroll
                    for (int d = 0; d < VC; ++d) lo[wave][m16][(g * 4 + y) * VC + d] = o[cc * VC + d][y] * mine * norm;
            }
        __syncthreads();
        // eight features of a row per thread
        for (int u = threadIdx.x; u < kTile * (COLS / 8); u += 64 * NW) {
            const int rr = u / (COLS / 8), f = (u % (COLS / 8)) * 8, ff = c * COLS + f, prr = first + rr;
            if (prr >= t.n * a.group || (PAD && ff >= hd)) continue;
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] = 0.f;
#pragma unroll
                for (int w = 0; w < NW; ++w) x[e] += lo[w][rr][f + e];
            }
            const int ri = prr / a.group;
            const int64_t orow = t.r0 + ri, oh = head * a.group + prr - ri * a.group;
            if (whole)
                store8(a.out.data, orow * a.out.row_stride + oh * a.out.head_stride + ff, a.out.dtype, x);
            else
                store8(reinterpret_cast<char*>(a.part), (((int64_t)split * a.r.rows + orow) * a.q.n_heads + oh) * hd + ff, HAWK_FP32, x);
        }
    }
}

// Joins the parts of a long axis: a wave per (row, head).
__global__ __launch_bounds__(256) void paged_join_kernel(AttnArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int row = (int)(unit / a.q.n_heads), qh = (int)(unit - (int64_t)row * a.q.n_heads);
    if (row >= a.r.rows) return;
    const int s = last_not_above(a.c.n_seq, lane, row, [&](int i) { return (int64_t)a.r.row_start[i]; });
    if (s < 0 || row >= a.r.row_start[s + 1]) return;
    const int first = ((row - max(a.r.row_start[s], 0)) * a.group + qh % a.group) / kTile * kTile;
    const Span t = span_of(a, s, first);
    const int n = used_splits(a, t.end);
    float mt = -INFINITY, lt = 0.f;
    for (int i = 0; i < n; ++i) mt = fmaxf(mt, a.part_ml[(((int64_t)i * a.r.rows + row) * a.q.n_heads + qh) * 2]);
    const float base = mt == -INFINITY ? 0.f : mt;
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const int f = lane * 8;
    for (int i = 0; i < n; ++i) {
        const int64_t at = ((int64_t)i * a.r.rows + row) * a.q.n_heads + qh;
        const float w = __builtin_amdgcn_exp2f(a.part_ml[at * 2] - base);
        lt += a.part_ml[at * 2 + 1] * w;
        if (f < a.c.hd) {
            float y[8];
            load8(reinterpret_cast<const char*>(a.part), at * a.c.hd + f, HAWK_FP32, y);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] += y[e] * w;
        }
    }
    if (f >= a.c.hd) return;
    const float norm = lt == 0.f ? 0.f : 1.f / lt;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= norm;
    store8(a.out.data, (int64_t)row * a.out.row_stride + (int64_t)qh * a.out.head_stride + f, a.out.dtype, x);
}

struct Plan { int tiles, splits, split_keys; size_t part_bytes, ml_bytes; };

// How a call is cut: parts of the long axis where the tiles alone would leave most of the chip's 256 units idle.
Plan plan_of(int n_seq, int rows, int n_heads, int n_q_heads, int hd, int64_t capacity, int max_len) {
    Plan p;
    const int group = n_q_heads / n_heads;
    p.tiles = (int)((int64_t)rows * group / kTile) + n_seq;
    const int64_t len = max_len < 1 || max_len > capacity ? capacity : max_len, blocks = (int64_t)p.tiles * n_heads;
    int64_t parts = 1024 / (blocks < 1 ? 1 : blocks);
    const int64_t most = len / 512;
    if (parts > most) parts = most;
    if (parts > 64) parts = 64;
    if (parts < 1) parts = 1;
    int64_t keys = (len + parts - 1) / parts;
    keys = (keys + 127) / 128 * 128;
    p.splits = (int)((len + keys - 1) / keys);
    if (p.splits < 1) p.splits = 1;
    p.split_keys = (int)keys;
    const size_t vectors = p.splits > 1 ? (size_t)p.splits * rows * n_q_heads : 0;
    p.part_bytes = (vectors * hd * sizeof(float) + 15) / 16 * 16;
    p.ml_bytes = (vectors * 2 * sizeof(float) + 15) / 16 * 16;
    return p;
}

bool shape_ok(const PagedView& c, int rows, int n_q_heads) {
    return rows >= 0 && n_q_heads >= 1 && n_q_heads <= 65535 && n_q_heads % c.n_heads == 0 &&
           ((int64_t)rows * (n_q_heads / c.n_heads) / kTile + c.n_seq) * c.n_heads <= (1 << 23);
}

template <int TYPE> void launch_typed(const AttnArgs& a, unsigned grid, hipStream_t stream) {
    const int hd = a.c.hd;
    if (hd <= 64) {
        if (hd == 64) paged_rows_kernel<TYPE, 64, false, 4><<<grid, 256, 0, stream>>>(a);
        else paged_rows_kernel<TYPE, 64, true, 4><<<grid, 256, 0, stream>>>(a);
    } else if (hd <= 128) {
        if (hd == 128) paged_rows_kernel<TYPE, 128, false, 4><<<grid, 256, 0, stream>>>(a);
        else paged_rows_kernel<TYPE, 128, true, 4><<<grid, 256, 0, stream>>>(a);
    } else {
        if (hd == 256) paged_rows_kernel<TYPE, 256, false, 4><<<grid, 256, 0, stream>>>(a);
        else paged_rows_kernel<TYPE, 256, true, 4><<<grid, 256, 0, stream>>>(a);
    }
}

}  // namespace

size_t paged_attention_workspace_bytes(const hawk_paged_cache* cache, int rows, int n_q_heads, int max_len) {
    PagedView c;
    if (!paged_view(cache, 0, &c) || !shape_ok(c, rows, n_q_heads)) return 0;
    const Plan p = plan_of(c.n_seq, rows, c.n_heads, n_q_heads, c.hd, (int64_t)c.max_pages * c.page_size, max_len);
    return p.part_bytes + p.ml_bytes;
}

int launch_paged_attention(const hawk_paged_cache* cache, int layer, const hawk_paged_rows* rows, const hawk_heads* q,
                           const uint64_t* tree, float scale, int max_len, const hawk_heads* out, void* workspace,
                           size_t workspace_bytes, hipStream_t stream) {
    AttnArgs a = {};
    if (!paged_view(cache, layer, &a.c)) return HAWK_EINVAL;
    if (nothing_to_do(cache, rows)) return HAWK_OK;
    if (!rows_view(rows, &a.r)) return HAWK_EINVAL;
    if (!heads_view(q, &a.q) || !heads_view(out, &a.out) || a.q.n_heads != a.out.n_heads) return HAWK_EINVAL;
    if (a.q.dtype != cache->dtype || !shape_ok(a.c, a.r.rows, a.q.n_heads)) return HAWK_EINVAL;
    if (!(scale > 0.f) || !(scale < 3.4e38f) || (reinterpret_cast<uintptr_t>(tree) & 7)) return HAWK_EINVAL;
    if (!room_for(a.out, a.r.rows, a.c.hd)) return HAWK_EINVAL;
    const Plan p = plan_of(a.c.n_seq, a.r.rows, a.c.n_heads, a.q.n_heads, a.c.hd, (int64_t)a.c.max_pages * a.c.page_size, max_len);
    if (p.part_bytes && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15))) return HAWK_EINVAL;
    if (workspace_bytes < p.part_bytes + p.ml_bytes) return p.part_bytes ? HAWK_ENOMEM : HAWK_EINVAL;
    a.tree = tree;
    a.scale2 = scale * 1.44269504f;
    a.group = a.q.n_heads / a.c.n_heads;
    a.tiles = p.tiles; a.splits = p.splits; a.split_keys = p.split_keys;
    a.part = static_cast<float*>(workspace);
    a.part_ml = reinterpret_cast<float*>(static_cast<char*>(workspace) + p.part_bytes);
    const int64_t grid = (int64_t)p.tiles * p.splits * a.c.n_heads;
    if (grid > (1 << 23)) return HAWK_EINVAL;
    if (cache->dtype == HAWK_FP32) launch_typed<HAWK_FP32>(a, (unsigned)grid, stream);
    else if (cache->dtype == HAWK_BF16) launch_typed<HAWK_BF16>(a, (unsigned)grid, stream);
    else launch_typed<HAWK_FP16>(a, (unsigned)grid, stream);
    if (p.splits > 1) {
        const int64_t units = (int64_t)a.r.rows * a.q.n_heads;
        paged_join_kernel<<<(unsigned)((units + 3) / 4), 256, 0, stream>>>(a);
    }
    return hipGetLastError() == hipSuccess ? HAWK_OK : HAWK_EDEVICE;
}

}  // namespace hawk
