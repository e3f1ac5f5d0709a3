// Attention of a step's rows over the pages of hawk_paged_cache.
//
// With S = scale Q K^T over the entries a row sees, out = softmax(S) V in one pass over the entries: a running maximum
// m and sum l per row, results rescaled when the maximum grows.  Everything is computed transposed, S^T = K Q^T and
// out^T = V^T P^T: a result lane of the matrix unit then holds one row's scores of four entries, which is what the next
// product takes as its operand if its entries are named in that order - the weights stay in the registers they are computed
// in, and a row's maximum, sum and rescaling are one value per lane.  Query heads that share a cache head are rows of the
// same tile: row r of a tile is (row of the sequence r / group, head r % group).
#include "paged.h"

// A score and its row's maximum are rounded alike, so that their difference is never above zero: nothing is fused but where it says so.
#pragma clang fp contract(off)

namespace hawk {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));

constexpr int kTile = 16;      // rows of a tile where a sequence has few (many: 128 or 256)

struct AttnArgs {
    PagedView c;
    RowsView r;
    HeadsView q, out;
    const uint64_t* tree;
    float scale2;              // scale * log2(e)
    Divisor group, heads, splits;   // query heads of a cache head; cache heads; parts of a long axis
    int tile, tiles;           // rows of a tile (2^tile), tiles of the launch
    int split_keys;            // entries of a part (the last one has the rest)
    float *part, *part_ml;     // [split][row][head][hd], [split][row][head][2]
};

// Which entries the rows of a tile are about.
struct Span {
    int s, first;              // sequence; the tile's first row * group + head
    int r0, n;                 // the sequence's first row, its rows
    int past;                  // committed entries (clamped to what an entry number can be)
    int end;                   // entries from this one on are seen by no row of the tile
    int all;                   // entries before this one are seen by every row of the tile
};
__host__ __device__ inline Span span_of(const AttnArgs& a, int s, int first, int start, int stop, int past) {
    Span t;
    t.s = s;
    t.first = first;
    t.r0 = min(max(start, 0), a.r.rows);
    t.n = max(min(max(stop, 0), a.r.rows) - t.r0, 0);
    t.past = min(max(past, -(1 << 30)), 1 << 30);
    const int lo = first / a.group, hi = min((first + (1 << a.tile) - 1) / a.group, t.n - 1);
    if (a.tree) {
        t.end = t.past + max(min(t.n, 64), hi + 1);
        t.all = t.past;
    } else {
        t.end = t.past + hi + 1;
        t.all = t.past + lo + 1;
    }
    t.end = max(min(t.end, a.c.capacity), 0);
    t.all = min(t.all, t.end);
    return t;
}
// Tiles are counted so that a sequence's first tile follows from its first row alone: base(s) = row_start[s] * group / tile + s,
// which leaves every sequence room for its tiles and at most one unused number per sequence.
__host__ __device__ inline int tile_base(const AttnArgs& a, int s, int start) {
    return (min(max(start, 0), a.r.rows) * a.group.d >> a.tile) + s;   // (rows * group is below 2^30)
}
// Tile `tile` as one of sequence s; false: it is none of its.  Where row starts do not ascend the search below may end at any
// sequence, one whose tiles lie behind this one (first below 0) among them.
__host__ __device__ inline bool tile_of(const AttnArgs& a, int s, int tile, int start, int stop, int past, Span& t) {
    t = span_of(a, s, (tile - tile_base(a, s, start)) * (1 << a.tile), start, stop, past);
    return t.first >= 0 && t.first < t.n * a.group.d;
}
// The sequence of a tile and its span; false: the tile is one of the unused numbers.  Up to 64 sequences every lane has one
// sequence's words, and the answer is there after one latency.
__device__ __forceinline__ bool find_tile(const AttnArgs& a, int lane, int tile, Span& t) {
    int s, start, stop, past;
    if (a.c.n_seq <= 64) {
        const int i = min(lane, a.c.n_seq - 1);
        const int b = a.r.row_start[i], e = a.r.row_start[i + 1], p = a.r.n_past[i];
        const int c = __popcll(__ballot(lane < a.c.n_seq && tile_base(a, i, b) <= tile));
        if (c == 0) return false;
        s = c - 1;
        start = __builtin_amdgcn_readlane(b, s);
        stop = __builtin_amdgcn_readlane(e, s);
        past = __builtin_amdgcn_readlane(p, s);
    } else {
        s = __builtin_amdgcn_readfirstlane(last_not_above(a.c.n_seq, lane, tile, [&](int i) { return (int64_t)tile_base(a, i, a.r.row_start[i]); }));
        if (s < 0) return false;
        start = a.r.row_start[s];
        stop = a.r.row_start[s + 1];
        past = a.r.n_past[s];
    }
    return tile_of(a, s, tile, start, stop, past, t);
}
// What a row of a tree sees; a row of a chain sees the entries up to its own.
__device__ __forceinline__ bool node_sees(const Span& t, int own, unsigned long long bits, int e) {
    const int j = e - t.past;
    return (int)(j < 0) | (int)(e == own) | ((int)(j < 64) & (int)((bits >> (j & 63)) & 1ull));
}
// Which of the 64 entries from e0 on a row sees, as bits: those before k1, of a chain up to its own, of a tree also by its ancestors' bits.
// One word a turn, so that a score costs a constant shift and a merge.
__device__ __forceinline__ unsigned long long first_bits(int n) { return n <= 0 ? 0ull : (n >= 64 ? ~0ull : (1ull << n) - 1ull); }
__device__ __forceinline__ unsigned long long seen_from(const AttnArgs& a, const Span& t, bool real, int own, unsigned long long bits, int e0, int k1) {
    unsigned long long w;
    if (a.tree) {
        const int j = e0 - t.past, m = own - e0;
        w = j >= 0 ? (j < 64 ? bits >> j : 0ull) : (j > -64 ? bits << -j : 0ull) | first_bits(-j);
        w |= m >= 0 && m < 64 ? 1ull << m : 0ull;
    } else {
        w = first_bits(own - e0 + 1);
    }
    return real ? w & first_bits(k1 - e0) : 0ull;
}
// z where bit c of the word is set, else minus infinity
__device__ __forceinline__ float if_seen(unsigned long long w, int c, float z) {
    const unsigned on = (unsigned)(((int)((unsigned)(w >> (c & 32)) << (31 - (c & 31)))) >> 31);
    return __uint_as_float((on & __float_as_uint(z)) | (~on & 0xFF800000u));
}
__device__ __forceinline__ int used_splits(const AttnArgs& a, int end) {
    return a.splits.shift < 0 ? 1 : min(a.splits.d, max(1, (end + a.split_keys - 1) / a.split_keys));
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

// Values of a type as words: the products, and which words hold an infinity or NaN (any sign bit of carry(w) set) and as which
// they are taken out.
template <int TYPE> struct Of;
template <class T> __device__ __forceinline__ unsigned carry(unsigned w) { return (w & T::kExp) + T::kCarry; }
template <class T> __device__ __forceinline__ bool odd(unsigned carries) { return (carries & (T::kExp ^ (T::kExp << 1)) & 0x80008000u) != 0u; }
template <> struct Of<HAWK_BF16> {
    static constexpr int kBytes = 2;
    static constexpr float kLift = 0.f;
    static __device__ __forceinline__ f32x4 mul(v4u a, v4u b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ unsigned short narrow(float x) { return __builtin_bit_cast(unsigned short, (__bf16)x); }
    static __device__ __forceinline__ float widen(unsigned short b) { return __uint_as_float((unsigned)b << 16); }
    static constexpr unsigned kExp = 0x7F807F80u, kCarry = 0x00800080u;   // an exponent of ones carries into the sign's place
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
    static constexpr unsigned kExp = 0x7C007C00u, kCarry = 0x04000400u;
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
    static constexpr unsigned kExp = 0x7F800000u, kCarry = 0x00800000u;
    static __device__ __forceinline__ unsigned clear(unsigned w) { return (w & kExp) == kExp ? 0u : w; }
};

// Infinities and NaN among the values, N features from f on of a row whose results are at dst.  An infinity that a row sees is in its result with
// its sign, however small its weight.
//   Of entries that only some rows of a tile see they would make NaN of the others' weights of zero: they are zeros in the products
// (entries from .. to - 1), and are added here, behind everything else.
//   Where every row sees an entry its values are multiplied as they are.  A weight's second part, which is zero or below it for every other
// weight, or a weight or factor that is zero in 32 bits then makes NaN of an infinity.  So a feature that is NaN is what the infinities and NaN
// among all values the row sees (entries begin .. to - 1) add up to; where there are none it stays.  (The row's sum of weights is a number above
// zero: that is looked at before.)
template <int TYPE, int N>
__device__ void add_odd(const AttnArgs& a, const Span& t, const char* vh, int own, unsigned long long bits, int begin, int from, int to, int f,
                        char* dst, int64_t at, int dtype) {
    const int32_t* pages = a.c.table + (int64_t)t.s * a.c.table_stride;
    auto stored = [&](int j) {
        float x, y;
        if (dtype == HAWK_FP32) return *reinterpret_cast<const float*>(dst + (at + j) * 4);
        widen2(*reinterpret_cast<const unsigned short*>(dst + (at + j) * 2), dtype, x, y);
        return x;
    };
    float sum[N];
    unsigned lost = 0u, some = 0u;   // features that are NaN; that have anything to add
#pragma unroll
    for (int j = 0; j < N; ++j) {
        sum[j] = 0.f;
        lost |= isnan(stored(j)) ? 1u << j : 0u;
    }
    for (int e = max(lost ? begin : from, 0); e < to; ++e) {
        const int64_t place = entry_at(a.c, pages, e);
        if (place < 0 || !(a.tree ? node_sees(t, own, bits, e) : e <= own)) continue;
        const unsigned take = e < from ? lost : ~0u;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            float v;
            if constexpr (TYPE == HAWK_FP32) v = *reinterpret_cast<const float*>(vh + (place + f + j) * 4);
            else v = Of<TYPE>::widen(*reinterpret_cast<const unsigned short*>(vh + (place + f + j) * 2));
            if (fabsf(v) <= 3.4028235e38f || !((take >> j) & 1u)) continue;
            sum[j] += v;
            some |= 1u << j;
        }
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
        if (!((some >> j) & 1u)) continue;
        const float x = (lost >> j) & 1u ? sum[j] : stored(j) + sum[j];
        if (dtype == HAWK_FP32) *reinterpret_cast<float*>(dst + (at + j) * 4) = x;
        else *reinterpret_cast<unsigned short*>(dst + (at + j) * 2) = (unsigned short)narrow2(x, 0.f, dtype);
    }
}

// Tile of 16 rows, NW waves that share the entries of its part in turns of 32 (16 of fp32).  Keys and values go from the pages straight
// into the operands' registers: a lane's 16 bytes of a key are its features of one product, and its piece of eight keys' values
// - the same few features of each - become the transposed operand by pairing words of two keys.  The next turn's keys and values
// are requested as soon as this turn's scores are there.
// EASY: groups of 16 entries lie within a page, so that their page number is one for the wave; otherwise every lane looks its
// entries up (48 sequences of six rows behind 1000 entries, 20 heads of 64: pages of 64 entries 38 us, of 60 45 us).
template <int TYPE, int DP, bool PAD, bool EASY, int NW>
__global__ __launch_bounds__(64 * NW, DP == 64 ? (NW == 4 ? 3 : (TYPE == HAWK_FP32 ? 2 : 4)) : (DP == 128 ? 2 : 1)) void paged_rows_kernel(AttnArgs a) {
    using T = Of<TYPE>;
    constexpr int ES = T::kBytes, VEC = 16 / ES, STEP = 4 * VEC, NS = DP / STEP;   // features of a lane's piece, of a product; products
    constexpr int VD = DP / 16, VC = VD < VEC ? VD : VEC, NC = VD / VC;            // a lane's features of a value, per piece; pieces
    constexpr int VW = VC * ES / 4;                                                // words of a piece
    constexpr int COLS = 16 * VC;                                                  // features of a round of pieces
    constexpr int KT = ES == 4 ? 1 : 2, KEYS = 16 * KT;                            // groups of 16 entries of a turn
    __shared__ float lo[NW][kTile][COLS + 4];
    __shared__ float lm[NW][kTile], ll[NW][kTile];
    __shared__ int lodd[NW];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), m16 = lane & 15, g = lane >> 4;
    const int rest = (int)blockIdx.x / a.heads, head = blockIdx.x - rest * a.heads.d, turned = rest / a.splits;
    const int split = rest - turned * a.splits.d, tile = a.tiles - 1 - turned;   // later tiles see more: they start first
    Span t;
    if (!find_tile(a, lane, tile, t) || split >= used_splits(a, t.end)) return;
    const int k0 = split * a.split_keys, k1 = split == a.splits.d - 1 ? t.end : min(t.end, k0 + a.split_keys);
    const int hd = a.c.hd;

    // page numbers of 64 pages from `window` on, one per lane
    const int32_t* pages = a.c.table + (int64_t)t.s * a.c.table_stride;
    int window = page_of(a.c, min(k0 + KEYS * wave, max(k1 - 1, 0)));
    int ids = pages[min(window + lane, a.c.max_pages - 1)];
    const char *kh = a.c.k + (int64_t)head * a.c.head_stride * ES, *vh = a.c.v + (int64_t)head * a.c.head_stride * ES;

    // this lane's row: its query, and what it sees
    const int pr = t.first + m16, i = pr / a.group;
    const bool real = pr < t.n * a.group.d;
    const int row = t.r0 + (real ? i : 0), qh = head * a.group.d + (real ? pr - i * a.group.d : 0);
    const int own = t.past + i;   // the row's own entry, the last one it sees of a chain
    const unsigned long long bits = a.tree && real ? a.tree[row] : 0ull;
    v4u q[NS];
#pragma unroll
    for (int ks = 0; ks < NS; ++ks) {
        q[ks] = (v4u){0u, 0u, 0u, 0u};
        const int f = ks * STEP + g * VEC;
        if (real && (!PAD || f < hd)) q[ks] = *reinterpret_cast<const v4u*>(a.q.data + ((int64_t)row * a.q.row_stride + (int64_t)qh * a.q.head_stride + f) * ES);
    }

    // Bytes from a head's start to a turn's groups of entries (EASY: of the group, in the wave's registers; otherwise of the lane's own
    // entry) and which entries there are.  Ones that do not exist read the pool's first entry: their scores are dropped.
    const int64_t es = a.c.entry_stride * ES;
    const int64_t klane = (EASY ? m16 * es : 0) + g * 16, vlane = (EASY ? g * 4 * es : 0) + m16 * VC * ES;
    int64_t at[KT];
    bool there[KT];                     // (EASY: of the page; the turn's end counts apart)
    auto places = [&](int kb) {
        const int p0 = page_of(a.c, kb), p1 = page_of(a.c, min(kb + KEYS, k1) - 1);
        if (p0 < window || p1 >= window + 64) {
            window = p0;
            ids = pages[min(window + lane, a.c.max_pages - 1)];
        }
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            const int e = EASY ? kb + kt * 16 : min(kb + kt * 16 + m16, k1 - 1);
            const int p = min(page_of(a.c, e), p1);   // (a group behind the end: any page)
            const int id = EASY ? __builtin_amdgcn_readlane(ids, p - window) : __shfl(ids, p - window);
            const int64_t x = place_in(a.c, id, e - p * a.c.page_size);
            // a group's first entry at or behind the end, or a lane's own entry there: the pool's first one
            there[kt] = x >= 0 && (EASY ? e < k1 : kb + kt * 16 + m16 < k1);
            at[kt] = there[kt] ? x * ES : 0;
        }
    };
    // EASY groups are read whole, past the end of the sequence too: the rest of the page is there, and dropped like any entry
    // that does not exist.
    v4u k[KT][NS];
    typedef unsigned piece __attribute__((ext_vector_type(VW)));
    typedef piece pieces[KT][4][NC];
    auto request = [&](pieces& v) {
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            const char* src = kh + at[kt] + (EASY && !there[kt] ? (int64_t)g * 16 : klane);
#pragma unroll
            for (int ks = 0; ks < NS; ++ks) {
                if (PAD && ks * STEP + g * VEC >= hd) k[kt][ks] = (v4u){0u, 0u, 0u, 0u};
                else k[kt][ks] = *reinterpret_cast<const v4u*>(src + ks * STEP * ES);
            }
        }
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const char* src;
                if (EASY) src = vh + at[kt] + (there[kt] ? vlane + r * es : (int64_t)m16 * VC * ES);
                else src = vh + __shfl((long long)at[kt], g * 4 + r) + vlane;
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    if (PAD && c * COLS + m16 * VC >= hd) v[kt][r][c] = (piece)0u;
                    else v[kt][r][c] = *reinterpret_cast<const piece*>(src + c * COLS * ES);
                }
            }
    };

    f32x4 o[VD];
#pragma unroll
    for (int d = 0; d < VD; ++d) o[d] = (f32x4){0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    bool found = false;   // values were taken out
    auto turn = [&](int kb, pieces& v, pieces& vn) {
        float z[KT][4];
        unsigned have = 0u;   // bit kt * 4 + r: entry g * 4 + r of group kt exists
        bool gone = false;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            gone = gone || !there[kt];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int ok = EASY ? (int)there[kt] & (int)(kb + kt * 16 + g * 4 + r < k1) : __shfl((int)there[kt], g * 4 + r);
                have |= ok ? 1u << (kt * 4 + r) : 0u;
            }
            f32x4 sc = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < NS; ++ks) sc = T::mul(k[kt][ks], q[ks], sc);
#pragma unroll
            for (int r = 0; r < 4; ++r) z[kt][r] = sc[r] * a.scale2;
        }
        if (kb + KEYS * NW < k1) {
            places(kb + KEYS * NW);
            request(vn);
        }
        const bool edge = kb + KEYS > t.all;   // not every row sees every entry
        if (edge || kb + KEYS > k1 || __any(gone)) {
            const unsigned long long w = seen_from(a, t, real, own, bits, kb + g * 4, k1);
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int r = 0; r < 4; ++r) z[kt][r] = if_seen(w, kt * 16 + r, z[kt][r]);
            if (__any(gone)) {
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) z[kt][r] = (have >> (kt * 4 + r)) & 1u ? z[kt][r] : -INFINITY;
            }
            // Weights of zero do not meet infinities and NaN: those of entries behind the end or without a page are dropped, others wait
            // for the rows that see them (add_odd).
            unsigned any = 0u;
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int c = 0; c < NC; ++c)
#pragma unroll
                        for (int x = 0; x < VW; ++x) any |= carry<T>(v[kt][r][c][x]);
            if (__any(odd<T>(any))) {
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const bool ok = (have >> (kt * 4 + r)) & 1u;
#pragma unroll
                        for (int c = 0; c < NC; ++c)
#pragma unroll
                            for (int x = 0; x < VW; ++x) v[kt][r][c][x] = ok && !edge ? v[kt][r][c][x] : T::clear(v[kt][r][c][x]);
                    }
                found = found || edge;
            }
        }
        float top = m;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int r = 0; r < 4; ++r) top = fmaxf(top, z[kt][r]);
        top = row_max(top);
        const float base = top == -INFINITY ? 0.f : top;
        if (__any(top > m)) {
            const float shrink = __builtin_amdgcn_exp2f(m - base);
            l *= shrink;
#pragma unroll
            for (int d = 0; d < VD; ++d) o[d] *= shrink;
        }
        m = top;
        float p[KT][4];
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                p[kt][r] = __builtin_amdgcn_exp2f(z[kt][r] - base + T::kLift);
                l += p[kt][r];
            }
        if constexpr (TYPE == HAWK_FP32) {
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int d = 0; d < VD; ++d)
                        o[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[kt][r][d / VC][d % VC]), p[kt][r], o[d], 0, 0, 0);
        } else {
            // the weights as two values of the type, the second the first one's remainder: about 16 bits
            v4u ph, pl;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float x = p[j >> 1][2 * j & 3], y = p[j >> 1][(2 * j & 3) + 1];
                ph[j] = narrow2(x, y, TYPE);
                pl[j] = narrow2(x - T::widen((unsigned short)ph[j]), y - T::widen((unsigned short)(ph[j] >> 16)), TYPE);
            }
#pragma unroll
            for (int d = 0; d < VD; ++d) {
                v4u w;
#pragma unroll
                for (int j = 0; j < 4; ++j)   // feature d of entries 2 j and 2 j + 1
                    w[j] = __builtin_amdgcn_perm(v[j >> 1][(2 * j & 3) + 1][d / VC][(d % VC) >> 1], v[j >> 1][2 * j & 3][d / VC][(d % VC) >> 1],
                                                 (d & 1) ? 0x07060302u : 0x05040100u);
                o[d] = T::mul(w, pl, o[d]);
                o[d] = T::mul(w, ph, o[d]);
            }
        }
    };
    int kb = k0 + KEYS * wave;
    pieces va, vb;
    if (kb < k1) {
        places(kb);
        request(va);
    }
    for (; kb < k1; kb += 2 * KEYS * NW) {
        turn(kb, va, vb);
        if (kb + KEYS * NW < k1) turn(kb + KEYS * NW, vb, va);
    }

    // the waves' parts: maximum and sum, then the results in rounds of COLS features
    l = row_sum(l);
    if (g == 0) {
        lm[wave][m16] = m;
        ll[wave][m16] = l;
    }
    if (lane == 0) lodd[wave] = found;
    __syncthreads();
    float mt = -INFINITY, lt = 0.f;
    bool any_odd = false;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        mt = fmaxf(mt, lm[w][m16]);
        any_odd = any_odd || lodd[w];
    }
    const float base = mt == -INFINITY ? 0.f : mt;
#pragma unroll
    for (int w = 0; w < NW; ++w) lt += ll[w][m16] * __builtin_amdgcn_exp2f(lm[w][m16] - base);
    const float mine = __builtin_amdgcn_exp2f(m - base);
    const bool whole = a.splits.d == 1;
    const float norm = whole ? (lt == 0.f ? 0.f : 1.f / lt) : 1.f;
    if (!whole && real && wave == 0 && g == 0) {
        float* ml = a.part_ml + (((int64_t)split * a.r.rows + row) * a.q.n_heads + qh) * 2;
        ml[0] = mt;
        ml[1] = lt;
    }
    // eight features of a row per thread
    const int type = whole ? a.out.dtype : HAWK_FP32;
    char* dst = whole ? a.out.data : reinterpret_cast<char*>(a.part);
    auto place_of = [&](int rr, int ff, int& ri) {
        const int prr = t.first + rr;
        ri = prr / a.group;
        const int64_t orow = t.r0 + ri, oh = head * a.group.d + prr - ri * a.group.d;
        return whole ? orow * a.out.row_stride + oh * a.out.head_stride + ff : (((int64_t)split * a.r.rows + orow) * a.q.n_heads + oh) * hd + ff;
    };
    bool lost = false;   // a result of this thread's is NaN
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        if (c > 0) __syncthreads();
#pragma unroll
        for (int y = 0; y < 4; ++y)
#pragma unroll
            for (int d = 0; d < VC; ++d) lo[wave][m16][(g * 4 + y) * VC + d] = o[c * VC + d][y] * (mine * norm);
        __syncthreads();
        for (int u = threadIdx.x; u < kTile * (COLS / 8); u += 64 * NW) {
            const int rr = u / (COLS / 8), f = (u % (COLS / 8)) * 8, ff = c * COLS + f;
            if (t.first + rr >= t.n * a.group.d || (PAD && ff >= hd)) continue;
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] = 0.f;
#pragma unroll
                for (int w = 0; w < NW; ++w) x[e] += lo[w][rr][f + e];
                lost = lost || isnan(x[e]);
            }
            int ri;
            store8(dst, place_of(rr, ff, ri), type, x);
        }
    }
    if (!lost && !any_odd) return;
    for (int c = 0; c < NC; ++c)
        for (int u = threadIdx.x; u < kTile * (COLS / 8); u += 64 * NW) {
            const int rr = u / (COLS / 8), ff = c * COLS + (u % (COLS / 8)) * 8;
            if (t.first + rr >= t.n * a.group.d || (PAD && ff >= hd)) continue;
            float sum = 0.f;   // of the row's weights: where it is NaN or zero, so is every feature
#pragma unroll
            for (int w = 0; w < NW; ++w) sum += ll[w][rr];
            int ri;
            const int64_t at = place_of(rr, ff, ri);
            const float none[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (sum == 0.f) store8(dst, at, type, none);
            else if (!isnan(sum))
                add_odd<TYPE, 8>(a, t, vh, t.past + ri, a.tree ? a.tree[t.r0 + ri] : 0ull, k0, max(k0, t.all - KEYS), k1, ff, dst, at, type);
        }
}

// Many rows: a workgroup of four or eight waves, 32 rows each, over turns of KB entries that all of them read from LDS.  The next
// turn's keys and values are in registers while this one is computed and are written behind it, two buffers, one barrier a
// turn.  Products of 32 x 32 x 16: a lane has one row's 16 scores of 32 entries - blocks of four entries, the other half of the
// wave the blocks between -, which in that order are the next product's operand; values are read transposed.
// Weights are rounded to the type once before the product with the values (their sum is not): a second part as in the tiles of 16 rows would be
// half of all products again, 374 us where this takes 291 (4001 rows x 4 behind 2048, heads of 128, bf16), and takes the relative error of
// bf16 results, which their own rounding makes 1.66e-3, from 2.34e-3 to 1.66e-3.
// LDS rows keep their 16-byte pieces in an order changed by the row number, so that the 16 rows (keys) or four rows (values) that a
// request touches lie on different banks.
template <int TYPE> struct Wide;
template <> struct Wide<HAWK_BF16> {
    static constexpr float kLift = 0.f;
    static __device__ __forceinline__ f32x16 mul(v4u a, v4u b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
    }
};
template <> struct Wide<HAWK_FP16> {
    static constexpr float kLift = 6.f;   // with what a maximum may lag behind (kLag) weights are at most 2^14
    static __device__ __forceinline__ f32x16 mul(v4u a, v4u b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
    }
};
constexpr float kLag = 8.f;   // results are rescaled when a row's maximum has grown by more than 2^8, not whenever it grows
constexpr float kFused = 0x1p20f;   // scaled scores up to this (half a step: 2^-5) are multiplied and added in one instruction

// EASY as above: a wave's part of a turn's rows lies in one group of 16, whose place is found once for the wave and added to by the
// requests themselves.
template <int TYPE, int DP, bool PAD, bool EASY, int KB, int NW>
__global__ __launch_bounds__(64 * NW, DP <= 128 ? 2 : 1) void paged_wide_kernel(AttnArgs a) {
    using T = Of<TYPE>;
    constexpr int ROW = DP * 2, CH = ROW / 16, TH = 64 * NW, PIECES = KB * CH / TH, NS = DP / 16, NT = DP / 32, SUB = KB / 32;
    __shared__ __attribute__((aligned(16))) char lk[2][KB * ROW];
    __shared__ __attribute__((aligned(16))) char lv[2][KB * ROW];
    __shared__ unsigned gone[4][SUB];   // of the turns in flight: which entries do not exist
    __shared__ int found;      // infinities or NaN were taken out of values

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r32 = lane & 31, hh = lane >> 5;
    const int rest = (int)blockIdx.x / a.heads, head = blockIdx.x - rest * a.heads.d, turned = rest / a.splits;
    const int split = rest - turned * a.splits.d, tile = a.tiles - 1 - turned;
    Span t;
    if (!find_tile(a, lane, tile, t) || split >= used_splits(a, t.end)) return;
    const int first = t.first;
    const int k0 = split * a.split_keys, k1 = split == a.splits.d - 1 ? t.end : min(t.end, k0 + a.split_keys);
    const int hd = a.c.hd;
    if (tid < 4 * SUB) gone[0][tid] = 0u;
    if (tid == 0) found = 0;

    const int pr = first + wave * 32 + r32, i = pr / a.group;
    const bool real = pr < t.n * a.group.d;
    const int row = t.r0 + (real ? i : 0), qh = head * a.group.d + (real ? pr - i * a.group.d : 0);
    const int own = t.past + i;
    const unsigned long long bits = a.tree && real ? a.tree[row] : 0ull;
    // entries that every row of the wave sees lie before `all`, none sees any from `end` on
    const int wlo = (first + wave * 32) / a.group, whi = min((first + wave * 32 + 31) / a.group, t.n - 1);
    const int all = a.tree ? t.past : t.past + wlo + 1;
    const int end = first + wave * 32 >= t.n * a.group.d ? 0 : (a.tree ? k1 : min(k1, t.past + whi + 1));
    v4u q[NS];
#pragma unroll
    for (int ks = 0; ks < NS; ++ks) {
        q[ks] = (v4u){0u, 0u, 0u, 0u};
        const int f = ks * 16 + hh * 8;
        if (real && (!PAD || f < hd)) q[ks] = *reinterpret_cast<const v4u*>(a.q.data + ((int64_t)row * a.q.row_stride + (int64_t)qh * a.q.head_stride + f) * 2);
    }
    f32x16 o[NT];
#pragma unroll
    for (int d = 0; d < NT; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
    float mb = -INFINITY, l = 0.f;   // the reference the weights are taken to, scaled; their sum

    const int32_t* pages = a.c.table + (int64_t)t.s * a.c.table_stride;
    const char *kh = a.c.k + (int64_t)head * a.c.head_stride * 2, *vh = a.c.v + (int64_t)head * a.c.head_stride * 2;
    // pieces of a turn that this thread brings: piece j is 16 bytes of row (tid + TH j) / CH
    const int chunk = tid % CH;
    const bool inside = !PAD || chunk * 8 < hd;
    int page[PIECES];           // EASY: of the wave's group; -1: behind the end
    v4u kr[PIECES], vr[PIECES];
    auto look_up = [&](int kb) {
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
            const int e = kb + (EASY ? (wave * 64 + TH * j) / CH & ~15 : (tid + TH * j) / CH);
            page[j] = e < k1 ? pages[page_of(a.c, e)] : -1;
            if (EASY) page[j] = __builtin_amdgcn_readfirstlane(page[j]);
        }
    };
    auto request = [&](int kb) {
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
            kr[j] = vr[j] = (v4u){0u, 0u, 0u, 0u};
            if (EASY) {
                const int e = kb + ((wave * 64 + TH * j) / CH & ~15);
                const int64_t at = place_in(a.c, page[j], e - page_of(a.c, e) * a.c.page_size) * 2;
                if (at >= 0) {
                    const unsigned off = (unsigned)((tid + TH * j) / CH & 15) * (unsigned)(a.c.entry_stride * 2) + chunk * 16;
                    if (inside) {
                        kr[j] = *reinterpret_cast<const v4u*>(kh + at + off);
                        vr[j] = *reinterpret_cast<const v4u*>(vh + at + off);
                    }
                }
            } else {
                const int e = kb + (tid + TH * j) / CH;
                const int64_t at = e < k1 ? place_in(a.c, page[j], e - page_of(a.c, e) * a.c.page_size) : -1;
                if (at >= 0 && inside) {
                    kr[j] = *reinterpret_cast<const v4u*>(kh + at * 2 + chunk * 16);
                    vr[j] = *reinterpret_cast<const v4u*>(vh + at * 2 + chunk * 16);
                }
            }
        }
    };
    auto put = [&](int kb, int turn) {
        const int buffer = (turn & 1) * (KB * ROW);
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
            const int r = EASY ? (wave * 64 + TH * j) / CH & ~15 : (tid + TH * j) / CH;
            if (kb + r < k1 && (unsigned)page[j] >= (unsigned)a.c.n_pages) atomicOr(&gone[turn & 3][r >> 5], (EASY ? 0xFFFFu : 1u) << (r & 31));
        }
        if (kb + KB > t.all) {   // not every row sees every entry
            unsigned any = 0u;
#pragma unroll
            for (int j = 0; j < PIECES; ++j)
#pragma unroll
                for (int x = 0; x < 4; ++x) any |= carry<T>(vr[j][x]);
            if (odd<T>(any)) {
                found = 1;
#pragma unroll
                for (int j = 0; j < PIECES; ++j)
#pragma unroll
                    for (int x = 0; x < 4; ++x) vr[j][x] = T::clear(vr[j][x]);
            }
        }
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
            const int r = (tid + TH * j) / CH;
            const int ck = DP == 64 ? chunk ^ ((r >> 1) & 7) : chunk ^ (r & 15);
            const int cv = DP == 64 ? chunk ^ (((r >> 1) & 1) << 2) : chunk ^ ((r & 3) << 2);
            *reinterpret_cast<v4u*>(lk[0] + buffer + r * ROW + ck * 16) = kr[j];
            *reinterpret_cast<v4u*>(lv[0] + buffer + r * ROW + cv * 16) = vr[j];
        }
    };

    const int turns = (k1 - k0 + KB - 1) / KB;
    // (kr, vr and page are of the same turn between request() and put(): look_up() of the next one comes behind put())
    if (turns > 0) {
        look_up(k0);
        request(k0);
        __syncthreads();   // gone is clear
        put(k0, 0);
        look_up(k0 + KB);
        request(k0 + KB);
    }
    __syncthreads();

    const int r16 = lane & 15, kbase = r32 * ROW + ((DP == 64 ? (r32 >> 1) & 7 : r32 & 15) ^ hh) * 16;
    const int vbase = (4 * hh + (r16 >> 2)) * ROW + ((((lane >> 4) & 1) * 2 + ((r16 & 3) >> 1)) ^ (DP == 64 ? (r16 >> 3) << 2 : (r16 >> 2) << 2)) * 16 + (r16 & 1) * 8;
    const float c = a.scale2;
    for (int turn = 0; turn < turns; ++turn) {
        const int kb = k0 + turn * KB;
        unsigned none[SUB], some = 0u;
#pragma unroll
        for (int u = 0; u < SUB; ++u) some |= none[u] = gone[turn & 3][u];
        if (kb < end) {
            const char *bk = lk[0] + (turn & 1) * (KB * ROW), *bv = lv[0] + (turn & 1) * (KB * ROW);
            float z[SUB][16];
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                f32x16 sc;
#pragma unroll
                for (int e = 0; e < 16; ++e) sc[e] = 0.f;
#pragma unroll
                for (int ks = 0; ks < NS; ++ks) {
                    const v4u k = *reinterpret_cast<const v4u*>(bk + u * 32 * ROW + (kbase ^ (ks * 32)));
                    sc = Wide<TYPE>::mul(k, q[ks], sc);
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) z[u][e] = sc[e];
            }
            if (some || kb + KB > all || kb + KB > k1) {
                unsigned long long w = seen_from(a, t, real, own, bits, kb + 4 * hh, k1);
                w &= ~(((unsigned long long)none[0] | (SUB > 1 ? (unsigned long long)none[SUB - 1] << 32 : 0ull)) >> (4 * hh));
#pragma unroll
                for (int u = 0; u < SUB; ++u)
#pragma unroll
                    for (int r = 0; r < 16; ++r) z[u][r] = if_seen(w, u * 32 + 8 * (r >> 2) + (r & 3), z[u][r]);
            }
            float top = -INFINITY;
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
                for (int r = 0; r < 16; ++r) top = fmaxf(top, z[u][r]);
            top = swap32(top, false) * c;
            if (__any(top > mb + kLag)) {
                const float now = fmaxf(mb, top), base = now == -INFINITY ? 0.f : now, shrink = __builtin_amdgcn_exp2f(mb - base);
                mb = now;
                l *= shrink;
#pragma unroll
                for (int d = 0; d < NT; ++d) o[d] *= shrink;
            }
            const float ref = mb == -INFINITY ? 0.f : mb;
            float by = c, off = Wide<TYPE>::kLift - ref;
            // The reference is a rounded product: an entry's own, not rounded, may lie above it by half a step.  Where that is more than a
            // small part of a power of two - a weight could leave the type, or every weight of a row be zero - both are rounded.
            if (__any(fabsf(ref) > kFused)) {
#pragma unroll
                for (int u = 0; u < SUB; ++u)
#pragma unroll
                    for (int r = 0; r < 16; ++r) z[u][r] = z[u][r] * c - ref;
                by = 1.f;
                off = Wide<TYPE>::kLift;
            }
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    z[u][r] = __builtin_amdgcn_exp2f(fmaf(z[u][r], by, off));
                    l += z[u][r];
                }
#pragma unroll
            for (int cc = 0; cc < KB / 16; ++cc) {
                v4u p;
#pragma unroll
                for (int j = 0; j < 4; ++j) p[j] = narrow2(z[cc >> 1][8 * (cc & 1) + 2 * j], z[cc >> 1][8 * (cc & 1) + 2 * j + 1], TYPE);
#pragma unroll
                for (int d = 0; d < NT; ++d) {
                    typedef short s4 __attribute__((ext_vector_type(4)));
                    const char* at = bv + cc * 16 * ROW + (vbase ^ (d * 64));
                    const v2u x = __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)const_cast<char*>(at)));
                    const v2u y = __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)const_cast<char*>(at + 8 * ROW)));
                    o[d] = Wide<TYPE>::mul((v4u){x[0], x[1], y[0], y[1]}, p, o[d]);
                }
            }
        }
        if (turn + 1 < turns) {
            put(kb + KB, turn + 1);
            look_up(kb + 2 * KB);
            request(kb + 2 * KB);
        }
        if (tid < SUB) gone[(turn + 3) & 3][tid] = 0u;   // the turn before this one's: nobody looks at it any more
        __syncthreads();
    }

    l = swap32(l, true);
    if (!real) return;
    const bool whole = a.splits.d == 1;
    const float norm = whole ? (l == 0.f ? 0.f : 1.f / l) : 1.f;
    const int64_t vec = ((int64_t)split * a.r.rows + row) * a.q.n_heads + qh;
    if (!whole && hh == 0) {
        a.part_ml[vec * 2] = mb;
        a.part_ml[vec * 2 + 1] = l;
    }
    char* dst = whole ? a.out.data : reinterpret_cast<char*>(a.part);
    const int64_t at = whole ? (int64_t)row * a.out.row_stride + (int64_t)qh * a.out.head_stride : vec * hd;
    const int type = whole ? a.out.dtype : HAWK_FP32;
    bool lost = false;
#pragma unroll
    for (int d = 0; d < NT; ++d)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int f = d * 32 + 8 * b + 4 * hh;
            if (PAD && f >= hd) continue;
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[e] = o[d][4 * b + e] * norm;
                lost = lost || isnan(x[e]);
            }
            store4(dst, at + f, type, x);
        }
    if (lost || found) {
        const float none[4] = {0.f, 0.f, 0.f, 0.f};
        for (int f = 4 * hh; f < hd; f += 8) {
            if (l == 0.f) store4(dst, at + f, type, none);
            else if (!isnan(l)) add_odd<TYPE, 4>(a, t, vh, own, bits, k0, max(k0, t.all - KB), k1, f, dst, at + f, type);
        }
    }
}

// Joins the parts of a long axis: a wave per (row, head).  Lane i has part i's maximum and sum; groups of lanes take a part's features each,
// eight a lane, so that several parts are on their way at once.
__global__ __launch_bounds__(256) void paged_join_kernel(AttnArgs a, int lanes) {
    const int lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int row = (int)(unit / a.q.n_heads), qh = (int)(unit - (int64_t)row * a.q.n_heads);
    if (row >= a.r.rows) return;
    const int s = last_not_above(a.c.n_seq, lane, row, [&](int i) { return (int64_t)a.r.row_start[i]; });
    if (s < 0) return;
    const int start = a.r.row_start[s], stop = a.r.row_start[s + 1];
    if (row < start || row >= stop) return;   // (the first only where row starts do not ascend)
    const Span t = span_of(a, s, ((row - max(start, 0)) * a.group.d + (qh - qh / a.group * a.group.d)) >> a.tile << a.tile, start, stop, a.r.n_past[s]);
    const int n = used_splits(a, t.end);
    const int64_t step = (int64_t)a.r.rows * a.q.n_heads, vec = (int64_t)row * a.q.n_heads + qh;
    const int f = (lane & (lanes - 1)) * 8, part0 = lane / lanes, per = 64 / lanes;
    float mt = -INFINITY, lt = 0.f, x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int i = lane; i < n; i += 64) mt = fmaxf(mt, a.part_ml[(i * step + vec) * 2]);
#pragma unroll
    for (int w = 1; w < 64; w <<= 1) mt = fmaxf(mt, __shfl_xor(mt, w));
    const float base = mt == -INFINITY ? 0.f : mt;
#pragma unroll 4
    for (int i = part0; i < n; i += per) {
        const float w = fmaxf(__builtin_amdgcn_exp2f(a.part_ml[(i * step + vec) * 2] - base), 0x1p-126f);   // (not zero: infinities stay what they are)
        lt += a.part_ml[(i * step + vec) * 2 + 1] * w;
        if (f < a.c.hd) {
            float y[8];
            load8(reinterpret_cast<const char*>(a.part), (i * step + vec) * a.c.hd + f, HAWK_FP32, y);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = fmaf(y[e], w, x[e]);
        }
    }
    for (int w = lanes; w < 64; w <<= 1) {
        lt += __shfl_xor(lt, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] += __shfl_xor(x[e], w);
    }
    if (lane >= lanes || f >= a.c.hd) return;
    const float norm = lt == 0.f ? 0.f : 1.f / lt;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= norm;
    store8(a.out.data, (int64_t)row * a.out.row_stride + (int64_t)qh * a.out.head_stride + f, a.out.dtype, x);
}

struct Plan { bool wide; int tile, waves, tiles, splits, split_keys; size_t part_bytes, ml_bytes; };

// How a call is cut.
// Tiles of 16 rows read a sequence's entries once for every 16 rows, but are there after 8 us; tiles of 128 through LDS want 64 rows a
// sequence (rows times query heads of a cache head) and some work.  16-row tiles times entries, 8 sequences, us for tiles of
// 16 / 128 rows: 32 heads of 128 on 8, 64 rows behind 300 entries (154 thousand) 12.7 / 18.3, 128 rows (307 thousand) 23.5 / 18.7, 32 behind
// 2000 (1 million) 44.6 / 44.2, 64 (2 million) 88.4 / 54.1; 20 heads of 64, 64 rows behind 300 (192 thousand) 12.8 / 12.3, behind 2000 49.4 / 39.2.
// Tiles of 256 rows halve what is brought and put, but eight waves meet at every barrier: 4001 rows x 4 behind 2048 292 us, in
// tiles of 128 337; 8 sequences of 512 rows x 4 behind 2000 199 / 223, of 256 rows x 4 142 / 110.
// Parts of the long axis where the tiles alone would leave many of the chip's 256 units idle: joining them is a launch of its own of 4 to
// 5 us, and a workgroup of 16 rows reads 35 to 70 KB a us, so 400 KB are worth parts, of 128 KB then (us whole / in two / in more: one
// row behind 1500 entries, 32 heads of 128 on 8, 18.3 / 16.5 / 13.5; four rows behind 9000 22.1 in 8, 18 in more; 4 x 6 rows behind 1100, 20
// heads of 64, 11.3 / 14.2 / 15.1).  Where every other unit has a tile, parts only even sequences out and have to be larger: 8 trees
// of 13 rows behind 64 to 1080, 32 heads of 128, 19.6 / 27.3; 16 x 1 behind 300 to 1500, 32 heads on 8, 20 in one, 25 in four; behind 100 to
// 8000 97 in one, 77 in three, 65 in eight; 32 x 1 behind 100 to 16000 231 in one, 200 in three, 233 in four.
// As many parts as make one workgroup of eight waves a unit, two for heads of up to 64 (us with one / two / four of four waves a unit: 4 x 1
// behind 70001 to 100000, 32 heads of 128 on 8, 228 / 236 / 258; 1 x 5 behind 16000 22.9 / 26.1 / 32; 6 x 6 behind 2500, 20 heads of 64, 27.0 / 21.7 / 21.6).
Plan plan_of(int dtype, int n_seq, int rows, int n_heads, int n_q_heads, int hd, int64_t capacity, int max_len) {
    Plan p;
    const int group = n_q_heads / n_heads, each = n_seq > 0 ? (int)(((int64_t)rows * group + n_seq - 1) / n_seq) : 0;
    const int64_t len = max_len < 1 || max_len > capacity ? capacity : max_len;
    p.wide = dtype != HAWK_FP32 && each >= 64 && (int64_t)((each + kTile - 1) / kTile) * n_seq * n_heads * len >= 300000;
    p.tile = !p.wide ? 4 : (each >= 2048 && hd <= 128 ? 8 : 7);
    p.tiles = (int)((int64_t)rows * group >> p.tile) + n_seq;
    // workgroups if the sequences are alike; the numbers that no tile has end at once
    const int size = 1 << p.tile;
    const int64_t blocks = (int64_t)((each + size - 1) / size) * n_seq * n_heads;
    int64_t room = 512, most = len / 512;   // workgroups; parts
    if (!p.wide) {
        room = blocks >= 128 && len > 2048 ? 1024 : (hd <= 64 ? 512 : 256);
        const int64_t kb = len * 2 * hd * (int64_t)type_bytes(dtype) >> 10;   // what a workgroup would read one piece after the other
        most = blocks >= 256 ? kb / 2048 : (blocks >= 128 ? kb / 1024 : (kb < 400 ? 1 : kb / 128));
    }
    int64_t parts = room / (blocks < 1 ? 1 : blocks);
    if (parts > most) parts = most;
    if (parts > 64) parts = 64;
    if (parts < 1) parts = 1;
    int64_t keys = (len + parts - 1) / parts;
    keys = (keys + 127) / 128 * 128;
    p.splits = (int)((len + keys - 1) / keys);
    if (p.splits < 1) p.splits = 1;
    p.split_keys = (int)keys;
    p.waves = blocks * p.splits <= (hd <= 64 ? 512 : 256) ? 8 : 4;
    const size_t vectors = p.splits > 1 ? (size_t)p.splits * rows * n_q_heads : 0;
    p.part_bytes = (vectors * hd * sizeof(float) + 15) / 16 * 16;
    p.ml_bytes = (vectors * 2 * sizeof(float) + 15) / 16 * 16;
    return p;
}

bool shape_ok(const PagedView& c, int rows, int n_q_heads) {
    return rows >= 0 && n_q_heads >= 1 && n_q_heads <= 65535 && n_q_heads % c.n_heads == 0 &&
           ((int64_t)rows * (n_q_heads / c.n_heads) / kTile + c.n_seq) * c.n_heads <= (1 << 22);
}

template <int TYPE, int DP, int NW> void launch_rows(const AttnArgs& a, unsigned grid, hipStream_t stream) {
    const bool easy = a.c.page_size % 16 == 0, exact = a.c.hd == DP;
    auto kern = !easy ? paged_rows_kernel<TYPE, DP, true, false, NW>
                      : (exact ? paged_rows_kernel<TYPE, DP, false, true, NW> : paged_rows_kernel<TYPE, DP, true, true, NW>);
    kern<<<grid, 64 * NW, 0, stream>>>(a);
}
template <int TYPE> void launch_typed(const AttnArgs& a, int waves, unsigned grid, hipStream_t stream) {
    const int hd = a.c.hd;
    if (hd > 128) launch_rows<TYPE, 256, 4>(a, grid, stream);
    else if (hd > 64) waves == 8 ? launch_rows<TYPE, 128, 8>(a, grid, stream) : launch_rows<TYPE, 128, 4>(a, grid, stream);
    else waves == 8 ? launch_rows<TYPE, 64, 8>(a, grid, stream) : launch_rows<TYPE, 64, 4>(a, grid, stream);
}

template <int TYPE, int DP, int KB, int NW> void launch_wide_of(const AttnArgs& a, unsigned grid, hipStream_t stream) {
    const bool easy = a.c.page_size % 16 == 0 && a.c.entry_stride <= (1 << 24), exact = a.c.hd == DP;
    auto kern = !easy ? paged_wide_kernel<TYPE, DP, true, false, KB, NW>
                      : (exact ? paged_wide_kernel<TYPE, DP, false, true, KB, NW> : paged_wide_kernel<TYPE, DP, true, true, KB, NW>);
    kern<<<grid, 64 * NW, 0, stream>>>(a);
}
template <int TYPE> void launch_wide(const AttnArgs& a, unsigned grid, hipStream_t stream) {
    if (a.c.hd > 128) launch_wide_of<TYPE, 256, 32, 4>(a, grid, stream);
    else if (a.c.hd > 64) a.tile == 8 ? launch_wide_of<TYPE, 128, 64, 8>(a, grid, stream) : launch_wide_of<TYPE, 128, 64, 4>(a, grid, stream);
    else a.tile == 8 ? launch_wide_of<TYPE, 64, 64, 8>(a, grid, stream) : launch_wide_of<TYPE, 64, 64, 4>(a, grid, stream);
}

}  // namespace

// log2 of a tile's rows * 10000 + waves of a workgroup * 100 + parts: the dispatch's rules, for the tests as well.
extern "C" int hawk_paged_attention_plan(int dtype, int n_seq, int rows, int n_heads, int n_q_heads, int hd, int capacity, int max_len) {
    if (n_seq < 0 || rows < 0 || n_heads < 1 || n_q_heads < n_heads || capacity < 1) return 0;
    const Plan p = plan_of(dtype, n_seq, rows, n_heads, n_q_heads, hd, capacity, max_len);
    return p.tile * 10000 + (p.wide ? (p.tile == 8 ? 8 : 4) : (hd > 128 ? 4 : p.waves)) * 100 + p.splits;
}

// The row of the buffers that row r of tile `tile` (of 2^tile_log2 rows) is, if the search for the tile ends at sequence s; -1: none. What the
// kernels compute, for the tests.
extern "C" int hawk_paged_attention_row(const int32_t* row_start, int n_past, int s, int rows, int group, int capacity, int tile_log2, int tile, int r) {
    AttnArgs a = {};
    a.r.rows = rows;
    a.group = divisor(group);
    a.c.capacity = capacity;
    a.tile = tile_log2;
    Span t;
    if (!tile_of(a, s, tile, row_start[s], row_start[s + 1], n_past, t)) return -1;
    const int pr = t.first + r;
    return pr < t.n * a.group.d ? t.r0 + pr / a.group : -1;
}

size_t paged_attention_workspace_bytes(const hawk_paged_cache* cache, int rows, int n_q_heads, int max_len) {
    PagedView c;
    if (!paged_view(cache, 0, &c) || !shape_ok(c, rows, n_q_heads)) return 0;
    const Plan p = plan_of(cache->dtype, c.n_seq, rows, c.n_heads, n_q_heads, c.hd, (int64_t)c.max_pages * c.page_size, max_len);
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
    const Plan p = plan_of(cache->dtype, a.c.n_seq, a.r.rows, a.c.n_heads, a.q.n_heads, a.c.hd, (int64_t)a.c.max_pages * a.c.page_size, max_len);
    if (p.part_bytes && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15))) return HAWK_EINVAL;
    if (workspace_bytes < p.part_bytes + p.ml_bytes) return p.part_bytes ? HAWK_ENOMEM : HAWK_EINVAL;
    a.tree = tree;
    a.scale2 = scale * 1.44269504f;
    a.group = divisor(a.q.n_heads / a.c.n_heads);
    a.heads = divisor(a.c.n_heads);
    a.splits = divisor(p.splits);
    a.tile = p.tile;
    a.tiles = p.tiles; a.split_keys = p.split_keys;
    a.part = static_cast<float*>(workspace);
    a.part_ml = reinterpret_cast<float*>(static_cast<char*>(workspace) + p.part_bytes);
    const int64_t grid = (int64_t)p.tiles * p.splits * a.c.n_heads;
    if (grid > (1 << 22)) return HAWK_EINVAL;   // a launch has fewer than 2^32 threads
    if (p.wide && cache->dtype == HAWK_BF16) launch_wide<HAWK_BF16>(a, (unsigned)grid, stream);
    else if (p.wide) launch_wide<HAWK_FP16>(a, (unsigned)grid, stream);
    else if (cache->dtype == HAWK_FP32) launch_typed<HAWK_FP32>(a, p.waves, (unsigned)grid, stream);
    else if (cache->dtype == HAWK_BF16) launch_typed<HAWK_BF16>(a, p.waves, (unsigned)grid, stream);
    else launch_typed<HAWK_FP16>(a, p.waves, (unsigned)grid, stream);
    if (p.splits > 1) {
        const int64_t units = (int64_t)a.r.rows * a.q.n_heads;
        int lanes = 1;
        while (lanes * 8 < a.c.hd) lanes *= 2;
        paged_join_kernel<<<(unsigned)((units + 3) / 4), 256, 0, stream>>>(a, lanes);
    }
    return hipGetLastError() == hipSuccess ? HAWK_OK : HAWK_EDEVICE;
}

}  // namespace hawk
