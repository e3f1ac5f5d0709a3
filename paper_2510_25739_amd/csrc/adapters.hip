// Low-rank adapters of many requests beside a shared projection: out[r] = base[r] + scale[a] B_a (A_a x[r]), a the adapter of row r's sequence.
//
// Rows are grouped by adapter into tiles of 16, once a step (the plan), so that an adapter that many requests use is read once for 16 of
// their rows.  One launch a projection: a workgroup has a tile and some of the columns.  Its waves share the sum over d_in, their parts are
// added in shared memory, and B h is added to base on the way out.  Where a few tiles' A would be a few units' to read, the sums are a launch of their
// own, shared by more workgroups (splits_of).  Both products are computed transposed (h^T = A x^T, out^T = B h^T): a result lane then has
// neighbouring elements of one row.
//
// What bounds it: of single tokens memory (200 rows of 64 adapters of rank 32, 4096 by 11008, 67 MB, 15.0 us with other inputs in turn: 4.5 TB/s), of prompts
// as well (4724 rows of 4096 by 4096, 117 MB, 32 us with other inputs in turn, 24 of one input that the last-level cache holds part of); of few rows a
// chain of latencies (plan, x and A, h, B; one row 3.8 us, where a call that launches nothing but an empty kernel takes 3.7); of large ranks the way of all of A
// into every tile's unit (1219 rows of rank 128, 1280 by 1000, 13.4 us: 412 KB a unit are 5.5 of it).
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

// Once a step, in one workgroup: 96 rows of 8 adapters 4.3 us, 200 single tokens of 64 8.6, 4724 rows of four prompts 13.2; it grows with the rows, and
// with the adapters that a wave's rows have (65536 rows: 102 us of 16 prompts, 550 of single tokens of 64 adapters; 2^20 of 256 13 ms).
//
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
    int n_adapters, rank, d_in, d_out, rows, tiles;
    Divisor parts;                   // workgroups of a tile
    int step;                        // kWhole; in two launches kShrink, kExpand
    int splits;                      // of the sum over d_in (two launches)
    float* sums;                     // [tile][split][rank / 16, rounded up][row][16]
};

enum { kWhole, kShrink, kExpand };

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

// 16 bytes of a type as they lie in memory: requested in one place, used in another.
template <int TYPE> struct Piece {
    static constexpr int kN = 16 / Of<TYPE>::kBytes;
    v4u w;
    __device__ __forceinline__ void load(const char* base, int64_t at) { w = *reinterpret_cast<const v4u*>(base + at * Of<TYPE>::kBytes); }
    __device__ __forceinline__ void store(char* base, int64_t at) const { *reinterpret_cast<v4u*>(base + at * Of<TYPE>::kBytes) = w; }
    __device__ __forceinline__ void widen(float (&x)[kN]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (TYPE == HAWK_FP32) x[i] = __uint_as_float(w[i]);
            else widen2(w[i], TYPE, x[2 * i], x[2 * i + 1]);
        }
    }
    __device__ __forceinline__ void narrow(const float (&x)[kN]) {   // to nearest, ties to even
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (TYPE == HAWK_FP32) w[i] = __float_as_uint(x[i]);
            else w[i] = narrow2(x[2 * i], x[2 * i + 1], TYPE);
        }
    }
};
// Between a wave's writes to shared memory and its other lanes' reads of them: the hardware keeps their order, the compiler has to as well.
__device__ __forceinline__ void wave_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// TYPE: of x and the weights; OUT: of base and out.  NR: groups of 16 of the rank.  NW waves.
// x, A, B, base and out pass between memory and registers as rows' whole 128 bytes, eight rows (four of 256) an instruction, and change places
// with the matrix units' layout - a lane has 16 bytes of one of 16 rows - in shared memory of the wave's own: read in that layout, with 64
// bytes of 16 rows an instruction, memory gave 3.3 instead of 4.4 TB/s, and x, base and out together, 4400 rows of 4096 without their products, took 35
// instead of 28 us.
template <int TYPE, int OUT, int NR, int NW>
__global__ __launch_bounds__(64 * NW, NR <= 2 ? 4 : 2) void adapter_apply_kernel(ApplyArgs a) {
    using T = Of<TYPE>;
    constexpr int ES = T::kBytes, VEC = 16 / ES;                               // values of a piece
    constexpr int RP = 16 * NR, LD = RP + 4;                                   // the rank, rounded up
    constexpr int P = TYPE == HAWK_FP32 ? 1 : (TYPE == HAWK_BF16 && OUT == HAWK_FP32 ? 3 : 2);   // parts of h
    constexpr bool PAIR = TYPE != HAWK_FP32 && NR == 1;                        // two parts of h share a product's 32 features
    constexpr int KS = TYPE == HAWK_FP32 ? NR : (NR + 1) / 2;                  // products over the rank
    constexpr int PP = PAIR ? (P + 1) / 2 : P;
    constexpr int D1 = NR <= 2 ? 2 : 1;                                        // stages of x and A that are requested ahead
    constexpr int D2 = NR == 1 && OUT != HAWK_FP32 ? 2 : 1;                   // columns that are
    constexpr int LR = OUT == HAWK_FP32 ? 16 : 8, NI = LR / 4;                 // lanes of a row of 64 columns, instructions of 16 rows
    // B of 32 bits, twice a stage's size, goes straight into the operands' places
    constexpr bool VIA = TYPE != HAWK_FP32;
    constexpr int PR = VIA ? RP / VEC : 4 * KS;                                // pieces of B that a lane brings for 64 columns (VIA: of a row)
    constexpr int kStage = 16 * (1 + NR) * 128, kSum = NR * 1024, kDelta = 16 * 68 * 4;
    constexpr int kOwn = kStage > kSum ? (kStage > kDelta ? kStage : kDelta) : (kSum > kDelta ? kSum : kDelta);
    static_assert(!VIA || 64 * PR * 16 <= kOwn, "64 columns' weights fit");
    __shared__ __align__(16) char own[NW][kOwn];                               // of a wave: a stage, its part of h, a block of B h
    __shared__ float h[kTile][LD];
    __shared__ float factor[kTile];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), m16 = lane & 15, g = lane >> 4;
    // the parts of a tile on one XCD (workgroups go round the eight of them), so that its rows and its adapter come from that one's L2
    const int turn = (int)blockIdx.x >> 3, eight = turn / a.parts, part = turn - eight * a.parts.d, tile = eight * 8 + ((int)blockIdx.x & 7);
    if (tile >= min(a.plan[0], a.tiles)) return;
    const int32_t* entry = a.plan + kHead + tile * kEntry;
    const int who = __builtin_amdgcn_readfirstlane(entry[0]);
    const bool none = who < 0 || who >= a.n_adapters;
    auto row_of = [&](int i) {
        const int r = entry[1 + i];
        return r < a.rows ? r : -1;
    };
    int row[NI];                         // of base and out
#pragma unroll
    for (int i = 0; i < NI; ++i) row[i] = row_of(i * (16 / NI) + lane / LR);
    const int groups = (a.d_out + 63) >> 6, step = a.parts.d * NW, piece = (lane & (LR - 1)) * Piece<OUT>::kN;
    int q = part * NW + wave;
    if (none) {                          // base alone
        if (a.base == a.out || a.step == kShrink) return;
        for (; q < groups; q += step)
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int c = q * 64 + piece;
                if (c >= a.d_out || row[i] < 0) continue;
                Piece<OUT> y = {};
                if (a.base) y.load(a.base, row[i] * a.base_row + c);
                y.store(a.out, row[i] * a.out_row + c);
            }
        return;
    }
    char* mine = own[wave];
    auto place = [&](int r, int p) { return r * 128 + ((p ^ r) & 7) * 16; };   // of a stage: pieces turned by the row, so that lanes do not meet

    // h^T = A x^T, the waves (of a tile's workgroups, where they share the sum) in turns of 128 bytes of every row
    if (a.step != kExpand) {
        f32x4 acc[NR];
#pragma unroll
        for (int j = 0; j < NR; ++j) acc[j] = (f32x4){0.f, 0.f, 0.f, 0.f};
        const int r8 = lane >> 3, bytes = a.d_in * ES, stages = (bytes + 127) >> 7;
        const int first = a.step == kShrink ? q : wave, turn = a.step == kShrink ? step : NW;
        const int xr[2] = {row_of(r8), row_of(8 + r8)};
        const char* x[2];
        const char* w[2 * NR];
#pragma unroll
        for (int i = 0; i < 2; ++i) x[i] = a.x + (int64_t)max(xr[i], 0) * a.x_row * ES;
#pragma unroll
        for (int i = 0; i < 2 * NR; ++i) w[i] = a.a + (who * a.a_adapter + min(8 * i + r8, a.rank - 1) * a.a_row) * ES;   // (rows behind the rank: see h)
        struct Stage { v4u x[2], w[2 * NR]; } ahead[D1];
        auto request = [&](int t, Stage& st) {
            const int at = t * 128 + (lane & 7) * 16;
            const bool in = at < bytes;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                st.x[i] = (v4u){0u, 0u, 0u, 0u};
                if (in && xr[i] >= 0) st.x[i] = *reinterpret_cast<const v4u*>(x[i] + at);
            }
#pragma unroll
            for (int i = 0; i < 2 * NR; ++i) {
                st.w[i] = (v4u){0u, 0u, 0u, 0u};
                if (in) st.w[i] = *reinterpret_cast<const v4u*>(w[i] + at);
            }
        };
#pragma unroll
        for (int d = 0; d < D1; ++d) request(first + d * turn, ahead[d]);
        for (int t = first; t < stages; t += D1 * turn)
#pragma unroll
            for (int d = 0; d < D1; ++d) {
                if (t + d * turn >= stages) break;
#pragma unroll
                for (int i = 0; i < 2; ++i) *reinterpret_cast<v4u*>(mine + place(8 * i + r8, lane)) = ahead[d].x[i];
#pragma unroll
                for (int i = 0; i < 2 * NR; ++i) *reinterpret_cast<v4u*>(mine + place(16 + 8 * i + r8, lane)) = ahead[d].w[i];
                wave_order();
                request(t + (d + D1) * turn, ahead[d]);
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const v4u xv = *reinterpret_cast<const v4u*>(mine + place(m16, 4 * s + g));
#pragma unroll
                    for (int j = 0; j < NR; ++j) acc[j] = T::mul(*reinterpret_cast<const v4u*>(mine + place(16 + 16 * j + m16, 4 * s + g)), xv, acc[j]);
                }
                wave_order();
            }
#pragma unroll
        for (int j = 0; j < NR; ++j) *reinterpret_cast<f32x4*>(mine + j * 1024 + m16 * 64 + g * 16) = acc[j];   // [..][row][..]
    }

    // 64 columns a wave: row mu of block i of the product stands for column 16 i + mu.  The first ones' weights and base are on their way while h is
    // put together, the next ones' while a wave works on its.
    const char* wb = a.b + who * a.b_adapter * ES;
    struct Columns {
        v4u w[PR];
        Piece<OUT> y[NI];
    } ahead[D2];
    auto weight_at = [&](int col, int p) { return (col * PR + (PR >= 8 ? p ^ (col & (PR - 1)) : p)) * 16; };   // of 64 columns' weights
    auto request = [&](int q, Columns& c) {
        if (q >= groups) return;
#pragma unroll
        for (int i = 0; i < PR; ++i) {       // (behind the rank, where h is zero: the last weights)
            const int n = lane + 64 * i;
            const int col = min(q * 64 + (VIA ? n / PR : 16 * (i / KS) + m16), a.d_out - 1), j = min((VIA ? n % PR : 4 * (i % KS) + g) * VEC, a.rank - VEC);
            c.w[i] = *reinterpret_cast<const v4u*>(wb + (col * a.b_row + j) * ES);
        }
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            c.y[i].w = (v4u){0u, 0u, 0u, 0u};
            if (a.base && row[i] >= 0 && q * 64 + piece < a.d_out) c.y[i].load(a.base, row[i] * a.base_row + q * 64 + piece);
        }
    };
    if (a.step != kShrink)
#pragma unroll
        for (int d = 0; d < D2; ++d) request(q + d * step, ahead[d]);

    __syncthreads();
    for (int i = threadIdx.x; i < kTile * RP; i += 64 * NW) {
        const int j = i / (kTile * 16), r = (i >> 4) & 15, c = i & 15;
        float s = 0.f;
        if (a.step == kExpand) {
            const float* from = a.sums + (int64_t)tile * a.splits * (kTile * RP) + i;
            for (int k0 = 0; k0 < a.splits; k0 += 8) {
                float v[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = k0 + k < a.splits ? from[(k0 + k) * (kTile * RP)] : 0.f;
#pragma unroll
                for (int k = 0; k < 8; ++k) s += v[k];
            }
        } else {
#pragma unroll
            for (int v = 0; v < NW; ++v) s += *reinterpret_cast<const float*>(own[v] + i * 4);
            s = j * 16 + c < a.rank ? s : 0.f;
            if (a.step == kShrink) a.sums[((int64_t)tile * a.splits + part) * (kTile * RP) + i] = s;
        }
        h[r][j * 16 + c] = s;
    }
    if (a.step == kShrink) return;
    __syncthreads();
    // of fp16 the power of two that brings a row's largest h below 2^14: half a step of a part of the smallest is then 2^-39 of the largest,
    // and nothing overflows
    if (TYPE == HAWK_FP16) {
        constexpr int N = 64 * NW / kTile;           // threads of a row
        const int r = (int)threadIdx.x / N;
        float top = 0.f;
#pragma unroll
        for (int j = threadIdx.x % N; j < RP; j += N) {
            const float v = fabsf(h[r][j]);
            top = fmaxf(top, v <= 3.4028235e38f ? v : 0.f);
        }
#pragma unroll
        for (int d = 1; d < N; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
        const int e = top > 0.f ? max(ilogbf(top) - 13, -126) : 0;
        if (threadIdx.x % N == 0) factor[r] = __uint_as_float((unsigned)(e + 127) << 23);
        __syncthreads();
    }
    v4u hv[PP][KS];
    const float up = TYPE == HAWK_FP16 ? factor[m16] : 1.f, scale = a.scale ? a.scale[who] * up : up, down = 1.f / up;
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
    for (; q < groups; q += D2 * step)
#pragma unroll
        for (int d = 0; d < D2; ++d) {
            const int at = q + d * step;
            if (at >= groups) break;
            if constexpr (VIA) {
#pragma unroll
                for (int i = 0; i < PR; ++i) *reinterpret_cast<v4u*>(mine + weight_at((lane + 64 * i) / PR, (lane + 64 * i) % PR)) = ahead[d].w[i];
                wave_order();
            }
            f32x4 o[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                o[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    const v4u w = VIA ? *reinterpret_cast<const v4u*>(mine + weight_at(16 * i + m16, PAIR ? g & 1 : 4 * k + g)) : ahead[d].w[(i * KS + k) % PR];
#pragma unroll
                    for (int p = 0; p < PP; ++p) o[i] = T::mul(w, hv[p][k], o[i]);
                }
            }
            wave_order();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
#pragma unroll
                for (int e = 0; e < 4; ++e) o[i][e] *= scale;
                *reinterpret_cast<f32x4*>(mine + (m16 * 68 + 16 * i + 4 * g) * 4) = o[i];   // [row][column]
            }
            wave_order();
            Piece<OUT> y[NI];
#pragma unroll
            for (int i = 0; i < NI; ++i) y[i] = ahead[d].y[i];
            request(at + D2 * step, ahead[d]);
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                float v[Piece<OUT>::kN];
                y[i].widen(v);
                const float* o = reinterpret_cast<const float*>(mine) + (i * (16 / NI) + lane / LR) * 68 + piece;
#pragma unroll
                for (int e = 0; e < Piece<OUT>::kN; e += 4) {
                    const f32x4 b = *reinterpret_cast<const f32x4*>(o + e);
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[e + k] += b[k];
                }
                y[i].narrow(v);
                if (row[i] >= 0 && at * 64 + piece < a.d_out) y[i].store(a.out, row[i] * a.out_row + at * 64 + piece);
            }
            wave_order();
        }
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
int status() { return hipGetLastError() == hipSuccess ? HAWK_OK : HAWK_EDEVICE; }
bool matrix_ok(const hawk_matrix* m, int width) {
    return m && m->data && aligned16(m->data) && is_type(m->dtype) && !(m->row_stride & 7) && m->row_stride >= 0 && width > 0;
}

constexpr int kWaves = 8;
template <int TYPE, int OUT> void launch_rank(const ApplyArgs& a, unsigned grid, hipStream_t stream) {
    auto kern = a.rank <= 16 ? adapter_apply_kernel<TYPE, OUT, 1, kWaves>
                             : (a.rank <= 32 ? adapter_apply_kernel<TYPE, OUT, 2, kWaves>
                                             : (a.rank <= 64 ? adapter_apply_kernel<TYPE, OUT, 4, kWaves> : adapter_apply_kernel<TYPE, OUT, 8, kWaves>));
    kern<<<grid, 64 * kWaves, 0, stream>>>(a);
}
template <int TYPE> void launch_typed(const ApplyArgs& a, int out, unsigned grid, hipStream_t stream) {
    if (out == HAWK_FP32) launch_rank<TYPE, HAWK_FP32>(a, grid, stream);
    else if (out == HAWK_BF16) launch_rank<TYPE, HAWK_BF16>(a, grid, stream);
    else launch_rank<TYPE, HAWK_FP16>(a, grid, stream);
}

// In how many workgroups a tile's sum over d_in is made, in a launch of its own (0: in every one that has some of its columns).  A unit reads A at 75 GB/s,
// whatever lies behind it; s of them save (s - 1) / s of that and cost a launch, 1.7 us in a graph and 5 for the host (us in one launch / two, in a
// graph: one row, 4096 by 4096, rank 32 7.6 / 6.1, 64 11.0 / 8.2, 128 20.2 / 13.4; 11008 by 4096, rank 16 10.3 / 5.9, 32 13.6 / 6.6, 128 38.5 / 17.1; three workgroups a
// tile, 64 rows of 64 adapters, 4096 by 4096, rank 64 16.3 / 18.1, 11008 by 4096, rank 32 17.9 / 16.2, 128 73 / 61; two, 1500 rows, 4096 by 4096, rank 128
// 30.4 / 30.8, 11008 by 4096, rank 64 29.5 / 26.2).  The border is where calls that are not captured lose nothing either (one row of 4096 by 4096, rank 64
// 11.4 / 13.3; of 11008, rank 32 13.8 / 12.9).
constexpr int64_t kSplitBytes = 400 << 10;
int splits_of(const hawk_adapters* w, int tiles) {
    const int64_t row = w->d_in * (int64_t)type_bytes(w->dtype), stages = (row + 127) / 128;
    const int64_t most = std::min<int64_t>(256 / std::max(tiles, 1), (stages + kWaves - 1) / kWaves);
    return most >= 2 && row * w->rank * (most - 1) >= kSplitBytes * (most + 1) ? (int)most : 0;
}
size_t sums_bytes(const hawk_adapters* w, int tiles, int splits) {
    const int nr = w->rank <= 16 ? 1 : (w->rank <= 32 ? 2 : (w->rank <= 64 ? 4 : 8));
    return (size_t)tiles * splits * kTile * 16 * nr * sizeof(float);
}
bool weights_ok(const hawk_adapters* w) {
    return w && is_type(w->dtype) && w->n_adapters >= 0 && w->rank >= 8 && w->rank <= 128 && w->rank % 8 == 0 && w->d_in >= 8 && w->d_in % 8 == 0 &&
           w->d_out >= 8 && w->d_out % 8 == 0 && w->d_in <= (1 << 24) && w->d_out <= (1 << 24);
}

}  // namespace

size_t adapter_apply_workspace_bytes(const hawk_adapters* w, int rows) {
    if (!weights_ok(w) || rows < 1 || adapter_plan_bytes(rows, w->n_adapters) == 0) return 0;
    const int tiles = most_tiles(rows, w->n_adapters);
    return sums_bytes(w, tiles, splits_of(w, tiles));
}

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
                         const hawk_matrix* out, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!weights_ok(w) || rows < 0) return HAWK_EINVAL;
    if ((w->a_adapter_stride | w->a_row_stride | w->b_adapter_stride | w->b_row_stride) & 7) return HAWK_EINVAL;
    if (w->a_adapter_stride < 0 || w->b_adapter_stride < 0 || w->a_row_stride < w->d_in || w->b_row_stride < w->rank) return HAWK_EINVAL;
    const size_t need = adapter_plan_bytes(rows, w->n_adapters);
    if (need == 0) return HAWK_EINVAL;
    if (rows == 0) return HAWK_OK;
    if (w->n_adapters > 0 && (!w->a || !w->b || !aligned16(w->a) || !aligned16(w->b))) return HAWK_EINVAL;
    if (!matrix_ok(x, w->d_in) || !matrix_ok(out, w->d_out) || (base && !matrix_ok(base, w->d_out))) return HAWK_EINVAL;
    if (x->dtype != w->dtype || (base && base->dtype != out->dtype) || (rows > 1 && out->row_stride < w->d_out)) return HAWK_EINVAL;
    // a tile's workgroups read its rows of x while others write theirs of out; base and out of one piece are read and written by the same lane
    auto over = [&](const hawk_matrix* m, int width) {
        const int64_t es = type_bytes(m->dtype), eo = type_bytes(out->dtype);
        return rows_meet(m->data, m->row_stride * es, width * es, out->data, out->row_stride * eo, w->d_out * eo, rows);
    };
    const bool in_place = base && base->data == out->data && (rows < 2 || base->row_stride == out->row_stride);
    if (over(x, w->d_in) || (base && !in_place && over(base, w->d_out))) return HAWK_EINVAL;
    if (!plan || !aligned16(plan)) return HAWK_EINVAL;
    if (plan_bytes < need) return HAWK_ENOMEM;
    ApplyArgs a = {};
    a.plan = static_cast<const int32_t*>(plan);
    a.a = static_cast<const char*>(w->a); a.b = static_cast<const char*>(w->b); a.scale = w->scale;
    a.x = static_cast<const char*>(x->data); a.base = base ? static_cast<const char*>(base->data) : nullptr; a.out = static_cast<char*>(out->data);
    a.a_adapter = w->a_adapter_stride; a.a_row = w->a_row_stride; a.b_adapter = w->b_adapter_stride; a.b_row = w->b_row_stride;
    a.x_row = x->row_stride; a.base_row = base ? base->row_stride : 0; a.out_row = out->row_stride;
    a.n_adapters = w->n_adapters; a.rank = w->rank; a.d_in = w->d_in; a.d_out = w->d_out; a.rows = rows;
    a.tiles = most_tiles(rows, w->n_adapters);
    // Every part of a tile's columns makes the tile's h again, so as many as there are idle units to do it (us with 1 / 2 / 3 / 4 / 6 / 8 parts, by the tiles there can be: 15 of
    // 1280 by 3456, rank 16, 8.8 / 6.6 / 6.0 / 5.4 / 5.3 / 4.7; 77 of 4096 by 11008, rank 32, 27.0 / 18.3 / 15.6 / 15.4 / 17.6 / 16.9; 304 of 4096 by 4096,
    // rank 16, 31.5 / 30.9 / 33.7 / 37.3 / 43.3 / 48; 80 of 1280 by 1000, rank 128, 15.6 / 13.1 / 13.2 / 23.3 / 23.4 / 29.8).
    const int groups = (a.d_out + 63) / 64, parts = std::max(1, std::min((groups + kWaves - 1) / kWaves, 256 / std::max(1, a.tiles)));
    auto launch = [&](int step, int n) {
        a.step = step;
        a.parts = divisor(n);
        const unsigned grid = (unsigned)((a.tiles + 7) / 8 * 8 * n);
        if (w->dtype == HAWK_FP32) launch_typed<HAWK_FP32>(a, out->dtype, grid, stream);
        else if (w->dtype == HAWK_BF16) launch_typed<HAWK_BF16>(a, out->dtype, grid, stream);
        else launch_typed<HAWK_FP16>(a, out->dtype, grid, stream);
    };
    a.splits = splits_of(w, a.tiles);
    if (a.splits == 0) {
        launch(kWhole, parts);
    } else {
        if (!workspace || !aligned16(workspace)) return HAWK_EINVAL;
        if (workspace_bytes < sums_bytes(w, a.tiles, a.splits)) return HAWK_ENOMEM;
        a.sums = static_cast<float*>(workspace);
        launch(kShrink, a.splits);
        launch(kExpand, parts);
    }
    return status();
}

}  // namespace hawk
