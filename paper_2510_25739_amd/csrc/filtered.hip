// One draw a row from logits cut by top-k, top-p and min-p, each row with parameters of its own.
//
// z = l / T in 32 bits, w = exp(z - reference).  Entries are ordered by z, equal ones by index; what is kept is a beginning of that order: the
// top_k first, of these the ones before which less than top_p of their mass lies, of these the ones with w >= min_p times the largest.  The token
// is the first in ascending index whose sum of kept weights exceeds u times the whole.
//
// Weights are whole multiples of 2^-S of the reference's (S as large as n of them still sum up in 64 bits: 48 for 16384 entries), rounded to
// nearest, so that a sum has one value whatever the order it is made in, and masses can be counted in bins by atomics.  What that
// rounding moves is n 2^-(S + 1) at most, 2^-35 for 16384 entries; the sum of random errors is a hundredth of it.  (Rows in parts: below.)
//
// The border of a cut - its last entry - is found by bins: linear ones of z below the maximum first, then, while more than a few entries share the
// border's bin, bins of the keys' bits in that range and, among equal ones, of the index.  The few are ranked against each other.
//
// Up to 16384 entries one workgroup of 1024 threads has a row in its registers (sample_filtered_kernel).  Longer rows are cut into parts, a
// workgroup each, in three launches: the parts' bins (filter_bins_kernel); sums of what is kept for certain, and the entries of the bins
// that a border may be in (filter_parts_kernel); the borders and the draw, a workgroup a row (filter_draw_kernel).  Where the border's bins
// hold more than a quarter of a part that last workgroup looks for it in the row itself; rows whose logits are beyond the bins' grid are its alone.
//
// What bounds it: not memory (48 rows of 65536 are 2.6 us of it) but a workgroup's instructions and barriers.  One row of 16384 entries, 15.5 us, is
// a dozen steps of sixteen waves with a barrier behind each, 1440 vector instructions a wave, which take 9.6 us to issue; 96 rows of which some have no top-k
// 21.6 us, the exponentials of 16 entries a thread among them; 48 rows of 65536 34.5 us one call among others, three launches of 10.7, 14.3 and 11.0 by
// themselves, of which nearly 4 each is a launch; 4 of 200003, 16 bits, 33.9 us.
#include "filtered.h"
#include "paged.h"
#include "sample_rows.h"

#include <algorithm>

// z is a rounded product wherever it is compared, binned or subtracted from the reference.
#pragma clang fp contract(off)

namespace hawk {

namespace {

typedef unsigned long long u64;

constexpr int kBinCount = 1024, kFine = 512;     // linear bins; those of a closer look
constexpr float kPerUnit = 32.f;     // bins of a unit of z
constexpr int kPartBins = 512;       // bins of a part of a long row
constexpr int kLooks = 7;             // closer looks there can be: 32 bits of a key and 20 of an index, nine at a time
constexpr int kFew = 64;             // entries that are ranked against each other (a look at 220 takes 1.6 us, ranking them 4)
constexpr int kChunk = 256;          // entries that a wave has of four a lane: sums of kept weights are held for each
constexpr int kMostEntries = 1 << 20, kChunks = kMostEntries / kChunk;
constexpr int kTop = 2 * NT;         // entries of a top-k that goes on as a list, two a thread

struct FilterArgs {
    const char* logits;
    int64_t row_stride;              // elements
    const int32_t *skip, *top_k;
    const float *u, *temperature, *top_p, *min_p;
    int dtype, n, unit;              // unit: S
    unsigned apart;                  // fp32 steps between scaled logits that differ, at least (see find_border)
    int32_t *out_token, *out_kept;
    float* out_prob;
    // rows in parts
    int parts;
    char* room;
};

struct Border { float z; int at; };  // entries are inside if z is larger, or equal and their index not above `at`
__device__ __forceinline__ bool inside(const Border& b, float z, int j) { return z > b.z || (z == b.z && j <= b.at); }
constexpr Border kNoBorder = {-3.4028235e38f, 0x7FFFFFFF};       // of all entries there are (minus infinity: none)
// An entry is before a cut if fewer than K entries and a mass below M lie before it, in order.
struct Cut { u64 M; unsigned K; };
// Where the border lies: entries and mass before, m entries with keys lo..hi, of equal keys with indices first..last.
struct Range { u64 before; unsigned ahead, m, lo, hi; int first, last; };
struct Found { Border border; u64 mass; };   // mass: of all entries up to the border

struct Picked { int bin; unsigned m, ahead; u64 before; };   // a bin: its entries; entries and mass before it
struct CutShared {
    u64 mass[kBinCount], fine_mass[kFine];
    unsigned count[kBinCount], fine[kFine];          // fine: zero between uses
    u64 w[kFew], base;
    unsigned key[kFew], lo, hi;
    int at[kFew], order[kFew], n, chunk;
    Picked picked;
    double steps[kSteps], log_p;
    u64 sum[NW];
    int isum[NW];
    float fmax[NW];
};

__device__ __forceinline__ u64 lane_u64(u64 v, int l) {
    return ((u64)(unsigned)__builtin_amdgcn_readlane((int)(v >> 32), l) << 32) | (unsigned)__builtin_amdgcn_readlane((int)(unsigned)v, l);
}
__device__ __forceinline__ u64 addu(u64 a, u64 b) { return a + b; }
__device__ __forceinline__ int addi(int a, int b) { return a + b; }
__device__ __forceinline__ u64 wave_sum_u64(u64 v) {
    ROW_ALLREDUCE(v, addu, dpp_u64)
    return (lane_u64(v, 0) + lane_u64(v, 16)) + (lane_u64(v, 32) + lane_u64(v, 48));
}
// Sums over the wave of four numbers a lane: halves of two change places, so that one addition is for both, then rows.  Lanes of row 0 have the
// first's sum, of row 2 the second's, of row 1 the third's, of row 3 the fourth's.
__device__ __forceinline__ u64 swap_add32(u64 a, u64 b) {
    const auto lo = __builtin_amdgcn_permlane32_swap((unsigned)a, (unsigned)b, false, false);
    const auto hi = __builtin_amdgcn_permlane32_swap((unsigned)(a >> 32), (unsigned)(b >> 32), false, false);
    return ((u64)hi[0] << 32 | lo[0]) + ((u64)hi[1] << 32 | lo[1]);
}
__device__ __forceinline__ u64 swap_add16(u64 a, u64 b) {
    const auto lo = __builtin_amdgcn_permlane16_swap((unsigned)a, (unsigned)b, false, false);
    const auto hi = __builtin_amdgcn_permlane16_swap((unsigned)(a >> 32), (unsigned)(b >> 32), false, false);
    return ((u64)hi[0] << 32 | lo[0]) + ((u64)hi[1] << 32 | lo[1]);
}
__device__ __forceinline__ u64 wave_sums_u64(u64 a, u64 b, u64 c, u64 d) {
    u64 v = swap_add16(swap_add32(a, b), swap_add32(c, d));
    ROW_ALLREDUCE(v, addu, dpp_u64)
    return v;
}
__device__ __forceinline__ int which_of_four(int lane) { return (lane >> 5) + 2 * (lane >> 4 & 1); }
__device__ __forceinline__ int wave_sum_i(int v) {
    ROW_ALLREDUCE(v, addi, dpp_i)
    return (__builtin_amdgcn_readlane(v, 0) + __builtin_amdgcn_readlane(v, 16)) + (__builtin_amdgcn_readlane(v, 32) + __builtin_amdgcn_readlane(v, 48));
}
__device__ __forceinline__ u64 wave_incl_scan_u64(u64 v) {
    v += dpp_u64<0x111>(v);
    v += dpp_u64<0x112>(v);
    v += dpp_u64<0x114>(v);
    v += dpp_u64<0x118>(v);
    const u64 r0 = lane_u64(v, 15), r1 = lane_u64(v, 31), r2 = lane_u64(v, 47);
    const int row = (threadIdx.x & 63) >> 4;
    return v + (row == 0 ? 0ull : row == 1 ? r0 : row == 2 ? r0 + r1 : r0 + r1 + r2);
}

// A weight as a whole number of 2^-S: a sum with 2^(52 - S) has it in its last 52 bits.
struct Weigh {
    double ref, magic;
    const double* steps;
    __device__ __forceinline__ double real(float z) const { return exp_below((double)z - ref, steps); }
    __device__ __forceinline__ u64 operator()(float z) const {   // (below -690 it is 0 whatever the weight)
        return (u64)__double_as_longlong(exp_near(fmax((double)z - ref, -690.0), steps) + magic) & 0xFFFFFFFFFFFFFull;
    }
};
__device__ __forceinline__ double magic_of(int unit) { return __hiloint2double((1075 - unit) << 20, 0); }

// ceil(p * mass), 0 < p < 1, exactly: p is a whole number of 24 bits times a power of two.
__device__ __forceinline__ u64 share_of(float p, u64 mass) {
    const unsigned b = __float_as_uint(p), e = b >> 23;
    const u64 m = e ? (b & 0x7FFFFFu) | 0x800000u : b & 0x7FFFFFu;
    const int s = 150 - (int)max(e, 1u);             // p = m / 2^s, s >= 24
    const u64 lo = m * mass, hi = __umul64hi(m, mass);
    if (s >= 128) return (lo | hi) ? 1ull : 0ull;
    u64 q, rest;
    if (s >= 64) {
        q = s == 64 ? hi : hi >> (s - 64);
        rest = lo | (s == 64 ? 0ull : hi << (128 - s));
    } else {
        q = (lo >> s) | (hi << (64 - s));
        rest = lo << (64 - s);
    }
    return q + (rest ? 1ull : 0ull);
}

// A row's values: z, minus infinity where there is nothing to draw (past the end, NaN).
struct Source {
    const char* l;
    int dtype, n;
    float inv_t;
    bool fours, infinite;            // four at a time can be read at once; the row's maximum is infinite
    __device__ __forceinline__ float scaled(float v) const {
        float z = v * inv_t;
        z = z == z ? z : -INFINITY;
        return infinite ? (z == INFINITY ? 0.f : -INFINITY) : z;
    }
    __device__ __forceinline__ float one(int j) const {
        if (dtype == HAWK_FP32) return reinterpret_cast<const float*>(l)[j];
        float a, b;
        widen2(reinterpret_cast<const unsigned short*>(l)[j], dtype, a, b);
        return a;
    }
    __device__ __forceinline__ void four(int j, float (&z)[4]) const {
        if (fours && j + 3 < n) {
            load4(l, j, dtype, z);
#pragma unroll
            for (int i = 0; i < 4; ++i) z[i] = scaled(z[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) z[i] = j + i < n ? scaled(one(j + i)) : -INFINITY;
        }
    }
};
// What a row asks for.
struct Asked {
    float T, top_p, min_p;
    unsigned k;
    bool greedy, by_k, by_p;
};
__device__ __forceinline__ Asked asked_of(const FilterArgs& a, int r) {
    Asked q;
    q.T = a.temperature ? a.temperature[r] : 1.f;
    q.greedy = !(q.T > 0.f);
    const int k = a.top_k ? a.top_k[r] : 0;
    q.by_k = k >= 1 && k < a.n;
    q.k = q.by_k ? (unsigned)k : 0xFFFFFFFFu;
    const float p = a.top_p ? a.top_p[r] : 1.f, m = a.min_p ? a.min_p[r] : 0.f;
    q.by_p = p < 1.f;
    q.top_p = fmaxf(p, 0.f);
    q.min_p = m > 1.f ? 1.f : (m > 0.f ? m : 0.f);   // (NaN: none)
    return q;
}
__device__ __forceinline__ Source source_of(const FilterArgs& a, int r, const Asked& q) {
    Source s;
    const int es = a.dtype == HAWK_FP32 ? 4 : 2;
    s.dtype = a.dtype;
    s.n = a.n;
    s.l = a.logits + r * a.row_stride * es;
    s.fours = (reinterpret_cast<uintptr_t>(s.l) & (4 * es - 1)) == 0;
    s.inv_t = q.greedy ? 1.f : (float)(1.0 / (double)q.T);
    s.infinite = false;
    return s;
}
__device__ __forceinline__ void give(const FilterArgs& a, int r, int token, float prob, int kept) {
    a.out_token[r] = token;
    if (a.out_prob) a.out_prob[r] = prob;
    if (a.out_kept) a.out_kept[r] = kept;
}
// The smallest z that min_p keeps, in 64 bits: held weights are too coarse for it, multiples of 2^-48 against a min_p that may be 2^-149.  zmax + log(min_p)
// is rounded to the nearest z, which is inside or the last one outside.  The logarithm is the second wave's while the first one fills the table of
// the exponential (300 rows of 20000 with top-k and min-p 46.9 us, with a logarithm in every wave 49.1).
__device__ __forceinline__ void fill_log(const Asked& q, double* log_p) {   // ends without a barrier
    if (threadIdx.x == 64) *log_p = q.min_p > 0.f ? log((double)q.min_p) : 0.0;
}
__device__ __forceinline__ float lowest_of(const Asked& q, float zmax, const double* steps, double log_p) {
    if (!(q.min_p > 0.f)) return -INFINITY;
    const float z = (float)((double)zmax + log_p);
    return exp_below((double)z - (double)zmax, steps) >= (double)q.min_p ? z : key_to_float(fkey(z) + 1u);
}

// Bins of which each thread has one, in order: its entries and mass, what lies before it, and all entries.  One barrier.
struct Bin { unsigned m, ahead, all; u64 mass, before; };
__device__ __forceinline__ Bin scan_bins(unsigned m, u64 mass, bool masses, int (&counts)[NW], u64 (&sums)[NW]) {
    const int lane = threadIdx.x & 63, wave = wave_id(), upto = wave_incl_scan_i((int)m);
    const u64 mass_upto = masses ? wave_incl_scan_u64(mass) : 0ull;
    if (lane == 63) {
        counts[wave] = upto;
        if (masses) sums[wave] = mass_upto;
    }
    __syncthreads();
    Bin b;
    int base;
    b.m = m;
    b.mass = mass;
    b.all = (unsigned)wave_base_i(counts, wave, base);
    b.ahead = (unsigned)(base + upto) - m;
    b.before = 0ull;
    if (masses) {
        const u64 s = lane < NW ? sums[lane] : 0ull, x = wave_incl_scan_u64(s);
        b.before = (wave > 0 ? lane_u64(x, wave - 1) : 0ull) + mass_upto - mass;
    }
    return b;
}
// Whether the bin holds the cut's border: it begins before the cut, and the cut is in it or there is nothing behind.
__device__ __forceinline__ bool holds(const Bin& b, const Cut& cut) {
    return b.m > 0u && b.ahead < cut.K && b.before < cut.M && (b.ahead + b.m >= cut.K || b.before + b.mass >= cut.M || b.ahead + b.m == b.all);
}
// Of the NB bins the one that holds a cut's border; all threads have the result, and sh.n is zero.  Two barriers, one of them at the end.
template <int NB>
__device__ __forceinline__ Picked pick_bin(const unsigned* count, const u64* mass, bool masses, const Cut& cut, unsigned ahead, u64 before, CutShared& sh) {
    const int tid = threadIdx.x;
    Bin b = scan_bins(tid < NB ? count[tid] : 0u, tid < NB && masses ? mass[tid] : 0ull, masses, sh.isum, sh.sum);
    b.ahead += ahead;
    b.all += ahead;
    b.before += before;
    if (holds(b, cut)) {
        const Picked p = {tid, b.m, b.ahead, b.before};
        sh.picked = p;
    }
    if (tid == 0) sh.n = 0;
    __syncthreads();
    return sh.picked;
}

// The border of a cut within a range.  each(f): f(index, z) of this thread's entries that may be in it.  masses: weights count.  All threads
// call, sh.n is zero; what it leaves in sh is read until the next barrier.
template <class Each>
__device__ __forceinline__ Found find_border(const Each& each, const Weigh& weigh, bool masses, const Cut& cut, Range r, CutShared& sh, unsigned apart) {
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_id();
    // keys of which there is one value at most: different ones of logits of 16 bits are `apart` (but for those too small to keep their distance)
    auto single = [&]() { return r.lo == r.hi || (r.hi - r.lo < apart && (r.lo >= 0x80800000u || r.hi <= 0x7F7FFFFFu)); };
    // logits of 16 bits: the many are a few values at most; where bins are wider than that, what the range really spans saves a look or two
    if (apart > 1u && r.m > (unsigned)kFew && (r.hi - r.lo) >> 9 >= apart) {
        unsigned lo = 0xFFFFFFFFu, hi = 0u;
        each([&](int, float z) {
            lo = min(lo, fkey(z));
            hi = max(hi, fkey(z));
        });
        if (tid == 0) { sh.lo = 0xFFFFFFFFu; sh.hi = 0u; }
        __syncthreads();
        for (int d = 1; d < 64; d <<= 1) {
            lo = min(lo, (unsigned)__shfl_xor((int)lo, d));
            hi = max(hi, (unsigned)__shfl_xor((int)hi, d));
        }
        if (lane == 0) {
            atomicMin(&sh.lo, lo);
            atomicMax(&sh.hi, hi);
        }
        __syncthreads();
        r.lo = sh.lo;
        r.hi = sh.hi;
    }
    for (int look = 0; look < kLooks && r.m > (unsigned)kFew; ++look) {
        const bool by_key = !single();
        const unsigned span = by_key ? r.hi - r.lo : (unsigned)(r.last - r.first);
        const int s = max(0, 32 - __clz((int)span) - 9);     // (nine bits: kFine bins)
        each([&](int j, float z) {
            const unsigned k = fkey(z);
            if (k < r.lo || k > r.hi || (!by_key && (j < r.first || j > r.last))) return;
            const unsigned d = (by_key ? r.hi - k : (unsigned)(j - r.first)) >> s;
            atomicAdd(&sh.fine[d], 1u);
            if (masses) atomicAdd(&sh.fine_mass[d], weigh(z));
        });
        __syncthreads();
        const Picked p = pick_bin<kFine>(sh.fine, sh.fine_mass, masses, cut, r.ahead, r.before, sh);
        const unsigned d = (unsigned)p.bin, up = ((d + 1u) << s) - 1u;
        r.m = p.m;
        r.ahead = p.ahead;
        r.before = p.before;
        if (by_key) {
            const unsigned hi = r.hi;
            r.lo = hi - min(hi - r.lo, up);
            r.hi = hi - (d << s);
        } else {
            const int first = r.first;
            r.first = first + (int)(d << s);
            r.last = (int)min((unsigned)r.last, (unsigned)first + up);
        }
        if (tid < kFine) { sh.fine[tid] = 0u; sh.fine_mass[tid] = 0ull; }
        __syncthreads();
    }
    each([&](int j, float z) {
        const unsigned k = fkey(z);
        if (k < r.lo || k > r.hi || j < r.first || j > r.last) return;
        const int i = atomicAdd(&sh.n, 1);
        if (i >= kFew) return;       // (there are r.m of them)
        sh.key[i] = k;
        sh.at[i] = j;
        sh.w[i] = masses ? weigh(z) : 0ull;
    });
    __syncthreads();
    // A wave ranks every sixteenth entry, its lanes compare it with all others.
    const int m = min((int)r.m, kFew);
    const unsigned k = lane < m ? sh.key[lane] : 0u;
    const int at = lane < m ? sh.at[lane] : 0x7FFFFFFF;
#pragma unroll
    for (int t = 0; t < kFew / NW; ++t) {
        const int i = t * NW + wave;
        if (i >= m) break;
        const unsigned mk = (unsigned)__builtin_amdgcn_readlane((int)k, i);
        const int ma = __builtin_amdgcn_readlane(at, i), rank = __popcll(__ballot(k > mk || (k == mk && at < ma)));
        if (lane == 0) sh.order[rank] = i;
    }
    __syncthreads();
    // Then in order: every wave finds the last entry before the cut.
    u64 own = 0ull;
    int n_in = (int)min((unsigned)m, cut.K - r.ahead);
    if (masses) {
        const u64 w = lane < m ? sh.w[sh.order[lane]] : 0ull, upto = wave_incl_scan_u64(w);
        n_in = min(n_in, __popcll(__ballot(lane < m && r.before + upto - w < cut.M)));
        own = lane_u64(upto, max(n_in, 1) - 1);
    }
    const int i = sh.order[max(n_in, 1) - 1];
    const Found out = {{key_to_float(sh.key[i]), sh.at[i]}, r.before + own};
    return out;
}

// Which keys bin b of the linear ones has: z is between its ends but for the rounding of zmax - z.
__device__ __forceinline__ int bin_of(float zmax, float z) { return (int)fminf((zmax - z) * kPerUnit, (float)(kBinCount - 1)); }
__device__ __forceinline__ Range bin_range(float zmax, const Picked& p) {
    Range r;
    const int b = p.bin;
    r.before = p.before;
    r.ahead = p.ahead;
    r.m = p.m;
    const double top = (double)zmax - b / (double)kPerUnit * (1.0 - 0x1p-23), low = (double)zmax - (b + 1) / (double)kPerUnit * (1.0 + 0x1p-23);
    r.hi = b == 0 ? fkey(zmax) : fkey((float)top) + 1u;
    r.lo = b == kBinCount - 1 ? 0u : fkey((float)low) - 1u;
    r.first = 0;
    r.last = kMostEntries - 1;
    return r;
}

// Four neighbouring entries of a lane, 256 of a wave: the one in which the sum of kept weights from `base` on first exceeds target.
template <class Kept>
__device__ __forceinline__ void draw_of_chunk(const FilterArgs& a, int r, int j, const float (&z)[4], const Kept& kept, const Weigh& weigh, u64 base, u64 target,
                                              u64 total) {
    u64 w[4], s = 0ull;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        w[i] = kept(z[i], j + i);
        s += w[i];
    }
    u64 at = base + wave_incl_scan_u64(s) - s;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (at <= target && target < at + w[i]) {
            a.out_token[r] = j + i;
            if (a.out_prob) a.out_prob[r] = (float)(weigh.real(z[i]) * __hiloint2double((1023 + a.unit) << 20, 0) / (double)total);
        }
        at += w[i];
    }
}
__device__ __forceinline__ u64 target_of(const FilterArgs& a, int r, u64 total) {   // the first sum above it
    return min((u64)(fmax((double)a.u[r], 0.0) * (double)total), total - 1ull);
}

// Sums of chunks (in sums, n of them): finds the one in which the sum first exceeds u times the whole.  All threads call and have the result.
__device__ __forceinline__ int pick_chunk(const FilterArgs& a, int r, const u64* sums, int n, CutShared& sh, u64& base, u64& target, u64& total) {
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_id();
    u64 s[kChunks / NT], own = 0ull;
#pragma unroll
    for (int i = 0; i < kChunks / NT; ++i) {
        s[i] = tid * (kChunks / NT) + i < n ? sums[tid * (kChunks / NT) + i] : 0ull;
        own += s[i];
    }
    const u64 upto = wave_incl_scan_u64(own);
    if (lane == 63) sh.sum[wave] = upto;
    if (tid == 0) { sh.chunk = 0; sh.base = 0ull; }
    __syncthreads();
    u64 before = 0ull;
    total = 0ull;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        before += w < wave ? sh.sum[w] : 0ull;
        total += sh.sum[w];
    }
    before += upto - own;
    target = target_of(a, r, total);
#pragma unroll
    for (int i = 0; i < kChunks / NT; ++i) {
        if (before <= target && target < before + s[i]) {
            sh.chunk = tid * (kChunks / NT) + i;
            sh.base = before;
        }
        before += s[i];
    }
    __syncthreads();
    base = sh.base;
    return sh.chunk;
}

// The entries inside a top-k's border, in index order: with a thousand of sixteen thousand left, exponentials and sums are one or two a thread
// instead of sixteen.
struct TopList {
    float z[kTop];
    int at[kTop], total[64];
};
// z: the row's entries as whole_row has them.  All threads call; returns how many there are.  Ends with a barrier.
template <int E> __device__ __forceinline__ int make_list(const float (&z)[E], const Border& border, TopList& list) {
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_id();
    u64 own = 0ull;                  // counts of the groups, 16 bits each
    unsigned in = 0u;
#pragma unroll
    for (int e = 0; e < E; ++e) in |= inside(border, z[e], entry<E>(e, tid)) ? 1u << e : 0u;
#pragma unroll
    for (int g = 0; g < E / 4; ++g) own |= (u64)__popc(in >> 4 * g & 15u) << 16 * g;
    const u64 upto = wave_incl_scan_u64(own);
    if (lane == 63)
#pragma unroll
        for (int g = 0; g < E / 4; ++g) list.total[g * NW + wave] = (int)(upto >> 16 * g & 0xFFFFull);
    __syncthreads();
    const int t = lane < E / 4 * NW ? list.total[lane] : 0, sum = wave_incl_scan_i(t), n = __builtin_amdgcn_readlane(sum, 63);
#pragma unroll
    for (int g = 0; g < E / 4; ++g) {
        int at = __builtin_amdgcn_readlane(sum - t, g * NW + wave) + (int)((upto - own) >> 16 * g & 0xFFFFull);
#pragma unroll
        for (int e = 4 * g; e < 4 * g + 4; ++e)
            if (in >> e & 1u) {
                list.z[at & (kTop - 1)] = z[e];
                list.at[at & (kTop - 1)] = entry<E>(e, tid);
                ++at;
            }
    }
    __syncthreads();
    return n;
}

// The draw from n entries of a list, two neighbours a thread.  sh.count and sh.mass: the counts of all entries, and zeros.
__device__ __forceinline__ void draw_of_list(const FilterArgs& a, int r, const Asked& q, float zmax, const Weigh& weigh, int n, const TopList& list, CutShared& sh) {
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_id();
    float z[2];
    int at[2];
    u64 w[2];
    sh.count[tid] = 0u;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const bool there = 2 * tid + i < n;
        z[i] = there ? list.z[2 * tid + i] : -INFINITY;
        at[i] = there ? list.at[2 * tid + i] : 0;
        w[i] = there ? weigh(z[i]) : 0ull;
    }
    Border border = kNoBorder;
    if (q.by_p) {
        u64 mass = wave_sum_u64(w[0] + w[1]);
        if (lane == 0) sh.sum[wave] = mass;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (z[i] > -INFINITY) {
                const int b = bin_of(zmax, z[i]);
                atomicAdd(&sh.count[b], 1u);
                atomicAdd(&sh.mass[b], w[i]);
            }
        mass = 0ull;
#pragma unroll
        for (int v = 0; v < NW; ++v) mass += sh.sum[v];
        __syncthreads();
        const Cut cut = {maxu64(share_of(q.top_p, mass), 1ull), 0xFFFFFFFFu};
        const Picked p = pick_bin<kBinCount>(sh.count, sh.mass, true, cut, 0u, 0ull, sh);
        border = find_border([&](auto f) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (z[i] > -INFINITY && bin_of(zmax, z[i]) == p.bin) f(at[i], z[i]);
        }, weigh, true, cut, bin_range(zmax, p), sh, 1u).border;
    }
    const float lowest = lowest_of(q, zmax, sh.steps, sh.log_p);
    int n_kept = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const bool kept = inside(border, z[i], at[i]) && z[i] >= lowest;
        w[i] = kept ? w[i] : 0ull;
        n_kept += __popcll(__ballot(kept));
    }
    const u64 upto = wave_incl_scan_u64(w[0] + w[1]);
    if (lane == 63) {
        sh.sum[wave] = upto;
        sh.isum[wave] = n_kept;
    }
    __syncthreads();
    u64 before = 0ull, total = 0ull;
    int all = 0;
#pragma unroll
    for (int v = 0; v < NW; ++v) {
        before += v < wave ? sh.sum[v] : 0ull;
        total += sh.sum[v];
        all += sh.isum[v];
    }
    before += upto - w[0] - w[1];
    const u64 target = target_of(a, r, total);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (before <= target && target < before + w[i])
            give(a, r, at[i], (float)(weigh.real(z[i]) * __hiloint2double((1023 + a.unit) << 20, 0) / (double)total), all);
        before += w[i];
    }
}

// One workgroup, one row.  E entries a thread in registers: group q of four starts at q * 4096 + 4 * thread; E = 0: read again for every look.
template <int E> __device__ __forceinline__ void whole_row(const FilterArgs& a, int r, CutShared& sh, u64* sums, TopList& list) {
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_id();
    const Asked q = asked_of(a, r);
    Source src = source_of(a, r, q);
    float z[E > 0 ? E : 1];
    u64 weights[E > 0 ? E : 1];      // of the row's entries, where they are asked for by top-p
    const int groups = E > 0 ? E / 4 : (a.n + 4 * NT - 1) / (4 * NT);
    auto load = [&]() {
        if constexpr (E > 0) {
#pragma unroll
            for (int g = 0; g < E / 4; ++g) {
                float v[4];
                src.four(g * 4 * NT + 4 * tid, v);
#pragma unroll
                for (int i = 0; i < 4; ++i) z[4 * g + i] = v[i];
            }
        }
    };
    auto each = [&](auto f) {        // f(index, z) of the entries there are
        if constexpr (E > 0) {
            const int th = this_thread();
#pragma unroll
            for (int e = 0; e < E; ++e) {
                float v = z[e];
                asm volatile("" : "+v"(v));      // (or the keys, bins and weights of all entries are kept for the next look: more than there are registers)
                if (v > -INFINITY) f(entry<E>(e, th), v);
            }
        } else {
            for (int g = 0; g < groups; ++g) {
                float v[4];
                const int j = g * 4 * NT + 4 * tid;
                src.four(j, v);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (v[i] > -INFINITY) f(j + i, v[i]);
            }
        }
    };
    __syncthreads();
    load();
    fill_steps(sh.steps);
    fill_log(q, &sh.log_p);
    static_assert(kBinCount == NT && kPartBins <= NT && kFine <= NT, "a thread has a bin");
    sh.count[tid] = 0u;
    sh.mass[tid] = 0ull;
    if (tid < kFine) { sh.fine[tid] = 0u; sh.fine_mass[tid] = 0ull; }

    if (q.greedy) {                  // the largest entry, lowest index first
        u64 best = 0ull;
        each([&](int j, float v) { best = maxu64(best, ((u64)fkey(v) << 32) | (0xFFFFFFFFu - (unsigned)j)); });
        best = max1(best, sh.sum);
        if (tid == 0) best == 0ull ? give(a, r, -1, 0.f, 0) : give(a, r, (int)(0xFFFFFFFFu - (unsigned)best), 1.f, 1);
        return;
    }
    float zmax = -INFINITY;
    each([&](int, float v) { zmax = fmaxf(zmax, v); });
    zmax = wave_max_f(zmax);
    if (lane == 0) sh.fmax[wave] = zmax;
    __syncthreads();
    zmax = sh.fmax[lane & 15];
    ROW_ALLREDUCE(zmax, fmaxf, dpp_f)
    zmax = lane_f(zmax, 0);
    if (zmax == -INFINITY) {
        if (tid == 0) give(a, r, -1, 0.f, 0);
        return;
    }
    if (zmax == INFINITY) {
        src.infinite = true;
        zmax = 0.f;
        load();
    }
    const Weigh weigh = {(double)zmax, magic_of(a.unit), sh.steps};
    if constexpr (E > 0) {
        if (q.by_k && q.k <= (unsigned)kTop) {
            each([&](int, float v) { atomicAdd(&sh.count[bin_of(zmax, v)], 1u); });
            __syncthreads();
            const Cut cut = {1ull << 63, q.k};
            const Picked p = pick_bin<kBinCount>(sh.count, sh.mass, false, cut, 0u, 0ull, sh);
            const Border border = find_border([&](auto f) {
                each([&](int j, float v) {
                    if (bin_of(zmax, v) == p.bin) f(j, v);
                });
            }, weigh, false, cut, bin_range(zmax, p), sh, 1u).border;
            draw_of_list(a, r, q, zmax, weigh, make_list<E>(z, border, list), list, sh);
            return;
        }
    }
    Border border = kNoBorder;
    if (q.by_k || q.by_p) {
        if constexpr (E > 0) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (e % 4 == 0) __builtin_amdgcn_sched_barrier(0);
                weights[e] = 0ull;
                if (z[e] > -INFINITY) {
                    const int b = bin_of(zmax, z[e]);
                    atomicAdd(&sh.count[b], 1u);
                    if (q.by_p) atomicAdd(&sh.mass[b], weights[e] = weigh(z[e]));
                }
            }
        } else {
            each([&](int, float v) {
                const int b = bin_of(zmax, v);
                atomicAdd(&sh.count[b], 1u);
                if (q.by_p) atomicAdd(&sh.mass[b], weigh(v));
            });
        }
        __syncthreads();
        u64 mass = 0ull;
        auto cut_at = [&](const Cut& cut) {
            const Picked p = pick_bin<kBinCount>(sh.count, sh.mass, q.by_p, cut, 0u, 0ull, sh);
            const int b = p.bin;
            const Range range = bin_range(zmax, p);
            auto in_bin = [&](auto f) {
                each([&](int j, float v) {
                    if (bin_of(zmax, v) == b) f(j, v);
                });
            };
            const Found found = find_border(in_bin, weigh, q.by_p, cut, range, sh, E > 0 ? 1u : a.apart);
            border = found.border;
            mass = found.mass;
        };
        if (q.by_k) {
            const Cut cut = {1ull << 63, q.k};
            cut_at(cut);
        } else {
            const u64 own = wave_sum_u64(sh.mass[tid]);
            if (lane == 0) sh.sum[wave] = own;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < NW; ++w) mass += sh.sum[w];
        }
        if (q.by_p) {
            __syncthreads();
            const Cut cut = {maxu64(share_of(q.top_p, mass), 1ull), q.k};   // (the first entry always)
            cut_at(cut);
        }
    }

    const float lowest = lowest_of(q, zmax, sh.steps, sh.log_p);
    int n_kept = 0;
    auto kept = [&](float v, int j) { return inside(border, v, j) && v >= lowest; };
    auto add_group = [&](int g, u64 s) {
        s = wave_sum_u64(s);
        if (lane == 0) sums[g * NW + wave] = s;
    };
    if constexpr (E > 0) {
        if (!q.by_p) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (e % 4 == 0) __builtin_amdgcn_sched_barrier(0);
                weights[e] = kept(z[e], entry<E>(e, tid)) ? weigh(z[e]) : 0ull;
            }
        }
        u64 s[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const bool k = kept(z[e], entry<E>(e, tid));
            weights[e] = k ? weights[e] : 0ull;
            s[e / 4] += weights[e];
            n_kept += k ? 1 : 0;
        }
        if constexpr (E == 16) {
            const u64 v = wave_sums_u64(s[0], s[1], s[2], s[3]);
            if ((lane & 15) == 0) sums[which_of_four(lane) * NW + wave] = v;
        } else {
#pragma unroll
            for (int g = 0; g < E / 4; ++g) add_group(g, s[g]);
        }
    } else {
        for (int g = 0; g < groups; ++g) {
            float v[4];
            u64 s = 0ull;
            const int j = g * 4 * NT + 4 * tid;
            src.four(j, v);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (!kept(v[i], j + i)) continue;
                s += weigh(v[i]);
                ++n_kept;
            }
            add_group(g, s);
        }
    }
    n_kept = wave_sum_i(n_kept);
    if (lane == 0) sh.isum[wave] = n_kept;
    __syncthreads();
    u64 base, target, total;
    int chunk;
    if constexpr (E > 0) {           // up to 64 sums: every wave looks for itself
        const u64 s = lane < groups * NW ? sums[lane] : 0ull, upto = wave_incl_scan_u64(s);
        total = lane_u64(upto, 63);
        target = target_of(a, r, total);
        chunk = __ffsll(__ballot(target < upto)) - 1;
        base = lane_u64(upto - s, chunk);
#pragma unroll
        for (int g = 0; g < E / 4; ++g)
            if (g * NW + wave == chunk) {
                const int j = g * 4 * NT + 4 * tid;
                const float v[4] = {z[4 * g], z[4 * g + 1], z[4 * g + 2], z[4 * g + 3]};
                draw_of_chunk(a, r, j, v, [&](float, int at) { return weights[4 * g + (at - j)]; }, weigh, base, target, total);
            }
    } else {
        chunk = pick_chunk(a, r, sums, groups * NW, sh, base, target, total);
        if (wave == 0) {
            float v[4];
            const int j = chunk * kChunk + 4 * lane;
            src.four(j, v);
            draw_of_chunk(a, r, j, v, [&](float x, int at) { return kept(x, at) ? weigh(x) : 0ull; }, weigh, base, target, total);
        }
    }
    if (tid == 0 && a.out_kept) {
        int all = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) all += sh.isum[w];
        a.out_kept[r] = all;
    }
}

template <int E> __global__ __launch_bounds__(NT) void sample_filtered_kernel(FilterArgs a, int row0) {
    __shared__ CutShared sh;
    __shared__ u64 sums[64];
    __shared__ TopList list;
    const int r = row0 + (int)blockIdx.x;
    if (a.skip && a.skip[r] < 0) {
        if (threadIdx.x == 0) give(a, r, -1, 0.f, 0);
        return;
    }
    whole_row<E>(a, r, sh, sums, list);
}

// ---- Long rows in parts of E * 1024 entries.  Their bins are cells of a fixed grid of z, 512 of them from the cell of the largest entry down (of a
// part, so that a part needs to know nothing of the others; the last one holds what lies behind), and weights are relative to the
// upper end of the largest's cell: parts are brought together by moving bins and scaling masses, in doubles (where a part's largest is in the
// row's cell they are the same whole numbers).  Between the borders' bins sums are whole numbers of the row's unit again.
constexpr int kMostParts = 32, kList = 4096;     // parts of a row; entries of the borders' bins that shared memory holds
__host__ __device__ constexpr int part_list(int E) { return 256 * E; }        // those of a part: a quarter of its entries
constexpr float kCells = 16.f;       // cells of a unit of z
constexpr int kFar = 1 << 29;        // cells from here on are not told apart
__device__ __forceinline__ int cell_of(float z) { return (int)fminf(fmaxf(floorf(z * kCells), -1073741824.f), 1073741824.f); }
__device__ __forceinline__ double ref_of(int top) { return (top + 1) * (double)(1.f / kCells); }

struct PartHead {
    u64 mass, best;                  // of all entries; the largest with the lowest index (greedy rows)
    float zmax;
    int top, valid, n_list, n_kept, pad;
};
struct RowHead {
    u64 total, k_before, p_before;   // of all entries; before the bins that the cuts lie in
    unsigned k_ahead, k_m;
    int k_bin, p_first, p_last, pad;
};
struct RowRoom {
    PartHead* head;
    RowHead* row;
    u64 *mass, *sums;                // [part][bin]; [part][chunk]
    unsigned* count;                 // [part][bin]
    int2* list;                      // [part][part_list]: z, index
};
__host__ __device__ inline size_t part_bytes(int E) { return sizeof(PartHead) + kPartBins * 12 + (size_t)part_list(E) * 8 + (size_t)E * 32; }
__host__ __device__ inline size_t row_bytes(int parts, int E) { return sizeof(RowHead) + parts * part_bytes(E); }
__device__ __forceinline__ RowRoom room_of(const FilterArgs& a, int row, int E) {
    char* p = a.room + row * row_bytes(a.parts, E);
    RowRoom r;
    r.row = reinterpret_cast<RowHead*>(p);
    r.head = reinterpret_cast<PartHead*>(p + sizeof(RowHead));
    r.mass = reinterpret_cast<u64*>(r.head + a.parts);
    r.sums = r.mass + (size_t)a.parts * kPartBins;
    r.list = reinterpret_cast<int2*>(r.sums + (size_t)a.parts * E * 4);
    r.count = reinterpret_cast<unsigned*>(r.list + (size_t)a.parts * part_list(E));
    return r;
}
template <int E> struct PartRow {
    float z[E];
    int j0;
    __device__ __forceinline__ void load(const Source& s, int part) {
        j0 = part * E * NT + 4 * (int)threadIdx.x;
#pragma unroll
        for (int g = 0; g < E / 4; ++g) {
            float v[4];
            s.four(j0 + g * 4 * NT, v);
#pragma unroll
            for (int i = 0; i < 4; ++i) z[4 * g + i] = v[i];
        }
    }
    __device__ __forceinline__ int index(int e) const { return j0 + (e >> 2) * 4 * NT + (e & 3); }
};

template <int E> __global__ __launch_bounds__(NT) void filter_bins_kernel(FilterArgs a, int row0) {
    __shared__ u64 mass[kPartBins], slot[NW];
    __shared__ unsigned count[kPartBins];
    __shared__ double steps[kSteps];
    __shared__ float top[NW];
    const int row = (int)blockIdx.x / a.parts, part = (int)blockIdx.x - row * a.parts, r = row0 + row, tid = threadIdx.x, lane = tid & 63, wave = wave_id();
    if (a.skip && a.skip[r] < 0) return;
    const Asked q = asked_of(a, r);
    const Source src = source_of(a, r, q);
    PartRow<E> p;
    p.load(src, part);
    const RowRoom room = room_of(a, row, E);
    if (q.greedy) {
        u64 best = 0ull;
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (p.z[e] > -INFINITY) best = maxu64(best, ((u64)fkey(p.z[e]) << 32) | (0xFFFFFFFFu - (unsigned)p.index(e)));
        best = max1(best, slot);
        if (tid == 0) room.head[part].best = best;
        return;
    }
    if (tid < kPartBins) {
        mass[tid] = 0ull;
        count[tid] = 0u;
    }
    fill_steps(steps);
    float zmax = -INFINITY;
#pragma unroll
    for (int e = 0; e < E; ++e) zmax = fmaxf(zmax, p.z[e]);
    zmax = wave_max_f(zmax);
    if (lane == 0) top[wave] = zmax;
    __syncthreads();
    zmax = top[lane & 15];
    ROW_ALLREDUCE(zmax, fmaxf, dpp_f)
    zmax = lane_f(zmax, 0);
    const int cell = cell_of(zmax);
    const bool bins = (q.by_k || q.by_p) && cell < kFar && cell > -kFar;
    if (bins) {
        const Weigh weigh = {ref_of(cell), magic_of(a.unit), steps};
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (p.z[e] > -INFINITY) {
                const int b = min(cell - cell_of(p.z[e]), kPartBins - 1);
                if (q.by_k) atomicAdd(&count[b], 1u);
                if (q.by_p) atomicAdd(&mass[b], weigh(p.z[e]));
            }
        __syncthreads();
        const u64 m = tid < kPartBins ? mass[tid] : 0ull;
        const int c = tid < kPartBins ? (int)count[tid] : 0;
        if (tid < kPartBins) {
            if (q.by_p) room.mass[part * kPartBins + tid] = m;
            if (q.by_k) room.count[part * kPartBins + tid] = (unsigned)c;
        }
        const u64 wm = wave_sum_u64(m);
        const int wc = wave_sum_i(c);
        if (lane == 0) { slot[wave] = wm; top[wave] = __int_as_float(wc); }
        __syncthreads();
    }
    if (tid == 0) {
        PartHead h = {};
        if (bins)
            for (int w = 0; w < NW; ++w) {
                h.mass += slot[w];
                h.valid += __float_as_int(top[w]);
            }
        h.zmax = zmax;
        h.top = cell;
        room.head[part] = h;
    }
}

// The largest entry of a row's parts and its cell; whether there is anything to draw, and whether any part's largest entry is off the grid.
struct Top { float zmax; int cell; bool any, far; };
__device__ __forceinline__ Top row_top(const FilterArgs& a, const RowRoom& room) {
    const int lane = threadIdx.x & 63;
    const float z = lane < a.parts ? room.head[lane].zmax : -INFINITY;
    Top t;
    t.zmax = wave_max_f(z);
    t.cell = cell_of(t.zmax);
    t.any = t.zmax > -INFINITY;
    t.far = __ballot(z > -INFINITY && (cell_of(z) >= kFar || cell_of(z) <= -kFar)) != 0ull;
    return t;
}

struct PartShared {
    u64 sums[NW], most_mass;
    double steps[kSteps], log_p, high[kPartBins], low[kPartBins];
    unsigned count[kPartBins];
    int counts[NW], n_list, n_kept;
    RowHead head;
};

template <int E> __global__ __launch_bounds__(NT) void filter_parts_kernel(FilterArgs a, int row0) {
    __shared__ PartShared ps;
    const int row = (int)blockIdx.x / a.parts, part = (int)blockIdx.x - row * a.parts, r = row0 + row, tid = threadIdx.x, lane = tid & 63, wave = wave_id();
    if (a.skip && a.skip[r] < 0) return;
    const Asked q = asked_of(a, r);
    if (q.greedy) return;
    const Source src = source_of(a, r, q);
    PartRow<E> p;
    p.load(src, part);
    const RowRoom room = room_of(a, row, E);
    const Top t = row_top(a, room);
    if (!t.any || t.far) return;
    const int top = t.cell;
    fill_steps(ps.steps);
    fill_log(q, &ps.log_p);
    const Weigh weigh = {ref_of(top), magic_of(a.unit), ps.steps};
    if (tid == 0) { ps.n_list = 0; ps.n_kept = 0; ps.head = RowHead{}; ps.head.k_bin = ps.head.p_first = kPartBins; ps.head.p_last = kPartBins - 1; }
    __syncthreads();
    if (q.by_k || q.by_p) {
        // lane i: how far part i's bins are moved, and what its masses are multiplied by
        int down = kFar, valid = 0;
        double scale = 0.0;
        u64 mass = 0ull;
        if (lane < a.parts) {
            const PartHead h = room.head[lane];
            if (h.zmax > -INFINITY) {
                down = top - h.top;
                scale = down == 0 ? 1.0 : exp_below(-(double)down * (double)(1.f / kCells), ps.steps);
                valid = h.valid;
                mass = down == 0 ? h.mass : (u64)((double)h.mass * scale);
            }
        }
        const unsigned all = (unsigned)wave_sum_i(valid);
        const u64 total = wave_sum_u64(mass);
        // Two threads a bin, each with every second part, four parts' bins requested at a time.  The halves of a mass are scaled and added as doubles,
        // whole numbers where parts are not moved: a third of the instructions of a whole mass, there and back for every part.
        static_assert(NT == 2 * kPartBins, "two threads a bin");
        const int half = wave >> 3, bin = tid & (kPartBins - 1);
        unsigned c = 0u;
        u64 m = 0ull;
        double high = 0.0, low = 0.0;
        for (int i0 = half; i0 < a.parts; i0 += 8) {
            unsigned cs[4];
            u64 ms[4];
            bool there[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int i = min(i0 + 2 * j, a.parts - 1), from = bin - __builtin_amdgcn_readlane(down, i), at = i * kPartBins + max(from, 0);
                there[j] = i0 + 2 * j < a.parts && from >= 0;
                cs[j] = q.by_k ? room.count[at] : 0u;
                ms[j] = q.by_p ? room.mass[at] : 0ull;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const double f = there[j] ? lane_d(scale, min(i0 + 2 * j, a.parts - 1)) : 0.0;
                c += there[j] ? cs[j] : 0u;
                high = fma((double)(unsigned)(ms[j] >> 32), f, high);
                low = fma((double)(unsigned)ms[j], f, low);
            }
        }
        if (half == 1) {
            ps.high[bin] = high;
            ps.low[bin] = low;
            ps.count[bin] = c;
        }
        __syncthreads();
        if (half == 0) {
            high += ps.high[bin];
            low += ps.low[bin];
            c += ps.count[bin];
            const double whole = floor(high);
            m = ((u64)whole << 32) + (u64)fma(high - whole, 0x1p32, low);
            if (!q.by_k) c = m > 0ull ? 1u : 0u;     // (entries are not counted then: a border by mass is in a bin that has some)
        } else {
            c = 0u;
        }
        Bin b = scan_bins(c, m, q.by_p, ps.counts, ps.sums);
        b.all = q.by_k ? all : 0xFFFFFFFFu;
        if (tid == kPartBins - 1) {
            b.mass = total > b.before ? total - b.before : 0ull;
            b.m = q.by_k ? all - b.ahead : (b.mass > 0ull ? 1u : 0u);
        } else if (tid >= kPartBins) {
            b.m = 0u;
        }
        u64 least_mass = total, most_mass = total;       // that a top-k keeps
        const Cut by_k = {1ull << 63, q.k};
        if (tid == 0) ps.head.total = total;
        if (q.by_k) {
            if (holds(b, by_k)) {
                ps.head.k_bin = tid;
                ps.head.k_m = b.m;
                ps.head.k_ahead = b.ahead;
                ps.head.k_before = b.before;
                ps.most_mass = b.before + b.mass;
            }
            __syncthreads();
            least_mass = ps.head.k_before;
            most_mass = ps.most_mass;
        }
        if (q.by_p) {
            // The cut's mass is `first` at least and, by the parts' sums, `last` at most.  The border is looked for with weights relative to the row's
            // maximum, each rounded to a unit, a part's own to a smaller one: sums of the same entries differ by a unit an entry at most, by one a
            // bin and part where scaled masses are rounded down, and by 2^-46 of the whole (exponentials are off by 2^-51, the sum of 32 products by
            // 2^-48).  That twice: for the cut's mass and for the sum that has to reach it.  A wider bracket lists a few more entries.
            const u64 first = share_of(q.top_p, least_mass), last = share_of(q.top_p, most_mass), off = (u64)a.n + kPartBins + kMostParts + (total >> 46);
            const Cut c0 = {maxu64(first, 1ull), q.k}, c1 = {last + 2ull * off + 1ull, q.k};
            if (holds(b, c0)) {
                ps.head.p_first = tid;
                ps.head.p_before = b.before;
            }
            if (holds(b, c1)) ps.head.p_last = tid;
        }
        __syncthreads();
        if (part == 0 && tid == 0) *room.row = ps.head;
    }
    const RowHead h = ps.head;
    const int sure = q.by_p ? h.p_first : (q.by_k ? h.k_bin : kPartBins);    // bins before this one are kept, but for min-p
    const float lowest = lowest_of(q, t.zmax, ps.steps, ps.log_p);
    int n_kept = 0;
    u64 sums[4];
#pragma unroll
    for (int g = 0; g < E / 4; ++g) {
        u64& s = sums[g & 3];
        s = 0ull;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float z = p.z[4 * g + i];
            if (!(z > -INFINITY)) continue;
            const int b = min(top - cell_of(z), kPartBins - 1);
            if (b < sure) {
                if (z >= lowest) {
                    s += weigh(z);
                    ++n_kept;
                }
            } else if ((q.by_k && b == h.k_bin) || (q.by_p && b <= h.p_last)) {
                const int at = atomicAdd(&ps.n_list, 1);
                if (at < part_list(E)) room.list[part * part_list(E) + at] = make_int2(__float_as_int(z), p.index(4 * g + i));
            }
        }
        if constexpr (E == 8) {
            s = wave_sum_u64(s);
            if (lane == 0) room.sums[(part * (E / 4) + g) * NW + wave] = s;
        } else if ((g & 3) == 3) {
            const u64 v = wave_sums_u64(sums[0], sums[1], sums[2], sums[3]);
            if ((lane & 15) == 0) room.sums[(part * (E / 4) + g - 3 + which_of_four(lane)) * NW + wave] = v;
        }
    }
    n_kept = wave_sum_i(n_kept);
    if (lane == 0) atomicAdd(&ps.n_kept, n_kept);
    __syncthreads();
    if (tid == 0) {
        room.head[part].n_list = ps.n_list;
        room.head[part].n_kept = ps.n_kept;
    }
}

struct ListShared {
    float z[kList];
    int at[kList], kept, m;
};

template <int E> __global__ __launch_bounds__(NT) void filter_draw_kernel(FilterArgs a, int row0) {
    __shared__ CutShared sh;
    __shared__ union { ListShared list; TopList top; } both;     // (a row that is read again needs no list)
    __shared__ u64 sums[kChunks];
    ListShared& ls = both.list;
    const int row = blockIdx.x, r = row0 + row, tid = threadIdx.x, lane = tid & 63, wave = wave_id();
    if (a.skip && a.skip[r] < 0) {
        if (tid == 0) give(a, r, -1, 0.f, 0);
        return;
    }
    const Asked q = asked_of(a, r);
    const RowRoom room = room_of(a, row, E);
    if (q.greedy) {
        u64 best = max1(tid < a.parts ? room.head[tid].best : 0ull, sh.sum);
        if (tid == 0) best == 0ull ? give(a, r, -1, 0.f, 0) : give(a, r, (int)(0xFFFFFFFFu - (unsigned)best), 1.f, 1);
        return;
    }
    const Top t = row_top(a, room);
    if (!t.any) {
        if (tid == 0) give(a, r, -1, 0.f, 0);
        return;
    }
    const int top = t.cell;
    if (t.far) {
        whole_row<0>(a, r, sh, sums, both.top);
        return;
    }
    const Source src = source_of(a, r, q);
    const int listed = lane < a.parts ? room.head[lane].n_list : 0, sure = lane < a.parts ? room.head[lane].n_kept : 0;
    const int upto = wave_incl_scan_i(listed), n_list = __builtin_amdgcn_readlane(upto, 63);
    const bool cut_short = __ballot(listed > part_list(E)) != 0ull;      // some are only in the row itself
    const int n_sure = wave_sum_i(sure);
    if (tid == 0) { ls.kept = n_sure; ls.m = 0; sh.n = 0; }
    fill_steps(sh.steps);
    fill_log(q, &sh.log_p);
    if (tid < kFine) { sh.fine[tid] = 0u; sh.fine_mass[tid] = 0ull; }
    const int chunks = a.parts * E * 4;
    for (int i = tid; i < chunks; i += NT) sums[i] = room.sums[i];
    const bool held = n_list <= kList && !cut_short;
    for (int i = wave; held && i < a.parts; i += NW) {
        const int n = __builtin_amdgcn_readlane(listed, i), from = __builtin_amdgcn_readlane(upto, i) - n;
        for (int k = lane; k < n; k += 64) {
            const int2 e = room.list[i * part_list(E) + k];
            ls.z[from + k] = __int_as_float(e.x);
            ls.at[from + k] = e.y;
        }
    }
    auto each_listed = [&](auto f) {     // f(index, z)
        if (held) {
            for (int i = tid; i < n_list; i += NT) f(ls.at[i], ls.z[i]);
        } else if (cut_short) {
            for (int j = 4 * tid; j < a.n; j += 4 * NT) {
                float v[4];
                src.four(j, v);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (v[i] > -INFINITY) f(j + i, v[i]);
            }
        } else {
            for (int i0 = 0; i0 < a.parts; i0 += 4) {            // four loads on their way together
                int n[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) n[i] = i0 + i < a.parts ? __builtin_amdgcn_readlane(listed, min(i0 + i, a.parts - 1)) : 0;
                const int most = max(max(n[0], n[1]), max(n[2], n[3]));
                for (int k = tid; k < most; k += NT) {
                    int2 e[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) e[i] = k < n[i] ? room.list[(i0 + i) * part_list(E) + k] : make_int2(0, 0);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (k < n[i]) f(e[i].y, __int_as_float(e[i].x));
                }
            }
        }
    };
    __syncthreads();
    const Weigh weigh = {ref_of(top), magic_of(a.unit), sh.steps};
    const float lowest = lowest_of(q, t.zmax, sh.steps, sh.log_p);
    Border border = kNoBorder;
    if (q.by_k || q.by_p) {
        const RowHead h = *room.row;
        auto bin = [&](float z) { return min(top - cell_of(z), kPartBins - 1); };
        auto range_of = [&](int first, int last) {       // of the keys of bins first .. last
            Range x = {};
            x.hi = fkey((float)ref_of(top - first)) + 1u;
            x.lo = last == kPartBins - 1 ? 0u : fkey((float)ref_of(top - last - 1)) - 1u;
            x.last = kMostEntries - 1;
            return x;
        };
        u64 mass = h.total;
        if (q.by_k) {
            const Cut cut = {1ull << 63, q.k};
            Range x = range_of(h.k_bin, h.k_bin);
            x.before = h.k_before; x.ahead = h.k_ahead; x.m = h.k_m;
            const Found f = find_border([&](auto f) {
                each_listed([&](int at, float z) {
                    if (bin(z) == h.k_bin) f(at, z);
                });
            }, weigh, q.by_p, cut, x, sh, a.apart);
            border = f.border;
            mass = f.mass;
            __syncthreads();
        }
        if (q.by_p) {
            const Border most = border;
            auto in = [&](int at, float z) {
                const int b = bin(z);
                return b >= h.p_first && b <= h.p_last && inside(most, z, at);
            };
            int m = n_list;          // (those before its bins are not listed, those behind neither, but for a top-k's bin)
            if (q.by_k) {
                m = 0;
                each_listed([&](int at, float z) { m += in(at, z) ? 1 : 0; });
                m = wave_sum_i(m);
                if (lane == 0) atomicAdd(&ls.m, m);
                if (tid == 0) sh.n = 0;
                __syncthreads();
                m = ls.m;
            }
            const Cut cut = {maxu64(share_of(q.top_p, mass), 1ull), 0xFFFFFFFFu};
            Range x = range_of(h.p_first, h.p_last);
            x.before = h.p_before; x.m = (unsigned)m;
            border = find_border([&](auto f) {
                each_listed([&](int at, float z) {
                    if (in(at, z)) f(at, z);
                });
            }, weigh, true, cut, x, sh, a.apart).border;
        }
        int n = 0;
        const int first = q.by_p ? h.p_first : h.k_bin;          // entries of bins before it are among the sums
        each_listed([&](int at, float z) {
            if (!inside(border, z, at) || z < lowest || (cut_short && bin(z) < first)) return;
            atomicAdd(&sums[at / kChunk], weigh(z));
            ++n;
        });
        n = wave_sum_i(n);
        if (lane == 0) atomicAdd(&ls.kept, n);
        __syncthreads();
    }
    u64 base, target, total;
    const int chunk = pick_chunk(a, r, sums, chunks, sh, base, target, total);
    if (wave == 0) {
        float v[4];
        const int j = chunk * kChunk + 4 * lane;
        src.four(j, v);
        draw_of_chunk(a, r, j, v, [&](float x, int at) { return inside(border, x, at) && x >= lowest ? weigh(x) : 0ull; }, weigh, base, target, total);
    }
    if (tid == 0 && a.out_kept) a.out_kept[r] = ls.kept;
}

// Rows in parts, as many at a time as kPartsAtOnce parts (so that the workspace does not grow with the rows).  Parts as small as keep them one to a
// unit: a larger part takes its unit longer, more parts than units take turns (us with 8 / 16 / 32 entries a thread: 16 rows of 65536,
// 128 / 64 / 32 parts, 29.5 / 34.4 / 46.1; 48 of them, 384 / 192 / 96, 39.3 / 36.0 / 46.4; 512 of them 195 / 178 / 158; 2 of 200003 33.1 / 39.7 / 56.5; 32 of
// them, 800 / 416 / 224, 73.6 / 67.3 / 61.7).
// 2048 parts of 72 KB are 150 MB.
constexpr int kPartsAtOnce = 2048;
struct Cutting { int E, parts, rows; };          // entries of a thread (0: rows are not cut), parts of a row, rows at a time
inline Cutting cutting_of(int rows, int n) {
    Cutting c = {0, 1, rows};
    if (n <= 16 * NT) return c;
    c.E = 8;
    auto parts = [&](int E) { return (n + E * NT - 1) / (E * NT); };
    while (c.E < 32 && (parts(c.E) > kMostParts || (int64_t)rows * parts(c.E) > 256)) c.E *= 2;
    c.parts = parts(c.E);
    c.rows = std::min(rows, kPartsAtOnce / c.parts);
    return c;
}
template <int E> void launch_rows(const FilterArgs& a, int rows, hipStream_t stream) {
    constexpr int kMost = 1 << 21;               // a launch has fewer than 2^32 threads
    for (int r = 0; r < rows; r += kMost) sample_filtered_kernel<E><<<(unsigned)std::min(kMost, rows - r), NT, 0, stream>>>(a, r);
}
template <int E> void launch_parts(FilterArgs a, const Cutting& c, int rows, hipStream_t stream) {
    for (int r = 0; r < rows; r += c.rows) {
        const int n = std::min(c.rows, rows - r);
        filter_bins_kernel<E><<<(unsigned)(n * c.parts), NT, 0, stream>>>(a, r);
        filter_parts_kernel<E><<<(unsigned)(n * c.parts), NT, 0, stream>>>(a, r);
        filter_draw_kernel<E><<<(unsigned)n, NT, 0, stream>>>(a, r);
    }
}

int status() { return hipGetLastError() == hipSuccess ? HAWK_OK : HAWK_EDEVICE; }

}  // namespace

size_t sample_filtered_workspace_bytes(int rows, int n) {
    if (rows < 1 || rows > (1 << 22) || n < 1 || n > kMostEntries) return 0;
    const Cutting c = cutting_of(rows, n);
    return c.E ? c.rows * row_bytes(c.parts, c.E) : 0;
}

int launch_sample_filtered(const void* logits, int dtype, int64_t row_stride, const int32_t* skip, const float* u, const float* temperature,
                           const int32_t* top_k, const float* top_p, const float* min_p, int rows, int n, int32_t* out_token, float* out_prob,
                           int32_t* out_kept, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!is_type(dtype) || rows < 0 || rows > (1 << 22) || n < 1 || n > kMostEntries || row_stride < n) return HAWK_EINVAL;
    if (rows == 0) return HAWK_OK;
    if (!logits || !u || !out_token || (reinterpret_cast<uintptr_t>(logits) & (type_bytes(dtype) - 1))) return HAWK_EINVAL;
    const Cutting c = cutting_of(rows, n);
    if (c.E && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15))) return HAWK_EINVAL;
    if (c.E && workspace_bytes < c.rows * row_bytes(c.parts, c.E)) return HAWK_ENOMEM;
    FilterArgs a = {};
    a.parts = c.parts; a.room = static_cast<char*>(workspace);
    a.logits = static_cast<const char*>(logits); a.row_stride = row_stride; a.dtype = dtype; a.n = n;
    a.skip = skip; a.u = u; a.temperature = temperature; a.top_k = top_k; a.top_p = top_p; a.min_p = min_p;
    a.out_token = out_token; a.out_prob = out_prob; a.out_kept = out_kept;
    int log = 0;
    while ((1 << log) < n) ++log;
    a.unit = std::min(51, 62 - log);
    // neighbours of 8 (11) bits are 2^15 (2^12) steps of 24 bits apart at least, times any number; each product is rounded by half a step
    a.apart = dtype == HAWK_BF16 ? (1u << 15) - 1u : (dtype == HAWK_FP16 ? (1u << 12) - 1u : 1u);
    if (n <= 4 * NT) launch_rows<4>(a, rows, stream);
    else if (n <= 8 * NT) launch_rows<8>(a, rows, stream);
    else if (n <= 16 * NT) launch_rows<16>(a, rows, stream);
    else if (c.E == 8) launch_parts<8>(a, c, rows, stream);
    else if (c.E == 16) launch_parts<16>(a, c, rows, stream);
    else launch_parts<32>(a, c, rows, stream);
    return status();
}

}  // namespace hawk
