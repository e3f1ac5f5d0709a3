// One draw a row from logits cut by top-k, top-p and min-p, each row with parameters of its own.
//
// z = l / T in 32 bits, w = exp(z - zmax).  Entries are ordered by z, equal ones by index; what is kept is a beginning of that order: the
// top_k first, of these the ones before which less than top_p of their mass lies, of these the ones with w >= min_p.  The token is the first
// in ascending index whose sum of kept weights exceeds u times the whole.
//
// Weights are whole multiples of 2^-S of the largest (S as large as n of them still sum up in 64 bits: 48 for 16384 entries),
// rounded to nearest, so that a sum has one value whatever the order it is made in, and masses can be counted in bins by atomics.  What
// that rounding moves is n 2^-(S + 1) of the largest weight at most, 2^-35 for 16384 entries; sums of random errors are a hundredth of it.
//
// A workgroup of 1024 threads has a row, in registers up to 65536 entries, read again for every look at a longer one.  The border of a cut is
// found by linear bins of z below the maximum; the entries of the border's bin are ranked against each other.  Bins of too many entries (ties,
// far tails) are searched by the bits of z instead.
#include "filtered.h"
#include "paged.h"
#include "sample_rows.h"

#include <algorithm>

// z is a rounded product wherever it is compared, binned or subtracted from the maximum.
#pragma clang fp contract(off)

namespace hawk {

namespace {

typedef unsigned long long u64;

constexpr int kCutBins = 2048;
constexpr float kCutReach = 32.f;       // bins reach so far below the maximum; what lies behind shares the last one
constexpr int kList = 2048;          // entries of a border's bin that are ranked

struct FilterArgs {
    const char* logits;
    int64_t row_stride;              // elements
    const int32_t *skip, *top_k;
    const float *u, *temperature, *top_p, *min_p;
    int dtype, n, unit;              // unit: S
    int32_t *out_token, *out_kept;
    float* out_prob;
};

struct FilterShared {
    u64 mass[kCutBins], list_mass[kList];
    unsigned count[kCutBins], list_key[kList], ranked_key[kList];
    int list_at[kList], ranked_at[kList];
    double steps[kSteps];
    u64 sum[NW];
    int isum[NW];
    float fmax[NW];
    u64 b_mass;                      // broadcasts
    unsigned b_key;
    int b_bin, b_count, b_at, n;
};

__device__ __forceinline__ u64 block_sum(u64 v, u64 (&slot)[NW]) {   // ends with a barrier
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
    __syncthreads();
    u64 s = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) s += slot[w];
    __syncthreads();
    return s;
}
template <class V> __device__ __forceinline__ V block_before(V v, V (&slot)[NW], V& all) {   // exclusive prefix; ends with a barrier
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    V x = v;
    for (int d = 1; d < 64; d <<= 1) {
        const V y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    if (lane == 63) slot[wave] = x;
    __syncthreads();
    V before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        const V s = slot[w];
        before += w < wave ? s : 0;
        all += s;
    }
    __syncthreads();
    return before + x - v;
}

// A row: groups of four neighbouring entries, group q of a thread starts at q * 4096 + 4 * thread.  Values are z, minus infinity where there is
// nothing to draw (past the end, NaN).
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
template <int E> struct Row {
    float z[E > 0 ? E : 1];
    Source s;
    __device__ __forceinline__ void load() {
        if (E > 0) {
#pragma unroll
            for (int q = 0; q < E / 4; ++q) {
                float v[4];
                s.four(q * 4 * NT + 4 * (int)threadIdx.x, v);
#pragma unroll
                for (int i = 0; i < 4; ++i) z[4 * q + i] = v[i];
            }
        }
    }
    __device__ __forceinline__ int groups() const { return E > 0 ? E / 4 : (s.n + 4 * NT - 1) / (4 * NT); }
    template <class F> __device__ __forceinline__ void each_group(F f) const {   // f(group, first index, four values)
        if (E > 0) {
#pragma unroll
            for (int q = 0; q < E / 4; ++q) {
                const float v[4] = {z[4 * q], z[4 * q + 1], z[4 * q + 2], z[4 * q + 3]};
                f(q, q * 4 * NT + 4 * (int)threadIdx.x, v);
            }
        } else {
            for (int q = 0; q < groups(); ++q) {
                float v[4];
                s.four(q * 4 * NT + 4 * (int)threadIdx.x, v);
                f(q, q * 4 * NT + 4 * (int)threadIdx.x, v);
            }
        }
    }
    template <class F> __device__ __forceinline__ void each(F f) const {         // f(index, z) of the entries there are
        each_group([&](int, int j, const float (&v)[4]) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (v[i] > -INFINITY) f(j + i, v[i]);
        });
    }
};

__device__ __forceinline__ int bin_of(float zmax, float z) { return (int)fminf((zmax - z) * (kCutBins / kCutReach), (float)(kCutBins - 1)); }

// Entries are kept if z is above the border's key, or equal and not behind index `at`.
struct Border { unsigned key; int at; };
__device__ __forceinline__ bool inside(const Border& b, float z, int j) {
    const unsigned k = fkey(z);
    return k > b.key || (k == b.key && j <= b.at);
}

// What a cut looks for: the first entry, in order, before which there are K entries or a mass of M.  (The other one is then never reached.)
struct Cut { u64 M; unsigned K; };

// The border of a cut: the last entry before it; mass: of all entries up to it.  Every thread has the result.
template <int E> __device__ Border find_border(const Row<E>& row, float zmax, const Cut& cut, int unit, FilterShared& sh, u64& mass) {
    const int tid = threadIdx.x;
    auto weight = [&](float z) { return (u64)__double_as_longlong(exp_below((double)z - (double)zmax, sh.steps) + __hiloint2double((1075 - unit) << 20, 0)) & 0xFFFFFFFFFFFFFull; };
    // the bin in which the cut lies
    {
        u64 m0 = sh.mass[2 * tid], m1 = sh.mass[2 * tid + 1], all_m;
        int c0 = (int)sh.count[2 * tid], c1 = (int)sh.count[2 * tid + 1], all_c;
        const u64 bm = block_before(m0 + m1, sh.sum, all_m);
        const int bc = block_before(c0 + c1, sh.isum, all_c);
        // the last bin that begins before the cut and is not empty
        const bool in0 = c0 > 0 && bm < cut.M && (unsigned)bc < cut.K, in1 = c1 > 0 && bm + m0 < cut.M && (unsigned)(bc + c0) < cut.K;
        if (tid == 0) sh.n = 0;
        if (in1 || in0) atomicMax(&sh.b_bin, in1 ? 2 * tid + 1 : 2 * tid);
        __syncthreads();
        const int b = sh.b_bin;
        if (b >> 1 == tid) {
            sh.b_mass = (b & 1) ? bm + m0 : bm;
            sh.b_count = (b & 1) ? bc + c0 : bc;
        }
        __syncthreads();
    }
    const int bin = sh.b_bin, m = (int)sh.count[bin];
    u64 before = sh.b_mass;
    unsigned ahead = (unsigned)sh.b_count;
    Border out;
    if (m <= kList) {
        row.each([&](int j, float z) {
            if (bin_of(zmax, z) == bin) {
                const int i = atomicAdd(&sh.n, 1);
                sh.list_key[i] = fkey(z);
                sh.list_at[i] = j;
            }
        });
        __syncthreads();
        for (int i = tid; i < m; i += NT) {
            const unsigned k = sh.list_key[i];
            const int at = sh.list_at[i];
            int r = 0;
            for (int x = 0; x < m; ++x) {
                const unsigned other = sh.list_key[x];
                r += other > k || (other == k && sh.list_at[x] < at) ? 1 : 0;
            }
            sh.ranked_key[r] = k;
            sh.ranked_at[r] = at;
        }
        __syncthreads();
        // two ranks a thread: sums of the masses before
        u64 w[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) w[i] = 2 * tid + i < m ? weight(key_to_float(sh.ranked_key[2 * tid + i])) : 0;
        u64 all, bm = before + block_before(w[0] + w[1], sh.sum, all);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = 2 * tid + i;
            if (r < m && bm < cut.M && ahead + r < cut.K) atomicMax(&sh.b_at, r);   // the last one inside
            bm += w[i];
            if (r < m) sh.list_mass[r] = bm;
        }
        __syncthreads();
        const int last = sh.b_at;
        out.key = sh.ranked_key[last];
        out.at = sh.ranked_at[last];
        mass = sh.list_mass[last];
        __syncthreads();
        return out;
    }
    // by the key's bits, eight at a time: the key of the last entry inside, and how many of the entries that have it are
    unsigned prefix = 0u, mask = 0u;
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        if (tid < 256) { sh.list_key[tid] = 0u; sh.list_mass[tid] = 0ull; }
        if (tid == 0) sh.b_at = -1;
        __syncthreads();
        row.each([&](int, float z) {
            const unsigned k = fkey(z);
            if (bin_of(zmax, z) == bin && (k & mask) == prefix) {
                atomicAdd(&sh.list_key[(k >> shift) & 255u], 1u);
                atomicAdd(&sh.list_mass[(k >> shift) & 255u], weight(z));
            }
        });
        __syncthreads();
        // descending: thread t has digit 255 - t
        const int c = tid < 256 ? (int)sh.list_key[255 - tid] : 0;
        const u64 w = tid < 256 ? sh.list_mass[255 - tid] : 0ull;
        int all_c;
        u64 all_w;
        const int bc = block_before(c, sh.isum, all_c);
        const u64 bw = block_before(w, sh.sum, all_w);
        if (c > 0 && before + bw < cut.M && ahead + (unsigned)bc < cut.K) atomicMax(&sh.b_at, tid);
        __syncthreads();
        const int t = sh.b_at;
        if (tid == t) { sh.b_mass = before + bw; sh.b_count = (int)ahead + bc; }
        __syncthreads();
        before = sh.b_mass;
        ahead = (unsigned)sh.b_count;
        prefix |= (unsigned)(255 - t) << shift;
        mask |= 255u << shift;
        if (shift == 0 && tid == 0) sh.n = (int)sh.list_key[255 - t];
    }
    __syncthreads();
    // of the equal ones entry i (from 0) is inside if before + i w < M and ahead + i < K
    const int equal = sh.n;
    const u64 w = weight(key_to_float(prefix));
    u64 c = min((u64)equal, (u64)(cut.K - ahead));
    if (w > 0) c = min(c, (cut.M - before + w - 1) / w);
    mass = before + c * w;
    int seen = 0;
    out.key = prefix;
    out.at = 0x7FFFFFFF;
    __syncthreads();
    if (tid == 0) sh.b_at = -1;
    row.each_group([&](int, int j, const float (&v)[4]) {
        int own = 0, all;
#pragma unroll
        for (int i = 0; i < 4; ++i) own += v[i] > -INFINITY && fkey(v[i]) == prefix ? 1 : 0;
        int k = seen + block_before(own, sh.isum, all);
        seen += all;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (v[i] > -INFINITY && fkey(v[i]) == prefix && (u64)++k == c) sh.b_at = j + i;
    });
    __syncthreads();
    out.at = sh.b_at;
    __syncthreads();
    return out;
}

template <int E>
__global__ __launch_bounds__(NT) void sample_filtered_kernel(FilterArgs a) {
    __shared__ FilterShared sh;
    const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    auto give = [&](int token, double prob, int kept) {
        if (tid == 0) {
            a.out_token[r] = token;
            if (a.out_prob) a.out_prob[r] = (float)prob;
            if (a.out_kept) a.out_kept[r] = kept;
        }
    };
    if (a.skip && a.skip[r] < 0) { give(-1, 0.0, 0); return; }
    const float T = a.temperature ? a.temperature[r] : 1.f;
    const bool greedy = !(T > 0.f);
    Row<E> row;
    row.s.dtype = a.dtype;
    row.s.n = a.n;
    const int es = a.dtype == HAWK_FP32 ? 4 : 2;
    row.s.l = a.logits + r * a.row_stride * es;
    row.s.fours = (reinterpret_cast<uintptr_t>(row.s.l) & (4 * es - 1)) == 0;
    row.s.inv_t = greedy ? 1.f : (float)(1.0 / (double)T);
    row.s.infinite = false;
    fill_steps(sh.steps);
    for (int i = tid; i < kCutBins; i += NT) { sh.count[i] = 0u; sh.mass[i] = 0ull; }
    if (tid == 0) { sh.b_bin = -1; sh.b_at = -1; sh.n = 0; }
    row.load();

    // the largest entry, lowest index first
    u64 best = 0ull;
    row.each([&](int j, float z) { best = maxu64(best, ((u64)fkey(z) << 32) | (0xFFFFFFFFu - (unsigned)j)); });
    for (int d = 1; d < 64; d <<= 1) best = maxu64(best, __shfl_xor(best, d));
    if (lane == 0) sh.sum[wave] = best;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) best = maxu64(best, sh.sum[w]);
    __syncthreads();
    if (best == 0ull) { give(-1, 0.0, 0); return; }
    float zmax = key_to_float((unsigned)(best >> 32));
    if (greedy) { give((int)(0xFFFFFFFFu - (unsigned)best), 1.0, 1); return; }
    if (zmax == INFINITY) {
        row.s.infinite = true;
        zmax = 0.f;
        row.load();
    }
    const int unit = a.unit;
    const double magic = __hiloint2double((1075 - unit) << 20, 0);   // 2^(52 - S): a sum with it has round(w 2^S) in its last 52 bits
    auto exact_weight = [&](float z) { return exp_below((double)z - (double)zmax, sh.steps); };
    auto whole = [&](double w) { return (u64)__double_as_longlong(w + magic) & 0xFFFFFFFFFFFFFull; };

    const int want = a.top_k ? a.top_k[r] : 0;
    const float top_p = a.top_p ? a.top_p[r] : 1.f, asked = a.min_p ? a.min_p[r] : 0.f, min_p = asked > 1.f ? 1.f : asked;   // (NaN: none)
    const bool by_k = want >= 1 && want < a.n, by_p = top_p < 1.f, by_m = min_p > 0.f;
    Border border = {0u, 0x7FFFFFFF};
    if (by_k || by_p) {
        row.each([&](int, float z) {
            const int b = bin_of(zmax, z);
            atomicAdd(&sh.count[b], 1u);
            if (by_p) atomicAdd(&sh.mass[b], whole(exact_weight(z)));
        });
        __syncthreads();
        u64 mass = 0ull;
        if (by_k) {
            const Cut cut = {1ull << 63, (unsigned)want};
            border = find_border<E>(row, zmax, cut, unit, sh, mass);
        } else {
            mass = block_sum(sh.mass[2 * tid] + sh.mass[2 * tid + 1], sh.sum);
        }
        if (by_p) {
            if (tid == 0) { sh.b_bin = -1; sh.b_at = -1; }
            __syncthreads();
            // an entry is inside if the mass before it is below top_p times the whole: of whole numbers, below that rounded up
            const Cut cut = {max((u64)ceil(fmax((double)top_p * (double)mass, 0.0)), 1ull), by_k ? (unsigned)want : 0xFFFFFFFFu};
            border = find_border<E>(row, zmax, cut, unit, sh, mass);
        }
    }

    // sums of the kept weights: of the four entries a thread has in a group, of a wave's 256, of all of them in index order
    auto kept = [&](float z, int j, double& w) {
        if (!(z > -INFINITY) || !inside(border, z, j)) return false;
        w = exact_weight(z);
        return !(by_m && w < (double)min_p);
    };
    const int groups = row.groups();
    u64* sums = sh.mass;             // [group][wave]: of up to 128 groups; further ones join the last
    int n_kept = 0;
    for (int i = tid; i < kCutBins; i += NT) sums[i] = 0ull;
    __syncthreads();
    constexpr int kGroups = kCutBins / NW;
    const int fold = (groups + kGroups - 1) / kGroups;               // groups that share a sum
    row.each_group([&](int q, int j, const float (&v)[4]) {
        u64 s = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            double w;
            if (kept(v[i], j + i, w)) {
                s += whole(w);
                ++n_kept;
            }
        }
        for (int d = 1; d < 64; d <<= 1) s += __shfl_xor(s, d);
        if (lane == 0) atomicAdd(&sums[fold == 1 ? q * NW + wave : q / fold * NW], s);
    });
    __syncthreads();
    u64 total;
    const u64 m0 = sums[2 * tid], m1 = sums[2 * tid + 1];
    const u64 before = block_before(m0 + m1, sh.sum, total);
    int all;
    (void)block_before(n_kept, sh.isum, all);
    const u64 target = min((u64)(fmax((double)a.u[r], 0.0) * (double)total), total - 1);   // the first sum above it
    if (before <= target && target < before + m0 + m1) {
        const bool second = target >= before + m0;
        sh.b_bin = 2 * tid + (second ? 1 : 0);
        sh.b_mass = second ? before + m0 : before;
    }
    __syncthreads();
    const int where = sh.b_bin;
    u64 base = sh.b_mass;
    row.each_group([&](int q, int j, const float (&v)[4]) {
        if (fold == 1) {
            if (q * NW + wave != where) return;                      // one wave's 256 entries of one group
        } else if (q / fold * NW != where) return;                   // the groups of one sum
        u64 w[4], s = 0;
        double x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = 0.0;
            w[i] = kept(v[i], j + i, x[i]) ? whole(x[i]) : 0;
            s += w[i];
        }
        u64 at, sum = 0;
        if (fold == 1) {
            u64 y = s;
            for (int d = 1; d < 64; d <<= 1) {
                const u64 o = __shfl_up(y, d);
                if (lane >= d) y += o;
            }
            at = base + y - s;
        } else {
            at = base + block_before(s, sh.sum, sum);
            base += sum;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (at <= target && target < at + w[i]) {
                a.out_token[r] = j + i;
                if (a.out_prob) a.out_prob[r] = (float)(x[i] * __hiloint2double((1023 + unit) << 20, 0) / (double)total);
            }
            at += w[i];
        }
    });
    if (tid == 0 && a.out_kept) a.out_kept[r] = all;
}

int status() { return hipGetLastError() == hipSuccess ? HAWK_OK : HAWK_EDEVICE; }

}  // namespace

size_t sample_filtered_workspace_bytes(int rows, int n) {
    (void)rows; (void)n;
    return 0;
}

int launch_sample_filtered(const void* logits, int dtype, int64_t row_stride, const int32_t* skip, const float* u, const float* temperature,
                           const int32_t* top_k, const float* top_p, const float* min_p, int rows, int n, int32_t* out_token, float* out_prob,
                           int32_t* out_kept, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    (void)workspace; (void)workspace_bytes;
    if (!is_type(dtype) || rows < 0 || rows > (1 << 22) || n < 1 || n > (1 << 20) || row_stride < n) return HAWK_EINVAL;
    if (rows == 0) return HAWK_OK;
    if (!logits || !u || !out_token || (reinterpret_cast<uintptr_t>(logits) & (type_bytes(dtype) - 1))) return HAWK_EINVAL;
    FilterArgs a = {};
    a.logits = static_cast<const char*>(logits); a.row_stride = row_stride; a.dtype = dtype; a.n = n;
    a.skip = skip; a.u = u; a.temperature = temperature; a.top_k = top_k; a.top_p = top_p; a.min_p = min_p;
    a.out_token = out_token; a.out_prob = out_prob; a.out_kept = out_kept;
    int log = 0;
    while ((1 << log) < n) ++log;
    a.unit = std::min(51, 62 - log);
    if (n <= 4 * NT) sample_filtered_kernel<4><<<(unsigned)rows, NT, 0, stream>>>(a);
    else if (n <= 16 * NT) sample_filtered_kernel<16><<<(unsigned)rows, NT, 0, stream>>>(a);
    else if (n <= 64 * NT) sample_filtered_kernel<64><<<(unsigned)rows, NT, 0, stream>>>(a);
    else sample_filtered_kernel<0><<<(unsigned)rows, NT, 0, stream>>>(a);
    return status();
}

}  // namespace hawk
