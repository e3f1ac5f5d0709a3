// Verification of drafted chains on logits the caller has: the statistics of every row that a sequence's drafts need, then per
// sequence the acceptance tests and one draw from the first rejected position's residual or the row behind the last draft.
//
// Rows whose kept entries fit a list (top-k up to 2048, slices up to 16384) and short slices are one workgroup a row and one a
// sequence.  Other slices are cut into up to 16 parts: a row of 65536 entries takes one compute unit 15 us for its exponentials
// alone, and a sequence's draw three passes over two of them.  Where every entry is kept, a part's statistics are its maximum and
// sum, and whoever needs a row's joins them; where top-k cuts a long slice, a workgroup finds a row's threshold.  Then a
// workgroup per sequence and part makes the tests (all of them the same ones) and sums its part of the residual, and one per sequence
// picks the part and the entry.
#include "sample_rows.h"

// Kernels here compute the same value more than once - an entry's bin in two passes, a weight where it is summed and where it is drawn - and
// compare what comes out: every product is rounded by itself, whatever it is added to.
#pragma clang fp contract(off)

namespace hawk {

namespace {

struct PartStat { double sum; float top; int arg; };                       // of a part of a row: sum of exp(z - top); entry of the maximum
struct ChainEnd { WarpStat ps, qs; int64_t row0; int acc, ended, d; };      // of a sequence: the position that ends it (acc < 0: it is left out)

struct ChainArgs {
    const float *p, *q;
    int64_t p_stride, q_seq, q_stride;
    const int32_t *p_start, *draft, *n_draft;
    const float *u_acc, *u_final;
    int p_rows, n_seq, k, n, top_k, greedy, n_parts;
    float inv_t;
    WarpStat* stat;            // [n_seq][2 k + 1]: the target's k + 1 rows, then the proposals'
    int32_t *llen, *lidx;      // lists of the target's rows, [n_seq][k + 1]
    double* lw;
    PartStat* parts;           // [n_seq][2 k + 1][16]
    double* mass;              // [n_seq][2][16]: the residual's and the target's sums of the parts
    ChainEnd* end;             // [n_seq]
    int32_t *out_n, *out_tok;
};

// Drafts of a sequence, -1 if it is left out; its first target row.
__device__ __forceinline__ int chain_of(const ChainArgs& a, int s, int64_t& row0) {
    row0 = a.p_start ? (int64_t)a.p_start[s] : (int64_t)s * (a.k + 1);
    const int nd = a.n_draft ? min(a.n_draft[s], a.k) : a.k;
    return nd < 0 || row0 < 0 || row0 + nd >= a.p_rows ? -1 : nd;
}

__device__ __forceinline__ const float* chain_row(const ChainArgs& a, int s, int64_t row0, int r) {
    return r <= a.k ? a.p + (row0 + r) * a.p_stride : a.q + s * a.q_seq + (int64_t)(r - a.k - 1) * a.q_stride;
}
__device__ __forceinline__ bool row_needed(const ChainArgs& a, int r, int nd) { return r <= a.k ? r <= nd : r - a.k - 1 < nd; }

// The threshold of a long row's top_k largest: linear bins below the maximum (whatever lies more than kReach below shares the last one),
// and an exact ranking of the entries of the threshold's bin.  Rows this does not thin out take the general form.  Both passes bin the rounded
// z (a product fused with the difference to the maximum would put entries at a border into another bin than the second pass).
constexpr float kReach = 32.f;
constexpr int kRank = 1024;
struct LongShared {
    unsigned hist[NT];
    float z[kRank], ranked[kRank];
    int idx[kRank];
    float queue[NW][128];
    unsigned n;
    int bin, want, count, cut;
    float tau;
};
template <class F> __device__ __forceinline__ void for_row(const float* l, int n, F f) {   // f(index, value), 16 bytes a request where they are aligned
    if ((n & 3) == 0 && (reinterpret_cast<uintptr_t>(l) & 15) == 0) {
        for (int j = threadIdx.x * 4; j < n; j += blockDim.x * 4) {
            const float4 v = *reinterpret_cast<const float4*>(l + j);
            f(j, v.x); f(j + 1, v.y); f(j + 2, v.z); f(j + 3, v.w);
        }
    } else {
        for (int j = threadIdx.x; j < n; j += blockDim.x) f(j, l[j]);
    }
}
__device__ WarpStat long_stats(const float* l, int n, float inv_t, int K, LongShared& ls, Shared& sh) {
    const bool vec = (n & 3) == 0 && (reinterpret_cast<uintptr_t>(l) & 15) == 0;
    float top = -INFINITY;
    for_row(l, n, [&](int, float v) { top = fmaxf(top, v * inv_t); });
    ls.hist[threadIdx.x] = 0u;
    if (threadIdx.x == 0) ls.n = 0u;
    top = block_max_f(top, sh);
    if (!(fabsf(top) < INFINITY)) return warp_stats(l, n, inv_t, K, 0, sh);
    const float scale = (float)NT / kReach;
    auto bin_of = [&](float z) { return (int)fminf((top - z) * scale, (float)(NT - 1)); };   // (NaN: the last one)
    __syncthreads();
    for_row(l, n, [&](int, float v) { atomicAdd(&ls.hist[bin_of(v * inv_t)], 1u); });
    __syncthreads();
    const int c = (int)ls.hist[threadIdx.x], before = block_excl_scan_i(c, sh);
    if (before < K && before + c >= K) {
        ls.bin = threadIdx.x;
        ls.want = K - before;
        ls.count = c;
    }
    __syncthreads();
    const int bin = ls.bin, want = ls.want, cnt = ls.count;
    if (bin == NT - 1 || cnt > kRank) return warp_stats(l, n, inv_t, K, 0, sh);
    // Few entries of a wave's turn lie above the threshold's bin: they queue up until every lane has one, so that a wave
    // evaluates an exponential for 64 of them, in an order that is always the same.
    const int lane = threadIdx.x & 63, wave = wave_id();
    int queued = 0;
    double sum = 0.0;
    for (int j0 = 0; j0 < n; j0 += 4 * NT) {
        float z[4];
        int at[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            at[i] = vec ? j0 + 4 * (int)threadIdx.x + i : j0 + i * NT + (int)threadIdx.x;
            z[i] = -INFINITY;
        }
        if (vec) {
            if (at[0] < n) {
                const float4 v = *reinterpret_cast<const float4*>(l + at[0]);
                z[0] = v.x * inv_t; z[1] = v.y * inv_t; z[2] = v.z * inv_t; z[3] = v.w * inv_t;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (at[i] < n) z[i] = l[at[i]] * inv_t;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int b = bin_of(z[i]);
            if (b == bin && at[i] < n) {
                const unsigned slot = atomicAdd(&ls.n, 1u);
                if (slot < kRank) {   // (the same count as in the histogram)
                    ls.z[slot] = z[i];
                    ls.idx[slot] = at[i];
                }
            }
            const unsigned long long above = __ballot(b < bin);
            if (above) {
                if (b < bin) ls.queue[wave][queued + (int)__builtin_amdgcn_mbcnt_hi((unsigned)(above >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)above, 0u))] = z[i];
                queued += __popcll(above);
                if (queued >= 64) {
                    queued -= 64;
                    sum += exp((double)ls.queue[wave][queued + lane] - (double)top);
                }
            }
        }
    }
    if (lane < queued) sum += exp((double)ls.queue[wave][lane] - (double)top);
    __syncthreads();
    if ((int)threadIdx.x < cnt) {   // larger value first, lower index first among equals
        const float z = ls.z[threadIdx.x];
        const int j = ls.idx[threadIdx.x];
        int rank = 0;
        for (int i = 0; i < cnt; ++i) rank += ls.z[i] > z || (ls.z[i] == z && ls.idx[i] < j);
        ls.ranked[rank] = z;
        if (rank == want - 1) {
            ls.tau = z;
            ls.cut = j;
        }
    }
    __syncthreads();
    if ((int)threadIdx.x < want) sum += exp((double)ls.ranked[threadIdx.x] - (double)top);
    WarpStat st;
    st.total = block_sum_d(sum, sh);
    st.zmax = top;
    st.tau = fkey(ls.tau);   // (behind the sum's barriers)
    st.tie_cut = ls.cut;
    st.onehot = -1;
    return st;
}

// E entries a thread in registers, 0: a long row from memory
template <int E>
__global__ __launch_bounds__(NT) void chain_stats_kernel(ChainArgs a) {
    const int per = a.q ? 2 * a.k + 1 : a.k + 1, s = blockIdx.x / per, r = blockIdx.x - s * per;
    int64_t row0;
    const int nd = chain_of(a, s, row0);
    if (!row_needed(a, r, nd)) return;
    const float* l = chain_row(a, s, row0, r);
    WarpStat st;
    if constexpr (E > 0) {
        __shared__ FastShared fs;
        __shared__ CompactList L;
        float z[E];
        load_row<E>(l, nullptr, 0.f, a.inv_t, nullptr, a.n, z);
        ListStore store = {nullptr, nullptr, nullptr};
        if (r <= a.k && a.llen) store = list_at(a.llen, a.lidx, a.lw, (size_t)s * (a.k + 1) + r);
        st = warp_and_draw<E>(z, a.n, a.top_k, a.greedy, fs, L, nullptr, nullptr, store);
    } else {
        __shared__ LongShared ls;
        __shared__ Shared sh;
        st = long_stats(l, a.n, a.inv_t, a.top_k, ls, sh);
    }
    if (threadIdx.x == 0) a.stat[(size_t)s * (2 * a.k + 1) + r] = st;
}

// ---- slices in parts ----
// A part is 4096 entries, 16 a thread, as far as 16 parts go; with 16 parts for every slice 48 chains over 5000 entries took 41 us,
// over 16384 49 us.
constexpr int kParts = 16, kPT = 256;   // parts of a slice at most, threads of a part's workgroup
inline int parts_of(int n) { return n > kParts * 16 * kPT ? kParts : (n + 16 * kPT - 1) / (16 * kPT); }
__device__ __forceinline__ int part_entries(const ChainArgs& a) { return ((a.n + a.n_parts - 1) / a.n_parts + 3) / 4 * 4; }
// weight_of by exp_below, of a scaled logit.
__device__ __forceinline__ double entry_weight(const WarpStat& st, float z, int j, bool whole, const double* steps) {
    return whole || kept(st, z, j) ? exp_below((double)z - (double)st.zmax, steps) : 0.0;
}

// 16 scaled logits of a thread: entries j + 4 threadIdx.x .. + 3 and those 4 kPT, 8 kPT, 12 kPT behind; minus infinity past cnt.
__device__ __forceinline__ void load_16(const float* l, int j, int cnt, bool vec, float inv_t, float (&z)[16]) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int at = j + q * 4 * kPT + 4 * (int)threadIdx.x;
        float4 v = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
        if (vec) {
            if (at < cnt) v = *reinterpret_cast<const float4*>(l + at);
        } else {
            if (at < cnt) v.x = l[at];
            if (at + 1 < cnt) v.y = l[at + 1];
            if (at + 2 < cnt) v.z = l[at + 2];
            if (at + 3 < cnt) v.w = l[at + 3];
        }
        z[4 * q] = v.x * inv_t; z[4 * q + 1] = v.y * inv_t; z[4 * q + 2] = v.z * inv_t; z[4 * q + 3] = v.w * inv_t;
    }
}
__device__ __forceinline__ bool in_fours(const float* l, int cnt) { return (reinterpret_cast<uintptr_t>(l) & 15) == 0 && (cnt & 3) == 0; }

// Maximum (lowest index first) and sum of one part of one row; a thread rescales its own sum when its maximum grows.
__global__ __launch_bounds__(kPT) void chain_part_kernel(ChainArgs a) {
    __shared__ double steps[kSteps];
    __shared__ double ssum[kPT / 64];
    __shared__ float smax[kPT / 64];
    __shared__ int sarg[kPT / 64];
    const int per = a.q ? 2 * a.k + 1 : a.k + 1, u = blockIdx.x / a.n_parts, part = blockIdx.x - u * a.n_parts, s = u / per, r = u - s * per;
    int64_t row0;
    const int nd = chain_of(a, s, row0);
    if (!row_needed(a, r, nd)) return;
    const int len = part_entries(a), j0 = min(part * len, a.n), cnt = min(len, a.n - j0);
    const float* l = chain_row(a, s, row0, r) + j0;
    float top = -INFINITY;
    int arg = 0x7FFFFFFF;
    double sum = 0.0;
    const bool vec = in_fours(l, cnt);
    fill_steps(steps);
    __syncthreads();
    for (int j = 0; j < cnt; j += 16 * kPT) {
        float z[16], most = -INFINITY;
        load_16(l, j, cnt, vec, a.inv_t, z);
#pragma unroll
        for (int i = 0; i < 16; ++i) most = fmaxf(most, z[i]);
        if (a.greedy) {
#pragma unroll
            for (int i = 15; i >= 0; --i)
                if (z[i] == most && most > top) arg = j0 + j + (i >> 2) * 4 * kPT + 4 * (int)threadIdx.x + (i & 3);
            top = fmaxf(top, most);
        } else {
            if (most > top) {
                sum *= top > -INFINITY ? exp((double)top - (double)most) : 0.0;
                top = most;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) sum += exp_below((double)z[i] - (double)top, steps);   // (top minus infinity: NaN, so 0)
        }
    }
    const float wtop = wave_max_f(top);
    sum = wave_sum_d(top > -INFINITY ? sum * exp((double)top - (double)wtop) : 0.0);
    arg = wave_min_i(top == wtop ? arg : 0x7FFFFFFF);
    if ((threadIdx.x & 63) == 0) {
        ssum[threadIdx.x >> 6] = sum;
        smax[threadIdx.x >> 6] = wtop;
        sarg[threadIdx.x >> 6] = arg;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        PartStat p = {0.0, -INFINITY, 0x7FFFFFFF};
        for (int w = 0; w < kPT / 64; ++w) p.top = fmaxf(p.top, smax[w]);
        for (int w = 0; w < kPT / 64; ++w) {
            p.sum += smax[w] > -INFINITY ? ssum[w] * exp((double)smax[w] - (double)p.top) : 0.0;
            if (smax[w] == p.top) p.arg = min(p.arg, sarg[w]);
        }
        a.parts[((size_t)s * (2 * a.k + 1) + r) * kParts + part] = p;
    }
}

// The acceptance tests of a sequence, lane i of every wave making test i: what a test needs besides the rows' statistics, which may be asked
// for before these are there, and how many drafts are accepted.
struct Test { float zp, zq, u; int d; };
__device__ __forceinline__ Test test_of(const ChainArgs& a, int s, int64_t row0, int nd) {
    const int lane = threadIdx.x & 63;
    Test t = {0.f, 0.f, 0.f, -1};
    if (lane < nd) {
        t.d = a.draft[(int64_t)s * a.k + lane];
        t.u = a.u_acc[(int64_t)s * a.k + lane];
        if ((unsigned)t.d < (unsigned)a.n) {
            t.zp = chain_row(a, s, row0, lane)[t.d] * a.inv_t;
            if (a.q) t.zq = chain_row(a, s, row0, a.k + 1 + lane)[t.d] * a.inv_t;
        }
    }
    return t;
}
__device__ __forceinline__ double scaled_weight(const WarpStat& st, float z, int j) {   // weight_of, of a scaled logit
    if (st.onehot >= 0) return j == st.onehot ? 1.0 : 0.0;
    return kept(st, z, j) ? exp((double)z - (double)st.zmax) : 0.0;
}
__device__ __forceinline__ int accepted(const ChainArgs& a, int nd, const Test& t, const WarpStat* stat) {
    const int lane = threadIdx.x & 63;
    bool rejected = false;
    if (lane < nd) {
        double pd = 0.0, qd = 1.0;
        if ((unsigned)t.d < (unsigned)a.n) {
            const WarpStat ps = stat[lane];
            pd = scaled_weight(ps, t.zp, t.d) / ps.total;
            if (a.q) {
                const WarpStat qs = stat[a.k + 1 + lane];
                qd = scaled_weight(qs, t.zq, t.d) / qs.total;
            }
        }
        rejected = !((double)t.u * qd < pd);
    }
    const unsigned long long rej = __ballot(rejected);
    return rej ? (int)__ffsll(rej) - 1 : nd;   // the first rejection is where the chain ends (k <= 63)
}
__device__ __forceinline__ void leave_out(const ChainArgs& a, int s) {
    for (int i = threadIdx.x; i <= a.k; i += blockDim.x) a.out_tok[(int64_t)s * (a.k + 1) + i] = -1;
    if (threadIdx.x == 0) a.out_n[s] = -1;
}
__device__ __forceinline__ void put_tokens(const ChainArgs& a, int s, int acc, int tok) {
    for (int i = threadIdx.x; i <= a.k; i += blockDim.x)
        a.out_tok[(int64_t)s * (a.k + 1) + i] =
            i < acc ? a.draft[(int64_t)s * a.k + i] : (i == acc ? ((unsigned)tok < (unsigned)a.n ? tok : 0) : -1);   // NaN logits: still a token of the slice
    if (threadIdx.x == 0) a.out_n[s] = acc;
}
// max(0, p - q) at entry j of a rejected position; without a proposal's row q is the point mass on the draft.
__device__ __forceinline__ double residual_at(double p, const ChainArgs& a, const WarpStat& qs, const float* qrow, int d, int j) {
    const double q = qrow ? weight_of(qs, qrow, a.inv_t, j) / qs.total : (j == d ? 1.0 : 0.0);
    return p - q > 0.0 ? p - q : 0.0;
}

// Workgroup (sequence, part): the tests, then the part's sums of the residual and of the target itself.
__global__ __launch_bounds__(kPT) void chain_residual_kernel(ChainArgs a) {
    __shared__ WarpStat stat[2 * kMaxK + 1];
    __shared__ double steps[kSteps];
    __shared__ double sr[kPT / 64], sp[kPT / 64];
    const int groups = a.greedy ? 1 : a.n_parts, s = blockIdx.x / groups, part = blockIdx.x - s * groups;
    int64_t row0;
    const int nd = chain_of(a, s, row0);
    if (nd < 0) {
        if (part == 0) leave_out(a, s);
        if (part == 0 && threadIdx.x == 0) a.end[s].acc = -1;
        return;
    }
    const int rows = a.q ? 2 * a.k + 1 : a.k + 1;
    const size_t first = (size_t)s * (2 * a.k + 1);
    const Test test = test_of(a, s, row0, nd);
    fill_steps(steps);
    if (a.parts) {
        for (int r0 = 0; r0 < rows; r0 += kPT / kParts) {   // 16 lanes a row
            const int r = r0 + (int)threadIdx.x / kParts;
            const bool mine = r < rows && row_needed(a, r, nd);
            PartStat p = {0.0, -INFINITY, 0x7FFFFFFF};
            if (mine && (int)(threadIdx.x & (kParts - 1)) < a.n_parts) p = a.parts[(first + r) * kParts + (threadIdx.x & (kParts - 1))];
            float top = p.top;
#pragma unroll
            for (int w = 1; w < kParts; w <<= 1) top = fmaxf(top, __shfl_xor(top, w));
            int arg = p.top == top ? p.arg : 0x7FFFFFFF;
            double sum = p.top > -INFINITY ? p.sum * exp((double)p.top - (double)top) : 0.0;
#pragma unroll
            for (int w = 1; w < kParts; w <<= 1) {
                sum += __shfl_xor(sum, w);
                arg = min(arg, __shfl_xor(arg, w));
            }
            if (mine && (threadIdx.x & (kParts - 1)) == 0) {
                WarpStat st;   // every entry above minus infinity is kept
                st.total = a.greedy ? 1.0 : sum; st.zmax = top; st.tau = 0x007FFFFFu; st.tie_cut = -1; st.onehot = a.greedy ? arg : -1;
                stat[r] = st;
            }
        }
    } else {
        for (int r = threadIdx.x; r < rows; r += kPT)
            if (row_needed(a, r, nd)) stat[r] = a.stat[first + r];
    }
    __syncthreads();
    const int acc = accepted(a, nd, test, stat);
    if (a.greedy) {   // point masses: what is left of the target's is the target's
        put_tokens(a, s, acc, stat[acc].onehot);
        return;
    }
    const bool ended = acc < nd;
    const WarpStat ps = stat[acc], qs = ended && a.q ? stat[a.k + 1 + acc] : ps;
    const float *prow = chain_row(a, s, row0, acc), *qrow = ended && a.q ? chain_row(a, s, row0, a.k + 1 + acc) : nullptr;
    const int d = ended ? a.draft[(int64_t)s * a.k + acc] : -1;
    const int len = part_entries(a), j0 = min(part * len, a.n), cnt = min(len, a.n - j0);
    const bool whole = a.parts != nullptr;   // every entry above minus infinity is kept
    const double ip = 1.0 / ps.total, iq = 1.0 / qs.total;
    double r = 0.0, p = 0.0;
    const bool vp = in_fours(prow + j0, cnt), vq = qrow && in_fours(qrow + j0, cnt);
    for (int j = 0; j < cnt; j += 16 * kPT) {
        float zp[16], zq[16];
        load_16(prow + j0, j, cnt, vp, a.inv_t, zp);
        if (qrow) load_16(qrow + j0, j, cnt, vq, a.inv_t, zq);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int at = j0 + j + (i >> 2) * 4 * kPT + 4 * (int)threadIdx.x + (i & 3);
            const double w = entry_weight(ps, zp[i], at, whole, steps) * ip;
            p += w;
            if (ended) {
                const double q = qrow ? entry_weight(qs, zq[i], at, whole, steps) * iq : (at == d ? 1.0 : 0.0);
                r += w - q > 0.0 ? w - q : 0.0;
            }
        }
    }
    r = wave_sum_d(r);
    p = wave_sum_d(p);
    if ((threadIdx.x & 63) == 0) {
        sr[threadIdx.x >> 6] = r;
        sp[threadIdx.x >> 6] = p;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        r = p = 0.0;
        for (int w = 0; w < kPT / 64; ++w) {
            r += sr[w];
            p += sp[w];
        }
        a.mass[(size_t)s * 2 * kParts + part] = r;
        a.mass[(size_t)s * 2 * kParts + kParts + part] = p;
        if (part == 0) {
            ChainEnd e = {ps, qs, row0, acc, ended, d};
            a.end[s] = e;
        }
    }
}

// The part of a sequence's draw, then the entry: the first whose running sum exceeds u times the total, else the last one with weight.
__global__ __launch_bounds__(NT) void chain_draw_kernel(ChainArgs a) {
    __shared__ Shared sh;
    __shared__ double steps[kSteps];
    const int s = blockIdx.x;
    const ChainEnd e = a.end[s];
    const double* mass = a.mass + (size_t)s * 2 * kParts;
    double mr[kParts], m[kParts], total = 0.0;   // (all requested at once)
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
        mr[i] = i < a.n_parts ? mass[i] : 0.0;
        m[i] = i < a.n_parts ? mass[kParts + i] : 0.0;
    }
    fill_steps(steps);
    if (e.acc < 0) return;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kParts; ++i) total += mr[i];
    const bool resid = e.ended && total > 0.0;
    if (resid) {
#pragma unroll
        for (int i = 0; i < kParts; ++i) m[i] = mr[i];
    } else {
        total = 0.0;
#pragma unroll
        for (int i = 0; i < kParts; ++i) total += m[i];
    }
    const double target = (double)a.u_final[s] * total;
    int part = -1, last = 0;
    double before = 0.0, base = 0.0, lower = 0.0;   // what lies before the part; before the last one with weight
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
        if (m[i] > 0.0) {
            last = i;
            lower = before;
        }
        if (part < 0 && before + m[i] > target) {
            part = i;
            base = before;
        }
        before += m[i];
    }
    if (part < 0) {
        part = last;
        base = lower;
    }
    const float *prow = chain_row(a, s, e.row0, e.acc), *qrow = resid && a.q ? chain_row(a, s, e.row0, a.k + 1 + e.acc) : nullptr;
    const int len = part_entries(a), j0 = min(part * len, a.n), j1 = min(j0 + len, a.n);
    const bool whole = a.parts != nullptr;
    const double ip = 1.0 / e.ps.total, iq = 1.0 / e.qs.total;
    int tok = -1;
    for (int j = j0; j < j1; j += 4 * NT) {   // four entries a thread
        double w[4], sum = 0.0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = j + 4 * (int)threadIdx.x + i;
            w[i] = 0.0;
            if (at < j1) {
                w[i] = entry_weight(e.ps, prow[at] * a.inv_t, at, whole, steps) * ip;
                if (resid) {
                    const double q = qrow ? entry_weight(e.qs, qrow[at] * a.inv_t, at, whole, steps) * iq : (at == e.d ? 1.0 : 0.0);
                    w[i] = w[i] - q > 0.0 ? w[i] - q : 0.0;
                }
            }
            sum += w[i];
        }
        double c = base + block_excl_scan_d(sum, sh);
        int hit = 0x7FFFFFFF, seen = -1;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            c += w[i];
            if (w[i] > 0.0) {
                seen = j + 4 * (int)threadIdx.x + i;
                if (hit == 0x7FFFFFFF && c > target) hit = seen;
            }
        }
        hit = block_min_i(hit, sh);
        if (hit != 0x7FFFFFFF) {
            tok = hit;
            break;
        }
        tok = max(tok, block_max_i(seen, sh));
        base += block_sum_d(sum, sh);
    }
    put_tokens(a, s, e.acc, tok);
}

// ---- one workgroup a sequence: lists, and slices short enough for passes over all of them (2048 entries 17 us, 4096 entries 25
// us; in parts 20) ----
constexpr int kShort = 2 * NT;
__global__ __launch_bounds__(NT) void chain_accept_kernel(ChainArgs a) {
    __shared__ Slots sl;
    __shared__ Shared sh;
    const int s = blockIdx.x;
    int64_t row0;
    const int nd = chain_of(a, s, row0);
    if (nd < 0) {
        leave_out(a, s);
        return;
    }
    if (threadIdx.x == 0) sl.pick = 0x7FFFFFFF;
    const WarpStat* stat = a.stat + (size_t)s * (2 * a.k + 1);
    const int acc = accepted(a, nd, test_of(a, s, row0, nd), stat);
    const float uf = a.u_final[s];
    const bool ended = acc < nd;
    const WarpStat ps = stat[acc], qs = ended && a.q ? stat[a.k + 1 + acc] : ps;
    const float *prow = chain_row(a, s, row0, acc), *qrow = ended && a.q ? chain_row(a, s, row0, a.k + 1 + acc) : nullptr;
    const int d = ended ? a.draft[(int64_t)s * a.k + acc] : -1;
    int tok;
    if (a.llen) {   // the kept entries of the target's row, which hold all of the residual's
        const ListStore src = list_at(a.llen, a.lidx, a.lw, (size_t)s * (a.k + 1) + acc);
        const int Kc = *src.len;
        int idx[kLH];
        double w[kLH], c[kLH];
#pragma unroll
        for (int h = 0; h < kLH; ++h) {
            const int i = (int)threadIdx.x + h * NT;
            idx[h] = -1;
            w[h] = 0.0;
            if (i < Kc) { idx[h] = src.idx[i]; w[h] = src.w[i]; }
        }
        int at = 0;
        bool resid = false;
        __syncthreads();   // sl.pick is set
        if (ended) {
            double r[kLH];
#pragma unroll
            for (int h = 0; h < kLH; ++h) r[h] = idx[h] >= 0 ? residual_at(w[h] / ps.total, a, qs, qrow, d, idx[h]) : 0.0;
            const double R = list_scan(r, Kc, c, sl.scan[0]);
            if (R > 0.0) {
                resid = true;
                at = list_pick(r, c, (double)uf * R, sl, sh);
            }
        }
        if (!resid) {
            (void)list_scan(w, Kc, c, sl.scan[1]);
            at = list_pick(w, c, (double)uf * ps.total, sl, sh);
        }
        tok = Kc > 0 ? src.idx[at] : 0;
    } else if (a.greedy) {   // point masses: what is left of the target's is the target's
        tok = ps.onehot;
    } else {
        auto wp = [&](int j) { return weight_of(ps, prow, a.inv_t, j); };
        auto left = [&](int j) { return residual_at(weight_of(ps, prow, a.inv_t, j) / ps.total, a, qs, qrow, d, j); };
        double R = 0.0;
        if (ended) {
            const Seg sg = my_segment(a.n);
            double sum = 0.0;
            for (int j = sg.j0; j < sg.j1; ++j) sum += left(j);
            R = block_sum_d(sum, sh);
        }
        tok = R > 0.0 ? inv_cdf(left, a.n, R, uf, sh) : inv_cdf(wp, a.n, ps.total, uf, sh);
    }
    put_tokens(a, s, acc, tok);
}

size_t up16(size_t x) { return (x + 15) / 16 * 16; }
struct ChainSizes { size_t stat, len, idx, w, parts, mass, end; };
// (the kernels of one call use the first, and the lists or the parts)
ChainSizes sizes_of(int n_seq, int k, int n) {
    const size_t rows = (size_t)n_seq * (k + 1), lists = n <= 16 * NT ? rows : 0, all = (size_t)n_seq * (2 * k + 1);
    return {up16(all * sizeof(WarpStat)), up16(list_len_bytes(lists)), up16(list_idx_bytes(lists)), up16(list_w_bytes(lists)),
            up16(all * kParts * sizeof(PartStat)), up16((size_t)n_seq * 2 * kParts * sizeof(double)), up16(n_seq * sizeof(ChainEnd))};
}

}  // namespace

size_t verify_chains_workspace_bytes(int n_seq, int k, int n) {
    const ChainSizes z = sizes_of(n_seq, k, n);
    const size_t lists = z.len + z.idx + z.w, parts = z.parts + z.mass + z.end;
    return z.stat + (lists > parts ? lists : parts);
}

int launch_verify_chains(const float* p_logits, int64_t p_stride, const int32_t* p_start, int p_rows, const float* q_logits,
                         int64_t q_seq_stride, int64_t q_stride, const int32_t* draft, const int32_t* n_draft,
                         const float* u_acc, const float* u_final, int n_seq, int k, int n, float temperature, int top_k,
                         int32_t* out_n_accept, int32_t* out_tokens, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    ChainArgs a = {};
    a.p = p_logits; a.q = k > 0 ? q_logits : nullptr;
    a.p_stride = p_stride; a.q_seq = q_seq_stride; a.q_stride = q_stride;
    a.p_start = p_start; a.draft = draft; a.n_draft = n_draft; a.u_acc = u_acc; a.u_final = u_final;
    a.p_rows = p_rows; a.n_seq = n_seq; a.k = k; a.n = n;
    a.greedy = temperature == 0.0f || top_k == 1;
    a.inv_t = a.greedy ? 1.0f : 1.0f / temperature;
    a.top_k = top_k < n ? top_k : n;
    a.out_n = out_n_accept; a.out_tok = out_tokens;
    const ChainSizes z = sizes_of(n_seq, k, n);
    char* w = static_cast<char*>(workspace);
    a.stat = reinterpret_cast<WarpStat*>(w);
    const int E = n <= 4 * NT ? 4 : (n <= 8 * NT ? 8 : (n <= 16 * NT ? 16 : 0));
    if (E && use_list(a.top_k, n, a.greedy)) {
        a.llen = reinterpret_cast<int32_t*>(w + z.stat);
        a.lidx = reinterpret_cast<int32_t*>(w + z.stat + z.len);
        a.lw = reinterpret_cast<double*>(w + z.stat + z.len + z.idx);
    }
    const unsigned rows = (unsigned)n_seq * (unsigned)(a.q ? 2 * k + 1 : k + 1);
    if (a.llen || n <= kShort) {
        auto stats = E == 4 ? chain_stats_kernel<4> : (E == 8 ? chain_stats_kernel<8> : chain_stats_kernel<16>);
        stats<<<rows, NT, 0, stream>>>(a);
        chain_accept_kernel<<<n_seq, NT, 0, stream>>>(a);
    } else {
        char* more = w + z.stat;
        a.n_parts = parts_of(n);
        a.mass = reinterpret_cast<double*>(more + z.parts);
        a.end = reinterpret_cast<ChainEnd*>(more + z.parts + z.mass);
        if (a.greedy || a.top_k == n) {
            a.parts = reinterpret_cast<PartStat*>(more);
            chain_part_kernel<<<rows * a.n_parts, kPT, 0, stream>>>(a);
        } else {
            auto stats = E == 4 ? chain_stats_kernel<4> : (E == 8 ? chain_stats_kernel<8> : (E == 16 ? chain_stats_kernel<16> : chain_stats_kernel<0>));
            stats<<<rows, NT, 0, stream>>>(a);
        }
        chain_residual_kernel<<<n_seq * (a.greedy ? 1 : a.n_parts), kPT, 0, stream>>>(a);
        if (!a.greedy) chain_draw_kernel<<<n_seq, NT, 0, stream>>>(a);
    }
    return hipGetLastError() == hipSuccess ? HAWK_OK : HAWK_EDEVICE;
}

}  // namespace hawk
