// Verification of drafted chains on logits the caller has: the statistics of every row that a sequence's drafts need, one
// workgroup a row, then per sequence the acceptance tests and one draw from the first rejected position's residual or
// the row behind the last draft.
#include "sample_rows.h"

namespace hawk {

namespace {

struct ChainArgs {
    const float *p, *q;
    int64_t p_stride, q_seq, q_stride;
    const int32_t *p_start, *draft, *n_draft;
    const float *u_acc, *u_final;
    int p_rows, n_seq, k, n, top_k, greedy;
    float inv_t;
    WarpStat* stat;            // [n_seq][2 k + 1]: the target's k + 1 rows, then the proposals'
    int32_t *llen, *lidx;      // lists of the target's rows, [n_seq][k + 1]
    double* lw;
    int32_t *out_n, *out_tok;
};

// Drafts of a sequence, -1 if it is left out; its first target row.
__device__ __forceinline__ int chain_of(const ChainArgs& a, int s, int64_t& row0) {
    row0 = a.p_start ? (int64_t)a.p_start[s] : (int64_t)s * (a.k + 1);
    const int nd = a.n_draft ? min(a.n_draft[s], a.k) : a.k;
    return nd < 0 || row0 < 0 || row0 + nd >= a.p_rows ? -1 : nd;
}

// E entries a thread in registers, 0: a row of any length from memory
template <int E>
__global__ __launch_bounds__(NT) void chain_stats_kernel(ChainArgs a) {
    const int per = a.q ? 2 * a.k + 1 : a.k + 1, s = blockIdx.x / per, r = blockIdx.x - s * per;
    int64_t row0;
    const int nd = chain_of(a, s, row0);
    const bool target = r <= a.k;
    if (target ? r > nd : r - a.k - 1 >= nd) return;
    const float* l = target ? a.p + (row0 + r) * a.p_stride : a.q + s * a.q_seq + (int64_t)(r - a.k - 1) * a.q_stride;
    WarpStat st;
    if constexpr (E > 0) {
        __shared__ FastShared fs;
        __shared__ CompactList L;
        float z[E];
        load_row<E>(l, nullptr, 0.f, a.inv_t, nullptr, a.n, z);
        ListStore store = {nullptr, nullptr, nullptr};
        if (target && a.llen) store = list_at(a.llen, a.lidx, a.lw, (size_t)s * (a.k + 1) + r);
        st = warp_and_draw<E>(z, a.n, a.top_k, a.greedy, fs, L, nullptr, nullptr, store);
    } else {
        __shared__ Shared sh;
        st = warp_stats(l, a.n, a.inv_t, a.top_k, a.greedy, sh);
    }
    if (threadIdx.x == 0) a.stat[(size_t)s * (2 * a.k + 1) + r] = st;
}

__device__ __forceinline__ int draw_dense(const ChainArgs& a, const float* prow, const WarpStat& ps, const float* qrow, const WarpStat& qs,
                                          bool resid, int d, float u, Shared& sh) {
    auto wp = [&](int j) { return weight_of(ps, prow, a.inv_t, j); };
    if (resid) {
        auto left = [&](int j) {
            const double q = qrow ? weight_of(qs, qrow, a.inv_t, j) / qs.total : (j == d ? 1.0 : 0.0);
            const double r = weight_of(ps, prow, a.inv_t, j) / ps.total - q;
            return r > 0.0 ? r : 0.0;
        };
        const Seg sg = my_segment(a.n);
        double sum = 0.0;
        for (int j = sg.j0; j < sg.j1; ++j) sum += left(j);
        const double R = block_sum_d(sum, sh);
        if (R > 0.0) return inv_cdf(left, a.n, R, u, sh);
    }
    return inv_cdf(wp, a.n, ps.total, u, sh);
}

__global__ __launch_bounds__(NT) void chain_accept_kernel(ChainArgs a) {
    __shared__ Slots sl;
    __shared__ Shared sh;
    const int s = blockIdx.x, lane = threadIdx.x & 63;
    int64_t row0;
    const int nd = chain_of(a, s, row0);
    int32_t* out = a.out_tok + (int64_t)s * (a.k + 1);
    if (nd < 0) {
        if ((int)threadIdx.x <= a.k) out[threadIdx.x] = -1;
        if (threadIdx.x == 0) a.out_n[s] = -1;
        return;
    }
    if (threadIdx.x == 0) sl.pick = 0x7FFFFFFF;
    const WarpStat* stat = a.stat + (size_t)s * (2 * a.k + 1);
    // lane i of every wave makes test i; the first rejection is where the chain ends (k <= 63)
    bool rejected = false;
    if (lane < nd) {
        const int d = a.draft[(int64_t)s * a.k + lane];
        double pd = 0.0, qd = 1.0;
        if ((unsigned)d < (unsigned)a.n) {
            const WarpStat ps = stat[lane];
            pd = weight_of(ps, a.p + (row0 + lane) * a.p_stride, a.inv_t, d) / ps.total;
            if (a.q) {
                const WarpStat qs = stat[a.k + 1 + lane];
                qd = weight_of(qs, a.q + s * a.q_seq + (int64_t)lane * a.q_stride, a.inv_t, d) / qs.total;
            }
        }
        rejected = !((double)a.u_acc[(int64_t)s * a.k + lane] * qd < pd);
    }
    const unsigned long long rej = __ballot(rejected);
    const int acc = rej ? (int)__ffsll(rej) - 1 : nd;
    const float uf = a.u_final[s];
    const bool ended = acc < nd;
    const float* prow = a.p + (row0 + acc) * a.p_stride;
    const float* qrow = ended && a.q ? a.q + s * a.q_seq + (int64_t)acc * a.q_stride : nullptr;
    const WarpStat ps = stat[acc];
    WarpStat qs = ps;
    if (qrow) qs = stat[a.k + 1 + acc];
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
            for (int h = 0; h < kLH; ++h) {
                r[h] = 0.0;
                if (idx[h] >= 0) {
                    const double q = qrow ? weight_of(qs, qrow, a.inv_t, idx[h]) / qs.total : (idx[h] == d ? 1.0 : 0.0);
                    const double v = w[h] / ps.total - q;
                    r[h] = v > 0.0 ? v : 0.0;
                }
            }
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
        tok = draw_dense(a, prow, ps, qrow, qs, ended, d, uf, sh);
    }
    const int i = threadIdx.x;
    if (i <= a.k) out[i] = i < acc ? a.draft[(int64_t)s * a.k + i] : (i == acc ? ((unsigned)tok < (unsigned)a.n ? tok : 0) : -1);   // NaN logits: still a token of the slice
    if (i == 0) a.out_n[s] = acc;
}

size_t up16(size_t x) { return (x + 15) / 16 * 16; }
struct ChainSizes { size_t stat, len, idx, w; };
ChainSizes sizes_of(int n_seq, int k, int n) {
    const size_t rows = (size_t)n_seq * (k + 1), lists = n <= 16 * NT ? rows : 0;
    return {up16((size_t)n_seq * (2 * k + 1) * sizeof(WarpStat)), up16(list_len_bytes(lists)), up16(list_idx_bytes(lists)), up16(list_w_bytes(lists))};
}

}  // namespace

size_t verify_chains_workspace_bytes(int n_seq, int k, int n) {
    const ChainSizes z = sizes_of(n_seq, k, n);
    return z.stat + z.len + z.idx + z.w;
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
    auto stats = E == 4 ? chain_stats_kernel<4> : (E == 8 ? chain_stats_kernel<8> : (E == 16 ? chain_stats_kernel<16> : chain_stats_kernel<0>));
    stats<<<rows, NT, 0, stream>>>(a);
    chain_accept_kernel<<<n_seq, NT, 0, stream>>>(a);
    return hipGetLastError() == hipSuccess ? HAWK_OK : HAWK_EDEVICE;
}

}  // namespace hawk
