// The cache of a target pass over many sequences: keys and values in pages.  Appending a step's rows (queries and keys
// normalised per head and rotated on the way) and moving the accepted path of a tree step into place.
// paged_attention.hip reads it.
#include "paged.h"

#include <algorithm>

namespace hawk {

namespace {

__global__ void rotary_table_kernel(float2* table, int64_t total, int half, double theta) {
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= total) return;
    const int64_t p = i / half;
    const double a = (double)p * pow(theta, -2.0 * (double)(i - p * half) / (2.0 * half));
    table[i] = make_float2((float)cos(a), (float)sin(a));
}

struct AppendArgs {
    PagedView c;
    RowsView r;
    HeadsView q, k, v, q_out;
    const float *q_gain, *k_gain, *rot;
    const int32_t* pos;
    float eps, inv_hd;
    int n_pos, rot_dim, pairs;
    int lanes, per_block;           // lanes of a vector (2^lanes), vectors that a workgroup's lanes take side by side
    Divisor blocks;                 // workgroups of a row
    int step;                       // rows between a workgroup's rows
};

template <int TYPE> struct Bytes { static constexpr int n = TYPE == HAWK_FP32 ? 4 : 2; };

// N values of a type as they lie in memory: requested in one place, used in another.
template <int TYPE, int N> struct Piece {
    static constexpr int kWords = N * Bytes<TYPE>::n / 4;
    typedef unsigned part __attribute__((ext_vector_type(kWords < 4 ? kWords : 4)));
    static constexpr int kParts = kWords < 4 ? 1 : kWords / 4;
    part w[kParts];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < kParts; ++i) w[i] = (part)0u;
    }
    __device__ __forceinline__ void load(const char* base, int at) {
#pragma unroll
        for (int i = 0; i < kParts; ++i) w[i] = reinterpret_cast<const part*>(base + at * Bytes<TYPE>::n)[i];
    }
    __device__ __forceinline__ void widen(float* x) const {
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            const unsigned v = w[i / 4][i % 4];
            if (TYPE == HAWK_FP32) x[i] = __uint_as_float(v);
            else widen2(v, TYPE, x[2 * i], x[2 * i + 1]);
        }
    }
};

// Sum over 2^n neighbouring lanes, the same value in each: quad permutes and mirrors inside a row of 16, a swap beyond it.
template <int CTRL> __device__ __forceinline__ float moved(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float sum_of_lanes(float v, int n) {
    if (n > 0) v += moved<0xB1>(v);    // quad_perm [1,0,3,2]
    if (n > 1) v += moved<0x4E>(v);    // quad_perm [2,3,0,1]
    if (n > 2) v += moved<0x141>(v);   // row_half_mirror
    if (n > 3) v += moved<0x140>(v);   // row_mirror
    if (n > 4) v += __shfl_xor(v, 16);
    return v;
}

// A workgroup has some vectors - a vector is one head of q, k or v - of every step-th row; a vector belongs to 2^lanes neighbouring lanes
// of one wave, eight elements each, so that its sum of squares is a few lane moves and its bytes are one request.  Every
// lane reads its elements' partners of the rotation itself where they are half a vector away: they are in the same lines.
// Dependent latencies (row starts and lengths, then table and rotation) stand against a few hundred bytes, so a workgroup stays for as
// many rows as make the chip full of workgroups once, holds what is the same for all of them - where its vectors come from and go
// to, their gains, the sequences - and has the next row's requests under way while it works on a row's.  4048 rows of 32 + 16 heads of
// 128, norms and rotation of halves: 25.9 us (3.9 TB/s of what is read and written; a copy of as much takes 21), with a workgroup for
// every two rows 34.4, for every row 37.3; 16000 rows of 16 + 4 heads of 256 99 us, with a workgroup for two rows 139.
constexpr int kResident = 1024;     // workgroups that are on the chip at a time: four to a unit
template <int FROM, int TO>   // types
__global__ __launch_bounds__(256, 4) void paged_append_kernel(AppendArgs a) {
    const int row0 = (int)blockIdx.x / a.blocks, part = blockIdx.x - row0 * a.blocks.d;
    const int lane = threadIdx.x & 63, e0 = (threadIdx.x & ((1 << a.lanes) - 1)) * 8, hd = a.c.hd;
    const int nq = a.q.n_heads, nk = a.c.n_heads, half = a.rot_dim >> 1;   // half: a multiple of four, so four elements' partners are four in a row
    const int vec = part * a.per_block + ((int)threadIdx.x >> a.lanes), what = vec < nq ? 0 : (vec < nq + nk ? 1 : 2);
    const int head = vec - (what == 0 ? 0 : (what == 1 ? nq : nq + nk));
    const bool mine = vec < nq + 2 * nk && e0 < hd, turned = a.rot && what < 2 && e0 < a.rot_dim, apart = turned && a.pairs;
    int other[2] = {e0, e0 + 4}, at_table[2] = {e0 >> 1, (e0 >> 1) + 2};   // partners' elements; rows of the table (pairs side by side: one piece)
    float sign[2] = {1.f, 1.f};
    if (apart) {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const bool low = e0 + 4 * g < half;
            other[g] += low ? half : -half;
            at_table[g] = low ? e0 + 4 * g : other[g];
            sign[g] = low ? -1.f : 1.f;
        }
    }
    const HeadsView& src = what == 0 ? a.q : (what == 1 ? a.k : a.v);
    const char* from = src.data + (int64_t)head * src.head_stride * Bytes<FROM>::n;
    const int64_t from_step = src.row_stride * Bytes<FROM>::n;
    char* to = what == 0 ? a.q_out.data + (int64_t)head * a.q_out.head_stride * Bytes<TO>::n
                         : (what == 1 ? a.c.k : a.c.v) + (int64_t)head * a.c.head_stride * Bytes<TO>::n;
    // the sequences; up to 64 of them every lane has one sequence's words, and one look answers for a row
    const bool few = a.c.n_seq <= 64;
    const int mine_s = min(lane, a.c.n_seq - 1);
    int starts = 0, stops = 0, pasts = 0;
    if (few) {
        starts = a.r.row_start[mine_s];
        stops = a.r.row_start[mine_s + 1];
        pasts = a.r.n_past[mine_s];
    }
    struct Row {            // of one row, as requested
        Piece<FROM, 8> x;
        Piece<FROM, 4> y[2];
        float2 f[8];
        int page, slot;     // of the entry
        bool there;
    };
    auto request_x = [&](int row, Row& r) {
        r.x.clear();
        r.y[0].clear();
        r.y[1].clear();
        if (mine && row < a.r.rows) {
            const char* p = from + row * from_step;
            r.x.load(p, e0);
            if (apart) {
                r.y[0].load(p, other[0]);
                r.y[1].load(p, other[1]);
            }
        }
    };
    auto request_place = [&](int row, Row& r) {
        int s, start, stop, past;
        if (few) {
            s = __popcll(__ballot(lane < a.c.n_seq && starts <= row)) - 1;
            start = __builtin_amdgcn_readlane(starts, max(s, 0));
            stop = __builtin_amdgcn_readlane(stops, max(s, 0));
            past = __builtin_amdgcn_readlane(pasts, max(s, 0));
        } else {
            s = __builtin_amdgcn_readfirstlane(last_not_above(a.c.n_seq, lane, row, [&](int i) { return (int64_t)a.r.row_start[i]; }));
            start = a.r.row_start[max(s, 0)];
            stop = a.r.row_start[max(s, 0) + 1];
            past = a.r.n_past[max(s, 0)];
        }
        r.there = row < a.r.rows && s >= 0 && row < stop;   // else in no sequence
        const int64_t entry = (int64_t)past + (row - start);
        int64_t p = entry;
        if (a.pos && r.there) p = a.pos[row];
        if (a.rot) r.there = r.there && p >= 0 && p < a.n_pos;
        r.page = -1;
        r.slot = 0;
        if (r.there && entry >= 0 && entry < a.c.capacity) {
            const int n = page_of(a.c, (int)entry);
            r.page = a.c.table[s * a.c.table_stride + n];
            r.slot = (int)entry - n * a.c.page_size;
        }
        if (turned && r.there) {
            const float2* cs = reinterpret_cast<const float2*>(a.rot) + p * half;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (a.pairs || i < 4) r.f[i] = cs[at_table[i >> 2] + (i & 3)];
        }
    };
    const float* gain = what == 0 ? a.q_gain : (what == 1 ? a.k_gain : nullptr);
    float g[8], gp[8];   // the elements' gains and, signed as the rotation has them, their partners'
    auto append = [&](int row, const Row& r) {
        float x[8], y[8], rs = 1.f;
        r.x.widen(x);
        if (a.q_gain || a.k_gain) {   // (every lane takes part in the sum)
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
            ss = sum_of_lanes(ss, a.lanes);
            if (gain) rs = rsqrtf(ss * a.inv_hd + a.eps);
        }
        if (!r.there) return;
        if (apart) {
            r.y[0].widen(y);
            r.y[1].widen(y + 4);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = rs * fmaf(y[i], gp[i] * r.f[i].y, x[i] * (g[i] * r.f[i].x));
        } else if (turned) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float v = x[2 * i] * g[2 * i], w = x[2 * i + 1] * g[2 * i + 1];
                x[2 * i] = rs * fmaf(-w, r.f[i].y, v * r.f[i].x);
                x[2 * i + 1] = rs * fmaf(w, r.f[i].x, v * r.f[i].y);
            }
        } else if (gain) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = rs * (x[i] * g[i]);
        }
        const int64_t place = place_in(a.c, r.page, r.slot);
        if (mine && (what == 0 || place >= 0)) store8(to, (what == 0 ? row * a.q_out.row_stride : place) + e0, TO, x);
    };

    Row r0, r1;
    request_x(row0, r0);
#pragma unroll
    for (int i = 0; i < 8; ++i) { g[i] = 1.f; gp[i] = sign[i >> 2]; }
    if (gain && mine) {
        load8(reinterpret_cast<const char*>(gain), e0, HAWK_FP32, g);
        if (apart) {
            load4(reinterpret_cast<const char*>(gain), other[0], HAWK_FP32, gp);
            load4(reinterpret_cast<const char*>(gain), other[1], HAWK_FP32, gp + 4);
#pragma unroll
            for (int i = 0; i < 8; ++i) gp[i] *= sign[i >> 2];
        }
    }
    request_place(row0, r0);
    for (int row = row0;; row += 2 * a.step) {
        const bool second = row + a.step < a.r.rows, third = row + 2 * a.step < a.r.rows;
        if (second) {
            request_x(row + a.step, r1);
            request_place(row + a.step, r1);
        }
        append(row, r0);
        if (!second) break;
        if (third) {
            request_x(row + 2 * a.step, r0);
            request_place(row + 2 * a.step, r0);
        }
        append(row + a.step, r1);
        if (!third) break;
    }
}

// A wave moves one head's keys or values of one sequence and layer.  Nodes lie at or behind the places they go to, so an
// accepted entry is never overwritten before it has been read as long as moves are made in ascending order; within a
// batch every lane has its piece before any lane stores.
__global__ __launch_bounds__(256) void paged_keep_kernel(PagedView c, const int32_t* n_past, const int32_t* path,
                                                         const int32_t* n_keep, int depth, int64_t layer_bytes, int pieces,
                                                         int lanes, int waves, int blocks, int esz) {
    const int s = blockIdx.x / blocks, unit = (blockIdx.x - s * blocks) * 4 + ((int)threadIdx.x >> 6);
    if (unit >= waves) return;
    const int lane = threadIdx.x & 63, layer = unit / (2 * c.n_heads), hv = unit - layer * 2 * c.n_heads, head = hv >> 1;
    const int keep = min(n_keep[s], depth);
    const int64_t past = n_past[s];
    char* pool = ((hv & 1) ? c.v : c.k) + layer * layer_bytes + (int64_t)head * c.head_stride * esz;
    const int32_t* row = c.table + s * c.table_stride;
    const int per = 64 / lanes, piece = lane & (lanes - 1);
    for (int j0 = 0; j0 < keep; j0 += per) {
        const int j = j0 + lane / lanes;
        int64_t from = -1, to = -1;
        if (j < keep && piece < pieces) {
            const int node = path[(int64_t)s * depth + j];
            if (node > j + 1) {
                from = entry_at(c, row, past + node);
                to = entry_at(c, row, past + j + 1);
            }
        }
        const bool move = from >= 0 && to >= 0;
        v4u w = {0u, 0u, 0u, 0u};
        if (move) w = *reinterpret_cast<const v4u*>(pool + from * esz + piece * 16);
        if (move) *reinterpret_cast<v4u*>(pool + to * esz + piece * 16) = w;
    }
}

template <int FROM> void launch_append_from(const AppendArgs& a, int to, unsigned grid, hipStream_t stream) {
    auto kern = to == HAWK_FP32 ? paged_append_kernel<FROM, HAWK_FP32>
                                : (to == HAWK_BF16 ? paged_append_kernel<FROM, HAWK_BF16> : paged_append_kernel<FROM, HAWK_FP16>);
    kern<<<grid, 256, 0, stream>>>(a);
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
int status() { return hipGetLastError() == hipSuccess ? HAWK_OK : HAWK_EDEVICE; }

}  // namespace

bool paged_view(const hawk_paged_cache* c, int layer, PagedView* out) {
    if (!c || !c->k || !c->v || (!c->table && c->n_seq > 0) || !is_type(c->dtype) || !aligned16(c->k) || !aligned16(c->v)) return false;
    if (c->head_dim < 8 || c->head_dim > 256 || c->head_dim % 8 || c->n_heads < 1 || c->n_layers < 1 || c->n_pages < 1 ||
        c->page_size < 1 || c->n_seq < 0 || c->max_pages < 1 || (int64_t)c->max_pages * c->page_size > (1 << 30))
        return false;
    if (c->n_heads > 65535 || layer < 0 || layer >= c->n_layers || c->table_stride < c->max_pages) return false;
    if ((c->page_stride | c->head_stride | c->entry_stride | c->layer_stride) & 7) return false;
    if (c->page_stride < c->head_dim || c->head_stride < c->head_dim || c->entry_stride < c->head_dim || c->layer_stride < 0) return false;
    const int64_t off = layer * c->layer_stride * (int64_t)type_bytes(c->dtype);
    out->k = static_cast<char*>(c->k) + off;
    out->v = static_cast<char*>(c->v) + off;
    out->page_stride = c->page_stride; out->head_stride = c->head_stride; out->entry_stride = c->entry_stride;
    out->table = c->table; out->table_stride = c->table_stride;
    out->n_pages = c->n_pages; out->page_size = c->page_size; out->n_heads = c->n_heads; out->hd = c->head_dim;
    out->n_seq = c->n_seq; out->max_pages = c->max_pages;
    out->capacity = c->max_pages * c->page_size;
    out->page = divisor(c->page_size);
    return true;
}

bool heads_view(const hawk_heads* h, HeadsView* out) {
    if (!h || !h->data || !aligned16(h->data) || !is_type(h->dtype) || h->n_heads < 1 || h->n_heads > 65535) return false;
    if (((h->row_stride | h->head_stride) & 7) || h->row_stride < 0 || h->head_stride < 0) return false;
    out->data = static_cast<char*>(h->data);
    out->row_stride = h->row_stride; out->head_stride = h->head_stride; out->n_heads = h->n_heads; out->dtype = h->dtype;
    return true;
}

int launch_rotary_table(float* table, int n_pos, int rot_dim, double theta, hipStream_t stream) {
    if ((!table && n_pos > 0) || n_pos < 0 || rot_dim < 2 || rot_dim % 2 || !(theta > 0.0) || (reinterpret_cast<uintptr_t>(table) & 7)) return HAWK_EINVAL;
    if (n_pos == 0) return HAWK_OK;
    const int64_t total = (int64_t)n_pos * (rot_dim / 2), blocks = (total + 255) / 256;
    if (blocks > (1 << 23)) return HAWK_EINVAL;
    rotary_table_kernel<<<(unsigned)blocks, 256, 0, stream>>>(reinterpret_cast<float2*>(table), total, rot_dim / 2, theta);
    return status();
}

int launch_paged_append(const hawk_paged_cache* cache, int layer, const hawk_paged_rows* rows, const hawk_heads* q,
                        const hawk_heads* k, const hawk_heads* v, const float* q_gain, const float* k_gain, float eps,
                        const float* rot, int n_pos, int rot_dim, int pairs, const int32_t* pos, const hawk_heads* q_out,
                        hipStream_t stream) {
    AppendArgs a = {};
    if (!paged_view(cache, layer, &a.c)) return HAWK_EINVAL;
    if (nothing_to_do(cache, rows)) return HAWK_OK;
    if (!rows_view(rows, &a.r)) return HAWK_EINVAL;
    const int hd = a.c.hd;
    if (!heads_view(k, &a.k) || !heads_view(v, &a.v) || a.k.n_heads != a.c.n_heads || a.v.n_heads != a.c.n_heads) return HAWK_EINVAL;
    if (a.k.dtype != a.v.dtype || (q == nullptr) != (q_out == nullptr)) return HAWK_EINVAL;
    if (q) {
        if (!heads_view(q, &a.q) || !heads_view(q_out, &a.q_out) || a.q.n_heads != a.q_out.n_heads) return HAWK_EINVAL;
        if (a.q.dtype != a.k.dtype || a.q_out.dtype != cache->dtype) return HAWK_EINVAL;
        // q itself only where every element is its own place
        if (!room_for(a.q_out, a.r.rows, hd)) return HAWK_EINVAL;
        if (a.q_out.data == a.q.data && (a.q_out.dtype != a.q.dtype || a.q_out.row_stride != a.q.row_stride ||
                                         a.q_out.head_stride != a.q.head_stride))
            return HAWK_EINVAL;
    }
    a.q_out.dtype = cache->dtype;
    if (!aligned16(q_gain) || !aligned16(k_gain) || (q_gain && !q) || ((q_gain || k_gain) && !(eps >= 0.f))) return HAWK_EINVAL;
    if (rot) {
        if (!aligned16(rot) || n_pos < 1 || rot_dim < 8 || rot_dim % 8 || rot_dim > hd || pairs < 0 || pairs > 1) return HAWK_EINVAL;
    } else if (pos) {
        return HAWK_EINVAL;
    }
    a.inv_hd = 1.f / (float)hd;
    a.q_gain = q_gain; a.k_gain = k_gain; a.eps = eps; a.rot = rot; a.n_pos = n_pos; a.rot_dim = rot ? rot_dim : 0; a.pairs = pairs; a.pos = pos;
    while ((8 << a.lanes) < hd) ++a.lanes;
    a.per_block = 256 >> a.lanes;
    const int vectors = a.q.n_heads + 2 * a.c.n_heads;
    a.blocks = divisor((vectors + a.per_block - 1) / a.per_block);
    if ((int64_t)a.r.rows * a.blocks.d > (1 << 23)) return HAWK_EINVAL;   // as other steps too large for one launch
    a.step = std::min(a.r.rows, std::max(1, kResident / a.blocks.d));
    const unsigned grid = (unsigned)(a.step * a.blocks.d);
    if (a.k.dtype == HAWK_FP32) launch_append_from<HAWK_FP32>(a, cache->dtype, grid, stream);
    else if (a.k.dtype == HAWK_BF16) launch_append_from<HAWK_BF16>(a, cache->dtype, grid, stream);
    else launch_append_from<HAWK_FP16>(a, cache->dtype, grid, stream);
    return status();
}

int launch_paged_keep(const hawk_paged_cache* cache, const int32_t* n_past, const int32_t* path, const int32_t* n_keep,
                      int depth, hipStream_t stream) {
    PagedView c;
    if (!paged_view(cache, 0, &c) || depth < 1 || depth > 64) return HAWK_EINVAL;
    if (cache->n_layers > 1 && cache->layer_stride < c.hd) return HAWK_EINVAL;   // layers in one another's place
    if (c.n_seq == 0) return HAWK_OK;
    if (!n_past || !path || !n_keep) return HAWK_EINVAL;
    const int esz = (int)type_bytes(cache->dtype), pieces = c.hd * esz / 16;
    int lanes = 1;
    while (lanes < pieces) lanes *= 2;
    const int64_t waves = (int64_t)cache->n_layers * 2 * c.n_heads, blocks = (waves + 3) / 4;
    if (waves > (1 << 25) || blocks * c.n_seq > (1 << 23)) return HAWK_EINVAL;
    paged_keep_kernel<<<(unsigned)(blocks * c.n_seq), 256, 0, stream>>>(c, n_past, path, n_keep, depth, cache->layer_stride * esz, pieces,
                                                                      lanes, (int)waves, (int)blocks, esz);
    return status();
}

}  // namespace hawk
