// The cache of a target pass over many sequences: keys and values in pages.  Appending a step's rows (queries and keys
// normalised per head and rotated on the way) and moving the accepted path of a tree step into place.
// paged_attention.hip reads it.
#include "paged.h"

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
    float eps;
    int n_pos, rot_dim, pairs;
    int lanes, per_block, blocks;   // lanes of a vector (a power of two), vectors of a workgroup, workgroups of a row
};

// Block (part of a row's vectors, row); a vector - one head of q, k or v - belongs to `lanes` neighbouring lanes of one wave,
// eight elements each, so that its sum of squares is a few lane swaps and its bytes are one request.  Every lane reads
// its elements' partners of the rotation itself where they are half a vector away: they are in the same lines.
__global__ __launch_bounds__(256) void paged_append_kernel(AppendArgs a) {
    const int row = blockIdx.x / a.blocks, part = blockIdx.x - row * a.blocks;
    const int lane = threadIdx.x & 63, e0 = (threadIdx.x & (a.lanes - 1)) * 8, hd = a.c.hd;
    const int vec = part * a.per_block + (int)threadIdx.x / a.lanes;
    const int nq = a.q.n_heads, nk = a.c.n_heads;
    const int what = vec < nq ? 0 : (vec < nq + nk ? 1 : 2), head = vec - (what == 0 ? 0 : (what == 1 ? nq : nq + nk));
    const bool mine = vec < nq + 2 * nk && e0 < hd;
    const HeadsView& src = what == 0 ? a.q : (what == 1 ? a.k : a.v);
    const int64_t at = (int64_t)row * src.row_stride + (int64_t)head * src.head_stride;
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (mine) load8(src.data, at + e0, src.dtype, x);

    const int s = last_not_above(a.c.n_seq, lane, row, [&](int i) { return (int64_t)a.r.row_start[i]; });
    if (s < 0 || row >= a.r.row_start[s + 1]) return;   // in no sequence
    const int64_t entry = (int64_t)a.r.n_past[s] + (row - a.r.row_start[s]);
    const float2* cs = nullptr;
    if (a.rot) {
        const int64_t p = a.pos ? (int64_t)a.pos[row] : entry;
        if (p < 0 || p >= a.n_pos) return;
        cs = reinterpret_cast<const float2*>(a.rot) + p * (a.rot_dim >> 1);
    }
    const int64_t place = entry_at(a.c, a.c.table + s * a.c.table_stride, entry);

    const float* gain = what == 0 ? a.q_gain : (what == 1 ? a.k_gain : nullptr);
    float rs = 1.f;
    if (gain) {
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
        for (int m = 1; m < a.lanes; m <<= 1) ss += __shfl_xor(ss, m);
        rs = 1.f / sqrtf(ss / (float)hd + a.eps);
        if (mine) {
            float g[8];
            load8(reinterpret_cast<const char*>(gain), e0, HAWK_FP32, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = x[i] * rs * g[i];
        }
    }
    if (cs && what < 2 && mine && e0 < a.rot_dim) {
        if (a.pairs == 0) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 t = cs[(e0 >> 1) + i];
                const float u = x[2 * i], w = x[2 * i + 1];
                x[2 * i] = u * t.x - w * t.y;
                x[2 * i + 1] = u * t.y + w * t.x;
            }
        } else {
            const int half = a.rot_dim >> 1;   // a multiple of four: four elements' partners are four in a row
#pragma unroll
            for (int g4 = 0; g4 < 2; ++g4) {
                const int e = e0 + 4 * g4;
                const bool low = e < half;
                const int other = low ? e + half : e - half, j = low ? e : e - half;
                float y[4];
                load4(src.data, at + other, src.dtype, y);
                if (gain) {
                    float g[4];
                    load4(reinterpret_cast<const char*>(gain), other, HAWK_FP32, g);
#pragma unroll
                    for (int i = 0; i < 4; ++i) y[i] = y[i] * rs * g[i];
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 t = cs[j + i];
                    float& v = x[4 * g4 + i];
                    v = low ? v * t.x - y[i] * t.y : y[i] * t.y + v * t.x;
                }
            }
        }
    }
    if (!mine) return;
    if (what == 0)
        store8(a.q_out.data, (int64_t)row * a.q_out.row_stride + (int64_t)head * a.q_out.head_stride + e0, a.q_out.dtype, x);
    else if (place >= 0)
        store8(what == 1 ? a.c.k : a.c.v, place + (int64_t)head * a.c.head_stride + e0, a.q_out.dtype, x);
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
    if (!table || n_pos < 0 || rot_dim < 2 || rot_dim % 2 || !(theta > 0.0) || (reinterpret_cast<uintptr_t>(table) & 7)) return HAWK_EINVAL;
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
    a.q_gain = q_gain; a.k_gain = k_gain; a.eps = eps; a.rot = rot; a.n_pos = n_pos; a.rot_dim = rot ? rot_dim : 0; a.pairs = pairs; a.pos = pos;
    a.lanes = 1;
    while (a.lanes * 8 < hd) a.lanes *= 2;
    a.per_block = 256 / a.lanes;
    a.blocks = (a.q.n_heads + 2 * a.c.n_heads + a.per_block - 1) / a.per_block;
    const int64_t grid = (int64_t)a.r.rows * a.blocks;
    if (grid > (1 << 23)) return HAWK_EINVAL;   // a launch has fewer than 2^32 threads
    paged_append_kernel<<<(unsigned)grid, 256, 0, stream>>>(a);
    return status();
}

int launch_paged_keep(const hawk_paged_cache* cache, const int32_t* n_past, const int32_t* path, const int32_t* n_keep,
                      int depth, hipStream_t stream) {
    PagedView c;
    if (!paged_view(cache, 0, &c) || !n_past || !path || !n_keep || depth < 1 || depth > 64) return HAWK_EINVAL;
    if (c.n_seq == 0) return HAWK_OK;
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
