// Pages of the cache of many sequences: which are taken, shared, given back and moved.  Everything is known from two arrays in device
// memory, the table (which page a place of a sequence has) and the counts (how many places have a page; 0: free), so that a step
// can be captured and replayed.  Lookups are one workgroup's work - they are a few thousand numbers, and what they cost is
// latency -, the entries are moved by a second launch that fills the chip.
#include "paged.h"

#include <algorithm>

namespace hawk {

namespace {

constexpr int kWide = 1024;         // threads of a workgroup that looks up
constexpr int kEach = 16;           // neighbouring counts a thread looks at in one round

// Exclusive prefix sum over the workgroup and the whole sum, the same in every thread.  `sums`: 17 words.  Ends with a barrier.
__device__ __forceinline__ int block_before(int v, int* sums, int& all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int x = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    if (lane == 63) sums[wave] = x;
    __syncthreads();
    int before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < kWide / 64; ++w) {
        const int s = sums[w];
        before += w < wave ? s : 0;
        all += s;
    }
    __syncthreads();
    return before + x - v;
}

__device__ __forceinline__ int pages_for(int64_t entries, const PagedView& c) {   // places that so many entries of a sequence fill
    if (entries <= 0) return 0;
    return entries >= c.capacity ? c.max_pages : page_of(c, (int)entries - 1) + 1;
}
__device__ __forceinline__ bool in_pool(const PagedView& c, int page) { return page >= 0 && page < c.n_pages; }

// A copy of the first n entries of a page, all layers and heads.
struct Move { int from, to, n; };
struct MoveList { int* count; Move* move; };

// Pair i: the sequence dst[i] has from now on the pages that hold src[i]'s committed entries, and what it had is given back.  A workgroup
// a pair.  Counts are sums of whole numbers: their order does not matter.  Every pair is compared with all others, which keeps the call without a
// workspace and a launch of its own for as many as there are (64 pairs 4.1 us; 16384 146 us, 65536 1.9 ms, 2^18 27 ms, beyond which it is refused).
constexpr int kMostPairs = 1 << 18;
__global__ __launch_bounds__(256) void paged_fork_kernel(PagedView c, int32_t* table, int32_t* refs, int32_t* n_past, const int32_t* src,
                                                         const int32_t* dst, int n) {
    const int i = blockIdx.x, from = src[i], to = dst[i];
    if (from < 0 || from >= c.n_seq || to < 0 || to >= c.n_seq || from == to) return;
    int lost = 0;
    for (int j = threadIdx.x; j < n; j += 256) {
        const int other = dst[j], base = src[j];
        const bool real = other >= 0 && other < c.n_seq && base >= 0 && base < c.n_seq && base != other;
        lost |= (other == to && j < i && real) || (other == from && real);   // a second pair for one sequence; a source that changes
    }
    if (__syncthreads_or(lost)) return;
    const int past = n_past[from], there = pages_for(past, c);
    const int32_t* a = table + from * c.table_stride;
    int32_t* b = table + to * c.table_stride;
    for (int p = threadIdx.x; p < c.max_pages; p += 256) {
        const int old = b[p], page = p < there ? a[p] : -1;
        if (in_pool(c, old)) atomicAdd(&refs[old], -1);
        if (in_pool(c, page)) atomicAdd(&refs[page], 1);
        b[p] = page;
    }
    if (threadIdx.x == 0) n_past[to] = past;
}

__global__ __launch_bounds__(256) void paged_trim_kernel(PagedView c, int32_t* table, int32_t* refs, const int32_t* n_past, Divisor blocks) {
    const int s = (int)blockIdx.x / blocks, p = ((int)blockIdx.x - s * blocks.d) * 256 + (int)threadIdx.x, past = n_past[s];
    if (p >= c.max_pages || past < 0 || p < pages_for(past, c)) return;
    int32_t* at = table + s * c.table_stride + p;
    const int page = *at;
    if (in_pool(c, page)) atomicAdd(&refs[page], -1);
    *at = -1;
}

struct TakeArgs {
    PagedView c;
    int32_t *table, *refs;
    const int32_t *n_past, *n_new;
    int32_t* short_by;              // [n_seq]
    int *free, *old;                // [n_pages]: free pages, lowest first, as many as are wanted; the page that a taken one stands in for
    MoveList moves;
    int lanes;                      // neighbouring lanes of a sequence (2^lanes)
};

// The pages that are written next.  First what every sequence lacks: places among those of entries n_past .. n_past + n_new - 1 that have no
// page or one that other places have too.  Then the free pages in ascending order, as many as are lacking.  Then they are handed
// out, sequences and places in ascending order, a sequence that would need more than there are (and all behind it) left as it
// was.  The counts that decide are those before the call: they are changed at the end.  72 sequences, 64 of which lack 2 pages of 700: 6.4 us, nearly
// all of it dependent latencies (8.2 with the counts requested once it was known how many are lacking).
__global__ __launch_bounds__(kWide) void paged_take_kernel(TakeArgs a) {
    __shared__ int sums[kWide / 64 + 1], given, moves;
    const PagedView& c = a.c;
    const int tid = threadIdx.x, per = kWide >> a.lanes, width = 1 << a.lanes, l = tid & (width - 1), group = (tid & 63) & ~(width - 1);
    const unsigned long long mine = width == 64 ? ~0ull : ((1ull << width) - 1ull) << group, before = mine & ((1ull << (tid & 63)) - 1ull);
    const bool once = c.n_seq <= per;                // what is found out at first still holds when pages are handed out
    auto lacks = [&](int s, int p, int& page) {
        page = a.table[s * c.table_stride + p];
        if (!in_pool(c, page)) { page = -1; return true; }
        return a.refs[page] > 1;
    };
    // A sequence's places that are written, entries of the first one that stay, pages it lacks; the lane's first place.
    int first = 0, stop = 0, inside = 0, need = 0, page0 = -1;
    bool lack0 = false;
    auto look = [&](int s) {
        first = stop = inside = need = 0;
        lack0 = false;
        if (s < c.n_seq) {
            const int past = a.n_past[s], add = a.n_new[s];
            if (past >= 0 && add > 0 && past < c.capacity) {
                first = page_of(c, past);
                stop = pages_for((int64_t)past + add, c);
                inside = past - first * c.page_size;
            }
        }
        if (first + l < stop) need = lack0 = lacks(s, first + l, page0);
        int page;
        for (int p = first + l + width; p < stop; p += width) need += lacks(s, p, page) ? 1 : 0;
        for (int w = 1; w < width; w <<= 1) need += __shfl_xor(need, w);
    };
    // Free pages among neighbouring counts: the first ones are requested before it is known how many are lacking.
    auto free_among = [&](int at) {
        unsigned bits = 0u;
        if (at + kEach <= c.n_pages) {
            typedef int i4 __attribute__((ext_vector_type(4), aligned(4)));
            i4 v[kEach / 4];
#pragma unroll
            for (int j = 0; j < kEach / 4; ++j) v[j] = *reinterpret_cast<const i4*>(a.refs + at + 4 * j);
#pragma unroll
            for (int j = 0; j < kEach; ++j) bits |= v[j / 4][j % 4] <= 0 ? 1u << j : 0u;
        } else {
            for (int j = 0; j < kEach && at + j < c.n_pages; ++j) bits |= a.refs[at + j] <= 0 ? 1u << j : 0u;
        }
        return bits;
    };
    const unsigned bits0 = free_among(tid * kEach);
    int wanted = 0;                                  // of this thread's sequences
    for (int s0 = 0; s0 < c.n_seq; s0 += per) {
        look(s0 + (tid >> a.lanes));
        wanted += l == 0 ? need : 0;
    }
    if (tid == 0) given = moves = 0;
    int total, n_free = 0;
    const int begin = block_before(wanted, sums, total);
    for (int p0 = 0; p0 < c.n_pages && n_free < total; p0 += kWide * kEach) {
        const int at = p0 + tid * kEach;
        unsigned bits = p0 == 0 ? bits0 : free_among(at);
        int all, k = n_free + block_before(__popc(bits), sums, all);
        for (; bits && k < total; bits &= bits - 1u) a.free[k++] = at + __ffs(bits) - 1;
        n_free += all;
    }
    __syncthreads();
    int asked = 0;                                   // of the sequences before this round's
    for (int s0 = 0; s0 < c.n_seq; s0 += per) {
        const int s = s0 + (tid >> a.lanes);
        int k = begin;
        if (!once) {
            look(s);
            int all;
            k = asked + block_before(l == 0 ? need : 0, sums, all);
            asked += all;
        }
        k = __shfl(k, group);                        // (the group's first lane counts for it)
        const bool served = k + need <= n_free;
        if (l == 0 && s < c.n_seq) {
            a.short_by[s] = served ? 0 : need;
            if (served && need > 0) atomicMax(&given, k + need);
            if (served && inside > 0 && lack0 && page0 >= 0) {
                // (the first place is the first that lacks a page, and gets the first page; copies may be made in any order)
                const Move mv = {page0, a.free[k], inside};
                a.moves.move[atomicAdd(&moves, 1)] = mv;
            }
        }
        if (!served || need == 0) continue;
        for (int p0 = first; p0 < stop; p0 += width) {
            const int p = p0 + l;
            int page = page0;
            const bool take = p < stop && (p0 == first ? lack0 : lacks(s, p, page));
            const unsigned long long who = __ballot(take);
            if (take) {
                const int at = k + __popcll(who & before), to = a.free[at];
                a.old[at] = page;
                a.table[s * c.table_stride + p] = to;
            }
            k += __popcll(who & mine);
        }
    }
    __syncthreads();
    if (tid == 0) *a.moves.count = moves;
    for (int i = tid; i < given; i += kWide) {
        a.refs[a.free[i]] = 1;
        if (a.old[i] >= 0) atomicAdd(&a.refs[a.old[i]], -1);
    }
}

// Of the pages in use those that lie behind as many places as there are pages in use, and the free ones before, are paired in ascending order.
__global__ __launch_bounds__(kWide) void paged_holes_kernel(PagedView c, const int32_t* refs, int32_t* refs_out, int* to, int* src, int* dst, MoveList moves,
                                                            int32_t* n_used) {
    __shared__ int sums[kWide / 64 + 1];
    const int tid = threadIdx.x;
    auto used = [&](int p) { return p < c.n_pages && refs[min(p, c.n_pages - 1)] > 0; };
    int n = 0;
    for (int p = tid; p < c.n_pages; p += kWide) n += used(p) ? 1 : 0;
    int total, holes = 0, behind = 0;
    block_before(n, sums, total);
    for (int p0 = 0; p0 < c.n_pages; p0 += kWide * kEach) {
        const int at = p0 + tid * kEach;
        unsigned bits = 0u;
#pragma unroll
        for (int j = 0; j < kEach; ++j) bits |= used(at + j) ? 1u << j : 0u;
        const int real = min(max(c.n_pages - at, 0), kEach), front = min(max(total - at, 0), real);   // of the thread's pages; before the border
        const unsigned low = (1u << front) - 1u, whole = (1u << real) - 1u;
        unsigned h = ~bits & low, b = bits & whole & ~low;
        int all;
        int k = holes + block_before(__popc(h), sums, all);
        holes += all;
        for (; h; h &= h - 1u) dst[k++] = at + __ffs(h) - 1;
        k = behind + block_before(__popc(b), sums, all);
        behind += all;
        for (; b; b &= b - 1u) src[k++] = at + __ffs(b) - 1;
        for (int j = 0; j < real; ++j) to[at + j] = (bits >> j) & 1u ? at + j : -1;
    }
    __syncthreads();
    for (int p = tid; p < c.n_pages; p += kWide) {   // (in place only what is below 0)
        const int r = refs[p];
        if (refs_out != refs || r < 0) refs_out[p] = max(r, 0);
    }
    __syncthreads();
    for (int i = tid; i < behind; i += kWide) {
        const Move mv = {src[i], dst[i], c.page_size};
        moves.move[i] = mv;
        to[mv.from] = mv.to;
        const int r = refs[mv.from];
        refs_out[mv.to] = r;
        refs_out[mv.from] = 0;
    }
    if (tid == 0) {
        *moves.count = behind;
        *n_used = total;
    }
}

struct CopyArgs {
    PagedView from, to;
    int64_t from_layer, to_layer;   // bytes
    const int32_t *src, *dst;       // pages of a list of the caller's (moves.count null)
    MoveList moves;
    int n, esz;
    int64_t batches;                // of the pieces of a whole page
    Divisor units, heads, pieces;   // of a page: layers times two pools times heads; heads; 16-byte pieces of an entry
    // tables on the way
    const int* map;                 // [n_pages]; null: none
    int32_t* table_out;
    int64_t table_out_stride, places;
};

// A wave moves 512 neighbouring pieces of 16 bytes of one page - heads one behind the other, of all layers and both pools -, eight a lane, requested
// together and then stored.  Parts of pages are as small as one entry: a wave that had one head of one layer at a time moved 640 bytes between
// two latencies (64 copies of 5 entries on average, 36 layers of 20 heads of 64: 36 us, so 26).  Workgroups stay for as many pieces as make the
// waves asked for: where there may be nothing to copy (a take), and where there are whole pages (us with 8192 / 16384 / 65536 waves: those 64
// with fork and take 38 / 36.3 / 37, 48 pages of 16.8 MB 344 / 337 / 326).
constexpr int kPartWaves = 16384, kPageWaves = 65536, kBatch = 512;
__global__ __launch_bounds__(256) void paged_copy_kernel(CopyArgs a) {
    const int lane = threadIdx.x & 63;
    if (a.map) {
        for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < a.places; i += (int64_t)gridDim.x * 256) {
            const int s = (int)(i / a.from.max_pages), p = (int)(i - (int64_t)s * a.from.max_pages), page = a.from.table[s * a.from.table_stride + p];
            a.table_out[s * a.table_out_stride + p] = in_pool(a.from, page) ? a.map[page] : -1;
        }
    }
    const int count = a.moves.count ? min(*a.moves.count, a.n) : a.n;
    const int64_t xs = a.from.entry_stride * a.esz, ys = a.to.entry_stride * a.esz;
    const int64_t items = (int64_t)count * a.batches;
    for (int64_t u = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); u < items; u += (int64_t)gridDim.x * 4) {
        const int m = __builtin_amdgcn_readfirstlane((int)(u / a.batches)), batch = __builtin_amdgcn_readfirstlane((int)(u - (int64_t)m * a.batches));
        Move mv = {-1, -1, a.from.page_size};
        if (a.moves.count) mv = a.moves.move[m];
        else { mv.from = a.src[m]; mv.to = a.dst[m]; }
        if (!in_pool(a.from, mv.from) || !in_pool(a.to, mv.to)) continue;
        // pieces of a head's entries; the batch's first head and its place in it
        const int per = mv.n * a.pieces.d;
        const int64_t head0 = (int64_t)batch * kBatch / per;         // (of a page of 2^30 pieces a part can be one: up to 2^39)
        if (head0 >= a.units.d) continue;
        const int unit0 = (int)head0, left = a.units.d - unit0, at0 = (int)((int64_t)batch * kBatch - head0 * per);
        const int64_t x0 = mv.from * a.from.page_stride, y0 = mv.to * a.to.page_stride;
        auto head_at = [&](int unit, const char*& from, char*& to) {
            const int lk = unit / a.heads, head = unit - lk * a.heads.d;
            from = ((lk & 1) ? a.from.v : a.from.k) + (lk >> 1) * a.from_layer + (x0 + head * a.from.head_stride) * a.esz;
            to = ((lk & 1) ? a.to.v : a.to.k) + (lk >> 1) * a.to_layer + (y0 + head * a.to.head_stride) * a.esz;
        };
        v4u w[8];
        if (at0 + kBatch <= per) {       // all of one head
            const char* from;
            char* to;
            head_at(unit0, from, to);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int i = at0 + lane + 64 * j, e = i / a.pieces, p = (i - e * a.pieces.d) * 16;
                w[j] = *reinterpret_cast<const v4u*>(from + e * xs + p);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int i = at0 + lane + 64 * j, e = i / a.pieces, p = (i - e * a.pieces.d) * 16;
                *reinterpret_cast<v4u*>(to + e * ys + p) = w[j];
            }
            continue;
        }
        // at0 + 511 < per + 512: the quotients by per are 0 and 1, or of numbers below 1024 and exact by 2^20 / per rounded up
        const unsigned magic = per < kBatch ? ((1u << 20) + per - 1u) / (unsigned)per : 0u;
        char* to[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = at0 + lane + 64 * j, q = per < kBatch ? (int)(((unsigned)i * magic) >> 20) : (i >= per ? 1 : 0);
            to[j] = nullptr;
            if (q < left) {
                const int k = i - q * per, e = k / a.pieces, p = (k - e * a.pieces.d) * 16;
                const char* from;
                head_at(unit0 + q, from, to[j]);
                to[j] += e * ys + p;
                w[j] = *reinterpret_cast<const v4u*>(from + e * xs + p);
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (to[j]) *reinterpret_cast<v4u*>(to[j]) = w[j];
    }
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
int status() { return hipGetLastError() == hipSuccess ? HAWK_OK : HAWK_EDEVICE; }
size_t round16(size_t n) { return (n + 15) / 16 * 16; }

// Lookups go through the counts in rounds of kWide * kEach: numbers of a round that begins behind the last page are still below 2^31.
constexpr int kMostPages = 0x7FFFFFFF - (2 * kWide * kEach - 1);
// A cache whose pages can be copied in all layers.
bool whole_view(const hawk_paged_cache* c, PagedView* v) {
    return paged_view(c, 0, v) && c->n_pages <= kMostPages && !(c->n_layers > 1 && c->layer_stride < c->head_dim) && (int64_t)c->n_layers * 2 * c->n_heads <= (1 << 25) &&
           (int64_t)c->page_size * (c->head_dim * (int)type_bytes(c->dtype) / 16) <= (1 << 30) && (int64_t)c->n_seq * c->max_pages <= (1 << 30) &&
           (int64_t)c->page_size * (c->head_dim * (int)type_bytes(c->dtype) / 16) * c->n_layers * 2 * c->n_heads <= (int64_t)kBatch << 30;
}
void copy_sides(const hawk_paged_cache* from, const hawk_paged_cache* to, CopyArgs* a) {
    a->esz = (int)type_bytes(from->dtype);
    a->from_layer = from->layer_stride * a->esz;
    a->to_layer = to->layer_stride * a->esz;
    a->units = divisor(from->n_layers * 2 * from->n_heads);
    a->heads = divisor(from->n_heads);
    a->pieces = divisor(from->head_dim * a->esz / 16);
    a->batches = ((int64_t)from->page_size * a->pieces.d * a->units.d + kBatch - 1) / kBatch;
}
void launch_copy(const CopyArgs& a, int64_t most, int waves_most, hipStream_t stream) {   // most: batches there can be
    const int64_t waves = std::min<int64_t>(waves_most, std::max<int64_t>(most, 1));
    paged_copy_kernel<<<(unsigned)((waves + 3) / 4), 256, 0, stream>>>(a);
}

// The workspace: a count, the moves, two lists of pages and where each page goes.
struct Room { int* count; Move* move; int *a, *b, *to; size_t bytes; };
Room room_of(const hawk_paged_cache* c, void* at) {
    Room r;
    char* p = static_cast<char*>(at);
    const size_t moves = round16(sizeof(Move) * (size_t)std::max(c->n_seq, c->n_pages / 2 + 1)), list = round16(sizeof(int) * (size_t)c->n_pages);
    r.count = reinterpret_cast<int*>(p);
    r.move = reinterpret_cast<Move*>(p + 16);
    r.a = reinterpret_cast<int*>(p + 16 + moves);
    r.b = reinterpret_cast<int*>(p + 16 + moves + list);
    r.to = reinterpret_cast<int*>(p + 16 + moves + 2 * list);
    r.bytes = 16 + moves + 3 * list;
    return r;
}

}  // namespace

size_t paged_pages_workspace_bytes(const hawk_paged_cache* cache) {
    PagedView v;
    return whole_view(cache, &v) ? room_of(cache, nullptr).bytes : 0;
}

int launch_paged_fork(const hawk_paged_cache* cache, int32_t* refs, int32_t* n_past, const int32_t* src, const int32_t* dst, int n, hipStream_t stream) {
    PagedView c;
    if (!paged_view(cache, 0, &c) || n < 0 || n > c.n_seq) return HAWK_EINVAL;
    if (n == 0) return HAWK_OK;
    if (!refs || !n_past || !src || !dst || n > kMostPairs) return HAWK_EINVAL;
    paged_fork_kernel<<<(unsigned)n, 256, 0, stream>>>(c, const_cast<int32_t*>(c.table), refs, n_past, src, dst, n);
    return status();
}

int launch_paged_trim(const hawk_paged_cache* cache, int32_t* refs, const int32_t* n_past, hipStream_t stream) {
    PagedView c;
    if (!paged_view(cache, 0, &c)) return HAWK_EINVAL;
    if (c.n_seq == 0) return HAWK_OK;
    if (!refs || !n_past) return HAWK_EINVAL;
    const int64_t blocks = (c.max_pages + 255) / 256;
    if (blocks * c.n_seq > (1 << 23)) return HAWK_EINVAL;
    paged_trim_kernel<<<(unsigned)(blocks * c.n_seq), 256, 0, stream>>>(c, const_cast<int32_t*>(c.table), refs, n_past, divisor((int)blocks));
    return status();
}

int launch_paged_take(const hawk_paged_cache* cache, int32_t* refs, const int32_t* n_past, const int32_t* n_new, int32_t* short_by, void* workspace,
                      size_t workspace_bytes, hipStream_t stream) {
    TakeArgs a = {};
    if (!whole_view(cache, &a.c)) return HAWK_EINVAL;
    if (a.c.n_seq == 0) return HAWK_OK;
    if (!refs || !n_past || !n_new || !short_by || !workspace || !aligned16(workspace)) return HAWK_EINVAL;
    const Room r = room_of(cache, workspace);
    if (workspace_bytes < r.bytes) return HAWK_ENOMEM;
    a.table = const_cast<int32_t*>(a.c.table);
    a.refs = refs; a.n_past = n_past; a.n_new = n_new; a.short_by = short_by;
    a.free = r.a; a.old = r.b;
    a.moves = {r.count, r.move};
    while (a.lanes < 6 && (int64_t)a.c.n_seq << (a.lanes + 1) <= kWide) ++a.lanes;
    paged_take_kernel<<<1, kWide, 0, stream>>>(a);
    CopyArgs m = {};
    m.from = m.to = a.c;
    m.moves = a.moves;
    m.n = a.c.n_seq;
    copy_sides(cache, cache, &m);
    launch_copy(m, m.n * m.batches, kPartWaves, stream);
    return status();
}

int launch_paged_compact(const hawk_paged_cache* cache, const int32_t* refs, int32_t* table_out, int64_t table_out_stride, int32_t* refs_out,
                         int32_t* n_used, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    CopyArgs m = {};
    if (!whole_view(cache, &m.from) || !refs || !refs_out || !n_used || !workspace || !aligned16(workspace)) return HAWK_EINVAL;
    if (m.from.n_seq > 0 && (!table_out || table_out_stride < m.from.max_pages)) return HAWK_EINVAL;
    // in place every thread writes what it has read itself; what lies over the old table or counts in any other way would be written before it is read
    const bool same_table = table_out == cache->table && (m.from.n_seq < 2 || table_out_stride == cache->table_stride);
    if (!same_table && rows_meet(cache->table, cache->table_stride * 4, cache->max_pages * 4ll, table_out, table_out_stride * 4, cache->max_pages * 4ll, cache->n_seq))
        return HAWK_EINVAL;
    if (refs_out != refs && rows_meet(refs, 0, cache->n_pages * 4ll, refs_out, 0, cache->n_pages * 4ll, 1)) return HAWK_EINVAL;
    const Room r = room_of(cache, workspace);
    if (workspace_bytes < r.bytes) return HAWK_ENOMEM;
    m.to = m.from;
    m.moves = {r.count, r.move};
    m.n = m.from.n_pages / 2;
    m.map = r.to;
    m.table_out = table_out;
    m.table_out_stride = table_out_stride;
    m.places = (int64_t)m.from.n_seq * m.from.max_pages;
    copy_sides(cache, cache, &m);
    paged_holes_kernel<<<1, kWide, 0, stream>>>(m.from, refs, refs_out, r.to, r.a, r.b, m.moves, n_used);
    launch_copy(m, std::max<int64_t>(m.n * m.batches, (m.places + 63) / 64), kPageWaves, stream);
    return status();
}

int launch_paged_copy(const hawk_paged_cache* from, const hawk_paged_cache* to, const int32_t* src, const int32_t* dst, int n, hipStream_t stream) {
    CopyArgs m = {};
    if (!whole_view(from, &m.from) || !whole_view(to, &m.to) || n < 0 || n > (1 << 20)) return HAWK_EINVAL;
    if (from->dtype != to->dtype || from->n_layers != to->n_layers || from->page_size != to->page_size || from->n_heads != to->n_heads ||
        from->head_dim != to->head_dim)
        return HAWK_EINVAL;
    if (n == 0) return HAWK_OK;
    if (!src || !dst) return HAWK_EINVAL;
    m.src = src; m.dst = dst; m.n = n;
    copy_sides(from, to, &m);
    launch_copy(m, n * m.batches, kPageWaves, stream);
    return status();
}

}  // namespace hawk
