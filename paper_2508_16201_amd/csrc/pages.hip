// specvlm_pages_assign and specvlm_pages_copy: which pages every request holds, and rows moved between pages.
//
// Assignment.  Every row of the new table goes on from a prefix of a row of the old one.  Whole pages of the prefix
// are shared.  The page that it ends in is written next: it stays with one row, the lowest that goes on in it, if no row
// holds it as a whole page; the others get a page of their own, with rows to copy into it.  With  whole/first(page) =
// minimum over the rows that keep it of (-1 if it is a whole page there, else the row),  row b keeps its page iff first == b.
// (A row whose prefix ends in an entry that is no page needs one there too, with nothing to copy.)
// Free pages (kept by no row) go out lowest first to the lowest rows first: page of rank r to the row whose prefix sum of needs
// holds r.  Everything is a sum, a minimum or a prefix sum of integers: the order of the atomics does not matter.
// Bound: launches and round trips (one launch where a workgroup can do it, else four: clear, mark, plan, write).
//
// Copy.  Bound by HBM: 16 bytes a lane and row, several rows in flight.  Where source and destination are one pool the rows of a
// request may lie in each other's way: a workgroup then has its columns of all the request's rows, and reads a run of them before
// it writes it, which is right as long as no row moves up.
#include "common.h"

#include <climits>

namespace specvlm {

struct AssignParams {
    const int32_t* old_table;
    int64_t old_row;
    const int32_t *parent, *keep_len, *new_len;
    int32_t* table;
    int64_t row;
    int32_t *copy_start, *copy_rows, *ref_counts, *status;
    int32_t *first, *start, *block_free;        // workspace: [n_pages], [batch + 1], [blocks of pages + 1]
    int batch, n_old, old_pages, max_pages, n_pages, page_size, window, n_sinks;
    uint32_t inv_page;
    int n_blocks;
    int row_chunks;
};

constexpr int kAssignThreads = 256;
constexpr int kPlanThreads = 1024;
constexpr int kPageBlock = 1024;                 // pages of a block, whose free ones are counted together
// What one workgroup takes: a wave goes over a row, 64 entries at a time, and over every sixteenth row.  Us a call, four launches / one, by
// rows, pages a row, pages of the pool:  1 x 100 of 1000 8.1 / 4.0;  8 x 129 of 4096 11.0 / 6.1;  16 x 500 of 6100 11.9 / 8.5;  32 x 240 of 6100 12.0 /
// 9.1;  128 x 40 of 6100 12.8 / 12.5;  8 x 800 of 8100 11.6 / 11.6;  but 64 x 250 of 12200 12.9 / 16.3, 120 x 16 of 12200 13.1 / 17.1, 64 x 100 of 8100 12.3 /
// 13.0, 250 x 48 of 15200 13.9 / 25.3.
constexpr int kSmallPages = 8192, kSmallTrips = 8, kSmallRows = kSmallTrips * kPlanThreads / kWave;

// A row of the new table: pages [0, whole) whole, one more if `part`; pages [0, wanted) in the end.
struct AssignRow { int parent, keep, whole, kept, wanted; bool valid; };
__device__ __forceinline__ AssignRow assign_row(const AssignParams& p, int b)
{
    AssignRow r;
    r.parent = p.parent[b]; r.keep = p.keep_len[b];
    const int n = p.new_len[b];
    // (lengths are compared in pages: a product with the page size might not fit)
    r.valid = r.parent >= -1 && r.parent < p.n_old && r.keep >= 0 && r.keep <= n && (r.keep == 0 || r.parent >= 0);
    const QuotRem k = divide(r.valid ? r.keep : 0, p.page_size, p.inv_page), w = divide(r.valid ? n : 0, p.page_size, p.inv_page);
    r.whole = k.q; r.kept = k.q + (k.r > 0); r.wanted = w.q + (w.r > 0);
    r.valid = r.valid && r.kept <= p.old_pages && r.wanted <= p.max_pages;
    if (!r.valid) r.whole = r.kept = r.wanted = 0;
    return r;
}
// Page i of the prefix, or -1: none of the pool's, or hidden for good by the window.
__device__ __forceinline__ int assign_page(const AssignParams& p, const AssignRow& r, int i)
{
    const int id = p.old_table[(int64_t)r.parent * p.old_row + i];
    if (p.window > 0) {
        const int64_t begin = (int64_t)i * p.page_size, end = begin + p.page_size;
        if (end <= (int64_t)r.keep - p.window + 1 && begin >= p.n_sinks) return -1;
    }
    return (uint32_t)id < (uint32_t)p.n_pages ? id : -1;
}
// Whether row b goes on in another page than the one that its prefix ends in (`page`), and whether it needs one.
__device__ __forceinline__ bool assign_leaves(const AssignParams& p, int page, int b) { return page >= 0 && p.first[page] != b; }

__global__ __launch_bounds__(kAssignThreads)
void assign_clear_kernel(const AssignParams p)
{
    const int i = blockIdx.x * kAssignThreads + threadIdx.x;
    if (i >= p.n_pages) return;
    p.ref_counts[i] = 0;
    if (p.batch) p.first[i] = INT_MAX;                // (no rows: no workspace)
}

__global__ __launch_bounds__(kAssignThreads)
void assign_mark_kernel(const AssignParams p)
{
    const int b = blockIdx.x / p.row_chunks, i = (blockIdx.x % p.row_chunks) * kAssignThreads + threadIdx.x;
    const AssignRow r = assign_row(p, b);
    if (i >= r.kept) return;
    const int page = assign_page(p, r, i);
    if (page < 0) return;
    atomicAdd(p.ref_counts + page, 1);
    atomicMin(p.first + page, i < r.whole ? -1 : b);
}

// Prefix sums over the workgroup's threads: what is before the thread's x and y, and the totals.
struct Pair { int x, y; };
template <int THREADS>
__device__ __forceinline__ Pair block_before(Pair v, Pair* total, Pair* s_wave)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Pair upto = {wave_prefix(v.x), wave_prefix(v.y)};
    __syncthreads();
    if (lane == kWave - 1) s_wave[wave] = upto;
    __syncthreads();
    Pair before = {upto.x - v.x, upto.y - v.y}, all = {0, 0};
#pragma unroll
    for (int i = 0; i < THREADS / kWave; ++i) {
        const Pair w = s_wave[i];
        if (i < wave) { before.x += w.x; before.y += w.y; }
        all.x += w.x; all.y += w.y;
    }
    *total = all;
    return before;
}

// Free pages of every block; the last workgroup has the rows: what each needs, and the sum of the needs before it.
__global__ __launch_bounds__(kAssignThreads)
void assign_plan_kernel(const AssignParams p)
{
    __shared__ Pair s_wave[kAssignThreads / kWave];
    if ((int)blockIdx.x < p.n_blocks) {
        int n = 0;
        Pair all;
#pragma unroll
        for (int i = 0; i < kPageBlock / kAssignThreads; ++i) {
            const int page = blockIdx.x * kPageBlock + i * kAssignThreads + threadIdx.x;
            n += page < p.n_pages && p.ref_counts[page] == 0;
        }
        block_before<kAssignThreads>({n, 0}, &all, s_wave);
        if (threadIdx.x == 0) p.block_free[blockIdx.x] = all.x;
        return;
    }
    int needed = 0;
    for (int base = 0; base < p.batch; base += kAssignThreads) {
        const int b = base + threadIdx.x;
        int need = 0;
        Pair all;
        if (b < p.batch) {
            const AssignRow r = assign_row(p, b);
            const int page = r.kept > r.whole ? assign_page(p, r, r.whole) : -1;
            need = r.wanted - (page >= 0 && !assign_leaves(p, page, b) ? r.kept : r.whole);
        }
        const int before = needed + block_before<kAssignThreads>({need, 0}, &all, s_wave).x;
        needed += all.x;
        if (b < p.batch) p.start[b] = before;
    }
    if (threadIdx.x == 0) p.start[p.batch] = needed;
}

// What the plan says of a row.
__device__ __forceinline__ void assign_tell(const AssignParams& p, const AssignRow& r, int b, bool leaves, bool fits)
{
    const bool copies = leaves && fits;
    p.status[b] = !r.valid ? SPECVLM_EINVAL : fits ? SPECVLM_OK : SPECVLM_ENOPAGES;
    p.copy_start[b] = copies ? r.whole * p.page_size : 0;
    p.copy_rows[b] = copies ? r.keep - r.whole * p.page_size : 0;
}
// The row that gets the free page of this rank: the last that starts at or before it.
__device__ __forceinline__ int assign_owner(const int32_t* start, int batch, int rank)
{
    int lo = 0, hi = batch;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= rank) lo = mid; else hi = mid;
    }
    return lo;
}

// The first workgroups hand out the free pages of a block each, the others write what the rows keep.
__global__ __launch_bounds__(kAssignThreads)
void assign_write_kernel(const AssignParams p)
{
    __shared__ Pair s_wave[kAssignThreads / kWave];
    const bool hands_out = (int)blockIdx.x < p.n_blocks;
    // free pages: all of them, and those of the blocks before (each wave for itself: no barrier)
    int before = 0, free = 0;
    for (int i = threadIdx.x & 63; i < p.n_blocks; i += kWave) {
        const int f = p.block_free[i];
        free += f;
        before += i < (int)blockIdx.x ? f : 0;
    }
    free = wave_total(free); before = wave_total(before);
    if (hands_out) {
        constexpr int EACH = kPageBlock / kAssignThreads;
        const int needed = p.start[p.batch];
        if (before >= needed) return;
        const int page0 = blockIdx.x * kPageBlock + threadIdx.x * EACH;
        bool is_free[EACH];
        int n = 0;
        Pair all;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            is_free[i] = page0 + i < p.n_pages && p.ref_counts[page0 + i] == 0;
            n += is_free[i];
        }
        int rank = before + block_before<kAssignThreads>({n, 0}, &all, s_wave).x;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            if (!is_free[i] || rank >= needed) continue;
            const int b = assign_owner(p.start, p.batch, rank), first = p.start[b], need = p.start[b + 1] - first;
            if (first + need <= free) {
                p.table[(int64_t)b * p.row + assign_row(p, b).wanted - need + rank - first] = page0 + i;
                p.ref_counts[page0 + i] = 1;
            }
            ++rank;
        }
        return;
    }
    const int w = blockIdx.x - p.n_blocks, b = w / p.row_chunks, i = (w % p.row_chunks) * kAssignThreads + threadIdx.x;
    const AssignRow r = assign_row(p, b);
    const int need = p.start[b + 1] - p.start[b];
    const bool fits = need == 0 || p.start[b] + need <= free;
    if (w % p.row_chunks == 0 && threadIdx.x == 0) {
        const int page = r.kept > r.whole ? assign_page(p, r, r.whole) : -1;
        const bool leaves = assign_leaves(p, page, b);
        if (leaves) atomicSub(p.ref_counts + page, 1);
        assign_tell(p, r, b, leaves, fits);
    }
    if (i >= p.max_pages) return;
    const bool handed_out = i >= r.wanted - need && i < r.wanted;
    if (handed_out && fits) return;
    p.table[(int64_t)b * p.row + i] = i < r.kept && !handed_out ? assign_page(p, r, i) : -1;
}

// All of it in one workgroup, with the counts in LDS (bound: its round trips; kSmallPages has both sides' times).
__global__ __launch_bounds__(kPlanThreads)
void assign_small_kernel(const AssignParams p)
{
    extern __shared__ int s_all[];
    int* const refs = s_all;                          // [n_pages]
    int* const first = refs + p.n_pages;              // [n_pages]
    int* const start = first + p.n_pages;             // [batch + 1]
    __shared__ Pair s_wave[kPlanThreads / kWave];
    __shared__ AssignRow s_row[kSmallRows];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    constexpr int WAVES = kPlanThreads / kWave;
    AssignRow mine = {};
    if (tid < p.batch) s_row[tid] = mine = assign_row(p, tid);
    for (int i = tid; i < p.n_pages; i += kPlanThreads) { refs[i] = 0; first[i] = INT_MAX; }
    __syncthreads();
    for (int b = wave; b < p.batch; b += WAVES) {
        const AssignRow r = s_row[b];
        for (int i = lane; i < r.kept; i += kWave) {
            const int page = assign_page(p, r, i);
            if (page < 0) continue;
            atomicAdd(refs + page, 1);
            atomicMin(first + page, i < r.whole ? -1 : b);
        }
    }
    __syncthreads();
    // the rows' needs; the free pages of this thread's share of the pool
    const int each = (p.n_pages + kPlanThreads - 1) / kPlanThreads, page0 = min(tid * each, p.n_pages), page1 = min(page0 + each, p.n_pages);
    int n = 0, need = 0, page = -1;
    for (int i = page0; i < page1; ++i) n += refs[i] == 0;
    if (mine.kept > mine.whole) page = assign_page(p, mine, mine.whole);
    const bool leaves = page >= 0 && first[page] != tid;
    need = mine.wanted - (page >= 0 && !leaves ? mine.kept : mine.whole);
    Pair all;
    const Pair sums = block_before<kPlanThreads>({n, need}, &all, s_wave);
    const int before = sums.y, free = all.x, needed = all.y;
    int rank = sums.x;
    if (tid < p.batch) start[tid] = before;
    if (tid == 0) start[p.batch] = needed;
    __syncthreads();
    if (tid < p.batch) assign_tell(p, mine, tid, leaves, need == 0 || before + need <= free);
    for (int i = page0; i < page1 && rank < needed; ++i) {
        if (refs[i] != 0) continue;
        const int b = assign_owner(start, p.batch, rank), begin = start[b], wants = start[b + 1] - begin;
        if (begin + wants <= free) {
            p.table[(int64_t)b * p.row + s_row[b].wanted - wants + rank - begin] = i;
            refs[i] = 1;                              // (nobody else looks at this page any more)
        }
        ++rank;
    }
    for (int b = wave; b < p.batch; b += WAVES) {
        const AssignRow r = s_row[b];
        const int wants = start[b + 1] - start[b];
        const bool fits = wants == 0 || start[b] + wants <= free;
        for (int i = lane; i < p.max_pages; i += kWave) {
            const bool handed_out = i >= r.wanted - wants && i < r.wanted;
            if (!(handed_out && fits)) p.table[(int64_t)b * p.row + i] = i < r.kept && !handed_out ? assign_page(p, r, i) : -1;
        }
    }
    if (leaves) atomicSub(refs + page, 1);
    __syncthreads();
    for (int i = tid; i < p.n_pages; i += kPlanThreads) p.ref_counts[i] = refs[i];
}

// ------------------------------------------------------------------------------------------------------- copy ----
struct CopySide { int64_t layer, page, tok, head; const int32_t* table; int64_t row; int n_pages, page_size, max_pages; uint32_t inv_page; };
struct CopyParams {
    const __bf16 *k_src, *v_src;
    __bf16 *k_dst, *v_dst;
    CopySide src, dst;
    const int32_t *src_row, *n_rows, *src_start, *dst_start, *row_idx, *cu_idx;
    int64_t idx_stride;
    int max_rows, n_table_rows, n_layers, batch, n_mats;
    int pieces, head_pieces, slice, slices, row_blocks;      // 16-byte pieces of a row, of a head, of a workgroup; workgroups that share a row; workgroups over the rows
    uint32_t inv_head;
};

constexpr int kCopyThreads = 256;
constexpr int kCopyEach = 2;
constexpr int kCopyTarget = 128 * kNumCu;       // workgroups of a launch
constexpr int64_t kCopyStreamBytes = 64 << 20;  // from this size on a copy is not kept near (the caches that it would fill hold 4 and 256 MB)

// The page of a token, and whether there may be one (else the first entry is read for nothing: no branch between the lookups).
struct CopyToken { int column, row; bool in; };
__device__ __forceinline__ CopyToken copy_token(const CopySide& s, int64_t token)
{
    CopyToken t;
    t.in = token >= 0 && token <= INT_MAX;
    const QuotRem at = divide(t.in ? (int)token : 0, s.page_size, s.inv_page);
    t.in = t.in && at.q < s.max_pages;
    t.column = t.in ? at.q : 0;
    t.row = at.r;
    return t;
}

// EACH rows of a thread at once; their places are looked up once and serve every layer of K and V that the workgroup has.
// IN_PLACE: a workgroup goes over all rows of its request, in order.  STREAM: what is copied is not kept near.
//   1254 rows of 2 KB in 80 layers (822 MB):  kept near 168 us, not 141;  four rows of a thread 6 us more, 32 workgroups to a CU, with more
//   layers each, 2 us more, 128 and none that share a lookup 50 us more.
//   32 pages of 1 to 63 rows of 1 KB in 28 layers, in place:  stores kept near 38 us, not 28 (and loads that are not 35: forks of one row read
//   one page);  a workgroup with whole rows, one run after the other, 31.6 us, with 16 pieces of each 25.1;  up to 5 rows in 28 layers of 8 requests
//   3.5 us, with four rows of a thread 3.9.
template <bool IN_PLACE, bool STREAM>
__global__ __launch_bounds__(kCopyThreads)
void pages_copy_kernel(const CopyParams p)
{
    constexpr int EACH = kCopyEach;
    const int b = blockIdx.y;
    const int slice = blockIdx.x % p.slices, block = blockIdx.x / p.slices;
    const int first = p.cu_idx ? p.cu_idx[b] : 0;
    int n = p.max_rows;
    if (p.cu_idx) n = min(n, p.cu_idx[b + 1] - first);
    if (p.n_rows) n = min(n, p.n_rows[b]);
    // the lanes lie over the pieces of a row, several rows at once where a row is short
    const int per_row = p.slice, rows = kCopyThreads / per_row, step = rows * EACH;
    if (block * step >= n) return;
    const int from = p.src_row ? p.src_row[b] : b;
    const bool there = from >= 0 && from < p.n_table_rows && p.src.max_pages > 0;
    const int32_t* const src_table = p.src.table + (there ? from : 0) * p.src.row;
    const int32_t* const dst_table = p.dst.table + b * p.dst.row;
    const int32_t* const idx = p.row_idx ? p.row_idx + (p.cu_idx ? (int64_t)first : b * p.idx_stride) : nullptr;
    const int64_t src0 = p.src_start ? p.src_start[b] : 0, dst0 = p.dst_start ? p.dst_start[b] : 0;
    const int lane_row = threadIdx.x / per_row, piece = slice * per_row + threadIdx.x % per_row;
    const bool on = lane_row < rows && piece < p.pieces && p.dst.max_pages > 0;
    const QuotRem at = divide(piece, p.head_pieces, p.inv_head);
    for (int i0 = block * step; i0 < n; i0 += IN_PLACE ? step : step * p.row_blocks) {
        int64_t to[EACH], of[EACH];                   // elements into a layer; -1: no such row
        int token[EACH];
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int i = min(i0 + e * rows + lane_row, n - 1);
            token[e] = i;
            if (idx && i0 + e * rows < n) token[e] = idx[i];
        }
        CopyToken s[EACH], d[EACH];
        int s_id[EACH], d_id[EACH];
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            s[e] = copy_token(p.src, src0 + token[e]);
            d[e] = copy_token(p.dst, dst0 + i0 + e * rows + lane_row);
            s_id[e] = d_id[e] = -1;
            if (i0 + e * rows < n) {
                if (there) s_id[e] = src_table[s[e].column];
                if (on) d_id[e] = dst_table[d[e].column];
            }
        }
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const bool live = on && i0 + e * rows + lane_row < n && d[e].in && (uint32_t)d_id[e] < (uint32_t)p.dst.n_pages;
            to[e] = live ? d_id[e] * p.dst.page + d[e].row * p.dst.tok + at.q * p.dst.head + at.r * 8 : -1;
            of[e] = live && s[e].in && (uint32_t)s_id[e] < (uint32_t)p.src.n_pages
                        ? s_id[e] * p.src.page + s[e].row * p.src.tok + at.q * p.src.head + at.r * 8 : -1;
        }
        for (int z = blockIdx.z; z < p.n_layers * p.n_mats; z += gridDim.z) {
            const int layer = p.n_mats == 2 ? z >> 1 : z;
            const bool is_v = p.n_mats == 2 && (z & 1);
            const __bf16* const src = (is_v ? p.v_src : p.k_src) + layer * p.src.layer;
            __bf16* const dst = (is_v ? p.v_dst : p.k_dst) + layer * p.dst.layer;
            u32x4 x[EACH];
#pragma unroll
            for (int e = 0; e < EACH; ++e) {
                x[e] = u32x4{0u, 0u, 0u, 0u};
                if (of[e] >= 0) {
                    if constexpr (STREAM && !IN_PLACE) x[e] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + of[e]));
                    else x[e] = *reinterpret_cast<const u32x4*>(src + of[e]);
                }
            }
            if constexpr (IN_PLACE) __syncthreads();
#pragma unroll
            for (int e = 0; e < EACH; ++e)
                if (to[e] >= 0) {
                    if constexpr (STREAM) __builtin_nontemporal_store(x[e], reinterpret_cast<u32x4*>(dst + to[e]));
                    else *reinterpret_cast<u32x4*>(dst + to[e]) = x[e];
                }
        }
        if constexpr (IN_PLACE) __syncthreads();
    }
}

template <bool IN_PLACE, bool STREAM>
static int launch_copy(CopyParams& p, hipStream_t stream)
{
    p.slice = p.pieces < kCopyThreads ? p.pieces : kCopyThreads;
    // in place a workgroup goes over its rows one run after the other: columns are shared out until a run has all of them, or is one of 16 pieces
    while (IN_PLACE && p.slice > 16 && kCopyThreads / p.slice * kCopyEach < p.max_rows) p.slice = p.slice / 2 > 16 ? p.slice / 2 : 16;
    p.slices = (p.pieces + p.slice - 1) / p.slice;
    const int step = kCopyThreads / p.slice * kCopyEach;
    p.row_blocks = IN_PLACE ? 1 : (p.max_rows + step - 1) / step;
    if (!launchable((int64_t)p.row_blocks * p.slices, kCopyThreads)) return SPECVLM_EUNSUPPORTED;
    // layers of K and V that share a workgroup, and its lookups: as many as leave workgroups enough
    const int64_t each = (int64_t)p.row_blocks * p.slices * p.batch;
    int64_t z = (kCopyTarget + each - 1) / each;
    if (z > p.n_layers * p.n_mats) z = p.n_layers * p.n_mats;
    hipLaunchKernelGGL((pages_copy_kernel<IN_PLACE, STREAM>), dim3(p.row_blocks * p.slices, p.batch, (int)z), dim3(kCopyThreads), 0, stream, p);
    return launch_status();
}

}  // namespace specvlm

using namespace specvlm;

// Whether two tables have a byte in common (columns of one table, cut side by side, have none).
static bool tables_overlap(const int32_t* a, int64_t a_stride, int a_rows, int a_width, const int32_t* b, int64_t b_stride, int b_rows, int b_width)
{
    if (a_rows == 0 || a_width == 0 || b_rows == 0 || b_width == 0) return false;
    const int64_t from_a = ((int64_t)(uintptr_t)b - (int64_t)(uintptr_t)a) / (int64_t)sizeof(int32_t);
    if (from_a >= (a_rows - 1) * a_stride + a_width || -from_a >= (b_rows - 1) * b_stride + b_width) return false;
    if (a_stride != b_stride || a_stride <= 0 || (a_rows == 1 && b_rows == 1)) return true;
    const int64_t column = ((from_a % a_stride) + a_stride) % a_stride;
    return column < a_width || column + b_width > a_stride;
}

static int assign_blocks(int n_pages) { return (n_pages + kPageBlock - 1) / kPageBlock; }

extern "C" size_t specvlm_pages_assign_workspace_bytes(int batch, int n_pages)
{
    if (batch <= 0 || n_pages < 0) return 0;
    return align256(sizeof(int32_t) * (size_t)n_pages) + align256(sizeof(int32_t) * ((size_t)batch + 1)) +
           align256(sizeof(int32_t) * ((size_t)assign_blocks(n_pages) + 1));
}

extern "C" int specvlm_pages_assign(
    const int32_t* old_table, int64_t old_stride, int old_rows, int old_max_pages,
    const int32_t* parent, const int32_t* keep_len, const int32_t* new_len, int batch,
    int32_t* page_table, int64_t table_stride, int max_pages, int n_pages, int page_size, int window, int n_sinks,
    int32_t* copy_start, int32_t* copy_rows, int32_t* ref_counts, int32_t* status,
    void* workspace, size_t workspace_bytes, void* stream)
{
    if (old_rows < 0 || old_max_pages < 0 || batch < 0 || max_pages < 0 || n_pages < 0 || page_size <= 0 || window < 0 || n_sinks < 0 ||
        old_stride < 0)
        return SPECVLM_EINVAL;
    if (page_size % 16) return SPECVLM_EUNSUPPORTED;
    if (batch == 0) {                                 // (nobody holds a page)
        if (n_pages == 0) return SPECVLM_OK;
        if (!ref_counts) return SPECVLM_EINVAL;
        AssignParams p = {};
        p.ref_counts = ref_counts; p.n_pages = n_pages;
        hipLaunchKernelGGL(assign_clear_kernel, dim3((n_pages - 1) / kAssignThreads + 1), dim3(kAssignThreads), 0, (hipStream_t)stream, p);
        return launch_status();
    }
    if (!parent || !keep_len || !new_len || !copy_start || !copy_rows || !status || (!ref_counts && n_pages > 0)) return SPECVLM_EINVAL;
    if ((!old_table && old_rows > 0 && old_max_pages > 0) || (!page_table && max_pages > 0)) return SPECVLM_EINVAL;
    if (batch > 1 && table_stride < max_pages) return SPECVLM_EINVAL;                  // (rows that overlap)
    if (tables_overlap(old_table, old_stride, old_rows, old_max_pages, page_table, table_stride, batch, max_pages)) return SPECVLM_EINVAL;
    const int most = old_max_pages > max_pages ? old_max_pages : max_pages;
    const int chunks = most ? (most + kAssignThreads - 1) / kAssignThreads : 1;
    if ((int64_t)batch * max_pages > INT_MAX / 2 || !launchable((int64_t)batch * chunks + assign_blocks(n_pages), kAssignThreads)) return SPECVLM_EUNSUPPORTED;
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < specvlm_pages_assign_workspace_bytes(batch, n_pages)) return SPECVLM_EWORKSPACE;

    AssignParams p;
    p.old_table = old_table; p.old_row = old_stride; p.parent = parent; p.keep_len = keep_len; p.new_len = new_len;
    p.table = page_table; p.row = table_stride;
    p.copy_start = copy_start; p.copy_rows = copy_rows; p.ref_counts = ref_counts; p.status = status;
    p.first = (int32_t*)workspace;
    p.start = (int32_t*)((char*)p.first + align256(sizeof(int32_t) * (size_t)n_pages));
    p.block_free = (int32_t*)((char*)p.start + align256(sizeof(int32_t) * ((size_t)batch + 1)));
    p.batch = batch; p.n_old = old_rows; p.old_pages = old_max_pages; p.max_pages = max_pages;
    p.n_pages = n_pages; p.page_size = page_size; p.window = window; p.n_sinks = n_sinks;
    p.inv_page = reciprocal(page_size);
    p.n_blocks = assign_blocks(n_pages);
    p.row_chunks = chunks;
    hipStream_t s = (hipStream_t)stream;
    int rc;
    constexpr int kWaves = kPlanThreads / kWave;
    if (n_pages <= kSmallPages && batch <= kSmallRows && most <= kSmallTrips * kWave &&
        (batch + kWaves - 1) / kWaves * ((most + kWave - 1) / kWave) <= kSmallTrips) {
        constexpr int kMostLds = (2 * kSmallPages + kSmallRows + 1) * (int)sizeof(int);
        if ((rc = allow_lds<&assign_small_kernel>(kMostLds)) != SPECVLM_OK) return rc;
        hipLaunchKernelGGL(assign_small_kernel, dim3(1), dim3(kPlanThreads), (2 * n_pages + batch + 1) * sizeof(int), s, p);
        return launch_status();
    }
    if (n_pages) {
        hipLaunchKernelGGL(assign_clear_kernel, dim3((n_pages + kAssignThreads - 1) / kAssignThreads), dim3(kAssignThreads), 0, s, p);
        if ((rc = launch_status()) != SPECVLM_OK) return rc;
        hipLaunchKernelGGL(assign_mark_kernel, dim3(batch * chunks), dim3(kAssignThreads), 0, s, p);
        if ((rc = launch_status()) != SPECVLM_OK) return rc;
    }
    hipLaunchKernelGGL(assign_plan_kernel, dim3(p.n_blocks + 1), dim3(kAssignThreads), 0, s, p);
    if ((rc = launch_status()) != SPECVLM_OK) return rc;
    hipLaunchKernelGGL(assign_write_kernel, dim3(p.n_blocks + batch * chunks), dim3(kAssignThreads), 0, s, p);
    return launch_status();
}

extern "C" int specvlm_pages_copy(
    const void* k_src, const void* v_src, int64_t src_layer_stride, int64_t src_page_stride, int64_t src_tok_stride, int64_t src_head_stride,
    int src_pages, int src_page_size, const int32_t* src_table, int64_t src_table_stride, int src_rows, int src_max_pages,
    void* k_dst, void* v_dst, int64_t dst_layer_stride, int64_t dst_page_stride, int64_t dst_tok_stride, int64_t dst_head_stride,
    int dst_pages, int dst_page_size, const int32_t* dst_table, int64_t dst_table_stride, int dst_max_pages,
    int n_layers, int batch, const int32_t* n_rows, int max_rows, const int32_t* src_row, const int32_t* src_start,
    const int32_t* dst_start, const int32_t* row_idx, int64_t idx_stride, const int32_t* cu_idx,
    int n_kv_heads, int head_dim, void* stream)
{
    if (src_pages < 0 || src_rows < 0 || src_max_pages < 0 || dst_pages < 0 || dst_max_pages < 0 || src_page_size <= 0 || dst_page_size <= 0 ||
        n_layers < 0 || batch < 0 || max_rows < 0 || n_kv_heads <= 0 || src_table_stride < 0 || dst_table_stride < 0 || idx_stride < 0)
        return SPECVLM_EINVAL;
    if ((v_src == nullptr) != (v_dst == nullptr)) return SPECVLM_EINVAL;
    if (cu_idx && !row_idx) return SPECVLM_EINVAL;
    if ((head_dim != 64 && head_dim != 128) || src_page_size % 16 || dst_page_size % 16) return SPECVLM_EUNSUPPORTED;
    if (n_layers == 0 || batch == 0 || max_rows == 0) return SPECVLM_OK;
    if (!k_src || !k_dst || !src_table || !dst_table) return SPECVLM_EINVAL;
    if (!src_row && src_rows < batch) return SPECVLM_EINVAL;
    const int64_t strides = src_layer_stride | src_page_stride | src_tok_stride | src_head_stride | dst_layer_stride | dst_page_stride |
                            dst_tok_stride | dst_head_stride;
    if ((strides & 7) || (((uintptr_t)k_src | (uintptr_t)v_src | (uintptr_t)k_dst | (uintptr_t)v_dst) & 15)) return SPECVLM_EUNSUPPORTED;
    const int mats = v_src ? 2 : 1;
    if (batch > 65535 || (int64_t)n_layers * mats > 65535 || n_kv_heads > (1 << 20) || max_rows > (1 << 30)) return SPECVLM_EUNSUPPORTED;

    CopyParams p;
    p.k_src = (const __bf16*)k_src; p.v_src = (const __bf16*)v_src; p.k_dst = (__bf16*)k_dst; p.v_dst = (__bf16*)v_dst;
    p.src = {src_layer_stride, src_page_stride, src_tok_stride, src_head_stride, src_table, src_table_stride, src_pages, src_page_size,
             src_max_pages, reciprocal(src_page_size)};
    p.dst = {dst_layer_stride, dst_page_stride, dst_tok_stride, dst_head_stride, dst_table, dst_table_stride, dst_pages, dst_page_size,
             dst_max_pages, reciprocal(dst_page_size)};
    p.src_row = src_row; p.n_rows = n_rows; p.src_start = src_start; p.dst_start = dst_start; p.row_idx = row_idx; p.cu_idx = cu_idx;
    p.idx_stride = idx_stride; p.max_rows = max_rows; p.n_table_rows = src_rows; p.n_layers = n_layers; p.batch = batch; p.n_mats = mats;
    p.head_pieces = head_dim / 8; p.pieces = n_kv_heads * p.head_pieces;
    p.inv_head = reciprocal(p.head_pieces);
    const bool in_place = k_src == k_dst || (v_src && v_src == v_dst);
    hipStream_t s = (hipStream_t)stream;
    if (in_place) return launch_copy<true, true>(p, s);
    const bool large = 16.0 * p.pieces * max_rows * batch * n_layers * mats >= kCopyStreamBytes;
    return large ? launch_copy<false, true>(p, s) : launch_copy<false, false>(p, s);
}
