// specvlm_paged_attn: grouped-query softmax attention of a short query block (one token, a verified chain, a draft
// tree) over a bf16 KV cache held in pages, with every key visible or only the first ones and a window of the last.
//
// Mathematics.  One pass over the keys with the running maximum m and sum l of each query row (online softmax); the
// key range of a request is cut into pieces, and pieces are joined by  o = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s.
// All statistics, sums and partial outputs are fp32; the probabilities go through the matrix instruction as two bf16
// each (16 bits), the output is rounded once.
//
// Bound.  Every visible K and V row is read once for up to 64 query rows of a kv head: HBM for long caches, launches and
// round trips for short ones.  More rows than 64 are groups that read the keys again: 208 rows (trees of 26 nodes of 64/8 heads), cut into four, load
// 520 MB through the L2, which alone takes 52 of the 72 us (the fourth group has one of the 13 row blocks).
//
// Pages.  A page holds a multiple of 16 keys, so 16 consecutive keys starting at a multiple of 16 lie in one page and
// one scalar table lookup serves them: the address of a wave-wide load is a scalar base plus a lane offset that never
// changes.  The loader waves look up the pages of a tile one tile before they load it.  With a window the keys are
// swept in the order  first keys (rounded up to 16), then the window (rounded down to 16): the pages between are never
// looked at, and may have been freed.
//
// Work decomposition.  The lengths are on the device.  Tiles of 64 keys of all requests are numbered request after
// request; group j (a workgroup for each kv head and row group) takes a run of equal length, which every workgroup
// finds by a prefix sum over the lengths, 64 requests at a time in the lanes of a wave (paged_cut: where the runs begin).  A captured
// launch so stays balanced as the caches grow.  A request that one group covers is written out directly; the others leave partial
// results that the second launch joins.  Short caches take one launch: a workgroup has a request's keys of a head whole (paged_takes_whole has the
// line), and where those would be few workgroups a slice of its value columns (paged_short_kernel, paged_short_chunks).
//
// A workgroup has MB*KS compute waves (row block mb, every KS-th 32-key chunk of a tile) and NLD loader waves that only issue
// direct-to-LDS loads into a ring of NS tiles (see decode_attn.hip for the matrix formulation and the swizzles).  The two roles plan for
// themselves, each its own way to its first instruction that matters:  a launch's 6 us over one tile were mostly instructions that it met
// for the first time.
#include <type_traits>

#include "attn_tile.h"

namespace specvlm {

#define SPECVLM_AS4 __attribute__((address_space(4)))

struct PagedParams {
    const __bf16* q;
    const __bf16* k;
    const __bf16* v;
    __bf16* out;
    float* lse;
    int64_t q_tok, q_head, page, tok, head;      // strides in elements
    const int32_t* table;
    int64_t table_row;
    const int32_t* kv_lens;
    const int32_t* cu_q;
    const uint64_t* block_mask;
    int n_pages, page_size;
    int batch, q_len, kv_len, n_q_heads, n_kv_heads, group;
    int window, n_sinks;
    uint32_t inv_page, inv_heads, inv_all_heads, inv_group, inv_rgroups, inv_groups, inv_fold;
    float scale_log2;
    int n_rgroups, rows_pad, max_groups;
    int fold;                // kFold * batch
    int n_units;             // (paged_short_kernel) requests' kv heads' blocks of 16 rows
    int last_units;          // of them, what is left of the last eight (1 to 8)
    uint32_t inv_last;
    float* part_o;           // [(groups + batch) * H_kv][rows_pad][D] unnormalised partial outputs
    float* part_ml;          // [(groups + batch) * H_kv][rows_pad][2] running maximum in log2 units, sum
    int32_t* part_of;        // [batch][2] (of a batch) the first group that has a piece of the request, and how many have
};

// A lane's sum of one chunk at or above this (or NaN), against the maximum of earlier chunks, is done once more with the maximum tracked.  It bounds what a probability
// can grow to before its product with a value:  with 2^100 values of 2^28 went beyond 32 bits (a logit 62 above those before it is a probability of 2^89), though
// the sum does not.
constexpr float kPagedRedo = 0x1p20f;
constexpr int kTileKeys = 64;
constexpr int kRing = 3;                 // tiles of a ring (four: 0.4 us more a call, no faster for long caches)
// A group takes a tile or more: as many as the launch's workgroups need, and up to four where a request (of the mean length) would else have more than
// the 32 pieces that eight groups of threads of the join fetch in one round.  Us a call, two tiles at least / this:  14/2 heads of size 64, 2000 keys 7.3 / 6.7, 5000
// 7.9 / 7.8;  28/4 of 128, 2000 8.0 / 7.6, 6 queries 6000 12.3 / 11.5, 8000 13.5 / 12.1;  three ragged requests of 2000 13.2 / 11.9;  4/1 of 64, 16000 9.9 / 9.0.
constexpr int kFold = 32, kFoldRun = 4;
constexpr int kTargetGroups = 256;       // workgroups of a launch
constexpr int kMostBlocks = 4;           // row blocks of a workgroup: two compute waves on each SIMD

// A word that all lanes of a wave read, of memory that nothing writes meanwhile: by a scalar load.
__device__ __forceinline__ int uniform_load(const int32_t* at, int i) { return ((const SPECVLM_AS4 int32_t*)(uintptr_t)at)[i]; }

// The keys of a request in the order of the sweep: place x < sinks is key x, the others key x + skip; n places.  Both are multiples of 16.
struct PagedView { int sinks, skip, n; };
__device__ __forceinline__ PagedView paged_view(const PagedParams& p, int ql, int kvl)
{
    if (ql <= 0 || ql > p.q_len || kvl < ql || kvl > p.kv_len) return {0, 0, 0};     // (nothing to do, or sizes beyond the call's)
    if (p.window == 0) return {0, 0, kvl};
    const int first = kvl - ql - p.window + 1, lo = first > 0 ? first & ~15 : 0;       // the first query's first key behind the sinks
    const int sinks = (min(p.n_sinks, kvl) + 15) & ~15;
    if (lo <= sinks) return {0, 0, kvl};
    return {sinks, lo - sinks, kvl - (lo - sinks)};
}
// A request's new tokens and length, and the tiles of its sweep: each lane's own request (one behind the last has no tiles).
struct PagedRequest { int q0, ql, kvl; };
__device__ __forceinline__ PagedRequest paged_lane_request(const PagedParams& p, int b)
{
    PagedRequest r = {0, 0, 0};
    if (b < p.batch) {
        r.kvl = p.kv_lens[b];
        r.q0 = p.cu_q ? p.cu_q[b] : b * p.q_len;
        r.ql = p.cu_q ? p.cu_q[b + 1] - r.q0 : p.q_len;
    }
    return r;
}
__device__ __forceinline__ int paged_tiles(const PagedParams& p, const PagedRequest& r) { return (paged_view(p, r.ql, r.kvl).n + kTileKeys - 1) / kTileKeys; }

// A request that all lanes have in common.
__device__ __forceinline__ PagedRequest paged_request(const PagedParams& p, int b)
{
    PagedRequest r;
    r.kvl = uniform_load(p.kv_lens, b);
    r.q0 = p.cu_q ? uniform_load(p.cu_q, b) : b * p.q_len;
    r.ql = p.cu_q ? uniform_load(p.cu_q, b + 1) - r.q0 : p.q_len;
    return r;
}

// Tiles that a group takes.
__device__ __forceinline__ int paged_run(const PagedParams& p, int total)
{
    const int fewest = min(kFoldRun, divide(total + p.fold - 1, p.fold, p.inv_fold).q);       // (total: 1 and more, or nobody asks)
    return max(fewest, divide(total + p.max_groups - 1, p.max_groups, p.inv_groups).q);
}

// How a batch is cut: runs of `run` tiles over all requests one behind the other, or (from_first: up to 64 requests, one to a lane) from each request's first tile on,
// where there are so many groups, with one tile more if need be.  A group with the end of one request and the start of another drains its ring and exchanges
// twice, 2 us;  a tile more is 0.5 to 1.3.  Us a call, one behind the other / this:  28/4 heads, 16 requests of 900 keys 13.1 / 11.7, 6 queries 18.5 / 15.5;  64/8 heads, 6
// queries, 8 ragged requests of 3000 20.0 / 17.8;  14/2 heads, 24 of 2000 10.6 / 9.2;  the worst 16 of 1500, 6 queries 10.8 / 11.0.  (Runs beyond 16 tiles: not worth the look.)
constexpr int kCutRun = 16;
struct PagedCut { int run; bool from_first; int pieces; };       // (pieces: the lane's request's)
__device__ __forceinline__ PagedCut paged_cut(const PagedParams& p, int tiles, int total)
{
    const int run = paged_run(p, total);
    if (run > 1 && run <= kCutRun) {
#pragma unroll
        for (int more = 0; more < 2; ++more) {
            const int r = run + more, x = tiles + r - 1;          // (x < 2^24 + 16: the product is off by less than one)
            int pieces = (int)((float)x * __builtin_amdgcn_rcpf((float)r));
            pieces += x >= (pieces + 1) * r;
            pieces -= x < pieces * r;
            if (wave_total(pieces) <= p.max_groups) return {r, true, pieces};
        }
    }
    return {run, false, 0};
}

// Places [x0, x0 + 16) of the sweep that hold keys k0.. : bit i is set if a query row sees key k0 + i.  before: keys before the block; seen: the
// row's mask of the block; hidden_to: the last key that the window hides (-1: none).
__device__ __forceinline__ uint32_t low_bits(int n) { return (1u << min(max(n, 0), 16)) - 1u; }
__device__ __forceinline__ uint32_t paged_sees(int k0, int before, int kvl, uint64_t seen, int hidden_to, int n_sinks)
{
    const int at = k0 - before;                               // the block's key that k0 is
    const uint64_t block = at >= 0 ? (at < 64 ? seen >> at : 0) : (at > -16 ? seen << -at : 0);
    const uint32_t window = low_bits(hidden_to + 1 - k0) & ~low_bits(n_sinks - k0);
    return ((uint32_t)block | low_bits(-at)) & low_bits(kvl - k0) & ~window;
}

// The runs of group j, request by request: f(request's number, request, first tile, end, whether that is all of it).  All waves of the
// workgroup pass here, and a barrier between two of them.  tells: this wave leaves the join where a request's pieces are.
template <class F>
__device__ __forceinline__ void paged_walk(const PagedParams& p, int lane, int j, bool tells, F&& f)
{
    // one request: its tiles are the numbering;  more: a prefix sum over the requests, 64 at a time
    int total, tiles = 0, upto = 0, base;                         // (upto: tiles up to and with the lane's request; base: with all 64)
    PagedRequest rq = {}, mine = {};                              // (the piece's request; the lane's)
    if (p.batch == 1) {
        rq = paged_request(p, 0);
        total = base = paged_tiles(p, rq);
    } else {
        mine = paged_lane_request(p, lane);
        tiles = paged_tiles(p, mine);
        upto = wave_prefix(tiles);
        total = base = __builtin_amdgcn_readlane(upto, kWave - 1);
        if (p.batch > kWave) {
            int more = 0;
            for (int c = kWave; c < p.batch; c += kWave) more += paged_tiles(p, paged_lane_request(p, c + lane));
            total += wave_total(more);
        }
    }
    int x, x_end, c64 = 0, run = 0;
    PagedCut cut = {0, false, 0};
    if (p.batch > 1 && p.batch <= kWave) cut = paged_cut(p, tiles, total);
    if (cut.from_first) {                                        // group j has piece j of all
        const int ends = wave_prefix(cut.pieces);
        x = x_end = 0;
        if (j < __builtin_amdgcn_readlane(ends, kWave - 1)) {
            const int at = __builtin_ctzll(__ballot(ends > j));
            const int last_of = __builtin_amdgcn_readlane(upto, at);
            x = last_of - __builtin_amdgcn_readlane(tiles, at) + (j - __builtin_amdgcn_readlane(ends, at) + __builtin_amdgcn_readlane(cut.pieces, at)) * cut.run;
            x_end = min(last_of, x + cut.run);
        }
    } else {
        run = paged_run(p, total);
        x = j * run;
        x_end = min(total, x + run);
    }
    while (x < x_end) {
        int b = 0, first = 0, last = total;
        if (p.batch > 1) {
            while (x >= base) {
                c64 += kWave;
                mine = paged_lane_request(p, c64 + lane);
                tiles = paged_tiles(p, mine);
                upto = base + wave_prefix(tiles);
                base = __builtin_amdgcn_readlane(upto, kWave - 1);
            }
            const int at = __builtin_ctzll(__ballot(upto > x));              // the request that holds tile x
            last = __builtin_amdgcn_readlane(upto, at);
            first = last - __builtin_amdgcn_readlane(tiles, at);
            b = c64 + at;
            rq.q0 = __builtin_amdgcn_readlane(mine.q0, at);
            rq.ql = __builtin_amdgcn_readlane(mine.ql, at);
            rq.kvl = __builtin_amdgcn_readlane(mine.kvl, at);
            if (tells && x == first) {
                const int live = cut.from_first ? __builtin_amdgcn_readlane(cut.pieces, at) : (last - 1) / run - j + 1;
                if (lane < 2) p.part_of[2 * b + lane] = lane ? live : j;
            }
        }
        const int to = min(last, x_end);
        f(b, rq, x - first, to - first, x == first && to == last);
        x = to;
        if (x < x_end) __syncthreads();          // the next piece reuses the ring and the exchange buffer
    }
}

// Waits until at most `younger` tiles of LPW loads each are on the way.
template <int LPW, int MOST>
__device__ __forceinline__ void wait_tiles(int younger)
{
    if constexpr (MOST > 0) {
        if (younger < MOST) return wait_tiles<LPW, MOST - 1>(younger);
    }
    wait_vmcnt<MOST * LPW>();
}

// A value that is no finite number (an infinity, rows never written) belongs only to the rows that see its key, and a product with 0 (by which it is
// found) or with both parts of a probability, of which the second may be negative, is no number: it is left out of the products, and the rows get it by
// how many such values they see.  sees: bits 0..3 and 16..19, the lane's keys that its row sees.
template <int DJ>
__device__ __forceinline__ void take_odd_values(bf16x8 (&vf)[DJ], uint32_t sees, floatx4 (&o_acc)[DJ])
{
    const floatx4 none = {0.f, 0.f, 0.f, 0.f};
    floatx4 odd = none;
#pragma unroll
    for (int jj = 0; jj < DJ; ++jj) odd = mfma16(vf[jj], __builtin_bit_cast(bf16x8, u32x4{}), odd);
    if (__builtin_expect(__any(!(odd[0] + odd[1] + odd[2] + odd[3] == 0.f)), 0)) {
        u32x4 seen;                                   // bf16 0 or 1
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t two = sees >> (e < 2 ? 2 * e : 2 * e + 12);
            seen[e] = (two & 1u) * 0x3f80u | (two & 2u) * (0x3f800000u / 2);
        }
#pragma unroll
        for (int jj = 0; jj < DJ; ++jj) {
            u32x4 w = __builtin_bit_cast(u32x4, vf[jj]), up, down, nan;
#pragma unroll
            for (int e = 0; e < 4; ++e) {             // (two halves a word: a carry into bit 15 says that a size is an infinity's or more, or more than one)
                const uint32_t size = w[e] & 0x7fff7fffu, odd2 = (size + 0x00800080u) >> 15 & 0x00010001u;
                nan[e] = (size + 0x007f007fu) >> 15 & 0x00010001u;
                down[e] = (odd2 ^ nan[e]) & w[e] >> 15;
                up[e] = odd2 ^ nan[e] ^ down[e];
                w[e] &= ~(odd2 * 0xffffu);
            }
            vf[jj] = __builtin_bit_cast(bf16x8, w);
            const auto count = [&](u32x4 x) { return mfma16(__builtin_bit_cast(bf16x8, x * 0x3f80u), __builtin_bit_cast(bf16x8, seen), none); };
            const floatx4 n_up = count(up), n_down = count(down), n_nan = count(nan);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (n_up[e] > 0.f) o_acc[jj][e] += INFINITY;
                if (n_down[e] > 0.f) o_acc[jj][e] += -INFINITY;
                if (n_nan[e] > 0.f) o_acc[jj][e] = NAN;
            }
            __builtin_amdgcn_sched_barrier(0);        // (one after the other: the registers of all at once would be the kernel's most)
        }
    }
}

// What is done twice where a sum comes out as no finite number: as fast as it goes, and then with an eye on such values.
typedef std::integral_constant<bool, false> Plain;
typedef std::integral_constant<bool, true> Careful;
// Whether one of these is no finite number (0 times it is no zero).
__device__ __forceinline__ bool any_odd(floatx4 x)
{
    x *= 0.f;
    return __any(!(x[0] + x[1] + x[2] + x[3] == 0.f));
}
template <int N> __device__ __forceinline__ bool any_odd(const floatx4 (&x)[N])
{
    floatx4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < N; ++i) sum += 0.f * x[i];
    return any_odd(sum);
}
// x by the weight w of a maximum that another has passed.  Careful: an infinity stays one however small its weight is, also where 32 bits take that for 0.
template <class HOW> __device__ __forceinline__ floatx4 weighted(float w, floatx4 x, HOW)
{
    if constexpr (!HOW::value) return w * x;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = fabsf(x[e]) == INFINITY ? x[e] : w * x[e];
    return x;
}

// MB: row blocks of 16, one to a compute wave.  KS: chunks of 32 keys of a tile, a wave for each.  NS: tiles of the ring.  NLD: loader waves.
// WHOLE: a workgroup has all keys of its request, and there is no plan.
template <int D, int MB, int KS, int NS, int NLD, bool WHOLE>
__global__ __launch_bounds__((MB * KS + NLD) * kWave)
void paged_split_kernel(const PagedParams p)
{
    constexpr int TK = KS * kChunkKeys;
    static_assert(WHOLE || TK == kTileKeys, "what the plan counts");
    constexpr int NW = MB * KS;                  // compute waves (row block, key split); the loader waves come after them
    constexpr int DJ = D / 16, KK = D / 32, CH = D / 8, ROW_BYTES = D * 2;
    constexpr int KEYS_PER_LOAD = kWave / CH;    // key rows of one wave-wide load (4 or 8)
    constexpr int TILE_BYTES = TK * ROW_BYTES;   // one of K or V
    constexpr int LOADS_PER_MAT = TK / KEYS_PER_LOAD;
    constexpr int LPW = 2 * LOADS_PER_MAT / NLD; // loads of a loader wave per tile: the first half of the waves K, the others V
    constexpr int GPW = LPW * KEYS_PER_LOAD / 16;        // groups of 16 keys of a loader wave
    constexpr int LPG = 16 / KEYS_PER_LOAD;      // loads per group
    constexpr int LDS_STRIDE = D + 4;
    static_assert(NLD == 2 || NLD == 4, "loader waves: half for K, half for V");
    static_assert(GPW == 2 || GPW == 4, "their pages' bytes are one word or half of one");

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool is_loader = wave >= NW;
    const int lw = wave - NW;                    // loader index
    const int mb = wave % MB, ks = wave / MB;    // (compute waves) row block, chunk of a tile
    const int r = lane & 15, c = lane >> 4;

    extern __shared__ __align__(1024) unsigned char smem[];      // stage s: K tile at s*2*TILE_BYTES, V tile right after it
    unsigned char* const s_ok = smem + NS * 2 * TILE_BYTES;       // per stage eight bytes, one for 16 keys: their page is there

    const QuotRem head = divide(blockIdx.x, p.n_kv_heads, p.inv_heads), rows_of = divide(head.q, p.n_rgroups, p.inv_rgroups);
    const int g = head.r, row0 = rows_of.r * (MB * 16), j = rows_of.q;       // (j: group of workgroups, or request)
    const auto work = [&](auto&& f) {
        if constexpr (WHOLE) {
            const PagedRequest rq = paged_request(p, j);
            const int n = paged_view(p, rq.ql, rq.kvl).n;
            if (n > 0) f(j, rq, 0, (n + TK - 1) / TK, true);
        } else {
            paged_walk(p, lane, j, g == 0 && row0 == 0 && wave == NW - 1, f);
        }
    };

    if (is_loader) {
        // this wave's matrix, its first group of a tile, and the lane offsets of the loads of a group
        const bool is_v = lw >= NLD / 2;
        const int group0 = (lw % (NLD / 2)) * GPW;
        const char* const mat = reinterpret_cast<const char*>((is_v ? p.v : p.k) + (int64_t)g * p.head);
        uint32_t lane_off[LPG];
#pragma unroll
        for (int i = 0; i < LPG; ++i) {
            const int kl = i * KEYS_PER_LOAD + lane / CH;             // key inside the group
            const int swz = is_v ? v_swizzle<D>(kl) : (D == 128 ? kl : kl >> 1);
            lane_off[i] = (uint32_t)kl * (uint32_t)(p.tok * 2) + (uint32_t)((lane % CH) ^ swz) * 16u;
        }
        work([&](const int b, const PagedRequest& rq, const int t_begin, const int t_end, bool) {
            const PagedView view = paged_view(p, rq.ql, rq.kvl);
            const int n = view.n, n_tiles = t_end - t_begin;      // >= 1
            if (row0 >= p.group * rq.ql) return;
            const SPECVLM_AS4 int32_t* const table = (const SPECVLM_AS4 int32_t*)(uintptr_t)(p.table + (int64_t)b * p.table_row);
            int id[GPW], row[GPW];                                    // pages of the next tile's groups, and the rows in them
            auto look_up = [&](int tile) {
#pragma unroll
                for (int i = 0; i < GPW; ++i) {
                    // (places behind the last are masked in the compute: its group of 16 is loaded again)
                    const int x = min(tile * TK + (group0 + i) * 16, (n - 1) & ~15);
                    const QuotRem at = divide(x < view.sinks ? x : x + view.skip, p.page_size, p.inv_page);
                    id[i] = table[at.q];
                    row[i] = at.r;
                }
            };
            auto issue_tile = [&](int stage) {
                unsigned char* const st = smem + stage * (2 * TILE_BYTES) + (is_v ? TILE_BYTES : 0) + group0 * 16 * ROW_BYTES;
                uint32_t ok = 0;
#pragma unroll
                for (int i = 0; i < GPW; ++i) {
                    // (a page that is not one of the pool's is not read: the pool's first is, and its keys are masked)
                    const bool there = (uint32_t)id[i] < (uint32_t)p.n_pages;
                    ok |= (there ? 1u : 0u) << (8 * i);
                    const char* const src = mat + 2 * ((there ? id[i] : 0) * p.page + row[i] * p.tok);
#pragma unroll
                    for (int l = 0; l < LPG; ++l)
                        __builtin_amdgcn_global_load_lds((const SPECVLM_AS1 void*)(src + lane_off[l]),
                                                         (SPECVLM_AS3 void*)(st + (i * LPG + l) * 1024), 16, 0, 2);
                }
                if (!is_v && lane == 0) {
                    if constexpr (GPW == 4) *reinterpret_cast<uint32_t*>(s_ok + 8 * stage + group0) = ok;
                    else *reinterpret_cast<uint16_t*>(s_ok + 8 * stage + group0) = (uint16_t)ok;
                }
            };
            int i = 1 - NS, stage = 0;
            look_up(t_begin);
            do {
                if (i >= 0) {
                    wait_tiles<LPW, NS - 2>(n_tiles - 1 - i);          // (the tiles behind tile i that are on the way)
                    __asm__ volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the bytes of s_ok are written
                    stage_barrier();                                  // tile i landed for everyone; the stage of tile i-1 is free
                }
                if (i + NS - 1 < n_tiles) {
                    issue_tile(stage);
                    look_up(t_begin + min(i + NS, n_tiles - 1));
                    stage = stage == NS - 1 ? 0 : stage + 1;
                }
            } while (++i < n_tiles);
            __syncthreads();                                      // the exchange of the others
            __syncthreads();
        });
        return;
    }

    const float sc = fmaxf(p.scale_log2, 1e-30f);                 // (a zero scale as a vanishing one: -inf stays -inf)

    // Tiles [t_begin, t_end) of request b; the result goes to partial slot slot0 + row, or straight to the output.
    work([&](const int b, const PagedRequest& rq, const int t_begin, const int t_end, const bool direct) {
        const PagedView view = paged_view(p, rq.ql, rq.kvl);
        const int kvl = rq.kvl, before = kvl - rq.ql, n_rows = p.group * rq.ql, n = view.n;
        if (row0 >= n_rows) return;
        const int n_tiles = t_end - t_begin;
        const int64_t slot0 = (int64_t)((j + b) * p.n_kv_heads + g) * p.rows_pad;
        float m_run = -INFINITY, l_run = 0.f;
        floatx4 o_acc[DJ];
#pragma unroll
        for (int jj = 0; jj < DJ; ++jj) o_acc[jj] = floatx4{0.f, 0.f, 0.f, 0.f};
        bf16x8 qf[KK];
        const int row = row0 + mb * 16 + r;
        const QuotRem q_at = divide(row < n_rows ? row : row0, p.group, p.inv_group);   // (padding rows take the first: never stored)
        const int t_blk = q_at.q;
        const __bf16* qp = p.q + (int64_t)(rq.q0 + t_blk) * p.q_tok + (int64_t)(g * p.group + q_at.r) * p.q_head + c * 8;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) qf[kk] = *reinterpret_cast<const bf16x8*>(qp + kk * 32);
        // places [n_sinks, edge) hold keys that the window hides from some query
        const int edge = p.window ? kvl - p.window - view.skip : 0;
        // where this lane reads in a stage: its keys' rows and its value rows.  A row's swizzle is an XOR of the piece's number, and so are the
        // kk-th quarter of a key and the jj-th pair of pieces of a value row, whose bits of the address are the row's own
        const uint32_t lds0 = (uint32_t)(uintptr_t)(SPECVLM_AS3 unsigned char*)smem;
        const int v_row = ks * kChunkKeys + 4 * c + (r >> 2);                   // (16 rows on the swizzles are the same)
        const uint32_t k_base = lds0 + (ks * kChunkKeys + r) * ROW_BYTES + (c ^ ((D == 128) ? (r & 15) : ((r >> 1) & 7))) * 16;
        const uint32_t v_base = lds0 + TILE_BYTES + v_row * ROW_BYTES + (r & 3) * 8 + (v_swizzle<D>(v_row) >> 1) * 32;
        bool fresh = true;                                        // some row has seen nothing yet
        // 32 places from `base` on:  their logits, values and pages (careful: with the same roundings, and every value looked at)
        const auto take = [&](const int base, const uint32_t ok, floatx4 s0, floatx4 s1, bf16x8 (&vf)[DJ], auto careful) {
            const bool need_mask = ok != 0x0101u || base + kChunkKeys > n - rq.ql || (base < edge && base + kChunkKeys > p.n_sinks);
            float s[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) { s[e] = s0[e]; s[4 + e] = s1[e]; }
            uint32_t sees = 0x000f000fu;                          // bits 0..3 and 16..19: the lane's keys that its row sees
            if (need_mask) {
                // block key b is visible where bit b is set: 0..t in a chain, the caller's ancestors in a tree
                const uint64_t seen = p.block_mask ? p.block_mask[rq.q0 + t_blk] : ((2ull << t_blk) - 1ull);
                const int hidden_to = p.window ? before + t_blk - p.window : -1;
                const int x1 = base + 16, ka = base < view.sinks ? base : base + view.skip, kb = x1 < view.sinks ? x1 : x1 + view.skip;
                const uint32_t lo = (ok & 1u) ? paged_sees(ka, before, kvl, seen, hidden_to, p.n_sinks) : 0u;
                const uint32_t hi = (ok & 0x100u) ? paged_sees(kb, before, kvl, seen, hidden_to, p.n_sinks) : 0u;
                sees = (lo | hi << 16) >> (4 * c);
#pragma unroll
                for (int e = 0; e < 8; ++e) s[e] = (sees >> (e < 4 ? e : e + 12)) & 1u ? s[e] : -INFINITY;
            }
            // Away from the masks the exponentials are taken against the reference that the earlier chunks left, and the
            // maximum is tracked only where a lane's sum does not stay moderate (see decode_attn.hip).
            floatx8 pv;
            bool settled = false;
            if (!need_mask && !fresh) {
                float psum = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) { pv[e] = fast_exp2(fmaf(s[e], sc, -m_run)); psum += pv[e]; }
                if (!__any(!(psum < kPagedRedo))) {
                    l_run += psum;
                    settled = true;
                }
            }
            if (!settled) {
                float mx = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
                mx = quad_max(mx) * sc;
                const float m_new = fmaxf(m_run, mx);
                const float m_ref = (m_new == -INFINITY) ? 0.f : m_new;
                const float alpha = fast_exp2(m_run - m_ref);
                const bool rescale = m_new != m_run;
                m_run = m_new;
                float psum = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) { pv[e] = fast_exp2(fmaf(s[e], sc, -m_ref)); psum += pv[e]; }
                l_run = l_run * alpha + psum;
                if (__any(rescale)) {
#pragma unroll
                    for (int jj = 0; jj < DJ; ++jj) o_acc[jj] = weighted(alpha, o_acc[jj], careful);
                }
            }
            if (need_mask || fresh) fresh = __any(!(m_run > -INFINITY));
            if (decltype(careful)::value || need_mask) take_odd_values(vf, sees, o_acc);
            // ---- O^T += V^T P^T, the probabilities as two bf16 each: rounded to one, their error (2^-9 of each term) was as large as the
            // output's own rounding, and the result 1.45 times as far from the sums in 64 bits as one that is only rounded at the end ----
            const bf16x8 pf = __builtin_convertvector(pv, bf16x8);
            const u32x4 two = __builtin_bit_cast(u32x4, pf);
            floatx8 rest;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                rest[2 * e] = pv[2 * e] - __uint_as_float(two[e] << 16);
                rest[2 * e + 1] = pv[2 * e + 1] - __uint_as_float(two[e] & 0xffff0000u);
            }
            const bf16x8 pf_rest = __builtin_convertvector(rest, bf16x8);
#pragma unroll
            for (int jj = 0; jj < DJ; ++jj) o_acc[jj] = mfma16(vf[jj], pf, o_acc[jj]);
#pragma unroll
            for (int jj = 0; jj < DJ; ++jj) o_acc[jj] = mfma16(vf[jj], pf_rest, o_acc[jj]);
        };
        uint32_t at_stage = 0;
        int base = t_begin * TK + ks * kChunkKeys;
        for (int i = 0; i < n_tiles; ++i, base += TK, at_stage = at_stage == (NS - 1) * 2 * TILE_BYTES ? 0 : at_stage + 2 * TILE_BYTES) {
            stage_barrier();
            if (base >= n) continue;
            const uint32_t ok = (uint32_t)__builtin_amdgcn_readfirstlane(*reinterpret_cast<const uint16_t*>(s_ok + at_stage / (TILE_BYTES / 4) + 2 * ks));
            // ---- S^T = K Q^T for 32 keys ----
            floatx4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                const SPECVLM_AS3 u32x4* const at = (const SPECVLM_AS3 u32x4*)(k_base + at_stage ^ kk * 64);
                const u32x4 k0 = at[0], k1 = at[16 * ROW_BYTES / 16];
                s0 = mfma16(__builtin_bit_cast(bf16x8, k0), qf[kk], s0);
                s1 = mfma16(__builtin_bit_cast(bf16x8, k1), qf[kk], s1);
            }
            // ---- V^T fragments of the lane's keys (4c+e and 16+4c+e) by the transposing LDS read ----
            bf16x8 vf[DJ];
#pragma unroll
            for (int jj = 0; jj < DJ; ++jj) {
                typedef short s16x4 __attribute__((ext_vector_type(4)));
                SPECVLM_AS3 s16x4* const at = (SPECVLM_AS3 s16x4*)(v_base + at_stage ^ jj * 32);
                const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(at);
                const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(at + 16 * ROW_BYTES / 8);
                vf[jj] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
            }
            take(base, ok, s0, s1, vf, Plain{});
        }
        // A sum that is no finite number, as a rule of an infinite value that a row sees away from the masks:  the wave takes its keys once more, carefully,
        // from where they lie.  (Us a call, without this / with it:  a chain block over 12806 keys 16.3 / 16.4, windows of 12 requests 40.0 / 40.3, trees of 26
        // nodes 73.0 / 74.9;  values looked at in every chunk, or the ring filled again, cost the chain block 1 us.)
        if (__builtin_expect(any_odd(o_acc), 0)) {
            m_run = -INFINITY; l_run = 0.f; fresh = true;
#pragma unroll
            for (int jj = 0; jj < DJ; ++jj) o_acc[jj] = floatx4{0.f, 0.f, 0.f, 0.f};
            // (the parameters are fetched again: kept since the kernel's start they would push others out of their registers)
            const SPECVLM_AS4 PagedParams* z = (const SPECVLM_AS4 PagedParams*)__builtin_amdgcn_kernarg_segment_ptr();
            __asm__ volatile("" : "+s"(z));
            uint32_t row_bytes = (uint32_t)z->tok * 2;
            for (int base = t_begin * TK + ks * kChunkKeys; base < min(n, t_end * TK); base += TK) {
                uint32_t lane_r = r, lane_c = c;
                __asm__ volatile("" : "+s"(row_bytes), "+v"(lane_r), "+v"(lane_c));       // (or the offsets of every load would live through the loop)
                uint32_t ok = 0;
                const char *k_at[2], *v_at[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int x = min(base + 16 * i, (n - 1) & ~15);
                    const QuotRem at = divide(x < view.sinks ? x : x + view.skip, z->page_size, z->inv_page);
                    const int id = uniform_load(z->table + (int64_t)b * z->table_row, at.q);
                    const bool there = (uint32_t)id < (uint32_t)z->n_pages;
                    ok |= (there ? 1u : 0u) << (8 * i);
                    const int64_t off = (there ? id : 0) * z->page + at.r * z->tok + (int64_t)g * z->head;
                    k_at[i] = reinterpret_cast<const char*>(z->k + off);
                    v_at[i] = reinterpret_cast<const char*>(z->v + off);
                }
                floatx4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kk = 0; kk < KK; ++kk) {
                    s0 = mfma16(*reinterpret_cast<const bf16x8*>(k_at[0] + (lane_r * row_bytes + lane_c * 16) + kk * 64), qf[kk], s0);
                    s1 = mfma16(*reinterpret_cast<const bf16x8*>(k_at[1] + (lane_r * row_bytes + lane_c * 16) + kk * 64), qf[kk], s1);
                    __builtin_amdgcn_sched_barrier(0);
                }
                bf16x8 vf[DJ];
#pragma unroll
                for (int jj = 0; jj < DJ; ++jj) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        vf[jj][e] = *reinterpret_cast<const __bf16*>(v_at[e / 4] + ((4 * lane_c + e % 4) * row_bytes + lane_r * 2) + jj * 32);
                    __builtin_amdgcn_sched_barrier(0);            // (one after the other, as in take_odd_values)
                }
                take(base, ok, s0, s1, vf, Careful{});
            }
        }

        // ---- the KS waves of a row block exchange their results through LDS; wave ks then owns D/KS columns of its rows ----
        constexpr int SLICE = D / KS, CPL = SLICE / 4;
        __syncthreads();                             // every wave is done with the ring
        float* sm_m = reinterpret_cast<float*>(smem);            // [KS][MB][16]
        float* sm_l = sm_m + KS * MB * 16;                       // [KS][MB][16]
        float* sm_o = sm_l + KS * MB * 16;                       // [KS][MB][16][LDS_STRIDE]
        const int at = (ks * MB + mb) * 16 + r;
        const float l = quad_sum(l_run);
        if (c == 0) { sm_m[at] = m_run; sm_l[at] = l; }
#pragma unroll
        for (int jj = 0; jj < DJ; ++jj) *reinterpret_cast<floatx4*>(sm_o + at * LDS_STRIDE + 4 * c + 16 * jj) = o_acc[jj];
        __syncthreads();
        if (row >= n_rows) return;
        float m_x[KS], m_all = -INFINITY, l_all = 0.f;
        bool lost = false;
#pragma unroll
        for (int kx = 0; kx < KS; ++kx) { m_x[kx] = sm_m[(kx * MB + mb) * 16 + r]; m_all = fmaxf(m_all, m_x[kx]); }
        const float m_ref = (m_all == -INFINITY) ? 0.f : m_all;
#pragma unroll
        for (int kx = 0; kx < KS; ++kx) {
            const float w = fast_exp2(m_x[kx] - m_ref);
            lost |= w == 0.f && m_x[kx] > -INFINITY;
            m_x[kx] = w;
            l_all += w * sm_l[(kx * MB + mb) * 16 + r];
        }
        const int col0 = ks * SLICE + c * CPL;
        floatx4 acc[CPL / 4];
        const auto sum = [&](auto careful) {
#pragma unroll
            for (int qd = 0; qd < CPL / 4; ++qd) acc[qd] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kx = 0; kx < KS; ++kx) {
                const float* buf = sm_o + ((kx * MB + mb) * 16 + r) * LDS_STRIDE + col0;
#pragma unroll
                for (int qd = 0; qd < CPL / 4; ++qd) acc[qd] += weighted(m_x[kx], *reinterpret_cast<const floatx4*>(buf + 4 * qd), careful);
            }
        };
        if (__builtin_expect(__any(lost), 0)) sum(Careful{}); else sum(Plain{});
        if (direct) {
            const int t = t_blk, h = g * p.group + q_at.r;
            const float inv = l_all == 0.f ? 0.f : 1.f / l_all;                   // (a row that sees nothing: 0)
            __bf16* op = p.out + (int64_t)(rq.q0 + t) * p.q_tok + (int64_t)h * p.q_head + col0;
#pragma unroll
            for (int qd = 0; qd < CPL / 4; ++qd)
                *reinterpret_cast<bf16x4*>(op + 4 * qd) = __builtin_convertvector(acc[qd] * inv, bf16x4);
            if (p.lse && c == 0 && ks == 0)
                p.lse[(int64_t)(rq.q0 + t) * p.n_q_heads + h] = (m_all + fast_log2(l_all)) * kLn2;
        } else {
            float* po = p.part_o + (slot0 + row) * D + col0;
#pragma unroll
            for (int qd = 0; qd < CPL / 4; ++qd) *reinterpret_cast<floatx4*>(po + 4 * qd) = acc[qd];
            if (c == 0 && ks == 0) { p.part_ml[(slot0 + row) * 2] = m_all; p.part_ml[(slot0 + row) * 2 + 1] = l_all; }
        }
    });
}

// Short caches of few heads and requests.  A workgroup has 16 query rows and 16 value COLUMNS over all keys: the column slices compute the same logits, and
// in return there are no partial results and one launch.  Sixteen waves have CH chunks of 32 places each and issue all their loads, through registers,
// before they wait for the first (the bytes in flight are then not bound by a ring in LDS: 1511 keys of size 64 in whole workgroups 10 us, here 6.8).  All logits of
// a wave are there before its maximum is taken, so nothing is rescaled; the waves meet once, at the end.  Without a window the pages are looked up while the
// lengths are on their way.  Tried: chunks dealt to the waves in turn (700 keys of size 64 5.6 us, not 5.1: more lines for masked places), helper workgroups
// that touch the rows for the XCD's L2 (size 128, 1000 keys 8.8 / 7.9, where the split takes 7.5; 512 and size 64 the same).
template <int D, int CH>
__global__ __launch_bounds__(16 * kWave)
void paged_short_kernel(const PagedParams p)
{
    constexpr int NW = 16, COLS = 16, SLICES = D / COLS, KK = D / 32, KP = D / 8, KPL = kWave / KP, LPG = 16 / KPL, KL = 2 * LPG;
    constexpr int ROW_BYTES = D * 2, K_BYTES = kChunkKeys * ROW_BYTES, WAVE_LDS = K_BYTES + kChunkKeys * COLS * 2;
    extern __shared__ __align__(16) unsigned char smem[];
    float (*s_m)[NW] = reinterpret_cast<float (*)[NW]>(smem + NW * WAVE_LDS);
    float (*s_l)[NW] = s_m + 16;
    // (the parameters together: fetched where each is first used, one wait after the other, 8 requests of 500 keys took 7.1 us, not 6.9)
    __asm__ volatile("" :: "s"(p.q), "s"(p.k), "s"(p.v), "s"(p.q_tok), "s"(p.q_head), "s"(p.page), "s"(p.tok), "s"(p.head), "s"(p.table), "s"(p.table_row),
                     "s"(p.kv_lens), "s"(p.cu_q), "s"(p.n_pages), "s"(p.page_size), "s"(p.q_len), "s"(p.kv_len), "s"(p.n_kv_heads), "s"(p.group),
                     "s"(p.window), "s"(p.n_sinks), "s"(p.inv_page), "s"(p.inv_heads), "s"(p.inv_group), "s"(p.inv_rgroups), "s"(p.n_rgroups));
    __asm__ volatile("" :: "s"(p.scale_log2), "s"(p.block_mask), "s"(p.n_units), "s"(p.last_units), "s"(p.inv_last));
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, c = lane >> 4;
    // ids go round the XCDs: the slices of a unit lie 8 apart (or as many as are left) and share an L2 where there are units enough (8 requests of 1024
    // keys, 14/2 heads 7.6 us with a request's heads side by side, 6.6 here)
    const int eights = blockIdx.x / (kNumXcd * SLICES), in = blockIdx.x % (kNumXcd * SLICES);
    QuotRem at_unit = {in / kNumXcd, in % kNumXcd};
    if (kNumXcd * (eights + 1) > p.n_units) at_unit = divide(in, p.last_units, p.inv_last);
    const int slice = at_unit.q, unit = kNumXcd * eights + at_unit.r;
    const QuotRem head = divide(unit, p.n_kv_heads, p.inv_heads), block = divide(head.q, p.n_rgroups, p.inv_rgroups);
    const int g = head.r, rb = block.r, b = block.q;
    const int x0 = wave * (CH * kChunkKeys);
    const SPECVLM_AS4 int32_t* const table = (const SPECVLM_AS4 int32_t*)(uintptr_t)(p.table + (int64_t)b * p.table_row);
    const PagedRequest rq = paged_request(p, b);
    const PagedView view = paged_view(p, rq.ql, rq.kvl);
    // the pages, which without a window do not wait for the lengths (places behind the last are masked)
    int id[2 * CH], at_row[2 * CH];
#pragma unroll
    for (int i = 0; i < 2 * CH; ++i) {
        int key;
        if (p.window == 0) key = min(x0 + 16 * i, (p.kv_len - 1) & ~15);
        else { const int x = max(min(x0 + 16 * i, (view.n - 1) & ~15), 0); key = x < view.sinks ? x : x + view.skip; }
        const QuotRem at = divide(key, p.page_size, p.inv_page);
        id[i] = table[at.q];
        at_row[i] = at.r;
    }
    const int kvl = rq.kvl, before = kvl - rq.ql, n_rows = p.group * rq.ql, n = view.n;
    if (n == 0 || rb * 16 >= n_rows) return;
    const int row = rb * 16 + r;
    const QuotRem q_at = divide(row < n_rows ? row : 0, p.group, p.inv_group);       // (padding rows take row 0: never stored)
    const int t_blk = q_at.q;
    unsigned char* const k_lds = smem + wave * WAVE_LDS;
    unsigned char* const v_lds = k_lds + K_BYTES;
    float m = -INFINITY, l = 0.f;
    floatx4 o_acc[1] = {floatx4{0.f, 0.f, 0.f, 0.f}};
    if (x0 < n) {
        bf16x8 qf[KK];
        u32x4 kraw[CH][KL], vraw[CH];
        const __bf16* qp = p.q + (int64_t)(rq.q0 + t_blk) * p.q_tok + (int64_t)(g * p.group + q_at.r) * p.q_head + c * 8;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) qf[kk] = *reinterpret_cast<const bf16x8*>(qp + kk * 32);
        const char* const kmat = reinterpret_cast<const char*>(p.k + (int64_t)g * p.head);
        const char* const vmat = reinterpret_cast<const char*>(p.v + (int64_t)g * p.head + slice * COLS);
        uint32_t k_off[LPG];
#pragma unroll
        for (int i = 0; i < LPG; ++i) k_off[i] = (uint32_t)(i * KPL + lane / KP) * (uint32_t)(p.tok * 2) + (uint32_t)(lane % KP) * 16u;
        const uint32_t v_off = (uint32_t)(lane / 2 % 16) * (uint32_t)(p.tok * 2) + (uint32_t)(lane % 2) * 16u;
        uint32_t ok = 0;
        int64_t page_at[2 * CH];
#pragma unroll
        for (int i = 0; i < 2 * CH; ++i) {
            // (looked up before the request's length was there: behind it an entry may hold anything, and the wave's first group is loaded again)
            const bool inside = i == 0 || x0 + 16 * i < n, there = inside && (uint32_t)id[i] < (uint32_t)p.n_pages;
            ok |= (there ? 1u : 0u) << i;
            page_at[i] = inside ? 2 * ((there ? id[i] : 0) * p.page + at_row[i] * p.tok) : page_at[0];
        }
#pragma unroll
        for (int ch = 0; ch < CH; ++ch)
#pragma unroll
            for (int i = 0; i < KL; ++i) kraw[ch][i] = *reinterpret_cast<const u32x4*>(kmat + page_at[2 * ch + i / LPG] + k_off[i % LPG]);
#pragma unroll
        for (int ch = 0; ch < CH; ++ch) {
            const int64_t first = page_at[2 * ch], second = page_at[2 * ch + 1] - first;
            vraw[ch] = *reinterpret_cast<const u32x4*>(vmat + first + ((lane < 32 ? 0 : second) + v_off));
        }
        const float sc = fmaxf(p.scale_log2, 1e-30f);
        const int edge = p.window ? kvl - p.window - view.skip : 0;
        const uint64_t row_mask = p.block_mask ? p.block_mask[rq.q0 + t_blk] : ((2ull << t_blk) - 1ull);
        const int hidden_to = p.window ? before + t_blk - p.window : -1;
        float s[CH][8], mx = -INFINITY;
        uint32_t sees[CH];
#pragma unroll
        for (int ch = 0; ch < CH; ++ch) {
#pragma unroll
            for (int i = 0; i < KL; ++i) {
                const int kl = i * KPL + lane / KP, swz = (D == 128) ? (kl & 15) : ((kl >> 1) & 7);
                *reinterpret_cast<u32x4*>(k_lds + kl * ROW_BYTES + (((lane % KP) ^ swz) * 16)) = kraw[ch][i];
            }
            floatx4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                const int x = (kk * 4 + c) ^ ((D == 128) ? r : (r >> 1));
                const u32x4 k0 = *reinterpret_cast<const u32x4*>(k_lds + r * ROW_BYTES + x * 16);
                const u32x4 k1 = *reinterpret_cast<const u32x4*>(k_lds + (r + 16) * ROW_BYTES + x * 16);
                s0 = mfma16(__builtin_bit_cast(bf16x8, k0), qf[kk], s0);
                s1 = mfma16(__builtin_bit_cast(bf16x8, k1), qf[kk], s1);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) { s[ch][e] = s0[e]; s[ch][4 + e] = s1[e]; }
            const int base = x0 + ch * kChunkKeys;
            sees[ch] = 0x000f000fu;
            if ((ok >> (2 * ch) & 3u) != 3u || base + kChunkKeys > n - rq.ql || (base < edge && base + kChunkKeys > p.n_sinks)) {
                uint32_t lo = 0, hi = 0;
                if (base < n) {
                    const int x1 = base + 16, ka = base < view.sinks ? base : base + view.skip, kb = x1 < view.sinks ? x1 : x1 + view.skip;
                    if (ok >> (2 * ch) & 1u) lo = paged_sees(ka, before, kvl, row_mask, hidden_to, p.n_sinks);
                    if (ok >> (2 * ch) & 2u) hi = paged_sees(kb, before, kvl, row_mask, hidden_to, p.n_sinks);
                }
                sees[ch] = (lo | hi << 16) >> (4 * c) & 0x000f000fu;
#pragma unroll
                for (int e = 0; e < 8; ++e) s[ch][e] = (sees[ch] >> (e < 4 ? e : e + 12)) & 1u ? s[ch][e] : -INFINITY;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) mx = fmaxf(mx, s[ch][e]);
        }
        m = quad_max(mx) * sc;
        const float m_ref = (m == -INFINITY) ? 0.f : m;
        const uint32_t v_addr = (uint32_t)(uintptr_t)(SPECVLM_AS3 const void*)(v_lds + (4 * c + (r >> 2)) * (COLS * 2) + (r & 3) * 8);
        const auto products = [&](const int ch, auto careful) {
            floatx8 pv, rest;
#pragma unroll
            for (int e = 0; e < 8; ++e) pv[e] = fast_exp2(fmaf(s[ch][e], sc, -m_ref));
            if constexpr (!decltype(careful)::value) {
#pragma unroll
                for (int e = 0; e < 8; ++e) l += pv[e];
            }
            const bf16x8 pf = __builtin_convertvector(pv, bf16x8);
            const u32x4 two = __builtin_bit_cast(u32x4, pf);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                rest[2 * e] = pv[2 * e] - __uint_as_float(two[e] << 16);
                rest[2 * e + 1] = pv[2 * e + 1] - __uint_as_float(two[e] & 0xffff0000u);
            }
            const bf16x8 pf_rest = __builtin_convertvector(rest, bf16x8);
            *reinterpret_cast<u32x4*>(v_lds + lane * 16) = vraw[ch];
            __asm__ volatile("" ::: "memory");
            u32x2 lo = lds_read_tr16<0>(v_addr), hi = lds_read_tr16<16 * COLS * 2>(v_addr);
            __asm__ volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __asm__ volatile("" : "+v"(lo), "+v"(hi));
            bf16x8 vf[1] = {__builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3))};
            if (decltype(careful)::value || __any(sees[ch] != 0x000f000fu)) take_odd_values(vf, sees[ch], o_acc);
            o_acc[0] = mfma16(vf[0], pf, o_acc[0]);
            o_acc[0] = mfma16(vf[0], pf_rest, o_acc[0]);
        };
#pragma unroll
        for (int ch = 0; ch < CH; ++ch) products(ch, Plain{});
        if (__builtin_expect(any_odd(o_acc), 0)) {                // (as in paged_split_kernel; the maximum is the wave's already)
            o_acc[0] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ch = 0; ch < CH; ++ch) products(ch, Careful{});
        }
        l = quad_sum(l);
    }
    // ---- the waves meet: lane (r, c) holds columns 4c .. 4c + 3 of row r; four lanes a piece sum the waves' results, a quarter of them each ----
    constexpr int LANES = 4, EACH = NW / LANES, PIECES = COLS / 4, SKEW = 256 / LANES;
    static_assert(16 * COLS * 4 + NW * SKEW <= WAVE_LDS, "a wave's result takes the place of its buffers");
    reinterpret_cast<floatx4*>(k_lds + wave * SKEW)[r * PIECES + (c ^ (r & 3))] = o_acc[0];
    if (c == 0) { s_m[r][wave] = m; s_l[r][wave] = l; }
    __syncthreads();
    const int w = threadIdx.x % LANES, orow = threadIdx.x / LANES / PIECES, piece = threadIdx.x / LANES % PIECES, grow = rb * 16 + orow;
    if (grow >= n_rows || threadIdx.x >= kWave * LANES) return;
    float m_w[EACH], l_w[EACH];
    floatx4 o_w[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        m_w[i] = s_m[orow][w + LANES * i];
        l_w[i] = s_l[orow][w + LANES * i];
        o_w[i] = reinterpret_cast<const floatx4*>(smem + (w + LANES * i) * (WAVE_LDS + SKEW))[orow * PIECES + (piece ^ (orow & 3))];
    }
    const auto over_lanes = [](float x, auto op) {
        x = op(x, row_move<0xB1>(x));
        return op(x, row_move<0x4E>(x));
    };
    const auto sum = [](float a, float b) { return a + b; };
    float m_all = m_w[0], l_all = 0.f;
#pragma unroll
    for (int i = 1; i < EACH; ++i) m_all = fmaxf(m_all, m_w[i]);
    m_all = over_lanes(m_all, [](float a, float b) { return fmaxf(a, b); });
    const float ref = (m_all == -INFINITY) ? 0.f : m_all;
    floatx4 tot = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        m_w[i] = fast_exp2(m_w[i] - ref);                    // 0 for a wave without keys
        tot += m_w[i] * o_w[i];
        l_all += m_w[i] * l_w[i];
    }
    if (__builtin_expect(any_odd(tot), 0)) {
        tot = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < EACH; ++i) tot += weighted(m_w[i], o_w[i], Careful{});
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) tot[i] = over_lanes(tot[i], sum);
    l_all = over_lanes(l_all, sum);
    if (w != 0) return;
    const QuotRem out_at = divide(grow, p.group, p.inv_group);
    const int t = out_at.q, h = g * p.group + out_at.r;
    tot *= l_all == 0.f ? 0.f : 1.f / l_all;                 // (a row that sees nothing: 0)
    *reinterpret_cast<bf16x4*>(p.out + (int64_t)(rq.q0 + t) * p.q_tok + (int64_t)h * p.q_head + slice * COLS + 4 * piece) =
        __builtin_convertvector(tot, bf16x4);
    if (p.lse && slice == 0 && piece == 0) p.lse[(int64_t)(rq.q0 + t) * p.n_q_heads + h] = (m_all + fast_log2(l_all)) * kLn2;
}

// Joins the pieces of the requests that were cut (one that was not is in its place already).  GP groups of threads share a row's
// pieces, each a fold against its own maximum; they meet in LDS.
template <int D, int GP>
__global__ __launch_bounds__(256)
void paged_join_kernel(const PagedParams p)
{
    constexpr int TPR = D / 4, ROWS = 256 / (TPR * GP), PRE = 4;
    __shared__ float s_m[ROWS][GP], s_l[ROWS][GP];
    __shared__ __align__(16) float s_o[ROWS][GP][D + 4];
    const int nbh = p.batch * p.n_kv_heads;
    const QuotRem at = divide(blockIdx.x, nbh, p.inv_all_heads), head = divide(at.r, p.n_kv_heads, p.inv_heads);
    const int b = head.q, g = head.r;
    const PagedRequest rq = paged_request(p, b);
    const int n_rows = p.group * rq.ql, row0 = at.q * ROWS, tiles = paged_tiles(p, rq);
    if (row0 >= n_rows || tiles == 0) return;
    int j0, live;                                    // the first group that has a piece, and how many have
    if (p.batch > 1) {
        j0 = uniform_load(p.part_of, 2 * b); live = uniform_load(p.part_of, 2 * b + 1);
    } else {
        j0 = 0; live = (tiles - 1) / paged_run(p, tiles) + 1;
    }
    if (live == 1) return;
    const int sub = threadIdx.x / TPR, grp = sub % GP, lr = sub / GP, col = (threadIdx.x % TPR) * 4, row = row0 + lr;
    const int64_t slot0 = (int64_t)((j0 + b) * p.n_kv_heads + g) * p.rows_pad + min(row, n_rows - 1);
    const int64_t step = (int64_t)p.n_kv_heads * p.rows_pad;
    float m, l;
    floatx4 acc;
    const auto fold = [&](auto careful) {
        m = -INFINITY; l = 0.f;
        acc = floatx4{0.f, 0.f, 0.f, 0.f};
        for (int s0 = grp; s0 < live; s0 += GP * PRE) {
            float2 ml[PRE];
            floatx4 o[PRE];
#pragma unroll
            for (int i = 0; i < PRE; ++i) {
                const int64_t slot = slot0 + min(s0 + GP * i, live - 1) * step;
                ml[i] = *reinterpret_cast<const float2*>(p.part_ml + slot * 2);
                o[i] = *reinterpret_cast<const floatx4*>(p.part_o + slot * D + col);
            }
            float m_new = m;
#pragma unroll
            for (int i = 0; i < PRE; ++i) if (s0 + GP * i < live) m_new = fmaxf(m_new, ml[i].x);
            const float ref = (m_new == -INFINITY) ? 0.f : m_new, old = fast_exp2(m - ref);
            acc = weighted(old, acc, careful); l *= old;
#pragma unroll
            for (int i = 0; i < PRE; ++i) {
                if (s0 + GP * i < live) {
                    const float w = fast_exp2(ml[i].x - ref);        // 0 for a piece of which the row sees nothing
                    acc += weighted(w, o[i], careful);
                    l += w * ml[i].y;
                }
            }
            m = m_new;
        }
    };
    fold(Plain{});
    if (__builtin_expect(any_odd(acc), 0)) fold(Careful{});
    if constexpr (GP > 1) {
        *reinterpret_cast<floatx4*>(&s_o[lr][grp][col]) = acc;
        if (col == 0) { s_m[lr][grp] = m; s_l[lr][grp] = l; }
        __syncthreads();
        if (grp != 0) return;
#pragma unroll
        for (int i = 0; i < GP; ++i) m = fmaxf(m, s_m[lr][i]);
        const float ref = (m == -INFINITY) ? 0.f : m;
        const auto sum = [&](auto careful) {
            acc = floatx4{0.f, 0.f, 0.f, 0.f}; l = 0.f;
#pragma unroll
            for (int i = 0; i < GP; ++i) {
                const float w = fast_exp2(s_m[lr][i] - ref);
                acc += weighted(w, *reinterpret_cast<const floatx4*>(&s_o[lr][i][col]), careful);
                l += w * s_l[lr][i];
            }
        };
        sum(Plain{});
        if (__builtin_expect(any_odd(acc), 0)) sum(Careful{});
    }
    if (row >= n_rows) return;
    acc *= l == 0.f ? 0.f : 1.f / l;
    const QuotRem out_at = divide(row, p.group, p.inv_group);
    const int t = out_at.q, h = g * p.group + out_at.r;
    *reinterpret_cast<bf16x4*>(p.out + (int64_t)(rq.q0 + t) * p.q_tok + (int64_t)h * p.q_head + col) = __builtin_convertvector(acc, bf16x4);
    if (p.lse && col == 0) p.lse[(int64_t)(rq.q0 + t) * p.n_q_heads + h] = (m + fast_log2(l)) * kLn2;
}

// ---------------------------------------------------------------- host side ----
struct PagedPlan { int n_rgroups, mb, rows_pad, max_groups; };

static PagedPlan paged_plan(int q_len, int n_q_heads, int n_kv_heads)
{
    PagedPlan s;
    const int blocks = (n_q_heads / n_kv_heads * q_len + 15) / 16;
    s.n_rgroups = (blocks + kMostBlocks - 1) / kMostBlocks;
    s.mb = (blocks + s.n_rgroups - 1) / s.n_rgroups;
    s.rows_pad = s.n_rgroups * s.mb * 16;
    s.max_groups = kTargetGroups / (n_kv_heads * s.n_rgroups);
    if (s.max_groups < 1) s.max_groups = 1;
    return s;
}

template <int D, int MB, int KS, int NS, int NLD, bool WHOLE>
static int launch_paged(const PagedParams& p, hipStream_t stream)
{
    constexpr int NW = MB * KS;
    constexpr size_t ring = (size_t)NS * (2 * KS * kChunkKeys * D * 2 + 8);
    constexpr size_t exchange = sizeof(float) * (size_t)(NW * 16 * (D + 4 + 2));
    constexpr size_t lds = ring > exchange ? ring : exchange;
    if (!launchable((int64_t)(WHOLE ? p.batch : p.max_groups) * p.n_rgroups * p.n_kv_heads, (NW + NLD) * kWave)) return SPECVLM_EUNSUPPORTED;
    if (lds > 64 * 1024)
        if (const int rc = allow_lds<&paged_split_kernel<D, MB, KS, NS, NLD, WHOLE>>((int)lds)) return rc;
    hipLaunchKernelGGL((paged_split_kernel<D, MB, KS, NS, NLD, WHOLE>), dim3((WHOLE ? p.batch : p.max_groups) * p.n_rgroups * p.n_kv_heads),
                       dim3((NW + NLD) * kWave), lds, stream, p);
    return launch_status();
}

// Whether a workgroup takes a request whole: one launch and no plan, but no more than a CU's share of the memory and two or four waves at
// work.  `places` is the most that a request's sweep can have.  Us a call, shared keys and join / whole, requests of equal lengths (where slices of the value
// columns take the call, see below, neither does):
//   size 64, 14/2 heads:   one request, 256 keys 6.2 / 4.6, 512 6.5 / 5.6, 1024 6.8 / 7.8 (42 rows, 512 7.4 / 7.5, 1024 7.7 / 10.5);  8 of 1024 8.0 / 8.2;  16 of 42 rows, 700
//     keys 9.9 / 9.2, 900 10.4 / 10.9;  32 of 1000 9.6 / 9.1, 1200 9.9 / 10.3;  64 of 1500 14.3 / 12.9, 2048 16.7 / 16.2
//   size 128, 28/4 heads:  one request, 256 keys 6.5 / 5.5, 512 6.4 / 7.5;  6 queries, 4 of 450 10.2 / 10.3, 580 10.7 / 11.7, 8 of 450 12.3 / 10.5, 700 12.2 / 12.4, 16 of 700 14.6 /
//     12.7, 900 15.7 / 16.0, 24 of 1200 21.9 / 19.6;  16 of 580 10.3 / 10.6;  32 of 1024 17.3 / 17.0
//   size 128, 64/8 heads:  8 of 450 9.5 / 9.4, 580 9.6 / 10.6, 6 queries 700 14.0 / 13.0;  32 of 1800 42.0 / 40.0, 6 queries 46.0 / 42.7 (2048 ragged 29.6 / 31.2)
static bool paged_takes_whole(int batch, int n_kv_heads, int n_rgroups, int mb, int head_dim, int64_t places)
{
    const int64_t wgs = (int64_t)batch * n_kv_heads * n_rgroups;
    const int eighths = batch == 1 ? 8 : wgs < 64 || (wgs < 96 && mb == 1) ? 9 : wgs < 96 ? 14 : wgs < 256 ? 20 : 32;
    return places * 8 <= (head_dim == 64 ? 768 : 448) * eighths;
}
static int64_t paged_most_places(int q_len, int kv_len, int window, int n_sinks)
{
    const int64_t seen = window ? (int64_t)window + q_len + 14 + ((n_sinks + 15ll) & ~15ll) : kv_len;
    return seen < kv_len ? seen : kv_len;
}

// Chunks of a wave of paged_short_kernel, or 0: not this one.  It takes one round of workgroups (slices of a unit wait for nobody, but two rounds of them read
// everything twice), and as many keys as its waves hold.  Us a call, the best of the others / this:
//   size 64, 14/2 heads:   one request, 256 keys 4.6 / 3.8, 512 5.6 / 4.4, 1024 6.8 / 5.7, 1511 6.8 / 6.8 in one launch for two (42 rows 7.7 / 7.2);  8 of 1024 7.9 / 6.6, 1300
//     8.3 / 8.6;  32 of 500 6.4 / 5.7, 1000 9.1 / 7.5, 1500 10.8 / 9.7;  but 64 of 100 4.4 / 6.9, 16 of 512 of 42 rows 7.8 / 10.2
//   size 128, 28/4 heads:  one request, 512 keys 6.5 / 5.4, 700 6.9 / 7.1, 42 rows 600 8.3 / 6.8, 800 8.4 / 8.2, 1000 8.6 / 8.9;  8 of 500 8.4 / 6.9, 700 9.0 / 8.1;  but
//     16 of 500 9.4 / 12.4, 250 6.5 / 9.5
//   size 128, 64/8 heads:  one request, 700 keys 6.9 / 6.5, 8 queries 9.4 / 7.6;  2 of 512 8.6 / 6.5, 1000 8.0 / 9.0, 4 of 800 10.3 / 9.0
static int paged_blocks(const PagedParams& p) { return (p.group * p.q_len + 15) / 16; }
static int paged_short_chunks(int batch, int n_kv_heads, int n_blocks, int head_dim, int64_t places)
{
    if ((int64_t)batch * n_kv_heads * n_blocks * (head_dim / 16) > kNumCu) return 0;
    if (places > (head_dim == 64 ? 1536 : 832)) return 0;
    return (int)(places + 511) / 512;
}

template <int D, int CH>
static int launch_short_paged(PagedParams p, hipStream_t stream)
{
    p.n_rgroups = paged_blocks(p); p.inv_rgroups = reciprocal(p.n_rgroups);
    p.n_units = p.batch * p.n_rgroups * p.n_kv_heads;
    p.last_units = (p.n_units - 1) % kNumXcd + 1; p.inv_last = reciprocal(p.last_units);
    constexpr size_t lds = (size_t)16 * (kChunkKeys * (D + 16) * 2 + 2 * 16 * sizeof(float));
    if (lds > 64 * 1024)
        if (const int rc = allow_lds<&paged_short_kernel<D, CH>>((int)lds)) return rc;
    hipLaunchKernelGGL((paged_short_kernel<D, CH>), dim3(p.n_units * (D / 16)), dim3(16 * kWave), lds, stream, p);
    return launch_status();
}

template <int D>
static int launch_paged_d(const PagedParams& p, int mb, bool whole, int short_chunks, hipStream_t stream)
{
    if (short_chunks) {
        if constexpr (D == 64) switch (short_chunks) {
            case 1: return launch_short_paged<D, 1>(p, stream);
            case 2: return launch_short_paged<D, 2>(p, stream);
            case 3: return launch_short_paged<D, 3>(p, stream);
        }
        else switch (short_chunks) {
            case 1: return launch_short_paged<D, 1>(p, stream);
            case 2: return launch_short_paged<D, 2>(p, stream);
        }
        return SPECVLM_EUNSUPPORTED;
    }
    if (whole) {
        if constexpr (D == 64) switch (mb) {
            case 1: return launch_paged<D, 1, 4, 3, 4, true>(p, stream);
            case 2: return launch_paged<D, 2, 4, 3, 4, true>(p, stream);
            case 3: return launch_paged<D, 3, 4, 3, 4, true>(p, stream);
            case 4: return launch_paged<D, 4, 2, 4, 4, true>(p, stream);
        }
        else switch (mb) {
            case 1: return launch_paged<D, 1, 2, 3, 4, true>(p, stream);
            case 2: return launch_paged<D, 2, 2, 3, 4, true>(p, stream);
            case 3: return launch_paged<D, 3, 2, 3, 2, true>(p, stream);
            case 4: return launch_paged<D, 4, 2, 3, 4, true>(p, stream);
        }
        return SPECVLM_EUNSUPPORTED;
    }
    // few rows: eight groups of threads share a row's pieces;  where the rows fill the chip two do, in a quarter of the workgroups.  Us a call, eight /
    // two:  64/8 heads, 12806 keys, 8 queries 18.1 / 19.4;  14/2 heads, one, 1511 keys 7.3 / 8.0;  but 64 requests of up to 1000 keys, 28/4 heads 22.2 / 21.1,
    // windows of 12 requests, 4 queries, 40/8 heads 43.1 / 41.5, trees of 208 rows, four requests, the join alone 11 / 5.2.
    const int rows = p.group * p.q_len;
    const bool few = (int64_t)rows * p.batch * p.n_kv_heads < 1024;
    const int join_rows = 256 / (D / 4 * (few ? 8 : 2));
    const int64_t joins = (int64_t)((rows + join_rows - 1) / join_rows) * p.batch * p.n_kv_heads;
    if (!launchable(joins, 256)) return SPECVLM_EUNSUPPORTED;
    int rc = SPECVLM_EUNSUPPORTED;
    switch (mb) {
        case 1: rc = launch_paged<D, 1, 2, kRing, 4, false>(p, stream); break;
        case 2: rc = launch_paged<D, 2, 2, kRing, 4, false>(p, stream); break;
        case 3: rc = launch_paged<D, 3, 2, kRing, 2, false>(p, stream); break;     // (four loader waves: one request of 128 keys 8.2 us, not 7.9, long ones the same)
        case 4: rc = launch_paged<D, 4, 2, kRing, 4, false>(p, stream); break;
    }
    if (rc != SPECVLM_OK) return rc;
    if (few) hipLaunchKernelGGL((paged_join_kernel<D, 8>), dim3((unsigned)joins), dim3(256), 0, stream, p);
    else     hipLaunchKernelGGL((paged_join_kernel<D, 2>), dim3((unsigned)joins), dim3(256), 0, stream, p);
    return launch_status();
}

}  // namespace specvlm

using namespace specvlm;

extern "C" size_t specvlm_paged_attn_workspace_bytes(int batch, int q_len, int n_q_heads, int n_kv_heads, int head_dim)
{
    if (batch <= 0 || q_len <= 0 || n_kv_heads <= 0 || n_q_heads <= 0 || n_q_heads % n_kv_heads || (head_dim != 64 && head_dim != 128) ||
        q_len > kMaxQueryBlock)
        return 0;
    const PagedPlan s = paged_plan(q_len, n_q_heads, n_kv_heads);
    const size_t slots = ((size_t)s.max_groups + batch) * n_kv_heads * s.rows_pad;
    return align256(slots * head_dim * sizeof(float)) + align256(slots * 2 * sizeof(float)) + align256((size_t)batch * 2 * sizeof(int32_t));
}

extern "C" int specvlm_paged_attn(
    const void* q, int64_t q_tok_stride, int64_t q_head_stride,
    const void* k_pages, const void* v_pages, int64_t page_stride, int64_t tok_stride, int64_t head_stride,
    int n_pages, int page_size, const int32_t* page_table, int64_t table_stride, int max_pages,
    const int32_t* kv_lens, const int32_t* cu_q, int batch, int q_len, int kv_len,
    int n_q_heads, int n_kv_heads, int head_dim, float softmax_scale, int window, int n_sinks,
    const uint64_t* ancestor_mask, void* out, float* lse,
    void* workspace, size_t workspace_bytes, void* stream)
{
    if (batch < 0 || q_len < 0 || kv_len < 0 || n_q_heads <= 0 || n_kv_heads <= 0 || n_pages < 0 || max_pages < 0) return SPECVLM_EINVAL;
    if (n_q_heads % n_kv_heads || page_size <= 0 || window < 0 || n_sinks < 0) return SPECVLM_EINVAL;
    if (!(softmax_scale >= 0.f) || !(softmax_scale < INFINITY)) return SPECVLM_EINVAL;
    if ((head_dim != 64 && head_dim != 128) || page_size % 16 || q_len > kMaxQueryBlock) return SPECVLM_EUNSUPPORTED;
    if (batch == 0 || q_len == 0) return SPECVLM_OK;
    if (q_len > kv_len || kv_len > (int64_t)max_pages * page_size || n_pages == 0 || table_stride < 0) return SPECVLM_EINVAL;
    if (!q || !k_pages || !v_pages || !out || !page_table || !kv_lens) return SPECVLM_EINVAL;
    if ((q_tok_stride | q_head_stride | page_stride | tok_stride | head_stride) & 7) return SPECVLM_EUNSUPPORTED;
    if (((uintptr_t)q | (uintptr_t)k_pages | (uintptr_t)v_pages | (uintptr_t)out) & 15) return SPECVLM_EUNSUPPORTED;
    // (a lane's offset inside 16 keys has 32 bits; tiles and places of the sweep are ints)
    if (tok_stride < 0 || tok_stride >= ((int64_t)1 << 26) || kv_len > (1 << 30)) return SPECVLM_EUNSUPPORTED;
    if ((int64_t)batch * ((kv_len + kTileKeys - 1) / kTileKeys) >= ((int64_t)1 << 30) || batch > (1 << 30) / kFold) return SPECVLM_EUNSUPPORTED;
    if ((int64_t)batch * q_len >= ((int64_t)1 << 31) / n_q_heads) return SPECVLM_EUNSUPPORTED;        // (rows are ints; a launch's threads: launchable)
    if (window >= kv_len) window = 0;                 // (no position is that far on; sums with the others stay in 32 bits)
    const PagedPlan s = paged_plan(q_len, n_q_heads, n_kv_heads);
    const size_t need = specvlm_paged_attn_workspace_bytes(batch, q_len, n_q_heads, n_kv_heads, head_dim);
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < need) return SPECVLM_EWORKSPACE;

    PagedParams p;
    p.q = (const __bf16*)q; p.k = (const __bf16*)k_pages; p.v = (const __bf16*)v_pages;
    p.out = (__bf16*)out; p.lse = lse;
    p.q_tok = q_tok_stride; p.q_head = q_head_stride; p.page = page_stride; p.tok = tok_stride; p.head = head_stride;
    p.table = page_table; p.table_row = table_stride; p.kv_lens = kv_lens; p.cu_q = cu_q; p.block_mask = ancestor_mask;
    p.n_pages = n_pages; p.page_size = page_size;
    p.batch = batch; p.q_len = q_len; p.kv_len = kv_len;
    p.n_q_heads = n_q_heads; p.n_kv_heads = n_kv_heads; p.group = n_q_heads / n_kv_heads;
    p.window = window; p.n_sinks = n_sinks;
    p.inv_page = reciprocal(page_size); p.inv_heads = reciprocal(n_kv_heads); p.inv_all_heads = reciprocal(batch * n_kv_heads);
    p.inv_group = reciprocal(p.group); p.inv_rgroups = reciprocal(s.n_rgroups); p.inv_groups = reciprocal(s.max_groups);
    p.fold = kFold * batch; p.inv_fold = reciprocal(p.fold);
    p.scale_log2 = softmax_scale * kLog2e;
    p.n_rgroups = s.n_rgroups; p.rows_pad = s.rows_pad; p.max_groups = s.max_groups;
    const size_t slots = ((size_t)s.max_groups + batch) * n_kv_heads * s.rows_pad;
    p.part_o = (float*)workspace;
    p.part_ml = (float*)((char*)workspace + align256(slots * head_dim * sizeof(float)));
    p.part_of = (int32_t*)((char*)p.part_ml + align256(slots * 2 * sizeof(float)));
    const int64_t places = paged_most_places(q_len, kv_len, window, n_sinks);
    const bool whole = paged_takes_whole(batch, n_kv_heads, s.n_rgroups, s.mb, head_dim, places);
    // (over the queries themselves the slices of a row would write what the others still read; in the other kernels a row is read by who writes it)
    const int short_chunks = out == q ? 0 : paged_short_chunks(batch, n_kv_heads, paged_blocks(p), head_dim, places);
    return head_dim == 128 ? launch_paged_d<128>(p, s.mb, whole, short_chunks, (hipStream_t)stream) : launch_paged_d<64>(p, s.mb, whole, short_chunks, (hipStream_t)stream);
}
