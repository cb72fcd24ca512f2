// How specvlm_shared_attn and specvlm_cross_attn number their work: entries, sets of rows, runs of units, rows of partial results.  Integer arithmetic on
// offsets, lengths and groups from device memory, which may be anything: by the kernels, and by the host in tests.
#pragma once

#include "common.h"

namespace specvlm {

constexpr int kRowsWaves = 8;
constexpr int kRowsThreads = kRowsWaves * kWave;
constexpr int kSetRows = kRowsWaves * 32;

// What is numbered.  Entry b is the keys that request b's group shares, if it is the group's first request; entry batch + b request b's own keys.
// (Flat: the call's entry b; with ranges a share of its queries, with the keys that any of them sees: RowsParams::spans.)  An item is an entry's set of rows of a
// kv head.  first: (paged, own keys) of the group that the request is taken with;  (flat) the call's entry.
struct Entry { int q0, n_q, key0, key1, first; };

struct RowsStart { int work, rows, q0, n_q, key0, key1, first, total; };       // in front of the entry; the entry; of all

struct RowsParams {
    const __bf16* q;
    const __bf16* k;
    const __bf16* v;
    __bf16* out;
    float* lse;
    int64_t q_tok, q_head, page, tok, head;      // strides in elements
    const int32_t* table;                        // (paged)
    int64_t table_row;
    const int32_t* kv_lens;
    const int32_t* groups;
    const uint64_t* block_mask;
    const int32_t* cu_q;
    const int32_t* cu_kv;                        // (flat)
    const int32_t* ranges;
    int n_pages, page_size;
    int batch, q_len, kv_len, n_queries;
    int n_q_heads, n_kv_heads, group;
    uint32_t inv_page, inv_group, inv_span;
    float scale_log2;
    int entries, span;                           // numbered; (ranges) queries of a share
    Entry* spans;
    int workgroups, padded;                      // that take runs; the launch
    float* part_o;                               // [rows_parts][D] unnormalised partial outputs (part_row)
    float* part_ml;                              // [rows_parts][2] running maximum in log2 units, sum
    RowsStart* starts;                           // [entries] what the join has to know of them
    int most_rows;                               // that the entries may have, for partial results
    // (paged) The output lies over the queries: a request that is taken alone may lie among those of a group, whose pieces read its queries too, so the join
    // writes all.
    bool over_q;
    bool far;                                    // entries that overlap may have more rows than an int holds
};

// What the call says of a request.
struct Request { int q0, n_q, kvl, first, members, shared; };
template <bool PAGED> __host__ __device__ __forceinline__ Request request_of(const RowsParams& p, int b)
{
    Request r = {b * p.q_len, p.q_len, 0, -1, 0, 0};
    if (p.cu_q) {
        r.q0 = p.cu_q[b];
        r.n_q = p.cu_q[b + 1] - r.q0;
    }
    if constexpr (PAGED) {
        r.kvl = p.kv_lens[b];
        r.first = p.groups[b];
        r.members = p.groups[p.batch + b];
        r.shared = p.groups[2 * p.batch + b];
    }
    return r;
}
// Whether b can be the first of a group of so many members that share so many tokens.
__host__ __device__ __forceinline__ bool leads(const RowsParams& p, int b, const Request& r)
{
    return r.first == b && r.members >= 2 && r.members <= p.batch - b && r.shared > 0 && r.shared % 16 == 0 && r.n_q > 0 && r.kvl >= r.n_q &&
           r.kvl <= p.kv_len && r.shared <= r.kvl - r.n_q;
}
// The keys that a group shares, with the queries of all of its requests, up to q_end; none where what is said of it does not fit together (its requests
// are then taken alone).
__host__ __device__ __forceinline__ Entry shared_entry(const RowsParams& p, const Request& r, int q_end)
{
    const int n_q = q_end - r.q0;
    if (n_q <= 0 || r.q0 < 0 || r.q0 > p.n_queries - n_q) return {0, 0, 0, 0, -1};
    return {r.q0, n_q, 0, r.shared, -1};
}
// A request's own keys, behind those that it shares with a group that begins at r.first, has so many members and the entry `all`:  if its queries are among
// the entry's (offsets that descend, of a request in between, leave others' outside).
__host__ __device__ __forceinline__ Entry own_entry(const RowsParams& p, int b, const Request& r, int members, const Entry& all)
{
    if (r.n_q <= 0 || r.n_q > p.q_len || r.q0 < 0 || r.q0 > p.n_queries - r.n_q || r.kvl < r.n_q || r.kvl > p.kv_len) return {0, 0, 0, 0, -1};
    const bool with = all.key1 > 0 && b - r.first < members && all.key1 <= r.kvl - r.n_q && all.q0 <= r.q0 && r.q0 + r.n_q <= all.q0 + all.n_q;
    return {r.q0, r.n_q, with ? all.key1 : 0, r.kvl, with ? r.first : -1};
}

template <bool PAGED> __host__ __device__ __forceinline__ Entry entry_of(const RowsParams& p, int e, bool grouped)
{
    if (e >= p.entries) return {0, 0, 0, 0, -1};
    const int b = PAGED && e >= p.batch ? e - p.batch : e;
    const Request r = request_of<PAGED>(p, b);
    if constexpr (!PAGED) {
        if (p.ranges) return p.spans[e];
        const int k0 = p.cu_kv ? p.cu_kv[e] : 0, n = p.cu_kv ? p.cu_kv[e + 1] - k0 : p.kv_len;
        // (offsets that leave the tensors: nothing is read or written by them)
        if (r.n_q <= 0 || r.q0 < 0 || r.q0 > p.n_queries - r.n_q || n < 0 || k0 < 0 || k0 > p.kv_len - n) return {0, 0, 0, 0, -1};
        return {r.q0, r.n_q, 0, n, e};
    } else {
        const int f = e < p.batch ? b : r.first;
        Entry all = {0, 0, 0, 0, -1};
        int members = 0;
        if (grouped && f >= 0 && f <= b) {
            const Request first = f == b ? r : request_of<true>(p, f);
            members = first.members;
            if (leads(p, f, first)) all = shared_entry(p, first, p.cu_q ? p.cu_q[f + members] : (f + members) * p.q_len);
        }
        return e < p.batch ? all : own_entry(p, b, r, members, all);
    }
}

__host__ __device__ __forceinline__ int chunks_of(const Entry& e) { return max(1, (e.key1 - e.key0 + 31) >> 5); }       // of 32 keys

__host__ __device__ __forceinline__ int padded_rows(const RowsParams& p, const Entry& e) { return (e.n_q * p.group + 31) & ~31; }      // of a kv head

// Work is counted in the time that 32 keys of a set take, and an item has kBegin more in front of its first: what a piece costs before and behind its keys.
// A set has 256 rows, the last one what is left. The figures are from the pieces' own clocks: 32 keys of up to four blocks of 32 rows 0.78 us, of more
// 1.15, a piece of one tile 9 to 12. (Trees of 26 nodes of eight requests about two videos of 12544 tokens: kBegin of 18 99 us a call, 27 89, 36 90;
// eight prompts of up to 256 tokens about one 345, 304, 304; 32 requests about five, which memory bounds, 125, 128, 130. With four blocks at 3: 107, 343 and 133 at 18.) No
// workgroup is begun for less than kLeastRun: of the smallest calls 6 and 12 take the same, 20 takes 1 us more.
constexpr int kBegin = 27, kLeastRun = 12;
struct Sets {
    int full, unit, whole, head;             // whole sets; work of 32 keys in the last; of a whole set; of a kv head
    __host__ __device__ __forceinline__ int unit_of(int set) const { return set < full ? 3 : unit; }
};
__host__ __device__ __forceinline__ Sets sets_of(int rows, int chunks)
{
    const int full = rows / kSetRows, blocks = ((rows + 31) >> 5) - full * kRowsWaves, unit = blocks <= 4 ? 2 : 3, whole = chunks * 3 + kBegin;
    return {full, unit, whole, full * whole + (blocks ? chunks * unit + kBegin : 0)};
}

struct Numbers { int work, rows; };          // of an entry, or in front of one
__host__ __device__ __forceinline__ Numbers numbers_of(const RowsParams& p, const Entry& e)
{
    if (e.n_q <= 0) return {0, 0};
    return {sets_of(e.n_q * p.group, chunks_of(e)).head * p.n_kv_heads, padded_rows(p, e) * p.n_kv_heads};
}

// The row of the partial results that workgroup j's piece of an item has: the rows of all items one after the other, and 256 on for every workgroup, so
// that two pieces of an item do not meet, nor two items of a workgroup.
__host__ __device__ __forceinline__ int64_t part_row(int j, int row_of_items) { return (int64_t)j * kSetRows + row_of_items; }

// The work is dealt to `n` workgroups: the first `more` have one more than `each`.
struct Shares {
    int n, each, more;
    __host__ __device__ __forceinline__ int begin(int j) const { return j * each + min(j, more); }
    __host__ __device__ __forceinline__ int of(int x) const
    {
        const int wide = more * (each + 1);
        return x < wide ? (int)((uint32_t)x / (uint32_t)(each + 1)) : more + (int)((uint32_t)(x - wide) / (uint32_t)max(each, 1));
    }
};
__host__ __device__ __forceinline__ Shares shares_of(const RowsParams& p, int total)
{
    const int n = min(p.workgroups, max(1, total / kLeastRun)), each = (int)((uint32_t)total / (uint32_t)n);
    return {n, each, total - each * n};
}

// A workgroup's way through the entries, a thread to each, from the first ones on.  Workgroup 0 goes through all once before, to tell of them, and begins again.
struct Walk {
    Numbers base;                            // in front of the entries at hand
    int c0;                                  // the first of them
    bool told;
    // Whether unit x is behind the entries at hand, which have so much work.  (Who has no unit to take looks for none: of skipped entries there is no work to find.)
    __host__ __device__ __forceinline__ bool goes_on(int x, int x_end, int work) const { return !told || (x < x_end && x >= base.work + work); }
    __host__ __device__ __forceinline__ void step(const Numbers& here, int entries)
    {
        base.work += here.work;
        base.rows += here.rows;
        c0 += kRowsThreads;
        if (c0 >= entries) {
            told = true;
            base = {0, 0};
            c0 = 0;
        }
    }
};

// A workgroup's part of an item: a set of rows of a kv head, and some of its keys.
struct Piece {
    int b, own;                              // request or entry; whether the keys are its own
    int q0, n_q, end;                        // the entry's queries, and the end of its keys
    int g, row0, n_rows;                     // kv head, the set's rows
    int key0, key1;                          // the piece's keys
    int direct;                              // whether they are all that the rows see
    int64_t part;                            // the first row of its partial results
};

// Whether an entry's offsets, or a request's, leave it queries: of those around it that do not, nothing else is true.
__host__ __device__ __forceinline__ bool has_queries(const RowsParams& p, int b)
{
    const int from = p.cu_q[b], to = p.cu_q[b + 1];
    return from >= 0 && from < to && to <= p.n_queries && (int64_t)to - from <= p.q_len;
}

// (Ranges) Shares of entry b's queries.  They are numbered behind those of the entries in front of it, wherever its queries lie; entries that have no query in
// common have no more than `entries` in all.
__host__ __device__ __forceinline__ int shares_of_entry(const RowsParams& p, int b)
{
    return b < p.batch && has_queries(p, b) ? divide(p.cu_q[b + 1] - p.cu_q[b] - 1, p.span, p.inv_span).q + 1 : 0;
}

}  // namespace specvlm
