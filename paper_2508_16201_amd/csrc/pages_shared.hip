// specvlm_pages_shared: which neighbouring requests of a batch share how many tokens, found from their rows of the page table.
//
// Integer arithmetic.  Request b has s_b = (kv_lens[b] - q_len_b) / page_size whole pages before its block; c_b is the number of first entries, up to
// min(s_{b-1}, s_b), in which its row agrees with the one before it and that are pages.  b goes with b - 1 if c_b * page_size >= min_tokens and
// 2 c_b >= max(c_{b-1}, c_{b+1}); a group is a run of requests that go with each other, and shares the least of its c.
//
// Bound.  Latency: the rows are read as far as they agree (0.8 MB for 250 requests of 784 shared pages, a microsecond), by a workgroup to a request, then one
// workgroup looks at a number a request (7.9 us a call).  A table that a workgroup reads at a look or two is compared by that one too, a wave to a request: 8
// rows of 140 pages 5.2 us in one launch, 7.8 in two.
#include <algorithm>

#include "common.h"

namespace specvlm {

constexpr int kSharedBatch = 8192;       // requests whose groups one workgroup holds in LDS
constexpr int kCompareThreads = 256, kGroupThreads = 1024;
constexpr int kAtOnce = kGroupThreads / kWave, kAtOncePages = 512;       // requests and pages of a table that is compared by one workgroup

struct SharedParams {
    const int32_t* table;
    int64_t table_row;
    const int32_t* kv_lens;
    const int32_t* cu_q;
    int32_t* groups;
    int32_t* common;                     // [batch] pages that each request has in common with the one before it
    int n_pages, page_size, max_pages, batch, q_len, min_tokens;
};

// Whole pages of a request before its block.
__device__ __forceinline__ int whole_pages(const SharedParams& p, int b)
{
    const int kvl = p.kv_lens[b], ql = p.cu_q ? p.cu_q[b + 1] - p.cu_q[b] : p.q_len;
    return ql <= 0 || kvl < ql ? 0 : min((kvl - ql) / p.page_size, p.max_pages);
}

// Entries of [from, from + 64) of the rows of b - 1 and b, up to `most`, that agree from the first on: by one wave.
__device__ __forceinline__ int agreeing(const SharedParams& p, const int32_t* above, const int32_t* row, int from, int most, int lane)
{
    const int i = from + lane;
    bool same = false;
    if (i < most) {
        const int id = row[i];
        same = id == above[i] && (uint32_t)id < (uint32_t)p.n_pages;
    }
    const uint64_t other = ~__ballot(same);
    return other ? __builtin_ctzll(other) : kWave;
}

// A workgroup to a request.
__global__ __launch_bounds__(kCompareThreads)
void shared_compare_kernel(const SharedParams p)
{
    constexpr int WAVES = kCompareThreads / kWave;
    __shared__ int s_stop[2];
    const int b = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (b == 0) {
        if (threadIdx.x == 0) p.common[0] = 0;
        return;
    }
    const int most = min(whole_pages(p, b - 1), whole_pages(p, b));
    const int32_t *const row = p.table + (int64_t)b * p.table_row, *const above = row - p.table_row;
    if (threadIdx.x < 2) s_stop[threadIdx.x] = most;
    __syncthreads();
    int n = most;
    for (int from = 0, turn = 0; from < most; from += WAVES * kWave, turn ^= 1) {
        const int at = from + wave * kWave, same = agreeing(p, above, row, at, most, lane);
        if (same < kWave && lane == 0) atomicMin(&s_stop[turn], min(at + same, most));
        __syncthreads();
        n = s_stop[turn];
        if (n < min(from + WAVES * kWave, most)) break;      // (the two words in turn: nobody writes the one that is read)
    }
    if (threadIdx.x == 0) p.common[b] = n;
}

template <bool ONE>                      // whether it compares the rows too
__global__ __launch_bounds__(kGroupThreads)
void shared_groups_kernel(const SharedParams p)
{
    extern __shared__ int smem[];
    int *const first = smem, *const members = smem + p.batch, *const least = members + p.batch;
    const int* common = p.common;
    __shared__ int s_wave[kGroupThreads / kWave];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if constexpr (ONE) {
        __shared__ int s_common[kAtOnce];
        common = s_common;
        if (wave < p.batch) {
            const int most = wave ? min(whole_pages(p, wave - 1), whole_pages(p, wave)) : 0;
            const int32_t *const row = p.table + (int64_t)wave * p.table_row, *const above = row - p.table_row;
            int n = 0;
            while (n < most) {                               // 256 entries at a look
                constexpr int LOOKS = 4;
                int same[LOOKS];
#pragma unroll
                for (int u = 0; u < LOOKS; ++u) same[u] = agreeing(p, above, row, n + u * kWave, most, lane);
                int u = 0;
#pragma unroll
                for (int w = 0; w < LOOKS; ++w) if (u == w && same[w] == kWave) ++u;
                int more = u * kWave;
#pragma unroll
                for (int w = 0; w < LOOKS; ++w) if (u == w) more += same[w];
                n += more;
                if (more < LOOKS * kWave) break;
            }
            if (lane == 0) s_common[wave] = n;
        }
        __syncthreads();
    }
    const auto linked = [&](int b, int c) {
        const int before = common[b - 1], behind = b + 1 < p.batch ? common[b + 1] : 0;
        return c > 0 && (int64_t)c * p.page_size >= p.min_tokens && 2 * (int64_t)c >= max(before, behind);
    };
    int carry = 0;                                           // the first request of the group at hand
    for (int b0 = 0; b0 < p.batch; b0 += kGroupThreads) {
        const int b = b0 + threadIdx.x;
        int f = 0;
        if (b < p.batch) {
            const int c = common[b];
            const bool goes_on = b > 0 && linked(b, c);
            f = goes_on ? 0 : b;
            members[b] = 0;
            least[b] = goes_on ? c : INT32_MAX;
        }
        // the last request up to here that begins a group
#pragma unroll
        for (int d = 1; d < kWave; d *= 2) {
            const int other = __shfl_up(f, d);
            if (lane >= d) f = max(f, other);
        }
        if (lane == kWave - 1) s_wave[wave] = f;
        __syncthreads();
        for (int w = 0; w < wave; ++w) f = max(f, s_wave[w]);
        f = max(f, carry);
        if (b < p.batch) first[b] = f;
        for (int w = 0; w < kGroupThreads / kWave; ++w) carry = max(carry, s_wave[w]);
        __syncthreads();
    }
    // a request's own number goes to its group's first: only those that begin one hold none
    for (int b = threadIdx.x; b < p.batch; b += kGroupThreads) {
        const int f = first[b];
        atomicAdd(&members[f], 1);
        if (f != b) atomicMin(&least[f], least[b]);
    }
    __syncthreads();
    for (int b = threadIdx.x; b < p.batch; b += kGroupThreads) {
        const int f = first[b];
        p.groups[b] = f;
        p.groups[p.batch + b] = members[b];
        p.groups[2 * p.batch + b] = members[f] > 1 ? least[f] * p.page_size : 0;
    }
}

}  // namespace specvlm

using namespace specvlm;

extern "C" size_t specvlm_pages_shared_workspace_bytes(int batch)
{
    return batch > 0 && batch <= kSharedBatch ? align256((size_t)batch * sizeof(int32_t)) : 0;
}

extern "C" int specvlm_pages_shared(
    const int32_t* page_table, int64_t table_stride, int max_pages, int n_pages, int page_size,
    const int32_t* kv_lens, const int32_t* cu_q, int batch, int q_len, int min_tokens,
    int32_t* groups, void* workspace, size_t workspace_bytes, void* stream)
{
    if (max_pages < 0 || n_pages < 0 || page_size <= 0 || batch < 0 || q_len < 0 || min_tokens < 0 || table_stride < 0) return SPECVLM_EINVAL;
    if (page_size % 16 || batch > kSharedBatch || (int64_t)max_pages * page_size > INT32_MAX) return SPECVLM_EUNSUPPORTED;
    if (batch == 0) return SPECVLM_OK;
    if (!page_table || !kv_lens || !groups) return SPECVLM_EINVAL;
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < specvlm_pages_shared_workspace_bytes(batch)) return SPECVLM_EWORKSPACE;
    SharedParams p = {};
    p.table = page_table; p.table_row = table_stride; p.kv_lens = kv_lens; p.cu_q = cu_q; p.groups = groups; p.common = (int32_t*)workspace;
    p.n_pages = n_pages; p.page_size = page_size; p.max_pages = max_pages; p.batch = batch; p.q_len = q_len; p.min_tokens = min_tokens;
    const int lds = 3 * batch * (int)sizeof(int);
    if (batch <= kAtOnce && max_pages <= kAtOncePages) {
        shared_groups_kernel<true><<<1, kGroupThreads, lds, (hipStream_t)stream>>>(p);
        return launch_status();
    }
    if (const int rc = allow_lds<&shared_groups_kernel<false>>(3 * kSharedBatch * (int)sizeof(int))) return rc;
    shared_compare_kernel<<<batch, kCompareThreads, 0, (hipStream_t)stream>>>(p);
    if (const int rc = launch_status()) return rc;
    shared_groups_kernel<false><<<1, kGroupThreads, lds, (hipStream_t)stream>>>(p);
    return launch_status();
}
