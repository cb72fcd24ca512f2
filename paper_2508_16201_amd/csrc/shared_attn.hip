// specvlm_shared_attn and specvlm_cross_attn: softmax attention in which many query rows meet the same keys.
//
// specvlm_shared_attn is attention of every request's block of new tokens over its paged cache, where neighbouring requests
// have the same first pages (several questions about one video): those keys are read once and meet the rows of all of the
// group's requests, then each request's rows meet its own keys.  specvlm_cross_attn is attention of texts of any length over an
// encoder's states, which no causal mask hides.
//
// Mathematics.  One pass over the keys with the running maximum m and sum l of each query row (online softmax); a row's keys are
// cut into pieces (of the shared keys, of its own), and pieces are joined by  o = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s.
// Statistics, sums and partial outputs are fp32, the output is rounded once.
//
// Work decomposition.  Rows of a kv head (query, head of the group) are taken 256 at a time ("a set"), keys 32 at a time.  The
// keys of all sets, heads and requests are numbered one after the other, and each workgroup takes a run of equal length, which it
// finds by a prefix sum over the requests: lengths and groups are on the device, and a captured launch serves them as they change.
// A piece that is all a row has is written out directly; the others leave partial results that the second launch joins.
//
// A workgroup has eight waves of 32 rows (v_mfma_f32_32x32x16_bf16 with the keys as rows of the product and the queries as its
// columns: a lane then holds 16 logits of one row, which are, packed, the second product's operand).  Where a set has fewer rows,
// two or four waves share them and take every second or fourth 32 keys.  Tiles of 128 keys go to LDS by direct loads, two in
// turn.
//
// Bound.  Wide sets: 128 keys of 256 rows take 7400 to 7900 cycles of a CU, of which the matrix unit works 4096 and the reads of the tiles' fragments from LDS
// take as many; the clock, 2.4 GHz without such work, falls to 1.9 to 1.55 under it.  2 x 2048 queries of 64 heads over 12544 states: 1.50 ms, 1.12 PFLOP/s (a
// library's product of 8192^3 1.22).  The loop alone, without masks, lookups and pages, took 6650 cycles, and 5950 without loads.  Narrow sets: memory, 32 requests
// about five videos of up to 32768 tokens at 3.7 TB/s.  Beside the keys a piece takes 7 to 9 us: its place 0.8, table and queries 2, the first tile's way
// through the maxima 2 more than another's, its results 2.5; and the second launch 3.5 to 23 us.
#include <climits>
#include <type_traits>

#include "attn_tile.h"
#include "rows_numbering.h"

namespace specvlm {

typedef float floatx16 __attribute__((ext_vector_type(16)));

constexpr int kRowsTile = 128;           // keys of a tile
constexpr int kChunks = kRowsTile / 32;
constexpr float kRowsRedo = 0x1p20f;     // a lane's sum of 32 keys above this (or NaN) is done again with the maximum tracked
// 32 keys with more than this times what their row had before have their probabilities in two bf16, where one costs up to 2^-9 of a probability: evened out
// over many keys of like weight, but not in a row that one key makes up. (48 viewers' tokens over one stream of 65536, errors against 64 bits in parts of those of
// outputs rounded once, over seeds: without 1.15 to 1.56, at 4 1.04 to 1.23, 2 1.03 to 1.22 (others 1.33), 1 1.03 to 1.20, 0.25 1.03 to 1.17;  91.1 us a call, and 90.8, 91.2,
// 92.4 and 100.)
constexpr float kRowsPeak = 2.f;

// D = A(32x16 bf16) * B(16x32 bf16) + C.  Per lane (r = lane % 32, h = lane / 32):
//   A holds row r, contraction indices 8h..8h+7;  B holds column r, the same;  C/D hold column r, element i row 8(i/4) + 4h + i%4
__device__ __forceinline__ floatx16 mfma32(bf16x8 a, bf16x8 b, floatx16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// LDS behind the tiles:  what a workgroup knows of 512 entries.
struct RowsPlan {
    Entry entry[kRowsThreads];
    Numbers front[kRowsThreads];
    int work[kRowsThreads];
    Numbers wave[kRowsWaves];
    union {
        uint64_t tree[kSetRows];             // the rows' masks of the block, then
        float ml[kSetRows * 2];              // maxima and sums of waves that share rows
    };
    alignas(8) int word[2][kRowsThreads / 2];        // of requests
    uint64_t missing[2][kRowsWaves];         // of 64 tiles, by their 16 keys:  those whose page is none of the pool's
    int found;
};

// entry_of of all entries, one to a thread, where there are no more than threads:  what requests say of each other goes through LDS, not by one look at memory
// after the other (15.0 us a call of four short dialogues, 15.3 without).
__device__ __forceinline__ Entry entry_at_once(const RowsParams& p, RowsPlan& s, bool grouped)
{
    const int t = threadIdx.x, b = t < p.batch ? t : t - p.batch;
    Request r = {0, 0, 0, -1, 0, 0};
    if (b < p.batch) r = request_of<true>(p, b);
    if (t < p.batch) {
        s.word[0][b] = r.q0 + r.n_q;
        s.word[1][b] = r.members;
    }
    __syncthreads();
    Entry e = {0, 0, 0, 0, -1};
    if (t < p.batch) {
        if (grouped && leads(p, b, r)) e = shared_entry(p, r, s.word[0][b + r.members - 1]);
        s.entry[b] = e;
    }
    __syncthreads();
    if (t >= p.batch && b < p.batch) {
        const bool in = grouped && r.first >= 0 && r.first <= b;
        e = own_entry(p, b, r, in ? s.word[1][r.first] : 0, in ? s.entry[r.first] : e);
    }
    return e;
}

// The sum over the workgroup's threads.
__device__ __forceinline__ int64_t block_sum(RowsPlan& s, int64_t x)
{
    unsigned long long* const sum = reinterpret_cast<unsigned long long*>(s.word);
    if (threadIdx.x == 0) *sum = 0;
    __syncthreads();
    atomicAdd(sum, (unsigned long long)x);
    __syncthreads();
    x = (int64_t)*sum;
    __syncthreads();
    return x;
}

// Lane i's word, to all.
__device__ __forceinline__ uint64_t lane_word(uint64_t x, int i)
{
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), i) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)x, i);
}

// Inclusive prefix sums over the workgroup's threads, and the total; `s` is free again behind the next barrier.
__device__ __forceinline__ Numbers block_prefix(RowsPlan& s, Numbers x, int wave, int lane, Numbers* total)
{
    Numbers up = {wave_prefix(x.work), wave_prefix(x.rows)};
    if (lane == kWave - 1) s.wave[wave] = up;
    __syncthreads();
    Numbers all = {0, 0};
#pragma unroll
    for (int w = 0; w < kRowsWaves; ++w) {
        const Numbers t = s.wave[w];
        if (w < wave) { up.work += t.work; up.rows += t.rows; }
        all.work += t.work;
        all.rows += t.rows;
    }
    *total = {__builtin_amdgcn_readfirstlane(all.work), __builtin_amdgcn_readfirstlane(all.rows)};
    __syncthreads();
    return up;
}

// A direct load of 16 bytes a lane to LDS, lane after lane from `lds` on (wave-uniform).  Issued as assembly: of the builtin the compiler knows that it writes
// LDS, and waits for all of them before every read of LDS that might be of the other stage.  (M0 takes one state to be seen by the load.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_to_lds(const char* base, uint32_t lane_offset, uint32_t lds)
{
    __asm__ volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(lane_offset), "s"(base) : "memory", "m0");
}
#pragma clang diagnostic pop

// How a tile lies in LDS.  A direct load brings 1 KB, of ROWS rows, and its lanes may take their 16 bytes from any of them: so the bytes lie as they are read, and
// every address is one of the lane and a constant.  Keys: piece (16 bytes) after piece, of each the rows;  32 lanes read the same piece of 32 rows, and with
// the loads PAD apart 16 of them touch all banks once.  Values: 32 columns after 32 columns, of each the rows;  32 lanes of a transposing read touch 4 rows.
template <int D> struct Layout {
    static constexpr int ROWS = 512 / D, PAD = ROWS * 16, LOAD = 1024 + PAD, TILE = kRowsTile / ROWS * LOAD;
};

template <class T> __device__ __forceinline__ SPECVLM_AS3 T* in_lds(uint32_t at) { return (SPECVLM_AS3 T*)(uintptr_t)at; }

__device__ __forceinline__ uint32_t first_bits(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; }

__device__ __forceinline__ float half_max(float x)
{
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float half_sum(float x)
{
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// What is computed from x stays where it is written: taken out of the loops, it would be in registers that the products need.
__device__ __forceinline__ void held(int& x) { __asm__ volatile("" : "+v"(x)); }
// (and the parameters are fetched where they are used: a kernel's, all held from its start, were more than there are scalar registers)
#define SPECVLM_AS4 __attribute__((address_space(4)))
__device__ __forceinline__ const SPECVLM_AS4 RowsParams& rows_params()
{
    const SPECVLM_AS4 RowsParams* z = (const SPECVLM_AS4 RowsParams*)__builtin_amdgcn_kernarg_segment_ptr();
    __asm__ volatile("" : "+s"(z));
    return *z;
}

// Takes a piece and writes what comes of it.
template <int D, bool PAGED>
__device__ __forceinline__ void rows_piece(RowsPlan& plan, const uint32_t lds0, const Piece& pc)
{
    constexpr int KK = D / 16, JB = D / 32, ROWS = Layout<D>::ROWS, LOAD_BYTES = Layout<D>::LOAD, TILE_BYTES = Layout<D>::TILE;
    constexpr int LOADS = 16 / ROWS, CHUNK_BYTES = 32 / ROWS * LOAD_BYTES;
    static_assert(kSetRows * D * 4 <= 4 * TILE_BYTES, "the exchange of waves that share rows");
    const SPECVLM_AS4 RowsParams& p = rows_params();
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int lane = threadIdx.x & 63;
    held(lane);
    const int r = lane & 31, h = lane >> 5;
    const float sc = fmaxf(p.scale_log2, 1e-30f);            // (a zero scale as a vanishing one: -inf stays -inf)
    const int n_blocks = (pc.n_rows + 31) >> 5, log_blocks = n_blocks > 4 ? 3 : n_blocks > 2 ? 2 : n_blocks - 1;       // waves of a kind
    const int blk = wave & ((1 << log_blocks) - 1), ks = wave >> log_blocks, n_ks = min(kChunks, kRowsWaves >> log_blocks);
    const bool works = blk < n_blocks && ks < n_ks;
    // Probabilities in two bf16 for one or two blocks, whose matrix products are hidden behind the loads (errors 1.03 times as large without, 1 % less time).
    const bool two_parts = n_blocks <= 2;
    const int key0 = pc.key0, key1 = pc.key1, tiles = (key1 - key0 + kRowsTile - 1) / kRowsTile;

    // ---- loads: wave w brings keys 16w..16w+15 of a tile ----
    const int64_t kv0 = (int64_t)pc.g * p.head + (PAGED ? 0 : (int64_t)(p.cu_kv ? __builtin_amdgcn_readfirstlane(p.cu_kv[pc.b]) : 0) * p.tok);
    const char* const k_at = reinterpret_cast<const char*>(p.k + kv0);
    const char* const v_at = reinterpret_cast<const char*>(p.v + kv0);
    uint64_t at = 0;                                     // of the next 64 tiles, one to a lane: the bytes from the pool's first row to this wave's 16 keys
    int id = 0, place = 0;
    const auto look_up = [&](int tile) {
        const int key = min(key0 + (tile + lane) * kRowsTile + wave * 16, (key1 - 1) & ~15);             // (a group behind the last: that one again)
        const QuotRem pg = divide(key, p.page_size, p.inv_page);
        id = p.table[(int64_t)pc.b * p.table_row + pg.q];
        place = pg.r;
    };
    const auto looked_up = [&](int tile) {
        // (a page that is not one of the pool's is not read: the pool's first is, and its keys are masked)
        const bool there = (uint32_t)id < (uint32_t)p.n_pages;
        at = (uint64_t)((there ? id : 0) * p.page + place * p.tok) * 2;
        const uint64_t missing = __ballot(!there && tile + lane < tiles);
        if (lane == 0) plan.missing[tile >> 6 & 1][wave] = missing;
    };
    const uint32_t k_from = (uint32_t)(lane % ROWS) * (uint32_t)(p.tok * 2) + lane / ROWS * 16;
    const uint32_t v_from = (uint32_t)((lane >> 2) % ROWS) * (uint32_t)(p.tok * 2) + (lane / (4 * ROWS) * 4 + (lane & 3)) * 16;
    const int64_t rows_bytes = p.tok * (ROWS * 2);
    const auto issue = [&](int tile, int stage) {
        const uint32_t to = lds0 + stage * 2 * TILE_BYTES + wave * LOADS * LOAD_BYTES;
        int64_t first;
        const int key = key0 + tile * kRowsTile + wave * 16;
        int last;                                        // the last of the 16 keys that there is: it stands for those behind it, whatever lies there
        if constexpr (PAGED) {
            const int l = tile & 63;
            if (l == 0 && tile > 0) {
                look_up(tile);
                looked_up(tile);
            }
            first = (int64_t)lane_word(at, l);
            last = key < key1 ? key1 - 1 - key : (key1 - 1) & 15;
        } else {
            first = (int64_t)min(key, key1 - 1) * (p.tok * 2);
            last = max(key1 - 1 - key, 0);
        }
        if (last >= 15) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                load_to_lds(k_at + first + i * rows_bytes, k_from, to + i * LOAD_BYTES);
                load_to_lds(v_at + first + i * rows_bytes, v_from, to + TILE_BYTES + i * LOAD_BYTES);
            }
            return;
        }
        const int k_row = lane % ROWS, v_of = (lane >> 2) % ROWS;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            load_to_lds(k_at + first, k_from + (uint32_t)(min(i * ROWS + k_row, last) - k_row) * (uint32_t)(p.tok * 2), to + i * LOAD_BYTES);
            load_to_lds(v_at + first, v_from + (uint32_t)(min(i * ROWS + v_of, last) - v_of) * (uint32_t)(p.tok * 2), to + TILE_BYTES + i * LOAD_BYTES);
        }
    };

    // this wave's rows; their queries are fetched while the first tile's pages are looked up
    if (PAGED && tiles > 0) look_up(0);
    const int my_row = blk * 32 + r;
    const QuotRem q_at = divide(pc.row0 + (my_row < pc.n_rows ? my_row : 0), p.group, p.inv_group);  // (padding rows take the first: never stored)
    const int64_t q_tok = pc.q0 + q_at.q;
    bf16x8 qf[KK];
    const __bf16* const qp = p.q + q_tok * p.q_tok + (int64_t)(pc.g * p.group + q_at.r) * p.q_head + h * 8;
#pragma unroll
    for (int s = 0; s < KK; ++s) qf[s] = *reinterpret_cast<const bf16x8*>(qp + s * 16);
    if (PAGED && tiles > 0) looked_up(0);
    if (tiles > 0) issue(0, 0);
    // the keys that it sees: [lo, hi), of the block those of a tree node's mask;  of all of the wave's rows: keys that all see, and that some see
    int lo = key0, hi = key1, all_lo = key0, all_hi = key1, any_lo = key0, any_hi = key1;
    const int before = pc.end - pc.n_q;                      // (own keys of a block)
    bool is_tree = false;
    if constexpr (PAGED) {
        if (pc.own) {
            is_tree = p.block_mask != nullptr;
            if (is_tree) {
                if (h == 0) plan.tree[my_row] = p.block_mask[q_tok];
                all_hi = min(before, key1);
            } else {
                hi = min(hi, before + q_at.q + 1);
                all_hi = min(key1, before + divide(pc.row0 + blk * 32, p.group, p.inv_group).q + 1);
                any_hi = min(key1, before + divide(pc.row0 + min(blk * 32 + 31, pc.n_rows - 1), p.group, p.inv_group).q + 1);
            }
        }
    } else if (p.ranges) {
        lo = min(max(p.ranges[2 * q_tok], 0), key1);
        hi = min(max(p.ranges[2 * q_tok + 1], 0), key1);
        all_lo = lo, all_hi = hi, any_lo = lo < hi ? lo : INT_MAX, any_hi = lo < hi ? hi : 0;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            all_lo = max(all_lo, __shfl_xor(all_lo, d)); all_hi = min(all_hi, __shfl_xor(all_hi, d));
            any_lo = min(any_lo, __shfl_xor(any_lo, d)); any_hi = max(any_hi, __shfl_xor(any_hi, d));
        }
        all_lo = __builtin_amdgcn_readfirstlane(all_lo); all_hi = __builtin_amdgcn_readfirstlane(all_hi);
        any_lo = __builtin_amdgcn_readfirstlane(any_lo); any_hi = __builtin_amdgcn_readfirstlane(any_hi);
    }

    float m_run, l_run;
    floatx16 o[JB];
    // where this lane reads in a stage
    const uint32_t k_base = lds0 + r / ROWS * LOAD_BYTES + r % ROWS * 16 + h * ROWS * 16;
    const int v_row = 4 * h + ((lane & 15) >> 2);
    const uint32_t v_base = lds0 + TILE_BYTES + v_row / ROWS * LOAD_BYTES + v_row % ROWS * 64 + (lane >> 4 & 1) * 32 + (lane & 3) * 8;
    // V^T fragments of 16 keys, by the transposing read
    const auto read_values = [&](bf16x8 (&vf)[JB], uint32_t at) {
#pragma unroll
        for (int jb = 0; jb < JB; ++jb) {
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            SPECVLM_AS3 s16x4* const src = in_lds<s16x4>(v_base + at) + jb * ROWS * 64 / 8;
            const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(src);
            const s16x4 c = __builtin_amdgcn_ds_read_tr16_b64_v4i16(src + 8 / ROWS * LOAD_BYTES / 8);
            vf[jb] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, c, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    };

    const auto read_keys = [&](bf16x8 (&kf)[KK], uint32_t at) {
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) kf[kk] = __builtin_bit_cast(bf16x8, in_lds<const u32x4>(k_base + at)[kk * 2 * ROWS]);
    };
    // S^T = K Q^T for 32 keys
    const auto logits = [&](const bf16x8 (&kf)[KK]) {
        floatx16 s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) s = mfma32(kf[kk], qf[kk], s);
        return s;
    };
    bool fresh = true;                                   // some row has seen nothing yet
    // Probabilities against the maximum with these logits too, to which the sums are brought.
    bool peak = false;                                   // the last 32 keys count for much of what some row has seen
    const auto raise = [&](const floatx16& s, float (&pv)[16]) {
        float mx = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
        const float m_new = fmaxf(m_run, half_max(mx) * sc);
        const float m_ref = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = fast_exp2(m_run - m_ref);
        const bool rescale = m_new != m_run;
        m_run = m_new;
        float psum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) { pv[i] = fast_exp2(fmaf(s[i], sc, -m_ref)); psum += pv[i]; }
        l_run *= alpha;
        peak = __any(psum > kRowsPeak * l_run);
        l_run += psum;
        if (__any(rescale)) {
#pragma unroll
            for (int jb = 0; jb < JB; ++jb)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[jb][i] *= alpha;
        }
    };
    // Probabilities of the keys from k0 on (two: whether the pages of the first and the second 16 are there), against the running maximum.
    const auto weigh = [&](floatx16 s, int k0, uint32_t two, float (&pv)[16]) {
        const bool need_mask = two != 0x101u || k0 < all_lo || k0 + 32 > all_hi;
        if (need_mask) {
            uint32_t sees = first_bits(hi - k0) & ~first_bits(lo - k0) & ((two & 1 ? 0xffffu : 0u) | (two & 0x100 ? 0xffff0000u : 0u));
            if (is_tree) {
                const int in = k0 - before;
                const uint64_t tree = plan.tree[my_row];
                const uint64_t block = in >= 0 ? (in < 64 ? tree >> in : 0) : (in > -32 ? tree << -in : 0);
                sees &= (uint32_t)block | first_bits(-in);
            }
            sees >>= 4 * h;                                  // bit 8(i/4) + i%4: the lane's i-th key
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = sees >> (8 * (i / 4) + i % 4) & 1u ? s[i] : -INFINITY;
        }
        // Away from the masks the exponentials are taken against the reference that the earlier keys left, and the maximum is tracked only where a
        // lane's sum does not stay moderate.
        if (!need_mask && !fresh) {
            float psum = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) { pv[i] = fast_exp2(fmaf(s[i], sc, -m_run)); psum += pv[i]; }
            if (!__any(!(psum <= kRowsRedo))) {
                peak = __any(psum > kRowsPeak * l_run);
                l_run += psum;
                return;
            }
        }
        raise(s, pv);
        fresh = __any(!(m_run > -INFINITY));
    };
    const auto begin_sums = [&] {
        m_run = -INFINITY;
        l_run = 0.f;
        fresh = true;
#pragma unroll
        for (int jb = 0; jb < JB; ++jb)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[jb][i] = 0.f;
    };
    const auto lds_done = [] { __asm__ volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };

    // A tile that all rows of the wave see whole, after others: while the vector unit weighs 32 keys, the matrix unit takes the products with the values of the last
    // 32 and then the logits of the next.  (The wave's keys of a tile: all, or every second 32.)  Returns how many it has taken: those that go beyond the maximum are left.
    // (Eight prompts of up to 256 tokens about one video 340 us a call without, 327 with; 48 viewers' tokens over a stream 102 and 96, 99.5 with tiles of all keys only; trees the same. Four
    // waves that share rows have one 32 keys of a tile: nothing to work on beside.)
    const auto whole_tile = [&](auto pieces, const uint32_t at) {
        constexpr int N = decltype(pieces)::value, STEP = kChunks / N * CHUNK_BYTES;
        floatx16 s;
        bf16x8 pf[2];
        {
            bf16x8 kf[KK];
            read_keys(kf, at);
            __builtin_amdgcn_sched_barrier(0);               // (the reads of all of them first: one by one, each waits for its own)
            s = logits(kf);
        }
#pragma unroll
        for (int ch = 0; ch <= N; ++ch) {
            float pv[16], psum = 0.f;
            __builtin_amdgcn_sched_barrier(0);
            // (the wave of a SIMD that is ahead stays ahead till its last products: one's exponentials then meet the other's products. 2 x 2048 queries over 12544
            // states 1.53 ms a call without, 1.50 with)
            if (N == kChunks && ch == 1) __builtin_amdgcn_s_setprio(1);
            if (N == kChunks && ch == N) __builtin_amdgcn_s_setprio(0);
            if (ch > 0) {
                bf16x8 vf[2][JB];
                read_values(vf[0], at + (ch - 1) * STEP);
                read_values(vf[1], at + (ch - 1) * STEP + CHUNK_BYTES / 2);
                __builtin_amdgcn_sched_barrier(0);
                if (ch < N) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) pv[i] = fast_exp2(fmaf(s[i], sc, -m_run));
                }
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int jb = 0; jb < JB; ++jb) o[jb] = mfma32(vf[u][jb], pf[u], o[jb]);
                if (ch < N) {
#pragma unroll
                    for (int i = 0; i < 2 * JB; ++i) {
                        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                        __builtin_amdgcn_sched_group_barrier(0x002, 16 / JB, 0);
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i) pv[i] = fast_exp2(fmaf(s[i], sc, -m_run));
            }
            __builtin_amdgcn_sched_barrier(0);
            if (ch == N) break;
            if (ch + 1 < N) {
                bf16x8 kf[KK];
                read_keys(kf, at + (ch + 1) * STEP);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < 16; ++i) psum += pv[i];
                s = logits(kf);
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    floatx8 pu;
#pragma unroll
                    for (int i = 0; i < 8; ++i) pu[i] = pv[8 * u + i];
                    pf[u] = __builtin_convertvector(pu, bf16x8);
                }
#pragma unroll
                for (int i = 0; i < KK; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x002, 24 / KK, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i) psum += pv[i];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    floatx8 pu;
#pragma unroll
                    for (int i = 0; i < 8; ++i) pu[i] = pv[8 * u + i];
                    pf[u] = __builtin_convertvector(pu, bf16x8);
                }
            }
            if (__builtin_expect(__any(!(psum <= fminf(kRowsRedo, kRowsPeak * l_run))), 0)) return ch;      // (these keys and the tile's others against another maximum)
            l_run += psum;
        }
        return N;
    };

    // The sweep.
    const auto sweep = [&] {
        begin_sums();
        if (tiles <= 0) return;
        uint64_t gone = 0;                                   // (pages) of 64 tiles, those with keys whose page is none
        for (int t = 0; t < tiles; ++t) {
            const int stage = t & 1;
            wait_vmcnt<0>();
            lds_done();
            stage_barrier();                             // the tile is there for everyone, and everyone has left the other stage
            if (t + 1 < tiles) issue(t + 1, stage ^ 1);
            if constexpr (PAGED) {
                if ((t & 63) == 0) {
                    gone = 0;
                    const uint64_t mine = plan.missing[t >> 6 & 1][lane % kRowsWaves];
                    if (__any(mine != 0))
#pragma unroll
                        for (int w = 0; w < kRowsWaves; ++w) gone |= lane_word(mine, w);
                }
            }
            if (!works) continue;
            const bool all_there = !PAGED || !(gone >> (t & 63) & 1);
            int ch0 = ks;
            if (n_ks <= 2 && !fresh && all_there && key0 + t * kRowsTile >= all_lo && key0 + (t + 1) * kRowsTile <= all_hi) {
                if (n_ks == 1) ch0 = whole_tile(std::integral_constant<int, kChunks>(), stage * 2 * TILE_BYTES);
                else ch0 = ks + 2 * whole_tile(std::integral_constant<int, kChunks / 2>(), stage * 2 * TILE_BYTES + ks * CHUNK_BYTES);
            }
            __builtin_amdgcn_s_setprio(0);                   // (keys were left)
            for (int ch = ch0; ch < kChunks; ch += n_ks) {
                const int k0 = key0 + t * kRowsTile + ch * 32;
                if (k0 >= any_hi || k0 + 31 < any_lo) continue;
                const uint32_t at_chunk = stage * 2 * TILE_BYTES + ch * CHUNK_BYTES;
                bf16x8 kf[KK], vf[2][JB];
                read_keys(kf, at_chunk);
                const floatx16 s = logits(kf);
                // (the reads of all of them first: one by one, each waits for its own)
                __builtin_amdgcn_sched_group_barrier(0x100, KK, 0);
                __builtin_amdgcn_sched_group_barrier(0x008, KK, 0);
                read_values(vf[0], at_chunk);
                float pv[16];
                uint32_t two = 0x101;
                if (!all_there) {
                    const auto there = [&](int half) { return (uint32_t)(__builtin_amdgcn_readfirstlane((int)(plan.missing[t >> 6 & 1][2 * ch + half] >> (t & 63))) & 1) ^ 1u; };
                    two = there(0) | there(1) << 8;
                }
                weigh(s, k0, two, pv);
                // ---- O^T += V^T P^T ----
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    floatx8 pu;
#pragma unroll
                    for (int i = 0; i < 8; ++i) pu[i] = pv[8 * u + i];
                    const bf16x8 pf = __builtin_convertvector(pu, bf16x8);
                    if (u == 0) read_values(vf[1], at_chunk + CHUNK_BYTES / 2);
                    if (PAGED && !(two >> (8 * u) & 1))      // (what lies in the place of a page that is none may be anything)
#pragma unroll
                        for (int jb = 0; jb < JB; ++jb) vf[u][jb] = __builtin_bit_cast(bf16x8, u32x4{});
#pragma unroll
                    for (int jb = 0; jb < JB; ++jb) o[jb] = mfma32(vf[u][jb], pf, o[jb]);
                    if (two_parts || peak) {
                        const u32x4 w = __builtin_bit_cast(u32x4, pf);
                        floatx8 rest;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            rest[2 * i] = pu[2 * i] - __uint_as_float(w[i] << 16);
                            rest[2 * i + 1] = pu[2 * i + 1] - __uint_as_float(w[i] & 0xffff0000u);
                        }
                        const bf16x8 pr = __builtin_convertvector(rest, bf16x8);
#pragma unroll
                        for (int jb = 0; jb < JB; ++jb) o[jb] = mfma32(vf[u][jb], pr, o[jb]);
                    }
                }
            }
        }
    };

    sweep();
    __syncthreads();                                         // everyone has left the tiles

    l_run = half_sum(l_run);
    int thread = threadIdx.x;
    held(thread);
    const SPECVLM_AS4 RowsParams& z = rows_params();
    const int row_in_block = thread & 31, half = thread >> 5 & 1;
    const auto inverse = [](float l) { return l > 0.f ? 1.f / l : l == 0.f ? 0.f : NAN; };
    // (the join looks after sums that are no finite numbers: such a row is not written here, where its queries may lie, and told of by a negative sum of its
    // probabilities)
    const auto tell = [&](int row, float m, float l, bool odd) { *reinterpret_cast<float2*>(z.part_ml + 2 * (pc.part + row)) = float2{m, odd ? -l : l}; };
    if (n_ks > 1) {
        // ---- waves that share rows: all sums to LDS (16-byte pieces of a row XORed by its number: its banks), then a row's four columns to a thread ----
        float* const s_o = (float*)in_lds<float>(lds0);
        if (works) {
            const int row = (ks * n_blocks + blk) * 32 + row_in_block;
            if (half == 0) *reinterpret_cast<float2*>(plan.ml + 2 * row) = float2{m_run, l_run};
#pragma unroll
            for (int jb = 0; jb < JB; ++jb)
#pragma unroll
                for (int i4 = 0; i4 < 4; ++i4)
                    *reinterpret_cast<floatx4*>(s_o + row * D + ((jb * 8 + i4 * 2 + half) ^ (row_in_block & (D / 4 - 1))) * 4) =
                        floatx4{o[jb][4 * i4], o[jb][4 * i4 + 1], o[jb][4 * i4 + 2], o[jb][4 * i4 + 3]};
        }
        __syncthreads();
        for (int at = thread; at < pc.n_rows * (D / 4); at += kRowsThreads) {
            const int row = at / (D / 4), c = at % (D / 4);
            float2 ml[kChunks];
            float m = -INFINITY, l = 0.f;
#pragma unroll
            for (int k = 0; k < kChunks; ++k) {
                ml[k] = k < n_ks ? *reinterpret_cast<const float2*>(plan.ml + 2 * (k * n_blocks * 32 + row)) : float2{-INFINITY, 0.f};
                m = fmaxf(m, ml[k].x);
            }
            const float m_ref = m == -INFINITY ? 0.f : m;
            floatx4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < kChunks; ++k) {
                if (k >= n_ks) break;
                const float w = fast_exp2(ml[k].x - m_ref);
                l += ml[k].y * w;
                const floatx4 y = *reinterpret_cast<const floatx4*>(s_o + (k * n_blocks * 32 + row) * D + (c ^ (row & 31 & (D / 4 - 1))) * 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[i] += y[i] * w;
            }
            if (pc.direct) {
                const QuotRem at_q = divide(pc.row0 + row, z.group, z.inv_group);
                const int64_t tok = pc.q0 + at_q.q;
                const int hd = pc.g * z.group + at_q.r;
                const bool odd = __ballot(!((sum[0] + sum[1] + sum[2] + sum[3]) * 0.f == 0.f)) >> (thread & 63 & ~(D / 4 - 1)) & (D == 128 ? 0xffffffffull : 0xffffull);
                if (!odd) *reinterpret_cast<bf16x4*>(z.out + tok * z.q_tok + (int64_t)hd * z.q_head + c * 4) = __builtin_convertvector(sum * inverse(l), bf16x4);
                if (z.lse && c == 0) z.lse[tok * z.n_q_heads + hd] = l == 0.f ? -INFINITY : (m + fast_log2(l)) * kLn2;
                if (c == 0) tell(row, m, l, odd);
            } else {
                *reinterpret_cast<floatx4*>(z.part_o + (pc.part + row) * D + c * 4) = sum;
                if (c == 0) tell(row, m, l, false);
            }
        }
    } else if (works && blk * 32 + row_in_block < pc.n_rows) {
        const int row = blk * 32 + row_in_block;
        if (pc.direct) {
            const QuotRem at_q = divide(pc.row0 + row, z.group, z.inv_group);
            const int64_t tok = pc.q0 + at_q.q;
            const int hd = pc.g * z.group + at_q.r;
            float odd = 0.f;
#pragma unroll
            for (int jb = 0; jb < JB; ++jb)
#pragma unroll
                for (int i = 0; i < 16; ++i) odd += 0.f * o[jb][i];
            odd = half_sum(odd);
            const float inv = inverse(l_run);
            __bf16* const op = z.out + tok * z.q_tok + (int64_t)hd * z.q_head + half * 4;
            if (odd == 0.f) {
#pragma unroll
                for (int jb = 0; jb < JB; ++jb)
#pragma unroll
                    for (int i4 = 0; i4 < 4; ++i4) {
                        const floatx4 y = floatx4{o[jb][4 * i4], o[jb][4 * i4 + 1], o[jb][4 * i4 + 2], o[jb][4 * i4 + 3]} * inv;
                        *reinterpret_cast<bf16x4*>(op + jb * 32 + i4 * 8) = __builtin_convertvector(y, bf16x4);
                    }
            }
            if (z.lse && half == 0) z.lse[tok * z.n_q_heads + hd] = l_run == 0.f ? -INFINITY : (m_run + fast_log2(l_run)) * kLn2;
            if (half == 0) tell(row, m_run, l_run, !(odd == 0.f));
        } else {
            if (half == 0) tell(row, m_run, l_run, false);
#pragma unroll
            for (int jb = 0; jb < JB; ++jb)
#pragma unroll
                for (int i4 = 0; i4 < 4; ++i4)
                    *reinterpret_cast<floatx4*>(z.part_o + (pc.part + row) * D + jb * 32 + i4 * 8 + half * 4) =
                        floatx4{o[jb][4 * i4], o[jb][4 * i4 + 1], o[jb][4 * i4 + 2], o[jb][4 * i4 + 3]};
        }
    }
}

__device__ __forceinline__ int first_of_last(int entries) { return (entries - 1) / kRowsThreads * kRowsThreads; }

template <int D, bool PAGED>
__global__ __launch_bounds__(kRowsThreads, 2)
void rows_kernel(const RowsParams p)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    extern __shared__ __align__(1024) unsigned char smem[];  // stage s: K tile at s * 2 * TILE_BYTES, V tile behind it
    RowsPlan& plan = *reinterpret_cast<RowsPlan*>(smem + 4 * Layout<D>::TILE);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(SPECVLM_AS3 unsigned char*)smem;

    // (neighbouring runs, which meet the same keys, on one XCD: 2 x 2048 queries over 12544 states 1.51 ms a call, dealt out over all of them 1.58)
    const int j = xcd_logical_id(blockIdx.x, p.padded);
    if (j >= p.workgroups) return;

    // ---- the numbering ----
    const int entries = p.entries;
    Numbers total, here;
    bool grouped = PAGED;
    const auto look_at = [&](int e) {                        // of 512 entries at a time, each thread one
        Entry entry;
        if (PAGED && entries <= kRowsThreads) entry = entry_at_once(p, plan, grouped);
        else entry = entry_of<PAGED>(p, e, grouped);
        const Numbers mine = numbers_of(p, entry), upto = block_prefix(plan, mine, wave, lane, &here);
        plan.entry[threadIdx.x] = entry;
        plan.front[threadIdx.x] = {upto.work - mine.work, upto.rows - mine.rows};
        plan.work[threadIdx.x] = mine.work;
        return mine.rows;
    };
    for (;;) {
        int64_t my_rows = 0;
        total = {0, 0};
        for (int c = first_of_last(entries); c >= 0; c -= kRowsThreads) {     // (the first 512 last: they are looked up next)
            my_rows += look_at(c + threadIdx.x);
            total.work += here.work;
            total.rows += here.rows;
        }
        // (groups that overlap would have rows more than once: there is no room for them)
        if (p.far && block_sum(plan, my_rows) > p.most_rows) total.rows = INT_MAX;
        if (total.rows <= p.most_rows || !grouped) break;
        grouped = false;
    }
    if (total.rows > p.most_rows) total.work = 0;            // (offsets that overlap)
    const Shares shares = shares_of(p, total.work);
    if (j >= shares.n) return;
    int x = shares.begin(j);
    const int x_end = shares.begin(j + 1);
    Walk at_hand = {{0, 0}, 0, entries <= kRowsThreads || j > 0};
    const Numbers& base = at_hand.base;
    const int& c0 = at_hand.c0;
    const auto tell = [&] {                                  // (the join reads where every entry begins)
        const int e = c0 + threadIdx.x;
        const Entry entry = plan.entry[threadIdx.x];
        const Numbers front = plan.front[threadIdx.x];
        if (e < entries)
            p.starts[e] = {base.work + front.work, base.rows + front.rows, entry.q0, entry.n_q, entry.key0, entry.key1, entry.first, total.work};
    };
    if (j == 0) tell();
    while (x < x_end || !at_hand.told) {
        while (at_hand.goes_on(x, x_end, here.work)) {
            at_hand.step(here, entries);
            __syncthreads();
            look_at(c0 + threadIdx.x);
            if (!at_hand.told) tell();
        }
        if (x >= x_end) break;
        const int there = base.work + plan.front[threadIdx.x].work;
        if (there <= x && x < there + plan.work[threadIdx.x]) plan.found = threadIdx.x;
        __syncthreads();
        const int at = __builtin_amdgcn_readfirstlane(plan.found), e = c0 + at;
        const Numbers front = {base.work + __builtin_amdgcn_readfirstlane(plan.front[at].work), base.rows + __builtin_amdgcn_readfirstlane(plan.front[at].rows)};
        const bool own = !PAGED || e >= p.batch;
        Entry en = plan.entry[at];
        en.q0 = __builtin_amdgcn_readfirstlane(en.q0); en.n_q = __builtin_amdgcn_readfirstlane(en.n_q);
        en.key0 = __builtin_amdgcn_readfirstlane(en.key0); en.key1 = __builtin_amdgcn_readfirstlane(en.key1);
        en.first = __builtin_amdgcn_readfirstlane(en.first);
        const int chunks = chunks_of(en), rows = en.n_q * p.group;
        const Sets sets = sets_of(rows, chunks);
        const int g = (int)((uint32_t)(x - front.work) / (uint32_t)sets.head), of_head = x - front.work - g * sets.head;
        const int set = min((int)((uint32_t)of_head / (uint32_t)sets.whole), sets.full), begin = of_head - set * sets.whole, unit = sets.unit_of(set);
        // (32 keys are a workgroup's that has their first unit)
        const auto chunk_at = [&](int u) { return max(0, unit == 2 ? (u - kBegin + 1) >> 1 : (int)((uint32_t)max(u - kBegin + 2, 0) / 3u)); };
        const int c_begin = chunk_at(begin), c_end = min(chunks, chunk_at(begin + x_end - x));
        x = min(x_end, x + chunks * unit + kBegin - begin);
        if (c_end <= c_begin) {                              // (the front of an item alone)
            __syncthreads();
            continue;
        }
        Piece pc;
        pc.b = !PAGED ? en.first : own ? e - p.batch : e; pc.own = own;
        pc.q0 = en.q0; pc.n_q = en.n_q; pc.end = en.key1;
        pc.g = g; pc.row0 = set * kSetRows; pc.n_rows = min(rows - pc.row0, kSetRows);
        pc.key0 = en.key0 + c_begin * 32; pc.key1 = min(en.key1, en.key0 + c_end * 32);
        pc.direct = own && !(PAGED && (en.key0 > 0 || p.over_q)) && c_begin == 0 && c_end == chunks;
        pc.part = part_row(j, front.rows + g * padded_rows(p, en) + pc.row0);
        rows_piece<D, PAGED>(plan, lds0, pc);
        __syncthreads();                                     // the ring, and what the plan holds, are free again
    }
}

// The shares up to those of 64 entries, a lane to each that has n, of which `before` are in front of them.  (What entries with queries in common have beyond the
// numbers that there are is not counted: an int holds it.)
__device__ __forceinline__ int shares_upto(const RowsParams& p, int before, int n) { return min(before, p.entries) + wave_prefix(n); }

// Each share of an entry's queries with the keys that any of them sees, a wave to a share: a workgroup's keys are then those that its rows see, and the work is
// dealt by them.
__global__ __launch_bounds__(256)
void rows_spans_kernel(const RowsParams p)
{
    const int lane = threadIdx.x & 63, e = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (e >= p.entries) return;
    int b = 0, of_entry = e;                                 // the entry, and the number in it
    if (p.cu_q) {
        b = -1;
        for (int c = 0, before = 0; c < p.batch && b < 0; c += kWave) {
            const int n = shares_of_entry(p, c + lane), upto = shares_upto(p, before, n);
            const uint64_t here = __ballot(upto - n <= e && e < upto);
            if (here) {
                const int i = __builtin_ctzll(here);
                b = c + i;
                of_entry = e - __builtin_amdgcn_readlane(upto - n, i);
            }
            before = __builtin_amdgcn_readlane(upto, kWave - 1);
        }
    }
    Entry s = {0, 0, 0, 0, b};
    if (b >= 0) {
        const int q0 = p.cu_q ? p.cu_q[b] : 0, n_q = p.cu_q ? p.cu_q[b + 1] - q0 : p.q_len, k0 = p.cu_kv ? p.cu_kv[b] : 0,
                  n = p.cu_kv ? p.cu_kv[b + 1] - k0 : p.kv_len;
        const int64_t at = (int64_t)of_entry * p.span;
        if (n_q > 0 && q0 >= 0 && q0 <= p.n_queries - n_q && n >= 0 && k0 >= 0 && k0 <= p.kv_len - n && at < n_q) {
            s.q0 = q0 + (int)at;
            s.n_q = min(p.span, n_q - (int)at);
            int lo = INT_MAX, hi = 0;
            for (int t = lane; t < s.n_q; t += kWave) {
                const int from = max(p.ranges[2 * (int64_t)(s.q0 + t)], 0), to = min(p.ranges[2 * (int64_t)(s.q0 + t) + 1], n);
                if (from < to) {
                    lo = min(lo, from);
                    hi = max(hi, to);
                }
            }
#pragma unroll
            for (int d = 1; d < kWave; d *= 2) {
                lo = min(lo, __shfl_xor(lo, d));
                hi = max(hi, __shfl_xor(hi, d));
            }
            s.key0 = min(lo, hi);
            s.key1 = hi;
        }
    }
    if (lane == 0) p.spans[e] = s;
}

// One row over all of its keys once more, by a wave, where its sum came out as no finite number: for an infinite value, which a row that sees it gets as it is,
// however small its weight, and a row that does not see it does not get, or for values whose sum is beyond 32 bits before it is divided.  m, l: the row's maximum and sum of probabilities.  (Every key takes its own loads and
// two rounds of the vector unit: 50 times what the matrix unit takes.)
template <int D, bool PAGED>
__device__ __forceinline__ void odd_row(const RowsParams& p, const RowsStart& own, int b, int tok, int hd, float m, float l, int lane)
{
    constexpr int COLS = D / kWave;
    const float sc = fmaxf(p.scale_log2, 1e-30f), m_ref = m == -INFINITY ? 0.f : m;
    const int g = hd / p.group, t = tok - own.q0;
    const __bf16* const q = p.q + (int64_t)tok * p.q_tok + (int64_t)hd * p.q_head;
    int lo = 0, hi = own.key1, before = own.key1;            // keys that the row sees;  of those from `before` on the tree's
    uint64_t tree = ~0ull;
    if constexpr (PAGED) {
        if (p.block_mask) {
            tree = p.block_mask[tok];
            before -= own.n_q;
        } else {
            hi -= own.n_q - 1 - t;
        }
    } else if (p.ranges) {
        lo = max(p.ranges[2 * (int64_t)tok], 0);
        hi = min(p.ranges[2 * (int64_t)tok + 1], own.key1);         // (what lies behind the share's keys is no range of its queries)
    }
    const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : NAN;      // (first of all: sums of the largest values stay within 32 bits so)
    float o[COLS];
#pragma unroll
    for (int c = 0; c < COLS; ++c) o[c] = 0.f;
    for (int k0 = lo; k0 < hi; k0 += kWave) {
        const int key = min(k0 + lane, hi - 1);
        bool sees = k0 + lane < hi && (key < before || (tree >> (key - before) & 1));
        int64_t at;
        if constexpr (PAGED) {
            const QuotRem pg = divide(key, p.page_size, p.inv_page);
            const int id = p.table[(int64_t)(key < own.key0 ? own.first : b) * p.table_row + pg.q];
            sees = sees && (uint32_t)id < (uint32_t)p.n_pages;
            at = (sees ? id : 0) * p.page + pg.r * p.tok;
        } else {
            at = (int64_t)((p.cu_kv ? p.cu_kv[b] : 0) + key) * p.tok;
        }
        at += (int64_t)g * p.head;
        float x = 0.f;
        for (int d = 0; d < D; d += 8) {
            const bf16x8 kv = *reinterpret_cast<const bf16x8*>(p.k + at + d), qv = *reinterpret_cast<const bf16x8*>(q + d);
#pragma unroll
            for (int i = 0; i < 8; ++i) x = fmaf((float)kv[i], (float)qv[i], x);
        }
        const float w = sees ? fast_exp2(fmaf(x, sc, -m_ref)) * inv : 0.f;
        uint64_t seen = __ballot(sees);
        while (seen) {
            const int i = __builtin_ctzll(seen);
            seen &= seen - 1;
            const float wi = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), i));
            const int64_t row = (int64_t)lane_word((uint64_t)at, i);
#pragma unroll
            for (int c = 0; c < COLS; ++c) {
                const float v = (float)p.v[row + lane * COLS + c];
                o[c] += fabsf(v) == INFINITY ? v : wi * v;
            }
        }
    }
    __bf16* const out = p.out + (int64_t)tok * p.q_tok + (int64_t)hd * p.q_head + lane * COLS;
#pragma unroll
    for (int c = 0; c < COLS; ++c) out[c] = (__bf16)o[c];
}

// Joins the pieces of the rows that were cut (one that was not is in its place already): D / 4 threads to a row, and `GP` groups of them take every GP-th
// of its pieces (GP = 1: a wave to as many rows as it holds, `TIMES` times: the token's request and entry, a look at memory after the other, are found once).
template <int D, bool PAGED, int GP, int TIMES>
__global__ __launch_bounds__(256)
void rows_join_kernel(const RowsParams p)
{
    constexpr int TPR = D / 4, RPW = kWave / TPR, WAVES = 4;       // threads of a row, rows of a wave
    static_assert(GP == 1 || GP == 256 / TPR, "a wave's row, or the workgroup's");
    __shared__ float s_ml[GP > 1 ? 2 * GP : 1];
    __shared__ __align__(16) float s_o[GP > 1 ? GP * D : 4];
    const int lane = threadIdx.x & 63, group = threadIdx.x / TPR, c = threadIdx.x % TPR;
    constexpr int HEADS = RPW * TIMES;
    const int units = (p.n_q_heads + HEADS - 1) / HEADS;
    int tok, hd0;
    if constexpr (GP == 1) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int64_t unit = (int64_t)blockIdx.x * WAVES + wave;
        tok = (int)(unit / units);
        hd0 = (int)(unit - (int64_t)tok * units) * HEADS;
    } else {
        tok = blockIdx.x / p.n_q_heads;
        hd0 = blockIdx.x - tok * p.n_q_heads;
    }
    if (tok >= p.n_queries) return;
    // the request;  (ranges) the shares in front of its own
    int b = 0, shares_before = 0;
    if (!p.cu_q) {
        b = PAGED ? tok / p.q_len : 0;
    } else {
        uint64_t behind = 0;
        for (; b < p.batch; b += kWave) {
            behind = __ballot(b + lane < p.batch && has_queries(p, b + lane) && p.cu_q[b + lane] <= tok && p.cu_q[b + lane + 1] > tok);
            if (!PAGED && p.ranges) {
                const int n = shares_of_entry(p, b + lane), upto = shares_upto(p, shares_before, n);
                shares_before = behind ? __builtin_amdgcn_readlane(upto - n, __builtin_ctzll(behind)) : __builtin_amdgcn_readlane(upto, kWave - 1);
            }
            if (behind) break;
        }
        if (!behind) return;                                 // (a row of no request)
        b += __builtin_ctzll(behind);
    }
    int e = PAGED ? p.batch + b : b;
    if (!PAGED && p.ranges) {
        e = shares_before + divide(tok - (p.cu_q ? p.cu_q[b] : 0), p.span, p.inv_span).q;
        if (e >= p.entries) return;                          // (there is none for queries of so many entries)
    }
    const RowsStart own = p.starts[e];
    const int total = own.total;
    const Shares shares = shares_of(p, total);
    if (total == 0 || own.n_q <= 0 || tok < own.q0) return;
    struct Pieces { int first, n, row; };                    // workgroups that have one, the row of their results
    const auto pieces_of = [&](const RowsStart& s, const QuotRem& head) {
        const Entry en = {s.q0, s.n_q, s.key0, s.key1, -1};
        const int row = (tok - en.q0) * p.group + head.r, chunks = chunks_of(en);
        const Sets sets = sets_of(en.n_q * p.group, chunks);
        const int set = row / kSetRows, unit = sets.unit_of(set), x = s.work + head.q * sets.head + set * sets.whole + kBegin;
        const int first = shares.of(x);
        return Pieces{first, shares.of(x + (chunks - 1) * unit) - first + 1, s.rows + head.q * padded_rows(p, en) + row};
    };
    const bool shares_keys = PAGED && own.key0 > 0;
    const RowsStart first = shares_keys ? p.starts[own.first] : own;
    // of the wave's heads, those that something is to be done for:  a row in one piece of finite sums is in its place
    uint64_t todo = ~0ull;
    if (TIMES > 1 && !shares_keys) {
        const int hd = hd0 + lane;
        bool mine = false;
        if (lane < HEADS && hd < p.n_q_heads) {
            const Pieces pieces = pieces_of(own, divide(hd, p.group, p.inv_group));
            mine = pieces.n != 1 || (PAGED && p.over_q);
            if (!mine) {
                const float l = p.part_ml[2 * part_row(pieces.first, pieces.row) + 1];
                mine = __float_as_uint(l) >> 31 || !(l == l);
            }
        }
        todo = __ballot(mine);
    }
    for (int k = 0; k < TIMES; ++k) {
        if (!(todo >> (k * RPW) & ((1u << RPW) - 1)) || hd0 + k * RPW >= p.n_q_heads) continue;
        const int of_lane = hd0 + k * RPW + (GP == 1 ? lane / TPR : 0), hd = min(of_lane, p.n_q_heads - 1);
        const bool mine_to_write = of_lane < p.n_q_heads && (GP == 1 || group == 0);      // (all lanes stay to the end: an odd row takes a whole wave)
        const QuotRem head = divide(hd, p.group, p.inv_group);
        const Pieces mine = pieces_of(own, head);
        Pieces theirs = {0, 0, 0};
        if (shares_keys) theirs = pieces_of(first, head);
        float m = -INFINITY, l = 0.f;
        floatx4 o = {0.f, 0.f, 0.f, 0.f};
        bool odd = false;
        const bool in_place = theirs.n == 0 && mine.n == 1 && !(PAGED && p.over_q);
        if (in_place) {
            const float2 ml = *reinterpret_cast<const float2*>(p.part_ml + 2 * part_row(mine.first, mine.row));
            odd = __float_as_uint(ml.y) >> 31 || !(ml.y == ml.y);
            m = ml.x;
            l = fabsf(ml.y);
        }
        const int n = in_place ? 0 : theirs.n + mine.n;
        const auto row_of = [&](int i) { return i < theirs.n ? part_row(theirs.first + i, theirs.row) : part_row(mine.first + i - theirs.n, mine.row); };
        const int g0 = GP == 1 ? 0 : group;                      // this group's first piece
        for (int i0 = g0; i0 < n; i0 += TPR * GP) {
            // a piece to a thread: its maximum and sum;  then the outputs, weighted by their thread's word
            float pm = -INFINITY, pl = 0.f;
            if (i0 + c * GP < n) {
                const float2 ml = *reinterpret_cast<const float2*>(p.part_ml + 2 * row_of(i0 + c * GP));
                pm = ml.x;
                pl = ml.y;
            }
            const int most = min(TPR, (n - i0 + GP - 1) / GP);
            floatx4 y[4];
            const auto fetch = [&](int i1) {                     // (behind the last piece: the last again, left out)
#pragma unroll
                for (int u = 0; u < 4; ++u) y[u] = *reinterpret_cast<const floatx4*>(p.part_o + row_of(i0 + min(i1 + u, most - 1) * GP) * D + c * 4);
            };
            fetch(0);
            float top = pm;
#pragma unroll
            for (int d = 1; d < TPR; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
            const float m_new = fmaxf(m, top), m_ref = m_new == -INFINITY ? 0.f : m_new;
            const float w = fast_exp2(pm - m_ref), keep = fast_exp2(m - m_ref);
            float sum = pl * w;
#pragma unroll
            for (int d = 1; d < TPR; d *= 2) sum += __shfl_xor(sum, d);
            l = l * keep + sum;
            m = m_new;
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = o[i] * keep;
            for (int i1 = 0; i1 < most; i1 += 4) {
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const float wi = __shfl(w, (lane & ~(TPR - 1)) + min(i1 + u, most - 1));
                    if (i1 + u < most)
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[i] += y[u][i] * wi;
                }
                if (i1 + 4 < most) fetch(i1 + 4);
            }
        }
        if (GP > 1 && !in_place) {
            if (c == 0) { s_ml[2 * group] = m; s_ml[2 * group + 1] = l; }
            *reinterpret_cast<floatx4*>(s_o + group * D + c * 4) = o;
            __syncthreads();
            for (int j = 0; j < GP; ++j) m = fmaxf(m, s_ml[2 * j]);
            const float m_ref = m == -INFINITY ? 0.f : m;
            l = 0.f;
            o = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < GP; ++j) {
                const float w = fast_exp2(s_ml[2 * j] - m_ref);
                l += s_ml[2 * j + 1] * w;
                const floatx4 y = *reinterpret_cast<const floatx4*>(s_o + j * D + c * 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] += y[i] * w;
            }
        }
        const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : NAN;
        if (!in_place) {
            const uint64_t odds = __ballot(!((o[0] + o[1] + o[2] + o[3]) * 0.f == 0.f));
            odd = odds >> (lane & ~(TPR - 1)) & (D == 128 ? 0xffffffffull : 0xffffull);
            if (mine_to_write) {
                if (!odd) *reinterpret_cast<bf16x4*>(p.out + (int64_t)tok * p.q_tok + (int64_t)hd * p.q_head + c * 4) = __builtin_convertvector(o * inv, bf16x4);
                if (p.lse && c == 0) p.lse[(int64_t)tok * p.n_q_heads + hd] = l == 0.f ? -INFINITY : (m + fast_log2(l)) * kLn2;
            }
        }
        for (uint64_t rows = __ballot(odd && mine_to_write && c == 0); __builtin_expect(rows != 0, 0); rows &= rows - 1) {
            const int i = __builtin_ctzll(rows);
            odd_row<D, PAGED>(p, own, b, tok, __builtin_amdgcn_readlane(hd, i), __shfl(m, i), __shfl(l, i), lane);
        }
    }
}

namespace {

// What a call numbers: requests' shared and own keys;  entries;  or, with ranges, shares of the entries' queries, as many queries as fill a set of rows.
int rows_span(int n_q_heads, int n_kv_heads) { const int group = n_q_heads / n_kv_heads; return group < kSetRows ? kSetRows / group : 1; }
int64_t rows_entries(bool paged, bool ranges, int batch, int n_queries, int n_q_heads, int n_kv_heads)
{
    return paged ? 2 * (int64_t)batch : ranges ? (int64_t)batch + n_queries / rows_span(n_q_heads, n_kv_heads) + 1 : batch;
}
// Rows of partial results: 256 for every workgroup, and those of all entries, each a multiple of 32 (a query is in one entry of own keys and at most one of
// shared ones, of which there are at most half as many as requests).
int64_t rows_parts(bool paged, bool ranges, int workgroups, int batch, int n_queries, int n_q_heads, int n_kv_heads)
{
    const int64_t rows = (int64_t)n_queries * n_q_heads * (paged ? 2 : 1),
                  entries = paged ? batch + batch / 2 : rows_entries(paged, ranges, batch, n_queries, n_q_heads, n_kv_heads);
    return (int64_t)workgroups * kSetRows + rows + entries * 32 * n_kv_heads;
}
// (asked without knowing of ranges: with them there are more entries)
size_t rows_workspace(bool paged, int batch, int n_queries, int n_q_heads, int n_kv_heads, int head_dim)
{
    const size_t rows = (size_t)rows_parts(paged, true, kNumCu, batch, n_queries, n_q_heads, n_kv_heads);
    const size_t entries = (size_t)rows_entries(paged, true, batch, n_queries, n_q_heads, n_kv_heads);
    return align256(rows * head_dim * sizeof(float)) + align256(rows * 2 * sizeof(float)) + align256(entries * sizeof(RowsStart)) + align256(entries * sizeof(Entry));
}
// Whether rows, and rows of partial results, are ints.  (Entries by themselves first: 32 times any number of them and of heads would pass 64 bits.)
bool rows_fit(bool paged, bool ranges, int batch, int n_queries, int n_q_heads, int n_kv_heads)
{
    const int64_t entries = rows_entries(paged, ranges, batch, n_queries, n_q_heads, n_kv_heads), most = (int64_t)1 << 29;
    return (int64_t)n_queries * n_q_heads < most && entries < most / 32 && entries * 32 * n_kv_heads < most;
}
// (no workspace for what the call refuses)
bool rows_shape(bool paged, int batch, int n_queries, int n_q_heads, int n_kv_heads, int head_dim)
{
    return batch > 0 && n_queries > 0 && n_kv_heads > 0 && n_q_heads > 0 && n_q_heads % n_kv_heads == 0 && (head_dim == 64 || head_dim == 128) &&
           rows_fit(paged, false, batch, n_queries, n_q_heads, n_kv_heads);
}

template <int D, bool PAGED>
int launch_rows(RowsParams& p, hipStream_t stream)
{
    constexpr int lds = 4 * Layout<D>::TILE + (int)sizeof(RowsPlan);
    static_assert(lds <= 160 * 1024, "a CU's");
    if (const int rc = allow_lds<&rows_kernel<D, PAGED>>(lds)) return rc;
    const int64_t rows = (int64_t)p.n_queries * p.n_q_heads;
    // Few rows of long keys have many pieces each: a workgroup to a row (8 tokens of 64 heads over 30000 states 36.7 us a call with a wave to two rows, so 33.3;
    // but 32 tokens over 2500 46.4 and 48.6, one of 14 heads over 1254 11.2 and 12.3).  Where there are more rows than waves for long, a wave looks at 8 heads of its token at once, of
    // which those in place cost no more than that look (2 texts of 2048 tokens and 64 heads 39 us, now 13;  but 60 thousand rows with two pieces each 18 and 24).
    const bool few = rows <= 512 && p.kv_len >= 2048, many = rows > 131072;
    const int heads = 256 / D * (many ? 8 : 1), units = (p.n_q_heads + heads - 1) / heads;
    const int64_t joins = few ? rows : ((int64_t)p.n_queries * units + 3) / 4;
    if (!launchable(joins, 256)) return SPECVLM_EUNSUPPORTED;
    if (!PAGED && p.ranges) {
        rows_spans_kernel<<<(p.entries + 3) / 4, 256, 0, stream>>>(p);
        if (const int rc = launch_status()) return rc;
    }
    p.workgroups = kNumCu;
    p.padded = round_up(p.workgroups, kNumXcd);
    rows_kernel<D, PAGED><<<p.padded, kRowsThreads, lds, stream>>>(p);
    if (const int rc = launch_status()) return rc;
    if (few) rows_join_kernel<D, PAGED, 1024 / D, 1><<<(unsigned)joins, 256, 0, stream>>>(p);
    else if (many) rows_join_kernel<D, PAGED, 1, 8><<<(unsigned)joins, 256, 0, stream>>>(p);
    else rows_join_kernel<D, PAGED, 1, 1><<<(unsigned)joins, 256, 0, stream>>>(p);
    return launch_status();
}

// What both calls ask of the queries, and what they share of the parameters.
int rows_start(RowsParams& p, bool paged, const void* q, int64_t q_tok, int64_t q_head, const void* k, const void* v, int64_t tok, int64_t head, int batch,
               int n_queries, int most_keys, int n_q_heads, int n_kv_heads, int head_dim, float scale, const int32_t* key_ranges, void* out, float* lse,
               void* workspace, size_t workspace_bytes)
{
    if (!q || !out || ((!k || !v) && most_keys > 0)) return SPECVLM_EINVAL;
    if ((q_tok | q_head | tok | head) & 7) return SPECVLM_EUNSUPPORTED;
    if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)out) & 15) return SPECVLM_EUNSUPPORTED;
    // (a lane's offset inside 16 keys has 32 bits; rows, and tiles of all sets and heads, are ints)
    if (tok < 0 || tok >= ((int64_t)1 << 26)) return SPECVLM_EUNSUPPORTED;
    const bool ranges = key_ranges != nullptr;
    if (!rows_fit(paged, ranges, batch, n_queries, n_q_heads, n_kv_heads)) return SPECVLM_EUNSUPPORTED;
    const int64_t rows = (int64_t)n_queries * n_q_heads, entries = rows_entries(paged, ranges, batch, n_queries, n_q_heads, n_kv_heads);
    const int64_t sets = (2 * rows / kSetRows + n_kv_heads) + entries * n_kv_heads;
    if (sets * 3 * (most_keys / 32 + 10) >= ((int64_t)1 << 31)) return SPECVLM_EUNSUPPORTED;
    const size_t need = rows_workspace(paged, batch, n_queries, n_q_heads, n_kv_heads, head_dim);
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < need) return SPECVLM_EWORKSPACE;
    p = {};
    p.q = (const __bf16*)q; p.k = (const __bf16*)k; p.v = (const __bf16*)v; p.out = (__bf16*)out; p.lse = lse;
    p.q_tok = q_tok; p.q_head = q_head; p.tok = tok; p.head = head;
    p.batch = batch; p.n_queries = n_queries; p.kv_len = most_keys;
    p.n_q_heads = n_q_heads; p.n_kv_heads = n_kv_heads; p.group = n_q_heads / n_kv_heads;
    p.inv_group = reciprocal(p.group);
    p.scale_log2 = scale * kLog2e;
    p.most_rows = (int)rows_parts(paged, ranges, 0, batch, n_queries, n_q_heads, n_kv_heads);
    p.over_q = q == out;
    p.far = entries * (rows + 32 * n_kv_heads) > INT_MAX;
    p.entries = (int)entries; p.ranges = key_ranges; p.span = rows_span(n_q_heads, n_kv_heads);
    p.inv_span = reciprocal(p.span);
    const size_t parts = (size_t)rows_parts(paged, true, kNumCu, batch, n_queries, n_q_heads, n_kv_heads);
    p.part_o = (float*)workspace;
    p.part_ml = (float*)((char*)workspace + align256(parts * head_dim * sizeof(float)));
    p.starts = (RowsStart*)((char*)p.part_ml + align256(parts * 2 * sizeof(float)));
    p.spans = (Entry*)((char*)p.starts + align256((size_t)rows_entries(paged, true, batch, n_queries, n_q_heads, n_kv_heads) * sizeof(RowsStart)));
    return SPECVLM_OK;
}

}  // namespace
}  // namespace specvlm

using namespace specvlm;

extern "C" size_t specvlm_shared_attn_workspace_bytes(int batch, int n_queries, int n_q_heads, int n_kv_heads, int head_dim)
{
    return rows_shape(true, batch, n_queries, n_q_heads, n_kv_heads, head_dim) ? rows_workspace(true, batch, n_queries, n_q_heads, n_kv_heads, head_dim) : 0;
}

extern "C" int specvlm_shared_attn(
    const void* q, int64_t q_tok_stride, int64_t q_head_stride,
    const void* k_pages, const void* v_pages, int64_t page_stride, int64_t tok_stride, int64_t head_stride,
    int n_pages, int page_size, const int32_t* page_table, int64_t table_stride, int max_pages,
    const int32_t* kv_lens, const int32_t* groups, const int32_t* cu_q, int batch, int n_queries, int q_len, int kv_len,
    int n_q_heads, int n_kv_heads, int head_dim, float softmax_scale,
    const uint64_t* ancestor_mask, void* out, float* lse,
    void* workspace, size_t workspace_bytes, void* stream)
{
    if (batch < 0 || n_queries < 0 || q_len < 0 || kv_len < 0 || n_q_heads <= 0 || n_kv_heads <= 0 || n_pages < 0 || max_pages < 0) return SPECVLM_EINVAL;
    if (n_q_heads % n_kv_heads || page_size <= 0) return SPECVLM_EINVAL;
    if (!(softmax_scale >= 0.f) || !(softmax_scale < INFINITY)) return SPECVLM_EINVAL;
    if ((head_dim != 64 && head_dim != 128) || page_size % 16 || (ancestor_mask && q_len > kMaxQueryBlock)) return SPECVLM_EUNSUPPORTED;
    if (batch == 0 || q_len == 0 || n_queries == 0) return SPECVLM_OK;
    if (!cu_q && (int64_t)batch * q_len != n_queries) return SPECVLM_EINVAL;
    if (q_len > kv_len || kv_len > (int64_t)max_pages * page_size || n_pages == 0 || table_stride < 0) return SPECVLM_EINVAL;
    if (!page_table || !kv_lens || !groups) return SPECVLM_EINVAL;
    if (page_stride & 7 || kv_len > (1 << 30)) return SPECVLM_EUNSUPPORTED;
    RowsParams p;
    if (const int rc = rows_start(p, true, q, q_tok_stride, q_head_stride, k_pages, v_pages, tok_stride, head_stride, batch, n_queries, kv_len, n_q_heads,
                                  n_kv_heads, head_dim, softmax_scale, nullptr, out, lse, workspace, workspace_bytes))
        return rc;
    p.page = page_stride; p.n_pages = n_pages; p.page_size = page_size; p.inv_page = reciprocal(page_size);
    p.table = page_table; p.table_row = table_stride;
    p.kv_lens = kv_lens; p.groups = groups; p.cu_q = cu_q; p.q_len = q_len; p.block_mask = ancestor_mask;
    return head_dim == 128 ? launch_rows<128, true>(p, (hipStream_t)stream) : launch_rows<64, true>(p, (hipStream_t)stream);
}

extern "C" size_t specvlm_cross_attn_workspace_bytes(int batch, int n_queries, int n_q_heads, int n_kv_heads, int head_dim)
{
    return rows_shape(false, batch, n_queries, n_q_heads, n_kv_heads, head_dim) ? rows_workspace(false, batch, n_queries, n_q_heads, n_kv_heads, head_dim) : 0;
}

extern "C" int specvlm_cross_attn(
    const void* q, int64_t q_tok_stride, int64_t q_head_stride,
    const void* k, const void* v, int64_t kv_tok_stride, int64_t kv_head_stride,
    const int32_t* cu_q, const int32_t* cu_kv, int batch, int n_queries, int n_states,
    int n_q_heads, int n_kv_heads, int head_dim, float softmax_scale,
    const int32_t* key_ranges, void* out, float* lse,
    void* workspace, size_t workspace_bytes, void* stream)
{
    if (batch < 0 || n_queries < 0 || n_states < 0 || n_q_heads <= 0 || n_kv_heads <= 0 || n_q_heads % n_kv_heads) return SPECVLM_EINVAL;
    if (!(softmax_scale >= 0.f) || !(softmax_scale < INFINITY)) return SPECVLM_EINVAL;
    if ((cu_q == nullptr) != (cu_kv == nullptr) || (!cu_q && batch > 1)) return SPECVLM_EINVAL;
    if (head_dim != 64 && head_dim != 128) return SPECVLM_EUNSUPPORTED;
    if (batch == 0 || n_queries == 0) return SPECVLM_OK;
    if (n_states > (1 << 30)) return SPECVLM_EUNSUPPORTED;
    RowsParams p;
    if (const int rc = rows_start(p, false, q, q_tok_stride, q_head_stride, k, v, kv_tok_stride, kv_head_stride, batch, n_queries, n_states, n_q_heads,
                                  n_kv_heads, head_dim, softmax_scale, key_ranges, out, lse, workspace, workspace_bytes))
        return rc;
    p.cu_q = cu_q; p.cu_kv = cu_kv; p.q_len = n_queries;
    return head_dim == 128 ? launch_rows<128, false>(p, (hipStream_t)stream) : launch_rows<64, false>(p, (hipStream_t)stream);
}
