// specvlm_paged_attn: grouped-query softmax attention of a short query block (one token, a verified chain, a draft
// tree) over a bf16 KV cache held in pages, with every key visible or only the first ones and a window of the last.
//
// Mathematics.  One pass over the keys with the running maximum m and sum l of each query row (online softmax); the
// key range of a request is cut into pieces, and pieces are joined by  o = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s.
// All statistics, sums and partial outputs are fp32; the probabilities go through the matrix instruction as two bf16
// each (16 bits), the output is rounded once.
//
// Bound.  Every visible K and V row is read once for up to 64 query rows of a kv head: HBM for long caches, launches and
// round trips for short ones.
//
// Pages.  A page holds a multiple of 16 keys, so 16 consecutive keys starting at a multiple of 16 lie in one page and
// one scalar table lookup serves them: the address of a wave-wide load is a scalar base plus a lane offset that never
// changes.  The loader waves look up the pages of a tile one tile before they load it.  With a window the keys are
// swept in the order  first keys (rounded up to 16), then the window (rounded down to 16): the pages between are never
// looked at, and may have been freed.
//
// Work decomposition.  The lengths are on the device.  Tiles of 64 keys of all requests are numbered request after
// request; group j (a workgroup for each kv head and row group) takes a run of equal length, which every workgroup
// finds by a prefix sum over the lengths, 64 requests at a time in the lanes of a wave.  A captured launch so stays
// balanced as the caches grow.  A request that one group covers is written out directly; the others leave partial
// results that the second launch joins.
//
// A workgroup has MB*KS compute waves (row block mb, every KS-th 32-key chunk of a tile) and NLD loader waves that only issue
// direct-to-LDS loads into a ring of NS tiles (see decode_attn.hip for the matrix formulation and the swizzles).
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
    uint32_t inv_page, inv_heads, inv_all_heads, inv_group, inv_rgroups;
    float scale_log2;
    int n_rgroups, rows_pad, max_groups;
    float* part_o;           // [(groups + batch) * H_kv][rows_pad][D] unnormalised partial outputs
    float* part_ml;          // [(groups + batch) * H_kv][rows_pad][2] running maximum in log2 units, sum
};

constexpr int kTileKeys = 64;
constexpr int kMinRun = 2;               // tiles a group takes at least
constexpr int kTargetGroups = 256;       // workgroups of a launch

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
__device__ __forceinline__ int paged_tiles(const PagedParams& p, int b)
{
    const int ql = p.cu_q ? p.cu_q[b + 1] - p.cu_q[b] : p.q_len;
    return (paged_view(p, ql, p.kv_lens[b]).n + kTileKeys - 1) / kTileKeys;
}

__device__ __forceinline__ int wave_prefix(int x, int lane)            // sum over the lanes up to this one
{
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const int y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    return x;
}
__device__ __forceinline__ int wave_total(int x)
{
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) x += __shfl_xor(x, d);
    return __builtin_amdgcn_readfirstlane(x);
}
// Tiles of the whole batch (all lanes of a wave together).
__device__ __forceinline__ int paged_total(const PagedParams& p, int lane)
{
    if (p.batch == 1) return paged_tiles(p, 0);
    int n = 0;
    for (int c = 0; c < p.batch; c += kWave) n += c + lane < p.batch ? paged_tiles(p, c + lane) : 0;
    return wave_total(n);
}
// Tiles that a group takes.
__device__ __forceinline__ int paged_run(const PagedParams& p, int total) { return max(kMinRun, (total + p.max_groups - 1) / p.max_groups); }

template <int D, int MB, int KS, int NS, int NLD, bool STREAM>
__global__ __launch_bounds__((MB * KS + NLD) * kWave)
void paged_split_kernel(const PagedParams p)
{
    constexpr int TK = kTileKeys;
    constexpr int NW = MB * KS;                  // compute waves (the loader waves come after them)
    constexpr int DJ = D / 16, KK = D / 32, CH = D / 8, ROW_BYTES = D * 2;
    constexpr int KEYS_PER_LOAD = kWave / CH;    // key rows of one wave-wide load (4 or 8)
    constexpr int TILE_BYTES = TK * ROW_BYTES;   // one of K or V
    constexpr int LOADS_PER_MAT = TK / KEYS_PER_LOAD;
    constexpr int LPW = 2 * LOADS_PER_MAT / NLD; // loads of a loader wave per tile: the first half of the waves K, the others V
    constexpr int GPW = LPW * KEYS_PER_LOAD / 16;        // groups of 16 keys of a loader wave
    constexpr int LPG = 16 / KEYS_PER_LOAD;      // loads per group
    constexpr int LDS_STRIDE = D + 4;
    static_assert(TK / kChunkKeys == KS, "one chunk of a tile per key-split wave");
    static_assert(NLD == 2 || NLD == 4, "loader waves");

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool is_loader = wave >= NW;
    const int lw = wave - NW;                    // loader index
    const int mb = wave % MB, ks = wave / MB;    // (compute waves)
    const int r = lane & 15, c = lane >> 4;

    extern __shared__ __align__(16) unsigned char smem[];        // stage s: K tile at s*2*TILE_BYTES, V tile right after it
    uint32_t* const s_ok = reinterpret_cast<uint32_t*>(smem + NS * 2 * TILE_BYTES);     // per stage a byte per 16 keys: their page is there

    const QuotRem head = divide(blockIdx.x, p.n_kv_heads, p.inv_heads), rows_of = divide(head.q, p.n_rgroups, p.inv_rgroups);
    const int g = head.r, row0 = rows_of.r * (MB * 16), j = rows_of.q;

    // loader: this wave's matrix, its first group of a tile, and the lane offsets of the loads of a group
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
    const float sc = fmaxf(p.scale_log2, 1e-30f);                 // (a zero scale as a vanishing one: -inf stays -inf)

    // Tiles [t_begin, t_end) of request b; the result goes to partial slot slot0 + row, or straight to the output.
    auto piece = [&](const int b, const int t_begin, const int t_end, const int64_t slot0, const bool direct) {
    const int q0 = p.cu_q ? p.cu_q[b] : b * p.q_len, ql = p.cu_q ? p.cu_q[b + 1] - q0 : p.q_len, kvl = p.kv_lens[b];
    const PagedView view = paged_view(p, ql, kvl);
    const int n_rows = p.group * ql, n = view.n;
    if (row0 >= n_rows) return;
    const int n_tiles = t_end - t_begin;                          // >= 1

    float m_run = -INFINITY, l_run = 0.f;
    floatx4 o_acc[DJ];
#pragma unroll
    for (int jj = 0; jj < DJ; ++jj) o_acc[jj] = floatx4{0.f, 0.f, 0.f, 0.f};

    if (is_loader) {
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
                                                     (SPECVLM_AS3 void*)(st + (i * LPG + l) * 1024), 16, 0, STREAM ? 2 : 0);
            }
            if (!is_v && lane == 0) {
                if constexpr (GPW == 4) s_ok[stage] = ok;
                else reinterpret_cast<uint16_t*>(s_ok + stage)[lw] = (uint16_t)ok;
            }
        };
        const int n_load = n_tiles > NS - 1 ? n_tiles : NS - 1;   // (a run shorter than the ring loads its last tile again)
        look_up(t_begin);
#pragma unroll
        for (int s = 0; s < NS - 1; ++s) {
            issue_tile(s);
            look_up(t_begin + min(s + 1, n_tiles - 1));
        }
        int i = 0;
        do {
            const int younger = min(NS - 2, n_load - 1 - i);      // tiles in flight behind tile i
            wait_vmcnt<(NS - 2) * LPW>();
            if constexpr (NS >= 4) { if (younger <= 1) wait_vmcnt<1 * LPW>(); }
            if constexpr (NS >= 3) { if (younger <= 0) wait_vmcnt<0>(); }
            __asm__ volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the bytes of s_ok are written
            stage_barrier();                                      // tile i landed for everyone; stage (i-1)%NS is free
            if (i + NS - 1 < n_load) {
                issue_tile((i + NS - 1) % NS);
                look_up(t_begin + min(i + NS, n_tiles - 1));
            }
        } while (++i < n_tiles);
        wait_vmcnt<0>();                                          // (spare copies may still be landing)
    } else {
        bf16x8 qf[KK];
        const int row = row0 + mb * 16 + r;
        const QuotRem at = divide(row < n_rows ? row : 0, p.group, p.inv_group);     // (padding rows take row 0: never stored)
        const int t_blk = at.q;
        const __bf16* qp = p.q + (int64_t)(q0 + t_blk) * p.q_tok + (int64_t)(g * p.group + at.r) * p.q_head + c * 8;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) qf[kk] = *reinterpret_cast<const bf16x8*>(qp + kk * 32);
        // places [n_sinks, edge) hold keys that the window hides from some query
        const int edge = p.window ? kvl - p.window - view.skip : 0;
        int i = 0;
        do {
            stage_barrier();
            const unsigned char* const kt = smem + (i % NS) * (2 * TILE_BYTES);
            const unsigned char* const vt = kt + TILE_BYTES;
            const int base = (t_begin + i) * TK + ks * kChunkKeys;
            if (base >= n) continue;
            const uint32_t ok = (uint32_t)__builtin_amdgcn_readfirstlane(s_ok[i % NS]) >> (16 * ks);
            // ---- S^T = K Q^T for 32 keys ----
            floatx4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                const int x = kk * 4 + c;
                const int key0 = ks * kChunkKeys + r;
                const int sw = (D == 128) ? (r & 15) : ((r >> 1) & 7);          // (the same for row r + 16)
                const u32x4 k0 = *reinterpret_cast<const u32x4*>(kt + key0 * ROW_BYTES + ((x ^ sw) * 16));
                const u32x4 k1 = *reinterpret_cast<const u32x4*>(kt + (key0 + 16) * ROW_BYTES + ((x ^ sw) * 16));
                s0 = mfma16(__builtin_bit_cast(bf16x8, k0), qf[kk], s0);
                s1 = mfma16(__builtin_bit_cast(bf16x8, k1), qf[kk], s1);
            }
            float s[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) { s[e] = s0[e]; s[4 + e] = s1[e]; }
            // ---- V^T fragments of the lane's keys (4c+e and 16+4c+e) by the transposing LDS read ----
            bf16x8 vf[DJ];
            {
                const int kl = ks * kChunkKeys + 4 * c + (r >> 2);
                const int pair_swz = v_swizzle<D>(kl) >> 1;                     // same for kl + 16
                const unsigned char* const vrow = vt + kl * ROW_BYTES + (r & 3) * 8;
#pragma unroll
                for (int jj = 0; jj < DJ; ++jj) {
                    typedef short s16x4 __attribute__((ext_vector_type(4)));
                    const unsigned char* const src = vrow + (jj ^ pair_swz) * 32;
                    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SPECVLM_AS3 s16x4*)src);
                    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SPECVLM_AS3 s16x4*)(src + 16 * ROW_BYTES));
                    vf[jj] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                }
            }
            const bool need_mask = (ok & 0xffffu) != 0x0101u || base + kChunkKeys > n - ql || (base < edge && base + kChunkKeys > p.n_sinks);
            if (need_mask) {
                // block key b is visible where bit b is set: 0..t in a chain, the caller's ancestors in a tree
                const uint64_t row_mask = p.block_mask ? p.block_mask[q0 + t_blk] : ((2ull << t_blk) - 1ull);
                const uint32_t mask_lo = (uint32_t)row_mask, mask_hi = (uint32_t)(row_mask >> 32);
                const int hidden_to = p.window ? kvl - ql + t_blk - p.window : -1;          // the window's last hidden key
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int x0 = base + (e < 4 ? 0 : 16), key = (x0 < view.sinks ? x0 : x0 + view.skip) + 4 * c + (e & 3);
                    const int bk = key - (kvl - ql);                                    // (negative: a context key)
                    const uint32_t bit = (((bk & 32) ? mask_hi : mask_lo) >> (bk & 31)) & 1u;
                    const bool hidden = (((ok >> (e < 4 ? 0 : 8)) & 1u) == 0u) | (key >= kvl) | ((key <= hidden_to) & (key >= p.n_sinks)) |
                                        ((bk >= 0) & (bit == 0u));
                    s[e] = hidden ? -INFINITY : s[e];
                }
            }
            // Away from the masks the exponentials are taken against the reference that the earlier chunks left, and the
            // maximum is tracked only where a lane's sum does not stay moderate (see decode_attn.hip).
            floatx8 pv;
            bool settled = false;
            if (!need_mask && !__any(!(m_run > -INFINITY))) {
                float psum = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) { pv[e] = fast_exp2(fmaf(s[e], sc, -m_run)); psum += pv[e]; }
                if (!__any(!(psum < kSumRedo))) {
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
                    for (int jj = 0; jj < DJ; ++jj) o_acc[jj] *= alpha;
                }
            }
            // the probabilities as two bf16 each: rounded to one, their error (2^-9 of each term) was as large as the output's own
            // rounding, and the result 1.45 times as far from the sums in 64 bits as one that is only rounded at the end
            const bf16x8 pf = __builtin_convertvector(pv, bf16x8);
            const bf16x8 pf_rest = __builtin_convertvector(pv - __builtin_convertvector(pf, floatx8), bf16x8);
            if (need_mask) {
                // A value that is no number (an infinity, rows never written) belongs only to the rows that see its key, and 0
                // times it is no zero: it is left out of the product, and the rows get it by how many such values they see.
                bool odd = false;
#pragma unroll
                for (int jj = 0; jj < DJ; ++jj) {
                    const u32x4 w = __builtin_bit_cast(u32x4, vf[jj]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) odd |= (w[e] & 0x7f80u) == 0x7f80u || (w[e] & 0x7f800000u) == 0x7f800000u;
                }
                if (__any(odd)) {
                    typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
                    u16x8 sees;
#pragma unroll
                    for (int e = 0; e < 8; ++e) sees[e] = s[e] == -INFINITY ? 0 : 0x3f80;       // bf16 0 or 1
#pragma unroll
                    for (int jj = 0; jj < DJ; ++jj) {
                        u16x8 w = __builtin_bit_cast(u16x8, vf[jj]), up, down, nan;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            up[e] = w[e] == 0x7f80 ? 0x3f80 : 0;
                            down[e] = w[e] == 0xff80 ? 0x3f80 : 0;
                            nan[e] = (w[e] & 0x7fff) > 0x7f80 ? 0x3f80 : 0;
                            w[e] = (w[e] & 0x7f80) == 0x7f80 ? 0 : w[e];
                        }
                        vf[jj] = __builtin_bit_cast(bf16x8, w);
                        const floatx4 none = {0.f, 0.f, 0.f, 0.f};
                        const bf16x8 see = __builtin_bit_cast(bf16x8, sees);
                        const floatx4 n_up = mfma16(__builtin_bit_cast(bf16x8, up), see, none);
                        const floatx4 n_down = mfma16(__builtin_bit_cast(bf16x8, down), see, none);
                        const floatx4 n_nan = mfma16(__builtin_bit_cast(bf16x8, nan), see, none);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if (n_up[e] > 0.f) o_acc[jj][e] += INFINITY;
                            if (n_down[e] > 0.f) o_acc[jj][e] += -INFINITY;
                            if (n_nan[e] > 0.f) o_acc[jj][e] = NAN;
                        }
                    }
                }
            }
            // ---- O^T += V^T P^T ----
#pragma unroll
            for (int jj = 0; jj < DJ; ++jj) o_acc[jj] = mfma16(vf[jj], pf, mfma16(vf[jj], pf_rest, o_acc[jj]));
        } while (++i < n_tiles);
    }

    // ---- the KS waves of a row block exchange their results through LDS; wave ks then owns D/KS columns of its 16 rows ----
    constexpr int SLICE = D / KS, CPL = SLICE / 4;
    l_run = quad_sum(l_run);
    const int row = row0 + mb * 16 + r;
    __syncthreads();                             // every wave is done with the ring
    float* sm_m = reinterpret_cast<float*>(smem);            // [NW][16]
    float* sm_l = sm_m + NW * 16;                            // [NW][16]
    float* sm_o = sm_l + NW * 16;                            // [NW][16][LDS_STRIDE]
    if (!is_loader) {
        if (c == 0) { sm_m[wave * 16 + r] = m_run; sm_l[wave * 16 + r] = l_run; }
        float* buf = sm_o + (wave * 16 + r) * LDS_STRIDE + 4 * c;
#pragma unroll
        for (int jj = 0; jj < DJ; ++jj) *reinterpret_cast<floatx4*>(buf + 16 * jj) = o_acc[jj];
    }
    __syncthreads();
    if (is_loader || row >= n_rows) return;
    float m_x[KS], m_all = -INFINITY, l_all = 0.f;
#pragma unroll
    for (int kx = 0; kx < KS; ++kx) { m_x[kx] = sm_m[(kx * MB + mb) * 16 + r]; m_all = fmaxf(m_all, m_x[kx]); }
    const float m_ref = (m_all == -INFINITY) ? 0.f : m_all;
#pragma unroll
    for (int kx = 0; kx < KS; ++kx) { m_x[kx] = fast_exp2(m_x[kx] - m_ref); l_all += m_x[kx] * sm_l[(kx * MB + mb) * 16 + r]; }
    const int col0 = ks * SLICE + c * CPL;
    floatx4 acc[CPL / 4];
#pragma unroll
    for (int qd = 0; qd < CPL / 4; ++qd) acc[qd] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kx = 0; kx < KS; ++kx) {
        const float* buf = sm_o + ((kx * MB + mb) * 16 + r) * LDS_STRIDE + col0;
#pragma unroll
        for (int qd = 0; qd < CPL / 4; ++qd) acc[qd] += m_x[kx] * *reinterpret_cast<const floatx4*>(buf + 4 * qd);
    }
    if (direct) {
        const QuotRem at = divide(row, p.group, p.inv_group);
        const int t = at.q, h = g * p.group + at.r;
        const float inv = l_all == 0.f ? 0.f : 1.f / l_all;                   // (a row that sees nothing: 0)
        __bf16* op = p.out + (int64_t)(q0 + t) * p.q_tok + (int64_t)h * p.q_head + col0;
#pragma unroll
        for (int qd = 0; qd < CPL / 4; ++qd)
            *reinterpret_cast<bf16x4*>(op + 4 * qd) = __builtin_convertvector(acc[qd] * inv, bf16x4);
        if (p.lse && c == 0 && ks == 0)
            p.lse[(int64_t)(q0 + t) * p.n_q_heads + h] = (m_all + fast_log2(l_all)) * kLn2;
    } else {
        float* po = p.part_o + (slot0 + row) * D + col0;
#pragma unroll
        for (int qd = 0; qd < CPL / 4; ++qd) *reinterpret_cast<floatx4*>(po + 4 * qd) = acc[qd];
        if (c == 0 && ks == 0) { p.part_ml[(slot0 + row) * 2] = m_all; p.part_ml[(slot0 + row) * 2 + 1] = l_all; }
    }
    };   // piece

    const auto slot_of = [&](int b) { return (int64_t)((j + b) * p.n_kv_heads + g) * p.rows_pad; };
    const int total = paged_total(p, lane), run = paged_run(p, total);
    int x = __builtin_amdgcn_readfirstlane(j * run);
    const int x_end = min(total, x + run);
    int base = 0;                                // tiles of the requests before the 64 at hand
    for (int c64 = 0; x < x_end; c64 += kWave) {
        const int tiles = p.batch == 1 ? total : c64 + lane < p.batch ? paged_tiles(p, c64 + lane) : 0;
        const int upto = p.batch == 1 ? total : base + wave_prefix(tiles, lane);
        base = __builtin_amdgcn_readlane(upto, kWave - 1);
        while (x < min(x_end, base)) {
            const int at = __builtin_ctzll(__ballot(upto > x));              // the request that holds tile x
            const int last = __builtin_amdgcn_readlane(upto, at), n = __builtin_amdgcn_readlane(tiles, at), first = last - n;
            const int to = min(last, x_end);
            piece(c64 + at, x - first, to - first, slot_of(c64 + at), x == first && to == last);
            x = to;
            __syncthreads();                     // the next piece reuses the ring and the exchange buffer
        }
    }
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
    const int b = head.q, g = head.r, lane = threadIdx.x & 63;
    const int q0 = p.cu_q ? p.cu_q[b] : b * p.q_len, ql = p.cu_q ? p.cu_q[b + 1] - q0 : p.q_len;
    const int n_rows = p.group * ql, row0 = at.q * ROWS;
    if (row0 >= n_rows) return;
    int first = 0, total = 0;
    if (p.batch == 1) total = paged_tiles(p, 0);
    else {
        int before = 0, all = 0;
        for (int c = 0; c < p.batch; c += kWave) {
            const int t = c + lane < p.batch ? paged_tiles(p, c + lane) : 0;
            all += t;
            before += c + lane < b ? t : 0;
        }
        total = wave_total(all); first = wave_total(before);
    }
    const int tiles = paged_tiles(p, b), run = paged_run(p, total);
    if (tiles == 0) return;
    const int j0 = first / run, live = (first + tiles - 1) / run - j0 + 1;
    if (live == 1) return;
    const int sub = threadIdx.x / TPR, grp = sub % GP, lr = sub / GP, col = (threadIdx.x % TPR) * 4, row = row0 + lr;
    const int64_t slot0 = (int64_t)((j0 + b) * p.n_kv_heads + g) * p.rows_pad + min(row, n_rows - 1);
    const int64_t step = (int64_t)p.n_kv_heads * p.rows_pad;
    float m = -INFINITY, l = 0.f;
    floatx4 acc = {0.f, 0.f, 0.f, 0.f};
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
        acc *= old; l *= old;
#pragma unroll
        for (int i = 0; i < PRE; ++i) {
            if (s0 + GP * i < live) {
                const float w = fast_exp2(ml[i].x - ref);        // 0 for a piece of which the row sees nothing
                acc += w * o[i];
                l += w * ml[i].y;
            }
        }
        m = m_new;
    }
    if constexpr (GP > 1) {
        *reinterpret_cast<floatx4*>(&s_o[lr][grp][col]) = acc;
        if (col == 0) { s_m[lr][grp] = m; s_l[lr][grp] = l; }
        __syncthreads();
        if (grp != 0) return;
#pragma unroll
        for (int i = 0; i < GP; ++i) m = fmaxf(m, s_m[lr][i]);
        const float ref = (m == -INFINITY) ? 0.f : m;
        acc = floatx4{0.f, 0.f, 0.f, 0.f}; l = 0.f;
#pragma unroll
        for (int i = 0; i < GP; ++i) {
            const float w = fast_exp2(s_m[lr][i] - ref);
            acc += w * *reinterpret_cast<const floatx4*>(&s_o[lr][i][col]);
            l += w * s_l[lr][i];
        }
    }
    if (row >= n_rows) return;
    acc *= l == 0.f ? 0.f : 1.f / l;
    const QuotRem out_at = divide(row, p.group, p.inv_group);
    const int t = out_at.q, h = g * p.group + out_at.r;
    *reinterpret_cast<bf16x4*>(p.out + (int64_t)(q0 + t) * p.q_tok + (int64_t)h * p.q_head + col) = __builtin_convertvector(acc, bf16x4);
    if (p.lse && col == 0) p.lse[(int64_t)(q0 + t) * p.n_q_heads + h] = (m + fast_log2(l)) * kLn2;
}

// ---------------------------------------------------------------- host side ----
struct PagedPlan { int n_rgroups, mb, rows_pad, max_groups; };

static PagedPlan paged_plan(int q_len, int n_q_heads, int n_kv_heads)
{
    PagedPlan s;
    attn_row_groups(n_q_heads / n_kv_heads * q_len, &s.n_rgroups, &s.mb);
    s.rows_pad = s.n_rgroups * s.mb * 16;
    s.max_groups = kTargetGroups / (n_kv_heads * s.n_rgroups);
    if (s.max_groups < 1) s.max_groups = 1;
    return s;
}

template <int D, int MB, int NLD>
static int launch_paged(const PagedParams& p, hipStream_t stream)
{
    constexpr int KS = 2, NS = 3, NW = MB * KS;
    constexpr size_t ring = (size_t)NS * 2 * kTileKeys * D * 2 + 64;
    constexpr size_t exchange = sizeof(float) * (size_t)(2 * NW * 16 + NW * 16 * (D + 4));
    constexpr size_t lds = ring > exchange ? ring : exchange;
    if (lds > 64 * 1024)
        if (const int rc = allow_lds<&paged_split_kernel<D, MB, KS, NS, NLD, true>>((int)lds)) return rc;
    hipLaunchKernelGGL((paged_split_kernel<D, MB, KS, NS, NLD, true>), dim3(p.max_groups * p.n_rgroups * p.n_kv_heads),
                       dim3((NW + NLD) * kWave), lds, stream, p);
    return launch_status();
}

template <int D>
static int launch_paged_d(const PagedParams& p, int mb, hipStream_t stream)
{
    int rc = SPECVLM_EUNSUPPORTED;
    switch (mb) {
        case 1: rc = launch_paged<D, 1, 2>(p, stream); break;
        case 2: rc = launch_paged<D, 2, 4>(p, stream); break;
        case 3: rc = launch_paged<D, 3, 2>(p, stream); break;
        case 4: rc = launch_paged<D, 4, 4>(p, stream); break;
    }
    if (rc != SPECVLM_OK) return rc;
    constexpr int GP = 8, ROWS = 256 / (D / 4 * GP);
    const int rows = p.group * p.q_len;
    hipLaunchKernelGGL((paged_join_kernel<D, GP>), dim3((rows + ROWS - 1) / ROWS * p.batch * p.n_kv_heads), dim3(256), 0, stream, p);
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
    return align256(slots * head_dim * sizeof(float)) + align256(slots * 2 * sizeof(float));
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
    if ((int64_t)batch * ((kv_len + kTileKeys - 1) / kTileKeys) >= ((int64_t)1 << 30)) return SPECVLM_EUNSUPPORTED;
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
    p.inv_group = reciprocal(p.group); p.inv_rgroups = reciprocal(s.n_rgroups);
    p.scale_log2 = softmax_scale * kLog2e;
    p.n_rgroups = s.n_rgroups; p.rows_pad = s.rows_pad; p.max_groups = s.max_groups;
    const size_t slots = ((size_t)s.max_groups + batch) * n_kv_heads * s.rows_pad;
    p.part_o = (float*)workspace;
    p.part_ml = (float*)((char*)workspace + align256(slots * head_dim * sizeof(float)));
    return head_dim == 128 ? launch_paged_d<128>(p, s.mb, (hipStream_t)stream) : launch_paged_d<64>(p, s.mb, (hipStream_t)stream);
}
