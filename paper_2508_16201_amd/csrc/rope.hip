// specvlm_rope_append: queries and keys of the new tokens turned to their positions, keys and values written to the
// pages of their requests' caches, in one launch.
//
// Mathematics.  Pair i of a head is turned by pos * f_i and scaled:  (a, b) -> m (a cos - b sin, b cos + a sin).  f_i is
// given in turns a position as a 64-bit fraction, and the angle is the product modulo 2^64, that is modulo one
// turn, exactly: at position 2^20 a product in 32-bit floating point would be off by 2^20 * 2^-24 rad.  The upper 32 bits of
// it go to the sine and the cosine.  The products are fp32 and rounded to bf16 once.
//
// Bound: every element is read once and written once, HBM for a prompt (5.7 TB/s at 151 MB), the launch for a block (3.3 us for 48 tokens).  A lane keeps the sines
// and cosines of its eight pairs (two 16-byte pieces of a row) and takes them to row after row of the token.
#include "common.h"

#include <cmath>

namespace specvlm {

struct RopeParams {
    const __bf16* q;
    __bf16* q_out;
    const __bf16* k;
    const __bf16* v;
    __bf16* k_pages;
    __bf16* v_pages;
    int64_t q_tok, q_head, out_tok, out_head, kv_tok, kv_head, page, tok, head;      // strides in elements
    const int32_t* table;
    int64_t table_row;
    const int32_t* kv_lens;
    const int32_t* cu_q;
    const int32_t* positions;
    const uint64_t* turns;
    int n_pages, page_size, max_pages, batch, q_len, n_q_heads, n_kv_heads;
    int rot_units, interleaved;
    float magnitude;
    int rows, passes, parts;             // rows a token (q, k, v heads), a wave's passes over rows, waves a token
    uint32_t inv_q_len, inv_page, inv_parts;
    int n_waves;
};

constexpr int kRopeWaves = 4;
constexpr int64_t kRopeStreamBytes = 128 << 20;      // read and written

// Sine and cosine of phase * 2^-32 turns.  The quarter turn nearest is taken off in integers; what is left, at most an eighth of a turn, goes
// into the Taylor polynomials (first terms left out: x^11 / 11! and x^12 / 12!, below 2^-29 of 1).
__device__ __forceinline__ void turn_sincos(uint32_t phase, float* sine, float* cosine)
{
    const uint32_t quarter = (phase + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(phase - (quarter << 30)) * 1.46291807926715968105e-9f;      // 2 pi / 2^32
    const float z = x * x;
    const float s = fmaf(x * z, fmaf(z, fmaf(z, fmaf(z, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), x);
    const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
    const bool swapped = quarter & 1u;
    const float a = swapped ? c : s, b = swapped ? s : c;
    *sine = quarter & 2u ? -a : a;
    *cosine = (quarter + 1u) & 2u ? -b : b;
}

// STREAM: results are not kept near, for they would not all stay there (8190 tokens of 28/4 heads of 128, 151 MB 33.4 us kept, 26.4 not;  4096 of
// 64/8, 168 MB 36.6 / 29.3;  2048, 84 MB 16.5 / 17.3, and what reads them next finds them).
template <int D, bool STREAM>
__global__ __launch_bounds__(kRopeWaves * kWave)
void rope_append_kernel(const RopeParams p)
{
    constexpr int UNITS = D / 16, ROWS = kWave / UNITS;      // units of 16 elements a row, rows of a pass
    const int lane = threadIdx.x & 63;
    const int w = __builtin_amdgcn_readfirstlane(blockIdx.x * kRopeWaves + (threadIdx.x >> 6));
    if (w >= p.n_waves) return;
    const QuotRem at = divide(w, p.parts, p.inv_parts);
    const int t = at.q, part = at.r;
    // the token's request: as many as end at or before it
    int b = 0;
    if (p.cu_q) {
        for (int c = 0; c < p.batch; c += kWave) b += __popcll(__ballot(c + lane < p.batch && p.cu_q[c + lane + 1] <= t));
        if (b >= p.batch) return;                            // (behind the last request)
    } else {
        b = divide(t, p.q_len, p.inv_q_len).q;
    }
    const int first = p.cu_q ? p.cu_q[b] : b * p.q_len, ql = p.cu_q ? p.cu_q[b + 1] - first : p.q_len;
    const int kvl = p.kv_lens ? p.kv_lens[b] : ql;
    if (kvl < ql || t < first) return;
    const int place = kvl - ql + (t - first);
    const int pos = p.positions ? p.positions[t] : place;
    int64_t page_at = -1;                                    // where the token's row of the cache begins; -1: it has none
    if (p.k) {
        const QuotRem in = divide(place, p.page_size, p.inv_page);
        const int id = in.q < p.max_pages ? p.table[(int64_t)b * p.table_row + in.q] : -1;
        if ((uint32_t)id < (uint32_t)p.n_pages) page_at = id * p.page + in.r * p.tok;
    }
    const int u = lane % UNITS;
    const bool turned = u < p.rot_units;
    float cs[8], sn[8];
    if (turned) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint64_t phase = p.turns[8 * u + i] * (uint64_t)(int64_t)pos;
            float s, c;
            turn_sincos((uint32_t)(phase >> 32), &s, &c);
            cs[i] = c * p.magnitude;
            sn[i] = s * p.magnitude;
        }
    }
    // this lane's two pieces of eight elements: side by side, or the two halves of its pairs
    const bool apart = turned && !p.interleaved;
    const int lo = apart ? 8 * u : 16 * u, hi = apart ? 8 * (p.rot_units + u) : 16 * u + 8;
    for (int pass = 0; pass < p.passes; ++pass) {
        const int row = (part * p.passes + pass) * ROWS + lane / UNITS;
        const int kv = row - p.n_q_heads;                     // (negative: a query row)
        const bool is_q = kv < 0, is_k = !is_q && kv < p.n_kv_heads;
        if (row >= p.rows || (!is_q && page_at < 0)) continue;
        const int h = is_q ? row : is_k ? kv : kv - p.n_kv_heads;
        const __bf16* src = is_q ? p.q + (int64_t)t * p.q_tok + (int64_t)h * p.q_head
                                 : (is_k ? p.k : p.v) + (int64_t)t * p.kv_tok + (int64_t)h * p.kv_head;
        __bf16* dst = is_q ? p.q_out + (int64_t)t * p.out_tok + (int64_t)h * p.out_head
                           : (is_k ? p.k_pages : p.v_pages) + page_at + (int64_t)h * p.head;
        bf16x8 x = *reinterpret_cast<const bf16x8*>(src + lo), y = *reinterpret_cast<const bf16x8*>(src + hi);
        if (turned && (is_q || is_k)) {
            const floatx8 a = __builtin_convertvector(x, floatx8), c = __builtin_convertvector(y, floatx8);
            floatx8 na, nc;
            if (p.interleaved) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    na[2 * i] = a[2 * i] * cs[i] - a[2 * i + 1] * sn[i];
                    na[2 * i + 1] = a[2 * i + 1] * cs[i] + a[2 * i] * sn[i];
                    nc[2 * i] = c[2 * i] * cs[4 + i] - c[2 * i + 1] * sn[4 + i];
                    nc[2 * i + 1] = c[2 * i + 1] * cs[4 + i] + c[2 * i] * sn[4 + i];
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    na[i] = a[i] * cs[i] - c[i] * sn[i];
                    nc[i] = c[i] * cs[i] + a[i] * sn[i];
                }
            }
            x = __builtin_convertvector(na, bf16x8);
            y = __builtin_convertvector(nc, bf16x8);
        }
        if constexpr (STREAM) {
            __builtin_nontemporal_store(__builtin_bit_cast(u32x4, x), reinterpret_cast<u32x4*>(dst + lo));
            __builtin_nontemporal_store(__builtin_bit_cast(u32x4, y), reinterpret_cast<u32x4*>(dst + hi));
        } else {
            *reinterpret_cast<bf16x8*>(dst + lo) = x;
            *reinterpret_cast<bf16x8*>(dst + hi) = y;
        }
    }
}

template <int D>
static int launch_rope(RopeParams& p, int n_tokens, hipStream_t stream)
{
    constexpr int ROWS = kWave / (D / 16);
    // a wave takes all rows of its token where there are tokens enough to fill the chip, else one pass
    const int all = (p.rows + ROWS - 1) / ROWS;
    p.passes = (int64_t)n_tokens * all > 8 * 4 * kNumCu ? all : 1;
    p.parts = (all + p.passes - 1) / p.passes;
    p.inv_parts = reciprocal(p.parts);
    if ((int64_t)n_tokens * p.parts > 0x7fffffff - kRopeWaves) return SPECVLM_EUNSUPPORTED;
    p.n_waves = n_tokens * p.parts;
    const dim3 grid((p.n_waves + kRopeWaves - 1) / kRopeWaves), block(kRopeWaves * kWave);
    if (!launchable(grid.x, kRopeWaves * kWave)) return SPECVLM_EUNSUPPORTED;
    if ((int64_t)n_tokens * p.rows * D * 4 >= kRopeStreamBytes) hipLaunchKernelGGL((rope_append_kernel<D, true>), grid, block, 0, stream, p);
    else                                                        hipLaunchKernelGGL((rope_append_kernel<D, false>), grid, block, 0, stream, p);
    return launch_status();
}

}  // namespace specvlm

using namespace specvlm;

extern "C" int specvlm_rope_turns(int rot_dim, const specvlm_rope_spec* spec, uint64_t* turns)
{
    if (rot_dim < 0 || (rot_dim & 1) || !spec || (!turns && rot_dim > 0)) return SPECVLM_EINVAL;
    const int kind = spec->kind;
    if (kind < SPECVLM_ROPE_PLAIN || kind > SPECVLM_ROPE_BY_PARTS || !(spec->base > 0.) || !(spec->base < INFINITY)) return SPECVLM_EINVAL;
    if (kind != SPECVLM_ROPE_PLAIN && (!(spec->factor >= 1.) || !(spec->factor < INFINITY))) return SPECVLM_EINVAL;
    if (kind == SPECVLM_ROPE_BY_PARTS && (!(spec->original_len > 0.) || !(spec->original_len < INFINITY) || !(spec->beta_slow >= 0.) ||
                                          !(spec->beta_fast > spec->beta_slow) || !(spec->beta_fast < INFINITY)))
        return SPECVLM_EINVAL;
    if (kind == SPECVLM_ROPE_BASE && rot_dim == 2) return SPECVLM_EINVAL;              // (one pair: it cannot be both)
    const long double two_pi = 6.283185307179586476925286766559005768L;
    long double base = spec->base;
    const long double factor = spec->factor, fast = spec->beta_fast, slow = spec->beta_slow;
    if (kind == SPECVLM_ROPE_BASE && rot_dim) base *= powl(factor, (long double)rot_dim / (rot_dim - 2));
    for (int i = 0; i < rot_dim / 2; ++i) {
        long double f = powl(base, -2.0L * i / rot_dim) / two_pi;                  // turns a position
        if (kind == SPECVLM_ROPE_LINEAR) f /= factor;
        if (kind == SPECVLM_ROPE_BY_PARTS) {
            const long double ramp = (spec->original_len * f - slow) / (fast - slow), keep = ramp < 0 ? 0 : ramp > 1 ? 1 : ramp;
            f = f * keep + f / factor * (1 - keep);
        }
        const long double x = floorl((f - floorl(f)) * 18446744073709551616.0L + 0.5L);
        turns[i] = x < 18446744073709551616.0L ? (uint64_t)x : 0;
    }
    return SPECVLM_OK;
}

extern "C" int specvlm_rope_append(
    const void* q, int64_t q_tok_stride, int64_t q_head_stride, void* q_out, int64_t out_tok_stride, int64_t out_head_stride,
    const void* k, const void* v, int64_t kv_tok_stride, int64_t kv_head_stride,
    void* k_pages, void* v_pages, int64_t page_stride, int64_t tok_stride, int64_t head_stride,
    int n_pages, int page_size, const int32_t* page_table, int64_t table_stride, int max_pages,
    const int32_t* kv_lens, const int32_t* cu_q, int batch, int n_tokens, const int32_t* positions,
    const uint64_t* turns, int rot_dim, int interleaved, float magnitude,
    int n_q_heads, int n_kv_heads, int head_dim, void* stream)
{
    if (batch < 0 || n_tokens < 0 || n_q_heads < 0 || n_kv_heads < 0 || n_pages < 0 || max_pages < 0 || rot_dim < 0) return SPECVLM_EINVAL;
    if (!(fabsf(magnitude) < INFINITY) || rot_dim > head_dim) return SPECVLM_EINVAL;
    if ((k == nullptr) != (v == nullptr)) return SPECVLM_EINVAL;
    if (head_dim != 64 && head_dim != 128) return SPECVLM_EUNSUPPORTED;
    if (rot_dim % 16) return SPECVLM_EUNSUPPORTED;
    if (!q) n_q_heads = 0;
    if (!k) n_kv_heads = 0;
    if (batch == 0 || n_tokens == 0 || n_q_heads + n_kv_heads == 0) return SPECVLM_OK;
    if (!cu_q && n_tokens % batch) return SPECVLM_EINVAL;
    if ((rot_dim > 0 && !turns) || (q && !q_out) || (!kv_lens && (k || !positions))) return SPECVLM_EINVAL;
    if (k) {
        if (!k_pages || !v_pages || !page_table || page_size <= 0 || table_stride < 0) return SPECVLM_EINVAL;
        if (page_size % 16) return SPECVLM_EUNSUPPORTED;
    }
    int64_t strides = 0;
    uintptr_t places = 0;
    if (q) { strides |= q_tok_stride | q_head_stride | out_tok_stride | out_head_stride; places |= (uintptr_t)q | (uintptr_t)q_out; }
    if (k) {
        strides |= kv_tok_stride | kv_head_stride | page_stride | tok_stride | head_stride;
        places |= (uintptr_t)k | (uintptr_t)v | (uintptr_t)k_pages | (uintptr_t)v_pages;
    }
    if ((strides & 7) || (places & 15)) return SPECVLM_EUNSUPPORTED;
    if (n_q_heads > (1 << 20) || n_kv_heads > (1 << 20)) return SPECVLM_EUNSUPPORTED;

    RopeParams p;
    p.q = (const __bf16*)q; p.q_out = (__bf16*)q_out; p.k = (const __bf16*)k; p.v = (const __bf16*)v;
    p.k_pages = (__bf16*)k_pages; p.v_pages = (__bf16*)v_pages;
    p.q_tok = q_tok_stride; p.q_head = q_head_stride; p.out_tok = out_tok_stride; p.out_head = out_head_stride;
    p.kv_tok = kv_tok_stride; p.kv_head = kv_head_stride; p.page = page_stride; p.tok = tok_stride; p.head = head_stride;
    p.table = page_table; p.table_row = table_stride; p.kv_lens = kv_lens; p.cu_q = cu_q; p.positions = positions; p.turns = turns;
    p.n_pages = n_pages; p.page_size = k ? page_size : 1; p.max_pages = max_pages;
    p.batch = batch; p.q_len = cu_q ? 1 : n_tokens / batch;
    p.n_q_heads = n_q_heads; p.n_kv_heads = n_kv_heads;
    p.rot_units = rot_dim / 16; p.interleaved = interleaved; p.magnitude = magnitude;
    p.rows = n_q_heads + 2 * n_kv_heads;
    p.inv_q_len = reciprocal(p.q_len); p.inv_page = reciprocal(p.page_size);
    return head_dim == 128 ? launch_rope<128>(p, n_tokens, (hipStream_t)stream) : launch_rope<64>(p, n_tokens, (hipStream_t)stream);
}
