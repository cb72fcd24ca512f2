// What the attention kernels share: waits and barriers of a ring of direct-to-LDS loads, the transposing LDS read of value tiles,
// reductions over the four lanes of a query row, and how query rows are cut into blocks.
#pragma once

#include "common.h"

namespace specvlm {

#define SPECVLM_AS1 __attribute__((address_space(1)))
#define SPECVLM_AS3 __attribute__((address_space(3)))

constexpr int kChunkKeys = 32;       // keys per PV contraction step
constexpr float kSumRedo = 0x1p100f;     // a lane's sum of one chunk at or above this (or NaN) is redone with the maximum tracked
constexpr int kMaxQueryBlock = 64;      // queries per request: a row's view of its block is one 64-bit mask

// s_waitcnt immediate (gfx9 encoding) that waits for vmcnt <= n only.
constexpr int vmcnt_imm(int n)
{
    return (n & 15) | ((n >> 4) << 14) | (7 << 4) | (15 << 8);
}

template <int N> __device__ __forceinline__ void wait_vmcnt()
{
    static_assert(N >= 0 && N < 64, "vmcnt is a 6-bit counter");
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(N));
}

// Workgroup barrier that does not drain the direct-to-LDS loads still in
// flight for younger stages (a fence would).  Ordering of this wave's own LDS
// traffic is handled by the s_waitcnt the compiler places before each use.
__device__ __forceinline__ void stage_barrier()
{
    __asm__ volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    __asm__ volatile("" ::: "memory");
}

// Reductions over the four lanes r, r+16, r+32, r+48 that share a query row,
// with the VALU lane-swap instructions of gfx950 (no LDS crossbar round trip):
// v_permlane32_swap exchanges the upper 32 lanes of one operand with the lower
// 32 of the other, v_permlane16_swap the odd 16-lane rows with the even ones.
__device__ __forceinline__ float quad_max(float x)
{
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

__device__ __forceinline__ float quad_sum(float x)
{
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

constexpr int largest_divisor_le(int n, int cap)
{
    int best = 1;
    for (int d = 1; d <= cap; ++d) if (n % d == 0) best = d;
    return best;
}

// XOR applied to the 16-byte chunk index of value row `key` inside a tile.  The transposing read of
// one PV step touches, per 32 lanes, 8 consecutive keys x 32 contiguous bytes (two chunks 2j, 2j+1):
// with the pair index XORed by the key (d = 128: key mod 8; d = 64, two rows per 256 bytes: key/2
// mod 4) those 8 x 32 bytes fall on 64 distinct banks.
template <int D> __device__ __forceinline__ constexpr int v_swizzle(int key)
{
    return (D == 128) ? ((key & 7) << 1) : (((key >> 1) & 3) << 1);
}

// ds_read_b64_tr_b16: every lane hands in the address of 8 bytes (four 16-bit elements); inside each
// group of 16 lanes, lanes 4x..4x+3 together hold "row" x (16 elements), and lane o receives element o
// of rows 0..3.  Issued as assembly, with the wait below: as a builtin the compiler cannot tell the
// read from one that aliases the direct-to-LDS loads still in flight and drains them (vmcnt 0) first.
template <int OFFSET>
__device__ __forceinline__ u32x2 lds_read_tr16(uint32_t lds_addr)
{
    u32x2 v;
    __asm__ volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=&v"(v) : "v"(lds_addr), "n"(OFFSET));
    return v;
}

// Waits for this wave's LDS reads; the fragments pass through so that their uses stay behind the wait.
template <int N>
__device__ __forceinline__ void lds_wait_fragments(bf16x8 (&f)[N])
{
    static_assert(N == 4 || N == 8, "one fragment per 16 value columns");
    if constexpr (N == 8)
        __asm__ volatile("s_waitcnt lgkmcnt(0)"
                         : "+v"(f[0]), "+v"(f[1]), "+v"(f[2]), "+v"(f[3]), "+v"(f[4]), "+v"(f[5]), "+v"(f[6]), "+v"(f[7]));
    else
        __asm__ volatile("s_waitcnt lgkmcnt(0)" : "+v"(f[0]), "+v"(f[1]), "+v"(f[2]), "+v"(f[3]));
}

// Query rows of a kv head beyond 64 (long chains, draft trees) are cut into groups of equal size,
// at most 4 row blocks of 16 each: n groups, mb row blocks per group.
inline void attn_row_groups(int rows, int* n_groups, int* mb)
{
    const int blocks = (rows + 15) / 16;
    *n_groups = (blocks + 3) / 4;
    *mb = (blocks + *n_groups - 1) / *n_groups;
}

}  // namespace specvlm
