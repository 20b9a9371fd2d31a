// What the kernels of attention over the quantized cache share: types, levels as half, arguments, outputs.
#pragma once
#include "kv_cache.h"
#include <math.h>
#include <algorithm>

struct AttendArgs {
    KvGeometry g; KvBatch q;
    const void* Q; long long ldq; void* O; long long ldo;
    const unsigned char* cache;
    float scale2;                 // scale log2 e
    int rep, window;
    int vec, out_piece;           // elements of Q that may be read together, 8, 4 or 0 (one by one); of O that may be written together: 8, 4 or 1
    int few;                      // sequences of more rows are kv_attend_tiles_kernel's
    const unsigned* tree; int tree_words, piece_rows;      // trees of drafted tokens (kv_tree_attention.hip): masks of a token's sequence's new tokens, rows of a piece
    int4* info;                   // per workgroup: the unit that begins in its share and ends in another: workgroups, first row of the sequence, row of the first | rows << 27, head
    float* tile_part; float2* tile_stat; int4* tile_info;      // kv_attend_tiles_kernel: per piece, its rows; of trees what the join needs
    float* part; float2* stat;    // per workgroup two pieces of 16 rows (of a unit that began before its share, of one that begins in it): averages; maximum, sum
};
// trees of drafted tokens: bf16 sequences of more than `few` rows by the kernel for many rows (kv_attention.hip)
size_t kv_tree_tiles_room(const KvGeometry& g, AttendArgs* a, void* ws);
bool kv_tree_tiles_takes(const KvGeometry& g, int n_seqs, long long n_tokens, int rep);
int kv_tree_tiles(tboa_ctx* ctx, const AttendArgs& a);

namespace {

typedef __hip_bfloat16 bf16;
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef unsigned u4 __attribute__((ext_vector_type(4)));
typedef unsigned u2 __attribute__((ext_vector_type(2)));
template <typename T> struct Four { typedef u4 type; };      // four elements
template <> struct Four<bf16> { typedef u2 type; };

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(bf16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16 from_f32<bf16>(float v) { return __float2bfloat16(v); }
__device__ __forceinline__ f4 by_power(f4 v, int e) { return f4{__builtin_amdgcn_ldexpf(v[0], e), __builtin_amdgcn_ldexpf(v[1], e), __builtin_amdgcn_ldexpf(v[2], e), __builtin_amdgcn_ldexpf(v[3], e)}; }
__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }

template <int N, int I = 0, typename F>
__device__ __forceinline__ void unroll(F&& f) {
    if constexpr (I < N) { f(std::integral_constant<int, I>{}); unroll<N, I + 1>(f); }
}
// lane n of a row of 16, in all of them
template <int N>
__device__ __forceinline__ unsigned row_lane(unsigned v) { return (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0x150 + N, 0xf, 0xf, true); }
template <int N>
__device__ __forceinline__ float row_lane(float v) { return __uint_as_float(row_lane<N>(__float_as_uint(v))); }
template <int X>
__device__ __forceinline__ float from_xor(float v) { return __shfl_xor(v, X, 64); }

// eight levels less the zeros in `off`, pairs of -(1024 + zero)
__device__ __forceinline__ h8 levels8(unsigned a, unsigned b, h2 o0, h2 o1, h2 o2, h2 o3) {
    constexpr unsigned ONE = 0x64646464u;      // half 1024 has the upper byte 0x64
    const h2 r0 = __builtin_bit_cast(h2, __builtin_amdgcn_perm(ONE, a, 0x04010400u)) + o0, r1 = __builtin_bit_cast(h2, __builtin_amdgcn_perm(ONE, a, 0x04030402u)) + o1;
    const h2 r2 = __builtin_bit_cast(h2, __builtin_amdgcn_perm(ONE, b, 0x04010400u)) + o2, r3 = __builtin_bit_cast(h2, __builtin_amdgcn_perm(ONE, b, 0x04030402u)) + o3;
    return h8{r0[0], r0[1], r1[0], r1[1], r2[0], r2[1], r3[0], r3[1]};
}
__device__ __forceinline__ f4 mma16(h8 a, h8 b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }


// channels c .. c + 3 of a row of the outputs
__device__ __forceinline__ void store4(float* out, int c, const AttendArgs& a, f4 v) {
    if (a.out_piece >= 4) { if (c < a.g.dh) *(f4*)(out + c) = v; return; }
#pragma unroll
    for (int j = 0; j < 4; ++j) if (c + j < a.g.dh) out[c + j] = v[j];
}
__device__ __forceinline__ uint2 pack4(f4 v) {
    union { bf16 e[4]; uint2 u; } p;
#pragma unroll
    for (int j = 0; j < 4; ++j) p.e[j] = from_f32<bf16>(v[j]);
    return p.u;
}
__device__ __forceinline__ void store4(bf16* out, int c, const AttendArgs& a, f4 v) {
    if (a.out_piece >= 4) { if (c < a.g.dh) *(uint2*)(out + c) = pack4(v); return; }
#pragma unroll
    for (int j = 0; j < 4; ++j) if (c + j < a.g.dh) out[c + j] = from_f32<bf16>(v[j]);
}

}  // namespace
