// Linear layers on packed weights (tboa_pack_codes): Y = X W^T (+ residual) and silu(X Wg^T) * (X Wu^T), W = scale (code - zero).
#include "internal.h"
#include <algorithm>

namespace {

typedef __hip_bfloat16 bf16;
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef unsigned u4 __attribute__((ext_vector_type(4)));

struct PackedArgs {
    const uint32_t* w[2]; const float* scale[2]; const float* zero[2];      // two: gate and up
    int d_out, d_in, words, group, n_groups;      // words of a row; channels of a group
    long long tokens;
    const void* X; long long ldx;
    const void* Res; long long ldr;
    void* Y; long long ldy;
    int vec;      // rows of X may be read 8 elements at a time
};

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(bf16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float from_f32(float v, float) { return v; }
__device__ __forceinline__ bf16 from_f32(float v, bf16) { return __float2bfloat16(v); }
__device__ __forceinline__ f4 mma16(b8 a, b8 b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ float silu(float g) { return g / (1.f + expf(-g)); }

// 24 bits as three terms of 8
__device__ __forceinline__ void split(float v, __bf16& hi, __bf16& mid, __bf16& lo) {
    hi = (__bf16)v;
    const float r = v - (float)hi;
    mid = (__bf16)r;
    lo = (__bf16)(r - (float)mid);
}

// Any group, any size: weights scale (code - zero) in fp32, as three bf16 terms, times X (bf16: as it is; fp32: three terms, products down to 2^-24).  A workgroup has 16 outputs of 16 MT tokens, its
// four wavefronts every fourth 32 channels.  GROUPS: 0: groups of a multiple of 8 channels, 1: of 8 and more (8 codes lie in at most two), 2: fewer.
template <typename T, int BITS, int GROUPS, int MT, bool GATED>
__global__ __launch_bounds__(256) void packed_any_kernel(PackedArgs a) {
    constexpr int NW = GATED ? 2 : 1, XT = sizeof(T) == 2 ? 1 : 3;
    __shared__ float part[4][NW][MT][16][17];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, grp = lane >> 4;
    const int n_tiles = (a.d_out + 15) / 16;
    const long long m_tiles = (a.tokens + 16 * MT - 1) / (16 * MT);
    for (long long tile = blockIdx.x; tile < n_tiles * m_tiles; tile += gridDim.x) {
        const int n0 = (int)(tile % n_tiles) * 16;
        const long long m0 = tile / n_tiles * (16 * MT);
        const long long row = min(n0 + col, a.d_out - 1);
        f4 acc[NW][MT];
#pragma unroll
        for (int w = 0; w < NW; ++w)
#pragma unroll
            for (int t = 0; t < MT; ++t) acc[w][t] = f4{0.f, 0.f, 0.f, 0.f};
        for (int k0 = wave * 32; k0 < a.d_in; k0 += 128) {
            const int k = k0 + 8 * grp, have = min(a.d_in - k, 8);      // codes of this lane (none: 0 or fewer)
            b8 wt[NW][3];
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = 0.f;
                if (have > 0) {
                    const uint32_t* const words = a.w[w] + row * a.words;
                    const float* const scale = a.scale[w] + row * a.n_groups, * const zero = a.zero[w] + row * a.n_groups;
                    const int at = (int)((long long)k * BITS >> 5), sh = k * BITS & 31;
                    const unsigned long long bits = (words[at] | (unsigned long long)words[min(at + 1, a.words - 1)] << 32) >> sh;
                    int g = k / a.group, left = a.group - (k - g * a.group);      // channels that the group still has
                    float s = scale[g], z = zero[g], s1 = s, z1 = z;
                    if (GROUPS == 1 && left < have) { s1 = scale[g + 1]; z1 = zero[g + 1]; }
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float c = (float)((unsigned)(bits >> (BITS * j)) & ((1u << BITS) - 1));
                        if (GROUPS == 1) v[j] = j < left ? s * (c - z) : s1 * (c - z1);
                        else v[j] = s * (c - z);
                        if (GROUPS == 2 && --left == 0 && j + 1 < have) { ++g; left = a.group; s = scale[g]; z = zero[g]; }
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j) if (j >= have) v[j] = 0.f;
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) { __bf16 hi, mid, lo; split(v[j], hi, mid, lo); wt[w][0][j] = hi; wt[w][1][j] = mid; wt[w][2][j] = lo; }
            }
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                const long long m = m0 + 16 * t + col;
                const T* const x = (const T*)a.X + min(m, a.tokens - 1) * a.ldx + k;
                b8 xt[XT];
                union { u4 u[sizeof(T) / 2]; T e[8]; } in;
#pragma unroll
                for (int i = 0; i < (int)sizeof(T) / 2; ++i) in.u[i] = u4{0, 0, 0, 0};
                if (m < a.tokens) {
                    if (a.vec && have >= 8) {
#pragma unroll
                        for (int i = 0; i < (int)sizeof(T) / 2; ++i) in.u[i] = ((const u4*)x)[i];
                    } else {
#pragma unroll
                        for (int j = 0; j < 8; ++j) if (j < have) in.e[j] = x[j];
                    }
                }
                if constexpr (XT == 1) xt[0] = __builtin_bit_cast(b8, in.u[0]);
                else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) { __bf16 hi, mid, lo; split(to_f32(in.e[j]), hi, mid, lo); xt[0][j] = hi; xt[1][j] = mid; xt[2][j] = lo; }
                }
#pragma unroll
                for (int w = 0; w < NW; ++w)
#pragma unroll
                    for (int i = 0; i < XT; ++i)
#pragma unroll
                        for (int j = 0; j + i < 3; ++j) acc[w][t] = mma16(xt[i], wt[w][j], acc[w][t]);
            }
        }
#pragma unroll
        for (int w = 0; w < NW; ++w)
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j) part[wave][w][t][4 * grp + j][col] = acc[w][t][j];
        __syncthreads();
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            const int r = threadIdx.x >> 4, n = n0 + (threadIdx.x & 15);
            const long long m = m0 + 16 * t + r;
            if (m < a.tokens && n < a.d_out) {
                float y[NW];
#pragma unroll
                for (int w = 0; w < NW; ++w) y[w] = (part[0][w][t][r][n - n0] + part[1][w][t][r][n - n0]) + (part[2][w][t][r][n - n0] + part[3][w][t][r][n - n0]);
                float v = GATED ? silu(y[0]) * y[NW - 1] : y[0];
                if (!GATED && a.Res) v += to_f32(((const T*)a.Res)[m * a.ldr + n]);
                ((T*)a.Y)[m * a.ldy + n] = from_f32(v, T());
            }
        }
        __syncthreads();
    }
}

template <typename T, int BITS, int GROUPS, bool GATED>
int launch_any(tboa_ctx* ctx, const PackedArgs& a) {
    const auto go = [&](auto MT) {
        constexpr int mt = decltype(MT)::value;
        const long long tiles = cdiv64(a.d_out, 16) * cdiv64(a.tokens, 16 * mt);
        hipLaunchKernelGGL((packed_any_kernel<T, BITS, GROUPS, mt, GATED>), dim3((unsigned)std::min<long long>(tiles, 1 << 20)), dim3(256), 0, ctx->stream, a);
    };
    if (a.tokens <= 16) go(std::integral_constant<int, 1>());
    else go(std::integral_constant<int, 4>());
    TB_KERNEL_CHECK(ctx);
    return 0;
}
template <typename T, int BITS, bool GATED>
int launch(tboa_ctx* ctx, const PackedArgs& a) {
    if (a.group % 8 == 0 || a.n_groups == 1) return launch_any<T, BITS, 0, GATED>(ctx, a);
    return a.group >= 8 ? launch_any<T, BITS, 1, GATED>(ctx, a) : launch_any<T, BITS, 2, GATED>(ctx, a);
}
template <typename T, bool GATED>
int launch(tboa_ctx* ctx, int bits, const PackedArgs& a) {
    switch (bits) {
        case 2: return launch<T, 2, GATED>(ctx, a);
        case 3: return launch<T, 3, GATED>(ctx, a);
        case 4: return launch<T, 4, GATED>(ctx, a);
        default: return launch<T, 8, GATED>(ctx, a);
    }
}

bool good_weight(const tboa_packed_weight* w) {
    return w && w->d_out > 0 && w->d_in > 0 && w->d_out <= 1 << 24 && w->d_in <= 1 << 24 && (w->bits == 2 || w->bits == 3 || w->bits == 4 || w->bits == 8) && w->group >= 0 &&
           (w->group == 0 || w->d_in % w->group == 0);
}

// what both calls check; up: the second matrix or NULL
int run(tboa_ctx* ctx, const char* who, const tboa_packed_weight* weight, const tboa_packed_weight* up, int64_t n_tokens, int dtype, const void* X, int64_t ldx, const void* Res, int64_t ldr, void* Y,
        int64_t ldy) {
    if (!good_weight(weight)) return tboa_fail(ctx, TBOA_EINVAL, "%s: a packed weight has 1 .. 2^24 rows and channels, codes of 2, 3, 4 or 8 bits and groups that divide its channels", who);
    if (dtype != TBOA_F32 && dtype != TBOA_BF16) return tboa_fail(ctx, TBOA_EINVAL, "%s: dtype must be fp32 or bf16", who);
    if (n_tokens < 0 || n_tokens > 1 << 24) return tboa_fail(ctx, TBOA_EINVAL, "%s: %lld tokens (at most 2^24)", who, (long long)n_tokens);
    if (n_tokens == 0) return 0;
    if (!weight->packed || !weight->scales || !weight->zeros || (up && (!up->packed || !up->scales || !up->zeros)) || !X || !Y) return tboa_fail(ctx, TBOA_EINVAL, "%s: null argument", who);
    if (ldx < weight->d_in || ldy < weight->d_out || (Res && ldr < weight->d_out)) return tboa_fail(ctx, TBOA_EINVAL, "%s: a row pitch is smaller than its row", who);
    const int size = dtype == TBOA_F32 ? 4 : 2;
    if ((uintptr_t)X % size || (uintptr_t)Y % size || (uintptr_t)Res % size) return tboa_fail(ctx, TBOA_EINVAL, "%s: an address that is no multiple of its elements' size", who);
    const TbDevice dev(ctx->device);
    PackedArgs a{};
    const tboa_packed_weight* both[2] = {weight, up ? up : weight};
    for (int i = 0; i < 2; ++i) { a.w[i] = both[i]->packed; a.scale[i] = both[i]->scales; a.zero[i] = both[i]->zeros; }
    a.d_out = weight->d_out; a.d_in = weight->d_in; a.words = (int)tboa_packed_words_per_row(weight->d_in, weight->bits);
    a.group = weight->group ? weight->group : weight->d_in; a.n_groups = weight->d_in / a.group;
    a.tokens = n_tokens; a.X = X; a.ldx = ldx; a.Res = Res; a.ldr = ldr; a.Y = Y; a.ldy = ldy;
    a.vec = (uintptr_t)X % 16 == 0 && ldx * size % 16 == 0;
    if (dtype == TBOA_F32) return up ? launch<float, true>(ctx, weight->bits, a) : launch<float, false>(ctx, weight->bits, a);
    return up ? launch<bf16, true>(ctx, weight->bits, a) : launch<bf16, false>(ctx, weight->bits, a);
}

}  // namespace

extern "C" size_t tboa_packed_workspace_bytes(const tboa_packed_weight* weight, int64_t n_tokens, int dtype) {
    return 0;
}

extern "C" int tboa_packed_linear(tboa_ctx* ctx, const tboa_packed_weight* weight, int64_t n_tokens, int dtype, const void* X, int64_t ldx, const void* Res, int64_t ldr, void* Y, int64_t ldy) {
    if (!ctx) return TBOA_EINVAL;
    return run(ctx, "packed_linear", weight, nullptr, n_tokens, dtype, X, ldx, Res, ldr, Y, ldy);
}

extern "C" int tboa_packed_swiglu(tboa_ctx* ctx, const tboa_packed_weight* gate, const tboa_packed_weight* up, int64_t n_tokens, int dtype, const void* X, int64_t ldx, void* Act, int64_t lda) {
    if (!ctx) return TBOA_EINVAL;
    if (!up || !gate || up->d_out != gate->d_out || up->d_in != gate->d_in || up->bits != gate->bits || up->group != gate->group)
        return tboa_fail(ctx, TBOA_EINVAL, "packed_swiglu: gate and up must have the same rows, channels, bits and groups");
    return run(ctx, "packed_swiglu", gate, up, n_tokens, dtype, X, ldx, nullptr, 0, Act, lda);
}
