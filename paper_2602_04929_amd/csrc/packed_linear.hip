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
    int vec;      // rows of X may be read 16 bytes at a time
    int runs_of_group, run_shift;      // packed_few_kernel: runs of channels that a group has, as a power of two or -1
};

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(bf16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float from_f32(float v, float) { return v; }
__device__ __forceinline__ bf16 from_f32(float v, bf16) { return __float2bfloat16(v); }
__device__ __forceinline__ f4 mma16(b8 a, b8 b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ float silu(float g) { return g / (1.f + expf(-g)); }

template <int N, int I = 0, typename F>
__device__ __forceinline__ void unroll(F&& f) {
    if constexpr (I < N) { f(std::integral_constant<int, I>{}); unroll<N, I + 1>(f); }
}

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

// ------------------------------------------------------------------------------------------------ few tokens
// Codes that a lane loads at a time, VW words of a row: CL of them, NF fragments of 8 for a 16 x 16 x 32 instruction.  Four lanes side by side hold CK = 4 CL consecutive channels of a row.
// Two codes become a pair of bf16 by a shift and an and-or: code c in the upper bits of the mantissa of 2^BITS is 2^BITS + c.  Pairs are codes that stand 16 bits apart in the stream (48 for 3 bits, as
// 16 is no multiple of 3), and X takes the same order.
template <int BITS, int VW>
struct Codes {
    static constexpr int CL = VW * 32 / BITS, NF = CL / 8, CK = 4 * CL, OFFSET = BITS == 8 ? 0 : 1 << BITS;
    // channels of pair p of fragment f
    static constexpr int first(int f, int p) { return BITS == 8 ? 8 * f + 2 * p : BITS == 4 ? 8 * f + p : BITS == 2 ? f / 2 * 16 + f % 2 * 4 + p : 4 * f + p; }
    static constexpr int second(int f, int p) { return BITS == 8 ? 8 * f + 2 * p + 1 : first(f, p) + (BITS == 4 ? 4 : BITS == 2 ? 8 : 16); }
    // the pair whose codes begin at bit `at` of either half of v
    template <int AT>
    static __device__ __forceinline__ unsigned pair(unsigned v) {
        constexpr int to = 7 - BITS;      // where a code begins in the mantissa
        constexpr unsigned mask = ((1u << BITS) - 1) << to, one = (unsigned)(127 + BITS) << 7;
        const unsigned u = AT < to ? v << (to - AT) : v >> (AT - to);
        return (u & (mask | mask << 16)) | (one | one << 16);
    }
    static __device__ __forceinline__ unsigned low_halves(unsigned a, unsigned b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
    static __device__ __forceinline__ unsigned high_halves(unsigned a, unsigned b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
    // fragment F of a lane's codes
    template <int F>
    static __device__ __forceinline__ void fragment(const unsigned (&w)[VW], unsigned (&out)[4]) {
        if constexpr (BITS == 4) {
            out[0] = pair<0>(w[F]); out[1] = pair<4>(w[F]); out[2] = pair<8>(w[F]); out[3] = pair<12>(w[F]);
        } else if constexpr (BITS == 2) {
            constexpr int at = F % 2 * 8;
            out[0] = pair<at>(w[F / 2]); out[1] = pair<at + 2>(w[F / 2]); out[2] = pair<at + 4>(w[F / 2]); out[3] = pair<at + 6>(w[F / 2]);
        } else if constexpr (BITS == 3) {
            const unsigned b = __builtin_amdgcn_alignbit(w[2], w[1], 16);      // the stream from bit 48 on
            // five codes of either half of the stream at a time, from bits 0, 15, 30 and 45 on
            auto five = [&](int k) {
                return k == 0 ? low_halves(w[0], b) : k == 1 ? low_halves(w[0] >> 15, b >> 15) : k == 2 ? low_halves(__builtin_amdgcn_alignbit(w[1], w[0], 30), w[2] >> 14) : low_halves(w[1] >> 13, w[2] >> 29);
            };
            out[0] = pair<4 * F % 5 * 3>(five(4 * F / 5)); out[1] = pair<(4 * F + 1) % 5 * 3>(five((4 * F + 1) / 5));
            out[2] = pair<(4 * F + 2) % 5 * 3>(five((4 * F + 2) / 5)); out[3] = pair<(4 * F + 3) % 5 * 3>(five((4 * F + 3) / 5));
        } else {
#pragma unroll
            for (int p = 0; p < 4; ++p) {      // whole numbers up to 255 are bf16
                const unsigned v = w[2 * F + p / 2] >> (p % 2 * 16);
                out[p] = high_halves(__float_as_uint((float)(v & 255u)), __float_as_uint((float)(v >> 8 & 255u)));
            }
        }
    }
};

// Up to 16 MT tokens per workgroup: bound by the codes' bytes.  A wavefront has 16 RT outputs (of either matrix) and every KW-th run of CK channels, which lie in one group; the wavefronts are joined through
// LDS.  bf16 X: codes enter with their offset, and (offset + zero) sum x, by a product with ones that all outputs share, is taken out again with every run:
//     y += scale (sum (offset + code) x - (offset + zero) sum x)
// fp32 X: codes less zeros, exact in bf16, times three bf16 terms.
template <typename T, int BITS, int VW, int MT, int RT, bool GATED>
__global__ __launch_bounds__(MT == 1 ? 1024 : 512) void packed_few_kernel(PackedArgs a) {
    typedef Codes<BITS, VW> C;
    constexpr bool EXACT = sizeof(T) == 4;
    constexpr int NW = GATED ? 2 : 1, NR = NW * RT, CL = C::CL, NF = C::NF, XT = EXACT ? 3 : 1, XW = CL * (int)sizeof(T) / 16;
    extern __shared__ float part[];      // [wavefronts][NR][16][17]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6, col = lane & 15, grp = lane >> 4;
    const int n0 = blockIdx.x * (16 * RT);
    const long long m0 = (long long)blockIdx.y * (16 * MT);
    const int runs = (a.d_in + C::CK - 1) / C::CK;
    const uint32_t* words[NR];
    const float *scale[NR], *zero[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        const long long row = min(n0 + (r % RT) * 16 + col, a.d_out - 1);
        words[r] = a.w[r / RT] + row * a.words;
        scale[r] = a.scale[r / RT] + row * a.n_groups; zero[r] = a.zero[r / RT] + row * a.n_groups;
    }
    const T* x[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) x[t] = (const T*)a.X + min(m0 + 16 * t + col, a.tokens - 1) * a.ldx;

    struct Run { unsigned w[NR][VW]; float s[NR], z[NR]; };
    auto load_weights = [&](int run, Run& o) {
        const int at = (run * 4 + grp) * VW, g = a.n_groups == 1 ? 0 : a.run_shift >= 0 ? run >> a.run_shift : run / a.runs_of_group;
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            if ((run + 1) * C::CK <= a.d_in) {
                struct __attribute__((packed, aligned(4))) Piece { unsigned u[VW]; };
                const Piece p = *(const Piece*)(words[r] + at);
#pragma unroll
                for (int i = 0; i < VW; ++i) o.w[r][i] = p.u[i];
            } else {
#pragma unroll
                for (int i = 0; i < VW; ++i) o.w[r][i] = words[r][min(at + i, a.words - 1)];
            }
            o.s[r] = scale[r][g]; o.z[r] = zero[r][g];
        }
    };
    f4 acc[NR][MT];
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[r][t] = f4{0.f, 0.f, 0.f, 0.f};
    b8 ones;
#pragma unroll
    for (int j = 0; j < 8; ++j) ones[j] = (__bf16)1.f;
    Run here, next;
    if (wave < runs) load_weights(wave, next);
    for (int run = wave; run < runs; run += waves) {
        here = next;
        const int k = run * C::CK + grp * CL;
        union Raw { u4 u[XW]; unsigned w[4 * XW]; T e[CL]; } raw[MT];
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            if (a.vec && (run + 1) * C::CK <= a.d_in) {
#pragma unroll
                for (int i = 0; i < XW; ++i) raw[t].u[i] = ((const u4*)(x[t] + k))[i];
            } else {
#pragma unroll
                for (int i = 0; i < XW; ++i) raw[t].u[i] = u4{0, 0, 0, 0};
#pragma unroll
                for (int j = 0; j < CL; ++j) if (k + j < a.d_in) raw[t].e[j] = x[t][k + j];
            }
        }
        if (run + waves < runs) load_weights(run + waves, next);
        f4 sum[MT], temp[NR][MT];
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            sum[t] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int r = 0; r < NR; ++r) temp[r][t] = f4{0.f, 0.f, 0.f, 0.f};
        }
        unroll<NF>([&](auto F) {
            constexpr int f = F;
            union { unsigned u[4]; b8 v; } wf[NR];
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                C::template fragment<f>(here.w[r], wf[r].u);
                if constexpr (EXACT) {
                    const float off = C::OFFSET + here.z[r];
#pragma unroll
                    for (int p = 0; p < 4; ++p)
                        wf[r].u[p] = C::high_halves(__float_as_uint(__uint_as_float(wf[r].u[p] << 16) - off), __float_as_uint(__uint_as_float(wf[r].u[p] & 0xffff0000u) - off));
                }
            }
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                union { unsigned u[4]; b8 v; } xf[XT];
                if constexpr (EXACT) {
#pragma unroll
                    for (int p = 0; p < 4; ++p)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            __bf16 hi, mid, lo;
                            split(to_f32(raw[t].e[j ? C::second(f, p) : C::first(f, p)]), hi, mid, lo);
                            xf[0].v[2 * p + j] = hi; xf[XT / 2].v[2 * p + j] = mid; xf[XT - 1].v[2 * p + j] = lo;
                        }
                } else {
#pragma unroll
                    for (int p = 0; p < 4; ++p) {
                        const int i = C::first(f, p), j = C::second(f, p);
                        xf[0].u[p] = BITS == 8 ? raw[t].w[i / 2] : i % 2 ? C::high_halves(raw[t].w[i / 2], raw[t].w[j / 2]) : C::low_halves(raw[t].w[i / 2], raw[t].w[j / 2]);
                    }
                    sum[t] = mma16(xf[0].v, ones, sum[t]);
                }
#pragma unroll
                for (int r = 0; r < NR; ++r)
#pragma unroll
                    for (int i = 0; i < XT; ++i) temp[r][t] = mma16(xf[i].v, wf[r].v, temp[r][t]);
            }
        });
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            const float off = -(C::OFFSET + here.z[r]);
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[r][t][j] = fmaf(here.s[r], EXACT ? temp[r][t][j] : fmaf(off, sum[t][j], temp[r][t][j]), acc[r][t][j]);
        }
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        if (t) __syncthreads();
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
            for (int j = 0; j < 4; ++j) part[((wave * NR + r) * 16 + 4 * grp + j) * 17 + col] = acc[r][t][j];
        __syncthreads();
        for (int i = threadIdx.x; i < RT * 256; i += blockDim.x) {
            const int r = i >> 8, row = i >> 4 & 15, c = i & 15, n = n0 + r * 16 + c;
            const long long m = m0 + 16 * t + row;
            if (m < a.tokens && n < a.d_out) {
                float y[NW];
#pragma unroll
                for (int w = 0; w < NW; ++w) {
                    y[w] = 0.f;
                    for (int v = 0; v < waves; ++v) y[w] += part[((v * NR + w * RT + r) * 16 + row) * 17 + c];
                }
                float v = GATED ? silu(y[0]) * y[NW - 1] : y[0];
                if (!GATED && a.Res) v += to_f32(((const T*)a.Res)[m * a.ldr + n]);
                ((T*)a.Y)[m * a.ldy + n] = from_f32(v, T());
            }
        }
    }
}

template <typename T, int BITS, int VW, int MT, int RT, bool GATED>
int launch_few(tboa_ctx* ctx, PackedArgs a) {
    typedef Codes<BITS, VW> C;
    constexpr int NR = GATED ? 2 * RT : RT;
    const int runs = (a.d_in + C::CK - 1) / C::CK, most = MT == 1 ? 16 : 8;
    int waves = 4;
    while (waves < most && waves < runs) waves *= 2;
    a.runs_of_group = a.group / C::CK;
    a.run_shift = a.n_groups > 1 && (a.runs_of_group & (a.runs_of_group - 1)) == 0 ? __builtin_ctz(a.runs_of_group) : -1;
    const int lds = waves * NR * 16 * 17 * 4;
    if (lds > 65536) TB_HIP(ctx, hipFuncSetAttribute((const void*)packed_few_kernel<T, BITS, VW, MT, RT, GATED>, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
    hipLaunchKernelGGL((packed_few_kernel<T, BITS, VW, MT, RT, GATED>), dim3((unsigned)cdiv64(a.d_out, 16 * RT), (unsigned)cdiv64(a.tokens, 16 * MT)), dim3(64 * waves), lds, ctx->stream, a);
    TB_KERNEL_CHECK(ctx);
    return 0;
}
template <typename T, int BITS, int VW, int MT, bool GATED>
int launch_few(tboa_ctx* ctx, const PackedArgs& a) {
    if constexpr (!GATED) { if (a.d_out >= 16 * 2 * 256) return launch_few<T, BITS, VW, MT, 2, GATED>(ctx, a); }
    return launch_few<T, BITS, VW, MT, 1, GATED>(ctx, a);
}
template <typename T, int BITS, int VW, bool GATED>
int launch_few(tboa_ctx* ctx, const PackedArgs& a) {
    constexpr int less = BITS == 2 && VW == 4 ? 2 : VW;      // (registers)
    if (a.tokens <= 16) return launch_few<T, BITS, VW, 1, GATED>(ctx, a);
    if constexpr (sizeof(T) == 2) { if (a.tokens > 32) return launch_few<T, BITS, less, 4, GATED>(ctx, a); }
    return launch_few<T, BITS, less, 2, GATED>(ctx, a);
}
// words that a lane may load at a time so that a run of channels lies in one group; 0: none
template <int BITS>
int words_of_run(const PackedArgs& a) {
    if (BITS == 3) return a.n_groups == 1 || a.group % 128 == 0 ? 3 : 0;
    for (int vw = 4; vw >= (BITS == 8 ? 2 : 1); vw /= 2) if (a.n_groups == 1 || a.group % (4 * vw * 32 / BITS) == 0) return vw;
    return 0;
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
    if (cdiv64(a.tokens, 16) <= 65535) switch (words_of_run<BITS>(a)) {
        case 4: if constexpr (BITS != 3) return launch_few<T, BITS, 4, GATED>(ctx, a); break;
        case 3: if constexpr (BITS == 3) return launch_few<T, BITS, 3, GATED>(ctx, a); break;
        case 2: if constexpr (BITS != 3) return launch_few<T, BITS, 2, GATED>(ctx, a); break;
        case 1: if constexpr (BITS != 3 && BITS != 8) return launch_few<T, BITS, 1, GATED>(ctx, a); break;
    }
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
