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
    unsigned piece_magic;      // packed_few_kernel: a group has 2^32 / piece_magic pieces of a run that share their scale (0: one; 1: all)
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

__device__ __forceinline__ unsigned low_halves(unsigned a, unsigned b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ unsigned high_halves(unsigned a, unsigned b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
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
// A run of CK = 128 VW / BITS consecutive channels of a row is 4 VW words, VW for each of the four lane groups of a 16 x 16 x 32 instruction, NF fragments of 8 codes for each lane.
// Two codes become a pair of bf16 by a shift and an and-or: code c in the upper bits of the mantissa of 2^BITS is 2^BITS + c.  Pairs are codes that stand 16 bits apart in the stream (48 for 3 bits, as
// 16 is no multiple of 3), and X takes the same order.
struct Masks { unsigned codes, one; };
template <int BITS, int VW>
struct Codes {
    static constexpr int CL = VW * 32 / BITS, NF = CL / 8, CK = 4 * CL, OFFSET = BITS == 8 ? 0 : 1 << BITS;
    // 2 and 4 bits: word r of lane group g is the run's word 4 r + g, so that a fragment's channels lie together (and so may groups of 32 or 64); else VW words in a row
    static constexpr bool TURNED = (BITS == 2 || BITS == 4) && VW == 4;
    // channels of pair p of fragment f, among the lane's
    static constexpr int first(int f, int p) { return BITS == 8 ? 8 * f + 2 * p : BITS == 4 ? 8 * f + p : BITS == 2 ? f / 2 * 16 + f % 2 * 4 + p : 4 * f + p; }
    static constexpr int second(int f, int p) { return BITS == 8 ? 8 * f + 2 * p + 1 : first(f, p) + (BITS == 4 ? 4 : BITS == 2 ? 8 : 16); }
    // the run's channel that is channel c of lane group g
    static __device__ __forceinline__ int channel(int c, int g) { return TURNED ? c / (32 / BITS) * (128 / BITS) + g * (32 / BITS) + c % (32 / BITS) : g * CL + c; }
    // the pair whose codes begin at bit AT of either half of v
    template <int AT>
    static __device__ __forceinline__ unsigned pair(unsigned v, const Masks& m) {
        constexpr int to = 7 - BITS;      // where a code begins in the mantissa
        return ((AT < to ? v << (to - AT) : v >> (AT - to)) & m.codes) | m.one;
    }
    static __device__ __forceinline__ Masks masks() {
        constexpr unsigned mask = BITS == 8 ? 0u : ((1u << BITS) - 1) << (7 - BITS), one = (unsigned)(127 + BITS) << 7;
        Masks m{mask | mask << 16, one | one << 16};
        asm("" : "+s"(m.codes), "+v"(m.one));      // (as literals they would be an instruction more for every pair)
        return m;
    }
    // fragment F of a lane's codes
    template <int F>
    static __device__ __forceinline__ void fragment(const unsigned (&w)[VW], unsigned (&out)[4], const Masks& m) {
        if constexpr (BITS == 4) {
            out[0] = pair<0>(w[F], m); out[1] = pair<4>(w[F], m); out[2] = pair<8>(w[F], m); out[3] = pair<12>(w[F], m);
        } else if constexpr (BITS == 2) {
            constexpr int at = F % 2 * 8;
            out[0] = pair<at>(w[F / 2], m); out[1] = pair<at + 2>(w[F / 2], m); out[2] = pair<at + 4>(w[F / 2], m); out[3] = pair<at + 6>(w[F / 2], m);
        } else if constexpr (BITS == 3) {
            const unsigned b = __builtin_amdgcn_alignbit(w[2], w[1], 16);      // the stream from bit 48 on
            // five codes of either half of the stream at a time, from bits 0, 15, 30 and 45 on
            auto five = [&](int k) {
                return k == 0 ? low_halves(w[0], b) : k == 1 ? low_halves(w[0] >> 15, b >> 15) : k == 2 ? low_halves(__builtin_amdgcn_alignbit(w[1], w[0], 30), w[2] >> 14) : low_halves(w[1] >> 13, w[2] >> 29);
            };
            out[0] = pair<4 * F % 5 * 3>(five(4 * F / 5), m); out[1] = pair<(4 * F + 1) % 5 * 3>(five((4 * F + 1) / 5), m);
            out[2] = pair<(4 * F + 2) % 5 * 3>(five((4 * F + 2) / 5), m); out[3] = pair<(4 * F + 3) % 5 * 3>(five((4 * F + 3) / 5), m);
        } else {
#pragma unroll
            for (int p = 0; p < 4; ++p) {      // whole numbers up to 255 are bf16
                const unsigned v = w[2 * F + p / 2] >> (p % 2 * 16);
                out[p] = high_halves(__float_as_uint((float)(v & 255u)), __float_as_uint((float)(v >> 8 & 255u)));
            }
        }
    }
};

constexpr int GRIDS = 8;      // groups whose scales and zeros a wavefront has in LDS
// 16-byte piece p of row n of 16 rows of 64 bytes in LDS: pieces exchanged by row, so that neither four lanes beside each other (written) nor 16 rows (read) meet in a bank
__device__ __forceinline__ int place16(int n, int p) { return n * 64 + ((p ^ (n >> 2 & 3)) << 4); }
// bytes of LDS that a wavefront has: runs of X (XR rows of it), of codes, scales and zeros
template <typename T, int BITS, int VW, int XR, int NR>
constexpr int few_bytes() { return XR * (Codes<BITS, VW>::CK) * (int)sizeof(T) + NR * 1024 + 2 * NR * 16 * GRIDS * 4; }
template <int XR, int NR>
constexpr int most_waves() { return XR <= 16 && NR == 1 ? 16 : 8; }

// Up to XR tokens (4, or 16 MT) per workgroup: bound by the codes' bytes.  A wavefront has 16 RT outputs (of either matrix) and an equal part of the runs of channels; the wavefronts are joined through LDS.  FF
// fragments of a run have one scale.  bf16 X: codes enter with their offset, and (offset + zero) sum x, by a product with ones that all outputs share, is taken out again with every scale:
//     y += scale (sum (offset + code) x - (offset + zero) sum x)
// fp32 X: codes less zeros, exact in bf16, times three bf16 terms.
// Rows of codes, of X and of scales are read by four lanes side by side, 64 bytes together, and handed to the lanes that multiply them through the wavefront's own part of LDS: read by those lanes
// themselves, a row each, every 16 bytes are an access of their own to the first cache (16 tokens of 8192 x 28672: 37 million accesses, 143000 cycles of every compute unit's, 67 us).
template <typename T, int BITS, int VW, int FF, int XR, int RT, bool GATED>
__global__ __launch_bounds__((64 * most_waves<XR, (GATED ? 2 : 1) * RT>())) void packed_few_kernel(PackedArgs a) {
    typedef Codes<BITS, VW> C;
    constexpr bool EXACT = sizeof(T) == 4;
    constexpr int MT = (XR + 15) / 16, NW = GATED ? 2 : 1, NR = NW * RT, NF = C::NF, NS = NF / FF, XT = EXACT ? 3 : 1, E = 16 / (int)sizeof(T), XB = C::CK * (int)sizeof(T) / 64;      // XB: 64-byte blocks of a row of X
    constexpr int XI = XR == 4 ? (XB + 3) / 4 : XB;      // loads that a row of X takes: of four rows, 64 lanes read four blocks at a time
    constexpr int P = XR == 4 ? 4 : MT == 1 && XB <= 4 ? 2 : 1;      // runs whose loads are under way together
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6, col = lane & 15, grp = lane >> 4;
    const int row4 = lane >> 2, quarter = lane & 3;      // as a reader: row of 16, 16-byte piece of 64
    char* const xs = lds + wave * few_bytes<T, BITS, VW, XR, NR>(), * const ws = xs + XR * 64 * XB;
    float* const grids = (float*)(ws + NR * 1024);      // [2][NR][16][GRIDS]
    const int n0 = blockIdx.x * (16 * RT);
    const long long m0 = (long long)blockIdx.y * XR;
    const int xrow = XR == 4 ? row4 & 3 : row4, xblock = XR == 4 ? lane >> 4 : 0;      // of X, as a reader
    // places within the workgroup's rows of codes and of X (32 bits beside a base that all lanes share)
    unsigned at_w[RT], at_x[MT];
#pragma unroll
    for (int r = 0; r < RT; ++r) at_w[r] = ((unsigned)min(r * 16 + row4, a.d_out - 1 - n0) * a.words + quarter * VW) * 4;
#pragma unroll
    for (int t = 0; t < MT; ++t) at_x[t] = (unsigned)min((long long)(16 * t + xrow), a.tokens - 1 - m0) * (unsigned)a.ldx * (unsigned)sizeof(T) + quarter * 16;
    const char* const x = (const char*)((const T*)a.X + m0 * a.ldx);
    const char* codes[NW];
#pragma unroll
    for (int w = 0; w < NW; ++w) codes[w] = (const char*)(a.w[w] + (long long)n0 * a.words);

    // block of X that this lane reads with load i; where that is in LDS; where a lane that multiplies finds byte `at` of its row of a run
    auto block_of = [&](int i) { return XR == 4 ? (XB < 4 ? xblock % XB : i * 4 + xblock) : i; };
    auto written = [&](int t, int i) { return (u4*)(xs + (XR == 4 ? block_of(i) * 256 + xrow * 64 + quarter * 16 : (t * XB + i) * 1024 + place16(row4, quarter))); };
    auto read = [&](int t, int at) { return xs + (XR == 4 ? (at >> 6) * 256 + (col & 3) * 64 + (at & 63) : (t * XB + (at >> 6)) * 1024 + place16(col, at >> 4 & 3) + (at & 15)); };
    struct Run { unsigned w[NR][VW]; u4 x[MT][XI]; };
    auto load = [&](int run, Run& o, auto WHOLE) {      // WHOLE: all of the run's channels are there, and X can be read 16 bytes at a time
        const int k0 = run * C::CK;
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            if constexpr (decltype(WHOLE)::value) {
                struct __attribute__((packed, aligned(4))) Piece { unsigned u[VW]; };
                const Piece p = *(const Piece*)(codes[r / RT] + (long long)run * (16 * VW) + at_w[r % RT]);
#pragma unroll
                for (int i = 0; i < VW; ++i) o.w[r][i] = p.u[i];
            } else {
                const uint32_t* const row = (const uint32_t*)(codes[r / RT] + (at_w[r % RT] - quarter * VW * 4));
#pragma unroll
                for (int i = 0; i < VW; ++i) o.w[r][i] = row[min((run * 4 + quarter) * VW + i, a.words - 1)];
            }
        }
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            if constexpr (decltype(WHOLE)::value) {
#pragma unroll
                for (int i = 0; i < XI; ++i) o.x[t][i] = *(const u4*)(x + (long long)k0 * sizeof(T) + (block_of(i) * 64 + at_x[t]));
            } else {
                const T* const row = (const T*)a.X + min(m0 + 16 * t + xrow, a.tokens - 1) * a.ldx;
#pragma unroll
                for (int i = 0; i < XI; ++i) {
                    union { u4 u; T e[E]; } v;
                    v.u = u4{0, 0, 0, 0};
#pragma unroll
                    for (int j = 0; j < E; ++j) { const int k = k0 + block_of(i) * 4 * E + quarter * E + j; if (k < a.d_in) v.e[j] = row[k]; }
                    o.x[t][i] = v.u;
                }
            }
        }
    };
    int grid0 = -GRIDS;      // first group whose scales are in LDS
    auto group_of = [&](unsigned piece) { return min((int)(a.piece_magic ? __umulhi(piece, a.piece_magic) : piece), a.n_groups - 1); };
    struct Grids { float f[2][NR][GRIDS / 4]; };
    auto load_grids = [&](int g, Grids& o) {      // of groups g .. for this lane's row of every 16
        grid0 = max(min(g, a.n_groups - GRIDS), 0);
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                const float* const row = (z ? a.zero : a.scale)[r / RT] + (long long)min(n0 + r % RT * 16 + row4, a.d_out - 1) * a.n_groups;
                const int first = min(grid0 + quarter * (GRIDS / 4), a.n_groups - 1), second = min(first + 1, a.n_groups - 1);
                o.f[z][r][0] = row[first]; o.f[z][r][1] = row[second];
            }
    };
    auto keep_grids = [&](const Grids& o) {
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
            for (int z = 0; z < 2; ++z)
#pragma unroll
                for (int i = 0; i < GRIDS / 4; ++i) grids[((z * NR + r) * 16 + row4) * GRIDS + ((quarter * (GRIDS / 4) + i) ^ (row4 >> 1))] = o.f[z][r][i];
    };
    auto grid = [&](int z, int r, int g) { return grids[((z * NR + r) * 16 + col) * GRIDS + ((g - grid0) ^ (col >> 1))]; };
    f4 acc[NR][MT];
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[r][t] = f4{0.f, 0.f, 0.f, 0.f};
    const Masks masks = C::masks();
    b8 ones;
#pragma unroll
    for (int j = 0; j < 8; ++j) ones[j] = (__bf16)1.f;
    auto in_order = [] { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); __builtin_amdgcn_wave_barrier(); };      // (a wavefront's own accesses to LDS)
    auto multiply = [&](int run, const Run& o) {
        in_order();
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            struct __attribute__((aligned(16))) Piece { unsigned u[VW]; } p;
#pragma unroll
            for (int i = 0; i < VW; ++i) p.u[i] = o.w[r][i];
            *(Piece*)(ws + r * 1024 + place16(row4, quarter)) = p;
        }
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int i = 0; i < XI; ++i) *written(t, i) = o.x[t][i];
        if (group_of(run * NS + NS - 1) >= grid0 + GRIDS) { Grids next; load_grids(group_of(run * NS), next); keep_grids(next); }
        in_order();
        unsigned w[NR][VW];
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
            for (int i = 0; i < VW; ++i) w[r][i] = *(const unsigned*)(ws + r * 1024 + (C::TURNED ? place16(col, i) + grp * 4 : place16(col, grp) + i * 4));
        f4 sum[MT], temp[NR][MT];
        unroll<NF>([&](auto F) {
            constexpr int f = F, s = f / FF;
            if constexpr (f % FF == 0) {
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    sum[t] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int r = 0; r < NR; ++r) temp[r][t] = f4{0.f, 0.f, 0.f, 0.f};
                }
            }
            const int g = group_of(run * NS + s);
            union { unsigned u[4]; b8 v; } wf[NR];
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                C::template fragment<f>(w[r], wf[r].u, masks);
                if constexpr (EXACT) {
                    const float off = C::OFFSET + grid(1, r, g);
#pragma unroll
                    for (int p = 0; p < 4; ++p)
                        wf[r].u[p] = high_halves(__float_as_uint(__uint_as_float(wf[r].u[p] << 16) - off), __float_as_uint(__uint_as_float(wf[r].u[p] & 0xffff0000u) - off));
                }
            }
            // the pieces of X that hold the fragment's channels: those of the first codes of its pairs, and of the second ones
            constexpr int c0 = C::first(f, 0), c1 = C::second(f, 0), B = BITS == 8 ? 8 : 4, H = BITS == 8 ? 1 : 2;      // B channels from c0 on, and from c1 on (H = 2)
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                T e[H][B];
#pragma unroll
                for (int h = 0; h < H; ++h) {
                    constexpr int N = B < E ? B : E;      // (a part of a piece, or pieces)
#pragma unroll
                    for (int i = 0; i < B; i += N) {
                        const int at = C::channel((h ? c1 : c0) + i, grp) * (int)sizeof(T);
                        struct __attribute__((aligned(N * sizeof(T)))) Part { T e[N]; };
                        const Part p = *(const Part*)read(t, at);
#pragma unroll
                        for (int j = 0; j < N; ++j) e[h][i + j] = p.e[j];
                    }
                }
                union { unsigned u[4]; b8 v; } xf[XT];
                if constexpr (EXACT) {
#pragma unroll
                    for (int p = 0; p < 4; ++p)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            __bf16 hi, mid, lo;
                            split(to_f32(BITS == 8 ? e[0][2 * p + j] : e[j * (H - 1)][p]), hi, mid, lo);
                            xf[0].v[2 * p + j] = hi; xf[XT / 2].v[2 * p + j] = mid; xf[XT - 1].v[2 * p + j] = lo;
                        }
                } else {
                    union { T e[H][B]; unsigned u[H][B / 2]; } in;
#pragma unroll
                    for (int h = 0; h < H; ++h)
#pragma unroll
                        for (int j = 0; j < B; ++j) in.e[h][j] = e[h][j];
#pragma unroll
                    for (int p = 0; p < 4; ++p) xf[0].u[p] = BITS == 8 ? in.u[0][p] : p % 2 ? high_halves(in.u[0][p / 2], in.u[H - 1][p / 2]) : low_halves(in.u[0][p / 2], in.u[H - 1][p / 2]);
                    sum[t] = mma16(xf[0].v, ones, sum[t]);
                }
#pragma unroll
                for (int r = 0; r < NR; ++r)
#pragma unroll
                    for (int i = 0; i < XT; ++i) temp[r][t] = mma16(xf[i].v, wf[r].v, temp[r][t]);
            }
            if constexpr (f % FF == FF - 1) {
#pragma unroll
                for (int r = 0; r < NR; ++r) {
                    const float scale = grid(0, r, g), off = -(C::OFFSET + grid(1, r, g));
#pragma unroll
                    for (int t = 0; t < MT; ++t)
#pragma unroll
                        for (int j = 0; j < 4; ++j) acc[r][t][j] = fmaf(scale, EXACT ? temp[r][t][j] : fmaf(off, sum[t][j], temp[r][t][j]), acc[r][t][j]);
                }
            }
        });
    };
    // P runs' loads are issued together; the wavefronts of a SIMD take turns
    const int runs = (a.d_in + C::CK - 1) / C::CK, whole = a.vec ? a.d_in / C::CK : 0, each = (runs + waves - 1) / waves;
    const int end = min((wave + 1) * each, runs);
    int run = wave * each;
    Grids first;
    load_grids(group_of(run * NS), first);
    auto several = [&](auto N) {
        constexpr int n = decltype(N)::value;
        for (; run + n <= min(whole, end); run += n) {
            Run o[n];
#pragma unroll
            for (int i = 0; i < n; ++i) load(run + i, o[i], std::true_type());
            __builtin_amdgcn_sched_barrier(0);
            if (run == wave * each) keep_grids(first);
#pragma unroll
            for (int i = 0; i < n; ++i) multiply(run + i, o[i]);
        }
    };
    several(std::integral_constant<int, P>());
    if constexpr (P == 4) several(std::integral_constant<int, 2>());
    for (; run < end; ++run) {
        Run o;
        if (run < whole) load(run, o, std::true_type()); else load(run, o, std::false_type());
        if (run == wave * each) keep_grids(first);
        multiply(run, o);
    }
    float* const part = (float*)lds;      // [wavefronts][NR][16][17]
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        __syncthreads();
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

template <typename T, int BITS, int VW, int FF, int XR, int RT, bool GATED>
int launch_few(tboa_ctx* ctx, PackedArgs a) {
    typedef Codes<BITS, VW> C;
    constexpr int NR = GATED ? 2 * RT : RT, bytes = few_bytes<T, BITS, VW, XR, NR>();
    const int runs = (a.d_in + C::CK - 1) / C::CK;
    const int most = a.d_out > 16 * RT * 512 ? 8 : most_waves<XR, NR>();      // (workgroups that all find room at once)
    int waves = 4;
    while (waves < most && waves * 2 < runs && 2 * waves * bytes <= 160 * 1024) waves *= 2;
    const int pieces = a.group / (32 * FF);
    a.piece_magic = a.n_groups == 1 ? 1 : pieces == 1 ? 0 : (unsigned)(((1ull << 32) + pieces - 1) / pieces);
    const auto kernel = packed_few_kernel<T, BITS, VW, FF, XR, RT, GATED>;
    if (waves * bytes > 65536) TB_HIP(ctx, hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, waves * bytes));
    hipLaunchKernelGGL(kernel, dim3((unsigned)cdiv64(a.d_out, 16 * RT), (unsigned)cdiv64(a.tokens, XR)), dim3(64 * waves), std::max(waves * bytes, waves * NR * 16 * 17 * 4), ctx->stream, a);
    TB_KERNEL_CHECK(ctx);
    return 0;
}
template <typename T, int BITS, int VW, int FF, int XR, bool GATED>
int launch_few(tboa_ctx* ctx, const PackedArgs& a) {
    if constexpr (!GATED && XR > 4) { if (a.d_out >= 16 * 2 * 256) return launch_few<T, BITS, VW, FF, XR, 2, GATED>(ctx, a); }
    return launch_few<T, BITS, VW, FF, XR, 1, GATED>(ctx, a);
}
template <typename T, int BITS, int VW, int FF, bool GATED>
int launch_few(tboa_ctx* ctx, const PackedArgs& a) {
    if (a.tokens <= 4) return launch_few<T, BITS, VW, FF, 4, GATED>(ctx, a);
    if (a.tokens <= 16) return launch_few<T, BITS, VW, FF, 16, GATED>(ctx, a);
    if constexpr (sizeof(T) == 2) { if (a.tokens > 32) return launch_few<T, BITS, VW, FF, 64, GATED>(ctx, a); }
    return launch_few<T, BITS, VW, FF, 32, GATED>(ctx, a);
}
// fragments (of 32 channels in all) that a group has at least: as many as a run, or the most of which it has a whole number; 0: none
int fragments_of_scale(const PackedArgs& a, int most, int least) {
    for (int ff = most; ff >= least; ff /= 2) if (a.n_groups == 1 || a.group % (32 * ff) == 0) return ff;
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
    if (cdiv64(a.tokens, 16) <= 65535) {
        if constexpr (BITS == 2) {
            const int ff = fragments_of_scale(a, 8, 2);
            if (ff) return ff == 8 ? launch_few<T, 2, 4, 8, GATED>(ctx, a) : ff == 4 ? launch_few<T, 2, 4, 4, GATED>(ctx, a) : launch_few<T, 2, 4, 2, GATED>(ctx, a);
        } else if constexpr (BITS == 3) {
            if (fragments_of_scale(a, 4, 4)) return launch_few<T, 3, 3, 4, GATED>(ctx, a);
        } else if constexpr (BITS == 4) {
            const int ff = fragments_of_scale(a, 4, 1);
            if (ff) return ff == 4 ? launch_few<T, 4, 4, 4, GATED>(ctx, a) : ff == 2 ? launch_few<T, 4, 4, 2, GATED>(ctx, a) : launch_few<T, 4, 4, 1, GATED>(ctx, a);
        } else {
            const int ff = fragments_of_scale(a, 2, 1);
            if (ff) return ff == 2 ? launch_few<T, 8, 4, 2, GATED>(ctx, a) : launch_few<T, 8, 2, 1, GATED>(ctx, a);
        }
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
    a.vec = (uintptr_t)X % 16 == 0 && ldx * size % 16 == 0 && ldx < 1 << 24;      // (the rows of a workgroup within 32 bits)
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
