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
    int d_out, d_in, bits, words, group, n_groups;      // words of a row; channels of a group
    long long tokens;
    const void* X; long long ldx;
    const void* Res; long long ldr;
    void* Y; long long ldy;
    int vec, out_vec;      // rows of X may be read 16 bytes at a time, of Y written four elements at a time
    float* partial; int splits;      // packed_few_kernel: parts of the channels that workgroups of their own have, and their sums [splits][tokens][d_out] (splits > 1)
    unsigned piece_magic, piece_all;      // packed_few_kernel: a group has 2^32 / piece_magic pieces of a run that share their scale (1: all), one where piece_all has all bits
};

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(bf16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float from_f32(float v, float) { return v; }
__device__ __forceinline__ bf16 from_f32(float v, bf16) { return __float2bfloat16(v); }
__device__ __forceinline__ f4 mma16(b8 a, b8 b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ float silu(float g) { return g / (1.f + expf(-g)); }

// x / d = umulhi(x, m) + (x & all) for x d < 2^32, 0 for d = 0
inline void magic(unsigned d, unsigned& m, unsigned& all) { m = d < 2 ? 0u : (unsigned)(((1ull << 32) + d - 1) / d); all = d == 1 ? ~0u : 0u; }
// whether that holds for all of a row's pieces of so many channels and those of its last, incomplete run (rows of millions of channels in a few groups: packed_any_kernel, which divides)
inline bool divides(const PackedArgs& a, int channels) { return a.n_groups == 1 || (a.d_in / channels + 64LL) * (a.group / channels) < 1LL << 32; }

template <int N, int I = 0, typename F>
__device__ __forceinline__ void unroll(F&& f) {
    if constexpr (I < N) { f(std::integral_constant<int, I>{}); unroll<N, I + 1>(f); }
}

__device__ __forceinline__ unsigned low_halves(unsigned a, unsigned b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ unsigned high_halves(unsigned a, unsigned b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
// 24 bits as three terms of 8, cut off (rounded, the largest numbers would become infinite)
__device__ __forceinline__ __bf16 upper(float v) { return __builtin_bit_cast(__bf16, (unsigned short)(__float_as_uint(v) >> 16)); }
__device__ __forceinline__ void split(float v, __bf16& hi, __bf16& mid, __bf16& lo) {
    hi = upper(v);
    const float r = v - (float)hi;
    mid = upper(r);
    lo = upper(r - (float)mid);
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
// 16 is no multiple of 3), and X takes the same order.  All of it times 2^-DOWN, which the sum over all channels takes back: 256 channels of the largest X then add up to a number, offsets included.
struct Masks { unsigned codes, one; };
template <int BITS, int VW>
struct Codes {
    static constexpr int CL = VW * 32 / BITS, NF = CL / 8, CK = 4 * CL, OFFSET = BITS == 8 ? 0 : 1 << BITS, DOWN = BITS + 10;
    // 2 and 4 bits: word r of lane group g is the run's word 4 r + g, so that a fragment's channels lie together (and so may groups of 32 or 64); else VW words in a row
    static constexpr bool TURNED = (BITS == 2 || BITS == 4) && VW == 4;
    static constexpr float LESS = 1.f / (1u << DOWN), MORE = 1u << DOWN;
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
        constexpr unsigned mask = BITS == 8 ? 0u : ((1u << BITS) - 1) << (7 - BITS), one = (unsigned)(127 + BITS - DOWN) << 7;
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
                out[p] = high_halves(__float_as_uint((float)(v & 255u) * LESS), __float_as_uint((float)(v >> 8 & 255u) * LESS));
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
//     y += scale (sum (offset + code) x - (offset + zero) sum x)      (all of it times 2^-DOWN)
// fp32 X: codes less zeros, exact in bf16, times three bf16 terms.
// Rows of codes, of X and of scales are read by four lanes side by side, 64 bytes together, and handed to the lanes that multiply them through the wavefront's own part of LDS: read by those lanes
// themselves, a row each, every 16 bytes are an access of their own to the first cache (16 tokens of 8192 x 28672: 37 million accesses, not 9.7; 67 us and not 34, the same weights again and again, 42.6 from memory).
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
    auto group_of = [&](unsigned piece) { return min((int)(__umulhi(piece, a.piece_magic) + (piece & a.piece_all)), a.n_groups - 1); };
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
    for (int j = 0; j < 8; ++j) ones[j] = (__bf16)C::LESS;
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
                    const float off = (C::OFFSET + grid(1, r, g)) * C::LESS;
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
    const int runs = (a.d_in + C::CK - 1) / C::CK, whole = a.vec ? a.d_in / C::CK : 0, each = (runs + waves * a.splits - 1) / (waves * a.splits), begin = min((blockIdx.z * waves + wave) * each, runs);
    const int end = min(begin + each, runs);
    int run = begin;
    Grids first;
    load_grids(group_of(run * NS), first);
    auto several = [&](auto N) {
        constexpr int n = decltype(N)::value;
        for (; run + n <= min(whole, end); run += n) {
            Run o[n];
#pragma unroll
            for (int i = 0; i < n; ++i) load(run + i, o[i], std::true_type());
            __builtin_amdgcn_sched_barrier(0);
            if (run == begin) keep_grids(first);
#pragma unroll
            for (int i = 0; i < n; ++i) multiply(run + i, o[i]);
        }
    };
    several(std::integral_constant<int, P>());
    if constexpr (P == 4) several(std::integral_constant<int, 2>());
    for (; run < end; ++run) {
        Run o;
        if (run < whole) load(run, o, std::true_type()); else load(run, o, std::false_type());
        if (run == begin) keep_grids(first);
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
                    y[w] *= C::MORE;
                }
                if (!GATED && a.splits > 1) { a.partial[(blockIdx.z * a.tokens + m) * a.d_out + n] = y[0]; continue; }
                float v = GATED ? silu(y[0]) * y[NW - 1] : y[0];
                if (!GATED && a.Res) v += to_f32(((const T*)a.Res)[m * a.ldr + n]);
                ((T*)a.Y)[m * a.ldy + n] = from_f32(v, T());
            }
        }
    }
}

// sums of the splits' partial results, an output a thread
template <typename T>
__global__ __launch_bounds__(256) void packed_few_join_kernel(PackedArgs a) {
    const int n = blockIdx.x * 256 + threadIdx.x;
    const long long m = blockIdx.y;
    if (n >= a.d_out) return;
    float v = 0.f;
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) v += a.partial[(s * a.tokens + m) * a.d_out + n];
    if (a.Res) v += to_f32(((const T*)a.Res)[m * a.ldr + n]);
    ((T*)a.Y)[m * a.ldy + n] = from_f32(v, T());
}

// Parts of the channels for 33 to 64 tokens of bf16, whose X (64 rows of it go through every workgroup) allows a compute unit one workgroup of eight wavefronts at a time: the fewest with which rounds of
// workgroups times runs of a wavefront is least, more of them for a fifth less (they are joined), each of at least 1024 channels.  64 tokens of 5120 x 13824, three bits: 320 workgroups of 16 outputs 61 us, 480 of 32
// outputs and a third of the channels 34, and 4 for the join.
int few_splits(const PackedArgs& a) {
    if (a.tokens > 64) return 1;
    const long long groups = cdiv64(a.d_out, 32), runs = cdiv64(a.d_in, a.bits == 2 ? 256 : 128);
    const auto cost = [&](int s) { return cdiv64(groups * s, 256) * cdiv64(runs, 8 * s); };
    int best = 1;
    for (int s = 2; s <= 8 && s <= a.d_in / 1024; ++s)
        if (cost(s) * 5 <= cost(best) * 4) best = s;
    return best;
}
size_t few_room(const PackedArgs& a) { const int splits = few_splits(a); return splits > 1 ? (size_t)splits * a.tokens * a.d_out * sizeof(float) : 0; }

template <typename T, int BITS, int VW, int FF, int XR, int RT, bool GATED>
int launch_few(tboa_ctx* ctx, PackedArgs a) {
    typedef Codes<BITS, VW> C;
    constexpr int NR = GATED ? 2 * RT : RT, bytes = few_bytes<T, BITS, VW, XR, NR>();
    a.splits = XR == 64 && !GATED ? few_splits(a) : 1;
    if (a.splits > 1) {
        TB_TRY(tboa_ws_reserve(ctx, few_room(a)));
        a.partial = (float*)ctx->ws;
    }
    const int runs = (a.d_in + C::CK - 1) / C::CK / a.splits + (a.splits > 1);      // (parts: eight wavefronts with a run each too)
    const int most = a.d_out > 16 * RT * 512 ? 8 : most_waves<XR, NR>();      // (workgroups that all find room at once)
    int waves = 4;
    while (waves < most && waves * 2 < runs && 2 * waves * bytes <= 160 * 1024) waves *= 2;
    const int pieces = a.group / (32 * FF);
    magic(a.n_groups == 1 ? 0 : pieces, a.piece_magic, a.piece_all);
    const auto kernel = packed_few_kernel<T, BITS, VW, FF, XR, RT, GATED>;
    if (waves * bytes > 65536) TB_HIP(ctx, hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, waves * bytes));
    hipLaunchKernelGGL(kernel, dim3((unsigned)cdiv64(a.d_out, 16 * RT), (unsigned)cdiv64(a.tokens, XR), a.splits), dim3(64 * waves), std::max(waves * bytes, waves * NR * 16 * 17 * 4), ctx->stream, a);
    TB_KERNEL_CHECK(ctx);
    if (a.splits > 1) {
        hipLaunchKernelGGL((packed_few_join_kernel<T>), dim3((unsigned)cdiv64(a.d_out, 256), (unsigned)a.tokens), dim3(256), 0, ctx->stream, a);
        TB_KERNEL_CHECK(ctx);
    }
    return 0;
}
template <typename T, int BITS, int VW, int FF, int XR, bool GATED>
int launch_few(tboa_ctx* ctx, const PackedArgs& a) {
    if constexpr (!GATED && XR == 64) return launch_few<T, BITS, VW, FF, XR, 2, GATED>(ctx, a);
    else if constexpr (!GATED && XR > 4) { if (a.d_out >= 16 * 2 * 256) return launch_few<T, BITS, VW, FF, XR, 2, GATED>(ctx, a); }
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
    for (int ff = most; ff >= least; ff /= 2) if (a.n_groups == 1 || a.group % (32 * ff) == 0) return divides(a, 32 * ff) ? ff : 0;
    return 0;
}

// ------------------------------------------------------------------------------------------------ many tokens
// Bound by the matrix instructions.  packed_rows_kernel makes X into half (bf16: exactly, fp32: as two terms), every row times a power of two that brings its largest channel to 2^14 .. 2^15, in the blocks of
// 16 rows x 32 channels that packed_many_kernel copies straight into LDS; and a table of the scales and zeros.  packed_many_kernel makes the codes into half on their way into LDS, once per tile of
// 256 outputs and TM tokens.
// Codes less zeros are exact in half.  A result is kept in the unit of the scale s_g of the group that its channels have come to: where a group begins, it is multiplied by s_(g-1) / s_g, so that the
// matrix instructions add to it what they add to any sum, and at the end by the last group's scale.  2048 tokens of 8192 x 4096, four bits, one scale a row 142 us, groups of 128 149, of 64 169, of 32 194, of 16
// 280; scale times code less zero as half instead, which is rounded twice to 11 bits (2e-4 of a result's size), 162 to 168 in groups.
struct ManyArgs {
    PackedArgs p;
    unsigned char* rows;          // X as half: [planes][token blocks of 16][kb][1 KB]
    float* row_scale;             // [tokens] power of two that takes a row's own back out
    unsigned* zeros;              // [n_groups][matrices][wide]: -(1024 + zero) as half, twice
    float* scales;                // [n_groups][matrices][wide]
    int wide, size;               // d_out rounded up to 256; bytes of an element of X and Y
    float* partial;               // [splits][tiles that are split][TM][256]: their channels are split over workgroups
    long long plane;              // bytes
    int kb, blocks;               // blocks of 32 channels, a multiple of four; of 16 tokens
    int full, splits;             // tiles that are not split (whole rounds of all compute units), how many ways the others are
    int tiles_m, tiles_n, segments, matrices;
    int units; unsigned unit_magic, unit_all;      // units of 16 channels that a group has, as PackedArgs::piece_magic
};
constexpr int KS = 32;      // channels of a stage

// the channels of a piece (8 of them, 16 bytes as half) in the order in which its codes are taken out of their word
template <int BITS>
constexpr int piece_channel(int i) { return BITS == 8 ? i : BITS == 4 ? i / 2 + i % 2 * 4 : BITS == 2 ? (i / 2) + i % 2 * 4 : i / 2 + i % 2 * 4; }

template <typename T, int BITS>
__global__ __launch_bounds__(1024) void packed_rows_kernel(ManyArgs a) {
    const PackedArgs& p = a.p;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if ((int)blockIdx.x >= a.blocks) {      // scales and zeros of 64 outputs, one a lane, a sixteenth of their groups a wavefront
        __shared__ float tops[16][64];
        const int b = blockIdx.x - a.blocks, per = a.wide / 64, which = b >= per, n = (b - which * per) * 64 + lane;
        const long long row = (long long)min(n, p.d_out - 1) * p.n_groups, at = (long long)which * a.wide + n, step = (long long)a.matrices * a.wide;
        const float* const scale = p.scale[which] + row, * const zero = p.zero[which] + row;
        float most = 0.f;
        for (int g = wave; g < p.n_groups; g += 16) { const float v = fabsf(scale[g]); most = v < __builtin_inff() ? fmaxf(most, v) : most; }
        tops[wave][lane] = most;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 16; ++i) most = fmaxf(most, tops[i][lane]);
        const float least = most > 0.f ? fmaxf(most * 0x1p-60f, 0x1p-149f) : 0.f;      // (quotients of scales stay numbers)
        for (int g = wave; g < p.n_groups; g += 16) {
            const unsigned z = __builtin_bit_cast(unsigned short, (_Float16)(-1024.f - zero[g]));
            a.zeros[g * step + at] = z | z << 16;
            const float v = scale[g];
            a.scales[g * step + at] = fabsf(v) < least ? least : v;
        }
        return;
    }
    __shared__ int exps[16];
    const long long m0 = (long long)blockIdx.x * 16;
    {      // a row per wavefront
        const T* const x = (const T*)p.X + min(m0 + wave, p.tokens - 1) * p.ldx;
        float most = 0.f;
        auto take = [&](float v) { v = fabsf(v); most = v < __builtin_inff() ? fmaxf(most, v) : most; };
        if (p.vec) {
            constexpr int E = 16 / (int)sizeof(T);
            const int whole = p.d_in / E * E;
            for (int k = lane * E; k < whole; k += 64 * E) {
                union { u4 u; T e[E]; } v;
                v.u = *(const u4*)(x + k);
#pragma unroll
                for (int j = 0; j < E; ++j) take(to_f32(v.e[j]));
            }
            for (int k = whole + lane; k < p.d_in; k += 64) take(to_f32(x[k]));
        } else for (int k = lane; k < p.d_in; k += 64) take(to_f32(x[k]));
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) most = fmaxf(most, __shfl_xor(most, o, 64));
        const int e = most > 0.f ? min(15 - __builtin_amdgcn_frexp_expf(most), 120) : 0;
        if (lane == 0) { exps[wave] = e; if (m0 + wave < p.tokens) a.row_scale[m0 + wave] = __builtin_amdgcn_ldexpf(1.f, -e); }
    }
    __syncthreads();
    const int row = threadIdx.x >> 1 & 15, half = threadIdx.x & 1, e = exps[row];      // a unit of 16 channels each: 32 lanes have a block
    const T* const x = (const T*)p.X + min(m0 + row, p.tokens - 1) * p.ldx;
    for (int kb = threadIdx.x >> 5; kb < a.kb; kb += 32) {
        const int k = kb * KS + half * 16;
        union { u4 u[sizeof(T)]; T e[16]; } in;
        if (p.vec && k + 16 <= p.d_in) {
#pragma unroll
            for (int i = 0; i < (int)sizeof(T); ++i) in.u[i] = ((const u4*)(x + k))[i];
        } else {
#pragma unroll
            for (int i = 0; i < (int)sizeof(T); ++i) in.u[i] = u4{0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < 16; ++j) if (k + j < p.d_in) in.e[j] = x[k + j];
        }
        union { _Float16 e[16]; u4 u[2]; } hi, lo;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float v = __builtin_amdgcn_ldexpf(to_f32(in.e[i / 8 * 8 + piece_channel<BITS>(i % 8)]), e);
            hi.e[i] = (_Float16)v;
            if constexpr (sizeof(T) == 4) lo.e[i] = (_Float16)(isfinite(v) ? v - (float)hi.e[i] : 0.f);
        }
        unsigned char* const out = a.rows + ((long long)blockIdx.x * a.kb + kb) * 1024 + row * 64;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int at = ((2 * half + i) ^ (row >> 2)) * 16;
            *(u4*)(out + at) = hi.u[i];
            if constexpr (sizeof(T) == 4) *(u4*)(out + a.plane + at) = lo.u[i];
        }
    }
}

// Codes of 128 channels of a row, as the four lanes of a quad load them: lane q has the 32 channels of stage q (8 bits: 16 channels of stages 0 and 1, 16 of stages 2 and 3)
template <int BITS> struct Codes128 { unsigned w[BITS == 8 ? 8 : BITS]; };
template <int P>
__device__ __forceinline__ unsigned quad(unsigned v) { return (unsigned)__builtin_amdgcn_mov_dpp((int)v, P, 0xf, 0xf, true); }
// the 8 codes of stage S that are lane j's of its quad, as half 1024 + code in pairs
template <int BITS, int S>
__device__ __forceinline__ void piece_halves(const Codes128<BITS>& in, int j, unsigned (&out)[4]) {
    constexpr unsigned ONE = 0x64006400u, OF = S * 0x55;      // quad_perm S S S S
    if constexpr (BITS == 8) {
        constexpr int a = S % 2 * 2, P = a | a << 2 | (a + 1) << 4 | (a + 1) << 6, at = S / 2 * 4;
        const unsigned q0 = quad<P>(in.w[at]), q1 = quad<P>(in.w[at + 1]), q2 = quad<P>(in.w[at + 2]), q3 = quad<P>(in.w[at + 3]);      // (of all lanes: not under a condition)
        const unsigned w0 = j & 1 ? q2 : q0, w1 = j & 1 ? q3 : q1;
        out[0] = __builtin_amdgcn_perm(0x64646464u, w0, 0x04010400u); out[1] = __builtin_amdgcn_perm(0x64646464u, w0, 0x04030402u);
        out[2] = __builtin_amdgcn_perm(0x64646464u, w1, 0x04010400u); out[3] = __builtin_amdgcn_perm(0x64646464u, w1, 0x04030402u);
    } else if constexpr (BITS == 4) {
        const unsigned q0 = quad<OF>(in.w[0]), q1 = quad<OF>(in.w[1]), q2 = quad<OF>(in.w[2]), q3 = quad<OF>(in.w[3]), a = j & 1 ? q1 : q0, b = j & 1 ? q3 : q2, w = j & 2 ? b : a;
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] = (w >> (4 * i) & 0x000f000fu) | ONE;
    } else if constexpr (BITS == 2) {
        const unsigned q0 = quad<OF>(in.w[0]), q1 = quad<OF>(in.w[1]), w = (j & 2 ? q1 : q0) >> (16 * (j & 1));      // 8 codes in 16 bits: 0 .. 3 below, 4 .. 7 brought above
        const unsigned v = (w & 0xffu) | (w & 0xff00u) << 8;
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] = (v >> (2 * i) & 0x00030003u) | ONE;
    } else {
        const unsigned w0 = quad<OF>(in.w[0]), w1 = quad<OF>(in.w[1]), w2 = quad<OF>(in.w[2]);
        const unsigned lo = j & 2 ? (j & 1 ? w2 : w1) : w0, hi = j & 2 ? w2 : w1;
        const unsigned w = __builtin_amdgcn_alignbit(hi, lo, j == 0 ? 0 : j == 1 ? 24 : j == 2 ? 16 : 8);      // 24 bits from 24 j on
        const unsigned v = (w & 0xfffu) | (w & 0xfff000u) << 4;
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] = (v >> (3 * i) & 0x00070007u) | ONE;
    }
}

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f16v __attribute__((ext_vector_type(16)));

// tile t in the order in which tiles are worked off: bands of four columns of tiles
__device__ __forceinline__ void tile_place(const ManyArgs& a, int t, int& tm, int& tn) {
    const int band = 4 * a.tiles_m, in = t % band, wide = min(4, a.tiles_n - t / band * 4);
    tn = t / band * 4 + in % wide; tm = in / wide;
}

// results n .. n + 3 of token m
template <typename T>
__device__ __forceinline__ void put4(const PackedArgs& p, long long m, int n, f4 v, bool may_add) {
    T* const y = (T*)p.Y + m * p.ldy + n;
    const T* const res = may_add && p.Res ? (const T*)p.Res + m * p.ldr + n : nullptr;
    struct __attribute__((aligned(4 * sizeof(T)))) Four { T e[4]; } o;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (n + k >= p.d_out) break;
        o.e[k] = from_f32(res ? v[k] + to_f32(res[k]) : v[k], T());
    }
    if (n + 4 <= p.d_out && p.out_vec) *(Four*)y = o;
    else for (int k = 0; k < 4; ++k) if (n + k < p.d_out) y[k] = o.e[k];
}

// A tile of TM tokens and 256 rows of codes (GATED: 128 of either matrix, 32 of one beside 32 of the other, so that a wavefront has both factors of its results); eight wavefronts, each TM / 2 tokens and 64 rows.
// A ring of NS stages of 32 channels in LDS: X is copied there, NS - 1 stages ahead; codes are loaded two stages before that, made into half and written by all wavefronts, 16 codes a lane and stage.
// Bound by the matrix instructions and the vector instructions that make codes into half beside them: 4096 tokens of 10240 x 8192, four bits in groups of 128, 651 us (1055 TFLOP/s), the matrix cores busy 51 %
// of the cycles and vector instructions issued in 48 %, at 1.85 GHz.  An earlier form, 677 us, against each wavefront making the codes of its own 64 rows 730 - 759, codes copied into LDS and made into half once
// for all 775.
// GRIDS_OF: 0: one scale a row; 1: groups of whole 128 channels, which begin where the ring does; 2: of whole 16, the depth of a matrix instruction, whose scales go through LDS.
template <int BITS, int GRIDS_OF, int TM, bool GATED>
__global__ __launch_bounds__(512) void packed_many_kernel(ManyArgs a) {
    constexpr int NS = 4, TI = TM / 64, TJ = 2, LPW = TM / 128, A_BYTES = TM * 64, STAGE = A_BYTES + 256 * 64, UNITS = 2 * NS;      // UNITS of 16 channels in a turn of the ring
    extern __shared__ __attribute__((aligned(1024))) unsigned char ring[];      // [NS][STAGE]; GRIDS_OF == 2: scales [3][UNITS][256]
    const PackedArgs& p = a.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, lh = lane >> 5;
    // tiles of one band of outputs after each other, an XCD (every eighth workgroup) its own run of them; then those that are split
    int tm, tn, split = 0, t;
    const int w = blockIdx.x, cut = a.tiles_m * a.tiles_n - a.full;
    if (w < a.full) t = (w & 7) * (a.full >> 3) + (w >> 3);
    else {
        const int total = cut * a.splits, per = (total + 7) / 8, v = w - a.full, item = (v & 7) * per + (v >> 3);
        if (v >> 3 >= per || item >= total) return;
        split = item % a.splits;
        t = a.full + item / a.splits;
    }
    const bool parts = w >= a.full && a.splits > 1;
    tile_place(a, t, tm, tn);
    const long long m0 = (long long)tm * TM;
    const int n0 = tn * (GATED ? 128 : 256);
    const int turns = a.kb / NS * a.segments, pieces = parts ? a.splits : 1, kt0 = (int)((long long)turns * split / pieces) * NS, nk = (int)((long long)turns * (split + 1) / pieces) * NS - kt0;      // (whole turns of the ring)

    // This thread's two rows of codes, of 256: row r of the tile and row r + 128, piece j of each in every stage
    const int r = threadIdx.x >> 2, j = threadIdx.x & 3;
    const int which = GATED ? r >> 5 & 1 : 0;
    auto output = [&](int row) { return GATED ? n0 + 32 * (row >> 6) + (row & 31) : n0 + row; };      // of a row of the tile (beyond the last one: tables go on, rows of codes do not)
    unsigned at_codes[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) at_codes[h] = (unsigned)(min(output(r + 128 * h), p.d_out - 1) - n0) * p.words * 4 + j * (BITS == 8 ? 16 : 4 * BITS);
    // (rows 32 .. 63 of every 64 are the second matrix's: the same for all of a wavefront's 16 rows)
    const uint32_t* const base = __builtin_amdgcn_readfirstlane(which) ? p.w[1] : p.w[0];
    const auto codes = __builtin_amdgcn_make_buffer_rsrc((void*)(base + (long long)n0 * p.words), 0, (int)(unsigned)min((long long)(p.d_out - n0) * p.words * 4, 0xfffffffcLL), 0x00020000);
    const long long table_step = (long long)a.matrices * a.wide;
    const unsigned at_zeros = which * a.wide + output(r);      // row r + 128: 128 outputs on, 64 of a gated tile
    const int wm = wave / 4 * (TM / 2), wn = wave % 4 * 64;
    const unsigned at_scales = output(wn) + l32;               // results: of the second 32 columns 32 outputs on, of a gated tile the other matrix's
    const unsigned next_scale = GATED ? a.wide : 32;
    constexpr int NG = GRIDS_OF == 2 ? NS : 1, NL = 2 * ((BITS == 8 ? 2 : 1) + (GRIDS_OF == 0 ? 0 : NG)) + (GRIDS_OF == 1 ? 2 : GRIDS_OF == 2);      // zeros of a row in NS stages; loads of `load`
    struct Load { Codes128<BITS> u[2]; unsigned z[2][NG]; float s[TJ]; };
    const unsigned ring_at = (unsigned)(unsigned long long)((__attribute__((address_space(3))) void*)ring);
    auto group_of = [&](unsigned unit) { return min((int)(__umulhi(unit, a.unit_magic) + (unit & a.unit_all)), p.n_groups - 1); };
    const unsigned row_zero[2] = {a.zeros[at_zeros], a.zeros[at_zeros + (GATED ? 64 : 128)]};      // GRIDS_OF == 0: the only ones
    int l_ks = kt0 % a.kb, l_slot = 0;      // of the next codes to be loaded, a multiple of NS; where their scales go
    auto load = [&](Load& o) {
        if constexpr (GRIDS_OF == 2) {      // a unit's scales a wavefront, four a lane
            const int row = 4 * lane;
            lds_direct_16(((GATED ? (row >> 5 & 1) * a.wide : 0) + output(row)) * 4, (const char*)(a.scales + group_of(l_ks * 2 + wave) * table_step), ring_at + NS * STAGE + (l_slot * UNITS + wave) * 1024);
            l_slot = l_slot == 2 ? 0 : l_slot + 1;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const unsigned at = at_codes[h] + l_ks * (BITS * 4);
            Codes128<BITS>& u = o.u[h];
            if constexpr (BITS == 8) {
#pragma unroll
                for (int i = 0; i < 2; ++i) { const u4 v = __builtin_amdgcn_raw_buffer_load_b128(codes, at + 64 * i, 0, 0); u.w[4 * i] = v[0]; u.w[4 * i + 1] = v[1]; u.w[4 * i + 2] = v[2]; u.w[4 * i + 3] = v[3]; }
            } else if constexpr (BITS == 4) { const u4 v = __builtin_amdgcn_raw_buffer_load_b128(codes, at, 0, 0); u.w[0] = v[0]; u.w[1] = v[1]; u.w[2] = v[2]; u.w[3] = v[3]; }
            else if constexpr (BITS == 2) { const auto v = __builtin_amdgcn_raw_buffer_load_b64(codes, at, 0, 0); u.w[0] = v[0]; u.w[1] = v[1]; }
            else { const auto v = __builtin_amdgcn_raw_buffer_load_b96(codes, at, 0, 0); u.w[0] = v[0]; u.w[1] = v[1]; u.w[2] = v[2]; }
#pragma unroll
            for (int i = 0; i < NG; ++i) o.z[h][i] = GRIDS_OF == 0 ? row_zero[h] : a.zeros[group_of((l_ks + i) * 2 + (GRIDS_OF == 2 ? j >> 1 : 0)) * table_step + at_zeros + h * (GATED ? 64 : 128)];
        }
        if constexpr (GRIDS_OF == 1) {
            const float* const s = a.scales + group_of(l_ks * 2) * table_step + at_scales;
            o.s[0] = s[0]; o.s[1] = s[next_scale];
        }
        l_ks += NS;
        if (l_ks >= a.kb) l_ks = 0;
    };
    unsigned char* const b_at = ring + A_BYTES + r * 64 + ((j ^ (r >> 2 & 3)) << 4);
    auto halves = [&](const Load& o, auto H, auto S, u4& out) {      // piece j of row h in stage S: codes less zeros
        constexpr int h = decltype(H)::value, st = decltype(S)::value;
        unsigned v[4];
        piece_halves<BITS, st>(o.u[h], j, v);
        const h2 z = __builtin_bit_cast(h2, o.z[h][GRIDS_OF == 2 ? st : 0]);
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] = __builtin_bit_cast(unsigned, __builtin_bit_cast(h2, v[i]) + z);
    };
    long long block[LPW];
#pragma unroll
    for (int i = 0; i < LPW; ++i) block[i] = min(m0 / 16 + wave * LPW + i, (long long)a.blocks - 1) * a.kb * 1024;
    int a_seg = kt0 / a.kb, a_ks = kt0 - a_seg * a.kb;      // of the next rows to be copied
    auto copy = [&](int slot) {
#pragma unroll
        for (int i = 0; i < LPW; ++i)
            lds_direct_16(lane * 16, (const char*)a.rows + (a_seg == 1 && a.segments > 1 ? a.plane : 0) + block[i] + (long long)a_ks * 1024, ring_at + slot * STAGE + (wave * LPW + i) * 1024);
        if (++a_ks == a.kb) { a_ks = 0; ++a_seg; }
    };
    auto x_piece = [&](int slot, int i, int ks) { const int row = wm + 32 * i + l32; return *(const h8*)(ring + slot * STAGE + row * 64 + (((2 * ks + lh) ^ (row >> 2 & 3)) << 4)); };
    auto w_piece = [&](int slot, int j, int ks) { const int row = wn + 32 * j + l32; return *(const h8*)(ring + slot * STAGE + A_BYTES + row * 64 + (((2 * ks + lh) ^ (row >> 2 & 3)) << 4)); };
    f16v acc[TI][TJ];
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
        for (int j = 0; j < TJ; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
    h8 fx[2][TI], fw[2][TJ];
    auto read = [&](int set, int slot, int ks) {
#pragma unroll
        for (int i = 0; i < TI; ++i) fx[set][i] = x_piece(slot, i, ks);
#pragma unroll
        for (int j = 0; j < TJ; ++j) fw[set][j] = w_piece(slot, j, ks);
    };
    float turn[TJ];      // from the unit of the results to that of the products that come
    auto multiply = [&](int set, auto TURNED) {
#pragma unroll
        for (int i = 0; i < TI; ++i)
#pragma unroll
            for (int j = 0; j < TJ; ++j) {
                if constexpr (decltype(TURNED)::value) acc[i][j] *= turn[j];
                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fx[set][i], fw[set][j], acc[i][j], 0, 0, 0);
            }
    };
    float scale[TJ];     // the unit of the results
    auto turn_to = [&](const float (&next)[TJ]) {
#pragma unroll
        for (int j = 0; j < TJ; ++j) { turn[j] = scale[j] == next[j] ? 1.f : scale[j] / next[j]; scale[j] = next[j]; }
    };
    auto arrived = [](Load& o) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (unsigned& w : o.u[h].w) asm volatile("" : "+v"(w));
#pragma unroll
            for (unsigned& z : o.z[h]) asm volatile("" : "+v"(z));
        }
        if constexpr (GRIDS_OF == 1) { asm volatile("" : "+v"(o.s[0])); asm volatile("" : "+v"(o.s[1])); }
    };
    // a run of matrix instructions: the next one's operands first, and vector instructions in the shadow of each
    auto beside = [](auto TURNED) {
        constexpr bool turned = decltype(TURNED)::value;
        __builtin_amdgcn_sched_group_barrier(0x100, TI + TJ, 0);
#pragma unroll
        for (int i = 0; i < TI * TJ; ++i) {
            if constexpr (turned) __builtin_amdgcn_sched_group_barrier(0x2, 16, 0);
            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0); __builtin_amdgcn_sched_group_barrier(0x2, TI == 4 ? 8 : 12, 0);
            if (i == TI * TJ * 5 / 8) __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);      // (what waits at the next barrier is then done)
        }
    };
    // As stage kt begins, stages kt .. kt + NS - 2 are in LDS or on their way there.  Codes are loaded for NS stages at once (kt and a.kb are multiples of NS) and written from the stage on that is NS - 1
    // before theirs: `here` has those of stages kt .. kt + NS - 1, `next` those of the NS after them.  Scales of GRIDS_OF == 2 are copied two turns ahead, the second of three slots being the next turn's.
    Load here, next, after_next;
    load(here);
    unroll<NS - 1>([&](auto S) {
        copy(S);
        unroll<2>([&](auto H) { u4 v; halves(here, H, S, v); *(u4*)(b_at + S * STAGE + H * 128 * 64) = v; });
    });
    load(next);
    arrived(next);
    wait_loads_but<0>();
    __syncthreads();
    const float* const scales_at = (const float*)(ring + NS * STAGE) + wn + l32;      // [slot][unit][256]
#pragma unroll
    for (int j = 0; j < TJ; ++j) scale[j] = GRIDS_OF == 2 ? scales_at[32 * j] : GRIDS_OF == 1 ? here.s[j] : 1.f;
    read(0, 0, 0);
    int slot = 0, unit = kt0 % a.kb * 2;      // GRIDS_OF == 2: of this turn's scales; of the row, its first unit
    for (int kt = 0; kt < nk; kt += NS) {
        if constexpr (GRIDS_OF == 1) turn_to(here.s);
        unroll<NS>([&](auto SS) {
            constexpr int s = SS, last = s == 0 ? NS - 1 : s - 1, after = s == NS - 1 ? 0 : s + 1;
            constexpr std::integral_constant<int, last> S;      // the written stage's number among its NS
            const Load& codes_of = s == 0 ? here : next;
            auto run = [&](auto H, auto TURNED) {
                constexpr int h = decltype(H)::value;
                u4 v;
                if constexpr (h == 0) read(1, s, 1); else read(0, after, 0);
                halves(codes_of, H, S, v);
                multiply(h, TURNED);
                *(u4*)(b_at + last * STAGE + h * 128 * 64) = v;
                beside(TURNED);
            };
            auto half_stage = [&](auto H) {
                constexpr int h = decltype(H)::value, u = 2 * s + h;
                if constexpr (GRIDS_OF == 2) {
                    const unsigned at = unit + u;
                    if ((__umulhi(at, a.unit_magic) + (at & a.unit_all)) * (unsigned)a.units == at) {      // a group begins
                        const float* const from = scales_at + (slot * UNITS + u) * 256;
                        const float more[TJ] = {from[0], from[32]};
                        turn_to(more);
#pragma unroll
                        for (int i = 0; i < TI; ++i)
#pragma unroll
                            for (int j = 0; j < TJ; ++j) acc[i][j] *= turn[j];
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                run(H, std::integral_constant<bool, GRIDS_OF == 1 && u == 0>());
            };
            copy(last);      // (the stage before this one has been read by everyone)
            if constexpr (s == 1) load(after_next);
            __builtin_amdgcn_sched_barrier(0);
            half_stage(std::integral_constant<int, 0>());
            // what the next stage has was copied two stages ago: two stages' copies may still be on their way, and the loads after the first of them (older ones are awaited with them)
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (s > 0) wait_loads_but<2 * LPW + NL>(); else wait_loads_but<2 * LPW>();
            __syncthreads();
            __builtin_amdgcn_sched_barrier(0);
            half_stage(std::integral_constant<int, 1>());
        });
        __builtin_amdgcn_sched_barrier(0);
        arrived(after_next);      // (here, where the newest copy is a stage old: the compiler, which does not know of the copies, waits for them too)
        here = next; next = after_next;
        if constexpr (GRIDS_OF == 2) { slot = slot == 2 ? 0 : slot + 1; unit += UNITS; if (unit == 2 * a.kb) unit = 0; }
    }
    // results through LDS, 32 tokens of a wavefront at a time: rows of 64 outputs
    if constexpr (GRIDS_OF == 0) { scale[0] = a.scales[at_scales]; scale[1] = a.scales[at_scales + next_scale]; }
    wait_loads_but<0>();
    __syncthreads();
    constexpr int WIDE = GATED ? 32 : 64, PITCH = WIDE + 4;
    float* const mine = (float*)(ring + wave * 32 * 68 * 4);
    const int c0 = GATED ? n0 + wn / 2 : n0 + wn;      // first output of the wavefront
#pragma unroll
    for (int i = 0; i < TI; ++i) {
        auto in_order = [] { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); __builtin_amdgcn_wave_barrier(); };
        const int sides = GATED && parts ? 2 : 1;
        for (int side = 0; side < sides; ++side) {      // (partial sums of a gated product: both factors, one after the other)
            in_order();
#pragma unroll
            for (int j = 0; j < (GATED ? 1 : TJ); ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const int row = 8 * (v / 4) + 4 * lh + v % 4;
                    float y = acc[i][j][v] * scale[j];
                    if constexpr (GATED) {
                        const float up = acc[i][1][v] * scale[1];
                        if (parts) y = side ? up : y;
                        else {
                            const float rs = a.row_scale[min(m0 + wm + 32 * i + row, p.tokens - 1)];
                            y = silu(y * rs) * (up * rs);      // (the row's power of two last: it alone may leave fp32, where the scale brings the product back)
                        }
                    }
                    mine[row * PITCH + 32 * j + l32] = y;
                }
            in_order();
            constexpr int LANES = WIDE / 4;      // that a row takes
#pragma unroll
            for (int q = 0; q < 32 * LANES / 64; ++q) {
                const int row = q * (64 / LANES) + lane / LANES, c = lane % LANES * 4, n = c0 + c;
                const long long m = m0 + wm + 32 * i + row;
                if (m >= p.tokens || n >= p.d_out) continue;
                f4 v = *(const f4*)(mine + row * PITCH + c);
                if (parts) {
                    *(f4*)(a.partial + (((long long)split * cut + (t - a.full)) * TM + (wm + 32 * i + row)) * 256 + (GATED ? side * 128 + wn / 2 : wn) + c) = v;
                    continue;
                }
                const float rs = GATED ? 1.f : a.row_scale[m];
                if (a.size == 2) put4<bf16>(p, m, n, v * rs, !GATED); else put4<float>(p, m, n, v * rs, !GATED);
            }
        }
    }
}

// sums of the splits' partial results of the tiles that are split
template <typename T, int TM, bool GATED>
__global__ __launch_bounds__(256) void packed_join_kernel(ManyArgs a) {
    constexpr int WIDE = GATED ? 128 : 256, LANES = WIDE / 4, ROWS = 256 / LANES;      // four outputs a thread
    const PackedArgs& p = a.p;
    const int cut = a.tiles_m * a.tiles_n - a.full, c = threadIdx.x % LANES * 4;
    for (int item = blockIdx.x; item < cut * (TM / ROWS); item += gridDim.x) {
        const int at = item / (TM / ROWS), row = item % (TM / ROWS) * ROWS + threadIdx.x / LANES;
        int tm, tn;
        tile_place(a, a.full + at, tm, tn);
        const long long m = (long long)tm * TM + row;
        const int n = tn * WIDE + c;
        if (m >= p.tokens || n >= p.d_out) continue;
        f4 y[2] = {f4{0.f, 0.f, 0.f, 0.f}, f4{0.f, 0.f, 0.f, 0.f}};
        const float* from = a.partial + ((long long)at * TM + row) * 256 + c;
#pragma unroll 4
        for (int s = 0; s < a.splits; ++s) { y[0] += *(const f4*)from; if (GATED) y[1] += *(const f4*)(from + 128); from += (long long)cut * TM * 256; }
        const float rs = a.row_scale[m];
        y[0] *= rs;
        if constexpr (GATED) {
            y[1] *= rs;
#pragma unroll
            for (int k = 0; k < 4; ++k) y[0][k] = silu(y[0][k]) * y[1][k];
        }
        put4<T>(p, m, n, y[0], !GATED);
    }
}

constexpr int CUS = 256;
constexpr long long MOST_ROWS = 8192;      // tokens of one round: more are worked off round by round, in the same workspace
// what a call of so many tokens is cut into, and the workspace for it
size_t many_room(const PackedArgs& p, bool gated, int size, long long tokens, ManyArgs& a, void* ws) {
    const int tm = tokens <= 128 ? 128 : 256;
    a.kb = (int)cdiv64(p.d_in, 4 * KS) * 4; a.blocks = (int)cdiv64(tokens, 16);
    a.segments = size == 2 ? 1 : 2; a.size = size;
    a.wide = (int)cdiv64(p.d_out, 256) * 256;
    a.tiles_m = (int)cdiv64(tokens, tm); a.tiles_n = (int)cdiv64(p.d_out, gated ? 128 : 256);
    const int tiles = a.tiles_m * a.tiles_n, cut = tiles % CUS;
    a.full = tiles - cut;
    a.splits = cut ? std::max(1, std::min(CUS / cut, a.kb / 4 * a.segments / 2)) : 1;
    if (a.splits == 1) a.full = tiles / 8 * 8;
    a.plane = (long long)a.blocks * a.kb * 1024;
    const int matrices = a.matrices = gated ? 2 : 1;
    Arena ar(ws);
    a.rows = ar.get<unsigned char>((size_t)a.plane * (size == 2 ? 1 : 2));
    a.row_scale = ar.get<float>((size_t)tokens);
    a.zeros = ar.get<unsigned>((size_t)matrices * a.wide * p.n_groups);
    a.scales = ar.get<float>((size_t)matrices * a.wide * p.n_groups);
    a.partial = ar.get<float>(a.splits > 1 ? (size_t)a.splits * cut * tm * 256 : 0);
    return ar.off;
}
// of all rounds of a call: the last one has fewer tokens and may still need more, where its tiles are split and those of a whole round are not
size_t rounds_room(const PackedArgs& p, bool gated, int size, long long tokens) {
    ManyArgs a{};
    const size_t first = many_room(p, gated, size, std::min(tokens, MOST_ROWS), a, nullptr), last = tokens % MOST_ROWS;
    return last ? std::max(first, many_room(p, gated, size, (long long)last, a, nullptr)) : first;
}
bool many_takes(const PackedArgs& p) { return (p.n_groups == 1 || p.group % 16 == 0) && divides(p, 16) && p.words <= 1 << 21; }

template <int BITS, int GRIDS_OF, int TM, bool GATED>
int launch_many(tboa_ctx* ctx, const ManyArgs& a) {
    constexpr int LDS = 4 * (TM + 256) * 64 + (GRIDS_OF == 2 ? 3 * 8 * 1024 : 0);
    const auto kernel = packed_many_kernel<BITS, GRIDS_OF, TM, GATED>;
    TB_HIP(ctx, hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, LDS));
    const int cut = a.tiles_m * a.tiles_n - a.full;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(a.full + cdiv64((a.tiles_m * a.tiles_n - a.full) * a.splits, 8) * 8)), dim3(512), LDS, ctx->stream, a);
    TB_KERNEL_CHECK(ctx);
    if (a.splits > 1) {
        const auto join = a.size == 2 ? packed_join_kernel<bf16, TM, GATED> : packed_join_kernel<float, TM, GATED>;
        hipLaunchKernelGGL(join, dim3((unsigned)std::min(cut * TM / (GATED ? 8 : 4), 1 << 16)), dim3(256), 0, ctx->stream, a);
        TB_KERNEL_CHECK(ctx);
    }
    return 0;
}
template <int BITS, int TM, bool GATED>
int launch_many(tboa_ctx* ctx, const ManyArgs& a) {
    if (a.p.n_groups == 1) return launch_many<BITS, 0, TM, GATED>(ctx, a);
    return a.p.group % 128 == 0 ? launch_many<BITS, 1, TM, GATED>(ctx, a) : launch_many<BITS, 2, TM, GATED>(ctx, a);
}
template <typename T, int BITS, bool GATED>
int launch_many(tboa_ctx* ctx, const PackedArgs& p) {
    ManyArgs a{};
    TB_TRY(tboa_ws_reserve(ctx, rounds_room(p, GATED, sizeof(T), p.tokens)));
    for (long long at = 0; at < p.tokens; at += MOST_ROWS) {
        a.p = p;
        a.p.tokens = std::min(p.tokens - at, MOST_ROWS);
        a.p.X = (const T*)p.X + at * p.ldx; a.p.Y = (T*)p.Y + at * p.ldy;
        if (p.Res) a.p.Res = (const T*)p.Res + at * p.ldr;
        if (many_room(p, GATED, sizeof(T), a.p.tokens, a, ctx->ws) > ctx->ws_bytes) return tboa_fail(ctx, TBOA_ENOMEM, "a workspace of %zu bytes is too small", ctx->ws_bytes);
        a.units = p.group / 16;
        magic(p.n_groups == 1 ? 0 : a.units, a.unit_magic, a.unit_all);
        hipLaunchKernelGGL((packed_rows_kernel<T, BITS>), dim3((unsigned)(a.blocks + a.matrices * (a.wide / 64))), dim3(1024), 0, ctx->stream, a);
        TB_KERNEL_CHECK(ctx);
        TB_TRY((a.p.tokens <= 128 ? launch_many<BITS, 128, GATED>(ctx, a) : launch_many<BITS, 256, GATED>(ctx, a)));
    }
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
    if (a.tokens > 64 && many_takes(a)) return launch_many<T, BITS, GATED>(ctx, a);
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

PackedArgs shape_of(const tboa_packed_weight& w) {
    PackedArgs a{};
    a.d_out = w.d_out; a.d_in = w.d_in; a.bits = w.bits; a.words = (int)tboa_packed_words_per_row(w.d_in, w.bits);
    a.group = w.group ? w.group : w.d_in; a.n_groups = w.d_in / a.group;
    return a;
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
    PackedArgs a = shape_of(*weight);
    const tboa_packed_weight* both[2] = {weight, up ? up : weight};
    for (int i = 0; i < 2; ++i) { a.w[i] = both[i]->packed; a.scale[i] = both[i]->scales; a.zero[i] = both[i]->zeros; }
    a.tokens = n_tokens; a.X = X; a.ldx = ldx; a.Res = Res; a.ldr = ldr; a.Y = Y; a.ldy = ldy;
    a.vec = (uintptr_t)X % 16 == 0 && ldx * size % 16 == 0 && ldx < 1 << 24;      // (the rows of a workgroup within 32 bits)
    a.out_vec = (uintptr_t)Y % (4 * size) == 0 && ldy % 4 == 0;
    if (dtype == TBOA_F32) return up ? launch<float, true>(ctx, weight->bits, a) : launch<float, false>(ctx, weight->bits, a);
    return up ? launch<bf16, true>(ctx, weight->bits, a) : launch<bf16, false>(ctx, weight->bits, a);
}

}  // namespace

extern "C" size_t tboa_packed_workspace_bytes(const tboa_packed_weight* weight, int64_t n_tokens, int dtype) {
    if (!good_weight(weight) || (dtype != TBOA_F32 && dtype != TBOA_BF16) || n_tokens <= 32 || n_tokens > 1 << 24) return 0;
    PackedArgs p = shape_of(*weight);
    size_t most = 0;
    if (dtype == TBOA_BF16) { p.tokens = std::min<long long>(n_tokens, 64); most = few_room(p); }
    if (n_tokens <= 64 || !many_takes(p)) return most;
    // a call of fewer tokens may need more (its tiles are split): the largest of all up to n_tokens, each the last with its number of tiles
    const long long last = std::min<long long>(n_tokens, MOST_ROWS);
    for (long long n = std::min(last, 128LL);; n = std::min(last, n / 256 * 256 + 256)) {
        ManyArgs a{};
        for (const bool gated : {false, true}) most = std::max(most, many_room(p, gated, dtype == TBOA_F32 ? 4 : 2, n, a, nullptr));
        if (n == last) return most;
    }
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
