// Norms and rotation of head vectors, and the append to a quantized key/value cache.
#include "kv_cache.h"
#include <math.h>
#include <algorithm>
#include <type_traits>

namespace {

typedef __hip_bfloat16 bf16;

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(bf16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16 from_f32<bf16>(float v) { return __float2bfloat16(v); }

__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
    const float4 a = ((const float4*)p)[0], b = ((const float4*)p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void load8(const bf16* p, float (&v)[8]) {
    const uint4 a = *(const uint4*)p;
    const unsigned w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
    ((float4*)p)[0] = make_float4(v[0], v[1], v[2], v[3]); ((float4*)p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(bf16* p, const float (&v)[8]) {
    union { bf16 h[8]; uint4 u; } o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o.h[i] = from_f32<bf16>(v[i]);
    *(uint4*)p = o.u;
}

struct Rotation { int dim, adjacent; long long positions; const float* table; };      // dim 0: none

template <typename T> struct RotateSide { const T* x; T* y; const float* w; long long ldx, ldy; int heads; };
template <typename T> struct RotateArgs { RotateSide<T> side[2]; long long tokens; int dh; double eps; Rotation rot; const int* positions; long long first; };      // first: head vector of this launch

// 1 / sqrt(mean of squares + eps) as 2^shift r, the sum in fp64: squares of 3e38 are within its range.  Values below 2^-64 or above 2^64 are moved there first (exactly, or where they would vanish
// beside the others anyway): fp32 holds the factor of 1e-39 not at all, that of 3e38 with fewer bits.
struct NormFactor { float r; int shift; };
__device__ __forceinline__ NormFactor norm_factor(double sum, int dh, double eps) {
    const double f = 1.0 / sqrt(sum / (double)dh + eps);
    const int shift = f > 0x1p64 ? 64 : f < 0x1p-64 ? -64 : 0;
    return NormFactor{(float)(shift ? ldexp(f, -shift) : f), shift};
}

// One lane per 16 channels, both halves of their pairs (channels 8 s .. and rot/2 + 8 s .., or 16 s .. where pairs are adjacent), `lpr` lanes per head vector.
// Every element is read and written once, in pieces of 16 bytes, and that is what bounds it: 16384 tokens, 64 + 8 heads of 128, bf16 (612 MB): 117 us, 5.2 TB/s; 16 tokens: 3.8 us.
template <typename T>
__global__ __launch_bounds__(256) void head_norm_rotate_kernel(RotateArgs<T> a, int lpr) {
    const int heads = a.side[0].heads + a.side[1].heads;
    const long long row = a.first + ((long long)blockIdx.x * 256 + threadIdx.x) / lpr;
    const int s = threadIdx.x & (lpr - 1);
    const bool live = row < a.tokens * heads;
    const long long t = live ? row / heads : 0;
    int h = live ? (int)(row % heads) : 0;
    const RotateSide<T>& d = a.side[h >= a.side[0].heads];
    if (h >= a.side[0].heads) h -= a.side[0].heads;
    const T* x = d.x + t * d.ldx + (long long)h * a.dh;
    T* y = d.y + t * d.ldy + (long long)h * a.dh;
    const bool mine = live && 16 * s < a.dh, turn = 16 * s < a.rot.dim;
    const int c0 = turn && !a.rot.adjacent ? 8 * s : 16 * s, c1 = turn && !a.rot.adjacent ? a.rot.dim / 2 + 8 * s : 16 * s + 8;
    float u[8] = {}, v[8] = {};
    if (mine) { load8(x + c0, u); load8(x + c1, v); }
    if (d.w) {
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += (double)u[i] * u[i] + (double)v[i] * v[i];
        for (int o = 1; o < lpr; o <<= 1) sum += __shfl_xor(sum, o, 64);
        const NormFactor f = norm_factor(sum, a.dh, a.eps);
        if (f.shift) {
#pragma unroll
            for (int i = 0; i < 8; ++i) { u[i] = __builtin_amdgcn_ldexpf(u[i], f.shift); v[i] = __builtin_amdgcn_ldexpf(v[i], f.shift); }
        }
        if (mine) {
#pragma unroll
            for (int i = 0; i < 8; ++i) { u[i] = u[i] * f.r * d.w[c0 + i]; v[i] = v[i] * f.r * d.w[c1 + i]; }
        }
    }
    if (!mine) return;
    if (turn) {
        const long long p = a.positions[t];
        float cs[8], sn[8];
        if (p >= 0 && p < a.rot.positions) {
            const float* tab = a.rot.table + p * a.rot.dim + 8 * s;
            load8(tab, cs); load8(tab + a.rot.dim / 2, sn);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) cs[i] = sn[i] = __builtin_nanf("");
        }
        if (a.rot.adjacent) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float e = u[2 * i], o = u[2 * i + 1], f = v[2 * i], g = v[2 * i + 1];
                u[2 * i] = e * cs[i] - o * sn[i]; u[2 * i + 1] = o * cs[i] + e * sn[i];
                v[2 * i] = f * cs[4 + i] - g * sn[4 + i]; v[2 * i + 1] = g * cs[4 + i] + f * sn[4 + i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) { const float e = u[i], o = v[i]; u[i] = e * cs[i] - o * sn[i]; v[i] = o * cs[i] + e * sn[i]; }
        }
    }
    store8(y + c0, u); store8(y + c1, v);
}

// channel that a channel is rotated with, and the pair's number
__device__ __forceinline__ int partner(int c, const Rotation& r, int& pair, bool& second) {
    if (r.adjacent) { pair = c >> 1; second = c & 1; return c ^ 1; }
    const int half = r.dim / 2;
    second = c >= half; pair = second ? c - half : c;
    return second ? c - half : c + half;
}

// Any sizes and alignment: one wavefront per head vector, a lane per channel; everything is read before anything is written (in place).  1003 tokens, 10 + 5 heads of 100, fp32 (12 MB): 10 us.
template <typename T>
__global__ __launch_bounds__(256) void head_norm_rotate_any_kernel(RotateArgs<T> a) {
    const int heads = a.side[0].heads + a.side[1].heads, lane = threadIdx.x & 63;
    const long long row = a.first + (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= a.tokens * heads) return;
    const long long t = row / heads;
    int h = (int)(row % heads);
    const RotateSide<T>& d = a.side[h >= a.side[0].heads];
    if (h >= a.side[0].heads) h -= a.side[0].heads;
    const T* x = d.x + t * d.ldx + (long long)h * a.dh;
    T* y = d.y + t * d.ldy + (long long)h * a.dh;
    float v[4], o[4];
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = lane + 64 * i;
        v[i] = o[i] = 0.f;
        if (c < a.dh) {
            v[i] = to_f32(x[c]);
            if (c < a.rot.dim) { int pair; bool second; o[i] = to_f32(x[partner(c, a.rot, pair, second)]); }
        }
        sum += (double)v[i] * v[i];
    }
    if (d.w) {
        for (int k = 1; k < 64; k <<= 1) sum += __shfl_xor(sum, k, 64);
        const NormFactor f = norm_factor(sum, a.dh, a.eps);
        if (f.shift) {
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[i] = __builtin_amdgcn_ldexpf(v[i], f.shift); o[i] = __builtin_amdgcn_ldexpf(o[i], f.shift); }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = lane + 64 * i;
            if (c < a.dh) {
                v[i] = v[i] * f.r * d.w[c];
                if (c < a.rot.dim) { int pair; bool second; o[i] = o[i] * f.r * d.w[partner(c, a.rot, pair, second)]; }
            }
        }
    }
    const long long p = a.rot.dim ? a.positions[t] : 0;
    const bool known = p >= 0 && p < a.rot.positions;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = lane + 64 * i;
        if (c >= a.dh) continue;
        float r = v[i];
        if (c < a.rot.dim) {
            int pair; bool second;
            partner(c, a.rot, pair, second);
            const float cs = known ? a.rot.table[p * a.rot.dim + pair] : __builtin_nanf(""), sn = known ? a.rot.table[p * a.rot.dim + a.rot.dim / 2 + pair] : __builtin_nanf("");
            r = second ? v[i] * cs + o[i] * sn : v[i] * cs - o[i] * sn;
        }
        y[c] = from_f32<T>(r);
    }
}

// ------------------------------------------------------------------------------------------------ append
template <typename T>
struct AppendArgs {
    KvGeometry g; KvBatch q;
    const T* x[2]; long long ld[2];      // K, V
    Rotation rot; const int* positions;
    unsigned char* cache; int unit_log, per; bool vec[2], vec_table;      // pieces of 8 channels, rows of the table in aligned pieces
};

// Scale and zero of a block from the ends of its new values and, where it has earlier tokens, from the stored grid; everything in fp64 on what is stored in fp32
struct Grid { double s, z, s0, z0; bool grown; };
__device__ __forceinline__ Grid block_grid(double lo, double hi, bool bad, bool had, float s_old, float z_old) {
    Grid r{0.0, 0.0, (double)s_old, (double)z_old, false};
    bad |= had && !(isfinite(s_old) && isfinite(z_old));
    if (bad) { r.s = __builtin_nan(""); return r; }
    if (had) {
        const double lo0 = -r.z0 * r.s0, hi0 = (255.0 - r.z0) * r.s0;
        if (lo >= lo0 - 0.5625 * r.s0 && hi <= hi0 + 0.5625 * r.s0) { r.s = r.s0; r.z = r.z0; return r; }
        lo = fmin(lo, lo0); hi = fmax(hi, hi0);
        r.grown = true;
    }
    if (lo == hi) { lo = -1.0; hi = 1.0; }
    r.s = fmax((double)(float)((hi - lo) / 255.0), 0x1p-126);
    r.z = rint(-lo / r.s);
    return r;
}
template <bool MOST, typename V>
__device__ __forceinline__ V pick(V a, V b) { return MOST ? fmax(a, b) : fmin(a, b); }
template <int CTRL>
__device__ __forceinline__ double dpp(double v) {
    const int lo = __builtin_amdgcn_mov_dpp(__double2loint(v), CTRL, 0xf, 0xf, true), hi = __builtin_amdgcn_mov_dpp(__double2hiint(v), CTRL, 0xf, 0xf, true);
    return __hiloint2double(hi, lo);
}
// over the LPT lanes of a token
template <int LPT, bool MOST>
__device__ __forceinline__ double of_token(double v) {
    v = pick<MOST>(v, dpp<0xB1>(v));      // quad_perm 1 0 3 2
    v = pick<MOST>(v, dpp<0x4E>(v));      // 2 3 0 1
    if constexpr (LPT > 4) v = pick<MOST>(v, dpp<0x141>(v));      // the other four of eight
    if constexpr (LPT > 8) v = pick<MOST>(v, dpp<0x140>(v));      // the other eight of sixteen
    return v;
}

template <typename T>
__device__ __forceinline__ void load_piece(const T* p, bool vec, int n, float (&o)[8]) {      // n of 8 channels are there
    if (vec && n == 8) { load8(p, o); return; }
#pragma unroll
    for (int j = 0; j < 8; ++j) { o[j] = 0.f; if (j < n) o[j] = to_f32(p[j]); }
}

// What a wavefront does with TOKENS tokens of a head.  LPT lanes per token, NP pieces of 8 channels in each (piece q + LPT i of a token is lane q's): the ends of a token are found in its lanes,
// whose grid is then theirs, and a token's levels leave as whole pieces; those of V turn by way of LDS into the tokens of a channel.
// Prompts of four sequences, 32 heads of 128, a grid per 16 tokens (147 MB): 89 us, three times what the bytes take at a copy's rate.  Half of the wavefronts' time is waiting for loads, which start
// tile after tile (two wavefronts per SIMD: FORM 4 for bf16 takes all 256 registers and spills 66, addresses of the branch for unaligned rows); 29 % is vector instructions, 36 a
// value on average (those of keys partly in fp64, which is what the grid is decided in).
// As many lanes per token as it has pieces, up to 16 (timed in graphs of 20 calls): four with up to eight pieces each took 14.4 us instead of 5.0 for a token of each of 64 sequences, 50 instead
// of 42 for four prompts of 2000 (8 heads, a grid per token).
// ROT: keys, rotated in fp64 (products of 24 bits are exact there); a piece's partners are read once more.  Else the inputs themselves, in fp32.  Levels come from fp32 products, and a piece with such
// a product within 2^-21 of a border from the fp64 quotients (three roundings are off by 3 * 2^-24 of it).
template <typename T, int LPT, int NP, bool ROT>
struct AppendTile {
    static constexpr int TOKENS = 64 / LPT;
    typedef typename std::conditional<ROT, double, float>::type V;
    const AppendArgs<T>& a;
    int kv, lane, tok, q;
    bool vec;
    V v[NP][8];

    __device__ __forceinline__ AppendTile(const AppendArgs<T>& args, int kv_) : a(args), kv(kv_) { lane = threadIdx.x & 63; tok = lane / LPT; q = lane % LPT; vec = a.vec[kv]; }
    __device__ __forceinline__ int channel(int i) const { return 8 * (q + LPT * i); }
    // row, p: of the tile's first token, its place; fresh: this lane's token is new
    __device__ __forceinline__ void fetch(int row, int p, int h, bool fresh) {
        const int dh = a.g.dh, rot = a.rot.dim, half = rot / 2;
        const T* const src = a.x[kv] + (long long)(row + tok) * a.ld[kv] + (long long)h * dh;
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = 0;
        if (!fresh) return;
        float raw[NP][8];
#pragma unroll
        for (int i = 0; i < NP; ++i) load_piece(src + channel(i), vec, min(max(dh - channel(i), 0), 8), raw[i]);
        if constexpr (!ROT) {
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] = raw[i][j];
        } else {
            const long long at = a.positions ? a.positions[row + tok] : p + tok;
            const bool known = at >= 0 && at < a.rot.positions, adjacent = a.rot.adjacent;
            const float* const tab = a.rot.table + (known ? at : 0) * rot;
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int c = channel(i);
                float other[8], cs[8], sn[8];
                if (c >= rot) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[i][j] = (double)raw[i][j];
                    continue;
                }
                if (adjacent) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) other[j] = raw[i][j ^ 1];
                    if (a.vec_table) {
                        const float4 x = *(const float4*)(tab + c / 2), y = *(const float4*)(tab + half + c / 2);
                        cs[0] = cs[1] = x.x; cs[2] = cs[3] = x.y; cs[4] = cs[5] = x.z; cs[6] = cs[7] = x.w;
                        sn[0] = -y.x; sn[1] = y.x; sn[2] = -y.y; sn[3] = y.y; sn[4] = -y.z; sn[5] = y.z; sn[6] = -y.w; sn[7] = y.w;
                    }
                } else if (a.vec_table && vec) {      // a piece is of one half
                    const bool second = c >= half;
                    load8(src + (second ? c - half : c + half), other);
                    load8(tab + (second ? c - half : c), cs); load8(tab + (second ? c : c + half), sn);
                    if (!second) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) sn[j] = -sn[j];
                    }
                }
                if (!a.vec_table || (!adjacent && !vec)) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        other[j] = cs[j] = sn[j] = 0.f;
                        if (c + j < rot) {
                            int pair; bool second;
                            other[j] = to_f32(src[partner(c + j, a.rot, pair, second)]);
                            cs[j] = tab[pair]; sn[j] = second ? tab[half + pair] : -tab[half + pair];
                        } else cs[j] = 1.f;
                    }
                }
                const double lost = known ? 0.0 : __builtin_nan("");
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    v[i][j] = fma((double)raw[i][j], (double)cs[j], (double)other[j] * (double)sn[j]);      // (the product is exact)
                    if (!known && c + j < rot) v[i][j] = lost;
                }
                __builtin_amdgcn_sched_barrier(0);      // a piece at a time: all pieces' operands side by side do not fit in the registers
            }
        }
    }
    // ends of this lane's token, and whether one of its values is no number
    __device__ __forceinline__ void ends(double& lo, double& hi, bool& bad) {
        V l = 0, u = 0, none = 0;
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) { l = pick<false>(l, v[i][j]); u = pick<true>(u, v[i][j]); none = fma(v[i][j], (V)0, none); }      // (an infinity or NaN leaves NaN)
        lo = of_token<LPT, false>((double)l); hi = of_token<LPT, true>((double)u);
        int wrong = none != 0;
        wrong |= __builtin_amdgcn_mov_dpp(wrong, 0xB1, 0xf, 0xf, true); wrong |= __builtin_amdgcn_mov_dpp(wrong, 0x4E, 0xf, 0xf, true);
        if constexpr (LPT > 4) wrong |= __builtin_amdgcn_mov_dpp(wrong, 0x141, 0xf, 0xf, true);
        if constexpr (LPT > 8) wrong |= __builtin_amdgcn_mov_dpp(wrong, 0x140, 0xf, 0xf, true);
        bad = wrong;
    }
    // levels of the token: new (fresh), or one of the `before` first ones of a block whose grid has grown
    __device__ __forceinline__ void put(unsigned char* tile, bool fresh, int before, const Grid& g, unsigned char* lds) {
        const int dp = a.g.dp, dh = a.g.dh;
        const bool moved = tok < before && g.grown, set = fresh || moved;
        const unsigned long long sets = __ballot(set);
        if (!sets) return;
        const float inv = (float)(1.0 / g.s), z = (float)g.z;
        unsigned w[NP][2] = {};
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int c = channel(i);
            float n[8];
            bool close = false;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float x = (float)v[i][j] * inv;
                n[j] = rintf(x);
                close |= !(fabsf(x - n[j]) < fmaf(fabsf(x), -0x1p-21f, 0.5f - 0x1p-21f));
            }
            if (close) {
#pragma unroll
                for (int j = 0; j < 8; ++j) n[j] = (float)rint((double)v[i][j] / g.s);
            }
            if (moved) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int ch = min(c + j, dh - 1);
                    n[j] = (float)(rint(((double)tile[kv ? ch * 16 + tok : tok * dp + ch] - g.z0) * g.s0 / g.s));
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) w[i][j >> 2] |= (unsigned)fminf(fmaxf(n[j] + z, 0.f), 255.f) << 8 * (j & 3);      // (NaN: 0)
        }
        if (!kv) {
            if (!set) return;
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int c = channel(i);
                unsigned char* const p = tile + tok * dp + c;
                if (c + 8 <= dh) *(uint2*)p = make_uint2(w[i][0], w[i][1]);
                else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) if (c + j < dh) p[j] = (unsigned char)(w[i][j >> 2] >> 8 * (j & 3));
                }
            }
        } else if (sets == ~0ull) {
            typedef unsigned Column __attribute__((ext_vector_type(TOKENS / 4)));
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) lds[(channel(i) + j) * TOKENS + tok] = (unsigned char)(w[i][j >> 2] >> 8 * (j & 3));
            __builtin_amdgcn_wave_barrier();      // (its own part of LDS)
#pragma unroll
            for (int i = 0; i < (8 * LPT * NP + 63) / 64; ++i) { const int c = lane + 64 * i; if (c < dh) *(Column*)(tile + c * 16) = *(const Column*)(lds + c * TOKENS); }
            __builtin_amdgcn_wave_barrier();
        } else if (set) {
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) if (channel(i) + j < dh) tile[(channel(i) + j) * 16 + tok] = (unsigned char)(w[i][j >> 2] >> 8 * (j & 3));
        }
    }
};

// A unit of max(TOKENS, scale_tokens) tokens of a sequence
constexpr int MOST_WAVES = 8;      // of a workgroup
struct Unit {
    int first, place, end, row0;      // first place that gets a token, the unit's first place and the end of its places; row of place p: row0 + p
    unsigned char* page;
    int in_page;
};

template <typename T, int LPT, int NP, bool ROT, int FORM>
__device__ __forceinline__ void append_unit(const AppendArgs<T>& a, const Unit& u, int kv, unsigned char* lds) {
    typedef AppendTile<T, LPT, NP, ROT> Tile;
    constexpr int TOKENS = Tile::TOKENS;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, st_log = a.g.st_log, st = 1 << st_log, pt = 1 << a.g.pt_log, tok = lane / LPT;
    auto is_new = [&](int p) { return p >= u.first && p < u.end; };
    auto grids_of = [&](int h) { return (float2*)(u.page + (kv ? a.g.vg_at : a.g.kg_at)) + ((long long)h << (a.g.pt_log - st_log)) + (u.in_page >> st_log); };
    auto levels_of = [&](int h, int j) {      // of the unit's tile j
        const int at = u.in_page + TOKENS * j;
        return kv ? u.page + a.g.v_at + ((long long)h * pt + (at & ~15)) * a.g.dp + (at & 15) : u.page + ((long long)h * pt + at) * a.g.dp;
    };
    if constexpr (FORM > 0) {
        const int t_block = FORM == 1 ? tok & ~(st - 1) : 0, p_block = u.place + t_block, tiles = FORM == 1 ? 1 : (1 << a.unit_log) / TOKENS;
        const bool touched = p_block < u.end && p_block + st > u.first, had = touched && p_block < u.first;
        const int h0 = ((int)blockIdx.y * 4 + wave) * a.per, h1 = min(h0 + a.per, a.g.heads);
        for (int h = h0; h < h1; ++h) {
            float2* const grid = grids_of(h) + (FORM == 1 ? tok >> st_log : 0);
            float2 old = make_float2(0.f, 0.f);
            if (had) old = *grid;
            Tile t[4] = {Tile(a, kv), Tile(a, kv), Tile(a, kv), Tile(a, kv)};
            double lo = 0.0, hi = 0.0;
            bool bad = false;
#pragma unroll
            for (int k = 0; k < FORM; ++k) {
                const int p = u.place + TOKENS * k;
                if (FORM > 1 && (k >= tiles || p >= u.end || p + TOKENS <= u.first)) continue;
                t[k].fetch(u.row0 + p, p, h, is_new(p + tok));
                double l, m;
                bool w;
                t[k].ends(l, m, w);
                lo = fmin(lo, l); hi = fmax(hi, m); bad |= w;
            }
            for (int o = LPT; o < (FORM == 1 ? LPT << st_log : 64); o <<= 1) { lo = fmin(lo, __shfl_xor(lo, o, 64)); hi = fmax(hi, __shfl_xor(hi, o, 64)); bad |= __shfl_xor((int)bad, o, 64) != 0; }
            const Grid g = block_grid(lo, hi, bad, had, old.x, old.y);
#pragma unroll
            for (int k = 0; k < FORM; ++k) {
                const int p = u.place + TOKENS * k;
                if (FORM > 1 && k >= tiles) continue;
                t[k].put(levels_of(h, k), is_new(p + tok), min(max(u.first - p, 0), TOKENS), g, lds);
            }
            if (touched && lane == LPT * t_block) *grid = make_float2((float)g.s, (float)g.z);
        }
    } else {
        __shared__ double ends[2][2][MOST_WAVES];
        __shared__ int bads[2][MOST_WAVES];
        constexpr int KEPT = NP == 1 ? 2 : 1;      // tiles that a wavefront keeps the values of
        const int tiles = (1 << a.unit_log) / TOKENS, waves = blockDim.x >> 6, h0 = (int)blockIdx.y * a.per, h1 = min(h0 + a.per, a.g.heads);
        const bool had = u.place < u.first, once = tiles <= KEPT * waves;
        auto some_new = [&](int p) { return p < u.end && p + TOKENS > u.first; };
        for (int h = h0; h < h1; ++h) {
            Tile t[2] = {Tile(a, kv), Tile(a, kv)};
            double lo = 0.0, hi = 0.0;
            bool bad = false;
            for (int j0 = wave; j0 < tiles; j0 += KEPT * waves)
#pragma unroll
                for (int k = 0; k < KEPT; ++k) {
                    const int j = j0 + k * waves, p = u.place + TOKENS * j;
                    if (j >= tiles || !some_new(p)) continue;
                    t[k].fetch(u.row0 + p, p, h, is_new(p + tok));
                    double l, m;
                    bool w;
                    t[k].ends(l, m, w);
                    lo = fmin(lo, l); hi = fmax(hi, m); bad |= w;
                }
#pragma unroll
            for (int o = LPT; o < 64; o <<= 1) { lo = fmin(lo, __shfl_xor(lo, o, 64)); hi = fmax(hi, __shfl_xor(hi, o, 64)); bad |= __shfl_xor((int)bad, o, 64) != 0; }
            const int turn = h & 1;      // (what the head before this one left is still read)
            if (lane == 0) { ends[turn][0][wave] = lo; ends[turn][1][wave] = hi; bads[turn][wave] = bad; }
            float2* const grid = grids_of(h);
            float2 old = make_float2(0.f, 0.f);
            if (had) old = *grid;
            __syncthreads();
            for (int w = 0; w < waves; ++w) { lo = fmin(lo, ends[turn][0][w]); hi = fmax(hi, ends[turn][1][w]); bad |= bads[turn][w] != 0; }
            const Grid g = block_grid(lo, hi, bad, had, old.x, old.y);
            if (threadIdx.x == 0) *grid = make_float2((float)g.s, (float)g.z);
            for (int j0 = wave; j0 < tiles; j0 += KEPT * waves)
#pragma unroll
                for (int k = 0; k < KEPT; ++k) {
                    const int j = j0 + k * waves, p = u.place + TOKENS * j;
                    if (j >= tiles) continue;
                    if (!once && some_new(p)) t[k].fetch(u.row0 + p, p, h, is_new(p + tok));
                    t[k].put(levels_of(h, j), is_new(p + tok), min(max(u.first - p, 0), TOKENS), g, lds);
                }
        }
    }
}

// One workgroup per unit and group of heads, K (blockIdx.z 0) or V.  FORM 1: a unit is one tile, of one or more blocks; 4: one block of at most four tiles.  In both, each of the four wavefronts
// has `per` heads of its own.  FORM 0: one block of more tiles, which all wavefronts share for the same `per` heads.
template <typename T, int LPT, int NP, int FORM>
__global__ __launch_bounds__(FORM ? 256 : 64 * MOST_WAVES, 2) void kv_append_kernel(AppendArgs<T> a) {
    __shared__ __align__(16) unsigned char turned[FORM ? 4 : MOST_WAVES][8 * LPT * NP * (64 / LPT)];
    const int ul = a.unit_log, room = a.q.room;
    int x = blockIdx.x, b;
    KvSeq s;
    if (!kv_find(a.q, kv_head(a.q), [ul, room](const KvSeq& e) {
            const int p0 = max(e.len - e.n, 0), end = min(e.len, room);
            return end > p0 && e.n > 0 ? ((end - 1) >> ul) - (p0 >> ul) + 1 : 0; }, x, b, s)) return;
    Unit u;
    u.first = max(s.len - s.n, 0);
    u.place = __builtin_amdgcn_readfirstlane(((u.first >> ul) + x) << ul);
    u.end = min(u.place + (1 << ul), min(s.len, room));
    u.row0 = s.start + s.n - s.len;
    const int page = a.q.pages[(long long)b * a.q.per_seq + (u.place >> a.g.pt_log)];
    if (page < 0 || page >= (int)a.g.n_pages) return;
    u.page = a.cache + (long long)page * a.g.page_bytes;
    u.in_page = u.place & ((1 << a.g.pt_log) - 1);
    unsigned char* const lds = turned[threadIdx.x >> 6];
    if (blockIdx.z == 0 && a.rot.dim) append_unit<T, LPT, NP, true, FORM>(a, u, 0, lds);
    else append_unit<T, LPT, NP, false, FORM>(a, u, blockIdx.z, lds);
}

template <typename T>
int head_norm_rotate(tboa_ctx* ctx, long long n_tokens, int dh, int nq, const void* Q, long long ldq, const float* wq, int nk, const void* K, long long ldk, const float* wk, double eps,
                     const Rotation& rot, const int* positions, void* Qo, long long ldqo, void* Ko, long long ldko) {
    RotateArgs<T> a{{{(const T*)Q, (T*)Qo, wq, ldq, ldqo, nq}, {(const T*)K, (T*)Ko, wk, ldk, ldko, nk}}, n_tokens, dh, eps, rot, positions, 0};
    const long long rows = n_tokens * (nq + nk);
    // 16-byte pieces where every head vector and table row starts on a 16-byte boundary and the pairs of 16 channels are whole pieces
    const int e = 16 / (int)sizeof(T);
    bool vec = dh % 16 == 0 && rot.dim % 16 == 0 && ((uintptr_t)rot.table & 15) == 0;
    for (const auto& d : a.side) vec &= !d.heads || ((((uintptr_t)d.x | (uintptr_t)d.y) & 15) == 0 && d.ldx % e == 0 && d.ldy % e == 0);
    int lpr = 1;
    while (16 * lpr < dh) lpr *= 2;
    const int per = vec ? 256 / lpr : 4;      // of a workgroup
    constexpr long long MOST_BLOCKS = 1 << 23;      // of a launch: of 2^32 work items and more the runtime starts what is left modulo 2^32
    for (; a.first < rows; a.first += MOST_BLOCKS * per) {
        const dim3 grid((unsigned)std::min<long long>(cdiv64(rows - a.first, per), MOST_BLOCKS));
        if (vec) hipLaunchKernelGGL((head_norm_rotate_kernel<T>), grid, dim3(256), 0, ctx->stream, a, lpr);
        else hipLaunchKernelGGL((head_norm_rotate_any_kernel<T>), grid, dim3(256), 0, ctx->stream, a);
        TB_KERNEL_CHECK(ctx);
    }
    return 0;
}

template <typename T, int LPT, int NP>
int append(tboa_ctx* ctx, AppendArgs<T> a) {
    int tile_log = 0;
    while (LPT << tile_log < 64) ++tile_log;
    a.unit_log = std::max(tile_log, a.g.st_log);
    const int tiles = 1 << (a.unit_log - tile_log), waves = tiles <= (NP == 1 ? 4 : 1) ? 1 : std::min(tiles, MOST_WAVES);
    const long long units = std::min<long long>(a.q.n_tokens, (a.q.n_tokens >> a.unit_log) + 2LL * a.q.n_seqs);
    // heads that one wavefront, or a workgroup of several tiles, goes through: as few as fill the chip (256 compute units, 16 wavefronts each), for the tile is found once for all of them
    const int most = (int)std::min<long long>(std::max<long long>(units * a.g.heads * 2 * waves / 4096, 1), 8) * (waves > 1 ? 1 : 4);      // of a workgroup
    const unsigned groups = (unsigned)((a.g.heads + most - 1) / most);
    a.per = (a.g.heads + (int)groups - 1) / (int)groups;
    if (waves == 1) a.per = (a.per + 3) / 4;
    if (waves > 1) hipLaunchKernelGGL((kv_append_kernel<T, LPT, NP, 0>), dim3((unsigned)units, groups, 2), dim3(64 * waves), 0, ctx->stream, a);
    else if (tiles == 1) hipLaunchKernelGGL((kv_append_kernel<T, LPT, NP, 1>), dim3((unsigned)units, groups, 2), dim3(256), 0, ctx->stream, a);
    else if constexpr (NP == 1) hipLaunchKernelGGL((kv_append_kernel<T, LPT, NP, 4>), dim3((unsigned)units, groups, 2), dim3(256), 0, ctx->stream, a);
    TB_KERNEL_CHECK(ctx);
    return 0;
}
template <typename T, int DP>
int append(tboa_ctx* ctx, const AppendArgs<T>& a) {
    constexpr int LANES = DP <= 32 ? 4 : DP <= 64 ? 8 : 16;
    return append<T, LANES, (DP / 8 + LANES - 1) / LANES>(ctx, a);
}
template <typename T>
int append(tboa_ctx* ctx, AppendArgs<T> a) {
    const int e = 16 / (int)sizeof(T);
    for (int i = 0; i < 2; ++i) a.vec[i] = a.g.dh % 8 == 0 && ((uintptr_t)a.x[i] & 15) == 0 && a.ld[i] % e == 0;
    a.vec_table = a.rot.dim % 16 == 0 && ((uintptr_t)a.rot.table & 15) == 0;
    switch (a.g.dp) {
        case 32: return append<T, 32>(ctx, a);
        case 64: return append<T, 64>(ctx, a);
        case 96: return append<T, 96>(ctx, a);
        case 128: return append<T, 128>(ctx, a);
        case 192: return append<T, 192>(ctx, a);
        default: return append<T, 256>(ctx, a);
    }
}

int check_rotation(tboa_ctx* ctx, const char* who, const tboa_rotation* r, int dh, Rotation& out) {
    out = Rotation{0, 0, 0, nullptr};
    if (!r || r->rot_dim == 0) return 0;
    if (r->rot_dim < 0 || r->rot_dim > dh || r->rot_dim % 2 || r->n_positions <= 0 || !r->cos_sin || ((uintptr_t)r->cos_sin & 3))
        return tboa_fail(ctx, TBOA_EINVAL, "%s: rotation of %d of %d channels (an even number), a table of at least one position", who, r->rot_dim, dh);
    out = Rotation{r->rot_dim, r->adjacent != 0, r->n_positions, r->cos_sin};
    return 0;
}

}  // namespace

bool kv_geometry(const tboa_kv_cache_desc* d, KvGeometry& g) {
    if (!d || d->n_kv_heads <= 0 || d->n_kv_heads > 65535 || d->head_dim <= 0 || d->head_dim > 256 || d->page_tokens < 16 || d->page_tokens > 1024 || d->scale_tokens < 1 ||
        d->scale_tokens > d->page_tokens || (d->page_tokens & (d->page_tokens - 1)) || (d->scale_tokens & (d->scale_tokens - 1)) || d->n_pages < 0 || d->n_pages > 2147483647LL) return false;
    g.heads = d->n_kv_heads; g.dh = d->head_dim; g.dp = kv_padded_head(d->head_dim); g.n_pages = d->n_pages;
    for (g.pt_log = 4; (1 << g.pt_log) < d->page_tokens;) ++g.pt_log;
    for (g.st_log = 0; (1 << g.st_log) < d->scale_tokens;) ++g.st_log;
    const long long levels = (long long)g.heads * d->page_tokens * g.dp, grids = (long long)g.heads * (d->page_tokens / d->scale_tokens) * 8;
    g.v_at = levels; g.kg_at = 2 * levels; g.vg_at = 2 * levels + grids;
    g.page_bytes = (2 * levels + 2 * grids + 255) & ~255LL;
    return d->n_pages == 0 || g.page_bytes <= (1LL << 62) / d->n_pages;
}

int kv_check(tboa_ctx* ctx, const char* who, const tboa_kv_cache_desc* d, const tboa_kv_batch* b, const void* cache, KvGeometry& g) {
    if (!d || !b) return tboa_fail(ctx, TBOA_EINVAL, "%s: null descriptor", who);
    if (!kv_geometry(d, g))
        return tboa_fail(ctx, TBOA_EINVAL, "%s: a cache has heads of 1 .. 256 channels, pages of 16 .. 1024 tokens and scales of 1 .. page_tokens tokens (powers of two)", who);
    if (b->n_seqs < 0 || b->n_tokens < 0 || b->n_tokens > 1 << 24 || b->n_seqs > 1 << 20 || b->pages_per_seq < 0 || b->max_new < 0)
        return tboa_fail(ctx, TBOA_EINVAL, "%s: bad batch (at most 2^24 tokens and 2^20 sequences)", who);
    if (b->n_seqs == 0 || b->n_tokens == 0) return 0;
    if (!b->starts || !b->lens || (b->pages_per_seq > 0 && !b->pages)) return tboa_fail(ctx, TBOA_EINVAL, "%s: null starts, lens or pages", who);
    if ((long long)b->pages_per_seq * d->page_tokens > KV_MOST_TOKENS) return tboa_fail(ctx, TBOA_EINVAL, "%s: sequences of at most 2^30 tokens", who);
    if (d->n_pages > 0 && (!cache || ((uintptr_t)cache & 15))) return tboa_fail(ctx, TBOA_EINVAL, "%s: the cache must be 16-byte aligned device memory", who);
    return 0;
}

extern "C" size_t tboa_kv_cache_page_bytes(const tboa_kv_cache_desc* desc) {
    KvGeometry g;
    return kv_geometry(desc, g) ? (size_t)g.page_bytes : 0;
}

extern "C" int tboa_head_norm_rotate(tboa_ctx* ctx, int64_t n_tokens, int head_dim, int dtype, int n_q_heads, const void* Q, int64_t ldq, const float* w_q, int n_k_heads, const void* K,
                                     int64_t ldk, const float* w_k, double eps, const tboa_rotation* rotation, const int* positions, void* Q_out, int64_t ldq_out, void* K_out,
                                     int64_t ldk_out) {
    if (!ctx) return TBOA_EINVAL;
    if (n_tokens < 0 || n_tokens > 2147483647LL || head_dim <= 0 || head_dim > 256 || n_q_heads < 0 || n_k_heads < 0 || n_q_heads > 65535 || n_k_heads > 65535)
        return tboa_fail(ctx, TBOA_EINVAL, "head_norm_rotate: heads of 1 .. 256 channels, at most 2^31 - 1 tokens");
    if (dtype != TBOA_F32 && dtype != TBOA_BF16) return tboa_fail(ctx, TBOA_EINVAL, "head_norm_rotate: dtype must be fp32 or bf16");
    Rotation rot;
    TB_TRY(check_rotation(ctx, "head_norm_rotate", rotation, head_dim, rot));
    if ((w_q || w_k) && !(eps >= 0.0 && eps <= 1e30)) return tboa_fail(ctx, TBOA_EINVAL, "head_norm_rotate: eps=%g", eps);
    if (n_tokens == 0 || n_q_heads + n_k_heads == 0) return 0;
    if ((n_q_heads && (!Q || !Q_out)) || (n_k_heads && (!K || !K_out)) || (rot.dim && !positions)) return tboa_fail(ctx, TBOA_EINVAL, "head_norm_rotate: null argument");
    const int64_t wide_q = (int64_t)n_q_heads * head_dim, wide_k = (int64_t)n_k_heads * head_dim;
    if ((n_q_heads && (ldq < wide_q || ldq_out < wide_q)) || (n_k_heads && (ldk < wide_k || ldk_out < wide_k)))
        return tboa_fail(ctx, TBOA_EINVAL, "head_norm_rotate: a row pitch is smaller than its heads");
    KvDevice dev(ctx->device);
    if (dtype == TBOA_F32) return head_norm_rotate<float>(ctx, n_tokens, head_dim, n_q_heads, Q, ldq, w_q, n_k_heads, K, ldk, w_k, eps, rot, positions, Q_out, ldq_out, K_out, ldk_out);
    return head_norm_rotate<bf16>(ctx, n_tokens, head_dim, n_q_heads, Q, ldq, w_q, n_k_heads, K, ldk, w_k, eps, rot, positions, Q_out, ldq_out, K_out, ldk_out);
}

extern "C" int tboa_kv_cache_append(tboa_ctx* ctx, const tboa_kv_cache_desc* desc, const tboa_kv_batch* batch, int dtype, const void* K, int64_t ldk, const void* V, int64_t ldv,
                                    const tboa_rotation* rotation, const int* positions, void* cache) {
    if (!ctx) return TBOA_EINVAL;
    KvGeometry g;
    TB_TRY(kv_check(ctx, "kv_cache_append", desc, batch, cache, g));
    if (dtype != TBOA_F32 && dtype != TBOA_BF16) return tboa_fail(ctx, TBOA_EINVAL, "kv_cache_append: dtype must be fp32 or bf16");
    Rotation rot;
    TB_TRY(check_rotation(ctx, "kv_cache_append", rotation, g.dh, rot));
    if (batch->n_seqs == 0 || batch->n_tokens == 0 || batch->pages_per_seq == 0 || g.n_pages == 0) return 0;
    if (!K || !V) return tboa_fail(ctx, TBOA_EINVAL, "kv_cache_append: null argument");
    if (ldk < (int64_t)g.heads * g.dh || ldv < (int64_t)g.heads * g.dh) return tboa_fail(ctx, TBOA_EINVAL, "kv_cache_append: a row pitch is smaller than its heads");
    const KvBatch q{batch->n_seqs, batch->pages_per_seq, (int)batch->n_tokens, batch->pages_per_seq * desc->page_tokens, batch->starts, batch->lens, batch->pages};
    KvDevice dev(ctx->device);
    if (dtype == TBOA_F32) return append<float>(ctx, AppendArgs<float>{g, q, {(const float*)K, (const float*)V}, {ldk, ldv}, rot, positions, (unsigned char*)cache, 0, 0, {}, false});
    return append<bf16>(ctx, AppendArgs<bf16>{g, q, {(const bf16*)K, (const bf16*)V}, {ldk, ldv}, rot, positions, (unsigned char*)cache, 0, 0, {}, false});
}
