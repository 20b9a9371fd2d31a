// Norms and rotation of head vectors, and the append to a quantized key/value cache.
#include "kv_cache.h"
#include <math.h>
#include <algorithm>

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
template <typename T> struct RotateArgs { RotateSide<T> side[2]; long long tokens; int dh; float eps; Rotation rot; const int* positions; };

// 1 / sqrt(mean of squares + eps), the sum in fp64: squares of 3e38 are within its range
__device__ __forceinline__ float norm_factor(double sum, int dh, float eps) { return (float)(1.0 / sqrt(sum / (double)dh + (double)eps)); }

// One lane per 16 channels, both halves of their pairs (channels 8 s .. and rot/2 + 8 s .., or 16 s .. where pairs are adjacent), `lpr` lanes per head vector.
template <typename T>
__global__ __launch_bounds__(256) void head_norm_rotate_kernel(RotateArgs<T> a, int lpr) {
    const int heads = a.side[0].heads + a.side[1].heads;
    const long long row = ((long long)blockIdx.x * 256 + threadIdx.x) / lpr;
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
        const float r = norm_factor(sum, a.dh, a.eps);
        if (mine) {
#pragma unroll
            for (int i = 0; i < 8; ++i) { u[i] = u[i] * r * d.w[c0 + i]; v[i] = v[i] * r * d.w[c1 + i]; }
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

// Any sizes and alignment: one wavefront per head vector, a lane per channel; everything is read before anything is written (in place)
template <typename T>
__global__ __launch_bounds__(256) void head_norm_rotate_any_kernel(RotateArgs<T> a) {
    const int heads = a.side[0].heads + a.side[1].heads, lane = threadIdx.x & 63;
    const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
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
        const float r = norm_factor(sum, a.dh, a.eps);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = lane + 64 * i;
            if (c < a.dh) {
                v[i] = v[i] * r * d.w[c];
                if (c < a.rot.dim) { int pair; bool second; o[i] = o[i] * r * d.w[partner(c, a.rot, pair, second)]; }
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
    unsigned char* cache; int unit_log;
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
__device__ __forceinline__ unsigned char level_of(double v, double s, double inv, double z) {
    const double t = v * inv;
    double r = rint(t);
    if (!(fabs(t - r) < 0.5 - 1e-6)) r = rint(v / s);      // next to a border the quotient itself decides (|t| below 2^10: the product is off by 2^-42 at most)
    return (unsigned char)fmin(fmax(r + z, 0.0), 255.0);
}

// One workgroup per unit of max(16, scale_tokens) tokens of a sequence, head, and K or V.  A tile of 16 tokens goes through LDS; 16 lanes per token hold its channels, rotated in fp64
// (products of 24 bits are exact there), find the ends, and after the block's grid stands turn them into levels.
template <typename T, int NC>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendArgs<T> a) {
    constexpr int DP = 16 * NC;
    __shared__ float xs[16][DP + 4];
    __shared__ __align__(16) unsigned char lev[16 * DP];
    __shared__ double tlo[16], thi[16];
    __shared__ int tbad[16];
    const int h = blockIdx.y, kv = blockIdx.z, ul = a.unit_log;
    int x = blockIdx.x, b;
    KvSeq s;
    const int room = a.q.room;
    if (!kv_find(a.q, kv_head(a.q), [ul, room](const KvSeq& e) {
            const int p0 = max(e.len - e.n, 0), end = min(e.len, room);
            return end > p0 && e.n > 0 ? ((end - 1) >> ul) - (p0 >> ul) + 1 : 0; }, x, b, s)) return;
    const int first = max(s.len - s.n, 0);                 // first position that gets a token
    const int p_unit = ((first >> ul) + x) << ul;
    const long long page = a.q.pages[(long long)b * a.q.per_seq + (p_unit >> a.g.pt_log)];
    if (page < 0 || page >= a.g.n_pages) return;
    const int row0 = s.start + s.n - s.len;                // row of position p: row0 + p
    unsigned char* const pg = a.cache + page * a.g.page_bytes;
    const int pt = 1 << a.g.pt_log, o_unit = p_unit & (pt - 1), st_log = a.g.st_log, st = 1 << st_log, dh = a.g.dh;
    float2* const grids = (float2*)(pg + (kv ? a.g.vg_at : a.g.kg_at)) + ((long long)h << (a.g.pt_log - st_log));
    const T* const X = a.x[kv] + (long long)h * dh;
    const long long ld = a.ld[kv];
    const int tok = threadIdx.x >> 4, sub = threadIdx.x & 15;
    const int tiles = 1 << (ul - 4), unit_end = min(p_unit + (1 << ul), min(s.len, room));
    const int rot = kv ? 0 : a.rot.dim;

    double v[NC];
    auto fetch = [&](int j) {      // values of tile j's tokens, channels sub + 16 i
        const int p0 = p_unit + 16 * j;
        __syncthreads();
        for (int i = threadIdx.x; i < 16 * dh; i += 256) {
            const int r = i / dh, c = i - r * dh, p = p0 + r;
            xs[r][c] = p >= first && p < unit_end ? to_f32(X[(row0 + p) * ld + c]) : 0.f;
        }
        __syncthreads();
        const int p = p0 + tok;
        const bool is_new = p >= first && p < unit_end;
        long long at = 0;
        bool known = true;
        if (rot && is_new) {
            at = a.positions ? a.positions[row0 + p] : p;
            known = at >= 0 && at < a.rot.positions;
        }
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int c = sub + 16 * i;
            v[i] = 0.0;
            if (c < dh && is_new) {
                v[i] = (double)xs[tok][c];
                if (c < rot) {
                    int pair; bool second;
                    const double w = (double)xs[tok][partner(c, a.rot, pair, second)];
                    const double cs = known ? (double)a.rot.table[at * rot + pair] : __builtin_nan(""), sn = known ? (double)a.rot.table[at * rot + rot / 2 + pair] : __builtin_nan("");
                    v[i] = second ? v[i] * cs + w * sn : v[i] * cs - w * sn;
                }
            }
        }
    };

    double lo = 0.0, hi = 0.0;
    int bad = 0;
    const int span = min(st, 16), t_first = tok & ~(span - 1);
    for (int j = 0; j < tiles; ++j) {
        if (p_unit + 16 * j >= unit_end || p_unit + 16 * j + 16 <= first) continue;
        fetch(j);
        double l = 0.0, u = 0.0;
        bool inf = false;
#pragma unroll
        for (int i = 0; i < NC; ++i) { l = fmin(l, v[i]); u = fmax(u, v[i]); inf |= !isfinite(v[i]); }
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) { l = fmin(l, __shfl_xor(l, o, 64)); u = fmax(u, __shfl_xor(u, o, 64)); inf |= __shfl_xor((int)inf, o, 64) != 0; }
        if (sub == 0) { tlo[tok] = l; thi[tok] = u; tbad[tok] = inf; }
        __syncthreads();
        for (int i = 0; i < span; ++i) { lo = fmin(lo, tlo[t_first + i]); hi = fmax(hi, thi[t_first + i]); bad |= tbad[t_first + i]; }
    }
    // this thread's block: the unit (st >= 16), or its token's within the only tile
    const int block = (o_unit >> st_log) + (st < 16 ? tok >> st_log : 0);
    const int p_block = p_unit + (st < 16 ? t_first : 0);
    const bool touched = p_block < unit_end && p_block + st > first;
    const bool had = touched && p_block < first;
    float2 old = make_float2(0.f, 0.f);
    if (had) old = grids[block];
    const Grid gr = block_grid(lo, hi, bad != 0, had, old.x, old.y);
    const double inv = 1.0 / gr.s;
    __syncthreads();      // every stored grid has been read
    if (touched && sub == 0 && (st < 16 ? (tok & (st - 1)) == 0 : tok == 0)) grids[block] = make_float2((float)gr.s, (float)gr.z);

    unsigned char* const levels = pg + (kv ? a.g.v_at : 0) + (long long)h * pt * DP + (long long)o_unit * DP;
    for (int j = 0; j < tiles; ++j) {
        const int p0 = p_unit + 16 * j;
        if (p0 >= unit_end) break;
        if (p0 + 16 <= first && !gr.grown) continue;      // (tiles > 1: one block, the same for all threads)
        if (tiles > 1) fetch(j);
        const int p = p0 + tok;
        unsigned char* const tile = levels + (long long)j * 16 * DP;
        const bool fresh = p >= first && p < unit_end, moved = p < first && gr.grown;      // a grown block: p lies in it, since it has earlier tokens
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int c = sub + 16 * i;
            unsigned char q = 0;
            if (fresh) q = level_of(v[i], gr.s, inv, gr.z);
            else if (moved && c < dh) {
                const double w = ((double)tile[kv ? c * 16 + tok : tok * DP + c] - gr.z0) * gr.s0;
                q = (unsigned char)fmin(fmax(rint(w / gr.s) + gr.z, 0.0), 255.0);
            }
            lev[kv ? c * 16 + tok : tok * DP + c] = q;
        }
        // K rows, V bytes of the tokens that have a new level
        const bool put = fresh || moved;
        if (sub == 0) tbad[tok] = put;
        __syncthreads();
        if (kv) {
            int all = 1;
            for (int i = 0; i < 16; ++i) all &= tbad[i];
            if (all) {
                for (int c = threadIdx.x; c < dh; c += 256) *(uint4*)(tile + c * 16) = *(const uint4*)(lev + c * 16);
            } else {
                for (int c = threadIdx.x; c < 16 * dh; c += 256) if (tbad[c & 15]) tile[c] = lev[c];
            }
        } else {
            const int whole = dh & ~15;
            for (int c = 16 * threadIdx.x; c < 16 * DP; c += 16 * 256) if (c % DP < whole && tbad[c / DP]) *(uint4*)(tile + c) = *(const uint4*)(lev + c);
            if (whole < dh)
                for (int i = threadIdx.x; i < 16 * (dh - whole); i += 256) {
                    const int r = i / (dh - whole), c = whole + i % (dh - whole);
                    if (tbad[r]) tile[r * DP + c] = lev[r * DP + c];
                }
        }
        __syncthreads();
    }
}

template <typename T>
int head_norm_rotate(tboa_ctx* ctx, long long n_tokens, int dh, int nq, const void* Q, long long ldq, const float* wq, int nk, const void* K, long long ldk, const float* wk, double eps,
                     const Rotation& rot, const int* positions, void* Qo, long long ldqo, void* Ko, long long ldko) {
    RotateArgs<T> a{{{(const T*)Q, (T*)Qo, wq, ldq, ldqo, nq}, {(const T*)K, (T*)Ko, wk, ldk, ldko, nk}}, n_tokens, dh, (float)eps, rot, positions};
    const long long rows = n_tokens * (nq + nk);
    // 16-byte pieces where every head vector and table row starts on a 16-byte boundary and the pairs of 16 channels are whole pieces
    const int e = 16 / (int)sizeof(T);
    bool vec = dh % 16 == 0 && rot.dim % 16 == 0 && ((uintptr_t)rot.table & 15) == 0;
    for (const auto& d : a.side) vec &= !d.heads || ((((uintptr_t)d.x | (uintptr_t)d.y) & 15) == 0 && d.ldx % e == 0 && d.ldy % e == 0);
    int lpr = 1;
    while (16 * lpr < dh) lpr *= 2;
    const long long blocks = vec ? cdiv64(rows, 256 / lpr) : cdiv64(rows, 4);
    if (blocks > 2147483647LL) return tboa_fail(ctx, TBOA_EINVAL, "head_norm_rotate: too many head vectors");
    if (vec) hipLaunchKernelGGL((head_norm_rotate_kernel<T>), dim3((unsigned)blocks), dim3(256), 0, ctx->stream, a, lpr);
    else hipLaunchKernelGGL((head_norm_rotate_any_kernel<T>), dim3((unsigned)blocks), dim3(256), 0, ctx->stream, a);
    TB_KERNEL_CHECK(ctx);
    return 0;
}

template <typename T>
int append(tboa_ctx* ctx, const AppendArgs<T>& a, long long units) {
    const dim3 grid((unsigned)units, (unsigned)a.g.heads, 2), block(256);
    switch (a.g.dp) {
        case 32: hipLaunchKernelGGL((kv_append_kernel<T, 2>), grid, block, 0, ctx->stream, a); break;
        case 64: hipLaunchKernelGGL((kv_append_kernel<T, 4>), grid, block, 0, ctx->stream, a); break;
        case 96: hipLaunchKernelGGL((kv_append_kernel<T, 6>), grid, block, 0, ctx->stream, a); break;
        case 128: hipLaunchKernelGGL((kv_append_kernel<T, 8>), grid, block, 0, ctx->stream, a); break;
        case 192: hipLaunchKernelGGL((kv_append_kernel<T, 12>), grid, block, 0, ctx->stream, a); break;
        default: hipLaunchKernelGGL((kv_append_kernel<T, 16>), grid, block, 0, ctx->stream, a);
    }
    TB_KERNEL_CHECK(ctx);
    return 0;
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
    const int unit_log = std::max(4, g.st_log);
    const long long units = std::min<long long>(batch->n_tokens, (batch->n_tokens >> unit_log) + 2LL * batch->n_seqs);
    const KvBatch q{batch->n_seqs, batch->pages_per_seq, (int)batch->n_tokens, batch->pages_per_seq * desc->page_tokens, batch->starts, batch->lens, batch->pages};
    KvDevice dev(ctx->device);
    if (dtype == TBOA_F32) return append<float>(ctx, AppendArgs<float>{g, q, {(const float*)K, (const float*)V}, {ldk, ldv}, rot, positions, (unsigned char*)cache, unit_log}, units);
    return append<bf16>(ctx, AppendArgs<bf16>{g, q, {(const bf16*)K, (const bf16*)V}, {ldk, ldv}, rot, positions, (unsigned char*)cache, unit_log}, units);
}
