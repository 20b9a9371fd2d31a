// Attention over a quantized key/value cache.
//
// One pass over the cache with the running maximum and sum of the softmax.  Levels minus their zero are whole numbers up to 255 and so exact in half; they are made in registers from the
// cache's bytes (a byte beside 0x64 is 1024 + level as half; one packed addition takes 1024 + zero away), and the scales multiply scores and probabilities:
//     x[t] = (scale s^K_t log2 e) q.(c^K_t - z^K_t),   p = 2^(x - max),   O += (p s^V_t 2^14 / ref) (c^V_t - z^V_t),   ref: a power of two above the scales seen so far
// Queries become half times a power of two that brings the largest of a tile to 2^13 .. 2^14 (bf16 queries stay exact down to 2^-31 of it); p s 2^14 / ref is rounded to half:
// 2^-11 of it at most, an eighth of an output's rounding to bf16.  fp32 queries and probabilities are split into two half terms (2^-22 of them at most).
#include "kv_cache.h"
#include <math.h>
#include <algorithm>

namespace {

typedef __hip_bfloat16 bf16;
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef unsigned u4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(bf16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16 from_f32<bf16>(float v) { return __float2bfloat16(v); }
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

struct AttendArgs {
    KvGeometry g; KvBatch q;
    const void* Q; long long ldq; void* O; long long ldo;
    const unsigned char* cache;
    float scale2;                 // scale log2 e
    int rep, window, target;      // target: items that fill the chip
    long long items;              // room in part and stat
    float* part; float2* stat;    // per item, head and row: unscaled outputs; maximum, sum
};

constexpr float HALF_TOP = 0x1p14f;      // what a probability of 1 with the largest scale becomes as half, at most: parts of 2^-28 of it are still normal numbers
constexpr int ROWS = 16, TILE = 64;      // rows (query token, head of the group) of an item, tokens a wavefront takes at a time

// how a sequence is cut: row tiles, tokens that its rows see
__device__ __forceinline__ int row_tiles(const KvSeq& s, int rep) { return (int)(((long long)s.n * rep + ROWS - 1) / ROWS); }
__device__ __forceinline__ int seen_tiles(const KvSeq& s, const AttendArgs& a) {
    const int end = min(s.len, a.q.room);
    return s.n == 0 ? 0 : (min(end, a.window ? (int)min((long long)a.window + s.n + TILE, 2147483647LL) : end) + TILE - 1) / TILE;
}
// tiles of TILE tokens that an item takes at least, so that all items are about `target`; a multiple of the four wavefronts
__device__ __forceinline__ int item_tiles(const AttendArgs& a) {
    const int lane = threadIdx.x & 63;
    long long total = 0;
    for (int b = lane; b < a.q.n_seqs; b += 64) {
        const KvSeq s = kv_sequence(a.q, b);
        total += (long long)row_tiles(s, a.rep) * seen_tiles(s, a);
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) total += __shfl_xor(total, o, 64);
    const long long c = (total * a.g.heads + a.target - 1) / a.target;
    return (int)min(max((c + 3) / 4 * 4, 4LL), 1LL << 26);
}
__device__ __forceinline__ int cuts(const KvSeq& s, const AttendArgs& a, int per) { return max((seen_tiles(s, a) + per - 1) / per, 1); }

// tokens that rows r0 .. of a sequence see
struct Span { int lo, hi; };
__device__ __forceinline__ Span row_span(const KvSeq& s, const AttendArgs& a, int r0, int rows) {
    const int p0 = s.len - s.n + r0 / a.rep, p1 = s.len - s.n + (r0 + rows - 1) / a.rep;
    return Span{a.window ? max(p0 - a.window + 1, 0) : 0, max(min(p1 + 1, a.q.room), 0)};
}

// One workgroup per item (16 rows of a sequence's query tokens and the heads of a KV group, a piece of the tokens they see) and KV head; its four wavefronts take every fourth tile of 64
// tokens and are joined through LDS at the end.  S^T = K Q^T with tile i's row 4 g + j of the matrix instruction being token 16 g + 4 i + j: lane group g then holds the probabilities of
// tokens 16 g .. 16 g + 15 for row lane % 16, which are the right operand of O^T += V^T P^T as they stand.
template <typename T, int DP>
__global__ __launch_bounds__(256) void kv_attend_rows_kernel(AttendArgs a) {
    constexpr int NT = sizeof(T) == 2 ? 1 : 2;      // half terms of queries and probabilities
    constexpr int K64 = DP / 64, K32 = (DP % 64) / 32, KS = DP / 32, CT = DP / 16;
    __shared__ float joined[4][ROWS][DP + 4];
    __shared__ float2 ends[4][ROWS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, grp = lane >> 4, h = blockIdx.y;
    const int per = item_tiles(a);
    int x = blockIdx.x, b;
    KvSeq s;
    if (!kv_find(a.q, [&](const KvSeq& e) { return e.n ? (int)min((long long)row_tiles(e, a.rep) * cuts(e, a, per), 1LL << 30) : 0; }, x, b, s)) return;
    const int n_cuts = cuts(s, a, per), r0 = x / n_cuts * ROWS, cut = x % n_cuts, n_rows = (int)min((long long)ROWS, (long long)s.n * a.rep - r0);
    const Span span = row_span(s, a, r0, n_rows);
    int lo, hi;
    {
        const int t0 = span.lo / TILE, t1 = (span.hi + TILE - 1) / TILE, each = max((t1 - t0 + n_cuts - 1) / n_cuts, 0);
        lo = (t0 + cut * each) * TILE; hi = min((t0 + (cut + 1) * each) * TILE, span.hi);
    }
    // this lane's row
    const bool row_live = col < n_rows;
    const int r = r0 + (row_live ? col : 0), pos = row_live ? s.len - s.n + r / a.rep : -1, low = a.window ? pos - a.window + 1 : 0;
    h8 qh[NT][KS];
    float unit;
    {
        const T* q = (const T*)a.Q + (long long)(s.start + r / a.rep) * a.ldq + (long long)(h * a.rep + r % a.rep) * a.g.dh;
        float v[KS][8], most = 0.f;
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int c = k < 2 * K64 ? (k >> 1) * 64 + grp * 16 + (k & 1) * 8 + j : K64 * 64 + grp * 8 + j;
                v[k][j] = row_live && c < a.g.dh ? to_f32(q[c]) : 0.f;
                const float m = fabsf(v[k][j]);
                most = m < __builtin_inff() ? fmaxf(most, m) : most;
            }
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) most = fmaxf(most, __shfl_xor(most, o, 64));
        int e = 0;
        if (most > 0.f) { frexpf(most, &e); e = min(14 - e, 100); }
        unit = ldexpf(a.scale2, -e);
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float w = ldexpf(v[k][j], e);
                const _Float16 hi16 = (_Float16)w;
                qh[0][k][j] = hi16;
                if constexpr (NT == 2) qh[1][k][j] = (_Float16)(isfinite(w) ? w - (float)hi16 : 0.f);
            }
    }

    float m = -__builtin_inff(), l = 0.f, ref = 0x1p-126f;
    f4 o[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) o[c] = f4{0.f, 0.f, 0.f, 0.f};

    const int end = min(s.len, a.q.room);
    const long long head_levels = (long long)h * DP << a.g.pt_log, head_grids = (long long)h << (a.g.pt_log - a.g.st_log);
    const int in_page = (1 << a.g.pt_log) - 1;
    const int* const pages = a.q.pages + (long long)b * a.q.per_seq;
    for (int t0 = lo + wave * TILE; t0 < hi; t0 += 4 * TILE) {
        const int tk = t0 + 16 * (col >> 2), tv = t0 + 16 * grp;      // 16 tokens that this lane takes levels of K, of V from
        const int pk = pages[min(tk >> a.g.pt_log, a.q.per_seq - 1)], pv = pages[min(tv >> a.g.pt_log, a.q.per_seq - 1)];
        const bool held = pv >= 0 && pv < a.g.n_pages;
        const unsigned char* const kp = a.cache + (long long)min(max(pk, 0), (int)a.g.n_pages - 1) * a.g.page_bytes;
        const unsigned char* const vp = a.cache + (long long)(held ? pv : 0) * a.g.page_bytes;
        const unsigned char* const kb = kp + head_levels + (long long)((tk & in_page) + (col & 3)) * DP + grp * 16;
        const unsigned char* const vb = vp + a.g.v_at + head_levels + (long long)(tv & in_page) * DP + col * 16;
        u4 kr[4][K64 + (K64 == 0)]; uint2 ks[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int k = 0; k < K64; ++k) kr[i][k] = *(const u4*)(kb + i * 4 * DP + k * 64);
            if constexpr (K32 != 0) ks[i] = *(const uint2*)(kb + i * 4 * DP + K64 * 64 - grp * 8);
        }
        u4 vr[CT];
#pragma unroll
        for (int c = 0; c < CT; ++c) vr[c] = *(const u4*)(vb + c * 256);
        // grids of token t0 + lane
        const int t = t0 + lane;
        const bool there = held && t < end;
        float2 gk = make_float2(1.f, 0.f), gv = make_float2(0.f, 0.f);
        if (there) {
            const long long at = head_grids + ((t & in_page) >> a.g.st_log);
            gk = ((const float2*)(vp + a.g.kg_at))[at]; gv = ((const float2*)(vp + a.g.vg_at))[at];
        }
        const float sk = gk.x * unit;

        // scores
        f4 st[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const _Float16 zo = (_Float16)(-1024.f - __shfl(gk.y, 16 * (col >> 2) + 4 * i + (col & 3), 64));
            const h2 z = {zo, zo};
            f4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                h8 lv;
                if (k < 2 * K64) lv = levels8(kr[i][k >> 1][(k & 1) * 2], kr[i][k >> 1][(k & 1) * 2 + 1], z, z, z, z);
                else lv = levels8(ks[i].x, ks[i].y, z, z, z, z);
#pragma unroll
                for (int n = 0; n < NT; ++n) acc = mma16(lv, qh[n][k], acc);
            }
            st[i] = acc;
        }
        float p[16];
        unroll<16>([&](auto I) { constexpr int i = I; p[i] = st[i >> 2][i & 3] * row_lane<i>(sk); });
        const bool all = t0 + TILE - 1 <= s.len - s.n + r0 / a.rep && t0 + TILE <= end && t0 >= (a.window ? span.lo + (n_rows - 1) / a.rep + 1 : 0) && __all(held);
        unsigned hidden = 0;
        if (!all) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int tt = tv + i;
                if (!(row_live && held && tt < end && tt <= pos && tt >= low)) { hidden |= 1u << i; p[i] = -__builtin_inff(); }
            }
        }
        float top = p[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, p[i]);
        top = fmaxf(top, from_xor<16>(top)); top = fmaxf(top, from_xor<32>(top));
        const float m_new = fmaxf(m, top), base = m_new == -__builtin_inff() ? 0.f : m_new;
        float turn = ex2(m - base);
        m = m_new;
        l *= turn;
#pragma unroll
        for (int i = 0; i < 16; ++i) { p[i] = ex2(p[i] - base); l += p[i]; }
        float s_top = gv.x;
#pragma unroll
        for (int q = 1; q < 64; q <<= 1) s_top = fmaxf(s_top, __shfl_xor(s_top, q, 64));
        if (s_top >= ref && s_top < __builtin_inff()) {
            int e;
            frexpf(s_top, &e);
            const float now = ldexpf(1.f, min(e, 127));
            turn *= ref / now; ref = now;
        }
        if (__any(turn != 1.f)) {
#pragma unroll
            for (int c = 0; c < CT; ++c) o[c] *= turn;
        }
        const float sv = gv.x * (HALF_TOP / ref);
        unroll<16>([&](auto I) { constexpr int i = I; p[i] *= row_lane<i>(sv); });
        if (!all) {
#pragma unroll
            for (int i = 0; i < 16; ++i) if (hidden >> i & 1) p[i] = 0.f;
        }
        h8 ph[NT][2];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const _Float16 w = (_Float16)p[8 * k + j];
                ph[0][k][j] = w;
                if constexpr (NT == 2) ph[1][k][j] = (_Float16)(p[8 * k + j] - (float)w);
            }
        // zeros of V's 16 tokens as pairs
        h2 zo[8];
        {
            const unsigned mine = __builtin_bit_cast(unsigned short, (_Float16)(-1024.f - gv.y));
            const unsigned next = (unsigned)__builtin_amdgcn_mov_dpp((int)mine, 0xB1, 0xf, 0xf, true);      // the neighbour's: quad_perm 1 0 3 2
            const unsigned pair = mine | next << 16;                                                             // (for even lanes)
            unroll<8>([&](auto I) { constexpr int i = I; zo[i] = __builtin_bit_cast(h2, row_lane<2 * i>(pair)); });
        }
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            const h8 v0 = levels8(vr[c][0], vr[c][1], zo[0], zo[1], zo[2], zo[3]), v1 = levels8(vr[c][2], vr[c][3], zo[4], zo[5], zo[6], zo[7]);
#pragma unroll
            for (int n = 0; n < NT; ++n) { o[c] = mma16(v0, ph[n][0], o[c]); o[c] = mma16(v1, ph[n][1], o[c]); }
        }
    }
    l += from_xor<16>(l); l += from_xor<32>(l);
    if (l != l) m = fmaxf(m, 0.f);      // scores that are all NaN leave the maximum where it was: the row has seen something
    if (grp == 0) ends[wave][col] = make_float2(m, l);
    __syncthreads();
    float top = ends[0][col].x;
#pragma unroll
    for (int w = 1; w < 4; ++w) top = fmaxf(top, ends[w][col].x);
    const float f = m == -__builtin_inff() ? 0.f : ex2(m - top) * ref * (1.f / HALF_TOP);
#pragma unroll
    for (int c = 0; c < CT; ++c) *(f4*)&joined[wave][col][c * 16 + grp * 4] = m == -__builtin_inff() ? f4{0.f, 0.f, 0.f, 0.f} : o[c] * f;
    __syncthreads();
    for (int i = threadIdx.x; i < n_rows * a.g.dh; i += 256) {
        const int rr = i / a.g.dh, c = i - rr * a.g.dh;
        float tp = ends[0][rr].x, sum = 0.f, v = 0.f;
#pragma unroll
        for (int w = 1; w < 4; ++w) tp = fmaxf(tp, ends[w][rr].x);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if (ends[w][rr].x != -__builtin_inff()) sum += ends[w][rr].y * ex2(ends[w][rr].x - tp);
            v += joined[w][rr][c];
        }
        if (n_cuts == 1) {
            const int row = r0 + rr;
            T* out = (T*)a.O + (long long)(s.start + row / a.rep) * a.ldo + (long long)(h * a.rep + row % a.rep) * a.g.dh;
            out[c] = from_f32<T>(sum == 0.f ? 0.f : v / sum);
        } else {
            const long long at = ((long long)blockIdx.x * a.g.heads + h) * ROWS + rr;
            a.part[at * DP + c] = v;
            if (c == 0) a.stat[at] = make_float2(tp, sum);
        }
    }
}

// Items of a row tile of a sequence that was cut: sum of 2^(max_i - max) O_i over that of the sums.  One workgroup per row tile, KV head and row.
template <typename T>
__global__ __launch_bounds__(256) void kv_attend_join_kernel(AttendArgs a) {
    const int h = blockIdx.y, rr = blockIdx.z, per = item_tiles(a);
    int x = blockIdx.x, b;
    KvSeq s;
    if (!kv_find(a.q, [&](const KvSeq& e) { return row_tiles(e, a.rep); }, x, b, s)) return;
    const int n_cuts = cuts(s, a, per);
    if (n_cuts == 1 || x * ROWS + rr >= s.n * a.rep) return;
    // number of the tile's first item: items of the sequences before, and of the tiles before
    long long before = 0;
    for (int i = threadIdx.x & 63; i < b; i += 64) { const KvSeq e = kv_sequence(a.q, i); if (e.n) before += (long long)row_tiles(e, a.rep) * cuts(e, a, per); }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) before += __shfl_xor(before, o, 64);
    const long long first = before + (long long)x * n_cuts;
    if (first + n_cuts > a.items) return;      // (starts that do not grow)
    __shared__ float sums[256], outs[256];
    float top = -__builtin_inff();
    for (int i = 0; i < n_cuts; ++i) top = fmaxf(top, a.stat[((first + i) * a.g.heads + h) * ROWS + rr].x);
    const int row = x * ROWS + rr;
    T* out = (T*)a.O + (long long)(s.start + row / a.rep) * a.ldo + (long long)(h * a.rep + row % a.rep) * a.g.dh;
    // 64 channels at a time, four shares of the items
    const int c0 = threadIdx.x & 63, share = threadIdx.x >> 6;
    for (int c = c0; c < a.g.dp; c += 64) {
        float v = 0.f, sum = 0.f;
        for (int i = share; i < n_cuts; i += 4) {
            const long long at = ((first + i) * a.g.heads + h) * ROWS + rr;
            const float2 st = a.stat[at];
            if (st.x == -__builtin_inff()) continue;
            const float f = ex2(st.x - top);
            sum += f * st.y;
            if (c < a.g.dh) v += f * a.part[at * a.g.dp + c];
        }
        sums[threadIdx.x] = sum; outs[threadIdx.x] = v;
        __syncthreads();
        if (share == 0 && c < a.g.dh) {
            sum = sums[c0] + sums[c0 + 64] + sums[c0 + 128] + sums[c0 + 192];
            v = outs[c0] + outs[c0 + 64] + outs[c0 + 128] + outs[c0 + 192];
            out[c] = from_f32<T>(sum == 0.f ? 0.f : v / sum);
        }
        __syncthreads();
    }
}

// Items that fill the chip: four workgroups of 256 compute units each
constexpr int TARGET = 1024;
struct AttendPlan { long long tiles, items; size_t bytes; };
AttendPlan plan(const KvGeometry& g, int n_seqs, long long n_tokens, int rep) {
    AttendPlan p;
    // row tiles of all sequences: at most rows / ROWS and one more per sequence, and no sequence with a token has more than ceil(rep / ROWS) per token
    p.tiles = std::min(n_tokens * rep / ROWS + std::min<long long>(n_seqs, n_tokens), n_tokens * cdiv64(rep, ROWS));
    p.items = p.tiles + cdiv64(TARGET, g.heads);
    Arena ar(nullptr);
    ar.get<float>((size_t)p.items * g.heads * ROWS * g.dp); ar.get<float2>((size_t)p.items * g.heads * ROWS);
    p.bytes = ar.off;
    return p;
}

template <typename T>
int attend(tboa_ctx* ctx, const AttendArgs& a, const AttendPlan& p) {
    const dim3 grid((unsigned)p.items, (unsigned)a.g.heads), block(256);
    switch (a.g.dp) {
        case 32: hipLaunchKernelGGL((kv_attend_rows_kernel<T, 32>), grid, block, 0, ctx->stream, a); break;
        case 64: hipLaunchKernelGGL((kv_attend_rows_kernel<T, 64>), grid, block, 0, ctx->stream, a); break;
        case 96: hipLaunchKernelGGL((kv_attend_rows_kernel<T, 96>), grid, block, 0, ctx->stream, a); break;
        case 128: hipLaunchKernelGGL((kv_attend_rows_kernel<T, 128>), grid, block, 0, ctx->stream, a); break;
        case 192: hipLaunchKernelGGL((kv_attend_rows_kernel<T, 192>), grid, block, 0, ctx->stream, a); break;
        default: hipLaunchKernelGGL((kv_attend_rows_kernel<T, 256>), grid, block, 0, ctx->stream, a);
    }
    TB_KERNEL_CHECK(ctx);
    hipLaunchKernelGGL((kv_attend_join_kernel<T>), dim3((unsigned)p.tiles, (unsigned)a.g.heads, ROWS), block, 0, ctx->stream, a);
    TB_KERNEL_CHECK(ctx);
    return 0;
}

}  // namespace

extern "C" size_t tboa_kv_cache_attention_workspace_bytes(const tboa_kv_cache_desc* desc, int n_q_heads, int n_seqs, int64_t n_tokens) {
    KvGeometry g;
    if (!kv_geometry(desc, g) || n_q_heads <= 0 || n_q_heads > 65535 || n_q_heads % g.heads || n_seqs < 0 || n_seqs > 1 << 20 || n_tokens < 0 || n_tokens > 1 << 24) return 0;
    return n_seqs == 0 || n_tokens == 0 ? 0 : plan(g, n_seqs, n_tokens, n_q_heads / g.heads).bytes;
}

extern "C" int tboa_kv_cache_attention(tboa_ctx* ctx, const tboa_kv_cache_desc* desc, const tboa_kv_batch* batch, int n_q_heads, int dtype, const void* Q, int64_t ldq,
                                       const void* cache, double scale, int window, void* O, int64_t ldo) {
    if (!ctx) return TBOA_EINVAL;
    KvGeometry g;
    TB_TRY(kv_check(ctx, "kv_cache_attention", desc, batch, cache, g));
    if (dtype != TBOA_F32 && dtype != TBOA_BF16) return tboa_fail(ctx, TBOA_EINVAL, "kv_cache_attention: dtype must be fp32 or bf16");
    if (n_q_heads <= 0 || n_q_heads > 65535 || n_q_heads % g.heads) return tboa_fail(ctx, TBOA_EINVAL, "kv_cache_attention: %d query heads for %d KV heads", n_q_heads, g.heads);
    if (!(scale >= 0.0 && scale <= 1e30) || window < 0) return tboa_fail(ctx, TBOA_EINVAL, "kv_cache_attention: scale=%g window=%d", scale, window);
    if (batch->n_seqs == 0 || batch->n_tokens == 0) return 0;
    if (batch->pages_per_seq == 0 || g.n_pages == 0) return tboa_fail(ctx, TBOA_EINVAL, "kv_cache_attention: no pages");
    if (!Q || !O) return tboa_fail(ctx, TBOA_EINVAL, "kv_cache_attention: null argument");
    if (ldq < (int64_t)n_q_heads * g.dh || ldo < (int64_t)n_q_heads * g.dh) return tboa_fail(ctx, TBOA_EINVAL, "kv_cache_attention: a row pitch is smaller than its heads");
    KvDevice dev(ctx->device);
    const int rep = n_q_heads / g.heads;
    const AttendPlan p = plan(g, batch->n_seqs, batch->n_tokens, rep);
    if (batch->n_tokens * rep > 1LL << 30) return tboa_fail(ctx, TBOA_EINVAL, "kv_cache_attention: too many rows");
    TB_TRY(tboa_ws_reserve(ctx, p.bytes));
    TB_TRY(tboa_ws_in_graph(ctx));
    AttendArgs a;
    a.g = g;
    a.q = KvBatch{batch->n_seqs, batch->pages_per_seq, (int)batch->n_tokens, batch->pages_per_seq * desc->page_tokens, batch->starts, batch->lens, batch->pages};
    a.Q = Q; a.ldq = ldq; a.O = O; a.ldo = ldo; a.cache = (const unsigned char*)cache;
    a.scale2 = (float)((scale == 0.0 ? 1.0 / sqrt((double)g.dh) : scale) * 1.4426950408889634);
    a.rep = rep; a.window = window; a.target = TARGET; a.items = p.items;
    Arena ar(ctx->ws);
    a.part = ar.get<float>((size_t)p.items * g.heads * ROWS * g.dp);
    a.stat = ar.get<float2>((size_t)p.items * g.heads * ROWS);
    return dtype == TBOA_F32 ? attend<float>(ctx, a, p) : attend<bf16>(ctx, a, p);
}
