// Attention over a quantized key/value cache.
//
// One pass over the cache with the running maximum and sum of the softmax.  Levels minus their zero are whole numbers up to 255 and so exact in half; they are made in registers from the
// cache's bytes (a byte beside 0x64 is 1024 + level as half; one packed addition takes 1024 + zero away), and the scales multiply scores and probabilities:
//     x[t] = (scale s^K_t log2 e) q.(c^K_t - z^K_t),   p = 2^(x - max),   O += (2^up p s^V_t) (c^V_t - z^V_t)
// A row's query becomes half times a power of two that brings its largest channel to 2^13 .. 2^14 (bf16 queries stay exact down to 2^-31 of it, whatever other rows hold); fp32 queries are split into two half
// terms (2^-22 of them at most), and so is 2^up p s; but one half (2^-11 of it at most, an eighth of an output's rounding to bf16) for bf16 queries of sequences of more than FEW rows, in
// either kernel, so that a row's bits do not hang on which one takes it: two prompts of 2048 tokens behind 4096, whose time is matrix instructions, would take 614 us, not 461.  Single tokens
// wait for the cache's bytes and pay one per cent for the second half (32 sequences 78.1 us, not 77.1; one of 131000 tokens 70.1, not 69.0).
// Trees of drafted tokens have two half terms whatever their rows (16 trees of up to 32 tokens, 64 / 8 heads, behind up to 8000 others, by the kernel for many rows: 215 us, not 203).
// `up` goes by the largest p s among the tokens that the row itself has seen so far, and falls and rises with it as the maximum moves: neither a token that is hidden from the row nor one of a huge
// scale and next to no probability takes bits from the others.
#include "kv_attention.h"

namespace {

constexpr float MOST_FLOAT = 0x1.fffffep127f;
constexpr int HALF_TOP = 14;      // a row's largest probability times scale becomes 2^14 .. 2^15 as half: parts of 2^-28 of it are still normal numbers
constexpr int ROWS = 16, TILE = 64;      // rows (query token, head of the group) of a unit, tokens a wavefront takes at a time
// workgroups that a compute unit holds at once (registers): the shares that the work is cut into are 256 times as many
template <int DP> constexpr int resident() { return DP <= 64 ? 3 : DP <= 128 ? 2 : 1; }

// Rows of a sequence up to which kv_attend_rows_kernel takes it in any call.  Both kernels, 32 sequences behind 2000 others, us, this kernel and the one for many rows:
//     heads (of dh)        32 of 32      64 / 8 of 32    32 of 64     64 / 8 of 64    32 of 128    64 / 8 of 128    8 of 256     16 / 2 of 256
//     32 rows              89   218      37   55         117  230     45   59         156  252     44   70          118  210     42   42
//     64 rows              145  233      53   57         198  246     68   60         283  270     76   73          227  224     61   61
// (heads of 32 would gain at 64 too)
constexpr int FEW = 32;

// how a sequence is cut: row tiles, tiles of tokens that its rows see
__device__ __forceinline__ int row_tiles(const KvSeq& s, int rep) { return (int)(((long long)s.n * rep + ROWS - 1) / ROWS); }
__device__ __forceinline__ int seen_tiles(const KvSeq& s, const AttendArgs& a) {
    const int end = min(s.len, a.q.room);
    return s.n == 0 ? 0 : max((min(end, a.window ? (int)min((long long)a.window + s.n + TILE, 2147483647LL) : end) + TILE - 1) / TILE, 1);
}
__device__ __forceinline__ long long unit_tiles(const KvSeq& s, const AttendArgs& a) { return s.n * a.rep > a.few ? 0 : (long long)row_tiles(s, a.rep) * seen_tiles(s, a) * a.g.heads; }

// tokens that rows r0 .. of a sequence see
struct Span { int lo, hi; };
__device__ __forceinline__ Span row_span(const KvSeq& s, const AttendArgs& a, int r0, int rows) {
    const int p0 = s.len - s.n + r0 / a.rep, p1 = s.len - s.n + (r0 + rows - 1) / a.rep;
    return Span{a.window ? max(p0 - a.window + 1, 0) : 0, max(min(p1 + 1, a.q.room), 0)};
}

// Units (16 rows of a sequence's query tokens and the heads of a KV group, all tokens that they see) follow each other as a list of tiles of 64 tokens, and every workgroup takes an equal
// share of that list, wherever units begin and end; its four wavefronts take every fourth tile and are joined through LDS.  A unit that lies in one share is finished there, pieces of the others go to
// kv_attend_join_kernel.  S^T = K Q^T with tile i's row 4 g + j of the matrix instruction being token 16 g + 4 i + j: lane group g then holds the probabilities of tokens 16 g .. 16 g + 15
// for row lane % 16, which are the right operand of O^T += V^T P^T as they stand.  The loads of V's tile are in flight while its scores are formed, those of K's next one while it is multiplied.
// Bound by the cache's bytes: 32 sequences of 1000 to 8000 tokens, 64 / 8 heads of 128 (319 MB): 68 us and 5 us for the pieces, 4.4 TB/s where a large copy reaches 4.7; one of 131000 tokens (285 MB):
// 52 + 9 us, repeated passes over so little finding part of it in the last cache.
template <typename T, int DP>
__global__ __launch_bounds__(256, resident<DP>()) void kv_attend_rows_kernel(AttendArgs a) {
    constexpr int NT = sizeof(T) == 2 ? 1 : 2;      // half terms of queries
    constexpr int K64 = DP / 64, K32 = (DP % 64) / 32, KS = DP / 32, CT = DP / 16;
    __shared__ float joined[4][ROWS][DP + 4];
    __shared__ float2 ends[4][ROWS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, grp = lane >> 4;
    KvSeq head{0, 0, 0};
    long long total = 0;
    int longest = 1;      // tiles of a unit, up to four
    for (int i = lane; i < a.q.n_seqs; i += 64) {
        const KvSeq e = kv_sequence(a.q, i);
        if (i < 64) head = e;
        const long long mine = unit_tiles(e, a);
        total += mine;
        if (mine) longest = max(longest, min(seen_tiles(e, a), 4));
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) total += __shfl_xor(total, o, 64);
    total = (long long)(unsigned)__builtin_amdgcn_readfirstlane((int)total) | (long long)__builtin_amdgcn_readfirstlane((int)(total >> 32)) << 32;
    const long long share = max((total + gridDim.x - 1) / gridDim.x, 1LL + (__any(longest > 1) != 0) + (__any(longest > 2) != 0) + (__any(longest > 3) != 0));      // (four: a tile for each wavefront)
    long long at = blockIdx.x * share;
    const long long at_end = min(at + share, total);
    if (threadIdx.x == 0) a.info[blockIdx.x] = make_int4(0, 0, 0, 0);
    while (at < at_end) {
        long long x = at;
        int b, h, k0, tile;
        KvSeq s;
        if (!kv_find(a.q, head, [&](const KvSeq& e) { return unit_tiles(e, a); }, x, b, s)) return;
        const int tiles = seen_tiles(s, a);
        if (x >> 31) { k0 = (int)(x % tiles); x /= tiles; h = (int)(x % a.g.heads); tile = (int)(x / a.g.heads); }
        else { const unsigned u = (unsigned)x / tiles; k0 = (unsigned)x - u * tiles; tile = u / a.g.heads; h = u - tile * a.g.heads; }
        h = __builtin_amdgcn_readfirstlane(h); k0 = __builtin_amdgcn_readfirstlane(k0); tile = __builtin_amdgcn_readfirstlane(tile);
        const bool two = NT == 2 || (a.q.n_seqs > 1 ? s.n : a.q.n_tokens) * a.rep <= FEW;      // half terms of probabilities (one sequence alone: as the host, which has only n_tokens, chooses its kernel)
        const int k1 = (int)min((long long)tiles, k0 + (at_end - at));      // tiles k0 .. k1 - 1 of the unit
        const int r0 = tile * ROWS, n_rows = (int)min((long long)ROWS, (long long)s.n * a.rep - r0);
        const Span span = row_span(s, a, r0, n_rows);
        const int lo = (span.lo / TILE + k0) * TILE, hi = min((span.lo / TILE + k1) * TILE, span.hi);
        // this lane's row
        const bool row_live = col < n_rows;
        const int r = r0 + (row_live ? col : 0), tok = r / a.rep, pos = row_live ? s.len - s.n + tok : -1, low = a.window ? pos - a.window + 1 : 0;
        const T* const q = (const T*)a.Q + (long long)(s.start + tok) * a.ldq + (long long)(h * a.rep + r - tok * a.rep) * a.g.dh;
        const int end = min(s.len, a.q.room);
        const long long head_levels = (long long)h * DP << a.g.pt_log, head_grids = (long long)h << (a.g.pt_log - a.g.st_log);
        const int in_page = (1 << a.g.pt_log) - 1;
        const int* const pages = a.q.pages + (long long)b * a.q.per_seq;

        // page of the 16 tokens that this lane takes levels of K from, of V from
        auto page_of = [&](int t) { return pages[min(t >> a.g.pt_log, a.q.per_seq - 1)]; };
        u4 kr[4][K64 + (K64 == 0)]; uint2 ks[4];
        float2 gk, gv;
        bool held = false;
        int pk = 0, pv = 0;
        const unsigned char* vb = a.cache;
        auto load_k = [&](int t0) {      // and the grids of token t0 + lane
            const int tk = t0 + 16 * (col >> 2), tv = t0 + 16 * grp, t = t0 + lane;
            held = pv >= 0 && pv < a.g.n_pages;
            const unsigned char* const kb = a.cache + (long long)min(max(pk, 0), (int)a.g.n_pages - 1) * a.g.page_bytes + head_levels + (long long)((tk & in_page) + (col & 3)) * DP + grp * 16;
            const unsigned char* const vp = a.cache + (long long)(held ? pv : 0) * a.g.page_bytes;
            vb = vp + a.g.v_at + head_levels + (long long)(tv & in_page) * DP + col * 16;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
#pragma unroll
                for (int k = 0; k < K64; ++k) kr[i][k] = *(const u4*)(kb + i * 4 * DP + k * 64);
                if constexpr (K32 != 0) ks[i] = *(const uint2*)(kb + i * 4 * DP + K64 * 64 - grp * 8);
            }
            gk = make_float2(1.f, 0.f); gv = make_float2(0.f, 0.f);
            if (held && t < end) {
                const long long gat = head_grids + ((t & in_page) >> a.g.st_log);
                gk = ((const float2*)(vp + a.g.kg_at))[gat]; gv = ((const float2*)(vp + a.g.vg_at))[gat];
            }
        };
        int t0 = lo + wave * TILE;
        int pk_next = 0, pv_next = 0;
        if (t0 < hi) {
            pk = page_of(t0 + 16 * (col >> 2)); pv = page_of(t0 + 16 * grp);
            load_k(t0);
            pk_next = page_of(t0 + 4 * TILE + 16 * (col >> 2)); pv_next = page_of(t0 + 4 * TILE + 16 * grp);
        }

        h8 qh[NT][KS];
        float unit;
        {
            float v[KS][8], most = 0.f;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const int c = k < 2 * K64 ? (k >> 1) * 64 + grp * 16 + (k & 1) * 8 : K64 * 64 + grp * 8;
                if (a.vec == 4) {
                    union { typename Four<T>::type u[2]; T e[8]; } in;
#pragma unroll
                    for (int j = 0; j < 2; ++j) in.u[j] = row_live && c + 4 * j < a.g.dh ? *(const typename Four<T>::type*)(q + c + 4 * j) : typename Four<T>::type{};
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[k][j] = to_f32(in.e[j]);
                } else if (a.vec) {
                    union { u4 u[sizeof(T) / 2]; T e[8]; } in;
#pragma unroll
                    for (int j = 0; j < (int)sizeof(T) / 2; ++j) in.u[j] = row_live && c < a.g.dh ? ((const u4*)(q + c))[j] : u4{0, 0, 0, 0};
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[k][j] = to_f32(in.e[j]);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[k][j] = row_live && c + j < a.g.dh ? to_f32(q[c + j]) : 0.f;
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) { const float m = fabsf(v[k][j]); most = m < __builtin_inff() ? fmaxf(most, m) : most; }
            }
            most = fmaxf(most, from_xor<16>(most)); most = fmaxf(most, from_xor<32>(most));      // of the row
            const int e = most > 0.f ? min(14 - __builtin_amdgcn_frexp_expf(most), 100) : 0;
            unit = __builtin_amdgcn_ldexpf(a.scale2, -e);
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float w = __builtin_amdgcn_ldexpf(v[k][j], e);
                    const _Float16 hi16 = (_Float16)w;
                    qh[0][k][j] = hi16;
                    if constexpr (NT == 2) qh[1][k][j] = (_Float16)(isfinite(w) ? w - (float)hi16 : 0.f);
                }
        }

        float m = -__builtin_inff(), l = 0.f, most_w = 0.f;      // most_w: largest probability times scale
        int up = HALF_TOP + 1 + 126;                             // brings it to 2^14 .. 2^15
        f4 o[CT];
#pragma unroll
        for (int c = 0; c < CT; ++c) o[c] = f4{0.f, 0.f, 0.f, 0.f};
        for (; t0 < hi; t0 += 4 * TILE) {
            u4 vr[CT];
#pragma unroll
            for (int c = 0; c < CT; ++c) vr[c] = *(const u4*)(vb + c * 256);
            const bool there = held;
            const float sk = gk.x, zk = -1024.f - gk.y, gvx = gv.x, zv = -1024.f - gv.y;
            // scores
            f4 st[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const _Float16 zo = (_Float16)__shfl(zk, 16 * (col >> 2) + 4 * i + (col & 3), 64);
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
            if (t0 + 4 * TILE < hi) {
                pk = pk_next; pv = pv_next;
                load_k(t0 + 4 * TILE);
                pk_next = page_of(t0 + 8 * TILE + 16 * (col >> 2)); pv_next = page_of(t0 + 8 * TILE + 16 * grp);
            }
            float p[16];
            unroll<16>([&](auto I) { constexpr int i = I; p[i] = st[i >> 2][i & 3] * (row_lane<i>(sk) * unit); });
            const bool all = t0 + TILE - 1 <= s.len - s.n + r0 / a.rep && t0 + TILE <= end && t0 >= (a.window ? span.lo + (n_rows - 1) / a.rep + 1 : 0) && __all(there);
            unsigned hidden = 0;
            if (!all) {
                const int tv = t0 + 16 * grp;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int tt = tv + i;
                    if (!(row_live && there && tt < end && tt <= pos && tt >= low)) { hidden |= 1u << i; p[i] = -__builtin_inff(); }
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
            unroll<16>([&](auto I) { constexpr int i = I; p[i] *= row_lane<i>(gvx); });
            if (!all) {      // whatever their scale is
#pragma unroll
                for (int i = 0; i < 16; ++i) if (hidden >> i & 1) p[i] = 0.f;
            }
            float w_top = p[0];
#pragma unroll
            for (int i = 1; i < 16; ++i) w_top = fmaxf(w_top, p[i]);
            w_top = fmaxf(w_top, from_xor<16>(w_top)); w_top = fmaxf(w_top, from_xor<32>(w_top));
            most_w = fmaxf(most_w * turn, fminf(w_top, MOST_FLOAT));
            const int up_was = up;
            up = HALF_TOP + 1 - (most_w > 0.f ? max(__builtin_amdgcn_frexp_expf(most_w), -126) : -126);
            turn = __builtin_amdgcn_ldexpf(turn, up - up_was);      // (up rises only as most_w falls with turn, to nothing at last: 2 at most)
            if (__any(turn != 1.f)) {
#pragma unroll
                for (int c = 0; c < CT; ++c) o[c] *= turn;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) p[i] = __builtin_amdgcn_ldexpf(p[i], up);
            h8 ph[2][2];
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const _Float16 w = (_Float16)p[8 * k + j];
                    ph[0][k][j] = w;
                    ph[1][k][j] = (_Float16)(p[8 * k + j] - (float)w);
                }
            // zeros of V's 16 tokens as pairs
            h2 zo[8];
            {
                const unsigned mine = __builtin_bit_cast(unsigned short, (_Float16)zv);
                const unsigned next = (unsigned)__builtin_amdgcn_mov_dpp((int)mine, 0xB1, 0xf, 0xf, true);      // the neighbour's: quad_perm 1 0 3 2
                const unsigned pair = mine | next << 16;                                                             // (for even lanes)
                unroll<8>([&](auto I) { constexpr int i = I; zo[i] = __builtin_bit_cast(h2, row_lane<2 * i>(pair)); });
            }
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                const h8 v0 = levels8(vr[c][0], vr[c][1], zo[0], zo[1], zo[2], zo[3]), v1 = levels8(vr[c][2], vr[c][3], zo[4], zo[5], zo[6], zo[7]);
                o[c] = mma16(v0, ph[0][0], o[c]); o[c] = mma16(v1, ph[0][1], o[c]);
                if (NT == 2 || two) { o[c] = mma16(v0, ph[1][0], o[c]); o[c] = mma16(v1, ph[1][1], o[c]); }
            }
        }
        l += from_xor<16>(l); l += from_xor<32>(l);
        if (l != l) m = fmaxf(m, 0.f);      // scores that are all NaN leave the maximum where it was: the row has seen something
        if (grp == 0) ends[wave][col] = make_float2(m, l);
        __syncthreads();
        float top = ends[0][col].x;
#pragma unroll
        for (int w = 1; w < 4; ++w) top = fmaxf(top, ends[w][col].x);
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) if (ends[w][col].x != -__builtin_inff()) sum += ends[w][col].y * ex2(ends[w][col].x - top);
        const float f = m == -__builtin_inff() ? 0.f : ex2(m - top) / sum;      // (averages from here on: weighted sums of the largest values leave fp32)
#pragma unroll
        for (int c = 0; c < CT; ++c) *(f4*)&joined[wave][col][c * 16 + grp * 4] = m == -__builtin_inff() ? f4{0.f, 0.f, 0.f, 0.f} : by_power(o[c] * f, -up);
        __syncthreads();
        const bool whole = k0 == 0 && k1 == tiles;
        const long long piece = (2LL * blockIdx.x + (k0 == 0)) * ROWS;
        if (threadIdx.x == 0 && k0 == 0 && !whole) a.info[blockIdx.x] = make_int4((int)((at + tiles - 1) / share) - (int)blockIdx.x + 1, s.start, r0 | (n_rows - 1) << 27, h);
        for (int i = threadIdx.x; i < n_rows * (DP / 4); i += 256) {
            const int rr = i / (DP / 4), c = i % (DP / 4) * 4;
            f4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < 4; ++w) v += *(const f4*)&joined[w][rr][c];
            if (whole) {
                const int row = r0 + rr, tk = row / a.rep;
                T* out = (T*)a.O + (long long)(s.start + tk) * a.ldo + (long long)(h * a.rep + row - tk * a.rep) * a.g.dh;
                store4(out, c, a, v);
            } else *(f4*)(a.part + (piece + rr) * DP + c) = v;
        }
        if (!whole && threadIdx.x < n_rows) a.stat[piece + threadIdx.x] = make_float2(top, sum);      // (lane col of the first wavefront: its row's)
        at += k1 - k0;
        if (at < at_end) __syncthreads();      // (what is in LDS has been read)
    }
}

// Rows of a unit that lies in several shares: averages O_i weighted with 2^(max_i - max) sum_i, over the weights' sum; a wavefront per row of the unit that begins in share blockIdx.x.  DP / 4 lanes hold a row;
// the first pieces are on their way before their weights are known.
template <typename T, int DP>
__global__ __launch_bounds__(256) void kv_attend_join_kernel(AttendArgs a) {
    constexpr int LANES = DP / 4, GROUPS = 64 / LANES, AHEAD = 16;
    const int4 info = a.info[blockIdx.x];
    const int pieces = min(info.x, (int)(gridDim.x - blockIdx.x)), r0 = info.z & ((1 << 27) - 1), n_rows = (int)((unsigned)info.z >> 27) + 1, h = info.w;
    const int lane = threadIdx.x & 63, rr = blockIdx.y * 4 + (threadIdx.x >> 6), c = lane % LANES, group = lane / LANES;
    if (pieces < 1 || rr >= n_rows) return;
    auto place = [&](int i) { return (2LL * (blockIdx.x + i) + (i == 0)) * ROWS + rr; };
    const float* const part = a.part + 4 * c;
    f4 v = {0.f, 0.f, 0.f, 0.f};
    float top = -__builtin_inff(), sum = 0.f;
    for (int i0 = 0; i0 < pieces; i0 += 64) {
        const float2 st = i0 + lane < pieces ? a.stat[place(i0 + lane)] : make_float2(-__builtin_inff(), 0.f);
        const int n = min(pieces - i0, 64);
        f4 ahead[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) { const int i = group + k * GROUPS; ahead[k] = group < GROUPS && i < n ? *(const f4*)(part + place(i0 + i) * DP) : f4{0.f, 0.f, 0.f, 0.f}; }
        float now = fmaxf(st.x, top);
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) now = fmaxf(now, __shfl_xor(now, o, 64));
        const float turn = top == now ? 1.f : ex2(top - now);
        float f = st.x == -__builtin_inff() ? 0.f : ex2(st.x - now) * st.y, more = f;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) more += __shfl_xor(more, o, 64);
        const float had = sum * turn;
        sum = had + more;
        const float part_of = sum == 0.f ? 0.f : 1.f / sum;
        v *= had * part_of; f *= part_of;
        top = now;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) v += ahead[k] * __shfl(f, min(group + k * GROUPS, 63), 64);
        for (int k0 = AHEAD * GROUPS; k0 < n; k0 += AHEAD * GROUPS) {
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) { const int i = k0 + group + k * GROUPS; ahead[k] = group < GROUPS && i < n ? *(const f4*)(part + place(i0 + i) * DP) : f4{0.f, 0.f, 0.f, 0.f}; }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) v += ahead[k] * __shfl(f, min(k0 + group + k * GROUPS, 63), 64);
        }
    }
    f4 all = v;
#pragma unroll
    for (int g = 1; g < GROUPS; ++g)
#pragma unroll
        for (int j = 0; j < 4; ++j) all[j] += __shfl(v[j], min(c + g * LANES, 63), 64);
    if (group == 0) {
        const int row = r0 + rr, tk = row / a.rep;
        T* out = (T*)a.O + (long long)(info.y + tk) * a.ldo + (long long)(h * a.rep + row - tk * a.rep) * a.g.dh;
        store4(out, 4 * c, a, all);
    }
}

// ------------------------------------------------------------------------------------------------ many rows
// Sequences of many new tokens: bound by the matrix instructions and the softmax's vector instructions, so what one workgroup reads of the cache serves 32 rows in each of its W wavefronts.
// A tile of 64 tokens is made into half once, by all of them, and kept in LDS (K by token, V by channel, 16-byte pieces XOR-permuted by row, two tiles of each).  S^T = K Q^T with 32 x 32 x 16
// instructions: the tokens of a tile's rows are ordered so that a lane's 32 scores, as half, are the right operand of O^T += V^T P^T as they stand.
// A wavefront alternates between a run of matrix instructions, scores of tile n and products with V of tile n - 1, and a run of vector instructions, the softmax of tile n and its part in making
// the next tile.  Runs end at a barrier; of the two wavefronts of a SIMD one is a run behind the other, so that one multiplies while the other exponentiates.
// A row's maximum is only followed where it has to be: as long as the sum of a lane's 32 probabilities stays below MOST, so does each of them, and they simply exceed 1 (MOST 2^TILE_TOP = 2^15 is
// within half); no maximum is formed then.
// Two sequences of up to 2048 new tokens behind up to 4096, 64 / 8 heads of 128 (367 GFLOP): 460 to 484 us, card by card, 760 to 800 TFLOP/s of the 1423 that a large product of half matrices reaches.
// What bounds it: a wavefront spends 30 % of its cycles issuing vector and matrix instructions (32 of the latter a tile, beside about 310 vector and 165 scalar ones), 28 % waiting to issue and 26 % at
// counters and barriers; and the units are uneven, the busiest compute unit having 194 tiles where the mean is 173.
constexpr float MOST = 0x1p7f;
constexpr int TILE_TOP = 8;      // halves are below 2^(TILE_TOP + 7): probabilities are up to MOST, scales below the row's bound
constexpr int SPARE = 8;         // a row's bound of scales is so many powers of two above its largest probability times scale: larger scales (the bound is then raised) are rare, and parts of 2^-13 of
                                 // that largest product are still normal halves, each off by 2^-24 of it at most
template <int DP> constexpr int waves() { return DP <= 128 ? 8 : 4; }      // (wider heads need twice the registers)
template <int DP> constexpr int permuted() { return DP % 128 == 0 ? 15 : DP % 64 == 0 ? 7 : 3; }      // bits of a piece's number that K's rows are XORed into
template <int DP> constexpr int tiles_lds() { return 2 * 2 * TILE * DP * 2; }
constexpr int TILES_TARGET = 256;                    // pieces that the units of a call are cut into where they are fewer: one for each compute unit, which holds one workgroup at a time.  1000 tokens of 64 / 8
                                                     // heads of 32, 64, 128, of 16 / 2 of 256: 39, 42, 53, 82 us; with 512: 50, 58, 77, 93 (1100 tokens of 256: 119 and 94)

struct TilesUnit { int b, h, tile, cut, n_cuts; KvSeq s; };
template <int RT>
__device__ __forceinline__ int unit_rows(const KvSeq& s, const AttendArgs& a) { return s.n * a.rep > a.few ? (s.n * a.rep + RT - 1) / RT : 0; }
// Piece x of the call: units by sequence, the last rows first (they see most), heads side by side (an XCD keeps to few heads: its cache holds them)
template <int RT>
__device__ __forceinline__ bool find_unit(const AttendArgs& a, int x, TilesUnit& u) {
    const int lane = threadIdx.x & 63;
    KvSeq head{0, 0, 0};
    int total = 0;
    for (int i = lane; i < a.q.n_seqs; i += 64) {
        const KvSeq e = kv_sequence(a.q, i);
        if (i < 64) head = e;
        total += unit_rows<RT>(e, a);
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) total += __shfl_xor(total, o, 64);
    const long long units = (long long)__builtin_amdgcn_readfirstlane(total) * a.g.heads;
    if (units == 0) return false;
    const int split = units >= TILES_TARGET ? 1 : (int)(TILES_TARGET / units);
    if (x >= units * split) return false;
    u.cut = x % split;
    const int unit = x / split;
    u.h = unit % a.g.heads;
    int at = unit / a.g.heads;
    if (!kv_find(a.q, head, [&](const KvSeq& e) { return unit_rows<RT>(e, a); }, at, u.b, u.s)) return false;
    u.tile = __builtin_amdgcn_readfirstlane(unit_rows<RT>(u.s, a) - 1 - at);
    u.n_cuts = max(min(split, seen_tiles(u.s, a) / 4), 1);
    return u.cut < u.n_cuts;
}

// Trees of drafted tokens: all rows of a sequence see as many tiles, and where units are fewer than compute units they are cut into pieces of at most `share` tiles, the least (in steps of an eighth) with which
// there are no more pieces than compute units: a piece more would begin when the others end.  16 trees of 32 tokens behind 1000 to 8000 others, 64 / 8 heads: 197 us,
// and 263 with some 340 pieces (either by this kernel, with one half term of probabilities).
constexpr int TREE_PIECES = TILES_TARGET;      // no call has more where units are cut
__device__ __forceinline__ Span tree_span(const KvSeq& s, const AttendArgs& a) {
    return Span{a.window ? max(s.len - s.n - a.window, 0) : 0, max(min(s.len, a.q.room), 0)};
}
__device__ __forceinline__ int tree_tiles(const KvSeq& s, const AttendArgs& a) { const Span p = tree_span(s, a); return max((p.hi + TILE - 1) / TILE - p.lo / TILE, 1); }
template <int RT>
__device__ __forceinline__ bool find_tree_unit(const AttendArgs& a, int x, TilesUnit& u) {
    const int lane = threadIdx.x & 63;
    KvSeq head{0, 0, 0};
    int units = 0;
    long long tiles = 0;
    for (int i = lane; i < a.q.n_seqs; i += 64) {
        const KvSeq e = kv_sequence(a.q, i);
        if (i < 64) head = e;
        const int mine = unit_rows<RT>(e, a);
        units += mine;
        if (mine) tiles += (long long)mine * tree_tiles(e, a);
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { units += __shfl_xor(units, o, 64); tiles += __shfl_xor(tiles, o, 64); }
    const long long all = (long long)__builtin_amdgcn_readfirstlane(units) * a.g.heads;
    if (all == 0) return false;
    long long share = all >= TILES_TARGET ? 1LL << 40 : max((tiles * a.g.heads + TILES_TARGET - 1) / TILES_TARGET, 4LL);
    auto cuts = [&](const KvSeq& e) { return (int)((tree_tiles(e, a) + share - 1) / share); };
    while (all < TILES_TARGET) {      // (with a share of the longest sequence's tiles there are as many pieces as units: it ends)
        long long pieces = 0;
        for (int i = lane; i < a.q.n_seqs; i += 64) { const KvSeq e = i < 64 ? head : kv_sequence(a.q, i); const int mine = unit_rows<RT>(e, a); if (mine) pieces += (long long)mine * cuts(e); }
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) pieces += __shfl_xor(pieces, o, 64);
        if (pieces * a.g.heads <= TILES_TARGET) break;
        share += share / 8 + 1;
    }
    long long at = x;
    if (!kv_find(a.q, head, [&](const KvSeq& e) { const int mine = unit_rows<RT>(e, a); return mine ? (long long)mine * a.g.heads * cuts(e) : 0LL; }, at, u.b, u.s)) return false;
    u.n_cuts = __builtin_amdgcn_readfirstlane(cuts(u.s));
    const int item = __builtin_amdgcn_readfirstlane((int)at), unit = item / u.n_cuts;
    u.cut = item - unit * u.n_cuts;
    u.h = unit % a.g.heads; u.tile = unit / a.g.heads;
    return true;
}

__device__ __forceinline__ f16v mma32(h8 a, h8 b, f16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

__device__ __forceinline__ float across_halves(float v) {      // maximum of lanes l and l ^ 32
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
template <typename F>
__device__ __forceinline__ int over_rows(int v, F&& f) {      // of the 32 rows of a wavefront, where lanes l and l ^ 32 hold the same
    v = f(v, __builtin_amdgcn_mov_dpp(v, 0xB1, 0xf, 0xf, true)); v = f(v, __builtin_amdgcn_mov_dpp(v, 0x4E, 0xf, 0xf, true));       // the others of four
    v = f(v, __builtin_amdgcn_mov_dpp(v, 0x141, 0xf, 0xf, true)); v = f(v, __builtin_amdgcn_mov_dpp(v, 0x140, 0xf, 0xf, true));     // of eight, of sixteen
    return f(__builtin_amdgcn_readlane(v, 0), __builtin_amdgcn_readlane(v, 16));
}
__device__ __forceinline__ int least(int a, int b) { return min(a, b); }
__device__ __forceinline__ int greatest(int a, int b) { return max(a, b); }
__device__ __forceinline__ void run_ends() {      // everything before it is before, what was written to LDS is there
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0xc07f);      // lgkmcnt(0), as an instruction that the compiler counts with
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// N times EACH matrix instructions with an LDS operand for EACH: the operands' loads AHEAD of them, no more (the registers would not hold them)
template <int N, int AHEAD, int EACH = 1>
__device__ __forceinline__ void operands_ahead() {
    __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
    for (int i = 0; i < N - AHEAD; ++i) { __builtin_amdgcn_sched_group_barrier(0x8, EACH, 0); __builtin_amdgcn_sched_group_barrier(0x100, 1, 0); }
    __builtin_amdgcn_sched_group_barrier(0x8, EACH * AHEAD, 0);
}

template <int DP, bool WIDE, bool TREE>      // WIDE: pages of 64 tokens and more, a tile lies in one; TREE: a row sees of its sequence's new tokens those that its mask names
__global__ __launch_bounds__(64 * waves<DP>(), waves<DP>() / 4) void kv_attend_tiles_kernel(AttendArgs a) {
    constexpr int W = waves<DP>(), RT = 32 * W, KS = DP / 16, CT = DP / 32, PIECES = 4 * DP, PP = (PIECES + 64 * W - 1) / (64 * W);      // 16-byte pieces of a tile of K (and of V), per thread
    constexpr bool EVEN = PIECES % (64 * W) == 0;
    constexpr int KROW = DP * 2, VROW = TILE * 2, AHEAD = 6;      // bytes of a row in LDS; operands on their way
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    unsigned char* const kbuf = lds;
    unsigned char* const vbuf = lds + 2 * TILE * KROW;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, half = lane >> 5, i16 = lane & 15;
    TilesUnit u;
    const bool any = TREE ? find_tree_unit<RT>(a, blockIdx.x, u) : find_unit<RT>(a, blockIdx.x, u);
    if constexpr (TREE) {      // for the join: pieces of the unit that this is the first one of, where its rows are
        if (tid == 0 && blockIdx.x < TREE_PIECES)
            a.tile_info[blockIdx.x] = any && u.cut == 0 ? make_int4(u.n_cuts, u.s.start, u.tile * RT, u.h | (min(RT, u.s.n * a.rep - u.tile * RT) - 1) << 16) : make_int4(0, 0, 0, 0);
    }
    if (!any) return;
    const KvSeq s = u.s;
    const int h = u.h, r0 = u.tile * RT, n_rows = min(RT, s.n * a.rep - r0);
    const Span span = TREE ? tree_span(s, a) : row_span(s, a, r0, n_rows);
    const int end = min(s.len, a.q.room);
    int lo, hi;      // tokens of this piece: whole tiles, the last one up to hi
    {
        const int t0 = span.lo / TILE, t1 = (span.hi + TILE - 1) / TILE, each = max((t1 - t0 + u.n_cuts - 1) / u.n_cuts, 0);
        lo = (t0 + u.cut * each) * TILE; hi = min((t0 + (u.cut + 1) * each) * TILE, span.hi);
    }
    const int n_tiles = __builtin_amdgcn_readfirstlane(max((hi - lo + TILE - 1) / TILE, 0));
    lo = __builtin_amdgcn_readfirstlane(lo);
    // this lane's row; the wavefront's rows
    const int w0 = wave * 32, w_rows = min(max(n_rows - w0, 0), 32);
    const bool row_live = col < w_rows;
    const int r = r0 + w0 + (row_live ? col : 0), tok = r / a.rep, pos = row_live ? s.len - s.n + tok : -1;
    const unsigned* const mask = TREE ? a.tree + (long long)(s.start + tok) * a.tree_words : nullptr;
    // tiles that the wavefront's rows see anything of, and places that all of them see
    int see0 = 0, see1 = 0, all0 = 0, all1 = -1;
    if (w_rows) {
        const Span mine = TREE ? span : row_span(s, a, r0 + w0, w_rows);
        see0 = max(mine.lo - lo, 0) / TILE; see1 = min((mine.hi - lo + TILE - 1) / TILE, n_tiles);
        all0 = a.window ? s.len - s.n + (r0 + w0 + w_rows - 1) / a.rep - a.window + 1 : 0; all1 = min(s.len - s.n + (r0 + w0) / a.rep, end - 1);
        if constexpr (TREE) { all0 = a.window ? s.len - a.window : 0; all1 = min(s.len - s.n, end) - 1; }
        if (w_rows < 32) all1 = -1;
    }
    see0 = __builtin_amdgcn_readfirstlane(see0); see1 = __builtin_amdgcn_readfirstlane(see1); all0 = __builtin_amdgcn_readfirstlane(all0); all1 = __builtin_amdgcn_readfirstlane(all1);

    const long long head_levels = (long long)h * DP << a.g.pt_log, head_grids = (long long)h << (a.g.pt_log - a.g.st_log);
    const int in_page = (1 << a.g.pt_log) - 1, st_log = a.g.st_log;
    const int* const pages = a.q.pages + (long long)u.b * a.q.per_seq;
    // pages of tile n: that of its 16 tokens lane % 4 (a vector load in either case: a scalar one would share its counter with LDS).  Place: where the tile's levels and grids lie, from
    // the head's in the cache's first page on, or the pages where they are several.
    auto pages_of = [&](int n) { return pages[min((lo + n * TILE + 16 * (lane & 3)) >> a.g.pt_log, a.q.per_seq - 1)]; };
    auto page_offset = [&](int pg) { return (long long)min(max(pg, 0), (int)a.g.n_pages - 1) * a.g.page_bytes; };
    struct Place { int ids; bool held; long long lev, grid; };
    auto place_of = [&](int n, int ids) {
        Place p{ids, false, 0, 0};
        if constexpr (WIDE) {
            const int pg = __builtin_amdgcn_readfirstlane(ids), o = (lo + n * TILE) & in_page;
            p.held = pg >= 0 && pg < (int)a.g.n_pages;
            const long long at = page_offset(pg);
            p.lev = at + o * DP; p.grid = at + (o >> st_log) * 8;
        }
        return p;
    };
    const unsigned char* const k_levels = a.cache + head_levels, * const v_levels = k_levels + a.g.v_at;
    const unsigned char* const k_grids = a.cache + a.g.kg_at + head_grids * 8, * const v_grids = a.cache + a.g.vg_at + head_grids * 8;

    // raw levels of K of one tile and V of the one before it, zero of a piece's token (K), of token 16 g + lane % 16 (V)
    u4 kraw[PP], vraw[PP];
    float kz[PP], vz[PP];
    auto fetch_k = [&](int n, const Place& at) {
#pragma unroll
        for (int j = 0; j < PP; ++j) {
            const unsigned i = tid + j * 64 * W, tk = i / (DP / 16);
            if (!EVEN && i >= PIECES) break;
            if constexpr (WIDE) {
                kraw[j] = *(const u4*)(k_levels + at.lev + i * 16);
                kz[j] = *(const float*)(k_grids + at.grid + ((tk >> st_log) * 8 + 4));
            } else {
                const long long page = page_offset(__shfl(at.ids, tk >> 4, 64));
                const int o = (lo + n * TILE + (int)tk) & in_page;
                kraw[j] = *(const u4*)(k_levels + page + (o * DP + i % (DP / 16) * 16));
                kz[j] = *(const float*)(k_grids + page + ((o >> st_log) * 8 + 4));
            }
        }
    };
    auto fetch_v = [&](int n, const Place& at) {
#pragma unroll
        for (int j = 0; j < PP; ++j) {
            const unsigned i = tid + j * 64 * W, g = i / DP;
            if (!EVEN && i >= PIECES) break;
            if constexpr (WIDE) {
                vraw[j] = *(const u4*)(v_levels + at.lev + i * 16);
                vz[j] = *(const float*)(v_grids + at.grid + (((16 * g + i16) >> st_log) * 8 + 4));
            } else {
                const long long page = page_offset(__shfl(at.ids, g, 64));
                const int o = (lo + n * TILE + 16 * (int)g) & in_page;
                vraw[j] = *(const u4*)(v_levels + page + (o * DP + i % DP * 16));
                vz[j] = *(const float*)(v_grids + page + (((o + i16) >> st_log) * 8 + 4));
            }
        }
    };
    auto store_k = [&](int buf) {
#pragma unroll
        for (int j = 0; j < PP; ++j) {
            const int i = tid + j * 64 * W, tk = i / (DP / 16), c = i % (DP / 16) * 2;
            if (!EVEN && i >= PIECES) break;
            const _Float16 zo = (_Float16)(-1024.f - kz[j]);
            const h2 z = {zo, zo};
            const int row = (tk & ~12) | (tk & 4) << 1 | (tk & 8) >> 1;      // the matrix instruction's row whose result is this token's
            unsigned char* const p = kbuf + buf * TILE * KROW + row * KROW;
            constexpr int M = permuted<DP>();
            *(h8*)(p + (((c & ~M) | ((c ^ row) & M)) << 4)) = levels8(kraw[j][0], kraw[j][1], z, z, z, z);
            *(h8*)(p + ((((c + 1) & ~M) | (((c + 1) ^ row) & M)) << 4)) = levels8(kraw[j][2], kraw[j][3], z, z, z, z);
        }
    };
    auto store_v = [&](int buf) {
#pragma unroll
        for (int j = 0; j < PP; ++j) {
            const int i = tid + j * 64 * W, g = i / DP, c = i % DP;
            if (!EVEN && i >= PIECES) break;
            h2 zo[8];
            const unsigned one = __builtin_bit_cast(unsigned short, (_Float16)(-1024.f - fminf(fmaxf(vz[j], 0.f), 255.f)));      // (what is behind the last token may be anything)
            const unsigned pair = one | (unsigned)__builtin_amdgcn_mov_dpp((int)one, 0xB1, 0xf, 0xf, true) << 16;
            unroll<8>([&](auto I) { constexpr int n = I; zo[n] = __builtin_bit_cast(h2, row_lane<2 * n>(pair)); });
            unsigned char* const p = vbuf + buf * DP * VROW + c * VROW;
            *(h8*)(p + (((2 * g) ^ (c & 7)) << 4)) = levels8(vraw[j][0], vraw[j][1], zo[0], zo[1], zo[2], zo[3]);
            *(h8*)(p + (((2 * g + 1) ^ (c & 7)) << 4)) = levels8(vraw[j][2], vraw[j][3], zo[4], zo[5], zo[6], zo[7]);
        }
    };
    // scales of tokens 32 k + 16 (i16 / 8) + 8 half + i16 % 8, k = 0, 1: those of a lane's scores, one in each lane of a row of 16; which groups of 16 tokens there are
    float gk[2], gv[2];
    unsigned there = 0;      // bit 2 k + i16 / 8
    auto fetch_grids = [&](int n, const Place& at) {
        const int t0 = lo + n * TILE;
        there = WIDE && at.held ? 15u : 0u;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const unsigned in = 32 * k + 16 * (i16 >> 3) + 8 * half + (i16 & 7);
            if constexpr (WIDE) { gk[k] = *(const float*)(k_grids + at.grid + (in >> st_log) * 8); gv[k] = *(const float*)(v_grids + at.grid + (in >> st_log) * 8); }
            else {
                const int pg = __shfl(at.ids, 2 * k + (i16 >> 3), 64), o = (t0 + (int)in) & in_page;
                const unsigned long long b = __ballot(pg >= 0 && pg < (int)a.g.n_pages);
                there |= (unsigned)(b & 1) << 2 * k | (unsigned)(b >> 8 & 1) << (2 * k + 1);
                const long long page = page_offset(pg) + (o >> st_log) * 8;
                gk[k] = *(const float*)(k_grids + page); gv[k] = *(const float*)(v_grids + page);
            }
        }
    };

    // Slot n of LDS, buffer n & 1: K of tile n and V of tile n - 1.  Run n of matrix instructions reads it: the first four wavefronts in the 2 n-th stretch between barriers, the others (`later`)
    // in the next one; its buffer is written in the two stretches before, by the later ones first.
    const int later = __builtin_amdgcn_readfirstlane(W > 4 ? wave >> 2 : 0);
    Place here{}, next{}, second{};      // of tiles n, n + 1, n + 2
    int ids = 0;                         // pages of tile n + 3
    if (n_tiles) {
        here = place_of(0, pages_of(0)); next = place_of(1, pages_of(1)); second = place_of(2, pages_of(2));
        ids = pages_of(3);
        fetch_k(0, here);
        store_k(0);
        if (later) { fetch_v(0, here); if (n_tiles > 1) fetch_k(1, next); }
    }
    h8 qf[KS];
    float unit, own;      // what multiplies a score: of the wavefront, of the row
    {
        const bf16* const q = (const bf16*)a.Q + (long long)(s.start + tok) * a.ldq + (long long)(h * a.rep + r - tok * a.rep) * a.g.dh;
        float most = 0.f;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            const int c = k * 16 + half * 8;
            union { u4 w; u2 f[2]; bf16 e[8]; h8 v; } in;
            if (a.vec == 8) in.w = row_live && c < a.g.dh ? *(const u4*)(q + c) : u4{0, 0, 0, 0};
            else if (a.vec) {
#pragma unroll
                for (int j = 0; j < 2; ++j) in.f[j] = row_live && c + 4 * j < a.g.dh ? *(const u2*)(q + c + 4 * j) : u2{0, 0};
            }
            else {
#pragma unroll
                for (int j = 0; j < 8; ++j) in.e[j] = row_live && c + j < a.g.dh ? q[c + j] : from_f32<bf16>(0.f);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) { const float m = fabsf(to_f32(in.e[j])); most = m < __builtin_inff() ? fmaxf(most, m) : most; }
            qf[k] = in.v;
        }
        most = across_halves(most);
        // the row's own power of two; what multiplies scores on the way is the same for all rows (one that leaves 2^100 between it and the smallest exponent), the rest a power of two
        const bool some = most > 0.f;
        const int e = some ? min(14 - __builtin_amdgcn_frexp_expf(most), 100) : 0;
        const int e0 = over_rows(some ? e : 128, least), e1 = over_rows(some ? e : -128, greatest), shared = e0 > e1 ? 0 : min(e1, e0 + 100);
        unit = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(__builtin_amdgcn_ldexpf(a.scale2, -shared))));
        own = some ? __builtin_amdgcn_ldexpf(1.f, shared - e) : 1.f;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            union { bf16 e[8]; h8 v; } in;
            in.v = qf[k];
#pragma unroll
            for (int j = 0; j < 8; ++j) qf[k][j] = (_Float16)__builtin_amdgcn_ldexpf(to_f32(in.e[j]), e);
        }
    }
    f16v o[CT], sc[2];
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[c][j] = 0.f;
    h8 pf[4], pl[TREE ? 4 : 1];
    float m = -__builtin_inff(), l = 0.f, most_w = 0.f;      // most_w: largest probability times scale that the row had when its bound was last set
    // A half is 2^(TILE_TOP - e_wave) scale, the same for all rows, times 2^d probability: 2^(e_wave - d) is the row's bound of scales, 2^SPARE above most_w.  Rows of 2^200 between them have that
    // (e_wave is at most 2^100 below the largest bound); what lies further below, if anything does, loses bits
    int e_wave = -126 + SPARE, d = 0;
    float limit = 0.f;                     // the least bound of a row
    // places 32 k + 16 (i / 8) + i % 8 + 8 half of the tile at t0 that this row of a tree sees, a bit each
    auto tree_sees = [&](int t0) {
        const int before = s.len - s.n;
        unsigned seen = 0;
        if (pos < 0) return seen;
        int low = 0;
        if (a.window) {
            int bits = 0;
            for (int i = 0; i < a.tree_words && 32 * i < s.n; ++i) bits += __popc(mask[i] & (s.n - 32 * i >= 32 ? ~0u : (1u << (s.n - 32 * i)) - 1));
            low = before + bits - a.window;
        }
        auto below = [](int n) { return n <= 0 ? 0u : n >= 8 ? 0xffu : (1u << n) - 1; };
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int t = t0 + 32 * (g >> 1) + 16 * (g & 1) + 8 * half, j = t - before;
            unsigned b = below(min(before, end) - t) & ~below(low - t);
            if (j > -8 && j < s.n) {
                auto word = [&](int i) { return i >= 0 && i < a.tree_words ? mask[i] : 0u; };
                const unsigned long long two = word(j >> 5) | (unsigned long long)word((j >> 5) + 1) << 32;
                b |= (unsigned)(two >> (j & 31)) & below(end - t) & ~below(-j);
            }
            seen |= b << 8 * g;
        }
        return seen;
    };
    // operands in LDS
    constexpr int M = permuted<DP>();
    auto k_piece = [&](int buf, int k, int c) {
        const int row = 32 * k + col, piece = 2 * c + half;
        return *(const h8*)(kbuf + buf * TILE * KROW + row * KROW + (((piece & ~M) | ((piece ^ col) & M)) << 4));
    };
    auto v_piece = [&](int buf, int k, int c) { return *(const h8*)(vbuf + buf * DP * VROW + (32 * c + col) * VROW + (((2 * k + half) ^ (col & 7)) << 4)); };
    run_ends();
    if (later) {
        if (n_tiles > 0) store_v(1);
        if (n_tiles > 1) store_k(1);
        run_ends();
    }
    for (int n = 0; n <= n_tiles && n_tiles; ++n) {
        // what this wavefront adds to slot n + 1, to slot n + 2 where it is a run behind
        const int slot = n + 1 + later;
        if (n < n_tiles) fetch_grids(n, here);
        if (slot <= n_tiles) fetch_v(slot - 1, later ? next : here);
        if (slot < n_tiles) fetch_k(slot, later ? second : next);
        const int ids_after = pages_of(n + 4);
        const int buf = n & 1;
        const bool qk = n >= see0 && n < see1, pv = n - 1 >= see0 && n - 1 < see1;
        if (qk) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int j = 0; j < 16; ++j) sc[k][j] = 0.f;
#pragma unroll
            for (int i = 0; i < 2 * KS; ++i) sc[i & 1] = mma32(k_piece(buf, i & 1, i >> 1), qf[i >> 1], sc[i & 1]);
            operands_ahead<2 * KS, (AHEAD < 2 * KS ? AHEAD : 2 * KS)>();
        }
        if (pv) {
#pragma unroll
            for (int i = 0; i < 4 * CT; ++i) {
                const h8 v = v_piece(buf, i / CT, i % CT);
                o[i % CT] = mma32(v, pf[i / CT], o[i % CT]);
                if constexpr (TREE) o[i % CT] = mma32(v, pl[i / CT], o[i % CT]);
            }
            operands_ahead<4 * CT, (TREE ? 2 : AHEAD < 4 * CT ? AHEAD : 4 * CT), TREE ? 2 : 1>();      // (trees: registers; 215 us as it is, 227 with 3 or 6, 222 unordered, for the 16 trees at the top)
        }
        run_ends();
        const int t0 = lo + n * TILE;
        if (qk) {
            if (t0 + TILE > end || there != 15u) {      // what is not there counts for no scale
#pragma unroll
                for (int k = 0; k < 2; ++k) if (t0 + 32 * k + 16 * (i16 >> 3) + 8 * half + (i16 & 7) >= end || !(there >> (2 * k + (i16 >> 3)) & 1)) { gk[k] = 1.f; gv[k] = 0.f; }
            }
            const float sk[2] = {gk[0] * unit, gk[1] * unit};
            float p[32], part[4] = {0.f, 0.f, 0.f, 0.f};
            unroll<32>([&](auto I) { constexpr int i = I; sc[i >> 4][i & 15] *= row_lane<i & 15>(sk[i >> 4]); p[i] = ex2(fmaf(sc[i >> 4][i & 15], own, (float)d - m)); part[i & 3] += p[i]; });
            float sum = __builtin_amdgcn_ldexpf((part[0] + part[1]) + (part[2] + part[3]), -d);
            const float s_most = fmaxf(gv[0], gv[1]);
            unsigned tree_bits = ~0u;
            const bool all = t0 >= all0 && t0 + TILE - 1 <= all1 && there == 15u;
            if (!all || __any(sum > MOST || s_most >= limit)) {
                // places 32 k + 16 (i / 8) + i % 8 from first_seen on, seen of them, are seen by this row
                int at = pos;
                asm("" : "+v"(at));      // (what follows from it is not kept in registers from the start on)
                const int low = a.window ? at - a.window + 1 : 0, first_seen = low - t0 - 8 * half;
                const unsigned seen = (unsigned)max(min(at, end - 1) - low + 1, 0), gone = ~there;
                if constexpr (TREE) tree_bits = all && row_live ? ~0u : tree_sees(t0);
                float top = -__builtin_inff();
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    if ((TREE ? !(tree_bits >> i & 1) : (unsigned)(32 * (i >> 4) + 16 * (i >> 3 & 1) + (i & 7) - first_seen) >= seen) || (gone >> (i >> 3) & 1)) sc[i >> 4][i & 15] = -__builtin_inff();
                    top = fmaxf(top, sc[i >> 4][i & 15]);
                }
                const float to = fmaxf(m, across_halves(top) * own);      // (-inf where nothing has been seen)
                __builtin_amdgcn_sched_barrier(0);      // (maximum, probabilities and bounds one after the other: mixed they took 2 % longer with heads of 32 and 64)
                float turn = m == -__builtin_inff() ? 0.f : ex2(m - to), w_top = 0.f;
                m = to; l *= turn;
                const float base = m == -__builtin_inff() ? 0.f : m;
                sum = 0.f;
                asm("" : "+v"(gv[0]), "+v"(gv[1]));      // (nor are scales, spread over a row's lanes, in 32 registers)
                unroll<32>([&](auto I) { constexpr int i = I; p[i] = ex2(fmaf(sc[i >> 4][i & 15], own, -base)); sum += p[i]; w_top = fmaxf(w_top, p[i] * row_lane<i & 15>(gv[i >> 4])); });
                most_w = fmaxf(most_w * turn, fminf(across_halves(w_top), MOST_FLOAT));
                const bool some = m != -__builtin_inff();
                __builtin_amdgcn_sched_barrier(0);
                const int e_was = e_wave - d, e_row = (most_w > 0.f ? max(__builtin_amdgcn_frexp_expf(most_w), -126) : -126) + SPARE;
                const int e_least = over_rows(some ? e_row : 128, least), e_most = over_rows(some ? e_row : -126 + SPARE, greatest);
                const float s_top = across_halves(fminf(fmaxf(gv[0], gv[1]), MOST_FLOAT));      // (seen or not: below, scales by themselves stay finite)
                e_wave = max(min(e_least, e_most), max(e_most - 100, __builtin_amdgcn_frexp_expf(__int_as_float(over_rows(__float_as_int(s_top), greatest))) - 118));
                limit = __uint_as_float((unsigned)(min(e_least, 128) + 127) << 23);
                d = min(e_wave - e_row, 100);
                const int rise = e_was - (e_wave - d), first = min(rise, 100);
                turn = __builtin_amdgcn_ldexpf(turn, first);
#pragma unroll
                for (int c = 0; c < CT; ++c) o[c] *= turn;
                if (__any(rise > first)) {      // (2^rise itself may be no number)
#pragma unroll
                    for (int c = 0; c < CT; ++c)
#pragma unroll
                        for (int j = 0; j < 16; ++j) o[c][j] = __builtin_amdgcn_ldexpf(o[c][j], rise - first);
                }
#pragma unroll
                for (int i = 0; i < 32; ++i) p[i] = __builtin_amdgcn_ldexpf(p[i], d);
            }
            l += sum;
            const float sv[2] = {__builtin_amdgcn_ldexpf(gv[0], TILE_TOP - e_wave), __builtin_amdgcn_ldexpf(gv[1], TILE_TOP - e_wave)};
            unroll<32>([&](auto I) { constexpr int i = I; p[i] *= row_lane<i & 15>(sv[i >> 4]); });
            if (!all && __any(sv[0] * 0.f + sv[1] * 0.f != 0.f)) {      // scales that are no numbers: what is not seen counts for nothing whatever its scale is
                int at = pos;
                asm("" : "+v"(at));
                const int low = a.window ? at - a.window + 1 : 0, first_seen = low - t0 - 8 * half;
                const unsigned seen = (unsigned)max(min(at, end - 1) - low + 1, 0), gone = ~there;
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if ((TREE ? !(tree_bits >> i & 1) : (unsigned)(32 * (i >> 4) + 16 * (i >> 3 & 1) + (i & 7) - first_seen) >= seen) || (gone >> (i >> 3) & 1)) p[i] = 0.f;
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    pf[k][j] = (_Float16)p[8 * k + j];
                    if constexpr (TREE) pl[k][j] = (_Float16)(p[8 * k + j] - (float)pf[k][j]);
                }
        }
        if (slot <= n_tiles) store_v(slot & 1);
        if (slot < n_tiles) store_k(slot & 1);
        here = next; next = second; second = place_of(n + 3, ids); ids = ids_after;
        run_ends();
    }
    if (W > 4 && !later) run_ends();      // as many as the others
    const int up = TILE_TOP - e_wave + d;
    l += from_xor<32>(l);
    if (l != l) m = fmaxf(m, 0.f);      // scores that are all NaN leave the maximum where it was
    const bool none = m == -__builtin_inff() || l == 0.f;
    const float f = none ? 0.f : 1.f / l;
    if (u.n_cuts == 1) {
        bf16* const out = (bf16*)a.O + (long long)(s.start + tok) * a.ldo + (long long)(h * a.rep + r - tok * a.rep) * a.g.dh;
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            f4 v[4];      // channels 32 c + 8 g + 4 half ..
#pragma unroll
            for (int g = 0; g < 4; ++g)
#pragma unroll
                for (int k = 0; k < 4; ++k) v[g][k] = none ? 0.f : __builtin_amdgcn_ldexpf(o[c][4 * g + k] * f, -up);
            if (a.out_piece == 8) {      // the two halves of the wavefront exchange theirs for whole 16-byte pieces
#pragma unroll
                for (int g = 0; g < 4; g += 2) {
                    const uint2 x = pack4(v[g]), y = pack4(v[g + 1]);
                    const auto p = __builtin_amdgcn_permlane32_swap(x.x, y.x, false, false), q = __builtin_amdgcn_permlane32_swap(x.y, y.y, false, false);
                    const int ch = 32 * c + 8 * (g + half);
                    if (row_live && ch < a.g.dh) *(uint4*)(out + ch) = make_uint4(p[0], q[0], p[1], q[1]);
                }
            } else if (row_live) {
#pragma unroll
                for (int g = 0; g < 4; ++g) store4(out, 32 * c + 8 * g + 4 * half, a, v[g]);
            }
        }
    } else {
        if (!row_live) return;
        const long long at = (long long)blockIdx.x * RT + w0 + col;
        if (half == 0) a.tile_stat[at] = make_float2(m, l);
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *(f4*)(a.tile_part + at * DP + 32 * c + 8 * i + 4 * half) = none ? f4{0.f, 0.f, 0.f, 0.f} : by_power(f4{o[c][4 * i], o[c][4 * i + 1], o[c][4 * i + 2], o[c][4 * i + 3]} * f, -up);
    }
}

// Rows of units that were cut: DP / 4 lanes per row, as kv_attend_join_kernel
template <int DP, int RT>
__global__ __launch_bounds__(256) void kv_attend_tiles_join_kernel(AttendArgs a) {
    constexpr int LANES = DP / 4, GROUPS = 64 / LANES;
    TilesUnit u;
    {   // unit blockIdx.x: the piece with cut 0 tells how many there are
        KvSeq head{0, 0, 0};
        int total = 0;
        for (int i = threadIdx.x & 63; i < a.q.n_seqs; i += 64) total += unit_rows<RT>(kv_sequence(a.q, i), a);
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) total += __shfl_xor(total, o, 64);
        const long long units = (long long)__builtin_amdgcn_readfirstlane(total) * a.g.heads;
        if (blockIdx.x >= units || units >= TILES_TARGET) return;
        const int split = (int)(TILES_TARGET / units);
        if (split < 2 || !find_unit<RT>(a, blockIdx.x * split, u) || u.n_cuts < 2) return;
        u.cut = blockIdx.x * split;      // (its number)
    }
    const int r0 = u.tile * RT, n_rows = min(RT, u.s.n * a.rep - r0), lane = threadIdx.x & 63, c = 4 * (lane % LANES), group = lane / LANES;
    if (group >= GROUPS || c >= a.g.dh) return;
    for (int rr = (blockIdx.y * 4 + (threadIdx.x >> 6)) * GROUPS + group; rr < n_rows; rr += 4 * gridDim.y * GROUPS) {
        float top = -__builtin_inff(), sum = 0.f;
#pragma unroll 4
        for (int i = 0; i < u.n_cuts; ++i) top = fmaxf(top, a.tile_stat[(long long)(u.cut + i) * RT + rr].x);
        auto weight = [&](long long at) { const float2 st = a.tile_stat[at]; return st.x == -__builtin_inff() ? 0.f : ex2(st.x - top) * st.y; };
#pragma unroll 4
        for (int i = 0; i < u.n_cuts; ++i) sum += weight((long long)(u.cut + i) * RT + rr);
        const float part_of = sum == 0.f ? 0.f : 1.f / sum;
        f4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int i = 0; i < u.n_cuts; ++i) {
            const long long at = (long long)(u.cut + i) * RT + rr;
            v += weight(at) * part_of * *(const f4*)(a.tile_part + at * DP + c);
        }
        const int row = r0 + rr, tk = row / a.rep;
        bf16* const out = (bf16*)a.O + (long long)(u.s.start + tk) * a.ldo + (long long)(u.h * a.rep + row - tk * a.rep) * a.g.dh;
        store4(out, c, a, v);
    }
}

// the same for trees: a lane group per row of the unit whose first piece this is
template <int DP, int RT>
__global__ __launch_bounds__(256) void kv_tree_tiles_join_kernel(AttendArgs a) {
    constexpr int LANES = DP / 4, GROUPS = 64 / LANES;
    const int4 info = a.tile_info[blockIdx.x];
    const int n_cuts = info.x, n_rows = (info.w >> 16) + 1, h = info.w & 0xffff, lane = threadIdx.x & 63, c = 4 * (lane % LANES), group = lane / LANES;
    if (n_cuts < 2 || group >= GROUPS || c >= a.g.dh) return;
    for (int rr = (blockIdx.y * 4 + (threadIdx.x >> 6)) * GROUPS + group; rr < n_rows; rr += 4 * gridDim.y * GROUPS) {
        const long long first = (long long)blockIdx.x * RT + rr;
        float top = -__builtin_inff(), sum = 0.f;
#pragma unroll 4
        for (int i = 0; i < n_cuts; ++i) top = fmaxf(top, a.tile_stat[first + (long long)i * RT].x);
        f4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int i = 0; i < n_cuts; ++i) {
            const long long at = first + (long long)i * RT;
            const float2 st = a.tile_stat[at];
            const f4 part = *(const f4*)(a.tile_part + at * DP + c);
            const float w = st.x == -__builtin_inff() ? 0.f : ex2(st.x - top) * st.y, more = sum + w;      // (averages all the way: the weighted sums of the largest values leave fp32)
            const float of = more == 0.f ? 0.f : 1.f / more;
            v = v * (sum * of) + part * (w * of);
            sum = more;
        }
        const int row = info.z + rr, tk = row / a.rep;
        bf16* const out = (bf16*)a.O + (long long)(info.y + tk) * a.ldo + (long long)(h * a.rep + row - tk * a.rep) * a.g.dh;
        store4(out, c, a, v);
    }
}

int shares(int dp) { return 256 * (dp == 32 ? resident<32>() : dp == 64 ? resident<64>() : dp <= 128 ? resident<128>() : resident<256>()); }
int unit_rows_of(int dp) { return 32 * (dp <= 128 ? waves<128>() : waves<256>()); }
// Calls whose units of 16 rows, by what the host knows, are few and short: the rows' kernel alone.  Two units (or a few of three) per workgroup of it are done before a tiles' workgroup has gone
// through the serial part of its first one: 36 new tokens behind 1093 others of six sequences (32 heads of 128, 576 units, 10000 tiles in all) 47 us, not 64; 256 new tokens of one (64 / 8 heads, 1024
// units) 28, not 33, with heads of 256 (16 / 2) 21, not 56, but of 64 32, not 26, and of 32 28, not 24; 64 behind 4000 others (256 units, 16000 tiles) 43 and 39, heads of 256 37 and 61; 16 behind 31000
// (64 units, 31000 tiles) 96 and 52, heads of 256 73 and 120; 16 sequences of 250 (8192 units) 158 and 62.  The host knows no lengths: a row of pages counts as if it were full, and one much wider than its
// sequences sends short calls to the other kernel.
bool is_small(const KvGeometry& g, const tboa_kv_batch& b, int rep, int window) {
    const long long room = ((long long)b.pages_per_seq << g.pt_log) + TILE, units = (b.n_tokens * rep / ROWS + std::min<long long>(b.n_seqs, b.n_tokens)) * g.heads;
    return units <= 9 * shares(g.dp) / 4 && units * ((window ? std::min<long long>(room, (long long)window + b.n_tokens + 2 * TILE) : room) / TILE) <= 16384;
}
// Row tiles of all sequences that kv_attend_tiles_kernel takes: at most one more per sequence than rows / RT, and one per token or more
long long most_units(const KvGeometry& g, int n_seqs, long long n_tokens, int rep) {
    const int rt = unit_rows_of(g.dp);
    return std::min(n_tokens * rep / rt + std::min<long long>(n_seqs, n_tokens), n_tokens * cdiv64(rep, rt)) * g.heads;
}
size_t room(const KvGeometry& g, bool tiles, long long units, AttendArgs* a, void* ws) {
    const size_t n = (size_t)shares(g.dp), pieces = tiles ? (size_t)std::min<long long>(TILES_TARGET, std::max<long long>(units, 1) * TILES_TARGET) : 0;
    Arena ar(ws);
    float* part = ar.get<float>(2 * n * ROWS * g.dp);
    float2* stat = ar.get<float2>(2 * n * ROWS);
    int4* info = ar.get<int4>(n);
    float* tile_part = ar.get<float>(pieces * unit_rows_of(g.dp) * g.dp);
    float2* tile_stat = ar.get<float2>(pieces * unit_rows_of(g.dp));
    if (a) { a->part = part; a->stat = stat; a->info = info; a->tile_part = tile_part; a->tile_stat = tile_stat; }
    return ar.off;
}

template <typename T, int DP>
int attend_rows(tboa_ctx* ctx, const AttendArgs& a) {
    hipLaunchKernelGGL((kv_attend_rows_kernel<T, DP>), dim3(256 * resident<DP>()), dim3(256), 0, ctx->stream, a);
    TB_KERNEL_CHECK(ctx);
    hipLaunchKernelGGL((kv_attend_join_kernel<T, DP>), dim3(256 * resident<DP>(), ROWS / 4), dim3(256), 0, ctx->stream, a);
    TB_KERNEL_CHECK(ctx);
    return 0;
}
template <int DP>
int attend_tiles(tboa_ctx* ctx, const AttendArgs& a, long long units) {
    constexpr int LDS = tiles_lds<DP>();
    const dim3 grid((unsigned)std::max<long long>(units, TILES_TARGET)), block(64 * waves<DP>());
    const unsigned cut = (unsigned)std::min<long long>(units, TILES_TARGET / 2);      // units that may be cut
    if (a.g.pt_log >= 6) {
        TB_HIP(ctx, hipFuncSetAttribute((const void*)kv_attend_tiles_kernel<DP, true, false>, hipFuncAttributeMaxDynamicSharedMemorySize, LDS));
        hipLaunchKernelGGL((kv_attend_tiles_kernel<DP, true, false>), grid, block, LDS, ctx->stream, a);
    } else {
        TB_HIP(ctx, hipFuncSetAttribute((const void*)kv_attend_tiles_kernel<DP, false, false>, hipFuncAttributeMaxDynamicSharedMemorySize, LDS));
        hipLaunchKernelGGL((kv_attend_tiles_kernel<DP, false, false>), grid, block, LDS, ctx->stream, a);
    }
    TB_KERNEL_CHECK(ctx);
    hipLaunchKernelGGL((kv_attend_tiles_join_kernel<DP, 32 * waves<DP>()>), dim3(cut, (unsigned)std::min<long long>(std::max(2048u / cut, 1u), 8 * waves<DP>())), dim3(256), 0, ctx->stream, a);
    TB_KERNEL_CHECK(ctx);
    return 0;
}
template <typename T, int DP>
int attend(tboa_ctx* ctx, const AttendArgs& a, bool rows, long long units) {
    if constexpr (sizeof(T) == 2) { if (units) TB_TRY(attend_tiles<DP>(ctx, a, units)); }
    return rows ? attend_rows<T, DP>(ctx, a) : 0;
}
template <typename T>
int attend(tboa_ctx* ctx, const AttendArgs& a, bool rows, long long units) {
    switch (a.g.dp) {
        case 32: return attend<T, 32>(ctx, a, rows, units);
        case 64: return attend<T, 64>(ctx, a, rows, units);
        case 96: return attend<T, 96>(ctx, a, rows, units);
        case 128: return attend<T, 128>(ctx, a, rows, units);
        case 192: return attend<T, 192>(ctx, a, rows, units);
        default: return attend<T, 256>(ctx, a, rows, units);
    }
}

template <int DP>
int attend_tree_tiles(tboa_ctx* ctx, const AttendArgs& a, long long units) {
    constexpr int LDS = tiles_lds<DP>(), RT = 32 * waves<DP>();
    const dim3 grid((unsigned)std::max<long long>(units, TREE_PIECES)), block(64 * waves<DP>());
    if (a.g.pt_log >= 6) {
        TB_HIP(ctx, hipFuncSetAttribute((const void*)kv_attend_tiles_kernel<DP, true, true>, hipFuncAttributeMaxDynamicSharedMemorySize, LDS));
        hipLaunchKernelGGL((kv_attend_tiles_kernel<DP, true, true>), grid, block, LDS, ctx->stream, a);
    } else {
        TB_HIP(ctx, hipFuncSetAttribute((const void*)kv_attend_tiles_kernel<DP, false, true>, hipFuncAttributeMaxDynamicSharedMemorySize, LDS));
        hipLaunchKernelGGL((kv_attend_tiles_kernel<DP, false, true>), grid, block, LDS, ctx->stream, a);
    }
    TB_KERNEL_CHECK(ctx);
    hipLaunchKernelGGL((kv_tree_tiles_join_kernel<DP, RT>), dim3(TREE_PIECES, 16), dim3(256), 0, ctx->stream, a);      // (pieces behind those are of units that are not cut)
    TB_KERNEL_CHECK(ctx);
    return 0;
}

}  // namespace

size_t kv_tree_tiles_room(const KvGeometry& g, AttendArgs* a, void* ws) {
    const size_t rows = (size_t)TREE_PIECES * unit_rows_of(g.dp);
    Arena ar(ws);
    float* part = ar.get<float>(rows * g.dp);
    float2* stat = ar.get<float2>(rows);
    int4* info = ar.get<int4>(TREE_PIECES);
    if (a) { a->tile_part = part; a->tile_stat = stat; a->tile_info = info; }
    return ar.off;
}
bool kv_tree_tiles_takes(const KvGeometry& g, int n_seqs, long long n_tokens, int rep) { return most_units(g, n_seqs, n_tokens, rep) < (1LL << 32) / (2 * unit_rows_of(g.dp)); }
int kv_tree_tiles(tboa_ctx* ctx, const AttendArgs& a) {
    const long long units = most_units(a.g, a.q.n_seqs, a.q.n_tokens, a.rep);
    switch (a.g.dp) {
        case 32: return attend_tree_tiles<32>(ctx, a, units);
        case 64: return attend_tree_tiles<64>(ctx, a, units);
        case 96: return attend_tree_tiles<96>(ctx, a, units);
        case 128: return attend_tree_tiles<128>(ctx, a, units);
        case 192: return attend_tree_tiles<192>(ctx, a, units);
        default: return attend_tree_tiles<256>(ctx, a, units);
    }
}

extern "C" size_t tboa_kv_cache_attention_workspace_bytes(const tboa_kv_cache_desc* desc, int n_q_heads, int n_seqs, int64_t n_tokens) {
    KvGeometry g;
    if (!kv_geometry(desc, g) || n_q_heads <= 0 || n_q_heads > 65535 || n_q_heads % g.heads || n_seqs < 0 || n_seqs > 1 << 20 || n_tokens < 0 || n_tokens > 1 << 24) return 0;
    return n_seqs == 0 || n_tokens == 0 ? 0 : room(g, n_tokens * (n_q_heads / g.heads) > FEW, most_units(g, n_seqs, n_tokens, n_q_heads / g.heads), nullptr, nullptr);
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
    const int rep = n_q_heads / g.heads, size = dtype == TBOA_F32 ? 4 : 2;
    if (batch->n_tokens * rep >= 1LL << 27) return tboa_fail(ctx, TBOA_EINVAL, "kv_cache_attention: too many rows");
    KvDevice dev(ctx->device);
    // sequences of more than FEW rows go to the tiles' kernel (16-bit inputs), the others to the rows'; what the caller says of the batch may spare one of the two launches
    const long long most = batch->max_new > 0 ? std::min<long long>(batch->max_new, batch->n_tokens) : batch->n_tokens;
    // (of 2^32 work items and more the runtime would start what is left modulo 2^32: such calls are the rows' kernel's, whose grid does not grow)
    const long long might = most_units(g, batch->n_seqs, batch->n_tokens, rep);
    const bool tiles = dtype == TBOA_BF16 && most * rep > FEW && !is_small(g, *batch, rep, window) && might < (1LL << 32) / (2 * unit_rows_of(g.dp));
    const bool rows = !tiles || batch->n_seqs > 1 || batch->n_tokens * rep <= FEW;
    const long long units = tiles ? might : 0;
    TB_TRY(tboa_ws_reserve(ctx, room(g, tiles, units, nullptr, nullptr)));
    AttendArgs a;
    a.g = g;
    a.q = KvBatch{batch->n_seqs, batch->pages_per_seq, (int)batch->n_tokens, batch->pages_per_seq * desc->page_tokens, batch->starts, batch->lens, batch->pages};
    a.Q = Q; a.ldq = ldq; a.O = O; a.ldo = ldo; a.cache = (const unsigned char*)cache;
    a.scale2 = (float)((scale == 0.0 ? 1.0 / sqrt((double)g.dh) : scale) * 1.4426950408889634);
    a.rep = rep; a.window = window < KV_MOST_TOKENS ? window : 0;      // (no sequence is longer)
    a.vec = g.dh % 8 == 0 && ((uintptr_t)Q & 15) == 0 && ldq * size % 16 == 0 ? 8 : g.dh % 4 == 0 && ldq % 4 == 0 && ((uintptr_t)Q & (4 * size - 1)) == 0 ? 4 : 0;
    a.out_piece = g.dh % 8 == 0 && ldo % 8 == 0 && ((uintptr_t)O & 15) == 0 ? 8 : g.dh % 4 == 0 && ldo % 4 == 0 && ((uintptr_t)O & (4 * size - 1)) == 0 ? 4 : 1;
    a.few = !tiles ? 1 << 30 : rows ? FEW : 0;
    room(g, tiles, units, &a, ctx->ws);
    return dtype == TBOA_F32 ? attend<float>(ctx, a, rows, units) : attend<bf16>(ctx, a, rows, units);
}
