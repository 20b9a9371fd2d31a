// Attention of a tree of drafted tokens over a quantized key/value cache: a row (drafted token, head of the group) sees the places before its sequence's new tokens, and of these the ones that
// its mask names.
//
// The same products and the same running softmax as attention of a chain (kv_attention.hip): levels less their zero are exact in half, scales multiply scores and probabilities,
//     x[t] = (scale s^K_t log2 e) q.(c^K_t - z^K_t),   p = 2^(x - max),   O += (2^up p s^V_t) (c^V_t - z^V_t)
// with a power of two per row for its query and one, `up`, by the largest p s among the tokens that the row itself has seen.  fp32 queries are two half terms, and so is
// 2^up p s, for bf16 queries too (2^-22 of it at most).
#include "kv_attention.h"

namespace {

constexpr float MOST_FLOAT = 0x1.fffffep127f;
constexpr int HALF_TOP = 14;      // a row's largest probability times scale becomes 2^14 .. 2^15 as half
constexpr int TILE = 64, RW = 16;      // tokens a wavefront takes at a time, its rows
template <int DP> constexpr int resident() { return DP <= 128 ? 2 : 1; }      // workgroups that a compute unit holds at once (registers)

// How a sequence is cut.  A workgroup's four wavefronts take `wr` blocks of RW rows side by side and 4 / wr tiles of 64 tokens at a time (a step).
struct Cut { int wr, wt, blocks, first, tiles, steps; };
__device__ __forceinline__ Cut cut_of(const KvSeq& s, const AttendArgs& a) {
    Cut c;
    const int rows = s.n * a.rep;
    const int most = min(rows, a.piece_rows);      // (a caller's max_new that is too small leaves room for fewer: then there are more blocks)
    c.wr = most <= RW ? 1 : most <= 2 * RW ? 2 : 4;
    c.wt = 4 / c.wr;
    c.blocks = (rows + RW * c.wr - 1) / (RW * c.wr);
    const int before = s.len - s.n, hi = min(s.len, a.q.room);
    c.first = (a.window ? max(before - a.window, 0) : 0) / TILE;      // (a mask may be empty: its row stands one place before the first new token)
    c.tiles = max((hi + TILE - 1) / TILE - c.first, 1);
    c.steps = (c.tiles + c.wt - 1) / c.wt;
    return c;
}
__device__ __forceinline__ long long steps_of(const KvSeq& s, const AttendArgs& a) {
    if (s.n == 0 || s.n * a.rep > a.few) return 0;
    const Cut c = cut_of(s, a);
    return (long long)c.blocks * a.g.heads * c.steps;
}
__device__ __forceinline__ unsigned below(int n) { return n <= 0 ? 0u : n >= 16 ? 0xffffu : (1u << n) - 1; }      // bits 0 .. n - 1 of 16

// Units (up to 4 RW rows of a sequence's drafted tokens and the heads of a KV group, all places that they see) follow each other as a list of steps, and every workgroup takes an equal share of
// that list; pieces of units that lie in several shares go to kv_tree_join_kernel.
// S^T = K Q^T with tile i's row 4 g + j of the matrix instruction being token 16 g + 4 i + j: lane group g then holds the probabilities of tokens 16 g .. 16 g + 15 for row lane % 16, which are
// the right operand of O^T += V^T P^T as they stand.
// Bound by the vector instructions that make levels into half and the softmax: 8 trees of up to 64 tokens behind up to 4000 others, 32 heads of 128, a row a token: 88 us and 10 for the join, where vector
// instructions are issued 59 % of the time and wavefronts wait 26 % of theirs (the levels take 37 at the rate of memory).  With two units of 16 rows a wavefront, which would make levels into half once for both,
// registers spill: 121 us, 61 % of the time waiting.
template <typename T, int DP>
__global__ __launch_bounds__(256, resident<DP>()) void kv_tree_kernel(AttendArgs a) {
    constexpr int NT = sizeof(T) == 2 ? 1 : 2;      // half terms of queries
    constexpr int K64 = DP / 64, K32 = (DP % 64) / 32, KS = DP / 32, CT = DP / 16;
    __shared__ float joined[4][RW][DP + 4];
    __shared__ float2 ends[4][RW];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, grp = lane >> 4;
    KvSeq head{0, 0, 0};
    long long total = 0;
    for (int i = lane; i < a.q.n_seqs; i += 64) {
        const KvSeq e = kv_sequence(a.q, i);
        if (i < 64) head = e;
        total += steps_of(e, a);
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) total += __shfl_xor(total, o, 64);
    total = (long long)(unsigned)__builtin_amdgcn_readfirstlane((int)total) | (long long)__builtin_amdgcn_readfirstlane((int)(total >> 32)) << 32;
    const long long share = max((total + gridDim.x - 1) / gridDim.x, 1LL);
    long long at = blockIdx.x * share;
    const long long at_end = min(at + share, total);
    if (threadIdx.x == 0) a.info[blockIdx.x] = make_int4(0, 0, 0, 0);
    while (at < at_end) {
        long long x = at;
        int b;
        KvSeq s;
        if (!kv_find(a.q, head, [&](const KvSeq& e) { return steps_of(e, a); }, x, b, s)) return;
        const Cut c = cut_of(s, a);
        const int step0 = __builtin_amdgcn_readfirstlane((int)(x % c.steps));
        x /= c.steps;
        const int h = __builtin_amdgcn_readfirstlane((int)(x % a.g.heads)), r0 = __builtin_amdgcn_readfirstlane((int)(x / a.g.heads) * (RW * c.wr));
        const int step1 = (int)min((long long)c.steps, step0 + (at_end - at));      // steps step0 .. step1 - 1 of the unit
        const int rows = s.n * a.rep, n_rows = min(RW * c.wr, rows - r0);
        const int before = s.len - s.n, end = min(s.len, a.q.room), group = wave / c.wr, rg = wave - group * c.wr;
        const int hi = min((c.first + step1 * c.wt) * TILE, end), stride = c.wt * TILE;
        // this lane's row
        const int r = r0 + rg * RW + col;
        const bool own = r < rows;
        const int tok = own ? r / a.rep : 0, hh = own ? r - tok * a.rep : 0;
        const bool live = own && before + tok >= 0;
        const T* const q = (const T*)a.Q + (long long)(s.start + tok) * a.ldq + (long long)(h * a.rep + hh) * a.g.dh;
        const unsigned* const mask = a.tree + (long long)(s.start + tok) * a.tree_words;
        int low = 0;
        if (a.window) {      // of the places before the new tokens, the last ones of the window that ends at the row's own, which is as far behind them as its mask has bits
            int bits = 0;
            for (int i = 0; i < a.tree_words && 32 * i < s.n; ++i) bits += __popc(mask[i] & (s.n - 32 * i >= 32 ? ~0u : (1u << (s.n - 32 * i)) - 1));
            low = before + bits - a.window;
        }
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
        int t0 = (c.first + step0 * c.wt + group) * TILE;
        int pk_next = 0, pv_next = 0;
        if (t0 < hi) {
            pk = page_of(t0 + 16 * (col >> 2)); pv = page_of(t0 + 16 * grp);
            load_k(t0);
            pk_next = page_of(t0 + stride + 16 * (col >> 2)); pv_next = page_of(t0 + stride + 16 * grp);
        }

        h8 qh[NT][KS];
        float unit;
        {
            float v[KS][8], most = 0.f;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const int ch = k < 2 * K64 ? (k >> 1) * 64 + grp * 16 + (k & 1) * 8 : K64 * 64 + grp * 8;
                if (a.vec == 4) {
                    union { typename Four<T>::type u[2]; T e[8]; } in;
#pragma unroll
                    for (int j = 0; j < 2; ++j) in.u[j] = live && ch + 4 * j < a.g.dh ? *(const typename Four<T>::type*)(q + ch + 4 * j) : typename Four<T>::type{};
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[k][j] = to_f32(in.e[j]);
                } else if (a.vec) {
                    union { u4 u[sizeof(T) / 2]; T e[8]; } in;
#pragma unroll
                    for (int j = 0; j < (int)sizeof(T) / 2; ++j) in.u[j] = live && ch < a.g.dh ? ((const u4*)(q + ch))[j] : u4{0, 0, 0, 0};
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[k][j] = to_f32(in.e[j]);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[k][j] = live && ch + j < a.g.dh ? to_f32(q[ch + j]) : 0.f;
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

        float m = -__builtin_inff(), l = 0.f, most_w = 0.f;      // maximum, sum, largest probability times scale
        int up = HALF_TOP + 1 + 126;                              // brings that to 2^14 .. 2^15
        f4 o[CT];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) o[ct] = f4{0.f, 0.f, 0.f, 0.f};
        for (; t0 < hi; t0 += stride) {
            u4 vr[CT];
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) vr[ct] = *(const u4*)(vb + ct * 256);
            const bool there = held;
            const float sk = gk.x, zk = -1024.f - gk.y, gvx = gv.x, zv = -1024.f - gv.y;
            // scores
            f4 st[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const _Float16 zo = (_Float16)__shfl(zk, 16 * (col >> 2) + 4 * i + (col & 3), 64);
                const h2 z = {zo, zo};
                st[i] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    h8 lv;
                    if (k < 2 * K64) lv = levels8(kr[i][k >> 1][(k & 1) * 2], kr[i][k >> 1][(k & 1) * 2 + 1], z, z, z, z);
                    else lv = levels8(ks[i].x, ks[i].y, z, z, z, z);
#pragma unroll
                    for (int n = 0; n < NT; ++n) st[i] = mma16(lv, qh[n][k], st[i]);
                }
            }
            if (t0 + stride < hi) {
                pk = pk_next; pv = pv_next;
                load_k(t0 + stride);
                pk_next = page_of(t0 + 2 * stride + 16 * (col >> 2)); pv_next = page_of(t0 + 2 * stride + 16 * grp);
            }
            const bool all = t0 + TILE <= min(before, end) && (!a.window || t0 >= before + s.n - a.window) && __all(there);
            h8 ph[2][2];
            float p[16];
            unroll<16>([&](auto I) { constexpr int i = I; p[i] = st[i >> 2][i & 3] * (row_lane<i>(sk) * unit); });
            unsigned seen = 0xffffu;
            if (!all) {
                const int tv = t0 + 16 * grp, j0 = tv - before;      // places tv .. tv + 15: before the new tokens, or the new tokens from the j0-th on
                seen = below(min(before, end) - tv) & ~below(low - tv);
                if (j0 > -16 && j0 < s.n) {
                    auto word = [&](int i) { return i >= 0 && i < a.tree_words ? mask[i] : 0u; };
                    const unsigned long long bits = word(j0 >> 5) | (unsigned long long)word((j0 >> 5) + 1) << 32;
                    seen |= (unsigned)(bits >> (j0 & 31)) & below(end - tv) & ~below(-j0);
                }
                if (!live || !there) seen = 0;
#pragma unroll
                for (int i = 0; i < 16; ++i) if (!(seen >> i & 1)) p[i] = -__builtin_inff();
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
                for (int i = 0; i < 16; ++i) if (!(seen >> i & 1)) p[i] = 0.f;
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
                for (int ct = 0; ct < CT; ++ct) o[ct] *= turn;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) p[i] = __builtin_amdgcn_ldexpf(p[i], up);
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
            for (int ct = 0; ct < CT; ++ct) {
                const h8 v0 = levels8(vr[ct][0], vr[ct][1], zo[0], zo[1], zo[2], zo[3]), v1 = levels8(vr[ct][2], vr[ct][3], zo[4], zo[5], zo[6], zo[7]);
                o[ct] = mma16(v0, ph[0][0], o[ct]); o[ct] = mma16(v1, ph[0][1], o[ct]);
                o[ct] = mma16(v0, ph[1][0], o[ct]); o[ct] = mma16(v1, ph[1][1], o[ct]);
            }
        }
        l += from_xor<16>(l); l += from_xor<32>(l);
        if (l != l) m = fmaxf(m, 0.f);      // scores that are all NaN leave the maximum where it was: the row has seen something
        if (grp == 0) ends[wave][col] = make_float2(m, l);
        __syncthreads();
        const bool whole = step0 == 0 && step1 == c.steps;
        const long long piece = (2LL * blockIdx.x + (step0 == 0)) * a.piece_rows;
        float top = -__builtin_inff(), sum = 0.f;
        for (int w = rg; w < 4; w += c.wr) top = fmaxf(top, ends[w][col].x);
        for (int w = rg; w < 4; w += c.wr) if (ends[w][col].x != -__builtin_inff()) sum += ends[w][col].y * ex2(ends[w][col].x - top);
        const float f = m == -__builtin_inff() ? 0.f : ex2(m - top) / sum;      // (averages from here on: weighted sums of the largest values leave fp32)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) *(f4*)&joined[wave][col][ct * 16 + grp * 4] = m == -__builtin_inff() ? f4{0.f, 0.f, 0.f, 0.f} : by_power(o[ct] * f, -up);
        if (!whole && grp == 0 && group == 0 && rg * RW + col < n_rows) a.stat[piece + rg * RW + col] = make_float2(top, sum);
        __syncthreads();
        if (threadIdx.x == 0 && step0 == 0 && !whole) a.info[blockIdx.x] = make_int4((int)((at + c.steps - 1) / share) - (int)blockIdx.x + 1, s.start, r0 / 16 | (n_rows - 1) << 23, h);
        for (int i = threadIdx.x; i < n_rows * (DP / 4); i += 256) {
            const int rr = i / (DP / 4), ch = i % (DP / 4) * 4;
            f4 v = {0.f, 0.f, 0.f, 0.f};
            for (int w = rr / RW; w < 4; w += c.wr) v += *(const f4*)&joined[w][rr % RW][ch];
            if (whole) {
                const int row = r0 + rr, tk = row / a.rep;
                T* out = (T*)a.O + (long long)(s.start + tk) * a.ldo + (long long)(h * a.rep + row - tk * a.rep) * a.g.dh;
                store4(out, ch, a, v);
            } else *(f4*)(a.part + (piece + rr) * DP + ch) = v;
        }
        at += step1 - step0;
        if (at < at_end) __syncthreads();      // (what is in LDS has been read)
    }
}

// Rows of a unit that lies in several shares: averages O_i weighted with 2^(max_i - max) sum_i, over the weights' sum; a wavefront per row of the unit that begins in share blockIdx.x.
template <typename T, int DP>
__global__ __launch_bounds__(256) void kv_tree_join_kernel(AttendArgs a) {
    constexpr int LANES = DP / 4, GROUPS = 64 / LANES;
    const int4 info = a.info[blockIdx.x];
    const int pieces = min(info.x, (int)(gridDim.x - blockIdx.x)), r0 = (info.z & ((1 << 23) - 1)) * 16, n_rows = (int)((unsigned)info.z >> 23) + 1, h = info.w;
    const int lane = threadIdx.x & 63, ch = 4 * (lane % LANES), group = lane / LANES;
    if (pieces < 1) return;
    for (int rr = blockIdx.y * 4 + (threadIdx.x >> 6); rr < n_rows; rr += 4 * gridDim.y) {
        auto place = [&](int i) { return (2LL * (blockIdx.x + i) + (i == 0)) * a.piece_rows + rr; };
        f4 v = {0.f, 0.f, 0.f, 0.f};
        float top = -__builtin_inff(), sum = 0.f;
        for (int i0 = 0; i0 < pieces; i0 += 64) {
            const float2 st = i0 + lane < pieces ? a.stat[place(i0 + lane)] : make_float2(-__builtin_inff(), 0.f);
            const int n = min(pieces - i0, 64);
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
#pragma unroll 4
            for (int k = 0; k < n; k += GROUPS) {
                const int i = k + group;
                const float w = __shfl(f, min(i, 63), 64);
                if (group < GROUPS && i < n) v += w * *(const f4*)(a.part + place(i0 + i) * DP + ch);
            }
        }
        f4 all = v;
#pragma unroll
        for (int g = 1; g < GROUPS; ++g)
#pragma unroll
            for (int j = 0; j < 4; ++j) all[j] += __shfl(v[j], min(lane % LANES + g * LANES, 63), 64);
        if (group == 0) {
            const int row = r0 + rr, tk = row / a.rep;
            T* out = (T*)a.O + (long long)(info.y + tk) * a.ldo + (long long)(h * a.rep + row - tk * a.rep) * a.g.dh;
            store4(out, ch, a, all);
        }
    }
}

int piece_rows(long long rows) { return rows <= RW ? RW : rows <= 2 * RW ? 2 * RW : 4 * RW; }
int shares(const KvGeometry& g) { return 256 * (g.dp <= 128 ? 2 : 1); }
// Rows of a bf16 sequence up to which it is this kernel's; with more the kernel for many rows of kv_attention.hip takes it, whose eight wavefronts share the levels that it makes into half.  Both, joins and
// launches included, us, this one and the one for many rows:
//     one tree behind 8000, 64 / 8 heads of 128: 128 rows 44 73, 256 52 124, 512 73 93, 1024 133 110, 2048 229 143;   16 of up to: 128 148 192, 256 229 214, 512 411 471;   8 behind 4000 of up to 2048: 496 428
//     16 trees behind 4000, 16 heads of 64: 100 rows 104 196, 128 114 196;   4 of up to 1000 behind 1000: 145 176;   4 behind 4000, 16 / 2 heads of 256: 256 rows 54 82
constexpr int FEW = 512;
size_t room(const KvGeometry& g, int rows_of_piece, bool tiles, AttendArgs* a, void* ws) {
    const size_t n = (size_t)shares(g);
    Arena ar(ws);
    float* part = ar.get<float>(2 * n * rows_of_piece * g.dp);
    float2* stat = ar.get<float2>(2 * n * rows_of_piece);
    int4* info = ar.get<int4>(n);
    if (a) { a->part = part; a->stat = stat; a->info = info; a->piece_rows = rows_of_piece; }
    return ar.off + (tiles ? kv_tree_tiles_room(g, a, a ? (char*)ws + ar.off : nullptr) : 0);
}

template <typename T, int DP>
int launch_heads(tboa_ctx* ctx, const AttendArgs& a) {
    hipLaunchKernelGGL((kv_tree_kernel<T, DP>), dim3(256 * resident<DP>()), dim3(256), 0, ctx->stream, a);
    TB_KERNEL_CHECK(ctx);
    hipLaunchKernelGGL((kv_tree_join_kernel<T, DP>), dim3(256 * resident<DP>(), std::min(a.piece_rows / 4, 16)), dim3(256), 0, ctx->stream, a);
    TB_KERNEL_CHECK(ctx);
    return 0;
}
template <typename T>
int launch(tboa_ctx* ctx, const AttendArgs& a) {
    switch (a.g.dp) {
        case 32: return launch_heads<T, 32>(ctx, a);
        case 64: return launch_heads<T, 64>(ctx, a);
        case 96: return launch_heads<T, 96>(ctx, a);
        case 128: return launch_heads<T, 128>(ctx, a);
        case 192: return launch_heads<T, 192>(ctx, a);
        default: return launch_heads<T, 256>(ctx, a);
    }
}

}  // namespace

extern "C" size_t tboa_kv_cache_tree_attention_workspace_bytes(const tboa_kv_cache_desc* desc, int n_q_heads, int n_seqs, int64_t n_tokens) {
    KvGeometry g;
    if (!kv_geometry(desc, g) || n_q_heads <= 0 || n_q_heads > 65535 || n_q_heads % g.heads || n_seqs < 0 || n_seqs > 1 << 20 || n_tokens < 0 || n_tokens > 1 << 24) return 0;
    if (n_seqs == 0 || n_tokens == 0) return 0;
    const long long rows = n_tokens * (n_q_heads / g.heads);
    return room(g, piece_rows(rows), rows > FEW, nullptr, nullptr);      // (fp32: without the second part)
}

extern "C" int tboa_kv_cache_tree_attention(tboa_ctx* ctx, const tboa_kv_cache_desc* desc, const tboa_kv_batch* batch, int n_q_heads, int dtype, const void* Q, int64_t ldq,
                                            const uint32_t* tree, int tree_words, const void* cache, double scale, int window, void* O, int64_t ldo) {
    if (!ctx) return TBOA_EINVAL;
    KvGeometry g;
    TB_TRY(kv_check(ctx, "kv_cache_tree_attention", desc, batch, cache, g));
    if (dtype != TBOA_F32 && dtype != TBOA_BF16) return tboa_fail(ctx, TBOA_EINVAL, "kv_cache_tree_attention: dtype must be fp32 or bf16");
    if (n_q_heads <= 0 || n_q_heads > 65535 || n_q_heads % g.heads) return tboa_fail(ctx, TBOA_EINVAL, "kv_cache_tree_attention: %d query heads for %d KV heads", n_q_heads, g.heads);
    if (!(scale >= 0.0 && scale <= 1e30) || window < 0) return tboa_fail(ctx, TBOA_EINVAL, "kv_cache_tree_attention: scale=%g window=%d", scale, window);
    if (tree_words < 1 || tree_words > 1024) return tboa_fail(ctx, TBOA_EINVAL, "kv_cache_tree_attention: masks of 1 .. 1024 words, not %d", tree_words);
    if (batch->max_new > 32 * tree_words) return tboa_fail(ctx, TBOA_EINVAL, "kv_cache_tree_attention: masks of %d words for %d drafted tokens", tree_words, batch->max_new);
    if (batch->n_seqs == 0 || batch->n_tokens == 0) return 0;
    if (batch->pages_per_seq == 0 || g.n_pages == 0) return tboa_fail(ctx, TBOA_EINVAL, "kv_cache_tree_attention: no pages");
    if (!Q || !O || !tree) return tboa_fail(ctx, TBOA_EINVAL, "kv_cache_tree_attention: null argument");
    if (ldq < (int64_t)n_q_heads * g.dh || ldo < (int64_t)n_q_heads * g.dh) return tboa_fail(ctx, TBOA_EINVAL, "kv_cache_tree_attention: a row pitch is smaller than its heads");
    const int rep = n_q_heads / g.heads, size = dtype == TBOA_F32 ? 4 : 2;
    if (batch->n_tokens * rep >= 1LL << 27) return tboa_fail(ctx, TBOA_EINVAL, "kv_cache_tree_attention: too many rows");
    KvDevice dev(ctx->device);
    const long long rows = (batch->max_new > 0 ? std::min<long long>(batch->max_new, batch->n_tokens) : batch->n_tokens) * rep;
    const int of_piece = piece_rows(rows);
    const bool tiles = dtype == TBOA_BF16 && rows > FEW && kv_tree_tiles_takes(g, batch->n_seqs, batch->n_tokens, rep);
    TB_TRY(tboa_ws_reserve(ctx, room(g, of_piece, tiles, nullptr, nullptr)));
    AttendArgs a{};
    a.g = g;
    a.q = KvBatch{batch->n_seqs, batch->pages_per_seq, (int)batch->n_tokens, batch->pages_per_seq * desc->page_tokens, batch->starts, batch->lens, batch->pages};
    a.Q = Q; a.ldq = ldq; a.O = O; a.ldo = ldo; a.cache = (const unsigned char*)cache;
    a.scale2 = (float)((scale == 0.0 ? 1.0 / sqrt((double)g.dh) : scale) * 1.4426950408889634);
    a.rep = rep; a.window = window < KV_MOST_TOKENS ? window : 0;      // (no sequence is longer)
    a.vec = g.dh % 8 == 0 && ((uintptr_t)Q & 15) == 0 && ldq * size % 16 == 0 ? 8 : g.dh % 4 == 0 && ldq % 4 == 0 && ((uintptr_t)Q & (4 * size - 1)) == 0 ? 4 : 0;
    a.out_piece = g.dh % 8 == 0 && ldo % 8 == 0 && ((uintptr_t)O & 15) == 0 ? 8 : g.dh % 4 == 0 && ldo % 4 == 0 && ((uintptr_t)O & (4 * size - 1)) == 0 ? 4 : 1;
    a.tree = tree; a.tree_words = tree_words;
    const bool all = tiles && batch->n_seqs == 1;      // one sequence: whatever its rows, one kernel
    a.few = all ? 0 : tiles ? FEW : 1 << 30;
    room(g, of_piece, tiles, &a, ctx->ws);
    if (tiles) TB_TRY(kv_tree_tiles(ctx, a));
    if (all) return 0;
    return dtype == TBOA_F32 ? launch<float>(ctx, a) : launch<bf16>(ctx, a);
}
