// Quantized key/value cache: geometry, and how a workgroup finds its part of a ragged batch.
#pragma once
#include "internal.h"

// A page holds 2^pt_log tokens of all heads: levels of K [head][token][dp], of V [head][token / 16][dp][token % 16], grids of K, of V [head][block of 2^st_log tokens][scale, zero].
// K by token and V by channel, 16 tokens together: what one lane of a 16 x 16 x 32 or 32 x 32 x 16 matrix instruction takes as its left operand of K Q^T and V^T P^T are consecutive
// bytes of either, so that nothing is transposed when the cache is read.
struct KvGeometry {
    int heads, dh, dp, pt_log, st_log;
    long long n_pages, page_bytes, v_at, kg_at, vg_at;      // offsets within a page
};
static inline int kv_padded_head(int dh) { return dh <= 32 ? 32 : dh <= 64 ? 64 : dh <= 96 ? 96 : dh <= 128 ? 128 : dh <= 192 ? 192 : 256; }
bool kv_geometry(const tboa_kv_cache_desc* d, KvGeometry& g);
int kv_check(tboa_ctx* ctx, const char* who, const tboa_kv_cache_desc* d, const tboa_kv_batch* b, const void* cache, KvGeometry& g);
// the context's device is current while a call runs, and the caller's is again after it
struct KvDevice {
    int before = -1, now = -1;
    explicit KvDevice(int device) { if (hipGetDevice(&before) == hipSuccess && before != device && hipSetDevice(device) == hipSuccess) now = device; }
    ~KvDevice() { if (now >= 0) (void)hipSetDevice(before); }
};

constexpr int KV_MOST_TOKENS = 1 << 30;      // of a sequence
struct KvBatch { int n_seqs, per_seq, n_tokens, room; const int *starts, *lens, *pages; };      // room: tokens that a row of `pages` stands for

struct KvSeq { int start, n, len; };      // first row of the new tokens, their number, tokens in the cache with them
__device__ __forceinline__ KvSeq kv_sequence(const KvBatch& q, int b) {
    const int a = min(max(q.starts[b], 0), q.n_tokens), e = min(max(q.starts[b + 1], a), q.n_tokens);
    return KvSeq{a, e - a, min(max(q.lens[b], 0), KV_MOST_TOKENS)};
}

__device__ __forceinline__ KvSeq kv_head(const KvBatch& q) { const int lane = threadIdx.x & 63; return lane < q.n_seqs ? kv_sequence(q, lane) : KvSeq{0, 0, 0}; }

// Item x of a list in which sequence b has count(sequence) items: its sequence, and x becomes the number within it.  Every wavefront finds its own, 64 sequences at a time.
// `head`: sequence threadIdx.x % 64, which the caller may have read already.
template <typename N, typename Count>
__device__ __forceinline__ bool kv_find(const KvBatch& q, const KvSeq& head, Count count, N& x, int& b, KvSeq& s) {
    const int lane = threadIdx.x & 63;
    for (int base = 0; base < q.n_seqs; base += 64) {
        KvSeq mine{0, 0, 0};
        N c = 0;
        if (base + lane < q.n_seqs) { mine = base ? kv_sequence(q, base + lane) : head; c = count(mine); }
        N sum = c;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) { const N v = __shfl_up(sum, o, 64); if (lane >= o) sum += v; }
        const unsigned long long past = __ballot(sum > x);
        if (past) {
            const int at = __builtin_ctzll(past);
            b = base + at;
            x -= __shfl(sum - c, at, 64);
            s = KvSeq{__builtin_amdgcn_readlane(mine.start, at), __builtin_amdgcn_readlane(mine.n, at), __builtin_amdgcn_readlane(mine.len, at)};
            return true;
        }
        x -= __shfl(sum, 63, 64);
    }
    return false;
}
