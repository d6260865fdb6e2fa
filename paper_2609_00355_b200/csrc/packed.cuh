// The 4-bit cache format: layout of a tile, and the conversions that kernels share.
//
// A tile is what one (layer, page, kv head) holds: K codes [64][d/2], K scales [64][d/16], V codes, V scales, 4.5 bits a
// value (9216 bytes at d 128, 4608 at d 64; a multiple of 16, so one bulk copy fetches it).  A code is e2m1 (sign, two
// exponent bits, one mantissa bit), a scale e4m3, value = scale * code: at most 2 + 4 significant bits, so the product is exact
// in bf16 and in fp16 (|value| <= 448 * 6, and the smallest that is not zero is 2^-10).
// Codes of a key are in order, eight to a word; the 16-byte pieces of a row are exchanged by key (code_at), so that eight keys
// read side by side meet no bank of shared memory twice.
#pragma once
#include <cuda_fp16.h>

#include "common.cuh"

namespace glance {
namespace packed {

constexpr int kGroup = 16;       // values along the head dimension that share a scale

template <int D>
struct Tile {
    static constexpr int ROW = D / 2;                        // bytes of a key's codes
    static constexpr int GROUPS = D / kGroup;
    static constexpr int SCALES = kPage * ROW;               // scales of K or V behind the codes
    static constexpr int HALF = kPage * (ROW + GROUPS);      // K, then V
    static constexpr int BYTES = 2 * HALF;
    static_assert(BYTES % 16 == 0 && HALF % 16 == 0 && SCALES % 16 == 0, "bulk copies");
};

__host__ __device__ inline int tile_bytes(int d) { return 2 * kPage * (d / 2 + d / kGroup); }

// byte offset of 16-byte piece c of key `key`'s codes
template <int D>
__device__ __forceinline__ int code_at(int key, int c) {
    if constexpr (D == 128) return key * 64 + ((c ^ ((key >> 1) & 3)) << 4);
    else return key * 32 + ((c ^ ((key >> 2) & 1)) << 4);
}

// eight codes of a word -> four fp16 pairs (even code in the low half); exact
__device__ __forceinline__ void codes_to_half(uint32_t w, uint32_t (&h)[4]) {
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
}
// two e4m3 scales -> an fp16 pair; exact
__device__ __forceinline__ uint32_t scales_to_half(uint32_t two) {
    uint32_t h;
    asm("{\n\t.reg .b16 x;\n\tcvt.u16.u32 x, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, x;\n\t}" : "=r"(h) : "r"(two));
    return h;
}
__device__ __forceinline__ uint32_t mul_half2(uint32_t a, uint32_t b) {
    uint32_t c;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(c) : "r"(a), "r"(b));
    return c;
}
// an fp16 pair as a bf16 pair (exact for values of this format)
__device__ __forceinline__ uint32_t half2_to_bf16(uint32_t h) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h));
    const __nv_bfloat162 b = __floats2bfloat162_rn(f.x, f.y);
    return *reinterpret_cast<const uint32_t *>(&b);
}

}  // namespace packed

// ---- where a row looks: sliding window, sinks, trees (attention over a cache that is not read whole) ----------------
// Positions of a sequence.  A length beyond the page table counts as one that fills it: the lists stay in 32 bits, and the page
// behind the table's last entry, which the new rows need, is reported.
__device__ __forceinline__ int positions(int seq_len, const KvGeom &g) { return min(max(seq_len, 0), g.max_pages_per_seq * kPage); }

// The pages that any row of a tile sees, as one list: pages [0, head), then pages [next, end).
struct PageList {
    int head, next, count;       // page of entry v: v < head ? v : v - head + next
    __device__ __forceinline__ int page(int v) const { return v < head ? v : v - head + next; }
};
// n_keys positions; the tile's rows see position p if p < sinks or p >= low (low <= 0: all)
__device__ __forceinline__ PageList page_list(int n_keys, int low, int sinks) {
    PageList l;
    const int end = (n_keys + kPage - 1) / kPage;
    l.next = max(low, 0) / kPage;
    l.head = (min(sinks, n_keys) + kPage - 1) / kPage;
    if (l.head >= l.next) l.head = l.next = 0;
    l.count = l.head + end - l.next;
    return l;
}

// What row `node` of a sequence sees: committed position p < P if p < sinks or p >= low; row j if bit j of `bits` is set (only
// where the rows are at most 128).
struct RowSight {
    int low;
    uint64_t bits[2];
};
__device__ __forceinline__ uint64_t bits_from(int n) { return n <= 0 ? ~0ull : n >= 64 ? 0ull : ~0ull << n; }   // bits n..63
__device__ __forceinline__ uint64_t bits_below(int n) { return ~bits_from(n); }                                  // bits 0..n-1

__device__ __forceinline__ int window_low(int at, int window) {      // first position inside the window of a row at position `at`
    return window > 0 ? (int)max((long long)at - window + 1, -(1ll << 30)) : -(1 << 30);
}

__device__ inline RowSight row_sight(const uint64_t *anc, int causal, int node, int T, int P, int window, int sinks) {
    RowSight r;
    const int keep = (int)min((long long)max(sinks - P, 0), 256ll);  // rows at the first `keep` positions stay visible
    if (!anc) {                                                     // block or chain: row j at position P + j
        r.low = window_low(P + node, window);
        const int last = causal ? min(node + 1, T) : T;             // rows 0..last-1
        const int lo = window > 0 ? max(node - window + 1, 0) : 0;
#pragma unroll
        for (int w = 0; w < 2; ++w)
            r.bits[w] = (bits_from(lo - 64 * w) | bits_below(keep - 64 * w)) & bits_below(last - 64 * w);
        return r;
    }
    const int W = (T + 63) / 64;
    const uint64_t *a = anc + (size_t)node * W;
    r.bits[0] = a[0] & bits_below(T);
    r.bits[1] = W > 1 ? a[1] & bits_below(T - 64) : 0ull;
    const int n = __popcll(r.bits[0]) + __popcll(r.bits[1]);
    r.low = window_low(P + max(n - 1, 0), window);
    if (window > 0 && window < n) {
        // the set's nodes in order are a path: all but the last `window` and the first `keep` leave
        int drop = n - window, skip = min(keep, n - window);
        drop -= skip;
        uint64_t kept[2] = {0ull, 0ull};
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            while (r.bits[w] && (skip > 0 || drop > 0)) {
                const uint64_t low_bit = r.bits[w] & (~r.bits[w] + 1ull);
                r.bits[w] ^= low_bit;
                if (skip > 0) { kept[w] |= low_bit; --skip; }
                else --drop;
            }
            r.bits[w] |= kept[w];
        }
    }
    return r;
}

// Whether a row sees anything.  One that does and has no weight has scores that are all -inf (an infinite query's): its outputs are
// NaN, the definition's 0 / 0, where those of a row that sees nothing are zeros.
__device__ __forceinline__ bool row_sees(const RowSight &r, int P, int sinks) {
    return (r.bits[0] | r.bits[1]) != 0ull || (P > 0 && (sinks > 0 || r.low < P));
}

}  // namespace glance
