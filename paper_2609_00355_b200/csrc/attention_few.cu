// Attention of few query rows (single tokens, short blocks and trees) over a long paged cache that is read in part (sliding
// window, sinks) or held in 4 bits: bound by the bytes of the cache, so everything is laid out around streaming them once.
//
// The pages that a launch has to read form one line: sequences, in each its kv heads, in each the pages that some row sees
// (packed.cuh).  The line is dealt out in stretches of equal cost to one CTA an SM, so ragged batches and long single
// sequences keep the whole GPU reading; a CTA finds its stretch from the device-resident lengths by one prefix sum.  Teams of four warps
// take its pages in turn, a warp 16 of a page's 64 keys, and nobody waits for another inside an item; a team's producer warp
// fetches its pages into its ring (bf16: tensor copies; 4 bits: one bulk copy of a 4.5-bit tile).
//     S^T[16 keys x 8 rows] = K Q^T,   O^T[d x 8 rows] += V^T P^T     (mma.sync m16n8k16, fp32 accumulators)
// Keys sit in the M dimension, so one token's 7 or 8 heads fill an instruction's N exactly; with rows in M half of it
// would idle, and 128-row tcgen05 tiles would run at 6 % and wait for their tensor memory round trips.  At 8 rows a page
// takes 128 to 250 clocks of mma against 1400 (bf16) or 400 (4 bits) of its share of HBM.
// 4-bit pages go from shared memory to registers in the order in which the mma wants them (16 consecutive d of a key per
// lane; the contraction order is free as long as Q has the same), fp16: code x scale is exact there, and fp16 has the
// conversion.  A row's queries are scaled by a power of two so that the largest lies in [1, 2): bf16 elements down to 2^-17 of it
// keep all their bits, smaller ones are rounded to multiples of 2^-24.  P is one fp16 term (half a step: 2^-11 relative; outputs
// then differ from those of an fp32 P by 7 to 9 x 10^-4 of their norm, half of what their own rounding to bf16 makes it, 1.7 x 10^-3),
// two where the caller has two-term queries (16 rows over 4096-32768 positions 45 -> 53 us).  bf16 pages stay bf16: Q as it
// is, P in two bf16 terms (one would cost 2^-8).
// A row's reference is raised only when a score exceeds the largest so far by 2^8; sums and accumulators are fp32.
// The warps' partial results meet in shared memory; an item that several CTAs share is finished by the one that comes last,
// which adds the parts in line order, or by its cluster through distributed shared memory: results do not depend on timing.
// Measured (us): 16 rows of 7 heads over 4096-32768 positions in 4 bits, 160 MB, 44.9 (3.6 TB/s); over 8192 positions in bf16,
// 268 MB, 50.7 (5.3 TB/s); one row over 32801 positions in 4 bits 14.9, of which 5.5 are the merge of 37 parts; one row over a
// window of 512 7.0.  In 4 bits the bound is the chain of a page in its warp (1300 clocks: first products 450, softmax 200,
// second products 620), of which 12 warps keep three pages going; variants without the conversions, the mma or V's products
// saved next to nothing.
#include <algorithm>
#include <type_traits>

#include "answers.h"
#include "kernels.cuh"
#include "packed.cuh"
#include "tc_ptx.cuh"

namespace glance {

namespace {

using namespace tc;
using namespace packed;

constexpr int kTeam = 4;                     // consumer warps that share a page, 16 keys each
constexpr int kMaxSeqs = 64;
constexpr float kRaise = 8.f;                // log2 units a score may exceed its reference by
constexpr float kHead = 7.f;                 // and the reference lies this far below the largest: fp16 probabilities reach from 2^15 down
                                             // to 2^-14 at full precision, 2^-21 of the largest
// Pages, in 4 bits and in bf16, that an item's end and the next one's start are worth (see the kernel).  Batches of 5, 16 and 40
// ragged sequences at d 64 and 128: in 4 bits 8 places are 0 to 10 % slower than 24, 40 places 0 to 5 %; in bf16 none are 1 to 17 %
// slower than 4, 12 places 3 % faster on average (1 % slower to 6 % faster).
constexpr int kLead4 = 24, kLead16 = 4;
constexpr int kMaxCluster = 8;
// Pages a CTA may have more to be in a cluster (see launch_few).  One to four rows over 600 to 1500 positions take 0.9 to 2.2 us
// more with 0; with 8 single rows over 2100 to 4300 positions take 2.3 to 3.4 less, the others the same.
constexpr int kMorePages = 3;

// NB: blocks of 8 query rows.  As many teams as the registers of NB blocks' accumulators leave room for: a page's chain
// (codes, first products, softmax, second products) is long, and only other warps' pages hide it.
template <int D, int NB>
struct Few {
    static constexpr int TEAMS = NB == 1 ? 3 : 2;
    static constexpr int WARPS = TEAMS * kTeam;              // consumers; one more fetches
    static constexpr int THREADS = (WARPS + TEAMS) * 32;
    // A team has a ring of its own, filled by a warp of its own: places of a bf16 page (K and V, multiples of 1024 for the
    // swizzle) or of three 4-bit tiles in its thirds, the team's next ones.  Three at once, because a thread takes 240 ns to
    // wait for a place and to announce what it fetches, more than a 4-bit page's share of HBM, and 30 for a copy.
    static constexpr int PAGE_BYTES = 2 * kPage * D * 2;
    static constexpr int THIRD = PAGE_BYTES / 3 / 16 * 16;
    static constexpr int PLACES = 2;                         // a team
    static constexpr int RING = TEAMS * PLACES * PAGE_BYTES;
    static constexpr int ROWF = D + 4;
    static constexpr int QB = 8 * D * 2;                     // one term of 8 rows' queries
    static constexpr int Q_AT = RING;                        // [fp16 | bf16][term][NB] fragments
    static constexpr int RED_AT = Q_AT + 4 * NB * QB;        // [warp of a team][8][ROWF] partial outputs of 8 rows
    static constexpr int TOTAL = RED_AT + kTeam * 8 * ROWF * 4 + 1024;
    static_assert(PAGE_BYTES % 1024 == 0 && THIRD >= Tile<D>::BYTES, "ring");
    static_assert(TEAMS * NB <= kTeam, "the teams' sums of an item fit the partial outputs' place");
    static_assert(TOTAL + 4 * 1024 <= 227 * 1024, "with the static arrays: one CTA an SM");
};

// key of row r of a 16-key tile (r < 8; the other eight follow 8 later): eight keys that lanes read side by side differ in
// the bits that pick a bank, for the 4-bit tile's rows as for 128-byte swizzled ones
__device__ __forceinline__ int key_of(int r) { return (r & 1) ? 4 + ((r >> 1) ^ 1) : r >> 1; }

template <bool HALF>
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (HALF)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// the same without an accumulator to add to
template <bool HALF>
__device__ __forceinline__ void mma_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (HALF)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
            : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
            : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t (&a)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(a[0]), "=r"(a[1]), "=r"(a[2]), "=r"(a[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t addr, uint32_t (&a)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(a[0]), "=r"(a[1]), "=r"(a[2]), "=r"(a[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
template <bool HALF>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    uint32_t r;
    if constexpr (HALF) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
}
template <bool HALF>
__device__ __forceinline__ float2 unpack2(uint32_t v) {
    if constexpr (HALF) return __half22float2(*reinterpret_cast<const __half2 *>(&v));
    else return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}
__device__ __forceinline__ void bulk_load(void *dst, const void *src, uint32_t bytes, uint64_t *bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(smem_u32(dst)), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
}

template <int TEAMS, int PLACES>
struct alignas(8) FewBars {
    uint64_t full[TEAMS][PLACES], empty[TEAMS][PLACES];
    int abort_flag, last;
};

struct alignas(16) RowMask {
    uint32_t bits[4];
    int low;
    float scale16;               // score scale in log2 units for the fp16 queries of this row
    int sees;                    // whether it sees anything
    int pad;
};

// The accumulators of a warp's 8 query rows from the 4-bit pages' order of d (lane g, register i: d = (D/8) g + i) to the mma's
// own (block mb, half e: 16 mb + 8 e + g): lane bits and register bits change places, one exchange of half the registers each.
template <int D>
__device__ __forceinline__ void reorder(float (&O)[D / 16][4], int g) {
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        float v[D / 8];
#pragma unroll
        for (int i = 0; i < D / 8; ++i) v[i] = O[i >> 1][(i & 1) * 2 + n];
#pragma unroll
        for (int bit = 0; bit < 3; ++bit) {
            const bool up = (g >> bit) & 1;
#pragma unroll
            for (int i = 0; i < D / 8; ++i)
                if (!((i >> bit) & 1)) {
                    const int j = i | 1 << bit;
                    const float got = __shfl_xor_sync(0xffffffffu, up ? v[i] : v[j], 4 << bit);
                    if (up) v[i] = got;
                    else v[j] = got;
                }
        }
        // register bits now: the lowest three are the lane's old ones
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
            if constexpr (D == 128) O[i & 7][(i >> 3) * 2 + n] = v[i];
            else O[i >> 1][(i & 1) * 2 + n] = v[i];
        }
    }
}

// What a lane keeps of its two query rows (2t, 2t + 1): the reference maximum (0 while the row has seen nothing), the score above
// which it is raised (-inf then), and its share of the row sum.  Log2 units.
struct RowState {
    float ref[2], limit[2], sum[2];
};

// One 16-key tile's softmax and the probabilities as the second product's B operand.  c: raw scores [key g | g + 8][rows 2t, 2t + 1],
// -inf where hidden; s: scale of each row.  True if a row's reference was raised: then everything summed so far takes the factor f.
template <bool HALF, bool TWO>
__device__ __forceinline__ bool softmax_tile(float (&c)[4], RowState &st, float s0, float s1, uint32_t (&b)[2], uint32_t (&blo)[2], float (&f)[2]) {
    float x0 = fmaxf(c[0], c[2]) * s0, x1 = fmaxf(c[1], c[3]) * s1;
    const bool raise = __any_sync(0xffffffffu, x0 > st.limit[0] || x1 > st.limit[1]);
    if (raise) {
#pragma unroll
        for (int o = 4; o <= 16; o <<= 1) {
            x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, o));
            x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, o));
        }
        f[0] = f[1] = 1.f;
        if (x0 > st.limit[0]) {
            f[0] = st.limit[0] == -INFINITY ? 0.f : ex2(st.ref[0] - (x0 - kHead));
            st.ref[0] = x0 - kHead;
            st.limit[0] = x0 + kRaise;
        }
        if (x1 > st.limit[1]) {
            f[1] = st.limit[1] == -INFINITY ? 0.f : ex2(st.ref[1] - (x1 - kHead));
            st.ref[1] = x1 - kHead;
            st.limit[1] = x1 + kRaise;
        }
        st.sum[0] *= f[0];
        st.sum[1] *= f[1];
    }
    c[0] = ex2(fmaf(c[0], s0, -st.ref[0]));
    c[1] = ex2(fmaf(c[1], s1, -st.ref[1]));
    c[2] = ex2(fmaf(c[2], s0, -st.ref[0]));
    c[3] = ex2(fmaf(c[3], s1, -st.ref[1]));
    st.sum[0] += c[0] + c[2];
    st.sum[1] += c[1] + c[3];
    const uint32_t h0 = pack2<HALF>(c[0], c[1]), h1 = pack2<HALF>(c[2], c[3]);
    b[0] = transpose8(h0);
    b[1] = transpose8(h1);
    if constexpr (TWO) {
        const float2 v0 = unpack2<HALF>(h0), v1 = unpack2<HALF>(h1);
        blo[0] = transpose8(pack2<HALF>(c[0] - v0.x, c[1] - v0.y));
        blo[1] = transpose8(pack2<HALF>(c[2] - v1.x, c[3] - v1.y));
    }
    return raise;
}

// shared-memory loads by address, so that a page's loads differ in their immediate offsets only
__device__ __forceinline__ uint4 lds16(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint2 lds8(uint32_t a) {
    uint2 v;
    asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t lds4(uint32_t a) {
    uint32_t v;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t lds2(uint32_t a) {
    uint32_t v;
    asm volatile("ld.shared.u16 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t lds1(uint32_t a) {
    uint32_t v;
    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}

// TWO: queries (and outputs) in two bf16 terms, and then probabilities of 4-bit pages in two fp16 terms
template <int D, int NB, bool TWO>
__global__ void __launch_bounds__(Few<D, NB>::THREADS, 1) attn_few_kernel(const __grid_constant__ CUtensorMap map_kv, AttnParams p) {
    using F = Few<D, NB>;
    constexpr int KS = D / 16, MB = D / 16, kWarps = F::WARPS;
    constexpr int CH = 2;                                    // independent sums of the first product (its chain of mma would wait for itself)
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);       // (an offset: the pointer stays a shared one)
    unsigned char *sQ = smem + F::Q_AT;
    float *red = reinterpret_cast<float *>(smem + F::RED_AT);
    __shared__ FewBars<F::TEAMS, F::PLACES> bars;
    __shared__ int upto[kMaxSeqs + 1];                       // pages (of all heads) of the sequences before
    __shared__ int lens[kMaxSeqs], helds[kMaxSeqs];          // positions; pages held in 4 bits
    __shared__ int most_pages[32];                           // of a (sequence, kv head)
    __shared__ float sum_m[8 * NB], sum_l[8 * NB];           // clusters: this CTA's part of its item (the outputs: in `red`)
    __shared__ RowMask mask[8 * NB];
    __shared__ int pages[F::TEAMS][64];
    __shared__ float red_m[kWarps][8 * NB], red_l[kWarps][8 * NB];

    // test hook: phases of the first CTA (entry, set up, predecessor done, queries staged, first page there, pages done, warps
    // merged, part handed over, end), and the grid's span
    unsigned long long *trace = p.trace && blockIdx.x == 0 && threadIdx.x == 0 ? p.trace : nullptr;
    if (trace) trace[0] = global_ns();
    if (p.trace && threadIdx.x == 0) atomicMin(p.trace + 14, (unsigned long long)global_ns());
    pdl_launch_dependents();
    static_assert(NB <= kTeam, "the teams' sums of an item fit the warps' places");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int G = p.Hq / p.Hkv, PR = p.T * G;
    volatile int *abort_flag = &bars.abort_flag;
    auto list_of = [&](int P) { return page_list(P + p.T, window_low(P, p.window), p.sinks); };
    if (warp == 0) {
        for (int i = lane; i < F::TEAMS * F::PLACES; i += 32) {
            mbar_init(&bars.full[0][0] + i, 1);
            mbar_init(&bars.empty[0][0] + i, kTeam);
        }
        if (lane == 0) bars.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x < 8 * NB) {
        sum_m[threadIdx.x] = -INFINITY;
        sum_l[threadIdx.x] = -1.f;                           // no pages yet
    }
    if (!p.early) pdl_wait();
    if (warp == 1) {
        // (inside a pass lengths may be read before the dependency wait: see attention_tc.cu)
        int run = 0, most = 0;
        for (int s0 = 0; s0 < p.batch; s0 += 32) {
            int n = 0;
            if (s0 + lane < p.batch) {
                const int P = positions(p.seq_len[s0 + lane], p.geom);
                const int h = p.held_len ? min(max(p.held_len[s0 + lane], 0), P) / kPage : 0;
                lens[s0 + lane] = P;
                helds[s0 + lane] = h;
                n = list_of(P).count;
                most = max(most, n);
                n *= p.Hkv;
            }
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, n, o);
                if (lane >= o) n += v;
            }
            if (s0 + lane < p.batch) upto[s0 + lane + 1] = run + n;
            run += __shfl_sync(0xffffffffu, n, 31);
        }
        most_pages[lane] = most;
        if (lane == 0) upto[0] = 0;
    }
    __syncthreads();
    // ---- this CTA's stretch of the line: with clusters, a share of its cluster's item ((sequence, kv head)).  Else the same number of
    // CTAs for every item, so that a CTA has one item to start and to finish, unless equal stretches, which may begin and end
    // inside an item, end earlier.  To finish an item and start the next takes a CTA as long as `lead` pages, so on the line every
    // item begins with that many places without a page (16 rows over 4096-32768 positions in 4 bits: without them CTAs with
    // one item ended after 37 us, those with two after 47; whole launch 49.4; with 24 places 44.9, 16 and 32 1.3 and 0.4 more) ----
    int chunk, lead = 0, s, kvh, pos, places;                // the first item's place to begin with (lead first); places of the stretch
    {
        const int items = p.batch * p.Hkv, grid = (int)gridDim.x, total = upto[p.batch];
        int per_item = p.S;
        if (p.S == 0) {
            int most = most_pages[lane];
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
            per_item = grid / items;
            lead = min(p.held_len ? kLead4 : kLead16, (total + grid - 1) / grid / 2);
            if (per_item > 0 && (most + per_item - 1) / per_item <= (total + lead * items + grid - 1) / grid) lead = 0;
            else per_item = 0;
        }
        if (per_item > 0) {
            const int item = (int)blockIdx.x / per_item;
            s = min(item / p.Hkv, p.batch - 1);
            kvh = item - s * p.Hkv;
            const int n = list_of(lens[s]).count;
            chunk = (n + per_item - 1) / per_item;
            pos = ((int)blockIdx.x - item * per_item) * chunk;
            places = item < items ? min(chunk, n - pos) : 0;
        } else {
            const int line = total + items * lead;
            chunk = (line + grid - 1) / grid;
            const int x = (int)blockIdx.x * chunk;
            places = min(chunk, line - x);
            s = 0;
            while (s + 1 < p.batch && upto[s + 1] + (s + 1) * p.Hkv * lead <= x) ++s;
            const int n = list_of(lens[s]).count + lead;
            pos = x - upto[s] - s * p.Hkv * lead;
            kvh = pos / n;
            pos -= kvh * n;
        }
    }
    // the part of item (s, kvh) from pos on that lies in the stretch, of which `at` places are behind: entries [v0, v1) of its
    // list; and on to the next item, or the end of the stretch
    struct Part {
        int v0, v1, from;                                    // from: place of the item's first page, counted from the stretch's begin
    };
    int at = 0;
    auto next_part = [&](int count) {
        const int end = min(count + lead, pos + places - at);
        const Part part{max(pos - lead, 0), max(end - lead, 0), at + lead - pos};
        at += end - pos;
        return part;
    };
    auto next_item = [&]() {
        pos = 0;
        if (++kvh == p.Hkv) {
            kvh = 0;
            ++s;
        }
    };

    // Page i of the CTA's stretch belongs to team i % TEAMS.
    const int team = warp < kWarps ? warp / kTeam : warp - kWarps;
    unsigned char *ring = smem + team * F::PLACES * F::PAGE_BYTES;
    uint64_t *full = bars.full[team], *empty = bars.empty[team];
    int place = 0;                                           // of the team's ring: next to be filled or taken, and how often round
    uint32_t phase = 0u;
    auto advance = [&]() {
        if (++place == F::PLACES) {
            place = 0;
            phase ^= 1u;
        }
    };
    // entries of a stretch [v0, v1) of a list that are held in 4 bits: a prefix
    auto held_of = [](const PageList &list, int held, int v0, int v1) {
        return min(max(held <= list.head ? held : list.head + max(held - max(list.next, list.head), 0), v0), v1) - v0;
    };

    if (warp >= kWarps) {
        // ---------------- a team's producer: lane 0 issues; all lanes look up page numbers, 32 at a time and ahead ----------------
        bool waited = false, ok = true;
        int *numbers = pages[team];
        int done = 0;                                        // pages of the stretch so far
        for (; at < places && ok; next_item()) {
            const int P = lens[s], held = helds[s];
            const PageList list = list_of(P);
            const Part part = next_part(list.count);
            const int v0 = part.v0, v1 = part.v1;
            if (v0 == v1) continue;
            auto look_up = [&](int v) {                      // page of entry v in its pool
                if (v >= v1) return 0;
                const int pg = list.page(v);
                const size_t entry = (size_t)s * p.geom.max_pages_per_seq + pg;
                int page = -1;
                if (pg < p.geom.max_pages_per_seq) page = pg < held ? p.held_table[entry] : p.page_table[entry];
                if (page < 0 || page >= (pg < held ? p.held_pages : p.geom.n_pages)) {
                    page = 0;
                    set_status(p.status, GLANCE_E_BOUNDS);
                }
                return page;
            };
            const int first = v0 + (team + F::TEAMS - done % F::TEAMS) % F::TEAMS, v_held = v0 + held_of(list, held, v0, v1);
            // this team's page k is entry first + TEAMS k; numbers of 64 of them, 32 replaced at a time
            numbers[lane] = look_up(first + F::TEAMS * lane);
            numbers[32 + lane] = look_up(first + F::TEAMS * (32 + lane));
            __syncwarp();
            int k = 0, upto_k = 64;
            for (int v = first; v < v1;) {
                if (k + 32 >= upto_k) {                      // lane 0 is past the older half
                    __syncwarp();
                    numbers[(upto_k + lane) & 63] = look_up(first + F::TEAMS * (upto_k + lane));
                    upto_k += 32;
                    __syncwarp();
                }
                const int n = v < v_held ? min(3, (v_held - v + F::TEAMS - 1) / F::TEAMS) : 1;       // pages of this place
                if (lane == 0 && ok) {
                    const int last = list.page(v + (n - 1) * F::TEAMS);
                    if (!waited && (last + 1) * kPage > P - kMaxBlock) {    // rows that this pass may write
                        pdl_wait();
                        waited = true;
                    }
                    ok = mbar_wait(&empty[place], phase ^ 1u, abort_flag, p.status);
                    if (ok) {
                        unsigned char *dst = ring + place * F::PAGE_BYTES;
                        if (v < v_held) {
                            mbar_expect_tx(&full[place], (uint32_t)(n * Tile<D>::BYTES));
                            for (int c = 0; c < n; ++c)
                                bulk_load(dst + c * F::THIRD, p.held_layer + ((size_t)numbers[(k + c) & 63] * p.Hkv + kvh) * Tile<D>::BYTES,
                                          Tile<D>::BYTES, &full[place]);
                        } else {
                            mbar_expect_tx(&full[place], F::PAGE_BYTES);
#pragma unroll
                            for (int kv = 0; kv < 2; ++kv) {
                                const int row = ((numbers[k & 63] * 2 + kv) * p.Hkv + kvh) * kPage;
#pragma unroll
                                for (int sl = 0; sl < D / 64; ++sl)
                                    tma_load_2d(dst + (kv * (D / 64) + sl) * (kPage * 128), &map_kv, &full[place], sl * 64, row);
                            }
                        }
                        advance();
                    }
                }
                v += n * F::TEAMS;
                k += n;
            }
            ok = __shfl_sync(0xffffffffu, ok ? 1 : 0, 0) != 0;
            done += v1 - v0;
        }
        if (lane == 0) {
            if (!waited) pdl_wait();
            if (*abort_flag) {                               // copies already issued must land before the CTA may exit
                for (int i = 0; i < F::PLACES; ++i) {
                    // the latest use of place i: in this round of the ring if it lies before `place`, else in the last one
                    const uint64_t t0 = global_ns();
                    while (!mbar_try_wait(&full[i], i < place ? phase : phase ^ 1u))
                        if (global_ns() - t0 > kWaitLimitNs) break;
                }
            }
        }
        __syncwarp();
        if (p.S > 0) {                                       // the two barriers of the clusters' merge
            cluster_sync_all();
            cluster_sync_all();
        }
        return;
    }

    // ---------------- consumers ----------------
    if (trace) trace[1] = global_ns();
    pdl_wait();
    if (trace) trace[2] = global_ns();
    const int g = lane >> 2, t = lane & 3, tid = threadIdx.x;
    const float sl2 = rsqrtf((float)D) * 1.4426950408889634f;
    const int first_key = warp % kTeam * 16;
    const int kA = first_key + key_of(g);                    // this lane's keys as rows of K: kA, kA + 8
    const int kV0 = first_key + t, kV1 = first_key + 4 + (t ^ 1);      // and as columns of V^T: kV0, kV1, kV0 + 8, kV1 + 8
    bool ok = true;
    // the whole warp waits; false (from then on) if a wait gave up
    auto wait_all = [&](uint64_t *bar, uint32_t parity) {
        if (!__all_sync(0xffffffffu, ok && mbar_try_wait(bar, parity))) {
            ok = ok && mbar_wait(bar, parity, abort_flag, p.status);
            ok = __all_sync(0xffffffffu, ok);
        }
        return ok;
    };
    // where a lane's codes and scales lie in a 4-bit tile (keys 8 later: 8 rows on, since the exchange of pieces repeats)
    const uint32_t ring_addr = smem_u32(ring);
    const uint32_t at_k = D == 128 ? code_at<D>(kA, t) : code_at<D>(kA, t >> 1) + (t & 1) * 8;
    const uint32_t at_ks = Tile<D>::SCALES + kA * Tile<D>::GROUPS + (D == 128 ? 2 * t : t);
    const uint32_t at_v0 = Tile<D>::HALF + (D == 128 ? code_at<D>(kV0, g >> 1) + (g & 1) * 8 : code_at<D>(kV0, g >> 2) + (g & 3) * 4);
    const uint32_t at_v1 = Tile<D>::HALF + (D == 128 ? code_at<D>(kV1, g >> 1) + (g & 1) * 8 : code_at<D>(kV1, g >> 2) + (g & 3) * 4);
    const uint32_t at_vs0 = Tile<D>::HALF + Tile<D>::SCALES + kV0 * Tile<D>::GROUPS + (D == 128 ? g : g >> 1);
    const uint32_t at_vs1 = Tile<D>::HALF + Tile<D>::SCALES + kV1 * Tile<D>::GROUPS + (D == 128 ? g : g >> 1);

    // (a warp whose wait gave up takes no more pages, but goes through every barrier and counts its items in)
    int done = 0;                                            // pages of the stretch so far
    for (; at < places; next_item()) {
        const int P = lens[s], held = helds[s];
        const PageList list = list_of(P);
        const Part part = next_part(list.count);
        const int v0 = part.v0, v1 = part.v1;
        if (v0 == v1) continue;
        const int n_keys = P + p.T;
        const int low_min = window_low(P, p.window);         // some row may see positions from here on
        const int low_max = p.window > 0 ? window_low(P + p.T - 1, p.window) : low_min;       // every row does

        // ---- the item's queries and what they see ----
        if (done > 0) asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory");      // the previous item's are no longer read
        for (int r = tid - (kWarps - 1) * 32; r >= 0 && r < 8 * NB; r += 32) {
            RowMask rm;
            rm.low = 0x7fffffff;                             // rows that do not exist see nothing
            rm.sees = 0;
            rm.bits[0] = rm.bits[1] = rm.bits[2] = rm.bits[3] = 0;
            if (r < PR) {
                const RowSight rs = row_sight(p.anc ? p.anc + (size_t)s * p.T * p.W : nullptr, p.causal, r / G, p.T, P, p.window, p.sinks);
                rm.low = rs.low;
                rm.sees = row_sees(rs, P, p.sinks);
                rm.bits[0] = (uint32_t)rs.bits[0]; rm.bits[1] = (uint32_t)(rs.bits[0] >> 32);
                rm.bits[2] = (uint32_t)rs.bits[1]; rm.bits[3] = (uint32_t)(rs.bits[1] >> 32);
            }
            mask[r].low = rm.low;
            mask[r].sees = rm.sees;
#pragma unroll
            for (int i = 0; i < 4; ++i) mask[r].bits[i] = rm.bits[i];
        }
        {
            constexpr int E = D / 32;                        // elements of a row that a lane stages: E * lane ..
            constexpr int NR = (8 * NB + kWarps - 1) / kWarps;     // rows of a warp, all in flight together
            uint32_t raw[NR][E / 2], raw_lo[NR][E / 2];
#pragma unroll
            for (int k = 0; k < NR; ++k) {
                const int r = warp + k * kWarps;
#pragma unroll
                for (int e = 0; e < E / 2; ++e) raw[k][e] = raw_lo[k][e] = 0u;
                if (r < PR) {
                    const size_t off = ((size_t)(s * p.T + r / G) * p.Hq + kvh * G + r % G) * D + lane * E;
                    if constexpr (E == 4) {
                        const uint2 v = *reinterpret_cast<const uint2 *>(p.q + off);
                        raw[k][0] = v.x; raw[k][1] = v.y;
                        if constexpr (TWO) {
                            const uint2 w = *reinterpret_cast<const uint2 *>(p.q_lo + off);
                            raw_lo[k][0] = w.x; raw_lo[k][1] = w.y;
                        }
                    } else {
                        raw[k][0] = *reinterpret_cast<const uint32_t *>(p.q + off);
                        if (TWO) raw_lo[k][0] = *reinterpret_cast<const uint32_t *>(p.q_lo + off);
                    }
                }
            }
#pragma unroll
            for (int k = 0; k < NR; ++k) {
                const int r = warp + k * kWarps;
                if (8 * NB % kWarps && r >= 8 * NB) break;
                float hi[E], lo[E];
#pragma unroll
                for (int e = 0; e < E; e += 2) {
                    const float2 v = unpack2<false>(raw[k][e / 2]), w = unpack2<false>(raw_lo[k][e / 2]);
                    hi[e] = v.x; hi[e + 1] = v.y;
                    lo[e] = w.x; lo[e + 1] = w.y;
                }
                float top = 0.f;
#pragma unroll
                for (int e = 0; e < E; ++e) top = fmaxf(top, fabsf(hi[e]));
                top = warp_max(top);
                // 2^-x brings the row's largest into [1, 2), which is undone in the score's scale
                const int x = top > 0.f && top < INFINITY ? min(max(ilogbf(top), -100), 120) : 0;
                const float down = exp2f((float)-x);
                if (lane == 0) mask[r].scale16 = sl2 * exp2f((float)x);
                const int n = r & 7, nb = r >> 3;
                uint32_t h16[E / 2], l16[E / 2], h32[E / 2], l32[E / 2];
#pragma unroll
                for (int e = 0; e < E; e += 2) {
                    const float a = (hi[e] + lo[e]) * down, b = (hi[e + 1] + lo[e + 1]) * down;
                    h16[e / 2] = pack2<true>(a, b);
                    const float2 v = unpack2<true>(h16[e / 2]);
                    l16[e / 2] = pack2<true>(a - v.x, b - v.y);
                    h32[e / 2] = pack2<false>(hi[e], hi[e + 1]);
                    l32[e / 2] = pack2<false>(lo[e], lo[e + 1]);
                }
                // fp16 fragments: lane (n, t') holds d = (D/4) t' + 4 j .. + 3 in its registers of k-step j
                // bf16 fragments: d = 16 j + 2 t' .. + 1 and the same 8 later
#pragma unroll
                for (int e = 0; e < E; e += 2) {
                    const int d0 = lane * E + e;
                    {
                        const int tt = d0 / (D / 4), j = d0 % (D / 4) / 4, reg = d0 % 4 / 2;
                        const int at = ((j >> 1) * 32 + n * 4 + tt) * 16 + (j & 1) * 8 + reg * 4;
                        *reinterpret_cast<uint32_t *>(sQ + (0 * NB + nb) * F::QB + at) = h16[e / 2];
                        *reinterpret_cast<uint32_t *>(sQ + (1 * NB + nb) * F::QB + at) = l16[e / 2];
                    }
                    {
                        const int j = d0 / 16, w = d0 % 16, reg = w / 8, tt = w % 8 / 2;
                        const int at = ((j >> 1) * 32 + n * 4 + tt) * 16 + (j & 1) * 8 + reg * 4;
                        *reinterpret_cast<uint32_t *>(sQ + (2 * NB + nb) * F::QB + at) = h32[e / 2];
                        *reinterpret_cast<uint32_t *>(sQ + (3 * NB + nb) * F::QB + at) = l32[e / 2];
                    }
                }
            }
        }
        asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory");

        if (trace) trace[3] = global_ns();
        float O[NB][MB][4];
        RowState rows_st[NB];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            rows_st[nb] = RowState{{0.f, 0.f}, {-INFINITY, -INFINITY}, {0.f, 0.f}};
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int i = 0; i < 4; ++i) O[nb][mb][i] = 0.f;
        }
        // masks a tile's scores; returns which of the lane's four V columns some row may see
        auto see = [&](int key) { return key < n_keys && (key < p.sinks || key >= low_min); };
        auto hide = [&](float (&c)[4], int nb, int key0) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const RowMask &rm = mask[nb * 8 + 2 * t + r];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int key = key0 + kA + 8 * k, e = key - P;
                    bool v;
                    if (e < 0) v = rm.low != 0x7fffffff && (key < p.sinks || key >= rm.low);
                    else v = e < 128 && ((rm.bits[(e >> 5) & 3] >> (e & 31)) & 1u);
                    if (!v) c[2 * k + r] = -INFINITY;
                }
            }
        };
        auto raise_acc = [&](int nb, const float (&f)[2]) {
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
                O[nb][mb][0] *= f[0]; O[nb][mb][1] *= f[1]; O[nb][mb][2] *= f[0]; O[nb][mb][3] *= f[1];
            }
        };
        // ---------------- pages in 4 bits: a prefix of the stretch's entries ----------------
        const int n_held = held_of(list, held, v0, v1);
        bool order4 = false;                                 // the accumulators have the 4-bit pages' order of d
        int i = (team + F::TEAMS - done % F::TEAMS) % F::TEAMS;              // this team's first entry
        done += v1 - v0;
        while (i < n_held) {
            if (!wait_all(&full[place], phase)) break;
            if (trace && !order4) trace[4] = global_ns();
            order4 = true;
            const uint32_t first_tile = ring_addr + (uint32_t)(place * F::PAGE_BYTES);
#pragma unroll 1
            for (uint32_t tile = first_tile; tile < first_tile + 3 * F::THIRD && i < n_held; tile += F::THIRD, i += F::TEAMS) {
                const int pg = list.page(v0 + i), key0 = pg * kPage;
                const bool open = key0 + kPage <= p.sinks || key0 >= low_max;        // every row sees all of it (it lies below P)
                float cc[CH][NB][4];
                {
                    constexpr int WORDS = D / 32;            // words of a key that a lane takes: d = (D/4) t ..
                    uint32_t wa[WORDS], wb[WORDS], sa, sb;
                    constexpr int ROW = Tile<D>::ROW, GROUPS = Tile<D>::GROUPS;
                    if constexpr (D == 128) {
                        const uint4 a = lds16(tile + at_k), b = lds16(tile + at_k + 8 * ROW);
                        wa[0] = a.x; wa[1] = a.y; wa[2] = a.z; wa[3] = a.w;
                        wb[0] = b.x; wb[1] = b.y; wb[2] = b.z; wb[3] = b.w;
                        sa = lds2(tile + at_ks);
                        sb = lds2(tile + at_ks + 8 * GROUPS);
                    } else {
                        const uint2 a = lds8(tile + at_k), b = lds8(tile + at_k + 8 * ROW);
                        wa[0] = a.x; wa[1] = a.y;
                        wb[0] = b.x; wb[1] = b.y;
                        sa = lds1(tile + at_ks) * 0x101u;
                        sb = lds1(tile + at_ks + 8 * GROUPS) * 0x101u;
                    }
                    sa = scales_to_half(sa);
                    sb = scales_to_half(sb);
#pragma unroll
                    for (int w = 0; w < WORDS; ++w) {
                        // two words to a scale
                        const uint32_t ga = __byte_perm(sa, 0, w < 2 ? 0x1010 : 0x3232), gb = __byte_perm(sb, 0, w < 2 ? 0x1010 : 0x3232);
                        uint32_t ha[4], hb[4];
                        codes_to_half(wa[w], ha);
                        codes_to_half(wb[w], hb);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            ha[k] = mul_half2(ha[k], ga);
                            hb[k] = mul_half2(hb[k], gb);
                        }
                        const uint32_t a0[4] = {ha[0], hb[0], ha[1], hb[1]}, a1[4] = {ha[2], hb[2], ha[3], hb[3]};
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb) {
                            const uint4 q = *reinterpret_cast<const uint4 *>(sQ + nb * F::QB + (w * 32 + lane) * 16);
                            if (2 * w < CH) mma_first<true>(cc[2 * w % CH][nb], a0, q.x, q.y);
                            else mma<true>(cc[2 * w % CH][nb], a0, q.x, q.y);
                            if (2 * w < CH) mma_first<true>(cc[(2 * w + 1) % CH][nb], a1, q.z, q.w);
                            else mma<true>(cc[(2 * w + 1) % CH][nb], a1, q.z, q.w);
                            if constexpr (TWO) {
                                const uint4 ql = *reinterpret_cast<const uint4 *>(sQ + (NB + nb) * F::QB + (w * 32 + lane) * 16);
                                mma<true>(cc[2 * w % CH][nb], a0, ql.x, ql.y);
                                mma<true>(cc[(2 * w + 1) % CH][nb], a1, ql.z, ql.w);
                            }
                        }
                    }
                }
                uint32_t b[NB][2], blo[NB][2];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    float (&c)[4] = cc[0][nb];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        c[e] += cc[1][nb][e];
                    }
                    const float s0 = mask[nb * 8 + 2 * t].scale16, s1 = mask[nb * 8 + 2 * t + 1].scale16;
                    if (!open) hide(c, nb, key0);
                    float f[2];
                    if (softmax_tile<true, TWO>(c, rows_st[nb], s0, s1, b[nb], blo[nb], f)) raise_acc(nb, f);
                }
                {
                    constexpr int WORDS = D / 64;            // words of a key that a lane takes: d = (D/8) g ..
                    constexpr int ROW = Tile<D>::ROW, GROUPS = Tile<D>::GROUPS;
                    uint32_t w[4][WORDS], sc[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {            // keys kV0, kV1, kV0 + 8, kV1 + 8
                        const uint32_t at = tile + ((k & 1) ? at_v1 : at_v0) + (k >> 1) * 8 * ROW, ats = tile + ((k & 1) ? at_vs1 : at_vs0) + (k >> 1) * 8 * GROUPS;
                        if constexpr (D == 128) {
                            const uint2 a = lds8(at);
                            w[k][0] = a.x; w[k][1] = a.y;
                        } else {
                            w[k][0] = lds4(at);
                        }
                        sc[k] = lds1(ats);
                    }
                    if (!open) {                             // what nobody sees may be anything, NaN included
#pragma unroll
                        for (int k = 0; k < 4; ++k) sc[k] = see(key0 + ((k & 1) ? kV1 : kV0) + (k >> 1) * 8) ? sc[k] : 0u;
                    }
                    const uint32_t s01 = scales_to_half(sc[0] | sc[1] << 8), s23 = scales_to_half(sc[2] | sc[3] << 8);
#pragma unroll
                    for (int wi = 0; wi < WORDS; ++wi) {
                        // (key 0, key 1) pairs of the same d: even d from the low nibbles, odd d from the high ones
                        uint32_t e01[4], o01[4], e23[4], o23[4];
                        constexpr uint32_t LOW = 0x0f0f0f0fu;
                        codes_to_half((w[0][wi] & LOW) | ((w[1][wi] << 4) & ~LOW), e01);
                        codes_to_half(((w[0][wi] >> 4) & LOW) | (w[1][wi] & ~LOW), o01);
                        codes_to_half((w[2][wi] & LOW) | ((w[3][wi] << 4) & ~LOW), e23);
                        codes_to_half(((w[2][wi] >> 4) & LOW) | (w[3][wi] & ~LOW), o23);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const uint32_t a[4] = {mul_half2(e01[k], s01), mul_half2(o01[k], s01), mul_half2(e23[k], s23), mul_half2(o23[k], s23)};
#pragma unroll
                            for (int nb = 0; nb < NB; ++nb) {
                                mma<true>(O[nb][wi * 4 + k], a, b[nb][0], b[nb][1]);
                                if constexpr (TWO) mma<true>(O[nb][wi * 4 + k], a, blo[nb][0], blo[nb][1]);
                            }
                        }
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&empty[place]);
            advance();
        }
        // ---------------- pages in bf16 ----------------
        if (ok && i < v1 - v0) {
            if (order4) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) reorder<D>(O[nb], g);
                order4 = false;
            }
            for (; i < v1 - v0; i += F::TEAMS) {
                const int pg = list.page(v0 + i), key0 = pg * kPage;
                const bool open = key0 + kPage <= P && (key0 + kPage <= p.sinks || key0 >= low_max);     // every row sees all of it
                if (!wait_all(&full[place], phase)) break;
                if (trace && n_held == 0 && i < F::TEAMS) trace[4] = global_ns();
                const uint32_t kbase = smem_u32(ring + place * F::PAGE_BYTES), vbase = kbase + kPage * D * 2;
                float cc[CH][NB][4];
                // lane's row of the four 8 x 8 matrices it addresses
                const int mi = lane >> 3, r = first_key + key_of(lane & 7);
#pragma unroll
                for (int j = 0; j < KS; ++j) {
                    // keys 0-7 | 8-15 of d 0-7, then of d 8-15
                    const int key = r + (mi & 1) * 8, ch = 2 * j + (mi >> 1);
                    uint32_t a[4];
                    ldmatrix4(kbase + (ch >> 3) * (kPage * 128) + key * 128 + (((ch & 7) ^ (key & 7)) << 4), a);
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        const uint2 q = *reinterpret_cast<const uint2 *>(sQ + (2 * NB + nb) * F::QB + ((j >> 1) * 32 + lane) * 16 + (j & 1) * 8);
                        if (j < CH) mma_first<false>(cc[j % CH][nb], a, q.x, q.y);
                        else mma<false>(cc[j % CH][nb], a, q.x, q.y);
                        if constexpr (TWO) {
                            const uint2 ql = *reinterpret_cast<const uint2 *>(sQ + (3 * NB + nb) * F::QB + ((j >> 1) * 32 + lane) * 16 + (j & 1) * 8);
                            mma<false>(cc[j % CH][nb], a, ql.x, ql.y);
                        }
                    }
                }
                uint32_t b[NB][2], blo[NB][2];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    float (&c)[4] = cc[0][nb];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        c[e] += cc[1][nb][e];
                    }
                    if (!open) hide(c, nb, key0);
                    float f[2];
                    if (softmax_tile<false, true>(c, rows_st[nb], sl2, sl2, b[nb], blo[nb], f)) raise_acc(nb, f);
                }
                uint32_t keep01 = ~0u, keep23 = ~0u;         // what nobody sees may be anything, NaN included
                if (!open) {
                    keep01 = (see(key0 + kV0) ? 0xffffu : 0u) | (see(key0 + kV1) ? 0xffff0000u : 0u);
                    keep23 = (see(key0 + kV0 + 8) ? 0xffffu : 0u) | (see(key0 + kV1 + 8) ? 0xffff0000u : 0u);
                }
#pragma unroll
                for (int mb = 0; mb < MB; ++mb) {
                    // d 0-7 | 8-15 of keys 0-7, then of keys 8-15
                    const int key = r + (mi >> 1) * 8, ch = 2 * mb + (mi & 1);
                    uint32_t a[4];
                    ldmatrix4_trans(vbase + (ch >> 3) * (kPage * 128) + key * 128 + (((ch & 7) ^ (key & 7)) << 4), a);
                    a[0] &= keep01; a[1] &= keep01; a[2] &= keep23; a[3] &= keep23;
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        mma<false>(O[nb][mb], a, b[nb][0], b[nb][1]);
                        mma<false>(O[nb][mb], a, blo[nb][0], blo[nb][1]);
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&empty[place]);
                advance();
            }
        }

        if (trace) trace[5] = global_ns();
        // ---- the warps' parts meet; this CTA's part of the item, or all of it ----
        // the item's first page lies in the stretch of CTA blockIdx - back; the item spreads over `parts` stretches
        const int back = part.from < 0 ? (chunk - 1 - part.from) / chunk : 0;
        const int parts = (part.from + back * chunk + list.count - 1) / chunk + 1;
        // a CTA may share an item that began before its stretch (its first part), and the one that begins in it last (its second)
        const int slot = 2 * (int)blockIdx.x + (part.from >= 0 ? 1 : 0);
        const int rows = min(PR, 8 * NB);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int o = 4; o <= 16; o <<= 1) rows_st[nb].sum[r] += __shfl_xor_sync(0xffffffffu, rows_st[nb].sum[r], o);
            if (g == 0) {
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    red_m[warp][nb * 8 + 2 * t + r] = rows_st[nb].limit[r] == -INFINITY ? -INFINITY : rows_st[nb].ref[r];
                    red_l[warp][nb * 8 + 2 * t + r] = rows_st[nb].sum[r];
                }
            }
        }
        // this warp's accumulators of 8 rows to dst [8][ROWF], element d at place_of(d): so neither order meets a bank twice
        auto place_of = [](int d) { return d ^ ((d >> 4 & 1) << 2); };
        auto put = [&](int nb, float *dst) {
            if (order4) {                                    // a lane has D / 8 consecutive d of rows 2t, 2t + 1
#pragma unroll
                for (int mb = 0; mb < MB; mb += 2)
#pragma unroll
                    for (int r = 0; r < 2; ++r)
                        *reinterpret_cast<float4 *>(dst + (2 * t + r) * F::ROWF + place_of((D / 8) * g + 2 * mb)) =
                            make_float4(O[nb][mb][r], O[nb][mb][2 + r], O[nb][mb + 1][r], O[nb][mb + 1][2 + r]);
            } else {
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                    for (int e = 0; e < 4; ++e) dst[(2 * t + (e & 1)) * F::ROWF + place_of(16 * mb + 8 * (e >> 1) + g)] = O[nb][mb][e];
            }
        };
        // element (row, d0 .. d0 + 3) over the warps w0 .. w0 + n - 1, whose accumulators lie `step` floats apart from src on
        auto add_warps = [&](const float *src, int step, int w0, int n, int row, int d0, float M, float4 &acc, float &L) {
#pragma unroll 4
            for (int w = 0; w < n; ++w) {
                const float mw = red_m[w0 + w][row], f = mw == -INFINITY ? 0.f : ex2(mw - M);
                const float4 a = *reinterpret_cast<const float4 *>(src + w * step + (row & 7) * F::ROWF + place_of(d0));
                L += f * red_l[w0 + w][row];
                acc.x += f * a.x; acc.y += f * a.y; acc.z += f * a.z; acc.w += f * a.w;
            }
        };
        auto top_of = [&](int row) {
            float M = -INFINITY;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) M = fmaxf(M, red_m[w][row]);
            return M;
        };
        auto emit = [&](int row, int d0, float M, float L, float4 acc) {
            if (row >= rows) return;
            if (p.S > 0) {
                *reinterpret_cast<float4 *>(red + row * F::ROWF + d0) = acc;
                if (d0 == 0) {
                    sum_m[row] = M;
                    sum_l[row] = L;
                }
            } else if (parts == 1) {
                const float inv = L > 0.f || mask[row].sees ? 1.f / L : 0.f;
                const size_t off = ((size_t)(s * p.T + row / G) * p.Hq + kvh * G + row % G) * D + d0;
                store_two_term(p.out + off, p.out_lo ? p.out_lo + off : nullptr, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
            } else {
                *reinterpret_cast<float4 *>(p.parts + ((size_t)slot * kFewRows + row) * D + d0) = acc;
                if (d0 == 0) reinterpret_cast<float2 *>(p.parts_ml)[(size_t)slot * kFewRows + row] = make_float2(M, L);
            }
        };
        constexpr int ELEMS = 8 * (D / 4), WARP_F = 8 * F::ROWF;             // of 8 rows
        if (places - at <= lead) {
            // The CTA's last item: no more pages come, so the rings hold the accumulators of all warps and blocks at once.
            asm volatile("bar.sync %0, %1;" ::"r"(2 + team), "n"(kTeam * 32) : "memory");        // the team has read its last page
            float *mine = reinterpret_cast<float *>(ring);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) put(nb, mine + (nb * kTeam + warp % kTeam) * WARP_F);
            asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory");
            for (int i = tid; i < NB * ELEMS; i += kWarps * 32) {
                const int nb = i / ELEMS, row = nb * 8 + i % ELEMS / (D / 4), d0 = i % (D / 4) * 4;
                const float M = top_of(row);
                float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
                float L = 0.f;
#pragma unroll
                for (int k = 0; k < F::TEAMS; ++k)
                    add_warps(reinterpret_cast<const float *>(smem + k * F::PLACES * F::PAGE_BYTES) + nb * kTeam * WARP_F, WARP_F, k * kTeam, kTeam, row, d0, M, acc, L);
                emit(row, d0, M, L, acc);
            }
        } else {
            // pages of the next item are under way: one team and block at a time, a thread keeps its element's sum over the teams
            constexpr int PER = (ELEMS + kWarps * 32 - 1) / (kWarps * 32);
            for (int nb = 0; nb < NB; ++nb) {
                float4 acc[PER];
                float M[PER], L[PER];
                for (int k = 0; k < F::TEAMS; ++k) {
                    if (team == k) {
#pragma unroll
                        for (int b = 0; b < NB; ++b)
                            if (b == nb) put(b, red + warp % kTeam * WARP_F);
                    }
                    asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory");
#pragma unroll
                    for (int e = 0; e < PER; ++e) {
                        const int i = tid + e * kWarps * 32, row = nb * 8 + i / (D / 4), d0 = i % (D / 4) * 4;
                        if (i >= ELEMS) break;
                        if (k == 0) {
                            M[e] = top_of(row);
                            L[e] = 0.f;
                            acc[e] = make_float4(0.f, 0.f, 0.f, 0.f);
                        }
                        add_warps(red, WARP_F, k * kTeam, kTeam, row, d0, M[e], acc[e], L[e]);
                        if (k == F::TEAMS - 1) emit(row, d0, M[e], L[e], acc[e]);
                    }
                    asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory");
                }
            }
        }
        if (trace) trace[6] = global_ns();
        if (p.S == 0 && parts > 1) {
            asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory");
            if (tid == 0) {
                // releases what the whole CTA wrote (the barrier orders it before this thread), acquires the others' parts
                int before;
                __threadfence();
                asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(before) : "l"(p.part_counters + s * p.Hkv + kvh) : "memory");
                bars.last = before == parts - 1;
                if (bars.last) p.part_counters[s * p.Hkv + kvh] = 0;    // for the next launch
            }
            asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory");
            if (trace) trace[7] = global_ns();
            if (bars.last) {
                // every team takes every TEAMS-th part, 8 elements a thread; the teams' sums meet in shared memory
                const int c_first = (int)blockIdx.x - back;
                float *team_m = &red_m[0][0], *team_l = &red_l[0][0];        // [team][8 NB]
                for (int i = tid % (kTeam * 32); i < rows * (D / 8); i += kTeam * 32) {
                    const int row = i / (D / 8), d0 = i % (D / 8) * 8;
                    float M = -INFINITY, L = 0.f;
                    float acc[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) acc[e] = 0.f;
                    constexpr int U = 7;                     // parts in flight
                    for (int c0 = team; c0 < parts; c0 += U * F::TEAMS) {
                        float2 ml[U];
                        float4 a[U][2];
#pragma unroll
                        for (int k = 0; k < U; ++k) {
                            const int c = min(c0 + k * F::TEAMS, parts - 1);
                            const size_t slot = (size_t)(2 * (c_first + c) + (c == 0 ? 1 : 0)) * kFewRows + row;
                            ml[k] = __ldcg(reinterpret_cast<const float2 *>(p.parts_ml) + slot);
                            a[k][0] = __ldcg(reinterpret_cast<const float4 *>(p.parts + slot * D + d0));
                            a[k][1] = __ldcg(reinterpret_cast<const float4 *>(p.parts + slot * D + d0) + 1);
                        }
                        float M2 = M;
#pragma unroll
                        for (int k = 0; k < U; ++k) {
                            if (c0 + k * F::TEAMS >= parts) ml[k] = make_float2(-INFINITY, 0.f);
                            M2 = fmaxf(M2, ml[k].x);
                        }
                        const float f0 = M == -INFINITY ? 0.f : ex2(M - M2);
                        L *= f0;
#pragma unroll
                        for (int e = 0; e < 8; ++e) acc[e] *= f0;
#pragma unroll
                        for (int k = 0; k < U; ++k) {
                            const float f = ml[k].x == -INFINITY ? 0.f : ex2(ml[k].x - M2);
                            L += ml[k].y * f;
                            acc[0] += a[k][0].x * f; acc[1] += a[k][0].y * f; acc[2] += a[k][0].z * f; acc[3] += a[k][0].w * f;
                            acc[4] += a[k][1].x * f; acc[5] += a[k][1].y * f; acc[6] += a[k][1].z * f; acc[7] += a[k][1].w * f;
                        }
                        M = M2;
                    }
                    float *dst = red + (team * 8 * NB + row) * F::ROWF + d0;
                    *reinterpret_cast<float4 *>(dst) = make_float4(acc[0], acc[1], acc[2], acc[3]);
                    *reinterpret_cast<float4 *>(dst + 4) = make_float4(acc[4], acc[5], acc[6], acc[7]);
                    if (d0 == 0) {
                        team_m[team * 8 * NB + row] = M;
                        team_l[team * 8 * NB + row] = L;
                    }
                }
                asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory");
                for (int i = tid; i < rows * (D / 4); i += kWarps * 32) {
                    const int row = i / (D / 4), d0 = i % (D / 4) * 4;
                    float M = -INFINITY, L = 0.f;
#pragma unroll
                    for (int k = 0; k < F::TEAMS; ++k) M = fmaxf(M, team_m[k * 8 * NB + row]);
                    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                    for (int k = 0; k < F::TEAMS; ++k) {
                        const float mk = team_m[k * 8 * NB + row], f = mk == -INFINITY ? 0.f : ex2(mk - M);
                        const float4 a = *reinterpret_cast<const float4 *>(red + (k * 8 * NB + row) * F::ROWF + d0);
                        L += f * team_l[k * 8 * NB + row];
                        acc.x += f * a.x; acc.y += f * a.y; acc.z += f * a.z; acc.w += f * a.w;
                    }
                    const float inv = L > 0.f || mask[row].sees ? 1.f / L : 0.f;
                    const size_t off = ((size_t)(s * p.T + row / G) * p.Hq + kvh * G + row % G) * D + d0;
                    store_two_term(p.out + off, p.out_lo ? p.out_lo + off : nullptr, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
                }
            }
        }
    }
    if (p.S > 0) {
        // ---- the cluster's CTAs hold a part of one item each: every CTA adds its share of the elements over all of them ----
        __syncwarp();
        cluster_sync_all();
        if (trace) trace[8] = global_ns();
        const int item = (int)blockIdx.x / p.S, sq = item / p.Hkv, kvh = item % p.Hkv;
        const int n = min(PR, 8 * NB) * (D / 4);
        for (int i = (int)cluster_rank() + p.S * tid; i < n; i += p.S * kWarps * 32) {
            const int row = i / (D / 4), d0 = i % (D / 4) * 4;
            float pm[kMaxCluster], pl[kMaxCluster], M = -INFINITY, L = 0.f;
            float4 a[kMaxCluster], acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < kMaxCluster; ++k) {
                const uint32_t from = (uint32_t)min(k, p.S - 1);
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(pm[k]) : "r"(map_to_rank(smem_u32(sum_m + row), from)) : "memory");
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(pl[k]) : "r"(map_to_rank(smem_u32(sum_l + row), from)) : "memory");
                asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(a[k].x), "=f"(a[k].y), "=f"(a[k].z), "=f"(a[k].w)
                             : "r"(map_to_rank(smem_u32(red + row * F::ROWF + d0), from)) : "memory");
            }
#pragma unroll
            for (int k = 0; k < kMaxCluster; ++k)
                if (k < p.S) M = fmaxf(M, pm[k]);
            if (M == -INFINITY) M = 0.f;
#pragma unroll
            for (int k = 0; k < kMaxCluster; ++k)
                if (k < p.S && !(pl[k] < 0.f)) {             // (a CTA without pages wrote no outputs)
                    const float f = ex2(pm[k] - M);          // 2^-inf = 0 for a part without a maximum: NaN where the row's scores were
                    L += f * pl[k];
                    acc.x += f * a[k].x; acc.y += f * a[k].y; acc.z += f * a[k].z; acc.w += f * a[k].w;
                }
            int sees = 1;
            if (!(L > 0.f))                                  // (the first CTA of a cluster has pages)
                asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(sees) : "r"(map_to_rank(smem_u32(&mask[row].sees), 0u)) : "memory");
            const float inv = sees ? 1.f / L : 0.f;
            const size_t off = ((size_t)(sq * p.T + row / G) * p.Hq + kvh * G + row % G) * D + d0;
            store_two_term(p.out + off, p.out_lo ? p.out_lo + off : nullptr, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
        }
        __syncwarp();
        cluster_sync_all();                                  // nobody leaves while a peer may read its part
    }
    if (trace) trace[11] = global_ns();
    if (p.trace && threadIdx.x == 0) atomicMax(p.trace + 15, (unsigned long long)global_ns());
}

template <int D, int NB>
cudaLaunchConfig_t few_config(cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(Few<D, NB>::THREADS, 1, 1);
    cfg.dynamicSmemBytes = Few<D, NB>::TOTAL;
    cfg.stream = st;
    return cfg;
}

// clusters of S CTAs that are resident at once (the kernel's attributes are set)
template <int D, int NB, bool TWO>
int few_clusters(int dev, int S) {
    static Answers<kMaxCluster + 1> answers;
    return answers.get(dev, S, 1, [&] {
        cudaLaunchConfig_t cfg = few_config<D, NB>(nullptr);
        cfg.gridDim = dim3(S, 1, 1);
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = S;
        attr[0].val.clusterDim.y = 1;
        attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        int n = 0;
        return cudaOccupancyMaxActiveClusters(&n, attn_few_kernel<D, NB, TWO>, &cfg) == cudaSuccess ? n : 0;
    });
}

template <int D, int NB, bool TWO>
cudaError_t launch_few(const AttnParams &p, const CUtensorMap &map_kv, long long pages, cudaStream_t st) {
    using F = Few<D, NB>;
    static Answers<1> ready;
    const int dev = current_device();
    if (!ready.get(dev, 0, 0, [] { return cudaFuncSetAttribute(attn_few_kernel<D, NB, TWO>, cudaFuncAttributeMaxDynamicSharedMemorySize, F::TOTAL) == cudaSuccess; }))
        return cudaErrorInvalidDevice;
    const int items = p.Hkv * p.batch;
    // A cluster an item, whose CTAs add their parts through distributed shared memory in 1.5 us, where that costs a CTA no more
    // than kMorePages pages (0.4 us in 4 bits, 0.8 in bf16) beyond its share of the line; there the parts of an item meet in
    // global memory, 3.5 us and more.
    AttnParams q = p;
    q.S = 0;
    for (int S = kMaxCluster; S > 1 && q.S == 0; S /= 2)
        if (items <= few_clusters<D, NB, TWO>(dev, S) && (pages + S - 1) / S <= (pages * items + 147) / 148 + kMorePages) q.S = S;
    cudaLaunchConfig_t cfg = few_config<D, NB>(st);
    // (no more CTAs than pages)
    cfg.gridDim = dim3((unsigned)(q.S > 0 ? (long long)items * q.S : std::min<long long>(148, pages * items)), 1, 1);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = q.S;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = q.S > 0 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, attn_few_kernel<D, NB, TWO>, map_kv, q);
}

}  // namespace

// (the places of a line are counted in 32 bits)
bool attention_few_takes(int T, int G, long long items, long long pages) { return (long long)T * G <= kFewRows && (double)items * pages < 1e9; }

// pages: as many as a row may see (the lengths themselves are on the device)
cudaError_t launch_attention_few(const AttnParams &p, const CUtensorMap &map_kv, long long pages, cudaStream_t st) {
    const int rows = p.T * (p.Hq / p.Hkv);
    auto pick = [&](auto d, auto two) {
        constexpr int D = decltype(d)::value;
        constexpr bool TWO = decltype(two)::value;
        return rows <= 8 ? launch_few<D, 1, TWO>(p, map_kv, pages, st) : launch_few<D, 2, TWO>(p, map_kv, pages, st);
    };
    using D128 = std::integral_constant<int, 128>;
    using D64 = std::integral_constant<int, 64>;
    if (p.d == 128) return p.q_lo ? pick(D128{}, std::true_type{}) : pick(D128{}, std::false_type{});
    return p.q_lo ? pick(D64{}, std::true_type{}) : pick(D64{}, std::false_type{});
}

}  // namespace glance
