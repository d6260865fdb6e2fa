// Attention of few query rows (single tokens, short blocks and trees) over a long paged cache that is read in part (sliding
// window, sinks) or held in 4 bits: bound by the bytes of the cache, so everything is laid out around streaming them once.
//
// The pages that a launch has to read form one line: sequences, in each its kv heads, in each the pages that some row sees
// (packed.cuh).  The line is dealt out in equal stretches to two CTAs an SM, so ragged batches and long single sequences
// keep the whole GPU reading; a CTA finds its stretch from the device-resident lengths by one prefix sum.  Warp 4 fetches
// pages into a ring (bf16: two tensor copies; 4 bits: one bulk copy of a 4.5-bit tile, three of which fit where a bf16 page
// does), warps 0..3 take 16 of a page's 64 keys each and never wait for one another inside an item.
//     S^T[16 keys x 8 rows] = K Q^T,   O^T[d x 8 rows] += V^T P^T     (mma.sync m16n8k16, fp32 accumulators)
// Keys sit in the M dimension, so one token's 7 or 8 heads fill an instruction's N exactly; with rows in M half of it
// would idle, and 128-row tcgen05 tiles would run at 6 % and wait for their tensor memory round trips.  At 8 rows a page
// takes 128 to 250 clocks of mma against 1400 (bf16) or 400 (4 bits) of its share of HBM.
// 4-bit pages go from shared memory to registers in the order in which the mma wants them (16 consecutive d of a key per
// lane; the contraction order is free as long as Q has the same), fp16: code x scale is exact there, and fp16 has the
// conversion.  A row's queries are scaled by a power of two into fp16's range (exact); P is one fp16 term (2^-12 relative), two
// where the caller has two-term queries.  bf16 pages stay bf16: Q as it is, P in two bf16 terms (one would cost 2^-9).
// A row's reference maximum is raised only when a score exceeds it by 2^8; sums and accumulators are fp32.
// The warps' partial results meet in shared memory; an item that several CTAs share is finished by the one that comes last,
// which adds the parts in line order, so results do not depend on timing.
#include <algorithm>

#include "kernels.cuh"
#include "packed.cuh"
#include "tc_ptx.cuh"

namespace glance {

namespace {

using namespace tc;
using namespace packed;

constexpr int kWarps = 4;                    // consumer warps
constexpr int kFewThreads = (kWarps + 1) * 32;
constexpr int kMaxSeqs = 64;
constexpr float kRaise = 8.f;                // log2 units a score may exceed its reference by

template <int D, int NB>
struct Few {
    static constexpr int SUB = D == 128 ? 11264 : 6144;      // one 4-bit tile (multiple of 1024: three make room for a bf16 page)
    static constexpr int SLOTS = NB == 4 ? 15 : 6;
    static constexpr int RING = SLOTS * SUB;
    static constexpr int PAGE_BYTES = 2 * kPage * D * 2;     // K and V of a bf16 page
    static constexpr int ROWF = D + 4;
    static constexpr int QB = 8 * D * 2;                     // one term of 8 rows' queries
    static constexpr int Q_AT = RING;                        // [fp16 | bf16][term][NB] fragments
    static constexpr int RED_AT = Q_AT + 4 * NB * QB;        // [warp][8][ROWF] partial outputs of 8 rows
    static constexpr int TOTAL = RED_AT + kWarps * 8 * ROWF * 4 + 1024;
    static constexpr int CTAS = NB == 4 ? 1 : 2;             // an SM
    static_assert(3 * SUB >= PAGE_BYTES && SUB >= Tile<D>::BYTES && SLOTS % 3 == 0, "ring");
    static_assert(CTAS * (TOTAL + 4096) <= 228 * 1024, "CTAs an SM");
};

// key of row r of a 16-key tile (r < 8; the other eight follow 8 later): eight keys that lanes read side by side differ in
// the bits that pick a bank, for the 4-bit tile's rows as for 128-byte swizzled ones
__device__ __forceinline__ int key_of(int r) { return (r & 1) ? 4 + ((r >> 1) ^ 1) : r >> 1; }

template <bool HALF>
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (HALF)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
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

template <int SLOTS>
struct alignas(8) FewBars {
    uint64_t full[SLOTS], empty[SLOTS];
    int abort_flag, last;
};

struct alignas(16) RowMask {
    uint32_t bits[4];
    int low;
    float scale16;               // score scale in log2 units for the fp16 queries of this row
    int pad[2];
};

// One 16-key tile's softmax and the probabilities as the second product's B operand.  c: scores [key g | g + 8][rows 2t, 2t+1].
template <bool HALF>
__device__ __forceinline__ void softmax_tile(float (&c)[4], float (&m)[2], float (&l)[2], float s0, float s1, bool two, uint32_t (&b)[2],
                                             uint32_t (&blo)[2], bool &raise, float (&f)[2]) {
    c[0] *= s0; c[1] *= s1; c[2] *= s0; c[3] *= s1;
    float x0 = fmaxf(c[0], c[2]), x1 = fmaxf(c[1], c[3]);
    raise = __any_sync(0xffffffffu, x0 > m[0] + kRaise || x1 > m[1] + kRaise);      // (m starts at -inf; a row that sees nothing stays there)
    f[0] = f[1] = 1.f;
    if (raise) {
#pragma unroll
        for (int o = 4; o <= 16; o <<= 1) {
            x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, o));
            x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, o));
        }
        if (x0 > m[0] + kRaise) { f[0] = ex2(m[0] - x0); m[0] = x0; }
        if (x1 > m[1] + kRaise) { f[1] = ex2(m[1] - x1); m[1] = x1; }
        l[0] *= f[0];
        l[1] *= f[1];
    }
    const float r0 = m[0] == -INFINITY ? 0.f : m[0], r1 = m[1] == -INFINITY ? 0.f : m[1];
    c[0] = ex2(c[0] - r0); c[1] = ex2(c[1] - r1); c[2] = ex2(c[2] - r0); c[3] = ex2(c[3] - r1);
    l[0] += c[0] + c[2];
    l[1] += c[1] + c[3];
    const uint32_t h0 = pack2<HALF>(c[0], c[1]), h1 = pack2<HALF>(c[2], c[3]);
    b[0] = transpose8(h0);
    b[1] = transpose8(h1);
    if (two) {
        const float2 v0 = unpack2<HALF>(h0), v1 = unpack2<HALF>(h1);
        blo[0] = transpose8(pack2<HALF>(c[0] - v0.x, c[1] - v0.y));
        blo[1] = transpose8(pack2<HALF>(c[2] - v1.x, c[3] - v1.y));
    }
}

template <int D, int NB>
__global__ void __launch_bounds__(kFewThreads, Few<D, NB>::CTAS) attn_few_kernel(const __grid_constant__ CUtensorMap map_kv, AttnParams p, int share) {
    using F = Few<D, NB>;
    constexpr int KS = D / 16, MB = D / 16;
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = reinterpret_cast<unsigned char *>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    unsigned char *ring = smem, *sQ = smem + F::Q_AT;
    float *red = reinterpret_cast<float *>(smem + F::RED_AT);
    __shared__ FewBars<F::SLOTS> bars;
    __shared__ int upto[kMaxSeqs + 1];                       // pages (of all heads) of the sequences before
    __shared__ RowMask mask[8 * NB];
    __shared__ float red_m[kWarps][8], red_l[kWarps][8];

    pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int G = p.Hq / p.Hkv, PR = p.T * G;
    volatile int *abort_flag = &bars.abort_flag;
    // positions that rows see, of a sequence (lengths may be read before the dependency wait: see attention_tc.cu)
    auto pages_of = [&](int s, int &P, PageList &l) {
        P = max(p.seq_len[s], 0);
        l = page_list(P + p.T, window_low(P, p.window), p.sinks);
    };
    if (threadIdx.x == 0) {
        for (int i = 0; i < F::SLOTS; ++i) {
            mbar_init(&bars.full[i], 1);
            mbar_init(&bars.empty[i], kWarps);
        }
        bars.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        int run = 0;
        for (int s0 = 0; s0 < p.batch; s0 += 32) {
            int n = 0;
            if (s0 + lane < p.batch) {
                int P;
                PageList l;
                pages_of(s0 + lane, P, l);
                n = l.count * p.Hkv;
            }
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, n, o);
                if (lane >= o) n += v;
            }
            if (s0 + lane < p.batch) upto[s0 + lane + 1] = run + n;
            run += __shfl_sync(0xffffffffu, n, 31);
        }
        if (lane == 0) upto[0] = 0;
    }
    __syncthreads();
    const int total = upto[p.batch];
    // equal stretches, of `share` pages at least
    const int chunk = max((total + (int)gridDim.x - 1) / (int)gridDim.x, share);
    const int x_begin = min((int)blockIdx.x * chunk, total), x_end = min(x_begin + chunk, total);
    int s = 0;
    while (s + 1 < p.batch && upto[s + 1] <= x_begin) ++s;

    if (warp == kWarps) {
        // ---------------- producer ----------------
        if (lane == 0) {
            bool waited = false, ok = true;
            int u = 0;                                       // sub-slots used so far
            auto take = [&](int n) {                         // waits until the next n sub-slots are free
                for (int i = 0; i < n && ok; ++i)
                    ok = mbar_wait(&bars.empty[(u + i) % F::SLOTS], (uint32_t)(((u + i) / F::SLOTS) & 1) ^ 1u, abort_flag, p.status);
                return ok;
            };
            for (int x = x_begin; x < x_end && ok;) {
                while (upto[s + 1] <= x) ++s;
                int P;
                PageList list;
                pages_of(s, P, list);
                const int held = p.held_len ? min(max(p.held_len[s], 0), P) / kPage : 0;
                const int kvh = (x - upto[s]) / list.count, v0 = (x - upto[s]) % list.count;
                const int v1 = min(list.count, v0 + (x_end - x));
                for (int v = v0; v < v1 && ok; ++v) {
                    const int pg = list.page(v);
                    if (!waited && (pg + 1) * kPage > P - kMaxBlock) {      // rows that this pass may write
                        pdl_wait();
                        waited = true;
                    }
                    const bool in_table = pg < p.geom.max_pages_per_seq;
                    const size_t entry = (size_t)s * p.geom.max_pages_per_seq + pg;
                    if (pg < held) {
                        int page = in_table ? p.held_table[entry] : -1;
                        if (page < 0 || page >= p.held_pages) { page = 0; set_status(p.status, GLANCE_E_BOUNDS); }
                        if (!take(1)) break;
                        uint64_t *bar = &bars.full[u % F::SLOTS];
                        mbar_expect_tx(bar, Tile<D>::BYTES);
                        bulk_load(ring + (u % F::SLOTS) * F::SUB, p.held_layer + ((size_t)page * p.Hkv + kvh) * Tile<D>::BYTES, Tile<D>::BYTES, bar);
                        u += 1;
                    } else {
                        int page = in_table ? p.page_table[entry] : -1;
                        if (page < 0 || page >= p.geom.n_pages) { page = 0; set_status(p.status, GLANCE_E_BOUNDS); }
                        const int skip = (3 - u % 3) % 3;    // to the next place for a whole bf16 page; nothing is put into these
                        if (!take(skip + 3)) break;
                        for (int i = 0; i < skip; ++i) mbar_arrive(&bars.full[(u + i) % F::SLOTS]);
                        u += skip;
                        const int at = u % F::SLOTS;
                        mbar_arrive(&bars.full[at + 1]);
                        mbar_arrive(&bars.full[at + 2]);
                        mbar_expect_tx(&bars.full[at], F::PAGE_BYTES);
#pragma unroll
                        for (int kv = 0; kv < 2; ++kv) {
                            const int row = ((page * 2 + kv) * p.Hkv + kvh) * kPage;
#pragma unroll
                            for (int sl = 0; sl < D / 64; ++sl)
                                tma_load_2d(ring + at * F::SUB + (kv * (D / 64) + sl) * (kPage * 128), &map_kv, &bars.full[at], sl * 64, row);
                        }
                        u += 3;
                    }
                }
                x += v1 - v0;
            }
            if (!waited) pdl_wait();
            if (*abort_flag) {                               // copies already issued must land before the CTA may exit
                for (int i = 0; i < F::SLOTS; ++i) {
                    const int w = u - 1 - i;
                    if (w < 0) break;
                    const uint64_t t0 = global_ns();
                    while (!mbar_try_wait(&bars.full[w % F::SLOTS], (uint32_t)(w / F::SLOTS) & 1u))
                        if (global_ns() - t0 > kWaitLimitNs) break;
                }
            }
        }
        __syncwarp();
        return;
    }

    // ---------------- consumers ----------------
    pdl_wait();
    const int g = lane >> 2, t = lane & 3, tid = threadIdx.x;
    const float sl2 = rsqrtf((float)D) * 1.4426950408889634f;
    const int kA = warp * 16 + key_of(g);                    // this lane's keys as rows of K: kA, kA + 8
    const int kV0 = warp * 16 + t, kV1 = warp * 16 + 4 + (t ^ 1);      // and as columns of V^T: kV0, kV1, kV0 + 8, kV1 + 8
    const bool two = p.q_lo != nullptr;
    int u = 0;
    bool ok = true;

    // (a warp whose wait gave up takes no more pages, but goes through every barrier and counts its items in)
    for (int x = x_begin; x < x_end;) {
        while (upto[s + 1] <= x) ++s;
        int P;
        PageList list;
        pages_of(s, P, list);
        const int held = p.held_len ? min(max(p.held_len[s], 0), P) / kPage : 0;
        const int kvh = (x - upto[s]) / list.count, v0 = (x - upto[s]) % list.count;
        const int v1 = min(list.count, v0 + (x_end - x));
        const int n_keys = P + p.T;
        const int low_min = window_low(P, p.window);         // some row may see positions from here on
        const int low_max = p.window > 0 ? window_low(P + p.T - 1, p.window) : low_min;       // every row does

        // ---- the item's queries and what they see ----
        asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory");      // the previous item's are no longer read
        for (int r = tid; r < 8 * NB; r += kWarps * 32) {
            RowMask rm;
            rm.low = 0x7fffffff;                             // rows that do not exist see nothing
            rm.bits[0] = rm.bits[1] = rm.bits[2] = rm.bits[3] = 0;
            if (r < PR) {
                const RowSight rs = row_sight(p.anc ? p.anc + (size_t)s * p.T * p.W : nullptr, p.causal, r / G, p.T, P, p.window, p.sinks);
                rm.low = rs.low;
                rm.bits[0] = (uint32_t)rs.bits[0]; rm.bits[1] = (uint32_t)(rs.bits[0] >> 32);
                rm.bits[2] = (uint32_t)rs.bits[1]; rm.bits[3] = (uint32_t)(rs.bits[1] >> 32);
            }
            mask[r].low = rm.low;
#pragma unroll
            for (int i = 0; i < 4; ++i) mask[r].bits[i] = rm.bits[i];
        }
        {
            constexpr int E = D / 32;                        // elements of a row that a lane stages: E * lane ..
            for (int r = warp; r < 8 * NB; r += kWarps) {
                float hi[E], lo[E];
#pragma unroll
                for (int e = 0; e < E; ++e) hi[e] = lo[e] = 0.f;
                if (r < PR) {
                    const size_t off = ((size_t)(s * p.T + r / G) * p.Hq + kvh * G + r % G) * D + lane * E;
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        hi[e] = __bfloat162float(p.q[off + e]);
                        if (two) lo[e] = __bfloat162float(p.q_lo[off + e]);
                    }
                }
                float top = 0.f;
#pragma unroll
                for (int e = 0; e < E; ++e) top = fmaxf(top, fabsf(hi[e]));
                top = warp_max(top);
                // 2^-x brings the row into [1, 2); exact, and undone in the score's scale
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

        float O[NB][MB][4], m[NB][2], l[NB][2];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            m[nb][0] = m[nb][1] = -INFINITY;
            l[nb][0] = l[nb][1] = 0.f;
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
        // O's rows: 4-bit pages: row g of block mb is d = (D/8) g + 2 mb, row g + 8 the next one; bf16 pages: 16 mb + g, + 8
        bool order4 = false;
        auto to_memory = [&](int nb, bool from4, float *dst) {       // dst [8 rows][ROWF]
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
                const int d0 = from4 ? (D / 8) * g + 2 * mb : 16 * mb + g, d1 = from4 ? d0 + 1 : d0 + 8;
                dst[(2 * t) * F::ROWF + d0] = O[nb][mb][0];
                dst[(2 * t + 1) * F::ROWF + d0] = O[nb][mb][1];
                dst[(2 * t) * F::ROWF + d1] = O[nb][mb][2];
                dst[(2 * t + 1) * F::ROWF + d1] = O[nb][mb][3];
            }
        };

        for (int v = v0; v < v1 && ok; ++v) {
            const int pg = list.page(v), key0 = pg * kPage;
            const bool open = key0 + kPage <= P && (key0 + kPage <= p.sinks || key0 >= low_max);     // every row sees all of it
            if (pg < held) {
                // ---------------- a page in 4 bits ----------------
                order4 = true;
                ok = mbar_wait(&bars.full[u % F::SLOTS], (uint32_t)(u / F::SLOTS) & 1u, abort_flag, p.status);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                const unsigned char *tile = ring + (u % F::SLOTS) * F::SUB;
                float c[NB][4];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) c[nb][0] = c[nb][1] = c[nb][2] = c[nb][3] = 0.f;
                {
                    constexpr int WORDS = D / 32;            // words of a key that a lane takes: d = (D/4) t ..
                    uint32_t wa[WORDS], wb[WORDS], sa, sb;
                    if constexpr (D == 128) {
                        const uint4 a = *reinterpret_cast<const uint4 *>(tile + code_at<D>(kA, t));
                        const uint4 b = *reinterpret_cast<const uint4 *>(tile + code_at<D>(kA + 8, t));
                        wa[0] = a.x; wa[1] = a.y; wa[2] = a.z; wa[3] = a.w;
                        wb[0] = b.x; wb[1] = b.y; wb[2] = b.z; wb[3] = b.w;
                        sa = *reinterpret_cast<const uint16_t *>(tile + Tile<D>::SCALES + kA * 8 + 2 * t);
                        sb = *reinterpret_cast<const uint16_t *>(tile + Tile<D>::SCALES + (kA + 8) * 8 + 2 * t);
                    } else {
                        const uint2 a = *reinterpret_cast<const uint2 *>(tile + code_at<D>(kA, t >> 1) + (t & 1) * 8);
                        const uint2 b = *reinterpret_cast<const uint2 *>(tile + code_at<D>(kA + 8, t >> 1) + (t & 1) * 8);
                        wa[0] = a.x; wa[1] = a.y;
                        wb[0] = b.x; wb[1] = b.y;
                        sa = tile[Tile<D>::SCALES + kA * 4 + t] * 0x101u;
                        sb = tile[Tile<D>::SCALES + (kA + 8) * 4 + t] * 0x101u;
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
                        for (int i = 0; i < 4; ++i) {
                            ha[i] = mul_half2(ha[i], ga);
                            hb[i] = mul_half2(hb[i], gb);
                        }
                        const uint32_t a0[4] = {ha[0], hb[0], ha[1], hb[1]}, a1[4] = {ha[2], hb[2], ha[3], hb[3]};
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb) {
                            const uint4 q = *reinterpret_cast<const uint4 *>(sQ + nb * F::QB + (w * 32 + lane) * 16);
                            mma<true>(c[nb], a0, q.x, q.y);
                            mma<true>(c[nb], a1, q.z, q.w);
                            if (two) {
                                const uint4 ql = *reinterpret_cast<const uint4 *>(sQ + (NB + nb) * F::QB + (w * 32 + lane) * 16);
                                mma<true>(c[nb], a0, ql.x, ql.y);
                                mma<true>(c[nb], a1, ql.z, ql.w);
                            }
                        }
                    }
                }
                uint32_t b[NB][2], blo[NB][2];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    const float s0 = mask[nb * 8 + 2 * t].scale16, s1 = mask[nb * 8 + 2 * t + 1].scale16;
                    if (!open) hide(c[nb], nb, key0);
                    bool raise;
                    float f[2];
                    softmax_tile<true>(c[nb], m[nb], l[nb], s0, s1, two, b[nb], blo[nb], raise, f);
                    if (raise) raise_acc(nb, f);
                }
                {
                    const unsigned char *vt = tile + Tile<D>::HALF;
                    constexpr int WORDS = D / 64;            // words of a key that a lane takes: d = (D/8) g ..
                    uint32_t w[4][WORDS], sc[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int key = ((k & 1) ? kV1 : kV0) + (k >> 1) * 8;
                        if constexpr (D == 128) {
                            const uint2 a = *reinterpret_cast<const uint2 *>(vt + code_at<D>(key, g >> 1) + (g & 1) * 8);
                            w[k][0] = a.x; w[k][1] = a.y;
                            sc[k] = vt[Tile<D>::SCALES + key * 8 + g];
                        } else {
                            w[k][0] = *reinterpret_cast<const uint32_t *>(vt + code_at<D>(key, g >> 2) + (g & 3) * 4);
                            sc[k] = vt[Tile<D>::SCALES + key * 4 + (g >> 1)];
                        }
                        if (!open && !see(key0 + key)) sc[k] = 0;      // what nobody sees may be anything, NaN included
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
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t a[4] = {mul_half2(e01[i], s01), mul_half2(o01[i], s01), mul_half2(e23[i], s23), mul_half2(o23[i], s23)};
#pragma unroll
                            for (int nb = 0; nb < NB; ++nb) {
                                mma<true>(O[nb][wi * 4 + i], a, b[nb][0], b[nb][1]);
                                if (two) mma<true>(O[nb][wi * 4 + i], a, blo[nb][0], blo[nb][1]);
                            }
                        }
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars.empty[u % F::SLOTS]);
                u += 1;
            } else {
                // ---------------- a page in bf16 ----------------
                for (; u % 3; ++u) {                         // the producer's way to the next place for a whole page
                    ok = ok && mbar_wait(&bars.full[u % F::SLOTS], (uint32_t)(u / F::SLOTS) & 1u, abort_flag, p.status);
                    ok = __all_sync(0xffffffffu, ok);
                    if (lane == 0) mbar_arrive(&bars.empty[u % F::SLOTS]);
                }
                ok = ok && mbar_wait(&bars.full[u % F::SLOTS], (uint32_t)(u / F::SLOTS) & 1u, abort_flag, p.status);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                if (order4) {                                // the accumulators so far to this page's order
                    order4 = false;
                    float *mine = red + warp * 8 * F::ROWF;
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        to_memory(nb, true, mine);
                        __syncwarp();
#pragma unroll
                        for (int mb = 0; mb < MB; ++mb) {
                            const int d0 = 16 * mb + g;
                            O[nb][mb][0] = mine[(2 * t) * F::ROWF + d0];
                            O[nb][mb][1] = mine[(2 * t + 1) * F::ROWF + d0];
                            O[nb][mb][2] = mine[(2 * t) * F::ROWF + d0 + 8];
                            O[nb][mb][3] = mine[(2 * t + 1) * F::ROWF + d0 + 8];
                        }
                        __syncwarp();
                    }
                }
                const uint32_t kbase = smem_u32(ring + (u % F::SLOTS) * F::SUB), vbase = kbase + kPage * D * 2;
                float c[NB][4];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) c[nb][0] = c[nb][1] = c[nb][2] = c[nb][3] = 0.f;
                // lane's row of the four 8 x 8 matrices it addresses
                const int mi = lane >> 3, r = warp * 16 + key_of(lane & 7);
#pragma unroll
                for (int j = 0; j < KS; ++j) {
                    // keys 0-7 | 8-15 of d 0-7, then of d 8-15
                    const int key = r + (mi & 1) * 8, ch = 2 * j + (mi >> 1);
                    uint32_t a[4];
                    ldmatrix4(kbase + (ch >> 3) * (kPage * 128) + key * 128 + (((ch & 7) ^ (key & 7)) << 4), a);
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        const uint2 q = *reinterpret_cast<const uint2 *>(sQ + (2 * NB + nb) * F::QB + ((j >> 1) * 32 + lane) * 16 + (j & 1) * 8);
                        mma<false>(c[nb], a, q.x, q.y);
                        if (two) {
                            const uint2 ql = *reinterpret_cast<const uint2 *>(sQ + (3 * NB + nb) * F::QB + ((j >> 1) * 32 + lane) * 16 + (j & 1) * 8);
                            mma<false>(c[nb], a, ql.x, ql.y);
                        }
                    }
                }
                uint32_t b[NB][2], blo[NB][2];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    if (!open) hide(c[nb], nb, key0);
                    bool raise;
                    float f[2];
                    softmax_tile<false>(c[nb], m[nb], l[nb], sl2, sl2, true, b[nb], blo[nb], raise, f);
                    if (raise) raise_acc(nb, f);
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
                if (lane < 3) mbar_arrive(&bars.empty[u % F::SLOTS + lane]);
                u += 3;
            }
        }

        // ---- the warps' parts meet; this CTA's part of the item, or all of it ----
        const int item = s * p.Hkv + kvh;
        const int first_x = x - v0, last_x = first_x + list.count - 1;       // the item's places in the line
        const int c_first = first_x / chunk, c_last = last_x / chunk, parts = c_last - c_first + 1;
        const int slot = 2 * (int)blockIdx.x + (first_x > x_begin ? 1 : 0);  // a CTA shares its first item, its last, or both
        const int rows = min(PR, 8 * NB);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int o = 4; o <= 16; o <<= 1) l[nb][r] += __shfl_xor_sync(0xffffffffu, l[nb][r], o);
            to_memory(nb, order4, red + warp * 8 * F::ROWF);
            if (g == 0) {
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    red_m[warp][2 * t + r] = m[nb][r];
                    red_l[warp][2 * t + r] = l[nb][r];
                }
            }
            asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory");
            for (int i = tid; i < 8 * (D / 4); i += kWarps * 32) {
                const int r = i / (D / 4), d0 = i % (D / 4) * 4, row = nb * 8 + r;
                float M = -INFINITY, L = 0.f;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) M = fmaxf(M, red_m[w][r]);
                float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < kWarps; ++w) {
                    const float f = red_m[w][r] == -INFINITY ? 0.f : ex2(red_m[w][r] - M);
                    const float4 a = *reinterpret_cast<const float4 *>(red + (w * 8 + r) * F::ROWF + d0);
                    L += f * red_l[w][r];
                    acc.x += f * a.x; acc.y += f * a.y; acc.z += f * a.z; acc.w += f * a.w;
                }
                if (row < rows) {
                    if (parts == 1) {
                        const float inv = L > 0.f ? 1.f / L : 0.f;
                        const size_t off = ((size_t)(s * p.T + row / G) * p.Hq + kvh * G + row % G) * D + d0;
                        store_two_term(p.out + off, p.out_lo ? p.out_lo + off : nullptr, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
                    } else {
                        *reinterpret_cast<float4 *>(p.parts + ((size_t)slot * kFewRows + row) * D + d0) = acc;
                        if (d0 == 0) reinterpret_cast<float2 *>(p.parts_ml)[(size_t)slot * kFewRows + row] = make_float2(M, L);
                    }
                }
            }
            asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory");
        }
        if (parts > 1) {
            __threadfence();
            asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory");
            if (tid == 0) {
                bars.last = atomicAdd(p.part_counters + item, 1) == parts - 1;
                if (bars.last) p.part_counters[item] = 0;    // for the next launch
                __threadfence();
            }
            asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory");
            if (bars.last) {
                for (int i = tid; i < rows * (D / 4); i += kWarps * 32) {
                    const int row = i / (D / 4), d0 = i % (D / 4) * 4;
                    // the part of the item's first CTA is its second one if another item came before
                    const int s_first = 2 * c_first + (first_x > c_first * chunk ? 1 : 0);
                    float M = -INFINITY, L = 0.f;
                    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
                    for (int c = 0; c < parts; ++c) {
                        const size_t at = (size_t)(c == 0 ? s_first : 2 * (c_first + c)) * kFewRows + row;
                        const float2 ml = __ldcg(reinterpret_cast<const float2 *>(p.parts_ml) + at);
                        const float4 a = __ldcg(reinterpret_cast<const float4 *>(p.parts + at * D + d0));
                        const float M2 = fmaxf(M, ml.x);
                        const float f0 = M == -INFINITY ? 0.f : ex2(M - M2), f1 = ml.x == -INFINITY ? 0.f : ex2(ml.x - M2);
                        M = M2;
                        L = L * f0 + ml.y * f1;
                        acc.x = acc.x * f0 + a.x * f1; acc.y = acc.y * f0 + a.y * f1;
                        acc.z = acc.z * f0 + a.z * f1; acc.w = acc.w * f0 + a.w * f1;
                    }
                    const float inv = L > 0.f ? 1.f / L : 0.f;
                    const size_t off = ((size_t)(s * p.T + row / G) * p.Hq + kvh * G + row % G) * D + d0;
                    store_two_term(p.out + off, p.out_lo ? p.out_lo + off : nullptr, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
                }
            }
        }
        x += v1 - v0;
    }
}

template <int D, int NB>
cudaError_t launch_few(const AttnParams &p, const CUtensorMap &map_kv, cudaStream_t st) {
    using F = Few<D, NB>;
    static bool once = false;
    if (!once) {
        const cudaError_t e = cudaFuncSetAttribute(attn_few_kernel<D, NB>, cudaFuncAttributeMaxDynamicSharedMemorySize, F::TOTAL);
        if (e != cudaSuccess) return e;
        once = true;
    }
    cudaLaunchConfig_t cfg = {};
    // no more CTAs than pages that a row can see: the lengths themselves are on the device
    long long pages = p.geom.max_pages_per_seq;
    if (p.window > 0) pages = std::min(pages, ((long long)p.window + p.T + kPage - 1) / kPage + 1 + ((long long)p.sinks + kPage - 1) / kPage);
    cfg.gridDim = dim3((unsigned)std::min<long long>(148 * F::CTAS, pages * p.Hkv * p.batch), 1, 1);
    cfg.blockDim = dim3(kFewThreads, 1, 1);
    cfg.dynamicSmemBytes = F::TOTAL;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, attn_few_kernel<D, NB>, map_kv, p, 1);
}

}  // namespace

bool attention_few_takes(int T, int G) { return (long long)T * G <= kFewRows; }

cudaError_t launch_attention_few(const AttnParams &p, const CUtensorMap &map_kv, cudaStream_t st) {
    const int rows = p.T * (p.Hq / p.Hkv);
    if (p.d == 128) {
        if (rows <= 8) return launch_few<128, 1>(p, map_kv, st);
        if (rows <= 16) return launch_few<128, 2>(p, map_kv, st);
        return launch_few<128, 4>(p, map_kv, st);
    }
    if (rows <= 8) return launch_few<64, 1>(p, map_kv, st);
    if (rows <= 16) return launch_few<64, 2>(p, map_kv, st);
    return launch_few<64, 4>(p, map_kv, st);
}

}  // namespace glance
