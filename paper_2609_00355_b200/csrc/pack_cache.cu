// Moves finished pages of the target's cache into the 4-bit pool and back (format: packed.cuh).
//
// HBM-bound: 2 bytes of a value are read and 9/16 of one written, or the other way round.  One wave of blocks takes the tiles
// (layer, page, kv head, K|V) in turn; which pages are due is worked out from the device-resident lengths by every block.  A
// lane takes one group of 16 values: one 32-byte load, the scale, eight conversions, one 8-byte store; the loads of a
// thread's next tile are in flight while it converts, and the page numbers of the one after it.  The block that is the last to
// have read the lengths publishes the new ones (nothing else in the launch reads what it writes), so nobody waits for the copies.
// Measured: 8704 positions of 28 layers (4 kv heads, d 128), 635 MB each way: 112 us to pack, 109 back (5.7 TB/s), 214 both in one
// graph; with a division a value, 16-byte accesses and page numbers looked up when due 158 and 144.
#include <cuda_fp8.h>

#include "kernels.cuh"
#include "packed.cuh"
#include "tc_ptx.cuh"

namespace glance {

namespace {

using namespace packed;

constexpr int kPackThreads = 256;
constexpr int kPackBlocks = 4;   // an SM
constexpr int kMaxSeqs = 64;

__device__ __forceinline__ int whole_pages(int n) { return max(n, 0) / kPage; }

// e4m3 of a / 6 for a = max|x| >= 0.  a has eight significant bits, so a / 6 is a border of e4m3 exactly or at least 2^-9 of
// itself away from one: rounding the product with 1 / 6 (off by 2^-23) to 12 bits (Veltkamp's splitting) makes borders exact again.
__device__ __forceinline__ uint32_t scale_code(float a) {
    const float q = fminf(a * (1.f / 6.f), 1024.f);      // (saturates at 448)
    const float wide = __fmul_rn(q, 4097.f), twelve = __fsub_rn(wide, __fsub_rn(wide, q));
    uint32_t r;
    asm("{\n\t.reg .b16 x;\n\tcvt.rn.satfinite.e4m3x2.f32 x, %1, %2;\n\tcvt.u32.u16 %0, x;\n\t}" : "=r"(r) : "f"(0.f), "f"(twelve));
    return r & 0xffu;
}
// e2m1 of x / s for the eight values of four words, first value in the lowest nibble; r = 1 / s rounded.  A quotient of an eight-bit
// and a four-bit significand is a border of e2m1 (an odd multiple of 1/4, 1/2 or 1) exactly or at least 2^-10 away from one.
// So it may be rounded to a multiple of 2^-13, which undoes the rounding of r (one place: 2^-19 at most where it matters) and
// keeps ties ties.
__device__ __forceinline__ uint32_t value_codes(const uint32_t (&w)[4], float r) {
    constexpr float kGrid = 1536.f;                      // 1.5 * 2^10: its last place is 2^-13
    const float2 r2 = make_float2(r, r), up = make_float2(kGrid, kGrid), down = make_float2(-kGrid, -kGrid);
    float2 q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        q[i] = tc::add2(tc::fma2(make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u)), r2, up), down);
    uint32_t c;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(c) : "f"(q[0].x), "f"(q[0].y), "f"(q[1].x), "f"(q[1].y), "f"(q[2].x), "f"(q[2].y), "f"(q[3].x), "f"(q[3].y));
    return c;
}

// A group's 32 bytes of bf16 in one access: as two of 16 a warp's accesses would cover half of every sector each time.
__device__ __forceinline__ void load32(const void *p, uint4 (&v)[2]) {
    asm volatile("ld.global.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(v[0].x), "=r"(v[0].y), "=r"(v[0].z), "=r"(v[0].w), "=r"(v[1].x), "=r"(v[1].y), "=r"(v[1].z), "=r"(v[1].w) : "l"(p) : "memory");
}
__device__ __forceinline__ void store32(void *p, const uint4 (&v)[2]) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 ::"l"(p), "r"(v[0].x), "r"(v[0].y), "r"(v[0].z), "r"(v[0].w), "r"(v[1].x), "r"(v[1].y), "r"(v[1].z), "r"(v[1].w) : "memory");
}

// 16 bf16 values -> 8 bytes of codes and the scale's code
__device__ __forceinline__ uint2 pack_group(const uint4 (&v)[2], uint32_t &scale) {
    const uint32_t w[2][4] = {{v[0].x, v[0].y, v[0].z, v[0].w}, {v[1].x, v[1].y, v[1].z, v[1].w}};
    uint32_t both = 0;                                   // the largest magnitude, by its bits
#pragma unroll
    for (int i = 0; i < 8; ++i) both = __vmaxu2(both, w[i >> 2][i & 3] & 0x7fff7fffu);
    const uint32_t top = max(both & 0xffffu, both >> 16);
    scale = top >= 0x7f80u ? 0x7fu : scale_code(__uint_as_float(top << 16));
    __half_raw h = __nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)scale, __NV_E4M3);
    const float s = __half2float(__half(h));
    const bool live = s > 0.f;                           // a scale of 0 or NaN: codes 0
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));
    const uint2 out = make_uint2(value_codes(w[0], r), value_codes(w[1], r));
    return live ? out : make_uint2(0u, 0u);
}

__device__ __forceinline__ void unpack_group(uint2 c, uint32_t scale, uint4 (&v)[2]) {
    const uint32_t s = scales_to_half(scale | scale << 8);
    uint32_t h[4], r[8];
    codes_to_half(c.x, h);
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = half2_to_bf16(mul_half2(h[i], s));
    codes_to_half(c.y, h);
#pragma unroll
    for (int i = 0; i < 4; ++i) r[4 + i] = half2_to_bf16(mul_half2(h[i], s));
    v[0] = make_uint4(r[0], r[1], r[2], r[3]);
    v[1] = make_uint4(r[4], r[5], r[6], r[7]);
}

template <int D, bool BACK>
__global__ void __launch_bounds__(kPackThreads, kPackBlocks) pack_kernel(PackParams p) {
    constexpr int GROUPS = Tile<D>::GROUPS;
    __shared__ int sh_first[kMaxSeqs], sh_upto[kMaxSeqs + 1], sh_len[kMaxSeqs];      // first page due, pages due up to here, new length in pages
    __shared__ int sh_ticket;
    const int t = threadIdx.x, cap = p.geom.max_pages_per_seq;
    if (t < p.batch) {
        const int seen = max(p.seq_len[t], 0);
        const int have = min(min(whole_pages(p.len[t]), whole_pages(seen)), cap);      // a length beyond seq_len counts for nothing
        int lo, hi;
        if (BACK) {
            lo = min(whole_pages(p.new_len[t]), have);
            hi = have;
            sh_len[t] = lo;
        } else {
            lo = have;
            hi = max(min(whole_pages(seen - p.keep), cap), have);
            sh_len[t] = hi;
            if (whole_pages(seen) > cap) set_status(p.status, GLANCE_E_CAPACITY);
        }
        sh_first[t] = lo;
        sh_upto[t + 1] = hi - lo;
    }
    __syncthreads();
    if (t < 32) {                                        // prefix sums
        int run = 0;
        for (int s0 = 0; s0 < p.batch; s0 += 32) {
            int n = s0 + t < p.batch ? sh_upto[s0 + t + 1] : 0;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, n, o);
                if (t >= o) n += v;
            }
            if (s0 + t < p.batch) sh_upto[s0 + t + 1] = run + n;
            run += __shfl_sync(0xffffffffu, n, 31);
        }
        if (t == 0) sh_upto[0] = 0;
    }
    __syncthreads();
    // counted in: this block has read the lengths (the answer is looked at when its tiles are done)
    int ticket = 0;
    if (t == 0) ticket = atomicAdd(p.counter, 1);

    const unsigned pages = (unsigned)sh_upto[p.batch], H2 = 2u * (unsigned)p.geom.n_kv_heads;
    const size_t layer4 = (size_t)p.n_pages4 * p.geom.n_kv_heads * Tile<D>::BYTES;
    // item: layer, page, (head, K|V)
    const unsigned items = pages * H2 * (unsigned)p.n_layers;
    constexpr int STEPS = kPage * GROUPS / kPackThreads;
    static_assert(kPage * GROUPS % kPackThreads == 0, "whole steps");
    struct Item {
        bf16 *rows;              // nullptr: nothing to move
        unsigned char *tile;
    };
    auto placed = [&](int from, int at4) { return from >= 0 && from < p.geom.n_pages && at4 >= 0 && at4 < p.n_pages4; };
    auto find = [&](unsigned it) {
        Item r{nullptr, nullptr};
        if (it >= items) return r;
        const unsigned kvh = it % H2, rest = it / H2, pg = rest % pages, layer = rest / pages;
        const int kv = (int)(kvh & 1u), head = (int)(kvh >> 1);
        int s = 0;
        while ((unsigned)sh_upto[s + 1] <= pg) ++s;
        const size_t entry = (size_t)s * cap + sh_first[s] + (int)pg - sh_upto[s];
        const int from = p.page_table[entry], at4 = p.page_table4[entry];
        if (!placed(from, at4)) {
            if (t == 0) set_status(p.status, GLANCE_E_BOUNDS);
            return r;
        }
        r.rows = p.kv_pool + (size_t)layer * p.geom.layer_stride() + p.geom.row(from, kv, head, 0);
        r.tile = p.pool4 + layer * layer4 + ((size_t)at4 * p.geom.n_kv_heads + head) * Tile<D>::BYTES + kv * Tile<D>::HALF;
        return r;
    };
    struct Data {
        uint4 v[STEPS][BACK ? 1 : 2];                    // two pieces of a row, or (way back) 8 bytes of codes and the scale
    };
    auto load = [&](const Item &it, Data &d) {
        if (!it.rows) return;
#pragma unroll
        for (int u = 0; u < STEPS; ++u) {
            const int g = u * kPackThreads + t;
            if constexpr (!BACK) {
                load32(it.rows + (size_t)g * kGroup, d.v[u]);
            } else {
                const int key = g / GROUPS, c = g % GROUPS;
                const uint2 codes = __ldcs(reinterpret_cast<const uint2 *>(it.tile + code_at<D>(key, c >> 1) + (c & 1) * 8));
                d.v[u][0] = make_uint4(codes.x, codes.y, it.tile[Tile<D>::SCALES + g], 0u);
            }
        }
    };
    // The next item's loads are issued, and the page numbers of the one after it looked up, before this one's are converted.
    Data now;
    Item item = find(blockIdx.x);
    load(item, now);
    // A page that has no place in one of the pools stays, and positions held in 4 bits are a prefix: a length rises to the first such
    // page only, and falls to behind the last one (what moves on the far side is not read there).  Every block looks at every entry
    // due while its first tile is on its way, 8 bytes a page for at least 20 KB that move: no time that was measured with one page
    // or many, 1 % with 84 pages of a small model; before the first tile's loads it took 0.5 us a launch.
    for (int pg = t, s = 0; pg < (int)pages; pg += kPackThreads) {
        while (sh_upto[s + 1] <= pg) ++s;
        const int at = sh_first[s] + pg - sh_upto[s];
        const size_t entry = (size_t)s * cap + at;
        if (placed(p.page_table[entry], p.page_table4[entry])) continue;
        if (BACK) atomicMax(&sh_len[s], at + 1);
        else atomicMin(&sh_len[s], at);
    }
    Item following = find(blockIdx.x + gridDim.x);
    for (unsigned it = blockIdx.x; it < items; it += gridDim.x) {
        Data next;
        load(following, next);
        const Item after = find(it + 2 * gridDim.x);
        if (item.rows) {
#pragma unroll
            for (int u = 0; u < STEPS; ++u) {
                const int g = u * kPackThreads + t, key = g / GROUPS, c = g % GROUPS;
                if constexpr (!BACK) {
                    uint32_t scale;
                    const uint2 codes = pack_group(now.v[u], scale);
                    *reinterpret_cast<uint2 *>(item.tile + code_at<D>(key, c >> 1) + (c & 1) * 8) = codes;
                    // four neighbours' scales in one store
                    uint32_t four = scale << (8 * (t & 3));
                    four |= __shfl_xor_sync(0xffffffffu, four, 1);
                    four |= __shfl_xor_sync(0xffffffffu, four, 2);
                    if ((t & 3) == 0) *reinterpret_cast<uint32_t *>(item.tile + Tile<D>::SCALES + g) = four;
                } else {
                    uint4 v[2];
                    unpack_group(make_uint2(now.v[u][0].x, now.v[u][0].y), now.v[u][0].z, v);
                    store32(item.rows + (size_t)g * kGroup, v);
                }
            }
        }
        item = following;
        following = after;
        now = next;
    }
    // the block that counted itself in last publishes the new lengths: every block has read the old ones
    if (t == 0) sh_ticket = ticket;
    __syncthreads();
    if (sh_ticket == (int)gridDim.x - 1) {
        if (t == 0) *p.counter = 0;                      // for the next launch
        if (t < p.batch) p.len[t] = sh_len[t] * kPage;
    }
}

}  // namespace

void launch_pack(const PackParams &p, bool back, cudaStream_t st) {
    // one wave; a block strides over the tiles
    const long long most = (long long)p.batch * p.geom.max_pages_per_seq * p.n_layers * p.geom.n_kv_heads * 2;
    const int blocks = (int)(most < 148 * kPackBlocks ? most : 148 * kPackBlocks);
    if (p.geom.head_dim == 128) {
        if (back) pack_kernel<128, true><<<blocks, kPackThreads, 0, st>>>(p);
        else pack_kernel<128, false><<<blocks, kPackThreads, 0, st>>>(p);
    } else {
        if (back) pack_kernel<64, true><<<blocks, kPackThreads, 0, st>>>(p);
        else pack_kernel<64, false><<<blocks, kPackThreads, 0, st>>>(p);
    }
}

}  // namespace glance
