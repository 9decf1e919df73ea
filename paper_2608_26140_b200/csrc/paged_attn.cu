// Attention of few query rows over a cache in pages.
//
//   o_r = sum_j p_rj V_j / sum_j p_rj,   p_rj = 2^(x_rj - M_r),   x_rj = log2(e) / sqrt(d) q_r K_j
//
// in one pass over the keys, M_r a running reference.  Keys and values are the long sides of both products,
//   S^T = K Q^T (keys x rows),   O^T += V^T P^T (d x rows),
// so that up to 8 rows (the query heads of a KV head, times the tokens) cost one matrix instruction for every 16 keys and 16 d; P only has
// to be transposed in 8 x 8 blocks (movmatrix).  P is rounded to bf16, as V is: 2^-8 of each probability at most; its sum is not.
//
// The work of all requests, KV heads and row tiles is one line of units of 64 keys (and a few behind each item's for what it costs by itself), cut into
// equal pieces, one a CTA, whatever the requests' lengths (they are known on the device only).  A CTA that does not have all keys of an item leaves a partial result
// and the last one to arrive adds the parts up, in their order.  Where there is too little for that, a cluster of CTAs has an item to itself.
// A warp streams 16 keys a step through a ring of its own in shared memory (cp.async, whole rows side by side, the page's number asked for two
// steps ahead), swizzled so that ldmatrix meets different banks.  Keys that do not count are not read: their places are zero.
//
// Up to 8 rows HBM bounds it: one token of 2 requests over 65537 keys of 32 heads (2148 MB) 305 us, 7.0 TB/s; of 64 requests over up to 8191 keys of
// 4 KV heads (794 MB) 121 us, 6.6 TB/s.  32 rows of 16 requests over 2560 keys of 32 heads, of which 2048 are the same pages for all, 103 us (8 rows 57, 16 69, 24
// 87): a step takes a warp 2000 clocks, two warps a scheduler that wait for their own results (issue slots 33 %, tensor pipe 41 % busy), 6.5 TB/s from L2; starts and ends
// of items are a fifth.  The fragments of a step's next product are asked for before the last one's products (108 without).  One token of one request over 1664 keys 7.5 us: four trips to memory one behind the other (arguments, page, keys, result) and a cluster's exchange.
//
// More than 32 rows of a KV head are tiles of 32, each of which reads all keys again, through L2 where they fit: 32 tokens on 28 query and 4 KV heads (224 rows, 7 tiles)
// of 16 requests over 2560 keys 94 us (floor 14: bytes and operations), of 32 requests over 8000 keys 424 (82; one token of each 104); a refresh of 16 x 922 rows
// over 2560 keys 2.9 ms on 32 KV heads (floor 0.37), 2.4 on 4.  215 to 277 TFLOP/s, the rate of one tile of 32 rows:
// nothing is gained from there being many.  Tiles of 128 rows on tcgen05, as the contiguous and the 8-bit cache have, are not written for pages.
#include <algorithm>
#include <climits>

#include "kernels.h"
#include "kv8.cuh"
#include "launch.h"
#include "per_device.h"
#include "tc_ptx.cuh"

namespace acache {
namespace {

constexpr int PW = 4;                    // warps of a CTA
constexpr int PSTEP = 16;                // keys of a warp's step
constexpr int PSTAGES = 3;
constexpr int kUnit = PW * PSTEP;        // keys of a unit of work
constexpr int kMinUnits = 2;             // fewest units that are worth a CTA
// What an item costs besides its keys (start, queries, joining the warps; 4.5 us beside units of 1.5), in units.  Without it a CTA may get a whole run of short
// requests' items, each of one unit: one token and 32 rows of 32 requests over 40 to 4000 keys of 32 heads 270 and 502 us; with 2 units 145 and 237, 3 141 and
// 197, 5 141 and 157, 8 140 and 158; 64 requests over 300 keys 62, 41, 40.5, 41.5, 43.
template <int NT>
constexpr unsigned kItemUnits = NT > 2 ? 5u : 3u;
constexpr int kPlaces = 2 * 148;         // CTAs that run at a time
static_assert(kPlaces <= kKv8Counters, "a counter for every CTA that an item may begin in");
constexpr float kPagedRaise = 8.f;       // M moves when a logit passes it by this (log2): P and sums stay within 2^8 of what they are with M the largest

__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ void cp_async16_or_zero(uint32_t dst, const void* src, bool on) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(dst), "l"(src) : "memory");
}
// the products' first step: nothing to add to
__device__ __forceinline__ void mma_bf16_16816_first(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
        "{%10,%10,%10,%10};\n"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
template <int N>
__device__ __forceinline__ void ring_wait() { asm volatile("cp.async.wait_group %0;\n" ::"n"(N) : "memory"); }

template <int D, int NT>
struct PagedLayout {
    static constexpr int ROWS = 8 * NT;
    static constexpr int HALF = PSTEP * D * 2;               // bytes of a stage's keys, then its values
    static constexpr int STAGE = 2 * HALF;
    static constexpr int RING = PW * PSTAGES * STAGE;
    static constexpr int MERGE = PW * ROWS * (D + 4) * 4;    // the warps' results, in the ring's place
    static constexpr int QS = (D / 16) * NT * 32 * 8;        // the queries as fragments
    static constexpr int RESULT = ROWS * D * 4;              // behind them, what a cluster's other CTAs read
    static constexpr int SMEM = (RING > MERGE + RESULT ? RING : MERGE + RESULT) + QS;
};

// Units of a request's items (row tile and KV head): one for an empty request too, which has outputs like any other.
__device__ __forceinline__ int units_of(int len) { return max(1, (len + kUnit - 1) / kUnit); }

template <int D, int NT>
__global__ void __launch_bounds__(PW * 32, 2) paged_attn_kernel(const PagedAttnArgs a) {
    using L = PagedLayout<D, NT>;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ float stat[2][PW][8 * NT];                    // references, denominators
    __shared__ uint32_t there_of[PW][PSTAGES];               // a stage's keys that count
    __shared__ unsigned sums[PW], at_request[2];             // (request, first unit of it) that this CTA begins with
    __shared__ int is_last;
    __shared__ float4 factor[8 * NT];
    __shared__ float lse2_of[8 * NT], lse_of[L::RING / (D * 4)];
    static_assert(PW == 4, "a factor for every warp");
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    pdl_wait();
    pdl_launch_dependents();
    const unsigned extra = a.cluster ? 0u : kItemUnits<NT>;     // units behind an item's that stand for no keys
    const int hkv = a.n_kv_heads, G = a.group, R = a.n * G, tiles = (R + L::ROWS - 1) / L::ROWS, per_request = hkv * tiles;
    uint2* qs = reinterpret_cast<uint2*>(smem + L::SMEM - L::QS);

    // where row r of KV head kvh of request b lies: query row r / G, head kvh G + r % G
    auto place_of = [&](int b, int kvh, int r) {
        const int i = a.group_inverse ? (int)__umulhi((unsigned)r, a.group_inverse) : G == 1 ? r : r / G;
        return (int64_t)(b * (int64_t)a.n + i) * a.n_heads + kvh * G + (r - i * G);
    };

    // ---- this CTA's share of the units ----
    auto len_of = [&](int b) { return a.lens ? min(max(a.lens[b], 0), a.ctx_len) : a.ctx_len; };
    unsigned base, rest;                                     // CTA c takes base units, the first `rest` ones one more
    int ctas;                                                // that have work
    auto first_of = [&](int c) { return (unsigned)c * base + min((unsigned)c, rest); };
    auto cta_of = [&](unsigned unit) { return unit < rest * (base + 1u) ? unit / (base + 1u) : rest + (unit - rest * (base + 1u)) / base; };
    auto share = [&](unsigned units) {
        ctas = (int)min(gridDim.x, max(1u, units / kMinUnits));
        base = units / (unsigned)ctas;
        rest = units - base * (unsigned)ctas;
    };
    int b;
    unsigned b_lo = 0u;                                      // first unit of request b
    unsigned unit, mine_hi;
    int cluster_item = 0;                                    // in a cluster: the item of request b that its CTAs share
    if (a.cluster) {
        const int item = blockIdx.x / a.cluster, rank = blockIdx.x % a.cluster;
        b = item / per_request;
        cluster_item = item - b * per_request;
        const unsigned units = units_of(len_of(b));
        unit = cluster_item * units + units * rank / a.cluster;
        mine_hi = cluster_item * units + units * (rank + 1) / a.cluster;
        if (a.lens && cluster_item == 0 && rank == 0 && tid == 0 && a.lens[b] != len_of(b)) atomicOr(a.status, kFlagBadIndex);
    } else if (!a.lens) {
        const unsigned u = (units_of(a.ctx_len) + extra) * per_request;
        share(u * a.batch);
        if ((int)blockIdx.x >= ctas) return;
        b = (int)(first_of(blockIdx.x) / u);
        b_lo = u * b;
    } else {
        // the threads count the units of equal runs of requests; the one whose run holds the first unit of the share finds its request
        const int run = (a.batch + PW * 32 - 1) / (PW * 32), r0 = min(tid * run, a.batch), r1 = min(r0 + run, a.batch);
        unsigned sum = 0u;
#pragma unroll 1
        for (int r = r0; r < r1; ++r) {
            const int len = a.lens[r];
            if (blockIdx.x == 0 && (len < 0 || len > a.ctx_len)) atomicOr(a.status, kFlagBadIndex);
            sum += (units_of(min(max(len, 0), a.ctx_len)) + extra) * per_request;
        }
        unsigned upto = sum;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const unsigned v = __shfl_up_sync(0xffffffffu, upto, off);
            if (lane >= off) upto += v;
        }
        if (lane == 31) sums[warp] = upto;
        __syncthreads();
        unsigned all = 0u;
#pragma unroll
        for (int w = 0; w < PW; ++w) {
            if (w == warp) upto += all;
            all += sums[w];
        }
        share(all);
        if ((int)blockIdx.x >= ctas) return;
        unsigned lo = upto - sum;
        const unsigned mine = first_of(blockIdx.x);
        if (lo <= mine && mine < upto) {
            int r = r0;
#pragma unroll 1
            for (; r < r1 - 1; ++r) {
                const unsigned u = (units_of(len_of(r)) + extra) * per_request;
                if (mine < lo + u) break;
                lo += u;
            }
            at_request[0] = (unsigned)r;
            at_request[1] = lo;
        }
        __syncthreads();
        b = (int)at_request[0];
        b_lo = at_request[1];
    }
    if (!a.cluster) {
        unit = first_of(blockIdx.x);
        mine_hi = first_of(blockIdx.x + 1);
    }

    const int page_mask = (1 << a.pages.log2_page) - 1;
    const bool whole = a.pages.log2_page >= 4;               // a step's keys lie in one page
    const __nv_bfloat16 *kp = static_cast<const __nv_bfloat16*>(a.k), *vp = static_cast<const __nv_bfloat16*>(a.v);
    constexpr int PIECES = D / 8;                            // 16-byte pieces of a row
    constexpr int PASS = 32 / PIECES, PASSES = PSTEP / PASS;
    const int row0 = lane / PIECES, piece = lane % PIECES;
    const uint32_t ring = smem_u32(smem) + warp * (PSTAGES * L::STAGE);
    constexpr int SWIZZLES = 8 / PASS;                       // a row's pieces are swizzled by its number modulo 8; the pass i is PASS rows further
    uint32_t put[SWIZZLES];
#pragma unroll
    for (int i = 0; i < SWIZZLES; ++i) put[i] = ring + row0 * D * 2 + ((piece ^ row0 ^ (i * PASS)) << 4);
    const int mrow = lane & 7, mj = lane >> 3;               // ldmatrix: this lane's row of the matrix mj
    const uint32_t k_get = ((mj & 1) * 8 + mrow) * D * 2 + (((mj >> 1) ^ mrow) << 4);
    const uint32_t v_get = L::HALF + ((mj >> 1) * 8 + mrow) * D * 2 + (((mj & 1) ^ mrow) << 4);

    for (;;) {
        // ---- the item and this CTA's keys of it ----
        int len = len_of(b);
        unsigned units = units_of(len);
        while (!a.cluster && unit >= b_lo + (units + extra) * per_request) {
            b_lo += (units + extra) * per_request;
            ++b;
            len = len_of(b);
            units = units_of(len);
        }
        const int item = a.cluster ? cluster_item : (int)((unit - b_lo) / (units + extra)), kvh = tiles == 1 ? item : item / tiles, tile = item - kvh * tiles;
        const unsigned item_lo = b_lo + (unsigned)item * (units + extra), item_hi = item_lo + units, seg_hi = min(item_hi, mine_hi);
        if (!a.cluster && unit >= item_hi) {                 // the others have all its keys
            unit = item_hi + extra;
            if (unit >= mine_hi) return;
            continue;
        }
        const int key_lo = (int)(unit - item_lo) * kUnit, key_hi = min(len, (int)(seg_hi - item_lo) * kUnit);
        const int steps = max(0, (key_hi - key_lo + PSTEP - 1) / PSTEP), my_steps = (steps - warp + PW - 1) / PW;
        const int32_t* table = a.pages.table + (int64_t)b * a.pages.table_stride;

        __syncthreads();                                     // nobody reads the last item's results or queries any more
        // ---- the ring ----
        // page of this lane's key, and the bits of keys that do not exist, of the next two steps to be fetched
        int entry = 0, entry2 = 0;
        uint32_t drop = 0u, drop2 = 0u;
        auto look_up = [&](int s, int& e, uint32_t& d) {
            if (s >= my_steps) return;
            const int key0 = key_lo + (warp + s * PW) * PSTEP, key = key0 + (whole ? 0 : lane & 15);
            e = key < key_hi ? __ldg(table + (key >> a.pages.log2_page)) : 0;
            d = a.key_drop ? __ldg(a.key_drop + (int64_t)b * a.drop_words + (key0 >> 5)) >> (key0 & 16) : 0u;
        };
        auto fetch = [&](int s, int stage) {
            if (s < my_steps) {
                const int key0 = key_lo + (warp + s * PW) * PSTEP, left = key_hi - key0;
                const bool good = entry >= 0 && entry < a.pages.n_pages;
                uint32_t there = (left >= PSTEP ? 0xFFFFu : (1u << left) - 1u) & ~drop;
                const uint32_t known = whole ? (good ? 0xFFFFu : 0u) : __ballot_sync(0xffffffffu, good);
                if ((there & ~known) != 0u) {                // keys in pages that are none do not count
                    if (lane == 0) atomicOr(a.status, kFlagBadIndex);
                    there &= known;
                }
                if (lane == 0) there_of[warp][stage] = there;
                const int64_t off = (good ? entry * a.pages.page_stride : 0) +
                                    (((int64_t)kvh << a.pages.log2_page) + ((key0 + (whole ? 0 : lane & 15)) & page_mask)) * D;
                if (whole && there == 0xFFFFu) {             // side by side
                    const __nv_bfloat16 *kf = kp + off + row0 * D + piece * 8, *vf = vp + off + row0 * D + piece * 8;
#pragma unroll
                    for (int i = 0; i < PASSES; ++i) {
                        const uint32_t dst = put[i % SWIZZLES] + stage * L::STAGE + i * PASS * D * 2;
                        cp_async16(dst, kf + i * PASS * D);
                        cp_async16(dst + L::HALF, vf + i * PASS * D);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < PASSES; ++i) {
                        const int row = i * PASS + row0;
                        const int64_t at = (whole ? off + row * D : __shfl_sync(0xffffffffu, off, row)) + piece * 8;
                        const bool on = (there >> row) & 1u;
                        const uint32_t dst = put[i % SWIZZLES] + stage * L::STAGE + i * PASS * D * 2;
                        cp_async16_or_zero(dst, kp + at, on);
                        cp_async16_or_zero(dst + L::HALF, vp + at, on);
                    }
                }
            }
            cp_async_commit();
        };
        look_up(0, entry, drop);
        look_up(1, entry2, drop2);
        int ahead = 0;                                       // the next step to be fetched
        auto advance = [&](int stage) {
            fetch(ahead, stage);
            entry = entry2; drop = drop2;
            look_up(ahead + 2, entry2, drop2);
            ++ahead;
        };
#pragma unroll 1
        while (ahead < PSTAGES - 1) advance(ahead);
        // ---- queries as fragments, the rows dealt out to the warps ----
        constexpr int FRAGS = (D / 16) * NT, PER_WARP = (FRAGS + PW - 1) / PW;
        {
            uint2 q[PER_WARP];
#pragma unroll
            for (int i = 0; i < PER_WARP; ++i) {
                const int f = warp + i * PW, r = tile * L::ROWS + (f % NT) * 8 + g;
                q[i] = make_uint2(0u, 0u);
                if (f < FRAGS && r < R) {
                    const uint32_t* from = reinterpret_cast<const uint32_t*>(static_cast<const __nv_bfloat16*>(a.q) + place_of(b, kvh, r) * D + f / NT * 16);
                    q[i] = make_uint2(__ldg(from + t), __ldg(from + t + 4));
                }
            }
#pragma unroll
            for (int i = 0; i < PER_WARP; ++i)
                if (warp + i * PW < FRAGS) qs[(warp + i * PW) * 32 + lane] = q[i];
        }
        __syncthreads();                                     // the queries are there

        constexpr bool Q_REGS = NT * D <= 256;
        uint2 qf[Q_REGS ? D / 16 : 1][Q_REGS ? NT : 1];
        if constexpr (Q_REGS) {
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) qf[ks][nt] = qs[(ks * NT + nt) * 32 + lane];
        }
        float o[D / 16][NT][4];
        float2 m[NT], l[NT];                                 // references, denominators of rows 2 t, 2 t + 1
        unsigned unset = (1u << (2 * NT)) - 1u;              // rows without a reference yet (no key, or none with a logit above -inf)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            m[nt] = l[nt] = make_float2(0.f, 0.f);
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[i][nt][j] = 0.f;
        }
        int stage = 0;                                       // step % PSTAGES
        for (int s = 0; s < my_steps; ++s) {
            const uint32_t st = ring + stage * L::STAGE;
            ring_wait<PSTAGES - 2>();
            __syncwarp();                                    // this step's stage is there for every lane, and every lane is done with the last one's
            const uint32_t there = there_of[warp][stage];
            advance(stage == 0 ? PSTAGES - 1 : stage - 1);
            stage = stage == PSTAGES - 1 ? 0 : stage + 1;
            if (there == 0u) continue;
            // ---- S^T = K Q^T ----
            float sv[NT][4];
            uint32_t fa[2][4];
            uint2 fq[2][NT];
            auto get = [&](int ks) {
                ldmatrix_x4(fa[ks & 1][0], fa[ks & 1][1], fa[ks & 1][2], fa[ks & 1][3], st + (k_get ^ (ks << 5)));
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    if constexpr (Q_REGS) fq[ks & 1][nt] = qf[ks][nt];
                    else fq[ks & 1][nt] = qs[(ks * NT + nt) * 32 + lane];
                }
            };
            get(0);
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                if (ks + 1 < D / 16) get(ks + 1);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const uint2 q = fq[ks & 1][nt];
                    if (ks == 0) mma_bf16_16816_first(sv[nt], fa[ks & 1], q.x, q.y);
                    else mma_bf16_16816(sv[nt], fa[ks & 1], q.x, q.y);
                }
            }
            const float2 scale2 = make_float2(a.scale_log2e, a.scale_log2e);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 4; j += 2) {
                    const float2 y = __ffma2_rn(make_float2(sv[nt][j], sv[nt][j + 1]), scale2, make_float2(-m[nt].x, -m[nt].y));
                    sv[nt][j] = y.x;
                    sv[nt][j + 1] = y.y;
                }
            if (there != 0xFFFFu) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (!((there >> ((j >> 1) * 8 + g)) & 1u))
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) sv[nt][j] = -INFINITY;
            }
            float top = fmaxf(fmaxf(sv[0][0], sv[0][1]), fmaxf(sv[0][2], sv[0][3]));
#pragma unroll
            for (int nt = 1; nt < NT; ++nt) top = fmaxf(fmaxf(fmaxf(fmaxf(top, sv[nt][0]), sv[nt][1]), sv[nt][2]), sv[nt][3]);
            if (__any_sync(0xffffffffu, top > kPagedRaise || unset != 0u)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        float x = fmaxf(sv[nt][r], sv[nt][r + 2]);
                        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
                        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
                        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
                        const unsigned bit = 1u << (2 * nt + r);
                        if (x > 0.f || ((unset & bit) && x > -INFINITY)) {
                            const float f = unset & bit ? 0.f : ex2(-x);
                            unset &= ~bit;
                            if (r == 0) { m[nt].x += x; l[nt].x *= f; }
                            else { m[nt].y += x; l[nt].y *= f; }
#pragma unroll
                            for (int i = 0; i < D / 16; ++i) {
                                o[i][nt][r] *= f;
                                o[i][nt][r + 2] *= f;
                            }
                            sv[nt][r] -= x;
                            sv[nt][r + 2] -= x;
                        }
                    }
            }
            // ---- P, and O^T += V^T P^T ----
            uint32_t pf[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float p0 = ex2(sv[nt][0]), p1 = ex2(sv[nt][1]), p2 = ex2(sv[nt][2]), p3 = ex2(sv[nt][3]);
                l[nt] = __fadd2_rn(l[nt], __fadd2_rn(make_float2(p0, p1), make_float2(p2, p3)));
                pf[nt][0] = transpose8x8(pack_bf16(p0, p1));
                pf[nt][1] = transpose8x8(pack_bf16(p2, p3));
            }
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                if (i == 0) ldmatrix_x4_trans(fa[0][0], fa[0][1], fa[0][2], fa[0][3], st + v_get);
                if (i + 1 < D / 16)
                    ldmatrix_x4_trans(fa[(i + 1) & 1][0], fa[(i + 1) & 1][1], fa[(i + 1) & 1][2], fa[(i + 1) & 1][3], st + (v_get ^ ((i + 1) << 5)));
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma_bf16_16816(o[i][nt], fa[i & 1], pf[nt][0], pf[nt][1]);
            }
        }

        // ---- the warps' results together, in their order ----
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                float x = r ? l[nt].y : l[nt].x;
                x += __shfl_xor_sync(0xffffffffu, x, 4);
                x += __shfl_xor_sync(0xffffffffu, x, 8);
                x += __shfl_xor_sync(0xffffffffu, x, 16);
                if (g == 0) {
                    stat[0][warp][nt * 8 + 2 * t + r] = (unset >> (2 * nt + r)) & 1u ? -INFINITY : r ? m[nt].y : m[nt].x;
                    stat[1][warp][nt * 8 + 2 * t + r] = x;
                }
            }
        ring_wait<0>();
        __syncthreads();                                     // nobody reads the ring any more
        float* os = reinterpret_cast<float*>(smem);          // [warp][row][D + 4]
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    os[(warp * L::ROWS + nt * 8 + 2 * t + (j & 1)) * (D + 4) + i * 16 + (j >> 1) * 8 + g] = o[i][nt][j];
        __syncthreads();
        const bool all_of_it = a.cluster ? a.cluster == 1 : unit == item_lo && seg_hi == item_hi;
        constexpr int TPR = D / 4;                           // threads of a row, 4 values each
        auto give = [&](int row, int c, const float4& v, float lse2) {
            const int64_t at = place_of(b, kvh, tile * L::ROWS + row);
            *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.o) + at * D + c * 4) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
            if (a.lse && c == 0) a.lse[at] = lse2 * 0.6931471805599453f;
        };
        // what a warp's sums of a row are multiplied by, and the log2 of the denominator
        if (tid < L::ROWS) {
            float mx = -INFINITY, den = 0.f, f[PW];
#pragma unroll
            for (int w = 0; w < PW; ++w) mx = fmaxf(mx, stat[0][w][tid]);
#pragma unroll
            for (int w = 0; w < PW; ++w) {
                f[w] = stat[0][w][tid] == -INFINITY ? 0.f : ex2(stat[0][w][tid] - mx);   // (a warp that met no key has sums of zero)
                den = fmaf(f[w], stat[1][w][tid], den);
            }
            const float inv = den == 0.f ? 0.f : 1.f / den;
            factor[tid] = make_float4(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv);
            lse2_of[tid] = den == 0.f ? -INFINITY : mx + log2f(den);
        }
        __syncthreads();
        // parts: [2 CTA + (whether the item began with it)][row][D], then [..][row] log2 of the denominators
        float* part_o = a.part;
        float* part_l = a.part + (int64_t)2 * gridDim.x * L::ROWS * D;
        const int64_t my_part = (int64_t)(2 * blockIdx.x + (unit == item_lo)) * L::ROWS;
        const int rows = min(L::ROWS, R - tile * L::ROWS);
        for (int i = tid; i < rows * TPR; i += PW * 32) {
            const int row = i / TPR, c = i % TPR;
            const float4 f4 = factor[row];
            const float f[PW] = {f4.x, f4.y, f4.z, f4.w};
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < PW; ++w) {
                const float4 x = *reinterpret_cast<const float4*>(os + (w * L::ROWS + row) * (D + 4) + c * 4);
                v.x = fmaf(f[w], x.x, v.x); v.y = fmaf(f[w], x.y, v.y); v.z = fmaf(f[w], x.z, v.z); v.w = fmaf(f[w], x.w, v.w);
            }
            if (all_of_it) {
                give(row, c, v, lse2_of[row]);
            } else if (a.cluster) {
                *reinterpret_cast<float4*>(os + L::MERGE / 4 + row * D + c * 4) = v;
            } else {
                *reinterpret_cast<float4*>(part_o + (my_part + row) * D + c * 4) = v;
                if (c == 0) part_l[my_part + row] = lse2_of[row];
            }
        }
        if (a.cluster > 1) {
            // ---- the CTAs of the cluster add their results up, each for a share of the values, in the order of their keys ----
            cluster_sync_all();
            const uint32_t res_at = smem_u32(os) + L::MERGE, lse_at = smem_u32(lse2_of);
            for (int i = tid + blockIdx.x % a.cluster * PW * 32; i < rows * TPR; i += a.cluster * PW * 32) {
                const int row = i / TPR, c = i % TPR;
                float x[8];
                float4 w[8];
#pragma unroll
                for (int p = 0; p < 8; ++p) {
                    x[p] = -INFINITY;
                    if (p < a.cluster) {
                        x[p] = ld_peer(mapa_u32(lse_at + row * 4, p));
                        w[p] = ld_peer4(mapa_u32(res_at + (row * D + c * 4) * 4, p));
                    }
                }
                Sum sum;
#pragma unroll
                for (int p = 0; p < 8; ++p) sum.add(x[p], w[p]);
                give(row, c, sum.mean(), sum.lse2());
            }
            cluster_sync_all();                              // nobody leaves while its results are read
            return;
        }
        if (!all_of_it) {
            // ---- the last of the item's CTAs adds the parts up, in their order ----
            const int c0 = (int)cta_of(item_lo), c1 = (int)cta_of(item_hi - 1u);
            auto part_of = [&](int q) { return (int64_t)(2 * q + (q == c0)) * L::ROWS; };
            __syncthreads();
            if (tid == 0) {
                unsigned* arrived = a.arrived + c0;          // an item that goes on past a CTA is the last one that begins there
                unsigned before;                             // (the other threads' parts are behind the barrier, and so told with this one's)
                asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(before) : "l"(arrived) : "memory");
                is_last = before == (unsigned)(c1 - c0);
                if (is_last) *arrived = 0u;
            }
            __syncthreads();
            if (is_last) {
                // This runs once: short loops (code that is met for the first time costs more than what it does), and the parts come as copies
                // into the ring's place, as many at a time as it holds, so that one wait stands for all of them.
                constexpr int HELD = L::RING / (L::ROWS * D * 4);
                float* held = os;                            // [part][row][D]
                float4 v[(L::ROWS * TPR) / (PW * 32)];
                float den[(L::ROWS * TPR) / (PW * 32)], top_l[(L::ROWS * TPR) / (PW * 32)];
#pragma unroll
                for (int k = 0; k < (L::ROWS * TPR) / (PW * 32); ++k) {
                    v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
                    den[k] = 0.f;
                    top_l[k] = -INFINITY;
                }
#pragma unroll 1
                for (int q0 = c0; q0 <= c1; q0 += HELD) {
                    const int n_here = min(HELD, c1 + 1 - q0), chunks = rows * TPR;
#pragma unroll 1
                    for (int p = warp; p < n_here; p += PW) {
                        const float* from = part_o + part_of(q0 + p) * D;
#pragma unroll 1
                        for (int i = lane; i < chunks; i += 32) cp_async16(smem_u32(held + p * (L::ROWS * D) + i * 4), from + i * 4);
                    }
                    cp_async_commit();
                    for (int i = tid; i < n_here * L::ROWS; i += PW * 32)
                        if (i % L::ROWS < rows) lse_of[i] = __ldcg(part_l + part_of(q0 + i / L::ROWS) + i % L::ROWS);
                    ring_wait<0>();
                    __syncthreads();
#pragma unroll 1
                    for (int p = 0; p < n_here; ++p) {
#pragma unroll
                        for (int k = 0; k < (L::ROWS * TPR) / (PW * 32); ++k) {
                            const int i = tid + k * PW * 32;
                            if (i >= chunks) break;
                            const float x = lse_of[p * L::ROWS + i / TPR];
                            if (x == -INFINITY) continue;    // no keys
                            const float4 w = *reinterpret_cast<const float4*>(held + p * (L::ROWS * D) + i * 4);
                            const float most = fmaxf(top_l[k], x), fo = top_l[k] == -INFINITY ? 0.f : ex2(top_l[k] - most), f = ex2(x - most);       // (a NaN comes through by f)
                            top_l[k] = most;
                            den[k] = fmaf(den[k], fo, f);
                            v[k].x = fmaf(v[k].x, fo, f * w.x); v[k].y = fmaf(v[k].y, fo, f * w.y);
                            v[k].z = fmaf(v[k].z, fo, f * w.z); v[k].w = fmaf(v[k].w, fo, f * w.w);
                        }
                    }
                    __syncthreads();
                }
#pragma unroll
                for (int k = 0; k < (L::ROWS * TPR) / (PW * 32); ++k) {
                    const int i = tid + k * PW * 32;
                    if (i >= rows * TPR) break;
                    const float inv = den[k] == 0.f ? 0.f : 1.f / den[k];
                    give(i / TPR, i % TPR, make_float4(v[k].x * inv, v[k].y * inv, v[k].z * inv, v[k].w * inv),
                         den[k] == 0.f ? -INFINITY : top_l[k] + log2f(den[k]));
                }
            }
        }
        unit = seg_hi == item_hi ? item_hi + extra : seg_hi;
        if (a.cluster || unit >= mine_hi) return;
    }
}

template <int D, int NT>
int paged_launch(PagedAttnArgs a, cudaStream_t stream) {
    using L = PagedLayout<D, NT>;
    static PerDevice<bool> ready;
    int device = 0;
    cudaGetDevice(&device);
    if (!ready.of(device, [](bool& ok) {
            ok = cudaFuncSetAttribute(paged_attn_kernel<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::SMEM) == cudaSuccess;
        }))
        return -1;
    a.group = a.n_heads / a.n_kv_heads;
    const int R = a.n * a.group, tiles = (R + L::ROWS - 1) / L::ROWS;
    // r / group as the upper half of a product, exact while r group stays below 2^32
    a.group_inverse = a.group > 1 && (int64_t)R * a.group < ((int64_t)1 << 32) ? (unsigned)((((int64_t)1 << 32) + a.group - 1) / a.group) : 0u;
    const int64_t items = (int64_t)tiles * a.batch * a.n_kv_heads, u = std::max(1, (a.ctx_len + kUnit - 1) / kUnit), units = (u + kItemUnits<NT>) * items;
    // Two ways to share the work.  In one line of units every CTA has as much to do, but a result in parts costs a trip through memory and
    // back (5 us, and the last CTA's time with each part); a cluster for each item joins its CTAs' parts in 1.6 us, but is as long as its item (lengths on
    // the device: a quarter longer than an equal share, say).  A unit of 128 columns takes a CTA 0.8 us alone on its SM and 1.3 beside another, or its share
    // of the memory's bandwidth.  One token of one request, 4 KV heads, 1664 keys: 9.1 us in one line, 7.5 in clusters; 5 rows of 7 requests, 251 keys: 10.5
    // and 6.7; 32 rows of one request, 4 KV heads of 64, 8000 keys: 40 and 17; one token of 32 requests, 4 KV heads, 40 to 2000 keys: 15 and 15.
    constexpr double kColumns = D / 128.0;
    const int ctas = (int)std::min<int64_t>(kPlaces, std::max<int64_t>(1, units / kMinUnits));
    auto unit_us = [&](int64_t active) {
        return kColumns * std::max(active > kPlaces / 2 ? 1.3 : 0.8, 1.5 * std::min<int64_t>(active, kPlaces) / kPlaces);
    };
    const double parts = ctas > items ? (double)ctas / items : 0.0;
    double best = (units + ctas - 1) / ctas * unit_us(ctas) + 6.0 + parts * 0.28 * NT * kColumns;
    a.cluster = 0;
    for (int c = 1; c <= 8 && c <= u && items * c <= 4 * kPlaces; c *= 2) {
        const double t = (items * c + kPlaces - 1) / kPlaces * ((u + c - 1) / c * unit_us(items * c) * (a.lens ? 1.25 : 1.0) + (c > 1 ? 2.6 : 1.0));
        if (t < best) {
            best = t;
            a.cluster = c;
        }
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(a.cluster ? (unsigned)items * a.cluster : ctas);
    cfg.blockDim = dim3(PW * 32);
    cfg.dynamicSmemBytes = L::SMEM;
    cfg.stream = stream;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = a.cluster; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = a.cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, paged_attn_kernel<D, NT>, a) == cudaSuccess ? 1 : -1;
}
// row tiles of 8 in a CTA for R rows of a KV head (24 rows as 32: 100 us for 87)
int tile_of(int64_t R) { return R <= 8 ? 1 : R <= 16 ? 2 : R <= 24 ? 3 : 4; }

template <int D>
int paged_dispatch(const PagedAttnArgs& a, cudaStream_t stream) {
    switch (tile_of((int64_t)a.n * (a.n_heads / a.n_kv_heads))) {
        case 1: return paged_launch<D, 1>(a, stream);
        case 2: return paged_launch<D, 2>(a, stream);
        case 3: return paged_launch<D, 3>(a, stream);
        default: return paged_launch<D, 4>(a, stream);
    }
}

}  // namespace

size_t paged_attention_scratch_bytes(int head_dim) { return (size_t)2 * kPlaces * 32 * (head_dim + 1) * sizeof(float); }

bool paged_attention_fits(int batch, int n, int ctx_len, int n_heads, int n_kv_heads) {
    const int64_t R = (int64_t)n * (n_heads / n_kv_heads);
    const int rows = 8 * tile_of(R);
    int64_t units = (R + rows - 1) / rows * batch;
    if (units > INT_MAX) return false;                       // (step by step: no product passes 64 bits)
    units *= n_kv_heads;
    if (units > INT_MAX) return false;
    return units * (std::max(1, (ctx_len + kUnit - 1) / kUnit) + (rows > 16 ? kItemUnits<4> : kItemUnits<1>)) <= INT_MAX;
}

int launch_paged_attention(const PagedAttnArgs& a, cudaStream_t stream) {
    if (a.batch == 0 || a.n == 0) return 0;
    return a.head_dim == 128 ? paged_dispatch<128>(a, stream) : paged_dispatch<64>(a, stream);
}

}  // namespace acache
