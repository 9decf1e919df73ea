// Attention over the 8-bit cache for many query rows per KV head (refreshes, decode blocks of grouped heads) on the
// 5th-generation tensor cores, head dimension 128.  The mathematics is that of kv8_attn.cu: products on the codes as f16, the
// key block's scale in the factor of the logits, the value block's in the exponent.
//
// A CTA takes SETS tiles of 128 query rows of one (request, KV head) - the heads of a group are rows like others, so a key is
// converted once for all of them - over a range of 128-key tiles:
//   converter warps    codes from the cache (registers one tile ahead, L2 further), to f16, into the 128-byte-swizzled shared
//                      tiles the tensor core reads: what a TMA load does for a bf16 cache
//   one issuing warp   S = Q K^T and O += P V by tcgen05.mma 128 x 128 x 16, P read from tensor memory, V MN-major
//   softmax warps      one thread per query row, S in two halves of 64 keys: y - M, maximum, exp2, P as f16 over S's columns
// Per 16 keys a table entry (the converters write it) gives the softmax both scales and the weight in l.
// Bound by the chain product - maximum - exponentials - product of a row tile: 4500 cycles a key tile with two row tiles, of which the
// tensor core is busy for 2170, the special-function units for 2050; with one thread a row, two softmax warps a scheduler are what there
// is to fill the gaps.  16 x 922 rows, 2560 keys, 32 heads: 790 us in int8 (0.78 PFLOP/s); 1639 rows, 8288 keys: 333 us (0.67: 224 CTAs on
// 148 SMs).  The bf16 kernel next door (attn_tc.cu: four threads a row, two S buffers, no codes to convert) takes 242 us for these.
// (Figures by which choices below were made are from references 2^4 above the largest logit: 1 to 5 % less.)
#include <algorithm>
#include <array>
#include <climits>

#include "kv8_tc.cuh"
#include "launch.h"
#include "per_device.h"

namespace acache {

namespace {

constexpr int kTcSplits = 8;                              // a portable cluster
// ns, measured, for one and for two row tiles: a key tile, the sum over a cluster; a CTA's start and end
template <int SETS>
constexpr int kTileNs = SETS == 2 ? 2300 : 2050;
template <int SETS>
constexpr int kSumNs = SETS == 2 ? 6000 : 2000;
constexpr int kCtaNs = 6000;

// Warps: converters, from warp 8 on softmax, one that issues.  128 registers a thread allow four warps a scheduler.  Two row tiles: 7
// converters and the issuing warp in front of 8 softmax warps (922 rows, 2560 keys, int8: 781 us; 3 converters 910, 4 and the issuing
// one behind them 805).  One: 8, 4 and the issuing one behind them (100 rows, 8192 keys: 501 us; 7 converters 509, 11 511).
template <int SETS>
constexpr int kConverters = SETS == 2 ? 7 : 8;
template <int SETS>
constexpr int kIssuer = SETS == 2 ? 7 : 12;
template <int SETS>
constexpr int kThreads = SETS == 2 ? 512 : 416;
constexpr int TT_SOFTMAX = 8;                             // the first softmax warp
constexpr int TT_SLACK = 1024;
constexpr int TT_TAIL = 2048;                             // tables, barriers; from kResL a float per row
constexpr int kResL = 1024;
static_assert(kTables * sizeof(KeyTable) + 256 <= kResL && kResL + 256 * 4 <= TT_TAIL);

template <int SETS>
constexpr int tt_smem() { return (SETS + 4) * TT_TILE + TT_TAIL + TT_SLACK; }
template <int SETS>
constexpr bool tt_res_fits() {           // the sums' weights behind the results; the first row tile's results off V
    return SETS * 128 * (132 + 8) * 4 <= (SETS + 4) * TT_TILE && 128 * 132 * 4 <= (SETS + 2) * TT_TILE;
}
static_assert(tt_res_fits<1>() && tt_res_fits<2>());
static_assert(tt_smem<1>() >= kAloneBytes && tt_smem<2>() <= 227 * 1024);

// The CTAs of a cluster add their results up, each for a share of the rows, in the order of their keys.  A function of its own: what
// it needs should not take registers from the loops before it.  (Its code runs once and comes from L2, so there is little of it.)
template <int SETS>
__device__ __noinline__ void tc_sum(unsigned char* base, unsigned char* tail, void* o, float* lse, int n, int n_heads, int G, int cs) {
    const float* res = reinterpret_cast<const float*>(base);                                // [row][132]
    const float* res_l = reinterpret_cast<const float*>(tail + kResL);
    float* weight = reinterpret_cast<float*>(base + SETS * 128 * 132 * 4);                  // [row][8]: of a CTA's part in the sum
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, n_kv = n_heads / G, row0 = blockIdx.y * SETS * 128;
    const int rows = min(n * G - row0, SETS * 128), rank = (int)cluster_ctarank();
    const int mine = rows > rank ? (rows - rank + cs - 1) / cs : 0;                         // rows rank, rank + cs, ..
    const int64_t first = (int64_t)(blockIdx.z / n_kv) * n * n_heads + blockIdx.z % n_kv * G;
    cluster_sync_all();                                   // (one that gave up takes part as well: the call reports it)
    for (int i = tid; i < mine * 8; i += kThreads<SETS>) {    // a whole group of eight lanes, or none of it
        const int row = rank + (i >> 3) * cs, part = i & 7;
        const float x = part < cs ? ld_peer(mapa_u32(smem_u32(res_l + row), part)) : -INFINITY;
        const uint32_t eight = 0xFFu << (lane & 24);
        float mx = x;
#pragma unroll
        for (int k = 4; k > 0; k >>= 1) mx = fmaxf(mx, __shfl_xor_sync(eight, mx, k));
        const float f = x == -INFINITY ? 0.f : ex2(x - mx);                                 // (a NaN comes through)
        float den = f;
#pragma unroll
        for (int k = 4; k > 0; k >>= 1) den += __shfl_xor_sync(eight, den, k);
        weight[i] = den == 0.f ? 0.f : f / den;
        const int r = row0 + row;
        if (part == 0 && lse) lse[first + (int64_t)(r / G) * n_heads + r % G] = den == 0.f ? -INFINITY : (mx + log2f(den)) * 0.6931471805599453f;
    }
    __syncthreads();
    for (int i = warp; i < mine; i += kThreads<SETS> / 32) {
        const int row = rank + i * cs, r = row0 + row;
        const uint32_t at = smem_u32(res + row * 132 + lane * 4);
        float4 w[8], v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int p = 0; p < 8; ++p) w[p] = p < cs ? ld_peer4(mapa_u32(at, p)) : v;
#pragma unroll
        for (int p = 0; p < 8; ++p) {
            const float f = weight[i * 8 + p];
            v.x = fmaf(f, w[p].x, v.x); v.y = fmaf(f, w[p].y, v.y); v.z = fmaf(f, w[p].z, v.z); v.w = fmaf(f, w[p].w, v.w);
        }
        *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(o) + (first + (int64_t)(r / G) * n_heads + r % G) * 128 + lane * 4) =
            make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
    }
    cluster_sync_all();                                   // nobody leaves while its results are read
}

template <int FMT, int SETS>
__global__ void __launch_bounds__(kThreads<SETS>, 1) kv8_attn_tc_kernel(const Kv8AttnArgs a) {
    constexpr int CW = kConverters<SETS>, ISSUER = kIssuer<SETS>;
    // Parts of a row tile's S, each a product of its own.  Alone, a row tile leaves the tensor core idle while its softmax runs, and
    // halves let the next S be made meanwhile (100 rows, 8192 keys, 512 pairs: 510 us, whole 535); two fill each other's gaps, and
    // products of 64 keys, which read Q twice as often from shared memory, only cost (922 rows, 2560 keys: 829 us, whole 805).
    constexpr int S_PARTS = SETS == 2 ? 1 : 2;
    constexpr int CT = CW * 32;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    unsigned char* base_ptr = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t sQ = base, sK0 = base + SETS * TT_TILE, sV0 = sK0 + 2 * TT_TILE;
    unsigned char* tail = base_ptr + (SETS + 4) * TT_TILE;
    KeyTable* tables = reinterpret_cast<KeyTable*>(tail);
    const uint32_t bars = smem_u32(tail + kTables * sizeof(KeyTable));
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(tail + kTables * sizeof(KeyTable) + 232);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tail + kTables * sizeof(KeyTable) + 236);
    // barriers: 0 q_full | 1,2 k_full | 3,4 k_empty | 5,6 v_full | 7,8 v_empty | 11 + 2 t + hb: p_full | 15 + 2 t + hb: pv_done |
    //           19 + j % 4: table of key tile j | 23 + 2 t + part: s_full   (row tile t, key half hb)
    auto bar = [&](int i) { return bars + 8 * i; };
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int split = blockIdx.x, tile = blockIdx.y, b = blockIdx.z / a.n_kv_heads, kvh = blockIdx.z % a.n_kv_heads;
    const int G = a.n_heads / a.n_kv_heads, R = a.n * G;
    const int row0 = tile * SETS * 128;
    const int n_sets = SETS == 2 && row0 + 128 < R ? 2 : 1;
    auto warps_of = [&](int t) { return min(4, (R - row0 - t * 128 + 31) / 32); };     // softmax warps with rows

    if (tid == 0) {
        mbar_init(bar(0), warps_of(0) + (n_sets == 2 ? warps_of(1) : 0));
        for (int i = 1; i <= 2; ++i) { mbar_init(bar(i), CW); mbar_init(bar(4 + i), CW); mbar_init(bar(2 + i), 1); mbar_init(bar(6 + i), 1); }
        for (int t = 0; t < 2; ++t) {
            for (int hb = 0; hb < 2; ++hb) {
                mbar_init(bar(23 + 2 * t + hb), 1);
                mbar_init(bar(11 + 2 * t + hb), t < n_sets ? warps_of(t) : 1);
                mbar_init(bar(15 + 2 * t + hb), 1);
            }
        }
        for (int i = 0; i < kTables; ++i) mbar_init(bar(19 + i), 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == ISSUER) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32(const_cast<uint32_t*>(tmem_slot))), "r"(SETS * 256) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    // columns: S of the row tiles, then O of the row tiles, 128 each
    constexpr uint32_t O_COL = SETS * 128;
    pdl_wait();
    pdl_launch_dependents();
    int len = a.ctx_len;
    if (a.lens) {
        len = a.lens[b];
        if (len < 0 || len > a.ctx_len) {
            if (tid == 0) atomicOr(a.status, kFlagBadIndex);
            len = min(max(len, 0), a.ctx_len);
        }
    }
    const int key_lo = split * a.split_keys, key_hi = min(len, key_lo + a.split_keys);
    const int n_tiles = key_hi > key_lo ? (key_hi - key_lo + 127) / 128 : 0;
    // This CTA's result, for the others of its cluster: [row][132] over the tiles of Q and K, which no product reads any more once
    // a row tile's last P V has completed (the other row tile's may still read V); the log2 of the denominators beside the tables.
    float* res = reinterpret_cast<float*>(base_ptr);
    float* res_l = reinterpret_cast<float*>(tail + kResL);

    if (warp < CW) {
        // ---------------- converters ----------------
        const int64_t cache_at = (int64_t)b * a.batch_stride + (int64_t)kvh * a.capacity * 128;
        const uint8_t *kb = a.k + cache_at, *vb = a.v + cache_at;
        const int64_t exps_at = ((int64_t)(a.shared ? 0 : b) * a.n_kv_heads + kvh) * a.n_blocks;
        const TileMeta meta_of{a.k_exp + exps_at, a.v_exp + exps_at, a.key_drop ? a.key_drop + (int64_t)b * a.drop_words : nullptr, a.log2_block, key_hi};
        TilePieces<CT> kr, vr;
        auto prefetch = [&](int j) {
            if (tid != 0 || j >= n_tiles) return;
            const int key0 = key_lo + j * 128, rows = min(128, key_hi - key0);
            l2_prefetch(kb + (int64_t)key0 * 128, rows * 128);
            l2_prefetch(vb + (int64_t)key0 * 128, rows * 128);
        };
        uint32_t meta = 0u;
        int e0 = 0;
        if (n_tiles > 0) {
            kr.load(kb, key_lo, key_hi, tid);
            meta = meta_of.load(key_lo, lane);
            vr.load(vb, key_lo, key_hi, tid);
            prefetch(1); prefetch(2); prefetch(3);
        }
        for (int j = 0; j < n_tiles; ++j) {
            const int s = j & 1;
            const uint32_t par = ((j >> 1) & 1) ^ 1;
            const uint32_t now = meta;
            // groups whose block holds nothing are zero; so are the values of keys that do not count
            const uint32_t empty = __ballot_sync(0xffffffffu, lane < 16 && now == 0u);
            uint32_t krows[4], vrows[4];
            rows_held(empty & 0xFFu, krows);
            rows_held(empty >> 8, vrows);
#pragma unroll
            for (int w = 0; w < 4; ++w) vrows[w] &= __shfl_sync(0xffffffffu, now, 16 + w);
            const bool k_all = (empty & 0xFFu) == 0u, v_all = (vrows[0] & vrows[1] & vrows[2] & vrows[3]) == ~0u;
            if (!__all_sync(0xffffffffu, tt_doze(bar(3 + s), par, abort_flag))) break;
            if (warp == 0) {
                write_table(tables[j & (kTables - 1)], now, lane, e0);
                if (lane == 0) mbar_arrive(bar(19 + (j & (kTables - 1))));
            }
            kr.template convert<FMT>(sK0 + s * TT_TILE, krows, k_all, tid);
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(1 + s));
            prefetch(j + 4);
            if (j + 1 < n_tiles) {
                kr.load(kb, key_lo + (j + 1) * 128, key_hi, tid);
                meta = meta_of.load(key_lo + (j + 1) * 128, lane);
            }
            if (!__all_sync(0xffffffffu, tt_doze(bar(7 + s), par, abort_flag))) break;
            vr.template convert<FMT>(sV0 + s * TT_TILE, vrows, v_all, tid);
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(5 + s));
            if (j + 1 < n_tiles) vr.load(vb, key_lo + (j + 1) * 128, key_hi, tid);
        }
    } else if (warp == ISSUER) {
        // ---------------- MMA issuer: the whole warp runs the loop, one lane issues ----------------
        const uint32_t idesc = (1u << 4) | ((uint32_t)(128 >> 4) << 24);                 // f16 x f16 -> fp32, 128 rows
        const uint32_t idesc_s = idesc | ((uint32_t)(128 / S_PARTS >> 3) << 17);         // keys of a part
        const uint32_t idesc_o = idesc | ((uint32_t)(128 >> 3) << 17) | (1u << 16);      // 128 columns of V, which is MN-major
        auto wait = [&](int i, uint32_t parity) { return __all_sync(0xffffffffu, tt_spin(bar(i), parity, abort_flag)); };
        auto issue_s = [&](int t, int j, int part) {
            const uint32_t k = sK0 + (j & 1) * TT_TILE + part * (64 * 128);
            if (!elect_lane()) return;
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) {
                const uint64_t da = smem_desc_sw128(sQ + t * TT_TILE + (ks >> 2) * TT_PANEL) + (uint64_t)((ks & 3) * 2);
                const uint64_t db = smem_desc_sw128(k + (ks >> 2) * TT_PANEL) + (uint64_t)((ks & 3) * 2);
                tc_mma(tmem_base + t * 128 + part * 64, da, db, idesc_s, ks > 0 ? 1u : 0u);
            }
            tc_commit(bar(23 + 2 * t + part));
        };
        bool ok = n_tiles > 0 && wait(0, 0) && wait(1, 0);
        if (ok) {
            tc_fence_after();
            for (int t = 0; t < n_sets; ++t)
                for (int part = 0; part < S_PARTS; ++part) {
                    issue_s(t, 0, part);
                    __syncwarp();
                }
            if (elect_lane()) tc_commit(bar(3));
            __syncwarp();
        }
        // The next key tile's S goes out right behind the P V that reads the P in its columns: the products execute in order.
        for (int j = 0; j < n_tiles && ok; ++j) {
            const int s = j & 1;
            const bool more = j + 1 < n_tiles;
            if (!(ok = wait(5 + s, (j >> 1) & 1))) break;
            if (more && !(ok = wait(1 + (s ^ 1), ((j + 1) >> 1) & 1))) break;
            const uint32_t v = sV0 + s * TT_TILE;
            for (int t = 0; t < n_sets && ok; ++t) {
                for (int hb = 0; hb < 2 && ok; ++hb) {
                    if (!(ok = wait(11 + 2 * t + hb, j & 1))) break;
                    tc_fence_after();
                    if (elect_lane()) {
#pragma unroll
                        for (int k4 = 0; k4 < 4; ++k4)
                            tt_mma_ta(tmem_base + O_COL + t * 128, tmem_base + t * 128 + hb * 64 + k4 * 8, tt_desc_mn(v + (hb * 4 + k4) * 2048), idesc_o,
                                      (j > 0 || hb > 0 || k4 > 0) ? 1u : 0u);
                        tc_commit(bar(15 + 2 * t + hb));
                    }
                    __syncwarp();
                    if (more && hb + S_PARTS >= 2) issue_s(t, j + 1, S_PARTS == 2 ? hb : 0);
                    __syncwarp();
                }
            }
            if (elect_lane()) {
                tc_commit(bar(7 + s));
                if (more) tc_commit(bar(3 + (s ^ 1)));
            }
            __syncwarp();
        }
    } else if (warp >= TT_SOFTMAX && warp < TT_SOFTMAX + 4 * n_sets) {
        // ---------------- softmax: one thread per query row ----------------
        const int t = (warp - TT_SOFTMAX) >> 2, q4 = warp & 3;    // the warp's TMEM lane quarter
        const int row = q4 * 32 + lane, r = row0 + t * 128 + row;
        const uint32_t lane_off = (uint32_t)(q4 * 32) << 16;
        const uint32_t tS = tmem_base + t * 128 + lane_off, tO = tmem_base + O_COL + t * 128 + lane_off;
        if (q4 * 32 < R - row0 - t * 128) {
            // the row of q as f16 over a power of two of its own, into the operand tile
            float rq = 0.f;
            if (n_tiles > 0) {
                const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(a.q) + ((int64_t)(b * (int64_t)a.n + r / G) * a.n_heads + kvh * G + r % G) * 128;
                uint4 x[16];
                uint32_t top2 = 0u;
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = r < R ? __ldg(reinterpret_cast<const uint4*>(q) + i) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    top2 = __vmaxu2(__vmaxu2(top2, x[i].x & 0x7F807F80u), __vmaxu2(__vmaxu2(x[i].y & 0x7F807F80u, x[i].z & 0x7F807F80u), x[i].w & 0x7F807F80u));
                const int field = min(max((int)(max(top2 & 0xFFFFu, top2 >> 16) >> 7), 1), 253);
                const float inv = __int_as_float((254 - field) << 23);
                rq = __int_as_float(field << 23) * a.scale_log2e;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
                    uint32_t f[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) f[k] = pack_f16(bf16_lo(w[k]) * inv, bf16_hi(w[k]) * inv);
                    st_shared16(sQ + t * TT_TILE + (i >> 3) * TT_PANEL + row * 128 + (((i & 7) ^ (row & 7)) << 4), f[0], f[1], f[2], f[3]);
                }
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0 && n_tiles > 0) mbar_arrive(bar(0));

            float m_use = -INFINITY, l = 0.f, top = -INFINITY;
            int e0 = 127;
            bool ok = true;
            for (int i = 0; i < 2 * n_tiles && ok; ++i) {
                const int hb = i & 1, j = i >> 1;
                const KeyTable& tab = tables[j & (kTables - 1)];
                if (hb == 0) {
                    // warp-uniform: the tensor-memory accesses below are collective
                    if (!(ok = __all_sync(0xffffffffu, tt_spin(bar(19 + (j & (kTables - 1))), (j >> 2) & 1, abort_flag)))) break;
                    l *= tab.grow;
                    m_use += tab.along;
                    e0 = tab.e0;
                }
                if (hb < S_PARTS) {
                    if (!(ok = __all_sync(0xffffffffu, tt_spin(bar(23 + 2 * t + hb), j & 1, abort_flag)))) break;
                    tc_fence_after();
                }
                const uint2 keep2 = *reinterpret_cast<const uint2*>(&tab.keep[2 * hb]);
                const uint32_t keep[2] = {keep2.x, keep2.y};
                float4 sc[4];
#pragma unroll
                for (int g = 0; g < 4; ++g) sc[g] = tab.group[hb * 4 + g];
                float sv[2][32];
                tt_ld32(tS + hb * 64, sv[0]);
                tt_ld32(tS + hb * 64 + 32, sv[1]);
                tt_wait_ld<32>(sv[0]);
                tt_wait_ld<32>(sv[1]);
                // y - M in place; M is 0 until a half with a key that counts
                const bool first = m_use == -INFINITY;
                const float m_ref = first ? 0.f : m_use;
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const float fa = rq * sc[g].x, fb = sc[g].y - m_ref;
                    const float2 fa2 = make_float2(fa, fa), fb2 = make_float2(fb, fb);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float* p = &sv[g >> 1][(g & 1) * 16 + 2 * e];
                        const float2 y = __ffma2_rn(make_float2(p[0], p[1]), fa2, fb2);
                        p[0] = y.x;
                        p[1] = y.y;
                    }
                }
                if ((keep[0] & keep[1]) != ~0u) {
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int e = 0; e < 32; ++e) sv[c][e] = ((keep[c] >> e) & 1u) ? sv[c][e] : -INFINITY;
                }
                float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int e = 0; e < 32; e += 2) m4[(e >> 1) & 3] = fmaxf(fmaxf(m4[(e >> 1) & 3], sv[c][e]), sv[c][e + 1]);
                float mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
                // The reference moves for the warp's rows together.  l and P take the new one at once; O, which waits for a product, once P is
                // out (in front of it: 673 us for 16 x 922 rows with their own lengths where it is 639; without that price, but with small
                // weights lost, 607: kv8.cuh).  top: the largest y - M met so far.
                top = fmaxf(top, mx);
                float f = 1.f;
                const bool moves = __any_sync(0xffffffffu, mx > kRaise || (first && mx > -INFINITY));
                if (moves) {
                    if (top > kStart || (first && mx > -INFINITY)) {
                        const float up = top - kStart;
                        f = first ? 0.f : ex2(-up);
                        m_use = m_ref + up;
                        top = kStart;
                        l *= f;
#pragma unroll
                        for (int c = 0; c < 2; ++c)
#pragma unroll
                            for (int e = 0; e < 32; ++e) sv[c][e] -= up;
                    }
                }
                // P as packed f16 over the first 32 of the half's 64 columns of S, which this thread has read
                uint32_t pk[32];
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    float2 sa = make_float2(0.f, 0.f), sb = make_float2(0.f, 0.f);
#pragma unroll
                    for (int e = 0; e < 16; e += 4) {
                        const float* x = &sv[g >> 1][(g & 1) * 16 + e];
                        const float2 pa = make_float2(ex2(x[0]), ex2(x[1])), pb = make_float2(ex2(x[2]), ex2(x[3]));
                        sa = __fadd2_rn(sa, pa);
                        sb = __fadd2_rn(sb, pb);
                        pk[g * 8 + (e >> 1)] = pack_f16(pa.x, pa.y);
                        pk[g * 8 + (e >> 1) + 1] = pack_f16(pb.x, pb.y);
                    }
                    l = fmaf((sa.x + sa.y) + (sb.x + sb.y), sc[g].z, l);
                }
                tt_st32(tS + hb * 64, pk);
                if (moves && i > 0) {
                    // O may only be touched once the P V of half i - 1 (and with it every earlier one) has completed: by now it has
                    if (!(ok = __all_sync(0xffffffffu, tt_spin(bar(15 + 2 * t + ((i - 1) & 1)), ((i - 1) >> 1) & 1, abort_flag)))) break;
                    tc_fence_after();
#pragma unroll 1
                    for (int c = 0; c < 2; ++c) {
                        float v[2][32];
                        tt_ld32(tO + c * 64, v[0]);
                        tt_ld32(tO + c * 64 + 32, v[1]);
                        tt_wait_ld<32>(v[0]);
                        tt_wait_ld<32>(v[1]);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            uint32_t u[32];
#pragma unroll
                            for (int e = 0; e < 32; ++e) u[e] = __float_as_uint(v[h][e] * f);
                            tt_st32(tO + c * 64 + h * 32, u);
                        }
                    }
                }
                tt_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(11 + 2 * t + hb));
            }
            // epilogue
            if (ok && n_tiles > 0) ok = __all_sync(0xffffffffu, mbar_wait(bar(15 + 2 * t + 1), (n_tiles - 1) & 1, abort_flag));
            if (ok) {
                tc_fence_after();
                const float inv = l == 0.f ? 0.f : 1.f / l, up = kv8_unbias(e0);
                const float lse2 = l == 0.f ? -INFINITY : m_use - (float)(e0 - 127 - kWeightBias) + log2f(l);
                const int64_t at = (int64_t)(b * (int64_t)a.n + r / G) * a.n_heads + kvh * G + r % G;
#pragma unroll 1
                for (int c = 0; c < 4; ++c) {
                    float v[32];
                    if (n_tiles > 0) {
                        tt_ld32(tO + c * 32, v);
                        tt_wait_ld<32>(v);
                    }
                    if (r < R) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = l == 0.f ? 0.f : v[e] * inv * up;
                        if (a.splits == 1) {
                            uint32_t u[8];
                            __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.o) + at * 128 + c * 32;
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
#pragma unroll
                                for (int k = 0; k < 8; ++k) u[k] = pack_bf16(v[h * 16 + 2 * k], v[h * 16 + 2 * k + 1]);
                                st_global32(out + h * 16, u, on_sector(a.o));
                            }
                        } else {
#pragma unroll
                            for (int k4 = 0; k4 < 8; ++k4)
                                *reinterpret_cast<float4*>(res + (t * 128 + row) * 132 + c * 32 + k4 * 4) =
                                    make_float4(v[k4 * 4], v[k4 * 4 + 1], v[k4 * 4 + 2], v[k4 * 4 + 3]);
                        }
                    }
                    __syncwarp();
                }
                if (r < R) {
                    if (a.splits > 1) res_l[t * 128 + row] = lse2;
                    else if (a.lse) a.lse[at] = lse2 * 0.6931471805599453f;
                }
            }
        }
    }
    // ---------------- teardown ----------------
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {
        if (tid == 0) {
            atomicOr(a.status, kFlagWaitExpired);
            for (int i = 0; i < 4096; ++i) __nanosleep(64);       // let products already in flight end
        }
        __syncthreads();
    }
    if (warp == ISSUER) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(SETS * 256));
    }
    if (a.splits == 1) return;
    tc_sum<SETS>(base_ptr, tail, a.o, a.lse, a.n, a.n_heads, G, a.splits);
}

template <int FMT, int SETS>
void tc_config(cudaLaunchConfig_t& cfg, cudaLaunchAttribute (&at)[2], dim3 grid, cudaStream_t stream) {
    cfg = cudaLaunchConfig_t{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(kThreads<SETS>);
    cfg.dynamicSmemBytes = tt_smem<SETS>();
    cfg.stream = stream;
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = grid.x; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = grid.x > 1 ? 2 : 1;
}
// [n]: clusters of n CTAs that the current device runs at a time (fewer than SMs / n: a cluster stays in one group of SMs)
template <int FMT, int SETS>
std::array<int, kTcSplits + 1> tc_clusters() {
    static PerDevice<std::array<int, kTcSplits + 1>> fits;
    int device = 0;
    cudaGetDevice(&device);
    return fits.of(device, [](std::array<int, kTcSplits + 1>& fit) {
        cudaFuncSetAttribute(kv8_attn_tc_kernel<FMT, SETS>, cudaFuncAttributeMaxDynamicSharedMemorySize, tt_smem<SETS>());
        for (int s = kTcSplits; s >= 1; --s) {
            cudaLaunchConfig_t cfg;
            cudaLaunchAttribute at[2];
            tc_config<FMT, SETS>(cfg, at, dim3(s), nullptr);
            cfg.attrs = at + 1;                           // the cluster alone
            cfg.numAttrs = 1;
            int most = 0;
            if (cudaOccupancyMaxActiveClusters(&most, kv8_attn_tc_kernel<FMT, SETS>, &cfg) != cudaSuccess) most = 0;
            fit[s] = std::max(most, 1);
        }
    });
}
struct TcPlan { int per, splits; int64_t cost; };         // key tiles of a split, splits, ns
// The number of splits with which the rounds of CTAs take least.  1639 rows of 32 heads, 8288 keys (224 items): whole 317 us, in
// thirds 325, in quarters 370; 100 rows, 8192 keys (32 items): whole 78 us, in quarters 42, in eighths (15 at a time) 75.
template <int FMT, int SETS>
TcPlan tc_plan(const Kv8AttnArgs& a) {
    const int R = a.n * (a.n_heads / a.n_kv_heads), tiles = (R + SETS * 128 - 1) / (SETS * 128);
    const int64_t items = (int64_t)tiles * a.batch * a.n_kv_heads;
    const int key_tiles = std::max(1, (a.ctx_len + 127) / 128);
    const std::array<int, kTcSplits + 1> fits = tc_clusters<FMT, SETS>();
    TcPlan best{key_tiles, 1, INT64_MAX};
    for (int s = 1; s <= kTcSplits && s <= key_tiles; ++s) {
        const int per = (key_tiles + s - 1) / s, n = (key_tiles + per - 1) / per, fit = fits[n];
        const int64_t cost = (items + fit - 1) / fit * (per * kTileNs<SETS> + kCtaNs + (n > 1 ? kSumNs<SETS> : 0));
        if (cost < best.cost) best = TcPlan{per, n, cost};
    }
    return best;
}
template <int FMT, int SETS>
int tc_launch(Kv8AttnArgs a, const TcPlan& plan, cudaStream_t stream) {
    const int R = a.n * (a.n_heads / a.n_kv_heads), tiles = (R + SETS * 128 - 1) / (SETS * 128);
    a.split_keys = plan.per * 128;
    a.splits = plan.splits;
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute at[2];
    tc_config<FMT, SETS>(cfg, at, dim3(a.splits, tiles, a.batch * a.n_kv_heads), stream);
    return cudaLaunchKernelEx(&cfg, kv8_attn_tc_kernel<FMT, SETS>, a) == cudaSuccess ? 1 : -1;
}
template <int FMT>
int tc_dispatch(const Kv8AttnArgs& a, int64_t limit, cudaStream_t stream) {
    const TcPlan one = tc_plan<FMT, 1>(a), two = tc_plan<FMT, 2>(a);
    if (std::min(one.cost, two.cost) > limit) return 0;
    return two.cost <= one.cost ? tc_launch<FMT, 2>(a, two, stream) : tc_launch<FMT, 1>(a, one, stream);
}

}  // namespace

int launch_kv8_attention_tc(const Kv8AttnArgs& a, int64_t limit, cudaStream_t stream) {
    return a.format == kKv8Int8 ? tc_dispatch<kKv8Int8>(a, limit, stream) : tc_dispatch<kKv8E4m3>(a, limit, stream);
}

}  // namespace acache
