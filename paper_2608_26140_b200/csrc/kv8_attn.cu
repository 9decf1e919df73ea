// Attention over the 8-bit cache.
//
//   o_r = sum_j 2^(x_rj - M) V_j / sum_j 2^(x_rj - M),   x_rj = log2(e) / sqrt(d) q_r K_j
//
// with K_j = 2^(ek) k_j, V_j = 2^(ev) v_j, k_j and v_j the codes: whole numbers or e4m3 values, exact in f16.  The products
// run on the codes; ek joins the factor that turns a product into x, ev the exponent:
//   y_rj = x_rj + ev,   p_rj = 2^(y_rj - M)  (M: running reference of y),   O = sum p v,   l = sum p 2^(E0 - ev)
// (l over 2^32: kv8.cuh) so that o = 2^E0 O / l with E0 the largest ev so far of values that count (l follows it), and no code is ever multiplied by its scale.  The
// scales of one head's values may differ by 2^100, which is where the weights in l end.  p is f16:
// V's codes are f16 whatever their scales, which leaves p 11 bits (with bf16 operands, 8).  q is f16 too, each row over a
// power of two of its own that brings its largest value to [1, 2).
//
// A warp streams keys on its own, 32 a step: the bytes go from the cache to a ring of its own in shared memory (cp.async, whole
// rows side by side; half rows stopped at 4.8 TB/s), swizzled so that the fragments' reads meet different banks, from there to
// registers, become matrix-instruction fragments there and are used for all the rows.  The order of d inside a product is free,
// so a thread's 16 contiguous bytes of a key row serve as its fragment of four products:
//   S^T = K Q^T (keys x rows)   O^T += V^T P^T (d x rows): keys and d are the long sides of both products, so up to 8 rows cost
//   one instruction, and P only has to be transposed in 8 x 8 blocks (movmatrix).
// Up to 8 rows HBM bounds it: one token over 2 x 65537 keys of 32 heads (1074 MB) 176 us in a row, 6.1 TB/s, 182 to 196 us among other
// passes.  At 32 rows (16 x 2560 keys of 32 heads, 344 MB, 102.6 us) the matrix instructions are busy for 42 % of the time, the issue slots for
// 35, HBM for half: with 255 registers a thread there are two warps a scheduler to hide each other's waits.
// The reference M moves only when a logit passes it by 2^15.9 (f16 ends at 2^16), found by a vote; then maxima are exchanged and O is scaled.
// It starts 2^8 below the first keys' largest (kv8.cuh); 2^4 above it, 32 rows took 98.8 us where they take 102.6, and lost small weights.
// (The figures by which splits and rows a CTA were chosen, further down, are from then: 32 rows took up to 4 % less.)
#include <algorithm>
#include <array>
#include <climits>

#include "kernels.h"
#include "kv8.cuh"
#include "launch.h"
#include "per_device.h"
#include "tc_ptx.cuh"

namespace acache {

// kernels launched, 0: it would take longer than `limit` ns, -1: failed
int launch_kv8_attention_tc(const Kv8AttnArgs& a, int64_t limit, cudaStream_t stream);

namespace {

constexpr int RW = 4;                    // warps of a CTA
constexpr int MT = 2;                    // 16-key tiles of a warp's step
constexpr int RSTEP = 16 * MT;
constexpr int RSTAGES = 3;
// Fewest keys of a split.  With 8 rows a CTA one cluster takes 128: one row, 1664 keys 6.7 us in 8 splits, 8.3 in 4; 32 rows and sums over
// clusters are worse off (32 rows, 1000 keys: 13.9 and 11.5 us).
constexpr int kMinSplit = 256, kMinSplitNarrow = 128;
constexpr int kSlots = 2;                // CTAs of an SM
// tenths of a nanosecond that a key takes a CTA
template <int D, int NT>
constexpr int kKeyNs = (NT == 4 ? 175 : 130) * D / 128;

__device__ __forceinline__ void mma_f16_16816(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16_16816_first(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};\n"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool on) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(dst), "l"(src) : "memory");
}
// the copies asked for are there but for the newest N groups; what is read from them stays behind this
template <int N>
__device__ __forceinline__ void ring_wait() { asm volatile("cp.async.wait_group %0;\n" ::"n"(N) : "memory"); }
template <int WORDS>
__device__ __forceinline__ void lds(const unsigned char* from, uint32_t* w) {
    if constexpr (WORDS == 4) {
        const uint4 v = *reinterpret_cast<const uint4*>(from);
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    } else {
        const uint2 v = *reinterpret_cast<const uint2*>(from);
        w[0] = v.x; w[1] = v.y;
    }
}

template <int D, int NT>
struct RowsLayout {
    static constexpr int ROWS = 8 * NT;
    static constexpr int KCH = D / 64;                       // 16-byte pieces of a key row per thread
    static constexpr int VB = D / 8;                         // bytes of a value row per thread (8 threads share a row)
    static constexpr int HALF = RSTEP * D;                   // bytes of a warp's stage: keys, then values
    static constexpr int STAGE = 2 * HALF;
    static constexpr int RING = RW * RSTAGES * STAGE;
    static constexpr int MERGE = (RW * ROWS * (D + 4) + ROWS * (D + 1)) * 4;    // after the loop: the warps' results, the CTA's
    static constexpr int SMEM = RING > MERGE ? RING : MERGE;
};

// item = (request, KV head, tile of 8 NT rows); rows of a KV head: query row i, head g of its group -> i G + g.
// grid (splits, row tiles, B Hkv).  The keys of a split are dealt out to the warps step by step.
template <int D, int NT, int FMT>
__global__ void __launch_bounds__(RW * 32, NT < 4 ? kSlots : 1) kv8_attn_rows_kernel(const Kv8AttnArgs a) {
    using L = RowsLayout<D, NT>;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float stat[2][RW][8 * NT];                    // reference, denominator
    __shared__ int top_v[RW], is_last;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    pdl_wait();
    pdl_launch_dependents();
    const int split = blockIdx.x, tile = blockIdx.y, b = blockIdx.z / a.n_kv_heads, kvh = blockIdx.z % a.n_kv_heads;
    const int G = a.n_heads / a.n_kv_heads, R = a.n * G;
    int len = a.ctx_len;
    if (a.lens) {
        len = a.lens[b];
        if (len < 0 || len > a.ctx_len) {
            if (tid == 0) atomicOr(a.status, kFlagBadIndex);
            len = min(max(len, 0), a.ctx_len);
        }
    }
    const int key_lo = split * a.split_keys, key_hi = min(len, key_lo + a.split_keys);
    const int steps = key_hi > key_lo ? (key_hi - key_lo + RSTEP - 1) / RSTEP : 0;
    const int64_t cache_at = (int64_t)b * a.batch_stride + (int64_t)kvh * a.capacity * D;
    const uint8_t *kb = a.k + cache_at, *vb = a.v + cache_at;
    const unsigned char* ring = smem + warp * (RSTAGES * L::STAGE);
    // A warp's copies take whole rows, side by side; where a row's 16-byte pieces lie in the ring depends on the row, so that the
    // fragments' reads (other rows in other threads) meet different banks.  Pieces per row: 8, at head dimension 64 4.
    constexpr int PIECES = D / 16;
    auto k_at = [](int row, int piece) { return row * D + ((D == 128 ? piece ^ ((row & 1) << 2) : piece ^ ((row >> 1) & 3)) << 4); };
    auto v_at = [](int row, int piece) { return row * D + ((D == 128 ? piece ^ (row & 6) : piece ^ ((row >> 1) & 3)) << 4); };

    // a lane's piece of the first rows of a copy; the next ones are 32 / PIECES rows further, in the ring's values with the
    // upper bit of the swizzle turned over
    constexpr int PASS = 32 / PIECES, PASSES = RSTEP / PASS;
    const int row0 = lane / PIECES, piece = lane % PIECES;
    const uint32_t ring_at = smem_u32(ring), k_to = k_at(row0, piece), v_to = L::HALF + v_at(row0, piece), v_to_odd = L::HALF + v_at(row0 + PASS, piece);
    auto fetch = [&](int step, int stage) {          // this warp's `step`-th step into its ring
        const int s = warp + step * RW;
        if (s < steps) {
            const int key0 = key_lo + s * RSTEP;
            const uint32_t st = ring_at + stage * L::STAGE;
            if (key0 + RSTEP <= key_hi) {
                const uint8_t* from = kb + (int64_t)(key0 + row0) * D + piece * 16;
                const uint8_t* from_v = vb + (int64_t)(key0 + row0) * D + piece * 16;
#pragma unroll
                for (int i = 0; i < PASSES; ++i) {
                    cp_async16(st + k_to + i * PASS * D, from + i * PASS * D);
                    cp_async16(i % 2 == 0 || PASS >= 8 ? st + v_to + i * PASS * D : st + v_to_odd + (i - 1) * PASS * D, from_v + i * PASS * D);
                }
            } else {
#pragma unroll
                for (int i = 0; i < PASSES; ++i) {
                    const int row = i * PASS + row0;
                    const bool on = key0 + row < key_hi;
                    const int64_t at = (int64_t)(on ? key0 + row : key_lo) * D + piece * 16;
                    cp_async16(st + k_at(row, piece), kb + at, on);
                    cp_async16(st + L::HALF + v_at(row, piece), vb + at, on);
                }
            }
        }
        cp_async_commit();
    };
#pragma unroll
    for (int s = 0; s < RSTAGES - 1; ++s) fetch(s, s);

    // exponent bytes of a step's two 16-key tiles: K, K, V, V (a block holds whole tiles)
    const int64_t exps_at = ((int64_t)(a.shared ? 0 : b) * a.n_kv_heads + kvh) * a.n_blocks;
    auto exponents = [&](int step, int (&e)[2 * MT]) {
        const int key0 = key_lo + min(warp + step * RW, steps - 1) * RSTEP;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const int64_t at = exps_at + (min(key0 + mt * 16, key_hi - 1) >> a.log2_block);
            e[mt] = __ldg(a.k_exp + at);
            e[MT + mt] = __ldg(a.v_exp + at);
        }
    };
    int e_next[2 * MT] = {};
    if (warp < steps) exponents(0, e_next);
    // q as f16, each row over a power of two of its own; kept in shared memory where the registers are needed for the sums
    constexpr bool Q_SMEM = NT * D > 256;
    __shared__ uint2 qs[Q_SMEM ? (D / 16) * NT * 32 : 1];
    uint32_t qf[Q_SMEM ? 1 : NT][D / 16][2];
    float2 rq[NT];                       // what a product of row 2 t (+ 1) is multiplied by, times the key's scale
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int r = tile * L::ROWS + nt * 8 + g;
        const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(a.q) + ((int64_t)(b * (int64_t)a.n + r / G) * a.n_heads + kvh * G + r % G) * D;
        uint32_t raw[D / 8];
        uint32_t top2 = 0u;
#pragma unroll
        for (int c = 0; c < L::KCH; ++c)
#pragma unroll
            for (int hlf = 0; hlf < 2; ++hlf) {
                const uint4 v = r < R ? __ldg(reinterpret_cast<const uint4*>(q + c * 64 + t * 16) + hlf) : make_uint4(0u, 0u, 0u, 0u);
                const int at = (c * 2 + hlf) * 4;
                raw[at] = v.x; raw[at + 1] = v.y; raw[at + 2] = v.z; raw[at + 3] = v.w;
            }
#pragma unroll
        for (int i = 0; i < D / 8; ++i) top2 = __vmaxu2(top2, raw[i] & 0x7F807F80u);
        top2 = __vmaxu2(top2, __shfl_xor_sync(0xffffffffu, top2, 1));
        top2 = __vmaxu2(top2, __shfl_xor_sync(0xffffffffu, top2, 2));
        // exponent field of the row's largest value; an infinity or a NaN stays what it is
        const int field = min(max((int)(max(top2 & 0xFFFFu, top2 >> 16) >> 7), 1), 253);
        const float inv = __int_as_float((254 - field) << 23);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
            const uint32_t q0 = pack_f16(bf16_lo(raw[2 * ks]) * inv, bf16_hi(raw[2 * ks]) * inv);
            const uint32_t q1 = pack_f16(bf16_lo(raw[2 * ks + 1]) * inv, bf16_hi(raw[2 * ks + 1]) * inv);
            if constexpr (Q_SMEM) {
                if (warp == 0) qs[(ks * NT + nt) * 32 + lane] = make_uint2(q0, q1);
            } else {
                qf[nt][ks][0] = q0;
                qf[nt][ks][1] = q1;
            }
        }
        const float mine = __int_as_float(field << 23) * a.scale_log2e;      // of row g; the products' columns are rows 2 t, 2 t + 1
        rq[nt].x = __shfl_sync(0xffffffffu, mine, 8 * t);
        rq[nt].y = __shfl_sync(0xffffffffu, mine, 8 * t + 4);
    }

    if constexpr (Q_SMEM) __syncthreads();

    float o[D / 16][NT][4];
    float2 m[NT], l[NT];                 // references and denominators of rows 2 t, 2 t + 1
    bool first = true;                   // no key yet: the same for all rows, a key counts for all of them or for none
    int e0 = 0;                          // E0, biased; 0: no value that counts met yet
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        m[nt] = l[nt] = make_float2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][nt][j] = 0.f;
    }

    int stage = 0;                       // step % RSTAGES
    for (int step = 0; warp + step * RW < steps; ++step) {
        const int s = warp + step * RW, key0 = key_lo + s * RSTEP;
        const uint32_t st = stage * L::STAGE;
        uint32_t there = key_hi - key0 >= RSTEP ? ~0u : (1u << (key_hi - key0)) - 1u;      // the step's keys that count
        if (a.key_drop) there &= ~__ldg(a.key_drop + (int64_t)b * a.drop_words + (key0 >> 5));
        int ek[MT], ev[MT];
        bool blank[MT], no_keys = false;      // a block that holds nothing has zero keys and values, whatever its codes
        int most = e0;                        // (nor has a tile without a key that counts any values)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            ek[mt] = e_next[mt];
            ev[mt] = e_next[MT + mt];
            no_keys |= ek[mt] == 0;
            blank[mt] = ev[mt] == 0 || ((there >> (mt * 16)) & 0xFFFFu) == 0u;
            most = blank[mt] ? most : max(most, ev[mt]);
        }
        if (most > e0) {
            // so far nothing but tiles without values, under E0 = 127: they have this scale as well as any, and M moves along with it
            const float grow = e0 ? kv8_scale(127 + min(most - e0, kFarApart)) : 1.f, along = e0 ? 0.f : (float)(most - 127);
            e0 = most;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                l[nt].x *= grow; l[nt].y *= grow;
                m[nt].x += along; m[nt].y += along;
            }
        }
        const int e_top = e0 ? e0 : 127;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) ev[mt] = blank[mt] ? e_top : ev[mt];
        exponents(step + 1, e_next);
        ring_wait<RSTAGES - 2>();
        __syncwarp();                        // this step's stage is there for every lane, and every lane is done with the last one's
        fetch(step + RSTAGES - 1, stage == 0 ? RSTAGES - 1 : stage - 1);
        stage = stage == RSTAGES - 1 ? 0 : stage + 1;
        // ---- S^T = K Q^T, then y - M in place ----
        float sv[MT][NT][4];
#pragma unroll
        for (int c = 0; c < L::KCH; ++c) {
            uint32_t kw[MT][2][4];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int r = 0; r < 2; ++r) lds<4>(ring + st + k_at(mt * 16 + r * 8 + g, c * 4 + t), kw[mt][r]);
            if (no_keys) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int r = 0; r < 2; ++r)
#pragma unroll
                        for (int w = 0; w < 4; ++w) kw[mt][r][w] = ek[mt] ? kw[mt][r][w] : 0u;
            }
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                uint32_t fa[MT][4];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    kv8_to_f16<FMT>(kw[mt][0][w], fa[mt][0], fa[mt][2]);
                    kv8_to_f16<FMT>(kw[mt][1][w], fa[mt][1], fa[mt][3]);
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    uint2 q;
                    if constexpr (Q_SMEM) q = qs[((c * 4 + w) * NT + nt) * 32 + lane];
                    else q = make_uint2(qf[nt][c * 4 + w][0], qf[nt][c * 4 + w][1]);
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {
                        if (c == 0 && w == 0) mma_f16_16816_first(sv[mt][nt], fa[mt], q.x, q.y);
                        else mma_f16_16816(sv[mt][nt], fa[mt], q.x, q.y);
                    }
                }
            }
        }
        float top = -INFINITY;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const float ks = kv8_scale(ek[mt]), vy = (float)(max(ev[mt], e_top - kFarApart) - 127);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float2 fa = __fmul2_rn(rq[nt], make_float2(ks, ks)), fb = __fadd2_rn(make_float2(vy, vy), make_float2(-m[nt].x, -m[nt].y));
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const float2 y = __ffma2_rn(make_float2(sv[mt][nt][2 * r], sv[mt][nt][2 * r + 1]), fa, fb);
                    sv[mt][nt][2 * r] = y.x;
                    sv[mt][nt][2 * r + 1] = y.y;
                }
            }
        }
        if (there != ~0u) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (!((there >> (mt * 16 + (j >> 1) * 8 + g)) & 1u))
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) sv[mt][nt][j] = -INFINITY;
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) top = fmaxf(fmaxf(fmaxf(fmaxf(top, sv[mt][nt][0]), sv[mt][nt][1]), sv[mt][nt][2]), sv[mt][nt][3]);
        if (__any_sync(0xffffffffu, top > kRaise || (first && there != 0u))) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    float x = sv[0][nt][r];
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) x = fmaxf(x, fmaxf(sv[mt][nt][r], sv[mt][nt][r + 2]));
                    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
                    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
                    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
                    if (x > kStart || (first && x > -INFINITY)) {       // (the others take the opportunity)
                        x -= kStart;
                        const float f = first ? 0.f : ex2(-x);       // before the first key there is nothing to scale
                        if (r == 0) { m[nt].x += x; l[nt].x *= f; }
                        else { m[nt].y += x; l[nt].y *= f; }
#pragma unroll
                        for (int i = 0; i < D / 16; ++i) {
                            o[i][nt][r] *= f;
                            o[i][nt][r + 2] *= f;
                        }
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) {
                            sv[mt][nt][r] -= x;
                            sv[mt][nt][r + 2] -= x;
                        }
                    }
                }
            first = false;
        }
        // ---- P, and O^T += V^T P^T ----
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            uint32_t pf[NT][2];
            const float lw = kv8_weight(e_top - ev[mt]);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float p0 = ex2(sv[mt][nt][0]), p1 = ex2(sv[mt][nt][1]), p2 = ex2(sv[mt][nt][2]), p3 = ex2(sv[mt][nt][3]);
                l[nt] = __ffma2_rn(__fadd2_rn(make_float2(p0, p1), make_float2(p2, p3)), make_float2(lw, lw), l[nt]);
                pf[nt][0] = transpose8(pack_f16(p0, p1));
                pf[nt][1] = transpose8(pack_f16(p2, p3));
            }
            constexpr int VW = L::VB / 4;
            uint32_t vw[4][VW];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                lds<VW>(ring + st + L::HALF + v_at(mt * 16 + 2 * t + (j & 1) + (j >> 1) * 8, g * L::VB / 16) + g * L::VB % 16, vw[j]);
            const uint32_t keys16 = (there >> (mt * 16)) & 0xFFFFu;
            if (keys16 != 0xFFFFu || blank[mt]) {              // values of keys that do not count may be anything
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bool on = !blank[mt] && ((keys16 >> (2 * t + (j & 1) + (j >> 1) * 8)) & 1u);
#pragma unroll
                    for (int w = 0; w < VW; ++w) vw[j][w] = on ? vw[j][w] : 0u;
                }
            }
#pragma unroll
            for (int w = 0; w < VW; ++w) {
                uint32_t fe[4], fo[4];       // d 2 w' and 2 w' + 1 of two products
                kv8_to_f16<FMT>(__byte_perm(vw[0][w], vw[1][w], 0x5140), fe[0], fe[1]);
                kv8_to_f16<FMT>(__byte_perm(vw[2][w], vw[3][w], 0x5140), fe[2], fe[3]);
                kv8_to_f16<FMT>(__byte_perm(vw[0][w], vw[1][w], 0x7362), fo[0], fo[1]);
                kv8_to_f16<FMT>(__byte_perm(vw[2][w], vw[3][w], 0x7362), fo[2], fo[3]);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    mma_f16_16816(o[2 * w][nt], fe, pf[nt][0], pf[nt][1]);
                    mma_f16_16816(o[2 * w + 1][nt], fo, pf[nt][0], pf[nt][1]);
                }
            }
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
                stat[0][warp][nt * 8 + 2 * t + r] = first ? -INFINITY : r ? m[nt].y : m[nt].x;
                stat[1][warp][nt * 8 + 2 * t + r] = x;
            }
        }
    if (lane == 0) top_v[warp] = e0;
    ring_wait<0>();
    __syncthreads();                         // nobody reads the ring any more
    float* os = reinterpret_cast<float*>(smem);      // [warp][row][D + 4]
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            float4* to = reinterpret_cast<float4*>(os + (warp * L::ROWS + nt * 8 + 2 * t + r) * (D + 4) + g * (D / 8));
#pragma unroll
            for (int i = 0; i < D / 32; ++i)
                to[i] = make_float4(o[2 * i][nt][r], o[2 * i][nt][r + 2], o[2 * i + 1][nt][r], o[2 * i + 1][nt][r + 2]);
        }
    __syncthreads();
    const int item = blockIdx.z * gridDim.y + tile;
#pragma unroll
    for (int w = 0; w < RW; ++w) e0 = max(e0, top_v[w]);
    e0 = e0 ? e0 : 127;
    const float up = kv8_unbias(e0);
    float along[RW], grow[RW];               // of a warp's reference and denominator, on the way to the CTA's E0 (as in the loop)
#pragma unroll
    for (int w = 0; w < RW; ++w) {
        along[w] = top_v[w] ? 0.f : (float)(e0 - 127);
        grow[w] = top_v[w] ? kv8_scale(127 + min(e0 - top_v[w], kFarApart)) : 1.f;
    }
    constexpr int TPR = D / 4;               // threads of a row, 4 values each
    const int cs = a.cluster, parts = a.splits / cs;
    float* part_o = a.part;                  // [item][part][row][D], then [item][part][row] log2 of the denominators
    float* part_l = a.part + (int64_t)gridDim.y * gridDim.z * parts * L::ROWS * D;
    const int64_t part0 = ((int64_t)item * parts + split / cs) * L::ROWS;
    auto give = [&](int row, int c, float4 v, float lse2) {          // a result of all that this launch has to add up, or of a part of it
        if (parts > 1) {
            *reinterpret_cast<float4*>(part_o + (part0 + row) * D + c * 4) = v;
            if (c == 0) part_l[part0 + row] = lse2;
            return;
        }
        const int r = tile * L::ROWS + row;
        const int64_t at = (int64_t)(b * (int64_t)a.n + r / G) * a.n_heads + kvh * G + r % G;
        *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.o) + at * D + c * 4) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
        if (a.lse && c == 0) a.lse[at] = lse2 * 0.6931471805599453f;
    };
    float* res = os + RW * L::ROWS * (D + 4);            // [row][D], then [row]: this CTA's result, for the others of its cluster
    for (int i = tid; i < L::ROWS * TPR; i += RW * 32) {
        const int row = i / TPR, c = i % TPR;
        if (tile * L::ROWS + row >= R) continue;
        float mx = -INFINITY;
#pragma unroll
        for (int w = 0; w < RW; ++w) mx = fmaxf(mx, stat[0][w][row] + along[w]);
        float den = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < RW; ++w) {
            const float mw = stat[0][w][row] + along[w];
            // a NaN in the sums has to come through; a warp that met no key has sums of zero
            const float f = mw == -INFINITY ? 1.f : ex2(mw - mx);
            const float4 x = *reinterpret_cast<const float4*>(os + (w * L::ROWS + row) * (D + 4) + c * 4);
            den = fmaf(f, stat[1][w][row] * grow[w], den);
            v.x = fmaf(f, x.x, v.x); v.y = fmaf(f, x.y, v.y); v.z = fmaf(f, x.z, v.z); v.w = fmaf(f, x.w, v.w);
        }
        const float s = den == 0.f ? 0.f : 1.f / den;
        v.x = v.x * s * up; v.y = v.y * s * up; v.z = v.z * s * up; v.w = v.w * s * up;
        const float lse2 = den == 0.f ? -INFINITY : mx - (float)(e0 - 127 - kWeightBias) + log2f(den);
        if (cs == 1) {
            give(row, c, v, lse2);
        } else {
            *reinterpret_cast<float4*>(res + row * D + c * 4) = v;
            if (c == 0) res[L::ROWS * D + row] = lse2;
        }
    }
    if (cs > 1) {
        // ---- the CTAs of a cluster add their results up, each for a share of the values, in the order of their keys ----
        cluster_sync_all();
        const uint32_t res_at = smem_u32(res);
        for (int i = tid + split % cs * RW * 32; i < L::ROWS * TPR; i += cs * RW * 32) {
            const int row = i / TPR, c = i % TPR;
            if (tile * L::ROWS + row >= R) continue;
            float x[8];
            float4 w[8];
#pragma unroll
            for (int p = 0; p < 8; ++p) {
                x[p] = -INFINITY;
                if (p < cs) {
                    x[p] = ld_peer(mapa_u32(res_at + (L::ROWS * D + row) * 4, p));
                    w[p] = ld_peer4(mapa_u32(res_at + (row * D + c * 4) * 4, p));
                }
            }
            Sum s;
#pragma unroll
            for (int p = 0; p < 8; ++p) s.add(x[p], w[p]);
            give(row, c, s.mean(), s.lse2());
        }
        cluster_sync_all();                  // nobody leaves while its results are read
    }
    if (parts == 1) return;
    // ---- of the CTAs with the same share, the last one adds the parts up, in their order ----
    const int rank = split % cs;
    __threadfence();
    __syncthreads();
    if (tid == 0) {
        unsigned* arrived = a.arrived + item * cs + rank;
        is_last = atomicAdd(arrived, 1u) == (unsigned)parts - 1u;
        if (is_last) *arrived = 0u;
    }
    __syncthreads();
    if (!is_last) return;
    __threadfence();
    const int64_t p0 = (int64_t)item * parts * L::ROWS;
    for (int i = tid + rank * RW * 32; i < L::ROWS * TPR; i += cs * RW * 32) {
        const int row = i / TPR, c = i % TPR, r = tile * L::ROWS + row;
        if (r >= R) continue;
        Sum s;
        for (int q0 = 0; q0 < parts; q0 += 8) {
            float x[8];
            float4 w[8];
#pragma unroll
            for (int p = 0; p < 8; ++p) {
                x[p] = -INFINITY;
                if (q0 + p < parts) {
                    x[p] = __ldcg(part_l + p0 + (int64_t)(q0 + p) * L::ROWS + row);
                    w[p] = __ldcg(reinterpret_cast<const float4*>(part_o + (p0 + (int64_t)(q0 + p) * L::ROWS + row) * D + c * 4));
                }
            }
#pragma unroll
            for (int p = 0; p < 8; ++p) s.add(x[p], w[p]);
        }
        const float4 v = s.mean();
        const int64_t at = (int64_t)(b * (int64_t)a.n + r / G) * a.n_heads + kvh * G + r % G;
        *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.o) + at * D + c * 4) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
        if (a.lse && c == 0) a.lse[at] = s.lse2() * 0.6931471805599453f;
    }
}

template <int D, int NT, int FMT>
void rows_config(cudaLaunchConfig_t& cfg, cudaLaunchAttribute (&at)[2], dim3 grid, int cluster, cudaStream_t stream) {
    cfg = cudaLaunchConfig_t{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(RW * 32);
    cfg.dynamicSmemBytes = RowsLayout<D, NT>::SMEM;
    cfg.stream = stream;
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
}
// [c]: clusters of 2^c CTAs that the current device runs at a time: fewer than the places for CTAs make up, as a cluster stays in one
// group of SMs
template <int D, int NT, int FMT>
std::array<int, 4> rows_clusters() {
    static PerDevice<std::array<int, 4>> fits;
    int device = 0;
    cudaGetDevice(&device);
    return fits.of(device, [](std::array<int, 4>& fit) {
        cudaFuncSetAttribute(kv8_attn_rows_kernel<D, NT, FMT>, cudaFuncAttributeMaxDynamicSharedMemorySize, RowsLayout<D, NT>::SMEM);
        for (int i = 3; i >= 0; --i) {
            cudaLaunchConfig_t cfg;
            cudaLaunchAttribute at[2];
            rows_config<D, NT, FMT>(cfg, at, dim3(1 << i), 1 << i, nullptr);
            cfg.attrs = at + 1;                           // the cluster alone
            cfg.numAttrs = 1;
            int most = 0;
            if (cudaOccupancyMaxActiveClusters(&most, kv8_attn_rows_kernel<D, NT, FMT>, &cfg) != cudaSuccess) most = 0;
            fit[i] = std::min(std::max(most, 1), (kSlots * 148) >> i);
        }
    });
}
struct RowsPlan { int cluster, splits; int64_t cost; };   // cost: ns
// Key splits, in clusters that add their results up; splits only where all their CTAs run at a time.  The estimate, with what was
// measured for 32 rows of 128 (and for fewer): a CTA takes 4 us and 17.5 (13) ns a key, where two share an SM 9 (5.2) us and the same;
// the sum over a cluster 5 (1.5) us, 1.5 us where two share an SM; the sum over clusters 2 us and 0.8 us for every eight of them and
// every value of a thread.  More CTAs than places take as many times longer, and a quarter for the last ones.  One
// sequence of 65536 keys, 4 KV heads, 35 rows (8 items): 49 us in 4 clusters of 8 each, 72 us in 9 of 4 (72, where 71 run at a time);
// 512 items of 8192 keys: 166 us whole, 180 us in halves.
template <int D, int NT, int FMT>
RowsPlan rows_plan(const Kv8AttnArgs& a) {
    using L = RowsLayout<D, NT>;
    const int R = a.n * (a.n_heads / a.n_kv_heads);
    const int64_t items = (int64_t)((R + L::ROWS - 1) / L::ROWS) * a.batch * a.n_kv_heads;
    RowsPlan best{1, 1, INT64_MAX};
    const int most = a.ctx_len / kMinSplit, most_one = a.ctx_len / (NT == 1 ? kMinSplitNarrow : kMinSplit);
    const std::array<int, 4> fits = rows_clusters<D, NT, FMT>();
    for (int c = 0; c < 4 && (c == 0 || 1 << c <= most_one); ++c) {
        const int fit = fits[c];
        if (c > 0 && items > fit) break;
        const int top = c == 0 ? 1 : std::max(1, (int)std::min<int64_t>(fit / items, most >> c));
        for (int k = 1;; k = top) {                       // one cluster an item, or as many as there is room for
            const int splits = k << c, keys = (a.ctx_len + splits - 1) / splits;
            const bool two = items * splits > 148;
            int64_t cost = (!two ? 4000 : NT == 4 ? 9000 : 5200) + (int64_t)keys * kKeyNs<D, NT> / 10;
            if (items > fit) cost = cost * (items * 4 + fit) / (fit * 4);
            if (c > 0) cost += NT == 4 && !two ? 5000 : 1500;
            if (k > 1) cost += 2000 + 800 * ((L::ROWS * D / (4 * RW * 32) + (1 << c) - 1) >> c) * ((k + 7) / 8);
            if (cost < best.cost) best = RowsPlan{1 << c, splits, cost};
            if (k == top) break;
        }
    }
    return best;
}
template <int D, int NT, int FMT>
int rows_launch(Kv8AttnArgs a, const RowsPlan& plan, cudaStream_t stream) {
    const int R = a.n * (a.n_heads / a.n_kv_heads), tiles = (R + 8 * NT - 1) / (8 * NT);
    a.cluster = plan.cluster;
    a.splits = plan.splits;
    a.split_keys = ((a.ctx_len + a.splits - 1) / a.splits + RSTEP - 1) / RSTEP * RSTEP;
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute at[2];
    rows_config<D, NT, FMT>(cfg, at, dim3(a.splits, tiles, a.batch * a.n_kv_heads), a.cluster, stream);
    return cudaLaunchKernelEx(&cfg, kv8_attn_rows_kernel<D, NT, FMT>, a) == cudaSuccess ? 1 : -1;
}
// Rows of a CTA: up to 32, so that a key is converted once for as many of them as there are; fewer where there are too few CTAs to
// go round.  us with 8, 16 and 32 rows a CTA: 4 KV heads, 28 rows, 1536 keys 8.3, 10.3, 14.3; 16 times as many requests 20.8, 17.5,
// 17.9, and 8192 keys 84, 56, 49; 32 KV heads, 1536 keys, 32 rows 12.8, 12.1, 15.6, 16 rows 9.8, 10.8.
// More than 32 rows: the tensor-memory kernel, where its plan takes less than this one's.  16 sequences, 32 KV heads, 100 rows,
// 8192 keys: 501 us there, 953 us here; one sequence of 300 keys: 12.3 and 10.0 us.  Up to 32 rows this one is ahead: 16 sequences, 32 KV
// heads, 32 rows, 2560 keys 183 us there, 109 here; one of 8288 keys 44 and 31; 64 of 28 rows, 4 KV heads, 8192 keys 274 and 151.
template <int D, int FMT>
int rows_dispatch(const Kv8AttnArgs& a, cudaStream_t stream) {
    const int R = a.n * (a.n_heads / a.n_kv_heads);
    const int64_t pairs = (int64_t)a.batch * a.n_kv_heads, splits = std::max(1, a.ctx_len / kMinSplit);
    auto ctas = [&](int rows) { return (R + rows - 1) / rows * pairs * splits; };
    const int few = R > 32 ? 148 : 222;                   // (of more than 32 rows, the tensor-memory kernel takes some of those between)
    const int nt = R <= 8 || ctas(16) < few ? 1 : R <= 16 || ctas(32) < few ? 2 : 4;
    if (nt == 1) return rows_launch<D, 1, FMT>(a, rows_plan<D, 1, FMT>(a), stream);
    if (nt == 2) return rows_launch<D, 2, FMT>(a, rows_plan<D, 2, FMT>(a), stream);
    const RowsPlan plan = rows_plan<D, 4, FMT>(a);
    if (D == 128 && R > 32) {
        const int r = launch_kv8_attention_tc(a, plan.cost, stream);
        if (r != 0) return r;
    }
    return rows_launch<D, 4, FMT>(a, plan, stream);
}

}  // namespace

size_t kv8_attention_scratch_bytes(int head_dim) {
    // keys are split only below an item per place for a CTA: no more results than places, of up to 32 rows
    return (size_t)kSlots * 148 * 32 * (head_dim + 1) * sizeof(float);
}

int launch_kv8_attention(const Kv8AttnArgs& a, cudaStream_t stream) {
    if (a.batch == 0 || a.n == 0) return 0;
    if (a.head_dim == 128) return a.format == kKv8Int8 ? rows_dispatch<128, kKv8Int8>(a, stream) : rows_dispatch<128, kKv8E4m3>(a, stream);
    return a.format == kKv8Int8 ? rows_dispatch<64, kKv8Int8>(a, stream) : rows_dispatch<64, kKv8E4m3>(a, stream);
}

}  // namespace acache
