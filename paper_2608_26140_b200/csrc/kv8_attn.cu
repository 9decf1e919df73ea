// Attention over the 8-bit cache.
//
//   o_r = sum_j 2^(x_rj - M) V_j / sum_j 2^(x_rj - M),   x_rj = log2(e) / sqrt(d) q_r K_j
//
// with K_j = 2^(ek) k_j, V_j = 2^(ev) v_j, k_j and v_j the codes: whole numbers or e4m3 values, exact in f16.  The products
// run on the codes; ek joins the factor that turns a product into x, ev the exponent:
//   y_rj = x_rj + ev,   p_rj = 2^(y_rj - M)  (M: running reference of y),   O = sum p v,   l = sum p 2^(E0 - ev)
// so that o = 2^E0 O / l with E0 the largest ev met so far (l follows it), and no code is ever multiplied by its scale.  The
// scales of one head's values may differ by 2^100, which is where the weights in l end.  p is f16:
// V's codes are f16 whatever their scales, which leaves p 11 bits (with bf16 operands, 8).  q is f16 too, each row over a
// power of two of its own that brings its largest value to [1, 2).
//
// Bound by HBM on the codes.  A warp streams keys on its own: the bytes go from the cache to a ring in shared memory in
// which every thread has its own slots (cp.async; a thread reads back what it asked for, so no barrier), from there to
// registers, become matrix-instruction fragments there and are used for all the rows.  The order of d inside a product is
// free, so a thread's 16 contiguous bytes of a key row serve as its fragment of four products:
//   S^T = K Q^T (keys x rows)   O^T += V^T P^T (d x rows): keys and d are the long sides of both products, so up to 8 rows cost
//   one instruction, and P only has to be transposed in 8 x 8 blocks (movmatrix).
// The reference M moves only when a logit passes it by 2^8, found by a vote; then maxima are exchanged and O is scaled.
#include "kernels.h"
#include "kv8.cuh"
#include "launch.h"

namespace acache {

namespace {

constexpr int RW = 4;                    // warps of a CTA
constexpr int RSTEP = 32;                // keys of a warp's step (two 16-key tiles)
constexpr int RSTAGES = 3;
constexpr float kRaise = 8.f;            // log2 units
constexpr int kFarApart = 100;           // most by which E0 is above an ev

__device__ __forceinline__ void mma_f16_16816(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
template <int BYTES>
__device__ __forceinline__ void cp_async(uint32_t dst, const void* src, bool on) {
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(dst), "l"(src), "r"(on ? 16 : 0));
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;\n" ::"r"(dst), "l"(src), "r"(on ? 8 : 0));
}
template <int WORDS>
__device__ __forceinline__ void lds(uint32_t addr, uint32_t* w) {
    if constexpr (WORDS == 4)
        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(addr));
    else asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(addr));
}

template <int D, int NT>
struct RowsLayout {
    static constexpr int ROWS = 8 * NT;
    static constexpr int KCH = D / 64;                       // 16-byte pieces of a key row per thread
    static constexpr int VB = D / 8;                         // bytes of a value row per thread (8 threads share a row)
    static constexpr int K_SLOTS = 2 * 2 * KCH, V_SLOTS = 2 * 4;
    static constexpr int K_BYTES = K_SLOTS * 16 * 32, V_BYTES = V_SLOTS * VB * 32;   // of a warp's stage
    static constexpr int STAGE = K_BYTES + V_BYTES;
    static constexpr int RING = RW * RSTAGES * STAGE;
    static constexpr int MERGE = RW * ROWS * (D + 4) * 4;    // the warps' results, after the loop
    static constexpr int SMEM = RING > MERGE ? RING : MERGE;
};

// item = (request, KV head, tile of 8 NT rows); rows of a KV head: query row i, head g of its group -> i G + g.
// grid (splits, row tiles, B Hkv).  The keys of a split are dealt out to the warps step by step.
template <int D, int NT, int FMT>
__global__ void __launch_bounds__(RW * 32) kv8_attn_rows_kernel(const Kv8AttnArgs a) {
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
    const uint32_t ring = smem_u32(smem) + warp * (RSTAGES * L::STAGE) + lane * 16;
    const uint32_t vring = smem_u32(smem) + warp * (RSTAGES * L::STAGE) + L::K_BYTES + lane * L::VB;

    auto fetch = [&](int step) {         // this warp's `step`-th step into its ring
        const int s = warp + step * RW;
        if (s < steps) {
            const int key0 = key_lo + s * RSTEP;
            const uint32_t st = (step % RSTAGES) * L::STAGE;
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int c = 0; c < L::KCH; ++c) {
                        const int key = key0 + mt * 16 + r * 8 + g;
                        cp_async<16>(ring + st + ((mt * 2 + r) * L::KCH + c) * 512, kb + (int64_t)min(key, key_hi - 1) * D + c * 64 + t * 16, key < key_hi);
                    }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int key = key0 + mt * 16 + 2 * t + (j & 1) + (j >> 1) * 8;
                    cp_async<L::VB>(vring + st + (mt * 4 + j) * (L::VB * 32), vb + (int64_t)min(key, key_hi - 1) * D + g * L::VB, key < key_hi);
                }
            }
        }
        cp_async_commit();
    };
#pragma unroll
    for (int s = 0; s < RSTAGES - 1; ++s) fetch(s);

    // exponent bytes of a step's two 16-key tiles: K, K, V, V (a block holds whole tiles)
    const int64_t exps_at = ((int64_t)(a.shared ? 0 : b) * a.n_kv_heads + kvh) * a.n_blocks;
    auto exponents = [&](int step, int (&e)[4]) {
        const int key0 = key_lo + min(warp + step * RW, steps - 1) * RSTEP;
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
            const int64_t at = exps_at + (min(key0 + mt * 16, key_hi - 1) >> a.log2_block);
            e[mt] = __ldg(a.k_exp + at);
            e[2 + mt] = __ldg(a.v_exp + at);
        }
    };
    int e_next[4] = {0, 0, 0, 0};
    if (warp < steps) exponents(0, e_next);
    // q as f16, each row over a power of two of its own
    uint32_t qf[NT][D / 16][2];
    float rq[NT][2];                     // what a product of row 2 t (+ 1) is multiplied by, times the key's scale
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
            qf[nt][ks][0] = pack_f16(bf16_lo(raw[2 * ks]) * inv, bf16_hi(raw[2 * ks]) * inv);
            qf[nt][ks][1] = pack_f16(bf16_lo(raw[2 * ks + 1]) * inv, bf16_hi(raw[2 * ks + 1]) * inv);
        }
        const float mine = __int_as_float(field << 23) * a.scale_log2e;      // of row g; the products' columns are rows 2 t, 2 t + 1
        rq[nt][0] = __shfl_sync(0xffffffffu, mine, 8 * t);
        rq[nt][1] = __shfl_sync(0xffffffffu, mine, 8 * t + 4);
    }

    float o[D / 16][NT][4];
    float m[NT][2], l[NT][2];
    int e0 = 0;                          // biased; 0: nothing met yet
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        m[nt][0] = m[nt][1] = -INFINITY;
        l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][nt][j] = 0.f;
    }

    for (int step = 0; warp + step * RW < steps; ++step) {
        const int s = warp + step * RW, key0 = key_lo + s * RSTEP;
        const uint32_t st = (step % RSTAGES) * L::STAGE;
        uint32_t there = key_hi - key0 >= 32 ? ~0u : (1u << (key_hi - key0)) - 1u;      // the step's keys that count
        if (a.key_drop) {
            // keys of a split start at a multiple of 32
            const int w = key0 >> 5;
            if (w < a.drop_words) there &= ~__ldg(a.key_drop + (int64_t)b * a.drop_words + w);
        }
        int ek[2], ev[2];
        bool blank[2];                       // a block that holds nothing has zero keys and values, whatever its codes
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
            ek[mt] = e_next[mt];
            ev[mt] = e_next[2 + mt];
            blank[mt] = ev[mt] == 0;
            if (blank[mt]) ev[mt] = e0 ? e0 : 127;      // its scale is of no account
            if (ev[mt] > e0) {
                const float grow = kv8_scale(127 + min(ev[mt] - e0, kFarApart));
                e0 = ev[mt];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) { l[nt][0] *= grow; l[nt][1] *= grow; }
            }
        }
        exponents(step + 1, e_next);
        cp_async_wait<RSTAGES - 2>();
        // ---- S^T = K Q^T, then y - M in place ----
        float sv[2][NT][4];
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 4; ++j) sv[mt][nt][j] = 0.f;
#pragma unroll
            for (int c = 0; c < L::KCH; ++c) {
                uint32_t k0[4], k1[4];
                lds<4>(ring + st + ((mt * 2 + 0) * L::KCH + c) * 512, k0);
                lds<4>(ring + st + ((mt * 2 + 1) * L::KCH + c) * 512, k1);
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    uint32_t fa[4];
                    kv8_to_f16<FMT>(k0[w], fa[0], fa[2]);
                    kv8_to_f16<FMT>(k1[w], fa[1], fa[3]);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma_f16_16816(sv[mt][nt], fa, qf[nt][c * 4 + w][0], qf[nt][c * 4 + w][1]);
                }
            }
        }
        bool raise = false;
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
            const float ks = kv8_scale(ek[mt]);
            const float vy = (float)(max(ev[mt], e0 - kFarApart) - 127);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float off = vy - (m[nt][j & 1] == -INFINITY ? 0.f : m[nt][j & 1]);
                    sv[mt][nt][j] = ek[mt] ? fmaf(sv[mt][nt][j], rq[nt][j & 1] * ks, off) : off;
                }
        }
        if (there != ~0u) {
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (!((there >> (mt * 16 + (j >> 1) * 8 + g)) & 1u))
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) sv[mt][nt][j] = -INFINITY;
        }
        float top[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                top[nt][r] = fmaxf(fmaxf(sv[0][nt][r], sv[0][nt][r + 2]), fmaxf(sv[1][nt][r], sv[1][nt][r + 2]));
                raise |= top[nt][r] > kRaise || (m[nt][r] == -INFINITY && top[nt][r] > -INFINITY);
            }
        if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    float x = top[nt][r];
                    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
                    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
                    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
                    const bool first = m[nt][r] == -INFINITY;
                    if (x > kRaise || (first && x > -INFINITY)) {
                        const float f = first ? 0.f : ex2(-x);
                        m[nt][r] = (first ? 0.f : m[nt][r]) + x;
                        l[nt][r] *= f;
#pragma unroll
                        for (int i = 0; i < D / 16; ++i) {
                            o[i][nt][r] *= f;
                            o[i][nt][r + 2] *= f;
                        }
#pragma unroll
                        for (int mt = 0; mt < 2; ++mt) {
                            sv[mt][nt][r] -= x;
                            sv[mt][nt][r + 2] -= x;
                        }
                    }
                }
        }
        // ---- P, and O^T += V^T P^T ----
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
            uint32_t pf[NT][2];
            const float lw = kv8_scale(127 + min(e0 - ev[mt], kFarApart));
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float p0 = ex2(sv[mt][nt][0]), p1 = ex2(sv[mt][nt][1]), p2 = ex2(sv[mt][nt][2]), p3 = ex2(sv[mt][nt][3]);
                l[nt][0] = fmaf(p0 + p2, lw, l[nt][0]);
                l[nt][1] = fmaf(p1 + p3, lw, l[nt][1]);
                pf[nt][0] = transpose8(pack_f16(p0, p1));
                pf[nt][1] = transpose8(pack_f16(p2, p3));
            }
            constexpr int VW = L::VB / 4;
            uint32_t vw[4][VW];
#pragma unroll
            for (int j = 0; j < 4; ++j) lds<VW>(vring + st + (mt * 4 + j) * (L::VB * 32), vw[j]);
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
        fetch(step + RSTAGES - 1);
    }

    // ---- the warps' results together, in their order ----
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            float x = l[nt][r];
            x += __shfl_xor_sync(0xffffffffu, x, 4);
            x += __shfl_xor_sync(0xffffffffu, x, 8);
            x += __shfl_xor_sync(0xffffffffu, x, 16);
            if (g == 0) {
                stat[0][warp][nt * 8 + 2 * t + r] = m[nt][r];
                stat[1][warp][nt * 8 + 2 * t + r] = x;
            }
        }
    if (lane == 0) top_v[warp] = e0;
    cp_async_wait<0>();
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
    const float up = kv8_scale(e0);          // 2^E0
    constexpr int TPR = D / 4;               // threads of a row, 4 values each
    float* part_o = a.part;                  // [item][split][row][D], then [item][split][row] log2 of the denominators
    float* part_l = a.part + (int64_t)gridDim.y * gridDim.z * a.splits * L::ROWS * D;
    auto finish = [&](int row, int c, float4 v, float lse2) {
        const int r = tile * L::ROWS + row;
        const int64_t at = (int64_t)(b * (int64_t)a.n + r / G) * a.n_heads + kvh * G + r % G;
        uint2 w = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
        *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.o) + at * D + c * 4) = w;
        if (a.lse && c == 0) a.lse[at] = lse2 * 0.6931471805599453f;
    };
    for (int i = tid; i < L::ROWS * TPR; i += RW * 32) {
        const int row = i / TPR, c = i % TPR;
        if (tile * L::ROWS + row >= R) continue;
        float mx = -INFINITY;
#pragma unroll
        for (int w = 0; w < RW; ++w) mx = fmaxf(mx, stat[0][w][row]);
        float den = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < RW; ++w) {
            const float mw = stat[0][w][row];
            // a NaN in the sums has to come through; a warp that met no key has sums of zero
            const float f = mw == -INFINITY ? 1.f : ex2(mw - mx);
            const float4 x = *reinterpret_cast<const float4*>(os + (w * L::ROWS + row) * (D + 4) + c * 4);
            den = fmaf(f, stat[1][w][row] * kv8_scale(127 + min(e0 - top_v[w], kFarApart)), den);
            v.x = fmaf(f, x.x, v.x); v.y = fmaf(f, x.y, v.y); v.z = fmaf(f, x.z, v.z); v.w = fmaf(f, x.w, v.w);
        }
        const float s = den == 0.f ? 0.f : up / den;
        v.x *= s; v.y *= s; v.z *= s; v.w *= s;
        const float lse2 = den == 0.f ? -INFINITY : mx - (float)(e0 - 127) + log2f(den);
        if (a.splits == 1) {
            finish(row, c, v, lse2);
        } else {
            const int64_t p = ((int64_t)item * a.splits + split) * L::ROWS + row;
            *reinterpret_cast<float4*>(part_o + p * D + c * 4) = v;
            if (c == 0) part_l[p] = lse2;
        }
    }
    if (a.splits == 1) return;
    // ---- the last CTA of the item adds the splits up, in their order ----
    __threadfence();
    __syncthreads();
    if (tid == 0) {
        const unsigned before = atomicAdd(a.arrived + item, 1u);
        is_last = before == (unsigned)a.splits - 1u;
        if (is_last) a.arrived[item] = 0u;
    }
    __syncthreads();
    if (!is_last) return;
    __threadfence();
    for (int i = tid; i < L::ROWS * TPR; i += RW * 32) {
        const int row = i / TPR, c = i % TPR;
        if (tile * L::ROWS + row >= R) continue;
        const int64_t p0 = (int64_t)item * a.splits * L::ROWS + row;
        float mx = -INFINITY;
        bool bad = false;
        for (int s = 0; s < a.splits; ++s) {
            const float x = __ldcg(part_l + p0 + (int64_t)s * L::ROWS);
            mx = fmaxf(mx, x);
            bad |= x != x;
        }
        float den = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int s = 0; s < a.splits; ++s) {
            const float x = __ldcg(part_l + p0 + (int64_t)s * L::ROWS);
            const float f = x == -INFINITY ? 0.f : ex2(x - mx);
            const float4 w = __ldcg(reinterpret_cast<const float4*>(part_o + (p0 + (int64_t)s * L::ROWS) * D + c * 4));
            den += f;
            v.x = fmaf(f, w.x, v.x); v.y = fmaf(f, w.y, v.y); v.z = fmaf(f, w.z, v.z); v.w = fmaf(f, w.w, v.w);
        }
        const float inv = bad ? __int_as_float(0x7FC00000) : (den == 0.f ? 0.f : 1.f / den);
        v.x *= inv; v.y *= inv; v.z *= inv; v.w *= inv;
        finish(row, c, v, bad ? __int_as_float(0x7FC00000) : (den == 0.f ? -INFINITY : mx + log2f(den)));
    }
}

template <int D, int NT, int FMT>
int rows_launch(Kv8AttnArgs a, cudaStream_t stream) {
    using L = RowsLayout<D, NT>;
    static bool attr = false;
    if (!attr) {
        cudaFuncSetAttribute(kv8_attn_rows_kernel<D, NT, FMT>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::SMEM);
        attr = true;
    }
    const int R = a.n * (a.n_heads / a.n_kv_heads), tiles = (R + L::ROWS - 1) / L::ROWS;
    const int64_t items = (int64_t)tiles * a.batch * a.n_kv_heads;
    // enough CTAs for two per SM, none with fewer than 128 keys
    const int slots = 2 * sm_count();
    int64_t splits = items >= slots ? 1 : (slots + items - 1) / items;
    if (splits > (a.ctx_len + 127) / 128) splits = (a.ctx_len + 127) / 128;
    if (splits < 1) splits = 1;
    a.split_keys = (int)(((a.ctx_len + splits - 1) / splits + RSTEP * RW - 1) / (RSTEP * RW)) * RSTEP * RW;
    a.splits = a.split_keys ? (a.ctx_len + a.split_keys - 1) / a.split_keys : 1;
    const dim3 grid(a.splits, tiles, a.batch * a.n_kv_heads);
    return launch_pdl(kv8_attn_rows_kernel<D, NT, FMT>, grid, dim3(RW * 32), L::SMEM, stream, a) == cudaSuccess ? 1 : -1;
}
template <int D, int FMT>
int rows_tiles(const Kv8AttnArgs& a, cudaStream_t stream) {
    const int R = a.n * (a.n_heads / a.n_kv_heads);
    return R <= 8 ? rows_launch<D, 1, FMT>(a, stream) : rows_launch<D, 2, FMT>(a, stream);
}

}  // namespace

size_t kv8_attention_scratch_bytes(int head_dim) {
    // keys are split only below two items per SM: fewer than four results per SM of up to 16 rows
    return (size_t)4 * 148 * 16 * (head_dim + 1) * sizeof(float);
}

int launch_kv8_attention(const Kv8AttnArgs& a, cudaStream_t stream) {
    if (a.batch == 0 || a.n == 0) return 0;
    if (a.head_dim == 128) return a.format == kKv8Int8 ? rows_tiles<128, kKv8Int8>(a, stream) : rows_tiles<128, kKv8E4m3>(a, stream);
    return a.format == kKv8Int8 ? rows_tiles<64, kKv8Int8>(a, stream) : rows_tiles<64, kKv8E4m3>(a, stream);
}

}  // namespace acache
