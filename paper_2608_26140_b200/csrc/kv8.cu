// The 8-bit cache: rows written into it (quantised), and read back.  Both are bound by HBM: 2 bytes read and 1 written a
// value, or the other way round; every value passes through registers once.
#include "kernels.h"
#include "kv8.cuh"
#include "launch.h"

namespace acache {

// ---- writing ----------------------------------------------------------------------------
// A unit is one (block of tokens, head, K or V).  Its threads hold all of it in registers, 8 pieces of 8 values each, so the
// block's largest value is known before anything is rounded and the rows are read once:
//   e_rows = exponent field of max |x| - top,   e = max(e_rows, e_old) if a row of the block stays, else e_rows,
//   code = round(x 2^(127 - e)),   rows that stay: round(code 2^(e_old - e)) where the exponent grew, untouched where not.
// Only the exponent of the largest value is needed, so the maximum is taken over the exponent fields, two to a word.
// A CTA takes the units of several heads of one block.  With positions given one by one it looks for the rows of its block
// in the list (the last of two that name a position wins): n loads per CTA from L2, no map and no second launch.
constexpr int kWriteThreads = 256;

template <int D, int BLOCK, int FMT, bool LIST>
__global__ void __launch_bounds__(kWriteThreads) kv8_write_kernel(const Kv8WriteArgs a) {
    constexpr int UT = BLOCK * D / 64;                  // threads of a unit
    constexpr int UNITS = kWriteThreads / UT;
    constexpr int CPR = D / 8;                          // pieces per row
    __shared__ int row_of[BLOCK];
    __shared__ uint32_t warp_max[kWriteThreads / 32];
    pdl_wait();
    pdl_launch_dependents();
    const int tid = threadIdx.x, b = blockIdx.z;
    const int32_t* list = LIST ? a.pos + (int64_t)b * a.n : nullptr;
    int blk = a.first_block + blockIdx.x;
    if (LIST && a.by_row) {
        // few rows, many blocks: the CTA of row i takes the block of its position, if no earlier row has it
        const int p = list[blockIdx.x];
        if (p < 0 || p >= a.ctx_len) {
            if (tid == 0 && blockIdx.y == 0) atomicOr(a.status, kFlagBadIndex);
            return;
        }
        blk = p / BLOCK;
        bool earlier = false;
        for (int i = tid; i < (int)blockIdx.x; i += kWriteThreads) {
            const int q = list[i];
            earlier |= q >= 0 && q < a.ctx_len && q / BLOCK == blk;
        }
        if (__syncthreads_or(earlier)) return;
    }
    const int t0 = blk * BLOCK;
    const int here = min(a.ctx_len - t0, BLOCK);        // the block's positions inside the context
    int n_written;
    if (LIST) {
        if (tid < BLOCK) row_of[tid] = -1;
        __syncthreads();
        bool bad = false;
        for (int i = tid; i < a.n; i += kWriteThreads) {
            const int p = list[i];
            if (p >= t0 && p < t0 + here) atomicMax(&row_of[p - t0], i);
            bad |= p < 0 || p >= a.ctx_len;
        }
        if (bad && !a.by_row && blockIdx.x == 0 && blockIdx.y == 0) atomicOr(a.status, kFlagBadIndex);
        __syncthreads();
        n_written = __syncthreads_count(tid < BLOCK && row_of[tid] >= 0);
        if (n_written == 0) return;
    } else {
        n_written = min(t0 + here, a.start + a.n) - max(t0, a.start);
    }
    auto source = [&](int r) {                          // the row that serves position t0 + r, or -1
        if (LIST) return row_of[r];
        const int i = t0 + r - a.start;
        return i >= 0 && i < a.n ? i : -1;
    };

    const int unit = blockIdx.y * UNITS + tid / UT, ut = tid % UT;
    const bool active = unit < 2 * a.n_kv_heads;
    const int h = active ? (unit < a.n_kv_heads ? unit : unit - a.n_kv_heads) : 0;
    const bool is_v = unit >= a.n_kv_heads;
    const __nv_bfloat16* rows = static_cast<const __nv_bfloat16*>(is_v ? a.v_rows : a.k_rows) + (int64_t)b * a.rows_batch_stride + h * D;
    uint4 x[8];
    uint32_t top2 = 0u;
    if (active) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = i * UT + ut, src = source(c / CPR);
            x[i] = make_uint4(0u, 0u, 0u, 0u);
            if (src >= 0) x[i] = __ldg(reinterpret_cast<const uint4*>(rows + (int64_t)src * a.n_kv_heads * D) + c % CPR);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            top2 = __vmaxu2(__vmaxu2(top2, x[i].x & 0x7F807F80u), __vmaxu2(__vmaxu2(x[i].y & 0x7F807F80u, x[i].z & 0x7F807F80u), x[i].w & 0x7F807F80u));
    }
    // over the unit's threads
    auto unit_max = [&](uint32_t m) {
#pragma unroll
        for (int o = (UT < 32 ? UT : 32) / 2; o > 0; o >>= 1) m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, o));
        if (UT > 32) {
            __syncthreads();
            if ((tid & 31) == 0) warp_max[tid >> 5] = m;
            __syncthreads();
            const int w0 = (tid / UT) * (UT / 32);
#pragma unroll
            for (int w = 0; w < UT / 32; ++w) m = __vmaxu2(m, warp_max[w0 + w]);
        }
        return (int)(max(m & 0xFFFFu, m >> 16) >> 7);
    };
    int field = unit_max(top2);
    bool careful = false;
    const bool odd = field == 255;                      // the unit has a value that is not finite
    if (__syncthreads_or(field == 255)) {               // something is not finite: the largest of the finite values counts
        careful = true;
        if (odd && ut == 0) atomicOr(a.status, kFlagNonFinite);
        top2 = 0u;
        if (active) {
            auto finite = [](uint32_t w) {
                const uint32_t lo = w & 0x7F80u, hi = w & 0x7F800000u;
                return (lo == 0x7F80u ? 0u : lo) | (hi == 0x7F800000u ? 0u : hi);
            };
#pragma unroll
            for (int i = 0; i < 8; ++i)
                top2 = __vmaxu2(__vmaxu2(top2, finite(x[i].x)), __vmaxu2(__vmaxu2(finite(x[i].y), finite(x[i].z)), finite(x[i].w)));
        }
        field = unit_max(top2);
    }
    if (!active) return;

    uint8_t* exps = (is_v ? a.v_exp : a.k_exp) + ((int64_t)(a.shared ? 0 : b) * a.n_kv_heads + h) * a.n_blocks + blk;
    uint8_t* codes = (is_v ? a.v : a.k) + (int64_t)b * a.batch_stride + ((int64_t)h * a.capacity + t0) * D;
    const int e_old = n_written < here ? *exps : 0;     // only counts where a row stays
    // (rows of zeros alone leave the block empty)
    const int e_rows = field == 0 && !odd ? 0 : min(max(field - kv8_top<FMT>(), kKv8MinExp), 254);
    const int e = max(e_rows, e_old);
    const float inv = __int_as_float((254 - e) << 23);
    if (field == 254 && FMT == kKv8E4m3) careful = true;
    const float limit = e == 254 - kv8_top<kKv8E4m3>() ? 240.f : 448.f;
    const float shrink = kv8_scale(127 + e_old - e);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int c = i * UT + ut, r = c / CPR;
        uint2* out = reinterpret_cast<uint2*>(codes + (int64_t)r * D) + c % CPR;
        if (source(r) >= 0 && e > 0) {
            const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
            float f[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                f[2 * j] = bf16_lo(w[j]) * inv;
                f[2 * j + 1] = bf16_hi(w[j]) * inv;
            }
            if (careful)
                *out = make_uint2(kv8_round_careful<FMT>(f[0], f[1], f[2], f[3], limit), kv8_round_careful<FMT>(f[4], f[5], f[6], f[7], limit));
            else
                *out = make_uint2(kv8_round<FMT>(f[0], f[1], f[2], f[3]), kv8_round<FMT>(f[4], f[5], f[6], f[7]));
        } else if (r >= here || e_old == 0) {           // past the context, or nothing there (e_old = 0 where e is)
            *out = make_uint2(0u, 0u);
        } else if (e != e_old) {                        // a row that stays, on the coarser scale
            const uint2 old = *out;
            uint32_t l0, h0, l1, h1;
            kv8_to_f16<FMT>(old.x, l0, h0);
            kv8_to_f16<FMT>(old.y, l1, h1);
            const float2 p0 = f16x2_to_f32(l0), p1 = f16x2_to_f32(h0), p2 = f16x2_to_f32(l1), p3 = f16x2_to_f32(h1);
            *out = make_uint2(kv8_round<FMT>(p0.x * shrink, p0.y * shrink, p1.x * shrink, p1.y * shrink),
                              kv8_round<FMT>(p2.x * shrink, p2.y * shrink, p3.x * shrink, p3.y * shrink));
        }
    }
    if (ut == 0) *exps = (uint8_t)e;
}

namespace {
template <int D, int BLOCK, int FMT>
void write_launch(const Kv8WriteArgs& a, unsigned blocks, cudaStream_t stream) {
    constexpr int UNITS = kWriteThreads / (BLOCK * D / 64);
    const dim3 grid(blocks, (2 * a.n_kv_heads + UNITS - 1) / UNITS, a.batch);
    if (a.pos) launch_pdl(kv8_write_kernel<D, BLOCK, FMT, true>, grid, kWriteThreads, 0, stream, a);
    else launch_pdl(kv8_write_kernel<D, BLOCK, FMT, false>, grid, kWriteThreads, 0, stream, a);
}
template <int D, int FMT>
void write_blocks(const Kv8WriteArgs& a, unsigned blocks, cudaStream_t stream) {
    switch (a.block) {
        case 16: return write_launch<D, 16, FMT>(a, blocks, stream);
        case 32: return write_launch<D, 32, FMT>(a, blocks, stream);
        case 64: return write_launch<D, 64, FMT>(a, blocks, stream);
        default: return write_launch<D, 128, FMT>(a, blocks, stream);
    }
}
}  // namespace

void launch_kv8_write(Kv8WriteArgs a, cudaStream_t stream) {
    unsigned blocks;
    if (a.pos) {
        const int all = (a.ctx_len + a.block - 1) / a.block;
        a.first_block = 0;
        a.by_row = a.n < all;
        blocks = a.by_row ? a.n : all;
    } else {
        a.first_block = a.start / a.block;
        blocks = (a.start + a.n - 1) / a.block - a.first_block + 1;
    }
    if (a.head_dim == 128) {
        if (a.format == kKv8Int8) write_blocks<128, kKv8Int8>(a, blocks, stream);
        else write_blocks<128, kKv8E4m3>(a, blocks, stream);
    } else {
        if (a.format == kKv8Int8) write_blocks<64, kKv8Int8>(a, blocks, stream);
        else write_blocks<64, kKv8E4m3>(a, blocks, stream);
    }
}

// ---- reading ----------------------------------------------------------------------------
// A thread turns pieces of 16 codes into 16 bf16 values (exact).  A warp takes 4 rows (8 at head dimension 64) of up to 4
// heads, K and V: eight loads in flight per thread; the codes of neighbouring rows of a head lie side by side.
template <int D, int FMT>
__global__ void __launch_bounds__(128) kv8_read_kernel(const Kv8ReadArgs a) {
    constexpr int LANES = D / 16, ROWS = 32 / LANES;    // lanes per row, rows per warp
    constexpr int HEADS = 4;
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31, b = blockIdx.z, h0 = blockIdx.y * HEADS;
    const int i = (blockIdx.x * 4 + (threadIdx.x >> 5)) * ROWS + lane / LANES, piece = lane % LANES;
    if (i >= a.n) return;
    const int p = a.pos ? __ldg(a.pos + (int64_t)b * a.n + i) : a.start + i;
    const bool ok = p >= 0 && p < a.ctx_len;
    if (!ok && h0 == 0 && piece == 0) atomicOr(a.status, kFlagBadIndex);
    uint4 w[2][HEADS];
    int e[2][HEADS];
#pragma unroll
    for (int u = 0; u < HEADS; ++u) {
        const int h = h0 + u;
        const bool there = ok && h < a.n_kv_heads;
        const int64_t at = (int64_t)b * a.batch_stride + ((int64_t)h * a.capacity + p) * D + piece * 16;
        const int64_t xat = ((int64_t)(a.shared ? 0 : b) * a.n_kv_heads + h) * a.n_blocks + (p >> a.log2_block);
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
            const bool on = there && (kv ? a.v_out : a.k_out) != nullptr;
            w[kv][u] = on ? __ldg(reinterpret_cast<const uint4*>((kv ? a.v : a.k) + at)) : make_uint4(0u, 0u, 0u, 0u);
            e[kv][u] = on ? __ldg((kv ? a.v_exp : a.k_exp) + xat) : 0;
        }
    }
#pragma unroll
    for (int u = 0; u < HEADS; ++u) {
        const int h = h0 + u;
        if (h >= a.n_kv_heads) break;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
            void* base = kv ? a.v_out : a.k_out;
            if (!base) continue;
            const float s = kv8_scale(e[kv][u]);
            const uint32_t in[4] = {w[kv][u].x, w[kv][u].y, w[kv][u].z, w[kv][u].w};
            uint32_t out[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t lo, hi;
                kv8_to_f16<FMT>(e[kv][u] ? in[j] : 0u, lo, hi);
                const float2 f0 = f16x2_to_f32(lo), f1 = f16x2_to_f32(hi);
                out[2 * j] = pack_bf16(f0.x * s, f0.y * s);
                out[2 * j + 1] = pack_bf16(f1.x * s, f1.y * s);
            }
            uint4* to = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(base) + (int64_t)b * a.out_batch_stride + ((int64_t)i * a.n_kv_heads + h) * D) + piece * 2;
            to[0] = make_uint4(out[0], out[1], out[2], out[3]);
            to[1] = make_uint4(out[4], out[5], out[6], out[7]);
        }
    }
}

void launch_kv8_read(const Kv8ReadArgs& a, cudaStream_t stream) {
    const int rows = 4 * (32 / (a.head_dim / 16));
    const dim3 grid((a.n + rows - 1) / rows, (a.n_kv_heads + 3) / 4, a.batch);
    if (a.head_dim == 128) {
        if (a.format == kKv8Int8) launch_pdl(kv8_read_kernel<128, kKv8Int8>, grid, 128, 0, stream, a);
        else launch_pdl(kv8_read_kernel<128, kKv8E4m3>, grid, 128, 0, stream, a);
    } else {
        if (a.format == kKv8Int8) launch_pdl(kv8_read_kernel<64, kKv8Int8>, grid, 128, 0, stream, a);
        else launch_pdl(kv8_read_kernel<64, kKv8E4m3>, grid, 128, 0, stream, a);
    }
}

}  // namespace acache
