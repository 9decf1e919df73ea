// The 8-bit cache: rows written into it (quantised), and read back.  Both are bound by HBM: 2 bytes read and 1 written a
// value, or the other way round; every value passes through registers once.
#include <type_traits>

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
// A CTA takes the units of one or several heads of a block.  With positions given one by one it looks for the rows of its block
// in the list (the last of two that name a position wins): n loads per CTA from L2, no map and no second launch; the rows found
// are packed, so that passes over the registers that a block's few rows leave empty are skipped.
// 16 requests of 2560 tokens, 32 heads of 128: all rows (1007 MB) 148 us, 6.8 TB/s; 922 rows each at positions of a list, int8
// (364 MB) 88 us: there 70 % of the issue slots are taken (search, packing, short loops), not DRAM.
constexpr int kWriteThreads = 256;

template <int D, int BLOCK, int FMT, bool LIST>
__global__ void __launch_bounds__(kWriteThreads, 4) kv8_write_kernel(const Kv8WriteArgs a) {
    constexpr int UT = BLOCK * D / 64;                  // threads of a unit
    constexpr int UNITS = kWriteThreads / UT;
    constexpr int CPR = D / 8;                          // pieces per row
    constexpr int RPP = UT / CPR;                       // rows of a pass: a thread's pieces are RPP rows apart
    __shared__ int row_of[LIST ? BLOCK : 1];            // row that serves a position, or -1
    __shared__ int2 write[LIST ? BLOCK : 1];            // of the k-th row to write: the row, its position
    __shared__ __align__(8) int warp_max[2][2][kWriteThreads / 32];
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
    int n_written, first = 0, from = 0;                 // rows to write; without a list: the first one's place, and its row
    if (LIST) {
        if (tid < BLOCK) row_of[tid] = -1;
        __syncthreads();
        bool bad = false;
        for (int i0 = tid; i0 < a.n; i0 += 4 * kWriteThreads) {      // four loads in flight
            int p[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) p[j] = i0 + j * kWriteThreads < a.n ? __ldg(list + i0 + j * kWriteThreads) : 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int i = i0 + j * kWriteThreads;
                if (i < a.n && (unsigned)(p[j] - t0) < (unsigned)here) atomicMax(&row_of[p[j] - t0], i);
                bad |= (unsigned)p[j] >= (unsigned)a.ctx_len;
            }
        }
        if (bad && !a.by_row && blockIdx.x == 0 && blockIdx.y == 0) atomicOr(a.status, kFlagBadIndex);
        __syncthreads();
        const int src = tid < BLOCK ? row_of[tid] : -1;
        const uint32_t in_warp = __ballot_sync(0xffffffffu, src >= 0);
        if (tid < BLOCK && (tid & 31) == 0) warp_max[0][0][tid >> 5] = __popc(in_warp);
        __syncthreads();
        int before = __popc(in_warp & ((1u << (tid & 31)) - 1u));
        n_written = 0;
#pragma unroll
        for (int w = 0; w < (BLOCK + 31) / 32; ++w) {
            if (w < tid >> 5) before += warp_max[0][0][w];
            n_written += warp_max[0][0][w];
        }
        if (n_written == 0) return;
        if (src >= 0) write[before] = make_int2(src, tid);
        __syncthreads();
    } else {
        first = max(a.start - t0, 0);
        from = t0 + first - a.start;
        n_written = min(t0 + here, a.start + a.n) - (t0 + first);
    }
    const int u = tid / UT, ut = tid % UT, k0 = ut / CPR;           // this thread's pieces: of rows k0, k0 + RPP, ..
    const int64_t row_elems = (int64_t)a.n_kv_heads * D, piece = ut % CPR * 8;
    auto write_at = [&](int k) { return LIST ? write[k] : make_int2(from + k, first + k); };
    auto largest = [](const uint4& x, auto of) { return __vmaxu2(__vmaxu2(of(x.x), of(x.y)), __vmaxu2(of(x.z), of(x.w))); };
    auto magnitude = [](uint32_t w) { return w & 0x7F807F80u; };
    auto finite = [](uint32_t w) {
        const uint32_t lo = w & 0x7F80u, hi = w & 0x7F800000u;
        return (lo == 0x7F80u ? 0u : lo) | (hi == 0x7F800000u ? 0u : hi);
    };
    // The largest over the unit's threads, of exponent fields; returned: whether one is 255 among all the threads that come together
    // here.  turn: which of two places, so that one barrier does.
    int turn = 0;
    auto unit_max = [&](auto& m) {
        constexpr int N = sizeof(m) / sizeof(m[0]);
        int top = 0;
#pragma unroll
        for (int p = 0; p < N; ++p) {
            int f = (int)(max(m[p] & 0xFFFFu, m[p] >> 16) >> 7);
            if constexpr (UT < 32) {
#pragma unroll
                for (int o = UT / 2; o > 0; o >>= 1) f = max(f, __shfl_xor_sync(0xffffffffu, f, o));
            } else {
                f = __reduce_max_sync(0xffffffffu, f);
                if (UT > 32 && (tid & 31) == 0) warp_max[turn][p][tid >> 5] = f;
            }
            m[p] = f;
            top = max(top, f);
        }
        if constexpr (UT > 32) {
            const bool any = __syncthreads_or(top == 255);
#pragma unroll
            for (int p = 0; p < N; ++p)
#pragma unroll
                for (int w = 0; w < UT / 32; w += 2) {
                    const int2 f = *reinterpret_cast<const int2*>(&warp_max[turn][p][u * (UT / 32) + w]);
                    m[p] = max((int)m[p], max(f.x, f.y));
                }
            turn ^= 1;
            return any;
        } else {
            if constexpr (UT < 32) top = max(top, __shfl_xor_sync(0xffffffffu, top, UT));
            return top == 255;
        }
    };
    // The units of this CTA, N of them at a time: one, or K and V of a head.
    auto run = [&](auto n_units) {
        constexpr int N = decltype(n_units)::value, SLOTS = 8 / N;
        const int all = 2 * a.n_kv_heads / N;
        int v0 = blockIdx.y * UNITS;
        while (v0 < all) {
            const int v = v0 + u;
            const bool active = v < all;
            auto is_v = [&](int p) { return N == 2 ? p == 1 : v >= a.n_kv_heads; };
            const int h = !active ? 0 : N == 2 || v < a.n_kv_heads ? v : v - a.n_kv_heads;
            const int64_t exps_at = ((int64_t)b * a.n_kv_heads + h) * a.n_blocks + blk;
            const int64_t rows_at = (int64_t)b * a.rows_batch_stride + h * D + piece;
            const int64_t codes_at = (int64_t)b * a.batch_stride + ((int64_t)h * a.capacity + t0) * D + piece;
            uint4 x[N][SLOTS];
            int e_old[N];
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) {
                if (LIST && i * RPP >= n_written) break;
                // (threads past the last row take it again: it changes no maximum)
                const int64_t at = rows_at + write_at(min(i * RPP + k0, n_written - 1)).x * row_elems;
#pragma unroll
                for (int p = 0; p < N; ++p)
                    x[p][i] = __ldg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(is_v(p) ? a.v_rows : a.k_rows) + at));
            }
            uint32_t field[N];
#pragma unroll
            for (int p = 0; p < N; ++p) {
                e_old[p] = active && n_written < here ? (is_v(p) ? a.v_exp : a.k_exp)[exps_at] : 0;      // only counts where a row stays
                field[p] = 0u;
            }
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) {
                if (LIST && i * RPP >= n_written) break;
#pragma unroll
                for (int p = 0; p < N; ++p) field[p] = __vmaxu2(field[p], largest(x[p][i], magnitude));
            }
            const bool any_odd = unit_max(field);
            bool odd[N];                                 // a unit has a value that is not finite: the largest of the others counts
#pragma unroll
            for (int p = 0; p < N; ++p) odd[p] = field[p] == 255;
            if (any_odd) {
#pragma unroll
                for (int p = 0; p < N; ++p) {
                    if (odd[p] && ut == 0) atomicOr(a.status, kFlagNonFinite);
                    field[p] = 0u;
#pragma unroll
                    for (int i = 0; i < SLOTS; ++i) {
                        if (LIST && i * RPP >= n_written) break;
                        field[p] = __vmaxu2(field[p], largest(x[p][i], finite));
                    }
                }
                unit_max(field);
            }
#pragma unroll
            for (int p = 0; p < N; ++p) {
                if (!active) break;
                // (rows of zeros alone leave the block empty)
                const int e_rows = field[p] == 0 && !odd[p] ? 0 : min(max((int)field[p] - kv8_top<FMT>(), kKv8MinExp), 254);
                const int e = max(e_rows, e_old[p]);
                const float inv = __int_as_float((254 - e) << 23);
                uint8_t* codes = (is_v(p) ? a.v : a.k) + codes_at;
                if (odd[p] || e == 0 || (field[p] == 254 && FMT == kKv8E4m3)) {
                    const float limit = e == 0 ? 0.f : e == 254 - kv8_top<kKv8E4m3>() ? 240.f : 448.f;
#pragma unroll 1
                    for (int i = 0; i < SLOTS; ++i) {
                        const int k = i * RPP + k0;
                        if (k >= n_written) break;
                        // (again from memory: a loop that is not unrolled cannot index registers)
                        const uint4 y = __ldg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(is_v(p) ? a.v_rows : a.k_rows) + rows_at + write_at(k).x * row_elems));
                        const uint2 w = make_uint2(kv8_round_careful<FMT>(bf16_lo(y.x) * inv, bf16_hi(y.x) * inv, bf16_lo(y.y) * inv, bf16_hi(y.y) * inv, limit),
                                                   kv8_round_careful<FMT>(bf16_lo(y.z) * inv, bf16_hi(y.z) * inv, bf16_lo(y.w) * inv, bf16_hi(y.w) * inv, limit));
                        *reinterpret_cast<uint2*>(codes + write_at(k).y * D) = e > 0 ? w : make_uint2(0u, 0u);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < SLOTS; ++i) {
                        if (LIST && i * RPP >= n_written) break;
                        const int k = i * RPP + k0;
                        if (k < n_written)
                            *reinterpret_cast<uint2*>(codes + write_at(k).y * D) =
                                make_uint2(kv8_round_bf16<FMT>(x[p][i].x, x[p][i].y, inv), kv8_round_bf16<FMT>(x[p][i].z, x[p][i].w, inv));
                    }
                }
                // the block's other rows: untouched where the exponent is what it was, and they count
                if (n_written < BLOCK && (e != e_old[p] || e_old[p] == 0 || here < BLOCK)) {
                    const float shrink = kv8_scale(127 + e_old[p] - e);
#pragma unroll 1
                    for (int r = k0; r < BLOCK; r += RPP) {
                        if (LIST ? row_of[r] >= 0 : r >= first && r < first + n_written) continue;
                        uint2* out = reinterpret_cast<uint2*>(codes + r * D);
                        if (r >= here || e_old[p] == 0) {        // past the context, or nothing there
                            *out = make_uint2(0u, 0u);
                        } else if (e != e_old[p]) {              // a row that stays, on the coarser scale
                            const uint2 old = *out;
                            uint32_t l0, h0, l1, h1;
                            kv8_to_f16<FMT>(old.x, l0, h0);
                            kv8_to_f16<FMT>(old.y, l1, h1);
                            const float2 p0 = f16x2_to_f32(l0), p1 = f16x2_to_f32(h0), p2 = f16x2_to_f32(l1), p3 = f16x2_to_f32(h1);
                            *out = make_uint2(kv8_round<FMT>(p0.x * shrink, p0.y * shrink, p1.x * shrink, p1.y * shrink),
                                              kv8_round<FMT>(p2.x * shrink, p2.y * shrink, p3.x * shrink, p3.y * shrink));
                        }
                    }
                }
                if (ut == 0) (is_v(p) ? a.v_exp : a.k_exp)[exps_at] = (uint8_t)e;
            }
            if constexpr (!LIST) break;                  // a CTA of a span has one turn
            else v0 += gridDim.y * UNITS;
        }
    };
    // K and V of a head together where both fit a thread's registers: twice the loads in flight, half the barriers and searches
    // (the 922 rows above, when this was measured: 91 us; 157 us one by one)
    if (LIST && 2 * n_written <= BLOCK) run(std::integral_constant<int, 2>{});
    else run(std::integral_constant<int, 1>{});
}

namespace {
template <int D, int BLOCK, int FMT>
void write_launch(const Kv8WriteArgs& a, unsigned blocks, cudaStream_t stream) {
    constexpr int UNITS = kWriteThreads / (BLOCK * D / 64);
    // a CTA of a span has one turn; one of a list has one of K and V together or, in a full block, two of them apart
    const int turns = (2 * a.n_kv_heads + UNITS - 1) / UNITS;
    const int pairs = (a.n_kv_heads + UNITS - 1) / UNITS;
    if (a.pos) launch_pdl(kv8_write_kernel<D, BLOCK, FMT, true>, dim3(blocks, pairs, a.batch), kWriteThreads, 0, stream, a);
    else launch_pdl(kv8_write_kernel<D, BLOCK, FMT, false>, dim3(blocks, turns, a.batch), kWriteThreads, 0, stream, a);
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
        const int all = a.ctx_len > 0 ? (a.ctx_len + a.block - 1) / a.block : 1;      // (none: one CTA says that no row has a place)
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
// A thread turns pieces of 16 codes into 16 bf16 values (exact) and stores them in one instruction of 32 bytes, a whole sector.
// A warp takes 4 rows (8 at head dimension 64) of two heads, K and V: four loads in flight per thread.  5 requests, 1639 rows
// of 32 heads of 128 each (200 MB): 34.6 us, 5.8 TB/s; with 16-byte stores 39.8 us; with four heads a warp 35.5 us.
constexpr int kReadHeads = 2;

template <int D, int FMT>
__global__ void __launch_bounds__(128) kv8_read_kernel(const Kv8ReadArgs a) {
    constexpr int LANES = D / 16, ROWS = 32 / LANES;    // lanes per row, rows per warp
    constexpr int HEADS = kReadHeads;
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
            void* to = static_cast<__nv_bfloat16*>(base) + (int64_t)b * a.out_batch_stride + ((int64_t)i * a.n_kv_heads + h) * D + piece * 16;
            st_global32(to, out, on_sector(base));
        }
    }
}

void launch_kv8_read(const Kv8ReadArgs& a, cudaStream_t stream) {
    const int rows = 4 * (32 / (a.head_dim / 16));
    const dim3 grid((a.n + rows - 1) / rows, (a.n_kv_heads + kReadHeads - 1) / kReadHeads, a.batch);
    if (a.head_dim == 128) {
        if (a.format == kKv8Int8) launch_pdl(kv8_read_kernel<128, kKv8Int8>, grid, 128, 0, stream, a);
        else launch_pdl(kv8_read_kernel<128, kKv8E4m3>, grid, 128, 0, stream, a);
    } else {
        if (a.format == kKv8Int8) launch_pdl(kv8_read_kernel<64, kKv8Int8>, grid, 128, 0, stream, a);
        else launch_pdl(kv8_read_kernel<64, kKv8E4m3>, grid, 128, 0, stream, a);
    }
}

}  // namespace acache
