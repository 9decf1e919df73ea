// Appending rows to a cache in pages, the rotary embedding applied on the way.
//
//   k'_i = k_i cos_i - k_{i + d/2} sin_i,   k'_{i + d/2} = k_{i + d/2} cos_i + k_i sin_i   (i < d / 2; the table's row: the token's position)
//
// in fp32, rounded once; queries likewise, values as they are.  A CTA takes a row: a thread the same eight pairs of every
// sixteenth (of 64 values, thirty-second) head, so that its angles are read once.  What is read depends on nothing but the row's
// number and is asked for before the position and the page are known.
//
// A row of a list looks for its position in the rest of the list, all threads together: nothing among hundreds of rows, and the square of their number beyond.
// Rows of 32 KV heads of one request, by list and behind a length: 4096 rows 31 and 29 us, 16 384 104 and 88, 65 536 748 and 326, 131 072 2554 and 641.
#include "common.cuh"
#include "kernels.h"
#include "launch.h"

namespace acache {
namespace {

// Threads of a CTA, heads that a thread asks for at once and CTAs of an SM: what is in flight is what counts, until writes of too many rows at a time
// get in each other's way.  us for 16 x 922 rows by list and for 16 x 2560 rows with 32 heads of queries (floors 74 and 308): 256 threads, 4, no
// bound 143 and 372; 256, 3, 4 103 and 309; 128, 2, 8 91 and 323; 128, 3, 8 87 and 316; 128, 6, 5 100 and 309; 64, 3, 14 90 and 331.
constexpr int kAppendThreads = 128, kAppendAhead = 3, kAppendCtas = 8;

struct Pair { uint4 lo, hi; };           // elements c .. c + 7 and d / 2 + c .. of a head

__device__ __forceinline__ uint32_t turn_lo(uint32_t a, uint32_t b, float2 c, float2 s) {
    return pack_bf16(bf16_lo(a) * c.x - bf16_lo(b) * s.x, bf16_hi(a) * c.y - bf16_hi(b) * s.y);
}
__device__ __forceinline__ uint32_t turn_hi(uint32_t a, uint32_t b, float2 c, float2 s) {
    return pack_bf16(bf16_lo(b) * c.x + bf16_lo(a) * s.x, bf16_hi(b) * c.y + bf16_hi(a) * s.y);
}

template <int D>
__global__ void __launch_bounds__(kAppendThreads, kAppendCtas) paged_append_kernel(const PagedAppendArgs a) {
    constexpr int SLOTS = D / 16;        // threads of a head
    constexpr int HEADS = kAppendThreads / SLOTS;
    constexpr int AHEAD = kAppendAhead;
    const int b = blockIdx.y, i = blockIdx.x, tid = threadIdx.x, c = tid % SLOTS * 8, head0 = tid / SLOTS;
    pdl_wait();
    pdl_launch_dependents();
    int count = a.n;
    if (a.counts) {
        count = a.counts[b];
        if (count < 0 || count > a.n) {
            if (i == 0 && tid == 0) atomicOr(a.status, kFlagBadIndex);
            count = min(count, a.n);
        }
    }
    if (i >= count) return;
    const int hkv = a.n_kv_heads, n_q = a.q_rows.p ? a.n_heads : 0, heads = n_q + 2 * hkv;
    auto from = [&](int h) {
        const Rows& r = h < n_q ? a.q_rows : h < n_q + hkv ? a.k_rows : a.v_rows;
        const int at = h < n_q ? h : h < n_q + hkv ? h - n_q : h - n_q - hkv;
        return static_cast<const __nv_bfloat16*>(r.p) + b * r.batch_stride + i * r.row_stride + (int64_t)at * D + c;
    };
    Pair x[AHEAD];
    auto load = [&](int h0) {
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int h = h0 + j * HEADS;
            if (h < heads) {
                const __nv_bfloat16* p = from(h);
                x[j].lo = __ldcs(reinterpret_cast<const uint4*>(p));
                x[j].hi = __ldcs(reinterpret_cast<const uint4*>(p + D / 2));
            }
        }
    };
    load(head0);
    const int64_t pos = a.pos ? a.pos[(int64_t)b * a.n + i] : (int64_t)a.lens[b] + i;
    bool skip = pos < 0 || pos >= a.ctx_len;
    int page = 0;
    if (!skip) {
        page = a.pages.table[(int64_t)b * a.pages.table_stride + (pos >> a.pages.log2_page)];
        skip = page < 0 || page >= a.pages.n_pages;
    }
    if (skip) {
        if (tid == 0) atomicOr(a.status, kFlagBadIndex);
        return;
    }
    if (a.pos) {
        // of rows of one position the last is written
        bool again = false;
        for (int j = i + 1 + tid; j < count; j += kAppendThreads) again |= a.pos[(int64_t)b * a.n + j] == pos;
        if (__syncthreads_or(again)) skip = true;
    }
    float2 cs[4] = {}, sn[4] = {};
    if (a.rope_cos) {
        const float4* pc = reinterpret_cast<const float4*>(a.rope_cos + pos * (D / 2) + c);
        const float4* ps = reinterpret_cast<const float4*>(a.rope_sin + pos * (D / 2) + c);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float4 u = __ldg(pc + j), w = __ldg(ps + j);
            cs[2 * j] = make_float2(u.x, u.y); cs[2 * j + 1] = make_float2(u.z, u.w);
            sn[2 * j] = make_float2(w.x, w.y); sn[2 * j + 1] = make_float2(w.z, w.w);
        }
    }
    const int64_t slot = page * a.pages.page_stride + (int64_t)((int)pos & ((1 << a.pages.log2_page) - 1)) * D + c;
    for (int h0 = head0; h0 < heads; h0 += AHEAD * HEADS) {
        if (h0 != head0) load(h0);
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int h = h0 + j * HEADS;
            if (h >= heads) break;
            Pair y = x[j];
            if (h < n_q + hkv && a.rope_cos) {
                const Pair& o = x[j];
                y.lo = make_uint4(turn_lo(o.lo.x, o.hi.x, cs[0], sn[0]), turn_lo(o.lo.y, o.hi.y, cs[1], sn[1]),
                                  turn_lo(o.lo.z, o.hi.z, cs[2], sn[2]), turn_lo(o.lo.w, o.hi.w, cs[3], sn[3]));
                y.hi = make_uint4(turn_hi(o.lo.x, o.hi.x, cs[0], sn[0]), turn_hi(o.lo.y, o.hi.y, cs[1], sn[1]),
                                  turn_hi(o.lo.z, o.hi.z, cs[2], sn[2]), turn_hi(o.lo.w, o.hi.w, cs[3], sn[3]));
            }
            __nv_bfloat16* to;
            if (h < n_q) {
                to = static_cast<__nv_bfloat16*>(a.q_out) + (((int64_t)b * a.n + i) * a.n_heads + h) * D + c;
            } else {
                if (skip) continue;
                const bool val = h >= n_q + hkv;
                to = static_cast<__nv_bfloat16*>(val ? a.v : a.k) + slot + ((int64_t)(h - n_q - (val ? hkv : 0)) << a.pages.log2_page) * D;
            }
            *reinterpret_cast<uint4*>(to) = y.lo;
            *reinterpret_cast<uint4*>(to + D / 2) = y.hi;
        }
    }
}

}  // namespace

int launch_paged_append(const PagedAppendArgs& a, cudaStream_t stream) {
    if (a.batch == 0 || a.n == 0) return 0;
    const dim3 grid(a.n, a.batch);
    const cudaError_t e = a.head_dim == 128 ? launch_pdl(paged_append_kernel<128>, grid, dim3(kAppendThreads), 0, stream, a)
                                            : launch_pdl(paged_append_kernel<64>, grid, dim3(kAppendThreads), 0, stream, a);
    return e == cudaSuccess ? 1 : -1;
}

}  // namespace acache
