// Parts of the tensor-memory kernel of the 8-bit attention (kv8_attn_tc.cu): PTX wrappers, the table of a key tile's scales, the
// conversion of a tile of codes.
#pragma once
#include "kernels.h"
#include "kv8.cuh"
#include "tc_ptx.cuh"

namespace acache {

constexpr int TT_TILE = 128 * 128 * 2;                    // 32 KB: 128 rows of f16 as two 64-column panels
constexpr int TT_PANEL = 128 * 64 * 2;

struct KeyTable {                                         // of one 128-key tile
    float4 group[8];                                      // per 16 keys: scale of K, log2 of V's scale, weight in l, -
    uint32_t keep[4];                                     // keys that count
    float grow, along;                                    // in front of this tile: what l is multiplied by, what M goes up by
    int e0;
    uint32_t pad;
};
constexpr int kTables = 4;

__device__ __forceinline__ uint4 ld_codes(const uint8_t* p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ void st_shared16(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void l2_prefetch(const void* p, int bytes) {
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p), "r"(bytes) : "memory");
}
// D += A B with A read from tensor memory
__device__ __forceinline__ void tt_mma_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(acc)
        : "memory");
}
// MN-major operand: rows of the K index are 128 bytes (64 elements of the MN index), the next 64 elements one panel further
__device__ __forceinline__ uint64_t tt_desc_mn(uint32_t saddr) {
    uint64_t d = (uint64_t)((saddr & 0x3FFFFu) >> 4);
    d |= (uint64_t)(TT_PANEL >> 4) << 16;
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}
__device__ __forceinline__ void tt_ld32(uint32_t taddr, float* v) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]),
          "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]),
          "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]),
          "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
        : "r"(taddr)
        : "memory");
}
// The loads above are complete after this; the values pass through it so that no use can move ahead of it.
template <int N>
__device__ __forceinline__ void tt_wait_ld(float* v) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]),
                   "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15])
                 :
                 : "memory");
    if constexpr (N > 16)
        asm volatile("" : "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]), "+f"(v[23]), "+f"(v[24]),
                          "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31]));
    if constexpr (N > 32) tt_wait_ld<N - 32>(v + 32);
}
__device__ __forceinline__ void tt_st32(uint32_t taddr, const uint32_t* v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
        ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]),
          "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]),
          "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]),
          "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31])
        : "memory");
}
__device__ __forceinline__ void tt_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// no sleep between polls: the softmax threads' waits are on the chain of every key tile
__device__ __forceinline__ bool tt_spin(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
    for (uint32_t i = 0; i < (TC_WAIT_LIMIT << 4); ++i) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((i & 4095u) == 4095u && *abort_flag) return false;
    }
    *abort_flag = 1;
    return false;
}

// For the converters, which are a stage ahead: a warp that polls takes issue slots from the softmax warps of its scheduler.
__device__ __forceinline__ bool tt_doze(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
    for (uint32_t i = 0; i < (TC_WAIT_LIMIT >> 1); ++i) {
        if (mbar_try_wait(bar, parity)) return true;
        __nanosleep(100);
        if (*abort_flag) return false;
    }
    *abort_flag = 1;
    return false;
}

// Lane l's share of what a warp needs to know of the 128-key tile at key0: lanes 0-7 the exponents of its 16-key groups of K,
// 8-15 V's, 16-19 the words of keys that count.
struct TileMeta {
    const uint8_t *k_exp, *v_exp;        // of the (request, KV head)
    const uint32_t* drop;                // of the request, or null
    int log2_block, key_hi;
    __device__ __forceinline__ uint32_t load(int key0, int lane) const {
        uint32_t v = 0u;
        if (lane < 16) {
            const int key = key0 + (lane & 7) * 16;
            if (key < key_hi) v = (lane < 8 ? k_exp : v_exp)[key >> log2_block];
        } else if (lane < 20) {
            const int k0 = key0 + (lane - 16) * 32, valid = key_hi - k0;
            v = valid >= 32 ? ~0u : (valid <= 0 ? 0u : (1u << valid) - 1u);
            if (drop && valid > 0) v &= ~__ldg(drop + (k0 >> 5));
        }
        return v;
    }
};
// A whole warp writes the table of a tile from its lanes' metas; e0: the largest ev so far of values that count (biased, 0: none), carried
// along.  Groups that hold nothing, or without a key that counts, have no scale; as long as there is nothing else it is taken to be 127,
// and M goes to the first real one with it.
__device__ __forceinline__ void write_table(KeyTable& t, uint32_t meta, int lane, int& e0) {
    const uint32_t keys = __shfl_sync(0xffffffffu, meta, 16 + ((lane & 7) >> 1)) >> ((lane & 1) * 16);
    const int held = __shfl_sync(0xffffffffu, (int)meta, 8 + (lane & 7)), ev = keys & 0xFFFFu ? held : 0;
    int top = ev;
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    top = max(top, e0);
    const int e_top = top ? top : 127;
    if (lane < 8) {
        const int e = ev ? ev : e_top;
        t.group[lane] = make_float4(kv8_scale((int)meta), (float)(max(e, e_top - kFarApart) - 127), kv8_weight(e_top - e), 0.f);
    }
    if (lane == 0) {
        t.grow = e0 ? kv8_scale(127 + min(top - e0, kFarApart)) : 1.f;
        t.along = e0 ? 0.f : (float)(e_top - 127);
        t.e0 = e_top;
    }
    if (lane >= 16 && lane < 20) t.keep[lane - 16] = meta;
    e0 = top;
    __syncwarp();
}
// 16-byte pieces of a [128 keys][128 codes] tile, piece i of a thread: row i CT / 8 + tid / 8, codes 16 (tid % 8) ..
template <int CT>
struct TilePieces {
    static constexpr int CH = (1024 + CT - 1) / CT;
    static __device__ __forceinline__ bool in_tile(int row) { return 1024 % CT == 0 || row < 128; }
    uint4 x[CH];
    __device__ __forceinline__ void load(const uint8_t* from, int key0, int key_hi, int tid) {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int row = i * (CT / 8) + (tid >> 3), key = key0 + row;
            x[i] = key < key_hi && in_tile(row) ? ld_codes(from + (int64_t)key * 128 + (tid & 7) * 16) : make_uint4(0u, 0u, 0u, 0u);
        }
    }
    // as f16 into a 128-byte-swizzled tile; rows whose bit is not set become zeros
    template <int FMT>
    __device__ __forceinline__ void convert(uint32_t dst, const uint32_t (&rows)[4], bool all, int tid) const {
        const int c8 = tid & 7, o = c8 >> 2;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int row = i * (CT / 8) + (tid >> 3);
            if (!in_tile(row)) break;
            uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w}, f[8];
            if (!all) {
                const uint32_t lo = row & 32 ? rows[1] : rows[0], hi = row & 32 ? rows[3] : rows[2];
                const bool on = ((row & 64 ? hi : lo) >> (row & 31)) & 1u;
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = on ? w[k] : 0u;
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) kv8_to_f16<FMT>(w[k], f[2 * k], f[2 * k + 1]);
            // two 16-byte units; the upper panel's threads store theirs the other way round (other banks)
            const uint32_t at = dst + o * TT_PANEL + row * 128, u = (c8 & 3) * 2, x7 = row & 7;
            const uint32_t a0 = at + (((u + o) ^ x7) << 4), a1 = at + (((u + 1 - o) ^ x7) << 4);
            if (o == 0) {
                st_shared16(a0, f[0], f[1], f[2], f[3]);
                st_shared16(a1, f[4], f[5], f[6], f[7]);
            } else {
                st_shared16(a0, f[4], f[5], f[6], f[7]);
                st_shared16(a1, f[0], f[1], f[2], f[3]);
            }
        }
    }
};
// the rows of a tile whose block holds something, from the ballot of its eight groups that do not
__device__ __forceinline__ void rows_held(uint32_t empty8, uint32_t (&rows)[4]) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const uint32_t e = (empty8 >> (2 * w)) & 3u;
        rows[w] = ~((e & 1u ? 0xFFFFu : 0u) | (e & 2u ? 0xFFFF0000u : 0u));
    }
}

}  // namespace acache
