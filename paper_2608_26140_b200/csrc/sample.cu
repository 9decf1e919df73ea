// Sampling of a token from a row of logits.
//
//   w_i = exp((l_i - max l) / T); in the order of falling l (equal ones by their index) a prefix is kept: the first top_k, the fewest of those that
//   make up top_p of their weight, those with w_i >= min_p, whatever is least; the token is the first of them whose running sum
//   passes u times the sum S of all that are kept.
//
// Nothing is sorted.  A weight is a whole number of 2^-shift (46 bits behind the point for up to 2^16 tokens, one less for every doubling), so that sums are exact and do not
// depend on their order; what is below half of that is never drawn.  Each of the three searches (the k-th token, the one
// at which top_p is reached, the one that is drawn) goes over a histogram of counts and weights, whose bins part the logits evenly from the largest
// to the smallest that counts, then over the tokens of one bin: by comparing them all with one another, where
// they are few, else by another histogram of their keys.  Searches end at a value; among the tokens that have it the index decides.
// The row lies in the shared memory of a cluster of CTAs, read once; what a CTA finds out is read by the others from there.  Every CTA takes
// every decision by itself, so that a search costs one barrier of the cluster, and a histogram two.
#include <algorithm>

#include "kernels.h"
#include "launch.h"
#include "per_device.h"
#include "tc_ptx.cuh"

namespace acache {
namespace {

using u64 = unsigned long long;

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBins = 2048;
constexpr int kFew = 512;                // tokens of a bin that are compared with one another
constexpr int kMaxCluster = 8;

__device__ __forceinline__ uint32_t order_key(float f) {     // larger float, larger key; 0 and -0 are one
    uint32_t u = __float_as_uint(f);
    if (u == 0x80000000u) u = 0u;
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float((key & 0x80000000u) ? key & 0x7FFFFFFFu : ~key); }

template <class T>
__device__ __forceinline__ const T* of_peer(const T* p, int rank) {
    u64 out;
    asm("mapa.u64 %0, %1, %2;" : "=l"(out) : "l"(reinterpret_cast<u64>(p)), "r"(rank));
    return reinterpret_cast<const T*>(out);
}

struct Totals {                          // of the bins that a CTA adds up for its cluster
    u64 mass;
    uint32_t count;
};
struct Found {                           // where a search ended: a value, how many have it, and what comes before them
    uint32_t key, equal;
    uint32_t count;
    u64 weight, mass;
};
struct Share {                           // what the others read
    float top, low;
    double confidence;
    u64 mass_min_p;
    Totals slice[2];                     // sums over this CTA's bins; [1]: of a histogram of keys
    int n[2];                            // list of a bin's tokens (two in turn)
    uint32_t key_lo[2], key_hi[2];
    uint32_t equal;
};
struct alignas(16) Scratch {
    Share share;
    float f[2][kWarps];
    double d[kWarps];
    u64 m[2][kWarps];
    uint32_t c[kWarps];
    int bin;
    uint32_t bin_count;
    u64 bin_mass;
    Found found;
    int list_n;
    uint32_t list_lo, list_hi;
};
struct Entry {
    u64 weight;
    uint32_t key, pad;
};

template <class T>
struct SampleSmem {
    static size_t bytes(int chunk, int cluster) {
        return sizeof(Scratch) + kBins * 12 + 2 * (kBins / cluster) * sizeof(Totals) + 3 * kFew * sizeof(Entry) + (chunk + 16) * sizeof(T) + 64;
    }
};

template <class T>
__global__ void __launch_bounds__(kThreads) sample_kernel(const SampleArgs a) {
    extern __shared__ __align__(16) unsigned char smem[];
    const int cluster = a.cluster, row = blockIdx.x / cluster, rank = blockIdx.x % cluster;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int slice = kBins / cluster;
    u64* hist_mass = reinterpret_cast<u64*>(smem);
    Entry* lists = reinterpret_cast<Entry*>(hist_mass + kBins);              // [2][kFew], then the cluster's
    Entry* merged = lists + 2 * kFew;
    Totals* totals = reinterpret_cast<Totals*>(merged + kFew);               // [2][slice]
    Scratch& s = *reinterpret_cast<Scratch*>(totals + 2 * slice);
    uint32_t* hist_count = reinterpret_cast<uint32_t*>(&s + 1);
    T* held = reinterpret_cast<T*>(hist_count + kBins);
    Share& share = s.share;

    for (int i = tid; i < kBins; i += kThreads) { hist_mass[i] = 0ull; hist_count[i] = 0u; }
    pdl_wait();
    pdl_launch_dependents();

    // ---- this CTA's part of the row into shared memory; largest and smallest finite logit ----
    const int e0 = min(rank * a.chunk, a.vocab), n = min(a.chunk, a.vocab - e0);
    const T* from = static_cast<const T*>(a.logits) + (int64_t)row * a.row_stride + e0;
    constexpr int VEC = 16 / sizeof(T);
    const int shift = (int)(reinterpret_cast<uintptr_t>(from) % 16 / sizeof(T));     // held[shift + i]: whole pieces of 16 bytes in both places
    T* mine = held + shift;
    float top = -INFINITY, low = INFINITY;
    bool nan = false;
    auto take = [&](float v) -> float {
        if (v != v) { nan = true; v = -INFINITY; }
        top = fmaxf(top, v);
        if (v > -INFINITY) low = fminf(low, v);
        return v;
    };
    auto to_f = [](T v) -> float { if constexpr (sizeof(T) == 2) return __bfloat162float(v); else return v; };
    auto from_f = [](float v) -> T { if constexpr (sizeof(T) == 2) return __float2bfloat16(v); else return v; };
    {
        const int lead = min(n, (VEC - shift) % VEC), body = (n - lead) / VEC;
        for (int i = tid; i < lead; i += kThreads) mine[i] = from_f(take(to_f(from[i])));
        for (int i = lead + body * VEC + tid; i < n; i += kThreads) mine[i] = from_f(take(to_f(from[i])));
        constexpr int AHEAD = 4;
        for (int i0 = tid; i0 < body; i0 += AHEAD * kThreads) {
            uint4 v[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j)
                if (i0 + j * kThreads < body) v[j] = __ldcs(reinterpret_cast<const uint4*>(from + lead) + i0 + j * kThreads);
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                if (i0 + j * kThreads >= body) break;
                T* x = reinterpret_cast<T*>(&v[j]);
#pragma unroll
                for (int k = 0; k < VEC; ++k) x[k] = from_f(take(to_f(x[k])));
                *(reinterpret_cast<uint4*>(mine + lead) + i0 + j * kThreads) = v[j];
            }
        }
    }
    if (nan) atomicOr(a.status, kFlagNonFinite);
    auto logit = [&](int i) { return to_f(mine[i]); };
#pragma unroll
    for (int off = 16; off; off >>= 1) {
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
        low = fminf(low, __shfl_xor_sync(0xffffffffu, low, off));
    }
    if (lane == 0) { s.f[0][warp] = top; s.f[1][warp] = low; }
    __syncthreads();
    if (warp == 0) {
        top = lane < kWarps ? s.f[0][lane] : -INFINITY;
        low = lane < kWarps ? s.f[1][lane] : INFINITY;
#pragma unroll
        for (int off = 16; off; off >>= 1) {
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
            low = fminf(low, __shfl_xor_sync(0xffffffffu, low, off));
        }
        if (lane == 0) { share.top = top; share.low = low; }
    }
    cluster_sync_all();
    top = share.top; low = share.low;
    for (int r = 0; r < cluster; ++r) {
        const Share* p = of_peer(&share, r);
        top = fmaxf(top, p->top);
        low = fminf(low, p->low);
    }
    if (top == -INFINITY) {                                  // nothing to draw
        if (rank == 0 && tid == 0) {
            a.token[row] = -1;
            if (a.prob) a.prob[row] = 0.f;
            if (a.confidence) a.confidence[row] = 0.f;
        }
        cluster_sync_all();                                  // nobody leaves while its shared memory is read
        return;
    }

    // ---- the row's settings ----
    const int at = row / a.rows_per_setting;
    const float temperature = a.temperature ? a.temperature[at] : 1.f;
    const bool greedy = !(temperature > 0.f);
    const float top_p = a.top_p ? a.top_p[at] : 1.f;
    const float min_p = a.min_p && a.min_p[at] > 0.f ? fminf(a.min_p[at], 1.f) : 0.f;
    const int top_k = a.top_k ? a.top_k[at] : 0;
    const double unit = (double)(1ull << a.shift);
    const double rate = 1.4426950408889634074 / (double)temperature;         // log2 of a weight per logit
    // half of the distance from the largest, which may be infinite (the whole of it would pass fp32's range between finite logits)
    const float half_top = 0.5f * top;
    auto behind = [&](float l) { return l == top ? 0.f : fmaf(-0.5f, l, half_top); };
    auto weight = [&](float l) -> u64 {
        const double y = l == top ? 0.0 : ((double)top - (double)l) * rate;
        return __double2ull_rn(exp2(-y) * unit);
    };
    // logits that count: their weight is not below half of the unit
    const float reach = fminf(fminf(behind(low), (float)(0.5 * (a.shift + 1.0) / rate)), 3.4028234663852886e38f);
    const float bins_per = (float)kBins / reach;             // (infinite where all are equal: they are in bin 0, as 0 times it is NaN and that a 0)
    auto bin_of = [&](float d) { return min((int)(d * bins_per), kBins - 1); };

    // ---- weights and counts by bins; the sum for the confidence; what min_p leaves ----
    const u64 least = (u64)ceil((double)min_p * unit);
    double conf = 0.0;
    u64 mass_min_p = 0ull;
    {
        float c = 0.f;
        for (int i = tid; i < n; i += kThreads) {
            const float l = logit(i), d = behind(l);
            c += exp2f(d * -2.8853900817779268f);
            if (!greedy && d <= reach) {
                const u64 w = weight(l);
                const int bin = bin_of(d);
                atomicAdd(&hist_mass[bin], w);
                atomicAdd(&hist_count[bin], 1u);
                if (w >= least) mass_min_p += w;
            }
        }
        conf = c;
    }
#pragma unroll
    for (int off = 16; off; off >>= 1) {
        conf += __shfl_xor_sync(0xffffffffu, conf, off);
        mass_min_p += __shfl_xor_sync(0xffffffffu, mass_min_p, off);
    }
    if (lane == 0) { s.d[warp] = conf; s.m[0][warp] = mass_min_p; }
    __syncthreads();
    if (tid == 0) {
        double x = 0.0;
        u64 y = 0ull;
        for (int w = 0; w < kWarps; ++w) { x += s.d[w]; y += s.m[0][w]; }
        share.confidence = x;
        share.mass_min_p = y;
    }

    // sums over the cluster of this CTA's bins; the histogram is clear afterwards
    auto add_up = [&](int level) {
        cluster_sync_all();
        u64 m = 0ull;
        uint32_t c = 0u;
        for (int i = tid; i < slice; i += kThreads) {
            Totals t{0ull, 0u};
            for (int r = 0; r < cluster; ++r) {
                t.mass += *of_peer(hist_mass + rank * slice + i, r);
                t.count += *of_peer(hist_count + rank * slice + i, r);
            }
            totals[level * slice + i] = t;
            m += t.mass;
            c += t.count;
        }
#pragma unroll
        for (int off = 16; off; off >>= 1) {
            m += __shfl_xor_sync(0xffffffffu, m, off);
            c += __shfl_xor_sync(0xffffffffu, c, off);
        }
        if (lane == 0) { s.m[0][warp] = m; s.c[warp] = c; }
        __syncthreads();
        if (tid == 0) {
            Totals t{0ull, 0u};
            for (int w = 0; w < kWarps; ++w) { t.mass += s.m[0][w]; t.count += s.c[w]; }
            share.slice[level] = t;
        }
        cluster_sync_all();
        for (int i = tid; i < kBins; i += kThreads) { hist_mass[i] = 0ull; hist_count[i] = 0u; }
    };

    // the first bin at which the running count (or weight) comes to `target`, from s.bin_count, s.bin_mass on: s.bin, and what is before it
    auto locate = [&](int level, bool by_count, u64 target) {
        uint32_t count = s.bin_count;
        u64 mass = s.bin_mass;
        int owner = 0;
        for (; owner < cluster - 1; ++owner) {
            const Totals t = of_peer(&share, owner)->slice[level];
            if ((by_count ? (u64)(count + t.count) : mass + t.mass) >= target) break;
            count += t.count;
            mass += t.mass;
        }
        const int per = (slice + kThreads - 1) / kThreads, i0 = tid * per;
        const Totals* from_owner = of_peer(totals + level * slice, owner);
        u64 m = 0ull;
        uint32_t c = 0u;
        for (int i = i0; i < min(i0 + per, slice); ++i) {
            const Totals t = from_owner[i];
            m += t.mass;
            c += t.count;
        }
        u64 m_to = m;
        uint32_t c_to = c;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const u64 x = __shfl_up_sync(0xffffffffu, m_to, off);
            const uint32_t y = __shfl_up_sync(0xffffffffu, c_to, off);
            if (lane >= off) { m_to += x; c_to += y; }
        }
        if (lane == 31) { s.m[0][warp] = m_to; s.c[warp] = c_to; }
        __syncthreads();                                     // (also: everyone has read where the search begins)
        for (int w = 0; w < warp; ++w) { mass += s.m[0][w]; count += s.c[w]; }
        mass += m_to - m;
        count += c_to - c;
        const bool last = i0 < slice && i0 + per >= slice;   // (whatever the target, some bin is found)
        for (int i = i0; i < min(i0 + per, slice); ++i) {
            const Totals t = from_owner[i];
            const u64 before = by_count ? (u64)count : mass, upto = by_count ? (u64)(count + t.count) : mass + t.mass;
            if (before < target && (target <= upto || (last && i == slice - 1))) {
                s.bin = owner * slice + i;
                s.bin_count = count;
                s.bin_mass = mass;
            }
            count += t.count;
            mass += t.mass;
        }
        __syncthreads();
    };

    // the value at which the running count (or weight) comes to `target`
    int turn = 0;
    auto find = [&](bool by_count, u64 target) -> Found {
        __syncthreads();
        if (tid == 0) { s.bin_count = 0u; s.bin_mass = 0ull; }
        __syncthreads();
        locate(0, by_count, target);
        uint32_t lo = 0u, hi = 0xffffffffu;                  // keys of the bin, once it is one of keys
        bool keys = false;
        for (;;) {
            // the bin's tokens, in a list of this CTA's
            if (tid == 0) { s.list_n = 0; s.list_lo = 0xffffffffu; s.list_hi = 0u; }
            __syncthreads();
            Entry* list = lists + turn * kFew;
            const int bin = s.bin;
            uint32_t k_lo = 0xffffffffu, k_hi = 0u;
            for (int i = tid; i < n; i += kThreads) {
                const float l = logit(i), d = behind(l);
                const uint32_t key = order_key(l);
                if (d <= reach && (keys ? key >= lo && key <= hi : bin_of(d) == bin)) {
                    k_lo = min(k_lo, key);
                    k_hi = max(k_hi, key);
                    const int slot = atomicAdd(&s.list_n, 1);
                    if (slot < kFew) { list[slot].key = key; list[slot].weight = weight(l); }
                }
            }
            k_lo = __reduce_min_sync(0xffffffffu, k_lo);
            k_hi = __reduce_max_sync(0xffffffffu, k_hi);
            if (lane == 0 && k_lo <= k_hi) { atomicMin(&s.list_lo, k_lo); atomicMax(&s.list_hi, k_hi); }
            __syncthreads();
            if (tid == 0) { share.n[turn] = s.list_n; share.key_lo[turn] = s.list_lo; share.key_hi[turn] = s.list_hi; }
            cluster_sync_all();
            int all = 0;
            lo = 0xffffffffu;
            hi = 0u;
            for (int r = 0; r < cluster; ++r) {
                const Share* p = of_peer(&share, r);
                all += p->n[turn];
                lo = min(lo, p->key_lo[turn]);
                hi = max(hi, p->key_hi[turn]);
            }
            const uint32_t count = s.bin_count;
            const u64 mass = s.bin_mass;
            if (lo == hi) {                                  // one value
                turn ^= 1;
                return Found{lo, (uint32_t)all, count, weight(value_of(lo)), mass};
            }
            if (all <= kFew) {
                int first = 0;
                for (int r = 0; r < cluster; ++r) {
                    const int m = of_peer(&share, r)->n[turn];
                    for (int i = tid; i < m; i += kThreads) merged[first + i] = *of_peer(list + i, r);
                    first += m;
                }
                turn ^= 1;
                __syncthreads();
                for (int i = warp; i < all; i += kWarps) {
                    const uint32_t key = merged[i].key;
                    const u64 w = merged[i].weight;
                    u64 m = 0ull;
                    uint32_t c = 0u, e = 0u;
                    for (int j = lane; j < all; j += 32) {
                        const uint32_t k = merged[j].key;
                        if (k > key) { m += merged[j].weight; ++c; }
                        e += k == key;
                    }
#pragma unroll
                    for (int off = 16; off; off >>= 1) m += __shfl_xor_sync(0xffffffffu, m, off);
                    c = __reduce_add_sync(0xffffffffu, c);
                    e = __reduce_add_sync(0xffffffffu, e);
                    m += mass;
                    c += count;
                    const u64 before = by_count ? (u64)c : m, upto = by_count ? (u64)(c + e) : m + w * e;
                    if (lane == 0 && before < target && target <= upto) s.found = Found{key, e, c, w, m};
                }
                __syncthreads();
                return s.found;
            }
            // too many: a histogram of their keys, the largest first
            turn ^= 1;
            const uint32_t width = hi - lo;
            const int by = max(0, 21 - __clz(width));        // at most 2048 bins
            for (int i = tid; i < n; i += kThreads) {
                const float l = logit(i);
                const uint32_t key = order_key(l);
                if (behind(l) <= reach && key >= lo && key <= hi) {
                    atomicAdd(&hist_mass[(hi - key) >> by], weight(l));
                    atomicAdd(&hist_count[(hi - key) >> by], 1u);
                }
            }
            add_up(1);
            locate(1, by_count, target);
            const uint32_t b_lo = (uint32_t)s.bin << by, b_hi = b_lo + ((1u << by) - 1u);
            const uint32_t top_key = hi;
            hi = top_key - b_lo;
            lo = max(lo, top_key - min(b_hi, width));
            keys = true;
        }
    };

    uint32_t token_key = order_key(top);
    u64 token_at = 0ull;                                     // which of the tokens of that value
    double prob = 1.0;
    if (!greedy) {
        add_up(0);
        u64 sum = 0ull, left = 0ull;
        uint32_t count = 0u;
        for (int r = 0; r < cluster; ++r) {
            const Share* p = of_peer(&share, r);
            sum += p->slice[0].mass;
            count += p->slice[0].count;
            left += p->mass_min_p;
        }
        if (top_k > 0 && (uint32_t)top_k < count) {
            const Found f = find(true, (u64)top_k);
            sum = f.mass + f.weight * ((u64)top_k - f.count);
        }
        u64 kept = sum;
        if (top_p < 1.f) {
            const u64 enough = min(max((u64)ceil((double)fmaxf(top_p, 0.f) * (double)sum), 1ull), sum);
            const Found f = find(false, enough);
            kept = f.mass + (enough - f.mass + f.weight - 1ull) / f.weight * f.weight;
        }
        if (least > 0ull) kept = min(kept, left);
        const float u = a.u[row];
        const u64 share_of = u > 0.f ? min((u64)((double)fminf(u, 1.f) * (double)kept), kept - 1ull) : 0ull;
        const Found f = find(false, share_of + 1ull);
        token_key = f.key;
        token_at = min((share_of - f.mass) / f.weight, (u64)(f.equal - 1u));
        prob = (double)f.weight / (double)kept;
    }

    // ---- among the tokens of the value, the one with that many before it ----
    const int seg = (n + kThreads - 1) / kThreads * 32, j0 = min(warp * seg, n), j1 = min(j0 + seg, n);
    uint32_t equal = 0u;
    for (int i = j0 + lane; i < j1; i += 32) equal += order_key(logit(i)) == token_key;
    equal = __reduce_add_sync(0xffffffffu, equal);
    __syncthreads();
    if (lane == 0) s.c[warp] = equal;
    __syncthreads();
    if (tid == 0) {
        uint32_t all = 0u;
        for (int w = 0; w < kWarps; ++w) all += s.c[w];
        share.equal = all;
    }
    cluster_sync_all();
    u64 before = 0ull;
    double total = 0.0;
    for (int r = 0; r < cluster; ++r) {
        const Share* p = of_peer(&share, r);
        if (r < rank) before += p->equal;
        total += p->confidence;
    }
    for (int w = 0; w < warp; ++w) before += s.c[w];
    if (before <= token_at && token_at < before + equal) {   // one warp of the cluster
        for (int i = j0; i < j1; i += 32) {
            const bool eq = i + lane < j1 && order_key(logit(i + lane)) == token_key;
            const uint32_t eqs = __ballot_sync(0xffffffffu, eq);
            if (eq && before + __popc(eqs & ((1u << lane) - 1u)) == token_at) {
                const float l = value_of(token_key);
                a.token[row] = e0 + i + lane;
                if (a.prob) a.prob[row] = (float)prob;
                if (a.confidence) a.confidence[row] = (float)((l == top ? 1.0 : exp((double)l - (double)top)) / total);
            }
            before += __popc(eqs);
        }
    }
    cluster_sync_all();                                      // nobody leaves while its shared memory is read
}

template <class T>
int sample_launch(SampleArgs a, cudaStream_t stream) {
    static PerDevice<int> ready;
    int device = 0;
    cudaGetDevice(&device);
    const int most = ready.of(device, [](int& bytes) {
        int optin = 0, dev = 0;
        cudaGetDevice(&dev);
        cudaDeviceGetAttribute(&optin, cudaDevAttrMaxSharedMemoryPerBlockOptin, dev);
        bytes = cudaFuncSetAttribute(sample_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, optin) == cudaSuccess ? optin : 0;
    });
    if (most == 0) return -1;
    auto chunk_of = [&](int c) { return ((a.vocab + c - 1) / c + 63) / 64 * 64; };
    int c = 1;
    while (c < kMaxCluster && chunk_of(c) > 16384) c *= 2;
    a.cluster = c;
    a.chunk = chunk_of(c);
    a.shift = 46;
    while (((int64_t)a.vocab << a.shift) > (int64_t)1 << 62) --a.shift;      // the sum of all weights stays below 2^63
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(a.rows * c);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = SampleSmem<T>::bytes(a.chunk, c);
    cfg.stream = stream;
    if (cfg.dynamicSmemBytes > (size_t)most) return -1;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = c; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, sample_kernel<T>, a) == cudaSuccess ? 1 : -1;
}

}  // namespace

int launch_sample(const SampleArgs& a, cudaStream_t stream) {
    if (a.rows == 0) return 0;
    return a.bf16 ? sample_launch<__nv_bfloat16>(a, stream) : sample_launch<float>(a, stream);
}

}  // namespace acache
