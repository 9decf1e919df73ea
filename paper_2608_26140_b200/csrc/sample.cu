// Sampling of a token from a row of logits.
//
//   w_i = exp((l_i - max l) / T); in the order of falling l (equal ones by their index) a prefix is kept: the first top_k, the fewest of those that
//   make up top_p of their weight, those with w_i >= min_p, whatever is least; the token is the first of them whose running sum
//   passes u times the sum S of all that are kept.
//
// A weight is a whole number of 2^-shift (46 bits behind the point for up to 2^16 tokens, one less for every doubling), so that sums are exact and do not
// depend on their order; what is below half of that is never drawn.  A row belongs to a cluster of CTAs, which keep it in shared memory or read it
// again from L2; what one finds out it writes to the others, and every CTA takes every decision by itself, so that a step of a search costs
// one or two barriers of the cluster.
//  - A top_k of up to kTop: while the row comes in every thread keeps its largest logit, and of those a bound follows that at least top_k tokens
//    reach and few others.  They go into a list of the first CTA, which sorts it, adds up their weights and decides.  No other weight is formed.
//    (Where too many reach the bound, those of the bins that hold the first top_k are taken.)
//  - Else the weights of all tokens are added up by bins, which part the logits evenly from the largest to the smallest that counts: in three parts of
//    16 bits, as a 32-bit atomic that returns nothing takes a twentieth of a 64-bit one's time.  Each of the searches (the k-th token, the one at
//    which top_p is reached, the one that is drawn) goes to a bin, then over the tokens of that bin: sorted, where they are few, else by
//    another histogram of their keys.  A search ends at a value; among the tokens that have it the index decides.
// The sum for the confidence is kept while the row comes in, against each thread's largest logit so far.
//
// What bounds it: 512 rows of 126464 fp32 logits, each with settings of its own, 233 us (floor 40), 128 bf16 rows with top_p 101 us, one row with top_k
// and top_p 11.0 us.  The chain of steps of a row, two CTAs an SM: of the 50 us that a CTA of 31616 bf16 logits takes without a top_k, 17 are the weights (conflicts
// of the atomics: random bins meet about four to a bank), 5 the row, 14 two searches, the rest barriers and sums; a word to another CTA is there after 0.6 us,
// a barrier of the cluster takes 0.25.  Issue slots are busy for half of the time.
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
constexpr int kTop = 1024, kList = 2048; // largest top_k whose tokens are sorted; room for them and those that come with them
constexpr int kMaxCluster = 8;
constexpr int kMostLogits = 65536;       // of a CTA: sums of as many parts of 16 bits fit in 32
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kSteps = 64, kCopies = 16; // a table of 2^(-j / 64), a copy for every lane of half a warp: no two in one bank

__device__ __forceinline__ uint32_t order_key(float f) {     // larger float, larger key; 0 and -0 are one
    uint32_t u = __float_as_uint(f);
    if (u == 0x80000000u) u = 0u;
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float((key & 0x80000000u) ? key & 0x7FFFFFFFu : ~key); }

// the same place in another CTA of the cluster
template <class T>
__device__ __forceinline__ T* of_peer(T* p, int rank) {
    u64 out;
    asm("mapa.u64 %0, %1, %2;" : "=l"(out) : "l"(reinterpret_cast<u64>(p)), "r"(rank));
    return reinterpret_cast<T*>(out);
}

struct Totals {
    u64 mass;
    uint32_t count;
};
struct Place {                           // a bin, what is before it, and with it
    Totals before, upto;
    int bin;
};
struct Found {                           // where a search ended: a value, how many have it, its weight, and what comes before it
    uint32_t key, equal;
    uint32_t count;                      // (of a search by count only)
    u64 weight, mass;
};
// What the CTAs of a cluster tell one another, each in the others' memory before a barrier: reading there takes a thousand clocks.
struct Inbox {
    float top[kMaxCluster], low[kMaxCluster], bound[kMaxCluster], bound_each[kMaxCluster];
    double confidence[kMaxCluster];
    u64 mass_min_p[kMaxCluster];
    Totals slice[2][kMaxCluster];        // of each CTA's share of the bins; [1]: of a histogram of keys
    Place place;
    int n[2][kMaxCluster];               // lengths of lists (two in turn)
    uint32_t key_lo[2][kMaxCluster], key_hi[2][kMaxCluster];
    uint32_t equal[kMaxCluster];
};
struct alignas(16) Scratch {
    Inbox box;
    double power[kSteps][kCopies];
    float f[2][kWarps];
    double d[kWarps];
    u64 m[2][kWarps];
    uint32_t c[kWarps];
    int list_n;
    uint32_t list_lo, list_hi;
    u64 reached[2];
};
struct Hist {                            // this CTA's counts, or its weights in three parts of 16 bits, whose sums fit in 32 bits: atomics that return nothing
    uint32_t part[3][kBins];
};
union Work {                             // one after the other
    Hist hist;
    u64 top[kList];                      // key and index of the tokens of the first bins, a word each: every CTA's in the first one's memory
    struct {
        uint32_t own[kFew];              // keys of a bin's tokens
        uint32_t key[2][2 * kFew];       // every CTA's, two in turn
        uint32_t merged[kFew];           // one after the other
        u64 upto[kFew];                  // sums of their weights, the largest first
    } few;
};

// kHold: the row's part stays in shared memory; else it is read again (from L2) for every pass that needs it.
template <class T>
size_t sample_smem(int chunk, int cluster, bool hold) {
    return sizeof(Work) + sizeof(Scratch) + 2 * (kBins / cluster) * (sizeof(u64) + sizeof(uint32_t)) + (hold ? (chunk + 32) * sizeof(T) : 0);
}

template <class T, bool kHold>
__global__ void __launch_bounds__(kThreads, 2) sample_kernel(const SampleArgs a) {
    extern __shared__ __align__(16) unsigned char smem[];
    const int cluster = a.cluster, row = blockIdx.x / cluster, rank = blockIdx.x % cluster;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int slice = kBins / cluster;
    Work& work = *reinterpret_cast<Work*>(smem);
    Hist& hist = work.hist;
    Scratch& s = *reinterpret_cast<Scratch*>(&work + 1);
    u64* masses = reinterpret_cast<u64*>(&s + 1);            // running sums of this CTA's bins, and of a histogram of keys: [2][slice]
    uint32_t* numbers = reinterpret_cast<uint32_t*>(masses + 2 * slice);
    T* held = reinterpret_cast<T*>(numbers + 2 * slice);
    Inbox& box = s.box;

    auto clear = [&] {
        __syncthreads();
        for (int i = tid; i < kBins; i += kThreads) hist.part[0][i] = hist.part[1][i] = hist.part[2][i] = 0u;
        __syncthreads();
    };
    cluster_arrive_relaxed();                                // waited for before the first word to another CTA: it has begun
    if (tid < kSteps) {
        const double x = exp2(-(double)tid / kSteps);
#pragma unroll 1
        for (int i = 0; i < kCopies; ++i) s.power[tid][i] = x;
    }
    pdl_wait();
    pdl_launch_dependents();

    // ---- the row's settings ----
    const int at = row / a.rows_per_setting;
    const float temperature = a.temperature ? a.temperature[at] : 1.f;
    const bool greedy = !(temperature > 0.f);
    const float top_p = a.top_p ? a.top_p[at] : 1.f;
    const float min_p = a.min_p && a.min_p[at] > 0.f ? fminf(a.min_p[at], 1.f) : 0.f;
    const int top_k = a.top_k ? a.top_k[at] : 0;
    const bool sampled = !greedy && top_k > 0, quick = sampled && top_k <= kTop && (top_k + cluster - 1) / cluster <= kThreads;

    // ---- this CTA's part of the row into shared memory; largest and smallest finite logit ----
    const int e0 = min(rank * a.chunk, a.vocab), n = min(a.chunk, a.vocab - e0);
    const T* from = static_cast<const T*>(a.logits) + (int64_t)row * a.row_stride + e0;
    constexpr int VEC = 16 / sizeof(T);
    const int shift = (int)(reinterpret_cast<uintptr_t>(from) % 16 / sizeof(T));     // held[shift + i]: whole pieces of 16 bytes in both places
    const int pieces = (shift + n + VEC - 1) / VEC;          // the first and the last filled up with -inf
    float top = -INFINITY, low = INFINITY;
    float conf = 0.f, conf_top = -3.4028234663852886e38f;    // sum of exp(l - conf_top) over this thread's logits, conf_top the largest of them so far
    bool nan = false;
    auto to_f = [](T v) -> float { if constexpr (sizeof(T) == 2) return __bfloat162float(v); else return v; };
    auto from_f = [](float v) -> T { if constexpr (sizeof(T) == 2) return __float2bfloat16(v); else return v; };
    auto unpack = [](const uint4& v, float (&x)[VEC]) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if constexpr (sizeof(T) == 2) { x[2 * k] = bf16_lo(w[k]); x[2 * k + 1] = bf16_hi(w[k]); }
            else x[k] = __uint_as_float(w[k]);
        }
    };
    auto ex2f = [](float x) {
        float e;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x));
        return e;
    };
    int top_piece = 0;                                       // where `top` is, and the largest logit of this thread's other pieces
    float next_top = -INFINITY;
    // a piece as it came: NaN out, its share of largest, smallest and sum
    auto take = [&](uint4& v, int i) {
        float x[VEC], high = -INFINITY;
        unpack(v, x);
        bool odd = false;
#pragma unroll
        for (int k = 0; k < VEC; ++k) odd |= x[k] != x[k];
        if (odd) {
            nan = true;
            T* w = reinterpret_cast<T*>(&v);
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
                x[k] = x[k] != x[k] ? -INFINITY : x[k];
                w[k] = from_f(x[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < VEC; ++k) high = fmaxf(high, x[k]);
        if (!greedy && !quick)                               // (who else needs the range of the bins takes all that weights allow)
#pragma unroll
            for (int k = 0; k < VEC; ++k) low = fminf(low, x[k] > -INFINITY ? x[k] : INFINITY);
        next_top = fmaxf(next_top, fminf(top, high));
        if (high > top) {
            top = high;
            top_piece = i;
        }
        if (a.confidence) {
            if (high > conf_top) {
                conf *= ex2f((conf_top - high) * kLog2e);
                conf_top = high;
            }
            float e[VEC];                                    // (added up by themselves: fewer roundings of the large sum)
#pragma unroll
            for (int k = 0; k < VEC; ++k) e[k] = ex2f((x[k] - conf_top) * kLog2e);
#pragma unroll
            for (int half = VEC / 2; half; half /= 2)
#pragma unroll
                for (int k = 0; k < half; ++k) e[k] += e[k + half];
            conf += e[0];
        }
    };
    // Piece i is thread i % kThreads', here and in every later pass.
    const int whole0 = shift ? 1 : 0, whole1 = (shift + n) / VEC;            // pieces that are all the row's
    const uint4* source = reinterpret_cast<const uint4*>(from - shift);      // (aligned; the first piece is not read here where it is not whole)
    auto partial = [&](int i) {
        uint4 v;
        T* w = reinterpret_cast<T*>(&v);
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
            const int e = i * VEC + k - shift;
            w[k] = e >= 0 && e < n ? from[e] : from_f(-INFINITY);
        }
        return v;
    };
    {
        auto alone = [&](int i) {
            uint4 v = partial(i);
            take(v, i);
            if (kHold) reinterpret_cast<uint4*>(held)[i] = v;
        };
        if (whole0 && tid == 0) alone(0);
        if (whole1 < pieces && whole1 >= whole0 && tid == whole1 % kThreads) alone(whole1);
        constexpr int AHEAD = 4;
        for (int i0 = tid; i0 < whole1; i0 += AHEAD * kThreads) {
            uint4 v[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                const int i = i0 + j * kThreads;
                if (i >= whole0 && i < whole1) v[j] = kHold ? __ldcs(source + i) : __ldcg(source + i);
            }
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                const int i = i0 + j * kThreads;
                if (i < whole0 || i >= whole1) continue;
                take(v[j], i);
                if (kHold) reinterpret_cast<uint4*>(held)[i] = v[j];
            }
        }
    }
    if (nan) atomicOr(a.status, kFlagNonFinite);
    bool endless = false;                                    // infinite logits: those are read as 0, all others as -inf, which has the same limits
    // a piece to f(logits, index of the first)
    auto one = [&](int i, auto&& f) {
        float x[VEC];
        if (kHold) {
            unpack(reinterpret_cast<const uint4*>(held)[i], x);
        } else {
            unpack(i >= whole0 && i < whole1 ? __ldcg(source + i) : partial(i), x);
            if (nan)
#pragma unroll
                for (int k = 0; k < VEC; ++k) x[k] = x[k] != x[k] ? -INFINITY : x[k];
        }
        if (endless)
#pragma unroll
            for (int k = 0; k < VEC; ++k) x[k] = x[k] == INFINITY ? 0.f : -INFINITY;
        f(x, i * VEC - shift);
    };
    auto each = [&](auto&& f) {
#pragma unroll 1
        for (int i = tid; i < pieces; i += kThreads) one(i, f);
    };
    // a value a thread, the largest to the first thread; room: threads that have one (a power of two, 32 and more)
    auto sorted = [&](auto v, int room, auto* exchange) {
#pragma unroll
        for (int size = 2; size <= kThreads; size *= 2) {
            if (size > room) break;
#pragma unroll
            for (int step = size / 2; step; step /= 2) {
                decltype(v) other;
                if (step >= 32) {
                    __syncthreads();
                    exchange[tid] = v;
                    __syncthreads();
                    other = exchange[tid ^ step];
                } else {
                    other = __shfl_xor_sync(0xffffffffu, v, step);
                }
                const bool larger = ((tid & size) == 0) == ((tid & step) == 0);
                v = (v > other) == larger ? v : other;
            }
        }
        return v;
    };
    float own_top = top;
    cluster_wait();
    // A bound that top_k tokens reach at least: the largest logits of that many threads.  Two bounds hold: top_k of one CTA's threads, and a share of
    // top_k in every CTA's.  (Of 31 logits a thread, those of 50 threads of 512: about 53 tokens of a CTA are as large; those of 7 threads in
    // each of 8 CTAs, the least of them: 80 of the row.)
    if (quick) {
        const uint32_t key = sorted(order_key(top), kThreads, work.few.merged);
        if (tid == top_k - 1) s.f[0][0] = value_of(key);
        if (tid == (top_k + cluster - 1) / cluster - 1) s.f[0][1] = value_of(key);
        __syncthreads();
        if (tid < cluster) {
            of_peer(&box, tid)->bound[rank] = top_k <= kThreads ? s.f[0][0] : -INFINITY;
            of_peer(&box, tid)->bound_each[rank] = s.f[0][1];
        }
        __syncthreads();
    }
#pragma unroll
    for (int off = 16; off; off >>= 1) {
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
        low = fminf(low, __shfl_xor_sync(0xffffffffu, low, off));
    }
    if (lane == 0) { s.f[0][warp] = top; s.f[1][warp] = low; }
    __syncthreads();
    if (warp == 0) {
        top = s.f[0][lane % kWarps];
        low = s.f[1][lane % kWarps];
#pragma unroll
        for (int off = kWarps / 2; off; off >>= 1) {
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
            low = fminf(low, __shfl_xor_sync(0xffffffffu, low, off));
        }
        if (lane < cluster) {
            Inbox* of = of_peer(&box, lane);
            of->top[rank] = top;
            of->low[rank] = low;
        }
    }
    if (!quick) clear();
    cluster_sync_all();
    float bound = -INFINITY;
    {
        float each_of = INFINITY;
        for (int r = 0; r < cluster; ++r) {
            top = r ? fmaxf(top, box.top[r]) : box.top[0];
            low = r ? fminf(low, box.low[r]) : box.low[0];
            if (quick) {
                bound = fmaxf(bound, box.bound[r]);
                each_of = fminf(each_of, box.bound_each[r]);
            }
        }
        if (quick) bound = fmaxf(bound, each_of);
    }
    if (top == -INFINITY) {                                  // nothing to draw
        if (rank == 0 && tid == 0) {
            a.token[row] = -1;
            if (a.prob) a.prob[row] = 0.f;
            if (a.confidence) a.confidence[row] = 0.f;
        }
        return;
    }

    endless = top == INFINITY;
    if (greedy || quick) low = -INFINITY;
    if (endless) {
        own_top = own_top == INFINITY ? 0.f : -INFINITY;
        next_top = next_top == INFINITY ? 0.f : -INFINITY;
        bound = bound == INFINITY ? 0.f : -INFINITY;
        top = low = 0.f;
    }
    const double unit = (double)(1ull << a.shift);
    const double rate = 1.4426950408889634074 / (double)temperature;         // log2 of a weight per logit
    const u64 least = (u64)ceil((double)min_p * unit);
    // half of the distance from the largest (the whole of it may pass fp32's range)
    const float half_top = 0.5f * top;
    auto behind = [&](float l) { return fmaf(-0.5f, l, half_top); };
    // 2^-y in units, for y up to shift + 1: y = j / 64 + r, the table's 2^(-j / 64) times 2^-r by its series, of which |r ln 2|^6 / 720 < 2^-54 is left
    // out; the last addition rounds to whole units
    auto weight = [&](float l) -> u64 {
        constexpr double kRound = 1.5 * 70368744177664.0;                    // 1.5 * 2^46: what is added to it is rounded to 1 / 64
        constexpr double kLn2 = -0.69314718055994530942;
        const double d = (double)top - (double)l, t = fma(d, rate, kRound), r = fma(d, rate, -(t - kRound));
        const int j = __double2loint(t);
        const double at = s.power[j & (kSteps - 1)][lane & (kCopies - 1)];
        const double scaled = __hiloint2double(__double2hiint(at) + ((a.shift - (j >> 6)) << 20), __double2loint(at));
        double p = fma(r, kLn2 * kLn2 * kLn2 * kLn2 * kLn2 / 120, kLn2 * kLn2 * kLn2 * kLn2 / 24);
        p = fma(r, p, kLn2 * kLn2 * kLn2 / 6);
        p = fma(r, p, kLn2 * kLn2 / 2);
        p = fma(r, p, kLn2);
        p = fma(r, p, 1.0);
        return (u64)__double_as_longlong(fma(scaled, p, 4503599627370496.0)) & 0xFFFFFFFFFFFFFull;
    };
    // logits that count: their weight is not below half of the unit
    const float reach = fminf(fminf(behind(low), (float)(0.5 * (a.shift + 1.0) / rate)), 3.4028234663852886e38f);
    const float bins_per = (float)(kBins - 1) / reach;       // (infinite where all are equal)
    auto bin_of = [&](float d) { return d > 0.f ? (int)(__float_as_uint(fmaf(fminf(d, reach), bins_per, 8388608.f)) & (kBins - 1)) : 0; };      // to the nearest

    // ---- counts and weights by bins, what min_p leaves ----
    u64 mass_min_p = 0ull;
    auto add_weight = [&](int bin, u64 w) {
#pragma unroll
        for (int p = 0; p < 3; ++p) atomicAdd(&hist.part[p][bin], (uint32_t)(w >> (16 * p)) & (p < 2 ? 0xFFFFu : 0xFFFFFFFFu));
    };
    // one pass over the logits, for counts or for weights; four at a time, without a branch until their weights are there
    auto pass = [&](bool counts) {
        each([&](const float (&x)[VEC], int) {
#pragma unroll
            for (int k0 = 0; k0 < VEC; k0 += 4) {
                int bin[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float d = behind(x[k0 + k]);
                    bin[k] = d <= reach ? bin_of(d) : -1;
                }
                if (counts) {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (bin[k] >= 0) atomicAdd(&hist.part[0][bin[k]], 1u);
                    continue;
                }
                u64 w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = weight(bin[k] >= 0 ? x[k0 + k] : top);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (bin[k] >= 0) add_weight(bin[k], w[k]);
                if (least)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (bin[k] >= 0 && w[k] >= least) mass_min_p += w[k];
            }
        });
    };
    // sum of a value over the CTA, in every thread of warp 0
    auto cta_sum = [&](auto v, auto* at_warp) {
#pragma unroll
        for (int off = 16; off; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
        if (lane == 0) at_warp[warp] = v;
        __syncthreads();
        if (warp == 0) {
            v = at_warp[lane % kWarps];
#pragma unroll
            for (int off = kWarps / 2; off; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
        }
        return v;
    };

    // sum of a value over the threads up to this one
    auto running = [&](u64 v) {
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const u64 x = __shfl_up_sync(0xffffffffu, v, off);
            if (lane >= off) v += x;
        }
        __syncthreads();
        if (lane == 31) s.m[0][warp] = v;
        __syncthreads();
        u64 before = lane < warp ? s.m[0][lane] : 0ull;      // (fewer warps than lanes)
#pragma unroll
        for (int off = kWarps / 2; off; off >>= 1) before += __shfl_xor_sync(0xffffffffu, before, off);
        return v + __shfl_sync(0xffffffffu, before, 0);
    };

    // running sums over the cluster of this CTA's bins, counts or weights (the others stay as they are); box.slice: every CTA's whole sum
    auto add_up = [&](int level, bool counts) {
        cluster_sync_all();
        // a thread kMine bins of one CTA: the CTAs side by side
        constexpr int kMine = kBins / kThreads;
        const int peer = tid & (cluster - 1), i0 = tid / cluster * kMine;
        const Hist* h = of_peer(&hist, peer);
        u64 m[kMine];
#pragma unroll
        for (int q = 0; q < kMine; q += 4) {
            auto four = [&](int p) { return *reinterpret_cast<const uint4*>(h->part[p] + rank * slice + i0 + q); };
            const uint4 x = four(0);
            m[q] = x.x; m[q + 1] = x.y; m[q + 2] = x.z; m[q + 3] = x.w;
            if (!counts) {
                const uint4 y = four(1), z = four(2);
                m[q] += ((u64)y.x << 16) + ((u64)z.x << 32); m[q + 1] += ((u64)y.y << 16) + ((u64)z.y << 32);
                m[q + 2] += ((u64)y.z << 16) + ((u64)z.z << 32); m[q + 3] += ((u64)y.w << 16) + ((u64)z.w << 32);
            }
        }
        for (int off = 1; off < cluster; off <<= 1)
#pragma unroll
            for (int j = 0; j < kMine; ++j) m[j] += __shfl_xor_sync(0xffffffffu, m[j], off);
#pragma unroll
        for (int j = 1; j < kMine; ++j) m[j] += m[j - 1];
        const u64 run = running(peer == 0 ? m[kMine - 1] : 0ull);
        if (peer == 0) {
#pragma unroll
            for (int j = 0; j < kMine; ++j) {
                if (counts) numbers[level * slice + i0 + j] = (uint32_t)(run - m[kMine - 1] + m[j]);
                else masses[level * slice + i0 + j] = run - m[kMine - 1] + m[j];
            }
        }
        if (warp == kWarps - 1) {
            const u64 all = __shfl_sync(0xffffffffu, run, 31);
            if (lane < cluster) {
                Totals& t = of_peer(&box, lane)->slice[level][rank];
                if (counts) t.count = (uint32_t)all;
                else t.mass = all;
            }
        }
        cluster_sync_all();
    };

    // The first bin at which the running count (or weight), `before` the first one, comes to `target`: the CTA that has it tells the others.  The sum that
    // is not searched by is there only if `both` have been added up; else it is not looked at, and the place's is zero.
    auto locate = [&](int level, bool by_count, bool both, u64 target, Totals before) -> Place {
        const bool counts = by_count || both, weights = !by_count || both;
        int owner = 0;
        for (; owner < cluster - 1; ++owner) {
            const Totals& t = box.slice[level][owner];
            const Totals with{before.mass + (weights ? t.mass : 0ull), before.count + (counts ? t.count : 0u)};
            if ((by_count ? (u64)with.count : with.mass) >= target) break;
            before = with;
        }
        if (rank == owner) {
            const u64* mass = masses + level * slice;
            const uint32_t* number = numbers + level * slice;
            for (int i = tid; i < slice; i += kThreads) {
                const Totals t0{before.mass + (weights && i > 0 ? mass[i - 1] : 0ull), before.count + (counts && i > 0 ? number[i - 1] : 0u)};
                const Totals t1{before.mass + (weights ? mass[i] : 0ull), before.count + (counts ? number[i] : 0u)};
                const u64 from_here = by_count ? (u64)t0.count : t0.mass, to_here = by_count ? (u64)t1.count : t1.mass;
                if ((from_here < target || i == 0) && (target <= to_here || i == slice - 1))     // (whatever the target, some bin is found)
                    for (int r = 0; r < cluster; ++r) of_peer(&box, r)->place = Place{t0, t1, owner * slice + i};
            }
        }
        cluster_sync_all();
        return box.place;
    };
    // The value at which the running count (or weight) comes to `target`.  By count: what comes before is counted and weighed; by weight: weighed only.
    int turn = 0;
    auto find = [&](bool by_count, u64 target) -> Found {
        Place at_bin = locate(0, by_count, by_count, target, Totals{0ull, 0u});
        uint32_t lo = 0u, hi = 0xffffffffu;                  // keys of the bin, once it is one of keys
        bool keys = false;
        for (int level = 0;; ++level) {                      // (a histogram of keys narrows them down to a 2048th of their range)
            // the bin's tokens, in a list of this CTA's
            if (tid == 0) { s.list_n = 0; s.list_lo = 0xffffffffu; s.list_hi = 0u; }
            __syncthreads();
            const int bin = at_bin.bin;
            // Logits of the bin lie less than a bin from its middle, whatever was rounded: the others are sorted out by two comparisons.
            float from_l = -INFINITY, to_l = INFINITY;
            if (!keys && bins_per < 1e30f) {
                from_l = __double2float_rd((double)top - 2.0 * (bin + 1) / (double)bins_per);
                to_l = __double2float_ru((double)top - 2.0 * (bin - 1) / (double)bins_per);
            }
            uint32_t k_lo = 0xffffffffu, k_hi = 0u;
            each([&](const float (&x)[VEC], int) {
#pragma unroll
                for (int k = 0; k < VEC; ++k) {
                    if (!(x[k] >= from_l && x[k] <= to_l)) continue;
                    const float d = behind(x[k]);
                    const uint32_t key = order_key(x[k]);
                    if (d <= reach && (keys ? key >= lo && key <= hi : bin_of(d) == bin)) {
                        k_lo = min(k_lo, key);
                        k_hi = max(k_hi, key);
                        const int slot = atomicAdd(&s.list_n, 1);
                        if (slot < kFew) work.few.own[slot] = key;
                    }
                }
            });
            k_lo = __reduce_min_sync(0xffffffffu, k_lo);
            k_hi = __reduce_max_sync(0xffffffffu, k_hi);
            if (lane == 0 && k_lo <= k_hi) { atomicMin(&s.list_lo, k_lo); atomicMax(&s.list_hi, k_hi); }
            __syncthreads();
            // to everyone: as many warps for each
            const int room_of = cluster == 1 ? kFew : 2 * kFew / cluster, mine_n = s.list_n;
            {
                const int peer = warp % cluster;
                uint32_t* to = of_peer(work.few.key[turn] + rank * room_of, peer);
                for (int i = warp / cluster * 32 + lane; i < min(mine_n, room_of); i += kWarps / cluster * 32) to[i] = work.few.own[i];
                if (warp < cluster && lane == 0) {
                    Inbox* of = of_peer(&box, peer);
                    of->n[turn][rank] = mine_n;
                    of->key_lo[turn][rank] = s.list_lo;
                    of->key_hi[turn][rank] = s.list_hi;
                }
            }
            cluster_sync_all();
            lo = 0xffffffffu;
            hi = 0u;
            int all = 0, longest = 0;
            for (int r = 0; r < cluster; ++r) {
                all += box.n[turn][r];
                longest = max(longest, box.n[turn][r]);
                lo = min(lo, box.key_lo[turn][r]);
                hi = max(hi, box.key_hi[turn][r]);
            }
            const uint32_t count = at_bin.before.count;
            const u64 mass = at_bin.before.mass;
            if (lo >= hi || level == 4) {                    // one value
                turn ^= 1;
                return Found{lo, (uint32_t)all, count, weight(value_of(lo)), mass};
            }
            if (all <= kFew && longest <= room_of) {
                uint32_t* merged = work.few.merged;
                const int r_of = warp % cluster;
                int first = 0;
                for (int r = 0; r < r_of; ++r) first += box.n[turn][r];
                for (int i = warp / cluster * 32 + lane; i < box.n[turn][r_of]; i += kWarps / cluster * 32)
                    merged[first + i] = work.few.key[turn][r_of * room_of + i];
                __syncthreads();
                turn ^= 1;
                int room = 32;
                while (room < all) room *= 2;
                static_assert(kFew == kThreads, "a thread has a key");
                const uint32_t key = sorted(tid < all ? merged[tid] : 0u, room, work.few.own);
                const u64 w = tid < all ? weight(value_of(key)) : 0ull;
                const u64 run = running(w) + mass;           // with this key
                const u64 before = by_count ? (u64)(count + tid) : run - w, upto = by_count ? (u64)(count + tid + 1) : run;
                work.few.upto[tid] = run;
                if (tid < all && before < target && target <= upto) s.list_lo = key;
                __syncthreads();
                const uint32_t found = s.list_lo;
                const int larger = __syncthreads_count(tid < all && key > found), equal = __syncthreads_count(tid < all && key == found);
                return Found{found, (uint32_t)equal, count + larger, weight(value_of(found)), larger ? work.few.upto[larger - 1] : mass};
            }
            // too many: a histogram of their keys, the largest first
            turn ^= 1;
            clear();
            const uint32_t width = hi - lo;
            const int by = max(0, 21 - __clz(width));        // at most 2048 bins
            for (int counts = by_count; counts >= 0; --counts) {
                if (by_count && !counts) clear();
                each([&](const float (&x)[VEC], int) {
#pragma unroll
                    for (int k = 0; k < VEC; ++k) {
                        const uint32_t key = order_key(x[k]);
                        if (behind(x[k]) <= reach && key >= lo && key <= hi) {
                            if (counts) atomicAdd(&hist.part[0][(hi - key) >> by], 1u);
                            else add_weight((hi - key) >> by, weight(x[k]));
                        }
                    }
                });
                add_up(1, counts);
            }
            at_bin = locate(1, by_count, by_count, target, at_bin.before);
            const uint32_t b_lo = (uint32_t)at_bin.bin << by, b_hi = b_lo + ((1u << by) - 1u);
            const uint32_t top_key = hi;
            hi = top_key - b_lo;
            lo = max(lo, top_key - min(b_hi, width));
            keys = true;
        }
    };
    // what is kept of a sum by top_p
    auto enough_of = [&](u64 sum) { return min(max((u64)ceil((double)fmaxf(top_p, 0.f) * (double)sum), 1ull), sum); };
    auto drawn_of = [&](u64 kept) {
        const float u = a.u[row];
        return u > 0.f ? min((u64)((double)fminf(u, 1.f) * (double)kept), kept - 1ull) : 0ull;
    };
    auto give = [&](int token, float l, double prob, double total) {
        a.token[row] = token;
        if (a.prob) a.prob[row] = (float)prob;
        if (a.confidence) a.confidence[row] = (float)(exp((double)l - (double)top) / total);
    };

    auto cluster_sum = [&](const auto (&v)[kMaxCluster], int n) {
        auto sum = v[0];
        sum = 0;
        for (int r = 0; r < n; ++r) sum += v[r];
        return sum;
    };
    if (a.confidence) {
        double c = 0.0;
        if (endless) each([&](const float (&x)[VEC], int) {                  // (the running sums say nothing then)
#pragma unroll
            for (int k = 0; k < VEC; ++k) c += x[k] == 0.f;
        });
        else c = (double)conf * (double)ex2f((conf_top - top) * kLog2e);
        c = cta_sum(c, s.d);
        if (tid < cluster) of_peer(&box, tid)->confidence[rank] = c;
    }
    auto total_of = [&] { return a.confidence ? cluster_sum(box.confidence, cluster) : 1.0; };

    // ---- a small top_k: its tokens in a list ----
    for (int attempt = quick ? 0 : 1; sampled && top_k <= kTop && attempt < 2; ++attempt) {
        int bin = -1;
        if (attempt == 1) {
            // by the counts of the bins
            if (quick) clear();                              // (too many tokens reach the bound)
            pass(true);
            add_up(0, true);
            uint32_t count = 0u;
            for (int r = 0; r < cluster; ++r) count += box.slice[0][r].count;
            const Place p = locate(0, true, false, min((u64)top_k, (u64)count), Totals{0ull, 0u});
            if (p.upto.count > kList) break;
            bin = p.bin;
        }
        if (tid == 0) s.list_n = 0;
        __syncthreads();
        const int room_of = kList / cluster;
        u64* to = of_peer(work.top + rank * room_of, 0);
        auto put = [&](float l, int i) {
            const int slot = atomicAdd(&s.list_n, 1);
            if (slot < room_of) to[slot] = (u64)order_key(l) << 32 | ~(uint32_t)(e0 + i);
        };
        if (attempt == 1 || own_top >= bound) {
            // (few threads have a token that reaches the bound, and those in one of their pieces, as a rule)
            const bool whole_share = attempt == 1 || next_top >= bound;
#pragma unroll 1
            for (int i = whole_share ? tid : top_piece; i < pieces; i += whole_share ? kThreads : pieces)
                one(i, [&](const float (&x)[VEC], int i0) {
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        const float d = behind(x[j]);
                        if (attempt == 0 ? x[j] >= bound && x[j] > -INFINITY : d <= reach && bin_of(d) <= bin) put(x[j], i0 + j);
                    }
                });
        }
        __syncthreads();
        if (tid < cluster) of_peer(&box, tid)->n[attempt][rank] = s.list_n;
        cluster_sync_all();
        int all = 0, longest = 0;
        for (int r = 0; r < cluster; ++r) {
            all += box.n[attempt][r];
            longest = max(longest, box.n[attempt][r]);
        }
        if (longest > room_of) continue;
        if (rank != 0) return;                               // nobody writes to its memory, or reads there, any more
        const double total = total_of();
        // sorted, kThreads apart
        constexpr int kMost = kList / kThreads;
        u64 word[kMost];
        int per = 1;
        if (all <= kThreads) {
            int i = tid, r = 0;
            while (r < cluster && i >= box.n[attempt][r]) i -= box.n[attempt][r++];
            int room = 32;
            while (room < all) room *= 2;
            word[0] = sorted(r < cluster ? work.top[r * room_of + i] : 0ull, room, work.top);
        } else {
            per = kMost;
            for (int i = tid; i < kList; i += kThreads)
                if (i % room_of >= box.n[attempt][i / room_of]) work.top[i] = 0ull;
#pragma unroll 1
            for (int size = 2; size <= kList; size *= 2)
#pragma unroll 1
                for (int step = size / 2; step; step /= 2) {
                    __syncthreads();
                    for (int i = tid; i < kList / 2; i += kThreads) {
                        const int x = 2 * i - (i & (step - 1)), y = x + step;
                        const u64 u = work.top[x], v = work.top[y];
                        if ((u < v) == ((x & size) == 0)) { work.top[x] = v; work.top[y] = u; }      // the largest first
                    }
                }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kMost; ++j) word[j] = work.top[j * kThreads + tid];
        }
        // running sums of the weights of the first top_k: upto, with this token
        u64 w[kMost], upto[kMost], kept = 0ull;
#pragma unroll
        for (int j = 0; j < kMost; ++j) {
            w[j] = upto[j] = 0ull;
            if (j >= per) continue;
            if (j * kThreads + tid < min(top_k, all)) {
                const float l = value_of((uint32_t)(word[j] >> 32));
                if (behind(l) <= reach) w[j] = weight(l);
            }
            upto[j] = running(w[j]) + kept;
            for (int v = 0; v < kWarps; ++v) kept += s.m[0][v];
        }
        // the sum at the first token where it comes to what top_p keeps; [1]: before the first that min_p does not leave
        const u64 enough = top_p < 1.f ? enough_of(kept) : kept;
        if (tid == 0) s.reached[1] = kept;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kMost; ++j) {
            if (w[j] == 0ull) continue;
            if (upto[j] - w[j] < enough && enough <= upto[j]) s.reached[0] = upto[j];
            if (w[j] < least) atomicMin(&s.reached[1], upto[j] - w[j]);
        }
        __syncthreads();
        kept = min(s.reached[0], s.reached[1]);
        const u64 target = drawn_of(kept) + 1ull;
#pragma unroll
        for (int j = 0; j < kMost; ++j)
            if (w[j] != 0ull && upto[j] - w[j] < target && target <= upto[j])
                give((int)~(uint32_t)word[j], value_of((uint32_t)(word[j] >> 32)), (double)w[j] / (double)kept, total);
        return;
    }
    if (sampled && top_k <= kTop) clear();                   // the list was too long

    uint32_t token_key = order_key(top);
    u64 token_at = 0ull;                                     // which of the tokens of that value
    uint32_t equal_all = 0u;                                 // how many there are, where that is known
    double prob = 1.0, total = 1.0;
    if (!greedy) {
        const bool counts = top_k > 0;
        if (counts) {
            pass(true);
            add_up(0, true);
            clear();
        }
        pass(false);
        const u64 left_here = cta_sum(mass_min_p, s.m[1]);
        if (tid < cluster) of_peer(&box, tid)->mass_min_p[rank] = left_here;
        add_up(0, false);
        u64 sum = 0ull;
        uint32_t count = 0u;
        for (int r = 0; r < cluster; ++r) {
            sum += box.slice[0][r].mass;
            if (counts) count += box.slice[0][r].count;
        }
        total = total_of();
        if (counts && (uint32_t)top_k < count) {
            const Found f = find(true, (u64)top_k);
            sum = f.mass + f.weight * ((u64)top_k - f.count);
        }
        u64 kept = sum;
        if (top_p < 1.f) {
            const u64 enough = enough_of(sum);
            const Found f = find(false, enough);
            kept = f.mass + (enough - f.mass + f.weight - 1ull) / f.weight * f.weight;
        }
        if (least > 0ull) kept = min(kept, cluster_sum(box.mass_min_p, cluster));
        const u64 drawn = drawn_of(kept);
        const Found f = find(false, drawn + 1ull);
        token_key = f.key;
        equal_all = f.equal;
        token_at = min((drawn - f.mass) / f.weight, (u64)(f.equal - 1u));
        prob = (double)f.weight / (double)kept;
    }
    if (equal_all == 1u) {
        each([&](const float (&x)[VEC], int i0) {
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (x[j] == value_of(token_key)) give(e0 + i0 + j, x[j], prob, total);
        });
        return;
    }

    // ---- among the tokens of the value, the one with that many before it ----
    // how many a warp's pieces have, round by round, which is the order of their indices
    const float value = value_of(token_key);
    uint32_t* count_of = reinterpret_cast<uint32_t*>(&work); // [round][warp]
    static_assert(((kMostLogits + 2 * VEC) / VEC / kThreads + 1) * kWarps * sizeof(uint32_t) <= sizeof(Work), "a word for every round and warp");
    const int rounds = (pieces + kThreads - 1) / kThreads;
    auto has = [&](int i) {                                  // tokens of piece i, a bit each
        uint32_t bits = 0u;
        if (i < pieces && own_top >= value) one(i, [&](const float (&x)[VEC], int) {
#pragma unroll
            for (int k = 0; k < VEC; ++k) bits |= x[k] == value && x[k] > -INFINITY ? 1u << k : 0u;
        });
        return bits;
    };
    __syncthreads();
    uint32_t here = 0u;
#pragma unroll 1
    for (int j = 0; j < rounds; ++j) {
        const uint32_t c = __reduce_add_sync(0xffffffffu, __popc(has(j * kThreads + tid)));
        if (lane == 0) count_of[j * kWarps + warp] = c;
        here += c;
    }
    here = cta_sum(lane == 0 ? here : 0u, s.c);
    if (tid < cluster) of_peer(&box, tid)->equal[rank] = here;
    cluster_sync_all();
    if (greedy) total = total_of();
    u64 before = cluster_sum(box.equal, rank);
    if (token_at < before || token_at >= before + box.equal[rank]) return;
    int group = 0;                                           // the round and warp that have it
    for (; before + count_of[group] <= token_at; ++group) before += count_of[group];
    if (group % kWarps != warp) return;
    const int i = group / kWarps * kThreads + tid;
    uint32_t bits = has(i), upto = __popc(bits);
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, upto, off);
        if (lane >= off) upto += x;
    }
    const int nth = (int)(token_at - before) - (int)(upto - __popc(bits));      // of this lane's
    if (nth < 0 || nth >= __popc(bits)) return;
    for (int k = 0; k < nth; ++k) bits &= bits - 1u;
    give(e0 + i * VEC - shift + __ffs(bits) - 1, value, prob, total);
}

int chunk_of(int vocab, int c) { return ((vocab + c - 1) / c + 63) / 64 * 64; }

template <class T, bool kHold>
int sample_launch(SampleArgs a, int c, cudaStream_t stream) {
    static PerDevice<bool> ready;
    int device = 0;
    cudaGetDevice(&device);
    if (!ready.of(device, [](bool& ok) {
            int optin = 0, dev = 0;
            cudaGetDevice(&dev);
            cudaDeviceGetAttribute(&optin, cudaDevAttrMaxSharedMemoryPerBlockOptin, dev);
            ok = cudaFuncSetAttribute(sample_kernel<T, kHold>, cudaFuncAttributeMaxDynamicSharedMemorySize, optin) == cudaSuccess;
        }))
        return -1;
    a.cluster = c;
    a.chunk = chunk_of(a.vocab, c);
    a.shift = 46;
    while (((int64_t)a.vocab << a.shift) > (int64_t)1 << 62) --a.shift;      // the sum of all weights stays below 2^63
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(a.rows * c);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = sample_smem<T>(a.chunk, c, kHold);
    cfg.stream = stream;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = c; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, sample_kernel<T, kHold>, a) == cudaSuccess ? 1 : -1;
}
// CTAs of a row: as many as pay while there are SMs for them, one each down to 4096 logits a CTA, two an SM down to 8192 (clusters of 8 find no more than 256 places
// at a time); us on average over settings, 32000 bf16 logits by 1, 2, 4, 8 CTAs: one row 22, 16, 13, 12; 37 rows 32, 24.6, 22.4, 32; 128 rows 32, 32, 42, 70.  With more
// rows than that a step's cost is spread over up to 40960 logits a CTA, up to twice as many with 4 CTAs: 300 bf16 rows of 151936 by 8 CTAs 234, by 4 183, of 262144 312
// and 261, fp32 379 and 321.  (Fewer CTAs wait for the row whose settings take longest: 512 fp32 rows of 126464 with settings of their own by 4 CTAs 236, by 2 254.)
// The row stays in shared memory where that leaves room for two CTAs in an SM, or there are so few that no two need share one, else it is read again from L2: 300 bf16
// rows of 8000 held with room for one CTA 45, read again 37; 5 fp32 rows of 151936 23.5 and 28, 16 rows 37.5 and 35.
template <class T>
int sample_dispatch(const SampleArgs& a, cudaStream_t stream) {
    constexpr size_t kHalfSm = 113 * 1024;
    int c = 1;
    for (; c < kMaxCluster; c *= 2) {
        const int chunk = chunk_of(a.vocab, c);
        const int64_t ctas = (int64_t)a.rows * 2 * c;
        if (!(chunk > kMostLogits || (chunk > 40960 && (c < 4 || ctas <= 2 * 148)) || (chunk > 8192 && ctas <= 256) || (chunk > 4096 && ctas <= 128))) break;
    }
    const bool hold = sample_smem<T>(chunk_of(a.vocab, c), c, true) <= kHalfSm || (int64_t)a.rows * c <= 64;
    return hold ? sample_launch<T, true>(a, c, stream) : sample_launch<T, false>(a, c, stream);
}

}  // namespace

int launch_sample(const SampleArgs& a, cudaStream_t stream) {
    if (a.rows == 0) return 0;
    return a.bf16 ? sample_dispatch<__nv_bfloat16>(a, stream) : sample_dispatch<float>(a, stream);
}

}  // namespace acache
