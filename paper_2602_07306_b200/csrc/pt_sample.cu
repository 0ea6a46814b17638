// Drawing one token per row of logits: temperature, top-k, top-p, min-p, then the inverse of the cumulative
// distribution at a given number u in [0, 1).  (The paper stops at h; sampling is part of the ends of the model that it
// leaves to "standard" practice, like the greedy choice.)
//
// With m = max x and w_i = exp((x_i - m) / temperature), every filter keeps a prefix of the tokens ordered by (logit
// descending, index ascending), so the kept set is "key above a threshold, or equal to it and index at most a cut":
//   top-k   the first k tokens
//   top-p   of those, the shortest prefix whose weight reaches p times their sum
//   min-p   of those, the tokens with w_i >= min_p
// and the token is the lowest kept index whose cumulative weight, summed in index order, exceeds u times the kept sum.
//
// Weights are whole multiples of 2^-44: integer sums do not depend on their order, so neither the number of blocks nor
// the order of atomics changes a result, and ties at a threshold are exact.  A weight below 2^-45 (45 ln 2 = 31.19 nats under
// the maximum) is zero: such a token is never drawn.  The exponential is evaluated in double; the multiple rounds it once,
// an absolute error of 2^-45 against a sum of at least 1.
//
// Three ways to take a row.  For few rows, whose time is latency, a cluster of up to 8 blocks, which exchange what they found
// through distributed shared memory; each holds its slice in shared memory, or, where that would leave one block on an SM,
// streams over it, the first pass from HBM and the later ones from L2.  For many rows, where exchanging between blocks costs
// more than it saves, one block streams over the row.
//
// Two ways to find the kept set.
// Few candidates (top-k up to kListK, or min-p alone): the k-th largest of the maxima that the threads found, four each, is a
// lower bound of the k-th largest logit, so a second pass collects the logits above it - little more than k - and one block
// sorts them and finishes the row alone.
// Everything else (top-p over the whole vocabulary, a large k, no filter): a histogram of the distance to the maximum in
// kBins bins bounds, from counts alone, which bins may hold the threshold: a weight in a bin is known to the bin's width,
// 0.8 % and half a unit, and so are the sums before and behind a bin.  One pass then sums the weights above those bins exactly and lists the
// logits inside them, and one block sorts that list and cuts it.  Where the list is too long (many equal logits), or top-p
// follows a large top-k, histograms with exact counts and weights narrow the threshold down to one key instead.
//
// Measured, top-k 50 / top-p 0.9 / no filter, in us: 1 x 32000 10.6 / 21 / 8.6 and 64 x 128000 19 / 53 / 24, latency of the
// exchanges and barriers; 1000 x 128000 181 / 457 / 230 (greedy 85; reading the logits once takes 79), bound by the instructions of
// the weights, with top-k by reading the rows twice: 296 rows in work at a time do not fit the L2.
#include <cooperative_groups.h>

#include "pt_internal.h"
#include "pt_sample.h"

namespace cg = cooperative_groups;

namespace pt {

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBins = 4096;                    // first histogram: distance to the maximum
constexpr int kFine = 2048;                    // later histograms: keys
constexpr int kCoarse = kThreads;              // histogram of the threads' maxima
constexpr int kList = 2048;                    // entries one block sorts
constexpr int kListK = 1024;                   // largest top-k that goes that way
constexpr int kBatch = 4;                      // quads a thread loads before it looks at them
constexpr int kBuckets = 1024;
constexpr int kFew = 128;                      // entries that are ranked by counting, not sorted
constexpr float kRange = 31.5f;                // nats below the maximum that the bins cover; beyond it weights are zero
constexpr float kSlack = 4e-7f;                // relative rounding of a distance and its bin number, three times over
constexpr int kMaxCluster = 8;
constexpr int kMaxSlice = 32768;               // elements of a slice: 128 KB
constexpr int kMaxVocab = 393216;

typedef unsigned long long u64;

// Distance-ordered key: smaller key = larger value.  -0 and +0 are one value.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);
    return (b & 0x80000000u) ? b : ~b & 0x7fffffffu;
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float((key & 0x80000000u) ? key : ~key & 0x7fffffffu); }

struct Row {
    float max, inv_bin;                        // bin of x = (max - x) * inv_bin
    double maxd, inv_t;                        // inv_t: log2(e) / temperature
    double inv16;                              // 16 inv_t
    float x_zero;                              // weights are zero below it
    float x_min;                               // min-p: kept values are >= x_min
    const double* root;                        // 2^(44 + j / 16), in shared memory
};

__constant__ double kRoot[16] = {1, 1.0442737824274138, 1.0905077326652577, 1.1387886347566916,
                                  1.189207115002721, 1.241857812073484, 1.2968395546510096, 1.3542555469368927,
                                  1.4142135623730951, 1.4768261459394993, 1.5422108254079407, 1.6104903319492543,
                                  1.681792830507429, 1.7562521603732995, 1.8340080864093424, 1.9152065613971474};

// w(x) * 2^44, rounded to the nearest whole number, as the low 52 bits of a double in [2^52, 2^53): 2^y with 16 y =
// 16 (x - max) log2(e) / temperature split into a whole number k and g in [-1/2, 1/2]; 2^(g / 16) by the polynomial of
// degree 5 that agrees with it at the six Chebyshev nodes of the interval (relative error 4.6e-15, a twelfth of the last
// place kept of the largest weight), 2^(44 + k / 16) from a table of sixteen and the exponent; adding 2^52 rounds to a whole
// number.  Logits below x_zero, where that gives 0, count as x_zero.  The loops are bound by the instructions they issue
// (70 a logit with the bits masked, compared and selected; the double-precision pipe was 19 % busy), so sums add the doubles'
// bits as they are and take kOffset off per term.
constexpr u64 kOffset = 0x4330000000000000ull;
__device__ __forceinline__ u64 weight_bits(const Row& r, float x) {
    const double d = (double)fmaxf(x, r.x_zero) - r.maxd;
    const double magic = 6755399441055744.0;   // 1.5 * 2^52: the sum's low word is round(16 y)
    const double k = fma(d, r.inv16, magic);
    const double g = fma(d, r.inv16, -(k - magic));
    double p = 1.2716085030349987e-09;
    p = fma(p, g, 1.467644462189871e-07);
    p = fma(p, g, 1.355080777749983e-05);
    p = fma(p, g, 0.000938384792486206);
    p = fma(p, g, 0.04332169878499661);
    p = fma(p, g, 1.0000000000000044);
    const int ki = __double2loint(k);
    p *= r.root[ki & 15];
    return (u64)__double_as_longlong(__hiloint2double(__double2hiint(p) + (ki & ~15) * 65536, __double2loint(p)) + 4503599627370496.0);
}
__device__ __forceinline__ u64 weight(const Row& r, float x) { return weight_bits(r, x) - kOffset; }

// elements of bins, and bounds of their weight; the three sums over the block share their barriers
struct BinSum { u64 n; double up, dn; };

struct Shared {
    union {
        uint32_t bins[kBins];
        struct { u64 mass[kFine]; uint32_t hist[kFine]; };      // narrowing by keys
        struct { u64 all[kList], list[kList]; };                // entries of the row (in the first block), of this block
    };
    union {
        uint32_t coarse[kCoarse];
        struct { uint32_t rank[kFew]; };
    };
    union {
        struct { u64 few_w[kFew], few_sum[kFew], few_total[2]; };
        struct { uint32_t bucket_n[kBuckets], bucket_0[kBuckets]; };
    };
    float red[kWarps];
    u64 wsum[kMaxCluster * kWarps];            // first block: weight kept by the part of every warp of the cluster
    u64 warp_tmp[kWarps], warp_tmp2[kWarps];
    uint32_t warp_cnt[kWarps];
    u64 blk_mass, blk_all;                     // weight of this block's elements above the searched bins, and of all
    u64 scan[kWarps + 1];
    BinSum bin_scan[kWarps];
    double root[16];
    double share[3];                           // totals of this block's share of the bins: counts, upper and lower bounds
    float4 edge[2];                            // streamed: the quads that the slice does not fill
    float max;
    int n_list, n_all;                         // entries of this block; of the row (in the first block)
    // found by a scan, or handed over by the block that found it
    int bin;
    u64 before_mass, before_cnt, total;
    int zone_a, zone_b, tail_a, tail_b, cut, first;
    uint32_t thr; int owner; u64 target, Z;
};

static_assert(kFew == 128, "the thread counts below");
static_assert(((sizeof(Shared) + 15) & ~15) + (kMaxSlice + 4) * 4 <= 232448, "shared memory of one block");

template <class V> __device__ __forceinline__ V warp_incl(V v) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const V u = __shfl_up_sync(0xffffffffu, v, o); if (lane >= o) v += u; }
    return v;
}
template <class V> __device__ __forceinline__ V warp_sum(V v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// exclusive prefix of v over the block's threads; total = the block's sum.  buf holds kWarps + 1 values.
template <class V> __device__ __forceinline__ V block_excl(V v, V* buf, V& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const V incl = warp_incl(v);
    __syncthreads();
    if (lane == 31) buf[warp] = incl;
    __syncthreads();
    V w = lane < kWarps ? buf[lane] : V(0);
    const V wi = warp_incl(w);
    total = __shfl_sync(0xffffffffu, wi, kWarps - 1);
    return __shfl_sync(0xffffffffu, wi - w, warp) + incl - v;
}

__device__ __forceinline__ BinSum warp_incl(BinSum v) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const u64 n = __shfl_up_sync(0xffffffffu, v.n, o);
        const double up = __shfl_up_sync(0xffffffffu, v.up, o), dn = __shfl_up_sync(0xffffffffu, v.dn, o);
        if (lane >= o) { v.n += n; v.up += up; v.dn += dn; }
    }
    return v;
}
__device__ __forceinline__ BinSum block_excl_bins(const BinSum& v, BinSum* buf, BinSum& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const BinSum incl = warp_incl(v);
    __syncthreads();
    if (lane == 31) buf[warp] = incl;
    __syncthreads();
    BinSum mine{incl.n - v.n, incl.up - v.up, incl.dn - v.dn};
    total = BinSum{0, 0., 0.};
#pragma unroll 1
    for (int w = 0; w < kWarps; ++w) {
        const BinSum s = buf[w];
        total.n += s.n; total.up += s.up; total.dn += s.dn;
        if (w < warp) { mine.n += s.n; mine.up += s.up; mine.dn += s.dn; }
    }
    return mine;
}

// The kList entries of a, ascending (bitonic).  A thread holds four neighbours: pairs up to 2 apart meet in its registers, up
// to 64 apart by shuffles, and only the ten steps of wider pairs go through shared memory and a barrier.
__device__ __forceinline__ void sort_list(u64* a) {
    static_assert(kList == 4 * kThreads, "four entries a thread");
    const int t = threadIdx.x;
    ulonglong2* mem = reinterpret_cast<ulonglong2*>(a);
    u64 x[4];
    { const ulonglong2 p = mem[2 * t], q = mem[2 * t + 1]; x[0] = p.x; x[1] = p.y; x[2] = q.x; x[3] = q.y; }
    auto order = [](u64& lo, u64& hi, bool up) { const u64 l = lo, h = hi; const bool swap = (l > h) == up; lo = swap ? h : l; hi = swap ? l : h; };
#pragma unroll 1
    for (int size = 2; size <= kList; size <<= 1) {
        const bool up = (4 * t & size) == 0;                  // (size 2 below: the thread's second pair the other way)
#pragma unroll 1
        for (int stride = size >> 1; stride >= 4; stride >>= 1) {
            const bool low = (4 * t & stride) == 0, take_min = low == up;
            u64 y[4];
            if (stride >= 128) {
                __syncthreads();                              // the last step's reads are done
                mem[2 * t] = make_ulonglong2(x[0], x[1]); mem[2 * t + 1] = make_ulonglong2(x[2], x[3]);
                __syncthreads();
                const int o = t ^ (stride >> 2);
                const ulonglong2 p = mem[2 * o], q = mem[2 * o + 1];
                y[0] = p.x; y[1] = p.y; y[2] = q.x; y[3] = q.y;
            } else {
#pragma unroll
                for (int c = 0; c < 4; ++c) y[c] = __shfl_xor_sync(0xffffffffu, x[c], stride >> 2);
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) x[c] = (x[c] < y[c]) == take_min ? x[c] : y[c];
        }
        if (size > 2) { order(x[0], x[2], up); order(x[1], x[3], up); }
        order(x[0], x[1], size > 2 ? up : true);
        order(x[2], x[3], size > 2 ? up : false);
    }
    __syncthreads();
    mem[2 * t] = make_ulonglong2(x[0], x[1]); mem[2 * t + 1] = make_ulonglong2(x[2], x[3]);
    __syncthreads();
}

// Four logits at p (which is aligned to them): -inf in place of NaN.
__device__ __forceinline__ float4 load4(const float* p) {
    const float4 v = __ldcg(reinterpret_cast<const float4*>(p));
    return make_float4(fmaxf(v.x, -INFINITY), fmaxf(v.y, -INFINITY), fmaxf(v.z, -INFINITY), fmaxf(v.w, -INFINITY));
}
__device__ __forceinline__ float4 load4(const __nv_bfloat16* p) {
    const uint2 b = __ldcg(reinterpret_cast<const uint2*>(p));
    return make_float4(fmaxf(__uint_as_float(b.x << 16), -INFINITY), fmaxf(__uint_as_float(b.x & 0xffff0000u), -INFINITY),
                       fmaxf(__uint_as_float(b.y << 16), -INFINITY), fmaxf(__uint_as_float(b.y & 0xffff0000u), -INFINITY));
}

struct Full { static constexpr int value = kBatch; };
struct One { static constexpr int value = 1; };

template <class E, bool CLUSTER, bool HELD>
__global__ void __launch_bounds__(kThreads, 2)
k_sample(const SampleP p, const int slice) {
    extern __shared__ __align__(16) unsigned char smem_raw[];
    Shared& sh = *reinterpret_cast<Shared*>(smem_raw);
    float4* xs = reinterpret_cast<float4*>(smem_raw + ((sizeof(Shared) + 15) & ~15));
    cg::cluster_group cluster = cg::this_cluster();
    const int CL = CLUSTER ? (int)cluster.num_blocks() : 1, rank = CLUSTER ? (int)cluster.block_rank() : 0;
    auto sync_row = [&]() { if (CLUSTER) cluster.sync(); else __syncthreads(); };
    auto remote = [&](auto* ptr, int q) { return CLUSTER ? cluster.map_shared_rank(ptr, q) : ptr; };
    const int64_t row = blockIdx.x / CL;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int count = max(0, min(slice, p.vocab - rank * slice));
    const E* src = reinterpret_cast<const E*>(p.logits) + row * p.row_stride + rank * slice;
    // quads of four, aligned as in global memory: element i of the slice is component (i + shift) % 4 of quad (i + shift) / 4
    // (slices are a multiple of four long: the same shift in every block)
    const int shift = (int)((reinterpret_cast<uintptr_t>(src) / sizeof(E)) & 3);
    const int base = rank * slice - shift;                    // index of component 0 of quad 0
    const int quads = count ? (count + shift + 3) >> 2 : 0;
    const int per_warp = (quads + kWarps - 1) / kWarps;       // every warp owns a contiguous part of the slice
    const int v0 = min(quads, warp * per_warp), v1 = min(quads, v0 + per_warp);
    const E* quad0 = src - shift;
    const int full0 = shift ? 1 : 0, full1 = (count + shift) >> 2;     // quads [full0, full1) lie inside the row

    // the row's settings, early: their latency hides behind the logits'
    float temperature = p.temperature ? p.temperature[row] : 1.0f;
    const float tp = p.top_p ? p.top_p[row] : 1.0f, mp = p.min_p ? p.min_p[row] : 0.f, u = p.u[row];
    const int k = tp <= 0.f ? 1 : p.top_k ? p.top_k[row] : 0; // a reach of nothing keeps one token

    // ---- the slice (NaN counts as masked) and its maximum
    sh.coarse[tid] = 0;
    if (tid < 16) sh.root[tid] = kRoot[tid] * 17592186044416.0;     // 2^44
    if (tid == 0) { sh.n_list = 0; sh.n_all = 0; sh.first = 0x7fffffff; sh.thr = 0xffffffffu; sh.cut = 0x7fffffff; }
    if (tid < 2) {                                            // the quads at the ends: filled up with -inf
        const int v = tid ? quads - 1 : 0;
        float e[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) { const int i = v * 4 + c - shift; e[c] = v >= 0 && i >= 0 && i < count ? fmaxf((float)src[i], -INFINITY) : -INFINITY; }
        sh.edge[tid] = make_float4(e[0], e[1], e[2], e[3]);
    }
    __syncthreads();
    // f(v, n, q): up to kBatch quads of the warp's part, q[i] being quad v + 32 i, all lanes together (past the end: v = -1 and
    // quads of -inf), from global memory: the full quads first
    const float4 none = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
    auto from_global = [&](auto&& f) {
        const int lo = max(v0, full0), hi = min(v1, full1);
        int vb = lo;
        for (; vb + 32 * kBatch <= hi; vb += 32 * kBatch) {   // the loads first: f may write to shared memory
            float4 q[kBatch];
#pragma unroll
            for (int i = 0; i < kBatch; ++i) q[i] = load4(quad0 + (vb + i * 32 + lane) * 4);
            f(vb + lane, q, Full{});
        }
#pragma unroll 1
        for (; vb < hi; vb += 32) { const int v = vb + lane; const float4 q = v < hi ? load4(quad0 + v * 4) : none; f(v < hi ? v : -1, &q, One{}); }
#pragma unroll 1
        for (int k = 0; k < 2; ++k) {
            const int v = k ? quads - 1 : 0;
            if (v >= v0 && v < v1 && (v < full0 || v >= full1) && !(k && quads == 1)) { const float4 q = lane ? none : sh.edge[k]; f(lane ? -1 : v, &q, One{}); }
        }
    };
    // the same from wherever the row is held
    auto each_batch = [&](auto&& f) {
        if (HELD) {
            int vb = v0;
            for (; vb + 32 * kBatch <= v1; vb += 32 * kBatch) {
                float4 q[kBatch];
#pragma unroll
                for (int i = 0; i < kBatch; ++i) q[i] = xs[vb + i * 32 + lane];
                f(vb + lane, q, Full{});
            }
#pragma unroll 1
            for (; vb < v1; vb += 32) { const int v = vb + lane; const float4 q = v < v1 ? xs[v] : none; f(v < v1 ? v : -1, &q, One{}); }
        } else from_global(f);
    };
    // quad by quad
    auto single = [](auto&& f) {
        return [&f](int v, const float4* q, auto n) {
#pragma unroll
            for (int i = 0; i < decltype(n)::value; ++i) f(v + i * 32, q[i]);
        };
    };
    auto each = [&](auto&& f) { each_batch(single(f)); };
    auto get = [&](int v) {                                   // one quad, wherever the row is held
        if (HELD) return xs[v];
        float4 q = sh.edge[v == 0 ? 0 : 1];
        if (v >= full0 && v < full1) q = load4(quad0 + v * 4);
        return q;
    };
    float4 tmax = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
    const bool choose = !(temperature > 0.f && temperature < INFINITY);      // greedy
    int top = -1;                                             // greedy: the first of this thread's quads that holds its maximum
    if (choose) {
        from_global(single([&](int v, float4 q) {
            const float m = fmaxf(fmaxf(q.x, q.y), fmaxf(q.z, q.w));
            if (m > tmax.x || (m == tmax.x && v < top)) { tmax.x = m; top = v; }
        }));
    } else {
        from_global(single([&](int v, float4 q) {
            if (HELD && v >= 0) xs[v] = q;
            tmax = make_float4(fmaxf(tmax.x, q.x), fmaxf(tmax.y, q.y), fmaxf(tmax.z, q.z), fmaxf(tmax.w, q.w));
        }));
    }
    {
        float m = fmaxf(fmaxf(tmax.x, tmax.y), fmaxf(tmax.z, tmax.w));
#pragma unroll
        for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        if (lane == 0) sh.red[warp] = m;
        __syncthreads();
        m = lane < kWarps ? sh.red[lane] : -INFINITY;
#pragma unroll
        for (int o = 8; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        if (tid == 0) sh.max = m;
    }
    sync_row();
    Row r;
    {
        float m = lane < CL ? *remote(&sh.max, lane) : -INFINITY;
#pragma unroll
        for (int o = kMaxCluster / 2; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        r.max = __shfl_sync(0xffffffffu, m, 0);
    }
    const bool nothing = r.max == -INFINITY;                  // every logit masked: token 0, probability 0
    if (nothing || choose) {
        // greedy: the lowest index of the maximum
        if (choose && !nothing && tmax.x == r.max) {
            float4 q = sh.edge[top == 0 ? 0 : 1];
            if (top >= full0 && top < full1) q = load4(quad0 + top * 4);
            atomicMin(&sh.first, base + top * 4 + (q.x == r.max ? 0 : q.y == r.max ? 1 : q.z == r.max ? 2 : 3));
        }
        sync_row();
        if (rank == 0 && warp == 0) {
            int at = lane < CL ? *remote(&sh.first, lane) : 0x7fffffff;
            at = nothing ? 0 : __reduce_min_sync(0xffffffffu, at);
            if (lane == 0) {
                if (p.token) p.token[row] = at;
                if (p.token2) p.token2[row * p.token2_stride] = at;
                if (p.prob) p.prob[row * p.prob_stride] = nothing ? 0.f : 1.f;
            }
        }
        sync_row();                                           // no block leaves while another still reads its shared memory
        return;
    }
    // so that bin widths are finite and not zero, a step of the logits below the maximum is no more than 600 temperatures (its
    // weight is zero either way) and x_zero is a number
    temperature = fminf(fmaxf(temperature, 1e-30f), 1e36f);
    temperature = fmaxf(temperature, (r.max - __fsub_rd(r.max, 1e-45f)) * (1.0f / 600.0f));
    temperature = fminf(temperature, (r.max + 3.4028235e38f) * (1.0f / 33.0f));
    r.maxd = (double)r.max;
    r.inv_t = 1.4426950408889634 / (double)temperature;
    r.inv16 = 16.0 * r.inv_t;
    r.x_zero = __fsub_rd(r.max, 31.885f * temperature);       // 2^-46 of the largest or less, and below it
    r.root = sh.root;
    r.inv_bin = (float)(kBins - 1) / (kRange * temperature);
    r.x_min = -INFINITY;
    if (mp > 0.f) r.x_min = mp >= 1.f ? r.max : __double2float_ru(r.maxd + (double)temperature * log((double)mp));
    const bool use_k = k > 0 && k < p.vocab, use_p = tp < 1.0f && tp > 0.f;
    const u64 frac64 = use_p ? (u64)__double2ull_rz((double)tp * 18446744073709551616.0) : 0ull;
    const u64 U = u >= 1.f ? ~0ull : (u > 0.f ? (u64)__double2ull_rz((double)u * 18446744073709551616.0) : 0ull);
    uint32_t thr = 0xffffffffu; int cut = 0x7fffffff;         // kept so far: key < thr, or key == thr and index <= cut
    auto store = [&](int tok, float x, u64 Z) {
        if (p.token) p.token[row] = tok;
        if (p.token2) p.token2[row * p.token2_stride] = tok;
        if (p.prob) p.prob[row * p.prob_stride] = (float)(exp2(((double)x - r.maxd) * r.inv_t) / ((double)Z * 0x1p-44));
    };
    // the reach of top-p: ceil(whole * p), at least 1
    auto reach = [&](u64 whole) { const u64 hi = __umul64hi(whole, frac64); return max((u64)1, hi + (whole * frac64 != 0)); };
    // The draw from the weights that the warps' parts keep (wsum, in the first block): that block finds the warp whose part
    // holds the token, that warp's block the token.  kept_of: what of the sum is kept (the first of it); weight_of: a logit's
    // kept weight.
    auto draw = [&](auto&& kept_of, auto&& weight_of, auto&& put) {
        if (rank == 0 && warp == 0) {
            constexpr int PL = kMaxCluster * kWarps / 32;
            u64 sum[PL], mine = 0;
#pragma unroll
            for (int j = 0; j < PL; ++j) { sum[j] = lane * PL + j < CL * kWarps ? sh.wsum[lane * PL + j] : 0; mine += sum[j]; }
            const u64 incl = warp_incl(mine), Z = kept_of(__shfl_sync(0xffffffffu, incl, 31));
            const u64 target = __umul64hi(Z, U);              // the token: lowest index with cumulative weight > target
            u64 before = incl - mine;
#pragma unroll
            for (int j = 0; j < PL; ++j) {
                if (before <= target && before + sum[j] > target) {
                    Shared* o = remote(&sh, (lane * PL + j) / kWarps);
                    o->thr = thr; o->cut = cut; o->target = target - before; o->Z = Z;
                    const int own = (lane * PL + j) % kWarps;
                    for (int q = 0; q < CL; ++q) remote(&sh, q)->owner = q == (lane * PL + j) / kWarps ? own : -1;
                }
                before += sum[j];
            }
        }
        sync_row();
        if (sh.owner < 0) return;
        thr = sh.thr; cut = sh.cut;
        const u64 target = sh.target;
        const int r0 = min(quads, sh.owner * per_warp), r1 = min(quads, r0 + per_warp), share = (r1 - r0 + kThreads - 1) / kThreads;
        const int q0 = min(r1, r0 + tid * share), q1 = min(r1, q0 + share);      // consecutive quads of this thread
        u64 mine = 0, tot;
        for (int v = q0; v < q1; ++v) {
            const float4 q = get(v);
            const float e[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int c = 0; c < 4; ++c) mine += weight_of(e[c], base + v * 4 + c);
        }
        u64 cum = block_excl<u64>(mine, sh.scan, tot);
        if (cum <= target && cum + mine > target) {
            for (int v = q0; v < q1; ++v) {
                const float4 q = get(v);
                const float e[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const u64 w = weight_of(e[c], base + v * 4 + c);
                    if (cum <= target && cum + w > target) put(base + v * 4 + c, e[c], sh.Z);
                    cum += w;
                }
            }
        }
    };

    if (r.max == INFINITY || r.max == -3.4028235e38f) {
        // +inf shares the whole weight, and nothing but a mask lies below the lowest number: every weight is 1 or 0
        u64 n = 0;
        each([&](int, float4 q) { n += (q.x == r.max) + (q.y == r.max) + (q.z == r.max) + (q.w == r.max); });
        n = warp_sum(n);
        if (lane == 0) remote(&sh.wsum[0], 0)[rank * kWarps + warp] = n;
        sync_row();
        draw([&](u64 all) { const u64 m = use_k ? min(all, (u64)k) : all; return use_p ? min(m, reach(m)) : m; },
             [&](float x, int) { return x == r.max ? 1ull : 0ull; },
             [&](int tok, float, u64 Z) {
                 if (p.token) p.token[row] = tok;
                 if (p.token2) p.token2[row * p.token2_stride] = tok;
                 if (p.prob) p.prob[row * p.prob_stride] = 1.0f / (float)Z;
             });
        return;
    }
    // the logits of a batch whose bits (4 i + c for component c of quad v + 32 i) are set in `hit` into this block's list; all
    // lanes of the warp call it.  One atomic a warp and batch: one a logit took 30 us for a list of 1400.
    auto append = [&](unsigned hit, int v, const float4* q) {
        if (!__any_sync(0xffffffffu, hit != 0)) return;
        const int incl = warp_incl(__popc(hit));
        int at = 0;
        if (lane == 31) at = atomicAdd(&sh.n_list, incl);
        at = __shfl_sync(0xffffffffu, at, 31) + incl - __popc(hit);
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
            if (hit >> 4 * i & 15) {
                const float e[4] = {q[i].x, q[i].y, q[i].z, q[i].w};
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (hit >> (4 * i + c) & 1) { if (at < kList) sh.list[at] = (u64)key_of(e[c]) << 32 | (uint32_t)(base + (v + i * 32) * 4 + c); ++at; }
            }
    };
    // brings the blocks' lists together in the first block; returns the entries of the row (more than kList: not brought)
    auto gather = [&]() {
        __syncthreads();
        const int n = sh.n_list;
        if (tid == 0) sh.bin = n ? atomicAdd(remote(&sh.n_all, 0), n) : 0;
        __syncthreads();
        u64* to = remote(&sh.all[0], 0) + sh.bin;
        if (n <= kList && sh.bin + n <= kList)
            for (int i = tid; i < n; i += kThreads) to[i] = sh.list[i];
        sync_row();
        return *remote(&sh.n_all, 0);
    };
    // Sorts the n entries of `all`, ascending.  bin_of is monotone: entries are spread over kBuckets bins and ranked inside
    // theirs by counting; where a bin gets more than 64 (equal logits), by the sorting network, which takes eight times as long.
    auto sort_all = [&](int n, auto&& bin_of) {
        uint32_t *cnt = sh.bucket_n, *pre = sh.bucket_0;
        for (int i = tid; i < kBuckets; i += kThreads) cnt[i] = 0;
        __syncthreads();
        u64 x[4]; int bin[4]; uint32_t slot[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = tid + j * kThreads;
            bin[j] = -1;
            if (i < n) { x[j] = sh.all[i]; bin[j] = max(0, min(kBuckets - 1, bin_of(x[j]))); slot[j] = atomicAdd(&cnt[bin[j]], 1u); }
        }
        __syncthreads();
        const uint32_t c0 = cnt[2 * tid], c1 = cnt[2 * tid + 1];
        if (__syncthreads_or(max(c0, c1) > 64)) {
            for (int i = n + tid; i < kList; i += kThreads) sh.all[i] = ~0ull;
            __syncthreads();
            sort_list(sh.all);
            return;
        }
        u64 tot;
        const uint32_t e = (uint32_t)block_excl<u64>(c0 + c1, sh.scan, tot);
        pre[2 * tid] = e; pre[2 * tid + 1] = e + c0;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) if (bin[j] >= 0) sh.all[pre[bin[j]] + slot[j]] = x[j];
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (bin[j] >= 0) {
                const uint32_t lo = pre[bin[j]], m = cnt[bin[j]];
                uint32_t before = 0;
                for (uint32_t i = 0; i < m; ++i) before += sh.all[lo + i] < x[j];
                slot[j] = lo + before;
            }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) if (bin[j] >= 0) sh.all[slot[j]] = x[j];
        __syncthreads();
    };
    auto by_value = [&](float from, float to) {               // bins over the logits from `from` down to `to`
        const float inv = from > to && to > -INFINITY ? (float)(kBuckets - 1) / (from - to) : 0.f;
        return [from, inv](u64 a) { return (int)fminf((from - value_of((uint32_t)(a >> 32))) * inv, (float)kBuckets); };
    };
    auto by_index = [&](u64 a) { return (int)(a >> 32) / ((p.vocab + kBuckets - 1) / kBuckets); };
    // Few entries (n <= kFew) are ranked by counting (64 to 256 as a limit measure alike; counting 400 took 12 us more than
    // sorting them).  Thread (i, part) compares entry i with every parts-th entry: `rank` and
    // few_sum get the number and the weight of the entries before it.  All threads call it; few_w holds the weights after.
    const auto few = [&](int n, int& i, bool& mine) {
        const int n2 = n <= 64 ? 64 : 128;
        i = tid & (n2 - 1);
        const int part = tid / n2;
        mine = part == 0 && i < n;
        if (tid < n2) { sh.rank[tid] = 0; sh.few_sum[tid] = 0; sh.few_w[tid] = tid < n ? weight(r, value_of((uint32_t)(sh.all[tid] >> 32))) : 0; }
        if (tid < 2) sh.few_total[tid] = 0;
        __syncthreads();
        if (i < n) {
            const u64 a = sh.all[i];
            uint32_t before = 0; u64 sum = 0;
            for (int j = part; j < n; j += kThreads / n2)
                if (sh.all[j] < a) { ++before; sum += sh.few_w[j]; }
            if (before) { atomicAdd(&sh.rank[i], before); atomicAdd(&sh.few_sum[i], sum); }
        }
        __syncthreads();
    };

    // ---- few candidates
    if ((use_k && k <= kListK) || (!use_k && !use_p && r.x_min > -INFINITY)) {
        float tau = r.max - kRange * (1.f + kSlack) * temperature - fabsf(r.max) * kSlack;      // below it weights are zero
        if (use_k) {
            const float inv = r.inv_bin * ((float)(kCoarse - 1) / (float)(kBins - 1));
            const float tm[4] = {tmax.x, tmax.y, tmax.z, tmax.w};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const float d = (r.max - tm[c]) * inv;
                if (d < (float)(kCoarse - 1)) atomicAdd(&sh.coarse[(int)d], 1u);
            }
            sync_row();
            u64 c = 0, tot;
            for (int q = 0; q < CL; ++q) c += remote(&sh.coarse[0], q)[tid];
            const u64 e = block_excl<u64>(c, sh.scan, tot);
            if (e < (u64)k && e + c >= (u64)k) sh.zone_a = tid;
            __syncthreads();
            if (tot >= (u64)k) {                              // so at least k logits are above the far edge of that bin
                const float t2 = r.max - ((float)(sh.zone_a + 1) * (1.f + kSlack)) / inv - fabsf(r.max) * kSlack;
                if (t2 > tau) tau = t2;                       // (an infinite or undefined edge leaves tau)
            }
        }
        if (!use_p && r.x_min > tau) tau = r.x_min;
        each_batch([&](int v, const float4* q, auto n) {
            unsigned hit = 0;
#pragma unroll
            for (int i = 0; i < decltype(n)::value; ++i) {
                const float e[4] = {q[i].x, q[i].y, q[i].z, q[i].w};
#pragma unroll
                for (int c = 0; c < 4; ++c) if (e[c] >= tau && e[c] > -INFINITY) hit |= 1u << (4 * i + c);
            }
            append(hit, v, q);
        });
        const int n = gather();
        sync_row();                                           // everybody has read it: from here the first block needs no other
        if (n <= kList) {
            if (rank != 0) return;
            if (n <= kFew) {
                int i; bool mine;
                few(n, i, mine);
                const u64 a = i < n ? sh.all[i] : 0, w = i < n ? sh.few_w[i] : 0;
                const bool in_k = i < n && (!use_k || sh.rank[i] < (uint32_t)k);
                u64 s = warp_sum(mine && in_k ? w : 0);
                if (lane == 0 && s) atomicAdd(&sh.few_total[0], s);
                __syncthreads();
                // kept: entries whose predecessors' weight is below the reach
                const bool in = in_k && (!use_p || sh.few_sum[i] < reach(sh.few_total[0])) && value_of((uint32_t)(a >> 32)) >= r.x_min;
                s = warp_sum(mine && in ? w : 0);
                if (lane == 0 && s) atomicAdd(&sh.few_total[1], s);
                __syncthreads();
                if (mine) { sh.few_sum[i] = 0; if (!in) sh.few_w[i] = 0; }
                __syncthreads();
                const u64 Z = sh.few_total[1], target = __umul64hi(Z, U);
                const int n2 = n <= 64 ? 64 : 128;
                if (in) {                                     // the kept weight in front of the entry, in index order
                    u64 sum = 0;
                    for (int j = tid / n2; j < n; j += kThreads / n2)
                        if ((uint32_t)sh.all[j] < (uint32_t)a) sum += sh.few_w[j];
                    if (sum) atomicAdd(&sh.few_sum[i], sum);
                }
                __syncthreads();
                if (mine && in && sh.few_sum[i] <= target && sh.few_sum[i] + w > target) store((int)(uint32_t)a, value_of((uint32_t)(a >> 32)), Z);
                return;
            }
            sort_all(n, by_value(r.max, tau));
            // four consecutive places a thread, in descending order of logits
            u64* wt = sh.list;
            u64 w4[4], mine = 0, tot;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int i = tid * 4 + j;
                w4[j] = i < n && (!use_k || i < k) ? weight(r, value_of((uint32_t)(sh.all[i] >> 32))) : 0;
                mine += w4[j];
            }
            u64 cum = block_excl<u64>(mine, sh.scan, tot);
            const u64 lim = use_p ? reach(tot) : ~0ull;       // kept: places whose predecessors' weight is below the reach
            u64 ksum = 0;
            uint32_t idx4[4];
            int kept = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int i = tid * 4 + j;
                const u64 a = i < n ? sh.all[i] : 0;
                const bool in = cum < lim && value_of((uint32_t)(a >> 32)) >= r.x_min;
                cum += w4[j];
                if (!in) w4[j] = 0;
                idx4[j] = (uint32_t)a;
                ksum += w4[j];
                kept += w4[j] > 0;
                if (i < kList) wt[i] = w4[j];
            }
            u64 Z;
            block_excl<u64>(ksum, sh.scan, Z);                // (its barriers also separate the reads of `all` from the writes below)
            // in index order: (index, place) of what is kept
            u64 kn;
            int at = (int)block_excl<u64>((u64)kept, sh.scan, kn);
#pragma unroll
            for (int j = 0; j < 4; ++j) if (w4[j] > 0) sh.all[at++] = (u64)idx4[j] << 32 | (uint32_t)(tid * 4 + j);
            sort_all((int)kn, by_index);
            const u64 target = __umul64hi(Z, U);
            mine = 0;
            u64 s4[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) { const int i = tid * 4 + j; s4[j] = i < (int)kn ? wt[(uint32_t)sh.all[i]] : 0; mine += s4[j]; }
            cum = block_excl<u64>(mine, sh.scan, tot);
            if (cum <= target && cum + mine > target) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (cum <= target && cum + s4[j] > target) {
                        const int tok = (int)(sh.all[tid * 4 + j] >> 32);     // its slice may be another block's: the logit from global memory
                        store(tok, (float)reinterpret_cast<const E*>(p.logits)[row * p.row_stride + tok], Z);
                    }
                    cum += s4[j];
                }
            }
            return;
        }
        if (tid == 0) { sh.n_list = 0; if (rank == 0) sh.n_all = 0; }
        sync_row();
    }

    // ---- whole distributions
    int za = 0, zb = kBins;                                   // bins that may hold the last threshold: elements before them are kept
    bool searched = false;                                    // za, zb hold a zone
    u64 ws = 0;                                               // weight of this warp's kept elements (before bin za, once searched)
    auto kept = [&](float x, int idx) {
        const uint32_t key = key_of(x);
        return x >= r.x_min && (key < thr || (key == thr && idx <= cut));
    };
    // the weights before bin za (`above`; into ws those that min-p keeps) and, with sum_all, of all; `inside` gets every
    // quad with a bit set for its elements of bins [za, zb], all lanes together.  No branch around the polynomials, four at a time: their chain is long.
    auto weigh = [&](bool sum_all, u64& above, u64& whole, auto&& inside) {
        const float fa = (float)za, fb = (float)(zb + 1), stop = sum_all ? (float)(kBins - 1) : fa;
        const bool with_min = r.x_min > -INFINITY;
        above = whole = ws = 0;
        unsigned n_above = 0, n_whole = 0, n_ws = 0;
        each([&](int v, const float4& q) {
            const float e[4] = {q.x, q.y, q.z, q.w};
            const float d[4] = {(r.max - q.x) * r.inv_bin, (r.max - q.y) * r.inv_bin, (r.max - q.z) * r.inv_bin, (r.max - q.w) * r.inv_bin};
            const float dm = fminf(fminf(d[0], d[1]), fminf(d[2], d[3]));
            if (dm < stop) {
                u64 w[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) w[c] = weight_bits(r, e[c]);
                if (sum_all) { whole += (w[0] + w[1]) + (w[2] + w[3]); n_whole += 4; }
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (d[c] < fa) {
                        above += w[c]; ++n_above;
                        if (with_min && e[c] >= r.x_min) { ws += w[c]; ++n_ws; }
                    }
            }
            unsigned in = 0;
#pragma unroll
            for (int c = 0; c < 4; ++c) if (d[c] >= fa && d[c] < fb) in |= 1u << c;
            inside(in, v, &q);
        });
        above -= n_above * kOffset; whole -= n_whole * kOffset; ws -= n_ws * kOffset;
        if (!with_min) ws = above;
        ws = warp_sum(ws);
        above = warp_sum(above); whole = warp_sum(whole);
        if (lane == 0) { sh.warp_tmp[warp] = above; sh.warp_tmp2[warp] = whole; }
        __syncthreads();
        if (tid == 0) { u64 s = 0, q = 0; for (int w = 0; w < kWarps; ++w) { s += sh.warp_tmp[w]; q += sh.warp_tmp2[w]; } sh.blk_mass = s; sh.blk_all = q; }
    };
    auto row_sum = [&](u64 Shared::*field) { u64 s = 0; for (int q = 0; q < CL; ++q) s += remote(&sh, q)->*field; return s; };

    bool by_keys = false;
    u64 above_cnt = 0;                                        // elements of the row before bin za
    int k_bin = -1;                                           // bin of the k-th element, with k_before elements before it
    u64 k_before = 0;
    if (use_k || use_p) {
        for (int i = tid; i < kBins / 4; i += kThreads) reinterpret_cast<uint4*>(sh.bins)[i] = make_uint4(0, 0, 0, 0);
        __syncthreads();
        each([&](int, float4 q) {
            const float d[4] = {(r.max - q.x) * r.inv_bin, (r.max - q.y) * r.inv_bin, (r.max - q.z) * r.inv_bin, (r.max - q.w) * r.inv_bin};
#pragma unroll
            for (int c = 0; c < 4; ++c) if (d[c] < (float)(kBins - 1)) atomicAdd(&sh.bins[(int)d[c]], 1u);
        });
        sync_row();
        // every block sums its share of the bins over the blocks: `per` of them a thread.  An element of bin b weighs between
        // e^-(b + 1)d and e^-bd (a hundredth of a bin more on either side for the rounding of its number), and its whole
        // number of units, which is what decides, lies up to half a unit outside (kHalf; the exponential's last bits are
        // relative, below).  Every one of many equal logits is rounded the same way: without it a reach within 1e-6 of 1
        // had its threshold in another bin than the bounds said.
        constexpr float kUnit = 0x1p-44f, kHalf = 0.5625f * kUnit;
        const int per = kBins / kThreads / CL, b0 = rank * (kBins / CL) + tid * per;
        const float d = kRange / (kBins - 1), step = __expf(-d);
        BinSum in{0, 0., 0.}, tot;
        {
            float fu = __expf(-d * ((float)b0 - 0.01f)), fd = __expf(-d * ((float)b0 + 1.01f));
#pragma unroll 1
            for (int b = b0; b < b0 + per; ++b) {
                uint32_t c = 0;
#pragma unroll
                for (int q = 0; q < (CLUSTER ? kMaxCluster : 1); ++q) if (q < CL) c += remote(&sh.bins[0], q)[b];
                if (CLUSTER) sh.bins[b] = c;                  // (no other block reads this block's own share here)
                in.n += c; in.up += (double)((float)c * (fu + kHalf)); in.dn += (double)((float)c * fmaxf(fd - kHalf, 0.f));
                fu *= step; fd *= step;
            }
        }
        const BinSum before = block_excl_bins(in, sh.bin_scan, tot);
        u64 tc = tot.n, ec = before.n; double tu = tot.up, td = tot.dn, eu = before.up, el = before.dn;
        if (tid == 0) { sh.share[0] = (double)tc; sh.share[1] = tu; sh.share[2] = td; sh.zone_a = sh.zone_b = sh.tail_a = sh.tail_b = kBins - 2; sh.bin = -1; sh.before_cnt = 0; }
        sync_row();
        tc = 0; tu = td = 0;
        for (int q = 0; q < CL; ++q) {
            const double* s = remote(&sh.share[0], q);
            if (q < rank) { ec += (u64)s[0]; eu += s[1]; el += s[2]; }
            tc += (u64)s[0]; tu += s[1]; td += s[2];
        }
        // (1e-5: the rounding of the bounds themselves, a product of up to 16 steps and a sum; a unit: the reach is a whole number)
        // The threshold lies in the first bin through which the weight reaches p times the whole, or, the same, behind which
        // at most 1 - p of it is left: both bounds are taken, the smaller part is the sharper one.
        const double t_lo = td * tp * (1 - 1e-5) - kUnit, t_hi = tu * tp * (1 + 1e-5) + kUnit;
        const double s_lo = td * (1.0 - (double)tp) * (1 - 1e-5) - kUnit, s_hi = tu * (1.0 - (double)tp) * (1 + 1e-5) + kUnit;
        // A bin is where a sum passes its limit if the sum before it does not and the sum through it does.  A thread's first sum
        // comes from the scan and the last of the thread before it from that thread: `eps`, far above their difference (1e-14
        // of the whole) and far below the 1e-5, keeps the passing from falling between the two.
        const double eps = 1e-11 * tu;
        float fu = __expf(-d * ((float)b0 - 0.01f)), fd = __expf(-d * ((float)b0 + 1.01f));
        const bool k_cuts = use_k && tc > (u64)k;             // otherwise top-k removes nothing that has weight
#pragma unroll 1
        for (int b = b0; b < b0 + per; ++b) {
            const uint32_t c = sh.bins[b];
            const double u1 = (double)((float)c * (fu + kHalf)), l1 = (double)((float)c * fmaxf(fd - kHalf, 0.f));
            if (k_cuts && ec < (u64)k && ec + c >= (u64)k)
                for (int q = 0; q < CL; ++q) { Shared* o = remote(&sh, q); o->bin = b; o->before_cnt = ec; }
            if (use_p && eu - eps < t_lo && eu + u1 >= t_lo) for (int q = 0; q < CL; ++q) atomicMin(&remote(&sh, q)->zone_a, b);
            if (use_p && el - eps < t_hi && el + l1 >= t_hi) for (int q = 0; q < CL; ++q) atomicMin(&remote(&sh, q)->zone_b, b);
            if (use_p && td - el + eps > s_hi && td - (el + l1) <= s_hi) for (int q = 0; q < CL; ++q) atomicMin(&remote(&sh, q)->tail_a, b);
            if (use_p && tu - eu + eps > s_lo && tu - (eu + u1) <= s_lo) for (int q = 0; q < CL; ++q) atomicMin(&remote(&sh, q)->tail_b, b);
            ec += c; eu += u1; el += l1;
            fu *= step; fd *= step;
        }
        sync_row();
        if (k_cuts) { k_bin = sh.bin; k_before = sh.before_cnt; }
        if (use_p && k_bin < 0) {
            const int ta = td <= s_hi ? 0 : sh.tail_a;        // already at most 1 - p before the first bin
            za = max(sh.zone_a, ta); zb = min(sh.zone_b, sh.tail_b);
            if (za > zb) { za = min(sh.zone_a, ta); zb = max(sh.zone_b, sh.tail_b); }
            searched = true;
        } else if (k_bin >= 0 && !use_p) {
            za = zb = k_bin; above_cnt = k_before;
            searched = true;
        } else by_keys = k_bin >= 0;                          // top-p behind a top-k that cuts
        __syncthreads();
    }

    u64 above, whole;
    if (!by_keys) {
        // ---- one pass: exact weights, and a list of the zone (without a filter: everything is kept)
        if (!searched && r.x_min == -INFINITY) {              // no filter: everything is kept (309 to 230 us for 1000 x 128000)
            ws = 0;
            unsigned n = 0;
            each([&](int, const float4& q) {
                if (fmaxf(fmaxf(q.x, q.y), fmaxf(q.z, q.w)) > r.x_zero) {
                    ws += (weight_bits(r, q.x) + weight_bits(r, q.y)) + (weight_bits(r, q.z) + weight_bits(r, q.w));
                    n += 4;
                }
            });
            ws = warp_sum(ws - n * kOffset);
        } else {
            if (!searched) { za = kBins; zb = kBins - 1; }
            weigh(use_p || !searched, above, whole, append);
        }
        if (lane == 0) remote(&sh.wsum[0], 0)[rank * kWarps + warp] = ws;
        const int n = searched ? gather() : 0;
        if (!searched) sync_row();
        by_keys = n > kList;
        if (!by_keys && searched && rank == 0) {
            const u64 above_mass = row_sum(&Shared::blk_mass);
            const u64 need = use_p ? reach(row_sum(&Shared::blk_all)) : 0;
            // entry `place` of the zone, `cum` the weight before it: in front of the threshold, on it, or behind
            auto decide = [&](u64 a, int place, u64 w, u64 cum) {
                const bool in = use_p ? cum < need : above_cnt + place < (u64)k;
                const bool last = in && (use_p ? cum + w >= need : above_cnt + place + 1 == (u64)k);
                const uint32_t key = (uint32_t)(a >> 32);
                const int idx = (int)(uint32_t)a;
                if (last) { sh.thr = key; sh.cut = idx; }
                if (in && value_of(key) >= r.x_min) {         // into the sum of the warp that owns it
                    const int q = idx / slice, i2 = idx - q * slice + shift;
                    const int qc = min(slice, p.vocab - q * slice), pw = (((qc + shift + 3) >> 2) + kWarps - 1) / kWarps;
                    atomicAdd(&sh.wsum[q * kWarps + (i2 >> 2) / pw], w);
                }
            };
            if (n <= kFew) {
                int i; bool mine;
                few(n, i, mine);
                if (mine) decide(sh.all[i], (int)sh.rank[i], sh.few_w[i], sh.few_sum[i] + above_mass);
            } else {
                sort_all(n, by_value(r.max - (float)za / r.inv_bin, r.max - (float)(zb + 1) / r.inv_bin));
                u64 w4[4], mine = 0, tot;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int i = tid * 4 + j;
                    w4[j] = i < n ? weight(r, value_of((uint32_t)(sh.all[i] >> 32))) : 0;
                    mine += w4[j];
                }
                u64 cum = block_excl<u64>(mine, sh.scan, tot) + above_mass;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int i = tid * 4 + j;
                    if (i < n) decide(sh.all[i], i, w4[j], cum);
                    cum += w4[j];
                }
            }
            __syncthreads();
            thr = sh.thr; cut = sh.cut;
        }
    }
    if (by_keys) {
        // ---- narrowing by keys.  Narrows (thr, cut) to the prefix whose count (by_mass false) or weight (true) first reaches
        // `target`, searching the elements of bins [za, zb] that are kept so far; `before` elements lie in earlier bins, all
        // kept.  By weight the target is the reach of top-p in the weight of everything kept so far: of `target` where that is
        // known, else of the sum that the first pass takes.  Returns the weight of the new prefix.
        auto refine = [&](bool by_mass, u64 before, u64 target, bool whole_known) -> u64 {
            // keys that the zone can hold: its distances, widened by the rounding of the subtraction and the product
            const float hi = za <= 0 ? r.max : r.max - ((float)za * (1.f - kSlack)) / r.inv_bin + fabsf(r.max) * kSlack;
            const float lo = r.max - ((float)(zb + 1) * (1.f + kSlack)) / r.inv_bin - fabsf(r.max) * kSlack;
            uint32_t klo = key_of(hi < r.max ? hi : r.max), khi = lo > -INFINITY ? key_of(lo) : 0xff800000u;   // the key of -inf is the largest used
            int shf = 0;
            while ((((uint64_t)khi - klo) >> shf) >= kFine) ++shf;
            u64 above_mass = 0;
            for (bool first = true;; first = false) {
                __syncthreads();
                for (int i = tid; i < kFine; i += kThreads) { sh.hist[i] = 0; sh.mass[i] = 0; }
                __syncthreads();
                auto inside = [&](float x, int idx) {
                    const uint32_t key = key_of(x);
                    if (key > thr || (key == thr && idx > cut) || key < klo || key > khi) return;
                    const int f = (int)((key - klo) >> shf);
                    if (f >= kFine) return;
                    atomicAdd(&sh.hist[f], 1u);
                    atomicAdd(&sh.mass[f], weight(r, x));
                };
                if (first)
                    weigh(by_mass && !whole_known, above, whole, [&](unsigned in, int v, const float4* q) {
                        const float e[4] = {q->x, q->y, q->z, q->w};
#pragma unroll
                        for (int c = 0; c < 4; ++c) if (in >> c & 1) inside(e[c], base + v * 4 + c);
                    });
                else {
                    const float fa = (float)za, fb = (float)(zb + 1);
                    for (int v = v0 + lane; v < v1; v += 32) {
                        const float4 q = get(v);
                        const float e[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                        for (int c = 0; c < 4; ++c) { const float d = (r.max - e[c]) * r.inv_bin; if (d >= fa && d < fb) inside(e[c], base + v * 4 + c); }
                    }
                }
                sync_row();
                constexpr int PB = kFine / kThreads;          // bins of this thread
                uint32_t cb[PB] = {}; u64 mb[PB] = {};
                for (int q = 0; q < CL; ++q)
#pragma unroll
                    for (int j = 0; j < PB; ++j) { cb[j] += remote(&sh.hist[0], q)[tid * PB + j]; mb[j] += remote(&sh.mass[0], q)[tid * PB + j]; }
                if (first) {
                    above_mass = row_sum(&Shared::blk_mass);
                    if (by_mass) target = reach(whole_known ? target : row_sum(&Shared::blk_all));
                }
                sync_row();                                   // everybody has read: the arrays may be overwritten
                u64 tot_c, tot_m, sc = 0, sm = 0;
#pragma unroll
                for (int j = 0; j < PB; ++j) { sc += cb[j]; sm += mb[j]; }
                u64 ec = block_excl<u64>(sc, sh.scan, tot_c) + before, em = block_excl<u64>(sm, sh.scan, tot_m) + above_mass;
                if (tid == 0) sh.bin = -1;
                __syncthreads();
#pragma unroll
                for (int j = 0; j < PB; ++j) {
                    const u64 e0 = by_mass ? em : ec, a = by_mass ? mb[j] : (u64)cb[j];
                    if (e0 < target && e0 + a >= target) { sh.bin = tid * PB + j; sh.before_cnt = ec; sh.before_mass = em; sh.total = cb[j]; }
                    ec += cb[j]; em += mb[j];
                }
                __syncthreads();
                if (sh.bin < 0) return above_mass + tot_m;    // everything kept so far is needed: no narrower threshold
                before = sh.before_cnt; above_mass = sh.before_mass;
                const uint32_t nlo = klo + ((uint32_t)sh.bin << shf);
                const u64 in_bin = sh.total;
                __syncthreads();
                if (shf == 0) {                               // one key: of its `in_bin` elements the first `take` by index
                    const u64 w = weight(r, value_of(nlo));
                    u64 take = in_bin;
                    if (!by_mass) take = target - before;
                    else if (w > 0) take = (target - above_mass + w - 1) / w;
                    const uint32_t old_thr = thr; const int old_cut = cut;
                    thr = nlo;
                    if (take >= in_bin) { cut = old_thr == thr ? old_cut : 0x7fffffff; return above_mass + in_bin * w; }
                    // index of the take-th element with that key: counts by warp, in index order
                    uint32_t mine = 0;
                    for (int v = v0 + lane; v < v1; v += 32) {
                        const float4 q = get(v);
                        mine += (key_of(q.x) == thr) + (key_of(q.y) == thr) + (key_of(q.z) == thr) + (key_of(q.w) == thr);
                    }
                    mine = warp_sum(mine);
                    if (lane == 0) sh.warp_cnt[warp] = mine;
                    sync_row();
                    u64 seen = 0;
                    for (int q = 0; q < CL * kWarps; ++q) {
                        const u64 cq = remote(&sh.warp_cnt[0], q / kWarps)[q % kWarps];
                        if (seen + cq >= take) {
                            if (q / kWarps == rank && q % kWarps == warp) {
                                uint32_t left = (uint32_t)(take - seen);      // 1 .. cq
                                for (int v = v0; v < v1; v += 32) {
                                    uint32_t hit = 0;
                                    if (v + lane < v1) {
                                        const float4 x = get(v + lane);
                                        hit = (key_of(x.x) == thr) | (key_of(x.y) == thr) << 1 | (key_of(x.z) == thr) << 2 | (key_of(x.w) == thr) << 3;
                                    }
                                    const uint32_t incl = warp_incl((uint32_t)__popc(hit)), here = __shfl_sync(0xffffffffu, incl, 31);
                                    if (left <= here) {
                                        uint32_t need = left - (incl - __popc(hit));
                                        if (left > incl - __popc(hit) && left <= incl)
                                            for (int c = 0; c < 4; ++c)
                                                if (hit >> c & 1 && --need == 0)
                                                    for (int z = 0; z < CL; ++z) *remote(&sh.cut, z) = base + (v + lane) * 4 + c;
                                        break;
                                    }
                                    left -= here;
                                }
                            }
                            break;
                        }
                        seen += cq;
                    }
                    sync_row();
                    cut = sh.cut;
                    return above_mass + take * w;
                }
                klo = nlo;
                khi = min(khi, (uint32_t)(klo + ((1u << shf) - 1)));
                shf = 0;
                while ((((uint64_t)khi - klo) >> shf) >= kFine) ++shf;
            }
        };
        u64 kept_mass = 0;
        if (k_bin >= 0) {
            za = zb = k_bin;
            kept_mass = refine(false, k_before, (u64)k, false);
        }
        if (use_p) {
            if (k_bin >= 0) { za = 0; zb = min(kBins - 2, (int)((r.max - value_of(thr)) * r.inv_bin)); }   // anywhere above the k-th
            refine(true, 0, kept_mass, k_bin >= 0);           // (otherwise the zone that the histogram gave)
        }
        // what every warp keeps: before the zone it is known
        const float fa = (float)za, fb = (float)(zb + 1);
        u64 z = 0;
        for (int v = v0 + lane; v < v1; v += 32) {
            const float4 q = get(v);
            const float e[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int c = 0; c < 4; ++c) { const float d = (r.max - e[c]) * r.inv_bin; if (d >= fa && d < fb && kept(e[c], base + v * 4 + c)) z += weight(r, e[c]); }
        }
        z = warp_sum(z);
        if (lane == 0) remote(&sh.wsum[0], 0)[rank * kWarps + warp] = ws + z;
        sync_row();
    }

    draw([&](u64 Z) { return Z; }, [&](float x, int idx) { return kept(x, idx) ? weight(r, x) : 0ull; },
         [&](int tok, float x, u64 Z) { store(tok, x, Z); });
}

template <class E, bool CLUSTER, bool HELD>
pt_status launch_kind(const SampleP& p, int64_t n, int cl, cudaStream_t st) {
    const int slice = ((p.vocab + cl - 1) / cl + 3) & ~3;
    const size_t head = (sizeof(Shared) + 15) & ~15;
    static bool done_[kMaxDevices] = {};
    bool& done = done_[current_device()];
    if (!done) {
        cudaError_t e = cudaFuncSetAttribute(k_sample<E, CLUSTER, HELD>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(head + (HELD ? (kMaxSlice + 4) * 4 : 0)));
        if (e != cudaSuccess) { set_error("cudaFuncSetAttribute: %s", cudaGetErrorString(e)); return PT_ERR_CUDA; }
        done = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(n * cl)); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = head + (HELD ? (size_t)(slice + 4) * 4 : 0); cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension; at[0].val.clusterDim.x = cl; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    cfg.attrs = at; cfg.numAttrs = CLUSTER ? 1 : 0;
    cudaError_t e = cudaLaunchKernelEx(&cfg, k_sample<E, CLUSTER, HELD>, p, slice);
    if (e != cudaSuccess) { set_error("k_sample launch: %s", cudaGetErrorString(e)); return PT_ERR_CUDA; }
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return PT_OK;
}

template <class E>
pt_status launch_t(const SampleP& p, int64_t n, cudaStream_t st) {
    // Clusters while all of their blocks are resident, two on an SM: up to 8 blocks for a row, one per 4096 logits, or 4 where
    // 8 are too many.  With 2 a row a cluster only broke even, so then, and for more rows, a block takes a row.  Measured with
    // top-k 50 / top-p 0.9 in us, cluster against row: 24 x 32000 11.7 / 23.6 against 12.7 / 31.0, 24 x 128000 15.6 / 39.0 against
    // 19.5 / 80.3, 64 x 32000 13.8 / 28.2 against 13.3 / 31.0, 64 x 128000 18.8 / 52.4 against 20.3 / 80.0; by twos 100 x 64000
    // 18.5 / 52.7 against 16.4 / 49.3.
    const int64_t slots = 2 * 148;
    int cl = 1;
    while (cl < kMaxCluster && (int64_t)cl * 4096 < p.vocab) cl *= 2;
    if (cl == kMaxCluster && n * cl > slots) cl = kMaxCluster / 2;
    else if (n * cl <= slots) {
        // slices of at most 16384 logits (64 KB: two blocks per SM); while a launch leaves SMs idle a row is spread further,
        // down to slices of 2048
        const int most = cl;
        for (cl = 1; cl < most && ((p.vocab + cl - 1) / cl > 16384 || (n * cl * 2 <= 148 && (p.vocab + cl - 1) / cl > 2048));) cl *= 2;
    }
    if (n * cl > slots) return launch_kind<E, false, false>(p, n, 1, st);
    // longer slices are held where an SM has one block anyway, else they are streamed as well (64 x 128000 by fours: held
    // 28.0 / 76.5)
    const int slice = (p.vocab + cl - 1) / cl;
    if (slice <= 16384 || (slice <= kMaxSlice && n * cl <= 148)) return launch_kind<E, true, true>(p, n, cl, st);
    return launch_kind<E, true, false>(p, n, cl, st);
}

}  // namespace

int sample_vocab_limit() { return kMaxVocab; }

pt_status launch_sample(const SampleP& p, int64_t n, bool bf16, cudaStream_t st) {
    return bf16 ? launch_t<__nv_bfloat16>(p, n, st) : launch_t<float>(p, n, st);
}

}  // namespace pt

using namespace pt;

extern "C" pt_status pt_sample(const void* logits, int32_t dtype, int64_t row_stride, int64_t n, int32_t vocab, const float* u,
                               const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                               int32_t* token, float* prob, void* stream) {
    if (!logits || !u || !token) { set_error("null argument"); return PT_ERR_INVALID_ARG; }
    if (dtype != PT_F32 && dtype != PT_BF16) { set_error("dtype must be PT_F32 or PT_BF16"); return PT_ERR_INVALID_ARG; }
    if (n < 1 || n > (1 << 24) || vocab < 1 || row_stride < vocab) { set_error("n outside [1, 2^24], vocab < 1 or row_stride < vocab"); return PT_ERR_INVALID_ARG; }
    if (vocab > sample_vocab_limit()) { set_error("vocab %d > %d", vocab, sample_vocab_limit()); return PT_ERR_UNSUPPORTED; }
    if ((uintptr_t)logits % (dtype == PT_F32 ? 4 : 2) || ((uintptr_t)u | (uintptr_t)temperature | (uintptr_t)top_k | (uintptr_t)top_p | (uintptr_t)min_p | (uintptr_t)token | (uintptr_t)prob) % 4) {
        set_error("the arrays must be aligned to their types"); return PT_ERR_MISALIGNED;
    }
    SampleP p{};
    p.logits = logits; p.row_stride = row_stride; p.vocab = vocab; p.u = u;
    p.temperature = temperature; p.top_k = top_k; p.top_p = top_p; p.min_p = min_p;
    p.token = token; p.prob = prob; p.prob_stride = 1;
    return launch_sample(p, n, dtype == PT_BF16, (cudaStream_t)stream);
}
