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
// the order of atomics changes a result, and ties at a threshold are exact.  A weight below 2^-45 (31 nats under the
// maximum) is zero: such a token is never drawn.  The exponential is evaluated in double; the multiple rounds it once,
// an absolute error of 2^-45 against a sum of at least 1.
//
// One cluster of CL blocks takes a row (CL = 1 for short rows): each block reads its slice from global memory once and
// keeps it in shared memory; everything after that runs there, and the blocks exchange histograms through distributed
// shared memory.  A threshold is found by radix selection: a histogram of the distance to the maximum (counts alone
// bound the cumulative weight within a bin's width), then histograms with exact counts and weights over the few bins
// that may hold the threshold, down to a single key.
#include <cooperative_groups.h>

#include "pt_internal.h"
#include "pt_sample.h"

namespace cg = cooperative_groups;

namespace pt {

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBins = 2048;                    // first histogram: distance to the maximum
constexpr int kFine = 1024;                    // later histograms: keys
constexpr int kFracBits = 44;
constexpr float kRange = 31.5f;                // nats below the maximum that the bins cover; beyond it weights are zero
constexpr int kMaxCluster = 8;
constexpr int kMaxSlice = 49152;               // elements of a slice: 192 KB

typedef unsigned long long u64;

// Distance-ordered key: smaller key = larger value.  -0 and +0 are one value.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);
    return (b & 0x80000000u) ? b : ~b & 0x7fffffffu;
}

struct Row {
    float max, inv_bin;                        // bin of x = (max - x) * inv_bin
    double inv_t;                              // log2(e) / temperature
    float x_min;                               // min-p: kept values are >= x_min
};

// w(x) * 2^44, rounded to the nearest whole number
__device__ __forceinline__ u64 weight(const Row& r, float x) {
    if (x == r.max) return 1ull << kFracBits;  // also for an infinite maximum, whose distance to itself has no value
    const double t = ((double)x - (double)r.max) * r.inv_t;
    if (!(t > -46.0)) return 0;
    return (u64)__double2ull_rn(exp2(t + (double)kFracBits));
}
__device__ __forceinline__ int bin_of(const Row& r, float x) {
    if (x == r.max) return 0;
    const float d = (r.max - x) * r.inv_bin;
    return d < (float)(kBins - 1) ? (int)d : kBins - 1;      // also for an infinite distance
}

struct Shared {
    uint32_t hist[kBins];
    u64 mass[kFine];
    float red[kWarps];
    int redi[kWarps];
    u64 warp_sum[kWarps];                      // weight kept by each warp's part of the slice
    uint32_t warp_cnt[kWarps];
    u64 blk_mass;                              // weight of this block's elements above the searched bins
    u64 scan[kWarps + 1];
    double dscan[kWarps + 1];
    float max;
    int arg;
    // found by a scan
    int bin;
    u64 before_mass, before_cnt, total;
    int zone_a, zone_b;
    int cut;
    int token;
};

template <class V> __device__ __forceinline__ V warp_incl(V v) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const V u = __shfl_up_sync(0xffffffffu, v, o); if (lane >= o) v += u; }
    return v;
}
// exclusive prefix of v over the block's threads; *total = the block's sum.  buf holds kWarps + 1 values.
template <class V> __device__ __forceinline__ V block_excl(V v, V* buf, V* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const V incl = warp_incl(v);
    __syncthreads();
    if (lane == 31) buf[warp] = incl;
    __syncthreads();
    if (warp == 0) {
        V w = lane < kWarps ? buf[lane] : V(0);
        const V wi = warp_incl(w);
        if (lane < kWarps) buf[lane] = wi - w;
        if (lane == kWarps - 1) buf[kWarps] = wi;
    }
    __syncthreads();
    *total = buf[kWarps];
    return buf[warp] + incl - v;
}

template <class E>
__global__ void __launch_bounds__(kThreads)
k_sample(const SampleP p, const int slice) {
    extern __shared__ __align__(16) unsigned char smem_raw[];
    Shared& sh = *reinterpret_cast<Shared*>(smem_raw);
    float* xs = reinterpret_cast<float*>(smem_raw + ((sizeof(Shared) + 15) & ~15));
    cg::cluster_group cluster = cg::this_cluster();
    const int CL = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int64_t row = blockIdx.x / CL;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int base = rank * slice;
    const int count = max(0, min(slice, p.vocab - base));
    const E* src = reinterpret_cast<const E*>(p.logits) + row * p.row_stride + base;
    const int per_warp = (count + kWarps - 1) / kWarps;       // every warp owns a contiguous part of the slice
    const int w0 = min(count, warp * per_warp), w1 = min(count, w0 + per_warp);

    // ---- the slice, and the maximum with its lowest index (NaN counts as masked)
    float best = -INFINITY; int arg = 0x7fffffff;
    for (int i = tid; i < count; i += kThreads) {
        float x = (float)src[i];
        if (!(x == x)) x = -INFINITY;
        xs[i] = x;
        if (x > best) { best = x; arg = base + i; }
    }
    auto better = [](float v, int i, float bv, int bi) { return v > bv || (v == bv && i < bi); };
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const float v = __shfl_xor_sync(0xffffffffu, best, o); const int i = __shfl_xor_sync(0xffffffffu, arg, o);
        if (better(v, i, best, arg)) { best = v; arg = i; }
    }
    if (lane == 0) { sh.red[warp] = best; sh.redi[warp] = arg; }
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < kWarps; ++w) if (better(sh.red[w], sh.redi[w], best, arg)) { best = sh.red[w]; arg = sh.redi[w]; }
        sh.max = best; sh.arg = arg;
    }
    cluster.sync();
    best = -INFINITY; arg = 0x7fffffff;
    for (int r = 0; r < CL; ++r) {
        const Shared* o = cluster.map_shared_rank(&sh, r);
        if (better(o->max, o->arg, best, arg)) { best = o->max; arg = o->arg; }
    }
    const float temperature = p.temperature ? p.temperature[row] : 1.0f;
    const bool nothing = best == -INFINITY;                   // every logit masked: token 0, probability 0
    const bool greedy = !(temperature > 0.f && temperature < INFINITY);
    if (nothing || greedy) {
        if (rank == 0 && tid == 0) {
            const int tok = nothing ? 0 : arg;
            if (p.token) p.token[row] = tok;
            if (p.token2) p.token2[row * p.token2_stride] = tok;
            if (p.prob) p.prob[row * p.prob_stride] = nothing ? 0.f : 1.f;
        }
        cluster.sync();                                       // no block leaves while another still reads its maximum
        return;
    }
    Row r;
    r.max = best;
    r.inv_t = 1.4426950408889634 / (double)temperature;
    r.inv_bin = (float)(kBins - 1) / (kRange * temperature);
    r.x_min = -INFINITY;
    if (p.min_p) {
        const float mp = p.min_p[row];
        if (mp > 0.f) r.x_min = mp >= 1.f ? best : __double2float_ru((double)best + (double)temperature * log((double)mp));
    }
    const int k = p.top_k ? p.top_k[row] : 0;
    const float tp = p.top_p ? p.top_p[row] : 1.0f;
    const bool use_k = k > 0 && k < p.vocab, use_p = tp < 1.0f;
    // kept so far: key < thr, or key == thr and index <= cut
    uint32_t thr = 0xffffffffu; int cut = 0x7fffffff;

    // ---- counts by distance to the maximum
    if (use_k || use_p) {
        for (int i = tid; i < kBins; i += kThreads) sh.hist[i] = 0;
        __syncthreads();
        for (int i = tid; i < count; i += kThreads) {
            const int b = bin_of(r, xs[i]);
            if (b < kBins - 1) atomicAdd(&sh.hist[b], 1u);
        }
    }
    // a thread's four bins of the whole row
    uint32_t c4[4] = {0, 0, 0, 0};
    auto row_hist = [&]() {
        cluster.sync();
        for (int q = 0; q < CL; ++q) {
            const uint4 v = *reinterpret_cast<const uint4*>(cluster.map_shared_rank(sh.hist, q) + tid * 4);
            c4[0] += v.x; c4[1] += v.y; c4[2] += v.z; c4[3] += v.w;
        }
        cluster.sync();
    };
    if (use_k || use_p) row_hist();

    // Narrows (thr, cut) to the prefix whose count (by_mass false) or weight (true) first reaches `target`, searching the
    // elements of bins [za, zb] that are kept so far; `above_cnt` elements lie in earlier bins, all kept.  By weight the
    // target is frac64 / 2^64 of the weight of everything kept so far: of `target` where that is known, else of the sum
    // that the first pass takes.  Returns the weight of the new prefix.
    auto refine = [&](bool by_mass, int za, int zb, u64 above_cnt, u64 target, bool whole_known, u64 frac64) -> u64 {
        // keys that the zone can hold: its distances, widened by the rounding of the subtraction and the product
        const float slack = 4e-7f;
        const float hi = za <= 0 ? r.max : r.max - ((float)za * (1.f - slack)) / r.inv_bin + fabsf(r.max) * slack;
        const float lo = r.max - ((float)(zb + 1) * (1.f + slack)) / r.inv_bin - fabsf(r.max) * slack;
        uint32_t klo = key_of(hi < r.max ? hi : r.max), khi = lo > -INFINITY ? key_of(lo) : 0xff800000u;   // the key of -inf is the largest used
        int shift = 0;
        while ((((uint64_t)khi - klo) >> shift) >= kFine) ++shift;
        u64 above_mass = 0;
        bool first = true;
        for (;;) {
            for (int i = tid; i < kFine; i += kThreads) { sh.hist[i] = 0; sh.mass[i] = 0; }
            if (tid == 0) sh.blk_mass = 0;
            __syncthreads();
            u64 am = 0, rest = 0;
            for (int i = tid; i < count; i += kThreads) {
                const float x = xs[i];
                const int b = bin_of(r, x);
                if (b > zb) { if (first && by_mass && !whole_known && b < kBins - 1) rest += weight(r, x); continue; }
                if (b < za) { if (first) am += weight(r, x); continue; }
                const uint32_t key = key_of(x);
                if (key > thr || (key == thr && base + i > cut)) continue;
                if (key < klo || key > khi) continue;
                const int f = (int)((key - klo) >> shift);
                if (f >= kFine) continue;
                atomicAdd(&sh.hist[f], 1u);
                atomicAdd(&sh.mass[f], weight(r, x));
            }
            if (first) {
#pragma unroll
                for (int o = 16; o; o >>= 1) { am += __shfl_xor_sync(0xffffffffu, am, o); rest += __shfl_xor_sync(0xffffffffu, rest, o); }
                if (lane == 0) { sh.warp_sum[warp] = am; sh.scan[warp] = rest; }
                __syncthreads();
                if (tid == 0) { u64 s = 0, q = 0; for (int w = 0; w < kWarps; ++w) { s += sh.warp_sum[w]; q += sh.scan[w]; } sh.blk_mass = s; sh.total = q; }
            }
            cluster.sync();
            uint32_t c2[2] = {0, 0}; u64 m2[2] = {0, 0}, below = 0;
            for (int q = 0; q < CL; ++q) {
                const uint2 c = *reinterpret_cast<const uint2*>(cluster.map_shared_rank(sh.hist, q) + tid * 2);
                const ulonglong2 m = *reinterpret_cast<const ulonglong2*>(cluster.map_shared_rank(sh.mass, q) + tid * 2);
                c2[0] += c.x; c2[1] += c.y; m2[0] += m.x; m2[1] += m.y;
                if (first) { above_mass += *cluster.map_shared_rank(&sh.blk_mass, q); below += *cluster.map_shared_rank(&sh.total, q); }
            }
            cluster.sync();                                   // everybody has read: the arrays may be overwritten
            u64 tot_c, tot_m;
            const u64 ec = block_excl<u64>((u64)c2[0] + c2[1], sh.scan, &tot_c) + above_cnt;
            const u64 em = block_excl<u64>(m2[0] + m2[1], sh.scan, &tot_m) + above_mass;
            if (first && by_mass) {                           // the target from the whole weight
                const u64 whole = whole_known ? target : above_mass + tot_m + below;
                const u64 lo64 = whole * frac64, hi64 = __umul64hi(whole, frac64);
                target = max((u64)1, hi64 + (lo64 != 0));
            }
            if (tid == 0) sh.bin = -1;
            __syncthreads();
            const u64 e0 = by_mass ? em : ec, a0 = by_mass ? m2[0] : (u64)c2[0], a1 = by_mass ? m2[1] : (u64)c2[1];
            if (e0 < target && e0 + a0 + a1 >= target) {
                const int sec = e0 + a0 >= target ? 0 : 1;
                sh.bin = tid * 2 + sec;
                sh.before_cnt = ec + (sec ? c2[0] : 0);
                sh.before_mass = em + (sec ? m2[0] : 0);
                sh.total = sec ? c2[1] : c2[0];
            }
            __syncthreads();
            if (sh.bin < 0) return above_mass + tot_m;        // everything kept so far is needed: no narrower threshold
            above_cnt = sh.before_cnt; above_mass = sh.before_mass;
            const uint32_t nlo = klo + ((uint32_t)sh.bin << shift);
            const u64 in_bin = sh.total;
            __syncthreads();
            if (shift == 0) {                                 // one key: of its `in_bin` elements the first `take` by index
                const float x = __uint_as_float((nlo & 0x80000000u) ? nlo : ~nlo & 0x7fffffffu);
                const u64 w = weight(r, x);
                u64 take = in_bin;
                if (!by_mass) take = target - above_cnt;
                else if (w > 0) take = (target - above_mass + w - 1) / w;
                const bool all = take >= in_bin;
                const uint32_t old_thr = thr; const int old_cut = cut;
                thr = nlo;
                if (all) { cut = old_thr == thr ? old_cut : 0x7fffffff; return above_mass + in_bin * w; }
                // index of the take-th element with that key: counts by warp, in index order
                uint32_t mine = 0;
                for (int i = w0 + lane; i < w1; i += 32) mine += key_of(xs[i]) == thr;
#pragma unroll
                for (int o = 16; o; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
                if (lane == 0) sh.warp_cnt[warp] = mine;
                cluster.sync();
                u64 seen = 0;
                for (int q = 0; q < CL * kWarps; ++q) {
                    const u64 c = cluster.map_shared_rank(sh.warp_cnt, q / kWarps)[q % kWarps];
                    if (seen + c >= take) {
                        if (q / kWarps == rank && q % kWarps == warp) {
                            u64 left = take - seen;           // 1 .. c
                            for (int i = w0; i < w1; i += 32) {
                                const bool hit = i + lane < w1 && key_of(xs[i + lane]) == thr;
                                const unsigned bal = __ballot_sync(0xffffffffu, hit);
                                if (left <= (u64)__popc(bal)) {
                                    if (hit && (u64)__popc(bal & ((2u << lane) - 1)) == left)
                                        for (int z = 0; z < CL; ++z) *cluster.map_shared_rank(&sh.cut, z) = base + i + lane;
                                    break;
                                }
                                left -= __popc(bal);
                            }
                        }
                        break;
                    }
                    seen += c;
                }
                cluster.sync();
                cut = sh.cut;
                return above_mass + take * w;
            }
            klo = nlo;
            khi = min(khi, (uint32_t)(klo + ((1u << shift) - 1)));
            shift = 0;
            while ((((uint64_t)khi - klo) >> shift) >= kFine) ++shift;
            first = false;
        }
    };

    u64 kept_mass = 0; bool mass_known = false;
    if (use_k) {
        u64 tot;
        const u64 mine = (u64)c4[0] + c4[1] + c4[2] + c4[3];
        u64 e = block_excl<u64>(mine, sh.scan, &tot);
        if (tot > (u64)k) {                                   // fewer elements with weight than k: top-k removes nothing that counts
            if (tid == 0) sh.bin = -1;
            __syncthreads();
            if (e < (u64)k && e + mine >= (u64)k)
                for (int j = 0; j < 4; ++j) { if (e + c4[j] >= (u64)k) { sh.bin = tid * 4 + j; sh.before_cnt = e; break; } e += c4[j]; }
            __syncthreads();
            const int zb = sh.bin; const u64 before = sh.before_cnt;
            __syncthreads();
            kept_mass = refine(false, zb, zb, before, (u64)k, false, 0);
            mass_known = true;
        }
    }
    if (use_p) {
        const u64 frac64 = tp > 0.f ? (u64)__double2ull_rz((double)tp * 18446744073709551616.0) : 0ull;
        // bins that may hold the threshold, from counts alone: an element of bin b weighs between e^-(b+1)d and e^-bd
        // (one more bin on either side for the rounding of the bin's number)
        const double d = (double)kRange / (kBins - 1);
        double up = 0, dn = 0;
        double u4[4], l4[4];
        for (int j = 0; j < 4; ++j) {
            const int b = tid * 4 + j;
            u4[j] = (double)c4[j] * exp(-d * max(0, b - 1)); l4[j] = (double)c4[j] * exp(-d * (b + 2));
            up += u4[j]; dn += l4[j];
        }
        double tot_up, tot_dn;
        double eu = block_excl<double>(up, sh.dscan, &tot_up), el = block_excl<double>(dn, sh.dscan, &tot_dn);
        const double t_lo = mass_known ? (double)kept_mass * 0x1p-44 * tp * (1 - 1e-9) : tot_dn * tp, t_hi = mass_known ? (double)kept_mass * 0x1p-44 * tp * (1 + 1e-9) : tot_up * tp;
        if (tid == 0) { sh.zone_a = kBins - 2; sh.zone_b = kBins - 2; }
        __syncthreads();
        for (int j = 0; j < 4; ++j) {
            const int b = tid * 4 + j;
            if (b < kBins - 1 && eu < t_lo && eu + u4[j] >= t_lo) atomicMin(&sh.zone_a, b);
            if (b < kBins - 1 && el < t_hi && el + l4[j] >= t_hi) atomicMin(&sh.zone_b, b);
            eu += u4[j]; el += l4[j];
        }
        __syncthreads();
        int za = max(0, min(sh.zone_a, sh.zone_b) - 1), zb = min(kBins - 2, max(sh.zone_a, sh.zone_b) + 1);
        if (!(t_lo > 0)) za = 0;
        if (mass_known) {                                     // the threshold of top-k bounds the zone from below
            const float xk = __uint_as_float((thr & 0x80000000u) ? thr : ~thr & 0x7fffffffu);
            zb = max(za, min(zb, bin_of(r, xk)));
            za = min(za, bin_of(r, xk));
        }
        __syncthreads();
        u64 before = 0, tot;
        {
            u64 mine = 0;
            for (int j = 0; j < 4; ++j) if (tid * 4 + j < za) mine += c4[j];
            block_excl<u64>(mine, sh.scan, &tot);
            before = tot;
        }
        __syncthreads();
        refine(true, za, zb, before, kept_mass, mass_known, frac64);
    }
    // ---- weight kept by every warp's part, then the draw
    auto kept = [&](float x, int idx) {
        const uint32_t key = key_of(x);
        return x >= r.x_min && (key < thr || (key == thr && idx <= cut));
    };
    u64 ws = 0;
    for (int i = w0 + lane; i < w1; i += 32) if (kept(xs[i], base + i)) ws += weight(r, xs[i]);
#pragma unroll
    for (int o = 16; o; o >>= 1) ws += __shfl_xor_sync(0xffffffffu, ws, o);
    __syncthreads();
    if (lane == 0) sh.warp_sum[warp] = ws;
    cluster.sync();
    u64 sum[kMaxCluster * kWarps / 32], Z = 0;
#pragma unroll
    for (int j = 0; j < kMaxCluster * kWarps / 32; ++j) {
        const int q = lane * (kMaxCluster * kWarps / 32) + j;
        sum[j] = q < CL * kWarps ? cluster.map_shared_rank(sh.warp_sum, q / kWarps)[q % kWarps] : 0;
        Z += sum[j];
    }
    const u64 mine = Z;
    const u64 incl = warp_incl(mine);
    Z = __shfl_sync(0xffffffffu, incl, 31);
    const float u = p.u[row];
    const u64 U = u >= 1.f ? ~0ull : (u > 0.f ? (u64)__double2ull_rz((double)u * 18446744073709551616.0) : 0ull);
    const u64 target = __umul64hi(Z, U);                      // the token: lowest index with cumulative weight > target
    u64 before = incl - mine; int owner = -1; u64 obefore = 0;
#pragma unroll
    for (int j = 0; j < kMaxCluster * kWarps / 32; ++j) {
        if (before <= target && before + sum[j] > target) { owner = lane * (kMaxCluster * kWarps / 32) + j; obefore = before; }
        before += sum[j];
    }
    const unsigned who = __ballot_sync(0xffffffffu, owner >= 0);
    owner = __shfl_sync(0xffffffffu, owner, __ffs(who) - 1);
    obefore = __shfl_sync(0xffffffffu, obefore, __ffs(who) - 1);
    if (owner / kWarps == rank && owner % kWarps == warp) {
        u64 run = obefore;
        for (int i = w0; i < w1; i += 32) {
            const float x = i + lane < w1 ? xs[i + lane] : -INFINITY;
            const u64 w = i + lane < w1 && kept(x, base + i + lane) ? weight(r, x) : 0;
            const u64 c = warp_incl(w) + run;
            const unsigned over = __ballot_sync(0xffffffffu, c > target);
            if (over) {
                if (lane == __ffs(over) - 1) {
                    const int tok = base + i + lane;
                    if (p.token) p.token[row] = tok;
                    if (p.token2) p.token2[row * p.token2_stride] = tok;
                    if (p.prob) p.prob[row * p.prob_stride] = (float)((x == r.max ? 1.0 : exp2(((double)x - (double)r.max) * r.inv_t)) / ((double)Z * 0x1p-44));
                }
                break;
            }
            run = __shfl_sync(0xffffffffu, c, 31);
        }
    }
    cluster.sync();                                           // no block leaves while another still reads its sums
}

template <class E>
pt_status launch_t(const SampleP& p, int64_t n, cudaStream_t st) {
    int cl = 1;
    while (cl < kMaxCluster && (p.vocab + cl - 1) / cl > 16384) cl *= 2;
    const int slice = ((p.vocab + cl - 1) / cl + 3) & ~3;
    const size_t smem = ((sizeof(Shared) + 15) & ~15) + (size_t)slice * 4;
    static bool done_[kMaxDevices] = {};
    bool& done = done_[current_device()];
    if (!done) {
        cudaError_t e = cudaFuncSetAttribute(k_sample<E>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(((sizeof(Shared) + 15) & ~15) + kMaxSlice * 4));
        if (e != cudaSuccess) { set_error("cudaFuncSetAttribute: %s", cudaGetErrorString(e)); return PT_ERR_CUDA; }
        done = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(n * cl)); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension; at[0].val.clusterDim.x = cl; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    cfg.attrs = at; cfg.numAttrs = 1;
    cudaError_t e = cudaLaunchKernelEx(&cfg, k_sample<E>, p, slice);
    if (e != cudaSuccess) { set_error("k_sample launch: %s", cudaGetErrorString(e)); return PT_ERR_CUDA; }
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return PT_OK;
}

}  // namespace

int sample_vocab_limit() { return kMaxCluster * kMaxSlice; }

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
    if ((uintptr_t)logits % (dtype == PT_F32 ? 4 : 2) || (uintptr_t)token % 4) { set_error("logits must be aligned to their type, token 4-byte aligned"); return PT_ERR_MISALIGNED; }
    SampleP p{};
    p.logits = logits; p.row_stride = row_stride; p.vocab = vocab; p.u = u;
    p.temperature = temperature; p.top_k = top_k; p.top_p = top_p; p.min_p = min_p;
    p.token = token; p.prob = prob; p.prob_stride = 1;
    return launch_sample(p, n, dtype == PT_BF16, (cudaStream_t)stream);
}
