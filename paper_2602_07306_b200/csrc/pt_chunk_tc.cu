// Attention of a ragged chunk over the paged KV cache on the 5th-generation tensor cores (tcgen05 + tensor memory).
//
// Rows.  The G query heads of a KV head read the same keys, so the rows of a tile are (token, head of the group): 128 / G
// tokens of G rows.  q[t][row][head][:] puts the heads of a group side by side, so a 4-D tensor map (head_dim, head, row,
// track) with a box of G heads x 128 / G tokens delivers such a tile in one copy per 64 columns.  A segment is up to two
// tiles of one (sequence, track, KV head) with the keys they see, in tiles of 128 keys.
//
// Split.  Every launch has one block per SM, and the list of all segments' key tiles, each weighed by what it costs, is cut
// into one range of equal cost per block.  A block works through its range; where a segment is cut, each part leaves its
// running maximum, sum and unnormalised output in scratch, and k_chunk_combine merges the parts.  The same code serves four
// speculated tokens on a long context (all ranges are parts of few segments) and a long prompt (hardly any segment is cut).
// Blocks find their range themselves from the lengths in device memory: nothing is planned on the host, and a captured
// launch may be replayed with other lengths.
//
// Inside a block the roles are those of the prefill kernel: warp 0 copies Q, K and V with TMA, warp 1 issues the products
// S = Q K^T and O += P V, warps 4-7 and 8-11 are the softmax of the two tiles, one thread per row.  Barriers count over all
// segments of a block, so the copies of the next segment start while the last one's output is being written.
// Every wait is bounded; on a timeout the block records PT_ERR_DEVICE_TIMEOUT and every role leaves.
#include "pt_chunk.h"
#include "pt_tcgen05.cuh"

namespace pt {

namespace {

constexpr int kChunkThreads = 384;
constexpr int kStK = 3, kStV = 2;              // ring depths: head_dim 128: 2 Q + 3 K + 2 V tiles of 32 KB fill a block's shared memory
constexpr int kMaxBlocks = 148;
// Cost of a segment in units: kCostSeg once, and per key tile kCost1 with one row tile, kCost2 with two.
constexpr int kCostSeg = 4, kCost1 = 4, kCost2 = 7;
constexpr int kMinUnits = kCostSeg + kCost1;   // a range is no shorter

enum { C_QFULL = 0, C_QEMPTY = 2, C_KFULL = 4, C_KEMPTY = 7, C_VFULL = 10, C_VEMPTY = 12, C_SFULL = 14, C_PFULL = 16, C_OREADY = 18, C_VRAW = 20, C_COUNT = 21 };

struct Plan { int64_t total, p0; int ranges, b, qrow0, tk, qb, u, len, pad; };

// cost of all segments of one (sequence, track, KV head)
__device__ __forceinline__ int64_t row_cost(int ql, int kl, int tpt) {
    int64_t c = 0;
    for (int t0 = 0; t0 < ql; t0 += 2 * tpt) {
        const int n = (kl - ql + min(t0 + 2 * tpt, ql) + 127) >> 7;
        c += kCostSeg + (int64_t)n * (t0 + tpt < ql ? kCost2 : kCost1);
    }
    return c;
}

// Walks the segments of a block's range.  Position of key tile k of a segment that starts at u (relative to the range):
// u for k = 0, u + kCostSeg + k w for the others; a tile belongs to the range its position lies in.
struct Seg {
    int b, qrow0, qlen, kvlen, tk, qb, u, len;     // len: length of the range
    int tok0, n0, n1, n, w, lo, hi;                // key tiles of the two row tiles, and the part [lo, hi) of max(n0, n1) that is ours
    __device__ __forceinline__ void start(const Plan& pl, const ChunkP& p, int tpt) {
        b = pl.b; qrow0 = pl.qrow0; tk = pl.tk; qb = pl.qb; u = pl.u; len = pl.len;
        if (len > 0) { qlen = p.qlen[b]; kvlen = p.kvlen[b]; derive(tpt); }
    }
    __device__ __forceinline__ static int first_at(int rel, int w) {       // first tile whose position, relative to the segment, is >= rel
        return rel <= 0 ? 0 : max(1, (rel - kCostSeg + w - 1) / w);
    }
    __device__ __forceinline__ void derive(int tpt) {
        tok0 = qb * 2 * tpt;
        n0 = (kvlen - qlen + min(tok0 + tpt, qlen) + 127) >> 7;
        n1 = tok0 + tpt < qlen ? (kvlen - qlen + min(tok0 + 2 * tpt, qlen) + 127) >> 7 : 0;
        n = max(n0, n1);
        w = n1 ? kCost2 : kCost1;
        lo = min(n, first_at(-u, w));
        hi = min(n, first_at(len - u, w));
    }
    // the next segment that starts inside the range
    __device__ __forceinline__ bool advance(const ChunkP& p, int tpt) {
        u += kCostSeg + n * w;
        if (u >= len) return false;
        if ((qb + 1) * 2 * tpt < qlen) ++qb;
        else {
            qb = 0;
            if (++tk == p.T * p.nkv) {
                tk = 0;
                do {
                    qrow0 += p.qlen[b];
                    if (++b >= p.B) return false;
                } while (p.qlen[b] == 0);
                qlen = p.qlen[b]; kvlen = p.kvlen[b];
            }
        }
        derive(tpt);
        return true;
    }
};

// Where range `c` of the launch starts: all threads of the block call it.  buf: 2 * (THREADS / 32 + 1) values.
template <int THREADS>
__device__ __forceinline__ void make_plan(const ChunkP& p, int tpt, int blocks, int c, Plan* out, int64_t* buf) {
    constexpr int NW = THREADS / 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int tkn = p.T * p.nkv;
    int64_t total = 0, rows = 0;
    int bad = 0;
    for (int b = tid; b < p.B; b += THREADS) {
        const int ql = p.qlen[b], kl = p.kvlen[b];
        const bool ok = ql >= 0 && kl >= ql && (int64_t)kl <= (int64_t)p.maxp * p.ps && ql <= p.M;
        bad |= !ok;
        rows += ok ? ql : 0;
        if (ok) total += row_cost(ql, kl, tpt);
    }
    bad = __syncthreads_or(bad);
    auto excl = [&](int64_t v, int64_t* b2, int64_t& sum) {                // exclusive prefix over the block
        int64_t incl = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const int64_t x = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += x; }
        __syncthreads();
        if (lane == 31) b2[warp] = incl;
        __syncthreads();
        int64_t before = 0, all = 0;
        for (int i = 0; i < NW; ++i) { if (i < warp) before += b2[i]; all += b2[i]; }
        sum = all;
        return before + incl - v;
    };
    int64_t all_rows;
    excl(total, buf, total);
    excl(rows, buf + NW, all_rows);
    total *= tkn;
    if (tid == 0) {
        out->len = 0;
        if ((bad || all_rows > p.M) && blockIdx.x == 0) report(p.status, PT_ERR_DEVICE_BOUNDS, LOC_CHUNK_LEN);
    }
    if (bad || all_rows > p.M || total == 0) { __syncthreads(); return; }
    const int64_t ranges = min((int64_t)blocks, max((int64_t)1, total / kMinUnits));
    if (c >= ranges) { __syncthreads(); return; }
    const int64_t p0 = total * c / ranges, p1 = total * (c + 1) / ranges;
    int64_t base = 0, row_base = 0;
    for (int b0 = 0; b0 < p.B; b0 += THREADS) {
        const int b = b0 + tid;
        const int ql = b < p.B ? p.qlen[b] : 0, kl = b < p.B ? p.kvlen[b] : 0;
        const int64_t one = row_cost(ql, kl, tpt), cost = one * tkn;
        int64_t sum, rsum;
        const int64_t at = base + excl(cost, buf, sum), row = row_base + excl((int64_t)ql, buf + NW, rsum);
        if (p0 >= at && p0 < at + cost) {
            const int64_t rem = p0 - at;
            const int tk = (int)(rem / one);
            int64_t in = rem - tk * one;
            int qb = 0;
            for (;; ++qb) {
                const int t0 = qb * 2 * tpt;
                const int n = (kl - ql + min(t0 + 2 * tpt, ql) + 127) >> 7;
                const int64_t cst = kCostSeg + (int64_t)n * (t0 + tpt < ql ? kCost2 : kCost1);
                if (in < cst) break;
                in -= cst;
            }
            out->b = b; out->qrow0 = (int)row; out->tk = tk; out->qb = qb; out->u = -(int)in; out->len = (int)(p1 - p0);
            out->total = total; out->ranges = (int)ranges; out->p0 = p0;
        }
        base += sum; row_base += rsum;
        if (base > p0) break;
    }
    __syncthreads();
}

template <int DH> struct ChunkCfg {
    static constexpr int HALVES = DH / 64;
    static constexpr int TILE = HALVES * kHalfBytes;               // one Q, K or V tile of 128 rows
    static constexpr int SMEM = (2 + kStK + kStV) * TILE + 1024 + 1024;
    static_assert(SMEM <= 232448, "shared memory of one block");
};

// Scratch: two slots per block (the part of a segment that began in an earlier range, the part of one that continues in
// a later range), each 256 rows of (maximum in powers of two, sum) and 256 rows of DH outputs.
template <int DH> struct Slots {
    float* base;
    __device__ __host__ static constexpr size_t floats() { return 256 * (2 + (size_t)DH); }
    __device__ __forceinline__ float2* stats(int block, int which) const { return reinterpret_cast<float2*>(base + ((size_t)block * 2 + which) * floats()); }
    __device__ __forceinline__ float* out(int block, int which) const { return base + ((size_t)block * 2 + which) * floats() + 512; }
};

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, uint64_t* bar, int c0, int c1, int c2, int c3) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(dst), "l"((uint64_t)map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(smem_u32(bar)) : "memory");
}

template <int DH>
__global__ void __launch_bounds__(kChunkThreads, 1)
k_chunk_tc(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kvmap, const ChunkP p, float* scratch, const int tpt,
           const uint32_t q_bytes) {
    using C = ChunkCfg<DH>;
    constexpr int HALVES = C::HALVES, TILE = C::TILE;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t* sq = smem;
    uint8_t* sk = sq + 2 * TILE;
    uint8_t* sv = sk + kStK * TILE;
    uint64_t* bars = (uint64_t*)(sv + kStV * TILE);
    int64_t* buf = (int64_t*)(bars + C_COUNT);                     // 2 * 12 values
    Plan* plan = (Plan*)(buf + 24);
    uint32_t* tmem_slot = (uint32_t*)(plan + 1);
    volatile int* abort_flag = (volatile int*)(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int G = p.nq / p.nkv;
    if (threadIdx.x == 0) {
        for (int i = 0; i < C_COUNT; ++i) mbar_init(&bars[i], (i == C_PFULL || i == C_PFULL + 1) ? 4 : 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    make_plan<kChunkThreads>(p, tpt, gridDim.x, blockIdx.x, plan, buf);
    if (plan->len == 0) return;                                    // nothing for this block, or bad lengths
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    Seg sg;
    sg.start(*plan, p, tpt);
    bool more = true;

    if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp == 0) {
        // ------------------------------------------------------------------ copies
        bool bad_page = false, ok = true;
        int jj = 0, qc[2] = {0, 0}, raw = 0;
        auto wait = [&](int bar, uint32_t parity) {
            if (!mbar_wait(&bars[bar], parity, abort_flag, true)) { if (lane == 0) { report(p.status, PT_ERR_DEVICE_TIMEOUT, LOC_CHUNK_WAIT); *abort_flag = 1; } ok = false; }
            ok = __all_sync(0xffffffffu, ok);
            return ok;
        };
        for (; more && ok; more = sg.advance(p, tpt)) {
            if (sg.lo >= sg.hi) continue;
            const int t = sg.tk / p.nkv, kvh = sg.tk % p.nkv;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (sg.lo >= (i ? sg.n1 : sg.n0)) continue;
                if (!wait(C_QEMPTY + i, (uint32_t)(qc[i] & 1) ^ 1u)) break;
                if (lane == 0) {
                    mbar_expect_tx(&bars[C_QFULL + i], q_bytes);
#pragma unroll
                    for (int h = 0; h < HALVES; ++h)
                        tma_load_4d(smem_u32(sq + i * TILE + h * kHalfBytes), &qmap, &bars[C_QFULL + i], h * 64, kvh * G, sg.qrow0 + sg.tok0 + i * tpt, t);
                }
                ++qc[i];
            }
            const int32_t* bt = p.bt + (size_t)sg.b * p.maxp;
            for (int j = sg.lo; j < sg.hi && ok; ++j, ++jj) {
                const int sK = jj % kStK, s = jj % kStV;
                const int key0 = j * 128;
                const int ng = min(8, (sg.kvlen - key0 + 15) >> 4);    // 16-key groups of this tile that hold keys
                int row_k = 0;
                if (lane < ng) {
                    const int key = key0 + lane * 16;
                    int page = bt[key / p.ps];
                    if (page < 0 || page >= p.num_pages) { bad_page = true; page = 0; }
                    row_k = (page * 2 * p.nkv + kvh) * p.ps + key % p.ps;
                }
                const uint32_t bytes = (uint32_t)ng * 16u * DH * 2u;
                if (!wait(C_KEMPTY + sK, (uint32_t)(jj / kStK & 1) ^ 1u)) break;
                if (lane == 0) mbar_expect_tx(&bars[C_KFULL + sK], bytes);
                __syncwarp();
                if (lane < ng) {
#pragma unroll
                    for (int h = 0; h < HALVES; ++h)
                        tma_load_3d(smem_u32(sk + sK * TILE + h * kHalfBytes + lane * 2048), &kvmap, &bars[C_KFULL + sK], h * 64, row_k, t);
                }
                if (!wait(C_VEMPTY + s, (uint32_t)(jj / kStV & 1) ^ 1u)) break;
                const bool partial = ((sg.kvlen - key0) & 15) && key0 + 128 > sg.kvlen;    // rows of the last group past the last key must read as zero
                uint64_t* vbar = partial ? &bars[C_VRAW] : &bars[C_VFULL + s];
                if (lane == 0) mbar_expect_tx(vbar, bytes);
                __syncwarp();
                if (lane < ng) {
#pragma unroll
                    for (int h = 0; h < HALVES; ++h)
                        tma_load_3d(smem_u32(sv + s * TILE + h * kHalfBytes + lane * 2048), &kvmap, vbar, h * 64, row_k + p.nkv * p.ps, t);
                }
                if (partial) {
                    if (!wait(C_VRAW, (uint32_t)raw & 1u)) break;
                    ++raw;
                    const int nvalid = sg.kvlen - key0;
                    for (int idx = lane; idx < (ng * 16 - nvalid) * HALVES * 8; idx += 32) {
                        const int row = nvalid + idx / (HALVES * 8), rem = idx % (HALVES * 8);
                        *reinterpret_cast<uint4*>(sv + s * TILE + (rem >> 3) * kHalfBytes + row * 128 + (rem & 7) * 16) = make_uint4(0, 0, 0, 0);
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bars[C_VFULL + s]);
                }
            }
        }
        if (bad_page) report(p.status, PT_ERR_DEVICE_BOUNDS, LOC_CHUNK_PAGE);
        if (!ok) {                                                 // copies still in flight get a bounded time to land
            WaitClock clock;
            for (int b = C_KFULL; b < C_VFULL + kStV; ++b)
                for (uint32_t i = 0; i < (1u << 16) && !clock.expired(100000000ull); ++i) __nanosleep(64);
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer
        constexpr uint32_t idesc_qk = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(128 >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
        constexpr uint32_t idesc_pv = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(DH >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
        bool ok = true;
        int jj = 0, qc[2] = {0, 0}, cnt[2] = {0, 0};
        auto wait = [&](int bar, uint32_t parity) {
            if (!ok) return;
            if (!__all_sync(0xffffffffu, mbar_wait(&bars[bar], parity, abort_flag))) { ok = false; if (lane == 0) { report(p.status, PT_ERR_DEVICE_TIMEOUT, LOC_CHUNK_WAIT); *abort_flag = 1; } }
            tc_fence_after();
        };
        auto qk = [&](int i, int s, bool last) {                   // S_i = Q_i K_s^T
            if (!ok) return;
            const uint32_t qa = smem_u32(sq + i * TILE), ka = smem_u32(sk + s * TILE);
#pragma unroll
            for (int ks = 0; ks < DH / 16; ++ks) {
                const uint32_t off = (uint32_t)(ks >> 2) * kHalfBytes + (uint32_t)(ks & 3) * 32u;
                mma_ss(tmem_base + i * 128, desc_kmajor(qa + off), desc_kmajor(ka + off), idesc_qk, ks != 0);
            }
            tc_commit(&bars[C_SFULL + i]);
            if (last) tc_commit(&bars[C_QEMPTY + i]);
        };
        for (; more && ok; more = sg.advance(p, tpt)) {
            if (sg.lo >= sg.hi) continue;
            const int end[2] = {min(sg.hi, sg.n0), min(sg.hi, sg.n1)};
            wait(C_KFULL + jj % kStK, (uint32_t)(jj / kStK) & 1u);
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (sg.lo < end[i]) { wait(C_QFULL + i, (uint32_t)qc[i] & 1u); ++qc[i]; qk(i, jj % kStK, sg.lo + 1 == end[i]); }
            if (ok) tc_commit(&bars[C_KEMPTY + jj % kStK]);
            for (int j = sg.lo; j < sg.hi && ok; ++j, ++jj) {
                const int s = jj % kStV, sn = (jj + 1) % kStK;
                const uint32_t phn = (uint32_t)((jj + 1) / kStK) & 1u;
                const int ng = min(8, (sg.kvlen - j * 128 + 15) >> 4);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if (j >= end[i]) continue;
                    const uint32_t va = smem_u32(sv + s * TILE);   // O_i (+)= P_i V_s over the groups that hold keys
                    wait(C_PFULL + i, (uint32_t)cnt[i] & 1u);
                    wait(C_VFULL + s, (uint32_t)(jj / kStV) & 1u);
                    ++cnt[i];
                    if (!ok) break;
                    for (int ks = 0; ks < ng; ++ks)
                        mma_ts(tmem_base + 256 + i * DH, tmem_base + i * 128 + ks * 8, desc_mnmajor(va + ks * 2048), idesc_pv, j > sg.lo || ks != 0);
                    tc_commit(&bars[C_OREADY + i]);
                    if (j + 1 < end[i]) { wait(C_KFULL + sn, phn); qk(i, sn, j + 2 == end[i]); }
                }
                if (ok) {
                    tc_commit(&bars[C_VEMPTY + s]);
                    if (j + 1 < sg.hi) tc_commit(&bars[C_KEMPTY + sn]);
                }
            }
        }
        __syncwarp();
    }
    } else {
        // ------------------------------------------------------------------ softmax groups
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        const int i = (warp - 4) >> 2;                             // row tile of this warp group
        const int w4 = warp & 3;                                   // tensor-memory lane quarter of this warp
        const int r = w4 * 32 + lane;                              // row inside the tile: token r / G, head r % G of the group
        const int tok = r / G, gh = r % G;
        const uint32_t t_s = tmem_base + ((uint32_t)(w4 * 32) << 16) + i * 128;
        const uint32_t t_o = tmem_base + ((uint32_t)(w4 * 32) << 16) + 256 + i * DH;
        const float c = p.scale_log2;
        const Slots<DH> slots{scratch};
        bool ok = true;
        int cnt = 0;
        auto wait = [&](int bar, uint32_t parity) {
            ok = __all_sync(0xffffffffu, mbar_wait(&bars[bar], parity, abort_flag));
            if (!ok && lane == 0) { report(p.status, PT_ERR_DEVICE_TIMEOUT, LOC_CHUNK_WAIT); *abort_flag = 1; }
            tc_fence_after();
            return ok;
        };
        for (; more && ok; more = sg.advance(p, tpt)) {
            const int n_i = i ? sg.n1 : sg.n0, end = min(sg.hi, n_i);
            if (sg.lo >= end) continue;
            const int start = sg.kvlen - sg.qlen, tok_i = sg.tok0 + i * tpt;
            const bool live = tok < tpt && tok_i + tok < sg.qlen;
            const int limit = min(start + tok_i + tok, sg.kvlen - 1);  // last visible key of this row
            const int tile_limit = min(start + tok_i, sg.kvlen - 1);   // last visible key of the tile's first row
            float m_ref = -INFINITY, l_run = 0.f;
            for (int j = sg.lo; j < end; ++j, ++cnt) {
                if (!wait(C_SFULL + i, (uint32_t)cnt & 1u)) break;
                const int key0 = j * 128;
                float v[128];
#pragma unroll
                for (int cc = 0; cc < 4; ++cc) tm_ld32(t_s + cc * 32, v + cc * 32);
                tm_wait_ld();
                if (key0 + 127 > tile_limit) {
#pragma unroll
                    for (int e = 0; e < 128; ++e) if (key0 + e > limit) v[e] = -INFINITY;
                }
                float mx0 = -INFINITY, mx1 = -INFINITY, mx2 = -INFINITY, mx3 = -INFINITY;
#pragma unroll
                for (int e = 0; e < 128; e += 8) {
                    mx0 = max3(mx0, v[e], v[e + 1]); mx1 = max3(mx1, v[e + 2], v[e + 3]);
                    mx2 = max3(mx2, v[e + 4], v[e + 5]); mx3 = max3(mx3, v[e + 6], v[e + 7]);
                }
                const float mx = fmaxf(fmaxf(mx0, mx1), fmaxf(mx2, mx3));
                if (j == sg.lo) {
                    m_ref = mx;                                    // -inf where the row sees nothing of this tile
                } else {
                    const bool grow = live && (mx - m_ref) * c > 8.0f;     // also from -inf, when mx is finite
                    if (__any_sync(0xffffffffu, grow)) {
                        // the previous P V product must have landed before the accumulator is rescaled
                        if (!wait(C_OREADY + i, (uint32_t)(cnt - 1) & 1u)) break;
                        const float corr = grow ? ex2((m_ref - mx) * c) : 1.0f;
                        if (grow) { m_ref = mx; l_run *= corr; }
#pragma unroll 1
                        for (int cc = 0; cc < DH / 32; ++cc) {
                            float o[32];
                            tm_ld32(t_o + cc * 32, o);
                            tm_wait_ld();
#pragma unroll
                            for (int e = 0; e < 32; ++e) o[e] *= corr;
                            tm_st32(t_o + cc * 32, o);
                        }
                    }
                }
                // P = exp2(c s - c m) as bf16 over the first half of the score columns (masked scores are -inf and give 0)
                float l0 = 0.f, l1 = 0.f, l2 = 0.f, l3 = 0.f;
                const float nmc = m_ref == -INFINITY ? 0.f : -m_ref * c;
#pragma unroll
                for (int cc = 0; cc < 4; ++cc) {
                    uint32_t pk[16];
#pragma unroll
                    for (int e = 0; e < 32; e += 4) {
                        float x0, x1, x2, x3;
                        fma2(x0, x1, v[cc * 32 + e], v[cc * 32 + e + 1], c, nmc);
                        fma2(x2, x3, v[cc * 32 + e + 2], v[cc * 32 + e + 3], c, nmc);
                        x0 = ex2(x0); x1 = ex2(x1); x2 = ex2(x2); x3 = ex2(x3);
                        add2(l0, l1, x0, x1);
                        add2(l2, l3, x2, x3);
                        pk[e >> 1] = pack_bf16(x0, x1);
                        pk[(e >> 1) + 1] = pack_bf16(x2, x3);
                    }
                    tm_st16(t_s + cc * 16, pk);
                }
                l_run += (l0 + l1) + (l2 + l3);
                tm_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars[C_PFULL + i]);
            }
            if (!ok || !wait(C_OREADY + i, (uint32_t)(cnt - 1) & 1u)) break;
            if (sg.lo == 0 && end == n_i) {                        // all of the tile's keys: the result
                const float inv = l_run > 0.f ? 1.0f / l_run : 0.f;
                const int t = sg.tk / p.nkv, head = (sg.tk % p.nkv) * G + gh;
                __nv_bfloat16* dst = p.o + ((size_t)t * p.M + sg.qrow0 + tok_i + tok) * (size_t)(p.nq * DH) + (size_t)head * DH;
#pragma unroll 1
                for (int cc = 0; cc < DH / 32; ++cc) {
                    float o[32];
                    tm_ld32(t_o + cc * 32, o);
                    tm_wait_ld();
                    if (live) {
#pragma unroll
                        for (int e = 0; e < 32; e += 8) {
                            uint4 u;
                            u.x = pack_bf16(o[e] * inv, o[e + 1] * inv); u.y = pack_bf16(o[e + 2] * inv, o[e + 3] * inv);
                            u.z = pack_bf16(o[e + 4] * inv, o[e + 5] * inv); u.w = pack_bf16(o[e + 6] * inv, o[e + 7] * inv);
                            *reinterpret_cast<uint4*>(dst + cc * 32 + e) = u;
                        }
                    }
                }
            } else {                                               // a part: merged by k_chunk_combine
                const int which = sg.lo > 0 ? 0 : 1;
                if (live) slots.stats(blockIdx.x, which)[i * 128 + r] = make_float2(m_ref * c, l_run);
                float* dst = slots.out(blockIdx.x, which) + (size_t)(i * 128 + r) * DH;
#pragma unroll 1
                for (int cc = 0; cc < DH / 32; ++cc) {
                    float o[32];
                    tm_ld32(t_o + cc * 32, o);
                    tm_wait_ld();
                    if (live) {
#pragma unroll
                        for (int e = 0; e < 32; e += 4) *reinterpret_cast<float4*>(dst + cc * 32 + e) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
                    }
                }
            }
            tc_fence_before();                                     // the accumulator has been read: the next segment's P may follow
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 2) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512) : "memory");
    }
}

// Merges the parts of cut segments.  Block (c, g) handles the segment that is cut at the start of range c + 1, if no earlier
// range's start cuts it too: parts lie in range c (second slot) and, as long as the segment goes on, in c + 1, c + 2, ...
// (first slot).  g: rows 32 g .. 32 g + 31 of its 256; one warp per row.
constexpr int kCombineThreads = 256;
template <int DH>
__global__ void __launch_bounds__(kCombineThreads)
k_chunk_combine(const ChunkP p, float* scratch, const int tpt, const int blocks) {
    __shared__ int64_t buf[2 * (kCombineThreads / 32)];
    __shared__ Plan plan;
    make_plan<kCombineThreads>(p, tpt, blocks, blockIdx.x + 1, &plan, buf);
    Seg sg;
    bool mine = plan.len > 0;
    int64_t seg_start = 0;
    auto lo_of = [&](int c) { const int64_t rel = plan.total * c / plan.ranges - seg_start; return rel >= (int64_t)0x7fffffff - sg.w ? sg.n : min(sg.n, Seg::first_at((int)max(rel, (int64_t)0), sg.w)); };
    if (mine) {
        sg.start(plan, p, tpt);
        seg_start = plan.p0 + plan.u;
        mine = sg.lo > 0 && sg.lo < sg.n && lo_of(blockIdx.x) == 0;     // cut at this range's start and at no earlier one
    }
    grid_dep_wait();
    grid_dep_launch();
    if (!mine) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int G = p.nq / p.nkv;
    const Slots<DH> slots{scratch};
    const int i = blockIdx.y >> 2;                                 // row tile
    const int n_i = i ? sg.n1 : sg.n0;
    if (sg.lo >= n_i) return;                                      // this tile's keys all lie in the first part: written there
    const int t = sg.tk / p.nkv, kvh = sg.tk % p.nkv;
    for (int rr = warp; rr < 32; rr += kCombineThreads / 32) {
        const int r = (blockIdx.y & 3) * 32 + rr;
        const int tok = r / G, tok_i = sg.tok0 + i * tpt;
        if (tok >= tpt || tok_i + tok >= sg.qlen) continue;
        float m = -INFINITY, l = 0.f, o[DH / 32];
#pragma unroll
        for (int e = 0; e < DH / 32; ++e) o[e] = 0.f;
        for (int c = blockIdx.x, lo = 0; lo < n_i; ++c) {
            const int hi = c == (int)blockIdx.x ? sg.lo : lo_of(c + 1);     // tiles [lo, hi) belong to range c
            const int top = min(hi, n_i);
            if (lo < top) {
                const int which = c == (int)blockIdx.x ? 1 : 0;
                const float2 st = slots.stats(c, which)[i * 128 + r];
                const float* src = slots.out(c, which) + (size_t)(i * 128 + r) * DH + lane;
                if (st.x > m) {
                    const float f = exp2f(m - st.x);
                    m = st.x; l *= f;
#pragma unroll
                    for (int e = 0; e < DH / 32; ++e) o[e] *= f;
                }
                if (st.x > -INFINITY) {
                    const float f = exp2f(st.x - m);
                    l += st.y * f;
#pragma unroll
                    for (int e = 0; e < DH / 32; ++e) o[e] += src[32 * e] * f;
                }
            }
            lo = hi;
        }
        const float inv = l > 0.f ? 1.0f / l : 0.f;
        __nv_bfloat16* dst = p.o + ((size_t)t * p.M + sg.qrow0 + tok_i + tok) * (size_t)(p.nq * DH) + (size_t)(kvh * G + r % G) * DH + lane;
#pragma unroll
        for (int e = 0; e < DH / 32; ++e) dst[32 * e] = __float2bfloat16_rn(o[e] * inv);
    }
}

template <int DH>
pt_status launch_t(const ChunkP& p, float* scratch, cudaStream_t st) {
    EncodeFn enc = get_encode();
    if (!enc) { set_error("cuTensorMapEncodeTiled is not available from this driver"); return PT_ERR_CUDA; }
    const int G = p.nq / p.nkv, tpt = 128 / G, box = std::min(tpt, p.M);
    CUtensorMap qmap, kvmap;
    cuuint64_t dims[4] = {(cuuint64_t)DH, (cuuint64_t)p.nq, (cuuint64_t)p.M, (cuuint64_t)p.T};
    cuuint64_t strides[3] = {(cuuint64_t)DH * 2, (cuuint64_t)p.nq * DH * 2, (cuuint64_t)p.M * p.nq * DH * 2};
    cuuint32_t bx[4] = {64, (cuuint32_t)G, (cuuint32_t)box, 1}, es[4] = {1, 1, 1, 1};
    CUresult r = enc(&qmap, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<__nv_bfloat16*>(p.q), dims, strides, bx, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                     CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) { set_error("cuTensorMapEncodeTiled (q) failed with code %d", (int)r); return PT_ERR_CUDA; }
    const int64_t rows = (int64_t)p.num_pages * 2 * p.nkv * p.ps;
    if (rows > 0x7fffffff) { set_error("a layer's slab of more than 2^31 cached vectors"); return PT_ERR_UNSUPPORTED; }
    pt_status s = make_map_bf16_strided(&kvmap, p.pool_l, DH, rows, p.T, p.pool_tstride * 2, 16);
    if (s != PT_OK) return s;
    static int sms_[kMaxDevices] = {};
    int& sms = sms_[current_device()];
    if (!sms) {
        int n = 0;
        cudaError_t e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, current_device());
        if (e == cudaSuccess) e = cudaFuncSetAttribute(k_chunk_tc<DH>, cudaFuncAttributeMaxDynamicSharedMemorySize, ChunkCfg<DH>::SMEM);
        if (e != cudaSuccess) { set_error("chunk attention setup: %s", cudaGetErrorString(e)); return PT_ERR_CUDA; }
        sms = n;
    }
    const int blocks = std::min(sms, kMaxBlocks);
    k_chunk_tc<DH><<<blocks, kChunkThreads, ChunkCfg<DH>::SMEM, st>>>(qmap, kvmap, p, scratch, tpt, (uint32_t)(128 * ChunkCfg<DH>::HALVES * G * box));
    g_launches.fetch_add(1, std::memory_order_relaxed);
    cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess && blocks > 1) {
        e = launch_dependent(k_chunk_combine<DH>, dim3(blocks - 1, 8), dim3(kCombineThreads), (size_t)0, st, p, scratch, tpt, blocks);
        g_launches.fetch_add(1, std::memory_order_relaxed);
    }
    if (e != cudaSuccess) { set_error("chunk attention launch: %s", cudaGetErrorString(e)); return PT_ERR_CUDA; }
    return PT_OK;
}

}  // namespace

size_t chunk_tc_scratch_bytes(int dh) { return (dh == 64 ? Slots<64>::floats() : Slots<128>::floats()) * 4 * 2 * kMaxBlocks; }

pt_status launch_chunk_attn_tc(const ChunkP& p, int dh, void* scratch, cudaStream_t st) {
    return dh == 64 ? launch_t<64>(p, (float*)scratch, st) : launch_t<128>(p, (float*)scratch, st);
}

}  // namespace pt
