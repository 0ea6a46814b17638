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
// launch may be replayed with other lengths.  One warp walks the range and hands the segments to the others through a ring
// in shared memory, so that the softmax threads, which hold a row of 128 scores each, carry nothing of the walk.
//
// Inside a block the roles are those of the prefill kernel: warps 0 and 3 copy Q and K, and V, with TMA, warp 1 issues the products
// S = Q K^T and O += P V, warps 4-7 and 8-11 are two softmax groups, one thread per row.  In a segment of two row tiles each
// group has one; in a segment of one, which is bound by the latency from a score to the next product, the groups take
// turns on its key tiles with a running maximum, sum and accumulator each, and the first merges both at the end.  Barriers
// count over all segments of a block, so the copies of the next segment start while the last one's output is being written.
// Weights are rounded to bf16 for the product with V, the operand type that the tensor core takes beside a bf16 V (their sum
// is taken unrounded; against 64 bits the outputs are off by 2.3e-3 of their size, 1.7e-3 of it the output's own rounding).
// Every wait is bounded; on a timeout the block records PT_ERR_DEVICE_TIMEOUT and every role leaves.
//
// Measured (head_dim 128): eight users' speculated tokens over 2k keys (8 tracks, 8 heads) 101 us, 0.74 of the copy bandwidth; four
// users' over 9k to 31k keys 127 us, 0.85: bound by the K and V stream and the start and merge around it.  2048 tokens over
// 32k keys (2 tracks, 8 heads on one KV head) 452 us, 1.15 PFLOP/s: a step of 128 keys of two tiles takes 4.0k cycles against 2.05k of
// products; a softmax takes 1.5 to 1.8k, bound by instruction issue, and waits for its own tile's products before and after.
// Scores in halves of 64 keys with two buffers per tile took 843 us (a product of 64 columns costs nearly one of 128).
#include "pt_chunk.h"
#include "pt_ring.cuh"
#include "pt_tcgen05.cuh"

namespace pt {

namespace {

constexpr int kChunkThreads = 384;
constexpr int kStK = 3, kStV = 2;              // ring depths: head_dim 128: 2 Q + 3 K + 2 V tiles of 32 KB fill a block's shared memory
constexpr int kMaxBlocks = 148;
// Cost of a segment in units of about 0.37 us: once for starting and writing it, and per key tile, with one row tile (bound
// by its share of the HBM bandwidth) and with two (bound by the softmax and the products).
// (Measured: 27 decoding sequences beside a 777-token chunk take 158 to 164 us with kCost2 from 7 to 9, 169 with kSeg2 = 14.)
constexpr int kSeg1 = 9, kSeg2 = 20, kCost1 = 4, kCost2 = 9;
constexpr int kMinUnits = kSeg1 + kCost1;      // a range is no shorter

enum { C_QFULL = 0, C_QEMPTY = 2, C_KFULL = 4, C_KEMPTY = 7, C_VFULL = 10, C_VEMPTY = 12, C_SFULL = 14, C_PFULL = 16, C_OREADY = 18, C_VRAW = 20, C_MREADY = 21, C_MDONE = 22,
       C_SEGFULL = 23, C_SEGEMPTY = 27, C_COUNT = 31 };
constexpr int kSegRing = 4;                    // segments handed out ahead
constexpr int kSegReaders = 11;                // warps 0, 1, 3 and the eight of the softmax

// Cost of one segment, of `left` tokens from its first one on and `keys` keys seen by its last row, in units of 2^sh (the
// host picks sh so that the sum over everything fits 31 bits); the + 1 keeps it above its last tile's position.
__device__ __forceinline__ int seg_cost(int left, int keys, int tpt, int sh) {
    const int n = (keys + 127) >> 7;
    return ((left > tpt ? kSeg2 + n * kCost2 : kSeg1 + n * kCost1) >> sh) + 1;
}

// Walks the segments of a range.  Position of key tile k of a segment that starts at u (relative to the range): u for k = 0,
// u + (kSeg + k w) / 2^sh for the others; a tile belongs to the range its position lies in.
// This code runs once per block and launch, so what it costs is fetching its instructions: it is written to be short.
struct Walk {
    int u, len, p0;                                // start of the segment relative to the range, length and start of the range
    int b, qrow0, qlen, kvlen, tk, qb;
    int tok0, n0, n1, n, cost, lo, hi;                // key tiles of the two row tiles, and the part [lo, hi) of max(n0, n1) that is ours
    __device__ __forceinline__ static int first_at(int rel, bool two, int sh) {    // first tile whose position, relative to the segment, is >= rel
        const int w = two ? kCost2 : kCost1;
        return rel <= 0 ? 0 : max(1, ((rel << sh) - (two ? kSeg2 : kSeg1) + w - 1) / w);
    }
    __device__ __forceinline__ void derive(int tpt, int sh) {
        tok0 = qb * 2 * tpt;
        n0 = (kvlen - qlen + min(tok0 + tpt, qlen) + 127) >> 7;
        n1 = tok0 + tpt < qlen ? (kvlen - qlen + min(tok0 + 2 * tpt, qlen) + 127) >> 7 : 0;
        n = max(n0, n1);
        cost = seg_cost(qlen - tok0, n * 128, tpt, sh);
        lo = u < 0 ? min(n, first_at(-u, n1 > 0, sh)) : 0;
        hi = len - u >= cost ? n : min(n, first_at(len - u, n1 > 0, sh));
    }
    // the next segment that starts inside the range
    __device__ __forceinline__ bool advance(const ChunkP& p, int tpt, int sh) {
        u += cost;
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
        derive(tpt, sh);
        return true;
    }

    // Finds range c of the launch; all lanes of a warp call it and get the same.  False: nothing in it.  Bad lengths are
    // reported by `reporter` and leave every range empty.
    __device__ __forceinline__ bool find(const ChunkP& p, int tpt, int sh, int blocks, int c, bool reporter) {
        const int lane = threadIdx.x & 31, tkn = p.T * p.nkv, span = 2 * tpt;
        int base = 0, row0 = 0, total = 0, start = 0;
        int64_t rows = 0;
        bool bad = false;
        // the first round over the sequences sums the costs, the second finds the one in which the range starts
        for (int round = 0; round < 2; ++round) {
#pragma unroll 1
            for (int b0 = 0; b0 < p.B; b0 += 32) {
                const bool in = b0 + lane < p.B;
                int ql = in ? p.qlen[b0 + lane] : 0;
                const int kl = in ? p.kvlen[b0 + lane] : 0;
                if (ql < 0 || kl < ql || (int64_t)kl > (int64_t)p.maxp * p.ps || ql > p.M) { bad = true; ql = 0; }
                int one = 0;                                   // cost of this lane's sequence for one (track, KV head)
                for (unsigned m = __ballot_sync(0xffffffffu, ql > span); m; m &= m - 1) {      // long chunks: the warp together
                    const int who = __ffs(m) - 1, q1 = __shfl_sync(0xffffffffu, ql, who), k1 = __shfl_sync(0xffffffffu, kl, who);
                    int s = 0;
#pragma unroll 1
                    for (int t0 = lane * span; t0 < q1; t0 += 32 * span) s += seg_cost(q1 - t0, k1 - q1 + min(t0 + span, q1), tpt, sh);
                    s = __reduce_add_sync(0xffffffffu, s);
                    if (lane == who) one = s;
                }
                if (ql > 0 && ql <= span) one = seg_cost(ql, kl, tpt, sh);
                if (round == 0) { total += one; rows += ql; continue; }
                int incl = one * tkn, rincl = ql;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int x = __shfl_up_sync(0xffffffffu, incl, o), y = __shfl_up_sync(0xffffffffu, rincl, o);
                    if (lane >= o) { incl += x; rincl += y; }
                }
                const unsigned m = __ballot_sync(0xffffffffu, start < base + incl);
                const int who = m ? __ffs(m) - 1 : 31;
                const int at = base + __shfl_sync(0xffffffffu, incl, who), rat = row0 + __shfl_sync(0xffffffffu, rincl, who);
                if (!m) { base = at; row0 = rat; continue; }
                const int per = __shfl_sync(0xffffffffu, one, who), rem = start - (at - per * tkn);
                b = b0 + who;
                qlen = __shfl_sync(0xffffffffu, ql, who); kvlen = __shfl_sync(0xffffffffu, kl, who);
                qrow0 = rat - qlen;
                tk = (int)((unsigned)rem / (unsigned)per);
                int left = rem - tk * per;                     // inside its segments of that (track, KV head)
#pragma unroll 1
                for (qb = 0;; qb += 32) {
                    const int t0 = (qb + lane) * span;
                    const int cst = t0 < qlen ? seg_cost(qlen - t0, kvlen - qlen + min(t0 + span, qlen), tpt, sh) : 0;
                    int cin = cst;
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) { const int x = __shfl_up_sync(0xffffffffu, cin, o); if (lane >= o) cin += x; }
                    const unsigned mq = __ballot_sync(0xffffffffu, left < cin);
                    if (mq) {
                        const int w2 = __ffs(mq) - 1;
                        qb += w2;
                        u = __shfl_sync(0xffffffffu, cin - cst, w2) - left;
                        return true;
                    }
                    left -= __shfl_sync(0xffffffffu, cin, 31);
                }
            }
            if (round) break;
            total = __reduce_add_sync(0xffffffffu, total) * tkn;
#pragma unroll
            for (int o = 16; o; o >>= 1) rows += __shfl_xor_sync(0xffffffffu, rows, o);
            if (__any_sync(0xffffffffu, bad) || rows > p.M) {
                if (reporter && lane == 0) report(p.status, PT_ERR_DEVICE_BOUNDS, LOC_CHUNK_LEN);
                return false;
            }
            const int ranges = max(1, min(blocks, total / (((kMinUnits - 1) >> sh) + 1)));
            if (total == 0 || c >= ranges) return false;
            const int each = total / ranges, more = total - each * ranges;     // the first `more` ranges are one longer
            start = p0 = each * c + min(c, more);
            len = each + (c < more);
        }
        return false;
    }
};

// What the other warps need of a segment; lo < 0: the end.
struct Seg { int row0, t, kvh, kvlen, pos0, left, n0, n1, lo, hi, b, pad; };

template <int DH> struct ChunkCfg {
    static constexpr int HALVES = DH / 64;
    static constexpr int TILE = HALVES * kHalfBytes;               // one Q, K or V tile of 128 rows
    static constexpr int SMEM = (2 + kStK + kStV) * TILE + 1024 + 2048;
    static_assert(SMEM <= 232448, "shared memory of one block");
};

// Where a range starts: the segment that holds its start, and what of it lies in earlier ranges.
struct Start { int p0, u, len, row0, t, kvh, left, n0, n1, lo, pad[6]; };

// Scratch: two slots per block (the part of a segment that began in an earlier range, the part of one that continues in
// a later range), each (maximum in powers of two, sum) of 256 rows and DH columns of 256 outputs; behind them the starts.
// Columns, because a thread holds a row: a warp's store is then 128 contiguous bytes, not 32 lines (a row-wise layout took
// 7 us per part of 256 rows, as long as three steps of the loop).
template <int DH> struct Slots {
    float* base;
    __device__ __host__ static constexpr size_t floats() { return 256 * (2 + (size_t)DH); }
    __device__ __forceinline__ float2* stats(int block, int which) const { return reinterpret_cast<float2*>(base + ((size_t)block * 2 + which) * floats()); }
    __device__ __forceinline__ Start* start(int block) const { return reinterpret_cast<Start*>(base + (size_t)kMaxBlocks * 2 * floats()) + block; }
    __device__ __forceinline__ float* out(int block, int which) const { return base + ((size_t)block * 2 + which) * floats() + 512; }
};

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, uint64_t* bar, int c0, int c1, int c2, int c3) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(dst), "l"((uint64_t)map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(smem_u32(bar)) : "memory");
}

__device__ __forceinline__ void st_global_32(void* p, const uint32_t* u) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(p), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]) : "memory");
}
// Eight products of 16 along the contraction with one election: an election and fresh descriptors for each product take the
// issuing warp longer than the tensor core takes for the product (88 cycles against 64 at 128 x 128).
// D[tmem] (+)= A[smem] * B[smem], 64 elements of the contraction at a time (HALVES of them, kHalfBytes apart)
template <int HALVES>
__device__ __forceinline__ void mma_ss_tile(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc) {
    static_assert(kHalfBytes >> 4 == 1024, "the second half's offset below");
    if constexpr (HALVES == 2)
        asm volatile("{\n .reg .pred e, o, z;\n .reg .b64 a<8>, b<8>;\n elect.sync _|e, 0xffffffff;\n setp.eq.b32 o, 0, 0;\n setp.ne.b32 z, 0, 0;\n"
                     " add.s64 a1, %1, 2;\n add.s64 b1, %2, 2;\n add.s64 a2, %1, 4;\n add.s64 b2, %2, 4;\n add.s64 a3, %1, 6;\n add.s64 b3, %2, 6;\n"
                     " add.s64 a4, %1, 1024;\n add.s64 b4, %2, 1024;\n add.s64 a5, %1, 1026;\n add.s64 b5, %2, 1026;\n"
                     " add.s64 a6, %1, 1028;\n add.s64 b6, %2, 1028;\n add.s64 a7, %1, 1030;\n add.s64 b7, %2, 1030;\n"
                     " @e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, z;\n @e tcgen05.mma.cta_group::1.kind::f16 [%0], a1, b1, %3, o;\n"
                     " @e tcgen05.mma.cta_group::1.kind::f16 [%0], a2, b2, %3, o;\n @e tcgen05.mma.cta_group::1.kind::f16 [%0], a3, b3, %3, o;\n"
                     " @e tcgen05.mma.cta_group::1.kind::f16 [%0], a4, b4, %3, o;\n @e tcgen05.mma.cta_group::1.kind::f16 [%0], a5, b5, %3, o;\n"
                     " @e tcgen05.mma.cta_group::1.kind::f16 [%0], a6, b6, %3, o;\n @e tcgen05.mma.cta_group::1.kind::f16 [%0], a7, b7, %3, o;\n}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc) : "memory");
    else
        asm volatile("{\n .reg .pred e, o, z;\n .reg .b64 a<4>, b<4>;\n elect.sync _|e, 0xffffffff;\n setp.eq.b32 o, 0, 0;\n setp.ne.b32 z, 0, 0;\n"
                     " add.s64 a1, %1, 2;\n add.s64 b1, %2, 2;\n add.s64 a2, %1, 4;\n add.s64 b2, %2, 4;\n add.s64 a3, %1, 6;\n add.s64 b3, %2, 6;\n"
                     " @e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, z;\n @e tcgen05.mma.cta_group::1.kind::f16 [%0], a1, b1, %3, o;\n"
                     " @e tcgen05.mma.cta_group::1.kind::f16 [%0], a2, b2, %3, o;\n @e tcgen05.mma.cta_group::1.kind::f16 [%0], a3, b3, %3, o;\n}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc) : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem] over 128 keys; acc = 0: D starts at zero
__device__ __forceinline__ void mma_ts_tile(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile("{\n .reg .pred p, e, o;\n .reg .b64 b<8>;\n .reg .b32 a<8>;\n elect.sync _|e, 0xffffffff;\n setp.eq.b32 o, 0, 0;\n setp.ne.b32 p, %4, 0;\n"
                 " add.u32 a1, %1, 8;\n add.s64 b1, %2, 128;\n add.u32 a2, %1, 16;\n add.s64 b2, %2, 256;\n add.u32 a3, %1, 24;\n add.s64 b3, %2, 384;\n"
                 " add.u32 a4, %1, 32;\n add.s64 b4, %2, 512;\n add.u32 a5, %1, 40;\n add.s64 b5, %2, 640;\n add.u32 a6, %1, 48;\n add.s64 b6, %2, 768;\n"
                 " add.u32 a7, %1, 56;\n add.s64 b7, %2, 896;\n"
                 " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n @e tcgen05.mma.cta_group::1.kind::f16 [%0], [a1], b1, %3, o;\n"
                 " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [a2], b2, %3, o;\n @e tcgen05.mma.cta_group::1.kind::f16 [%0], [a3], b3, %3, o;\n"
                 " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [a4], b4, %3, o;\n @e tcgen05.mma.cta_group::1.kind::f16 [%0], [a5], b5, %3, o;\n"
                 " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [a6], b6, %3, o;\n @e tcgen05.mma.cta_group::1.kind::f16 [%0], [a7], b7, %3, o;\n}"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}

template <int DH>
__global__ void __launch_bounds__(kChunkThreads, 1)
k_chunk_tc(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kvmap, const ChunkP p, float* scratch, const int tpt,
           const uint32_t q_bytes, const int box, const int sh) {
    using C = ChunkCfg<DH>;
    constexpr int HALVES = C::HALVES, TILE = C::TILE;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t* sq = smem;
    uint8_t* sk = sq + 2 * TILE;
    uint8_t* sv = sk + kStK * TILE;
    uint64_t* bars = (uint64_t*)(sv + kStV * TILE);
    uint32_t* tmem_slot = (uint32_t*)(bars + C_COUNT);
    volatile int* abort_flag = (volatile int*)(tmem_slot + 1);
    Seg* ring = (Seg*)(bars + 40);                                 // kSegRing segments
    float2* odd_stats = (float2*)(bars + 80);                      // maximum and sum of the second group, one-tile segments

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int G = p.nq / p.nkv;
    if (threadIdx.x == 0) {
        for (int i = 0; i < C_COUNT; ++i)
            mbar_init(&bars[i], (i == C_PFULL || i == C_PFULL + 1 || i == C_MREADY || i == C_MDONE) ? 4 : i >= C_SEGEMPTY ? kSegReaders : 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    grid_dep_wait();                                               // everything that this kernel reads or writes may be an earlier kernel's
    grid_dep_launch();
    // the next segment of the block; false at the end, or after a wait that ran out
    int seg_i = 0;
    auto next_seg = [&](Seg& sg) {
        const int s = seg_i % kSegRing;
        if (!__all_sync(0xffffffffu, mbar_wait(&bars[C_SEGFULL + s], (uint32_t)(seg_i / kSegRing) & 1u, abort_flag))) {
            if (lane == 0) { report(p.status, PT_ERR_DEVICE_TIMEOUT, LOC_CHUNK_WAIT); *abort_flag = 1; }
            return false;
        }
        sg = ring[s];
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars[C_SEGEMPTY + s]);
        ++seg_i;
        return sg.lo >= 0;
    };
    Seg sg;

    if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp == 0 || warp == 3) {
        // ------------------------------------------------------------------ copies: warp 0 Q and K, warp 3 V
        // A key tile is 128 / box boxes of `box` keys (a divisor of the page, so a box lies in one page), one lane each; the
        // page numbers of the next tile are fetched before this one's ring slot is waited for.
        const bool is_v = warp == 3;
        bool bad_page = false, ok = true;
        int jj = 0, qc[2] = {0, 0}, raw = 0, turn = 0;
        auto wait = [&](int bar, uint32_t parity) {
            if (!mbar_wait(&bars[bar], parity, abort_flag, true, 32)) { if (lane == 0) { report(p.status, PT_ERR_DEVICE_TIMEOUT, LOC_CHUNK_WAIT); *abort_flag = 1; } ok = false; }
            ok = __all_sync(0xffffffffu, ok);
            return ok;
        };
        while (ok && next_seg(sg)) {
            const int t = sg.t, kvh = sg.kvh;
            const int32_t* bt = p.bt + (size_t)sg.b * p.maxp;
            auto row_of = [&](int j) {                             // first cache row of this lane's box of tile j
                const int key = j * 128 + lane * box;
                if (lane * box >= 128 || key >= sg.kvlen) return -1;
                int page = bt[key / p.ps];
                if (page < 0 || page >= p.num_pages) { bad_page = true; page = 0; }
                return ((page * 2 + (is_v ? 1 : 0)) * p.nkv + kvh) * p.ps + key % p.ps;
            };
            int row = row_of(sg.lo);
            if (!is_v) {
                const bool one = sg.n1 == 0;                       // one row tile: the two Q buffers take turns
                if (one) turn ^= 1;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if (one ? i != turn : sg.lo >= (i ? sg.n1 : sg.n0)) continue;
                    if (!wait(C_QEMPTY + i, (uint32_t)(qc[i] & 1) ^ 1u)) break;
                    if (lane == 0) {
                        mbar_expect_tx(&bars[C_QFULL + i], q_bytes);
#pragma unroll
                        for (int h = 0; h < HALVES; ++h)
                            tma_load_4d(smem_u32(sq + i * TILE + h * kHalfBytes), &qmap, &bars[C_QFULL + i], h * 64, kvh * G, sg.row0 + (one ? 0 : i) * tpt, t);
                    }
                    ++qc[i];
                }
            }
            for (int j = sg.lo; j < sg.hi && ok; ++j, ++jj) {
                const int key0 = j * 128;
                const int next = j + 1 < sg.hi ? row_of(j + 1) : -1;
                const int ng = min(128 / box, (sg.kvlen - key0 + box - 1) / box);     // boxes of this tile that hold keys
                const uint32_t bytes = (uint32_t)(ng * box) * DH * 2u;
                const int s = jj % (is_v ? kStV : kStK);
                uint8_t* dst = is_v ? sv + s * TILE : sk + s * TILE;
                if (is_v ? !wait(C_VEMPTY + s, (uint32_t)(jj / kStV & 1) ^ 1u) : !wait(C_KEMPTY + s, (uint32_t)(jj / kStK & 1) ^ 1u)) break;
                // rows of the last 16-key group past the last key must read as zero where P (also zero) meets them
                const bool partial = is_v && key0 + 128 > sg.kvlen && ((sg.kvlen - key0) & 15);
                uint64_t* bar = &bars[partial ? C_VRAW : is_v ? C_VFULL + s : C_KFULL + s];
                if (lane == 0) mbar_expect_tx(bar, bytes);
                __syncwarp();
                if (row >= 0) {
#pragma unroll
                    for (int h = 0; h < HALVES; ++h)
                        tma_load_3d(smem_u32(dst + h * kHalfBytes + lane * box * 128), &kvmap, bar, h * 64, row, t);
                }
                if (partial) {
                    if (!wait(C_VRAW, (uint32_t)raw & 1u)) break;
                    ++raw;
                    const int nvalid = sg.kvlen - key0, top = (nvalid + 15) & ~15;
                    for (int idx = lane; idx < (top - nvalid) * HALVES * 8; idx += 32) {
                        const int rr = nvalid + idx / (HALVES * 8), rem = idx % (HALVES * 8);
                        *reinterpret_cast<uint4*>(dst + (rem >> 3) * kHalfBytes + rr * 128 + (rem & 7) * 16) = make_uint4(0, 0, 0, 0);
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bars[C_VFULL + s]);
                }
                row = next;
            }
        }
        if (bad_page) report(p.status, PT_ERR_DEVICE_BOUNDS, LOC_CHUNK_PAGE);
    } else if (warp == 2) {
        // ------------------------------------------------------------------ the walk
        Walk wk;
        bool more = wk.find(p, tpt, sh, gridDim.x, blockIdx.x, blockIdx.x == 0), ok = true;
        if (more) wk.derive(tpt, sh);
        if (lane == 0) {                                           // for the blocks that merge cut segments
            Start st;
            st.p0 = wk.p0; st.u = wk.u; st.len = more ? wk.len : 0;
            st.row0 = wk.qrow0 + wk.tok0; st.t = wk.tk / p.nkv; st.kvh = wk.tk % p.nkv; st.left = wk.qlen - wk.tok0;
            st.n0 = wk.n0; st.n1 = wk.n1; st.lo = wk.lo;
            Slots<DH>{scratch}.start(blockIdx.x)[0] = st;
        }
        for (int i = 0; ok; ++i) {
            while (more && wk.lo >= wk.hi) more = wk.advance(p, tpt, sh);
            const int s = i % kSegRing;
            ok = __all_sync(0xffffffffu, mbar_wait(&bars[C_SEGEMPTY + s], ((uint32_t)(i / kSegRing) & 1u) ^ 1u, abort_flag, true));
            if (!ok) { if (lane == 0) { report(p.status, PT_ERR_DEVICE_TIMEOUT, LOC_CHUNK_WAIT); *abort_flag = 1; } break; }
            if (lane == 0) {
                Seg o;
                o.row0 = wk.qrow0 + wk.tok0; o.t = wk.tk / p.nkv; o.kvh = wk.tk % p.nkv; o.kvlen = wk.kvlen;
                o.pos0 = wk.kvlen - wk.qlen + wk.tok0; o.left = wk.qlen - wk.tok0;
                o.n0 = wk.n0; o.n1 = wk.n1; o.lo = more ? wk.lo : -1; o.hi = wk.hi; o.b = wk.b; o.pad = 0;
                ring[s] = o;
                mbar_arrive(&bars[C_SEGFULL + s]);
            }
            __syncwarp();
            if (!more) break;
            more = wk.advance(p, tpt, sh);
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer
        constexpr uint32_t idesc_qk = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(128 >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
        constexpr uint32_t idesc_pv = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(DH >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
        bool ok = true;
        int jj = 0, qc[2] = {0, 0}, cnt[2] = {0, 0}, turn = 0;
        auto wait = [&](int bar, uint32_t parity) {
            if (!ok) return;
            if (!__all_sync(0xffffffffu, mbar_wait(&bars[bar], parity, abort_flag))) { ok = false; if (lane == 0) { report(p.status, PT_ERR_DEVICE_TIMEOUT, LOC_CHUNK_WAIT); *abort_flag = 1; } }
            tc_fence_after();
        };
        auto qk = [&](int i, int qb, int s, bool last) {           // S_i = Q_qb K_s^T
            if (!ok) return;
            const uint32_t qa = smem_u32(sq + qb * TILE), ka = smem_u32(sk + s * TILE);
            mma_ss_tile<HALVES>(tmem_base + i * 128, desc_kmajor(qa), desc_kmajor(ka), idesc_qk);
            tc_commit(&bars[C_SFULL + i]);
            if (last) tc_commit(&bars[C_QEMPTY + qb]);
        };
        auto pv = [&](int i, int jv, int ng, bool fresh, bool last) {   // O_i (+)= P_i V over the groups that hold keys
            wait(C_PFULL + i, (uint32_t)cnt[i] & 1u);
            ++cnt[i];
            if (!ok) return;
            const uint32_t va = smem_u32(sv + (jv % kStV) * TILE);
            if (ng == 8) mma_ts_tile(tmem_base + 256 + i * DH, tmem_base + i * 128, desc_mnmajor(va), idesc_pv, !fresh);
            else for (int ks = 0; ks < ng; ++ks)
                mma_ts(tmem_base + 256 + i * DH, tmem_base + i * 128 + ks * 8, desc_mnmajor(va + ks * 2048), idesc_pv, !fresh || ks != 0);
            if (last) tc_commit(&bars[C_OREADY + i]);              // before: the next scores say that this product is done
        };
        while (ok && next_seg(sg)) {
            if (sg.n1 == 0) {                                      // one row tile: scores two key tiles ahead, in turns
                turn ^= 1;
                const int qb = turn;
                wait(C_QFULL + qb, (uint32_t)qc[qb] & 1u);
                ++qc[qb];
                for (int j = sg.lo; j < sg.hi + 2 && ok; ++j) {
                    if (j - 2 >= sg.lo) {
                        wait(C_VFULL + jj % kStV, (uint32_t)(jj / kStV) & 1u);
                        pv((j - sg.lo) & 1, jj, min(8, (sg.kvlen - (j - 2) * 128 + 15) >> 4), j - 4 < sg.lo, j >= sg.hi);
                        if (ok) tc_commit(&bars[C_VEMPTY + jj % kStV]);
                        ++jj;
                    }
                    if (j < sg.hi) {
                        const int jk = jj + min(j - sg.lo, 1);          // jj: the tile behind the last product with V
                        wait(C_KFULL + jk % kStK, (uint32_t)(jk / kStK) & 1u);
                        qk((j - sg.lo) & 1, qb, jk % kStK, j + 1 == sg.hi);
                        if (ok) tc_commit(&bars[C_KEMPTY + jk % kStK]);
                    }
                }
                continue;
            }
            const int end[2] = {min(sg.hi, sg.n0), min(sg.hi, sg.n1)};
            wait(C_KFULL + jj % kStK, (uint32_t)(jj / kStK) & 1u);
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (sg.lo < end[i]) { wait(C_QFULL + i, (uint32_t)qc[i] & 1u); ++qc[i]; qk(i, i, jj % kStK, sg.lo + 1 == end[i]); }
            if (ok) tc_commit(&bars[C_KEMPTY + jj % kStK]);
            // What does not depend on the softmax groups is waited for before their P, and a tile's stages are given back
            // behind the next product: between two products the tensor core has nothing to do.
            for (int j = sg.lo; j < sg.hi && ok; ++j, ++jj) {
                const int sn = (jj + 1) % kStK;
                const int ng = min(8, (sg.kvlen - j * 128 + 15) >> 4);
                wait(C_VFULL + jj % kStV, (uint32_t)(jj / kStV) & 1u);
                if (j + 1 < sg.hi) wait(C_KFULL + sn, (uint32_t)((jj + 1) / kStK) & 1u);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if (j < end[i]) pv(i, jj, ng, j == sg.lo, j + 1 == end[i]);
                    if (i == 0 && ok && j > sg.lo) {
                        tc_commit(&bars[C_VEMPTY + (jj - 1) % kStV]);
                        tc_commit(&bars[C_KEMPTY + jj % kStK]);
                    }
                    if (j + 1 < end[i]) qk(i, i, sn, j + 2 == end[i]);
                }
            }
            if (ok) tc_commit(&bars[C_VEMPTY + (jj - 1) % kStV]);
        }
        __syncwarp();
    }
    } else {
        // ------------------------------------------------------------------ softmax groups
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        const int i = (warp - 4) >> 2;                             // group: its row tile, or its share of the key tiles
        const int w4 = warp & 3;                                   // tensor-memory lane quarter of this warp
        const int r = w4 * 32 + lane;                              // row inside the tile: token r / G, head r % G of the group
        const int tok = r / G, gh = r % G;
        const uint32_t t_s = tmem_base + ((uint32_t)(w4 * 32) << 16) + i * 128;
        const uint32_t t_o = tmem_base + ((uint32_t)(w4 * 32) << 16) + 256 + i * DH;
        const float c = p.scale_log2;
        const Slots<DH> slots{scratch};
        bool ok = true;
        int cnt = 0, merges = 0, segs = 0;                         // tiles, one-tile segments, segments with a tile of this group
        auto wait = [&](int bar, uint32_t parity) {
            ok = __all_sync(0xffffffffu, mbar_wait(&bars[bar], parity, abort_flag));
            if (!ok && lane == 0) { report(p.status, PT_ERR_DEVICE_TIMEOUT, LOC_CHUNK_WAIT); *abort_flag = 1; }
            tc_fence_after();
            return ok;
        };
        while (ok && next_seg(sg)) {
            const bool one = sg.n1 == 0;
            const int n_i = !one && i ? sg.n1 : sg.n0, end = min(sg.hi, n_i);
            if (sg.lo >= end) continue;
            const int tok_i = (one ? 0 : i) * tpt;                     // first token of the tile, from the segment's first
            const bool live = tok < tpt && tok_i + tok < sg.left;
            const bool any = __any_sync(0xffffffffu, live);            // a warp without rows only keeps the barriers going
            const int limit = min(sg.pos0 + tok_i + tok, sg.kvlen - 1);  // last visible key of this row
            const int tile_limit = min(sg.pos0 + tok_i, sg.kvlen - 1);   // last visible key of the tile's first row
            const int first = sg.lo + (one ? i : 0), step = one ? 2 : 1;
            float m_ref = -INFINITY, l_run = 0.f;
            for (int j = first; j < end; j += step, ++cnt) {
                if (!wait(C_SFULL + i, (uint32_t)cnt & 1u)) break;
                if (!any) { if (lane == 0) mbar_arrive(&bars[C_PFULL + i]); continue; }
                const int key0 = j * 128;
                float v[128];
#pragma unroll
                for (int cc = 0; cc < 4; ++cc) tm_ld32(t_s + cc * 32, v + cc * 32);
                tm_wait_ld<128>(v);
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
                if (j == first) {
                    m_ref = mx;                                    // -inf where the row sees nothing of this tile
                } else {
                    const bool grow = live && (mx - m_ref) * c > 8.0f;     // also from -inf, when mx is finite
                    if (__any_sync(0xffffffffu, grow)) {
                        // (these scores were issued behind the previous P V, so that has landed)
                        const float corr = grow ? ex2((m_ref - mx) * c) : 1.0f;
                        if (grow) { m_ref = mx; l_run *= corr; }
#pragma unroll 1
                        for (int cc = 0; cc < DH / 32; ++cc) {
                            float o[32];
                            tm_ld32(t_o + cc * 32, o);
                            tm_wait_ld<32>(o);
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
            if (!ok || (first < end && !wait(C_OREADY + i, (uint32_t)segs++ & 1u))) break;
            float m = m_ref * c, f0 = 1.f, f1 = 0.f;                   // the maximum in powers of two, the groups' factors
            if (one) {
                if (i == 1) {
                    odd_stats[r] = make_float2(m, l_run);
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bars[C_MREADY]);
                    if (!wait(C_MDONE, (uint32_t)merges++ & 1u)) break;
                    continue;
                }
                if (!wait(C_MREADY, (uint32_t)merges++ & 1u)) break;
                const float2 odd = odd_stats[r];
                const float top = fmaxf(m, odd.x);
                f0 = m > -INFINITY ? ex2(m - top) : 0.f;
                f1 = odd.x > -INFINITY ? ex2(odd.x - top) : 0.f;
                m = top;
                l_run = l_run * f0 + odd.y * f1;
            }
            // 32 columns of the output, merged
            auto columns = [&](int cc, float* o) {
                tm_ld32(t_o + cc * 32, o);
                if (one && sg.lo + 1 < end) {
                    float o1[32];
                    tm_ld32(t_o + DH + cc * 32, o1);
                    tm_wait_ld<32>(o, o1);
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] = o[e] * f0 + (f1 > 0.f ? o1[e] * f1 : 0.f);
                } else {
                    tm_wait_ld<32>(o);
                }
            };
            if (any) {
            if (sg.lo == 0 && end == n_i) {                        // all of the tile's keys: the result
                const float inv = 1.0f / l_run;                    // every live row sees a key: a sum of 0 or NaN is NaN in the definition too
                __nv_bfloat16* dst = p.o + ((size_t)sg.t * p.M + sg.row0 + tok_i + tok) * (size_t)(p.nq * DH) + (size_t)(sg.kvh * G + gh) * DH;
#pragma unroll 1
                for (int cc = 0; cc < DH / 32; ++cc) {
                    float o[32];
                    columns(cc, o);
                    if (live) {
#pragma unroll
                        for (int e = 0; e < 32; e += 16) {         // whole 32-byte sectors: a warp's store touches 32 rows
                            uint32_t u[8];
#pragma unroll
                            for (int x = 0; x < 8; ++x) u[x] = pack_bf16(o[e + 2 * x] * inv, o[e + 2 * x + 1] * inv);
                            st_global_32(dst + cc * 32 + e, u);
                        }
                    }
                }
            } else {                                               // a part: merged by k_chunk_combine
                const int which = sg.lo > 0 ? 0 : 1;
                const int slot_row = (one ? 0 : i) * 128 + r;
                if (live) slots.stats(blockIdx.x, which)[slot_row] = make_float2(m, l_run);
                float* dst = slots.out(blockIdx.x, which) + slot_row;
#pragma unroll 1
                for (int cc = 0; cc < DH / 32; ++cc) {
                    float o[32];
                    columns(cc, o);
                    if (live) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) dst[(cc * 32 + e) * 256] = o[e];
                    }
                }
            }
            }
            if (one) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars[C_MDONE]);
            }
            tc_fence_before();                                     // the accumulator has been read: the next segment's P may follow
        }
    }
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) settle_copies();
    if (warp == 2) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512) : "memory");
    }
}

// Merges the parts of cut segments.  Block (c, g) handles the segment that is cut at the start of range c + 1, if no earlier
// range's start cuts it too: parts lie in range c (second slot) and, as long as the segment goes on, in c + 1, c + 2, ...
// (first slot).  g: rows 32 g .. 32 g + 31 of its 256, a lane each, 16 columns a warp (128 / 16 warps at most).
constexpr int kCombineThreads = 256;
template <int DH>
__global__ void __launch_bounds__(kCombineThreads)
k_chunk_combine(const ChunkP p, float* scratch, const int tpt, const int blocks, const int sh) {
    grid_dep_wait();
    grid_dep_launch();
    const Slots<DH> at{scratch};
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Start sg = *at.start(blockIdx.x + 1);
    // A lane has the start of range c + base + lane: the ranges of a segment are looked up 32 at a time.
    int base = 0, from_p0, from_len;
    auto look = [&]() {
        const int c = blockIdx.x + base + lane;
        const Start* st = at.start(min(c, blocks - 1));
        from_p0 = st->p0; from_len = c < blocks ? st->len : 0;
    };
    look();
    const int n = max(sg.n0, sg.n1);
    if (sg.len == 0 || sg.lo == 0 || sg.lo >= n) return;           // the segment is not cut at this range's start
    const int seg_start = sg.p0 + sg.u, seg_len = seg_cost(sg.left, n * 128, tpt, sh);
    // first key tile of the segment that belongs to range c + k or a later one (k ascending); behind the last range, all are before
    auto lo_of = [&](int k) {
        if (k - base >= 32) { base = k; look(); }
        const int lo = from_len == 0 ? n : min(n, Walk::first_at(min(from_p0 - seg_start, seg_len), sg.n1 > 0, sh));
        return __shfl_sync(0xffffffffu, lo, k - base);
    };
    if (lo_of(0) > 0) return;                                      // an earlier range's start cuts it already
    const int G = p.nq / p.nkv;
    const int i = blockIdx.y >> 2;                                 // row tile
    const int n_i = i ? sg.n1 : sg.n0;
    if (sg.lo >= n_i) return;                                      // this tile's keys all lie in the first part: written there
    const int r = (blockIdx.y & 3) * 32 + lane, tok = r / G, tok_i = i * tpt;
    const bool live = tok < tpt && tok_i + tok < sg.left;
    const int col = warp * 16;
    if (col >= DH) return;
    float m = -INFINITY, l = 0.f, o[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) o[e] = 0.f;
    constexpr int kAhead = 2;                                      // parts that are loaded before the first of them is merged (4: no faster)
    for (int k = 0, lo = 0; lo < n_i;) {
        float2 st[kAhead];
        float x[kAhead][16];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            const int hi = k == 0 ? sg.lo : lo < n_i ? lo_of(k + 1) : lo;     // tiles [lo, hi) belong to range c + k
            const bool some = lo < min(hi, n_i);
            st[a] = make_float2(-INFINITY, 0.f);
            if (some && live) {
                const int which = k == 0 ? 1 : 0;
                st[a] = at.stats(blockIdx.x + k, which)[i * 128 + r];
                const float* src = at.out(blockIdx.x + k, which) + (size_t)col * 256 + i * 128 + r;
#pragma unroll
                for (int e = 0; e < 16; ++e) x[a][e] = src[e * 256];
            }
            if (lo < n_i) { lo = hi; ++k; }
        }
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            const float top = fmaxf(m, st[a].x);
            if (st[a].x > -INFINITY) {
                const float f0 = exp2f(m - top), f1 = exp2f(st[a].x - top);
                m = top; l = l * f0 + st[a].y * f1;
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] = o[e] * f0 + x[a][e] * f1;
            } else {
                l += st[a].y;                                      // 0, or NaN: the maximum skips scores that are NaN, the sum does not
            }
        }
    }
    if (!live) return;
    const float inv = 1.0f / l;
    uint32_t u[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = pack_bf16(o[2 * e] * inv, o[2 * e + 1] * inv);
    st_global_32(p.o + ((size_t)sg.t * p.M + sg.row0 + tok_i + tok) * (size_t)(p.nq * DH) + (size_t)(sg.kvh * G + r % G) * DH + col, u);
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
    const int kv_box = p.ps % 64 == 0 ? 64 : p.ps % 32 == 0 ? 32 : 16;      // a divisor of the page and of the key tile: fewer, larger copies
    pt_status s = make_map_bf16_strided(&kvmap, p.pool_l, DH, rows, p.T, p.pool_tstride * 2, kv_box);
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
    // no more than this can be asked of a launch: every block of rows with every key that the table can name
    const double most = (double)p.T * p.nkv * ((double)p.M / (2 * tpt) + p.B + 1) * (kSeg2 + 1 + ((double)p.maxp * p.ps / 128 + 1) * kCost2);
    int sh = 0;
    while (most / (double)(1ll << sh) + (double)p.T * p.nkv * ((double)p.M / (2 * tpt) + p.B + 1) > 1e9 && sh < 20) ++sh;
    if (most / (double)(1ll << sh) > 1e9) { set_error("chunk attention: too many sequences, rows or pages for one call"); return PT_ERR_UNSUPPORTED; }
    cudaError_t e = launch_dependent(k_chunk_tc<DH>, dim3(blocks), dim3(kChunkThreads), (size_t)ChunkCfg<DH>::SMEM, st, qmap, kvmap, p, scratch, tpt, (uint32_t)(128 * ChunkCfg<DH>::HALVES * G * box), kv_box, sh);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    if (e == cudaSuccess && blocks > 1) {
        e = launch_dependent(k_chunk_combine<DH>, dim3(blocks - 1, 8), dim3(kCombineThreads), (size_t)0, st, p, scratch, tpt, blocks, sh);
        g_launches.fetch_add(1, std::memory_order_relaxed);
    }
    if (e != cudaSuccess) { set_error("chunk attention launch: %s", cudaGetErrorString(e)); return PT_ERR_CUDA; }
    return PT_OK;
}

}  // namespace

size_t chunk_tc_scratch_bytes(int dh) { return (dh == 64 ? Slots<64>::floats() : Slots<128>::floats()) * 4 * 2 * kMaxBlocks + kMaxBlocks * sizeof(Start); }

pt_status launch_chunk_attn_tc(const ChunkP& p, int dh, void* scratch, cudaStream_t st) {
    return dh == 64 ? launch_t<64>(p, (float*)scratch, st) : launch_t<128>(p, (float*)scratch, st);
}

}  // namespace pt
