// Attention of one or a few new tokens per sequence straight from a 4-bit cache (pt_kv_dtype PT_KV_E2M1).
//
//   out[r] = sum_j 2^(s_rj - m_r) v_j / sum_j 2^(s_rj - m_r),   s_rj = log2(e) / sqrt(dh) q_r . k_j,
//   k_j[d] = code * scale of d's group of 32, v_j likewise; r runs over the (token, head) rows of a sequence and KV head.
//
// What bounds it: 17 bytes bring 32 values, so at the copy rate an SM has 2.3 cycles for every 100 values, and the codes'
// way into the matrix instructions takes more than that.  No unit is full (256 ragged sequences, 149 us: issue slots 57 %, ALU 57,
// tensor pipe 28, DRAM 60; 4 x 5 tokens of 9-31k keys, 75 us: 41, 32, 37, 26): the time is that of dependent steps, with three
// warps a scheduler to cover them, or two.  So:
//  * The products run on mma.sync m16n8k16 in f16 with the cached vectors on the 16-row side and the rows r on the 8-column
//    side: K^T q and V^T p take their 4-bit operand from registers, where cvt.rn.f16x2.e2m1x2 puts two codes an instruction.
//    (tcgen05 takes its operands from shared memory or tensor memory: 4-bit codes would be converted in registers all the
//    same, written and fetched again, and its block scales are powers of two, which these are not.  With one row tile that looks
//    like more work than it takes away.  With several, where K's codes are converted and scaled once for all rows here too, it
//    would take the products and the accumulators off the warps.  Neither is built or measured.)
//  * The order of a block of 16 tokens is that of the instruction's operands: a lane loads its codes of K (two tokens, 32 dims
//    each) and V (four tokens, 16 dims each) with 128-bit loads free of bank conflicts.  Of V a byte holds two dims of one
//    token and the operand wants two tokens of one dim: eight codes of two tokens change places in four instructions.
//  * A scale of K multiplies the partial score of its group in fp32 (with several row tiles: its codes, exactly), a scale of V
//    the weights, once for 32 dims.  Weight times scale is one f16 number, kept within f16's normal range from both sides: the
//    weights' reference (m above) lags behind the maximum by up to 2^6, so that a part's largest weight is 2^8 to 2^14, and the
//    scales of a group of 32 columns are divided by a power of two that puts the largest of the tile's into [2^-5, 2).  (So 2^-28 of
//    the row's largest weight times that scale is the least that f16 holds; 256 ragged sequences take 149.5 us with it and 148.9
//    with the scales as they are, which loses the small weights behind a dominant key.)  The fp32
//    sums of the group carry that power and are rescaled, exactly, where it changes, which in ordinary data is once a segment.
//    q is divided by a power of two that puts a row's largest magnitude at 2^13, K codes are below 8, sums are fp32.
//  * A warp works alone: a ring of 32-key stages filled by bulk copies (a block of 16 tokens, K, V and scales, is one piece
//    of 17 * dh bytes), its own plan from the device's lengths, its own contiguous share of all key tiles of the call, so
//    that no barrier stands in the loop and a captured call may be replayed with other lengths.  A segment (sequence, track, KV
//    head, a block of 8, 16 or 24 rows, the last one shorter) that is cut leaves parts (sums, reference): those of a block's warps
//    are merged in its shared memory, those of several blocks by k_kv4_merge.  Twelve warps of 168 registers with one and two row
//    tiles, eight of up to 255 with three.
#include <algorithm>
#include <type_traits>

#include "pt_kv4.cuh"
#include "pt_tc.h"
#include "pt_ring.cuh"

namespace pt {

namespace {

constexpr int kTile = 32;                 // keys a warp takes at a time: two blocks of 16
constexpr int kMaxBlocks = 160;           // thread blocks whose parts the scratch has room for
constexpr int kSegCost = 2;               // cost of beginning a segment, in tiles
constexpr int kWholeTiles = 3;            // tiles of a warp up to which a block takes a whole segment: 1000 keys 11.1 us (12.8 cut up), 1500 keys 12.8 (12.0)
constexpr uint32_t kSpin = 1u << 24;
constexpr float kTop = 14.f, kStart = 8.f; // weights stay below 2^kTop; a reference is set so that the largest is 2^kStart
// V's unit 2^e of a group (e >= -14): the tile's largest scale of the group is in [2^(e - kBand), 2^(e + 1)), as fp16 bits in the
// upper half of a word from (e + 15 - kBand) << 26 on
constexpr int kBand = 5;
constexpr uint32_t kBandBits = (uint32_t)(kBand + 1) << 26;
constexpr float kNone = -3.0e38f;         // reference of a row that has seen nothing

// Warps and ring stages (32 keys each at head_dim 128) by row tiles: what registers (168 a lane with 12 warps, 255 with 8) and
// shared memory allow.  256 ragged sequences with one tile: 12 x 3 148 us; 16 x 2, which spills, 147 (but 301 keys 1 us more);
// 14 x 2 173, 10 x 4 180, 8 x 5 177 - warps have to divide evenly among the four schedulers.
template <int DH, int NT> struct Cfg {
    static constexpr int NG = DH / 32, RB = 8 * NT, BLK = kv4_block(DH);
    static constexpr int WARPS = NT <= 2 ? 12 : 8, STAGES = (NT == 2 ? 2 : 3) * (128 / DH), THREADS = WARPS * 32;
    // several tiles: queries in shared memory instead of registers, and head parts in the scratch instead of there
    static constexpr bool QS = NT > 1;
    // K's scales multiply its codes, 64 instructions a tile, instead of the partial scores, 32 for each row tile (20 rows: 84 to 82 us)
    static constexpr bool KOP = NT > 1;
    static constexpr int SCALE_BYTES = kTile * NG * 6;                     // a tile's scales, decoded: K as fp32, V as fp16 pairs
    static constexpr int STAGE = 2 * BLK, ROW = DH + 4, PART = RB * ROW + 2 * RB;      // floats of a part: rows, then (reference, sum) of each
    static constexpr int RING = STAGES * STAGE > PART * 4 ? STAGES * STAGE : PART * 4;  // bytes of a warp's ring, which its last part takes when it is empty
    static constexpr int HEADS = WARPS * RING, SCALES = HEADS + (QS ? 0 : WARPS * PART * 4), QUERIES = SCALES + WARPS * SCALE_BYTES, BARS = QUERIES + (QS ? WARPS * NG * NT * 512 : 0);
    static constexpr int SMEM = BARS + WARPS * STAGES * 8;
    static_assert(SMEM <= 227 * 1024 - 6144, "shared memory");
};

// A segment: the (token, head) rows [r0, r0 + rows) of one sequence, track and KV head, with the keys they see.
struct SegInfo { int t, h, row0, r0, rows; };
// What a thread block leaves for the merge: a part whose segment began before it (head) and one that goes on behind it (tail).
struct Leftover { int head, tail, tail_begins; SegInfo seg; };

template <int DH, int NT> struct Scratch {
    using C = Cfg<DH, NT>;
    static constexpr int PART = C::RB * (DH + 2);                          // floats of a block's part: rows, then (reference, sum) of each
    static constexpr size_t bytes = (size_t)kMaxBlocks * (64 + 2 * PART * 4 + (C::QS ? C::WARPS * C::PART * 4 : 0));
    char* p;
    __device__ explicit Scratch(void* p_) : p((char*)p_) {}
    __device__ Leftover* left() const { return (Leftover*)p; }
    __device__ float* part(int block, int which) const { return (float*)(p + kMaxBlocks * 64) + (size_t)(2 * block + which) * PART; }
    // head part of a warp: its ring is still in use
    __device__ float* head(int block, int warp, uint8_t* smem) const {
        if (!C::QS) return (float*)(smem + C::HEADS) + warp * C::PART;
        return (float*)(p + kMaxBlocks * (64 + 2 * PART * 4)) + (size_t)(block * C::WARPS + warp) * C::PART;
    }
};

__device__ __forceinline__ float ex2f(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t half2_of(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t mul2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
// K's scales of a word as the scores take them, in order: fp32, or (OP: they multiply the operand) fp16 pairs of 2^-4 of each,
// which keeps six times the largest inside fp16 and the product with a code exact
template <bool OP> __device__ __forceinline__ void k_scales(uint32_t even, uint32_t odd, uint32_t* f) {
    if constexpr (OP) {
        even = mul2(even, 0x2c002c00u);
        odd = mul2(odd, 0x2c002c00u);
        f[0] = __byte_perm(even, even, 0x1010); f[1] = __byte_perm(odd, odd, 0x1010);
        f[2] = __byte_perm(even, even, 0x3232); f[3] = __byte_perm(odd, odd, 0x3232);
    } else {
        const float2 a = __half22float2(*reinterpret_cast<__half2*>(&even)), b = __half22float2(*reinterpret_cast<__half2*>(&odd));
        f[0] = __float_as_uint(a.x); f[1] = __float_as_uint(b.x); f[2] = __float_as_uint(a.y); f[3] = __float_as_uint(b.y);
    }
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
__device__ __forceinline__ void mma(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// the same with an accumulator of zeros
__device__ __forceinline__ void mma0(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// four scale bytes (low first) -> fp16 pairs (bytes 0 and 2), (bytes 1 and 3)
__device__ __forceinline__ void scales4(uint32_t w, uint32_t& even, uint32_t& odd) { even = (w << 7) & 0x7f807f80u; odd = (w >> 1) & 0x7f807f80u; }
// the largest of them, in the upper half of a word whose lower half is below every border of a comparison
__device__ __forceinline__ uint32_t top_scale(uint32_t even, uint32_t odd) {
    const uint32_t m = __vmaxu2(even, odd);
    return __vmaxu2(m, m << 16);
}
template <int N> __device__ __forceinline__ void lds(uint32_t at, uint32_t* w) {
    if constexpr (N == 4) asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at));
    else if constexpr (N == 2) asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at));
    else asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(at));
}
__device__ __forceinline__ void bulk_copy(uint32_t dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
}

// Where a warp is in the list of segments: (track, KV head), sequence, row block; and which of the segment's tiles are its own.
struct Cursor {
    int th, b, rb, row0, S, K, seen, n, lo, hi;   // row0: the sequence's first row; seen: keys that the block's last row sees; n: tiles of those
    long long left;                               // units of cost of the warp's range behind this segment's
};

template <int DH, int NT> struct Walk {
    static constexpr int RB = Cfg<DH, NT>::RB;
    const Kv4AttnP& p;
    const int G;
    const bool whole;                             // a block takes one whole segment
    __device__ Walk(const Kv4AttnP& p_, bool w) : p(p_), G(p_.nq / p_.slab.nkv), whole(w) {}
    __device__ int seen(int S, int K, int rb) const { return (rb + 1) * RB >= S * G ? K : K - S + ((rb + 1) * RB - 1) / G + 1; }
    __device__ void load(int b, int& S, int& K) const { S = p.qlen ? p.qlen[b] : 1; K = p.kvlen[b]; }
    __device__ int cost(int seen) const { return whole ? 1 : (seen + kTile - 1) / kTile + kSegCost; }
    // of all row blocks of a sequence (the host has checked that those of all sequences fit)
    __device__ int cost(int S, int K) const {
        int n = 0;
        for (int rb = 0; rb * RB < S * G; ++rb) n += cost(seen(S, K, rb));
        return n;
    }
    // the cursor at unit `in` of its segment; takes what the range has of it
    __device__ void enter(Cursor& c, int in) const {
        c.seen = seen(c.S, c.K, c.rb);
        c.n = (c.seen + kTile - 1) / kTile;
        const int take = (int)min((long long)(c.n + kSegCost - in), c.left);
        c.lo = max(0, in - kSegCost);
        c.hi = max(0, in + take - kSegCost);
        c.left -= take;
    }
    // to the next segment of the range with tiles in it; false: there is none
    __device__ bool next(Cursor& c) const {
        while (c.left > 0) {
            if (++c.rb * RB >= c.S * G) {
                c.rb = 0;
                do {
                    c.row0 += c.S;
                    if (++c.b == p.B) { c.b = 0; ++c.th; c.row0 = 0; }
                    load(c.b, c.S, c.K);
                } while (c.S == 0);
            }
            enter(c, 0);
            if (c.lo < c.hi) return true;
        }
        return false;
    }
    // Every warp plans for itself: a lane sums the costs of 1 / 32 of the sequences, the lane in whose sum the warp's range
    // begins is found by a ballot, and its sequences are looked through the same way.  false: nothing to do (or `bad` lengths)
    __device__ bool plan(Cursor& c, bool& bad) const {
        const int lane = threadIdx.x & 31, per = (p.B + 31) / 32;
        int mine = 0, S = 0, K = 0;
        long long rows = 0;
        bad = false;
        for (int b = lane * per; b < min(p.B, (lane + 1) * per); ++b) {
            load(b, S, K);
            if (S < 0 || K < S || S > p.M || K > (long long)p.maxp * p.slab.ps) { bad = true; break; }
            rows += S;
            mine += cost(S, K);
        }
        int up = kv4_scan(mine);
        long long up_rows = 0;
        if (p.qlen) up_rows = kv4_scan(rows);
        bad = __any_sync(0xffffffffu, bad) || __shfl_sync(0xffffffffu, up_rows, 31) > p.M;
        const int per_head = __shfl_sync(0xffffffffu, up, 31);
        const long long units = (long long)per_head * p.slab.nkv * p.T;
        if (bad || units == 0) return false;
        // the call's units go in equal shares to the warps of as many blocks as have one for each warp
        constexpr int W = Cfg<DH, NT>::WARPS;
        long long u0 = blockIdx.x;
        if (whole) {
            if (u0 >= units) return false;
        } else {
            const int all = (int)min((long long)gridDim.x, (units + W - 1) / W) * W, gw = blockIdx.x * W + (threadIdx.x >> 5);
            if (gw >= all) return false;
            const long long share = kv4_quotient(units, all), more = units - share * all;
            u0 = share * gw + min((long long)gw, more);
            c.left = share + (gw < more);
            if (c.left == 0) return false;
        }
        c.th = (int)kv4_quotient(u0, per_head);
        int in = (int)(u0 - (long long)c.th * per_head);
        const int l = __popc(__ballot_sync(0xffffffffu, up <= in));
        in -= __shfl_sync(0xffffffffu, up - mine, l);
        c.row0 = p.qlen ? (int)__shfl_sync(0xffffffffu, up_rows - rows, l) : l * per;
        int at = l;
        if (per > 1) {
            for (int b0 = l * per;; b0 += 32) {
                const int b = b0 + lane;
                S = K = 0;
                if (b < min(p.B, (l + 1) * per)) load(b, S, K);
                mine = cost(S, K);
                up = kv4_scan(mine);
                at = __popc(__ballot_sync(0xffffffffu, up <= in));
                int sum = lane < at ? S : 0;
#pragma unroll
                for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                c.row0 += sum;
                if (at < 32) { c.b = b0 + at; break; }
                in -= __shfl_sync(0xffffffffu, up, 31);
            }
            in -= __shfl_sync(0xffffffffu, up - mine, at);
        } else {
            c.b = l;
        }
        c.S = __shfl_sync(0xffffffffu, S, at);
        c.K = __shfl_sync(0xffffffffu, K, at);
        for (c.rb = 0;; ++c.rb) {
            const int n = cost(seen(c.S, c.K, c.rb));
            if (in < n) break;
            in -= n;
        }
        if (whole) {                                               // its tiles in equal shares to the block's warps
            const int w = threadIdx.x >> 5;
            c.seen = seen(c.S, c.K, c.rb);
            c.n = (c.seen + kTile - 1) / kTile;
            c.lo = (int)((long long)c.n * w / W); c.hi = (int)((long long)c.n * (w + 1) / W);
            c.left = 0;
            return c.lo < c.hi;
        }
        enter(c, in);
        return c.lo < c.hi || next(c);
    }
};

template <int DH, int NT>
__global__ void __launch_bounds__(Cfg<DH, NT>::THREADS, 1) k_kv4_attn(const Kv4AttnP p, void* scratch, const bool whole) {
    using C = Cfg<DH, NT>;
    constexpr int NG = C::NG, RB = C::RB;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ SegInfo info[C::WARPS][2];
    __shared__ Cursor cursors[C::WARPS][2];               // of what is computed, of what is fetched: read at a segment's ends only
    __shared__ int flags[C::WARPS];                       // bit 0: a head part, 1: a tail part, 2: the tail's segment begins here
    __shared__ float factor[RB][32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, q4 = lane & 3;
    uint64_t* bars = (uint64_t*)(smem + C::BARS) + warp * C::STAGES;
    if (lane == 0) {
        for (int i = 0; i < C::STAGES; ++i) mbar_init(&bars[i], 2);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    grid_dep_wait();
    grid_dep_launch();
    const Walk<DH, NT> walk(p, whole);
    const int G = walk.G, nkv = p.slab.nkv, ps = p.slab.ps;
    const Scratch<DH, NT> sc(scratch);
    Cursor cur{};
    bool bad = false, any = walk.plan(cur, bad);
    if (bad) {                                            // every warp of the call finds the same
        if (tid == 0) { report(p.status, PT_ERR_DEVICE_BOUNDS, LOC_KV4_LEN); sc.left()[blockIdx.x] = Leftover{}; }
        return;
    }
    // ---- the ring: lanes 0 and 1 fetch a block of 16 keys each; pages are looked up one tile ahead
    uint8_t* ring = smem + warp * C::RING;
    if (lane == 0) cursors[warp][0] = cursors[warp][1] = cur;
    __syncwarp();
    // the next segment of a cursor; registers hold no more of it than its tiles need
    auto step = [&](Cursor& at, bool& some) {
        Cursor c = at;
        __syncwarp();
        some = walk.next(c);
        if (lane == 0) at = c;
        __syncwarp();
        return c;
    };
    const int bpp = ps / 16, step_col = 2 / bpp, step_in = 2 % bpp;            // blocks of a page: 1 .. 4
    const uint32_t page_bytes = (uint32_t)nkv * bpp * C::BLK;
    int a_tile = 0, a_hi = 0, a_seen = 0, a_col = 0, a_in = 0, a_page = -1;
    bool a_any = any, bad_page = false;
    const char* a_base = nullptr;                         // the head's first block in page 0
    const int32_t* a_bt = nullptr;
    auto look = [&]() { if (lane < 2 && a_tile * kTile + 16 * lane < a_seen) a_page = a_bt[a_col]; };
    auto aim = [&](const Cursor& ahead) {
        const int t = ahead.th / nkv, h = ahead.th - t * nkv, blk = 2 * ahead.lo + lane;
        a_base = p.slab.pool_l + (size_t)t * p.slab.tstride + (size_t)h * bpp * C::BLK;
        a_bt = p.bt + (size_t)ahead.b * p.maxp;
        a_tile = ahead.lo; a_hi = ahead.hi; a_seen = ahead.seen;
        a_col = blk / bpp; a_in = blk - a_col * bpp;
        look();
    };
    auto issue = [&](int slot) {
        if (lane < 2) {                                   // each expects its own bytes: none behind the last key
            const bool some = a_tile * kTile + 16 * lane < a_seen, go = some && (uint32_t)a_page < (uint32_t)p.slab.num_pages;
            bad_page |= some != go;
            mbar_expect_tx(&bars[slot], go ? C::BLK : 0);
            if (go) bulk_copy(smem_u32(ring + slot * C::STAGE + lane * C::BLK), a_base + (uint64_t)(uint32_t)a_page * page_bytes + a_in * C::BLK, C::BLK, &bars[slot]);
        }
        if (++a_tile == a_hi) {
            const Cursor c = step(cursors[warp][1], a_any);
            if (a_any) aim(c);
        } else {
            a_col += step_col; a_in += step_in;
            if (a_in >= bpp) { a_in -= bpp; ++a_col; }
            look();
        }
    };
    // a segment's queries, of row tile nt: lane (g, q4) has row g's octet q4 of every group
    uint4 raw[NG];
    auto fetch = [&](const Cursor& cur, int nt) {
        const int t = cur.th / nkv, h = cur.th - t * nkv;
        const int r = cur.rb * RB + nt * 8 + g, tok = r / G;
        const __nv_bfloat16* src = p.q + (((size_t)t * p.M + cur.row0 + tok) * p.nq + h * G + (r - tok * G)) * DH + 8 * q4;
#pragma unroll
        for (int j = 0; j < NG; ++j) raw[j] = r < cur.S * G ? *reinterpret_cast<const uint4*>(src + 32 * j) : make_uint4(0, 0, 0, 0);
    };
    if (a_any) { aim(cur); fetch(cur, 0); }
    __syncwarp();
    for (int s = 0; s < C::STAGES; ++s) if (a_any) issue(s);

    int slot = 0, my_flags = 0, pending = 0;              // pending: tiles of the range that a wait that gave up has left
    uint32_t parity = 0;
    bool timed_out = false;
    while (any && !timed_out) {
        // ---- a segment: its queries
        uint32_t qf[C::QS ? 1 : NG][C::QS ? 1 : NT][4];
        const uint32_t qs = smem_u32(smem + C::QUERIES + warp * NG * NT * 512 + lane * 16);
        float unit[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            if (nt) fetch(cursors[warp][0], nt);
            uint32_t top = 0;
#pragma unroll
            for (int j = 0; j < NG; ++j) {
                const uint32_t w[4] = {raw[j].x, raw[j].y, raw[j].z, raw[j].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) top = __vmaxu2(top, w[i] & 0x7fff7fffu);
            }
            top = max(top & 0xffffu, top >> 16);
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            // divided by the power of two that puts the row's largest magnitude into [2^13, 2^14)
            int e = (int)(top >> 7) - 127;
            if (top >= 0x7f80u) e = 13;                   // not finite: as it is
            e = max(e, -100);
            const float inv = __uint_as_float((uint32_t)(13 - e + 127) << 23);
            const float un = __uint_as_float((uint32_t)(e - 13 + 127) << 23) * (C::KOP ? 16.f * p.scale_log2 : p.scale_log2);
#pragma unroll
            for (int j = 0; j < NG; ++j) {
                const uint32_t w[4] = {raw[j].x, raw[j].y, raw[j].z, raw[j].w};
                uint32_t f[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) f[i] = half2_of(__uint_as_float(w[i] << 16) * inv, __uint_as_float(w[i] & 0xffff0000u) * inv);
                if constexpr (C::QS) {                            // read back by the lane that wrote it
                    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(qs + (j * NT + nt) * 512), "r"(f[0]), "r"(f[1]), "r"(f[2]), "r"(f[3]) : "memory");
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) qf[j][nt][i] = f[i];
                }
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) unit[nt][c] = __shfl_sync(0xffffffffu, un, (2 * q4 + c) * 4);
        }
        const int seen = cursors[warp][0].seen, hi = cursors[warp][0].hi, all_see = cursors[warp][0].K - cursors[warp][0].S + cursors[warp][0].rb * RB / G + 1;
        float o[NG][2][NT][4] = {}, ref[NT][2], l[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) { ref[nt][c] = kNone; l[nt][c] = 0.f; }
        int e_v = -14;                                            // V's unit of group lane % NG
        uint32_t inv_v = 0x74007400u;                             // 2^-e_v, an fp16 pair
        for (int tile = cursors[warp][0].lo; tile < hi; ++tile) {
            bool ok = mbar_try(&bars[slot], parity);
            if (!__all_sync(0xffffffffu, ok)) {
                WaitClock clock;
                for (uint32_t spin = 0; spin < kSpin && !ok; ++spin) {
                    ok = mbar_try(&bars[slot], parity);
                    if ((spin & 255) == 255 && clock.expired()) break;
                }
                if (!__all_sync(0xffffffffu, ok)) { timed_out = true; pending = hi - tile; break; }
            }
            const uint32_t base = smem_u32(ring + slot * C::STAGE), dec = smem_u32(smem + C::SCALES + warp * C::SCALE_BYTES);
            const int key0 = tile * kTile;
            // ---- the tile's scales, each decoded once: lane l has key l's of K and word l (block, q, group) of V's
            uint32_t high;
            bool over;                                            // a scale of V out of its unit's band
            {
                const int hb = lane >> 4, l = lane & 15;
                uint32_t kb = 0, vb = 0, even, odd, f[4];
                if constexpr (NG == 4) {
                    lds<1>(base + hb * C::BLK + kv4_codes(DH) + l * 4, &kb);
                    lds<1>(base + hb * C::BLK + 2 * kv4_codes(DH) + kv4_scales(DH) + l * 4, &vb);
                    if (key0 + kTile > seen) {                    // nothing behind the last key counts
                        const int nv = min(max(seen - (key0 + 16 * hb + (l & ~3)), 0), 4);
                        vb &= nv == 4 ? 0xffffffffu : (1u << (8 * nv)) - 1u;
                    }
                    scales4(kb, even, odd);
                    k_scales<C::KOP>(even, odd, f);
                    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(dec + lane * 16), "r"(f[0]), "r"(f[1]), "r"(f[2]), "r"(f[3]) : "memory");
                    scales4(vb, even, odd);
                    asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(dec + kTile * 16 + lane * 8), "r"(mul2(even, inv_v)), "r"(mul2(odd, inv_v)) : "memory");
                } else if (l < 8) {                               // two groups: a word of K's has two keys, eight words of V's are a block's
                    lds<1>(base + hb * C::BLK + kv4_codes(DH) + l * 4, &kb);
                    lds<1>(base + hb * C::BLK + 2 * kv4_codes(DH) + kv4_scales(DH) + l * 4, &vb);
                    if (key0 + kTile > seen) {
                        const int nv = min(max(seen - (key0 + 16 * hb + 4 * (l >> 1)), 0), 4);
                        vb &= nv == 4 ? 0xffffffffu : (1u << (8 * nv)) - 1u;
                    }
                    scales4(kb, even, odd);
                    k_scales<C::KOP>(even, odd, f);
                    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(dec + (hb * 8 + l) * 16), "r"(f[0]), "r"(f[1]), "r"(f[2]), "r"(f[3]) : "memory");
                    scales4(vb, even, odd);
                    asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(dec + kTile * 8 + (hb * 8 + l) * 8), "r"(mul2(even, inv_v)), "r"(mul2(odd, inv_v)) : "memory");
                } else {
                    even = odd = 0;
                }
                high = vb;
                const uint32_t top = top_scale(even, odd);        // of four keys: seldom out of the band where the tile's is in it
                over = top && top - ((uint32_t)(e_v + 15 - kBand) << 26) >= kBandBits;
                __syncwarp();
            }
            // ---- scores
            float s[2][NT][4];
#pragma unroll
            for (int hb = 0; hb < 2; ++hb) {
                const uint32_t kb = base + hb * C::BLK;
                uint32_t kw[2][NG], ks[2 * NG];
                lds<NG>(kb + g * (DH / 2) + q4 * (DH / 8), kw[0]);
                lds<NG>(kb + (g + 8) * (DH / 2) + q4 * (DH / 8), kw[1]);
                lds<NG>(dec + (16 * hb + 2 * g) * NG * 4, ks);
                lds<NG>(dec + (16 * hb + 2 * g + 1) * NG * 4, ks + NG);
#pragma unroll
                for (int j = 0; j < NG; ++j) {
                    uint32_t h0[4], h1[4];
                    kv4_codes8(kw[0][j], h0);
                    kv4_codes8(kw[1][j], h1);
                    if constexpr (C::KOP) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) { h0[i] = mul2(h0[i], ks[j]); h1[i] = mul2(h1[i], ks[NG + j]); }
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float c[4];
                        uint32_t f[4];
                        if constexpr (C::QS) {
                            lds<4>(qs + (j * NT + nt) * 512, f);
                        } else {
#pragma unroll
                            for (int i = 0; i < 4; ++i) f[i] = qf[j][nt][i];
                        }
                        if constexpr (C::KOP) {
                            if (j) mma(s[hb][nt], h0[0], h1[0], h0[1], h1[1], f[0], f[1]);
                            else mma0(s[hb][nt], h0[0], h1[0], h0[1], h1[1], f[0], f[1]);
                            mma(s[hb][nt], h0[2], h1[2], h0[3], h1[3], f[2], f[3]);
                        } else {
                            mma0(c, h0[0], h1[0], h0[1], h1[1], f[0], f[1]);
                            mma(c, h0[2], h1[2], h0[3], h1[3], f[2], f[3]);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const float f = __uint_as_float(ks[(i >> 1) * NG + j]);
                                s[hb][nt][i] = j ? fmaf(c[i], f, s[hb][nt][i]) : c[i] * f;
                            }
                        }
                    }
                }
            }
            // ---- weights 2^(score - reference).  The reference lags behind the maximum: it is raised, and what has been summed
            // scaled down, only where a weight would pass 2^kTop
            if (key0 + kTile > all_see) {                         // some row does not see all of the tile
                const Cursor& at = cursors[warp][0];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int end = at.K - at.S + min((at.rb * RB + nt * 8 + 2 * q4 + c) / G, at.S - 1) + 1 - key0 - 2 * g;
#pragma unroll
                        for (int hb = 0; hb < 2; ++hb)
#pragma unroll
                            for (int i = 0; i < 2; ++i)
                                if (16 * hb + i >= end) s[hb][nt][2 * i + c] = -INFINITY;
                    }
                // a group of V that is not finite must not meet the weights 0 of rows that do not see it: its codes are 0, its
                // scale is made 0, and the others' sums become NaN here
                const uint32_t nan = __vcmpeq4(high, 0xffffffffu);
                if (__any_sync(0xffffffffu, nan != 0)) {
                    uint32_t even, odd;
                    high &= ~nan;
                    scales4(high, even, odd);
                    const int hb = lane >> 4, l = lane & 15;
                    if (l < 4 * NG) asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(dec + kTile * NG * 4 + (hb * 4 * NG + l) * 8), "r"(mul2(even, inv_v)), "r"(mul2(odd, inv_v)) : "memory");
                    __syncwarp();
                    const int mine = nan ? 16 * hb + l / NG * 4 + (__ffs(nan) - 1) / 8 : kTile;
#pragma unroll
                    for (int j = 0; j < NG; ++j) {
                        const int first = __reduce_min_sync(0xffffffffu, l % NG == j ? mine : kTile);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int c = 0; c < 2; ++c)
                                if (first < kTile && key0 + first <= at.K - at.S + min((at.rb * RB + nt * 8 + 2 * q4 + c) / G, at.S - 1)) {
#pragma unroll
                                    for (int mt = 0; mt < 2; ++mt) o[j][mt][nt][c] = o[j][mt][nt][2 + c] = __uint_as_float(0x7fffffffu);
                                }
                    }
                }
            }
            float mx[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    mx[nt][c] = fmaxf(fmaxf(s[0][nt][c], s[0][nt][2 + c]), fmaxf(s[1][nt][c], s[1][nt][2 + c]));
                    over = over || fmaf(mx[nt][c], unit[nt][c], -ref[nt][c]) > kTop;
                }
            if (__any_sync(0xffffffffu, over)) {
                // V's units: those whose band the tile's largest scale (a NaN does not count) has left move there
                float shift[NG];
                {
                    uint32_t even, odd;
                    scales4(high & ~__vcmpeq4(high, 0xffffffffu), even, odd);
                    uint32_t top = top_scale(even, odd);
#pragma unroll
                    for (int m = NG; m < 32; m <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, m));
                    const int was = e_v;
                    if (top && top - ((uint32_t)(e_v + 15 - kBand) << 26) >= kBandBits) {
                        e_v = max((int)(top >> 26) - 15, -14);
                        inv_v = (e_v < 15 ? (uint32_t)(15 - e_v) << 10 : 0x200u) * 0x10001u;
                    }
#pragma unroll
                    for (int j = 0; j < NG; ++j) shift[j] = __uint_as_float((uint32_t)(__shfl_sync(0xffffffffu, was - e_v, j) + 127) << 23);
                    scales4(high, even, odd);
                    const int hb = lane >> 4, l = lane & 15;
                    if (l < 4 * NG) asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(dec + kTile * NG * 4 + (hb * 4 * NG + l) * 8), "r"(mul2(even, inv_v)), "r"(mul2(odd, inv_v)) : "memory");
                    __syncwarp();
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float corr[2];
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float m = mx[nt][c];
                        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
                        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
                        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16)) * unit[nt][c];
                        float nr = ref[nt][c];
                        if (m - nr > kTop) nr = m - kStart;
                        corr[c] = ex2f(ref[nt][c] - nr);
                        l[nt][c] *= corr[c];
                        ref[nt][c] = nr;
                    }
#pragma unroll
                    for (int j = 0; j < NG; ++j)
#pragma unroll
                        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                            for (int i = 0; i < 4; ++i) o[j][mt][nt][i] *= corr[i & 1] * shift[j];
                }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
#pragma unroll
                    for (int hb = 0; hb < 2; ++hb) s[hb][nt][i] = ex2f(fmaf(s[hb][nt][i], unit[nt][i & 1], -ref[nt][i & 1]));
                    l[nt][i & 1] += s[0][nt][i] + s[1][nt][i];
                }
            // ---- weights times V
#pragma unroll
            for (int hb = 0; hb < 2; ++hb) {
                const uint32_t vb = base + hb * C::BLK + kv4_codes(DH) + kv4_scales(DH);
                uint32_t b0[NT], b1[NT], vs[2 * NG];              // scales of keys 4 q4 + (0, 2) and + (1, 3), group by group
#pragma unroll
                for (int i = 0; i < NG / 2; ++i) lds<4>(dec + kTile * NG * 4 + (hb * 4 + q4) * NG * 8 + i * 16, vs + 4 * i);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    b0[nt] = transpose8x8(half2_of(s[hb][nt][0], s[hb][nt][1]));
                    b1[nt] = transpose8x8(half2_of(s[hb][nt][2], s[hb][nt][3]));
                }
                uint32_t x[4][NG / 2];                            // codes of keys 4 q4 + i
                if constexpr (NG == 4) {
                    uint32_t w[4];
                    lds<4>(vb + lane * 16, w);
                    x[0][0] = w[0]; x[0][1] = w[1]; x[1][0] = w[2]; x[1][1] = w[3];
                    lds<4>(vb + 512 + lane * 16, w);
                    x[2][0] = w[0]; x[2][1] = w[1]; x[3][0] = w[2]; x[3][1] = w[3];
                } else {
                    uint32_t w[4];
                    lds<4>(vb + lane * 16, w);
                    x[0][0] = w[0]; x[1][0] = w[1]; x[2][0] = w[2]; x[3][0] = w[3];
                }
#pragma unroll
                for (int jj = 0; jj < NG / 2; ++jj) {
                    constexpr uint32_t m = 0x0f0f0f0fu;
                    uint32_t a0[4], a1[4], a2[4], a3[4];          // byte e / 2 of group 2 jj, then of group 2 jj + 1
                    kv4_codes8((x[0][jj] & m) | ((x[2][jj] << 4) & ~m), a0);
                    kv4_codes8(((x[0][jj] >> 4) & m) | (x[2][jj] & ~m), a1);
                    kv4_codes8((x[1][jj] & m) | ((x[3][jj] << 4) & ~m), a2);
                    kv4_codes8(((x[1][jj] >> 4) & m) | (x[3][jj] & ~m), a3);
#pragma unroll
                    for (int jl = 0; jl < 2; ++jl) {
                        const int j = 2 * jj + jl;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            const uint32_t p0 = mul2(b0[nt], vs[2 * j]), p1 = mul2(b1[nt], vs[2 * j + 1]);
                            mma(o[j][0][nt], a0[2 * jl], a1[2 * jl], a2[2 * jl], a3[2 * jl], p0, p1);
                            mma(o[j][1][nt], a0[2 * jl + 1], a1[2 * jl + 1], a2[2 * jl + 1], a3[2 * jl + 1], p0, p1);
                        }
                    }
                }
            }
            __syncwarp();                                         // every lane is done with the slot
            if (a_any) { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); issue(slot); }
            if (++slot == C::STAGES) { slot = 0; parity ^= 1; }
        }
        if (timed_out) break;
        // ---- the end of the piece
        float unit_v[NG];
#pragma unroll
        for (int j = 0; j < NG; ++j) unit_v[j] = __uint_as_float((uint32_t)(__shfl_sync(0xffffffffu, e_v, j) + 127) << 23);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int m = 4; m < 32; m <<= 1) l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], m);
        const Cursor at = cursors[warp][0];
        const int t = at.th / nkv, h = at.th - t * nkv, r0 = at.rb * RB;
        const bool begins = at.lo == 0, ends = at.hi == at.n;
        const SegInfo si{t, h, at.row0, r0, min(RB, at.S * G - r0)};
        if (begins && ends) {                                     // all of the segment's keys: the result
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int r = nt * 8 + 2 * q4 + c;
                    if (r >= si.rows) continue;
                    const int tok = (r0 + r) / G, hd = r0 + r - tok * G;
                    const float inv = 1.0f / l[nt][c];
                    __nv_bfloat16* dst = p.o + (((size_t)t * p.M + si.row0 + tok) * p.nq + h * G + hd) * DH + 4 * g;
#pragma unroll
                    for (int j = 0; j < NG; ++j) {
                        const float f = inv * unit_v[j];
                        *reinterpret_cast<uint2*>(dst + 32 * j) = make_uint2(kv4_bf16(o[j][0][nt][c] * f, o[j][0][nt][2 + c] * f),
                                                                            kv4_bf16(o[j][1][nt][c] * f, o[j][1][nt][2 + c] * f));
                    }
                }
        } else {                                                  // a part: merged below, or by k_kv4_merge
            float* part = ends ? sc.head(blockIdx.x, warp, smem) : (float*)ring;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int r = nt * 8 + 2 * q4 + c;
#pragma unroll
                    for (int j = 0; j < NG; ++j)
                        *reinterpret_cast<float4*>(part + r * C::ROW + 32 * j + 4 * g) = make_float4(o[j][0][nt][c] * unit_v[j], o[j][0][nt][2 + c] * unit_v[j], o[j][1][nt][c] * unit_v[j], o[j][1][nt][2 + c] * unit_v[j]);
                    if (g == 0) { part[RB * C::ROW + 2 * r] = ref[nt][c]; part[RB * C::ROW + 2 * r + 1] = l[nt][c]; }
                }
            my_flags |= ends ? 1 : begins ? 6 : 2;
            if (lane == 0) info[warp][ends ? 0 : 1] = si;
        }
        const Cursor c = step(cursors[warp][0], any);
        if (any) fetch(c, 0);
    }
    if (timed_out) {
        while (pending < C::STAGES) {                     // the ring is kept as full as the range's rest allows
            const Cursor c = step(cursors[warp][0], any);
            if (!any) break;
            pending += c.hi - c.lo;
        }
        drain_ring(bars, C::STAGES, slot, pending);
        if (lane == 0) report(p.status, PT_ERR_DEVICE_TIMEOUT, LOC_KV4_WAIT);
        my_flags = 0;
    }
    if (bad_page) report(p.status, PT_ERR_DEVICE_BOUNDS, LOC_KV4_PAGE);
    if (lane == 0) flags[warp] = my_flags;
    __syncthreads();

    // ---- parts of one segment side by side in this block's warps: to the result, or to one part for the merge.
    // Lane 2 w + 0 / 1 stands for warp w's head / tail; parts of one segment (a chain) follow one another
    static_assert(2 * C::WARPS <= 32, "a lane for each part");
    const int fl = lane < 2 * C::WARPS ? flags[lane >> 1] : 0;
    const bool exists = lane & 1 ? (fl & 2) != 0 : (fl & 1) != 0;
    const uint32_t members = __ballot_sync(0xffffffffu, exists), closers = members & 0x55555555u;
    const uint32_t begins = __ballot_sync(0xffffffffu, exists && (lane & 1) && (fl & 4));
    if (members) {
        const uint32_t starts = begins | (members & (0u - members));
        // last lane of the chain that begins in lane f
        auto last_of = [&](int f) {
            const uint32_t c = closers >> f;
            return c ? f + __ffs(c) - 1 : 31 - __clz(members);
        };
        auto part_of = [&](int l) { return l & 1 ? (const float*)(smem + (l >> 1) * C::RING) : (const float*)sc.head(blockIdx.x, l >> 1, smem); };
        const uint32_t before = starts & ((2u << lane) - 1u);
        const int mine_first = before ? 31 - __clz(before) : lane, mine_last = exists ? last_of(mine_first) : lane;
        const bool whole = ((begins >> mine_first) & 1) && !(mine_last & 1);      // the chain has all of the segment's keys
        for (int r = warp; r < RB; r += C::WARPS) {
            float m = kNone, sum = 0.f;
            if (exists) { const float2 st = *reinterpret_cast<const float2*>(part_of(lane) + RB * C::ROW + 2 * r); m = st.x; sum = st.y; }
            float top = m;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const float x = __shfl_up_sync(0xffffffffu, top, o);
                if (lane - o >= mine_first) top = fmaxf(top, x);
            }
            top = __shfl_sync(0xffffffffu, top, mine_last);
            const float f = ex2f(m - top);
            sum *= f;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const float x = __shfl_up_sync(0xffffffffu, sum, o);
                if (lane - o >= mine_first) sum += x;
            }
            sum = __shfl_sync(0xffffffffu, sum, mine_last);
            factor[r][lane] = whole ? f / sum : f;
            if (exists && !whole && lane == mine_last) {
                float* to = sc.part(blockIdx.x, lane & 1) + RB * DH + 2 * r;
                to[0] = top; to[1] = sum;
            }
        }
        __syncthreads();
        // a warp per chain and row
        uint32_t rest = starts;
        for (int task = warp, chain = 0; rest; task += C::WARPS) {
            while (rest && task >= (chain + 1) * RB) { rest &= rest - 1; ++chain; }
            if (!rest) break;
            const int r = task - chain * RB, first = __ffs(rest) - 1, last = last_of(first);
            const SegInfo si = info[first >> 1][first & 1];
            if (r >= si.rows) continue;
            const uint32_t chain_of = members & ((2u << last) - 1u) & ~((1u << first) - 1u);
            constexpr int V = DH / 32;                            // columns of a lane
            using Vec = std::conditional_t<V == 4, float4, float2>;
            alignas(16) float acc[V] = {};
#pragma unroll(C::QS ? 4 : 2 * C::WARPS)
            for (int l = 0; l < 2 * C::WARPS; ++l) {              // straight-line: all loads in flight at once
                Vec x{};
                float f = 0.f;
                if ((chain_of >> l) & 1) { f = factor[r][l]; x = *reinterpret_cast<const Vec*>(part_of(l) + r * C::ROW + lane * V); }
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] += f * reinterpret_cast<const float*>(&x)[i];
            }
            if (((begins >> first) & 1) && !(last & 1)) {
                const int tok = (si.r0 + r) / G, hd = si.r0 + r - tok * G;
                __nv_bfloat16* dst = p.o + (((size_t)si.t * p.M + si.row0 + tok) * p.nq + si.h * G + hd) * DH + lane * V;
#pragma unroll
                for (int i = 0; i < V; i += 2) *reinterpret_cast<uint32_t*>(dst + i) = kv4_bf16(acc[i], acc[i + 1]);
            } else {
                *reinterpret_cast<Vec*>(sc.part(blockIdx.x, last & 1) + r * DH + lane * V) = *reinterpret_cast<const Vec*>(acc);
            }
        }
    }
    if (tid == 0) {
        Leftover left{};
        if (members) {
            const int top = 31 - __clz(members), low = __ffs(members) - 1;
            const uint32_t starts = begins | (1u << low);
            // the first chain is cut at its front unless it begins here; the last is cut at its end unless a head closes it
            if (!((begins >> low) & 1) && closers) left.head = __ffs(closers) - 1 < (begins ? __ffs(begins) - 1 : 32);
            if (top & 1) {
                const int first = 31 - __clz(starts);
                left.tail = 1; left.tail_begins = (begins >> first) & 1; left.seg = info[first >> 1][first & 1];
            }
        }
        sc.left()[blockIdx.x] = left;
    }
}

// Merges the parts of the segments that thread blocks cut: block (c, r) has row r of the segment that begins in block c and
// goes on behind it.
constexpr int kMergeThreads = 256;
template <int DH, int NT>
__global__ void __launch_bounds__(kMergeThreads) k_kv4_merge(const Kv4AttnP p, void* scratch, const int blocks) {
    constexpr int WARPS = kMergeThreads / 32, RB = Cfg<DH, NT>::RB, V = DH / 32;      // columns of a lane
    using Vec = std::conditional_t<V == 4, float4, float2>;
    __shared__ __align__(16) float sums[WARPS][DH];
    __shared__ float tops[WARPS], dens[WARPS];
    grid_dep_wait();
    grid_dep_launch();
    const Scratch<DH, NT> sc(scratch);
    const int r = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c0 = blockIdx.x;
    const Leftover first = sc.left()[c0];
    if (!first.tail || !first.tail_begins || r >= first.seg.rows) return;
    // the block that ends the segment: the first behind c0 with a head
    int last = blocks - 1;
    for (int base = c0 + 1; base < blocks; base += 32) {
        const uint32_t heads = __ballot_sync(0xffffffffu, base + lane < blocks && sc.left()[base + lane].head);
        if (heads) { last = base + __ffs(heads) - 1; break; }
    }
    float top = kNone, sum = 0.f;
    alignas(16) float acc[V] = {};
#pragma unroll 4
    for (int c = c0 + warp; c <= last; c += WARPS) {               // tails, and the last one's head: a warp each
        const float* part = sc.part(c, c == last ? 0 : 1);
        const float2 st = *reinterpret_cast<const float2*>(part + RB * DH + 2 * r);
        const Vec x = *reinterpret_cast<const Vec*>(part + r * DH + lane * V);
        const float nt = fmaxf(top, st.x), f0 = ex2f(top - nt), f1 = ex2f(st.x - nt);
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] = acc[i] * f0 + reinterpret_cast<const float*>(&x)[i] * f1;
        sum = sum * f0 + st.y * f1;
        top = nt;
    }
    *reinterpret_cast<Vec*>(&sums[warp][lane * V]) = *reinterpret_cast<const Vec*>(acc);
    if (lane == 0) { tops[warp] = top; dens[warp] = sum; }
    __syncthreads();
    const int d = threadIdx.x;
    if (d >= DH) return;
    float all = kNone, o = 0.f;
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < WARPS; ++i) all = fmaxf(all, tops[i]);
#pragma unroll
    for (int i = 0; i < WARPS; ++i) {
        const float f = ex2f(tops[i] - all);
        o += sums[i][d] * f;
        sum += dens[i] * f;
    }
    const int G = p.nq / p.slab.nkv, tok = (first.seg.r0 + r) / G, hd = first.seg.r0 + r - tok * G;
    p.o[(((size_t)first.seg.t * p.M + first.seg.row0 + tok) * p.nq + first.seg.h * G + hd) * DH + d] = __float2bfloat16_rn(o / sum);
}

template <int DH, int NT> pt_status launch_t(const Kv4AttnP& p, void* scratch, cudaStream_t st) {
    using C = Cfg<DH, NT>;
    // units of one head are counted in 32 bits: every block of rows with every key that the table can name
    const double most = ((double)p.M * (p.nq / p.slab.nkv) / C::RB + p.B) * ((double)p.maxp * p.slab.ps / kTile + 1 + kSegCost);
    if (most > 2e9) { set_error("4-bit attention: too many sequences, rows or pages for one call"); return PT_ERR_UNSUPPORTED; }
    const double bytes = (double)p.T * p.M * p.nq * DH * 2;
    if (kv4_meet(p.q, bytes, p.o, bytes)) { set_error("out must not overlap q"); return PT_ERR_INVALID_ARG; }
    static int sms_[kMaxDevices] = {};
    int& sms = sms_[current_device()];
    if (!sms) {
        int n = 0;
        cudaError_t e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, current_device());
        if (e == cudaSuccess) e = cudaFuncSetAttribute(k_kv4_attn<DH, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
        if (e != cudaSuccess) { set_error("4-bit attention setup: %s", cudaGetErrorString(e)); return PT_ERR_CUDA; }
        sms = n;
    }
    const int blocks = std::min(sms, kMaxBlocks);
    // Few segments of few keys: a block for each, and no second launch
    const double segments = ((double)p.M * (p.nq / p.slab.nkv) / C::RB + p.B) * p.slab.nkv * p.T;
    const bool whole = segments <= blocks && (int64_t)p.maxp * p.slab.ps <= kWholeTiles * kTile * C::WARPS;
    cudaError_t e = launch_dependent(k_kv4_attn<DH, NT>, dim3(whole ? (unsigned)segments : blocks), dim3(C::THREADS), (size_t)C::SMEM, st, p, scratch, whole);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    if (e == cudaSuccess && !whole && blocks > 1) {
        e = launch_dependent(k_kv4_merge<DH, NT>, dim3(blocks - 1, p.qlen ? C::RB : p.nq / p.slab.nkv), dim3(kMergeThreads), (size_t)0, st, p, scratch, blocks);
        g_launches.fetch_add(1, std::memory_order_relaxed);
    }
    if (e != cudaSuccess) { set_error("4-bit attention launch: %s", cudaGetErrorString(e)); return PT_ERR_CUDA; }
    return PT_OK;
}

}  // namespace

template <int NT> constexpr size_t scratch_of(int dh) { return dh == 64 ? Scratch<64, NT>::bytes : Scratch<128, NT>::bytes; }
size_t kv4_attn_scratch_bytes(int dh) { return std::max(scratch_of<1>(dh), std::max(scratch_of<2>(dh), scratch_of<3>(dh))); }

template <int DH> static pt_status launch_dh(const Kv4AttnP& p, void* scratch, cudaStream_t st) {
    return p.tiles <= 1 ? launch_t<DH, 1>(p, scratch, st) : p.tiles == 2 ? launch_t<DH, 2>(p, scratch, st) : launch_t<DH, 3>(p, scratch, st);
}

// The mean number of rows of a sequence in as few passes over its keys as can be, in equal shares: up to three tiles of 8 rows a
// pass.  (Four sequences of 20k keys, 4 tracks, 4 KV heads: 44, 66 and 83 us a pass of 1, 2 and 3 tiles; with four, whose
// accumulators take 128 registers a lane, 134 us, as much as two passes of two.)
int kv4_mean_tiles(int64_t rows, int B) {
    const int64_t eights = ((rows + B - 1) / B + 7) / 8, passes = (eights + 2) / 3;
    return (int)((eights + passes - 1) / passes);
}

pt_status launch_kv4_attn(const Kv4AttnP& p, int dh, void* scratch, cudaStream_t st) {
    return dh == 64 ? launch_dh<64>(p, scratch, st) : launch_dh<128>(p, scratch, st);
}

}  // namespace pt
