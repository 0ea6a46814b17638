// Pages of the KV cache as units of their own: copies inside a pool or between two pools, sequences that share pages
// (fork, copy on write) and compaction.  The paper has no cache; all of this is the library's.
//
// One page id stands for one block in every (track, layer) slab, so "copy page s to page d" is slabs = T * L copies of
// page_bytes each, s and d a fixed distance apart in every slab.  The list of pairs travels in the kernel's parameters
// (no upload, no buffer, and a captured launch keeps its own list).
#include <algorithm>
#include <cstring>
#include <new>
#include <vector>

#include "pt_internal.h"
#include "pt_kernels.h"

namespace pt {

namespace {

constexpr int kPairs = 448;               // pairs per launch: 3.5 KB of the 4 KB of parameters
struct PagePairs { int32_t src[kPairs], dst[kPairs]; };

// A run of equal blocks: block p of slab s at base + s * slab_bytes + p * page_bytes.
struct Plane { const char* src; char* dst; int64_t src_slab, dst_slab; int64_t page_bytes; };

constexpr int kPieceVecs = 4;             // 16-byte loads a lane keeps in flight
constexpr int64_t kPieceBytes = 32 * 16 * kPieceVecs;

// One warp per piece of kPieceBytes of one page of one slab; neighbouring warps take neighbouring pieces.  A plain copy at the
// rate of the HBM: 150 pages of an 8-bit cache (192 slabs, 1.9 GB moved) in 294 us, 1.02 of the measured copy bandwidth; one
// page to 24 (writes all but alone, 0.42 GB) in 68 us, 0.95.  A warp per piece and as many blocks as that takes: with a grid
// of 148 x 8 blocks that loop it was 317 and 78 us (a warp waits for its stores' slots before its next loads), with 148 x 32
// 304 and 71; pieces of 1 KB 335 and 88, of 4 KB in the large grid 295 and 68.
__global__ void __launch_bounds__(256)
k_copy_pages(const Plane pl, const PagePairs pairs, int n, int64_t pieces, int pieces_per_page) {
    const int lane = threadIdx.x & 31;
    const int64_t warps = (int64_t)gridDim.x * (blockDim.x >> 5);
    for (int64_t w = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5); w < pieces; w += warps) {
        const int piece = (int)(w % pieces_per_page);
        const int64_t rest = w / pieces_per_page;
        const int pair = (int)(rest % n);
        const int64_t slab = rest / n;
        const char* s = pl.src + slab * pl.src_slab + pairs.src[pair] * pl.page_bytes;
        char* d = pl.dst + slab * pl.dst_slab + pairs.dst[pair] * pl.page_bytes;
        const int64_t at = piece * kPieceBytes + lane * 16;
        uint4 v[kPieceVecs];
#pragma unroll
        for (int i = 0; i < kPieceVecs; ++i)
            if (at + i * 512 < pl.page_bytes) v[i] = __ldcs(reinterpret_cast<const uint4*>(s + at + i * 512));
#pragma unroll
        for (int i = 0; i < kPieceVecs; ++i)
            if (at + i * 512 < pl.page_bytes) __stcs(reinterpret_cast<uint4*>(d + at + i * 512), v[i]);
    }
}

pt_status copy_plane(const Plane& pl, int64_t slabs, const int32_t* src, const int32_t* dst, int n, cudaStream_t st) {
    if (n == 0) return PT_OK;
    const int per_page = (int)((pl.page_bytes + kPieceBytes - 1) / kPieceBytes);
    for (int i = 0; i < n; i += kPairs) {
        const int m = std::min(kPairs, n - i);
        PagePairs pp;
        std::memcpy(pp.src, src + i, (size_t)m * 4);
        std::memcpy(pp.dst, dst + i, (size_t)m * 4);
        const int64_t pieces = slabs * m * per_page;
        const unsigned blocks = (unsigned)std::min<int64_t>((pieces + 7) / 8, 0x7fffffff);
        k_copy_pages<<<blocks, 256, 0, st>>>(pl, pp, m, pieces, per_page);
        g_launches.fetch_add(1, std::memory_order_relaxed);
    }
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) { set_error("k_copy_pages launch: %s", cudaGetErrorString(e)); return PT_ERR_CUDA; }
    return PT_OK;
}

}  // namespace

pt_status launch_copy_pages(const pt_kv_cache* c, const char* src_pool, const float* src_scales, int32_t src_pages,
                            char* dst_pool, float* dst_scales, int32_t dst_pages, const int32_t* src, const int32_t* dst, int n, cudaStream_t st) {
    const int64_t slabs = (int64_t)c->m->cfg.T * c->m->cfg.L;
    Plane pl{};
    pl.page_bytes = c->page_elems * (int64_t)c->esz;
    pl.src = src_pool; pl.dst = dst_pool; pl.src_slab = src_pages * pl.page_bytes; pl.dst_slab = dst_pages * pl.page_bytes;
    pt_status s = copy_plane(pl, slabs, src, dst, n, st);
    if (s != PT_OK || !src_scales) return s;
    pl.page_bytes = c->page_elems / c->m->dh * 4;
    pl.src = (const char*)src_scales; pl.dst = (char*)dst_scales; pl.src_slab = src_pages * pl.page_bytes; pl.dst_slab = dst_pages * pl.page_bytes;
    return copy_plane(pl, slabs, src, dst, n, st);
}

// Gives sequences pages of their own where the coming call writes: pages that hold positions >= lens[i] of sequence
// seqs[i], up to lens[i] + adds[i].  A shared page whose earlier positions are kept is copied, one that only holds
// positions to be written is replaced.  The last owner of a page keeps it.  `pages_needed` counts the pages taken from
// the free list; plan() changes nothing, commit() moves references and table entries.
void CowPlan::plan(const pt_kv_cache* c, const int32_t* seqs, const int32_t* adds, int n) {
    entries.clear(); src.clear(); dst.clear(); pages_needed = 0;
    std::unordered_map<int32_t, int32_t> left;            // references that remain on a page once the planned entries are done
    for (int i = 0; i < n; ++i) {
        auto it = c->seqs.find(seqs[i]);
        if (it == c->seqs.end() || adds[i] <= 0) continue;
        const Seq& s = it->second;
        const int64_t end = (int64_t)s.len + adds[i];
        for (size_t p = (size_t)(s.len / c->ps); p < s.pages.size() && (int64_t)p * c->ps < end; ++p) {
            const int32_t page = s.pages[p];
            if (c->ref[page] <= 1) continue;
            auto l = left.emplace(page, c->ref[page]).first;
            if (l->second <= 1) continue;
            l->second -= 1;
            const bool keep = (int64_t)p * c->ps < s.len;
            if (++pages_needed > c->free_list.size()) return;     // too many: the call is refused
            const int32_t fresh = c->free_list[pages_needed - 1];
            entries.push_back({seqs[i], (int32_t)p, fresh});
            if (keep) { src.push_back(page); dst.push_back(fresh); }
        }
    }
}

void CowPlan::commit(pt_kv_cache* c) const {
    for (const Entry& e : entries) {
        int32_t& page = c->seqs[e.seq].pages[e.index];
        c->ref[page] -= 1;
        page = e.page;
        c->ref[page] = 1;
        c->free_list.pop_front();
    }
}

}  // namespace pt

using namespace pt;

#define KV_FAIL(code, ...) do { set_error(__VA_ARGS__); return (code); } while (0)
// Host memory that runs out ends a call here, with the cache as it was: what can throw comes before what changes it.
#define KV_CATCH catch (const std::bad_alloc&) { KV_FAIL(PT_ERR_INVALID_ARG, "out of host memory"); }

extern "C" {

pt_status pt_kv_seq_fork(pt_kv_cache* c, int32_t src, int32_t dst, int32_t len) try {
    if (!c) KV_FAIL(PT_ERR_INVALID_ARG, "null argument");
    auto it = c->seqs.find(src);
    if (it == c->seqs.end()) KV_FAIL(PT_ERR_STATE, "unknown sequence %d", src);
    if (dst < 0) KV_FAIL(PT_ERR_INVALID_ARG, "negative sequence id %d", dst);
    if (c->seqs.count(dst)) KV_FAIL(PT_ERR_STATE, "sequence %d exists already", dst);
    if (len < 0 || len > it->second.len) KV_FAIL(PT_ERR_INVALID_ARG, "len %d outside [0, %d]", len, it->second.len);
    Seq s;
    s.len = len;
    s.pages.assign(it->second.pages.begin(), it->second.pages.begin() + (len + c->ps - 1) / c->ps);
    const auto& pages = c->seqs.emplace(dst, std::move(s)).first->second.pages;
    for (int32_t p : pages) c->ref[p] += 1;
    return PT_OK;
} KV_CATCH

pt_status pt_kv_free_pages(const pt_kv_cache* c, int32_t* n) {
    if (!c || !n) KV_FAIL(PT_ERR_INVALID_ARG, "null argument");
    *n = (int32_t)c->free_list.size();
    return PT_OK;
}

pt_status pt_kv_page_refs(const pt_kv_cache* c, int32_t page, int32_t* refs) {
    if (!c || !refs) KV_FAIL(PT_ERR_INVALID_ARG, "null argument");
    if (page < 0 || page >= c->num_pages) KV_FAIL(PT_ERR_INVALID_ARG, "page %d outside [0, %d)", page, c->num_pages);
    *refs = c->ref[page];
    return PT_OK;
}

pt_status pt_kv_compact(pt_kv_cache* c, int32_t* moved, void* stream) try {
    if (!c) KV_FAIL(PT_ERR_INVALID_ARG, "null argument");
    const int32_t used = c->num_pages - (int32_t)c->free_list.size();
    std::vector<int32_t> src, dst, to(c->num_pages, -1);
    int32_t hole = 0;
    for (int32_t p = used; p < c->num_pages; ++p) {
        if (!c->ref[p]) continue;
        while (c->ref[hole]) ++hole;                       // a page below `used` that nobody owns: there is one for each p
        src.push_back(p); dst.push_back(hole);
        to[p] = hole++;
    }
    std::deque<int32_t> free_list;
    for (int32_t p = used; p < c->num_pages; ++p) free_list.push_back(p);
    pt_status s = launch_copy_pages(c, c->pool, c->scales, c->num_pages, c->pool, c->scales, c->num_pages, src.data(), dst.data(), (int)src.size(), (cudaStream_t)stream);
    if (s != PT_OK) return s;
    for (auto& e : c->seqs)
        for (int32_t& p : e.second.pages) if (to[p] >= 0) p = to[p];
    for (size_t i = 0; i < src.size(); ++i) { c->ref[dst[i]] = c->ref[src[i]]; c->ref[src[i]] = 0; }
    c->free_list.swap(free_list);
    if (moved) *moved = (int32_t)src.size();
    return PT_OK;
} KV_CATCH

pt_status pt_kv_move_pool(pt_kv_cache* c, int32_t num_pages, void* dev_pool, size_t bytes, void* stream) try {
    if (!c || !dev_pool) KV_FAIL(PT_ERR_INVALID_ARG, "null argument");
    size_t need = 0, codes = 0;
    pt_status s = kv_pool_layout(c->m, num_pages, c->ps, c->kv_dtype, &codes, &need);
    if (s != PT_OK) return s;
    if (bytes < need) KV_FAIL(PT_ERR_BUFFER_TOO_SMALL, "KV pool: %zu < %zu bytes", bytes, need);
    if ((uintptr_t)dev_pool % 256) KV_FAIL(PT_ERR_MISALIGNED, "KV pool must be 256-byte aligned");
    const int32_t used = c->num_pages - (int32_t)c->free_list.size();
    if (used > num_pages) KV_FAIL(PT_ERR_CACHE_FULL, "%d pages are in use, the new pool holds %d", used, num_pages);
    if ((char*)dev_pool < c->pool + c->bytes && c->pool < (char*)dev_pool + bytes) KV_FAIL(PT_ERR_INVALID_ARG, "the pools overlap");
    std::vector<int32_t> src, dst, to(c->num_pages, -1), ref(num_pages, 0);
    for (int32_t p = 0; p < c->num_pages; ++p)
        if (c->ref[p]) { to[p] = (int32_t)src.size(); ref[src.size()] = c->ref[p]; dst.push_back(to[p]); src.push_back(p); }
    std::deque<int32_t> free_list;
    for (int32_t p = used; p < num_pages; ++p) free_list.push_back(p);
    float* scales = c->scales ? (float*)((char*)dev_pool + codes) : nullptr;
    s = launch_copy_pages(c, c->pool, c->scales, c->num_pages, (char*)dev_pool, scales, num_pages, src.data(), dst.data(), (int)src.size(), (cudaStream_t)stream);
    if (s != PT_OK) return s;
    for (auto& e : c->seqs)
        for (int32_t& p : e.second.pages) p = to[p];
    c->pool = (char*)dev_pool; c->scales = scales; c->bytes = bytes; c->num_pages = num_pages;
    c->slab_elems = c->page_elems * num_pages;
    c->ref.swap(ref);
    c->free_list.swap(free_list);
    return PT_OK;
} KV_CATCH

pt_status pt_kernel_kv_copy_pages(const void* src_pool, int32_t src_pages, void* dst_pool, int32_t dst_pages,
                                  int64_t slabs, int64_t page_bytes, const int32_t* src, const int32_t* dst, int32_t n, void* stream) try {
    if (!src_pool || !dst_pool || n < 0 || (n > 0 && (!src || !dst))) KV_FAIL(PT_ERR_INVALID_ARG, "bad argument");
    if (src_pages < 1 || dst_pages < 1 || slabs < 1 || page_bytes < 16 || page_bytes % 16 || page_bytes > (1 << 30))
        KV_FAIL(PT_ERR_INVALID_ARG, "sizes must be positive, page_bytes a multiple of 16 up to 2^30");
    if (slabs > (1ll << 62) / page_bytes / std::max(src_pages, dst_pages)) KV_FAIL(PT_ERR_INVALID_ARG, "a pool of more than 2^62 bytes");
    if ((uintptr_t)src_pool % 16 || (uintptr_t)dst_pool % 16) KV_FAIL(PT_ERR_MISALIGNED, "pools must be 16-byte aligned");
    const bool same = src_pool == dst_pool;
    if (same && src_pages != dst_pages) KV_FAIL(PT_ERR_INVALID_ARG, "one pool, two page counts");
    const char *a = (const char*)src_pool, *b = (const char*)dst_pool;
    if (!same && a < b + slabs * dst_pages * page_bytes && b < a + slabs * src_pages * page_bytes) KV_FAIL(PT_ERR_INVALID_ARG, "the pools overlap");
    std::vector<uint64_t> written(((size_t)dst_pages + 63) / 64, 0);
    for (int i = 0; i < n; ++i) {
        if (src[i] < 0 || src[i] >= src_pages || dst[i] < 0 || dst[i] >= dst_pages) KV_FAIL(PT_ERR_INVALID_ARG, "pair %d (%d -> %d) is outside the pools", i, src[i], dst[i]);
        uint64_t &w = written[dst[i] >> 6], bit = 1ull << (dst[i] & 63);
        if (w & bit) KV_FAIL(PT_ERR_INVALID_ARG, "page %d is written twice", dst[i]);
        w |= bit;
    }
    for (int i = 0; same && i < n; ++i)
        if (written[src[i] >> 6] >> (src[i] & 63) & 1) KV_FAIL(PT_ERR_INVALID_ARG, "page %d is read and written", src[i]);
    Plane pl{a, (char*)dst_pool, src_pages * page_bytes, dst_pages * page_bytes, page_bytes};
    return copy_plane(pl, slabs, src, dst, n, (cudaStream_t)stream);
} KV_CATCH

}  // extern "C"
