// paged_accept.cu -- the end of a step over a paged cache: greedy acceptance of
// every request, the accepted rows moved within their pages, the lengths
// advanced.
//
// Acceptance is the bitset form of accept.cu: with match the set of nodes whose
// draft token is their parent's greedy token, node i is accepted when
// (anc[i] & ~match & ~root) == 0; the deepest accepted node (smallest id among
// equals) ends the path, which is its ancestor set in increasing order.  Slot
// L + j of every layer and kv head then takes slot L + path[j], through the
// block table.  path is strictly increasing with path[j] >= j, so a thread that
// holds one 16-byte piece of a (layer, kv head, K or V) and goes through j in
// order, a few loads ahead of their stores, reads no slot that it has written.
//
// A cluster of CTAs shares a request: each repeats the (tiny) acceptance, moves
// its share of the pieces, and the first writes the length after all have read
// it (a cluster barrier whose halves lie before and behind the moves), so that the
// lengths may be advanced in place.
#include "paged_q4.cuh"

namespace tv {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxCluster = 8;  // CTAs of a request
constexpr int kAhead = 2, kPieces = 4;  // moves in flight per thread: kAhead of each of kPieces

struct AcceptArgs {
    const TreeDesc *trees;
    int n_trees, batch, max_pages, page_log2, n_rows, vocab;
    const int32_t *tree, *lens, *row_start, *table, *draft, *argmax;
    tb_result *results;
    int32_t *lens_out;
    uint16_t *k, *v;
    long long layer_stride, page_stride, head_stride, slot_stride;  // 2-byte units
    int n_layers, n_pages, Hkv, d, cluster_log2;
    int scale_first, scale_stride;  // 4-bit pages: of a slot's scales in a page's block (slot_stride: of its codes)
};

// What one request accepts; warp 0 of each CTA fills it in.
template <bool kQ4>
struct Accepted {
    int len, bonus, status, L;
    int given;  // the accept_len that a given result says
    bool live;  // the request takes part in the step
    int path[TB_MAX_NODES];
    long long at[TB_MAX_NODES];   // elements from the layer's first head to slot L + j, -1: no such slot
    long long src[TB_MAX_NODES];  // the same for slot L + path[j]
    // 4-bit pages: at and src are of the codes, these of the scales
    long long scale_at[kQ4 ? TB_MAX_NODES : 1], scale_src[kQ4 ? TB_MAX_NODES : 1];
};

// Two round trips: the request's lengths, then its tree, tokens and block table together.
template <bool kQ4>
__device__ void accept_one(const AcceptArgs &p, int b, Accepted<kQ4> &a)
{
    const int lane = threadIdx.x;
    const int t = load_now(p.tree + b), L = load_now(p.lens + b);
    const int row0 = load_now(p.row_start + b), n_here = load_now(p.row_start + b + 1) - row0;
    const bool tree_ok = t >= 0 && t < p.n_trees;
    const TreeDesc *td = p.trees + (tree_ok ? t : 0);
    const int n = load_now(&td->n);
    const tb_result &r = p.results[b];
    const int given = p.draft ? 0 : load_now(&r.accept_len);
    uint64_t anc[2];
    int par[2], dep[2], tok[2], best_tok[2], path[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int i = lane + 32 * h;
        anc[h] = load_now(td->anc + i);
        par[h] = td->parent[i];
        dep[h] = td->depth[i];
        const bool row = p.draft && row0 >= 0 && i < n_here && i < p.n_rows - row0;
        tok[h] = row ? load_now(p.draft + row0 + i) : 0;
        best_tok[h] = row ? load_now(p.argmax + row0 + i) : 0;
        path[h] = p.draft ? 0 : load_now(r.path + i);
    }
    // the pages of slots L .. L + 63, one per lane
    const int mask = (1 << p.page_log2) - 1, first = L >= 0 ? L >> p.page_log2 : 0, in_page = L & mask;
    const int spanned = ((TB_MAX_NODES - 1) >> p.page_log2) + 2;
    const int id = p.k && L >= 0 && lane < spanned && first + lane < p.max_pages
                       ? load_now(p.table + (size_t)b * p.max_pages + first + lane)
                       : -1;
    const auto slot_offset = [&](int j) {  // by the whole warp
        const int x = in_page + j, page = __shfl_sync(0xffffffffu, id, x >> p.page_log2);
        return page < 0 || page >= p.n_pages ? -1ll : page * p.page_stride + (x & mask) * p.slot_stride;
    };

    // a request that paged_plan gave no rows takes no part in the step
    const bool live = tree_ok && L >= 0 && row0 >= 0 && n_here == n && row0 + n <= p.n_rows;
    int len = 0, bonus = -1, status = t >= p.n_trees ? TB_EINVAL : TB_OK;
    if (live && p.draft) {
        bool match[2], badtok[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int i = lane + 32 * h;
            const int of_parent[2] = {__shfl_sync(0xffffffffu, best_tok[0], par[h] & 31),
                                      __shfl_sync(0xffffffffu, best_tok[1], par[h] & 31)};
            badtok[h] = i > 0 && i < n && (tok[h] < 0 || tok[h] >= p.vocab);
            match[h] = i < n && (i == 0 || (!badtok[h] && tok[h] == (par[h] < 32 ? of_parent[0] : of_parent[1])));
        }
        const uint64_t m = (uint64_t)__ballot_sync(0xffffffffu, match[0]) |
                           ((uint64_t)__ballot_sync(0xffffffffu, match[1]) << 32);
        if (__any_sync(0xffffffffu, badtok[0] || badtok[1]))
            status = TB_EINVAL;
        // the deepest accepted node, smallest id among equals
        int best = -1;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int i = lane + 32 * h;
            if (i < n && (anc[h] & ~m) == 0)
                best = max(best, dep[h] * 64 + 63 - i);
        }
        best = __reduce_max_sync(0xffffffffu, best);
        const int j = 63 - (best & 63);
        const uint64_t on = __shfl_sync(0xffffffffu, j < 32 ? anc[0] : anc[1], j & 31);
        len = __popcll(on);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int i = lane + 32 * h;
            if ((on >> i) & 1)
                a.path[__popcll(on & ((1ull << i) - 1))] = i;
        }
        bonus = __shfl_sync(0xffffffffu, j < 32 ? best_tok[0] : best_tok[1], j & 31);
    } else if (live) {
        len = min(max(given, 0), n);
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (lane + 32 * h < len)
                a.path[lane + 32 * h] = min(max(path[h], lane + 32 * h), n - 1);
    }
    __syncwarp();
    if (p.k && live) {
        bool hole = false;  // in the table, where a row should move from or to
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int j = lane + 32 * h, from = j < len ? a.path[j] : j;
            const long long at = slot_offset(j), src = slot_offset(from);
            if constexpr (kQ4) {
                const auto scales = [&](int j, long long codes) {
                    return codes + p.scale_first + ((in_page + j) & mask) * (p.scale_stride - p.slot_stride);
                };
                a.scale_at[j] = scales(j, at);
                a.scale_src[j] = scales(from, src);
            }
            if (j < len) {
                a.at[j] = at;
                a.src[j] = from == j ? -1 : src;  // in place already: nothing moves
                hole |= from != j && (at < 0 || src < 0);
            }
        }
        if (__any_sync(0xffffffffu, hole))
            status = TB_EINVAL;
    }
    if (lane == 0) {
        a.len = len;
        a.bonus = bonus;
        a.status = status;
        a.L = L;
        a.given = given;
        a.live = live;
    }
}

// Pieces of a head's row that a thread moves: 16 bytes, and in 4-bit pages the scales of 2 or 4.
template <bool kQ4>
__host__ __device__ constexpr unsigned pieces_of(int d)
{
    return kQ4 ? code_bytes(d) / 16 + 1 : d / 8;
}

// This CTA's share of the accepted rows.
template <bool kQ4>
__device__ __forceinline__ void move_rows(const AcceptArgs &p, const Accepted<kQ4> &a, int rank)
{
    if (!p.k || a.len < 2)
        return;
    // pieces of one (layer, kv head, K or V), several per thread in flight
    const unsigned per_head = p.d == 64 ? pieces_of<kQ4>(64) : pieces_of<kQ4>(128);
    const unsigned pieces = 2u * p.n_layers * p.Hkv * per_head;  // < 2^30 (the host's check)
    const unsigned stride = (unsigned)kThreads << p.cluster_log2;
    for (unsigned x0 = rank * kThreads + threadIdx.x; x0 < pieces; x0 += kPieces * stride) {
        uint16_t *base[kPieces];
        bool scales[kPieces];
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const unsigned x = x0 + i * stride, y = p.d == 64 ? x / pieces_of<kQ4>(64) : x / pieces_of<kQ4>(128);
            const unsigned c = x - y * per_head;
            const unsigned lv = y / (unsigned)p.Hkv, g = y - lv * (unsigned)p.Hkv;
            scales[i] = kQ4 && c == per_head - 1;
            base[i] = x < pieces ? ((lv & 1) ? p.v : p.k) + (lv >> 1) * p.layer_stride + g * p.head_stride +
                                       (scales[i] ? 0 : 8 * c)
                                 : nullptr;
        }
        for (int j0 = 1; j0 < a.len; j0 += kAhead) {
            uint4 buf[kPieces][kAhead];
            long long src[kAhead], at[kAhead], scale_src[kAhead], scale_at[kAhead];
#pragma unroll
            for (int m = 0; m < kAhead; ++m) {
                const int j = j0 + m;
                const bool move = j < a.len && a.src[j] >= 0 && a.at[j] >= 0;
                src[m] = move ? a.src[j] : -1;
                at[m] = move ? a.at[j] : -1;
                scale_src[m] = kQ4 && move ? a.scale_src[j] : 0;
                scale_at[m] = kQ4 && move ? a.scale_at[j] : 0;
            }
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
#pragma unroll
                for (int m = 0; m < kAhead; ++m)
                    if (src[m] >= 0 && base[i]) {
                        if (!scales[i])
                            buf[i][m] = *reinterpret_cast<const uint4 *>(base[i] + src[m]);
                        else if (p.d == 128)
                            buf[i][m].x = *reinterpret_cast<const uint32_t *>(base[i] + scale_src[m]);
                        else
                            buf[i][m].x = base[i][scale_src[m]];
                    }
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
#pragma unroll
                for (int m = 0; m < kAhead; ++m)
                    if (at[m] >= 0 && base[i]) {
                        if (!scales[i])
                            *reinterpret_cast<uint4 *>(base[i] + at[m]) = buf[i][m];
                        else if (p.d == 128)
                            *reinterpret_cast<uint32_t *>(base[i] + scale_at[m]) = buf[i][m].x;
                        else
                            base[i][scale_at[m]] = (uint16_t)buf[i][m].x;
                    }
        }
    }
}

// Bound by the latency of the chain lengths, tree and tokens and table, rows (one
// request of two layers: 2.8 us; 3.6 with each of these loads behind the one before);
// with many requests by the scattered 128- or 256-byte rows, read and written (64
// requests of 32 layers and 8 heads, 36 MB: 9.4 us, 3.8 TB/s; 512 of them 50 us, 5.0).
// In 4-bit pages a row is 64 bytes of codes and 4 of scales: the same 64 requests
// 7.8 us; 8.8 to 9.8 with four or eight rows of fewer pieces in flight.
template <bool kQ4>
__global__ void __launch_bounds__(kThreads) k_paged_accept(const __grid_constant__ AcceptArgs p)
{
    __shared__ Accepted<kQ4> a;
    pdl_wait();
    pdl_trigger();
    const int b = blockIdx.x >> p.cluster_log2, rank = blockIdx.x & ((1 << p.cluster_log2) - 1);
    if (threadIdx.x < 32)
        accept_one(p, b, a);
    __syncthreads();
    cluster_arrive();  // this CTA has read the request's length and result
    move_rows(p, a, rank);
    cluster_wait();  // and so have the others, which frees them to be written
    if (rank == 0) {
        tb_result &r = p.results[b];
        if (p.draft) {
            if (threadIdx.x < TB_MAX_NODES)
                r.path[threadIdx.x] = threadIdx.x < a.len ? a.path[threadIdx.x] : 0;
            if (threadIdx.x == 0) {
                r.accept_len = a.len;
                r.bonus_token = a.bonus;
                r.status = a.status;
            }
        } else {
            if (a.given != a.len) {
                // cut off, or left there by an earlier step for a request that takes no part in this one
                if (threadIdx.x < TB_MAX_NODES && !a.live)
                    r.path[threadIdx.x] = 0;
                if (threadIdx.x == 0) {
                    r.accept_len = a.len;
                    if (!a.live)
                        r.bonus_token = -1;
                }
            }
            if (threadIdx.x == 0 && a.status != TB_OK)
                r.status = a.status;
        }
        if (threadIdx.x == 0) {
            r.new_L = a.L + a.len;
            p.lens_out[b] = a.L + a.len;
        }
    }
}

// What both calls do once the pages are checked and put into `a` (a.k NULL: none).
template <bool kQ4>
tb_status accept_requests(AcceptArgs &a, const tb_requests *req, const int32_t *draft_tokens, const int32_t *argmax,
                          int n_rows, int vocab, tb_result *results, int32_t *lens_out, tb_stream stream, const char *fn)
{
    a.batch = req->batch;
    a.max_pages = req->max_pages;
    while ((1 << a.page_log2) < req->page_size)
        ++a.page_log2;
    a.n_rows = n_rows;
    a.vocab = vocab;
    a.tree = req->tree;
    a.lens = req->lens;
    a.row_start = req->row_start;
    a.table = req->table;
    a.draft = draft_tokens;
    a.argmax = argmax;
    a.results = results;
    a.lens_out = lens_out;
    // as many CTAs per request as it has rounds of pieces, or while there are SMs for them one piece per
    // thread (512 requests of 8 layers: 16.6 us, 33 with 8 CTAs each; 8 of them 3.5 us, 4.3 with 2)
    const int n_sm = device_sms(-1);
    if (n_sm <= 0)
        return record_error(TB_ECUDA, "%s: no current device", fn);
    const long long pieces = a.k ? 2ll * a.n_layers * a.Hkv * pieces_of<kQ4>(a.d) : 0;
    int cluster = 1;
    while (cluster < kMaxCluster && cluster * kThreads * (req->batch * cluster < n_sm / 2 ? 1 : kPieces) < pieces)
        cluster *= 2;
    while ((1 << a.cluster_log2) < cluster)
        ++a.cluster_log2;
    return launch_result(launch_kernel_cluster(k_paged_accept<kQ4>, dim3(req->batch * cluster), dim3(kThreads), 0,
                                               (cudaStream_t)stream, true, cluster, a),
                         fn);
}

tb_status check_accept(AcceptArgs &a, const tb_bank *bank, const tb_requests *req, const int32_t *draft_tokens,
                       const int32_t *argmax, int n_rows, int vocab, const tb_result *results, const int32_t *lens_out,
                       const char *fn)
{
    tb_status st = check_device_bank(bank, fn, &a.trees, &a.n_trees);
    if (st != TB_OK || (st = check_requests(req, true, fn)) != TB_OK)
        return st;
    if (!req->tree)
        return record_error(TB_EINVAL, "%s: req->tree is NULL", fn);
    if (!results || !lens_out)
        return record_error(TB_EINVAL, "%s: results or lens_out is NULL", fn);
    if (draft_tokens && (!argmax || vocab < 1))
        return record_error(TB_EINVAL, "%s: argmax is NULL or vocab %d < 1", fn, vocab);
    if (n_rows < 0)
        return record_error(TB_EINVAL, "%s: n_rows %d", fn, n_rows);
    return TB_OK;
}

// Pages of a table whose pages have page_size slots.
template <typename Pages>
tb_status check_fit(const Pages *pages, const tb_requests *req, const char *fn)
{
    if (pages->page_size != req->page_size)
        return record_error(TB_EINVAL, "%s: pages of %d slots, a table of %d", fn, pages->page_size, req->page_size);
    if ((long long)pages->n_layers * pages->n_kv_heads > 1 << 24)
        return record_error(TB_EUNSUPPORTED, "%s: %d layers of %d kv heads", fn, pages->n_layers, pages->n_kv_heads);
    return TB_OK;
}

}  // namespace

TB_BOUNDS_COUNTER(bounds_violations_paged_accept)

}  // namespace tv

using namespace tv;

extern "C" tb_status paged_accept(const tb_bank *bank, const tb_requests *req, const tb_pages *pages,
                                  const int32_t *draft_tokens, const int32_t *argmax, int n_rows, int vocab,
                                  tb_result *results, int32_t *lens_out, tb_stream stream)
{
    const char *fn = "paged_accept";
    AcceptArgs a{};
    tb_status st = check_accept(a, bank, req, draft_tokens, argmax, n_rows, vocab, results, lens_out, fn);
    if (st != TB_OK)
        return st;
    if (pages) {
        if ((st = check_pages(pages, fn)) != TB_OK || (st = check_fit(pages, req, fn)) != TB_OK)
            return st;
        a.k = static_cast<uint16_t *>(pages->k);
        a.v = static_cast<uint16_t *>(pages->v);
        a.layer_stride = pages->layer_stride;
        a.page_stride = pages->page_stride;
        a.head_stride = pages->head_stride;
        a.slot_stride = pages->slot_stride;
        a.n_layers = pages->n_layers;
        a.n_pages = pages->n_pages;
        a.Hkv = pages->n_kv_heads;
        a.d = pages->head_dim;
    }
    return accept_requests<false>(a, req, draft_tokens, argmax, n_rows, vocab, results, lens_out, stream, fn);
}

extern "C" tb_status paged_accept_q4(const tb_bank *bank, const tb_requests *req, const tb_pages_q4 *pages,
                                     const int32_t *draft_tokens, const int32_t *argmax, int n_rows, int vocab,
                                     tb_result *results, int32_t *lens_out, tb_stream stream)
{
    const char *fn = "paged_accept_q4";
    AcceptArgs a{};
    tb_status st = check_accept(a, bank, req, draft_tokens, argmax, n_rows, vocab, results, lens_out, fn);
    if (st != TB_OK)
        return st;
    if (pages) {
        if ((st = check_pages_q4(pages, fn)) != TB_OK || (st = check_fit(pages, req, fn)) != TB_OK)
            return st;
        a.k = static_cast<uint16_t *>(pages->k);
        a.v = static_cast<uint16_t *>(pages->v);
        a.layer_stride = pages->layer_stride / 2;
        a.page_stride = pages->page_stride / 2;
        a.head_stride = pages->head_stride / 2;
        a.slot_stride = code_bytes(pages->head_dim) / 2;
        a.scale_first = pages->page_size * code_bytes(pages->head_dim) / 2;
        a.scale_stride = scale_bytes(pages->head_dim) / 2;
        a.n_layers = pages->n_layers;
        a.n_pages = pages->n_pages;
        a.Hkv = pages->n_kv_heads;
        a.d = pages->head_dim;
    }
    return accept_requests<true>(a, req, draft_tokens, argmax, n_rows, vocab, results, lens_out, stream, fn);
}
