// paged_plan.cu -- the step of a batch laid out on the GPU from its lengths:
// pages taken and given back, row offsets, slots, positions, and the work split
// of the paged attention.
//
// With n[b] the tokens that request b brings and P the page size,
//   need[b] = ceil((len[b] + n[b]) / P),  take[b] = max(0, need - held),
//   give[b] = max(0, held - need),  row_start = exclusive sum of n,
// and the j-th page that b takes is the ring's entry at head + (exclusive sum of
// take)[b] + j.  Everything follows from exclusive sums over the requests, which
// each CTA takes for itself (a few thousand values from L2) rather than waiting
// for another: one launch, no barrier between CTAs.  The rows and the pages that
// change hands are then shared out over the grid, each by a binary search in the
// sums, while the first CTA makes the attention's split.  Taken ids come from the
// ring's free part and given ones go behind it, so no CTA reads what another
// writes; `held` and the ring's state, which may be updated in place, are written by
// the CTA that finishes last (an arrival ticket in the plan).  A further plan of the
// same step has `held` but no ring: it refuses what the first one refused.
//
// The attention's split.  Requests are put in order of their row blocks (blocks of
// 128 query rows per kv head), the most first, and their key tiles behind one
// another; row block s of all requests that have one is a prefix of that sequence
// of tiles.  Every CTA takes W tiles of one sequence, so that CTA k of each of
// them reads the same keys at the same time, once from HBM and then from L2, where
// row blocks behind one another read them again from HBM.  With one row block
// (decoding, small trees) the tiles are split evenly.
#include "paged.cuh"

namespace tv {

namespace {

constexpr int kThreads = 256;
// Tiles of an attention CTA at least: fewer CTAs on a small problem, but fewer
// partials to join.  Neither 1 nor 2 is better throughout.  In us with 1 and with 2:
// 64 nodes over 512 keys, 32 / 8 heads 13.7 and 16.2, 32 / 32 heads 14.7 and 13.8,
// 2 / 2 heads 11.2 and 12.7; over 4096 keys, 2 / 2 heads 18.1 and 16.4, 8 / 2 heads
// 20.3 and 19.8; one ragged capped tree 15.9 and 14.9; one token 12.6 with either.
constexpr int kMinTiles = 2;

struct PlanArgs {
    const TreeDesc *trees;
    int n_trees, batch, max_pages, page_log2, n_pages;
    const int32_t *tree, *n_new, *lens, *key_begin;
    int32_t *table, *row_start, *ring;
    const int32_t *state, *held;
    int32_t *state_out, *held_out;
    int64_t *slots;
    int32_t *positions, *status;
    int max_rows, Hq, Hkv, window, sink, P;
    void *plan;
};

// Exclusive sums over the block of K values a thread; the totals in `total`.
template <int K>
__device__ void block_scan(long long (&v)[K], long long (&total)[K])
{
    __shared__ long long part[kThreads / 32][K];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long in[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        long long x = v[k];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o)
                x += y;
        }
        in[k] = x - v[k];
        if (lane == 31)
            part[warp][k] = x;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        long long before = 0, all = 0;
        for (int w = 0; w < kThreads / 32; ++w) {
            if (w < warp)
                before += part[w][k];
            all += part[w][k];
        }
        v[k] = before + in[k];
        total[k] = all;
    }
    __syncthreads();
}

// The last b with sums[b] <= x, sums[0 .. n] non-decreasing, sums[0] <= x < sums[n].
template <typename T>
__device__ __forceinline__ int owner_of(const T *sums, int n, T x)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (sums[mid] <= x)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

// The key tiles of a request (see PlanReq).  Its rows see slots from lo on, and
// with a window the first `sink` from `begin`.
__device__ void tiles_of(PlanReq &q, int window, int sink)
{
    const long long end = (long long)q.L + q.n;
    const long long lo = window > 0 ? max((long long)q.begin, (long long)q.L - window + 1) : q.begin;
    const long long far_end = min((long long)q.begin + sink, 0x7fffffffll);
    q.far_end = (int)far_end;
    q.a0 = 0;
    q.n1 = 0;
    q.b0 = (int)(min(lo, end - 1) / kTileKeys);
    const long long near_far = min(far_end, lo);  // the kept first tokens that the window no longer covers
    if (window > 0 && near_far > q.begin) {
        const int a0 = q.begin / kTileKeys, a1 = (int)((near_far + kTileKeys - 1) / kTileKeys);
        if (a1 >= q.b0) {
            q.b0 = a0;
        } else {
            q.a0 = a0;
            q.n1 = a1 - a0;
        }
    }
    q.T = q.n1 + (int)((end - 1) / kTileKeys) - q.b0 + 1;
}

// The first tile of CTA c's range when `total` tiles are split evenly over P CTAs,
// and the CTA whose range holds tile t.
__device__ __forceinline__ long long div_up_to(long long a, long long b)
{
    return (a | b) >> 32 ? a / b : (long long)((uint32_t)a / (uint32_t)b);
}
__device__ __forceinline__ long long split_begin(long long total, int P, int c)
{
    const long long q = div_up_to(total, P), r = total - q * P;
    return q * c + (c < r ? c : r);
}
__device__ __forceinline__ int split_owner(long long total, int P, long long t)
{
    const long long q = div_up_to(total, P), r = total - q * P, wide = r * (q + 1);
    return (int)(t < wide ? div_up_to(t, q + 1) : r + div_up_to(t - wide, q));
}

// The requests' sums and sizes in shared memory.
struct Sums {
    long long *tile;  // in order of row blocks: tiles before
    int *row, *take, *give, *need, *held, *len, *n, *tree, *order;
};

// The attention's work split, by one CTA.
__device__ void make_split(const PlanArgs &p, const Sums &s)
{
    __shared__ int bins[kMaxRowBlocks + 2], warp_bins[kThreads / 32][kMaxRowBlocks + 2];
    __shared__ int s_start[kMaxRowBlocks + 1], s_W, s_seqs, s_P;
    __shared__ long long s_tiles[kMaxRowBlocks];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, B = p.batch, group = p.Hq / p.Hkv;
    PlanHeader *hd = static_cast<PlanHeader *>(p.plan);
    PlanReq *out = plan_reqs(p.plan);
    auto blocks_of = [&](int b) { return (s.n[b] * group + 127) / 128; };
    // stable counting sort by row blocks, the most first (bin kMaxRowBlocks - blocks; requests
    // without rows last)
    for (int x = tid; x < kMaxRowBlocks + 2; x += kThreads)
        bins[x] = 0;
    __syncthreads();
    for (int b = tid; b < B; b += kThreads)
        atomicAdd(&bins[kMaxRowBlocks - blocks_of(b)], 1);
    __syncthreads();
    if (warp == 0) {  // exclusive sums of the bins
        static_assert(kMaxRowBlocks == 32, "a lane per bin, and the last");
        const int n = bins[lane];
        int x = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, o);
            x += lane >= o ? y : 0;
        }
        bins[lane] = x - n;
        if (lane == 31)
            bins[32] = x;
    }
    __syncthreads();
    const int n_active = bins[kMaxRowBlocks];
    __shared__ int base[kMaxRowBlocks + 1];
    if (tid <= kMaxRowBlocks)
        base[tid] = bins[tid];
    for (int b0 = 0; b0 < B; b0 += kThreads) {
        for (int x = tid; x < (kThreads / 32) * (kMaxRowBlocks + 2); x += kThreads)
            (&warp_bins[0][0])[x] = 0;
        __syncthreads();
        const int b = b0 + tid, bin = b < B ? kMaxRowBlocks - blocks_of(b) : kMaxRowBlocks + 1;
        const unsigned same = __match_any_sync(0xffffffffu, bin);
        const int rank = __popc(same & ((1u << lane) - 1));
        if (rank == 0)
            warp_bins[warp][bin] = __popc(same);
        __syncthreads();
        if (tid < kMaxRowBlocks) {
            int at = base[tid];
            for (int w = 0; w < kThreads / 32; ++w) {
                const int n = warp_bins[w][tid];
                warp_bins[w][tid] = at;
                at += n;
            }
            base[tid] = at;
        }
        __syncthreads();
        if (bin < kMaxRowBlocks)
            s.order[warp_bins[warp][bin] + rank] = b;
        __syncthreads();
    }

    // the records in that order, and the tiles before each
    auto record = [&](int b) {
        PlanReq q;
        q.b = b;
        q.L = s.len[b];
        q.n = s.n[b];
        q.tree = s.tree[b];
        q.row0 = s.row[b];
        q.begin = p.key_begin ? min(max(p.key_begin[b], 0), q.L + q.n) : 0;
        tiles_of(q, p.window, p.sink);
        return q;
    };
    const int items = (n_active + kThreads - 1) / kThreads;
    long long v[1] = {0}, total[1];
    for (int i = 0; i < items; ++i)
        if (tid * items + i < n_active)
            v[0] += (long long)record(s.order[tid * items + i]).T * p.Hkv;
    block_scan<1>(v, total);
    for (int i = 0; i < items; ++i) {
        const int x = tid * items + i;
        if (x < n_active) {
            PlanReq q = record(s.order[x]);
            q.tile_base = v[0];
            s.tile[x] = v[0];
            out[x] = q;
            v[0] += (long long)q.T * p.Hkv;
        }
    }
    if (tid == 0) {
        s.tile[n_active] = total[0];
        PlanReq end = {};
        end.tile_base = total[0];
        out[n_active] = end;
    }
    __syncthreads();
    if (warp == 0) {
        // sequence `lane`: row block `lane` of the requests with more blocks than that
        const long long mine = s.tile[bins[kMaxRowBlocks - lane]];
        const int seqs = __popc(__ballot_sync(0xffffffffu, mine > 0));
        long long all = mine;
#pragma unroll
        for (int o = 16; o >= 1; o >>= 1)
            all += __shfl_xor_sync(0xffffffffu, all, o);
        // sum over the sequences of ceil(tiles / W) <= all / W + seqs <= P
        const int W = (int)max((long long)kMinTiles, all > 0 ? div_up_to(all - 1, max(p.P - seqs, 1)) + 1 : 1);
        const int P1 = (int)min((long long)p.P, max(div_up_to(all + kMinTiles - 1, kMinTiles), 1ll));
        const int ctas = seqs <= 1 ? (lane == 0 ? P1 : 0) : (int)div_up_to(mine + W - 1, W);
        int x = ctas;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, o);
            x += lane >= o ? y : 0;
        }
        s_tiles[lane] = mine;
        s_start[lane] = x - ctas;
        if (lane == 31) {
            s_start[32] = x;
            s_W = W;
            s_seqs = seqs;
            s_P = P1;
        }
    }
    __syncthreads();
    // the CTAs' ranges, and each unit that a range starts inside, once: at its second CTA
    PlanCta *ctas = plan_ctas(p.plan);
    int n_splits = 0;
    for (int c0 = 0; c0 < p.P; c0 += kThreads) {
        const int c = c0 + tid;
        PlanCta x = {};
        PlanSplit sp = {};
        if (c < p.P && n_active > 0 && c < s_start[32]) {
            int q = 0;
            while (c >= s_start[q + 1])
                ++q;
            const bool even = s_seqs <= 1;
            const long long tiles = s_tiles[q];
            auto begin_of = [&](int k) { return even ? split_begin(tiles, s_P, k) : min((long long)k * s_W, tiles); };
            auto owner = [&](long long t) { return even ? split_owner(tiles, s_P, t) : (int)div_up_to(t, s_W); };
            const int k = c - s_start[q];
            x.t0 = begin_of(k);
            x.t1 = begin_of(k + 1);
            x.rb = q;
            x.idx = owner_of(s.tile, n_active, x.t0);
            x.req = out[x.idx];
            const PlanReq &r = x.req;
            const int u = (int)div_up_to(x.t0 - r.tile_base, r.T);
            const long long first = r.tile_base + (long long)u * r.T;
            if (k > 0 && x.t0 > first && begin_of(k - 1) <= first) {
                sp.c_lo = c - 1;
                sp.nseg = owner(first + r.T - 1) - (k - 1) + 1;
                sp.lo_slot = begin_of(k - 1) == first ? 0 : 1;
                sp.row0 = r.row0;
                sp.rb = (int16_t)q;
                sp.head = u;
                sp.rows = (int16_t)min(128, r.n * group - q * 128);
                sp.tree = r.tree;
                sp.n = r.n;
            }
        }
        if (c < p.P)
            ctas[c] = x;
        long long at[1] = {sp.rows > 0}, n[1];
        block_scan<1>(at, n);
        if (sp.rows > 0)
            plan_splits(p.plan)[n_splits + at[0]] = sp;
        n_splits += (int)n[0];
    }
    if (tid == 0) {
        hd->valid = 1;
        hd->batch = B;
        hd->n_q_heads = p.Hq;
        hd->n_kv_heads = p.Hkv;
        hd->window = p.window;
        hd->n_splits = n_splits;
    }
}

// Bound by latency: every CTA's chain is a handful of dependent loads (length, tree,
// page id) and the sums; the first CTA's ends with the split.  8 requests 7.0 us,
// 1024 requests with 31000 rows 12.8 us.
__global__ void __launch_bounds__(kThreads) k_paged_plan(const __grid_constant__ PlanArgs p)
{
    extern __shared__ __align__(16) uint8_t smem[];
    const int B = p.batch, ld = B + 1, tid = threadIdx.x;
    Sums s;
    s.tile = reinterpret_cast<long long *>(smem);
    s.row = reinterpret_cast<int *>(s.tile + ld);
    s.take = s.row + ld;
    s.give = s.take + ld;
    s.need = s.give + ld;
    s.held = s.need + ld;
    s.len = s.held + ld;
    s.n = s.len + ld;
    s.tree = s.n + ld;
    s.order = s.tree + ld;
    __shared__ int s_last;
    pdl_wait();
    pdl_trigger();
    const bool pool = p.ring != nullptr, attend = p.Hq > 0, bad_write = blockIdx.x == gridDim.x - 1;
    int head = 0, count = 0;
    if (pool) {
        head = min(max(p.state[0], 0), p.n_pages - 1);
        count = min(max(p.state[1], 0), p.n_pages);
    }
    for (int b = tid; b < B; b += kThreads) {
        const int len = p.lens[b], tree = p.tree ? p.tree[b] : -1;
        int n = p.tree ? 0 : p.n_new[b], held = p.held ? p.held[b] : 0;
        if (tree >= 0 && tree < p.n_trees)
            n = p.trees[tree].n;
        const bool ok = len >= 0 && n >= 0 && tree >= -1 && tree < p.n_trees && held >= 0 && held <= p.max_pages;
        const long long want = ok ? ((long long)len + n + (1ll << p.page_log2) - 1) >> p.page_log2 : 0;
        const int bad = !ok ? TB_EINVAL : want > p.max_pages ? TB_ECAPACITY : TB_OK;
        // without `held` every page is there; with it but no ring, no page changes hands, so that a request
        // which needs more than it holds is refused as one that the ring has nothing left for
        held = p.held ? min(max(held, 0), p.max_pages) : bad ? 0 : (int)want;
        s.len[b] = len;
        s.tree[b] = tree;
        s.n[b] = bad ? 0 : n;
        s.held[b] = held;
        s.need[b] = bad ? held : pool ? (int)want : max((int)want, held);
        s.order[b] = bad;  // the status, until the split sorts
    }
    __syncthreads();

    // sums of rows, of pages taken and given; a request that does not fit gets nothing
    const int items = (B + kThreads - 1) / kThreads, b0 = min(tid * items, B), b1 = min(b0 + items, B);
    long long v[3], total[3];
    auto sum = [&] {
        v[0] = v[1] = v[2] = 0;
        for (int b = b0; b < b1; ++b) {
            v[0] += s.n[b];
            v[1] += max(0, s.need[b] - s.held[b]);
            v[2] += max(0, s.held[b] - s.need[b]);
        }
        block_scan<3>(v, total);
    };
    auto refuse = [&](int b) {
        s.order[b] = TB_ECAPACITY;
        s.n[b] = 0;
        s.need[b] = s.held[b];
    };
    sum();
    if (total[0] > p.max_rows) {  // the same for every thread
        long long at = v[0];
        for (int b = b0; b < b1; ++b) {
            at += s.n[b];
            if (s.n[b] > 0 && at > p.max_rows)
                refuse(b);
        }
        sum();
    }
    if (total[1] > count) {
        long long at = v[1];
        for (int b = b0; b < b1; ++b) {
            const int take = max(0, s.need[b] - s.held[b]);
            at += take;
            if (take > 0 && at > count)
                refuse(b);
        }
        sum();
    }
    const int rows = (int)total[0], n_take = (int)total[1], n_give = (int)total[2];
    for (int b = b0; b < b1; ++b) {
        s.row[b] = (int)v[0];
        s.take[b] = (int)v[1];
        s.give[b] = (int)v[2];
        v[0] += s.n[b];
        v[1] += max(0, s.need[b] - s.held[b]);
        v[2] += max(0, s.held[b] - s.need[b]);
        if (bad_write)
            p.status[b] = s.order[b];
    }
    if (tid == 0) {
        s.row[B] = rows;
        s.take[B] = n_take;
        s.give[B] = n_give;
    }
    __syncthreads();
    PlanHeader *hd = static_cast<PlanHeader *>(p.plan);
    if (bad_write) {
        for (int b = tid; b <= B; b += kThreads)
            p.row_start[b] = s.row[b];
        if (!attend && tid == 0)
            hd->valid = 0;
    }
    if (attend && blockIdx.x == 0) {
        make_split(p, s);
    } else {
        // the rows
        const int ctas = gridDim.x - (attend ? 1 : 0), stride = ctas * kThreads;
        const int from = (blockIdx.x - (attend ? 1 : 0)) * kThreads + tid;
        const int ring_n = p.n_pages;
        for (int r = from; r < p.max_rows; r += stride) {
            int64_t slot = -1;
            int pos = 0;
            if (r < rows) {
                const int b = owner_of(s.row, B, r), i = r - s.row[b];
                const int at = s.len[b] + i, pg = at >> p.page_log2;
                int id;
                if (pg < s.held[b]) {
                    id = p.table[(size_t)b * p.max_pages + pg];
                } else {
                    int x = head + s.take[b] + pg - s.held[b];
                    x -= x >= ring_n ? ring_n : 0;
                    id = p.ring[x];
                }
                if (id >= 0)
                    slot = ((int64_t)id << p.page_log2) + (at & ((1 << p.page_log2) - 1));
                pos = s.len[b] + (p.tree ? p.trees[s.tree[b]].depth[i] : i);
            }
            p.slots[r] = slot;
            p.positions[r] = pos;
        }
        // the pages that change hands
        for (int x = from; x < n_take; x += stride) {
            const int b = owner_of(s.take, B, x);
            int at = head + x;
            at -= at >= ring_n ? ring_n : 0;
            const int pg = s.held[b] + x - s.take[b];
            if (in_bounds(pg < p.max_pages && at < ring_n, nullptr))
                p.table[(size_t)b * p.max_pages + pg] = p.ring[at];
        }
        for (int x = from; x < n_give; x += stride) {
            const int b = owner_of(s.give, B, x);
            const int at = (int)(((long long)head + count + x) % ring_n);
            p.ring[at] = p.table[(size_t)b * p.max_pages + s.need[b] + x - s.give[b]];
        }
    }
    if (!pool)
        return;
    // every CTA has read `held` and the state by the time the last one arrives
    __syncthreads();
    if (tid == 0) {
        bool last = true;
        if (gridDim.x > 1) {
            __threadfence();
            last = atomicAdd(&hd->ticket, 1) == (int)gridDim.x - 1;
            if (last)
                hd->ticket = 0;
        }
        s_last = last;
    }
    __syncthreads();
    if (!s_last)
        return;
    for (int b = tid; b < B; b += kThreads)
        p.held_out[b] = s.need[b];
    if (tid == 0) {
        p.state_out[0] = (int)(((long long)head + n_take) % p.n_pages);
        p.state_out[1] = count - n_take + n_give;
    }
}

int log2_of(int x)
{
    int l = 0;
    while ((1 << l) < x)
        ++l;
    return l;
}

}  // namespace

TB_BOUNDS_COUNTER(bounds_violations_paged_plan)

}  // namespace tv

using namespace tv;

extern "C" size_t tb_paged_plan_size(int batch, int device)
{
    if (batch < 1 || batch > TB_MAX_REQUESTS || device_sms(device) <= 0)
        return 0;
    return plan_bytes_for(batch);
}

extern "C" tb_status paged_plan(const tb_bank *bank, const tb_requests *req, const tb_page_pool *pool, int64_t *slots,
                                int32_t *positions, int max_rows, int32_t *status, int n_q_heads, int n_kv_heads,
                                int window, int sink, void *plan, size_t plan_bytes, tb_stream stream)
{
    const char *fn = "paged_plan";
    tb_status st = check_requests(req, true, fn);
    if (st != TB_OK)
        return st;
    PlanArgs a{};
    if (req->tree) {
        if ((st = check_device_bank(bank, fn, &a.trees, &a.n_trees)) != TB_OK)
            return st;
    } else if (!req->n_new) {
        return record_error(TB_EINVAL, "%s: neither tree nor n_new", fn);
    }
    if (!status || max_rows < 0 || (max_rows > 0 && (!slots || !positions)))
        return record_error(TB_EINVAL, "%s: slots, positions or status is NULL, or max_rows %d < 0", fn, max_rows);
    if (n_q_heads < 0 || (n_q_heads > 0 && (n_kv_heads < 1 || n_q_heads % n_kv_heads)))
        return record_error(TB_EINVAL, "%s: n_q_heads %d not a multiple of n_kv_heads %d", fn, n_q_heads, n_kv_heads);
    if (n_q_heads > 0 && n_q_heads / n_kv_heads > kMaxGroup)
        return record_error(TB_EUNSUPPORTED, "%s: %d query heads per kv head (%d supported)", fn,
                            n_q_heads / n_kv_heads, kMaxGroup);
    if (n_q_heads > 0 && !req->tree)
        return record_error(TB_EINVAL, "%s: an attention plan is for trees", fn);
    if (window < 0 || sink < 0)
        return record_error(TB_EINVAL, "%s: window %d, sink %d", fn, window, sink);
    if ((st = check_workspace(plan, plan_bytes, plan_bytes_for(req->batch), fn)) != TB_OK)
        return st;
    if (pool) {
        const bool held_only = !pool->ring && !pool->state && !pool->state_out && !pool->held_out;
        if (!pool->held || (!held_only && (pool->n_pages < 1 || pool->n_pages > 1 << 30 || !pool->ring ||
                                           !pool->state || !pool->state_out || !pool->held_out)))
            return record_error(TB_EINVAL, "%s: pool of %d pages or with a NULL pointer", fn, pool->n_pages);
        a.n_pages = pool->n_pages;
        a.ring = pool->ring;
        a.state = pool->state;
        a.state_out = pool->state_out;
        a.held = pool->held;
        a.held_out = pool->held_out;
    }
    const int n_sm = device_sms(-1);
    if (n_sm <= 0)
        return record_error(TB_ECUDA, "%s: no current device", fn);
    a.batch = req->batch;
    a.max_pages = req->max_pages;
    a.page_log2 = log2_of(req->page_size);
    a.tree = req->tree;
    a.n_new = req->n_new;
    a.lens = req->lens;
    a.key_begin = req->key_begin;
    a.table = req->table;
    a.row_start = req->row_start;
    a.slots = slots;
    a.positions = positions;
    a.status = status;
    a.max_rows = max_rows;
    a.Hq = n_q_heads;
    a.Hkv = n_q_heads > 0 ? n_kv_heads : 1;
    a.window = window;
    a.sink = sink;
    a.P = n_sm < kMaxPlanCtas ? n_sm : kMaxPlanCtas;  // the grid of the attention
    a.plan = plan;
    // a CTA for every 512 rows (more of them repeat the sums for nothing), and one for the split
    const long long ctas = ((long long)max_rows + 2ll * req->batch + 511) / 512;
    const int grid = (int)(ctas < 1 ? 1 : ctas > n_sm ? n_sm : ctas) + (n_q_heads > 0 ? 1 : 0);
    const size_t smem = (size_t)(req->batch + 1) * (sizeof(long long) + 9 * sizeof(int));
    cudaError_t e = allow_max_smem((const void *)k_paged_plan);
    if (e == cudaSuccess)
        e = launch_kernel(k_paged_plan, dim3(grid), dim3(kThreads), smem, (cudaStream_t)stream, true, a);
    return launch_result(e, fn);
}
