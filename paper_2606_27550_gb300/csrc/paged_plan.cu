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
// for another: one launch, no barrier between CTAs.  The rows, the pages that
// change hands and the records are then shared out over the grid, each by a
// binary search in the sums.  Taken ids come from the ring's free part and given
// ones go behind it, so no CTA reads what another writes; `held` and the ring's
// state, which may be updated in place, are written by the CTA that finishes
// last (an arrival ticket in the plan).
#include "paged.cuh"

namespace tv {

namespace {

constexpr int kThreads = 512;
constexpr int kItems = TB_MAX_REQUESTS / kThreads;
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
static_assert(kMaxPlanCtas <= kThreads, "a split per thread");

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

// Bound by latency: 8 requests of 4 to 64 nodes and 1024 requests with 15 000
// rows differ little, since every chain is a handful of dependent loads (length,
// tree, page id) and the sums.
__global__ void __launch_bounds__(kThreads) k_paged_plan(const __grid_constant__ PlanArgs p)
{
    extern __shared__ __align__(16) uint8_t smem[];
    const int B = p.batch, ld = B + 1;
    long long *s_tile = reinterpret_cast<long long *>(smem);
    int *s_row = reinterpret_cast<int *>(s_tile + ld);
    int *s_take = s_row + ld, *s_give = s_take + ld, *s_need = s_give + ld, *s_held = s_need + ld;
    __shared__ int s_last;
    pdl_wait();
    pdl_trigger();
    const int items = (B + kThreads - 1) / kThreads, b0 = threadIdx.x * items;
    const bool pool = p.ring != nullptr;
    int head = 0, count = 0;
    if (pool) {
        head = min(max(p.state[0], 0), p.n_pages - 1);
        count = min(max(p.state[1], 0), p.n_pages);
    }

    // the requests of this thread
    int len[kItems], n[kItems], held[kItems], need[kItems], tree[kItems], bad[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const int b = b0 + i;
        const bool mine = i < items && b < B;
        len[i] = mine ? p.lens[b] : 0;
        tree[i] = mine && p.tree ? p.tree[b] : -1;
        n[i] = mine && !p.tree ? p.n_new[b] : 0;
        held[i] = mine && pool ? p.held[b] : 0;
    }
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        if (tree[i] >= 0 && tree[i] < p.n_trees)
            n[i] = p.trees[tree[i]].n;
        const bool ok = len[i] >= 0 && n[i] >= 0 && tree[i] >= -1 && tree[i] < p.n_trees && held[i] >= 0 &&
                        held[i] <= p.max_pages;
        const long long want = ok ? ((long long)len[i] + n[i] + (1ll << p.page_log2) - 1) >> p.page_log2 : 0;
        bad[i] = !ok ? TB_EINVAL : want > p.max_pages ? TB_ECAPACITY : TB_OK;
        need[i] = (int)want;
        if (!pool)
            held[i] = need[i];
        if (bad[i] != TB_OK) {
            n[i] = 0;
            held[i] = min(max(held[i], 0), p.max_pages);
            need[i] = held[i];
        }
    }

    // sums of rows and of pages taken; a request that does not fit gets nothing
    long long sum[2], total2[2];
    auto totals = [&] {
        sum[0] = sum[1] = 0;
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            sum[0] += n[i];
            sum[1] += max(0, need[i] - held[i]);
        }
    };
    totals();
    block_scan<2>(sum, total2);
    if (total2[0] > p.max_rows) {  // the same for every thread
        long long at = sum[0];
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            at += n[i];
            if (n[i] > 0 && at > p.max_rows)
                bad[i] = TB_ECAPACITY, n[i] = 0, need[i] = held[i];
        }
        totals();
        block_scan<2>(sum, total2);
    }
    if (total2[1] > count) {
        long long at = sum[1];
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int take = max(0, need[i] - held[i]);
            at += take;
            if (take > 0 && at > count)
                bad[i] = TB_ECAPACITY, n[i] = 0, need[i] = held[i];
        }
        totals();
        block_scan<2>(sum, total2);
    }

    // offsets of rows, pages, records and tiles
    const int group = p.Hq > 0 ? p.Hq / p.Hkv : 0;
    auto record = [&](int i) {
        PlanReq q;
        q.b = b0 + i;
        q.L = len[i];
        q.n = n[i];
        q.tree = tree[i];
        q.row_blocks = (n[i] * group + 127) / 128;
        q.begin = p.key_begin ? min(max(p.key_begin[q.b], 0), len[i] + n[i]) : 0;
        tiles_of(q, p.window, p.sink);
        return q;
    };
    long long v[3] = {0, 0, 0}, total3[3];
    const bool attend = group > 0 && p.tree;
#pragma unroll 1
    for (int i = 0; i < items; ++i) {
        v[0] += max(0, held[i] - need[i]);
        if (n[i] > 0 && attend) {
            const PlanReq q = record(i);
            v[1] += 1;
            v[2] += (long long)q.T * p.Hkv * q.row_blocks;
        }
    }
    block_scan<3>(v, total3);
    const int rows = (int)total2[0], n_take = (int)total2[1], n_give = (int)total3[0], n_active = (int)total3[1];
    PlanHeader *hd = static_cast<PlanHeader *>(p.plan);
    PlanReq *out = plan_reqs(p.plan);
    const bool first = blockIdx.x == 0;
    // a CTA has kMinTiles tiles at least: fewer CTAs on a small problem, but whole
    // units and no partials to merge
    const int P = (int)min((long long)p.P, max((total3[2] + kMinTiles - 1) / kMinTiles, 1ll));
#pragma unroll 1
    for (int i = 0; i < items; ++i) {
        const int b = b0 + i;
        if (b >= B)
            break;
        s_row[b] = (int)sum[0];
        s_take[b] = (int)sum[1];
        s_give[b] = (int)v[0];
        s_need[b] = need[i];
        s_held[b] = held[i];
        if (first) {
            p.row_start[b] = (int)sum[0];
            p.status[b] = bad[i];
            if (n[i] > 0 && attend) {
                PlanReq q = record(i);
                q.tile_base = v[2];
                q.row0 = (int)sum[0];
                out[v[1]] = q;
                s_tile[v[1]] = v[2];
                v[1] += 1;
                v[2] += (long long)q.T * p.Hkv * q.row_blocks;
            }
        }
        sum[0] += n[i];
        sum[1] += max(0, need[i] - held[i]);
        v[0] += max(0, held[i] - need[i]);
    }
    if (threadIdx.x == 0) {
        s_row[B] = rows;
        s_take[B] = n_take;
        s_give[B] = n_give;
        if (first) {
            s_tile[n_active] = total3[2];
            p.row_start[B] = rows;
            PlanReq end = {};
            end.tile_base = total3[2];
            out[n_active] = end;
            hd->valid = attend ? 1 : 0;
            hd->batch = B;
            hd->n_q_heads = p.Hq;
            hd->n_kv_heads = p.Hkv;
            hd->window = p.window;
            hd->sink = p.sink;
            hd->n_active = n_active;
            hd->P = P;
            hd->total = total3[2];
            hd->rows = rows;
        }
    }
    __syncthreads();
    if (first) {
        PlanCta *ctas = plan_ctas(p.plan);
        for (int c = threadIdx.x; c < p.P; c += kThreads) {
            PlanCta x = {};
            x.total = total3[2];
            x.P = P;
            if (c < P && n_active > 0) {
                x.t0 = plan_split(total3[2], P, c);
                x.t1 = plan_split(total3[2], P, c + 1);
                x.idx = owner_of(s_tile, n_active, x.t0);
                x.req = out[x.idx];
            }
            ctas[c] = x;
        }
        // the units that a CTA's range starts inside, each once: at its second CTA
        PlanSplit sp = {};
        const int c = threadIdx.x;  // P <= kThreads
        if (c > 0 && c < P && n_active > 0) {
            const long long t = plan_split(total3[2], P, c);
            const PlanReq r = out[owner_of(s_tile, n_active, t)];
            const long long tl = t - r.tile_base;
            const int u = (int)(tl / r.T);
            const long long begin = r.tile_base + (long long)u * r.T;
            if (t > begin && plan_split(total3[2], P, c - 1) <= begin) {
                sp.c_lo = c - 1;
                sp.nseg = plan_cta_of(total3[2], P, begin + r.T - 1) - sp.c_lo + 1;
                sp.lo_slot = plan_split(total3[2], P, c - 1) == begin ? 0 : 1;
                sp.row0 = r.row0;
                sp.rb = u % r.row_blocks;
                sp.head = u / r.row_blocks;
                sp.rows = min(128, r.n * group - sp.rb * 128);
            }
        }
        long long v1[1] = {sp.rows > 0}, n_splits[1];
        block_scan<1>(v1, n_splits);
        if (sp.rows > 0)
            plan_splits(p.plan)[v1[0]] = sp;
        if (threadIdx.x == 0)
            hd->n_splits = (int)n_splits[0];
    }

    // the rows
    const int stride = gridDim.x * kThreads, tid = blockIdx.x * kThreads + threadIdx.x;
    const int ring_n = p.n_pages;
    for (int r = tid; r < p.max_rows; r += stride) {
        int64_t slot = -1;
        int pos = 0;
        if (r < rows) {
            const int b = owner_of(s_row, B, r), i = r - s_row[b];
            const int L = p.lens[b], s = L + i, pg = s >> p.page_log2;
            int id;
            if (pg < s_held[b]) {
                id = p.table[(size_t)b * p.max_pages + pg];
            } else {
                int at = head + s_take[b] + pg - s_held[b];
                at -= at >= ring_n ? ring_n : 0;
                id = p.ring[at];
            }
            if (id >= 0)
                slot = ((int64_t)id << p.page_log2) + (s & ((1 << p.page_log2) - 1));
            pos = L + (p.tree ? p.trees[p.tree[b]].depth[i] : i);
        }
        p.slots[r] = slot;
        p.positions[r] = pos;
    }
    // the pages that change hands
    for (int x = tid; x < n_take; x += stride) {
        const int b = owner_of(s_take, B, x);
        int at = head + x;
        at -= at >= ring_n ? ring_n : 0;
        const int pg = s_held[b] + x - s_take[b];
        if (in_bounds(pg < p.max_pages && at < ring_n, nullptr))
            p.table[(size_t)b * p.max_pages + pg] = p.ring[at];
    }
    for (int x = tid; x < n_give; x += stride) {
        const int b = owner_of(s_give, B, x);
        const int at = (int)(((long long)head + count + x) % ring_n);
        p.ring[at] = p.table[(size_t)b * p.max_pages + s_need[b] + x - s_give[b]];
    }
    if (!pool)
        return;
    // every CTA has read `held` and the state by the time the last one arrives
    __syncthreads();
    if (threadIdx.x == 0) {
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
    for (int b = threadIdx.x; b < B; b += kThreads)
        p.held_out[b] = s_need[b];
    if (threadIdx.x == 0) {
        p.state_out[0] = (int)(((long long)head + n_take) % ring_n);
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
    if (!slots || !positions || !status || max_rows < 1)
        return record_error(TB_EINVAL, "%s: slots, positions or status is NULL, or max_rows %d < 1", fn, max_rows);
    if (n_q_heads < 0 || (n_q_heads > 0 && (n_kv_heads < 1 || n_q_heads % n_kv_heads || n_q_heads > 65536)))
        return record_error(TB_EINVAL, "%s: n_q_heads %d not a multiple of n_kv_heads %d", fn, n_q_heads, n_kv_heads);
    if (n_q_heads > 0 && !req->tree)
        return record_error(TB_EINVAL, "%s: an attention plan is for trees", fn);
    if (window < 0 || sink < 0)
        return record_error(TB_EINVAL, "%s: window %d, sink %d", fn, window, sink);
    if ((st = check_workspace(plan, plan_bytes, plan_bytes_for(req->batch), fn)) != TB_OK)
        return st;
    if (pool) {
        if (pool->n_pages < 1 || pool->n_pages > 1 << 30 || !pool->ring || !pool->state || !pool->state_out ||
            !pool->held || !pool->held_out)
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
    // a CTA for every 512 rows: more of them repeat the sums for nothing
    const long long ctas = ((long long)max_rows + 2ll * req->batch + kThreads - 1) / kThreads;
    const int grid = (int)(ctas < 1 ? 1 : ctas > n_sm ? n_sm : ctas);
    const size_t smem = (size_t)(req->batch + 1) * (sizeof(long long) + 5 * sizeof(int));
    cudaError_t e = allow_max_smem((const void *)k_paged_plan);
    if (e == cudaSuccess)
        e = launch_kernel(k_paged_plan, dim3(grid), dim3(kThreads), smem, (cudaStream_t)stream, true, a);
    return launch_result(e, fn);
}
