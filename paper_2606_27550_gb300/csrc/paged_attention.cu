// paged_attention.cu -- tree attention over the pages of one layer: ancestor
// masks, an optional window with the first tokens kept, capped scores, a bias by
// distance.
//
// One CTA per (row, query head): its warps share the visible slots, each lane
// holds d / 32 elements of the query and of the output, and every warp keeps a
// running maximum m and sum l of its slots (z in units of ln 2),
//   m' = max(m, z),  l' = l 2^(m - m') + 2^(z - m'),  o' = o 2^(m - m') + 2^(z - m') v,
// which the first warp joins at the end.
#include "paged.cuh"

#include <cuda_fp16.h>

#include <cmath>

namespace tv {

namespace {

constexpr int kThreads = 128, kWarps = kThreads / 32;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct PagedArgs {
    const TreeDesc *trees;
    const int32_t *table;
    int max_pages, page_log2, n_pages, batch;
    const uint16_t *k, *v;  // of the layer
    long long page_stride, head_stride, slot_stride;
    const uint16_t *q;
    uint16_t *out;
    float *lse;
    const float *slopes;
    int n_rows, Hq, Hkv, d;
    float scale, softcap;
    void *plan;
    int *status;
};

template <bool kF16>
__device__ __forceinline__ float2 unpack(uint32_t w)
{
    if constexpr (kF16)
        return __half22float2(*reinterpret_cast<const __half2 *>(&w));
    else
        return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}

template <bool kF16>
__device__ __forceinline__ uint32_t pack(float lo, float hi)
{
    if constexpr (kF16) {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&h);
    } else {
        return pack_bf16x2(lo, hi);
    }
}

// kD / 32 elements of a lane
template <bool kF16, int kD>
struct Lane {
    float v[kD / 32];
    __device__ __forceinline__ void load(const uint16_t *row, int lane)
    {
#pragma unroll
        for (int i = 0; i < kD / 64; ++i) {
            const float2 x = unpack<kF16>(reinterpret_cast<const uint32_t *>(row)[lane * (kD / 64) + i]);
            v[2 * i] = x.x, v[2 * i + 1] = x.y;
        }
    }
};

template <bool kF16, int kD>
__global__ void __launch_bounds__(kThreads) k_paged_attention(const __grid_constant__ PagedArgs p)
{
    __shared__ float s_o[kWarps][kD], s_m[kWarps], s_l[kWarps];
    pdl_wait();
    pdl_trigger();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const PlanHeader *hd = static_cast<const PlanHeader *>(p.plan);
    if (!hd->valid || hd->batch != p.batch || hd->n_q_heads != p.Hq || hd->n_kv_heads != p.Hkv) {
        if (threadIdx.x == 0)
            atomicOr(p.status, kStatusBounds);
        return;
    }
    const int row = blockIdx.x, h = blockIdx.y;
    if (row >= hd->rows)
        return;
    const PlanReq *reqs = plan_reqs(p.plan);
    int lo = 0, hi = hd->n_active;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (reqs[mid].row0 <= row)
            lo = mid;
        else
            hi = mid;
    }
    const PlanReq rq = reqs[lo];
    const int i = row - rq.row0, L = rq.L, g = h / (p.Hq / p.Hkv);
    const TreeDesc &td = p.trees[rq.tree];
    const uint64_t anc = td.anc[i];
    const int pos = L + td.depth[i];
    const float slope = p.slopes ? p.slopes[h] : 0.f;
    Lane<kF16, kD> q;
    q.load(p.q + ((size_t)row * p.Hq + h) * kD, lane);
    float o[kD / 32] = {}, m = -INFINITY, l = 0.f;
    for (int s = rq.begin + warp; s < L + rq.n; s += kWarps) {
        const int j = s - L;
        if (j >= 0 && !((anc >> j) & 1))
            continue;
        const int at = j < 0 ? s : L + td.depth[j];
        if (hd->window > 0 && pos - at >= hd->window && s >= rq.far_end)
            continue;
        const int id = p.table[(size_t)rq.b * p.max_pages + (s >> p.page_log2)];
        if (id < 0 || id >= p.n_pages)
            continue;
        const long long off = id * p.page_stride + g * p.head_stride + (s & ((1 << p.page_log2) - 1)) * p.slot_stride;
        Lane<kF16, kD> k, v;
        k.load(p.k + off, lane);
        v.load(p.v + off, lane);
        float z = 0.f;
#pragma unroll
        for (int x = 0; x < kD / 32; ++x)
            z += q.v[x] * k.v[x];
#pragma unroll
        for (int x = 16; x >= 1; x >>= 1)
            z += __shfl_xor_sync(0xffffffffu, z, x);
        z *= p.scale;
        if (p.softcap > 0.f)
            z = p.softcap * tanhf(z / p.softcap);
        z = (z - slope * (float)(pos - at)) * kLog2e;
        const float m2 = fmaxf(m, z), w = exp2f(m - m2), e = exp2f(z - m2);
        m = m2;
        l = l * w + e;
#pragma unroll
        for (int x = 0; x < kD / 32; ++x)
            o[x] = o[x] * w + e * v.v[x];
    }
#pragma unroll
    for (int x = 0; x < kD / 32; ++x)
        s_o[warp][lane * (kD / 32) + x] = o[x];
    if (lane == 0)
        s_m[warp] = m, s_l[warp] = l;
    __syncthreads();
    if (warp)
        return;
    float M = -INFINITY, sum = 0.f;
    for (int w = 0; w < kWarps; ++w)
        M = fmaxf(M, s_m[w]);
    float acc[kD / 32] = {};
    for (int w = 0; w < kWarps; ++w) {
        const float f = s_m[w] == -INFINITY ? 0.f : exp2f(s_m[w] - M);
        sum += f * s_l[w];
#pragma unroll
        for (int x = 0; x < kD / 32; ++x)
            acc[x] += f * s_o[w][lane * (kD / 32) + x];
    }
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    uint32_t *dst = reinterpret_cast<uint32_t *>(p.out + ((size_t)row * p.Hq + h) * kD) + lane * (kD / 64);
#pragma unroll
    for (int x = 0; x < kD / 64; ++x)
        dst[x] = pack<kF16>(acc[2 * x] * inv, acc[2 * x + 1] * inv);
    if (p.lse && lane == 0)
        p.lse[(size_t)row * p.Hq + h] = sum > 0.f ? M * kLn2 + logf(sum) : -INFINITY;
}

}  // namespace

TB_BOUNDS_COUNTER(bounds_violations_paged_attention)

}  // namespace tv

using namespace tv;

extern "C" tb_status paged_tree_attention(const tb_bank *bank, const tb_requests *req, const tb_pages *pages,
                                          int layer, const void *plan, size_t plan_bytes, const void *q, int n_rows,
                                          int n_q_heads, float scale, float softcap, const float *slopes, void *out,
                                          float *lse, void *workspace, size_t workspace_bytes, tb_stream stream)
{
    const char *fn = "paged_tree_attention";
    PagedArgs a{};
    int n_trees = 0;
    tb_status st = check_device_bank(bank, fn, &a.trees, &n_trees);
    if (st != TB_OK || (st = check_requests(req, true, fn)) != TB_OK || (st = check_pages(pages, fn)) != TB_OK)
        return st;
    if (!req->tree)
        return record_error(TB_EINVAL, "%s: req->tree is NULL", fn);
    if (pages->page_size != req->page_size)
        return record_error(TB_EINVAL, "%s: pages of %d slots, a table of %d", fn, pages->page_size, req->page_size);
    if (layer < 0 || layer >= pages->n_layers)
        return record_error(TB_EINVAL, "%s: layer %d of %d", fn, layer, pages->n_layers);
    if (n_q_heads < pages->n_kv_heads || n_q_heads % pages->n_kv_heads || n_q_heads > 65535)
        return record_error(TB_EINVAL, "%s: n_q_heads %d not a multiple of n_kv_heads %d", fn, n_q_heads,
                            pages->n_kv_heads);
    if (!(scale > 0.f) || !std::isfinite(scale) || !(softcap >= 0.f) || !std::isfinite(softcap))
        return record_error(TB_EINVAL, "%s: scale %g, softcap %g", fn, scale, softcap);
    if (n_rows < 0)
        return record_error(TB_EINVAL, "%s: n_rows %d", fn, n_rows);
    if (!q || !out || !ptr_aligned(q, 16) || !ptr_aligned(out, 16))
        return record_error(TB_EINVAL, "%s: q / out NULL or not 16-byte aligned", fn);
    if ((st = check_workspace(plan, plan_bytes, plan_bytes_for(req->batch), fn)) != TB_OK)
        return st;
    if ((st = check_workspace(workspace, workspace_bytes,
                              tb_workspace_size(0, 1, pages->n_kv_heads, n_q_heads, pages->head_dim, 0, -1), fn)) !=
        TB_OK)
        return st;
    if (n_rows == 0)
        return launch_result(cudaSuccess, fn);
    a.table = req->table;
    a.max_pages = req->max_pages;
    while ((1 << a.page_log2) < req->page_size)
        ++a.page_log2;
    a.n_pages = pages->n_pages;
    a.batch = req->batch;
    a.k = static_cast<const uint16_t *>(pages->k) + (long long)layer * pages->layer_stride;
    a.v = static_cast<const uint16_t *>(pages->v) + (long long)layer * pages->layer_stride;
    a.page_stride = pages->page_stride;
    a.head_stride = pages->head_stride;
    a.slot_stride = pages->slot_stride;
    a.q = static_cast<const uint16_t *>(q);
    a.out = static_cast<uint16_t *>(out);
    a.lse = lse;
    a.slopes = slopes;
    a.n_rows = n_rows;
    a.Hq = n_q_heads;
    a.Hkv = pages->n_kv_heads;
    a.d = pages->head_dim;
    a.scale = scale;
    a.softcap = softcap;
    a.plan = const_cast<void *>(plan);
    a.status = static_cast<int *>(workspace);
    const bool f16 = pages->dtype == TB_F16;
    const auto kernel = pages->head_dim == 64 ? (f16 ? k_paged_attention<true, 64> : k_paged_attention<false, 64>)
                                              : (f16 ? k_paged_attention<true, 128> : k_paged_attention<false, 128>);
    return launch_result(launch_kernel(kernel, dim3(n_rows, n_q_heads), dim3(kThreads), 0, (cudaStream_t)stream, true,
                                       a),
                         fn);
}
