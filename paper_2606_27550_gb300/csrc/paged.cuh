// paged.cuh -- what the kernels of a serving step over a paged cache share: the
// plan of a step (written by paged_plan, read by paged_tree_attention) and the
// argument checks of their entry points.
#pragma once

#include "kernels.cuh"

#include <cuda_fp16.h>

namespace tv {

constexpr int kTileKeys = 128;  // keys per tile of the paged attention

// One request of a plan.  Its tiles, kv head after kv head, are key tiles [a0, a0 +
// n1) (the first tokens that a window keeps) and [b0, b0 + T - n1).
struct PlanReq {
    long long tile_base;  // first of its tiles in the flattened tile space
    int L, n, row0, tree;
    int T, a0, n1, b0;
    int begin, far_end, b;  // keys before far_end are seen beyond the window
    int pad;                // whole words: a tail of four bytes is copied apart (plan of 1024 requests 13.1 us, 12.7 so)
};
static_assert(sizeof(PlanReq) == 56, "eight-byte aligned records");

struct PlanHeader {
    int ticket;  // of paged_plan's CTAs; zero between calls
    int valid;
    int batch, n_q_heads, n_kv_heads, window, n_splits;
    int pad[9];
};
static_assert(sizeof(PlanHeader) == 64, "");

// The tiles [t0, t1) of one attention CTA, for row block rb of the requests that
// they belong to; req is the one that t0 lies in, idx its place among the records.
struct PlanCta {
    long long t0, t1;
    int rb, idx;
    PlanReq req;
};
static_assert(sizeof(PlanCta) == 80, "eight-byte aligned records");

// A unit, (request, kv head, row block), that several CTAs share: what joining its
// partials needs.
struct PlanSplit {
    int c_lo, nseg;  // its CTAs
    int lo_slot;     // which of c_lo's two partial slots is the unit's (of the others: their first)
    int row0;        // the request's first row
    int16_t rows, rb;  // of the unit
    int head, tree, n;
};
static_assert(sizeof(PlanSplit) == 32, "");

constexpr int kMaxPlanCtas = 512;
constexpr int kMaxGroup = 64;                                   // query heads per kv head
constexpr int kMaxRowBlocks = kMaxNodes * kMaxGroup / 128;

// header, one PlanCta per attention CTA, as many PlanSplits, then the requests
// with rows and one more record whose tile_base is the sum of all tiles
inline size_t plan_bytes_for(int batch)
{
    return sizeof(PlanHeader) + kMaxPlanCtas * (sizeof(PlanCta) + sizeof(PlanSplit)) + (size_t)(batch + 1) * sizeof(PlanReq);
}
__host__ __device__ inline PlanCta *plan_ctas(void *plan)
{
    return reinterpret_cast<PlanCta *>(static_cast<unsigned char *>(plan) + sizeof(PlanHeader));
}
__host__ __device__ inline PlanSplit *plan_splits(void *plan)
{
    return reinterpret_cast<PlanSplit *>(plan_ctas(plan) + kMaxPlanCtas);
}
__host__ __device__ inline PlanReq *plan_reqs(void *plan)
{
    return reinterpret_cast<PlanReq *>(plan_splits(plan) + kMaxPlanCtas);
}

// argument checks (treeverify.cu); each returns TB_OK or records the error
tb_status check_device_bank(const tb_bank *bank, const char *fn, const TreeDesc **trees, int *n_trees);
tb_status check_requests(const tb_requests *req, bool table, const char *fn);
tb_status check_pages(const tb_pages *pages, const char *fn);
tb_status check_workspace(const void *ws, size_t bytes, size_t need, const char *fn);
tb_status launch_result(cudaError_t e, const char *fn);
// the attention's partials in a workspace of tb_workspace_size
float *attention_parts(void *ws);
int device_sms(int device);  // -1: the current one
bool ptr_aligned(const void *p, size_t a);

// What the stores share (paged_store.cu).
constexpr int kMaxAxes = 4;

struct Rows {
    uint16_t *p;
    long long row_stride, head_stride;
};
inline Rows rows_of(const tb_rows *r)
{
    return Rows{static_cast<uint16_t *>(r->ptr), r->row_stride, r->head_stride};
}

struct RopeAxes {
    const int32_t *pos;
    long long axis_stride;
    int axis_end[kMaxAxes];       // first pair past the axis
    uint64_t freq[kRopeMaxHalf];  // turns per position, times 2^64
};
tb_status check_rows(const tb_rows *r, const char *what, const char *fn);
tb_status check_store(int layer, int n_layers, const int64_t *slots, int n_rows, const tb_rows *k, const tb_rows *v,
                      const tb_rows *q, const tb_rows *q_out, int n_q_heads, const char *fn);
tb_status rope_axes(const tb_rope *rope, int d, int n_rows, RopeAxes *a, const char *fn);
tb_status check_pages_q4(const tb_pages_q4 *pages, const char *fn);

// K or V of one layer's pages: (d, slots of a page, kv heads, pages), box (64, box_slots, 1, 1)
bool make_tmap_pages(CUtensorMap *map, const tb_pages *pages, const void *base, int box_slots, const char **err);

unsigned int bounds_violations_paged_plan();
unsigned int bounds_violations_paged_store();
unsigned int bounds_violations_paged_rows();
unsigned int bounds_violations_paged_attention();
unsigned int bounds_violations_paged_attention_q4();
unsigned int bounds_violations_logits();
unsigned int bounds_violations_paged_accept();

// Loads that are issued where they stand: a short CTA's life is its round trips to
// memory, and a compiler that moves a load behind the branch that uses it adds one.
__device__ __forceinline__ int load_now(const int *p)
{
    int v;
    asm volatile("ld.global.b32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ float load_now(const float *p)
{
    float v;
    asm volatile("ld.global.b32 %0, [%1];" : "=f"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ uint64_t load_now(const uint64_t *p)
{
    uint64_t v;
    asm volatile("ld.global.b64 %0, [%1];" : "=l"(v) : "l"(p) : "memory");
    return v;
}

// The angle of pair i of a row, in 2^-64 of a turn (whole turns overflow).
__device__ __forceinline__ uint64_t turn_of(const RopeAxes &rope, int row, int i)
{
    int axis = 0;
#pragma unroll
    for (int a = 0; a < kMaxAxes - 1; ++a)
        axis += i >= rope.axis_end[a];
    const long long pos = rope.pos[axis * rope.axis_stride + row];
    return (uint64_t)pos * rope.freq[i];
}

// Two 16-bit elements of a word.
template <bool kF16>
__device__ __forceinline__ float2 unpack_pair(uint32_t w)
{
    if constexpr (kF16) {
        return __half22float2(*reinterpret_cast<const __half2 *>(&w));
    } else {
        return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    }
}
template <bool kF16>
__device__ __forceinline__ uint32_t pack_pair(float lo, float hi)
{
    if constexpr (kF16) {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&h);
    } else {
        return pack_bf16x2(lo, hi);
    }
}

// Two 32-bit floats in one instruction (softmax loops are bound by their issue slots).
__device__ __forceinline__ uint64_t two(float lo, float hi)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 halves(uint64_t v)
{
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ uint64_t fma_two(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t mul_two(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t add_two(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

}  // namespace tv
