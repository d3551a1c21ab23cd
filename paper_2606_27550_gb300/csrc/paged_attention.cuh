// paged_attention.cuh -- tree attention over the pages of one layer: ancestor
// masks, an optional window with the first tokens kept, capped scores, a bias by
// distance.  On the 5th-generation tensor cores, as the attention over a
// contiguous cache (attention_tc.cu) is, with the work split read from the plan
// of the step.
//
// A unit is one (request, kv head, block of 128 query rows); its 128-key tiles lie
// behind one another in a flattened tile space that paged_plan has split evenly
// over the CTAs.  Per tile
//   S   = Q K^T   M = 128 rows, N = 128 keys; Q is the TMEM operand, the K tile a
//                 K-major shared-memory operand
//   O  += P V     N = head_dim; P = 2^(z - m) is the TMEM operand, the V tile an
//                 MN-major one
// with the scores z in units of ln 2 and a reference maximum m that is raised (and
// O and the sum rescaled) only when the row's maximum has grown past it by 2^8
// (2^7 in fp16).  A unit split between CTAs leaves one (O, m, l) per CTA, which
// k_paged_merge joins by log-sum-exp in CTA order: the same sums every time.
//
// A tile's 128 slots are 128 / page_size pages (or a part of one): the lanes of a
// producer warp look their pages up one tile ahead and issue one TMA box each.
// Pages past the request's end, and ids outside the pool, are addressed past the
// last page, where TMA fills zeros; such an id where some row looks is reported.
// Slots of a landed tile that no row may see (a page's rest behind the last token, before a document's beginning, between the
// kept first tokens and the window) can hold anything: their scores are replaced
// (not multiplied) by -inf, and the softmax threads overwrite their V rows with
// zeros before P V reads them, since 0 * NaN is NaN.
//
// One CTA per SM, 16 warps: 0 and 3 load K and V tiles through separate rings, 1
// issues Q K^T (S double-buffered) and holds the TMEM, 2 issues P V, 4-7 and 12-15
// are the softmax (two threads per row, half of a tile's columns each), 8-11 stage
// the next unit's queries and write the finished unit's output.
// TMEM columns: S0 [0, 128), S1 [128, 256), of each the halves' P on their first 32
// columns, O [256, 256 + kD), Q0 [384, 384 + kD / 2), Q1 behind it.  Row
// r sits in lane 32 (r % 4) + r / 4, so that few rows spread over the four SM
// sub-partitions.
//
// Bound by HBM where rows are few (64 requests of one token, 8 kv heads of 128, prefixes
// of 512 to 8192: 182 us, 6.37 TB/s, 94 % of a copy's bandwidth, 206 us with a cap and 201
// with a bias, whose special functions run for 128 rows where 4 are there; 32 kv heads at
// 65536 keys 166 us, 95 %), by the softmax's chain per tile with 128 rows per kv head (two row
// blocks of 64 nodes at 65536 keys: 76 us, 0.91 PFLOP/s; 2060 cycles a tile, 700 of them
// for the weights, 260 for the exchange between the halves, 340 waiting for S, whose
// 16 MMAs with P V take over 100 cycles each), and by
// the way to the first tile, unit boundaries and the join in short calls (9.1 us for a
// tree of 7 nodes at 128 keys, 52 us for 32 heads at 16384 keys).  Eight ragged trees with
// capped scores take 44.5 us; they took 51.7 with one softmax thread per row, 47.9 with two,
// and 43.6 with packed pairs and one reciprocal for four caps, before holes in the table
// were reported.
//
// 4-bit pages (kQ4), units of few rows: paged_attention_few.cuh.  The others: warps 0
// and 1 copy pages as they lie into rings of packed tiles of K and V, and warps 8-11 (K)
// and 0-2 (V) turn them into the tiles above, each element exactly: 32 codes and their
// scale per thread, four 16-byte pieces into the swizzled rows.  Within 8 elements those
// stand in the order 0 4 1 5 2 6 3 7, in which four codes come out of one shift; the
// queries are staged in that order too, and the output's columns put back.  Warp 3 issues
// both products, whichever is ready.  Bound by the way of a tile through its stages, 2600
// to 3000 cycles (the 16-bit pages' 2060): the seven warps that unpack it, 16 products that
// take 1800 to issue and run, and the instruction caches, which five roles' code contends
// for (a chain of 4 nodes at 131000 keys, 4 query heads on each of 8 kv heads: 92 us, 19 %
// of a copy's bandwidth; eight ragged trees with capped scores and a window 55 us).  The
// trees took 81 us with four warps that unpacked both operands in unrolled code, 73 with
// seven in short loops, 67 with one warp that issues whichever product is ready, 63 with
// its addresses in uniform registers, 55 with units of 9 to 16 rows here and not among the
// few.
#pragma once

#include "paged_q4.cuh"

#include <cmath>
#include <type_traits>

namespace tv {

namespace {

constexpr int kBN = kTileKeys;
constexpr int kAtom = 128 * 128;  // bytes of a 64-column swizzle atom of 128 rows
constexpr int kThreads = 512;
constexpr int kHalf = kBN / 2;  // columns of a softmax thread
constexpr int kMaxStages = 3;
constexpr int kPackedStages = 4;  // of the packed tiles of 4-bit pages
constexpr uint32_t kColS = 0, kColO = 256, kColQ = 384;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// score forms
constexpr int kPlain = 0, kCap = 1, kBias = 2;  // kBias: a bias by distance, capped or not

constexpr int tile_bytes(int d)
{
    return d / 64 * kAtom;
}
constexpr int k_stages(bool q4)
{
    return q4 ? 2 : 3;
}
constexpr int kVStages = 2;
constexpr int packed_bytes(int d)
{
    return kBN * row_bytes(d);
}
// A capped score carries an error of up to cap 2^-20 from the 32-bit tanh: 2^-10 at this cap, where
// rounding a weight costs 2^-8 (bf16) or 2^-11 (fp16).
constexpr float kMaxCap = 1024.f;

float cap_in(float scale, float softcap)
{
    return (float)(2.0 * 1.4426950408889634 * (double)scale / (double)softcap);
}

struct PagedArgs {
    CUtensorMap tk, tv;  // of the layer
    const uint8_t *k_pages, *v_pages;  // 4-bit pages: the layer's, strides in bytes
    long long head_stride;
    uint32_t page_units;  // 16 bytes each
    const TreeDesc *trees;
    int n_trees;
    const int32_t *table;
    int max_pages, page_log2, n_pages, batch;
    const uint16_t *q;
    uint16_t *out;
    float *lse;
    const float *slopes;
    int n_rows, Hq, Hkv, group;
    float scale;      // of the raw scores, times log2(e)
    float cap, cap_in;  // cap log2(e); 2 scale / cap, times log2(e)
    void *plan;
    float *part;
    int *status;
    int expire_wait;  // test hook: P V waits on a barrier that nothing arrives on
};

template <bool kF16>
__device__ __forceinline__ uint32_t pack(float lo, float hi)
{
    if constexpr (kF16) {
        uint32_t r;
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    } else {
        return pack_bf16x2(lo, hi);
    }
}

// Instruction descriptor of a kind::f16 MMA with M = 128 and f32 accumulation.
template <bool kF16>
__device__ constexpr uint32_t idesc(int N, bool b_mn)
{
    const uint32_t bf = idesc_bf16_f32(128, N, false, b_mn);
    return kF16 ? bf & ~((1u << 7) | (1u << 10)) : bf;  // both operand types: 0 is f16, 1 bf16
}

__device__ __forceinline__ float rcp_approx(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ float min_or_nan(float a, float b)
{
    float y;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}

// A capped score is cap tanh y = cap - 2 cap w with w = 1 / (1 + e^(2y)), y = scale s / cap.
// w of four scores in their place: from e^(2y) = 2^30 on, 2 w is below half a unit in the
// last place of 1, so that the exponent stops there and one reciprocal, of the product of
// all four denominators (at most 2^120), serves them: 1/a = b (cd / abcd).  The special
// functions bound a capped tile: two row blocks over 65536 keys (8 kv heads) take 98 us
// with this, 107 us with a reciprocal each, 113 us with an odd polynomial for small
// arguments, and 75 us without a cap.
__device__ __forceinline__ void cap_four(uint32_t *r, float cap_in)
{
    float e[4];
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
        const float2 y = halves(mul_two(two(__uint_as_float(r[i]), __uint_as_float(r[i + 1])), two(cap_in, cap_in)));
        e[i] = ex2_approx(min_or_nan(y.x, 30.f)), e[i + 1] = ex2_approx(min_or_nan(y.y, 30.f));
    }
    const uint64_t ac = add_two(two(e[0], e[2]), two(1.f, 1.f)), bd = add_two(two(e[1], e[3]), two(1.f, 1.f));
    const float2 ab_cd = halves(mul_two(ac, bd));
    const float y = rcp_approx(ab_cd.x * ab_cd.y);
    const uint64_t inv = mul_two(two(ab_cd.y, ab_cd.x), two(y, y));  // 1 / ab, 1 / cd
    const float2 w02 = halves(mul_two(bd, inv)), w13 = halves(mul_two(ac, inv));
    r[0] = __float_as_uint(w02.x), r[2] = __float_as_uint(w02.y);
    r[1] = __float_as_uint(w13.x), r[3] = __float_as_uint(w13.y);
}

// The verdict of a wait by a whole warp.  Its lanes may see a barrier complete and the time run out
// in one instant, and leave the kernel's loops together or not at all.
__device__ __forceinline__ bool warp_agrees(bool ok)
{
    return __all_sync(0xffffffffu, ok);
}

// The bits of [lo, hi) relative to s0, of 32.
__device__ __forceinline__ uint32_t range_bits(int s0, int lo, int hi)
{
    const int a = max(lo - s0, 0), b = min(hi - s0, 32);
    if (a >= b)
        return 0u;
    return (0xffffffffu >> (32 - (b - a))) << a;
}

// The bits of a node set of the 32 slots from s0 on (the tree begins at slot L).
__device__ __forceinline__ uint32_t tree_bits(int s0, int L, uint64_t nodes)
{
    if (s0 >= L)
        return s0 - L < 64 ? (uint32_t)(nodes >> (s0 - L)) : 0u;
    return s0 + 32 > L ? (uint32_t)(nodes << (L - s0)) : 0u;
}

// A CTA's position: the request that its next tile lies in, the one after it
// fetched ahead.
struct Cursor {
    PlanReq r, next;
    const PlanReq *reqs;
    int idx;
    long long end, t1;  // first tile past the request; past the CTA's range

    __device__ __forceinline__ void start(const PlanCta &c, long long past, const PlanReq *all, int Hkv)
    {
        r = c.req;
        reqs = all;
        idx = c.idx;
        t1 = past;
        set_end(Hkv);
        if (end < t1)
            next = reqs[idx + 1];
    }
    __device__ __forceinline__ void set_end(int Hkv) { end = r.tile_base + (long long)r.T * Hkv; }
    // moves on to the request of tile t
    __device__ __forceinline__ void seek(long long t, int Hkv)
    {
        while (t >= end) {
            r = next;
            ++idx;
            set_end(Hkv);
            if (end < t1)
                next = reqs[idx + 1];
        }
    }
};

// A run of tiles of one unit.
struct Seg {
    int head, j0, n;
};
__device__ __forceinline__ Seg seg_at(const Cursor &c, long long t)
{
    Seg g;
    const long long tl = t - c.r.tile_base;
    g.head = (unsigned long long)tl <= 0xffffffffull ? (int)((uint32_t)tl / (uint32_t)c.r.T) : (int)(tl / c.r.T);
    g.j0 = (int)(tl - (long long)g.head * c.r.T);
    const long long left = c.t1 - t;
    g.n = left < c.r.T - g.j0 ? (int)left : c.r.T - g.j0;
    return g;
}
__device__ __forceinline__ int tile_key(int j, int a0, int n1, int b0)
{
    return (j < n1 ? a0 + j : b0 + j - n1) * kBN;
}

// What the softmax needs of a segment, written with its queries.
struct SegInfo {
    int n, j0, a0, n1, b0;
    int L, end, begin, far, lo_min, lo_max;  // far: end of the kept first tokens within the prefix
    int lo[128];         // per row: the first prefix slot that its window sees
    uint64_t anc[128];   // tree nodes that it sees
    uint64_t path[128];  // its root path
    int pos[128];
    float slope[128];    // times log2(e)
    float m[128], l[2][128];  // written back by the softmax (a sum of each half)
};

// 8 elements of two bytes in the order that codes are unpacked in, and back.
__device__ __forceinline__ uint4 code_order(const uint4 &x)
{
    return make_uint4(__byte_perm(x.x, x.z, 0x5410), __byte_perm(x.x, x.z, 0x7632), __byte_perm(x.y, x.w, 0x5410),
                      __byte_perm(x.y, x.w, 0x7632));
}
// where element e of 8 stands in that order
__device__ constexpr int code_place(int e)
{
    return e < 4 ? 2 * e : 2 * (e - 4) + 1;
}

// Shared memory by its 32-bit address.
__device__ __forceinline__ uint32_t lds8(uint32_t a)
{
    uint32_t x;
    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(x) : "r"(a));
    return x;
}
__device__ __forceinline__ uint32_t lds32(uint32_t a)
{
    uint32_t x;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(x) : "r"(a));
    return x;
}
__device__ __forceinline__ uint2 lds64(uint32_t a)
{
    uint2 x;
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(x.x), "=r"(x.y) : "r"(a));
    return x;
}
__device__ __forceinline__ uint4 lds128(uint32_t a)
{
    uint4 x;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(a));
    return x;
}

__device__ __forceinline__ void sts128(uint32_t a, const uint32_t (&x)[4])
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3])
                 : "memory");
}

// The packed tile of 128 keys: pieces of min(page_size, 128) keys, each as it lies in its page: its keys'
// codes, then their scales.
struct PackedTile {
    int log2;  // keys of a piece
    __device__ __forceinline__ explicit PackedTile(int page_log2) : log2(min(page_log2, 7)) {}
    template <int kD>
    __device__ __forceinline__ int codes(int key) const
    {
        return key * code_bytes(kD) + (key & -(1 << log2)) * scale_bytes(kD);
    }
    template <int kD>
    __device__ __forceinline__ int scales(int key) const
    {
        return (key & -(1 << log2)) * code_bytes(kD) + key * scale_bytes(kD) + (code_bytes(kD) << log2);
    }
};

template <int kD>
constexpr int kTileBlocks = kBN * kD / kGroup / 32;

// Part of a packed tile into one of 16-bit elements, by a warp: 32 elements of a key per lane and block, 8 keys
// of 128 elements or 16 of 64; blocks first to first + n - 1.  holes: the pieces that are not there, whose
// elements count as zeros.

template <int kD, bool kF16>
__device__ __forceinline__ void unpack_blocks(uint32_t packed, uint32_t tile, const PackedTile &pt, uint32_t holes, int first,
                                              int n)
{
    constexpr int kChunks = kD / kGroup, kKeys = 32 / kChunks;
    const int lane = threadIdx.x & 31, chunk = lane % kChunks;
    // eight neighbouring lanes write eight different 16-byte columns: those of the second atom in another order
    const bool flip = kD == 128 && chunk >= 2;
    int key = first * kKeys + lane / kChunks;
    const auto load = [&](uint4 &w, float &f) {
        const uint32_t at = packed + pt.codes<kD>(key) + 16 * chunk;
        const uint2 a = lds64(at + (flip ? 8 : 0)), b = lds64(at + (flip ? 0 : 8));
        w = make_uint4(a.x, a.y, b.x, b.y);
        f = scale_of(lds8(packed + pt.scales<kD>(key) + chunk));
        if (holes)
            f = (holes >> (key >> pt.log2)) & 1u ? 0.f : f;
    };
    uint32_t to = tile + (flip ? kAtom : 0) + key * 128;
    uint32_t column[4];  // (a block's keys are a multiple of 8: key & 7 stays)
#pragma unroll
    for (int j = 0; j < 4; ++j)
        column[j] = (((chunk & 1) * 4 + (flip ? j ^ 2 : j)) ^ (key & 7)) * 16;
    uint4 w, next{};
    float f, next_f = 0.f;
    load(w, f);
    // (a short loop: four roles' unrolled code does not fit the instruction caches)
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
        key += kKeys;
        if (i + 1 < n)
            load(next, next_f);
        const OperandScale<kF16> s = operand_scale<kF16>(f, f);
        const uint32_t words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t e[4];
            dequant_four<kF16>(words[j], s, e);
            sts128(to + column[j], e);
        }
        to += kKeys * 128;
        w = next;
        f = next_f;
    }
}

}  // namespace

}  // namespace tv

#include "paged_attention_few.cuh"

namespace tv {

namespace {

// What the kernel keeps in dynamic shared memory: the tiles of K and V; for 4-bit pages also the packed
// tiles and the segments' records, or all that few rows take.
template <int kD, bool kQ4>
constexpr int smem_bytes()
{
    const int tiles = (k_stages(kQ4) + kVStages) * tile_bytes(kD);
    const int many = tiles + (kQ4 ? 2 * kPackedStages * packed_bytes(kD) + 2 * (int)sizeof(SegInfo) : 0);
    const int few = kQ4 ? (int)sizeof(FewSmem<kD>) : 0;
    return (many > few ? many : few) + 1024;
}

template <int kD, bool kF16, int kForm, bool kQ4>
__global__ void __launch_bounds__(kThreads, 1) k_paged_attention(const __grid_constant__ PagedArgs p)
{
    constexpr int kTile = tile_bytes(kD), kSlot = slot_floats(kD), kKStages = k_stages(kQ4);
    constexpr int kPacked = packed_bytes(kD);
    // fp16 weights are held 2^8 larger, so that small ones keep their bits above the
    // subnormals; the largest stays below 2^15
    constexpr float kShift = kF16 ? 8.f : 0.f, kGrow = kF16 ? 7.f : 8.f;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t k_full[kMaxStages], k_empty[kMaxStages], v_full[kMaxStages], v_empty[kMaxStages];
    __shared__ __align__(8) uint64_t s_full[2], p_full[2], pv_done[2], q_full[2], ml_full[2], o_free[2], drain_bar;
    __shared__ __align__(8) uint64_t never_bar[2];
    __shared__ __align__(8) uint64_t mx_full[4][2];  // per lane quadrant: both halves' row maxima are there
    __shared__ float s_mx[2][2][128];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag, s_ok;
    __shared__ __align__(8) PlanCta s_cta;
    struct None {
    };
    __shared__ std::conditional_t<kQ4, None, SegInfo[2]> info;
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *sK = smem, *sV = smem + (size_t)kKStages * kTile;
    // 4-bit pages: the packed tiles of K, filled by warp 0 and emptied by warps 8-11, and of V, filled by warp 1 and
    // emptied by warps 0-2
    uint8_t *const packed = sV + (size_t)kVStages * kTile;
    __shared__ __align__(8) uint64_t packed_full[kQ4 ? 2 : 1][kPackedStages], packed_empty[kQ4 ? 2 : 1][kPackedStages];
    __shared__ uint32_t packed_holes[kQ4 ? 2 : 1][kPackedStages];
    __shared__ int s_rows;  // 4-bit pages: of the CTA's largest unit
    SegInfo *const s_info = [&] {
        if constexpr (kQ4)
            return reinterpret_cast<SegInfo *>(packed + 2 * kPackedStages * kPacked);
        else
            return info;
    }();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = blockIdx.x;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kMaxStages; ++s) {
            mbar_init(&k_full[s], kQ4 ? 4 : 1);
            mbar_init(&k_empty[s], 1);
            mbar_init(&v_full[s], kQ4 ? 3 : 1);
            mbar_init(&v_empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&s_full[b], 1);
            mbar_init(&p_full[b], 8);
            mbar_init(&pv_done[b], 1);
            mbar_init(&q_full[b], 4);
            mbar_init(&ml_full[b], 8);
            mbar_init(&o_free[b], 4);
            mbar_init(&never_bar[b], 1);
            for (int q = 0; q < 4; ++q)
                mbar_init(&mx_full[q][b], 2);
        }
        if constexpr (kQ4) {
            for (int s = 0; s < 2 * kPackedStages; ++s) {
                mbar_init(&packed_full[s / kPackedStages][s % kPackedStages], 1);
                mbar_init(&packed_empty[s / kPackedStages][s % kPackedStages], s < kPackedStages ? 4 : 3);
            }
        }
        mbar_init(&drain_bar, kQ4 ? 1 : 2);  // issuing threads
        abort_flag = 0;
        fence_mbar_init();
        if constexpr (!kQ4) {
            prefetch_tmap(&p.tk);
            prefetch_tmap(&p.tv);
        }
    }
    if (warp == 1) {
        tmem_alloc(&tmem_slot, 512);
        tmem_relinquish();
    }
    pdl_wait();
    pdl_trigger();
    if (warp == 2) {
        if (lane < (int)(sizeof(PlanCta) / 8))
            reinterpret_cast<long long *>(&s_cta)[lane] = reinterpret_cast<const long long *>(plan_ctas(p.plan) + c)[lane];
        if (lane == 31) {
            const PlanHeader *hd = static_cast<const PlanHeader *>(p.plan);
            s_ok = hd->valid && hd->batch == p.batch && hd->n_q_heads == p.Hq && hd->n_kv_heads == p.Hkv;
            if (!s_ok)
                atomicOr(p.status, kStatusBounds);
        }
        if constexpr (kQ4) {
            // the requests of this CTA's range follow one another
            __syncwarp();
            const PlanReq *all = plan_reqs(p.plan);
            int rows = s_cta.req.n * p.group - s_cta.rb * 128;
            const bool several = s_cta.req.tile_base + (long long)s_cta.req.T * p.Hkv < s_cta.t1;
            for (int i0 = s_cta.idx; several; i0 += 32) {
                const int i = i0 + lane;
                const bool in = i < p.batch && all[i].tile_base < s_cta.t1;
                const uint32_t run = __ballot_sync(0xffffffffu, in);
                const int n = run == 0xffffffffu ? 32 : __ffs((int)~run) - 1;
                rows = max(rows, lane < n ? all[i].n * p.group - s_cta.rb * 128 : 0);
                if (n < 32)
                    break;
            }
            rows = __reduce_max_sync(0xffffffffu, rows);
            if (lane == 0)
                s_rows = rows;
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    const long long t0 = s_ok ? s_cta.t0 : 0, t1 = s_ok ? s_cta.t1 : 0;
    const PlanReq *reqs = plan_reqs(p.plan);
    // Few rows, unless the CTA's share is short: their way there and the join of 16 runs cost 7 us more than a tile's
    // way through the tensor cores (4 rows of 8 kv heads at 2000 keys: 18.2 and 16.8 us, at 8000 keys 23.7 and
    // 26.6, at 131000 keys 55 and 107).  All threads of the CTA alike.
    const bool few = kQ4 && s_rows <= kFewRows && t1 - t0 > kFewTiles;

    // 4-bit pages: this warp's blocks of tile i (of K or V)
    [[maybe_unused]] const auto unpack = [&](bool is_v, int i, int first, int n) {
        const int ps = i % kPackedStages, S = is_v ? kVStages : kKStages, s = i % S;
        if (!warp_agrees(mbar_wait_bounded(&packed_full[is_v][ps], (uint32_t)(i / kPackedStages) & 1u, &abort_flag,
                                           p.status)) ||
            !warp_agrees(mbar_wait_bounded(is_v ? &v_empty[s] : &k_empty[s], ((uint32_t)(i / S) & 1u) ^ 1u, &abort_flag,
                                           p.status)))
            return false;
        unpack_blocks<kD, kF16>(smem_u32(packed) + ((is_v ? kPackedStages : 0) + ps) * kPacked,
                                smem_u32(is_v ? sV : sK) + s * kTile, PackedTile(p.page_log2), packed_holes[is_v][ps], first,
                                n);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
            mbar_arrive(&packed_empty[is_v][ps]);
            mbar_arrive(is_v ? &v_full[s] : &k_full[s]);
        }
        return true;
    };
    // K's blocks lie with warps 8-11, V's with 0-2 so that none takes much longer than the others: copying a tile
    // costs warps 0 and 1 as much as four blocks or so
    constexpr int kBlocks = kTileBlocks<kD>, kShare = kBlocks / 4;  // of V, for warps 0 and 1
    if (kQ4 && few) {
        if constexpr (kQ4) {
            FewSmem<kD> &sm = *reinterpret_cast<FewSmem<kD> *>(smem);
            few_rows<kD, kF16, kForm>(p, s_cta, sm, &abort_flag, &never_bar[0]);
        }
    } else if (kQ4 && warp < 4) {
        if constexpr (kQ4) {
            const int all = (int)(t1 - t0);
            if (warp == 3) {
                // ------------------------------------------------ both products, whichever is ready.  The whole warp
                // goes through this (what it decides by is voted on) and one lane issues: addresses and descriptors
                // then stay in uniform registers
                struct Walk {
                    Cursor cur;
                    Seg g{0, 0, 0};
                    long long t;
                    int it = 0, j = 0, sg = -1;
                    bool first = false;  // tile `it` begins a segment
                } wq, wp;
                wq.cur.start(s_cta, t1, reqs, p.Hkv);
                wp.cur.start(s_cta, t1, reqs, p.Hkv);
                wq.t = wp.t = t0;
                const auto next = [&](Walk &w) {
                    w.first = w.j == w.g.n;
                    if (!w.first)
                        return;
                    w.t += w.g.n;
                    w.cur.seek(w.t, p.Hkv);
                    w.g = seg_at(w.cur, w.t);
                    w.g.n = __shfl_sync(0xffffffffu, w.g.n, 0);
                    w.j = 0;
                    ++w.sg;
                };
                const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
                const uint64_t k_desc = smem_desc_sw128(smem_u32(sK), 0, 1024), v_desc = smem_desc_sw128(smem_u32(sV), kAtom, 1024);
                const auto scores_ready = [&] {
                    const int it = wq.it;
                    return warp_agrees(mbar_test(&k_full[it % kKStages], (uint32_t)(it / kKStages) & 1u) &&
                                       (it < 2 || mbar_test(&pv_done[it & 1], (uint32_t)((it - 2) >> 1) & 1u)) &&
                                       (!wq.first || mbar_test(&q_full[wq.sg & 1], (uint32_t)(wq.sg >> 1) & 1u)));
                };
                const auto scores = [&] {
                    const int b = wq.it & 1, s = wq.it % kKStages;
                    tc_fence_after();
                    if (elect_one()) {
                        const uint32_t q_col = tm + kColQ + (wq.sg & 1) * (kD / 2);
                        const uint64_t desc = k_desc + (uint32_t)(s * (kTile >> 4));
#pragma unroll
                        for (int kk = 0; kk < kD / 16; ++kk)
                            tc_mma_f16_ts(tm + kColS + b * 128, q_col + kk * 8,
                                          desc + (((kk >> 2) * kAtom + (kk & 3) * 32) >> 4), idesc<kF16>(kBN, false),
                                          kk > 0 ? 1u : 0u);
                        tc_commit(&s_full[b]);
                        tc_commit(&k_empty[s]);
                    }
                    __syncwarp();
                    ++wq.j;
                    if (++wq.it < all)
                        next(wq);
                };
                uint64_t *const p_ready = p.expire_wait ? never_bar : p_full;
                const auto outputs_ready = [&] {
                    const int it = wp.it;
                    return warp_agrees(mbar_test(&p_ready[it & 1], (uint32_t)(it >> 1) & 1u) &&
                                       (!wp.first || wp.sg == 0 ||
                                        mbar_test(&o_free[(wp.sg - 1) & 1], (uint32_t)((wp.sg - 1) >> 1) & 1u)) &&
                                       mbar_test(&v_full[it % kVStages], (uint32_t)(it / kVStages) & 1u));
                };
                const auto outputs = [&] {
                    const int b = wp.it & 1, s = wp.it % kVStages;
                    tc_fence_after();
                    if (elect_one()) {
                        const uint64_t desc = v_desc + (uint32_t)(s * (kTile >> 4));
                        const uint32_t fresh = wp.first ? 0u : 1u;
#pragma unroll
                        for (int ks = 0; ks < kBN / 16; ++ks)
                            tc_mma_f16_ts(tm + kColO, tm + kColS + b * 128 + (ks >> 2) * 64 + (ks & 3) * 8,
                                          desc + ((ks * 2048) >> 4), idesc<kF16>(kD, true), ks == 0 ? fresh : 1u);
                        tc_commit(&v_empty[s]);
                        tc_commit(&pv_done[b]);
                    }
                    __syncwarp();
                    ++wp.j;
                    if (++wp.it < all)
                        next(wp);
                };
                if (all > 0)
                    next(wq), next(wp);
                long long idle = cycles();
                while (wp.it < all) {
                    if (outputs_ready()) {  // (tile `it`'s weights are there, so its scores have been issued)
                        outputs();
                    } else if (wq.it < all && scores_ready()) {
                        scores();
                    } else {
                        if (!warp_agrees(*const_cast<volatile int *>(&abort_flag) == 0))
                            break;
                        if (!warp_agrees(cycles() - idle <= kWaitLimitCycles)) {
                            *const_cast<volatile int *>(&abort_flag) = 1;
                            if (lane == 0)
                                atomicOr(p.status, kStatusTimeout);
                            break;
                        }
                        continue;
                    }
                    idle = cycles();
                }
                if (elect_one())
                    tc_commit(&drain_bar);
                __syncwarp();
            } else {
                // ------------------------------------------------ V; warp 0 copies K's tiles, warp 1 V's
                const bool is_v = warp == 1;
                uint64_t *full = packed_full[is_v], *empty = packed_empty[is_v];
                uint8_t *ring = packed + (is_v ? kPackedStages * kPacked : 0);
                const int pages_log2 = p.page_log2 >= 7 ? 0 : 7 - p.page_log2;  // pages of a tile: one per lane
                const int keys = min(1 << p.page_log2, kBN);
                const bool box = lane < 1 << pages_log2;
                Cursor cur;
                cur.start(s_cta, t1, reqs, p.Hkv);
                const auto report_hole = [&](int slot) {
                    const int window = static_cast<const PlanHeader *>(p.plan)->window, past = slot + keys;
                    const int lo_min = window > 0 ? max(cur.r.begin, cur.r.L - window + 1) : cur.r.begin;
                    if (past > lo_min ||
                        (window > 0 && past > cur.r.begin && slot < min(cur.r.far_end, cur.r.L)))
                        atomicOr(p.status, kStatusBounds);
                };
                // of the segment that is being copied: where its pages lie, its tile and past its last one; this
                // lane's page of the next tile, looked up a tile ahead
                const int32_t *table = nullptr;
                const uint8_t *pages = nullptr;
                Seg g{0, 0, 0};
                int j = 0, past = 0, copied = 0, id = -1, slot = 0;
                const auto look_up = [&] {
                    slot = tile_key(j, cur.r.a0, cur.r.n1, cur.r.b0) + (lane << p.page_log2);
                    const int at = slot >> p.page_log2;
                    id = -1;
                    if (box && slot < past && at < p.max_pages)
                        id = table[at];
                };
                const auto copy_tile = [&] {  // the next one, once its stage is free
                    if (copied == 0 || j == g.j0 + g.n) {
                        const long long t = t0 + copied;
                        cur.seek(t, p.Hkv);
                        g = seg_at(cur, t);
                        j = g.j0;
                        past = cur.r.L + cur.r.n;
                        table = p.table + (size_t)cur.r.b * p.max_pages;
                        pages = (is_v ? p.v_pages : p.k_pages) + g.head * p.head_stride;
                        look_up();
                    }
                    const int s = copied % kPackedStages;
                    if (!warp_agrees(mbar_wait_bounded(&empty[s], ((uint32_t)(copied / kPackedStages) & 1u) ^ 1u,
                                                       &abort_flag, p.status)))
                        return false;
                    // a page's block, or a tile's part of its codes and of its scales; nothing for holes
                    const bool inside = box && slot < past, there = inside && (unsigned)id < (unsigned)p.n_pages;
                    const uint32_t found = __ballot_sync(0xffffffffu, there);
                    const uint32_t holes = __ballot_sync(0xffffffffu, inside) & ~found;
                    if (lane == 0) {
                        packed_holes[is_v][s] = holes;
                        mbar_arrive_expect_tx(&full[s], __popc(found) * keys * row_bytes(kD));
                    }
                    __syncwarp();
                    if (there) {
                        const uint8_t *src = pages + ((unsigned long long)(unsigned)id * p.page_units << 4);
                        uint8_t *dst = ring + s * kPacked + lane * keys * row_bytes(kD);
                        if (p.page_log2 <= 7) {
                            bulk_load(dst, src, keys * row_bytes(kD), &full[s]);
                        } else {
                            const int at = slot & ((1 << p.page_log2) - 1);
                            bulk_load(dst, src + at * code_bytes(kD), kBN * code_bytes(kD), &full[s]);
                            bulk_load(dst + kBN * code_bytes(kD),
                                      src + ((long long)code_bytes(kD) << p.page_log2) + at * scale_bytes(kD),
                                      kBN * scale_bytes(kD), &full[s]);
                        }
                    }
                    if (holes && inside && !there && !is_v)
                        report_hole(slot);
                    ++copied;
                    if (++j < g.j0 + g.n)
                        look_up();
                    return true;
                };
                bool ok = true;
                for (int it = 0; ok && it < all; ++it) {
                    while (ok && warp < 2 && copied < min(all, it + kPackedStages))
                        ok = copy_tile();
                    ok = ok && unpack(true, it, warp * kShare, warp < 2 ? kShare : kBlocks - 2 * kShare);
                }
                if (lane == 0 && warp < 2)  // (some other warp may have given up)
                    for (int x = max(copied - kPackedStages, 0); x < copied; ++x)
                        mbar_wait_drain(&full[x % kPackedStages], (uint32_t)(x / kPackedStages) & 1u);
                __syncwarp();
            }
        }
    } else if (warp < 4) {
        Cursor cur;  // (a CTA without tiles has an empty one)
        cur.start(s_cta, t1, reqs, p.Hkv);
        if (warp == 0 || warp == 3) {
            // ------------------------------------------------ producers: a page per lane
            const bool is_v = warp == 3;
            uint64_t *full = is_v ? v_full : k_full;
            uint64_t *empty = is_v ? v_empty : k_empty;
            const int S = is_v ? kVStages : kKStages;
            uint8_t *ring = is_v ? sV : sK;
            const CUtensorMap *map = is_v ? &p.tv : &p.tk;
            const int pages_log2 = p.page_log2 >= 7 ? 0 : 7 - p.page_log2;  // pages of a tile
            const int a = lane >> pages_log2, pg = lane & ((1 << pages_log2) - 1);
            const bool box = a < kD / 64;
            const uint32_t dst_off = (uint32_t)a * kAtom + ((uint32_t)pg << (p.page_log2 + 7));
            const int page_mask = (1 << p.page_log2) - 1;
            // this lane's page of tile j of the current request; nothing is asked of it before its tile's turn
            struct Page {
                int id;
                bool inside;  // the request has slots in it
            };
            auto first_slot = [&](int j) { return tile_key(j, cur.r.a0, cur.r.n1, cur.r.b0) + (pg << p.page_log2); };
            auto page_of = [&](int j) {
                const int slot = first_slot(j), at = slot >> p.page_log2;
                Page x{-1, box && slot < cur.r.L + cur.r.n};
                if (x.inside && at < p.max_pages)
                    x.id = p.table[(size_t)cur.r.b * p.max_pages + at];
                return x;
            };
            // a hole in the table: reported, if some row may see one of the slots
            auto report_hole = [&](int slot) {
                const int window = static_cast<const PlanHeader *>(p.plan)->window, past = slot + min(1 << p.page_log2, kBN);
                const int lo_min = window > 0 ? max(cur.r.begin, cur.r.L - window + 1) : cur.r.begin;
                if (past > lo_min || (window > 0 && past > cur.r.begin && slot < min(cur.r.far_end, cur.r.L)))
                    atomicOr(p.status, kStatusBounds);
            };
            long long issued = 0;
            int s = 0;
            uint32_t ph = 0;
            bool ok = true;
            for (long long t = t0; ok && t < t1;) {
                cur.seek(t, p.Hkv);
                const Seg g = seg_at(cur, t);
                Page page = page_of(g.j0);
                for (int j = 0; j < g.n; ++j) {
                    const Page next = j + 1 < g.n ? page_of(g.j0 + j + 1) : Page{-1, false};
                    if (lane == 0)
                        ok = mbar_wait_bounded(&empty[s], ph ^ 1u, &abort_flag, p.status);
                    ok = __shfl_sync(0xffffffffu, ok, 0);
                    if (!ok)
                        break;
                    if (lane == 0)
                        mbar_arrive_expect_tx(&full[s], kTile);
                    __syncwarp();
                    const bool there = page.id >= 0 && page.id < p.n_pages;
                    if (box)  // past the last page: zeros
                        tma_load_4d(ring + (size_t)s * kTile + dst_off, map, &full[s], 64 * a,
                                    p.page_log2 > 7 ? tile_key(g.j0 + j, cur.r.a0, cur.r.n1, cur.r.b0) & page_mask : 0,
                                    g.head, there ? page.id : p.n_pages);
                    if (page.inside && !there && !is_v)
                        report_hole(first_slot(g.j0 + j));
                    page = next;
                    ++issued;
                    if (++s == S) {
                        s = 0;
                        ph ^= 1u;
                    }
                }
                t += g.n;
            }
            if (!ok && lane == 0)
                for (long long it = (issued > S ? issued - S : 0); it < issued; ++it)
                    mbar_wait_drain(&full[it % S], (uint32_t)(it / S) & 1u);
            __syncwarp();
        } else if (lane == 0 && warp == 1) {
            // ------------------------------------------------ Q K^T issuer
            long long it = 0;
            int s = 0, sg = 0;
            uint32_t ph = 0;
            bool ok = true;
            for (long long t = t0; ok && t < t1; ++sg) {
                cur.seek(t, p.Hkv);
                const Seg g = seg_at(cur, t);
                const uint32_t q_col = tmem + kColQ + (sg & 1) * (kD / 2);
                for (int j = 0; j < g.n; ++j, ++it) {
                    const int b = (int)(it & 1);
                    // K landed; P V(it - 2) has read P_b, whose columns are S_b's; at a segment's
                    // first tile, its queries are staged
                    if (!mbar_wait_bounded(&k_full[s], ph, &abort_flag, p.status) ||
                        (it >= 2 &&
                         !mbar_wait_bounded(&pv_done[b], (uint32_t)((it - 2) >> 1) & 1u, &abort_flag, p.status)) ||
                        (j == 0 &&
                         !mbar_wait_bounded(&q_full[sg & 1], (uint32_t)(sg >> 1) & 1u, &abort_flag, p.status))) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t k_base = smem_u32(sK + (size_t)s * kTile);
#pragma unroll
                    for (int kk = 0; kk < kD / 16; ++kk) {
                        const uint32_t off = (uint32_t)(kk >> 2) * kAtom + (uint32_t)(kk & 3) * 32;
                        tc_mma_f16_ts(tmem + kColS + b * 128, q_col + kk * 8, smem_desc_sw128(k_base + off, 0, 1024),
                                      idesc<kF16>(kBN, false), kk > 0 ? 1u : 0u);
                    }
                    tc_commit(&s_full[b]);
                    tc_commit(&k_empty[s]);
                    if (++s == kKStages) {
                        s = 0;
                        ph ^= 1u;
                    }
                }
                t += g.n;
            }
            tc_commit(&drain_bar);
        } else if (lane == 0) {
            // ------------------------------------------------ P V issuer
            uint64_t *const p_ready = p.expire_wait ? never_bar : p_full;
            long long it = 0;
            int s = 0, sg = 0;
            uint32_t ph = 0;
            bool ok = true;
            for (long long t = t0; ok && t < t1; ++sg) {
                cur.seek(t, p.Hkv);
                const Seg g = seg_at(cur, t);
                for (int j = 0; j < g.n; ++j, ++it) {
                    const int b = (int)(it & 1);
                    // P written; at a segment's first tile, the previous segment's O has been read
                    if (!mbar_wait_bounded(&p_ready[b], (uint32_t)(it >> 1) & 1u, &abort_flag, p.status) ||
                        (j == 0 && sg > 0 &&
                         !mbar_wait_bounded(&o_free[(sg - 1) & 1], (uint32_t)((sg - 1) >> 1) & 1u, &abort_flag,
                                            p.status)) ||
                        !mbar_wait_bounded(&v_full[s], ph, &abort_flag, p.status)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t v_base = smem_u32(sV + (size_t)s * kTile);
#pragma unroll
                    for (int ks = 0; ks < kBN / 16; ++ks)
                        tc_mma_f16_ts(tmem + kColO, tmem + kColS + b * 128 + (ks >> 2) * 64 + (ks & 3) * 8,
                                      smem_desc_sw128(v_base + ks * 2048, kAtom, 1024), idesc<kF16>(kD, true),
                                      (j == 0 && ks == 0) ? 0u : 1u);
                    tc_commit(&v_empty[s]);
                    tc_commit(&pv_done[b]);
                    if (++s == kVStages) {
                        s = 0;
                        ph ^= 1u;
                    }
                }
                t += g.n;
            }
            tc_commit(&drain_bar);
        }
    } else if (warp < 8 || warp >= 12) {
        // ---------------------------------------------------- softmax (warps 4-7 and 12-15)
        // two threads per row: the lower half of a tile's columns and the upper one
        const int q4 = warp & 3, half = warp >= 12 ? 1 : 0;
        const uint32_t lane_addr = tmem + ((uint32_t)(32 * q4) << 16);
        const int rloc = 4 * lane + q4;
        long long it = 0;
        bool aborted = false;
        int sg = 0;
        for (long long t = t0; t < t1 && !aborted; ++sg) {
            SegInfo &si = s_info[sg & 1];
            if (!warp_agrees(mbar_wait_bounded(&q_full[sg & 1], (uint32_t)(sg >> 1) & 1u, &abort_flag, p.status)))
                break;
            const int n = si.n, L = si.L, end = si.end, lo = si.lo[rloc], pos = si.pos[rloc];
            const uint64_t anc = si.anc[rloc], path = kForm == kBias ? si.path[rloc] : 0;
            const float slope = si.slope[rloc];
            t += n;
            float m_ref = -INFINITY, l = 0.f;
            for (int j = 0; j < n; ++j, ++it) {
                const int b = (int)(it & 1);
                const int key0 = tile_key(si.j0 + j, si.a0, si.n1, si.b0);
                // (a wait that ran out is looked at where the warp votes anyway, below; until then it
                // goes on with whatever S holds)
                bool ok = mbar_wait_bounded(&s_full[b], (uint32_t)(it >> 1) & 1u, &abort_flag, p.status);
                tc_fence_after();
                const uint32_t sa = lane_addr + kColS + b * 128 + half * kHalf;
                const int h0 = key0 + half * kHalf;  // this thread's first slot
                const bool masked = h0 + kHalf > L || h0 < si.lo_max;
                const auto visible = [&](int s0) {  // which of the 32 slots from s0 on this row sees
                    return range_bits(s0, lo, L) | range_bits(s0, si.begin, si.far) | tree_bits(s0, L, anc);
                };
                // this half's scores (kCap: their w), held in registers until they are weights
                constexpr uint32_t kHidden = kForm == kCap ? 0x7f800000u : 0xff800000u;  // z = -inf
                uint32_t r[kHalf];
                tmem_ld_32x32b_x32(sa, r);
                tmem_ld_32x32b_x32(sa + 32, r + 32);
                tmem_ld_wait();
                if constexpr (kForm != kPlain) {
                    if (kForm == kCap || p.cap > 0.f) {
                        // a NaN in a hidden slot must not reach its neighbours through the common reciprocal
                        if (masked) {
#pragma unroll
                            for (int y = 0; y < kHalf; y += 32) {
                                const uint32_t allow = visible(h0 + y);
#pragma unroll
                                for (int x = 0; x < 32; ++x)
                                    r[y + x] = (allow >> x) & 1u ? r[y + x] : 0xff800000u;
                            }
                        }
#pragma unroll
                        for (int x = 0; x < kHalf; x += 4)
                            cap_four(r + x, p.cap_in);
                        if constexpr (kForm == kBias) {
#pragma unroll
                            for (int x = 0; x < kHalf; x += 2) {
                                const float2 z = halves(fma_two(two(__uint_as_float(r[x]), __uint_as_float(r[x + 1])),
                                                                two(-2.f * p.cap, -2.f * p.cap), two(p.cap, p.cap)));
                                r[x] = __float_as_uint(z.x), r[x + 1] = __float_as_uint(z.y);
                            }
                        }
                    } else {
#pragma unroll
                        for (int x = 0; x < kHalf; ++x)
                            r[x] = __float_as_uint(__uint_as_float(r[x]) * p.scale);
                    }
                }
                if (masked) {
#pragma unroll
                    for (int y = 0; y < kHalf; y += 32) {
                        const int s0 = h0 + y;
                        if constexpr (kForm == kBias) {
                            // the distance falls by one from slot to slot of the prefix, and behind
                            // each node of the row's root path (its nodes are in order of depth)
                            float dist = (float)(s0 <= L ? pos - s0
                                                         : pos - L - (s0 - L < 64 ? __popcll(path & ((1ull << (s0 - L)) - 1))
                                                                                  : __popcll(path)));
                            const uint32_t fall = range_bits(s0, s0, L) | tree_bits(s0, L, path);
#pragma unroll
                            for (int x = 0; x < 32; ++x) {
                                r[y + x] = __float_as_uint(fmaf(-slope, dist, __uint_as_float(r[y + x])));
                                dist -= (fall >> x) & 1u ? 1.f : 0.f;
                            }
                        }
                        const uint32_t allow = visible(s0);
#pragma unroll
                        for (int x = 0; x < 32; ++x)
                            r[y + x] = (allow >> x) & 1u ? r[y + x] : kHidden;
                    }
                } else if constexpr (kForm == kBias) {
                    const float d0 = (float)(pos - h0);
                    uint64_t dist = two(d0, d0 - 1.f);
#pragma unroll
                    for (int x = 0; x < kHalf; x += 2) {
                        const float2 z = halves(fma_two(two(-slope, -slope), dist,
                                                        two(__uint_as_float(r[x]), __uint_as_float(r[x + 1]))));
                        r[x] = __float_as_uint(z.x), r[x + 1] = __float_as_uint(z.y);
                        dist = add_two(dist, two(-2.f, -2.f));
                    }
                }
                // z = f r + f0; f < 0 where r is a capped score's w
                float mx = kForm == kCap ? INFINITY : -INFINITY;
#pragma unroll
                for (int x = 0; x < kHalf; ++x)
                    mx = kForm == kCap ? fminf(mx, __uint_as_float(r[x])) : fmaxf(mx, __uint_as_float(r[x]));
                const float f = kForm == kCap ? -2.f * p.cap : kForm == kPlain ? p.scale : 1.f;
                const float f0 = kForm == kCap ? p.cap : 0.f;
                mx = fmaf(f, mx, f0);
                // the other half's
                s_mx[b][half][rloc] = mx;
                __syncwarp();
                if (lane == 0)
                    mbar_arrive(&mx_full[q4][b]);
                ok = mbar_wait_bounded(&mx_full[q4][b], (uint32_t)(it >> 1) & 1u, &abort_flag, p.status) && ok;
                mx = fmaxf(mx, s_mx[b][half ^ 1][rloc]);

                // the lazily raised reference, the same in both halves
                float alpha = 1.f;
                bool rescale = false;
                if (j == 0) {
                    m_ref = mx - kShift;
                } else if (mx > m_ref + kShift + kGrow) {
                    alpha = m_ref == -INFINITY ? 0.f : ex2_approx(m_ref - (mx - kShift));
                    m_ref = mx - kShift;
                    rescale = true;
                }
                if (__any_sync(0xffffffffu, rescale || !ok)) {
                    // O holds the previous tiles' P V: wait for the last one, then scale in place
                    const long long jp = it - 1;
                    if (!warp_agrees(ok) ||
                        !warp_agrees(mbar_wait_bounded(&pv_done[jp & 1], (uint32_t)(jp >> 1) & 1u, &abort_flag, p.status))) {
                        aborted = true;
                        break;
                    }
                    tc_fence_after();
                    l *= alpha;
#pragma unroll 1
                    for (int c0 = half * (kD / 2); c0 < (half + 1) * (kD / 2); c0 += 32) {
                        uint32_t o[32];
                        tmem_ld_32x32b_x32(lane_addr + kColO + c0, o);
                        tmem_ld_wait();
#pragma unroll
                        for (int x = 0; x < 32; ++x)
                            o[x] = __float_as_uint(__uint_as_float(o[x]) * alpha);
                        tmem_st_32x32b_x32(lane_addr + kColO + c0, o);
                    }
                    tmem_st_wait();
                }

                // P in the pages' type on the first columns of this half, its 32-bit sum into l
                const float mu = m_ref == -INFINITY ? 0.f : m_ref;
                uint64_t rs = two(0.f, 0.f);
#pragma unroll
                for (int x = 0; x < kHalf / 2; ++x) {
                    const float2 z = halves(fma_two(two(__uint_as_float(r[2 * x]), __uint_as_float(r[2 * x + 1])), two(f, f),
                                                    two(f0 - mu, f0 - mu)));
                    const float p0 = ex2_approx(z.x), p1 = ex2_approx(z.y);
                    rs = add_two(rs, two(p0, p1));
                    r[x] = pack<kF16>(p0, p1);
                }
                tmem_st_32x32b_x32(sa, r);
                l += halves(rs).x + halves(rs).y;
                if (key0 + kBN > end || key0 < si.lo_min) {
                    // V rows that nobody sees may hold anything: zeros, once the tile has landed
                    const int sv = (int)(it % kVStages);
                    if (!warp_agrees(
                            mbar_wait_bounded(&v_full[sv], (uint32_t)(it / kVStages) & 1u, &abort_flag, p.status))) {
                        aborted = true;
                        break;
                    }
                    const int slot = key0 + rloc;
                    if (slot >= end || slot < si.begin || (slot < si.lo_min && slot >= si.far)) {
                        uint8_t *row = sV + (size_t)sv * kTile + rloc * 128;
#pragma unroll
                        for (int x = half * (kD / 16); x < (half + 1) * (kD / 16); ++x)
                            *reinterpret_cast<uint4 *>(row + (x >> 3) * kAtom + (x & 7) * 16) = make_uint4(0, 0, 0, 0);
                    }
                    fence_proxy_async_smem();
                }
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0)
                    mbar_arrive(&p_full[b]);
            }
            if (aborted)
                break;
            if (sg >= 2 &&
                !warp_agrees(mbar_wait_bounded(&o_free[sg & 1], (uint32_t)((sg >> 1) - 1) & 1u, &abort_flag, p.status)))
                break;
            if (half == 0)
                si.m[rloc] = m_ref;
            si.l[half][rloc] = l;
            __syncwarp();
            if (lane == 0)
                mbar_arrive(&ml_full[sg & 1]);
        }
    } else if (t0 < t1) {
        // ---------------------------------------------------- staging and epilogue (warps 8-11)
        const int q4 = warp & 3;
        const uint32_t lane_addr = tmem + ((uint32_t)(32 * q4) << 16);
        const int rloc = 4 * lane + q4;
        struct Unit {
            int n, j0, T;
            bool first, valid;
            PlanReq r;
            size_t row;  // (row, query head) of this thread
            int node, qh;
        };
        Cursor cur;
        cur.start(s_cta, t1, reqs, p.Hkv);
        const int window = static_cast<const PlanHeader *>(p.plan)->window;
        auto describe = [&](long long t) {
            cur.seek(t, p.Hkv);
            const Seg g = seg_at(cur, t);
            Unit u;
            u.n = g.n;
            u.j0 = g.j0;
            u.T = cur.r.T;
            u.first = t == t0;
            u.r = cur.r;
            const int grow = s_cta.rb * 128 + rloc;
            u.node = grow / p.group;
            u.qh = g.head * p.group + grow % p.group;
            u.valid = u.node < cur.r.n && cur.r.row0 + u.node < p.n_rows;
            if (u.valid && (unsigned)cur.r.tree >= (unsigned)p.n_trees) {  // a plan of another bank
                atomicOr(p.status, kStatusBounds);
                u.valid = false;
            }
            if (u.valid)
                u.valid = in_bounds(u.node < kMaxNodes && u.qh < p.Hq && cur.r.row0 >= 0, p.status);
            u.row = u.valid ? (size_t)(cur.r.row0 + u.node) * p.Hq + u.qh : 0;
            return u;
        };
        auto stage = [&](Unit &u, int sg) {
            SegInfo &si = s_info[sg & 1];
            const uint32_t col = lane_addr + kColQ + (sg & 1) * (kD / 2);
            const uint4 *src = reinterpret_cast<const uint4 *>(p.q + u.row * kD);
            uint4 qv[kD / 8];
#pragma unroll
            for (int i = 0; i < kD / 8; ++i)
                qv[i] = u.valid ? src[i] : make_uint4(0, 0, 0, 0);
            // what this row sees
            const TreeDesc &td = p.trees[(unsigned)u.r.tree < (unsigned)p.n_trees ? u.r.tree : 0];
            const int L = u.r.L, node = u.valid ? u.node : 0;
            int dep = td.depth[node];
            uint64_t anc = td.anc[node];
            if (u.valid && td.n != u.r.n) {
                atomicOr(p.status, kStatusBounds);
                u.valid = false;
            }
            dep = u.valid ? dep : 0;
            anc = u.valid ? anc : 0ull;
            if constexpr (kForm == kBias)
                si.path[rloc] = anc;
            if (window > 0 && dep >= window) {
                // ancestors that the window has left behind
                uint64_t near = 0;
                for (int node = u.node; node >= 0; node = td.parent[node])
                    if (dep - td.depth[node] < window || L + node < u.r.far_end)
                        near |= 1ull << node;
                anc &= near;
            }
            if (u.r.begin > L)
                anc &= u.r.begin - L < 64 ? ~0ull << (u.r.begin - L) : 0ull;
            const int lo_min = window > 0 ? max(u.r.begin, L - window + 1) : u.r.begin;
            si.anc[rloc] = anc;
            si.lo[rloc] = window > 0 ? max(u.r.begin, L + dep - window + 1) : u.r.begin;
            si.pos[rloc] = L + dep;
            si.slope[rloc] = kForm == kBias && u.valid && p.slopes ? p.slopes[u.qh] * kLog2e : 0.f;
            if (lane == 0) {  // the same words from every warp
                si.n = u.n;
                si.j0 = u.j0;
                si.a0 = u.r.a0;
                si.n1 = u.r.n1;
                si.b0 = u.r.b0;
                si.L = L;
                si.end = L + u.r.n;
                si.begin = u.r.begin;
                si.far = window > 0 ? min(u.r.far_end, L) : u.r.begin;
                si.lo_min = lo_min;
                si.lo_max = window > 0 ? max(u.r.begin, L + td.max_depth - window + 1) : u.r.begin;
            }
#pragma unroll
            for (int qc = 0; qc < kD / 32; ++qc) {
                uint32_t w[16];
#pragma unroll
                for (int ch = 0; ch < 4; ++ch) {
                    const uint4 x = kQ4 ? code_order(qv[qc * 4 + ch]) : qv[qc * 4 + ch];
                    w[4 * ch] = x.x;
                    w[4 * ch + 1] = x.y;
                    w[4 * ch + 2] = x.z;
                    w[4 * ch + 3] = x.w;
                }
                tmem_st_32x32b_x16(col + qc * 16, w);
            }
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0)
                mbar_arrive(&q_full[sg & 1]);
        };
        // 4-bit pages: K's tiles unpacked so far
        [[maybe_unused]] int k_done = 0;
        [[maybe_unused]] const auto unpack_to = [&](int n) {
            for (n = min(n, (int)(t1 - t0)); k_done < n; ++k_done)
                if (!unpack(false, k_done, q4 * (kBlocks / 4), kBlocks / 4))
                    return false;
            return true;
        };
        long long t = t0;
        Unit now = describe(t);
        stage(now, 0);
        t += now.n;
        Unit nxt{};
        bool has_next = t < t1;
        if (has_next) {
            nxt = describe(t);
            stage(nxt, 1);
            t += nxt.n;
        }
        long long it = 0;
        for (int sg = 0;; ++sg) {
            it += now.n;
            Unit fut{};
            const bool has_fut = t < t1;
            if (has_fut) {
                fut = describe(t);
                t += fut.n;
                if (fut.valid) {
#pragma unroll
                    for (int off = 0; off < 2 * kD; off += 128)
                        asm volatile("prefetch.global.L2 [%0];" ::"l"(reinterpret_cast<const char *>(p.q + fut.row * kD) +
                                                                      off));
                }
            }
            const long long last = it - 1;
            if constexpr (kQ4) {
                // through the next unit's first two tiles: their scores do not wait for this unit's output to be read
                if (!unpack_to((int)it + 2))
                    break;
            }
            if (!warp_agrees(mbar_wait_bounded(&ml_full[sg & 1], (uint32_t)(sg >> 1) & 1u, &abort_flag, p.status)))
                break;
            const float m_ref = s_info[sg & 1].m[rloc], l = s_info[sg & 1].l[0][rloc] + s_info[sg & 1].l[1][rloc];
            if (!warp_agrees(mbar_wait_bounded(&pv_done[last & 1], (uint32_t)(last >> 1) & 1u, &abort_flag, p.status)))
                break;
            tc_fence_after();
            const bool whole = now.n == now.T;
            // of 4-bit pages, the elements entered times a power of two
            constexpr float kBack = kQ4 ? 1.f / kOperandScale<kF16> : 1.f;
            const float inv = l == 0.f ? 0.f : kBack / l;  // a NaN stays one
            uint4 *dst = reinterpret_cast<uint4 *>(p.out + now.row * kD);
            float *slot = p.part + ((size_t)c * 2 + (now.first ? 0 : 1)) * kSlot;
            float4 *pdst = reinterpret_cast<float4 *>(slot + rloc * kD);
#pragma unroll 1
            for (int c0 = 0; c0 < kD; c0 += 32) {
                uint32_t r[32];
                tmem_ld_32x32b_x32(lane_addr + kColO + c0, r);
                tmem_ld_wait();
                if constexpr (kQ4) {
                    uint32_t o[32];
#pragma unroll
                    for (int x = 0; x < 32; ++x)
                        o[x] = r[(x & ~7) + code_place(x & 7)];
#pragma unroll
                    for (int x = 0; x < 32; ++x)
                        r[x] = o[x];
                }
                if (c0 + 32 == kD) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0)
                        mbar_arrive(&o_free[sg & 1]);
                }
                if (!now.valid)
                    continue;
                if (whole) {
#pragma unroll
                    for (int ch = 0; ch < 4; ++ch) {
                        uint4 v;
                        v.x = pack<kF16>(__uint_as_float(r[8 * ch + 0]) * inv, __uint_as_float(r[8 * ch + 1]) * inv);
                        v.y = pack<kF16>(__uint_as_float(r[8 * ch + 2]) * inv, __uint_as_float(r[8 * ch + 3]) * inv);
                        v.z = pack<kF16>(__uint_as_float(r[8 * ch + 4]) * inv, __uint_as_float(r[8 * ch + 5]) * inv);
                        v.w = pack<kF16>(__uint_as_float(r[8 * ch + 6]) * inv, __uint_as_float(r[8 * ch + 7]) * inv);
                        dst[c0 / 8 + ch] = v;
                    }
                } else {
#pragma unroll
                    for (int x = 0; x < 8; ++x)
                        pdst[c0 / 4 + x] =
                            make_float4(__uint_as_float(r[4 * x]) * kBack, __uint_as_float(r[4 * x + 1]) * kBack,
                                        __uint_as_float(r[4 * x + 2]) * kBack, __uint_as_float(r[4 * x + 3]) * kBack);
                }
            }
            if (now.valid && whole) {
                if (p.lse)
                    p.lse[now.row] = l == 0.f ? -INFINITY : (m_ref + log2f(l)) * kLn2;
            } else if (now.valid) {
                slot[128 * kD + rloc] = m_ref;
                slot[128 * kD + 128 + rloc] = l;
            }
            if (!has_next)
                break;
            if (has_fut)
                stage(fut, sg + 2);
            now = nxt;
            nxt = fut;
            has_next = has_fut;
        }
    }

    tc_fence_before();
    __syncwarp();
    __syncthreads();
    if (warp == 1) {
        if (lane == 0 && !few)
            mbar_wait_drain(&drain_bar, 0);
        __syncwarp();
        tmem_dealloc(tmem, 512);
    }
}

// Log-sum-exp join of the partials of the units that CTAs share, in CTA order (the
// same sums every time).  A group of 8 lanes takes a row, kD / 8 columns each:
// group w row w % 2^rows_log2 of split w / 2^rows_log2, and so on.  Bound by its round
// trips (the split; the row's maxima, sums and first four partials together), so
// all rows are under way at once.  Joined by the last CTA of a unit instead,
// without this launch, the one SM needed 10 us for 64 rows of six partials.
template <int kD, bool kF16>
__global__ void __launch_bounds__(256, 2) k_paged_merge(const __grid_constant__ PagedArgs p, int rows_log2)
{
    constexpr int kSlot = slot_floats(kD), kVec = kD / 32, kAhead = 4;  // kVec: float4s of a lane
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, sub = lane & 7;
    const PlanHeader *hd = static_cast<const PlanHeader *>(p.plan);
    int item = (blockIdx.x * 256 + threadIdx.x) >> 3;
    auto split_at = [&](int i) { return plan_splits(p.plan)[min(i >> rows_log2, kMaxPlanCtas - 1)]; };
    PlanSplit s, next = split_at(item);
    // What the CTAs have reported, looked at before the first write: a wait that ran out, or a request
    // whose tree is another here (a load per row for that would be one more on every call's way).
    const int reported = load_now(p.status);
    const auto left_out = [&](const PlanSplit &s) {
        return (reported & kStatusTimeout) || (unsigned)s.tree >= (unsigned)p.n_trees || p.trees[s.tree].n != s.n;
    };
    const int items = hd->n_splits << rows_log2, stride = gridDim.x * 32;
    if (!hd->valid || hd->batch != p.batch || hd->n_q_heads != p.Hq || hd->n_kv_heads != p.Hkv)
        return;
    for (; __any_sync(0xffffffffu, item < items); item += stride) {
        s = next;
        if (item + stride < items)
            next = split_at(item + stride);
        int x = item & ((1 << rows_log2) - 1);
        const int grow = s.rb * 128 + x, node = grow / p.group, qh = s.head * p.group + grow % p.group;
        const bool live = item < items && x < s.rows && s.row0 + node < p.n_rows &&
                          in_bounds(qh < p.Hq && s.c_lo >= 0, p.status);
        if (!__any_sync(0xffffffffu, live))
            continue;
        const int nseg = live ? s.nseg : 0;
        const float *rest = p.part + (live ? (size_t)s.c_lo * 2 * kSlot : 0);  // CTA k > 0: + 2 k slots
        const float *first = rest + (live ? s.lo_slot * kSlot : 0);
        float M = -INFINITY, sum = 0.f;
        float4 acc[kVec] = {};
        for (int k0 = 0; __any_sync(0xffffffffu, k0 < nseg); k0 += 8) {
            // lane k of the group has the (k0 + k)-th CTA's maximum and sum
            const int k = k0 + sub;
            const float *sl = k == 0 ? first : rest + (size_t)(k < nseg ? k : 0) * 2 * kSlot;
            const float ms = k < nseg ? __ldcg(sl + 128 * kD + x) : -INFINITY;
            const float ls = k < nseg ? __ldcg(sl + 128 * kD + 128 + x) : 0.f;
            float w = 0.f;
            for (int z = 0; z < 8; z += kAhead) {
                if (!__any_sync(0xffffffffu, k0 + z < nseg))
                    break;
                float4 v[kAhead][kVec];
#pragma unroll
                for (int y = 0; y < kAhead; ++y) {
                    const int c = k0 + z + y;
                    const float4 *from = reinterpret_cast<const float4 *>((c == 0 ? first : rest + (size_t)c * 2 * kSlot) + x * kD);
#pragma unroll
                    for (int i = 0; i < kVec; ++i)
                        v[y][i] = c < nseg ? __ldcg(from + sub + 8 * i) : make_float4(0.f, 0.f, 0.f, 0.f);
                }
                if (z == 0) {
                    float m2 = ms;
#pragma unroll
                    for (int o = 4; o >= 1; o >>= 1)
                        m2 = fmaxf(m2, __shfl_xor_sync(0xffffffffu, m2, o));
                    m2 = fmaxf(m2, M);
                    const float keep = M == -INFINITY ? 0.f : ex2_approx(M - m2);
                    w = ms == -INFINITY ? 0.f : ex2_approx(ms - m2);
                    float ws = w * ls;
#pragma unroll
                    for (int o = 4; o >= 1; o >>= 1)
                        ws += __shfl_xor_sync(0xffffffffu, ws, o);
                    M = m2;
                    sum = sum * keep + ws;
#pragma unroll
                    for (int i = 0; i < kVec; ++i)
                        acc[i].x *= keep, acc[i].y *= keep, acc[i].z *= keep, acc[i].w *= keep;
                }
#pragma unroll
                for (int y = 0; y < kAhead; ++y) {
                    const float f = __shfl_sync(0xffffffffu, w, z + y, 8);
#pragma unroll
                    for (int i = 0; i < kVec; ++i) {
                        acc[i].x = fmaf(f, v[y][i].x, acc[i].x);
                        acc[i].y = fmaf(f, v[y][i].y, acc[i].y);
                        acc[i].z = fmaf(f, v[y][i].z, acc[i].z);
                        acc[i].w = fmaf(f, v[y][i].w, acc[i].w);
                    }
                }
            }
        }
        if (!live || (reported && left_out(s)))
            continue;
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        const size_t row = (size_t)(s.row0 + node) * p.Hq + qh;
        uint2 *dst = reinterpret_cast<uint2 *>(p.out + row * kD) + sub;
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            dst[8 * i] = make_uint2(pack<kF16>(acc[i].x * inv, acc[i].y * inv), pack<kF16>(acc[i].z * inv, acc[i].w * inv));
        if (p.lse && sub == 0)
            p.lse[row] = sum == 0.f ? -INFINITY : (M + log2f(sum)) * kLn2;
    }
}

template <int kD, bool kF16, int kForm, bool kQ4>
cudaError_t launch(const PagedArgs &a, int n_sm, int max_rows, cudaStream_t stream)
{
    cudaError_t e = allow_max_smem((const void *)k_paged_attention<kD, kF16, kForm, kQ4>);
    if (e != cudaSuccess)
        return e;
    e = launch_kernel(k_paged_attention<kD, kF16, kForm, kQ4>, dim3(n_sm), dim3(kThreads),
                      (size_t)smem_bytes<kD, kQ4>(), stream, true, a);
    if (e != cudaSuccess || n_sm < 2)
        return e;
    int rows_log2 = 0;
    while ((1 << rows_log2) < max_rows)
        ++rows_log2;
    const long long rows = (long long)(n_sm - 1) << rows_log2;  // of every possible split
    const int blocks = (int)((rows + 31) / 32);
    return launch_kernel(k_paged_merge<kD, kF16>, dim3(blocks < 2 * n_sm ? blocks : 2 * n_sm), dim3(256), 0, stream, true,
                         a, rows_log2);
}

template <int kD, bool kF16, bool kQ4>
cudaError_t launch_form(const PagedArgs &a, int n_sm, int max_rows, cudaStream_t stream)
{
    if (a.slopes)
        return launch<kD, kF16, kBias, kQ4>(a, n_sm, max_rows, stream);
    return a.cap > 0.f ? launch<kD, kF16, kCap, kQ4>(a, n_sm, max_rows, stream)
                       : launch<kD, kF16, kPlain, kQ4>(a, n_sm, max_rows, stream);
}

// What both calls do: their checks but for the pages' own, the arguments, the launches.  fill(a): the layer's
// pages, or what is wrong with them.
template <bool kQ4, typename Pages, typename Fill>
tb_status attend(const tb_bank *bank, const tb_requests *req, const Pages *pages, int layer, const void *plan,
                 size_t plan_bytes, const void *q, int n_rows, int n_q_heads, float scale, float softcap,
                 const float *slopes, void *out, float *lse, void *workspace, size_t workspace_bytes, tb_stream stream,
                 const char *fn, tb_status (*check)(const Pages *, const char *), Fill fill)
{
    PagedArgs a{};
    tb_status st = check_device_bank(bank, fn, &a.trees, &a.n_trees);
    if (st != TB_OK || (st = check_requests(req, true, fn)) != TB_OK || (st = check(pages, fn)) != TB_OK)
        return st;
    if (!req->tree)
        return record_error(TB_EINVAL, "%s: req->tree is NULL", fn);
    if (pages->page_size != req->page_size)
        return record_error(TB_EINVAL, "%s: pages of %d slots, a table of %d", fn, pages->page_size, req->page_size);
    a.expire_wait = (layer & TB_DEBUG_EXPIRE_WAIT) ? 1 : 0;
    layer &= ~TB_DEBUG_EXPIRE_WAIT;
    if (layer < 0 || layer >= pages->n_layers)
        return record_error(TB_EINVAL, "%s: layer %d of %d", fn, layer, pages->n_layers);
    if (n_q_heads < pages->n_kv_heads || n_q_heads % pages->n_kv_heads)
        return record_error(TB_EINVAL, "%s: n_q_heads %d not a multiple of n_kv_heads %d", fn, n_q_heads,
                            pages->n_kv_heads);
    if (n_q_heads / pages->n_kv_heads > kMaxGroup)
        return record_error(TB_EUNSUPPORTED, "%s: %d query heads per kv head (%d supported)", fn,
                            n_q_heads / pages->n_kv_heads, kMaxGroup);
    if (!(scale > 0.f) || !std::isfinite(scale) || !(softcap >= 0.f) || !std::isfinite(softcap))
        return record_error(TB_EINVAL, "%s: scale %g, softcap %g", fn, scale, softcap);
    if (softcap > kMaxCap || (softcap > 0.f && !std::isfinite(cap_in(scale, softcap))))
        return record_error(TB_EUNSUPPORTED, "%s: scale %g with softcap %g (%g at most)", fn, scale, softcap, kMaxCap);
    if (n_rows < 0)
        return record_error(TB_EINVAL, "%s: n_rows %d", fn, n_rows);
    if (n_rows > 0 && (!q || !out || !ptr_aligned(q, 16) || !ptr_aligned(out, 16)))
        return record_error(TB_EINVAL, "%s: q / out NULL or not 16-byte aligned", fn);
    if ((st = check_workspace(plan, plan_bytes, plan_bytes_for(req->batch), fn)) != TB_OK)
        return st;
    if ((st = check_workspace(workspace, workspace_bytes,
                              tb_workspace_size(0, 1, pages->n_kv_heads, n_q_heads, pages->head_dim, 0, -1), fn)) !=
        TB_OK)
        return st;
    if (n_rows == 0)
        return launch_result(cudaSuccess, fn);
    const int n_sm = device_sms(-1);
    if (n_sm <= 0 || n_sm > kMaxPlanCtas)
        return record_error(TB_ECUDA, "%s: no current device, or one of %d SMs", fn, n_sm);
    a.table = req->table;
    a.max_pages = req->max_pages;
    while ((1 << a.page_log2) < req->page_size)
        ++a.page_log2;
    a.n_pages = pages->n_pages;
    a.batch = req->batch;
    a.q = static_cast<const uint16_t *>(q);
    a.out = static_cast<uint16_t *>(out);
    a.lse = lse;
    a.slopes = slopes;
    a.n_rows = n_rows;
    a.Hq = n_q_heads;
    a.Hkv = pages->n_kv_heads;
    a.group = n_q_heads / pages->n_kv_heads;
    a.scale = scale * kLog2e;
    a.cap = softcap * kLog2e;
    a.cap_in = softcap > 0.f ? cap_in(scale, softcap) : 0.f;
    a.plan = const_cast<void *>(plan);
    a.part = attention_parts(workspace);
    a.status = static_cast<int *>(workspace);
    if (kQ4 && pages->dtype == TB_BF16) {
        a.scale *= 1.f / kOperandScale<false>;
        a.cap_in *= 1.f / kOperandScale<false>;
        if (!std::isfinite(a.scale) || !std::isfinite(a.cap_in))
            return record_error(TB_EUNSUPPORTED, "%s: scale %g with softcap %g", fn, scale, softcap);
    }
    if (const char *err = fill(a, layer))
        return record_error(kQ4 ? TB_EUNSUPPORTED : TB_EINVAL, "%s: %s", fn, err);
    const long long most = (long long)(n_rows < kMaxNodes ? n_rows : kMaxNodes) * a.group;
    const int max_rows = most < 128 ? (int)most : 128;
    const bool f16 = pages->dtype == TB_F16;
    const cudaStream_t s = (cudaStream_t)stream;
    const cudaError_t e = pages->head_dim == 64 ? (f16 ? launch_form<64, true, kQ4>(a, n_sm, max_rows, s)
                                                       : launch_form<64, false, kQ4>(a, n_sm, max_rows, s))
                                                : (f16 ? launch_form<128, true, kQ4>(a, n_sm, max_rows, s)
                                                       : launch_form<128, false, kQ4>(a, n_sm, max_rows, s));
    return launch_result(e, fn);
}

}  // namespace

}  // namespace tv
