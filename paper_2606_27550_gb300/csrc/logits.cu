// logits.cu -- penalties for repeated tokens, biases and grammar masks on the
// logits of every row, and the statistics that the acceptance rules read, in one
// pass over the logits.
//
// A CTA takes one request, a slice of the vocabulary and up to 8 of the request's
// rows, and builds the slice's rules once in shared memory for all of them: how
// often each token was generated, whether the prompt has it, its bias, and a
// bitmap of the tokens that any rule touches.  A warp takes a row's slice (or a
// part of it where there are few rows) in chunks of 512 tokens through a ring of its
// own in shared memory, the next chunk on its way.  A chunk's touched tokens (a few
// percent of a vocabulary, but some lane of nearly every warp has one) take the rules one
// per lane, in shared memory, and so do the draft tokens on the row's root path that
// lie in it; then every lane takes its sixteen logits.  (With the rules on all of a
// chunk's logits wherever more than 32 were touched, eight trees at 128256 tokens took
// 81 us.)
//
// Bound by HBM while the logits stream (at that pace three CTAs of an SM together would
// take 9 TB/s), but half of a CTA's life goes into its rules, where it waits for memory
// in turn: parameters, history and tree, the rows' first chunks.  Eight trees (358 rows)
// at 128256 tokens 77 us, 4.9 TB/s; 68 without rules; 256 requests of one row 154 us.
// 16-bit logits take as long (76 us, a quarter fewer bytes): instructions bound them.
//
// With x = z - m, m the warp's running maximum, each lane keeps s = sum e^x, u = sum
// x e^x and the two sums at temperature T, rescaled when a chunk has a new maximum;
// parts join in shared memory, slices by the last CTA of the rows (an arrival ticket) or
// by k_logits_join, always in index order: outputs do not depend on the placement.
//   top1 = 1 / s,  H = ln s - u / s,  ln Z_T = m / T + ln s_T
// Penalties and biases are 32-bit operations in the documented order, each rounded
// to nearest (nothing is contracted).
#include "paged.cuh"

#include <cuda_fp16.h>

#include <cmath>

namespace tv {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kVec = 4, kChunk = 128 * kVec;  // tokens a warp takes at a time: kVec groups of four per lane
constexpr int kRows = kWarps;   // rows of a CTA
constexpr int kPerSm = 3;        // CTAs of an SM
constexpr int kMaxSlice = 3584;  // kPerSm of them fit its shared memory
constexpr int kMaxRowsCall = 65536;
constexpr int kStages = 2;      // chunks of a warp's ring: one in work, the others on their way
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// How far below a row's maximum a part's maximum counts as: its weight is 0 long before, but a
// difference that overflows (a part of nothing but the type's lowest value, which stands for "masked"
// in many models' logits, or a temperature near 0) would make 0 x inf of it.
constexpr float kFar = -1e30f;

// logits that a chunk's stage of the ring holds: 16-bit ones may begin and end in the middle of a word
__host__ __device__ constexpr int stage_elems(int bytes)
{
    return bytes == 4 ? kChunk : kChunk + 8;
}

struct Part {
    float m;
    int arg;
    float s, u, st, ut;
    int pad[2];
};

struct LogitArgs {
    const TreeDesc *trees;
    int n_trees, batch, n_rows, V, slices, size;  // size: tokens per slice
    int ring_off, mask_off, copy_off;             // in the dynamic shared memory
    const int32_t *tree, *row_start;
    const void *in;
    long long in_stride, out_stride;
    float *out;
    tb_logit_rules r;
    tb_logit_stats st;
    float temperature, inv_t;
    bool join;  // by the last CTA of a piece's rows, else by k_logits_join
    int mask_rows, n_bias;       // that mask_row may name; entries of all biases
    int *status;
    int *ticket;                 // [pieces of rows]
    Part *parts;                 // [rows][slices]
};

__device__ __forceinline__ Part empty_part()
{
    return Part{-INFINITY, 0x7fffffff, 0.f, 0.f, 0.f, 0.f, {0, 0}};
}

// a and b over disjoint tokens; equal maxima: the lower token
__device__ __forceinline__ Part combine(const Part &a, const Part &b, float inv_t)
{
    Part o;
    const bool take_b = b.m > a.m || (b.m == a.m && b.arg < a.arg);
    o.m = take_b ? b.m : a.m;
    o.arg = take_b ? b.arg : a.arg;
    // the sums of an empty part are 0 (or NaN), whatever its weight
    const float da = a.m == -INFINITY ? 0.f : fmaxf(a.m - o.m, kFar);
    const float db = b.m == -INFINITY ? 0.f : fmaxf(b.m - o.m, kFar);
    const float wa = ex2_approx(da * kLog2e), wb = ex2_approx(db * kLog2e);
    o.s = wa * a.s + wb * b.s;
    o.u = wa * (a.u + da * a.s) + wb * (b.u + db * b.s);
    const float ta = fmaxf(da * inv_t, kFar), tb = fmaxf(db * inv_t, kFar);
    const float va = ex2_approx(ta * kLog2e), vb = ex2_approx(tb * kLog2e);
    o.st = va * a.st + vb * b.st;
    o.ut = va * (a.ut + ta * a.st) + vb * (b.ut + tb * b.st);
    return o;
}

template <int kType>
struct In;
template <>
struct In<TB_F32> {
    using T = float;
    static __device__ __forceinline__ float one(const T *p) { return *p; }
    static __device__ __forceinline__ float4 four(const T *p) { return *reinterpret_cast<const float4 *>(p); }
};
template <>
struct In<TB_BF16> {
    using T = __nv_bfloat16;
    static __device__ __forceinline__ float one(const T *p) { return __bfloat162float(*p); }
    static __device__ __forceinline__ float4 four(const T *p)
    {
        const uint2 w = *reinterpret_cast<const uint2 *>(p);
        return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u),
                           __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u));
    }
};
template <>
struct In<TB_F16> {
    using T = __half;
    static __device__ __forceinline__ float one(const T *p) { return __half2float(*p); }
    static __device__ __forceinline__ float4 four(const T *p)
    {
        const uint2 w = *reinterpret_cast<const uint2 *>(p);
        const float2 a = __half22float2(*reinterpret_cast<const __half2 *>(&w.x));
        const float2 b = __half22float2(*reinterpret_cast<const __half2 *>(&w.y));
        return make_float4(a.x, a.y, b.x, b.y);
    }
};

// The penalties of a request.
struct Penalty {
    float rep, freq, pres;
};

template <int kBytes>
__device__ __forceinline__ void copy_async(void *dst, const void *src)
{
    if constexpr (kBytes == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(smem_u32(dst)), "l"(src), "n"(kBytes) : "memory");
}

// The rules on one logit.  n: generated occurrences; seen: they or the prompt have
// the token.
__device__ __forceinline__ float penalise(float z, float n, bool seen, float bias, const Penalty &p)
{
    const float b = seen ? p.rep : 1.f;
    z = z > 0.f ? __fdiv_rn(z, b) : __fmul_rn(z, b);
    z = __fsub_rn(z, __fmul_rn(p.freq, n));
    z = __fsub_rn(z, n > 0.f ? p.pres : 0.f);
    return __fadd_rn(z, bias);
}

// Notes an occurrence of the slice's token `loc`, if it is below `here`: the history has
// it, and if it was generated, once more.  Predicated: one lane in 36 has a token of the
// slice, some lane of most warps, and as a branch per token this took longer than the
// tokens' way from memory.
__device__ __forceinline__ void note_token(uint32_t *count, uint32_t *seen, unsigned loc, unsigned here, bool generated)
{
    asm volatile("{\n\t"
                 ".reg .pred p, q;\n\t"
                 "setp.ne.s32 q, %4, 0;\n\t"
                 "setp.lt.u32 p, %2, %3;\n\t"
                 "setp.lt.and.u32 q, %2, %3, q;\n\t"
                 "@p red.shared.or.b32 [%1], %5;\n\t"
                 "@q red.shared.add.u32 [%0], 1;\n\t"
                 "}" ::"r"(smem_u32(count) + 4 * loc), "r"(smem_u32(seen) + 4 * (loc >> 5)), "r"(loc), "r"(here),
                 "r"((int)generated), "r"(1u << (loc & 31))
                 : "memory");
}

// The largest of the warp's values (NaN only where all are).
__device__ __forceinline__ float warp_max(float x)
{
    float y;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
    return y;
}

// The last request whose rows begin at or before row g, by the whole warp (one round
// trip to memory for every 32-fold).
__device__ __forceinline__ int owner_of(const int32_t *row_start, int batch, int g, int lane)
{
    int lo = 0, n = batch;  // among requests lo .. lo + n - 1; row_start[lo] <= g
    while (n > 1) {
        const int step = (n + 31) / 32, at = lo + lane * step;
        const bool before = lane * step < n && (lane == 0 || row_start[at] <= g);
        const int k = __popc(__ballot_sync(0xffffffffu, before)) - 1;
        lo += k * step;
        n = min(step, n - k * step);
    }
    return lo;
}

// A row's statistics so far: the warp's maximum and where it is, and this lane's sums over
// the tokens of even and odd index, x in units of ln 2.
struct Running {
    float m;
    int arg;
    uint64_t s, u, st, ut;
};

// The lane's parts k and k + 32 of a row, on their way.
struct TwoParts {
    Part x[2];
};
__device__ __forceinline__ TwoParts load_parts(const LogitArgs &p, int row, int k)
{
    TwoParts t{{empty_part(), empty_part()}};
#pragma unroll
    for (int y = 0; y < 2; ++y)
        if (k + 32 * y < p.slices) {
            const Part *from = p.parts + (size_t)row * p.slices + k + 32 * y;
            float4 *to = reinterpret_cast<float4 *>(&t.x[y]);
#pragma unroll
            for (int h = 0; h < 2; ++h)
                asm volatile("ld.global.cg.v4.f32 {%0, %1, %2, %3}, [%4];"
                             : "=f"(to[h].x), "=f"(to[h].y), "=f"(to[h].z), "=f"(to[h].w)
                             : "l"(reinterpret_cast<const float4 *>(from) + h)
                             : "memory");
        }
    return t;
}

// One warp joins the slices of a row and writes its statistics, and the draft tokens'
// logits of its children.  The request's rows are row0 .. row1 - 1; first: the lane's
// parts from `lane` on.
template <int kStats>
__device__ __forceinline__ void join_row(const LogitArgs &p, int row, int row0, int row1, const TreeDesc *td, int lane,
                                         const TwoParts &first)
{
    const float inv_t = p.inv_t;
    // the draft tokens of the row's children
    float draft_logit[2];
    bool child[2] = {};
    if (p.st.draft_logit && td) {
        const int nodes = min(load_now(&td->n), row1 - row0);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int j = lane + 32 * h, v = row0 + j < row1 ? load_now(p.r.draft + row0 + j) : -1;
            const int8_t parent = td->parent[j];
            child[h] = j > 0 && j < nodes && row - row0 < nodes && parent == row - row0 && v >= 0 && v < p.V;
            draft_logit[h] = child[h] ? __ldcg(p.out + row * p.out_stride + v) : 0.f;
        }
    }
    Part a = combine(first.x[0], first.x[1], inv_t);
    for (int k = 64 + lane; k - lane < p.slices; k += 64) {
        const TwoParts t = load_parts(p, row, k);
        a = combine(combine(a, t.x[0], inv_t), t.x[1], inv_t);
    }
    // the lanes' parts relative to the row's maximum, then plain sums
    const float m = warp_max(a.m);
    const unsigned arg = __reduce_min_sync(0xffffffffu, a.m == m ? (unsigned)a.arg : 0x7fffffffu);
    Part top = empty_part();
    top.m = m;
    a = combine(a, top, inv_t);
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) {
        a.s += __shfl_xor_sync(0xffffffffu, a.s, o);
        a.u += __shfl_xor_sync(0xffffffffu, a.u, o);
        a.st += __shfl_xor_sync(0xffffffffu, a.st, o);
        a.ut += __shfl_xor_sync(0xffffffffu, a.ut, o);
    }
    if (lane == 0) {
        // a row without an allowed token: sums 0 (NaN where its allowed logits are)
        const bool none = !(m > -INFINITY);
        const bool empty = none && a.s == 0.f;
        if (p.st.argmax)
            p.st.argmax[row] = none ? -1 : (int)arg;
        if (p.st.top1)
            p.st.top1[row] = empty ? 0.f : 1.f / a.s;
        if (p.st.entropy)
            p.st.entropy[row] = empty ? 0.f : logf(a.s) - a.u / a.s;
        const float sT = kStats > 1 ? a.st : a.s, uT = kStats > 1 ? a.ut : a.u;
        if (p.st.logz_t)
            p.st.logz_t[row] = empty ? -INFINITY : __fdiv_rn(m, p.temperature) + logf(sT);
        if (p.st.entropy_t)
            p.st.entropy_t[row] = empty ? 0.f : logf(sT) - uT / sT;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
        if (child[h])
            p.st.draft_logit[row0 + lane + 32 * h] = draft_logit[h];
}

// kStats: 0 none, 1 at temperature 1 only, 2 also at T
template <int kType, int kStats>
__global__ void __launch_bounds__(kThreads, kPerSm) k_logits(const __grid_constant__ LogitArgs p)
{
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ Part s_part[kRows][kWarps];
    __shared__ uint64_t s_anc[TB_MAX_NODES];
    __shared__ int s_draft[TB_MAX_NODES];
    __shared__ int s_last;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int slice = blockIdx.y, size = p.size, v0 = slice * size;  // v0 < V (the host's split)
    uint32_t *count = reinterpret_cast<uint32_t *>(smem);  // generated occurrences; then as floats
    float *bias = reinterpret_cast<float *>(count + size);
    uint32_t *touched = reinterpret_cast<uint32_t *>(bias + size);  // bitmap: a rule has the token
    uint32_t *seen = touched + size / 32;                           // bitmap: the history has it
    uint16_t *before = reinterpret_cast<uint16_t *>(seen + size / 32);  // touched tokens before a word's
    uint16_t *list = before + size / 32 + 8;                            // the touched tokens, in order
    using T = typename In<kType>::T;
    constexpr int kStage = stage_elems(sizeof(T));
    T *ring = reinterpret_cast<T *>(smem + p.ring_off) + warp * kStage;  // a stage of all warps behind another
    // the second stage holds tokens of the history until the rules are built
    int *early = reinterpret_cast<int *>(smem + p.ring_off + kWarps * kStage * sizeof(T));
    constexpr int kEarly = kWarps * kStage * sizeof(T) / 4;
    static_assert(kStages >= 2, "tokens of the history in the second stage");
    uint32_t *mask_ring = reinterpret_cast<uint32_t *>(smem + p.mask_off) + warp * kStages * (kChunk / 32);
    float *copy = reinterpret_cast<float *>(smem + p.copy_off) + warp * kChunk;  // (16-bit logits only)
    const bool rules = p.r.history || p.r.bias_start;
    if (rules) {
        for (int x = threadIdx.x; x < size / 4; x += kThreads) {
            reinterpret_cast<uint4 *>(count)[x] = make_uint4(0, 0, 0, 0);
            reinterpret_cast<uint4 *>(bias)[x] = make_uint4(0, 0, 0, 0);
        }
        for (int x = threadIdx.x; x < size / 32; x += kThreads)
            touched[x] = seen[x] = 0;
    }
    pdl_wait();
    pdl_trigger();
    // Rows are grouped in blocks of 8 of the whole batch, cut at the requests' ends.
    // CTA x < batch takes the first piece of request x, CTA batch + e the block e if
    // it begins inside a request.
    int b = blockIdx.x, g0 = 0, g1;
    const bool head = b < p.batch;
    if (!head) {
        g0 = (b - p.batch) * kRows;
        b = owner_of(p.row_start, p.batch, g0, lane);
    }
    // the request's parameters, one round trip
    const int row0 = load_now(p.row_start + b), row_end = load_now(p.row_start + b + 1);
    const int t = p.tree ? load_now(p.tree + b) : -1;
    const int said = p.r.history ? load_now(p.r.history_len + b) : 0;
    const int asked = p.r.history && p.r.prompt_len ? load_now(p.r.prompt_len + b) : 0;
    const int bias0 = p.r.bias_start ? load_now(p.r.bias_start + b) : 0;
    const int bias_said = p.r.bias_start ? load_now(p.r.bias_start + b + 1) : 0;
    Penalty pen;
    pen.rep = p.r.repetition ? load_now(p.r.repetition + b) : 1.f;
    pen.freq = p.r.frequency ? load_now(p.r.frequency + b) : 0.f;
    pen.pres = p.r.presence ? load_now(p.r.presence + b) : 0.f;
    const int row1 = min(row_end, p.n_rows);
    if (head)
        g0 = row0;
    if (row0 < 0 || g0 >= row1 || (!head && g0 <= row0))
        return;
    g1 = min((g0 / kRows + 1) * kRows, row1);
    const int here = min(size, p.V - v0);  // tokens of the slice that exist
    // parts of a row: every warp has work where there are chunks enough
    static_assert(kWarps == 8 && kRows == 8, "warps per row as powers of two");
    const int rows = g1 - g0, parts_log2 = rows == 1 ? 3 : rows == 2 ? 2 : rows <= 4 ? 1 : 0, parts = 1 << parts_log2;
    const int part_size = (((here + kChunk - 1) / kChunk + parts - 1) >> parts_log2) * kChunk;
    // the item (row, part) in work
    const T *src = nullptr;
    const int32_t *mask = nullptr;
    bool unknown = false;  // the row names a mask that there is not: no token is allowed
    int row = 0, c_first = 0, c_end = 0;
    float *dst = nullptr;
    bool vec = false;  // four logits at a time, in and out
    int odd = 0;       // 16-bit logits from between two 32-bit words on
    auto fetch = [&](int c) {  // chunk c on its way; always one group of copies
        if (c < c_end) {
            const int st = ((c - c_first) / kChunk) % kStages;
            T *to = ring + st * (kWarps * kStage);
            if (vec && c + kChunk <= here) {
#pragma unroll
                for (int k = 0; k < kVec; ++k)
                    copy_async<4 * sizeof(T)>(to + k * 128 + lane * 4, src + c + k * 128 + lane * 4);
            } else if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int k = 0; k < 4 * kVec; ++k)
                    if (c + 32 * k + lane < here)
                        copy_async<4>(to + 32 * k + lane, src + c + 32 * k + lane);
            } else {
                // pairs of 16-bit logits, from the element before where the row begins between two
                // (the tensor begins on 16 bytes); those that would end past the slice stay out
#pragma unroll
                for (int k = 0; k <= 2 * kVec; ++k) {
                    const int o = 64 * k + 2 * lane - odd;
                    if ((k < 2 * kVec || (lane == 0 && odd)) && c + o + 1 < here)
                        copy_async<4>(to + o + odd, src + c + o);
                }
            }
            if (mask && lane < kChunk / 32 && c + 32 * lane < here)
                copy_async<4>(mask_ring + st * (kChunk / 32) + lane, mask + (c >> 5) + lane);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    // The first tokens of the history (some in registers, others by way of shared
    // memory) and the first biases, then the logits and the tree: one round trip.
    constexpr int kAhead = 16, kInRegs = kAhead * kThreads, kBiasAhead = 2;
    const int n_said = (int)min((long long)max(said, 0), (long long)p.r.history_stride);
    const int n_asked = min(max(asked, 0), n_said);
    const int32_t *h = p.r.history + (p.r.history ? b * p.r.history_stride : 0);
    const int bias_end = min(bias_said, p.n_bias);
    int word_of[kAhead], bias_tok[kBiasAhead];
    float bias_val[kBiasAhead];
#pragma unroll
    for (int m = 0; m < kAhead; ++m) {
        const int i = threadIdx.x + m * kThreads;
        word_of[m] = i < n_said ? load_now(h + i) : -1;
    }
    const auto load_biases = [&](int e) {
#pragma unroll
        for (int m = 0; m < kBiasAhead; ++m) {
            bias_tok[m] = e + m * kThreads < bias_end ? load_now(p.r.bias_token + e + m * kThreads) : -1;
            bias_val[m] = e + m * kThreads < bias_end ? load_now(p.r.bias_value + e + m * kThreads) : 0.f;
        }
    };
    load_biases(max(bias0, 0) + threadIdx.x);
    for (int i = threadIdx.x; i < min(n_said - kInRegs, kEarly); i += kThreads)
        copy_async<4>(early + i, h + kInRegs + i);
    asm volatile("cp.async.commit_group;" ::: "memory");
    const int gr = warp >> parts_log2, part = warp & (parts - 1);  // this warp's row and part of it
    if (gr < rows) {
        row = g0 + gr;
        c_first = part * part_size;
        c_end = min(c_first + part_size, here);
        src = static_cast<const T *>(p.in) + row * p.in_stride + v0;
        dst = p.out + row * p.out_stride + v0;
        odd = sizeof(T) == 2 ? (int)(reinterpret_cast<uintptr_t>(src) >> 1) & 1 : 0;
        vec = (reinterpret_cast<uintptr_t>(src) & (4 * sizeof(T) - 1)) == 0 && (reinterpret_cast<uintptr_t>(dst) & 15) == 0;
        const int mrow = !p.r.mask ? -1 : p.r.mask_row ? p.r.mask_row[row] : row;
        unknown = mrow >= p.mask_rows;
        mask = mrow >= 0 ? p.r.mask + (unknown ? 0 : mrow) * p.r.mask_stride + (v0 >> 5) : nullptr;
        // on their way while the rules are built
#pragma unroll
        for (int k = 0; k < kStages - 1; ++k)
            fetch(c_first + k * kChunk);
    } else {
#pragma unroll
        for (int k = 0; k < kStages - 1; ++k)
            asm volatile("cp.async.commit_group;" ::: "memory");
    }

    const TreeDesc *td = t >= 0 && t < p.n_trees ? p.trees + t : nullptr;
    const bool paths = td && p.r.draft;
    uint64_t node_anc = 0;
    int node_tok = -1;
    if (paths && threadIdx.x < TB_MAX_NODES) {
        const int n = load_now(&td->n), here_rows = row1 - row0;
        const uint64_t anc = load_now(td->anc + threadIdx.x);
        const int token = (int)threadIdx.x < here_rows ? load_now(p.r.draft + row0 + threadIdx.x) : -1;
        if ((int)threadIdx.x < min(n, here_rows)) {
            node_anc = anc & ~1ull;
            node_tok = token;
        }
    }
    __shared__ int s_sum[kWarps], s_again;
    if (threadIdx.x < TB_MAX_NODES) {
        s_anc[threadIdx.x] = node_anc;
        s_draft[threadIdx.x] = node_tok;
    }
    if (threadIdx.x == 0)
        s_again = 0;
    asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");  // all but the logits
    __syncthreads();
#pragma unroll
    for (int m = 0; m < kAhead; ++m) {
        if (m * kThreads >= n_said)
            break;
        note_token(count, seen, (unsigned)(word_of[m] - v0), (unsigned)here, (int)threadIdx.x + m * kThreads >= n_asked);
    }
#pragma unroll 4
    for (int i = threadIdx.x; i < min(n_said - kInRegs, kEarly); i += kThreads)
        note_token(count, seen, (unsigned)(early[i] - v0), (unsigned)here, kInRegs + i >= n_asked);
    for (int i0 = kInRegs + kEarly + threadIdx.x; i0 < n_said; i0 += kInRegs) {
#pragma unroll
        for (int m = 0; m < kAhead; ++m)
            word_of[m] = i0 + m * kThreads < n_said ? load_now(h + i0 + m * kThreads) : -1;
#pragma unroll
        for (int m = 0; m < kAhead; ++m)
            note_token(count, seen, (unsigned)(word_of[m] - v0), (unsigned)here, i0 + m * kThreads >= n_asked);
    }
    if (bias_said > p.n_bias && threadIdx.x == 0)
        atomicOr(p.status, kStatusBounds);
    // Biases, in any order as long as no token comes up twice; where one does, all again
    // by one warp in list order, so that its entries add up in a fixed order.
    for (int e = max(bias0, 0) + threadIdx.x; e < bias_end;) {
#pragma unroll
        for (int m = 0; m < kBiasAhead; ++m) {
            const unsigned loc = (unsigned)(bias_tok[m] - v0);
            if (loc < (unsigned)here) {
                if ((atomicOr(&touched[loc >> 5], 1u << (loc & 31)) >> (loc & 31)) & 1)
                    s_again = 1;
                else
                    bias[loc] = bias_val[m];
            }
        }
        e += kThreads * kBiasAhead;
        load_biases(e);
    }
    __syncthreads();
    if (s_again) {
        for (int x = threadIdx.x; x < size; x += kThreads)
            bias[x] = 0.f;
        __syncthreads();
        for (int e0 = max(bias0, 0); warp == 0 && e0 < bias_end; e0 += 32) {
            const int e = e0 + lane;
            const unsigned loc = e < bias_end ? (unsigned)(load_now(p.r.bias_token + e) - v0) : 0xffffffffu;
            const float value = e < bias_end ? load_now(p.r.bias_value + e) : 0.f;
            const bool mine = loc < (unsigned)here;
            const unsigned same = __match_any_sync(0xffffffffu, mine ? (int)loc : -1 - lane);
            const bool leader = mine && (same & ((1u << lane) - 1)) == 0;
            float acc = leader ? bias[loc] : 0.f;
            for (int k = 0; k < 32; ++k) {
                const float v = __shfl_sync(0xffffffffu, value, k);
                acc += (same >> k) & 1 ? v : 0.f;
            }
            if (leader)
                bias[loc] = acc;
            __syncwarp();
        }
    }

    if (rules) {
        // the touched tokens as a list, their counts as floats
        const int words = size / 32;
        static_assert(kMaxSlice / 32 <= kThreads, "a word of the bitmap per thread");
        const uint32_t mine = threadIdx.x < words ? touched[threadIdx.x] | seen[threadIdx.x] : 0u;
        int at = __popc(mine);
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, at, o);
            at += lane >= o ? y : 0;
        }
        if (lane == 31)
            s_sum[warp] = at;
        __syncthreads();
        for (int k = 0; k < warp; ++k)
            at += s_sum[k];
        if (threadIdx.x < words) {
            if (threadIdx.x == words - 1)
                before[words] = (uint16_t)at;
            at -= __popc(mine);
            before[threadIdx.x] = (uint16_t)at;
            for (uint32_t rest = mine; rest; rest &= rest - 1) {
                const int x = threadIdx.x * 32 + __ffs(rest) - 1;
                list[at++] = (uint16_t)x;
                reinterpret_cast<float *>(count)[x] = (float)count[x];
            }
        }
        __syncthreads();
    }
    const float *generated = reinterpret_cast<const float *>(count);

    const float inv_t = p.inv_t;
    if (gr < rows) {
        // the draft tokens on this row's root path, relative to the slice
        int tok[2] = {-1, -1};
        if (paths && row - row0 < TB_MAX_NODES) {
            const uint64_t anc = s_anc[row - row0];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int j = lane + 32 * h, x = s_draft[j] - v0;
                if (((anc >> j) & 1) && s_draft[j] >= 0 && x >= 0 && x < here)
                    tok[h] = x;
            }
        }
        Running a{-INFINITY, 0x7fffffff, 0, 0, 0, 0};
        auto add = [&](float v0, float v1, float mu) {
            const uint64_t y = mul_two(add_two(two(v0, v1), two(-mu, -mu)), two(kLog2e, kLog2e));
            const float2 x = halves(y);
            const uint64_t yc = two(fmaxf(x.x, -3e38f), fmaxf(x.y, -3e38f));  // finite where the weight is 0
            const uint64_t q = two(ex2_approx(x.x), ex2_approx(x.y));
            a.s = add_two(a.s, q);
            a.u = fma_two(q, yc, a.u);
            if constexpr (kStats > 1) {
                const float2 t = halves(mul_two(y, two(inv_t, inv_t)));
                const uint64_t qt = two(ex2_approx(t.x), ex2_approx(t.y));
                a.st = add_two(a.st, qt);
                a.ut = fma_two(qt, yc, a.ut);
            }
        };
#pragma unroll 1
        for (int c = c_first; c < c_end; c += kChunk) {
            float z[kVec][4];
            uint32_t word = 0xffffffffu;  // lane w holds word w of the chunk's mask
            __syncwarp();  // a chunk of another order (a slice's end) takes the place of what other lanes read
            fetch(c + (kStages - 1) * kChunk);
            asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
            const int st = ((c - c_first) / kChunk) % kStages;
            T *from = ring + st * (kWarps * kStage);  // 32-bit logits: every lane reads what it copied
            int l0 = 0, nl = 0;  // the chunk's touched tokens in the list
            if (rules) {
                l0 = before[c >> 5];
                nl = before[(c + kChunk) >> 5] - l0;
            }
            const int o0 = tok[0] - c, o1 = tok[1] - c;
            const bool in0 = (unsigned)o0 < (unsigned)kChunk, in1 = (unsigned)o1 < (unsigned)kChunk;
            const bool on_path = paths && __any_sync(0xffffffffu, in0 || in1);
            const bool touched_here = nl > 0 || on_path;
            // the rules on the chunk's touched tokens, one per lane, in a 32-bit copy of it
            const auto touch = [&](float *copy) {
                __syncwarp();  // the other lanes' copies have landed
                // tokens of the root path: up to two per lane, each once, with how often it comes up
                int at[2] = {-1, -1}, more[2] = {0, 0}, n = 0;
                float value[2];
                if (on_path) {
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        for (unsigned with = __ballot_sync(0xffffffffu, h ? in1 : in0); with; with &= with - 1) {
                            const int o = __shfl_sync(0xffffffffu, h ? o1 : o0, __ffs(with) - 1);
                            const bool known = __any_sync(0xffffffffu, at[0] == o || at[1] == o);
#pragma unroll
                            for (int y = 0; y < 2; ++y) {
                                if (!known && lane + 32 * y == n)
                                    at[y] = o;
                                more[y] += at[y] == o;
                            }
                            n += !known;
                        }
#pragma unroll
                    for (int y = 0; y < 2; ++y)
                        if (at[y] >= 0) {
                            const int x = c + at[y];
                            value[y] = penalise(copy[at[y]], (rules ? generated[x] : 0.f) + (float)more[y], true,
                                                rules ? bias[x] : 0.f, pen);
                        }
                    __syncwarp();
                }
                for (int i = lane; i < nl; i += 32) {
                    const int x = list[l0 + i];
                    copy[x - c] = penalise(copy[x - c], generated[x], (seen[x >> 5] >> (x & 31)) & 1, bias[x], pen);
                }
                __syncwarp();
                if (on_path) {
#pragma unroll
                    for (int y = 0; y < 2; ++y)
                        if (at[y] >= 0)
                            copy[at[y]] = value[y];
                    __syncwarp();
                }
            };
            if constexpr (sizeof(T) == 4) {
                if (touched_here)
                    touch(from);
            }
            // a lane's logits: four in a row of each 128, or where that is not aligned (and at a slice's
            // end) one of each 32: eight trees at 128255 tokens 88 us, 98 with four in a row one by one;
            // bf16 107 us, 150 without the ring
            const bool four = vec && c + kChunk <= here;
            const int mine = four ? 4 * lane : lane, next = four ? 1 : 32;
            if (four) {
#pragma unroll
                for (int k = 0; k < kVec; ++k) {
                    const float4 x = In<kType>::four(from + k * 128 + mine);
                    z[k][0] = x.x, z[k][1] = x.y, z[k][2] = x.z, z[k][3] = x.w;
                }
            } else {
                if constexpr (sizeof(T) != 4)
                    __syncwarp();  // other lanes' copies
#pragma unroll
                for (int k = 0; k < kVec; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int o = k * 128 + e * 32 + lane;
                        const bool landed = sizeof(T) == 4 || c + ((o + odd) | 1) - odd < here;
                        z[k][e] = c + o < here ? In<kType>::one(landed ? from + o + odd : src + c + o) : -INFINITY;
                    }
                if constexpr (sizeof(T) != 4)
                    __syncwarp();
            }
            if (mask && lane < kChunk / 32 && c + 32 * lane < here)
                word = unknown ? 0u : mask_ring[st * (kChunk / 32) + lane];
            if constexpr (sizeof(T) != 4) {
                if (touched_here) {
                    if (four) {
#pragma unroll
                        for (int k = 0; k < kVec; ++k)
                            *reinterpret_cast<float4 *>(copy + k * 128 + mine) =
                                make_float4(z[k][0], z[k][1], z[k][2], z[k][3]);
                    } else {
#pragma unroll
                        for (int k = 0; k < kVec; ++k)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                copy[k * 128 + e * 32 + lane] = z[k][e];
                    }
                    touch(copy);
                    if (four) {
#pragma unroll
                        for (int k = 0; k < kVec; ++k) {
                            const float4 x = *reinterpret_cast<const float4 *>(copy + k * 128 + mine);
                            z[k][0] = x.x, z[k][1] = x.y, z[k][2] = x.z, z[k][3] = x.w;
                        }
                    } else {
#pragma unroll
                        for (int k = 0; k < kVec; ++k)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                z[k][e] = copy[k * 128 + e * 32 + lane];
                    }
                }
            }
            if (mask && four) {
#pragma unroll
                for (int k = 0; k < kVec; ++k) {
                    const uint32_t w = __shfl_sync(0xffffffffu, word, 4 * k + (lane >> 3)) >> (4 * (lane & 7));
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        z[k][e] = (w >> e) & 1 ? z[k][e] : -INFINITY;
                }
            } else if (mask) {
#pragma unroll
                for (int k = 0; k < kVec; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        z[k][e] = (__shfl_sync(0xffffffffu, word, 4 * k + e) >> lane) & 1 ? z[k][e] : -INFINITY;
            }
            if (four) {
#pragma unroll
                for (int k = 0; k < kVec; ++k)
                    *reinterpret_cast<float4 *>(dst + c + k * 128 + mine) = make_float4(z[k][0], z[k][1], z[k][2], z[k][3]);
            } else {
#pragma unroll
                for (int k = 0; k < kVec; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int o = c + k * 128 + e * 32 + lane;
                        if (o < here)
                            dst[o] = z[k][e];
                    }
            }
            if constexpr (kStats > 0) {
                float m = -INFINITY;
#pragma unroll
                for (int k = 0; k < kVec; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        m = fmaxf(m, z[k][e]);
                m = warp_max(m);
                if (m > a.m) {
                    // a new maximum: its lowest token, and the sums relative to it
                    unsigned arg = 0x7fffffffu;
#pragma unroll
                    for (int k = 0; k < kVec; ++k)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (z[k][e] == m)
                                arg = min(arg, (unsigned)(v0 + c + k * 128 + mine + e * next));
                    a.arg = (int)__reduce_min_sync(0xffffffffu, arg);
                    const float d = a.m == -INFINITY ? 0.f : a.m - m;  // (sums of nothing: 0)
                    const float dy = fmaxf(d * kLog2e, kFar), w = ex2_approx(dy);
                    a.u = mul_two(two(w, w), fma_two(two(dy, dy), a.s, a.u));
                    a.s = mul_two(two(w, w), a.s);
                    if constexpr (kStats > 1) {
                        const float wt = ex2_approx(dy * inv_t);
                        a.ut = mul_two(two(wt, wt), fma_two(two(dy, dy), a.st, a.ut));
                        a.st = mul_two(two(wt, wt), a.st);
                    }
                    a.m = m;
                }
                const float mu = a.m == -INFINITY ? 0.f : a.m;
#pragma unroll
                for (int k = 0; k < kVec; ++k)
#pragma unroll
                    for (int e = 0; e < 4; e += 2)
                        add(z[k][e], z[k][e + 1], mu);
            }
        }
        if (unknown && lane == 0)
            atomicOr(p.status, kStatusBounds);
        if constexpr (kStats > 0) {
            float sum[4] = {halves(a.s).x + halves(a.s).y, (halves(a.u).x + halves(a.u).y) * kLn2,
                            halves(a.st).x + halves(a.st).y, (halves(a.ut).x + halves(a.ut).y) * kLn2};
#pragma unroll
            for (int o = 16; o >= 1; o >>= 1)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    sum[k] += __shfl_xor_sync(0xffffffffu, sum[k], o);
            if (lane == 0)
                s_part[gr][part] = Part{a.m, a.arg, sum[0], sum[1], sum[2], sum[3] * inv_t, {0, 0}};
        }
    }
    if (kStats == 0)
        return;

    __syncthreads();
    if (threadIdx.x < rows) {
        Part a = s_part[threadIdx.x][0];
        for (int k = 1; k < parts; ++k)
            a = combine(a, s_part[threadIdx.x][k], inv_t);
        p.parts[(size_t)(g0 + threadIdx.x) * p.slices + slice] = a;
    }
    if (!p.join)
        return;
    // the last CTA of these rows joins their slices
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        int *ticket = &p.ticket[blockIdx.x];
        s_last = atomicAdd(ticket, 1) == p.slices - 1;
        if (s_last)
            *ticket = 0;
        __threadfence();
    }
    __syncthreads();
    if (!s_last)
        return;
    if (warp < rows)
        join_row<kStats>(p, g0 + warp, row0, row1, td, lane, load_parts(p, g0 + warp, lane));
}

// Where CTAs follow one another on an SM, each one's way to the ticket and back (its
// stores have to land first) costs more than another launch: 256 requests of one row of
// 128256 tokens took 162 us with this kernel and 189 with the last CTA's join when it was
// chosen (154 now), 16 of them 17.2 and 18.3 (16.3 now).  Below that it is one launch less at the same time (9.7 us for a tree
// of 26 nodes at 32000 tokens).
template <int kStats>
__global__ void __launch_bounds__(kThreads) k_logits_join(const __grid_constant__ LogitArgs p)
{
    const int lane = threadIdx.x & 31, row = blockIdx.x * kWarps + (threadIdx.x >> 5);
    pdl_wait();
    pdl_trigger();
    if (row >= p.n_rows)
        return;
    const TwoParts first = load_parts(p, row, lane);
    const int b = owner_of(p.row_start, p.batch, row, lane);
    const int row0 = load_now(p.row_start + b), row1 = min(load_now(p.row_start + b + 1), p.n_rows);
    const int t = p.tree ? load_now(p.tree + b) : -1;
    if (row0 < 0 || row < row0 || row >= row1)  // nobody's row
        return;
    join_row<kStats>(p, row, row0, row1, t >= 0 && t < p.n_trees ? p.trees + t : nullptr, lane, first);
}

// The tokens of a slice.
int slice_of(int batch, int n_rows, int vocab, int n_sm)
{
    // as many slices as fill every SM once; longer ones scan a history less often
    // (4 requests of one row of 128256 tokens: 11.6 us, 14.6 with a third more CTAs)
    const long long rows = (n_rows + batch - 1) / batch, groups = (rows + kRows - 1) / kRows;
    const long long per_slice = (long long)batch * groups;
    const long long slices = ((long long)kPerSm * n_sm + per_slice - 1) / per_slice;
    const long long size = (vocab + slices * kChunk - 1) / (slices * kChunk) * kChunk;
    return (int)(size > kMaxSlice ? kMaxSlice : size);
}

template <int kType>
auto kernel_of(int stats_kind)
{
    return stats_kind == 0 ? k_logits<kType, 0> : stats_kind == 1 ? k_logits<kType, 1> : k_logits<kType, 2>;
}

// tickets for every piece of rows that a call may have
constexpr size_t kPartsOff = 256 + (size_t)(TB_MAX_REQUESTS + kMaxRowsCall / kRows) * sizeof(int);

}  // namespace

TB_BOUNDS_COUNTER(bounds_violations_logits)

}  // namespace tv

using namespace tv;

extern "C" size_t tb_logits_workspace_size(int batch, int n_rows, int vocab)
{
    if (batch < 1 || batch > TB_MAX_REQUESTS || n_rows < 0 || n_rows > kMaxRowsCall || vocab < 1)
        return 0;
    return kPartsOff + (size_t)n_rows * ((vocab + kChunk - 1) / kChunk) * sizeof(Part);  // the shortest slices
}

extern "C" tb_status logits_process(const tb_bank *bank, const tb_requests *req, const void *logits, int dtype,
                                    int64_t logit_stride, int n_rows, int vocab, const tb_logit_rules *rules,
                                    float temperature, float *out, int64_t out_stride, const tb_logit_stats *stats,
                                    void *workspace, size_t workspace_bytes, tb_stream stream)
{
    const char *fn = "logits_process";
    LogitArgs a{};
    tb_status st = check_requests(req, false, fn);
    if (st != TB_OK)
        return st;
    if (req->tree && (st = check_device_bank(bank, fn, &a.trees, &a.n_trees)) != TB_OK)
        return st;
    if (dtype != TB_F32 && dtype != TB_BF16 && dtype != TB_F16)
        return record_error(TB_EUNSUPPORTED, "%s: logits of type %d", fn, dtype);
    if (n_rows < 0 || n_rows > kMaxRowsCall || vocab < 1 || logit_stride < vocab || out_stride < vocab)
        return record_error(TB_EINVAL, "%s: n_rows %d, vocab %d, strides %lld, %lld", fn, n_rows, vocab,
                            (long long)logit_stride, (long long)out_stride);
    if (n_rows > 0 && (!logits || !out || !ptr_aligned(logits, 16) || !ptr_aligned(out, 16)))
        return record_error(TB_EINVAL, "%s: logits / out NULL or not 16-byte aligned", fn);
    if (n_rows > 0 && (const void *)out == logits && (dtype != TB_F32 || logit_stride != out_stride))
        return record_error(TB_EINVAL, "%s: in place with another type or stride", fn);
    if (!(temperature > 0.f) || !std::isfinite(temperature) || !std::isfinite(1.f / temperature))
        return record_error(TB_EINVAL, "%s: temperature %g", fn, temperature);
    if (rules)
        a.r = *rules;
    if (stats)
        a.st = *stats;
    if (a.r.history && (!a.r.history_len || a.r.history_stride < 1))
        return record_error(TB_EINVAL, "%s: history without history_len, or its stride %lld", fn,
                            (long long)a.r.history_stride);
    if (a.r.bias_start && (!a.r.bias_token || !a.r.bias_value))
        return record_error(TB_EINVAL, "%s: bias_start without bias_token or bias_value", fn);
    if (a.r.bias_start && (a.r.n_bias < 1 || a.r.n_bias > 0x7fffffff))
        return record_error(TB_EINVAL, "%s: bias_start into %lld entries", fn, (long long)a.r.n_bias);
    if (a.r.mask && a.r.mask_stride < (vocab + 31) / 32)
        return record_error(TB_EINVAL, "%s: mask_stride %lld below %d words", fn, (long long)a.r.mask_stride,
                            (vocab + 31) / 32);
    if (a.r.mask && a.r.mask_row && a.r.mask_rows < 1)
        return record_error(TB_EINVAL, "%s: mask_row into %lld mask rows", fn, (long long)a.r.mask_rows);
    if (a.st.draft_logit && (!a.r.draft || !req->tree))
        return record_error(TB_EINVAL, "%s: draft_logit without draft tokens or trees", fn);
    if ((st = check_workspace(workspace, workspace_bytes, tb_logits_workspace_size(req->batch, n_rows, vocab), fn)) !=
        TB_OK)
        return st;
    if (n_rows == 0)
        return launch_result(cudaSuccess, fn);
    const int n_sm = device_sms(-1);
    if (n_sm <= 0)
        return record_error(TB_ECUDA, "%s: no current device", fn);
    a.batch = req->batch;
    a.n_rows = n_rows;
    a.V = vocab;
    a.tree = req->tree;
    a.row_start = req->row_start;
    a.in = logits;
    a.in_stride = logit_stride;
    a.out = out;
    a.out_stride = out_stride;
    a.temperature = temperature;
    a.inv_t = 1.f / temperature;
    a.n_bias = (int)a.r.n_bias;
    a.mask_rows = a.r.mask_row && a.r.mask_rows < 0x7fffffff ? (int)a.r.mask_rows : 0x7fffffff;
    a.status = static_cast<int *>(workspace);
    a.ticket = reinterpret_cast<int *>(static_cast<uint8_t *>(workspace) + 256);
    a.parts = reinterpret_cast<Part *>(static_cast<uint8_t *>(workspace) + kPartsOff);
    a.size = slice_of(req->batch, n_rows, vocab, n_sm);
    a.slices = (vocab + a.size - 1) / a.size;
    if (a.slices > 65535)
        return record_error(TB_EUNSUPPORTED, "%s: vocab %d", fn, vocab);
    // count, bias, two bitmaps, the list and its offsets; then the rings
    a.ring_off = (a.size * 10 + a.size / 4 + a.size / 16 + 16 + 127) / 128 * 128;
    const int elem = dtype == TB_F32 ? 4 : 2;
    a.mask_off = a.ring_off + kWarps * kStages * stage_elems(elem) * elem;
    a.copy_off = a.mask_off + kWarps * kStages * (kChunk / 32) * 4;
    const size_t smem = (size_t)a.copy_off + (dtype == TB_F32 ? 0 : kWarps * kChunk * 4);
    const bool want = a.st.argmax || a.st.top1 || a.st.entropy || a.st.logz_t || a.st.entropy_t || a.st.draft_logit;
    const int stats_kind = !want ? 0 : (a.st.logz_t || a.st.entropy_t) && temperature != 1.f ? 2 : 1;
    const auto kernel = dtype == TB_F32    ? kernel_of<TB_F32>(stats_kind)
                        : dtype == TB_BF16 ? kernel_of<TB_BF16>(stats_kind)
                                           : kernel_of<TB_F16>(stats_kind);
    const long long pieces = req->batch + (n_rows + kRows - 1) / kRows;
    a.join = pieces * a.slices <= (long long)kPerSm * n_sm;
    cudaError_t e = allow_max_smem((const void *)kernel);
    if (e == cudaSuccess)
        e = launch_kernel(kernel, dim3((unsigned)pieces, a.slices), dim3(kThreads), smem, (cudaStream_t)stream, true, a);
    if (e == cudaSuccess && want && !a.join)
        e = launch_kernel(stats_kind == 1 ? k_logits_join<1> : k_logits_join<2>, dim3((n_rows + kWarps - 1) / kWarps),
                          dim3(kThreads), 0, (cudaStream_t)stream, true, a);
    return launch_result(e, fn);
}
