// logits.cu -- penalties for repeated tokens, biases and grammar masks on the
// logits of every row, and the statistics that the acceptance rules read, in one
// pass over the logits.
//
// A CTA takes one request and a slice of the vocabulary and builds the slice's
// rules once in shared memory for all rows of the request: how often each token
// was generated, whether the prompt has it, its bias, and a bitmap of the tokens
// that any rule touches (most of a vocabulary is touched by none).  Its warps
// then take (row, chunk) items: the chunk is read into registers at once, so its
// maximum is known before the first exponential and nothing is rescaled.  A tree
// row also counts the tokens on its root path; those inside the chunk (rarely
// any) go to a small table of the warp.  With x = z - m and m the chunk's
// maximum each item leaves (m, argmax, sum e^x, sum x e^x, and the two sums at
// temperature T); items combine to slices in shared memory and slices to rows by
// the request's last CTA (an arrival ticket), both in index order: outputs do not
// depend on the placement.
//   top1 = 1 / s,  H = ln s - u / s,  ln Z_T = m / T + ln s_T
// Penalties and biases are exact 32-bit operations in the documented order
// (nothing is contracted), counts are integers.
#include "paged.cuh"

#include <cuda_fp16.h>

#include <cmath>

namespace tv {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxChunks = 8;   // chunks per slice
constexpr int kRowGroup = 64;   // rows whose partials are in shared memory together
constexpr uint32_t kInPrompt = 0x80000000u;
constexpr float kLog2e = 1.4426950408889634f;

struct Part {
    float m;
    int arg;
    float s, u, st, ut;
    int pad[2];
};

struct LogitArgs {
    const TreeDesc *trees;
    int n_trees, batch, n_rows, V, slices, chunks;  // chunks per slice
    const int32_t *tree, *row_start;
    const void *in;
    long long in_stride, out_stride;
    float *out;
    tb_logit_rules r;
    tb_logit_stats st;
    float temperature, scale_t;  // scale_t = log2(e) / T
    int want, want_t;            // statistics at temperature 1 (with the argmax), and at T != 1
    int *ticket;                 // [batch]
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
    const float da = a.m == -INFINITY ? 0.f : a.m - o.m, db = b.m == -INFINITY ? 0.f : b.m - o.m;
    const float wa = ex2_approx(da * kLog2e), wb = ex2_approx(db * kLog2e);
    o.s = wa * a.s + wb * b.s;
    o.u = wa * (a.u + da * a.s) + wb * (b.u + db * b.s);
    const float ta = da * inv_t, tb = db * inv_t;
    const float va = ex2_approx(ta * kLog2e), vb = ex2_approx(tb * kLog2e);
    o.st = va * a.st + vb * b.st;
    o.ut = va * (a.ut + ta * a.st) + vb * (b.ut + tb * b.st);
    return o;
}

__device__ __forceinline__ Part shfl_part(const Part &a, int mask)
{
    Part o;
    o.m = __shfl_xor_sync(0xffffffffu, a.m, mask);
    o.arg = __shfl_xor_sync(0xffffffffu, a.arg, mask);
    o.s = __shfl_xor_sync(0xffffffffu, a.s, mask);
    o.u = __shfl_xor_sync(0xffffffffu, a.u, mask);
    o.st = __shfl_xor_sync(0xffffffffu, a.st, mask);
    o.ut = __shfl_xor_sync(0xffffffffu, a.ut, mask);
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

// The rules of a slice, in shared memory.
struct Slice {
    uint32_t *count;    // generated occurrences; kInPrompt: the prompt has the token
    float *bias;
    uint32_t *touched;  // bitmap
    uint8_t *extra;     // this warp's: occurrences on the row's path within its chunk
    uint32_t *path_bits;
};

__device__ __forceinline__ float penalise(float z, uint32_t c, int extra, float bias, float rep, float freq, float pres)
{
    const int n = (int)(c & ~kInPrompt) + extra;
    if (n > 0 || (c & kInPrompt))
        z = z > 0.f ? __fdiv_rn(z, rep) : __fmul_rn(z, rep);
    if (n > 0)
        z = __fsub_rn(__fsub_rn(z, __fmul_rn(freq, (float)n)), pres);
    return __fadd_rn(z, bias);
}

// kVec: groups of four tokens per lane in a chunk of 128 kVec tokens.
template <int kType, int kVec>
__global__ void __launch_bounds__(kThreads) k_logits(const __grid_constant__ LogitArgs p)
{
    constexpr int kChunk = 128 * kVec;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ Part s_part[kRowGroup][kMaxChunks];
    __shared__ uint8_t s_extra[kWarps][kChunk];
    __shared__ uint32_t s_path[kWarps][kChunk / 32];
    __shared__ int s_last;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int b = blockIdx.y, slice = blockIdx.x;
    const int size = p.chunks * kChunk, v0 = slice * size;  // v0 < V (the host's split)
    Slice sl;
    sl.count = reinterpret_cast<uint32_t *>(smem);
    sl.bias = reinterpret_cast<float *>(sl.count + size);
    sl.touched = reinterpret_cast<uint32_t *>(sl.bias + size);
    sl.extra = s_extra[warp];
    sl.path_bits = s_path[warp];
    const bool rules = p.r.history || p.r.bias_start;
    if (rules) {
        for (int x = threadIdx.x; x < size / 4; x += kThreads) {
            reinterpret_cast<uint4 *>(sl.count)[x] = make_uint4(0, 0, 0, 0);
            reinterpret_cast<uint4 *>(sl.bias)[x] = make_uint4(0, 0, 0, 0);
        }
        for (int x = threadIdx.x; x < size / 32; x += kThreads)
            sl.touched[x] = 0;
    }
    for (int x = lane; x < kChunk / 4; x += 32)
        reinterpret_cast<uint32_t *>(sl.extra)[x] = 0;
    for (int x = lane; x < kChunk / 32; x += 32)
        sl.path_bits[x] = 0;
    pdl_wait();
    pdl_trigger();
    const int row0 = max(p.row_start[b], 0), row1 = min(p.row_start[b + 1], p.n_rows);
    if (row0 >= row1)
        return;
    const int t = p.tree ? p.tree[b] : -1;
    const TreeDesc *td = t >= 0 && t < p.n_trees ? p.trees + t : nullptr;
    const float rep = p.r.repetition ? p.r.repetition[b] : 1.f;
    const float freq = p.r.frequency ? p.r.frequency[b] : 0.f;
    const float pres = p.r.presence ? p.r.presence[b] : 0.f;
    __syncthreads();
    if (p.r.history) {
        const int32_t *h = p.r.history + b * p.r.history_stride;
        const int n = (int)min((long long)max(p.r.history_len[b], 0), (long long)p.r.history_stride);
        const int prompt = p.r.prompt_len ? min(max(p.r.prompt_len[b], 0), n) : 0;
        auto note = [&](int i, int tok) {
            const unsigned loc = (unsigned)(tok - v0);
            if (loc < (unsigned)size && tok < p.V) {
                if (i < prompt)
                    atomicOr(&sl.count[loc], kInPrompt);
                else
                    atomicAdd(&sl.count[loc], 1u);
                atomicOr(&sl.touched[loc >> 5], 1u << (loc & 31));
            }
        };
        constexpr int kAhead = 8;
        for (int i0 = threadIdx.x; i0 < n; i0 += kThreads * kAhead) {
            int tok[kAhead];
#pragma unroll
            for (int m = 0; m < kAhead; ++m)
                tok[m] = i0 + m * kThreads < n ? h[i0 + m * kThreads] : -1;
#pragma unroll
            for (int m = 0; m < kAhead; ++m)
                if (tok[m] >= 0)
                    note(i0 + m * kThreads, tok[m]);
        }
    }
    if (p.r.bias_start && warp == 0) {
        // in list order: entries of one token add up in a fixed order
        const int e1 = p.r.bias_start[b + 1];
        for (int e0 = max(p.r.bias_start[b], 0); e0 < e1; e0 += 32) {
            const int e = e0 + lane;
            const int tok = e < e1 ? p.r.bias_token[e] : -1;
            const unsigned loc = (unsigned)(tok - v0);
            const bool mine = tok >= 0 && tok < p.V && loc < (unsigned)size;
            const float val = mine ? p.r.bias_value[e] : 0.f;
            const unsigned same = __match_any_sync(0xffffffffu, mine ? (int)loc : -1 - lane);
            const bool leader = mine && (same & ((1u << lane) - 1)) == 0;
            float acc = leader ? sl.bias[loc] : 0.f;
            for (int k = 0; k < 32; ++k) {
                const float other = __shfl_sync(0xffffffffu, val, k);
                if ((same >> k) & 1)
                    acc += other;
            }
            if (leader) {
                sl.bias[loc] = acc;
                atomicOr(&sl.touched[loc >> 5], 1u << (loc & 31));
            }
            __syncwarp();
        }
    }
    __syncthreads();

    const int n_chunks = min(p.chunks, (p.V - v0 + kChunk - 1) / kChunk);
    const float inv_t = 1.f / p.temperature;
    using T = typename In<kType>::T;
    for (int g0 = row0; g0 < row1; g0 += kRowGroup) {
        const int rows = min(kRowGroup, row1 - g0);
        for (int item = warp; item < rows * n_chunks; item += kWarps) {
            const int gr = item / n_chunks, ch = item - gr * n_chunks, row = g0 + gr;
            const int c0 = v0 + ch * kChunk, room = p.V - c0;  // tokens of the chunk that exist
            const T *src = static_cast<const T *>(p.in) + row * p.in_stride + c0;
            float *dst = p.out + row * p.out_stride + c0;
            float z[kVec][4];
            const bool in_vec = (reinterpret_cast<uintptr_t>(src) & (4 * sizeof(T) - 1)) == 0 && room >= kChunk;
            if (in_vec) {
#pragma unroll
                for (int k = 0; k < kVec; ++k) {
                    const float4 x = In<kType>::four(src + k * 128 + lane * 4);
                    z[k][0] = x.x, z[k][1] = x.y, z[k][2] = x.z, z[k][3] = x.w;
                }
            } else {
#pragma unroll
                for (int k = 0; k < kVec; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int o = k * 128 + lane * 4 + e;
                        z[k][e] = o < room ? In<kType>::one(src + o) : -INFINITY;
                    }
            }
            // this row's mask words of the chunk: lane's four tokens lie in word 4 k + lane / 8
            uint32_t allow[kVec];
            const int mrow = !p.r.mask ? -1 : p.r.mask_row ? p.r.mask_row[row] : row;
            const int32_t *mask = mrow >= 0 ? p.r.mask + mrow * p.r.mask_stride + (c0 >> 5) : nullptr;
#pragma unroll
            for (int k = 0; k < kVec; ++k) {
                const int w = 4 * k + (lane >> 3);
                allow[k] = 0xfu;
                if (mask && w * 32 < room)
                    allow[k] = ((uint32_t)mask[w] >> (4 * (lane & 7))) & 0xfu;
            }
            // the draft tokens on this row's root path that fall into the chunk
            bool on_path = false;
            int tok[2] = {-1, -1};
            if (td && p.r.draft && row - row0 < td->n) {
                const uint64_t anc = td->anc[row - row0] & ~1ull;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int j = lane + 32 * h;
                    if ((anc >> j) & 1) {
                        const int x = p.r.draft[row0 + j] - c0;
                        if (x >= 0 && x < kChunk && x < room)
                            tok[h] = x;
                    }
                }
                on_path = __any_sync(0xffffffffu, tok[0] >= 0 || tok[1] >= 0);
            }
            if (on_path) {
                for (int h = 0; h < 2; ++h)
                    for (int k = 0; k < 32; ++k) {
                        const int x = __shfl_sync(0xffffffffu, tok[h], k);
                        if (x >= 0 && lane == 0) {
                            sl.extra[x] += 1;
                            sl.path_bits[x >> 5] |= 1u << (x & 31);
                        }
                    }
                __syncwarp();
            }
            if (rules || on_path) {
#pragma unroll
                for (int k = 0; k < kVec; ++k) {
                    const int o = k * 128 + lane * 4, loc = ch * kChunk + o;
                    uint32_t bits = rules ? sl.touched[loc >> 5] : 0u;
                    if (on_path)
                        bits |= sl.path_bits[o >> 5];
                    bits = (bits >> (o & 31)) & 0xfu;
                    if (bits) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if ((bits >> e) & 1)
                                z[k][e] = penalise(z[k][e], rules ? sl.count[loc + e] : 0u,
                                                   on_path ? sl.extra[o + e] : 0, rules ? sl.bias[loc + e] : 0.f, rep,
                                                   freq, pres);
                    }
                }
            }
            if (on_path) {
                __syncwarp();
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    if (tok[h] >= 0) {
                        sl.extra[tok[h]] = 0;
                        sl.path_bits[tok[h] >> 5] = 0;
                    }
                __syncwarp();
            }
#pragma unroll
            for (int k = 0; k < kVec; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (!((allow[k] >> e) & 1))
                        z[k][e] = -INFINITY;
            if ((reinterpret_cast<uintptr_t>(dst) & 15) == 0 && room >= kChunk) {
#pragma unroll
                for (int k = 0; k < kVec; ++k)
                    *reinterpret_cast<float4 *>(dst + k * 128 + lane * 4) =
                        make_float4(z[k][0], z[k][1], z[k][2], z[k][3]);
            } else {
#pragma unroll
                for (int k = 0; k < kVec; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int o = k * 128 + lane * 4 + e;
                        if (o < room)
                            dst[o] = z[k][e];
                    }
            }
            if (!p.want)
                continue;
            // the chunk's maximum, then its sums
            Part a = empty_part();
#pragma unroll
            for (int k = 0; k < kVec; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (z[k][e] > a.m) {
                        a.m = z[k][e];
                        a.arg = c0 + k * 128 + lane * 4 + e;
                    }
            float m = a.m;
            int arg = a.arg;
#pragma unroll
            for (int o = 16; o >= 1; o >>= 1) {
                const float om = __shfl_xor_sync(0xffffffffu, m, o);
                const int oa = __shfl_xor_sync(0xffffffffu, arg, o);
                if (om > m || (om == m && oa < arg))
                    m = om, arg = oa;
            }
            const float mu = m == -INFINITY ? 0.f : m;
            float s = 0.f, u = 0.f, st = 0.f, ut = 0.f;
#pragma unroll
            for (int k = 0; k < kVec; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = z[k][e] - mu;
                    const float q = ex2_approx(x * kLog2e);
                    s += q;
                    u += q > 0.f ? q * x : 0.f;
                    if (p.want_t) {
                        const float qt = ex2_approx(x * p.scale_t);
                        st += qt;
                        ut += qt > 0.f ? qt * x : 0.f;
                    }
                }
#pragma unroll
            for (int o = 16; o >= 1; o >>= 1) {
                s += __shfl_xor_sync(0xffffffffu, s, o);
                u += __shfl_xor_sync(0xffffffffu, u, o);
                st += __shfl_xor_sync(0xffffffffu, st, o);
                ut += __shfl_xor_sync(0xffffffffu, ut, o);
            }
            if (lane == 0)
                s_part[gr][ch] = Part{m, arg, s, u, st, ut * inv_t, {0, 0}};
        }
        if (!p.want)
            continue;
        __syncthreads();
        for (int gr = threadIdx.x; gr < rows; gr += kThreads) {
            Part a = s_part[gr][0];
            for (int ch = 1; ch < n_chunks; ++ch)
                a = combine(a, s_part[gr][ch], inv_t);
            p.parts[(size_t)(g0 + gr) * p.slices + slice] = a;
        }
        __syncthreads();
    }
    if (!p.want)
        return;

    // the request's last CTA combines the slices of its rows
    if (threadIdx.x == 0) {
        __threadfence();
        s_last = atomicAdd(&p.ticket[b], 1) == p.slices - 1;
        if (s_last) {
            p.ticket[b] = 0;
            __threadfence();
        }
    }
    __syncthreads();
    if (!s_last)
        return;
    for (int row = row0 + warp; row < row1; row += kWarps) {
        const Part *parts = p.parts + (size_t)row * p.slices;
        Part a = empty_part();
        for (int k = lane; k < p.slices; k += 32) {
            Part x;
            *reinterpret_cast<float4 *>(&x) = __ldcg(reinterpret_cast<const float4 *>(parts + k));
            *(reinterpret_cast<float4 *>(&x) + 1) = __ldcg(reinterpret_cast<const float4 *>(parts + k) + 1);
            a = combine(a, x, inv_t);
        }
#pragma unroll
        for (int o = 16; o >= 1; o >>= 1)
            a = combine(a, shfl_part(a, o), inv_t);
        if (lane == 0) {
            // a row without an allowed token: sums 0 (NaN where its allowed logits are)
            const bool none = a.m == -INFINITY;
            const bool empty = none && a.s == 0.f;
            if (p.st.argmax)
                p.st.argmax[row] = none ? -1 : a.arg;
            if (p.st.top1)
                p.st.top1[row] = empty ? 0.f : 1.f / a.s;
            if (p.st.entropy)
                p.st.entropy[row] = empty ? 0.f : logf(a.s) - a.u / a.s;
            const float sT = p.want_t ? a.st : a.s, uT = p.want_t ? a.ut : a.u;
            if (p.st.logz_t)
                p.st.logz_t[row] = empty ? -INFINITY : __fdiv_rn(a.m, p.temperature) + logf(sT);
            if (p.st.entropy_t)
                p.st.entropy_t[row] = empty ? 0.f : logf(sT) - uT / sT;
        }
        const int j = row - row0;
        if (p.st.draft_logit && lane == 0 && td && j > 0 && j < td->n) {
            const int tok = p.r.draft[row], par = row0 + td->parent[j];
            if (tok >= 0 && tok < p.V && par < p.n_rows)
                p.st.draft_logit[row] = __ldcg(p.out + par * p.out_stride + tok);
        }
    }
}

// Tokens per chunk: large ones where the batch fills the GPU with them, else
// small ones, so that one request's rows spread over the SMs.
int chunk_of(int batch, int vocab)
{
    return (long long)batch * ((vocab + 1023) / 1024) >= 512 ? 1024 : 256;
}

constexpr size_t kPartsOff = 256 + (size_t)TB_MAX_REQUESTS * sizeof(int);

template <int kVec>
cudaError_t launch(const LogitArgs &a, int dtype, cudaStream_t stream)
{
    const int size = a.chunks * 128 * kVec;
    const size_t smem = (size_t)size * 8 + size / 8;
    const auto kernel = dtype == TB_F32    ? k_logits<TB_F32, kVec>
                        : dtype == TB_BF16 ? k_logits<TB_BF16, kVec>
                                           : k_logits<TB_F16, kVec>;
    const cudaError_t e = allow_max_smem((const void *)kernel);
    return e != cudaSuccess ? e : launch_kernel(kernel, dim3(a.slices, a.batch), dim3(kThreads), smem, stream, true, a);
}

}  // namespace

TB_BOUNDS_COUNTER(bounds_violations_logits)

}  // namespace tv

using namespace tv;

extern "C" size_t tb_logits_workspace_size(int batch, int n_rows, int vocab)
{
    if (batch < 1 || batch > TB_MAX_REQUESTS || n_rows < 0 || vocab < 1)
        return 0;
    const int chunk = chunk_of(batch, vocab);
    return kPartsOff + (size_t)n_rows * ((vocab + chunk - 1) / chunk) * sizeof(Part);
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
    if (n_rows < 0 || vocab < 1 || logit_stride < vocab || out_stride < vocab)
        return record_error(TB_EINVAL, "%s: n_rows %d, vocab %d, strides %lld, %lld", fn, n_rows, vocab,
                            (long long)logit_stride, (long long)out_stride);
    if (!logits || !out || !ptr_aligned(logits, 16) || !ptr_aligned(out, 16))
        return record_error(TB_EINVAL, "%s: logits / out NULL or not 16-byte aligned", fn);
    if ((const void *)out == logits && (dtype != TB_F32 || logit_stride != out_stride))
        return record_error(TB_EINVAL, "%s: in place with another type or stride", fn);
    if (!(temperature > 0.f) || !std::isfinite(temperature))
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
    if (a.r.mask && a.r.mask_stride < (vocab + 31) / 32)
        return record_error(TB_EINVAL, "%s: mask_stride %lld below %d words", fn, (long long)a.r.mask_stride,
                            (vocab + 31) / 32);
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
    a.scale_t = (float)(1.4426950408889634 / (double)temperature);
    a.want = a.st.argmax || a.st.top1 || a.st.entropy || a.st.logz_t || a.st.entropy_t || a.st.draft_logit;
    a.want_t = (a.st.logz_t || a.st.entropy_t) && temperature != 1.f;
    a.ticket = reinterpret_cast<int *>(static_cast<uint8_t *>(workspace) + 256);
    a.parts = reinterpret_cast<Part *>(static_cast<uint8_t *>(workspace) + kPartsOff);
    const int chunk = chunk_of(req->batch, vocab), n_chunks = (vocab + chunk - 1) / chunk;
    // chunks per slice: about six CTAs for each SM; a longer slice scans a
    // request's history less often
    long long per = ((long long)n_chunks * req->batch + 6ll * n_sm - 1) / (6ll * n_sm);
    a.chunks = (int)(per < 1 ? 1 : per > kMaxChunks ? kMaxChunks : per);
    a.slices = (n_chunks + a.chunks - 1) / a.chunks;
    const cudaError_t e = chunk == 1024 ? launch<8>(a, dtype, (cudaStream_t)stream)
                                        : launch<2>(a, dtype, (cudaStream_t)stream);
    return launch_result(e, fn);
}
