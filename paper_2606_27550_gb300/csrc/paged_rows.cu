// paged_rows.cu -- the store with norms of the heads before the rotation, into
// pages of 16 bits or of 4, and the way back from 4 bits to rows of 16.
//
// What follows the rotation may be a rounding to 4 bits, where the last bit of a
// 32-bit number decides between two values a seventh of the largest apart.  So
// the steps before it are those of the documented formulas, each rounded once,
// and what goes into them is right to the last bit but for rare near-ties: sines,
// cosines and the norm's reciprocal root are computed with a second float that
// holds what the first leaves (a sum's or product's rounding error is a float
// itself: Dekker 1971, Knuth's two-sum).  Another program that follows the formulas
// gets the same values, and the same keys but for such near-ties (fewer than 1 of 10^7 elements, as a sine's
// last bit moves an element by 2^-23 of the head's size; without a rotation and norms, all of them).
//
// A CTA takes a few rows: their (cos, sin) once into shared memory (they serve
// all heads), then every (row, head, 16-byte piece of the lower half of the head
// and its partner in the upper half).  A head's pieces lie in 4 or 8 neighbouring
// lanes, which add up its squares; four of them hold a scale's 32 elements.
#include "paged_q4.cuh"

#include <cmath>

namespace tv {

namespace {

constexpr int kThreads = 256;
constexpr int kCtas = 4;  // of an SM
constexpr int kMaxRows = 8;  // rows per CTA

struct RowsArgs {
    uint8_t *k_pages, *v_pages;  // of the layer
    long long page_stride, head_stride, slot_stride;  // bytes; 4-bit pages have no slot stride
    int n_pages, page_log2, Hkv, Hq, n_rows, rows_per_cta;
    const int64_t *slots;
    Rows k, v, q, q_out;
    const uint16_t *q_weight, *k_weight;  // NULL: not normed
    float eps, weight_offset;
    int turn;
    RopeAxes rope;
};

// A number as the sum of two floats, the second below half a unit in the last place of the first.
struct Two {
    float hi, lo;
};
__device__ __forceinline__ Two sum_of(float a, float b)
{
    const float s = __fadd_rn(a, b), t = __fsub_rn(s, a);
    return {s, __fadd_rn(__fsub_rn(a, __fsub_rn(s, t)), __fsub_rn(b, t))};
}
__device__ __forceinline__ Two near_sum(float a, float b)  // |a| >= |b|
{
    const float s = __fadd_rn(a, b);
    return {s, __fsub_rn(b, __fsub_rn(s, a))};
}
__device__ __forceinline__ Two product(Two a, Two b)
{
    const float p = __fmul_rn(a.hi, b.hi);
    float e = __fmaf_rn(a.hi, b.hi, -p);
    e = __fmaf_rn(a.hi, b.lo, e);
    e = __fmaf_rn(a.lo, b.hi, e);
    return {p, e};
}
__device__ __forceinline__ Two plus(Two c, Two x)  // |c| >= |x|
{
    const Two s = near_sum(c.hi, x.hi);
    return {s.hi, __fadd_rn(s.lo, __fadd_rn(c.lo, x.lo))};
}

// Cosine and sine of an angle in 2^-64 of a turn: the nearest quarter turn, and the Taylor series of
// the rest, at most pi / 4, its first terms in two floats.  Off by 2^-34 of itself at most before the one
// rounding: the series' ends are 2^-36 of it (sine) and 2^-41, the last terms' own roundings 2^-35.
__device__ float2 cos_sin(uint64_t turn)
{
    const int quarter = (int)((turn + (1ull << 61)) >> 62);
    const int64_t r = (int64_t)(turn - ((uint64_t)quarter << 62));  // in [-2^61, 2^61)
    // its leading bits, wherever they stand: 24 in one float, the next 32 rounded to 24 in another (2^-47 of it).
    // Small angles take the same way as large ones
    const uint64_t size = r < 0 ? 0 - (uint64_t)r : (uint64_t)r;
    const int zeros = __clzll((long long)(size | 1));
    const uint64_t m = size << zeros;
    const float h = __uint2float_rn((uint32_t)(m >> 40)), l = __fmul_rn(__uint2float_rn((uint32_t)(m >> 8)), 0x1p-32f);
    // times 2 pi / 2^24, then 2^-zeros and the sign
    Two y = product(near_sum(h, l), Two{6.28318548202514648f * 0x1p-24f, -1.74845553146951715e-07f * 0x1p-24f});
    y = near_sum(y.hi, y.lo);
    const float unit = __int_as_float((int)((uint32_t)(127 - zeros) << 23 | (r < 0 ? 0x80000000u : 0u)));
    y = Two{__fmul_rn(y.hi, unit), __fmul_rn(y.lo, unit)};
    const Two z = product(y, y);
    // sin y = y + y z S(z), cos y = 1 + z C(z)
    float f = __fmaf_rn(z.hi, __fmaf_rn(z.hi, -1.f / 39916800.f, 1.f / 362880.f), -1.f / 5040.f);
    Two s = plus(Two{8.33333376795053482e-03f, -4.34617203337595e-10f}, Two{__fmul_rn(z.hi, f), 0.f});  // 1 / 120
    s = plus(Two{-1.66666671633720398e-01f, 4.96705373128283e-09f}, product(z, s));                     // -1 / 6
    s = product(y, product(z, s));
    Two e = near_sum(y.hi, s.hi);
    const float sine = __fadd_rn(e.hi, __fadd_rn(e.lo, __fadd_rn(y.lo, s.lo)));
    f = __fmaf_rn(z.hi, __fmaf_rn(z.hi, __fmaf_rn(z.hi, 1.f / 479001600.f, -1.f / 3628800.f), 1.f / 40320.f), -1.f / 720.f);
    Two c = plus(Two{4.16666679084300995e-02f, -1.24176343282071e-09f}, Two{__fmul_rn(z.hi, f), 0.f});  // 1 / 24
    c = plus(Two{-0.5f, 0.f}, product(z, c));
    c = product(z, c);
    e = near_sum(1.f, c.hi);
    const float cosine = __fadd_rn(e.hi, __fadd_rn(e.lo, c.lo));
    switch (quarter & 3) {
    case 0:
        return make_float2(cosine, sine);
    case 1:
        return make_float2(-sine, cosine);
    case 2:
        return make_float2(-cosine, -sine);
    default:
        return make_float2(sine, -cosine);
    }
}

__device__ __forceinline__ uint64_t minus(uint64_t a, uint64_t b)  // of two numbers each
{
    return fma_two(b, two(-1.f, -1.f), a);
}

// 1 / sqrt(mean of squares + eps) of the head whose 16 elements each are held by kLanes neighbouring
// lanes.  By the whole warp; what it returns where `normed` is false is not read.
template <int kLanes>
__device__ __forceinline__ float inverse_norm(const uint64_t (&x)[8], float eps, bool normed)
{
    // two sums, each with what its roundings left
    uint64_t hi = mul_two(x[0], x[0]), lo = two(0.f, 0.f);
#pragma unroll
    for (int i = 1; i < 8; ++i) {
        const uint64_t b = mul_two(x[i], x[i]);  // 11 bits at most: the squares are exact
        const uint64_t s = add_two(hi, b), t = minus(s, hi);
        lo = add_two(lo, add_two(minus(hi, minus(s, t)), minus(b, t)));
        hi = s;
    }
    Two s = sum_of(halves(hi).x, halves(hi).y);
    s.lo = __fadd_rn(s.lo, __fadd_rn(halves(lo).x, halves(lo).y));
#pragma unroll
    for (int m = 1; m < kLanes; m *= 2) {
        const float h = __shfl_xor_sync(0xffffffffu, s.hi, m), l = __shfl_xor_sync(0xffffffffu, s.lo, m);
        const Two t = sum_of(s.hi, h);
        s = {t.hi, __fadd_rn(__fadd_rn(s.lo, l), t.lo)};
    }
    constexpr float kMean = 1.f / (16 * kLanes);
    const bool fits = !normed || (s.hi > 0x1p-60f && s.hi < 0x1p120f);
    if (__any_sync(0xffffffffu, !fits)) {
        // squares that leave the range of 32 bits (all zeros among them): in 64
        double t = 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 f = halves(x[i]);
            t += (double)f.x * f.x + (double)f.y * f.y;
        }
#pragma unroll
        for (int m = 1; m < kLanes; m *= 2)
            t += __shfl_xor_sync(0xffffffffu, t, m);
        if (!fits)
            return (float)(1.0 / sqrt(t * kMean + eps));
    }
    Two v = sum_of(s.hi * kMean, eps);
    v = near_sum(v.hi, __fadd_rn(v.lo, s.lo * kMean));
    // one Newton step from the 32-bit root, its residual 1 - v y^2 with y^2 in two floats
    const float y = rsqrtf(v.hi);
    const float a = __fmul_rn(y, y), b = __fmaf_rn(y, y, -a);
    float t = __fmaf_rn(-v.hi, a, 1.f);
    t = __fmaf_rn(-v.hi, b, t);
    t = __fmaf_rn(-v.lo, a, t);
    return __fmaf_rn(0.5f * y, t, y);
}

template <bool kF16>
__device__ __forceinline__ void widen(const uint4 &w, uint64_t *x)
{
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = unpack_pair<kF16>(u[i]);
        x[i] = two(f.x, f.y);
    }
}
template <bool kF16>
__device__ __forceinline__ uint4 narrow(const uint64_t *x)
{
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        u[i] = pack_pair<kF16>(halves(x[i]).x, halves(x[i]).y);
    return make_uint4(u[0], u[1], u[2], u[3]);
}
// 8 floats of shared memory
__device__ __forceinline__ void four_pairs(const float *from, uint64_t (&x)[4])
{
    const float4 a = *reinterpret_cast<const float4 *>(from), b = *reinterpret_cast<const float4 *>(from + 4);
    x[0] = two(a.x, a.y), x[1] = two(a.z, a.w), x[2] = two(b.x, b.y), x[3] = two(b.z, b.w);
}
__device__ __forceinline__ float max_or_nan(float a, float b)
{
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}
__device__ __forceinline__ float max_or_nan(float a, float2 b)  // of magnitudes
{
    float y;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b.x), "f"(b.y));
    return y;
}
// to one unit in the last place
__device__ __forceinline__ float reciprocal(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Bound by HBM where rows stay in 16 bits: each element is read once and written once (8191 rows of 32 + 2 * 32
// heads of 128, normed and turned: 74 us, 5.4 TB/s, 80 % of a copy's bandwidth; 87 us with a division for each
// piece to find its place), and by its instructions where they become 4 bits (the same
// rows: 91 us, 73 without norms, 79 without the rotation, 63 with neither, which rows of 16 bits take too; the
// largest of 32, the scale and 32 corrected quotients on top; 149 us with a division each and one number at a time)
// and what they wait for: 70 % of the issue slots are taken.  One to eight rows per CTA: the sines serve all of a row's heads, and
// few rows still reach all SMs (eight trees, 32 + 2 * 8 heads: 5.3 us).
template <int kD, bool kF16, bool kQ4>
__global__ void __launch_bounds__(kThreads, kCtas) k_paged_rows(const __grid_constant__ RowsArgs p)
{
    constexpr int kHalf = kD / 2, kLanes = kHalf / 8;  // lanes of a head
    __shared__ __align__(16) float s_cos[kMaxRows][kHalf], s_sin[kMaxRows][kHalf];
    __shared__ __align__(16) float s_weight[2][kD];
    __shared__ long long s_slot[kMaxRows];
    pdl_wait();
    pdl_trigger();
    const int r0 = blockIdx.x * p.rows_per_cta, n_rows = min(p.rows_per_cta, p.n_rows - r0);
    const int threads = blockDim.x;
    const bool norms = p.q_weight || p.k_weight;
    for (int x = threadIdx.x; x < n_rows; x += threads)
        s_slot[x] = p.slots[r0 + x];
    if (norms && threadIdx.x < kD) {
        const int x = threadIdx.x;
        const uint16_t *w[2] = {p.q_weight, p.k_weight};
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (w[i])
                s_weight[i][x] = p.weight_offset + unpack_pair<kF16>(w[i][x]).x;
    }
    if (p.turn)
        for (int x = threadIdx.x; x < n_rows * kHalf; x += threads) {
            const float2 cs = cos_sin(turn_of(p.rope, r0 + x / kHalf, x % kHalf));
            s_cos[x / kHalf][x % kHalf] = cs.x;
            s_sin[x / kHalf][x % kHalf] = cs.y;
        }
    __syncthreads();
    // A thread keeps its place in a row, (head, 16 bytes of either half), and takes row after row; where a row
    // has fewer places than the CTA threads, several rows stand abreast.  Whole warps go through the loops: a
    // head's lanes add up together, and what lies outside does a valid row's work and writes nothing.
    const int per_row = (p.Hq + 2 * p.Hkv) * kLanes, abreast = per_row < threads ? threads / per_row : 1;
    const int sub = per_row < threads ? (int)threadIdx.x / per_row : 0;
    constexpr int kAhead = 2;  // rows per thread in flight
    const int c = (int)(threadIdx.x % kLanes) * 8;  // (the threads are a multiple of a head's lanes)
    for (int y0 = 0; y0 < per_row; y0 += threads) {
        const int y = y0 + (int)threadIdx.x - sub * per_row;
        const bool live = y < per_row && sub < abreast;
        int h = live ? y / kLanes : 0;
        const int kind = h < p.Hq ? 0 : h < p.Hq + p.Hkv ? 1 : 2;  // a query, a key, a value
        h -= kind == 0 ? 0 : kind == 1 ? p.Hq : p.Hq + p.Hkv;
        const Rows &rows = kind == 0 ? p.q : kind == 1 ? p.k : p.v;
        const uint16_t *src = rows.p + r0 * rows.row_stride + h * rows.head_stride + c;
        const long long src_stride = rows.row_stride;
        uint16_t *const q_out = p.q_out.p + r0 * p.q_out.row_stride + h * p.q_out.head_stride + c;
        uint8_t *const pages = (kind == 2 ? p.v_pages : p.k_pages) + h * p.head_stride;
        const bool normed = live && (kind == 0 ? p.q_weight != nullptr : kind == 1 && p.k_weight != nullptr);
        const bool any_normed = __any_sync(0xffffffffu, normed), turns = p.turn && kind < 2;
        const bool any_key = __any_sync(0xffffffffu, live && kind > 0);
        const bool as_is = !kQ4 && __all_sync(0xffffffffu, kind == 2 || !live);  // values stay as they are
        for (int rr = 0; rr < n_rows; rr += kAhead * abreast) {
            uint4 in[kAhead][2];
#pragma unroll
            for (int m = 0; m < kAhead; ++m) {
                const uint16_t *from = src + min(rr + m * abreast + sub, n_rows - 1) * src_stride;
                in[m][0] = *reinterpret_cast<const uint4 *>(from);
                in[m][1] = *reinterpret_cast<const uint4 *>(from + kHalf);
            }
#pragma unroll
            for (int m = 0; m < kAhead; ++m) {
                if (rr + m * abreast >= n_rows)
                    break;
                const int r = min(rr + m * abreast + sub, n_rows - 1);
                bool there = live && rr + m * abreast + sub < n_rows;
                uint8_t *dst, *scales_to = nullptr;
                if (kind == 0) {
                    dst = reinterpret_cast<uint8_t *>(q_out + r * p.q_out.row_stride);
                } else {
                    const long long slot = s_slot[r], page = slot >> p.page_log2;
                    there = there && slot >= 0 && page < p.n_pages;  // else padding
                    const int in_page = (int)slot & ((1 << p.page_log2) - 1);
                    dst = pages + page * p.page_stride;
                    if constexpr (kQ4) {
                        scales_to = dst + ((long long)code_bytes(kD) << p.page_log2) + in_page * scale_bytes(kD);
                        dst += in_page * code_bytes(kD) + c / 2;
                    } else {
                        dst += in_page * p.slot_stride + 2 * c;
                    }
                }
                if (as_is) {
                    if (there) {
                        *reinterpret_cast<uint4 *>(dst) = in[m][0];
                        *reinterpret_cast<uint4 *>(dst + 2 * kHalf) = in[m][1];
                    }
                    continue;
                }
                uint64_t v[8];  // the lower half's 8 elements, the upper half's
                widen<kF16>(in[m][0], v);
                widen<kF16>(in[m][1], v + 4);
                if (any_normed) {
                    const float inv = inverse_norm<kLanes>(v, p.eps, normed);
                    if (normed) {
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            uint64_t w[4];
                            four_pairs(s_weight[kind] + c + i * kHalf, w);
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                v[4 * i + j] = mul_two(mul_two(v[4 * i + j], two(inv, inv)), w[j]);
                        }
                    }
                }
                if (turns) {
                    uint64_t co[4], si[4];
                    four_pairs(s_cos[r] + c, co);
                    four_pairs(s_sin[r] + c, si);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint64_t a = v[i], b = v[4 + i];
                        const float2 ac = halves(mul_two(a, co[i])), bs = halves(mul_two(b, si[i]));
                        const float2 bc = halves(mul_two(b, co[i])), as = halves(mul_two(a, si[i]));
                        // (one by one: the assembler makes one fma of a product and a sum of pairs)
                        v[i] = two(__fsub_rn(ac.x, bs.x), __fsub_rn(ac.y, bs.y));
                        v[4 + i] = two(__fadd_rn(bc.x, as.x), __fadd_rn(bc.y, as.y));
                    }
                }
                if ((!kQ4 || kind == 0) && there) {
                    *reinterpret_cast<uint4 *>(dst) = narrow<kF16>(v);
                    *reinterpret_cast<uint4 *>(dst + 2 * kHalf) = narrow<kF16>(v + 4);
                }
                if (kQ4 && any_key) {
                    uint32_t sb[2], word[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint64_t x[4] = {v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
                        float top = 0.f;
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            top = max_or_nan(top, halves(x[j]));
                        top = max_or_nan(top, __shfl_xor_sync(0xffffffffu, top, 1));
                        top = max_or_nan(top, __shfl_xor_sync(0xffffffffu, top, 2));
                        sb[i] = scale_byte(top);
                        const float s = scale_of(sb[i]);
                        word[i] = quantize8(x, s, s == 0.f ? 0.f : reciprocal(s),
                                             __any_sync(0xffffffffu, sb[i] >= kMaxScaleByte));
                    }
                    // the head's scales from its lanes 0 and 4 (kD = 64: lane 0)
                    uint32_t scales = sb[0] | sb[1] << (8 * kD / (2 * kGroup));
                    if constexpr (kLanes == 8)
                        scales |= __shfl_xor_sync(0xffffffffu, scales, 4) << 8;
                    if (kind > 0 && there) {
                        *reinterpret_cast<uint32_t *>(dst) = word[0];
                        *reinterpret_cast<uint32_t *>(dst + kHalf / 2) = word[1];
                        if (c == 0) {
                            if constexpr (kD == 128)
                                *reinterpret_cast<uint32_t *>(scales_to) = scales;
                            else
                                *reinterpret_cast<uint16_t *>(scales_to) = (uint16_t)scales;
                        }
                    }
                }
            }
        }
    }
}

// ------------------------------------------------------------------ back to 16 bits

struct LoadArgs {
    const uint8_t *k_pages, *v_pages;  // of the first layer
    long long layer_stride, page_stride, head_stride;
    int n_pages, page_log2, Hkv, n_rows;
    const int64_t *slots;
    Rows k, v;
    long long row_layer_stride;
};

// 16 codes (8 bytes, half a scale's) become 32 bytes, a sector, written at once.
constexpr int kLoadCodes = 16, kLoadAhead = 4;

// A thread keeps its place in a row, (K or V, head, 16 elements), and takes a few rows.  Bound by HBM: 0.53
// bytes read and 2 written per element (8000 rows of 32 layers and 8 heads of 128: 197 us, 6.7 TB/s, 99 % of
// a copy's bandwidth; 240 us in stores of 16 bytes, which fill half a sector each).
template <int kD, bool kF16>
__global__ void __launch_bounds__(kThreads) k_paged_load(const __grid_constant__ LoadArgs p, int rows_per_cta)
{
    constexpr int kPieces = kD / kLoadCodes;
    pdl_wait();
    pdl_trigger();
    const int per_row = 2 * p.Hkv * kPieces, layer = blockIdx.y;
    // rows at a time: as many as the CTA's threads cover
    const int abreast = per_row < kThreads ? kThreads / per_row : 1;
    const int first = (int)blockIdx.x * rows_per_cta, end = min(first + rows_per_cta, p.n_rows);
    const int sub = per_row < kThreads ? (int)threadIdx.x / per_row : 0;
    if (sub >= abreast)
        return;
    for (int y = (int)threadIdx.x - sub * per_row; y < per_row; y += kThreads) {
        int h = y / kPieces;
        const int w = y % kPieces;
        const bool is_v = h >= p.Hkv;
        h -= is_v ? p.Hkv : 0;
        const uint8_t *codes = (is_v ? p.v_pages : p.k_pages) + layer * p.layer_stride + h * p.head_stride + 8 * w;
        const uint8_t *scales = codes - 8 * w + ((long long)code_bytes(kD) << p.page_log2) + w / 2;
        const Rows &to = is_v ? p.v : p.k;
        uint16_t *out = to.p + layer * p.row_layer_stride + h * to.head_stride + kLoadCodes * w;
        for (int r0 = first + sub; r0 < end; r0 += kLoadAhead * abreast) {
            uint2 code[kLoadAhead];
            uint32_t scale[kLoadAhead];
            bool there[kLoadAhead];
#pragma unroll
            for (int m = 0; m < kLoadAhead; ++m) {
                const int r = r0 + m * abreast;
                const long long slot = r < end ? p.slots[r] : -1, page = slot >> p.page_log2;
                there[m] = slot >= 0 && page < p.n_pages;  // else padding
                if (!there[m])
                    continue;
                const int in_page = (int)slot & ((1 << p.page_log2) - 1);
                code[m] = *reinterpret_cast<const uint2 *>(codes + page * p.page_stride + in_page * code_bytes(kD));
                scale[m] = scales[page * p.page_stride + in_page * scale_bytes(kD)];
            }
#pragma unroll
            for (int m = 0; m < kLoadAhead; ++m) {
                if (!there[m])
                    continue;
                const float f = scale_of(scale[m]);
                const Scale<kF16> s = scale_pair<kF16>(f, f);
                uint32_t e[8];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t x = i ? code[m].y : code[m].x;
                    uint32_t a[4];  // elements j and j + 4
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        a[j] = dequant_pair<kF16>(x >> (4 * j), s);
                    e[4 * i] = __byte_perm(a[0], a[1], 0x5410), e[4 * i + 1] = __byte_perm(a[2], a[3], 0x5410);
                    e[4 * i + 2] = __byte_perm(a[0], a[1], 0x7632), e[4 * i + 3] = __byte_perm(a[2], a[3], 0x7632);
                }
                uint16_t *dst = out + (long long)(r0 + m * abreast) * to.row_stride;
                if ((reinterpret_cast<uintptr_t>(dst) & 31) == 0) {
                    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst), "r"(e[0]), "r"(e[1]),
                                 "r"(e[2]), "r"(e[3]), "r"(e[4]), "r"(e[5]), "r"(e[6]), "r"(e[7])
                                 : "memory");
                } else {
                    reinterpret_cast<uint4 *>(dst)[0] = make_uint4(e[0], e[1], e[2], e[3]);
                    reinterpret_cast<uint4 *>(dst)[1] = make_uint4(e[4], e[5], e[6], e[7]);
                }
            }
        }
    }
}

tb_status check_norm(const tb_head_norm *norm, const char *fn)
{
    if (!norm)
        return TB_OK;
    if (!ptr_aligned(norm->q_weight, 16) || !ptr_aligned(norm->k_weight, 16))
        return record_error(TB_EINVAL, "%s: norm weights must be 16-byte aligned", fn);
    if (!(norm->eps >= 0.f) || !std::isfinite(norm->eps) || !std::isfinite(norm->weight_offset))
        return record_error(TB_EINVAL, "%s: norm eps %g, weight_offset %g", fn, norm->eps, norm->weight_offset);
    return TB_OK;
}

// What both stores do once their pages are checked and put into `a`.
tb_status store_rows(RowsArgs &a, bool q4, int layer, int n_layers, int n_kv_heads, int page_size, int d, int dtype,
                     const int64_t *slots, int n_rows, const tb_rows *k, const tb_rows *v, const tb_rows *q,
                     const tb_rows *q_out, int n_q_heads, const tb_head_norm *norm, const tb_rope *rope,
                     cudaStream_t stream, const char *fn)
{
    tb_status st = check_store(layer, n_layers, slots, n_rows, k, v, q, q_out, n_q_heads, fn);
    if (st != TB_OK || (st = check_norm(norm, fn)) != TB_OK)
        return st;
    if (n_kv_heads > 1 << 20)
        return record_error(TB_EUNSUPPORTED, "%s: %d kv heads", fn, n_kv_heads);
    const bool has_q = q && q->ptr;
    a.turn = rope && rope->theta != 0.f;
    if (a.turn && (st = rope_axes(rope, d, n_rows, &a.rope, fn)) != TB_OK)
        return st;
    if (n_rows == 0)
        return launch_result(cudaSuccess, fn);
    const int n_sm = device_sms(-1);
    if (n_sm <= 0)
        return record_error(TB_ECUDA, "%s: no current device", fn);
    while ((1 << a.page_log2) < page_size)
        ++a.page_log2;
    a.Hkv = n_kv_heads;
    a.Hq = has_q ? n_q_heads : 0;
    a.n_rows = n_rows;
    a.slots = slots;
    a.k = rows_of(k);
    a.v = rows_of(v);
    if (has_q) {
        a.q = rows_of(q);
        a.q_out = rows_of(q_out);
    }
    if (norm) {
        a.q_weight = has_q ? static_cast<const uint16_t *>(norm->q_weight) : nullptr;
        a.k_weight = static_cast<const uint16_t *>(norm->k_weight);
        a.eps = norm->eps;
        a.weight_offset = norm->weight_offset;
    }
    // The rows of a CTA: all CTAs that the SMs hold at once have as many, or in several rounds, kMaxRows at most.
    const auto rows_for = [&](int threads) {
        const long long slots = (long long)(kCtas * kThreads / threads) * n_sm, rounds = (n_rows - 1) / (kMaxRows * slots) + 1;
        return (int)((n_rows - 1) / (rounds * slots)) + 1;
    };
    // Fewer threads than kThreads, if a row's places (or whole rows) fill them and not kThreads, where CTAs have one
    // row or get fewer.  With 384 places 192 threads: 358 rows 5.3 us (6.2 with 256), 700 rows 6.8 (8.6), 4000
    // rows 24.6 (26.0); where both have as many rows, 1000 rows 9.6 (8.9), 2400 rows 16.6 (14.8).
    const int per_row = (a.Hq + 2 * a.Hkv) * (d / 16);
    const auto fills = [&](int t) { return per_row % t == 0 || t % per_row == 0; };
    int threads = kThreads;
    for (int t = kThreads - 32; t >= kThreads / 2 && !fills(threads); t -= 32)
        if (fills(t) && (rows_for(t) == 1 || rows_for(t) < rows_for(kThreads)))
            threads = t;
    a.rows_per_cta = rows_for(threads);
    using Kernel = void (*)(RowsArgs);
    static const Kernel kernels[2][2][2] = {
        {{k_paged_rows<64, false, false>, k_paged_rows<64, false, true>},
         {k_paged_rows<64, true, false>, k_paged_rows<64, true, true>}},
        {{k_paged_rows<128, false, false>, k_paged_rows<128, false, true>},
         {k_paged_rows<128, true, false>, k_paged_rows<128, true, true>}}};
    const int grid = (n_rows - 1) / a.rows_per_cta + 1;
    return launch_result(launch_kernel(kernels[d == 128][dtype == TB_F16][q4], dim3(grid), dim3(threads), 0, stream,
                                       true, a),
                         fn);
}

}  // namespace

TB_BOUNDS_COUNTER(bounds_violations_paged_rows)

tb_status check_pages_q4(const tb_pages_q4 *pages, const char *fn)
{
    if (!pages || !pages->k || !pages->v)
        return record_error(TB_EINVAL, "%s: pages, pages->k or pages->v is NULL", fn);
    if (!ptr_aligned(pages->k, 16) || !ptr_aligned(pages->v, 16))
        return record_error(TB_EINVAL, "%s: pages->k / pages->v must be 16-byte aligned", fn);
    if (pages->dtype != TB_BF16 && pages->dtype != TB_F16)
        return record_error(TB_EUNSUPPORTED, "%s: rows of type %d (TB_BF16 or TB_F16)", fn, pages->dtype);
    if (pages->head_dim != 64 && pages->head_dim != 128)
        return record_error(TB_EUNSUPPORTED, "%s: head_dim %d (64 or 128 supported)", fn, pages->head_dim);
    if (pages->n_layers < 1 || pages->n_pages < 1 || pages->n_kv_heads < 1)
        return record_error(TB_EINVAL, "%s: n_layers=%d n_pages=%d n_kv_heads=%d", fn, pages->n_layers, pages->n_pages,
                            pages->n_kv_heads);
    if (pages->page_size < 8 || pages->page_size > 1024 || (pages->page_size & (pages->page_size - 1)))
        return record_error(TB_EINVAL, "%s: page_size %d (a power of two from 8 to 1024)", fn, pages->page_size);
    const int64_t block = (int64_t)pages->page_size * row_bytes(pages->head_dim);
    for (int64_t s : {pages->layer_stride, pages->page_stride, pages->head_stride})
        if (s < 0 || s % 16)
            return record_error(TB_EINVAL, "%s: strides must be multiples of 16 bytes, none negative", fn);
    if ((pages->n_kv_heads > 1 && pages->head_stride < block) || (pages->n_pages > 1 && pages->page_stride < block) ||
        (pages->n_layers > 1 && pages->layer_stride < block))
        return record_error(TB_EINVAL, "%s: layer, page or head stride below a page's %lld bytes", fn, (long long)block);
    return TB_OK;
}

}  // namespace tv

using namespace tv;

extern "C" tb_status paged_kv_store_norm(const tb_pages *pages, int layer, const int64_t *slots, int n_rows,
                                         const tb_rows *k, const tb_rows *v, const tb_rows *q, const tb_rows *q_out,
                                         int n_q_heads, const tb_head_norm *norm, const tb_rope *rope, tb_stream stream)
{
    const char *fn = "paged_kv_store_norm";
    const tb_status st = check_pages(pages, fn);
    if (st != TB_OK)
        return st;
    RowsArgs a{};
    const long long off = 2ll * layer * pages->layer_stride;
    a.k_pages = static_cast<uint8_t *>(pages->k) + off;
    a.v_pages = static_cast<uint8_t *>(pages->v) + off;
    a.page_stride = 2 * pages->page_stride;
    a.head_stride = 2 * pages->head_stride;
    a.slot_stride = 2 * pages->slot_stride;
    a.n_pages = pages->n_pages;
    return store_rows(a, false, layer, pages->n_layers, pages->n_kv_heads, pages->page_size, pages->head_dim,
                      pages->dtype, slots, n_rows, k, v, q, q_out, n_q_heads, norm, rope, (cudaStream_t)stream, fn);
}

extern "C" tb_status paged_kv_store_q4(const tb_pages_q4 *pages, int layer, const int64_t *slots, int n_rows,
                                       const tb_rows *k, const tb_rows *v, const tb_rows *q, const tb_rows *q_out,
                                       int n_q_heads, const tb_head_norm *norm, const tb_rope *rope, tb_stream stream)
{
    const char *fn = "paged_kv_store_q4";
    const tb_status st = check_pages_q4(pages, fn);
    if (st != TB_OK)
        return st;
    RowsArgs a{};
    const long long off = (long long)layer * pages->layer_stride;
    a.k_pages = static_cast<uint8_t *>(pages->k) + off;
    a.v_pages = static_cast<uint8_t *>(pages->v) + off;
    a.page_stride = pages->page_stride;
    a.head_stride = pages->head_stride;
    a.n_pages = pages->n_pages;
    return store_rows(a, true, layer, pages->n_layers, pages->n_kv_heads, pages->page_size, pages->head_dim,
                      pages->dtype, slots, n_rows, k, v, q, q_out, n_q_heads, norm, rope, (cudaStream_t)stream, fn);
}

extern "C" tb_status paged_kv_load_q4(const tb_pages_q4 *pages, int layer, int n_layers, const int64_t *slots,
                                      int n_rows, const tb_rows *k, const tb_rows *v, int64_t row_layer_stride,
                                      tb_stream stream)
{
    const char *fn = "paged_kv_load_q4";
    tb_status st = check_pages_q4(pages, fn);
    if (st != TB_OK)
        return st;
    if (layer < 0 || n_layers < 1 || n_layers > pages->n_layers - layer)
        return record_error(TB_EINVAL, "%s: layers %d to %d of %d", fn, layer, layer + n_layers, pages->n_layers);
    if (n_layers > 65535)
        return record_error(TB_EUNSUPPORTED, "%s: %d layers", fn, n_layers);
    if (n_rows < 0 || (n_rows > 0 && !slots))
        return record_error(TB_EINVAL, "%s: n_rows %d, or slots is NULL", fn, n_rows);
    if (n_rows > 0 && ((st = check_rows(k, "k", fn)) != TB_OK || (st = check_rows(v, "v", fn)) != TB_OK))
        return st;
    if (n_rows > 1 << 30 || pages->n_kv_heads > 1 << 20)
        return record_error(TB_EUNSUPPORTED, "%s: %d rows of %d kv heads", fn, n_rows, pages->n_kv_heads);
    if (row_layer_stride % 8)
        return record_error(TB_EINVAL, "%s: row_layer_stride must be a multiple of 8 elements", fn);
    if (n_rows == 0)
        return launch_result(cudaSuccess, fn);
    const int n_sm = device_sms(-1);
    if (n_sm <= 0)
        return record_error(TB_ECUDA, "%s: no current device", fn);
    LoadArgs a{};
    const long long off = (long long)layer * pages->layer_stride;
    a.k_pages = static_cast<const uint8_t *>(pages->k) + off;
    a.v_pages = static_cast<const uint8_t *>(pages->v) + off;
    a.layer_stride = pages->layer_stride;
    a.page_stride = pages->page_stride;
    a.head_stride = pages->head_stride;
    a.n_pages = pages->n_pages;
    while ((1 << a.page_log2) < pages->page_size)
        ++a.page_log2;
    a.Hkv = pages->n_kv_heads;
    a.n_rows = n_rows;
    a.slots = slots;
    a.k = rows_of(k);
    a.v = rows_of(v);
    a.row_layer_stride = row_layer_stride;
    // kLoadAhead rows per thread, fewer rows per CTA where that would leave SMs without one, more where it would
    // make more than 64 CTAs for each
    const long long per_row = 2ll * a.Hkv * (pages->head_dim / kLoadCodes), abreast = per_row < kThreads ? kThreads / per_row : 1;
    long long rows = kLoadAhead * abreast;
    while (rows > abreast && (n_rows + rows - 1) / rows * n_layers < 2 * n_sm)
        rows -= abreast;
    while ((n_rows + rows - 1) / rows * n_layers > 64ll * n_sm && rows < n_rows)
        rows *= 2;
    const dim3 grid((unsigned)((n_rows + rows - 1) / rows), n_layers);
    const bool f16 = pages->dtype == TB_F16;
    const auto kernel = pages->head_dim == 64 ? (f16 ? k_paged_load<64, true> : k_paged_load<64, false>)
                                              : (f16 ? k_paged_load<128, true> : k_paged_load<128, false>);
    return launch_result(launch_kernel(kernel, grid, dim3(kThreads), 0, (cudaStream_t)stream, true, a, (int)rows),
                         fn);
}
