// paged_store.cu -- rotary embedding with several position axes, and keys and
// values into their pages.
//
// Pair i of a head, (x_i, x_{i + d/2}), turns by the angle pos * theta^(-2i/d),
// pos taken from the axis that owns pair i.  Only the fraction of a turn
// matters, so the frequency in turns, theta^(-2i/d) / (2 pi) < 1, is held as a
// 64-bit fixed-point fraction and pos * frequency is one 64-bit integer product,
// whose overflow is the whole turns: the fraction is as right as the frequency,
// to pos * 2^-65 of a turn where the host's long double has 113 bits (Arm), and
// to pos * 2^-62 where it has 64 (2^-64 for theta of 100 and more), where a
// 32-bit float product loses it after a few thousand turns.
//
// A CTA takes a few rows: their (cos, sin) once into shared memory (they serve
// all heads), then every (row, head, 16-byte piece of the lower half of the head
// and its partner in the upper half).
#include "paged.cuh"

#include <cuda_fp16.h>

#include <cmath>

namespace tv {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxRows = 8;  // rows per CTA

struct StoreArgs {
    uint16_t *k_pages, *v_pages;  // of the layer
    long long page_stride, head_stride, slot_stride;
    int n_pages, page_log2, Hkv, Hq, n_rows, d_log2, rows_per_cta;
    const int64_t *slots;
    Rows k, v, q, q_out;
    RopeAxes rope;
};

// kRope: queries and keys turn.  Bound by HBM: each element is read once and
// written once.  8191 rows of a prompt, 32 heads of 128 (403 MB): 65.7 us, 6.13 TB/s,
// 90 % of a copy's bandwidth, with two items per thread in flight (69.4 with one); a
// step's few hundred rows (8.9 MB): 3.4 us, a launch and one round trip.
template <bool kF16, bool kRope>
__global__ void __launch_bounds__(kThreads) k_paged_store(const __grid_constant__ StoreArgs p)
{
    __shared__ float2 s_cs[kMaxRows][kRopeMaxHalf];
    __shared__ long long s_slot[kMaxRows];
    pdl_wait();
    pdl_trigger();
    const int r0 = blockIdx.x * p.rows_per_cta, n_rows = min(p.rows_per_cta, p.n_rows - r0);
    const int half_log2 = p.d_log2 - 1, half = 1 << half_log2;
    for (int x = threadIdx.x; x < n_rows; x += kThreads)
        s_slot[x] = p.slots[r0 + x];
    if constexpr (kRope) {
        for (int x = threadIdx.x; x < n_rows << half_log2; x += kThreads) {
            const int r = x >> half_log2, i = x & (half - 1);
            // the fraction of a turn in [-1/2, 1/2), as an angle in units of pi
            const int turn = (int)(turn_of(p.rope, r0 + r, i) >> 32);
            float2 cs;
            sincospif((float)turn * 0x1p-31f, &cs.y, &cs.x);
            s_cs[r][i] = cs;
        }
    }
    __syncthreads();
    // items: a 16-byte piece of the lower half of a head and its partner; queries, keys,
    // values; kAhead of them in flight per thread
    constexpr int kAhead = 2;
    const int pc_log2 = half_log2 - 3, heads = p.Hq + 2 * p.Hkv;
    const unsigned per_row = (unsigned)heads << pc_log2, items = n_rows * per_row;
    for (unsigned x0 = threadIdx.x; x0 < items; x0 += kAhead * kThreads) {
        uint4 lo[kAhead], hi[kAhead];
        uint16_t *dst[kAhead];
        const float2 *turn[kAhead];
#pragma unroll
        for (int m = 0; m < kAhead; ++m) {
            const unsigned x = x0 + m * kThreads;
            dst[m] = nullptr;
            turn[m] = nullptr;
            if (x >= items)
                continue;
            const unsigned r = x / per_row, y = x - r * per_row;
            int h = (int)(y >> pc_log2);
            const int c = (int)(y & ((1u << pc_log2) - 1)) * 8;
            const long long row = r0 + r;
            const uint16_t *src;
            if (h < p.Hq) {
                src = p.q.p + row * p.q.row_stride + h * p.q.head_stride;
                dst[m] = p.q_out.p + row * p.q_out.row_stride + h * p.q_out.head_stride + c;
                turn[m] = &s_cs[r][c];
            } else {
                h -= p.Hq;
                const bool is_v = h >= p.Hkv;
                h -= is_v ? p.Hkv : 0;
                const long long slot = s_slot[r], page = slot >> p.page_log2;
                if (slot < 0 || page >= p.n_pages)
                    continue;  // padding
                const Rows &in = is_v ? p.v : p.k;
                src = in.p + row * in.row_stride + h * in.head_stride;
                dst[m] = (is_v ? p.v_pages : p.k_pages) + page * p.page_stride + h * p.head_stride +
                         (slot & ((1 << p.page_log2) - 1)) * p.slot_stride + c;
                turn[m] = is_v ? nullptr : &s_cs[r][c];
            }
            lo[m] = *reinterpret_cast<const uint4 *>(src + c);
            hi[m] = *reinterpret_cast<const uint4 *>(src + c + half);
        }
#pragma unroll
        for (int m = 0; m < kAhead; ++m) {
            if (!dst[m])
                continue;
            if (kRope && turn[m]) {
                uint32_t *a = &lo[m].x, *b = &hi[m].x;
                const float2 *cs = turn[m];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 t0 = cs[2 * e], t1 = cs[2 * e + 1];
                    const float2 u = unpack_pair<kF16>(a[e]), w = unpack_pair<kF16>(b[e]);
                    a[e] = pack_pair<kF16>(u.x * t0.x - w.x * t0.y, u.y * t1.x - w.y * t1.y);
                    b[e] = pack_pair<kF16>(w.x * t0.x + u.x * t0.y, w.y * t1.x + u.y * t1.y);
                }
            }
            *reinterpret_cast<uint4 *>(dst[m]) = lo[m];
            *reinterpret_cast<uint4 *>(dst[m] + half) = hi[m];
        }
    }
}

using u128 = unsigned __int128;

// The upper half of a 128 x 128 bit product: the product of two fractions of 2^128.
u128 mul_fraction(u128 a, u128 b)
{
    const uint64_t a1 = (uint64_t)(a >> 64), a0 = (uint64_t)a, b1 = (uint64_t)(b >> 64), b0 = (uint64_t)b;
    const u128 mid = (u128)a1 * b0 + (((u128)a0 * b0) >> 64);
    const u128 mid2 = (u128)a0 * b1 + (uint64_t)mid;
    return (u128)a1 * b1 + (mid >> 64) + (mid2 >> 64);
}

u128 fraction_of(long double x)  // 0 <= x < 1
{
    const long double two64 = 18446744073709551616.0L;
    const long double y = x * two64;
    const uint64_t hi = (uint64_t)y;
    return ((u128)hi << 64) | (uint64_t)((y - (long double)hi) * two64);
}

// freq[i] = theta^(-2i/d) / (2 pi) as a fraction of 2^64, a geometric series in
// 128 bits whose ratio r = theta^(-2/d) is Newton's step on r^(d/2) = 1 / theta
// from its double value, in long double: half a unit of 2^-64 off where that has
// 113 bits; with 64 bits up to 0.8 units for theta of 100 and more, 3.1 at theta 2,
// since the ratio's error grows with i (64 calls of a long-double pow took 90 us a call on the
// GB300's host).
void turns(double theta, int d, uint64_t *freq)
{
    const int half = d / 2;
    u128 f = fraction_of(0.159154943091895335768883763372514362L);  // 1 / (2 pi)
    const double r0 = pow(theta, -2.0 / d);
    long double power = r0;
    for (int k = 1; k < half; k *= 2)  // half is a power of two
        power *= power;
    const long double r = r0 * (1.0L + (1.0L / ((long double)theta * power) - 1.0L) / half);
    const u128 ratio = r < 1.0L ? fraction_of(r) : ~(u128)0;
    for (int i = 0; i < half; ++i, f = mul_fraction(f, ratio))
        freq[i] = (uint64_t)(f >> 64) + (uint64_t)((f >> 63) & 1);
}

}  // namespace

tb_status check_rows(const tb_rows *r, const char *what, const char *fn)
{
    if (!r || !r->ptr || !ptr_aligned(r->ptr, 16))
        return record_error(TB_EINVAL, "%s: %s NULL or not 16-byte aligned", fn, what);
    if (r->row_stride % 8 || r->head_stride % 8)
        return record_error(TB_EINVAL, "%s: strides of %s must be multiples of 8 elements", fn, what);
    return TB_OK;
}

tb_status check_store(int layer, int n_layers, const int64_t *slots, int n_rows, const tb_rows *k, const tb_rows *v,
                      const tb_rows *q, const tb_rows *q_out, int n_q_heads, const char *fn)
{
    if (layer < 0 || layer >= n_layers)
        return record_error(TB_EINVAL, "%s: layer %d of %d", fn, layer, n_layers);
    if (n_rows < 0 || (n_rows > 0 && !slots))
        return record_error(TB_EINVAL, "%s: n_rows %d, or slots is NULL", fn, n_rows);
    const bool has_q = q && q->ptr;
    tb_status st;
    if (n_rows > 0 && ((st = check_rows(k, "k", fn)) != TB_OK || (st = check_rows(v, "v", fn)) != TB_OK))
        return st;
    if (n_rows > 0 && has_q && ((st = check_rows(q, "q", fn)) != TB_OK || (st = check_rows(q_out, "q_out", fn)) != TB_OK))
        return st;
    if (has_q && (n_q_heads < 1 || n_q_heads > 65536))
        return record_error(TB_EINVAL, "%s: n_q_heads %d", fn, n_q_heads);
    return TB_OK;
}

tb_status rope_axes(const tb_rope *rope, int d, int n_rows, RopeAxes *a, const char *fn)
{
    if (!(rope->theta >= 1.f) || !std::isfinite(rope->theta))
        return record_error(TB_EINVAL, "%s: rope theta %g (1 or more)", fn, rope->theta);
    if (rope->n_axes < 1 || rope->n_axes > kMaxAxes || (n_rows > 0 && !rope->positions) || rope->axis_stride < 0 ||
        (rope->n_axes > 1 && rope->axis_stride < n_rows))
        return record_error(TB_EINVAL, "%s: %d axes, positions NULL or axis_stride %lld below n_rows", fn, rope->n_axes,
                            (long long)rope->axis_stride);
    int end = 0;
    for (int x = 0; x < kMaxAxes; ++x) {
        if (x < rope->n_axes && (rope->sections[x] < 0 || rope->sections[x] > d / 2))
            return record_error(TB_EINVAL, "%s: section %d of %d pairs", fn, x, rope->sections[x]);
        end += x < rope->n_axes ? rope->sections[x] : 0;
        a->axis_end[x] = x < rope->n_axes - 1 ? end : d;
    }
    if (end != d / 2)
        return record_error(TB_EINVAL, "%s: the sections have %d pairs, a head %d", fn, end, d / 2);
    turns((double)rope->theta, d, a->freq);
    a->pos = rope->positions;
    a->axis_stride = rope->axis_stride;
    return TB_OK;
}

TB_BOUNDS_COUNTER(bounds_violations_paged_store)

}  // namespace tv

using namespace tv;

extern "C" tb_status paged_kv_store(const tb_pages *pages, int layer, const int64_t *slots, int n_rows,
                                    const tb_rows *k, const tb_rows *v, const tb_rows *q, const tb_rows *q_out,
                                    int n_q_heads, const tb_rope *rope, tb_stream stream)
{
    const char *fn = "paged_kv_store";
    tb_status st = check_pages(pages, fn);
    if (st != TB_OK)
        return st;
    if ((st = check_store(layer, pages->n_layers, slots, n_rows, k, v, q, q_out, n_q_heads, fn)) != TB_OK)
        return st;
    const bool has_q = q && q->ptr;
    StoreArgs a{};
    const bool turn = rope && rope->theta != 0.f;
    const int d = pages->head_dim;
    if (turn && (st = rope_axes(rope, d, n_rows, &a.rope, fn)) != TB_OK)
        return st;
    if (n_rows == 0)
        return launch_result(cudaSuccess, fn);
    const int n_sm = device_sms(-1);
    if (n_sm <= 0)
        return record_error(TB_ECUDA, "%s: no current device", fn);
    a.k_pages = static_cast<uint16_t *>(pages->k) + (long long)layer * pages->layer_stride;
    a.v_pages = static_cast<uint16_t *>(pages->v) + (long long)layer * pages->layer_stride;
    a.page_stride = pages->page_stride;
    a.head_stride = pages->head_stride;
    a.slot_stride = pages->slot_stride;
    a.n_pages = pages->n_pages;
    while ((1 << a.page_log2) < pages->page_size)
        ++a.page_log2;
    a.d_log2 = d == 64 ? 6 : 7;
    a.Hkv = pages->n_kv_heads;
    a.Hq = has_q ? n_q_heads : 0;
    a.n_rows = n_rows;
    a.slots = slots;
    a.k = rows_of(k);
    a.v = rows_of(v);
    if (has_q) {
        a.q = rows_of(q);
        a.q_out = rows_of(q_out);
    }
    // one row per CTA while there are SMs for more, up to kMaxRows of them otherwise
    const int per = n_rows / (8 * n_sm);
    a.rows_per_cta = per < 1 ? 1 : per > kMaxRows ? kMaxRows : per;
    const bool f16 = pages->dtype == TB_F16;
    const auto kernel = f16 ? (turn ? k_paged_store<true, true> : k_paged_store<true, false>)
                            : (turn ? k_paged_store<false, true> : k_paged_store<false, false>);
    const int grid = (n_rows + a.rows_per_cta - 1) / a.rows_per_cta;
    return launch_result(launch_kernel(kernel, dim3(grid), dim3(kThreads), 0, (cudaStream_t)stream, true, a), fn);
}
