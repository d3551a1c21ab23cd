// paged_attention_few.cuh -- the attention over 4-bit pages for units of up to 16
// query rows per kv head: single tokens, chains and small trees of drafts.
//
// With so few rows the bytes bound, and a score tile of 128 rows would be work for
// rows that are not there.  So keys lie on the rows of the products here and
// queries on their columns (8 or 16), in registers:
//   S^T = K Q^T   16 keys x 8 queries x 16 elements per mma
//   O^T += V^T P^T   16 elements x 8 queries x 16 keys
// Any order of the summed index will do, as long as both operands have it.  For
// S^T a thread's share of a k step are elements of one 16-byte piece of its key's
// row (32 codes under one scale), the queries staged to match; for V^T it takes four
// keys' codes of 8 or 16 neighbouring elements, two keys at a time in the halves of a
// word.  Codes become 16-bit operands in registers and never go back to
// shared memory.  P moves from the layout of a result (keys by queries) to that of an
// operand by an 8 x 8 transpose in the warp.
//
// Each warp walks its own pieces of 32 keys (every 16th of the CTA's), copied whole
// from the pages into a ring of its own, with its own maxima, sums and output;
// at a unit's end the CTA adds the 16 of them up, in a fixed order.
#pragma once

namespace tv {

namespace {

constexpr int kFewRows = 16;
constexpr int kFewKeys = 32;  // of a piece
constexpr int kFewSegs = 64;  // units laid out at a time
constexpr int kFewWarps = kThreads / 32;

constexpr int few_stages(int d)
{
    return d == 64 ? 4 : 2;
}

// A run of tiles of one unit.
struct FewSeg {
    int first, end;  // its pieces, from the CTA's first tile on
    int head, j0, whole;
    PlanReq r;
};

// A query row of a unit.
struct FewRow {
    uint64_t anc, path;
    long long out;  // (row, query head); -1: none
    int lo, pos;
    float slope;
    int pad;
};

template <int kD>
struct FewSmem {
    static constexpr int kStage = 2 * kFewKeys * row_bytes(kD), kRing = few_stages(kD) * kStage;
    static constexpr int kQueryRow = 2 * kD + 16;  // bytes: rows begin in different banks
    uint8_t ring[kFewWarps][kRing];
    float4 sum[8][2 * kD / 16][32];       // O^T of 8 warps, fragment by fragment
    uint8_t query[2][kFewRows * kQueryRow];  // of this unit and of the next
    FewRow row[2][kFewRows];
    float m[kFewWarps][kFewRows], l[kFewWarps][kFewRows];
    FewSeg seg[kFewSegs];
    uint32_t holes[kFewWarps][few_stages(kD)];
    uint64_t full[kFewWarps][few_stages(kD)];
    int n_segs;
};

template <bool kF16>
__device__ __forceinline__ void mma_16x8x16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                            uint32_t b0, uint32_t b1)
{
    if constexpr (kF16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                     "{%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                     "{%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x)
{
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// kN: columns of 8 queries.
template <int kD, bool kF16, int kForm, int kN>
__device__ __forceinline__ void few_rows(const PagedArgs &p, const PlanCta &cta, FewSmem<kD> &sm, int *abort_flag,
                                         uint64_t *never_bar)
{
    constexpr int kStages = few_stages(kD), kSlot = slot_floats(kD), kTilesD = kD / 16;
    constexpr float kShift = kF16 ? 8.f : 0.f, kGrow = kF16 ? 7.f : 8.f;  // as for many rows
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const PlanReq *reqs = plan_reqs(p.plan);
    const int window = static_cast<const PlanHeader *>(p.plan)->window;
    const long long t0 = cta.t0, t1 = cta.t1;
    uint8_t *ring = sm.ring[warp];

    // ---- a warp's copies: lane (kind, piece) copies K's or V's part of a piece of min(page_size, 32) keys, with
    // larger pages its codes or its scales
    const int part_log2 = min(p.page_log2, 5);
    const bool split = p.page_log2 > 5;
    const int parts = split ? 2 : kFewKeys >> part_log2;
    const bool copies = lane < 2 * parts, copies_v = lane >= parts;
    const int part = copies_v ? lane - parts : lane, part_key = split ? 0 : part << part_log2;
    struct Fetch {
        int id, key0, head;
        bool inside;
    };
    auto seg_key = [&](const FewSeg &s, int piece) {
        return tile_key(s.j0 + ((piece - s.first) >> 2), s.r.a0, s.r.n1, s.r.b0) + ((piece & 3) * kFewKeys);
    };
    int ahead_seg = 0, issued = 0, taken = 0;
    auto fetch = [&](int piece) {
        while (piece >= sm.seg[ahead_seg].end)
            ++ahead_seg;
        const FewSeg &s = sm.seg[ahead_seg];
        Fetch f{-1, seg_key(s, piece), s.head, false};
        const int slot = f.key0 + part_key, at = slot >> p.page_log2;
        f.inside = copies && slot < s.r.L + s.r.n;
        if (f.inside && at < p.max_pages)
            f.id = p.table[(size_t)s.r.b * p.max_pages + at];
        return f;
    };
    auto report_hole = [&](int slot) {
        const PlanReq &r = sm.seg[ahead_seg].r;
        const int past = slot + (1 << part_log2);
        const int lo_min = window > 0 ? max(r.begin, r.L - window + 1) : r.begin;
        if (past > lo_min || (window > 0 && past > r.begin && slot < min(r.far_end, r.L)))
            atomicOr(p.status, kStatusBounds);
    };
    auto issue = [&](const Fetch &f) {
        const int s = issued % kStages;
        const bool there = f.inside && f.id >= 0 && f.id < p.n_pages;
        const uint32_t holes = __ballot_sync(0xffffffffu, f.inside && !there);
        const uint32_t found = __ballot_sync(0xffffffffu, there);
        if (lane == 0) {
            sm.holes[warp][s] = holes & ((1u << parts) - 1);
            mbar_arrive_expect_tx(&sm.full[warp][s], split ? (found ? 2 * kFewKeys * row_bytes(kD) : 0)
                                                           : (__popc(found) << part_log2) * row_bytes(kD));
        }
        __syncwarp();
        if (there) {
            const uint8_t *src = (copies_v ? p.v_pages : p.k_pages) + f.id * p.page_stride + f.head * p.head_stride;
            uint8_t *dst = ring + s * FewSmem<kD>::kStage + (copies_v ? kFewKeys * row_bytes(kD) : 0);
            if (!split) {
                bulk_load(dst + part_key * row_bytes(kD), src, row_bytes(kD) << part_log2, &sm.full[warp][s]);
            } else {
                const int at = f.key0 & ((1 << p.page_log2) - 1);
                if (part == 0)
                    bulk_load(dst, src + at * code_bytes(kD), kFewKeys * code_bytes(kD), &sm.full[warp][s]);
                else
                    bulk_load(dst + kFewKeys * code_bytes(kD),
                              src + ((long long)code_bytes(kD) << p.page_log2) + at * scale_bytes(kD),
                              kFewKeys * scale_bytes(kD), &sm.full[warp][s]);
            }
        }
        if (f.inside && !there && !copies_v && (!split || part == 0))
            report_hole(f.key0 + part_key);
        ++issued;
    };

    // ---- where this thread's keys and values lie in a piece.  Row i of a product's 16 keys is key i with its
    // lowest two bits swapped, so that the four keys which V's loads take at once lie in different banks.
    const int key_k = (g & 4) | ((g & 1) << 1) | ((g >> 1) & 1), key_v = (t >> 1) * 4 + (t & 1);
    const int per_part = 1 << part_log2;
    const int code8 = part_log2 == 3 ? 8 * row_bytes(kD) : 8 * code_bytes(kD);
    const int code16 = part_log2 == 5 ? 16 * code_bytes(kD) : 16 * row_bytes(kD);
    const int scale8 = part_log2 == 3 ? 8 * row_bytes(kD) : 8 * scale_bytes(kD);
    const int scale16 = part_log2 == 5 ? 16 * scale_bytes(kD) : 16 * row_bytes(kD);
    const int k_code = key_k * code_bytes(kD) + t * (kD / 8);
    const int k_scale = per_part * code_bytes(kD) + key_k * scale_bytes(kD) + t * (kD / 4) / kGroup;
    const int v_code = kFewKeys * row_bytes(kD) + key_v * code_bytes(kD) + g * (kD / 16);
    const int v_scale = kFewKeys * row_bytes(kD) + per_part * code_bytes(kD) + key_v * scale_bytes(kD) +
                        g * (kD / 8) / kGroup;

    if (lane == 0)
        for (int s = 0; s < kStages; ++s)
            mbar_init(&sm.full[warp][s], 1);
    fence_mbar_init();
    __syncwarp();

    // ---- a unit's rows: warp w takes row w, its query and what it sees
    auto stage = [&](const FewSeg &s, int buf) {
        const int row = cta.rb * 128 + warp, node = row / p.group, qh = s.head * p.group + row % p.group;
        bool valid = node < s.r.n && s.r.row0 + node < p.n_rows;
        const bool known = (unsigned)s.r.tree < (unsigned)p.n_trees;
        if (valid && !known)
            atomicOr(p.status, kStatusBounds);
        const TreeDesc &td = p.trees[known ? s.r.tree : 0];
        if (valid && known && td.n != s.r.n)
            atomicOr(p.status, kStatusBounds);
        valid = valid && known && td.n == s.r.n;
        valid = valid && in_bounds(node < kMaxNodes && qh < p.Hq && s.r.row0 >= 0, p.status);
        const size_t at = valid ? (size_t)(s.r.row0 + node) * p.Hq + qh : 0;
        uint32_t *dst = reinterpret_cast<uint32_t *>(sm.query[buf] + warp * FewSmem<kD>::kQueryRow);
        const uint32_t *src = reinterpret_cast<const uint32_t *>(p.q + at * kD);
#pragma unroll
        for (int i = 0; i < kD / 64; ++i)
            dst[lane + 32 * i] = valid ? src[lane + 32 * i] : 0u;
        if (lane == 0) {
            const int L = s.r.L, dep = valid ? td.depth[node] : 0;
            uint64_t anc = valid ? td.anc[node] : 0;
            FewRow &r = sm.row[buf][warp];
            r.path = anc;
            if (window > 0 && dep >= window) {
                // ancestors that the window has left behind
                uint64_t near = 0;
                for (int u = node; u >= 0; u = td.parent[u])
                    if (dep - td.depth[u] < window || L + u < s.r.far_end)
                        near |= 1ull << u;
                anc &= near;
            }
            if (s.r.begin > L)
                anc &= s.r.begin - L < 64 ? ~0ull << (s.r.begin - L) : 0ull;
            r.anc = anc;
            r.out = valid ? (long long)at : -1;
            r.lo = window > 0 ? max(s.r.begin, L + dep - window + 1) : s.r.begin;
            r.pos = L + dep;
            r.slope = kForm == kBias && valid && p.slopes ? p.slopes[qh] * kLog2e : 0.f;
        }
    };

    bool ok = true;
    int unit0 = 0;  // units before this round's
    const int head0 = (int)((t0 - cta.req.tile_base) / cta.req.T);
    for (bool more = true; more; unit0 += kFewSegs) {
        // ---- the next units: those whose tiles begin before t1, in order
        __syncthreads();
        if (threadIdx.x < kFewSegs) {
            const int u = head0 + unit0 + threadIdx.x, i = cta.idx + u / p.Hkv;
            FewSeg s{};
            bool in = i < p.batch;
            if (in) {
                s.r = reqs[i];
                s.head = u % p.Hkv;
                const long long first = s.r.tile_base + (long long)s.head * s.r.T;
                in = first < t1 && s.r.T > 0;
                const long long from = max(first, t0), to = min(first + s.r.T, t1);
                s.j0 = (int)(from - first);
                s.first = 4 * (int)(from - t0);
                s.end = 4 * (int)(to - t0);
                s.whole = to - from == s.r.T;
            }
            // records behind the last request hold anything: only what follows without a gap counts
            const uint32_t all = __ballot_sync(0xffffffffu, in);
            const int n = all == 0xffffffffu ? 32 : __ffs((int)~all) - 1;
            if (lane < n)
                sm.seg[threadIdx.x] = s;
            if (threadIdx.x == 0)
                sm.n_segs = n;
            asm volatile("bar.sync 1, 64;" ::: "memory");
            if (threadIdx.x == 32 && sm.n_segs == 32)
                sm.n_segs = 32 + n;
        }
        __syncthreads();
        const int n_segs = sm.n_segs;
        if (n_segs == 0)
            break;
        const int last = sm.seg[n_segs - 1].end;
        more = last < 4 * (int)(t1 - t0);
        // this warp's pieces of the round: the ring filled, the next page looked up
        int next = sm.seg[0].first + ((warp - sm.seg[0].first) & (kFewWarps - 1));
        int piece = next;
        ahead_seg = 0;
        Fetch ahead{};
        bool has_ahead = next < last;
        if (has_ahead)
            ahead = fetch(next);
        auto refill = [&] {
            issue(ahead);
            next += kFewWarps;
            has_ahead = next < last;
            if (has_ahead)
                ahead = fetch(next);
        };
        for (int s = 0; s < kStages && has_ahead && ok; ++s)
            refill();
        stage(sm.seg[0], 0);
        __syncthreads();

        for (int si = 0; si < n_segs; ++si) {
            const FewSeg &seg = sm.seg[si];
            const int buf = si & 1, L = seg.r.L, end = L + seg.r.n, begin = seg.r.begin;
            const int far = window > 0 ? min(seg.r.far_end, L) : begin;
            const int lo_min = window > 0 ? max(begin, L - window + 1) : begin;
            const int lo_max = window > 0 ? lo_min + kMaxNodes : begin;  // past any row's
            const FewRow *rows = sm.row[buf];
            // queries of columns g (and 8 + g) in the order of the keys' elements
            uint32_t q[kD / 16][kN][2];
#pragma unroll
            for (int n = 0; n < kN; ++n)
#pragma unroll
                for (int i = 0; i < kD / 32; ++i) {
                    const uint4 x = code_order(*reinterpret_cast<const uint4 *>(
                        sm.query[buf] + (8 * n + g) * FewSmem<kD>::kQueryRow + t * (kD / 2) + 16 * i));
                    q[2 * i][n][0] = x.x, q[2 * i][n][1] = x.y;
                    q[2 * i + 1][n][0] = x.z, q[2 * i + 1][n][1] = x.w;
                }
            if (si + 1 < n_segs)
                stage(sm.seg[si + 1], buf ^ 1);
            float o[kTilesD][kN][4] = {};
            float m[kN][2], l[kN][2];  // of columns 8 n + 2 t and the one after it; l: this thread's keys
#pragma unroll
            for (int n = 0; n < kN; ++n)
                m[n][0] = m[n][1] = -INFINITY, l[n][0] = l[n][1] = 0.f;

            for (; piece < seg.end; piece += kFewWarps) {
                const int st = taken % kStages;
                ok = ok && warp_agrees(mbar_wait_bounded(p.expire_wait ? never_bar : &sm.full[warp][st],
                                                         p.expire_wait ? 0u : (uint32_t)(taken / kStages) & 1u, abort_flag,
                                                         p.status));
                if (!ok)
                    continue;
                ++taken;
                const int key0 = seg_key(seg, piece);
                const uint8_t *base = ring + st * FewSmem<kD>::kStage;
                const uint32_t holes = sm.holes[warp][st];
                if (key0 < end) {
                    const bool masked = key0 + kFewKeys > L || key0 < lo_max || holes;
                    // a key's or value's scale: 0 in a hole, of a value also where no row looks
                    auto there = [&](int key) { return !((holes >> (split ? 0 : key >> part_log2)) & 1u); };
                    auto looked_at = [&](int key) {
                        const int slot = key0 + key;
                        return there(key) && slot < end && slot >= begin && (slot >= lo_min || slot < far);
                    };
                    float s[2][kN][4] = {};
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        uint32_t w[2][kD / 32];
                        Scale<kF16> sc[2];
#pragma unroll
                        for (int a = 0; a < 2; ++a) {
                            const uint8_t *c = base + k_code + a * code8 + b * code16;
                            if constexpr (kD == 128) {
                                const uint4 x = *reinterpret_cast<const uint4 *>(c);
                                w[a][0] = x.x, w[a][1] = x.y, w[a][2] = x.z, w[a][3] = x.w;
                            } else {
                                const uint2 x = *reinterpret_cast<const uint2 *>(c);
                                w[a][0] = x.x, w[a][1] = x.y;
                            }
                            float f = scale_of(base[k_scale + a * scale8 + b * scale16]);
                            if (masked)
                                f = there(key_k + 8 * a + 16 * b) ? f : 0.f;
                            sc[a] = scale_pair<kF16>(f, f);
                        }
#pragma unroll
                        for (int i = 0; i < kD / 32; ++i)
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const uint32_t a0 = dequant_pair<kF16>(w[0][i] >> (8 * h), sc[0]);
                                const uint32_t a1 = dequant_pair<kF16>(w[1][i] >> (8 * h), sc[1]);
                                const uint32_t a2 = dequant_pair<kF16>(w[0][i] >> (8 * h + 4), sc[0]);
                                const uint32_t a3 = dequant_pair<kF16>(w[1][i] >> (8 * h + 4), sc[1]);
#pragma unroll
                                for (int n = 0; n < kN; ++n)
                                    mma_16x8x16<kF16>(s[b][n], a0, a1, a2, a3, q[2 * i + h][n][0], q[2 * i + h][n][1]);
                            }
                    }
                    // scores: element c of s[b][n] is key 16 b + 8 (c / 2) + key_k, column 8 n + 2 t + c % 2
                    auto visible = [&](int slot, const FewRow &r) {
                        if (slot < L)
                            return slot >= r.lo || (slot >= begin && slot < far);
                        return slot - L < 64 && ((r.anc >> (slot - L)) & 1);
                    };
                    constexpr float kHidden = kForm == kCap ? INFINITY : -INFINITY;  // z = -inf
                    uint32_t sees = 0xffffffffu;  // bit 8 n + 4 b + c... of this thread's scores
                    if (masked) {
                        sees = 0;
#pragma unroll
                        for (int n = 0; n < kN; ++n)
#pragma unroll
                            for (int b = 0; b < 2; ++b)
#pragma unroll
                                for (int c = 0; c < 4; ++c)
                                    if (visible(key0 + 16 * b + 8 * (c >> 1) + key_k, rows[8 * n + 2 * t + (c & 1)]))
                                        sees |= 1u << (8 * n + 4 * b + c);
                    }
                    if constexpr (kForm != kPlain) {
                        if (kForm == kCap || p.cap > 0.f) {
                            // four of one row together: what is not a number there makes that row none anyway,
                            // unless it is hidden
#pragma unroll
                            for (int n = 0; n < kN; ++n)
#pragma unroll
                                for (int c = 0; c < 2; ++c) {
                                    uint32_t r[4];
#pragma unroll
                                    for (int i = 0; i < 4; ++i) {
                                        const int b = i >> 1, e = c + 2 * (i & 1);
                                        r[i] = (sees >> (8 * n + 4 * b + e)) & 1u ? __float_as_uint(s[b][n][e]) : 0xff800000u;
                                    }
                                    cap_four(r, p.cap_in);
#pragma unroll
                                    for (int i = 0; i < 4; ++i)
                                        s[i >> 1][n][c + 2 * (i & 1)] =
                                            kForm == kCap ? __uint_as_float(r[i])
                                                          : fmaf(-2.f * p.cap, __uint_as_float(r[i]), p.cap);
                                }
                        } else {
#pragma unroll
                            for (int n = 0; n < kN; ++n)
#pragma unroll
                                for (int c = 0; c < 8; ++c)
                                    s[c >> 2][n][c & 3] *= p.scale;
                        }
                    }
#pragma unroll
                    for (int n = 0; n < kN; ++n)
#pragma unroll
                        for (int b = 0; b < 2; ++b) {
                            float(&z)[4] = s[b][n];
                            if constexpr (kForm == kBias) {
#pragma unroll
                                for (int c = 0; c < 4; ++c) {
                                    const FewRow &r = rows[8 * n + 2 * t + (c & 1)];
                                    const int slot = key0 + 16 * b + 8 * (c >> 1) + key_k;
                                    // in the tree: one step for each node of the row's root path before this one
                                    const int dist =
                                        slot <= L ? r.pos - slot
                                                  : r.pos - L - (slot - L < 64 ? __popcll(r.path & ((1ull << (slot - L)) - 1))
                                                                               : __popcll(r.path));
                                    z[c] = fmaf(-r.slope, (float)dist, z[c]);
                                }
                            }
                            if (masked) {
#pragma unroll
                                for (int c = 0; c < 4; ++c)
                                    z[c] = (sees >> (8 * n + 4 * b + c)) & 1u ? z[c] : kHidden;
                            }
                        }
                    // z = f s + f0; f < 0 where s is a capped score's w
                    const float f = kForm == kCap ? -2.f * p.cap : kForm == kPlain ? p.scale : 1.f;
                    const float f0 = kForm == kCap ? p.cap : 0.f;
                    float alpha[kN][2];
                    bool raise = false;
#pragma unroll
                    for (int n = 0; n < kN; ++n)
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            float mx;
                            if constexpr (kForm == kCap) {
                                mx = fminf(fminf(s[0][n][c], s[0][n][c + 2]), fminf(s[1][n][c], s[1][n][c + 2]));
#pragma unroll
                                for (int x = 4; x < 32; x *= 2)
                                    mx = fminf(mx, __shfl_xor_sync(0xffffffffu, mx, x));
                            } else {
                                mx = fmaxf(fmaxf(s[0][n][c], s[0][n][c + 2]), fmaxf(s[1][n][c], s[1][n][c + 2]));
#pragma unroll
                                for (int x = 4; x < 32; x *= 2)
                                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, x));
                            }
                            mx = fmaf(f, mx, f0);
                            alpha[n][c] = 1.f;
                            if (mx > m[n][c] + kShift + kGrow) {
                                alpha[n][c] = m[n][c] == -INFINITY ? 0.f : ex2_approx(m[n][c] - (mx - kShift));
                                m[n][c] = mx - kShift;
                                raise = true;
                            }
                        }
                    if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
                        for (int n = 0; n < kN; ++n) {
                            l[n][0] *= alpha[n][0], l[n][1] *= alpha[n][1];
#pragma unroll
                            for (int j = 0; j < kTilesD; ++j)
#pragma unroll
                                for (int c = 0; c < 4; ++c)
                                    o[j][n][c] *= alpha[n][c & 1];
                        }
                    }
                    uint32_t w[2][kN][2];  // P^T as an operand
#pragma unroll
                    for (int n = 0; n < kN; ++n) {
                        const float mu0 = f0 - (m[n][0] == -INFINITY ? 0.f : m[n][0]);
                        const float mu1 = f0 - (m[n][1] == -INFINITY ? 0.f : m[n][1]);
#pragma unroll
                        for (int b = 0; b < 2; ++b)
#pragma unroll
                            for (int a = 0; a < 2; ++a) {
                                const float p0 = ex2_approx(fmaf(f, s[b][n][2 * a], mu0));
                                const float p1 = ex2_approx(fmaf(f, s[b][n][2 * a + 1], mu1));
                                l[n][0] += p0, l[n][1] += p1;
                                w[b][n][a] = transpose_8x8(pack<kF16>(p0, p1));
                            }
                    }
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        uint32_t v[2][2][kD / 64];  // [keys 0-7, 8-15][first key, second][8 codes each]
                        Scale<kF16> sc[2];
#pragma unroll
                        for (int a = 0; a < 2; ++a) {
                            float f[2];
#pragma unroll
                            for (int x = 0; x < 2; ++x) {
                                const uint8_t *c = base + v_code + 2 * x * code_bytes(kD) + a * code8 + b * code16;
                                if constexpr (kD == 128) {
                                    const uint2 y = *reinterpret_cast<const uint2 *>(c);
                                    v[a][x][0] = y.x, v[a][x][1] = y.y;
                                } else {
                                    v[a][x][0] = *reinterpret_cast<const uint32_t *>(c);
                                }
                                f[x] = scale_of(base[v_scale + 2 * x * scale_bytes(kD) + a * scale8 + b * scale16]);
                                if (masked)
                                    f[x] = looked_at(key_v + 2 * x + 8 * a + 16 * b) ? f[x] : 0.f;
                            }
                            sc[a] = scale_pair<kF16>(f[0], f[1]);
                        }
#pragma unroll
                        for (int i = 0; i < kD / 64; ++i)
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                // four elements of two keys
                                const uint32_t sel = h ? 0x7632 : 0x5410;
                                const uint32_t u0 = __byte_perm(v[0][0][i], v[0][1][i], sel);
                                const uint32_t u1 = __byte_perm(v[1][0][i], v[1][1][i], sel);
#pragma unroll
                                for (int x = 0; x < 2; ++x) {
                                    const uint32_t a0 = dequant_pair<kF16>(u0 >> (8 * x), sc[0]);
                                    const uint32_t a1 = dequant_pair<kF16>(u0 >> (8 * x + 4), sc[0]);
                                    const uint32_t a2 = dequant_pair<kF16>(u1 >> (8 * x), sc[1]);
                                    const uint32_t a3 = dequant_pair<kF16>(u1 >> (8 * x + 4), sc[1]);
#pragma unroll
                                    for (int n = 0; n < kN; ++n)
                                        mma_16x8x16<kF16>(o[4 * i + 2 * h + x][n], a0, a1, a2, a3, w[b][n][0], w[b][n][1]);
                                }
                            }
                    }
                }
                __syncwarp();
                if (has_ahead)
                    refill();
            }

            // ---- the unit's end: 16 warps' maxima, sums and outputs, added up in their order
#pragma unroll
            for (int n = 0; n < kN; ++n)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
#pragma unroll
                    for (int x = 4; x < 32; x *= 2)
                        l[n][c] += __shfl_xor_sync(0xffffffffu, l[n][c], x);
                    if (g == 0) {
                        sm.m[warp][8 * n + 2 * t + c] = m[n][c];
                        sm.l[warp][8 * n + 2 * t + c] = l[n][c];
                    }
                }
            __syncthreads();
            const bool stop = *const_cast<volatile int *>(abort_flag) != 0;  // (nobody waits until the next unit)
            float M[kN][2], sum[kN][2];
#pragma unroll
            for (int n = 0; n < kN; ++n)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int col = 8 * n + 2 * t + c;
                    float x = -INFINITY, y = 0.f;
#pragma unroll
                    for (int k = 0; k < kFewWarps; ++k)
                        x = fmaxf(x, sm.m[k][col]);
#pragma unroll
                    for (int k = 0; k < kFewWarps; ++k)
                        y += (sm.m[k][col] == -INFINITY ? 0.f : ex2_approx(sm.m[k][col] - x)) * sm.l[k][col];
                    const float scale = m[n][c] == -INFINITY ? 0.f : ex2_approx(m[n][c] - x);
                    M[n][c] = x;
                    sum[n][c] = y;
#pragma unroll
                    for (int j = 0; j < kTilesD; ++j)
                        o[j][n][c] *= scale, o[j][n][c + 2] *= scale;
                }
            // fragment (j, n) is written by warp j kN + n: elements (kD / 8) g + 2 j and the next of columns
            // 8 n + 2 t and the next.  (Where to is read here: the next unit's rows may be staged from the last
            // barrier on.)
            const int write_j = warp / kN, write_n = warp % kN;
            long long write_at[2];
#pragma unroll
            for (int c = 0; c < 2; ++c)
                write_at[c] = rows[8 * write_n + 2 * t + c].out;
            float4(*part)[32] = sm.sum[warp & 7];
            if (warp >= 8) {
#pragma unroll
                for (int j = 0; j < kTilesD; ++j)
#pragma unroll
                    for (int n = 0; n < kN; ++n)
                        part[j * kN + n][lane] = make_float4(o[j][n][0], o[j][n][1], o[j][n][2], o[j][n][3]);
            }
            __syncthreads();
            if (warp < 8) {
#pragma unroll
                for (int j = 0; j < kTilesD; ++j)
#pragma unroll
                    for (int n = 0; n < kN; ++n) {
                        const float4 x = part[j * kN + n][lane];
                        part[j * kN + n][lane] =
                            make_float4(o[j][n][0] + x.x, o[j][n][1] + x.y, o[j][n][2] + x.z, o[j][n][3] + x.w);
                    }
            }
            __syncthreads();
            if (warp < kTilesD * kN && !stop) {
                float4 a = sm.sum[0][warp][lane];
#pragma unroll
                for (int k = 1; k < 8; ++k) {
                    const float4 x = sm.sum[k][warp][lane];
                    a.x += x.x, a.y += x.y, a.z += x.z, a.w += x.w;
                }
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int col = 8 * write_n + 2 * t + c, e = (kD / 8) * g + 2 * write_j;
                    const long long at = write_at[c];
                    if (at < 0)
                        continue;
                    const float Mc = write_n == 0 ? M[0][c] : M[kN - 1][c];
                    const float lc = write_n == 0 ? sum[0][c] : sum[kN - 1][c];
                    const float x = c ? a.y : a.x, y = c ? a.w : a.z;
                    if (seg.whole) {
                        const float inv = lc == 0.f ? 0.f : 1.f / lc;  // a NaN stays one
                        *reinterpret_cast<uint32_t *>(p.out + at * kD + e) = pack<kF16>(x * inv, y * inv);
                        if (p.lse && write_j == 0 && g == 0)
                            p.lse[at] = lc == 0.f ? -INFINITY : (Mc + log2f(lc)) * kLn2;
                    } else {
                        float *slot = p.part + ((size_t)blockIdx.x * 2 + (seg.first == 0 ? 0 : 1)) * kSlot;
                        *reinterpret_cast<float2 *>(slot + col * kD + e) = make_float2(x, y);
                        if (write_j == 0 && g == 0) {
                            slot[128 * kD + col] = Mc;
                            slot[128 * kD + 128 + col] = lc;
                        }
                    }
                }
            }
        }
    }
    if (!ok && lane == 0)
        for (; taken < issued; ++taken)
            mbar_wait_drain(&sm.full[warp][taken % kStages], (uint32_t)(taken / kStages) & 1u);
    __syncwarp();
}

}  // namespace

}  // namespace tv
