// paged_attention_few.cuh -- the attention over 4-bit pages for units of up to 8
// query rows per kv head: single tokens and the shortest chains of drafts.
//
// With so few rows a score tile of 128 rows would be work for rows that are not
// there, and unpacked tiles would go through shared memory for one use.  So keys
// lie on the rows of the products here and queries on their 8 columns, in registers:
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
// The CTA's tiles, as pieces of 32 keys, are split evenly over its 16 warps, a run
// each, and a warp walks its run alone: its own ring of copied pieces, its own maxima,
// sums and output, nothing to wait for.  A unit that lies within a run is written out
// by its warp.  Of those that do not, the warps leave their parts (the first of a run
// in the CTA's slots of the workspace, the last in shared memory once all rings are
// done with), and the CTA joins them in order.
//
// Bound by its instructions and by the way from one to the next: about 740 of a warp per piece, 288
// of them from codes to operands (masks and shifts at half rate) and 76 for scales and pairs, with four
// warps on a scheduler, which find 62 % of its slots; the largest wait is for fixed latencies (64
// requests of one token, 8 kv heads of 128 with 4 query heads each, prefixes of 512 to 16384: 155 us, 55 %
// of a copy's bandwidth; 16 requests at 65536 keys: 65 %); and by about 10 us to the first piece and through
// the join.  The registers that the kernel spills (372 bytes of stores at head_dim 128) are not the
// loop's: 0.07 % of that call's instructions touch local memory.  The batch took 582 us through the tiles of many rows, 246 with pieces that all warps
// shared, 172 with runs and copies of each warp's own, 157 with one shift for four codes.
#pragma once

namespace tv {

namespace {

constexpr int kFewRows = 8;
constexpr int kFewTiles = 2;  // of a CTA: with so many or fewer, as for many rows
constexpr int kFewKeys = 32;  // of a piece
constexpr int kFewSegs = 8;  // units that a warp lays out at a time
constexpr int kFewWarps = kThreads / 32;

constexpr int few_stages(int d)
{
    return d == 64 ? 6 : 3;
}

// The pieces of one unit in a warp's run.
struct FewSeg {
    int first, from, to;  // the unit's first piece, the run's own: pieces of the CTA's tiles, counted from t0
    int head;
    PlanReq r;
};

// A query row of a unit.
struct FewRow {
    uint64_t anc, path;
    int lo, pos;
    float slope;
};

// A warp's part of a unit that others have parts of too.
struct FewPart {
    int unit;  // its first piece; parts of one unit follow one another
    int begins, ends;  // whether the unit does, in this part
    int last;          // of its run: in shared memory
    int head;
    int row0, n;  // the request's rows; n 0: none to write
};
constexpr int kNoUnit = 0x7fffffff;

template <int kD>
struct FewSmem {
    static constexpr int kStage = 2 * kFewKeys * row_bytes(kD), kRing = few_stages(kD) * kStage;
    union {
        uint8_t ring[kFewWarps][kRing];
        float4 last[kFewWarps][kD / 16][32];  // O^T of the runs' last parts, fragment by fragment
    };
    FewRow row[kFewWarps][kFewRows];
    FewSeg seg[kFewWarps][kFewSegs];
    FewPart part[kFewWarps][2];
    float m[kFewWarps][2][kFewRows], l[kFewWarps][2][kFewRows];
};

// 16 bytes into shared memory, behind this thread's back: n of them (0 or 16) from src, else zeros.
__device__ __forceinline__ void copy16(uint32_t dst, const uint8_t *src, uint32_t n)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void copies_end()  // of a group
{
    asm volatile("cp.async.commit_group;" ::: "memory");
}
template <int kLeft>
__device__ __forceinline__ void copies_wait()  // for all groups but the last kLeft
{
    asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory");
}

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

template <int kD, bool kF16, int kForm>
__device__ __forceinline__ void few_rows(const PagedArgs &p, const PlanCta &cta, FewSmem<kD> &sm, int *abort_flag,
                                         uint64_t *never_bar)
{
    constexpr int kStages = few_stages(kD), kSlot = slot_floats(kD), kTilesD = kD / 16;
    constexpr float kShift = kF16 ? 8.f : 0.f, kGrow = kF16 ? 7.f : 8.f;  // as for many rows
    constexpr float kBack = 1.f / kOperandScale<kF16>;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const PlanReq *reqs = plan_reqs(p.plan);
    const int window = static_cast<const PlanHeader *>(p.plan)->window;
    const long long t0 = cta.t0;
    const int pieces = 4 * (int)(cta.t1 - t0);
    const int run0 = (int)((long long)pieces * warp / kFewWarps), run1 = (int)((long long)pieces * (warp + 1) / kFewWarps);
    uint8_t *ring = sm.ring[warp];
    FewSeg *segs = sm.seg[warp];
    FewRow *rows = sm.row[warp];

    // ---- a warp's copies.  A piece's blocks are parts of min(page_size, 32) keys, first K's, then V's; 16, 8 or 4
    // lanes copy a block, its codes in kD / 16 rounds and its scales in one more, to where those of all 32 keys lie.
    const int part_log2 = min(p.page_log2, 5);
    const int block_log2 = 1 + 5 - part_log2;  // blocks of a piece
    const int lanes_log2 = 5 - block_log2;     // lanes of a block
    const int block = lane >> lanes_log2, in_block = lane & ((1 << lanes_log2) - 1);
    const bool copies_v = block >> (block_log2 - 1);
    const int part_key = (block & ((1 << (block_log2 - 1)) - 1)) << part_log2;
    const uint32_t ring_a = smem_u32(ring);
    constexpr int kScales = kFewKeys * code_bytes(kD), kV = kFewKeys * row_bytes(kD);  // in a stage
    const uint32_t copy_to = ring_a + (copies_v ? kV : 0) + part_key * code_bytes(kD) + 16 * in_block;
    const uint32_t scales_to = ring_a + (copies_v ? kV : 0) + kScales + part_key * scale_bytes(kD) + 16 * in_block;
    constexpr int kRounds = kD / 16;
    const bool in_scales = in_block < (scale_bytes(kD) << part_log2) / 16;
    const int in_page = p.page_log2 > 5 ? (1 << p.page_log2) - 1 : 0;
    const long long scales_from = (long long)code_bytes(kD) << p.page_log2;
    struct Fetch {
        int id, key0, seg;
        bool inside;
    };
    int ahead_seg = 0, issue_at = 0, take_at = 0;
    // of the unit that is being fetched: its first piece not fetched, where its window's gap is, the key of piece
    // 0 before and behind that, its last token, its pages' ids and where this lane's blocks of them begin
    int a_to = run0, a_gap = 0, a_key = 0, a_key2 = 0, a_end = 0;
    const int32_t *a_table = nullptr;
    const uint8_t *a_pages = nullptr, *f_pages = nullptr;
    auto fetch = [&](int piece) {
        if (piece >= a_to) {
            while (piece >= segs[ahead_seg].to)
                ++ahead_seg;
            const FewSeg &s = segs[ahead_seg];
            a_to = s.to;
            a_gap = s.first + 4 * s.r.n1;
            a_key = s.r.a0 * kBN - kFewKeys * s.first;
            a_key2 = (s.r.b0 - s.r.n1) * kBN - kFewKeys * s.first;
            a_end = s.r.L + s.r.n;
            a_table = p.table + (size_t)s.r.b * p.max_pages;
            a_pages = (copies_v ? p.v_pages : p.k_pages) + s.head * p.head_stride + 16 * in_block;
        }
        Fetch f{-1, (piece < a_gap ? a_key : a_key2) + kFewKeys * piece, ahead_seg, false};
        const int slot = f.key0 + part_key, at = slot >> p.page_log2;
        f.inside = slot < a_end;
        if (f.inside && at < p.max_pages)
            f.id = a_table[at];  // (looked up here, used a piece later)
        f_pages = a_pages;
        return f;
    };
    auto report_hole = [&](int slot, const PlanReq &r) {
        const int past = slot + (1 << part_log2);
        const int lo_min = window > 0 ? max(r.begin, r.L - window + 1) : r.begin;
        if (past > lo_min || (window > 0 && past > r.begin && slot < min(r.far_end, r.L)))
            atomicOr(p.status, kStatusBounds);
    };
    auto copy_codes = [&](auto log2, uint32_t to, const uint8_t *src, uint32_t n) {
        constexpr int kStep = 16 << decltype(log2)::value;
#pragma unroll
        for (int i = 0; i < kRounds; ++i)
            copy16(to + i * kStep, src + i * kStep, n);
    };
    // Past the request's end and where a page is not there: zeros, whose scales make every element 0.
    auto issue = [&](const Fetch &f) {
        const bool there = f.inside && (unsigned)f.id < (unsigned)p.n_pages;
        const uint32_t n = there ? 16 : 0;
        const uint8_t *src = f_pages + ((unsigned long long)(there ? (unsigned)f.id : 0u) * p.page_units << 4);
        const int at = f.key0 & in_page;  // in a page of more than 32 slots
        const uint8_t *codes = src + at * code_bytes(kD);
        const uint32_t stage = issue_at * FewSmem<kD>::kStage;
        if (in_scales)
            copy16(scales_to + stage, src + scales_from + at * scale_bytes(kD), n);
        if (part_log2 == 4)
            copy_codes(std::integral_constant<int, 3>{}, copy_to + stage, codes, n);
        else if (part_log2 == 3)
            copy_codes(std::integral_constant<int, 2>{}, copy_to + stage, codes, n);
        else
            copy_codes(std::integral_constant<int, 4>{}, copy_to + stage, codes, n);
        copies_end();
        if (f.inside && !there && !copies_v && in_block == 0)
            report_hole(f.key0 + part_key, segs[f.seg].r);
        issue_at = issue_at + 1 == kStages ? 0 : issue_at + 1;
    };

    // ---- where this thread's keys and values lie in a piece.  Row i of a product's 16 keys is key i with its
    // lowest two bits swapped, so that the four keys which V's loads take at once lie in different banks.
    const int key_k = (g & 4) | ((g & 1) << 1) | ((g >> 1) & 1), key_v = (t >> 1) * 4 + (t & 1);
    const int k_code = key_k * code_bytes(kD) + t * (kD / 8);
    const int k_scale = kScales + key_k * scale_bytes(kD) + t * (kD / 4) / kGroup;
    const int v_code = kV + key_v * code_bytes(kD) + g * (kD / 16);
    const int v_scale = kV + kScales + key_v * scale_bytes(kD) + g * (kD / 8) / kGroup;

    // where row r of a unit goes, (row, query head); -1: no such row
    auto row_at = [&](const FewSeg &s, int r) {
        const int row = cta.rb * 128 + r, node = row / p.group, qh = s.head * p.group + row % p.group;
        const bool valid = node < s.r.n && s.r.row0 + node < p.n_rows &&
                           in_bounds(node < kMaxNodes && qh < p.Hq && s.r.row0 >= 0, p.status);
        return valid ? (long long)(s.r.row0 + node) * p.Hq + qh : -1ll;
    };
    // what the rows see: a lane each; false if the call's bank has not the plan's tree
    auto stage = [&](const FewSeg &s) {
        const bool known = (unsigned)s.r.tree < (unsigned)p.n_trees;
        const TreeDesc &td = p.trees[known ? s.r.tree : 0];
        const bool same = known && td.n == s.r.n;
        if (lane < kFewRows) {
            const int row = cta.rb * 128 + lane, node = row / p.group, qh = s.head * p.group + row % p.group;
            const bool valid = same && node < s.r.n && node < kMaxNodes;
            const int L = s.r.L, dep = valid ? td.depth[node] : 0;
            uint64_t anc = valid ? td.anc[node] : 0;
            FewRow &r = rows[lane];
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
            r.lo = window > 0 ? max(s.r.begin, L + dep - window + 1) : s.r.begin;
            r.pos = L + dep;
            r.slope = kForm == kBias && valid && qh < p.Hq && p.slopes ? p.slopes[qh] * kLog2e : 0.f;
        }
        if (!same && lane == 0)
            atomicOr(p.status, kStatusBounds);
        __syncwarp();
        return same;
    };

    // ---- the run's first unit
    bool ok = true;
    int request = cta.idx, head0 = 0;
    if (run0 < run1) {
        const long long tile = t0 + (run0 >> 2);
        long long base = cta.req.tile_base;
        int T = cta.req.T;
        if (tile >= base + (long long)T * p.Hkv) {  // not of the request that the CTA begins in
            for (int i0 = cta.idx;; i0 += 32) {
                const int i = i0 + lane;
                const uint32_t before = __ballot_sync(0xffffffffu, i < p.batch && reqs[i].tile_base <= tile);
                const int n = before == 0xffffffffu ? 32 : __ffs((int)~before) - 1;
                request = i0 + n - 1;
                if (n < 32)
                    break;
            }
            base = reqs[request].tile_base;
            T = reqs[request].T;
        }
        const long long in = tile - base;
        head0 = (unsigned long long)in <= 0xffffffffull ? (int)((uint32_t)in / (uint32_t)T) : (int)(in / T);
    }
    if (lane < 2)
        sm.part[warp][lane] = FewPart{kNoUnit, 0, 0, 0, 0, 0, 0};
    float o[kTilesD][4];
    float m[2], l[2];          // of columns 2 t and 2 t + 1; l: this thread's keys
    bool last_here = false;    // o, m and l are the run's last part
    int n_parts = 0;
    for (int piece = run0; piece < run1; head0 += kFewSegs) {
        // ---- the next units
        int n_segs;
        {
            const int u = head0 + lane, i = request + u / p.Hkv;
            FewSeg s{};
            bool in = lane < kFewSegs && i < p.batch;
            if (in) {
                s.r = i == cta.idx ? cta.req : reqs[i];
                s.head = u % p.Hkv;
                const long long first = s.r.tile_base + (long long)s.head * s.r.T - t0;
                in = first < (run1 + 3) / 4;
                s.first = in ? 4 * (int)first : 0;
                s.from = max(s.first, run0);
                s.to = min(s.first + 4 * s.r.T, run1);
                in = in && s.from < s.to;
            }
            // records behind the last request hold anything: only what follows without a gap counts
            const uint32_t all = __ballot_sync(0xffffffffu, in);
            n_segs = __ffs((int)~all) - 1;  // (at most kFewSegs lanes)
            __syncwarp();
            if (lane < n_segs)
                segs[lane] = s;
            __syncwarp();
        }
        if (n_segs == 0)
            break;
        const int last = segs[n_segs - 1].to;
        // the ring filled, the next page looked up
        issue_at = take_at = 0;
        ahead_seg = 0;
        a_to = piece;
        int next = piece;
        Fetch ahead = fetch(next);
        auto refill = [&] {  // one group of copies each time, an empty one at the end
            if (next >= last) {
                copies_end();
                return;
            }
            issue(ahead);
            if (++next < last)
                ahead = fetch(next);
        };
        for (int s = 0; s < kStages; ++s)
            refill();

        for (int si = 0; si < n_segs; ++si) {
            const FewSeg &seg = segs[si];
            const int L = seg.r.L, end = L + seg.r.n, begin = seg.r.begin;
            const int far = window > 0 ? min(seg.r.far_end, L) : begin;
            const int lo_min = window > 0 ? max(begin, L - window + 1) : begin;
            const int lo_max = window > 0 ? lo_min + kMaxNodes : begin;  // past any row's
            const int gap = seg.first + 4 * seg.r.n1, to = seg.to;
            const int key_a = seg.r.a0 * kBN - kFewKeys * seg.first;
            const int key_b = (seg.r.b0 - seg.r.n1) * kBN - kFewKeys * seg.first;
            // the query of column g in the order of the keys' elements
            uint32_t q[kD / 16][2];
            {
                const long long at = row_at(seg, g);
                const uint4 *src = reinterpret_cast<const uint4 *>(p.q + max(at, 0ll) * kD + t * (kD / 4));
#pragma unroll
                for (int i = 0; i < kD / 32; ++i) {
                    const uint4 x = code_order(at >= 0 ? src[i] : make_uint4(0, 0, 0, 0));
                    q[2 * i][0] = x.x, q[2 * i][1] = x.y;
                    q[2 * i + 1][0] = x.z, q[2 * i + 1][1] = x.w;
                }
            }
            const bool known = stage(seg);
            m[0] = m[1] = -INFINITY, l[0] = l[1] = 0.f;
#pragma unroll
            for (int j = 0; j < kTilesD; ++j)
                o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;

            for (; piece < to; ++piece) {
                if (p.expire_wait)
                    ok = ok && warp_agrees(mbar_wait_bounded(never_bar, 0, abort_flag, p.status));
                copies_wait<kStages - 1>();
                __syncwarp();
                const int key0 = (piece < gap ? key_a : key_b) + kFewKeys * piece;
                const uint32_t base = ring_a + take_at * FewSmem<kD>::kStage;
                take_at = take_at + 1 == kStages ? 0 : take_at + 1;
                const auto work = [&](auto is_masked) {
                    constexpr bool masked = decltype(is_masked)::value;
                    // whether some row looks at a value: the others may be anything
                    auto looked_at = [&](int key) {
                        const int slot = key0 + key;
                        return slot < end && slot >= begin && (slot >= lo_min || slot < far);
                    };
                    float s[2][4] = {};
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        uint32_t w[2][kD / 32];
                        OperandScale<kF16> sc[2];
#pragma unroll
                        for (int a = 0; a < 2; ++a) {
                            const uint32_t c = base + k_code + (8 * a + 16 * b) * code_bytes(kD);
                            if constexpr (kD == 128) {
                                const uint4 x = lds128(c);
                                w[a][0] = x.x, w[a][1] = x.y, w[a][2] = x.z, w[a][3] = x.w;
                            } else {
                                const uint2 x = lds64(c);
                                w[a][0] = x.x, w[a][1] = x.y;
                            }
                            const float f = scale_of(lds8(base + k_scale + (8 * a + 16 * b) * scale_bytes(kD)));
                            sc[a] = operand_scale<kF16>(f, f);
                        }
#pragma unroll
                        for (int i = 0; i < kD / 32; ++i) {
                            uint32_t x[4], y[4];
                            dequant_four<kF16>(w[0][i], sc[0], x);
                            dequant_four<kF16>(w[1][i], sc[1], y);
#pragma unroll
                            for (int h = 0; h < 2; ++h)
                                mma_16x8x16<kF16>(s[b], x[2 * h], y[2 * h], x[2 * h + 1], y[2 * h + 1], q[2 * i + h][0],
                                                  q[2 * i + h][1]);
                        }
                    }
                    // scores: element c of s[b] is key 16 b + 8 (c / 2) + key_k, column 2 t + c % 2
                    constexpr float kHidden = kForm == kCap ? INFINITY : -INFINITY;  // z = -inf
                    uint32_t sees = 0xffu;  // bit 4 b + c of this thread's scores
                    if constexpr (masked) {
                        sees = 0;
#pragma unroll
                        for (int x = 0; x < 8; ++x) {
                            const FewRow &r = rows[2 * t + (x & 1)];
                            const int slot = key0 + 8 * (x >> 1) + key_k;
                            const bool see = slot < L ? slot >= r.lo || (slot >= begin && slot < far)
                                                      : slot - L < 64 && ((r.anc >> (slot - L)) & 1);
                            sees |= see ? 1u << x : 0u;
                        }
                    }
                    if constexpr (kForm != kPlain) {
                        if (kForm == kCap || p.cap > 0.f) {
                            // four of one row together: what is not a number there makes that row none anyway,
                            // unless it is hidden
#pragma unroll
                            for (int c = 0; c < 2; ++c) {
                                uint32_t r[4];
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    const int b = i >> 1, e = c + 2 * (i & 1);
                                    r[i] = !masked || ((sees >> (4 * b + e)) & 1u) ? __float_as_uint(s[b][e]) : 0xff800000u;
                                }
                                cap_four(r, p.cap_in);
#pragma unroll
                                for (int i = 0; i < 4; ++i)
                                    s[i >> 1][c + 2 * (i & 1)] = kForm == kCap
                                                                     ? __uint_as_float(r[i])
                                                                     : fmaf(-2.f * p.cap, __uint_as_float(r[i]), p.cap);
                            }
                        } else {
#pragma unroll
                            for (int x = 0; x < 8; ++x)
                                s[x >> 2][x & 3] *= p.scale;
                        }
                    }
#pragma unroll
                    for (int x = 0; x < 8; ++x) {
                        float &z = s[x >> 2][x & 3];
                        if constexpr (kForm == kBias) {
                            const FewRow &r = rows[2 * t + (x & 1)];
                            const int slot = key0 + 8 * (x >> 1) + key_k;
                            // in the tree: one step for each node of the row's root path before this one
                            const int dist = slot <= L ? r.pos - slot
                                                       : r.pos - L - (slot - L < 64
                                                                          ? __popcll(r.path & ((1ull << (slot - L)) - 1))
                                                                          : __popcll(r.path));
                            z = fmaf(-r.slope, (float)dist, z);
                        }
                        if constexpr (masked)
                            z = (sees >> x) & 1u ? z : kHidden;
                    }
                    // z = f s + f0; f < 0 where s is a capped score's w
                    const float f = kForm == kCap ? -2.f * p.cap : kForm == kPlain ? p.scale : 1.f;
                    const float f0 = kForm == kCap ? p.cap : 0.f;
                    float alpha[2];
                    bool raise = false;
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float mx;
                        if constexpr (kForm == kCap) {
                            mx = fminf(fminf(s[0][c], s[0][c + 2]), fminf(s[1][c], s[1][c + 2]));
#pragma unroll
                            for (int x = 4; x < 32; x *= 2)
                                mx = fminf(mx, __shfl_xor_sync(0xffffffffu, mx, x));
                        } else {
                            mx = fmaxf(fmaxf(s[0][c], s[0][c + 2]), fmaxf(s[1][c], s[1][c + 2]));
#pragma unroll
                            for (int x = 4; x < 32; x *= 2)
                                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, x));
                        }
                        mx = fmaf(f, mx, f0);
                        alpha[c] = 1.f;
                        if (mx > m[c] + kShift + kGrow) {
                            alpha[c] = m[c] == -INFINITY ? 0.f : ex2_approx(m[c] - (mx - kShift));
                            m[c] = mx - kShift;
                            raise = true;
                        }
                    }
                    if (__any_sync(0xffffffffu, raise)) {
                        l[0] *= alpha[0], l[1] *= alpha[1];
#pragma unroll
                        for (int j = 0; j < kTilesD; ++j)
#pragma unroll
                            for (int c = 0; c < 4; ++c)
                                o[j][c] *= alpha[c & 1];
                    }
                    uint32_t w[2][2];  // P^T as an operand
                    const float mu0 = f0 - (m[0] == -INFINITY ? 0.f : m[0]), mu1 = f0 - (m[1] == -INFINITY ? 0.f : m[1]);
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int a = 0; a < 2; ++a) {
                            const float p0 = ex2_approx(fmaf(f, s[b][2 * a], mu0));
                            const float p1 = ex2_approx(fmaf(f, s[b][2 * a + 1], mu1));
                            l[0] += p0, l[1] += p1;
                            w[b][a] = transpose_8x8(pack<kF16>(p0, p1));
                        }
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        uint32_t v[2][2][kD / 64];  // [keys 0-7, 8-15][first key, second][8 codes each]
                        OperandScale<kF16> sc[2];
#pragma unroll
                        for (int a = 0; a < 2; ++a) {
                            float f[2];
#pragma unroll
                            for (int x = 0; x < 2; ++x) {
                                const uint32_t c = base + v_code + (2 * x + 8 * a + 16 * b) * code_bytes(kD);
                                if constexpr (kD == 128) {
                                    const uint2 y = lds64(c);
                                    v[a][x][0] = y.x, v[a][x][1] = y.y;
                                } else {
                                    v[a][x][0] = lds32(c);
                                }
                                f[x] = scale_of(lds8(base + v_scale + (2 * x + 8 * a + 16 * b) * scale_bytes(kD)));
                                if constexpr (masked)
                                    f[x] = looked_at(key_v + 2 * x + 8 * a + 16 * b) ? f[x] : 0.f;
                            }
                            sc[a] = operand_scale<kF16>(f[0], f[1]);
                        }
#pragma unroll
                        for (int i = 0; i < kD / 64; ++i)
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                // four elements of two keys
                                const uint32_t sel = h ? 0x7632 : 0x5410;
                                uint32_t x[4], y[4];
                                dequant_four<kF16>(__byte_perm(v[0][0][i], v[0][1][i], sel), sc[0], x);
                                dequant_four<kF16>(__byte_perm(v[1][0][i], v[1][1][i], sel), sc[1], y);
#pragma unroll
                                for (int e = 0; e < 2; ++e)
                                    mma_16x8x16<kF16>(o[4 * i + 2 * h + e], x[2 * e], x[2 * e + 1], y[2 * e], y[2 * e + 1],
                                                      w[b][0], w[b][1]);
                            }
                    }
                };
                if (key0 + kFewKeys > L || key0 < lo_max) {
                    if (key0 < end)
                        work(std::true_type{});
                } else {
                    work(std::false_type{});
                }
                __syncwarp();
                refill();
            }

            // ---- the unit's end here
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int x = 4; x < 32; x *= 2)
                    l[c] += __shfl_xor_sync(0xffffffffu, l[c], x);
            const bool begins = seg.from == seg.first, ends = seg.to == seg.first + 4 * seg.r.T;
            if (begins && ends) {
                // columns 2 t and 2 t + 1: kD / 8 elements from (kD / 8) g on
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const long long at = row_at(seg, 2 * t + c);
                    if (at < 0 || !known || !ok)
                        continue;
                    const float inv = l[c] == 0.f ? 0.f : kBack / l[c];  // a NaN stays one
                    uint32_t w[kTilesD];
#pragma unroll
                    for (int j = 0; j < kTilesD; ++j)
                        w[j] = pack<kF16>(o[j][c] * inv, o[j][c + 2] * inv);
                    uint4 *dst = reinterpret_cast<uint4 *>(p.out + at * kD + g * (kD / 8));
#pragma unroll
                    for (int j = 0; j < kTilesD / 4; ++j)
                        dst[j] = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
                    if (p.lse && g == 0)
                        p.lse[at] = l[c] == 0.f ? -INFINITY : (m[c] + log2f(l[c])) * kLn2;
                }
                continue;
            }
            // a part: at most two of a run, the second at its end
            if (lane == 0)
                sm.part[warp][n_parts] =
                    FewPart{seg.first, begins, ends, seg.to == run1, seg.head, seg.r.row0, known ? seg.r.n : 0};
            if (g == 0) {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    sm.m[warp][n_parts][2 * t + c] = m[c];
                    sm.l[warp][n_parts][2 * t + c] = l[c];
                }
            }
            if (seg.to < run1) {
                float4 *to = reinterpret_cast<float4 *>(p.part + (size_t)blockIdx.x * 2 * kSlot) + warp * kTilesD * 32;
#pragma unroll
                for (int j = 0; j < kTilesD; ++j)
                    to[j * 32 + lane] = make_float4(o[j][0], o[j][1], o[j][2], o[j][3]);
            } else {
                last_here = true;  // the last of the run
            }
            ++n_parts;
        }
    }
    copies_wait<0>();

    // ---- the units that runs share
    __syncthreads();  // all rings are done with
    if (last_here) {
#pragma unroll
        for (int j = 0; j < kTilesD; ++j)
            sm.last[warp][j][lane] = make_float4(o[j][0], o[j][1], o[j][2], o[j][3]);
    }
    __syncthreads();
    // warp j takes fragment j of every unit, elements (kD / 8) g + 2 j and the next; at most two units are also other
    // CTAs', and go to the slots that the first parts lie in: once all have read those
    const bool mine = warp < kTilesD;
    const bool stop = *const_cast<volatile int *>(abort_flag) != 0;  // (nobody waits any more)
    const float4 *firsts = reinterpret_cast<const float4 *>(p.part + (size_t)blockIdx.x * 2 * kSlot) + threadIdx.x;
    float4 kept[2];
    float kept_m[2][2], kept_l[2][2];
    bool keep[2] = {false, false};
    for (int x = 0; mine && x < 2 * kFewWarps;) {
        const FewPart head = sm.part[x >> 1][x & 1];
        int y = x + 1;
        if (head.unit == kNoUnit) {
            x = y;
            continue;
        }
        while (y < 2 * kFewWarps && (sm.part[y >> 1][y & 1].unit == head.unit || sm.part[y >> 1][y & 1].unit == kNoUnit))
            ++y;
        bool ends = false;
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
        float M[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};
        for (int z = x; z < y; ++z)
            if (sm.part[z >> 1][z & 1].unit == head.unit)
#pragma unroll
                for (int c = 0; c < 2; ++c)
                    M[c] = fmaxf(M[c], sm.m[z >> 1][z & 1][2 * t + c]);
#pragma unroll 4
        for (int z = x; z < y; ++z) {
            const FewPart &part = sm.part[z >> 1][z & 1];
            if (part.unit != head.unit)
                continue;
            ends = part.ends;
            const float4 v = part.last ? sm.last[z >> 1][warp][lane] : __ldcg(firsts + (z >> 1) * kTilesD * 32);
            float f[2];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const float mz = sm.m[z >> 1][z & 1][2 * t + c];
                f[c] = mz == -INFINITY ? 0.f : ex2_approx(mz - M[c]);
                sum[c] = fmaf(f[c], sm.l[z >> 1][z & 1][2 * t + c], sum[c]);
            }
            a.x = fmaf(f[0], v.x, a.x), a.y = fmaf(f[1], v.y, a.y);
            a.z = fmaf(f[0], v.z, a.z), a.w = fmaf(f[1], v.w, a.w);
        }
        if (head.begins && ends) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                FewSeg s{};
                s.head = head.head, s.r.n = head.n, s.r.row0 = head.row0;
                const long long at = row_at(s, 2 * t + c);
                if (at < 0 || stop)
                    continue;
                const float inv = sum[c] == 0.f ? 0.f : kBack / sum[c];
                *reinterpret_cast<uint32_t *>(p.out + at * kD + g * (kD / 8) + 2 * warp) =
                    pack<kF16>((c ? a.y : a.x) * inv, (c ? a.w : a.z) * inv);
                if (p.lse && warp == 0 && g == 0)
                    p.lse[at] = sum[c] == 0.f ? -INFINITY : (M[c] + log2f(sum[c])) * kLn2;
            }
        } else {
            // of the CTA's first tile on: slot 0, as for many rows
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (i == (head.unit <= 0 ? 0 : 1)) {
                    keep[i] = true;
                    kept[i] = a;
#pragma unroll
                    for (int c = 0; c < 2; ++c)
                        kept_m[i][c] = M[c], kept_l[i][c] = sum[c];
                }
        }
        x = y;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (!keep[i])
            continue;
        float *slot = p.part + ((size_t)blockIdx.x * 2 + i) * kSlot;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int col = 2 * t + c;
            *reinterpret_cast<float2 *>(slot + col * kD + g * (kD / 8) + 2 * warp) =
                c ? make_float2(kept[i].y * kBack, kept[i].w * kBack) : make_float2(kept[i].x * kBack, kept[i].z * kBack);
            if (warp == 0 && g == 0) {
                slot[128 * kD + col] = kept_m[i][c];
                slot[128 * kD + 128 + col] = kept_l[i][c];
            }
        }
    }
}

}  // namespace

}  // namespace tv
