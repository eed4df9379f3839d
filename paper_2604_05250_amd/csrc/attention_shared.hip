// Attention over a paged cache of a batch whose sequences share prefixes (the answers to one prompt): a row's keys are those of its group's
// prefix and its sequence's own.  A softmax can be taken in parts: with the states (m, l, o) of two sets of keys, reference, sum of weights
// and weighted sum of values, that of both is  M = max(m, m'),  2^(m-M) l + 2^(m'-M) l',  2^(m-M) o + 2^(m'-M) o'.  So the rows of all
// sequences of a group meet the prefix together, as the rows of one very long block, and its keys are read once for all of them; the own
// keys are met sequence by sequence; a second kernel merges the states.  The workgroups are those of attention_paged.h, of either kind in
// one launch where both take as many row blocks, as neither fills the card in a serving batch's step.  Where that pays (plan_of), a sequence's
// rows take prefix and own keys in one go instead, and there is nothing to merge.
// One token of 16 sequences, 32/8 heads, e4m3, over 4096 keys and 512 of their own: 15.3 us, of which two launches that find no key take
// 6.2 and either part alone some 6 more; with dd_paged_attention on whole tables, where caches hold what sequences share, 22.  Of 64
// over 32768 and 256: 60 to 65, 0.55 PFLOP/s, the own keys' workgroups behind the others some 10 of it; on whole tables 285.
#include "attention_paged.h"

namespace dd {
namespace {

// Every state of a row, merged by D / 4 lanes: the prefix's splits, then those of the own keys.  Two or four such lots of lanes have a half or
// a quarter of the states each where one would have to go to memory more than once (one token of 32 sequences over 4000 keys, nine states
// 16.5 -> 14.3 us).  All that a row can have are asked for before it is known how many it has.
struct SharedMerge {
    const int32_t *kv_lens, *group_starts, *prefix_lens;
    uint8_t *O;
    int rows_total, Hkv, max_pages, max_prefix_pages, groups, page_log2, own_splits, prefix_splits;
};
template <int D, int PARTS>
__global__ __launch_bounds__(256) void shared_merge_kernel(const float *part_ml, const float *part_o, int slots, int rows, SharedMerge a)
{
    constexpr int LANES = D / 4, U = 8, ROWS = 256 / LANES / PARTS;
    const int lot = threadIdx.x / LANES, part = lot % PARTS, mine = lot / PARTS, d0 = (threadIdx.x % LANES) * 4;
    const int row = min((int)blockIdx.x * ROWS + mine, rows - 1);
    const float2 *ml = reinterpret_cast<const float2 *>(part_ml) + (size_t)row * slots;
    const floatx4 *po = reinterpret_cast<const floatx4 *>(part_o + (size_t)row * slots * D + d0);
    float2 st[U];
    floatx4 v[U];
    auto fetch = [&](int s0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int s = min(s0 + u * PARTS, slots - 1);
            st[u] = ml[s];
            v[u] = po[(size_t)s * (D / 4)];
        }
    };
    fetch(part);
    const int b = (int)((unsigned)row / (unsigned)a.rows_total / (unsigned)a.Hkv);
    const int own = shared_share_of(a.kv_lens[b], a.max_pages, a.page_log2, a.own_splits, kSplitTiles).used;
    int lo = 0, hi = a.groups;                       // the last group that begins at b or before
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.group_starts[mid] <= b) lo = mid;
        else hi = mid;
    }
    const bool member = a.group_starts[lo] <= b && b < a.group_starts[lo + 1];
    const int shared = shared_share_of(member ? a.prefix_lens[lo] : 0, a.max_prefix_pages, a.page_log2, a.prefix_splits, kSplitTiles).used;
    auto counts = [&](int s) __attribute__((always_inline)) { return s < shared || (s >= a.prefix_splits && s < a.prefix_splits + own); };
    float M = kNone, L = 0;
    floatx4 x = {0, 0, 0, 0};
    for (int s0 = part;;) {
        float top = M;
#pragma unroll
        for (int u = 0; u < U; ++u) top = fmaxf(top, counts(s0 + u * PARTS) ? st[u].x : M);
        const float by = __builtin_amdgcn_exp2f(M - top);
        M = top;
        L *= by;
        x *= by;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (counts(s0 + u * PARTS)) {
                const float f = __builtin_amdgcn_exp2f(st[u].x - M);
                L += f * st[u].y;
                x += f * v[u];
            }
        }
        s0 += U * PARTS;
        if (s0 >= slots) break;
        fetch(s0);
    }
    if constexpr (PARTS > 1) {
        __shared__ float2 ml_of[256 / LANES];
        __shared__ floatx4 x_of[256];
        if (threadIdx.x % LANES == 0) ml_of[lot] = make_float2(M, L);
        x_of[threadIdx.x] = x;
        __syncthreads();
        if (part != 0) return;
        float2 all[PARTS];
        float top = kNone;
#pragma unroll
        for (int k = 0; k < PARTS; ++k) {
            all[k] = ml_of[lot + k];
            top = fmaxf(top, all[k].x);
        }
        L = 0;
        x = floatx4{0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < PARTS; ++k) {
            const float f = __builtin_amdgcn_exp2f(all[k].x - top);
            L += f * all[k].y;
            x += f * x_of[threadIdx.x + k * LANES];
        }
    }
    if ((int)blockIdx.x * ROWS + mine >= rows) return;
    const float inv = L > 0 ? 1.0f / L : 0.0f;       // no key at all: zeros
    *reinterpret_cast<uint2 *>(a.O + ((size_t)row * D + d0) * 2) = make_uint2(pack_bf16(x[0] * inv, x[1] * inv), pack_bf16(x[2] * inv, x[3] * inv));
}

constexpr int kLongSplitTiles = 32;          // tiles of 64 keys of a long split
// One kind of workgroup: 32-row blocks each takes, splits of the keys, row tiles, workgroups.
struct Kind { int rg, splits; long row_tiles, wgs; };
struct Plan { Kind prefix, own; int slots; bool whole; };
Plan plan_of(const SharedAttnShape &s)
{
    const long rows = (long)(s.H / s.Hkv) * s.n, all = rows * s.B;
    auto blocks_of = [](long r) { return (r + 31) / 32; };
    auto group_rows = [&](long blocks, bool few, bool full) { return few || blocks <= (s.fp8 ? 512 : 256) ? 1 : full && blocks > (s.fp8 ? 1792 : 1024) ? 4 : 2; };
    auto is_full = [](long r) { return (r + 127) / 128 * 128 * 8 <= r * 9; };
    auto splits_of = [](long room, long base, long tiles, int least) {
        const long most = (tiles + least - 1) / least;       // (a tile for each wave; the last split may have less)
        const long n = room / base < most ? room / base : most;
        return (int)(n < 1 ? 1 : n > kMaxSplits ? kMaxSplits : n);
    };
    Plan p;
    p.own.rg = group_rows(s.B * (long)s.Hkv * blocks_of(rows), rows <= kFewRows, is_full(rows));
    p.own.row_tiles = (rows + 32 * p.own.rg - 1) / (32 * p.own.rg);
    const long own_base = (long)s.B * s.Hkv * p.own.row_tiles;
    p.own.splits = splits_of(kUnits, own_base, ((long)s.max_pages << s.page_log2) / 64, kSplitTiles);
    p.own.wgs = own_base * p.own.splits;
    p.prefix.rg = group_rows((long)s.Hkv * blocks_of(all), all <= kFewRows, is_full(all));
    p.prefix.row_tiles = all / (32 * p.prefix.rg) + s.G;      // (every group may end within a tile)
    if (s.G == 1) p.prefix.row_tiles = (all + 32 * p.prefix.rg - 1) / (32 * p.prefix.rg);
    const long base = (long)s.Hkv * p.prefix.row_tiles;
    // Splits of the prefix: as many workgroups as run at once, but for the room that the own keys' ones take where splits are short and a
    // second round of workgroups costs (one token of 32 sequences over 4000 e4m3 keys and 64 of their own 23.4 -> 16.6 us, of 64 over 8192
    // and 256 30.2 -> 25.3; of 64 over 32768 61.4 without, 62.8 with).
    const long prefix_tiles = ((long)s.max_prefix_pages << s.page_log2) / 64;
    long room = 2 * kUnits;
    if (prefix_tiles < room / base * kLongSplitTiles) room = room - p.own.wgs > kUnits ? room - p.own.wgs : kUnits;
    p.prefix.splits = splits_of(room, base, prefix_tiles, kSplitTiles);
    p.prefix.wgs = base * p.prefix.splits;
    // Sequence by sequence, prefix and own keys in one go and nothing to merge, or the prefix together?  What either has to do is row blocks
    // times keys; the first has more blocks where a sequence's rows fill less than one, and they are as long as all keys.  us, sequence by
    // sequence / together, 32/8 heads, by sequences x rows and keys (64 of them a sequence's own):
    //     e4m3    4 x 1     512   7.2 / 10.7    1024   9.8 / 10.3    2048  16.3 / 12.3       16 x 8   1280  13.6 / 19.5    2964  23.4 / 23.5
    //            16 x 1     512   7.4 / 11.3    1024  11.0 / 11.7    1280  12.6 / 11.6        4 x 64  1024  12.0 / 26.1    4064  29.6 / 37.8
    //            64 x 1    1024  15.0 / 18.4    1280  16.8 / 21.2    2048  23.3 / 21.0        4 x 64 16064  97.0 / 90.3
    //             8 x 8    1280  13.3 / 15.6    2048  17.6 / 19.5    2964  23.3 / 19.7       16 x 64  1024  26.4 / 49.5    4064  78.4 / 96.8
    //     bf16    4 x 1     512   8.3 / 11.2     768  11.0 / 11.3    1024  12.8 / 11.2       16 x 8   1280  16.1 / 19.7    2964  29.0 / 25.3
    //            64 x 1     768  16.0 / 18.4    1024  19.1 / 19.6    1280  22.4 / 19.4        4 x 64  4064  36.5 / 42.9   16064 125.8 / 120
    //             8 x 8     768  12.3 / 13.2    1280  16.0 / 16.7    2048  21.3 / 19.4       16 x 64  1024  29.6 / 49.8    4064  90.0 / 106
    // So up to a length that grows with the row blocks that there are in all; where compute units have two workgroups or more, less of
    // it, unless the blocks are full.
    const long together = s.Hkv * blocks_of(all), apart = s.B * (long)s.Hkv * blocks_of(rows), keys = ((long)s.max_prefix_pages + s.max_pages) << s.page_log2;
    const long least = s.fp8 ? 1024 : 768, grown = (s.fp8 ? 28 : 20) * together, most = least > grown ? least : grown;
    const bool full = apart * 4 <= together * 5;
    p.whole = full && together >= 2 * kUnits ? true
            : keys <= (full || apart <= kUnits ? most : apart <= 2 * kUnits ? most * 3 / 4 : most * 3 * kUnits / (2 * apart));
    const int hook = tune("DD_TUNE_SHARED_WHOLE", -1);
    if (hook >= 0) p.whole = hook != 0;
    // In one go a sequence's positions are those of both tables, counted in 32 bits, with up to 127 between them and a thousand asked for behind
    // the last.  Tables that may hold more together than one may are taken by two kinds of workgroups.
    if (keys >= 1l << 30) p.whole = false;
    if (p.whole) {
        p.own.splits = 1;
        p.own.wgs = own_base;
        p.prefix.splits = 0;
        p.prefix.wgs = 0;
    }
    p.slots = p.prefix.splits + p.own.splits;
    return p;
}

unsigned eights(long wgs) { return (unsigned)((wgs + 7) / 8 * 8); }

template <int D, bool FP8, int NT, bool ONE>
hipError_t attend(const SharedAttnArgs &a, const SharedTail &tail, int rg, unsigned grid, unsigned launched, unsigned shape, hipStream_t stream)
{
    auto run = [&](auto kernel) {
        return launch(kernel, dim3(grid), dim3(256), stream, a.table, a.kv_lens, static_cast<const uint8_t *>(a.Kc), static_cast<const uint8_t *>(a.Vc), a.s.Hkv,
                      (a.s.H / a.s.Hkv) * a.s.n, a.num_pages, a.s.max_pages, launched, shape, tail);
    };
    return rg == 1 ? run(attn_paged_kernel<D, FP8, NT, ONE, 1, SharedTail>)
         : rg == 2 ? run(attn_paged_kernel<D, FP8, NT, ONE, 2, SharedTail>) : run(attn_paged_kernel<D, FP8, NT, ONE, 4, SharedTail>);
}
template <int D, bool FP8>
hipError_t attend(const SharedAttnArgs &a, const SharedTail &tail, int rg, unsigned grid, unsigned launched, unsigned shape, hipStream_t stream)
{
    constexpr int NT = FP8 ? 2 : 1;
    return (1 << a.s.page_log2) >= 32 * NT ? attend<D, FP8, NT, true>(a, tail, rg, grid, launched, shape, stream)
                                           : attend<D, FP8, NT, false>(a, tail, rg, grid, launched, shape, stream);
}

}  // namespace

bool shared_attention_fits(const SharedAttnShape &s)
{
    const double rows = (double)(s.H / s.Hkv) * s.n;
    // (fewer than 2^22 workgroups of either kind, of 256 threads, and fewer than 2^27 rows, for which the merge has a workgroup per eight or more,
    // less only where rows are few: launches of fewer than 2^32 threads)
    return rows * s.B * s.Hkv < 1073741824.0 && ((__builtin_ceil(rows / 32) + 1) * s.B + s.G) * s.Hkv < 4194304.0;
}

size_t shared_attention_workspace_bytes(const SharedAttnShape &s)
{
    const Plan p = plan_of(s);
    return p.whole ? 0 : (size_t)s.B * s.H * s.n * (size_t)p.slots * (size_t)(s.d + 2) * sizeof(float);
}

hipError_t launch_attention_shared(const SharedAttnArgs &a, hipStream_t stream)
{
    const SharedAttnShape &s = a.s;
    const Plan p = plan_of(s);
    const size_t rows = (size_t)s.B * s.H * s.n;
    SharedTail tail;
    static_cast<PagedTail &>(tail) = PagedTail{static_cast<const uint8_t *>(a.Q), a.k_scale, a.v_scale, static_cast<uint8_t *>(a.O), static_cast<float *>(a.workspace),
                                               static_cast<float *>(a.workspace) + rows * p.slots * s.d, (float)(1.4426950408889634 / __builtin_sqrt((double)s.d))};
    tail.prefix_table = a.prefix_table; tail.prefix_lens = a.prefix_lens; tail.group_starts = a.group_starts;
    tail.groups = s.G; tail.max_prefix_pages = s.max_prefix_pages; tail.B = s.B;
    tail.prefix_tiles = (unsigned)p.prefix.row_tiles; tail.prefix_splits = p.prefix.splits; tail.slots = p.slots;
    tail.least = kSplitTiles; tail.whole = p.whole;
    const unsigned shape = (unsigned)p.own.row_tiles << 8 | (unsigned)(p.own.splits - 1) << 2 | (unsigned)(s.page_log2 - 4);
    auto part = [&](int rg, long prefix_wgs, long own_wgs) {
        tail.prefix_wgs = eights(prefix_wgs); tail.own_wgs = (unsigned)own_wgs;
        const unsigned grid = tail.prefix_wgs + eights(own_wgs);
        auto go = [&](auto attends) { return attends(a, tail, rg, grid, (unsigned)prefix_wgs, shape, stream); };
        return s.d == 128 ? (s.fp8 ? go(attend<128, true>) : go(attend<128, false>)) : (s.fp8 ? go(attend<64, true>) : go(attend<64, false>));
    };
    hipError_t e;
    if (p.whole || p.prefix.rg == p.own.rg) {
        e = part(p.own.rg, p.prefix.wgs, p.own.wgs);
    } else {
        e = part(p.prefix.rg, p.prefix.wgs, 0);
        if (e == hipSuccess) e = part(p.own.rg, 0, p.own.wgs);
    }
    if (e != hipSuccess || p.whole) return e;
    const int parts = p.slots > 16 ? 4 : p.slots > 8 ? 2 : 1;
    const unsigned per_wg = 256 / (s.d / 4) / parts;
    const dim3 grid((unsigned)((rows + per_wg - 1) / per_wg));
    const SharedMerge m{a.kv_lens, a.group_starts, a.prefix_lens, tail.O, (s.H / s.Hkv) * s.n, s.Hkv, s.max_pages, s.max_prefix_pages, s.G, s.page_log2, p.own.splits,
                        p.prefix.splits};
    auto merge = [&](auto kernel) { return launch(kernel, grid, dim3(256), stream, tail.part_ml, tail.part_o, p.slots, (int)rows, m); };
    return s.d == 128 ? (parts == 4 ? merge(shared_merge_kernel<128, 4>) : parts == 2 ? merge(shared_merge_kernel<128, 2>) : merge(shared_merge_kernel<128, 1>))
                      : (parts == 4 ? merge(shared_merge_kernel<64, 4>) : parts == 2 ? merge(shared_merge_kernel<64, 2>) : merge(shared_merge_kernel<64, 1>));
}

}  // namespace dd
