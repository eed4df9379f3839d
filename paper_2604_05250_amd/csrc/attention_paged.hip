// Attention over a paged cache: the merge of splits, and how a call is shared out.  The kernel is in attention_paged.h.
#include "attention_paged.h"

namespace dd {
namespace {

// The splits' states of a row, merged by D / 4 lanes; rows whose sequence took one split are finished already.
// The first states are asked for before it is known how many of them there are (one token, 4 x 4096 keys 12.1 -> 11.5 us with this and
// with leading scalar arguments, as above).
template <int D>
__global__ __launch_bounds__(256) void paged_merge_kernel(const float *part_ml, const float *part_o, const int32_t *kv_lens, uint8_t *O, int Hkv, int rows_total,
                                                          int max_pages, unsigned shape, unsigned launched, int rows)
{
    constexpr int LANES = D / 4;
    const int row = blockIdx.x * (256 / LANES) + threadIdx.x / LANES, d0 = (threadIdx.x % LANES) * 4;
    if (row >= rows) return;
    const int splits = (int)(shape >> 2 & 63) + 1;
    const float2 *ml = reinterpret_cast<const float2 *>(part_ml) + (size_t)row * splits;
    const floatx4 *po = reinterpret_cast<const floatx4 *>(part_o + (size_t)row * splits * D + d0);
    constexpr int U = 8;                             // states on their way: a round trip to memory for eight of them
    float2 st[U];
    floatx4 v[U];
    auto fetch = [&](int s0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int s = min(s0 + u, splits - 1);
            st[u] = ml[s];
            v[u] = po[(size_t)s * (D / 4)];
        }
    };
    fetch(0);
    const unsigned b = (unsigned)row / (unsigned)rows_total / (unsigned)Hkv;
    const int used = share_of(kv_lens[b], max_pages, 4 + (int)(shape & 3), splits, rows_total, launched).used;
    if (used <= 1) return;
    float M = kNone, L = 0;
    floatx4 x = {0, 0, 0, 0};
    for (int s0 = 0;;) {
        float top = M;
#pragma unroll
        for (int u = 0; u < U; ++u) top = fmaxf(top, s0 + u < used ? st[u].x : M);
        const float by = __builtin_amdgcn_exp2f(M - top);
        M = top;
        L *= by;
        x *= by;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (s0 + u < used) {
                const float f = __builtin_amdgcn_exp2f(st[u].x - M);
                L += f * st[u].y;
                x += f * v[u];
            }
        }
        s0 += U;
        if (s0 >= used) break;
        fetch(s0);
    }
    const float inv = L > 0 ? 1.0f / L : 0.0f;
    *reinterpret_cast<uint2 *>(O + ((size_t)row * D + d0) * 2) = make_uint2(pack_bf16(x[0] * inv, x[1] * inv), pack_bf16(x[2] * inv, x[3] * inv));
}

struct Plan { int rg, splits; long row_tiles, wgs; bool long_splits; };      // splits: at most kMaxSplits, row tiles: less than 2^24
Plan plan_of(int n, int B, int H, int Hkv, long capacity, bool fp8)
{
    const long rows = (long)(H / Hkv) * n, heads = (long)B * Hkv, blocks = heads * ((rows + 31) / 32), tiles = capacity / 64;
    const bool few = rows <= kFewRows;               // no two workgroups read the same keys: memory bounds them
    Plan p;
    // Two or four row blocks per workgroup read the cache once for all, but the workgroups are fewer and their waves wait for each other.
    // 256 compute units hold two workgroups each, so that up to 512 of one block run at once; bf16 pages wait for memory sooner.
    // us with one / two / four row blocks, unsplit, by blocks x positions:
    //     e4m3    128 x 2048    15.5 / 25.2 / -           bf16    256 x 1024    14.6 / 19.3 / -
    //             512 x 2048    25.0 / 27.1 / 46.1                320 x 2048    28.8 / 32.0 / -
    //            1024 x 2048    45.5 / 40.0 / 46.6                512 x 4096    75.5 / 68.0 / 104
    //            1536 x 2048    73.9 / 62.2 / 65.6               1024 x 2048    76.3 / 50.7 / 57.3
    //            1920 x 2048    91.5 / 78.2 / 75.5               1152 x 2048    89.5 / 74.5 / 71.0
    //            8192 x 2048     335 /  290 /  272               2048 x 1024    80.0 / 56.5 / 50.0
    // Where a workgroup's last rows are missing, their work is not: 320 rows of 128 heads, 700 positions 35.3 / 32.6 / 34.7.
    const bool full = (rows + 127) / 128 * 128 * 8 <= rows * 9;
    p.rg = few || blocks <= (fp8 ? 512 : 256) ? 1 : full && blocks > (fp8 ? 1792 : 1024) ? 4 : 2;
    p.row_tiles = (rows + 32 * p.rg - 1) / (32 * p.rg);
    const long base = heads * p.row_tiles;
    // Splits: the merge's launch costs some 1.5 us and each split a state per row, written and read again, for 32 rows as many bytes as a
    // tile of 64 keys; so up to one workgroup per compute unit, and up to two where arithmetic bounds them and the splits stay long.
    // us with 1 / 2 / 4 / 8 / 16 splits, 32/8 heads, e4m3, by sequences x positions:
    //     one token    1 x 512      6.1 /  7.4 /  7.4 / - / -         64 tokens    1 x 1024     9.9 / 10.7 / 10.8 / - / -
    //                  1 x 1024     8.6 /  8.6 /  7.4 / - / -                      1 x 1500    12.5 / 12.3 / 11.8 / - / -
    //                  1 x 4096    22.2 / 15.6 / 11.0 / 8.8 / 8.4                  1 x 2048    14.8 / 13.1 / 12.0 / - / -
    //                  4 x 4096    25.1 / 17.5 / 12.7 / 11.3 / 13.1                1 x 16384   83.2 / 47.6 / 29.1 / 28.9 / 33.8
    //                 24 x 4096    35.2 / 40.9 / 39.5 / 42.3 / -                   3 x 2048    16.1 / 20.6 / 23.9 / - / -
    //                                                                              3 x 8192    46.6 / 42.9 / 41.1 / 46.0 / -
    //                                                                              4 x 2048    16.3 / 22.8 / 26.1 / - / -
    //                                                                              4 x 8192    47.7 / 48.3 / 51.3 / 59.6 / -
    // Calls a little past one or two workgroups per compute unit wait for the few that share one: 264 of 3937 positions 34.1 / 38.5 / 37.9 / - / -.
    auto up_to = [&](long want, long least) { return want < tiles / least ? want : tiles / least; };
    long s = p.rg == 1 ? up_to(kUnits / base, kSplitTiles) : 1;
    if (!few && p.rg < 4) {
        const long twice = up_to(2 * kUnits / base, kSplitTilesShared);
        s = s > twice ? s : twice;
    }
    if (capacity < (few ? 1024 : 1200)) s = 1;
    if (s > kMaxSplits) s = kMaxSplits;
    p.splits = s < 1 ? 1 : (int)s;
    p.wgs = base * p.splits;
    p.long_splits = !few && p.wgs > kUnits && p.splits > 1 && base % 8 == 0;
    return p;
}

unsigned launched_of(const Plan &p) { return (unsigned)p.wgs | (p.long_splits ? kLongSplits : 0u); }       // (fewer than 2^24)

template <int D, bool FP8, int NT, bool ONE> hipError_t attend(const PagedAttnArgs &a, const PagedTail &tail, const Plan &p, unsigned shape, hipStream_t stream)
{
    auto run = [&](auto kernel) {
        return launch(kernel, dim3((unsigned)p.wgs), dim3(256), stream, a.table, a.kv_lens, static_cast<const uint8_t *>(a.Kc), static_cast<const uint8_t *>(a.Vc), a.Hkv,
                      (a.H / a.Hkv) * a.n, a.num_pages, a.max_pages, launched_of(p), shape, tail);
    };
    return p.rg == 1 ? run(attn_paged_kernel<D, FP8, NT, ONE, 1, PagedTail>) : p.rg == 2 ? run(attn_paged_kernel<D, FP8, NT, ONE, 2, PagedTail>) : run(attn_paged_kernel<D, FP8, NT, ONE, 4, PagedTail>);
}
template <int D, bool FP8> hipError_t attend(const PagedAttnArgs &a, const PagedTail &tail, const Plan &p, unsigned shape, hipStream_t stream)
{
    constexpr int NT = FP8 ? 2 : 1;                  // (bf16 pieces take twice the registers)
    return (1 << a.page_log2) >= 32 * NT ? attend<D, FP8, NT, true>(a, tail, p, shape, stream) : attend<D, FP8, NT, false>(a, tail, p, shape, stream);
}

}  // namespace

size_t paged_attention_workspace_bytes(int n, int B, int H, int Hkv, int d, long capacity, bool fp8)
{
    const Plan p = plan_of(n, B, H, Hkv, capacity, fp8);
    return p.splits <= 1 ? 0 : (size_t)B * H * n * (size_t)p.splits * (size_t)(d + 2) * sizeof(float);
}

hipError_t launch_attention_paged(const PagedAttnArgs &a, hipStream_t stream)
{
    const bool fp8 = a.k_scale != nullptr;
    const Plan p = plan_of(a.n, a.B, a.H, a.Hkv, (long)a.max_pages << a.page_log2, fp8);
    const size_t rows = (size_t)a.B * a.H * a.n;
    const PagedTail tail{static_cast<const uint8_t *>(a.Q), a.k_scale, a.v_scale, static_cast<uint8_t *>(a.O), static_cast<float *>(a.workspace),
                         static_cast<float *>(a.workspace) + rows * p.splits * a.d, (float)(1.4426950408889634 / __builtin_sqrt((double)a.d))};
    const unsigned shape = (unsigned)p.row_tiles << 8 | (unsigned)(p.splits - 1) << 2 | (unsigned)(a.page_log2 - 4);
    const hipError_t e = a.d == 128 ? (fp8 ? attend<128, true>(a, tail, p, shape, stream) : attend<128, false>(a, tail, p, shape, stream))
                                    : (fp8 ? attend<64, true>(a, tail, p, shape, stream) : attend<64, false>(a, tail, p, shape, stream));
    if (e != hipSuccess || p.splits <= 1) return e;
    const unsigned per_wg = 256 / (a.d / 4);
    const dim3 grid((unsigned)((rows + per_wg - 1) / per_wg));
    auto merge = [&](auto kernel) {
        return launch(kernel, grid, dim3(256), stream, tail.part_ml, tail.part_o, a.kv_lens, tail.O, a.Hkv, (a.H / a.Hkv) * a.n, a.max_pages, shape,
                      launched_of(p), (int)rows);
    };
    return a.d == 128 ? merge(paged_merge_kernel<128>) : merge(paged_merge_kernel<64>);
}

}  // namespace dd
