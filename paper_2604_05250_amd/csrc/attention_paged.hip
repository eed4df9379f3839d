// Attention over a paged cache (the drafter's call of Sec. 2.3 on a cache that is kept in pages), bf16 pages or e4m3 pages with one scale
// per page and head.
//     O = softmax(Q K^T / sqrt(d_k)) V   (Eq. 3)   over the keys that a sequence holds
// S^T = K Q^T and O^T = V^T P^T on 32x32x16 matrix instructions, a tile of 64 keys at a time.  The cache is laid out for them: a lane's
// operand of the first product is 16-byte pieces of one key's row, of the second one 16 keys of one head dim, which lie side by side
// in a page, so both go from memory to registers without LDS, and the tile's keys are dealt to the rows of S^T in such a way that the
// weights that a lane gets are the ones that it has to give to the second product:
//     lane half h, score tile T (0, 1), accumulator i (0 .. 15)  <->  key 32 h + 16 T + i of the tile
// A unit of 16 keys (h, T) lies in one page whatever the page size, so its page and its scales are one value per lane and T.
// Every wave takes every fourth tile with a state (reference, sum, O) of its own; the states are merged through LDS at the end, the
// key range is split over workgroups where those are few, and the splits' states are merged by a second kernel.
// e4m3 codes become bf16 exactly in registers; k_scale goes into the factor of the exponent, v_scale onto the weights before they are
// rounded to bf16 (bf16 for its range: scales span 2^-126 .. 2^119).
#include "attention_common.h"
#include "dd_internal.h"

namespace dd {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr float kNone = -1.0e30f;        // the reference of a row that has met no key
constexpr float kRaise = 8.0f;           // a reference is raised when a score is this far above it (log2 units)
constexpr int kMaxSplits = 64;

__device__ __forceinline__ unsigned pack_bf16(float lo, float hi)
{
    floatx2 f = {lo, hi};
    return __builtin_bit_cast(unsigned, __builtin_convertvector(f, bf16x2));
}
__device__ __forceinline__ bf16x8 decode8(unsigned w0, unsigned w1)                  // eight e4m3 codes, exactly
{
    const u32x4 r = {__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, 1.0f, false)),
                     __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, 1.0f, true)),
                     __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, 1.0f, false)),
                     __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, 1.0f, true))};
    return __builtin_bit_cast(bf16x8, r);
}
// fragment `f` (eight elements) of a lane's consecutive elements
template <bool FP8> __device__ __forceinline__ bf16x8 fragment(const u32x4 *raw, int f)
{
    if constexpr (FP8) return decode8(raw[f / 2][(f % 2) * 2], raw[f / 2][(f % 2) * 2 + 1]);
    else return __builtin_bit_cast(bf16x8, raw[f]);
}
__device__ __forceinline__ float halves_max(float x) { return fmaxf(x, __shfl_xor(x, 32)); }

struct PagedKernelArgs {
    const uint8_t *Q, *Kc, *Vc;
    const int32_t *table, *kv_lens;
    const float *k_scale, *v_scale;
    uint8_t *O;
    float *part_o, *part_ml;             // [rows][splits][d], [rows][splits][2]
    int Hkv, rows_total, num_pages, max_pages, page_log2, row_tiles, splits, wgs;
    float scale_log2;                    // log2(e) / sqrt(d)
};

// How a sequence's tiles are shared out over the splits of a call: tiles per split and splits that have any.
struct Share { int tiles, per_split, used, len; };
__device__ __forceinline__ Share share_of(int len, int max_pages, int page_log2, int splits)
{
    Share s;
    const long most = (long)max_pages << page_log2;
    s.len = len < 0 ? 0 : (long)len > most ? (int)most : len;
    s.tiles = (int)(((unsigned)s.len + 63u) >> 6);
    s.per_split = (s.tiles + splits - 1) / splits;
    s.used = s.tiles == 0 ? 0 : (s.tiles + s.per_split - 1) / s.per_split;
    return s;
}

template <int D, bool FP8, int RB, int W>
__global__ __launch_bounds__(64 * W, RB == 1 && (FP8 || D == 64) ? 2 : 1) void attn_paged_kernel(PagedKernelArgs a)
{
    constexpr int EB = FP8 ? 1 : 2;
    constexpr int ROWB = D * EB;                     // bytes per key
    constexpr int KR = ROWB / 2 / 16;                // 16-byte pieces of a lane's half of a key
    constexpr int VR = EB;                           // 16-byte pieces of a unit's 16 keys of one head dim
    constexpr int DT = D / 32, KS = D / 16;          // head-dim tiles, k steps of S
    constexpr int ROWS = 32 * RB, PITCH = D + 4;
    __shared__ __attribute__((aligned(16))) float o_sh[W][ROWS][PITCH];
    __shared__ float ml_sh[W][2][ROWS];

    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    unsigned bid = blockIdx.x;
    {                                                // workgroups that share keys: on one XCD
        const unsigned total = a.wgs, per = total >> 3, rem = total & 7;
        const unsigned xcd = bid & 7, slot = bid >> 3;
        bid = xcd * per + min(xcd, rem) + slot;
    }
    const int rt = bid % (unsigned)a.row_tiles; bid /= (unsigned)a.row_tiles;
    const int sp = bid % (unsigned)a.splits; bid /= (unsigned)a.splits;
    const int head = bid, b = head / a.Hkv, g = head - b * a.Hkv;
    const Share sh = share_of(uniform_load(a.kv_lens + b), a.max_pages, a.page_log2, a.splits);
    if (sp >= sh.used && sp > 0) return;
    const int v_first = rt * ROWS;
    const size_t row_base = (size_t)head * a.rows_total;

    // ---- queries: of row l32 of each block, half of the head dims
    bf16x8 q[RB][KS];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int r = min(v_first + rb * 32 + l32, a.rows_total - 1);
        const u32x4 *p = reinterpret_cast<const u32x4 *>(a.Q + (row_base + r) * (D * 2) + hh * D);
#pragma unroll
        for (int s = 0; s < KS; ++s) q[rb][s] = __builtin_bit_cast(bf16x8, p[s]);
    }

    const int t_end = min((sp + 1) * sh.per_split, sh.tiles);
    int t = sp * sh.per_split + wave;
    const int32_t *const row_of_table = a.table + (size_t)b * a.max_pages;
    const int P_log2 = a.page_log2;
    const unsigned in_page = (1u << P_log2) - 1;
    const int kh = (l32 >> 2) & 1;                   // half of the tile that row l32 of S^T is in
    const int kslot = ((l32 >> 4) & 1) * 8 + ((l32 >> 3) & 1) * 4 + (l32 & 3);     // its key within a unit

    struct Pages { int id[4]; };
    auto pages_of = [&](int tile) __attribute__((always_inline)) {
        Pages p;
#pragma unroll
        for (int u = 0; u < 4; ++u) p.id[u] = uniform_load(row_of_table + min((tile * 4 + u) >> (P_log2 - 4), a.max_pages - 1));
        return p;
    };
    auto valid = [&](int id) __attribute__((always_inline)) { return (unsigned)id < (unsigned)a.num_pages; };
    auto place = [&](int id) __attribute__((always_inline)) { return (size_t)((valid(id) ? id : 0) * (long)a.Hkv + g); };      // page and head

    u32x4 kraw[2][KR], vraw[DT][2][VR];
    auto load_k = [&](const Pages &p, int tile) __attribute__((always_inline)) {
#pragma unroll
        for (int T = 0; T < 2; ++T) {
            const size_t pl = kh ? place(p.id[2 + T]) : place(p.id[T]);
            const unsigned off = ((unsigned)(tile * 64) + 32 * kh + 16 * T) & in_page;
            const u32x4 *src = reinterpret_cast<const u32x4 *>(a.Kc + ((pl << P_log2) + off + kslot) * ROWB + hh * (ROWB / 2));
#pragma unroll
            for (int i = 0; i < KR; ++i) kraw[T][i] = src[i];
        }
    };
    auto load_v = [&](const Pages &p, int tile) __attribute__((always_inline)) {
#pragma unroll
        for (int T = 0; T < 2; ++T) {
            const size_t pl = hh ? place(p.id[2 + T]) : place(p.id[T]);
            const unsigned off = ((unsigned)(tile * 64) + 32 * hh + 16 * T) & in_page;
            const uint8_t *src = a.Vc + (((pl * D + l32) << P_log2) + off) * EB;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int i = 0; i < VR; ++i)
                    vraw[dt][T][i] = reinterpret_cast<const u32x4 *>(src + (((size_t)dt * 32) << P_log2) * EB)[i];
        }
    };

    floatx16 o[RB][DT];
    float m[RB], l[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        m[rb] = kNone;
        l[rb] = 0;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[rb][dt][i] = 0;
    }

    Pages now, next;
    float ks[2], vs[2], ks_next[2], vs_next[2];
    auto load_scales = [&](const Pages &p, float *k, float *v) __attribute__((always_inline)) {
        if constexpr (FP8) {
#pragma unroll
            for (int T = 0; T < 2; ++T) {
                const float k0 = uniform_load(a.k_scale + place(p.id[T])), k1 = uniform_load(a.k_scale + place(p.id[2 + T]));
                const float v0 = uniform_load(a.v_scale + place(p.id[T])), v1 = uniform_load(a.v_scale + place(p.id[2 + T]));
                k[T] = hh ? k1 : k0;
                v[T] = hh ? v1 : v0;
            }
        }
    };
    if (t < t_end) {
        now = pages_of(t);
        load_k(now, t);
        load_v(now, t);
        load_scales(now, ks, vs);
        next = pages_of(t + W);
    }
    for (; t < t_end; t += W) {
        const bool more = t + W < t_end;
        // ---- scores
        floatx16 s[RB][2];
#pragma unroll
        for (int T = 0; T < 2; ++T)
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[rb][T][i] = 0;
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int T = 0; T < 2; ++T) {
                const bf16x8 f = fragment<FP8>(kraw[T], k);
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) s[rb][T] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, q[rb][k], s[rb][T], 0, 0, 0);
            }
        if (more) {
            load_k(next, t + W);
            load_scales(next, ks_next, vs_next);
        }
        // ---- the last tile's end, and units without a page: their keys take no part
        const bool whole = t * 64 + 64 <= sh.len && valid(now.id[0]) && valid(now.id[1]) && valid(now.id[2]) && valid(now.id[3]);
        float c[2];
#pragma unroll
        for (int T = 0; T < 2; ++T) c[T] = FP8 ? a.scale_log2 * ks[T] : a.scale_log2;
        if (!whole) {
#pragma unroll
            for (int T = 0; T < 2; ++T) {
                const bool there = hh ? valid(now.id[2 + T]) : valid(now.id[T]);
                const int left = there ? sh.len - (t * 64 + 32 * hh + 16 * T) : 0;      // keys of the unit that count
                if (left <= 0) {
                    c[T] = 1.0f;
                    if (FP8) vs[T] = 1.0f;
                }
#pragma unroll
                for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[rb][T][i] = i < left ? s[rb][T][i] : -__builtin_inff();
                // what lies there may be no number, and 0 times it would be none
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                    for (int w = 0; w < 4 * VR; ++w) {
                        constexpr int PER = 4 / EB;
                        const int n = left - w * PER;
                        const unsigned keep = n >= PER ? ~0u : n <= 0 ? 0u : (1u << (n * 8 * EB)) - 1;
                        vraw[dt][T][w / 4][w % 4] &= keep;
                    }
            }
        }
        // ---- weights
        bf16x8 p[RB][4];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            float mx[2];
#pragma unroll
            for (int T = 0; T < 2; ++T) {
                mx[T] = s[rb][T][0];
#pragma unroll
                for (int i = 1; i < 16; ++i) mx[T] = fmaxf(mx[T], s[rb][T][i]);
                mx[T] *= c[T];
            }
            const float top = halves_max(fmaxf(mx[0], mx[1]));
            if (__any(top > m[rb] + kRaise)) {
                const float to = fmaxf(top, m[rb]), by = __builtin_amdgcn_exp2f(m[rb] - to);
                m[rb] = to;
                l[rb] *= by;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[rb][dt][i] *= by;
            }
#pragma unroll
            for (int T = 0; T < 2; ++T) {
                float w[16], sum = 0;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    w[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rb][T][i], c[T], -m[rb]));
                    sum += w[i];
                    if constexpr (FP8) w[i] *= vs[T];
                }
                l[rb] += sum;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const u32x4 r = {pack_bf16(w[8 * j], w[8 * j + 1]), pack_bf16(w[8 * j + 2], w[8 * j + 3]),
                                     pack_bf16(w[8 * j + 4], w[8 * j + 5]), pack_bf16(w[8 * j + 6], w[8 * j + 7])};
                    p[rb][2 * T + j] = __builtin_bit_cast(bf16x8, r);
                }
            }
        }
        // ---- output
#pragma unroll
        for (int T = 0; T < 2; ++T)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    const bf16x8 f = fragment<FP8>(vraw[dt][T], j);
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) o[rb][dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, p[rb][2 * T + j], o[rb][dt], 0, 0, 0);
                }
        if (more) {
            load_v(next, t + W);
            now = next;
            if constexpr (FP8) {
#pragma unroll
                for (int T = 0; T < 2; ++T) { ks[T] = ks_next[T]; vs[T] = vs_next[T]; }
            }
            next = pages_of(t + 2 * W);
        }
    }

    // ---- the waves' states, merged: every thread finishes eight head dims of a row at a time
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        l[rb] += __shfl_xor(l[rb], 32);
        if (hh == 0) {
            ml_sh[wave][0][rb * 32 + l32] = m[rb];
            ml_sh[wave][1][rb * 32 + l32] = l[rb];
        }
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<float4 *>(&o_sh[wave][rb * 32 + l32][dt * 32 + 8 * i + 4 * hh]) =
                    make_float4(o[rb][dt][4 * i], o[rb][dt][4 * i + 1], o[rb][dt][4 * i + 2], o[rb][dt][4 * i + 3]);
    }
    __syncthreads();
    for (int u = tid; u < ROWS * (D / 8); u += 64 * W) {
        const int r = u / (D / 8), d0 = (u % (D / 8)) * 8;
        if (v_first + r >= a.rows_total) break;
        float M = ml_sh[0][0][r];
#pragma unroll
        for (int w = 1; w < W; ++w) M = fmaxf(M, ml_sh[w][0][r]);
        float L = 0, x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float f = __builtin_amdgcn_exp2f(ml_sh[w][0][r] - M);
            L += f * ml_sh[w][1][r];
            const float4 lo = *reinterpret_cast<const float4 *>(&o_sh[w][r][d0]), hi = *reinterpret_cast<const float4 *>(&o_sh[w][r][d0 + 4]);
            x[0] += f * lo.x; x[1] += f * lo.y; x[2] += f * lo.z; x[3] += f * lo.w;
            x[4] += f * hi.x; x[5] += f * hi.y; x[6] += f * hi.z; x[7] += f * hi.w;
        }
        const size_t row = row_base + v_first + r;
        if (sh.used <= 1) {
            const float inv = L > 0 ? 1.0f / L : 0.0f;       // no key at all: zeros
            *reinterpret_cast<uint4 *>(a.O + (row * D + d0) * 2) = make_uint4(pack_bf16(x[0] * inv, x[1] * inv), pack_bf16(x[2] * inv, x[3] * inv),
                                                                             pack_bf16(x[4] * inv, x[5] * inv), pack_bf16(x[6] * inv, x[7] * inv));
        } else {
            float *to = a.part_o + (row * a.splits + sp) * D + d0;
            *reinterpret_cast<float4 *>(to) = make_float4(x[0], x[1], x[2], x[3]);
            *reinterpret_cast<float4 *>(to + 4) = make_float4(x[4], x[5], x[6], x[7]);
            if (d0 == 0) {
                a.part_ml[(row * a.splits + sp) * 2] = M;
                a.part_ml[(row * a.splits + sp) * 2 + 1] = L;
            }
        }
    }
}

// The splits' states of a row, merged by D / 4 lanes; rows whose sequence took one split are finished already.
template <int D> __global__ __launch_bounds__(256) void paged_merge_kernel(PagedKernelArgs a, int rows)
{
    constexpr int LANES = D / 4;
    const int row = blockIdx.x * (256 / LANES) + threadIdx.x / LANES, d0 = (threadIdx.x % LANES) * 4;
    if (row >= rows) return;
    const int b = row / a.rows_total / a.Hkv;
    const int used = share_of(a.kv_lens[b], a.max_pages, a.page_log2, a.splits).used;
    if (used <= 1) return;
    const float *ml = a.part_ml + (size_t)row * a.splits * 2, *po = a.part_o + (size_t)row * a.splits * D + d0;
    float M = kNone;
    for (int s = 0; s < used; ++s) M = fmaxf(M, ml[2 * s]);
    float L = 0, x[4] = {0, 0, 0, 0};
    for (int s = 0; s < used; ++s) {
        const float f = __builtin_amdgcn_exp2f(ml[2 * s] - M);
        L += f * ml[2 * s + 1];
        const float4 v = *reinterpret_cast<const float4 *>(po + (size_t)s * D);
        x[0] += f * v.x; x[1] += f * v.y; x[2] += f * v.z; x[3] += f * v.w;
    }
    const float inv = L > 0 ? 1.0f / L : 0.0f;
    *reinterpret_cast<uint2 *>(a.O + ((size_t)row * D + d0) * 2) = make_uint2(pack_bf16(x[0] * inv, x[1] * inv), pack_bf16(x[2] * inv, x[3] * inv));
}

struct Plan { int rb, splits; long row_tiles, wgs; };
Plan plan_of(int n, int B, int H, int Hkv, long capacity)
{
    const long rows = (long)(H / Hkv) * n, heads = (long)B * Hkv;
    Plan p;
    p.rb = rows > 64 ? 2 : 1;
    p.row_tiles = (rows + 32 * p.rb - 1) / (32 * p.rb);
    const long base = heads * p.row_tiles, target = p.rb == 1 ? 512 : 256;
    long s = (target + base - 1) / base;
    const long most = capacity / 256;                // a tile for each wave of a split
    if (s > most) s = most;
    if (s > kMaxSplits) s = kMaxSplits;
    p.splits = s < 1 ? 1 : (int)s;
    p.wgs = base * p.splits;
    return p;
}

template <int D, bool FP8> hipError_t attend(const PagedKernelArgs &k, const Plan &p, hipStream_t stream)
{
    return p.rb == 1 ? launch(attn_paged_kernel<D, FP8, 1, 4>, dim3((unsigned)p.wgs), dim3(256), stream, k)
                     : launch(attn_paged_kernel<D, FP8, 2, 4>, dim3((unsigned)p.wgs), dim3(256), stream, k);
}

}  // namespace

size_t paged_attention_workspace_bytes(int n, int B, int H, int Hkv, int d, long capacity, bool fp8)
{
    (void)fp8;
    const Plan p = plan_of(n, B, H, Hkv, capacity);
    return p.splits <= 1 ? 0 : (size_t)B * H * n * (size_t)p.splits * (size_t)(d + 2) * sizeof(float);
}

hipError_t launch_attention_paged(const PagedAttnArgs &a, hipStream_t stream)
{
    const Plan p = plan_of(a.n, a.B, a.H, a.Hkv, (long)a.max_pages << a.page_log2);
    const size_t rows = (size_t)a.B * a.H * a.n;
    const bool fp8 = a.k_scale != nullptr;
    PagedKernelArgs k{static_cast<const uint8_t *>(a.Q), static_cast<const uint8_t *>(a.Kc), static_cast<const uint8_t *>(a.Vc), a.table, a.kv_lens,
                      a.k_scale, a.v_scale, static_cast<uint8_t *>(a.O), static_cast<float *>(a.workspace),
                      static_cast<float *>(a.workspace) + rows * p.splits * a.d, a.Hkv, (a.H / a.Hkv) * a.n, a.num_pages, a.max_pages, a.page_log2,
                      (int)p.row_tiles, p.splits, (int)p.wgs, (float)(1.4426950408889634 / __builtin_sqrt((double)a.d))};
    const hipError_t e = a.d == 128 ? (fp8 ? attend<128, true>(k, p, stream) : attend<128, false>(k, p, stream))
                                    : (fp8 ? attend<64, true>(k, p, stream) : attend<64, false>(k, p, stream));
    if (e != hipSuccess || p.splits <= 1) return e;
    const unsigned per_wg = 256 / (a.d / 4);
    const dim3 grid((unsigned)((rows + per_wg - 1) / per_wg));
    return a.d == 128 ? launch(paged_merge_kernel<128>, grid, dim3(256), stream, k, (int)rows) : launch(paged_merge_kernel<64>, grid, dim3(256), stream, k, (int)rows);
}

}  // namespace dd
