// What happens to a projection's rows before attention (Sec. 2.2, Sec. 2.3): head norms, the rotation by position, and the way of
// keys and values into a paged cache.
//
//   norm      y = x / sqrt(mean(x^2) + eps) * w                             over the d elements of one head
//   rotation  (u, v) -> (u cos a - v sin a, v cos a + u sin a),  a = position * inv_freq[k],  for the pair k of the first rot dims
//   e4m3      code = rne(x / s), s = 2^e: one scale per page and head
//
// A row of d elements belongs to d / 16 lanes, each with two chunks of eight elements (16-byte accesses in bf16).  The chunks of a lane
// are chosen so that the two members of every pair are in one lane, and so a rotation needs no exchange; and so that the first chunks of
// the lanes lie side by side, and the second ones.  (Both of a lane side by side - every other piece of a row for each load and store -
// made the pairing of neighbours slower: 4 x 2046 rows of 64 heads of 64, fp32, 122 us, 13 x 2613 of 32 heads of 128, bf16, 178.)
// Angles: position * inv_freq in revolutions, in fp64, and its distance from the nearest whole one to fp32 (a product in fp32 is off by
// 2^-24 of the angle: a hundredth of a radian at position 130000).  Where a result is bf16, the hardware's sine and cosine, which take
// revolutions and are off by 2^-23 (measured over [0, 1] against fp64), and its reciprocal root: far below its half step of 2^-8.  Where
// fp32 arithmetic shows - fp32 rows, and e4m3 pages, on which a key next to a border between two codes goes the other way as often as its
// error is large - sine and cosine to a step of fp32, and the reciprocal root to half of one.
#include "attention_common.h"
#include "dd_internal.h"

#include <type_traits>

namespace dd {
namespace {

typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float bf16_lo(unsigned w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float bf16_hi(unsigned w) { return __builtin_bit_cast(float, w & 0xffff0000u); }

struct Bf16 { static constexpr int bytes = 2; };
struct F32 { static constexpr int bytes = 4; };

// eight consecutive elements as they are in memory
template <typename T> struct Chunk { u32x4 w[T::bytes / 2]; };
template <typename T> __device__ __forceinline__ Chunk<T> load_chunk(const uint8_t *row, int element)
{
    Chunk<T> c;
    const u32x4 *p = reinterpret_cast<const u32x4 *>(row + element * T::bytes);
#pragma unroll
    for (int i = 0; i < T::bytes / 2; ++i) c.w[i] = p[i];
    return c;
}
__device__ __forceinline__ void unpack(const Chunk<Bf16> &c, float *x)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = bf16_lo(c.w[0][i]); x[2 * i + 1] = bf16_hi(c.w[0][i]); }
}
__device__ __forceinline__ void unpack(const Chunk<F32> &c, float *x)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = as_float(c.w[i / 4][i % 4]);
}
template <typename T, bool STREAM> __device__ __forceinline__ void store_chunk(uint8_t *row, int element, const float *x)
{
    u32x4 *p = reinterpret_cast<u32x4 *>(row + element * T::bytes);
#pragma unroll
    for (int i = 0; i < T::bytes / 2; ++i) {
        u32x4 v;
        if constexpr (std::is_same<T, Bf16>::value) v = u32x4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
        else v = __builtin_bit_cast(u32x4, floatx4{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]});
        if constexpr (STREAM) __builtin_nontemporal_store(v, p + i);
        else p[i] = v;
    }
}

// exchanges among the 4 or 8 lanes of a row (lanes of one row are neighbours and start at a multiple of their number)
template <int CTRL> __device__ __forceinline__ float across(float x)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
template <int LANES> __device__ __forceinline__ float row_sum(float x)
{
    static_assert(LANES == 4 || LANES == 8, "a row is 64 or 128 elements");
    x += across<0xB1>(x);                                    // lane ^ 1
    x += across<0x4E>(x);                                    // lane ^ 2
    if (LANES == 8) x += across<0x141>(x);                   // mirrored within eight lanes: the other four
    return x;
}

struct Pairing {                                             // where a lane's two chunks are, and how they are paired
    int a, b;                                                // first elements
    int fa, fb;                                              // which angles: of the first four pairs, of the last four
    bool ta, tb;                                             // whether those turn
};
template <int D> __device__ __forceinline__ Pairing pairing(int lane, int rot, bool interleaved)
{
    Pairing p;
    if (interleaved) {                                       // pairs within a chunk
        p.a = 8 * lane;
        p.b = D / 2 + 8 * lane;
        p.ta = p.a < rot;
        p.tb = p.b < rot;
        p.fa = p.a / 2;
        p.fb = p.b / 2;
    } else {                                                 // chunk and chunk + rot / 2; what stays as it is behind them
        const int rest = 8 * lane - rot / 2;
        p.ta = p.tb = rest < 0;
        p.a = p.ta ? 8 * lane : rot + rest;
        p.b = p.ta ? rot / 2 + 8 * lane : rot + (D - rot) / 2 + rest;
        p.fa = 8 * lane;
        p.fb = 8 * lane + 4;
    }
    return p;
}

enum { kNoTurn = 0, kHalves = 1, kNeighbours = 2 };

// cos and sin of an angle within half a turn or so, off by little more than a step of fp32: the angle from the nearest quarter of a turn,
// rounded once, and the power series of both functions over an eighth of a turn on either side; what they leave out is under 2^-28.
__device__ __forceinline__ void cos_sin(double turns, float &c, float &s)
{
    const double quarters = 4.0 * turns, nearest = __builtin_rint(quarters);
    const float x = (float)(1.5707963267948966 * (quarters - nearest)), xx = x * x;
    const int q = (int)nearest;
    const float sn = __builtin_fmaf(x * xx, __builtin_fmaf(xx, __builtin_fmaf(xx, __builtin_fmaf(xx, 1.0f / 362880, -1.0f / 5040), 1.0f / 120), -1.0f / 6), x);
    const float cs = __builtin_fmaf(xx, __builtin_fmaf(xx, __builtin_fmaf(xx, __builtin_fmaf(xx, __builtin_fmaf(xx, -1.0f / 3628800, 1.0f / 40320), -1.0f / 720),
                                                                       1.0f / 24), -0.5f), 1.0f);
    c = as_float(__builtin_bit_cast(unsigned, (q & 1) ? sn : cs) ^ (unsigned)((q + 1) & 2) << 30);
    s = as_float(__builtin_bit_cast(unsigned, (q & 1) ? cs : sn) ^ (unsigned)(q & 2) << 30);
}
// cos and sin of the eight angles of a lane at a position; elements that stay as they are get 1 and 0.  EXACT: to a step of fp32; FAR: at
// positions past 2^30 too.  Relative error of fp32 rows against fp64, rms: 3.9e-8, with the hardware's functions 9.3e-8; codes that are not
// the exact ones' of 33 million normed keys on e4m3 pages: 32 and 80 (plain fp32 arithmetic: 45).  us exact / hardware: 4 x 2048 fp32 rows of
// 40 heads 62 / 75 (neighbours paired 64 / 64), 16 x 64 7.7 / 9.9 (7.6 / 7.0); append of 16 x 2048 rows of 8 heads to e4m3 pages 43.2 / 42.5,
// 16 x 64 5.9 / 5.7, 1 x 512 4.2 / 3.9, 11 x 16 4.5 / 4.5.
template <bool EXACT, bool FAR> __device__ __forceinline__ void turn_of(const float *inv_freq, const Pairing &p, double position, float *c, float *s)
{
    constexpr double kTurn = 0.15915494309189535, kTurnRest = -9.839338337591243e-18;        // 1 / 2 pi, and what the first number lacks
    const double q = position * kTurn;
    const float *const fa = inv_freq + (p.ta ? p.fa : 0), *const fb = inv_freq + (p.tb ? p.fb : 0);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const double f = (double)(i < 4 ? fa[i] : fb[i - 4]);
        float cs, sn;
        if constexpr (EXACT) {
            double turns, rest = 0.0;
            if constexpr (FAR) {
                const double a = position * f;                                               // (the product has 55 bits)
                turns = a * kTurn;
                rest = __builtin_fma(a, kTurn, -turns) + __builtin_fma(__builtin_fma(position, f, -a), kTurn, a * kTurnRest);
            } else {
                turns = f * q;
            }
            cos_sin((turns - __builtin_rint(turns)) + rest, cs, sn);
        } else {
            const double turns = f * q;
            const float r = (float)(turns - __builtin_rint(turns));
            cs = __builtin_amdgcn_cosf(r);
            sn = __builtin_amdgcn_sinf(r);
        }
        const bool turns = i < 4 ? p.ta : p.tb;
        c[i] = turns ? cs : 1.0f;
        s[i] = turns ? sn : 0.0f;
    }
}
template <int PAIR> __device__ __forceinline__ void rotate(float *x, const float *c, const float *s)     // x: both chunks, 16 values
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float &u = PAIR == kHalves ? x[i] : x[2 * i], &v = PAIR == kHalves ? x[8 + i] : x[2 * i + 1];
        const float u0 = u, v0 = v;
        u = u0 * c[i] - v0 * s[i];
        v = v0 * c[i] + u0 * s[i];
    }
}
// weights of a lane's elements, 1 where there are none; norm() of a row without weights leaves it as it is
template <typename T> __device__ __forceinline__ void weights_of(const void *weight, const Pairing &p, float *w)
{
    if (weight == nullptr) {
#pragma unroll
        for (int i = 0; i < 16; ++i) w[i] = 1.0f;
        return;
    }
    unpack(load_chunk<T>(static_cast<const uint8_t *>(weight), p.a), w);
    unpack(load_chunk<T>(static_cast<const uint8_t *>(weight), p.b), w + 8);
}
// EXACT: the root to half a step of fp32 or so, by a correction of the hardware's, and what the elements are to be multiplied by after their
// rotation, which leaves out a rounding of each (bf16 rows times bf16 weights are exact); else they are normed when it returns.
template <int D, bool EXACT> __device__ __forceinline__ float norm(float *x, const float *w, float eps, bool normed)
{
    if constexpr (EXACT) {
        float q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = __builtin_fmaf(x[2 * i + 1], x[2 * i + 1], x[2 * i] * x[2 * i]);
        const float m = __builtin_fmaf(row_sum<D / 16>(((q[0] + q[1]) + (q[2] + q[3])) + ((q[4] + q[5]) + (q[6] + q[7]))), 1.0f / D, eps);
        const float r = __builtin_amdgcn_rsqf(m), p = m * r, e = __builtin_fmaf(-p, r, 1.0f) - __builtin_fmaf(m, r, -p) * r;
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] *= w[i];
        return normed ? __builtin_fmaf(0.5f * r, e, r) : 1.0f;
    }
    float q = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) q += x[i] * x[i];
    const float root = __builtin_amdgcn_rsqf(row_sum<D / 16>(q) * (1.0f / D) + eps), r = normed ? root : 1.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = x[i] * r * w[i];
    return 1.0f;
}
template <bool EXACT> __device__ __forceinline__ void times(float *x, float r)
{
    if constexpr (EXACT) {
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] *= r;
    }
}

// ---------------------------------------------------------------- queries and keys for dense attention
// A lane keeps its place in the row and its token, and goes through `per_wg` heads: the angles and the weights are made once for all
// of them.  Reads and writes every row once: bound by memory where tokens are many.
// Every load and store of the loop is unconditional (the last heads' prefetch reads the last row again), so that a wave waits for one
// row's loads and not for all that are on their way.  Stores are non-temporal: 16 x 2048 rows of 40 heads 141 -> 137 us (4.9 TB/s read and
// written, what a copy reaches), 16 x 64 rows 7.0 -> 6.0; with dd_bidir_attention after it 1 x 1024 rows of 32 + 8 heads 31.3 -> 29.3, 1 x 4096
// of 32 + 32 224.5 -> 223.7, but 8 x 1024 of 32 + 32 168.5 -> 174.5, where all that is written would have stayed in the last cache.
template <typename T, int D, bool NORM, int PAIR>
__global__ __launch_bounds__(256) void norm_rotate_kernel(NormRotateArgs a)
{
    constexpr int LANES = D / 16, TOKENS = 256 / LANES;
    constexpr bool EXACT = std::is_same<T, F32>::value;
    constexpr int U = 4 / (T::bytes / 2);                    // heads on their way
    const int lane = threadIdx.x % LANES;
    const unsigned token = blockIdx.x * TOKENS + threadIdx.x / LANES;
    if (token >= a.tokens) return;                           // (whole rows: the lanes of a row stay together)
    const unsigned b = token / (unsigned)a.n, i = token - b * (unsigned)a.n;
    const bool is_q = (int)blockIdx.y < a.q_groups;
    const NormRotateSide &side = is_q ? a.q : a.k;
    const int first = ((int)blockIdx.y - (is_q ? 0 : a.q_groups)) * a.per_wg, count = min(a.per_wg, side.heads - first);
    const Pairing p = pairing<D>(lane, a.rot, PAIR == kNeighbours);

    const uint8_t *src = static_cast<const uint8_t *>(side.x) + ((long)b * side.batch + first * side.head + (long)i * side.row) * T::bytes;
    uint8_t *dst = static_cast<uint8_t *>(side.y) + (((long)b * side.heads + first) * a.n + i) * D * T::bytes;
    Chunk<T> in[U][2];
    auto fetch = [&](int h, int u) __attribute__((always_inline)) {
        const uint8_t *row = src + (long)min(h, count - 1) * side.head * T::bytes;
        in[u][0] = load_chunk<T>(row, p.a);
        in[u][1] = load_chunk<T>(row, p.b);
    };
#pragma unroll
    for (int u = 0; u < U; ++u) fetch(u, u);

    float w[16], c[8], s[8];
    if constexpr (NORM) weights_of<T>(side.weight, p, w);
    if constexpr (PAIR != kNoTurn) turn_of<EXACT, true>(a.inv_freq, p, a.positions != nullptr ? (double)a.positions[token] : (double)i, c, s);
    const bool normed = NORM && side.weight != nullptr;
    for (int h0 = 0; h0 < count; h0 += U) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float x[16];
            unpack(in[u][0], x);
            unpack(in[u][1], x + 8);
            fetch(h0 + U + u, u);
            float root = 1.0f;
            if constexpr (NORM) root = norm<D, EXACT>(x, w, a.eps, normed);
            if constexpr (PAIR != kNoTurn) rotate<PAIR>(x, c, s);
            if constexpr (NORM) times<EXACT>(x, root);
            if (h0 + u < count) {
                uint8_t *row = dst + (long)(h0 + u) * a.n * D * T::bytes;
                store_chunk<T, true>(row, p.a, x);
                store_chunk<T, true>(row, p.b, x + 8);
            }
        }
    }
}

// ---------------------------------------------------------------- keys and values into pages
__device__ __forceinline__ unsigned codes4(float a, float b, float c, float d)      // e4m3, to nearest even; |x| <= 448
{
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}
__device__ __forceinline__ unsigned regrown4(unsigned codes, float by)              // codes of `by` times the values that they stand for
{
    const floatx2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
    return codes4(lo[0] * by, lo[1] * by, hi[0] * by, hi[1] * by);
}
// The least power of two, 2^-126 at least, that 448 times is no less than a: 448 = 1.75 * 2^8.
__device__ __forceinline__ float scale_for(float a)
{
    const unsigned bits = __builtin_bit_cast(unsigned, a);
    const int e = (int)(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);  // its biased exponent
    return __builtin_bit_cast(float, (unsigned)(e < 1 ? 1 : e) << 23);
}
__device__ __forceinline__ float wave_largest(float x)       // over the 64 lanes of a wave
{
    typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
    x = fmaxf(x, across<0xB1>(x));
    x = fmaxf(x, across<0x4E>(x));
    x = fmaxf(x, across<0x141>(x));
    x = fmaxf(x, across<0x140>(x));                          // mirrored within sixteen lanes
    u32x2 r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    x = fmaxf(as_float(r[0]), as_float(r[1]));
    r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    return fmaxf(as_float(r[0]), as_float(r[1]));
}
struct Divide {                                              // x / s, by a product where that is the same number
    float s, inverse;
    bool exact;
    __device__ __forceinline__ explicit Divide(float scale) : s(scale), inverse(1.0f / scale), exact((__builtin_bit_cast(unsigned, scale) & 0x7fffffu) == 0) {}
    __device__ __forceinline__ void operator()(float *x) const
    {
        if (exact) {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] *= inverse;
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] /= s;
        }
    }
};

// One workgroup has one page of one sequence, its keys or its values, for `per_wg` heads one after the other, and one row per d / 16
// lanes: ROWS rows, all of the page or, where a call has no more than that for each sequence, the ones from its first new row on.  It is the only one that writes this page and these heads, so the page's scale, its old rows and its new ones are
// decided here without an atomic.  The rows stay in registers between the maximum over the page and their storage; the next head's are
// on their way meanwhile, and its angles and weights are this one's.
// Values are stored with the keys of one head dim side by side, and are turned over in LDS.
// Bound by memory: 16 x 2048 rows of 8 heads to e4m3 pages of 64 43 us, 4.7 TB/s read and written.
template <typename T, int D, int PAGE, int ROWS, bool FP8, bool VALUES>
__device__ __forceinline__ void append_page(const PageAppendArgs &a, unsigned bid, unsigned *turned, float *wave_max)
{
    constexpr int LANES = D / 16, THREADS = ROWS * LANES, WAVES = (THREADS + 63) / 64;
    constexpr int EB = FP8 ? 1 : 2;                          // bytes per stored element
    constexpr int PITCH = D * EB / 4 + 1;                    // words per row in LDS: an odd number
    constexpr int KEYS = 16 / EB, DIMS = 4 / EB;             // a thread stores KEYS values of DIMS head dims
    constexpr int JOBS = D / DIMS * (PAGE / KEYS), TURNS = (JOBS + THREADS - 1) / THREADS;
    const int tid = threadIdx.x, lane = tid % LANES;
    const int group = bid % a.head_groups;
    bid /= a.head_groups;
    const int b = bid / a.pages_per_seq, j = bid % a.pages_per_seq;

    // ---- which rows of the page this call writes, and which it finds there
    const long start = uniform_load(a.starts + b);
    const long rows = a.n_rows != nullptr ? min(max(uniform_load(a.n_rows + b), 0), a.n) : a.n;
    const long held = a.kv_lens != nullptr ? (long)uniform_load(a.kv_lens + b) : start;
    const long page_index = (start >> a.page_log2) + j, first = page_index * PAGE;       // first: position of the page's first row
    if (page_index < 0 || page_index >= a.max_pages) return;
    if (first >= start + rows || rows == 0) return;          // (first + PAGE > start: j >= 0)
    const int page = uniform_load(a.table + (long)b * a.max_pages + page_index);
    if (page < 0 || page >= a.num_pages) return;
    const long base = ROWS == PAGE || start < first ? first : start;                     // position of the first row that this workgroup has
    const int slot = (int)(base - first) + tid / LANES;      // (ROWS < PAGE: may be behind the page; nothing is written there)
    const long pos = first + slot;
    const bool written = slot < PAGE && pos >= start && pos < start + rows;
    const bool keeps = min(start, held) > first || min(held, first + PAGE) > start + rows;       // some row is kept

    const Pairing p = pairing<D>(lane, VALUES ? 0 : a.rot, a.interleaved);
    const PageAppendSide &side = VALUES ? a.v : a.k;
    const long r = written ? pos - start : (start > first ? 0 : first - start);          // (a row that exists)
    const uint8_t *src = static_cast<const uint8_t *>(side.x) + (b * side.batch + r * side.row) * T::bytes;
    const int g_begin = group * a.per_wg, g_end = min(g_begin + a.per_wg, a.Hkv);
    Chunk<T> in[2];
    auto fetch = [&](int g) __attribute__((always_inline)) {
        const uint8_t *row = src + (long)g * side.head * T::bytes;
        in[0] = load_chunk<T>(row, p.a);
        in[1] = load_chunk<T>(row, p.b);
    };
    fetch(g_begin);
    float w[16], c[8], s[8];
    const bool normed = a.weight != nullptr, turns = a.rot > 0;
    if constexpr (!VALUES) {
        weights_of<T>(a.weight, p, w);
        if (turns) turn_of<FP8, false>(a.inv_freq, p, (double)pos, c, s);
    }

    // the keys and head dims of values that this thread stores: TURNS times 16 bytes of each of DIMS head dims
    int k0[TURNS], dw[TURNS];                                // first key, word of a row in LDS
    bool stores[TURNS], all[TURNS], some[TURNS];
#pragma unroll
    for (int t = 0; t < TURNS; ++t) {
        const int job = tid + t * THREADS;
        k0[t] = job % (PAGE / KEYS) * KEYS;
        dw[t] = job / (PAGE / KEYS);
        stores[t] = job < JOBS;
        const long at0 = first + k0[t];
        all[t] = at0 >= start && at0 + KEYS <= start + rows;
        some[t] = at0 < start + rows && at0 + KEYS > start;
    }

    for (int g = g_begin, turn = 0; g < g_end; ++g, turn ^= 1) {
        const long at = (long)page * a.Hkv + g;              // page and head
        uint8_t *const store = static_cast<uint8_t *>(side.cache) + at * PAGE * D * EB;
        auto place = [&](int t, int q) __attribute__((always_inline)) { return reinterpret_cast<u32x4 *>(store + ((long)(dw[t] * DIMS + q) * PAGE + k0[t]) * EB); };
        u32x4 was[TURNS][DIMS];                              // vectors of which only some keys are written
#pragma unroll
        for (int t = 0; t < TURNS; ++t)
            if (VALUES && stores[t] && some[t] && !all[t]) {
#pragma unroll
                for (int q = 0; q < DIMS; ++q) was[t][q] = *place(t, q);
            }
        float old = 0.0f;
        if (FP8 && keeps) old = side.scale[at];
        float x[16];
        unpack(in[0], x);
        unpack(in[1], x + 8);
        fetch(min(g + 1, g_end - 1));
        if constexpr (!VALUES) {
            const float root = normed ? norm<D, FP8>(x, w, a.eps, true) : 1.0f;
            if (turns) {
                if (a.interleaved) rotate<kNeighbours>(x, c, s);
                else rotate<kHalves>(x, c, s);
            }
            if (normed) times<FP8>(x, root);
        }
        float by = 1.0f;                                     // kept codes: their old scale over the new one
        if constexpr (FP8) {
            float m = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) m = fmaxf(m, fabsf(x[i]));
            m = wave_largest(written ? m : 0.0f);
            if ((tid & 63) == 0) wave_max[turn * WAVES + (tid >> 6)] = m;
            __syncthreads();
#pragma unroll
            for (int k = 0; k < WAVES; ++k) m = fmaxf(m, wave_max[turn * WAVES + k]);
            float scale = scale_for(m);
            if (keeps) {
                scale = fmaxf(scale, old);
                by = old / scale;
            }
            if (tid == 0) side.scale[at] = scale;            // (the old one was read before the barrier)
            const Divide divide(scale);
            divide(x);
        }
        if constexpr (!VALUES) {
            uint8_t *const row = store + (long)slot * D * EB;
            if constexpr (FP8) {
                if (written) {
                    *reinterpret_cast<uint2 *>(row + p.a) = make_uint2(codes4(x[0], x[1], x[2], x[3]), codes4(x[4], x[5], x[6], x[7]));
                    *reinterpret_cast<uint2 *>(row + p.b) = make_uint2(codes4(x[8], x[9], x[10], x[11]), codes4(x[12], x[13], x[14], x[15]));
                }
                if (by != 1.0f) {
#pragma unroll
                    for (int k = 0; k < PAGE / ROWS; ++k) {
                        const int s1 = k * ROWS + tid / LANES;
                        const long at1 = first + s1;
                        if (at1 >= held || (at1 >= start && at1 < start + rows)) continue;
                        uint2 *const pa = reinterpret_cast<uint2 *>(store + (long)s1 * D + p.a), *const pb = reinterpret_cast<uint2 *>(store + (long)s1 * D + p.b);
                        const uint2 ca = *pa, cb = *pb;
                        *pa = make_uint2(regrown4(ca.x, by), regrown4(ca.y, by));
                        *pb = make_uint2(regrown4(cb.x, by), regrown4(cb.y, by));
                    }
                }
            } else if (written) {
                store_chunk<Bf16, false>(row, p.a, x);
                store_chunk<Bf16, false>(row, p.b, x + 8);
            }
        } else {
            // ---- values: rows into LDS, and out by words of the rows, four (bf16: two) head dims of one key
            unsigned *const at_a = turned + tid / LANES * PITCH + p.a * EB / 4, *const at_b = turned + tid / LANES * PITCH + p.b * EB / 4;
            if constexpr (FP8) {
#pragma unroll
                for (int i = 0; i < 4; ++i) (i < 2 ? at_a : at_b)[i % 2] = codes4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) (i < 4 ? at_a : at_b)[i % 4] = pack_bf16(x[2 * i], x[2 * i + 1]);
            }
            __syncthreads();
#pragma unroll
            for (int t = 0; t < TURNS; ++t) {
                if (!stores[t] || !(some[t] || by != 1.0f)) continue;
                const int from = k0[t] - (int)(base - first);            // row of the first key in LDS; (ROWS < PAGE) of keys that are not there, any row
                unsigned in_row[KEYS];
#pragma unroll
                for (int k = 0; k < KEYS; ++k) in_row[k] = turned[(ROWS == PAGE ? from + k : min(max(from + k, 0), ROWS - 1)) * PITCH + dw[t]];
                if (!some[t]) {
#pragma unroll
                    for (int q = 0; q < DIMS; ++q) was[t][q] = *place(t, q);
                }
#pragma unroll
                for (int q = 0; q < DIMS; ++q) {
                    u32x4 out;
#pragma unroll
                    for (int o = 0; o < 4; ++o) {
                        if constexpr (FP8) {
                            const unsigned lo = __builtin_amdgcn_perm(in_row[4 * o + 1], in_row[4 * o], 0x0c0c0000u | (unsigned)(q | (q + 4) << 8));
                            const unsigned hi = __builtin_amdgcn_perm(in_row[4 * o + 3], in_row[4 * o + 2], 0x0c0c0000u | (unsigned)(q | (q + 4) << 8));
                            out[o] = lo | hi << 16;
                        } else {
                            out[o] = __builtin_amdgcn_perm(in_row[2 * o + 1], in_row[2 * o], q ? 0x07060302u : 0x05040100u);
                        }
                    }
                    if (!all[t]) {                              // the other keys of the vector: kept codes in the new scale, the rest as it was
#pragma unroll
                        for (int o = 0; o < 4; ++o) {
                            unsigned grown = was[t][q][o], is_new = 0, is_kept = 0;
                            if constexpr (FP8) grown = by != 1.0f ? regrown4(was[t][q][o], by) : was[t][q][o];
#pragma unroll
                            for (int e = 0; e < KEYS / 4; ++e) {
                                const long at1 = first + k0[t] + o * (KEYS / 4) + e;
                                const unsigned field = (FP8 ? 0xffu : 0xffffu) << (e * 8 * EB);
                                if (at1 >= start && at1 < start + rows) is_new |= field;
                                else if (at1 < held) is_kept |= field;
                            }
                            out[o] = (out[o] & is_new) | (grown & is_kept) | (was[t][q][o] & ~(is_new | is_kept));
                        }
                    }
                    *place(t, q) = out;
                }
            }
            if (g + 1 < g_end) __syncthreads();
        }
    }
}

template <typename T, int D, int PAGE, int ROWS, bool FP8>
__global__ __launch_bounds__(ROWS *D / 16) void page_append_kernel(PageAppendArgs a)
{
    constexpr int EB = FP8 ? 1 : 2, WAVES = (ROWS * D / 16 + 63) / 64;
    __shared__ unsigned turned[ROWS * (D * EB / 4 + 1)];
    __shared__ float wave_max[2 * WAVES];
    if (blockIdx.x & 1) append_page<T, D, PAGE, ROWS, FP8, true>(a, blockIdx.x >> 1, turned, wave_max);
    else append_page<T, D, PAGE, ROWS, FP8, false>(a, blockIdx.x >> 1, turned, wave_max);
}

// Rows of a workgroup: as many as a sequence can have, of 16, 64 or all of the page: a workgroup of few waves starts and meets sooner.  us
// with this / with all: one token, 8 sequences, 32 heads, e4m3 pages of 128 6.8 / 9.7, ten 6.4 / 14.2, 16 rows of 11 sequences, 8 heads, pages of 64
// 5.2 / 5.9.
int rows_of(int n, int page) { return n <= 16 ? 16 : n <= 64 && page > 64 ? 64 : page; }
template <typename T, int D, int PAGE> hipError_t append_rows(const PageAppendArgs &a, bool fp8, unsigned wgs, hipStream_t stream)
{
    const int rows = rows_of(a.n, PAGE);
    auto run = [&](auto kernel) { return launch(kernel, dim3(wgs), dim3(rows * D / 16), stream, a); };
    if constexpr (PAGE > 16)
        if (rows == 16) return fp8 ? run(page_append_kernel<T, D, PAGE, 16, true>) : run(page_append_kernel<T, D, PAGE, 16, false>);
    if constexpr (PAGE > 64)
        if (rows == 64) return fp8 ? run(page_append_kernel<T, D, PAGE, 64, true>) : run(page_append_kernel<T, D, PAGE, 64, false>);
    return fp8 ? run(page_append_kernel<T, D, PAGE, PAGE, true>) : run(page_append_kernel<T, D, PAGE, PAGE, false>);
}
template <typename T, int D> hipError_t append_rows(const PageAppendArgs &a, bool fp8, unsigned wgs, hipStream_t stream)
{
    switch (a.page_log2) {
    case 4: return append_rows<T, D, 16>(a, fp8, wgs, stream);
    case 5: return append_rows<T, D, 32>(a, fp8, wgs, stream);
    case 6: return append_rows<T, D, 64>(a, fp8, wgs, stream);
    default: return append_rows<T, D, 128>(a, fp8, wgs, stream);
    }
}

template <typename T, int D> hipError_t norm_rotate(const NormRotateArgs &a, dim3 grid, hipStream_t stream)
{
    const int pair = a.rot == 0 ? kNoTurn : a.interleaved ? kNeighbours : kHalves;
    if (a.q.weight != nullptr || a.k.weight != nullptr)
        return pair == kNoTurn ? launch(norm_rotate_kernel<T, D, true, kNoTurn>, grid, dim3(256), stream, a)
             : pair == kHalves ? launch(norm_rotate_kernel<T, D, true, kHalves>, grid, dim3(256), stream, a)
                               : launch(norm_rotate_kernel<T, D, true, kNeighbours>, grid, dim3(256), stream, a);
    return pair == kNoTurn ? launch(norm_rotate_kernel<T, D, false, kNoTurn>, grid, dim3(256), stream, a)
         : pair == kHalves ? launch(norm_rotate_kernel<T, D, false, kHalves>, grid, dim3(256), stream, a)
                           : launch(norm_rotate_kernel<T, D, false, kNeighbours>, grid, dim3(256), stream, a);
}

}  // namespace

hipError_t launch_norm_rotate(NormRotateArgs a, int d, bool bf16, hipStream_t stream)
{
    const int per_wg_tokens = 256 / (d / 16);
    const long tiles = ((long)a.tokens + per_wg_tokens - 1) / per_wg_tokens;
    const int heads = a.q.heads + a.k.heads;
    // Heads per workgroup: as many as leave two workgroups per compute unit, as each makes the angles of its tokens once.  us at 512 / 2048
    // workgroups: 16 x 64 rows of 40 heads 6.0 / 7.2, 3 x 700 rows of 32 heads in fp32 14.7 / 17.3, 16 x 2048 rows of 40 heads the same.
    long groups = (512 + tiles - 1) / tiles;
    if (groups > heads) groups = heads;
    a.per_wg = (int)((heads + groups - 1) / groups);
    a.q_groups = (a.q.heads + a.per_wg - 1) / a.per_wg;
    const int k_groups = (a.k.heads + a.per_wg - 1) / a.per_wg;
    const dim3 grid((unsigned)tiles, (unsigned)(a.q_groups + k_groups));
    if (bf16) return d == 128 ? norm_rotate<Bf16, 128>(a, grid, stream) : norm_rotate<Bf16, 64>(a, grid, stream);
    return d == 128 ? norm_rotate<F32, 128>(a, grid, stream) : norm_rotate<F32, 64>(a, grid, stream);
}

hipError_t launch_page_append(PageAppendArgs a, int d, bool rows_bf16, bool fp8, hipStream_t stream)
{
    const long page = 1L << a.page_log2;
    a.pages_per_seq = (int)((a.n + page - 2) / page + 1);    // that n rows can touch, wherever they begin
    // Heads per workgroup: as many as leave two thousand threads per compute unit, what fits there; more workgroups make the angles and
    // look up the page once more each.  us at one head / all heads / this: 16 x 2048 rows, 8 heads, e4m3 67 / 42 / 42, 4096 rows, 32 heads,
    // bf16 pages of 16 32 / 33 / 31 (with the hardware's sine); short calls have one head each.
    const long threads = 2L * a.B * a.pages_per_seq * a.Hkv * (rows_of(a.n, (int)page) * d / 16), per = threads / (256 * 2048);
    a.per_wg = per < 1 ? 1 : per > a.Hkv ? a.Hkv : (int)per;
    a.head_groups = (a.Hkv + a.per_wg - 1) / a.per_wg;
    const unsigned wgs = (unsigned)(2L * a.B * a.pages_per_seq * a.head_groups);
    if (rows_bf16) return d == 128 ? append_rows<Bf16, 128>(a, fp8, wgs, stream) : append_rows<Bf16, 64>(a, fp8, wgs, stream);
    return d == 128 ? append_rows<F32, 128>(a, fp8, wgs, stream) : append_rows<F32, 64>(a, fp8, wgs, stream);
}

}  // namespace dd
