// Verification of drafted tokens with given random numbers.  For sequence b with drafts x_0 .. x_{n-1}, the verifier's probabilities
// p_i = softmax(l_V,i / T) and the drafter's q_i = softmax(l_D,i / T):
//     draft i stands iff  u_i q_i(x_i) < p_i(x_i);   a = drafts that stand before the first that does not
//     the token behind them is the lowest x with  sum_{y <= x} w(y) > u_n sum_y w(y),   w = max(p_a - q_a, 0) where a draft was turned
//     down, p_a where none was
// so that every token is distributed as the verifier's.  A decision is a comparison with a border that is one of V, some 10^-5 apart and
// closer: exponentials and sums are held in 64 bits, and no order of addition or rounding of an exponential decides (fp32 sums would
// move a border by 10^-3 of a token's width and more).  An fp64 instruction takes a wave as long here as an fp32 one.
// Three launches, as every step needs all of the one before:
//   draft_sums_kernel   every logit once: reference and sum of 2^((l - ref) c), c = log2(e) / T, of every part of a row
//   draft_decide_kernel the drafts' fate, and the weights' sums over the parts of the row that a token is drawn from
//   draft_pick_kernel   the part in which the sum passes its mark, and there the token
#include "dd_internal.h"

#include <type_traits>

namespace dd {
namespace {

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kLoads = 4;                    // vectors of 16 bytes of a lane on their way
constexpr int kMostSplits = 64;              // of a row: a lane of a wave for each
constexpr int kMostParts = kThreads;         // of the row that is drawn from: a thread of a workgroup for each
[[maybe_unused]] constexpr float kCold = 1.0e-6f;             // temperatures up to here: all of the probability on the largest logit
[[maybe_unused]] constexpr double kLog2e = 1.4426950408889634;
[[maybe_unused]] constexpr float kRaise = 500.0f;             // log2 units: a reference may be exceeded by as much, 2^kRaise sums fit fp64
[[maybe_unused]] constexpr double kFloor = -1020.0;           // below that a power of two is none

struct State { float ref; int first; double sum; };      // reference, its first index (temperature 0), sum
struct Sums { double w, p; };                            // of a part of the row that is drawn from: of the weights, and of p alone
enum { kDone = 0, kDraw = 1, kDrawP = 2 };
struct Verdict { int kind, at; float ref_p, ref_q; double inv_p, inv_q, c; };      // how the token at `at` is drawn

struct DraftKernelArgs {
    const uint8_t *lv, *ld;
    const int32_t *tokens, *n_draft;
    const float *uniforms, *temperature;
    int32_t *out_tokens, *out_accepted;
    float *out_chances;
    State *states;                           // [B nv + B n][splits]
    Sums *sums;                              // [B][parts]
    Verdict *verdicts;                       // [B]
    int B, n, nv, bonus, vecs;               // nv: verifier rows of a sequence; vecs: 16-byte vectors of a row
    int splits, per_split, parts, per_part;  // vectors per split and part
};

// 2^t for t <= 1000, 0 below -1020: the nearest integer by a number so large that fractions fall off, the rest on [-1/2, 1/2] by a
// polynomial through 2^f at the Chebyshev nodes (error 1.1e-12 at most).
__device__ __forceinline__ double power(double t)
{
    constexpr double kWhole = 6755399441055744.0;            // 1.5 2^52
    t = __builtin_fmax(t, kFloor);
    const double w = t + kWhole, f = t - (w - kWhole);
    double p = 0x1.63d136366db24p-20;
    p = __builtin_fma(p, f, 0x1.00dc4a532fb8ep-16);
    p = __builtin_fma(p, f, 0x1.4308ac85aa947p-13);
    p = __builtin_fma(p, f, 0x1.5d8745a728441p-10);
    p = __builtin_fma(p, f, 0x1.3b2ab7181b755p-7);
    p = __builtin_fma(p, f, 0x1.c6b08dd6fd234p-5);
    p = __builtin_fma(p, f, 0x1.ebfbdff823cedp-3);
    p = __builtin_fma(p, f, 0x1.62e42fef84cf0p-1);
    p = __builtin_fma(p, f, 1.0);
    u32x2 r = __builtin_bit_cast(u32x2, p);
    r.y += __builtin_bit_cast(u32x2, w).x << 20;
    return __builtin_bit_cast(double, r);
}
// the same, exactly 0 where it is nothing next to 1: what is impossible has no weight at all
__device__ __forceinline__ double weight_of(float l, double c, double at) { return power(__builtin_fma((double)l, c, at)) - 0x1p-1020; }

template <bool BF16> __device__ __forceinline__ void unpack(const u32x4 &v, float *x)
{
    if constexpr (BF16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __builtin_bit_cast(float, (unsigned)v[i] << 16);
            x[2 * i + 1] = __builtin_bit_cast(float, (unsigned)v[i] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __builtin_bit_cast(float, (unsigned)v[i]);
    }
}
template <bool BF16> __device__ __forceinline__ float logit(const uint8_t *row, int x)
{
    if constexpr (BF16) return __builtin_bit_cast(float, (unsigned)reinterpret_cast<const uint16_t *>(row)[x] << 16);
    else return reinterpret_cast<const float *>(row)[x];
}

// ---- across a wave and a workgroup, every lane with the result, always in the same order
__device__ __forceinline__ double other(double v, int mask)
{
    u32x2 r = __builtin_bit_cast(u32x2, v);
    r.x = __shfl_xor((int)r.x, mask);
    r.y = __shfl_xor((int)r.y, mask);
    return __builtin_bit_cast(double, r);
}
__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) v += other(v, m);
    return v;
}
__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) v = fmaxf(v, __shfl_xor(v, m));
    return v;
}
__device__ __forceinline__ int wave_min(int v)
{
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) v = min(v, __shfl_xor(v, m));
    return v;
}
__device__ __forceinline__ void merge_first(float &ref, int &first, float r, int f)
{
    if (r > ref || (r == ref && f < first)) { ref = r; first = f; }
}

__device__ __forceinline__ int drafts_of(const DraftKernelArgs &a, int b) { return a.n_draft ? min(max(a.n_draft[b], 0), a.n) : a.n; }
// log2(e) / T; 0 for a temperature that takes the largest logit
__device__ __forceinline__ double factor_of(const DraftKernelArgs &a, int b)
{
    const float t = a.temperature ? a.temperature[b] : 1.0f;
    return t > kCold ? kLog2e / (double)fminf(t, 3.0e38f) : 0.0;
}

// One part of one row.  A lane's reference is set by its first vectors and raised only where one passes it by 2^kRaise.
template <bool BF16> __global__ __launch_bounds__(kThreads) void draft_sums_kernel(DraftKernelArgs a)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int E = BF16 ? 8 : 4;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const unsigned row = blockIdx.x / (unsigned)a.splits, sp = blockIdx.x - row * (unsigned)a.splits;
    const bool verifier = row < (unsigned)a.B * (unsigned)a.nv;
    const unsigned in = verifier ? row : row - (unsigned)a.B * (unsigned)a.nv;
    const int b = (int)(in / (unsigned)(verifier ? a.nv : a.n)), i = (int)(in - (unsigned)b * (unsigned)(verifier ? a.nv : a.n));
    const int drafts = drafts_of(a, b);
    if (i > drafts || (i == drafts && !(verifier && a.bonus))) return;       // no draft, and not the row behind the last one
    const int begin = (int)sp * a.per_split, count = min(a.per_split, a.vecs - begin);
    const u32x4 *const p = reinterpret_cast<const u32x4 *>((verifier ? a.lv : a.ld) + (size_t)in * a.vecs * 16) + begin;
    const double c = factor_of(a, b);
    float ref = -3.0e38f;
    int first = 0x7fffffff;
    double sum = 0;
    if (c == 0) {
        ref = -__builtin_inff();
        for (int v = tid; v < count; v += kThreads) {
            float x[E];
            unpack<BF16>(p[v], x);
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (x[e] > ref || first == 0x7fffffff) { ref = x[e]; first = (begin + v) * E + e; }
        }
    } else {
        const float margin = (float)(kRaise / c);
        double at = -(double)ref * c, s[2] = {0, 0};
        for (int v = tid; v < count; v += kThreads * kLoads) {
            u32x4 w[kLoads];
#pragma unroll
            for (int u = 0; u < kLoads; ++u) {
                const int j = v + u * kThreads;
                w[u] = p[min(j, count - 1)];
            }
#pragma unroll
            for (int u = 0; u < kLoads; ++u) {
                if (v + u * kThreads >= count) break;
                float x[E], top;
                unpack<BF16>(w[u], x);
                top = x[0];
#pragma unroll
                for (int e = 1; e < E; ++e) top = fmaxf(top, x[e]);
                if (top - ref > margin) {                    // (the first vectors too)
                    const double by = power(((double)ref - (double)top) * c);
                    s[0] *= by;
                    s[1] *= by;
                    ref = top;
                    at = -(double)ref * c;
                }
#pragma unroll
                for (int e = 0; e < E; ++e) s[e & 1] += power(__builtin_fma((double)x[e], c, at));
            }
        }
        sum = s[0] + s[1];
    }
    __shared__ State of_wave[kThreads / 64];
    if (c == 0) {
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) merge_first(ref, first, __shfl_xor(ref, m), __shfl_xor(first, m));
    } else {
        const float top = wave_max(ref);
        sum = wave_sum(sum * power(((double)ref - (double)top) * c));
        ref = top;
    }
    if (lane == 0) of_wave[wave] = State{ref, first, sum};
    __syncthreads();
    if (tid == 0) {
        State r = of_wave[0];
        for (int w = 1; w < kThreads / 64; ++w) {
            const State o = of_wave[w];
            if (c == 0) merge_first(r.ref, r.first, o.ref, o.first);
            else {
                const float top = fmaxf(r.ref, o.ref);
                r.sum = r.sum * power(((double)r.ref - (double)top) * c) + o.sum * power(((double)o.ref - (double)top) * c);
                r.ref = top;
            }
        }
        a.states[(size_t)row * a.splits + sp] = r;
    }
#endif
}

// A row's state, merged by a wave.
__device__ __forceinline__ State row_state(const DraftKernelArgs &a, size_t row, double c)
{
    const int lane = threadIdx.x & 63;
    State r{-__builtin_inff(), 0x7fffffff, 0};
    if (lane < a.splits) r = a.states[row * a.splits + lane];
    if (c == 0) {
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) merge_first(r.ref, r.first, __shfl_xor(r.ref, m), __shfl_xor(r.first, m));
    } else {
        const float top = wave_max(r.ref);
        r.sum = wave_sum(lane < a.splits ? r.sum * power(((double)r.ref - (double)top) * c) : 0.0);
        r.ref = top;
    }
    return r;
}

// The drafts' fate, by every workgroup of a sequence for itself; the first one of them writes it.
template <bool BF16> __global__ __launch_bounds__(kThreads) void draft_decide_kernel(DraftKernelArgs a)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int E = BF16 ? 8 : 4;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int b = (int)(blockIdx.x / (unsigned)a.parts), part = (int)(blockIdx.x - (unsigned)b * (unsigned)a.parts);
    const int drafts = drafts_of(a, b), V = a.vecs * E;
    const double c = factor_of(a, b);
    const size_t v_row = (size_t)b * a.nv, d_row = (size_t)a.B * a.nv + (size_t)b * a.n;
    const size_t row_bytes = (size_t)a.vecs * 16;
    __shared__ int turned;
    if (tid == 0) turned = drafts;
    __syncthreads();
    for (int i = wave; i < a.n; i += kThreads / 64) {
        float chance = 0;
        if (i < drafts) {
            const int x = a.tokens[(size_t)b * a.n + i];
            const bool known = x >= 0 && x < V;
            const State sp = row_state(a, v_row + i, c);
            double px, qx = 1;
            if (c == 0) px = sp.first == x ? 1 : 0;
            else px = known && sp.sum > 0 ? weight_of(logit<BF16>(a.lv + (v_row + i) * row_bytes, x), c, -(double)sp.ref * c) / sp.sum : 0;
            if (a.ld) {
                const State sq = row_state(a, d_row + i, c);
                if (c == 0) qx = sq.first == x ? 1 : 0;
                else qx = known && sq.sum > 0 ? weight_of(logit<BF16>(a.ld + ((size_t)b * a.n + i) * row_bytes, x), c, -(double)sq.ref * c) / sq.sum : 0;
            }
            const double u = a.uniforms[(size_t)b * (a.n + 1) + i];
            if (lane == 0 && !(u * qx < px)) atomicMin(&turned, i);
            chance = qx > px ? (float)(px / qx) : px > 0 ? 1.0f : 0.0f;
        }
        if (part == 0 && lane == 0) a.out_chances[(size_t)b * a.n + i] = chance;
    }
    __syncthreads();
    const int at = turned;
    const bool down = at < drafts, draws = down || a.bonus;
    if (part == 0) {
        for (int j = tid; j <= a.n; j += kThreads)
            if (j != at || !draws) a.out_tokens[(size_t)b * (a.n + 1) + j] = j < at ? a.tokens[(size_t)b * a.n + j] : -1;
        if (tid == 0) a.out_accepted[b] = at;
    }
    Verdict verdict{kDone, at, 0, 0, 0, 0, c};
    State p{}, q{};
    const bool minus = down && a.ld != nullptr;
    const int without = down && a.ld == nullptr ? a.tokens[(size_t)b * a.n + at] : -1;       // a drafter without probabilities was sure of this one
    if (draws) {
        p = row_state(a, v_row + at, c);
        if (c == 0) {
            // one token has all of the probability, and what the drafter has there does not matter: if it has all of it too, nothing is
            // left, and the draw is p's
            if (part == 0 && tid == 0) a.out_tokens[(size_t)b * (a.n + 1) + at] = p.first < V ? p.first : -1;
        } else {
            if (minus) q = row_state(a, d_row + at, c);
            verdict = Verdict{kDraw, at, p.ref, q.ref, p.sum > 0 ? 1.0 / p.sum : 0.0, q.sum > 0 ? 1.0 / q.sum : 0.0, c};
        }
    }
    if (part == 0 && tid == 0) a.verdicts[b] = verdict;
    if (verdict.kind == kDone) return;
    // ---- this part of the row that the token is drawn from
    const int begin = part * a.per_part, count = min(a.per_part, a.vecs - begin);
    const u32x4 *const pv = reinterpret_cast<const u32x4 *>(a.lv + (v_row + at) * row_bytes) + begin;
    const u32x4 *const pd = minus ? reinterpret_cast<const u32x4 *>(a.ld + ((size_t)b * a.n + at) * row_bytes) + begin : pv;
    const double at_p = -(double)p.ref * c, at_q = -(double)q.ref * c;
    double sw = 0, sp = 0;
    for (int v = tid; v < count; v += kThreads) {
        float x[E], y[E];
        unpack<BF16>(pv[v], x);
        unpack<BF16>(pd[v], y);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const double px = weight_of(x[e], c, at_p) * verdict.inv_p;
            double w = px;
            if (minus) w = __builtin_fmax(px - weight_of(y[e], c, at_q) * verdict.inv_q, 0.0);
            if ((begin + v) * E + e == without) w = 0;
            sw += w;
            sp += px;
        }
    }
    sw = wave_sum(sw);
    sp = wave_sum(sp);
    __shared__ Sums of_wave[kThreads / 64];
    if (lane == 0) of_wave[wave] = Sums{sw, sp};
    __syncthreads();
    if (tid == 0) {
        Sums s = of_wave[0];
        for (int w = 1; w < kThreads / 64; ++w) { s.w += of_wave[w].w; s.p += of_wave[w].p; }
        a.sums[(size_t)b * a.parts + part] = s;
    }
#endif
}

// Sums of the threads before, in the threads' order, and the sum of all.
__device__ __forceinline__ double before(double v, double *of_wave, double &all)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    double s = v;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        u32x2 r = __builtin_bit_cast(u32x2, s);
        r.x = __shfl_up((int)r.x, m);
        r.y = __shfl_up((int)r.y, m);
        if (lane >= m) s += __builtin_bit_cast(double, r);
    }
    u32x2 r = __builtin_bit_cast(u32x2, s);
    r.x = __shfl_up((int)r.x, 1);
    r.y = __shfl_up((int)r.y, 1);
    __syncthreads();
    if (lane == 63) of_wave[wave] = s;
    __syncthreads();
    double pre = 0;
    all = 0;
    for (int w = 0; w < kThreads / 64; ++w) {
        if (w == wave) pre = all;
        all += of_wave[w];
    }
    return pre + (lane == 0 ? 0.0 : __builtin_bit_cast(double, r));
}

template <bool BF16> __global__ __launch_bounds__(kThreads) void draft_pick_kernel(DraftKernelArgs a)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int E = BF16 ? 8 : 4;
    const int tid = threadIdx.x, b = blockIdx.x;
    const Verdict verdict = a.verdicts[b];
    if (verdict.kind == kDone) return;
    const int at = verdict.at;
    __shared__ double of_wave[kThreads / 64];
    __shared__ int found, last;
    __shared__ double start;
    const Sums s = tid < a.parts ? a.sums[(size_t)b * a.parts + tid] : Sums{0, 0};
    // what is left of p without q; where p is nowhere above q, p itself
    double all_w, all_p;
    const double pre_w = before(s.w, of_wave, all_w), pre_p = before(s.p, of_wave, all_p);
    const bool left = all_w > 0;
    const double mine = left ? s.w : s.p, pre = left ? pre_w : pre_p;
    const double mark = __builtin_fmax((double)a.uniforms[(size_t)b * (a.n + 1) + a.n], 0.0) * (left ? all_w : all_p);
    if (tid == 0) { found = a.parts; last = -1; }
    __syncthreads();
    if (tid < a.parts && mine > 0) {
        if (pre + mine > mark) atomicMin(&found, tid);
        atomicMax(&last, tid);
    }
    __syncthreads();
    const int part = found < a.parts ? found : last;
    if (part < 0) {                                          // no probability anywhere
        if (tid == 0) a.out_tokens[(size_t)b * (a.n + 1) + at] = -1;
        return;
    }
    if (tid == part) start = pre;
    __syncthreads();
    if (tid == 0) { found = 0x7fffffff; last = -1; }
    // ---- within the part, neighbouring vectors per thread
    const int drafts = drafts_of(a, b);
    const bool down = at < drafts, minus = left && down && a.ld != nullptr;
    const int without = left && down && a.ld == nullptr ? a.tokens[(size_t)b * a.n + at] : -1;
    const size_t row_bytes = (size_t)a.vecs * 16;
    const int begin = part * a.per_part, count = min(a.per_part, a.vecs - begin), each = (count + kThreads - 1) / kThreads;
    const u32x4 *const pv = reinterpret_cast<const u32x4 *>(a.lv + ((size_t)b * a.nv + at) * row_bytes) + begin;
    const u32x4 *const pd = minus ? reinterpret_cast<const u32x4 *>(a.ld + ((size_t)b * a.n + at) * row_bytes) + begin : pv;
    const double c = verdict.c, at_p = -(double)verdict.ref_p * c, at_q = -(double)verdict.ref_q * c;
    auto weights = [&](int v, double *w) __attribute__((always_inline)) {
        float x[E], y[E];
        unpack<BF16>(pv[v], x);
        unpack<BF16>(pd[v], y);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            w[e] = weight_of(x[e], c, at_p) * verdict.inv_p;
            if (minus) w[e] = __builtin_fmax(w[e] - weight_of(y[e], c, at_q) * verdict.inv_q, 0.0);
            if ((begin + v) * E + e == without) w[e] = 0;
        }
    };
    double sum = 0;
    for (int v = tid * each; v < min((tid + 1) * each, count); ++v) {
        double w[E];
        weights(v, w);
#pragma unroll
        for (int e = 0; e < E; ++e) sum += w[e];
    }
    double all;
    double so_far = start + before(sum, of_wave, all);
    // (threads that begin behind the mark have nothing to look for, but that rounding may have taken the mark past the part's end)
    for (int v = tid * each; v < min((tid + 1) * each, count); ++v) {
        double w[E];
        weights(v, w);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            so_far += w[e];
            if (w[e] > 0) {
                if (so_far > mark) atomicMin(&found, (begin + v) * E + e);
                atomicMax(&last, (begin + v) * E + e);
            }
        }
    }
    __syncthreads();
    if (tid == 0) a.out_tokens[(size_t)b * (a.n + 1) + at] = found != 0x7fffffff ? found : last;
#endif
}

struct Plan { int vecs, splits, per_split, parts, per_part; size_t states, sums, bytes; };
Plan plan_of(int B, int n, int nv, int V, bool bf16, bool drafter)
{
    Plan p;
    p.vecs = (int)((long)V * (bf16 ? 2 : 4) / 16);
    const long rows = (long)B * nv + (drafter ? (long)B * n : 0);
    auto divide = [&](long rows, long want, int most, int &per, int &count) {
        long v = (long)p.vecs * rows / want;                 // vectors per workgroup
        const long least = ((long)p.vecs + most - 1) / most;
        v = v > least ? v : least;
        v = (v + kThreads - 1) / kThreads * kThreads;
        per = (int)(v < 0x7fffff00 ? v : 0x7fffff00);
        count = (int)(((long)p.vecs + per - 1) / per);
    };
    divide(rows, 8192, kMostSplits, p.per_split, p.splits);
    divide(B, 1024, kMostParts, p.per_part, p.parts);
    p.states = ((size_t)rows * p.splits * sizeof(State) + 255) / 256 * 256;
    p.sums = ((size_t)B * p.parts * sizeof(Sums) + 255) / 256 * 256;
    p.bytes = p.states + p.sums + (size_t)B * sizeof(Verdict);
    return p;
}

}  // namespace

size_t verify_draft_workspace_bytes(int B, int n, int nv, int V, bool bf16, bool drafter) { return plan_of(B, n, nv, V, bf16, drafter).bytes; }
// workgroups of the largest launch
double verify_draft_workgroups(int B, int n, int nv, int V, bool bf16, bool drafter)
{
    const Plan p = plan_of(B, n, nv, V, bf16, drafter);
    const double rows = (double)B * nv + (drafter ? (double)B * n : 0), first = rows * p.splits, second = (double)B * p.parts;
    return first > second ? first : second;
}

hipError_t launch_verify_draft(const DraftArgs &d, hipStream_t stream)
{
    const Plan p = plan_of(d.B, d.n, d.nv, d.V, d.bf16, d.logits_d != nullptr);
    uint8_t *const ws = static_cast<uint8_t *>(d.workspace);
    const DraftKernelArgs a{static_cast<const uint8_t *>(d.logits_v), static_cast<const uint8_t *>(d.logits_d), d.tokens, d.n_draft, d.uniforms, d.temperature,
                            d.out_tokens, d.out_accepted, d.out_chances, reinterpret_cast<State *>(ws), reinterpret_cast<Sums *>(ws + p.states),
                            reinterpret_cast<Verdict *>(ws + p.states + p.sums), d.B, d.n, d.nv, d.bonus ? 1 : 0, p.vecs, p.splits, p.per_split, p.parts, p.per_part};
    const unsigned rows = (unsigned)d.B * (unsigned)d.nv + (d.logits_d ? (unsigned)d.B * (unsigned)d.n : 0u);
    auto all = [&](auto sums, auto decide, auto pick) {
        hipError_t e = launch(sums, dim3(rows * (unsigned)p.splits), dim3(kThreads), stream, a);
        if (e == hipSuccess) e = launch(decide, dim3((unsigned)d.B * (unsigned)p.parts), dim3(kThreads), stream, a);
        return e == hipSuccess ? launch(pick, dim3((unsigned)d.B), dim3(kThreads), stream, a) : e;
    };
    return d.bf16 ? all(draft_sums_kernel<true>, draft_decide_kernel<true>, draft_pick_kernel<true>)
                  : all(draft_sums_kernel<false>, draft_decide_kernel<false>, draft_pick_kernel<false>);
}

}  // namespace dd
