// Verification of drafted tokens with given random numbers.  For sequence b with drafts x_0 .. x_{n-1}, the verifier's probabilities
// p_i = softmax(l_V,i / T) and the drafter's q_i = softmax(l_D,i / T):
//     draft i stands iff  u_i q_i(x_i) < p_i(x_i);   a = drafts that stand before the first that does not
//     the token behind them is the lowest x with  sum_{y <= x} w(y) > u_n sum_y w(y),   w = max(p_a - q_a, 0) where a draft was turned
//     down, p_a where none was
// so that every token is distributed as the verifier's.  A decision is a comparison with a border, and a draw one with borders that are
// V, some 10^-5 apart and closer: no rounding may decide them (fp32 sums would move a border by 10^-3 of a token's width and more).
// Three launches, as every step needs all of the one before:
//   draft_sums_kernel   every logit once: reference and sum of 2^((l - ref) c), c = log2(e) / T, of every part of a row; fp32
//                       exponentials, whose sums are good to kNear: memory bounds it
//   draft_decide_kernel the drafts' fate; a draft nearer to its border than kNear is decided again on fp64 sums of its rows (one in some
//                       ten thousand).  Then, of the one row that a token is drawn from, in fp64 by parts: sums of p's and q's
//                       exponentials, all and where p is the larger.  Which of the two is the larger goes by the fp32 sums, and may be
//                       wrong for tokens where they agree to kNear: of those there is a sum too
//   draft_pick_kernel   the part in which the running sum passes its mark, and there the token.  Now S_p and S_q are known in fp64, and with
//                       them by how much the quotient that decided was off, e: no border is off by more than e times the probability of
//                       the tokens that were near.  A mark closer than that to its token's borders is taken again, with the parts that
//                       have such tokens summed by the true quotient: fewer than one row in ten thousand where drafter and
//                       verifier differ; every row where they agree to 10^-5, or on a token that outweighs all others.  (One
//                       sequence, 126464 fp32 logits: 14.5 us, 22 with such a token, 88 where all tokens are near; 64 of them 36, 51, 105.)
// An fp64 instruction takes a wave as long here as an fp32 one (2.2 and 1.9 ns), a power of two 18 of them; with fp64 sums in the
// first kernel too, that one took 100 us for 64 sequences of 8 drafts, 126464 bf16 logits.  As it is the three take 47.5 (5.8 TB/s), 24.4 and 5.6:
// the second's workgroups are 7 us at the decisions, which are chains of loads just behind 275 MB of others, and 5 to 8 at their part of the
// row.  (The drafts' fate by a launch of its own: 7.5 + 17 for the 24.  All of a row's loads before its arithmetic, and logits picked up
// by the first kernel: no difference.  Exponentials of 15 instructions for 18: 24.6.  The last of a sequence's workgroups as the third launch: 194
// for 24 and 5, as every workgroup's fence writes its cache back.)
#include "dd_internal.h"

#include <type_traits>

namespace dd {
namespace {

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kLoads = 4;                    // vectors of 16 bytes of a lane on their way
constexpr int kMostSplits = 64;              // of a row: a lane of a wave for each
constexpr int kMostParts = 64;               // workgroups of the row that is drawn from: a thread of a workgroup for each of their waves
[[maybe_unused]] constexpr float kCold = 1.0e-6f;             // temperatures up to here: all of the probability on the largest logit
[[maybe_unused]] constexpr double kLog2e = 1.4426950408889634;
[[maybe_unused]] constexpr float kRaise = 16.0f;              // log2 units by which logits may exceed a reference
[[maybe_unused]] constexpr double kFloor = -1020.0;           // below that a power of two is none
// What a quotient of two of the first kernel's sums and of two probabilities may be off by: per exponential the roundings of l - ref and
// of its product with c, as rounded, 2^-24 each of an exponent of 40 and less (what is below adds nothing), ln 2 of that, its own
// of 2^-23, and three additions: 5.5e-6 per sum.
[[maybe_unused]] constexpr double kNear = 2.0e-5;

struct State { float ref; int first; double sum; };      // reference, its first index (temperature 0), sum
struct Sums { double p, q, above_p, above_q, near_p; };  // of exponentials, of a part of the row that is drawn from: all, where p > q, of vectors where that is open
enum { kDone = 0, kDraw = 1 };
struct Verdict { int kind, at, minus, without; float ref_p, ref_q; double c, even; };        // how the token at `at` is drawn; S_p / S_q of the fp32 sums

struct DraftKernelArgs {
    const uint8_t *lv, *ld;
    const int32_t *tokens, *n_draft;
    const float *uniforms, *temperature;
    int32_t *out_tokens, *out_accepted;
    float *out_chances;
    State *states;                           // [B nv + B n][splits]
    Sums *sums;                              // [B][parts][kWaves]
    Verdict *verdicts;                       // [B]
    int B, n, nv, bonus, vecs;               // nv: verifier rows of a sequence; vecs: 16-byte vectors of a row
    int splits, per_split, parts, per_part;  // vectors per split and part (of a part, a quarter per wave)
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

// ---- across a wave, every lane with the result (the same bits: the two that meet are added in either order): neighbours, pairs of two,
// halves of eight and of sixteen lanes, then the halves of 32 and of 64
template <int STEP> __device__ __forceinline__ u32x2 meet(unsigned v)
{
    if constexpr (STEP < 4) {
        constexpr int CTRL = STEP == 0 ? 0xB1 : STEP == 1 ? 0x4E : STEP == 2 ? 0x141 : 0x140;
        return u32x2{v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true)};
    } else if constexpr (STEP == 4) {
        return __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(v, v, false, false));
    } else {
        return __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(v, v, false, false));
    }
}
template <int STEP = 0> __device__ __forceinline__ double wave_sum(double v)
{
    const u32x2 r = __builtin_bit_cast(u32x2, v), lo = meet<STEP>(r.x), hi = meet<STEP>(r.y);
    v = __builtin_bit_cast(double, u32x2{lo.x, hi.x}) + __builtin_bit_cast(double, u32x2{lo.y, hi.y});
    if constexpr (STEP < 5) return wave_sum<STEP + 1>(v);
    else return v;
}
template <int STEP = 0> __device__ __forceinline__ float wave_max(float v)
{
    const u32x2 r = meet<STEP>(__builtin_bit_cast(unsigned, v));
    v = fmaxf(__builtin_bit_cast(float, (unsigned)r.x), __builtin_bit_cast(float, (unsigned)r.y));
    if constexpr (STEP < 5) return wave_max<STEP + 1>(v);
    else return v;
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

// One part of one row.  A lane's reference is set by its first vectors and raised only where one passes it by kRaise.
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
        const float by = (float)c, margin = (float)(kRaise / c);
        for (int v = tid; v < count; v += kThreads * kLoads) {
            u32x4 w[kLoads];
#pragma unroll
            for (int u = 0; u < kLoads; ++u) w[u] = __builtin_nontemporal_load(p + min(v + u * kThreads, count - 1));
#pragma unroll
            for (int u = 0; u < kLoads; ++u) {
                float x[E], top;
                unpack<BF16>(w[u], x);
                top = x[0];
#pragma unroll
                for (int e = 1; e < E; ++e) top = fmaxf(top, x[e]);
                if (top - ref > margin) {                    // (the first vectors too)
                    sum *= power(((double)ref - (double)top) * c);
                    ref = top;
                }
                float s[E];
#pragma unroll
                for (int e = 0; e < E; ++e) s[e] = __builtin_amdgcn_exp2f((x[e] - ref) * by);
#pragma unroll
                for (int k = 1; k < E; k *= 2)
#pragma unroll
                    for (int e = 0; e + k < E; e += 2 * k) s[e] += s[e + k];
                sum += v + u * kThreads < count ? (double)s[0] : 0.0;
            }
        }
    }
    __shared__ State of_wave[kWaves];
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
        for (int w = 1; w < kWaves; ++w) {
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

// The sum of a whole row's exponentials in fp64, by a workgroup.
template <bool BF16> __device__ double exact_sum(const uint8_t *row, int vecs, double c, float ref)
{
    constexpr int E = BF16 ? 8 : 4;
    const u32x4 *const p = reinterpret_cast<const u32x4 *>(row);
    const double at = -(double)ref * c;
    double s = 0;
    for (int v = threadIdx.x; v < vecs; v += kThreads) {
        float x[E];
        unpack<BF16>(p[v], x);
#pragma unroll
        for (int e = 0; e < E; ++e) s += weight_of(x[e], c, at);
    }
    s = wave_sum(s);
    __shared__ double of_wave[kWaves];
    __syncthreads();
    if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x >> 6] = s;
    __syncthreads();
    s = of_wave[0];
    for (int w = 1; w < kWaves; ++w) s += of_wave[w];
    return s;
}

// The drafts' fate, by every workgroup of a sequence for itself; the first one of them writes it.
template <bool BF16> __global__ __launch_bounds__(kThreads) void draft_decide_kernel(DraftKernelArgs a)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int E = BF16 ? 8 : 4;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int b = (int)(blockIdx.x / (unsigned)a.parts), part = (int)(blockIdx.x - (unsigned)b * (unsigned)a.parts);
    const int drafts = drafts_of(a, b), V = a.vecs * E;
    const double c = factor_of(a, b);
    const size_t v_row = (size_t)b * a.nv, d_row = (size_t)a.B * a.nv + (size_t)b * a.n, row_bytes = (size_t)a.vecs * 16;
    auto row_v = [&](int i) { return a.lv + (v_row + i) * row_bytes; };
    auto row_d = [&](int i) { return a.ld + ((size_t)b * a.n + i) * row_bytes; };
    // an exponential at a token, 0 at one that is none
    auto weight_at = [&](const uint8_t *row, int x, float ref) { return x >= 0 && x < V ? weight_of(logit<BF16>(row, x), c, -(double)ref * c) : 0.0; };
    auto over = [](double w, double sum) { return sum > 0 ? w / sum : 0.0; };
    auto chance_of = [](double px, double qx) { return qx > px ? (float)(px / qx) : px > 0 ? 1.0f : 0.0f; };
    __shared__ int stop;                     // the first draft that does not stand for sure: twice its place, and 1 where it falls for sure
    int at = 0;
    for (int from = 0;;) {
        if (tid == 0) stop = 2 * drafts;
        __syncthreads();
        for (int i = from + wave; i < a.n; i += kWaves) {
            float chance = 0;
            if (i < drafts) {
                const int x = a.tokens[(size_t)b * a.n + i];
                const double u = a.uniforms[(size_t)b * (a.n + 1) + i];
                const State sp = row_state(a, v_row + i, c);
                const double px = c == 0 ? (sp.first == x ? 1 : 0) : over(weight_at(row_v(i), x, sp.ref), sp.sum);
                double qx = 1;
                if (a.ld) {
                    const State sq = row_state(a, d_row + i, c);
                    qx = c == 0 ? (sq.first == x ? 1 : 0) : over(weight_at(row_d(i), x, sq.ref), sq.sum);
                }
                const double uq = u * qx;
                const bool near = c != 0 && px > 0 && uq > 0 && __builtin_fabs(uq - px) <= kNear * px;
                if (lane == 0 && (near || !(uq < px))) atomicMin(&stop, 2 * i + (near ? 0 : 1));
                chance = chance_of(px, qx);
            }
            if (part == 0 && lane == 0) a.out_chances[(size_t)b * a.n + i] = chance;
        }
        __syncthreads();
        const int s = stop;
        at = s >> 1;
        if (at >= drafts || (s & 1)) break;
        // as near to the border as that: again, on sums in fp64
        const int x = a.tokens[(size_t)b * a.n + at];
        const double u = a.uniforms[(size_t)b * (a.n + 1) + at];
        const float ref = row_state(a, v_row + at, c).ref;
        const double px = over(weight_at(row_v(at), x, ref), exact_sum<BF16>(row_v(at), a.vecs, c, ref));
        double qx = 1;
        if (a.ld) {
            const float rd = row_state(a, d_row + at, c).ref;
            qx = over(weight_at(row_d(at), x, rd), exact_sum<BF16>(row_d(at), a.vecs, c, rd));
        }
        if (part == 0 && tid == 0) a.out_chances[(size_t)b * a.n + at] = chance_of(px, qx);
        if (!(u * qx < px)) break;
        from = at + 1;
        __syncthreads();                                     // (`stop` has been read by all)
    }
    const bool down = at < drafts, draws = down || a.bonus;
    if (part == 0) {
        for (int j = tid; j <= a.n; j += kThreads)
            if (j != at || !draws) a.out_tokens[(size_t)b * (a.n + 1) + j] = j < at ? a.tokens[(size_t)b * a.n + j] : -1;
        if (tid == 0) a.out_accepted[b] = at;
    }
    Verdict verdict{kDone, at, 0, -1, 0, 0, c, 0};
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
            // p > q as e_p > e_q S_p / S_q; a row without any probability is below whatever there is
            verdict = Verdict{kDraw, at, minus, without, p.ref, q.ref, c, minus && q.sum > 0 ? p.sum / q.sum : 0};
        }
    }
    if (part == 0 && tid == 0) a.verdicts[b] = verdict;
    if (verdict.kind == kDone) return;
    // ---- this wave's part of the row that the token is drawn from
    const int per_wave = a.per_part / kWaves, begin = part * a.per_part + wave * per_wave, end = min(begin + per_wave, a.vecs);
    const u32x4 *const pv = reinterpret_cast<const u32x4 *>(row_v(at)), *const pd = minus ? reinterpret_cast<const u32x4 *>(row_d(at)) : pv;
    const double at_p = -(double)p.ref * c, at_q = -(double)q.ref * c;
    Sums s{0, 0, 0, 0, 0};
    if (begin < end) {
        u32x4 wv = pv[min(begin + lane, end - 1)], wd = pd[min(begin + lane, end - 1)];
        for (int v = begin + lane; v < end; v += 64) {
            float x[E], y[E];
            unpack<BF16>(wv, x);
            unpack<BF16>(wd, y);
            wv = pv[min(v + 64, end - 1)];                   // (the next ones, on their way meanwhile)
            wd = pd[min(v + 64, end - 1)];
            if (minus) {
                double of_vector = 0;
                bool open = false;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const double ep = weight_of(x[e], c, at_p), eq = weight_of(y[e], c, at_q);
                    const double more = __builtin_fma(-eq, verdict.even, ep);
                    const bool above = more > 0;
                    of_vector += ep;
                    s.q += eq;
                    s.above_p += above ? ep : 0;
                    s.above_q += above ? eq : 0;
                    open = open || __builtin_fabs(more) < kNear * ep;      // (not where both are 0)
                }
                s.p += of_vector;
                s.near_p += open ? of_vector : 0;
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const double ep = weight_of(x[e], c, at_p);
                    s.p += ep;
                    s.above_p += v * E + e != without ? ep : 0;
                }
            }
        }
    }
    s.q = wave_sum(s.q);
    s.above_q = wave_sum(s.above_q);
    s.near_p = wave_sum(s.near_p);
    s.p = wave_sum(s.p);
    s.above_p = wave_sum(s.above_p);
    if (lane == 0) a.sums[((size_t)b * a.parts + part) * kWaves + wave] = s;
#endif
}

// in a wave, the sum of a lane's value and all before it: within rows of sixteen lanes, then the rows' last lanes to the rows behind them
template <int CTRL, int ROWS> __device__ __forceinline__ double moved(double v)
{
    const u32x2 r = __builtin_bit_cast(u32x2, v);
    return __builtin_bit_cast(double, u32x2{(unsigned)__builtin_amdgcn_update_dpp(0, (int)r.x, CTRL, ROWS, 0xF, false),
                                            (unsigned)__builtin_amdgcn_update_dpp(0, (int)r.y, CTRL, ROWS, 0xF, false)});
}
__device__ __forceinline__ double up_to(double v)
{
    v += moved<0x111, 0xF>(v);                               // row_shr by 1, 2, 4, 8
    v += moved<0x112, 0xF>(v);
    v += moved<0x114, 0xF>(v);
    v += moved<0x118, 0xF>(v);
    v += moved<0x142, 0xA>(v);                               // row_bcast:15 to the second and fourth row
    v += moved<0x143, 0xC>(v);                               // row_bcast:31 to the upper half
    return v;
}
__device__ __forceinline__ double from_lane(double v, int lane)
{
    const u32x2 r = __builtin_bit_cast(u32x2, v);
    return __builtin_bit_cast(double, u32x2{(unsigned)__builtin_amdgcn_readlane((int)r.x, lane), (unsigned)__builtin_amdgcn_readlane((int)r.y, lane)});
}

// Of the threads' values v >= 0 in the threads' order, the first at which the running sum, begun at `base`, passes base + u * (their sum)
// or, if it is given, `mark`: which thread, and the sum before it.  Where rounding or u >= 1 leaves none, the last v > 0; -1 where
// there is none of those either.
struct Spot { int thread; double before, mark; };
__device__ __forceinline__ Spot spot_of(double v, double base, bool given, double mark, double u, double (*of_wave)[4])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const double upto = up_to(v), last = from_lane(upto, 63);
    if (lane == 0) of_wave[0][wave] = last;
    __syncthreads();
    double all = 0, pre = base;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const double x = of_wave[0][w];
        pre += w < wave ? x : 0;
        all += x;
    }
    if (!given) mark = base + u * all;
    const unsigned long long passed = __ballot(v > 0 && pre + upto > mark), some = __ballot(v > 0);
    const int first = passed ? __builtin_ctzll(passed) : -1, end = some ? 63 - __builtin_clzll(some) : -1;
    // per wave: the place, and what was before it
    const int at = first >= 0 ? first : end;
    const double before = pre + (at >= 0 ? from_lane(upto, at) - from_lane(v, at) : 0.0);
    if (lane == 0) {
        of_wave[1][wave] = first >= 0 ? 2 * 64 + first : end >= 0 ? 64 + end : 0;
        of_wave[2][wave] = before;
    }
    __syncthreads();
    Spot r{-1, 0, mark};
    bool done = false;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const int code = (int)of_wave[1][w];
        if (!done && code >= 64) {                           // (a later wave's last one counts only where nobody has passed)
            r.thread = w * 64 + (code & 63);
            r.before = of_wave[2][w];
        }
        done = done || code >= 128;
    }
    return r;
}

template <bool BF16> __global__ __launch_bounds__(kThreads) void draft_pick_kernel(DraftKernelArgs a)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int E = BF16 ? 8 : 4;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, b = blockIdx.x, pieces = a.parts * kWaves, per_piece = a.per_part / kWaves;
    __shared__ double of_wave[6][kWaves], again[kThreads];
    const Verdict verdict = a.verdicts[b];
    Sums s{0, 0, 0, 0, 0};
    if (verdict.kind == kDone) return;
    if (tid < pieces) s = a.sums[(size_t)b * pieces + tid];
    const double u = __builtin_fmax((double)a.uniforms[(size_t)b * (a.n + 1) + a.n], 0.0);
    const int at = verdict.at;
    const bool minus = verdict.minus != 0;
    const size_t row_bytes = (size_t)a.vecs * 16;
    const uint8_t *const row_v = a.lv + ((size_t)b * a.nv + at) * row_bytes, *const row_d = minus ? a.ld + ((size_t)b * a.n + at) * row_bytes : row_v;
    const u32x4 *const pv = reinterpret_cast<const u32x4 *>(row_v), *const pd = reinterpret_cast<const u32x4 *>(row_d);
    const double c = verdict.c, at_p = -(double)verdict.ref_p * c, at_q = -(double)verdict.ref_q * c;
    const double wave_p = wave_sum(s.p), wave_q = wave_sum(s.q), wave_near = wave_sum(s.near_p);
    if (lane == 0) {
        of_wave[3][wave] = wave_p;
        of_wave[4][wave] = wave_q;
        of_wave[5][wave] = wave_near;
    }
    __syncthreads();
    double all_p = 0, all_q = 0, near_p = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        all_p += of_wave[3][w];
        all_q += of_wave[4][w];
        near_p += of_wave[5][w];
    }
    const double inv_p = all_p > 0 ? 1.0 / all_p : 0.0, inv_q = all_q > 0 ? 1.0 / all_q : 0.0;
    // How far borders may be off as tokens stand on the wrong side of S_p / S_q:  such a token's p and q differ by no more than that quotient is
    // off, relative, and all of them go the same way.  Twice that.  (Values that are none: everything is taken again.)
    const double off = minus && near_p > 0 ? 2 * __builtin_fabs(verdict.even * (all_q * inv_p) - 1) * (near_p * inv_p) : 0.0;
    int token = -1;
    // what is left of p without q, on the sums at hand, then, where that leaves it open, on true ones; where p is nowhere above q, p itself
    enum { kLeft = 2, kAgain = 1, kAll = 0 };
    for (int how = kLeft; how >= kAll && token < 0; --how) {
        const bool left = how != kAll;
        auto weight = [&](float x, float y, int e) __attribute__((always_inline)) {
            double w = weight_of(x, c, at_p) * inv_p;
            if (left && minus) w = __builtin_fmax(w - weight_of(y, c, at_q) * inv_q, 0.0);
            return left && e == verdict.without ? 0.0 : w;
        };
        auto weights = [&](const u32x4 &wv, const u32x4 &wd, int v) __attribute__((always_inline)) {       // of a vector of the row
            float x[E], y[E];
            unpack<BF16>(wv, x);
            unpack<BF16>(wd, y);
            double sum = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) sum += weight(x[e], y[e], v * E + e);
            return sum;
        };
        double mine = left ? s.above_p * inv_p - s.above_q * inv_q : s.p * inv_p;
        if (how == kAgain) {
            if (off == 0) continue;
            again[tid] = s.near_p != 0 ? -1 : mine;          // (parts without such tokens stay as they are)
            __syncthreads();
            for (int k = wave; k < pieces; k += kWaves) {
                if (again[k] > -0.5) continue;
                const int begin = k * per_piece, end = min(begin + per_piece, a.vecs);
                u32x4 wv = pv[min(begin + lane, end - 1)], wd = pd[min(begin + lane, end - 1)];
                double sum = 0;
                for (int v = begin + lane; v < end; v += 64) {
                    const u32x4 now_v = wv, now_d = wd;
                    wv = pv[min(v + 64, end - 1)];
                    wd = pd[min(v + 64, end - 1)];
                    sum += weights(now_v, now_d, v);
                }
                sum = wave_sum(sum);
                if (lane == 0) again[k] = sum;
            }
            __syncthreads();
            mine = again[tid];
        }
        const Spot piece = spot_of(mine, 0, false, 0, u, of_wave);
        if (piece.thread < 0) continue;
        // ---- within the piece, neighbouring vectors per thread
        const int begin = piece.thread * per_piece, end = min(begin + per_piece, a.vecs), each = (end - begin + kThreads - 1) / kThreads;
        double sum = 0;
        const int first = begin + tid * each;
        for (int v = first; v < min(first + each, end); ++v) sum += weights(pv[v], pd[v], v);
        __syncthreads();                                     // (`of_wave` has been read)
        const Spot who = spot_of(sum, piece.before, true, piece.mark, 0, of_wave);
        if (who.thread >= 0) {
            // ---- within that thread's vectors, an element per lane, of every wave the same
            const int from = (begin + who.thread * each) * E, to = min(begin + (who.thread + 1) * each, end) * E;
            double done = who.before;
            int last = -1;
            bool clear = false;
            for (int e0 = from; e0 < to && token < 0; e0 += 64) {
                const int e = min(e0 + lane, to - 1);
                const double w = e0 + lane < to ? weight(logit<BF16>(row_v, e), logit<BF16>(row_d, e), e) : 0.0, upto = up_to(w);
                const unsigned long long passed = __ballot(w > 0 && done + upto > who.mark), some = __ballot(w > 0);
                if (passed) {
                    const int l = __builtin_ctzll(passed);
                    const double behind = done + from_lane(upto, l);
                    token = e0 + l;
                    clear = behind - who.mark > off && who.mark - (behind - from_lane(w, l)) > off;
                }
                if (some) last = e0 + 63 - __builtin_clzll(some);
                done += from_lane(upto, 63);
            }
            if (token < 0) token = last;
            if (how == kLeft && off != 0 && !clear) token = -1;
        }
        __syncthreads();
    }
    if (tid == 0) a.out_tokens[(size_t)b * (a.n + 1) + at] = token;      // (-1: no probability anywhere)
#endif
}

struct Plan { int vecs, splits, per_split, parts, per_part; size_t states, sums, bytes; };
Plan plan_of(int B, int n, int nv, int V, bool bf16, bool drafter)
{
    Plan p;
    p.vecs = (int)((long)V * (bf16 ? 2 : 4) / 16);
    const long rows = (long)B * nv + (drafter ? (long)B * n : 0);
    // about `want` workgroups, each of whole rounds of `unit` vectors once it has as many (a round that is short takes as long: 32 x 4 rows of
    // 152064 logits in lots of 1536 vectors 30.1 us, of 2048 27.4), at most `most` of a row
    auto divide = [&](long rows, long want, int most, long unit, int &per, int &count) {
        long v = (long)p.vecs * rows / want;                 // vectors per workgroup
        const long least = ((long)p.vecs + most - 1) / most;
        v = v > least ? v : least;
        const long whole = v > unit / 2 ? unit : kThreads;   // (256 at least: of a part a quarter per wave)
        v = (v + whole - 1) / whole * whole;
        per = (int)(v < 0x7ffff000 ? v : 0x7ffff000);
        count = (int)(((long)p.vecs + per - 1) / per);
    };
    divide(rows, 2048, kMostSplits, kThreads * kLoads, p.per_split, p.splits);
    divide(B, 1024, kMostParts, kThreads, p.per_part, p.parts);
    p.states = ((size_t)rows * p.splits * sizeof(State) + 255) / 256 * 256;
    p.sums = ((size_t)B * p.parts * kWaves * sizeof(Sums) + 255) / 256 * 256;
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
