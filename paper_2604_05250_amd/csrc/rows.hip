// What happens to a projection's rows before attention (Sec. 2.2, Sec. 2.3): head norms, the rotation by position, and the way of
// keys and values into a paged cache.
//
//   norm      y = x / sqrt(mean(x^2) + eps) * w                             over the d elements of one head
//   rotation  (u, v) -> (u cos a - v sin a, v cos a + u sin a),  a = position * inv_freq[k],  for the pair k of the first rot dims
//   e4m3      code = rne(x / s), s = 2^e: one scale per page and head
//
// A row of d elements belongs to d / 16 lanes, each with two chunks of eight elements (16-byte accesses in bf16).  The chunks of a lane
// are chosen so that the two members of every pair are in one lane - chunk c and chunk c + rot/2 where halves are paired, neighbours
// otherwise - so a rotation needs no exchange, and lane c needs the angles 8c .. 8c + 7 in both pairings.
// Angles: position * inv_freq in revolutions, in fp64, and its fraction to fp32 (a product in fp32 is off by 2^-24 of the angle:
// a hundredth of a radian at position 130000).  bf16 and e4m3 results take the hardware's sine (off by some 2^-20), fp32 results sinpi.
#include "dd_internal.h"

#include <type_traits>

namespace dd {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ unsigned pack_bf16(float lo, float hi)
{
    floatx2 f = {lo, hi};
    return __builtin_bit_cast(unsigned, __builtin_convertvector(f, bf16x2));
}
__device__ __forceinline__ float bf16_lo(unsigned w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float bf16_hi(unsigned w) { return __builtin_bit_cast(float, w & 0xffff0000u); }

struct Bf16 { static constexpr int bytes = 2; };
struct F32 { static constexpr int bytes = 4; };

// eight consecutive elements as they are in memory
template <typename T> struct Chunk { uint4 w[T::bytes / 2]; };
template <typename T> __device__ __forceinline__ Chunk<T> load_chunk(const uint8_t *row, int element)
{
    Chunk<T> c;
    const uint4 *p = reinterpret_cast<const uint4 *>(row + element * T::bytes);
#pragma unroll
    for (int i = 0; i < T::bytes / 2; ++i) c.w[i] = p[i];
    return c;
}
__device__ __forceinline__ void unpack(const Chunk<Bf16> &c, float *x)
{
    const unsigned w[4] = {c.w[0].x, c.w[0].y, c.w[0].z, c.w[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = bf16_lo(w[i]); x[2 * i + 1] = bf16_hi(w[i]); }
}
__device__ __forceinline__ void unpack(const Chunk<F32> &c, float *x)
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        x[4 * i] = __builtin_bit_cast(float, c.w[i].x); x[4 * i + 1] = __builtin_bit_cast(float, c.w[i].y);
        x[4 * i + 2] = __builtin_bit_cast(float, c.w[i].z); x[4 * i + 3] = __builtin_bit_cast(float, c.w[i].w);
    }
}
__device__ __forceinline__ uint4 pack8_bf16(const float *x)
{
    return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}
template <typename T> __device__ __forceinline__ void store_chunk(uint8_t *row, int element, const float *x)
{
    uint4 *p = reinterpret_cast<uint4 *>(row + element * T::bytes);
    if constexpr (std::is_same<T, Bf16>::value) {
        p[0] = pack8_bf16(x);
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            p[i] = make_uint4(__builtin_bit_cast(unsigned, x[4 * i]), __builtin_bit_cast(unsigned, x[4 * i + 1]),
                              __builtin_bit_cast(unsigned, x[4 * i + 2]), __builtin_bit_cast(unsigned, x[4 * i + 3]));
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
    bool turns, halves;
};
__device__ __forceinline__ Pairing pairing(int lane, int rot, bool interleaved)
{
    Pairing p;
    p.turns = 16 * lane < rot;
    p.halves = p.turns && !interleaved;
    p.a = p.halves ? 8 * lane : 16 * lane;
    p.b = p.halves ? rot / 2 + 8 * lane : 16 * lane + 8;
    return p;
}

// cos and sin of the eight angles of a lane
template <bool EXACT> __device__ __forceinline__ void turn_of(const double *turns_per_step, long position, float *c, float *s)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const double r = (double)position * turns_per_step[i];
        const float f = (float)(r - __builtin_floor(r));     // revolutions, in [0, 1]
        if constexpr (EXACT) {
            s[i] = sinpif(2.0f * f);
            c[i] = cospif(2.0f * f);
        } else {
            s[i] = __builtin_amdgcn_sinf(f);
            c[i] = __builtin_amdgcn_cosf(f);
        }
    }
}
__device__ __forceinline__ void turns_per_step(const float *inv_freq, int lane, double *t)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = (double)inv_freq[8 * lane + i] * 0.15915494309189533577;      // 1 / 2 pi
}
__device__ __forceinline__ void rotate(float *x, const Pairing &p, const float *c, const float *s)     // x: both chunks, 16 values
{
    if (p.halves) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float u = x[i], v = x[8 + i];
            x[i] = u * c[i] - v * s[i];
            x[8 + i] = v * c[i] + u * s[i];
        }
    } else if (p.turns) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float u = x[2 * i], v = x[2 * i + 1];
            x[2 * i] = u * c[i] - v * s[i];
            x[2 * i + 1] = v * c[i] + u * s[i];
        }
    }
}
template <int D> __device__ __forceinline__ void norm(float *x, const float *w, float eps)
{
    float q = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) q += x[i] * x[i];
    const float r = 1.0f / sqrtf(row_sum<D / 16>(q) * (1.0f / D) + eps);
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = x[i] * r * w[i];
}

// ---------------------------------------------------------------- queries and keys for dense attention
// A lane keeps its place in the row and its token, and goes through `per_wg` heads: the angles and the weights are made once for all
// of them.  Reads and writes every row once: bound by memory where tokens are many.
template <typename T, int D>
__global__ __launch_bounds__(256) void norm_rotate_kernel(NormRotateArgs a)
{
    constexpr int LANES = D / 16, TOKENS = 256 / LANES;
    const int lane = threadIdx.x % LANES;
    const unsigned token = blockIdx.x * TOKENS + threadIdx.x / LANES;
    const bool live = token < a.tokens;
    const unsigned at = live ? token : a.tokens - 1;
    const long b = at / (unsigned)a.n, i = at - (unsigned)b * (unsigned)a.n;
    const bool is_q = (int)blockIdx.y < a.q_groups;
    const NormRotateSide &side = is_q ? a.q : a.k;
    const int first = ((int)blockIdx.y - (is_q ? 0 : a.q_groups)) * a.per_wg, last = min(first + a.per_wg, side.heads);
    const Pairing p = pairing(lane, a.rot, a.interleaved);

    const uint8_t *src = static_cast<const uint8_t *>(side.x) + (b * side.batch + i * side.row) * T::bytes;
    uint8_t *dst = static_cast<uint8_t *>(side.y) + ((b * side.heads) * a.n + i) * D * T::bytes;
    constexpr int U = 2;                                     // heads on their way
    Chunk<T> in[U][2];
    auto fetch = [&](int h, int u) __attribute__((always_inline)) {
        const uint8_t *row = src + (long)min(h, last - 1) * side.head * T::bytes;
        in[u][0] = load_chunk<T>(row, p.a);
        in[u][1] = load_chunk<T>(row, p.b);
    };
#pragma unroll
    for (int u = 0; u < U; ++u) fetch(first + u, u);

    float w[16], c[8], s[8];
    if (side.weight != nullptr) {
        unpack(load_chunk<T>(static_cast<const uint8_t *>(side.weight), p.a), w);
        unpack(load_chunk<T>(static_cast<const uint8_t *>(side.weight), p.b), w + 8);
    }
    if (p.turns) {
        double t[8];
        turns_per_step(a.inv_freq, lane, t);
        turn_of<std::is_same<T, F32>::value>(t, a.positions != nullptr ? (long)a.positions[at] : i, c, s);
    }
    for (int h0 = first; h0 < last; h0 += U) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = h0 + u;
            float x[16];
            unpack(in[u][0], x);
            unpack(in[u][1], x + 8);
            if (h0 + U < last) fetch(h + U, u);
            if (side.weight != nullptr) norm<D>(x, w, a.eps);
            rotate(x, p, c, s);
            if (live && h < last) {
                uint8_t *row = dst + (long)h * a.n * D * T::bytes;
                store_chunk<T>(row, p.a, x);
                store_chunk<T>(row, p.b, x + 8);
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

// One workgroup has one page of one sequence, its keys or its values, for `per_wg` heads one after the other, and one row of the page
// per d / 16 lanes.  It is the only one that writes this page and these heads, so the page's scale, its old rows and its new ones are
// decided here without an atomic.  The rows stay in registers between the maximum over the page and their storage.
// Values are stored with the keys of one head dim side by side, and are turned over in LDS.
template <typename T, int D, int PAGE, bool FP8>
__global__ __launch_bounds__(PAGE *D / 16) void page_append_kernel(PageAppendArgs a)
{
    constexpr int LANES = D / 16, THREADS = PAGE * LANES, WAVES = (THREADS + 63) / 64;
    constexpr int EB = FP8 ? 1 : 2;                          // bytes per stored element
    constexpr int PITCH = D * EB + 4;                        // bytes per row in LDS: an odd number of words
    __shared__ unsigned turned[PAGE * PITCH / 4];
    __shared__ float wave_max[2][WAVES];

    const int tid = threadIdx.x, lane = tid % LANES, slot = tid / LANES;
    unsigned bid = blockIdx.x;
    const bool values = bid & 1;
    bid >>= 1;
    const int group = bid % a.head_groups;
    bid /= a.head_groups;
    const int b = bid / a.pages_per_seq, j = bid % a.pages_per_seq;

    // ---- which rows of the page this call writes, and which it finds there
    const long start = a.starts[b];
    const long rows = a.n_rows != nullptr ? min(max(a.n_rows[b], 0), a.n) : a.n;
    const long held = a.kv_lens != nullptr ? (long)a.kv_lens[b] : start;
    const long page_index = (start >> a.page_log2) + j, first = page_index * PAGE;       // first: position of the page's first row
    if (page_index < 0 || page_index >= a.max_pages) return;
    if (first >= start + rows || rows == 0) return;          // (first + PAGE > start: j >= 0)
    const int page = a.table[(long)b * a.max_pages + page_index];
    if (page < 0 || page >= a.num_pages) return;
    const long pos = first + slot;
    const bool written = pos >= start && pos < start + rows;
    const bool kept = !written && pos < held;
    const bool keeps = min(start, held) > first || min(held, first + PAGE) > start + rows;       // some row is kept

    Pairing p = pairing(lane, values ? 0 : a.rot, a.interleaved);
    const PageAppendSide &side = values ? a.v : a.k;
    const long r = written ? pos - start : (start > first ? 0 : first - start);          // (a row that exists)
    const uint8_t *src = static_cast<const uint8_t *>(side.x) + (b * side.batch + r * side.row) * T::bytes;
    float w[16], c[8], s[8];
    if (!values) {
        if (a.weight != nullptr) {
            unpack(load_chunk<T>(static_cast<const uint8_t *>(a.weight), p.a), w);
            unpack(load_chunk<T>(static_cast<const uint8_t *>(a.weight), p.b), w + 8);
        }
        if (p.turns) {
            double t[8];
            turns_per_step(a.inv_freq, lane, t);
            turn_of<false>(t, pos, c, s);
        }
    }
    const int g_end = min((group + 1) * a.per_wg, a.Hkv);
    for (int g = group * a.per_wg, turn = 0; g < g_end; ++g, turn ^= 1) {
        float x[16];
        unpack(load_chunk<T>(src + (long)g * side.head * T::bytes, p.a), x);
        unpack(load_chunk<T>(src + (long)g * side.head * T::bytes, p.b), x + 8);
        if (!values) {
            if (a.weight != nullptr) norm<D>(x, w, a.eps);
            rotate(x, p, c, s);
        }
        const long at = (long)page * a.Hkv + g;              // page and head
        uint8_t *const store = static_cast<uint8_t *>(side.cache) + at * PAGE * D * EB;
        float by = 1.0f;                                     // kept codes: their old scale over the new one
        if constexpr (FP8) {
            float m = 0;
            if (written) {
#pragma unroll
                for (int i = 0; i < 16; ++i) m = fmaxf(m, fabsf(x[i]));
            }
            for (int k = 32; k; k >>= 1) m = fmaxf(m, __shfl_xor(m, k));
            if ((tid & 63) == 0) wave_max[turn][tid >> 6] = m;
            const float old = keeps ? side.scale[at] : 0.0f;
            __syncthreads();
            for (int k = 0; k < WAVES; ++k) m = fmaxf(m, wave_max[turn][k]);
            float scale = scale_for(m);
            if (keeps) {
                scale = fmaxf(scale, old);
                by = old / scale;
            }
            if (tid == 0) side.scale[at] = scale;            // (the old one was read before the barrier)
            const Divide divide(scale);
            divide(x);
        }
        if (!values) {
            uint8_t *const row = store + (long)slot * D * EB;
            if constexpr (FP8) {
                uint2 *const pa = reinterpret_cast<uint2 *>(row + p.a), *const pb = reinterpret_cast<uint2 *>(row + p.b);
                if (written) {
                    *pa = make_uint2(codes4(x[0], x[1], x[2], x[3]), codes4(x[4], x[5], x[6], x[7]));
                    *pb = make_uint2(codes4(x[8], x[9], x[10], x[11]), codes4(x[12], x[13], x[14], x[15]));
                } else if (kept && by != 1.0f) {
                    const uint2 ca = *pa, cb = *pb;
                    *pa = make_uint2(regrown4(ca.x, by), regrown4(ca.y, by));
                    *pb = make_uint2(regrown4(cb.x, by), regrown4(cb.y, by));
                }
            } else if (written) {
                store_chunk<Bf16>(row, p.a, x);
                store_chunk<Bf16>(row, p.b, x + 8);
            }
            continue;
        }
        // ---- values: rows into LDS, then for four head dims the sixteen (bf16: two head dims, the eight) keys of a vector
        unsigned *const mine = turned + slot * (PITCH / 4) + lane * (4 * EB);
        if constexpr (FP8) {
#pragma unroll
            for (int i = 0; i < 4; ++i) mine[i] = codes4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) mine[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
        }
        __syncthreads();
        constexpr int KEYS = 16 / EB, DIMS = 4 / EB, UNITS = (PAGE / KEYS) * (D / DIMS);
        for (int u = tid; u < UNITS; u += THREADS) {
            const int k0 = (u % (PAGE / KEYS)) * KEYS, dw = u / (PAGE / KEYS);           // first key, word of the row
            const long at0 = first + k0;
            const bool all = at0 >= start && at0 + KEYS <= start + rows;
            const bool some = at0 < start + rows && at0 + KEYS > start;
            if (!some && by == 1.0f) continue;
            unsigned in[KEYS];
#pragma unroll
            for (int k = 0; k < KEYS; ++k) in[k] = turned[(k0 + k) * (PITCH / 4) + dw];
#pragma unroll
            for (int q = 0; q < DIMS; ++q) {
                unsigned out[4];
#pragma unroll
                for (int o = 0; o < 4; ++o) {
                    if constexpr (FP8) {
                        const unsigned lo = __builtin_amdgcn_perm(in[4 * o + 1], in[4 * o], 0x0c0c0000u | (unsigned)(q | (q + 4) << 8));
                        const unsigned hi = __builtin_amdgcn_perm(in[4 * o + 3], in[4 * o + 2], 0x0c0c0000u | (unsigned)(q | (q + 4) << 8));
                        out[o] = lo | hi << 16;
                    } else {
                        out[o] = __builtin_amdgcn_perm(in[2 * o + 1], in[2 * o], q ? 0x07060302u : 0x05040100u);
                    }
                }
                uint4 *const to = reinterpret_cast<uint4 *>(store + ((long)(dw * DIMS + q) * PAGE + k0) * EB);
                if (!all) {                                  // the other keys of the vector: kept codes in the new scale, the rest as it was
                    const uint4 was = *to;
                    const unsigned old[4] = {was.x, was.y, was.z, was.w};
#pragma unroll
                    for (int o = 0; o < 4; ++o) {
                        unsigned grown = old[o], is_new = 0, is_kept = 0;
                        if constexpr (FP8) grown = by != 1.0f ? regrown4(old[o], by) : old[o];
#pragma unroll
                        for (int e = 0; e < KEYS / 4; ++e) {
                            const long at1 = at0 + o * (KEYS / 4) + e;
                            const unsigned field = (FP8 ? 0xffu : 0xffffu) << (e * 8 * EB);
                            if (at1 >= start && at1 < start + rows) is_new |= field;
                            else if (at1 < held) is_kept |= field;
                        }
                        out[o] = (out[o] & is_new) | (grown & is_kept) | (old[o] & ~(is_new | is_kept));
                    }
                }
                *to = make_uint4(out[0], out[1], out[2], out[3]);
            }
        }
        __syncthreads();
    }
}

template <typename T, int D, int PAGE>
hipError_t append_rows(const PageAppendArgs &a, bool fp8, unsigned wgs, hipStream_t stream)
{
    const dim3 block(PAGE * D / 16);
    return fp8 ? launch(page_append_kernel<T, D, PAGE, true>, dim3(wgs), block, stream, a) : launch(page_append_kernel<T, D, PAGE, false>, dim3(wgs), block, stream, a);
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

}  // namespace

hipError_t launch_norm_rotate(NormRotateArgs a, int d, bool bf16, hipStream_t stream)
{
    const int per_wg_tokens = 256 / (d / 16);
    const long tiles = ((long)a.tokens + per_wg_tokens - 1) / per_wg_tokens;
    const int heads = a.q.heads + a.k.heads;
    // heads per workgroup: as many as leave eight workgroups per compute unit
    long groups = (2048 + tiles - 1) / tiles;
    if (groups > heads) groups = heads;
    a.per_wg = (int)((heads + groups - 1) / groups);
    a.q_groups = (a.q.heads + a.per_wg - 1) / a.per_wg;
    const int k_groups = (a.k.heads + a.per_wg - 1) / a.per_wg;
    const dim3 grid((unsigned)tiles, (unsigned)(a.q_groups + k_groups));
    if (bf16) return d == 128 ? launch(norm_rotate_kernel<Bf16, 128>, grid, dim3(256), stream, a) : launch(norm_rotate_kernel<Bf16, 64>, grid, dim3(256), stream, a);
    return d == 128 ? launch(norm_rotate_kernel<F32, 128>, grid, dim3(256), stream, a) : launch(norm_rotate_kernel<F32, 64>, grid, dim3(256), stream, a);
}

long page_append_wgs(int n, int B, int Hkv, int page_log2)
{
    const long page = 1L << page_log2;
    return 2L * B * Hkv * ((n + page - 2) / page + 1);
}

hipError_t launch_page_append(PageAppendArgs a, int d, bool rows_bf16, bool fp8, hipStream_t stream)
{
    const long page = 1L << a.page_log2;
    a.pages_per_seq = (int)((a.n + page - 2) / page + 1);    // that n rows can touch, wherever they begin
    a.per_wg = 1;
    a.head_groups = (a.Hkv + a.per_wg - 1) / a.per_wg;
    const unsigned wgs = (unsigned)(2L * a.B * a.pages_per_seq * a.head_groups);
    if (rows_bf16) return d == 128 ? append_rows<Bf16, 128>(a, fp8, wgs, stream) : append_rows<Bf16, 64>(a, fp8, wgs, stream);
    return d == 128 ? append_rows<F32, 128>(a, fp8, wgs, stream) : append_rows<F32, 64>(a, fp8, wgs, stream);
}

}  // namespace dd
