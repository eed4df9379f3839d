// Attention over a paged cache (the drafter's call of Sec. 2.3 on a cache that is kept in pages), bf16 pages or e4m3 pages with one scale
// per page and head.
//     O = softmax(Q K^T / sqrt(d_k)) V   (Eq. 3)   over the keys that a sequence holds
// S^T = K Q^T and O^T = V^T P^T on 32x32x16 matrix instructions, a tile of 64 keys (bf16 pages: 32) at a time.  The cache is laid out
// for them: a lane's operand of the first product is 16-byte pieces of one key's row, of the second one keys of one head dim, which
// lie side by side in a page, so neither has to be turned over.  The tile's keys are dealt to the rows of S^T in such a way that the
// weights that a lane gets are the ones that it has to give to the second product:
//     lane half h, score tile T (0 .. NT - 1), accumulator i (0 .. 15)  <->  key 16 NT h + 16 T + i of the tile
// A unit of 16 keys (h, T) lies in one page whatever the page size, so its page and its scales are one value per lane and T.
// Tiles go to LDS by loads that no register waits for, a kilobyte of memory each in the order in which it lies there: the operands'
// own order, taken straight into registers, is sixteen bytes out of each of 32 rows per load, and cost more than the arithmetic (16
// sequences x 64 rows, 32/8 heads, 2048 e4m3 keys 51 us, with all loads from the nearest cache 50, with none 37; by LDS 43).
// A workgroup's four waves are one row block x 4 streams of keys, each with a state (reference, sum, O) of its own and a tile of its
// own in LDS, whose K is asked for again as soon as it is in registers, and V likewise; or two blocks x 2 streams with doubled tiles
// that two waves share.  The states are merged through LDS, the key range is split over workgroups where those are few, and the
// splits' states are merged by a second kernel.
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
[[maybe_unused]] constexpr float kRaise = 4096.0f;        // a reference is raised when a lane's weights of a tile add up to more
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
// across the two halves of a wave
__device__ __forceinline__ float as_float(unsigned w) { return __builtin_bit_cast(float, w); }       // (by value: in place it takes a vector's element 0)
__device__ __forceinline__ float halves_max(float x)
{
    typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
    const u32x2 r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    return fmaxf(as_float(r[0]), as_float(r[1]));
}
__device__ __forceinline__ float halves_other(float x) { return __shfl_xor(x, 32); }

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

// One 16-byte piece per lane from memory to LDS, 1 KB of it from `lds` on in the lanes' order; not known to the compiler, which neither
// counts nor waits for it.
__device__ __forceinline__ void to_lds(unsigned lds, const uint8_t *base, unsigned lane_offset)
{
    asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(lane_offset), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void to_lds(unsigned lds, const uint8_t *lane_address)
{
    asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(lane_address) : "memory", "m0");
}
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// NT: score tiles of 32 keys, 32 NT keys at a time.  ONE: those lie in one page (page_size >= 32 NT).  RG: row blocks of 32 per
// workgroup; its four waves are RG blocks x 4 / RG streams of keys.
template <int D, bool FP8, int NT, bool ONE, int RG>
__global__ __launch_bounds__(256, 2) void attn_paged_kernel(PagedKernelArgs a)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int EB = FP8 ? 1 : 2;
    constexpr int ROWB = D * EB, CH = ROWB / 16;     // bytes and 16-byte pieces per key
    constexpr int KR = CH / 2;                       // pieces of a lane's half of a key
    constexpr int DT = D / 32, KS = D / 16;          // head-dim tiles, k steps of S
    constexpr int TILE = 32 * NT, STREAMS = 4 / RG, UNITS = 2 * NT;
    constexpr int KB = TILE * ROWB, VB = D * TILE * EB, NK = KB / 1024, NV = VB / 1024;      // a tile in LDS: bytes and wave-wide loads
    constexpr int KPI = 1024 / ROWB;                 // keys per load
    constexpr int BUFS = RG == 1 ? 1 : 2;            // a wave's own tile is asked for piece by piece as it is used up; a shared one is doubled
    constexpr int PITCH = D + 4;
    constexpr int KVB = STREAMS * BUFS * (KB + VB), MERGEB = STREAMS == 1 ? 0 : 4 * 32 * PITCH * 4;
    static_assert(TILE * EB == 64, "a head dim's keys of a tile are four pieces");
    static_assert(NK % RG == 0 && NV % RG == 0, "the waves of a stream share its loads out");
    __shared__ __attribute__((aligned(1024))) uint8_t lds[KVB > MERGEB ? KVB : MERGEB];

    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int block = wave % RG, stream = wave / RG;
    unsigned bid = blockIdx.x;
    {                                                // workgroups that share keys: on one XCD
        const unsigned total = a.wgs, per = total >> 3, rem = total & 7;
        const unsigned xcd = bid & 7, slot = bid >> 3;
        bid = xcd * per + min(xcd, rem) + slot;
    }
    int rt, sp;
    place_of(bid, a.row_tiles, rt);
    place_of(bid, a.splits, sp);
    const int head = bid, b = head / a.Hkv, g = head - b * a.Hkv;
    const Share sh = share_of(uniform_load(a.kv_lens + b), a.max_pages, a.page_log2, a.splits);
    if (sp >= sh.used && sp > 0) return;
    const int v_first = (rt * RG + block) * 32;
    const size_t row_base = (size_t)head * a.rows_total;

    // ---- queries: of row l32 of the block, half of the head dims
    bf16x8 q[KS];
    {
        const int r = min(v_first + l32, a.rows_total - 1);
        const u32x4 *p = reinterpret_cast<const u32x4 *>(a.Q + (row_base + r) * (D * 2) + hh * D);
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = __builtin_bit_cast(bf16x8, p[s]);
    }

    const int t_begin = sp * sh.per_split * (2 / NT), t_end = min(t_begin + sh.per_split * (2 / NT), (sh.len + TILE - 1) / TILE);
    const int32_t *const row_of_table = a.table + (size_t)b * a.max_pages;
    const int P_log2 = a.page_log2;
    const unsigned in_page = (1u << P_log2) - 1;

    // ---- pages: of each unit of 16 keys, or of the tile
    constexpr int IDS = ONE ? 1 : UNITS;
    struct Pages { int id[IDS]; };
    auto pages_of = [&](int tile) __attribute__((always_inline)) {
        Pages p;
#pragma unroll
        for (int u = 0; u < IDS; ++u) p.id[u] = uniform_load(row_of_table + min((tile * TILE + 16 * u) >> P_log2, a.max_pages - 1));
        return p;
    };
    auto valid = [&](int id) __attribute__((always_inline)) { return (unsigned)id < (unsigned)a.num_pages; };
    auto place = [&](int id) __attribute__((always_inline)) { return (size_t)((valid(id) ? id : 0) * (long)a.Hkv + g); };      // page and head

    // ---- a tile's way into LDS: K [key][piece ^ sw(key)], V [head dim][piece ^ (dim / 2) % 4], so that the eight lanes that read at a time
    // are on different banks: lanes r of S^T's rows are keys (r & 3) + 16 NT (r & 4) / 4 + 4 (r & 24) / 8
    const unsigned tile_lds = (unsigned)(size_t)(__attribute__((address_space(3))) uint8_t *)lds + stream * (BUFS * (KB + VB));
    uint8_t *const tile_ptr = lds + stream * (BUFS * (KB + VB));
    auto sw = [&](int key, int upper) __attribute__((always_inline)) { return CH >= 8 ? (key & 3) | upper << 2 : (key >> 1 & 1) | upper << 1; };
    const int k_key = lane / CH, k_piece = lane % CH;
    const unsigned k_off[2] = {(unsigned)(k_key * ROWB + (k_piece ^ sw(k_key, 0)) * 16), (unsigned)(k_key * ROWB + (k_piece ^ sw(k_key, 1)) * 16)};
    const int v_piece = lane % 4 ^ (lane >> 3 & 3);
    const unsigned v_off = (((unsigned)lane / 4) << P_log2) * EB + v_piece * 16;
    auto load_k = [&](const Pages &p, int tile, unsigned buf) __attribute__((always_inline)) {
        const uint8_t *base[IDS];
#pragma unroll
        for (int u = 0; u < IDS; ++u) base[u] = a.Kc + ((place(p.id[u]) << P_log2) + ((unsigned)(tile * TILE + 16 * u) & in_page)) * ROWB;
#pragma unroll
        for (int i = 0; i < NK / RG; ++i) {
            // (with one block the loads' numbers are constants, and so are the units that they are in)
            const int I = RG == 1 ? i : block * (NK / RG) + i, u = I * KPI / 16;
            const uint8_t *from;
            if constexpr (ONE) {
                from = base[0] + I * 1024;
            } else {
                from = base[0] + I * 1024;
#pragma unroll
                for (int k = 1; k < IDS; ++k) from = u == k ? base[k] + (I * KPI - 16 * k) * ROWB : from;
            }
            to_lds(buf + I * 1024, from, u >= NT ? k_off[1] : k_off[0]);
        }
    };
    auto load_v = [&](const Pages &p, int tile, unsigned buf) __attribute__((always_inline)) {
        const int first = RG == 1 ? 0 : block * (NV / RG);
        const size_t step = ((size_t)16 << P_log2) * EB;             // sixteen head dims
        if constexpr (ONE) {
            const uint8_t *from = a.Vc + (((place(p.id[0]) * D) << P_log2) + ((unsigned)(tile * TILE) & in_page)) * EB + first * step;
#pragma unroll
            for (int i = 0; i < NV / RG; ++i) to_lds(buf + KB + (first + i) * 1024, from + i * step, v_off);
        } else {
            // the page of the lane's piece, by the bits of its unit (not by an index, which would put the pages into memory)
            const unsigned u = EB == 1 ? v_piece : v_piece >> 1, m0 = 0u - (u & 1), m1 = 0u - (u >> 1);
            unsigned id = ((unsigned)p.id[0] & ~m0) | ((unsigned)p.id[1] & m0);
            if constexpr (IDS == 4) id = (id & ~m1) | ((((unsigned)p.id[2] & ~m0) | ((unsigned)p.id[3] & m0)) & m1);
            const uint8_t *from = a.Vc + (((place((int)id) * D) << P_log2) + ((unsigned)(tile * TILE + 16 * u) & in_page)) * EB + (v_off - 16 * u * EB) + first * step;
#pragma unroll
            for (int i = 0; i < NV / RG; ++i) to_lds(buf + KB + (first + i) * 1024, from + i * step);
        }
    };
    // scales stay in scalar registers until they are used, so that nothing waits for them where they are asked for
    struct Scales { float k[IDS], v[IDS]; };
    auto load_scales = [&](const Pages &p) __attribute__((always_inline)) {
        Scales s;
#pragma unroll
        for (int u = 0; u < IDS; ++u) {
            s.k[u] = FP8 ? uniform_load(a.k_scale + place(p.id[u])) : 1.0f;
            s.v[u] = FP8 ? uniform_load(a.v_scale + place(p.id[u])) : 1.0f;
        }
        return s;
    };
    const unsigned upper = 0u - (unsigned)hh;
    auto of_half = [&](const float *x, int T) __attribute__((always_inline)) {
        if constexpr (ONE) return x[0];
        else return as_float((__builtin_bit_cast(unsigned, (float)x[T]) & ~upper) | (__builtin_bit_cast(unsigned, (float)x[NT + T]) & upper));
    };

    // ---- where a lane reads: its key's half of the head dims, its head dim's half of the keys
    const int kh = l32 >> 2 & 1;
    const int my_key = 16 * NT * kh + (l32 >> 4 & 1) * 8 + (l32 >> 3 & 1) * 4 + (l32 & 3), my_sw = sw(l32 & 3, kh);

    floatx16 o[DT];
    float m = kNone, l = 0;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[dt][i] = 0;

    Pages now, next, after{};
    Scales sc{}, sc_next{};
    const int mine = t_begin + stream;
    now = pages_of(mine);
    next = pages_of(mine + STREAMS);
    if (mine < t_end) {
        load_k(now, mine, tile_lds);
        load_v(now, mine, tile_lds);
    }
    sc = load_scales(now);
    // (the compiler's wait for the queries: here, as in the loop it would wait for every load on its way, every time)
#pragma unroll
    for (int k = 0; k < KS; ++k) asm volatile("" ::"v"(q[k]));
    const int rounds = (t_end - t_begin + STREAMS - 1) / STREAMS;
    for (int it = 0; it < rounds; ++it) {
        const int t = mine + it * STREAMS;
        const bool more = t + STREAMS < t_end;
        const unsigned buf_at = BUFS == 1 ? 0 : (it & 1) * (KB + VB);
        const uint8_t *const buf = tile_ptr + buf_at;
        if constexpr (RG == 1) {
            if (t >= t_end) break;
            wait_loads<NV>();
        } else {
            wait_loads<0>();
            asm volatile("s_barrier" ::: "memory");  // the tile is there for all, and the other buffer has been read by all
            if (more) {
                load_k(next, t + STREAMS, tile_lds + (KB + VB) - buf_at);
                load_v(next, t + STREAMS, tile_lds + (KB + VB) - buf_at);
            }
            sc_next = load_scales(next);             // (the scalar loads are unconditional: a branch would wait for them at its end)
            after = pages_of(t + 2 * STREAMS);
            if (t >= t_end) continue;
        }
        // ---- scores
        u32x4 kraw[NT][KR];
#pragma unroll
        for (int T = 0; T < NT; ++T)
#pragma unroll
            for (int i = 0; i < KR; ++i) kraw[T][i] = *reinterpret_cast<const u32x4 *>(buf + (my_key + 16 * T) * ROWB + ((hh * KR + i) ^ my_sw) * 16);
        if constexpr (RG == 1) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (more) load_k(next, t + STREAMS, tile_lds);
            sc_next = load_scales(next);             // (the scalar loads are unconditional: a branch would wait for them at its end)
            after = pages_of(t + 2 * STREAMS);
        }
        floatx16 s[NT];
#pragma unroll
        for (int T = 0; T < NT; ++T)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[T][i] = 0;
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int T = 0; T < NT; ++T) s[T] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fragment<FP8>(kraw[T], k), q[k], s[T], 0, 0, 0);
        // ---- the last tile's end, and units without a page: their keys take no part
        bool whole = t * TILE + TILE <= sh.len;
#pragma unroll
        for (int u = 0; u < IDS; ++u) whole = whole && valid(now.id[u]);
        float c[NT], vs[NT];
        int left[NT];                                // keys of the lane's unit that count
#pragma unroll
        for (int T = 0; T < NT; ++T) {
            c[T] = FP8 ? a.scale_log2 * of_half(sc.k, T) : a.scale_log2;
            vs[T] = of_half(sc.v, T);
            left[T] = 16;
        }
        if (!whole) {
#pragma unroll
            for (int T = 0; T < NT; ++T) {
                const bool there = ONE ? valid(now.id[0]) : (((unsigned)valid(now.id[T % IDS]) & ~upper) | ((unsigned)valid(now.id[(NT + T) % IDS]) & upper)) != 0;
                left[T] = there ? sh.len - (t * TILE + 16 * (NT * hh + T)) : 0;
                if (left[T] <= 0) c[T] = vs[T] = 1.0f;
#pragma unroll
                for (int i = 0; i < 16; ++i) s[T][i] = i < left[T] ? s[T][i] : -__builtin_inff();
            }
        }
        // ---- weights: with the reference in use; a sum that is too large (the first always is) raises it, and they are taken again
        float w[NT][16], sum;
        auto weigh = [&]() __attribute__((always_inline)) {
            sum = 0;
#pragma unroll
            for (int T = 0; T < NT; ++T)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    w[T][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[T][i], c[T], -m));
                    sum += w[T][i];
                }
        };
        weigh();
        if (__any(sum > kRaise)) {
            float top = -__builtin_inff();
#pragma unroll
            for (int T = 0; T < NT; ++T) {
                float x = s[T][0];
#pragma unroll
                for (int i = 1; i < 16; ++i) x = fmaxf(x, s[T][i]);
                top = fmaxf(top, x * c[T]);
            }
            const float to = fmaxf(halves_max(top), m), by = __builtin_amdgcn_exp2f(m - to);
            m = to;
            l *= by;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[dt][i] *= by;
            weigh();
        }
        l += sum;
        bf16x8 p[2 * NT];
#pragma unroll
        for (int T = 0; T < NT; ++T)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                u32x4 r;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x0 = w[T][8 * j + 2 * e], x1 = w[T][8 * j + 2 * e + 1];
                    r[e] = FP8 ? pack_bf16(x0 * vs[T], x1 * vs[T]) : pack_bf16(x0, x1);
                }
                p[2 * T + j] = __builtin_bit_cast(bf16x8, r);
            }
        // ---- output
        if constexpr (RG == 1) {
            if (more) wait_loads<NK>();
            else wait_loads<0>();
        }
        u32x4 vraw[DT][2];
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int i = 0; i < 2; ++i)
                vraw[dt][i] = *reinterpret_cast<const u32x4 *>(buf + KB + (dt * 32 + l32) * 64 + ((2 * hh + i) ^ (l32 >> 1 & 3)) * 16);
        if constexpr (RG == 1) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (more) load_v(next, t + STREAMS, tile_lds);
        }
        if (!whole) {                                // what lies behind may be no number, and 0 times it would be none
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    constexpr int PER = 4 / EB;
                    const int n = (FP8 ? left[i % NT] : left[0] - 8 * i) - x * PER;
                    const unsigned keep = n >= PER ? ~0u : n <= 0 ? 0u : (1u << (n * 8 * EB)) - 1;
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) vraw[dt][i][x] &= keep;
                }
        }
#pragma unroll
        for (int f = 0; f < 2 * NT; ++f)
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fragment<FP8>(vraw[dt], f), p[f], o[dt], 0, 0, 0);
        now = next;
        sc = sc_next;
        next = after;
    }
    l += halves_other(l);

    if constexpr (STREAMS == 1) {                    // a row is in one wave: four head dims of it at a time
        if (v_first + l32 >= a.rows_total) return;
        const size_t row = row_base + v_first + l32;
        const float inv = sh.used > 1 ? 1.0f : l > 0 ? 1.0f / l : 0.0f;              // no key at all: zeros
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int d0 = dt * 32 + 8 * i + 4 * hh;
                const float x0 = o[dt][4 * i] * inv, x1 = o[dt][4 * i + 1] * inv, x2 = o[dt][4 * i + 2] * inv, x3 = o[dt][4 * i + 3] * inv;
                if (sh.used <= 1) *reinterpret_cast<uint2 *>(a.O + (row * D + d0) * 2) = make_uint2(pack_bf16(x0, x1), pack_bf16(x2, x3));
                else *reinterpret_cast<float4 *>(a.part_o + (row * a.splits + sp) * D + d0) = make_float4(x0, x1, x2, x3);
            }
        if (sh.used > 1 && hh == 0) {
            a.part_ml[(row * a.splits + sp) * 2] = m;
            a.part_ml[(row * a.splits + sp) * 2 + 1] = l;
        }
    } else {
        // ---- the streams' states, merged: every thread finishes eight head dims of a row at a time
        float (*const o_sh)[32][PITCH] = reinterpret_cast<float (*)[32][PITCH]>(lds);
        __shared__ float ml_sh[4][2][32];
        __syncthreads();                             // the tiles have been read
        if (hh == 0) {
            ml_sh[wave][0][l32] = m;
            ml_sh[wave][1][l32] = l;
        }
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<float4 *>(&o_sh[wave][l32][dt * 32 + 8 * i + 4 * hh]) =
                    make_float4(o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]);
        __syncthreads();
        for (int u = tid; u < 32 * RG * (D / 8); u += 256) {
            const int r = u / (D / 8), d0 = (u % (D / 8)) * 8, blk = r / 32, in = r % 32;
            const int v = rt * RG * 32 + r;
            if (v >= a.rows_total) break;
            float M = ml_sh[blk][0][in];
#pragma unroll
            for (int k = 1; k < STREAMS; ++k) M = fmaxf(M, ml_sh[blk + k * RG][0][in]);
            float L = 0, x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < STREAMS; ++k) {
                const int w = blk + k * RG;
                const float f = __builtin_amdgcn_exp2f(ml_sh[w][0][in] - M);
                L += f * ml_sh[w][1][in];
                const float4 lo = *reinterpret_cast<const float4 *>(&o_sh[w][in][d0]), hi = *reinterpret_cast<const float4 *>(&o_sh[w][in][d0 + 4]);
                x[0] += f * lo.x; x[1] += f * lo.y; x[2] += f * lo.z; x[3] += f * lo.w;
                x[4] += f * hi.x; x[5] += f * hi.y; x[6] += f * hi.z; x[7] += f * hi.w;
            }
            const size_t row = row_base + v;
            if (sh.used <= 1) {
                const float inv = L > 0 ? 1.0f / L : 0.0f;
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
#endif
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

struct Plan { int rg, splits; long row_tiles, wgs; };
Plan plan_of(int n, int B, int H, int Hkv, long capacity)
{
    const long rows = (long)(H / Hkv) * n, heads = (long)B * Hkv;
    Plan p;
    p.rg = rows > 32 ? 2 : 1;
    p.row_tiles = (rows + 32 * p.rg - 1) / (32 * p.rg);
    const long base = heads * p.row_tiles, target = 256;
    long s = (target + base - 1) / base;
    const long most = capacity / 1024;
    if (s > most) s = most;
    if (s > kMaxSplits) s = kMaxSplits;
    p.splits = s < 1 ? 1 : (int)s;
    p.wgs = base * p.splits;
    return p;
}

template <int D, bool FP8, int NT, bool ONE> hipError_t attend(const PagedKernelArgs &k, const Plan &p, hipStream_t stream)
{
    const dim3 grid((unsigned)p.wgs), block(256);
    return p.rg == 1 ? launch(attn_paged_kernel<D, FP8, NT, ONE, 1>, grid, block, stream, k)
                     : launch(attn_paged_kernel<D, FP8, NT, ONE, 2>, grid, block, stream, k);
}
template <int D, bool FP8> hipError_t attend(const PagedKernelArgs &k, const Plan &p, hipStream_t stream)
{
    constexpr int NT = FP8 ? 2 : 1;                  // (bf16 pieces take twice the registers)
    return (1 << k.page_log2) >= 32 * NT ? attend<D, FP8, NT, true>(k, p, stream) : attend<D, FP8, NT, false>(k, p, stream);
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
