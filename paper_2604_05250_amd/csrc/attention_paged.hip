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
// sequences x 64 rows, 32/8 heads, 2048 e4m3 keys 51 us, with all loads from the nearest cache 50, with none 37; by LDS 43, in three
// stages 40).
// A workgroup's four waves are one row block x 4 streams of keys, each with a state (reference, sum, O) of its own and a tile of its
// own in LDS, whose K is asked for again as soon as it is in registers, and V likewise; or two blocks x 2 streams or four x 1, with
// doubled tiles that two or four waves share (as above 44.5, 40.2 and 49.0 us; four blocks x 2 streams in eight waves 42.9).  The next
// keys' scores are computed beside these keys' weights, for e4m3 pages the last keys' output beside both, so that the matrix cores and
// the vector units have work at the same time (with e4m3 pages as above they are at it 44 and 48 % of a wave's cycles, and the clock at 1.8
// GHz; a wave waits 26 % of them for data and others).  The states are merged through LDS, the key range is split over workgroups where
// those are few, and the splits' states are merged by a second kernel.
// e4m3 codes become bf16 exactly in registers.  k_scale goes into the factor of the exponent; of v_scale the power of two goes into the
// decoding of V, which is exact (bf16 for its range: scales span 2^-126 .. 2^88), and the rest, 1 where this library made the scale,
// into the exponent.  Weights are rounded to bf16 (2^-8 of each at most, as the result is), their sum is the one of the rounded ones.
#include "attention_common.h"
#include "dd_internal.h"

#include <type_traits>

namespace dd {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr float kNone = -1.0e30f;        // the reference of a row that has met no key
[[maybe_unused]] constexpr float kMargin = 7.0f;          // a reference is set this far above a tile's maximum (log2 units)
constexpr int kMaxSplits = 64;
[[maybe_unused]] constexpr int kWaves = 4;           // per workgroup
constexpr int kFewRows = 32;             // of a key/value head: one row block
constexpr int kUnits = 256;              // compute units
// tiles of 64 keys that a split has at least: with few rows, with more, and with more where workgroups share a compute unit
constexpr int kSplitTiles = 4, kSplitTilesMany = 8, kSplitTilesShared = 32;

// eight e4m3 codes times the power of two in `scale` (the instruction takes no more of it), exactly
__device__ __forceinline__ bf16x8 decode8(unsigned w0, unsigned w1, float scale)
{
    const u32x4 r = {__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, false)),
                     __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, true)),
                     __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, false)),
                     __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, true))};
    return __builtin_bit_cast(bf16x8, r);
}
// fragment `f` (eight elements) of a lane's consecutive elements
template <bool FP8> __device__ __forceinline__ bf16x8 fragment(const u32x4 *raw, int f, float scale)
{
    if constexpr (FP8) return decode8(raw[f / 2][(f % 2) * 2], raw[f / 2][(f % 2) * 2 + 1], scale);
    else return __builtin_bit_cast(bf16x8, raw[f]);
}
// across the two halves of a wave
__device__ __forceinline__ float halves_max(float x)
{
    const u32x2 r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    return fmaxf(as_float(r[0]), as_float(r[1]));
}
__device__ __forceinline__ float halves_other(float x) { return __shfl_xor(x, 32); }

// What the first loads need is in registers when a wave starts, as leading scalar arguments (fourteen words); the rest arrives meanwhile.
struct PagedTail {
    const uint8_t *Q;
    const float *k_scale, *v_scale;
    uint8_t *O;
    float *part_o, *part_ml;             // [rows][splits][d], [rows][splits][2]
    float scale_log2;                    // log2(e) / sqrt(d)
};
#define DD_PAGED_HEAD const int32_t *table, const int32_t *kv_lens, const uint8_t *Kc, const uint8_t *Vc, int Hkv, int rows_total, int num_pages, \
                      int max_pages, unsigned launched, unsigned shape // launched: workgroups, kLongSplits; shape: row tiles, splits - 1 (6
                                                                       // bits), log2(page_size / 16) (2 bits)

// How a sequence's tiles are shared out over the splits of a call: tiles per split and splits that have any.  The call's splits go by what
// its table can hold, a sequence's by what it holds: with many rows and more workgroups than compute units (kLongSplits) only long ones
// pay.  Workgroups that have none may not sit between the others (26.0 us where the first figure below is 20.8), so this is for calls whose
// row blocks the eight XCDs share evenly.  us with this / with splits of half of the keys, and at a table that is no wider than that,
// 64 rows, 32/8 heads:
//     sequences x keys, table     e4m3                  bf16
//     4 x 2048, 8192              20.8 / 23.4, 18.3     23.4 / 25.2, 21.1
//     3 x 2048, 8192              19.0 / 20.3, 16.1     22.2 / 23.0, 19.1
//     4 x 3008, 4096              26.0 / 26.8           30.2 / 31.8
//     3 x 3008, 4096              24.6 / 24.7, 21.9     29.3 / 28.3, 26.3
constexpr unsigned kLongSplits = 1u << 31;
struct Share { int tiles, per_split, used, len; };
__device__ __forceinline__ Share share_of(int len, int max_pages, int page_log2, int splits, int rows_total, unsigned launched)
{
    Share s;
    s.len = min(max(len, 0), max_pages << page_log2);        // (less than 2^30)
    s.tiles = (int)(((unsigned)s.len + 63u) >> 6);
    if (launched & kLongSplits) splits = min(splits, max(s.tiles / kSplitTilesShared, 1));
    s.per_split = max((s.tiles + splits - 1) / splits, rows_total <= kFewRows ? kSplitTiles : kSplitTilesMany);
    s.used = s.tiles == 0 ? 0 : (s.tiles + s.per_split - 1) / s.per_split;
    return s;
}

// One 16-byte piece per lane from memory to LDS, 1 KB of it from `lds` on in the lanes' order; not known to the compiler, which neither
// counts nor waits for it.
__device__ __forceinline__ void to_lds(unsigned lds, const uint8_t *base, unsigned lane_offset)
{
    asm volatile(DD_SET_M0_BASE "global_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(lane_offset), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void to_lds(unsigned lds, const uint8_t *lane_address)
{
    asm volatile(DD_SET_M0 "global_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(lane_address) : "memory", "m0");
}
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// NT: score tiles of 32 keys, 32 NT keys at a time.  ONE: those lie in one page (page_size >= 32 NT).  RG: row blocks of 32 per
// workgroup; its four waves are RG blocks x 4 / RG streams of keys.
template <int D, bool FP8, int NT, bool ONE, int RG>
__global__ __launch_bounds__(256, 2) void attn_paged_kernel(DD_PAGED_HEAD, PagedTail a)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int EB = FP8 ? 1 : 2;
    constexpr int ROWB = D * EB, CH = ROWB / 16;     // bytes and 16-byte pieces per key
    constexpr int KR = CH / 2;                       // pieces of a lane's half of a key
    constexpr int DT = D / 32, KS = D / 16;          // head-dim tiles, k steps of S
    constexpr int TILE = 32 * NT, STREAMS = kWaves / RG, UNITS = 2 * NT;
    constexpr int KB = TILE * ROWB, VB = D * TILE * EB, NK = KB / 1024, NV = VB / 1024;      // a tile in LDS: bytes and wave-wide loads
    constexpr int KPI = 1024 / ROWB;                 // keys per load
    constexpr int BUFS = RG == 1 ? 1 : 2;            // a wave's own tile is asked for piece by piece as it is used up; a shared one is doubled
    constexpr int PITCH = D + 4;
    constexpr int KVB = STREAMS * BUFS * (KB + VB), MERGEB = STREAMS == 1 ? 0 : kWaves * 32 * PITCH * 4;
    static_assert(TILE * EB == 64, "a head dim's keys of a tile are four pieces");
    static_assert(NK % RG == 0 && NV % RG == 0, "the waves of a stream share its loads out");
    static_assert(RG == 1 || (NK + NV) / RG <= 8, "eight loads are asked for in a round");
    __shared__ __attribute__((aligned(1024))) uint8_t lds[KVB > MERGEB ? KVB : MERGEB];

    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int block = wave % RG, stream = wave / RG;
    const int P_log2 = 4 + (int)(shape & 3), splits = (int)(shape >> 2 & 63) + 1;
    unsigned bid = blockIdx.x;
    {                                                // workgroups that share keys: on one XCD
        const unsigned wgs = launched & ~kLongSplits, per = wgs >> 3, rem = wgs & 7;
        const unsigned xcd = bid & 7, slot = bid >> 3;
        bid = xcd * per + min(xcd, rem) + slot;
        if (launched & kLongSplits) {                // and there split after split, each of all of them: units get as much of each
            const unsigned each = per / (unsigned)splits, s = slot / each, pair = xcd * each + (slot - s * each), tiles = shape >> 8;
            bid = (pair / tiles * (unsigned)splits + s) * tiles + pair % tiles;
        }
    }
    int rt, sp;
    place_of(bid, shape >> 8, rt);
    place_of(bid, splits, sp);
    const unsigned head = bid, b = head / (unsigned)Hkv, g = head - b * (unsigned)Hkv;
    const int32_t *const row_of_table = table + (size_t)b * max_pages;
    const unsigned in_page = (1u << P_log2) - 1;
    constexpr int IDS = ONE ? 1 : UNITS;             // pages: of the tile, or of each unit of 16 keys
    struct Pages { int id[IDS]; };
    auto pages_of = [&](int tile) __attribute__((always_inline)) {
        Pages p;
#pragma unroll
        for (int u = 0; u < IDS; ++u) p.id[u] = uniform_load(row_of_table + min((tile * TILE + 16 * u) >> P_log2, max_pages - 1));
        return p;
    };
    const int held = uniform_load(kv_lens + b);
    Pages now, next, after;
    if (splits == 1) {                               // (not after the length: the pages are known without it)
        now = pages_of(stream);
        next = pages_of(stream + STREAMS);
        after = pages_of(stream + 2 * STREAMS);
    }
    const Share sh = share_of(held, max_pages, P_log2, splits, rows_total, launched);
    if (sp >= sh.used && sp > 0) return;
    const int v_first = (rt * RG + block) * 32;
    const size_t row_base = (size_t)head * rows_total;
    const int t_begin = sp * sh.per_split * (2 / NT), t_end = min(t_begin + sh.per_split * (2 / NT), (sh.len + TILE - 1) / TILE);
    const int mine = t_begin + stream;
    if (splits > 1) {
        now = pages_of(mine);
        next = pages_of(mine + STREAMS);
        after = pages_of(mine + 2 * STREAMS);
    }

    // ---- queries: of row l32 of the block, half of the head dims
    bf16x8 q[KS];
    {
        const int r = min(v_first + l32, rows_total - 1);
        const u32x4 *p = reinterpret_cast<const u32x4 *>(a.Q + (row_base + r) * (D * 2) + hh * D);
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = __builtin_bit_cast(bf16x8, p[s]);
    }

    // every stream takes as many tiles; those behind the split's last key are masked whole
    const int rounds = (t_end - t_begin + STREAMS - 1) / STREAMS, key_end = min(sh.len, t_end * TILE);
    auto valid = [&](int id) __attribute__((always_inline)) { return (unsigned)id < (unsigned)num_pages; };
    auto place = [&](int id) __attribute__((always_inline)) { return (size_t)((valid(id) ? id : 0) * (long)Hkv + g); };      // page and head

    // ---- a tile's way into LDS: K [key][piece ^ sw(key)], V [head dim][piece ^ (dim / 2) % 4], so that the eight lanes that read at a time
    // are on different banks: lanes r of S^T's rows are keys (r & 3) + 16 NT (r & 4) / 4 + 4 (r & 24) / 8
    uint8_t *const tile_ptr = lds + stream * (BUFS * (KB + VB));
    const unsigned k_lds = (unsigned)(size_t)(__attribute__((address_space(3))) uint8_t *)lds + stream * (BUFS * (KB + VB)), v_lds = k_lds + BUFS * KB;
    auto sw = [&](int key, int upper) __attribute__((always_inline)) { return CH >= 8 ? (key & 3) | upper << 2 : (key >> 1 & 1) | upper << 1; };
    const int k_key = lane / CH, k_piece = lane % CH;
    const unsigned k_off[2] = {(unsigned)(k_key * ROWB + (k_piece ^ sw(k_key, 0)) * 16), (unsigned)(k_key * ROWB + (k_piece ^ sw(k_key, 1)) * 16)};
    const int v_piece = lane % 4 ^ (lane >> 3 & 3);
    const unsigned v_off = (((unsigned)lane / 4) << P_log2) * EB + v_piece * 16;
    struct KFrom { const uint8_t *base[IDS]; };
    auto k_from = [&](const Pages &p, int tile) __attribute__((always_inline)) {
        KFrom f;
#pragma unroll
        for (int u = 0; u < IDS; ++u) f.base[u] = Kc + ((place(p.id[u]) << P_log2) + ((unsigned)(tile * TILE + 16 * u) & in_page)) * ROWB;
        return f;
    };
    auto put_k = [&](const KFrom &f, unsigned buf, int i) __attribute__((always_inline)) {
        // (with one block the loads' numbers are constants, and so are the units that they are in)
        const int I = RG == 1 ? i : block * (NK / RG) + i, u = I * KPI / 16;
        const uint8_t *from = f.base[0] + I * 1024;
        if constexpr (!ONE) {
#pragma unroll
            for (int k = 1; k < IDS; ++k) from = u == k ? f.base[k] + (I * KPI - 16 * k) * ROWB : from;
        }
        to_lds(buf + I * 1024, from, u >= NT ? k_off[1] : k_off[0]);
    };
    const size_t v_step = ((size_t)16 << P_log2) * EB;               // sixteen head dims
    const int v_begin = RG == 1 ? 0 : block * (NV / RG);
    auto v_from = [&](const Pages &p, int tile) __attribute__((always_inline)) {         // the tile's, or the lane's, first address
        if constexpr (ONE) {
            return Vc + (((place(p.id[0]) * D) << P_log2) + ((unsigned)(tile * TILE) & in_page)) * EB + v_begin * v_step;
        } else {
            // the page of the lane's piece, by the bits of its unit (not by an index, which would put the pages into memory)
            const unsigned u = EB == 1 ? v_piece : v_piece >> 1, m0 = 0u - (u & 1), m1 = 0u - (u >> 1);
            unsigned id = ((unsigned)p.id[0] & ~m0) | ((unsigned)p.id[1] & m0);
            if constexpr (IDS == 4) id = (id & ~m1) | ((((unsigned)p.id[2] & ~m0) | ((unsigned)p.id[3] & m0)) & m1);
            return Vc + (((place((int)id) * D) << P_log2) + ((unsigned)(tile * TILE + 16 * u) & in_page)) * EB + (v_off - 16 * u * EB) + v_begin * v_step;
        }
    };
    auto put_v = [&](const uint8_t *from, unsigned buf, int i) __attribute__((always_inline)) {
        if constexpr (ONE) to_lds(buf + (v_begin + i) * 1024, from + i * v_step, v_off);
        else to_lds(buf + (v_begin + i) * 1024, from + i * v_step);
    };
    auto load_k = [&](const Pages &p, int tile, unsigned buf) __attribute__((always_inline)) {
        const KFrom f = k_from(p, tile);
#pragma unroll
        for (int i = 0; i < NK / RG; ++i) put_k(f, buf, i);
    };
    auto load_v = [&](const Pages &p, int tile, unsigned buf) __attribute__((always_inline)) {
        const uint8_t *const f = v_from(p, tile);
#pragma unroll
        for (int i = 0; i < NV / RG; ++i) put_v(f, buf, i);
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

    // ---- a tile's K from LDS, a half of the keys (T) at a time, and its V
    auto read_k = [&](u32x4 *kraw, int T, int turn) __attribute__((always_inline)) {
        const uint8_t *const buf = tile_ptr + (BUFS == 1 ? 0 : (turn & 1) * KB);
#pragma unroll
        for (int i = 0; i < KR; ++i) kraw[i] = *reinterpret_cast<const u32x4 *>(buf + (my_key + 16 * T) * ROWB + ((hh * KR + i) ^ my_sw) * 16);
    };
    auto read_v = [&](u32x4 (*vraw)[2], int first, int last, int turn) __attribute__((always_inline)) {     // pieces first .. last
        const uint8_t *const buf = tile_ptr + BUFS * KB + (BUFS == 1 ? 0 : (turn & 1) * VB);
#pragma unroll
        for (int i = first; i <= last; ++i)
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
                vraw[dt][i] = *reinterpret_cast<const u32x4 *>(buf + (dt * 32 + l32) * 64 + ((2 * hh + i) ^ (l32 >> 1 & 3)) * 16);
    };
    auto zeros = [&]() __attribute__((always_inline)) {
        floatx16 z;
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i] = 0;
        return z;
    };
    // ---- what a tile's scores and values are multiplied by: the factor of the exponent, v_scale, of its significand in [1, 2) the
    // logarithm and the reciprocal (its power of two goes into the decoding of V)
    struct Factors {
        float c[NT], vs[NT], shift[NT], part[NT];
        int left[NT];                                // keys of the lane's unit that count
        bool whole;
    };
    auto factors_of = [&](const Pages &p, const Scales &x, int t) __attribute__((always_inline)) {
        Factors f;
        f.whole = t * TILE + TILE <= key_end;
#pragma unroll
        for (int u = 0; u < IDS; ++u) f.whole = f.whole && valid(p.id[u]);
#pragma unroll
        for (int T = 0; T < NT; ++T) {
            f.c[T] = FP8 ? a.scale_log2 * of_half(x.k, T) : a.scale_log2;
            f.vs[T] = of_half(x.v, T);
            f.left[T] = 16;
        }
        if (!f.whole) {                              // the last tile's end, and units without a page: their keys take no part
#pragma unroll
            for (int T = 0; T < NT; ++T) {
                const bool there = ONE ? valid(p.id[0]) : (((unsigned)valid(p.id[T % IDS]) & ~upper) | ((unsigned)valid(p.id[(NT + T) % IDS]) & upper)) != 0;
                f.left[T] = there ? key_end - (t * TILE + 16 * (NT * hh + T)) : 0;
                if (f.left[T] <= 0) f.c[T] = f.vs[T] = 1.0f;
            }
        }
#pragma unroll
        for (int T = 0; T < NT; ++T) {
            const float x = as_float((__builtin_bit_cast(unsigned, (float)f.vs[T]) & 0x7fffffu) | 0x3f800000u);
            f.shift[T] = FP8 ? __builtin_amdgcn_logf(x) : 0.0f;
            f.part[T] = FP8 ? __builtin_amdgcn_rcpf(x) : 1.0f;
        }
        return f;
    };
    auto mask = [&](floatx16 &s, int left) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = i < left ? s[i] : -__builtin_inff();
    };
    auto mask_v = [&](u32x4 (*vraw)[2], int first, int last, const Factors &f) __attribute__((always_inline)) {
        // what lies behind may be no number, and 0 times it would be none
#pragma unroll
        for (int i = first; i <= last; ++i)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                constexpr int PER = 4 / EB;
                const int n = (FP8 ? f.left[i % NT] : f.left[0] - 8 * i) - x * PER;
                const unsigned keep = n >= PER ? ~0u : n <= 0 ? 0u : (1u << (n * 8 * EB)) - 1;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) vraw[dt][i][x] &= keep;
            }
    };
    // ---- weights 2^(s c - m) of 32 keys.  The reference only has to be near the running maximum: the first keys set it to their maximum
    // + 7; later ones take their weights with the one in use, and only if some weight reached 2 - one bit of its bf16 pattern - the
    // reference is raised and they are taken again: of the rows that are over alone, a row's result is its own, whatever the others are.
    struct Weights { u32x4 w[2]; };
    auto weigh = [&](Weights &w, const floatx16 &s, int e, float c, float at) __attribute__((always_inline)) {     // two of them
        const unsigned x = pack_bf16(__builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * e], c, at)), __builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * e + 1], c, at)));
        w.w[e / 4][e % 4] = x;
        return x;
    };
    auto raise = [&](Weights &w, const floatx16 &s, float c, float shift, unsigned over) __attribute__((always_inline)) {
        if (!__any((over & 0x40004000u) != 0)) return;
        float top = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
        const float to = halves_max((over & 0x40004000u) != 0 ? 1.0f : 0.0f) > 0 ? fmaxf(halves_max(top * c) + kMargin, m) : m, by = __builtin_amdgcn_exp2f(m - to);
        m = to;
        l *= by;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[dt][i] *= by;
#pragma unroll
        for (int e = 0; e < 8; ++e) weigh(w, s, e, c, shift - m);
    };
    // their sum as they are multiplied, by the matrix instruction of sixteen 4 x 4 blocks: with ones as its A every lane gets the sum of
    // its own; four at a time
    auto sum4 = [&](floatx4 sum, const Weights &w, int j) __attribute__((always_inline)) {
        const u32x2 four = {w.w[j / 2][j % 2 * 2], w.w[j / 2][j % 2 * 2 + 1]};
        return __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(short4v{0x3F80, 0x3F80, 0x3F80, 0x3F80}, __builtin_bit_cast(short4v, four), sum, 0, 0, 0);
    };

    Pages third{};
    Scales sc = load_scales(now), sc_next = load_scales(next);
    if (rounds > 0) {
        load_k(now, mine, k_lds);
        load_v(now, mine, v_lds);
        if (RG > 1 && rounds > 1) load_k(next, mine + STREAMS, k_lds + KB);
    }
    // (the compiler's wait for the queries: here, as in the loop it would wait for every load on its way, every time)
#pragma unroll
    for (int k = 0; k < KS; ++k) asm volatile("" ::"v"(q[k]));
    if constexpr (RG > 1) {
        wait_loads<0>();
        asm volatile("s_barrier" ::: "memory");
    }
    floatx16 s[NT];
    if (rounds > 0) {
        if constexpr (RG == 1) wait_loads<NV>();
        u32x4 kraw[NT][KR];
#pragma unroll
        for (int T = 0; T < NT; ++T) read_k(kraw[T], T, 0);
        if constexpr (RG == 1) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (rounds > 1) load_k(next, mine + STREAMS, k_lds);
        }
#pragma unroll
        for (int T = 0; T < NT; ++T) s[T] = zeros();
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int T = 0; T < NT; ++T) s[T] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fragment<FP8>(kraw[T], k, 1.0f), q[k], s[T], 0, 0, 0);
    }
    if constexpr (NT == 1) {
        // ---- tile by tile: the scores of the next one on the matrix cores beside this one's weights, then its output.  MORE: there is a next.
        auto round = [&](auto more_tag, int it, bool more2) __attribute__((always_inline)) {
            constexpr bool MORE = decltype(more_tag)::value;
            const int t = mine + it * STREAMS;
            if constexpr (RG > 1) {
                wait_loads<0>();
                asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");         // what was asked for is there for all, and all have read the other buffers
                if (more2) load_k(after, t + 2 * STREAMS, k_lds + (it & 1) * KB);
                if constexpr (MORE) load_v(next, t + STREAMS, v_lds + (~it & 1) * VB);
            }
            third = pages_of(t + 3 * STREAMS);           // (scalar loads are unconditional: a branch would wait for them at its end)
            const Factors f = factors_of(now, sc, t);
            sc = sc_next;
            sc_next = load_scales(after);
            if (!f.whole) mask(s[0], f.left[0]);
            u32x4 kraw[KR];
            floatx16 s_next = zeros();
            if constexpr (MORE) {
                if constexpr (RG == 1) {
                    if (it == 0) wait_loads<0>();        // (this tile's V was asked for before the next one's K)
                    else wait_loads<NV>();
                }
                read_k(kraw, 0, it + 1);
                if constexpr (RG == 1) {
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                    if (more2) load_k(after, t + 2 * STREAMS, k_lds);
                }
            }
            Weights w;
            unsigned over = 0;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                if constexpr (MORE) s_next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fragment<FP8>(kraw, k, 1.0f), q[k], s_next, 0, 0, 0);
#pragma unroll
                for (int e = k * 8 / KS; e < (k + 1) * 8 / KS; ++e) over |= weigh(w, s[0], e, f.c[0], f.shift[0] - m);
                __builtin_amdgcn_sched_barrier(0);       // (left to itself the compiler puts one after the other)
            }
            raise(w, s[0], f.c[0], f.shift[0], over);
            floatx4 sum = {0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < 4; ++j) sum = sum4(sum, w, j);
            l = __builtin_fmaf(sum[0], f.part[0], l);
            if constexpr (RG == 1) {
                if (MORE && more2) wait_loads<NK>();
                else wait_loads<0>();
            }
            u32x4 vraw[DT][2];
            read_v(vraw, 0, 1, it);
            if constexpr (RG == 1) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                if constexpr (MORE) load_v(next, t + STREAMS, v_lds);
            }
            if (!f.whole) mask_v(vraw, 0, 1, f);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
                    o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fragment<FP8>(vraw[dt], j, 1.0f), __builtin_bit_cast(bf16x8, w.w[j]), o[dt], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
            s[0] = s_next;
            now = next;
            next = after;
            after = third;
        };
        for (int it = 0; it + 1 < rounds; ++it) round(std::true_type{}, it, it + 2 < rounds);
        if (rounds > 0) round(std::false_type{}, rounds - 1, false);
    } else {
        // ---- half a tile, 32 keys, at a time, in three stages at once: the output of keys u, the weights of keys u + 32, the scores of keys
        // u + 64.  A matrix instruction, the decoding of the next one's operand and a share of the weights take turns, so that neither the
        // matrix cores nor the vector units wait for the other.  MORE, MORE2: one tile, two follow
        // (MORE2 for shared tiles, others go by more2).
        Factors f = factors_of(now, sc, mine);
        Weights w;
        unsigned over = 0;
        if (rounds > 0) {
            if (!f.whole) mask(s[0], f.left[0]);
#pragma unroll
            for (int e = 0; e < 8; ++e) over |= weigh(w, s[0], e, f.c[0], f.shift[0] - m);
            raise(w, s[0], f.c[0], f.shift[0], over);
        }
        auto round = [&](auto tag, int it, bool more2) __attribute__((always_inline)) {
            constexpr bool MORE = decltype(tag)::value > 0, MORE2 = decltype(tag)::value > 1;
            const int t = mine + it * STREAMS;
            wait_loads<0>();
            if constexpr (RG > 1) {
                asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");         // what was asked for is there for all, and all have read the other buffers
            }
            u32x4 kraw[NT][KR], vraw[DT][2];
            constexpr int READ = RG == 1 ? 1 : 0;        // the halves that are read now: a wave's own tile is to be free for the next one
            read_v(vraw, 0, READ, it);
            if constexpr (MORE) {
#pragma unroll
                for (int T = 0; T <= READ; ++T) read_k(kraw[T], T, it + 1);
            }
            if constexpr (RG == 1) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                if (more2) load_k(after, t + 2 * STREAMS, k_lds);
                if constexpr (MORE) load_v(next, t + STREAMS, v_lds);
            }
            // Shared tiles are asked for one load at a time, beside the arithmetic: a wave waits where it asks faster than they are taken (16 x 64
            // rows as above, 8192 keys 156.6 -> 151.9 us; bf16 pages, which wait for memory, take 29.2 at once and 31.0 one by one).
            KFrom kf;
            const uint8_t *vf;
            if constexpr (RG > 1 && MORE2) kf = k_from(after, t + 2 * STREAMS);
            if constexpr (RG > 1 && MORE) vf = v_from(next, t + STREAMS);
            auto ask = [&](int i) __attribute__((always_inline)) {
                if constexpr (RG > 1 && MORE) {
                    if (i < NV / RG) put_v(vf, v_lds + (~it & 1) * VB, i);
                }
                if constexpr (RG > 1 && MORE2) {
                    if (i >= NV / RG && i < NV / RG + NK / RG) put_k(kf, k_lds + (it & 1) * KB, i - NV / RG);
                }
            };
            third = pages_of(t + 3 * STREAMS);           // (scalar loads are unconditional: a branch would wait for them at its end)
            const Factors fn = factors_of(next, sc_next, t + STREAMS);
            sc_next = load_scales(after);
            if (!f.whole) {
                mask_v(vraw, 0, READ, f);
                mask(s[1], f.left[1]);
            }
            auto step = [&](auto t_tag, auto s_tag, auto w_tag, const Factors &fw, floatx16 &from, floatx16 &to) __attribute__((always_inline)) {
                constexpr int T = decltype(t_tag)::value;
                constexpr bool SCORES = decltype(s_tag)::value, WEIGHTS = decltype(w_tag)::value;
                constexpr int TW = 1 - T;                // the half that is weighed
                Weights wn;
                unsigned over = 0;
                floatx4 sum = {0, 0, 0, 0};
                floatx16 acc = zeros();
                const float c = fw.c[TW], at = fw.shift[TW] - m;
                constexpr int SLOTS = 2 * DT;            // output instructions; KS of scores beside them
                bf16x8 fk, fv = fragment<FP8>(vraw[0], 2 * T, f.vs[T]);
                if constexpr (SCORES) fk = fragment<FP8>(kraw[T], 0, 1.0f);
#pragma unroll
                for (int i = 0; i < SLOTS; ++i) {
                    const int dt = i % DT, j = i / DT;
                    if constexpr (SCORES) {
                        if (i < KS) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fk, q[i % KS], acc, 0, 0, 0);
                        if (i + 1 < KS) fk = fragment<FP8>(kraw[T], (i + 1) % KS, 1.0f);
                    }
                    if constexpr (WEIGHTS) {
                        if (i < 8) over |= weigh(wn, from, i % 8, c, at);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                    o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fv, __builtin_bit_cast(bf16x8, w.w[j]), o[dt], 0, 0, 0);
                    if (i + 1 < SLOTS) fv = fragment<FP8>(vraw[(i + 1) % DT], 2 * T + (i + 1) / DT, f.vs[T]);
                    if constexpr (T == 0) {
#pragma unroll
                        for (int e = i * 8 / SLOTS; e < (i + 1) * 8 / SLOTS; ++e) ask(e);
                    }
                    if (i < 4) sum = sum4(sum, w, i);
                    if constexpr (WEIGHTS && SLOTS < 8) over |= weigh(wn, from, (SLOTS + i) % 8, c, at);
                    __builtin_amdgcn_sched_barrier(0);
                }
                l = __builtin_fmaf(sum[0], f.part[T], l);
                if constexpr (WEIGHTS) {
                    raise(wn, from, c, fw.shift[TW], over);
                    w = wn;
                }
                if constexpr (SCORES) to = acc;
            };
            step(std::integral_constant<int, 0>{}, std::integral_constant<bool, MORE>{}, std::true_type{}, f, s[1], s[0]);
            if constexpr (READ == 0) {
                read_v(vraw, 1, 1, it);
                if constexpr (MORE) read_k(kraw[1], 1, it + 1);
                if (!f.whole) mask_v(vraw, 1, 1, f);
            }
            if constexpr (MORE) {
                if (!fn.whole) mask(s[0], fn.left[0]);
            }
            step(std::integral_constant<int, 1>{}, std::integral_constant<bool, MORE>{}, std::integral_constant<bool, MORE>{}, fn, s[0], s[1]);
            f = fn;
            now = next;
            next = after;
            after = third;
        };
        if constexpr (RG == 1) {
            for (int it = 0; it + 1 < rounds; ++it) round(std::integral_constant<int, 1>{}, it, it + 2 < rounds);
        } else {
            for (int it = 0; it + 2 < rounds; ++it) round(std::integral_constant<int, 2>{}, it, true);
            if (rounds > 1) round(std::integral_constant<int, 1>{}, rounds - 2, false);
        }
        if (rounds > 0) round(std::integral_constant<int, 0>{}, rounds - 1, false);
    }
    l += halves_other(l);

    if constexpr (STREAMS == 1) {                    // a row is in one wave, four head dims of it at a time (and its keys are not split)
        if (v_first + l32 >= rows_total) return;
        const size_t row = row_base + v_first + l32;
        const float inv = l > 0 ? 1.0f / l : 0.0f;   // no key at all: zeros
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int d0 = dt * 32 + 8 * i + 4 * hh;
                const float x0 = o[dt][4 * i] * inv, x1 = o[dt][4 * i + 1] * inv, x2 = o[dt][4 * i + 2] * inv, x3 = o[dt][4 * i + 3] * inv;
                *reinterpret_cast<uint2 *>(a.O + (row * D + d0) * 2) = make_uint2(pack_bf16(x0, x1), pack_bf16(x2, x3));
            }
    } else {
        // ---- the streams' states, merged: every thread finishes eight head dims of a row at a time
        float (*const o_sh)[32][PITCH] = reinterpret_cast<float (*)[32][PITCH]>(lds);
        __shared__ float ml_sh[kWaves][2][32];
        __syncthreads();                             // the tiles have been read
        if (hh == 0) {
            ml_sh[wave][0][l32] = m;
            ml_sh[wave][1][l32] = l;
        }
        if (v_first + l32 < rows_total)
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
            if (v >= rows_total) break;
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
                float *to = a.part_o + (row * splits + sp) * D + d0;
                *reinterpret_cast<float4 *>(to) = make_float4(x[0], x[1], x[2], x[3]);
                *reinterpret_cast<float4 *>(to + 4) = make_float4(x[4], x[5], x[6], x[7]);
                if (d0 == 0) {
                    a.part_ml[(row * splits + sp) * 2] = M;
                    a.part_ml[(row * splits + sp) * 2 + 1] = L;
                }
            }
        }
    }
#endif
}

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
    return p.rg == 1 ? run(attn_paged_kernel<D, FP8, NT, ONE, 1>) : p.rg == 2 ? run(attn_paged_kernel<D, FP8, NT, ONE, 2>) : run(attn_paged_kernel<D, FP8, NT, ONE, 4>);
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
