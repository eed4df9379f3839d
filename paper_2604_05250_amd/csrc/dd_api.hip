// C ABI of the library: argument validation (host only, before any GPU call) and dispatch
// to the kernels.  See include/dd.h for the contract of every entry point.
#include "../../include/dd.h"
#include "dd_internal.h"

#include <cstdlib>
#include <mutex>

namespace {

// Scratch memory of dd_verify_remask_static: one copy per GPU, at its own address on each, held from the moment
// the library's code is loaded on that GPU until the process ends.  The name below is a host-side handle only;
// the device address is looked up once per device (scratch_of_current_device) and is what the kernels get.
constexpr size_t kStaticScratchBytes = 128u * 1024u;
static __device__ __align__(256) unsigned char scratch[kStaticScratchBytes];
constexpr int kMaxDevices = 64;
void *g_scratch_ptr[kMaxDevices];            // device address of `scratch` on device i, or nullptr: not looked up yet
std::mutex g_scratch_mutex;

int scratch_of_current_device(void **out)
{
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return DD_ERR_LAUNCH;
    std::lock_guard<std::mutex> lock(g_scratch_mutex);
    if (g_scratch_ptr[dev] == nullptr) {
        void *p = nullptr;
        if (hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)) != hipSuccess || p == nullptr) return DD_ERR_LAUNCH;
        g_scratch_ptr[dev] = p;
    }
    *out = g_scratch_ptr[dev];
    return DD_OK;
}

inline bool misaligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

int check_attention_common(int B, int H, int Hkv, int N, int d, dd_dtype qk_dtype, dd_dtype v_dtype,
                           const float *q_scale, const float *k_scale, const float *v_scale = nullptr)
{
    if (B < 1 || H < 1 || Hkv < 1 || N < 1) return DD_ERR_SHAPE;
    if (H % Hkv != 0) return DD_ERR_SHAPE;
    if (d != 64 && d != 128) return DD_ERR_SHAPE;
    if ((double)B * H * N * d >= 1099511627776.0) return DD_ERR_SHAPE;
    // (fp8 V - with fp8 Q/K - only through the entry points that carry its scale)
    const bool ok = (qk_dtype == DD_F32 && v_dtype == DD_F32) || (qk_dtype == DD_BF16 && v_dtype == DD_BF16) ||
                    (qk_dtype == DD_FP8_E4M3 && v_dtype == DD_BF16) ||
                    (qk_dtype == DD_FP8_E4M3 && v_dtype == DD_FP8_E4M3 && v_scale != nullptr);
    if (!ok) return DD_ERR_DTYPE;
    if (qk_dtype == DD_FP8_E4M3 && (!q_scale || !k_scale)) return DD_ERR_NULL;
    return DD_OK;
}

int check_workspace(const void *ws, size_t have, size_t need)
{
    if (need == 0) return DD_OK;
    if (!ws || have < need) return DD_ERR_WORKSPACE;
    if ((reinterpret_cast<uintptr_t>(ws) & 255u) != 0) return DD_ERR_WORKSPACE;
    return DD_OK;
}

}  // namespace

namespace dd {

int tune(const char *name, int dflt)
{
    static const bool hooks = [] { const char *e = getenv("DD_TUNE"); return e && e[0] == '1'; }();
    if (!hooks) return dflt;
    const char *e = getenv(name);
    return e && *e ? atoi(e) : dflt;
}

// Query rows per workgroup of the drafter's MFMA kernel.  Smaller row tiles (64, 32: more workgroups that
// stream the same K/V side by side) were measured and lose on every benchmark shape.
int attn_block_rows_per_wg(int block_len, int B, int H, int Hkv)
{
    (void)block_len; (void)B; (void)H; (void)Hkv;
    return 128;
}

int attn_block_splits(int block_len, int B, int H, int Hkv, int N, int d, int qk_dtype)
{
    const int group = H / Hkv;
    const int r = attn_block_rows_per_wg(block_len, B, H, Hkv);
    const long base = (long)B * Hkv * ((group * block_len + r - 1) / r);
    // Every extra split adds partial-state traffic and merge work, so the key range is only split until
    // there is about one workgroup per compute unit.
    const int target = 256;
    long s = (target + base - 1) / base;
    // The streaming kernel's bf16 form at d = 128 fills a compute unit's LDS, so there workgroup 257 is a second round of
    // them all: one split less where the last one would cross that line.  us per call: 88 row tiles, 1237 keys 28.2 -> 20.1 (3
    // splits -> 2), 96 row tiles, 1000 keys 23.4 -> 16.6, 104, 600 keys 18.3 -> 14.1, 20, 2048 keys 15.5 -> 14.2 (13 -> 12).  The
    // other forms fit two workgroups on a compute unit.
    if (qk_dtype == DD_BF16 && d == 128 && (long)group * block_len <= 64 && base <= target) s = target / base;
    const long forced = tune("DD_TUNE_BLOCK_SPLITS", 0);
    if (forced >= 1) s = forced;
    const long max_s = N / 128 > 1 ? N / 128 : 1;   // at least 128 keys per split
    if (s > max_s) s = max_s;
    if (s > 16) s = 16;
    if (s < 1) s = 1;
    return (int)s;
}

size_t attn_partial_bytes(int B, int H, int Nq, int d, int splits)
{
    if (splits <= 1) return 0;
    return (size_t)B * H * Nq * (size_t)splits * (size_t)(d + 2) * sizeof(float);
}

}  // namespace dd

extern "C" {

const char *dd_strerror(int status)
{
    switch (status) {
    case DD_OK: return "ok";
    case DD_ERR_NULL: return "a required pointer is NULL";
    case DD_ERR_SHAPE: return "a size is out of range or inconsistent";
    case DD_ERR_DTYPE: return "unsupported element type or combination";
    case DD_ERR_MODE: return "unknown remask mode";
    case DD_ERR_WORKSPACE: return "workspace is NULL, too small or not 256-byte aligned";
    case DD_ERR_ALIGN: return "a pointer or row pitch is not 16-byte aligned";
    case DD_ERR_LAUNCH: return "the HIP runtime refused a kernel launch";
    default: return "unknown status";
    }
}

int dd_version(void) { return 100; }

size_t dd_bidir_attention_workspace_bytes(int, int, int, int, int, dd_dtype, dd_dtype) { return 0; }

int dd_bidir_attention(const void *Q, const void *K, const void *V, void *O,
                       int B, int H, int Hkv, int N, int d, dd_dtype qk_dtype, dd_dtype v_dtype,
                       const float *q_scale, const float *k_scale,
                       void *workspace, size_t workspace_bytes, void *stream)
{
    (void)workspace; (void)workspace_bytes;
    if (!Q || !K || !V || !O) return DD_ERR_NULL;
    const int rc = check_attention_common(B, H, Hkv, N, d, qk_dtype, v_dtype, q_scale, k_scale);
    if (rc != DD_OK) return rc;
    if (misaligned16(Q) || misaligned16(K) || misaligned16(V) || misaligned16(O)) return DD_ERR_ALIGN;
    dd::AttnArgs a{};
    a.Q = Q; a.K = K; a.V = V; a.Kblk = nullptr; a.Vblk = nullptr; a.O = O;
    a.q_scale = q_scale; a.k_scale = k_scale;
    a.B = B; a.H = H; a.Hkv = Hkv; a.Nq = N; a.N = N; a.d = d;
    a.block_start = 0; a.block_len = 0;
    a.qk_dtype = qk_dtype; a.v_dtype = v_dtype;
    a.splits = 1; a.workspace = nullptr;
    const hipError_t e = (qk_dtype == DD_F32) ? dd::launch_attention_f32(a, static_cast<hipStream_t>(stream))
                                              : dd::launch_attention_mfma(a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? DD_OK : DD_ERR_LAUNCH;
}

size_t dd_block_attention_cached_workspace_bytes(int block_len, int B, int H, int Hkv, int N, int d,
                                                 dd_dtype qk_dtype, dd_dtype v_dtype)
{
    if (check_attention_common(B, H, Hkv, N, d, qk_dtype, v_dtype, (const float *)16, (const float *)16) != DD_OK) return 0;
    if (block_len < 1 || block_len > N) return 0;
    // which kernel serves the call also depends on block_start: enough for either plan
    const size_t narrow = dd::attn_partial_bytes(B, H, block_len, d, dd::attn_block_splits(block_len, B, H, Hkv, N, d, qk_dtype));
    const size_t wide = dd::attn_partial_bytes(B, H, block_len, d, dd::attn_wide_block_splits(block_len, B, H, Hkv, N));
    const size_t duo = dd::attn_partial_bytes(B, H, block_len, d, dd::attn_duo_plan((long)(H / Hkv) * block_len, (long)B * Hkv, N, qk_dtype == DD_FP8_E4M3 || d == 64).splits);
    const size_t most = narrow > wide ? narrow : wide;
    return duo > most ? duo : most;
}

}  // extern "C"

// test hooks: a drafter call is sent to one of the kernels it may run on besides attention_duo.hip's and attention_solo.hip's
static bool other_kernel_forced()
{
    return dd::tune("DD_TUNE_BLOCK_WIDE", -1) >= 0 || dd::tune("DD_TUNE_BLOCK_STREAM", -1) >= 0 || dd::tune("DD_TUNE_BLOCK_WIDE_ROWS", 0) > 0 ||
           dd::tune("DD_TUNE_BLOCK_WIDE_MIN_ROWS", 0) > 0 || dd::tune("DD_TUNE_STREAM_NT", -1) >= 0;
}

// the drafter's call, with (refresh) or without the block's rows written back into the cache, over the
// whole cache (win_len == 0) or over the key rows [win_start, win_start + win_len) only
static int block_attention(const void *Qblk, const void *Kc, const void *Vc, void *O,
                           int block_start, int block_len, const void *Kblk, const void *Vblk,
                           int B, int H, int Hkv, int N, int d, dd_dtype qk_dtype, dd_dtype v_dtype,
                           const float *q_scale, const float *k_scale,
                           void *workspace, size_t workspace_bytes, void *stream, bool refresh,
                           int win_start = 0, int win_len = 0, const int32_t *block_starts = nullptr,
                           const float *v_scale = nullptr)
{
    if (!Qblk || !Kc || !Vc || !O) return DD_ERR_NULL;
    if ((Kblk == nullptr) != (Vblk == nullptr)) return DD_ERR_NULL;
    if (refresh && !Kblk) return DD_ERR_NULL;
    if (refresh && block_len > (1 << 25)) return DD_ERR_SHAPE;   // the copy indexes a block's 16-byte chunks with 32 bits
    int rc = check_attention_common(B, H, Hkv, N, d, qk_dtype, v_dtype, q_scale, k_scale, v_scale);
    if (rc != DD_OK) return rc;
    if (block_start < 0 || block_len < 1 || (long)block_start + block_len > N) return DD_ERR_SHAPE;
    const int full_N = N;
    if (win_len != 0) {
        // a window is a shorter sequence that starts win_start rows into every (batch, kv head) of the cache:
        // same kernels, K/V based at the window's first row, the cache's own row count as the stride
        if (win_start < 0 || win_len < 1 || (long)win_start + win_len > N) return DD_ERR_SHAPE;
        if (block_start < win_start || (long)block_start + block_len > (long)win_start + win_len) return DD_ERR_SHAPE;
        const size_t ebk = qk_dtype == DD_F32 ? 4 : qk_dtype == DD_BF16 ? 2 : 1;
        const size_t ebv = v_dtype == DD_F32 ? 4 : v_dtype == DD_BF16 ? 2 : 1;
        Kc = static_cast<const uint8_t *>(Kc) + (size_t)win_start * d * ebk;
        Vc = static_cast<const uint8_t *>(Vc) + (size_t)win_start * d * ebv;
        block_start -= win_start;
        N = win_len;
    }
    if (misaligned16(Qblk) || misaligned16(Kc) || misaligned16(Vc) || misaligned16(O) ||
        misaligned16(Kblk) || misaligned16(Vblk))
        return DD_ERR_ALIGN;
    dd::AttnArgs a{};
    a.Q = Qblk; a.K = Kc; a.V = Vc; a.Kblk = Kblk; a.Vblk = Vblk; a.O = O;
    a.q_scale = q_scale; a.k_scale = k_scale; a.v_scale = v_scale;
    a.B = B; a.H = H; a.Hkv = Hkv; a.Nq = block_len; a.N = N; a.d = d;
    a.block_start = block_start; a.block_len = block_len;
    a.qk_dtype = qk_dtype; a.v_dtype = v_dtype;
    a.workspace = workspace;
    a.kv_stride = full_N;
    a.block_starts = block_starts;
    if (refresh) {
        a.K_refresh = const_cast<void *>(Kc);
        a.V_refresh = const_cast<void *>(Vc);
    }
    const bool wide = dd::tune("DD_TUNE_BLOCK_WIDE", 1) != 0 && dd::attn_wide_block_fits(a);
    const long rows = (long)(H / Hkv) * block_len, heads = (long)B * Hkv;
    const int narrow_splits = dd::attn_block_splits(block_len, B, H, Hkv, N, d, qk_dtype);
    const int wide_rows = dd::attn_wide_block_rows(block_len, B, H, Hkv, N);
    const long wide_wgs = wide ? heads * ((rows + wide_rows - 1) / wide_rows) * dd::attn_wide_block_splits(block_len, B, H, Hkv, N) : 0;
    dd::SoloPlan solo{false, 0, 1};
    if (dd::attn_solo_serves(a) && dd::tune("DD_TUNE_DUO", -1) <= 0 && !other_kernel_forced())
        solo = dd::attn_solo_plan(rows, heads, N, d, qk_dtype == DD_FP8_E4M3, v_dtype == DD_FP8_E4M3, refresh, Kblk ? block_len : 0, wide_wgs, wide_rows,
                                  narrow_splits);
    dd::DuoPlan duo{0, 1};
    if (!solo.take && dd::attn_duo_serves(a) && (rows > 64 || dd::tune("DD_TUNE_DUO", 0) > 0) && !other_kernel_forced()) {
        duo = dd::attn_duo_plan(rows, heads, N, qk_dtype == DD_FP8_E4M3 || d == 64);
        // Where the wide kernel cannot take the call (block rows spliced in from a block shorter than a tile), the MFMA kernel's 128-row
        // workgroups, two to a compute unit, are faster on few keys: than 128-row ones here below 256 keys, where it splits (bf16 176 heads, 80 rows, 178
        // keys 11.0 against 12.1, 192 x 96 rows, 123 keys 10.1 / 11.1; d = 64 144 x 110, 94 keys 6.2 / 6.9), than 64-row ones up to 64 keys
        // (bf16 112 x 80, 40 keys 6.4 / 7.2) and, with 64 head dims, 128 (96 x 96, 89 keys 5.7 / 6.4; 128 x 128, 81 keys 6.1 / 6.5).
        if (!wide && N <= (duo.blocks == 4 ? 255 : d == 64 ? 128 : 64) && dd::tune("DD_TUNE_DUO", -1) < 0) duo.blocks = 0;
        // Past one round of 128-row workgroups the wide kernel's 256-row tiles are faster (24 x 32/8 heads, 64 rows, 1024 keys
        // 43.3 against 48.5 us, fp8 36.3 / 42.5), its 128-row tiles, for up to 128 rows, are not (40 x 16/8: 60.9 / 52.6, fp8
        // 51.7 / 45.0); the MFMA kernel, where the wide one cannot take the call, is (64 x 32/8, 32 rows: 62.8 / 66.8).
        if (duo.blocks == 0 && wide && rows <= 128 && dd::tune("DD_TUNE_DUO", -1) != 0) duo.blocks = 4;
    }
    // Long bf16 streams that the splits here leave a fifth of the compute units without: the wide kernel's larger tiles split finer (48 heads x 192
    // rows, 3709 keys: 39.2 on 240 workgroups against 43.3 on 192; 24 x 512, 3857 keys 43.1 / 46.3; at 2600 keys still 0.96).
    if (duo.splits > 1 && wide && qk_dtype == DD_BF16 && d == 128 && N >= 3072 && dd::tune("DD_TUNE_DUO", -1) < 0) {
        const long here = heads * ((rows + 32 * duo.blocks - 1) / (32 * duo.blocks)) * duo.splits;
        if (5 * here <= 4 * wide_wgs) duo.blocks = 0;
    }
    const int general = wide ? dd::attn_wide_block_splits(block_len, B, H, Hkv, N) : narrow_splits;
    const int splits = duo.blocks ? duo.splits : solo.take ? solo.splits : general;
    // (what the kernels of every shape ask for is asked for here too, whichever serves the call)
    rc = check_workspace(workspace, workspace_bytes, dd::attn_partial_bytes(B, H, block_len, d, splits > general ? splits : general));
    if (rc != DD_OK) return rc;
    a.splits = splits;
    if (duo.blocks)
        return dd::launch_attention_duo(a, duo.blocks, static_cast<hipStream_t>(stream)) == hipSuccess ? DD_OK : DD_ERR_LAUNCH;
    if (solo.take)
        return dd::launch_attention_solo(a, solo.form, static_cast<hipStream_t>(stream)) == hipSuccess ? DD_OK : DD_ERR_LAUNCH;
    if (wide)
        return dd::launch_attention_wide_block(a, static_cast<hipStream_t>(stream)) == hipSuccess ? DD_OK : DD_ERR_LAUNCH;
    const hipError_t e = (qk_dtype == DD_F32) ? dd::launch_attention_f32(a, static_cast<hipStream_t>(stream))
                                              : dd::launch_attention_mfma(a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? DD_OK : DD_ERR_LAUNCH;
}

extern "C" {

int dd_block_attention_cached(const void *Qblk, const void *Kc, const void *Vc, void *O,
                              int block_start, int block_len, const void *Kblk, const void *Vblk,
                              int B, int H, int Hkv, int N, int d, dd_dtype qk_dtype, dd_dtype v_dtype,
                              const float *q_scale, const float *k_scale,
                              void *workspace, size_t workspace_bytes, void *stream)
{
    return block_attention(Qblk, Kc, Vc, O, block_start, block_len, Kblk, Vblk, B, H, Hkv, N, d, qk_dtype, v_dtype,
                           q_scale, k_scale, workspace, workspace_bytes, stream, false);
}

int dd_bidir_attention_fp8v(const void *Q, const void *K, const void *V, void *O,
                            int B, int H, int Hkv, int N, int d,
                            const float *q_scale, const float *k_scale, const float *v_scale, void *stream)
{
    if (!Q || !K || !V || !O || !v_scale) return DD_ERR_NULL;
    const int rc = check_attention_common(B, H, Hkv, N, d, DD_FP8_E4M3, DD_FP8_E4M3, q_scale, k_scale, v_scale);
    if (rc != DD_OK) return rc;
    if (misaligned16(Q) || misaligned16(K) || misaligned16(V) || misaligned16(O)) return DD_ERR_ALIGN;
    dd::AttnArgs a{};
    a.Q = Q; a.K = K; a.V = V; a.Kblk = nullptr; a.Vblk = nullptr; a.O = O;
    a.q_scale = q_scale; a.k_scale = k_scale; a.v_scale = v_scale;
    a.B = B; a.H = H; a.Hkv = Hkv; a.Nq = N; a.N = N; a.d = d;
    a.block_start = 0; a.block_len = 0;
    a.qk_dtype = DD_FP8_E4M3; a.v_dtype = DD_FP8_E4M3;
    a.splits = 1; a.workspace = nullptr;
    return dd::launch_attention_mfma(a, static_cast<hipStream_t>(stream)) == hipSuccess ? DD_OK : DD_ERR_LAUNCH;
}

int dd_bidir_attention_mx(const void *Q, const void *Qs, const void *K, const void *Ks, const void *V, const void *Vs,
                          void *O, int B, int H, int Hkv, int N, int d, void *stream)
{
    if (!Q || !Qs || !K || !Ks || !V || !Vs || !O) return DD_ERR_NULL;
    const float one = 1.0f;                    // (the per-head scales of the plain fp8 form are not part of this one)
    const int rc = check_attention_common(B, H, Hkv, N, d, DD_FP8_E4M3, DD_BF16, &one, &one);
    if (rc != DD_OK) return rc;
    if (misaligned16(Q) || misaligned16(K) || misaligned16(V) || misaligned16(O)) return DD_ERR_ALIGN;
    // (a row's scale bytes are read as one word)
    if (((reinterpret_cast<uintptr_t>(Qs) | reinterpret_cast<uintptr_t>(Ks) | reinterpret_cast<uintptr_t>(Vs)) & 3u) != 0) return DD_ERR_ALIGN;
    dd::AttnArgs a{};
    a.Q = Q; a.K = K; a.V = V; a.Kblk = nullptr; a.Vblk = nullptr; a.O = O;
    a.q_scale = nullptr; a.k_scale = nullptr;
    a.q_mx = static_cast<const uint8_t *>(Qs); a.k_mx = static_cast<const uint8_t *>(Ks); a.v_mx = static_cast<const uint8_t *>(Vs);
    a.B = B; a.H = H; a.Hkv = Hkv; a.Nq = N; a.N = N; a.d = d;
    a.block_start = 0; a.block_len = 0;
    a.qk_dtype = DD_FP8_E4M3; a.v_dtype = DD_BF16;     // (storage of V: packed e2m1; its decoded form is bf16)
    a.splits = 1; a.workspace = nullptr;
    return dd::launch_attention_mfma(a, static_cast<hipStream_t>(stream)) == hipSuccess ? DD_OK : DD_ERR_LAUNCH;
}

size_t dd_block_attention_cached_fp8v_workspace_bytes(int block_len, int B, int H, int Hkv, int N, int d)
{
    return dd_block_attention_cached_workspace_bytes(block_len, B, H, Hkv, N, d, DD_FP8_E4M3, DD_BF16);
}

int dd_block_attention_cached_fp8v(const void *Qblk, const void *Kc, const void *Vc, void *O,
                                   int block_start, int block_len, const void *Kblk, const void *Vblk,
                                   int B, int H, int Hkv, int N, int d,
                                   const float *q_scale, const float *k_scale, const float *v_scale,
                                   void *workspace, size_t workspace_bytes, void *stream)
{
    if (!v_scale) return DD_ERR_NULL;
    return block_attention(Qblk, Kc, Vc, O, block_start, block_len, Kblk, Vblk, B, H, Hkv, N, d, DD_FP8_E4M3,
                           DD_FP8_E4M3, q_scale, k_scale, workspace, workspace_bytes, stream, false, 0, 0, nullptr, v_scale);
}

size_t dd_block_attention_refresh_workspace_bytes(int block_len, int B, int H, int Hkv, int N, int d,
                                                  dd_dtype qk_dtype, dd_dtype v_dtype)
{
    return dd_block_attention_cached_workspace_bytes(block_len, B, H, Hkv, N, d, qk_dtype, v_dtype);
}

int dd_block_attention_refresh(const void *Qblk, void *Kc, void *Vc, void *O,
                               int block_start, int block_len, const void *Kblk, const void *Vblk,
                               int B, int H, int Hkv, int N, int d, dd_dtype qk_dtype, dd_dtype v_dtype,
                               const float *q_scale, const float *k_scale,
                               void *workspace, size_t workspace_bytes, void *stream)
{
    return block_attention(Qblk, Kc, Vc, O, block_start, block_len, Kblk, Vblk, B, H, Hkv, N, d, qk_dtype, v_dtype,
                           q_scale, k_scale, workspace, workspace_bytes, stream, true);
}

size_t dd_block_attention_batched_workspace_bytes(int block_len, int B, int H, int Hkv, int N, int d,
                                                  dd_dtype qk_dtype, dd_dtype v_dtype)
{
    return dd_block_attention_cached_workspace_bytes(block_len, B, H, Hkv, N, d, qk_dtype, v_dtype);
}

int dd_block_attention_batched(const void *Qblk, const void *Kc, const void *Vc, void *O,
                               const int32_t *block_starts, int block_len, const void *Kblk, const void *Vblk,
                               int B, int H, int Hkv, int N, int d, dd_dtype qk_dtype, dd_dtype v_dtype,
                               const float *q_scale, const float *k_scale,
                               void *workspace, size_t workspace_bytes, void *stream)
{
    if (!block_starts || !Kblk || !Vblk) return DD_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(block_starts) & 3u) != 0) return DD_ERR_ALIGN;
    return block_attention(Qblk, Kc, Vc, O, 0, block_len, Kblk, Vblk, B, H, Hkv, N, d, qk_dtype, v_dtype,
                           q_scale, k_scale, workspace, workspace_bytes, stream, false, 0, 0, block_starts);
}

size_t dd_block_attention_window_workspace_bytes(int block_len, int win_len, int B, int H, int Hkv, int N, int d,
                                                 dd_dtype qk_dtype, dd_dtype v_dtype)
{
    if (win_len < 1 || win_len > N) return 0;
    if (check_attention_common(B, H, Hkv, N, d, qk_dtype, v_dtype, (const float *)16, (const float *)16) != DD_OK) return 0;
    return dd_block_attention_cached_workspace_bytes(block_len, B, H, Hkv, win_len, d, qk_dtype, v_dtype);
}

int dd_block_attention_window(const void *Qblk, const void *Kc, const void *Vc, void *O,
                              int block_start, int block_len, int win_start, int win_len,
                              const void *Kblk, const void *Vblk,
                              int B, int H, int Hkv, int N, int d, dd_dtype qk_dtype, dd_dtype v_dtype,
                              const float *q_scale, const float *k_scale,
                              void *workspace, size_t workspace_bytes, void *stream)
{
    if (win_len < 1) return DD_ERR_SHAPE;
    return block_attention(Qblk, Kc, Vc, O, block_start, block_len, Kblk, Vblk, B, H, Hkv, N, d, qk_dtype, v_dtype,
                           q_scale, k_scale, workspace, workspace_bytes, stream, false, win_start, win_len);
}

int dd_cache_insert_rows(void *Kc, void *Vc, const void *Krows, const void *Vrows, const int32_t *positions, int n,
                         int B, int Hkv, int N, int d, dd_dtype qk_dtype, dd_dtype v_dtype, void *stream)
{
    if (n < 0) return DD_ERR_SHAPE;
    const int rc = check_attention_common(B, Hkv, Hkv, N, d, qk_dtype, v_dtype, (const float *)16, (const float *)16);
    if (rc != DD_OK) return rc;
    if ((double)B * Hkv * n * d >= 1099511627776.0) return DD_ERR_SHAPE;
    if (n == 0) return DD_OK;
    if (!Kc || !Vc || !Krows || !Vrows || !positions) return DD_ERR_NULL;
    if (misaligned16(Kc) || misaligned16(Vc) || misaligned16(Krows) || misaligned16(Vrows)) return DD_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(positions) & 3u) != 0) return DD_ERR_ALIGN;
    const int ebk = qk_dtype == DD_F32 ? 4 : qk_dtype == DD_BF16 ? 2 : 1, ebv = v_dtype == DD_F32 ? 4 : 2;
    const hipError_t e = dd::launch_cache_insert_rows(Krows, Vrows, Kc, Vc, positions, n, B, Hkv, N, d, ebk, ebv,
                                                      static_cast<hipStream_t>(stream));
    return e == hipSuccess ? DD_OK : DD_ERR_LAUNCH;
}

// strides of rows (elements): non-negative, and a multiple of 16 bytes where an axis has more than one entry
static int check_strides(const int64_t *st, const int *extent, int eb)
{
    double last = 0;
    for (int i = 0; i < 3; ++i) {
        if (extent[i] <= 1) continue;
        if (st[i] < 0) return DD_ERR_SHAPE;
        last += (double)st[i] * (extent[i] - 1);
        if (last >= 1099511627776.0) return DD_ERR_SHAPE;
        if (st[i] * eb % 16 != 0) return DD_ERR_ALIGN;
    }
    return DD_OK;
}
// bytes from the first element that rows by strides reach
static uintptr_t reach(const int64_t *st, const int *extent, int d, int eb)
{
    uintptr_t last = (uintptr_t)d;
    for (int i = 0; i < 3; ++i)
        if (extent[i] > 1) last += (uintptr_t)st[i] * (uintptr_t)(extent[i] - 1);
    return last * (uintptr_t)eb;
}
static bool overlap(const void *a, uintptr_t na, const void *b, uintptr_t nb)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + nb && y < x + na;
}
static int check_rotation(const void *weight, float eps, const float *inv_freq, int rot_dim, int d)
{
    if (rot_dim < 0 || rot_dim > d || rot_dim % 16 != 0) return DD_ERR_SHAPE;
    if (rot_dim > 0 && !inv_freq) return DD_ERR_NULL;
    if (weight && !(eps >= 1.17549435e-38f && eps <= 3.402823466e38f)) return DD_ERR_SHAPE;        // (normal: the reciprocal root takes others for 0)
    if (misaligned16(weight) || (reinterpret_cast<uintptr_t>(inv_freq) & 3u) != 0) return DD_ERR_ALIGN;
    return DD_OK;
}

int dd_qk_norm_rope(const void *Q, int64_t q_batch, int64_t q_head, int64_t q_row,
                    const void *K, int64_t k_batch, int64_t k_head, int64_t k_row,
                    const void *q_weight, const void *k_weight, float eps,
                    const float *inv_freq, int rot_dim, int interleaved, const int32_t *positions,
                    void *Qo, void *Ko, int B, int H, int Hkv, int n, int d, dd_dtype dtype, void *stream)
{
    if (dtype != DD_F32 && dtype != DD_BF16) return DD_ERR_DTYPE;
    if (n == 0 && B >= 1 && H >= 1 && Hkv >= 0 && (d == 64 || d == 128)) return DD_OK;
    if (!Q || !Qo || (K == nullptr) != (Ko == nullptr)) return DD_ERR_NULL;
    if (B < 1 || H < 1 || n < 0 || (K && Hkv < 1) || (d != 64 && d != 128)) return DD_ERR_SHAPE;
    const int kv = K ? Hkv : 0, eb = dtype == DD_BF16 ? 2 : 4;
    // (a thread has 16 elements of a token, and a launch fewer than 2^32 threads along an axis)
    if ((double)B * n >= 2147483648.0 || (double)B * n * d >= 68719476736.0 || (double)B * (H > kv ? H : kv) * n * d >= 1099511627776.0) return DD_ERR_SHAPE;
    int rc = check_rotation(q_weight ? q_weight : K ? k_weight : nullptr, eps, inv_freq, rot_dim, d);
    if (rc != DD_OK) return rc;
    const int64_t qs[3] = {q_batch, q_head, q_row}, ks[3] = {k_batch, k_head, k_row};
    const int qe[3] = {B, H, n}, ke[3] = {B, kv, n};
    if ((rc = check_strides(qs, qe, eb)) != DD_OK || (K && (rc = check_strides(ks, ke, eb)) != DD_OK)) return rc;
    if (misaligned16(Q) || misaligned16(K) || misaligned16(Qo) || misaligned16(Ko) || misaligned16(q_weight) || misaligned16(k_weight) ||
        (reinterpret_cast<uintptr_t>(positions) & 3u) != 0)
        return DD_ERR_ALIGN;
    // an output may be its own dense input (a row is read whole by the lanes that write it) and shares memory with nothing else
    const uintptr_t qb = (uintptr_t)B * H * n * d * eb, kb = (uintptr_t)B * kv * n * d * eb;
    const uintptr_t qr = reach(qs, qe, d, eb), kr = K ? reach(ks, ke, d, eb) : 0;
    auto dense = [&](const int64_t *st, int heads) {
        return (B == 1 || st[0] == (int64_t)heads * n * d) && (heads == 1 || st[1] == (int64_t)n * d) && (n == 1 || st[2] == d);
    };
    const bool q_in_place = Qo == Q && dense(qs, H), k_in_place = K && Ko == K && dense(ks, kv);
    if ((!q_in_place && overlap(Qo, qb, Q, qr)) || (K && overlap(Qo, qb, K, kr))) return DD_ERR_SHAPE;
    if (K && ((!k_in_place && overlap(Ko, kb, K, kr)) || overlap(Ko, kb, Q, qr) || overlap(Ko, kb, Qo, qb))) return DD_ERR_SHAPE;
    dd::NormRotateArgs a;
    auto side = [](dd::NormRotateSide &s, const void *x, void *y, const void *w, int heads, const int64_t *st, const int *extent) {
        s.x = x; s.y = y; s.weight = w; s.heads = heads;
        s.batch = extent[0] > 1 ? st[0] : 0; s.head = extent[1] > 1 ? st[1] : 0; s.row = extent[2] > 1 ? st[2] : 0;
    };
    side(a.q, Q, Qo, q_weight, H, qs, qe);
    if (K) side(a.k, K, Ko, k_weight, kv, ks, ke);
    a.inv_freq = inv_freq; a.positions = positions;
    a.tokens = (unsigned)((long)B * n); a.n = n; a.rot = rot_dim;
    a.interleaved = interleaved != 0;
    a.eps = eps;
    const hipError_t e = dd::launch_norm_rotate(a, d, dtype == DD_BF16, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? DD_OK : DD_ERR_LAUNCH;
}

static int page_log2_of(int page_size) { return page_size == 16 ? 4 : page_size == 32 ? 5 : page_size == 64 ? 6 : page_size == 128 ? 7 : -1; }
// what the calls on a paged cache have in common
static int check_pages(const void *Kc, const void *Vc, const float *k_scale, const float *v_scale, const int32_t *table, const int32_t *lens,
                       int n, int B, int Hkv, int d, int num_pages, int page_size, int max_pages, dd_dtype cache_dtype)
{
    if (!Kc || !Vc || !table || !lens) return DD_ERR_NULL;
    if (cache_dtype != DD_BF16 && cache_dtype != DD_FP8_E4M3) return DD_ERR_DTYPE;
    if (cache_dtype == DD_FP8_E4M3 && (!k_scale || !v_scale)) return DD_ERR_NULL;
    if (n < 0 || B < 1 || Hkv < 1 || (d != 64 && d != 128) || num_pages < 1 || max_pages < 1 || page_log2_of(page_size) < 0) return DD_ERR_SHAPE;
    if ((double)max_pages * page_size >= 1073741824.0 || (double)num_pages * Hkv * page_size * d >= 1099511627776.0) return DD_ERR_SHAPE;
    if (misaligned16(Kc) || misaligned16(Vc)) return DD_ERR_ALIGN;
    const uintptr_t words = reinterpret_cast<uintptr_t>(k_scale) | reinterpret_cast<uintptr_t>(v_scale) | reinterpret_cast<uintptr_t>(table) |
                            reinterpret_cast<uintptr_t>(lens);
    return (words & 3u) != 0 ? DD_ERR_ALIGN : DD_OK;
}

int dd_paged_cache_append(void *Kc, void *Vc, float *k_scale, float *v_scale,
                          const void *K, int64_t k_batch, int64_t k_head, int64_t k_row,
                          const void *V, int64_t v_batch, int64_t v_head, int64_t v_row,
                          const int32_t *block_table, const int32_t *starts, const int32_t *kv_lens, const int32_t *n_rows,
                          const void *k_weight, float eps, const float *inv_freq, int rot_dim, int interleaved,
                          int n, int B, int Hkv, int d, int num_pages, int page_size, int max_pages,
                          dd_dtype row_dtype, dd_dtype cache_dtype, void *stream)
{
    int rc = check_pages(Kc, Vc, k_scale, v_scale, block_table, starts, n, B, Hkv, d, num_pages, page_size, max_pages, cache_dtype);
    if (rc != DD_OK || n == 0) return rc;
    if (!K || !V) return DD_ERR_NULL;
    if (row_dtype != DD_BF16 && row_dtype != DD_F32) return DD_ERR_DTYPE;
    if ((double)B * Hkv * n * d >= 1099511627776.0) return DD_ERR_SHAPE;
    if ((rc = check_rotation(k_weight, eps, inv_freq, rot_dim, d)) != DD_OK) return rc;
    const int eb = row_dtype == DD_BF16 ? 2 : 4;
    const int64_t ks[3] = {k_batch, k_head, k_row}, vs[3] = {v_batch, v_head, v_row};
    const int extent[3] = {B, Hkv, n};
    if ((rc = check_strides(ks, extent, eb)) != DD_OK || (rc = check_strides(vs, extent, eb)) != DD_OK) return rc;
    if (misaligned16(K) || misaligned16(V) || ((reinterpret_cast<uintptr_t>(kv_lens) | reinterpret_cast<uintptr_t>(n_rows)) & 3u) != 0) return DD_ERR_ALIGN;
    const int log2 = page_log2_of(page_size);
    // (2 B pages (page_size d / 16) threads, for up to n + 2 page_size positions' pages: fewer than 2^31)
    if ((double)B * ((double)n + 2.0 * page_size) * d >= 17179869184.0) return DD_ERR_SHAPE;
    const uintptr_t cache_bytes = (uintptr_t)num_pages * Hkv * page_size * d * (cache_dtype == DD_BF16 ? 2 : 1);
    const uintptr_t k_reach = reach(ks, extent, d, eb), v_reach = reach(vs, extent, d, eb);
    if (overlap(Kc, cache_bytes, Vc, cache_bytes) || overlap(Kc, cache_bytes, K, k_reach) || overlap(Kc, cache_bytes, V, v_reach) ||
        overlap(Vc, cache_bytes, K, k_reach) || overlap(Vc, cache_bytes, V, v_reach))
        return DD_ERR_SHAPE;
    if (cache_dtype == DD_FP8_E4M3) {                        // each is read and written by one of a page's two workgroups, unordered with the other
        const uintptr_t scale_bytes = (uintptr_t)num_pages * Hkv * sizeof(float);
        if (overlap(k_scale, scale_bytes, v_scale, scale_bytes)) return DD_ERR_SHAPE;
        for (const float *scale : {k_scale, v_scale})
            if (overlap(scale, scale_bytes, Kc, cache_bytes) || overlap(scale, scale_bytes, Vc, cache_bytes) || overlap(scale, scale_bytes, K, k_reach) ||
                overlap(scale, scale_bytes, V, v_reach))
                return DD_ERR_SHAPE;
    }
    dd::PageAppendArgs a;
    auto side = [&](dd::PageAppendSide &s, const void *x, void *cache, float *scale, const int64_t *st) {
        s.x = x; s.cache = cache; s.scale = cache_dtype == DD_FP8_E4M3 ? scale : nullptr;
        s.batch = B > 1 ? st[0] : 0; s.head = Hkv > 1 ? st[1] : 0; s.row = n > 1 ? st[2] : 0;
    };
    side(a.k, K, Kc, k_scale, ks);
    side(a.v, V, Vc, v_scale, vs);
    a.table = block_table; a.starts = starts; a.kv_lens = kv_lens; a.n_rows = n_rows;
    a.weight = k_weight; a.inv_freq = inv_freq; a.eps = eps;
    a.n = n; a.B = B; a.Hkv = Hkv; a.num_pages = num_pages; a.max_pages = max_pages; a.page_log2 = log2; a.rot = rot_dim;
    a.interleaved = interleaved != 0;
    const hipError_t e = dd::launch_page_append(a, d, row_dtype == DD_BF16, cache_dtype == DD_FP8_E4M3, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? DD_OK : DD_ERR_LAUNCH;
}

// rows, and row blocks of 32 of each key/value head, that one launch of 256 threads for a row block can have
static bool attends_in_one_launch(int n, int B, int H, int Hkv)
{
    const double rows = (double)(H / Hkv) * n;
    return rows * B * Hkv < 1073741824.0 && __builtin_ceil(rows / 32) * B * Hkv < 16777216.0;
}

size_t dd_paged_attention_workspace_bytes(int n, int B, int H, int Hkv, int d, int page_size, int max_pages, dd_dtype cache_dtype)
{
    if (n < 1 || B < 1 || H < 1 || Hkv < 1 || H % Hkv != 0 || (d != 64 && d != 128) || max_pages < 1 || page_log2_of(page_size) < 0) return 0;
    if (cache_dtype != DD_BF16 && cache_dtype != DD_FP8_E4M3) return 0;
    if ((double)max_pages * page_size >= 1073741824.0 || !attends_in_one_launch(n, B, H, Hkv)) return 0;
    return dd::paged_attention_workspace_bytes(n, B, H, Hkv, d, (long)max_pages * page_size, cache_dtype == DD_FP8_E4M3);
}

int dd_paged_attention(const void *Q, const void *Kc, const void *Vc, const float *k_scale, const float *v_scale,
                       const int32_t *block_table, const int32_t *kv_lens, void *O,
                       int n, int B, int H, int Hkv, int d, int num_pages, int page_size, int max_pages,
                       dd_dtype cache_dtype, void *workspace, size_t workspace_bytes, void *stream)
{
    int rc = check_pages(Kc, Vc, k_scale, v_scale, block_table, kv_lens, n, B, Hkv, d, num_pages, page_size, max_pages, cache_dtype);
    if (rc != DD_OK) return rc;
    if (H < 1 || H % Hkv != 0) return DD_ERR_SHAPE;
    if (n == 0) return DD_OK;
    if (!Q || !O) return DD_ERR_NULL;
    if (!attends_in_one_launch(n, B, H, Hkv)) return DD_ERR_SHAPE;
    if (misaligned16(Q) || misaligned16(O)) return DD_ERR_ALIGN;
    const bool fp8 = cache_dtype == DD_FP8_E4M3;
    rc = check_workspace(workspace, workspace_bytes, dd::paged_attention_workspace_bytes(n, B, H, Hkv, d, (long)max_pages * page_size, fp8));
    if (rc != DD_OK) return rc;
    const uintptr_t rows_bytes = (uintptr_t)B * H * n * d * 2, cache_bytes = (uintptr_t)num_pages * Hkv * page_size * d * (fp8 ? 1 : 2);
    if (overlap(O, rows_bytes, Q, rows_bytes) || overlap(O, rows_bytes, Kc, cache_bytes) || overlap(O, rows_bytes, Vc, cache_bytes)) return DD_ERR_SHAPE;
    const uintptr_t scale_bytes = (uintptr_t)num_pages * Hkv * sizeof(float);
    if (fp8 && (overlap(O, rows_bytes, k_scale, scale_bytes) || overlap(O, rows_bytes, v_scale, scale_bytes))) return DD_ERR_SHAPE;
    dd::PagedAttnArgs a;
    a.Q = Q; a.Kc = Kc; a.Vc = Vc; a.O = O;
    a.k_scale = fp8 ? k_scale : nullptr; a.v_scale = fp8 ? v_scale : nullptr;
    a.table = block_table; a.kv_lens = kv_lens;
    a.n = n; a.B = B; a.H = H; a.Hkv = Hkv; a.d = d; a.num_pages = num_pages; a.max_pages = max_pages; a.page_log2 = page_log2_of(page_size);
    a.workspace = workspace;
    const hipError_t e = dd::launch_attention_paged(a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? DD_OK : DD_ERR_LAUNCH;
}

static bool resize_sizes(int n, int B, int page_size, int max_pages)
{
    if (n < 0 || B < 1 || max_pages < 1 || page_log2_of(page_size) < 0) return false;
    if ((double)max_pages * page_size >= 1073741824.0 || (double)B * max_pages >= 2147483648.0 || n >= 1073741824 || (double)B * n >= 2147483648.0) return false;
    return dd::paged_resize_workgroups(n, B, max_pages) < 16777216.0;
}

size_t dd_paged_resize_workspace_bytes(int n, int B, int page_size, int max_pages)
{
    return resize_sizes(n, B, page_size, max_pages) ? dd::paged_resize_workspace_bytes(n, B, max_pages) : 0;
}

int dd_paged_resize(int32_t *block_table, int32_t *free_pages, int32_t *num_free, const int32_t *lens, const int32_t *new_lens,
                    int32_t *out_lens, int32_t *positions, int32_t *slots,
                    int n, int B, int num_pages, int page_size, int max_pages, void *workspace, size_t workspace_bytes, void *stream)
{
    if (B == 0 && n >= 0 && num_pages >= 1 && max_pages >= 1 && page_log2_of(page_size) >= 0) return DD_OK;
    if (!resize_sizes(n, B, page_size, max_pages) || num_pages < 1 || (double)num_pages * page_size >= 2147483648.0) return DD_ERR_SHAPE;
    if (!block_table || !free_pages || !num_free || !lens || !new_lens || !out_lens || (n > 0 && (!positions || !slots))) return DD_ERR_NULL;
    struct Range { const void *at; uintptr_t bytes; };
    const uintptr_t seqs = (uintptr_t)B * 4, rows = (uintptr_t)B * n * 4;
    const Range all[8] = {{block_table, (uintptr_t)B * max_pages * 4}, {free_pages, (uintptr_t)num_pages * 4}, {num_free, 4}, {out_lens, seqs},
                          {positions, rows}, {slots, rows}, {lens, seqs}, {new_lens, seqs}};
    for (const Range &r : all)
        if ((reinterpret_cast<uintptr_t>(r.at) & 3u) != 0) return DD_ERR_ALIGN;
    const int rc = check_workspace(workspace, workspace_bytes, dd::paged_resize_workspace_bytes(n, B, max_pages));
    if (rc != DD_OK) return rc;
    for (int i = 0; i < 6; ++i)                              // (what is written, against everything)
        for (int j = i + 1; j < 8; ++j)
            if (all[i].bytes && all[j].bytes && !(i == 3 && j >= 6 && all[i].at == all[j].at) && overlap(all[i].at, all[i].bytes, all[j].at, all[j].bytes)) return DD_ERR_SHAPE;
    dd::TableArgs a;
    a.table = block_table; a.stack = free_pages; a.num_free = num_free; a.lens = lens; a.new_lens = new_lens; a.out_lens = out_lens; a.positions = positions; a.slots = slots;
    a.n = n; a.B = B; a.page_log2 = page_log2_of(page_size); a.max_pages = max_pages; a.capacity = num_pages; a.workspace = workspace;
    const hipError_t e = dd::launch_paged_resize(a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? DD_OK : DD_ERR_LAUNCH;
}

static dd::SharedAttnShape shared_shape(int n, int B, int H, int Hkv, int d, int page_size, int G, int max_prefix_pages, int max_pages, dd_dtype t)
{
    dd::SharedAttnShape s;
    s.n = n; s.B = B; s.H = H; s.Hkv = Hkv; s.d = d; s.G = G; s.max_prefix_pages = max_prefix_pages; s.max_pages = max_pages;
    s.page_log2 = page_log2_of(page_size); s.fp8 = t == DD_FP8_E4M3;
    return s;
}

size_t dd_paged_attention_shared_workspace_bytes(int n, int B, int H, int Hkv, int d, int page_size, int G, int max_prefix_pages, int max_pages,
                                                 dd_dtype cache_dtype)
{
    if (n < 1 || B < 1 || H < 1 || Hkv < 1 || H % Hkv != 0 || (d != 64 && d != 128) || G < 1 || max_prefix_pages < 1 || max_pages < 1) return 0;
    if (page_log2_of(page_size) < 0 || (cache_dtype != DD_BF16 && cache_dtype != DD_FP8_E4M3)) return 0;
    if ((double)max_pages * page_size >= 1073741824.0 || (double)max_prefix_pages * page_size >= 1073741824.0) return 0;
    const dd::SharedAttnShape s = shared_shape(n, B, H, Hkv, d, page_size, G, max_prefix_pages, max_pages, cache_dtype);
    return dd::shared_attention_fits(s) ? dd::shared_attention_workspace_bytes(s) : 0;
}

int dd_paged_attention_shared(const void *Q, const void *Kc, const void *Vc, const float *k_scale, const float *v_scale,
                              const int32_t *prefix_table, const int32_t *prefix_lens, const int32_t *group_starts,
                              const int32_t *block_table, const int32_t *kv_lens, void *O,
                              int n, int B, int H, int Hkv, int d, int num_pages, int page_size, int G, int max_prefix_pages,
                              int max_pages, dd_dtype cache_dtype, void *workspace, size_t workspace_bytes, void *stream)
{
    int rc = check_pages(Kc, Vc, k_scale, v_scale, block_table, kv_lens, n, B, Hkv, d, num_pages, page_size, max_pages, cache_dtype);
    if (rc != DD_OK) return rc;
    if (!prefix_table || !prefix_lens || !group_starts) return DD_ERR_NULL;
    if (H < 1 || H % Hkv != 0 || G < 1 || max_prefix_pages < 1 || (double)max_prefix_pages * page_size >= 1073741824.0) return DD_ERR_SHAPE;
    if (((reinterpret_cast<uintptr_t>(prefix_table) | reinterpret_cast<uintptr_t>(prefix_lens) | reinterpret_cast<uintptr_t>(group_starts)) & 3u) != 0) return DD_ERR_ALIGN;
    if (n == 0) return DD_OK;
    if (!Q || !O) return DD_ERR_NULL;
    const dd::SharedAttnShape s = shared_shape(n, B, H, Hkv, d, page_size, G, max_prefix_pages, max_pages, cache_dtype);
    if (!dd::shared_attention_fits(s)) return DD_ERR_SHAPE;
    if (misaligned16(Q) || misaligned16(O)) return DD_ERR_ALIGN;
    rc = check_workspace(workspace, workspace_bytes, dd::shared_attention_workspace_bytes(s));
    if (rc != DD_OK) return rc;
    const uintptr_t rows_bytes = (uintptr_t)B * H * n * d * 2, cache_bytes = (uintptr_t)num_pages * Hkv * page_size * d * (s.fp8 ? 1 : 2);
    const uintptr_t scale_bytes = (uintptr_t)num_pages * Hkv * sizeof(float);
    if (overlap(O, rows_bytes, Q, rows_bytes) || overlap(O, rows_bytes, Kc, cache_bytes) || overlap(O, rows_bytes, Vc, cache_bytes)) return DD_ERR_SHAPE;
    if (s.fp8 && (overlap(O, rows_bytes, k_scale, scale_bytes) || overlap(O, rows_bytes, v_scale, scale_bytes))) return DD_ERR_SHAPE;
    if (overlap(O, rows_bytes, prefix_table, (uintptr_t)G * max_prefix_pages * 4) || overlap(O, rows_bytes, prefix_lens, (uintptr_t)G * 4) ||
        overlap(O, rows_bytes, group_starts, ((uintptr_t)G + 1) * 4) || overlap(O, rows_bytes, block_table, (uintptr_t)B * max_pages * 4) ||
        overlap(O, rows_bytes, kv_lens, (uintptr_t)B * 4))
        return DD_ERR_SHAPE;
    dd::SharedAttnArgs a;
    a.s = s;
    a.Q = Q; a.Kc = Kc; a.Vc = Vc; a.O = O;
    a.k_scale = s.fp8 ? k_scale : nullptr; a.v_scale = s.fp8 ? v_scale : nullptr;
    a.prefix_table = prefix_table; a.prefix_lens = prefix_lens; a.group_starts = group_starts; a.table = block_table; a.kv_lens = kv_lens;
    a.num_pages = num_pages; a.workspace = workspace;
    const hipError_t e = dd::launch_attention_shared(a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? DD_OK : DD_ERR_LAUNCH;
}

size_t dd_verify_remask_workspace_bytes(int B, int G, int V, dd_dtype logit_dtype)
{
    if (B < 0 || G < 0 || V < 1 || (logit_dtype != DD_F32 && logit_dtype != DD_BF16)) return 0;
    if ((double)B * G >= 2147483648.0) return 0;
    return dd::verify_workspace_bytes(B * G, V, logit_dtype == DD_BF16 ? 2 : 4);
}

}  // extern "C"

// everything dd_verify_remask checks before it launches, except the workspace; DD_OK with *empty set for a no-op
static int check_verify_remask(const void *logits_d, const void *logits_v, const uint8_t *mask, int mode, float threshold,
                               const uint8_t *out_mask, const int32_t *out_tokens, const float *out_scores,
                               int B, int G, int V, int logit_dtype, bool *empty)
{
    *empty = false;
    if (mode < DD_TRUST || mode > DD_CONF_TOPK) return DD_ERR_MODE;
    if ((mode == DD_KL_TOPK || mode == DD_CONF_TOPK) && !(threshold >= 0.0f && threshold <= 3.0e38f)) return DD_ERR_SHAPE;
    if (logit_dtype != DD_F32 && logit_dtype != DD_BF16) return DD_ERR_DTYPE;
    if (B < 0 || G < 0 || V < 1) return DD_ERR_SHAPE;
    if ((double)B * G >= 2147483648.0) return DD_ERR_SHAPE;
    const int eb = logit_dtype == DD_BF16 ? 2 : 4;
    if (((long)V * eb) % 16 != 0) return DD_ERR_ALIGN;
    if (B == 0 || G == 0) {
        *empty = true;
        return DD_OK;
    }
    const bool kl = (mode == DD_KL_THRESH || mode == DD_KL_PROB || mode == DD_KL_TOPK);
    if (!logits_v || !mask || !out_mask || !out_tokens || !out_scores) return DD_ERR_NULL;
    if (kl && !logits_d) return DD_ERR_NULL;
    {
        // The per-row rules read mask[i] and write out_mask[i] in one lane, so updating the mask in place is
        // safe; the per-sequence rules (Eq. 6, the budgeted ones) read every mask byte of a sequence while other
        // workgroups write out_mask.  Ranges that overlap without being identical are never meaningful.
        const uintptr_t m0 = reinterpret_cast<uintptr_t>(mask), o0 = reinterpret_cast<uintptr_t>(out_mask);
        const uintptr_t n = (uintptr_t)B * (uintptr_t)G;
        const bool overlap = m0 < o0 + n && o0 < m0 + n;
        const bool per_sequence = mode == DD_KL_PROB || mode == DD_KL_TOPK || mode == DD_CONF_TOPK;
        if (overlap && (per_sequence || m0 != o0)) return DD_ERR_SHAPE;
    }
    if (misaligned16(logits_v) || (kl && misaligned16(logits_d))) return DD_ERR_ALIGN;
    return DD_OK;
}

static int verify_remask(const void *logits_d, const void *logits_v, const uint8_t *mask, int mode, float threshold,
                         uint64_t seed, uint8_t *out_mask, int32_t *out_tokens, float *out_scores, int B, int G, int V,
                         int logit_dtype, void *workspace, size_t workspace_bytes, void *stream, bool static_scratch)
{
    bool empty = false;
    int rc = check_verify_remask(logits_d, logits_v, mask, mode, threshold, out_mask, out_tokens, out_scores, B, G, V,
                                 logit_dtype, &empty);
    if (rc != DD_OK || empty) return rc;
    const int eb = logit_dtype == DD_BF16 ? 2 : 4;
    if (static_scratch) {
        const size_t need = dd::verify_workspace_bytes(B * G, V, eb);
        if (need > kStaticScratchBytes) return DD_ERR_WORKSPACE;  // more partial states than the static array holds
        workspace = nullptr;
        workspace_bytes = need;
        if (need > 0 && (rc = scratch_of_current_device(&workspace)) != DD_OK) return rc;
    }
    rc = check_workspace(workspace, workspace_bytes, dd::verify_least_workspace_bytes(B * G, V, eb));
    if (rc != DD_OK) return rc;
    const bool kl = (mode == DD_KL_THRESH || mode == DD_KL_PROB || mode == DD_KL_TOPK);
    const hipError_t e = dd::launch_verify(kl ? logits_d : nullptr, logits_v, mask, mode, threshold, seed,
                                           out_mask, out_tokens, out_scores, B, G, V, logit_dtype == DD_BF16,
                                           workspace, workspace_bytes, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? DD_OK : DD_ERR_LAUNCH;
}

extern "C" {

int dd_verify_remask(const void *logits_d, const void *logits_v, const uint8_t *mask,
                     dd_mode mode, float threshold, uint64_t seed,
                     uint8_t *out_mask, int32_t *out_tokens, float *out_scores,
                     int B, int G, int V, dd_dtype logit_dtype,
                     void *workspace, size_t workspace_bytes, void *stream)
{
    return verify_remask(logits_d, logits_v, mask, (int)mode, threshold, seed, out_mask, out_tokens, out_scores, B, G, V,
                         (int)logit_dtype, workspace, workspace_bytes, stream, false);
}

int dd_verify_remask_static(const void *logits_d, const void *logits_v, const uint8_t *mask,
                            dd_mode mode, float threshold, uint64_t seed,
                            uint8_t *out_mask, int32_t *out_tokens, float *out_scores,
                            int B, int G, int V, dd_dtype logit_dtype, void *stream)
{
    // every partial state the finishing kernel reads is written by the streaming kernel of the same call:
    // nothing in the static array has to be cleared between calls
    return verify_remask(logits_d, logits_v, mask, (int)mode, threshold, seed, out_mask, out_tokens, out_scores, B, G, V,
                         (int)logit_dtype, nullptr, 0, stream, true);
}

size_t dd_unmask_workspace_bytes(int B, int G, int V, dd_dtype logit_dtype)
{
    return dd_verify_remask_workspace_bytes(B, G, V, logit_dtype);
}

int dd_unmask(const void *logits_d, const uint8_t *mask, dd_unmask_mode mode, float threshold,
              int32_t *x_tokens, uint8_t *out_mask, int32_t *out_tokens, float *out_conf,
              int B, int G, int V, dd_dtype logit_dtype,
              void *workspace, size_t workspace_bytes, void *stream)
{
    if (mode != DD_UNMASK_THRESH && mode != DD_UNMASK_TOPK) return DD_ERR_MODE;
    if (mode == DD_UNMASK_TOPK && !(threshold >= 0.0f && threshold <= 3.0e38f)) return DD_ERR_SHAPE;
    if (logit_dtype != DD_F32 && logit_dtype != DD_BF16) return DD_ERR_DTYPE;
    if (B < 0 || G < 0 || V < 1) return DD_ERR_SHAPE;
    if ((double)B * G >= 2147483648.0) return DD_ERR_SHAPE;
    const int eb = logit_dtype == DD_BF16 ? 2 : 4;
    if (((long)V * eb) % 16 != 0) return DD_ERR_ALIGN;
    if (B == 0 || G == 0) return DD_OK;
    if (!logits_d || !mask || !out_mask || !out_tokens || !out_conf) return DD_ERR_NULL;
    {
        // the selection reads every mask byte of a sequence while other lanes write out_mask
        const uintptr_t m0 = reinterpret_cast<uintptr_t>(mask), o0 = reinterpret_cast<uintptr_t>(out_mask);
        const uintptr_t n = (uintptr_t)B * (uintptr_t)G;
        if (m0 < o0 + n && o0 < m0 + n) return DD_ERR_SHAPE;
    }
    if (misaligned16(logits_d)) return DD_ERR_ALIGN;
    const int rc = check_workspace(workspace, workspace_bytes, dd::verify_least_workspace_bytes(B * G, V, eb));
    if (rc != DD_OK) return rc;
    const hipError_t e = dd::launch_verify(nullptr, logits_d, mask,
                                           mode == DD_UNMASK_TOPK ? dd::kModeUnmaskTopk : dd::kModeUnmaskThresh,
                                           threshold, 0, out_mask, out_tokens, out_conf, B, G, V,
                                           logit_dtype == DD_BF16, workspace, workspace_bytes, static_cast<hipStream_t>(stream), x_tokens);
    return e == hipSuccess ? DD_OK : DD_ERR_LAUNCH;
}

size_t dd_verify_scores_workspace_bytes(int P, int V, dd_dtype logit_dtype)
{
    return dd_verify_remask_workspace_bytes(1, P, V, logit_dtype);
}

int dd_verify_scores(const void *logits_d, const void *logits_v,
                     float *out_kl, float *out_conf_v, int32_t *out_tok_v, float *out_conf_d, int32_t *out_tok_d,
                     int P, int V, dd_dtype logit_dtype, void *workspace, size_t workspace_bytes, void *stream)
{
    if (logit_dtype != DD_F32 && logit_dtype != DD_BF16) return DD_ERR_DTYPE;
    if (P < 0 || V < 1) return DD_ERR_SHAPE;
    const int eb = logit_dtype == DD_BF16 ? 2 : 4;
    if (((long)V * eb) % 16 != 0) return DD_ERR_ALIGN;
    if (P == 0) return DD_OK;
    if (!logits_d || !logits_v || !out_kl || !out_conf_v || !out_tok_v) return DD_ERR_NULL;
    if (misaligned16(logits_v) || misaligned16(logits_d)) return DD_ERR_ALIGN;
    const int rc = check_workspace(workspace, workspace_bytes, dd::verify_least_workspace_bytes(P, V, eb));
    if (rc != DD_OK) return rc;
    dd::VerifyExtra ex;
    ex.conf_v = out_conf_v;
    ex.conf_d = out_conf_d;
    ex.tok_d = out_tok_d;
    const hipError_t e = dd::launch_verify(logits_d, logits_v, nullptr, dd::kModeScores, 0.0f, 0, nullptr, out_tok_v,
                                           out_kl, 1, P, V, logit_dtype == DD_BF16, workspace, workspace_bytes,
                                           static_cast<hipStream_t>(stream), nullptr, &ex);
    return e == hipSuccess ? DD_OK : DD_ERR_LAUNCH;
}

static bool draft_sizes(int B, int n, int bonus, int V, int with_drafter, dd_dtype t)
{
    const int nv = n + (bonus ? 1 : 0);
    if (B < 1 || n < 0 || n == 0x7fffffff || nv < 1 || V < 1) return false;
    if ((double)B * (n + 1.0) >= 1073741824.0) return false;
    return dd::verify_draft_workgroups(B, n, nv, V, t == DD_BF16, with_drafter != 0) < 16777216.0;
}

size_t dd_verify_draft_workspace_bytes(int B, int n, int bonus, int V, int with_drafter, dd_dtype logit_dtype)
{
    if (logit_dtype != DD_F32 && logit_dtype != DD_BF16) return 0;
    if (!draft_sizes(B, n, bonus, V, with_drafter, logit_dtype)) return 0;
    return dd::verify_draft_workspace_bytes(B, n, n + (bonus ? 1 : 0), V, logit_dtype == DD_BF16, with_drafter != 0);
}

int dd_verify_draft(const void *logits_v, const void *logits_d, const int32_t *tokens, const int32_t *n_draft,
                    const float *uniforms, const float *temperature,
                    int32_t *out_tokens, int32_t *out_accepted, float *out_chances,
                    int B, int n, int bonus, int V, dd_dtype logit_dtype, void *workspace, size_t workspace_bytes, void *stream)
{
    if (logit_dtype != DD_F32 && logit_dtype != DD_BF16) return DD_ERR_DTYPE;
    if (B < 0 || n < 0 || V < 1) return DD_ERR_SHAPE;
    const int eb = logit_dtype == DD_BF16 ? 2 : 4, nv = n + (bonus ? 1 : 0);
    if (((long)V * eb) % 16 != 0) return DD_ERR_ALIGN;
    if (B == 0) return DD_OK;
    if (!draft_sizes(B, n, bonus, V, logits_d != nullptr, logit_dtype)) return DD_ERR_SHAPE;
    if (!logits_v || !uniforms || !out_tokens || !out_accepted || (n > 0 && (!tokens || !out_chances))) return DD_ERR_NULL;
    uintptr_t words = 0;
    for (const void *p : {(const void *)tokens, (const void *)n_draft, (const void *)uniforms, (const void *)temperature, (const void *)out_tokens,
                          (const void *)out_accepted, (const void *)out_chances})
        words |= reinterpret_cast<uintptr_t>(p);
    if (misaligned16(logits_v) || misaligned16(logits_d) || (words & 3u) != 0) return DD_ERR_ALIGN;
    const int rc = check_workspace(workspace, workspace_bytes, dd::verify_draft_workspace_bytes(B, n, nv, V, logit_dtype == DD_BF16, logits_d != nullptr));
    if (rc != DD_OK) return rc;
    // (a sequence's inputs are read by some workgroups while others write outputs)
    struct Range { const void *at; uintptr_t bytes; };
    const uintptr_t seqs = (uintptr_t)B * 4, drafts = (uintptr_t)B * n * 4, both = seqs + drafts;
    const Range outs[3] = {{out_tokens, both}, {out_accepted, seqs}, {out_chances, drafts}};
    const Range ins[6] = {{logits_v, (uintptr_t)B * nv * V * eb}, {logits_d, (uintptr_t)B * n * V * eb}, {tokens, drafts}, {n_draft, seqs}, {uniforms, both},
                          {temperature, seqs}};
    for (int o = 0; o < 3; ++o) {
        for (int i = 0; i < 6; ++i)
            if (ins[i].at && outs[o].bytes && ins[i].bytes && overlap(outs[o].at, outs[o].bytes, ins[i].at, ins[i].bytes)) return DD_ERR_SHAPE;
        for (int i = 0; i < o; ++i)
            if (outs[o].bytes && outs[i].bytes && overlap(outs[o].at, outs[o].bytes, outs[i].at, outs[i].bytes)) return DD_ERR_SHAPE;
    }
    dd::DraftArgs a;
    a.logits_v = logits_v; a.logits_d = n > 0 ? logits_d : nullptr; a.tokens = tokens; a.n_draft = n_draft; a.uniforms = uniforms; a.temperature = temperature;
    a.out_tokens = out_tokens; a.out_accepted = out_accepted; a.out_chances = out_chances;
    a.B = B; a.n = n; a.nv = nv; a.V = V; a.bonus = bonus != 0; a.bf16 = logit_dtype == DD_BF16;
    a.workspace = workspace;
    const hipError_t e = dd::launch_verify_draft(a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? DD_OK : DD_ERR_LAUNCH;
}

}  // extern "C"
