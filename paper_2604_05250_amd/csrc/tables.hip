// Block tables, positions and slots from request lengths.  Sequence b holds  have = ceil(len / P)  pages and shall hold  need = ceil(new
// len / P):  what is over goes back to a stack of free pages, what is missing is taken from it, for all sequences at once.  Where a page
// goes or comes from follows from sums over the sequences before:  with R pages given back, F free before and F' = F + R after that,
//     the i-th page given back is stack[F' - 1 - i],   the t-th page taken was stack[F' - 1 - t],   i and t in the sequences' order
// so that a call and its opposite leave tables and stack as they were.  A sequence gets all it asks for if the pages asked for up to and
// with it are free, else it stays as it is.  There is next to nothing to read or to compute: what it takes is launches, and round trips to
// memory one after the other, of which the sums are one.  us for both ways of a step, two calls: a token of 16 sequences 10.4 (the calls cost the
// host 8), 57 sequences in mid-flight with up to 64 rows 13.7, 64 prompts of 2048 positions, 8192 pages of 16, 17.1.  One workgroup of 256
// threads takes as long for the first and 5 us more for the others.
#include "dd_internal.h"

namespace dd {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;

struct TableKernelArgs {
    int32_t *table, *stack, *num_free;
    const int32_t *lens, *new_lens;
    int32_t *out_lens, *positions, *slots;
    int n, B, page_log2, max_pages, capacity;
    int *between;                            // [1 + 2 B] of a call of two launches: F', each sequence's pages taken before it and its length
};

struct Growth { int len, have, want, need; bool fits; };
__device__ __forceinline__ Growth growth_of(const TableKernelArgs &a, int b)
{
    const int most = a.max_pages << a.page_log2, up = (1 << a.page_log2) - 1;
    Growth g;
    g.len = min(max(a.lens[b], 0), most);
    g.have = (g.len + up) >> a.page_log2;
    g.want = max(a.new_lens[b], 0);
    g.fits = g.want <= most;
    g.need = g.fits ? (g.want + up) >> a.page_log2 : g.have;
    return g;
}

// Two counts at once, given back above 32 bits, taken below: sums over the threads before, and over all (a table has fewer than 2^31 entries).
__device__ __forceinline__ void before(unsigned long long v, unsigned long long *of_wave, unsigned long long &pre, unsigned long long &all)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    unsigned long long s = v;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const unsigned long long x = __shfl_up(s, m);
        if (lane >= m) s += x;
    }
    __syncthreads();
    if (lane == 63) of_wave[wave] = s;
    __syncthreads();
    pre = s - v;
    all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const unsigned long long x = of_wave[w];
        pre += w < wave ? x : 0;
        all += x;
    }
}

// Row r of [0, n) of sequence b: its position and its place in the pages.  `first`: pages taken before the sequence's.
__device__ __forceinline__ void place_row(const TableKernelArgs &a, int b, int r, int len, int out, int have, int first, int top)
{
    const int p = len + r;                           // (less than 2^30 + n: no overflow)
    const size_t at = (size_t)b * a.n + r;
    a.positions[at] = p;
    int slot = -1;
    if (p < out) {
        const int j = p >> a.page_log2, page = j < have ? a.table[(size_t)b * a.max_pages + j] : a.stack[top - 1 - (first + j - have)];
        slot = (unsigned)page < (unsigned)a.capacity ? (page << a.page_log2) + (p & ((1 << a.page_log2) - 1)) : -1;
    }
    a.slots[at] = slot;
}

// One workgroup: sums, pages given back, and (ALL) everything else too; otherwise what the second launch needs to know.
template <bool ALL> __global__ __launch_bounds__(kThreads) void tables_kernel(TableKernelArgs a)
{
    __shared__ unsigned long long of_wave[kWaves];
    __shared__ int len_of[kThreads], out_of[kThreads], first_of[kThreads], most;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, up = (1 << a.page_log2) - 1;
    const int free_before = min(max(*a.num_free, 0), a.capacity);
    if (tid == 0) most = 0;
    // ---- of kThreads sequences from b0 on, a thread's: its pages, and those of the sequences before it in this lot
    Growth g{};
    unsigned long long pre = 0, lot = 0;
    auto count = [&](int b0) {
        g = Growth{};
        if (b0 + tid < a.B) g = growth_of(a, b0 + tid);
        before((unsigned long long)max(g.have - g.need, 0) << 32 | (unsigned)max(g.need - g.have, 0), of_wave, pre, lot);
    };
    const bool once = a.B <= kThreads;
    long long back = 0;
    for (int b0 = 0; b0 < a.B; b0 += kThreads) {
        count(b0);
        back += (long long)(lot >> 32);
    }
    const int top = (int)min(free_before + back, (long long)a.capacity);           // (a stack that is too small for its pages loses some)
    // ---- what comes back goes onto the stack, a wave per sequence
    if (back > 0) {
        long long so_far = 0;
        for (int b0 = 0; b0 < a.B; b0 += kThreads) {
            if (!once) count(b0);
            len_of[tid] = g.have;
            out_of[tid] = g.need;
            first_of[tid] = (int)(so_far + (long long)(pre >> 32));
            __syncthreads();
            for (int k = wave; k < min(kThreads, a.B - b0); k += kWaves) {
                const int have = len_of[k], need = out_of[k];
                int32_t *const row = a.table + (size_t)(b0 + k) * a.max_pages;
                for (int j = need + lane; j < have; j += 64) {
                    const int at = top - 1 - (first_of[k] + j - need);
                    if (at >= 0) a.stack[at] = row[j];
                    row[j] = -1;
                }
            }
            so_far += (long long)(lot >> 32);
            __syncthreads();
        }
    }
    // ---- who gets what
    long long so_far = 0;
    for (int b0 = 0; b0 < a.B; b0 += kThreads) {
        if (!once) count(b0);
        const int b = b0 + tid, take = max(g.need - g.have, 0);
        const long long end = so_far + (long long)(pre & 0xffffffffu) + take;
        const bool granted = g.fits && (take == 0 || end <= top);
        const int out = granted ? g.want : g.len, first = granted ? (int)(end - take) : 0;
        if (granted && take > 0) atomicMax(&most, (int)end);
        if (b < a.B) {
            a.out_lens[b] = out;
            if constexpr (!ALL) {
                a.between[1 + 2 * b] = first;
                a.between[2 + 2 * b] = g.len;
            }
        }
        if constexpr (ALL) {
            len_of[tid] = g.len;
            out_of[tid] = out;
            first_of[tid] = first;
            __syncthreads();
            const int lot_size = min(kThreads, a.B - b0);
            for (int k = wave; k < lot_size; k += kWaves) {
                const int have = (len_of[k] + up) >> a.page_log2, need = (out_of[k] + up) >> a.page_log2;
                int32_t *const row = a.table + (size_t)(b0 + k) * a.max_pages;
                for (int j = have + lane; j < need; j += 64) row[j] = a.stack[top - 1 - (first_of[k] + j - have)];
            }
            for (int i = tid; i < lot_size * a.n; i += kThreads) {
                const int k = i / a.n;
                place_row(a, b0 + k, i - k * a.n, len_of[k], out_of[k], (len_of[k] + up) >> a.page_log2, first_of[k], top);
            }
            __syncthreads();
        }
        so_far += (long long)(lot & 0xffffffffu);
    }
    __syncthreads();
    if (tid == 0) {
        *a.num_free = top - most;
        if constexpr (!ALL) a.between[0] = top;
    }
}

// The rest of a large call: entries of the table and places of rows, a piece of a sequence per workgroup.
constexpr int kPiece = 2048;
__global__ __launch_bounds__(256) void places_kernel(TableKernelArgs a, int pieces)
{
    const int b = (int)(blockIdx.x / (unsigned)pieces), from = (int)(blockIdx.x - (unsigned)b * (unsigned)pieces) * kPiece;
    const int up = (1 << a.page_log2) - 1, top = a.between[0], first = a.between[1 + 2 * b], len = a.between[2 + 2 * b], out = a.out_lens[b];
    const int have = (len + up) >> a.page_log2, need = (out + up) >> a.page_log2;
    int32_t *const row = a.table + (size_t)b * a.max_pages;
    for (int j = have + from + (int)threadIdx.x; j < min(need, have + from + kPiece); j += 256) row[j] = a.stack[top - 1 - (first + j - have)];
    for (int r = from + (int)threadIdx.x; r < min(a.n, from + kPiece); r += 256) place_row(a, b, r, len, out, have, first, top);
}

int pieces_of(int n, int max_pages) { return ((n > max_pages ? n : max_pages) + kPiece - 1) / kPiece; }
// One workgroup for everything, or a second launch for entries and rows.  us for a call and its opposite, one / two launches, pages of 16:
//     16 sequences, a token, tables of 64 entries         7.9 / 11.4       8192 rows: 16 x 512      11.6 / 12.4     128 x 64    17.5 / 17.1
//     the same, tables of 4096                            7.7 / 12.0       16384: 16 x 1024         14.4 / 12.7
//     all 65536 entries there and back: 16 x 4096        30.0 / 33.9       32768: 32 x 1024         21.0 / 13.8     1 x 32768   25.4 / 17.9
//     64 x 1024  32.1 / 37.8      256 x 256  35.9 / 38.2
// So two from 8192 rows on; entries that move cost as much either way, as what comes back is one workgroup's in both (a wave per sequence),
// and those that do not move cost nothing, so 65536 of them is as far as this was timed.  Many sequences are slower in one launch
// than they need be, a token of 1000 on 16 entries 20.0 / 12.1, of 4000 76.4 / 33.0: the rule does not go by that.
bool small(int n, int B, int max_pages) { return (double)B * n <= 8192 && (double)B * max_pages <= 65536; }

}  // namespace

double paged_resize_workgroups(int n, int B, int max_pages) { return (double)B * pieces_of(n, max_pages); }
size_t paged_resize_workspace_bytes(int n, int B, int max_pages) { return small(n, B, max_pages) ? 0 : ((size_t)B * 2 + 1) * sizeof(int); }

hipError_t launch_paged_resize(const TableArgs &t, hipStream_t stream)
{
    const TableKernelArgs a{t.table, t.stack, t.num_free, t.lens, t.new_lens, t.out_lens, t.positions, t.slots, t.n, t.B, t.page_log2, t.max_pages, t.capacity,
                            static_cast<int *>(t.workspace)};
    if (small(t.n, t.B, t.max_pages)) return launch(tables_kernel<true>, dim3(1), dim3(kThreads), stream, a);
    const hipError_t e = launch(tables_kernel<false>, dim3(1), dim3(kThreads), stream, a);
    if (e != hipSuccess) return e;
    const int pieces = pieces_of(t.n, t.max_pages);
    return launch(places_kernel, dim3((unsigned)t.B * (unsigned)pieces), dim3(256), stream, a, pieces);
}

}  // namespace dd
