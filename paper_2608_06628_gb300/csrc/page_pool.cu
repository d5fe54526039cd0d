// page_pool.cu -- block tables and slot maps from request lengths, and the ring
// of free pages (hybrid_page_append, hybrid_page_release).
//
// Append: with P = page_size, request r needs
//     need_r = ceil((len_r + new_r) / P) - ceil(len_r / P)
// pages; exclusive sums of need and of new give its first page in the ring and
// its first slot.  A token at position p lies in page p / P, which is either in
// the table already (p / P < ceil(len_r / P)) or the ring's entry
// head + first_r + p / P - ceil(len_r / P).
//
// The work is a scan over requests (a few KB, in L2) and two ints written per
// token: latency at decoding sizes, and the write of slots for prompts.  One
// launch: every block scans all requests itself, 1024 at a time in shared
// memory, and writes the slots of its own range; a block-to-block scan would
// cost a second launch, about as long as the whole call at these sizes.
// Nothing a block reads is written by another one (table entries of new pages
// are only written, the ring and lengths are read from one array and written to
// another), so no block waits on another.
#include "hybrid_common.cuh"
#include "softmax_kernels.h"
#include "tc_pipeline.cuh"

namespace hyb {
namespace {

constexpr int kThreads = 256;
constexpr int kPer = 4;                     // requests per thread in a chunk
constexpr int kChunk = kThreads * kPer;

struct Scan2 {
    long long a, b;
};

// Exclusive scan of (a, b) over the block in thread order; `total` gets the sums.
__device__ Scan2 block_scan(Scan2 v, Scan2 &total, Scan2 *warp_sums)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Scan2 inc = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long a = __shfl_up_sync(0xffffffffu, inc.a, o), b = __shfl_up_sync(0xffffffffu, inc.b, o);
        if (lane >= o) {
            inc.a += a;
            inc.b += b;
        }
    }
    __syncthreads();                        // warp_sums free for reuse
    if (lane == 31) warp_sums[warp] = inc;
    __syncthreads();
    Scan2 before{0, 0};
    total = {0, 0};
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
        if (w < warp) {
            before.a += warp_sums[w].a;
            before.b += warp_sums[w].b;
        }
        total.a += warp_sums[w].a;
        total.b += warp_sums[w].b;
    }
    return {before.a + inc.a - v.a, before.b + inc.b - v.b};
}

// Pages of a context of len tokens.
__device__ __forceinline__ long long pages_of(long long len, int lg) { return (len + (1ll << lg) - 1) >> lg; }

// The ring's head and count, or an empty ring if they are out of range.
__device__ bool load_ring(const int *ring, int n_pages, int &head, int &count)
{
    head = ring[0];
    count = ring[1];
    if (head >= 0 && head < n_pages && count >= 0 && count <= n_pages) return true;
    head = count = 0;
    return false;
}

// out[t0 + i] = v[i] for the i with b <= t0 + i < e.
template <int V> __device__ __forceinline__ void write(int *out, int t0, int b, int e, const int (&v)[V])
{
    if (V == 4 && t0 >= b && t0 + 4 <= e && (reinterpret_cast<uintptr_t>(out) & 15) == 0) {
        *reinterpret_cast<int4 *>(out + t0) = make_int4(v[0], v[V > 1], v[V > 2 ? 2 : 0], v[V > 3 ? 3 : 0]);
        return;
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (t0 + i >= b && t0 + i < e) out[t0 + i] = v[i];
}

struct AppendArgs {
    const int *lens, *n_new, *free_pages, *ring_in;
    int *table, *slots, *positions, *tok_offsets, *lens_out, *ring_out;
    int n_req, n_slots, lg, n_pages, max_pages;   // page size 1 << lg
    unsigned *err;
};

// V slots in a row per thread: 4 share a search and 16-byte stores where there are
// many, 1 is the shorter chain where there are few.
template <int V> __global__ __launch_bounds__(kThreads) void k_page_append(const AppendArgs a)
{
    __shared__ int s_tok[kChunk + 1];       // first slot of each request, capped at n_slots
    __shared__ int s_len[kChunk], s_page[kChunk];
    __shared__ bool s_served[kChunk];
    __shared__ Scan2 s_warp[kThreads / 32];
    __shared__ int s_taken;
    const int tid = threadIdx.x;
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    int head, count;
    const bool ring_ok = load_ring(a.ring_in, a.n_pages, head, count);
    bool bad = !ring_ok;
    // this block's slots, a multiple of four
    const long long per = ((a.n_slots + (long long)gridDim.x - 1) / gridDim.x + 3) & ~3ll;
    const long long lo = per * blockIdx.x < a.n_slots ? per * blockIdx.x : a.n_slots;
    const long long hi = lo + per < a.n_slots ? lo + per : a.n_slots;
    long long tok0 = 0, page0 = 0;          // tokens and pages of the chunks before
    if (tid == 0) s_taken = 0;
    for (int r0 = 0, chunk = 0; r0 < a.n_req; r0 += kChunk, ++chunk) {
        const int nr = a.n_req - r0 < kChunk ? a.n_req - r0 : kChunk;
        const bool mine = chunk % gridDim.x == blockIdx.x;   // writes the per-request outputs
        int len[kPer], nw[kPer], need[kPer];
        bool valid[kPer];
        Scan2 sum{0, 0};
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int r = r0 + tid * kPer + i;
            len[i] = nw[i] = need[i] = 0;
            valid[i] = false;
            if (r < a.n_req) {
                len[i] = a.lens[r];
                nw[i] = a.n_new[r];
                const long long end = (long long)len[i] + nw[i];
                valid[i] = len[i] >= 0 && nw[i] >= 0 && end <= ((long long)a.max_pages << a.lg);
                if (valid[i]) need[i] = (int)(pages_of(end, a.lg) - pages_of(len[i], a.lg));
                if (nw[i] < 0) nw[i] = 0;
            }
            sum.a += nw[i];
            sum.b += need[i];
        }
        Scan2 total;
        Scan2 at = block_scan(sum, total, s_warp);
        at.a += tok0;
        at.b += page0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int l = tid * kPer + i, r = r0 + l;
            if (r < a.n_req) {
                const bool served =
                    valid[i] && (need[i] == 0 || at.b + need[i] <= count) && at.a + nw[i] <= a.n_slots;
                s_tok[l] = (int)(at.a < a.n_slots ? at.a : a.n_slots);
                s_len[l] = len[i];
                s_page[l] = served ? (int)at.b : 0;
                s_served[l] = served;
                bad |= !served;
                // the requests that take pages come before all that find too few, so
                // the pages taken are the first of the ring
                if (served && need[i] > 0) atomicMax(&s_taken, (int)at.b + need[i]);
                if (mine) {
                    a.lens_out[r] = served ? len[i] + nw[i] : len[i];
                    if (a.tok_offsets) a.tok_offsets[r] = s_tok[l];
                }
            }
            at.a += nw[i];
            at.b += need[i];
        }
        tok0 += total.a;
        page0 += total.b;
        if (tid == 0) s_tok[nr] = (int)(tok0 < a.n_slots ? tok0 : a.n_slots);
        __syncthreads();
        // the slots of this chunk that lie in this block's range
        const int b = s_tok[0] > lo ? s_tok[0] : (int)lo, e = s_tok[nr] < hi ? s_tok[nr] : (int)hi;
        for (int t0 = b / V * V + V * tid; t0 < e && b < e; t0 += V * kThreads) {
            int x = 0, y = nr;              // last request whose first slot is <= the first of them
            const int first = t0 > b ? t0 : b;
            while (y - x > 1) {
                const int m = (x + y) >> 1;
                if (s_tok[m] <= first) x = m;
                else y = m;
            }
            int slot[V], pos[V], entry_new[V], page[V];
            const int *from[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int t = t0 + i;
                slot[i] = -1;
                pos[i] = 0;
                entry_new[i] = -1;
                from[i] = nullptr;
                if (t < b || t >= e) continue;
                while (x + 1 < nr && s_tok[x + 1] <= t) ++x;
                if (!s_served[x]) continue;
                pos[i] = s_len[x] + (t - s_tok[x]);         // of a served request: fits
                const int j = pos[i] >> a.lg, old = (int)pages_of(s_len[x], a.lg);
                if (j >= old) {
                    const long long k = (long long)head + s_page[x] + (j - old);
                    from[i] = a.free_pages + (k < a.n_pages ? k : k - a.n_pages);
                    // a new page's first token is always a new one
                    if ((pos[i] & ((1 << a.lg) - 1)) == 0) entry_new[i] = x;
                } else {
                    from[i] = a.table + (size_t)(r0 + x) * a.max_pages + j;
                }
            }
#pragma unroll
            for (int i = 0; i < V; ++i) page[i] = from[i] ? *from[i] : 0;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (!from[i]) continue;
                if (entry_new[i] >= 0) a.table[(size_t)(r0 + entry_new[i]) * a.max_pages + (pos[i] >> a.lg)] = page[i];
                if (page[i] >= 0 && page[i] < a.n_pages) slot[i] = (page[i] << a.lg) + (pos[i] & ((1 << a.lg) - 1));
                else bad = true;
            }
            write<V>(a.slots, t0, b, e, slot);
            if (a.positions) write<V>(a.positions, t0, b, e, pos);
        }
        __syncthreads();                    // the chunk's arrays are read no more
    }
    // beyond the last token
    for (long long t = (tok0 > lo ? tok0 : lo) + tid; t < hi; t += kThreads) {
        a.slots[t] = -1;
        if (a.positions) a.positions[t] = 0;
    }
    if (blockIdx.x == 0) {
        __syncthreads();
        if (tid == 0) {
            const long long h = (long long)head + s_taken;
            a.ring_out[0] = ring_ok ? (int)(h < a.n_pages ? h : h - a.n_pages) : a.ring_in[0];
            a.ring_out[1] = ring_ok ? count - s_taken : a.ring_in[1];
            if (a.tok_offsets) a.tok_offsets[a.n_req] = (int)(tok0 < a.n_slots ? tok0 : a.n_slots);
        }
    }
    if (bad) raise_error(a.err, ERR_BAD_INDEX);
}

struct ReleaseArgs {
    const int *rows, *lens, *table, *ring_in;
    int *free_pages, *ring_out;
    int n_req, n_rows, lg, n_pages, max_pages;
    unsigned *err;
};

// Whether a released row has ever held an entry that is no page, on this device.
__device__ unsigned g_bad_entry;

// Page i of all released pages, in order, goes to the ring's entry head + count + i.
// Blocks take runs of kThreads pages in turn.  Entries that are no pages are taken out
// again by k_page_release_drop.
__global__ __launch_bounds__(kThreads) void k_page_release(const ReleaseArgs a)
{
    __shared__ int s_row[kChunk];
    __shared__ long long s_first[kChunk + 1];
    __shared__ Scan2 s_warp[kThreads / 32];
    const int tid = threadIdx.x;
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    int head, count;
    const bool ring_ok = load_ring(a.ring_in, a.n_pages, head, count);
    const long long room = ring_ok ? a.n_pages - count : 0;
    bool bad = !ring_ok;
    long long page0 = 0;
    for (int i0 = 0; i0 < a.n_rows; i0 += kChunk) {
        const int nr = a.n_rows - i0 < kChunk ? a.n_rows - i0 : kChunk;
        int k[kPer];
        Scan2 sum{0, 0};
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int l = tid * kPer + i;
            k[i] = 0;
            if (i0 + l < a.n_rows) {
                const int r = a.rows[i0 + l];
                const bool row_ok = r >= 0 && r < a.n_req;
                const int len = row_ok ? a.lens[r] : -1;
                const bool ok = len >= 0 && len <= ((long long)a.max_pages << a.lg);
                if (ok) k[i] = (int)pages_of(len, a.lg);
                s_row[l] = ok ? r : 0;
                bad |= !ok;
            }
            sum.a += k[i];
        }
        Scan2 total;
        Scan2 at = block_scan(sum, total, s_warp);
        at.a += page0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int l = tid * kPer + i;
            if (l < nr) s_first[l] = at.a;
            at.a += k[i];
        }
        const long long begin = page0;
        page0 += total.a;
        if (tid == 0) s_first[nr] = page0;
        __syncthreads();
        const long long end = page0 < room ? page0 : room;
        long long run = begin / kThreads;
        run += (blockIdx.x + gridDim.x - run % gridDim.x) % gridDim.x;   // first run of this block
        for (; run * kThreads < end; run += gridDim.x) {
            const long long i = run * kThreads + tid;
            if (i >= begin && i < end) {
                int x = 0, y = nr;
                while (y - x > 1) {
                    const int m = (x + y) >> 1;
                    if (s_first[m] <= i) x = m;
                    else y = m;
                }
                const int page = a.table[(size_t)s_row[x] * a.max_pages + (size_t)(i - s_first[x])];
                if (page < 0 || page >= a.n_pages) {
                    bad = true;
                    *const_cast<volatile unsigned *>(&g_bad_entry) = 1u;
                }
                const long long to = (long long)head + count + i;      // < 2 n_pages
                a.free_pages[to < a.n_pages ? to : to - a.n_pages] = page;
            }
        }
        __syncthreads();
    }
    if (page0 > room) bad = true;
    if (blockIdx.x == 0 && tid == 0) {
        a.ring_out[0] = a.ring_in[0];
        a.ring_out[1] = ring_ok ? count + (int)(page0 < room ? page0 : room) : a.ring_in[1];
    }
    if (bad) raise_error(a.err, ERR_BAD_INDEX);
}

// The pages of the release just before it without the entries that are no pages, closed up
// in order, by one block.  The healthy case is a look at a word that nothing sets, for a
// launch (2 us of the host's time, 0.6 us on the GPU): the blocks of the release know of each
// other's pages only when they are done, and the word outlives the call because calls on
// several streams share it.
__global__ __launch_bounds__(kThreads) void k_page_release_drop(const ReleaseArgs a)
{
    __shared__ Scan2 s_warp[kThreads / 32];
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    if (*const_cast<volatile unsigned *>(&g_bad_entry) == 0u) return;
    int head, count;
    if (!load_ring(a.ring_in, a.n_pages, head, count)) return;
    const int n = a.ring_out[1] - count;                        // entries of the release
    int kept = 0;
    for (int i0 = 0; i0 < n; i0 += kThreads) {
        const long long from = (long long)head + count + i0 + threadIdx.x;
        const int page = i0 + (int)threadIdx.x < n ? a.free_pages[from < a.n_pages ? from : from - a.n_pages] : -1;
        const bool keep = page >= 0 && page < a.n_pages;
        Scan2 total;
        const Scan2 at = block_scan({keep ? 1 : 0, 0}, total, s_warp);      // (a barrier behind the loads)
        const long long to = (long long)head + count + kept + at.a;
        if (keep) a.free_pages[to < a.n_pages ? to : to - a.n_pages] = page;
        kept += (int)total.a;
        __syncthreads();                                        // before the next entries are loaded
    }
    if (threadIdx.x == 0) a.ring_out[1] = count + kept;
}

// A thread per item (slots, a page) while that takes no more blocks than the GPU holds at once.
int blocks_for(long long items)
{
    const long long n = (items + kThreads - 1) / kThreads;
    return (int)(n < 1 ? 1 : (n > 608 ? 608 : n));
}

constexpr int kFewSlots = 608 * kThreads;   // a thread per slot

int log2_of(int page_size)
{
    int lg = 0;
    while ((1 << lg) < page_size) ++lg;
    return lg;
}

}  // namespace

cudaError_t launch_page_append(const hybrid_page_cfg &pg, int n_req, const int *lens, const int *n_new,
                               const int *free_pages, const int *ring_in, int *block_table, int *slots,
                               int *positions, int n_slots, int *tok_offsets, int *lens_out, int *ring_out,
                               unsigned *err, cudaStream_t st)
{
    AppendArgs a{lens,      n_new,    free_pages, ring_in, block_table,  slots,      positions,    tok_offsets,
                 lens_out,  ring_out, n_req,      n_slots, log2_of(pg.page_size), pg.n_pages, pg.max_pages, err};
    // 2048 slots 3.7 us with one slot a thread, 4.8 with four; 1024000 slots 12 and 9
    if (n_slots <= kFewSlots)
        return pipe::launch_early(k_page_append<1>, dim3(blocks_for(n_slots)), dim3(kThreads), 0, st, a);
    return pipe::launch_early(k_page_append<4>, dim3(blocks_for((n_slots + 3ll) / 4)), dim3(kThreads), 0, st, a);
}

cudaError_t launch_page_release(const hybrid_page_cfg &pg, int n_req, const int *rows, int n_rows, const int *lens,
                                const int *block_table, int *free_pages, const int *ring_in, int *ring_out,
                                unsigned *err, cudaStream_t st)
{
    ReleaseArgs a{rows,     lens,  block_table, ring_in,      free_pages, ring_out,
                  n_req,    n_rows, log2_of(pg.page_size), pg.n_pages, pg.max_pages, err};
    // at most the pool's pages move
    long long most = (long long)n_rows * pg.max_pages;
    if (most > pg.n_pages) most = pg.n_pages;
    const cudaError_t e = pipe::launch_early(k_page_release, dim3(blocks_for(most)), dim3(kThreads), 0, st, a);
    if (e != cudaSuccess || n_rows == 0) return e;
    return pipe::launch_early(k_page_release_drop, dim3(1), dim3(kThreads), 0, st, a);
}

}  // namespace hyb
