// paged_plan.cuh -- how one paged-attention call is cut over the GPU, and the
// format of the partial results.
//
// A unit is (row tile, request, key head): n_gt * n_bt row tiles, all units of a
// request with the same visible keys.  The visible keys of a request are cut into
// tiles of kTile keys.  Work is counted in quarters of a tile: a unit of n tiles is
// 4 n + extra quarters, `extra` for what a change of units costs a block: 3 where rows
// are copied, else 7 (128 requests of 1-2000 tokens, one token 55.3 us with 1, 52.2 with
// 3, 53.4 with 4; block of 32 72.0 with 4, 65.2 with 7, 64.4 with 12, where 64 requests of
// 256-8192 tokens lose 1 us).  The quarters of all units, in the order (row tile, request,
// key head, tile), are shared out evenly over the blocks, at least four to a block,
// and a tile belongs to the block that has its first quarter.  So every block is
// busy for the same time whatever the lengths are, and a long request is split over
// as many blocks as it is worth.  Where there are several row tiles, the blocks of one are at the
// same keys as the blocks of another at any time, and all but the first find them
// in L2.  The lengths are on the device, so each block finds its share
// itself by a scan over the requests (a few KB).
//
// A run of tiles of one unit is a segment.  A segment that covers its unit writes
// the output; any other writes (m, l, O) -- running maximum in units of log2,
// sum and unnormalised output -- to partial 2 c (the segment goes on with a unit of
// an earlier block c - 1) or 2 c + 1 (it begins one that later blocks go on with).  A
// second launch joins them, told by notes what to join.
//
// Workspace: n_cta notes, then 2 n_cta partials.
#pragma once

#include "hybrid_common.cuh"
#include "softmax_kernels.h"
#include "tc_ptx.cuh"

namespace hyb {
namespace paged {

constexpr int kTile = 128;

// Visible keys of a context of len tokens: [0, sink) and [lo, len), sink <= lo;
// as tiles: `ns` tiles from 0 (those of the sinks), then `first`, first + 1, ...
struct Visible {
    int len, lo, sink;
    int ns, first, tiles;
};

__device__ __forceinline__ Visible visible_keys(const PagedArgs &a, int len)
{
    Visible v;
    const int cap = a.max_pages * a.page_size;              // < 2^31 - 255 (the host's check)
    if (len < 0) len = 0;
    if (len > cap) len = cap;
    v.len = len;
    v.lo = a.window > 0 && len > a.window ? len - a.window : 0;
    v.sink = v.lo > 0 ? (a.sink < v.lo ? a.sink : v.lo) : 0;
    v.ns = (v.sink + kTile - 1) / kTile;
    v.first = v.lo / kTile > v.ns ? v.lo / kTile : v.ns;
    const int last = (len + kTile - 1) / kTile;
    v.tiles = v.ns + (last > v.first ? last - v.first : 0);
    return v;
}
__device__ __forceinline__ bool length_ok(const PagedArgs &a, int len)
{
    return len >= 0 && len <= a.max_pages * a.page_size;
}
// key tile of the i-th visible tile
__device__ __forceinline__ int key_tile(const Visible &v, int i) { return i < v.ns ? i : v.first + (i - v.ns); }
__device__ __forceinline__ bool key_visible(const Visible &v, int j) { return j < v.len && (j >= v.lo || j < v.sink); }

// Whether the n keys from j hold a visible one.
__device__ __forceinline__ bool any_visible(const Visible &v, int j, int n)
{
    return (j < v.len && j + n > v.lo) || j < v.sink;
}

__device__ __forceinline__ int row_tiles(const PagedArgs &a) { return a.n_gt * a.n_bt; }

// Quarters of a unit of n tiles.
__device__ __forceinline__ int unit_quarters(const PagedArgs &a, int tiles) { return tiles > 0 ? 4 * tiles + a.extra : 0; }

// Shares of T quarters over C blocks: the first T % C blocks take one more.
// T < 2^31 (the host's check).
struct Shares {
    int per, rem, C;
    __device__ Shares(int T, int n_cta)
    {
        C = T / 4 < n_cta ? T / 4 : n_cta;
        per = C == 0 ? 0 : T / C;
        rem = T - per * C;
    }
    __device__ int start(int c) const { return per * c + (c < rem ? c : rem); }
    // block of a quarter
    __device__ int block_of(int t) const
    {
        const int big = rem * (per + 1);
        return t < big ? t / (per + 1) : rem + (t - big) / per;
    }
};

// What the join does at the boundary between blocks c and c + 1: written by block c
// when its last segment is the first part of a unit that later blocks go on with.
struct JoinNote {
    int cut;               // 0: nothing to join
    int req, head, rt;     // the unit
    int last;              // block of its last tile: partials 2 c + 1, 2 (c + 1), ... 2 last
    int pad[3];
};

// Scratch of the search for a block's share.
struct PlanSmem {
    int warp[16];
    int req, before, len;
};

// The segments of a block's share, one after another.
struct Walk {
    int t, t1;             // next quarter, end of the share
    int base;              // quarters of the row tiles before, and of the requests before `req`
    int req, rt;           // request and row tile
    Visible vis;
    // the current segment: tiles [i0, i1) of key head `head` of request `req`
    int head, i0, i1;

    __device__ bool next(const PagedArgs &a)
    {
        while (t < t1) {
            int unit = unit_quarters(a, vis.tiles);
            while (t >= base + unit * a.Hkv) {              // next request with visible keys
                base += unit * a.Hkv;
                if (++req == a.n_req) {
                    req = 0;
                    ++rt;
                }
                vis = visible_keys(a, __ldg(a.lens + req));
                unit = unit_quarters(a, vis.tiles);
            }
            const int rel = t - base;
            const int h = (unsigned)rel / (unsigned)unit;
            const int q0 = rel - h * unit, q1 = unit - q0 < t1 - t ? unit : q0 + (t1 - t);
            t += q1 - q0;
            const int first = (q0 + 3) >> 2, end = (q1 + 3) >> 2;       // tiles whose first quarter is here
            if (first >= vis.tiles) continue;
            head = h;
            i0 = first;
            i1 = end < vis.tiles ? end : vis.tiles;
            return true;
        }
        return false;
    }
    __device__ bool whole() const { return i0 == 0 && i1 == vis.tiles; }
    __device__ int slot() const { return 2 * (int)blockIdx.x + (i0 == 0 ? 1 : 0); }
};

// The walk up to the request, which the caller fills in; returns the first quarter's
// place in its row tile (of `total` quarters per key head).
__device__ __forceinline__ int start_walk(const PagedArgs &a, int total, const Shares &sh, Walk &w)
{
    const int t0 = sh.start(blockIdx.x), row_tile = total * a.Hkv;
    w.t = t0;
    w.t1 = sh.start(blockIdx.x + 1);
    w.rt = row_tiles(a) == 1 ? 0 : t0 / row_tile;
    w.base = w.rt * row_tile;
    w.i0 = 1;                                               // no segment yet
    w.i1 = 0;
    return t0 - w.base;
}

// Find the block's share; false if it has none.  By each warp for itself, for few
// requests (kPerLane a lane): no barrier and no shared memory between the lengths
// and the first use of the share.
constexpr int kPerLane = 4, kFewRequests = 32 * kPerLane;
__device__ __forceinline__ bool find_share_warp(const PagedArgs &a, Walk &w, Shares &sh)
{
    const int lane = threadIdx.x & 31, M = a.Hkv;
    int len[kPerLane], n[kPerLane], sum = 0;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) {
        const int r = lane * kPerLane + i;
        len[i] = r < a.n_req ? __ldg(a.lens + r) : 0;
        bad |= !length_ok(a, len[i]);
    }
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) {
        n[i] = unit_quarters(a, visible_keys(a, len[i]).tiles);
        sum += n[i];
    }
    if (bad) raise_error(a.err, ERR_BAD_INDEX);
    int inc = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += v;
    }
    const int total = __shfl_sync(0xffffffffu, inc, 31);
    sh = Shares(total * M * row_tiles(a), a.n_cta);
    if ((int)blockIdx.x >= sh.C) return false;
    const int at = start_walk(a, total, sh, w);
    int b = inc - sum, req = lane * kPerLane, length = len[0];
    const unsigned holder = __ballot_sync(0xffffffffu, at >= b * M && at < inc * M);
#pragma unroll
    for (int i = 0; i + 1 < kPerLane; ++i)
        if (at >= (b + n[i]) * M && req == lane * kPerLane + i) {
            b += n[i];
            ++req;
            length = len[i + 1];
        }
    const int from = __ffs(holder) - 1;
    w.req = __shfl_sync(0xffffffffu, req, from);
    w.base += M * __shfl_sync(0xffffffffu, b, from);
    w.vis = visible_keys(a, __shfl_sync(0xffffffffu, length, from));
    return true;
}

// By a scan over the requests with the whole block, NT threads (a multiple of 32),
// each with a run of them, for any number.  May synchronise the block (also where
// it returns false).
template <int NT>
__device__ __forceinline__ bool find_share(const PagedArgs &a, PlanSmem &s, Walk &w, Shares &sh)
{
    if (a.n_req <= kFewRequests) return find_share_warp(a, w, sh);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int M = a.Hkv, per = (a.n_req + NT - 1) / NT;
    const int q0 = tid * per < a.n_req ? tid * per : a.n_req, q1 = q0 + per < a.n_req ? q0 + per : a.n_req;
    int sum = 0;
    bool bad = false;
    for (int r = q0; r < q1; ++r) {
        const int len = __ldg(a.lens + r);
        bad |= !length_ok(a, len);
        sum += unit_quarters(a, visible_keys(a, len).tiles);
    }
    if (bad) raise_error(a.err, ERR_BAD_INDEX);
    int inc = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += v;
    }
    if (lane == 31) s.warp[warp] = inc;
    __syncthreads();
    int b = inc - sum, total = 0;
#pragma unroll
    for (int x = 0; x < NT / 32; ++x) {
        if (x < warp) b += s.warp[x];
        total += s.warp[x];
    }
    sh = Shares(total * M * row_tiles(a), a.n_cta);
    const bool work = (int)blockIdx.x < sh.C;
    if (work) {
        const int at = start_walk(a, total, sh, w);
        if (at >= b * M && at < (b + sum) * M) {            // one thread's run holds the first quarter
            for (int r = q0; r < q1; ++r) {
                const int len = __ldg(a.lens + r), n = unit_quarters(a, visible_keys(a, len).tiles);
                if (at < (b + n) * M) {
                    s.req = r;
                    s.before = b;
                    s.len = len;
                    break;
                }
                b += n;
            }
        }
    }
    __syncthreads();
    if (!work) return false;
    w.req = s.req;
    w.base += M * s.before;
    w.vis = visible_keys(a, s.len);
    return true;
}

// The note of this block, from its last segment (one thread).
__device__ __forceinline__ void write_note(const PagedArgs &a, bool work, const Walk &w, const Shares &sh)
{
    JoinNote n{};
    if (work && w.i0 == 0 && w.i1 < w.vis.tiles) {
        n.cut = 1;
        n.req = w.req;
        n.head = w.head;
        n.rt = w.rt;
        n.last = sh.block_of(w.base + w.head * unit_quarters(a, w.vis.tiles) + 4 * (w.vis.tiles - 1));
    }
    a.notes[blockIdx.x] = n;
}

// Zeros for the requests without a visible key, shared over the blocks.
template <typename T, int NT>
__device__ __forceinline__ void write_empty(const PagedArgs &a, int thread)
{
    for (int r = blockIdx.x; r < a.n_req; r += gridDim.x) {
        if (visible_keys(a, __ldg(a.lens + r)).tiles > 0) continue;
        constexpr int kPer = 16 / sizeof(T);
        uint4 *out = reinterpret_cast<uint4 *>(static_cast<T *>(a.O) + (size_t)r * a.B * a.Hq * a.d);
        const int n = a.B * a.Hq * a.d / kPer;
        for (int x = thread; x < n; x += NT) out[x] = make_uint4(0, 0, 0, 0);
    }
}

// A unit's rows: row rho is token i0 + rho / Gt, query head g0 + rho % Gt of the group.
struct Unit {
    int head, g0, i0;
};
__device__ __forceinline__ Unit unit_of(const PagedArgs &a, int head, int rt)
{
    Unit u;
    u.head = head;
    u.g0 = u.i0 = 0;
    if (row_tiles(a) > 1) {
        u.g0 = rt / a.n_bt * a.Gt;
        u.i0 = rt % a.n_bt * a.Bt;
    }
    return u;
}
// Element offset of row rho of a unit in Q and O, and whether the row exists.
__device__ __forceinline__ bool row_at(const PagedArgs &a, int req, const Unit &u, int rho, size_t &at)
{
    const int i = u.i0 + rho / a.Gt, g = u.g0 + rho % a.Gt;
    at = (((size_t)req * a.B + i) * a.Hq + (size_t)u.head * a.G + g) * a.d;
    return rho < a.Bt * a.Gt && i < a.B && g < a.G;
}

// 16 bytes to shared memory by cp.async, `bytes` (16 or 0) of them read and the rest zeros.
__device__ __forceinline__ void copy16(void *dst, const float *src, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(ptx::smem_u32(dst)), "l"(src), "r"(bytes)
                 : "memory");
}
// 16 bytes as two pairs
__device__ __forceinline__ void load_pairs(const void *p, ptx::f32x2 &a, ptx::f32x2 &b)
{
    const ulonglong2 v = *static_cast<const ulonglong2 *>(p);
    a.v = v.x;
    b.v = v.y;
}

// Partial slot: m[rows], l[rows], O[d][rows] (feature-major, so that the threads of a
// warp, one row each, write runs of memory), rows = Bt * Gt.
__host__ __device__ __forceinline__ size_t partial_floats(int rows, int d) { return ((size_t)rows * (d + 2) + 3) / 4 * 4; }

}  // namespace paged
}  // namespace hyb
