// paged_attn_few.cu -- attention over the paged cache for row tiles of at most 8 rows,
// float32 (hybrid_paged_attn): decoding.
//
// D / 8 lanes hold the queries of the R = 4 or 8 rows and a step's two keys, 8 features
// each:
//     x = q . k log2(e) / sqrt(d)    2 R partial products, added over the lanes by halves,
//                                    so that each lane ends with one (or two) of them
//     p = 2^(x - m), l += p          by that lane
//     o += p v                       p from its lane; o as R rows of 8 features a lane
// A row's maximum is moved, and its output rescaled, only when a score exceeds it by
// more than 8 (as in paged_attn_tc.cu).  Each group of D / 8 lanes has an m, l and o of
// its own; nothing is shared until the end of a segment, when the groups of a warp are
// added by shuffles and the warps in shared memory, in a fixed order.  A lane copies
// what it alone reads (cp.async, kStages - 1 steps ahead), so the loop has no barrier.
//
// Bound by memory with 4 rows: 64 requests of 256-8192 tokens, 4 key heads, d = 128
// 173 us (6.4 TB/s), d = 64 92 us, where a version with chunks of 32 or 64 keys, two barriers
// each and scores through shared memory took 297 us.  With 8 rows the queries and
// outputs fill 128 registers, so one block to a multiprocessor, 179 and 103 us (one key
// to a step 223 and 121 us: 2 warps to a scheduler, and each step waits for its sums).
#include "paged_plan.cuh"
#include "tc_pipeline.cuh"

namespace hyb {
namespace {

using namespace paged;
using ptx::f32x2;
using ptx::pair2;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kKeys = 2;                        // of a lane in a step
constexpr int kRun = kTile / kWarps;            // keys of a warp in a tile, side by side: of one page
constexpr float kSlack = 8.f;

template <int D, int R> struct Smem {
    static constexpr int kStages = R == 4 ? 3 : 4;
    float4 ring[kWarps][kStages][4 * kKeys][32];            // [2 key + half]: K, then V
    float o[kWarps][R][D];
    float m[kWarps][R], l[kWarps][R];
    PlanSmem plan;
};

template <int D, int R>
__global__ __launch_bounds__(kThreads, R == 4 ? 2 : 1) void k_paged_attn_few(const PagedArgs a, int page_lg)
{
    constexpr int kStages = Smem<D, R>::kStages;
    constexpr int LPK = D / 8, SLOTS = 32 / LPK;            // lanes of a key, groups of a warp
    constexpr int kSteps = kRun / (kKeys * SLOTS);          // steps of a tile
    // the products key * R + row of a step: lane i ends with kOwn from kOwn (i % kSpread)
    constexpr int kProducts = kKeys * R, kSpread = kProducts < LPK ? kProducts : LPK, kOwn = kProducts / kSpread;
    static_assert(kStages * kKeys < 32, "bits of `seen`");
    extern __shared__ __align__(16) unsigned char raw[];
    Smem<D, R> &s = *reinterpret_cast<Smem<D, R> *>(raw);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int sub = lane % LPK, group = lane / LPK, lane0 = lane - sub;
    const int rows = a.Bt * a.Gt;
    const float to_log2 = pipe::kLog2e * rsqrtf((float)D);
    float4 (*ring)[4 * kKeys][32] = s.ring[warp];

    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    Walk w;
    Shares sh(0, 1);
    const bool work = find_share<kThreads>(a, s.plan, w, sh);
    bool go = work && w.next(a);
    // the copies, of the segment w: tile, step within it, stage
    int i = 0, at = 0, slot = 0;
    unsigned seen = 0;                                      // a bit for each key, the latest lowest
    int key = 0, ahead = 0;                                 // this group's first key of the run; page of the next run
    size_t run = 0;                                         // place of that key in the cache
    auto look_up = [&](int tile) {
        ahead = 0;
        if (tile >= w.i1) return;
        const int j = key_tile(w.vis, tile) * kTile + warp * kRun;
        if (any_visible(w.vis, j, kRun)) ahead = __ldg(a.table + (size_t)w.req * a.max_pages + (j >> page_lg));
    };
    auto fetch = [&]() {
        if (i < w.i1) {
            if (at == 0) {
                key = key_tile(w.vis, i) * kTile + warp * kRun + group;
                int page = ahead;
                if (page < 0 || page >= a.n_pages) {
                    raise_error(a.err, ERR_BAD_INDEX);
                    page = 0;
                }
                run = ((((size_t)page * a.Hkv + w.head) << page_lg) + (key & ((1 << page_lg) - 1))) * D + 4 * sub;
                look_up(i + 1);
            }
#pragma unroll
            for (int x = 0; x < kKeys; ++x) {
                const int step = (kKeys * at + x) * SLOTS;
                const bool see = key_visible(w.vis, key + step);
                const int bytes = see ? 16 : 0;             // masked keys and values are zeros
                const size_t from = see ? run + step * D : 0;
                seen = 2 * seen + see;
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const int c = y * 4 * LPK;
                    copy16(&ring[slot][2 * x + y][lane], static_cast<const float *>(a.K) + from + c, bytes);
                    copy16(&ring[slot][2 * (kKeys + x) + y][lane], static_cast<const float *>(a.V) + from + c, bytes);
                }
            }
            if (++at == kSteps) {
                at = 0;
                ++i;
            }
        } else {
            seen <<= kKeys;
        }
        slot = slot + 1 == kStages ? 0 : slot + 1;
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto first_page = [&]() {
        i = w.i0;
        at = slot = 0;
        look_up(i);
    };
    auto first_steps = [&]() {
#pragma unroll
        for (int x = 0; x < kStages - 1; ++x) fetch();
    };
    if (go) {
        first_page();
        first_steps();
    }
    while (go) {
        const Unit u = unit_of(a, w.head, w.rt);
        f32x2 q[R][4], o[R][4];
#pragma unroll
        for (int y = 0; y < R; ++y) {
            size_t from;
            const bool live = row_at(a, w.req, u, y, from);
#pragma unroll
            for (int c = 0; c < 4; ++c) q[y][c] = o[y][c] = pair2(0.f, 0.f);
            if (live) {
                const float *row = static_cast<const float *>(a.Q) + from + 4 * sub;
                load_pairs(row, q[y][0], q[y][1]);
                load_pairs(row + 4 * LPK, q[y][2], q[y][3]);
            }
        }
        float m[kOwn], l[kOwn];                             // of rows kOwn sub % R ...; l of this lane's key
#pragma unroll
        for (int e = 0; e < kOwn; ++e) {
            m[e] = -INFINITY;
            l[e] = 0.f;
        }
        const int steps = (w.i1 - w.i0) * kSteps;
        for (int n = 0, b = 0; n < steps; ++n, b = b + 1 == kStages ? 0 : b + 1) {
            fetch();                                        // into the stage of the step before
            asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
            float x[kProducts];
#pragma unroll
            for (int k = 0; k < kKeys; ++k) {
                f32x2 c[4];
                load_pairs(&ring[b][2 * k][lane], c[0], c[1]);
                load_pairs(&ring[b][2 * k + 1][lane], c[2], c[3]);
#pragma unroll
                for (int y = 0; y < R; ++y) {
                    const f32x2 t = ptx::fma2(c[2], q[y][2], ptx::fma2(c[1], q[y][1], ptx::mul2(c[0], q[y][0])));
                    float lo, hi;
                    ptx::unpair2(ptx::fma2(c[3], q[y][3], t), lo, hi);
                    x[R * k + y] = lo + hi;
                }
            }
            // add over the lanes, each time half of the products to half of the lanes
#pragma unroll
            for (int f = kSpread / 2; f > 0; f >>= 1)
#pragma unroll
                for (int y = 0; y < kOwn * f; ++y) {
                    const bool up = sub & f;
                    const float give = up ? x[y] : x[y + kOwn * f];
                    x[y] = (up ? x[y + kOwn * f] : x[y]) + __shfl_xor_sync(0xffffffffu, give, f);
                }
#pragma unroll
            for (int f = kSpread; f < LPK; f <<= 1) x[0] += __shfl_xor_sync(0xffffffffu, x[0], f);
            const bool see = seen >> (kKeys * kStages - 1 - sub % kSpread * kOwn / R) & 1;
            bool above = false;
#pragma unroll
            for (int e = 0; e < kOwn; ++e) {
                x[e] = see ? x[e] * to_log2 : -INFINITY;
                above |= x[e] > m[e] + kSlack;
            }
            if (__any_sync(0xffffffffu, above)) {
                float f[kOwn];
#pragma unroll
                for (int e = 0; e < kOwn; ++e) {
                    float now = x[e] > m[e] + kSlack ? x[e] : m[e];
                    now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, kSpread / 2));   // the lane of the other key
                    f[e] = m[e] == -INFINITY ? 1.f : exp2f(m[e] - now);                 // (o and l are zero, or NaN)
                    m[e] = now;
                    l[e] *= f[e];
                }
#pragma unroll
                for (int y = 0; y < R; ++y) {
                    const float g = __shfl_sync(0xffffffffu, f[y % kOwn], lane0 + y / kOwn);
                    const f32x2 gg = pair2(g, g);
#pragma unroll
                    for (int c = 0; c < 4; ++c) o[y][c] = ptx::mul2(o[y][c], gg);
                }
            }
#pragma unroll
            for (int e = 0; e < kOwn; ++e) {
                x[e] = exp2f(x[e] - (m[e] == -INFINITY ? 0.f : m[e]));
                l[e] += x[e];
            }
#pragma unroll
            for (int k = 0; k < kKeys; ++k) {
                f32x2 c[4];
                load_pairs(&ring[b][2 * (kKeys + k)][lane], c[0], c[1]);
                load_pairs(&ring[b][2 * (kKeys + k) + 1][lane], c[2], c[3]);
#pragma unroll
                for (int y = 0; y < R; ++y) {
                    const float t = __shfl_sync(0xffffffffu, x[(R * k + y) % kOwn], lane0 + (R * k + y) / kOwn);
                    const f32x2 tt = pair2(t, t);
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[y][e] = ptx::fma2(tt, c[e], o[y][e]);
                }
            }
        }
        // the segment after this one: its first page, then its first copies, are under way meanwhile
        const bool whole = w.whole();
        const int req = w.req;
        float *part = a.part + w.slot() * partial_floats(rows, D);
        go = w.next(a);
        if (go) first_page();
        {   // the groups of the warp
            float f[kOwn];
#pragma unroll
            for (int e = 0; e < kOwn; ++e) {
                float top = m[e];
#pragma unroll
                for (int x = LPK; x < 32; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
                f[e] = m[e] == -INFINITY ? 0.f : exp2f(m[e] - top);
                l[e] = (l[e] + __shfl_xor_sync(0xffffffffu, l[e], kSpread / 2)) * f[e];
#pragma unroll
                for (int x = LPK; x < 32; x <<= 1) l[e] += __shfl_xor_sync(0xffffffffu, l[e], x);
                if (lane < R / kOwn) {
                    s.m[warp][lane * kOwn + e] = top;
                    s.l[warp][lane * kOwn + e] = l[e];
                }
            }
#pragma unroll
            for (int y = 0; y < R; ++y) {
                const float g = __shfl_sync(0xffffffffu, f[y % kOwn], lane0 + y / kOwn);
                float e[8];
#pragma unroll
                for (int c = 0; c < 4; ++c) ptx::unpair2(o[y][c], e[2 * c], e[2 * c + 1]);
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    e[c] *= g;
#pragma unroll
                    for (int x = LPK; x < 32; x <<= 1) e[c] += __shfl_xor_sync(0xffffffffu, e[c], x);
                }
                if (lane < LPK) {
                    *reinterpret_cast<float4 *>(&s.o[warp][y][4 * sub]) = make_float4(e[0], e[1], e[2], e[3]);
                    *reinterpret_cast<float4 *>(&s.o[warp][y][4 * (sub + LPK)]) = make_float4(e[4], e[5], e[6], e[7]);
                }
            }
        }
        if (go) first_steps();
        __syncthreads();
        // the warps
        for (int x = tid; x < rows * D; x += kThreads) {
            const int rho = x / D, c = x % D;
            float top = s.m[0][rho], sum = 0.f, out = 0.f;
#pragma unroll
            for (int y = 1; y < kWarps; ++y) top = fmaxf(top, s.m[y][rho]);
            const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int y = 0; y < kWarps; ++y) {
                const float f = exp2f(s.m[y][rho] - base);
                sum = fmaf(f, s.l[y][rho], sum);
                out = fmaf(f, s.o[y][rho][c], out);
            }
            if (whole) {
                size_t to;
                if (row_at(a, req, u, rho, to)) static_cast<float *>(a.O)[to + c] = out / sum;
            } else {
                part[2 * rows + (size_t)c * rows + rho] = out;
                if (c == 0) {
                    part[rho] = top;
                    part[rows + rho] = sum;
                }
            }
        }
        __syncthreads();                                    // before the next segment's results
    }
    if (tid == 0) write_note(a, work, w, sh);
    write_empty<float, kThreads>(a, tid);
}

template <int D, int R> cudaError_t launch(const PagedArgs &a, cudaStream_t st)
{
    using S = Smem<D, R>;
    static std::atomic<unsigned long long> opted{0};
    const cudaError_t e = pipe::opt_in(reinterpret_cast<const void *>(&k_paged_attn_few<D, R>), (int)sizeof(S), opted);
    if (e != cudaSuccess) return e;
    int lg = 4;
    while ((1 << lg) < a.page_size) ++lg;
    return pipe::launch_early(k_paged_attn_few<D, R>, dim3(a.n_cta), dim3(kThreads), sizeof(S), st, a, lg);
}

}  // namespace

cudaError_t launch_paged_attn_few(const PagedArgs &a, cudaStream_t st)
{
    const bool four = a.Bt * a.Gt <= 4;
    if (a.d == 128) return four ? launch<128, 4>(a, st) : launch<128, 8>(a, st);
    return four ? launch<64, 4>(a, st) : launch<64, 8>(a, st);
}

}  // namespace hyb
