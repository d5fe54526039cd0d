// paged_attn_quant_few.cu -- attention over the 8-bit paged cache on the CUDA cores, row tiles of
// at most 8 rows (hybrid_paged_attn_quant): float32 queries.
//
// As paged_attn_few.cu, with codes instead of values: a lane copies 8 features of a key (8 bytes) and
// decodes them where it uses them (exact, by way of half precision).  The scales stay out of the
// products: with ks, vs those of a key's group of 16,
//     x = (q . codes) ks log2(e) / sqrt(d),   p = 2^(x - m),   l += p,   o += (p vs) codes
// A warp's run of 16 keys in a tile is one group, so it has two scales a tile, copied with its
// codes.
#include "paged_plan.cuh"
#include "quant.cuh"
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

static_assert(kRun == HYBRID_QUANT_TOKENS, "two scales a run");

// 8 codes as pairs of float32
__device__ __forceinline__ void decode8(const uint2 &v, f32x2 (&c)[4])
{
    float lo[4], hi[4];
    quant::decode4(v.x, lo);
    quant::decode4(v.y, hi);
    c[0] = pair2(lo[0], lo[1]);
    c[1] = pair2(lo[2], lo[3]);
    c[2] = pair2(hi[0], hi[1]);
    c[3] = pair2(hi[2], hi[3]);
}
__device__ __forceinline__ void copy8(void *dst, const uint8_t *src, int bytes)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(ptx::smem_u32(dst)), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy4(void *dst, const float *src, int bytes)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(ptx::smem_u32(dst)), "l"(src), "r"(bytes) : "memory");
}

template <typename T> __device__ __forceinline__ void load8(const T *p, f32x2 (&c)[4]);
template <> __device__ __forceinline__ void load8(const float *p, f32x2 (&c)[4])
{
    load_pairs(p, c[0], c[1]);
    load_pairs(p + 4, c[2], c[3]);
}
template <> __device__ __forceinline__ void load8(const __nv_bfloat16 *p, f32x2 (&c)[4])
{
    const uint4 v = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = pair2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}

template <int D, int R> struct Smem {
    static constexpr int kStages = 4;
    static constexpr int kScales = 8;                       // tiles whose scales are in flight or in use
    uint2 ring[kWarps][kStages][2 * kKeys][32];             // K, then V
    float scales[kWarps][kScales][2];
    float o[kWarps][R][D];
    float m[kWarps][R], l[kWarps][R];
    PlanSmem plan;
};

template <typename T, int D, int R>
__global__ __launch_bounds__(kThreads, R == 4 ? 2 : 1) void k_paged_attn_quant_few(const PagedArgs a, int page_lg)
{
    constexpr int kStages = Smem<D, R>::kStages, kScales = Smem<D, R>::kScales;
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
    uint2 (*ring)[2 * kKeys][32] = s.ring[warp];
    const uint8_t *K = static_cast<const uint8_t *>(a.K), *V = static_cast<const uint8_t *>(a.V);

    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    Walk w;
    Shares sh(0, 1);
    const bool work = find_share<kThreads>(a, s.plan, w, sh);
    bool go = work && w.next(a);
    // the copies, of the segment w: tile, step within it, stage
    int i = 0, at = 0, slot = 0, to_scale = 0;
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
                run = (((size_t)page * a.Hkv + w.head) << page_lg) + (key & ((1 << page_lg) - 1));
                if (lane < 2) {
                    const bool see = any_visible(w.vis, key - group, kRun);
                    copy4(&s.scales[warp][to_scale][lane], (lane ? a.V_scale : a.K_scale) + (see ? run / kRun : 0), see ? 4 : 0);
                }
                to_scale = to_scale + 1 == kScales ? 0 : to_scale + 1;
                run = run * D + 8 * sub;
                look_up(i + 1);
            }
#pragma unroll
            for (int x = 0; x < kKeys; ++x) {
                const int step = (kKeys * at + x) * SLOTS;
                const bool see = key_visible(w.vis, key + step);
                const size_t from = see ? run + step * D : 0;   // masked keys and values are zeros
                seen = 2 * seen + see;
                copy8(&ring[slot][x][lane], K + from, see ? 8 : 0);
                copy8(&ring[slot][kKeys + x][lane], V + from, see ? 8 : 0);
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
        at = slot = to_scale = 0;
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
                load8(static_cast<const T *>(a.Q) + from + 8 * sub, q[y]);
            }
        }
        float m[kOwn], l[kOwn];                             // of rows kOwn sub % R ...; l of this lane's key
#pragma unroll
        for (int e = 0; e < kOwn; ++e) {
            m[e] = -INFINITY;
            l[e] = 0.f;
        }
        const int steps = (w.i1 - w.i0) * kSteps;
        float ks = 0.f, vs = 0.f;                           // of the run; log2(e) / sqrt(d) in ks
        for (int n = 0, b = 0; n < steps; ++n, b = b + 1 == kStages ? 0 : b + 1) {
            fetch();                                        // into the stage of the step before
            asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
            if (n % kSteps == 0) {
                __syncwarp();                               // the scales are other lanes' copies
                const float2 both = *reinterpret_cast<const float2 *>(s.scales[warp][n / kSteps % kScales]);
                ks = both.x * to_log2;
                vs = both.y;
            }
            float x[kProducts];
#pragma unroll
            for (int k = 0; k < kKeys; ++k) {
                f32x2 c[4];
                decode8(ring[b][k][lane], c);
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
                x[e] = see ? x[e] * ks : -INFINITY;
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
                x[e] *= vs;
            }
#pragma unroll
            for (int k = 0; k < kKeys; ++k) {
                f32x2 c[4];
                decode8(ring[b][kKeys + k][lane], c);
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
                    *reinterpret_cast<float4 *>(&s.o[warp][y][8 * sub]) = make_float4(e[0], e[1], e[2], e[3]);
                    *reinterpret_cast<float4 *>(&s.o[warp][y][8 * sub + 4]) = make_float4(e[4], e[5], e[6], e[7]);
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
                if (row_at(a, req, u, rho, to)) static_cast<T *>(a.O)[to + c] = from_f32<T>(out / sum);
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
    write_empty<T, kThreads>(a, tid);
}

template <typename T, int D, int R> cudaError_t launch(const PagedArgs &a, cudaStream_t st)
{
    using S = Smem<D, R>;
    static std::atomic<unsigned long long> opted{0};
    const cudaError_t e = pipe::opt_in(reinterpret_cast<const void *>(&k_paged_attn_quant_few<T, D, R>), (int)sizeof(S), opted);
    if (e != cudaSuccess) return e;
    int lg = 4;
    while ((1 << lg) < a.page_size) ++lg;
    return pipe::launch_early(k_paged_attn_quant_few<T, D, R>, dim3(a.n_cta), dim3(kThreads), sizeof(S), st, a, lg);
}
template <typename T> cudaError_t launch(const PagedArgs &a, cudaStream_t st)
{
    const bool four = a.Bt * a.Gt <= 4;
    if (a.d == 128) return four ? launch<T, 128, 4>(a, st) : launch<T, 128, 8>(a, st);
    return four ? launch<T, 64, 4>(a, st) : launch<T, 64, 8>(a, st);
}

}  // namespace

void paged_quant_geometry(const hybrid_cfg &c, PagedArgs &a)
{
    a.B = c.block_size;
    a.Hq = c.n_q_heads;
    a.Hkv = c.n_kv_heads;
    a.G = c.n_q_heads / c.n_kv_heads;
    a.d = c.head_dim;
    paged_cut_rows(a, kFewestRows);
    a.extra = 7;
    a.n_cta = (a.Bt * a.Gt > 4 ? 1 : 2) * pipe::sm_count();  // resident blocks
}

cudaError_t launch_paged_attn_quant(hybrid_dtype dt, const PagedArgs &a, cudaStream_t st)
{
    const cudaError_t e = dt == HYBRID_BF16 ? launch<__nv_bfloat16>(a, st) : launch<float>(a, st);
    return e != cudaSuccess ? e : launch_paged_join(dt, a, st);
}

}  // namespace hyb
