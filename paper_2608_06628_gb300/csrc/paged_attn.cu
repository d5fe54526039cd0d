// paged_attn.cu -- attention over the paged cache on the CUDA cores (float32),
// and the join of the requests that were split (hybrid_paged_attn).
//
// Per row: running maximum m, sum l and output O over the visible keys, in one
// pass; scores are kept in units of log2, x = q . k log2(e) / sqrt(d).
#include "paged_plan.cuh"
#include "tc_pipeline.cuh"

namespace hyb {
namespace {

using namespace paged;

constexpr int kThreads = 256;
constexpr int kRows = 16;       // rows of a tile
constexpr int kKeys = 64;       // keys in shared memory at a time

template <typename T> __device__ __forceinline__ float4 load4(const T *p);
template <> __device__ __forceinline__ float4 load4<float>(const float *p) { return *reinterpret_cast<const float4 *>(p); }
template <> __device__ __forceinline__ float4 load4<__nv_bfloat16>(const __nv_bfloat16 *p)
{
    const uint2 v = *reinterpret_cast<const uint2 *>(p);
    return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16),
                       __uint_as_float(v.y & 0xffff0000u));
}
template <typename T> __device__ __forceinline__ void store4(T *p, float4 v);
template <> __device__ __forceinline__ void store4<float>(float *p, float4 v) { *reinterpret_cast<float4 *>(p) = v; }
template <> __device__ __forceinline__ void store4<__nv_bfloat16>(__nv_bfloat16 *p, float4 v)
{
    *reinterpret_cast<uint2 *>(p) = make_uint2(pipe::pack_bf16x2(v.x, v.y), pipe::pack_bf16x2(v.z, v.w));
}

template <int D> struct Smem {
    float q[kRows][D];
    float k[kKeys][D + 4];      // rows 16 bytes apart modulo 128: a warp's 16-byte reads of 32 keys do not collide
    float v[kKeys][D];
    float p[kRows][kKeys];
    float m[kRows], l[kRows], scale[kRows];
    PlanSmem plan;
};

// Output columns: thread = 4 columns (tid % (D/4)) of rows tid / (D/4) + i * kRowStep.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void k_paged_attn(const PagedArgs a)
{
    constexpr int kCols = D / 4, kRowStep = kThreads / kCols, kOwn = kRows / kRowStep;
    extern __shared__ __align__(16) unsigned char raw[];
    Smem<D> &s = *reinterpret_cast<Smem<D> *>(raw);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rows = a.Bt * a.Gt;
    const float to_log2 = pipe::kLog2e * rsqrtf((float)D);

    const Plan plan = make_plan<kThreads>(a, s.plan);
    const long long M = units_per_request(a), T_all = plan.total * M;
    const int C = T_all < a.n_cta ? (int)T_all : a.n_cta;
    if ((int)blockIdx.x >= C) return;
    long long t = share_start(T_all, C, blockIdx.x);
    const long long t0 = t, t1 = share_start(T_all, C, blockIdx.x + 1);
    int req;
    long long before;
    locate(a, plan, t, s.plan, req, before);

    while (t < t1) {
        Visible vis = visible_keys(a, a.lens[req]);
        while (t >= (before + vis.tiles) * M) {             // next request with visible keys
            before += vis.tiles;
            vis = visible_keys(a, a.lens[++req]);
        }
        const long long rel = t - before * M;
        const int m = (int)(rel / vis.tiles), i0 = (int)(rel % vis.tiles);
        const int i1 = (int)(vis.tiles - i0 < t1 - t ? vis.tiles : i0 + (t1 - t));
        const Unit u = unit_of(a, m);
        const int *pages = a.table + (size_t)req * a.max_pages;

        __syncthreads();                                     // the last segment's reads are done
        for (int x = tid; x < kRows * kCols; x += kThreads) {
            const int rho = x / kCols, c = x % kCols * 4;
            size_t at;
            const bool live = row_at(a, req, u, rho, at);
            *reinterpret_cast<float4 *>(&s.q[rho][c]) =
                live ? load4(static_cast<const T *>(a.Q) + at + c) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
        if (tid < kRows) {
            s.m[tid] = -INFINITY;
            s.l[tid] = 0.f;
        }
        float4 o[kOwn];
#pragma unroll
        for (int i = 0; i < kOwn; ++i) o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        const int col = tid % kCols * 4, row0 = tid / kCols;

        for (int i = i0; i < i1; ++i) {
            const int tile = key_tile(vis, i);
#pragma unroll 1
            for (int half = 0; half < kTile / kKeys; ++half) {
                const int j0 = tile * kTile + half * kKeys;
                if (j0 >= vis.len) break;
                __syncthreads();                             // keys and values free
                for (int x = tid; x < kKeys * kCols; x += kThreads) {
                    const int r = x / kCols, c = x % kCols * 4, j = j0 + r;
                    float4 k = make_float4(0.f, 0.f, 0.f, 0.f), v = k;
                    if (key_visible(vis, j)) {
                        int page = pages[j / a.page_size];
                        if (page < 0 || page >= a.n_pages) {
                            raise_error(a.err, ERR_BAD_INDEX);
                            page = 0;
                        }
                        const size_t at =
                            (((size_t)page * a.Hkv + u.head) * a.page_size + j % a.page_size) * D + c;
                        k = load4(static_cast<const T *>(a.K) + at);
                        v = load4(static_cast<const T *>(a.V) + at);
                    }
                    *reinterpret_cast<float4 *>(&s.k[r][c]) = k;
                    *reinterpret_cast<float4 *>(&s.v[r][c]) = v;
                }
                __syncthreads();
                {   // scores: thread = one key, four rows
                    const int r = tid % kKeys, g = tid / kKeys * 4;
                    float acc[4] = {0.f, 0.f, 0.f, 0.f};
                    if (g < rows) {
#pragma unroll 8
                        for (int c = 0; c < D; c += 4) {
                            const float4 k = *reinterpret_cast<const float4 *>(&s.k[r][c]);
#pragma unroll
                            for (int y = 0; y < 4; ++y) {
                                const float4 q = *reinterpret_cast<const float4 *>(&s.q[g + y][c]);
                                acc[y] = fmaf(k.x, q.x, acc[y]);
                                acc[y] = fmaf(k.y, q.y, acc[y]);
                                acc[y] = fmaf(k.z, q.z, acc[y]);
                                acc[y] = fmaf(k.w, q.w, acc[y]);
                            }
                        }
                    }
                    const bool see = key_visible(vis, j0 + r);
#pragma unroll
                    for (int y = 0; y < 4; ++y) s.p[g + y][r] = see ? acc[y] * to_log2 : -INFINITY;
                }
                __syncthreads();
                // softmax: warp = two rows
                for (int rho = warp * 2; rho < warp * 2 + 2; ++rho) {
                    const float x0 = s.p[rho][lane], x1 = s.p[rho][lane + 32];
                    const float old = s.m[rho], now = fmaxf(old, warp_max(fmaxf(x0, x1)));
                    const float base = now == -INFINITY ? 0.f : now;
                    const float p0 = exp2f(x0 - base), p1 = exp2f(x1 - base);
                    const float sum = warp_sum(p0 + p1), f = exp2f(old - base);
                    s.p[rho][lane] = p0;
                    s.p[rho][lane + 32] = p1;
                    __syncwarp();
                    if (lane == 0) {
                        s.m[rho] = now;
                        s.l[rho] = s.l[rho] * f + sum;
                        s.scale[rho] = f;
                    }
                }
                __syncthreads();
#pragma unroll
                for (int y = 0; y < kOwn; ++y) {
                    const int rho = row0 + y * kRowStep;
                    if (rho >= rows) break;
                    const float f = s.scale[rho];
                    float4 c = o[y];
                    c.x *= f;
                    c.y *= f;
                    c.z *= f;
                    c.w *= f;
#pragma unroll 8
                    for (int r = 0; r < kKeys; ++r) {
                        const float4 v = *reinterpret_cast<const float4 *>(&s.v[r][col]);
                        const float p = s.p[rho][r];
                        c.x = fmaf(p, v.x, c.x);
                        c.y = fmaf(p, v.y, c.y);
                        c.z = fmaf(p, v.z, c.z);
                        c.w = fmaf(p, v.w, c.w);
                    }
                    o[y] = c;
                }
            }
        }
        const bool whole = i0 == 0 && i1 == vis.tiles;
        float *part = a.part + (size_t)(2 * blockIdx.x + (t != t0)) * partial_floats(rows, D);
#pragma unroll
        for (int y = 0; y < kOwn; ++y) {
            const int rho = row0 + y * kRowStep;
            if (rho >= rows) break;
            size_t at;
            const bool live = row_at(a, req, u, rho, at);
            float4 c = o[y];
            if (whole) {
                const float f = 1.f / s.l[rho];
                c.x *= f;
                c.y *= f;
                c.z *= f;
                c.w *= f;
                if (live) store4(static_cast<T *>(a.O) + at + col, c);
            } else {
                float *out = part + 2 * rows + (size_t)rho * D + col;
                out[0] = c.x;
                out[1] = c.y;
                out[2] = c.z;
                out[3] = c.w;
                if (col == 0) {
                    part[rho] = s.m[rho];
                    part[rows + rho] = s.l[rho];
                }
            }
        }
        t += i1 - i0;
    }
}

// Join: block x looks at the boundary between shares x and x + 1.  If it cuts a
// unit, and is the first one to cut it, the block joins all of the unit's
// partials, in their order; blocks along y take kJoinRows rows each.  Requests
// without a visible key get their zeros here, shared over the blocks.
constexpr int kJoinRows = 4;

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void k_paged_join(const PagedArgs a)
{
    __shared__ PlanSmem s_plan;
    const int tid = threadIdx.x, rows = a.Bt * a.Gt;
    const Plan plan = make_plan<kThreads>(a, s_plan);
    for (int r = blockIdx.x; r < a.n_req; r += gridDim.x) {
        if (visible_keys(a, a.lens[r]).tiles > 0) continue;
        T *out = static_cast<T *>(a.O) + (size_t)r * a.B * a.Hq * D;
        const int n = a.B * a.Hq * D / 4;
        for (int x = blockIdx.y * kThreads + tid; x < n; x += gridDim.y * kThreads)
            store4(out + (size_t)x * 4, make_float4(0.f, 0.f, 0.f, 0.f));
    }
    const long long M = units_per_request(a), T_all = plan.total * M;
    const int C = T_all < a.n_cta ? (int)T_all : a.n_cta;
    const int c = blockIdx.x;
    if (c + 1 >= C) return;
    const long long cut = share_start(T_all, C, c + 1);
    int req;
    long long before;
    locate(a, plan, cut, s_plan, req, before);
    const Visible vis = visible_keys(a, a.lens[req]);
    const long long rel = cut - before * M;
    const int m = (int)(rel / vis.tiles);
    const long long start = before * M + (long long)m * vis.tiles, end = start + vis.tiles;
    if (cut == start || share_start(T_all, C, c) > start) return;
    int last = c + 1;                                        // block of the unit's last tile
    while (share_start(T_all, C, last + 1) < end) ++last;
    const Unit u = unit_of(a, m);
    const size_t size = partial_floats(rows, D);
    const float *first = a.part + (size_t)(2 * c + (share_start(T_all, C, c) != start)) * size;

    constexpr int kCols = D / 4;
    for (int x = tid; x < kJoinRows * kCols; x += kThreads) {
        const int rho = blockIdx.y * kJoinRows + x / kCols, col = x % kCols * 4;
        size_t at;
        if (rho >= rows || !row_at(a, req, u, rho, at)) continue;
        float mx = first[rho];
        for (int b = c + 1; b <= last; ++b) mx = fmaxf(mx, a.part[(size_t)2 * b * size + rho]);
        const float base = mx == -INFINITY ? 0.f : mx;
        float l = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int b = c; b <= last; ++b) {
            const float *p = b == c ? first : a.part + (size_t)2 * b * size;
            const float f = exp2f(p[rho] - base);
            l = fmaf(f, p[rows + rho], l);
            const float *po = p + 2 * rows + (size_t)rho * D + col;
            o.x = fmaf(f, po[0], o.x);
            o.y = fmaf(f, po[1], o.y);
            o.z = fmaf(f, po[2], o.z);
            o.w = fmaf(f, po[3], o.w);
        }
        const float f = 1.f / l;
        store4(static_cast<T *>(a.O) + at + col, make_float4(o.x * f, o.y * f, o.z * f, o.w * f));
    }
}

template <typename T, int D> cudaError_t launch(const PagedArgs &a, cudaStream_t st)
{
    static_assert(sizeof(Smem<D>) < 100 * 1024, "two blocks per multiprocessor");
    PagedArgs b = a;
    void *args[] = {&b};
    const void *f = reinterpret_cast<const void *>(&k_paged_attn<T, D>);
    cudaError_t e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Smem<D>));
    if (e != cudaSuccess) return e;
    e = cudaLaunchKernel(f, dim3(a.n_cta), dim3(kThreads), args, sizeof(Smem<D>), st);
    if (e != cudaSuccess) return e;
    const int rows = a.Bt * a.Gt;
    return cudaLaunchKernel(reinterpret_cast<const void *>(&k_paged_join<T, D>),
                            dim3(a.n_cta, (rows + kJoinRows - 1) / kJoinRows), dim3(kThreads), args, 0, st);
}

}  // namespace

void paged_geometry(const hybrid_cfg &c, PagedArgs &a)
{
    const int max_rows = kRows;
    a.B = c.block_size;
    a.Hq = c.n_q_heads;
    a.Hkv = c.n_kv_heads;
    a.G = c.n_q_heads / c.n_kv_heads;
    a.d = c.head_dim;
    a.Gt = a.G < max_rows ? a.G : max_rows;
    a.n_gt = (a.G + a.Gt - 1) / a.Gt;
    a.Bt = max_rows / a.Gt < a.B ? max_rows / a.Gt : a.B;
    a.n_bt = (a.B + a.Bt - 1) / a.Bt;
    a.n_cta = 2 * pipe::sm_count();
}

size_t paged_partial_bytes(const PagedArgs &a)
{
    return (size_t)2 * a.n_cta * partial_floats(a.Bt * a.Gt, a.d) * sizeof(float);
}

cudaError_t launch_paged_attn(hybrid_dtype dt, const PagedArgs &a, cudaStream_t st)
{
    if (dt == HYBRID_BF16)
        return a.d == 128 ? launch<__nv_bfloat16, 128>(a, st) : launch<__nv_bfloat16, 64>(a, st);
    return a.d == 128 ? launch<float, 128>(a, st) : launch<float, 64>(a, st);
}

}  // namespace hyb
