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

__device__ __forceinline__ float4 load4(const float *p) { return *reinterpret_cast<const float4 *>(p); }
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
template <int D>
__global__ __launch_bounds__(kThreads) void k_paged_attn(const PagedArgs a)
{
    constexpr int kCols = D / 4, kRowStep = kThreads / kCols, kOwn = kRows / kRowStep;
    extern __shared__ __align__(16) unsigned char raw[];
    Smem<D> &s = *reinterpret_cast<Smem<D> *>(raw);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rows = a.Bt * a.Gt;
    const float to_log2 = pipe::kLog2e * rsqrtf((float)D);

    ptx::griddep_launch_dependents();                        // the join may start its scan
    const Plan plan = make_plan<kThreads>(a, s.plan);
    const long long M = units_per_request(a), T_all = plan.total * M;
    const int C = T_all < a.n_cta ? (int)T_all : a.n_cta;
    if ((int)blockIdx.x >= C) return;
    const long long t = share_start(T_all, C, blockIdx.x), t1 = share_start(T_all, C, blockIdx.x + 1);
    int req;
    long long before;
    locate(a, plan, t, s.plan, req, before);

    Walk w;
    w.begin(a, t, t1, req, before);
    while (w.next(a, M)) {
        const Visible vis = w.vis;
        const int i0 = w.i0, i1 = w.i1;
        req = w.req;
        const Unit u = unit_of(a, w.m);
        const int *pages = a.table + (size_t)req * a.max_pages;

        __syncthreads();                                     // the last segment's reads are done
        for (int x = tid; x < kRows * kCols; x += kThreads) {
            const int rho = x / kCols, c = x % kCols * 4;
            size_t at;
            const bool live = row_at(a, req, u, rho, at);
            *reinterpret_cast<float4 *>(&s.q[rho][c]) =
                live ? load4(static_cast<const float *>(a.Q) + at + c) : make_float4(0.f, 0.f, 0.f, 0.f);
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
                        k = load4(static_cast<const float *>(a.K) + at);
                        v = load4(static_cast<const float *>(a.V) + at);
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
        const bool whole = w.whole();
        float *part = a.part + (size_t)(2 * blockIdx.x + (w.at_start ? 0 : 1)) * partial_floats(rows, D);
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
                if (live) store4(static_cast<float *>(a.O) + at + col, c);
            } else {
                float *out = part + 2 * rows + (size_t)col * rows + rho;
                out[0] = c.x;
                out[rows] = c.y;
                out[2 * rows] = c.z;
                out[3 * rows] = c.w;
                if (col == 0) {
                    part[rho] = s.m[rho];
                    part[rows + rho] = s.l[rho];
                }
            }
        }
    }
}

// Join: block x looks at the boundary between shares x and x + 1.  If it cuts a
// unit, and is the first one to cut it, the block joins all of the unit's
// partials; blocks along y take kJoinCols features each.  Where a unit has few
// rows (decoding) and so may have many partials, groups of threads take every
// n-th partial and are added in order.  Requests without a visible key get their
// zeros here, shared over the blocks.  Launched programmatically behind the
// attention kernel: the scan over the requests overlaps its end.
constexpr int kJoinCols = 32;
constexpr int kMaxRows = 128;

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void k_paged_join(const PagedArgs a)
{
    __shared__ PlanSmem s_plan;
    __shared__ float s_base[kMaxRows], s_inv[kMaxRows];
    __shared__ float s_o[kMaxRows * (kJoinCols + 1)];        // [group][row][kJoinCols + 1]
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rows = a.Bt * a.Gt;
    const int col0 = blockIdx.y * kJoinCols;
    const Plan plan = make_plan<kThreads>(a, s_plan);
    const long long M = units_per_request(a), T_all = plan.total * M;
    const int C = T_all < a.n_cta ? (int)T_all : a.n_cta;
    const int c = blockIdx.x;
    int req = 0, last = 0;
    Unit u{};
    const float *first = nullptr;
    bool cut_here = false;
    if (c + 1 < C) {
        const long long cut = share_start(T_all, C, c + 1);
        long long before;
        locate(a, plan, cut, s_plan, req, before);
        const Visible vis = visible_keys(a, a.lens[req]);
        const int m = (int)((cut - before * M) / vis.tiles);
        const long long mine = share_start(T_all, C, c), start = before * M + (long long)m * vis.tiles;
        cut_here = cut != start && mine <= start;
        if (cut_here) {
            last = c + 1;                                    // block of the unit's last tile
            while (share_start(T_all, C, last + 1) < start + vis.tiles) ++last;
            u = unit_of(a, m);
            first = a.part + (size_t)(2 * c + (mine != start)) * partial_floats(rows, D);
        }
    }
    ptx::griddep_wait();
    for (int r = blockIdx.x; r < a.n_req; r += gridDim.x) {
        if (visible_keys(a, a.lens[r]).tiles > 0) continue;
        T *out = static_cast<T *>(a.O) + (size_t)r * a.B * a.Hq * D;
        const int n = a.B * a.Hq * D / 4;
        for (int x = blockIdx.y * kThreads + tid; x < n; x += gridDim.y * kThreads)
            store4(out + (size_t)x * 4, make_float4(0.f, 0.f, 0.f, 0.f));
    }
    if (!cut_here) return;
    const size_t size = partial_floats(rows, D);
    auto part_of = [&](int b) { return b == c ? first : a.part + (size_t)2 * b * size; };

    // maximum and sum of each row: warp = row, lanes over the partials
    for (int rho = warp; rho < rows; rho += kThreads / 32) {
        float mx = -INFINITY;
        for (int b = c + lane; b <= last; b += 32) mx = fmaxf(mx, part_of(b)[rho]);
        mx = warp_max(mx);
        const float base = mx == -INFINITY ? 0.f : mx;
        float l = 0.f;
        for (int b = c + lane; b <= last; b += 32) l = fmaf(exp2f(part_of(b)[rho] - base), part_of(b)[rows + rho], l);
        l = warp_sum(l);
        if (lane == 0) {
            s_base[rho] = base;
            s_inv[rho] = 1.f / l;
        }
    }
    __syncthreads();
    // sums over the partials; item = (feature, row), row fastest as in memory
    const int items = rows * kJoinCols, groups = items <= kThreads / 2 ? kThreads / items : 1;
    const int step = groups > 1 ? items * groups : kThreads;
    for (int x = tid; x < items * groups; x += step) {
        const int item = x % items, g = x / items, rho = item % rows, col = item / rows;
        const float base = s_base[rho];
        float o = 0.f;
#pragma unroll 4
        for (int b = c + g; b <= last; b += groups) {
            const float *p = part_of(b);
            o = fmaf(exp2f(p[rho] - base), p[2 * rows + (size_t)(col0 + col) * rows + rho], o);
        }
        s_o[(g * rows + rho) * (kJoinCols + 1) + col] = o;
    }
    __syncthreads();
    for (int x = tid; x < rows * (kJoinCols / 4); x += kThreads) {
        const int rho = x / (kJoinCols / 4), col = x % (kJoinCols / 4) * 4;
        size_t at;
        if (!row_at(a, req, u, rho, at)) continue;
        float o[4] = {0.f, 0.f, 0.f, 0.f};
        for (int g = 0; g < groups; ++g) {
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] += s_o[(g * rows + rho) * (kJoinCols + 1) + col + i];
        }
        const float f = s_inv[rho];
        store4(static_cast<T *>(a.O) + at + col0 + col, make_float4(o[0] * f, o[1] * f, o[2] * f, o[3] * f));
    }
}

// The join of a call whose attention kernel was launched just before.
template <typename T, int D> cudaError_t launch_join(const PagedArgs &a, cudaStream_t st)
{
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3(a.n_cta, D / kJoinCols);
    lc.blockDim = dim3(kThreads);
    lc.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = attr;
    lc.numAttrs = 1;
    return cudaLaunchKernelEx(&lc, k_paged_join<T, D>, a);
}

template <int D> cudaError_t launch_f32(const PagedArgs &a, cudaStream_t st)
{
    static_assert(sizeof(Smem<D>) < 100 * 1024, "two blocks per multiprocessor");
    PagedArgs b = a;
    void *args[] = {&b};
    const void *f = reinterpret_cast<const void *>(&k_paged_attn<D>);
    cudaError_t e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Smem<D>));
    if (e != cudaSuccess) return e;
    e = cudaLaunchKernel(f, dim3(a.n_cta), dim3(kThreads), args, sizeof(Smem<D>), st);
    if (e != cudaSuccess) return e;
    return launch_join<float, D>(a, st);
}

}  // namespace

void paged_geometry(const hybrid_cfg &c, PagedArgs &a)
{
    const bool tc = c.io_dtype == HYBRID_BF16;
    const int max_rows = tc ? kMaxRows : kRows;
    a.B = c.block_size;
    a.Hq = c.n_q_heads;
    a.Hkv = c.n_kv_heads;
    a.G = c.n_q_heads / c.n_kv_heads;
    a.d = c.head_dim;
    a.Gt = a.G < max_rows ? a.G : max_rows;
    a.n_gt = (a.G + a.Gt - 1) / a.Gt;
    a.Bt = max_rows / a.Gt < a.B ? max_rows / a.Gt : a.B;
    a.n_bt = (a.B + a.Bt - 1) / a.Bt;
    a.n_cta = (tc ? 1 : 2) * pipe::sm_count();
}

size_t paged_partial_bytes(const PagedArgs &a)
{
    return (size_t)2 * a.n_cta * partial_floats(a.Bt * a.Gt, a.d) * sizeof(float);
}

cudaError_t launch_paged_attn(hybrid_dtype dt, const PagedArgs &a, cudaStream_t st)
{
    if (dt == HYBRID_F32) return a.d == 128 ? launch_f32<128>(a, st) : launch_f32<64>(a, st);
    const cudaError_t e = launch_paged_attn_tc(a, st);
    if (e != cudaSuccess) return e;
    return a.d == 128 ? launch_join<__nv_bfloat16, 128>(a, st) : launch_join<__nv_bfloat16, 64>(a, st);
}

}  // namespace hyb
