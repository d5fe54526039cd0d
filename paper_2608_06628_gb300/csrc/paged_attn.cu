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

    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    Walk w;
    Shares sh(0, 1);
    const bool work = find_share<kThreads>(a, s.plan, w, sh);
    const int M = units_per_request(a);
    while (work && w.next(a, M)) {
        const Visible vis = w.vis;
        const int i0 = w.i0, i1 = w.i1;
        const int req = w.req;
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
        float *part = a.part + w.slot() * partial_floats(rows, D);
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
    if (tid == 0) write_note(a, work, w, sh);
    write_empty<float, kThreads>(a, tid);
}

// Join: block x reads the note of boundary x and, if a unit is cut there for the
// first time, adds up the unit's partials; blocks along y take COLS features each.
// A thread has one row and every n-th feature; it loads references, sums and
// outputs of a partial together and merges them into its own (m, l, o), so that two
// rounds of loads (the note, then the partials) are all the latency.  Where a unit
// has few rows (decoding) it may have many partials: then groups of threads take
// every n-th one, and the groups are merged in order.  Launched programmatically
// behind the attention kernel.
constexpr int kMaxRows = 128;

// (m, l, o) <- (m, l, o) + (mi, li, oi): weights of both in units of the larger reference
struct Merge {
    float keep, add;
    __device__ Merge(float &m, float mi)
    {
        const float top = fmaxf(m, mi), base = top == -INFINITY ? 0.f : top;
        keep = exp2f(m - base);
        add = exp2f(mi - base);
        m = top;
    }
};

template <typename T, int COLS, int ROWS>
__global__ __launch_bounds__(kThreads) void k_paged_join(const PagedArgs a)
{
    constexpr int kIter = ROWS * COLS > kThreads ? ROWS * COLS / kThreads : 1;   // features per thread, at most
    constexpr int kOut = ROWS * (COLS + 1) > kThreads ? ROWS * (COLS + 1) : kThreads;
    __shared__ float s_o[kOut];                              // [row][COLS + 1], or one value a thread
    __shared__ float s_m[kThreads], s_l[kThreads];
    const int tid = threadIdx.x, rows = a.Bt * a.Gt, c = blockIdx.x, col0 = blockIdx.y * COLS;
    ptx::griddep_wait();
    const JoinNote note = a.notes[c];
    if (!note.cut) return;
    const size_t size = partial_floats(rows, a.d);
    const int n = note.last - c + 1;                         // partials
    auto part_of = [&](int i) { return a.part + (size_t)(i == 0 ? note.slot : 2 * (c + i)) * size; };

    const int rho = tid % rows, lane = tid / rows, lanes = kThreads / rows;   // threads of a row
    const int groups = lanes >= COLS ? lanes / COLS : 1, step = lanes >= COLS ? COLS : lanes;
    const int g = lane / step, first = lane % step;          // features first, first + step, ...
    float m = -INFINITY, l = 0.f, o[kIter];
#pragma unroll
    for (int k = 0; k < kIter; ++k) o[k] = 0.f;
    if (g < groups) {
#pragma unroll 2
        for (int i = g; i < n; i += groups) {
            const float *p = part_of(i);
            const float mi = p[rho], li = p[rows + rho];
            float v[kIter];
#pragma unroll
            for (int k = 0; k < kIter; ++k) {
                const int col = first + k * step;
                v[k] = col < COLS ? p[2 * rows + (size_t)(col0 + col) * rows + rho] : 0.f;
            }
            const Merge w(m, mi);
            l = l * w.keep + li * w.add;
#pragma unroll
            for (int k = 0; k < kIter; ++k) o[k] = o[k] * w.keep + v[k] * w.add;
        }
    }
    if (groups > 1) {                                        // one feature a thread
        s_m[tid] = m;
        s_l[tid] = l;
        s_o[tid] = o[0];
        __syncthreads();
        if (g == 0) {
            for (int y = 1; y < groups; ++y) {
                const int other = tid + y * COLS * rows;
                const Merge w(m, s_m[other]);
                l = l * w.keep + s_l[other] * w.add;
                o[0] = o[0] * w.keep + s_o[other] * w.add;
            }
        }
        __syncthreads();
    }
    if (g == 0) {
        const float inv = 1.f / l;
#pragma unroll
        for (int k = 0; k < kIter; ++k) {
            const int col = first + k * step;
            if (col < COLS) s_o[rho * (COLS + 1) + col] = o[k] * inv;
        }
    }
    __syncthreads();
    const Unit u = unit_of(a, note.m);
    for (int x = tid; x < rows * (COLS / 4); x += kThreads) {
        const int r = x / (COLS / 4), col = x % (COLS / 4) * 4;
        size_t at;
        if (!row_at(a, note.req, u, r, at)) continue;
        const float *v = s_o + r * (COLS + 1) + col;
        store4(static_cast<T *>(a.O) + at + col0 + col, make_float4(v[0], v[1], v[2], v[3]));
    }
}

// The join of a call whose attention kernel was launched just before.
template <typename T> cudaError_t launch_join(const PagedArgs &a, cudaStream_t st)
{
    // many partials of few rows: more blocks of fewer features, with little shared
    // memory, so that they are in place before the attention kernel ends
    const int rows = a.Bt * a.Gt;
    if (rows <= 16)
        return pipe::launch_early(k_paged_join<T, 16, 16>, dim3(a.n_cta, a.d / 16), dim3(kThreads), 0, st, a);
    return pipe::launch_early(k_paged_join<T, 32, kMaxRows>, dim3(a.n_cta, a.d / 32), dim3(kThreads), 0, st, a);
}

template <int D> cudaError_t launch_f32(const PagedArgs &a, cudaStream_t st)
{
    static_assert(sizeof(Smem<D>) < 100 * 1024, "two blocks per multiprocessor");
    cudaError_t e =
        cudaFuncSetAttribute(k_paged_attn<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Smem<D>));
    if (e != cudaSuccess) return e;
    e = pipe::launch_early(k_paged_attn<D>, dim3(a.n_cta), dim3(kThreads), sizeof(Smem<D>), st, a);
    if (e != cudaSuccess) return e;
    return launch_join<float>(a, st);
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

size_t paged_workspace_bytes(const PagedArgs &a)
{
    return (size_t)a.n_cta * sizeof(JoinNote) + (size_t)2 * a.n_cta * partial_floats(a.Bt * a.Gt, a.d) * sizeof(float);
}

void paged_set_workspace(PagedArgs &a, void *workspace)
{
    a.notes = static_cast<JoinNote *>(workspace);
    a.part = reinterpret_cast<float *>(a.notes + a.n_cta);
}

cudaError_t launch_paged_attn(hybrid_dtype dt, const PagedArgs &a, cudaStream_t st)
{
    if (dt == HYBRID_F32) return a.d == 128 ? launch_f32<128>(a, st) : launch_f32<64>(a, st);
    const cudaError_t e = launch_paged_attn_tc(a, st);
    if (e != cudaSuccess) return e;
    return launch_join<__nv_bfloat16>(a, st);
}

}  // namespace hyb
