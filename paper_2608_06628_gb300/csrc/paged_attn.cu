// paged_attn.cu -- attention over the paged cache on the CUDA cores (float32),
// and the join of the requests that were split (hybrid_paged_attn).
//
// Per row: running maximum m, sum l and output O over the visible keys, in one
// pass; scores are kept in units of log2, x = q . k log2(e) / sqrt(d).
//
// A block of 8 warps walks its share of the tiles (paged_plan.cuh) in chunks of 64
// (d = 64) or 32 keys, copied by cp.async one or two chunks ahead, across requests; masked
// keys are zero-filled, their pages not read.  For the scores a lane has its keys
// (row pitch d + 4 floats: 16-byte reads of 8 keys do not collide) and a warp every
// eighth row, so maximum, sum and probabilities of a row stay in one warp's
// registers; for O a thread has 4 features of every (1024 / d)-th row.  16 rows to a
// tile where a key head has no more, else 64, so that each key read from shared memory
// meets 8 rows (bound by the FMA pipe).  Up to 8 rows: paged_attn_few.cu.
#include <type_traits>

#include "paged_plan.cuh"
#include "tc_pipeline.cuh"

namespace hyb {
namespace {

using namespace paged;
using ptx::f32x2;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kFewRows = 16, kManyRows = 64;    // rows of a tile

__device__ __forceinline__ float4 load4(const float *p) { return *reinterpret_cast<const float4 *>(p); }
template <typename T> __device__ __forceinline__ void store4(T *p, float4 v);
template <> __device__ __forceinline__ void store4<float>(float *p, float4 v) { *reinterpret_cast<float4 *>(p) = v; }
template <> __device__ __forceinline__ void store4<__nv_bfloat16>(__nv_bfloat16 *p, float4 v)
{
    *reinterpret_cast<uint2 *>(p) = make_uint2(pipe::pack_bf16x2(v.x, v.y), pipe::pack_bf16x2(v.z, v.w));
}
// 16 bytes of shared memory as two pairs
__device__ __forceinline__ void load_pairs(const float *p, f32x2 &a, f32x2 &b)
{
    const ulonglong2 v = *reinterpret_cast<const ulonglong2 *>(p);
    a.v = v.x;
    b.v = v.y;
}

// 16 bytes to shared memory, `bytes` of them read and the rest zeros
__device__ __forceinline__ void copy16(uint32_t dst, const float *src, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

template <int D, int ROWS> struct Smem {
    static constexpr int kKeys = D == 64 ? 64 : 32;
    static constexpr int kStages = ROWS == kFewRows ? 3 : 2;   // chunks in place or on their way
    float q[ROWS][D];
    struct {
        float k[kKeys][D + 4];
        float v[kKeys][D];
    } chunk[kStages];
    float p[ROWS][kKeys];
    float m[ROWS], l[ROWS], scale[ROWS];
    PlanSmem plan;
};

// The chunks of a block's share, those without a visible key left out.
template <int KEYS> struct Chunks {
    Walk w;
    int i, j0;             // tile of the segment, first key
    bool live;

    __device__ void begin(const PagedArgs &a, const Walk &walk)
    {
        w = walk;
        live = w.next(a);
        if (!live) return;
        i = w.i0;
        j0 = key_tile(w.vis, i) * kTile;
        skip(a);
    }
    // Advance; true if the chunk is the first of a segment.
    __device__ bool step(const PagedArgs &a)
    {
        j0 += KEYS;
        return skip(a);
    }
    __device__ bool skip(const PagedArgs &a)
    {
        bool first = false;
        while (true) {
            if (j0 < (key_tile(w.vis, i) + 1) * kTile) {
                if (any_visible(w.vis, j0, KEYS)) return first;
                j0 += KEYS;
                continue;
            }
            if (++i == w.i1) {
                first = true;
                live = w.next(a);
                if (!live) return first;
                i = w.i0;
            }
            j0 = key_tile(w.vis, i) * kTile;
        }
    }
};

template <int D, int ROWS>
__global__ __launch_bounds__(kThreads, 2) void k_paged_attn(const PagedArgs a, int page_lg)
{
    using S = Smem<D, ROWS>;
    constexpr int KEYS = S::kKeys, KL = KEYS / 32, RW = ROWS / kWarps;      // keys of a lane, rows of a warp
    constexpr int kCols = D / 4, kRowStep = kThreads / kCols;               // O: threads per row, rows at a time
    constexpr int kOwn = ROWS / kRowStep;                                   // rows of a thread
    constexpr int kCopies = KEYS * kCols / kThreads;                        // 16-byte copies of K per thread
    extern __shared__ __align__(16) unsigned char raw[];
    S &s = *reinterpret_cast<S *>(raw);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rows = a.Bt * a.Gt;
    const float to_log2 = pipe::kLog2e * rsqrtf((float)D);

    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    Walk w;
    Shares sh(0, 1);
    const bool work = find_share<kThreads>(a, s.plan, w, sh);
    if (work) {
        const int col = tid % kCols * 4, row0 = tid / kCols;
        Chunks<KEYS> at, ahead;
        at.begin(a, w);
        ahead = at;
        auto issue = [&](int b) {
            if (ahead.live) {
                const int *pages = a.table + (size_t)ahead.w.req * a.max_pages;
                // this thread's 16 bytes of a key in the cache, from its page
                auto in_cache = [&](int j) {
                    int page = __ldg(pages + (j >> page_lg));
                    if (page < 0 || page >= a.n_pages) {
                        raise_error(a.err, ERR_BAD_INDEX);
                        page = 0;
                    }
                    return ((((size_t)page * a.Hkv + ahead.w.head) << page_lg) + (j & ((1 << page_lg) - 1))) * D + col;
                };
                const uint32_t to_k = ptx::smem_u32(&s.chunk[b].k[row0][col]), to_v = ptx::smem_u32(&s.chunk[b].v[row0][col]);
                if (ahead.j0 >= ahead.w.vis.lo && ahead.j0 + KEYS <= ahead.w.vis.len) {
                    // all keys visible: a page is looked up once for 16 keys in a row
                    constexpr int kRun = 16 / kRowStep > 1 ? 16 / kRowStep : 1;
#pragma unroll
                    for (int x = 0; x < kCopies; x += kRun) {
                        const size_t from = in_cache(ahead.j0 + row0 + x * kRowStep);
#pragma unroll
                        for (int y = 0; y < kRun; ++y) {
                            copy16(to_k + (x + y) * kRowStep * (D + 4) * 4,
                                   static_cast<const float *>(a.K) + from + y * kRowStep * D, 16);
                            copy16(to_v + (x + y) * kRowStep * D * 4,
                                   static_cast<const float *>(a.V) + from + y * kRowStep * D, 16);
                        }
                    }
                } else {
#pragma unroll 1
                    for (int x = 0; x < kCopies; ++x) {
                        const int j = ahead.j0 + row0 + x * kRowStep;
                        const bool see = key_visible(ahead.w.vis, j);
                        const size_t from = see ? in_cache(j) : 0;
                        const int bytes = see ? 16 : 0;      // masked keys are zero-filled
                        copy16(to_k + x * kRowStep * (D + 4) * 4, static_cast<const float *>(a.K) + from, bytes);
                        copy16(to_v + x * kRowStep * D * 4, static_cast<const float *>(a.V) + from, bytes);
                    }
                }
                ahead.step(a);
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        constexpr int kAhead = S::kStages - 1;
#pragma unroll
        for (int x = 0; x < kAhead; ++x) issue(x);
        bool first = true;
        float m[RW], l[RW];                                  // of rows warp + 8 y
        float4 o[kOwn];                                      // features col ... of rows row0 + y kRowStep
        Unit u{};
        for (int b = 0; at.live; b = b + 1 == S::kStages ? 0 : b + 1) {
            const int req = at.w.req;
            issue(b == 0 ? kAhead : b - 1);
            if (first) {
                u = unit_of(a, at.w.head, at.w.rt);
                for (int x = tid; x < rows * kCols; x += kThreads) {
                    const int rho = x / kCols, c = x % kCols * 4;
                    size_t from;
                    const bool live = row_at(a, req, u, rho, from);
                    *reinterpret_cast<float4 *>(&s.q[rho][c]) =
                        live ? load4(static_cast<const float *>(a.Q) + from + c) : make_float4(0.f, 0.f, 0.f, 0.f);
                }
#pragma unroll
                for (int y = 0; y < RW; ++y) {
                    m[y] = -INFINITY;
                    l[y] = 0.f;
                }
#pragma unroll
                for (int y = 0; y < kOwn; ++y) o[y] = make_float4(0.f, 0.f, 0.f, 0.f);
            }
            asm volatile("cp.async.wait_group %0;" ::"n"(kAhead) : "memory");
            __syncthreads();
            {   // scores of keys lane, lane + 32 with rows warp, warp + 8, ...
                f32x2 acc[KL][RW];
#pragma unroll
                for (int x = 0; x < KL; ++x)
#pragma unroll
                    for (int y = 0; y < RW; ++y) acc[x][y] = ptx::pair2(0.f, 0.f);
                auto products = [&](auto full) {
#pragma unroll 4
                    for (int c = 0; c < D; c += 4) {
                        f32x2 k0[KL], k1[KL];
#pragma unroll
                        for (int x = 0; x < KL; ++x) load_pairs(&s.chunk[b].k[lane + 32 * x][c], k0[x], k1[x]);
#pragma unroll
                        for (int y = 0; y < RW; ++y) {
                            if (!full && warp + 8 * y >= rows) break;
                            f32x2 q0, q1;
                            load_pairs(&s.q[warp + 8 * y][c], q0, q1);
#pragma unroll
                            for (int x = 0; x < KL; ++x)
                                acc[x][y] = ptx::fma2(k1[x], q1, ptx::fma2(k0[x], q0, acc[x][y]));
                        }
                    }
                };
                // (a full tile without the checks of each row)
                if (rows == ROWS) products(std::true_type{});
                else if (warp < rows) products(std::false_type{});
                bool see[KL];
#pragma unroll
                for (int x = 0; x < KL; ++x) see[x] = key_visible(at.w.vis, at.j0 + lane + 32 * x);
#pragma unroll
                for (int y = 0; y < RW; ++y) {
                    const int rho = warp + 8 * y;
                    if (rho >= rows) break;
                    float x[KL], mx = -INFINITY, sum = 0.f;
#pragma unroll
                    for (int k = 0; k < KL; ++k) {
                        float lo, hi;
                        ptx::unpair2(acc[k][y], lo, hi);
                        x[k] = see[k] ? (lo + hi) * to_log2 : -INFINITY;
                        mx = fmaxf(mx, x[k]);
                    }
                    const float now = fmaxf(m[y], warp_max(mx)), base = now == -INFINITY ? 0.f : now;
#pragma unroll
                    for (int k = 0; k < KL; ++k) {
                        const float p = exp2f(x[k] - base);
                        s.p[rho][lane + 32 * k] = p;
                        sum += p;
                    }
                    const float f = exp2f(m[y] - base);
                    l[y] = l[y] * f + warp_sum(sum);
                    m[y] = now;
                    if (lane == 0) {
                        s.scale[rho] = f;
                        s.m[rho] = now;
                        s.l[rho] = l[y];
                    }
                }
            }
            __syncthreads();
            {   // O <- O scale + P V
                f32x2 acc[kOwn][2];
#pragma unroll
                for (int y = 0; y < kOwn; ++y) {
                    const int rho = row0 + y * kRowStep;
                    const float f = rho < rows ? s.scale[rho] : 0.f;
                    acc[y][0] = ptx::pair2(o[y].x * f, o[y].y * f);
                    acc[y][1] = ptx::pair2(o[y].z * f, o[y].w * f);
                }
                auto products = [&](auto full) {
#pragma unroll 2
                    for (int r = 0; r < KEYS; r += 4) {
                        f32x2 v[4][2];
#pragma unroll
                        for (int k = 0; k < 4; ++k) load_pairs(&s.chunk[b].v[r + k][col], v[k][0], v[k][1]);
#pragma unroll
                        for (int y = 0; y < kOwn; ++y) {
                            const int rho = row0 + y * kRowStep;
                            if (!full && y > 0 && rho >= rows) break;
                            const float4 p4 = load4(&s.p[rho][r]);
                            const float p[4] = {p4.x, p4.y, p4.z, p4.w};
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const f32x2 pp = ptx::pair2(p[k], p[k]);
                                acc[y][0] = ptx::fma2(pp, v[k][0], acc[y][0]);
                                acc[y][1] = ptx::fma2(pp, v[k][1], acc[y][1]);
                            }
                        }
                    }
                };
                if (rows == ROWS) products(std::true_type{});
                else if (row0 < rows) products(std::false_type{});
#pragma unroll
                for (int y = 0; y < kOwn; ++y) {
                    ptx::unpair2(acc[y][0], o[y].x, o[y].y);
                    ptx::unpair2(acc[y][1], o[y].z, o[y].w);
                }
            }
            const Walk here = at.w;
            first = at.step(a);
            if (first) {                                     // the segment's output
                const bool whole = here.whole();
                float *part = a.part + here.slot() * partial_floats(rows, D);
#pragma unroll
                for (int y = 0; y < kOwn; ++y) {
                    const int rho = row0 + y * kRowStep;
                    if (rho >= rows) break;
                    size_t to;
                    const bool live = row_at(a, req, u, rho, to);
                    const float4 c = o[y];
                    if (whole) {
                        const float f = 1.f / s.l[rho];
                        if (live)
                            store4(static_cast<float *>(a.O) + to + col, make_float4(c.x * f, c.y * f, c.z * f, c.w * f));
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
            __syncthreads();                                 // the chunk, Q and P may be overwritten
        }
        w = at.w;
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
    auto part_of = [&](int i) { return a.part + (size_t)(i == 0 ? 2 * c + 1 : 2 * (c + i)) * size; };

    const int rho = tid % rows, lane = tid / rows, lanes = kThreads / rows;   // threads of a row
    const int groups = lanes >= COLS ? lanes / COLS : 1, step = lanes >= COLS ? COLS : lanes;
    const int g = lane / step, first = lane % step;          // features first, first + step, ...
    float m = -INFINITY, l = 0.f, o[kIter];
#pragma unroll
    for (int k = 0; k < kIter; ++k) o[k] = 0.f;
    if (g < groups) {
        constexpr int kLoad = 4;                             // partials loaded at a time
        for (int i0 = g; i0 < n; i0 += kLoad * groups) {
            float mi[kLoad], li[kLoad], v[kLoad][kIter];
#pragma unroll
            for (int x = 0; x < kLoad; ++x) {
                const int i = i0 + x * groups;
                const float *p = part_of(i < n ? i : i0);
                mi[x] = i < n ? p[rho] : -INFINITY;
                li[x] = p[rows + rho];
#pragma unroll
                for (int k = 0; k < kIter; ++k) {
                    const int col = first + k * step;
                    v[x][k] = i < n && col < COLS ? p[2 * rows + (size_t)(col0 + col) * rows + rho] : 0.f;
                }
            }
#pragma unroll
            for (int x = 0; x < kLoad; ++x) {
                if (i0 + x * groups >= n) break;
                const Merge w(m, mi[x]);
                l = l * w.keep + li[x] * w.add;
#pragma unroll
                for (int k = 0; k < kIter; ++k) o[k] = o[k] * w.keep + v[x][k] * w.add;
            }
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
    const Unit u = unit_of(a, note.head, note.rt);
    for (int x = tid; x < rows * (COLS / 4); x += kThreads) {
        const int r = x / (COLS / 4), col = x % (COLS / 4) * 4;
        size_t at;
        if (!row_at(a, note.req, u, r, at)) continue;
        const float *v = s_o + r * (COLS + 1) + col;
        store4(static_cast<T *>(a.O) + at + col0 + col, make_float4(v[0], v[1], v[2], v[3]));
    }
}

// The join of a call whose attention kernel was launched just before; none where no
// unit can be cut (one block, or contexts of one tile at most).
template <typename T> cudaError_t launch_join(const PagedArgs &a, cudaStream_t st)
{
    if (a.n_cta == 1 || a.max_pages * a.page_size <= kTile) return cudaSuccess;
    // few rows: little shared memory, so that the blocks are in place before the
    // attention kernel ends
    const int rows = a.Bt * a.Gt;
    if (rows <= 16)
        return pipe::launch_early(k_paged_join<T, 16, 16>, dim3(a.n_cta, a.d / 16), dim3(kThreads), 0, st, a);
    return pipe::launch_early(k_paged_join<T, 16, kMaxRows>, dim3(a.n_cta, a.d / 16), dim3(kThreads), 0, st, a);
}

template <int D, int ROWS> cudaError_t launch_f32(const PagedArgs &a, cudaStream_t st)
{
    using S = Smem<D, ROWS>;
    static_assert(sizeof(S) < 113 * 1024, "two blocks per multiprocessor");
    int lg = 4;
    while ((1 << lg) < a.page_size) ++lg;
    static std::atomic<unsigned long long> opted{0};
    cudaError_t e = pipe::opt_in(reinterpret_cast<const void *>(&k_paged_attn<D, ROWS>), (int)sizeof(S), opted);
    if (e != cudaSuccess) return e;
    return pipe::launch_early(k_paged_attn<D, ROWS>, dim3(a.n_cta), dim3(kThreads), sizeof(S), st, a, lg);
}

template <int D> cudaError_t launch_f32(const PagedArgs &a, cudaStream_t st)
{
    return a.Bt * a.Gt <= kFewRows ? launch_f32<D, kFewRows>(a, st) : launch_f32<D, kManyRows>(a, st);
}

}  // namespace

// Row tiles of at most `most` rows, of about equal size along the tokens.
static void cut_rows(PagedArgs &a, int most)
{
    a.Gt = a.G < most ? a.G : most;
    a.n_gt = (a.G + a.Gt - 1) / a.Gt;
    a.Bt = most / a.Gt < a.B ? most / a.Gt : a.B;
    a.n_bt = (a.B + a.Bt - 1) / a.Bt;
    a.Bt = (a.B + a.n_bt - 1) / a.n_bt;
}

void paged_geometry(const hybrid_cfg &c, PagedArgs &a)
{
    const bool tc = c.io_dtype == HYBRID_BF16;
    a.B = c.block_size;
    a.Hq = c.n_q_heads;
    a.Hkv = c.n_kv_heads;
    a.G = c.n_q_heads / c.n_kv_heads;
    a.d = c.head_dim;
    if (tc) {
        cut_rows(a, kMaxRows);
    } else {
        // The kernel of paged_attn_few.cu also for two row tiles, but not for three: 64
        // requests of 256-8192 tokens, 4 key heads, d = 128, 16 rows 425 us against 539
        // here (d = 64 230 and 292), 15 rows as three times 5 628 against 548.
        cut_rows(a, kFewestRows);
        if (a.n_gt * a.n_bt > 2) cut_rows(a, a.G * a.B <= kFewRows ? kFewRows : kManyRows);
    }
    const int rows = a.Bt * a.Gt;
    a.extra = tc && rows <= 64 ? 3 : 7;
    a.n_cta = (tc || (rows > 4 && rows <= kFewestRows) ? 1 : 2) * pipe::sm_count();   // resident blocks
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
    const bool bf16 = dt == HYBRID_BF16;
    const int rows = a.Bt * a.Gt;
    cudaError_t e;
    if (bf16) e = launch_paged_attn_tc(a, st);
    else if (rows <= kFewestRows) e = launch_paged_attn_few(a, st);
    else e = a.d == 128 ? launch_f32<128>(a, st) : launch_f32<64>(a, st);
    if (e != cudaSuccess) return e;
    return bf16 ? launch_join<__nv_bfloat16>(a, st) : launch_join<float>(a, st);
}

}  // namespace hyb
