// paged_attn.cu -- attention over the paged cache on the CUDA cores (float32),
// and the join of the requests that were split (hybrid_paged_attn).
//
// Per row: running maximum m, sum l and output O over the visible keys, in one
// pass; scores are kept in units of log2, x = q . k log2(e) / sqrt(d).
//
// A block of 8 warps takes the tiles of its share (paged_plan.cuh) one after another,
// 64 rows x 128 keys (rows beyond the tile's are zeros: checks in the loops cost more).
// For the scores a thread has 8 rows x 4 keys (12 16-byte reads of shared memory for 64
// packed FMAs), for O 4 rows x 8 features (the same), with all keys at d = 128 and every
// second 64 of them at d = 64, added at a segment's end.  K, V and P have one buffer each:
// K of the next tile comes while P V is computed, V while the scores are; masked keys are
// zero-filled, their pages not read.  A row's maximum is moved only when a score exceeds
// it by more than 8, which the block votes on, so that a tile takes three barriers and no
// reduction; sums are added over the threads at a segment's end.  Row tiles of up to 8
// rows: paged_attn_few.cu.
//
// Bound by reads of shared memory and the FMA pipe in turn (about 60% of the peak of
// each): 64 requests of 256-8192 tokens, blocks of 32, 16 query and 4 key heads, d = 128
// 1530 us (47 TFLOP/s), d = 64 848 us; with 8 rows x 2 keys and 4 x 4 to a thread, and a
// maximum of each row found for each tile, 2440 us.
#include "paged_plan.cuh"
#include "tc_pipeline.cuh"

namespace hyb {
namespace {

using namespace paged;
using ptx::f32x2;
using ptx::pair2;

constexpr int kThreads = 256;
constexpr int kRows = 64;                       // rows of a tile
constexpr int kPitchP = kTile + 8;              // 4 rows x 8 keys written by a warp meet 32 banks
constexpr float kSlack = 8.f;

template <typename T> __device__ __forceinline__ void store4(T *p, float4 v);
template <> __device__ __forceinline__ void store4<float>(float *p, float4 v) { *reinterpret_cast<float4 *>(p) = v; }
template <> __device__ __forceinline__ void store4<__nv_bfloat16>(__nv_bfloat16 *p, float4 v)
{
    *reinterpret_cast<uint2 *>(p) = make_uint2(pipe::pack_bf16x2(v.x, v.y), pipe::pack_bf16x2(v.z, v.w));
}

template <int D> struct Smem {
    static constexpr int kPitch = D + 4;        // 16-byte reads of 8 keys, or 4 rows, meet 32 banks
    float q[kRows][kPitch];
    float k[kTile][kPitch];
    float v[kTile][D];
    float p[kRows][kPitchP];
    float sum[kRows][4], top[kRows][4];         // of a row, by the warps that share it
    float m[kRows], scale[kRows];
    PlanSmem plan;
};

template <int D> __global__ __launch_bounds__(kThreads, 1) void k_paged_attn(const PagedArgs a, int page_lg)
{
    using S = Smem<D>;
    constexpr int kCols = D / 4, kKeyStep = 32 / kCols;     // copies of a warp: 16 bytes of kKeyStep keys at a time
    constexpr int kOwnKeys = kTile / 8;                     // keys that a warp copies, side by side: of one page
    extern __shared__ __align__(16) unsigned char raw[];
    S &s = *reinterpret_cast<S *>(raw);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rows = a.Bt * a.Gt;
    const float to_log2 = pipe::kLog2e * rsqrtf((float)D);

    // scores: rows row_s + 8 y, keys key_s + 8 x
    const int row_s = lane / 8 + 4 * (warp & 1), key_s = lane % 8 + 32 * (warp >> 1);
    // outputs: rows row_o + 16 y, features col_o + 32 x + (0 ... 3); half of the keys (d = 64)
    const int row_o = lane / 8 + 4 * (warp & 3), half = warp >> 2;
    const int col_o = lane % 8 * 4 + (D == 128 ? 64 * half : 0);
    constexpr int kKeysO = D == 128 ? kTile : kTile / 2;
    const int key_o = D == 128 ? 0 : half * kKeysO;

    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    Walk w;
    Shares sh(0, 1);
    const bool work = find_share<kThreads>(a, s.plan, w, sh);
    if (work) {
        // the tile to copy next: segment and tile, and this warp's page
        Walk ahead = w;
        int i = 0, page = 0;
        bool more = ahead.next(a);
        i = ahead.i0;
        auto look_up = [&]() {                              // the page of this warp's keys
            const int j = key_tile(ahead.vis, i) * kTile + warp * kOwnKeys;
            page = 0;
            if (more && any_visible(ahead.vis, j, kOwnKeys))
                page = __ldg(a.table + (size_t)ahead.req * a.max_pages + (j >> page_lg));
        };
        auto copy_q = [&]() {
            const Unit u = unit_of(a, ahead.head, ahead.rt);
            for (int x = tid; x < kRows * kCols; x += kThreads) {
                const int rho = x / kCols, c = x % kCols * 4;
                size_t from;
                const bool live = row_at(a, ahead.req, u, rho, from);
                copy16(&s.q[rho][c], static_cast<const float *>(a.Q) + (live ? from + c : 0), live ? 16 : 0);
            }
        };
        // this warp's keys of a tile to shared memory
        auto copy_tile = [&](const Visible &vis, int tile, size_t from, const void *cache, float *to, int pitch) {
            const int j0 = key_tile(vis, tile) * kTile + warp * kOwnKeys + lane / kCols, c = lane % kCols * 4;
            const float *src = static_cast<const float *>(cache) + from + c;
            float *dst = to + (size_t)(warp * kOwnKeys + lane / kCols) * pitch + c;
            const int in_page = j0 & ((1 << page_lg) - 1);
#pragma unroll
            for (int x = 0; x < kOwnKeys; x += kKeyStep) {
                const bool see = key_visible(vis, j0 + x);
                copy16(dst + x * pitch, see ? src + (in_page + x) * D : static_cast<const float *>(cache), see ? 16 : 0);
            }
        };
        auto from_page = [&]() {
            if (page < 0 || page >= a.n_pages) {
                raise_error(a.err, ERR_BAD_INDEX);
                page = 0;
            }
            return (((size_t)page * a.Hkv + ahead.head) << page_lg) * D;
        };
        auto commit = [&]() { asm volatile("cp.async.commit_group;" ::: "memory"); };

        size_t from = 0;
        Visible vis_v{};                                    // of the tile whose values are to be copied
        int i_v = 0;
        look_up();
        if (more) {
            from = from_page();
            copy_q();
            copy_tile(ahead.vis, i, from, a.K, &s.k[0][0], S::kPitch);
            commit();
            copy_tile(ahead.vis, i, from, a.V, &s.v[0][0], D);
        }
        commit();
        asm volatile("cp.async.wait_group 1;" ::: "memory");
        __syncthreads();
        while (w.next(a)) {
            const Unit u = unit_of(a, w.head, w.rt);
            float m[8], l[8];                               // of this thread's rows; its own keys' sum
            f32x2 o[4][4];
#pragma unroll
            for (int y = 0; y < 8; ++y) {
                m[y] = -INFINITY;
                l[y] = 0.f;
            }
#pragma unroll
            for (int y = 0; y < 4; ++y)
#pragma unroll
                for (int x = 0; x < 4; ++x) o[y][x] = pair2(0.f, 0.f);
            for (int tile = w.i0; tile < w.i1; ++tile) {
                // the next tile to copy
                bool segment = false;
                if (++i >= ahead.i1) {
                    more = ahead.next(a);
                    segment = more;
                    i = ahead.i0;
                }
                look_up();
                float x[8][4];
                {
                    f32x2 acc[8][4];
#pragma unroll
                    for (int y = 0; y < 8; ++y)
#pragma unroll
                        for (int k = 0; k < 4; ++k) acc[y][k] = pair2(0.f, 0.f);
#pragma unroll 2
                    for (int c = 0; c < D; c += 4) {
                        f32x2 k0[4], k1[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) load_pairs(&s.k[key_s + 8 * k][c], k0[k], k1[k]);
#pragma unroll
                        for (int y = 0; y < 8; ++y) {
                            f32x2 q0, q1;
                            load_pairs(&s.q[row_s + 8 * y][c], q0, q1);
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                acc[y][k] = ptx::fma2(k1[k], q1, ptx::fma2(k0[k], q0, acc[y][k]));
                        }
                    }
                    const int j = key_tile(w.vis, tile) * kTile + key_s;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const bool see = key_visible(w.vis, j + 8 * k);
#pragma unroll
                        for (int y = 0; y < 8; ++y) {
                            float lo, hi;
                            ptx::unpair2(acc[y][k], lo, hi);
                            x[y][k] = see ? (lo + hi) * to_log2 : -INFINITY;
                        }
                    }
                }
                bool above = false;
#pragma unroll
                for (int y = 0; y < 8; ++y)
#pragma unroll
                    for (int k = 0; k < 4; ++k) above |= x[y][k] > m[y] + kSlack;
                const bool moved = __syncthreads_or(above);     // also: K and Q have been read
                vis_v = ahead.vis;
                i_v = i;
                if (more) {
                    from = from_page();
                    if (segment) copy_q();
                    copy_tile(vis_v, i_v, from, a.K, &s.k[0][0], S::kPitch);
                }
                commit();
                if (moved) {
#pragma unroll
                    for (int y = 0; y < 8; ++y) {
                        float t = fmaxf(fmaxf(x[y][0], x[y][1]), fmaxf(x[y][2], x[y][3]));
#pragma unroll
                        for (int f = 4; f > 0; f >>= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, f));
                        if (lane % 8 == 0) s.top[row_s + 8 * y][warp >> 1] = t;
                    }
                    __syncthreads();
#pragma unroll
                    for (int y = 0; y < 8; ++y) {
                        const float4 t = *reinterpret_cast<const float4 *>(s.top[row_s + 8 * y]);
                        const float all = fmaxf(fmaxf(t.x, t.y), fmaxf(t.z, t.w));
                        const float now = all > m[y] + kSlack ? all : m[y];
                        const float f = m[y] == -INFINITY ? 1.f : exp2f(m[y] - now);    // (l and O are zero, or NaN)
                        m[y] = now;
                        l[y] *= f;
                        if (lane % 8 == 0 && warp < 2) s.scale[row_s + 8 * y] = f;
                    }
                }
#pragma unroll
                for (int y = 0; y < 8; ++y) {
                    const float base = m[y] == -INFINITY ? 0.f : m[y];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float p = exp2f(x[y][k] - base);
                        l[y] += p;
                        s.p[row_s + 8 * y][key_s + 8 * k] = p;
                    }
                }
                asm volatile("cp.async.wait_group 1;" ::: "memory");
                __syncthreads();                            // P and V are in place
                if (moved) {
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        const float f = s.scale[row_o + 16 * y];
                        const f32x2 ff = pair2(f, f);
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[y][e] = ptx::mul2(o[y][e], ff);
                    }
                }
#pragma unroll 4
                for (int r = 0; r < kKeysO; r += 4) {
                    f32x2 v[4][4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float *at = &s.v[key_o + r + k][col_o];
                        load_pairs(at, v[k][0], v[k][1]);
                        load_pairs(at + 32, v[k][2], v[k][3]);
                    }
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        const float4 p4 = *reinterpret_cast<const float4 *>(&s.p[row_o + 16 * y][key_o + r]);
                        const float p[4] = {p4.x, p4.y, p4.z, p4.w};
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const f32x2 pp = pair2(p[k], p[k]);
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[y][e] = ptx::fma2(pp, v[k][e], o[y][e]);
                        }
                    }
                }
                asm volatile("cp.async.wait_group 0;" ::: "memory");
                __syncthreads();                            // the next K and Q are in place, V and P have been read
                if (more) copy_tile(vis_v, i_v, from, a.V, &s.v[0][0], D);
                commit();
            }
            // the segment's output
#pragma unroll
            for (int y = 0; y < 8; ++y) {
#pragma unroll
                for (int f = 4; f > 0; f >>= 1) l[y] += __shfl_xor_sync(0xffffffffu, l[y], f);
                if (lane % 8 == 0) {
                    s.sum[row_s + 8 * y][warp >> 1] = l[y];
                    if (warp < 2) s.m[row_s + 8 * y] = m[y];
                }
            }
            if (D == 64 && half == 1) {
#pragma unroll
                for (int y = 0; y < 4; ++y)
#pragma unroll
                    for (int e = 0; e < 4; e += 2) {
                        ulonglong2 t;
                        t.x = o[y][e].v;
                        t.y = o[y][e + 1].v;
                        *reinterpret_cast<ulonglong2 *>(&s.p[row_o + 16 * y][col_o + 16 * e]) = t;
                    }
            }
            __syncthreads();
            if (D == 128 || half == 0) {
                const bool whole = w.whole();
                float *part = a.part + w.slot() * partial_floats(rows, D);
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const int rho = row_o + 16 * y;
                    if (rho >= rows) break;
                    const float4 t = *reinterpret_cast<const float4 *>(s.sum[rho]);
                    const float sum = (t.x + t.y) + (t.z + t.w), f = 1.f / sum;
                    size_t to;
                    const bool live = row_at(a, w.req, u, rho, to);
#pragma unroll
                    for (int e = 0; e < 4; e += 2) {
                        const int col = col_o + 16 * e;
                        if (D == 64) {
                            f32x2 b0, b1;
                            load_pairs(&s.p[rho][col], b0, b1);
                            o[y][e] = ptx::add2(o[y][e], b0);
                            o[y][e + 1] = ptx::add2(o[y][e + 1], b1);
                        }
                        float4 c;
                        ptx::unpair2(o[y][e], c.x, c.y);
                        ptx::unpair2(o[y][e + 1], c.z, c.w);
                        if (whole) {
                            if (live)
                                store4(static_cast<float *>(a.O) + to + col, make_float4(c.x * f, c.y * f, c.z * f, c.w * f));
                        } else {
                            float *out = part + 2 * rows + (size_t)col * rows + rho;
                            out[0] = c.x;
                            out[rows] = c.y;
                            out[2 * rows] = c.z;
                            out[3 * rows] = c.w;
                        }
                    }
                    if (!whole && col_o == 0) {
                        part[rho] = s.m[rho];
                        part[rows + rho] = sum;
                    }
                }
            }
        }
    }
    if (tid == 0) write_note(a, work, w, sh);
    write_empty<float, kThreads>(a, tid);
}

// Join: block x reads the note of boundary x and, if a unit is cut there for the
// first time, adds up the unit's partials; blocks along y take kJoinCols features each.
// A thread has one row and some of the features; it loads references, sums and
// outputs of a partial together and merges them into its own (m, l, o), so that two
// rounds of loads (the note, then the partials) are all the latency.  Launched
// programmatically behind the attention kernel.
constexpr int kMaxRows = 128;
constexpr int kJoinCols = 16;

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

// At most 16 rows (decoding): a unit may have many partials, so groups of kJoinCols
// threads a row, one feature each, take every n-th one, and the groups are merged in
// order.
template <typename T> __global__ __launch_bounds__(kThreads) void k_paged_join_few(const PagedArgs a)
{
    constexpr int kPitch = kJoinCols + 1;
    __shared__ float s_o[16 * kPitch];                       // one value a thread, then [row][kPitch]
    __shared__ float s_m[kThreads], s_l[kThreads];
    static_assert(16 * kPitch >= kThreads, "a value of each thread");
    const int tid = threadIdx.x, rows = a.Bt * a.Gt, c = blockIdx.x, col0 = blockIdx.y * kJoinCols;
    ptx::griddep_wait();
    const JoinNote note = a.notes[c];
    if (!note.cut) return;
    const size_t size = partial_floats(rows, a.d);
    const int n = note.last - c + 1;                         // partials
    const int rho = tid % rows, lane = tid / rows, groups = kThreads / rows / kJoinCols;
    const int g = lane / kJoinCols, col = lane % kJoinCols;
    float m = -INFINITY, l = 0.f, o = 0.f;
    if (g < groups) {
        constexpr int kLoad = 4;                             // partials loaded at a time
        for (int i0 = g; i0 < n; i0 += kLoad * groups) {
            float mi[kLoad], li[kLoad], v[kLoad];
#pragma unroll
            for (int x = 0; x < kLoad; ++x) {
                const int i = i0 + x * groups;
                const float *p = a.part + (size_t)(i == 0 ? 2 * c + 1 : 2 * (c + i)) * size + rho;
                mi[x] = i < n ? p[0] : -INFINITY;
                li[x] = i < n ? p[rows] : 0.f;
                v[x] = i < n ? p[(2 + col0 + col) * rows] : 0.f;
            }
#pragma unroll
            for (int x = 0; x < kLoad; ++x) {
                if (i0 + x * groups >= n) break;
                const Merge w(m, mi[x]);
                l = l * w.keep + li[x] * w.add;
                o = o * w.keep + v[x] * w.add;
            }
        }
    }
    if (groups > 1) {
        s_m[tid] = m;
        s_l[tid] = l;
        s_o[tid] = o;
        __syncthreads();
        if (g == 0) {
            for (int y = 1; y < groups; ++y) {
                const int other = tid + y * kJoinCols * rows;
                const Merge w(m, s_m[other]);
                l = l * w.keep + s_l[other] * w.add;
                o = o * w.keep + s_o[other] * w.add;
            }
        }
        __syncthreads();
    }
    if (g == 0) s_o[rho * kPitch + col] = o / l;
    __syncthreads();
    const Unit u = unit_of(a, note.head, note.rt);
    for (int x = tid; x < rows * (kJoinCols / 4); x += kThreads) {
        const int r = x / (kJoinCols / 4), at_col = x % (kJoinCols / 4) * 4;
        size_t at;
        if (!row_at(a, note.req, u, r, at)) continue;
        const float *v = s_o + r * kPitch + at_col;
        store4(static_cast<T *>(a.O) + at + col0 + at_col, make_float4(v[0], v[1], v[2], v[3]));
    }
}

// More than 16 rows: kJoinCols / FEAT threads to a row, each with FEAT features side by
// side, which it writes itself; two partials at a time, as most units have, so that five
// blocks are in place on a multiprocessor.  (Four partials at a time and the output by way
// of shared memory, three blocks: blocks of 32 tokens for 64 requests 104 us, here 100.)
template <typename T, int FEAT> __global__ __launch_bounds__(kThreads, 4) void k_paged_join_many(const PagedArgs a)
{
    constexpr int kSpan = kThreads * FEAT / kJoinCols;       // rows
    const int rows = a.Bt * a.Gt, rho = threadIdx.x % kSpan, c = blockIdx.x;
    const int col = blockIdx.y * kJoinCols + threadIdx.x / kSpan * FEAT;
    ptx::griddep_wait();
    const JoinNote note = a.notes[c];
    if (!note.cut || rho >= rows) return;
    const size_t size = partial_floats(rows, a.d);
    const int n = note.last - c + 1;                         // partials
    float m = -INFINITY, l = 0.f, o[FEAT];
#pragma unroll
    for (int k = 0; k < FEAT; ++k) o[k] = 0.f;
    for (int i0 = 0; i0 < n; i0 += 2) {
        float mi[2], li[2], v[2][FEAT];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int i = i0 + x;
            const float *p = a.part + (size_t)(i == 0 ? 2 * c + 1 : 2 * (c + i)) * size + rho;
            mi[x] = i < n ? p[0] : -INFINITY;
            li[x] = i < n ? p[rows] : 0.f;
#pragma unroll
            for (int k = 0; k < FEAT; ++k) v[x][k] = i < n ? p[(2 + col + k) * rows] : 0.f;
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            if (i0 + x >= n) break;
            const Merge w(m, mi[x]);
            l = l * w.keep + li[x] * w.add;
#pragma unroll
            for (int k = 0; k < FEAT; ++k) o[k] = o[k] * w.keep + v[x][k] * w.add;
        }
    }
    size_t at;
    if (!row_at(a, note.req, unit_of(a, note.head, note.rt), rho, at)) return;
    const float inv = 1.f / l;
#pragma unroll
    for (int k = 0; k < FEAT; ++k) o[k] *= inv;
    T *out = static_cast<T *>(a.O) + at + col;
    if constexpr (FEAT == 2) {
        if constexpr (sizeof(T) == 4) *reinterpret_cast<float2 *>(out) = make_float2(o[0], o[1]);
        else *reinterpret_cast<uint32_t *>(out) = pipe::pack_bf16x2(o[0], o[1]);
    } else if constexpr (FEAT == 8 && sizeof(T) == 2) {
        *reinterpret_cast<uint4 *>(out) = make_uint4(pipe::pack_bf16x2(o[0], o[1]), pipe::pack_bf16x2(o[2], o[3]),
                                                     pipe::pack_bf16x2(o[4], o[5]), pipe::pack_bf16x2(o[6], o[7]));
    } else {
#pragma unroll
        for (int k = 0; k < FEAT; k += 4) store4(out + k, make_float4(o[k], o[k + 1], o[k + 2], o[k + 3]));
    }
}

// The join of a call whose attention kernel was launched just before; none where no
// unit can be cut (one block, or contexts of one tile at most).
template <typename T> cudaError_t launch_join(const PagedArgs &a, cudaStream_t st)
{
    if (a.n_cta == 1 || a.max_pages * a.page_size <= kTile) return cudaSuccess;
    const dim3 grid(a.n_cta, a.d / kJoinCols), block(kThreads);
    const int rows = a.Bt * a.Gt;
    if (rows <= 16) return pipe::launch_early(k_paged_join_few<T>, grid, block, 0, st, a);
    if (rows <= 32) return pipe::launch_early(k_paged_join_many<T, 2>, grid, block, 0, st, a);
    if (rows <= 64) return pipe::launch_early(k_paged_join_many<T, 4>, grid, block, 0, st, a);
    return pipe::launch_early(k_paged_join_many<T, 8>, grid, block, 0, st, a);
}

template <int D> cudaError_t launch_f32(const PagedArgs &a, cudaStream_t st)
{
    int lg = 4;
    while ((1 << lg) < a.page_size) ++lg;
    static std::atomic<unsigned long long> opted{0};
    const cudaError_t e = pipe::opt_in(reinterpret_cast<const void *>(&k_paged_attn<D>), (int)sizeof(Smem<D>), opted);
    if (e != cudaSuccess) return e;
    return pipe::launch_early(k_paged_attn<D>, dim3(a.n_cta), dim3(kThreads), sizeof(Smem<D>), st, a, lg);
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
        // The kernel of paged_attn_few.cu also for a few row tiles: 64 requests of 256-8192
        // tokens, 4 key heads, d = 128, here 786 us for any rows up to 64, there four tiles
        // of 8 rows 650 us, five 813, six 969 (one request of 777 tokens: 25 us here, 14
        // there).
        cut_rows(a, kFewestRows);
        if (a.n_gt * a.n_bt > 5) cut_rows(a, kRows);
    }
    const int rows = a.Bt * a.Gt;
    a.extra = tc && rows <= 64 ? 3 : 7;
    a.n_cta = (tc || rows > 4 ? 1 : 2) * pipe::sm_count();   // resident blocks
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
