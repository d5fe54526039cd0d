// qk_norm_rope.cu -- norm of each query and key head with the rotary position
// in the same pass, into dense outputs or the paged cache, and its gradient
// (hybrid_qk_norm_rope, _cache, _backward).
//
// For a head x of d features, r = (mean x^2 + eps)^(-1/2), xh = x r, n = w xh:
//     y = R(t) n,   (a, b) -> scale (a cos t - b sin t, b cos t + a sin t)
// and backwards, with dn = R(t)^T dy (the rotation by -t) and u = w dn:
//     dx = r (u - xh mean(u xh)),   dw = sum dn xh.
// Forward and backward read each input once and write each output once; memory
// bounds them.
//
// A warp takes a run of rows (heads of Q, of K, of V, token by token).  A row lies across D / E lanes, E = 16 bytes of elements each: the
// first members of E / 2 pairs and their second members, so a pair is always in one
// lane.  With interleaved pairs these are 16 bytes in a row, with the half layout
// twice 8 bytes (rot is a multiple of 16, so they are aligned, and a lane's pairs
// are all rotated or all not).  Each thread copies what it will need next into a
// ring of its own in shared memory (cp.async), kDepth steps ahead, across tokens:
// that keeps 64 KB and more in flight per SM without holding registers, and needs
// no barrier, since a thread reads only what it has copied.  The angles depend on
// the token only: the lanes of a warp form them once, two each at most, and read
// their own from shared memory.  Beside memory the issue slots count: at the
// memory's rate an SM has about 170 (backward 260) for the 512 (2 x 512) bytes of a
// step, so what depends on the kind of row is set where the kind changes, and a
// step only advances pointers.  Everything is float32; outputs are rounded once.
#include "hybrid_common.cuh"
#include "softmax_kernels.h"
#include "tc_pipeline.cuh"

namespace hyb {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxBackwardBlocks = 512;     // partial sums of dw

template <typename T> struct Vec {
    static constexpr int E = 16 / sizeof(T);
    __device__ static void unpack(const uint4 &v, float (&x)[E]);
    __device__ static uint4 pack(const float (&x)[E]);
};
template <> __device__ __forceinline__ void Vec<float>::unpack(const uint4 &v, float (&x)[4])
{
    x[0] = __uint_as_float(v.x);
    x[1] = __uint_as_float(v.y);
    x[2] = __uint_as_float(v.z);
    x[3] = __uint_as_float(v.w);
}
template <> __device__ __forceinline__ uint4 Vec<float>::pack(const float (&x)[4])
{
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}
template <> __device__ __forceinline__ void Vec<__nv_bfloat16>::unpack(const uint4 &v, float (&x)[8])
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
template <> __device__ __forceinline__ uint4 Vec<__nv_bfloat16>::pack(const float (&x)[8])
{
    return make_uint4(pipe::pack_bf16x2(x[0], x[1]), pipe::pack_bf16x2(x[2], x[3]), pipe::pack_bf16x2(x[4], x[5]),
                      pipe::pack_bf16x2(x[6], x[7]));
}

// Sum over the L lanes of a head.
template <int L> __device__ __forceinline__ float head_sum(float v)
{
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

constexpr int kMaxPairs = 64;
constexpr int kDepth = 4;           // steps ahead

// Where a lane's features lie in a row: two pieces of E / 2.
template <int D, int E, bool kInter> struct Pieces {
    int first, second;              // offsets of the pieces
    int pair;                       // its first pair
    bool on;                        // its pairs are rotated
    __device__ Pieces(const RopeArgs &a, int l)
    {
        pair = l * (E / 2);
        const int half = a.rot >> 1;
        on = pair < half;
        if (kInter) {
            first = l * E;
            second = first + E / 2;
        } else if (on) {
            first = pair;
            second = half + pair;
        } else {                    // beyond the rotated part, halves of what is left
            first = a.rot + (pair - half);
            second = first + (D / 2 - half);
        }
    }
};

template <int E, bool kInter, typename T>
__device__ __forceinline__ void copy_async(uint4 *dst, const T *row, int first, int second)
{
    if (kInter) {
        ptx::cp_async16(dst, row + first);
    } else {
        asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(ptx::smem_u32(dst)), "l"(row + first) : "memory");
        asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(ptx::smem_u32(dst) + 8), "l"(row + second)
                     : "memory");
    }
}
template <int E, bool kInter, typename T>
__device__ __forceinline__ void store(T *row, int first, int second, const uint4 &v)
{
    if (kInter) {
        *reinterpret_cast<uint4 *>(row + first) = v;
    } else {
        *reinterpret_cast<uint2 *>(row + first) = make_uint2(v.x, v.y);
        *reinterpret_cast<uint2 *>(row + second) = make_uint2(v.z, v.w);
    }
}
template <int E, bool kInter, typename T>
__device__ __forceinline__ uint4 load(const T *row, int first, int second)
{
    if (kInter) return __ldg(reinterpret_cast<const uint4 *>(row + first));
    const uint2 x = __ldg(reinterpret_cast<const uint2 *>(row + first));
    const uint2 y = __ldg(reinterpret_cast<const uint2 *>(row + second));
    return make_uint4(x.x, x.y, y.x, y.y);
}

// Cosine and sine (times scale) of a lane's E / 2 pairs.
template <int E> struct Rotation {
    float c[E / 2], s[E / 2];
};

// The angles of token t, by the whole warp; `table` is the warp's own.
template <int E>
__device__ __forceinline__ void make_rotation(const RopeArgs &a, int t, int pair0, bool on, float2 *table,
                                              Rotation<E> &r)
{
    const int lane = threadIdx.x & 31, half = a.rot >> 1;
    if (half == 0) return;
    __syncwarp();                                   // the last token's have been read
    const unsigned long long p = (unsigned long long)(long long)__ldg(a.positions + t);
#pragma unroll
    for (int i = 0; i < kMaxPairs / 32; ++i) {
        const int pair = lane + 32 * i;
        if (pair < half) {
            // fraction of a turn, exact modulo 1, as a signed number of half turns
            const int frac = (int)(unsigned)((p * __ldg(a.freqs + pair)) >> 32);
            float s, c;
            sincospif((float)frac * 0x1p-31f, &s, &c);
            table[pair] = make_float2(c * a.scale, s * a.scale);
        }
    }
    __syncwarp();
    if (on) {
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            const float2 v = table[pair0 + i];
            r.c[i] = v.x;
            r.s[i] = v.y;
        }
    }
}

// x <- R x (kInverse: R^T x) for a lane whose pairs are rotated.
template <int E, bool kInter, bool kInverse>
__device__ __forceinline__ void rotate(float (&x)[E], const Rotation<E> &r)
{
#pragma unroll
    for (int i = 0; i < E / 2; ++i) {
        float &a = x[kInter ? 2 * i : i], &b = x[kInter ? 2 * i + 1 : E / 2 + i];
        const float s = kInverse ? -r.s[i] : r.s[i], a0 = a;
        a = a0 * r.c[i] - b * s;
        b = b * r.c[i] + a0 * s;
    }
}

// The rows of a token in steps of RPW: kinds 0 (Q), 1 (K) and, with the cache, 2
// (V), each padded to whole steps.  The steps of all tokens are shared out evenly:
// each warp takes a run of them, wherever in a token it begins.
struct Split {
    int steps, steps_q, steps_k;    // steps of a token, of its Q and of its K
    int n_kinds;
    int warps, run, rem;            // warps with work; the first rem take run + 1 steps
    bool wide;                      // more than 2^32 steps in all
};

// A warp's place in its steps.
template <int RPW> struct Cursor {
    int t, kind, h;                 // token, kind, first row of the step
    int left;                       // steps to go

    // Start of a warp's run; false if it has none.
    __device__ bool begin(const Split &s, unsigned warp)
    {
        left = 0;
        if (warp >= (unsigned)s.warps) return false;
        left = s.run + ((int)warp < s.rem ? 1 : 0);
        const unsigned extra = warp < (unsigned)s.rem ? warp : (unsigned)s.rem;
        int at;
        if (s.wide) {
            const unsigned long long start = (unsigned long long)s.run * warp + extra;
            t = (int)(start / (unsigned)s.steps);
            at = (int)(start - (unsigned long long)t * s.steps);
        } else {
            const unsigned start = (unsigned)s.run * warp + extra;
            t = (int)(start / (unsigned)s.steps);
            at = (int)(start - (unsigned)t * s.steps);
        }
        kind = 0;
        if (at >= s.steps_q) {
            at -= s.steps_q;
            kind = 1;
            if (at >= s.steps_k) {
                at -= s.steps_k;
                kind = 2;
            }
        }
        h = at * RPW;
        return true;
    }
    // Advance; true if there is no step left or it is of another kind or token.
    __device__ bool step(const Split &s, int n_heads)
    {
        h += RPW;
        if (--left == 0) return true;
        if (h < n_heads) return false;
        h = 0;
        if (++kind == s.n_kinds) {
            kind = 0;
            ++t;
        }
        return true;
    }
};

template <int N> __device__ __forceinline__ void async_wait()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }

template <typename T, int D, bool kInter>
__global__ __launch_bounds__(kThreads, 4) void k_qk_norm_rope(const RopeArgs a, const Split split)
{
    constexpr int E = Vec<T>::E, L = D / E, RPW = 32 / L;
    __shared__ uint4 s_ring[kDepth][kThreads];
    __shared__ float2 s_angles[kWarps][kMaxPairs];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, sub = lane / L;
    const Pieces<D, E, kInter> piece(a, lane % L);
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    Cursor<RPW> at;
    if (!at.begin(split, blockIdx.x * kWarps + warp)) return;
    Cursor<RPW> ahead = at;
    auto heads = [&](int kind) { return kind == 0 ? a.Hq : a.Hkv; };

    // loads, kDepth steps ahead
    const T *src = nullptr;                 // this lane group's row of the step
    auto source = [&]() {
        const T *base = ahead.kind == 0   ? static_cast<const T *>(a.Q) + (size_t)ahead.t * a.q_stride
                        : ahead.kind == 1 ? static_cast<const T *>(a.K) + (size_t)ahead.t * a.k_stride
                                          : static_cast<const T *>(a.V) + (size_t)ahead.t * a.v_stride;
        src = base + (size_t)(ahead.h + sub) * D;
    };
    int ahead_heads = 0;
    auto issue = [&](int slot) {
        if (ahead.left > 0) {
            if (ahead.h + sub < ahead_heads) copy_async<E, kInter>(&s_ring[slot][tid], src, piece.first, piece.second);
            src += RPW * D;
            if (ahead.step(split, ahead_heads) && ahead.left > 0) {
                ahead_heads = heads(ahead.kind);
                source();
            }
        }
        async_commit();
    };
    ahead_heads = heads(ahead.kind);
    source();
#pragma unroll
    for (int i = 0; i < kDepth; ++i) issue(i);

    Rotation<E> rot;
    float w[E];                             // the kind's weight
    bool norm = false, write = true;
    T *dst = nullptr;                       // this lane group's row of the output
    size_t step = 0;                        // rows RPW apart in the output
    int n_heads = 0, token = -1, slot_of = -1;
    auto enter = [&]() {                    // another kind or token
        n_heads = heads(at.kind);
        if (at.t != token) {
            token = at.t;
            make_rotation<E>(a, token, piece.pair, piece.on, s_angles[warp], rot);
            if (a.slots) slot_of = __ldg(a.slots + token);
        }
        const void *wp = at.kind == 0 ? a.wq : (at.kind == 1 ? a.wk : nullptr);
        norm = wp != nullptr;
        if (norm) Vec<T>::unpack(load<E, kInter>(static_cast<const T *>(wp), piece.first, piece.second), w);
        write = true;
        step = (size_t)RPW * D;
        if (at.kind == 0) {
            dst = static_cast<T *>(a.Qo) + ((size_t)token * a.Hq + at.h + sub) * D;
        } else if (!a.slots) {
            dst = static_cast<T *>(a.Ko) + ((size_t)token * a.Hkv + at.h + sub) * D;
        } else {
            const int page = slot_of / a.page_size;
            write = slot_of >= 0 && page < a.n_pages;
            if (slot_of >= 0 && !write && lane == 0) raise_error(a.err, ERR_BAD_INDEX);
            step *= a.page_size;
            dst = static_cast<T *>(at.kind == 1 ? a.K_cache : a.V_cache);
            if (write)
                dst += (((size_t)page * a.Hkv + at.h + sub) * a.page_size + (size_t)(slot_of % a.page_size)) * D;
        }
    };
    enter();
    for (int slot = 0;; slot = (slot + 1) % kDepth) {
        async_wait<kDepth - 1>();
        const uint4 raw = s_ring[slot][tid];
        uint4 out = raw;
        if (at.kind < 2) {
            float x[E];
            Vec<T>::unpack(raw, x);
            if (norm) {
                float ss = 0.f;
#pragma unroll
                for (int i = 0; i < E; ++i) ss = fmaf(x[i], x[i], ss);
                const float r = rsqrtf(head_sum<L>(ss) * (1.f / D) + a.eps);
#pragma unroll
                for (int i = 0; i < E; ++i) x[i] = x[i] * r * w[i];
            }
            if (piece.on) rotate<E, kInter, false>(x, rot);
            out = Vec<T>::pack(x);
        }
        issue(slot);
        if (write && at.h + sub < n_heads) store<E, kInter>(dst, piece.first, piece.second, out);
        dst += step;
        if (at.step(split, n_heads)) {
            if (at.left == 0) break;
            enter();
        }
    }
}

template <typename T, int D, bool kInter>
__global__ __launch_bounds__(kThreads, 2) void k_qk_norm_rope_backward(const RopeArgs a, const Split split)
{
    constexpr int E = Vec<T>::E, L = D / E, RPW = 32 / L;
    __shared__ uint4 s_ring[kDepth][2][kThreads];
    __shared__ float2 s_angles[kWarps][kMaxPairs];
    __shared__ float s_dw[kWarps][2][D];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, sub = lane / L;
    const Pieces<D, E, kInter> piece(a, lane % L);
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    Cursor<RPW> at;
    const bool work = at.begin(split, blockIdx.x * kWarps + warp);
    Cursor<RPW> ahead = at;
    auto heads = [&](int kind) { return kind == 0 ? a.Hq : a.Hkv; };
    // start of a token's rows of a kind in Q or K (or its gradient)
    auto offset = [&](const Cursor<RPW> &c) {
        return (size_t)c.t * (c.kind == 0 ? a.q_stride : a.k_stride) + (size_t)(c.h + sub) * D;
    };

    const T *src = nullptr, *src_dy = nullptr;
    int ahead_heads = 0;
    auto source = [&]() {
        ahead_heads = heads(ahead.kind);
        src = static_cast<const T *>(ahead.kind == 0 ? a.Q : a.K) + offset(ahead);
        src_dy = static_cast<const T *>(ahead.kind == 0 ? a.dQo : a.dKo) +
                 ((size_t)ahead.t * ahead_heads + ahead.h + sub) * D;
    };
    auto issue = [&](int slot) {
        if (ahead.left > 0) {
            if (ahead.h + sub < ahead_heads) {
                copy_async<E, kInter>(&s_ring[slot][0][tid], src, piece.first, piece.second);
                copy_async<E, kInter>(&s_ring[slot][1][tid], src_dy, piece.first, piece.second);
            }
            src += RPW * D;
            src_dy += RPW * D;
            if (ahead.step(split, ahead_heads) && ahead.left > 0) source();
        }
        async_commit();
    };
    // sums of dw over the rows of the current kind and of the other one
    float dw[E], dw_other[E];
#pragma unroll
    for (int i = 0; i < E; ++i) dw[i] = dw_other[i] = 0.f;
    int kind = 0;                           // of `dw`
    if (work) {
        source();
#pragma unroll
        for (int i = 0; i < kDepth; ++i) issue(i);

        Rotation<E> rot;
        float w[E];
        bool norm = false;
        T *dst = nullptr;
        int n_heads = 0, token = -1;
        auto enter = [&]() {                // another kind or token
            n_heads = heads(at.kind);
            if (at.t != token) {
                token = at.t;
                make_rotation<E>(a, token, piece.pair, piece.on, s_angles[warp], rot);
            }
            const void *wp = at.kind == 0 ? a.wq : a.wk;
            norm = wp != nullptr;
            if (norm) Vec<T>::unpack(load<E, kInter>(static_cast<const T *>(wp), piece.first, piece.second), w);
            dst = static_cast<T *>(at.kind == 0 ? a.Qo : a.Ko) + offset(at);
            if (at.kind != kind) {
                kind = at.kind;
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const float x = dw[i];
                    dw[i] = dw_other[i];
                    dw_other[i] = x;
                }
            }
        };
        enter();
        for (int slot = 0;; slot = (slot + 1) % kDepth) {
            async_wait<kDepth - 1>();
            float x[E], g[E];
            Vec<T>::unpack(s_ring[slot][1][tid], g);
            if (piece.on) rotate<E, kInter, true>(g, rot);          // dn
            const bool live = at.h + sub < n_heads;
            if (norm) {
                Vec<T>::unpack(s_ring[slot][0][tid], x);
                float xx = 0.f, ux = 0.f, u[E];
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    u[i] = g[i] * w[i];
                    xx = fmaf(x[i], x[i], xx);
                    ux = fmaf(u[i], x[i], ux);
                }
                const float r = rsqrtf(head_sum<L>(xx) * (1.f / D) + a.eps);
                const float m = r * r * head_sum<L>(ux) * (1.f / D);    // r mean(u xh)
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const float xh = x[i] * r;
                    if (live) dw[i] = fmaf(g[i], xh, dw[i]);
                    g[i] = r * u[i] - xh * m;
                }
            }
            issue(slot);
            if (live) store<E, kInter>(dst, piece.first, piece.second, Vec<T>::pack(g));
            dst += RPW * D;
            if (at.step(split, n_heads)) {
                if (at.left == 0) break;
                enter();
            }
        }
    }
    // heads of the warp, then warps of the block, in a fixed order
#pragma unroll
    for (int i = 0; i < E; ++i) {
#pragma unroll
        for (int o = L; o < 32; o <<= 1) {
            dw[i] += __shfl_xor_sync(0xffffffffu, dw[i], o);
            dw_other[i] += __shfl_xor_sync(0xffffffffu, dw_other[i], o);
        }
        if (sub == 0) {
            const int c = i < E / 2 ? piece.first + i : piece.second + i - E / 2;
            s_dw[warp][kind][c] = dw[i];
            s_dw[warp][1 - kind][c] = dw_other[i];
        }
    }
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * D; c += kThreads) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) v += s_dw[w][c / D][c % D];
        a.partial[(size_t)blockIdx.x * 2 * D + c] = v;
    }
}

// dw[c] = sum over blocks of partial[b][c], in a fixed order: 8 threads a column,
// each every eighth block.
__global__ __launch_bounds__(kThreads) void k_dw_reduce(const float *partial, int blocks, int d, float *dwq, float *dwk)
{
    __shared__ float s[8][32];
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), y = threadIdx.x >> 5;
    float v = 0.f;
    for (int b = y; b < blocks; b += 8) v += partial[(size_t)b * 2 * d + c];
    s[y][threadIdx.x & 31] = v;
    __syncthreads();
    if (y == 0) {
#pragma unroll
        for (int i = 1; i < 8; ++i) v += s[i][threadIdx.x & 31];
        float *out = c < d ? dwq : dwk;
        if (out) out[c < d ? c : c - d] = v;
    }
}

// Shares of the steps: a warp per step while the GPU holds them, per_sm blocks a
// multiprocessor.  Beyond that, with `waves`, short runs of about 16 to 24 steps
// (whole tokens where those are short): the blocks at work then keep to a narrow
// window of memory, which the DRAM serves better than runs that span all of it
// (20011 tokens of 32 float32 heads: 53 against 62 us; 65536 tokens of 24 bfloat16
// rows: 142 against 153; runs of 4 steps 62 and 180, for the angles).  Returns the
// number of blocks.
int split_rows(const RopeArgs &a, int rpw, int per_sm, bool waves, Split &s)
{
    s.steps_q = (a.Hq + rpw - 1) / rpw;
    s.steps_k = (a.Hkv + rpw - 1) / rpw;
    s.n_kinds = a.slots ? 3 : 2;
    s.steps = s.steps_q + (s.n_kinds - 1) * s.steps_k;
    const long long total = (long long)a.n_tok * s.steps, held = (long long)per_sm * pipe::sm_count() * kWarps;
    long long warps = total < held ? total : held;
    const int run = s.steps >= 16 ? (s.steps < 24 ? s.steps : 24) : (16 + s.steps - 1) / s.steps * s.steps;
    if (waves && total / run > warps) warps = total / run;
    s.warps = (int)warps;
    s.run = (int)(total / warps);
    s.rem = (int)(total % warps);
    s.wide = total > 0xffffffffll;
    return (int)((warps + kWarps - 1) / kWarps);
}

template <typename T, int D, bool kInter> cudaError_t forward(const RopeArgs &a, cudaStream_t st)
{
    Split s;
    const int blocks = split_rows(a, 32 * 16 / (int)sizeof(T) / D, 4, true, s);
    return pipe::launch_early(k_qk_norm_rope<T, D, kInter>, dim3(blocks), dim3(kThreads), 0, st, a, s);
}

template <typename T, int D, bool kInter> cudaError_t backward(const RopeArgs &a, cudaStream_t st)
{
    int blocks = 0;
    if (a.n_tok > 0) {
        Split s;
        blocks = split_rows(a, 32 * 16 / (int)sizeof(T) / D, 2, false, s);
        if (blocks > kMaxBackwardBlocks) return cudaErrorInvalidConfiguration;   // a GPU of more than 256 multiprocessors
        const cudaError_t e =
            pipe::launch_early(k_qk_norm_rope_backward<T, D, kInter>, dim3(blocks), dim3(kThreads), 0, st, a, s);
        if (e != cudaSuccess) return e;
    }
    if (!a.dwq && !a.dwk) return cudaSuccess;
    return pipe::launch_early(k_dw_reduce, dim3(2 * D / 32), dim3(kThreads), 0, st, (const float *)a.partial, blocks, D,
                              a.dwq, a.dwk);
}

template <typename T, int D> cudaError_t either(const RopeArgs &a, bool back, cudaStream_t st)
{
    if (back) return a.interleaved ? backward<T, D, true>(a, st) : backward<T, D, false>(a, st);
    return a.interleaved ? forward<T, D, true>(a, st) : forward<T, D, false>(a, st);
}

cudaError_t launch(hybrid_dtype dt, const RopeArgs &a, bool back, cudaStream_t st)
{
    if (dt == HYBRID_BF16)
        return a.d == 128 ? either<__nv_bfloat16, 128>(a, back, st) : either<__nv_bfloat16, 64>(a, back, st);
    return a.d == 128 ? either<float, 128>(a, back, st) : either<float, 64>(a, back, st);
}

}  // namespace

size_t qk_norm_rope_partial_bytes(int d, int n_tok)
{
    (void)n_tok;                            // the number of blocks is capped
    return (size_t)kMaxBackwardBlocks * 2 * d * sizeof(float);
}

cudaError_t launch_qk_norm_rope(hybrid_dtype dt, const RopeArgs &a, cudaStream_t st) { return launch(dt, a, false, st); }

cudaError_t launch_qk_norm_rope_backward(hybrid_dtype dt, const RopeArgs &a, cudaStream_t st)
{
    return launch(dt, a, true, st);
}

}  // namespace hyb
