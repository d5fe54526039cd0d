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
// A warp takes one token and a run of its heads.  A head lies across D / E lanes,
// E = 16 bytes of elements each, so every load and store is 16 bytes a lane and
// 512 a warp.  The angles depend on the token only: each lane forms the cosines
// and sines of its own features once and uses them for all heads of the run.  A
// pair's other member is in the same lane (interleaved) or rot / 2 features away,
// which is a whole number of lanes because rot is a multiple of 16: one shuffle
// per feature.  Everything is float32; outputs are rounded once.
#include <math_constants.h>

#include "hybrid_common.cuh"
#include "softmax_kernels.h"
#include "tc_pipeline.cuh"

namespace hyb {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxBackwardBlocks = 608;     // partial sums of dw: 4 blocks per SM of 152

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

// What a lane needs to rotate its E features: cos and sin (times scale) of each,
// and the lane that holds the other member of its pairs (half layout).
template <int E> struct Rotation {
    float c[E], s[E];
    int partner;        // lane offset of the other member
    bool on;            // the lane's features are rotated
};

template <int E>
__device__ __forceinline__ Rotation<E> make_rotation(const RopeArgs &a, int t, int e0)
{
    Rotation<E> r;
    const int half = a.rot >> 1;
    r.on = e0 < a.rot;
    r.partner = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        r.c[i] = 1.f;
        r.s[i] = 0.f;
    }
    if (!r.on) return r;
    const unsigned long long p = (unsigned long long)(long long)a.positions[t];
    const bool second = !a.interleaved && e0 >= half;
    if (!a.interleaved) r.partner = second ? -(half / E) : half / E;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        if (a.interleaved && (i & 1)) {             // the pair's angle again
            r.c[i] = r.c[i - 1];
            r.s[i] = -r.s[i - 1];
            continue;
        }
        const int pair = a.interleaved ? (e0 + i) >> 1 : (second ? e0 - half : e0) + i;
        // fraction of a turn, exact modulo 1, as a signed number of half turns
        const int frac = (int)(unsigned)((p * a.freqs[pair]) >> 32);
        float s, c;
        sincospif((float)frac * 0x1p-31f, &s, &c);
        r.c[i] = c * a.scale;
        // the first member gets -b sin, the second +a sin
        r.s[i] = (second ? s : -s) * a.scale;
    }
    return r;
}

// x <- R x (kInverse: R^T x).  All lanes of the warp take part.
template <int E, bool kInverse>
__device__ __forceinline__ void rotate(float (&x)[E], const Rotation<E> &r, bool interleaved, int lane)
{
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < E; i += 2) {
            const float a = x[i], b = x[i + 1];
            const float sa = kInverse ? -r.s[i] : r.s[i], sb = kInverse ? -r.s[i + 1] : r.s[i + 1];
            if (r.on) {
                x[i] = a * r.c[i] + b * sa;
                x[i + 1] = b * r.c[i + 1] + a * sb;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const float o = __shfl_sync(0xffffffffu, x[i], lane + r.partner);
            if (r.on) x[i] = x[i] * r.c[i] + o * (kInverse ? -r.s[i] : r.s[i]);
        }
    }
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads, 3) void k_qk_norm_rope(const RopeArgs a, int parts, int rows_per_part)
{
    constexpr int E = Vec<T>::E, L = D / E, RPW = 32 / L, U = E == 8 ? 2 : 4;
    const int lane = threadIdx.x & 31, sub = lane / L, e0 = (lane % L) * E;
    const long long item = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    if (item >= (long long)a.n_tok * parts) return;
    const int t = (int)(item / parts), part = (int)(item % parts);
    const int n_rows = a.Hq + (a.slots ? 2 : 1) * a.Hkv;    // q heads, k heads, v heads
    const int begin = part * rows_per_part;
    const int end = begin + rows_per_part < n_rows ? begin + rows_per_part : n_rows;

    const T *Q = static_cast<const T *>(a.Q) + (size_t)t * a.q_stride + e0;
    const T *K = static_cast<const T *>(a.K) + (size_t)t * a.k_stride + e0;
    const T *V = static_cast<const T *>(a.V) + (size_t)t * a.v_stride + e0;
    T *Qo = static_cast<T *>(a.Qo) + (size_t)t * a.Hq * D + e0;
    // key head h of the token: base + h * step
    T *Ko, *Vo = nullptr;
    size_t step = D;
    bool write_kv = true;
    if (a.slots) {
        const int slot = a.slots[t];
        const int page = slot / a.page_size;
        write_kv = slot >= 0 && page < a.n_pages;
        if (slot >= 0 && !write_kv && lane == 0) raise_error(a.err, ERR_BAD_INDEX);
        const size_t at =
            write_kv ? ((size_t)page * a.Hkv * a.page_size + (size_t)(slot % a.page_size)) * D + e0 : 0;
        step = (size_t)a.page_size * D;
        Ko = static_cast<T *>(a.K_cache) + at;
        Vo = static_cast<T *>(a.V_cache) + at;
    } else {
        Ko = static_cast<T *>(a.Ko) + (size_t)t * a.Hkv * D + e0;
    }
    // U rows a lane group are loaded before the angles are formed, and the next U
    // while these are worked on
    uint4 raw[U], next[U];
    auto load = [&](int h0, uint4 (&r)[U]) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = h0 + u * RPW + sub;
            r[u] = make_uint4(0, 0, 0, 0);
            if (h < end) {
                const T *src = h < a.Hq ? Q + (size_t)h * D
                                        : (h < a.Hq + a.Hkv ? K + (size_t)(h - a.Hq) * D
                                                            : V + (size_t)(h - a.Hq - a.Hkv) * D);
                r[u] = *reinterpret_cast<const uint4 *>(src);
            }
        }
    };
    load(begin, next);
    const Rotation<E> rot = make_rotation<E>(a, t, e0);

    for (int h0 = begin; h0 < end; h0 += U * RPW) {
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = next[u];
        if (h0 + U * RPW < end) load(h0 + U * RPW, next);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = h0 + u * RPW + sub;
            if (h0 + u * RPW >= end) break;                 // the whole warp
            float x[E];
            Vec<T>::unpack(raw[u], x);
            const bool is_q = h < a.Hq, is_k = !is_q && h < a.Hq + a.Hkv;
            const void *w = is_q ? a.wq : (is_k ? a.wk : nullptr);
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < E; ++i) ss = fmaf(x[i], x[i], ss);
            ss = head_sum<L>(ss);
            if (w) {
                const float r = rsqrtf(ss * (1.f / D) + a.eps);
                float g[E];
                Vec<T>::unpack(*reinterpret_cast<const uint4 *>(static_cast<const T *>(w) + e0), g);
#pragma unroll
                for (int i = 0; i < E; ++i) x[i] = x[i] * r * g[i];
            }
            rotate<E, false>(x, rot, a.interleaved, lane);
            if (h >= end) continue;
            if (is_q) {
                *reinterpret_cast<uint4 *>(Qo + (size_t)h * D) = Vec<T>::pack(x);
            } else if (write_kv) {
                if (is_k) *reinterpret_cast<uint4 *>(Ko + (size_t)(h - a.Hq) * step) = Vec<T>::pack(x);
                else *reinterpret_cast<uint4 *>(Vo + (size_t)(h - a.Hq - a.Hkv) * step) = raw[u];
            }
        }
    }
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads, 2) void k_qk_norm_rope_backward(const RopeArgs a, int parts, int rows_per_part)
{
    constexpr int E = Vec<T>::E, L = D / E, RPW = 32 / L, U = 2;
    __shared__ float s_dw[kWarps][2][D];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane / L, e0 = (lane % L) * E;
    const int n_rows = a.Hq + a.Hkv;
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    // the weights stay packed: they are unpacked where they are used
    uint4 wq = make_uint4(0, 0, 0, 0), wk = wq;
    float dwq[E], dwk[E];
#pragma unroll
    for (int i = 0; i < E; ++i) dwq[i] = dwk[i] = 0.f;
    if (a.wq) wq = *reinterpret_cast<const uint4 *>(static_cast<const T *>(a.wq) + e0);
    if (a.wk) wk = *reinterpret_cast<const uint4 *>(static_cast<const T *>(a.wk) + e0);
    const long long items = (long long)a.n_tok * parts, stride = (long long)gridDim.x * kWarps;

    // A warp's rows, U lane groups' worth at a time, over all of its tokens: the next
    // ones are loaded while these are worked on.
    struct Place {
        long long item;
        int h0;             // first row of the batch
        int end;            // end of the token's rows
    };
    auto rows_of = [&](Place &p) {
        const int begin = (int)(p.item % parts) * rows_per_part;
        p.h0 = begin;
        p.end = begin + rows_per_part < n_rows ? begin + rows_per_part : n_rows;
    };
    auto step = [&](Place &p) {
        p.h0 += U * RPW;
        if (p.h0 < p.end) return;
        p.item += stride;
        if (p.item < items) rows_of(p);
    };
    auto place_of = [&](const Place &p, int u, bool &live, bool &is_q, size_t &at, size_t &dy) {
        const int t = (int)(p.item / parts), h = p.h0 + u * RPW + sub;
        live = h < p.end;
        is_q = h < a.Hq;
        at = is_q ? (size_t)t * a.q_stride + (size_t)h * D + e0 : (size_t)t * a.k_stride + (size_t)(h - a.Hq) * D + e0;
        dy = is_q ? ((size_t)t * a.Hq + h) * D + e0 : ((size_t)t * a.Hkv + (h - a.Hq)) * D + e0;
    };
    uint4 nx[U], ny[U];
    auto load = [&](const Place &p) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            bool live, is_q;
            size_t at, dy;
            place_of(p, u, live, is_q, at, dy);
            nx[u] = ny[u] = make_uint4(0, 0, 0, 0);
            if (live) {
                nx[u] = *reinterpret_cast<const uint4 *>(static_cast<const T *>(is_q ? a.Q : a.K) + at);
                ny[u] = *reinterpret_cast<const uint4 *>(static_cast<const T *>(is_q ? a.dQo : a.dKo) + dy);
            }
        }
    };
    Place p{(long long)blockIdx.x * kWarps + warp, 0, 0};
    if (p.item < items) {
        rows_of(p);
        load(p);
    }
    long long rotated = -1;                 // token of `rot`
    Rotation<E> rot;
    while (p.item < items) {
        const Place now = p;
        uint4 rx[U], ry[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            rx[u] = nx[u];
            ry[u] = ny[u];
        }
        step(p);
        if (p.item < items) load(p);
        if (now.item / parts != rotated) {
            rotated = now.item / parts;
            rot = make_rotation<E>(a, (int)rotated, e0);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (now.h0 + u * RPW >= now.end) break;         // the whole warp
            bool live, is_q;
            size_t at, dy;
            place_of(now, u, live, is_q, at, dy);
            float x[E], g[E], w[E];
            Vec<T>::unpack(rx[u], x);
            Vec<T>::unpack(ry[u], g);
            Vec<T>::unpack(is_q ? wq : wk, w);
            rotate<E, true>(g, rot, a.interleaved, lane);   // dn
            float xx = 0.f, ux = 0.f;
            const bool norm = is_q ? a.wq != nullptr : a.wk != nullptr;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                xx = fmaf(x[i], x[i], xx);
                ux = fmaf(g[i] * w[i], x[i], ux);
            }
            xx = head_sum<L>(xx);
            ux = head_sum<L>(ux);
            if (!live) continue;
            if (norm) {
                const float r = rsqrtf(xx * (1.f / D) + a.eps), m = r * ux * (1.f / D);   // m = mean(u xh)
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const float xh = x[i] * r, dw = g[i] * xh;
                    if (is_q) dwq[i] += dw;
                    else dwk[i] += dw;
                    g[i] = r * (g[i] * w[i] - xh * m);
                }
            }
            *reinterpret_cast<uint4 *>(static_cast<T *>(is_q ? a.Qo : a.Ko) + at) = Vec<T>::pack(g);
        }
    }
    // heads of the warp, then warps of the block, in a fixed order
#pragma unroll
    for (int i = 0; i < E; ++i) {
#pragma unroll
        for (int o = L; o < 32; o <<= 1) {
            dwq[i] += __shfl_xor_sync(0xffffffffu, dwq[i], o);
            dwk[i] += __shfl_xor_sync(0xffffffffu, dwk[i], o);
        }
        if (sub == 0) {
            s_dw[warp][0][e0 + i] = dwq[i];
            s_dw[warp][1][e0 + i] = dwk[i];
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

// Heads per warp: all heads of a token when there are enough tokens to fill the
// GPU, else runs short enough that about 16 warps a multiprocessor have one.
void split_heads(long long n_tok, int n_rows, int rpw, int &parts, int &rows_per_part)
{
    const long long want = 152 * 16;
    const int most = (n_rows + rpw - 1) / rpw;              // parts of one row a lane group
    long long p = (want + n_tok - 1) / n_tok;
    if (p > most) p = most;
    if (p < 1) p = 1;
    rows_per_part = (int)((n_rows + p - 1) / p);
    rows_per_part = (rows_per_part + rpw - 1) / rpw * rpw;
    parts = (n_rows + rows_per_part - 1) / rows_per_part;
}

template <typename T, int D> cudaError_t forward(const RopeArgs &a, cudaStream_t st)
{
    constexpr int RPW = 32 * 16 / (int)sizeof(T) / D;
    int parts, rpp;
    split_heads(a.n_tok, a.Hq + (a.slots ? 2 : 1) * a.Hkv, RPW, parts, rpp);
    const long long blocks = ((long long)a.n_tok * parts + kWarps - 1) / kWarps;
    return pipe::launch_early(k_qk_norm_rope<T, D>, dim3((unsigned)blocks), dim3(kThreads), 0, st, a, parts, rpp);
}

template <typename T, int D> cudaError_t backward(const RopeArgs &a, cudaStream_t st)
{
    constexpr int RPW = 32 * 16 / (int)sizeof(T) / D;
    int blocks = 0;
    if (a.n_tok > 0) {
        int parts, rpp;
        split_heads(a.n_tok, a.Hq + a.Hkv, RPW, parts, rpp);
        const long long want = ((long long)a.n_tok * parts + kWarps - 1) / kWarps;
        blocks = (int)(want < kMaxBackwardBlocks ? want : kMaxBackwardBlocks);
        const cudaError_t e =
            pipe::launch_early(k_qk_norm_rope_backward<T, D>, dim3(blocks), dim3(kThreads), 0, st, a, parts, rpp);
        if (e != cudaSuccess) return e;
    }
    if (!a.dwq && !a.dwk) return cudaSuccess;
    return pipe::launch_early(k_dw_reduce, dim3(2 * D / 32), dim3(kThreads), 0, st, (const float *)a.partial, blocks, D,
                              a.dwq, a.dwk);
}

}  // namespace

size_t qk_norm_rope_partial_bytes(int d, int n_tok)
{
    (void)n_tok;                            // the number of blocks is capped
    return (size_t)kMaxBackwardBlocks * 2 * d * sizeof(float);
}

cudaError_t launch_qk_norm_rope(hybrid_dtype dt, const RopeArgs &a, cudaStream_t st)
{
    if (dt == HYBRID_BF16)
        return a.d == 128 ? forward<__nv_bfloat16, 128>(a, st) : forward<__nv_bfloat16, 64>(a, st);
    return a.d == 128 ? forward<float, 128>(a, st) : forward<float, 64>(a, st);
}

cudaError_t launch_qk_norm_rope_backward(hybrid_dtype dt, const RopeArgs &a, cudaStream_t st)
{
    if (dt == HYBRID_BF16)
        return a.d == 128 ? backward<__nv_bfloat16, 128>(a, st) : backward<__nv_bfloat16, 64>(a, st);
    return a.d == 128 ? backward<float, 128>(a, st) : backward<float, 64>(a, st);
}

}  // namespace hyb
