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

using ptx::f32x2;
using ptx::pair2;

// 16 bytes of elements as pairs of float32.
template <typename T> struct Vec {
    static constexpr int E = 16 / sizeof(T);
    __device__ static void unpack(const uint4 &v, f32x2 (&x)[E / 2]);
    __device__ static uint4 pack(const f32x2 (&x)[E / 2]);
};
template <> __device__ __forceinline__ void Vec<float>::unpack(const uint4 &v, f32x2 (&x)[2])
{
    x[0] = pair2(__uint_as_float(v.x), __uint_as_float(v.y));
    x[1] = pair2(__uint_as_float(v.z), __uint_as_float(v.w));
}
template <> __device__ __forceinline__ uint4 Vec<float>::pack(const f32x2 (&x)[2])
{
    float f[4];
    ptx::unpair2(x[0], f[0], f[1]);
    ptx::unpair2(x[1], f[2], f[3]);
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
template <> __device__ __forceinline__ void Vec<__nv_bfloat16>::unpack(const uint4 &v, f32x2 (&x)[4])
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = pair2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}
template <> __device__ __forceinline__ uint4 Vec<__nv_bfloat16>::pack(const f32x2 (&x)[4])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a, b;
        ptx::unpair2(x[i], a, b);
        w[i] = pipe::pack_bf16x2(a, b);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
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

// Layout of the pairs: interleaved, halves of part of the head, halves of all of it
// (where the pieces' distance is known to the compiler).
enum Layout { kInterleaved, kHalves, kAllHalves };

// Where a lane's features lie in a row: two pieces of E / 2, in elements.
template <int D, int E, Layout kLayout> struct Pieces {
    int first, distance;            // the first piece, and from it to the second
    int pair;                       // its first pair
    bool on;                        // its pairs are rotated
    __device__ Pieces(const RopeArgs &a, int l)
    {
        pair = l * (E / 2);
        const int half = a.rot >> 1;
        on = pair < half;
        if (kLayout == kInterleaved) {
            first = l * E;
            distance = E / 2;
        } else if (on) {
            first = pair;
            distance = half;
        } else {                    // beyond the rotated part, halves of what is left
            first = a.rot + (pair - half);
            distance = D / 2 - half;
        }
    }
    __device__ int apart() const { return kLayout == kAllHalves ? D / 2 : (kLayout == kInterleaved ? E / 2 : distance); }
};

// Copies of a lane's pieces; `row` points at its first piece.  No branch: a copy of
// a row that is not there is predicated off.
template <Layout kLayout, typename T>
__device__ __forceinline__ void copy_async(uint32_t dst, const T *row, int apart, bool live)
{
    if (kLayout == kInterleaved) {
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %2, 0;\n\t@p cp.async.cg.shared.global [%0], [%1], 16;\n\t}" ::"r"(
                         dst),
                     "l"(row), "r"((int)live)
                     : "memory");
    } else {
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %3, 0;\n\t@p cp.async.ca.shared.global [%0], [%1], 8;\n\t"
            "@p cp.async.ca.shared.global [%0 + 8], [%2], 8;\n\t}" ::"r"(dst),
            "l"(row), "l"(row + apart), "r"((int)live)
            : "memory");
    }
}
template <Layout kLayout, typename T>
__device__ __forceinline__ void store(T *row, int apart, const uint4 &v, bool live)
{
    if (kLayout == kInterleaved) {
        if (live) *reinterpret_cast<uint4 *>(row) = v;
    } else if (live) {
        *reinterpret_cast<uint2 *>(row) = make_uint2(v.x, v.y);
        *reinterpret_cast<uint2 *>(row + apart) = make_uint2(v.z, v.w);
    }
}
template <Layout kLayout, typename T> __device__ __forceinline__ uint4 load(const T *row, int apart)
{
    if (kLayout == kInterleaved) return __ldg(reinterpret_cast<const uint4 *>(row));
    const uint2 x = __ldg(reinterpret_cast<const uint2 *>(row));
    const uint2 y = __ldg(reinterpret_cast<const uint2 *>(row + apart));
    return make_uint4(x.x, x.y, y.x, y.y);
}
__device__ __forceinline__ uint4 ring_load(uint32_t at)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
    return v;
}
__device__ __forceinline__ void ring_store(uint32_t at, uint32_t v)
{
    asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(at), "r"(v) : "memory");
}

// Cosines and sines (times scale) of a lane's E / 2 pairs, as the packed arithmetic
// wants them.  Half layout: c[i], s[i], ns[i] hold those of pairs 2 i and 2 i + 1
// (i < E / 4).  Interleaved: c[i] = (cos, cos) and s[i] = (-sin, sin) of pair i.
template <int E, bool kInter> struct Rotation {
    static constexpr int N = kInter ? E / 2 : E / 4;
    f32x2 c[N], s[N], ns[kInter ? 1 : N];
};

// The angles of token t, by the whole warp; `table` is the warp's own.  kInverse:
// the rotation by -t.
template <int E, bool kInter, bool kInverse>
__device__ __forceinline__ void make_rotation(const RopeArgs &a, int t, int pair0, bool on, float2 *table,
                                              Rotation<E, kInter> &r)
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
            table[pair] = make_float2(c * a.scale, (kInverse ? -s : s) * a.scale);
        }
    }
    __syncwarp();
    if (on) {
        if (kInter) {
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
                const float2 v = table[pair0 + i];
                r.c[i] = pair2(v.x, v.x);
                r.s[i] = pair2(-v.y, v.y);
            }
        } else {
#pragma unroll
            for (int i = 0; i < E / 4; ++i) {
                const float2 v = table[pair0 + 2 * i], w = table[pair0 + 2 * i + 1];
                r.c[i] = pair2(v.x, w.x);
                r.s[i] = pair2(v.y, w.y);
                r.ns[i] = pair2(-v.y, -w.y);
            }
        }
    }
}

// x <- R x for a lane whose pairs are rotated.
template <int E, bool kInter> __device__ __forceinline__ void rotate(f32x2 (&x)[E / 2], const Rotation<E, kInter> &r)
{
    if (kInter) {
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            float a, b;
            ptx::unpair2(x[i], a, b);
            x[i] = ptx::fma2(pair2(b, a), r.s[i], ptx::mul2(x[i], r.c[i]));
        }
    } else {
#pragma unroll
        for (int i = 0; i < E / 4; ++i) {
            f32x2 &a = x[i], &b = x[E / 4 + i];
            const f32x2 a0 = a;
            a = ptx::fma2(b, r.ns[i], ptx::mul2(a0, r.c[i]));
            b = ptx::fma2(a0, r.s[i], ptx::mul2(b, r.c[i]));
        }
    }
}

// Sum of the two halves.
__device__ __forceinline__ float both(const f32x2 &x)
{
    float a, b;
    ptx::unpair2(x, a, b);
    return a + b;
}

// The rows of a token in steps of RPW: kinds 0 (Q), 1 (K) and, with the cache, 2
// (V), each padded to whole steps.  The steps of all tokens are shared out evenly:
// each warp takes a share of them, wherever in a token it begins.
struct Split {
    int steps, steps_q, steps_k;    // steps of a token, of its Q and of its K
    int n_kinds;
    int warps, share, rem;          // warps with work; the first rem take share + 1 steps
    bool wide;                      // more than 2^32 steps in all
};

// A warp's place: runs of steps of one token and kind.
template <int RPW> struct Cursor {
    int t, kind, h;                 // token, kind, first row of the run
    int run;                        // steps of the run
    int left;                       // steps of the share after the run

    // Start of a warp's share; false if it has none.
    __device__ bool begin(const Split &s, unsigned warp)
    {
        if (warp >= (unsigned)s.warps) return false;
        left = s.share + ((int)warp < s.rem ? 1 : 0);
        const unsigned extra = warp < (unsigned)s.rem ? warp : (unsigned)s.rem;
        int at;
        if (s.wide) {
            const unsigned long long start = (unsigned long long)s.share * warp + extra;
            t = (int)(start / (unsigned)s.steps);
            at = (int)(start - (unsigned long long)t * s.steps);
        } else {
            const unsigned start = (unsigned)s.share * warp + extra;
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
        take(s, (kind == 0 ? s.steps_q : s.steps_k) - at);
        return true;
    }
    // The next run; false if there is none.
    __device__ bool next(const Split &s)
    {
        if (left == 0) return false;
        h = 0;
        if (++kind == s.n_kinds) {
            kind = 0;
            ++t;
        }
        take(s, kind == 0 ? s.steps_q : s.steps_k);
        return true;
    }
    __device__ void take(const Split &s, int steps)
    {
        run = steps < left ? steps : left;
        left -= run;
    }
};

template <int N> __device__ __forceinline__ void async_wait()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }

template <typename T, int D, Layout kLayout>
__global__ __launch_bounds__(kThreads, 4) void k_qk_norm_rope(const RopeArgs a, const Split split)
{
    constexpr int E = Vec<T>::E, L = D / E, RPW = 32 / L;
    constexpr bool kInter = kLayout == kInterleaved;
    constexpr uint32_t kSlot = kThreads * 16;
    __shared__ uint4 s_ring[kDepth * kThreads];
    __shared__ float2 s_angles[kWarps][kMaxPairs];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, sub = lane / L;
    const Pieces<D, E, kLayout> piece(a, lane % L);
    const int apart = piece.apart();
    const uint32_t ring0 = ptx::smem_u32(&s_ring[tid]), ring_end = ring0 + kDepth * kSlot;
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    Cursor<RPW> at;
    if (!at.begin(split, blockIdx.x * kWarps + warp)) return;
    Cursor<RPW> ahead = at;

    // loads, kDepth steps ahead
    const T *src = nullptr;                 // this lane's piece in the next row to load
    int src_rows = 0, src_steps = 0;        // rows from its lane group's on, steps of its run
    auto source = [&]() {
        const T *base = ahead.kind == 0   ? static_cast<const T *>(a.Q) + (size_t)ahead.t * a.q_stride
                        : ahead.kind == 1 ? static_cast<const T *>(a.K) + (size_t)ahead.t * a.k_stride
                                          : static_cast<const T *>(a.V) + (size_t)ahead.t * a.v_stride;
        src = base + (size_t)(ahead.h + sub) * D + piece.first;
        src_rows = (ahead.kind == 0 ? a.Hq : a.Hkv) - ahead.h - sub;
        src_steps = ahead.run;
    };
    auto issue = [&](uint32_t slot) {
        if (src_steps > 0) {
            copy_async<kLayout>(slot, src, apart, src_rows > 0);
            src += RPW * D;
            src_rows -= RPW;
            if (--src_steps == 0 && ahead.next(split)) source();
        }
        async_commit();
    };
    source();
#pragma unroll
    for (int i = 0; i < kDepth; ++i) issue(ring0 + i * kSlot);

    Rotation<E, kInter> rot;
    int token = -1, to = -1;                // token of `rot`, its slot in the cache
    uint32_t slot = ring0;
    do {
        // what depends on the run's token and kind
        if (at.t != token) {
            token = at.t;
            make_rotation<E, kInter, false>(a, token, piece.pair, piece.on, s_angles[warp], rot);
            if (a.slots) to = __ldg(a.slots + token);
        }
        bool write = true;
        size_t step = (size_t)RPW * D;      // rows RPW apart in the output
        T *dst;                             // this lane's piece in the output's row
        if (at.kind == 0) {
            dst = static_cast<T *>(a.Qo) + ((size_t)token * a.Hq + at.h + sub) * D;
        } else if (!a.slots) {
            dst = static_cast<T *>(a.Ko) + ((size_t)token * a.Hkv + at.h + sub) * D;
        } else {
            const int page = to / a.page_size;
            write = to >= 0 && page < a.n_pages;
            if (to >= 0 && !write && lane == 0) raise_error(a.err, ERR_BAD_INDEX);
            step *= a.page_size;
            dst = static_cast<T *>(at.kind == 1 ? a.K_cache : a.V_cache);
            if (write) dst += (((size_t)page * a.Hkv + at.h + sub) * a.page_size + (size_t)(to % a.page_size)) * D;
        }
        dst += piece.first;
        int n = write ? (at.kind == 0 ? a.Hq : a.Hkv) - at.h - sub : 0;     // rows to write
        auto advance = [&](const uint4 &v) {
            issue(slot);
            slot = slot + kSlot == ring_end ? ring0 : slot + kSlot;
            store<kLayout>(dst, apart, v, n > 0);
            n -= RPW;
            dst += step;
        };
        if (at.kind == 2) {
            for (int i = at.run; i > 0; --i) {
                async_wait<kDepth - 1>();
                advance(ring_load(slot));
            }
            continue;
        }
        const void *wp = at.kind == 0 ? a.wq : a.wk;
        f32x2 w[E / 2];
        if (wp) Vec<T>::unpack(load<kLayout>(static_cast<const T *>(wp) + piece.first, apart), w);
        for (int i = at.run; i > 0; --i) {
            async_wait<kDepth - 1>();
            f32x2 x[E / 2];
            Vec<T>::unpack(ring_load(slot), x);
            if (wp) {
                f32x2 ss = ptx::mul2(x[0], x[0]);
#pragma unroll
                for (int k = 1; k < E / 2; ++k) ss = ptx::fma2(x[k], x[k], ss);
                const float r = rsqrtf(head_sum<L>(both(ss)) * (1.f / D) + a.eps);
                const f32x2 rr = pair2(r, r);
#pragma unroll
                for (int k = 0; k < E / 2; ++k) x[k] = ptx::mul2(ptx::mul2(x[k], rr), w[k]);
            }
            if (kLayout == kAllHalves || piece.on) rotate<E, kInter>(x, rot);
            advance(Vec<T>::pack(x));
        }
    } while (at.next(split));
}

template <typename T, int D, Layout kLayout>
__global__ __launch_bounds__(kThreads, 2) void k_qk_norm_rope_backward(const RopeArgs a, const Split split)
{
    constexpr int E = Vec<T>::E, L = D / E, RPW = 32 / L;
    constexpr bool kInter = kLayout == kInterleaved;
    constexpr uint32_t kHalf = kThreads * 16, kSlot = 2 * kHalf;            // x, then dy
    __shared__ uint4 s_ring[kDepth * 2 * kThreads];
    __shared__ float2 s_angles[kWarps][kMaxPairs];
    __shared__ float s_dw[kWarps][2][D];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, sub = lane / L;
    const Pieces<D, E, kLayout> piece(a, lane % L);
    const int apart = piece.apart();
    const uint32_t ring0 = ptx::smem_u32(&s_ring[tid]), ring_end = ring0 + kDepth * kSlot;
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    Cursor<RPW> at;
    const bool work = at.begin(split, blockIdx.x * kWarps + warp);
    Cursor<RPW> ahead = at;
    // this lane's piece of a run's first row in Q or K (or its gradient)
    auto offset = [&](const Cursor<RPW> &c) {
        return (size_t)c.t * (c.kind == 0 ? a.q_stride : a.k_stride) + (size_t)(c.h + sub) * D + piece.first;
    };

    const T *src = nullptr, *src_dy = nullptr;
    int src_rows = 0, src_steps = 0;
    auto source = [&]() {
        const int heads = ahead.kind == 0 ? a.Hq : a.Hkv;
        src = static_cast<const T *>(ahead.kind == 0 ? a.Q : a.K) + offset(ahead);
        src_dy = static_cast<const T *>(ahead.kind == 0 ? a.dQo : a.dKo) +
                 ((size_t)ahead.t * heads + ahead.h + sub) * D + piece.first;
        src_rows = heads - ahead.h - sub;
        src_steps = ahead.run;
    };
    auto issue = [&](uint32_t slot) {
        if (src_steps > 0) {
            copy_async<kLayout>(slot, src, apart, src_rows > 0);
            copy_async<kLayout>(slot + kHalf, src_dy, apart, src_rows > 0);
            if (src_rows <= 0) {            // beyond the heads: x = 1, dy = 0, which adds nothing to dw
                ring_store(slot, sizeof(T) == 2 ? 0x3f803f80u : 0x3f800000u);
                ring_store(slot + kHalf, 0u);
            }
            src += RPW * D;
            src_dy += RPW * D;
            src_rows -= RPW;
            if (--src_steps == 0 && ahead.next(split)) source();
        }
        async_commit();
    };
    // sums of dw over the rows of the current kind and of the other one
    f32x2 dw[E / 2], dw_other[E / 2];
#pragma unroll
    for (int i = 0; i < E / 2; ++i) dw[i] = dw_other[i] = pair2(0.f, 0.f);
    int kind = 0;                           // of `dw`
    if (work) {
        source();
#pragma unroll
        for (int i = 0; i < kDepth; ++i) issue(ring0 + i * kSlot);

        Rotation<E, kInter> rot;
        int token = -1;
        uint32_t slot = ring0;
        do {
            if (at.t != token) {
                token = at.t;
                make_rotation<E, kInter, true>(a, token, piece.pair, piece.on, s_angles[warp], rot);
            }
            if (at.kind != kind) {
                kind = at.kind;
#pragma unroll
                for (int i = 0; i < E / 2; ++i) {
                    const f32x2 x = dw[i];
                    dw[i] = dw_other[i];
                    dw_other[i] = x;
                }
            }
            const void *wp = kind == 0 ? a.wq : a.wk;
            f32x2 w[E / 2];
            if (wp) Vec<T>::unpack(load<kLayout>(static_cast<const T *>(wp) + piece.first, apart), w);
            T *dst = static_cast<T *>(kind == 0 ? a.Qo : a.Ko) + offset(at);
            int n = (kind == 0 ? a.Hq : a.Hkv) - at.h - sub;                // rows to write
            for (int i = at.run; i > 0; --i) {
                async_wait<kDepth - 1>();
                f32x2 x[E / 2], g[E / 2];
                Vec<T>::unpack(ring_load(slot + kHalf), g);
                if (kLayout == kAllHalves || piece.on) rotate<E, kInter>(g, rot);       // dn
                if (wp) {
                    Vec<T>::unpack(ring_load(slot), x);
                    f32x2 u[E / 2], xx = pair2(0.f, 0.f), ux = xx;
#pragma unroll
                    for (int k = 0; k < E / 2; ++k) {
                        u[k] = ptx::mul2(g[k], w[k]);
                        xx = ptx::fma2(x[k], x[k], xx);
                        ux = ptx::fma2(u[k], x[k], ux);
                    }
                    const float r = rsqrtf(head_sum<L>(both(xx)) * (1.f / D) + a.eps);
                    const float m = r * r * head_sum<L>(both(ux)) * (-1.f / D);         // -r mean(u xh)
                    const f32x2 rr = pair2(r, r), mm = pair2(m, m);
#pragma unroll
                    for (int k = 0; k < E / 2; ++k) {
                        const f32x2 xh = ptx::mul2(x[k], rr);
                        dw[k] = ptx::fma2(g[k], xh, dw[k]);
                        g[k] = ptx::fma2(xh, mm, ptx::mul2(u[k], rr));
                    }
                }
                issue(slot);
                slot = slot + kSlot == ring_end ? ring0 : slot + kSlot;
                store<kLayout>(dst, apart, Vec<T>::pack(g), n > 0);
                n -= RPW;
                dst += RPW * D;
            }
        } while (at.next(split));
    }
    // heads of the warp, then warps of the block, in a fixed order
#pragma unroll
    for (int i = 0; i < E / 2; ++i) {
        float v[2][2];
        ptx::unpair2(dw[i], v[0][0], v[0][1]);
        ptx::unpair2(dw_other[i], v[1][0], v[1][1]);
#pragma unroll
        for (int y = 0; y < 2; ++y) {
#pragma unroll
            for (int o = L; o < 32; o <<= 1) {
                v[0][y] += __shfl_xor_sync(0xffffffffu, v[0][y], o);
                v[1][y] += __shfl_xor_sync(0xffffffffu, v[1][y], o);
            }
            const int e = 2 * i + y, c = e < E / 2 ? piece.first + e : piece.first + apart + e - E / 2;
            if (sub == 0) {
                s_dw[warp][kind][c] = v[0][y];
                s_dw[warp][1 - kind][c] = v[1][y];
            }
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

// dw[c] = sum over blocks of partial[b][c], in a fixed order: 32 threads a column,
// each every 32nd block.
constexpr int kReduceThreads = 1024;
__global__ __launch_bounds__(kReduceThreads) void k_dw_reduce(const float *partial, int blocks, int d, float *dwq,
                                                              float *dwk)
{
    __shared__ float s[32][33];
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5, c = blockIdx.x * 32 + x;
    float v = 0.f;
#pragma unroll 4
    for (int b = y; b < blocks; b += 32) v += partial[(size_t)b * 2 * d + c];
    s[y][x] = v;
    __syncthreads();
    // warp y adds up column y of this block's 32
    v = warp_sum(s[x][y]);
    const int col = blockIdx.x * 32 + y;
    float *out = col < d ? dwq : dwk;
    if (x == 0 && out) out[col < d ? col : col - d] = v;
}

// Shares of the steps: a warp per step while the GPU holds them, per_sm blocks a
// multiprocessor.  Beyond that, with `waves`, short shares of about 16 to 24 steps
// (whole tokens where those are short): the blocks at work then keep to a narrow
// window of memory and fast multiprocessors take more of them (20011 tokens of 32
// float32 heads: 54 against 62 us; 65536 tokens of 24 bfloat16 rows: 142 against
// 153; shares of 4 steps 62 and 180, for the angles).  Returns the number of blocks.
int split_rows(const RopeArgs &a, int rpw, int per_sm, bool waves, Split &s)
{
    s.steps_q = (a.Hq + rpw - 1) / rpw;
    s.steps_k = (a.Hkv + rpw - 1) / rpw;
    s.n_kinds = a.slots ? 3 : 2;
    s.steps = s.steps_q + (s.n_kinds - 1) * s.steps_k;
    const long long total = (long long)a.n_tok * s.steps, held = (long long)per_sm * pipe::sm_count() * kWarps;
    long long warps = total < held ? total : held;
    const int share = s.steps >= 16 ? (s.steps < 24 ? s.steps : 24) : (16 + s.steps - 1) / s.steps * s.steps;
    if (waves && total / share > warps) warps = total / share;
    if (warps > 1 << 30) warps = 1 << 30;
    s.warps = (int)warps;
    s.share = (int)(total / warps);
    s.rem = (int)(total % warps);
    s.wide = total > 0xffffffffll;
    return (int)((warps + kWarps - 1) / kWarps);
}

template <typename T, int D, Layout kLayout> cudaError_t forward(const RopeArgs &a, cudaStream_t st)
{
    Split s;
    const int blocks = split_rows(a, 32 * 16 / (int)sizeof(T) / D, 4, true, s);
    return pipe::launch_early(k_qk_norm_rope<T, D, kLayout>, dim3(blocks), dim3(kThreads), 0, st, a, s);
}

template <typename T, int D, Layout kLayout> cudaError_t backward(const RopeArgs &a, cudaStream_t st)
{
    int blocks = 0;
    if (a.n_tok > 0) {
        // one wave: each further one costs about 4 us for its sums of dw
        Split s;
        blocks = split_rows(a, 32 * 16 / (int)sizeof(T) / D, 2, false, s);
        if (blocks > kMaxBackwardBlocks) return cudaErrorInvalidConfiguration;   // a GPU of more than 256 multiprocessors
        const cudaError_t e =
            pipe::launch_early(k_qk_norm_rope_backward<T, D, kLayout>, dim3(blocks), dim3(kThreads), 0, st, a, s);
        if (e != cudaSuccess) return e;
    }
    if (!a.dwq && !a.dwk) return cudaSuccess;
    return pipe::launch_early(k_dw_reduce, dim3(2 * D / 32), dim3(kReduceThreads), 0, st, (const float *)a.partial, blocks,
                              D, a.dwq, a.dwk);
}

template <typename T, int D> cudaError_t any(const RopeArgs &a, bool back, cudaStream_t st)
{
    if (a.interleaved) return back ? backward<T, D, kInterleaved>(a, st) : forward<T, D, kInterleaved>(a, st);
    if (a.rot == D) return back ? backward<T, D, kAllHalves>(a, st) : forward<T, D, kAllHalves>(a, st);
    return back ? backward<T, D, kHalves>(a, st) : forward<T, D, kHalves>(a, st);
}

cudaError_t launch(hybrid_dtype dt, const RopeArgs &a, bool back, cudaStream_t st)
{
    if (dt == HYBRID_BF16)
        return a.d == 128 ? any<__nv_bfloat16, 128>(a, back, st) : any<__nv_bfloat16, 64>(a, back, st);
    return a.d == 128 ? any<float, 128>(a, back, st) : any<float, 64>(a, back, st);
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
