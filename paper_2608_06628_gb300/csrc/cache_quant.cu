// cache_quant.cu -- the paged cache in 8 bits: keys and values rounded as they are written, with
// the keys' norm and rotation in the same pass (hybrid_qk_norm_rope_cache_quant), and tokens read
// back (hybrid_cache_dequant).  The format is in quant.cuh.
//
// Write.  A scale belongs to 16 tokens of a head, so the tokens of one group that a call writes
// (a run: they stand side by side, but for tokens without a slot) are held together: a warp has a run's rows of one head, of K
// or of V, in registers, up to 16 rows of d float32 (64 registers a lane at d = 128), and
//     y = norm and rotation of x (K),   amax = max |y| over the run
//     E = least power of two with amax <= 448 * 2^E; no less than the group's old one, unless
//         the run has the group's first slot
//     code = e4m3(y / 2^E)
// then brings the group's other tokens to 2^E (zeros where the group starts afresh).  A block
// takes a window of the packed tokens and the runs that begin in it, one after another; its warps
// share a run's angles and take its heads.  Queries go through qk_norm_rope.cu's kernel.
#include "quant.cuh"
#include "rope_rows.cuh"

namespace hyb {
namespace {

using namespace rope;
using namespace quant;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

struct Run {
    int t, n;                   // first token, and tokens up to the last one
    unsigned members;           // those of them that are written: a bit each (others have no slot)
    int page, off;              // place of the group in the cache: page, first token in it
    unsigned written;           // a bit for each token of the group that the run has
    int slot;                   // of this lane's token (lane < n)
    __device__ bool has(int r) const { return members >> r & 1u; }
};

// One head of a run, K (kLayout: of the rotated pairs) or V (norm and rotation left out).
template <typename T, int D, Layout kLayout, bool kKey>
__device__ __forceinline__ void write_head(const RopeArgs &a, const Run &run, int head, const float2 *angles)
{
    constexpr int E = Vec<T>::E, L = D / E, RPW = 32 / L, kSteps = kGroup / RPW;
    const int lane = threadIdx.x & 31, sub = lane / L;
    const Pieces<D, E, kLayout> piece(a, lane % L);
    const int apart = piece.apart();
    const T *src = static_cast<const T *>(kKey ? a.K : a.V) + (size_t)head * D + piece.first;
    const size_t stride = kKey ? a.k_stride : a.v_stride;

    uint4 raw[kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const int r = i * RPW + sub;
        raw[i] = run.has(r) ? load<kLayout>(src + (size_t)(run.t + r) * stride, apart) : make_uint4(0, 0, 0, 0);
    }
    f32x2 x[kSteps][E / 2];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) Vec<T>::unpack(raw[i], x[i]);
    if (kKey && a.wk) {
        f32x2 w[E / 2];
        Vec<T>::unpack(load<kLayout>(static_cast<const T *>(a.wk) + piece.first, apart), w);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            if (i * RPW >= run.n) break;
            f32x2 ss = ptx::mul2(x[i][0], x[i][0]);
#pragma unroll
            for (int k = 1; k < E / 2; ++k) ss = ptx::fma2(x[i][k], x[i][k], ss);
            const float r = rsqrtf(head_sum<L>(both(ss)) * (1.f / D) + a.eps);
            const f32x2 rr = pair2(r, r);
#pragma unroll
            for (int k = 0; k < E / 2; ++k) x[i][k] = ptx::mul2(ptx::mul2(x[i][k], rr), w[k]);
        }
    }
    if (kKey && a.rot > 0 && piece.on) {
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int r = i * RPW + sub;
            if (!run.has(r)) continue;
            Rotation<E, kLayout == kInterleaved> rot;
            read_rotation(angles + r * kMaxPairs, piece.pair, rot);
            rotate<E, kLayout == kInterleaved>(x[i], rot);
        }
    }
    // the largest magnitude, as bits; beyond 0x7f7fffff there are infinities or NaN, which are left out
    uint32_t amax = 0;
    auto each = [&](auto f) {
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
            if (run.has(i * RPW + sub))
#pragma unroll
                for (int k = 0; k < E / 2; ++k) {
                    float lo, hi;
                    ptx::unpair2(x[i][k], lo, hi);
                    f(lo, hi);
                    x[i][k] = pair2(lo, hi);
                }
    };
    auto magnitude = [](float v) { return __float_as_uint(v) & 0x7fffffffu; };
    each([&](float &lo, float &hi) { amax = max(amax, max(magnitude(lo), magnitude(hi))); });
    amax = __reduce_max_sync(0xffffffffu, amax);
    if (amax >= 0x7f800000u) {
        amax = 0;
        each([&](float &lo, float &hi) {
            for (float *v : {&lo, &hi}) {
                if (magnitude(*v) < 0x7f800000u) amax = max(amax, magnitude(*v));
                else *v = __uint_as_float(0x7fc00000u);
            }
        });
        amax = __reduce_max_sync(0xffffffffu, amax);
    }
    const size_t row = (((size_t)run.page * a.Hkv + head) * a.page_size + run.off);     // the group's first token
    float *scale = (kKey ? a.K_scale : a.V_scale) + row / kGroup;
    uint8_t *codes = static_cast<uint8_t *>(kKey ? a.K_cache : a.V_cache) + row * D;
    const bool fresh = run.written & 1u;
    int e = scale_of_amax(amax), has = e;
    if (!fresh) {
        has = scale_of_bits(__float_as_uint(*scale));
        e = max(e, has);
    }
    const float inv = scale_inverse(e);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const int r = i * RPW + sub;
        const int to = __shfl_sync(0xffffffffu, run.slot, r) % kGroup;
        if (!run.has(r)) continue;
        uint32_t c[E / 4];
#pragma unroll
        for (int k = 0; k < E / 2; k += 2) {
            float v0, v1, v2, v3;
            ptx::unpair2(x[i][k], v0, v1);
            ptx::unpair2(x[i][k + 1], v2, v3);
            c[k / 2] = encode4(v0 * inv, v1 * inv, v2 * inv, v3 * inv);
        }
        uint8_t *dst = codes + to * D + piece.first;
        if constexpr (E == 8) {
            if (kLayout == kInterleaved) {
                *reinterpret_cast<uint2 *>(dst) = make_uint2(c[0], c[1]);
            } else {
                *reinterpret_cast<uint32_t *>(dst) = c[0];
                *reinterpret_cast<uint32_t *>(dst + apart) = c[1];
            }
        } else {
            if (kLayout == kInterleaved) {
                *reinterpret_cast<uint32_t *>(dst) = c[0];
            } else {
                *reinterpret_cast<uint16_t *>(dst) = (uint16_t)c[0];
                *reinterpret_cast<uint16_t *>(dst + apart) = (uint16_t)(c[0] >> 16);
            }
        }
    }
    if (run.written != 0xffffu && (fresh || e != has)) {
        // the group's other tokens, 4 features a lane
        const float down = scale_ratio(has, e);
#pragma unroll 1
        for (int r = lane / (D / 4); r < kGroup; r += 128 / D) {
            if (run.written >> r & 1u) continue;
            uint32_t *at = reinterpret_cast<uint32_t *>(codes + r * D) + lane % (D / 4);
            uint32_t v = 0;
            if (!fresh) {
                float f[4];
                decode4(*at, f);
                v = encode4(f[0] * down, f[1] * down, f[2] * down, f[3] * down);
            }
            *at = v;
        }
    }
    if (lane == 0 && (fresh || e != has)) *scale = scale_value(e);
}

template <typename T, int D, Layout kLayout>
__global__ __launch_bounds__(kThreads, 2) void k_cache_quant(const RopeArgs a, int window)
{
    __shared__ float2 s_angles[kGroup * kMaxPairs];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int t0 = blockIdx.x * window, t1 = min(t0 + window, a.n_tok);
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    for (int t = t0; t < t1; ++t) {
        // the run that begins at token t
        // tokens t ... t + 15, and in the upper lanes t - 16 ... t - 1
        const int token = lane < kGroup ? t + lane : t - 32 + lane;
        Run run;
        run.slot = token >= 0 && token < a.n_tok ? __ldg(a.slots + token) : -1;
        const int of = run.slot >= 0 && run.slot < a.n_pages * a.page_size ? run.slot / kGroup : -1;
        const int group = __shfl_sync(0xffffffffu, of, 0);
        if (group < 0) {
            if (tid == 0 && run.slot >= 0) raise_error(a.err, ERR_BAD_INDEX);
            continue;
        }
        // no token of the group in the 15 before, up to the last one of another group
        const unsigned same = __ballot_sync(0xffffffffu, of == group), other = __ballot_sync(0xffffffffu, of >= 0 && of != group);
        const unsigned before = other >> 16;
        if ((same >> 17 & ~0u << (before ? 31 - __clz(before) : 0)) != 0) continue;
        run.members = same & 0xffffu & ((other & 0xffffu) != 0 ? (1u << (__ffs(other) - 1)) - 1 : 0xffffu);
        run.t = t;
        run.n = 32 - __clz(run.members);
        run.written = __reduce_or_sync(0xffffffffu, lane < kGroup && run.has(lane) ? 1u << run.slot % kGroup : 0u);
        run.page = group * kGroup / a.page_size;
        run.off = group * kGroup - run.page * a.page_size;
        const int half = a.rot >> 1;
        if (half > 0) {
            __syncthreads();                        // the last run's have been read
            for (int x = tid; x < run.n * kMaxPairs; x += kThreads) {
                const int pair = x % kMaxPairs;
                if (pair < half && run.has(x / kMaxPairs)) s_angles[x] = angle(a, t + x / kMaxPairs, pair);
            }
            __syncthreads();
        }
        for (int x = blockIdx.y * kWarps + warp; x < 2 * a.Hkv; x += gridDim.y * kWarps) {
            if (x < a.Hkv) write_head<T, D, kLayout, true>(a, run, x, s_angles);
            else write_head<T, D, kInterleaved, false>(a, run, x - a.Hkv, s_angles);
        }
    }
}

template <typename T, int D, Layout kLayout> cudaError_t launch_write(const RopeArgs &a, cudaStream_t st)
{
    // A block to a token while the GPU holds them (each may be a run of its own), else windows
    // of up to 16, in which about one run of a prompt begins.
    const int held = 2 * pipe::sm_count();
    int window = (a.n_tok + held - 1) / held;
    if (window > kGroup) window = kGroup;
    const int blocks = (a.n_tok + window - 1) / window, rounds = (2 * a.Hkv + kWarps - 1) / kWarps;
    int y = held / blocks;
    y = y < 1 ? 1 : (y > rounds ? rounds : y);
    return pipe::launch_early(k_cache_quant<T, D, kLayout>, dim3(blocks, y), dim3(kThreads), 0, st, a, window);
}
template <typename T, int D> cudaError_t launch_write(const RopeArgs &a, cudaStream_t st)
{
    if (a.interleaved) return launch_write<T, D, kInterleaved>(a, st);
    return a.rot == D ? launch_write<T, D, kAllHalves>(a, st) : launch_write<T, D, kHalves>(a, st);
}

// Reading back: a thread has 8 features of a token's head, of K and of V.
template <typename T, int D> __global__ __launch_bounds__(kThreads) void k_cache_dequant(const DequantArgs a)
{
    constexpr int kPer = D / 8;
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    const size_t total = (size_t)a.n_tok * a.Hkv * kPer;
    for (size_t x = (size_t)blockIdx.x * kThreads + threadIdx.x; x < total; x += (size_t)gridDim.x * kThreads) {
        const int c = (int)(x % kPer);
        const size_t th = x / kPer;
        const int h = (int)(th % a.Hkv), t = (int)(th / a.Hkv);
        const int slot = __ldg(a.slots + t), page = slot / a.page_size;
        const bool there = slot >= 0 && page < a.n_pages;
        if (slot >= 0 && !there) raise_error(a.err, ERR_BAD_INDEX);
        const size_t row = there ? ((size_t)page * a.Hkv + h) * a.page_size + slot % a.page_size : 0;
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (there) {
                const uint2 v = __ldg(reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(y ? a.V_cache : a.K_cache) + row * D + 8 * c));
                const float s = __ldg((y ? a.V_scale : a.K_scale) + row / kGroup);
                float lo[4], hi[4];
                decode4(v.x, lo);
                decode4(v.y, hi);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    f[i] = lo[i] * s;
                    f[i + 4] = hi[i] * s;
                }
            }
            T *out = static_cast<T *>(y ? a.V : a.K) + x * 8;
            if constexpr (sizeof(T) == 2) {
                *reinterpret_cast<uint4 *>(out) = make_uint4(pipe::pack_bf16x2(f[0], f[1]), pipe::pack_bf16x2(f[2], f[3]),
                                                             pipe::pack_bf16x2(f[4], f[5]), pipe::pack_bf16x2(f[6], f[7]));
            } else {
                *reinterpret_cast<float4 *>(out) = make_float4(f[0], f[1], f[2], f[3]);
                *reinterpret_cast<float4 *>(out + 4) = make_float4(f[4], f[5], f[6], f[7]);
            }
        }
    }
}

template <typename T, int D> cudaError_t launch_read(const DequantArgs &a, cudaStream_t st)
{
    const size_t total = (size_t)a.n_tok * a.Hkv * (D / 8), most = (size_t)8 * pipe::sm_count();
    const size_t blocks = (total + kThreads - 1) / kThreads;
    return pipe::launch_early(k_cache_dequant<T, D>, dim3((unsigned)(blocks < most ? blocks : most)), dim3(kThreads), 0, st, a);
}

}  // namespace

cudaError_t launch_qk_norm_rope_cache_quant(hybrid_dtype dt, const RopeArgs &a, cudaStream_t st)
{
    if (a.Q) {
        RopeArgs q = a;                             // the queries alone
        q.K = nullptr;
        q.slots = nullptr;
        const cudaError_t e = launch_qk_norm_rope(dt, q, st);
        if (e != cudaSuccess) return e;
    }
    if (dt == HYBRID_BF16) return a.d == 128 ? launch_write<__nv_bfloat16, 128>(a, st) : launch_write<__nv_bfloat16, 64>(a, st);
    return a.d == 128 ? launch_write<float, 128>(a, st) : launch_write<float, 64>(a, st);
}

cudaError_t launch_cache_dequant(hybrid_dtype dt, const DequantArgs &a, cudaStream_t st)
{
    if (dt == HYBRID_BF16) return a.d == 128 ? launch_read<__nv_bfloat16, 128>(a, st) : launch_read<__nv_bfloat16, 64>(a, st);
    return a.d == 128 ? launch_read<float, 128>(a, st) : launch_read<float, 64>(a, st);
}

}  // namespace hyb
