// cache_quant.cu -- the paged cache in 8 bits: keys and values rounded as they are written, with
// the norms and rotations of keys and queries in the same pass (hybrid_qk_norm_rope_cache_quant),
// and tokens read back (hybrid_cache_dequant).  The format is in quant.cuh.
//
// Write.  A scale belongs to 16 tokens of a head, so the tokens of one group that a call writes
// (a run: they stand side by side, but for tokens without a slot) are held together: a warp has a
// run's rows of one head, of K or of V, and
//     y = norm and rotation of x (K),   amax = max |y| over the run
//     E = least power of two with amax <= 448 * 2^E; no less than the group's old one, unless
//         the run has the group's first slot
//     code = e4m3(y / 2^E)
// then brings the group's other tokens to 2^E (zeros where the group starts afresh).  A block has
// a window of the packed tokens: its queries, and the runs that begin in it.  It forms the window's
// angles once; its warps share the pieces of work (a run's head; some steps of queries), and each
// copies the rows of its next piece to shared memory while it works on one (cp.async, a lane
// only what it reads itself).  A run's rows are formed twice, for the maximum and for the codes: that
// costs less than 64 registers a lane to keep them, and loops over the steps instead of unrolled
// ones keep the code within the instruction cache.
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

template <typename T, int D> struct Rows {
    static constexpr int E = Vec<T>::E, L = D / E, RPW = 32 / L;        // elements of a lane, lanes of a row, rows of a step
    static constexpr int kSteps = kGroup / RPW;                         // of a run, and of a piece of queries
    static constexpr int kStage = kSteps * 512;                         // bytes of a warp's rows
    static constexpr int kAngles = (2 * kGroup - 1) * kMaxPairs;
    static constexpr int kBytes = kWarps * 2 * kStage + kAngles * (int)sizeof(float2);
};

// A row's norm (w: the weights, null without) and rotation.
template <int D, int E, bool kInter>
__device__ __forceinline__ void norm_rotate(f32x2 (&x)[E / 2], bool norm, const f32x2 (&w)[E / 2], float eps, bool turn,
                                            const float2 *angles, int pair)
{
    if (norm) {
        f32x2 ss = ptx::mul2(x[0], x[0]);
#pragma unroll
        for (int k = 1; k < E / 2; ++k) ss = ptx::fma2(x[k], x[k], ss);
        const float r = rsqrtf(head_sum<D / E>(both(ss)) * (1.f / D) + eps);
        const f32x2 rr = pair2(r, r);
#pragma unroll
        for (int k = 0; k < E / 2; ++k) x[k] = ptx::mul2(ptx::mul2(x[k], rr), w[k]);
    }
    if (turn) {
        Rotation<E, kInter> rot;
        read_rotation(angles, pair, rot);
        rotate<E, kInter>(x, rot);
    }
}

// One head of a run, K or V (norm and rotation left out), into the cache.  `rows`: this lane's place in its stage;
// `angles`: of the run's first token.
template <typename T, int D, Layout kLayout>
__device__ __forceinline__ void write_head(const RopeArgs &a, const Run &run, bool key, int head, uint32_t rows, const float2 *angles)
{
    using R = Rows<T, D>;
    constexpr int E = R::E;
    const int lane = threadIdx.x & 31, sub = lane / R::L;
    const Pieces<D, E, kLayout> piece(a, lane % R::L);
    const int apart = piece.apart();
    const size_t row = (((size_t)run.page * a.Hkv + head) * a.page_size + run.off);     // the group's first token
    float *scale = (key ? a.K_scale : a.V_scale) + row / kGroup;
    uint8_t *codes = static_cast<uint8_t *>(key ? a.K_cache : a.V_cache) + row * D;
    const bool fresh = run.written & 1u;
    const float old = fresh ? 0.f : *scale;                 // under way beside the arithmetic
    const bool norm = key && a.wk, turn = key && a.rot > 0 && piece.on;
    f32x2 w[E / 2];
    if (norm) Vec<T>::unpack(load<kLayout>(static_cast<const T *>(a.wk) + piece.first, apart), w);
    const int steps = (run.n + R::RPW - 1) / R::RPW;
    // this lane's part of row step * RPW + sub (zeros where the run has none)
    auto form = [&](int step, float (&y)[E]) {
        const int r = step * R::RPW + sub;
        f32x2 x[E / 2];
        Vec<T>::unpack(ring_load(rows + 512 * step), x);
        norm_rotate<D, E, kLayout == kInterleaved>(x, norm, w, a.eps, turn, angles + r * kMaxPairs, piece.pair);
        const bool has = run.has(r);
#pragma unroll
        for (int k = 0; k < E / 2; ++k) {
            ptx::unpair2(x[k], y[2 * k], y[2 * k + 1]);
            if (!has) y[2 * k] = y[2 * k + 1] = 0.f;
        }
    };
    auto magnitude = [](float v) { return __float_as_uint(v) & 0x7fffffffu; };
    // the largest magnitude, as bits; from 0x7f800000 on there are infinities or NaN, which are left out
    uint32_t amax = 0;
#pragma unroll 2
    for (int i = 0; i < steps; ++i) {
        float y[E];
        form(i, y);
#pragma unroll
        for (int k = 0; k < E; ++k) amax = max(amax, magnitude(y[k]));
    }
    amax = __reduce_max_sync(0xffffffffu, amax);
    const bool wild = amax >= 0x7f800000u;
    if (wild) {
        amax = 0;
#pragma unroll 1
        for (int i = 0; i < steps; ++i) {
            float y[E];
            form(i, y);
#pragma unroll
            for (int k = 0; k < E; ++k)
                if (magnitude(y[k]) < 0x7f800000u) amax = max(amax, magnitude(y[k]));
        }
        amax = __reduce_max_sync(0xffffffffu, amax);
    }
    int e = scale_of_amax(amax), has = e;
    if (!fresh) {
        has = scale_of_bits(__float_as_uint(old));
        e = max(e, has);
    }
    const float inv = scale_inverse(e);
#pragma unroll 2
    for (int i = 0; i < steps; ++i) {
        const int r = i * R::RPW + sub, to = __shfl_sync(0xffffffffu, run.slot, r & 31) % kGroup;
        float y[E];
        form(i, y);
        uint32_t c[E / 4];
#pragma unroll
        for (int k = 0; k < E; ++k) {
            if (wild && magnitude(y[k]) >= 0x7f800000u) y[k] = __uint_as_float(0x7fc00000u);
            y[k] *= inv;
        }
#pragma unroll
        for (int k = 0; k < E; k += 4) c[k / 4] = encode4(y[k], y[k + 1], y[k + 2], y[k + 3]);
        if (!run.has(r)) continue;
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

// Steps of queries of a window: step s has RPW heads of its token s / steps.
struct Steps {
    int token, head;
    __device__ Steps(int s, int steps, int rpw, int sub)
    {
        token = s / steps;
        head = (s - token * steps) * rpw + sub;
    }
    __device__ void next(int heads, int rpw, int sub)       // (`head` may lie behind the last: a padded step)
    {
        head += rpw;
        if (head - sub >= heads) {
            head = sub;
            ++token;
        }
    }
};

template <typename T, int D, Layout kLayout>
__global__ __launch_bounds__(kThreads, 2) void k_cache_write(const RopeArgs a, int window)
{
    using R = Rows<T, D>;
    constexpr int E = R::E, RPW = R::RPW;
    extern __shared__ __align__(16) unsigned char s_raw[];
    float2 *s_angles = reinterpret_cast<float2 *>(s_raw + kWarps * 2 * R::kStage);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, sub = lane / R::L;
    const int t0 = blockIdx.x * window, n_win = min(window, a.n_tok - t0);
    const uint32_t stage0 = ptx::smem_u32(s_raw) + warp * (2 * R::kStage) + 16 * lane;
    const Pieces<D, E, kLayout> piece(a, lane % R::L);
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    // Groups of the tokens t0 - 16 ... t0 + 15 and t0 + 16 ... t0 + 31, -1 without a slot; each warp for itself.
    auto slot_at = [&](int t) { return t >= 0 && t < a.n_tok ? __ldg(a.slots + t) : -1; };
    const int slot0 = slot_at(t0 - kGroup + lane), slot1 = lane < kGroup ? slot_at(t0 + kGroup + lane) : -1;
    const int slots = a.n_pages * a.page_size;
    const int of0 = slot0 >= 0 && slot0 < slots ? slot0 / kGroup : -1, of1 = slot1 >= 0 && slot1 < slots ? slot1 / kGroup : -1;
    if (blockIdx.y == 0 && warp == 0 && lane >= kGroup && lane < kGroup + n_win && slot0 >= slots) raise_error(a.err, ERR_BAD_INDEX);
    // A run begins at a token of the window unless the last token with a slot before it, of the 15 before, is of its group.
    const unsigned live = __ballot_sync(0xffffffffu, of0 >= 0);
    const unsigned earlier = live & ((1u << lane) - 1);
    const int last = earlier ? 31 - __clz(earlier) : 0;
    const int group_before = __shfl_sync(0xffffffffu, of0, last);
    const unsigned starts = __ballot_sync(0xffffffffu, of0 >= 0 && lane >= kGroup && lane < kGroup + n_win &&
                                                           !(earlier && lane - last < kGroup && group_before == of0));
    auto run_from = [&](int at) {                           // lane `at` of of0
        Run run;
        const int group = __shfl_sync(0xffffffffu, of0, at), from = at + lane;          // tokens t ... t + 15
        const int g0 = __shfl_sync(0xffffffffu, of0, from & 31), g1 = __shfl_sync(0xffffffffu, of1, from & 31);
        const int s0 = __shfl_sync(0xffffffffu, slot0, from & 31), s1 = __shfl_sync(0xffffffffu, slot1, from & 31);
        const int of = from < 32 ? g0 : g1;
        run.slot = from < 32 ? s0 : s1;
        const unsigned same = __ballot_sync(0xffffffffu, lane < kGroup && of == group);
        const unsigned other = __ballot_sync(0xffffffffu, lane < kGroup && of >= 0 && of != group);
        run.members = other ? same & ((1u << (__ffs(other) - 1)) - 1) : same;
        run.t = t0 + at - kGroup;
        run.n = 32 - __clz(run.members);
        run.written = __reduce_or_sync(0xffffffffu, lane < kGroup && run.has(lane) ? 1u << run.slot % kGroup : 0u);
        run.page = group * kGroup / a.page_size;
        run.off = group * kGroup - run.page * a.page_size;
        return run;
    };
    const int heads = 2 * a.Hkv, n_heads = __popc(starts) * heads;
    const int steps = (a.Hq + RPW - 1) / RPW, n_steps = a.Q ? n_win * steps : 0;
    const int n_work = n_heads + (n_steps + R::kSteps - 1) / R::kSteps;
    // the run of a piece of work that is a head
    auto run_of = [&](int work, int &head) {
        const int nth = work / heads;
        unsigned left = starts;
        for (int x = 0; x < nth; ++x) left &= left - 1;
        head = work - nth * heads;
        return run_from(__ffs(left) - 1);
    };
    // copies of a piece's rows, as one group of them
    auto copy = [&](int work, uint32_t to) {
        if (work < n_heads) {
            int head;
            const Run run = run_of(work, head);
            const bool key = head < a.Hkv;
            const size_t stride = key ? a.k_stride : a.v_stride;
            const T *src = static_cast<const T *>(key ? a.K : a.V) + (size_t)(run.t + sub) * stride +
                           (size_t)(key ? head : head - a.Hkv) * D + piece.first;
#pragma unroll 4
            for (int i = 0; i * RPW < run.n; ++i) {
                copy_async<kLayout>(to + 512 * i, src, piece.apart(), run.has(i * RPW + sub));
                src += RPW * stride;
            }
        } else if (work < n_work) {
            const int s0 = (work - n_heads) * R::kSteps, n = min(R::kSteps, n_steps - s0);
            Steps at(s0, steps, RPW, sub);
#pragma unroll 4
            for (int i = 0; i < n; ++i) {
                const T *src = static_cast<const T *>(a.Q) + (size_t)(t0 + at.token) * a.q_stride + (size_t)at.head * D + piece.first;
                copy_async<kLayout>(to + 512 * i, src, piece.apart(), at.head < a.Hq);
                at.next(a.Hq, RPW, sub);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    int work = blockIdx.y * kWarps + warp, b = 0;
    copy(work, stage0);
    const int half = a.rot >> 1;
    if (half > 0) {
        // the tokens whose angles are used: the window's for queries, the runs' for keys
        int n_angles = a.Q ? n_win : 0;
        if (starts) {
            const Run tail = run_from(31 - __clz(starts));
            n_angles = max(n_angles, tail.t - t0 + tail.n);
        }
        for (int x = tid; x < n_angles * kMaxPairs; x += kThreads) {
            const int pair = x % kMaxPairs;
            if (pair < half) s_angles[x] = angle(a, t0 + x / kMaxPairs, pair);
        }
        __syncthreads();
    }
#pragma unroll 1
    for (; work < n_work; b ^= 1) {
        const int now = work;
        const uint32_t rows = stage0 + b * R::kStage;
        work += gridDim.y * kWarps;
        copy(work, stage0 + (b ^ 1) * R::kStage);
        asm volatile("cp.async.wait_group 1;" ::: "memory");
        if (now < n_heads) {
            int head;
            const Run run = run_of(now, head);
            const bool key = head < a.Hkv;
            write_head<T, D, kLayout>(a, run, key, key ? head : head - a.Hkv, rows, s_angles + (run.t - t0) * kMaxPairs);
        } else {
            const int s0 = (now - n_heads) * R::kSteps, n = min(R::kSteps, n_steps - s0);
            f32x2 w[E / 2];
            if (a.wq) Vec<T>::unpack(load<kLayout>(static_cast<const T *>(a.wq) + piece.first, piece.apart()), w);
            Steps at(s0, steps, RPW, sub);
#pragma unroll 4
            for (int i = 0; i < n; ++i) {
                f32x2 x[E / 2];
                Vec<T>::unpack(ring_load(rows + 512 * i), x);
                norm_rotate<D, E, kLayout == kInterleaved>(x, a.wq, w, a.eps, a.rot > 0 && piece.on, s_angles + at.token * kMaxPairs, piece.pair);
                store<kLayout>(static_cast<T *>(a.Qo) + ((size_t)(t0 + at.token) * a.Hq + at.head) * D + piece.first, piece.apart(),
                               Vec<T>::pack(x), at.head < a.Hq);
                at.next(a.Hq, RPW, sub);
            }
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
    const int blocks = (a.n_tok + window - 1) / window;
    const int steps = a.Q ? (a.Hq + Rows<T, D>::RPW - 1) / Rows<T, D>::RPW * window : 0;
    const int pieces = 2 * a.Hkv + (steps + Rows<T, D>::kSteps - 1) / Rows<T, D>::kSteps, rounds = (pieces + kWarps - 1) / kWarps;
    int y = held / blocks;
    y = y < 1 ? 1 : (y > rounds ? rounds : y);
    static std::atomic<unsigned long long> opted{0};
    const cudaError_t e = pipe::opt_in(reinterpret_cast<const void *>(&k_cache_write<T, D, kLayout>), Rows<T, D>::kBytes, opted);
    if (e != cudaSuccess) return e;
    return pipe::launch_early(k_cache_write<T, D, kLayout>, dim3(blocks, y), dim3(kThreads), Rows<T, D>::kBytes, st, a, window);
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
    if (dt == HYBRID_BF16) return a.d == 128 ? launch_write<__nv_bfloat16, 128>(a, st) : launch_write<__nv_bfloat16, 64>(a, st);
    return a.d == 128 ? launch_write<float, 128>(a, st) : launch_write<float, 64>(a, st);
}

cudaError_t launch_cache_dequant(hybrid_dtype dt, const DequantArgs &a, cudaStream_t st)
{
    if (dt == HYBRID_BF16) return a.d == 128 ? launch_read<__nv_bfloat16, 128>(a, st) : launch_read<__nv_bfloat16, 64>(a, st);
    return a.d == 128 ? launch_read<float, 128>(a, st) : launch_read<float, 64>(a, st);
}

}  // namespace hyb
