// paged_attn_tc.cu -- attention over the paged cache on the tensor cores
// (bfloat16; hybrid_paged_attn).
//
// A row tile has up to 128 query rows (tokens x query heads of one key head), the
// M of the products.  For each tile of 128 keys
//     S = Q K^T          bf16, accumulator in Tensor Memory (two buffers)
//     p = 2^(S c - ref)  c = log2(e) / sqrt(d); one thread per row
//     O += P V           P bf16 in Tensor Memory, V as the MN-major operand
// with a running reference per row instead of the running maximum: ref is the
// maximum when it was last moved, and O and the sum are rescaled only when a
// row's maximum exceeds it by more than 8, so p <= 2^8 and most tiles touch O
// with the products alone.
//
// The cache is read once per row tile by TMA boxes of one page of one head (64
// features x page_size rows, 128-byte swizzle), which land in a ring of K and V
// tiles: 5 or 6 slots of 32 KB for d = 128, so that 160 to 192 KB are in flight or
// in use per SM.  One block per SM walks its share of all requests' tiles
// (paged_plan.cuh) without a pause between segments: the producer and the MMA
// issuer run ahead into the next segment.  With few rows (decoding) the tensor
// pipe works on padding, which costs nothing here: a tile's products take about
// 0.6 us, its bytes 1.5 us at an SM's share of the memory bandwidth.
//
// Keys that no query sees: pages without a visible key are not loaded, scores of
// masked keys are replaced before use, and of V only groups of 16 keys with a
// visible one enter the product, their masked rows zeroed in shared memory, so
// nothing in those places (NaN included) reaches the output.
//
// Warps: 0-3 softmax and epilogue (row = thread; warps beyond the rows idle),
// 4 producer, 5 MMA issuer.  Every wait is bounded (tc_pipeline.cuh).
#include <atomic>

#include "paged_plan.cuh"
#include "tc_pipeline.cuh"

namespace hyb {
namespace {

using namespace paged;
using namespace pipe;

constexpr int kThreads = 192;
constexpr int kSmemLimit = 232448;
constexpr int kMaxSlots = 12;
constexpr float kSlack = 8.f;             // log2 of the largest p

struct TcArgs {
    CUtensorMap tmQ, tmK, tmV;
    PagedArgs p;
    int NS;                               // ring slots
    uint32_t q_bytes;                     // one Q buffer
    uint32_t off_ring, off_bar, bytes;
};

// Whether the 16 keys from j hold a visible one (for pages, `n` keys from j).
__device__ __forceinline__ bool any_visible(const Visible &v, int j, int n)
{
    return (j < v.len && j + n > v.lo) || j < v.sink;
}
__device__ __forceinline__ bool all_visible(const Visible &v, int j)
{
    return (j >= v.lo && j + kTile <= v.len) || j + kTile <= v.sink;
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1) k_paged_attn_tc(const __grid_constant__ TcArgs ta)
{
    using namespace ptx;
    constexpr int kHalves = D / 64;                        // 64-feature panels of a tile
    constexpr uint32_t kPanel = kTile * 128;               // bytes of one panel of a K or V tile
    constexpr uint32_t kSlot = kHalves * kPanel;
    // Tensor Memory columns: S (2 x 128), P (2 x 64), O
    constexpr uint32_t cS = 0, cP = 256, cO = 384;
    const PagedArgs &a = ta.p;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, NS = ta.NS;
    const int rows = a.Bt * a.Gt, n_soft = (rows + 31) / 32;   // warps with rows

    uint8_t *ring = smem + ta.off_ring;
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem + ta.off_bar);
    uint64_t *full = bars;               // [NS] the K or V tile has landed
    uint64_t *empty = full + kMaxSlots;  // [NS] its products are done
    uint64_t *qfull = empty + kMaxSlots; // [2]
    uint64_t *qempty = qfull + 2;        // [2] the segment's last S is formed
    uint64_t *sready = qempty + 2;       // [2] S is formed
    uint64_t *sfree = sready + 2;        // [2] S has been read
    uint64_t *pready = sfree + 2;        // [2] P is written (and O rescaled, V's masked rows zeroed)
    uint64_t *pvdone = pready + 2;       // [2] O includes the tile's P V
    uint64_t *ofree = pvdone + 2;        // the epilogue has read O
    uint64_t *drained = ofree + 1;       // every MMA has completed
    uint32_t *tmem_holder = reinterpret_cast<uint32_t *>(drained + 1);
    volatile int *fail = reinterpret_cast<volatile int *>(tmem_holder + 1);
    PlanSmem *plan_smem = reinterpret_cast<PlanSmem *>(tmem_holder + 2);

    if (warp == 5) {
        tmem_alloc(tmem_holder, 512);
        tmem_relinquish();
    }
    if (warp == 4 && lane == 0) {
        prefetch_tensormap(&ta.tmQ);
        prefetch_tensormap(&ta.tmK);
        prefetch_tensormap(&ta.tmV);
        for (int i = 0; i < NS; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&qfull[i], 1);
            mbar_init(&qempty[i], 1);
            mbar_init(&sready[i], 1);
            mbar_init(&sfree[i], n_soft);
            mbar_init(&pready[i], n_soft);
            mbar_init(&pvdone[i], 1);
        }
        mbar_init(ofree, n_soft);
        mbar_init(drained, 1);
        *fail = 0;
        fence_mbar_init();
    }
    // what comes before in the stream is complete from here on; the join may start its scan
    griddep_wait();
    griddep_launch_dependents();
    tc_fence_before();
    const Plan plan = make_plan<kThreads>(a, *plan_smem);  // synchronises the block
    tc_fence_after();
    const uint32_t tmem = *tmem_holder;
    const long long M = units_per_request(a), T_all = plan.total * M;
    const int C = T_all < a.n_cta ? (int)T_all : a.n_cta;
    const bool work = (int)blockIdx.x < C;
    Walk w;
    if (work) {
        const long long t0 = share_start(T_all, C, blockIdx.x), t1 = share_start(T_all, C, blockIdx.x + 1);
        int req;
        long long before;
        locate(a, plan, t0, *plan_smem, req, before);
        w.begin(a, t0, t1, req, before);
    }

    if (work && warp == 4) {
        // ------------------------------------------------------------- producer
        const int P = a.page_size, per = kTile / P;        // pages of a tile
        const uint32_t page_bytes = (uint32_t)P * D * 2;
        uint32_t q = 0, ns = 0;                            // ring items and segments issued
        bool ok = true;
        while (ok && w.next(a, M)) {
            const Unit u = unit_of(a, w.m);
            const uint32_t qb = ns & 1;
            ok = wait_bar(&qempty[qb], ((ns >> 1) & 1u) ^ 1u, fail);
            if (__any_sync(0xffffffffu, !ok)) break;
            if (lane == 0) {
                const uint32_t panel = ta.q_bytes / kHalves;
                mbar_arrive_expect_tx(&qfull[qb], (uint32_t)rows * D * 2);
#pragma unroll
                for (int h = 0; h < kHalves; ++h)
                    tma_load_4d(smem + qb * ta.q_bytes + h * panel, &ta.tmQ, 64 * h, u.head * a.G + u.g0, u.i0, w.req,
                                &qfull[qb]);
            }
            ++ns;
            const int *pages = a.table + (size_t)w.req * a.max_pages;
            auto page_at = [&](int i) -> int {             // this lane's page of tile i, -1: nothing visible in it
                if (i >= w.i1 || lane >= per) return -1;
                const int j = key_tile(w.vis, i) * per + lane;
                if (!any_visible(w.vis, j * P, P)) return -1;
                const int page = __ldg(pages + j);
                if (page >= 0 && page < a.n_pages) return page;
                raise_error(a.err, ERR_BAD_INDEX);
                return 0;
            };
            int next_page = page_at(w.i0);
            for (int i = w.i0; i < w.i1; ++i) {
                const int page = next_page;
                next_page = page_at(i + 1);                // a tile ahead of its use
                const uint32_t bytes = page_bytes * __popc(__ballot_sync(0xffffffffu, page >= 0));
#pragma unroll 1
                for (int kv = 0; kv < 2; ++kv) {
                    const int slot = q % NS;
                    ok = wait_bar(&empty[slot], ((q / NS) & 1u) ^ 1u, fail);
                    if (__any_sync(0xffffffffu, !ok)) {
                        ok = false;
                        break;
                    }
                    if (lane == 0) mbar_arrive_expect_tx(&full[slot], bytes);
                    __syncwarp();
                    if (page >= 0) {
                        uint8_t *dst = ring + (size_t)slot * kSlot + lane * P * 128;
#pragma unroll
                        for (int h = 0; h < kHalves; ++h)
                            tma_load_4d(dst + h * kPanel, kv ? &ta.tmV : &ta.tmK, 64 * h, 0, u.head, page, &full[slot]);
                    }
                    ++q;
                }
                if (!ok) break;
            }
        }
        if (*fail && lane == 0) {
            // let copies in flight land before the block exits
            for (int s = 0; s < NS; ++s) {
                const uint32_t n = q / NS + ((uint32_t)s < q % NS ? 1u : 0u);
                if (n) mbar_wait(&full[s], (n - 1) & 1u, kWaitNs);
            }
            for (uint32_t s = 0; s < 2; ++s) {
                const uint32_t n = ns / 2 + (s < ns % 2 ? 1u : 0u);
                if (n) mbar_wait(&qfull[s], (n - 1) & 1u, kWaitNs);
            }
        }
    } else if (work && warp == 5) {
        // ----------------------------------------------------------- MMA issuer
        if (lane == 0) {
            const uint32_t id_s = instr_desc(FMT_BF16, FMT_BF16, false, false, 128, kTile);
            const uint32_t id_o = instr_desc(FMT_BF16, FMT_BF16, false, true, 128, D);
            const uint32_t ring_u = smem_u32(ring), q_u = smem_u32(smem), q_panel = ta.q_bytes / kHalves;
            uint32_t n = 0, seg = 0;                       // tiles and segments whose S was issued
            // the tile whose P V is still to be issued
            bool have = false, pv_first = false, pv_last = false;
            uint32_t pv_n = 0, pv_seg = 0, pv_groups = 0;
            // O += P V of the pending tile
            auto issue_pv = [&]() -> bool {
                const uint32_t b = pv_n & 1, item = 2 * pv_n + 1, slot = item % NS;
                // O is overwritten by a segment's first product: the last epilogue has read it
                if (pv_first && pv_seg > 0 && !wait_bar(ofree, (pv_seg - 1) & 1u, fail)) return false;
                if (!wait_bar(&pready[b], (pv_n >> 1) & 1u, fail)) return false;
                if (!wait_bar(&full[slot], (item / NS) & 1u, fail)) return false;
                tc_fence_after();
                uint32_t acc = pv_first ? 0u : 1u;
                for (int g = 0; g < kTile / 16; ++g) {
                    if (!(pv_groups >> g & 1u)) continue;
                    const uint64_t bv = smem_desc(ring_u + slot * kSlot + g * 2048, kPanel, 1024, SWZ_128B);
                    mma_bf16_ts(tmem + cO, tmem + cP + 64 * b + 8 * g, bv, id_o, acc);
                    acc = 1;
                }
                mma_commit(&empty[slot]);
                mma_commit(&pvdone[b]);
                return true;
            };
            bool ok = true;
            while (ok && w.next(a, M)) {
                const uint32_t qb = seg & 1;
                ok = wait_bar(&qfull[qb], (seg >> 1) & 1u, fail);
                for (int i = w.i0; ok && i < w.i1; ++i) {
                    const uint32_t b = n & 1, item = 2 * n, slot = item % NS;
                    if (!wait_bar(&sfree[b], ((n >> 1) & 1u) ^ 1u, fail) ||
                        !wait_bar(&full[slot], (item / NS) & 1u, fail)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint64_t aq =
                            smem_desc(q_u + qb * ta.q_bytes + (k >> 2) * q_panel + (k & 3) * 32, 16, 1024, SWZ_128B);
                        const uint64_t bk =
                            smem_desc(ring_u + slot * kSlot + (k >> 2) * kPanel + (k & 3) * 32, 16, 1024, SWZ_128B);
                        mma_bf16_ss(tmem + cS + 128 * b, aq, bk, id_s, k > 0);
                    }
                    mma_commit(&empty[slot]);
                    mma_commit(&sready[b]);
                    if (i + 1 == w.i1) mma_commit(&qempty[qb]);
                    if (have) ok = issue_pv();
                    const int j = key_tile(w.vis, i) * kTile;
                    pv_groups = 0;
                    for (int g = 0; g < kTile / 16; ++g)
                        pv_groups |= (any_visible(w.vis, j + 16 * g, 16) ? 1u : 0u) << g;
                    have = true;
                    pv_first = i == w.i0;
                    pv_n = n++;
                    pv_seg = seg;
                }
                ++seg;
            }
            if (ok && have) issue_pv();
            mma_commit(drained);
            mbar_wait(drained, 0, kWaitNs);
            (void)pv_last;
        }
    } else if (work && warp < n_soft) {
        // --------------------------------------------------- softmax, epilogue
        const int row = tid;
        const uint32_t lane_off = (uint32_t)(32 * warp) << 16;
        const float to_log2 = kLog2e * rsqrtf((float)D);
        uint32_t n = 0;                                    // tiles so far
        bool ok = true;
        while (ok && w.next(a, M)) {
            const Unit u = unit_of(a, w.m);
            float ref = -INFINITY, l = 0.f;
            for (int i = w.i0; i < w.i1; ++i, ++n) {
                const uint32_t b = n & 1;
                const int j0 = key_tile(w.vis, i) * kTile;
                const bool edge = !all_visible(w.vis, j0);
                if (edge) {
                    // masked rows of V in the groups that enter the product
                    const uint32_t item = 2 * n + 1, slot = item % NS;
                    ok = wait_bar(&full[slot], (item / NS) & 1u, fail);
                    if (__any_sync(0xffffffffu, !ok)) { ok = false; break; }
                    for (int c = tid; c < kTile; c += 32 * n_soft) {
                        const int j = j0 + c;
                        if (!key_visible(w.vis, j) && any_visible(w.vis, j & ~15, 16)) {
#pragma unroll
                            for (int x = 0; x < kHalves * 8; ++x)
                                *reinterpret_cast<uint4 *>(ring + (size_t)slot * kSlot + (x >> 3) * kPanel + c * 128 +
                                                           (x & 7) * 16) = make_uint4(0, 0, 0, 0);
                        }
                    }
                    fence_proxy_async_smem();
                }
                ok = wait_bar(&sready[b], (n >> 1) & 1u, fail);
                if (__any_sync(0xffffffffu, !ok)) { ok = false; break; }
                tc_fence_after();
                float s[4][32];
#pragma unroll
                for (int x = 0; x < 4; ++x) tmem_ld32(tmem + cS + 128 * b + 32 * x + lane_off, s[x]);
                tmem_wait_ld();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sfree[b]);
                if (edge) {
#pragma unroll
                    for (int x = 0; x < 4; ++x)
#pragma unroll
                        for (int y = 0; y < 32; ++y)
                            if (!key_visible(w.vis, j0 + 32 * x + y)) s[x][y] = -INFINITY;
                }
                float mx = -INFINITY;
#pragma unroll
                for (int x = 0; x < 4; ++x)
#pragma unroll
                    for (int y = 0; y < 32; ++y) mx = fmaxf(mx, s[x][y]);
                mx *= to_log2;
                float f = 1.f;
                if (i == w.i0) {
                    ref = mx == -INFINITY ? 0.f : mx;
                } else if (mx > ref + kSlack) {
                    f = ex2(ref - mx);
                    ref = mx;
                }
                const bool rescale = __any_sync(0xffffffffu, row < rows && f != 1.f);
                // P's buffer is free, and O is at rest, once earlier products are done
                if (rescale || n >= 2) {
                    const uint32_t k = rescale ? n - 1 : n - 2;
                    ok = wait_bar(&pvdone[k & 1], (k >> 1) & 1u, fail);
                    if (__any_sync(0xffffffffu, !ok)) { ok = false; break; }
                    tc_fence_after();
                }
                if (rescale) {
                    l *= f;
#pragma unroll 1
                    for (int x = 0; x < D / 32; ++x) {
                        float o[32];
                        tmem_ld32(tmem + cO + 32 * x + lane_off, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int y = 0; y < 32; ++y) o[y] *= f;
                        tmem_st32(tmem + cO + 32 * x + lane_off, o);
                    }
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float p[32];                           // pairs of bf16
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int y = 0; y < 32; y += 2) {
                            const float p0 = ex2(fmaf(s[2 * h + x][y], to_log2, -ref));
                            const float p1 = ex2(fmaf(s[2 * h + x][y + 1], to_log2, -ref));
                            l += p0 + p1;
                            p[16 * x + y / 2] = __uint_as_float(pack_bf16x2(p0, p1));
                        }
                    tmem_st32(tmem + cP + 64 * b + 32 * h + lane_off, p);
                }
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&pready[b]);
            }
            if (!ok) break;
            // the segment's output
            ok = wait_bar(&pvdone[(n - 1) & 1], ((n - 1) >> 1) & 1u, fail);
            if (__any_sync(0xffffffffu, !ok)) { ok = false; break; }
            tc_fence_after();
            size_t at;
            const bool live = row_at(a, w.req, u, row, at), whole = w.whole();
            bf16 *out = static_cast<bf16 *>(a.O) + at;
            float *part = a.part + (size_t)(2 * blockIdx.x + (w.at_start ? 0 : 1)) * partial_floats(rows, D);
            const float inv = 1.f / l;
            if (!whole && row < rows) {
                part[row] = ref;
                part[rows + row] = l;
            }
#pragma unroll 1
            for (int x = 0; x < D / 32; ++x) {
                float o[32];
                tmem_ld32(tmem + cO + 32 * x + lane_off, o);
                tmem_wait_ld();
                if (x == D / 32 - 1) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(ofree);
                }
                if (whole) {
                    if (live) {
#pragma unroll
                        for (int y = 0; y < 32; y += 8)
                            *reinterpret_cast<uint4 *>(out + 32 * x + y) = make_uint4(
                                pack_bf16x2(o[y] * inv, o[y + 1] * inv), pack_bf16x2(o[y + 2] * inv, o[y + 3] * inv),
                                pack_bf16x2(o[y + 4] * inv, o[y + 5] * inv), pack_bf16x2(o[y + 6] * inv, o[y + 7] * inv));
                    }
                } else if (row < rows) {
                    float *po = part + 2 * rows + (size_t)(32 * x) * rows + row;
#pragma unroll
                    for (int y = 0; y < 32; ++y) po[(size_t)y * rows] = o[y];
                }
            }
        }
        if (tid == 0 && *fail) raise_error(a.err, ERR_WAIT_TIMEOUT);
    }
    __syncthreads();
    if (warp == 5) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

template <int D> cudaError_t launch(const PagedArgs &a, cudaStream_t st)
{
    TcArgs ta;
    ta.p = a;
    const int rows = a.Bt * a.Gt;
    // Q buffers (two), K/V ring, barriers and the plan's scratch
    ta.q_bytes = (uint32_t)((rows + 7) / 8) * 1024 * (D / 64);
    const uint32_t bar_bytes = 1024, slot = kTile * D * 2;
    int ns = (int)((kSmemLimit - 1024 - bar_bytes - 2 * ta.q_bytes) / slot);
    if (ns > kMaxSlots) ns = kMaxSlots;
    ta.NS = ns;
    ta.off_ring = 2 * ta.q_bytes;
    ta.off_bar = ta.off_ring + ns * slot;
    ta.bytes = ta.off_bar + bar_bytes + 1024;
    {
        const cuuint64_t dq[4] = {(cuuint64_t)D, (cuuint64_t)a.Hq, (cuuint64_t)a.B, (cuuint64_t)a.n_req};
        const cuuint64_t sq[3] = {(cuuint64_t)D * 2, (cuuint64_t)a.Hq * D * 2, (cuuint64_t)a.B * a.Hq * D * 2};
        const cuuint32_t bq[4] = {64, (cuuint32_t)a.Gt, (cuuint32_t)a.Bt, 1};
        const cuuint64_t dk[4] = {(cuuint64_t)D, (cuuint64_t)a.page_size, (cuuint64_t)a.Hkv, (cuuint64_t)a.n_pages};
        const cuuint64_t sk[3] = {(cuuint64_t)D * 2, (cuuint64_t)a.page_size * D * 2,
                                  (cuuint64_t)a.Hkv * a.page_size * D * 2};
        const cuuint32_t bk[4] = {64, (cuuint32_t)a.page_size, 1, 1};
        if (!encode_bf16(&ta.tmQ, a.Q, 4, dq, sq, bq) || !encode_bf16(&ta.tmK, a.K, 4, dk, sk, bk) ||
            !encode_bf16(&ta.tmV, a.V, 4, dk, sk, bk))
            return cudaErrorInvalidValue;
    }
    // opt in to the shared memory once per device
    static std::atomic<unsigned long long> opted{0};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    const unsigned long long bit = 1ull << dev;
    if (!(opted.load(std::memory_order_acquire) & bit)) {
        const cudaError_t e =
            cudaFuncSetAttribute(k_paged_attn_tc<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit);
        if (e != cudaSuccess) return e;
        opted.fetch_or(bit, std::memory_order_release);
    }
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3(a.n_cta);
    lc.blockDim = dim3(kThreads);
    lc.dynamicSmemBytes = ta.bytes;
    lc.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = attr;
    lc.numAttrs = 1;
    return cudaLaunchKernelEx(&lc, k_paged_attn_tc<D>, ta);
}

}  // namespace

cudaError_t launch_paged_attn_tc(const PagedArgs &a, cudaStream_t st)
{
    return a.d == 128 ? launch<128>(a, st) : launch<64>(a, st);
}

}  // namespace hyb
