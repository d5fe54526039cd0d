// paged_attn_tc.cu -- attention over the paged cache on the tensor cores
// (bfloat16; hybrid_paged_attn).
//
// A row tile has up to 128 query rows (tokens x query heads of one key head), the
// M of the products.  For each tile of 128 keys
//     S = Q K^T          bf16, accumulator in Tensor Memory (two buffers)
//     p = 2^(S c - ref)  c = log2(e) / sqrt(d); two threads per row, 64 keys each
//     O += P V           P bf16 in Tensor Memory, V as the MN-major operand
// with a running reference per row instead of the running maximum: ref is the
// maximum when it was last moved, and O and the sum are rescaled only when a
// row's maximum exceeds it by more than 8, so p <= 2^8 and most tiles touch O
// with the products alone.  The two threads of a row lie in different warps (a
// warp reaches one quarter of Tensor Memory's lanes): they agree by one barrier
// vote per tile that no reference has to move, and exchange maxima only if one has.
//
// The cache is read once per row tile by TMA boxes of one page of one head (64
// features x page_size rows, 128-byte swizzle), which land in a ring of K tiles
// and one of V tiles: 5 or 6 slots of 32 KB for d = 128, so that 160 to 192 KB are
// in flight or in use per SM.  (Two rings, because a wait knows a phase by its
// parity alone: each issuer must itself have seen every phase of its slots.)  One block per SM walks its share of all requests' tiles
// (paged_plan.cuh) without a pause between segments: the producers and the issuer
// of S run ahead into the next segment.  With few rows (decoding) the tensor
// pipe works on padding, which costs nothing here: a tile's products take about
// 0.6 us, its bytes 1.5 us at an SM's share of the memory bandwidth.
//
// Keys that no query sees: pages without a visible key are not loaded, scores of
// masked keys are replaced before use, and of V only groups of 16 keys with a
// visible one enter the product, their masked rows zeroed in shared memory, so
// nothing in those places (NaN included) reaches the output.
//
// Warps: 0-7 softmax and epilogue (warp w: rows 32 (w % 4) ..., half w / 4 of the
// keys and of the output's features; warps beyond the rows idle), 8 and 9
// producers of K (with Q) and V, 10 and 11 issuers of S and O.  Every wait is bounded (tc_pipeline.cuh).
#include <atomic>

#include "paged_plan.cuh"
#include "tc_pipeline.cuh"

namespace hyb {
namespace {

using namespace paged;
using namespace pipe;

constexpr int kParts = 2;                 // threads per row: each has kTile / kParts keys
constexpr int kSoftWarps = 4 * kParts;
constexpr int kThreads = 32 * (kSoftWarps + 4);
constexpr int kLoadK = kSoftWarps, kLoadV = kSoftWarps + 1, kIssueS = kSoftWarps + 2, kIssueO = kSoftWarps + 3;
constexpr int kSmemLimit = 232448;
constexpr int kMaxSlots = 12;
constexpr uint32_t kBarBytes = 1024;      // barriers, TMEM address, failure flag, the plan's scratch
constexpr float kSlack = 8.f;             // log2 of the largest p

struct TcArgs {
    CUtensorMap tmQ, tmK, tmV;
    PagedArgs p;
    int NK, NV;                           // slots of the K ring, then of the V ring
    uint32_t q_bytes;                     // one Q buffer
    uint32_t off_ring, off_bar, bytes;
};

// As wait_bar, but reads the timer only after some tries: its latency would delay
// the common short wait.
__device__ __forceinline__ bool wait_soon(uint64_t *bar, uint32_t parity, volatile int *fail)
{
    for (int i = 0; i < 32; ++i)
        if (ptx::mbar_try_wait(bar, parity)) return true;
    return wait_bar(bar, parity, fail);
}

// Position in a ring: slot and phase of the next item.
struct RingPos {
    uint32_t slot, phase;
    __device__ void step(uint32_t n_slots)
    {
        if (++slot == n_slots) {
            slot = 0;
            phase ^= 1u;
        }
    }
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
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, NK = ta.NK, NV = ta.NV;
    const int rows = a.Bt * a.Gt, n_quads = (rows + 31) / 32;  // quarters of the lanes with rows
    const int n_soft = n_quads * kParts;                       // softmax warps at work

    uint8_t *ring = smem + ta.off_ring;
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem + ta.off_bar);
    uint64_t *full = bars;               // [NK + NV] the K or V tile has landed
    uint64_t *empty = full + kMaxSlots;  // [NK + NV] its products are done
    uint64_t *qfull = empty + kMaxSlots; // [2]
    uint64_t *qempty = qfull + 2;        // [2] the segment's last S is formed
    uint64_t *sready = qempty + 2;       // [2] S is formed
    uint64_t *sfree = sready + 2;        // [2] S has been read
    uint64_t *pready = sfree + 2;        // [2] P is written (and O rescaled, V's masked rows zeroed)
    uint64_t *pvdone = pready + 2;       // [2] O includes the tile's P V
    uint64_t *ofree = pvdone + 2;        // the epilogue has read O
    uint64_t *drained = ofree + 1;       // [2] every MMA of an issuer has completed
    uint32_t *tmem_holder = reinterpret_cast<uint32_t *>(drained + 2);
    volatile int *fail = reinterpret_cast<volatile int *>(tmem_holder + 1);
    PlanSmem *plan_smem = reinterpret_cast<PlanSmem *>(tmem_holder + 2);
    float *exchange = reinterpret_cast<float *>(smem + ta.off_bar + kBarBytes);   // [kParts][128]

    if (warp == kIssueS) {
        tmem_alloc(tmem_holder, 512);
        tmem_relinquish();
    }
    if (warp == kLoadK && lane == 0) {
        prefetch_tensormap(&ta.tmQ);
        prefetch_tensormap(&ta.tmK);
        prefetch_tensormap(&ta.tmV);
        for (int i = 0; i < NK + NV; ++i) {
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
        mbar_init(&drained[0], 1);
        mbar_init(&drained[1], 1);
        *fail = 0;
        fence_mbar_init();
    }
    // what comes before in the stream is complete from here on
    griddep_wait();
    griddep_launch_dependents();
    tc_fence_before();
    Walk w;
    Shares sh(0, 1);
    const bool work = find_share<kThreads>(a, *plan_smem, w, sh);   // synchronises the block
    tc_fence_after();
    const uint32_t tmem = *tmem_holder;
    const long long M = units_per_request(a);

    if (work && (warp == kLoadK || warp == kLoadV)) {
        // ------------------------------------------- producers: Q and K; V
        const bool is_v = warp == kLoadV;
        const int P = a.page_size, per = kTile / P;        // pages of a tile
        const uint32_t page_bytes = (uint32_t)P * D * 2, n_slots = is_v ? NV : NK;
        const CUtensorMap *map = is_v ? &ta.tmV : &ta.tmK;
        uint64_t *my_full = is_v ? full + NK : full, *my_empty = is_v ? empty + NK : empty;
        uint8_t *my_ring = is_v ? ring + (size_t)NK * kSlot : ring;
        uint32_t n = 0, ns = 0;                            // tiles and segments issued
        RingPos pos{0, 1};                                 // phase of `empty`: the first round is free
        bool ok = true;
        while (ok && w.next(a, M)) {
            const Unit u = unit_of(a, w.m);
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
            if (!is_v) {
                const uint32_t qb = ns & 1;
                ok = wait_soon(&qempty[qb], ((ns >> 1) & 1u) ^ 1u, fail);
                if (__any_sync(0xffffffffu, !ok)) break;
                if (lane == 0) {
                    const uint32_t panel = ta.q_bytes / kHalves;
                    mbar_arrive_expect_tx(&qfull[qb], (uint32_t)rows * D * 2);
#pragma unroll
                    for (int h = 0; h < kHalves; ++h)
                        tma_load_4d(smem + qb * ta.q_bytes + h * panel, &ta.tmQ, 64 * h, u.head * a.G + u.g0, u.i0,
                                    w.req, &qfull[qb]);
                }
                ++ns;
            }
            for (int i = w.i0; i < w.i1; ++i) {
                const int page = next_page;
                next_page = page_at(i + 1);                // a tile ahead of its use
                const uint32_t bytes = page_bytes * __popc(__ballot_sync(0xffffffffu, page >= 0));
                ok = wait_soon(&my_empty[pos.slot], pos.phase, fail);
                if (__any_sync(0xffffffffu, !ok)) {
                    ok = false;
                    break;
                }
                if (lane == 0) mbar_arrive_expect_tx(&my_full[pos.slot], bytes);
                __syncwarp();
                if (page >= 0) {
                    uint8_t *dst = my_ring + (size_t)pos.slot * kSlot + lane * P * 128;
#pragma unroll
                    for (int h = 0; h < kHalves; ++h)
                        tma_load_4d(dst + h * kPanel, map, 64 * h, 0, u.head, page, &my_full[pos.slot]);
                }
                pos.step(n_slots);
                ++n;
            }
        }
        if (*fail && lane == 0) {
            // let copies in flight land before the block exits
            auto land = [&](uint64_t *bar, uint32_t slots, uint32_t items) {
                for (uint32_t s = 0; s < slots; ++s) {
                    const uint32_t k = items / slots + (s < items % slots ? 1u : 0u);
                    if (k) mbar_wait(&bar[s], (k - 1) & 1u, kWaitNs);
                }
            };
            land(my_full, n_slots, n);
            land(qfull, 2, ns);
        }
    } else if (work && warp == kIssueS) {
        // ------------------------------------------------------ issuer of S = Q K^T
        if (lane == 0) {
            const uint32_t id = instr_desc(FMT_BF16, FMT_BF16, false, false, 128, kTile);
            const uint64_t q_desc = smem_desc(smem_u32(smem), 16, 1024, SWZ_128B);
            const uint64_t k_desc = smem_desc(smem_u32(ring), 16, 1024, SWZ_128B);
            const uint32_t q_panel = ta.q_bytes / kHalves;
            uint32_t n = 0, seg = 0;                       // tiles and segments so far
            RingPos pos{0, 0};
            bool ok = true;
            while (ok && w.next(a, M)) {
                const uint32_t qb = seg & 1;
                const uint64_t aq = q_desc + qb * (ta.q_bytes >> 4);
                ok = wait_soon(&qfull[qb], (seg >> 1) & 1u, fail);
                for (int i = w.i0; ok && i < w.i1; ++i, ++n) {
                    const uint32_t b = n & 1;
                    ok = wait_soon(&sfree[b], ((n >> 1) & 1u) ^ 1u, fail) && wait_soon(&full[pos.slot], pos.phase, fail);
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t bk = k_desc + pos.slot * (kSlot >> 4);
#pragma unroll
                    for (int k = 0; k < D / 16; ++k)
                        mma_bf16_ss(tmem + cS + 128 * b, aq + (k >> 2) * (q_panel >> 4) + (k & 3) * 2,
                                    bk + (k >> 2) * (kPanel >> 4) + (k & 3) * 2, id, k > 0);
                    mma_commit(&sready[b]);
                    mma_commit(&empty[pos.slot]);
                    if (i + 1 == w.i1) mma_commit(&qempty[qb]);
                    pos.step(NK);
                }
                ++seg;
            }
            mma_commit(&drained[0]);
            mbar_wait(&drained[0], 0, kWaitNs);
        }
    } else if (work && warp == kIssueO) {
        // ------------------------------------------------------ issuer of O += P V
        if (lane == 0) {
            const uint32_t id = instr_desc(FMT_BF16, FMT_BF16, false, true, 128, D);
            const uint64_t v_desc = smem_desc(smem_u32(ring), kPanel, 1024, SWZ_128B);
            uint32_t n = 0, seg = 0;
            RingPos pos{0, 0};
            bool ok = true;
            while (ok && w.next(a, M)) {
                // O is overwritten by a segment's first product: the last epilogue has read it
                if (seg > 0) ok = wait_soon(ofree, (seg - 1) & 1u, fail);
                for (int i = w.i0; ok && i < w.i1; ++i, ++n) {
                    const uint32_t b = n & 1;
                    const int j = key_tile(w.vis, i) * kTile;
                    ok = wait_soon(&full[NK + pos.slot], pos.phase, fail) && wait_soon(&pready[b], (n >> 1) & 1u, fail);
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t bv = v_desc + (NK + pos.slot) * (kSlot >> 4);
                    if (all_visible(w.vis, j)) {
#pragma unroll
                        for (int g = 0; g < kTile / 16; ++g)
                            mma_bf16_ts(tmem + cO, tmem + cP + 64 * b + 8 * g, bv + g * (2048 >> 4), id,
                                        g > 0 || i > w.i0);
                    } else {
                        uint32_t acc = i > w.i0;
                        for (int g = 0; g < kTile / 16; ++g) {
                            if (!any_visible(w.vis, j + 16 * g, 16)) continue;
                            mma_bf16_ts(tmem + cO, tmem + cP + 64 * b + 8 * g, bv + g * (2048 >> 4), id, acc);
                            acc = 1;
                        }
                    }
                    mma_commit(&pvdone[b]);
                    mma_commit(&empty[NK + pos.slot]);
                    pos.step(NV);
                }
                ++seg;
            }
            mma_commit(&drained[1]);
            mbar_wait(&drained[1], 0, kWaitNs);
        }
    } else if (work && (warp & 3) < n_quads) {
        // --------------------------------------------------- softmax, epilogue
        constexpr int kKeys = kTile / kParts, kFeat = D / kParts;   // this thread's keys and features
        const int quad = warp & 3, part = warp >> 2, row = 32 * quad + lane;
        const int worker = 32 * (part * n_quads + quad) + lane;     // among the threads at work
        const uint32_t lane_off = (uint32_t)(32 * quad) << 16;
        const uint32_t pair_bar = 1 + quad;                         // the kParts warps of these rows
        const float to_log2 = kLog2e * rsqrtf((float)D);
        float *mine = exchange + part * 128 + row, *row_x = exchange + row;
        uint32_t n = 0;                                    // tiles so far
        bool bad = false;                                  // a wait gave up: leave at the next vote
        auto wait = [&](uint64_t *bar, uint32_t parity) {
            bad = __any_sync(0xffffffffu, bad || !wait_soon(bar, parity, fail));
        };
        while (w.next(a, M)) {              // left by a vote only, so that the warps of a row stay together
            const Unit u = unit_of(a, w.m);
            float ref = 0.f, l2[2] = {0.f, 0.f};           // the row's sum over this thread's keys, in two
            bool left = false;
            for (int i = w.i0; i < w.i1; ++i, ++n) {
                const uint32_t b = n & 1;
                const int j0 = key_tile(w.vis, i) * kTile;
                const bool edge = !all_visible(w.vis, j0), first = i == w.i0;
                if (edge) {
                    // masked rows of V in the groups that enter the product.  (An earlier
                    // tile's product first, so that the slot's last item has landed and the
                    // wait cannot take its phase for this one's.)
                    if (n >= 2) wait(&pvdone[b], ((n - 2) >> 1) & 1u);
                    const uint32_t slot = NK + n % NV;
                    wait(&full[slot], (n / NV) & 1u);
                    for (int c = worker; c < kTile; c += 32 * n_soft) {
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
                wait(&sready[b], (n >> 1) & 1u);
                tc_fence_after();
                float s[kKeys / 32][32];
#pragma unroll
                for (int x = 0; x < kKeys / 32; ++x)
                    tmem_ld32(tmem + cS + 128 * b + kKeys * part + 32 * x + lane_off, s[x]);
                tmem_wait_ld();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sfree[b]);
                if (edge) {
#pragma unroll
                    for (int x = 0; x < kKeys / 32; ++x)
#pragma unroll
                        for (int y = 0; y < 32; ++y)
                            if (!key_visible(w.vis, j0 + kKeys * part + 32 * x + y)) s[x][y] = -INFINITY;
                }
                float mx4[4] = {s[0][0], s[0][1], s[0][2], s[0][3]};
#pragma unroll
                for (int x = 0; x < kKeys / 32; ++x)
#pragma unroll
                    for (int y = 0; y < 32; ++y) mx4[y & 3] = fmaxf(mx4[y & 3], s[x][y]);
                float mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3])) * to_log2;
                bool rescale = false;
                float f = 1.f;
                if (group_sync_failed(pair_bar, 32 * kParts, bad || first || (row < rows && mx > ref + kSlack))) {
                    *mine = mx;
                    if (group_sync_failed(pair_bar, 32 * kParts, bad)) {
                        left = true;
                        break;
                    }
#pragma unroll
                    for (int x = 0; x < kParts; ++x) mx = fmaxf(mx, row_x[x * 128]);
                    if (first) {
                        ref = mx == -INFINITY ? 0.f : mx;
                    } else if (mx > ref + kSlack) {
                        f = ex2(ref - mx);
                        ref = mx;
                    }
                    rescale = __any_sync(0xffffffffu, row < rows && f != 1.f);
                }
                // P's buffer is free, and O is at rest, once earlier products are done
                if (rescale || n >= 2) {
                    const uint32_t k = rescale ? n - 1 : n - 2;
                    wait(&pvdone[k & 1], (k >> 1) & 1u);
                    tc_fence_after();
                }
                if (rescale) {
                    l2[0] *= f;
                    l2[1] *= f;
#pragma unroll 1
                    for (int x = 0; x < kFeat / 32; ++x) {
                        const uint32_t at = tmem + cO + kFeat * part + 32 * x + lane_off;
                        float o[32];
                        tmem_ld32(at, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int y = 0; y < 32; ++y) o[y] *= f;
                        tmem_st32(at, o);
                    }
                }
#pragma unroll
                for (int h = 0; h < kKeys / 64; ++h) {
                    float p[32];                           // pairs of bf16
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int y = 0; y < 32; y += 2) {
                            const float p0 = ex2(fmaf(s[2 * h + x][y], to_log2, -ref));
                            const float p1 = ex2(fmaf(s[2 * h + x][y + 1], to_log2, -ref));
                            l2[0] += p0;
                            l2[1] += p1;
                            p[16 * x + y / 2] = __uint_as_float(pack_bf16x2(p0, p1));
                        }
                    tmem_st32(tmem + cP + 64 * b + (kKeys / 2) * part + 32 * h + lane_off, p);
                }
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0 && !bad) mbar_arrive(&pready[b]);
            }
            if (left) break;
            // the segment's output: the row's sum from its threads, then O
            group_sync_failed(pair_bar, 32 * kParts, false);       // the exchanged maxima have been read
            *mine = l2[0] + l2[1];
            group_sync_failed(pair_bar, 32 * kParts, false);
            float l = 0.f;
#pragma unroll
            for (int x = 0; x < kParts; ++x) l += row_x[x * 128];
            wait(&pvdone[(n - 1) & 1], ((n - 1) >> 1) & 1u);
            tc_fence_after();
            size_t at;
            const bool live = row_at(a, w.req, u, row, at) && !bad, whole = w.whole();
            bf16 *out = static_cast<bf16 *>(a.O) + at + kFeat * part;
            float *partial = a.part + w.slot() * partial_floats(rows, D);
            const float inv = 1.f / l;
            if (!whole && row < rows && part == 0) {
                partial[row] = ref;
                partial[rows + row] = l;
            }
#pragma unroll 1
            for (int x = 0; x < kFeat / 32; ++x) {
                float o[32];
                tmem_ld32(tmem + cO + kFeat * part + 32 * x + lane_off, o);
                tmem_wait_ld();
                if (x == kFeat / 32 - 1) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0 && !bad) mbar_arrive(ofree);
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
                    float *po = partial + 2 * rows + (size_t)(kFeat * part + 32 * x) * rows + row;
#pragma unroll
                    for (int y = 0; y < 32; ++y) po[(size_t)y * rows] = o[y];
                }
            }
        }
        if (tid == 0 && *fail) raise_error(a.err, ERR_WAIT_TIMEOUT);
        if (worker == 0) write_note(a, true, w, sh);
    }
    if (!work && tid == 0) write_note(a, false, w, sh);
    write_empty<bf16, kThreads>(a, tid);
    __syncthreads();
    if (warp == kIssueS) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

template <int D> cudaError_t launch(const PagedArgs &a, cudaStream_t st)
{
    TcArgs ta;
    ta.p = a;
    const int rows = a.Bt * a.Gt;
    // Q buffers (two), K/V ring, barriers, exchange, and 1 KB for alignment
    ta.q_bytes = (uint32_t)((rows + 7) / 8) * 1024 * (D / 64);
    const uint32_t tail = kBarBytes + kParts * 128 * sizeof(float) + 1024, slot = kTile * D * 2;
    int ns = (int)((kSmemLimit - tail - 2 * ta.q_bytes) / slot);
    if (ns > kMaxSlots) ns = kMaxSlots;
    ta.NK = (ns + 1) / 2;
    ta.NV = ns / 2;
    ta.off_ring = 2 * ta.q_bytes;
    ta.off_bar = ta.off_ring + ns * slot;
    ta.bytes = ta.off_bar + tail;
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
    return pipe::launch_early(k_paged_attn_tc<D>, dim3(a.n_cta), dim3(kThreads), ta.bytes, st, ta);
}

}  // namespace

cudaError_t launch_paged_attn_tc(const PagedArgs &a, cudaStream_t st)
{
    return a.d == 128 ? launch<128>(a, st) : launch<64>(a, st);
}

}  // namespace hyb
