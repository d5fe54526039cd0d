// paged_attn_tc.cu -- attention over the paged cache on the tensor cores
// (bfloat16; hybrid_paged_attn).
//
// A row tile has up to 128 query rows (tokens x query heads of one key head), the
// M of the products.  For each tile of 128 keys
//     S = Q K^T          bf16, accumulator in Tensor Memory (two buffers)
//     p = 2^(S c - ref)  c = log2(e) / sqrt(d)
//     O += P V           P bf16 in Tensor Memory, V as the MN-major operand
// with a running reference per row instead of the running maximum: ref is the
// maximum when it was last moved, and O and the sum are rescaled only when a
// row's maximum exceeds it by more than 8, so p <= 2^8 and most tiles touch O
// with the products alone.
//
// A warp reaches one quarter of Tensor Memory's lanes, and the four warps of a
// quarter share one scheduler.  With few rows (decoding) that would leave the whole
// softmax to one scheduler, so the rows are copied: with at most 32 (64) rows, Q
// stands 4 (2) times in the 128 rows of the product, and each copy takes a quarter
// (half) of every tile's keys: it has a reference and a sum of its own, and O is the
// sum of the copies' rows, formed at the end of a segment.  The products of a copy's
// keys with V write its lanes alone: with zeros in the other copies' P instead, an
// infinite V would make NaN of their rows, for the same time (64 requests of 256-8192
// tokens 92.5 us both, 45 requests of 86-249 tokens with 16 key heads 34.5, here 34.7; 39.3
// with a loop for each copy, which the instruction cache does not hold).  The products'
// padding costs nothing: a tile's products take about 0.6 us, its bytes 1.5 us at an SM's share of the memory
// bandwidth.  With more rows, two threads share a row, 64 keys of every tile each, with
// a reference, a sum and an accumulator O of its own; P then takes the place of the S
// it was made from (Tensor Memory holds two S and two O), and the halves are added at
// the end of a segment.  So no warp waits for another between the tiles of a segment.
//
// The cache is read once per row tile by TMA boxes of one page of one head (64
// features x page_size rows, 128-byte swizzle), issued by one warp for K and one
// for V (one warp alone cannot issue the 32 boxes of a tile with pages of 16 in
// time).  They land in a ring of K tiles and one of V tiles, together 5 or 6 slots
// of 32 KB for d = 128, so that 160 to 192 KB are in flight or in use per SM.  (Two
// rings, because a wait knows a phase by its parity alone: each issuer must itself
// have seen every phase of its slots.)  One block per SM walks its share of all
// requests' tiles (paged_plan.cuh) without a pause between segments: the producers
// run ahead into the next segment.
//
// Keys that no query sees: pages without a visible key are not loaded, scores of
// masked keys are replaced before use, and of V only groups of 16 keys with a
// visible one enter the product, their masked rows zeroed in shared memory, so
// nothing in those places (NaN included) reaches the output.
//
// Warps: softmax and epilogue (4 with copies, else 8: warp w reaches the lanes
// 32 (w % 4) ...), producers of K and V, issuers of S (and loads of Q) and of O.
// Every wait is bounded (tc_pipeline.cuh).
#include "paged_plan.cuh"
#include "tc_pipeline.cuh"

namespace hyb {
namespace {

using namespace paged;
using namespace pipe;

constexpr int kSmemLimit = 232448;
constexpr int kMaxSlots = 12;
constexpr uint32_t kBarBytes = 1024;      // barriers, TMEM address, failure flag, the plan's scratch
constexpr uint32_t kExchange = 1024;      // two floats a row
// with copies: 64 inverse sums, and 128 rows of 32 + 4 features (a quarter of the rows: 128 + 4)
constexpr uint32_t kStage = 256 + 128 * 36 * 4;
constexpr float kSlack = 8.f;             // log2 of the largest p

struct TcArgs {
    CUtensorMap tmQ, tmK, tmV;
    PagedArgs p;
    int NK, NV;                           // slots of the K ring, then of the V ring
    uint32_t off_bar, off_stage, bytes;
};

// kCopies: 4, 2 or 1 copies of the rows (at most 32, 64, 128 of them).
template <int kCopies> struct Roles {
    static constexpr int kParts = kCopies == 1 ? 2 : 1;    // threads per row of a copy
    static constexpr int kSoft = 4 * kParts;               // softmax warps
    static constexpr int kLoadK = kSoft, kLoadV = kSoft + 1, kIssueS = kSoft + 2, kIssueO = kSoft + 3;
    static constexpr int kThreads = 32 * (kSoft + 4);
};

template <int D, int kCopies>
__global__ void __launch_bounds__(Roles<kCopies>::kThreads, 1) k_paged_attn_tc(const __grid_constant__ TcArgs ta)
{
    using namespace ptx;
    using W = Roles<kCopies>;
    constexpr int kParts = W::kParts, kThreads = W::kThreads;
    constexpr int kHalves = D / 64;                        // 64-feature panels of a tile
    constexpr uint32_t kPanel = kTile * 128;               // bytes of one panel of a Q, K or V tile
    constexpr uint32_t kSlot = kHalves * kPanel;
    constexpr int kCopyRows = 128 / kCopies;
    // Tensor Memory columns: S (2 x 128); with copies P (2 x 64) and O, else the O of
    // both halves of the keys, and P in the first 32 columns of its half of S
    constexpr uint32_t cS = 0, cP = 256, cO = kCopies > 1 ? 384 : 256;
    const PagedArgs &a = ta.p;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, NK = ta.NK, NV = ta.NV;
    const int rows = a.Bt * a.Gt;
    // quarters of the lanes with rows, softmax warps at work
    const int n_quads = kCopies > 1 ? 4 : (rows + 31) / 32, n_soft = n_quads * kParts;

    uint8_t *ring = smem + kSlot;                          // behind Q
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem + ta.off_bar);
    uint64_t *full = bars;               // [NK + NV] the K or V tile has landed
    uint64_t *empty = full + kMaxSlots;  // [NK + NV] its products are done
    uint64_t *sready = empty + kMaxSlots;// [2] S is formed
    uint64_t *sfree = sready + 2;        // [2] S has been read (with copies; else pvdone tells it)
    uint64_t *pready = sfree + 2;        // [2][kParts] P is written (and O rescaled, V's masked rows zeroed)
    uint64_t *pvdone = pready + 4;       // [2] O includes the tile's P V
    uint64_t *qfull = pvdone + 2;
    uint64_t *qempty = qfull + 1;        // the segment's last S is formed
    uint64_t *ofree = qempty + 1;        // the epilogue has read O
    uint64_t *drained = ofree + 1;       // [2] every MMA of an issuer has completed
    uint32_t *tmem_holder = reinterpret_cast<uint32_t *>(drained + 2);
    volatile int *fail = reinterpret_cast<volatile int *>(tmem_holder + 1);
    PlanSmem *plan_smem = reinterpret_cast<PlanSmem *>(tmem_holder + 2);
    float *exchange = reinterpret_cast<float *>(smem + ta.off_bar + kBarBytes);   // [2][128]
    float *inv_of = exchange + 256;                        // [64], with copies

    if (warp == W::kIssueS) {
        tmem_alloc(tmem_holder, 512);
        tmem_relinquish();
    }
    if (warp == W::kLoadK && lane == 0) {
        prefetch_tensormap(&ta.tmQ);
        prefetch_tensormap(&ta.tmK);
        prefetch_tensormap(&ta.tmV);
        for (int i = 0; i < NK + NV; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sready[i], 1);
            mbar_init(&sfree[i], n_soft);
            for (int p = 0; p < kParts; ++p) mbar_init(&pready[i * kParts + p], n_quads);
            mbar_init(&pvdone[i], 1);
            mbar_init(&drained[i], 1);
        }
        mbar_init(qfull, 1);
        mbar_init(qempty, 1);
        mbar_init(ofree, n_soft);
        *fail = 0;
        fence_mbar_init();
    }
    tc_fence_before();
    __syncthreads();                                       // barriers and Tensor Memory are in place
    tc_fence_after();
    // what comes before in the stream is complete from here on
    griddep_wait();
    griddep_launch_dependents();
    Walk w;
    Shares sh(0, 1);
    const bool work = find_share<kThreads>(a, *plan_smem, w, sh);
    const uint32_t tmem = *tmem_holder;

    if (warp == W::kLoadK || warp == W::kLoadV) {
        // ------------------------------------------------------ producers of K and V
        const bool is_v = warp == W::kLoadV;
        if (work) {
            const int P = a.page_size, per = kTile / P;    // pages of a tile
            const uint32_t page_bytes = (uint32_t)P * D * 2, n_slots = is_v ? NV : NK;
            const CUtensorMap *map = is_v ? &ta.tmV : &ta.tmK;
            uint64_t *my_full = is_v ? full + NK : full, *my_empty = is_v ? empty + NK : empty;
            uint8_t *my_ring = is_v ? ring + (size_t)NK * kSlot : ring;
            // a cache that is read once need not push tables, lengths and partials out of L2
            const bool once = row_tiles(a) == 1;
            const uint64_t policy = policy_evict_first();
            uint32_t n = 0;                                // tiles issued
            RingPos pos{0, 1};                             // phase of `empty`: the first round is free
            bool ok = true;
            while (ok && w.next(a)) {
                const int head = w.head;
                const int *pages = a.table + (size_t)w.req * a.max_pages;
                auto page_at = [&](int i) -> int {         // this lane's page of tile i, -1: nothing visible in it
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
                    next_page = page_at(i + 1);            // a tile ahead of its use
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
                            if (once) tma_load_4d_policy(dst + h * kPanel, map, 64 * h, 0, head, page, &my_full[pos.slot], policy);
                            else tma_load_4d(dst + h * kPanel, map, 64 * h, 0, head, page, &my_full[pos.slot]);
                    }
                    pos.step(n_slots);
                    ++n;
                }
            }
            if (*fail && lane == 0) {
                // let copies in flight land before the block exits
                for (uint32_t s = 0; s < n_slots; ++s) {
                    const uint32_t k = n / n_slots + (s < n % n_slots ? 1u : 0u);
                    if (k) mbar_wait(&my_full[s], (k - 1) & 1u, kWaitNs);
                }
            }
        }
        if (is_v) {
            if (lane == 0) write_note(a, work, w, sh);
            write_empty<bf16, 32>(a, lane);
        }
    } else if (work && warp == W::kIssueS) {
        // --------------------------------------------- issuer of S = Q K^T, loads of Q
        if (lane == 0) {
            const uint32_t id = instr_desc(FMT_BF16, FMT_BF16, false, false, 128, kTile);
            const uint64_t aq = smem_desc(smem_u32(smem), 16, 1024, SWZ_128B);
            const uint64_t k_desc = smem_desc(smem_u32(ring), 16, 1024, SWZ_128B);
            uint32_t n = 0, seg = 0;                       // tiles and segments so far
            RingPos pos{0, 0};
            bool ok = true;
            while (ok && w.next(a)) {
                const Unit u = unit_of(a, w.head, w.rt);
                if (seg > 0 && !wait_soon(qempty, (seg - 1) & 1u, fail)) break;
                mbar_arrive_expect_tx(qfull, (uint32_t)(kCopies * rows * D * 2));
#pragma unroll
                for (int x = 0; x < kCopies * kHalves; ++x)
                    tma_load_4d(smem + (x % kHalves) * kPanel + (x / kHalves) * kCopyRows * 128, &ta.tmQ,
                                64 * (x % kHalves), u.head * a.G + u.g0, u.i0, w.req, qfull);
                ok = wait_soon(qfull, seg & 1u, fail);
                ++seg;
                for (int i = w.i0; ok && i < w.i1; ++i, ++n) {
                    const uint32_t b = n & 1;
                    // S's buffer is free: read, or (P being in it) multiplied
                    ok = wait_soon(kCopies > 1 ? &sfree[b] : &pvdone[b], ((n >> 1) & 1u) ^ 1u, fail) &&
                         wait_soon(&full[pos.slot], pos.phase, fail);
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t bk = k_desc + pos.slot * (kSlot >> 4);
#pragma unroll
                    for (int k = 0; k < D / 16; ++k)
                        mma_bf16_ss(tmem + cS + 128 * b, aq + (k >> 2) * (kPanel >> 4) + (k & 3) * 2,
                                    bk + (k >> 2) * (kPanel >> 4) + (k & 3) * 2, id, k > 0);
                    mma_commit(&sready[b]);
                    mma_commit(&empty[pos.slot]);
                    if (i + 1 == w.i1) mma_commit(qempty);
                    pos.step(NK);
                }
            }
            mma_commit(&drained[0]);
            mbar_wait(&drained[0], 0, kWaitNs);
            if (*fail && seg > 0) mbar_wait(qfull, (seg - 1) & 1u, kWaitNs);
        }
    } else if (work && warp == W::kIssueO) {
        // ------------------------------------------------------ issuer of O += P V
        if (lane == 0) {
            const uint32_t id = instr_desc(FMT_BF16, FMT_BF16, false, true, 128, D);
            const uint64_t v_desc = smem_desc(smem_u32(ring + (size_t)NK * kSlot), kPanel, 1024, SWZ_128B);
            uint32_t n = 0, seg = 0;
            RingPos pos{0, 0};
            bool ok = true;
            while (ok && w.next(a)) {
                // O is overwritten by a segment's first product: the last epilogue has read it
                if (seg > 0) ok = wait_soon(ofree, (seg - 1) & 1u, fail);
                uint32_t acc = 0;                          // bits: accumulators, or copies, that the segment has written
                for (int i = w.i0; ok && i < w.i1; ++i, ++n) {
                    const uint32_t b = n & 1;
                    const int j = key_tile(w.vis, i) * kTile;
                    const bool all = all_visible(w.vis, j);
                    // steps of 16 keys: of a part, of a copy
                    constexpr int kSteps = kTile / 16 / kParts, kOwn = kSteps / kCopies;
                    ok = wait_soon(&full[NK + pos.slot], pos.phase, fail);
                    const uint64_t bv = v_desc + pos.slot * (kSlot >> 4);
#pragma unroll
                    for (int p = 0; p < kParts; ++p) {
                        ok = ok && wait_soon(&pready[b * kParts + p], (n >> 1) & 1u, fail);
                        if (!ok) break;
                        tc_fence_after();
                        const uint32_t o = tmem + cO + 128 * p, pa = tmem + (kCopies > 1 ? cP + 64 * b : cS + 128 * b + 64 * p);
                        auto product = [&](int g, uint32_t accumulate) {
                            const uint64_t v = bv + (p * kSteps + g) * (2048 >> 4);
                            if constexpr (kCopies > 1) mma_bf16_ts_lanes(o, pa + 8 * g, v, id, accumulate, kCopies, g / kOwn);
                            else mma_bf16_ts(o, pa + 8 * g, v, id, accumulate);
                        };
                        if (all) {
#pragma unroll
                            for (int g = 0; g < kSteps; ++g)
                                product(g, g % kOwn > 0 ? 1u : acc >> (p + g / kOwn) & 1u);
                            acc |= ((1u << kCopies) - 1) << p;
                        } else {
#pragma unroll 1
                            for (int g = 0; g < kSteps; ++g) {
                                if (!any_visible(w.vis, j + 16 * (p * kSteps + g), 16)) continue;
                                product(g, acc >> (p + g / kOwn) & 1u);
                                acc |= 1u << (p + g / kOwn);
                            }
                        }
                    }
                    if (!ok) break;
                    mma_commit(&pvdone[b]);
                    mma_commit(&empty[NK + pos.slot]);
                    pos.step(NV);
                }
                ++seg;
            }
            mma_commit(&drained[1]);
            mbar_wait(&drained[1], 0, kWaitNs);
        }
    } else if (work && warp < W::kSoft && (warp & 3) < n_quads) {
        // --------------------------------------------------- softmax, epilogue
        constexpr int kKeys = kTile / (kParts * kCopies);   // keys of a tile of this thread
        constexpr int kFeat = D / kParts;                   // features of the output that it writes
        constexpr int kGroup = 32 * (kCopies > 1 ? 4 : kParts);   // threads that share rows
        const int quad = warp & 3, part = kCopies > 1 ? 0 : warp >> 2;
        const int copy = kCopies > 1 ? tid / kCopyRows : 0, row = kCopies > 1 ? tid % kCopyRows : 32 * quad + lane;
        const int key0 = kKeys * (kCopies > 1 ? copy : part);
        const int worker = kCopies > 1 ? tid : 32 * (part * n_quads + quad) + lane;   // among the threads at work
        const uint32_t lane_off = (uint32_t)(32 * quad) << 16;
        const uint32_t group_bar = kCopies > 1 ? 1 : 1 + quad;
        const uint32_t my_o = tmem + cO + 128 * part + lane_off;
        const float to_log2 = kLog2e * rsqrtf((float)D);
        float *stage = reinterpret_cast<float *>(smem + ta.off_stage);   // with copies
        uint32_t n = 0;                                    // tiles so far
        bool bad = false;                                  // a wait gave up: leave at the next vote
        auto wait = [&](uint64_t *bar, uint32_t parity) {
            bad = __any_sync(0xffffffffu, bad || !wait_soon(bar, parity, fail));
        };
        // arrival of the warp, after its Tensor Memory accesses
        auto arrive = [&](uint64_t *bar) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0 && !bad) mbar_arrive(bar);
        };
        while (w.next(a)) {     // left by a vote at a segment's end only, so that the warps of a row stay together
            float ref = -INFINITY;
            f32x2 l2 = pair2(0.f, 0.f);                    // the row's sum over this thread's keys, in two
            for (int i = w.i0; i < w.i1; ++i, ++n) {
                const uint32_t b = n & 1;
                const int j0 = key_tile(w.vis, i) * kTile;
                const bool edge = !all_visible(w.vis, j0);
                if (edge) {
                    // masked rows of V in the groups that enter the product.  (An earlier
                    // tile's product first, so that the slot's last item has landed and the
                    // wait cannot take its phase for this one's.)
                    if (n >= 2) wait(&pvdone[b], ((n - 2) >> 1) & 1u);
                    const uint32_t slot = n % (uint32_t)NV;
                    wait(&full[NK + slot], (n / (uint32_t)NV) & 1u);
                    for (int c = worker; c < kTile; c += 32 * n_soft) {
                        const int j = j0 + c;
                        if (!bad && !key_visible(w.vis, j) && any_visible(w.vis, j & ~15, 16)) {
                            uint8_t *v = ring + (size_t)(NK + slot) * kSlot + c * 128;
#pragma unroll
                            for (int x = 0; x < kHalves * 8; ++x)
                                *reinterpret_cast<uint4 *>(v + (x >> 3) * kPanel + (x & 7) * 16) = make_uint4(0, 0, 0, 0);
                        }
                    }
                    fence_proxy_async_smem();
                }
                wait(&sready[b], (n >> 1) & 1u);
                tc_fence_after();
                float s[kKeys / 32][32];
#pragma unroll
                for (int x = 0; x < kKeys / 32; ++x)
                    tmem_ld32(tmem + cS + 128 * b + key0 + 32 * x + lane_off, s[x]);
                tmem_wait_ld();
                if (kCopies > 1) arrive(&sfree[b]);
                if (edge) {
                    const int k0 = j0 + key0, hi = w.vis.len - k0, lo = w.vis.lo - k0, sink = w.vis.sink - k0;
#pragma unroll
                    for (int x = 0; x < kKeys / 32; ++x)
#pragma unroll
                        for (int y = 0; y < 32; ++y) {
                            const int k = 32 * x + y;
                            if (!(k < hi && (k >= lo || k < sink))) s[x][y] = -INFINITY;
                        }
                }
                float mx4[4] = {s[0][0], s[0][1], s[0][2], s[0][3]};
#pragma unroll
                for (int x = 0; x < kKeys / 32; ++x)
#pragma unroll
                    for (int y = 0; y < 32; ++y) mx4[y & 3] = fmaxf(mx4[y & 3], s[x][y]);
                float mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3])) * to_log2;
                float f = 1.f;
                if (mx > ref + kSlack) {                   // from -inf: whenever a key is visible
                    if (ref != -INFINITY) f = ex2(ref - mx);        // (else O and the sum are zero)
                    ref = mx;
                }
                // P's buffer is free, and O is at rest, once earlier products are done
                const bool rescale = __any_sync(0xffffffffu, f != 1.f && row < rows);
                if (rescale || (kCopies > 1 && n >= 2)) {
                    const uint32_t k = rescale ? n - 1 : n - 2;
                    wait(&pvdone[k & 1], (k >> 1) & 1u);
                    tc_fence_after();
                }
                if (rescale) {
                    l2 = mul2(l2, pair2(f, f));
#pragma unroll 1
                    for (int x = 0; x < D / 32; ++x) {
                        float o[32];
                        tmem_ld32(my_o + 32 * x, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int y = 0; y < 32; ++y) o[y] *= f;
                        tmem_st32(my_o + 32 * x, o);
                    }
                }
                const float base = ref == -INFINITY ? 0.f : ref;
                const f32x2 c2 = pair2(to_log2, to_log2), base2 = pair2(-base, -base);
#pragma unroll
                for (int x = 0; x < kKeys / 32; ++x) {
                    float p[16];                           // pairs of bf16
#pragma unroll
                    for (int y = 0; y < 32; y += 2) {
                        float p0, p1;
                        unpair2(fma2(pair2(s[x][y], s[x][y + 1]), c2, base2), p0, p1);
                        p0 = ex2(p0);
                        p1 = ex2(p1);
                        l2 = add2(l2, pair2(p0, p1));
                        p[y / 2] = __uint_as_float(pack_bf16x2(p0, p1));
                    }
                    tmem_st16(tmem + lane_off + 16 * x + (kCopies > 1 ? cP + 64 * b + key0 / 2 : cS + 128 * b + 64 * part), p);
                }
                tmem_wait_st();
                arrive(&pready[b * kParts + part]);
            }
            // the segment's output
            const Unit u = unit_of(a, w.head, w.rt);
            size_t at;
            const bool live = row_at(a, w.req, u, row, at), whole = w.whole();
            bf16 *out = static_cast<bf16 *>(a.O) + at;
            float *partial = a.part + w.slot() * partial_floats(rows, D);
            float l, l_odd, f = 1.f, f0 = 0.f, f1 = 0.f;
            unpair2(l2, l, l_odd);
            l += l_odd;
            if (kCopies > 1) {
                // reference and sum of the row over its copies
                exchange[tid] = ref;
                exchange[128 + tid] = l;
                if (group_sync_failed(group_bar, kGroup, bad)) break;
                float top = exchange[row];
#pragma unroll
                for (int c = 1; c < kCopies; ++c) top = fmaxf(top, exchange[c * kCopyRows + row]);
                const float base = top == -INFINITY ? 0.f : top;
                f = ex2(ref - base);
                ref = top;
                l = 0.f;
#pragma unroll
                for (int c = 0; c < kCopies; ++c)
                    l = fmaf(exchange[128 + c * kCopyRows + row], ex2(exchange[c * kCopyRows + row] - base), l);
                if (copy == 0) inv_of[row] = 1.f / l;              // read after the next barrier
            } else {
                // the same over the two halves of the keys
                exchange[part * 128 + row] = ref;
                if (group_sync_failed(group_bar, kGroup, bad)) break;
                const float r0 = exchange[row], r1 = exchange[128 + row], top = fmaxf(r0, r1);
                const float base = top == -INFINITY ? 0.f : top;
                f0 = ex2(r0 - base);
                f1 = ex2(r1 - base);
                group_sync_failed(group_bar, kGroup, false);
                exchange[part * 128 + row] = l * (part == 0 ? f0 : f1);
                group_sync_failed(group_bar, kGroup, false);
                l = exchange[row] + exchange[128 + row];
                group_sync_failed(group_bar, kGroup, false);       // read before the next segment's are written
                ref = top;
            }
            const float inv = 1.f / l;
            if (!whole && row < rows && (kCopies > 1 ? copy == 0 : part == 0)) {
                partial[row] = ref;
                partial[rows + row] = l;
            }
            wait(&pvdone[(n - 1) & 1], ((n - 1) >> 1) & 1u);
            tc_fence_after();
            if constexpr (kCopies > 1) {
                // The copies' rows are added in order, in shared memory, as many features
                // (32, 64 or 128) at a time as it holds of these rows: [copy][row][width + 4].
                const int width = rows <= kCopyRows / 4 ? 128 : (rows <= kCopyRows / 2 ? 64 : 32);
                const int span = width < D ? width : D, pitch = span + 4;
#pragma unroll 1
                for (int x0 = 0; x0 < D; x0 += span) {
                    float *mine = stage + (copy * rows + row) * pitch;
#pragma unroll 1
                    for (int x = 0; x < span; x += 32) {
                        float o[32];
                        tmem_ld32(tmem + cO + x0 + x + lane_off, o);
                        tmem_wait_ld();
                        if (row < rows) {                  // (a copy without a visible key has not written O)
#pragma unroll
                            for (int y = 0; y < 32; y += 4)
                                *reinterpret_cast<float4 *>(mine + x + y) =
                                    f != 0.f ? make_float4(o[y] * f, o[y + 1] * f, o[y + 2] * f, o[y + 3] * f)
                                             : make_float4(0.f, 0.f, 0.f, 0.f);
                        }
                    }
                    if (x0 + span == D) arrive(ofree);
                    group_sync_failed(group_bar, kGroup, false);
                    if (!bad) {
                        if (whole) {                       // eight features of a row
                            for (int x = tid; x < rows * (span / 8); x += 128) {
                                const int r = x / (span / 8), col = x % (span / 8) * 8;
                                const float *src = stage + r * pitch + col;
                                float4 v0 = make_float4(0.f, 0.f, 0.f, 0.f), v1 = v0;
#pragma unroll
                                for (int c = 0; c < kCopies; ++c) {
                                    const float4 s0 = *reinterpret_cast<const float4 *>(src + c * rows * pitch);
                                    const float4 s1 = *reinterpret_cast<const float4 *>(src + c * rows * pitch + 4);
                                    v0 = make_float4(v0.x + s0.x, v0.y + s0.y, v0.z + s0.z, v0.w + s0.w);
                                    v1 = make_float4(v1.x + s1.x, v1.y + s1.y, v1.z + s1.z, v1.w + s1.w);
                                }
                                const float k = inv_of[r];
                                size_t to;
                                if (row_at(a, w.req, u, r, to))
                                    *reinterpret_cast<uint4 *>(static_cast<bf16 *>(a.O) + to + x0 + col) = make_uint4(
                                        pack_bf16x2(v0.x * k, v0.y * k), pack_bf16x2(v0.z * k, v0.w * k),
                                        pack_bf16x2(v1.x * k, v1.y * k), pack_bf16x2(v1.z * k, v1.w * k));
                            }
                        } else {                           // feature-major, as the join reads it
                            for (int x = tid; x < rows * span; x += 128) {
                                const int r = x % rows, col = x / rows;
                                float v = 0.f;
#pragma unroll
                                for (int c = 0; c < kCopies; ++c) v += stage[(c * rows + r) * pitch + col];
                                partial[2 * rows + (size_t)x0 * rows + x] = v;
                            }
                        }
                    }
                    group_sync_failed(group_bar, kGroup, false);
                }
            } else {
#pragma unroll 1
                for (int x = 0; x < kFeat / 32; ++x) {
                    const uint32_t from = tmem + cO + kFeat * part + 32 * x + lane_off;
                    float o[32], o1[32];
                    tmem_ld32(from, o);
                    tmem_ld32(from + 128, o1);
                    tmem_wait_ld();
                    if (x == kFeat / 32 - 1) arrive(ofree);
                    if (bad) continue;
                    // (a half without a visible key in the segment may not have been written)
#pragma unroll
                    for (int y = 0; y < 32; ++y) o[y] = (f0 != 0.f ? o[y] * f0 : 0.f) + (f1 != 0.f ? o1[y] * f1 : 0.f);
                    const int col = kFeat * part + 32 * x;
                    if (whole) {
                        if (live) {
#pragma unroll
                            for (int y = 0; y < 32; y += 8)
                                *reinterpret_cast<uint4 *>(out + col + y) = make_uint4(
                                    pack_bf16x2(o[y] * inv, o[y + 1] * inv), pack_bf16x2(o[y + 2] * inv, o[y + 3] * inv),
                                    pack_bf16x2(o[y + 4] * inv, o[y + 5] * inv), pack_bf16x2(o[y + 6] * inv, o[y + 7] * inv));
                        }
                    } else if (row < rows) {
                        float *po = partial + 2 * rows + (size_t)col * rows + row;
#pragma unroll
                        for (int y = 0; y < 32; ++y) po[(size_t)y * rows] = o[y];
                    }
                }
            }
        }
        if (tid == 0 && *fail) raise_error(a.err, ERR_WAIT_TIMEOUT);
    }
    __syncthreads();
    if (warp == W::kIssueS) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

template <int D, int kCopies> cudaError_t launch(const PagedArgs &a, cudaStream_t st)
{
    TcArgs ta;
    ta.p = a;
    // Q, K/V rings, barriers, exchange, stage (with copies), and 1 KB for alignment
    const uint32_t slot = kTile * D * 2, stage = kCopies > 1 ? kStage : 0;
    const uint32_t tail = kBarBytes + kExchange + stage + 1024;
    int ns = (int)((kSmemLimit - tail) / slot) - 1;
    if (ns > kMaxSlots) ns = kMaxSlots;
    // S has two buffers of its own, so V waits longer for its product than K
    ta.NK = ns / 2;
    ta.NV = ns - ta.NK;
    ta.off_bar = (1 + ns) * slot;
    ta.off_stage = ta.off_bar + kBarBytes + kExchange + 256;
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
    static std::atomic<unsigned long long> opted{0};
    const cudaError_t e = opt_in(reinterpret_cast<const void *>(&k_paged_attn_tc<D, kCopies>), kSmemLimit, opted);
    if (e != cudaSuccess) return e;
    return pipe::launch_early(k_paged_attn_tc<D, kCopies>, dim3(a.n_cta), dim3(Roles<kCopies>::kThreads), ta.bytes, st, ta);
}

template <int D> cudaError_t launch_rows(const PagedArgs &a, cudaStream_t st)
{
    // as many copies of the rows as fit in 128
    const int rows = a.Bt * a.Gt;
    if (rows <= 32) return launch<D, 4>(a, st);
    return rows <= 64 ? launch<D, 2>(a, st) : launch<D, 1>(a, st);
}

}  // namespace

cudaError_t launch_paged_attn_tc(const PagedArgs &a, cudaStream_t st)
{
    return a.d == 128 ? launch_rows<128>(a, st) : launch_rows<64>(a, st);
}

}  // namespace hyb
