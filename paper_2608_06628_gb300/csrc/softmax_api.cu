// softmax_api.cu -- the extern "C" entry points declared in
// include/hybrid_softmax.h: argument validation and launches.
#include <cmath>

#include "hybrid_common.cuh"
#include "softmax_kernels.h"

namespace {

bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
bool good(const void *p, uintptr_t a) { return p && aligned(p, a); }
bool good_or_null(const void *p, uintptr_t a) { return aligned(p, a); }

// n ints of a call's argument
struct Ints {
    const int *p;
    size_t n;
};
// Whether one of the outputs shares memory with an input or another output.  (The blocks of
// a call do not wait for one another: one may write what another has yet to read.)
template <int O, int I> bool overlap(const Ints (&out)[O], const Ints (&in)[I])
{
    auto meet = [](const Ints &a, const Ints &b) {
        const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
        return a.p && b.p && a.n && b.n && x < y + b.n * sizeof(int) && y < x + a.n * sizeof(int);
    };
    for (int i = 0; i < O; ++i) {
        for (int j = 0; j < I; ++j)
            if (meet(out[i], in[j])) return true;
        for (int j = 0; j < i; ++j)
            if (meet(out[i], out[j])) return true;
    }
    return false;
}

hybrid_status from_cuda(cudaError_t e) { return e == cudaSuccess ? HYBRID_OK : HYBRID_ERR_CUDA; }

constexpr int kMaxRequests = 65536;

hybrid_status check_cfg(const hybrid_cfg *c)
{
    if (!c) return HYBRID_ERR_INVALID_ARG;
    if (c->io_dtype != HYBRID_F32 && c->io_dtype != HYBRID_BF16) return HYBRID_ERR_UNSUPPORTED;
    if (c->head_dim != 64 && c->head_dim != 128) return HYBRID_ERR_UNSUPPORTED;
    if (c->n_kv_heads < 1 || c->n_q_heads < 1 || c->n_q_heads > 256) return HYBRID_ERR_UNSUPPORTED;
    if (c->n_kv_heads > c->n_q_heads || c->n_q_heads % c->n_kv_heads != 0) return HYBRID_ERR_INVALID_ARG;
    return HYBRID_OK;
}

hybrid_status check_pages(const hybrid_page_cfg *p)
{
    if (!p) return HYBRID_ERR_INVALID_ARG;
    if (p->page_size != 16 && p->page_size != 32 && p->page_size != 64 && p->page_size != 128)
        return HYBRID_ERR_UNSUPPORTED;
    if (p->n_pages < 1 || p->max_pages < 1) return HYBRID_ERR_INVALID_ARG;
    // slots and positions are ints (with room for the end of a tile)
    if ((long long)p->n_pages * p->page_size > 0x7fffffffll || (long long)p->max_pages * p->page_size > 0x7fffff00ll)
        return HYBRID_ERR_UNSUPPORTED;
    return HYBRID_OK;
}

// Checks shared by the three rotation entry points, for n_tok > 0.
hybrid_status check_rope(const hybrid_cfg *cfg, const hybrid_rope_cfg *rope, const void *Q, size_t q_stride,
                         const void *K, size_t k_stride, int n_tok, const void *wq, const void *wk,
                         const int *positions, const unsigned long long *freqs)
{
    hybrid_status s = check_cfg(cfg);
    if (s != HYBRID_OK) return s;
    if (!rope || n_tok < 0) return HYBRID_ERR_INVALID_ARG;
    if (rope->interleaved != 0 && rope->interleaved != 1) return HYBRID_ERR_INVALID_ARG;
    if (rope->rot_dim < 0 || rope->rot_dim > cfg->head_dim || rope->rot_dim % 16 != 0) return HYBRID_ERR_UNSUPPORTED;
    if (!(rope->eps >= 0.f) || !std::isfinite(rope->eps) || !std::isfinite(rope->scale)) return HYBRID_ERR_INVALID_ARG;
    if (n_tok == 0) return HYBRID_OK;
    const size_t unit = cfg->io_dtype == HYBRID_BF16 ? 8 : 4;   // elements of 16 bytes
    if (q_stride % unit != 0 || k_stride % unit != 0) return HYBRID_ERR_INVALID_ARG;
    if (q_stride < (size_t)cfg->n_q_heads * cfg->head_dim || k_stride < (size_t)cfg->n_kv_heads * cfg->head_dim)
        return HYBRID_ERR_INVALID_ARG;
    if (!good(Q, 16) || !good(K, 16) || !good_or_null(wq, 16) || !good_or_null(wk, 16)) return HYBRID_ERR_INVALID_ARG;
    if (rope->rot_dim > 0 && (!good(positions, 4) || !good(freqs, 8))) return HYBRID_ERR_INVALID_ARG;
    return HYBRID_OK;
}

hyb::RopeArgs rope_args(const hybrid_cfg *cfg, const hybrid_rope_cfg *rope, const void *Q, size_t q_stride,
                        const void *K, size_t k_stride, int n_tok, const void *wq, const void *wk,
                        const int *positions, const unsigned long long *freqs)
{
    hyb::RopeArgs a{};
    a.Q = Q;
    a.K = K;
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.wq = wq;
    a.wk = wk;
    a.positions = positions;
    a.freqs = freqs;
    a.n_tok = n_tok;
    a.Hq = cfg->n_q_heads;
    a.Hkv = cfg->n_kv_heads;
    a.d = cfg->head_dim;
    a.rot = rope->rot_dim;
    a.interleaved = rope->interleaved;
    a.scale = rope->scale;
    a.eps = rope->eps;
    return a;
}

}  // namespace

extern "C" {

hybrid_status hybrid_page_append(const hybrid_page_cfg *pg, int n_req, const int *lens, const int *n_new,
                                 const int *free_pages, const int *ring_in, int *block_table, int *slots,
                                 int *positions, int n_slots, int *tok_offsets, int *lens_out, int *ring_out,
                                 cudaStream_t stream)
{
    hybrid_status s = check_pages(pg);
    if (s != HYBRID_OK) return s;
    if (n_req < 0 || n_slots < 0) return HYBRID_ERR_INVALID_ARG;
    if (n_req > kMaxRequests) return HYBRID_ERR_UNSUPPORTED;
    if (n_req == 0 && n_slots == 0 && !ring_out && !tok_offsets) return HYBRID_OK;
    if (!good(free_pages, 4) || !good(ring_in, 4) || !good(ring_out, 4)) return HYBRID_ERR_INVALID_ARG;
    if (n_req > 0 && (!good(lens, 4) || !good(n_new, 4) || !good(block_table, 4) || !good(lens_out, 4)))
        return HYBRID_ERR_INVALID_ARG;
    if (n_slots > 0 && !good(slots, 4)) return HYBRID_ERR_INVALID_ARG;
    if (!good_or_null(positions, 4) || !good_or_null(tok_offsets, 4)) return HYBRID_ERR_INVALID_ARG;
    const size_t n = n_req, table = n * pg->max_pages;
    if (overlap<6, 4>({{block_table, table}, {slots, (size_t)n_slots}, {positions, (size_t)n_slots}, {tok_offsets, n + 1},
                       {lens_out, n}, {ring_out, 2}},
                      {{lens, n}, {n_new, n}, {free_pages, (size_t)pg->n_pages}, {ring_in, 2}}))
        return HYBRID_ERR_INVALID_ARG;
    unsigned *err = hyb::error_word();
    if (!err) return HYBRID_ERR_CUDA;
    return from_cuda(hyb::launch_page_append(*pg, n_req, lens, n_new, free_pages, ring_in, block_table, slots,
                                             positions, n_slots, tok_offsets, lens_out, ring_out, err, stream));
}

hybrid_status hybrid_page_release(const hybrid_page_cfg *pg, int n_req, const int *rows, int n_rows,
                                  const int *lens, const int *block_table, int *free_pages, const int *ring_in,
                                  int *ring_out, cudaStream_t stream)
{
    hybrid_status s = check_pages(pg);
    if (s != HYBRID_OK) return s;
    if (n_req < 0 || n_rows < 0) return HYBRID_ERR_INVALID_ARG;
    if (n_req > kMaxRequests || n_rows > kMaxRequests) return HYBRID_ERR_UNSUPPORTED;
    if (n_rows == 0 && !ring_out) return HYBRID_OK;
    if (!good(free_pages, 4) || !good(ring_in, 4) || !good(ring_out, 4)) return HYBRID_ERR_INVALID_ARG;
    if (n_rows > 0 && (!good(rows, 4) || !good(lens, 4) || !good(block_table, 4))) return HYBRID_ERR_INVALID_ARG;
    if (overlap<2, 4>({{free_pages, (size_t)pg->n_pages}, {ring_out, 2}},
                      {{rows, (size_t)n_rows}, {lens, (size_t)n_req}, {block_table, (size_t)n_req * pg->max_pages}, {ring_in, 2}}))
        return HYBRID_ERR_INVALID_ARG;
    unsigned *err = hyb::error_word();
    if (!err) return HYBRID_ERR_CUDA;
    return from_cuda(hyb::launch_page_release(*pg, n_req, rows, n_rows, lens, block_table, free_pages, ring_in,
                                              ring_out, err, stream));
}

hybrid_status hybrid_rope_freqs(const hybrid_rope_scaling *sc, int rot_dim, unsigned long long *freqs, float *scale)
{
    if (!sc || !freqs || !scale) return HYBRID_ERR_INVALID_ARG;
    if (rot_dim < 16 || rot_dim > 128 || rot_dim % 16 != 0) return HYBRID_ERR_UNSUPPORTED;
    if (sc->kind < HYBRID_ROPE_NONE || sc->kind > HYBRID_ROPE_YARN) return HYBRID_ERR_UNSUPPORTED;
    if (!(sc->base > 1.0) || !std::isfinite(sc->base)) return HYBRID_ERR_INVALID_ARG;
    const bool scaled = sc->kind != HYBRID_ROPE_NONE, yarn = sc->kind == HYBRID_ROPE_YARN;
    if (scaled && (!(sc->factor >= 1.0) || !std::isfinite(sc->factor))) return HYBRID_ERR_INVALID_ARG;
    if (yarn && (!(sc->orig_len > 0.0) || !std::isfinite(sc->orig_len) || !(sc->beta_slow >= 0.0) ||
                 !(sc->beta_fast > sc->beta_slow) || !std::isfinite(sc->beta_fast)))
        return HYBRID_ERR_INVALID_ARG;
    const double two_pi = 6.283185307179586476925;
    const double base =
        sc->kind == HYBRID_ROPE_NTK ? sc->base * std::pow(sc->factor, (double)rot_dim / (rot_dim - 2)) : sc->base;
    for (int i = 0; i < rot_dim / 2; ++i) {
        double t = std::pow(base, -2.0 * i / rot_dim) / two_pi;   // turns per position, < 1/6
        if (sc->kind == HYBRID_ROPE_LINEAR) t /= sc->factor;
        if (yarn) {
            double keep = (sc->orig_len * t - sc->beta_slow) / (sc->beta_fast - sc->beta_slow);
            keep = keep < 0.0 ? 0.0 : (keep > 1.0 ? 1.0 : keep);
            t = t / sc->factor * (1.0 - keep) + t * keep;
        }
        freqs[i] = (unsigned long long)std::ldexp(t, 64);         // below 2^62: fits
    }
    *scale = yarn ? (float)(0.1 * std::log(sc->factor) + 1.0) : 1.0f;
    return HYBRID_OK;
}

hybrid_status hybrid_qk_norm_rope(const hybrid_cfg *cfg, const hybrid_rope_cfg *rope, const void *Q,
                                  size_t q_stride, const void *K, size_t k_stride, int n_tok, const void *wq,
                                  const void *wk, const int *positions, const unsigned long long *freqs, void *Qo,
                                  void *Ko, cudaStream_t stream)
{
    hybrid_status s = check_rope(cfg, rope, Q, q_stride, K, k_stride, n_tok, wq, wk, positions, freqs);
    if (s != HYBRID_OK || n_tok == 0) return s;
    if (!good(Qo, 16) || !good(Ko, 16)) return HYBRID_ERR_INVALID_ARG;
    if ((Qo == Q && q_stride != (size_t)cfg->n_q_heads * cfg->head_dim) ||
        (Ko == K && k_stride != (size_t)cfg->n_kv_heads * cfg->head_dim))
        return HYBRID_ERR_INVALID_ARG;
    hyb::RopeArgs a = rope_args(cfg, rope, Q, q_stride, K, k_stride, n_tok, wq, wk, positions, freqs);
    a.Qo = Qo;
    a.Ko = Ko;
    return from_cuda(hyb::launch_qk_norm_rope(cfg->io_dtype, a, stream));
}

hybrid_status hybrid_qk_norm_rope_cache(const hybrid_cfg *cfg, const hybrid_rope_cfg *rope,
                                        const hybrid_page_cfg *pg, const void *Q, size_t q_stride, const void *K,
                                        size_t k_stride, const void *V, size_t v_stride, int n_tok, const void *wq,
                                        const void *wk, const int *positions, const unsigned long long *freqs,
                                        const int *slots, void *Qo, void *K_cache, void *V_cache,
                                        cudaStream_t stream)
{
    hybrid_status s = check_rope(cfg, rope, Q, q_stride, K, k_stride, n_tok, wq, wk, positions, freqs);
    if (s != HYBRID_OK) return s;
    s = check_pages(pg);
    if (s != HYBRID_OK || n_tok == 0) return s;
    if (!good(V, 16) || !good(slots, 4) || !good(Qo, 16) || !good(K_cache, 16) || !good(V_cache, 16))
        return HYBRID_ERR_INVALID_ARG;
    if (v_stride % (cfg->io_dtype == HYBRID_BF16 ? 8 : 4) != 0 || v_stride < (size_t)cfg->n_kv_heads * cfg->head_dim)
        return HYBRID_ERR_INVALID_ARG;
    if (Qo == Q && q_stride != (size_t)cfg->n_q_heads * cfg->head_dim) return HYBRID_ERR_INVALID_ARG;
    unsigned *err = hyb::error_word();
    if (!err) return HYBRID_ERR_CUDA;
    hyb::RopeArgs a = rope_args(cfg, rope, Q, q_stride, K, k_stride, n_tok, wq, wk, positions, freqs);
    a.V = V;
    a.v_stride = v_stride;
    a.slots = slots;
    a.Qo = Qo;
    a.K_cache = K_cache;
    a.V_cache = V_cache;
    a.page_size = pg->page_size;
    a.n_pages = pg->n_pages;
    a.err = err;
    return from_cuda(hyb::launch_qk_norm_rope(cfg->io_dtype, a, stream));
}

size_t hybrid_qk_norm_rope_workspace_bytes(const hybrid_cfg *cfg, int n_tok)
{
    if (check_cfg(cfg) != HYBRID_OK || n_tok < 0) return 0;
    return hyb::qk_norm_rope_partial_bytes(cfg->head_dim, n_tok);
}

hybrid_status hybrid_qk_norm_rope_backward(const hybrid_cfg *cfg, const hybrid_rope_cfg *rope, const void *Q,
                                           size_t q_stride, const void *K, size_t k_stride, const void *dQo,
                                           const void *dKo, int n_tok, const void *wq, const void *wk,
                                           const int *positions, const unsigned long long *freqs, void *workspace,
                                           size_t workspace_bytes, void *dQ, void *dK, float *dwq, float *dwk,
                                           cudaStream_t stream)
{
    hybrid_status s = check_rope(cfg, rope, Q, q_stride, K, k_stride, n_tok, wq, wk, positions, freqs);
    if (s != HYBRID_OK) return s;
    // the weight gradients are written for every n_tok (zeros without tokens)
    if ((wq != nullptr) != (dwq != nullptr) || (wk != nullptr) != (dwk != nullptr)) return HYBRID_ERR_INVALID_ARG;
    if (!good_or_null(dwq, 4) || !good_or_null(dwk, 4)) return HYBRID_ERR_INVALID_ARG;
    if (n_tok == 0 && !dwq && !dwk) return HYBRID_OK;
    if (n_tok > 0 && (!good(dQo, 16) || !good(dKo, 16) || !good(dQ, 16) || !good(dK, 16)))
        return HYBRID_ERR_INVALID_ARG;
    if (!good(workspace, 16) || workspace_bytes < hyb::qk_norm_rope_partial_bytes(cfg->head_dim, n_tok))
        return HYBRID_ERR_INVALID_ARG;
    hyb::RopeArgs a = rope_args(cfg, rope, Q, q_stride, K, k_stride, n_tok, wq, wk, positions, freqs);
    a.dQo = dQo;
    a.dKo = dKo;
    a.Qo = dQ;
    a.Ko = dK;
    a.partial = static_cast<float *>(workspace);
    a.dwq = dwq;
    a.dwk = dwk;
    return from_cuda(hyb::launch_qk_norm_rope_backward(cfg->io_dtype, a, stream));
}

size_t hybrid_paged_attn_workspace_bytes(const hybrid_cfg *cfg, const hybrid_page_cfg *pg, int n_req)
{
    if (check_cfg(cfg) != HYBRID_OK || check_pages(pg) != HYBRID_OK || n_req < 0 || n_req > kMaxRequests) return 0;
    if (cfg->block_size < 1 || cfg->block_size > 128) return 0;
    hyb::PagedArgs a{};
    hyb::paged_geometry(*cfg, a);
    return hyb::paged_workspace_bytes(a);
}

hybrid_status hybrid_paged_attn(const hybrid_cfg *cfg, const hybrid_page_cfg *pg, const void *Q,
                                const void *K_cache, const void *V_cache, const int *block_table,
                                const int *kv_len, int n_req, int window, int n_sink, void *O, void *workspace,
                                size_t workspace_bytes, cudaStream_t stream)
{
    hybrid_status s = check_cfg(cfg);
    if (s != HYBRID_OK) return s;
    s = check_pages(pg);
    if (s != HYBRID_OK) return s;
    if (cfg->block_size < 1 || cfg->block_size > 128) return HYBRID_ERR_UNSUPPORTED;
    if (n_req < 0 || window < 0 || n_sink < 0) return HYBRID_ERR_INVALID_ARG;
    if (n_req > kMaxRequests) return HYBRID_ERR_UNSUPPORTED;
    if (n_req == 0) return HYBRID_OK;
    if (!good(Q, 16) || !good(K_cache, 16) || !good(V_cache, 16) || !good(O, 16) || !good(block_table, 4) ||
        !good(kv_len, 4) || !good(workspace, 16))
        return HYBRID_ERR_INVALID_ARG;
    hyb::PagedArgs a{};
    hyb::paged_geometry(*cfg, a);
    if (workspace_bytes < hyb::paged_workspace_bytes(a)) return HYBRID_ERR_INVALID_ARG;
    // the kernels count quarters of tiles of 128 keys, of all row tiles, in an int
    const long long quarters = 4 * (((long long)pg->max_pages * pg->page_size + 127) / 128) + a.extra;
    if (quarters * n_req > 0x7fffffffll / ((long long)a.Hkv * a.n_gt * a.n_bt)) return HYBRID_ERR_UNSUPPORTED;
    // no more blocks than the longest possible contexts give work, four quarters each
    const long long most = quarters * n_req * a.Hkv * a.n_gt * a.n_bt / 4;
    if (most < a.n_cta) a.n_cta = (int)most;
    unsigned *err = hyb::error_word();
    if (!err) return HYBRID_ERR_CUDA;
    a.Q = Q;
    a.K = K_cache;
    a.V = V_cache;
    a.table = block_table;
    a.lens = kv_len;
    a.O = O;
    hyb::paged_set_workspace(a, workspace);
    a.n_req = n_req;
    a.page_size = pg->page_size;
    a.n_pages = pg->n_pages;
    a.max_pages = pg->max_pages;
    a.window = window;
    a.sink = n_sink;
    a.err = err;
    return from_cuda(hyb::launch_paged_attn(cfg->io_dtype, a, stream));
}

}  // extern "C"
