// softmax_kernels.h -- internal launchers of the softmax-layer operators
// (hybrid_softmax.h), and the description of one attention call.
#pragma once

#include <cuda_runtime.h>

#include "hybrid_softmax.h"

namespace hyb {

// The device error word of the current device (hybrid_api.cu); null on failure.
unsigned *error_word();

// page_pool.cu
cudaError_t launch_page_append(const hybrid_page_cfg &pg, int n_req, const int *lens, const int *n_new,
                               const int *free_pages, const int *ring_in, int *block_table, int *slots,
                               int *positions, int n_slots, int *tok_offsets, int *lens_out, int *ring_out,
                               unsigned *err, cudaStream_t st);
cudaError_t launch_page_release(const hybrid_page_cfg &pg, int n_req, const int *rows, int n_rows, const int *lens,
                                const int *block_table, int *free_pages, const int *ring_in, int *ring_out,
                                unsigned *err, cudaStream_t st);

// qk_norm_rope.cu
struct RopeArgs {
    const void *Q, *K, *V;            // K null: queries alone; V: cache writes only
    size_t q_stride, k_stride, v_stride;
    const void *wq, *wk;              // null: no norm
    const int *positions;
    const unsigned long long *freqs;
    const int *slots;                 // null: dense keys
    void *Qo, *Ko;                    // dense outputs (Ko null with slots)
    void *K_cache, *V_cache;
    const void *dQo, *dKo;            // backward
    float *partial;                   // backward: [blocks][2][d]
    float *dwq, *dwk;
    float *K_scale, *V_scale;         // 8-bit caches
    int n_tok, Hq, Hkv, d;
    int rot, interleaved, page_size, n_pages;
    float scale, eps;
    unsigned *err;
    bool beside;                      // runs beside the kernel before it in the stream (see qk_norm_rope.cu)
};
cudaError_t launch_qk_norm_rope(hybrid_dtype dt, const RopeArgs &a, cudaStream_t st);
cudaError_t launch_qk_norm_rope_backward(hybrid_dtype dt, const RopeArgs &a, cudaStream_t st);
size_t qk_norm_rope_partial_bytes(int d, int n_tok);

// cache_quant.cu
cudaError_t launch_qk_norm_rope_cache_quant(hybrid_dtype dt, const RopeArgs &a, cudaStream_t st);   // Q may be null
struct DequantArgs {
    const void *K_cache, *V_cache;
    const float *K_scale, *V_scale;
    const int *slots;
    void *K, *V;
    int n_tok, Hkv, d, page_size, n_pages;
    unsigned *err;
};
cudaError_t launch_cache_dequant(hybrid_dtype dt, const DequantArgs &a, cudaStream_t st);

// paged_attn.cu (float32, and the join of split requests), paged_attn_tc.cu (bfloat16)
namespace paged {
struct JoinNote;
}
struct PagedArgs {
    const void *Q, *K, *V;
    const float *K_scale, *V_scale;   // 8-bit caches
    const int *table, *lens;
    void *O;
    paged::JoinNote *notes;           // workspace, see paged_plan.cuh
    float *part;
    int n_req, B, Hq, Hkv, G, d;
    int page_size, n_pages, max_pages, window, sink;
    // a row tile is Bt tokens x Gt query heads of one key head
    int Gt, n_gt, Bt, n_bt;
    int n_cta;                        // blocks that share the tiles
    int extra;                        // quarters of a tile that a unit costs besides its tiles
    unsigned *err;
};
// Geometry (row tiles, number of blocks) of a call; pointers left to the caller.
void paged_geometry(const hybrid_cfg &c, PagedArgs &a);
size_t paged_workspace_bytes(const PagedArgs &a);
void paged_set_workspace(PagedArgs &a, void *workspace);
// Without the join: bfloat16; float32 with row tiles of at most kFewestRows rows.
cudaError_t launch_paged_attn_tc(const PagedArgs &a, cudaStream_t st);
constexpr int kFewestRows = 8;
cudaError_t launch_paged_attn_few(const PagedArgs &a, cudaStream_t st);
cudaError_t launch_paged_attn(hybrid_dtype dt, const PagedArgs &a, cudaStream_t st);
// The join of a call whose attention kernel was launched just before.
cudaError_t launch_paged_join(hybrid_dtype dt, const PagedArgs &a, cudaStream_t st);
// The same over an 8-bit cache: paged_attn_quant.cu (float32, and few rows), paged_attn_quant_tc.cu
void paged_quant_geometry(const hybrid_cfg &c, PagedArgs &a);
cudaError_t launch_paged_attn_quant_tc(const PagedArgs &a, cudaStream_t st);     // without the join
cudaError_t launch_paged_attn_quant(hybrid_dtype dt, const PagedArgs &a, cudaStream_t st);
// Row tiles of at most `most` rows, of about equal size along the tokens.
void paged_cut_rows(PagedArgs &a, int most);

}  // namespace hyb
