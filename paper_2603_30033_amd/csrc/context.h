// What the host files of the library share: the context, workspace carving, weight preparation, per-kernel timing.
#pragma once
#include "../../include/tucker_attn.h"

#include <hip/hip_runtime.h>

#include <cstring>

#include "common.h"
#include "params.h"

namespace ta {
constexpr int kMaxKernels = 40;
constexpr size_t kAlign = 256;
constexpr long kMaxTokens = 65535l * 32;   // token rows of a call (32-row tiles along a grid dimension)
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
}  // namespace ta

struct tucker_attn_ctx {
  tucker_attn_config cfg;
  int R2, RT2, D, dp;          // padded ranks, common K/V width, padded d
  int es;                      // bytes per stored element
  float4* rope;                // device [D/4][max_positions] (cos, sin, cos, sin) or null
  float qscale;                // log2(e) / sqrt(d_head), folded into the head-mixed core
  int n_cus;                   // compute units of the device current at create (256 if none could be asked)
  int profile;
  int n_kernels;
  const char* names[ta::kMaxKernels];
  hipEvent_t ev[ta::kMaxKernels + 1];
  hipEvent_t kev[2];           // start and end of the dominant kernel itself (attached to its dispatch)
  const char* kev_name;        // null until such a launch has been made with profiling on
  bool ev_created;
  // prepared weights (tucker_attn_prepare_weights): caller-owned buffer in the layout of
  // carve_weights, and the weight pointers it was made from
  void* prepared;
  tucker_attn_weights prepared_from;
};

namespace ta {

struct Carver {
  char* base;
  size_t off;
  template <typename P> P* take(size_t bytes) {
    P* p = reinterpret_cast<P*>(base + off);
    off += align_up(bytes);
    return p;
  }
};

inline void carve_weights(const tucker_attn_ctx* c, Carver& cv, void*& Gt, void*& Gtil2, void*& Wcat, void*& Ut2p) {
  const tucker_attn_config& f = c->cfg;
  Gt = cv.take<char>((size_t)f.n_heads * c->D * c->R2 * c->es);
  Gtil2 = cv.take<char>((size_t)c->RT2 * f.n_heads * c->D * c->es);
  Wcat = cv.take<char>((size_t)(c->R2 + 2 * c->D) * c->dp * c->es);
  Ut2p = cv.take<char>((size_t)c->dp * c->RT2 * c->es);
}

// Head-mixed query core as rows [n_heads * D][R2]: the calls over pages keep their queries in memory and make them with one
// product.  Behind carve_weights in a prepared buffer.
inline void* carve_query_core(const tucker_attn_ctx* c, Carver& cv) {
  return cv.take<char>((size_t)c->cfg.n_heads * c->D * c->R2 * c->es);
}

// The operand-layout copies of the weights: a piece of the call's workspace, or the caller's
// prepared buffer when one is registered (then no preparation kernel runs).
template <typename W> inline void use_prepared(const tucker_attn_ctx* c, W& w) {
  if (!c->prepared) return;
  Carver cv{static_cast<char*>(c->prepared), 0};
  carve_weights(c, cv, w.Gt, w.Gtil2, w.Wcat, w.Ut2p);
}

inline bool same_weights(const tucker_attn_weights& a, const tucker_attn_weights& b) {
  return a.C == b.C && a.U1 == b.U1 && a.U2 == b.U2 && a.U3 == b.U3 && a.Ct == b.Ct && a.Ut1 == b.Ut1 &&
         a.Ut2 == b.Ut2 && a.Ut3 == b.Ut3;
}

inline void add_job(PrepArgs& pa, const void* src, const void* coef, void* out, int A, int rows, int cols, int Z,
             int rows_pad, int cols_pad, long sz, long su, int transposed, int perm, float scale, int frag = 0) {
  PrepJob& j = pa.job[pa.n_jobs++];
  j.src = src; j.coef = coef; j.out = out;
  j.A = A; j.rows = rows; j.cols = cols; j.Z = Z;
  j.rows_pad = rows_pad; j.cols_pad = cols_pad;
  j.out_stride_z = sz; j.out_stride_u = su;
  j.transposed = transposed; j.perm = perm; j.scale = scale; j.frag = frag;
  j.first_block = pa.total_blocks;
  pa.total_blocks += prep_job_blocks(j);
}

// head-mixed cores (Gt or Gq null: not that one) and factor matrices in MFMA operand layout; returns the output-factor pointer
inline PrepArgs make_prep(const tucker_attn_ctx* c, const tucker_attn_weights* w, void* Gt, void* Gtil2, void* Wcat,
                   void* Ut2p, const void** ut2_used, long* ut2_ld, bool with_wcat = true, void* Gq = nullptr) {
  const tucker_attn_config& f = c->cfg;
  const int es = c->es;
  PrepArgs pa;
  std::memset(&pa, 0, sizeof(pa));
  const long nHD = (long)f.n_heads * c->D;
  // Gt[i][c][b] = qscale * sum_a U1[i,a] C[a,b,c], fragment-major 32x32 blocks of (c, b)
  if (Gt)
    add_job(pa, w->C, w->U1, Gt, f.r1, f.r2, f.r3, f.n_heads, c->R2, c->D, (long)c->D * c->R2, c->R2, 1, 1, c->qscale, 1);
  // Gq[i*D + c][b] = sum_a U1[i,a] C[a,b,c], b in acc order like the query latents
  if (Gq) add_job(pa, w->C, w->U1, Gq, f.r1, f.r2, f.r3, f.n_heads, c->R2, c->D, (long)c->D * c->R2, c->R2, 1, 1, 1.f);
  // Gtil2[b][i*D + c] = sum_a U~1[i,a] C~[a,b,c]
  add_job(pa, w->Ct, w->Ut1, Gtil2, f.rt1, f.rt2, f.rt3, f.n_heads, c->RT2, c->D, c->D, nHD, 0, 1, 1.f);
  // Wcat rows: U2^T | U3^T | U~3^T, each [rank_pad][dp]
  char* wc = static_cast<char*>(Wcat);
  if (with_wcat) {
    add_job(pa, w->U2, nullptr, wc, 1, f.d_model, f.r2, 1, c->dp, c->R2, 0, c->dp, 1, 0, 1.f);
    add_job(pa, w->U3, nullptr, wc + (size_t)c->R2 * c->dp * es, 1, f.d_model, f.r3, 1, c->dp, c->D, 0, c->dp, 1, 0, 1.f);
    if (!f.shared_kv)
      add_job(pa, w->Ut3, nullptr, wc + (size_t)(c->R2 + c->D) * c->dp * es, 1, f.d_model, f.rt3, 1, c->dp, c->D, 0,
              c->dp, 1, 0, 1.f);
  }
  if (f.rt2 != c->RT2) {
    add_job(pa, w->Ut2, nullptr, Ut2p, 1, f.d_model, f.rt2, 1, c->dp, c->RT2, 0, c->RT2, 0, 0, 1.f);
    *ut2_used = Ut2p;
  } else {
    *ut2_used = w->Ut2;
  }
  *ut2_ld = c->RT2;
  return pa;
}

struct Recorder {
  tucker_attn_ctx* c;
  hipStream_t s;
  bool on;
  hipError_t begin() {
    c->n_kernels = 0;
    if (!on) return hipSuccess;
    return hipEventRecord(c->ev[0], s);
  }
  hipError_t after(const char* name) {
    if (!on) return hipSuccess;
    if (c->n_kernels >= kMaxKernels) return hipSuccess;
    c->names[c->n_kernels] = name;
    ++c->n_kernels;
    return hipEventRecord(c->ev[c->n_kernels], s);
  }
};

// Z = O Gtil2^T (latent merge of the heads) and Y = Z U~2^T, over B x Npad token rows of which N of every Npad exist
inline GemmArgs merge_product(const tucker_attn_ctx* c, const void* Gtil2, const void* O, void* Z, int B, int N, int Npad) {
  GemmArgs z;
  std::memset(&z, 0, sizeof(z));
  z.A = Gtil2; z.lda = (long)c->cfg.n_heads * c->D; z.M = c->RT2;
  z.Bsrc = O; z.ldb = (long)c->cfg.n_heads * c->D; z.K = c->cfg.n_heads * c->D;
  z.Bsz = B; z.N = N; z.Npad = Npad; z.src_padded = 1;
  z.epi = 1; z.Out = Z; z.ldo = c->RT2; z.ksplit = 1; z.R2 = 0; z.D = 0;
  return z;
}
inline hipError_t launch_output(const tucker_attn_ctx* c, const void* ut2, long ut2_ld, const void* Z, void* Y, int B, int N, int Npad,
                                hipStream_t s) {
  GemmArgs y;
  std::memset(&y, 0, sizeof(y));
  y.A = ut2; y.lda = ut2_ld; y.M = c->cfg.d_model;
  y.Bsrc = Z; y.ldb = c->RT2; y.K = c->RT2;
  y.Bsz = B; y.N = N; y.Npad = Npad; y.src_padded = 1;
  y.epi = 2; y.Out = Y; y.ldo = c->cfg.d_model; y.ksplit = 1;
  return out_proj_supported(c->cfg.dtype, y) ? launch_out_proj(c->cfg.dtype, y, s) : launch_gemm(c->cfg.dtype, y, s);
}

inline bool weights_ok(const tucker_attn_ctx* c, const tucker_attn_weights* w) {
  return c && w && w->C && w->U1 && w->U2 && w->U3 && w->Ct && w->Ut1 && w->Ut2 && (w->Ut3 || c->cfg.shared_kv);
}

}  // namespace ta
