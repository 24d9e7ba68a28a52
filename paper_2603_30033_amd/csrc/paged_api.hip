// Host side of the paged latent cache: argument checks, the split of a call's work, launches.
#include <algorithm>

#include "context.h"
#include "paged.h"

using namespace ta;

namespace {

// (no kernel here has events of its own: what a forward call left there is not this call's)
hipError_t begin(Recorder& rec) {
  if (rec.on) rec.c->kev_name = nullptr;
  return rec.begin();
}

constexpr long kMaxRows = 1l << 31;   // (token, head) rows of a call
constexpr int kMaxLen = (int)((1l << 31) - (1l << 17));   // cached rows of a sequence: the kernels round row numbers up, to whole units and parts

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

int check_batch(const tucker_attn_ctx* c, const tucker_attn_batch* b) {
  if (!c || !b || b->B < 1 || b->T < 1 || b->max_pages < 1 || b->max_new < 1 || b->max_len < 1) return TUCKER_ATTN_INVALID_ARG;
  const tucker_attn_config& f = c->cfg;
  if (f.use_rope && b->max_len > f.max_positions) return TUCKER_ATTN_INVALID_ARG;
  if ((long)b->T * f.n_heads >= kMaxRows || b->max_len > kMaxLen) return TUCKER_ATTN_UNSUPPORTED_SHAPE;
  if ((f.r3 * c->es) % 16 != 0 || (f.rt3 * c->es) % 16 != 0) return TUCKER_ATTN_UNSUPPORTED_SHAPE;
  return TUCKER_ATTN_OK;
}

int check_pool(const tucker_attn_ctx* c, const tucker_attn_pages* p, const tucker_attn_batch* b) {
  if (!p || !p->K || p->n_pages < 1 || p->page_size < 1) return TUCKER_ATTN_INVALID_ARG;
  const tucker_attn_config& f = c->cfg;
  if (f.shared_kv ? p->V != nullptr : p->V == nullptr) return TUCKER_ATTN_INVALID_ARG;
  if (!aligned16(p->K) || !aligned16(p->V)) return TUCKER_ATTN_INVALID_ARG;
  auto stride_ok = [&](int64_t s, int r) { return s == 0 || (s >= (int64_t)p->page_size * r && (s * c->es) % 16 == 0); };
  if (!stride_ok(p->k_stride, f.r3) || (!f.shared_kv && !stride_ok(p->v_stride, f.rt3))) return TUCKER_ATTN_INVALID_ARG;
  // (the kernels count 16-byte units of a pool in 32 bits)
  auto small = [&](int64_t s, int r) { return (double)p->n_pages * (s ? s : (double)p->page_size * r) * c->es < 16.0 * 0xffffffffu; };
  if (!small(p->k_stride, f.r3) || (!f.shared_kv && !small(p->v_stride, f.rt3))) return TUCKER_ATTN_UNSUPPORTED_SHAPE;
  if (!b->q_start || !b->kv_len || !b->page_table) return TUCKER_ATTN_INVALID_ARG;
  if (b->max_len > (long)b->max_pages * p->page_size) return TUCKER_ATTN_INVALID_ARG;
  return TUCKER_ATTN_OK;
}

// Most new tokens of a sequence: the caller's bound, which may be any number, cut to the tokens there are (so that rows of a sequence are
// counted in 31 bits like those of the call)
int most_new(const tucker_attn_batch* b) { return std::min(b->max_new, b->T); }

template <typename A> void fill(A& a, const tucker_attn_ctx* c, const tucker_attn_pages* p, const tucker_attn_batch* b) {
  const tucker_attn_config& f = c->cfg;
  a.K = p->K; a.V = p->V;
  a.k_stride = p->k_stride ? p->k_stride : (long)p->page_size * f.r3;
  a.v_stride = p->v_stride ? p->v_stride : (long)p->page_size * f.rt3;
  a.n_pages = p->n_pages; a.page_size = p->page_size; a.ps = divisor(p->page_size);
  a.q_start = b->q_start; a.kv_len = b->kv_len; a.table = b->page_table;
  a.B = b->B; a.T = b->T; a.max_pages = b->max_pages; a.max_new = most_new(b); a.max_len = b->max_len;
  a.nH = f.n_heads; a.r3 = f.r3; a.rt3 = f.rt3;
  a.rope = c->rope; a.rope_ld = f.max_positions;
}

// Parts that the keys of a product of `blocks` row blocks are dealt to: `wgs` workgroups for every compute unit, and no more parts than
// ones of `least` keys would be
int key_parts(const tucker_attn_ctx* c, long blocks, int keys, int wgs, int least) {
  const long most = (keys + least - 1) / least, want = (long)wgs * c->n_cus / (blocks < 1 ? 1 : blocks);
  return (int)(want < 1 || most < 1 ? 1 : want < most ? want : most);
}

// Keys of each of these parts, whole tiles; and the parts that then hold any (4097 keys in 16 parts: 13 of 320)
int part_keys(int keys, int& parts) {
  if (keys < 1) return 64;
  const int each = ((keys + parts - 1) / parts + 63) / 64 * 64;
  parts = (keys + each - 1) / each;
  return each;
}

// Longest keys that one workgroup takes alone rather than several and a second launch that joins their results.  us with 256, 512, 1024, 32
// heads of 128 channels: one sequence of 300 rows 15.8, 12.4, 12.5; of 500 15.5, 14.4, 14.4; of 700 15.4, 15.4, 18.3; of 1000 15.4, 15.5,
// 22.1; 64 of 1000 19.2, 19.0, 23.4.
constexpr int kStreamWhole = 512;

// What of a call depends on its bounds alone: which kernels, the parts of their work, the workspace.  Returns its bytes.
size_t plan(const tucker_attn_ctx* c, const tucker_attn_batch* b, int prefix, void* ws, PagedArgs& a) {
  const tucker_attn_config& f = c->cfg;
  a.B = b->B; a.T = b->T; a.nH = f.n_heads; a.D = c->D; a.prefix = prefix;
  const long rows = (long)b->T * f.n_heads, most = (long)most_new(b) * f.n_heads;
  const int keys = b->max_len - prefix;
  const bool tile = f.dtype == TUCKER_ATTN_BF16;                  // (fp32 rows go through paged_rows)
  const int block = tile ? kTileRows : 32;
  // least keys of a prefix's part, us with half, these, twice: seven sequences behind 777 rows, 12 heads of 64, 12.3, 12.9, 15.2 (fp32 19.3,
  // 19.6, 22.9); four behind 2000, 32 heads of 128, 14.1, 16.6, 22.5; two behind 16384 15.5, 16.4, 21.3; 32 behind 16384 30.7, 30.8, 30.9
  a.prefix_parts = prefix > 0 ? key_parts(c, (rows + block - 1) / block, prefix, tile ? 1 : 2, tile ? 256 : 128) : 0;
  if (tile && prefix > 0) {
    // ... and no more of the two workgroups a compute unit than its share of the work, the sequences' own keys at half their bound (128
    // sequences of up to 2048 rows behind 2048: 33 us, with one workgroup a compute unit for the prefix 39)
    const double work = (double)prefix * ((rows + block - 1) / block), own = .5 * paged_rows_blocks(a, block) * (keys + kTileBlock * kTileUnit);
    const long share = (long)(2 * c->n_cus * work / (work + own)) / ((rows + block - 1) / block);
    a.prefix_parts = (int)std::max(1l, std::min(share, (long)a.prefix_parts));
  }
  a.prefix_keys = a.prefix_parts > 0 ? part_keys(prefix, a.prefix_parts) : 0;
  const long pieces = (rows + block - 1) / block * a.prefix_parts;
  a.prefix_wgs = (int)((pieces + 7) / 8 * 8);
  // Few rows and no prefix: paged_stream, unless there are so many sequences that its workgroups could not have equal shares.  us,
  // 32 heads of 128 channels, paged_stream and paged_tile: 128 sequences of up to 1024 rows 20.4, 23.1; 140: 25.2, 23.3; 200: 28.2, 25.4;
  // 16 of 4096 19.2, 21.4; one of 32768 17.9, 19.9; 12 heads of 64: one of 257 8.4, 11.2; 140 of up to 3000 30.6, 21.9, of 3000 42.2, 28.7; a
  // shared latent (twice the workgroups): 140 of 3000 55.4, 57.6, 250 72.1, 102.7.
  // One more row than paged_stream takes: 16 sequences of 4096 with 32 heads 18.1, with 33 23.2, with 64 27.1, with 2 tokens of 32 27.9.
  // A prompt's piece sends the single tokens beside it to paged_tile: 32 of them on 2000 rows 18.4, 512 tokens on 2048 46.8, in one call 50.3.
  // Behind a prefix their keys go with the prefix's own launch, which paged_tile does (with this kernel beside it, in two launches, before
  // the joins became what they are: 32 sequences behind 16384 rows 44, in one 35; 128 with up to 1024 rows of their own 46, 33; 16 with
  // 32768 68, 57).
  const int wgs = (stream_late(c->D, f.shared_kv && f.use_rope ? 1 : 0) ? 2 : 1) * c->n_cus;
  const bool split = keys > kStreamWhole;
  const bool even = 2 * (long)b->B <= wgs && b->B <= 256 && (long)b->B * (keys / kStreamUnit + 1) < (1l << 31);   // (units in 32 bits)
  a.hb = !tile || prefix > 0 || (split && !even) ? 0 : most <= 32 ? 1 : most <= 64 && c->D < 128 ? 2 : 0;
  a.stream_wgs = a.tile_wgs = 0;
  a.own_parts = prefix > 0 ? 1 : 0;                               // rows that one workgroup does alone
  long shared = 0;                                                // rows of partial results that workgroups share
  if (a.hb > 0) {
    if (split) {
      a.stream_wgs = wgs;
      shared = (long)wgs * a.hb * 32;
    }
  } else if (tile) {
    const long blocks = paged_rows_blocks(a, block), units = (keys + kTileUnit - 1) / kTileUnit;
    if (const long work = blocks * (units + kTileBlock); units > kTileLeast && work < (1l << 31)) {
      // every die's workgroups have a place at once beside the prefix's; no more than there can be shares
      a.tile_wgs = std::max(2 * c->n_cus - std::min(a.prefix_wgs, 2 * c->n_cus), c->n_cus);
      a.tile_wgs = (int)std::min((long)a.tile_wgs, (work + kTileLeast - 1) / kTileLeast);
    }
    a.tile_per_key = 1. / (kTileUnit * (double)f.n_heads);
    shared = 2l * a.tile_wgs * kTileRows;
  } else {
    // (least keys 64, 128, 256: five proposed tokens on 700 rows, three sequences of 12 heads of 64, 12.6, 12.9, 16.2 us; one token on 257
    // 11.8, 11.8, 14.8)
    int parts = key_parts(c, paged_rows_blocks(a, block), keys, 2, 128);
    a.own_keys = part_keys(keys, parts);
    if (parts > 1) a.own_parts = parts;
  }
  const size_t parts = a.prefix_parts + a.own_parts;
  Carver cv{static_cast<char*>(ws), 0};
  a.part_o = cv.take<float>(parts * rows * c->D * 4);
  a.part_ml = cv.take<float2>(parts * rows * 8);
  a.stream_o = cv.take<float>(shared * c->D * 4);
  a.stream_ml = cv.take<float2>(shared * 8);
  a.stream_parts = cv.take<int2>(a.stream_wgs > 0 ? b->B * sizeof(int2) : 0);
  a.tile_cuts = cv.take<int4>(prefix > 0 ? 0 : a.tile_wgs * sizeof(int4));
  a.tile_rows = cv.take<int2>(tile && prefix > 0 ? rows * sizeof(int2) : 0);
  return cv.off;
}

// Whether the launches of a planned call can be made: none has more workgroups than one takes.  (So rows counted in whole blocks stay
// within 31 bits too.)  Joins that go row by row: D/4 threads each where there are so many rows.
bool fits(const PagedArgs& a, bool bf16) {
  const long rows = (long)a.T * a.nH, blocks = paged_rows_blocks(a, bf16 ? kTileRows : 32);
  if (a.hb > 0) return a.B <= kMaxGroups;
  if (blocks + (bf16 ? a.prefix_wgs : 0) > kMaxGroups) return false;
  return a.prefix_parts + a.own_parts == 0 || (rows * (a.D / 4) + 255) / 256 <= kMaxGroups;
}

int check_prefix(const tucker_attn_batch* b, const int32_t* table, int32_t prefix) {
  return prefix < 0 || prefix > b->max_len || (prefix > 0 && !table) ? TUCKER_ATTN_INVALID_ARG : TUCKER_ATTN_OK;
}

// arguments of the attention over checked pages; returns the bytes of workspace it needs
size_t attend_args(PagedArgs& a, const tucker_attn_ctx* c, const tucker_attn_pages* pages, const tucker_attn_batch* batch,
                   const int32_t* prefix_table, int32_t prefix, void* workspace) {
  const tucker_attn_config& f = c->cfg;
  std::memset(&a, 0, sizeof(a));
  fill(a, c, pages, batch);
  a.prefix_table = prefix_table; a.q_row = f.r3; a.o_row = f.rt3;
  a.heads = divisor(f.n_heads); a.scale = c->qscale; a.causal = f.causal; a.shared_kv = f.shared_kv;
  return plan(c, batch, prefix, workspace, a);
}

int launch_attend(const tucker_attn_ctx* c, const PagedArgs& a, hipStream_t s, Recorder& rec) {
  const bool tile = c->cfg.dtype == TUCKER_ATTN_BF16;
  if (a.prefix > 0) {
    if ((tile ? launch_paged_tile(a, true, s) : launch_paged_rows(a, true, s)) != hipSuccess) return TUCKER_ATTN_HIP_ERROR;
    (void)rec.after("prefix_attention");
  }
  if (a.prefix == 0 || !tile) {                                   // (that launch of paged_tile did the sequences' own keys as well)
    if ((a.hb > 0 ? launch_paged_stream(a, s) : tile ? launch_paged_tile(a, false, s) : launch_paged_rows(a, false, s)) != hipSuccess)
      return TUCKER_ATTN_HIP_ERROR;
    (void)rec.after("paged_attention");
  }
  if (a.prefix_parts + a.own_parts + a.stream_wgs + a.tile_wgs > 0) {
    if ((a.hb > 0 ? launch_paged_join(a, s) : tile ? launch_paged_tile_join(a, s) : launch_paged_merge(a, s)) != hipSuccess)
      return TUCKER_ATTN_HIP_ERROR;
    (void)rec.after("paged_merge");
  }
  return TUCKER_ATTN_OK;
}

int attend(tucker_attn_ctx* c, const tucker_attn_pages* pages, const tucker_attn_batch* batch, const int32_t* prefix_table,
           int32_t prefix, const void* Q, void* O, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (int st = check_batch(c, batch)) return st;
  if (int st = check_pool(c, pages, batch)) return st;
  if (!Q || !O || !aligned16(Q) || !aligned16(O) || reinterpret_cast<uintptr_t>(lse) % 4 != 0) return TUCKER_ATTN_INVALID_ARG;
  if (int st = check_prefix(batch, prefix_table, prefix)) return st;
  if (reinterpret_cast<uintptr_t>(workspace) % kAlign != 0) return TUCKER_ATTN_INVALID_ARG;
  PagedArgs a;
  const size_t need = attend_args(a, c, pages, batch, prefix_table, prefix, workspace);
  if (!fits(a, c->cfg.dtype == TUCKER_ATTN_BF16)) return TUCKER_ATTN_UNSUPPORTED_SHAPE;
  a.Q = Q; a.O = O; a.lse = lse;
  if (need > 0 && !workspace) return TUCKER_ATTN_INVALID_ARG;
  if (workspace_bytes < need) return TUCKER_ATTN_WORKSPACE_TOO_SMALL;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  Recorder rec{c, s, c->profile != 0};
  if (begin(rec) != hipSuccess) return TUCKER_ATTN_HIP_ERROR;
  return launch_attend(c, a, s, rec);
}

// Workspace of the layer over pages: operand copies of the weights, the tokens' latents, per-head queries and outputs (rows of D
// channels, the outputs' in acc order), merged latents; behind them that of the attention.
struct LayerWs {
  void *Gt, *Gtil2, *Wcat, *Ut2p, *Gq, *Qlat, *K, *V, *Q, *O, *Z;
  size_t bytes;
};
LayerWs carve_layer(const tucker_attn_ctx* c, void* ws, long T) {
  const tucker_attn_config& f = c->cfg;
  const size_t es = c->es, heads = (size_t)T * f.n_heads * c->D * es;
  Carver cv{static_cast<char*>(ws), 0};
  LayerWs w;
  carve_weights(c, cv, w.Gt, w.Gtil2, w.Wcat, w.Ut2p);
  w.Gq = w.Gt;                                                    // the same size, and this one is not needed
  w.Gt = nullptr;
  w.Qlat = cv.take<char>(T * c->R2 * es);
  w.K = cv.take<char>(T * f.r3 * es);
  w.V = cv.take<char>(f.shared_kv ? 0 : T * f.rt3 * es);
  w.Q = cv.take<char>(heads);
  w.O = cv.take<char>(heads);
  w.Z = cv.take<char>(T * c->RT2 * es);
  w.bytes = cv.off;
  return w;
}

}  // namespace

extern "C" {

int tucker_attn_append_paged(tucker_attn_ctx* c, const tucker_attn_pages* pages, const tucker_attn_batch* batch, const void* K,
                             int64_t ldk, const void* V, int64_t ldv, const void* Q, void* Qrot, int32_t rotate,
                             void* hip_stream) {
  if (int st = check_batch(c, batch)) return st;
  if (int st = check_pool(c, pages, batch)) return st;
  const tucker_attn_config& f = c->cfg;
  if (!K || (f.shared_kv ? V != nullptr : V == nullptr) || (Q == nullptr) != (Qrot == nullptr)) return TUCKER_ATTN_INVALID_ARG;
  if (rotate != 0 && rotate != 1) return TUCKER_ATTN_INVALID_ARG;
  if (!rotate && Q) return TUCKER_ATTN_INVALID_ARG;
  if (ldk < f.r3 || (V && ldv < f.rt3)) return TUCKER_ATTN_INVALID_ARG;
  for (const void* p : {K, V, Q, static_cast<const void*>(Qrot)})
    if (reinterpret_cast<uintptr_t>(p) % c->es != 0) return TUCKER_ATTN_INVALID_ARG;
  PagedAppendArgs a;
  std::memset(&a, 0, sizeof(a));
  fill(a, c, pages, batch);
  a.Kin = K; a.ldk = ldk; a.Vin = V; a.ldv = ldv; a.Qin = Q; a.Qout = Qrot; a.q_row = f.r3;
  a.rotate_k = rotate && !f.shared_kv;
  if (!paged_append_fits(f.dtype, a)) return TUCKER_ATTN_UNSUPPORTED_SHAPE;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  Recorder rec{c, s, c->profile != 0};
  if (begin(rec) != hipSuccess) return TUCKER_ATTN_HIP_ERROR;
  if (launch_paged_append(f.dtype, a, s) != hipSuccess) return TUCKER_ATTN_HIP_ERROR;
  (void)rec.after("paged_append");
  return TUCKER_ATTN_OK;
}

size_t tucker_attn_attend_workspace_bytes(const tucker_attn_ctx* c, const tucker_attn_batch* batch, int32_t prefix_len) {
  if (check_batch(c, batch) != TUCKER_ATTN_OK || prefix_len < 0 || prefix_len > batch->max_len) return 0;
  PagedArgs a;
  const size_t bytes = plan(c, batch, prefix_len, nullptr, a);
  return fits(a, c->cfg.dtype == TUCKER_ATTN_BF16) ? bytes : 0;
}

int tucker_attn_attend_paged(tucker_attn_ctx* c, const tucker_attn_pages* pages, const tucker_attn_batch* batch, const void* Q,
                             void* O, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
  return attend(c, pages, batch, nullptr, 0, Q, O, lse, workspace, workspace_bytes, hip_stream);
}

int tucker_attn_attend_prefix(tucker_attn_ctx* c, const tucker_attn_pages* pages, const tucker_attn_batch* batch,
                              const int32_t* prefix_table, int32_t prefix_len, const void* Q, void* O, float* lse,
                              void* workspace, size_t workspace_bytes, void* hip_stream) {
  return attend(c, pages, batch, prefix_table, prefix_len, Q, O, lse, workspace, workspace_bytes, hip_stream);
}

size_t tucker_attn_forward_paged_workspace_bytes(const tucker_attn_ctx* c, const tucker_attn_batch* batch, int32_t prefix_len) {
  if (check_batch(c, batch) != TUCKER_ATTN_OK || prefix_len < 0 || prefix_len > batch->max_len || batch->T > kMaxTokens) return 0;
  PagedArgs a;
  const size_t bytes = plan(c, batch, prefix_len, nullptr, a);
  return fits(a, c->cfg.dtype == TUCKER_ATTN_BF16) ? carve_layer(c, nullptr, batch->T).bytes + bytes : 0;
}

int tucker_attn_forward_paged(tucker_attn_ctx* c, const tucker_attn_weights* w, const void* X, void* Y, const tucker_attn_pages* pages,
                              const tucker_attn_batch* batch, const int32_t* prefix_table, int32_t prefix_len, void* workspace,
                              size_t workspace_bytes, void* hip_stream) {
  if (int st = check_batch(c, batch)) return st;
  if (int st = check_pool(c, pages, batch)) return st;
  if (!weights_ok(c, w) || !X || !Y || !workspace) return TUCKER_ATTN_INVALID_ARG;
  if (int st = check_prefix(batch, prefix_table, prefix_len)) return st;
  if (batch->T > kMaxTokens) return TUCKER_ATTN_UNSUPPORTED_SHAPE;
  if (reinterpret_cast<uintptr_t>(workspace) % kAlign != 0) return TUCKER_ATTN_INVALID_ARG;
  if (c->prepared && !same_weights(*w, c->prepared_from)) return TUCKER_ATTN_INVALID_ARG;
  const tucker_attn_config& f = c->cfg;
  const int T = batch->T;
  LayerWs ws = carve_layer(c, workspace, T);
  PagedArgs a;
  const size_t attend_bytes = attend_args(a, c, pages, batch, prefix_table, prefix_len, static_cast<char*>(workspace) + ws.bytes);
  PagedAppendArgs p;
  std::memset(&p, 0, sizeof(p));
  fill(p, c, pages, batch);
  p.Kin = ws.K; p.ldk = f.r3; p.Vin = f.shared_kv ? nullptr : ws.V; p.ldv = f.rt3;
  p.Qin = p.Qout = f.use_rope ? ws.Q : nullptr; p.q_row = c->D;   // (queries in place)
  p.rotate_k = !f.shared_kv;
  if (!fits(a, f.dtype == TUCKER_ATTN_BF16) || !paged_append_fits(f.dtype, p)) return TUCKER_ATTN_UNSUPPORTED_SHAPE;
  if (workspace_bytes < ws.bytes + attend_bytes) return TUCKER_ATTN_WORKSPACE_TOO_SMALL;

  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  Recorder rec{c, s, c->profile != 0};
  if (begin(rec) != hipSuccess) return TUCKER_ATTN_HIP_ERROR;
  if (c->prepared) {
    Carver cv{static_cast<char*>(c->prepared), 0};
    carve_weights(c, cv, ws.Gt, ws.Gtil2, ws.Wcat, ws.Ut2p);
    ws.Gq = carve_query_core(c, cv);
  }
  const void* ut2;
  long ut2_ld;
  const PrepArgs pa = make_prep(c, w, nullptr, ws.Gtil2, ws.Wcat, ws.Ut2p, &ut2, &ut2_ld, true, ws.Gq);
  if (!c->prepared) {
    if (launch_prep(f.dtype, pa, s) != hipSuccess) return TUCKER_ATTN_HIP_ERROR;
    (void)rec.after("prep_weights");
  }

  // the tokens of all sequences are the rows of each product; their latents are not rotated here
  GemmArgs g;
  std::memset(&g, 0, sizeof(g));
  g.A = ws.Wcat; g.lda = c->dp; g.M = c->R2 + (f.shared_kv ? 1 : 2) * c->D; g.shared_kv = f.shared_kv;
  g.Bsrc = X; g.ldb = f.d_model; g.K = f.d_model;
  g.Bsz = 1; g.N = T; g.Npad = T; g.src_padded = 1;
  g.epi = 0;
  g.Qlat = ws.Qlat; g.R2 = c->R2; g.D = c->D;
  g.Kcache = ws.K; g.Vcache = f.shared_kv ? nullptr : ws.V; g.Lmax = T; g.r3 = f.r3; g.rt3 = f.rt3;
  g.ksplit = 1;
  if (launch_gemm(f.dtype, g, s) != hipSuccess) return TUCKER_ATTN_HIP_ERROR;
  (void)rec.after("factor_projection");

  GemmArgs q;
  std::memset(&q, 0, sizeof(q));
  q.A = ws.Gq; q.lda = c->R2; q.M = f.n_heads * c->D;
  q.Bsrc = ws.Qlat; q.ldb = c->R2; q.K = c->R2;
  q.Bsz = 1; q.N = T; q.Npad = T; q.src_padded = 1;
  q.epi = 1; q.Out = ws.Q; q.ldo = q.M; q.ksplit = 1;
  if (launch_gemm(f.dtype, q, s) != hipSuccess) return TUCKER_ATTN_HIP_ERROR;
  (void)rec.after("head_queries");

  if (launch_paged_append(f.dtype, p, s) != hipSuccess) return TUCKER_ATTN_HIP_ERROR;
  (void)rec.after("paged_append");

  a.Q = ws.Q; a.q_row = c->D; a.O = ws.O; a.o_row = c->D; a.o_acc = 1;
  if (int st = launch_attend(c, a, s, rec)) return st;

  if (launch_gemm(f.dtype, merge_product(c, ws.Gtil2, ws.O, ws.Z, 1, T, T), s) != hipSuccess) return TUCKER_ATTN_HIP_ERROR;
  (void)rec.after("latent_merge");
  if (launch_output(c, ut2, ut2_ld, ws.Z, Y, 1, T, T, s) != hipSuccess) return TUCKER_ATTN_HIP_ERROR;
  (void)rec.after("output_projection");
  return TUCKER_ATTN_OK;
}

}  // extern "C"
