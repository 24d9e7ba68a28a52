// The paged latent cache: arguments and launchers of the append and attention kernels, and the device functions they share
// (sequence bounds, page lookup, output rows).
#pragma once
#include "common.h"
#include "params.h"

namespace ta {

// n / d for 0 <= n < 2^31 by one high product: mul = ceil(2^(31+shift) / d), shift = ceil(log2 d)
struct Divisor {
  uint32_t mul;
  int shift;
};
inline Divisor divisor(int d) {
  int s = 0;
  while ((1l << s) < d) ++s;
  return {(uint32_t)(((1ul << (31 + s)) + d - 1) / d), s};
}

struct PagedArgs {
  // pool: page j of the keys starts k_stride * j elements behind K, its rows r3 wide; values alike (null: shared latent)
  const void *K, *V;
  long k_stride, v_stride;
  int n_pages, page_size;
  Divisor ps;
  // batch: device arrays as the header describes them, and the bounds that keep every access inside the buffers
  const int *q_start, *kv_len, *table;
  int B, T, max_pages, max_new, max_len;
  const int* prefix_table;      // pages of rows 0 .. prefix-1 of every sequence
  int prefix;                   // 0: none
  // queries [T][nH] rows of q_row elements, outputs [T][nH] rows of o_row elements, log-sum-exp [T][nH] (nullable)
  const void* Q;
  void* O;
  float* lse;
  int q_row, o_row, o_acc;      // o_acc: output channels at their acc-order positions, all D of them
  int nH, r3, rt3, D;
  Divisor heads;
  float scale;                  // of a score, times log2(e)
  int causal, shared_kv;
  const float4* rope;           // [D/4][rope_ld] as in GemmArgs, or null; read for a shared latent only
  int rope_ld;
  // partial results of a row (un-normalised output in fp32; running maximum in the base-2 domain and sum)
  float* part_o;                // [parts][T * nH][D]
  float2* part_ml;              // [parts][T * nH]
  int prefix_parts;             // parts 0 .. prefix_parts-1: the prefix
  int own_parts;                // then those of the sequence's own rows (bf16: one, of rows that one workgroup does alone); 0: written to O
  int prefix_keys, own_keys;    // keys of such parts (a short sequence leaves the last parts empty: no output, a sum of 0)
  // The keys of all sequences dealt to this many workgroups (0: a workgroup for every sequence, or row block): of paged_stream, which
  // takes a sequence's `hb` blocks of 32 rows at once, and of paged_tile.  Rows that several workgroups share leave partial results:
  // [workgroups][hb * 32] rows, [2 * workgroups][kTileRows].
  int hb, stream_wgs, tile_wgs;
  float* stream_o;
  float2* stream_ml;
  int2* stream_parts;           // paged_stream: for every sequence its first workgroup and how many share it
  double tile_per_key;          // paged_tile: work of a key of a row block, 1 / (kTileUnit nH)
  // paged_tile: [0]: number of shares, then for each, if its start is the first in a row block behind the block's own: first row of the
  // block, its rows (0 otherwise), last share in it, whether the first share in it begins in an earlier block
  int4* tile_cuts;
  // with a prefix: workgroups of its pieces (a multiple of 8; those above follow in the same launch), and for every row where the
  // first share left its result and how many shares follow (0: that result is the row's own)
  int prefix_wgs;
  int2* tile_rows;
};
// Keys of a unit of paged_stream's work, least units of a workgroup.  us with 1, 2, 4 of them, 32 heads of 128 channels: one sequence of
// 4096 rows 14.2, 15.5, 19.4; 24 of up to 2000 14.6, 15.8, 19.2; 16 of 4096 19.4, 19.5, 20.8.
constexpr int kStreamUnit = 128, kStreamLeast = 2;
// whether two of its workgroups share a compute unit by design (KIND 1: one pool, keys rotated on use)
constexpr bool stream_late(int D, int kind) { return D == 128 && kind == 1; }
// Latent rows into their pages, keys (and the per-head queries, if given) rotated to the tokens' positions
struct PagedAppendArgs {
  void *K, *V;                  // pools as above
  long k_stride, v_stride;
  int n_pages, page_size;
  Divisor ps;
  const int *q_start, *kv_len, *table;
  int B, T, max_pages, max_new, max_len;
  const void *Kin, *Vin, *Qin;  // rows of ldk, ldv elements; [T][nH] rows of q_row elements
  void* Qout;
  long ldk, ldv;
  int q_row, nH, r3, rt3;
  int rotate_k;                 // 0: key rows are stored as they come
  const float4* rope;           // null: nothing is rotated
  int rope_ld;
};

constexpr long kMaxGroups = (1l << 24) - 1;            // workgroups of 256 that a launch takes along x (2^32 threads are refused)
int paged_rows_blocks(const PagedArgs& a, int rows);   // row blocks of `rows` rows that a batch can have
bool paged_append_fits(int dtype, const PagedAppendArgs& a);   // into one launch
hipError_t launch_paged_append(int dtype, const PagedAppendArgs& a, hipStream_t s);
hipError_t launch_paged_rows(const PagedArgs& a, bool prefix_pass, hipStream_t s);   // fp32
hipError_t launch_paged_stream(const PagedArgs& a, hipStream_t s);   // bf16
hipError_t launch_paged_join(const PagedArgs& a, hipStream_t s);     // of its partial results
hipError_t launch_paged_tile(const PagedArgs& a, bool prefix_pass, hipStream_t s);   // bf16
// Rows of a workgroup of paged_tile, keys of a unit of its work, units that a row block costs besides, least units of a share.  us with 2, 4,
// 8 of these, 32 heads of 128 channels: five sequences with four new tokens on 3012 rows 20.4, 22.3, 27.1; 100 on 600, twice 25.1, 25.7,
// 30.0; 140 single tokens on up to 1024 22.5, 23.2, 27.0; four times 512 on 4097 170, 169, 169.
constexpr int kTileRows = 128, kTileUnit = 64, kTileBlock = 3, kTileLeast = 4;
hipError_t launch_paged_tile_join(const PagedArgs& a, hipStream_t s);
hipError_t launch_paged_merge(const PagedArgs& a, hipStream_t s);   // fp32

// ---- device -----------------------------------------------------------------------------------------------------
__device__ __forceinline__ int divide(int n, Divisor d) { return (int)(__umulhi((uint32_t)n * 2u, d.mul) >> d.shift); }

// Sequence b of a batch.  What the arrays hold is bounded here, so that no value in them leads outside a buffer.
struct PagedSeq {
  int q0, nq;                   // its new tokens
  int len;                      // its cached rows
};
template <typename A> __device__ __forceinline__ PagedSeq paged_seq(const A& p, int b) {
  PagedSeq s;
  const int q1 = min(max(p.q_start[b + 1], 0), p.T);
  s.q0 = min(max(p.q_start[b], 0), p.T);
  s.nq = min(max(q1 - s.q0, 0), p.max_new);
  s.len = min(max(p.kv_len[b], 0), p.max_len);
  return s;
}

// Page of a table entry; a number that is no page of the pool reads page 0
__device__ __forceinline__ int paged_page(int entry, int n_pages) { return (uint32_t)entry < (uint32_t)n_pages ? entry : 0; }

// Which sequence item target(total) belongs to when every sequence has items(b) of them, one behind the other, `total` together: the
// sequence's number (-1: behind the last, or before the first), the item's index in it.  All 256 threads call; `sh` holds 6 words.
template <class G, class F>
__device__ __forceinline__ int paged_locate(int B, G target, F items, int* sh, int& index, int& total) {
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int per = (B + 255) / 256, first = tid * per, last = min(B, first + per);
  int mine = 0;
  for (int b = first; b < last; ++b) mine += items(b);
  int x = mine;
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) {
    const int y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  constexpr int W = 256 / kWave;
  if (lane == kWave - 1) sh[wave] = x;
  if (tid == 0) sh[W] = -1;
  __syncthreads();
  int before = x - mine;
  total = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    total += sh[w];
    before += w < wave ? sh[w] : 0;
  }
  const int at = target(total);
  if (at >= before && at < before + mine) {
    int b = first;
    if (per > 1)
      for (int n; at >= before + (n = items(b)); ++b) before += n;
    sh[W] = b;
    sh[W + 1] = at - before;
  }
  __syncthreads();
  index = sh[W + 1];
  const int found = sh[W];
  __syncthreads();
  return found;
}

// `units` units of work in equal shares for at most `wgs` workgroups, at least `least` units each (the first units % G have one more)
struct Shares {
  int n, more, G;
  __device__ __forceinline__ Shares(int units, int wgs, int least) {
    G = max(1, min(wgs, (units + least - 1) / least));
    n = units / G;
    more = units % G;
  }
  __device__ __forceinline__ int first(int g) const { return g * n + min(g, more); }         // unit of workgroup g
  __device__ __forceinline__ int group(int u) const {                                        // workgroup of unit u
    const int m = more * (n + 1);
    return u < m ? u / (n + 1) : more + (u - m) / n;
  }
};

// four output channels c .. c+3 of one row
template <typename T>
__device__ __forceinline__ void paged_store4(const PagedArgs& p, long row, int c, f32x4 v) {
  T* o = static_cast<T*>(p.O) + row * p.o_row;
  if (p.o_acc) {
    if (c >= p.rt3) v = f32x4{0.f, 0.f, 0.f, 0.f};
    store4(o + (c & ~31) + acc_pos(c & 31), v[0], v[1], v[2], v[3]);
  }
  else if (c < p.rt3) store4(o + c, v[0], v[1], v[2], v[3]);
}
constexpr float kLn2 = 0.69314718055994531f;

}  // namespace ta
