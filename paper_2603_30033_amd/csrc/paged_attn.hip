// Attention over the paged latent cache in fp32, and the join of its partial results.
//
// One latent key and value row serves all heads, so the rows of the product are the (token, head) pairs of a sequence, token by
// token: row r is head r % nH of new token r / nH.  Online softmax over the keys; a row sees the keys up to its token's own.
//
//   paged_rows   32 rows a workgroup, its four waves taking every fourth block of 32 keys straight from the pages
//   paged_merge  joins the partial results of a row: sum_i 2^(m_i - m) (l_i, O_i), m = max m_i
//
// The fp32 matrix instructions (64 cycles for 2 channels of 32 x 32) bound many rows; few rows are a chain of dependent loads (where
// the rows are, page, keys), so the keys of a row block are dealt to two workgroups a compute unit, down to 128 keys, one block a
// wave, and a block's value loads are on their way beside its key loads.
#include "paged_block.h"

namespace ta {

// ------------------------------------------------------------------------------------------------------------------
// 32 rows a workgroup
// ------------------------------------------------------------------------------------------------------------------
// Grid: row blocks x parts of the keys.  Key fragments come from memory as they are (a lane reads 16 channels of its key row);
// value fragments one element a lane, 32 consecutive channels of a row in half a wave.
template <int D, bool SH, bool PREFIX>
__global__ __launch_bounds__(256) void paged_rows_kernel(PagedArgs p) {
  using T = float;
  constexpr int CB = D / 32;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int h = lane / 32, lr = lane % 32;
  const int part = blockIdx.y;

  // ---- which rows, which keys ----
  int rb, n_rows, row0;                                           // block, rows of its sequence, first row of that in [T * nH]
  int first, len, nq, pages;
  const int* table;
  if constexpr (PREFIX) {
    rb = blockIdx.x;
    row0 = 0;
    nq = min(max(p.q_start[p.B], 0), p.T);
    n_rows = nq * p.nH;
    first = 0;
    len = p.prefix;
    table = p.prefix_table;
    pages = divide(p.prefix - 1, p.ps) + 1;
    if (rb * 32 >= n_rows) return;
  } else {
    int total;
    const int b = paged_locate(p.B, [](int) { return (int)blockIdx.x; }, [&](int i) { return (paged_seq(p, i).nq * p.nH + 31) / 32; },
                               reinterpret_cast<int*>(smem_raw), rb, total);
    if (b < 0) return;
    const PagedSeq s = paged_seq(p, b);
    nq = s.nq;
    row0 = s.q0 * p.nH;
    n_rows = nq * p.nH;
    first = p.prefix;
    len = s.len;
    table = p.table + (long)b * p.max_pages;
    pages = p.max_pages;
  }
  const bool causal = !PREFIX && p.causal;
  const int r = min(rb * 32 + lr, n_rows - 1);                    // rows behind the last repeat it and are not stored
  const int limit = causal ? len - nq + divide(r, p.heads) + 1 : len;          // keys that the row sees
  const int hi = causal ? len - nq + divide(min(rb * 32 + 31, n_rows - 1), p.heads) + 1 : len;
  const int lo = causal ? len - nq + divide(rb * 32, p.heads) + 1 : len;       // keys that all rows of the block see
  const int blocks = hi > first ? (hi - first + 31) / 32 : 0;
  const int per = (PREFIX ? p.prefix_keys : p.own_keys) / 32;
  const int k0 = part * per, k1 = min(blocks, k0 + per);

  Frag<T> qf[CB];
  {
    const T* q = static_cast<const T*>(p.Q) + (long)(row0 + r) * p.q_row;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) qf[cb] = load_frag_upto<T>(q, cb * 32 + 16 * h, p.r3);
  }
  f32x16 oacc[CB];
  float m_run = -INFINITY, l_run = 0.f;
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int e = 0; e < 16; ++e) oacc[cb][e] = 0.f;

  for (int k = k0 + wave; k < k1; k += 4) {
    const int n0 = first + k * 32;
    const int n = min(n0 + lr, hi - 1);                           // keys behind the last repeat it and are masked
    const int pi = divide(n, p.ps);
    const int page = paged_page(table[min(pi, pages - 1)], p.n_pages), at = n - pi * p.page_size;
    const T* krow = static_cast<const T*>(p.K) + page * p.k_stride + (long)at * p.r3;
    Frag<T> vf[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      const int c = min(cb * 32 + lr, p.rt3 - 1);                 // channels behind the last repeat it and are not stored
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int key = 8 * (e / 4) + 4 * h + e % 4;
        const long pg = __shfl(page, key), off = __shfl(at, key);
        const T* src = SH ? static_cast<const T*>(p.K) + pg * p.k_stride + off * p.r3
                          : static_cast<const T*>(p.V) + pg * p.v_stride + off * p.rt3;
        frag_set(vf[cb], e, src[c]);
      }
    }
    f32x16 s;
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      Frag<T> kf = load_frag_upto<T>(krow, cb * 32 + 16 * h, p.r3);
      if (SH && p.rope != nullptr) {
        const f32x4* tab = reinterpret_cast<const f32x4*>(p.rope) + (long)(8 * cb + 4 * h) * p.rope_ld + min(n, p.rope_ld - 1);
        f32x4 cs[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) cs[q] = tab[(long)q * p.rope_ld];
        turn_frag(kf, cs);
      }
      mma32(s, kf, qf[cb]);
    }
    const bool partly = n0 + 32 > lo;
    float mx = -INFINITY;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      s[e] *= p.scale;
      if (partly && n0 + 8 * (e / 4) + 4 * h + e % 4 >= limit) s[e] = -INFINITY;
      mx = fmaxf(mx, s[e]);
    }
    mx = halves_max(mx);
    const float m_new = fmaxf(m_run, mx), m_use = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = fast_exp2(m_run - m_use);
    m_run = m_new;
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = fast_exp2(s[e] - m_use);
    l_run = block_sum(s, l_run * alpha);
    const Frag<T> pf = to_frag<T>(s);
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
#pragma unroll
      for (int e = 0; e < 16; ++e) oacc[cb][e] *= alpha;
      if (__builtin_amdgcn_ballot_w64(!frag_finite(vf[cb])) != 0ull) take_nonfinite<T>(vf[cb], limit - n0 - 4 * h, oacc[cb]);
      mma32(oacc[cb], vf[cb], pf);
    }
  }

  __syncthreads();                                                // (the plan's words are done with)
  const bool direct = !PREFIX && p.own_parts == 0;
  const long row_first = (long)row0 + rb * 32;
  join_waves<D, 1>(reinterpret_cast<float*>(smem_raw), &oacc, &m_run, &l_run, n_rows - rb * 32, [&](int row, int c, float m, float l, f32x4 o) {
    if (direct) paged_result<T>(p, row_first + row, c, m, l, o);
    else paged_partial<D>(p.part_o, p.part_ml, (long)((PREFIX ? 0 : p.prefix_parts) + part) * p.T * p.nH + row_first + row, c, m, l, o);
  });
}

// ------------------------------------------------------------------------------------------------------------------
// partial results of a row joined: a row by D/4 threads, or by `groups` times as many that take every groups-th part
// ------------------------------------------------------------------------------------------------------------------
template <int D>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedArgs p, int groups) {
  constexpr int L = D / 4, SLOTS = 256 / L;
  __shared__ float4 po[256];
  __shared__ float2 pml[SLOTS];
  const int tid = threadIdx.x, slot = tid / L, c = tid % L * 4, per = SLOTS / groups, group = slot / per;
  const long rows = (long)p.T * p.nH, row = (long)blockIdx.x * per + slot % per;
  RowSum sum;
  if (row < rows)
    sum.add_parts(p.prefix_parts + p.own_parts, group, groups, [&](int i, const float2*& ml, const float*& o) {
      ml = p.part_ml + i * rows + row;
      o = p.part_o + (i * rows + row) * D + c;
    });
  const int q0 = min(max(p.q_start[0], 0), p.T), q1 = min(max(p.q_start[p.B], 0), p.T);
  const bool live = row >= (long)q0 * p.nH && row < (long)q1 * p.nH;   // not behind the last sequence
  sum.add_groups(po, pml, slot, group, groups, per, L);
  if (group == 0 && live) paged_result<float>(p, row, c, sum.m, sum.l, sum.o);
}

// ------------------------------------------------------------------------------------------------------------------
int paged_rows_blocks(const PagedArgs& a, int rows) {
  const long all = ((long)a.T * a.nH + rows - 1) / rows + (a.B < a.T ? a.B : a.T);
  return (int)(all < 0x7fffffffl ? all : 0x7fffffffl);
}

template <int D, bool SH, bool PREFIX> static hipError_t rows_one(const PagedArgs& a, hipStream_t s) {
  const size_t smem = join_bytes<D, 1>();
  auto kern = paged_rows_kernel<D, SH, PREFIX>;
  static LdsOnce lds_once;                                       // one per kernel instantiation
  if (hipError_t e = allow_dynamic_lds(lds_once, kern, smem); e != hipSuccess) return e;
  const int blocks = PREFIX ? (int)(((long)a.T * a.nH + 31) / 32) : paged_rows_blocks(a, 32);
  hipLaunchKernelGGL(kern, dim3(blocks, PREFIX ? a.prefix_parts : a.own_parts > 0 ? a.own_parts : 1), dim3(256), smem, s, a);
  return hipGetLastError();
}
template <int D> static hipError_t rows_variant(const PagedArgs& a, bool prefix, hipStream_t s) {
  if (a.shared_kv) return prefix ? rows_one<D, true, true>(a, s) : rows_one<D, true, false>(a, s);
  return prefix ? rows_one<D, false, true>(a, s) : rows_one<D, false, false>(a, s);
}
hipError_t launch_paged_rows(const PagedArgs& a, bool prefix, hipStream_t s) {
  switch (a.D) {
    case 32: return rows_variant<32>(a, prefix, s);
    case 64: return rows_variant<64>(a, prefix, s);
    case 128: return rows_variant<128>(a, prefix, s);
  }
  return hipErrorInvalidValue;
}

hipError_t launch_paged_merge(const PagedArgs& a, hipStream_t s) {
  const long rows = (long)a.T * a.nH;
  int groups = 1;                                                 // 8 parts a thread
  while (groups < 8 && 8 * groups < a.prefix_parts + a.own_parts) groups *= 2;
  auto grid = [&](int slots) { return dim3((uint32_t)((rows + slots / groups - 1) / (slots / groups))); };
  switch (a.D) {
    case 32: hipLaunchKernelGGL(paged_merge_kernel<32>, grid(32), dim3(256), 0, s, a, groups); break;
    case 64: hipLaunchKernelGGL(paged_merge_kernel<64>, grid(16), dim3(256), 0, s, a, groups); break;
    case 128: hipLaunchKernelGGL(paged_merge_kernel<128>, grid(8), dim3(256), 0, s, a, groups); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace ta
