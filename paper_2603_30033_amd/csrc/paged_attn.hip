// Attention over the paged latent cache.
//
// One latent key and value row serves all heads, so the rows of the product are the (token, head) pairs of a sequence, token by
// token: row r is head r % nH of new token r / nH.  Online softmax over the keys; a row sees the keys up to its token's own.
//
//   paged_rows   32 rows a workgroup, its four waves taking every fourth block of 32 keys straight from the pages
//   paged_merge  joins the partial results of a row: sum_i 2^(m_i - m) (l_i, O_i), m = max m_i
#include "paged.h"

namespace ta {

// 16 channels c0 .. of a row of r channels (whole 16-byte chunks), zeros behind them
template <typename T> __device__ __forceinline__ Frag<T> load_frag_upto(const T* row, int c0, int r) {
  constexpr int CE = 16 / (int)sizeof(T), NC = 16 / CE;
  Frag<T> f = zero_frag<T>();
#pragma unroll
  for (int i = 0; i < NC; ++i)
    if (c0 + i * CE < r) f.v[i] = *reinterpret_cast<const decltype(f.v[0] + f.v[0])*>(row + c0 + i * CE);
  return f;
}

// the fragment's 8 channel pairs turned by the table entries of their 4 quads
__device__ __forceinline__ void turn_frag(Frag<bf16>& f, const f32x4 (&cs)[4]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    u32x4 raw = __builtin_bit_cast(u32x4, f.v[i]);
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      const float c = cs[2 * i + d / 2][2 * (d % 2)], s = cs[2 * i + d / 2][2 * (d % 2) + 1];
      const float x0 = __uint_as_float(raw[d] << 16), x1 = __uint_as_float(raw[d] & 0xffff0000u);
      const f32x2 two = {x0 * c - x1 * s, x0 * s + x1 * c};
      raw[d] = __builtin_bit_cast(uint32_t, __builtin_convertvector(two, bf16x2));
    }
    f.v[i] = __builtin_bit_cast(bf16x8, raw);
  }
}
__device__ __forceinline__ void turn_frag(Frag<float>& f, const f32x4 (&cs)[4]) {
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int e = 0; e < 4; e += 2) {
      const float c = cs[q][e], s = cs[q][e + 1], x0 = f.v[q][e], x1 = f.v[q][e + 1];
      f.v[q][e] = x0 * c - x1 * s;
      f.v[q][e + 1] = x0 * s + x1 * c;
    }
}

// Values that are not finite, where some rows do not see their key: 0 * Inf would reach those rows.  Such values are taken out of
// the fragment, and out of 0/1 products over the rows that see the key comes which sums they belong to.
__device__ __forceinline__ bool frag_finite(const Frag<bf16>& f) {
  bool ok = true;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const u32x4 w = __builtin_bit_cast(u32x4, f.v[i]);
#pragma unroll
    for (int d = 0; d < 4; ++d) ok = ok && (w[d] & 0x7f80u) != 0x7f80u && (w[d] & 0x7f800000u) != 0x7f800000u;
  }
  return ok;
}
__device__ __forceinline__ bool frag_finite(const Frag<float>& f) {
  bool ok = true;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) ok = ok && (__float_as_uint(f.v[i][j]) & 0x7f800000u) != 0x7f800000u;
  return ok;
}
__device__ __forceinline__ float frag_at(const Frag<bf16>& f, int e) { return (float)f.v[e / 8][e % 8]; }
__device__ __forceinline__ float frag_at(const Frag<float>& f, int e) { return f.v[e / 4][e % 4]; }
__device__ __forceinline__ void frag_set(Frag<bf16>& f, int e, float x) { f.v[e / 8][e % 8] = (bf16)x; }
__device__ __forceinline__ void frag_set(Frag<float>& f, int e, float x) { f.v[e / 4][e % 4] = x; }
// seen: 1 where the row sees the key; o: the accumulator block of the fragment's 32 channels
template <typename T> __device__ __forceinline__ void take_nonfinite(Frag<T>& v, const Frag<T>& seen, f32x16& o) {
  Frag<T> one[3];                                                 // where the value is +Inf, -Inf, NaN
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const float x = frag_at(v, e);
    frag_set(one[0], e, x == INFINITY ? 1.f : 0.f);
    frag_set(one[1], e, x == -INFINITY ? 1.f : 0.f);
    frag_set(one[2], e, x != x ? 1.f : 0.f);
    if (!(x - x == 0.f)) frag_set(v, e, 0.f);
  }
  const float what[3] = {INFINITY, -INFINITY, NAN};
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    f32x16 n;
#pragma unroll
    for (int e = 0; e < 16; ++e) n[e] = 0.f;
    mma32(n, one[k], seen);
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (n[e] > 0.f) o[e] += what[k];
  }
}

// What the rounding of a probability to bf16 left over, as a second operand: without it that rounding (2^-8 at most) would weigh
// as much in the result as the result's own
template <typename T> __device__ __forceinline__ Frag<T> rest_of(const f32x16& pr, const Frag<T>& f) {
  f32x16 r;
#pragma unroll
  for (int e = 0; e < 16; ++e) r[e] = pr[e] - frag_at(f, e);
  return to_frag<T>(r);
}

// ---- partial results of the waves of a workgroup, joined through LDS -----------------------------------------------
template <int D, int W> struct WaveJoin {
  static constexpr int RE = D + 4;                                // padded row
  static constexpr size_t bytes(int rows) { return (size_t)W * rows * (RE + 2) * sizeof(float); }
};

// ------------------------------------------------------------------------------------------------------------------
// 32 rows a workgroup
// ------------------------------------------------------------------------------------------------------------------
// Grid: row blocks x parts of the keys.  Key fragments come from memory as they are (a lane reads 16 channels of its key row);
// value fragments one element a lane, 32 consecutive channels of a row in half a wave.
template <typename T, int D, bool SH, bool PREFIX>
__global__ __launch_bounds__(256) void paged_rows_kernel(PagedArgs p) {
  constexpr int CB = D / 32;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int h = lane / 32, lr = lane % 32;
  const int parts = PREFIX ? p.prefix_parts : max(p.own_parts, 1), part = blockIdx.y;

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
    const int b = paged_locate(p.B, blockIdx.x, [&](int i) { return (paged_seq(p, i).nq * p.nH + 31) / 32; },
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
  const int per = (blocks + parts - 1) / parts;
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
    const int page = paged_page(table, min(pi, pages - 1), p.n_pages), at = n - pi * p.page_size;
    const T* krow = static_cast<const T*>(p.K) + page * p.k_stride + (long)at * p.r3;
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
    Frag<T> seen;
    if (partly)
#pragma unroll
      for (int e = 0; e < 16; ++e) frag_set(seen, e, s[e] == -INFINITY ? 0.f : 1.f);
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = fast_exp2(s[e] - m_use);
    l_run = block_sum(s, l_run * alpha);
    const Frag<T> pf = to_frag<T>(s);
    Frag<T> ph;
    if constexpr (sizeof(T) == 2) ph = rest_of<T>(s, pf);
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
#pragma unroll
      for (int e = 0; e < 16; ++e) oacc[cb][e] *= alpha;
      Frag<T> vf;
      const int c = min(cb * 32 + lr, p.rt3 - 1);                 // channels behind the last repeat it and are not stored
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int key = 8 * (e / 4) + 4 * h + e % 4;
        const long pg = __shfl(page, key), off = __shfl(at, key);
        const T* src = SH ? static_cast<const T*>(p.K) + pg * p.k_stride + off * p.r3
                          : static_cast<const T*>(p.V) + pg * p.v_stride + off * p.rt3;
        frag_set(vf, e, to_f32(src[c]));
      }
      if (partly && __builtin_amdgcn_ballot_w64(!frag_finite(vf)) != 0ull) take_nonfinite<T>(vf, seen, oacc[cb]);
      mma32(oacc[cb], vf, pf);
      if constexpr (sizeof(T) == 2) mma32(oacc[cb], vf, ph);
    }
  }

  // ---- the waves' sums joined; one row of D channels by D/4 threads ----
  constexpr int RE = WaveJoin<D, 4>::RE;
  float* mo = reinterpret_cast<float*>(smem_raw);                 // [4][32][RE], then references and sums [4][32]
  float* mm = mo + 4 * 32 * RE;
  float* ml = mm + 4 * 32;
  __syncthreads();                                                // (the plan's words are done with)
  const float l_tot = halves_sum(l_run);
  if (h == 0) {
    mm[wave * 32 + lr] = m_run;
    ml[wave * 32 + lr] = l_tot;
  }
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      store4(mo + (wave * 32 + lr) * RE + cb * 32 + 8 * q + 4 * h, oacc[cb][4 * q], oacc[cb][4 * q + 1], oacc[cb][4 * q + 2],
             oacc[cb][4 * q + 3]);
  __syncthreads();
  const bool direct = !PREFIX && p.own_parts == 0;
  for (int i = threadIdx.x; i < 32 * (D / 4); i += 256) {
    const int row = i / (D / 4), c = i % (D / 4) * 4;
    if (rb * 32 + row >= n_rows) break;
    float m = -INFINITY, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) m = fmaxf(m, mm[w * 32 + row]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = mm[w * 32 + row] == -INFINITY ? 0.f : fast_exp2(mm[w * 32 + row] - m);
      l += f * ml[w * 32 + row];
      o += f * *reinterpret_cast<const f32x4*>(mo + (w * 32 + row) * RE + c);
    }
    const long at = (long)row0 + rb * 32 + row;
    if (direct) {
      const float inv = l == 0.f ? 0.f : 1.f / l;                 // no key: the row is zero
      paged_store4<T>(p, at, c, o * inv);
      if (c == 0 && p.lse != nullptr) p.lse[at] = l == 0.f ? -INFINITY : (m + __log2f(l)) * kLn2;
    } else {
      const long slot = (long)((PREFIX ? 0 : p.prefix_parts) + part) * p.T * p.nH + at;
      *reinterpret_cast<f32x4*>(p.part_o + slot * D + c) = o;
      if (c == 0) p.part_ml[slot] = float2{m, l};
    }
  }
}

// ------------------------------------------------------------------------------------------------------------------
// partial results of a row joined: one row by D/4 threads
// ------------------------------------------------------------------------------------------------------------------
template <typename T, int D>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedArgs p) {
  constexpr int L = D / 4;
  const long rows = (long)p.T * p.nH, row = (long)blockIdx.x * (256 / L) + threadIdx.x / L;
  const int c = threadIdx.x % L * 4;
  const int q0 = min(max(p.q_start[0], 0), p.T), q1 = min(max(p.q_start[p.B], 0), p.T);
  if (row < (long)q0 * p.nH || row >= (long)q1 * p.nH) return;    // behind the last sequence
  const int parts = p.prefix_parts + p.own_parts;
  float m = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int i = 0; i < parts; ++i) {
    const float2 ml = p.part_ml[i * rows + row];
    const f32x4 v = *reinterpret_cast<const f32x4*>(p.part_o + (i * rows + row) * D + c);
    if (ml.x == -INFINITY) continue;
    const float m_new = fmaxf(m, ml.x), a = fast_exp2(m - m_new), b = fast_exp2(ml.x - m_new);
    m = m_new;
    l = l * a + ml.y * b;
    o = o * a + v * b;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  paged_store4<T>(p, row, c, o * inv);
  if (c == 0 && p.lse != nullptr) p.lse[row] = l == 0.f ? -INFINITY : (m + __log2f(l)) * kLn2;
}

// ------------------------------------------------------------------------------------------------------------------
int paged_rows_blocks(const PagedArgs& a, int rows) {
  const long all = ((long)a.T * a.nH + rows - 1) / rows + (a.B < a.T ? a.B : a.T);
  return (int)(all < 0x7fffffffl ? all : 0x7fffffffl);
}

template <typename T, int D, bool SH, bool PREFIX> static hipError_t rows_one(const PagedArgs& a, hipStream_t s) {
  const size_t smem = WaveJoin<D, 4>::bytes(32);
  auto kern = paged_rows_kernel<T, D, SH, PREFIX>;
  static LdsOnce lds_once;                                       // one per kernel instantiation
  if (hipError_t e = allow_dynamic_lds(lds_once, kern, smem); e != hipSuccess) return e;
  const int blocks = PREFIX ? (int)(((long)a.T * a.nH + 31) / 32) : paged_rows_blocks(a, 32);
  hipLaunchKernelGGL(kern, dim3(blocks, PREFIX ? a.prefix_parts : a.own_parts > 0 ? a.own_parts : 1), dim3(256), smem, s, a);
  return hipGetLastError();
}
template <typename T, int D> static hipError_t rows_variant(const PagedArgs& a, bool prefix, hipStream_t s) {
  if (a.shared_kv) return prefix ? rows_one<T, D, true, true>(a, s) : rows_one<T, D, true, false>(a, s);
  return prefix ? rows_one<T, D, false, true>(a, s) : rows_one<T, D, false, false>(a, s);
}
template <typename T> static hipError_t rows_dispatch(const PagedArgs& a, bool prefix, hipStream_t s) {
  switch (a.D) {
    case 32: return rows_variant<T, 32>(a, prefix, s);
    case 64: return rows_variant<T, 64>(a, prefix, s);
    case 128: return rows_variant<T, 128>(a, prefix, s);
  }
  return hipErrorInvalidValue;
}
hipError_t launch_paged_rows(int dtype, const PagedArgs& a, bool prefix_pass, hipStream_t s) {
  return dtype == 0 ? rows_dispatch<float>(a, prefix_pass, s) : rows_dispatch<bf16>(a, prefix_pass, s);
}

template <typename T> static hipError_t merge_dispatch(const PagedArgs& a, hipStream_t s) {
  const long rows = (long)a.T * a.nH;
  auto grid = [&](int per) { return dim3((uint32_t)((rows + per - 1) / per)); };
  switch (a.D) {
    case 32: hipLaunchKernelGGL((paged_merge_kernel<T, 32>), grid(32), dim3(256), 0, s, a); break;
    case 64: hipLaunchKernelGGL((paged_merge_kernel<T, 64>), grid(16), dim3(256), 0, s, a); break;
    case 128: hipLaunchKernelGGL((paged_merge_kernel<T, 128>), grid(8), dim3(256), 0, s, a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}
hipError_t launch_paged_merge(int dtype, const PagedArgs& a, hipStream_t s) {
  return dtype == 0 ? merge_dispatch<float>(a, s) : merge_dispatch<bf16>(a, s);
}

}  // namespace ta
