// Device functions of the attention kernels over pages: operand fragments of cached rows, values that are not finite, partial
// results of the waves of a workgroup.
#pragma once
#include "paged.h"

namespace ta {

// 16 channels c0 .. of a row of r channels (whole 16-byte chunks), zeros behind them
template <typename T> __device__ __forceinline__ Frag<T> load_frag_upto(const T* row, int c0, int r) {
  constexpr int CE = 16 / (int)sizeof(T), NC = 16 / CE;
  Frag<T> f;
#pragma unroll
  for (int i = 0; i < NC; ++i) {                                  // (no branches: the loads go together)
    const int c = c0 + i * CE;
    const u32x4 x = *reinterpret_cast<const u32x4*>(row + (c < r ? c : 0));
    f.v[i] = __builtin_bit_cast(__typeof__(f.v[0] + f.v[0]), c < r ? x : u32x4{0u, 0u, 0u, 0u});
  }
  return f;
}

// the fragment's 8 channel pairs turned by the table entries of their 4 quads
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

__device__ __forceinline__ float frag_at(const Frag<bf16>& f, int e) { return (float)f.v[e / 8][e % 8]; }
__device__ __forceinline__ void frag_set(Frag<float>& f, int e, float x) { f.v[e / 4][e % 4] = x; }

// Values that are not finite where some rows do not see their key: 0 * Inf in a product would reach those rows.  Such values are taken
// out of the operand, and one product of small numbers that stand for them with 0/1 (the row sees the key) says which sums they
// belong to.  The other sums get the bits of the plain product.  (Rare; integer arithmetic on the packed words, since as many
// comparisons as a fragment has elements would each hold a pair of scalar registers.)
template <typename T> struct Bits;                                // of a 32-bit word that holds one or two elements
template <> struct Bits<bf16> {
  static constexpr uint32_t kExp = 0x7f807f80u, kLow = 0x00800080u, kTop = 0x80008000u, kMant = 0x007f007fu, kUnit = 0x00010001u, kAll = 0xffffu;
  static constexpr int kSign = 15, kMantBits = 7;
  static constexpr uint32_t kPlus = 0x3f80u, kMinus = 0x3a80u, kNan = 0x4480u;        // 1, 2^-10, 2^10
};
template <> struct Bits<float> {
  static constexpr uint32_t kExp = 0x7f800000u, kLow = 0x00800000u, kTop = 0x80000000u, kMant = 0x007fffffu, kUnit = 1u, kAll = ~0u;
  static constexpr int kSign = 31, kMantBits = 23;
  static constexpr uint32_t kPlus = 0x3f800000u, kMinus = 0x3a800000u, kNan = 0x44800000u;
};
template <typename T> __device__ __forceinline__ bool frag_finite(const Frag<T>& f) {
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < (int)sizeof(Frag<T>) / 16; ++i) {
    const u32x4 w = __builtin_bit_cast(u32x4, f.v[i]);
#pragma unroll
    for (int d = 0; d < 4; ++d) any |= (w[d] & Bits<T>::kExp) + Bits<T>::kLow;
  }
  return (any & Bits<T>::kTop) == 0;
}
// element pair (element) d of part i of a fragment for the keys of a block that the row sees -- `live` of them, as this lane counts
// (minus 4h) -- : ones, else zeros
template <typename T> __device__ __forceinline__ uint32_t seen_word(int i, int d, int live) {
  if constexpr (sizeof(T) == 2) {                                 // elements 8i + 2d, + 1: keys 8 (e / 4) + e % 4 (+ 4h)
    const int key = 16 * i + 8 * (d / 2) + 2 * (d % 2);
    return ((uint32_t)((key - live) >> 31) & 0x3f80u) | ((uint32_t)((key + 1 - live) >> 31) & 0x3f800000u);
  } else {
    return (uint32_t)((8 * i + d - live) >> 31) & 0x3f800000u;
  }
}
__device__ __forceinline__ void mma_part(f32x16& n, const bf16x8& a, const bf16x8& b) { n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, n, 0, 0, 0); }
__device__ __forceinline__ void mma_part(f32x16& n, const f32x4& a, const f32x4& b) {
#pragma unroll
  for (int j = 0; j < 4; ++j) n = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], n, 0, 0, 0);
}
// v without its elements that are not finite, which go to the sums o of its 32 channels and of the rows that see their key
template <typename T> __device__ __forceinline__ void take_nonfinite(Frag<T>& v, int live, f32x16& o) {
  using B = Bits<T>;
  using Part = __typeof__(v.v[0] + v.v[0]);
  f32x16 n;
#pragma unroll
  for (int e = 0; e < 16; ++e) n[e] = 0.f;
#pragma unroll
  for (int i = 0; i < (int)sizeof(Frag<T>) / 16; ++i) {
    __builtin_amdgcn_sched_barrier(0);                            // (one part at a time: few registers)
    u32x4 w = __builtin_bit_cast(u32x4, v.v[i]), x, y;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      const uint32_t bad = (((w[d] & B::kExp) + B::kLow) >> B::kSign) & B::kUnit;
      const uint32_t nan = (((w[d] & B::kMant) + B::kMant) >> B::kMantBits) & bad, minus = (w[d] >> B::kSign) & bad & ~nan;
      x[d] = nan * B::kNan + minus * B::kMinus + (bad & ~nan & ~minus) * B::kPlus;
      w[d] &= ~(bad * B::kAll);
      y[d] = seen_word<T>(i, d, live);
    }
    v.v[i] = __builtin_bit_cast(Part, w);
    mma_part(n, __builtin_bit_cast(Part, x), __builtin_bit_cast(Part, y));   // up to 32 of each kind: exact
  }
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    if (e % 4 == 0) __builtin_amdgcn_sched_barrier(0);
    o[e] += n[e] >= 1.f ? INFINITY : 0.f;
    o[e] += __builtin_amdgcn_fractf(n[e]) > 0.f ? -INFINITY : 0.f;
    o[e] += n[e] >= 1024.f ? NAN : 0.f;
  }
  __builtin_amdgcn_sched_barrier(0);
}

// What the rounding of a probability to bf16 left over, as a second operand: without it that rounding (2^-8 at most) would weigh
// as much in the result as the result's own
__device__ __forceinline__ Frag<bf16> rest_of(const f32x16& pr, const Frag<bf16>& f) {
  f32x16 r;
#pragma unroll
  for (int e = 0; e < 16; ++e) r[e] = pr[e] - frag_at(f, e);
  return to_frag<bf16>(r);
}

// lane l's 16 bytes at `from` to chunk l of `to` (the same for the whole wave)
__device__ __forceinline__ void chunk_to_lds(const void* from, void* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}

// Join of the partial results of a workgroup's four waves: reference m = max of theirs, sums and outputs scaled by 2^(m_w - m).
// A wave's lane (row = lane % 32 of block hb, half h) holds channels 32 cb + 8q + 4h + r in o[hb][cb][4q + r]; emit(row, c, m, l,
// four channels) for every row below `rows`.  The LDS at `lds` must be free and is free again behind the next barrier.
template <int D, int HB> constexpr size_t join_bytes() { return 4ul * HB * 32 * (D + 4 + 2) * sizeof(float); }
template <int D, int HB, class Emit>
__device__ __forceinline__ void join_waves(float* lds, const f32x16 (*o)[D / 32], const float* m_run, const float* l_run, int rows, Emit emit) {
  constexpr int RE = D + 4, R = HB * 32;                          // padded row; rows
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, h = lane / 32, lr = lane % 32;
  float* mm = lds + 4 * R * RE;                                   // references and sums [4][R]
  float* ml = mm + 4 * R;
#pragma unroll
  for (int hb = 0; hb < HB; ++hb) {
    const float l = halves_sum(l_run[hb]);
    if (h == 0) {
      mm[wave * R + hb * 32 + lr] = m_run[hb];
      ml[wave * R + hb * 32 + lr] = l;
    }
#pragma unroll
    for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        store4(lds + (wave * R + hb * 32 + lr) * RE + cb * 32 + 8 * q + 4 * h, o[hb][cb][4 * q], o[hb][cb][4 * q + 1],
               o[hb][cb][4 * q + 2], o[hb][cb][4 * q + 3]);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < R * (D / 4); i += 256) {
    const int row = i / (D / 4), c = i % (D / 4) * 4;
    if (row >= rows) break;
    float m = -INFINITY, l = 0.f;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) m = fmaxf(m, mm[w * R + row]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = mm[w * R + row] == -INFINITY ? 0.f : fast_exp2(mm[w * R + row] - m);
      l += f * ml[w * R + row];
      v += f * *reinterpret_cast<const f32x4*>(lds + (w * R + row) * RE + c);
    }
    emit(row, c, m, l, v);
  }
}

// four channels of a finished row (no key: zero, and a log-sum-exp of -infinity) ...
template <typename T> __device__ __forceinline__ void paged_result(const PagedArgs& p, long row, int c, float m, float l, f32x4 o) {
  paged_store4<T>(p, row, c, o * (l == 0.f ? 0.f : 1.f / l));
  if (c == 0 && p.lse != nullptr) p.lse[row] = l == 0.f ? -INFINITY : (m + __log2f(l)) * kLn2;
}
// ... and of a partial result
template <int D> __device__ __forceinline__ void paged_partial(float* po, float2* pml, long slot, int c, float m, float l, f32x4 o) {
  *reinterpret_cast<f32x4*>(po + slot * D + c) = o;
  if (c == 0) pml[slot] = float2{m, l};
}

// Partial results of one row, four channels a thread: (m, l, o) with sum and output relative to 2^m
struct RowSum {
  float m = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  __device__ __forceinline__ void add(float2 ml, f32x4 v, bool live = true) {
    // An empty part has a sum of 0, and its output may never have been written.  Its maximum says nothing: that of NaN scores alone is
    // -infinity too, and their sum and output are NaN.
    live = live && ml.y != 0.f;
    const float top = fmaxf(m, live ? ml.x : -INFINITY), ref = top == -INFINITY ? 0.f : top;
    const float a = fast_exp2(m - ref), f = live ? fast_exp2(ml.x - ref) : 0.f;
    m = top;
    l = l * a + (live ? ml.y * f : 0.f);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = o[e] * a + (live ? v[e] * f : 0.f);
  }
  // U of the parts base + group, + groups, ..; where(i, ml, o): where part i is.  The loads are in flight together.
  template <int U, class W> __device__ __forceinline__ void add_batch(int base, int parts, int group, int groups, W where) {
    float2 ml[U];
    f32x4 v[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const float2* pm;
      const float* po;
      where(min(base + group + k * groups, parts - 1), pm, po);
      ml[k] = *pm;
      v[k] = *reinterpret_cast<const f32x4*>(po);
    }
#pragma unroll
    for (int k = 0; k < U; ++k) add(ml[k], v[k], base + group + k * groups < parts);
  }
  // parts group, group + groups, ..
  template <class W> __device__ __forceinline__ void add_parts(int parts, int group, int groups, W where) {
    for (int base = 0; base < parts;) {
      const int left = parts - base;
      if (left > 4 * groups) {
        add_batch<8>(base, parts, group, groups, where);
        base += 8 * groups;
      } else if (left > 2 * groups) {
        add_batch<4>(base, parts, group, groups, where);
        base += 4 * groups;
      } else {
        add_batch<2>(base, parts, group, groups, where);
        base += 2 * groups;
      }
    }
  }
  // the sums of a row's other groups of threads, in their order, into group 0's.  po [256], pml [256 / L]; all threads call.
  __device__ __forceinline__ void add_groups(float4* po, float2* pml, int slot, int group, int groups, int per, int L) {
    if (groups == 1) return;
    const int tid = threadIdx.x;
    po[tid] = float4{o[0], o[1], o[2], o[3]};
    if (tid % L == 0) pml[slot] = float2{m, l};
    __syncthreads();
    if (group > 0) return;
    for (int k = 1; k < groups; ++k) {
      const float4 v = po[tid + k * per * L];
      add(pml[slot + k * per], f32x4{v.x, v.y, v.z, v.w});
    }
  }
};

}  // namespace ta
