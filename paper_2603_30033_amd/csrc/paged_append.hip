// Appending latent rows to the paged cache, with the position rotation on the way.
//
// Token t of sequence b sits at position p = kv_len[b] - q_start[b+1] + t.  Its key latent is rotated to p (channel pairs by
// p * base^(-2j/r3), from the context's table) and stored, with its value latent, in row p % page_size of page
// page_table[b][p / page_size]; its per-head queries are rotated by the same angles.  Every element is read and written once: HBM
// bound for many tokens, and for few a chain of four dependent reads (batch bounds, length, table entry, rotation).
//
// A group of CH = r3/8 (bf16) lanes takes one token's rows by 16-byte chunks, a lane the same channels of every row: it reads its
// rotation once and applies it to up to kAppendHeads query rows, whose loads are all in flight before the token's sequence is looked
// for (8189 tokens of 32 heads of 128 channels: 37.1 us, looked for first 38.5; with 4, 16 heads a group 38.6, 45.0).  Rotated queries
// that no L2 can hold until they are read go past the caches, which leaves these to what the call still has to read: the same call
// 26 us (5.5 TB/s; a large copy has 4.9), together with the attention behind it 407 us for two prompts of 4096 tokens and 404
// without.  Queries in place are in the caches already.  One token of 12 heads of 64 channels: 5.0 us (a kernel that writes one element: 1.4).
#include "paged.h"

namespace ta {

constexpr int kAppendHeads = 8;         // query rows of a group
constexpr int kAppendStarts = 1024;     // batch bounds looked through at a time
constexpr long kL2Bytes = 32l << 20;    // of all eight dies

template <typename T> struct Row16 {    // 16 bytes of a row as fp32
  static constexpr int N = 16 / (int)sizeof(T);
  float x[N];
};
template <typename T, bool WIDE> __device__ __forceinline__ void load16(const T* p, Row16<T>& r) {
  if constexpr (WIDE) {
    const u32x4 raw = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 2) {
        r.x[2 * i] = __uint_as_float(raw[i] << 16);
        r.x[2 * i + 1] = __uint_as_float(raw[i] & 0xffff0000u);
      } else {
        r.x[i] = __uint_as_float(raw[i]);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < Row16<T>::N; ++i) r.x[i] = to_f32(p[i]);
  }
}
template <typename T, bool WIDE, bool PAST = false> __device__ __forceinline__ void store16(T* p, const Row16<T>& r) {
  if constexpr (WIDE) {
    u32x4 raw;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 2) {
        const f32x2 two = {r.x[2 * i], r.x[2 * i + 1]};
        raw[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(two, bf16x2));
      } else {
        raw[i] = __float_as_uint(r.x[i]);
      }
    }
    if constexpr (PAST) __builtin_nontemporal_store(raw, reinterpret_cast<u32x4*>(p));
    else *reinterpret_cast<u32x4*>(p) = raw;
  } else {
#pragma unroll
    for (int i = 0; i < Row16<T>::N; ++i) store1(p + i, r.x[i]);
  }
}
template <typename T> __device__ __forceinline__ void turn(Row16<T>& r, const f32x4 (&cs)[Row16<T>::N / 4]) {
#pragma unroll
  for (int i = 0; i < Row16<T>::N; i += 2) {
    const float c = cs[i / 4][i % 4], s = cs[i / 4][i % 4 + 1], x0 = r.x[i], x1 = r.x[i + 1];
    r.x[i] = x0 * c - x1 * s;
    r.x[i + 1] = x0 * s + x1 * c;
  }
}

// WIDE: every row starts on 16 bytes.  PAST: rotated queries go past the caches.  parts: groups that a token's rows are dealt to, the
// last of them its key and value row
template <typename T, bool WIDE, bool PAST>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedAppendArgs p, int lanes, int parts) {
  constexpr int N = Row16<T>::N;
  __shared__ int starts[kAppendStarts];
  const int slots = 256 / lanes, slot = threadIdx.x / lanes, ch = threadIdx.x % lanes;
  const long item = (long)blockIdx.x * slots + slot;
  const int t = (int)min(item / parts, (long)p.T), part = (int)(item % parts);
  const bool live = slot < slots && t < p.T;

  // the rows are on their way while the token's sequence is looked for
  const int c = ch * N, h0 = part * kAppendHeads;
  const bool queries = part < parts - 1;
  const long qrow = ((long)t * p.nH + h0) * p.q_row + c;
  Row16<T> r[kAppendHeads];
  if (live && queries && c < p.r3) {
#pragma unroll
    for (int i = 0; i < kAppendHeads; ++i)
      if (h0 + i < p.nH) load16<T, WIDE>(static_cast<const T*>(p.Qin) + qrow + (long)i * p.q_row, r[i]);
  } else if (live && !queries) {
    if (c < p.r3) load16<T, WIDE>(static_cast<const T*>(p.Kin) + t * p.ldk + c, r[0]);
    if (p.V != nullptr && c < p.rt3) load16<T, WIDE>(static_cast<const T*>(p.Vin) + t * p.ldv + c, r[1]);
  }

  // sequence of the token: as many of q_start[1 ..] as are not behind it
  int b = 0;
  for (int at = 1; at <= p.B; at += kAppendStarts) {
    const int n = min(kAppendStarts, p.B + 1 - at);
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += 256) starts[i] = p.q_start[at + i];
    __syncthreads();
    int lo = 0, hi = n;
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (starts[mid] <= t) lo = mid + 1;
      else hi = mid;
    }
    b += lo;
    if (!__syncthreads_or(lo == n)) break;
  }
  if (!live || b >= p.B) return;                                  // behind the last sequence
  const PagedSeq s = paged_seq(p, b);
  if (t < s.q0 || t >= s.q0 + s.nq) return;
  const int pos = s.len - s.nq + (t - s.q0);                      // negative: before the sequence's first row

  f32x4 cs[N / 4];
#pragma unroll
  for (int q = 0; q < N / 4; ++q) cs[q] = f32x4{1.f, 0.f, 1.f, 0.f};
  if (p.rope != nullptr && c < p.r3) {
    const f32x4* tab = reinterpret_cast<const f32x4*>(p.rope) + (long)(c / 4) * p.rope_ld + min(max(pos, 0), p.rope_ld - 1);
#pragma unroll
    for (int q = 0; q < N / 4; ++q) cs[q] = tab[(long)q * p.rope_ld];
  }
  if (queries) {
    if (c >= p.r3) return;
    T* dst = static_cast<T*>(p.Qout) + qrow;
#pragma unroll
    for (int i = 0; i < kAppendHeads; ++i)
      if (h0 + i < p.nH) {
        if (p.rope != nullptr) turn<T>(r[i], cs);
        store16<T, WIDE, PAST>(dst + (long)i * p.q_row, r[i]);
      }
    return;
  }
  if (pos < 0) return;
  const int i = divide(pos, p.ps);
  if (i >= p.max_pages) return;
  const int page = p.table[(long)b * p.max_pages + i];
  if ((uint32_t)page >= (uint32_t)p.n_pages) return;              // no page: nothing is stored
  const int at = pos - i * p.page_size;
  if (c < p.r3) {
    if (p.rope != nullptr && p.rotate_k) turn<T>(r[0], cs);
    store16<T, true>(static_cast<T*>(p.K) + page * p.k_stride + (long)at * p.r3 + c, r[0]);
  }
  if (p.V != nullptr && c < p.rt3) store16<T, true>(static_cast<T*>(p.V) + page * p.v_stride + (long)at * p.rt3 + c, r[1]);
}

// lanes of a group (a power of two), groups of a token, workgroups
struct AppendGrid {
  int lanes = 1, parts;
  long blocks;
};
static AppendGrid append_grid(int es, const PagedAppendArgs& a) {
  AppendGrid g;
  const int widest = a.V != nullptr && a.rt3 > a.r3 ? a.rt3 : a.r3;
  while (g.lanes * 16 < widest * es) g.lanes *= 2;
  g.parts = 1 + (a.Qin != nullptr ? (a.nH + kAppendHeads - 1) / kAppendHeads : 0);
  const long slots = 256 / g.lanes;
  g.blocks = ((long)a.T * g.parts + slots - 1) / slots;
  return g;
}
bool paged_append_fits(int dtype, const PagedAppendArgs& a) { return append_grid(dtype == 0 ? 4 : 2, a).blocks <= kMaxGroups; }

template <typename T> static hipError_t append_one(const PagedAppendArgs& a, hipStream_t s) {
  const bool past = a.Qout != a.Qin && (long)a.T * a.nH * a.q_row * (long)sizeof(T) > kL2Bytes;
  const AppendGrid g = append_grid(sizeof(T), a);
  auto wide = [&](const void* q, long ld) { return reinterpret_cast<uintptr_t>(q) % 16 == 0 && ld * (long)sizeof(T) % 16 == 0; };
  const bool all = wide(a.Kin, a.ldk) && wide(a.Vin, a.ldv) && wide(a.Qin, a.q_row) && wide(a.Qout, a.q_row);
  const auto kern = !all ? paged_append_kernel<T, false, false>
                    : past ? paged_append_kernel<T, true, true> : paged_append_kernel<T, true, false>;
  hipLaunchKernelGGL(kern, dim3((uint32_t)g.blocks), dim3(256), 0, s, a, g.lanes, g.parts);
  return hipGetLastError();
}
hipError_t launch_paged_append(int dtype, const PagedAppendArgs& a, hipStream_t s) {
  return dtype == 0 ? append_one<float>(a, s) : append_one<bf16>(a, s);
}

}  // namespace ta
