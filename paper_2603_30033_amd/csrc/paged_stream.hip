// Attention over the paged latent cache for few rows a sequence (bf16, up to 32 (token, head) rows, 64 where the latents are at most 64
// wide: decode, proposed tokens).
//
// The cached rows are read once, in order, and every one serves all heads: 2 nH flops a byte, so HBM bounds it.  What counts is
// that all compute units stream all the time:
//   - The key rows of a sequence are cut into units of 128 and dealt to workgroups, the same number to each whatever the
//     sequence: as many as give every compute unit one workgroup.  (A workgroup finds its part by a scan over the lengths, which
//     live on the device.)  Where several share a sequence each leaves (max, sum, output) of its rows, which paged_join adds up.
//     More sequences than half the workgroups would leave parts of very different lengths: those go through paged_tile.
//   - Wave w takes keys 32w .. 32w+31 of a unit and does all the work for them (scores of every row, its own running softmax,
//     product with the values): nothing is shared between the waves while they stream, so there is no barrier in the loop.
//   - Rows go from the pages straight into the wave's two LDS stages, two units ahead.
#include "paged_block.h"

namespace ta {

constexpr int kUnit = kStreamUnit;      // keys of a unit

// KIND 0: key and value pools; 1: one pool, keys rotated when they are used; 2: one pool, nothing rotated
template <int D, int KIND> struct StreamLds {
  static constexpr int kTile = 32 * D;                            // elements of 32 rows
  static constexpr int kStage = kTile * (KIND == 0 ? 2 : 1) + (KIND == 1 ? 512 : 0);   // KIND 1: 1 KB of rotation entries
  static constexpr size_t kStages = 4ul * 2 * kStage * sizeof(bf16);
  static constexpr size_t kRows = KIND == 1 ? (size_t)(D / 4) * 16 * 16 : 0;           // rotation by 0 .. 15, behind the stages
  static constexpr size_t kAll = kStages + kRows;
  template <int HB> static constexpr size_t bytes() { return kAll > join_bytes<D, HB>() ? kAll : join_bytes<D, HB>(); }
};

// units of sequence b (no new token: none; no key of its own: one, which leaves its rows' empty result)
__device__ __forceinline__ int stream_units(const PagedArgs& p, int b) {
  const PagedSeq s = paged_seq(p, b);
  return (int)(s.nq != 0) * max(1, (s.len + kUnit - 1) / kUnit);  // (no branch: the loads go together)
}
// sum of every thread's number; all 256 threads call, sh holds 4 words
__device__ __forceinline__ int block_total(int x, int* sh) {
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) x += __shfl_xor(x, d);
  __syncthreads();
  if (threadIdx.x % kWave == 0) sh[threadIdx.x / kWave] = x;
  __syncthreads();
  return sh[0] + sh[1] + sh[2] + sh[3];
}
template <int D, int HB, int KIND>
// Wide latents with two pools: LDS leaves one wave to a SIMD, which may then use all registers.  With one pool whose keys are rotated on
// use the vector unit is busier than memory: two workgroups share a compute unit, and a stage is filled again at a round's end.
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(stream_late(D, KIND) ? 2 : 1, HB == 1 && (D < 128 || KIND == 1) ? 2 : 1)))
void paged_stream_kernel(PagedArgs p) {
  using T = bf16;
  using L = StreamLds<D, KIND>;
  constexpr int CB = D / 32, CPR = D / 8, RPP = 64 / CPR;         // 16-byte chunks of a row, rows of a 1 KB piece
  constexpr int PIECES = L::kTile / 512;
  constexpr bool ROT = KIND == 1, kLate = stream_late(D, KIND);
  extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int h = lane / 32, lr = lane % 32;

  int b, off = 0, cnt;                                            // sequence, first unit in it, units
  if (p.stream_wgs == 0) {                                        // a workgroup for every sequence
    b = blockIdx.x;
    cnt = stream_units(p, b);
  } else {
    int* sh = reinterpret_cast<int*>(smem_raw);
    // Units of a workgroup: one round of workgroups over the compute units, the units' share of each, or, where the sequences' last
    // parts make too many of these, a share that is larger by as much.  (At most 256 sequences, thread i's is i, and no more than half
    // the workgroups.)
    const int mine = (int)threadIdx.x < p.B ? stream_units(p, threadIdx.x) : 0, n_all = block_total(mine, sh);
    int units = max(kStreamLeast, (n_all + p.stream_wgs - 1) / p.stream_wgs), part, all;
    auto me = [](int) { return (int)blockIdx.x; };
    auto parts = [&](int) { return (mine + units - 1) / units; };
    __syncthreads();
    b = paged_locate(p.B, me, parts, sh, part, all);
    if (all > p.stream_wgs) {
      units = max(units, (n_all + p.stream_wgs - p.B - 1) / (p.stream_wgs - p.B));
      b = paged_locate(p.B, me, parts, sh, part, all);
    }
    if (b < 0) return;
    b = __builtin_amdgcn_readfirstlane(b);
    off = __builtin_amdgcn_readfirstlane(part) * units;
    const int n = stream_units(p, b);
    cnt = min(units, n - off);
    if (off == 0 && threadIdx.x == 0) p.stream_parts[b] = int2{(int)blockIdx.x, (n + units - 1) / units};   // for the join
  }
  if (cnt == 0) return;

  T* wbase = reinterpret_cast<T*>(smem_raw) + (long)wave * 2 * L::kStage;
  f32x4* rowtab = reinterpret_cast<f32x4*>(smem_raw + L::kStages);
  const PagedSeq s = paged_seq(p, b);
  const int all = stream_units(p, b);
  const int keys = s.len, n_rows = s.nq * p.nH, row0 = s.q0 * p.nH;
  const int unit0 = off * kUnit;                                // first key
  const int* table = p.table + (long)b * p.max_pages;
  const int lo = p.causal ? keys - s.nq + 1 : keys;             // keys that every row sees

  f32x16 oacc[HB][CB];
  float m_run[HB], l_run[HB];
  int limit[HB];                                                // keys that this lane's row sees
#pragma unroll
  for (int hb = 0; hb < HB; ++hb) {
    m_run[hb] = -INFINITY;
    l_run[hb] = 0.f;
    limit[hb] = p.causal ? lo + divide(min(hb * 32 + lr, n_rows - 1), p.heads) : keys;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int e = 0; e < 16; ++e) oacc[hb][cb][e] = 0.f;
  }

  if (unit0 < keys) {                                           // (the same for the whole workgroup)
    // 16 rows in one page (the usual sizes): their number comes by a scalar read, there is one start for the wave, and lanes add
    // their row and chunk to it.  Rows behind the sequence's last are whatever the page holds, chunks behind a row's end (which meet
    // zeros of the queries, or become channels that are not stored) repeat its last.  Else every lane looks up its own rows.
    constexpr int PPG = 16 / RPP;                                 // pieces of 16 rows
    const bool straight = p.page_size % 16 == 0;
    auto block_at = [&](int j) { return unit0 + min(j, cnt - 1) * kUnit + wave * 32; };   // past the end: the last again, unused
    const auto* entries = (const __attribute__((address_space(4))) int*)table;
    auto entry_at = [&](int j, int half) {
      return entries[min(divide(min(block_at(j) + 16 * half, keys - 1), p.ps), p.max_pages - 1)];
    };
    int entry[2] = {entry_at(0, 0), entry_at(0, 1)};              // of the block that is issued next
    auto issue = [&](int j, int st) {
      const int n0 = block_at(j);
      T* kt = wbase + (long)st * L::kStage;
      int l = lane;
      asm volatile("" : "+v"(l));                                 // (chunks of the pieces are formed afresh, not kept across the loop)
      if (straight) {
        const char *k = nullptr, *v = nullptr;
#pragma unroll
        for (int q = 0; q < PIECES; ++q) {
          if (q % PPG == 0) {                                     // the next 16 rows
            const int n = n0 + q * RPP;
            const long pg = paged_page(entry[q / PPG], p.n_pages), a = n - divide(n, p.ps) * p.page_size;
            k = static_cast<const char*>(p.K) + (pg * p.k_stride + a * p.r3) * 2;
            if constexpr (KIND == 0) v = static_cast<const char*>(p.V) + (pg * p.v_stride + a * p.rt3) * 2;
          }
          const uint32_t row = q % PPG * RPP + l / CPR, c = (l % CPR) ^ swz_x<CPR>(q * RPP + l / CPR);
          chunk_to_lds(k + row * (p.r3 * 2) + min(c * 16, p.r3 * 2u - 16), kt + q * 512);
          if constexpr (KIND == 0) chunk_to_lds(v + row * (p.rt3 * 2) + min(c * 16, p.rt3 * 2u - 16), kt + L::kTile + q * 512);
        }
        entry[0] = entry_at(j + 1, 0);
        entry[1] = entry_at(j + 1, 1);
      } else {
        int pages[PIECES];                                       // (all on their way before one is waited for)
#pragma unroll
        for (int q = 0; q < PIECES; ++q) pages[q] = table[min(divide(min(n0 + q * RPP + l / CPR, keys - 1), p.ps), p.max_pages - 1)];
#pragma unroll
        for (int q = 0; q < PIECES; ++q) {
          const int row = q * RPP + l / CPR, c = ((l % CPR) ^ swz_x<CPR>(row)) * 8;
          const int n = min(n0 + row, keys - 1);
          const long pg = paged_page(pages[q], p.n_pages), a = n - divide(n, p.ps) * p.page_size;
          const T* kp = static_cast<const T*>(p.K) + pg * p.k_stride + a * p.r3;
          chunk_to_lds(kp + min(c, p.r3 - 8), kt + q * 512);
          if constexpr (KIND == 0) {
            const T* vp = static_cast<const T*>(p.V) + pg * p.v_stride + a * p.rt3;
            chunk_to_lds(vp + min(c, p.rt3 - 8), kt + L::kTile + q * 512);
          }
        }
      }
      if constexpr (ROT) {                                        // rotation of the block's rows 0 and 16
        const int quad = l % (D / 4), n = n0 + 16 * (l / (D / 4) % 2);
        chunk_to_lds(reinterpret_cast<const f32x4*>(p.rope) + (long)quad * p.rope_ld + min(n, p.rope_ld - 1), kt + L::kTile);
      }
    };
    // vector-memory operations behind those of block j when round j begins (looking up rows one by one: those at least)
    constexpr int OPS = PIECES * (KIND == 0 ? 2 : 1) + (ROT ? 1 : 0);

    Frag<T> qf[HB][CB];
#pragma unroll
    for (int hb = 0; hb < HB; ++hb) {
      const T* q = static_cast<const T*>(p.Q) + (long)(row0 + min(hb * 32 + lr, n_rows - 1)) * p.q_row;
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) qf[hb][cb] = load_frag_upto<T>(q, cb * 32 + 16 * h, p.r3);
    }
    if constexpr (ROT) {
      for (int i = threadIdx.x; i < (D / 4) * 16; i += 256)
        rowtab[i] = reinterpret_cast<const f32x4*>(p.rope)[(long)(i / 16) * p.rope_ld + min(i % 16, p.rope_ld - 1)];
    }
    wait_vm<0>();                                               // plain loads out of the way of the counted ones
    wait_lds();
    if constexpr (ROT) __syncthreads();
    issue(0, 0);
    issue(1, 1);

    constexpr float kLazy = 8.f;
    const int xs = swz_x<CPR>(lr);
    auto round = [&](int j, int st) {
      const int n0 = block_at(j);
      const T* kt = wbase + (long)st * L::kStage;
      wait_vm<OPS>();
      f32x16 sc[HB];
#pragma unroll
      for (int hb = 0; hb < HB; ++hb)
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[hb][e] = 0.f;
      if constexpr (ROT) {
        // products with the keys' second parts have sums of their own: where a key is infinite, what its first part leaves over is
        // Inf - Inf, and that score is the first part's alone (a finite number added to it changes nothing)
        f32x16 sr[HB];
#pragma unroll
        for (int hb = 0; hb < HB; ++hb)
#pragma unroll
          for (int e = 0; e < 16; ++e) sr[hb][e] = 0.f;
        const f32x4* rl = reinterpret_cast<const f32x4*>(kt + L::kTile);
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
          const Frag<T> raw = load_frag_swz<T>(kt + lr * D, 4 * cb + 2 * h, xs);
          f32x16 x;                                             // the row's 16 channels, turned by (key 0 or 16 of the block) + (row)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const f32x4 t = rl[lr / 16 * (D / 4) + 8 * cb + 4 * h + q], a = rowtab[(8 * cb + 4 * h + q) * 16 + lr % 16];
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
              const float c = a[e] * t[e] - a[e + 1] * t[e + 1], sn = a[e + 1] * t[e] + a[e] * t[e + 1];
              const float x0 = frag_at(raw, 4 * q + e), x1 = frag_at(raw, 4 * q + e + 1);
              x[4 * q + e] = x0 * c - x1 * sn;
              x[4 * q + e + 1] = x0 * sn + x1 * c;
            }
          }
          const Frag<T> kf = to_frag<T>(x), rest = rest_of(x, kf);
#pragma unroll
          for (int hb = 0; hb < HB; ++hb) {
            mma32(sc[hb], kf, qf[hb][cb]);
            mma32(sr[hb], rest, qf[hb][cb]);
          }
        }
#pragma unroll
        for (int hb = 0; hb < HB; ++hb)
#pragma unroll
          for (int e = 0; e < 16; ++e) sc[hb][e] += __builtin_amdgcn_fmed3f(sr[hb][e], -3.4e38f, 3.4e38f);   // (of a NaN: a bound)
      } else {
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
          const Frag<T> kf = load_frag_swz<T>(kt + lr * D, 4 * cb + 2 * h, xs);
#pragma unroll
          for (int hb = 0; hb < HB; ++hb) mma32(sc[hb], kf, qf[hb][cb]);
        }
      }
      // the value fragments (transposing reads) are taken before the stage is filled again
      constexpr int TF = CB < 2 ? 1 : 2;
      Frag<T> vf[CB / TF][TF];
      const T* vt = kt + (KIND == 0 ? L::kTile : 0);
      if constexpr (!kLate) {
#pragma unroll
        for (int k = 0; k < CB / TF; ++k) load_frags_tr_swz<CPR, false>(vf[k], vt, 0, k * TF * 32, lane);
        wait_lds();
        issue(j + 2, st);
      }

      const bool partly = n0 + 32 > lo;
#pragma unroll
      for (int hb = 0; hb < HB; ++hb) {
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[hb][e] *= p.scale;
        if (partly)
#pragma unroll
          for (int e = 0; e < 16; ++e) sc[hb][e] = n0 + 8 * (e / 4) + 4 * h + e % 4 < limit[hb] ? sc[hb][e] : -INFINITY;
      }
      // online softmax with a lazily raised reference: O and l are rescaled only when a block's maximum exceeds the
      // reference by more than kLazy (probabilities stay below 2^kLazy)
      Frag<T> pf[HB], ph[HB];
#pragma unroll
      for (int hb = 0; hb < HB; ++hb) {
        float mx = -INFINITY;
#pragma unroll
        for (int e = 0; e < 16; ++e) mx = fmaxf(mx, sc[hb][e]);
        mx = halves_max(mx);
        const bool raise = mx > m_run[hb] + kLazy;              // -inf + kLazy = -inf: the first block with a key raises
        if (__builtin_amdgcn_ballot_w64(raise) != 0ull) {
          const float alpha = raise ? fast_exp2(m_run[hb] - mx) : 1.f;
          if (raise) m_run[hb] = mx;
          l_run[hb] *= alpha;
#pragma unroll
          for (int cb = 0; cb < CB; ++cb)
#pragma unroll
            for (int e = 0; e < 16; ++e) oacc[hb][cb][e] *= alpha;
        }
        const float m_use = m_run[hb] == -INFINITY ? 0.f : m_run[hb];
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[hb][e] = fast_exp2(sc[hb][e] - m_use);
        l_run[hb] = block_sum(sc[hb], l_run[hb]);
        pf[hb] = to_frag<T>(sc[hb]);
        ph[hb] = rest_of(sc[hb], pf[hb]);
      }
      if constexpr (kLate) {
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
          Frag<T> v[1];
          load_frags_tr_swz<CPR>(v, vt, 0, cb * 32, lane);
          if (__builtin_amdgcn_ballot_w64(!frag_finite(v[0])) != 0ull) take_nonfinite<T>(v[0], limit[0] - n0 - 4 * h, oacc[0][cb]);
          mma32(oacc[0][cb], v[0], pf[0]);
          mma32(oacc[0][cb], v[0], ph[0]);
        }
        wait_lds();
        issue(j + 2, st);
        return;
      }
      bool fine = true;
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) fine = fine && frag_finite(vf[cb / TF][cb % TF]);
      if (__builtin_amdgcn_ballot_w64(!fine) == 0ull) {
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
          for (int hb = 0; hb < HB; ++hb) {
            mma32(oacc[hb][cb], vf[cb / TF][cb % TF], pf[hb]);
            mma32(oacc[hb][cb], vf[cb / TF][cb % TF], ph[hb]);
          }
      } else {
#pragma unroll
        for (int hb = 0; hb < HB; ++hb) {
#pragma unroll
          for (int cb = 0; cb < CB; ++cb) {
            Frag<T> v = vf[cb / TF][cb % TF];
            take_nonfinite<T>(v, limit[hb] - n0 - 4 * h, oacc[hb][cb]);
            mma32(oacc[hb][cb], v, pf[hb]);
            mma32(oacc[hb][cb], v, ph[hb]);
          }
        }
      }
    };
    for (int j = 0; j < cnt; ++j) {
      round(j, j & 1);
    }
    wait_vm<0>();                                               // tiles requested past the end still land in LDS
  }
  __syncthreads();

  const bool complete = off == 0 && cnt == all;
  join_waves<D, HB>(reinterpret_cast<float*>(smem_raw), oacc, m_run, l_run, n_rows, [&](int row, int c, float m, float l, f32x4 o) {
    if (complete) paged_result<T>(p, (long)row0 + row, c, m, l, o);
    else paged_partial<D>(p.stream_o, p.stream_ml, (long)blockIdx.x * (HB * 32) + row, c, m, l, o);
  });
}

// ------------------------------------------------------------------------------------------------------------------
// The partial results of a sequence's rows, from the workgroups that the first of them has named.  Grid: sequences x groups of rows; a
// row by D/4 threads, as many rows a workgroup as leave every part of a row a group of threads of its own (up to 8 groups).
// ------------------------------------------------------------------------------------------------------------------
template <int D>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedArgs p, int groups) {
  using T = bf16;
  constexpr int L = D / 4, SLOTS = 256 / L;                       // threads of a row, rows or groups of a workgroup
  __shared__ float4 po[256];
  __shared__ float2 pml[SLOTS];
  const int b = blockIdx.x, tid = threadIdx.x;
  const PagedSeq s = paged_seq(p, b);
  const int2 parts = p.stream_parts[b];                           // (of a sequence without a new token: anything)
  const int n_rows = s.nq * p.nH, per = SLOTS / groups;
  if ((int)blockIdx.y * per >= n_rows || parts.y == 1) return;    // one workgroup did it all and has written the result
  const int slot = tid / L, c = tid % L * 4, group = slot / per, r = (int)blockIdx.y * per + slot % per;
  RowSum sum;
  if (r < n_rows)
    sum.add_parts(parts.y, group, groups, [&](int i, const float2*& ml, const float*& o) {
      const long at = (long)(parts.x + i) * (p.hb * 32) + r;
      ml = p.stream_ml + at;
      o = p.stream_o + at * D + c;
    });
  sum.add_groups(po, pml, slot, group, groups, per, L);
  if (group == 0 && r < n_rows) paged_result<T>(p, (long)s.q0 * p.nH + r, c, sum.m, sum.l, sum.o);
}

// ------------------------------------------------------------------------------------------------------------------
template <int D, int HB, int KIND> static hipError_t stream_one(const PagedArgs& a, hipStream_t s) {
  const size_t smem = StreamLds<D, KIND>::template bytes<HB>();
  auto kern = paged_stream_kernel<D, HB, KIND>;
  static LdsOnce lds_once;                                       // one per kernel instantiation
  if (hipError_t e = allow_dynamic_lds(lds_once, kern, smem); e != hipSuccess) return e;
  hipLaunchKernelGGL(kern, dim3(a.stream_wgs > 0 ? a.stream_wgs : a.B), dim3(256), smem, s, a);
  return hipGetLastError();
}
template <int D> static hipError_t stream_variant(const PagedArgs& a, hipStream_t s) {
  const int kind = !a.shared_kv ? 0 : a.rope != nullptr ? 1 : 2;
  if (a.hb == 1) return kind == 0 ? stream_one<D, 1, 0>(a, s) : kind == 1 ? stream_one<D, 1, 1>(a, s) : stream_one<D, 1, 2>(a, s);
  if constexpr (D < 128) return kind == 0 ? stream_one<D, 2, 0>(a, s) : kind == 1 ? stream_one<D, 2, 1>(a, s) : stream_one<D, 2, 2>(a, s);
  return hipErrorInvalidValue;                                    // (two blocks of 128 channels do not fit the registers)
}
hipError_t launch_paged_stream(const PagedArgs& a, hipStream_t s) {
  switch (a.D) {
    case 32: return stream_variant<32>(a, s);
    case 64: return stream_variant<64>(a, s);
    case 128: return stream_variant<128>(a, s);
  }
  return hipErrorInvalidValue;
}

template <int D> static hipError_t join_one(const PagedArgs& a, hipStream_t s) {
  constexpr int SLOTS = 256 / (D / 4);
  // one group of threads for every 8 parts that a sequence has on average
  const int parts = a.stream_wgs / a.B + 1;
  int groups = 1;
  while (groups < 8 && 8 * groups < parts) groups *= 2;
  const int per = SLOTS / groups, most = a.max_new * a.nH;
  hipLaunchKernelGGL(paged_join_kernel<D>, dim3(a.B, (most + per - 1) / per), dim3(256), 0, s, a, groups);
  return hipGetLastError();
}
hipError_t launch_paged_join(const PagedArgs& a, hipStream_t s) {
  switch (a.D) {
    case 32: return join_one<32>(a, s);
    case 64: return join_one<64>(a, s);
    case 128: return join_one<128>(a, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace ta
