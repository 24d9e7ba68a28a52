// Attention over the paged latent cache for many rows of one sequence (bf16: pieces of prompts, and the rows of a whole batch on a
// common prefix).
//
// A cached row serves all (token, head) rows, so with R of them a key costs 4 D R flops and 4 D bytes: from a few dozen rows on the
// matrix pipe bounds it.  A workgroup of four waves takes 128 rows, a wave 32 of them, and all keys (or a part of them) in tiles that
// its waves share in LDS.  Tiles go from the pages straight into one of two LDS stages, a tile ahead.  Two workgroups share a
// compute unit: between two barriers a workgroup's waves do the same at the same time (reads, products, exponentials), and another
// workgroup that is not in step with it fills the gaps (eight waves in step, on tiles of the same size: 135 against 96 us for four
// sequences with up to 512 new tokens on up to 4097 rows).  Probabilities are rounded to bf16 once for the value product, as the
// result is: the relative error of the sum is that of one more rounding of the result.
#include "paged_block.h"

#include <type_traits>

namespace ta {

// KIND 0: key and value pools; 1: one pool, keys rotated on their way into LDS, kept as two bf16 parts; 2: one pool, nothing rotated
template <int D, int KIND> struct TileLds {
  static constexpr int kKeys = KIND == 1 ? 32 : 64;               // of a tile
  static constexpr int kTile = kKeys * D;                         // elements
  static constexpr int kStage = kTile * (KIND == 0 ? 2 : KIND == 1 ? 3 : 1);
  static constexpr size_t kEntries = KIND == 1 ? 0 : 4ul * 4 * 64 * sizeof(int);      // table entries of four tiles a wave
  static constexpr size_t kTiles = 2ul * kStage * sizeof(bf16);
  static constexpr size_t kBytes = kTiles + kEntries;
};

template <int D, int KIND, bool PREFIX>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void paged_tile_kernel(PagedArgs p) {
  using T = bf16;
  using L = TileLds<D, KIND>;
  constexpr int CB = D / 32, CPR = D / 8, RPP = 64 / CPR;         // 16-byte chunks of a row, rows of a 1 KB piece
  constexpr int BC = L::kKeys, NB = BC / 32, RB = kTileRows;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
  T* smem = reinterpret_cast<T*>(smem_raw);
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
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
    if (rb * RB >= n_rows) return;
  } else {
    int total;
    const int b = paged_locate(p.B, blockIdx.x, [&](int i) { return (paged_seq(p, i).nq * p.nH + RB - 1) / RB; },
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
  const int r0 = rb * RB, rw = r0 + wave * 32;                 // first row of the workgroup, of this wave
  const int r = min(rw + lr, n_rows - 1);                         // rows behind the last repeat it and are not stored
  auto sees = [&](int row) { return causal ? len - nq + divide(min(row, n_rows - 1), p.heads) + 1 : len; };
  const int limit = sees(r), lo_all = sees(r0), hi_all = sees(r0 + RB - 1);     // keys that the row sees, that all and any rows of the workgroup see
  const int hi = sees(rw + 31);                                   // keys that any row of the wave sees
  const int tiles = hi_all > first ? (hi_all - first + BC - 1) / BC : 0;
  const int per = (tiles + parts - 1) / parts;
  const int k0 = part * per, cnt = max(min(tiles, k0 + per) - k0, 0);
  const int key0 = first + k0 * BC;

  f32x16 oacc[CB];
  float m_run = -INFINITY, l_run = 0.f;
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int e = 0; e < 16; ++e) oacc[cb][e] = 0.f;

  if (cnt > 0) {                                                  // (the same for the whole workgroup)
    auto tile_at = [&](int j) { return key0 + min(j, cnt - 1) * BC; };   // past the end: the last again, unused

    Frag<T> qf[CB];
    {
      const T* q = static_cast<const T*>(p.Q) + (long)(row0 + r) * p.q_row;
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) qf[cb] = load_frag_upto<T>(q, cb * 32 + 16 * h, p.r3);
    }

    constexpr float kLazy = 8.f;
    const int xs = swz_x<CPR>(lr);
    // the 32 keys from key n0 on, rows kr .. of stage st; between(): work that is done while the first products run; careful: some
    // rows may not see some of the keys
    auto block = [&](auto careful, int n0, int kr, int st, auto between) {
      constexpr bool CAREFUL = decltype(careful)::value;
      const T* kt = smem + (long)st * L::kStage + kr * D;
      const T* vt = kt + (KIND == 0 ? L::kTile : KIND == 1 ? 2 * L::kTile : 0);
      f32x16 s;
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = 0.f;
      constexpr int G = KIND == 1 && CB > 2 ? 2 : CB;             // channel blocks whose reads are all on their way before a product
#pragma unroll
      for (int g = 0; g < CB; g += G) {
        Frag<T> kf[G], rest[KIND == 1 ? G : 1];
#pragma unroll
        for (int i = 0; i < G; ++i) {
          kf[i] = load_frag_swz<T>(kt + lr * D, 4 * (g + i) + 2 * h, xs);
          if constexpr (KIND == 1) rest[i] = load_frag_swz<T>(kt + L::kTile + lr * D, 4 * (g + i) + 2 * h, xs);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < G; ++i) {
          mma32(s, kf[i], qf[g + i]);
          if constexpr (KIND == 1) mma32(s, rest[i], qf[g + i]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      between();
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (CAREFUL) {
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = n0 + 8 * (e / 4) + 4 * h + e % 4 < limit ? s[e] : -INFINITY;
      }
      // online softmax with a lazily raised reference: O and l are rescaled only when a block's maximum exceeds the reference by
      // more than kLazy (probabilities stay below 2^kLazy)
      float mx = -INFINITY;
#pragma unroll
      for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[e]);
      mx = halves_max(mx) * p.scale;
      const bool raise = mx > m_run + kLazy;                      // -inf + kLazy = -inf: the first block with a key raises
      if (__builtin_amdgcn_ballot_w64(raise) != 0ull) {
        const float alpha = raise ? fast_exp2(m_run - mx) : 1.f;
        if (raise) m_run = mx;
        l_run *= alpha;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
          for (int e = 0; e < 16; ++e) oacc[cb][e] *= alpha;
      }
      const float m_use = m_run == -INFINITY ? 0.f : m_run;
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = fast_exp2(s[e] * p.scale - m_use);
      l_run = block_sum(s, l_run);
      const Frag<T> pf = to_frag<T>(s);
      constexpr int TF = CB < 2 ? 1 : 2;
#pragma unroll
      for (int k = 0; k < CB / TF; ++k) {
        Frag<T> vf[TF];
        load_frags_tr_swz<CPR>(vf, vt, 0, k * TF * 32, lane);
        if constexpr (CAREFUL) {
          bool fine = true;
#pragma unroll
          for (int f = 0; f < TF; ++f) fine = fine && frag_finite(vf[f]);
          if (__builtin_amdgcn_ballot_w64(!fine) != 0ull) {       // (rare)
#pragma unroll
            for (int f = 0; f < TF; ++f) take_nonfinite<T>(vf[f], frag_seen(limit - n0 - 4 * h, T()), oacc[k * TF + f]);
          }
        }
#pragma unroll
        for (int f = 0; f < TF; ++f) mma32(oacc[k * TF + f], vf[f], pf);
      }
    };
    // tile j from stage st: one that all rows of the workgroup see, and any other (a block that no row of the wave sees is passed over)
    auto whole = [&](int j, int st, auto between) {
      const int n0 = tile_at(j);
      block(std::false_type(), n0, 0, st, between);
#pragma unroll
      for (int nb = 1; nb < NB; ++nb) block(std::false_type(), n0 + nb * 32, nb * 32, st, [] {});
    };
    auto edge = [&](int j, int st, auto between) {
      const int n0 = tile_at(j);
      between();
#pragma unroll 1
      for (int nb = 0; nb < NB; ++nb)
        if (n0 + nb * 32 < hi) block(std::true_type(), n0 + nb * 32, nb * 32, st, [] {});
    };
    const int n_whole = min(max(lo_all - key0, 0) / BC, cnt);

    if constexpr (KIND != 1) {
      int* entries = reinterpret_cast<int*>(smem_raw + L::kTiles) + wave * 4 * 64;
      // table entries of tile j's rows, by way of LDS: an entry in a register would be waited for with every tile behind it.
      // Rows behind the last repeat it and are masked.
      auto fetch_entries = [&](int j) {
        const int n = min(tile_at(j) + lane, hi_all - 1);
        word_to_lds(table + min(divide(n, p.ps), pages - 1), entries + (j & 3) * 64);
      };
      // A wave's pieces of a tile: 1 KB each, NK of the keys and as many, of the same rows, of the values.  Where this lane's
      // chunks of them come from, in 16-byte units behind the pools' starts (a chunk behind the row's end: negative):
      constexpr int NK = BC * D / 512 / 4;
      const uint32_t k16 = (uint32_t)(p.k_stride / 8), v16 = (uint32_t)(p.v_stride / 8);
      long kfrom[NK], vfrom[KIND == 0 ? NK : 1];
      auto find = [&](int j) {
        const int* ids = entries + (j & 3) * 64;
        int l = lane;
        asm volatile("" : "+v"(l));                               // (rows and chunks of the pieces are formed afresh, not kept across the loop)
#pragma unroll
        for (int i = 0; i < NK; ++i) {
          const int row = (wave + 4 * i) * RPP + l / CPR, c = (l % CPR) ^ swz_x<CPR>(row);
          const int n = min(tile_at(j) + row, hi_all - 1);
          const uint32_t page = paged_page(ids[row], p.n_pages), at = n - divide(n, p.ps) * p.page_size;
          kfrom[i] = (long)((unsigned long)page * k16 + (at * (uint32_t)(p.r3 / 8) + c));
          if (c * 8 >= p.r3) kfrom[i] = -1;
          if constexpr (KIND == 0) {
            vfrom[i] = (long)((unsigned long)page * v16 + (at * (uint32_t)(p.rt3 / 8) + c));
            if (c * 8 >= p.rt3) vfrom[i] = -1;
          }
        }
      };
      auto issue = [&](int st) {
        T* kt = smem + (long)st * L::kStage;
        auto source = [&](const void* pool, long at) {
          const u32x4* from = static_cast<const u32x4*>(pool) + at;
          return p.r3 == D && p.rt3 == D ? from : at < 0 ? paged_zeros : from;
        };
#pragma unroll
        for (int i = 0; i < NK; ++i) {
          chunk_to_lds(source(p.K, kfrom[i]), kt + (wave + 4 * i) * 512);
          if constexpr (KIND == 0) chunk_to_lds(source(p.V, vfrom[i]), kt + L::kTile + (wave + 4 * i) * 512);
        }
      };
      fetch_entries(0);
      fetch_entries(1);
      fetch_entries(2);
      wait_vm<0>();                                               // entries, and plain loads out of the way of the counted ones
      find(0);
      issue(0);
      fetch_entries(3);
      find(1);
      auto next = [&](int j) {
        wait_vm<1>();                                             // this wave's part of tile j is there (entries may be on their way),
        wait_lds();                                               // its reads of tile j - 1 are done
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        issue((j + 1) & 1);                                       // the stage of tile j - 1
        fetch_entries(j + 4);
      };
      int j = 0;
      for (; j < n_whole; ++j) {
        next(j);
        whole(j, j & 1, [&] { find(j + 2); });
      }
      for (; j < cnt; ++j) {
        next(j);
        edge(j, j & 1, [&] { find(j + 2); });
      }
      wait_vm<0>();                                               // tiles requested past the end still land in LDS
    } else {
      // a thread's chunks of a tile are those of one row, eight apart: neighbouring lanes read neighbouring positions of the
      // rotation table
      constexpr int CPT = CPR / 8 > 0 ? CPR / 8 : 1;
      const int row = threadIdx.x % 32, ch0 = threadIdx.x / 32;
      struct Set { u32x4 x[CPT]; f32x4 cs[CPT][2]; } reg;
      auto load = [&](int j) {
        const int n = min(tile_at(j) + row, hi_all - 1);
        const int pi = divide(n, p.ps);
        const long pg = paged_page(table[min(pi, pages - 1)], p.n_pages), a = n - pi * p.page_size;
        const T* src = static_cast<const T*>(p.K) + pg * p.k_stride + a * p.r3;
#pragma unroll
        for (int i = 0; i < CPT; ++i) {
          const int ch = min(ch0 + 8 * i, CPR - 1);
          reg.x[i] = ch * 8 < p.r3 ? *reinterpret_cast<const u32x4*>(src + ch * 8) : u32x4{0u, 0u, 0u, 0u};
          const f32x4* tab = reinterpret_cast<const f32x4*>(p.rope) + (long)(2 * ch) * p.rope_ld + min(n, p.rope_ld - 1);
          reg.cs[i][0] = tab[0];
          reg.cs[i][1] = tab[p.rope_ld];
        }
      };
      auto store = [&](int st) {
        T* kt = smem + (long)st * L::kStage;
#pragma unroll
        for (int i = 0; i < CPT; ++i) {
          const int ch = ch0 + 8 * i;
          if (ch >= CPR) break;
          u32x4 hi16, lo16;
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            const float c = reg.cs[i][d / 2][2 * (d % 2)], sn = reg.cs[i][d / 2][2 * (d % 2) + 1];
            const float x0 = __uint_as_float(reg.x[i][d] << 16), x1 = __uint_as_float(reg.x[i][d] & 0xffff0000u);
            const f32x2 y = {x0 * c - x1 * sn, x0 * sn + x1 * c};
            hi16[d] = __builtin_bit_cast(uint32_t, __builtin_convertvector(y, bf16x2));
            const f32x2 z = {y[0] - __uint_as_float(hi16[d] << 16), y[1] - __uint_as_float(hi16[d] & 0xffff0000u)};
            lo16[d] = __builtin_bit_cast(uint32_t, __builtin_convertvector(z, bf16x2));
          }
          const int at = row * D + ((ch ^ swz_x<CPR>(row)) * 8);
          *reinterpret_cast<u32x4*>(kt + at) = hi16;
          *reinterpret_cast<u32x4*>(kt + L::kTile + at) = lo16;
          *reinterpret_cast<u32x4*>(kt + 2 * L::kTile + at) = reg.x[i];
        }
      };
      load(0);
      __syncthreads();                                            // (the plan's words are done with)
      store(0);
      load(1);
      int j = 0;
      for (; j < n_whole; ++j) {
        __syncthreads();
        store((j + 1) & 1);                                       // the stage of tile j - 1
        load(j + 2);
        whole(j, j & 1, [] {});
      }
      for (; j < cnt; ++j) {                                      // (nothing is kept in registers for later: they are all in use)
        __syncthreads();
        load(j + 1);
        store((j + 1) & 1);
        edge(j, j & 1, [] {});
      }
    }
  }

  const float l = halves_sum(l_run);
  if (rw + lr >= n_rows) return;
  const long at = (long)row0 + rw + lr;
  const bool direct = !PREFIX && p.own_parts == 0;
  const long slot = (long)((PREFIX ? 0 : p.prefix_parts) + part) * p.T * p.nH + at;
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x4 o = {oacc[cb][4 * q], oacc[cb][4 * q + 1], oacc[cb][4 * q + 2], oacc[cb][4 * q + 3]};
      const int c = cb * 32 + 8 * q + 4 * h;
      if (direct) paged_result<T>(p, at, c, m_run, l, o);
      else paged_partial<D>(p.part_o, p.part_ml, slot, c, m_run, l, o);
    }
}

template <int D, int KIND, bool PREFIX> static hipError_t tile_one(const PagedArgs& a, hipStream_t s) {
  const size_t smem = TileLds<D, KIND>::kBytes;
  auto kern = paged_tile_kernel<D, KIND, PREFIX>;
  static LdsOnce lds_once;                                       // one per kernel instantiation
  if (hipError_t e = allow_dynamic_lds(lds_once, kern, smem); e != hipSuccess) return e;
  const int blocks = PREFIX ? (int)(((long)a.T * a.nH + kTileRows - 1) / kTileRows) : paged_rows_blocks(a, kTileRows);
  hipLaunchKernelGGL(kern, dim3(blocks, PREFIX ? a.prefix_parts : a.own_parts > 0 ? a.own_parts : 1), dim3(256), smem, s, a);
  return hipGetLastError();
}
template <int D> static hipError_t tile_variant(const PagedArgs& a, bool prefix, hipStream_t s) {
  const int kind = !a.shared_kv ? 0 : a.rope != nullptr ? 1 : 2;
  if (prefix) return kind == 0 ? tile_one<D, 0, true>(a, s) : kind == 1 ? tile_one<D, 1, true>(a, s) : tile_one<D, 2, true>(a, s);
  return kind == 0 ? tile_one<D, 0, false>(a, s) : kind == 1 ? tile_one<D, 1, false>(a, s) : tile_one<D, 2, false>(a, s);
}
hipError_t launch_paged_tile(const PagedArgs& a, bool prefix_pass, hipStream_t s) {
  switch (a.D) {
    case 32: return tile_variant<32>(a, prefix_pass, s);
    case 64: return tile_variant<64>(a, prefix_pass, s);
    case 128: return tile_variant<128>(a, prefix_pass, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace ta
