// Attention over the paged latent cache for many rows of one sequence (bf16: pieces of prompts, and the rows of a whole batch on a
// common prefix).
//
// A cached row serves all (token, head) rows, so with R of them a key costs 4 D R flops and 4 D bytes: from a few dozen rows on the
// matrix pipe bounds it.  A workgroup of eight waves takes 32 WR rows, a wave 32 of them and every (8 / WR)-th block of keys of the
// 64-key tiles that all waves share in LDS.  Tiles go from the pages straight into one of three LDS stages, two tiles ahead, so
// that one barrier a tile suffices.  Probabilities are rounded to bf16 once for the value product, as the result is: the relative
// error of the sum is that of one more rounding of the result.
#include "paged_block.h"

namespace ta {

constexpr int kTileKeys = 64;

// KIND 0: key and value pools; 1: one pool, keys rotated on their way into LDS, kept as two bf16 parts; 2: one pool, nothing rotated
template <int D, int KIND> struct TileLds {
  static constexpr int kTile = kTileKeys * D;                     // elements
  static constexpr int kStages = KIND == 1 ? 2 : 3;
  static constexpr int kStage = kTile * (KIND == 0 ? 2 : KIND == 1 ? 3 : 1);
  static constexpr size_t kEntries = KIND == 1 ? 0 : 8ul * 4 * 64 * sizeof(int);      // table entries of four tiles a wave
  static constexpr size_t kTiles = (size_t)kStages * kStage * sizeof(bf16);
  // the waves of other keys hand their sums over here: [WR][16 CB + 2][64]
  static constexpr size_t kSums = 4ul * (D / 2 + 2) * 64 * sizeof(float);
  static constexpr size_t kBytes = kTiles + kEntries > kSums ? kTiles + kEntries : kSums;
};

template <int D, int WR, int KIND, bool PREFIX>
__global__ __launch_bounds__(512) void paged_tile_kernel(PagedArgs p) {
  using T = bf16;
  using L = TileLds<D, KIND>;
  constexpr int CB = D / 32, CPR = D / 8, RPP = 64 / CPR;         // 16-byte chunks of a row, rows of a 1 KB piece
  constexpr int WK = 8 / WR, KPW = kTileKeys / WK, NB = KPW / 32; // waves that share a row's keys, keys and blocks of a wave
  extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
  T* smem = reinterpret_cast<T*>(smem_raw);
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int h = lane / 32, lr = lane % 32, wr = wave % WR, wk = wave / WR;
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
    if (rb * 32 * WR >= n_rows) return;
  } else {
    int total;
    const int b = paged_locate<512>(p.B, blockIdx.x, [&](int i) { return (paged_seq(p, i).nq * p.nH + 32 * WR - 1) / (32 * WR); },
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
  const int r0 = rb * 32 * WR, rw = r0 + wr * 32;                 // first row of the workgroup, of this wave
  const int r = min(rw + lr, n_rows - 1);                         // rows behind the last repeat it and are not stored
  auto sees = [&](int row) { return causal ? len - nq + divide(min(row, n_rows - 1), p.heads) + 1 : len; };
  const int limit = sees(r), hi_all = sees(r0 + 32 * WR - 1);     // keys that the row sees, that any row of the workgroup sees
  const int lo = sees(rw), hi = sees(rw + 31);                    // keys that all rows, any row of the wave see
  const int tiles = hi_all > first ? (hi_all - first + kTileKeys - 1) / kTileKeys : 0;
  const int per = (tiles + parts - 1) / parts;
  const int k0 = part * per, cnt = max(min(tiles, k0 + per) - k0, 0);
  const int key0 = first + k0 * kTileKeys;

  f32x16 oacc[CB];
  float m_run = -INFINITY, l_run = 0.f;
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int e = 0; e < 16; ++e) oacc[cb][e] = 0.f;

  if (cnt > 0) {                                                  // (the same for the whole workgroup)
    auto tile_at = [&](int j) { return key0 + min(j, cnt - 1) * kTileKeys; };   // past the end: the last again, unused

    Frag<T> qf[CB];
    {
      const T* q = static_cast<const T*>(p.Q) + (long)(row0 + r) * p.q_row;
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) qf[cb] = load_frag_upto<T>(q, cb * 32 + 16 * h, p.r3);
    }

    constexpr float kLazy = 8.f;
    const int xs = swz_x<CPR>(lr);
    // this wave's keys of tile j from stage st
    auto compute = [&](int j, int st) {
      const T* kt = smem + (long)st * L::kStage;
      const T* vt = kt + (KIND == 0 ? L::kTile : KIND == 1 ? 2 * L::kTile : 0);
      const int n0 = tile_at(j) + wk * KPW, kr = wk * KPW;
      if (n0 >= hi) return;                                       // no row of the wave sees these keys
      f32x16 s[NB];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
        for (int e = 0; e < 16; ++e) s[nb][e] = 0.f;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
          mma32(s[nb], load_frag_swz<T>(kt + (kr + nb * 32 + lr) * D, 4 * cb + 2 * h, xs), qf[cb]);
          if constexpr (KIND == 1)
            mma32(s[nb], load_frag_swz<T>(kt + L::kTile + (kr + nb * 32 + lr) * D, 4 * cb + 2 * h, xs), qf[cb]);
        }
      }
      const bool partly = n0 + KPW > lo;
      if (partly) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int e = 0; e < 16; ++e) s[nb][e] = n0 + nb * 32 + 8 * (e / 4) + 4 * h + e % 4 < limit ? s[nb][e] : -INFINITY;
      }
      // online softmax with a lazily raised reference: O and l are rescaled only when a tile's maximum exceeds the reference by
      // more than kLazy (probabilities stay below 2^kLazy)
      float mx = -INFINITY;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[nb][e]);
      mx = halves_max(mx) * p.scale;
      const bool raise = mx > m_run + kLazy;                      // -inf + kLazy = -inf: the first tile with a key raises
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
      for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
        for (int e = 0; e < 16; ++e) s[nb][e] = fast_exp2(s[nb][e] * p.scale - m_use);
        l_run = block_sum(s[nb], l_run);
        const Frag<T> pf = to_frag<T>(s[nb]);
        constexpr int TF = CB < 2 ? 1 : 2;
#pragma unroll
        for (int k = 0; k < CB / TF; ++k) {
          Frag<T> vf[TF];
          load_frags_tr_swz<CPR, false>(vf, vt, kr + nb * 32, k * TF * 32, lane);
          bool fine = true;
          if (partly)
#pragma unroll
            for (int f = 0; f < TF; ++f) fine = fine && frag_finite(vf[f]);
          if (__builtin_amdgcn_ballot_w64(!fine) == 0ull) {
#pragma unroll
            for (int f = 0; f < TF; ++f) mma32(oacc[k * TF + f], vf[f], pf);
          } else {
            const Frag<T> seen = frag_seen(limit - n0 - nb * 32 - 4 * h, T());
#pragma unroll
            for (int f = 0; f < TF; ++f) {
              take_nonfinite<T>(vf[f], seen, oacc[k * TF + f]);
              mma32(oacc[k * TF + f], vf[f], pf);
            }
          }
        }
      }
    };

    if constexpr (KIND != 1) {
      int* entries = reinterpret_cast<int*>(smem_raw + L::kTiles) + wave * 4 * 64;
      // table entries of tile j's rows, by way of LDS: an entry in a register would be waited for with every tile behind it.
      // Rows behind the last repeat it and are masked.
      auto fetch_entries = [&](int j) {
        const int n = min(tile_at(j) + lane, hi_all - 1);
        word_to_lds(table + min(divide(n, p.ps), pages - 1), entries + (j & 3) * 64);
      };
      constexpr int PK = D / 8, PIECES = KIND == 0 ? D / 32 : D / 64 > 0 ? D / 64 : 1;  // pieces of a tile, of a wave
      auto issue = [&](int j, int st) {
        const int n0 = tile_at(j);
        const int* ids = entries + (j & 3) * 64;
        T* kt = smem + (long)st * L::kStage;
        int l = lane;
        asm volatile("" : "+v"(l));                               // (rows and chunks of the pieces are formed afresh, not kept across the loop)
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
          const int q = wave + 8 * i, q1 = q % PK;
          const bool value = q >= PK;
          if (KIND == 2 && value) break;                          // (narrow tiles: half of the waves)
          const int row = q1 * RPP + l / CPR, c = ((l % CPR) ^ swz_x<CPR>(row)) * 8;
          const int n = min(n0 + row, hi_all - 1);
          const long pg = paged_page(ids[row], p.n_pages), a = n - divide(n, p.ps) * p.page_size;
          const T* at = value ? static_cast<const T*>(p.V) + pg * p.v_stride + a * p.rt3 + c
                              : static_cast<const T*>(p.K) + pg * p.k_stride + a * p.r3 + c;
          chunk_to_lds(c < (value ? p.rt3 : p.r3) ? at : reinterpret_cast<const T*>(paged_zeros), kt + (value ? L::kTile : 0) + q1 * 512);
        }
      };
      // vector-memory operations behind those of tile j when round j begins: entries, a stage, entries
      constexpr int OPS = PIECES + 2;
      fetch_entries(0);
      fetch_entries(1);
      fetch_entries(2);
      wait_vm<0>();                                               // entries, and plain loads out of the way of the counted ones
      issue(0, 0);
      fetch_entries(3);
      issue(1, 1);
      int st = 0;
      for (int j = 0; j < cnt; ++j) {
        fetch_entries(j + 4);
        wait_vm<OPS>();                                           // this wave's part of tile j is there, its reads of tile j - 1 are done
        wait_lds();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        const int st2 = st == 0 ? 2 : st - 1;                     // (j + 2) % 3, the stage of tile j - 1
        issue(j + 2, st2);
        compute(j, st);
        st = st == 2 ? 0 : st + 1;
      }
      wait_vm<0>();                                               // tiles requested past the end still land in LDS
    } else {
      // a thread's chunks of a tile: channels 8 ch of row tid % 64 (+ 0 .. of the chunks 8 apart): neighbouring lanes read
      // neighbouring positions of the rotation table
      constexpr int CPT = kTileKeys * CPR / 512 > 0 ? kTileKeys * CPR / 512 : 1;
      const int row = threadIdx.x % 64, ch0 = threadIdx.x / 64;
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
      for (int j = 0; j < cnt; ++j) {
        __syncthreads();
        store((j + 1) & 1);                                       // the stage of tile j - 1
        load(j + 2);
        compute(j, j & 1);
      }
    }
  }

  // ---- the sums of the waves that share rows, then the rows themselves ----
  if constexpr (WK > 1) {
    static_assert(WK == 2, "one wave hands over");
    __syncthreads();
    float* sums = reinterpret_cast<float*>(smem_raw) + (long)wr * (16 * CB + 2) * 64 + lane;
    if (wk == 1) {
      sums[0] = m_run;
      sums[64] = l_run;
#pragma unroll
      for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int e = 0; e < 16; ++e) sums[(2 + 16 * cb + e) * 64] = oacc[cb][e];
    }
    __syncthreads();
    if (wk == 1) return;
    const float m2 = sums[0], top = fmaxf(m_run, m2);
    const float f1 = m_run == -INFINITY ? 0.f : fast_exp2(m_run - top), f2 = m2 == -INFINITY ? 0.f : fast_exp2(m2 - top);
    m_run = top;
    l_run = l_run * f1 + sums[64] * f2;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int e = 0; e < 16; ++e) oacc[cb][e] = oacc[cb][e] * f1 + sums[(2 + 16 * cb + e) * 64] * f2;
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

template <int D, int WR, int KIND, bool PREFIX> static hipError_t tile_one(const PagedArgs& a, hipStream_t s) {
  const size_t smem = TileLds<D, KIND>::kBytes;
  auto kern = paged_tile_kernel<D, WR, KIND, PREFIX>;
  static LdsOnce lds_once;                                       // one per kernel instantiation
  if (hipError_t e = allow_dynamic_lds(lds_once, kern, smem); e != hipSuccess) return e;
  const int rows = 32 * WR, blocks = PREFIX ? (int)(((long)a.T * a.nH + rows - 1) / rows) : paged_rows_blocks(a, rows);
  hipLaunchKernelGGL(kern, dim3(blocks, PREFIX ? a.prefix_parts : a.own_parts > 0 ? a.own_parts : 1), dim3(512), smem, s, a);
  return hipGetLastError();
}
template <int D, int WR> static hipError_t tile_variant(const PagedArgs& a, bool prefix, hipStream_t s) {
  const int kind = !a.shared_kv ? 0 : a.rope != nullptr ? 1 : 2;
  if (prefix) return kind == 0 ? tile_one<D, WR, 0, true>(a, s) : kind == 1 ? tile_one<D, WR, 1, true>(a, s) : tile_one<D, WR, 2, true>(a, s);
  return kind == 0 ? tile_one<D, WR, 0, false>(a, s) : kind == 1 ? tile_one<D, WR, 1, false>(a, s) : tile_one<D, WR, 2, false>(a, s);
}
hipError_t launch_paged_tile(const PagedArgs& a, bool prefix_pass, hipStream_t s) {
  switch (a.D) {
    case 32: return tile_variant<32, kTileWaves>(a, prefix_pass, s);
    case 64: return tile_variant<64, kTileWaves>(a, prefix_pass, s);
    case 128: return tile_variant<128, kTileWaves>(a, prefix_pass, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace ta
