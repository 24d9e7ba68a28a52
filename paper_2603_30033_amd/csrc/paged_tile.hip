// Attention over the paged latent cache for many rows of one sequence (bf16: pieces of prompts, and the rows of a whole batch on a
// common prefix).
//
// A cached row serves all (token, head) rows, so with R of them a key costs 4 D R flops and 4 D bytes: from a few dozen rows on the
// matrix pipe bounds it.  A workgroup of four waves takes 128 rows, a wave 32 of them, and all keys (or a part of them) in tiles that
// its waves share in LDS.  Tiles go from the pages straight into one of two LDS stages, a tile ahead.  Two workgroups share a
// compute unit: between two barriers a workgroup's waves do the same at the same time (reads, products, exponentials), and another
// workgroup that is not in step with it fills the gaps (four sequences with up to 512 new tokens on up to 4097 rows, 32 heads of 128
// channels: 123 us, eight waves of one workgroup in step 135).  With shares of equal work (below) that call takes 67 us, its largest
// part at 0.8 PFLOP/s; the rest is the launches, the first loads and the partial results.
//
// Probabilities are rounded to bf16 once for the value product, as the result is, where paged_stream keeps two parts: a second part is as
// many matrix instructions again as the value product has, which bounds this kernel and not that one.  The relative error of the sum
// is that of one more rounding of the result (0.0018 to 0.0023 in the root mean square, with both parts 0.0013 to 0.0017).
#include "paged_block.h"

namespace ta {

// KIND 0: key and value pools; 1: one pool, keys rotated on their way into LDS, kept as two bf16 parts; 2: one pool, nothing rotated
template <int D, int KIND> struct TileLds {
  static constexpr int kKeys = KIND == 1 ? 32 : 64;               // of a tile
  static constexpr int kTile = kKeys * D;                         // elements
  static constexpr int kStage = kTile * (KIND == 0 ? 2 : KIND == 1 ? 3 : 1);
  static constexpr size_t kBytes = 2ul * kStage * sizeof(bf16);
};

__device__ __forceinline__ int tile_blocks(const PagedArgs& p, const PagedSeq& s) { return (s.nq * p.nH + kTileRows - 1) / kTileRows; }
// The work of a sequence's first i row blocks: kTileBlock for each, and one for every kTileUnit keys that its last row sees (in closed
// form: a block more sees kTileRows / nH keys more; doubles hold these integers exactly).  Not decreasing, and at most
// i (kTileBlock + units of the sequence's own keys), whatever its lengths are.  Two prompts of 4096 tokens, 32 heads of 128 channels:
// 354 us, with kTileBlock 1, 6, 12: 471, 357, 374, with blocks that count alike 577.  Eight of 1024 tokens, 12 heads of 64: 44, 55,
// 45, 46, 49.
__device__ __forceinline__ int tile_work(const PagedArgs& p, const PagedSeq& s, int i) {
  constexpr double R = kTileRows;
  const int own = max(s.len - p.prefix, 0), seen = p.causal ? max(s.len - s.nq - p.prefix, 0) : own;
  const double n = i, keys = n * seen * p.nH + (p.causal ? R / 2 * n * (n + 1) : 0.);   // times nH
  return i * kTileBlock + min((int)fmin(keys * p.tile_per_key, 2147483647.), i * ((own + kTileUnit - 1) / kTileUnit));
}
// the row block in which item `at` of the sequence's work lies
__device__ __forceinline__ int tile_block(const PagedArgs& p, const PagedSeq& s, int at) {
  int lo = 0, hi = tile_blocks(p, s);                             // work(lo) <= at < work(hi)
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (tile_work(p, s, mid) <= at) lo = mid;
    else hi = mid;
  }
  return lo;
}
__device__ __forceinline__ int tile_work(const PagedArgs& p, int b) {
  const PagedSeq s = paged_seq(p, b);
  return tile_work(p, s, tile_blocks(p, s));
}

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

  // ---- which rows, which keys ----
  // Workgroups go to the eight dies in turn, and each die has a cache of its own: workgroup i of a die takes piece i of the die's
  // share of consecutive pieces, which read the same keys.
  const bool pre = PREFIX && (int)blockIdx.x < p.prefix_wgs;      // the prefix's pieces come first, then shares of the sequences' own keys
  const int wg = PREFIX && !pre ? blockIdx.x - p.prefix_wgs : blockIdx.x;
  const int die = wg % 8, in_die = wg / 8;
  // sequence, row block, items of its work that others do before, all its items, items to do
  int b = 0, rb, item = 0, items = 1, left = 1, part = 0, me = 0;
  Shares shares(0, 1, 1);
  int done = 0;                                                   // items in front of this share and of the segments behind
  if (pre) {
    const int blocks = (p.T * p.nH + RB - 1) / RB, per = (blocks * p.prefix_parts + 7) / 8, piece = die * per + in_die;
    if (in_die >= per || piece >= blocks * p.prefix_parts) return;
    part = piece / blocks;
    rb = piece % blocks;
  } else {
    int index, all;
    if (p.tile_wgs == 0) {                                        // a workgroup for every row block
      b = paged_locate(p.B, [=](int) { return wg; }, [&](int i) { return tile_blocks(p, paged_seq(p, i)); },
                       reinterpret_cast<int*>(smem_raw), rb, all);
      if (b < 0) return;
    } else {
      auto start = [&](int total) {                               // of this workgroup's share; behind all if it has none
        shares = Shares(total, p.tile_wgs, kTileLeast);
        const int per = (shares.G + 7) / 8;
        me = die * per + in_die;
        return in_die < per && me < shares.G ? shares.first(me) : total;
      };
      b = paged_locate(p.B, start, [&](int i) { return tile_work(p, i); }, reinterpret_cast<int*>(smem_raw), index, all);
      if (b < 0) {
        if (!PREFIX && all == 0 && blockIdx.x == 0 && threadIdx.x == 0) p.tile_cuts[0].x = 0;
        return;
      }
      done = shares.first(me);
      left = shares.first(me + 1) - done;
      b = __builtin_amdgcn_readfirstlane(b);
      index = __builtin_amdgcn_readfirstlane(index);
      const PagedSeq s = paged_seq(p, b);
      rb = tile_block(p, s, index);
      item = index - tile_work(p, s, rb);
      items = tile_work(p, s, rb + 1) - tile_work(p, s, rb);
      if (!PREFIX && threadIdx.x == 0) {                          // for the join: how many shares there are, what starts in a block
        const int at = done - item;
        if (me == 0) p.tile_cuts[0].x = shares.G;
        else if (item == 0 || shares.group(at) != me - 1) p.tile_cuts[me].y = 0;   // at its start; behind another share's start
        else
          p.tile_cuts[me] = int4{s.q0 * p.nH + rb * RB, min(s.nq * p.nH - rb * RB, RB), shares.group(at + items - 1), shares.first(me - 1) < at};
      }
    }
    rb = __builtin_amdgcn_readfirstlane(rb);
    item = __builtin_amdgcn_readfirstlane(item);
    items = __builtin_amdgcn_readfirstlane(items);
  }

  for (int segment = 0; left > 0; ++segment) {
    int row0 = 0, first = 0, nq, len = p.prefix, pages;           // first row of the sequence in [T * nH], its first key, ..
    const int* table = p.prefix_table;
    if (pre) {
      nq = min(max(p.q_start[p.B], 0), p.T);
      pages = divide(p.prefix - 1, p.ps) + 1;
      if (rb * RB >= nq * p.nH) return;
    } else {
      const PagedSeq s = paged_seq(p, b);
      nq = s.nq;
      row0 = s.q0 * p.nH;
      first = p.prefix;
      len = s.len;
      table = p.table + (long)b * p.max_pages;
      pages = p.max_pages;
    }
    const int n_rows = nq * p.nH, now = pre ? 1 : max(1, min(left, items - item));
    const bool causal = !pre && p.causal;
    const int r0 = rb * RB, rw = r0 + wave * 32;               // first row of the workgroup, of this wave
    const int r = min(rw + lr, n_rows - 1);                       // rows behind the last repeat it and are not stored
    auto sees = [&](int row) { return causal ? len - nq + divide(min(row, n_rows - 1), p.heads) + 1 : len; };
    // keys that the row sees, that all and any rows of the workgroup see
    const int limit = sees(r), lo_all = sees(r0), hi_all = sees(r0 + RB - 1);
    const int hi = sees(rw + 31);                                 // keys that any row of the wave sees
    // items dealt to whole units of the keys that the block sees; who ends here and who goes on from here count alike
    const int units = max(0, hi_all - first + kTileUnit - 1) / kTileUnit;
    auto unit_at = [&](int i) { return i == 0 ? 0 : i == items ? units : __builtin_amdgcn_readfirstlane((int)((double)i * units / items)); };
    const int key0 = pre ? part * p.prefix_keys : first + unit_at(item) * kTileUnit;
    const int key1 = min(hi_all, pre ? key0 + p.prefix_keys : first + unit_at(item + now) * kTileUnit);
    const int cnt = key1 > key0 ? (key1 - key0 + BC - 1) / BC : 0;  // tiles
    const bool busy = rw < n_rows;                                // a wave without rows helps with the loads only

    f32x16 oacc[CB];
    float m_run = -INFINITY, l_run = 0.f;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int e = 0; e < 16; ++e) oacc[cb][e] = 0.f;

    if (cnt > 0) {                                                // (the same for the whole workgroup)
      auto tile_at = [&](int j) { return key0 + min(j, cnt - 1) * BC; }; // past the end: the last again, unused

      Frag<T> qf[CB];
      auto load_queries = [&] {
        const T* q = static_cast<const T*>(p.Q) + (long)(row0 + r) * p.q_row;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) qf[cb] = load_frag_upto<T>(q, cb * 32 + 16 * h, p.r3);
      };

      constexpr float kLazy = 8.f;
      const int xs = swz_x<CPR>(lr);
      // ---- a block of 32 keys, rows kr .. of stage st: scores, probabilities, O += V P ----
      auto scores = [&](int kr, int st, f32x16& s) {
        const T* kt = smem + (long)st * L::kStage + kr * D;
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = 0.f;
        constexpr int G = KIND == 1 && CB > 2 ? 2 : CB;           // channel blocks whose reads are all on their way before a product
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
      };
      // online softmax with a lazily raised reference: O and l are rescaled only when a block's maximum exceeds the reference by more
      // than kLazy (probabilities stay below 2^kLazy)
      auto probabilities = [&](f32x16& s) {
        float mx = -INFINITY;
#pragma unroll
        for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[e]);
        mx = halves_max(mx) * p.scale;
        const bool raise = mx > m_run + kLazy;                    // -inf + kLazy = -inf: the first block with a key raises
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
        return to_frag<T>(s);
      };
      // some rows may not see some of the keys, n0 ..
      auto values = [&](int n0, int kr, int st, const Frag<T>& pf) {
        const T* vt = smem + (long)st * L::kStage + kr * D + (KIND == 0 ? L::kTile : KIND == 1 ? 2 * L::kTile : 0);
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
          Frag<T> vf[1];
          load_frags_tr_swz<CPR>(vf, vt, 0, cb * 32, lane);
          if (__builtin_amdgcn_ballot_w64(!frag_finite(vf[0])) != 0ull) take_nonfinite<T>(vf[0], limit - n0 - 4 * h, oacc[cb]); // (rare)
          mma32(oacc[cb], vf[0], pf);
        }
      };
      // A tile that all rows of the workgroup see: the scores of its two blocks, then exponentials and value product of one block and of the
      // other.  A wave issues in order, so little of a product runs under this wave's own exponentials (4050 cycles a tile alone on a SIMD,
      // 1024 of them matrix instructions); the other workgroup's wave on the SIMD fills some of the rest.
      auto whole = [&](int st) {
        f32x16 s[NB];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) scores(nb * 32, st, s[nb]);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          __builtin_amdgcn_sched_barrier(0);
          // the first value fragments are on their way under the exponentials
          constexpr int TF = CB < 2 ? 1 : 2;
          const T* vt = smem + (long)st * L::kStage + nb * 32 * D + (KIND == 0 ? L::kTile : KIND == 1 ? 2 * L::kTile : 0);
          Frag<T> vf[TF];
          load_frags_tr_swz<CPR>(vf, vt, 0, 0, lane);
          const Frag<T> pf = probabilities(s[nb]);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int k = 0; k < CB / TF; ++k) {
            if (k > 0) load_frags_tr_swz<CPR>(vf, vt, 0, k * TF * 32, lane);
#pragma unroll
            for (int f = 0; f < TF; ++f) mma32(oacc[k * TF + f], vf[f], pf);
          }
        }
      };
      // any other, a block that no row of the wave sees passed over
      auto edge = [&](int j, int st) {
#pragma unroll 1
        for (int nb = 0; nb < NB; ++nb) {
          const int n0 = tile_at(j) + nb * 32;
          if (n0 >= hi) break;
          f32x16 s;
          scores(nb * 32, st, s);
#pragma unroll
          for (int e = 0; e < 16; ++e) s[e] = n0 + 8 * (e / 4) + 4 * h + e % 4 < limit ? s[e] : -INFINITY;
          const Frag<T> pf = probabilities(s);
          values(n0, nb * 32, st, pf);
        }
      };
      const int n_whole = min(max(lo_all - key0, 0) / BC, cnt);

      if constexpr (KIND != 1) {
        // A wave takes BC / 4 consecutive rows of a tile: NK pieces of 1 KB of the keys, and as many of the values.  Rows that lie in
        // one page (the usual sizes): its number comes by a scalar read, there is one start for the wave, in 16-byte units (32 bits:
        // 64 GiB), and lanes add their row and chunk to it.  Rows behind the last are whatever the page holds, chunks behind a row's
        // end (which meet zeros of the queries, or become channels that are not stored) repeat its last.  Else every lane looks up its
        // own rows.
        constexpr int NK = BC * D / 512 / 4, ROWS = BC / 4;
        static_assert(ROWS == 16, "rows of a wave");
        const uint32_t k16 = (uint32_t)(p.k_stride / 8), v16 = (uint32_t)(p.v_stride / 8), rk = p.r3 / 8, rv = p.rt3 / 8;
        const bool straight = p.page_size % ROWS == 0 && first % ROWS == 0;
        const auto* entries = (const __attribute__((address_space(4))) int*)table;
        auto entry_at = [&](int j) { return entries[min(divide(min(tile_at(j) + wave * ROWS, hi_all - 1), p.ps), pages - 1)]; };
        int entry = entry_at(0);                                  // of the tile that is filled next
        auto fill = [&](int j, int st) {
          T* kt = smem + (long)st * L::kStage + wave * NK * 512;
          const int n0 = tile_at(j) + wave * ROWS;
          int l = lane;
          asm volatile("" : "+v"(l));                             // (chunks of the pieces are formed afresh, not kept across the loop)
          if (straight) {
            const uint32_t page = paged_page(entry, p.n_pages), at = n0 - divide(n0, p.ps) * p.page_size;
            const char* k = static_cast<const char*>(p.K) + (unsigned long)(page * k16 + at * rk) * 16;
            const char* v = KIND == 0 ? static_cast<const char*>(p.V) + (unsigned long)(page * v16 + at * rv) * 16 : nullptr;
#pragma unroll
            for (int i = 0; i < NK; ++i) {
              const uint32_t row = i * RPP + l / CPR, c = (l % CPR) ^ swz_x<CPR>(i * RPP + l / CPR);
              chunk_to_lds(k + (row * rk + min(c, rk - 1)) * 16, kt + i * 512);
              if constexpr (KIND == 0) chunk_to_lds(v + (row * rv + min(c, rv - 1)) * 16, kt + L::kTile + i * 512);
            }
            entry = entry_at(j + 1);
          } else {
            int found[NK];                                        // (all on their way before one is waited for)
#pragma unroll
            for (int i = 0; i < NK; ++i) found[i] = table[min(divide(min(n0 + i * RPP + l / CPR, hi_all - 1), p.ps), pages - 1)];
#pragma unroll
            for (int i = 0; i < NK; ++i) {
              const uint32_t row = i * RPP + l / CPR, c = (l % CPR) ^ swz_x<CPR>(row);
              const int n = min(n0 + (int)row, hi_all - 1);
              const uint32_t page = paged_page(found[i], p.n_pages), at = n - divide(n, p.ps) * p.page_size;
              chunk_to_lds(static_cast<const u32x4*>(p.K) + (page * k16 + at * rk + min(c, rk - 1)), kt + i * 512);
              if constexpr (KIND == 0)
                chunk_to_lds(static_cast<const u32x4*>(p.V) + (page * v16 + at * rv + min(c, rv - 1)), kt + L::kTile + i * 512);
            }
          }
        };
        fill(0, 0);
        load_queries();                                           // (behind the first tile, whose way is the longer one)
        auto arrived = [] {
          wait_vm<0>();                                           // this wave's part of tile j is there,
          wait_lds();                                             // its reads of tile j - 1 are done
          __builtin_amdgcn_s_barrier();
          asm volatile("" ::: "memory");
        };
        int j = 0;
        for (; j < n_whole; ++j) {
          arrived();
          fill(j + 1, (j + 1) & 1);                               // into the stage of tile j - 1
          if (busy) whole(j & 1);
        }
        for (; j < cnt; ++j) {
          arrived();
          fill(j + 1, (j + 1) & 1);
          if (busy) edge(j, j & 1);
        }
        wait_vm<0>();                                             // tiles requested past the end still land in LDS
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
            float most = 0.f;
#pragma unroll
            for (int d = 0; d < 4; ++d) {
              const float c = reg.cs[i][d / 2][2 * (d % 2)], sn = reg.cs[i][d / 2][2 * (d % 2) + 1];
              const float x0 = __uint_as_float(reg.x[i][d] << 16), x1 = __uint_as_float(reg.x[i][d] & 0xffff0000u);
              const f32x2 y = {x0 * c - x1 * sn, x0 * sn + x1 * c};
              most = fmaxf(fmaxf(fabsf(y[0]), fabsf(y[1])), most);
              hi16[d] = __builtin_bit_cast(uint32_t, __builtin_convertvector(y, bf16x2));
              const f32x2 z = {y[0] - __uint_as_float(hi16[d] << 16), y[1] - __uint_as_float(hi16[d] & 0xffff0000u)};
              lo16[d] = __builtin_bit_cast(uint32_t, __builtin_convertvector(z, bf16x2));
            }
            // the first part of an infinite channel leaves Inf - Inf: nothing of it is kept
            if (most > 3.38e38f)                                    // (rare)
#pragma unroll
              for (int d = 0; d < 4; ++d) {
                const uint32_t bad = (((hi16[d] & Bits<T>::kExp) + Bits<T>::kLow) >> Bits<T>::kSign) & Bits<T>::kUnit;
                lo16[d] &= ~(bad * Bits<T>::kAll);
              }
            const int at = row * D + ((ch ^ swz_x<CPR>(row)) * 8);
            *reinterpret_cast<u32x4*>(kt + at) = hi16;
            *reinterpret_cast<u32x4*>(kt + L::kTile + at) = lo16;
            *reinterpret_cast<u32x4*>(kt + 2 * L::kTile + at) = reg.x[i];
          }
        };
        load(0);
        load_queries();
        __syncthreads();                                          // (the plan's words are done with)
        store(0);
        load(1);
        int j = 0;
        for (; j < n_whole; ++j) {
          __syncthreads();
          store((j + 1) & 1);                                     // the stage of tile j - 1
          load(j + 2);
          if (busy) whole(j & 1);
        }
        for (; j < cnt; ++j) {                                    // (nothing is kept in registers for later: they are all in use)
          __syncthreads();
          load(j + 1);
          store((j + 1) & 1);
          if (busy) edge(j, j & 1);
        }
      }
    }

    // ---- the rows: a result, or a part of one ----
    const float l = halves_sum(l_run);
    const bool complete = !pre && now == items;                   // nobody else has keys of these rows
    if (rw + lr < n_rows) {
      const long at = (long)row0 + rw + lr;
      const bool direct = complete && !PREFIX;
      const bool by_row = pre || complete;
      const int shared = (2 * me + (segment > 0)) * RB + wave * 32 + lr;
      const long slot = by_row ? (long)(pre ? part : p.prefix_parts) * p.T * p.nH + at : shared;
      float* po = by_row ? p.part_o : p.stream_o;
      float2* pml = by_row ? p.part_ml : p.stream_ml;
      // for the join: this share, the first of the row's, and how many more there are
      if (PREFIX && !pre && item == 0 && h == 0)
        p.tile_rows[at] = int2{shared, complete ? 0 : shares.group(done + items - 1) - me};
#pragma unroll
      for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4 o = {oacc[cb][4 * q], oacc[cb][4 * q + 1], oacc[cb][4 * q + 2], oacc[cb][4 * q + 3]};
          const int c = cb * 32 + 8 * q + 4 * h;
          if (direct) paged_result<T>(p, at, c, m_run, l, o);
          else paged_partial<D>(po, pml, slot, c, m_run, l, o);
        }
    }
    left -= now;
    done += now;
    if (pre || left == 0) break;
    item = 0;
    PagedSeq s = paged_seq(p, b);
    if (++rb == tile_blocks(p, s)) {
      rb = 0;
      do {
        if (++b >= p.B) return;                                   // (work is left, so a sequence follows if q_start never decreases)
        s = paged_seq(p, b);
      } while (s.nq == 0);
    }
    items = __builtin_amdgcn_readfirstlane(tile_work(p, s, rb + 1) - tile_work(p, s, rb));
    __syncthreads();
  }
}

// ------------------------------------------------------------------------------------------------------------------
// The partial results of rows that several workgroups share, or that have a prefix.  A row by D/4 threads, or by `groups` times as
// many.  Without a prefix only the row blocks in which a share starts have something to join (grid: shares x groups of rows), with one
// all rows have.  What there is to join for a block or row the workgroup that did its first share has left in memory (to look for it
// here again: 20 us more).
// ------------------------------------------------------------------------------------------------------------------
template <int D, bool PREFIX>
__global__ __launch_bounds__(256) void paged_tile_join_kernel(PagedArgs p, int groups) {
  using T = bf16;
  constexpr int L = D / 4, SLOTS = 256 / L;
  __shared__ float4 po[256];
  __shared__ float2 pml[SLOTS];
  const int tid = threadIdx.x, per = SLOTS / groups, slot = tid / L, c = tid % L * 4, group = slot / per;
  const long rows = (long)p.T * p.nH;
  long row;
  int first, more;                                                // slot of the first share's result; shares behind it
  bool live;
  if constexpr (PREFIX) {
    row = (long)blockIdx.x * per + slot % per;
    const int q0 = min(max(p.q_start[0], 0), p.T), q1 = min(max(p.q_start[p.B], 0), p.T);
    live = row >= (long)q0 * p.nH && row < (long)q1 * p.nH;       // not behind the last sequence
    const int2 e = row < rows ? p.tile_rows[row] : int2{0, 0};
    // (bounded: a row that no sequence has finds anything here)
    first = min(max(e.x, 0), max(2 * p.tile_wgs * kTileRows - 1, 0));
    more = min(max(e.y, 0), max(p.tile_wgs - 1 - first / (2 * kTileRows), 0));
  } else {
    const int g = (int)blockIdx.x + 1, r = (int)blockIdx.y * per + slot % per, shares = p.tile_cuts[0].x;
    const int4 e = p.tile_cuts[g];
    if (g >= shares || (int)blockIdx.y * per >= e.y) return;
    live = r < e.y;
    row = (long)e.x + r;
    first = (2 * (g - 1) + e.w) * kTileRows + r;
    more = max(min(e.z, p.tile_wgs - 1) - (g - 1), 0);
  }
  RowSum sum;
  if (PREFIX ? row < rows : live) {
    auto by_row = [&](int i, const float2*& ml, const float*& o) {
      ml = p.part_ml + i * rows + row;
      o = p.part_o + (i * rows + row) * D + c;
    };
    if (PREFIX) sum.add_parts(p.prefix_parts, group, groups, by_row);   // (waits for nothing that is read above)
    if (PREFIX && (more == 0 || !live))
      sum.add_parts(1, group, groups, [&](int, const float2*& ml, const float*& o) { by_row(p.prefix_parts, ml, o); });
    else
      sum.add_parts(more + 1, group, groups, [&](int i, const float2*& ml, const float*& o) {
        // share i's first segment, but the first share's last
        const long at = i == 0 ? first : (first / (2 * kTileRows) + i) * 2l * kTileRows + first % kTileRows;
        ml = p.stream_ml + at;
        o = p.stream_o + at * D + c;
      });
  }
  sum.add_groups(po, pml, slot, group, groups, per, L);
  if (group == 0 && live) paged_result<T>(p, row, c, sum.m, sum.l, sum.o);
}

template <int D, int KIND, bool PREFIX> static hipError_t tile_one(const PagedArgs& a, hipStream_t s) {
  const size_t smem = TileLds<D, KIND>::kBytes;
  auto kern = paged_tile_kernel<D, KIND, PREFIX>;
  static LdsOnce lds_once;                                       // one per kernel instantiation
  if (hipError_t e = allow_dynamic_lds(lds_once, kern, smem); e != hipSuccess) return e;
  const uint32_t own = a.tile_wgs == 0 ? paged_rows_blocks(a, kTileRows) : (a.tile_wgs + 7) / 8 * 8, grid = own + (PREFIX ? a.prefix_wgs : 0);
  hipLaunchKernelGGL(kern, dim3(grid), dim3(256), smem, s, a);
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

template <int D> static hipError_t tile_join_one(const PagedArgs& a, hipStream_t s) {
  constexpr int SLOTS = 256 / (D / 4);
  const int blocks = paged_rows_blocks(a, kTileRows), parts = a.prefix_parts + (a.tile_wgs > 0 ? a.tile_wgs / blocks : 0) + 1;
  int groups = 1;                                                 // one for every 8 parts that a row has on average
  while (groups < 8 && 8 * groups < parts) groups *= 2;
  const int per = SLOTS / groups, most = kTileRows < a.max_new * a.nH ? kTileRows : a.max_new * a.nH;
  if (a.prefix_parts > 0)
    hipLaunchKernelGGL((paged_tile_join_kernel<D, true>), dim3(((long)a.T * a.nH + per - 1) / per), dim3(256), 0, s, a, groups);
  else
    hipLaunchKernelGGL((paged_tile_join_kernel<D, false>), dim3(a.tile_wgs - 1, (most + per - 1) / per), dim3(256), 0, s, a, groups);
  return hipGetLastError();
}
hipError_t launch_paged_tile_join(const PagedArgs& a, hipStream_t s) {
  switch (a.D) {
    case 32: return tile_join_one<32>(a, s);
    case 64: return tile_join_one<64>(a, s);
    case 128: return tile_join_one<128>(a, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace ta
