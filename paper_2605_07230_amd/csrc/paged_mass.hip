// paged_mass kernels for gfx950: the attention weight that positions of a cache in pages gather,
//     w(y) = sum over tokens j and query heads g of a kv head:  exp(scale <q_jg, k_y> - lse_jg).
//
// lse is known, so there is no maximum to follow and nothing to rescale: one product S = Q K^T, an exponential per score and a sum down each column.  The keys stand still - a
// wave holds 16 KW of them in registers - and the query rows go past them, so a column's sum stays in one wave from its first term to its last: no atomics, no partial results
// in memory, and an order that depends on the call's sizes alone.
//
// S = Q K^T (queries as A, keys as B): a lane owns a key of each group of 16 and adds up the queries 4 g .. 4 g + 3 of every product; the four 16-lane rows meet once at the end.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "common.h"

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr int WAVES = 4, STAGE = 64 * WAVES;   // query rows that are looked up together, a thread each

struct MassParams {
  paged_mass_args a;
  int group, most_len;   // query heads of a kv head; the longest row that the bounds allow
  int key_blocks;        // workgroups that a row's keys may need
  int wave_tiles;        // (few query rows) tiles that a wave goes through
  float scale_log2e;
  unsigned group_inv;    // floor(2^32 / group) + 1: a query row's token as a high product (rows times group stay below 2^32); 0 for one head
  int* dev_status;
};

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// ---- 16 rows as an operand: lane (l16, g) holds row l16, and of its elements those that stand at k = g of some product
template <typename T, int D, bool VEC>
struct Operand;
template <int D, bool VEC>
struct Operand<uint16_t, D, VEC> {
  static constexpr int N = D / 32;
  bf16x8 x[N];
  __device__ __forceinline__ void load(const uint16_t* row, int g, int) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = *(const bf16x8*)(row + 32 * i + 8 * g);
  }
  __device__ __forceinline__ static f32x4 product(const Operand& a, const Operand& b) {
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < N; ++i) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.x[i], b.x[i], s, 0, 0, 0);
    return s;
  }
};
// f32, D: head_dim rounded up to 16s: element c of the 16 bytes at 16 i + 4 g of both operands meets in product (i, c)
template <int D, bool VEC>
struct Operand<float, D, VEC> {
  static constexpr int N = D / 16;
  f32x4 x[N];
  __device__ __forceinline__ void load(const float* row, int g, int head_dim) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int d = 16 * i + 4 * g;
      if (VEC) x[i] = d < head_dim ? *(const f32x4*)(row + d) : f32x4{0.f, 0.f, 0.f, 0.f};
      else
#pragma unroll
        for (int c = 0; c < 4; ++c) x[i][c] = d + c < head_dim ? row[d + c] : 0.f;
    }
  }
  __device__ __forceinline__ static f32x4 product(const Operand& a, const Operand& b) {
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int c = 0; c < 4; ++c) s = __builtin_amdgcn_mfma_f32_16x16x4f32(a.x[i][c], b.x[i][c], s, 0, 0, 0);
    return s;
  }
};

// ---- a row of the batch: its tokens, where they stand, the first position that is asked for; n = 0: nothing to do
struct MassRow {
  int s, lo, n, L, Lp, first;
};
__device__ __forceinline__ MassRow row_of(const MassParams& p, int s, bool report) {
  const paged_mass_args& a = p.a;
  const int lo = a.q_off[s], hi = a.q_off[s + 1], L = a.seq_len[s], first = a.first ? max(a.first[s], 0) : 0;
  int flag = 0;
  if (lo < 0 || hi > a.n_tokens || lo > hi || hi - lo > a.max_new) flag = CASCADE_FLAG_TREE_SIZE;
  else if (L < hi - lo || L > p.most_len) flag = CASCADE_FLAG_CAPACITY;   // (negative lengths among them)
  if (a.prefix_len) {
    const int before = a.prefix_len[s];
    if (!flag && before == L) return MassRow{s, 0, 0, 0, 0, 0};
    if (!flag && before != L - (hi - lo)) flag = CASCADE_FLAG_CAPACITY;
  }
  if (flag) {
    if (report) atomicOr(p.dev_status, flag);
    return MassRow{s, 0, 0, 0, 0, 0};
  }
  return MassRow{s, lo, hi - lo, L, L - (hi - lo), first};
}

// A wave's keys, groups of 16 from kb on; returns the groups that hold some.  A group that no token attends, or none of whose positions is asked for, is not read, nor
// is its entry of the table.
template <typename Op, typename T, int KW>
__device__ __forceinline__ unsigned load_keys(const MassParams& p, const MassRow& r, int kvh, int kb, Op (&key)[KW]) {
  const paged_mass_args& a = p.a;
  const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4;
  unsigned there = 0;
  const int reach = a.window > 0 ? max(r.Lp - a.window + 1, 0) : 0;   // the first position that a token sees through the window
#pragma unroll
  for (int kt = 0; kt < KW; ++kt) {
    const int y0 = kb + 16 * kt;
    if (y0 >= r.L || y0 + 15 < r.first || (y0 + 15 < reach && y0 >= a.n_sink)) continue;
    const int e = y0 / a.page_size, page = __builtin_amdgcn_readfirstlane(a.block_table[r.s * a.table_stride + e]);
    if ((unsigned)page >= (unsigned)a.n_pages) {
      if (lane == 0) atomicOr(p.dev_status, CASCADE_FLAG_PAGE);
      continue;
    }
    there |= 1u << kt;
    const int inside = y0 - e * a.page_size + min(l16, r.L - 1 - y0);   // behind the last key: that one again, masked
    key[kt].load((const T*)a.k_pages + page * a.stride_page + kvh * a.stride_head + inside * a.stride_pos, g, a.head_dim);
  }
  return there;
}

// The sums of a wave's groups: lane (l16, g) has position 16 g + l16 of them.
template <int KW>
__device__ __forceinline__ float own_sum(const float (&sum)[KW]) {
  const int g = (threadIdx.x & 63) >> 4;
  float mine = 0.f;
#pragma unroll
  for (int kt = 0; kt < KW; ++kt) {
    const float all = rows4_sum(sum[kt]);
    if (g == kt) mine = all;
  }
  return mine;
}
template <int KW>
__device__ __forceinline__ void write_sums(const MassParams& p, const MassRow& r, int kvh, int kb, const float (&sum)[KW]) {
  const int lane = threadIdx.x & 63;
  const float mine = own_sum<KW>(sum);
  const int y = kb + lane;
  if (lane < 16 * KW && y >= r.first && y < r.L) {
    float* m = p.a.mass + r.s * p.a.mass_stride_row + kvh * p.a.mass_stride_head + y;
    *m = y >= r.Lp ? mine : *m + mine;
  }
}

// ------------------------------------------------------------------------------------------------------------- bf16, few query rows
// Up to 16 NB query rows (single tokens, accepted paths): bound by the stream of keys.  A wave has a tile or two of 64 positions and everything else that it needs on its way before
// them - query rows, lse, the sums so far - so one trip to memory follows the place of a tile, and no wave waits for another.  One token of 64 rows x 4200 keys, 8 kv heads
// of 4, head_dim 128 (568 MB): 116 us = 4.9 TB/s from memory (a large copy: 4.9).
template <int D, int NB, bool DEALT>
__global__ __launch_bounds__(64 * WAVES, NB == 1 ? 4 : 3) void paged_mass_few_kernel(MassParams p) {
  constexpr int KW = 4;
  typedef Operand<uint16_t, D, true> Op;
  const paged_mass_args& a = p.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, g = lane >> 4, G = p.group;
  const int kvh = blockIdx.x % a.n_kv_heads, b = blockIdx.x / a.n_kv_heads;
  int kblk;
  MassRow row;
  if constexpr (!DEALT) {
    kblk = b / a.n_rows;   // (long rows' last tiles come last, from all of them)
    row = row_of(p, b % a.n_rows, kblk == 0 && kvh == 0 && tid == 0);
  } else {
    MassRow mine = {0, 0, 0, 0, 0, 0};
    if (lane < a.n_rows) mine = row_of(p, lane, b == 0 && kvh == 0 && wave == 0);
    const int per = 16 * KW * WAVES * p.wave_tiles, cnt = mine.n > 0 ? (mine.L + per - 1) / per : 0, incl = wave_scan_incl_i(cnt);
    const unsigned long long who = __ballot(incl > b);
    if (!who) return;
    const int l = __ffsll((long long)who) - 1;
    auto of = [&](int x) { return __builtin_amdgcn_readlane(x, l); };
    kblk = b - of(incl - cnt);
    row = MassRow{l, of(mine.lo), of(mine.n), of(mine.L), of(mine.Lp), of(mine.first)};
  }
  const int lo = row.lo, n = row.n, M = n * G, Lp = row.Lp, W = a.window;
  const int kb0 = 16 * KW * (WAVES * p.wave_tiles * kblk + wave), kb1 = min(row.L, kb0 + 16 * KW * WAVES * p.wave_tiles);   // tiles WAVES apart
  if (n == 0 || kb0 >= row.L || kb1 <= row.first) return;
  auto token_of = [&](int r) { return (int)(p.group_inv ? __umulhi((unsigned)r, p.group_inv) : (unsigned)r); };
  Op q[NB];
  float lse[NB][4];
  int x[NB][4];   // positions of rows 4 g + c; -1: the row counts nothing
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int r = min(16 * nb + l16, M - 1), j = token_of(r);
    int t = a.source ? a.source[lo + j] : lo + j;
    if ((unsigned)t >= (unsigned)a.n_source) {
      if (t != -1) atomicOr(p.dev_status, CASCADE_FLAG_PATH);
      t = 0;
    }
    q[nb].load((const uint16_t*)a.q + t * a.q_stride + (kvh * G + r - j * G) * D, g, D);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int rc = 16 * nb + 4 * g + c, jc = token_of(min(rc, M - 1)), tc = a.source ? a.source[lo + jc] : lo + jc;
      x[nb][c] = rc < M && (unsigned)tc < (unsigned)a.n_source ? Lp + jc : -1;
      lse[nb][c] = a.lse[(long long)max(min(tc, a.n_source - 1), 0) * a.n_heads + kvh * G + min(rc, M - 1) - jc * G];
    }
  }
  bool all_count = true;
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      if (!(fabsf(lse[nb][c]) < INFINITY)) x[nb][c] = -1;
      all_count = all_count && x[nb][c] >= 0;
      lse[nb][c] *= LOG2E;
    }
  all_count = __all(all_count);
  for (int kb = kb0; kb < kb1; kb += 16 * KW * WAVES) {
    if (kb + 16 * KW <= row.first) continue;
    const int y = kb + lane;
    float* const at = a.mass + row.s * a.mass_stride_row + kvh * a.mass_stride_head + y;
    const bool wanted = y >= row.first && y < row.L;
    const float before = wanted && y < Lp ? *at : 0.f;
    Op key[KW];
    const unsigned there = load_keys<Op, uint16_t, KW>(p, row, kvh, kb, key);
    // whether every row sees all of the keys
    const bool whole = all_count && there == (1u << KW) - 1 && kb + 16 * KW - 1 <= Lp && (W == 0 || Lp + n - 1 - kb < W);
    float sum[KW];
#pragma unroll
    for (int kt = 0; kt < KW; ++kt) {
      sum[kt] = 0.f;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        if (nb > 0 && 16 * nb >= M) continue;
        f32x4 w = Op::product(q[nb], key[kt]);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          w[c] = fast_exp2(fmaf(w[c], p.scale_log2e, -lse[nb][c]));
          if (!whole) {
            const int yk = kb + 16 * kt + l16;
            const bool seen = yk <= x[nb][c] && (W == 0 || x[nb][c] - yk < W || yk < a.n_sink) && ((there >> kt) & 1);
            w[c] = seen ? w[c] : 0.f;
          }
        }
        sum[kt] += (w[0] + w[1]) + (w[2] + w[3]);
      }
    }
    const float mine = own_sum<KW>(sum);
    if (wanted) *at = before + mine;   // (a new token's own: before is 0)
  }
}

// -------------------------------------------------------------------------------------------------------------------------------- f32
// Workgroup = (row, kv head, 64 KW positions), a wave to 16 KW of them.  Query rows come straight from memory, 16 at a time, for each wave.
template <int D, int KW, bool VEC>
__global__ __launch_bounds__(64 * WAVES) void paged_mass_kernel(MassParams p) {
  typedef Operand<float, D, VEC> Op;
  const paged_mass_args& a = p.a;
  __shared__ long long s_q[STAGE];   // where a query row lies
  __shared__ __align__(16) int s_x[STAGE];      // its position; -1: it counts nothing
  __shared__ __align__(16) float s_lse[STAGE];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, g = lane >> 4, G = p.group;
  const int kvh = blockIdx.x % a.n_kv_heads, b = blockIdx.x / a.n_kv_heads, kblk = b % p.key_blocks;
  const MassRow row = row_of(p, b / p.key_blocks, kblk == 0 && kvh == 0 && tid == 0);
  const int lo = row.lo, n = row.n, M = n * G, Lp = row.Lp, W = a.window;
  const int kb0 = 16 * KW * WAVES * kblk;
  if (n == 0 || kb0 >= row.L || kb0 + 16 * KW * WAVES <= row.first) return;
  const int kb = kb0 + 16 * KW * wave;
  Op key[KW];
  const unsigned there = load_keys<Op, float, KW>(p, row, kvh, kb, key);
  // ---- the query rows that see some of them, in blocks of 16
  int from = 0, to = M;
  if (!there) to = 0;
  else {
    if (kb > Lp) from = min(kb - Lp, n) * G / 16 * 16;
    if (W > 0 && kb >= a.n_sink) to = (int)min((long long)M, max(0ll, (long long)(kb + 16 * KW - 1) + W - Lp) * G);
  }
  float sum[KW];
#pragma unroll
  for (int kt = 0; kt < KW; ++kt) sum[kt] = 0.f;
  const int wg_from = kb0 > Lp ? min(kb0 - Lp, n) * G / 16 * 16 : 0;
  for (int c0 = wg_from; c0 < M; c0 += STAGE) {
    __syncthreads();
    bool counts = false;
    {
      const int r = c0 + tid;
      int x = -1;
      float lse = 0.f;
      long long at = 0;
      if (r < M) {
        const int j = r / G, h = kvh * G + r - j * G;
        int t = lo + j;
        if (a.source) t = a.source[t];
        if ((unsigned)t < (unsigned)a.n_source) {
          at = t * a.q_stride + (long long)h * a.head_dim;
          lse = a.lse[(long long)t * a.n_heads + h];
          if (fabsf(lse) < INFINITY) { x = Lp + j; counts = true; lse *= LOG2E; }
          else lse = 0.f;
        } else if (t != -1) {
          atomicOr(p.dev_status, CASCADE_FLAG_PATH);
        }
      }
      s_q[tid] = at;
      s_x[tid] = x;
      s_lse[tid] = lse;
    }
    const bool all_count = __syncthreads_and(counts || c0 + tid >= M);
    for (int r0 = max(c0, from); r0 < min(c0 + STAGE, to); r0 += 16) {
      const int i0 = r0 - c0, rows = min(16, M - r0);
      Op q;
      q.load((const float*)a.q + s_q[i0 + min(l16, rows - 1)], g, a.head_dim);
      const f32x4 lse = *(const f32x4*)(s_lse + i0 + 4 * g);
      // whether every row sees all of the wave's keys
      const int x0 = Lp + r0 / G, x1 = Lp + (r0 + rows - 1) / G;
      const bool whole = all_count && rows == 16 && there == (1u << KW) - 1 && kb + 16 * KW - 1 <= x0 && (W == 0 || x1 - kb < W);
#pragma unroll
      for (int kt = 0; kt < KW; ++kt) {
        f32x4 w = Op::product(q, key[kt]);
#pragma unroll
        for (int c = 0; c < 4; ++c) w[c] = fast_exp2(fmaf(w[c], p.scale_log2e, -lse[c]));
        if (!whole) {
          const int y = kb + 16 * kt + l16;
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int x = s_x[i0 + 4 * g + c];
            const bool seen = y <= x && (W == 0 || x - y < W || y < a.n_sink) && ((there >> kt) & 1);
            w[c] = seen ? w[c] : 0.f;
          }
        }
        sum[kt] += (w[0] + w[1]) + (w[2] + w[3]);
      }
    }
  }
  write_sums<KW>(p, row, kvh, kb, sum);
}

// ------------------------------------------------------------------------------------------------------------ bf16, many query rows
// Workgroup = (row, kv head, 64 KG positions), 64 to a wave; where KG is less than 4 the waves of the same keys share the query rows of a block.  Blocks of 64 query rows and their
// lse pass through a ring in LDS, filled by LDS-direct loads (M0 = the LDS address of a wave's 1 KiB) two blocks ahead of their use: a wave waits for its own loads of the block
// needed next (vmcnt), then one bare barrier makes everybody's visible and the oldest place free.  Such a load puts lane l's 16 bytes at 16 l, so rows cannot be padded;
// slot q of row r holds piece q ^ swz(r), and the 16 rows of an operand meet in no bank.  lse of rows that are not there, and of tokens without a source, come from a place that
// holds infinity: they count nothing.  Bound by products and exponentials, which take turns (matrix cores 28 % and vector ALU 44 % of the cycles where rows differ in length): 16 rows of 1000
// tokens behind 3000, 8 kv heads of 4, 550 us = 835 TFLOP/s (a large product: 1214); 8 rows of 500 to 1000 behind up to 2000 110 to 115.  Three places in the ring: two wait for memory,
// four leave room for two workgroups only.
// Workgroup `b` of a kv head: with up to 64 rows the blocks of keys come in the order of the tokens that see them, min(n, L - y) for the block that begins at y, so what the launch ends
// with is short: 8 rows of 500 to 1000 tokens behind up to 2000 122 -> 115 us (other lengths of them 149 -> 145, 132 -> 105), 16 rows of 100 to 1000 behind up to 4000 223 -> 195, 40 of up to 300
// behind up to 3000 152 -> 120; rows of one length 277 -> 274, of 100 tokens 58 -> 62, for the search.  A lane to a row; how many blocks have at least w tokens is a sum over the rows, and
// w is found bit by bit.
template <int KEYS>
__device__ __forceinline__ MassRow longest_first(const MassParams& p, int b, bool report, int* kblk) {
  const paged_mass_args& a = p.a;
  const int lane = threadIdx.x & 63;
  if (a.n_rows > 64) {   // positions that all tokens see come first, rows one further with every block
    *kblk = b / a.n_rows;
    return row_of(p, (b + *kblk + (*kblk >> 2)) % a.n_rows, report && *kblk == 0 && lane == 0);
  }
  MassRow mine = {0, 0, 0, 0, 0, 0};
  if (lane < a.n_rows) mine = row_of(p, lane, report && b == 0);
  auto at_least = [&](int w) { return mine.n >= w ? (mine.L - w) / KEYS + 1 : 0; };   // (0 < w <= n <= L)
  int w = 0;
  for (int bit = 1 << (31 - __clz(a.max_new)); bit; bit >>= 1)
    if (wave_sum_i(at_least(w | bit)) > b) w |= bit;
  if (w == 0) return MassRow{0, 0, 0, 0, 0, 0};   // fewer blocks than that
  const int above = at_least(w + 1), before = b - wave_sum_i(above), incl = wave_scan_incl_i(at_least(w) - above);   // of blocks with just w tokens the `before`-th
  const int l = __ffsll((long long)__ballot(incl > before)) - 1;
  auto of = [&](int x) { return __builtin_amdgcn_readlane(x, l); };
  // a row's blocks with w tokens follow one another: the last of them that has so many
  *kblk = of((mine.L - w) / KEYS) - (of(incl) - 1 - before);
  return MassRow{l, of(mine.lo), of(mine.n), of(mine.L), of(mine.Lp), of(mine.first)};
}

constexpr int QB = 64, STAGES = 3;   // query rows of a block, places of the ring
__device__ const float s_nothing = INFINITY;

template <int D>
struct ManyGeom {
  static constexpr int RB = 2 * D;          // bytes of a row
  static constexpr int PPR = RB / 16;       // 16-byte pieces of a row
  static constexpr int RPL = 1024 / RB;     // rows of a wave-wide load
  static constexpr int LPW = QB / RPL / WAVES;   // such loads of a wave in a block
  static constexpr int BLOCK = QB * RB, LSE = WAVES * QB * 4;   // a block in LDS; its lse, a copy to a wave
  static constexpr int LDS = STAGES * (BLOCK + LSE);
  __device__ static constexpr int swz(int r) { return D == 128 ? (r & 15) : ((r >> 1) & 7); }
};
template <int N>
__device__ __forceinline__ void wait_and_sync() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

template <int D, int KG, bool SOURCE>
__global__ __launch_bounds__(64 * WAVES, 3) void paged_mass_ring_kernel(MassParams p) {
  using GM = ManyGeom<D>;
  constexpr int KW = 4, KEYS = 16 * KW * KG, KS = D / 32, NQ = KG;   // NQ: groups of 16 query rows of a block that a wave takes
  typedef Operand<uint16_t, D, true> Op;
  extern __shared__ __align__(1024) char many_smem[];
  __shared__ float s_join[KG < WAVES ? WAVES * 64 : 1];
  const paged_mass_args& a = p.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, g = lane >> 4, G = p.group;
  const int kvh = blockIdx.x % a.n_kv_heads, b = blockIdx.x / a.n_kv_heads;
  int kblk;
  const MassRow row = longest_first<KEYS>(p, b, kvh == 0 && wave == 0, &kblk);
  const int lo = row.lo, n = row.n, M = n * G, Lp = row.Lp, W = a.window;
  const int kb0 = KEYS * kblk, kb = kb0 + 16 * KW * (wave % KG), qw = wave / KG;
  if (n == 0 || kb0 >= row.L || kb0 + KEYS <= row.first) return;
  auto token_of = [&](int r) { return (int)(p.group_inv ? __umulhi((unsigned)r, p.group_inv) : (unsigned)r); };
  // ---- the query rows that see some of the workgroup's keys, and of the wave's
  auto rows_of = [&](int k0, int keys, int* from, int* to) {
    *from = k0 > Lp ? min(k0 - Lp, n) * G : 0;
    *to = W > 0 && k0 >= a.n_sink ? (int)min((long long)M, max(0ll, (long long)(k0 + keys - 1) + W - Lp) * G) : M;
  };
  int wg_from, wg_to, from, to;
  rows_of(kb0, KEYS, &wg_from, &wg_to);
  rows_of(kb, 16 * KW, &from, &to);
  wg_from &= ~(QB - 1);

  const unsigned lds0 = __builtin_amdgcn_readfirstlane((unsigned)(size_t)many_smem);
  // Whole blocks of tokens in a row, whose heads divide a block: a lane's rows lie at constant distances from the block's first (per block no vector instruction but the loads)
  const bool regular = !SOURCE && QB % G == 0 && a.q_stride <= (1 << 24);
  const int block_tokens = QB / G;
  unsigned q_at[GM::LPW], lse_at;
#pragma unroll
  for (int i = 0; i < GM::LPW; ++i) {
    const int in = (GM::LPW * wave + i) * GM::RPL + lane / GM::PPR, j = token_of(in);
    q_at[i] = 2u * (unsigned)(j * (int)min(a.q_stride, (int64_t)1 << 24) + (in - j * G) * D + 8 * ((lane % GM::PPR) ^ GM::swz(in)));
  }
  {
    const int j = token_of(lane);
    lse_at = 4u * (unsigned)(j * a.n_heads + lane - j * G);
  }
  auto request = [&](int r0, int stage) {   // (rows behind the last: that one again, and nothing for its lse)
    if (regular && r0 + QB <= M) {
      const long long t = lo + (long long)(r0 / QB) * block_tokens;   // (r0 is a multiple of QB)
      const uintptr_t qs = (uintptr_t)((const uint16_t*)a.q + t * a.q_stride + kvh * G * D), ls = (uintptr_t)(a.lse + t * a.n_heads + kvh * G);
      const auto uniform = [](uintptr_t x) {
        return (const char*)(((uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32) | (unsigned)__builtin_amdgcn_readfirstlane((int)x));
      };
#pragma unroll
      for (int i = 0; i < GM::LPW; ++i) {
        const unsigned l = lds0 + stage * GM::BLOCK + (GM::LPW * wave + i) * 1024;
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(l), "v"(q_at[i]), "s"(uniform(qs)) : "memory");
      }
      const unsigned l = lds0 + STAGES * GM::BLOCK + stage * GM::LSE + wave * (QB * 4);
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(l), "v"(lse_at), "s"(uniform(ls)) : "memory");
      return;
    }
#pragma unroll
    for (int i = 0; i < GM::LPW; ++i) {
      const int in = (GM::LPW * wave + i) * GM::RPL + lane / GM::PPR, r = min(r0 + in, M - 1), j = token_of(r);
      int t = SOURCE ? a.source[lo + j] : lo + j;
      if (SOURCE && (unsigned)t >= (unsigned)a.n_source) t = 0;
      const uint16_t* at = (const uint16_t*)a.q + t * a.q_stride + (kvh * G + r - j * G) * D + 8 * ((lane % GM::PPR) ^ GM::swz(in));
      const unsigned l = lds0 + stage * GM::BLOCK + (GM::LPW * wave + i) * 1024;
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(l), "v"(at) : "memory");
    }
    const int r = r0 + lane, j = token_of(min(r, M - 1)), h = kvh * G + min(r, M - 1) - j * G;
    int t = SOURCE ? a.source[lo + j] : lo + j;
    if (SOURCE && t != -1 && (unsigned)t >= (unsigned)a.n_source) { atomicOr(p.dev_status, CASCADE_FLAG_PATH); t = -1; }
    const float* at = r < M && t >= 0 ? a.lse + (long long)t * a.n_heads + h : &s_nothing;
    const unsigned l = lds0 + STAGES * GM::BLOCK + stage * GM::LSE + wave * (QB * 4);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(l), "v"(at) : "memory");
  };
  constexpr int LOADS = GM::LPW + 1;
  if (wg_from < wg_to)
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) request(wg_from + i * QB, i);
  Op key[KW];
  const unsigned there = load_keys<Op, uint16_t, KW>(p, row, kvh, kb, key);
  if (!there) to = 0;
  float sum[KW];
#pragma unroll
  for (int kt = 0; kt < KW; ++kt) sum[kt] = 0.f;

  auto block = [&](int r0, auto stage_const) {
    constexpr int ST = decltype(stage_const)::value;
    wait_and_sync<LOADS*(STAGES - 2)>();
    request(r0 + (STAGES - 1) * QB, (ST + STAGES - 1) % STAGES);
    if (r0 + QB <= from || r0 >= to) return;
    const uint16_t* qs = (const uint16_t*)(many_smem + ST * GM::BLOCK);
    float* ls = (float*)(many_smem + STAGES * GM::BLOCK + ST * GM::LSE) + wave * QB;
    int own_at = 8 * (g ^ GM::swz(l16));
    auto operand = [&](Op& q, int qb) {
      if constexpr (D == 128 && KG == 4) asm volatile("" : "+v"(own_at));   // (piece 4 ks + g is one xor away: these addresses, held for every ks, spilled here, and are faster held elsewhere)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) q.x[ks] = *(const bf16x8*)(qs + (16 * qb + l16) * D + (own_at ^ 32 * ks));
    };
    // whether every row sees all of the wave's keys
    const int rows = min(QB, M - r0), x0 = Lp + token_of(r0), x1 = Lp + token_of(r0 + rows - 1);
    const float mine = ls[lane] * LOG2E;   // (the wave's own copy)
    ls[lane] = mine;
    __builtin_amdgcn_wave_barrier();
    const bool all_count = __all(fabsf(mine) < INFINITY), whole = all_count && there == (1u << KW) - 1 && kb + 16 * KW - 1 <= x0 && (W == 0 || x1 - kb < W);
    if (whole) {
      // the products of the next 16 rows stand among the exponentials of these
      Op q[2];
      f32x4 w[2][KW];
      operand(q[0], NQ * qw);
      if (NQ > 1) operand(q[1], NQ * qw + 1);
#pragma unroll
      for (int kt = 0; kt < KW; ++kt) w[0][kt] = Op::product(q[0], key[kt]);
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
        const f32x4 lse = *(const f32x4*)(ls + 16 * (NQ * qw + i) + 4 * g);
        if (i + 2 < NQ) operand(q[i & 1], NQ * qw + i + 2);
#pragma unroll
        for (int kt = 0; kt < KW; ++kt) {
          if (i + 1 < NQ) w[(i + 1) & 1][kt] = Op::product(q[(i + 1) & 1], key[kt]);
          f32x4 e;
#pragma unroll
          for (int c = 0; c < 4; ++c) e[c] = fast_exp2(fmaf(w[i & 1][kt][c], p.scale_log2e, -lse[c]));
          sum[kt] += (e[0] + e[1]) + (e[2] + e[3]);
        }
      }
    } else {
#pragma unroll 1
      for (int i = 0; i < NQ; ++i) {
        const int qb = NQ * qw + i, r = r0 + 16 * qb + 4 * g;
        if (r0 + 16 * qb >= M) break;
        const int x_lo = Lp + token_of(r0 + 16 * qb), x_hi = Lp + token_of(min(r0 + 16 * qb + 15, M - 1));   // positions of these rows
        if (kb > x_hi) continue;
        Op q;
        operand(q, qb);
        const f32x4 lse = *(const f32x4*)(ls + 16 * qb + 4 * g);
        int at[4];   // positions; -1: the row counts nothing
#pragma unroll
        for (int c = 0; c < 4; ++c) at[c] = fabsf(lse[c]) < INFINITY ? Lp + token_of(r + c) : -1;
#pragma unroll
        for (int kt = 0; kt < KW; ++kt) {
          const int y0 = kb + 16 * kt, y = y0 + l16;
          if (y0 > x_hi || !((there >> kt) & 1)) continue;   // none of them sees any of these keys
          const f32x4 w = Op::product(q, key[kt]);
          f32x4 e;
#pragma unroll
          for (int c = 0; c < 4; ++c) e[c] = fast_exp2(fmaf(w[c], p.scale_log2e, -lse[c]));
          if (!all_count || y0 + 15 > x_lo || (W > 0 && x_hi - y0 >= W))
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const bool seen = y <= at[c] && (W == 0 || at[c] - y < W || y < a.n_sink);
              e[c] = seen ? e[c] : 0.f;
            }
          sum[kt] += (e[0] + e[1]) + (e[2] + e[3]);
        }
      }
    }
  };
  for (int r0 = wg_from; r0 < wg_to; r0 += STAGES * QB) {
    block(r0, std::integral_constant<int, 0>{});
    if (r0 + QB < wg_to) block(r0 + QB, std::integral_constant<int, 1>{});
    if (r0 + 2 * QB < wg_to) block(r0 + 2 * QB, std::integral_constant<int, 2>{});
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the loads that nothing uses must not outlive the workgroup's LDS
  if constexpr (KG < WAVES) {   // the waves that share keys join, in order
#pragma unroll
    for (int kt = 0; kt < KW; ++kt) {
      const float all = rows4_sum(sum[kt]);
      if (g == 0) s_join[wave * 64 + 16 * kt + l16] = all;
    }
    __syncthreads();
    if (qw > 0) return;
#pragma unroll
    for (int kt = 0; kt < KW; ++kt) {
      sum[kt] = 0.f;
      if (g == 0)
#pragma unroll
        for (int w = 0; w < WAVES / KG; ++w) sum[kt] += s_join[(wave + KG * w) * 64 + 16 * kt + l16];
    }
  }
  write_sums<KW>(p, row, kvh, kb, sum);
}

template <int D, int KW, bool VEC>
hipError_t launch_k(cascade_ctx* ctx, MassParams& p) {
  constexpr int KEYS = 16 * KW * WAVES;
  p.key_blocks = (p.a.max_seq_len + KEYS - 1) / KEYS;
  const int64_t blocks = (int64_t)p.a.n_rows * p.a.n_kv_heads * p.key_blocks;
  KernelTimer t(ctx, CASCADE_K_MASS);
  CASCADE_TIMED_LAUNCH(t, (paged_mass_kernel<D, KW, VEC>), dim3((unsigned)blocks), dim3(64 * WAVES), 0, ctx->stream, p);
  return hipGetLastError();
}
template <auto KERNEL>
hipError_t allow_lds(int bytes, int device) {   // more than a launch may have by default: said once per kernel and device
  static std::atomic<unsigned long long> done{0};
  const unsigned long long bit = 1ull << (device & 63);
  if (device < 64 && (done.load(std::memory_order_relaxed) & bit)) return hipSuccess;
  const hipError_t e = hipFuncSetAttribute((const void*)KERNEL, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == hipSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}
template <int D, int KG, bool SOURCE>
hipError_t launch_ring_k(cascade_ctx* ctx, MassParams& p) {
  constexpr auto kern = paged_mass_ring_kernel<D, KG, SOURCE>;
  const hipError_t e = allow_lds<kern>(ManyGeom<D>::LDS, ctx->device);
  if (e != hipSuccess) return e;
  p.key_blocks = (p.a.max_seq_len + 64 * KG - 1) / (64 * KG);
  KernelTimer t(ctx, CASCADE_K_MASS);
  CASCADE_TIMED_LAUNCH(t, kern, dim3((unsigned)((int64_t)p.a.n_rows * p.a.n_kv_heads * p.key_blocks)), dim3(64 * WAVES), ManyGeom<D>::LDS, ctx->stream, p);
  return hipGetLastError();
}
template <int D, bool SOURCE>
hipError_t launch_ring(cascade_ctx* ctx, MassParams& p) {
  // Wider workgroups read the queries less often, narrower ones fill the chip.  With 256, 128 and 64 positions, prompts of 8 kv heads of 4: 16 rows x 1000 tokens behind 3000 (2048
  // workgroups of 256 positions) 548, 581, 781 us; 32 x 100 behind 1000 (1280) 58, 68, 103; 16 x 1000 behind 1000 (1024) 273, 279, 347; rows of 500 to 1000 behind up to 2000 (768)
  // 166, 120, 128; 8 x 300 behind 1000 (384) 74, 50, 54; 8 x 100 behind 500 (192) 24, 21, 22, with head_dim 64 (384) 64, 42, 37.
  const int64_t blocks = (int64_t)p.a.n_rows * p.a.n_kv_heads * ((p.a.max_seq_len + 255) / 256);
  if (blocks >= 4 * ctx->n_cu) return launch_ring_k<D, 4, SOURCE>(ctx, p);
  return blocks >= ctx->n_cu ? launch_ring_k<D, 2, SOURCE>(ctx, p) : launch_ring_k<D, 1, SOURCE>(ctx, p);
}
template <int D, int NB>
hipError_t launch_few_k(cascade_ctx* ctx, MassParams& p) {
  const int64_t tiles = (int64_t)p.a.n_rows * p.a.n_kv_heads * ((p.a.max_seq_len + 255) / 256);
  // Two tiles to a wave spare queries and workgroups, four leave rows of different lengths ends of their own: one token of 64 rows of 2145 keys 66, 62, 61 us with one, two, four; of 90 to 4200
  // keys 75, 71, 78; paths of 11 tokens, 16 rows x 32 heads of 600 to 2356 keys 53, 51, 49.
  p.wave_tiles = tiles >= 8 * ctx->n_cu ? 2 : 1;
  p.key_blocks = (p.a.max_seq_len + 256 * p.wave_tiles - 1) / (256 * p.wave_tiles);
  const dim3 grid((unsigned)((int64_t)p.a.n_rows * p.a.n_kv_heads * p.key_blocks));
  // Of few rows the workgroups that have keys come one behind the other, the others last; of others the last tiles of all rows come last.  The second way and the first, one token, 8 kv heads of 4,
  // us: rows of 100 to 16000 keys: 3 rows 14.1, 12.3; 4 19.9, 12.2; 8 41.0, 25.5; 16 66.6, 56.0; of 90 to 4200: 4 9.3, 9.1; 8 11.8, 9.9; 16 21.0, 19.1; all of 2145: 4 8.6, 9.2; 8 11.1, 11.6;
  // 16 18.3, 19.4 (32 kv heads: of 90 to 4200 8 27.7, 28.1; 16 74.6, 75.4; of 2145 8 33.8, 38.3; 16 64.9, 68.4; paths of 16 rows 45.4, 45.6).  Two rows leave nothing to gain (6.6, 6.9; paths 9.7,
  // 10.2).  Of 17 to 64 rows it is 5 to 17 % less where they differ (32: 38.8, 32.1; 64: 70.7, 65.6) and 2 to 10 % more where they do not (32: 35.5, 39.2; 64: 62.6, 66.6), as images
  // that began together: neither is the rule for them, and the search is left out
  const bool dealt = p.a.n_rows > 2 && p.a.n_rows <= 16;
  KernelTimer t(ctx, CASCADE_K_MASS);
  if (dealt) CASCADE_TIMED_LAUNCH(t, (paged_mass_few_kernel<D, NB, true>), grid, dim3(64 * WAVES), 0, ctx->stream, p);
  else CASCADE_TIMED_LAUNCH(t, (paged_mass_few_kernel<D, NB, false>), grid, dim3(64 * WAVES), 0, ctx->stream, p);
  return hipGetLastError();
}
template <int D>
hipError_t launch_bf16(cascade_ctx* ctx, MassParams& p) {
  // 64 rows of 8 tokens x 4 heads behind 2000: 60 us straight from memory, 72 through the ring (the stream of keys bounds both); 16 rows of 16 x 4: 22.4 both, head_dim 64 15.2 and 12.8
  const int64_t rows = (int64_t)p.a.max_new * p.group;
  if (rows <= 32) return rows <= 16 ? launch_few_k<D, 1>(ctx, p) : launch_few_k<D, 2>(ctx, p);
  return p.a.source ? launch_ring<D, true>(ctx, p) : launch_ring<D, false>(ctx, p);
}
template <bool VEC>
hipError_t launch_f32(cascade_ctx* ctx, MassParams& p) {
  if (p.a.head_dim <= 64) return launch_k<64, 4, VEC>(ctx, p);
  return p.a.head_dim <= 128 ? launch_k<128, 2, VEC>(ctx, p) : launch_k<256, 1, VEC>(ctx, p);
}

}  // namespace

hipError_t launch_paged_mass(cascade_ctx* ctx, const paged_mass_args* a) {
  MassParams p;
  p.a = *a;
  p.group = a->n_heads / a->n_kv_heads;
  p.most_len = (int)std::min<int64_t>({a->max_seq_len, (int64_t)a->table_width * a->page_size, a->mass_cap});
  p.scale_log2e = (a->scale != 0.f ? a->scale : 1.f / sqrtf((float)a->head_dim)) * LOG2E;
  p.dev_status = ctx->dev_status;
  p.group_inv = p.group == 1 ? 0u : (unsigned)((1ull << 32) / p.group + 1);
  if (a->dtype == CASCADE_BF16) return a->head_dim == 128 ? launch_bf16<128>(ctx, p) : launch_bf16<64>(ctx, p);
  // 16 bytes at a time where everything lies on such boundaries, otherwise element by element
  const bool vec = ((a->head_dim | a->q_stride | a->stride_page | a->stride_head | a->stride_pos) % 4) == 0 && (((uintptr_t)a->q | (uintptr_t)a->k_pages) & 15) == 0;
  return vec ? launch_f32<true>(ctx, p) : launch_f32<false>(ctx, p);
}
