// paged_evict kernels for gfx950: rows over their budget give up the positions that gathered the least attention weight, in every layer and kv head their own.
//
// Attention over a cache does not ask in which order keys lie, so nothing is compacted: a kept position moves only if it lies behind the places that remain, and it moves into a
// place that was given up.  With N of L positions left that is at most L - N of them, whatever N is, where closing the gaps would move nearly all N.  The last n_recent positions stay in
// order, so that the next call finds the newest ones at the end again: if any position goes, all of these move too.
//
// What stays (the N-th largest weight by radix selection, then the lists of places and of positions that go there) is found by every workgroup that shares a unit's moves, with the
// list in its LDS; only rows of more than 16384 positions take two launches, with lists in memory.  Bound by the moves, scattered keys of 256 bytes, where there are many: 30 layers
// of 8 rows x 8 kv heads, 1289 to 2356 positions down to 1024 (1.2 GB read and written) 279 us, 4.4 TB/s, of which choosing takes 20; a layer of two rows, 500 positions down to 312,
// 12 us, one workgroup's chain.  Where n_recent is more than what goes, the recent ones are what a call costs: rows of 1024 and a few more down to 1024 with 256 recent, 30 layers of 8 rows x 8
// kv heads: one more 127 us (at the rate of a large copy 106), 16 more 133 (111), 64 more 149 (129); head_dim 64 79 (54), 84 (57), 92 (66); a layer of two rows x 8 kv heads 13 to 14 (1), x 32
// heads 18.5 (4).
#include <algorithm>

#include "common.h"

namespace {

typedef unsigned long long u64;
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr int THREADS = 256;   // of a workgroup that moves

struct EvictParams {
  paged_evict_args a;
  int most_len;     // the longest row that the bounds allow
  int units;        // (layer, row, kv head)
  int most_moves;   // pairs that a unit's list has room for
  int* dev_status;
  int2* list;       // [units][1 + most_moves]: how many of the first and the second kind, then pairs {place, position that goes there}, the second kind from the list's end
  int pieces;       // 16-byte pieces of a key
  int splits;       // workgroups that share a unit's moves of keys (and of values)
  unsigned page16_inv;   // floor(2^32 / (page_size / 16)) + 1: a position's page as a high product (positions / 16 stay below 2^26); 0 for pages of 16
};
__device__ __forceinline__ int page_index(const EvictParams& p, int y) {
  return p.page16_inv ? (int)__umulhi((unsigned)y >> 4, p.page16_inv) : y >> 4;
}

// ---- what remains of a row
struct RowPlan {
  int L, f, r, N;   // positions, those at the front and at the end that stay anyhow, what remains
  bool ok;
};
__device__ __forceinline__ RowPlan plan_row(const EvictParams& p, int s) {
  const paged_evict_args& a = p.a;
  RowPlan w;
  w.L = a.seq_len[s];
  w.ok = w.L >= 0 && w.L <= p.most_len;
  const int L = w.ok ? w.L : 0;
  w.f = min(a.n_first ? max(a.n_first[s], 0) : 0, L);
  w.r = min(a.n_recent, L - w.f);
  w.N = max(min(max(a.budget[s], 0), L), w.f + w.r);
  return w;
}
__device__ __forceinline__ int pages_of(const EvictParams& p, int positions) { return (positions + p.a.page_size - 1) / p.a.page_size; }
__device__ __forceinline__ int pages_back(const EvictParams& p, const RowPlan& w) { return w.ok ? pages_of(p, w.L) - pages_of(p, w.N) : 0; }

// larger weights have larger numbers; zeros of both signs the same; NaN the least
__device__ __forceinline__ unsigned rank_of(float v) {
  if (!(v == v)) return 0u;
  const unsigned u = __float_as_uint(v + 0.f);
  return u >> 31 ? ~u : u | 0x80000000u;
}

// The lengths, the pages that go back and their list: a wave to a row, behind the units' workgroups.
__device__ __forceinline__ void give_back(const EvictParams& p, int s) {
  const paged_evict_args& a = p.a;
  const int lane = threadIdx.x & 63;
  if (s >= a.n_rows) return;
  const int listed = a.free_count[0], base = min(max(listed, 0), a.free_capacity);
  int before = 0;   // entries of the rows in front
  for (int r0 = 0; r0 < s; r0 += 64) {
    int n = 0;
    if (r0 + lane < s) n = pages_back(p, plan_row(p, r0 + lane));
    before += wave_sum_i(n);
  }
  const RowPlan w = plan_row(p, s);
  const int from = w.ok ? pages_of(p, w.N) : 0, n = pages_back(p, w), room = max(min(n, a.free_capacity - base - before), 0);
  int flag = w.ok ? 0 : CASCADE_FLAG_CAPACITY;
  if (room < n || listed != base) flag |= CASCADE_FLAG_PAGE;
  for (int i = lane; i < room; i += 64) {
    const int page = a.block_table[s * a.table_stride + from + i];
    if ((unsigned)page >= (unsigned)a.n_pages) flag |= CASCADE_FLAG_PAGE;
    a.free_pages[base + before + i] = page;
  }
  if (flag) atomicOr(p.dev_status, flag);
  if (lane == 0) {
    a.seq_len_out[s] = w.ok ? w.N : w.L;
    if (a.dropped) a.dropped[s] = w.ok ? w.L - w.N : 0;
    if (s == a.n_rows - 1) a.free_count_out[0] = min(base + before + n, a.free_capacity);
  }
}

// What stays of a (layer, row, kv head): the pairs of its list, which lies in LDS or in the workspace, and, by one workgroup (`lead`), its weights; at: where these begin.
// Returns how many pairs there are of the first and of the second kind.
// The weight that decides is found by radix selection of the ranks, 12, 10 and 10 bits: with the whole exponent and three bits of the fraction in the first digit, weights that spread
// over some octaves spread over the bins.  Once no more than a wave of candidates begin like the one that decides they are ranked against each other, by weight and position, and the
// other digits are left out.  A thread holds HELD consecutive positions in registers (rows of up to HELD NT positions are read once), so one scan over the threads' counts gives everything
// its place in the order of positions.
template <int NT, int HELD>
__device__ __forceinline__ int2 decide(const EvictParams& p, const RowPlan& w, long long at, bool lead, int2* pairs, int cap) {
  constexpr int NW = NT / 64, BINS = 4096, WORDS = BINS + BINS / 16, SPAN = HELD * NT;
  typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));   // (such loads need the boundary of a word)
  const paged_evict_args& a = p.a;
  __shared__ int s_bin[WORDS];   // (a word between runs of 16: threads that each go through a run meet in no bank)
  __shared__ int s_sum[2][NW];
  __shared__ int s_digit, s_left, s_same, s_count;
  __shared__ int2 s_near[64];    // candidates: rank, position
  auto bin = [](int i) { return i + (i >> 4); };
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  for (int i = tid; i < WORDS; i += NT) s_bin[i] = 0;
  if (tid == 0) s_count = 0;
  const float* mass = a.mass + at;
  float* out = a.mass_out + at;
  const int L = w.L, f = w.f, m = w.N - w.r, end = L - w.r, keep = m - f;   // `keep` of f .. end - 1; places f .. m - 1
  unsigned u[HELD];
  const int spans = (end - f + SPAN - 1) / SPAN;
  auto first_of = [&](int span) { return f + span * SPAN + HELD * tid; };
  auto load = [&](int span) {
    const int y0 = first_of(span);
#pragma unroll
    for (int i = 0; i < HELD; i += 4) {
      f32x4 v = {0.f, 0.f, 0.f, 0.f};
      if (y0 + i + 3 < end) v = *(const f32x4_any*)(mass + y0 + i);
      else
#pragma unroll
        for (int c = 0; c < 3; ++c)
          if (y0 + i + c < end) v[c] = mass[y0 + i + c];
#pragma unroll
      for (int c = 0; c < 4; ++c) u[i + c] = rank_of(v[c]);
    }
  };
  if (spans == 1) load(0);
  // (places that are given up get the weights that come there below)
  if (lead) {
    for (int y = tid; y < m; y += NT) out[y] = mass[y];
    for (int y = tid; y < w.r; y += NT) out[m + y] = mass[end + y];
  }
  // what is in front of this thread's counts, and their sum; two buffers in turn, so that one barrier does
  int turn = 0;
  auto before_me = [&](int v, int* total) {
    const int incl = wave_scan_incl_i(v);
    if (lane == 63) s_sum[turn][wave] = incl;
    __syncthreads();
    int base = 0, all = 0;
#pragma unroll
    for (int x = 0; x < NW; ++x) {
      const int n = s_sum[turn][x];
      base += x < wave ? n : 0;
      all += n;
    }
    turn ^= 1;
    *total = all;
    return base + incl - v;
  };
  // ---- what is kept: ranks above `least`, and of those equal to it the positions up to `last`; (rank >> shift) is compared
  unsigned least = 0xffffffffu;
  int last = -1, shift = 0, left = 0;
  bool by_order = false;   // of equal ones the first `left`, as they come
  if (keep > 0) {
    least = 0;
    left = keep;
    last = 0x7fffffff;
    for (int digit = 0; digit < 3; ++digit) {
      const int bits = digit == 0 ? 12 : 10, bins = 1 << bits;
      shift = digit == 0 ? 20 : (digit == 1 ? 10 : 0);
      if (digit > 0)
        for (int i = tid; i < bin(bins); i += NT) s_bin[i] = 0;
      __syncthreads();
      for (int span = 0; span < spans; ++span) {
        if (spans > 1) load(span);
        const int y0 = first_of(span);
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
          const bool in = y0 + i < end && (digit == 0 || u[i] >> (shift + bits) == least);
          if (in) atomicAdd(&s_bin[bin((u[i] >> shift) & (bins - 1))], 1);
        }
      }
      __syncthreads();
      // from the largest digit down, some bins to a thread
      const int each = bins / NT > 0 ? bins / NT : 1;
      int mine = 0;
      if (tid * each < bins)
        for (int i = 0; i < each; ++i) mine += s_bin[bin(bins - 1 - (tid * each + i))];
      int total;
      int before = before_me(mine, &total);
      if (before < left && before + mine >= left) {   // one thread's
        int d = bins - 1 - tid * each;
        while (before + s_bin[bin(d)] < left) before += s_bin[bin(d--)];
        s_digit = d;
        s_left = left - before;
        s_same = s_bin[bin(d)];
      }
      __syncthreads();
      least = (digit == 0 ? 0u : least << bits) | (unsigned)s_digit;
      left = s_left;
      const int same = s_same;
      if (left == same) break;   // all that begin so are kept
      if (same <= 64) {
        for (int span = 0; span < spans; ++span) {
          if (spans > 1) load(span);
          const int y0 = first_of(span);
#pragma unroll
          for (int i = 0; i < HELD; ++i)
            if (y0 + i < end && u[i] >> shift == least) s_near[atomicAdd(&s_count, 1)] = int2{(int)u[i], y0 + i};
        }
        __syncthreads();
        const int2 c = lane < same ? s_near[lane] : int2{0, 0x7fffffff};   // every wave for itself
        int ahead = 0;
        for (int j = 0; j < same; ++j) {
          const unsigned other = (unsigned)__builtin_amdgcn_readlane(c.x, j);
          const int where = __builtin_amdgcn_readlane(c.y, j);
          ahead += other > (unsigned)c.x || (other == (unsigned)c.x && where < c.y) ? 1 : 0;
        }
        const int who = __ffsll((long long)__ballot(lane < same && ahead == left - 1)) - 1;   // (positions differ, so do the ranks)
        least = (unsigned)__builtin_amdgcn_readlane(c.x, who);
        last = __builtin_amdgcn_readlane(c.y, who);
        shift = 0;
        break;
      }
      by_order = digit == 2;
      __syncthreads();   // the bins have been looked at
    }
  }
  const bool in_order = w.r > L - w.N;   // the last ones move onto places of their own: the other kernel takes them one run after the other
  int ties = 0, holes = 0, fills = 0, plain = 0;   // so far
  for (int span = 0; span < spans; ++span) {
    if (spans > 1) load(span);
    const int y0 = first_of(span);
    unsigned kept = 0;
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
      const unsigned x = u[i] >> shift;
      if (y0 + i < end && keep > 0 && (x > least || (x == least && y0 + i <= last))) kept |= 1u << i;
    }
    if (by_order) {
      unsigned tie = 0;
#pragma unroll
      for (int i = 0; i < HELD; ++i)
        if (((kept >> i) & 1) && u[i] == least) tie |= 1u << i;
      int all;
      int at_tie = ties + before_me(__popc(tie), &all);
#pragma unroll
      for (int i = 0; i < HELD; ++i)
        if ((tie >> i) & 1) {
          if (at_tie >= left) kept &= ~(1u << i);
          ++at_tie;
        }
      ties += all;
    }
    // three kinds of positions that the lists are made of: places given up below m; kept positions from m on; and, where the last ones come from behind all places, those of
    // their places that nothing has to leave first.  Bits of this thread's positions:
    auto bits_below = [&](int limit) { return limit <= y0 ? 0u : (limit - y0 >= HELD ? (1u << HELD) - 1u : (1u << (limit - y0)) - 1u); };
    const unsigned there = bits_below(end), low = bits_below(m);
    const unsigned hole = low & ~kept, fill = kept & ~low, free = in_order ? 0u : there & ~low & ~kept & bits_below(w.N);
    int all;   // (at most 2^14 of each in a span)
    const int at_both = before_me(__popc(hole) | __popc(fill) << 16, &all);
    int h = holes + (at_both & 0xffff), q = fills + (at_both >> 16);
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
      if ((hole >> i) & 1) pairs[h++].x = y0 + i;
      if ((fill >> i) & 1) pairs[q++].y = y0 + i;
    }
    holes += all & 0xffff;
    fills += all >> 16;
    if (!in_order) {
      int n_free;
      int x = plain + before_me(__popc(free), &n_free);
#pragma unroll
      for (int i = 0; i < HELD; ++i)
        if ((free >> i) & 1) pairs[cap - 1 - x++] = int2{y0 + i, y0 + i + L - w.N};
      plain += n_free;
    }
  }
  __syncthreads();
  if (lead)
    for (int i = tid; i < holes; i += NT) {
      const int2 pair = pairs[i];
      out[pair.x] = mass[pair.y];
    }
  return int2{holes, plain};
}

// The moves of keys or of values of a unit, this workgroup's share of them (`mine` of `splits`).
// Pairs of the first kind bring a kept position to a place that was given up.  Where it stood may be a place of the last n_recent: then the thread that has taken the old
// key away brings the new one, and no other has anything to do with it.  The second kind are the other places of the last ones.  So nobody waits for anybody.
// Only if more of the last ones move than positions go (n_recent > L - N), some move onto places of others of them: then the pairs go first, in workgroups that share the
// 16-byte pieces of all keys - whole lines of 128 bytes, so at keys of 128 bytes one workgroup moves all keys of a unit and one all values -, and the last ones follow in runs, each in
// registers before its places are written; every later run comes from behind those.
template <int NT>
__device__ __forceinline__ void move(const EvictParams& p, const RowPlan& w, int layer, int s, int kvh, bool values, int mine, int splits, const int2* list, int cap, int2 counts) {
  const paged_evict_args& a = p.a;
  const int tid = threadIdx.x;
  const int gone = w.L - w.N;
  const bool in_order = w.r > gone;
  int pieces = p.pieces, slice = 0;
  if (in_order) {   // whole lines of 128 bytes
    const int slices = p.pieces % 8 == 0 ? min(splits, p.pieces / 8) : 1, per = p.pieces / 8 / max(slices, 1) * 8;
    if (slices > 1 && p.pieces % (8 * slices) == 0) {
      if (mine >= slices) return;
      pieces = per;
      slice = mine * per;
    } else if (mine > 0) {
      return;
    }
    splits = 1;
    mine = 0;
  }
  const long long esize = a.dtype == CASCADE_BF16 ? 2 : 4, stride_page = a.stride_page * esize, stride_pos = a.stride_pos * esize;
  const int each = NT / pieces, entry = tid / pieces, piece = tid - entry * pieces;   // keys that the workgroup moves at a time; this thread's
  if (each == 0) return;   // (the host asks for no more pieces than threads)
  const bool idle = entry >= each;
  char* const base = (char*)(values ? a.v_pages : a.k_pages) + (layer * a.stride_layer + kvh * a.stride_head) * esize + 16 * (slice + piece);
  const int32_t* table = a.block_table + s * a.table_stride;
  auto at = [&](int page, int y) {   // (outside the pool: its first page)
    return base + ((unsigned)page < (unsigned)a.n_pages ? page : 0) * stride_page + (y - page_index(p, y) * a.page_size) * stride_pos;
  };
  auto good = [&](int from, int to) {
    const bool ok = (unsigned)from < (unsigned)a.n_pages && (unsigned)to < (unsigned)a.n_pages;
    if (!ok) atomicOr(p.dev_status, CASCADE_FLAG_PAGE);
    return ok;
  };
  constexpr int U = 4;
  const int n = counts.x + (in_order ? 0 : counts.y), step = splits * U * each;
  // (Loads without conditions, so that a round's are on their way together: behind the last pair that one again, outside the pool its first page; what must not be written is not.)
  if (!idle)
    for (int i0 = mine * U * each + entry; i0 < n; i0 += step) {
      u32x4 x[U];
      int2 pair[U];
      int from_page[U], to_page[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = min(i0 + u * each, n - 1);
        pair[u] = list[i < counts.x ? i : cap - 1 - (i - counts.x)];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        from_page[u] = table[page_index(p, pair[u].y)];
        to_page[u] = table[page_index(p, pair[u].x)];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) x[u] = *(const u32x4*)at(from_page[u], pair[u].y);
      bool chain = false;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i0 + u * each < n && good(from_page[u], to_page[u])) *(u32x4*)at(to_page[u], pair[u].x) = x[u];
        chain |= !in_order && pair[u].y < w.N;
      }
      if (chain)   // places that these keys have left and that the last ones come to
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (i0 + u * each < n && pair[u].y < w.N) {
            const int page = table[page_index(p, pair[u].y + gone)];
            if (good(from_page[u], page)) *(u32x4*)at(from_page[u], pair[u].y) = *(const u32x4*)at(page, pair[u].y + gone);
          }
    }
  if (!in_order) return;
  __syncthreads();
  const int m = w.N - w.r, end = w.L - w.r;
  for (int i0 = 0; i0 < w.r; i0 += U * each) {
    u32x4 x[U];
    int from_page[U], to_page[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = min(i0 + u * each + entry, w.r - 1);
      from_page[u] = table[page_index(p, end + i)];
      to_page[u] = table[page_index(p, m + i)];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = *(const u32x4*)at(from_page[u], end + min(i0 + u * each + entry, w.r - 1));
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the run is in registers
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * each + entry;
      if (!idle && i < w.r && good(from_page[u], to_page[u])) *(u32x4*)at(to_page[u], m + i) = x[u];
    }
  }
}

struct Unit {
  int kvh, s, layer;
  long long mass;   // where its weights begin
};
__device__ __forceinline__ Unit unit_of(const EvictParams& p, int unit) {
  const paged_evict_args& a = p.a;
  const int kvh = unit % a.n_kv_heads, sl = unit / a.n_kv_heads, s = sl % a.n_rows, layer = sl / a.n_rows;
  return Unit{kvh, s, layer, layer * a.mass_stride_layer + s * a.mass_stride_row + kvh * a.mass_stride_head};
}
__device__ __forceinline__ void copy_weights(const EvictParams& p, long long at, int n, int threads) {
  for (int y = threadIdx.x; y < n; y += threads) p.a.mass_out[at + y] = p.a.mass[at + y];
}

// Rows whose list fits in LDS, all in one launch: the workgroups that share a unit's moves each find out by themselves what stays.
template <int NT, int HELD>
__global__ __launch_bounds__(NT, 4) void evict_kernel(EvictParams p) {
  __shared__ int2 s_pairs[NT * HELD / 2];
  if ((int)blockIdx.x >= p.units * p.splits) {
    give_back(p, ((int)blockIdx.x - p.units * p.splits) * (NT / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
    return;
  }
  const int split = blockIdx.x % p.splits;
  const Unit unit = unit_of(p, blockIdx.x / p.splits);
  const RowPlan w = plan_row(p, unit.s);
  if (!w.ok || w.N >= w.L) {
    if (w.ok && split == 0) copy_weights(p, unit.mass, w.L, NT);
    return;
  }
  const int2 counts = decide<NT, HELD>(p, w, unit.mass, split == 0, s_pairs, NT * HELD / 2);
  // keys by the even workgroups, values by the odd ones; one alone does both
  const int shares = max(p.splits >> 1, 1);
#pragma unroll 1
  for (int v = p.splits > 1 ? split & 1 : 0; v < 2; v += p.splits > 1 ? 2 : 1)
    move<NT>(p, w, unit.layer, unit.s, unit.kvh, v, p.splits > 1 ? split >> 1 : 0, shares, s_pairs, NT * HELD / 2, counts);
}

// Longer rows: the lists go through the workspace, {counts} and the pairs of each unit.
constexpr int LONG_THREADS = 1024, LONG_HELD = 16;
__global__ __launch_bounds__(LONG_THREADS) void evict_stay_kernel(EvictParams p) {
  if ((int)blockIdx.x >= p.units) {
    give_back(p, ((int)blockIdx.x - p.units) * (LONG_THREADS / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
    return;
  }
  const Unit unit = unit_of(p, blockIdx.x);
  const RowPlan w = plan_row(p, unit.s);
  int2* list = p.list + (long long)blockIdx.x * (1 + p.most_moves);
  if (!w.ok || w.N >= w.L) {
    if (w.ok) copy_weights(p, unit.mass, w.L, LONG_THREADS);
    return;
  }
  const int2 counts = decide<LONG_THREADS, LONG_HELD>(p, w, unit.mass, true, list + 1, p.most_moves);
  if (threadIdx.x == 0) list[0] = counts;
}
__global__ __launch_bounds__(THREADS) void evict_move_kernel(EvictParams p) {
  const int split = blockIdx.x % p.splits, b = blockIdx.x / p.splits;
  const Unit unit = unit_of(p, b >> 1);
  const int2* list = p.list + (long long)(b >> 1) * (1 + p.most_moves);
  const RowPlan w = plan_row(p, unit.s);
  if (!w.ok || w.N >= w.L) return;
  move<THREADS>(p, w, unit.layer, unit.s, unit.kvh, b & 1, split, p.splits, list + 1, p.most_moves, list[0]);
}

int most_moves(const paged_evict_args* a) { return a->max_seq_len / 2; }   // as many places as positions: at most half of them together

constexpr int MOST_LOCAL = 1024 * 16;   // positions of a row whose list fits in LDS

}  // namespace

int64_t plan_paged_evict(const paged_evict_args* a) {
  if (a->max_seq_len <= MOST_LOCAL) return 0;
  return (int64_t)a->n_layers * a->n_rows * a->n_kv_heads * (1 + most_moves(a)) * (int64_t)sizeof(int2);
}

hipError_t launch_paged_evict(cascade_ctx* ctx, const paged_evict_args* a) {
  EvictParams p;
  p.a = *a;
  p.most_len = (int)std::min<int64_t>({a->max_seq_len, (int64_t)a->table_width * a->page_size, a->mass_cap});
  p.units = a->n_layers * a->n_rows * a->n_kv_heads;
  p.most_moves = most_moves(a);
  p.dev_status = ctx->dev_status;
  p.list = (int2*)a->workspace;
  p.pieces = a->head_dim * (a->dtype == CASCADE_BF16 ? 2 : 4) / 16;
  const int page16 = a->page_size / 16;
  p.page16_inv = page16 == 1 ? 0u : (unsigned)((1ull << 32) / page16 + 1);
  auto waves_of_rows = [&](int nt) { return (a->n_rows + nt / 64 - 1) / (nt / 64); };
  if (a->max_seq_len <= MOST_LOCAL) {
    auto run = [&](auto kernel, int nt, int per_cu) {
      // an even number of workgroups to a unit, as many as the chip holds at a time, with 64 keys to move at least
      const int64_t want = std::min<int64_t>((int64_t)per_cu * ctx->n_cu / p.units, 2 * ((p.most_moves + 63) / 64));
      p.splits = want < 2 ? 1 : (int)(want / 2 * 2);
      KernelTimer t(ctx, CASCADE_K_EVICT);
      CASCADE_TIMED_LAUNCH(t, kernel, dim3((unsigned)(p.units * p.splits + waves_of_rows(nt))), dim3(nt), 0, ctx->stream, p);
      return hipGetLastError();
    };
    if (a->max_seq_len <= 4 * 256) return run(evict_kernel<256, 4>, 256, 4);
    if (a->max_seq_len <= 8 * 512) return run(evict_kernel<512, 8>, 512, 2);
    return run(evict_kernel<1024, 16>, 1024, 1);
  }
  {
    KernelTimer t(ctx, CASCADE_K_EVICT);
    CASCADE_TIMED_LAUNCH(t, evict_stay_kernel, dim3((unsigned)(p.units + waves_of_rows(LONG_THREADS))), dim3(LONG_THREADS), 0, ctx->stream, p);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // eight workgroups to a compute unit, 64 keys to each
  const int64_t want = std::min<int64_t>(8 * ctx->n_cu / (2 * p.units) + 1, (p.most_moves + 63) / 64);
  p.splits = (int)std::max<int64_t>(want, 1);
  KernelTimer t(ctx, CASCADE_K_EVICT_MOVE);
  CASCADE_TIMED_LAUNCH(t, evict_move_kernel, dim3((unsigned)(p.units * 2 * p.splits)), dim3(THREADS), 0, ctx->stream, p);
  return hipGetLastError();
}
