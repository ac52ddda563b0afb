// paged_evict kernels for gfx950: rows over their budget give up the positions that gathered the least attention weight, in every layer and kv head their own.
//
// Attention over a cache does not ask in which order keys lie, so nothing is compacted: a kept position moves only if it lies behind the places that remain, and it moves into a
// place that was given up.  With N of L positions left that is at most (L - N) rows of keys and values, whatever N is, where closing the gaps would move nearly all N.  Only the
// last n_recent positions stay in order, so that the next call finds the newest ones at the end again.
//
// Two launches: what stays (the N-th largest weight by radix selection, then the lists of places and of positions that go there), and the moves.
#include <algorithm>

#include "common.h"

namespace {

typedef unsigned long long u64;
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr int THREADS = 256, PER = 4, STRIP = THREADS * PER;   // positions that a workgroup ranks at a time, four to a thread

struct EvictParams {
  paged_evict_args a;
  int most_len;     // the longest row that the bounds allow
  int units;        // (layer, row, kv head)
  int most_moves;   // pairs that a unit's list has room for
  int* dev_status;
  int2* list;       // [units][1 + most_moves]: {number of pairs, 0}, then {place, position that goes there}
  int pieces, slices;   // 16-byte pieces of a key; workgroups that share them
};

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

// inclusive sum over the workgroup's threads, and the total
__device__ __forceinline__ int block_scan(int* s_wave, int v, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  v = wave_scan_incl_i(v);
  __syncthreads();
  if (lane == 63) s_wave[wave] = v;
  __syncthreads();
  int base = 0, all = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    if (w < wave) base += s_wave[w];
    all += s_wave[w];
  }
  *total = all;
  return base + v;
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

// Workgroup = (layer, row, kv head): the pairs of its list, and its weights.
__global__ __launch_bounds__(THREADS) void evict_stay_kernel(EvictParams p) {
  const paged_evict_args& a = p.a;
  __shared__ int s_bin[256];
  __shared__ int s_wave[THREADS / 64];
  __shared__ int s_digit, s_left;
  const int tid = threadIdx.x;
  if ((int)blockIdx.x >= p.units) {
    give_back(p, ((int)blockIdx.x - p.units) * (THREADS / 64) + (tid >> 6));
    return;
  }
  const int kvh = blockIdx.x % a.n_kv_heads, b = blockIdx.x / a.n_kv_heads, s = b % a.n_rows, layer = b / a.n_rows;
  int2* list = p.list + (long long)blockIdx.x * (1 + p.most_moves);
  const RowPlan w = plan_row(p, s);
  const float* mass = a.mass + layer * a.mass_stride_layer + s * a.mass_stride_row + kvh * a.mass_stride_head;
  float* out = a.mass_out + (mass - a.mass);
  const int L = w.ok ? w.L : 0, f = w.f, m = w.N - w.r, end = L - w.r, keep = m - f;   // `keep` of f .. end - 1; places f .. m - 1
  if (w.N >= L) {
    if (tid == 0) list[0] = int2{0, 0};
    for (int y = tid; y < L; y += THREADS) out[y] = mass[y];
    return;
  }
  // ---- the keep-th largest rank, eight bits at a time; `left` of those that have it are kept
  unsigned least = 0;
  int left = keep;
  if (keep > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      s_bin[tid] = 0;
      __syncthreads();
      const unsigned above = shift == 24 ? 0u : ~0u << (shift + 8);
      for (int y = f + tid; y < end; y += THREADS) {
        const unsigned u = rank_of(mass[y]);
        if ((u & above) == least) atomicAdd(&s_bin[(u >> shift) & 255], 1);
      }
      __syncthreads();
      // bins from the largest digit down: thread t holds digit 255 - t
      const int mine = s_bin[255 - tid];
      int total;
      const int upto = block_scan(s_wave, mine, &total);
      if (upto >= left && upto - mine < left) { s_digit = 255 - tid; s_left = left - (upto - mine); }
      __syncthreads();
      least |= (unsigned)s_digit << shift;
      left = s_left;
      __syncthreads();
    }
  }
  // ---- the lists, in order of positions
  int ties = 0, holes = 0, fills = 0;   // so far
  for (int y0 = f; y0 < end; y0 += STRIP) {
    unsigned u[PER];
    int n_tie = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int y = y0 + PER * tid + i;
      u[i] = y < end ? rank_of(mass[y]) : 0u;
      n_tie += y < end && u[i] == least ? 1 : 0;
    }
    int all_ties, all;
    int tie = ties + block_scan(s_wave, n_tie, &all_ties) - n_tie;
    // holes in the low half of a word, fills in the high one: a strip has at most 1024 of both
    int marks = 0;
    bool hole[PER], fill[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int y = y0 + PER * tid + i;
      const bool kept = keep > 0 && (u[i] > least || (u[i] == least && tie < left));
      if (y < end && u[i] == least) ++tie;
      hole[i] = y < m && !kept;
      fill[i] = y >= m && y < end && kept;
      marks += (hole[i] ? 1 : 0) + (fill[i] ? 1 << 16 : 0);
    }
    const int at = block_scan(s_wave, marks, &all) - marks;
    int h = holes + (at & 0xffff), q = fills + (at >> 16);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int y = y0 + PER * tid + i;
      if (hole[i]) list[1 + h++].x = y;
      if (fill[i]) list[1 + q++].y = y;
      if (y < m && !hole[i]) out[y] = mass[y];
    }
    ties += all_ties;
    holes += all & 0xffff;
    fills += all >> 16;
  }
  if (tid == 0) list[0] = int2{holes, 0};
  __syncthreads();
  for (int i = tid; i < holes; i += THREADS) {
    const int2 pair = list[1 + i];
    out[pair.x] = mass[pair.y];
  }
  for (int y = tid; y < f; y += THREADS) out[y] = mass[y];
  for (int y = tid; y < w.r; y += THREADS) out[m + y] = mass[end + y];
}

// Workgroup = (unit, keys or values, part of their 16-byte pieces).  First the pairs, whose places and positions are different ones; then the last r, which may go to places
// that others of them leave: a run of them is in registers before its places are written, and every later run comes from behind those.
__global__ __launch_bounds__(THREADS) void evict_move_kernel(EvictParams p) {
  const paged_evict_args& a = p.a;
  const int tid = threadIdx.x, per = p.pieces / p.slices;
  int b = blockIdx.x;
  const int slice = b % p.slices;
  b /= p.slices;
  const bool values = b & 1;
  const int unit = b >> 1, kvh = unit % a.n_kv_heads, s = unit / a.n_kv_heads % a.n_rows, layer = unit / a.n_kv_heads / a.n_rows;
  const RowPlan w = plan_row(p, s);
  if (!w.ok || w.N >= w.L) return;
  const long long esize = a.dtype == CASCADE_BF16 ? 2 : 4;
  char* const base = (char*)(values ? a.v_pages : a.k_pages) + (layer * a.stride_layer + kvh * a.stride_head) * esize + 16ll * slice * per;
  const int32_t* table = a.block_table + s * a.table_stride;
  auto place = [&](int y) -> char* {   // nullptr: outside the pool
    const int e = y / a.page_size, page = table[e];
    if ((unsigned)page >= (unsigned)a.n_pages) {
      atomicOr(p.dev_status, CASCADE_FLAG_PAGE);
      return nullptr;
    }
    return base + (page * a.stride_page + (long long)(y - e * a.page_size) * a.stride_pos) * esize;
  };
  const int2* list = p.list + (long long)unit * (1 + p.most_moves);
  const long long n = (long long)list[0].x * per;
  constexpr int U = 4;
  for (long long i0 = tid; i0 < n; i0 += U * THREADS) {
    u32x4 x[U];
    char* to[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long i = i0 + u * THREADS;
      to[u] = nullptr;
      if (i < n) {
        const int k = (int)(i / per), piece = (int)(i - (long long)k * per);
        const int2 pair = list[1 + k];
        const char* from = place(pair.y);
        to[u] = from ? place(pair.x) : nullptr;
        if (to[u]) { x[u] = *(const u32x4*)(from + 16 * piece); to[u] += 16 * piece; }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (to[u]) *(u32x4*)to[u] = x[u];
  }
  __syncthreads();
  const int m = w.N - w.r, end = w.L - w.r;
  const long long nr = (long long)w.r * per;
  for (long long i0 = 0; i0 < nr; i0 += U * THREADS) {
    u32x4 x[U];
    char* to[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long i = i0 + u * THREADS + tid;
      to[u] = nullptr;
      if (i < nr) {
        const int k = (int)(i / per), piece = (int)(i - (long long)k * per);
        const char* from = place(end + k);
        to[u] = from ? place(m + k) : nullptr;
        if (to[u]) { x[u] = *(const u32x4*)(from + 16 * piece); to[u] += 16 * piece; }
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the run is in registers
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (to[u]) *(u32x4*)to[u] = x[u];
  }
}

int most_moves(const paged_evict_args* a) { return a->max_seq_len / 2; }   // as many places as positions: at most half of them together

}  // namespace

int64_t plan_paged_evict(const paged_evict_args* a) {
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
  p.slices = p.pieces % 8 == 0 ? p.pieces / 8 : 1;   // whole lines of 128 bytes
  {
    KernelTimer t(ctx, CASCADE_K_EVICT);
    CASCADE_TIMED_LAUNCH(t, evict_stay_kernel, dim3((unsigned)(p.units + (a->n_rows + THREADS / 64 - 1) / (THREADS / 64))), dim3(THREADS), 0, ctx->stream, p);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.units == 0) return e;
  KernelTimer t(ctx, CASCADE_K_EVICT_MOVE);
  CASCADE_TIMED_LAUNCH(t, evict_move_kernel, dim3((unsigned)(p.units * 2 * p.slices)), dim3(THREADS), 0, ctx->stream, p);
  return hipGetLastError();
}
