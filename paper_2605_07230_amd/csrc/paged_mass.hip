// paged_mass kernels for gfx950: the attention weight that positions of a cache in pages gather,
//     w(y) = sum over tokens j and query heads g of a kv head:  exp(scale <q_jg, k_y> - lse_jg).
//
// lse is known, so there is no maximum to follow and nothing to rescale: one product S = Q K^T, an exponential per score and a sum down each column.  The keys stand still - a
// wave holds 16 KW of them in registers - and the query rows go past them, so a column's sum stays in one wave from its first term to its last: no atomics, no partial results
// in memory, and an order that depends on the call's sizes alone.
//
// S = Q K^T (queries as A, keys as B): a lane owns a key of each group of 16 and adds up the queries 4 g .. 4 g + 3 of every product; the four 16-lane rows meet once at the end.
#include <algorithm>

#include "common.h"

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr int WAVES = 4, STAGE = 64 * WAVES;   // query rows that are looked up together, a thread each

typedef unsigned long long u64;

struct MassParams {
  paged_mass_args a;
  int group, most_len;   // query heads of a kv head; the longest row that the bounds allow
  int key_blocks;        // workgroups that a row's keys may need
  float scale_log2e;
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

// Workgroup = (row, kv head, 64 KW positions), a wave to 16 KW of them.
template <typename T, int D, int KW, bool VEC>
__global__ __launch_bounds__(64 * WAVES) void paged_mass_kernel(MassParams p) {
  const paged_mass_args& a = p.a;
  __shared__ long long s_q[STAGE];   // where a query row lies
  __shared__ __align__(16) int s_x[STAGE];      // its position; -1: it counts nothing
  __shared__ __align__(16) float s_lse[STAGE];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, g = lane >> 4, G = p.group;
  const int kvh = blockIdx.x % a.n_kv_heads, b = blockIdx.x / a.n_kv_heads, kblk = b % p.key_blocks, s = b / p.key_blocks;
  const int lo = a.q_off[s], hi = a.q_off[s + 1], L = a.seq_len[s];
  int flag = 0;
  if (lo < 0 || hi > a.n_tokens || lo > hi || hi - lo > a.max_new) flag = CASCADE_FLAG_TREE_SIZE;
  else if (L < hi - lo || L > p.most_len) flag = CASCADE_FLAG_CAPACITY;   // (negative lengths among them)
  if (flag) {
    if (kblk == 0 && kvh == 0 && tid == 0) atomicOr(p.dev_status, flag);
    return;
  }
  const int n = hi - lo, M = n * G, Lp = L - n, first = a.first ? max(a.first[s], 0) : 0, W = a.window;
  const int kb0 = 16 * KW * WAVES * kblk;
  if (n == 0 || kb0 >= L || kb0 + 16 * KW * WAVES <= first) return;

  // ---- this wave's keys.  A group of 16 that no token attends, or none of whose positions is asked for, is not read, nor is its entry of the table.
  const int kb = kb0 + 16 * KW * wave;
  Operand<T, D, VEC> key[KW];
  unsigned there = 0;   // groups that hold keys
  const int reach = W > 0 ? max(Lp - W + 1, 0) : 0;   // the first position that a token sees through the window
#pragma unroll
  for (int kt = 0; kt < KW; ++kt) {
    const int y0 = kb + 16 * kt;
    if (y0 >= L || y0 + 15 < first || (y0 + 15 < reach && y0 >= a.n_sink)) continue;
    const int e = y0 / a.page_size, page = __builtin_amdgcn_readfirstlane(a.block_table[s * a.table_stride + e]);
    if ((unsigned)page >= (unsigned)a.n_pages) {
      if (lane == 0) atomicOr(p.dev_status, CASCADE_FLAG_PAGE);
      continue;
    }
    there |= 1u << kt;
    const int inside = y0 - e * a.page_size + min(l16, L - 1 - y0);   // behind the last key: that one again, masked
    key[kt].load((const T*)a.k_pages + page * a.stride_page + kvh * a.stride_head + inside * a.stride_pos, g, a.head_dim);
  }
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
      Operand<T, D, VEC> q;
      q.load((const T*)a.q + s_q[i0 + min(l16, rows - 1)], g, a.head_dim);
      const f32x4 lse = *(const f32x4*)(s_lse + i0 + 4 * g);
      // whether every row sees all of the wave's keys
      const int x0 = Lp + r0 / G, x1 = Lp + (r0 + rows - 1) / G;
      const bool whole = all_count && rows == 16 && there == (1u << KW) - 1 && kb + 16 * KW - 1 <= x0 && (W == 0 || x1 - kb < W);
#pragma unroll
      for (int kt = 0; kt < KW; ++kt) {
        f32x4 w = Operand<T, D, VEC>::product(q, key[kt]);
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
  // ---- lane (l16, g) writes position 16 g + l16 of the wave's
  float mine = 0.f;
#pragma unroll
  for (int kt = 0; kt < KW; ++kt) {
    const float all = rows4_sum(sum[kt]);
    if (g == kt) mine = all;
  }
  const int y = kb + lane;
  if (lane < 16 * KW && y >= first && y < L) {
    float* m = a.mass + s * a.mass_stride_row + kvh * a.mass_stride_head + y;
    *m = y >= Lp ? mine : *m + mine;
  }
}

template <typename T, int D, int KW, bool VEC>
hipError_t launch_k(cascade_ctx* ctx, MassParams& p) {
  constexpr int KEYS = 16 * KW * WAVES;
  p.key_blocks = (p.a.max_seq_len + KEYS - 1) / KEYS;
  const int64_t blocks = (int64_t)p.a.n_rows * p.a.n_kv_heads * p.key_blocks;
  KernelTimer t(ctx, CASCADE_K_MASS);
  CASCADE_TIMED_LAUNCH(t, (paged_mass_kernel<T, D, KW, VEC>), dim3((unsigned)blocks), dim3(64 * WAVES), 0, ctx->stream, p);
  return hipGetLastError();
}
template <bool VEC>
hipError_t launch_f32(cascade_ctx* ctx, MassParams& p) {
  if (p.a.head_dim <= 64) return launch_k<float, 64, 4, VEC>(ctx, p);
  return p.a.head_dim <= 128 ? launch_k<float, 128, 2, VEC>(ctx, p) : launch_k<float, 256, 1, VEC>(ctx, p);
}

}  // namespace

hipError_t launch_paged_mass(cascade_ctx* ctx, const paged_mass_args* a) {
  MassParams p;
  p.a = *a;
  p.group = a->n_heads / a->n_kv_heads;
  p.most_len = (int)std::min<int64_t>({a->max_seq_len, (int64_t)a->table_width * a->page_size, a->mass_cap});
  p.scale_log2e = (a->scale != 0.f ? a->scale : 1.f / sqrtf((float)a->head_dim)) * LOG2E;
  p.dev_status = ctx->dev_status;
  if (a->dtype == CASCADE_BF16) return a->head_dim == 128 ? launch_k<uint16_t, 128, 4, true>(ctx, p) : launch_k<uint16_t, 64, 4, true>(ctx, p);
  // 16 bytes at a time where everything lies on such boundaries, otherwise element by element
  const bool vec = ((a->head_dim | a->q_stride | a->stride_page | a->stride_head | a->stride_pos) % 4) == 0 && (((uintptr_t)a->q | (uintptr_t)a->k_pages) & 15) == 0;
  return vec ? launch_f32<true>(ctx, p) : launch_f32<false>(ctx, p);
}
