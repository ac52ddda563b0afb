// paged_attn kernels for gfx950: attention of new tokens (a chain, or a drafted tree) over a cache in pages and over themselves.
#include "common.h"

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

struct PagedParams {
  paged_attn_args a;
  int group;
  float scale_log2e;
  int* dev_status;
};

// One wave per (token, query head): a lane takes a key of 64, then head elements.
template <typename T>
__global__ __launch_bounds__(256) void paged_attn_simple_kernel(PagedParams p) {
  const paged_attn_args& a = p.a;
  __shared__ float s_q[4][256];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long long at = (long long)blockIdx.x * 4 + wave;
  if (at >= (long long)a.n_tokens * a.n_heads) return;
  const int t = (int)(at / a.n_heads), h = (int)(at % a.n_heads), kvh = h / p.group, D = a.head_dim;
  int s = -1;
  for (int base = 0; base < a.n_rows && s < 0; base += 64) {
    const int r = base + lane;
    const bool hit = r < a.n_rows && a.q_off[r] <= t && t < a.q_off[r + 1];
    const unsigned long long who = __ballot(hit);
    if (who) s = base + __ffsll((long long)who) - 1;
  }
  if (s < 0) return;
  const int lo = a.q_off[s], n = a.q_off[s + 1] - lo, P = a.prefix_len[s];
  T* out = (T*)a.out + at * D;
  auto put = [&](int d, float v) {
    if constexpr (sizeof(T) == 2) out[d] = f32_to_bf16_bits(v);
    else out[d] = v;
  };
  int flag = 0;
  if (lo < 0 || a.q_off[s + 1] > a.n_tokens || n > a.max_new) flag = CASCADE_FLAG_TREE_SIZE;
  else if (P < 0 || P > a.max_prefix_len || P > (long long)a.table_width * a.page_size) flag = CASCADE_FLAG_CAPACITY;
  if (flag) {
    if (lane == 0) atomicOr(p.dev_status, flag);
    for (int d = lane; d < D; d += 64) put(d, 0.f);
    if (lane == 0 && a.lse) a.lse[at] = -INFINITY;
    return;
  }
  const T* q = (const T*)a.q + (long long)t * a.q_stride + (long long)h * D;
  for (int d = lane; d < D; d += 64) s_q[wave][d] = load_f32(q + d);
  const int i = t - lo;
  // the node's depth (a chain: its index)
  int depth = i;
  if (a.parent) {
    depth = 0;
    for (int x = i; x > 0; ++depth) {
      const int up = a.parent[lo + x];
      if (up >= x || up < 0) { if (lane == 0) atomicOr(p.dev_status, CASCADE_FLAG_PARENT); x = 0; }
      else x = up;
    }
  }
  const int qpos = P + depth;
  auto near = [&](int kpos) { return a.window == 0 || qpos - kpos < a.window || kpos < a.n_sink; };
  float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  const int n_pt = (P + 63) / 64, n_nt = i / 64 + 1;
  for (int c = 0; c < n_pt + n_nt; ++c) {
    const bool fresh = c >= n_pt;
    const int key = 64 * (fresh ? c - n_pt : c) + lane;
    bool sees = false;
    const T *k = nullptr, *v = nullptr;
    if (!fresh) {
      if (key < P && near(key)) {
        int g = a.block_table[s * a.table_stride + key / a.page_size];
        if (g < 0 || g >= a.n_pages) { atomicOr(p.dev_status, CASCADE_FLAG_PAGE); g = 0; }
        const long long off = g * a.stride_page + kvh * a.stride_head + (key % a.page_size) * a.stride_pos;
        k = (const T*)a.k_pages + off;
        v = (const T*)a.v_pages + off;
        sees = true;
      }
    } else if (key <= i) {
      int kdepth = key;
      sees = true;
      if (a.parent) {
        sees = false;
        int x = i;
        kdepth = depth;
        while (x > key) {
          const int up = a.parent[lo + x];
          x = up >= x || up < 0 ? 0 : up;
          --kdepth;
        }
        sees = x == key;
      }
      sees = sees && near(P + kdepth);
      if (sees) {
        const long long off = (lo + key) * a.kv_stride + (long long)kvh * D;
        k = (const T*)a.k_new + off;
        v = (const T*)a.v_new + off;
      }
    }
    float z = -INFINITY;
    if (sees) {
      float dot = 0.f;
      for (int d = 0; d < D; ++d) dot = fmaf(s_q[wave][d], load_f32(k + d), dot);
      z = dot * p.scale_log2e;
    }
    const float m_new = fmaxf(m, wave_max(z)), use = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = exp2f(m - use), e = sees ? exp2f(z - use) : 0.f;
    l = l * alpha + wave_sum(e);
    m = m_new;
    for (int x = 0; x < 4; ++x) o[x] *= alpha;
    unsigned long long who = __ballot(sees);
    while (who) {
      const int j = __ffsll((long long)who) - 1;
      who &= who - 1;
      const float w = __shfl(e, j);
      const T* vj = (const T*)__shfl((unsigned long long)v, j);
      for (int x = 0; x < 4; ++x)
        if (lane + 64 * x < D) o[x] = fmaf(w, load_f32(vj + lane + 64 * x), o[x]);
    }
  }
  for (int x = 0; x < 4; ++x)
    if (lane + 64 * x < D) put(lane + 64 * x, l == 0.f ? 0.f : o[x] / l);
  if (lane == 0 && a.lse) a.lse[at] = m * LN2 + logf(l);
}

}  // namespace

hipError_t launch_paged_attn(cascade_ctx* ctx, const paged_attn_args* a) {
  PagedParams p;
  p.a = *a;
  p.group = a->n_heads / a->n_kv_heads;
  p.scale_log2e = (a->scale != 0.f ? a->scale : 1.f / sqrtf((float)a->head_dim)) * LOG2E;
  p.dev_status = ctx->dev_status;
  const unsigned grid = (unsigned)(((long long)a->n_tokens * a->n_heads + 3) / 4);
  KernelTimer t(ctx, CASCADE_K_PAGED_ATTN);
  if (a->dtype == CASCADE_BF16) CASCADE_TIMED_LAUNCH(t, paged_attn_simple_kernel<uint16_t>, dim3(grid), dim3(256), 0, ctx->stream, p);
  else CASCADE_TIMED_LAUNCH(t, paged_attn_simple_kernel<float>, dim3(grid), dim3(256), 0, ctx->stream, p);
  return hipGetLastError();
}

int64_t plan_paged_attn(const cascade_ctx* ctx, const paged_attn_args* a) { return 0; }
