// paged_slots and paged_append kernels for gfx950: pages for rows that grow, and the copy of their new tokens into them.
#include "common.h"

namespace {

// ---------------------------------------------------------------------------------------------------------------- paged_slots
// Rows are served in order: row s takes the pages behind those of the rows before it, from the end of the list of free ones, if
// they reach; where they stop reaching, no later row gets any either.  That is one exclusive scan over the rows (of new tokens, which
// also places them, then of pages), which every workgroup makes by itself from the lengths: two or three values of a few
// hundred rows cost less than a second launch.  A workgroup then writes the tokens of its row, or of a part of it, a token to a thread.
// Bound by launch and the chain lengths -> scan -> table -> slot: 16 rows 4.2 us, 256 rows with 159052 tokens 6.6.
struct SlotParams {
  paged_slots_args a;
  int* dev_status;
};

constexpr int SLOT_THREADS = 256;

// additions that stop at the largest value keep any order of them the same
__device__ __forceinline__ unsigned sat_add(unsigned a, unsigned b) { return a + b < a ? 0xffffffffu : a + b; }

__device__ __forceinline__ unsigned wave_scan_sat(unsigned v) {
  v = sat_add((unsigned)dpp_i32<0x111, 0xf>(0, (int)v), v);
  v = sat_add((unsigned)dpp_i32<0x112, 0xf>(0, (int)v), v);
  v = sat_add((unsigned)dpp_i32<0x114, 0xf>(0, (int)v), v);
  v = sat_add((unsigned)dpp_i32<0x118, 0xf>(0, (int)v), v);
  v = sat_add((unsigned)dpp_i32<0x142, 0xa>(0, (int)v), v);
  v = sat_add((unsigned)dpp_i32<0x143, 0xc>(0, (int)v), v);
  return v;
}

// inclusive scan over the workgroup's threads, and their sum
__device__ __forceinline__ unsigned block_scan_sat(unsigned* s_wave, unsigned v, unsigned* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  v = wave_scan_sat(v);
  __syncthreads();
  if (lane == 63) s_wave[wave] = v;
  __syncthreads();
  unsigned base = 0, all = 0;
#pragma unroll
  for (int w = 0; w < SLOT_THREADS / 64; ++w) {
    if (w < wave) base = sat_add(base, s_wave[w]);
    all = sat_add(all, s_wave[w]);
  }
  *total = all;
  return sat_add(base, v);
}

__global__ __launch_bounds__(SLOT_THREADS) void paged_slots_kernel(SlotParams p) {
  const paged_slots_args& a = p.a;
  __shared__ unsigned s_wave[SLOT_THREADS / 64];
  __shared__ unsigned s_base, s_end, s_page0, s_taken, s_served;
  const int tid = threadIdx.x, s = blockIdx.x, part = blockIdx.y, parts = gridDim.y;
  const bool path = a.new_len == nullptr;
  const unsigned cap = (unsigned)a.max_tokens;
  if (tid == 0) { s_base = 0; s_end = 0; s_page0 = 0; s_taken = 0; s_served = 0; }
  unsigned free_n = 0;
  {
    const int f = a.free_count[0];
    free_n = f < 0 ? 0u : min((unsigned)f, (unsigned)a.free_capacity);
    if (s == 0 && part == 0 && tid == 0 && (unsigned)f != free_n) atomicOr(p.dev_status, CASCADE_FLAG_PAGE);
  }
  unsigned tokens = 0, pages = 0;   // of the rows before these
  for (int r0 = 0; r0 < a.n_rows; r0 += SLOT_THREADS) {
    const int r = r0 + tid;
    int len = 0, n = 0, flag = 0;
    if (r < a.n_rows) {
      len = a.seq_len[r];
      if (path) {
        const int b = a.row_prompt[r];
        if (b < 0 || b >= a.n_prompts) flag = CASCADE_FLAG_PATH;
        else {
          n = a.accept_len[b];
          if (n < 0 || n > a.max_depth) { flag = CASCADE_FLAG_DEPTH; n = 0; }
          else ++n;
        }
      } else {
        n = a.new_len[r];
        if (n < 0) { flag = CASCADE_FLAG_CAPACITY; n = 0; }
      }
    }
    unsigned sum;
    const unsigned end = sat_add(tokens, block_scan_sat(s_wave, (unsigned)n, &sum)), begin = end == 0xffffffffu ? end : end - (unsigned)n;
    // a row whose tokens, or whose pages in the table, do not all have a place asks for nothing
    bool fits = !flag && r < a.n_rows && len >= 0 && end <= cap && (long long)len + n <= (long long)a.table_width * a.page_size;
    if (!fits && !flag && r < a.n_rows) flag = CASCADE_FLAG_CAPACITY;
    const unsigned ps = (unsigned)a.page_size;
    const unsigned need = fits ? (unsigned)(((long long)len + n + ps - 1) / ps) - (unsigned)(((long long)len + ps - 1) / ps) : 0u;
    unsigned page_sum;
    const unsigned page_end = sat_add(pages, block_scan_sat(s_wave, need, &page_sum)), page0 = page_end == 0xffffffffu ? page_end : page_end - need;
    if (fits && need && page_end > free_n) { fits = false; flag = CASCADE_FLAG_CAPACITY; }
    if (fits && need) atomicMax(&s_taken, page_end);
    if (r == s) { s_base = min(begin, cap); s_end = min(end, cap); s_page0 = page0; s_served = fits; }
    if (s == 0 && part == 0 && r < a.n_rows) {
      if (flag) atomicOr(p.dev_status, flag);
      if (r == 0) a.q_off[0] = 0;
      a.q_off[r + 1] = (int)min(end, cap);
      a.seq_len_out[r] = fits ? len + n : len;
    }
    tokens = sat_add(tokens, sum);
    pages = sat_add(pages, page_sum);
    if (r0 + SLOT_THREADS >= a.n_rows) {   // places behind the last token, dealt to all workgroups
      for (unsigned t = min(tokens, cap) + (unsigned)((s * parts + part) * SLOT_THREADS + tid); t < cap; t += gridDim.x * parts * SLOT_THREADS) {
        a.slot_map[t] = -1;
        if (a.position) a.position[t] = -1;
        if (a.source) a.source[t] = -1;
      }
    }
  }
  __syncthreads();
  if (s == 0 && part == 0 && tid == 0) a.free_count_out[0] = (int)(free_n - s_taken);
  const bool served = s_served != 0;
  const unsigned base = s_base, n = s_end - base, ps = (unsigned)a.page_size;
  const unsigned len = (unsigned)max(a.seq_len[s], 0), have = (len + ps - 1) / ps;
  const int32_t* table = a.block_table + (long long)s * a.table_stride;
  const unsigned top = free_n - 1 - s_page0 + have;   // page e of the table comes from free_pages[top - e]
  auto fresh = [&](unsigned e) {
    const int g = a.free_pages[top - e];
    return g >= 0 && g < a.n_pages ? g : -1;
  };
  if (served) {
    const unsigned last = (len + n + ps - 1) / ps;
    for (unsigned e = have + part * SLOT_THREADS + tid; e < last; e += parts * SLOT_THREADS) {
      const int g = fresh(e);
      if (g < 0) atomicOr(p.dev_status, CASCADE_FLAG_PAGE);
      a.block_table[(long long)s * a.table_stride + e] = g;
    }
  }
  int off = 0, nodes = 0, prompt = 0;
  if (path && n) {
    prompt = a.row_prompt[s];
    off = a.node_off[s];
    nodes = a.node_off[s + 1] - off;
  }
  for (unsigned j = part * SLOT_THREADS + tid; j < n; j += parts * SLOT_THREADS) {
    const unsigned pos = len + j, e = pos / ps;
    int slot = -1, src = (int)(base + j);
    if (served) {
      const int g = e >= have ? fresh(e) : table[e];
      if (g >= 0 && g < a.n_pages) slot = g * (int)ps + (int)(pos - e * ps);
      else if (e < have) atomicOr(p.dev_status, CASCADE_FLAG_PAGE);
    }
    if (path) {
      const int node = j ? a.path_nodes[(long long)prompt * a.max_depth + j - 1] : 0;
      if (node < 0 || node >= nodes || off < 0 || off > a.n_nodes_total - 1 - node) {
        atomicOr(p.dev_status, CASCADE_FLAG_PATH);
        slot = src = -1;
      } else {
        src = off + node;
      }
    }
    a.slot_map[base + j] = slot;
    if (a.position) a.position[base + j] = (int)pos;
    if (a.source) a.source[base + j] = src;
  }
}

// --------------------------------------------------------------------------------------------------------------- paged_append
// A gather / scatter of 16-byte pieces, like kv_commit: workgroup = (a run of pieces, layer, keys or values); a thread
// requests its pieces' slots, then the pieces themselves, and stores them past the caches.  Bound by the copy: 495 MB (30 layers, 2000 tokens of 8 x 128) 85 us =
// 5.9 TB/s, read and write counted; one token of 16 rows x 30 layers (16 MB) 4.7.
struct AppendParams {
  paged_append_args a;
  int* dev_status;
  int row_vec, head_vec;            // 16-byte pieces of a token, of one of its heads
  unsigned total;                   // pieces of all tokens in a layer
  long long sl, sg, sh, sp;         // strides of the pool in 16-byte pieces
  long long src_layer;              // pieces of a layer of k_new / v_new
};

constexpr int APPEND_THREADS = 256, APPEND_EACH = 4;
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

__global__ __launch_bounds__(APPEND_THREADS) void paged_append_kernel(AppendParams p) {
  const paged_append_args& a = p.a;
  const int layer = blockIdx.y;
  const bool values = blockIdx.z;
  const u32x4* src = (const u32x4*)(values ? a.v_new : a.k_new) + layer * p.src_layer;
  u32x4* dst = (u32x4*)(values ? a.v_pages : a.k_pages) + layer * p.sl;
  const int n_slots = a.n_pages * a.page_size;
  const unsigned first = blockIdx.x * (APPEND_THREADS * APPEND_EACH) + threadIdx.x;
  u32x4 piece[APPEND_EACH];
  int slot[APPEND_EACH];
  unsigned v[APPEND_EACH];
#pragma unroll
  for (int i = 0; i < APPEND_EACH; ++i) {
    const unsigned at = min(first + i * APPEND_THREADS, p.total - 1), t = at / (unsigned)p.row_vec;
    v[i] = at - t * p.row_vec;
    slot[i] = a.slot_map[t];
    int from = (int)t;
    if (a.source) from = a.source[t];
    const bool in = first + i * APPEND_THREADS < p.total;
    if (slot[i] < -1 || slot[i] >= n_slots || (slot[i] >= 0 && (from < 0 || from >= a.n_source))) {
      if (in && v[i] == 0 && layer == 0 && !values) atomicOr(p.dev_status, CASCADE_FLAG_PAGE);
      slot[i] = -1;
    }
    if (!in) slot[i] = -1;
    if (slot[i] >= 0) piece[i] = src[(long long)from * p.row_vec + v[i]];
  }
#pragma unroll
  for (int i = 0; i < APPEND_EACH; ++i)
    if (slot[i] >= 0) {
      const unsigned page = (unsigned)slot[i] / (unsigned)a.page_size, head = v[i] / (unsigned)p.head_vec;
      __builtin_nontemporal_store(piece[i], dst + page * p.sg + (slot[i] - page * a.page_size) * p.sp + head * p.sh + (v[i] - head * p.head_vec));
    }
}

}  // namespace

hipError_t launch_paged_slots(cascade_ctx* ctx, const paged_slots_args* a) {
  SlotParams p = {*a, ctx->dev_status};
  // a workgroup writes about a thousand tokens, at most four workgroups per compute unit
  int64_t parts = ((int64_t)a->max_tokens / a->n_rows + 1023) / 1024;
  const int64_t most = 4 * ctx->n_cu / a->n_rows;
  if (parts > most) parts = most;
  if (parts < 1) parts = 1;
  KernelTimer t(ctx, CASCADE_K_SLOTS);
  CASCADE_TIMED_LAUNCH(t, paged_slots_kernel, dim3((unsigned)a->n_rows, (unsigned)parts), dim3(SLOT_THREADS), 0, ctx->stream, p);
  return hipGetLastError();
}

hipError_t launch_paged_append(cascade_ctx* ctx, const paged_append_args* a) {
  const int e = a->dtype == CASCADE_BF16 ? 2 : 4;
  AppendParams p;
  p.a = *a;
  p.dev_status = ctx->dev_status;
  p.head_vec = a->head_dim * e / 16;
  p.row_vec = a->n_kv_heads * p.head_vec;
  p.total = (unsigned)a->n_tokens * (unsigned)p.row_vec;
  p.sl = a->stride_layer * e / 16;
  p.sg = a->stride_page * e / 16;
  p.sh = a->stride_head * e / 16;
  p.sp = a->stride_pos * e / 16;
  p.src_layer = (long long)a->n_source * p.row_vec;
  const unsigned each = APPEND_THREADS * APPEND_EACH;
  dim3 grid((p.total + each - 1) / each, (unsigned)a->n_layers, 2);
  KernelTimer t(ctx, CASCADE_K_APPEND);
  CASCADE_TIMED_LAUNCH(t, paged_append_kernel, grid, dim3(APPEND_THREADS), 0, ctx->stream, p);
  return hipGetLastError();
}
