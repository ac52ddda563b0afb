// paged_attn kernels for gfx950: attention of new tokens (a chain, or a drafted tree) over a cache in pages and over themselves.
//
// The query rows of a (row of the batch, kv head) are its tokens times the query heads that share the kv head, token by token, so that a block of rows is a
// short run of positions: what a chain's mask or a window leaves it is one run of key tiles (two with sinks), and no other tile is touched.
//
// Keys come in tiles of 64, first those of the pages, then those of the new tokens.  A page holds a multiple of 16 positions, so 16 keys that begin
// at a multiple of 16 lie in one page, one stride apart: a wave looks one entry of the table up for them, in scalar registers.
//
// Scores are produced transposed, S^T = K Q^T (v_mfma_f32_16x16x32_bf16): a lane owns one query column, so the running maximum and sum are
// per-lane scalars, a mask is one 64-bit word per lane and tile, made from three comparisons, and the probabilities are already the B operand of
// O^T = V^T P^T, whose A operand the transposing LDS read (ds_read_b64_tr_b16) takes from row-major values.
//
// Probabilities enter that product as bf16, the only type in which the matrix cores take them next to bf16 values at this rate: at most half a step, 2^-8 of each, which leaves
// outputs 0.0022 from float64 (relative 2-norm) where probabilities in float32 leave 0.0017, the rounding of the result.  Sums, maxima and lse are of unrounded float32 ones.
//
// A masked key has probability 0, but 0 x inf and 0 x NaN are NaN.  Places that no token of the workgroup sees are never taken from memory, or are
// zeroed on the way; a tile that some tokens see and others do not, or whose places behind the last key hold that key again, is looked through for such values, and if
// it holds any they are taken out of the product and added to the tokens that see them, once what was summed before has its scale (the first scale is 0).
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "common.h"

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
constexpr int KT = 64;   // keys per tile

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef unsigned long long u64;

struct PagedParams {
  paged_attn_args a;
  int group;
  unsigned group_inv;    // floor(2^32 / group) + 1: a query row's token as a high product (rows times group stay below 2^32); 0 for one head
  int most_prefix;       // the longest prefix that the bound and the table allow
  float scale_log2e;
  int* dev_status;
  int page16;            // 16-key groups of a page
  unsigned page16_inv;   // floor(2^32 / page16) + 1: group / page16 as a high product (groups stay below 2^26, page16 <= 64); 0 for page16 1
  int parts;             // that the keys of a row are cut into at most; 1: results are written at once
  int part_tiles;        // tiles of a part (few rows)
  bool in_order;         // (other kernels) rows of the batch are taken in order, not longest first
  float* ws_o;           // [parts][n_tokens * n_heads][head_dim]
  float* ws_ml;          // [parts][n_tokens * n_heads][2]
};

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ uint32_t pack_bf16x2(float a, float b) {
  const bf16x2_t v = __builtin_convertvector(f32x2_t{a, b}, bf16x2_t);
  return *(const uint32_t*)&v;
}
union Frag8 {
  bf16x8 v;
  uint4 u;
};

// bits 0 .. n - 1
__device__ __forceinline__ u64 below(int n) { return n <= 0 ? 0ull : (n >= 64 ? ~0ull : (1ull << n) - 1ull); }

// ---- one row of the batch
struct RowInfo {
  int s, lo, T, P;
  int flag;   // what is wrong with it; then T counts the tokens of it that exist, for zeros
};
__device__ __forceinline__ RowInfo check_row(const PagedParams& p, int s, int lo, int hi, int P) {
  const paged_attn_args& a = p.a;
  RowInfo r = {s, lo, hi - lo, P, 0};
  if (lo < 0 || hi > a.n_tokens || lo > hi || hi - lo > a.max_new) {
    r.flag = CASCADE_FLAG_TREE_SIZE;
    r.lo = max(lo, 0);
    r.T = max(min(hi, a.n_tokens) - r.lo, 0);
  } else if (P < 0 || P > p.most_prefix) {
    r.flag = CASCADE_FLAG_CAPACITY;
  }
  return r;
}

// The tiles that query tokens i0 .. i1 of a row see: n_p of the pages, then n_n of the new tokens.  A window leaves those of the sinks and those from
// its beginning on; `skip` tiles between them are left out.
struct Tiles {
  int n_p, sinks_p, skip_p;
  int n_n, sinks_n, skip_n;
  int first;   // the first position that some of these tokens sees through the window (all: 0)
  __device__ __forceinline__ int prefix_tile(int t) const { return t < sinks_p ? t : t + skip_p; }
  __device__ __forceinline__ int new_tile(int t) const { return t < sinks_n ? t : t + skip_n; }
};
template <int TS = KT>   // keys per tile
__device__ __forceinline__ Tiles tiles_of(const PagedParams& p, int P, int i0, int i1, bool tree) {
  const int W = p.a.window, n_pt = (P + TS - 1) / TS, n_nt = i1 / TS + 1;
  Tiles t = {n_pt, 0, 0, n_nt, 0, 0, 0};
  if (W > 0) {
    if (tree) i0 = 0;   // a node's position is its depth
    t.first = max(0, P + i0 - W + 1);
    const int from_p = t.first < P ? t.first / TS : n_pt;
    t.sinks_p = (min(p.a.n_sink, P) + TS - 1) / TS;
    t.skip_p = max(0, from_p - t.sinks_p);
    t.n_p = n_pt - t.skip_p;
    if (!tree) {
      t.sinks_n = min((min(max(p.a.n_sink - P, 0), i1 + 1) + TS - 1) / TS, n_nt);
      t.skip_n = max(0, max(0, i0 - W + 1) / TS - t.sinks_n);
      t.n_n = n_nt - t.skip_n;
    }
  }
  return t;
}

// keys kb .. kb + 63 of the pages that a token at position x sees; of a chain's new tokens, that token i sees
__device__ __forceinline__ u64 sees_prefix(const PagedParams& p, int P, int kb, int x) {
  u64 v = below(P - kb);
  if (p.a.window > 0) v &= ~below(x - p.a.window + 1 - kb) | below(p.a.n_sink - kb);
  return v;
}
__device__ __forceinline__ u64 sees_chain(const PagedParams& p, int P, int kb, int i) {
  u64 v = below(i + 1 - kb);
  if (p.a.window > 0) v &= ~below(i - p.a.window + 1 - kb) | below(p.a.n_sink - P - kb);
  return v;
}

// The group of 16 keys to load for group g: itself, or, where none of its keys exists or is seen, one with such keys.
__device__ __forceinline__ int needed_group(const PagedParams& p, const Tiles& ti, int P, int g) {
  g = min(g, (P - 1) >> 4);
  if (p.a.window > 0 && 16 * g >= p.a.n_sink && 16 * g + 15 < ti.first) g = ti.first < P ? ti.first >> 4 : (min(p.a.n_sink, P) - 1) >> 4;
  return g;
}
__device__ __forceinline__ int token_of(const PagedParams& p, int row) { return p.group_inv ? (int)__umulhi((unsigned)row, p.group_inv) : row; }
__device__ __forceinline__ int page_index(const PagedParams& p, int g) { return p.page16_inv ? (int)__umulhi((unsigned)g, p.page16_inv) : g; }

// an entry of the table; one outside the pool is flagged and stands for the first page
__device__ __forceinline__ int checked_page(const PagedParams& p, int page) {
  if ((unsigned)page < (unsigned)p.a.n_pages) return page;
  if ((threadIdx.x & 63) == 0) atomicOr(p.dev_status, CASCADE_FLAG_PAGE);
  return 0;
}
typedef const __attribute__((address_space(4))) int32_t* ConstTable;   // loads through the scalar cache
__device__ __forceinline__ int table_entry(const PagedParams& p, int s, int e) {
  return *((ConstTable)(uintptr_t)p.a.block_table + ((long long)s * p.a.table_stride + e));
}
// element offset of the first key of group g in page `page` (e-th of the row), kv head kvh
__device__ __forceinline__ long long group_offset(const PagedParams& p, int page, int e, int g, int kvh) {
  return page * p.a.stride_page + kvh * p.a.stride_head + (long long)(16 * (g - e * p.page16)) * p.a.stride_pos;
}

// infinities and NaN among packed bf16 pairs: adding one to an exponent of ones reaches the sign's place
__device__ __forceinline__ uint32_t odd_exponent(uint32_t x) { return (x & 0x7f807f80u) + 0x00800080u; }   // & 0x80008000
__device__ __forceinline__ uint32_t finite_only(uint32_t x) {
  const uint32_t bad = odd_exponent(x) & 0x80008000u;
  return x & ~(bad | (bad - (bad >> 15)));
}

// zeros for the tokens of a row that cannot be computed, query heads of one kv head; empty parts where there are several
template <typename T>
__device__ __forceinline__ void write_nothing(const PagedParams& p, const RowInfo& r, int kvh, int part, int tid, int threads) {
  const int D = p.a.head_dim, G = p.group;
  if (tid == 0 && part == 0) atomicOr(p.dev_status, r.flag);
  for (int i = tid; i < r.T * G; i += threads) {
    const long long row = (long long)(r.lo + i / G) * p.a.n_heads + kvh * G + i % G;
    if (p.parts > 1) {
      float* ml = p.ws_ml + ((long long)part * p.a.n_tokens * p.a.n_heads + row) * 2;
      ml[0] = -INFINITY;
      ml[1] = 0.f;
    } else if (part == 0) {
      for (int d = 0; d < D; ++d) ((T*)p.a.out)[row * D + d] = 0;
      if (p.a.lse) p.a.lse[row] = -INFINITY;
    }
  }
}

// ------------------------------------------------------------------------------------------------------------ bf16, few query rows
// Up to 16 query rows (single tokens, a few of them): bound by the stream of keys and values, so every wave of a workgroup takes its own tiles - w, w + NW, ... of the part
// - and needs no barrier until their end, where the waves' maxima, sums and outputs meet in LDS.  Keys are loaded in operand order (16 bytes of
// a key per lane), values through a region of LDS of the wave's own.  A workgroup works through parts (row, kv head, run of part_tiles tiles) until
// none is left: rows of very different lengths share the chip, and no workgroup is launched for nothing.
// One token of 64 rows x 4200 keys, 8 kv heads of 4, head_dim 128 (1.1 GB): 193 us = 5.7 TB/s; of 90 to 4200 keys (602 MB) 120 us and the join's 4; two rows x 312 keys, 32 kv heads: 9.8 us, of
// which the chain row -> table -> tile -> join of the waves is all, and the way of its instructions from memory: lookups of a lane per group of keys on scalar bases and masks only where
// something is masked (3600 -> 3000 instructions) took 1 us off every small call.  (The look at a last key's values, 20
// instructions, takes 0.35 of one.)  Sixty-four rows dealt longest first, every second round backwards: no faster (131 -> 146 then).  Sixteen trees of 15 nodes x 600 keys, 32 heads: 37 us = 4.5 TB/s.
// Waves per SIMD: two, at head_dim 64, whose tiles are half as large, three of four-wave workgroups (64 rows of 90 to 4200 keys 70 -> 67 us, of 300 to 600 with 16 heads 28.3 -> 26.9).
template <int D, int NW>
constexpr int few_per_unit() { return D == 64 && NW == 4 ? 3 : 8 / NW; }
template <int D, int NW, bool TREE>
__global__ __launch_bounds__(64 * NW, (few_per_unit<D, NW>())) void paged_few_kernel(PagedParams p) {
  constexpr int NT = 64 * NW, KS = D / 32, DB = D / 16, DC = D / 8, VP = D + 16, OP = D + 4, NVC = KT * DC / 64, R = 16;
  extern __shared__ __align__(16) char few_smem[];
  const paged_attn_args& a = p.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g = lane >> 4, G = p.group;
  uint16_t* vt = (uint16_t*)few_smem + (size_t)wave * KT * VP;

  for (int item = blockIdx.x;; item += gridDim.x) {
    const int kvh = item % a.n_kv_heads;
    int part = item / a.n_kv_heads;
    // which row this part belongs to
    RowInfo r = {-1, 0, 0, 0, 0};
    int n_parts = 0;
    for (int base = 0; base < a.n_rows && r.s < 0; base += 64) {
      const int at = base + lane;
      RowInfo mine = {at, 0, 0, 0, 0};
      int n = 0;
      if (at < a.n_rows) {
        mine = check_row(p, at, a.q_off[at], a.q_off[at + 1], a.prefix_len[at]);
        if (mine.flag) {
          n = 1;   // (reported even if it holds no token)
        } else if (mine.T > 0) {
          const Tiles ti = tiles_of(p, mine.P, 0, mine.T - 1, TREE);
          n = (ti.n_p + ti.n_n + p.part_tiles - 1) / p.part_tiles;
        }
      }
      const int incl = wave_scan_incl_i(n);
      const u64 who = __ballot(part < incl);
      if (who) {
        const int l = __ffsll((long long)who) - 1;
        r.s = base + l;
        r.lo = __builtin_amdgcn_readlane(mine.lo, l);
        r.T = __builtin_amdgcn_readlane(mine.T, l);
        r.P = __builtin_amdgcn_readlane(mine.P, l);
        r.flag = __builtin_amdgcn_readlane(mine.flag, l);
        n_parts = __builtin_amdgcn_readlane(n, l);
        part -= __builtin_amdgcn_readlane(incl - n, l);
      } else {
        part -= __builtin_amdgcn_readlane(incl, 63);
      }
    }
    if (r.s < 0) return;
    if (r.flag) {
      for (int q = 0; q < p.parts; ++q) write_nothing<uint16_t>(p, r, kvh, q, tid, NT);
      continue;
    }
    const int lo = r.lo, T = r.T, P = r.P, M = T * G;
    const Tiles ti = tiles_of(p, P, 0, T - 1, TREE);
    const int nt = ti.n_p + ti.n_n, t_begin = part * p.part_tiles, t_end = min(nt, t_begin + p.part_tiles);
    if (part == 0 && p.parts > n_parts)   // parts that this row has not
      for (int i = tid; i < M * (p.parts - n_parts); i += NT) {
        const int q = i % M;
        float* ml = p.ws_ml + ((long long)(n_parts + i / M) * a.n_tokens * a.n_heads + (long long)(lo + q / G) * a.n_heads + kvh * G + q % G) * 2;
        ml[0] = -INFINITY;
        ml[1] = 0.f;
      }

    // ---- a tile: kf[kt][ks] = key 16 kt + l16, d 32 ks + 8 g .. + 7; value pieces c = lane + 64 it of the row-major tile.  Groups of 16 keys begin
    // anywhere; inside one, 32-bit offsets do.  Keys past the end are the last one again.
    u32x4 kf[4][KS], vr[NVC];
    const char *kn = (const char*)((const uint16_t*)a.k_new + lo * a.kv_stride + kvh * D), *vn = (const char*)((const uint16_t*)a.v_new + lo * a.kv_stride + kvh * D);
    constexpr int GV = NVC / 4, KEYS = 64 / DC;   // value pieces of a lane in a group, keys between two of them
    auto request = [&](int t) {
      const bool fresh = t >= ti.n_p;
      const int end = (fresh ? T : P) - 1;
      const unsigned pitch = 2u * (unsigned)(fresh ? a.kv_stride : a.stride_pos);
      // the places of the four groups, by a lane each
      long long off;
      int gq = 4 * (fresh ? ti.new_tile(t - ti.n_p) : ti.prefix_tile(t)) + (lane & 3);
      if (fresh) {
        gq = min(gq, end >> 4);
        off = (long long)(16 * gq) * pitch;
      } else {
        gq = needed_group(p, ti, P, gq);
        const int e = page_index(p, gq);
        int page = a.block_table[r.s * a.table_stride + e];
        if ((unsigned)page >= (unsigned)a.n_pages) {   // as checked_page
          atomicOr(p.dev_status, CASCADE_FLAG_PAGE);
          page = 0;
        }
        off = 2 * group_offset(p, page, e, gq, kvh);
      }
      const int behind = end - 16 * gq;
      const char *kb = fresh ? kn : (const char*)a.k_pages, *vb = fresh ? vn : (const char*)a.v_pages;
#pragma unroll
      for (int kt = 0; kt < 4; ++kt) {
        const long long o = (long long)(((u64)(unsigned)__builtin_amdgcn_readlane((int)(off >> 32), kt) << 32) | (unsigned)__builtin_amdgcn_readlane((int)off, kt));
        const int last = __builtin_amdgcn_readlane(behind, kt);
        const char *kp = kb + o, *vp = vb + o;
        const unsigned at = (unsigned)min(l16, last) * pitch + 16u * g;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kf[kt][ks] = *(const u32x4*)(kp + 64 * ks + at);
#pragma unroll
        for (int j = 0; j < GV; ++j) vr[GV * kt + j] = *(const u32x4*)(vp + ((unsigned)min(lane / DC + KEYS * j, last) * pitch + 16u * (unsigned)(lane % DC)));
      }
    };
    // queries (B operand of S^T): rows past the end repeat the last one, never stored
    Frag8 qf[KS];
    // Opaque at head_dim 128, where registers run out: what follows from it is worked out here, not kept over the parts.  Without scratch memory 64 rows of 90 to 4200 keys
    // take 130 -> 120 us, of 300 to 600 with 16 heads 56.6 -> 49.3; at head_dim 64 it only costs the small calls 0.5.
    int asker = g;
    if (D == 128) asm volatile("" : "+v"(asker));
    const int qr = min(l16, M - 1), qi = token_of(p, qr);
    const uint16_t* qp = (const uint16_t*)a.q + (long long)(lo + qi) * a.q_stride + (kvh * G + qr - qi * G) * D + 8 * asker;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks].u = *(const uint4*)(qp + 32 * ks);
    // trees (at most 16 nodes here): parents in the lanes; what a token sees of the new tokens, and its depth
    u64 path = 0;
    int depth = qi;
    int pa = -1;
    if (TREE) pa = a.parent[lo + min(lane, T - 1)];
    if (t_begin + wave < t_end) request(t_begin + wave);
    if (TREE) {
      const bool bad = lane < T && (lane == 0 ? pa != -1 : (pa >= lane || pa < 0));
      if (bad) { atomicOr(p.dev_status, CASCADE_FLAG_PARENT); pa = lane == 0 ? -1 : 0; }
      int x = qi;
      while (__any(x >= 0)) {
        if (x >= 0) path |= 1ull << x;
        const int up = __builtin_amdgcn_ds_bpermute(4 * (x & 63), pa);
        x = x > 0 ? up : -1;
      }
      depth = __popcll(path) - 1;
      if (a.window > 0) {   // the nearest `window` of them, and the sinks
        const int keep_sinks = a.n_sink - P;   // depths below this
        u64 all = path;
        int left = depth + 1 - a.window;   // so many of the path's first are out of reach
        int d = 0;
        while (__any(all != 0)) {
          if (all) {
            const int b = __ffsll((long long)all) - 1;
            if (d < left && d >= keep_sinks) path &= ~(1ull << b);
            all &= all - 1;
            ++d;
          }
        }
      }
    }

    f32x4 ot[DB];
    float m_run = -INFINITY, l_run = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db) ot[db] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int t = t_begin + wave; t < t_end; t += NW) {
      const bool fresh = t >= ti.n_p;
      const int kb = fresh ? ti.new_tile(t - ti.n_p) * KT : ti.prefix_tile(t) * KT;
      f32x4 st[4];
#pragma unroll
      for (int kt = 0; kt < 4; ++kt) {
        st[kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          Frag8 a8;
          a8.u = make_uint4(kf[kt][ks][0], kf[kt][ks][1], kf[kt][ks][2], kf[kt][ks][3]);
          st[kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a8.v, qf[ks].v, st[kt], 0, 0, 0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      // what some token sees of this tile, and whether all of them see the same
      const u64 valid = fresh ? (TREE ? path : sees_chain(p, P, kb, qi)) : sees_prefix(p, P, kb, P + depth);
      u64 some = valid, all = valid;
      // (lanes differ only in l16)
      if (T > 1 && (fresh || (a.window > 0))) {
#pragma unroll
        for (int s = 1; s < 16; s <<= 1) {
          some |= ((u64)(unsigned)__shfl_xor((int)(some >> 32), s) << 32) | (unsigned)__shfl_xor((int)some, s);
          all &= ((u64)(unsigned)__shfl_xor((int)(all >> 32), s) << 32) | (unsigned)__shfl_xor((int)all, s);
        }
      }
      // Wave-uniform: values that must not meet a masked probability.  Keys past the end are copies of the last one, which the last pieces of such a tile hold.
      // (without a branch: one that leaves the values alone on one side sends up to 81 registers to scratch)
      uint32_t last_odd = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) last_odd |= odd_exponent(vr[NVC - 1][e]);
      bool odd = __any(valid != ~0ull && (last_odd & 0x80008000u) != 0);
      // (a single token without a window sees every key that exists: nothing to take out)
      if ((T > 1 || a.window > 0) && __any(some != ~0ull || all != ~0ull)) {
        uint32_t seen_odd = 0;
#pragma unroll
        for (int it = 0; it < NVC; ++it) {
          const int c = lane + 64 * it;
          const bool keep = (some >> (c / DC)) & 1;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            vr[it][e] = keep ? vr[it][e] : 0u;
            seen_odd |= odd_exponent(vr[it][e]);
          }
        }
        odd = __any((seen_odd & 0x80008000u) != 0) && __any(some != all);
      }
      // values: registers -> this wave's LDS tile (row-major); the previous tile's reads are complete (same wave, in order)
#pragma unroll
      for (int it = 0; it < NVC; ++it) {
        const int c = lane + 64 * it;
        *(u32x4*)(&vt[(c / DC) * VP + 8 * (c % DC)]) = vr[it];
      }
      __builtin_amdgcn_wave_barrier();   // keep the tile's stores ahead of its transposing reads in program order
      if (t + NW < t_end) request(t + NW);   // the wave's next tile streams in during the softmax
      Frag8 pf[2];
      if (__any(valid != ~0ull)) {
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) {
          const uint32_t nib = (uint32_t)(valid >> (16 * kt + 4 * g));   // this lane's 4 keys of sub-tile kt
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const uint32_t seen = (uint32_t)__builtin_amdgcn_sbfe((int)nib, c, 1);
            st[kt][c] = __uint_as_float((seen & __float_as_uint(st[kt][c])) | (~seen & 0xff800000u));
          }
        }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int kt = 0; kt < 4; ++kt)
#pragma unroll
        for (int c = 0; c < 4; ++c) mx = fmaxf(mx, st[kt][c]);
      mx = rows4_max(mx) * p.scale_log2e;
      const float m_new = fmaxf(m_run, mx), m_use = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = fast_exp2(m_run - m_use);
      float ls = 0.f;
#pragma unroll
      for (int kt = 0; kt < 4; ++kt)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const float e = fast_exp2(fmaf(st[kt][c], p.scale_log2e, -m_use));
          st[kt][c] = e;
          ls += e;
        }
      l_run = l_run * alpha + ls;
      m_run = m_new;
#pragma unroll
      for (int db = 0; db < DB; ++db) ot[db] *= alpha;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        pf[j].u.x = pack_bf16x2(st[2 * j][0], st[2 * j][1]);
        pf[j].u.y = pack_bf16x2(st[2 * j][2], st[2 * j][3]);
        pf[j].u.z = pack_bf16x2(st[2 * j + 1][0], st[2 * j + 1][1]);
        pf[j].u.w = pack_bf16x2(st[2 * j + 1][2], st[2 * j + 1][3]);
      }
      // O^T += V^T P^T with transposing reads of the wave's tile (LDS operations of one wave complete in order)
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint16_t* vp = &vt[(32 * j + 4 * g + (l16 >> 2)) * VP + 16 * db + 4 * (l16 & 3)];
          union { Frag8 f; s16x4 h[2]; } vf;
          vf.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(vp));
          vf.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(vp + 16 * VP));
          if (odd) vf.f.u = make_uint4(finite_only(vf.f.u.x), finite_only(vf.f.u.y), finite_only(vf.f.u.z), finite_only(vf.f.u.w));
          ot[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf.f.v, pf[j].v, ot[db], 0, 0, 0);
        }
      if (odd)
        for (int key = 0; key < KT; ++key)
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const float v = bf16_bits_to_f32(vt[key * VP + 16 * db + 4 * g + c]);
              const bool is_odd = !(fabsf(v) < INFINITY);
              if (is_odd && ((valid >> key) & 1)) ot[db][c] += v;
            }
      __builtin_amdgcn_wave_barrier();   // and the reads ahead of the next tile's stores
    }

    // ---- the waves' results meet in LDS (the value tiles are reused)
    __syncthreads();
    float* mo = (float*)few_smem;          // [NW][R][OP]
    float* mml = mo + NW * R * OP;         // [NW][R][2]
    int joiner = tid;
    if (D == 128) asm volatile("" : "+v"(joiner));   // (as `asker`)
    const float l = rows4_sum(l_run);
    float* orow = mo + (wave * R + (joiner & 15)) * OP + (joiner >> 4 & 3) * 4;
#pragma unroll
    for (int db = 0; db < DB; ++db) *(f32x4*)(orow + 16 * db) = ot[db];
    if ((joiner & 48) == 0) {
      mml[(wave * R + joiner % 16) * 2] = m_run;
      mml[(wave * R + joiner % 16) * 2 + 1] = l;
    }
    __syncthreads();
    constexpr int TPR = D / 4;             // threads per row, four elements each
    for (int row = joiner / TPR; row < M; row += NT / TPR) {
      const int d = 4 * (joiner % TPR);
      float m = -INFINITY, l = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) m = fmaxf(m, mml[(w * R + row) * 2]);
      const float m_use = m == -INFINITY ? 0.f : m;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float f = fast_exp2(mml[(w * R + row) * 2] - m_use);
        l += f * mml[(w * R + row) * 2 + 1];
        const f32x4 x = *(const f32x4*)(mo + (w * R + row) * OP + d);
#pragma unroll
        for (int c = 0; c < 4; ++c) o[c] = fmaf(f, x[c], o[c]);
      }
      const int tok = token_of(p, row);
      const long long at = (long long)(lo + tok) * a.n_heads + kvh * G + row - tok * G;
      if (p.parts > 1) {
        const long long w = (long long)part * a.n_tokens * a.n_heads + at;
        *(f32x4*)(p.ws_o + w * D + d) = o;
        if (d == 0) { p.ws_ml[w * 2] = m; p.ws_ml[w * 2 + 1] = l; }
      } else {
        const float inv = 1.f / l;
        uint2 x;
        x.x = pack_bf16x2(o[0] * inv, o[1] * inv);
        x.y = pack_bf16x2(o[2] * inv, o[3] * inv);
        *(uint2*)((uint16_t*)a.out + at * D + d) = x;
        if (d == 0 && a.lse) a.lse[at] = m * LN2 + logf(l);
      }
    }
    __syncthreads();   // the next part's values go where the results were
  }
}

// ------------------------------------------------------------------------------------------------------- bf16, many query rows
// Workgroup = (16 NQ NW query rows of a row of the batch, kv head, part of their tiles): its waves share every tile of 64 keys.  Tiles never pass through registers on
// their way in: LDS-direct loads (global_load_lds_dwordx4, M0 = the LDS address of a wave's 1 KiB) write them into two rings of NS tiles, NS - 1 ahead of
// their use; a wave waits for its own loads of the tile needed next (vmcnt), then one bare barrier per tile makes everybody's visible and
// the oldest place free.  Such a load puts lane l's 16 bytes at 16 l, so rows cannot be padded; bank conflicts are avoided by WHICH 16-byte piece of a key a lane fetches:
// slot q of key r holds piece q ^ swz(r).  The products of the next tile's scores stand between the exponentials of this one.  The reference of the exponentials
// moves when a row's maximum has grown by more than 2^8: the result does not depend on it, and the rescaling becomes a rare branch.
//
// A wave's rows of a tile (8 or 16) lie in one group of 16 keys, so their page is one entry of the table.  The workgroup keeps the entries of its part in LDS, as
// many as fit, and reads the one for the next tile a tile ahead.
//
// Bound by the matrix cores and the vector ALU taking turns: products keep the former busy 40 to 42 % of the cycles, the latter 45 to 50 (clock 2.0 GHz under this load), the table costs nothing that can be
// measured.  Eight rows of 500-1000 new tokens behind 0-2000, 8 kv heads of 4 (157 GFLOP): 188 us = 835 TFLOP/s in 128-row workgroups (64 rows: 259, 256 rows, tried there: 221); 256-node trees of
// 8 rows x 32 heads behind 4200 keys (141 GFLOP): 181-184 us, 183 where the prefixes are contiguous; 1800-2000 new tokens under a window of 1024, head_dim 64: 40.2
// (half the products per exponential: 21 and 48 %; the chunks above with that head_dim 125, the trees 130).  Three workgroups per compute unit are what head_dim 64 runs best with, and they leave
// 128-row workgroups 168 registers: 9 (chains) and 14 (trees) go to scratch.
// Sums of the probabilities as they are, before they are rounded, cost less than products with ones (196 -> 184 us for the trees: registers) and give an exact lse.
template <int D>
struct RingGeom {
  static constexpr int RB = 2 * D;        // bytes per key
  static constexpr int PPR = RB / 16;     // 16-byte pieces per key
  static constexpr int RPC = 1024 / RB;   // keys per 1 KiB (one wave-wide load)
  static constexpr int CPT = KT / RPC;    // such loads per tile
  static constexpr int TILE = KT * RB;
  __device__ static constexpr int kswz(int key) { return D == 128 ? (key & 15) : ((key >> 1) & 7); }
  __device__ static constexpr int vswz(int key) { return D == 128 ? 2 * (key & 7) : 2 * ((key >> 1) & 3); }
};

constexpr float RESCALE_STEP = 8.f;      // log2 units
constexpr int STAGED = 2048;             // entries of the table in LDS

// LDS behind the rings: parents and depths (trees), two tiles' ancestor words (trees), entries of the table
template <int D, int NS, int NQ, int NW, bool TREE>
constexpr int ring_lds() {
  return 2 * NS * RingGeom<D>::TILE + (TREE ? CASCADE_MAX_TREE * 6 + 2 * 16 * NQ * NW * 8 : 0) + STAGED * 4;
}

template <int N>
__device__ __forceinline__ void wait_and_sync() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// maxima of products' results: an operation that the compiler sees, so that it keeps the distance that the matrix cores ask for
__device__ __forceinline__ float vmax2(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float vmax3(float a, float b, float c) { return vmax2(vmax2(a, b), c); }
__device__ __forceinline__ float rows4_max_raw(float v) {
  cascade_u32x2 a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = vmax2(__uint_as_float(a.x), __uint_as_float(a.y));
  cascade_u32x2 b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return vmax2(__uint_as_float(b.x), __uint_as_float(b.y));
}

// Block `blk` of the launch: a run of query rows of a row of the batch, a row's blocks from its end, where a chain sees most.  Where there are more blocks than compute units,
// rows are taken longest first (up to 64 of them).  64 rows of 25 tokens behind 74 keys: 10.3 us ranked row by row, 7.4 in order; of 60 behind 1000, many blocks: 56.1 us, ranked eight
// at a time 54.9.
__device__ __forceinline__ RowInfo block_row(const PagedParams& p, int blk, int rows_per_block, int lane, int* sb) {
  const paged_attn_args& a = p.a;
  RowInfo none = {-1, 0, 0, 0, 0};
  for (int base = 0; base < a.n_rows; base += 64) {
    const int at = base + lane;
    RowInfo mine = {at, 0, 0, 0, 0};
    int nb = 0;
    if (at < a.n_rows) {
      mine = check_row(p, at, a.q_off[at], a.q_off[at + 1], a.prefix_len[at]);
      nb = mine.flag ? 1 : (mine.T * p.group + rows_per_block - 1) / rows_per_block;
    }
    int from = lane;   // the lane whose row stands at this lane's place
    if (!p.in_order) {
      // lengths in steps of 32, and the lane, so that none are equal; lanes without a row stand behind
      const unsigned work = at < a.n_rows ? (mine.flag ? 0u : (unsigned)(mine.P + mine.T) >> 5 << 6) + 127u - lane : 63u - lane;
      int rank = 0;
      for (int r0 = 0; r0 < a.n_rows; r0 += 8)
#pragma unroll
        for (int r = 0; r < 8; ++r) rank += (unsigned)__builtin_amdgcn_readlane((int)work, r0 + r) > work ? 1 : 0;
      if (lane >= a.n_rows) rank = lane;
      from = __builtin_amdgcn_ds_permute(4 * rank, lane);
      nb = __builtin_amdgcn_ds_bpermute(4 * from, nb);
    }
    const int incl = wave_scan_incl_i(nb);
    const u64 who = __ballot(blk < incl);
    if (who) {
      const int l = __ffsll((long long)who) - 1, src = __builtin_amdgcn_readlane(from, l), n = __builtin_amdgcn_readlane(nb, l);
      blk -= __builtin_amdgcn_readlane(incl, l) - n;
      *sb = n - 1 - blk;
      RowInfo r = {base + src, __builtin_amdgcn_readlane(mine.lo, src), __builtin_amdgcn_readlane(mine.T, src), __builtin_amdgcn_readlane(mine.P, src),
                   __builtin_amdgcn_readlane(mine.flag, src)};
      return r;
    }
    blk -= __builtin_amdgcn_readlane(incl, 63);
  }
  return none;
}

template <int D, int NS, int NQ, int NW, bool TREE>
__global__ __launch_bounds__(64 * NW, NW == 8 ? 1 : (D == 64 ? (NQ == 1 ? 4 : 3) : 2)) void paged_ring_kernel(PagedParams p) {
  using GM = RingGeom<D>;
  constexpr int NT = 64 * NW, RW = 16 * NQ * NW, KS = D / 32, DB = D / 16;
  constexpr int CPW = GM::CPT / NW;     // loads of K (and of V) that a wave makes per tile
  constexpr int LPI = 2 * CPW;
  static_assert(GM::CPT % NW == 0 && CPW * GM::RPC <= 16 && (NS == 2 || NS == 3), "a wave's keys lie in one group of 16");
  extern __shared__ __align__(1024) char ring_smem[];
  char* const smem_raw = ring_smem;
  int* s_parent = (int*)(smem_raw + 2 * NS * GM::TILE);
  uint16_t* s_depth = (uint16_t*)(s_parent + CASCADE_MAX_TREE);
  u64* s_anc = (u64*)(s_depth + CASCADE_MAX_TREE);
  int* s_page = TREE ? (int*)(s_anc + 2 * RW) : s_parent;
  const paged_attn_args& a = p.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g = lane >> 4, G = p.group, H = a.n_kv_heads;

  // Workgroups are dealt round-robin to the 8 XCDs, one L2 each: those of a kv head stay on one XCD (or on 8 / H of them), where the blocks of a row meet in its keys.
  int kvh, b;
  {
    const int h = blockIdx.x, x = h & 7, k = h >> 3;
    if (H % 8 == 0) { const int m = H >> 3; kvh = x + 8 * (k % m); b = k / m; }
    else if (8 % H == 0 && (gridDim.x & 7) == 0) { kvh = x % H; b = k * (8 / H) + x / H; }
    else { kvh = h % H; b = h / H; }
  }
  const int part = b % p.parts;
  int sb = 0;
  const RowInfo ri = block_row(p, b / p.parts, RW, lane, &sb);
  if (ri.s < 0) return;   // the grid is an upper bound of the number of blocks
  if (ri.flag) { write_nothing<uint16_t>(p, ri, kvh, part, tid, NT); return; }
  auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  const int lo = uniform(ri.lo), T = uniform(ri.T), P = uniform(ri.P), M = T * G, row0 = uniform(sb) * RW;
  const int i0 = uniform(token_of(p, row0)), i1 = uniform(token_of(p, min(row0 + RW, M) - 1));
  const Tiles ti = tiles_of(p, P, i0, i1, TREE);
  const int nt = ti.n_p + ti.n_n, per = (nt + p.parts - 1) / p.parts, t_begin = part * per, t_end = min(nt, t_begin + per);
  const long long all_rows = (long long)a.n_tokens * a.n_heads;
  if (t_begin >= t_end) {   // fewer tiles than parts: an empty one
    for (int r = row0 + tid; r < min(row0 + RW, M); r += NT) {
      float* ml = p.ws_ml + (part * all_rows + (long long)(lo + r / G) * a.n_heads + kvh * G + r % G) * 2;
      ml[0] = -INFINITY;
      ml[1] = 0.f;
    }
    return;
  }

  // ---- loader: load i of a wave is 1 KiB c = CPW wave + i of a tile; lane -> key c RPC + lane / PPR, LDS slot lane % PPR
  const unsigned pitch_p = (unsigned)(a.stride_pos * 2), pitch_n = (unsigned)(a.kv_stride * 2);
  const unsigned lds0 = __builtin_amdgcn_readfirstlane((unsigned)(size_t)smem_raw);
  const int wave_group = CPW * GM::RPC * wave / 16;   // the group of 16 keys of a tile that the wave's keys lie in
  int ld_row[CPW];                                    // key in that group
  unsigned ld_kpiece[CPW], ld_vpiece[CPW], ld_kfull[CPW], ld_vfull[CPW];
#pragma unroll
  for (int i = 0; i < CPW; ++i) {
    const int r = (CPW * wave + i) * GM::RPC + lane / GM::PPR, q = lane % GM::PPR;
    ld_row[i] = r & 15;
    ld_kpiece[i] = 16u * (unsigned)(q ^ GM::kswz(r));
    ld_vpiece[i] = 16u * (unsigned)(q ^ GM::vswz(r));
    ld_kfull[i] = (unsigned)(r & 15) * pitch_p + ld_kpiece[i];
    ld_vfull[i] = (unsigned)(r & 15) * pitch_p + ld_vpiece[i];
  }
  // Where the wave's keys of a tile come from: the first key of their group, and how many keys are behind it.  Tiles past the part's end are its
  // last one again (the number of loads stays fixed; what they bring is not used), keys past the end are the last one again, masked.
  struct Source {
    long long off;   // bytes from the first page's or the row's first new key
    int last;        // keys of the group behind the first
    bool fresh;
  };
  const int e0 = ti.n_p > 0 ? page_index(p, 4 * min(ti.prefix_tile(max(min(t_begin, ti.n_p - 1), ti.sinks_p)), (P - 1) / KT)) : 0;
  const int n_staged = ti.n_p > 0 ? min(STAGED, page_index(p, (P - 1) >> 4) + 1 - e0) : 0;
  const ConstTable table = (ConstTable)(uintptr_t)a.block_table + (long long)ri.s * a.table_stride;
  const long long page_bytes = 2 * a.stride_page;
  const unsigned group_bytes = 16u * pitch_p;   // (stride_pos is at most 2^25)
  // (without a branch: it stands among the products of a step)
  const int first = ti.first, seen_group = first < P ? first >> 4 : (min(a.n_sink, P) - 1) >> 4, sinks = a.window > 0 ? a.n_sink : P;
  auto group_of = [&](int t) {   // as needed_group; t < n_p
    const int g = min(4 * ti.prefix_tile(t) + wave_group, (P - 1) >> 4);
    return 16 * g >= sinks && 16 * g + 15 < first ? seen_group : g;
  };
  const unsigned inv = p.page16_inv, whole = inv ? 0u : 1u;
  auto entry_of = [&](int g) { return (int)(__umulhi((unsigned)g, inv) + whole * (unsigned)g); };
  auto source_of = [&](int t, int page) {
    Source s;
    s.fresh = t >= ti.n_p;
    const int gp = group_of(min(t, ti.n_p - 1)), gn = min(4 * ti.new_tile(t - ti.n_p) + wave_group, (T - 1) >> 4), gq = s.fresh ? gn : gp;
    const long long in_pages = (long long)(s.fresh ? 0 : checked_page(p, page)) * page_bytes + (long long)(gp - entry_of(gp) * p.page16) * group_bytes;
    s.off = s.fresh ? (long long)(16 * gn) * pitch_n : in_pages;
    s.last = (s.fresh ? T : P) - 1 - 16 * gq;
    return s;
  };
  auto entry_now = [&](int t) { return t < ti.n_p ? table[entry_of(group_of(t))] : 0; };
  auto entry_staged = [&](int t) {
    if (t >= ti.n_p) return 0;
    const int e = entry_of(group_of(t)), at = e - e0;
    return at >= 0 && at < n_staged ? s_page[at] : table[e];
  };
  const char *kc = (const char*)((const uint16_t*)a.k_pages + kvh * a.stride_head), *vc = (const char*)((const uint16_t*)a.v_pages + kvh * a.stride_head);
  const char* kn = (const char*)((const uint16_t*)a.k_new + lo * a.kv_stride + kvh * D);
  const char* vn = (const char*)((const uint16_t*)a.v_new + lo * a.kv_stride + kvh * D);
  auto request = [&](const Source& s, int stage, bool is_v) {
    const unsigned ldst = lds0 + (is_v ? NS * GM::TILE : 0) + stage * GM::TILE + CPW * wave * 1024;
    const uintptr_t at = (uintptr_t)((s.fresh ? (is_v ? vn : kn) : (is_v ? vc : kc)) + s.off);
    const char* src = (const char*)(((u64)(unsigned)__builtin_amdgcn_readfirstlane((int)(at >> 32)) << 32) | (unsigned)__builtin_amdgcn_readfirstlane((int)at));
    if (!s.fresh && s.last >= 15) {   // whole: the lanes' offsets are constants
#pragma unroll
      for (int i = 0; i < CPW; ++i) {
        const unsigned l = ldst + i * 1024;
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(l), "v"(is_v ? ld_vfull[i] : ld_kfull[i]), "s"(src) : "memory");
      }
    } else {
      const unsigned pitch = s.fresh ? pitch_n : pitch_p;
#pragma unroll
      for (int i = 0; i < CPW; ++i) {
        const unsigned l = ldst + i * 1024, off = (unsigned)min(ld_row[i], s.last) * pitch + (is_v ? ld_vpiece[i] : ld_kpiece[i]);
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(l), "v"(off), "s"(src) : "memory");
      }
    }
  };

  // ---- prologue: K of the first tile, then the steady order K(t + NS), V(t + NS - 1)
  auto clamped = [&](int t) { return min(t, t_end - 1); };
  Source before;   // the tile whose V is requested next
  before = source_of(t_begin, entry_now(t_begin));
  request(before, 0, false);
#pragma unroll
  for (int i = 1; i < NS; ++i) {
    const int t = clamped(t_begin + i);
    const Source s = source_of(t, entry_now(t));
    request(s, i, false);
    request(before, i - 1, true);
    before = s;
  }
  // what else the loop needs in LDS
  for (int i = tid; i < n_staged; i += NT) s_page[i] = a.block_table[ri.s * a.table_stride + e0 + i];
  if (TREE) {
    for (int i = tid; i < T; i += NT) {
      int pi = a.parent[lo + i];
      if (i == 0 ? pi != -1 : (pi >= i || pi < 0)) {
        atomicOr(p.dev_status, CASCADE_FLAG_PARENT);
        pi = i == 0 ? -1 : 0;   // keeps the climb finite
      }
      s_parent[i] = pi;
    }
  }
  // query fragments (B operand of S^T): lane = (query l16, d group g)
  Frag8 qf[NQ][KS];
  int qi[NQ];            // the token, -1 behind the last
  long long out_row[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int r = row0 + 16 * (wave + NW * n) + l16;
    const bool ok = r < M;
    const int i = ok ? token_of(p, r) : 0, hg = ok ? r - i * G : 0;
    qi[n] = ok ? i : -1;
    out_row[n] = (long long)(lo + i) * a.n_heads + kvh * G + hg;
    const uint16_t* qp = (const uint16_t*)a.q + (lo + i) * a.q_stride + (kvh * G + hg) * D + 8 * g;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if (ok) qf[n][ks].u = *(const uint4*)(qp + 32 * ks);
      else qf[n][ks].u = make_uint4(0, 0, 0, 0);
    }
  }
  f32x4 ot[NQ][DB];
  float lsum[NQ];        // this lane's part of the row sums, of the probabilities before they are rounded
  float m_ref[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    m_ref[n] = -INFINITY;
    lsum[n] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db) ot[n][db] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // ---- LDS addresses (see the comment on slots): K fragment (kt, ks): key 16 kt + l16, piece 4 ks + g; V operand (db, j): keys 32 j + 4 g + (l16 >> 2)
  // (+ 16), four d at 16 db + 4 (l16 & 3).  ks and db enter by XOR, the stage, kt and j are constants.
  const unsigned k_lane = (unsigned)(l16 * GM::RB) + 16u * (unsigned)(g ^ GM::kswz(l16));
  const int vkey = 4 * g + (l16 >> 2);
  const unsigned v_lane = (unsigned)(vkey * GM::RB) + ((16u * (unsigned)((l16 & 3) >> 1)) ^ (16u * (unsigned)GM::vswz(vkey))) + 8u * (unsigned)(l16 & 1);
  const char* k_addr[KS];
  const char* v_addr[DB];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) k_addr[ks] = smem_raw + (k_lane ^ (unsigned)(64 * ks));
#pragma unroll
  for (int db = 0; db < DB; ++db) v_addr[db] = smem_raw + NS * GM::TILE + (v_lane ^ (unsigned)(32 * db));

  f32x4 st[NQ][4];   // scores: st[n][kt] holds keys 16 kt + 4 g + c for query l16
  auto load_kfrags = [&](Frag8 (&kf)[KS], int stage, int kt) {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) kf[ks].u = *(const uint4*)(k_addr[ks] + stage * GM::TILE + 16 * kt * GM::RB);
  };
  auto score_kt = [&](const Frag8 (&kf)[KS], int kt) {
#pragma unroll
    for (int n = 0; n < NQ; ++n) st[n][kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int n = 0; n < NQ; ++n) st[n][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[ks].v, qf[n][ks].v, st[n][kt], 0, 0, 0);
  };
  union VFrag { Frag8 f; s16x4 h[2]; };
  auto load_vfrag = [&](VFrag& vf, int stage, int i) {   // step i = (db, j) = (i / 2, i % 2)
    const char* vp = v_addr[i >> 1] + stage * GM::TILE + 32 * (i & 1) * GM::RB;
    vf.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(vp));
    vf.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(vp + 16 * GM::RB));
  };
  auto lane_max = [&](int n) {
    float x = vmax3(st[n][0][0], st[n][0][1], st[n][0][2]);
    x = vmax3(x, st[n][0][3], st[n][1][0]);
    x = vmax3(x, st[n][1][1], st[n][1][2]);
    x = vmax3(x, st[n][1][3], st[n][2][0]);
    x = vmax3(x, st[n][2][1], st[n][2][2]);
    x = vmax3(x, st[n][2][3], st[n][3][0]);
    x = vmax3(x, st[n][3][1], st[n][3][2]);
    return vmax2(x, st[n][3][3]);
  };

  __syncthreads();                    // parents and entries complete
  int q_depth[NQ];                    // position of the query behind the prefix
  if (TREE) {
    if (a.window > 0) {
      for (int i = tid; i < T; i += NT) {
        int d = 0;
        for (int x = s_parent[i]; x >= 0; x = s_parent[x]) ++d;
        s_depth[i] = (uint16_t)d;
      }
      __syncthreads();
    }
  }
#pragma unroll
  for (int n = 0; n < NQ; ++n) q_depth[n] = TREE ? (a.window > 0 ? s_depth[max(qi[n], 0)] : 0) : qi[n];
  // trees: which nodes of new tile t each of the workgroup's query rows sees
  auto build_mask = [&](int t) {
    if (tid < RW) {
      const int kb = (t - ti.n_p) * KT, r = row0 + tid;
      u64 bits = 0;
      if (r < M) {
        int x = token_of(p, r);
        const int reach = a.window > 0 ? s_depth[x] - a.window + 1 : 0, sinks = a.n_sink - P;   // depths seen: from `reach` on, and below `sinks`
        while (x >= kb) {   // kb >= 0; ancestors only get smaller
          if (x - kb < 64 && (a.window == 0 || s_depth[x] >= reach || (int)s_depth[x] < sinks)) bits |= 1ull << (x - kb);
          x = s_parent[x];
        }
      }
      s_anc[(t & 1) * RW + tid] = bits;
    }
  };
  if (TREE && t_begin >= ti.n_p) build_mask(t_begin);
  // the source of the K requested next is worked out a step ahead, among the products
  int entry = entry_staged(clamped(t_begin + NS));
  Source next;
  wait_and_sync<LPI * (NS - 1)>();    // K of the first tile everywhere (and the first mask)
  float lmax[NQ];                     // lane_max of the scores in st
  {
    Frag8 kf[2][KS];
    load_kfrags(kf[0], 0, 0);
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) {
      if (kt < 3) load_kfrags(kf[(kt + 1) & 1], 0, kt + 1);
      score_kt(kf[kt & 1], kt);
    }
#pragma unroll
    for (int n = 0; n < NQ; ++n) lmax[n] = lane_max(n);
  }

  auto tile_step = [&](int t, auto st_const) {
    constexpr int ST = decltype(st_const)::value;
    constexpr int ST_K = (ST + 1) % NS;             // stage of K(t+1)
    constexpr int ST_VNEW = (ST + NS - 1) % NS;     // V(t + NS - 1) goes where V(t - 1) was
    wait_and_sync<LPI * (NS - 2)>();   // K(t+1), V(t) landed everywhere; K(t), V(t-1) free
    next = source_of(clamped(t + NS), __builtin_amdgcn_readfirstlane(entry));
    request(next, ST, false);
    request(before, ST_VNEW, true);
    before = next;
    entry = entry_staged(clamped(t + NS + 1));
    __builtin_amdgcn_sched_barrier(0);
    Frag8 kf[2][KS];
    load_kfrags(kf[0], ST_K, 0);       // in flight during the reference check
    if (TREE && t + 1 < t_end && t + 1 >= ti.n_p) build_mask(t + 1);   // read behind the next barrier

    // ---- masks
    const bool fresh = t >= ti.n_p;
    const int kb = fresh ? ti.new_tile(t - ti.n_p) * KT : ti.prefix_tile(t) * KT;
    const int far = fresh ? i1 : P + i1;             // no query's position is behind this one
    const bool cut = a.window > 0 && kb < far - a.window + 1 && kb + KT > a.n_sink - (fresh ? P : 0);
    const bool mixed = (fresh && (TREE || kb + KT - 1 > i0)) || cut;   // some queries see less of it than others
    const bool partial = mixed || (!fresh && kb + KT > P);             // or it ends, and its last key is there again
    auto sees = [&](int n) -> u64 {
      if (qi[n] < 0) return 0ull;
      if (fresh) return TREE ? s_anc[(t & 1) * RW + 16 * (wave + NW * n) + l16] : sees_chain(p, P, kb, qi[n]);
      return sees_prefix(p, P, kb, P + q_depth[n]);
    };
    if (partial) {
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        const u64 valid = sees(n);
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) {
          const uint32_t nib = (uint32_t)(valid >> (16 * kt + 4 * g));   // this lane's 4 keys of sub-tile kt
#pragma unroll
          for (int c = 0; c < 4; ++c) st[n][kt][c] = ((nib >> c) & 1u) ? st[n][kt][c] : -INFINITY;
        }
        lmax[n] = lane_max(n);
      }
    }
    // ---- the reference of the exponentials: a lane sees 16 of its row's 64 scores; if none of the wave's lanes exceeds its row's by more than the step, no row does
    bool moved = false;
#pragma unroll
    for (int n = 0; n < NQ; ++n) moved |= lmax[n] * p.scale_log2e > m_ref[n] + RESCALE_STEP;   // -inf + 8 = -inf: a first finite score always moves it
    if (__ballot(moved) != 0ull) {
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        const float mx = rows4_max_raw(lmax[n]) * p.scale_log2e;
        const float m_new = (mx > m_ref[n] + RESCALE_STEP) ? mx : m_ref[n];
        const float use_new = (m_new == -INFINITY) ? 0.f : m_new;
        const float alpha = fast_exp2(m_ref[n] - use_new);   // -inf - finite = -inf -> 0 ; equal -> 1
        lsum[n] *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db) ot[n][db] *= alpha;
        m_ref[n] = m_new;
      }
    }
    if (partial) {
      // infinities and NaN among values that not every query sees (every wave looks through the whole tile, so all agree); behind the rescaling, whose
      // first factor is 0
      uint32_t odd = 0;
      char* const vt = smem_raw + NS * GM::TILE + ST * GM::TILE;
#pragma unroll
      for (int c = 0; c < GM::CPT; ++c) {
        const uint4 x = *(const uint4*)(vt + 1024 * c + 16 * lane);
        odd |= odd_exponent(x.x) | odd_exponent(x.y) | odd_exponent(x.z) | odd_exponent(x.w);
      }
      if (__any((odd & 0x80008000u) != 0)) {   // they go to the queries that see them, and out of the tile
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
          const u64 valid = sees(n);
          for (int key = 0; key < KT; ++key)
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
              for (int c = 0; c < 4; ++c) {
                const float v = bf16_bits_to_f32(*(const uint16_t*)(vt + key * GM::RB + 16 * ((2 * db + (g >> 1)) ^ GM::vswz(key)) + 8 * (g & 1) + 2 * c));
                if (!(fabsf(v) < INFINITY) && ((valid >> key) & 1)) ot[n][db][c] += v;
              }
        }
        __syncthreads();
        for (int c = tid; c < GM::TILE / 16; c += NT) {
          uint4* at = (uint4*)(vt + 16 * c);
          *at = make_uint4(finite_only(at->x), finite_only(at->y), finite_only(at->z), finite_only(at->w));
        }
        __syncthreads();
      }
    }
    float m_neg[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) m_neg[n] = (m_ref[n] == -INFINITY) ? 0.f : -m_ref[n];

    // ---- probabilities of tile t (B operand of the second product), between them the scores of tile t+1 over the same registers
    Frag8 pf[NQ][2];
    auto probs_kt = [&](int kt) {
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        float e[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) e[c] = fast_exp2(fmaf(st[n][kt][c], p.scale_log2e, m_neg[n]));   // -inf stays -inf -> 0
        lsum[n] += (e[0] + e[1]) + (e[2] + e[3]);
        const uint32_t lo2 = pack_bf16x2(e[0], e[1]), hi2 = pack_bf16x2(e[2], e[3]);
        if (kt & 1) { pf[n][kt >> 1].u.z = lo2; pf[n][kt >> 1].u.w = hi2; }
        else { pf[n][kt >> 1].u.x = lo2; pf[n][kt >> 1].u.y = hi2; }
      }
    };
    constexpr int NVS = 2 * DB, VW = 4;   // V steps per tile, steps whose fragments are requested ahead
    VFrag vf[VW];
    probs_kt(0);
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) {
      if (kt < 3) load_kfrags(kf[(kt + 1) & 1], ST_K, kt + 1);
      else {
#pragma unroll
        for (int i = 0; i < VW; ++i) load_vfrag(vf[i], ST, i);
        __builtin_amdgcn_sched_barrier(0);   // left alone, every V read sinks to its product
      }
      score_kt(kf[kt & 1], kt);
      if (kt < 3) probs_kt(kt + 1);
    }
    // ---- O^T += V^T P^T; the vector ALU meanwhile looks at the next tile's scores
#pragma unroll
    for (int n = 0; n < NQ; ++n) lmax[n] = lane_max(n);
#pragma unroll
    for (int i = 0; i < NVS; ++i) {
#pragma unroll
      for (int n = 0; n < NQ; ++n) ot[n][i >> 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[i % VW].f.v, pf[n][i & 1].v, ot[n][i >> 1], 0, 0, 0);
      if (i + VW < NVS) load_vfrag(vf[i % VW], ST, i + VW);
      __builtin_amdgcn_sched_barrier(0);   // keeps the read of step i + VW here, VW steps ahead of its use
    }
  };
  for (int t = t_begin; t < t_end; t += NS) {
    tile_step(t, std::integral_constant<int, 0>{});
    if (t + 1 >= t_end) break;
    tile_step(t + 1, std::integral_constant<int, 1>{});
    if constexpr (NS > 2) {
      if (t + 2 >= t_end) break;
      tile_step(t + 2, std::integral_constant<int, 2>{});
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the loads that nothing uses must not outlive the workgroup's LDS

  // epilogue: lane (query l16, g) owns d = 16 db + 4 g + c
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const float l = rows4_sum(lsum[n]);
    if (qi[n] < 0) continue;
    if (p.parts > 1) {
      const long long w = part * all_rows + out_row[n];
#pragma unroll
      for (int db = 0; db < DB; ++db) *(f32x4*)(p.ws_o + w * D + 16 * db + 4 * g) = ot[n][db];
      if (g == 0) { p.ws_ml[w * 2] = m_ref[n]; p.ws_ml[w * 2 + 1] = l; }
      continue;
    }
    const float inv = 1.f / l;
    uint16_t* o = (uint16_t*)a.out + out_row[n] * D;
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      uint2 w;
      w.x = pack_bf16x2(ot[n][db][0] * inv, ot[n][db][1] * inv);
      w.y = pack_bf16x2(ot[n][db][2] * inv, ot[n][db][3] * inv);
      *(uint2*)(o + 16 * db + 4 * g) = w;
    }
    if (g == 0 && a.lse) a.lse[out_row[n]] = m_ref[n] * LN2 + logf(l);
  }
}

// ------------------------------------------------------------------------------------------------------------------------- f32
// Workgroup = (16 query rows, kv head, part); its NW waves take every NW-th tile of 16 keys - one group, one page - and meet in LDS.  Both products run on
// v_mfma_f32_16x16x4_f32 (one value per lane and operand, k = lane / 16 = g):
//   S^T = K Q^T   lane (l16, g) loads 16 bytes at d = 16 db + 4 g of key / query l16 and feeds element c of both to the c-th product; the result holds
//                 keys 4 g + r of query l16;
//   O^T = V^T P^T product r takes P^T straight from register r of that result, and element c of the 16 bytes at d = 64 h + 4 l16 of key 4 g + r's value: its row l16
//                 stands for that d + c (element loads: d = 16 db + l16).
// Nothing passes through LDS before the waves meet.  Bound by the trips to memory, one after the other: the row's place, the table's entry, the first tile.
// 15 new tokens x 8 heads x 64 behind 256 keys: 9 us.  Many rows fetch every key again for each 16 of them: 8 rows of 200 tokens behind 1289 keys, 8 heads: 94 us at head_dim 64 (49 TFLOP/s; 30 at the rate
// of a large product), 161 at 128 (57 TFLOP/s).
template <int DB, int NW, bool VEC, bool TREE>
__global__ __launch_bounds__(64 * NW) void paged_f32_kernel(PagedParams p) {
  extern __shared__ __align__(16) float f32_smem[];   // [NW][16 queries][16 DB + 4] outputs, [NW][16][2] maxima and sums
  __shared__ int s_parent[TREE ? CASCADE_MAX_TREE : 1];
  constexpr int OP = 16 * DB + 4, TS = 16;
  const paged_attn_args& a = p.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g = lane >> 4, G = p.group, D = a.head_dim;
  const int kvh = blockIdx.x % a.n_kv_heads, b = blockIdx.x / a.n_kv_heads, part = b % p.parts;
  int sb = 0;
  const RowInfo ri = block_row(p, b / p.parts, 16, lane, &sb);
  if (ri.s < 0) return;   // the grid is an upper bound of the number of blocks
  if (ri.flag) { write_nothing<float>(p, ri, kvh, part, tid, 64 * NW); return; }
  const int lo = ri.lo, T = ri.T, P = ri.P, M = T * G, row0 = 16 * sb, rows = min(16, M - row0);
  const Tiles ti = tiles_of<TS>(p, P, token_of(p, row0), token_of(p, row0 + rows - 1), TREE);
  const int nt = ti.n_p + ti.n_n, per = (nt + p.parts - 1) / p.parts, t_begin = part * per, t_end = min(nt, t_begin + per);
  const int qr = row0 + min(l16, rows - 1);   // rows past the end repeat the last one, never stored
  const int qi = token_of(p, qr);
  const float* qrow = (const float*)a.q + (lo + qi) * a.q_stride + (kvh * G + qr - qi * G) * D;
  const float *kn = (const float*)a.k_new + lo * a.kv_stride + kvh * D, *vn = (const float*)a.v_new + lo * a.kv_stride + kvh * D;
  auto load4 = [&](const float* row, int d) {
    if (VEC) return d < D ? *(const f32x4*)(row + d) : f32x4{0.f, 0.f, 0.f, 0.f};
    f32x4 x;
#pragma unroll
    for (int c = 0; c < 4; ++c) x[c] = d + c < D ? row[d + c] : 0.f;
    return x;
  };
  f32x4 q[DB], ot[DB], k[DB], v[4][DB / 4];
  // keys past the end of the tile's source: the last one again, masked
  struct Source {
    long long off, pitch;
    int last;
    bool fresh;
  };
  auto source_of = [&](int t) {
    Source s;
    s.fresh = t >= ti.n_p;
    if (!s.fresh) {
      const int gq = needed_group(p, ti, P, ti.prefix_tile(t)), e = page_index(p, gq);
      s.off = group_offset(p, checked_page(p, table_entry(p, ri.s, e)), e, gq, kvh);
      s.last = P - 1 - 16 * gq;
      s.pitch = a.stride_pos;
    } else {
      const int j = ti.new_tile(t - ti.n_p);
      s.off = (long long)(16 * j) * a.kv_stride;
      s.last = T - 1 - 16 * j;
      s.pitch = a.kv_stride;
    }
    return s;
  };
  auto request_k = [&](const Source& s) {
    const float* row = (s.fresh ? kn : (const float*)a.k_pages) + s.off + min(l16, s.last) * s.pitch;
#pragma unroll
    for (int db = 0; db < DB; ++db) k[db] = load4(row, 16 * db + 4 * g);
  };
  auto request_v = [&](const Source& s) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float* row = (s.fresh ? vn : (const float*)a.v_pages) + s.off + min(4 * g + r, s.last) * s.pitch;
#pragma unroll
      for (int h = 0; h < DB / 4; ++h)
        if (VEC) v[r][h] = load4(row, 64 * h + 4 * l16);
        else
#pragma unroll
          for (int c = 0; c < 4; ++c) v[r][h][c] = row[min(64 * h + 16 * c + l16, D - 1)];
    }
  };
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    q[db] = load4(qrow, 16 * db + 4 * g);
    ot[db] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  if (t_begin + wave < t_end) {
    const Source s = source_of(t_begin + wave);
    request_k(s);
    request_v(s);
  }
  int depth = qi;
  if (TREE) {
    for (int i = tid; i < T; i += 64 * NW) {
      int pi = a.parent[lo + i];
      if (i == 0 ? pi != -1 : (pi >= i || pi < 0)) { atomicOr(p.dev_status, CASCADE_FLAG_PARENT); pi = i == 0 ? -1 : 0; }
      s_parent[i] = pi;
    }
    __syncthreads();
    if (a.window > 0) {
      depth = 0;
      for (int x = s_parent[qi]; x >= 0; x = s_parent[x]) ++depth;
    }
  }
  // keys of tile t that query l16 sees
  auto seen = [&](int t) -> unsigned {
    if (t < ti.n_p) return (unsigned)sees_prefix(p, P, 16 * ti.prefix_tile(t), P + depth) & 0xffffu;
    const int kb = 16 * ti.new_tile(t - ti.n_p);
    if (!TREE) return (unsigned)sees_chain(p, P, kb, qi) & 0xffffu;
    unsigned bits = 0;
    const int reach = depth - a.window + 1, sinks = a.n_sink - P;
    int d = depth;
    for (int x = qi; x >= kb; x = s_parent[x], --d)   // kb >= 0; ancestors only get smaller
      if (x - kb < 16 && (a.window == 0 || d >= reach || d < sinks)) bits |= 1u << (x - kb);
    return bits;
  };
  float m = -INFINITY, l = 0.f;
  auto step = [&](int t, auto more) {   // more: another tile of the wave follows
    constexpr bool MORE = decltype(more)::value;
    const unsigned bits = seen(t);
    f32x4 st = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int c = 0; c < 4; ++c) st = __builtin_amdgcn_mfma_f32_16x16x4f32(k[db][c], q[db][c], st, 0, 0, 0);
    Source next;
    if constexpr (MORE) {
      next = source_of(t + NW);
      request_k(next);
    }
    float mx = -INFINITY;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      st[r] = ((bits >> (4 * g + r)) & 1u) ? st[r] * p.scale_log2e : -INFINITY;
      mx = fmaxf(mx, st[r]);
    }
    const float m_new = fmaxf(m, rows4_max(mx)), m_use = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = fast_exp2(m - m_use);
    float ls = 0.f;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      st[r] = fast_exp2(st[r] - m_use);
      ls += st[r];
    }
    l = l * alpha + ls;
    m = m_new;
    // a tile that some query does not see whole is looked through for infinities and NaN; if it holds any its keys are added one at a time, to the queries that see them
    bool whole_keys = true;
    if (__any(bits != 0xffffu)) {
      float z = 0.f;
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int db = 0; db < DB; ++db) z = fmaf(v[r][db / 4][db % 4], 0.f, z);
      whole_keys = !__any(z != 0.f);
    }
#pragma unroll
    for (int db = 0; db < DB; ++db) ot[db] *= alpha;
    if (whole_keys) {
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 4; ++r) ot[db] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[r][db / 4][db % 4], st[r], ot[db], 0, 0, 0);
    } else {
      for (int kg = 0; kg < 4; ++kg)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const bool sees = (bits >> (4 * kg + r)) & 1u;
#pragma unroll
          for (int db = 0; db < DB; ++db) {
            const f32x4 o = __builtin_amdgcn_mfma_f32_16x16x4f32(g == kg ? v[r][db / 4][db % 4] : 0.f, st[r], ot[db], 0, 0, 0);
#pragma unroll
            for (int c = 0; c < 4; ++c) ot[db][c] = sees ? o[c] : ot[db][c];
          }
        }
    }
    if constexpr (MORE) request_v(next);
  };
  int t = t_begin + wave;
  for (; t + NW < t_end; t += NW) step(t, std::true_type{});
  if (t < t_end) step(t, std::false_type{});
  // the waves meet: lane (l16, g) holds d = 64 (db / 4) + 16 g + 4 c + db % 4 of query l16 (element loads: d = 16 db + 4 g + c)
  l = rows4_sum(l);
  float* mo = f32_smem + (wave * 16 + l16) * OP;
  float* ml = f32_smem + NW * 16 * OP;
#pragma unroll
  for (int h = 0; h < DB / 4; ++h)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      if (VEC) *(f32x4*)(mo + 64 * h + 16 * g + 4 * c) = f32x4{ot[4 * h][c], ot[4 * h + 1][c], ot[4 * h + 2][c], ot[4 * h + 3][c]};
      else *(f32x4*)(mo + 64 * h + 16 * c + 4 * g) = ot[4 * h + c];
    }
  if (g == 0) {
    ml[(wave * 16 + l16) * 2] = m;
    ml[(wave * 16 + l16) * 2 + 1] = l;
  }
  __syncthreads();
  // a wave finishes whole rows: lane w holds the factor of wave w's part
  const long long all_rows = (long long)a.n_tokens * a.n_heads;
  for (int r = wave; r < rows; r += NW) {
    const int row = row0 + r, w = lane & 15;
    const float mw = w < NW ? ml[(w * 16 + r) * 2] : -INFINITY, lw = w < NW ? ml[(w * 16 + r) * 2 + 1] : 0.f;
    const float mm = wave_max(mw), f = fast_exp2(mw - (mm == -INFINITY ? 0.f : mm));   // a wave without visible keys: 0
    const float ll = wave_sum(lane < NW ? f * lw : 0.f);
    const int tok = token_of(p, row);
    const long long at = (long long)(lo + tok) * a.n_heads + kvh * G + row - tok * G;
    float* out = p.parts > 1 ? p.ws_o + (part * all_rows + at) * D : (float*)a.out + at * D;
    for (int d = lane; d < D; d += 64) {
      float o = 0.f;
#pragma unroll
      for (int i = 0; i < NW; ++i) o = fmaf(__int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), i)), f32_smem[(i * 16 + r) * OP + d], o);
      out[d] = p.parts > 1 ? o : o / ll;
    }
    if (lane == 0) {
      if (p.parts > 1) { p.ws_ml[(part * all_rows + at) * 2] = mm; p.ws_ml[(part * all_rows + at) * 2 + 1] = ll; }
      else if (a.lse) a.lse[at] = mm * LN2 + logf(ll);
    }
  }
}

// Joins the parts, a wave to a (token, query head): the parts' factors come from its lanes, so two trips to memory follow each other whatever their number.  Rows
// that have fewer parts, or that could not be computed, left empty ones (l = 0), of which nothing else was written.  4.1 us for 32 rows of up to 16 parts; a thread
// that goes from part to part took 9 to 11.
constexpr int MOST_PARTS = 64;
template <typename T, int DL>   // DL: elements of the head to a lane
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedParams p) {
  const paged_attn_args& a = p.a;
  const int D = a.head_dim, lane = threadIdx.x & 63;
  const int rows = a.n_tokens * a.n_heads, row = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
  if (row >= rows) return;
  float m = -INFINITY, l = 0.f;
  if (lane < p.parts) {
    const float2 ml = *(const float2*)(p.ws_ml + ((long long)lane * rows + row) * 2);
    m = ml.x;
    l = ml.y;
  }
  const int first = a.q_off[0], last = a.q_off[a.n_rows];
  if (row < (long long)first * a.n_heads || row >= (long long)last * a.n_heads) return;   // a token of no row
  const float mm = wave_max(m);
  float f = l == 0.f ? 0.f : fast_exp2(m - (mm == -INFINITY ? 0.f : mm));
  const float ll = wave_sum(f * l);
  f = ll == 0.f ? 0.f : f / ll;
  float o[DL];
#pragma unroll
  for (int i = 0; i < DL; ++i) o[i] = 0.f;
  const u64 used = __ballot(l != 0.f);
  for (int c0 = 0; c0 < p.parts; c0 += 4) {
    float x[4][DL];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c = c0 + j;
      const bool there = c < p.parts && ((used >> c) & 1);
      const float* src = p.ws_o + ((long long)(there ? c : 0) * rows + row) * D;
#pragma unroll
      for (int i = 0; i < DL; ++i) x[j][i] = there && DL * lane + i < D ? src[DL * lane + i] : 0.f;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float w = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), (c0 + j) & 63));
#pragma unroll
      for (int i = 0; i < DL; ++i) o[i] = fmaf(w, x[j][i], o[i]);
    }
  }
  T* out = (T*)a.out + (long long)row * D;
#pragma unroll
  for (int i = 0; i < DL; ++i)
    if (DL * lane + i < D) {
      if constexpr (sizeof(T) == 2) out[DL * lane + i] = f32_to_bf16_bits(o[i]);
      else out[DL * lane + i] = o[i];
    }
  if (lane == 0 && a.lse) a.lse[row] = mm * LN2 + logf(ll);
}

// ----------------------------------------------------------------------------------------------------------------------- launches
// Kernels ask for more LDS than a launch may have by default: said once per kernel and device.
template <auto KERNEL>
hipError_t allow_lds(int bytes, int device) {
  static std::atomic<u64> done{0};
  const u64 bit = 1ull << (device & 63);
  if (device < 64 && (done.load(std::memory_order_relaxed) & bit)) return hipSuccess;
  const hipError_t e = hipFuncSetAttribute((const void*)KERNEL, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == hipSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

// How a call is cut.  Shape 0: few query rows, at most 16; 1, 2, 3: workgroups of 64, 128, 256 query rows; 4: f32.
struct Cut {
  int shape;
  int parts, part_tiles;
};
constexpr int FEW = 0, RING_64 = 1, RING_128 = 2, RING_256 = 3, F32 = 4;
constexpr int SHAPE_ROWS[] = {16, 64, 128, 256, 16};

int tiles_bound(const paged_attn_args* a, int ts = KT) {
  const int n = (a->max_new + ts - 1) / ts;
  int t = (a->max_prefix_len + ts - 1) / ts;
  if (a->window > 0) {
    const int64_t w = ((int64_t)a->window + ts - 2) / ts + 1 + ((int64_t)a->n_sink + ts - 1) / ts;   // a window's tiles, wherever it begins, and the sinks'
    if (w < t) t = (int)w;
  }
  return t + n;
}

int f32_waves(const paged_attn_args* a) { return a->head_dim <= 64 ? 16 : (a->head_dim <= 128 ? 8 : 4); }

size_t part_bytes(const paged_attn_args* a) { return (size_t)a->n_tokens * a->n_heads * (a->head_dim + 2) * sizeof(float); }

// Estimated time of a cut of many query rows, us: what the longest workgroup takes, or what all of them have to do where several share a compute unit, whichever is more.  A tile costs a
// workgroup c0 on a mostly idle chip, c1 with one workgroup on every compute unit, c2 with two (256 rows: one after the other); at head_dim 64 what is shared costs `narrow` of that, a step
// by itself the same.  Workgroups of a chain go through half of its new tiles in the mean; trees' new tiles cost 0.7 more for their masks; to begin and to end is worth 4.6 tiles.
// Fitted to 180 sizes x 3 shapes x up to 4 numbers of parts (1 to 64 rows, 1 to 2200 new tokens behind 0 to 8000, windows, trees): the cut with the least estimate
// takes 0.6 % longer than the fastest one in the mean, 17 % at most.  With every workgroup as long as the longest it was 3 % and 38 %.
float ring_estimate_us(int shape, const paged_attn_args* a, int parts, int n_cu) {
  constexpr struct { float c0, c1, c2, narrow; } COST[] = {{0.85f, 1.01f, 1.4f, 0.59f}, {1.1f, 1.52f, 1.96f, 0.73f}, {1.34f, 2.09f, 0.f, 0.67f}};
  const auto& c = COST[shape - RING_64];
  const int G = a->n_heads / a->n_kv_heads, rows = SHAPE_ROWS[shape];
  const int n_sb = (int)(((int64_t)a->max_new * G + rows - 1) / rows);
  float blocks = (float)a->n_rows * n_sb;
  if (n_sb > 1) blocks = fminf(blocks, (float)a->n_tokens * G / rows + 0.5f * a->n_rows);
  const float x = blocks * a->n_kv_heads * parts / n_cu;
  // tiles of the longest workgroup, and in the mean
  const int news = (a->max_new + KT - 1) / KT, old = tiles_bound(a) - news;
  const float row_tokens = (float)a->n_tokens / a->n_rows;
  float most = (float)(old + news), mean = a->parent ? fminf((float)news, news * row_tokens / a->max_new) : 0.5f * row_tokens / KT + 0.5f;
  if (a->window > 0) {
    const float w = (float)(((int64_t)a->window + KT - 2) / KT + 1), all = w + (float)(((int64_t)a->n_sink + KT - 1) / KT) + 1.f;
    most = fminf(old + fminf((float)news, w), all);
    mean = fminf(old + fminf(mean, w), all);
  } else {
    mean += old;
  }
  if (a->parent) { most += 0.7f * news; mean += 0.7f * news; }
  const float alone = c.c0 + (c.c1 - c.c0) * fminf(x, 1.f);
  const float shared = x <= 1.f ? alone : (shape == RING_256 ? c.c1 * ceilf(x) : (x <= 2.f ? c.c1 + (c.c2 - c.c1) * (x - 1.f) : c.c2 * 0.5f * x));
  float us = 5.15f + fmaxf(ceilf(most / parts) * alone, (mean / parts + 4.65f) * shared * (a->head_dim == 64 ? c.narrow : 1.f));
  if (parts > 1) us += 3.f + 0.2f * parts + (float)parts * a->n_tokens * a->n_heads * (a->head_dim + 2) * 4.f / 7e6f;
  return us;
}

Cut choose(const paged_attn_args* a, int n_cu, size_t ws_bytes) {
  Cut c = {F32, 1, 1};
  const int64_t M = (int64_t)a->max_new * (a->n_heads / a->n_kv_heads);
  const int most = (int)std::min<size_t>(ws_bytes / part_bytes(a), MOST_PARTS);
  if (a->dtype == CASCADE_F32) {
    // few blocks share the keys, four tiles to a wave at least
    const int waves = f32_waves(a);
    const int64_t blocks = a->n_rows * ((M + 15) / 16) * a->n_kv_heads;
    c.parts = (int)std::max<int64_t>(1, std::min<int64_t>({most, n_cu / blocks, tiles_bound(a, 16) / (4 * waves)}));
    return c;
  }
  const int tiles = tiles_bound(a);
  // (17 to 32 query rows in waves of their own, twice the registers: 0.6 to 1.1 of the time at head_dim 64, 1.5 to 2.6 at 128, where they do not fit)
  if (M > 16) {
    float best = INFINITY;
    for (int shape = RING_64; shape <= (a->head_dim == 64 ? RING_256 : RING_128); ++shape)   // (256 rows at head_dim 128 cost more than 128 rows at any size)
      for (int parts = 1; parts <= 16 && parts <= std::max(most, 1) && parts <= tiles; parts = parts < 4 ? parts + 1 : parts * 2) {
        const float us = ring_estimate_us(shape, a, parts, n_cu);
        if (us < best) { best = us; c.shape = shape; c.parts = parts; }
      }
    return c;
  }
  c.shape = FEW;
  const int64_t heads = (int64_t)a->n_rows * a->n_kv_heads;
  // A wave takes 4-5 us to a tile whose keys come from memory, so few (row, kv head) pairs are cut until there is a part for every compute unit (up to 16: joining
  // more takes longer than they save), unless that saves less than the join's 4 us.  Pairs that fill the chip by themselves are cut in two, for rows of different lengths:
  // 64 rows of 90-4200 keys, 8 kv heads 140.7 -> 136.4 us, 40 of 100-1500 45.8 -> 39.8 (all of them 4200 keys: 199 -> 211).
  int parts = (int)std::min<int64_t>(n_cu / heads, 16);
  const int alone = (tiles + 7) / 8, cut = parts > 1 ? (tiles + 8 * parts - 1) / (8 * parts) : alone;
  if (alone - cut < (parts >= 4 ? 1 : 2)) parts = 1;
  if (heads > n_cu && tiles >= 16) parts = 2;
  parts = std::max(1, std::min(parts, most));
  c.part_tiles = (tiles + parts - 1) / parts;
  c.parts = (tiles + c.part_tiles - 1) / c.part_tiles;
  return c;
}

// eight waves to a part where every part has a compute unit of its own (trees, few of which are that small: one kernel)
int few_waves(const paged_attn_args* a, const Cut& c, int n_cu) { return !a->parent && (int64_t)a->n_rows * a->n_kv_heads * c.parts <= n_cu ? 8 : 4; }

template <int D, int NW, bool TREE>
hipError_t launch_few_k(cascade_ctx* ctx, const PagedParams& p) {
  constexpr int v_bytes = NW * KT * (D + 16) * 2, o_bytes = NW * 16 * (D + 4 + 2) * 4, smem = v_bytes > o_bytes ? v_bytes : o_bytes;
  constexpr auto kern = paged_few_kernel<D, NW, TREE>;
  hipError_t e = allow_lds<kern>(smem, ctx->device);
  if (e != hipSuccess) return e;
  const int64_t items = (int64_t)p.a.n_rows * p.a.n_kv_heads * p.parts, slots = (int64_t)ctx->n_cu * few_per_unit<D, NW>();
  KernelTimer t(ctx, CASCADE_K_PAGED_ATTN);
  CASCADE_TIMED_LAUNCH(t, kern, dim3((unsigned)std::min(items, slots)), dim3(64 * NW), smem, ctx->stream, p);
  return hipGetLastError();
}
template <int D>
hipError_t launch_few(cascade_ctx* ctx, const PagedParams& p, const Cut& c) {
  if (p.a.parent) return launch_few_k<D, 4, true>(ctx, p);
  return few_waves(&p.a, c, ctx->n_cu) == 8 ? launch_few_k<D, 8, false>(ctx, p) : launch_few_k<D, 4, false>(ctx, p);
}

// no more blocks of so many query rows than this, whatever the rows' lengths are; a row out of order is one
int64_t most_blocks(const PagedParams& p, int rows) {
  const int64_t each = ((int64_t)p.a.max_new * p.group + rows - 1) / rows;
  return std::min((int64_t)p.a.n_tokens * p.group / rows + p.a.n_rows, each * p.a.n_rows) * p.parts;
}

template <int D, int NS, int NQ, int NW, bool TREE>
hipError_t launch_ring_k(cascade_ctx* ctx, PagedParams& p) {
  constexpr int smem = ring_lds<D, NS, NQ, NW, TREE>();
  constexpr auto kern = paged_ring_kernel<D, NS, NQ, NW, TREE>;
  hipError_t e = allow_lds<kern>(smem, ctx->device);
  if (e != hipSuccess) return e;
  const paged_attn_args& a = p.a;
  const int64_t blocks = most_blocks(p, 16 * NQ * NW);
  // (8 / n_kv_heads XCDs share a kv head: every one gets as many)
  const int64_t share = 8 % a.n_kv_heads == 0 ? 8 / a.n_kv_heads : 1;
  p.in_order = a.n_rows == 1 || a.n_rows > 64 || blocks * a.n_kv_heads <= ctx->n_cu;
  KernelTimer t(ctx, CASCADE_K_PAGED_ATTN);
  CASCADE_TIMED_LAUNCH(t, kern, dim3((unsigned)((blocks + share - 1) / share * share * a.n_kv_heads)), dim3(64 * NW), smem, ctx->stream, p);
  return hipGetLastError();
}
template <int D, bool TREE>
hipError_t launch_ring(cascade_ctx* ctx, PagedParams& p, const Cut& c) {
  if (c.shape == RING_64) return launch_ring_k<D, 2, 1, 4, TREE>(ctx, p);
  if constexpr (D == 64)
    if (c.shape == RING_256) return launch_ring_k<D, 3, 2, 8, TREE>(ctx, p);
  return launch_ring_k<D, 2, 2, 4, TREE>(ctx, p);
}
template <int DB, int NW, bool VEC, bool TREE>
hipError_t launch_f32_k(cascade_ctx* ctx, PagedParams& p) {
  constexpr int smem = (NW * 16 * (16 * DB + 4) + NW * 32) * 4;
  constexpr auto kern = paged_f32_kernel<DB, NW, VEC, TREE>;
  hipError_t e = allow_lds<kern>(smem, ctx->device);
  if (e != hipSuccess) return e;
  const int64_t blocks = most_blocks(p, 16) * p.a.n_kv_heads;
  p.in_order = p.a.n_rows == 1 || p.a.n_rows > 64 || blocks <= ctx->n_cu;
  KernelTimer t(ctx, CASCADE_K_PAGED_ATTN);
  CASCADE_TIMED_LAUNCH(t, kern, dim3((unsigned)blocks), dim3(64 * NW), smem, ctx->stream, p);
  return hipGetLastError();
}
template <int DB, int NW>
hipError_t launch_f32_t(cascade_ctx* ctx, PagedParams& p) {
  const paged_attn_args& a = p.a;
  // keys, values and queries 16 bytes at a time where everything lies on such boundaries, otherwise element by element
  const bool vec = ((a.head_dim | a.q_stride | a.kv_stride | a.stride_page | a.stride_head | a.stride_pos) % 4) == 0 &&
                   (((uintptr_t)a.q | (uintptr_t)a.k_new | (uintptr_t)a.v_new | (uintptr_t)a.k_pages | (uintptr_t)a.v_pages) & 15) == 0;
  if (a.parent) return vec ? launch_f32_k<DB, NW, true, true>(ctx, p) : launch_f32_k<DB, NW, false, true>(ctx, p);
  return vec ? launch_f32_k<DB, NW, true, false>(ctx, p) : launch_f32_k<DB, NW, false, false>(ctx, p);
}
hipError_t launch_f32(cascade_ctx* ctx, PagedParams& p) {
  if (p.a.head_dim <= 64) return launch_f32_t<4, 16>(ctx, p);
  return p.a.head_dim <= 128 ? launch_f32_t<8, 8>(ctx, p) : launch_f32_t<16, 4>(ctx, p);
}
template <int D>
hipError_t launch_bf16(cascade_ctx* ctx, PagedParams& p, const Cut& c) {
  if (c.shape == FEW) return launch_few<D>(ctx, p, c);
  return p.a.parent ? launch_ring<D, true>(ctx, p, c) : launch_ring<D, false>(ctx, p, c);
}

}  // namespace

hipError_t launch_paged_attn(cascade_ctx* ctx, const paged_attn_args* a) {
  PagedParams p;
  p.a = *a;
  p.group = a->n_heads / a->n_kv_heads;
  p.group_inv = p.group == 1 ? 0u : (unsigned)((1ull << 32) / p.group + 1);
  p.most_prefix = (int)std::min<int64_t>(a->max_prefix_len, (int64_t)a->table_width * a->page_size);
  p.scale_log2e = (a->scale != 0.f ? a->scale : 1.f / sqrtf((float)a->head_dim)) * LOG2E;
  p.dev_status = ctx->dev_status;
  p.page16 = a->page_size / 16;
  p.page16_inv = p.page16 == 1 ? 0u : (unsigned)((1ull << 32) / p.page16 + 1);
  char* ws = a->workspace ? (char*)a->workspace : ctx->attn_ws;
  size_t ws_bytes = a->workspace ? (size_t)a->workspace_bytes : (recorded(ctx->stream) ? 0 : ctx->attn_ws_bytes);
  const Cut c = choose(a, ctx->n_cu, ws_bytes);
  p.parts = c.parts;
  p.part_tiles = c.part_tiles;
  p.ws_o = (float*)ws;
  p.ws_ml = (float*)ws + (size_t)c.parts * a->n_tokens * a->n_heads * a->head_dim;
  hipError_t e = c.shape == F32 ? launch_f32(ctx, p) : (a->head_dim == 128 ? launch_bf16<128>(ctx, p, c) : launch_bf16<64>(ctx, p, c));
  if (e != hipSuccess) return e;
  if (c.parts > 1) {
    const dim3 grid((unsigned)((a->n_tokens * a->n_heads + 3) / 4));
    KernelTimer t(ctx, CASCADE_K_PAGED_MERGE);
    if (a->dtype == CASCADE_F32) CASCADE_TIMED_LAUNCH(t, (paged_merge_kernel<float, 4>), grid, dim3(256), 0, ctx->stream, p);
    else if (a->head_dim == 128) CASCADE_TIMED_LAUNCH(t, (paged_merge_kernel<uint16_t, 2>), grid, dim3(256), 0, ctx->stream, p);
    else CASCADE_TIMED_LAUNCH(t, (paged_merge_kernel<uint16_t, 1>), grid, dim3(256), 0, ctx->stream, p);
  }
  return hipGetLastError();
}

int64_t plan_paged_attn(const cascade_ctx* ctx, const paged_attn_args* a) {
  const Cut c = choose(a, ctx->n_cu, (size_t)1 << 40);
  return c.parts > 1 ? (int64_t)c.parts * (int64_t)part_bytes(a) : 0;
}

void plan_paged_cut(const paged_attn_args* a, int n_cu, size_t ws_bytes, int32_t* query_rows, int32_t* key_parts, int32_t* waves) {
  const Cut c = choose(a, n_cu, ws_bytes);
  *query_rows = SHAPE_ROWS[c.shape];
  *key_parts = c.parts;
  *waves = c.shape == FEW ? few_waves(a, c, n_cu) : (c.shape == F32 ? f32_waves(a) : (c.shape == RING_256 ? 8 : 4));
}
