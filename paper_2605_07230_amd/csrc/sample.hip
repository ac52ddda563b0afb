// sample_tokens kernel for gfx950: one workgroup per row, the row in its registers from the first load to the draw.
//
//   m = max l,  w_v = exp((l_v - m) / T)
//   kept: l_v >= the k-th largest entry; of those, l_v >= the largest t with  mass{l >= t} >= p * mass;  w_v >= min_p
//   token = the smallest v whose running mass (vocabulary order) exceeds u * the kept mass,  prob = w_token / the kept mass
//
// A draw has to land on the same token whatever the order of additions, so a weight is a double from a polynomial in doubles (relative error
// 3e-13) - single precision puts the running sum of 65536 entries on the wrong side of a border once in a few thousand rows.
// Thresholds come from one pass of 2048 bins, linear in (m - l) / T, that are added up from the top until the k entries (the mass) are
// reached; the entries of the bin where that happens (some hundred) go to a list and are ranked against each other.  A bin of more than
// 1024 entries - masked rows, ties, rows of one value - is divided by the bits of its values until one value is left.
// Masses are added as integers, so that no sum depends on the order in which lanes arrive.
// Once at most 4096 entries are kept they move to a list in vocabulary order, four to a thread, and the rest runs there.
#include "common.h"

namespace {

typedef unsigned long long u64;
constexpr int BINS = 2048, LIST = 1024, KEPT = 4096;
constexpr float REACH = 45.f;   // temperatures below the maximum that the bins cover; the last one takes everything beyond

template <int CTRL, int ROW_MASK>
__device__ __forceinline__ u64 dpp_u64(u64 v) {
  const unsigned lo = (unsigned)dpp_i32<CTRL, ROW_MASK>(0, (int)(unsigned)v), hi = (unsigned)dpp_i32<CTRL, ROW_MASK>(0, (int)(unsigned)(v >> 32));
  return ((u64)hi << 32) | lo;
}
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ double dpp_f64(double v) { return __longlong_as_double((long long)dpp_u64<CTRL, ROW_MASK>((u64)__double_as_longlong(v))); }

__device__ __forceinline__ u64 wave_scan_incl_u64(u64 v) {
  v += dpp_u64<0x111, 0xf>(v);
  v += dpp_u64<0x112, 0xf>(v);
  v += dpp_u64<0x114, 0xf>(v);
  v += dpp_u64<0x118, 0xf>(v);
  v += dpp_u64<0x142, 0xa>(v);
  v += dpp_u64<0x143, 0xc>(v);
  return v;
}
__device__ __forceinline__ double wave_scan_incl_d(double v) {
  v += dpp_f64<0x111, 0xf>(v);
  v += dpp_f64<0x112, 0xf>(v);
  v += dpp_f64<0x114, 0xf>(v);
  v += dpp_f64<0x118, 0xf>(v);
  v += dpp_f64<0x142, 0xa>(v);
  v += dpp_f64<0x143, 0xc>(v);
  return v;
}
__device__ __forceinline__ u64 readlane_u64(u64 v, int l) {
  return ((u64)(unsigned)__builtin_amdgcn_readlane((int)(unsigned)(v >> 32), l) << 32) | (unsigned)__builtin_amdgcn_readlane((int)(unsigned)v, l);
}
__device__ __forceinline__ double readlane_d(double v, int l) { return __longlong_as_double((long long)readlane_u64((u64)__double_as_longlong(v), l)); }

// 2^y for y <= 0: 2^n e^(r ln 2) with |r| <= 1/2; the series of e^x to x^10 leaves 2.3e-13 at 0.347
__device__ __forceinline__ double exp2_d(double y) {
  y = fmax(y, -1100.0);   // below the smallest double
  const double n = rint(y), x = (y - n) * 0.693147180559945309417;
  double e = 1.0 / 3628800;
  e = fma(e, x, 1.0 / 362880);
  e = fma(e, x, 1.0 / 40320);
  e = fma(e, x, 1.0 / 5040);
  e = fma(e, x, 1.0 / 720);
  e = fma(e, x, 1.0 / 120);
  e = fma(e, x, 1.0 / 24);
  e = fma(e, x, 1.0 / 6);
  e = fma(e, x, 0.5);
  e = fma(e, x, 1.0);
  e = fma(e, x, 1.0);
  return __builtin_amdgcn_ldexp(e, (int)n);
}
// a weight (at most 1) in units of 2^-46: its bits behind 64, whose last place that is.  65536 of them stay below 2^63.
__device__ __forceinline__ u64 mass_of(double w) { return (u64)__double_as_longlong(w + 64.0) - (u64)__double_as_longlong(64.0); }

// unsigned integers in the order of the floats
__device__ __forceinline__ unsigned order_of(float x) {
  const unsigned b = __float_as_uint(x == 0.f ? 0.f : x);   // -0 and 0 are one value
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(unsigned k) { return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k); }

template <int NT>
struct Shared {
  u64 bin[BINS];          // (counts: the lower halves)
  float list[LIST];
  u64 list_mass[LIST];
  float kept[KEPT];
  int kept_at[KEPT];
  u64 wave_u[NT / 64];
  double wave_d[NT / 64];
  double chunk[CASCADE_MAX_VOCAB / 256];
  unsigned wave_lo[NT / 64], wave_hi[NT / 64];
  int n_list, at_bin, token;
  u64 before;
  unsigned found;
  double base;
};

// What a row's weights are measured in.
struct Row {
  double m, c;      // maximum, log2(e) / T
  float m32, scale; // the maximum again, bins per unit below it
  __device__ __forceinline__ double weight(float x) const { return x == -INFINITY ? 0.0 : exp2_d(((double)x - m) * c); }
  __device__ __forceinline__ int bin(float x) const { return (int)fminf((m32 - x) * scale, (float)(BINS - 1)); }
};

template <int NT>
__device__ __forceinline__ u64 block_scan_excl(Shared<NT>& sh, u64 v, u64* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const u64 incl = wave_scan_incl_u64(v);
  if (lane == 63) sh.wave_u[wave] = incl;
  __syncthreads();
  u64 base = 0, all = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    const u64 x = sh.wave_u[w];
    base += w < wave ? x : 0;
    all += x;
  }
  *total = all;
  __syncthreads();
  return base + incl - v;
}

// Adds up the bins from the first until `amount` is reached: at_bin, and what lies before it.  Behind a barrier that completes the bins.
template <int NT>
__device__ __forceinline__ void crossing(Shared<NT>& sh, u64 amount) {
  constexpr int PER = BINS / NT;
  u64 v[PER], sum = 0, total;
#pragma unroll
  for (int i = 0; i < PER; ++i) { v[i] = sh.bin[threadIdx.x * PER + i]; sum += v[i]; }
  u64 run = block_scan_excl(sh, sum, &total);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (run < amount && run + v[i] >= amount) { sh.at_bin = threadIdx.x * PER + i; sh.before = run; }
    run += v[i];
  }
  __syncthreads();
}

template <int NT>
__device__ __forceinline__ void clear_bins(Shared<NT>& sh) {
#pragma unroll
  for (int i = 0; i < BINS / NT; ++i) sh.bin[threadIdx.x + i * NT] = 0;
}

// The largest t with amount{x >= t} >= amount, where an entry counts one or its mass.  0 < amount <= the sum over all entries that
// are not -inf; entries below `floor_` do not count.
template <int NT, int R, bool MASS>
__device__ float threshold(Shared<NT>& sh, const float (&x)[R], const Row& row, u64 amount, float floor_) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  auto in = [&](float v) { return v >= floor_ && v > -INFINITY; };
  auto worth = [&](float v) -> u64 { return MASS ? mass_of(row.weight(v)) : 1ull; };
  clear_bins(sh);
  if (tid == 0) sh.n_list = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (in(x[i])) {
      if (MASS) atomicAdd(&sh.bin[row.bin(x[i])], worth(x[i]));
      else atomicAdd((unsigned*)&sh.bin[row.bin(x[i])], 1u);
    }
  __syncthreads();
  crossing(sh, amount);
  const int b = sh.at_bin;
  u64 before = sh.before;
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (in(x[i]) && row.bin(x[i]) == b) {
      const int at = atomicAdd(&sh.n_list, 1);
      if (at < LIST) { sh.list[at] = x[i]; if (MASS) sh.list_mass[at] = worth(x[i]); }
    }
  if (tid == 0) sh.found = 0;
  __syncthreads();
  const int n = sh.n_list;
  if (n <= LIST) {
    // entry i is a threshold if it and what is above it suffice; the largest such one is taken
    for (int i = tid; i < n; i += NT) {
      const float v = sh.list[i];
      u64 sum = before;
      for (int j = 0; j < n; ++j) sum += sh.list[j] >= v ? (MASS ? sh.list_mass[j] : 1ull) : 0ull;
      if (sum >= amount) atomicMax(&sh.found, order_of(v));
    }
    __syncthreads();
    const float t = value_of(sh.found);
    __syncthreads();
    return t;
  }
  // many entries in one bin: by the bits of their values
  unsigned lo = 0xffffffffu, hi = 0;
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (in(x[i]) && row.bin(x[i]) == b) { const unsigned k = order_of(x[i]); lo = min(lo, k); hi = max(hi, k); }
  for (int s = 32; s; s >>= 1) { lo = min(lo, (unsigned)__shfl_xor((int)lo, s)); hi = max(hi, (unsigned)__shfl_xor((int)hi, s)); }
  if (lane == 0) { sh.wave_lo[wave] = lo; sh.wave_hi[wave] = hi; }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) { lo = min(lo, sh.wave_lo[w]); hi = max(hi, sh.wave_hi[w]); }
  while (lo < hi) {   // a round leaves at most 1 / 2048 of the range: three at most
    const int shift = max(0, 32 - __clz((int)(hi - lo)) - 11);   // (hi - lo) >> shift < 2048
    __syncthreads();
    clear_bins(sh);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const unsigned k = order_of(x[i]);
      if (in(x[i]) && row.bin(x[i]) == b && k >= lo && k <= hi) {
        if (MASS) atomicAdd(&sh.bin[(hi - k) >> shift], worth(x[i]));
        else atomicAdd((unsigned*)&sh.bin[(hi - k) >> shift], 1u);
      }
    }
    __syncthreads();
    crossing(sh, amount - before);
    before += sh.before;
    hi -= (unsigned)sh.at_bin << shift;
    const unsigned width = (1u << shift) - 1u;
    lo = hi - lo > width ? hi - width : lo;
  }
  __syncthreads();
  return value_of(hi);
}

struct SampleParams {
  const void* logits;
  long long stride;
  int vocab;
  const float* temperature;
  const int32_t* top_k;
  const float *top_p, *min_p, *u;
  int32_t* token;
  float* prob;
};

// R entries per thread (a multiple of 4): entry 4 (j NT + tid) + i of the row is x[4 j + i], so a wave holds 256 consecutive entries for every j
template <typename T, int NT, int R, bool VEC>
__global__ __launch_bounds__(NT) void sample_kernel(SampleParams p) {
  constexpr int NW = NT / 64, J = R / 4;
  __shared__ Shared<NT> sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), row_id = blockIdx.x;
  const int V = p.vocab;
  const T* l = (const T*)p.logits + (long long)row_id * p.stride;
  float x[R];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int at = 4 * (j * NT + tid);
    if constexpr (VEC) {   // vocab a multiple of 4, rows on 4-entry boundaries
      const int from = min(at, V - 4);
      if constexpr (sizeof(T) == 4) {
        const f32x4 v = *(const f32x4*)(l + from);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[4 * j + i] = v[i];
      } else {
        const uint2 v = *(const uint2*)(l + from);
        x[4 * j] = bf16_bits_to_f32((uint16_t)v.x); x[4 * j + 1] = bf16_bits_to_f32((uint16_t)(v.x >> 16));
        x[4 * j + 2] = bf16_bits_to_f32((uint16_t)v.y); x[4 * j + 3] = bf16_bits_to_f32((uint16_t)(v.y >> 16));
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[4 * j + i] = load_f32(l + min(at + i, V - 1));
    }
  }
  float temp = p.temperature ? p.temperature[row_id] : 1.f, u = p.u[row_id];
  const int k = p.top_k ? p.top_k[row_id] : 0;
  const float top_p = p.top_p ? p.top_p[row_id] : 1.f, min_p = p.min_p ? p.min_p[row_id] : 0.f;
  float mx = -INFINITY;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    // entries past the row and NaN are never drawn
    if (4 * ((i / 4) * NT + tid) + i % 4 >= V || x[i] != x[i]) x[i] = -INFINITY;
    mx = fmaxf(mx, x[i]);
  }
  mx = wave_max(mx);
  if (lane == 0) sh.wave_lo[wave] = __float_as_uint(mx);
  if (tid == 0) { sh.token = 0x7fffffff; sh.base = 0.0; }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NW; ++w) mx = fmaxf(mx, __uint_as_float(sh.wave_lo[w]));
  __syncthreads();
  if (mx == -INFINITY) {   // nothing to draw
    if (tid == 0) { p.token[row_id] = -1; if (p.prob) p.prob[row_id] = 0.f; }
    return;
  }
  if (!(temp > 0.f)) {   // greedy: the first of the largest
    int first = 0x7fffffff;
#pragma unroll
    for (int i = R - 1; i >= 0; --i)
      if (x[i] == mx) first = 4 * ((i / 4) * NT + tid) + i % 4;
    first = wave_min_i(first);
    if (lane == 0) atomicMin(&sh.token, first);
    __syncthreads();
    if (tid == 0) { p.token[row_id] = sh.token; if (p.prob) p.prob[row_id] = 1.f; }
    return;
  }
  if (mx == INFINITY) {   // entries at infinity share the mass, whatever the temperature
#pragma unroll
    for (int i = 0; i < R; ++i) x[i] = x[i] == INFINITY ? 0.f : -INFINITY;
    mx = 0.f;
  }
  Row row;
  row.m = mx;
  row.m32 = mx;
  row.c = 1.44269504088896340736 / (double)temp;
  row.scale = (float)BINS / (REACH * temp);
  if (!(row.scale <= 3e38f)) row.scale = 3e38f;
  if (!(u >= 0.f)) u = 0.f;   // outside [0, 1): the first or the last kept entry

  float least_w = -INFINITY;   // w >= min_p, as a value of x
  if (min_p > 0.f) {
    const double least = (double)mx + (double)temp * log((double)fminf(min_p, 1.f));
    least_w = (float)least;
    if ((double)least_w < least) least_w = value_of(order_of(least_w) + 1);
    if (least_w != least_w) least_w = -INFINITY;   // an infinite temperature: every weight is 1
  }
  // kept: x >= thr and x > -inf.  The mass that top-p is a share of holds what min-p takes out.
  float thr = top_p < 1.f ? -INFINITY : least_w;
  auto count_kept = [&](float t) {
    int n = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) n += x[i] >= t && x[i] > -INFINITY;
    u64 total;
    (void)block_scan_excl(sh, (u64)wave_sum_i(n) * (lane == 0), &total);
    return (int)total;
  };
  if (k > 0 && k < V && k < count_kept(thr)) thr = fmaxf(thr, threshold<NT, R, false>(sh, x, row, (u64)k, thr));
  const int n_kept = count_kept(thr);   // at least the maximum

  if (n_kept <= KEPT) {
    // ---- the kept entries in vocabulary order, in LDS
    int mine = 0;   // of this wave, chunk by chunk: their places follow from the counts of all chunks
    int* chunk_n = (int*)sh.chunk;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      int n = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) n += __popcll(__ballot(x[4 * j + i] >= thr && x[4 * j + i] > -INFINITY));
      if (lane == 0) chunk_n[j * NW + wave] = n;
      mine += n;
    }
    __syncthreads();
    {
      constexpr int PER = (J * NW + 63) / 64;   // chunks of a lane of wave 0
      if (wave == 0) {
        int c[PER], sum = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) { c[i] = lane * PER + i < J * NW ? chunk_n[lane * PER + i] : 0; sum += c[i]; }
        int run = wave_scan_incl_i(sum) - sum;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          if (lane * PER + i < J * NW) chunk_n[lane * PER + i] = run;
          run += c[i];
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < J; ++j) {
      int n = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) n += x[4 * j + i] >= thr && x[4 * j + i] > -INFINITY;
      int at = chunk_n[j * NW + wave] + wave_scan_incl_i(n) - n;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (x[4 * j + i] >= thr && x[4 * j + i] > -INFINITY) {
          sh.kept[at] = x[4 * j + i];
          sh.kept_at[at] = 4 * (j * NT + tid) + i;
          ++at;
        }
    }
    __syncthreads();
    constexpr int PER = KEPT / NT;   // consecutive entries of a thread
    float y[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) y[i] = tid * PER + i < n_kept ? sh.kept[tid * PER + i] : -INFINITY;
    if (top_p < 1.f) {
      u64 sum = 0, total;
#pragma unroll
      for (int i = 0; i < PER; ++i) sum += mass_of(row.weight(y[i]));
      (void)block_scan_excl(sh, sum, &total);
      const double share = (double)fmaxf(top_p, 0.f) * (double)total;
      u64 amount = (u64)share;
      amount += (double)amount < share;
      thr = fmaxf(thr, threshold<NT, PER, true>(sh, y, row, amount < 1 ? 1 : (amount > total ? total : amount), thr));
    }
    thr = fmaxf(thr, least_w);
    double w[PER], sum = 0.0;
#pragma unroll
    for (int i = 0; i < PER; ++i) { w[i] = y[i] >= thr ? row.weight(y[i]) : 0.0; sum += w[i]; }
    const double incl = wave_scan_incl_d(sum);
    if (lane == 63) sh.wave_d[wave] = incl;
    __syncthreads();
    double base = 0.0, total = 0.0;
#pragma unroll
    for (int q = 0; q < NW; ++q) { base += q < wave ? sh.wave_d[q] : 0.0; total += sh.wave_d[q]; }
    const double target = (double)u * total;
    double run = base + (incl - sum);
    int cand = 0x7fffffff, last = -1;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      run += w[i];
      if (w[i] > 0.0) last = tid * PER + i;
      if (cand == 0x7fffffff && w[i] > 0.0 && run > target) cand = tid * PER + i;
    }
    cand = wave_min_i(cand);
    last = wave_max_i(last);
    if (lane == 0) { atomicMin(&sh.token, cand); sh.wave_hi[wave] = (unsigned)last; }
    __syncthreads();
    int at = sh.token;
    if (at == 0x7fffffff) {   // rounding, or u >= 1, kept the running mass at or below the target: the last entry
      at = -1;
#pragma unroll
      for (int q = 0; q < NW; ++q) at = max(at, (int)sh.wave_hi[q]);
    }
    if (tid == 0) {
      p.token[row_id] = sh.kept_at[at];
      if (p.prob) p.prob[row_id] = (float)(row.weight(sh.kept[at]) / total);
    }
    return;
  }

  // ---- many kept entries: they stay in the registers
  if (top_p < 1.f) {
    u64 sum = 0, total;
#pragma unroll
    for (int i = 0; i < R; ++i) sum += x[i] >= thr ? mass_of(row.weight(x[i])) : 0;
    (void)block_scan_excl(sh, sum, &total);
    const double share = (double)fmaxf(top_p, 0.f) * (double)total;
    u64 amount = (u64)share;
    amount += (double)amount < share;
    thr = fmaxf(thr, threshold<NT, R, true>(sh, x, row, amount < 1 ? 1 : (amount > total ? total : amount), thr));
  }
  thr = fmaxf(thr, least_w);
  // sums of chunks of 256 entries, the chunk in which the running mass crosses the target, the entry in it
#pragma unroll
  for (int j = 0; j < J; ++j) {
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < 4; ++i) s += x[4 * j + i] >= thr ? row.weight(x[4 * j + i]) : 0.0;
    s = wave_scan_incl_d(s);
    if (lane == 63) sh.chunk[j * NW + wave] = s;
  }
  __syncthreads();
  constexpr int PER = (J * NW + 63) / 64;
  if (wave == 0) {
    double c[PER], s = 0.0;
#pragma unroll
    for (int i = 0; i < PER; ++i) { c[i] = lane * PER + i < J * NW ? sh.chunk[lane * PER + i] : 0.0; s += c[i]; }
    const double incl = wave_scan_incl_d(s), total = readlane_d(incl, 63), target = (double)u * total;
    double run = incl - s;
    int cand = 0x7fffffff, last = -1;
    double base = 0.0, last_base = 0.0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (c[i] > 0.0) { last = lane * PER + i; last_base = run; }
      if (cand == 0x7fffffff && c[i] > 0.0 && run + c[i] > target) { cand = lane * PER + i; base = run; }
      run += c[i];
    }
    int at = wave_min_i(cand);
    const bool none = at == 0x7fffffff;
    if (none) at = wave_max_i(last);
    const unsigned long long who = __ballot((none ? last : cand) == at);
    const double b = readlane_d(none ? last_base : base, __ffsll((long long)who) - 1);
    if (lane == 0) { sh.at_bin = at; sh.base = b; sh.wave_d[0] = total; }
  }
  __syncthreads();
  const int at = sh.at_bin;
  const double base = sh.base, total = sh.wave_d[0], target = (double)u * total;
  if (at % NW == wave) {
    float y[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = j == at / NW ? x[4 * j + i] : y[i];
    double w[4], s = 0.0;
#pragma unroll
    for (int i = 0; i < 4; ++i) { w[i] = y[i] >= thr ? row.weight(y[i]) : 0.0; s += w[i]; }
    double run = base + (wave_scan_incl_d(s) - s);
    int cand = 0x7fffffff, last = -1;
    double wc = 0.0, wl = 0.0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      run += w[i];
      if (w[i] > 0.0) { last = 4 * lane + i; wl = w[i]; }
      if (cand == 0x7fffffff && w[i] > 0.0 && run > target) { cand = 4 * lane + i; wc = w[i]; }
    }
    int e = wave_min_i(cand);
    const bool none = e == 0x7fffffff;
    if (none) e = wave_max_i(last);
    if ((none ? last : cand) == e) {
      p.token[row_id] = at * 256 + e;
      if (p.prob) p.prob[row_id] = (float)((none ? wl : wc) / total);
    }
  }
}

template <typename T, int NT, int R>
hipError_t launch_t(cascade_ctx* ctx, const SampleParams& p, int rows, bool vec) {
  KernelTimer t(ctx, CASCADE_K_SAMPLE);
  if (vec) CASCADE_TIMED_LAUNCH(t, (sample_kernel<T, NT, R, true>), dim3(rows), dim3(NT), 0, ctx->stream, p);
  else CASCADE_TIMED_LAUNCH(t, (sample_kernel<T, NT, R, false>), dim3(rows), dim3(NT), 0, ctx->stream, p);
  return hipGetLastError();
}
template <typename T>
hipError_t launch_v(cascade_ctx* ctx, const SampleParams& p, int rows, bool vec) {
  if (p.vocab <= 4096) return launch_t<T, 256, 16>(ctx, p, rows, vec);
  if (p.vocab <= 16384) return launch_t<T, 1024, 16>(ctx, p, rows, vec);
  if (p.vocab <= 36864) return launch_t<T, 1024, 36>(ctx, p, rows, vec);
  return launch_t<T, 1024, 64>(ctx, p, rows, vec);
}

}  // namespace

hipError_t launch_sample(cascade_ctx* ctx, const sample_args* a) {
  SampleParams p = {a->logits, a->row_stride, a->vocab, a->temperature, a->top_k, a->top_p, a->min_p, a->u, a->token, a->prob};
  const int size = a->dtype == CASCADE_BF16 ? 2 : 4;
  const bool vec = a->vocab % 4 == 0 && a->row_stride % 4 == 0 && ((uintptr_t)a->logits % (4 * size)) == 0;
  return a->dtype == CASCADE_BF16 ? launch_v<uint16_t>(ctx, p, a->n_rows, vec) : launch_v<float>(ctx, p, a->n_rows, vec);
}
