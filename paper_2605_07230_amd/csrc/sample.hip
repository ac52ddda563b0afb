// sample_tokens kernel for gfx950: one workgroup per row.
//
//   m = max l,  w_v = exp((l_v - m) / T)
//   kept: l_v >= the k-th largest entry; of those, l_v >= the largest t with  mass{l >= t} >= p * mass;  w_v >= min_p
//   token = the smallest v whose running mass (vocabulary order) exceeds u * the kept mass,  prob = w_token / the kept mass
//
// A draw has to land on the same token whatever the order of additions, so a weight is a double from a polynomial in doubles (relative error
// 1e-12): single precision puts the running sum of 65536 entries on the wrong side of a border once in a few thousand rows.  Sums are made in an order
// that the row's length alone decides; what lanes add in the order of their arrival are integers, or decides about nothing but time.
//
// The row passes through the registers, 1024 entries of a wave at a time, the next ones on their way.  What a pass has to know beforehand - near which
// value the weights are of size 1, above which value some more than k entries lie - is taken from a sample of four entries per thread that the whole row is
// checked against: a sample that misleads costs another pass.
//   - greedy: one pass.
//   - top-k up to 2700, min-p, or 4096 entries at most: entries above the sample's cut go to a list in LDS, in vocabulary order, and the rest runs on that list.
//   - no cut: one pass adds the weights of every chunk of 256 entries, and the chunk in which the sum crosses the target is read again.
//   - top-p over a long row: the first pass counts what falls into 2048 bins, linear in (m - l) / T; the second adds, chunk by chunk, what is above the bins
//     around the one in which the share is reached and lists these bins' entries.
// A threshold among listed entries comes from bins as well: they are added up from the top until the k entries (the mass) are reached, and the entries of
// the bin where that happens, if they are 256 at most, are ranked against each other; more of them (masked rows, ties, narrow rows) are divided by the bits of their values.
//
// What bounds it: one row, the chain of passes, barriers and instruction fetches (code that a workgroup runs through once costs 10 to 20 ns an instruction); a full
// chip, a compute unit's vector instructions: without a cut 40 an entry, 17 of them on doubles, are 41 of the 60 thousand cycles that a row of 65536 takes (greedy 13 of 34,
// top-k 32 of 61, top-p 86 of 127), and rows without top-p wait for those with it.  Measured, one row of 16384, one of 65536 and 256 of 65536 (67 MB, 13 us at the rate of a large
// copy): greedy 4.0, 7.3, 17 us; no cut 9, 21, 30; top-k 2000 13, 20, 30; top-k 5000 18, 47, 64; top-p 0.9 23, 47, 61; top-k 2000 and top-p 16, 24, 34.
// A row kept in registers, 64 entries to a thread, is read once for certain, but every loop over it is unrolled: its code does not fit the instruction cache, 52 us
// for one row of 65536 without a cut and 57 with top-k 2000.
#include "common.h"

namespace {

typedef unsigned long long u64;
constexpr int BINS = 2048, LIST = 256, AROUND = 1024, KEPT = 4096;
constexpr int MOST_SAMPLED = 2700;   // top-k up to which a sample cuts the row: k + k / 4 + 300 entries, some hundred more or less, are not more than KEPT
constexpr int MAXCHUNKS = CASCADE_MAX_VOCAB / 256;
constexpr int LONG = 1024;   // threads of a row of more than 4096 entries
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

// 2^y for y <= 0: 2^n 2^r with |r| <= 1/2, 2^r = 1 + r Q(r) with Q of degree 7 fitted for the least relative error (8.2e-13; exactly 1 at 0).  n is
// what adding 3 2^51 leaves in the last places, and goes to the exponent.  Below 2^-1000 weights stay there.
__device__ __forceinline__ double exp2_d(double y) {
  y = fmax(y, -1000.0);
  const double shifted = y + 6755399441055744.0, r = y - (shifted - 6755399441055744.0);
  double e = 1.3178932928720322e-06;
  e = fma(e, r, 1.5309156636482046e-05);
  e = fma(e, r, 0.00015403825469434995);
  e = fma(e, r, 0.0013333454858479137);
  e = fma(e, r, 0.009618128616103836);
  e = fma(e, r, 0.055504109352689346);
  e = fma(e, r, 0.2402265069811076);
  e = fma(e, r, 0.6931471805482115);
  e = fma(e, r, 1.0);
  return __hiloint2double(__double2hiint(e) + (__double2loint(shifted) << 20), __double2loint(e));
}
// a weight (at most 1) in units of 2^-46: its bits behind 64, whose last place that is.  65536 of them stay below 2^63.
__device__ __forceinline__ u64 mass_of(double w) { return (u64)__double_as_longlong(w + 64.0) - (u64)__double_as_longlong(64.0); }

// unsigned integers in the order of the floats
__device__ __forceinline__ unsigned order_of(float x) {
  const unsigned b = __float_as_uint(x == 0.f ? 0.f : x);   // -0 and 0 are one value
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(unsigned k) { return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k); }

struct Entry {
  float x;
  int at;
};

template <int NT>
struct Shared {
  u64 bin[BINS];          // (counts: the lower halves)
  union {
    Entry kept[KEPT];
    struct {
      double chunk[MAXCHUNKS];   // masses of the chunks of 256 entries
      u64 extra[MAXCHUNKS];      // what listed entries add to them
      float around[AROUND];      // entries of the bins around a share: value, mass, chunk
      u64 around_mass[AROUND];
      int around_at[AROUND];
    };
  };
  float list[LIST];
  u64 list_mass[LIST];
  int chunk_n[MAXCHUNKS], chunk_at[MAXCHUNKS];   // kept entries of the chunks, and where they lie in the list
  u64 wave_u[NT / 64];
  double wave_d[NT / 64];
  unsigned wave_lo[NT / 64], wave_hi[NT / 64];
  int n_list, at_bin, token, bounds[10];
  u64 before;
  unsigned found;
  double base;
};

// What a row's weights are measured in.
struct Row {
  double m, c;        // where a weight is 1, log2(e) / T
  float m32, scale;   // where the bins begin, bins per unit below it
  __device__ __forceinline__ void at(float top, float temp) {
    m = top;
    m32 = top;
    c = 1.44269504088896340736 / (double)temp;
    scale = (float)BINS / (REACH * temp);
    if (!(scale <= 3e38f)) scale = 3e38f;
  }
  __device__ __forceinline__ double weight(float x) const { return exp2_d(((double)x - m) * c); }   // the difference first: 1 for the maximum, however large
  __device__ __forceinline__ int bin(float x) const { return (int)__builtin_amdgcn_fmed3f((m32 - x) * scale, 0.f, (float)(BINS - 1)); }
};

// What the waves left in `per_wave`, added up by every wave for itself: the sum, and what the waves before it left.  (One load and a scan over lanes: the code that
// a workgroup runs through once costs the time to fetch it, 10 to 20 ns an instruction.)
template <int NT>
__device__ __forceinline__ double waves_sum(const double* per_wave, int wave, double* before) {
  const int lane = threadIdx.x & 63;
  const double incl = wave_scan_incl_d(lane < NT / 64 ? per_wave[lane] : 0.0);
  *before = wave ? readlane_d(incl, wave - 1) : 0.0;
  return readlane_d(incl, 63);
}

// exclusive scan over the threads, and the sum; wave_u takes turns, so that one barrier does
template <int NT>
__device__ __forceinline__ u64 block_scan_excl(Shared<NT>& sh, u64 v, u64* total) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const u64 incl = wave_scan_incl_u64(v);
  __syncthreads();
  if (lane == 63) sh.wave_u[wave] = incl;
  __syncthreads();
  const u64 all = wave_scan_incl_u64(lane < NT / 64 ? sh.wave_u[lane] : 0ull);
  *total = readlane_u64(all, 63);
  return (wave ? readlane_u64(all, wave - 1) : 0ull) + incl - v;
}

// Adds up the bins from the first until `amount` (of their sum) is reached: at_bin, and what lies before it.  Behind a barrier that completes the bins.
template <int NT, class Amount>
__device__ __forceinline__ u64 crossing(Shared<NT>& sh, Amount amount_of) {
  constexpr int PER = BINS / NT;
  u64 v[PER], sum = 0, total;
#pragma unroll
  for (int i = 0; i < PER; ++i) { v[i] = sh.bin[threadIdx.x * PER + i]; sum += v[i]; }
  u64 run = block_scan_excl(sh, sum, &total);
  const u64 amount = amount_of(total);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (run < amount && run + v[i] >= amount) { sh.at_bin = threadIdx.x * PER + i; sh.before = run; }
    run += v[i];
  }
  __syncthreads();
  return amount;
}

template <int NT>
__device__ __forceinline__ void clear_bins(Shared<NT>& sh) {
#pragma unroll
  for (int i = 0; i < BINS / NT; ++i) sh.bin[threadIdx.x + i * NT] = 0;
}

// Of the n listed entries the largest one that, with what is above it, makes up `rest` (masses, or one each): a fourth of a quad of lanes adds up a fourth of the
// list.  Behind a barrier that completes the list and sets `found` to 0; in front of one.
template <int NT, bool MASS, class Enough>
__device__ __forceinline__ void rank_list(Shared<NT>& sh, int n, Enough enough) {
  const int quarter = threadIdx.x & 3;
  for (int i = threadIdx.x >> 2; i < n; i += NT / 4) {
    const float v = sh.list[i];
    u64 sum = 0;
#pragma unroll 4
    for (int j = quarter; j < n; j += 4) sum += sh.list[j] >= v ? (MASS ? sh.list_mass[j] : 1ull) : 0ull;
    sum += dpp_u64<0xb1, 0xf>(sum);   // the other lane of the pair
    sum += dpp_u64<0x4e, 0xf>(sum);   // the other pair of the quad
    if (quarter == 0 && enough(sum)) atomicMax(&sh.found, order_of(v));
  }
}

// The largest t with amount{x >= t} >= amount, where an entry counts one or its mass, and amount <= the sum over all entries is made of that sum.
// each(f) calls f with the thread's entries; each_again does so too, where that is seldom needed.
// bin_of: 0 .. BINS - 1, no larger for a larger value.
template <int NT, bool MASS, class Bin, class Mass, class Amount, class Each, class Again>
__device__ __forceinline__ float threshold(Shared<NT>& sh, Bin bin_of, Mass mass, Amount amount_of, Each each, Again each_again) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  auto add = [&](int bin, float x) {
    if (MASS) atomicAdd(&sh.bin[bin], mass(x));
    else atomicAdd((unsigned*)&sh.bin[bin], 1u);
  };
  clear_bins(sh);
  if (tid == 0) { sh.n_list = 0; sh.found = 0; }
  __syncthreads();
  each([&](float x) { add(bin_of(x), x); });
  __syncthreads();
  const u64 amount = crossing(sh, amount_of);
  const int b = sh.at_bin;
  u64 before = sh.before;
  each([&](float x) {
    if (bin_of(x) == b) {
      const int at = atomicAdd(&sh.n_list, 1);
      if (at < LIST) sh.list[at] = x;
    }
  });
  __syncthreads();
  const int n = sh.n_list;
  if (n <= LIST) {
    if (MASS) {
      for (int i = tid; i < n; i += NT) sh.list_mass[i] = mass(sh.list[i]);
      __syncthreads();
    }
    rank_list<NT, MASS>(sh, n, [&](u64 sum) { return before + sum >= amount; });   // an entry is a threshold if it and what is above it suffice
    __syncthreads();
    const float t = value_of(sh.found);
    __syncthreads();
    return t;
  }
  // many entries in one bin: by the bits of their values
  unsigned lo = 0xffffffffu, hi = 0;
  each_again([&](float x) {
    if (bin_of(x) == b) { const unsigned k = order_of(x); lo = min(lo, k); hi = max(hi, k); }
  });
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
    each_again([&](float x) {
      const unsigned k = order_of(x);
      if (bin_of(x) == b && k >= lo && k <= hi) add((hi - k) >> shift, x);
    });
    __syncthreads();
    crossing(sh, [&](u64) { return amount - before; });
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

// the smallest share of a total that is at least p of it, and not nothing
__device__ __forceinline__ u64 share_of(float p, u64 total) {
  const double share = (double)fmaxf(p, 0.f) * (double)total;
  u64 n = (u64)share;
  n += (double)n < share;
  return n < 1 ? 1 : (n > total ? total : n);
}

// w >= min_p, as a value of the logits: at least the lowest one
__device__ __forceinline__ float least_of(float mx, float temp, float min_p) {
  const float LOWEST = -3.402823466e38f;
  if (!(min_p > 0.f)) return LOWEST;
  const double least = (double)mx + (double)temp * log((double)fminf(min_p, 1.f));
  float x = (float)least;
  if ((double)x < least) x = value_of(order_of(x) + 1);
  return x >= LOWEST ? x : LOWEST;   // (an infinite temperature: every weight is 1)
}

// Sums over the wave of four values at once: the 16 lanes of row 0 receive those of the first, of row 1 of the third, of row 2 of the second, of row 3 of the
// fourth; lane 15 of a row the whole sum.
__device__ __forceinline__ double swap_add(double a, double b, bool by32) {
  const u64 x = (u64)__double_as_longlong(a), y = (u64)__double_as_longlong(b);
  cascade_u32x2 lo, hi;
  if (by32) {
    lo = __builtin_amdgcn_permlane32_swap((unsigned)x, (unsigned)y, false, false);
    hi = __builtin_amdgcn_permlane32_swap((unsigned)(x >> 32), (unsigned)(y >> 32), false, false);
  } else {
    lo = __builtin_amdgcn_permlane16_swap((unsigned)x, (unsigned)y, false, false);
    hi = __builtin_amdgcn_permlane16_swap((unsigned)(x >> 32), (unsigned)(y >> 32), false, false);
  }
  return __longlong_as_double((long long)(((u64)hi.x << 32) | lo.x)) + __longlong_as_double((long long)(((u64)hi.y << 32) | lo.y));
}
__device__ __forceinline__ double rows_of_four(double s0, double s1, double s2, double s3) {
  double d = swap_add(swap_add(s0, s1, true), swap_add(s2, s3, true), false);
  d += dpp_f64<0x111, 0xf>(d);
  d += dpp_f64<0x112, 0xf>(d);
  d += dpp_f64<0x114, 0xf>(d);
  d += dpp_f64<0x118, 0xf>(d);
  return d;
}
template <int NT>
__device__ __forceinline__ double sum_of_chunks(const Shared<NT>& sh, int lane) {   // every wave for itself
  double s = 0.0;
#pragma unroll
  for (int i = 0; i < MAXCHUNKS / 64; ++i) s += sh.chunk[lane * (MAXCHUNKS / 64) + i];
  return readlane_d(wave_scan_incl_d(s), 63);
}
// 2^ceil(y), |y| below 900
__device__ __forceinline__ double exp_up(double y) { return __longlong_as_double((long long)((u64)(1023 + (int)ceil(fmax(y, -900.0))) << 52)); }

template <typename T, int NT, bool VEC>
__global__ __launch_bounds__(NT) void sample_kernel(SampleParams p) {
  constexpr int NW = NT / 64, B = 4;   // B: chunks that a wave takes at a time
  __shared__ Shared<NT> sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), row_id = blockIdx.x;
  const int V = p.vocab, chunks = (V + 255) >> 8;
  const T* l = (const T*)p.logits + (long long)row_id * p.stride;
  // four entries from `at` on, at most the row's last ones
  auto load4 = [&](int at) {
    f32x4 v;
    if constexpr (VEC) {   // vocab a multiple of 4, rows on 4-entry boundaries
      const int from = min(at, V - 4);
      if constexpr (sizeof(T) == 4) v = *(const f32x4*)(l + from);
      else {
        const uint2 r = *(const uint2*)(l + from);
        v = f32x4{bf16_bits_to_f32((uint16_t)r.x), bf16_bits_to_f32((uint16_t)(r.x >> 16)), bf16_bits_to_f32((uint16_t)r.y), bf16_bits_to_f32((uint16_t)(r.y >> 16))};
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = load_f32(l + min(at + i, V - 1));
    }
    return v;
  };
  // f(chunk, entries of the lane's four) for the wave's chunks, B of them at a time: chunk, chunk + NW, ...; entries past the row, and NaN, are -inf: never drawn.  What is
  // past the row's last chunk is -inf as well.
  auto over_row = [&](auto f) {
    f32x4 next[B];
#pragma unroll
    for (int b = 0; b < B; ++b) next[b] = load4(256 * (wave + b * NW) + 4 * lane);
#pragma unroll 1
    for (int c = wave; c < chunks; c += B * NW) {
      f32x4 v[B];
#pragma unroll
      for (int b = 0; b < B; ++b) v[b] = next[b];
      if (c + B * NW < chunks)
#pragma unroll
        for (int b = 0; b < B; ++b) next[b] = load4(256 * (c + (B + b) * NW) + 4 * lane);
#pragma unroll
      for (int b = 0; b < B; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) v[b][i] = 256 * (c + b * NW) + 4 * lane + i < V && v[b][i] == v[b][i] ? v[b][i] : -INFINITY;
      f(c, v);
    }
  };
  auto all_max = [&](float v) {   // over the workgroup
    v = wave_max(v);
    __syncthreads();
    if (lane == 0) sh.wave_lo[wave] = __float_as_uint(v);
    __syncthreads();
    return wave_max(lane < NW ? __uint_as_float(sh.wave_lo[lane]) : -INFINITY);
  };
  auto write = [&](int token, double prob) {
    p.token[row_id] = token;
    if (p.prob) p.prob[row_id] = (float)prob;
  };

  const f32x4 sample = load4((int)((long long)tid * (V >> 2) / NT) * 4);
  const float temp = p.temperature ? p.temperature[row_id] : 1.f;
  float u = p.u[row_id];
  const int k = p.top_k ? p.top_k[row_id] : 0;
  const float top_p = p.top_p ? p.top_p[row_id] : 1.f, min_p = p.min_p ? p.min_p[row_id] : 0.f;
  if (!(u >= 0.f)) u = 0.f;   // outside [0, 1): the first or the last kept entry

  if (!(temp > 0.f)) {   // greedy: the first of the largest
    float mx = -INFINITY;
    int at = 0x7fffffff;
    over_row([&](int c, const f32x4 (&v)[B]) {
#pragma unroll
      for (int b = 0; b < B; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (v[b][i] > mx) { mx = v[b][i]; at = 256 * (c + b * NW) + 4 * lane + i; }   // (a thread's entries come in ascending order)
    });
    const float m = all_max(mx);
    if (tid == 0) sh.token = 0x7fffffff;
    __syncthreads();
    at = wave_min_i(mx == m && m > -INFINITY ? at : 0x7fffffff);
    if (lane == 0) atomicMin(&sh.token, at);
    __syncthreads();
    if (tid == 0) { if (m == -INFINITY) write(-1, 0.0); else write(sh.token, 1.0); }
    return;
  }

  // ---- what the sample says
  const float LOWEST = -3.402823466e38f;   // what is above it is not -inf
  float near_max = fmaxf(fmaxf(sample[0], sample[1]), fmaxf(sample[2], sample[3]));   // (fmaxf passes over NaN)
  near_max = all_max(near_max);
  const bool sampled = near_max > -INFINITY && near_max < INFINITY;
  Row row;
  // The row's maximum is mostly above the sample's: bins begin fifteen temperatures above that (five left a third of the rows of a normal distribution of 6.7
  // temperatures above the bins).  A weight of exactly 1 at the sample's maximum keeps the sums of rows of one value whole numbers.
  row.at(sampled ? near_max : 0.f, temp);
  if (sampled && near_max + 15.f * temp < INFINITY) row.m32 = near_max + 15.f * temp;
  auto row_bin = [&](float x) { return row.bin(x); };
  auto row_mass = [&](float x) { return mass_of(row.weight(x)); };
  const bool top_k = k > 0 && k < V;
  float cut = LOWEST;
  bool list_all = V <= KEPT, cut_by_k = false;
  if (sampled && top_p >= 1.f && min_p > 0.f) {
    cut = fmaxf(cut, near_max + temp * logf(fminf(min_p, 1.f)) * 1.0001f - 1e-5f * fabsf(near_max));   // the maximum is no smaller, so no w >= min_p is below
    if (!(cut >= LOWEST)) cut = LOWEST;
  }
  if (sampled && !list_all && ((top_k && k <= MOST_SAMPLED) || cut > LOWEST)) {
    // some more than k entries, as a share of the sample; bins sixteen times as wide where these lie too far below the maximum
    const float share = top_k && k <= MOST_SAMPLED ? (float)max(k + k / 4 + 300, 1500) * (4.f * NT) / (float)V : 4.f * NT;
    u64 hits = 0;
    float scale = row.scale;
#pragma unroll 1
    for (int wide = 0; wide < 3; ++wide, scale *= 1.f / 16) {
      clear_bins(sh);
      if (tid == 0) sh.at_bin = BINS - 1;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (sample[i] >= cut) atomicAdd((unsigned*)&sh.bin[(int)__builtin_amdgcn_fmed3f((row.m32 - sample[i]) * scale, 0.f, (float)(BINS - 1))], 1u);
      __syncthreads();
      crossing(sh, [&](u64 total) { hits = total; return (u64)share + 1; });
      if (!((float)hits > share) || sh.at_bin < BINS - 1) break;
      __syncthreads();
    }
    if ((float)hits > share && sh.at_bin < BINS - 1) { cut = fmaxf(cut, row.m32 - (float)(sh.at_bin + 1) / scale); cut_by_k = true; }
    list_all = (cut_by_k || !((float)hits > share)) && fminf((float)hits, share) * (float)V < 3900.f * 4.f * NT;   // (the estimate of what is above the cut)
  } else if (!list_all) {
    cut = LOWEST;
  }

  float mx = -INFINITY;
  if (list_all) {
    // ---- entries from the cut on go to the list, chunk by chunk in the order in which they are met
    if (tid == 0) sh.n_list = 0;
    for (int c = tid; c < MAXCHUNKS; c += NT) sh.chunk_n[c] = 0;
    __syncthreads();
    over_row([&](int c, const f32x4 (&v)[B]) {
#pragma unroll
      for (int b = 0; b < B; ++b) {
        u64 is[4];
        int n = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          mx = fmaxf(mx, v[b][i]);
          is[i] = __ballot(v[b][i] >= cut);
          n += __popcll(is[i]);
        }
        if (n == 0) continue;
        int at = 0;
        if (lane == 0) at = atomicAdd(&sh.n_list, n);
        at = __builtin_amdgcn_readfirstlane(at);
        if (lane == 0) { sh.chunk_n[c + b * NW] = n; sh.chunk_at[c + b * NW] = at; }
        if (at + n <= KEPT) {
#pragma unroll
          for (int i = 0; i < 4; ++i) at = __builtin_amdgcn_mbcnt_hi((unsigned)(is[i] >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)is[i], at));
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (v[b][i] >= cut) sh.kept[at++] = Entry{v[b][i], 256 * (c + b * NW) + 4 * lane + i};
        }
      }
    });
    mx = all_max(mx);
    const int n_kept = sh.n_list;   // (behind a barrier)
    if (mx == -INFINITY) { if (tid == 0) write(-1, 0.0); return; }
    if (n_kept <= KEPT && (!cut_by_k || n_kept >= k) && mx < INFINITY) {
      // vocabulary order: the chunks' places follow from their counts
      if (wave == 0) {
        constexpr int PER = MAXCHUNKS / 64;
        int c[PER], sum = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) { c[i] = sh.chunk_n[lane * PER + i]; sum += c[i]; }
        int run = wave_scan_incl_i(sum) - sum;
#pragma unroll
        for (int i = 0; i < PER; ++i) { sh.chunk_n[lane * PER + i] = run; run += c[i]; }
      }
      constexpr int PER = KEPT / NT;
      Entry mine[PER];
#pragma unroll
      for (int i = 0; i < PER; ++i) mine[i] = sh.kept[min(tid + i * NT, n_kept - 1)];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (tid + i * NT < n_kept) {
          const int c = mine[i].at >> 8;
          sh.kept[sh.chunk_n[c] + tid + i * NT - sh.chunk_at[c]] = mine[i];
        }
      __syncthreads();
      row.at(mx, temp);
      float y[PER];   // consecutive entries of a thread
#pragma unroll
      for (int i = 0; i < PER; ++i) y[i] = tid * PER + i < n_kept ? sh.kept[tid * PER + i].x : -INFINITY;
      float thr = cut;
      const float least = least_of(mx, temp, min_p);
      if (top_p >= 1.f) thr = fmaxf(thr, least);   // the mass that top-p is a share of holds what min-p takes out
      auto each_kept = [&](auto f) {
#pragma unroll
        for (int i = 0; i < PER; ++i)
          if (y[i] >= thr) f(y[i]);
      };
      if (top_k && k < n_kept) {
        int n = 0;   // (min-p may have left fewer than k)
        each_kept([&](float) { ++n; });
        u64 total;
        (void)block_scan_excl(sh, (u64)n, &total);
        if ((u64)k < total) thr = threshold<NT, false>(sh, row_bin, row_mass, [&](u64) { return (u64)k; }, each_kept, each_kept);
      }
      if (top_p < 1.f) thr = threshold<NT, true>(sh, row_bin, row_mass, [&](u64 total) { return share_of(top_p, total); }, each_kept, each_kept);
      thr = fmaxf(thr, least);
      double w[PER], sum = 0.0;
#pragma unroll
      for (int i = 0; i < PER; ++i) { w[i] = y[i] >= thr ? row.weight(y[i]) : 0.0; sum += w[i]; }
      const double incl = wave_scan_incl_d(sum);
      if (lane == 63) sh.wave_d[wave] = incl;
      if (tid == 0) { sh.token = 0x7fffffff; sh.at_bin = 0; }
      __syncthreads();
      double base;
      const double total = waves_sum<NT>(sh.wave_d, wave, &base), target = (double)u * total;
      double run = base + (incl - sum);
      int cand = 0x7fffffff, last = 0;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        run += w[i];
        if (w[i] > 0.0) last = tid * PER + i;
        if (cand == 0x7fffffff && w[i] > 0.0 && run > target) cand = tid * PER + i;
      }
      cand = wave_min_i(cand);
      last = wave_max_i(last);
      if (lane == 0) { atomicMin(&sh.token, cand); atomicMax(&sh.at_bin, last); }
      __syncthreads();
      if (tid == 0) {
        const int at = sh.token != 0x7fffffff ? sh.token : sh.at_bin;   // rounding, or u >= 1, kept the running mass at or below the target: the last entry
        write(sh.kept[at].at, row.weight(sh.kept[at].x) / total);
      }
      return;
    }
  }

  // ---- long rows.  Chunk sums: weights of the entries that `keep` says, in an order that only the row's length decides.
  float thr = LOWEST;
  bool infinite = false;   // entries at infinity share the mass, whatever the temperature
  auto weight = [&](float x) { return infinite ? (x == INFINITY ? 1.0 : 0.0) : row.weight(x); };
  auto chunk_sums = [&](auto f) {   // f(chunk, place in it, x): a double
    over_row([&](int c, const f32x4 (&v)[B]) {
      double s[B];
#pragma unroll
      for (int b = 0; b < B; ++b) {
        s[b] = 0.0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          mx = fmaxf(mx, v[b][i]);
          s[b] += f(c + b * NW, i, v[b][i]);
        }
      }
      // four sums over 64 lanes: rows of 16 lanes take one chunk each
      const double d = rows_of_four(s[0], s[1], s[2], s[3]);
      // (row_of_four: lanes 0-15 chunk 0, 16-31 chunk 2, 32-47 chunk 1, 48-63 chunk 3)
      const int b = (lane >> 5) + 2 * ((lane >> 4) & 1), at = c + b * NW;
      if ((lane & 15) == 15 && at < chunks) sh.chunk[at] = d;
    });
  };
  auto each_again = [&](auto f) {
    over_row([&](int c, const f32x4 (&v)[B]) {
#pragma unroll
      for (int b = 0; b < B; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (v[b][i] >= thr) f(v[b][i]);
    });
  };
  // weights are measured from the sample's maximum, unless that is far from the row's
  auto measure_again = [&]() {
    mx = all_max(mx);
    infinite = mx == INFINITY;
    const bool far = !infinite && !(sampled && fabs(((double)mx - row.m) * row.c) < 500.0);
    if (far) row.at(mx, temp);
    return far || infinite;
  };
  const bool cut_k = top_k, cut_p = top_p < 1.f;
  __syncthreads();
  if (cut_k || cut_p || min_p > 0.f) {
    // the maximum, for thresholds among values, the number of entries, which top-k may reach, and for top-p how many entries each bin holds
    clear_bins(sh);
    __syncthreads();
    int n = 0;
    over_row([&](int c, const f32x4 (&v)[B]) {
#pragma unroll
      for (int b = 0; b < B; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          mx = fmaxf(mx, v[b][i]);
          n += v[b][i] > -INFINITY;
          if (cut_p && !cut_k && v[b][i] > -INFINITY) atomicAdd((unsigned*)&sh.bin[row.bin(v[b][i])], 1u);
        }
    });
    const bool bins_are_off = measure_again();
    u64 counted;
    (void)block_scan_excl(sh, (u64)n, &counted);
    if (counted == 0) { if (tid == 0) write(-1, 0.0); return; }
    if (!infinite && cut_k && (u64)k < counted) {
      row.at(mx, temp);
      thr = threshold<NT, false>(sh, row_bin, row_mass, [&](u64) { return (u64)k; }, each_again, each_again);
    }
    const float least = least_of(mx, temp, min_p);
    if (!infinite && cut_p) {
      bool done = false;
      if (!cut_k && !bins_are_off) {
        // The bins around the one in which the share is reached, as far as the bins' numbers of entries at the weight of their middles say: from where a little
        // less than the share is reached to where a little more is, 1 % of the mass or, where that would be too many entries (a peaked row has few there and bins that say
        // little, a flat one the contrary), less.  The exact masses say whether it is among these.
        constexpr int PER = BINS / NT, STEPS = 5, NOWHERE = (BINS - 1) << 17;   // a bin and the number of entries up to it
        constexpr float WIDTH = REACH * 1.44269504f / BINS;
        float mass[PER], sum = 0.f;
        int count[PER], total_n = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const int b = tid * PER + i;
          count[i] = (int)(unsigned)sh.bin[b];
          mass[i] = (float)count[i] * __builtin_amdgcn_exp2f(b == 0 ? fmaxf(0.f, (mx - row.m32) * (float)row.c) : -WIDTH * ((float)b + 0.5f));
          sum += mass[i];
          total_n += count[i];
        }
        const float incl = wave_scan_incl_f(sum);
        u64 counted_too;
        int run_n = (int)block_scan_excl(sh, (u64)total_n, &counted_too);
        if (tid < 2 * STEPS) sh.bounds[tid] = tid < STEPS ? 0 : NOWHERE | (int)counted_too;
        if (tid == 0) { sh.n_list = 0; sh.found = 0; }
        if (lane == 63) sh.wave_lo[wave] = __float_as_uint(incl);
        for (int c = tid; c < MAXCHUNKS; c += NT) { sh.chunk[c] = 0.0; sh.extra[c] = 0; }
        __syncthreads();
        const float waves = wave_scan_incl_f(lane < NW ? __uint_as_float(sh.wave_lo[lane]) : 0.f);
        const float near_all = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(waves), 63)), share = fmaxf(top_p, 0.f) * near_all;
        float run = incl - sum + (wave ? __int_as_float(__builtin_amdgcn_readlane(__float_as_int(waves), wave - 1)) : 0.f);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const float end = run + mass[i];
          if (count[i] && end >= share - 0.01f * near_all && run < share + 0.01f * near_all) {
            float more = 0.01f * near_all;
            const int b = (tid * PER + i) << 17;
#pragma unroll 1
            for (int e = 0; e < STEPS; ++e) {
              if (run < share - more || (e == STEPS - 1 && run < share)) atomicMax(&sh.bounds[e], b | run_n);   // the last bin that begins before the share less `more`
              if (end >= share + more || (e == STEPS - 1 && end >= share)) atomicMin(&sh.bounds[STEPS + e], b | (run_n + count[i]));
              more *= 0.25f;
            }
          }
          run = end;
          run_n += count[i];
        }
        __syncthreads();
        int e = 0;
        while (e < STEPS - 1 && (sh.bounds[STEPS + e] & 0x1ffff) - (sh.bounds[e] & 0x1ffff) > AROUND - 100) ++e;
        const int b0 = sh.bounds[e] >> 17, b1 = sh.bounds[STEPS + e] >> 17;
        double all_mine = 0.0;
        if ((sh.bounds[STEPS + e] & 0x1ffff) - (sh.bounds[e] & 0x1ffff) > AROUND) { if (tid == 0) sh.n_list = AROUND + 1; }
        else chunk_sums([&](int c, int i, float x) {
          const int at = x > -INFINITY ? row.bin(x) : BINS;
          if (at >= b0 && at <= b1) {
            const int q = atomicAdd(&sh.n_list, 1);
            if (q < AROUND) { sh.around[q] = x; sh.around_at[q] = c; }
          }
          const double w = at < BINS ? row.weight(x) : 0.0;
          all_mine += w;
          return at < b0 ? w : 0.0;
        });
        const double all_incl = wave_scan_incl_d(all_mine);
        if (lane == 63) sh.wave_d[wave] = all_incl;
        __syncthreads();
        const int n_list = sh.n_list;
        if (n_list <= AROUND) {
          double ahead;
          const double all = waves_sum<NT>(sh.wave_d, wave, &ahead);
          const double amount = fmax((double)fmaxf(top_p, 0.f) * all, 1e-300), before = sum_of_chunks(sh, lane);
          // masses of the listed as integers, which no order of additions changes: no weight is larger than `one`
          const double one = exp_up(((double)mx - row.m) * row.c), step = one * 0x1p-46;
          u64 mine = 0, listed;
          for (int i = tid; i < n_list; i += NT) {
            const u64 q = mass_of(row.weight(sh.around[i]) / one);
            sh.around_mass[i] = q;
            mine += q;
          }
          (void)block_scan_excl(sh, mine, &listed);
          if (before < amount && before + (double)listed * step >= amount) {
            const double rest = ceil((amount - before) / step);
            const float finer = (float)BINS / (float)(b1 - b0 + 1);
            auto each_listed = [&](auto f) {
#pragma unroll 1
              for (int i = tid; i < n_list; i += NT) f(sh.around[i]);
            };
            thr = threshold<NT, true>(
                sh, [&](float x) { return (int)__builtin_amdgcn_fmed3f(((row.m32 - x) * row.scale - (float)b0) * finer, 0.f, (float)(BINS - 1)); },
                [&](float x) { return mass_of(row.weight(x) / one); }, [&](u64 total) { return rest < (double)total ? (u64)rest : total; }, each_listed, each_listed);
            if (least <= thr) {   // min-p takes nothing more: the chunks' sums stand, with the listed entries above the threshold
              for (int i = tid; i < n_list; i += NT)
                if (sh.around[i] >= thr) atomicAdd(&sh.extra[sh.around_at[i]], sh.around_mass[i]);
              __syncthreads();
              for (int c = tid; c < chunks; c += NT) sh.chunk[c] += (double)sh.extra[c] * step;
              __syncthreads();
            }
            done = true;
          }
        }
      }
      if (!done) {
        row.at(mx, temp);
        thr = threshold<NT, true>(sh, row_bin, row_mass, [&](u64 total) { return share_of(top_p, total); }, each_again, each_again);
      }
      if (!done || least > thr) {
        thr = fmaxf(thr, least);
        chunk_sums([&](int, int, float x) { return x >= thr ? row.weight(x) : 0.0; });
      }
    } else {
      thr = infinite ? LOWEST : fmaxf(thr, least);
      chunk_sums([&](int, int, float x) { return x >= thr ? weight(x) : 0.0; });
    }
  } else {
    chunk_sums([&](int, int, float x) { return x >= thr ? weight(x) : 0.0; });
    if (measure_again()) {
      if (mx == -INFINITY) { if (tid == 0) write(-1, 0.0); return; }
      chunk_sums([&](int, int, float x) { return x >= thr ? weight(x) : 0.0; });
    }
  }
  __syncthreads();

  // ---- the chunk in which the running mass crosses the target, the entry in it
  if (wave == 0) {
    constexpr int PER = MAXCHUNKS / 64;
    double c[PER], s = 0.0;
#pragma unroll
    for (int i = 0; i < PER; ++i) { c[i] = lane * PER + i < chunks ? sh.chunk[lane * PER + i] : 0.0; s += c[i]; }
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
    bool none = at == 0x7fffffff;
    if (none) at = wave_max_i(last);
    const u64 who = __ballot((none ? last : cand) == at);
    const double b = readlane_d(none ? last_base : base, __ffsll((long long)who) - 1);
    const f32x4 y = load4(256 * at + 4 * lane);
    double w[4];
    s = 0.0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool in = 256 * at + 4 * lane + i < V && y[i] >= thr;
      w[i] = in ? weight(y[i]) : 0.0;
      s += w[i];
    }
    run = b + (wave_scan_incl_d(s) - s);
    cand = 0x7fffffff;
    last = -1;
    double wc = 0.0, wl = 0.0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      run += w[i];
      if (w[i] > 0.0) { last = 4 * lane + i; wl = w[i]; }
      if (cand == 0x7fffffff && w[i] > 0.0 && run > target) { cand = 4 * lane + i; wc = w[i]; }
    }
    int e = wave_min_i(cand);
    none = e == 0x7fffffff;
    if (none) e = wave_max_i(last);
    if ((none ? last : cand) == e) write(at * 256 + e, (none ? wl : wc) / total);
  }
}

template <typename T>
hipError_t launch_t(cascade_ctx* ctx, const SampleParams& p, int rows, bool vec) {
  KernelTimer t(ctx, CASCADE_K_SAMPLE);
  // rows of at most 4096 entries: four chunks to each of four waves, several rows to a compute unit
  if (p.vocab <= 4096) {
    if (vec) CASCADE_TIMED_LAUNCH(t, (sample_kernel<T, 256, true>), dim3(rows), dim3(256), 0, ctx->stream, p);
    else CASCADE_TIMED_LAUNCH(t, (sample_kernel<T, 256, false>), dim3(rows), dim3(256), 0, ctx->stream, p);
  } else {
    if (vec) CASCADE_TIMED_LAUNCH(t, (sample_kernel<T, LONG, true>), dim3(rows), dim3(LONG), 0, ctx->stream, p);
    else CASCADE_TIMED_LAUNCH(t, (sample_kernel<T, LONG, false>), dim3(rows), dim3(LONG), 0, ctx->stream, p);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_sample(cascade_ctx* ctx, const sample_args* a) {
  SampleParams p = {a->logits, a->row_stride, a->vocab, a->temperature, a->top_k, a->top_p, a->min_p, a->u, a->token, a->prob};
  const int size = a->dtype == CASCADE_BF16 ? 2 : 4;
  const bool vec = a->vocab % 4 == 0 && a->row_stride % 4 == 0 && ((uintptr_t)a->logits % (4 * size)) == 0;
  return a->dtype == CASCADE_BF16 ? launch_t<uint16_t>(ctx, p, a->n_rows, vec) : launch_t<float>(ctx, p, a->n_rows, vec);
}
