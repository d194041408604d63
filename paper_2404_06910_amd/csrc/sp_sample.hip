// A token for every row of logits, drawn with temperature, min-p, top-k and top-p from a given random number
// (Alg. 3's Sample).
//
// The tokens of a row are put in order: logit descending, ties by the lower index.  Token v weighs w_v = exp((x_v - m) / T), m the
// largest logit.  Every filter leaves a prefix of the order: min-p a range of values, top-k a number of tokens, top-p the
// shortest prefix whose weight reaches p of what the others left.  The draw is the token at which the running weight of the
// order passes u times the weight that is left.  So all that is asked of a row is: at which token does the running count, or
// the running weight, reach a given number?  That is one search over the bits of the (order of the value, index) key, from the
// top: a histogram of counts and weights over the key's first bits, then the bin that holds the place in question again.
// Weights are integers, exp(.) in 64 bits times a power of two such that a row's sum fits 62 bits: their sums do not depend on
// the order of the additions (equal calls give equal tokens), and a weight is off by at most 2^-(62 - bits of the vocabulary), 2^-45 of
// the largest at 128256 tokens.  Tokens lighter than that cannot be drawn.
//
// One workgroup per row.  bf16 rows take counts alone: there are 65536 values, so a histogram of all of them in LDS is the sorted row, and a
// weight is computed once per value that occurs, not per token (sample_counts).  fp32, and the bf16 rows that the 16-bit counts cannot
// hold, build histograms of weights over the first 13 bits and go on inside a bin (RowSearch).
//
// Measured, us: one bf16 row of 50432 with top-p 14.9; 64 of 128256, each with filters of its own, 29.0 (reading them once: 3.2);
// 1024 of 50432 63 (20); 96 fp32 rows of 50257, the best 50 and a nucleus of them, 25.5 (3.8).  A workgroup fills a compute unit's LDS, so a
// row's phases follow each other: of 15 us the load takes 4, the counts' atomics 4 (random bins: bank conflicts), and the rest are
// latencies of scans and barriers.
#include <algorithm>
#include <type_traits>

#include "sp_device.h"
#include "sp_internal.h"

namespace sp {

namespace {

constexpr int kSampleThreads = 1024;
constexpr int kSampleWaves = kSampleThreads / 64;
constexpr int kBinBits = 13, kBins = 1 << kBinBits;
constexpr int kSortedList = 256;                // keys that top-k leaves, up to which they are sorted
constexpr int kList = 2048;                     // keys of one bin that are searched in LDS
constexpr uint32_t kNegInfKey = 0x007fffffu;    // value_key(-inf)

// Order of a value as an unsigned number (the larger the earlier); -0 counts as +0.
__device__ __forceinline__ uint32_t value_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return (u >> 31) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float((k >> 31) ? k & 0x7fffffffu : ~k); }

typedef unsigned long long u64;
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// Place of the search in the order: what lies before the token, or bin, that was found, and what that holds.
struct Place {
  u64 mass_before, mass;
  uint32_t count_before, count, bin;
};

struct SampleLds {
  u64 mass[kBins];
  uint32_t count[kBins];
  u64 list[kList];
  u64 dmass[256];
  uint32_t dcount[256];
  u64 wave_mass[kSampleWaves], wave_top[kSampleWaves];
  uint32_t wave_count[kSampleWaves];
  double table[64];
  Place place;
  uint32_t n_list, n_kept, found_key, found_index;
  u64 kept[kList];                              // the tokens that top-k leaves, and those with equal first bits
};

// exp(.) by a table of 2^(i/64) in LDS and a polynomial for what is left, |r| <= ln 2 / 128 (table-driven reduction; the sixth-order rest
// is below 4e-17): about half the instructions of the library's.
struct Weights {
  float m;          // largest logit
  double inv_t;     // log2 e * 64 / temperature
  int s_bits;       // weights are multiples of 2^-s_bits
  const double *table;
  __device__ __forceinline__ u64 operator()(float x) const {
    // in 64ths of an octave; at m itself the weight is 2^s_bits, from -64 octaves on it is 0 (NaN, and what is not infinite beside infinity)
    const double z = x == m ? 0.0 : fmax((double(x) - double(m)) * inv_t, -65.0 * 64.0);
    const double n = rint(z), r = (z - n) * (0.69314718055994530942 / 64.0);
    const int i = int(n);
    double p = fma(r, 1.0 / 120.0, 1.0 / 24.0);
    p = fma(p, r, 1.0 / 6.0);
    p = fma(p, r, 0.5);
    p = fma(p * r, r, r);
    const double t = table[i & 63];
    return u64(ldexp(fma(t, p, t), (i >> 6) + s_bits));
  }
};
// the table; threads below 64
__device__ __forceinline__ void fill_table(double *table) {
  if (threadIdx.x < 64) table[threadIdx.x] = exp2(double(threadIdx.x) / 64.0);
}

// fn(x, index) for every element of a row, in no order
template <typename T, class F>
__device__ __forceinline__ void for_row(const T *row, int vocab, F &&fn) {
  constexpr int EV = Elem<T>::kVec, U = 4;       // loads in flight
  const int n_vec = vocab / EV;
  for (int v0 = threadIdx.x; v0 < n_vec; v0 += U * kSampleThreads) {
    u32x4 raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u] = ld16(row + int64_t(min(v0 + u * kSampleThreads, n_vec - 1)) * EV);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int v = v0 + u * kSampleThreads;
      if (v >= n_vec) break;
      float x[EV];
      Elem<T>::unpack(raw[u], x);
#pragma unroll
      for (int e = 0; e < EV; ++e) fn(x[e], v * EV + e);
    }
  }
  const int i = n_vec * EV + threadIdx.x;
  if (i < vocab) fn(Elem<T>::load1(row + i), i);
}

// x of the lane that the DPP control names, 0 where it names none (or the row mask leaves the row out)
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp(uint32_t x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false); }
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 dpp(u64 x) { return u64(dpp<CTRL, ROWS>(uint32_t(x >> 32))) << 32 | dpp<CTRL, ROWS>(uint32_t(x)); }
// Sum over the lanes up to this one: in the rows of 16 by shifts, then the last lanes of rows to the rows behind.  (Through LDS, by
// shuffles, a scan of weights and counts takes three times as long, and a row is a chain of them.)
template <class X>
__device__ __forceinline__ X row_scan(X x) {
  x += dpp<0x111, 0xf>(x);                       // row_shr 1, 2, 4, 8
  x += dpp<0x112, 0xf>(x);
  x += dpp<0x114, 0xf>(x);
  x += dpp<0x118, 0xf>(x);
  return x;
}
template <class X>
__device__ __forceinline__ X wave_scan(X x) {
  x = row_scan(x);
  x += dpp<0x142, 0xa>(x);                       // row_bcast 15, 31
  x += dpp<0x143, 0xc>(x);
  return x;
}
__device__ __forceinline__ u64 lane_value(u64 x, int lane) {
  return u64(uint32_t(__builtin_amdgcn_readlane(uint32_t(x >> 32), lane))) << 32 | uint32_t(__builtin_amdgcn_readlane(uint32_t(x), lane));
}
__device__ __forceinline__ uint32_t lane_value(uint32_t x, int lane) { return __builtin_amdgcn_readlane(x, lane); }

// sums over the threads before this one
template <class Lds>
__device__ __forceinline__ void scan_before(Lds &s, u64 &mass, uint32_t &count) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const u64 m = wave_scan(mass);
  const uint32_t c = wave_scan(count);
  __syncthreads();
  if (lane == 63) { s.wave_mass[wave] = m; s.wave_count[wave] = c; }
  __syncthreads();
  // the waves' sums are scanned by the lanes below 16 of every wave
  const u64 wm = wave_scan(lane < kSampleWaves ? s.wave_mass[lane & (kSampleWaves - 1)] : 0);
  const uint32_t wc = wave_scan(lane < kSampleWaves ? s.wave_count[lane & (kSampleWaves - 1)] : 0);
  mass = m - mass + (wave ? lane_value(wm, wave - 1) : 0);
  count = c - count + (wave ? lane_value(wc, wave - 1) : 0);
}

// The bin, from the highest down, at which the running weight (or count) reaches target.
__device__ __forceinline__ Place find_bin(SampleLds &s, const u64 *mass, const uint32_t *count, int n_bins, u64 target, bool by_mass) {
  const int per = (n_bins + kSampleThreads - 1) / kSampleThreads;
  const int top = n_bins - 1 - int(threadIdx.x) * per;
  u64 m = 0;
  uint32_t c = 0;
  for (int j = 0; j < per; ++j)
    if (top - j >= 0) { m += mass[top - j]; c += count[top - j]; }
  u64 mb = m;
  uint32_t cb = c;
  scan_before(s, mb, cb);
  const bool here = by_mass ? mb < target && target <= mb + m : cb < target && target <= u64(cb) + c;
  if (here) {
    int b = top;
    while (b > 0 && (by_mass ? mb + mass[b] : u64(cb) + count[b]) < target) {
      mb += mass[b];
      cb += count[b];
      --b;
    }
    s.place = Place{mb, mass[b], cb, count[b], uint32_t(b)};
  }
  __syncthreads();
  return s.place;
}

__device__ __forceinline__ void reset_place(SampleLds &s) {
  if (threadIdx.x == 0) s.place = Place{0, 0, 0, 0, 0};
  __syncthreads();
}

template <typename T>
struct RowSearch {
  const T *row;
  int vocab;
  uint32_t least;        // value keys below it take no part
  Weights weight;
  SampleLds &s;
  bool few = false;      // what takes part is in s.kept

  template <class F>
  __device__ __forceinline__ void each(F &&fn) const {
    if (few) {
      for (uint32_t i = threadIdx.x; i < s.n_kept; i += kSampleThreads) fn(key_value(uint32_t(s.kept[i] >> 32)), int(~uint32_t(s.kept[i])));
    } else {
      for_row(row, vocab, fn);
    }
  }

  __device__ __forceinline__ bool in(float x, uint32_t k) const { return x == x && k >= least; }

  // histogram over the `bits` bits of the value key above `shift`, of the keys that begin with prefix
  template <bool MASS = true>
  __device__ __forceinline__ void histogram(int shift, int bits, uint32_t prefix) {
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += kSampleThreads) { s.mass[i] = 0; s.count[i] = 0; }
    __syncthreads();
    each([&](float x, int) {
      const uint32_t k = value_key(x);
      if (!in(x, k) || (shift + bits < 32 && (k >> (shift + bits)) != prefix)) return;
      const uint32_t b = (k >> shift) & ((1u << bits) - 1);
      if (MASS) atomicAdd(&s.mass[b], weight(x));
      atomicAdd(&s.count[b], 1u);
    });
    __syncthreads();
  }

  // the n-th (from 0) of the elements with this value key, by index
  __device__ __forceinline__ uint32_t nth_equal(uint32_t key, uint32_t n) {
    constexpr int EV = Elem<T>::kVec;
    const int n_vec = (vocab + EV - 1) / EV;
    uint32_t base = 0;
    for (int v0 = 0; v0 < n_vec; v0 += kSampleThreads) {
      const int v = v0 + threadIdx.x;
      uint32_t hits = 0;
      for (int e = 0; e < EV; ++e) {
        const int i = v * EV + e;
        if (v < n_vec && i < vocab) {
          const float x = Elem<T>::load1(row + i);
          if (x == x && value_key(x) == key) hits |= 1u << e;
        }
      }
      u64 none = 0;
      uint32_t before = __popc(hits);
      scan_before(s, none, before);
      before += base;
      if (before <= n && n < before + __popc(hits)) {
        for (; before < n; ++before) hits &= hits - 1;
        s.found_index = uint32_t(v * EV + __ffs(hits) - 1);
      }
      uint32_t all = 0;
      for (int w = 0; w < kSampleWaves; ++w) all += s.wave_count[w];
      base += all;
      if (n < base) break;
    }
    __syncthreads();
    return s.found_index;
  }

  // The token at which the running weight (or count) reaches target, 1 <= target <= what there is in all: its place; its key and index in
  // s.found_key, s.found_index.  The histogram of the first bits is there before and, if `keep`, after.
  __device__ __forceinline__ Place select(u64 target, bool by_mass, bool keep) {
    reset_place(s);
    Place p = find_bin(s, s.mass, s.count, kBins, target, by_mass);
    uint32_t prefix = p.bin;
    u64 mass_before = p.mass_before;
    uint32_t count_before = p.count_before;
    target -= by_mass ? p.mass_before : p.count_before;
    int shift = 32 - kBinBits;
    while (p.count > kList && shift > 0) {
      const int bits = min(shift, kBinBits);
      shift -= bits;
      histogram(shift, bits, prefix);
      reset_place(s);
      p = find_bin(s, s.mass, s.count, kBins, target, by_mass);
      prefix = (prefix << bits) | p.bin;
      mass_before += p.mass_before;
      count_before += p.count_before;
      target -= by_mass ? p.mass_before : p.count_before;
    }
    const bool lost = shift < 32 - kBinBits;
    if (p.count > kList) {                       // equal values: the index decides
      const float x = key_value(prefix);
      const u64 w = weight(x), n = by_mass ? (target - 1) / w : target - 1;
      nth_equal(prefix, uint32_t(n));
      if (threadIdx.x == 0) s.found_key = prefix;
      p = Place{mass_before + n * w, w, uint32_t(count_before + n), 1, 0};
    } else {
      __syncthreads();
      if (threadIdx.x == 0) s.n_list = 0;
      __syncthreads();
      each([&](float x, int i) {
        const uint32_t k = value_key(x);
        if (in(x, k) && (k >> shift) == prefix) s.list[atomicAdd(&s.n_list, 1u)] = (u64(k) << 32) | uint32_t(~i);
      });
      __syncthreads();
      constexpr int PER = kList / kSampleThreads;
      const uint32_t n = s.n_list;
      u64 key[PER], w[PER];
      bool live[PER];
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        const uint32_t i = threadIdx.x + j * kSampleThreads;
        live[j] = i < n;
        key[j] = live[j] ? s.list[i] : 0;
        w[j] = live[j] ? weight(key_value(uint32_t(key[j] >> 32))) : 0;
      }
      for (int sh = 56; sh >= 0; sh -= 8) {
        if (threadIdx.x < 256) { s.dmass[threadIdx.x] = 0; s.dcount[threadIdx.x] = 0; }
        reset_place(s);
#pragma unroll
        for (int j = 0; j < PER; ++j)
          if (live[j]) {
            atomicAdd(&s.dmass[(key[j] >> sh) & 255], w[j]);
            atomicAdd(&s.dcount[(key[j] >> sh) & 255], 1u);
          }
        __syncthreads();
        p = find_bin(s, s.dmass, s.dcount, 256, target, by_mass);
        mass_before += p.mass_before;
        count_before += p.count_before;
        target -= by_mass ? p.mass_before : p.count_before;
#pragma unroll
        for (int j = 0; j < PER; ++j) live[j] = live[j] && ((key[j] >> sh) & 255) == p.bin;
        __syncthreads();
        if (p.count == 1) break;
      }
#pragma unroll
      for (int j = 0; j < PER; ++j)
        if (live[j]) { s.found_key = uint32_t(key[j] >> 32); s.found_index = ~uint32_t(key[j]); }
      p.mass_before = mass_before;
      p.count_before = count_before;
    }
    __syncthreads();
    if (lost && keep) histogram(32 - kBinBits, kBinBits, 0);
    return p;
  }
};

// The settings of a row.
struct Settings {
  float temperature, top_p, min_p, u;
  int32_t top_k;
};
__device__ __forceinline__ Settings settings_of(const SampleArgs &a, int64_t r) {
  const uint32_t set = uint32_t(r) / uint32_t(a.rows_per_set);        // at most 2^21 rows
  return {a.temperature ? a.temperature[set] : 1.f, a.top_p ? a.top_p[set] : 1.f, a.min_p ? a.min_p[set] : 0.f,
          fminf(fmaxf(a.u[r], 0.f), 0x1.fffffep-1f), a.top_k ? a.top_k[set] : 0};      // u: NaN counts as 0
}
__device__ __forceinline__ Weights weights_of(float m, float temperature, int vocab, const double *table) {
  return Weights{m, 64.0 * 1.44269504088896340736 / double(temperature), 62 - (32 - __clz((vocab - 1) | 1)), table};
}
// least value that min-p leaves
__device__ __forceinline__ float min_p_value(float m, float temperature, float min_p) {
  if (!(min_p > 0.f)) return -INFINITY;
  if (min_p >= 1.f || m == INFINITY) return m;
  const double limit = double(m) + double(temperature) * log(double(min_p));
  const float f = float(limit);
  return double(f) < limit ? nextafterf(f, INFINITY) : f;
}
// what top-p leaves of a total weight begins at the token that reaches this; the draw is the token that reaches that
__device__ __forceinline__ u64 top_p_target(float top_p, u64 total) {
  const double want = ceil(double(fmaxf(top_p, 0.f)) * double(total));
  return want < 1.0 ? 1 : min(u64(want), total);
}
__device__ __forceinline__ u64 draw_target(float u, u64 total) { return min(u64(floor(double(u) * double(total))) + 1, total); }
__device__ __forceinline__ void write_result(const SampleArgs &a, int64_t r, int32_t token, float x, const Weights &w, float temperature,
                                             u64 total) {
  a.token[r] = token;
  if (a.logprob) {
    const double z = x == w.m ? 0.0 : (double(x) - double(w.m)) / double(temperature);
    a.logprob[r] = float(z - log(ldexp(double(total), -w.s_bits)));
  }
}

template <typename T>
__device__ __forceinline__ void sample_general(const SampleArgs &a, int64_t r, SampleLds &s) {
  const T *row = static_cast<const T *>(a.logits) + r * a.row_stride;
  const int vocab = int(a.vocab);
  const Settings set = settings_of(a, r);
  fill_table(s.table);

  // the first token of the order
  u64 top = 0;
  for_row(row, vocab, [&](float x, int i) {
    const uint32_t k = value_key(x);
    if (x == x && k > kNegInfKey) { const u64 c = (u64(k) << 32) | uint32_t(~i); top = c > top ? c : top; }
  });
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) { const u64 o = __shfl_xor(top, off); top = o > top ? o : top; }
  if ((threadIdx.x & 63) == 0) s.wave_top[threadIdx.x >> 6] = top;
  __syncthreads();
  for (int w = 0; w < kSampleWaves; ++w) top = s.wave_top[w] > top ? s.wave_top[w] : top;
  if (top == 0 || !(set.temperature > 0.f)) {
    if (threadIdx.x == 0) {
      a.token[r] = top ? int32_t(~uint32_t(top)) : -1;
      if (a.logprob) a.logprob[r] = top ? 0.f : -INFINITY;
    }
    return;
  }
  const float m = key_value(uint32_t(top >> 32));
  const uint32_t least = max(kNegInfKey + 1, value_key(min_p_value(m, set.temperature, set.min_p)));
  RowSearch<T> find{row, vocab, least, weights_of(m, set.temperature, vocab, s.table), s};
  // what takes part in all
  auto totals = [&](u64 &mass, uint32_t &n) {
    mass = 0;
    n = 0;
    for (int i = threadIdx.x; i < kBins; i += kSampleThreads) { mass += s.mass[i]; n += s.count[i]; }
    const u64 own = mass;
    const uint32_t own_n = n;
    scan_before(s, mass, n);
    if (threadIdx.x == kSampleThreads - 1) s.place = Place{0, mass + own, 0, n + own_n, 0};
    __syncthreads();
    mass = s.place.mass;
    n = s.place.count;
    __syncthreads();
  };
  constexpr int kShift = 32 - kBinBits;
  u64 total = 0;
  uint32_t n = 0;
  bool cut = false;
  if (set.top_k > 0) {
    // Counts tell which bins the first top_k tokens lie in.  The tokens of those bins (and no others) are weighed, and where they
    // are few they are put aside, so that nothing below reads the row again.
    find.template histogram<false>(kShift, kBinBits, 0);
    totals(total, n);
    cut = uint32_t(set.top_k) < n;
    if (cut) {
      reset_place(s);
      const Place p = find_bin(s, s.mass, s.count, kBins, u64(set.top_k), false);
      find.least = max(find.least, p.bin << kShift);
      if (p.count_before + p.count <= kList) {
        __syncthreads();
        if (threadIdx.x == 0) s.n_kept = 0;
        __syncthreads();
        for_row(row, vocab, [&](float x, int i) {
          const uint32_t k = value_key(x);
          if (find.in(x, k)) s.kept[atomicAdd(&s.n_kept, 1u)] = (u64(k) << 32) | uint32_t(~i);
        });
        __syncthreads();
        find.few = true;
        if (s.n_kept <= kSortedList) {
          // So few are sorted, each by the number that come before it (1.5 us), and every search is one comparison.
          const uint32_t kept = s.n_kept, tid = threadIdx.x;
          if (tid < kept) {
            const u64 mine = s.kept[tid];
            uint32_t rank = 0;
#pragma unroll 8
            for (uint32_t j = 0; j < kept; ++j) rank += s.kept[j] > mine;
            s.list[rank] = mine;
          }
          __syncthreads();
          const u64 mine = tid < min(kept, uint32_t(set.top_k)) ? s.list[tid] : 0;
          const float x = key_value(uint32_t(mine >> 32));
          const u64 w = mine ? find.weight(x) : 0;
          u64 before = w;
          uint32_t none = 0;
          scan_before(s, before, none);
          // the weight up to the token that reaches a target, and the token itself
          auto reach = [&](u64 target) {
            if (before < target && target <= before + w) {
              s.place.mass = before + w;
              s.found_key = uint32_t(mine >> 32);
              s.found_index = ~uint32_t(mine);
            }
            __syncthreads();
            const u64 mass = s.place.mass;
            __syncthreads();
            return mass;
          };
          if (tid == kSampleThreads - 1) s.place.mass = before + w;
          __syncthreads();
          total = s.place.mass;
          __syncthreads();
          if (set.top_p < 1.f) total = reach(top_p_target(set.top_p, total));
          reach(draw_target(set.u, total));
          if (tid == 0) write_result(a, r, int32_t(s.found_index), key_value(s.found_key), find.weight, set.temperature, total);
          return;
        }
      }
    }
  }
  find.histogram(kShift, kBinBits, 0);
  if (cut) {
    const Place p = find.select(u64(set.top_k), false, true);
    total = p.mass_before + find.weight(key_value(s.found_key));
  } else {
    totals(total, n);
  }
  if (set.top_p < 1.f) {
    const Place p = find.select(top_p_target(set.top_p, total), true, true);
    total = p.mass_before + find.weight(key_value(s.found_key));
  }
  find.select(draw_target(set.u, total), true, false);
  if (threadIdx.x == 0) write_result(a, r, int32_t(s.found_index), key_value(s.found_key), find.weight, set.temperature, total);
}

__global__ __launch_bounds__(kSampleThreads) void sample_f32_kernel(SampleArgs a) {
  __shared__ SampleLds s;
  sample_general<float>(a, blockIdx.x, s);
}
__global__ __launch_bounds__(kSampleThreads) void sample_bf16_long_kernel(SampleArgs a) {
  __shared__ SampleLds s;
  sample_general<__bf16>(a, blockIdx.x, s);
}

// ---- bf16: a row as a histogram of its values ---------------------------------------------------------------------------

// 16-bit order of a bf16 value: like value_key, but -0 comes right behind +0 (they weigh the same; only the search for a token's
// index has to take them together).  Keys up to 0x7f are -inf and negative NaN, above 0xff80 (+inf) positive NaN.
constexpr uint32_t kFirst16 = 0x80, kLast16 = 0xff80, kZero16 = 0x8000, kMinusZero16 = 0x7fff;
__device__ __forceinline__ float key16_value(uint32_t k) { return __uint_as_float((k >> 15 ? k & 0x7fffu : ~k & 0xffffu) << 16); }

struct CountLds {
  uint32_t hist[1 << 15];               // two 16-bit counts each
  u64 g_mass[1024];                     // of 64 keys: weight and number of the tokens that take part
  uint32_t g_count[1024];
  u64 flags[128];                       // a byte per group: has it any token?
  u64 some[kSampleWaves];               // a bit per group
  uint16_t groups[1024];                // those that have any, ascending
  u64 wave_mass[kSampleWaves];
  uint32_t wave_count[kSampleWaves];
  double table[64];
  u64 f_mass, total;
  uint32_t f_group, f_count, n, counted, index, hits[16], wave_hits[kSampleWaves];
};

// A row of at most 8192 NV logits, NV vectors per thread.
template <int NV>
struct RowVectors {
  static constexpr uint32_t kPad = 0xff80ff80u;   // -inf
  const uint16_t *row;
  int vocab;
  u32x4 tail;                                     // the last, partial vector, in place of the padding that its thread has there
  int tail_i;
  __device__ __forceinline__ RowVectors(const SampleArgs &a, int64_t r)
      : row(static_cast<const uint16_t *>(a.logits) + r * a.row_stride), vocab(int(a.vocab)), tail{kPad, kPad, kPad, kPad} {
    tail_i = vocab % 8 && int(threadIdx.x) == vocab / 8 % kSampleThreads ? vocab / 8 / kSampleThreads : -1;
    if (tail_i >= 0) {
#pragma unroll
      for (int e = 0; e < 7; ++e)
        if (e < vocab % 8) {
          const uint32_t x = row[vocab / 8 * 8 + e];
          tail[e / 2] = e & 1 ? (tail[e / 2] & 0xffffu) | x << 16 : (tail[e / 2] & 0xffff0000u) | x;
        }
    }
  }
  __device__ __forceinline__ u32x4 operator()(int i) const {
    const int at = i * kSampleThreads + threadIdx.x;
    u32x4 x = {kPad, kPad, kPad, kPad};
    if (at < vocab / 8) x = ld16(row + int64_t(at) * 8);
    return x;
  }
};

// The vectors of a row are in registers if there is room for them (KEEP: v), or are read when they are counted and again, from the caches,
// when the token's index is looked for.  Returns false, having written nothing, if a value occurs too often for a 16-bit count.
template <int NV, bool KEEP>
__device__ __forceinline__ bool sample_counts(const SampleArgs &a, int64_t r, const RowVectors<NV> &load, u32x4 (&v)[KEEP ? NV : 1],
                                              CountLds &s) {
  static_assert(KEEP || NV % 4 == 0, "read in fours");
  constexpr uint32_t kPad = RowVectors<NV>::kPad;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int vocab = int(a.vocab), n_vec = (vocab + 7) / 8, tail_i = load.tail_i;
  const u32x4 tail = load.tail;
  const Settings set = settings_of(a, r);
  fill_table(s.table);
#pragma unroll
  for (int i = 0; i < 8; ++i) reinterpret_cast<u32x4 *>(s.hist)[i * kSampleThreads + tid] = u32x4{0, 0, 0, 0};
  s.g_mass[tid] = 0;
  s.g_count[tid] = 0;
  if (tid < 16) s.hits[tid] = 0;
  if (tid == 0) s.counted = 0;
  __syncthreads();

  // two keys of a word at once: all bits of a negative number flip, the sign of a positive one
  auto keys = [](uint32_t w) { const uint32_t sign = (w >> 15) & 0x00010001u; return w ^ ((sign << 16) - sign | 0x80008000u); };
  // -inf (padding, masked tokens: often most of a row) is no value, and its atomics would all be one after the other
  uint32_t out = 0;
  const bool may_overflow = NV > 7 && n_vec * 8 > 65535;
  // fn(vector, i) for all vectors of the thread; read from memory, four in flight
  auto vectors = [&](auto first, auto &&fn) {
    if constexpr (KEEP) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (decltype(first)::value) v[i] = i == tail_i ? tail : v[i];
        fn(v[i], i);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
#pragma unroll 1
      for (int i0 = 0; i0 < NV; i0 += 4) {
        u32x4 x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = load(i0 + j);
#pragma unroll
        for (int j = 0; j < 4; ++j) fn(i0 + j == tail_i ? tail : x[j], i0 + j);
      }
    }
  };
  vectors(std::true_type{}, [&](const u32x4 &x, int) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t k = keys(x[e]), lo = k & 0xffffu, hi = k >> 16;
      if (may_overflow) out += (lo == 0x7f) + (hi == 0x7f);
      if (lo != 0x7f) atomicAdd(&s.hist[lo >> 1], (lo & 1) * 0xffffu + 1);
      if (hi != 0x7f) atomicAdd(&s.hist[hi >> 1], (hi & 1) * 0xffffu + 1);
    }
  });
  __syncthreads();

  // which groups of 64 keys hold any token: a wave reads 8 groups at a time, eight lanes a group
  uint32_t counted = out;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int w0 = wave * 2048 + j * 256 + lane * 4;
    const u32x4 c = *reinterpret_cast<const u32x4 *>(&s.hist[w0]);
    const u64 some = __ballot((c[0] | c[1] | c[2] | c[3]) != 0);
    if (lane == 0) s.flags[wave * 8 + j] = some;
    if (may_overflow)
#pragma unroll
      for (int e = 0; e < 4; ++e) counted += (c[e] & 0xffffu) + (c[e] >> 16);
  }
  if (may_overflow) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) counted += __shfl_xor(counted, off);
    if (lane == 0) atomicAdd(&s.counted, counted);
  }
  __syncthreads();
  // (a count that overflows loses 65536, or loses it and adds one to its neighbour)
  if (may_overflow && s.counted != uint32_t(NV * kSampleThreads * 8)) return false;
  const bool some = (s.flags[tid >> 3] >> (8 * (tid & 7)) & 0xff) != 0 && tid >= int(kFirst16 / 64) && tid <= int(kLast16 / 64);
  const u64 some_here = __ballot(some);
  if (lane == 0) s.some[wave] = some_here;
  __syncthreads();
  const uint32_t groups_to = row_scan(uint32_t(__popcll(s.some[lane & (kSampleWaves - 1)])));
  const int n_groups = int(lane_value(groups_to, kSampleWaves - 1));
  if (some)
    s.groups[(wave ? lane_value(groups_to, wave - 1) : 0) + uint32_t(__popcll(some_here & ((u64(1) << lane) - 1)))] = uint16_t(tid);
  __syncthreads();
  auto count_of = [&](uint32_t key) { return (s.hist[key >> 1] >> (16 * (key & 1))) & 0xffffu; };
  // the largest value
  uint32_t top = 0;
  for (int i = n_groups - 1; i >= 0 && top == 0; --i) {
    const uint32_t first = uint32_t(s.groups[i]) * 64, key = first + lane;
    const u64 here = __ballot(key <= kLast16 && count_of(key) > 0);
    if (here) top = first + (63 - __builtin_clzll(here));
  }
  const float m = key16_value(top);

  // the n-th (from 0) token with this key, by index; `several`: there are more
  auto index_of = [&](uint32_t key, uint32_t n, bool several) {
    const uint32_t raw = key >> 15 ? key & 0x7fffu : ~key & 0xffffu, pair = raw | raw << 16;
    const uint32_t mask = raw << 17 ? ~0u : 0x7fff7fffu;              // zeros of both signs
    auto hits = [&](const u32x4 &x) {
      uint32_t h = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t d = (x[e] ^ pair) & mask;
        h |= uint32_t((d & 0xffffu) == 0) << (2 * e) | uint32_t((d >> 16) == 0) << (2 * e + 1);
      }
      return h;
    };
    auto any = [&](const u32x4 &x) {      // halves without a difference, found by the least of four words' halves
      u16x2 least_of = {0xffff, 0xffff};
#pragma unroll
      for (int e = 0; e < 4; ++e) least_of = __builtin_elementwise_min(least_of, __builtin_bit_cast(u16x2, (x[e] ^ pair) & mask));
      return least_of[0] == 0 || least_of[1] == 0;
    };
    vectors(std::false_type{}, [&](const u32x4 &x, int i) {
      if (any(x)) {
        const uint32_t h = hits(x);
        if (several) atomicAdd(&s.hits[i], uint32_t(__popc(h)));
        else s.index = uint32_t(i * kSampleThreads + tid) * 8 + __ffs(h) - 1;
      }
    });
    __syncthreads();
    if (several) {
      int i = 0;
      while (i < NV - 1 && n >= s.hits[i]) n -= s.hits[i++];
      u32x4 x = {kPad, kPad, kPad, kPad};
      if constexpr (KEEP) {
#pragma unroll
        for (int j = 0; j < NV; ++j) x = i == j ? v[j] : x;
      } else {
        x = load(i);
      }
      const uint32_t h = hits(i == tail_i ? tail : x);
      uint32_t before = wave_scan(uint32_t(__popc(h)));
      if (lane == 63) s.wave_hits[wave] = before;
      __syncthreads();
      before -= __popc(h);
      for (int w = 0; w < wave; ++w) before += s.wave_hits[w];
      if (before <= n && n < before + __popc(h)) {
        uint32_t left = h;
        for (; before < n; ++before) left &= left - 1;
        s.index = uint32_t(i * kSampleThreads + tid) * 8 + __ffs(left) - 1;
      }
      __syncthreads();
    }
    return int32_t(s.index);
  };

  if (top == 0 || !(set.temperature > 0.f)) {
    const bool zero = top == kZero16 || top == kMinusZero16;
    const int32_t token = top ? index_of(top, 0, zero ? count_of(kZero16) + count_of(kMinusZero16) > 1 : count_of(top) > 1) : -1;
    if (tid == 0) {
      a.token[r] = token;
      if (a.logprob) a.logprob[r] = top ? 0.f : -INFINITY;
    }
    return true;
  }
  const Weights weight = weights_of(m, set.temperature, vocab, s.table);
  const float least = min_p_value(m, set.temperature, set.min_p);

  // weigh the groups that hold any: a wave four at a time, sixteen lanes a group, four keys a lane
  for (int i0 = wave * 4; i0 < n_groups; i0 += kSampleWaves * 4) {
    const int i = i0 + (lane >> 4);
    const uint32_t g = s.groups[min(i, n_groups - 1)], key0 = g * 64 + (lane & 15) * 4;
    const uint2 counts = *reinterpret_cast<const uint2 *>(&s.hist[key0 >> 1]);
    u64 mass = 0;
    uint32_t n = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float x = key16_value(key0 + e);
      uint32_t c = ((e < 2 ? counts.x : counts.y) >> (16 * (e & 1))) & 0xffffu;
      if (key0 + e > kLast16 || !(x >= least)) c = 0;
      mass += c * weight(c ? x : m);
      n += c;
    }
    mass = row_scan(mass);
    if ((lane & 15) == 15 && i < n_groups) s.g_mass[g] = mass;
    if (set.top_k > 0) {
      n = row_scan(n);
      if ((lane & 15) == 15 && i < n_groups) s.g_count[g] = n;
    }
  }
  __syncthreads();
  // thread t has the group that is t-th from the top
  const u64 g_mass = s.g_mass[1023 - tid];
  const uint32_t g_count = s.g_count[1023 - tid];
  u64 mass_before = g_mass;
  uint32_t count_before = g_count;
  scan_before(s, mass_before, count_before);
  if (tid == kSampleThreads - 1) { s.total = mass_before + g_mass; s.n = count_before + g_count; }
  __syncthreads();

  struct Found {
    uint32_t key, count, nth;             // the value, its tokens, and which of them
    u64 mass;                             // of the order up to that token
  };
  auto find = [&](u64 target, bool by_mass) {
    if (by_mass ? mass_before < target && target <= mass_before + g_mass
                : count_before < target && target <= u64(count_before) + g_count) {
      s.f_group = 1023 - tid;
      s.f_mass = mass_before;
      s.f_count = count_before;
    }
    __syncthreads();
    // every wave for itself: lane L has key 63 - L of the group
    const uint32_t key = s.f_group * 64 + 63 - lane;
    const float x = key16_value(key);
    const uint32_t c = key <= kLast16 && x >= least ? count_of(key) : 0;
    const u64 w = c ? weight(x) : 0;
    u64 mass = c * w;
    uint32_t count = c;
    mass = wave_scan(mass);
    count = wave_scan(count);
    mass += s.f_mass;
    count += s.f_count;
    const int at = __builtin_ctzll(__ballot(by_mass ? target <= mass : target <= count) | u64(1) << 63);
    const u64 after = lane_value(mass, at), wf = lane_value(w, at);
    Found f;
    f.key = lane_value(key, at);
    f.count = lane_value(c, at);
    const u64 before = after - f.count * wf;
    f.nth = 0;
    if (!by_mass) {
      f.nth = uint32_t(target - 1) - (lane_value(count, at) - f.count);
    } else if (f.count > 1) {             // (target - before - 1) / wf, by a quotient in 64 bits and what it is off
      const u64 rest = target - before - 1;
      u64 n = u64(double(rest) / double(wf));
      if (n * wf > rest) --n;
      else if (rest - n * wf >= wf) ++n;
      f.nth = uint32_t(n);
    }
    f.mass = before + u64(f.nth + 1) * wf;
    __syncthreads();                      // everybody has read what the next search writes
    return f;
  };
  u64 total = s.total;
  if (set.top_k > 0 && uint32_t(set.top_k) < s.n) total = find(u64(set.top_k), false).mass;
  if (set.top_p < 1.f) total = find(top_p_target(set.top_p, total), true).mass;
  Found f = find(draw_target(set.u, total), true);
  bool several = f.count > 1;
  if (f.key == kZero16 || f.key == kMinusZero16) {
    const uint32_t plus = count_of(kZero16);
    if (f.key == kMinusZero16) f.nth += plus;
    several = plus + count_of(kMinusZero16) > 1;
  }
  const int32_t token = index_of(f.key, f.nth, several);
  if (tid == 0) write_result(a, r, token, key16_value(f.key), weight, set.temperature, total);
  return true;
}

// Out of line: its registers are none of the path that rows take.  The arguments come in LDS: as a reference to the kernel's they were copied
// to memory by every workgroup (64 rows of 128256 32.2 / 29.0 us, 1024 rows 150 / 127).
struct AgainLds {
  SampleLds general;
  SampleArgs args;
};
__attribute__((noinline)) __device__ void sample_again(AgainLds &s, int64_t r) { sample_general<__bf16>(s.args, r, s.general); }

template <int NV>
__global__ __launch_bounds__(kSampleThreads) void sample_bf16_kernel(SampleArgs a) {
  __shared__ CountLds s;
  const RowVectors<NV> row(a, blockIdx.x);
  u32x4 v[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) v[i] = row(i);
  sample_counts<NV, true>(a, blockIdx.x, row, v, s);
}

template <int NV>
__global__ __launch_bounds__(kSampleThreads) void sample_bf16_wide_kernel(SampleArgs a) {
  __shared__ union { CountLds counts; AgainLds again; } s;
  const RowVectors<NV> row(a, blockIdx.x);
  u32x4 none[1] = {};
  if (sample_counts<NV, false>(a, blockIdx.x, row, none, s.counts)) return;
  __syncthreads();
  if (threadIdx.x == 0) s.again.args = a;
  __syncthreads();
  sample_again(s.again, blockIdx.x);
}

}  // namespace

hipError_t launch_sample(const SampleArgs &a, sp_dtype dtype, hipStream_t s) {
  // A launch has fewer than 2^32 threads.  More rows go in several, each of whole sets of settings, or of a part of one set.
  constexpr int64_t kMost = int64_t(1) << 21;
  const int64_t per = a.rows_per_set, esz = dtype == SP_F32 ? 4 : 2;
  auto go = [&](auto kernel) {
    for (int64_t r = 0, n; r < a.n_rows; r += n) {
      n = std::min(a.n_rows - r, per <= kMost ? kMost / per * per : std::min(kMost, per - r % per));
      SampleArgs part = a;
      part.logits = static_cast<const char *>(a.logits) + r * a.row_stride * esz;
      part.u = a.u + r;
      part.token = a.token + r;
      if (a.logprob) part.logprob = a.logprob + r;
      if (a.temperature) part.temperature = a.temperature + r / per;
      if (a.top_k) part.top_k = a.top_k + r / per;
      if (a.top_p) part.top_p = a.top_p + r / per;
      if (a.min_p) part.min_p = a.min_p + r / per;
      hipLaunchKernelGGL(kernel, dim3(unsigned(n)), dim3(kSampleThreads), 0, s, part);
    }
  };
  // bf16, by the vectors of 8 logits that a thread has.  Up to 4 and 7 are kept in registers (with more there are not enough of them, and
  // a 16-bit count could overflow); up to 16, as many as CountLds::hits has places for, are read again.  Beyond that the general
  // search reads a row several times: right, and slow, and nothing but its being written stands against counting longer rows as well.  64 / 1024 rows
  // with top-p, us: 32768 tokens 14.7 / 55, 32776 16.1 / 60, 57344 17.2 / 70, 57352 25.6 / 102, 131072 30.4 / 130, 131080 126 / 486,
  // 152064 139 / 577, 256000 369 / 1212.
  const int64_t nv = (a.vocab + 8 * kSampleThreads - 1) / (8 * kSampleThreads);
  if (dtype == SP_F32) go(sample_f32_kernel);
  else if (nv <= 4) go(sample_bf16_kernel<4>);
  else if (nv <= 7) go(sample_bf16_kernel<7>);
  else if (nv <= 16) go(sample_bf16_wide_kernel<16>);
  else go(sample_bf16_long_kernel);
  return hipGetLastError();
}

}  // namespace sp
