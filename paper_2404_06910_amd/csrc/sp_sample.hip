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
// One workgroup per row.
#include "sp_device.h"
#include "sp_internal.h"

namespace sp {

namespace {

constexpr int kSampleThreads = 1024;
constexpr int kSampleWaves = kSampleThreads / 64;
constexpr int kBinBits = 13, kBins = 1 << kBinBits;
constexpr int kList = 4096;                     // keys of one bin that are searched in LDS
constexpr uint32_t kNegInfKey = 0x007fffffu;    // value_key(-inf)

// Order of a value as an unsigned number (the larger the earlier); -0 counts as +0.
__device__ __forceinline__ uint32_t value_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return (u >> 31) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float((k >> 31) ? k & 0x7fffffffu : ~k); }

typedef unsigned long long u64;

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
  Place place;
  uint32_t n_list, found_key, found_index;
};

struct Weights {
  float m;          // largest logit
  double inv_t, scale;
  __device__ __forceinline__ u64 operator()(float x) const {
    if (x == m) return u64(scale);
    if (m == INFINITY) return 0;
    return u64(exp((double(x) - double(m)) * inv_t) * scale);
  }
};

// fn(x, index) for every element of a row, in no order
template <typename T, class F>
__device__ __forceinline__ void for_row(const T *row, int vocab, F &&fn) {
  constexpr int EV = Elem<T>::kVec;
  const int n_vec = vocab / EV;
  for (int v = threadIdx.x; v < n_vec; v += kSampleThreads) {
    float x[EV];
    Elem<T>::unpack(ld16(row + int64_t(v) * EV), x);
#pragma unroll
    for (int e = 0; e < EV; ++e) fn(x[e], v * EV + e);
  }
  const int i = n_vec * EV + threadIdx.x;
  if (i < vocab) fn(Elem<T>::load1(row + i), i);
}

// sums over the threads before this one
__device__ __forceinline__ void scan_before(SampleLds &s, u64 &mass, uint32_t &count) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const u64 own_mass = mass;
  const uint32_t own_count = count;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const u64 m = __shfl_up(mass, off);
    const uint32_t c = __shfl_up(count, off);
    if (lane >= off) { mass += m; count += c; }
  }
  __syncthreads();
  if (lane == 63) { s.wave_mass[wave] = mass; s.wave_count[wave] = count; }
  __syncthreads();
  mass -= own_mass;
  count -= own_count;
  for (int w = 0; w < wave; ++w) { mass += s.wave_mass[w]; count += s.wave_count[w]; }
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

  __device__ __forceinline__ bool in(float x, uint32_t k) const { return x == x && k >= least; }

  // histogram over the `bits` bits of the value key above `shift`, of the keys that begin with prefix
  __device__ __forceinline__ void histogram(int shift, int bits, uint32_t prefix) {
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += kSampleThreads) { s.mass[i] = 0; s.count[i] = 0; }
    __syncthreads();
    for_row(row, vocab, [&](float x, int) {
      const uint32_t k = value_key(x);
      if (!in(x, k) || (shift + bits < 32 && (k >> (shift + bits)) != prefix)) return;
      const uint32_t b = (k >> shift) & ((1u << bits) - 1);
      atomicAdd(&s.mass[b], weight(x));
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
      for_row(row, vocab, [&](float x, int i) {
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

template <typename T>
__global__ __launch_bounds__(kSampleThreads) void sample_kernel(SampleArgs a) {
  __shared__ SampleLds s;
  const int64_t r = blockIdx.x;
  const int64_t set = r / a.rows_per_set;
  const T *row = static_cast<const T *>(a.logits) + r * a.row_stride;
  const int vocab = int(a.vocab);
  const float temperature = a.temperature ? a.temperature[set] : 1.f;
  const int32_t top_k = a.top_k ? a.top_k[set] : 0;
  const float top_p = a.top_p ? a.top_p[set] : 1.f, min_p = a.min_p ? a.min_p[set] : 0.f;

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
  if (top == 0 || !(temperature > 0.f)) {
    if (threadIdx.x == 0) {
      a.token[r] = top ? int32_t(~uint32_t(top)) : -1;
      if (a.logprob) a.logprob[r] = top ? 0.f : -INFINITY;
    }
    return;
  }
  const float m = key_value(uint32_t(top >> 32));
  const int s_bits = 62 - (32 - __clz(vocab - 1 | 1));
  RowSearch<T> find{row, vocab, kNegInfKey + 1, Weights{m, 1.0 / double(temperature), ldexp(1.0, s_bits)}, s};
  if (min_p > 0.f) {
    const double limit = min_p >= 1.f ? double(m) : double(m) + double(temperature) * log(double(min_p));
    float f = float(limit);
    if (double(f) < limit) f = nextafterf(f, INFINITY);
    find.least = max(find.least, value_key(f));
  }
  find.histogram(32 - kBinBits, kBinBits, 0);
  // what takes part in all
  u64 total = 0;
  uint32_t n = 0;
  for (int i = threadIdx.x; i < kBins; i += kSampleThreads) { total += s.mass[i]; n += s.count[i]; }
  {
    const u64 own = total;
    const uint32_t own_n = n;
    scan_before(s, total, n);
    total += own;
    n += own_n;
    if (threadIdx.x == kSampleThreads - 1) s.place = Place{0, total, 0, n, 0};
    __syncthreads();
    total = s.place.mass;
    n = s.place.count;
    __syncthreads();
  }
  if (top_k > 0 && uint32_t(top_k) < n) {
    const Place p = find.select(u64(top_k), false, true);
    total = p.mass_before + find.weight(key_value(s.found_key));
  }
  if (top_p < 1.f) {
    const double want = ceil(double(fmaxf(top_p, 0.f)) * double(total));
    const u64 target = want < 1.0 ? 1 : min(u64(want), total);
    const Place p = find.select(target, true, true);
    total = p.mass_before + find.weight(key_value(s.found_key));
  }
  const float u = fminf(fmaxf(a.u[r], 0.f), 0x1.fffffep-1f);      // NaN: 0
  const u64 target = min(u64(floor(double(u) * double(total))) + 1, total);
  find.select(target, true, false);
  if (threadIdx.x == 0) {
    a.token[r] = int32_t(s.found_index);
    if (a.logprob) {
      const float x = key_value(s.found_key);
      const double z = x == m ? 0.0 : (double(x) - double(m)) * find.weight.inv_t;
      a.logprob[r] = float(z - log(double(total) / find.weight.scale));
    }
  }
}

}  // namespace

hipError_t launch_sample(const SampleArgs &a, sp_dtype dtype, int64_t n_rows, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(n_rows)), block(kSampleThreads);
  if (dtype == SP_BF16) hipLaunchKernelGGL(sample_kernel<__bf16>, grid, block, 0, s, a);
  else hipLaunchKernelGGL(sample_kernel<float>, grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace sp
