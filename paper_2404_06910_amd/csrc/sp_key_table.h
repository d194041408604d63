// What the decode kernels share: the key list of one (prompt, KV head) as ranges in LDS.  Args is a kernel's argument struct
// (kept, k, Kp, Vp and their strides, Kr, Vr, pos_resp, resp_capacity, resp_len, resp_len_add, k_new, v_new, new_pos, few_wgs).
#pragma once

#include "sp_device.h"
#include "sp_internal.h"

namespace sp {

constexpr int kDecMaxRanges = 128;

// The key list of one (prompt, KV head) as ranges with running key counts, in LDS: the prefill ranges of the
// shared part and of the kept paths, the response cache, the new token or tokens.
struct KeyTable {
  int32_t cum[kDecMaxRanges + 3];
  int64_t stride[kDecMaxRanges + 2];           // bytes from one token to the next
  const char *k[kDecMaxRanges + 2], *v[kDecMaxRanges + 2];
  const float *pos[kDecMaxRanges + 2];
  int32_t s_cnt[kDecMaxRanges], s_keys[kDecMaxRanges];
  int32_t n_total, n_ranges;
};

// The rows of k_new / v_new (and new_pos) that a prompt adds: n consecutive ones, `stride` bytes apart.
struct NewKeys {
  int32_t row, n;
  int64_t stride;
};

// One thread per source (the workgroup has min(k, kDecMaxRanges - 1) + 1 of them at least) follows the tables (kept -> path slot descriptor, which carries the first range), so the
// dependent loads of all sources run side by side; a prefix over the sources puts the ranges in order.
// Where no prompt has more than 64 paths, the descriptors of a prompt's paths lie at a fixed place (path_stride; upload_plan
// says where not) and the first wave reads all of them while `kept` is on its way, and picks from its lanes: one memory latency less for every
// launch, and no barrier between the two halves, which one wave does (four tokens of six prompts of 32/8 heads 47.0 -> 45.1 us,
// a request with five tokens of one prompt of 32 heads 89.1 -> 86.2).  With more than four workgroups to a compute unit the
// others' streams hide the latency, and the reads of paths that are not kept cost 0.2 % (64 prompts, 32 heads: 91.1 / 91.4).
template <typename T, int D, class Args>
__device__ __forceinline__ void build_key_table(const PlanDev &pd, const Args &a, int b, int g, int len_r, NewKeys added, bool bias,
                                                KeyTable &t) {
  const int tid = threadIdx.x, Hkv = pd.n_kv_heads;
  const int n_src = min(a.k, kDecMaxRanges - 1) + 1;      // k beyond that: prompts without paths, nothing to keep
  const bool one_wave = a.few_wgs && pd.path_stride > 0 && n_src <= 64;
  RangeDesc src{0, 0, 0, 0};
  if (one_wave) {
    if (tid < 64) {
      RangeDesc path{0, 0, 0, 0};
      int kp = -1;
      if (tid < pd.path_stride) path = pd.path_desc[b * pd.path_stride + tid];
      if (tid > 0 && tid < n_src) kp = a.kept[(int64_t)b * a.k + (tid - 1)];
      const RangeDesc shared = pd.shared_desc[b];
      const RangeDesc mine{__shfl(path.beg, kp & 63), __shfl(path.end, kp & 63), __shfl(path.tok_start, kp & 63),
                           __shfl(path.len, kp & 63)};
      if (tid == 0) src = shared;
      else if (kp >= 0 && kp < pd.path_stride) src = mine;   // paths that the prompt does not have are empty
    }
  } else if (tid == 0) {
    src = pd.shared_desc[b];
  } else if (tid < n_src) {
    const int p0 = pd.path_off[b], np = pd.path_off[b + 1] - p0;
    const int kp = a.kept[(int64_t)b * a.k + (tid - 1)];
    if (kp >= 0 && kp < np) src = pd.path_desc[pd.path_stride > 0 ? b * pd.path_stride + kp : p0 + kp];
  }
  const int beg = src.beg, end = src.end;
  if (tid < n_src) {
    int keys = end > beg ? src.len : 0;
    for (int r = beg + 1; r < end; ++r) keys += pd.dec_ranges[r].len;
    t.s_cnt[tid] = end - beg;
    t.s_keys[tid] = keys;
  }
  if (one_wave) {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  } else {
    __syncthreads();
  }
  if (tid < n_src) {
    int at = 0, cum = 0;
    for (int i = 0; i < tid; ++i) { at += t.s_cnt[i]; cum += t.s_keys[i]; }
    const char *kb = static_cast<const char *>(a.Kp) + (int64_t)g * a.kv_head_stride * int64_t(sizeof(T));
    const char *vb = static_cast<const char *>(a.Vp) + (int64_t)g * a.kv_head_stride * int64_t(sizeof(T));
    const int64_t stride = a.kv_tok_stride * int64_t(sizeof(T));
    for (int r = beg; r < end && at < kDecMaxRanges; ++r, ++at) {
      const KeyRange kr = r == beg ? KeyRange{src.tok_start, src.len} : pd.dec_ranges[r];
      t.cum[at] = cum;
      t.stride[at] = stride;
      t.k[at] = kb + kr.tok_start * stride;
      t.v[at] = vb + kr.tok_start * stride;
      t.pos[at] = bias ? pd.tok_pos + kr.tok_start : nullptr;
      cum += kr.len;
    }
    if (tid == n_src - 1) {
      const int64_t row = int64_t(b) * a.resp_capacity * Hkv + g;
      if (len_r > 0) {
        t.cum[at] = cum;
        t.stride[at] = int64_t(Hkv) * D * int64_t(sizeof(T));
        t.k[at] = reinterpret_cast<const char *>(static_cast<const T *>(a.Kr) + row * D);
        t.v[at] = reinterpret_cast<const char *>(static_cast<const T *>(a.Vr) + row * D);
        t.pos[at] = bias ? a.pos_resp + int64_t(b) * a.resp_capacity : nullptr;
        cum += len_r;
        ++at;
      }
      t.cum[at] = cum;
      t.stride[at] = added.stride;
      t.k[at] = reinterpret_cast<const char *>(static_cast<const T *>(a.k_new) + ((int64_t)added.row * Hkv + g) * D);
      t.v[at] = reinterpret_cast<const char *>(static_cast<const T *>(a.v_new) + ((int64_t)added.row * Hkv + g) * D);
      t.pos[at] = bias ? a.new_pos + added.row : nullptr;
      t.cum[at + 1] = cum + added.n;
      t.n_total = cum + added.n;
      t.n_ranges = at + 1;
    }
  }
  __syncthreads();
}

// K, V and positions are read through pointers from the table: see global_ptr
template <bool STREAM>
__device__ __forceinline__ u32x4 ld16_kv(const char *p) {
  if constexpr (STREAM) return __builtin_nontemporal_load(global_ptr<u32x4>(p));
  else return *global_ptr<u32x4>(p);
}

// Range of a key (vk < n_total, so every search ends at the latest on the new tokens' range).  Every lane keeps one
// running count, so that the range of a wave-uniform key is one comparison and a bit count; walking the counts in LDS
// instead costs a dependent LDS read per range, which a piece of a few dozen keys feels (1 us of 4).
struct RangeSearch {
  const KeyTable &t;
  int32_t my_end;                              // end of range `lane`
  __device__ __forceinline__ explicit RangeSearch(const KeyTable &tab) : t(tab) {
    const int lane = threadIdx.x & 63;
    my_end = lane < t.n_ranges ? t.cum[lane + 1] : INT32_MAX;
  }
  __device__ __forceinline__ int from(int i, int vk) const {
    while (t.cum[i + 1] <= vk) ++i;
    return i;
  }
  // vk wave-uniform
  __device__ __forceinline__ int uniform(int vk) const {
    const int i = __popcll(__ballot(my_end <= vk));
    return i < 64 ? i : __builtin_amdgcn_readfirstlane(from(64, vk));
  }
};

__device__ __forceinline__ int64_t uniform64(int64_t x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane(uint32_t(x)), hi = __builtin_amdgcn_readfirstlane(uint32_t(x >> 32));
  return int64_t((uint64_t(hi) << 32) | lo);
}

// rows of the response cache that take part (the new tokens are not among them), and the row the first new token goes to
struct RespRows { int read, write; };
template <class Args>
__device__ __forceinline__ RespRows resp_rows(const Args &a, int b) {
  const int len_b = (a.resp_len ? a.resp_len[b] : 0) + a.resp_len_add;
  return {len_b < a.resp_capacity ? (len_b < 0 ? 0 : len_b) : a.resp_capacity, len_b};
}

}  // namespace sp
