// a5: attention of a tree of drafted tokens over the joined cache.
//
// Node i sees the joined cache and the response cache completely, and of the tree itself and its ancestors: a bit mask of 64 nodes.
// One workgroup per (prompt, KV head, node); a wave per query head walks the keys 64 at a time with a running maximum and sum.
#include "sp_device.h"
#include "sp_internal.h"
#include "sp_key_table.h"

namespace sp {

constexpr int kTreeThreads = 256;

// Bit j of lane i's mask: node j is node i or an ancestor of it.  Six doublings reach all of 64 nodes, since parents come first.
__device__ __forceinline__ uint64_t ancestor_mask(const int32_t *parent, int64_t base, int n) {
  const int i = threadIdx.x & 63;
  int up = -1;
  if (i < n) {
    up = parent ? parent[base + i] : i - 1;
    if (up < 0 || up >= i) up = -1;
  }
  uint32_t lo = i < 32 ? 1u << i : 0u, hi = i >= 32 ? 1u << (i - 32) : 0u;
#pragma unroll
  for (int r = 0; r < 6; ++r) {
    const int from = up < 0 ? i : up;
    const uint32_t l = __shfl(lo, from), h = __shfl(hi, from);
    const int u = __shfl(up, from);
    lo |= l;
    hi |= h;
    up = up < 0 ? -1 : u;
  }
  return uint64_t(hi) << 32 | lo;
}

// the nodes' K and V (and positions) to the response cache: one workgroup per (prompt, KV head)
template <typename T, int D>
__device__ __forceinline__ void append_nodes(const PlanDev &pd, const TreeArgs &a, int b, int g, int row0, int n) {
  constexpr int EV = Elem<T>::kVec, LPK = D / EV;
  const int Hkv = pd.n_kv_heads;
  for (int i = threadIdx.x; i < n * LPK; i += blockDim.x) {
    const int node = i / LPK, sub = i % LPK, row = row0 + node;
    if (row0 < 0 || row >= a.resp_capacity) continue;
    const int64_t to = (((int64_t)b * a.resp_capacity + row) * Hkv + g) * D + sub * EV;
    const int64_t from = (((int64_t)b * a.max_nodes + node) * Hkv + g) * D + sub * EV;
    st16(static_cast<T *>(a.Kr) + to, ld16(static_cast<const T *>(a.k_new) + from));
    st16(static_cast<T *>(a.Vr) + to, ld16(static_cast<const T *>(a.v_new) + from));
    if (g == 0 && sub == 0 && a.pos_resp && a.new_pos)
      a.pos_resp[(int64_t)b * a.resp_capacity + row] = a.new_pos[(int64_t)b * a.max_nodes + node];
  }
}

template <typename T, int D>
__global__ __launch_bounds__(kTreeThreads) void tree_simple_kernel(PlanDev pd, TreeArgs a) {
  constexpr int EV = Elem<T>::kVec;
  const int Hq = pd.n_q_heads, Hkv = pd.n_kv_heads, G = Hq / Hkv;
  const int b = blockIdx.x / Hkv, g = blockIdx.x % Hkv, node = blockIdx.y;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int n = a.n_nodes ? min(max(a.n_nodes[b], 0), a.max_nodes) : a.max_nodes;
  if (node >= n) return;
  __shared__ KeyTable tab;
  __shared__ float s_p[4][64], s_q[4][D];
  const RespRows rr = resp_rows(a, b);
  if (node == 0) append_nodes<T, D>(pd, a, b, g, rr.write, n);
  const bool bias = pd.slopes != nullptr;
  build_key_table<T, D>(pd, a, b, g, rr.read, NewKeys{b * a.max_nodes, n, int64_t(Hkv) * D * int64_t(sizeof(T))}, bias, tab);
  const uint64_t all = ancestor_mask(a.parent, (int64_t)b * a.max_nodes, n);
  const uint64_t mask = uint64_t(__shfl(uint32_t(all >> 32), node)) << 32 | __shfl(uint32_t(all), node);
  const int old = tab.n_total - n;
  const float pos_q = bias ? a.new_pos[(int64_t)b * a.max_nodes + node] : 0.f;
  for (int h0 = 0; h0 < G; h0 += 4) {
    const int h = h0 + wave;
    const int head = g * G + min(h, G - 1);
    const int64_t qrow = (((int64_t)b * a.max_nodes + node) * Hq + head) * D;
    __syncthreads();
    for (int d = lane; d < D; d += 64) s_q[wave][d] = Elem<T>::load1(static_cast<const T *>(a.q_new) + qrow + d) * a.scale * kLog2e;
    __syncthreads();
    const float slope2 = bias ? pd.slopes[head] * kLog2e : 0.f;
    float m = kNegBig, l = 0.f, acc[D / 64] = {};
    for (int t0 = 0; t0 < tab.n_total; t0 += 64) {
      const int key = min(t0 + lane, tab.n_total - 1);
      int r = 0;
      while (tab.cum[r + 1] <= key) ++r;
      const bool see = t0 + lane < tab.n_total && (key < old || (mask >> (key - old) & 1));
      float t = 0.f;
      const char *kp = tab.k[r] + int64_t(key - tab.cum[r]) * tab.stride[r];
      for (int d = 0; d < D; d += EV) {
        float x[EV];
        const u32x4 raw = *global_ptr<u32x4>(kp + d * sizeof(T));
        Elem<T>::unpack(raw, x);
#pragma unroll
        for (int e = 0; e < EV; ++e) t = fmaf(x[e], s_q[wave][d + e], t);
      }
      if (bias) t -= slope2 * (pos_q - tab.pos[r][key - tab.cum[r]]);
      if (!see) t = -INFINITY;
      float mx = t;
#pragma unroll
      for (int off = 32; off >= 1; off >>= 1) mx = fmaxf(mx, __shfl_xor(mx, off));
      const float m_new = fmaxf(m, mx), alpha = fast_exp2(m - m_new), p = fast_exp2(t - m_new);
      m = m_new;
      float ps = p;
#pragma unroll
      for (int off = 32; off >= 1; off >>= 1) ps += __shfl_xor(ps, off);
      l = l * alpha + ps;
      s_p[wave][lane] = p;
      __syncthreads();
#pragma unroll
      for (int c = 0; c < D / 64; ++c) acc[c] *= alpha;
      for (int j = 0; j < min(64, tab.n_total - t0); ++j) {
        const int vk = t0 + j;
        if (vk >= old && !(mask >> (vk - old) & 1)) continue;
        int rv = 0;
        while (tab.cum[rv + 1] <= vk) ++rv;
        const T *vp = reinterpret_cast<const T *>(tab.v[rv] + int64_t(vk - tab.cum[rv]) * tab.stride[rv]);
#pragma unroll
        for (int c = 0; c < D / 64; ++c) acc[c] = fmaf(s_p[wave][j], Elem<T>::load1(vp + lane + 64 * c), acc[c]);
      }
      __syncthreads();
    }
    if (h < G)
#pragma unroll
      for (int c = 0; c < D / 64; ++c) Elem<T>::store1(static_cast<T *>(a.o_out) + qrow + lane + 64 * c, acc[c] / l);
  }
}

hipError_t launch_tree_decode(const sp_plan *plan, TreeArgs a, hipStream_t s) {
  const dim3 grid(unsigned(plan->n_prompts) * unsigned(plan->n_kv_heads), unsigned(a.max_nodes)), block(kTreeThreads);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, plan->dev, a); };
  if (plan->dtype == SP_BF16) plan->head_dim == 128 ? go(tree_simple_kernel<__bf16, 128>) : go(tree_simple_kernel<__bf16, 64>);
  else plan->head_dim == 128 ? go(tree_simple_kernel<float, 128>) : go(tree_simple_kernel<float, 64>);
  return hipGetLastError();
}

}  // namespace sp
