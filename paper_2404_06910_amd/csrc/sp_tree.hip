// a5: attention of a tree of drafted tokens over the joined cache.
//
// Node i sees the joined cache and the response cache completely, and of the tree itself and its ancestors.  The nodes' rows
// of all query heads that share a KV head are the rows of one small product with that head's keys: row node * G + head.  The keys are the
// list of build_key_table, the nodes last, so that only its last steps know a mask: one bit mask of 64 nodes per row.
//
// A wave walks the keys 32 (fp32: 16) at a time for RT tiles of 16 rows, with a running maximum and sum per row.  The waves of a
// workgroup either take different keys (few rows: nothing is shared, each wave streams through two LDS slots of its own and waits for
// nobody, their sums are added up at the end) or different rows (many rows: K and V are staged once for all of them).
// Where that leaves most of the chip idle, the key list is cut into pieces too, one workgroup each, and a
// second, small kernel adds the pieces up in their order.
#include <algorithm>
#include <type_traits>

#include "sp_key_table.h"
#include "sp_lds_dma.h"

namespace sp {

namespace {

struct TreeDev {
  TreeArgs a;
  int32_t n_pieces;
  float *part;               // n_pieces > 1: [piece][prompt, node, query head][D] sums, then {max, sum} for each
  int64_t rows;              // prompts * nodes * query heads
};

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
  if (row0 < 0) return;
  for (int i = threadIdx.x; i < n * LPK; i += blockDim.x) {
    const int node = i / LPK, sub = i % LPK, row = row0 + node;
    if (row >= a.resp_capacity) continue;
    const int64_t to = (((int64_t)b * a.resp_capacity + row) * Hkv + g) * D + sub * EV;
    const int64_t from = (((int64_t)b * a.max_nodes + node) * Hkv + g) * D + sub * EV;
    st16(static_cast<T *>(a.Kr) + to, ld16(static_cast<const T *>(a.k_new) + from));
    st16(static_cast<T *>(a.Vr) + to, ld16(static_cast<const T *>(a.v_new) + from));
    if (g == 0 && sub == 0 && a.pos_resp && a.new_pos)
      a.pos_resp[(int64_t)b * a.resp_capacity + row] = a.new_pos[(int64_t)b * a.max_nodes + node];
  }
}

// value of a row's four lanes (L, L ^ 16, L ^ 32, L ^ 48) combined
__device__ __forceinline__ float rows_max(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return xhalf_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float rows_sum(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return xhalf_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// What a wave needs to know of its rows: lane L holds row L % 16 of each tile.
template <int RT>
struct Rows {
  int32_t node[RT], head[RT];        // rows past the last repeat it
  bool real[RT];
  uint64_t mask[RT];                 // nodes that the row sees
  float slope2[RT], bias0[RT];       // with a distance penalty: slope * log2 e, and that times minus the row's position
};
template <int RT, bool BIAS>
__device__ __forceinline__ void find_rows(const PlanDev &pd, const TreeArgs &a, int b, int g, int n, int row0, Rows<RT> &r) {
  const int G = pd.n_q_heads / pd.n_kv_heads, l16 = threadIdx.x & 15;
  const uint64_t all = ancestor_mask(a.parent, (int64_t)b * a.max_nodes, n);
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int row = min(row0 + 16 * t + l16, n * G - 1);
    r.real[t] = row0 + 16 * t + l16 < n * G;
    r.node[t] = row / G;
    r.head[t] = g * G + row % G;
    r.mask[t] = uint64_t(__shfl(uint32_t(all >> 32), r.node[t])) << 32 | __shfl(uint32_t(all), r.node[t]);
    r.slope2[t] = BIAS ? pd.slopes[r.head[t]] * kLog2e : 0.f;
    r.bias0[t] = BIAS ? -r.slope2[t] * a.new_pos[(int64_t)b * a.max_nodes + r.node[t]] : 0.f;
  }
}

// Ends a workgroup.  Every wave has m, l (complete, the same in a row's four lanes) and the weighted sums of its rows; Put says
// which dims a lane holds: put(t, fn) calls fn(first dim, four sums) for each of its groups of four.  Waves that took different keys
// (KEYS of them) are added up in LDS, in their order.
template <typename T, int D>
__device__ __forceinline__ void store4(const TreeDev &d, int64_t row, int dim, f32x4 v, float inv) {
  if constexpr (sizeof(T) == 2) {
    bf16x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = static_cast<__bf16>(v[e] * inv);
    *reinterpret_cast<bf16x4 *>(static_cast<__bf16 *>(d.a.o_out) + row * D + dim) = w;
  } else {
    *reinterpret_cast<f32x4 *>(static_cast<float *>(d.a.o_out) + row * D + dim) = v * inv;
  }
}
template <typename T, int D, int RT, int KEYS, class Put>
__device__ __forceinline__ void finish(const PlanDev &pd, const TreeDev &d, int b, const Rows<RT> &r, const float *m, const float *l,
                                       float *lds, Put &&put) {
  constexpr int PITCH = D + 4;                       // 16 rows' vectors fall into different banks
  const int lane = threadIdx.x & 63, l16 = lane & 15, wave = threadIdx.x >> 6;
  const int64_t base = (int64_t)b * d.a.max_nodes * pd.n_q_heads;
  auto out = [&](int64_t row, int dim, f32x4 v, float mm, float ll, bool first) {
    if (d.n_pieces == 1) {
      store4<T, D>(d, row, dim, v, 1.f / ll);
    } else {
      const int64_t at = int64_t(blockIdx.z) * d.rows + row;
      *reinterpret_cast<f32x4 *>(d.part + at * D + dim) = v;
      if (first) {
        d.part[d.n_pieces * d.rows * D + 2 * at] = mm;
        d.part[d.n_pieces * d.rows * D + 2 * at + 1] = ll;
      }
    }
  };
  if constexpr (KEYS == 1) {
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int64_t row = base + (int64_t)r.node[t] * pd.n_q_heads + r.head[t];
      put(t, [&](int dim, f32x4 v) {
        if (r.real[t]) out(row, dim, v, m[t], l[t], dim == 0);
      });
    }
  } else {
    __shared__ float s_m[KEYS][16 * RT], s_l[KEYS][16 * RT];
    __syncthreads();                                 // all waves are done with their slots
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      put(t, [&](int dim, f32x4 v) { *reinterpret_cast<f32x4 *>(lds + ((wave * RT + t) * 16 + l16) * PITCH + dim) = v; });
      if (lane < 16) { s_m[wave][16 * t + lane] = m[t]; s_l[wave][16 * t + lane] = l[t]; }
    }
    __syncthreads();
    constexpr int PER = D / 4;
    const int G = pd.n_q_heads / pd.n_kv_heads;
    for (int i = threadIdx.x; i < 16 * RT * PER; i += 64 * KEYS) {
      const int at = i / PER, dim = i % PER * 4;
      float mm = s_m[0][at], ll = 0.f;
      f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 1; w < KEYS; ++w) mm = fmaxf(mm, s_m[w][at]);
#pragma unroll
      for (int w = 0; w < KEYS; ++w) {
        const float f = fast_exp2(s_m[w][at] - mm);
        const f32x4 x = *reinterpret_cast<const f32x4 *>(lds + (w * 16 * RT + at) * PITCH + dim);
        ll = fmaf(f, s_l[w][at], ll);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = fmaf(f, x[e], v[e]);
      }
      // the row itself: that of tile at / 16, lane at % 16
      const int first = int(blockIdx.y) * 16 * RT, rr = first + at;
      const int n = d.a.n_nodes ? min(max(d.a.n_nodes[b], 0), d.a.max_nodes) : d.a.max_nodes;
      if (rr < n * G) out(base + int64_t(rr / G) * pd.n_q_heads + int64_t(blockIdx.x % pd.n_kv_heads) * G + rr % G, dim, v, mm, ll, dim == 0);
    }
  }
}

__device__ __forceinline__ bool not_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }

}  // namespace

// bf16 on v_mfma_f32_16x16x32_bf16.  Per step of 32 keys (two tiles of 16):
//   S^T[key, row]  = K[key, :] . Q[row, :]         A = K (LDS), B = Q (registers)
//   O^T[d, row]   += V^T[d, key] . P^T[key, row]   A = V (LDS, transpose reads), B = P as it is
// In the accumulator lane L holds row L % 16 and keys 4 (L / 16) + i of each tile, which are bound to the k-slots that the lane feeds in
// the second product.  P is rounded to bf16 there, as the output is (the sum of the weights is not); that is half a step of every weight, and the
// result is as far off as two roundings of it instead of one.
// SHARED: the NW waves take different rows and fill each stage together; otherwise each takes every NW-th step and fills its own.
template <int D, int RT, int NW, bool SHARED, bool BIAS>
__global__ __launch_bounds__(64 * NW) void tree_bf16_kernel(PlanDev pd, TreeDev d) {
  constexpr int ROWB = D * 2, CPR = D / 8, RPC = 256 / ROWB, RG = 64 / CPR;   // LDS row, its 16-byte chunks, rows per 256 bytes, rows per DMA
  constexpr int HALFB = 32 * ROWB, SLOTB = 2 * HALFB;
  constexpr int NI = 32 / RG;                    // DMA instructions per half
  constexpr int KEYS = SHARED ? 1 : NW;
  constexpr int RINGB = 2 * SLOTB * KEYS;
  constexpr int MERGEB = KEYS > 1 ? KEYS * RT * 16 * (D + 4) * 4 : 0;
  constexpr int NJ = D / 32, NC = D / 16;
  __shared__ __attribute__((aligned(1024))) unsigned char ring[RINGB > MERGEB ? RINGB : MERGEB];
  __shared__ __attribute__((aligned(256))) float s_pos[BIAS ? 2 * KEYS : 1][64];
  __shared__ KeyTable tab;
  const TreeArgs &a = d.a;
  const int Hq = pd.n_q_heads, Hkv = pd.n_kv_heads, G = Hq / Hkv;
  const int b = blockIdx.x / Hkv, g = blockIdx.x % Hkv;
  const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = a.n_nodes ? min(max(a.n_nodes[b], 0), a.max_nodes) : a.max_nodes;
  const int row0 = (int(blockIdx.y) * (SHARED ? NW : 1) + (SHARED ? wave : 0)) * 16 * RT;
  if (int(blockIdx.y) * (SHARED ? NW : 1) * 16 * RT >= n * G) return;

  Rows<RT> rows;
  find_rows<RT, BIAS>(pd, a, b, g, n, row0, rows);
  bf16x8 qf[RT][NJ];
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int j = 0; j < NJ; ++j)
      qf[t][j] = *reinterpret_cast<const bf16x8 *>(static_cast<const __bf16 *>(a.q_new) +
                                                   (((int64_t)b * a.max_nodes + rows.node[t]) * Hq + rows.head[t]) * D + (q + 4 * j) * 8);
  const float scale2 = a.scale * kLog2e;
  const RespRows rr = resp_rows(a, b);
  if (blockIdx.y == 0 && blockIdx.z == 0) append_nodes<__bf16, D>(pd, a, b, g, rr.write, n);
  build_key_table<__bf16, D>(pd, a, b, g, rr.read, NewKeys{b * a.max_nodes, n, int64_t(Hkv) * D * 2}, BIAS, tab);
  const RangeSearch find(tab);
  const int n_total = tab.n_total, old = n_total - n;
  // pieces are multiples of 32 keys, so that only steps at the end of the list reach beyond it
  const int piece = ((n_total + d.n_pieces - 1) / d.n_pieces + 31) & ~31;
  const int key0 = min(int(blockIdx.z) * piece, n_total), key1 = min(key0 + piece, n_total);
  const int n_steps = (key1 - key0 + 31) / 32;

  // LDS rows are unpadded; the 16-byte chunks of a row are swizzled on the global side, so that row reads of K (16 rows, one
  // chunk) and transpose reads of V (8 rows of one chunk pair at a time) spread over the banks.
  auto fK = [](int row) { return (row / RPC) % CPR; };
  auto fV = [](int row) { return ((row / RPC) % (CPR / 4)) * 4 | ((row >> 2) & 1) * 2; };
  const uint32_t ring_base = (uint32_t)(size_t)(lds_byte *)ring + (SHARED ? 0 : wave * 2 * SLOTB);
  const uint32_t pos_base = (uint32_t)(size_t)(lds_byte *)&s_pos[0][0] + (SHARED ? 0 : wave * 2 * 256);
  const unsigned char *ringp = ring + (SHARED ? 0 : wave * 2 * SLOTB);
  const int drow = lane / CPR, dslot = lane % CPR;
  constexpr int MINE = SHARED ? (2 * NI + NW - 1) / NW : 2 * NI;           // DMA instructions of a wave per stage

  auto issue = [&](int s, int slot) {
    const int t0 = key0 + 32 * s;
    const int i0 = find.uniform(t0);
    const int c0 = __builtin_amdgcn_readfirstlane(tab.cum[i0]), c1 = __builtin_amdgcn_readfirstlane(tab.cum[i0 + 1]);
    const int64_t stride = uniform64(tab.stride[i0]);
    const uint32_t lds = ring_base + slot * SLOTB;
    // rows RG m .. of the half: consecutive tokens of one range, or each row looked up by itself (past the end: the last key again)
    const bool plain = t0 + 32 <= c1 && stride < (int64_t(1) << 27);
    const char *kb = reinterpret_cast<const char *>(uniform64(reinterpret_cast<int64_t>(tab.k[i0]))) + (t0 - c0) * stride;
    const char *vb = reinterpret_cast<const char *>(uniform64(reinterpret_cast<int64_t>(tab.v[i0]))) + (t0 - c0) * stride;
    const uint32_t row_off = uint32_t(drow) * uint32_t(stride);
#pragma unroll
    for (int x = 0; x < MINE; ++x) {
      const int m2 = SHARED ? wave + x * NW : x;
      if (SHARED && 2 * NI % NW != 0 && m2 >= 2 * NI) break;
      const bool is_v = m2 >= NI;
      const int m = is_v ? m2 - NI : m2, row = RG * m + drow;
      const uint32_t chunk = uint32_t(dslot ^ (is_v ? fV(row) : fK(row))) * 16;
      const uint32_t to = lds + (is_v ? HALFB : 0) + m * (RG * ROWB);
      if (plain) {
        dma16s((is_v ? vb : kb) + RG * m * stride, row_off + chunk, to);
      } else {
        const int vk = min(t0 + row, n_total - 1), i = find.from(i0, vk);
        dma16((is_v ? tab.v[i] : tab.k[i]) + int64_t(vk - tab.cum[i]) * tab.stride[i] + chunk, to);
      }
    }
    if (BIAS && (!SHARED || wave == 0)) {
      const int vk = min(t0 + (lane & 31), n_total - 1), i = find.from(i0, vk);
      dma4(tab.pos[i] + (vk - tab.cum[i]), pos_base + slot * 256);
    }
  };

  float m_run[RT], l_run[RT];
  f32x4 o[RT][NC];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    m_run[t] = kNegBig;
    l_run[t] = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) o[t][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const int tr_row = l16 >> 2, tr_x = (lane & 3) >> 1, tr_sub8 = (lane & 1) * 8;

  // one step on a slot; MASKED: it holds nodes (or reaches beyond them)
  auto step = [&](int t0, int slot, auto masked) {
    constexpr bool MASKED = decltype(masked)::value;
    const unsigned char *sl = ringp + slot * SLOTB;
    f32x4 s[RT][2];
#pragma unroll
    for (int t = 0; t < RT; ++t) s[t][0] = s[t][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const int row = 16 * h + l16;
        const bf16x8 k = *reinterpret_cast<const bf16x8 *>(sl + row * ROWB + ((4 * j + q) ^ fK(row)) * 16);
#pragma unroll
        for (int t = 0; t < RT; ++t) s[t][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, qf[t][j], s[t][h], 0, 0, 0);
      }
    f32x4 kp[2];
    if (BIAS) {
      const float *ps = &s_pos[(SHARED ? 0 : 2 * wave) + slot][0];
#pragma unroll
      for (int h = 0; h < 2; ++h) kp[h] = *reinterpret_cast<const f32x4 *>(ps + 16 * h + 4 * q);
    }
    bf16x8 pb[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      float mx = -INFINITY;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float x = BIAS ? fmaf(s[t][h][i], scale2, fmaf(rows.slope2[t], kp[h][i], rows.bias0[t])) : s[t][h][i] * scale2;
          if (MASKED) {
            const int at = t0 + 16 * h + 4 * q + i - old;          // node of this key
            if (at >= n || (at >= 0 && !(rows.mask[t] >> (at & 63) & 1))) x = -INFINITY;
          }
          s[t][h][i] = x;
          mx = fmaxf(mx, x);
        }
      // The reference may lag behind the maximum by 8 (weights up to 256, which bf16 and the sums absorb): the lanes of a row need
      // not agree on a maximum in every step.
      if (__any(mx > m_run[t] + 8.f)) {
        const float m_new = fmaxf(m_run[t], rows_max(mx)), alpha = fast_exp2(m_run[t] - m_new);
        m_run[t] = m_new;
        l_run[t] *= alpha;
#pragma unroll
        for (int c = 0; c < NC; ++c) o[t][c] *= alpha;
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p = fast_exp2(s[t][h][i] - m_run[t]);
          l_run[t] += p;
          pb[t][4 * h + i] = static_cast<__bf16>(p);
        }
    }
    bf16x8 vf[NC];
    const unsigned char *vs = sl + HALFB + tr_sub8;
    uint32_t bad = 0;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int r0 = 4 * q + tr_row;
      const unsigned char *vp = vs + r0 * ROWB + ((2 * c + tr_x) ^ fV(r0)) * 16;
      const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4 *)vp);
      const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4 *)(vp + 16 * ROWB));
      vf[c] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      if (MASKED) {
        const u32x4 w = __builtin_bit_cast(u32x4, vf[c]);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          bad |= uint32_t((w[e] & 0x7f80u) == 0x7f80u) | uint32_t((w[e] & 0x7f800000u) == 0x7f800000u);
      }
    }
    if (MASKED && __any(bad)) {
      // An infinite V, or NaN, must not reach rows that do not see its key (0 times infinity is NaN): such elements are taken out of
      // the product and added key by key where the weight is not zero.
      const int i0 = find.uniform(t0);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll 1
          for (int from = 0; from < 4; ++from) {
            const int vk = min(t0 + 16 * h + 4 * from + i, n_total - 1), r = find.from(i0, vk);
            const __bf16 *v = reinterpret_cast<const __bf16 *>(tab.v[r] + int64_t(vk - tab.cum[r]) * tab.stride[r]);
#pragma unroll
            for (int t = 0; t < RT; ++t) {
              const float p = __shfl(static_cast<float>(pb[t][4 * h + i]), 16 * from + l16);
#pragma unroll
              for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const float x = static_cast<float>(v[16 * c + 4 * q + e]);
                  if (not_finite(x) && p != 0.f) o[t][c][e] += p * x;
                }
            }
          }
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (not_finite(static_cast<float>(vf[c][e]))) vf[c][e] = static_cast<__bf16>(0.f);
    }
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int t = 0; t < RT; ++t) o[t][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[c], pb[t], o[t][c], 0, 0, 0);
  };
  auto compute = [&](int s, int slot) {
    const int t0 = key0 + 32 * s;
    if (t0 + 32 > old) step(t0, slot, std::true_type{});
    else step(t0, slot, std::false_type{});
  };

  if constexpr (SHARED) {
    if (n_steps > 0) issue(0, 0);
    for (int s = 0; s < n_steps; ++s) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();                             // stage s is there, and nobody reads the other slot any more
      if (s + 1 < n_steps) issue(s + 1, (s + 1) & 1);
      compute(s, s & 1);
    }
  } else {
    // two stages of this wave are in flight whenever it waits
    if (wave < n_steps) issue(wave, 0);
    if (wave + NW < n_steps) issue(wave + NW, 1);
    int slot = 0;
    for (int s = wave; s < n_steps; s += NW, slot ^= 1) {
      if (s + NW < n_steps) {
        if constexpr (BIAS) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(MINE + 1) : "memory");
        else asm volatile("s_waitcnt vmcnt(%0)" ::"n"(MINE) : "memory");
      } else {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      }
      compute(s, slot);
      // the reads of this slot have returned before the next stage may overwrite it
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (s + 2 * NW < n_steps) issue(s + 2 * NW, slot);
    }
  }
#pragma unroll
  for (int t = 0; t < RT; ++t) l_run[t] = rows_sum(l_run[t]);
  finish<__bf16, D, RT, KEYS>(pd, d, b, rows, m_run, l_run, reinterpret_cast<float *>(ring), [&](int t, auto &&fn) {
#pragma unroll
    for (int c = 0; c < NC; ++c) fn(16 * c + 4 * q, o[t][c]);
  });
}

// fp32 on v_mfma_f32_16x16x4_f32, 16 keys a step, everything in 32 bits; K and V come from memory straight into registers.
//   S^T[key, row] = K[key, :] . Q[row, :]       slots bound to dims 16 i + 4 (L / 16) + e
//   O^T[d, row]  += V^T[d, key] . P^T[key, row] slot L / 16 of step r bound to key 4 (L / 16) + r; rows of O^T to dims 64 h + 4 (L % 16) + c
// Sums are kept in short chains that are added up (a single chain of D products rounds several times as much).
template <int D, int RT, int NW, bool BIAS>
__global__ __launch_bounds__(64 * NW) void tree_f32_kernel(PlanDev pd, TreeDev d) {
  constexpr int NI = D / 16, NH = D / 64;
  __shared__ __attribute__((aligned(16))) float merge[NW > 1 ? NW * RT * 16 * (D + 4) : 4];
  __shared__ KeyTable tab;
  const TreeArgs &a = d.a;
  const int Hq = pd.n_q_heads, Hkv = pd.n_kv_heads, G = Hq / Hkv;
  const int b = blockIdx.x / Hkv, g = blockIdx.x % Hkv;
  const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = a.n_nodes ? min(max(a.n_nodes[b], 0), a.max_nodes) : a.max_nodes;
  const int row0 = int(blockIdx.y) * 16 * RT;
  if (row0 >= n * G) return;

  Rows<RT> rows;
  find_rows<RT, BIAS>(pd, a, b, g, n, row0, rows);
  float qf[RT][4 * NI];
  const float scale2 = a.scale * kLog2e;
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const float *qp = static_cast<const float *>(a.q_new) + (((int64_t)b * a.max_nodes + rows.node[t]) * Hq + rows.head[t]) * D + 4 * q;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const f32x4 v = *reinterpret_cast<const f32x4 *>(qp + 16 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) qf[t][4 * i + e] = v[e] * scale2;
    }
  }
  const RespRows rr = resp_rows(a, b);
  if (blockIdx.y == 0 && blockIdx.z == 0) append_nodes<float, D>(pd, a, b, g, rr.write, n);
  build_key_table<float, D>(pd, a, b, g, rr.read, NewKeys{b * a.max_nodes, n, int64_t(Hkv) * D * 4}, BIAS, tab);
  const RangeSearch find(tab);
  const int n_total = tab.n_total, old = n_total - n;
  const int piece = ((n_total + d.n_pieces - 1) / d.n_pieces + 31) & ~31;
  const int key0 = min(int(blockIdx.z) * piece, n_total), key1 = min(key0 + piece, n_total);

  float m_run[RT], l_run[RT];
  f32x4 o[RT][NI];                   // o[t][4h + c][r]: dim 64h + 16 q + 4r + c of the lane's row
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    m_run[t] = kNegBig;
    l_run[t] = 0.f;
#pragma unroll
    for (int c = 0; c < NI; ++c) o[t][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  struct Stage {
    f32x4 k[NI], v[NH][4];
    float pos[4];
  };
  auto load = [&](int t0, Stage &st) {
    const int i0 = find.uniform(t0);
    const int c0 = __builtin_amdgcn_readfirstlane(tab.cum[i0]), c1 = __builtin_amdgcn_readfirstlane(tab.cum[i0 + 1]);
    const bool plain = t0 + 16 <= c1;
    const int64_t stride = uniform64(tab.stride[i0]);
    auto at = [&](int key, bool v) -> const char * {
      if (plain) return (v ? tab.v[i0] : tab.k[i0]) + int64_t(key - c0) * stride;
      const int vk = min(key, n_total - 1), i = find.from(i0, vk);
      return (v ? tab.v[i] : tab.k[i]) + int64_t(vk - tab.cum[i]) * tab.stride[i];
    };
    const char *kp = at(t0 + l16, false) + 16 * q;
#pragma unroll
    for (int i = 0; i < NI; ++i) st.k[i] = *global_ptr<f32x4>(kp + 64 * i);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const char *vp = at(t0 + 4 * q + r, true) + 16 * l16;
#pragma unroll
      for (int h = 0; h < NH; ++h) st.v[h][r] = *global_ptr<f32x4>(vp + 256 * h);
      if (BIAS) {
        const int vk = min(t0 + 4 * q + r, n_total - 1), i = find.from(i0, vk);
        st.pos[r] = global_ptr<float>(tab.pos[i])[vk - tab.cum[i]];
      }
    }
  };
  auto step = [&](int t0, Stage &st, auto masked) {
    constexpr bool MASKED = decltype(masked)::value;
    float p[RT][4];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      f32x4 s[NI];
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = x;
        x = __builtin_amdgcn_mfma_f32_16x16x4f32(st.k[i][0], qf[t][4 * i], x, 0, 0, 0);
        y = __builtin_amdgcn_mfma_f32_16x16x4f32(st.k[i][1], qf[t][4 * i + 1], y, 0, 0, 0);
        x = __builtin_amdgcn_mfma_f32_16x16x4f32(st.k[i][2], qf[t][4 * i + 2], x, 0, 0, 0);
        y = __builtin_amdgcn_mfma_f32_16x16x4f32(st.k[i][3], qf[t][4 * i + 3], y, 0, 0, 0);
        s[i] = x + y;
      }
#pragma unroll
      for (int w = NI / 2; w >= 1; w /= 2)
#pragma unroll
        for (int i = 0; i < w; ++i) s[i] += s[i + w];
      float mx = -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float x = s[0][i];
        if (BIAS) x += fmaf(rows.slope2[t], st.pos[i], rows.bias0[t]);
        if (MASKED) {
          const int at = t0 + 4 * q + i - old;
          if (at >= n || (at >= 0 && !(rows.mask[t] >> (at & 63) & 1))) x = -INFINITY;
        }
        p[t][i] = x;
        mx = fmaxf(mx, x);
      }
      if (__any(mx > m_run[t])) {
        const float m_new = fmaxf(m_run[t], rows_max(mx)), alpha = fast_exp2(m_run[t] - m_new);
        m_run[t] = m_new;
        l_run[t] *= alpha;
#pragma unroll
        for (int c = 0; c < NI; ++c) o[t][c] *= alpha;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[t][i] = fast_exp2(p[t][i] - m_run[t]);
        l_run[t] += p[t][i];
      }
    }
    if (MASKED) {
      bool bad = false;
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int e = 0; e < 4; ++e) bad |= not_finite(st.v[h][r][e]);
      if (__any(bad)) {                            // as in the bf16 kernel
        const int i0 = find.uniform(t0);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll 1
          for (int from = 0; from < 4; ++from) {
            const int vk = min(t0 + 4 * from + i, n_total - 1), r = find.from(i0, vk);
            const float *v = reinterpret_cast<const float *>(tab.v[r] + int64_t(vk - tab.cum[r]) * tab.stride[r]);
#pragma unroll
            for (int t = 0; t < RT; ++t) {
              const float w = __shfl(p[t][i], 16 * from + l16);
#pragma unroll
              for (int c = 0; c < NI; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const float x = v[64 * (c / 4) + 16 * q + 4 * e + c % 4];
                  if (not_finite(x) && w != 0.f) o[t][c][e] += w * x;
                }
            }
          }
#pragma unroll
        for (int h = 0; h < NH; ++h)
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (not_finite(st.v[h][r][e])) st.v[h][r][e] = 0.f;
      }
    }
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int r = 0; r < 4; ++r) x = __builtin_amdgcn_mfma_f32_16x16x4f32(st.v[h][r][c], p[t][r], x, 0, 0, 0);
          o[t][4 * h + c] += x;
        }
  };
  auto compute = [&](int t0, Stage &st) {
    if (t0 + 16 > old) step(t0, st, std::true_type{});
    else step(t0, st, std::false_type{});
  };
  for (int t0 = key0 + 16 * wave; t0 < key1; t0 += 16 * NW) {
    Stage st;
    load(t0, st);
    compute(t0, st);
  }
#pragma unroll
  for (int t = 0; t < RT; ++t) l_run[t] = rows_sum(l_run[t]);
  finish<float, D, RT, NW>(pd, d, b, rows, m_run, l_run, merge, [&](int t, auto &&fn) {
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        fn(64 * h + 16 * q + 4 * r, f32x4{o[t][4 * h][r], o[t][4 * h + 1][r], o[t][4 * h + 2][r], o[t][4 * h + 3][r]});
  });
}

// Adds up the pieces of a row in their order: a thread per four dims.
template <typename T, int D>
__global__ __launch_bounds__(256) void tree_merge_kernel(PlanDev pd, TreeDev d) {
  constexpr int PER = D / 4;
  const int64_t at = int64_t(blockIdx.x) * 256 + threadIdx.x, row = at / PER;
  if (row >= d.rows) return;
  const int dim = int(at % PER) * 4;
  if (d.a.n_nodes) {
    const int64_t node = row / pd.n_q_heads;
    if (node % d.a.max_nodes >= d.a.n_nodes[node / d.a.max_nodes]) return;
  }
  const float *ml = d.part + d.n_pieces * d.rows * D;
  float m = kNegBig, l = 0.f;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  for (int p = 0; p < d.n_pieces; ++p) {
    const int64_t i = p * d.rows + row;
    const float pm = ml[2 * i], pl = ml[2 * i + 1], m_new = fmaxf(m, pm), wa = fast_exp2(m - m_new), wb = fast_exp2(pm - m_new);
    const f32x4 x = *reinterpret_cast<const f32x4 *>(d.part + i * D + dim);
    l = l * wa + pl * wb;
    m = m_new;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = v[e] * wa + x[e] * wb;
  }
  store4<T, D>(d, row, dim, v, 1.f / l);
}

template <typename T, int D>
static hipError_t launch_tree(const sp_plan *plan, TreeDev &d, int64_t keys, hipStream_t s, bool *no_scratch) {
  constexpr bool kBf16 = sizeof(T) == 2;
  const int G = plan->n_q_heads / plan->n_kv_heads, rows = d.a.max_nodes * G, pairs = plan->n_prompts * plan->n_kv_heads;
  const int n_cu = plan->ctx->n_cu;
  int rt = rows <= 16 ? 1 : 2;
  int nw = 4;
  bool shared = kBf16 && rows > 64;
  const int block_rows = 16 * rt * (shared ? nw : 1);
  const int blocks = (rows + block_rows - 1) / block_rows;
  d.n_pieces = 1;
  const int64_t wgs = int64_t(pairs) * blocks;
  int64_t pieces = std::min<int64_t>((n_cu + wgs - 1) / wgs, keys / 256);
  pieces = std::min<int64_t>(pieces, int64_t(kTreePartBytes) / (d.rows * (D + 2) * 4));
  if (pieces > 1) {
    d.part = static_cast<float *>(tree_scratch(plan, s));
    if (!d.part) { *no_scratch = true; return hipSuccess; }
    d.n_pieces = int(pieces);
  }
  d.a.few_wgs = wgs * d.n_pieces <= int64_t(kDecFewWgsPerCu) * n_cu;
  const dim3 grid(static_cast<unsigned>(pairs), static_cast<unsigned>(blocks), static_cast<unsigned>(d.n_pieces)), block(64u * unsigned(nw));
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, plan->dev, d); };
  auto pick = [&](auto bias) {
    constexpr bool BIAS = decltype(bias)::value;
    if constexpr (kBf16) {
      if (shared) go(tree_bf16_kernel<D, 2, 4, true, BIAS>);
      else if (rt == 1) go(tree_bf16_kernel<D, 1, 4, false, BIAS>);
      else go(tree_bf16_kernel<D, 2, 4, false, BIAS>);
    } else {
      if (rt == 1) go(tree_f32_kernel<D, 1, 4, BIAS>);
      else go(tree_f32_kernel<D, 2, 4, BIAS>);
    }
  };
  if (plan->has_slopes) pick(std::true_type{}); else pick(std::false_type{});
  if (d.n_pieces > 1)
    hipLaunchKernelGGL((tree_merge_kernel<T, D>), dim3(unsigned((d.rows * (D / 4) + 255) / 256)), dim3(256), 0, s, plan->dev, d);
  return hipGetLastError();
}

hipError_t launch_tree_decode(const sp_plan *plan, const TreeArgs &a, hipStream_t s, bool *no_scratch) {
  TreeDev d{a, 1, nullptr, int64_t(plan->n_prompts) * a.max_nodes * plan->n_q_heads};
  const int64_t resp = int64_t(a.resp_len_add) + (a.resp_len ? a.resp_capacity / 2 : 0);
  const int64_t keys = plan->max_shared_keys + int64_t(a.k) * plan->max_path_keys + std::min<int64_t>(resp, a.resp_capacity);
  *no_scratch = false;
  if (plan->dtype == SP_BF16)
    return plan->head_dim == 128 ? launch_tree<__bf16, 128>(plan, d, keys, s, no_scratch) : launch_tree<__bf16, 64>(plan, d, keys, s, no_scratch);
  return plan->head_dim == 128 ? launch_tree<float, 128>(plan, d, keys, s, no_scratch) : launch_tree<float, 64>(plan, d, keys, s, no_scratch);
}

}  // namespace sp
