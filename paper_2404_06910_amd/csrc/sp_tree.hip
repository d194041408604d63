// a5: attention of a tree of drafted tokens over the joined cache.
//
// Node i sees the joined cache and the response cache completely, and of the tree itself and its ancestors.  The nodes' rows
// of all query heads that share a KV head are the rows of one small product with that head's keys: row node * G + head.  The keys are the
// list of build_key_table, the nodes last, so that only its last steps know a mask: one bit mask of 64 nodes per row.
//
// A wave walks the keys 32 (fp32: 16) at a time for RT tiles of 16 rows, with a running maximum and sum per row.  The waves of a
// workgroup either take different keys (few rows: nothing is shared, each wave streams through two LDS slots of its own and waits for
// nobody, their sums are added up at the end) or different rows (many rows: K and V are staged once for all of them).
// Where that leaves most of the chip idle, the key list is cut into pieces too, one workgroup each, and the workgroup that
// finishes last adds the pieces up in their order.
//
// Measured, us for one layer (bytes that have to move at a large copy's 5.1 TB/s: floor), bf16 unless said:
//   64 prompts of 32 heads, 16 nodes, 2 kept paths     121.5 (floor 125): HBM, 5.2 TB/s
//   16 prompts of 32/8 heads, 64 nodes, 950 keys        38.3 (17): 2048 rows to 256 workgroups, the steps' barriers and issue of products and exponents
//   2 prompts of 32/4 heads of 64 dims, 33 nodes, up to 12000 keys   27.9 (3.6): a piece's chain of steps
//   6 prompts of 32/8 heads, 12 nodes, 890 keys, fp32 with positions 31.2 (8.8): fp32 matrix pipe, a piece's chain
//   one prompt of 32 heads, 5 nodes                     11.1 (1.4): latencies (launch, tables, K and V, merge)
#include <algorithm>
#include <type_traits>

#include "sp_key_table.h"
#include "sp_lds_dma.h"

namespace sp {

namespace {

typedef __attribute__((ext_vector_type(2))) unsigned long long u64x2;

struct TreeDev {
  TreeArgs a;
  int32_t n_pieces;
  float *part;               // n_pieces > 1: [piece][prompt, node, query head][D] sums, then {max, sum} for each
  int64_t rows;              // prompts * nodes * query heads
  uint32_t *count;           // and an arrival counter per (prompt, KV head, block of rows), zero between launches
};

// The parent of lane i's node as the table has it (the request leaves early, the mask is built when K and V are on their way).
__device__ __forceinline__ int load_parent(const TreeArgs &a, int b) {
  const int i = threadIdx.x & 63;
  return a.parent && i < a.max_nodes ? a.parent[(int64_t)b * a.max_nodes + i] : i - 1;
}
// Bit j of lane i's mask: node j is node i or an ancestor of it.  Six doublings reach all of 64 nodes, since parents come first.
__device__ __forceinline__ uint64_t ancestor_mask(int up, int n) {
  const int i = threadIdx.x & 63;
  if (i >= n || up < 0 || up >= i) up = -1;
  uint32_t lo = i < 32 ? 1u << i : 0u, hi = i >= 32 ? 1u << (i - 32) : 0u;
  for (int r = 1; r < n; r *= 2) {
    const int from = up < 0 ? i : up;
    const uint32_t l = __shfl(lo, from), h = __shfl(hi, from);
    const int u = __shfl(up, from);
    lo |= l;
    hi |= h;
    up = up < 0 ? -1 : u;
  }
  return uint64_t(hi) << 32 | lo;
}

// the nodes' K and V (and positions) to the response cache: workgroups of their own, one per (prompt, KV head), beside the others
template <typename T, int D>
__device__ __forceinline__ void append_nodes(const PlanDev &pd, const TreeArgs &a, int b, int g, int row0, int n) {
  constexpr int EV = Elem<T>::kVec, LPK = D / EV;
  const int Hkv = pd.n_kv_heads;
  if (row0 < 0 || row0 >= a.resp_capacity) return;           // before any sum: row0 + node passes 31 bits for the largest lengths
  n = min(n, a.resp_capacity - row0);
  for (int i = threadIdx.x; i < n * LPK; i += blockDim.x) {
    const int node = i / LPK, sub = i % LPK, row = row0 + node;
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
  int32_t node[RT], head[RT];        // rows past max_nodes repeat the last one
  bool real[RT];
  uint64_t mask[RT];                 // nodes that the row sees
  float slope2[RT], bias0[RT];       // with a distance penalty: slope * log2 e, and that times minus the row's position
};
template <int RT, bool BIAS>
__device__ __forceinline__ void find_rows(const PlanDev &pd, const TreeArgs &a, int b, int g, int row0, Rows<RT> &r) {
  const int G = pd.n_q_heads / pd.n_kv_heads, l16 = threadIdx.x & 15;
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int row = min(row0 + 16 * t + l16, a.max_nodes * G - 1);
    r.node[t] = row / G;
    r.head[t] = g * G + row % G;
    r.slope2[t] = BIAS ? pd.slopes[r.head[t]] * kLog2e : 0.f;
    r.bias0[t] = BIAS ? -r.slope2[t] * a.new_pos[(int64_t)b * a.max_nodes + r.node[t]] : 0.f;
  }
}
template <int RT>
__device__ __forceinline__ void find_masks(const PlanDev &pd, int n, int up, int row0, Rows<RT> &r) {
  const int G = pd.n_q_heads / pd.n_kv_heads, l16 = threadIdx.x & 15;
  const uint64_t all = ancestor_mask(up, n);
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    r.real[t] = row0 + 16 * t + l16 < n * G;
    r.mask[t] = uint64_t(__shfl(uint32_t(all >> 32), r.node[t])) << 32 | __shfl(uint32_t(all), r.node[t]);
  }
}

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

// Four floats that other workgroups write or read: agent-scope accesses go past the L2 that is not theirs (a fence would write
// back and invalidate all of it).
__device__ __forceinline__ void store_shared(float *p, f32x4 v) {
  const auto w = __builtin_bit_cast(u64x2, v);
  __hip_atomic_store(reinterpret_cast<unsigned long long *>(p), w[0], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __hip_atomic_store(reinterpret_cast<unsigned long long *>(p) + 1, w[1], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x4 load_shared(const float *p) {
  u64x2 w;
  w[0] = __hip_atomic_load(reinterpret_cast<const unsigned long long *>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  w[1] = __hip_atomic_load(reinterpret_cast<const unsigned long long *>(p) + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return __builtin_bit_cast(f32x4, w);
}

// Ends a workgroup.  Every wave has m, l (complete, the same in a row's four lanes) and the weighted sums of its rows, NV vectors of
// four dims of which the i-th begins at dim(i).  The KS groups of waves that took different keys are added up in LDS, in their order, by the
// first group; pieces, if there are several, by the workgroup that arrives last, in theirs.
template <typename T, int D, int RT, int RW, int KS, class Dim>
__device__ __forceinline__ void finish(const PlanDev &pd, const TreeDev &d, int b, int g, int n, const Rows<RT> &r, float *m, float *l,
                                       f32x4 (*o)[D / 16], float *lds, Dim &&dim) {
  constexpr int PITCH = D + 4, NV = D / 16;          // 16 rows' vectors fall into different banks
  const int lane = threadIdx.x & 63, l16 = lane & 15, wave = threadIdx.x >> 6, rw = wave % RW, ks = wave / RW;
  if constexpr (KS > 1) {
    __shared__ float s_ml[KS - 1][RW][2][16 * RT];
    __syncthreads();                                 // all waves are done with their slots
    if (ks > 0) {
#pragma unroll
      for (int t = 0; t < RT; ++t) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
          *reinterpret_cast<f32x4 *>(lds + ((((ks - 1) * RW + rw) * RT + t) * 16 + l16) * PITCH + dim(i)) = o[t][i];
        if (lane < 16) { s_ml[ks - 1][rw][0][16 * t + lane] = m[t]; s_ml[ks - 1][rw][1][16 * t + lane] = l[t]; }
      }
    }
    __syncthreads();
    if (ks == 0) {
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int k = 0; k < KS - 1; ++k) {
          const float pm = s_ml[k][rw][0][16 * t + l16], m_new = fmaxf(m[t], pm), wa = fast_exp2(m[t] - m_new), wb = fast_exp2(pm - m_new);
          l[t] = l[t] * wa + s_ml[k][rw][1][16 * t + l16] * wb;
          m[t] = m_new;
#pragma unroll
          for (int i = 0; i < NV; ++i) {
            const f32x4 x = *reinterpret_cast<const f32x4 *>(lds + (((k * RW + rw) * RT + t) * 16 + l16) * PITCH + dim(i));
#pragma unroll
            for (int e = 0; e < 4; ++e) o[t][i][e] = o[t][i][e] * wa + x[e] * wb;
          }
        }
    }
  }
  const int64_t base = (int64_t)b * d.a.max_nodes * pd.n_q_heads;
  float *const part_ml = d.part + d.n_pieces * d.rows * D;
  if (ks == 0) {
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      if (!r.real[t]) continue;
      const int64_t row = base + (int64_t)r.node[t] * pd.n_q_heads + r.head[t];
      if (d.n_pieces == 1) {
        const float inv = 1.f / l[t];
#pragma unroll
        for (int i = 0; i < NV; ++i) store4<T, D>(d, row, dim(i), o[t][i], inv);
      } else {
        const int64_t at = int64_t(blockIdx.z) * d.rows + row;
#pragma unroll
        for (int i = 0; i < NV; ++i) store_shared(d.part + at * D + dim(i), o[t][i]);
        if (lane < 16) {
          const uint64_t w = uint64_t(__float_as_uint(l[t])) << 32 | __float_as_uint(m[t]);
          __hip_atomic_store(reinterpret_cast<unsigned long long *>(part_ml + 2 * at), w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
      }
    }
  }
  if (d.n_pieces == 1) return;
  __shared__ int s_last;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // this wave's stores have been performed
  __syncthreads();
  if (threadIdx.x == 0) {
    uint32_t *ctr = d.count + blockIdx.x + gridDim.x * blockIdx.y;
    s_last = __hip_atomic_fetch_add(ctr, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == uint32_t(d.n_pieces - 1);
    if (s_last) __hip_atomic_store(ctr, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (!s_last) return;
  // a thread per row and four dims
  constexpr int PER = D / 4;
  const int G = pd.n_q_heads / pd.n_kv_heads, row0 = int(blockIdx.y) * RW * RT * 16, rows = min(RW * RT * 16, n * G - row0);
  constexpr int NT = 64 * RW * KS;
  auto merge = [&](auto items) {                     // as many of a thread's at once, with four pieces' loads each
    constexpr int U = decltype(items)::value;
    for (int i0 = threadIdx.x; i0 < rows * PER; i0 += U * NT) {
      int64_t row[U];
      int at_dim[U];
      float mm[U], ll[U];
      f32x4 v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = min(i0 + u * NT, rows * PER - 1), rr = row0 + i / PER;
        at_dim[u] = i % PER * 4;
        row[u] = base + int64_t(rr / G) * pd.n_q_heads + g * G + rr % G;
        mm[u] = kNegBig;
        ll[u] = 0.f;
        v[u] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
      for (int p0 = 0; p0 < d.n_pieces; p0 += 4) {
        f32x4 x[U][4];
        uint64_t w[U][4];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int64_t at = min(p0 + j, d.n_pieces - 1) * d.rows + row[u];
            x[u][j] = load_shared(d.part + at * D + at_dim[u]);
            w[u][j] = __hip_atomic_load(reinterpret_cast<unsigned long long *>(part_ml + 2 * at), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (p0 + j >= d.n_pieces) break;
            const float pm = __uint_as_float(uint32_t(w[u][j])), pl = __uint_as_float(uint32_t(w[u][j] >> 32));
            const float m_new = fmaxf(mm[u], pm), wa = fast_exp2(mm[u] - m_new), wb = fast_exp2(pm - m_new);
            ll[u] = ll[u] * wa + pl * wb;
            mm[u] = m_new;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[u][e] = v[u][e] * wa + x[u][j][e] * wb;
          }
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i0 + u * NT < rows * PER) store4<T, D>(d, row[u], at_dim[u], v[u], 1.f / ll[u]);
    }  };
    if (rows * PER <= NT) merge(std::integral_constant<int, 1>{});
    else merge(std::integral_constant<int, 2>{});
  }

// bf16: what the second product sums is the weights times this.  The upper half of a weight (its bits cut off) leaves less than 2^-7 of it; with the
// factor the rest is never zero either (2^-10 of the weight at least), so that an infinite V that a row sees stays infinite: zero times
// infinity is NaN.  The sum of the weights is multiplied by the same factor at the end.
constexpr float kWeightScale = 1.f + 0x1p-10f;

__device__ __forceinline__ bool not_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }

}  // namespace

// A step is 32 keys in bf16 (two tiles of 16), 16 in fp32.
// bf16, v_mfma_f32_16x16x32_bf16:
//   S^T[key, row]  = K[key, :] . Q[row, :]         A = K (LDS), B = Q (registers)
//   O^T[d, row]   += V^T[d, key] . P^T[key, row]   A = V (LDS, transpose reads), B = P as it is
// In the accumulator lane L holds row L % 16 and keys 4 (L / 16) + i of each tile, which are bound to the k-slots that the lane feeds in
// the second product.  A weight goes into it as two bf16 numbers, its upper half and what that leaves (kWeightScale), so that it is off by at most
// 2^-15 of itself, and the result by little more than its one rounding (1.7e-3 of the outputs' norm from 64 bits, as the rounding alone; with weights of
// one bf16 number 2.3e-3).  The product more costs nothing where HBM bounds a launch (64 prompts 121.6 / 121.7 us), and 33.5 / 38.3 and 25.4 / 27.9
// in the two cases above where issue does.
// fp32, v_mfma_f32_16x16x4_f32, everything in 32 bits:
//   S^T[key, row] = K[key, :] . Q[row, :]       slots bound to dims 16 i + 4 (L / 16) + e
//   O^T[d, row]  += V^T[d, key] . P^T[key, row] slot L / 16 of product r bound to key 4 (L / 16) + r; rows of O^T to dims 64 h + 4 (L % 16) + c
// Sums are kept in short chains that are added up (a single chain of D products rounds several times as much).
// RW waves take different rows and fill each stage together; KS such groups take every KS-th step and have slots of their own.
template <typename T, int D, int RT, int RW, int KS, int NS, bool BIAS>
__global__ __launch_bounds__(64 * RW * KS, 2) void tree_kernel(PlanDev pd, TreeDev d) {
  constexpr bool kBf16 = sizeof(T) == 2;
  constexpr int STEP = kBf16 ? 32 : 16;
  constexpr int ROWB = D * int(sizeof(T)), CPR = ROWB / 16, RG = 64 / CPR;    // LDS row, its 16-byte chunks, rows per DMA
  constexpr int RPC = ROWB < 256 ? 256 / ROWB : 1;                            // rows per 256 bytes (all banks)
  constexpr int HALFB = STEP * ROWB, SLOTB = 2 * HALFB;
  constexpr int NI = STEP / RG;                  // DMA instructions per half
  // Keys that one workgroup reads (bf16; fp32 up to 16 rows) are not kept in the caches.  fp32 has up to four blocks of 16 rows to a key, and they gain
  // from the hint all the same, or lose nothing.  us with / without it: 64 prompts of 32/8 heads, 16 rows 96 / 106; 32 prompts, 32 rows 90 / 96, 64 rows
  // 140 / 139; 6 prompts, 48 rows 32.0 / 31.8.
  constexpr bool STREAM = RW == 1;
  constexpr int RINGB = NS * SLOTB * KS;
  constexpr int MERGEB = (KS - 1) * RW * RT * 16 * (D + 4) * 4;
  constexpr int NQ = CPR / 4, NC = D / 16;       // 16-byte vectors of a row per lane; output vectors
  __shared__ __attribute__((aligned(1024))) unsigned char ring[RINGB > MERGEB ? RINGB : MERGEB];
  __shared__ __attribute__((aligned(256))) float s_pos[BIAS ? NS * KS : 1][64];
  __shared__ KeyTable tab;
  const TreeArgs &a = d.a;
  const int Hq = pd.n_q_heads, Hkv = pd.n_kv_heads, G = Hq / Hkv;
  const int b = blockIdx.x / Hkv, g = blockIdx.x % Hkv;
  const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rw = wave % RW, ks = wave / RW;
  const RespRows rr = resp_rows(a, b);
  const int n = a.n_nodes ? min(max(a.n_nodes[b], 0), a.max_nodes) : a.max_nodes;
  if (blockIdx.y == gridDim.y - 1) {
    if (blockIdx.z == 0) append_nodes<T, D>(pd, a, b, g, rr.write, n);
    return;
  }
  const int row0 = (int(blockIdx.y) * RW + rw) * 16 * RT;

  Rows<RT> rows;
  find_rows<RT, BIAS>(pd, a, b, g, row0, rows);
  const int up = load_parent(a, b);
  u32x4 qf[RT][NQ];
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int j = 0; j < NQ; ++j)
      qf[t][j] = ld16(static_cast<const T *>(a.q_new) + (((int64_t)b * a.max_nodes + rows.node[t]) * Hq + rows.head[t]) * D +
                      (q + 4 * j) * (16 / int(sizeof(T))));
  const float scale2 = a.scale * kLog2e;
  if (int(blockIdx.y) * RW * 16 * RT >= n * G) return;
  build_key_table<T, D>(pd, a, b, g, rr.read, NewKeys{b * a.max_nodes, n, int64_t(Hkv) * ROWB}, BIAS, tab);
  const RangeSearch find(tab);
  // The compiler waits for a load of its own at the first use, which would be in the loop, with all the DMA in flight there.
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int j = 0; j < NQ; ++j) asm volatile("" : "+v"(qf[t][j]));
  int up_here = up;
  asm volatile("" : "+v"(up_here));
  const int n_total = tab.n_total, old = n_total - n;
  // pieces are multiples of a step, so that only steps at the end of the list reach beyond it
  const int piece = ((n_total + d.n_pieces - 1) / d.n_pieces + STEP - 1) & ~(STEP - 1);
  const int key0 = min(int(blockIdx.z) * piece, n_total), key1 = min(key0 + piece, n_total);
  const int n_steps = (key1 - key0 + STEP - 1) / STEP;

  // LDS rows are unpadded; the 16-byte chunks of a row are swizzled on the global side, so that row reads of K (16 rows, one
  // chunk) and, in bf16, transpose reads of V (8 rows of one chunk pair at a time) spread over the banks.
  auto fK = [](int row) { return (row / RPC) % (CPR < 16 ? CPR : 16); };
  auto fV = [](int row) { return kBf16 ? ((row / RPC) % (CPR / 4)) * 4 | ((row >> 2) & 1) * 2 : 0; };
  const uint32_t ring_base = (uint32_t)(size_t)(lds_byte *)ring + ks * NS * SLOTB;
  const uint32_t pos_base = (uint32_t)(size_t)(lds_byte *)&s_pos[0][0] + ks * NS * 256;
  const unsigned char *ringp = ring + ks * NS * SLOTB;
  const int drow = lane / CPR, dslot = lane % CPR;
  static_assert(2 * NI % RW == 0, "the waves of a group share a stage evenly");
  constexpr int MINE = 2 * NI / RW;              // DMA instructions of a wave per stage

  // the range that the last stage began in, wave-uniform: looking it up takes longer than the requests
  int c0 = 0, c1 = 0, i0 = 0;
  int64_t stride = 0;
  const char *k0 = nullptr, *v0 = nullptr;
  auto issue = [&](int s, int slot) {
    const int t0 = key0 + STEP * s;
    const uint32_t lds = ring_base + slot * SLOTB;
    if (t0 >= c1) {
      i0 = find.uniform(t0);
      c0 = __builtin_amdgcn_readfirstlane(tab.cum[i0]);
      c1 = __builtin_amdgcn_readfirstlane(tab.cum[i0 + 1]);
      stride = uniform64(tab.stride[i0]);
      k0 = reinterpret_cast<const char *>(uniform64(reinterpret_cast<int64_t>(tab.k[i0])));
      v0 = reinterpret_cast<const char *>(uniform64(reinterpret_cast<int64_t>(tab.v[i0])));
    }
    // rows RG m .. of the half: consecutive tokens of one range, or each row looked up by itself (past the end: the last key again)
    const bool plain = t0 + STEP <= c1 && stride < (int64_t(1) << 27);
    const char *kb = k0 + (t0 - c0) * stride, *vb = v0 + (t0 - c0) * stride;
    const uint32_t row_off = uint32_t(drow) * uint32_t(stride);
    if (plain) {
#pragma unroll
      for (int x = 0; x < MINE; ++x) {
        const int m2 = rw + x * RW;
        const bool is_v = m2 >= NI;
        const int m = is_v ? m2 - NI : m2, row = RG * m + drow;
        const uint32_t chunk = uint32_t(dslot ^ (is_v ? fV(row) : fK(row))) * 16;
        dma16s<STREAM>((is_v ? vb : kb) + RG * m * stride, row_off + chunk, lds + (is_v ? HALFB : 0) + m * (RG * ROWB));
      }
    } else {
#pragma unroll
      for (int x = 0; x < MINE; ++x) {
        const int m2 = rw + x * RW;
        const bool is_v = m2 >= NI;
        const int m = is_v ? m2 - NI : m2, row = RG * m + drow;
        const uint32_t chunk = uint32_t(dslot ^ (is_v ? fV(row) : fK(row))) * 16;
        const int vk = min(t0 + row, n_total - 1), i = find.from(i0, vk);
        dma16((is_v ? tab.v[i] : tab.k[i]) + int64_t(vk - tab.cum[i]) * tab.stride[i] + chunk, lds + (is_v ? HALFB : 0) + m * (RG * ROWB));
      }
    }
    if (BIAS && rw == 0) {
      const int vk = min(t0 + (lane & (STEP - 1)), n_total - 1), i = find.from(i0, vk);
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

  // bit k: the row of tile t sees key t0 + k (all keys before the nodes)
  auto seen = [&](int t, int t0) {
    const int at = t0 - old;
    return at >= 0 ? uint32_t(rows.mask[t] >> at) : uint32_t(rows.mask[t]) << -at | ((1u << -at) - 1);
  };
  // An infinite V, or NaN, must not reach rows that do not see its key (0 times infinity is NaN).  Steps with nodes look for such
  // elements, take them out of the product and add them key by key where the weight is not zero: weight(t, i) is that of key
  // 4 (L / 16) + i of the keys from t0 on, dim(c, e) the place of o[t][c][e].
  auto add_infinite = [&](int t0, auto &&weight, auto &&dim) {
    if (t0 >= n_total) return;                       // half a step behind the list (bf16): no key, and no weight but zero
    const int i0 = find.uniform(t0);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll 1
      for (int from = 0; from < 4; ++from) {
        const int vk = min(t0 + 4 * from + i, n_total - 1), r = find.from(i0, vk);
        const char *v = tab.v[r] + int64_t(vk - tab.cum[r]) * tab.stride[r];
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          const float p = __shfl(weight(t, i), 16 * from + l16);
#pragma unroll
          for (int c = 0; c < NC; ++c) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float x = static_cast<float>(*global_ptr<T>(v + dim(c, e) * sizeof(T)));
              o[t][c][e] += not_finite(x) && p != 0.f ? p * x : 0.f;
            }
            __builtin_amdgcn_sched_barrier(0);       // few masks at a time: the loop around has no scalar registers to spare
          }
        }
      }
  };

  // one step on a slot
  auto compute_bf16 = [&](int step, int slot) {
    constexpr int NJ = D / 32;
    const int t0 = key0 + STEP * step;
    const bool masked = t0 + STEP > old;             // it holds nodes, or reaches beyond them
    const unsigned char *sl = ringp + slot * SLOTB;
    f32x4 s[RT][2];
#pragma unroll
    for (int t = 0; t < RT; ++t) s[t][0] = s[t][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int row = 16 * h + l16;
        const bf16x8 k = *reinterpret_cast<const bf16x8 *>(sl + row * ROWB + ((4 * j + q) ^ fK(row)) * 16);
#pragma unroll
        for (int t = 0; t < RT; ++t) s[t][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, __builtin_bit_cast(bf16x8, qf[t][j]), s[t][h], 0, 0, 0);
      }
    bf16x8 vf[NC];                                   // on its way under the softmax
    const unsigned char *vs = sl + HALFB + tr_sub8;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int r0 = 4 * q + tr_row;
      const unsigned char *vp = vs + r0 * ROWB + ((2 * c + tr_x) ^ fV(r0)) * 16;
      const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4 *)vp);
      const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4 *)(vp + 16 * ROWB));
      vf[c] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    if (BIAS) {
      const float *ps = &s_pos[NS * ks + slot][0];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const f32x4 kp = *reinterpret_cast<const f32x4 *>(ps + 16 * h + 4 * q);
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[t][h][i] = fmaf(s[t][h][i], scale2, fmaf(rows.slope2[t], kp[i], rows.bias0[t]));
      }
    }
    auto largest = [](const f32x4 (&x)[2]) {
      return fmaxf(fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[0][2], x[0][3])), fmaxf(fmaxf(x[1][0], x[1][1]), fmaxf(x[1][2], x[1][3])));
    };
    float mx[RT];
    if (!masked) {
#pragma unroll
      for (int t = 0; t < RT; ++t) mx[t] = largest(s[t]);
    } else {
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const uint32_t see = seen(t, t0) >> (4 * q);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[t][h][i] = see >> (16 * h + i) & 1 ? s[t][h][i] : -INFINITY;
        mx[t] = largest(s[t]);
      }
    }
    u32x4 pb[RT], pr[RT];                            // weights as pairs of bf16: upper halves, and the rest
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      if (!BIAS) mx[t] *= scale2;                    // scale2 > 0
      // The reference may lag behind the maximum by 8 (weights up to 256, which bf16 and the sums absorb): the lanes of a row need
      // not agree on a maximum in every step.
      if (__any(mx[t] > m_run[t] + 8.f)) {
        const float m_new = fmaxf(m_run[t], rows_max(mx[t])), alpha = fast_exp2(m_run[t] - m_new);
        m_run[t] = m_new;
        l_run[t] *= alpha;
#pragma unroll
        for (int c = 0; c < NC; ++c) o[t][c] *= alpha;
      }
      float ls[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = fast_exp2(BIAS ? s[t][h][i] - m_run[t] : fmaf(s[t][h][i], scale2, -m_run[t]));
        ls[h] = (p[0] + p[1]) + (p[2] + p[3]);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float a = p[2 * i], b = p[2 * i + 1];
          const uint32_t w = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
          pb[t][2 * h + i] = w;
          pr[t][2 * h + i] = __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(fmaf(a, kWeightScale, -bf16_lo(w))),
                                                                 static_cast<__bf16>(fmaf(b, kWeightScale, -bf16_hi(w)))});
        }
      }
      l_run[t] += ls[0] + ls[1];
    }
    if (masked) {
      uint32_t bad = 0;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const u32x4 w = __builtin_bit_cast(u32x4, vf[c]);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          bad |= uint32_t((w[e] & 0x7f80u) == 0x7f80u) | uint32_t((w[e] & 0x7f800000u) == 0x7f800000u);
      }
      if (__any(bad)) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
          add_infinite(t0 + 16 * h, [&](int t, int i) { return i & 1 ? bf16_hi(pb[t][2 * h + i / 2]) : bf16_lo(pb[t][2 * h + i / 2]); },
                       [&](int c, int e) { return 16 * c + 4 * q + e; });
#pragma unroll
        for (int c = 0; c < NC; ++c) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (not_finite(static_cast<float>(vf[c][e]))) vf[c][e] = static_cast<__bf16>(0.f);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int t = 0; t < RT; ++t) o[t][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[c], __builtin_bit_cast(bf16x8, pr[t]), o[t][c], 0, 0, 0);
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int t = 0; t < RT; ++t) o[t][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[c], __builtin_bit_cast(bf16x8, pb[t]), o[t][c], 0, 0, 0);
  };

  auto compute_f32 = [&](int step, int slot) {
    constexpr int NH = D / 64;
    const int t0 = key0 + STEP * step;
    const bool masked = t0 + STEP > old;
    const unsigned char *sl = ringp + slot * SLOTB;
    f32x4 s[RT];
    {
      f32x4 part[RT][NQ];
#pragma unroll
      for (int j0 = 0; j0 < NQ; j0 += 4) {           // eight chains side by side
        f32x4 k[4], z[RT][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) k[j] = *reinterpret_cast<const f32x4 *>(sl + l16 * ROWB + ((4 * (j0 + j) + q) ^ fK(l16)) * 16);
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int h = 0; h < 4; ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const f32x4 x = __builtin_bit_cast(f32x4, qf[t][j0 + j]), none = {0.f, 0.f, 0.f, 0.f};
              f32x4 &y = h & 1 ? z[t][j] : part[t][j0 + j];
              y = __builtin_amdgcn_mfma_f32_16x16x4f32(k[j][h], x[h], h < 2 ? none : y, 0, 0, 0);
            }
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int j = 0; j < 4; ++j) part[t][j0 + j] += z[t][j];
      }
#pragma unroll
      for (int t = 0; t < RT; ++t) {
#pragma unroll
        for (int w = NQ / 2; w >= 1; w /= 2)
#pragma unroll
          for (int j = 0; j < w; ++j) part[t][j] += part[t][j + w];
        s[t] = part[t][0];
      }
    }
    f32x4 vf[NH][4];                                 // [h][r]: dims 64h + 4 l16 + (0..3) of key 4q + r
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        vf[h][r] = *reinterpret_cast<const f32x4 *>(sl + HALFB + (4 * q + r) * ROWB + (16 * h + l16) * 16);
    f32x4 kp;
    if (BIAS) kp = *reinterpret_cast<const f32x4 *>(&s_pos[NS * ks + slot][4 * q]);
    float p[RT][4];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const uint32_t see = (masked ? seen(t, t0) : ~0u) >> (4 * q);
      float mx = -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = BIAS ? fmaf(s[t][i], scale2, fmaf(rows.slope2[t], kp[i], rows.bias0[t])) : s[t][i] * scale2;
        p[t][i] = see >> i & 1 ? x : -INFINITY;
        mx = fmaxf(mx, p[t][i]);
      }
      if (__any(mx > m_run[t])) {                    // the reference is the maximum itself (see the fp32 prefill)
        const float m_new = fmaxf(m_run[t], rows_max(mx)), alpha = fast_exp2(m_run[t] - m_new);
        m_run[t] = m_new;
        l_run[t] *= alpha;
#pragma unroll
        for (int c = 0; c < NC; ++c) o[t][c] *= alpha;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) p[t][i] = fast_exp2(p[t][i] - m_run[t]);
      l_run[t] += (p[t][0] + p[t][1]) + (p[t][2] + p[t][3]);
    }
    if (masked) {
      bool bad = false;
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int e = 0; e < 4; ++e) bad |= not_finite(vf[h][r][e]);
      if (__any(bad)) {
        add_infinite(t0, [&](int t, int i) { return p[t][i]; }, [&](int c, int e) { return 64 * (c / 4) + 16 * q + 4 * e + c % 4; });
#pragma unroll
        for (int h = 0; h < NH; ++h)
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (not_finite(vf[h][r][e])) vf[h][r][e] = 0.f;
      }
    }
    // o[t][4h + c][r]: dim 64h + 16 q + 4r + c of the lane's row
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int h = 0; h < NH; ++h) {
        f32x4 x[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) x[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int c = 0; c < 4; ++c) x[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[h][r][c], p[t][r], x[c], 0, 0, 0);
#pragma unroll
        for (int c = 0; c < 4; ++c) o[t][4 * h + c] += x[c];
      }
  };
  auto compute = [&](int step, int slot) {
    if constexpr (kBf16) compute_bf16(step, slot);
    else compute_f32(step, slot);
  };

  // RW waves: NS - 1 stages are on their way when a step begins; one wave: NS when it waits
  constexpr int AHEAD = RW > 1 ? NS - 1 : NS;
#pragma unroll
  for (int i = 0; i < AHEAD; ++i)
    if (ks + i * KS < n_steps) issue(ks + i * KS, i);
  find_masks(pd, n, up_here, row0, rows);
  // the stages behind the one that is waited for: what the wave that also fetches positions has in flight is more, never less
  constexpr int LATER = (AHEAD - 1) * (RW > 1 ? MINE : MINE + (BIAS ? 1 : 0));
  int slot = 0;
  for (int s0 = 0; s0 < n_steps; s0 += KS) {
    const int s = s0 + ks;
    if (s + (AHEAD - 1) * KS < n_steps) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LATER) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if constexpr (RW > 1) {
      __syncthreads();                             // this stage is there, and nobody reads the slot of the one before any more
      if (s + AHEAD * KS < n_steps) issue(s + AHEAD * KS, slot == 0 ? NS - 1 : slot - 1);
      if (s < n_steps && row0 < n * G) compute(s, slot);      // a wave without rows only fetches
    } else {
      if (s < n_steps) compute(s, slot);
      // the reads of this slot have returned before the next stage may overwrite it
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (s + AHEAD * KS < n_steps) issue(s + AHEAD * KS, slot);
    }
    slot = slot + 1 == NS ? 0 : slot + 1;
  }
#pragma unroll
  for (int t = 0; t < RT; ++t) l_run[t] = rows_sum(l_run[t]) * (kBf16 ? kWeightScale : 1.f);
  if constexpr (kBf16) {
    finish<T, D, RT, RW, KS>(pd, d, b, g, n, rows, m_run, l_run, o, reinterpret_cast<float *>(ring), [&](int c) { return 16 * c + 4 * q; });
  } else {
    f32x4 ov[RT][NC];                // [4h + r]: four dims from 64h + 16 q + 4r on
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int h = 0; h < NC / 4; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) ov[t][4 * h + r] = f32x4{o[t][4 * h][r], o[t][4 * h + 1][r], o[t][4 * h + 2][r], o[t][4 * h + 3][r]};
    finish<T, D, RT, RW, KS>(pd, d, b, g, n, rows, m_run, l_run, ov, reinterpret_cast<float *>(ring),
                             [&](int i) { return 64 * (i / 4) + 16 * q + 4 * (i % 4); });
  }
}

// How a launch is shared out, a function of the call's sizes alone.  Measured, bf16, 128 dims (64 dims take half the LDS, and the same rule), us for
// one layer (~500 keys, 32 KV heads; 950 keys with 60 rows and more), by waves that take different keys / different rows:
//   up to 16 rows to a KV head, 6 / 8 / 10 / 16 / 20 / 32 prompts: 1 wave 30 / 29 / 32 / 36 / 43 / 58, 2 key groups
//     20 / 22 / 27 / 32 / 49 / 61, 4 key groups 19 / 21 / 33 / 39 / 51 / 73
//   60 rows, 4 / 8 / 16 / 32 prompts: 2 row waves 45 / 48 / 72 / 121, times 2 key groups 34 / 41 / 66 / 127, times 4 29 / 39 / 76 / 146
//   256 rows, 4 / 8 / 16 / 32 prompts of 8 KV heads: 2 row waves times 4 key groups 26 / 29 / 53 / 118, 4 times 2 31 / 35 / 39 / 82,
//     4 row waves 34 / 43 / 44 / 69
// Hence: as many key groups as leave a workgroup to every compute unit (their slots fill its LDS), none where there are more
// workgroups than that; four waves to share a stage once two would give more workgroups than compute units.
//   fp32, 48 pairs of 890 keys, up to 48 / 192 rows: 1 row wave times 4 key groups 45 / 125, in 2 pieces 33 / 139; 4 row waves 116 / 122,
//     in 5 pieces 52 / 79.  512 / 1024 pairs, up to 16 rows: 1 wave 128 / 168, 2 key groups 83 / 166, 4 87 / 177
// The key table takes a thread per kept path and one for the shared part: above 63 kept paths never a single wave.
// Lists are cut into pieces, of at least a step for every key group, where that leaves compute units without a workgroup (fp32
// with four row waves, of which three workgroups are resident: without three).
struct TreeShape {
  int rt, rw, ks, blocks, pieces;
};
static TreeShape tree_shape(const sp_plan *plan, int max_nodes, int k, int64_t keys, int64_t part_rows, int n_cu) {
  const int G = plan->n_q_heads / plan->n_kv_heads, rows = max_nodes * G;
  const int64_t pairs = int64_t(plan->n_prompts) * plan->n_kv_heads;
  TreeShape t{rows <= 16 ? 1 : 2, 1, 1, 1, 1};
  auto wgs = [&]() {
    t.blocks = (rows + 16 * t.rt * t.rw - 1) / (16 * t.rt * t.rw);
    return pairs * t.blocks;
  };
  if (plan->dtype == SP_BF16) {
    if (rows > 32) t.rw = 2;
    if (rows > 64 && wgs() > n_cu) t.rw = 4;
    const int64_t n = wgs();
    if (n <= n_cu) t.ks = t.rw == 4 ? 2 : 4;
    else if (t.rw == 1 && (n <= 2 * n_cu || k > 63)) t.ks = 2;
  } else {
    t.rt = 1;
    if (rows > 64) t.rw = 4;
    else t.ks = wgs() <= 2 * n_cu ? 4 : 2;
  }
  const int64_t n = wgs();
  if (n <= kTreeCounters) {
    int64_t p = ((plan->dtype == SP_F32 && t.rw == 4 ? 3 : 1) * n_cu + n / 2) / n;
    p = std::min<int64_t>(p, (keys + 16 * t.ks) / (32 * t.ks));
    p = std::min<int64_t>(p, int64_t(kTreePartBytes) / (part_rows * (plan->head_dim + 2) * 4));
    t.pieces = int(std::max<int64_t>(p, 1));
  }
  return t;
}

template <typename T, int D>
static hipError_t launch_tree(const sp_plan *plan, TreeDev &d, const TreeShape &t, hipStream_t s) {
  const int64_t pairs = int64_t(plan->n_prompts) * plan->n_kv_heads;
  const dim3 grid(static_cast<unsigned>(pairs), unsigned(t.blocks) + 1, unsigned(t.pieces)), block(64u * unsigned(t.rw * t.ks));
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, plan->dev, d); };
  auto pick = [&](auto bias) {
    constexpr bool BIAS = decltype(bias)::value;
    if constexpr (sizeof(T) == 4) t.rw == 4 ? go(tree_kernel<T, D, 1, 4, 1, 3, BIAS>) : t.ks == 4 ? go(tree_kernel<T, D, 1, 1, 4, 2, BIAS>)
                                                                                                 : go(tree_kernel<T, D, 1, 1, 2, 2, BIAS>);
    else if (t.rw == 4) t.ks == 2 ? go(tree_kernel<T, D, 2, 4, 2, 4, BIAS>) : go(tree_kernel<T, D, 2, 4, 1, 3, BIAS>);
    else if (t.rw == 2) t.ks == 4 ? go(tree_kernel<T, D, 2, 2, 4, 2, BIAS>) : go(tree_kernel<T, D, 2, 2, 1, 2, BIAS>);
    else if (t.rt == 1) t.ks == 4 ? go(tree_kernel<T, D, 1, 1, 4, 2, BIAS>) : t.ks == 2 ? go(tree_kernel<T, D, 1, 1, 2, 2, BIAS>)
                                                                                          : go(tree_kernel<T, D, 1, 1, 1, 2, BIAS>);
    else t.ks == 4 ? go(tree_kernel<T, D, 2, 1, 4, 2, BIAS>) : t.ks == 2 ? go(tree_kernel<T, D, 2, 1, 2, 2, BIAS>)
                                                                           : go(tree_kernel<T, D, 2, 1, 1, 2, BIAS>);
  };
  if (plan->has_slopes) pick(std::true_type{}); else pick(std::false_type{});
  return hipGetLastError();
}

hipError_t launch_tree_decode(const sp_plan *plan, const TreeArgs &a, hipStream_t s, bool *no_scratch) {
  TreeDev d{a, 1, nullptr, int64_t(plan->n_prompts) * a.max_nodes * plan->n_q_heads, nullptr};
  const int64_t resp = int64_t(a.resp_len_add) + (a.resp_len ? a.resp_capacity / 2 : 0);
  const int64_t keys = plan->max_shared_keys + int64_t(a.k) * plan->max_path_keys + std::min<int64_t>(resp, a.resp_capacity);
  const int n_cu = plan->ctx->n_cu;
  const TreeShape t = tree_shape(plan, a.max_nodes, a.k, keys, d.rows, n_cu);
  *no_scratch = false;
  d.n_pieces = t.pieces;
  if (t.pieces > 1) {
    const DecodeRegion *region = tree_region(plan, s, size_t(t.pieces) * size_t(d.rows) * size_t(plan->head_dim + 2) * 4);
    if (!region) { *no_scratch = true; return hipSuccess; }
    d.part = static_cast<float *>(region->part);
    d.count = region->count;
  }
  d.a.few_wgs = int64_t(plan->n_prompts) * plan->n_kv_heads * t.blocks * t.pieces <= int64_t(kDecFewWgsPerCu) * n_cu;
  if (plan->dtype == SP_BF16)
    return plan->head_dim == 128 ? launch_tree<__bf16, 128>(plan, d, t, s) : launch_tree<__bf16, 64>(plan, d, t, s);
  return plan->head_dim == 128 ? launch_tree<float, 128>(plan, d, t, s) : launch_tree<float, 64>(plan, d, t, s);
}

}  // namespace sp
