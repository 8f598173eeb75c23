// Rotary positions on Q and K: in token order, and on the way of the group gather and its inverse.
//
// Pair j of the rotated channels turns by the angle p theta_j, p the position on the pair's axis:
// (x, y) -> amplitude (x cos - y sin, x sin + y cos).  Angles are kept in turns as 64-bit fixed point:
// theta / 2 pi as a fraction of 2^64 (made once, on the host), times the integer position, wraps modulo
// one turn exactly as the angle does, so the phase of any 32-bit position is good to 2^-32 turns with one
// integer product, without tables in memory and without fp64 on the device.  The sine and cosine take its upper
// 32 bits as an fp32 number of half turns between -1 and 1: at most 2^-26 turns more, near half a turn.
//
// HBM-bound: each thread forms the cosines and sines of its channels of a token once and applies them to
// all heads of its share, so the trigonometry is a few percent of the time of the row copies (40 heads of 126,360
// tokens, Q and K: 0.79 - 0.81 ms, 6.4 - 6.5 TB/s; the inverse gather of a top-2 routing of them: 1.78 ms,
// 6.5 TB/s).  With one head there is nothing to share it with: 600,000 tokens take 0.13 - 0.16 ms, 3.8 - 4.7 TB/s.
// Half layouts whose halves are not whole 16-byte vectors use narrower ones (88 of 128 channels, 60,000 tokens,
// 12 heads: 0.13 - 0.14 ms, 5.2 - 5.8 TB/s; 84 channels: 0.18 - 0.19 ms, 3.8 - 4.1 TB/s; odd halves by shuffles:
// 0.28 - 0.29 ms, 2.5 - 2.6 TB/s).

#include <math.h>

#include "block_common.cuh"

namespace moga {
namespace {

constexpr int kRopeThreads = 256;
constexpr int kMaxPairs = 64;

enum RopePath {
  PATH_INTERLEAVED = 0,   // pairs (2j, 2j+1): inside one 16-byte vector
  PATH_HALF = 1,          // pairs (j, j + rot/2): a thread takes both vectors of a pair of vectors, of 16, 8 or 4
                          // bytes, the widest of which rot/2 channels are a whole number
  PATH_HALF_ANY = 2       // bf16 with odd rot/2: partners come from the row's other lanes, by shuffles
};

struct RopeArgs {
  moga_rope_plan plan;
  const int32_t* pos;           // [N, axes] (pos_stride_b = 0) or [B, N, axes], or null
  long long pos_stride_b;
  int N, H, D;
  int heads_per_block;
  int slots;                    // threads of a row
  float sign;                   // -1: transpose
  // token-order side, in elements
  long long sb, sh, sn;
};

// Copies the plan's per-pair values where lanes can index them.
struct PairTable {
  uint64_t turns[kMaxPairs];
  int axis[kMaxPairs];
};
__device__ __forceinline__ void load_pairs(PairTable& t, const moga_rope_plan& p) {
  for (int j = threadIdx.x; j < kMaxPairs; j += blockDim.x) {
    t.turns[j] = j < p.pairs ? p.turns[j] : 0;
    t.axis[j] = j < p.axis_pairs[0] ? 0 : j < p.axis_pairs[0] + p.axis_pairs[1] ? 1 : 2;
  }
  __syncthreads();
}

__device__ __forceinline__ void token_position(const RopeArgs& a, int b, int n, long long (&at)[3]) {
  const moga_rope_plan& p = a.plan;
  if (a.pos != nullptr) {
    const int32_t* q = a.pos + b * a.pos_stride_b + (long long)n * p.n_axes;
    at[0] = __ldg(q);
    at[1] = p.n_axes > 1 ? __ldg(q + 1) : 0;
    at[2] = p.n_axes > 2 ? __ldg(q + 2) : 0;
  } else if (p.n_axes == 1) {
    at[0] = n;
    at[1] = at[2] = 0;
  } else {
    const int y = n / p.grid_w;
    const int x = n - y * p.grid_w;
    if (p.n_axes == 2) {
      at[0] = y, at[1] = x, at[2] = 0;
    } else {
      const int f = y / p.grid_h;
      at[0] = f, at[1] = y - f * p.grid_h, at[2] = x;
    }
  }
  at[0] += p.start[0];
  at[1] += p.start[1];
  at[2] += p.start[2];
}

__device__ __forceinline__ void pair_cos_sin(const RopeArgs& a, const PairTable& t, int j, const long long (&at)[3],
                                             float& c, float& s) {
  const int ax = t.axis[j];
  const long long p = ax == 0 ? at[0] : ax == 1 ? at[1] : at[2];
  const uint64_t phase = t.turns[j] * (uint64_t)p + (1ull << 31);     // turns * 2^64, rounded to 32 bits
  sincospif((float)(int32_t)(phase >> 32) * 0x1p-31f, &s, &c);        // half turns in [-1, 1]
  c *= a.plan.amplitude;
  s *= a.plan.amplitude * a.sign;
}

template <typename XT, typename VT, int E>
__device__ __forceinline__ void unpack_channels(const VT& r, float (&f)[E]) {
  const uint32_t* w = reinterpret_cast<const uint32_t*>(&r);
#pragma unroll
  for (int i = 0; i < (int)sizeof(VT) / 4; ++i) {
    if constexpr (sizeof(XT) == 2) f[2 * i] = __uint_as_float(w[i] << 16), f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    else f[i] = __uint_as_float(w[i]);
  }
}
template <typename XT, typename VT, int E>
__device__ __forceinline__ VT pack_channels(const float (&f)[E]) {
  VT r;
  uint32_t* w = reinterpret_cast<uint32_t*>(&r);
#pragma unroll
  for (int i = 0; i < (int)sizeof(VT) / 4; ++i) {
    if constexpr (sizeof(XT) == 2) {
      const __nv_bfloat162 t = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&t);
    } else {
      w[i] = __float_as_uint(f[i]);
    }
  }
  return r;
}

// OUT words from word `skip` (below N) on of the 2 N words that lanes s0 and s0 + 1 of the row hold in w; lane
// numbers are taken modulo width, the lanes of a row.  Every lane of the warp takes part.
template <int N, int OUT>
__device__ __forceinline__ void window(const uint32_t (&w)[N], int s0, int width, int skip, uint32_t (&out)[OUT]) {
  uint32_t t[2 * N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    t[i] = __shfl_sync(0xffffffffu, w[i], s0, width);
    t[N + i] = __shfl_sync(0xffffffffu, w[i], s0 + 1, width);
  }
#pragma unroll
  for (int step = N / 2; step > 0; step /= 2) {
    const bool on = skip & step;
#pragma unroll
    for (int i = 0; i + step < 2 * N; ++i) t[i] = on ? t[i + step] : t[i];
  }
#pragma unroll
  for (int i = 0; i < OUT; ++i) out[i] = t[i];
}

// The share of one thread in a row: which vectors it holds and their rotation.
//   INTERLEAVED: vector v, E / 2 pairs.      HALF: vectors v0 and v1 (partners), E pairs; or v0 alone, copied.
//   HALF_ANY: vector v, and the E partner channels.
template <typename XT, int PATH, typename VT>
struct Share {
  static constexpr int E = sizeof(VT) / sizeof(XT);
  static constexpr int NV = PATH == PATH_HALF ? 2 : 1;             // vectors held
  static constexpr int NP = PATH == PATH_INTERLEAVED ? E / 2 : E;  // rotations held
  int v[NV];
  bool rotated;           // HALF: both vectors belong to pairs
  int first;              // INTERLEAVED: its first pair; HALF_ANY: its first channel
  int from, skip;         // HALF_ANY: the partners start at channel `skip` of lane `from`'s vector
  float c[NP], s[NP];

  __device__ __forceinline__ void place(const RopeArgs& a, int slot) {
    const int pairs = a.plan.pairs;
    if constexpr (PATH == PATH_INTERLEAVED) {
      v[0] = slot;
      first = slot * (E / 2);
      rotated = first < pairs;
    } else if constexpr (PATH == PATH_HALF) {
      const int hv = pairs / E;
      rotated = slot < hv;
      v[0] = rotated ? slot : slot + hv;
      v[1] = rotated ? slot + hv : v[0];
    } else {
      v[0] = slot;
      first = slot * E;
      rotated = first < 2 * pairs;
      const bool lower = first < pairs;
      from = lower ? slot + pairs / E : slot - pairs / E - 1;
      skip = lower ? pairs % E : E - pairs % E;     // pairs is not a multiple of E here
    }
  }
  __device__ __forceinline__ void turn(const RopeArgs& a, const PairTable& t, int slot, const long long (&at)[3]) {
    const int pairs = a.plan.pairs;
    if constexpr (PATH == PATH_INTERLEAVED) {
#pragma unroll
      for (int i = 0; i < NP; ++i)
        if (first + i < pairs) pair_cos_sin(a, t, first + i, at, c[i], s[i]);
    } else if constexpr (PATH == PATH_HALF) {
      if (rotated) {
#pragma unroll
        for (int i = 0; i < NP; ++i) pair_cos_sin(a, t, slot * E + i, at, c[i], s[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int ch = first + i;
        if (ch < 2 * pairs) pair_cos_sin(a, t, ch < pairs ? ch : ch - pairs, at, c[i], s[i]);
      }
    }
  }

  // HALF_ANY: the partners y of this lane's channels, from the raw vectors of the row's lanes.  The one vector
  // that holds channels of both halves takes its upper ones' partners from the start of the row (lane 0).
  __device__ __forceinline__ void partners(const RopeArgs& a, const uint4& raw, float (&y)[E]) const {
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
    constexpr int PER = E / 4;                      // channels of a word
    const int pairs = a.plan.pairs, both_at = pairs % E;
    uint32_t t[5], z[5];
    window<4, 5>(w, from, a.slots, skip / PER, t);
    window<4, 5>(w, a.slots - 1, a.slots, (E - both_at) / PER, z);    // lanes slots - 1 and 0
    const bool mixed = first < pairs && first + E > pairs, odd = PER == 2 && (both_at & 1);
    uint4 r, s;
    if (odd) {
      r = make_uint4(__funnelshift_r(t[0], t[1], 16), __funnelshift_r(t[1], t[2], 16), __funnelshift_r(t[2], t[3], 16), __funnelshift_r(t[3], t[4], 16));
      s = make_uint4(__funnelshift_r(z[0], z[1], 16), __funnelshift_r(z[1], z[2], 16), __funnelshift_r(z[2], z[3], 16), __funnelshift_r(z[3], z[4], 16));
    } else {
      r = make_uint4(t[0], t[1], t[2], t[3]);
      s = make_uint4(z[0], z[1], z[2], z[3]);
    }
    unpack_channels<XT>(r, y);
    float up[E];
    unpack_channels<XT>(s, up);
#pragma unroll
    for (int i = 0; i < E; ++i) y[i] = mixed && i >= both_at ? up[i] : y[i];
  }
  // The same for values already summed in fp32.
  __device__ __forceinline__ void partners(const RopeArgs& a, const float (&x)[E], float (&y)[E]) const {
    const int pairs = a.plan.pairs, both_at = pairs % E;
    uint32_t w[E], t[E], z[E];
#pragma unroll
    for (int i = 0; i < E; ++i) w[i] = __float_as_uint(x[i]);
    window<E, E>(w, from, a.slots, skip, t);
    window<E, E>(w, a.slots - 1, a.slots, E - both_at, z);
    const bool mixed = first < pairs && first + E > pairs;
#pragma unroll
    for (int i = 0; i < E; ++i) y[i] = __uint_as_float(mixed && i >= both_at ? z[i] : t[i]);
  }

  // x: the held vectors as floats; y: HALF_ANY's partners.
  __device__ __forceinline__ void rotate(const RopeArgs& a, float (&x)[NV][E], const float (&y)[E]) const {
    if (!rotated) return;
    const int pairs = a.plan.pairs;
    if constexpr (PATH == PATH_INTERLEAVED) {
#pragma unroll
      for (int i = 0; i < NP; ++i)
        if (first + i < pairs) {
          const float u = x[0][2 * i], w = x[0][2 * i + 1];
          x[0][2 * i] = fmaf(u, c[i], -(w * s[i]));
          x[0][2 * i + 1] = fmaf(u, s[i], w * c[i]);
        }
    } else if constexpr (PATH == PATH_HALF) {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const float u = x[0][i], w = x[1][i];
        x[0][i] = fmaf(u, c[i], -(w * s[i]));
        x[1][i] = fmaf(u, s[i], w * c[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int ch = first + i;
        if (ch < pairs) x[0][i] = fmaf(x[0][i], c[i], -(y[i] * s[i]));
        else if (ch < 2 * pairs) x[0][i] = fmaf(y[i], s[i], x[0][i] * c[i]);
      }
    }
  }
};

// Q and K (and V, copied) of token order, rotated: to token order, in place or not, or,
// SORTED: to the k sorted rows inv[b, n, 0..k) of contiguous [B, H, N k, D] tensors.
// grid: (token tiles, head shares, B).  Each thread keeps its channels' rotation over its share of the heads and
// has the next head's rows on the way while it turns the present ones; the first rows are asked for before the
// sines are formed.  Rotating gather of 32,760 tokens, 12 heads, top-1: 98 us, 6.1 TB/s, of the 114 with its sort
// (without the next rows on the way 17 us more; with its natural 88 registers, two blocks to an SM, 2 us more).
// Five blocks to an SM for the interleaved layout in token order: 0.795 ms for the 40 heads, 0.809 with four.
struct RotateTensors {
  const void *Q, *K, *V;
  void *Qo, *Ko, *Vo;
  const int32_t* inv;
  int k;
};
template <typename XT, int PATH, typename VT, bool SORTED>
__global__ void __launch_bounds__(kRopeThreads, SORTED ? 3 : PATH == PATH_INTERLEAVED ? 5 : 0) rope_kernel(const __grid_constant__ RopeArgs a,
                                                            const __grid_constant__ RotateTensors t) {
  using S = Share<XT, PATH, VT>;
  constexpr int E = S::E, NV = S::NV;
  constexpr int NT = SORTED ? 3 : 2;
  __shared__ PairTable table;
  const int rows = kRopeThreads / a.slots;
  const int slot = threadIdx.x % a.slots, r = threadIdx.x / a.slots;
  const int b = blockIdx.z;
  const long long n_long = (long long)blockIdx.x * rows + r;
  const bool live = r < rows && n_long < a.N;
  const int n = live ? (int)n_long : 0;
  const long long src_row = (long long)b * a.sb + (long long)n * a.sn;
  const int h0 = blockIdx.y * a.heads_per_block, h1 = min(h0 + a.heads_per_block, a.H);
  const void* in[3] = {t.Q, t.K, t.V};
  void* out[3] = {t.Qo, t.Ko, t.Vo};
  S sh;
  sh.place(a, slot);
  VT next[NT][NV];
  auto load = [&](int h) {
#pragma unroll
    for (int q = 0; q < NT; ++q)
      if (live && in[q] != nullptr) {
        const XT* row = static_cast<const XT*>(in[q]) + src_row + (long long)h * a.sh;
#pragma unroll
        for (int i = 0; i < NV; ++i) next[q][i] = load_stream(reinterpret_cast<const VT*>(row) + sh.v[i]);
      }
  };
#pragma unroll
  for (int q = 0; q < NT; ++q)
#pragma unroll
    for (int i = 0; i < NV; ++i) next[q][i] = VT{};
  load(h0);
  load_pairs(table, a.plan);
  long long at[3];
  token_position(a, b, n, at);
  sh.turn(a, table, slot, at);
  for (int h = h0; h < h1; ++h) {
    VT raw[NT][NV];
#pragma unroll
    for (int q = 0; q < NT; ++q)
#pragma unroll
      for (int i = 0; i < NV; ++i) raw[q][i] = next[q][i];
    if (h + 1 < h1) load(h + 1);
#pragma unroll
    for (int q = 0; q < NT; ++q) {
      if (in[q] == nullptr) continue;               // the same for all threads
      if (q < 2) {
        float x[NV][E], y[E];
        if constexpr (PATH == PATH_HALF_ANY) sh.partners(a, raw[q][0], y);   // shuffles: every lane takes part
        if (sh.rotated) {
#pragma unroll
          for (int i = 0; i < NV; ++i) unpack_channels<XT>(raw[q][i], x[i]);
          sh.rotate(a, x, y);
#pragma unroll
          for (int i = 0; i < NV; ++i) {
            const VT keep = raw[q][i];
            raw[q][i] = pack_channels<XT, VT>(x[i]);
            // a vector that ends outside the rotated channels keeps those bits
            if constexpr (PATH != PATH_HALF) {
              const int inside = PATH == PATH_INTERLEAVED ? 2 * (a.plan.pairs - sh.first) : 2 * a.plan.pairs - sh.first;
              uint32_t* o = reinterpret_cast<uint32_t*>(&raw[q][i]);
              const uint32_t* kept = reinterpret_cast<const uint32_t*>(&keep);
#pragma unroll
              for (int w = 0; w < 4; ++w)
                if (w * (E / 4) >= inside) o[w] = kept[w];           // rot is even: whole words for bf16
            }
          }
        }
      }
      if (!live) continue;
      if constexpr (SORTED) {
        const long long T = (long long)a.N * t.k;
        const long long head = ((long long)b * a.H + h) * T;
        for (int j = 0; j < t.k; ++j) {
          const long long p = __ldg(t.inv + (long long)b * T + (long long)n * t.k + j);
          VT* dst = reinterpret_cast<VT*>(static_cast<XT*>(out[q]) + (head + p) * a.D);
#pragma unroll
          for (int i = 0; i < NV; ++i)
            if (i == 0 || sh.rotated) store_stream(dst + sh.v[i], raw[q][i]);
        }
      } else {
        VT* dst = reinterpret_cast<VT*>(static_cast<XT*>(out[q]) + src_row + (long long)h * a.sh);
#pragma unroll
        for (int i = 0; i < NV; ++i)
          if (i == 0 || sh.rotated) store_stream(dst + sh.v[i], raw[q][i]);
      }
    }
  }
}

// The inverse: dQ[n] = R^T sum_j dQp[inv[n, j]], dK the same, dV without the rotation; fp32 sums in slot
// order, one rounding.
struct UnrotateTensors {
  const void *in[3];
  void *out[3];
  const int32_t* inv;
  int k;
};
template <typename XT, int PATH, typename VT, int K>
__global__ void __launch_bounds__(kRopeThreads) rope_back_kernel(const __grid_constant__ RopeArgs a,
                                                                 const __grid_constant__ UnrotateTensors t) {
  using S = Share<XT, PATH, VT>;
  constexpr int E = S::E, NV = S::NV;
  __shared__ PairTable table;
  load_pairs(table, a.plan);
  const int rows = kRopeThreads / a.slots;
  const int slot = threadIdx.x % a.slots, r = threadIdx.x / a.slots;
  const int b = blockIdx.z;
  const long long n_long = (long long)blockIdx.x * rows + r;
  const bool live = r < rows && n_long < a.N;
  if (PATH != PATH_HALF_ANY && !live) return;       // HALF_ANY: lanes of a warp exchange partners
  const int n = live ? (int)n_long : 0;
  S sh;
  long long at[3];
  token_position(a, b, n, at);
  sh.place(a, slot);
  sh.turn(a, table, slot, at);
  const int k = K > 0 ? K : t.k;
  const long long T = (long long)a.N * k;
  const int32_t* iv = t.inv + (long long)b * T + (long long)n * k;
  constexpr int KK = K > 0 ? K : 1;
  long long p[KK];
#pragma unroll
  for (int j = 0; j < KK; ++j) p[j] = min(max((long long)__ldg(iv + j), 0ll), T - 1);   // a bad index reads a wrong row, never past the tensor
  const int h0 = blockIdx.y * a.heads_per_block, h1 = min(h0 + a.heads_per_block, a.H);
  const long long dst_row = (long long)b * a.sb + (long long)n * a.sn;
  for (int h = h0; h < h1; ++h) {
    const long long head = ((long long)b * a.H + h) * T;
    VT raw[3][KK][NV];
    float x[3][NV][E];
#pragma unroll
    for (int q = 0; q < 3; ++q)
#pragma unroll
      for (int j = 0; j < KK; ++j)
#pragma unroll
        for (int i = 0; i < NV; ++i)
          raw[q][j][i] = load_stream(reinterpret_cast<const VT*>(static_cast<const XT*>(t.in[q]) + (head + p[j]) * a.D) + sh.v[i]);
#pragma unroll
    for (int q = 0; q < 3; ++q) {
#pragma unroll
      for (int i = 0; i < NV; ++i) unpack_channels<XT>(raw[q][0][i], x[q][i]);
#pragma unroll
      for (int j = 1; j < KK; ++j) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          float f[E];
          unpack_channels<XT>(raw[q][j][i], f);
#pragma unroll
          for (int e = 0; e < E; ++e) x[q][i][e] += f[e];
        }
      }
      if constexpr (K == 0) {
        for (int j = 1; j < k; ++j) {
          const long long pj = min(max((long long)__ldg(iv + j), 0ll), T - 1);
#pragma unroll
          for (int i = 0; i < NV; ++i) {
            float f[E];
            unpack_channels<XT>(load_stream(reinterpret_cast<const VT*>(static_cast<const XT*>(t.in[q]) + (head + pj) * a.D) + sh.v[i]), f);
#pragma unroll
            for (int e = 0; e < E; ++e) x[q][i][e] += f[e];
          }
        }
      }
      if (q < 2) {
        float y[E];
        if constexpr (PATH == PATH_HALF_ANY) sh.partners(a, x[q][0], y);
        sh.rotate(a, x[q], y);
      }
      if (!live) continue;
      VT* dst = reinterpret_cast<VT*>(static_cast<XT*>(t.out[q]) + dst_row + (long long)h * a.sh);
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (i == 0 || sh.rotated) store_stream(dst + sh.v[i], pack_channels<XT, VT>(x[q][i]));
    }
  }
}

// The path and the bytes of its vectors.
struct RopeWay {
  int path, bytes;
};
RopeWay rope_way(const moga_shape& s, const moga_rope_plan& p) {
  if (p.layout == MOGA_ROPE_INTERLEAVED) return {PATH_INTERLEAVED, 16};
  for (int bytes = 16; bytes >= 4; bytes /= 2)
    if (p.pairs * (int)elem_size(s.dtype) % bytes == 0) return {PATH_HALF, bytes};
  return {PATH_HALF_ANY, 16};
}

// The common arguments and the grid: blocks of whole rows, heads split so that every SM has work.
RopeArgs rope_args(const moga_shape& s, const moga_rope_plan& p, const int32_t* pos, int pos_per_batch, bool transpose,
                   const RopeWay& way, int blocks_per_sm, dim3* grid) {
  RopeArgs a{};
  a.plan = p;
  a.pos = pos;
  a.pos_stride_b = pos_per_batch ? (long long)s.N * p.n_axes : 0;
  a.N = s.N;
  a.H = s.H;
  a.D = s.D;
  const int e = way.bytes / (int)elem_size(s.dtype);
  a.slots = way.path == PATH_HALF ? s.D / e - p.pairs / e : s.D / e;
  a.sign = transpose ? -1.f : 1.f;
  const Strides sd = qkv_strides(s);
  a.sb = sd.b;
  a.sh = sd.h;
  a.sn = sd.n;
  const int rows = kRopeThreads / a.slots;
  const long long tiles = (s.N + rows - 1) / rows;
  // at least so many blocks for each of the 148 SMs, as far as there are heads
  long long shares = (148ll * blocks_per_sm + tiles * s.B - 1) / (tiles * s.B);
  if (shares > s.H) shares = s.H;
  a.heads_per_block = (int)((s.H + shares - 1) / shares);
  *grid = dim3((unsigned)tiles, (s.H + a.heads_per_block - 1) / a.heads_per_block, s.B);
  return a;
}

template <typename XT, bool SORTED>
moga_status run_rope(const RopeArgs& a, const RotateTensors& t, const RopeWay& way, dim3 grid, cudaStream_t st) {
  if (way.path == PATH_INTERLEAVED) rope_kernel<XT, PATH_INTERLEAVED, uint4, SORTED><<<grid, kRopeThreads, 0, st>>>(a, t);
  else if (way.path == PATH_HALF && way.bytes == 16) rope_kernel<XT, PATH_HALF, uint4, SORTED><<<grid, kRopeThreads, 0, st>>>(a, t);
  else if (way.path == PATH_HALF && way.bytes == 8) rope_kernel<XT, PATH_HALF, uint2, SORTED><<<grid, kRopeThreads, 0, st>>>(a, t);
  else if (way.path == PATH_HALF) rope_kernel<XT, PATH_HALF, uint32_t, SORTED><<<grid, kRopeThreads, 0, st>>>(a, t);
  else if constexpr (sizeof(XT) == 2) rope_kernel<XT, PATH_HALF_ANY, uint4, SORTED><<<grid, kRopeThreads, 0, st>>>(a, t);
  MOGA_CUDA_OK(cudaGetLastError());
  return MOGA_OK;
}

template <typename XT, int PATH, typename VT>
void run_back(const RopeArgs& a, const UnrotateTensors& t, dim3 grid, cudaStream_t st) {
  if (t.k == 1) rope_back_kernel<XT, PATH, VT, 1><<<grid, kRopeThreads, 0, st>>>(a, t);
  else if (t.k == 2) rope_back_kernel<XT, PATH, VT, 2><<<grid, kRopeThreads, 0, st>>>(a, t);
  else rope_back_kernel<XT, PATH, VT, 0><<<grid, kRopeThreads, 0, st>>>(a, t);
}
template <typename XT>
moga_status run_back_path(const RopeArgs& a, const UnrotateTensors& t, const RopeWay& way, dim3 grid, cudaStream_t st) {
  if (way.path == PATH_INTERLEAVED) run_back<XT, PATH_INTERLEAVED, uint4>(a, t, grid, st);
  else if (way.path == PATH_HALF && way.bytes == 16) run_back<XT, PATH_HALF, uint4>(a, t, grid, st);
  else if (way.path == PATH_HALF && way.bytes == 8) run_back<XT, PATH_HALF, uint2>(a, t, grid, st);
  else if (way.path == PATH_HALF) run_back<XT, PATH_HALF, uint32_t>(a, t, grid, st);
  else if constexpr (sizeof(XT) == 2) run_back<XT, PATH_HALF_ANY, uint4>(a, t, grid, st);
  MOGA_CUDA_OK(cudaGetLastError());
  return MOGA_OK;
}

}  // namespace

moga_status launch_rope(const moga_shape& s, const moga_rope_plan& p, const int32_t* pos, int pos_per_batch,
                        const void* Q, const void* K, void* Qo, void* Ko, bool transpose, cudaStream_t st) {
  const RopeWay way = rope_way(s, p);
  dim3 grid;
  const RopeArgs a = rope_args(s, p, pos, pos_per_batch, transpose, way, 8, &grid);
  const RotateTensors t{Q, K, nullptr, Qo, Ko, nullptr, nullptr, 0};
  return s.dtype == MOGA_BF16 ? run_rope<__nv_bfloat16, false>(a, t, way, grid, st) : run_rope<float, false>(a, t, way, grid, st);
}

moga_status launch_rope_gather(const moga_shape& s, const moga_rope_plan& p, const int32_t* pos, int pos_per_batch,
                               const int32_t* inv, const void* Q, const void* K, const void* V, void* Qp, void* Kp,
                               void* Vp, cudaStream_t st) {
  const RopeWay way = rope_way(s, p);
  dim3 grid;
  const RopeArgs a = rope_args(s, p, pos, pos_per_batch, false, way, 8, &grid);
  const RotateTensors t{Q, K, V, Qp, Kp, Vp, inv, s.k};
  return s.dtype == MOGA_BF16 ? run_rope<__nv_bfloat16, true>(a, t, way, grid, st) : run_rope<float, true>(a, t, way, grid, st);
}

moga_status launch_rope_ungather(const moga_shape& s, const moga_rope_plan& p, const int32_t* pos, int pos_per_batch,
                                 const void* dQp, const void* dKp, const void* dVp, const int32_t* inv, void* dQ,
                                 void* dK, void* dV, cudaStream_t st) {
  const RopeWay way = rope_way(s, p);
  dim3 grid;
  const RopeArgs a = rope_args(s, p, pos, pos_per_batch, true, way, 16, &grid);
  const UnrotateTensors t{{dQp, dKp, dVp}, {dQ, dK, dV}, inv, s.k};
  return s.dtype == MOGA_BF16 ? run_back_path<__nv_bfloat16>(a, t, way, grid, st) : run_back_path<float>(a, t, way, grid, st);
}

// Host only: the plan of a configuration.
moga_status rope_build(const moga_rope_config& c, moga_rope_plan* out) {
  const bool scaled = c.scaling != MOGA_ROPE_SCALE_NONE;
  if ((c.layout != MOGA_ROPE_INTERLEAVED && c.layout != MOGA_ROPE_HALF) || c.scaling < MOGA_ROPE_SCALE_NONE ||
      c.scaling > MOGA_ROPE_SCALE_BY_PARTS || c.n_axes < 1 || c.n_axes > 3 || !(c.base >= 1.0) || !isfinite(c.base) ||
      !isfinite(c.amplitude))
    return MOGA_ERR_INVALID_ARG;
  if (c.n_axes > 1 && (c.grid_w < 0 || c.grid_h < 0)) return MOGA_ERR_INVALID_ARG;
  if (c.scaling == MOGA_ROPE_SCALE_BY_PARTS &&
      (!(c.original_length > 0.0) || !isfinite(c.original_length) || !(c.beta_fast > c.beta_slow) || !(c.beta_slow >= 0.0) ||
       !isfinite(c.beta_fast)))
    return MOGA_ERR_INVALID_ARG;
  moga_rope_plan p{};
  p.layout = c.layout;
  p.n_axes = c.n_axes;
  p.grid_h = c.grid_h;
  p.grid_w = c.grid_w;
  p.amplitude = c.amplitude;
  const long double two_pi = 6.283185307179586476925286766559005768L;
  for (int x = 0; x < c.n_axes; ++x) {
    const int d = c.axis_dim[x];
    if (d < 2 || (d & 1)) return MOGA_ERR_INVALID_ARG;
    if (p.pairs + d / 2 > kMaxPairs) return MOGA_ERR_UNSUPPORTED;
    if (scaled && (!(c.factor[x] > 0.0) || !isfinite(c.factor[x]))) return MOGA_ERR_INVALID_ARG;
    const long double f = scaled ? (long double)c.factor[x] : 1.0L;
    long double base = c.base;
    if (c.scaling == MOGA_ROPE_SCALE_BASE && d > 2) base *= powl(f, (long double)d / (d - 2));
    p.start[x] = c.start[x];
    p.axis_pairs[x] = d / 2;
    for (int i = 0; i < d / 2; ++i) {
      long double theta = powl(base, -2.0L * i / d);
      if (c.scaling == MOGA_ROPE_SCALE_LINEAR) {
        theta /= f;
      } else if (c.scaling == MOGA_ROPE_SCALE_BY_PARTS) {
        const long double turns = (long double)c.original_length * theta / two_pi;
        long double g = (turns - c.beta_slow) / ((long double)c.beta_fast - c.beta_slow);
        g = g < 0.0L ? 0.0L : g > 1.0L ? 1.0L : g;
        theta = (1.0L - g) * theta / f + g * theta;
      }
      const long double frac = fmodl(theta / two_pi, 1.0L) * 18446744073709551616.0L;   // theta > 0
      p.turns[p.pairs++] = frac >= 18446744073709551615.0L ? 0 : (uint64_t)(frac + 0.5L);
    }
  }
  *out = p;
  return MOGA_OK;
}

}  // namespace moga
