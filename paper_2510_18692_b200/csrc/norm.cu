// Layer norm over the channels of a token, forward and backward, and the same with the residual
// addition (and dropout) in front of it: the norm whose output the router and the projections read.
//
// Forward, one row x of C channels: m = mean x, v = mean (x - m)^2, y = (x - m) / sqrt(v + eps) w + b.
// The row is read from memory once and stays in registers; sums and statistics are fp32, taken so that rows
// far from zero keep their digits.  HBM-bound: two (with the residual four) tensor passes.
//
// Backward: with g = dy w and xh = (x - m) r, dx = r (g - mean g - xh mean(g xh)), dw = sum dy xh and
// db = sum dy over the rows.  One pass over x and dy: a block owns a run of rows and all channels, its
// threads keep their channels' dw and db in registers, and the block writes one partial row; a second
// launch adds the partials in a fixed order (no atomics, the same bits every run).
//
// What bounds these kernels on a B200 (times below: bf16, under sustained load, at which the board sits at its
// power limit and the SMs run at 1.6 - 1.8 GHz instead of 1.97): the HBM while a kernel spends fewer than about
// two instructions on a byte it moves, above that the issue slots at the lowered clock.
//   forward, 561,600 x 5,120           1.76 - 1.78 ms, 6.5 TB/s (a device copy of as many bytes: 1.75 ms)
//   backward, 126,360 x 5,120          0.63 - 0.67 ms, 5.8 - 6.1 TB/s;  fp32, 20,000 x 5,120: 0.199 ms, 6.2 TB/s
//   residual forward, 65,520 x 1,536   0.137 - 0.145 ms, 5.6 - 5.9 TB/s;  fp32, 20,000 x 5,120: 0.242 ms, 6.8 TB/s
//   residual backward, 32,760 x 5,120  0.303 - 0.319 ms, 5.3 - 5.5 TB/s;  fp32, 20,000 x 5,120: 0.336 ms, 6.1 TB/s
#include "block_common.cuh"

namespace moga {
namespace {

// How rows are dealt to blocks that keep per-channel values for a run of rows.  The SMs of a B200 do not get
// equal shares of the memory's bandwidth (a row copy with equal static shares ends on the fastest SMs after
// 70 % of its time, and reaches 5.9 TB/s where first-come blocks reach 6.8), so the runs shrink: a first tier of
// one long run for each resident block, then tiers of shorter ones, which the block scheduler hands to whichever
// SM is free.  Which rows a block has depends on its index alone, so sums over a run keep their order.
// Where a longest run is set, as many tiers of it come first as it takes; they are stored as one.
constexpr int kMaxTiers = 48;
struct Tiers {
  int items, blocks;               // of a tier, blocks for each item
  int count;                       // tiers, of which the first `alike` have the rows of size[0]
  int alike;
  int size[kMaxTiers];             // rows of a block, from the last of those tiers on
  int start[kMaxTiers + 1];        // rows of an item before that tier (start[0]: before the first)
};
// rows: of an item (below 2^31); resident: blocks that run at once; most, least: rows of a run.
inline Tiers make_tiers(long long rows, int items, int resident, int most, int least) {
  Tiers t{};
  t.items = items;
  t.blocks = resident / items < 1 ? 1 : resident / items;
  if (t.blocks > rows) t.blocks = (int)rows;
  long long done = 0;
  int stored = 0;
  while (done < rows) {
    const long long left = rows - done, share = (left + t.blocks - 1) / t.blocks;
    long long size = stored == 0 ? share * 5 / 8 : share / 2;
    if (size < least || share - size < least / 2) size = share < 2 * least ? share : least;
    if (stored == kMaxTiers - 1) size = share;
    else if (size > most) size = most;
    if (stored == 0) t.size[stored++] = (int)size;
    else if (stored > 1 || size != most || t.size[0] != most) {
      t.start[stored] = (int)done;
      t.size[stored++] = (int)size;
    }
    if (stored == 1) t.alike++;
    t.count++;
    done += size * t.blocks < left ? size * t.blocks : left;
  }
  t.start[stored] = (int)rows;
  return t;
}
// The run of block `block`: its item, first row inside the item, and rows (0 for the last of an uneven tier).
__device__ __forceinline__ void block_run(const Tiers& t, int block, int& item, int& lo, int& rows) {
  const int per = t.items * t.blocks, tier = block / per, at = max(tier - t.alike + 1, 0);
  item = block % per / t.blocks;
  const int size = t.size[at], end = t.start[at + 1];
  const long long first = at > 0 ? t.start[at] : (long long)tier * size * t.blocks;
  lo = (int)min(first + (long long)(block % t.blocks) * size, (long long)end);
  rows = min(size, end - lo);
}

struct FwdArgs {
  const void *X, *R;           // X: input, or what is dropped; R: residual (RES only)
  const float *W, *bias;       // [C] or [items, C]; may be null
  void *Hout, *Y;
  float *mean, *rstd;          // may be null
  long long rows;              // rows of one item
  int nvec;                    // vectors of a row
  int C;
  int param_stride;            // C if W, bias are given for each item, else 0
  float eps;
  DropArgs drop;
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" :: "n"(N) : "memory"); }
__device__ __forceinline__ uint4 lds128(uint32_t at) {
  uint4 r;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(at) : "memory");
  return r;
}

template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int o = (LANES < 32 ? LANES : 32) / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// How many lanes hold the partial results of a block's warps (a power of two, every such group of lanes holds
// all of them): what the second step of a sum over the block has to exchange over.
__host__ __device__ constexpr int warp_lanes(int max_threads) { return max_threads <= 128 ? 4 : max_threads <= 256 ? 8 : max_threads <= 512 ? 16 : 32; }

// (x - mean) rstd: the difference first, so that rows far from zero, and constant rows, lose nothing (one fused
// step with mean rstd rounded turns a constant row of 1,000 into 0.02 instead of 0, and measured the same time).
__device__ __forceinline__ float2 centred(const float2& x, float mean, float rstd) {
  return __fmul2_rn(__fadd2_rn(x, both(-mean)), both(rstd));
}

// NV (2 or 4) sums over the warps of a block, one barrier; red holds [NV][32] words and the caller alternates
// between two such buffers.  The lanes of a warp exchange halves first (each keeps half of the values, then a
// quarter), so that four sums cost six shuffles instead of twenty.
template <int NV, int WL>
__device__ __forceinline__ void block_sums(float (&v)[NV], float* red, int warps) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int half = NV / 2, bit = 1; half > 0; half /= 2, bit *= 2) {
    const bool up = lane & bit;
#pragma unroll
    for (int i = 0; i < half; ++i) {
      const float keep = up ? v[i + half] : v[i], send = up ? v[i] : v[i + half];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, send, bit);
    }
  }
  float t = v[0];                                 // of value number: the lane's low bits, reversed
#pragma unroll
  for (int o = NV; o < 32; o *= 2) t += __shfl_xor_sync(0xffffffffu, t, o);
  const int mine = NV == 2 ? lane : (lane & 1) * 2 + (lane >> 1);
  if (lane < NV) red[mine * 32 + (threadIdx.x >> 5)] = t;
  __syncthreads();
  if constexpr (WL <= 8) {                        // few warps: read them all
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = 0.f;
    for (int w = 0; w < warps; ++w)
#pragma unroll
      for (int i = 0; i < NV; ++i) v[i] += red[i * 32 + w];
  } else {                                        // 32 / NV lanes for each value
    constexpr int G = 32 / NV;
    t = 0.f;
    for (int w = lane % G; w < warps; w += G) t += red[lane / G * 32 + w];
#pragma unroll
    for (int o = 1; o < G; o *= 2) t += __shfl_xor_sync(0xffffffffu, t, o);
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = __shfl_sync(0xffffffffu, t, i * G);
  }
}

// Two sums for each of a thread's ROWS rows over the threads of the row.  A block has one group of
// threads when a row has several warps; red is then read by all of them behind one barrier.
template <int TPR, int ROWS>
__device__ __forceinline__ void row_sum2(float (&a)[ROWS], float (&b)[ROWS], float2 (*red)[ROWS]) {
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    a[r] = lanes_sum<TPR>(a[r]);
    b[r] = lanes_sum<TPR>(b[r]);
  }
  if constexpr (TPR > 32) {
    const int warp = threadIdx.x >> 5;
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
      for (int r = 0; r < ROWS; ++r) red[warp][r] = make_float2(a[r], b[r]);
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      a[r] = b[r] = 0.f;
#pragma unroll
      for (int i = 0; i < TPR / 32; ++i) {
        const float2 t = red[i][r];
        a[r] += t.x;
        b[r] += t.y;
      }
    }
  }
}

// Few rows, short rows, and the residual form.  TPR threads share ROWS consecutive rows, each holds VPT vectors
// VT of each.  Short rows come several to a thread, because W and bias are two to four times as wide as the
// channels they belong to and their loads through L1 bound the kernel otherwise (400,000 x 256: 78 us with four
// rows, 98 with one).  The mean is the first of two sums over registers; the second also sums x - m, which
// corrects mean and variance for the rounding of the first.
template <typename XT, typename VT, int TPR, int VPT, int ROWS, bool RES>
__global__ void __launch_bounds__(TPR > 32 ? TPR : 128) norm_fwd_kernel(const __grid_constant__ FwdArgs a) {
  constexpr int E = sizeof(VT) / sizeof(XT), P = E / 2;
  constexpr int kThreads = TPR > 32 ? TPR : 128;
  constexpr int kGroups = kThreads / TPR;
  __shared__ float2 red[2][TPR > 32 ? TPR / 32 : 1][ROWS];
  const int lane = threadIdx.x % TPR;
  const long long row_in = ((long long)blockIdx.x * kGroups + threadIdx.x / TPR) * ROWS;
  const int live = (int)min((long long)ROWS, a.rows - row_in);   // a group without rows still joins the sums
  const long long row = (long long)blockIdx.y * a.rows + (live > 0 ? row_in : 0);
  const uint64_t base = (uint64_t)row * a.nvec;
  const VT *X = static_cast<const VT*>(a.X) + base;
  VT x[ROWS][VPT];
  const uint64_t offset = RES ? drop_offset(a.drop) : 0;
#pragma unroll
  for (int r = 0; r < ROWS; ++r)
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int v = lane + i * TPR;
      x[r][i] = r < live && v < a.nvec ? load_stream(X + (uint64_t)r * a.nvec + v) : VT{};
    }
  if constexpr (RES) {
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      VT res[VPT];
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        const int v = lane + i * TPR;
        res[i] = r < live && v < a.nvec ? load_stream(static_cast<const VT*>(a.R) + base + (uint64_t)r * a.nvec + v) : VT{};
      }
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        const int v = lane + i * TPR;
        const uint64_t at = base + (uint64_t)r * a.nvec + v;
        float2 f[P], g[P];
        unpack(x[r][i], f);
        unpack(res[i], g);
        drop_vec(a.drop, offset, at, f);
#pragma unroll
        for (int e = 0; e < P; ++e) f[e] = __fadd2_rn(f[e], g[e]);
        x[r][i] = pack_as<VT>(f);                       // the stream is stored in its type, and normed as stored
        if (r < live && v < a.nvec) store_stream(static_cast<VT*>(a.Hout) + at, x[r][i]);
      }
    }
  }
  float s[ROWS], s1[ROWS], s2[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    float2 t = both(0.f);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {              // lanes past the row hold zeros
      float2 f[P];
      unpack(x[r][i], f);
#pragma unroll
      for (int e = 0; e < P; ++e) t = __fadd2_rn(t, f[e]);
    }
    s[r] = t.x + t.y;
    s1[r] = 0.f;
  }
  row_sum2<TPR, ROWS>(s, s1, red[0]);
  const float inv_c = 1.f / (float)a.C;
  float mean[ROWS], rstd[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    mean[r] = s[r] * inv_c;
    float2 t1 = both(0.f), t2 = both(0.f);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      if (lane + i * TPR < a.nvec) {
        float2 f[P];
        unpack(x[r][i], f);
#pragma unroll
        for (int e = 0; e < P; ++e) {
          const float2 d = __fadd2_rn(f[e], both(-mean[r]));
          t1 = __fadd2_rn(t1, d);
          t2 = __ffma2_rn(d, d, t2);
        }
      }
    }
    s1[r] = t1.x + t1.y;
    s2[r] = t2.x + t2.y;
  }
  row_sum2<TPR, ROWS>(s1, s2, red[1]);
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    const float fix = s1[r] * inv_c;
    const float var = fmaxf(fmaf(-fix, fix, s2[r] * inv_c), 0.f);
    mean[r] += fix;
    rstd[r] = s2[r] == s2[r] ? rsqrtf(var + a.eps) : s2[r];   // fmaxf would turn a NaN into 0
    if (lane == 0 && r < live) {
      if (a.mean != nullptr) a.mean[row + r] = mean[r];
      if (a.rstd != nullptr) a.rstd[row + r] = rstd[r];
    }
  }
  const long long po = (long long)blockIdx.y * a.param_stride;
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int v = lane + i * TPR;
    if (v >= a.nvec) continue;
    float2 w[P], b[P];
#pragma unroll
    for (int q = 0; q < P / 2; ++q) {
      float4 t = make_float4(1.f, 1.f, 1.f, 1.f);
      if (a.W != nullptr) t = __ldg(reinterpret_cast<const float4*>(a.W + po + (size_t)v * E) + q);
      w[2 * q] = make_float2(t.x, t.y);
      w[2 * q + 1] = make_float2(t.z, t.w);
      t = make_float4(0.f, 0.f, 0.f, 0.f);
      if (a.bias != nullptr) t = __ldg(reinterpret_cast<const float4*>(a.bias + po + (size_t)v * E) + q);
      b[2 * q] = make_float2(t.x, t.y);
      b[2 * q + 1] = make_float2(t.z, t.w);
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (r >= live) continue;
      float2 f[P];
      unpack(x[r][i], f);
#pragma unroll
      for (int e = 0; e < P; ++e)
        f[e] = __ffma2_rn(__fmul2_rn(__fadd2_rn(f[e], both(-mean[r])), both(rstd[r])), w[e], b[e]);
      store_stream(static_cast<VT*>(a.Y) + base + (uint64_t)r * a.nvec + v, pack_as<VT>(f));
    }
  }
}

template <typename XT, typename VT, int TPR, int VPT, int ROWS, bool RES>
moga_status run_fwd_v(FwdArgs a, int items, cudaStream_t st) {
  constexpr int threads = TPR > 32 ? TPR : 128, rows = threads / TPR * ROWS;
  a.nvec = (int)(a.C * sizeof(XT) / sizeof(VT));
  const long long blocks = (a.rows + rows - 1) / rows;
  if (blocks > 0x7fffffffll) return MOGA_ERR_UNSUPPORTED;
  norm_fwd_kernel<XT, VT, TPR, VPT, ROWS, RES><<<dim3((unsigned)blocks, items), threads, 0, st>>>(a);
  MOGA_CUDA_OK(cudaGetLastError());
  return MOGA_OK;
}

// VPT counts 16-byte vectors.  The plain norm of bf16 takes them as twice as many 8-byte ones.
template <typename XT, int TPR, int VPT, int ROWS, bool RES>
moga_status run_fwd(const FwdArgs& a, int items, cudaStream_t st) {
  if constexpr (RES || sizeof(XT) == 4) return run_fwd_v<XT, uint4, TPR, VPT, ROWS, RES>(a, items, st);
  else return run_fwd_v<XT, uint2, TPR, 2 * VPT, ROWS, RES>(a, items, st);
}

// The norm of many rows.  One block of 512 threads stays on each SM, with W and bias in
// shared memory (read per row through L1 they would be two to four times the row's own traffic, and rows two
// by two halve it again).  A row belongs to a group of 32 WPG threads, each with VPT vectors, only the last
// of which may lie past the row; groups go their own way, with a barrier of their own.  A ring of cp.async
// copies keeps the next rows on the way: each thread fetches its own vectors into its own slots and reads
// them back itself, so the ring needs no barrier.
// Long rows of few threads keep the instructions for a channel low, and the shrinking runs keep all SMs busy to
// the end: 561,600 x 5,120 takes 1.76 ms; blocks of 320 threads to a row with W and bias in registers and equal
// runs took 2.01, the same with shrinking runs 2.03 (1.75 at full clocks), this kernel with equal runs 1.99.
// Statistics by merging (Chan, Golub, LeVeque 1979): a thread takes the mean m and the sum q of squared
// deviations of its own n channels; (n, m, q) and (n', m', q') with d = m' - m give m + d n' / (n + n') and
// q + q' + d^2 n n' / (n + n').  The counts, so the factors too, are the same for every row.  No cancellation
// for rows far from zero.
constexpr int kStreamThreads = 512, kStreamRows = 2, kStreamStages = 2;
template <typename XT, int WPG, int VPT>
__global__ void __launch_bounds__(kStreamThreads, 1) norm_stream_kernel(const __grid_constant__ FwdArgs a,
                                                                        const __grid_constant__ Tiers tiers) {
  constexpr int E = VecTraits<XT>::E, P = E / 2, Q = E / 4, ROWS = kStreamRows, STAGES = kStreamStages;
  constexpr int T = kStreamThreads, G = 32 * WPG, GROUPS = T / G;
  extern __shared__ __align__(16) uint4 ring[];
  __shared__ float2 red[2][GROUPS][ROWS][WPG];
  const int tid = threadIdx.x, lane = tid & 31, at = tid % G, group = tid / G, warp = at >> 5;
  int item, lo, total;
  block_run(tiers, blockIdx.x, item, lo, total);
  if (total <= 0) return;
  const size_t first = (size_t)item * a.rows + lo;
  constexpr int stride = GROUPS * ROWS;           // the run's rows, dealt out to the groups two by two
  const bool whole = at + (VPT - 1) * G < a.nvec;                   // all VPT vectors are the row's
  auto has = [&](int i) { return i < VPT - 1 || whole; };
  // W and bias as float4 planes [2 Q][nvec]: a warp's reads are contiguous
  float4* params = reinterpret_cast<float4*>(ring + STAGES * ROWS * VPT * T);
  for (int v = tid; v < a.nvec; v += T) {
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const size_t c = (size_t)item * a.param_stride + (size_t)v * E + 4 * q;
      params[q * a.nvec + v] = a.W != nullptr ? __ldg(reinterpret_cast<const float4*>(a.W + c)) : make_float4(1.f, 1.f, 1.f, 1.f);
      params[(Q + q) * a.nvec + v] = a.bias != nullptr ? __ldg(reinterpret_cast<const float4*>(a.bias + c)) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
  }
  __syncthreads();
  int row = group * ROWS;
  const size_t step = (size_t)stride * a.nvec;
  const uint4* src = static_cast<const uint4*>(a.X) + (first + row) * a.nvec + at;
  uint4* dst = static_cast<uint4*>(a.Y) + (first + row) * a.nvec + at;
  const uint32_t smem = (uint32_t)__cvta_generic_to_shared(ring) + tid * 16;
  constexpr uint32_t plane = T * 16, row_bytes = plane * VPT, stage_bytes = row_bytes * ROWS;
  auto fetch = [&](int row, uint32_t stage) {
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
      if (row + r < total) {
#pragma unroll
        for (int i = 0; i < VPT; ++i)
          if (has(i)) cp_async16(stage + r * row_bytes + i * plane, src + (size_t)r * a.nvec + i * G);
      }
    cp_async_commit();
    src += step;
  };
  fetch(row, smem);
  fetch(row + stride, smem + stage_bytes);
  // factors of the five merges inside the warp
  float part[5], weight[5], n = (float)(whole ? VPT * E : (VPT - 1) * E);
  const float inv_n = 1.f / n, inv_c = 1.f / (float)a.C;
#pragma unroll
  for (int s = 0; s < 5; ++s) {
    const float next = __shfl_xor_sync(0xffffffffu, n, 1 << s);
    part[s] = next / (n + next);
    weight[s] = n * part[s];
    n += next;
  }
  int buf = 0;
  for (uint32_t stage = smem; row < total; row += stride) {
    cp_async_wait<STAGES - 1>();
    uint4 x[ROWS][VPT];
    float m[ROWS], q[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {              // past the last row: an older row's values, never stored
#pragma unroll
      for (int i = 0; i < VPT; ++i)
        if (has(i)) x[r][i] = lds128(stage + r * row_bytes + i * plane);
      float2 t = both(0.f);
      if constexpr (E == 8) {
        // one pass around k, the mean of the thread's first vector: m = k + sum d / n, q = sum d^2 - (sum d)^2 / n.
        // 8 (k - m)^2 <= q, so the difference loses at most a factor 1 + n / 8 (6 for 40 channels).
        float2 f[P], d1 = both(0.f);
        unpack(x[r][0], f);
#pragma unroll
        for (int e = 0; e < P; ++e) t = __fadd2_rn(t, f[e]);
        const float k = (t.x + t.y) * (1.f / E);
        t = both(0.f);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
          if (has(i)) {
            unpack(x[r][i], f);
#pragma unroll
            for (int e = 0; e < P; ++e) {
              const float2 d = __fadd2_rn(f[e], both(-k));
              d1 = __fadd2_rn(d1, d);
              t = __ffma2_rn(d, d, t);
            }
          }
        }
        const float s1 = d1.x + d1.y, mean_d = s1 * inv_n;
        m[r] = k + mean_d;
        q[r] = fmaf(-s1, mean_d, t.x + t.y);
      } else {                                    // fp32: the thread's mean first, then sums around it that correct it,
                                                  // or a constant row of 1,000.1 would lie 6e-5 off its mean (0.02 in Y)
        float2 f[VPT][P];
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
          if (has(i)) {
            unpack(x[r][i], f[i]);
#pragma unroll
            for (int e = 0; e < P; ++e) t = __fadd2_rn(t, f[i][e]);
          }
        }
        m[r] = (t.x + t.y) * inv_n;
        float2 d1 = both(0.f);
        t = both(0.f);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
          if (has(i)) {
#pragma unroll
            for (int e = 0; e < P; ++e) {
              const float2 d = __fadd2_rn(f[i][e], both(-m[r]));
              d1 = __fadd2_rn(d1, d);
              t = __ffma2_rn(d, d, t);
            }
          }
        }
        const float s1 = d1.x + d1.y, fix = s1 * inv_n;
        m[r] += fix;
        q[r] = fmaf(-s1, fix, t.x + t.y);
      }
    }
    fetch(row + STAGES * stride, stage);   // the values are in registers
    stage = stage == smem ? smem + stage_bytes : smem;
#pragma unroll
    for (int s = 0; s < 5; ++s)
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        const float d = __shfl_xor_sync(0xffffffffu, m[r], 1 << s) - m[r];
        q[r] = fmaf(d * d, weight[s], q[r] + __shfl_xor_sync(0xffffffffu, q[r], 1 << s));
        m[r] = fmaf(d, part[s], m[r]);
      }
    float mean[ROWS], rstd[ROWS];
    if constexpr (WPG > 1) {
      if (lane == 0) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r) red[buf][group][r][warp] = make_float2(m[r], q[r]);
      }
      asm volatile("bar.sync %0, %1;" :: "r"(1 + group), "n"(G) : "memory");
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        const float ref = red[buf][group][r][0].x;
        float s = 0.f, dev = 0.f;
        float2 part_of[WPG];
#pragma unroll
        for (int k = 0; k < WPG; ++k) {
          const float channels = (float)(E * (32 * (VPT - 1) + min(max(a.nvec - (VPT - 1) * G - 32 * k, 0), 32)));
          part_of[k] = red[buf][group][r][k];
          s = fmaf(channels, part_of[k].x - ref, s);
        }
        mean[r] = fmaf(s, inv_c, ref);
#pragma unroll
        for (int k = 0; k < WPG; ++k) {
          const float channels = (float)(E * (32 * (VPT - 1) + min(max(a.nvec - (VPT - 1) * G - 32 * k, 0), 32)));
          const float d = part_of[k].x - mean[r];
          dev += fmaf(channels * d, d, part_of[k].y);
        }
        q[r] = dev;
      }
      buf ^= 1;                                   // the next barrier comes before this half is written again
    } else {
#pragma unroll
      for (int r = 0; r < ROWS; ++r) mean[r] = m[r];
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      rstd[r] = rsqrtf(fmaf(q[r] < 0.f ? 0.f : q[r], inv_c, a.eps));
      if (at == 0 && row + r < total) {
        if (a.mean != nullptr) a.mean[first + row + r] = mean[r];
        if (a.rstd != nullptr) a.rstd[first + row + r] = rstd[r];
      }
    }
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      if (has(i)) {
        float2 w[P], b[P];
#pragma unroll
        for (int q4 = 0; q4 < Q; ++q4) {
          const float4 u = params[q4 * a.nvec + at + i * G], v = params[(Q + q4) * a.nvec + at + i * G];
          w[2 * q4] = make_float2(u.x, u.y), w[2 * q4 + 1] = make_float2(u.z, u.w);
          b[2 * q4] = make_float2(v.x, v.y), b[2 * q4 + 1] = make_float2(v.z, v.w);
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
          if (row + r < total) {
            float2 f[P];
            unpack(x[r][i], f);
#pragma unroll
            for (int e = 0; e < P; ++e) f[e] = __ffma2_rn(centred(f[e], mean[r], rstd[r]), w[e], b[e]);
            store_stream(dst + (size_t)r * a.nvec + i * G, pack(f));
          }
        }
      }
    }
    dst += step;
  }
  cp_async_wait<0>();
}

template <typename XT, int WPG, int VPT>
moga_status run_stream(const FwdArgs& a, int items, cudaStream_t st) {
  auto kernel = norm_stream_kernel<XT, WPG, VPT>;
  const int smem = kStreamStages * kStreamRows * VPT * kStreamThreads * 16 + 2 * a.C * (int)sizeof(float);
  const Tiers tiers = make_tiers(a.rows, items, 148, 1 << 20, 32);   // a block for each SM
  MOGA_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  kernel<<<tiers.items * tiers.blocks * tiers.count, kStreamThreads, smem, st>>>(a, tiers);
  MOGA_CUDA_OK(cudaGetLastError());
  return MOGA_OK;
}
template <typename XT, int WPG>
moga_status dispatch_stream(const FwdArgs& a, int items, cudaStream_t st) {
  if (a.nvec <= 96 * WPG) return run_stream<XT, WPG, 3>(a, items, st);
  if (a.nvec <= 128 * WPG) return run_stream<XT, WPG, 4>(a, items, st);
  return run_stream<XT, WPG, 5>(a, items, st);
}

// The split of a row over threads.  Many rows: the streaming kernel (from 148 x 8 rows on: 1,560 x 5,120 takes
// 8.4 us, 9.3 with a block to a row; 4,000 x 5,120 14.8 and 16.5), or, for short rows and the residual form,
// threads that hold the row in registers.  With the residual a block of 128 threads to a row is best for long
// rows (30,000 x 5,120: 186 us at full clocks, 317 with a warp to a row, 204 with 160 threads, 205 in the streaming
// kernel), of 64 for middle ones (50,000 x 2,560: 158 us, 175 with 128 threads; 60,000 x 2,048: 164 us, 185 with a
// warp), a warp below (120,000 x 1,000: 162 us, 182 with 64 threads).
// Few rows: the row is spread over more threads.
template <typename XT, bool RES>
moga_status dispatch_fwd(const FwdArgs& a, int items, cudaStream_t st) {
  const int n = a.nvec;
  const bool many = a.rows * items > 148 * 8;
  if (many) {
    if (n <= 8) return run_fwd<XT, 8, 1, RES ? 2 : 4, RES>(a, items, st);
    if (n <= 16) return run_fwd<XT, 16, 1, RES ? 2 : 4, RES>(a, items, st);
    if (n <= 32) return run_fwd<XT, 32, 1, RES ? 2 : 4, RES>(a, items, st);
    if (n <= 64) return run_fwd<XT, 32, 2, 2, RES>(a, items, st);
    if constexpr (RES) {
      if (n <= 96) return run_fwd<XT, 32, 3, 1, RES>(a, items, st);
      if (n <= 128) return run_fwd<XT, 32, 4, 1, RES>(a, items, st);
      if (n <= 192) return run_fwd<XT, 64, 3, 1, RES>(a, items, st);
      if (n <= 256) return run_fwd<XT, 64, 4, 1, RES>(a, items, st);
      if (n <= 320) return run_fwd<XT, 64, 5, 1, RES>(a, items, st);
      if (n <= 384) return run_fwd<XT, 64, 6, 1, RES>(a, items, st);
      if (n <= 512) return run_fwd<XT, 128, 4, 1, RES>(a, items, st);
      if (n <= 640) return run_fwd<XT, 128, 5, 1, RES>(a, items, st);
    } else {
      if (n <= 160) return dispatch_stream<XT, 1>(a, items, st);
      if (n <= 320) return dispatch_stream<XT, 2>(a, items, st);
      if (n <= 640) return dispatch_stream<XT, 4>(a, items, st);
      if (n <= (sizeof(XT) == 2 ? 1024 : 1280)) return dispatch_stream<XT, 8>(a, items, st);   // ring and W, bias: 200 KB
    }
  } else {
    if (n <= 8) return run_fwd<XT, 8, 1, 1, RES>(a, items, st);
    if (n <= 16) return run_fwd<XT, 16, 1, 1, RES>(a, items, st);
    if (n <= 32) return run_fwd<XT, 32, 1, 1, RES>(a, items, st);
    if (n <= 128) return run_fwd<XT, 128, 1, 1, RES>(a, items, st);
    if (n <= 256) return run_fwd<XT, 256, 1, 1, RES>(a, items, st);
    if (n <= 512) return run_fwd<XT, 512, 1, 1, RES>(a, items, st);
  }
  if (n <= 1024) return run_fwd<XT, 256, 4, 1, RES>(a, items, st);
  if (n <= 1280) return run_fwd<XT, 256, 5, 1, RES>(a, items, st);
  return run_fwd<XT, 512, 4, 1, RES>(a, items, st);
}

// ---------------------------------------------------------------- backward
struct BwdArgs {
  const uint4 *X, *dY, *dH;    // dH (RES only): gradient that reaches the stored stream from elsewhere, may be null
  const float *W, *mean, *rstd;
  uint4 *dX, *dR;
  float* part;                 // [blocks, 2, C] partial dW, dbias
  long long rows;              // rows of one item
  int nvec, C, param_stride;
  Tiers tiers;                 // the runs of rows; a block writes one partial row
  int want;                    // bit 0: dW, bit 1: dbias
  DropArgs drop;
};


// Rows of at most 64 vectors: TPR threads of a warp share a row, the groups of a block take consecutive rows.
// Each thread copies its own vectors into its own slots of a ring with cp.async and reads them back itself,
// so there is no barrier until the block adds up its groups' parameter gradients.
constexpr int kGroupThreads = 256, kGroupStages = 4;
template <typename XT, int TPR, int VPT, bool RES>
__global__ void __launch_bounds__(kGroupThreads, 2) norm_bwd_group_kernel(const __grid_constant__ BwdArgs a) {
  constexpr int E = VecTraits<XT>::E, P = E / 2, NT = RES ? 3 : 2, T = kGroupThreads, GROUPS = T / TPR;
  constexpr int STAGES = kGroupStages;
  extern __shared__ __align__(16) uint4 ring[];
  const int tid = threadIdx.x, lane = tid % TPR, group = tid / TPR;
  int item, lo, run;
  block_run(a.tiers, blockIdx.x, item, lo, run);
  const size_t first = (size_t)item * a.rows + lo + group, at0 = first * a.nvec + lane, step = (size_t)GROUPS * a.nvec;
  const int total = run - group, most = run;      // this group: rows 0, GROUPS, 2 GROUPS, ... below total
  auto has = [&](int i) { return lane + i * TPR < a.nvec; };
  constexpr uint32_t plane = T * 16, row_bytes = plane * VPT * NT;
  const uint32_t smem = (uint32_t)__cvta_generic_to_shared(ring) + tid * 16;
  const bool has_h = RES && a.dH != nullptr;
  const uint4 *fx = a.X + at0, *fy = a.dY + at0, *fh = has_h ? a.dH + at0 : nullptr;
  uint32_t fstage = smem;
  int fetched = 0;
  auto fetch = [&]() {
    if (fetched < total) {
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        if (has(i)) {
          cp_async16(fstage + (i * NT) * plane, fx + i * TPR);
          cp_async16(fstage + (i * NT + 1) * plane, fy + i * TPR);
          if (has_h) cp_async16(fstage + (i * NT + 2) * plane, fh + i * TPR);
        }
      }
    }
    cp_async_commit();
    fetched += GROUPS;
    fx += step;
    fy += step;
    if (has_h) fh += step;
    fstage += row_bytes;
    if (fstage == smem + STAGES * row_bytes) fstage = smem;
  };
#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) fetch();
  float2 w[VPT][P], dw[VPT][P], db[VPT][P];
#pragma unroll
  for (int i = 0; i < VPT; ++i)
#pragma unroll
    for (int e = 0; e < P; ++e) {
      dw[i][e] = db[i][e] = both(0.f);
      const size_t c = (size_t)item * a.param_stride + (size_t)(lane + i * TPR) * E;
      w[i][e] = both(1.f);
      if (a.W != nullptr && has(i)) w[i][e] = __ldg(reinterpret_cast<const float2*>(a.W + c) + e);
    }
  const uint64_t offset = RES ? drop_offset(a.drop) : 0;
  const float inv_c = 1.f / (float)a.C;
  const float *pm = a.mean + first, *pr = a.rstd + first;
  float mean = total > 0 ? __ldg(pm) : 0.f, rstd = total > 0 ? __ldg(pr) : 0.f;
  uint4 *dx = a.dX + at0, *dr = RES ? a.dR + at0 : nullptr;
  uint64_t vec = at0;
  uint32_t stage = smem;
  for (int row = 0; row < most; row += GROUPS) {  // the same trips for all groups: they share warps' shuffles
    fetch();
    cp_async_wait<STAGES - 1>();
    const bool live = row < total;
    const float next_mean = row + GROUPS < total ? __ldg(pm + row + GROUPS) : 0.f;
    const float next_rstd = row + GROUPS < total ? __ldg(pr + row + GROUPS) : 0.f;
    const float2 nm = both(-mean), rs = both(rstd);
    float2 t1 = both(0.f), t2 = both(0.f);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      if (live && has(i)) {
        float2 x[P], dy[P];
        unpack(lds128(stage + (i * NT) * plane), x);
        unpack(lds128(stage + (i * NT + 1) * plane), dy);
#pragma unroll
        for (int e = 0; e < P; ++e) {
          const float2 xh = __fmul2_rn(__fadd2_rn(x[e], nm), rs), g = __fmul2_rn(dy[e], w[i][e]);
          dw[i][e] = __ffma2_rn(dy[e], xh, dw[i][e]);
          db[i][e] = __fadd2_rn(db[i][e], dy[e]);
          t1 = __fadd2_rn(t1, g);
          t2 = __ffma2_rn(g, xh, t2);
        }
      }
    }
    // r (g - c1 - xh c2) = r g + (x - m) (-r^2 c2) - r c1
    const float2 c1 = both(-rstd * (lanes_sum<TPR>(t1.x + t1.y) * inv_c)),
                 c2 = both(-rstd * rstd * (lanes_sum<TPR>(t2.x + t2.y) * inv_c));
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      if (live && has(i)) {
        float2 x[P], dy[P];
        unpack(lds128(stage + (i * NT) * plane), x);
        unpack(lds128(stage + (i * NT + 1) * plane), dy);
#pragma unroll
        for (int e = 0; e < P; ++e)
          x[e] = __ffma2_rn(__fmul2_rn(dy[e], w[i][e]), rs, __ffma2_rn(__fadd2_rn(x[e], nm), c2, c1));
        if constexpr (RES) {
          if (has_h) {
            unpack(lds128(stage + (i * NT + 2) * plane), dy);
#pragma unroll
            for (int e = 0; e < P; ++e) x[e] = __fadd2_rn(x[e], dy[e]);
          }
          store_stream(dr + i * TPR, pack(x));
          drop_vec(a.drop, offset, vec + i * TPR, x);
        }
        store_stream(dx + i * TPR, pack(x));
      }
    }
    dx += step;
    if constexpr (RES) {
      dr += step;
      vec += step;
    }
    mean = next_mean;
    rstd = next_rstd;
    stage += row_bytes;
    if (stage == smem + STAGES * row_bytes) stage = smem;
  }
  cp_async_wait<0>();
  if (a.want == 0) return;
  // the block's partial row: the groups' sums through shared memory, added in order
  float* out = a.part + (size_t)blockIdx.x * 2 * a.C;
  float* sum = reinterpret_cast<float*>(ring);    // [2 * E][T]
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    __syncthreads();
#pragma unroll
    for (int e = 0; e < P; ++e) {
      sum[2 * e * T + tid] = dw[i][e].x;
      sum[(2 * e + 1) * T + tid] = dw[i][e].y;
      sum[(E + 2 * e) * T + tid] = db[i][e].x;
      sum[(E + 2 * e + 1) * T + tid] = db[i][e].y;
    }
    __syncthreads();
    for (int j = tid; j < TPR * 2 * E; j += T) {
      const int l = j % TPR, e = j / TPR, v = l + i * TPR;
      if (v >= a.nvec) continue;
      float t = 0.f;
#pragma unroll
      for (int q = 0; q < GROUPS; ++q) t += sum[e * T + q * TPR + l];
      out[(e >= E ? a.C : 0) + (size_t)v * E + e % E] = t;
    }
  }
}

// Rows of 65 to 128 vectors, a warp to a row and 16 rows side by side in the one block of an SM.  Each lane has
// VPT vectors, only the last of which may lie past the row, and keeps their dw and db for the block's whole
// run; W lies in shared memory.  No barrier until the block adds up its warps' parameter gradients.  120,000 x
// 1,000: 136 us, 153 with a block of two warps to a row; for 640 vectors five warps to a row in this manner are
// slower (824 us against 700 on 126,360 rows: three rows in flight on an SM do not cover the exchanges).
constexpr int kWarpRows = 16;
template <typename XT, int VPT, bool RES>
__global__ void __launch_bounds__(32 * kWarpRows, 1) norm_bwd_warp_kernel(const __grid_constant__ BwdArgs a) {
  constexpr int E = VecTraits<XT>::E, P = E / 2, Q = E / 4, NT = RES ? 3 : 2, STAGES = RES ? 2 : 3;
  constexpr int G = 32, GROUPS = kWarpRows, T = G * GROUPS;
  extern __shared__ __align__(16) uint4 ring[];
  const int tid = threadIdx.x, at = tid & 31, group = tid >> 5;
  int item, lo, run;
  block_run(a.tiers, blockIdx.x, item, lo, run);
  const size_t first = (size_t)item * a.rows + lo + group, at0 = first * a.nvec + at, step = (size_t)GROUPS * a.nvec;
  const bool whole = at + (VPT - 1) * G < a.nvec;
  auto has = [&](int i) { return i < VPT - 1 || whole; };
  float4* weights = reinterpret_cast<float4*>(ring + STAGES * NT * VPT * T);   // [Q][nvec]
  for (int v = tid; v < a.nvec; v += T) {
#pragma unroll
    for (int q = 0; q < Q; ++q)
      weights[q * a.nvec + v] = a.W != nullptr
                                    ? __ldg(reinterpret_cast<const float4*>(a.W + (size_t)item * a.param_stride + (size_t)v * E) + q)
                                    : make_float4(1.f, 1.f, 1.f, 1.f);
  }
  constexpr uint32_t plane = T * 16, row_bytes = plane * VPT * NT;
  const uint32_t smem = (uint32_t)__cvta_generic_to_shared(ring) + tid * 16;
  const bool has_h = RES && a.dH != nullptr;
  const uint4 *fx = a.X + at0, *fy = a.dY + at0, *fh = has_h ? a.dH + at0 : nullptr;
  uint32_t fstage = smem;
  int fetched = group;
  auto fetch = [&]() {
    if (fetched < run) {
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        if (has(i)) {
          cp_async16(fstage + (i * NT) * plane, fx + i * G);
          cp_async16(fstage + (i * NT + 1) * plane, fy + i * G);
          if (has_h) cp_async16(fstage + (i * NT + 2) * plane, fh + i * G);
        }
      }
    }
    cp_async_commit();
    fetched += GROUPS;
    fx += step;
    fy += step;
    if (has_h) fh += step;
    fstage += row_bytes;
    if (fstage == smem + STAGES * row_bytes) fstage = smem;
  };
#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) fetch();
  float2 dw[VPT][P], db[VPT][P];
#pragma unroll
  for (int i = 0; i < VPT; ++i)
#pragma unroll
    for (int e = 0; e < P; ++e) dw[i][e] = db[i][e] = both(0.f);
  const uint64_t offset = RES ? drop_offset(a.drop) : 0;
  const float inv_c = 1.f / (float)a.C;
  const float *pm = a.mean + first, *pr = a.rstd + first;
  float mean = group < run ? __ldg(pm) : 0.f, rstd = group < run ? __ldg(pr) : 0.f;
  uint4 *dx = a.dX + at0, *dr = RES ? a.dR + at0 : nullptr;
  uint64_t vec = at0;
  uint32_t stage = smem;
  __syncthreads();                                // the weights are there
  auto weight = [&](int i, float2 (&w)[P]) {
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const float4 u = weights[q * a.nvec + at + i * G];
      w[2 * q] = make_float2(u.x, u.y), w[2 * q + 1] = make_float2(u.z, u.w);
    }
  };
  for (int row = group; row < run; row += GROUPS) {
    fetch();
    cp_async_wait<STAGES - 1>();
    pm += GROUPS;
    pr += GROUPS;
    const float next_mean = row + GROUPS < run ? __ldg(pm) : 0.f, next_rstd = row + GROUPS < run ? __ldg(pr) : 0.f;
    float2 t1 = both(0.f), t2 = both(0.f);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      if (has(i)) {
        float2 x[P], dy[P], w[P];
        unpack(lds128(stage + (i * NT) * plane), x);
        unpack(lds128(stage + (i * NT + 1) * plane), dy);
        weight(i, w);
#pragma unroll
        for (int e = 0; e < P; ++e) {
          // dw is fp32 for bf16 rows too, so the difference is taken first here
          const float2 p = __fmul2_rn(dy[e], __fmul2_rn(__fadd2_rn(x[e], both(-mean)), both(rstd)));
          dw[i][e] = __fadd2_rn(dw[i][e], p);
          db[i][e] = __fadd2_rn(db[i][e], dy[e]);
          t1 = __ffma2_rn(dy[e], w[e], t1);
          t2 = __ffma2_rn(p, w[e], t2);
        }
      }
    }
    const float s1 = lanes_sum<32>(t1.x + t1.y), s2 = lanes_sum<32>(t2.x + t2.y);
    __syncwarp();                                 // keeps the two halves of the row apart, or registers run out
    // r (g - c1 - xh c2) = r g + (x - m) (-r^2 c2) - r c1
    const float slope = -rstd * rstd * (s2 * inv_c), shift = -rstd * (s1 * inv_c);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      if (has(i)) {
        float2 x[P], dy[P], w[P];
        unpack(lds128(stage + (i * NT) * plane), x);
        unpack(lds128(stage + (i * NT + 1) * plane), dy);
        weight(i, w);
#pragma unroll
        for (int e = 0; e < P; ++e) {
          float2 t;
          if constexpr (E == 8) t = __ffma2_rn(x[e], both(slope), both(fmaf(-mean, slope, shift)));
          else t = __ffma2_rn(__fadd2_rn(x[e], both(-mean)), both(slope), both(shift));
          x[e] = __ffma2_rn(__fmul2_rn(dy[e], w[e]), both(rstd), t);
        }
        if constexpr (RES) {
          if (has_h) {
            unpack(lds128(stage + (i * NT + 2) * plane), dy);
#pragma unroll
            for (int e = 0; e < P; ++e) x[e] = __fadd2_rn(x[e], dy[e]);
          }
          store_stream(dr + i * G, pack(x));
          drop_vec(a.drop, offset, vec + i * G, x);
        }
        store_stream(dx + i * G, pack(x));
      }
    }
    dx += step;
    if constexpr (RES) {
      dr += step;
      vec += step;
    }
    mean = next_mean;
    rstd = next_rstd;
    stage += row_bytes;
    if (stage == smem + STAGES * row_bytes) stage = smem;
  }
  cp_async_wait<0>();
  if (a.want == 0) return;
  // the block's partial row: the groups' sums through the ring, added in order
  float2* sum = reinterpret_cast<float2*>(ring);  // [GROUPS][2][P][nvec]
  __syncthreads();
#pragma unroll
  for (int i = 0; i < VPT; ++i)
    if (has(i)) {
#pragma unroll
      for (int e = 0; e < P; ++e) {
        sum[((group * 2) * P + e) * a.nvec + at + i * G] = dw[i][e];
        sum[((group * 2 + 1) * P + e) * a.nvec + at + i * G] = db[i][e];
      }
    }
  __syncthreads();
  float2* out = reinterpret_cast<float2*>(a.part + (size_t)blockIdx.x * 2 * a.C);
  for (int v = tid; v < a.nvec; v += T)
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int e = 0; e < P; ++e) {
        float2 t = both(0.f);
#pragma unroll
        for (int q = 0; q < GROUPS; ++q) t = __fadd2_rn(t, sum[((q * 2 + k) * P + e) * a.nvec + v]);
        out[(size_t)k * (a.C / 2) + (size_t)v * P + e] = t;
      }
}

// Longer rows, a block to a row: only the last of a thread's VPT vectors may lie past the row (blockDim <=
// nvec <= blockDim VPT; none with EVEN), and ROWS rows cost one barrier.  Two rows a barrier measured 0.67 ms on
// 126,360 x 5,120, one row 0.71 with a ring of the same bytes; at full clocks both take 0.61, 6.4 TB/s.
template <typename XT, int VPT, bool EVEN, bool RES, int ROWS, int STAGES, int MAXT, int MINB>
__global__ void __launch_bounds__(MAXT, MINB) norm_bwd_row_kernel(const __grid_constant__ BwdArgs a) {
  constexpr int E = VecTraits<XT>::E, P = E / 2, NT = RES ? 3 : 2;
  extern __shared__ __align__(16) uint4 ring[];
  __shared__ float red[2][2 * ROWS * 32];
  const int T = blockDim.x, tid = threadIdx.x, warps = T >> 5;
  int item, lo, run;
  block_run(a.tiers, blockIdx.x, item, lo, run);
  const size_t first = (size_t)item * a.rows + lo, at0 = first * a.nvec + tid;
  const bool whole = EVEN || tid + (VPT - 1) * T < a.nvec;          // all VPT vectors are the row's
  auto has = [&](int i) { return i < VPT - 1 || whole; };
  const uint32_t plane = T * 16, row_bytes = plane * VPT * NT, stage_bytes = row_bytes * ROWS;
  const uint32_t smem = (uint32_t)__cvta_generic_to_shared(ring) + tid * 16;
  const bool has_h = RES && a.dH != nullptr;
  const uint4 *fx = a.X + at0, *fy = a.dY + at0, *fh = has_h ? a.dH + at0 : nullptr;
  uint32_t fstage = smem;
  int fetched = 0;                                // rows asked for so far
  auto fetch = [&]() {
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (fetched + r < run) {
        const uint32_t to = fstage + r * row_bytes;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
          if (has(i)) {
            cp_async16(to + (i * NT) * plane, fx + (size_t)r * a.nvec + i * T);
            cp_async16(to + (i * NT + 1) * plane, fy + (size_t)r * a.nvec + i * T);
            if (has_h) cp_async16(to + (i * NT + 2) * plane, fh + (size_t)r * a.nvec + i * T);
          }
        }
      }
    }
    cp_async_commit();
    fetched += ROWS;
    fx += ROWS * a.nvec;
    fy += ROWS * a.nvec;
    if (has_h) fh += ROWS * a.nvec;
    fstage += stage_bytes;
    if (fstage == smem + STAGES * stage_bytes) fstage = smem;
  };
#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) fetch();
  float2 w[VPT][P], dw[VPT][P], db[VPT][P];
#pragma unroll
  for (int i = 0; i < VPT; ++i)
#pragma unroll
    for (int e = 0; e < P; ++e) {
      dw[i][e] = db[i][e] = both(0.f);
      const size_t c = (size_t)item * a.param_stride + (size_t)(tid + i * T) * E;
      w[i][e] = both(1.f);
      if (a.W != nullptr && has(i)) w[i][e] = __ldg(reinterpret_cast<const float2*>(a.W + c) + e);
    }
  const uint64_t offset = RES ? drop_offset(a.drop) : 0;
  const float inv_c = 1.f / (float)a.C;
  const float *pm = a.mean + first, *pr = a.rstd + first;
  float mean[ROWS], rstd[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    mean[r] = r < run ? __ldg(pm + r) : 0.f;
    rstd[r] = r < run ? __ldg(pr + r) : 0.f;
  }
  uint4 *dx = a.dX + at0, *dr = RES ? a.dR + at0 : nullptr;
  uint64_t vec = at0;
  uint32_t stage = smem;
  int buf = 0;
  for (int row = 0; row < run; row += ROWS) {
    fetch();
    cp_async_wait<STAGES - 1>();
    float next_mean[ROWS], next_rstd[ROWS], v[2 * ROWS];
    pm += ROWS;
    pr += ROWS;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      next_mean[r] = row + ROWS + r < run ? __ldg(pm + r) : 0.f;
      next_rstd[r] = row + ROWS + r < run ? __ldg(pr + r) : 0.f;
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      float2 t1 = both(0.f), t2 = both(0.f);
      if (ROWS == 1 || row + r < run) {           // the same for the whole block
        const float2 nm = both(-mean[r]), rs = both(rstd[r]);
        const uint32_t from = stage + r * row_bytes;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
          if (has(i)) {
            float2 x[P], dy[P];
            unpack(lds128(from + (i * NT) * plane), x);
            unpack(lds128(from + (i * NT + 1) * plane), dy);
#pragma unroll
            for (int e = 0; e < P; ++e) {
              const float2 xh = __fmul2_rn(__fadd2_rn(x[e], nm), rs), g = __fmul2_rn(dy[e], w[i][e]);
              dw[i][e] = __ffma2_rn(dy[e], xh, dw[i][e]);
              db[i][e] = __fadd2_rn(db[i][e], dy[e]);
              t1 = __fadd2_rn(t1, g);
              t2 = __ffma2_rn(g, xh, t2);
            }
          }
        }
      }
      v[2 * r] = t1.x + t1.y;
      v[2 * r + 1] = t2.x + t2.y;
    }
    block_sums<2 * ROWS, warp_lanes(MAXT)>(v, red[buf], warps);
    buf ^= 1;                                     // the next barrier comes before this half is written again
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (ROWS == 1 || row + r < run) {
        // r (g - c1 - xh c2) = r g + (x - m) slope + shift, slope = -r^2 c2, shift = -r c1
        const float slope = -rstd[r] * rstd[r] * (v[2 * r + 1] * inv_c), shift = -rstd[r] * (v[2 * r] * inv_c);
        const float2 rs = both(rstd[r]), sl = both(slope), nm = both(-mean[r]),
                     sh = both(E == 8 ? fmaf(-mean[r], slope, shift) : shift);
        const uint32_t from = stage + r * row_bytes;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
          if (has(i)) {
            float2 x[P], dy[P];
            unpack(lds128(from + (i * NT) * plane), x);
            unpack(lds128(from + (i * NT + 1) * plane), dy);
#pragma unroll
            for (int e = 0; e < P; ++e) {
              // bf16 results have eight bits, so x slope + (shift - m slope) is exact enough there
              const float2 t = __ffma2_rn(E == 8 ? x[e] : __fadd2_rn(x[e], nm), sl, sh);
              x[e] = __ffma2_rn(__fmul2_rn(dy[e], w[i][e]), rs, t);
            }
            if constexpr (RES) {
              if (has_h) {
                unpack(lds128(from + (i * NT + 2) * plane), dy);
#pragma unroll
                for (int e = 0; e < P; ++e) x[e] = __fadd2_rn(x[e], dy[e]);
              }
              store_stream(dr + i * T, pack(x));
              drop_vec(a.drop, offset, vec + i * T, x);
            }
            store_stream(dx + i * T, pack(x));
          }
        }
      }
      dx += a.nvec;
      if constexpr (RES) {
        dr += a.nvec;
        vec += a.nvec;
      }
      mean[r] = next_mean[r];
      rstd[r] = next_rstd[r];
    }
    stage += stage_bytes;
    if (stage == smem + STAGES * stage_bytes) stage = smem;
  }
  cp_async_wait<0>();
  if (a.want == 0) return;
  float* out = a.part + (size_t)blockIdx.x * 2 * a.C + (size_t)tid * E;
#pragma unroll
  for (int i = 0; i < VPT; ++i)
    if (has(i)) {
#pragma unroll
      for (int e = 0; e < P; ++e) {
        reinterpret_cast<float2*>(out + (size_t)i * T * E)[e] = dw[i][e];
        reinterpret_cast<float2*>(out + a.C + (size_t)i * T * E)[e] = db[i][e];
      }
    }
}

// dW[p, c] = sum of the partial rows of item p, in 64 bits and in a fixed order.  The rows of an item are
// `blocks` neighbours in each of `tiers` tiers of items * blocks.  32 channels to a block, eight threads by
// four of them, 32 such sets of threads down the partial rows.
// grid: (ceil(C / 32), 2, items), block (8, 32).
__global__ void __launch_bounds__(256) norm_reduce_kernel(const float* __restrict__ part, int tiers, int blocks, int C,
                                                          float* dW, float* dbias) {
  __shared__ double sum[32][33];
  float* out = blockIdx.y == 0 ? dW : dbias;
  if (out == nullptr) return;
  const int c = blockIdx.x * 32 + threadIdx.x * 4, n = tiers * blocks;
  const size_t row = 2 * (size_t)C, jump = (size_t)(gridDim.z - 1) * blocks;   // partial rows between an item's tiers
  const float* p = part + (size_t)blockIdx.z * blocks * row + (size_t)blockIdx.y * C + c;
  double t[4] = {0.0, 0.0, 0.0, 0.0};
  if (c < C) {
    constexpr int U = 10;                         // loads in flight: 320 partial rows in one go
    for (int q0 = threadIdx.y; q0 < n; q0 += 32 * U) {
      float4 x[U];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int q = q0 + 32 * i;
        x[i] = q < n ? __ldg(reinterpret_cast<const float4*>(p + (q + (tiers > 1 ? q / blocks * jump : 0)) * row))
                     : make_float4(0.f, 0.f, 0.f, 0.f);
      }
#pragma unroll
      for (int i = 0; i < U; ++i) t[0] += (double)x[i].x, t[1] += (double)x[i].y, t[2] += (double)x[i].z, t[3] += (double)x[i].w;
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) sum[threadIdx.y][threadIdx.x * 4 + i] = t[i];
  __syncthreads();
  const int tid = threadIdx.y * 8 + threadIdx.x, mine = tid >> 3, slice = tid & 7;   // eight threads add a channel's 32
  double s = 0.0;
#pragma unroll
  for (int q = 0; q < 4; ++q) s += sum[slice * 4 + q][mine];
#pragma unroll
  for (int o = 1; o < 8; o *= 2) s += __shfl_xor_sync(0xffffffffu, s, o);
  const int ch = blockIdx.x * 32 + mine;
  if (slice == 0 && ch < C) out[(size_t)blockIdx.z * C + ch] = (float)s;
}

// How the backward splits a problem: the same on the host that sizes the workspace and the one that launches.
struct BwdPlan {
  int tpr, threads, vpt;
  long long rows;
  Tiers tiers;
  int blocks() const { return tiers.items * tiers.blocks * tiers.count; }
};
BwdPlan bwd_plan(const moga_shape& s, bool per_batch) {
  BwdPlan p{};
  const int items = per_batch ? s.B : 1;
  p.rows = per_batch ? (long long)s.N : (long long)s.B * s.N;
  const int nvec = (int)((size_t)s.C * elem_size(s.dtype) / 16);
  p.vpt = nvec <= 32 ? 1 : nvec <= 1280 ? 2 : 4;
  if (nvec <= 64) {                               // short rows: groups of threads side by side in a block
    p.tpr = nvec <= 8 ? 8 : nvec <= 16 ? 16 : 32;
    p.threads = kGroupThreads;
  } else if (nvec <= 128) {                       // a warp to a row
    p.vpt = nvec <= 96 ? 3 : 4;
    p.tpr = 32;
    p.threads = 32 * kWarpRows;
  } else {
    p.tpr = p.threads = (int)align_up((nvec + p.vpt - 1) / p.vpt, 32);
  }
  // blocks: one to an SM where a block has W in shared memory, else as many as make up 640 threads (two at least);
  // at least four rows for each group of threads, and no partial sum over more than 512 rows of a thread.  The
  // workspace size, which both forms share and which no CUDA call may be made for, fixes these counts, so they do
  // not follow what fits an SM in every form: of five blocks of 128 threads four do with the residual (1,544 - 2,048
  // bf16 channels; 50,000 x 2,048: 212 us, 4.8 TB/s), of two of more than 320 threads one does (fp32, 20,000 x 5,120:
  // 199 us, 6.2 TB/s); the others start as those end.
  // Equal runs: a partial row costs as much traffic as three rows, more than shorter runs at the end would level
  // (126,360 x 5,120: 0.65 ms at full clocks with them, 0.61 without).
  const int groups = p.threads / p.tpr;
  const int per_sm = nvec > 64 && nvec <= 128 ? 1 : 640 / p.threads < 2 ? 2 : 640 / p.threads;
  long long resident = 148ll * per_sm, most = (p.rows * items + 4 * groups - 1) / (4 * groups);
  resident = resident > most ? most : resident;
  p.tiers = make_tiers(p.rows, items, (int)(resident < 1 ? 1 : resident), 512 * groups, 1 << 20);
  return p;
}

template <typename XT, int TPR, int VPT, bool RES>
moga_status run_bwd_groups(const BwdArgs& a, const BwdPlan& p, cudaStream_t st) {
  auto kernel = norm_bwd_group_kernel<XT, TPR, VPT, RES>;
  // the ring, which also holds the sum of the groups
  const int ring = kGroupStages * VPT * (RES ? 3 : 2) * kGroupThreads * 16;
  const int merge = kGroupThreads * 2 * VecTraits<XT>::E * (int)sizeof(float), smem = ring > merge ? ring : merge;
  if (smem > 40 * 1024) MOGA_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  kernel<<<p.blocks(), kGroupThreads, smem, st>>>(a);
  MOGA_CUDA_OK(cudaGetLastError());
  return MOGA_OK;
}

template <typename XT, int VPT, bool RES>
moga_status run_bwd_warps(const BwdArgs& a, const BwdPlan& p, cudaStream_t st) {
  auto kernel = norm_bwd_warp_kernel<XT, VPT, RES>;
  // the ring (2 tensors x 3 stages, or 3 x 2) and W, or the sum of the warps
  const int ring = 6 * VPT * p.threads * 16 + a.C * (int)sizeof(float), sums = kWarpRows * 2 * a.C * (int)sizeof(float);
  const int smem = ring > sums ? ring : sums;
  MOGA_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  kernel<<<p.blocks(), p.threads, smem, st>>>(a);
  MOGA_CUDA_OK(cudaGetLastError());
  return MOGA_OK;
}

template <typename XT, int VPT, bool EVEN, bool RES, int ROWS, int STAGES, int MAXT, int MINB>
moga_status run_bwd_rows(const BwdArgs& a, const BwdPlan& p, cudaStream_t st) {
  auto kernel = norm_bwd_row_kernel<XT, VPT, EVEN, RES, ROWS, STAGES, MAXT, MINB>;
  const int smem = STAGES * ROWS * VPT * (RES ? 3 : 2) * p.threads * 16;
  if (smem > 40 * 1024) MOGA_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  kernel<<<p.blocks(), p.threads, smem, st>>>(a);
  MOGA_CUDA_OK(cudaGetLastError());
  return MOGA_OK;
}
template <typename XT, bool RES, int ROWS, int STAGES, int MAXT, int MINB>
moga_status run_bwd_even(const BwdArgs& a, const BwdPlan& p, cudaStream_t st) {
  return a.nvec == 2 * p.threads ? run_bwd_rows<XT, 2, true, RES, ROWS, STAGES, MAXT, MINB>(a, p, st)
                                 : run_bwd_rows<XT, 2, false, RES, ROWS, STAGES, MAXT, MINB>(a, p, st);
}

template <typename XT, bool RES>
moga_status dispatch_bwd(const BwdArgs& a, const BwdPlan& p, cudaStream_t st) {
  if (p.tpr == 8) return run_bwd_groups<XT, 8, 1, RES>(a, p, st);
  if (p.tpr == 16) return run_bwd_groups<XT, 16, 1, RES>(a, p, st);
  if (p.threads == 32 * kWarpRows && p.tpr == 32)
    return p.vpt == 3 ? run_bwd_warps<XT, 3, RES>(a, p, st) : run_bwd_warps<XT, 4, RES>(a, p, st);
  if (p.tpr < p.threads)
    return p.vpt == 1 ? run_bwd_groups<XT, 32, 1, RES>(a, p, st) : run_bwd_groups<XT, 32, 2, RES>(a, p, st);
  // Two rows to a barrier where two rings of two stages fit an SM's 227 KB beside each other
  if (p.vpt == 4) return run_bwd_rows<XT, 4, false, RES, 1, RES ? 2 : 3, 512, 1>(a, p, st);
  if (p.threads <= 128) return run_bwd_even<XT, RES, 2, 2, 128, 5>(a, p, st);
  if (p.threads > 320) return run_bwd_even<XT, RES, 1, RES ? 2 : 3, 640, 1>(a, p, st);
  if constexpr (RES) return run_bwd_even<XT, RES, 1, 2, 320, 2>(a, p, st);
  else return run_bwd_even<XT, RES, 2, 2, 320, 2>(a, p, st);
}

}  // namespace

size_t norm_backward_bytes(const moga_shape& s, const moga_norm& n) {
  const BwdPlan p = bwd_plan(s, n.per_batch != 0);
  return align_up(256 + sizeof(float) * 2 * (size_t)s.C * p.blocks(), kWsAlign);
}

static DropArgs drop_args(const moga_dropout* d) {
  DropArgs a{};
  a.scale = 1.f;
  if (d != nullptr) {
    for (uint32_t r = 0; r < 10; ++r) {
      a.key[2 * r] = (uint32_t)d->seed + r * 0x9E3779B9u;
      a.key[2 * r + 1] = (uint32_t)(d->seed >> 32) + r * 0xBB67AE85u;
    }
    a.offset = d->offset;
    a.step = d->step;
    const double t = d->p * 65536.0 + 0.5;
    a.threshold = t >= 65535.0 ? 65535u : (uint32_t)t;
    a.scale = 65536.f / (float)(65536u - a.threshold);
  }
  return a;
}

moga_status launch_norm(const moga_shape& s, const moga_norm& n, const moga_dropout* d, const void* X, const void* R,
                        const float* W, const float* bias, void* Hout, void* Y, float* mean, float* rstd,
                        cudaStream_t st) {
  FwdArgs a{};
  a.X = X;
  a.R = R;
  a.W = W;
  a.bias = bias;
  a.Hout = Hout;
  a.Y = Y;
  a.mean = mean;
  a.rstd = rstd;
  a.rows = n.per_batch ? (long long)s.N : (long long)s.B * s.N;
  a.C = s.C;
  a.nvec = (int)((size_t)s.C * elem_size(s.dtype) / 16);
  a.param_stride = n.per_batch ? s.C : 0;
  a.eps = n.eps;
  a.drop = drop_args(d);
  const int items = n.per_batch ? s.B : 1;
  if (s.dtype == MOGA_BF16)
    return R != nullptr ? dispatch_fwd<__nv_bfloat16, true>(a, items, st) : dispatch_fwd<__nv_bfloat16, false>(a, items, st);
  return R != nullptr ? dispatch_fwd<float, true>(a, items, st) : dispatch_fwd<float, false>(a, items, st);
}

moga_status launch_norm_backward(const moga_shape& s, const moga_norm& n, const moga_dropout* d, const void* X,
                                 const float* W, const float* mean, const float* rstd, const void* dY, const void* dH,
                                 void* dX, void* dR, float* dW, float* dbias, char* ws, cudaStream_t st) {
  const BwdPlan p = bwd_plan(s, n.per_batch != 0);
  BwdArgs a{};
  a.X = static_cast<const uint4*>(X);
  a.dY = static_cast<const uint4*>(dY);
  a.dH = static_cast<const uint4*>(dH);
  a.W = W;
  a.mean = mean;
  a.rstd = rstd;
  a.dX = static_cast<uint4*>(dX);
  a.dR = static_cast<uint4*>(dR);
  a.part = reinterpret_cast<float*>(ws + 256);
  a.rows = p.rows;
  a.C = s.C;
  a.nvec = (int)((size_t)s.C * elem_size(s.dtype) / 16);
  a.param_stride = n.per_batch ? s.C : 0;
  a.tiers = p.tiers;
  a.want = (dW != nullptr ? 1 : 0) | (dbias != nullptr ? 2 : 0);
  a.drop = drop_args(d);
  moga_status r;
  if (s.dtype == MOGA_BF16)
    r = dR != nullptr ? dispatch_bwd<__nv_bfloat16, true>(a, p, st) : dispatch_bwd<__nv_bfloat16, false>(a, p, st);
  else
    r = dR != nullptr ? dispatch_bwd<float, true>(a, p, st) : dispatch_bwd<float, false>(a, p, st);
  if (r != MOGA_OK || a.want == 0) return r;
  norm_reduce_kernel<<<dim3((s.C + 31) / 32, 2, p.tiers.items), dim3(8, 32), 0, st>>>(a.part, p.tiers.count, p.tiers.blocks,
                                                                                         s.C, dW, dbias);
  MOGA_CUDA_OK(cudaGetLastError());
  return MOGA_OK;
}

// ---------------------------------------------------------------- dropout with a residual
namespace {

constexpr int kDropThreads = 256;
constexpr int kDropUnits = 4;     // units of eight elements in flight per thread

// Y = R + keep X scale, eight elements (one generator call) at a time.  HBM-bound: the generator's forty integer
// operations for eight elements fit under the 32 to 48 bytes they move (126,360 x 5,120 bf16 with the residual:
// 0.56 - 0.59 ms, 6.6 - 6.9 TB/s; fp32, 20,000 x 5,120: 176 us, 7.0 TB/s, and without the residual 131 us, 6.3 TB/s).
template <typename XT, bool RES>
__global__ void __launch_bounds__(kDropThreads) dropout_kernel(const uint4* X, const uint4* R, uint4* Y, uint64_t nvec,
                                                               const __grid_constant__ DropArgs d) {
  constexpr int E = VecTraits<XT>::E, P = E / 2, V = 8 / E;    // 16-byte vectors of a unit
  const uint64_t offset = drop_offset(d);
  const uint64_t first = (uint64_t)blockIdx.x * kDropThreads * kDropUnits + threadIdx.x;
  uint4 x[kDropUnits][V], r[kDropUnits][V];
#pragma unroll
  for (int i = 0; i < kDropUnits; ++i)
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const uint64_t v = (first + i * kDropThreads) * V + j;
      if (v < nvec) {
        x[i][j] = load_stream(X + v);
        if (RES) r[i][j] = load_stream(R + v);
      }
    }
#pragma unroll
  for (int i = 0; i < kDropUnits; ++i) {
    const uint64_t unit = first + i * kDropThreads;
    if (unit * V >= nvec) continue;
    uint4 bits = make_uint4(0, 0, 0, 0);
    if (d.threshold != 0) bits = philox(d, unit, offset);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if (unit * V + j >= nvec) continue;
      float2 f[P];
      unpack(x[i][j], f);
      if (d.threshold != 0) {
        if constexpr (E == 8) drop_bits(d, bits, f);
        else drop_bits(d, j ? bits.z : bits.x, j ? bits.w : bits.y, f);
      }
      if constexpr (RES) {
        float2 g[P];
        unpack(r[i][j], g);
#pragma unroll
        for (int e = 0; e < P; ++e) f[e] = __fadd2_rn(f[e], g[e]);
      }
      store_stream(Y + unit * V + j, pack(f));
    }
  }
}

template <typename XT>
moga_status run_dropout(const void* X, const void* R, void* Y, uint64_t nvec, const DropArgs& d, cudaStream_t st) {
  constexpr uint64_t per_block = (uint64_t)kDropThreads * kDropUnits * (8 / VecTraits<XT>::E);
  const uint64_t blocks = (nvec + per_block - 1) / per_block;
  if (blocks > 0x7fffffffull) return MOGA_ERR_UNSUPPORTED;
  const uint4 *x = static_cast<const uint4*>(X), *r = static_cast<const uint4*>(R);
  if (R != nullptr)
    dropout_kernel<XT, true><<<(unsigned)blocks, kDropThreads, 0, st>>>(x, r, static_cast<uint4*>(Y), nvec, d);
  else
    dropout_kernel<XT, false><<<(unsigned)blocks, kDropThreads, 0, st>>>(x, r, static_cast<uint4*>(Y), nvec, d);
  MOGA_CUDA_OK(cudaGetLastError());
  return MOGA_OK;
}

}  // namespace

moga_status launch_dropout(const moga_shape& s, const moga_dropout& d, const void* X, const void* R, void* Y,
                           cudaStream_t st) {
  const uint64_t nvec = (uint64_t)s.B * s.N * ((uint64_t)s.C * elem_size(s.dtype) / 16);
  return s.dtype == MOGA_BF16 ? run_dropout<__nv_bfloat16>(X, R, Y, nvec, drop_args(&d), st)
                              : run_dropout<float>(X, R, Y, nvec, drop_args(&d), st);
}

}  // namespace moga
