// Norms of queries and keys for each head with the position rotation in the same pass, and its gradient.
//
//   forward   y = R(t) (x r w),  r = 1 / sqrt(mean(x^2) + eps)
//   gradient  g = R(-t) dy;  dw = sum over rows of g x r;  u = g w;  dx = r (u - x r mean(u x r))
//
// Bound: reading x (and dy) and writing y (dx) once. A workgroup takes 64 (d = 64) or 32 rows of a few heads of queries or of
// keys: the rotation's angles, as many bytes as a bf16 row, are loaded once for all of them, and all their rows are asked
// for before the first is worked on. Weight gradients are summed over a workgroup's rows in registers and LDS, then over workgroups by
// a second kernel: no atomics.
// Measured, us: B1 N4096 H32 Hkv8 d64 bf16 forward 10.5 (42 MB, launch and ramp 2-3 of it); B4 N8192 H16 Hkv16 d128 bf16 forward and gradient 252
// (5.35 TB/s); N2047 H8 Hkv8 d64 float, a weight a head, 18 (7.0, 8.5 and the weights' sums 2.5); 64 single tokens, a kernel of 3.5.
#include "paged.h"
#include "token_rows.h"

namespace da {

namespace {

constexpr int kRowThreads = 256;

struct HeadsOf {   // one of the two tensors
  const void* x;
  const void* g;       // gradient: dy
  void* y;             // forward: y, gradient: dx
  int heads;
  int64_t x_stride[3], g_stride[3], y_stride[3];
  const void* weight;
};
struct QkArgs {
  HeadsOf t[2];        // queries, keys
  int N, rows;         // rows of a head in a batch, in all of them
  int chunk, chunks_q; // heads of a workgroup, workgroups for the query heads of the same rows
  Rotary r;
  const int* positions;
};

template <typename E, int D, int ROPE, int HC, bool ONCE>
__global__ __launch_bounds__(kRowThreads) void qk_forward_kernel(const QkArgs a, int chunks) {
  constexpr int LPR = D / 16;
  const int chunk = blockIdx.x % chunks;
  const bool keys = chunk >= a.chunks_q;
  const HeadsOf& t = a.t[keys];
  const int h0 = (keys ? chunk - a.chunks_q : chunk) * HC;
  const int row = blockIdx.x / chunks * (kRowThreads / LPR) + threadIdx.x / LPR;
  const int row_ld = min(row, a.rows - 1);   // (surplus rows: a valid one, never stored)
  const LanePlace<ROPE> at(threadIdx.x % LPR, a.r.rot_dim);
  const int b = row_ld / a.N, n = row_ld % a.N;
  const E* x = (const E*)t.x + b * t.x_stride[0] + n * t.x_stride[2];
  E* y = (E*)t.y + b * t.y_stride[0] + n * t.y_stride[2];
  Eight<E> lo[HC], hi[HC];
#pragma unroll
  for (int i = 0; i < HC; ++i) {
    const E* p = x + min(h0 + i, t.heads - 1) * t.x_stride[1];
    lo[i].template load<ONCE>(p + at.lo);
    hi[i].template load<ONCE>(p + at.hi);
  }
  Angles angles;
  angles.load(a.r, a.positions ? a.positions[row_ld] : n, at.pair, at.turn);
  float w[16];
  if (a.r.norm && !a.r.weight_heads) load_weight<D>(w, t.weight, a.r, 0, at);
#pragma unroll
  for (int i = 0; i < HC; ++i) {
    if (h0 + i >= t.heads) break;
    float v[16];
    lo[i].values(v);
    hi[i].values(v + 8);
    if (a.r.norm) {
      if (a.r.weight_heads) load_weight<D>(w, t.weight, a.r, h0 + i, at);
      const float r = inverse_rms<LPR>(v, a.r.eps);
#pragma unroll
      for (int j = 0; j < 16; ++j) v[j] = v[j] * r * w[j];
    }
    if (at.turn) rotate<ROPE, 1>(v, angles);
    if (row < a.rows) {
      E* p = y + (h0 + i) * t.y_stride[1];
      Eight<E>::template store<ONCE>(p + at.lo, v);
      Eight<E>::template store<ONCE>(p + at.hi, v + 8);
    }
  }
}

// part: [chunks][gridDim.x / chunks][D] sums of a workgroup's rows, null where no weight gradient is asked for
template <typename E, int D, int ROPE, bool ONCE>
__global__ __launch_bounds__(kRowThreads) void qk_backward_kernel(const QkArgs a, int chunks, float* part) {
  constexpr int LPR = D / 16, ROWS = kRowThreads / LPR;
  const int chunk = blockIdx.x % chunks, group = blockIdx.x / chunks, groups = gridDim.x / chunks;
  const bool keys = chunk >= a.chunks_q;
  const HeadsOf& t = a.t[keys];
  const int h0 = (keys ? chunk - a.chunks_q : chunk) * a.chunk, h1 = min(h0 + a.chunk, t.heads);
  const LanePlace<ROPE> at(threadIdx.x % LPR, a.r.rot_dim);
  float w[16], dw[16];
#pragma unroll
  for (int j = 0; j < 16; ++j) dw[j] = 0.0f;
  if (a.r.norm) load_weight<D>(w, t.weight, a.r, h0, at);   // (a weight for each head: the chunk is one head)
  for (int r0 = group * ROWS; r0 < a.rows; r0 += groups * ROWS) {
    const int row = r0 + threadIdx.x / LPR, row_ld = min(row, a.rows - 1);
    const int b = row_ld / a.N, n = row_ld % a.N;
    const E* x = (const E*)t.x + b * t.x_stride[0] + n * t.x_stride[2];
    const E* g = (const E*)t.g + b * t.g_stride[0] + n * t.g_stride[2];
    E* y = (E*)t.y + b * t.y_stride[0] + n * t.y_stride[2];
    Angles angles;
    angles.load(a.r, a.positions ? a.positions[row_ld] : n, at.pair, at.turn);
    for (int64_t h = h0; h < h1; ++h) {
      Eight<E> xl, xh, gl, gh;
      gl.template load<ONCE>(g + h * t.g_stride[1] + at.lo);
      gh.template load<ONCE>(g + h * t.g_stride[1] + at.hi);
      if (a.r.norm) {
        xl.template load<ONCE>(x + h * t.x_stride[1] + at.lo);
        xh.template load<ONCE>(x + h * t.x_stride[1] + at.hi);
      }
      float u[16];
      gl.values(u);
      gh.values(u + 8);
      if (at.turn) rotate<ROPE, -1>(u, angles);
      if (a.r.norm) {
        float v[16];
        xl.values(v);
        xh.values(v + 8);
        const float r = inverse_rms<LPR>(v, a.r.eps);
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          v[j] *= r;
          if (row < a.rows) dw[j] = __builtin_fmaf(u[j], v[j], dw[j]);
          u[j] *= w[j];
          s = __builtin_fmaf(u[j], v[j], s);
        }
        s = row_sum<LPR>(s) * (1.0f / D);
#pragma unroll
        for (int j = 0; j < 16; ++j) u[j] = r * __builtin_fmaf(-s, v[j], u[j]);
      }
      if (row < a.rows) {
        E* p = y + h * t.y_stride[1];
        Eight<E>::template store<ONCE>(p + at.lo, u);
        Eight<E>::template store<ONCE>(p + at.hi, u + 8);
      }
    }
  }
  if (part == nullptr) return;
  __shared__ float sums[ROWS][D + 4];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    sums[threadIdx.x / LPR][at.lo + j] = dw[j];
    sums[threadIdx.x / LPR][at.hi + j] = dw[8 + j];
  }
  __syncthreads();
  if (threadIdx.x < D) {
    float s = 0.0f;
#pragma unroll 8
    for (int i = 0; i < ROWS; ++i) s += sums[i][threadIdx.x];
    part[((size_t)chunk * groups + group) * D + threadIdx.x] = s;
  }
}

// One workgroup sums eight channels of one weight: over the `n` rows of part from row `first` on.
struct WeightSums {
  const float* part;
  float* out[2];
  int weights[2];      // weights of the tensor (1, or one for each head)
  int first[2], n[2];  // part rows of its first weight, of each of its weights
  int d;
};
__global__ __launch_bounds__(256) void qk_weight_kernel(const WeightSums a) {
  const int pieces = a.d / 8;
  int id = blockIdx.x / pieces;
  const int c = blockIdx.x % pieces * 8 + (threadIdx.x & 7);
  const int of = id >= a.weights[0] ? 1 : 0;
  id -= of ? a.weights[0] : 0;
  if (a.out[of] == nullptr) return;
  const float* p = a.part + (size_t)(a.first[of] + id * a.n[of]) * a.d + c;
  float s = 0.0f;
#pragma unroll 8
  for (int i = threadIdx.x >> 3; i < a.n[of]; i += 32) s += p[(size_t)i * a.d];
  __shared__ float sums[32][8];
  sums[threadIdx.x >> 3][threadIdx.x & 7] = s;
  __syncthreads();
  if (threadIdx.x >= 8) return;
  s = 0.0f;
#pragma unroll
  for (int i = 0; i < 32; ++i) s += sums[i][threadIdx.x];
  a.out[of][id * a.d + c] = s;
}

QkArgs arguments(const QkProblem& p, int chunk, bool backward) {
  QkArgs a = {};
  for (int i = 0; i < 2; ++i) {
    HeadsOf& t = a.t[i];
    t.x = p.x[i];
    t.g = p.g[i];
    t.y = p.y[i];
    t.heads = p.heads[i];
    for (int j = 0; j < 3; ++j) {
      t.x_stride[j] = p.in_stride[i][j];
      t.g_stride[j] = p.out_stride[i][j];
      t.y_stride[j] = backward ? p.in_stride[i][j] : p.out_stride[i][j];
    }
    t.weight = p.weight[i];
  }
  a.N = p.N;
  a.rows = p.B * p.N;
  a.chunk = chunk;
  a.chunks_q = (p.heads[0] + chunk - 1) / chunk;
  a.r = Rotary{p.rotary.norm, p.rotary.eps, p.rotary.weight_dtype, p.rotary.weight_heads, p.rotary.rope,
               p.rotary.rope ? p.rotary.rot_dim : 0, p.rotary.n_pos, p.rotary.cos_table, p.rotary.sin_table};
  a.positions = p.positions;
  return a;
}
int all_chunks(const QkProblem& p, int chunk) { return (p.heads[0] + chunk - 1) / chunk + (p.heads[1] + chunk - 1) / chunk; }
// whether the call reads and writes, `tensors` of them in all, more than the caches are asked to hold
bool past_caches(const QkProblem& p, int tensors) {
  return (long long)tensors * p.B * p.N * (p.heads[0] + p.heads[1]) * p.d * (p.dtype == 0 ? 2 : 4) > kPastCaches;
}
int row_groups(const QkProblem& p) { return (p.B * p.N + kRowThreads * 16 / p.d - 1) / (kRowThreads * 16 / p.d); }

template <typename E, int D, int ROPE>
void forward(const QkProblem& p, hipStream_t stream) {
  const int groups = row_groups(p);
  // Two heads to a workgroup, which share its angles, where that still leaves two workgroups to a compute unit (one | two | four heads, us: H32 Hkv8
  // N4096 d64 11.5 | 11.3 | 12.1, H8 Hkv8 N4096 d128 10.4 | 11.1 | 10.9, with its gradient H32 Hkv8 N4096 d128 51.4 | 49.8 | 51.4).
  const bool two = (long long)groups * all_chunks(p, 2) >= 2 * kComputeUnits;
  const int chunk = two ? 2 : 1, chunks = all_chunks(p, chunk);
  const dim3 grid((unsigned)(groups * chunks)), block(kRowThreads);
  const QkArgs a = arguments(p, chunk, false);
  constexpr bool kCan = sizeof(E) == 2;
  if (kCan && two && past_caches(p, 2)) hipLaunchKernelGGL((qk_forward_kernel<E, D, ROPE, 2, kCan>), grid, block, 0, stream, a, chunks);
  else if (two) hipLaunchKernelGGL((qk_forward_kernel<E, D, ROPE, 2, false>), grid, block, 0, stream, a, chunks);
  else hipLaunchKernelGGL((qk_forward_kernel<E, D, ROPE, 1, false>), grid, block, 0, stream, a, chunks);
}

// Backward: heads of a workgroup and workgroups along the rows.
struct BackwardSplit {
  int chunk, chunks, groups;
};
BackwardSplit backward_split(const QkProblem& p) {
  BackwardSplit s;
  s.chunk = p.rotary.norm && p.rotary.weight_heads ? 1 : 4;
  s.chunks = all_chunks(p, s.chunk);
  // Workgroups that walk the rows: four to a compute unit, two for tensors that come from memory (B4 H16 Hkv16 N8192 d128 252 | 247 us; but H32 Hkv8
  // N4096 d64 29.5 | 32.3): fewer sums to add up.
  const int most = ((past_caches(p, 3) ? 2 : 4) * kComputeUnits + s.chunks - 1) / s.chunks;
  s.groups = std::max(1, std::min(row_groups(p), most));
  return s;
}

template <typename E, int D, int ROPE>
void backward(const QkProblem& p, float* part, hipStream_t stream) {
  const BackwardSplit s = backward_split(p);
  constexpr bool kCan = sizeof(E) == 2;
  const bool once = kCan && past_caches(p, p.rotary.norm ? 3 : 2);
  hipLaunchKernelGGL((once ? qk_backward_kernel<E, D, ROPE, kCan> : qk_backward_kernel<E, D, ROPE, false>), dim3((unsigned)(s.groups * s.chunks)),
                     dim3(kRowThreads), 0, stream, arguments(p, s.chunk, true), s.chunks, part);
}

#define DA_QK_DISPATCH(CALL)                                                        \
  const bool halves = p.rotary.rope == 1;                                           \
  if (p.dtype == 0) {                                                               \
    if (p.d == 64) halves ? CALL(bf16, 64, 1) : CALL(bf16, 64, 2);                  \
    else halves ? CALL(bf16, 128, 1) : CALL(bf16, 128, 2);                          \
  } else {                                                                          \
    if (p.d == 64) halves ? CALL(float, 64, 1) : CALL(float, 64, 2);                \
    else halves ? CALL(float, 128, 1) : CALL(float, 128, 2);                        \
  }

}  // namespace

hipError_t launch_qk_forward(const QkProblem& p, hipStream_t stream) {
#define DA_QK(E, D, R) forward<E, D, R>(p, stream)
  DA_QK_DISPATCH(DA_QK)
#undef DA_QK
  return hipGetLastError();
}

size_t qk_backward_scratch_bytes(const QkProblem& p) {
  if (!p.rotary.norm) return 0;
  const BackwardSplit s = backward_split(p);
  return (size_t)s.chunks * s.groups * p.d * 4;
}

hipError_t launch_qk_backward(const QkProblem& p, float* const dweight[2], float* part, hipStream_t stream) {
#define DA_QK(E, D, R) backward<E, D, R>(p, part, stream)
  DA_QK_DISPATCH(DA_QK)
#undef DA_QK
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || part == nullptr) return e;
  const BackwardSplit s = backward_split(p);
  const bool each = p.rotary.weight_heads != 0;
  const int chunks_q = (p.heads[0] + s.chunk - 1) / s.chunk, chunks_k = s.chunks - chunks_q;
  WeightSums a = {part, {dweight[0], dweight[1]}, {each ? p.heads[0] : 1, each ? p.heads[1] : (p.heads[1] ? 1 : 0)},
                  {0, chunks_q * s.groups}, {each ? s.groups : chunks_q * s.groups, each ? s.groups : chunks_k * s.groups}, p.d};
  hipLaunchKernelGGL(qk_weight_kernel, dim3((unsigned)((a.weights[0] + a.weights[1]) * (p.d / 8))), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace da
