// The losses that a gate is trained with, and their gradients with respect to its scores s [T,E]:
//   moe_balance_loss    counts c_e and probability sums P_e = sum_t p[t,e], p = softmax_E(s);
//                       L = E k sum_e c_e P_e / (sum c)^2
//   moe_route_backward  the gradient of the routing weights and of coef * L
//   moe_gate_distill    the mean over tokens of KL(softmax(target) || p), and its gradient
// All three stream tables of T x E floats once: HBM-bound for large batches, launch-bound for small ones.
//
// One wave per token; lane l holds the scores of experts l, l + 64, ...  Sums over tokens stay in registers (a lane
// keeps its experts), meet in LDS at the end of the block and go to the workspace as one row per block; a single
// block then adds the rows in 64 bits, in a fixed order.
#include "moe_internal.h"

namespace moe {

constexpr int GL_THREADS = 256;
constexpr int GL_WAVES = GL_THREADS / MOE_WAVE;
constexpr int GL_BLOCKS = 512;        // most blocks of a launch that leaves partial sums
constexpr int GL_FINISH = 1024;       // threads of the block that adds them

__device__ __forceinline__ float gl_wave_sum(float v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off);
  return v;
}
__device__ __forceinline__ float gl_wave_max(float v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v = fmaxf(v, __shfl_xor(v, off));
  return v;
}

// The scores of token t, -inf past the last expert.
template <int QE>
__device__ __forceinline__ void gl_load(const float* __restrict__ scores, int64_t t, int E, int lane, float (&s)[QE]) {
#pragma unroll
  for (int q = 0; q < QE; ++q) {
    const int e = lane + q * MOE_WAVE;
    s[q] = e < E ? scores[t * E + e] : -INFINITY;
  }
}

// p = softmax(s), zeros where every score is -inf; returns log(sum_e exp(s_e)) (-inf there).
template <int QE> __device__ __forceinline__ float gl_softmax(const float (&s)[QE], float (&p)[QE]) {
  float m = s[0];
#pragma unroll
  for (int q = 1; q < QE; ++q) m = fmaxf(m, s[q]);
  m = gl_wave_max(m);
  const bool empty = m == -INFINITY;
  if (empty) m = 0.f;
  float sum = 0.f;
#pragma unroll
  for (int q = 0; q < QE; ++q) {
    p[q] = expf(s[q] - m);
    sum += p[q];
  }
  sum = fmaxf(gl_wave_sum(sum), 1e-30f);     // 1 or more unless all are zero
#pragma unroll
  for (int q = 0; q < QE; ++q) p[q] /= sum;
  return empty ? -INFINITY : m + logf(sum);
}

template <int QE>
__global__ __launch_bounds__(GL_THREADS) void balance_kernel(const float* __restrict__ scores,
                                                             const int32_t* __restrict__ topk_idx,
                                                             const uint8_t* __restrict__ mask, int T, int E, int k,
                                                             float* __restrict__ part_p, int32_t* __restrict__ part_c) {
  __shared__ float sum_p[GL_WAVES][MOE_MAX_E];
  __shared__ int32_t cnt[MOE_MAX_E];
  const int lane = lane_id(), wave = threadIdx.x / MOE_WAVE;
  cnt[threadIdx.x] = 0;
  __syncthreads();
  float acc[QE];
#pragma unroll
  for (int q = 0; q < QE; ++q) acc[q] = 0.f;
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * GL_WAVES + wave; t < T; t += static_cast<int64_t>(gridDim.x) * GL_WAVES) {
    if (mask && !mask[t]) continue;
    float s[QE], p[QE];
    gl_load(scores, t, E, lane, s);
    if (lane < k) {
      const int e = topk_idx[t * k + lane];
      if (static_cast<unsigned>(e) < static_cast<unsigned>(E)) atomicAdd(&cnt[e], 1);
    }
    gl_softmax(s, p);
#pragma unroll
    for (int q = 0; q < QE; ++q) acc[q] += p[q];
  }
#pragma unroll
  for (int q = 0; q < QE; ++q) sum_p[wave][lane + q * MOE_WAVE] = acc[q];
  __syncthreads();
  const int e = threadIdx.x;
  if (e < E) {
    float v = 0.f;
    for (int w = 0; w < GL_WAVES; ++w) v += sum_p[w][e];
    part_p[static_cast<int64_t>(blockIdx.x) * E + e] = v;
    part_c[static_cast<int64_t>(blockIdx.x) * E + e] = cnt[e];
  }
}

// Sum over the block of one value per thread, in a fixed order; valid on thread 0.
template <class V> __device__ __forceinline__ V gl_block_sum(V v, V* lds) {
  lds[threadIdx.x] = v;
  __syncthreads();
  for (int half = blockDim.x / 2; half >= 1; half >>= 1) {
    if (threadIdx.x < static_cast<unsigned>(half)) lds[threadIdx.x] += lds[threadIdx.x + half];
    __syncthreads();
  }
  const V r = lds[0];
  __syncthreads();
  return r;
}

__global__ __launch_bounds__(GL_FINISH) void balance_finish_kernel(const float* __restrict__ part_p,
                                                                   const int32_t* __restrict__ part_c, int blocks, int E,
                                                                   int k, int32_t* __restrict__ counts,
                                                                   float* __restrict__ prob_sum, float* __restrict__ loss) {
  __shared__ double sp[GL_FINISH];
  __shared__ double sc[GL_FINISH];
  const int e = threadIdx.x & (MOE_MAX_E - 1), g = threadIdx.x / MOE_MAX_E;
  double p = 0.0, c = 0.0;
  if (e < E)
    for (int b = g; b < blocks; b += GL_FINISH / MOE_MAX_E) {
      p += part_p[static_cast<int64_t>(b) * E + e];
      c += part_c[static_cast<int64_t>(b) * E + e];
    }
  sp[threadIdx.x] = p;
  sc[threadIdx.x] = c;
  __syncthreads();
  if (g == 0) {
    for (int i = 1; i < GL_FINISH / MOE_MAX_E; ++i) {
      p += sp[i * MOE_MAX_E + e];
      c += sc[i * MOE_MAX_E + e];
    }
    if (e < E) {
      counts[e] = static_cast<int32_t>(c);
      prob_sum[e] = static_cast<float>(p);
    }
  }
  __syncthreads();
  const double total = gl_block_sum(g == 0 ? c : 0.0, sc);
  const double dot = gl_block_sum(g == 0 ? c * p : 0.0, sp);
  if (threadIdx.x == 0) *loss = total > 0.0 ? static_cast<float>(dot * E * k / (total * total)) : 0.f;
}

// ds = gradient of sum_j d_topk_w[j] w_j (w: the routing weights of moe_route) + gradient of coef * L.
//   renorm 0: w_j = p[i_j]:                 ds_e = p_e (g_e - sum_l p_l g_l),  g_e = sum of d_topk_w[j] with i_j = e
//   renorm 1: w = softmax over the chosen:  ds[i_j] = w_j (d_topk_w[j] - sum_l w_l d_topk_w[l])
//   balance:  b_e = coef E k c_e / (sum c)^2, ds_e = p_e (b_e - sum_l p_l b_l)
template <int QE>
__global__ __launch_bounds__(GL_THREADS) void route_backward_kernel(const float* __restrict__ scores,
                                                                    const int32_t* __restrict__ topk_idx,
                                                                    const float* __restrict__ d_topk_w,
                                                                    const int32_t* __restrict__ counts, float coef,
                                                                    const uint8_t* __restrict__ mask, int T, int E, int k,
                                                                    int renorm, int accumulate, float* __restrict__ d_scores) {
  const int lane = lane_id(), wave = threadIdx.x / MOE_WAVE;
  float b[QE];
#pragma unroll
  for (int q = 0; q < QE; ++q) b[q] = 0.f;
  if (counts) {
    int64_t total = 0;
    for (int e = 0; e < E; ++e) total += counts[e];
    const double c = total > 0 ? static_cast<double>(coef) * E * k / (static_cast<double>(total) * static_cast<double>(total)) : 0.0;
#pragma unroll
    for (int q = 0; q < QE; ++q) {
      const int e = lane + q * MOE_WAVE;
      if (e < E) b[q] = static_cast<float>(c * counts[e]);
    }
  }
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * GL_WAVES + wave; t < T; t += static_cast<int64_t>(gridDim.x) * GL_WAVES) {
    float d[QE];
#pragma unroll
    for (int q = 0; q < QE; ++q) d[q] = 0.f;
    if (!mask || mask[t]) {
      float s[QE], p[QE], g[QE], chosen[QE];
      gl_load(scores, t, E, lane, s);
      gl_softmax(s, p);
#pragma unroll
      for (int q = 0; q < QE; ++q) {
        g[q] = b[q];
        chosen[q] = 0.f;
      }
      if (d_topk_w) {
        int my_e = lane < k ? topk_idx[t * k + lane] : -1;
        if (static_cast<unsigned>(my_e) >= static_cast<unsigned>(E)) my_e = -1;
        float my_d = my_e >= 0 ? d_topk_w[t * k + lane] : 0.f;
        if (renorm) {
          const float my_s = my_e >= 0 ? scores[t * E + my_e] : -INFINITY;
          float m = gl_wave_max(my_s);
          if (m == -INFINITY) m = 0.f;
          float w = my_e >= 0 ? expf(my_s - m) : 0.f;
          w /= fmaxf(gl_wave_sum(w), 1e-30f);
          my_d = w * (my_d - gl_wave_sum(w * my_d));
        }
        for (int j = 0; j < k; ++j) {
          const int e = __shfl(my_e, j);
          const float v = __shfl(my_d, j);
#pragma unroll
          for (int q = 0; q < QE; ++q)
            if (e == lane + q * MOE_WAVE) (renorm ? chosen[q] : g[q]) += v;
        }
      }
      float dot = 0.f;
#pragma unroll
      for (int q = 0; q < QE; ++q) dot += p[q] * g[q];
      dot = gl_wave_sum(dot);
#pragma unroll
      for (int q = 0; q < QE; ++q) d[q] = p[q] * (g[q] - dot) + chosen[q];
    }
#pragma unroll
    for (int q = 0; q < QE; ++q) {
      const int e = lane + q * MOE_WAVE;
      if (e < E) d_scores[t * E + e] = accumulate ? d_scores[t * E + e] + d[q] : d[q];
    }
  }
}

// Tokens that the mask keeps, one number per block.
__global__ __launch_bounds__(GL_THREADS) void mask_count_kernel(const uint8_t* __restrict__ mask, int T, int32_t* __restrict__ part) {
  __shared__ int32_t lds[GL_THREADS];
  int n = 0;
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * GL_THREADS + threadIdx.x; t < T; t += static_cast<int64_t>(gridDim.x) * GL_THREADS)
    n += mask[t] != 0;
  n = gl_block_sum(n, lds);
  if (threadIdx.x == 0) part[blockIdx.x] = n;
}

// Tokens that count, from the blocks of mask_count_kernel (T without a mask); the same on every thread.
__device__ __forceinline__ double gl_tokens(const int32_t* __restrict__ part_n, int n_blocks, int T) {
  if (!part_n) return T;
  double n = 0.0;
  for (int b = 0; b < n_blocks; ++b) n += part_n[b];
  return n;
}

template <int QE>
__global__ __launch_bounds__(GL_THREADS) void distill_kernel(const float* __restrict__ scores,
                                                             const float* __restrict__ target,
                                                             const uint8_t* __restrict__ mask,
                                                             const int32_t* __restrict__ part_n, int n_blocks, int T, int E,
                                                             float coef, int accumulate, double* __restrict__ part_loss,
                                                             float* __restrict__ d_scores) {
  __shared__ double lds[GL_THREADS];
  const int lane = lane_id(), wave = threadIdx.x / MOE_WAVE;
  const double n = gl_tokens(part_n, n_blocks, T);
  const float scale = n > 0.0 ? static_cast<float>(coef / n) : 0.f;
  double loss = 0.0;
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * GL_WAVES + wave; t < T; t += static_cast<int64_t>(gridDim.x) * GL_WAVES) {
    float d[QE];
#pragma unroll
    for (int q = 0; q < QE; ++q) d[q] = 0.f;
    if (!mask || mask[t]) {
      float s[QE], u[QE], p[QE], w[QE];
      gl_load(scores, t, E, lane, s);
      gl_load(target, t, E, lane, u);
      const float lp = gl_softmax(s, p), lq = gl_softmax(u, w);
      if (lp > -INFINITY && lq > -INFINITY) {
        float row = 0.f;
#pragma unroll
        for (int q = 0; q < QE; ++q) {
          const int e = lane + q * MOE_WAVE;
          if (e < E && w[q] > 0.f) row += w[q] * ((u[q] - lq) - (s[q] - lp));
          d[q] = scale * (p[q] - w[q]);
        }
        loss += row;
      }
    }
    if (d_scores) {
#pragma unroll
      for (int q = 0; q < QE; ++q) {
        const int e = lane + q * MOE_WAVE;
        if (e < E) d_scores[t * E + e] = accumulate ? d_scores[t * E + e] + d[q] : d[q];
      }
    }
  }
  loss = gl_block_sum(loss, lds);
  if (threadIdx.x == 0) part_loss[blockIdx.x] = loss;
}

__global__ __launch_bounds__(GL_FINISH) void distill_finish_kernel(const double* __restrict__ part_loss, int blocks,
                                                                   const int32_t* __restrict__ part_n, int n_blocks, int T,
                                                                   float* __restrict__ loss) {
  __shared__ double lds[GL_FINISH];
  const double sum = gl_block_sum(static_cast<int>(threadIdx.x) < blocks ? part_loss[threadIdx.x] : 0.0, lds);
  const double n = gl_tokens(part_n, n_blocks, T);
  if (threadIdx.x == 0) *loss = n > 0.0 ? static_cast<float>(sum / n) : 0.f;
}

static_assert(GL_BLOCKS <= GL_FINISH, "one partial loss per thread");

static int gl_blocks(int T) {
  const int64_t b = (static_cast<int64_t>(T) + GL_WAVES - 1) / GL_WAVES;
  return static_cast<int>(b < GL_BLOCKS ? b : GL_BLOCKS);
}
constexpr int GL_COUNT_BLOCKS = 64;

// Kernel variant by the number of scores per lane.
#define GL_BY_E(E, CALL) \
  do {                   \
    if ((E) <= 64) {     \
      constexpr int QE = 1; CALL; \
    } else if ((E) <= 128) { \
      constexpr int QE = 2; CALL; \
    } else {             \
      constexpr int QE = 4; CALL; \
    }                    \
  } while (0)

size_t gate_loss_workspace_bytes(const moe_shape_t* shape) {
  const size_t b = static_cast<size_t>(gl_blocks(shape->T));
  const size_t balance = b * shape->E * 8, distill = b * 8 + GL_COUNT_BLOCKS * 4;
  return balance > distill ? balance : distill;
}

}  // namespace moe

extern "C" int moe_balance_loss(const moe_shape_t* shape, const float* scores, const int32_t* topk_idx,
                                const uint8_t* token_mask, int32_t* counts, float* prob_sum, float* loss,
                                void* workspace, size_t workspace_bytes, void* hip_stream) {
  using namespace moe;
  const int rc = check_shape(shape);
  if (rc != MOE_OK) return rc;
  if (!counts || !prob_sum || !loss || !workspace || !aligned16(workspace)) return MOE_ERR_INVALID_ARG;
  if (!aligned4(topk_idx) || !aligned4(counts) || !aligned4(prob_sum) || !aligned4(loss)) return MOE_ERR_INVALID_ARG;
  if (shape->T > 0 && (!scores || !topk_idx || !aligned16(scores))) return MOE_ERR_INVALID_ARG;
  if (workspace_bytes < gate_loss_workspace_bytes(shape)) return MOE_ERR_WORKSPACE;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const int T = shape->T, E = shape->E, k = shape->k, blocks = gl_blocks(T);
  float* part_p = static_cast<float*>(workspace);
  int32_t* part_c = reinterpret_cast<int32_t*>(part_p + static_cast<size_t>(blocks) * E);
  if (blocks > 0)
    GL_BY_E(E, hipLaunchKernelGGL((balance_kernel<QE>), dim3(blocks), dim3(GL_THREADS), 0, st, scores, topk_idx,
                                  token_mask, T, E, k, part_p, part_c));
  hipLaunchKernelGGL(balance_finish_kernel, dim3(1), dim3(GL_FINISH), 0, st, part_p, part_c, blocks, E, k, counts,
                     prob_sum, loss);
  return launch_status();
}

extern "C" int moe_route_backward(const moe_shape_t* shape, const float* scores, const int32_t* topk_idx,
                                  const float* d_topk_w, const int32_t* counts, float balance_coef,
                                  const uint8_t* token_mask, float* d_scores, int accumulate, void* hip_stream) {
  using namespace moe;
  const int rc = check_shape(shape);
  if (rc != MOE_OK) return rc;
  if (accumulate != 0 && accumulate != 1) return MOE_ERR_INVALID_ARG;
  if (shape->T == 0) return MOE_OK;
  if (!d_topk_w && !counts) return MOE_ERR_INVALID_ARG;
  if (!scores || !d_scores || (d_topk_w && !topk_idx)) return MOE_ERR_INVALID_ARG;
  if (!aligned16(scores) || !aligned16(d_scores) || !aligned4(topk_idx) || !aligned4(d_topk_w) || !aligned4(counts))
    return MOE_ERR_INVALID_ARG;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const int T = shape->T, E = shape->E, k = shape->k;
  GL_BY_E(E, hipLaunchKernelGGL((route_backward_kernel<QE>), dim3(gl_blocks(T)), dim3(GL_THREADS), 0, st, scores, topk_idx,
                                d_topk_w, counts, balance_coef, token_mask, T, E, k, shape->renorm, accumulate, d_scores));
  return launch_status();
}

extern "C" int moe_gate_distill(const moe_shape_t* shape, const float* scores, const float* target_scores,
                                const uint8_t* token_mask, float coef, float* loss, float* d_scores, int accumulate,
                                void* workspace, size_t workspace_bytes, void* hip_stream) {
  using namespace moe;
  const int rc = check_shape(shape);
  if (rc != MOE_OK) return rc;
  if (accumulate != 0 && accumulate != 1) return MOE_ERR_INVALID_ARG;
  if (!loss || !workspace || !aligned16(workspace)) return MOE_ERR_INVALID_ARG;
  if (shape->T > 0 && (!scores || !target_scores || !aligned16(scores) || !aligned16(target_scores))) return MOE_ERR_INVALID_ARG;
  if (!aligned16(d_scores) || !aligned4(loss)) return MOE_ERR_INVALID_ARG;
  if (workspace_bytes < gate_loss_workspace_bytes(shape)) return MOE_ERR_WORKSPACE;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const int T = shape->T, E = shape->E, blocks = gl_blocks(T);
  double* part_loss = static_cast<double*>(workspace);
  int32_t* part_n = token_mask ? reinterpret_cast<int32_t*>(part_loss + blocks) : nullptr;
  if (token_mask && T > 0)
    hipLaunchKernelGGL(mask_count_kernel, dim3(GL_COUNT_BLOCKS), dim3(GL_THREADS), 0, st, token_mask, T, part_n);
  if (blocks > 0)
    GL_BY_E(E, hipLaunchKernelGGL((distill_kernel<QE>), dim3(blocks), dim3(GL_THREADS), 0, st, scores, target_scores,
                                  token_mask, part_n, GL_COUNT_BLOCKS, T, E, coef, accumulate, part_loss, d_scores));
  hipLaunchKernelGGL(distill_finish_kernel, dim3(1), dim3(GL_FINISH), 0, st, part_loss, blocks, T > 0 ? part_n : nullptr,
                     GL_COUNT_BLOCKS, T, loss);
  return launch_status();
}
