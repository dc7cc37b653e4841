// moe_gate_backward: the gradients of the gate product score[t,e] = sum_i x[t,i] w_gate[e,i] + gate_bias[e]:
//   d_w_gate[e,:] = sum_t d_scores[t,e] x[t,:]      d_gate_bias[e] = sum_t d_scores[t,e]
//   d_x[t,:]      = sum_e d_scores[t,e] w_gate[e,:]
// One thread per column and eight experts for the weights' gradient, the tokens split over blocks whose sums
// meet in the workspace; one block per token for the hidden states'.
#include "moe_internal.h"

namespace moe {

constexpr int GB_THREADS = 256;
constexpr int GB_EXPERTS = 8;

template <bool BF16> __device__ __forceinline__ float gb_load(const void* p, int64_t i) {
  return BF16 ? bf16_to_f32(static_cast<const bf16_t*>(p)[i]) : static_cast<const float*>(p)[i];
}

template <bool BF16>
__global__ __launch_bounds__(GB_THREADS) void gate_weight_grad_kernel(const void* __restrict__ x,
                                                                      const float* __restrict__ d_scores,
                                                                      const uint8_t* __restrict__ mask, int T, int d, int E,
                                                                      int per_split, float* __restrict__ part_w,
                                                                      float* __restrict__ part_b) {
  const int i = blockIdx.x * GB_THREADS + threadIdx.x, e0 = blockIdx.y * GB_EXPERTS;
  const int64_t t0 = static_cast<int64_t>(blockIdx.z) * per_split, t1 = min(t0 + per_split, static_cast<int64_t>(T));
  float acc[GB_EXPERTS] = {}, bias[GB_EXPERTS] = {};
  for (int64_t t = t0; t < t1; ++t) {
    if (mask && !mask[t]) continue;
    const float xv = i < d ? gb_load<BF16>(x, t * d + i) : 0.f;
#pragma unroll
    for (int u = 0; u < GB_EXPERTS; ++u) {
      const float v = e0 + u < E ? d_scores[t * E + e0 + u] : 0.f;
      acc[u] = fmaf(v, xv, acc[u]);
      bias[u] += v;
    }
  }
#pragma unroll
  for (int u = 0; u < GB_EXPERTS; ++u) {
    if (e0 + u >= E) continue;
    if (i < d) part_w[(static_cast<int64_t>(blockIdx.z) * E + e0 + u) * d + i] = acc[u];
    if (i == 0) part_b[static_cast<int64_t>(blockIdx.z) * E + e0 + u] = bias[u];
  }
}

__global__ __launch_bounds__(GB_THREADS) void gate_weight_sum_kernel(const float* __restrict__ part, int splits, int64_t n,
                                                                     int accumulate, float* __restrict__ out) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * GB_THREADS + threadIdx.x;
  if (i >= n) return;
  float v = accumulate ? out[i] : 0.f;
  for (int s = 0; s < splits; ++s) v += part[s * n + i];
  out[i] = v;
}

template <bool BF16>
__global__ __launch_bounds__(GB_THREADS) void gate_x_grad_kernel(const void* __restrict__ w, const float* __restrict__ d_scores,
                                                                 const uint8_t* __restrict__ mask, int T, int d, int E,
                                                                 int accumulate, void* __restrict__ d_x) {
  __shared__ float ds[MOE_MAX_E];
  for (int64_t t = blockIdx.x; t < T; t += gridDim.x) {
    const bool real = !mask || mask[t];
    __syncthreads();
    if (static_cast<int>(threadIdx.x) < E) ds[threadIdx.x] = real ? d_scores[t * E + threadIdx.x] : 0.f;
    __syncthreads();
    for (int i = threadIdx.x; i < d; i += GB_THREADS) {
      float v = 0.f;
      for (int e = 0; e < E; ++e) v = fmaf(ds[e], gb_load<BF16>(w, static_cast<int64_t>(e) * d + i), v);
      if (accumulate) v += gb_load<BF16>(d_x, t * d + i);
      if (BF16)
        static_cast<bf16_t*>(d_x)[t * d + i] = f32_to_bf16(v);
      else
        static_cast<float*>(d_x)[t * d + i] = v;
    }
  }
}

// Tokens are cut into this many parts, each of 64 tokens or more.
static int gb_splits(int T) {
  const int64_t s = (static_cast<int64_t>(T) + 63) / 64;
  return static_cast<int>(s < 32 ? s : 32);
}

size_t gate_backward_workspace_bytes(const moe_shape_t* shape) {
  return static_cast<size_t>(gb_splits(shape->T)) * shape->E * (static_cast<size_t>(shape->d) + 1) * sizeof(float);
}

template <bool BF16>
static int gate_backward(const moe_shape_t* shape, const void* x, const void* w_gate, const float* d_scores, const uint8_t* mask,
                         float* d_w_gate, float* d_gate_bias, void* d_x, int accumulate, float* part, hipStream_t st) {
  const int T = shape->T, d = shape->d, E = shape->E, splits = gb_splits(T);
  const int acc_w = accumulate & MOE_ACCUMULATE_WEIGHTS ? 1 : 0, acc_x = accumulate & MOE_ACCUMULATE_X ? 1 : 0;
  if (d_w_gate || d_gate_bias) {
    float* part_b = part + static_cast<size_t>(splits) * E * d;
    if (splits > 0)
      hipLaunchKernelGGL((gate_weight_grad_kernel<BF16>), dim3((d + GB_THREADS - 1) / GB_THREADS, (E + GB_EXPERTS - 1) / GB_EXPERTS, splits),
                         dim3(GB_THREADS), 0, st, x, d_scores, mask, T, d, E, (T + splits - 1) / splits, part, part_b);
    auto sum = [&](const float* p, int64_t n, float* out) {
      hipLaunchKernelGGL(gate_weight_sum_kernel, dim3(static_cast<unsigned>((n + GB_THREADS - 1) / GB_THREADS)), dim3(GB_THREADS), 0,
                         st, p, splits, n, acc_w, out);
    };
    if (d_w_gate) sum(part, static_cast<int64_t>(E) * d, d_w_gate);
    if (d_gate_bias) sum(part_b, E, d_gate_bias);
  }
  if (d_x && T > 0)
    hipLaunchKernelGGL((gate_x_grad_kernel<BF16>), dim3(T < 8192 ? T : 8192), dim3(GB_THREADS), 0, st, w_gate, d_scores, mask, T, d,
                       E, acc_x, d_x);
  return launch_status();
}

}  // namespace moe

extern "C" int moe_train_workspace_bytes(const moe_shape_t* shape, size_t* out_bytes) {
  const int rc = moe::check_shape(shape);
  if (rc != MOE_OK) return rc;
  if (!out_bytes) return MOE_ERR_INVALID_ARG;
  const size_t a = moe::gate_loss_workspace_bytes(shape), b = moe::gate_backward_workspace_bytes(shape);
  *out_bytes = ((a > b ? a : b) + 255) / 256 * 256;
  if (*out_bytes == 0) *out_bytes = 256;
  return MOE_OK;
}

extern "C" int moe_gate_backward(const moe_shape_t* shape, const void* x, const void* w_gate, const float* d_scores,
                                 const uint8_t* token_mask, float* d_w_gate, float* d_gate_bias, void* d_x, int accumulate,
                                 void* workspace, size_t workspace_bytes, void* hip_stream) {
  using namespace moe;
  const int rc = check_shape(shape);
  if (rc != MOE_OK) return rc;
  if (accumulate & ~(MOE_ACCUMULATE_WEIGHTS | MOE_ACCUMULATE_X)) return MOE_ERR_INVALID_ARG;
  if (!d_w_gate && !d_gate_bias && !d_x) return shape->T == 0 ? MOE_OK : MOE_ERR_INVALID_ARG;
  if (!aligned16(d_w_gate) || !aligned4(d_gate_bias) || !aligned16(d_x) || !aligned16(x) || !aligned16(w_gate) || !aligned16(d_scores))
    return MOE_ERR_INVALID_ARG;
  if (shape->T > 0 && (!d_scores || (d_w_gate && !x) || (d_x && !w_gate))) return MOE_ERR_INVALID_ARG;
  if (d_w_gate || d_gate_bias) {
    if (!workspace || !aligned16(workspace)) return MOE_ERR_INVALID_ARG;
    if (workspace_bytes < gate_backward_workspace_bytes(shape)) return MOE_ERR_WORKSPACE;
  }
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  return shape->dtype == MOE_BF16
             ? gate_backward<true>(shape, x, w_gate, d_scores, token_mask, d_w_gate, d_gate_bias, d_x, accumulate, static_cast<float*>(workspace), st)
             : gate_backward<false>(shape, x, w_gate, d_scores, token_mask, d_w_gate, d_gate_bias, d_x, accumulate, static_cast<float*>(workspace), st);
}
