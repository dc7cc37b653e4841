// moe_grad_norm, moe_clip_grads: the Euclidean norm of a list of tensors taken together, and the tensors scaled to a
// largest norm:  norm = sqrt(sum over all elements of g^2),  out = g * min(1, max_norm / norm).
// HBM-bound: every element is read once for the norm, and once more with a write for the scaling.
//
// The list travels in the kernels' arguments, so no table has to reach the device first and a captured graph holds its
// own copy.  Every block takes one piece of one tensor.  Squares and their sums are 64-bit (an fp32 square overflows
// from 1.8e19 on and loses all bits below 1e-23); a block leaves one sum in the workspace and one block adds those in
// a fixed order.
#include "moe_internal.h"

namespace moe {

constexpr int GR_THREADS = 256;
constexpr int GR_TENSORS = 128;        // tensors of one launch
constexpr int64_t GR_PIECE = 4096;     // least elements of a piece; all pieces of a call have the same size
constexpr int64_t GR_PIECES = 2048;    // pieces of a call that is large enough

struct GradTable {
  const void* data[GR_TENSORS];
  void* out[GR_TENSORS];
  int64_t n[GR_TENSORS];               // elements * 2 + 1 for bf16
  int32_t first[GR_TENSORS];           // first block of each tensor
};
static_assert(sizeof(GradTable) <= 3900, "arguments of a launch");

struct GradPiece {
  const void* data;
  void* out;
  int64_t begin, end;
  bool bf16;
};

// The piece of this block: the last tensor whose first block is not behind it (tensors without elements have no block).
__device__ __forceinline__ GradPiece grad_piece(const GradTable& tab, int count, int64_t piece) {
  int lo = 0, hi = count - 1;
  const int b = blockIdx.x;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (tab.first[mid] <= b) lo = mid; else hi = mid - 1;
  }
  GradPiece g;
  const int64_t n = tab.n[lo] >> 1;
  g.data = tab.data[lo];
  g.out = tab.out[lo];
  g.bf16 = tab.n[lo] & 1;
  g.begin = static_cast<int64_t>(b - tab.first[lo]) * piece;
  g.end = g.begin + piece < n ? g.begin + piece : n;
  return g;
}

__device__ __forceinline__ float grad_load(const void* p, int64_t i, bool bf16) {
  return bf16 ? bf16_to_f32(static_cast<const bf16_t*>(p)[i]) : static_cast<const float*>(p)[i];
}

__device__ __forceinline__ double grad_block_sum(double v, double* lds) {
  lds[threadIdx.x] = v;
  __syncthreads();
  for (int half = GR_THREADS / 2; half >= 1; half >>= 1) {
    if (threadIdx.x < static_cast<unsigned>(half)) lds[threadIdx.x] += lds[threadIdx.x + half];
    __syncthreads();
  }
  return lds[0];
}

__global__ __launch_bounds__(GR_THREADS) void grad_square_kernel(GradTable tab, int count, int64_t piece, double* __restrict__ part) {
  __shared__ double lds[GR_THREADS];
  const GradPiece g = grad_piece(tab, count, piece);
  double s = 0.0;
  for (int64_t i = g.begin + threadIdx.x; i < g.end; i += GR_THREADS) {
    const double v = grad_load(g.data, i, g.bf16);
    s = fma(v, v, s);
  }
  s = grad_block_sum(s, lds);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// coef[0] = min(1, max_norm / norm); 1 where the norm is no finite number (the caller sees it in `norm`).
__global__ __launch_bounds__(GR_THREADS) void grad_finish_kernel(const double* __restrict__ part, int64_t pieces, double max_norm,
                                                                 float* __restrict__ norm, float* __restrict__ coef) {
  __shared__ double lds[GR_THREADS];
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < pieces; i += GR_THREADS) s += part[i];
  s = sqrt(grad_block_sum(s, lds));
  if (threadIdx.x == 0) {
    *norm = static_cast<float>(s);
    *coef = s > max_norm && s < INFINITY ? static_cast<float>(max_norm / s) : 1.f;
  }
}

__global__ __launch_bounds__(GR_THREADS) void grad_scale_kernel(GradTable tab, int count, int64_t piece, const float* __restrict__ coef) {
  const GradPiece g = grad_piece(tab, count, piece);
  const float c = *coef;
  if (c == 1.f && g.out == g.data) return;
  for (int64_t i = g.begin + threadIdx.x; i < g.end; i += GR_THREADS) {
    const float v = grad_load(g.data, i, g.bf16) * c;
    if (g.bf16)
      static_cast<bf16_t*>(g.out)[i] = f32_to_bf16(v);
    else
      static_cast<float*>(g.out)[i] = v;
  }
}

static int check_grads(int32_t count, const moe_tensor_t* tensors, bool with_out) {
  if (count < 0 || (count > 0 && !tensors)) return MOE_ERR_INVALID_ARG;
  int64_t total = 0;
  for (int32_t i = 0; i < count; ++i) {
    const moe_tensor_t& t = tensors[i];
    if (t.dtype != MOE_F32 && t.dtype != MOE_BF16) return MOE_ERR_INVALID_ARG;
    if (t.n < 0) return MOE_ERR_INVALID_ARG;
    if (t.n == 0) continue;
    const uintptr_t off = static_cast<uintptr_t>(elem_bytes(t.dtype)) - 1;
    if (!t.data || (reinterpret_cast<uintptr_t>(t.data) & off)) return MOE_ERR_INVALID_ARG;
    if (with_out && (!t.out || (reinterpret_cast<uintptr_t>(t.out) & off))) return MOE_ERR_INVALID_ARG;
    if (t.n > (int64_t(1) << 40)) return MOE_ERR_UNSUPPORTED;
    total += t.n;
    if (total > (int64_t(1) << 40)) return MOE_ERR_UNSUPPORTED;
  }
  return MOE_OK;
}

// Elements of a piece, and the number of pieces of all tensors.
static int64_t grad_pieces(int32_t count, const moe_tensor_t* tensors, int64_t* piece) {
  int64_t total = 0, pieces = 0;
  for (int32_t i = 0; i < count; ++i) total += tensors[i].n;
  int64_t p = (total + GR_PIECES - 1) / GR_PIECES;
  p = (p + GR_PIECE - 1) / GR_PIECE * GR_PIECE;
  if (p < GR_PIECE) p = GR_PIECE;
  for (int32_t i = 0; i < count; ++i) pieces += (tensors[i].n + p - 1) / p;
  *piece = p;
  return pieces;
}

// Calls launch(table, tensors in it, blocks) for up to GR_TENSORS tensors that have elements at a time.
template <class F> static void for_tables(int32_t count, const moe_tensor_t* tensors, int64_t piece, F launch) {
  GradTable tab;
  int n = 0;
  int64_t blocks = 0;
  for (int32_t i = 0; i < count; ++i) {
    if (tensors[i].n == 0) continue;
    tab.data[n] = tensors[i].data;
    tab.out[n] = tensors[i].out;
    tab.n[n] = tensors[i].n * 2 + (tensors[i].dtype == MOE_BF16 ? 1 : 0);
    tab.first[n] = static_cast<int32_t>(blocks);
    blocks += (tensors[i].n + piece - 1) / piece;
    if (++n == GR_TENSORS) {
      launch(tab, n, static_cast<int>(blocks));
      n = 0;
      blocks = 0;
    }
  }
  if (n > 0) launch(tab, n, static_cast<int>(blocks));
}

static int grads_call(int32_t count, const moe_tensor_t* tensors, bool clip, double max_norm, float* norm, void* workspace,
                      size_t workspace_bytes, hipStream_t st) {
  const int rc = check_grads(count, tensors, clip);
  if (rc != MOE_OK) return rc;
  if (!norm || (reinterpret_cast<uintptr_t>(norm) & 3) || !workspace || !aligned16(workspace)) return MOE_ERR_INVALID_ARG;
  int64_t piece = 0;
  const int64_t pieces = grad_pieces(count, tensors, &piece);
  if (workspace_bytes < static_cast<size_t>(pieces) * 8 + 16) return MOE_ERR_WORKSPACE;
  float* coef = static_cast<float*>(workspace);
  double* part = static_cast<double*>(workspace) + 2;
  int64_t at = 0;
  for_tables(count, tensors, piece, [&](const GradTable& tab, int n, int blocks) {
    hipLaunchKernelGGL(grad_square_kernel, dim3(blocks), dim3(GR_THREADS), 0, st, tab, n, piece, part + at);
    at += blocks;
  });
  hipLaunchKernelGGL(grad_finish_kernel, dim3(1), dim3(GR_THREADS), 0, st, part, pieces, max_norm, norm, coef);
  if (clip)
    for_tables(count, tensors, piece, [&](const GradTable& tab, int n, int blocks) {
      hipLaunchKernelGGL(grad_scale_kernel, dim3(blocks), dim3(GR_THREADS), 0, st, tab, n, piece, coef);
    });
  return launch_status();
}

}  // namespace moe

extern "C" int moe_grad_workspace_bytes(int32_t count, const moe_tensor_t* tensors, size_t* out_bytes) {
  const int rc = moe::check_grads(count, tensors, false);
  if (rc != MOE_OK) return rc;
  if (!out_bytes) return MOE_ERR_INVALID_ARG;
  int64_t piece = 0;
  *out_bytes = (static_cast<size_t>(moe::grad_pieces(count, tensors, &piece)) * 8 + 16 + 255) / 256 * 256;
  return MOE_OK;
}

extern "C" int moe_grad_norm(int32_t count, const moe_tensor_t* tensors, float* norm, void* workspace, size_t workspace_bytes,
                             void* hip_stream) {
  return moe::grads_call(count, tensors, false, 0.0, norm, workspace, workspace_bytes, static_cast<hipStream_t>(hip_stream));
}

extern "C" int moe_clip_grads(int32_t count, const moe_tensor_t* tensors, float max_norm, float* norm, void* workspace,
                              size_t workspace_bytes, void* hip_stream) {
  if (!(max_norm >= 0.f)) return MOE_ERR_INVALID_ARG;
  return moe::grads_call(count, tensors, true, max_norm, norm, workspace, workspace_bytes, static_cast<hipStream_t>(hip_stream));
}
