// moe_grad_norm, moe_clip_grads: the Euclidean norm of a list of tensors taken together, and the tensors scaled to a
// largest norm:  norm = sqrt(sum over all elements of g^2),  out = g * min(1, max_norm / norm).
// HBM-bound: every element is read once for the norm, and once more with a write for the scaling.  (Measured: 60 tensors
// of 5 to 14336 x 4096 elements, 844 MB of fp32 and bf16, 447 us, of it the norm 143 = 5.9 TB/s and the scaling 300 =
// 5.6 TB/s read and written; 32 tensors of 512 KiB 11.6 us.)
//
// The list travels in the kernels' arguments, so no table has to reach the device first and a captured graph holds its
// own copy.  Every block takes one piece of one tensor.  Squares and their sums are 64-bit (an fp32 square overflows
// from 1.8e19 on and loses all bits below 1e-23); a block leaves one sum in the workspace and one block adds those in
// a fixed order.
#include "moe_internal.h"

namespace moe {

constexpr int GR_THREADS = 256;
constexpr int GR_TENSORS = 128;        // tensors of one launch
// Least elements of a piece (all pieces of a call have the same size), and the pieces of a call that is large enough: small
// pieces fill the chip, few of them are less to add up, which every block does.  (Measured, pieces of 4096 / 8192 / 16384,
// us: one tensor of 100000 5.9 / 6.4 / 7.1, 32 of 131072 12.4 / 11.6 / 11.5, 40 of up to 2000000 22.9 / 20.8 / 20.4.
// 2048 / 4096 / 8192 pieces: 844 MB 470 / 459 / 446, 512 MiB of bf16 282 / 281 / 288.)
constexpr int64_t GR_PIECE = 8192;
constexpr int64_t GR_PIECES = 4096;

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

// Piece b of the table: of the last tensor whose first block is not behind it (tensors without elements have no block).
__device__ __forceinline__ GradPiece grad_piece(const GradTable& tab, int count, int64_t piece, int b) {
  int lo = 0, hi = count - 1;
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

// The elements [begin, end) of a tensor: those in whole, aligned 16-byte chunks by `chunk`(pointer to it, its first
// element's number), the others, at most 7 at either end, by `one`(number).  LAST: nothing is read again.  (The scaling's
// loads marked so, us: 844 MB 458 -> 447, 512 MiB of bf16 280 -> 270, 40 tensors of up to 2000000 21.0 -> 20.4.)
template <bool BF16, bool LAST, class Chunk, class One>
__device__ __forceinline__ void grad_for_each(const GradPiece& g, Chunk chunk, One one) {
  constexpr int PER = BF16 ? 8 : 4, UNROLL = 4;
  const int64_t skip = -static_cast<int64_t>(reinterpret_cast<uintptr_t>(g.data) / (16 / PER)) & (PER - 1);   // elements before an aligned one
  int64_t first = (g.begin - skip + PER - 1) / PER * PER + skip, last = (g.end - skip) / PER * PER + skip;
  if (g.begin <= skip) first = skip;
  if (first >= last) first = last = g.end;
  if (g.begin + threadIdx.x < first) one(g.begin + threadIdx.x);
  if (last + threadIdx.x < g.end) one(last + threadIdx.x);
  const int64_t n = (last - first) / PER;
  const uint4* p = reinterpret_cast<const uint4*>(static_cast<const char*>(g.data) + first * (16 / PER));
  int64_t i = threadIdx.x;
  for (; i + (UNROLL - 1) * GR_THREADS < n; i += UNROLL * GR_THREADS) {
    uint4 v[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) v[u] = LAST ? nt_load(p + i + u * GR_THREADS) : p[i + u * GR_THREADS];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) chunk(v[u], first + (i + u * GR_THREADS) * PER);
  }
  for (; i < n; i += GR_THREADS) chunk(p[i], first + i * PER);
}

// Sum over the block, in a fixed order, on every thread.
__device__ __forceinline__ double grad_block_sum(double v, double* lds) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off);
  if (lane_id() == 0) lds[threadIdx.x / MOE_WAVE] = v;
  __syncthreads();
  v = 0.0;
#pragma unroll
  for (int w = 0; w < GR_THREADS / MOE_WAVE; ++w) v += lds[w];
  return v;
}

template <bool BF16> __device__ __forceinline__ double grad_squares(const GradPiece& g) {
  double s[4] = {};
  auto add = [&](int k, float f) {
    const double d = f;
    s[k & 3] = fma(d, d, s[k & 3]);
  };
  grad_for_each<BF16, false>(
      g,
      [&](uint4 v, int64_t) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if constexpr (BF16) {
            add(2 * k, bf16lo(w[k]));
            add(2 * k + 1, bf16hi(w[k]));
          } else {
            add(k, __uint_as_float(w[k]));
          }
        }
      },
      [&](int64_t i) { add(0, BF16 ? bf16_to_f32(static_cast<const bf16_t*>(g.data)[i]) : static_cast<const float*>(g.data)[i]); });
  return (s[0] + s[1]) + (s[2] + s[3]);
}

__global__ __launch_bounds__(GR_THREADS) void grad_square_kernel(GradTable tab, int count, int64_t piece, double* __restrict__ part) {
  __shared__ double lds[GR_THREADS / MOE_WAVE];
  const GradPiece g = grad_piece(tab, count, piece, blockIdx.x);
  const double s = grad_block_sum(g.bf16 ? grad_squares<true>(g) : grad_squares<false>(g), lds);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// The norm from the pieces' sums, the same on every thread of every block.
__device__ __forceinline__ double grad_total_norm(const double* __restrict__ part, int64_t pieces, double* lds) {
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < pieces; i += GR_THREADS) s += part[i];
  return sqrt(grad_block_sum(s, lds));
}

__global__ __launch_bounds__(GR_THREADS) void grad_finish_kernel(const double* __restrict__ part, int64_t pieces, float* __restrict__ norm) {
  __shared__ double lds[GR_THREADS / MOE_WAVE];
  const double s = grad_total_norm(part, pieces, lds);
  if (threadIdx.x == 0) *norm = static_cast<float>(s);
}

template <bool BF16, class C> __device__ __forceinline__ void grad_scale(const GradPiece& g, C c) {
  auto times = [&](float v) { return static_cast<float>(v * c); };
  auto one = [&](int64_t i) {
    if constexpr (BF16)
      static_cast<bf16_t*>(g.out)[i] = f32_to_bf16(times(bf16_to_f32(static_cast<const bf16_t*>(g.data)[i])));
    else
      static_cast<float*>(g.out)[i] = times(static_cast<const float*>(g.data)[i]);
  };
  if ((reinterpret_cast<uintptr_t>(g.out) ^ reinterpret_cast<uintptr_t>(g.data)) & 15) {   // no common alignment
    for (int64_t i = g.begin + threadIdx.x; i < g.end; i += GR_THREADS) one(i);
    return;
  }
  grad_for_each<BF16, true>(
      g,
      [&](uint4 v, int64_t i) {
        uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k)
          w[k] = BF16 ? pack_bf16x2(times(bf16lo(w[k])), times(bf16hi(w[k]))) : __float_as_uint(times(__uint_as_float(w[k])));
        nt_store(reinterpret_cast<uint4*>(static_cast<char*>(g.out) + i * (BF16 ? 2 : 4)), make_uint4(w[0], w[1], w[2], w[3]));
      },
      one);
}

// Every block makes the factor from the pieces' sums by itself, which saves a launch.  The pieces are taken from the last
// eight to the first: what the norm's pass read last is in the memory-side cache, and in the L2 of the XCD that block b
// of both passes runs on (b % 8).  The grid is a multiple of 8.  (Measured, first to last / last to first, us: 844 MB 486 /
// 459, 512 MiB of bf16 301 / 281.  What is written is not read soon and goes past the L2: with ordinary stores 490, 312.)
__global__ __launch_bounds__(GR_THREADS) void grad_scale_kernel(GradTable tab, int count, int blocks, int64_t piece, const double* __restrict__ part,
                                                                int64_t pieces, double max_norm, float* __restrict__ norm) {
  __shared__ double lds[GR_THREADS / MOE_WAVE];
  const double s = grad_total_norm(part, pieces, lds);
  if (blockIdx.x == 0 && threadIdx.x == 0) *norm = static_cast<float>(s);
  // 1 where `norm`, which the caller sees, is no finite number
  const double exact = s > max_norm && static_cast<float>(s) < INFINITY ? max_norm / s : 1.0;
  const float c = static_cast<float>(exact);
  const int b = (gridDim.x / 8 - 1 - blockIdx.x / 8) * 8 + blockIdx.x % 8;
  if (b >= blocks) return;
  const GradPiece g = grad_piece(tab, count, piece, b);
  if (c == 1.f && g.out == g.data) return;
  if (exact > 0.0 && exact < 0x1p-126) {             // few bits of it, or none, are left in 32
    if (g.bf16)
      grad_scale<true>(g, exact);
    else
      grad_scale<false>(g, exact);
  } else if (g.bf16) {
    grad_scale<true>(g, c);
  } else {
    grad_scale<false>(g, c);
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

// One 64-bit sum per piece.
static size_t grad_workspace_bytes(int64_t pieces) { return pieces > 0 ? (static_cast<size_t>(pieces) * 8 + 255) / 256 * 256 : 256; }

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
  if (workspace_bytes < grad_workspace_bytes(pieces)) return MOE_ERR_WORKSPACE;
  double* part = static_cast<double*>(workspace);
  int64_t at = 0;
  for_tables(count, tensors, piece, [&](const GradTable& tab, int n, int blocks) {
    hipLaunchKernelGGL(grad_square_kernel, dim3(blocks), dim3(GR_THREADS), 0, st, tab, n, piece, part + at);
    at += blocks;
  });
  if (clip && pieces > 0)
    for_tables(count, tensors, piece, [&](const GradTable& tab, int n, int blocks) {
      hipLaunchKernelGGL(grad_scale_kernel, dim3((blocks + 7) / 8 * 8), dim3(GR_THREADS), 0, st, tab, n, blocks, piece, part, pieces, max_norm, norm);
    });
  else
    hipLaunchKernelGGL(grad_finish_kernel, dim3(1), dim3(GR_THREADS), 0, st, part, pieces, norm);
  return launch_status();
}

}  // namespace moe

extern "C" int moe_grad_workspace_bytes(int32_t count, const moe_tensor_t* tensors, size_t* out_bytes) {
  const int rc = moe::check_grads(count, tensors, false);
  if (rc != MOE_OK) return rc;
  if (!out_bytes) return MOE_ERR_INVALID_ARG;
  int64_t piece = 0;
  *out_bytes = moe::grad_workspace_bytes(moe::grad_pieces(count, tensors, &piece));
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
