// moe_gate_backward: the gradients of the gate product score[t,e] = sum_i x[t,i] w_gate[e,i] + gate_bias[e]:
//   d_w_gate[e,:] = sum_t d_scores[t,e] x[t,:]      d_gate_bias[e] = sum_t d_scores[t,e]
//   d_x[t,:]      = sum_e d_scores[t,e] w_gate[e,:]
// x is read once and d_x written once; everything else is small beside them, so both products are HBM-bound up to about
// 128 experts and bound by the matrix instructions above.
//
// Both run on v_mfma_f32_16x16x32_bf16 with fp32 accumulators, operands straight from global memory into registers:
//   - a lane that holds V consecutive columns of 8 consecutive rows of a matrix (one load per row) turns them, with
//     byte permutes inside the lane, into the 8 values along the reduction that the instruction wants of it, for
//     V column tiles: tile i holds the columns V c + i of the lanes c = 0..15.  x (reduction over tokens) and w_gate
//     (reduction over experts) need no LDS and no transposed copy, and the V results of a lane are V consecutive
//     columns again: 16-byte stores;
//   - d_scores (fp32) enters in bf16 pieces: three that hold all its 24 bits for the weights' gradient, which is
//     stored in fp32; two (16 bits, 2^-16 of each term) for the d_x of bf16 layers, which is rounded to 8 bits.
//     fp32 layers cut x and w_gate into three pieces as well and leave out the products below 2^-22 of a term.
#include "moe_internal.h"

namespace moe {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 gb_bf16x8;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float gb_f32x4;

__device__ __forceinline__ gb_f32x4 gb_mfma(uint4 a, uint4 b, gb_f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(gb_bf16x8, a), __builtin_bit_cast(gb_bf16x8, b), c, 0, 0, 0);
}

// High halves of two words, the second one's on top.
__device__ __forceinline__ uint32_t gb_high(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
__device__ __forceinline__ uint32_t gb_low(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }

// Two fp32 values as three bf16 pieces each that add up to them exactly.  The first is cut off, so that no finite value
// becomes an infinity; what it leaves has 16 bits, the second is rounded and leaves 8 bits or fewer.
__device__ __forceinline__ void gb_split(float a, float b, uint32_t& h, uint32_t& m, uint32_t& l) {
  h = gb_high(__float_as_uint(a), __float_as_uint(b));
  a -= __uint_as_float(__float_as_uint(a) & 0xFFFF0000u);
  b -= __uint_as_float(__float_as_uint(b) & 0xFFFF0000u);
  m = pack_bf16x2(a, b);
  l = pack_bf16x2(a - bf16lo(m), b - bf16hi(m));
}

// The operand fragments of V column tiles from a lane's V columns of 8 rows along the reduction; P pieces each.
template <bool BF16, int V> struct GbFrag {
  static constexpr int P = BF16 ? 1 : 3;
  uint4 f[P][V];
};

// V consecutive elements of a row: 8 or 16 bytes.
template <bool BF16, int V> struct GbRow {
  static constexpr int W = V * (BF16 ? 2 : 4) / 4;
  uint32_t w[W];
  __device__ __forceinline__ void load(const char* p) {
    if constexpr (W == 4) {
      const uint4 v = *reinterpret_cast<const uint4*>(p);
      w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    } else {
      const uint2 v = *reinterpret_cast<const uint2*>(p);
      w[0] = v.x, w[1] = v.y;
    }
  }
  __device__ __forceinline__ void keep(bool real) {
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = real ? w[i] : 0u;
  }
};

template <bool BF16, int V> __device__ __forceinline__ void gb_transpose(const GbRow<BF16, V> (&r)[8], GbFrag<BF16, V>& o) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    uint32_t q[3][4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      if constexpr (BF16) {
        const uint32_t a = r[2 * p].w[i / 2], b = r[2 * p + 1].w[i / 2];
        q[0][p] = i % 2 ? gb_high(a, b) : gb_low(a, b);
      } else {
        gb_split(__uint_as_float(r[2 * p].w[i]), __uint_as_float(r[2 * p + 1].w[i]), q[0][p], q[1][p], q[2][p]);
      }
    }
#pragma unroll
    for (int u = 0; u < GbFrag<BF16, V>::P; ++u) o.f[u][i] = make_uint4(q[u][0], q[u][1], q[u][2], q[u][3]);
  }
}

// ------------------------------------------------------------------------------------------------ weights' gradient
// A block owns 16 V columns of x for a range of tokens and up to 16 MT experts; its waves take 32 tokens each in turn,
// keep their own sums in registers and add them up in LDS at the end.  (Waves side by side over the columns would
// share the pieces of d_scores, but leave eight times the sums to be written and read again: for 65536 tokens, d = 2048,
// 64 experts half of what x itself has.)
constexpr int GW_THREADS = 512;
constexpr int GW_WAVES = GW_THREADS / MOE_WAVE;

template <bool BF16, int MT, int V>
__global__ __launch_bounds__(GW_THREADS) void gate_weight_kernel(const char* __restrict__ x, const float* __restrict__ d_scores,
                                                                 const uint8_t* __restrict__ mask, int T, int d, int E, int tiles,
                                                                 int splits, int per_split, int accumulate,
                                                                 float* __restrict__ out_w, float* __restrict__ out_b) {
  __shared__ gb_f32x4 red[GW_WAVES][4][MOE_WAVE];
  __shared__ float red_b[GW_WAVES][16 * MT];
  constexpr int B = BF16 ? 2 : 4;
  const int lane = lane_id(), wave = threadIdx.x / MOE_WAVE, c = lane & 15, g = lane >> 4;
  // All column tiles of a token range on one XCD (blocks are dealt to the 8 XCDs in turn): its L2 then gets d_scores
  // once, and whole rows of x.
  const int chunk = blockIdx.y;
  int split, tile;
  if (splits % 8 == 0) {
    tile = blockIdx.x / 8 % tiles;
    split = blockIdx.x / 8 / tiles * 8 + blockIdx.x % 8;
  } else {
    tile = blockIdx.x % tiles;
    split = blockIdx.x / tiles;
  }
  const int e0 = chunk * 16 * MT;
  const int col = tile * 16 * V + V * c;
  const int64_t begin = static_cast<int64_t>(split) * per_split;
  const int64_t end = min(begin + per_split, static_cast<int64_t>(T));
  const char* x_lane = x + static_cast<int64_t>(min(col, d - V)) * B;
  const int64_t pitch = static_cast<int64_t>(d) * B;
  const bool with_bias = out_b && tile == 0;

  gb_f32x4 acc[MT][V];
  float bias[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    bias[m] = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) acc[m][i] = gb_f32x4{0.f, 0.f, 0.f, 0.f};
  }

  for (int64_t t0 = begin + 32 * wave; t0 < end; t0 += 32 * GW_WAVES) {
    GbRow<BF16, V> r[8];
    const int left = static_cast<int>(min(end - t0, static_cast<int64_t>(32)));     // 1 .. 32 tokens
    // bit i: token t0 + i counts
    const int at = lane & 31;
    const uint32_t real = static_cast<uint32_t>(__ballot(at < left && (!mask || mask[t0 + min(at, left - 1)])));
    if (out_w) {
#pragma unroll
      for (int j = 0; j < 8; ++j) r[j].load(x_lane + (t0 + min(8 * g + j, left - 1)) * pitch);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) r[j].keep(false);
    }
    if (real != 0xFFFFFFFFu) {
#pragma unroll
      for (int j = 0; j < 8; ++j) r[j].keep(real >> (8 * g + j) & 1);
    }
    GbFrag<BF16, V> b;
    gb_transpose<BF16, V>(r, b);
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      // rows of experts that do not exist repeat the last one's; their sums are not stored
      const float* p = d_scores + t0 * E + min(e0 + 16 * m + c, E - 1);
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = p[static_cast<int64_t>(min(8 * g + j, left - 1)) * E];
      if (real != 0xFFFFFFFFu) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = real >> (8 * g + j) & 1 ? v[j] : 0.f;
      }
      if (with_bias) {
#pragma unroll
        for (int j = 0; j < 8; ++j) bias[m] += v[j];
      }
      uint32_t q[3][4];
#pragma unroll
      for (int u = 0; u < 4; ++u) gb_split(v[2 * u], v[2 * u + 1], q[0][u], q[1][u], q[2][u]);
      const uint4 ah = make_uint4(q[0][0], q[0][1], q[0][2], q[0][3]), am = make_uint4(q[1][0], q[1][1], q[1][2], q[1][3]),
                  al = make_uint4(q[2][0], q[2][1], q[2][2], q[2][3]);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        gb_f32x4 s = acc[m][i];
        s = gb_mfma(al, b.f[0][i], s);
        if constexpr (!BF16) {
          s = gb_mfma(ah, b.f[2][i], s);
          s = gb_mfma(am, b.f[1][i], s);
        }
        s = gb_mfma(am, b.f[0][i], s);
        if constexpr (!BF16) s = gb_mfma(ah, b.f[1][i], s);
        acc[m][i] = gb_mfma(ah, b.f[0][i], s);
      }
    }
  }

  // sums of the waves, 16 experts at a time: lane 16 g + c of a wave holds experts 4 g + 0..3 of the columns V c + i
  const int64_t n = static_cast<int64_t>(E) * d;
  float* to = out_w + (splits > 1 ? split * n : 0);
  const bool add = accumulate && splits == 1;
  if (out_w) {
#pragma unroll
    for (int m = 0; m < MT; ++m) {
#pragma unroll
      for (int quad = 0; quad < V / 4; ++quad) {    // four columns of a lane at a time
        if (m + quad > 0) __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) red[wave][i][lane] = acc[m][4 * quad + i];
        __syncthreads();
        const int cc = threadIdx.x & 15, row = threadIdx.x >> 4;
        const int e = e0 + 16 * m + row, at = tile * 16 * V + V * cc + 4 * quad;
        if (row < 16 && e < E && at < d) {
          const int from = row / 4 * 16 + cc;
          float4* o = reinterpret_cast<float4*>(to + static_cast<int64_t>(e) * d + at);
          float4 s = add ? *o : make_float4(0.f, 0.f, 0.f, 0.f);
          for (int w = 0; w < GW_WAVES; ++w) {
            s.x += red[w][0][from][row % 4];
            s.y += red[w][1][from][row % 4];
            s.z += red[w][2][from][row % 4];
            s.w += red[w][3][from][row % 4];
          }
          *o = s;
        }
      }
    }
  }
  if (with_bias) {
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      float v = bias[m];
      v += __shfl_xor(v, 16);
      v += __shfl_xor(v, 32);
      if (g == 0) red_b[wave][16 * m + c] = v;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * MT; i += GW_THREADS) {
      const int e = e0 + i;
      if (e < E) {
        float v = add ? out_b[e] : 0.f;
        for (int w = 0; w < GW_WAVES; ++w) v += red_b[w][i];
        out_b[(splits > 1 ? static_cast<int64_t>(split) * E : 0) + e] = v;
      }
    }
  }
}

// out[i] (+)= the sum of the parts' elements i, in order; four consecutive ones per thread.
constexpr int GS_THREADS = 256;
__global__ __launch_bounds__(GS_THREADS) void gate_sum_kernel(const float* __restrict__ part_w, float* __restrict__ out_w, int64_t n,
                                                              const float* __restrict__ part_b, float* __restrict__ out_b, int E,
                                                              int splits, int accumulate) {
  const int64_t i = (static_cast<int64_t>(blockIdx.x) * GS_THREADS + threadIdx.x) * 4;
  if (out_w && i < n) {
    float4* o = reinterpret_cast<float4*>(out_w + i);
    float4 s = accumulate ? *o : make_float4(0.f, 0.f, 0.f, 0.f);
    for (int p = 0; p < splits; ++p) {
      const float4 v = *reinterpret_cast<const float4*>(part_w + p * n + i);
      s = make_float4(s.x + v.x, s.y + v.y, s.z + v.z, s.w + v.w);
    }
    *o = s;
  }
  if (out_b && blockIdx.x == 0 && static_cast<int>(threadIdx.x) < E) {
    float s = accumulate ? out_b[threadIdx.x] : 0.f;
    for (int p = 0; p < splits; ++p) s += part_b[static_cast<int64_t>(p) * E + threadIdx.x];
    out_b[threadIdx.x] = s;
  }
}
static_assert(GS_THREADS >= MOE_MAX_E, "one thread per expert");

// ------------------------------------------------------------------------------------------------ hidden states' gradient
// A wave keeps the fragments of w_gate of its 16 V columns (KS steps of 32 experts) in registers and runs over tokens,
// 16 at a time: d_scores in, d_x out.  The four waves of a block lie side by side.
constexpr int GX_THREADS = 256;
constexpr int GX_WAVES = GX_THREADS / MOE_WAVE;

template <bool BF16, int KS, int V>
__global__ __launch_bounds__(GX_THREADS) void gate_x_kernel(const char* __restrict__ w_gate, const float* __restrict__ d_scores,
                                                            const uint8_t* __restrict__ mask, int T, int d, int E, int tiles,
                                                            int per_split, int accumulate, char* __restrict__ d_x) {
  constexpr int B = BF16 ? 2 : 4;
  const int lane = lane_id(), wave = threadIdx.x / MOE_WAVE, c = lane & 15, g = lane >> 4;
  const int tile = static_cast<int>(blockIdx.x % tiles) * GX_WAVES + wave;
  const int col = tile * 16 * V + V * c;
  if (tile * 16 * V >= d) return;
  const int64_t begin = static_cast<int64_t>(blockIdx.x / tiles) * per_split;
  const int64_t end = min(begin + per_split, static_cast<int64_t>(T));
  const int64_t pitch = static_cast<int64_t>(d) * B;
  const char* w_lane = w_gate + static_cast<int64_t>(min(col, d - V)) * B;
  GbFrag<BF16, V> w[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    GbRow<BF16, V> r[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = 32 * s + 8 * g + j;
      r[j].load(w_lane + min(e, E - 1) * pitch);
      r[j].keep(e < E);
    }
    gb_transpose<BF16, V>(r, w[s]);
  }
  const bool whole = E % 4 == 0;                     // rows of d_scores start at multiples of 16 bytes
  for (int64_t t0 = begin; t0 < end; t0 += 16) {
    const int64_t t = min(t0 + c, end - 1);          // this lane's token of d_scores
    const bool real = !mask || mask[t];
    gb_f32x4 acc[V];
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = gb_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int e = 32 * s + 8 * g;
      const float* p = d_scores + t * E;
      float v[8];
      if (whole) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float4 q = e + 4 * h < E ? *reinterpret_cast<const float4*>(p + e + 4 * h) : make_float4(0.f, 0.f, 0.f, 0.f);
          v[4 * h] = q.x, v[4 * h + 1] = q.y, v[4 * h + 2] = q.z, v[4 * h + 3] = q.w;
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = e + j < E ? p[e + j] : 0.f;
      }
      uint32_t q[3][4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float a = real ? v[2 * u] : 0.f, b = real ? v[2 * u + 1] : 0.f;
        gb_split(a, b, q[0][u], q[1][u], q[2][u]);
      }
      const uint4 ah = make_uint4(q[0][0], q[0][1], q[0][2], q[0][3]), am = make_uint4(q[1][0], q[1][1], q[1][2], q[1][3]),
                  al = make_uint4(q[2][0], q[2][1], q[2][2], q[2][3]);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if constexpr (!BF16) {
          acc[i] = gb_mfma(al, w[s].f[0][i], acc[i]);
          acc[i] = gb_mfma(ah, w[s].f[2][i], acc[i]);
          acc[i] = gb_mfma(am, w[s].f[1][i], acc[i]);
        }
        acc[i] = gb_mfma(am, w[s].f[0][i], acc[i]);
        if constexpr (!BF16) acc[i] = gb_mfma(ah, w[s].f[1][i], acc[i]);
        acc[i] = gb_mfma(ah, w[s].f[0][i], acc[i]);
      }
    }
    // lane 16 g + c holds tokens t0 + 4 g + 0..3 of its V columns
    const uint64_t keep = __ballot(real);            // bit i of the first 16: token t0 + i counts
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int64_t to = t0 + 4 * g + r;
      if (to >= end || col >= d || (accumulate && !(keep >> (4 * g + r) & 1))) continue;
      char* o = d_x + to * pitch + static_cast<int64_t>(col) * B;
      GbRow<BF16, V> old;
      if (accumulate) old.load(o);
      if constexpr (BF16) {
        uint32_t q[V / 2];
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
          float a = acc[2 * i][r], b = acc[2 * i + 1][r];
          if (accumulate) {
            a += bf16lo(old.w[i]);
            b += bf16hi(old.w[i]);
          }
          q[i] = pack_bf16x2(a, b);
        }
        if constexpr (V == 8)
          *reinterpret_cast<uint4*>(o) = make_uint4(q[0], q[1], q[2], q[3]);
        else
          *reinterpret_cast<uint2*>(o) = make_uint2(q[0], q[1]);
      } else {
        float q[V];
#pragma unroll
        for (int i = 0; i < V; ++i) q[i] = acc[i][r] + (accumulate ? __uint_as_float(old.w[i]) : 0.f);
        if constexpr (V == 4)
          *reinterpret_cast<float4*>(o) = make_float4(q[0], q[1], q[2], q[3]);
        else
          *reinterpret_cast<float2*>(o) = make_float2(q[0], q[1]);
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------ launches
// Blocks of the weights' gradient: column tiles, groups of experts, and parts of the tokens, of which there are as many
// as fill the chip twice, each of 32 tokens per wave or more.
struct GwPlan {
  int mt, v, tiles, chunks, splits, per_split;
};
static GwPlan gw_plan(const moe_shape_t* s) {
  GwPlan p{};
  p.mt = s->E <= 16 ? 1 : s->E <= 32 ? 2 : s->E <= 64 ? 4 : 8;
  p.v = s->dtype == MOE_F32 || p.mt == 8 ? 4 : 8;
  p.tiles = (s->d + 16 * p.v - 1) / (16 * p.v);
  p.chunks = (s->E + 16 * p.mt - 1) / (16 * p.mt);
  const int64_t most = (static_cast<int64_t>(s->T) + 32 * GW_WAVES - 1) / (32 * GW_WAVES);
  int64_t n = 512 / (static_cast<int64_t>(p.tiles) * p.chunks);
  if (n > most) n = most;
  if (n > 8) n = n / 8 * 8;
  if (n < 1) n = 1;
  int64_t per = (s->T + n - 1) / n;
  per = (per + 31) / 32 * 32;
  p.per_split = static_cast<int>(per < 32 ? 32 : per);
  p.splits = static_cast<int>(n);
  return p;
}

size_t gate_backward_workspace_bytes(const moe_shape_t* shape) {
  const GwPlan p = gw_plan(shape);
  return p.splits > 1 ? static_cast<size_t>(p.splits) * shape->E * (static_cast<size_t>(shape->d) + 1) * sizeof(float) : 0;
}

template <bool BF16>
static void launch_weight(const GwPlan& p, const moe_shape_t* s, const void* x, const float* ds, const uint8_t* mask, int accumulate,
                          float* out_w, float* out_b, hipStream_t st) {
  constexpr int V8 = BF16 ? 8 : 4;
  const auto kernel = p.mt == 1 ? gate_weight_kernel<BF16, 1, V8> : p.mt == 2 ? gate_weight_kernel<BF16, 2, V8>
                    : p.mt == 4 ? gate_weight_kernel<BF16, 4, V8> : gate_weight_kernel<BF16, 8, 4>;
  hipLaunchKernelGGL(kernel, dim3(p.tiles * p.splits, p.chunks), dim3(GW_THREADS), 0, st, static_cast<const char*>(x), ds, mask, s->T,
                     s->d, s->E, p.tiles, p.splits, p.per_split, accumulate, out_w, out_b);
}

template <bool BF16>
static void launch_x(const moe_shape_t* s, const void* w, const float* ds, const uint8_t* mask, int accumulate, void* d_x, hipStream_t st) {
  constexpr int V8 = BF16 ? 8 : 4, V4 = BF16 ? 4 : 2;
  const int ks = s->E <= 32 ? 1 : s->E <= 64 ? 2 : s->E <= 128 ? 4 : 8;
  const int v = ks <= 2 ? V8 : V4;
  const auto kernel = ks == 1 ? gate_x_kernel<BF16, 1, V8> : ks == 2 ? gate_x_kernel<BF16, 2, V8>
                    : ks == 4 ? gate_x_kernel<BF16, 4, V4> : gate_x_kernel<BF16, 8, V4>;
  const int tiles = (s->d + 16 * v * GX_WAVES - 1) / (16 * v * GX_WAVES);
  int64_t splits = 2048 / tiles;
  const int64_t most = (static_cast<int64_t>(s->T) + 15) / 16;
  if (splits > most) splits = most;
  if (splits < 1) splits = 1;
  int64_t per = (s->T + splits - 1) / splits;
  per = (per + 15) / 16 * 16;
  splits = (s->T + per - 1) / per;
  hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(tiles * splits)), dim3(GX_THREADS), 0, st, static_cast<const char*>(w), ds, mask,
                     s->T, s->d, s->E, tiles, static_cast<int>(per), accumulate, static_cast<char*>(d_x));
}

template <bool BF16>
static int gate_backward(const moe_shape_t* shape, const void* x, const void* w_gate, const float* d_scores, const uint8_t* mask,
                         float* d_w_gate, float* d_gate_bias, void* d_x, int accumulate, float* part, hipStream_t st) {
  const int acc_w = accumulate & MOE_ACCUMULATE_WEIGHTS ? 1 : 0, acc_x = accumulate & MOE_ACCUMULATE_X ? 1 : 0;
  if (d_w_gate || d_gate_bias) {
    const GwPlan p = gw_plan(shape);
    const int64_t n = static_cast<int64_t>(shape->E) * shape->d;
    const bool parts = p.splits > 1;
    float* part_b = part + p.splits * n;
    launch_weight<BF16>(p, shape, x, d_scores, mask, acc_w, d_w_gate ? (parts ? part : d_w_gate) : nullptr,
                        d_gate_bias ? (parts ? part_b : d_gate_bias) : nullptr, st);
    if (parts) {
      const int64_t threads = d_w_gate ? n / 4 : 1;
      hipLaunchKernelGGL(gate_sum_kernel, dim3(static_cast<unsigned>((threads + GS_THREADS - 1) / GS_THREADS)), dim3(GS_THREADS), 0, st, part,
                         d_w_gate, n, part_b, d_gate_bias, shape->E, p.splits, acc_w);
    }
  }
  if (d_x && shape->T > 0) launch_x<BF16>(shape, w_gate, d_scores, mask, acc_x, d_x, st);
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
