// The losses that a gate is trained with, and their gradients with respect to its scores s [T,E]:
//   moe_balance_loss    counts c_e and probability sums P_e = sum_t p[t,e], p = softmax_E(s);
//                       L = E k sum_e c_e P_e / (sum c)^2
//   moe_route_backward  the gradient of the routing weights and of coef * L
//   moe_gate_distill    the mean over tokens of KL(softmax(target) || p), and its gradient
// All three stream tables of T x E floats once: HBM-bound for large batches, launch-bound for small ones.  (Measured, in
// a captured graph, 65536 tokens: distill with a gradient, 128 experts, 100 MB, 23.8 us, of it 4 for the sum of the loss,
// and 28 with a mask; balance and its gradient, 64 experts, 52 MB, 19.4 us in three launches; route backward, 128
// experts, k = 8, 71 MB, 16.2 us = 4.4 TB/s.  A single small call takes 4 to 6 us.)
//
// G lanes share a token, the least power of two with 4 G >= E; a lane holds four scores: consecutive ones in one load if
// E is a multiple of 4 (VEC), those of experts l, l + G, ... otherwise.  So a wave reads 64 / G neighbouring rows at a
// time, 1 KiB in one piece, whatever E is, and the sums over a row take log2(G) steps between lanes.
//
// Powers are taken of 2: with m the row's maximum and c = log2(e), e^(s-m) = 2^(c s - c m) is one fused multiply-add
// (rounded once) and one v_exp_f32.  The rounding of c m is the same for a whole row and divides out of p, as long as
// it is small: from |m| of some 1e9 on it is more than what a power of 2 can hold (GL_FAR).
#include <type_traits>

#include "moe_internal.h"

namespace moe {

constexpr int GL_SUM_THREADS = 1024;  // of a block that leaves a row of sums, and of the block that adds these rows
constexpr int GL_THREADS = 256;       // of the others
constexpr float GL_LOG2E = 1.44269504088896340736f;
constexpr float GL_LN2 = 0.693147180559945309417f;

// Sum and maximum over the G lanes of a token, on each of them: DPP steps inside a row of 16 lanes (xor 1, xor 2, then
// the mirrors of 8 and of 16, as the lanes that they join hold equal values by then), beyond it swaps, which leave the
// even rows' (the lower half's) values in one register and the odd rows' (the upper half's) in the other.
template <int CTRL> __device__ __forceinline__ float gl_dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
template <int G, class Op> __device__ __forceinline__ float gl_reduce(float v, Op op) {
  if constexpr (G >= 2) v = op(v, gl_dpp<0xB1>(v));      // quad_perm [1,0,3,2]
  if constexpr (G >= 4) v = op(v, gl_dpp<0x4E>(v));      // quad_perm [2,3,0,1]
  if constexpr (G >= 8) v = op(v, gl_dpp<0x141>(v));     // row_half_mirror
  if constexpr (G >= 16) v = op(v, gl_dpp<0x140>(v));    // row_mirror
  if constexpr (G >= 32) {
    const auto q = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(__uint_as_float(q[0]), __uint_as_float(q[1]));
  }
  if constexpr (G >= 64) {
    const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(__uint_as_float(q[0]), __uint_as_float(q[1]));
  }
  return v;
}
template <int G> __device__ __forceinline__ float gl_sum(float v) {
  return gl_reduce<G>(v, [](float a, float b) { return a + b; });
}
template <int G> __device__ __forceinline__ float gl_max(float v) {
  return gl_reduce<G>(v, [](float a, float b) { return fmaxf(a, b); });
}

// The expert of value j of lane l of a token.
template <int G, bool VEC> __device__ __forceinline__ int gl_expert(int l, int j) { return VEC ? 4 * l + j : l + G * j; }

// Row `row` of a block's rows of a table of `width` columns of 4 bytes.  (The block's rows have less than 2^32 bytes, being
// 1/256 of a table at most, and number less than 2^24: the table's address stays in scalar registers.)
template <class V> __device__ __forceinline__ V* gl_row(V* rows, int row, int width, int column) {
  const uint32_t at = __umul24(row, 4 * width) + 4 * column;
  if constexpr (std::is_const<V>::value)
    return reinterpret_cast<V*>(reinterpret_cast<const char*>(rows) + at);
  else
    return reinterpret_cast<V*>(reinterpret_cast<char*>(rows) + at);
}

// A lane's four values of a row of a table, `fill` past the last expert.  (No load is behind a branch: lanes past the end
// read the last values again.  The compiler counts on no load that a branch may skip, and would wait for all of them.)
template <int G, bool VEC>
__device__ __forceinline__ void gl_load(const float* __restrict__ rows, int row, int E, int l, float fill, float (&v)[4]) {
  if constexpr (VEC) {
    const float4 q = *reinterpret_cast<const float4*>(gl_row(rows, row, E, min(4 * l, E - 4)));
    const bool there = 4 * l < E;
    v[0] = there ? q.x : fill, v[1] = there ? q.y : fill, v[2] = there ? q.z : fill, v[3] = there ? q.w : fill;
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int e = l + G * j;
      v[j] = *gl_row(rows, row, E, min(e, E - 1));
      v[j] = e < E ? v[j] : fill;
    }
  }
}

template <int G, bool VEC> __device__ __forceinline__ void gl_store(float* __restrict__ rows, int row, int E, int l, const float (&v)[4]) {
  if constexpr (VEC) {
    if (4 * l < E) *reinterpret_cast<float4*>(gl_row(rows, row, E, 4 * l)) = make_float4(v[0], v[1], v[2], v[3]);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int e = l + G * j;
      if (e < E) *gl_row(rows, row, E, e) = v[j];
    }
  }
}

// The exponents c (s - m) of a row with the maximum m.  Beyond GL_FAR, up to which the rounding of c m is 2^-8 at most, m is
// subtracted first; m = -inf: every s is, and so are the exponents.  Returns m's own exponent, what is left of c m.
constexpr float GL_FAR = 65536.f;
__device__ __forceinline__ float gl_exponents(const float (&s)[4], float m, float (&t)[4]) {
  const bool far = fabsf(m) > GL_FAR;
  float scaled = GL_LOG2E * m, top = m;
#pragma unroll
  for (int j = 0; j < 4; ++j) t[j] = s[j];
  if (__any(far)) {                                  // rarely
    const float shift = far && m > -INFINITY ? m : 0.f;
    scaled = far ? 0.f : scaled;
    top -= shift;
#pragma unroll
    for (int j = 0; j < 4; ++j) t[j] -= shift;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) t[j] = fmaf(GL_LOG2E, t[j], -scaled);
  return fmaf(GL_LOG2E, top, -scaled);
}

// The powers v divided by their sum, zeros where there is none: v_rcp_f32 and a step of correction, so that what is alone in
// its sum becomes 1.
__device__ __forceinline__ void gl_divide(float (&v)[4], float sum, bool some) {
  const float inv = some ? __builtin_amdgcn_rcpf(sum) : 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float q = v[j] * inv;
    v[j] = fmaf(fmaf(-q, sum, v[j]), inv, q);
  }
}

// Logarithms (of base 2) of a row's probabilities, and of the largest, that of the score m.
struct GlLogs {
  float p[4], m, top;
};

// p = softmax of a row, zeros where every score is -inf, NaN where one is NaN (which a maximum does not show).  Returns
// whether anything is left of the row.
template <int G> __device__ __forceinline__ bool gl_softmax(const float (&s)[4], float (&p)[4], GlLogs* logs = nullptr) {
  const float m = gl_max<G>(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])));
  float t[4];
  const float top = gl_exponents(s, m, t);
#pragma unroll
  for (int j = 0; j < 4; ++j) p[j] = __builtin_amdgcn_exp2f(t[j]);
  const float sum = gl_sum<G>((p[0] + p[1]) + (p[2] + p[3]));
  const bool some = sum != 0.f;
  gl_divide(p, sum, some);
  if (logs) {
    // the logarithm of a sum of one power is its exponent
    const float log2sum = sum == __builtin_amdgcn_exp2f(top) ? top : __builtin_amdgcn_logf(some ? sum : 1.f);
#pragma unroll
    for (int j = 0; j < 4; ++j) logs->p[j] = t[j] - log2sum;
    logs->m = m;
    logs->top = top - log2sum;
  }
  return some;
}

// Sum over the block of one value per thread, in a fixed order, on every thread.  lds: one value per wave.
template <class V> __device__ __forceinline__ V gl_block_sum(V v, V* lds) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off);
  __syncthreads();
  if (lane_id() == 0) lds[threadIdx.x / MOE_WAVE] = v;
  __syncthreads();
  v = 0;
  for (int w = 0; w < static_cast<int>(blockDim.x / MOE_WAVE); ++w) v += lds[w];
  return v;
}

// A block's rows: the first one, and their number.
struct GlRows {
  int64_t begin;
  int n;
  __device__ __forceinline__ GlRows(int T, int per_block)
      : begin(static_cast<int64_t>(blockIdx.x) * per_block), n(static_cast<int>(min(static_cast<int64_t>(per_block), T - begin))) {}
};

// The n > 0 rows of a block, in turns of its waves, 64 / G rows at a time: load(data, row), then use(data, row, whether there
// is such a row, whether it counts); rows are counted from the block's first, as are the bytes of `mask`.  The loads of a
// turn are on their way during the turn before, those of the first during `first`; past the end the last row is read again.
// `table`: n bytes or more, read where there is no mask.  (Two batches of rows to a turn: route backward of 65536 tokens, 64
// experts 12.7 us instead of 12.0, of 4096 tokens, 128 experts 4.9 instead of 4.5.)
template <int G, class Data, class Load, class First, class Use>
__device__ __forceinline__ void gl_rows(int n, const uint8_t* __restrict__ mask, const void* table, Load load, First first, Use use) {
  constexpr int ROWS = MOE_WAVE / G;
  struct Turn {
    Data data;
    uint8_t mask;
  };
  const uint8_t* some_bytes = mask ? mask : static_cast<const uint8_t*>(table);
  auto start = [&](Turn& next, int t0) {
    const int row = min(t0 + lane_id() / G, n - 1);
    next.mask = some_bytes[static_cast<uint32_t>(row)];
    load(next.data, row);
  };
  const int step = blockDim.x / MOE_WAVE * ROWS;
  int t0 = __builtin_amdgcn_readfirstlane(threadIdx.x / MOE_WAVE) * ROWS;
  Turn now;
  start(now, t0);
  first();
  while (t0 < n) {
    Turn next;
    start(next, t0 + step);
    const int t = t0 + lane_id() / G;
    use(now.data, t, t < n, t < n && (!mask || now.mask));
    now = next;
    t0 += step;
  }
}

// A block's row of sums in the workspace, whole 16-byte chunks.
constexpr int gl_part_pitch(int E) { return (E + 3) / 4 * 4; }

// The loss from c_e and c_e P_e of expert e on thread e, 0 on threads without an expert.
__device__ __forceinline__ void gl_finish_loss(double total, double dot, int E, int k, double (&lds)[2][MOE_MAX_E / MOE_WAVE], float* __restrict__ loss) {
  const int wave = threadIdx.x / MOE_WAVE;
  if (wave < MOE_MAX_E / MOE_WAVE) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) {
      total += __shfl_xor(total, off);
      dot += __shfl_xor(dot, off);
    }
    if (lane_id() == 0) lds[0][wave] = total, lds[1][wave] = dot;
  }
  __syncthreads();
  if (threadIdx.x != 0) return;
  total = (lds[0][0] + lds[0][1]) + (lds[0][2] + lds[0][3]);
  dot = (lds[1][0] + lds[1][1]) + (lds[1][2] + lds[1][3]);
  *loss = total > 0.0 ? static_cast<float>(dot * E * k / (total * total)) : 0.f;
}
static_assert(MOE_MAX_E == 4 * MOE_WAVE, "four waves of experts");

// Counts and sums of a block's rows.  A single block finishes by itself (part_p is then not used), others leave a row of
// the workspace each.
template <int G, bool VEC>
__global__ __launch_bounds__(GL_SUM_THREADS) void balance_kernel(const float* __restrict__ scores, const int32_t* __restrict__ topk_idx,
                                                             const uint8_t* __restrict__ mask, int T, int E, int k, int per_block,
                                                             float* __restrict__ part_p, int32_t* __restrict__ part_c,
                                                             int32_t* __restrict__ counts, float* __restrict__ prob_sum,
                                                             float* __restrict__ loss) {
  constexpr int WAVES = GL_SUM_THREADS / MOE_WAVE;
  __shared__ float sum_p[WAVES][MOE_MAX_E];
  __shared__ int32_t cnt[MOE_MAX_E];
  __shared__ double sums[2][MOE_MAX_E / MOE_WAVE];
  const int lane = lane_id(), wave = threadIdx.x / MOE_WAVE, l = lane % G;
  if (threadIdx.x < MOE_MAX_E) cnt[threadIdx.x] = 0;
  __syncthreads();
  float acc[4] = {};
  struct Row {
    float s[4];
  };
  const GlRows rows(T, per_block);
  scores += rows.begin * E;
  topk_idx += rows.begin * k;
  if (mask) mask += rows.begin;
  gl_rows<G, Row>(
      rows.n, mask, scores, [&](Row& r, int t) { gl_load<G, VEC>(scores, t, E, l, -INFINITY, r.s); },
      [&] {
        const uint32_t choices = static_cast<uint32_t>(rows.n) * k;      // T k < 2^31
        for (uint32_t a = threadIdx.x; a < choices; a += GL_SUM_THREADS) {
          const int e = topk_idx[a];
          if ((!mask || mask[a / k]) && static_cast<unsigned>(e) < static_cast<unsigned>(E)) atomicAdd(&cnt[e], 1);
        }
      },
      [&](Row& r, int, bool, bool real) {
        float p[4];
        gl_softmax<G>(r.s, p);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] += real ? p[j] : 0.f;
      });
#pragma unroll
  for (int off = G; off < MOE_WAVE; off <<= 1)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] += __shfl_xor(acc[j], off);
  if (lane < G) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int e = gl_expert<G, VEC>(l, j);
      if (e < E) sum_p[wave][e] = acc[j];
    }
  }
  __syncthreads();
  const int e = threadIdx.x;
  float v = 0.f;
  int32_t c = 0;
  if (e < E) {
    for (int w = 0; w < WAVES; ++w) v += sum_p[w][e];
    c = cnt[e];
  }
  if (gridDim.x > 1) {
    const int pitch = gl_part_pitch(E);
    if (e < pitch) {
      part_p[blockIdx.x * pitch + e] = v;
      part_c[blockIdx.x * pitch + e] = c;
    }
    return;
  }
  if (e < E) {
    counts[e] = c;
    prob_sum[e] = v;
  }
  gl_finish_loss(static_cast<double>(c), static_cast<double>(c) * v, E, k, sums, loss);
}

// Adds the blocks' rows: L lanes of a wave (a power of two) for the experts of a row, four to a lane, so that a wave has
// 64 / L rows at a time; the waves' sums meet in LDS.
__global__ __launch_bounds__(GL_SUM_THREADS) void balance_finish_kernel(const float* __restrict__ part_p,
                                                                        const int32_t* __restrict__ part_c, int blocks, int E,
                                                                        int k, int L, int32_t* __restrict__ counts,
                                                                        float* __restrict__ prob_sum, float* __restrict__ loss) {
  constexpr int WAVES = GL_SUM_THREADS / MOE_WAVE;
  __shared__ double sp[WAVES][MOE_MAX_E];
  __shared__ int32_t sc[WAVES][MOE_MAX_E];
  __shared__ double sums[2][MOE_MAX_E / MOE_WAVE];
  const int lane = lane_id(), wave = threadIdx.x / MOE_WAVE, l = lane & (L - 1), pitch = gl_part_pitch(E);
  const int rows = GL_SUM_THREADS / L;
  double p[4] = {};
  int32_t c[4] = {};
  if (4 * l < E)
    for (int b = threadIdx.x / L; b < blocks; b += 4 * rows) {
      float4 vp[4];
      int4 vc[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int at = (b + u * rows) * pitch + 4 * l;
        const bool there = b + u * rows < blocks;
        vp[u] = there ? *reinterpret_cast<const float4*>(part_p + at) : make_float4(0.f, 0.f, 0.f, 0.f);
        vc[u] = there ? *reinterpret_cast<const int4*>(part_c + at) : make_int4(0, 0, 0, 0);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        p[0] += vp[u].x, p[1] += vp[u].y, p[2] += vp[u].z, p[3] += vp[u].w;
        c[0] += vc[u].x, c[1] += vc[u].y, c[2] += vc[u].z, c[3] += vc[u].w;
      }
    }
  for (int off = L; off < MOE_WAVE; off <<= 1)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      p[j] += __shfl_xor(p[j], off);
      c[j] += __shfl_xor(c[j], off);
    }
  if (lane < L && 4 * l < E)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      sp[wave][4 * l + j] = p[j];
      sc[wave][4 * l + j] = c[j];
    }
  __syncthreads();
  const int e = threadIdx.x;
  double sum = 0.0;
  int32_t count = 0;
  if (e < E)
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      sum += sp[w][e];
      count += sc[w][e];
    }
  if (e < E) {
    counts[e] = count;
    prob_sum[e] = static_cast<float>(sum);
  }
  gl_finish_loss(static_cast<double>(count), count * sum, E, k, sums, loss);
}

// ds = gradient of sum_j d_topk_w[j] w_j (w: the routing weights of moe_route) + gradient of coef * L.
//   renorm 0: w_j = p[i_j]:                 ds_e = p_e (g_e - sum_l p_l g_l),  g_e = sum of d_topk_w[j] with i_j = e
//   renorm 1: w = softmax over the chosen:  ds[i_j] = w_j (d_topk_w[j] - sum_l w_l d_topk_w[l])
//   balance:  b_e = coef E k c_e / (sum c)^2, ds_e = p_e (b_e - sum_l p_l b_l);  as the p_l add up to 1 a constant may be
//             taken off the b_e, their mean: what is left of even loads is then not the rounding of large numbers
// Every lane finds out, for its experts, how often each was chosen (n_e) and g_e.
// renorm 1 needs no more: with v_e = e^(s_e) / sum_l n_l e^(s_l),  ds_e = v_e (g_e - n_e sum_l v_l g_l) where n_e > 0.
// Q: choices per lane, 0 without d_topk_w.  ACC: d_scores is added to.
//
// Up to one choice per lane, the choices' lanes write their numbers into a table of the wave's tokens and experts in LDS, from
// which every lane reads who chose its experts; where a lane does not find its own number an expert was chosen twice, and
// the wave goes through the choices one after the other, as it does for more choices.  (Measured, one after the other /
// table, us: 65536 tokens, 128 experts, k = 8 24.2 / 18.2, renorm 1 28.2 / 22.0; 64, 6 13.9 / 11.7; 8 experts, two lanes
// to a token, k = 2 4.4 / 4.6.)
constexpr int GL_TABLE_FROM = 4;       // lanes of a token
template <int G, bool VEC, int Q, bool ACC>
__global__ __launch_bounds__(GL_THREADS) void route_backward_kernel(const float* __restrict__ scores,
                                                                    const int32_t* __restrict__ topk_idx,
                                                                    const float* __restrict__ d_topk_w,
                                                                    const int32_t* __restrict__ counts, float coef,
                                                                    const uint8_t* __restrict__ mask, int T, int E, int k,
                                                                    int renorm, int per_block, float* __restrict__ d_scores) {
  __shared__ __align__(16) int table[Q == 1 && G >= GL_TABLE_FROM ? GL_THREADS / MOE_WAVE : 1][4 * MOE_WAVE];
  const int lane = lane_id(), l = lane % G;
  float b[4] = {};
  const bool with_p = counts || !renorm;             // the softmax over all experts has a part in it
  struct Row {
    float s[4], old[4], d[Q > 0 ? Q : 1];
    int e[Q > 0 ? Q : 1];
  };
  const GlRows rows(T, per_block);
  scores += rows.begin * E;
  d_scores += rows.begin * E;
  if (Q > 0) topk_idx += rows.begin * k, d_topk_w += rows.begin * k;
  if (mask) mask += rows.begin;
  gl_rows<G, Row>(
      rows.n, mask, scores,
      [&](Row& r, int t) {
        gl_load<G, VEC>(scores, t, E, l, -INFINITY, r.s);
        if constexpr (ACC) gl_load<G, VEC>(d_scores, t, E, l, 0.f, r.old);
        // choices l, l + G, ... of the token are on lane l: k <= E <= 4 G
#pragma unroll
        for (int q = 0; q < Q; ++q) {
          const int choice = min(l + G * q, k - 1);
          r.e[q] = *gl_row(topk_idx, t, k, choice);
          r.d[q] = *gl_row(d_topk_w, t, k, choice);
        }
      },
      [&] {
        if (!counts) return;
        int64_t total = 0;
        for (int e = lane; e < E; e += MOE_WAVE) total += counts[e];
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) total += __shfl_xor(total, off);
        const double n = static_cast<double>(total), c = total > 0 ? static_cast<double>(coef) * k / (n * n) : 0.0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int e = gl_expert<G, VEC>(l, j);
          if (e < E) b[j] = static_cast<float>(c * static_cast<double>(static_cast<int64_t>(counts[e]) * E - total));
        }
      },
      [&](Row& r, int t, bool there, bool real) {
        float p[4], d[4] = {}, g[4] = {}, times[4] = {};
        bool distinct = false;
        if constexpr (Q == 1 && G >= GL_TABLE_FROM) {
          const bool chooses = l < k && static_cast<unsigned>(r.e[0]) < static_cast<unsigned>(E);
          int* mine = &table[threadIdx.x / MOE_WAVE][lane / G * (4 * G)];
          *reinterpret_cast<int4*>(mine + 4 * l) = make_int4(-1, -1, -1, -1);
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
          if (chooses) mine[r.e[0]] = lane;
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
          distinct = !__any(chooses && mine[r.e[0]] != lane);
          int from[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) from[j] = mine[gl_expert<G, VEC>(l, j)];
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float v = __shfl(r.d[0], from[j]);
            times[j] = from[j] >= 0 ? 1.f : 0.f;
            g[j] = from[j] >= 0 ? v : 0.f;
          }
        }
        if (!distinct) {
#pragma unroll
          for (int j = 0; j < 4; ++j) g[j] = times[j] = 0.f;
#pragma unroll
          for (int q = 0; q < Q; ++q) {
            const int n = min(k - G * q, G);         // the same for all lanes
            if (static_cast<unsigned>(r.e[q]) >= static_cast<unsigned>(E)) r.e[q] = -1;
            for (int i = 0; i < n; ++i) {
              const int e = __shfl(r.e[q], (lane & ~(G - 1)) + i);
              const float v = __shfl(r.d[q], (lane & ~(G - 1)) + i);
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const bool same = e == gl_expert<G, VEC>(l, j);
                g[j] += same ? v : 0.f;
                times[j] += same ? 1.f : 0.f;
              }
            }
          }
        }
        if (Q > 0 && renorm) {
          float v[4], t[4], sum = 0.f;
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] = times[j] > 0.f ? r.s[j] : -INFINITY;
          const float m = gl_max<G>(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])));
          gl_exponents(v, m, t);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            v[j] = __builtin_amdgcn_exp2f(t[j]);
            sum += times[j] * v[j];
          }
          sum = gl_sum<G>(sum);
          gl_divide(v, sum, sum != 0.f);
          const float dot = gl_sum<G>((v[0] * g[0] + v[1] * g[1]) + (v[2] * g[2] + v[3] * g[3]));
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            d[j] = v[j] * (g[j] - times[j] * dot);
            g[j] = 0.f;
          }
        }
        if (with_p) {
          gl_softmax<G>(r.s, p);
#pragma unroll
          for (int j = 0; j < 4; ++j) g[j] += b[j];
          const float dot = gl_sum<G>((p[0] * g[0] + p[1] * g[1]) + (p[2] * g[2] + p[3] * g[3]));
#pragma unroll
          for (int j = 0; j < 4; ++j) d[j] += p[j] * (g[j] - dot);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          d[j] = real ? d[j] : 0.f;
          if constexpr (ACC) d[j] += r.old[j];
        }
        if (there && (real || !ACC)) gl_store<G, VEC>(d_scores, t, E, l, d);
      });
}

// Bytes of a mask that are not 0, over the block; the same on every thread.
__device__ __forceinline__ int gl_count_mask(const uint8_t* __restrict__ mask, int64_t begin, int64_t end, int* lds) {
  int n = 0;
  auto word = [](uint32_t v) { return __popc(((v & 0x7F7F7F7Fu) + 0x7F7F7F7Fu | v) & 0x80808080u); };
  int64_t first = begin + (-static_cast<int64_t>(reinterpret_cast<uintptr_t>(mask) + begin) & 15);
  if (first > end) first = end;
  const int64_t chunks = (end - first) / 16;
  for (int64_t t = begin + threadIdx.x; t < first; t += blockDim.x) n += mask[t] != 0;
  for (int64_t t = first + chunks * 16 + threadIdx.x; t < end; t += blockDim.x) n += mask[t] != 0;
  for (int64_t i = threadIdx.x; i < chunks; i += blockDim.x) {
    const uint4 v = *reinterpret_cast<const uint4*>(mask + first + i * 16);
    n += word(v.x) + word(v.y) + word(v.z) + word(v.w);
  }
  return gl_block_sum(n, lds);
}

constexpr int GL_COUNT_BLOCKS = 64;
__global__ __launch_bounds__(GL_THREADS) void mask_count_kernel(const uint8_t* __restrict__ mask, int T, int32_t* __restrict__ part) {
  __shared__ int lds[GL_THREADS / MOE_WAVE];
  const int64_t per = (static_cast<int64_t>(T) + GL_COUNT_BLOCKS - 1) / GL_COUNT_BLOCKS;
  const int64_t begin = min(blockIdx.x * per, static_cast<int64_t>(T));
  const int n = gl_count_mask(mask, begin, min(begin + per, static_cast<int64_t>(T)), lds);
  if (threadIdx.x == 0) part[blockIdx.x] = n;
}

// Tokens that count: T without a mask; from mask_count_kernel's parts; or counted by the block.
__device__ __forceinline__ double gl_tokens(const uint8_t* __restrict__ mask, const int32_t* __restrict__ part_n, int T, int* lds) {
  if (!mask) return T;
  if (!part_n) return gl_count_mask(mask, 0, T, lds);
  int n = part_n[lane_id()];
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) n += __shfl_xor(n, off);
  return n;
}
static_assert(GL_COUNT_BLOCKS == MOE_WAVE, "one part per lane");

struct GlRowPair {
  float s[4], u[4];
};

// ACC: d_scores is added to.
template <int G, bool VEC, bool ACC>
__global__ __launch_bounds__(GL_THREADS) void distill_kernel(const float* __restrict__ scores, const float* __restrict__ target,
                                                             const uint8_t* __restrict__ mask, const int32_t* __restrict__ part_n,
                                                             int T, int E, float coef, int per_block,
                                                             double* __restrict__ part_loss, float* __restrict__ loss,
                                                             float* __restrict__ d_scores) {
  __shared__ double lds[GL_THREADS / MOE_WAVE];
  __shared__ int lds_n[GL_THREADS / MOE_WAVE];
  const int lane = lane_id(), l = lane % G;
  double n = 0.0, sum = 0.0;
  float scale = 0.f;
  struct Row {
    float s[4], u[4], old[4];
  };
  const GlRows rows(T, per_block);
  scores += rows.begin * E;
  target += rows.begin * E;
  if (d_scores) d_scores += rows.begin * E;
  gl_rows<G, Row>(
      rows.n, mask ? mask + rows.begin : nullptr, scores,
      [&](Row& r, int t) {
        gl_load<G, VEC>(scores, t, E, l, -INFINITY, r.s);
        gl_load<G, VEC>(target, t, E, l, -INFINITY, r.u);
        if constexpr (ACC) gl_load<G, VEC>(d_scores, t, E, l, 0.f, r.old);
      },
      [&] {
        n = gl_tokens(mask, part_n, T, lds_n);
        scale = n > 0.0 ? static_cast<float>(coef / n) : 0.f;
      },
      [&](Row& r, int t, bool there, bool real) {
        float p[4], q[4], d[4];
        GlLogs lp, lq;
        const bool left_p = gl_softmax<G>(r.s, p, &lp), left_q = gl_softmax<G>(r.u, q, &lq);
        const bool counts = real && left_p && left_q;
        float row = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          row += q[j] != 0.f ? q[j] * (lq.p[j] - lp.p[j]) : 0.f;     // q = 0 has no part
          d[j] = counts ? scale * (p[j] - q[j]) : 0.f;
          if constexpr (ACC) d[j] += r.old[j];
        }
        sum += counts ? row : 0.f;
        if (d_scores && there && (real || !ACC)) gl_store<G, VEC>(d_scores, t, E, l, d);
      });
  if (__any(!(fabs(sum) < INFINITY))) {
    // rarely: finite scores so far below their row's maximum that the difference, or what it is multiplied by, passes the
    // largest number.  The wave's rows once more, in 64 bits (in the loop above that costs a single small call 0.5 us of 4.3).
    sum = 0.0;
    gl_rows<G, GlRowPair>(
        rows.n, mask ? mask + rows.begin : nullptr, scores,
        [&](GlRowPair& r, int t) {
          gl_load<G, VEC>(scores, t, E, l, -INFINITY, r.s);
          gl_load<G, VEC>(target, t, E, l, -INFINITY, r.u);
        },
        [] {},
        [&](GlRowPair& r, int, bool, bool real) {
          float p[4], q[4];
          GlLogs lp, lq;
          const bool left_p = gl_softmax<G>(r.s, p, &lp), left_q = gl_softmax<G>(r.u, q, &lq);
          double row = 0.0;
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (q[j] != 0.f) row += q[j] * (lq.p[j] - lp.top - (static_cast<double>(r.s[j]) - lp.m) * 1.4426950408889634);
          sum += real && left_p && left_q ? row : 0.0;
        });
  }
  sum = gl_block_sum(sum * GL_LN2, lds);
  if (threadIdx.x != 0) return;
  if (gridDim.x > 1)
    part_loss[blockIdx.x] = sum;
  else
    *loss = n > 0.0 ? static_cast<float>(sum / n) : 0.f;
}

// The mean of the blocks' losses.  (T == 0: no blocks, and 0.)
__global__ __launch_bounds__(GL_SUM_THREADS) void distill_finish_kernel(const double* __restrict__ part_loss, int blocks,
                                                                   const uint8_t* __restrict__ mask, const int32_t* __restrict__ part_n,
                                                                   int T, float* __restrict__ loss) {
  __shared__ double lds[GL_SUM_THREADS / MOE_WAVE];
  __shared__ int lds_n[GL_SUM_THREADS / MOE_WAVE];
  const double n = gl_tokens(mask, part_n, T, lds_n);
  const double sum = gl_block_sum(static_cast<int>(threadIdx.x) < blocks ? part_loss[threadIdx.x] : 0.0, lds);
  if (threadIdx.x == 0) *loss = n > 0.0 ? static_cast<float>(sum / n) : 0.f;
}

// Calls f with the lanes per token and whether rows are whole 16-byte chunks.
template <class F> static void gl_by_experts(int E, F f) {
  auto with = [&](auto g) {
    if (E % 4 == 0)
      f(g, std::true_type{});
    else
      f(g, std::false_type{});
  };
  if (E <= 4) with(std::integral_constant<int, 1>{});
  else if (E <= 8) with(std::integral_constant<int, 2>{});
  else if (E <= 16) with(std::integral_constant<int, 4>{});
  else if (E <= 32) with(std::integral_constant<int, 8>{});
  else if (E <= 64) with(std::integral_constant<int, 16>{});
  else if (E <= 128) with(std::integral_constant<int, 32>{});
  else with(std::integral_constant<int, 64>{});
}

// Lanes that share a token.
static int gl_lanes(int E) {
  int g = 1;
  while (4 * g < E) g <<= 1;
  return g;
}

// Blocks of a call and the rows of each: a turn of the block's waves, or as many as the limit on
// blocks asks for; a batch of up to `alone` turns is one block, which needs no launch to add up sums.  (Measured, one
// block / two launches, us: balance 64 experts, 200 tokens 7.4 / 9.3, 500 9.5 / 9.4; 8 experts, 1500 tokens 7.5 / 11.2;
// distill 8 experts, 500 tokens 4.0 / 5.2, 64 experts, 60 tokens 4.1 / 5.3, 120 5.7 / 5.4.)
struct GlPlan {
  int blocks, per_block;
};
static GlPlan gl_plan(int T, int E, int threads, int alone, int most_blocks) {
  const int64_t pass = threads / gl_lanes(E);
  int64_t per = (static_cast<int64_t>(T) + most_blocks - 1) / most_blocks;
  per = (per + pass - 1) / pass * pass;
  if (T <= alone * pass) per = T;
  return {T > 0 ? static_cast<int>((T + per - 1) / per) : 0, static_cast<int>(per)};
}
// Sums for every expert: one block adds up the blocks' rows, so there are 256 blocks at most (65536 tokens, 64 experts
// 18.4 us; with 512 blocks 21.0).
static GlPlan gl_balance_plan(const moe_shape_t* s) { return gl_plan(s->T, s->E, GL_SUM_THREADS, 4, 256); }
// One sum: as many blocks as the finishing block has threads (65536 tokens, 128 experts 22.8 us; with half as many 25.9).
static GlPlan gl_distill_plan(const moe_shape_t* s) { return gl_plan(s->T, s->E, GL_THREADS, 4, GL_SUM_THREADS); }
// (512 / 1024 / 2048 blocks: 65536 tokens, 128 experts 17.9 / 15.8 / 16.0 us, 64 experts 12.8 / 12.0 / 12.5.)
static GlPlan gl_route_plan(const moe_shape_t* s) { return gl_plan(s->T, s->E, GL_THREADS, 1, 1024); }

// From this many tokens on the mask is counted by a launch of its own, not by every block.  (Measured, every block / a
// launch, us: E = 64, 4000 tokens 7.7 / 9.7, 16384 9.4 / 10.3, 30000 14.5 / 14.7; E = 128, 65536 tokens 31.1 / 27.2.)
constexpr int GL_COUNT_FROM = 1 << 15;

size_t gate_loss_workspace_bytes(const moe_shape_t* shape) {
  const size_t balance = static_cast<size_t>(gl_balance_plan(shape).blocks) * gl_part_pitch(shape->E) * 8;
  const size_t distill = static_cast<size_t>(gl_distill_plan(shape).blocks) * 8 + GL_COUNT_BLOCKS * 4;
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
  if (workspace_bytes < train_workspace_bytes(shape)) return MOE_ERR_WORKSPACE;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const int T = shape->T, E = shape->E, k = shape->k;
  const GlPlan plan = gl_balance_plan(shape);
  float* part_p = static_cast<float*>(workspace);
  int32_t* part_c = reinterpret_cast<int32_t*>(part_p + static_cast<size_t>(plan.blocks) * gl_part_pitch(E));
  if (T > 0)
    gl_by_experts(E, [&](auto g, auto vec) {
      hipLaunchKernelGGL((balance_kernel<decltype(g)::value, decltype(vec)::value>), dim3(plan.blocks), dim3(GL_SUM_THREADS), 0, st, scores, topk_idx, token_mask, T, E, k,
                         plan.per_block, part_p, part_c, counts, prob_sum, loss);
    });
  if (plan.blocks != 1)
    hipLaunchKernelGGL(balance_finish_kernel, dim3(1), dim3(GL_SUM_THREADS), 0, st, part_p, part_c, plan.blocks, E, k, gl_lanes(E), counts,
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
  const int64_t table = int64_t(4) * shape->T * shape->E, choices = int64_t(4) * shape->T * shape->k;
  if (!apart(d_scores, table, scores, table) || !apart(d_scores, table, d_topk_w, choices) || !apart(d_scores, table, topk_idx, choices))
    return MOE_ERR_INVALID_ARG;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const int T = shape->T, E = shape->E, k = shape->k;
  const GlPlan plan = gl_route_plan(shape);
  gl_by_experts(E, [&](auto g, auto vec) {
    constexpr int G = decltype(g)::value;
    constexpr bool VEC = decltype(vec)::value;
    const auto with = [&](auto q) {
      return accumulate ? route_backward_kernel<G, VEC, decltype(q)::value, true> : route_backward_kernel<G, VEC, decltype(q)::value, false>;
    };
    const auto kernel = !d_topk_w ? with(std::integral_constant<int, 0>{})
                        : k <= G  ? with(std::integral_constant<int, 1>{})
                                  : with(std::integral_constant<int, 4>{});
    hipLaunchKernelGGL(kernel, dim3(plan.blocks), dim3(GL_THREADS), 0, st, scores, topk_idx, d_topk_w, counts, balance_coef, token_mask, T, E,
                       k, shape->renorm, plan.per_block, d_scores);
  });
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
  if (workspace_bytes < train_workspace_bytes(shape)) return MOE_ERR_WORKSPACE;
  const int64_t table = int64_t(4) * shape->T * shape->E;
  if (!apart(d_scores, table, scores, table) || !apart(d_scores, table, target_scores, table)) return MOE_ERR_INVALID_ARG;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const int T = shape->T, E = shape->E;
  const GlPlan plan = gl_distill_plan(shape);
  double* part_loss = static_cast<double*>(workspace);
  int32_t* part_n = nullptr;
  if (token_mask && T >= GL_COUNT_FROM) {
    part_n = reinterpret_cast<int32_t*>(part_loss + plan.blocks);
    hipLaunchKernelGGL(mask_count_kernel, dim3(GL_COUNT_BLOCKS), dim3(GL_THREADS), 0, st, token_mask, T, part_n);
  }
  if (T > 0)
    gl_by_experts(E, [&](auto g, auto vec) {
      constexpr int G = decltype(g)::value;
      constexpr bool VEC = decltype(vec)::value;
      const auto kernel = accumulate && d_scores ? distill_kernel<G, VEC, true> : distill_kernel<G, VEC, false>;
      hipLaunchKernelGGL(kernel, dim3(plan.blocks), dim3(GL_THREADS), 0, st, scores, target_scores, token_mask, part_n, T, E, coef,
                         plan.per_block, part_loss, loss, d_scores);
    });
  if (plan.blocks != 1)
    hipLaunchKernelGGL(distill_finish_kernel, dim3(1), dim3(GL_SUM_THREADS), 0, st, part_loss, plan.blocks, token_mask, part_n, T, loss);
  return launch_status();
}
