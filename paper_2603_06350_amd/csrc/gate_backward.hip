// moe_gate_backward: the gradients of the gate product score[t,e] = sum_i x[t,i] w_gate[e,i] + gate_bias[e]:
//   d_w_gate[e,:] = sum_t d_scores[t,e] x[t,:]      d_gate_bias[e] = sum_t d_scores[t,e]
//   d_x[t,:]      = sum_e d_scores[t,e] w_gate[e,:]
// x is read once and d_x written once; everything else is small beside them.  Up to 32 experts both products are bound by
// HBM; beyond, the weights' gradient has as much to do in the matrix instructions and the splitting into pieces as in its
// loads, and neither hides the other entirely.
//
// Measured (bf16 layers; a copy on this card reads and writes 4.6 to 5.4 TB/s): both gradients of 65536 tokens, d = 4096, E = 8
// 217 us = 5.0 TB/s; 65536 tokens, d = 2048, E = 64 113 to 117 us = 4.8 TB/s, of it the weights' 55
// and 7 for the sums of the parts and the hidden states' 48 to 50 = 5.5 TB/s written; weights alone of 16384 tokens, d = 4096,
// E = 128 50 us and 6.5.
//
// Both run on v_mfma_f32_16x16x32_bf16 with fp32 accumulators, operands straight from global memory into registers:
//   - a lane that holds V consecutive columns of 8 consecutive rows of a matrix (one load per row) turns them, with
//     byte permutes inside the lane, into the 8 values along the reduction that the instruction wants of it, for
//     V column tiles: tile i holds the columns V c + i of the lanes c = 0..15.  x (reduction over tokens) and w_gate
//     (reduction over experts) need no LDS and no transposed copy, and the V results of a lane are V consecutive
//     columns again: 16-byte stores;
//   - d_scores (fp32) enters in three bf16 pieces that hold all its 24 bits.  (Two would do for a d_x that is rounded to
//     8 bits only where the terms of a sum do not cancel: rows of d_scores add up to nothing, so what gate rows have
//     in common does.  Measured for d_x, two / three, us: 65536 tokens, d = 2048, E = 64 52 / 51; 16384, d = 4096, E = 128
//     39 / 48; 8000, d = 5120, E = 250 54 / 63.)  fp32 layers cut x and w_gate into three pieces as well and multiply
//     eight of the nine products (gb_products), so that a sum of one product is as good as rounded: within 1.02 x 2^-24 of
//     it.  (Six products and one sum for all, which leave up to 5 x 2^-24, us: 8192 tokens, d = 2048, E = 8 27.4, with eight
//     29; 40000, d = 1024, E = 64 80 and 87; 8000, d = 4096, E = 128 104 and 123; 8000, d = 1024, E = 256 58 and 67.)
#include "moe_internal.h"

namespace moe {

// Of x and d_x: the most rows that a descriptor covers (128 of d_x) stay within 2^31 bytes, and GB_NOWHERE and as many
// rows within 2^32.
constexpr int64_t GB_ROW_BYTES = int64_t(1) << 24;

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

// The pieces of eight values.
__device__ __forceinline__ void gb_split8(const float (&v)[8], uint4 (&p)[3]) {
  uint32_t q[3][4];
#pragma unroll
  for (int u = 0; u < 4; ++u) gb_split(v[2 * u], v[2 * u + 1], q[0][u], q[1][u], q[2][u]);
#pragma unroll
  for (int i = 0; i < 3; ++i) p[i] = make_uint4(q[i][0], q[i][1], q[i][2], q[i][3]);
}

// The sum of a lane's eight gradients of an expert, for d_gate_bias, which is summed in 64 bits beyond these (sums in 32 were
// off by up to 3e-7, relative, where these are by 7e-8).
__device__ __forceinline__ float gb_sum8(const float (&v)[8]) {
  return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
}

// The operand fragments of V column tiles from a lane's V columns of 8 rows along the reduction; P pieces each.
template <bool BF16, int V> struct GbFrag {
  static constexpr int P = BF16 ? 1 : 3;
  uint4 f[P][V];
};

// A step's rows are read and written through a buffer descriptor of exactly these rows: the place of a lane in them is 32
// bits, and a lane that is past the last row, or has nothing to do, reads zeros and writes nothing.  No load or store is
// behind a branch, so that the waits for one step's operands can leave the next one's on their way.
constexpr uint32_t GB_NOWHERE = 0x80000000u;          // a place outside every descriptor (with a few rows added as well)
__device__ __forceinline__ __amdgpu_buffer_rsrc_t gb_rows(const void* first, int rows, uint32_t pitch) {
  // (the clamp may become an instruction of the vector unit; a descriptor has to be in scalar registers)
  const uint32_t n = __builtin_amdgcn_readfirstlane(max(rows, 0));
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(first), 0, static_cast<int>(n * pitch), 0x00020000);
}
// The same number, but nothing that is computed from it is kept from one step to the next: sixteen offsets of rows would
// take as many registers, where an addition for each is cheap.
__device__ __forceinline__ uint32_t gb_anew(uint32_t v) {
  asm volatile("" : "+s"(v));
  return v;
}
__device__ __forceinline__ float gb_load_f32(__amdgpu_buffer_rsrc_t rows, uint32_t at) {
  return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rows, static_cast<int>(at), 0, 0));
}
typedef uint32_t gb_u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t gb_u32x2 __attribute__((ext_vector_type(2)));

// What is not used again by the launch (d_x as it is stored, x of large batches) is marked as a stream, so that it leaves the
// caches first: d_x displaces less of the x that follows, and x nothing.  (Measured for both gradients, neither / stores /
// stores and the loads of blocks of 64 experts, us: 65536 tokens, d = 2048, E = 64 152 / 129 / 117; 16384, d = 4096, E = 128
// 115 / 109 / 108; 30000, d = 4096, E = 16 109 / 104; 8192, d = 2048, E = 64 30.9 / 31.8.  In the blocks of 16 and 32 experts
// marked loads are slower: 4096 tokens, d = 4096, E = 8 18.3 / 20.4 with them.)
constexpr int GB_STREAM = 2;

// V consecutive elements of a row: 8 or 16 bytes.
template <bool BF16, int V> struct GbRow {
  static constexpr int W = V * (BF16 ? 2 : 4) / 4;
  uint32_t w[W];
  template <int CACHE = 0> __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t rows, uint32_t at) {
    if constexpr (W == 4) {
      const auto v = __builtin_amdgcn_raw_buffer_load_b128(rows, static_cast<int>(at), 0, CACHE);
      w[0] = v[0], w[1] = v[1], w[2] = v[2], w[3] = v[3];
    } else {
      const auto v = __builtin_amdgcn_raw_buffer_load_b64(rows, static_cast<int>(at), 0, CACHE);
      w[0] = v[0], w[1] = v[1];
    }
  }
  __device__ __forceinline__ void store(__amdgpu_buffer_rsrc_t rows, uint32_t at) const {
    if constexpr (W == 4)
      __builtin_amdgcn_raw_buffer_store_b128(gb_u32x4{w[0], w[1], w[2], w[3]}, rows, static_cast<int>(at), 0, GB_STREAM);
    else
      __builtin_amdgcn_raw_buffer_store_b64(gb_u32x2{w[0], w[1]}, rows, static_cast<int>(at), 0, GB_STREAM);
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

// acc[i] += the products of the pieces of an fp32 operand with those of column tile i, the small ones first.  Products with
// the same sum are V instructions apart: one that follows directly waits for the sum.  fp32 layers: without the product of
// the last pieces, 2^-31 of the whole or less; the matrix instruction does not round its sum to nearest, so all but
// the leading products, 2^-6 of them and less, have sums of their own, `low`, that the caller adds (gb_add).
template <bool BF16, int V> using GbLow = gb_f32x4[BF16 ? 1 : V];
template <bool BF16, int V>
__device__ __forceinline__ void gb_products(uint4 h, uint4 m, uint4 l, const GbFrag<BF16, V>& b, gb_f32x4 (&acc)[V], GbLow<BF16, V>& low) {
  auto step = [&](uint4 a, const uint4 (&f)[V], gb_f32x4 (&to)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) to[i] = gb_mfma(a, f[i], to[i]);
  };
  if constexpr (BF16) {
    step(l, b.f[0], acc);
    step(m, b.f[0], acc);
    step(h, b.f[0], acc);
  } else {
    step(l, b.f[1], low);
    step(m, b.f[2], low);
    step(l, b.f[0], low);
    step(h, b.f[2], low);
    step(h, b.f[0], acc);
    step(m, b.f[1], low);
    step(m, b.f[0], low);
    step(h, b.f[1], low);
  }
}
template <bool BF16, int V> __device__ __forceinline__ void gb_add(gb_f32x4 (&acc)[V], const GbLow<BF16, V>& low) {
  if constexpr (!BF16) {
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] += low[i];
  }
}

// ------------------------------------------------------------------------------------------------ weights' gradient
// A block owns 16 V columns of x for a range of tokens and up to 16 MT experts; its waves take 32 tokens each in turn,
// keep their own sums in registers and add them up in LDS at the end, so that a block leaves few columns' sums to be
// written and read again.  With 16 experts it reads x at 5.65 TB/s (65536 tokens, d = 4096, without d_x).
constexpr int GW_WAVES = 8;
constexpr int GW_THREADS = GW_WAVES * MOE_WAVE;

struct GwArgs {
  const char* x;
  const float* d_scores;
  const uint8_t* mask;
  float* out_w;
  float* out_b;
  int T, d, E, tiles, chunks, splits, per_split, accumulate;
};

// The block's place: column tile, group of experts, part of the tokens.  All tiles and groups of a part are on one XCD
// (blocks are dealt to the 8 XCDs in turn): its L2 then gets d_scores once, and whole rows of x once.
struct GwPlace {
  int tile, chunk, split;
};
__device__ __forceinline__ GwPlace gw_place(int tiles, int chunks, int splits, int b) {
  const int n = tiles * chunks;
  const int rest = splits % 8 == 0 ? b / 8 % n : b % n;
  return {rest / chunks, rest % chunks, splits % 8 == 0 ? b / 8 / n * 8 + b % 8 : b / n};
}

// 16 or 32 experts to a block: a lane loads the values of d_scores that it needs (8 tokens of an expert) one by one, and
// every wave cuts the pieces of its own.
constexpr int GW_LDS = GW_WAVES * 4 * MOE_WAVE * 16;
template <bool BF16, int MT, int V>
__device__ __forceinline__ void gate_weight_block(const GwArgs& a, int block, unsigned char* lds, double (*red_b)[16 * MT]) {
  constexpr int B = BF16 ? 2 : 4;
  auto red = reinterpret_cast<gb_f32x4(*)[4][MOE_WAVE]>(lds);
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / MOE_WAVE), c = lane & 15, g = lane >> 4;
  const int d = a.d, E = a.E, splits = a.splits;
  const GwPlace place = gw_place(a.tiles, a.chunks, splits, block);
  const int tile = place.tile, split = place.split, e0 = place.chunk * 16 * MT;
  // (token numbers in 32 unsigned bits: T < 2^31, and no number passes it by more than the blocks' steps)
  const uint32_t begin = static_cast<uint32_t>(split) * a.per_split;
  const uint32_t end = min(begin + a.per_split, static_cast<uint32_t>(a.T));
  const uint32_t pitch = static_cast<uint32_t>(d) * B, pitch_s = static_cast<uint32_t>(E) * 4;
  // Columns past the last and experts that do not exist repeat the last ones'; their sums are not stored.
  const uint32_t at_x = 8 * g * pitch + static_cast<uint32_t>(min(tile * 16 * V + V * c, d - V)) * B;
  const bool with_w = a.out_w, with_bias = a.out_b && tile == 0;

  gb_f32x4 acc[MT][V];
  double bias[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    bias[m] = 0.0;
#pragma unroll
    for (int i = 0; i < V; ++i) acc[m][i] = gb_f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // What a wave multiplies in one step: 32 tokens, lane 16 g + c the tokens 8 g + 0..7 of its columns and experts.
  GbRow<BF16, V> x[8];
  float ds[MT][8];
  uint32_t mask;                                     // of token t0 + (lane & 31)
  auto load = [&](uint32_t t0) {
    const int left = min(static_cast<int>(end - t0), 32);
    // a descriptor for every row that the lanes have in common: what differs between lanes stays the same
    const char* x0 = a.x + static_cast<int64_t>(t0) * pitch;
    const char* s0 = reinterpret_cast<const char*>(a.d_scores) + static_cast<int64_t>(t0) * pitch_s;
    mask = __builtin_amdgcn_raw_buffer_load_b8(gb_rows(a.mask + t0, a.mask ? left : 0, 1), lane & 31, 0, 0);
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int j = 0; j < 8; ++j)
        ds[m][j] = gb_load_f32(gb_rows(s0 + j * pitch_s, left - j, pitch_s),
                               8 * g * pitch_s + static_cast<uint32_t>(min(e0 + 16 * m + c, E - 1)) * 4);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j].load(gb_rows(x0 + static_cast<int64_t>(j) * pitch, with_w ? left - j : 0, pitch), at_x);
  };
  // A step's operands go over to the registers that the products read, and the next step's are requested into the ones
  // that are free then; behind the last step nothing is read.
  uint32_t t0 = begin + 32 * wave;
  load(t0);
  while (t0 < end) {
    const int left = static_cast<int>(end - t0);
    if (a.mask || left < 32) {
      // bit j: token t0 + 8 g + j counts
      const uint32_t real = static_cast<uint32_t>(__ballot((lane & 31) < left && (!a.mask || mask))) >> (8 * g);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[j].keep(real >> j & 1);
#pragma unroll
        for (int m = 0; m < MT; ++m) ds[m][j] = real >> j & 1 ? ds[m][j] : 0.f;
      }
    }
    GbFrag<BF16, V> b;
    gb_transpose<BF16, V>(x, b);
    uint4 p[MT][3];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      if (with_bias) bias[m] += gb_sum8(ds[m]);
      gb_split8(ds[m], p[m]);
    }
    __builtin_amdgcn_sched_barrier(0);
    t0 += 32 * GW_WAVES;
    load(t0);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      GbLow<BF16, V> low = {};
      gb_products<BF16, V>(p[m][0], p[m][1], p[m][2], b, acc[m], low);
      gb_add<BF16, V>(acc[m], low);
    }
  }

  // sums of the waves, 16 experts at a time: lane 16 g + c of a wave holds experts 4 g + 0..3 of the columns V c + i
  const int64_t n = static_cast<int64_t>(E) * d;
  float* to = a.out_w + (splits > 1 ? split * n : 0);
  const bool add = a.accumulate && splits == 1;
  if (with_w) {
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
      double v = bias[m];
      v += __shfl_xor(v, 16);
      v += __shfl_xor(v, 32);
      if (g == 0) red_b[wave][16 * m + c] = v;
    }
    __syncthreads();
    const int e = e0 + threadIdx.x;
    if (threadIdx.x < 16 * MT && e < E) {
      double v = add ? a.out_b[e] : 0.f;
      for (int w = 0; w < GW_WAVES; ++w) v += red_b[w][threadIdx.x];
      a.out_b[(splits > 1 ? static_cast<int64_t>(split) * E : 0) + e] = static_cast<float>(v);
    }
  }
}

// 64 experts and 64 V columns to a block (gw_plan says when): its waves lie side by side over the columns, four for the
// first 32 tokens of a step and four for the next, and share the pieces of d_scores, which the block makes once and keeps
// in LDS in the order in which the lanes want them: thread 64 w + i of a step cuts 8 tokens (8 (w % 4) of half w / 4) of
// expert i.
//
// A step's loads are on their way while the one before is multiplied.  Measured, us: 16384 tokens, d = 4096, E = 128 50 (its
// matrix instructions alone 26, without products 43), 65536 tokens 171; d = 2048, E = 64, 65536 tokens 58.  Where the waves
// met between two steps, all of them splitting and transposing at the same time, it took 10 % longer with 128 experts.
// Loads one, two and four steps further ahead (spills, or one wave per SIMD), loads between the products, the 32x32x16
// instruction (1.9 PFLOP/s in a loop of its own, the 16x16x32 2.0 to 2.2), and two blocks of four waves were not faster.
constexpr int GWW_PIECES = 4 * MOE_WAVE * 16;         // bytes of a piece of 32 tokens, 64 experts
constexpr int GWW_STEP = 2 * 3 * GWW_PIECES;
constexpr int GWW_LDS = 3 * GWW_STEP;                 // (the waves' sums need 64 KiB of it)
static_assert(GWW_LDS >= GW_WAVES * 8 * MOE_WAVE * 16, "sums of the waves");

template <bool BF16, int V>
__device__ __forceinline__ void gate_weight_wide_block(const GwArgs& a, unsigned char* lds, double* red_b) {
  constexpr int B = BF16 ? 2 : 4, MT = 4;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / MOE_WAVE), c = lane & 15, g = lane >> 4;
  const int half = wave >> 2;
  const int d = a.d, E = a.E, splits = a.splits;
  const GwPlace place = gw_place(a.tiles, a.chunks, splits, blockIdx.x);
  const int e0 = place.chunk * 64;
  const uint32_t begin = static_cast<uint32_t>(place.split) * a.per_split;
  const uint32_t end = min(begin + a.per_split, static_cast<uint32_t>(a.T));
  const uint32_t pitch = static_cast<uint32_t>(d) * B, pitch_s = static_cast<uint32_t>(E) * 4;
  const int col = (place.tile * 4 + (wave & 3)) * 16 * V + V * c;
  const uint32_t at_x = 8 * g * pitch + static_cast<uint32_t>(min(col, d - V)) * B;
  const bool with_w = a.out_w, with_bias = a.out_b && place.tile == 0;

  // this thread's part of d_scores: 8 tokens of an expert
  const uint32_t at_s = 8 * (wave & 3) * pitch_s + static_cast<uint32_t>(min(e0 + lane, E - 1)) * 4;
  const int at_piece = half * 3 * GWW_PIECES + (lane / 16 * MOE_WAVE + 16 * (wave & 3) + lane % 16) * 16;
  float ds[8];
  double bias = 0.0;
  GbRow<BF16, V> x[8];
  uint32_t mask;
  auto left_of = [&](uint32_t t0) { return min(static_cast<int>(end - t0) - 32 * half, 32); };
  auto load_x = [&](uint32_t t0) {
    const auto rows = gb_rows(a.x + (static_cast<int64_t>(t0) + 32 * half) * pitch, with_w ? left_of(t0) : 0, pitch);
    const uint32_t p = gb_anew(pitch);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j].template load<GB_STREAM>(rows, at_x + j * p);
  };
  auto load_s = [&](uint32_t t0) {
    const int64_t t = static_cast<int64_t>(t0) + 32 * half;
    const auto rows = gb_rows(reinterpret_cast<const char*>(a.d_scores) + t * pitch_s, left_of(t0), pitch_s);
    const uint32_t p = gb_anew(pitch_s);
#pragma unroll
    for (int j = 0; j < 8; ++j) ds[j] = gb_load_f32(rows, at_s + j * p);
    mask = __builtin_amdgcn_raw_buffer_load_b8(gb_rows(a.mask + t, a.mask ? left_of(t0) : 0, 1), lane & 31, 0, 0);
  };
  // Pieces of a step's gradients, of which bit i of the result says whether token t0 + 32 half + i counts.
  auto put = [&](uint32_t t0, unsigned char* to) {
    uint32_t real = 0xFFFFFFFFu;
    if (a.mask || static_cast<int>(end - t0) < 64) {
      real = static_cast<uint32_t>(__ballot((lane & 31) < left_of(t0) && (!a.mask || mask)));
      const uint32_t mine = real >> (8 * (wave & 3));
#pragma unroll
      for (int j = 0; j < 8; ++j) ds[j] = mine >> j & 1 ? ds[j] : 0.f;
    }
    if (with_bias) bias += gb_sum8(ds);
    uint4 p[3];
    gb_split8(ds, p);
#pragma unroll
    for (int q = 0; q < 3; ++q) *reinterpret_cast<uint4*>(to + at_piece + q * GWW_PIECES) = p[q];
    return real;
  };

  gb_f32x4 acc[MT][V];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int i = 0; i < V; ++i) acc[m][i] = gb_f32x4{0.f, 0.f, 0.f, 0.f};
  // x of a step goes over to the registers that the products read, and the next step's is requested into the ones that are
  // free then.  The next step's gradients, which are a step ahead of x, are cut into pieces halfway through the products:
  // the waves meet there, and need not start the next step together.  A third place for pieces in LDS is for the waves
  // that are behind by half a step.  Behind the last step nothing is read.
  load_s(begin);
  load_x(begin);
  uint32_t real = put(begin, lds);
  load_s(begin + 64);
  __syncthreads();
  uint32_t at_lds = 0;
  for (uint32_t t0 = begin; t0 < end; t0 += 64) {
    if (real != 0xFFFFFFFFu) {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j].keep(real >> (8 * g) >> j & 1);
    }
    GbFrag<BF16, V> b;
    gb_transpose<BF16, V>(x, b);
    __builtin_amdgcn_sched_barrier(0);
    load_x(t0 + 64);
    __builtin_amdgcn_sched_barrier(0);
    const uint32_t next = at_lds == 2 * GWW_STEP ? 0 : at_lds + GWW_STEP;
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      if (m == MT / 2) {
        real = put(t0 + 64, lds + next);
        load_s(t0 + 128);
        __syncthreads();
      }
      uint4 p[3];
#pragma unroll
      for (int q = 0; q < 3; ++q)
        p[q] = *reinterpret_cast<const uint4*>(lds + at_lds + (half * 3 + q) * GWW_PIECES + (m * MOE_WAVE + lane) * 16);
      GbLow<BF16, V> low = {};
      gb_products<BF16, V>(p[0], p[1], p[2], b, acc[m], low);
      gb_add<BF16, V>(acc[m], low);
    }
    at_lds = next;
  }
  __syncthreads();

  // The halves' sums meet in LDS: the first half's waves finish the experts 0..31, the second's 32..63.
  const int64_t n = static_cast<int64_t>(E) * d;
  float* to = a.out_w + (splits > 1 ? place.split * n : 0);
  const bool add = a.accumulate && splits == 1;
  auto red = reinterpret_cast<gb_f32x4(*)[V][MOE_WAVE]>(lds);
  auto finish = [&](const gb_f32x4 (&mine)[V], int m) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int e = e0 + 16 * m + 4 * g + r;
      if (e >= E || col >= d) continue;
#pragma unroll
      for (int i = 0; i < V; i += 4) {
        float4* o = reinterpret_cast<float4*>(to + static_cast<int64_t>(e) * d + col + i);
        float4 s = add ? *o : make_float4(0.f, 0.f, 0.f, 0.f);
        s.x += mine[i][r], s.y += mine[i + 1][r], s.z += mine[i + 2][r], s.w += mine[i + 3][r];
        *o = s;
      }
    }
  };
  if (with_w) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      if (q > 0) __syncthreads();
      if (half == 0) {
#pragma unroll
        for (int i = 0; i < V; ++i) red[wave][i][lane] = acc[2 + q][i];
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) red[wave][i][lane] = acc[q][i];
      }
      __syncthreads();
      if (half == 0) {
#pragma unroll
        for (int i = 0; i < V; ++i) acc[q][i] += red[wave + 4][i][lane];
        finish(acc[q], q);
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) acc[2 + q][i] += red[wave - 4][i][lane];
        finish(acc[2 + q], 2 + q);
      }
    }
  }
  if (with_bias) {
    red_b[threadIdx.x] = bias;
    __syncthreads();
    const int e = e0 + threadIdx.x;
    if (threadIdx.x < 64 && e < E) {
      double v = add ? a.out_b[e] : 0.f;
      for (int w = 0; w < GW_WAVES; ++w) v += red_b[64 * w + threadIdx.x];
      a.out_b[(splits > 1 ? static_cast<int64_t>(place.split) * E : 0) + e] = static_cast<float>(v);
    }
  }
}

template <bool BF16, int V>
__global__ __launch_bounds__(GW_THREADS) void gate_weight_wide_kernel(GwArgs a) {
  extern __shared__ __align__(16) unsigned char lds[];
  __shared__ double red_b[GW_THREADS];
  gate_weight_wide_block<BF16, V>(a, lds, red_b);
}

// out[i] (+)= the sum of the parts' elements i: four consecutive ones per thread, every GROUPS-th part, eight of them on
// their way at a time; the groups' sums of an element meet in LDS.  The order of the additions is fixed.  Many parts are of
// few elements and want many groups, few parts large blocks of elements.  (Measured, 2 / 4 / 8 groups, us: 256 parts of 8 x
// 64 10.3 / 6.1 / 3.9; 64 of 64 x 2048 6.4 / 6.4 / 7.8; 16 of 128 x 4096 6.2 / 9.6 / 6.5.)
constexpr int GS_THREADS = 256;
__device__ __forceinline__ float4 gs_add(float4 a, float4 b) { return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w); }
__device__ __forceinline__ double gs_add(double a, double b) { return a + b; }
template <int GROUPS, class S, class V>
__device__ __forceinline__ void gs_column(const V* part, V* out, int64_t n, int64_t i, int splits, int accumulate, S* lds) {
  constexpr int COLUMNS = GS_THREADS / GROUPS;
  const int column = threadIdx.x % COLUMNS, group = threadIdx.x / COLUMNS;
  S s{};
  if (i < n) {
    for (int p = group; p < splits; p += 8 * GROUPS) {
      V v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        v[u] = V{};
        if (p + u * GROUPS < splits) v[u] = part[(p + u * GROUPS) * n + i];
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) s = gs_add(s, v[u]);
    }
  }
  if (group > 0) lds[(group - 1) * COLUMNS + column] = s;
  __syncthreads();
  if (group == 0 && i < n) {
#pragma unroll
    for (int u = 0; u < GROUPS - 1; ++u) s = gs_add(s, lds[u * COLUMNS + column]);
    if (accumulate) s = gs_add(s, out[i]);
    out[i] = static_cast<V>(s);
  }
}
// Blocks: the first blocks_w for d_w_gate (n elements), the others for d_gate_bias.
template <int GROUPS>
__global__ __launch_bounds__(GS_THREADS) void gate_sum_kernel(const float* __restrict__ part_w, float* __restrict__ out_w, int64_t n,
                                                              int blocks_w, const float* __restrict__ part_b,
                                                              float* __restrict__ out_b, int E, int splits, int accumulate) {
  constexpr int COLUMNS = GS_THREADS / GROUPS;
  __shared__ float4 lds[(GROUPS - 1) * COLUMNS];
  const int column = threadIdx.x % COLUMNS, block = blockIdx.x;
  if (block < blocks_w)
    gs_column<GROUPS, float4>(reinterpret_cast<const float4*>(part_w), reinterpret_cast<float4*>(out_w), n / 4,
                      static_cast<int64_t>(block) * COLUMNS + column, splits, accumulate, lds);
  else
    gs_column<GROUPS, double>(part_b, out_b, static_cast<int64_t>(E), static_cast<int64_t>(block - blocks_w) * COLUMNS + column, splits, accumulate,
                      reinterpret_cast<double*>(lds));
}

// ------------------------------------------------------------------------------------------------ hidden states' gradient
// A wave keeps the fragments of w_gate of its 16 V columns (KS steps of 32 experts) in registers; the four waves of a
// block lie side by side and run over tokens, GT at a time.  The block reads d_scores of its next GT tokens in whole
// rows, cuts them into pieces once and keeps these in LDS, from where the waves take their operands.  (Every wave
// reading its operands straight from global memory, 64 lanes in 64 places, which the L1 serves one after the other:
// 65536 tokens, d = 2048, E = 64 80 us instead of 52.)
constexpr int GX_SIDE = 4;                            // waves side by side

struct GxArgs {
  const char* w_gate;
  const float* d_scores;
  const uint8_t* mask;
  char* d_x;
  int T, d, E, tiles, splits, per_split;
};

// THREADS: 256, or 512 for two groups of waves side by side, each with GT tokens of a step of its own.
template <bool BF16, int KS, int THREADS> struct GxTile {
  static constexpr int P = 3;                        // pieces of d_scores
  static constexpr int GT = KS <= 2 ? 64 : 128 / KS; // tokens of a wave's step
  static constexpr int STEP = GT * THREADS / 256;    // tokens of the block's step
  static constexpr int CPT = 8 * KS;                 // chunks of four experts of a token
  static constexpr int LOADS = STEP * CPT / THREADS;
  static constexpr int PITCH = 64 * KS + 16;         // bytes of a row in LDS: 16 more than the experts take, against bank conflicts
  static constexpr int PIECE = STEP * PITCH;
  static constexpr int LDS = 2 * P * PIECE;
};

// WHOLE: E is a multiple of 4, so that rows of d_scores are whole 16-byte chunks.  ACC: d_x is added to.
template <bool BF16, int KS, int V, int THREADS, bool WHOLE, bool ACC>
__device__ __forceinline__ void gate_x_block(const GxArgs& a, int block, unsigned char* lds, uint32_t* reals) {
  using Tile = GxTile<BF16, KS, THREADS>;
  constexpr int B = BF16 ? 2 : 4, P = Tile::P, GT = Tile::GT, STEP = Tile::STEP, CPT = Tile::CPT, LOADS = Tile::LOADS, PITCH = Tile::PITCH,
                PIECE = Tile::PIECE;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / MOE_WAVE), c = lane & 15, g = lane >> 4;
  const int d = a.d, E = a.E, first = wave / GX_SIDE * GT;             // of this wave's tokens in a step
  const GwPlace place = gw_place(a.tiles, 1, a.splits, block);
  const int col = (place.tile * GX_SIDE + wave % GX_SIDE) * 16 * V + V * c;
  const uint32_t begin = static_cast<uint32_t>(place.split) * a.per_split;
  const uint32_t end = min(begin + a.per_split, static_cast<uint32_t>(a.T));
  if (begin >= end) return;                          // the whole block
  const uint32_t pitch = static_cast<uint32_t>(d) * B, pitch_s = static_cast<uint32_t>(E) * 4;

  // Chunk threadIdx.x + THREADS i of a step: four experts of one token.
  float v[LOADS][4];
  uint32_t mask[LOADS];
  auto load = [&](uint32_t t0) {
    const int rows = min(static_cast<int>(end - t0), STEP);
    const auto sr = gb_rows(a.d_scores + static_cast<int64_t>(t0) * E, rows, pitch_s);
    const auto mr = gb_rows(a.mask + t0, a.mask ? rows : 0, 1);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int at = threadIdx.x + THREADS * i, row = at / CPT, e = at % CPT * 4;
      mask[i] = __builtin_amdgcn_raw_buffer_load_b8(mr, row, 0, 0);
      if constexpr (WHOLE) {
        const auto q = __builtin_amdgcn_raw_buffer_load_b128(sr, static_cast<int>(e < E ? row * pitch_s + e * 4 : GB_NOWHERE), 0, 0);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i][j] = __uint_as_float(q[j]);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i][j] = gb_load_f32(sr, e + j < E ? row * pitch_s + (e + j) * 4 : GB_NOWHERE);
      }
    }
  };
  auto put = [&](int buf) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int at = threadIdx.x + THREADS * i, row = at / CPT, e = at % CPT * 4;
      const bool real = !a.mask || mask[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) v[i][j] = real ? v[i][j] : 0.f;
      uint32_t q[3][2];
#pragma unroll
      for (int u = 0; u < 2; ++u) gb_split(v[i][2 * u], v[i][2 * u + 1], q[0][u], q[1][u], q[2][u]);
#pragma unroll
      for (int p = 0; p < P; ++p) *reinterpret_cast<uint2*>(lds + (buf * P + p) * PIECE + row * PITCH + e * 2) = make_uint2(q[p][0], q[p][1]);
      if (ACC && e == 0) reinterpret_cast<uint8_t*>(reals + buf * (STEP / 4))[row] = real;
    }
  };
  load(begin);
  GbFrag<BF16, V> w[KS];
  {
    const uint32_t at = 8 * g * pitch + static_cast<uint32_t>(min(col, d - V)) * B;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const auto rows = gb_rows(a.w_gate + static_cast<int64_t>(32 * k) * pitch, min(E - 32 * k, 32), pitch);
      GbRow<BF16, V> r[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) r[j].load(rows, at + j * pitch);      // zeros for experts that do not exist
      gb_transpose<BF16, V>(r, w[k]);
    }
  }
  put(0);
  __syncthreads();
  // lane 16 g + c: tokens 4 g + 0..3 of every 16, its V columns
  const uint32_t at_out = col < d ? 4 * g * pitch + static_cast<uint32_t>(col) * B : GB_NOWHERE;
  int buf = 0;
  for (uint32_t t0 = begin; t0 < end; t0 += STEP, buf ^= 1) {
    load(t0 + STEP);                                   // behind the last step nothing is read
    const int rows = min(static_cast<int>(end - t0), STEP);
    const auto out = gb_rows(a.d_x + static_cast<int64_t>(t0) * pitch, rows, pitch);
#pragma unroll
    for (int m = 0; m < GT / 16; ++m) {
      GbRow<BF16, V> old[ACC ? 4 : 1];
      if constexpr (ACC) {
#pragma unroll
        for (int r = 0; r < 4; ++r) old[r].load(out, at_out + (first + 16 * m + r) * pitch);
      }
      gb_f32x4 acc[V];
#pragma unroll
      for (int i = 0; i < V; ++i) acc[i] = gb_f32x4{0.f, 0.f, 0.f, 0.f};
      GbLow<BF16, V> low = {};
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        // lane 16 g + c: experts 32 k + 8 g + 0..7 of token 16 m + c of this wave's
        const int at = (first + 16 * m + c) * PITCH + 64 * k + 16 * g;
        uint4 q[P];
#pragma unroll
        for (int p = 0; p < P; ++p) q[p] = *reinterpret_cast<const uint4*>(lds + (buf * P + p) * PIECE + at);
        gb_products<BF16, V>(q[0], q[1], q[2], w[k], acc, low);
      }
      gb_add<BF16, V>(acc, low);
      __builtin_amdgcn_sched_barrier(0);               // (with the next tokens' operands on top of these, registers spill)
      uint32_t keep = 0x01010101u;                   // padded tokens: zeros, or nothing where d_x is added to
      if constexpr (ACC) keep = reals[buf * (STEP / 4) + first / 4 + 4 * m + g];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        GbRow<BF16, V> o;
#pragma unroll
        for (int i = 0; i < o.W; ++i) {
          if constexpr (BF16) {
            float lo = acc[2 * i][r], hi = acc[2 * i + 1][r];
            if constexpr (ACC) lo += bf16lo(old[r].w[i]), hi += bf16hi(old[r].w[i]);
            o.w[i] = pack_bf16x2(lo, hi);
          } else {
            float s = acc[i][r];
            if constexpr (ACC) s += __uint_as_float(old[r].w[i]);
            o.w[i] = __float_as_uint(s);
          }
        }
        o.store(out, keep >> (8 * r) & 1 ? at_out + (first + 16 * m + r) * pitch : GB_NOWHERE);
      }
    }
    put(buf ^ 1);
    __syncthreads();
  }
}

// A launch of its own (launch_narrow says when 17 to 32 experts have one; more always do).  Two blocks to a CU, also
// where that spills a few registers: fp32 layers of 200 experts, 2000 tokens, d = 4096 33.6 us instead of 42 with one.
template <bool BF16, int KS, int V, bool WHOLE, bool ACC>
__global__ __launch_bounds__(256, 2) void gate_x_kernel(GxArgs a) {
  using Tile = GxTile<BF16, KS, 256>;
  __shared__ __align__(16) unsigned char lds[Tile::LDS];
  __shared__ uint32_t reals[Tile::STEP / 2];
  gate_x_block<BF16, KS, V, 256, WHOLE, ACC>(a, blockIdx.x, lds, reals);
}

// Up to 32 experts, where either gradient's blocks leave room for the other's: both in one launch, eight blocks of the one
// and eight of the other in turn (one per XCD each), so that x is read while d_x is written.  (Two blocks to a CU up to 16
// experts of bf16 layers; fp32 layers' pieces would spill: 8192 tokens, d = 2048, E = 8 34 us instead of 29.)
template <bool BF16, int MT, bool WHOLE, bool ACC>
__global__ __launch_bounds__(GW_THREADS, BF16 && MT == 1 && !ACC ? 4 : 2) void gate_narrow_kernel(GwArgs w, int blocks_w, GxArgs x, int blocks_x) {
  constexpr int V = BF16 ? 8 : 4;
  using Tile = GxTile<BF16, 1, GW_THREADS>;
  __shared__ __align__(16) unsigned char lds[Tile::LDS > GW_LDS ? Tile::LDS : GW_LDS];
  __shared__ double red_b[GW_WAVES][16 * MT];
  __shared__ uint32_t reals[Tile::STEP / 2];
  const int group = blockIdx.x / 8, both = min((blocks_w + 7) / 8, (blocks_x + 7) / 8);
  const bool of_w = group < 2 * both ? group % 2 == 0 : blocks_w > blocks_x;
  const int block = (group < 2 * both ? group / 2 : group - both) * 8 + blockIdx.x % 8;
  if (of_w) {
    if (block < blocks_w) gate_weight_block<BF16, MT, V>(w, block, lds, red_b);
  } else {
    if (block < blocks_x) gate_x_block<BF16, 1, V, GW_THREADS, WHOLE, ACC>(x, block, lds, reals);
  }
}

// ------------------------------------------------------------------------------------------------ launches
// Blocks of the weights' gradient: column tiles, groups of experts, and parts of the tokens, of which there are as many
// as fill the chip (twice with 16 or 32 experts to a block), each of a step of the block or more.
//
// Up to 1024 tokens are one part, whose sums are stored at once: that saves a launch.  (Measured, one part / as many as
// fit, us: d = 4096, 501 tokens, E = 8 10.8 / 14.1; 1000 tokens, E = 128 11.9 / 19.8; d = 1048, 1000 tokens, E = 12
// 10.2 / 13.4.)
//
// More than 32 experts: blocks of 32 read x once for every 32, blocks of 64 are four times as wide and leave that many more
// parts to be added up.  So the former take what is small, counted in bytes of x read.  (Measured, blocks of 32 / of 64,
// us: d = 2048, E = 64, 16384 tokens 27 / 32, 32768 50 / 42, 65536 82 / 63; d = 4096, E = 128, 2000 tokens 24 / 26, 4096
// 33 / 31, 8192 52 / 39; E = 256, 3000 tokens 43 / 33; d = 1048, E = 100, 8192 tokens 23 / 25.)
struct GwPlan {
  int mt, tiles, chunks, splits, per_split;
};
static GwPlan gw_plan(const moe_shape_t* s) {
  GwPlan p{};
  const int64_t x_reads = static_cast<int64_t>(s->T) * s->d * elem_bytes(s->dtype) * ((s->E + 31) / 32);
  const bool wide = s->E > 32 && x_reads > (int64_t(s->E <= 64 ? 128 : 64) << 20);
  p.mt = s->E <= 16 ? 1 : wide ? 4 : 2;
  const int v = s->dtype == MOE_F32 ? 4 : 8, cols = 16 * v * (p.mt == 4 ? 4 : 1);
  p.tiles = (s->d + cols - 1) / cols;
  p.chunks = (s->E + 16 * p.mt - 1) / (16 * p.mt);
  const int step = p.mt == 4 ? 64 : 32 * GW_WAVES;
  const int64_t most = (static_cast<int64_t>(s->T) + step - 1) / step;
  int64_t n = (p.mt == 4 ? 256 : 512) / (static_cast<int64_t>(p.tiles) * p.chunks);
  if (n > most) n = most;
  if (s->T <= 1024 && !wide) n = 1;
  if (n > 8) n = n / 8 * 8;
  if (n < 1) n = 1;
  int64_t per = (s->T + n - 1) / n;
  const int unit = p.mt == 4 ? 64 : 32;
  per = (per + unit - 1) / unit * unit;
  p.per_split = static_cast<int>(per < unit ? unit : per);
  p.splits = static_cast<int>(n);
  return p;
}

size_t gate_backward_workspace_bytes(const moe_shape_t* shape) {
  const GwPlan p = gw_plan(shape);
  return p.splits > 1 ? static_cast<size_t>(p.splits) * shape->E * (static_cast<size_t>(shape->d) + 1) * sizeof(float) : 0;
}

// Column tiles and parts of the tokens of the hidden states' gradient, for blocks of `step` tokens at a time.
static GxArgs gx_plan(GxArgs a, int cols, int step, int most_blocks) {
  a.tiles = (a.d + cols - 1) / cols;
  const int64_t most = (static_cast<int64_t>(a.T) + step - 1) / step;
  int64_t n = most_blocks / a.tiles;
  if (n > most) n = most;
  if (n > 8) n = n / 8 * 8;
  if (n < 1) n = 1;
  const int64_t per = (a.T + n - 1) / n;
  a.splits = static_cast<int>(n);
  a.per_split = static_cast<int>((per + step - 1) / step * step);
  return a;
}

// (Measured for both gradients, 256 / 512 / 1024 blocks, us: 3000 tokens, d = 4096, E = 200 56 / 52 / 55; 4000, d = 5120,
// E = 100 61 / 52 / 52; 30000, d = 2048, E = 32 62 / 65 / 68; 65536, d = 2048, E = 64 116 to 123 / 117 / 115.)
template <bool BF16, int KS> static void launch_x(GxArgs x, bool accumulate, hipStream_t st) {
  constexpr int V = KS <= 2 ? (BF16 ? 8 : 4) : (BF16 ? 4 : 2);
  x = gx_plan(x, 16 * V * GX_SIDE, GxTile<BF16, KS, 256>::STEP, 512);
  const bool whole = x.E % 4 == 0;
  const auto kernel = accumulate ? (whole ? gate_x_kernel<BF16, KS, V, true, true> : gate_x_kernel<BF16, KS, V, false, true>)
                                 : (whole ? gate_x_kernel<BF16, KS, V, true, false> : gate_x_kernel<BF16, KS, V, false, false>);
  hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(x.tiles * x.splits)), dim3(256), 0, st, x);
}

// One launch for both gradients, but two for 17 to 32 experts beyond a round of blocks: their weights' blocks have a CU to
// themselves, which costs the hidden states' more than the launch.  (Measured in a captured graph, one launch / two, us: E = 8,
// d = 4096, 501 tokens 6.4 / 9.7, 4096 19.0 / 20.2, 65536 217 / 195; E = 16, 30000 tokens 104 / 97; E = 32, 2000 tokens,
// d = 2048 10.7 / 14.5; E = 24, 32768 tokens, d = 4096 139 / 118.  So up to 16 experts, too, large batches would gain from two.)
template <bool BF16, int MT> static void launch_narrow(const GwArgs& w, const GxArgs& gx, bool with_w, bool with_x, bool accumulate, hipStream_t st) {
  const GxArgs x = gx_plan(gx, 16 * (BF16 ? 8 : 4) * GX_SIDE, GxTile<BF16, 1, GW_THREADS>::STEP, 512);
  const int blocks_w = with_w ? w.tiles * w.chunks * w.splits : 0;
  int blocks_x = with_x ? x.tiles * x.splits : 0;
  if (MT == 2 && blocks_w + blocks_x > 256 && with_x) {
    launch_x<BF16, 1>(gx, accumulate, st);
    blocks_x = 0;
  }
  const bool whole = x.E % 4 == 0;
  const auto kernel = accumulate ? (whole ? gate_narrow_kernel<BF16, MT, true, true> : gate_narrow_kernel<BF16, MT, false, true>)
                                 : (whole ? gate_narrow_kernel<BF16, MT, true, false> : gate_narrow_kernel<BF16, MT, false, false>);
  const unsigned groups = static_cast<unsigned>((blocks_w + 7) / 8 + (blocks_x + 7) / 8);
  if (groups > 0) hipLaunchKernelGGL(kernel, dim3(8 * groups), dim3(GW_THREADS), 0, st, w, blocks_w, x, blocks_x);
}

template <bool BF16> static int launch_wide(const GwArgs& w, hipStream_t st) {
  const auto kernel = gate_weight_wide_kernel<BF16, BF16 ? 8 : 4>;
  static LdsOnce once;
  const int rc = ensure_dynamic_lds(once, reinterpret_cast<const void*>(kernel), GWW_LDS);
  if (rc != MOE_OK) return rc;
  hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(w.tiles * w.chunks * w.splits)), dim3(GW_THREADS), GWW_LDS, st, w);
  return MOE_OK;
}

template <bool BF16>
static int gate_backward(const moe_shape_t* s, const void* x, const void* w_gate, const float* d_scores, const uint8_t* mask,
                         float* d_w_gate, float* d_gate_bias, void* d_x, int accumulate, float* part, hipStream_t st) {
  const int acc_w = accumulate & MOE_ACCUMULATE_WEIGHTS ? 1 : 0, acc_x = accumulate & MOE_ACCUMULATE_X ? 1 : 0;
  const bool with_w = d_w_gate || d_gate_bias, with_x = d_x && s->T > 0;
  const GwPlan p = gw_plan(s);
  const int64_t n = static_cast<int64_t>(s->E) * s->d;
  const bool parts = p.splits > 1;
  float* part_b = part + p.splits * n;
  const GwArgs gw = {static_cast<const char*>(x), d_scores, mask, d_w_gate ? (parts ? part : d_w_gate) : nullptr,
                     d_gate_bias ? (parts ? part_b : d_gate_bias) : nullptr, s->T, s->d, s->E, p.tiles, p.chunks, p.splits, p.per_split, acc_w};
  const GxArgs gx = {static_cast<const char*>(w_gate), d_scores, mask, static_cast<char*>(d_x), s->T, s->d, s->E, 0, 0, 0};
  if (s->E <= 16) {
    launch_narrow<BF16, 1>(gw, gx, with_w, with_x, acc_x, st);
  } else if (s->E <= 32) {
    launch_narrow<BF16, 2>(gw, gx, with_w, with_x, acc_x, st);
  } else {
    if (with_w && p.mt == 2) {
      launch_narrow<BF16, 2>(gw, gx, true, false, false, st);
    } else if (with_w) {
      const int rc = launch_wide<BF16>(gw, st);
      if (rc != MOE_OK) return rc;
    }
    if (with_x) {
      if (s->E <= 64) launch_x<BF16, 2>(gx, acc_x, st);
      else if (s->E <= 128) launch_x<BF16, 4>(gx, acc_x, st);
      else launch_x<BF16, 8>(gx, acc_x, st);
    }
  }
  if (with_w && parts) {
    const int columns = GS_THREADS / (p.splits > 64 ? 8 : 2);
    const int blocks_w = d_w_gate ? static_cast<int>((n / 4 + columns - 1) / columns) : 0;
    const int blocks_b = d_gate_bias ? (s->E + columns - 1) / columns : 0;
    const auto kernel = p.splits > 64 ? gate_sum_kernel<8> : gate_sum_kernel<2>;
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(blocks_w + blocks_b)), dim3(GS_THREADS), 0, st, part, d_w_gate, n, blocks_w, part_b,
                       d_gate_bias, s->E, p.splits, acc_w);
  }
  return launch_status();
}

}  // namespace moe

extern "C" int moe_train_workspace_bytes(const moe_shape_t* shape, size_t* out_bytes) {
  const int rc = moe::check_shape(shape);
  if (rc != MOE_OK) return rc;
  if (!out_bytes) return MOE_ERR_INVALID_ARG;
  *out_bytes = moe::train_workspace_bytes(shape);
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
  if (static_cast<int64_t>(shape->d) * elem_bytes(shape->dtype) > GB_ROW_BYTES) return MOE_ERR_UNSUPPORTED;
  if (shape->T > 0 && (!d_scores || (d_w_gate && !x) || (d_x && !w_gate))) return MOE_ERR_INVALID_ARG;
  if (d_w_gate || d_gate_bias) {
    if (!workspace || !aligned16(workspace)) return MOE_ERR_INVALID_ARG;
    if (workspace_bytes < train_workspace_bytes(shape)) return MOE_ERR_WORKSPACE;
  }
  const int64_t rows = static_cast<int64_t>(shape->T) * shape->d * elem_bytes(shape->dtype);
  const int64_t gate = static_cast<int64_t>(shape->E) * shape->d * elem_bytes(shape->dtype);
  const int64_t table = int64_t(4) * shape->T * shape->E, d_gate = int64_t(4) * shape->E * shape->d;
  if (!apart(d_x, rows, x, rows) || !apart(d_x, rows, w_gate, gate) || !apart(d_x, rows, d_scores, table) || !apart(d_w_gate, d_gate, x, rows) ||
      !apart(d_w_gate, d_gate, w_gate, gate) || !apart(d_w_gate, d_gate, d_scores, table) || !apart(d_w_gate, d_gate, d_x, rows))
    return MOE_ERR_INVALID_ARG;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  return shape->dtype == MOE_BF16
             ? gate_backward<true>(shape, x, w_gate, d_scores, token_mask, d_w_gate, d_gate_bias, d_x, accumulate, static_cast<float*>(workspace), st)
             : gate_backward<false>(shape, x, w_gate, d_scores, token_mask, d_w_gate, d_gate_bias, d_x, accumulate, static_cast<float*>(workspace), st);
}
