// The dense FP8 projection and its gradients: E4M3 operands with a power-of-two scale for every block of 128 along the contraction
// (weights: every 128 x 128 tile), float32 accumulation on the block-scaled tensor cores.
//   forward       out[T, N] = Q(x) Q(W)^T         blocks of 128 channels           bf16
//   input's       dx[T, K]  = Q(dy) Q(W)          blocks of 128 output features    bf16
//   weight's      dW[N, K]  = Q'(dy)^T Q'(x)      Q': blocks of 128 tokens         float32
// One layout of the codes serves all three: an operand whose contraction runs along its rows is loaded as it lies and read by the
// MMA in its "MN-major" form, so that neither W nor dy nor x is ever transposed.  A scale is one byte per (row or column, block); the
// tensor core wants it as atoms of 128 rows x 4 bytes (a byte per 32 elements of the contraction: the same four times).
#include "fp8.cuh"
#include "kernels.cuh"
#include "split_k.cuh"
#include <climits>

namespace quads {
namespace {

// ---------------------------------------------------------------------------
// Quantization.  One CTA per tile of 128 x 128 values, read once and kept in registers (thread = 8 columns of 8 rows); by rows
// (blocks of 128 columns) and / or by columns (blocks of 128 rows).  Maxima are packed 16-bit integer maxima of the bf16 magnitudes.
// Elements beyond the tensor count as zeros; the atoms' bytes for rows beyond it are those of a zero row.
// ---------------------------------------------------------------------------
// 16 bytes that this SM does not read again.
__device__ __forceinline__ uint4 ldg128_once(const void* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) { return __vmaxu2(a, b); }

__global__ void __launch_bounds__(256)
fp8_quantize_tiles_kernel(const Fp8QuantArgs a0, const Fp8QuantArgs a1, int tiles0, int32_t* __restrict__ status) {
  pdl_sync();
  if (blockIdx.x == 0 && threadIdx.x == 0) *status = 0;
  const bool second = (int)blockIdx.x >= tiles0;
  const Fp8QuantArgs& a = second ? a1 : a0;
  const int tile = (int)blockIdx.x - (second ? tiles0 : 0);
  const int ct = (a.cols + 127) >> 7;                       // column tiles
  const int tr = tile / ct, tc = tile - tr * ct;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int col = tc * 128 + tx * 8;
  const int64_t row0 = (int64_t)tr * 128 + ty;
  __shared__ uint32_t s_col[8][64];
  __shared__ uint8_t s_rcode[128], s_ccode[128];
  uint4 v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t r = row0 + 16 * i;
    v[i] = make_uint4(0u, 0u, 0u, 0u);
    if (r < a.rows && col < a.cols) v[i] = ldg128_once(a.v + r * a.ld + col);
  }
  if (a.codes_c) {
    uint32_t m[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      m[0] = max2(m[0], v[i].x & 0x7FFF7FFFu);
      m[1] = max2(m[1], v[i].y & 0x7FFF7FFFu);
      m[2] = max2(m[2], v[i].z & 0x7FFF7FFFu);
      m[3] = max2(m[3], v[i].w & 0x7FFF7FFFu);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) m[k] = max2(m[k], __shfl_xor_sync(0xFFFFFFFFu, m[k], 16));
    if (lane < 16) {
#pragma unroll
      for (int k = 0; k < 4; ++k) s_col[warp][tx * 4 + k] = m[k];
    }
  }
  uint32_t rcode[8];
  if (a.codes_r) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      // the maxima of two rows, one in each half of a word
      const uint32_t p = absmax8(v[i]), q = absmax8(v[i + 1]);
      uint32_t m = max2(__byte_perm(p, q, 0x5410), __byte_perm(p, q, 0x7632));
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) m = max2(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
      rcode[i] = fp8_scale_code(__uint_as_float(m << 16));
      rcode[i + 1] = fp8_scale_code(__uint_as_float(m & 0xFFFF0000u));
    }
    if (tx == 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) s_rcode[ty + 16 * i] = (uint8_t)rcode[i];
    }
  }
  if (a.codes_c) {
    __syncthreads();
    if (threadIdx.x < 64) {
      uint32_t m = s_col[0][threadIdx.x];
#pragma unroll
      for (int w = 1; w < 8; ++w) m = max2(m, s_col[w][threadIdx.x]);
      s_ccode[2 * threadIdx.x] = (uint8_t)fp8_scale_code(__uint_as_float(m << 16));
      s_ccode[2 * threadIdx.x + 1] = (uint8_t)fp8_scale_code(__uint_as_float(m & 0xFFFF0000u));
    }
  }
  __syncthreads();
  float csc[8];
  if (a.codes_c) {
    const uint2 c8 = *reinterpret_cast<const uint2*>(s_ccode + tx * 8);
#pragma unroll
    for (int k = 0; k < 8; ++k) csc[k] = fp8_inv_scale(((k < 4 ? c8.x : c8.y) >> (8 * (k & 3))) & 0xFFu);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t r = row0 + 16 * i;
    if (r >= a.rows || col >= a.cols) continue;
    float f[8];
    unpack8(v[i], f);
    if (a.codes_r) {
      const float sc = fp8_inv_scale(rcode[i]);
      *reinterpret_cast<uint2*>(a.codes_r + r * a.cols + col) =
          make_uint2(f32x4_to_e4m3x4(__fmul_rn(f[0], sc), __fmul_rn(f[1], sc), __fmul_rn(f[2], sc), __fmul_rn(f[3], sc)),
                     f32x4_to_e4m3x4(__fmul_rn(f[4], sc), __fmul_rn(f[5], sc), __fmul_rn(f[6], sc), __fmul_rn(f[7], sc)));
    }
    if (a.codes_c)
      *reinterpret_cast<uint2*>(a.codes_c + r * a.cols + col) =
          make_uint2(f32x4_to_e4m3x4(__fmul_rn(f[0], csc[0]), __fmul_rn(f[1], csc[1]), __fmul_rn(f[2], csc[2]), __fmul_rn(f[3], csc[3])),
                     f32x4_to_e4m3x4(__fmul_rn(f[4], csc[4]), __fmul_rn(f[5], csc[5]), __fmul_rn(f[6], csc[6]), __fmul_rn(f[7], csc[7])));
  }
  // atoms: word (row % 32) * 4 + row / 32 is the row's scale byte, four times
  const int w = threadIdx.x & 127, wrow = (w & 3) * 32 + (w >> 2);
  if (threadIdx.x < 128) {
    if (a.codes_r) reinterpret_cast<uint32_t*>(a.atoms_r + ((size_t)tr * ct + tc) * 512)[w] = s_rcode[wrow] * 0x01010101u;
  } else if (a.codes_c) {
    const size_t rt = (size_t)((a.rows + 127) >> 7);
    reinterpret_cast<uint32_t*>(a.atoms_c + ((size_t)tc * rt + tr) * 512)[w] = s_ccode[wrow] * 0x01010101u;
  }
}

// The same for smaller tensors, which are bound by latency: by rows 16 rows of 128 columns to a CTA, by columns 128 rows of 64, so that the
// work spreads over more SMs and a thread's chain is one row or four long (a tensor that needs both is read twice, out of L2 the second time).
// Whole calls, us, so / in tiles of 128 x 128: forward (rows alone, a kernel of its own: with the columns' registers 512 rows take 15.0)
// 61 x 2048 -> 1536 7.1 / 7.8, 512 x 4096 -> 4096 13.6 / 16.3, 2048 x 4096 34.1 / 34.5, 4096 x 4096 63.7 / 63.5, 8192 x 4096 118.4 / 115.9; both
// gradients 16 x 2048 -> 1536 10.5 / 11.0, 333 x 2048 -> 1536 13.2 / 14.3, 1024 x 2048 -> 2048 22.3 / 21.9, 2048 x 4096 -> 4096 78 / 73.
constexpr int64_t kQuantRowsElements = 12 << 20, kQuantSmallElements = 5 << 19;
__device__ __forceinline__ void quantize_row_tile(const Fp8QuantArgs& a, int tile) {
  const int ct = (a.cols + 127) >> 7, tr = tile / ct, tc = tile - tr * ct;
  const int tx = threadIdx.x & 15, r = tr * 16 + (threadIdx.x >> 4), col = tc * 128 + tx * 8;
  const bool on = r < a.rows && col < a.cols;
  uint4 v = make_uint4(0u, 0u, 0u, 0u);
  if (on) v = ldg128_once(a.v + r * a.ld + col);
  uint32_t m = absmax8(v);
  m = max(m & 0xFFFFu, m >> 16);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
  const uint32_t code = fp8_scale_code(__uint_as_float(m << 16));
  const float sc = fp8_inv_scale(code);
  float f[8];
  unpack8(v, f);
  if (on)
    *reinterpret_cast<uint2*>(a.codes_r + (int64_t)r * a.cols + col) =
        make_uint2(f32x4_to_e4m3x4(__fmul_rn(f[0], sc), __fmul_rn(f[1], sc), __fmul_rn(f[2], sc), __fmul_rn(f[3], sc)),
                   f32x4_to_e4m3x4(__fmul_rn(f[4], sc), __fmul_rn(f[5], sc), __fmul_rn(f[6], sc), __fmul_rn(f[7], sc)));
  // (the atom's words of rows beyond the tensor are left: the products read them for rows that nobody stores)
  if (tx == 0 && r < a.rows)
    reinterpret_cast<uint32_t*>(a.atoms_r + ((size_t)(r >> 7) * ct + tc) * 512)[(r & 31) * 4 + ((r >> 5) & 3)] = code * 0x01010101u;
}

__device__ __forceinline__ void quantize_column_tile(const Fp8QuantArgs& a, int tile, uint32_t (*s_max)[32]) {
  const int ct = (a.cols + 63) >> 6, tr = tile / ct, tc = tile - tr * ct;
  const int tx = threadIdx.x & 7, ty = threadIdx.x >> 3, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int col = tc * 64 + tx * 8;
  const int64_t row0 = (int64_t)tr * 128 + ty;
  uint4 v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t r = row0 + 32 * i;
    v[i] = make_uint4(0u, 0u, 0u, 0u);
    if (r < a.rows && col < a.cols) v[i] = ldg128_once(a.v + r * a.ld + col);
  }
  uint32_t m[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m[0] = max2(m[0], v[i].x & 0x7FFF7FFFu);
    m[1] = max2(m[1], v[i].y & 0x7FFF7FFFu);
    m[2] = max2(m[2], v[i].z & 0x7FFF7FFFu);
    m[3] = max2(m[3], v[i].w & 0x7FFF7FFFu);
  }
#pragma unroll
  for (int o = 8; o < 32; o <<= 1) {
#pragma unroll
    for (int k = 0; k < 4; ++k) m[k] = max2(m[k], __shfl_xor_sync(0xFFFFFFFFu, m[k], o));
  }
  if (lane < 8) *reinterpret_cast<uint4*>(&s_max[warp][tx * 4]) = make_uint4(m[0], m[1], m[2], m[3]);
  __syncthreads();
  // every thread: the scales of its eight columns
  uint32_t code[8];
#pragma unroll
  for (int w = 0; w < 8; ++w) {
    const uint4 o = *reinterpret_cast<const uint4*>(&s_max[w][tx * 4]);
    if (w == 0) { m[0] = o.x; m[1] = o.y; m[2] = o.z; m[3] = o.w; }
    else { m[0] = max2(m[0], o.x); m[1] = max2(m[1], o.y); m[2] = max2(m[2], o.z); m[3] = max2(m[3], o.w); }
  }
  float sc[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    code[k] = fp8_scale_code(__uint_as_float((k & 1) ? m[k >> 1] & 0xFFFF0000u : m[k >> 1] << 16));
    sc[k] = fp8_inv_scale(code[k]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t r = row0 + 32 * i;
    if (r >= a.rows || col >= a.cols) continue;
    float f[8];
    unpack8(v[i], f);
    *reinterpret_cast<uint2*>(a.codes_c + r * a.cols + col) =
        make_uint2(f32x4_to_e4m3x4(__fmul_rn(f[0], sc[0]), __fmul_rn(f[1], sc[1]), __fmul_rn(f[2], sc[2]), __fmul_rn(f[3], sc[3])),
                   f32x4_to_e4m3x4(__fmul_rn(f[4], sc[4]), __fmul_rn(f[5], sc[5]), __fmul_rn(f[6], sc[6]), __fmul_rn(f[7], sc[7])));
  }
  if (ty == 0 && col < a.cols) {
    const size_t rt = (size_t)((a.rows + 127) >> 7);
    uint32_t* atom = reinterpret_cast<uint32_t*>(a.atoms_c + ((size_t)(col >> 7) * rt + tr) * 512);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int c = (col + k) & 127;
      atom[(c & 31) * 4 + (c >> 5)] = code[k] * 0x01010101u;
    }
  }
}

__global__ void __launch_bounds__(256)
fp8_quantize_rows_kernel(const Fp8QuantArgs a, int32_t* __restrict__ status) {
  pdl_sync();
  if (blockIdx.x == 0 && threadIdx.x == 0) *status = 0;
  quantize_row_tile(a, (int)blockIdx.x);
}
// CTAs: a0's rows, a0's columns, a1's columns (each may be none).
__global__ void __launch_bounds__(256)
fp8_quantize_small_kernel(const Fp8QuantArgs a0, const Fp8QuantArgs a1, int rows0, int cols0, int32_t* __restrict__ status) {
  pdl_sync();
  __shared__ __align__(16) uint32_t s_max[8][32];
  if (blockIdx.x == 0 && threadIdx.x == 0) *status = 0;
  const int b = (int)blockIdx.x;
  if (b < rows0) quantize_row_tile(a0, b);
  else if (b < rows0 + cols0) quantize_column_tile(a0, b - rows0, s_max);
  else quantize_column_tile(a1, b - rows0 - cols0, s_max);
}

// ---------------------------------------------------------------------------
// Shared by the two products
// ---------------------------------------------------------------------------
constexpr int kChunkBlocks = 32;                       // of 128: the contraction's piece of a float32 result
constexpr int kLTile = 128 * 128;                      // 128 rows of 128 bytes (or 128 steps of the contraction x 128 rows)
constexpr uint32_t kLSwHi = (uint32_t)((8 * 128) >> 4) | (1u << 14) | (2u << 29);      // 128-byte swizzle, groups of eight 1 KB apart
constexpr uint32_t kLSfHi = (uint32_t)(128 >> 4) | (1u << 14);

// An operand of the MMA: low word of its shared-memory descriptor, and what 32 steps of the contraction add to it.  K-major: 32 bytes
// inside the swizzled 128-byte rows; MN-major: 32 rows of 128 bytes (128 of M or N are one swizzle pattern wide: the leading offset is
// not used).
__device__ __forceinline__ uint32_t operand_lo(uint32_t saddr, bool mn) { return ((saddr & 0x3FFFFu) >> 4) | (mn ? (uint32_t)(kLTile >> 4) << 16 : 1u << 16); }
__device__ __forceinline__ uint32_t operand_step(bool mn) { return mn ? (32u * 128u) >> 4 : 2u; }
// E4M3 x E4M3, UE8M0 block scales, m x n outputs; the MMA's scale byte (bits 4 and 29 on) is added where it is issued.
__device__ __forceinline__ uint32_t fp8_idesc(int m, int n, bool a_mn, bool b_mn) {
  return (1u << 23) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ void load_operand(uint32_t dst, const CUtensorMap* map, bool mn, int kb, int row0, uint32_t bar) {
  tma_load_2d(dst, map, mn ? row0 : kb * 128, mn ? kb * 128 : row0, bar);
}
__device__ __forceinline__ void load_operand_pair(uint32_t dst, const CUtensorMap* map, bool mn, int kb, int row0, uint32_t bar) {
  tma_load_2d_pair(dst, map, mn ? row0 : kb * 128, mn ? kb * 128 : row0, bar);
}

// Stores a warp's 32 rows of 128 bytes (thread = row, w[32]: 64 bf16 or 32 float32) to rows `pitch` bytes apart, the first `bytes`
// bytes (a multiple of 32) of the first `rows` rows; transposed in groups of four lanes as in store_y_rows, so that a store writes
// complete lines.  kF32 and add: added to what is there.  wide: the addresses are aligned to 32 bytes, else to 16.
template <bool kF32>
__device__ __forceinline__ void store_lines(uint32_t* w, uint8_t* dst, size_t pitch, int bytes, int rows, bool wide, bool add, int lane) {
#pragma unroll
  for (int s = 1; s < 4; s <<= 1) {
    const bool up = (lane & s) != 0;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      if (c & s) continue;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const uint32_t lo = w[8 * c + k], hi = w[8 * (c | s) + k];
        const uint32_t got = __shfl_xor_sync(0xFFFFFFFFu, up ? lo : hi, s);
        w[8 * c + k] = up ? got : lo;
        w[8 * (c | s) + k] = up ? hi : got;
      }
    }
  }
  const int g = lane >> 2, j = lane & 3;
  if (32 * j >= bytes) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = 4 * g + i;
    if (r >= rows) continue;
    uint8_t* d = dst + (size_t)r * pitch + 32 * j;
    uint32_t* v = w + 8 * i;
    if (kF32 && add) {
      const float4 a = reinterpret_cast<const float4*>(d)[0], b = reinterpret_cast<const float4*>(d)[1];
      const float o[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = __float_as_uint(__fadd_rn(o[k], __uint_as_float(v[k])));
    }
    if (wide) {
      stg256(d, v);
    } else {
      reinterpret_cast<uint4*>(d)[0] = make_uint4(v[0], v[1], v[2], v[3]);
      reinterpret_cast<uint4*>(d)[1] = make_uint4(v[4], v[5], v[6], v[7]);
    }
  }
}

// 64 accumulator columns (bits of float32) of a warp's 32 rows to the output at (row0, n0).
__device__ __forceinline__ void store_acc(uint32_t* v, const Fp8Problem& q, int64_t row0, int n0, bool add, int lane) {
  const int rows = (int)min((int64_t)32, q.M - row0), cols = min(64, q.N - n0);
  if (rows <= 0 || cols <= 0) return;                             // (the whole warp)
  const bool wide = (reinterpret_cast<size_t>(q.out) & 31) == 0;
  if (q.f32) {
    uint8_t* dst = reinterpret_cast<uint8_t*>(static_cast<float*>(q.out) + row0 * q.N + n0);
    store_lines<true>(v, dst, (size_t)q.N * 4, cols * 4, rows, wide, add, lane);
    if (cols > 32) store_lines<true>(v + 32, dst + 128, (size_t)q.N * 4, (cols - 32) * 4, rows, wide, add, lane);
  } else {
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = f32x2_to_bf16x2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1]));
    store_lines<false>(v, reinterpret_cast<uint8_t*>(static_cast<uint16_t*>(q.out) + row0 * q.N + n0), (size_t)q.N * 2, cols * 2, rows, wide, false, lane);
  }
}

// 32 consecutive accumulator columns of this thread's tensor-memory lane, as bits.
__device__ __forceinline__ void tmem_ld32_bits(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr) : "memory");
}

// ---------------------------------------------------------------------------
// Large products: persistent pairs of CTAs, 256 x 256 or 256 x 192 tiles (cta_group::2), each CTA with its own 128 rows of A and half of B's
// -- 32 or 28 KB a stage and 128 of K, six or seven stages.  One float32 accumulator of 256 columns (two do not fit beside the scales), drained
// by sixteen warps into registers at once.  (96 registers a thread leave the form of 256 columns a stack of 16 bytes: 24 bytes of spill stores, 64 of
// loads.  The form of 192 columns has none.)
// ---------------------------------------------------------------------------
template <int kN>
struct PCfg {
  static constexpr int kB = kN / 2 * 128;                // bytes of B in a stage
  static constexpr int kOffSfA = kLTile + kB, kOffSfB = kOffSfA + 512;
  static constexpr int kStageBytes = (kOffSfB + 1024 + 1023) / 1024 * 1024;
  static constexpr int kStages = kN == 256 ? 6 : 7;
  static constexpr int kBarOffset = kStages * kStageBytes;
  static constexpr int kSmemBytes = kBarOffset + 256 + 1024;
  static_assert(kN == 256 || kN == 192, "columns of a tile");
  static_assert(kSmemBytes <= 232448, "shared memory");
};
constexpr int kPThreads = 608;
constexpr int kPEpiWarps = 16;
constexpr int kPLoadB = 18;                              // warp 0 loads A

struct __align__(8) PBarriers {
  uint64_t full[7];
  uint64_t empty[7];
  uint64_t tmem_full;
  uint64_t tmem_empty;
  uint32_t tmem_base;
  int abort_flag;
};

template <int kN>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPThreads, 1)
fp8_pair_kernel(const Fp8LinearParams p, const __grid_constant__ Fp8LinearMaps maps) {
  using C = PCfg<kN>;
  constexpr int kPStages = C::kStages, kPStageBytes = C::kStageBytes;
  extern __shared__ uint8_t smem_dyn[];
  const uint32_t smem_base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
  uint8_t* smem_gen = smem_dyn + (smem_base - smem_u32(smem_dyn));
  PBarriers* bars = reinterpret_cast<PBarriers*>(smem_gen + C::kBarOffset);
  const uint32_t bar_full = smem_u32(&bars->full[0]), bar_empty = smem_u32(&bars->empty[0]);
  const uint32_t bar_tfull = smem_u32(&bars->tmem_full), bar_tempty = smem_u32(&bars->tmem_empty);
  volatile int* abort_flag = &bars->abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const bool leader = rank == 0;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kPStages; ++s) { mbar_init(bar_full + 8 * s, leader ? 4 : 1); mbar_init(bar_empty + 8 * s, 1); }
    mbar_init(bar_tfull, 1);
    mbar_init(bar_tempty, kPEpiWarps * 2);
    bars->abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    prefetch_tmap(&maps.a[0]);
    prefetch_tmap(&maps.b[0]);
  }
  if (warp == 1) tmem_alloc<2>(smem_u32(&bars->tmem_base), 512);
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem = bars->tmem_base;
  // The problems' tiles are dealt in rounds, those of problem 1 from pair first_1 on; a pair does its tiles of problem 0 first.  Those that
  // have one more tile of problem 0 come to problem 1 some rounds later.
  const int pair = (int)blockIdx.x / 2, n_pairs = (int)gridDim.x / 2;
  auto my_first = [&](int i) {
    const int at = pair - p.first[i] + (pair < p.first[i] ? n_pairs : 0);
    return at < p.ctas[i] / 2 ? at + (i == 1 && pair < p.first[1] ? p.early_tiles : 0) : INT_MAX;
  };
  auto my_next = [&](int i, int tile) { return tile + (i == 1 && tile < p.early_tiles ? p.early_step : p.ctas[i] / 2); };
  // Weights are older than the kernel in front, this call's quantization, which waited for its own predecessor before this one could
  // start: their loader goes ahead until it comes to the other problem's operand.
  bool waited = warp != kPLoadB;
  if (waited) pdl_sync();

  if (warp == 0 || warp == kPLoadB) {
    // ------------------------------------------------------------ loaders
    const bool issuer = elect_one(), loads_b = warp == kPLoadB;
    uint32_t stage = 0, phase = 0;
    bool ok = true;
    const uint32_t leader_full = map_to_cta(bar_full, 0);
    for (int i = 0; i < 2 && ok; ++i) {
      const Fp8Problem& q = p.pr[i];
      const CUtensorMap *tm = loads_b ? &maps.b[i] : &maps.a[i], *tm_sf = loads_b ? &maps.sfb[i] : &maps.sfa[i];
      const bool mn = loads_b ? q.b_mn : q.a_mn;
      const int last = ((loads_b ? q.N : q.M) + 127) / 128 - 1, n_tiles = q.n_tiles, total = p.tiles[i], k_blocks = q.k_blocks;
      const int sf_tile = loads_b ? q.b_sf_tile : q.a_sf_tile, sf_kb = loads_b ? q.b_sf_kb : q.a_sf_kb;
      for (int tile = my_first(i); tile < total && ok; tile = my_next(i, tile)) {
        if (!waited && !q.b_early) { pdl_sync(); waited = true; }
        const int mt = tile / n_tiles, nt = tile - mt * n_tiles;
        // (a tile beyond the operand is loaded as zeros, with the scales of the last one)
        const int t128 = loads_b ? nt * kN / 128 : mt * 2, row0 = loads_b ? nt * kN + (int)rank * (kN / 2) : (t128 + (int)rank) * 128;
        const int sf0 = min(loads_b ? t128 : t128 + (int)rank, last) * sf_tile, sf1 = min(t128 + 1, last) * sf_tile;
        for (int ks = 0; ks < k_blocks; ++ks) {
          ok = mbar_wait(bar_empty + 8 * stage, phase ^ 1u, abort_flag, p.status);
          if (!ok) break;
          if (issuer) {
            const uint32_t sb = smem_base + stage * kPStageBytes, full = leader_full + 8 * stage;
            mbar_expect_tx_cluster(full, loads_b ? C::kB + 1024u : kLTile + 512u);
            load_operand_pair(sb + (loads_b ? kLTile : 0), tm, mn, ks, row0, full);
            tma_load_2d_pair(sb + (loads_b ? C::kOffSfB : C::kOffSfA), tm_sf, 0, sf0 + ks * sf_kb, full);
            if (loads_b) tma_load_2d_pair(sb + C::kOffSfB + 512, tm_sf, 0, sf1 + ks * sf_kb, full);
          }
          __syncwarp();
          if (++stage == kPStages) { stage = 0; phase ^= 1u; }
        }
      }
    }
    for (int s = 0; s < kPStages && ok; ++s) {             // drain: every armed stage lands and is consumed
      ok = mbar_wait(bar_empty + 8 * stage, phase ^ 1u, abort_flag, p.status);
      if (++stage == kPStages) { stage = 0; phase ^= 1u; }
    }
  } else if (warp == 1 && !leader) {
    // the leader CTA issues the MMAs of the pair
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer
    const bool issuer = elect_one();
    uint32_t stage = 0, phase = 0, kcount = 0;
    int it = 0;
    bool ok = true;
    for (int i = 0; i < 2 && ok; ++i) {
      const bool a_mn = p.pr[i].a_mn, b_mn = p.pr[i].b_mn;
      const uint32_t idesc = fp8_idesc(256, kN, a_mn, b_mn), a_step = operand_step(a_mn), b_step = operand_step(b_mn);
      const int total = p.tiles[i], k_blocks = p.pr[i].k_blocks, chunk = p.pr[i].chunk;
      for (int tile = my_first(i); tile < total && ok; tile = my_next(i, tile)) {
        // a tile of 192 columns may start in the middle of 128: two words of 32 columns behind the first atom's start
        const uint32_t sfb = kN == 192 ? 4u + ((uint32_t)(tile % p.pr[i].n_tiles) & 1u) * 2u : 4u;
        for (int k0 = 0; k0 < k_blocks && ok; k0 += chunk, ++it) {
          ok = mbar_wait_cluster(bar_tempty, (uint32_t)(it & 1) ^ 1u, abort_flag, p.status);
          if (!ok) break;
          tc_fence_after();
          const int k1 = min(k_blocks, k0 + chunk);
          for (int ks = k0; ks < k1; ++ks, ++kcount) {
            ok = mbar_wait_cluster(bar_full + 8 * stage, phase, abort_flag, p.status);
            if (!ok) break;
            tc_fence_after();
            if (issuer) {
              const uint32_t sb = smem_base + stage * kPStageBytes, sfcol = tmem + 256 + (kcount & 1u) * 16;
              const uint32_t a_lo = operand_lo(sb, a_mn), b_lo = operand_lo(sb + kLTile, b_mn);
              tc_cp_sf<2>(sfcol, ((uint64_t)kLSfHi << 32) | (((sb + C::kOffSfA) & 0x3FFFFu) >> 4));
              tc_cp_sf<2>(sfcol + 4, ((uint64_t)kLSfHi << 32) | (((sb + C::kOffSfB) & 0x3FFFFu) >> 4));
              tc_cp_sf<2>(sfcol + 8, ((uint64_t)kLSfHi << 32) | (((sb + C::kOffSfB + 512) & 0x3FFFFu) >> 4));
#pragma unroll
              for (int j = 0; j < 4; ++j)
                tc_mma_mxf8<2>(tmem, ((uint64_t)kLSwHi << 32) | (a_lo + a_step * j), ((uint64_t)kLSwHi << 32) | (b_lo + b_step * j),
                               idesc | ((uint32_t)j << 4) | ((uint32_t)j << 29), sfcol, sfcol + sfb, (ks > k0 || j > 0) ? 1u : 0u);
              tc_commit<2>(bar_empty + 8 * stage);
            }
            __syncwarp();
            if (++stage == kPStages) { stage = 0; phase ^= 1u; }
          }
          if (ok && issuer) tc_commit<2>(bar_tfull);
          __syncwarp();
        }
      }
    }
  } else {
    // ------------------------------------------------------------ epilogue: thread = row, 64 columns
    const int q4 = warp & 3, cq = (warp - 2) >> 2;
    const uint32_t lane_addr = tmem + ((uint32_t)(q4 * 32) << 16) + (uint32_t)(cq * 64);
    const uint32_t tempty_addr = map_to_cta(bar_tempty, 0);
    int it = 0;
    bool ok = true;
    for (int i = 0; i < 2 && ok; ++i) {
      const Fp8Problem& q = p.pr[i];
      const int n_tiles = q.n_tiles, total = p.tiles[i], k_blocks = q.k_blocks, chunk = q.chunk;
      for (int tile = my_first(i); tile < total && ok; tile = my_next(i, tile)) {
        const int mt = tile / n_tiles, nt = tile - mt * n_tiles;
        for (int k0 = 0; k0 < k_blocks; k0 += chunk, ++it) {
          ok = mbar_wait(bar_tfull, (uint32_t)(it & 1), abort_flag, p.status);
          if (!ok) break;
          __syncwarp();
          tc_fence_after();
          uint32_t v[64];
          if (cq * 64 < kN) {
            tmem_ld32_bits(lane_addr, v);
            tmem_ld32_bits(lane_addr + 32, v + 32);
            tmem_ld_wait();
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_remote_relaxed(tempty_addr);             // the accumulator is free again
          if (cq * 64 < kN) store_acc(v, q, (int64_t)(mt * 2 + (int)rank) * 128 + q4 * 32, nt * kN + cq * 64, q.add || k0 > 0, lane);
        }
      }
    }
  }
  __syncwarp();                         // the instructions from here on want whole warps, the lanes come out of loops
  tc_fence_before();
  __syncthreads();
  if (warp == 0) settle_if_abandoned(abort_flag);
  cluster_sync_all();                   // the peer may still be signalling this CTA's barriers
  tc_fence_after();
  if (warp == 1) tmem_dealloc<2>(tmem, 512);
}

// ---------------------------------------------------------------------------
// Small products and few rows: tiles of 128 x 128, one CTA each or (where the tiles leave SMs free) a cluster that splits the
// contraction and adds its partial tiles up over distributed shared memory in the order of the ranks.  Warp 0 loads A, warp 10 B; an
// operand older than the preceding kernel (the weights) is loaded without waiting for that one, so the quantization of x hides behind
// the stream of weights.  kRows: rows of A in a stage (128; 64 or 16 where no tile has more: more stages fit; the MMA still reads 128, and
// what it finds behind them gives accumulator rows that nobody reads).
// kQuantize: at most 16 rows, A comes from bf16 x: the warps that store later quantize it into the stages, one stage each at a
// time, and the call is this kernel alone.
// ---------------------------------------------------------------------------
constexpr int kSThreads = 352;
constexpr int kSLoadB = 10;

template <int kRows>
struct SCfg {
  static constexpr int kOffB = kRows * 128;
  static constexpr int kOffSfA = kOffB + kLTile, kOffSfB = kOffSfA + 512;
  static constexpr int kStageBytes = kOffSfB + 512;
  static constexpr int kStages = kRows == 128 ? 6 : kRows == 64 ? 8 : 11;
  static constexpr int kBarOffset = kStages * kStageBytes;
  static constexpr int kSmemBytes = kBarOffset + 256 + 1024;
  static_assert(kStages <= 11 && sizeof(uint64_t) * (2 * 11 + 4) + 8 <= 256, "barriers");
  static_assert(kStageBytes % 1024 == 0, "swizzled tiles");
  static_assert(128 * 4 * (128 + 4 * kSplitMax) <= kBarOffset, "the exchange fits the ring");
  static_assert(kSmemBytes <= 232448, "shared memory");
};

struct __align__(8) SBarriers {
  uint64_t full[11];
  uint64_t empty[11];
  uint64_t tmem_full[2];
  uint64_t tmem_empty[2];
  uint32_t tmem_base;
  int abort_flag;
};

// The (at most sixteen) rows of x's block ks, quantized into a stage: codes in the 128-byte swizzle, scale bytes in the atom.  One warp,
// two rows at a time with 16 lanes each, all loads in flight.
__device__ __forceinline__ void quantize_stage(const Fp8LinearParams& p, int rows, int ks, uint32_t codes, uint32_t atom, int lane) {
  const int c = ks * 128 + (lane & 15) * 8, h = lane >> 4;
  uint4 v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = 2 * i + h;
    v[i] = make_uint4(0u, 0u, 0u, 0u);
    if (r < rows && c < p.K) v[i] = __ldg(reinterpret_cast<const uint4*>(p.x + r * p.ldx + c));
  }
#pragma unroll
  for (int half = 0; half < 8; half += 4) {
    if (2 * half >= rows) break;                                // (the whole warp)
    uint32_t m[2];                                              // four rows side by side, two maxima in a word
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t a = absmax8(v[half + 2 * i]), b = absmax8(v[half + 2 * i + 1]);
      m[i] = max2(__byte_perm(a, b, 0x5410), __byte_perm(a, b, 0x7632));
    }
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) {
#pragma unroll
      for (int i = 0; i < 2; ++i) m[i] = max2(m[i], __shfl_xor_sync(0xFFFFFFFFu, m[i], o));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 2 * (half + i) + h;
      const uint32_t code = fp8_scale_code(__uint_as_float((i & 1) ? m[i >> 1] & 0xFFFF0000u : m[i >> 1] << 16));
      const float sc = fp8_inv_scale(code);
      float f[8];
      unpack8(v[half + i], f);
      const uint32_t lo = f32x4_to_e4m3x4(__fmul_rn(f[0], sc), __fmul_rn(f[1], sc), __fmul_rn(f[2], sc), __fmul_rn(f[3], sc));
      const uint32_t hi = f32x4_to_e4m3x4(__fmul_rn(f[4], sc), __fmul_rn(f[5], sc), __fmul_rn(f[6], sc), __fmul_rn(f[7], sc));
      if (r < rows) {
        const uint32_t at = codes + r * 128 + ((((lane & 15) >> 1) ^ (r & 7)) << 4) + (lane & 1) * 8;
        asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(at), "r"(lo), "r"(hi) : "memory");
        if ((lane & 15) == 0) asm volatile("st.shared.u32 [%0], %1;" ::"r"(atom + r * 16), "r"(code * 0x01010101u) : "memory");
      }
    }
  }
}

template <int kRows, bool kQuantize>
__global__ void __launch_bounds__(kSThreads, 1)
fp8_wave_kernel(const Fp8LinearParams p, const __grid_constant__ Fp8LinearMaps maps) {
  using C = SCfg<kRows>;
  constexpr int kStages = C::kStages;
  extern __shared__ uint8_t smem_dyn[];
  const uint32_t smem_base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
  uint8_t* smem_gen = smem_dyn + (smem_base - smem_u32(smem_dyn));
  SBarriers* bars = reinterpret_cast<SBarriers*>(smem_gen + C::kBarOffset);
  const uint32_t bar_full = smem_u32(&bars->full[0]), bar_empty = smem_u32(&bars->empty[0]);
  const uint32_t bar_tfull = smem_u32(&bars->tmem_full[0]), bar_tempty = smem_u32(&bars->tmem_empty[0]);
  volatile int* abort_flag = &bars->abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // this CTA's problem; CTAs of problem 0 come first
  const int which = (int)blockIdx.x >= p.ctas[0] ? 1 : 0;
  const Fp8Problem& q = p.pr[which];
  const CUtensorMap *tm_a = &maps.a[which], *tm_b = &maps.b[which];
  const int cta = (int)blockIdx.x - (which ? p.ctas[0] : 0);
  const int split = 1 << q.split_log2, part = split > 1 ? (int)cluster_ctarank() : 0;      // (a split has the clusters' size, or is 1)
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) { mbar_init(bar_full + 8 * s, 2); mbar_init(bar_empty + 8 * s, 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(bar_tfull + 8 * b, 1); mbar_init(bar_tempty + 8 * b, 8); }
    bars->abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (!kQuantize) prefetch_tmap(tm_a);
    prefetch_tmap(tm_b);
  }
  if (warp == 1) tmem_alloc<1>(smem_u32(&bars->tmem_base), 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bars->tmem_base;

  const int n_tiles = q.n_tiles, total = p.tiles[which];
  const int first_tile = cta >> q.split_log2, tile_step = p.ctas[which] >> q.split_log2;       // (a split: one tile per cluster)
  const int ks0 = (part * q.k_blocks) >> q.split_log2, ks1 = ((part + 1) * q.k_blocks) >> q.split_log2;      // never empty: split <= k_blocks
  const bool a_mn = q.a_mn, b_mn = q.b_mn;
  // The kernel in front is this call's quantization, which waited for its own predecessor before this one could start.
  const bool early = !kQuantize && q.b_early && (warp == kSLoadB || warp == 1);
  if (!early) pdl_sync();
  else if (warp == 1) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (kQuantize && blockIdx.x == 0 && threadIdx.x == 64) *p.status = 0;       // (the call's only kernel)

  if (warp == kSLoadB || (!kQuantize && warp == 0)) {
    // ------------------------------------------------------------ loaders
    const bool issuer = elect_one(), loads_b = warp == kSLoadB;
    uint32_t stage = 0, phase = 0;
    bool ok = true;
    for (int tile = first_tile; tile < total && ok; tile += tile_step) {
      const int mt = tile / n_tiles, nt = tile - mt * n_tiles;
      const uint8_t* sf = loads_b ? q.b_sf + (size_t)nt * q.b_sf_tile * 512u : q.a_sf + (size_t)mt * q.a_sf_tile * 512u;
      const size_t sf_step = (size_t)(loads_b ? q.b_sf_kb : q.a_sf_kb) * 512u;
      for (int ks = ks0; ks < ks1; ++ks) {
        ok = mbar_wait(bar_empty + 8 * stage, phase ^ 1u, abort_flag, p.status);
        if (!ok) break;
        if (issuer) {
          const uint32_t sb = smem_base + stage * C::kStageBytes, full = bar_full + 8 * stage;
          mbar_expect_tx(full, (uint32_t)(loads_b ? kLTile : kRows * 128) + 512u);
          if (loads_b) load_operand(sb + C::kOffB, tm_b, b_mn, ks, nt * 128, full);
          else load_operand(sb, tm_a, a_mn, ks, mt * 128, full);
          bulk_load(sb + (loads_b ? C::kOffSfB : C::kOffSfA), sf + ks * sf_step, 512u, full);
        }
        __syncwarp();
        if (++stage == kStages) { stage = 0; phase ^= 1u; }
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer
    const bool issuer = elect_one();
    uint32_t stage = 0, phase = 0, kcount = 0;
    int it = 0;
    bool ok = true;
    const uint32_t idesc = fp8_idesc(128, 128, a_mn, b_mn), a_step = operand_step(a_mn), b_step = operand_step(b_mn);
    for (int tile = first_tile; tile < total && ok; tile += tile_step) {
      for (int k0 = ks0; k0 < ks1 && ok; k0 += q.chunk, ++it) {
        const int buf = it & 1, k1 = min(ks1, k0 + q.chunk);
        ok = mbar_wait(bar_tempty + 8 * buf, (uint32_t)((it >> 1) & 1) ^ 1u, abort_flag, p.status);
        if (!ok) break;
        tc_fence_after();
        for (int ks = k0; ks < k1; ++ks, ++kcount) {
          ok = mbar_wait(bar_full + 8 * stage, phase, abort_flag, p.status);
          if (!ok) break;
          tc_fence_after();
          if (issuer) {
            const uint32_t sb = smem_base + stage * C::kStageBytes, sfcol = tmem + 256 + (kcount & 1u) * 8;
            const uint32_t a_lo = operand_lo(sb, a_mn), b_lo = operand_lo(sb + C::kOffB, b_mn);
            tc_cp_sf<1>(sfcol, ((uint64_t)kLSfHi << 32) | (((sb + C::kOffSfA) & 0x3FFFFu) >> 4));
            tc_cp_sf<1>(sfcol + 4, ((uint64_t)kLSfHi << 32) | (((sb + C::kOffSfB) & 0x3FFFFu) >> 4));
#pragma unroll
            for (int j = 0; j < 4; ++j)
              tc_mma_mxf8<1>(tmem + buf * 128, ((uint64_t)kLSwHi << 32) | (a_lo + a_step * j), ((uint64_t)kLSwHi << 32) | (b_lo + b_step * j),
                             idesc | ((uint32_t)j << 4) | ((uint32_t)j << 29), sfcol, sfcol + 4, (ks > k0 || j > 0) ? 1u : 0u);
            tc_commit<1>(bar_empty + 8 * stage);
          }
          __syncwarp();
          if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
        if (ok && issuer) tc_commit<1>(bar_tfull + 8 * buf);
        __syncwarp();
      }
    }
  } else if (warp >= 2 && (kQuantize || split == 1)) {
    // ------------------------------------------------------------ quantization of x, and the epilogue without a split: thread = row, 64 columns
    const int quad = warp & 3, c0 = ((warp - 2) >> 2) * 64;
    int it = 0, tiles = 0;
    bool ok = true;
    for (int tile = first_tile; tile < total && ok; tile += tile_step, ++tiles) {
      const int mt = tile / n_tiles, nt = tile - mt * n_tiles;
      const int64_t row0 = (int64_t)mt * 128 + quad * 32;
      if (kQuantize) {
        // the tile's stages dealt to the eight warps.  (No more warps than stages in the ring: a warp that comes to a stage's next turn but one
        // would take the parity of a turn that has not been for one that is over.)
        static_assert(!kQuantize || 8 <= kStages, "turns told apart by their parity");
        const int n = ks1 - ks0;
        for (int ks = warp - 2; ks < n && ok; ks += 8) {
          const int count = tiles * n + ks, stage = count % kStages;
          ok = mbar_wait(bar_empty + 8 * stage, (uint32_t)((count / kStages) & 1) ^ 1u, abort_flag, p.status);
          if (!ok) break;
          __syncwarp();
          const uint32_t sb = smem_base + stage * C::kStageBytes;
          quantize_stage(p, q.M, ks0 + ks, sb, sb + C::kOffSfA, lane);
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");          // the MMA and the copy to tensor memory read them
          __syncwarp();
          if (lane == 0) mbar_arrive(bar_full + 8 * stage);
        }
        if (!ok || split > 1) break;
      }
      for (int k0 = ks0; k0 < ks1; k0 += q.chunk, ++it) {
        const int buf = it & 1;
        ok = mbar_wait(bar_tfull + 8 * buf, (uint32_t)((it >> 1) & 1), abort_flag, p.status);
        if (!ok) break;
        __syncwarp();
        tc_fence_after();
        uint32_t v[64];
        if (row0 < q.M) {
          tmem_ld32_bits(tmem + buf * 128 + ((uint32_t)(quad * 32) << 16) + c0, v);
          tmem_ld32_bits(tmem + buf * 128 + ((uint32_t)(quad * 32) << 16) + c0 + 32, v + 32);
          tmem_ld_wait();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_tempty + 8 * buf);
        if (row0 < q.M) store_acc(v, q, row0, nt * 128 + c0, q.add || k0 > ks0, lane);
      }
    }
  }
  // ------------------------------------------------------------ the split's partial tiles.  The cluster's barriers are met by every warp,
  // also when a wait was abandoned.
  const bool epi = split > 1 && warp >= 2 && warp < kSLoadB;
  const int mt = first_tile / n_tiles, nt = first_tile - mt * n_tiles;
  const int quad = warp & 3, row = quad * 32 + lane, rows_valid = (int)min((int64_t)128, q.M - (int64_t)mt * 128);
  const int w_log2 = 7 - q.split_log2, w = 1 << w_log2, ld = w + 4;       // columns a CTA owns, their row pitch
  if (epi) {
    mbar_wait(bar_tfull, 0u, abort_flag, p.status);         // all MMAs are done, so every stage of the ring has been read
    tc_fence_after();
  }
  __syncwarp();                                          // the instructions from here on want whole warps, the lanes come out of loops
  if (split > 1) cluster_sync_all();                     // ... in the whole cluster
  if (epi) {
    const int c0 = ((warp - 2) >> 2) * 64;
    if (quad * 32 < rows_valid) {
#pragma unroll
      for (int h = 0; h < 64; h += 32) {
        float v[32];
        __syncwarp();                                    // (some lanes stored the half before)
        tmem_ld32(tmem + ((uint32_t)(quad * 32) << 16) + c0 + h, v);
        tmem_ld_wait();
        if (row < rows_valid) {
          const uint32_t own = smem_base + (uint32_t)((part * 128 + row) * ld) * 4u;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int c = c0 + h + 4 * i;
            st_cluster_f4(map_to_cta(own + (uint32_t)(c & (w - 1)) * 4u, (uint32_t)(c >> w_log2)), v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
          }
        }
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  if (split > 1) cluster_sync_all(); else __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_dealloc<1>(tmem, 512);
  if (warp == 0) settle_if_abandoned(abort_flag);
  if (!epi) return;
  const float* sums = reinterpret_cast<const float*>(smem_gen);
  const int r_log2 = w_log2 - 3, n0 = nt * 128 + part * w;     // a thread takes eight columns of a row
  for (int i = threadIdx.x - 64; i < rows_valid << r_log2; i += 256) {
    const int r = i >> r_log2, c = (i & ((1 << r_log2) - 1)) * 8;
    if (n0 + c >= q.N) continue;
    float4 lo, hi;
    sum_parts(sums + r * ld + c, 128 * ld, split, lo, hi);
    const int64_t at = ((int64_t)mt * 128 + r) * q.N + n0 + c;
    if (q.f32) {
      float4* d = reinterpret_cast<float4*>(static_cast<float*>(q.out) + at);
      if (q.add) {
        const float4 a = d[0], b = d[1];
        lo.x += a.x; lo.y += a.y; lo.z += a.z; lo.w += a.w;
        hi.x += b.x; hi.y += b.y; hi.z += b.z; hi.w += b.w;
      }
      d[0] = lo;
      d[1] = hi;
    } else {
      *reinterpret_cast<uint4*>(static_cast<uint16_t*>(q.out) + at) =
          make_uint4(f32x2_to_bf16x2(lo.x, lo.y), f32x2_to_bf16x2(lo.z, lo.w), f32x2_to_bf16x2(hi.x, hi.y), f32x2_to_bf16x2(hi.z, hi.w));
    }
  }
}

template <int kN>
quads_status launch_pairs(const Fp8LinearParams& p, const Fp8LinearMaps& m, int grid, cudaStream_t st) {
  QUADS_CUDA_OK(set_max_dynamic_smem<fp8_pair_kernel<kN>>(PCfg<kN>::kSmemBytes));
  QUADS_CUDA_OK(launch_kernel(fp8_pair_kernel<kN>, dim3(grid), dim3(kPThreads), (size_t)PCfg<kN>::kSmemBytes, st, p, m));
  return QUADS_OK;
}

template <int kRows, bool kQuantize>
quads_status launch_wave(const Fp8LinearParams& p, const Fp8LinearMaps& m, int cluster_log2, cudaStream_t st) {
  constexpr int smem = SCfg<kRows>::kSmemBytes;
  const int grid = p.ctas[0] + p.ctas[1];
  QUADS_CUDA_OK((set_max_dynamic_smem<fp8_wave_kernel<kRows, kQuantize>>(smem)));
  if (cluster_log2 == 0) QUADS_CUDA_OK(launch_kernel(fp8_wave_kernel<kRows, kQuantize>, dim3(grid), dim3(kSThreads), (size_t)smem, st, p, m));
  else QUADS_CUDA_OK(launch_clusters(fp8_wave_kernel<kRows, kQuantize>, grid, 1 << cluster_log2, kSThreads, (size_t)smem, st, p, m));
  return QUADS_OK;
}

}  // namespace

quads_status launch_fp8_quantize_tiles(const Fp8QuantArgs& a0, const Fp8QuantArgs& a1, int32_t* status, cudaStream_t st) {
  const int64_t t0 = (int64_t)((a0.rows + 127) / 128) * ((a0.cols + 127) / 128), t1 = (int64_t)((a1.rows + 127) / 128) * ((a1.cols + 127) / 128);
  if (t0 + t1 > 0x7FFFFFFF) return QUADS_ERR_SHAPE;
  const int64_t elements = (int64_t)a0.rows * a0.cols + (int64_t)a1.rows * a1.cols;
  const int64_t r0 = a0.codes_r ? (int64_t)((a0.rows + 15) / 16) * ((a0.cols + 127) / 128) : 0;
  if (!a0.codes_c && t1 == 0 && elements <= kQuantRowsElements) {
    QUADS_CUDA_OK(launch_kernel(fp8_quantize_rows_kernel, dim3((unsigned)r0), dim3(256), (size_t)0, st, a0, status));
    return QUADS_OK;
  }
  if (elements <= kQuantSmallElements) {
    const int64_t c0 = a0.codes_c ? (int64_t)((a0.rows + 127) / 128) * ((a0.cols + 63) / 64) : 0;
    const int64_t c1 = (int64_t)((a1.rows + 127) / 128) * ((a1.cols + 63) / 64);
    QUADS_CUDA_OK(launch_kernel(fp8_quantize_small_kernel, dim3((unsigned)(r0 + c0 + c1)), dim3(256), (size_t)0, st, a0, a1, (int)r0, (int)c0, status));
    return QUADS_OK;
  }
  QUADS_CUDA_OK(launch_kernel(fp8_quantize_tiles_kernel, dim3((unsigned)(t0 + t1)), dim3(256), (size_t)0, st, a0, a1, (int)t0, status));
  return QUADS_OK;
}

// Two problems on pairs, in rounds: problem 0, and 1 from where 0 ends, after as many rounds without the x pairs that still have a tile of 0 as
// balances the two.  64 x 4096 -> 4096 (16 tiles of 32 blocks, 256 of one) 24.2 us with five such rounds, 31.7 with one; 64 x 8192 -> 8192
// 71 with seven, 82 with one; 8192 x 768 -> 2048 51 with two, 66 with one, 57 with pairs of their own for each.  Returns the longest pair's cost.
int64_t plan_rounds(const int64_t* tiles, const int64_t* cost, int n_pairs, Fp8LinearParams* p) {
  const int64_t pairs = std::min<int64_t>(n_pairs, tiles[0] + tiles[1]), x = tiles[0] % pairs, m = pairs - x, full = tiles[0] / pairs * cost[0];
  int64_t best = INT64_MAX, both = 0, rounds = 1;
  for (int64_t r = 1; r <= (x ? 16 : 1); ++r) {
    const int64_t rest = std::max<int64_t>(0, tiles[1] - r * m);
    const int64_t late = full + (x ? cost[0] + (rest + pairs - 1) / pairs * cost[1] : 0);
    const int64_t early = full + (rest ? r + rest / pairs + (x < rest % pairs ? 1 : 0) : (tiles[1] + m - 1) / m) * cost[1];
    const int64_t c = std::max(late, early);
    if (c < best || (c == best && late + early < both)) { best = c; both = late + early; rounds = r; }
  }
  p->first[1] = (int)x;
  p->early_tiles = (int)((rounds - 1) * m);
  p->early_step = (int)m;
  return best;
}

// The launch of one product, or of the two of a backward call together.
quads_status plan_fp8_linear(Fp8LinearParams* p, int n_problems, bool bf16_x, int n_sms, Fp8LinearPlan* plan) {
  int64_t t128[2] = {0, 0}, t256[2] = {0, 0};
  for (int i = 0; i < n_problems; ++i) {
    const Fp8Problem& q = p->pr[i];
    t128[i] = (int64_t)((q.M + 127) / 128) * ((q.N + 127) / 128);
    t256[i] = (int64_t)((q.M + 255) / 256) * ((q.N + 255) / 256);
  }
  if (t128[0] + t128[1] > 0x3FFFFFFF) return QUADS_ERR_SHAPE;
  *plan = Fp8LinearPlan{};
  plan->a_rows = n_problems == 1 && !p->pr[0].a_mn && p->pr[0].M <= 64 ? 64 : 128;
  plan->quantize = bf16_x && p->pr[0].M <= 16;
  // A float32 result leaves the tensor core every 4096 steps of the contraction and is added up in float32: that adds to the accumulator
  // by cutting off, so its error grows with the steps (2-norm, relative, normal values: 6.0e-8 at 1024, 2.2e-7 at 4096 and, in one piece, 4.8e-7 at 8192
  // and 1.16e-6 at 16384; where the tokens' gradients spread by factors of e some 2.4 times that).
  for (int i = 0; i < n_problems; ++i) p->pr[i].chunk = p->pr[i].f32 ? kChunkBlocks : p->pr[i].k_blocks;
  auto may_split = [&](int i, int lg) { return 1 << lg <= p->pr[i].k_blocks && (p->pr[i].k_blocks + (1 << lg) - 1) >> lg <= p->pr[i].chunk; };
  auto us = [&](int i, int l) {                              // (tiles of 128 x 128, one to a CTA)
    return ((p->pr[i].k_blocks + (1 << l) - 1) >> l) * 0.2 + 4.0 + (l ? std::min(p->pr[i].M, 128) / 128.0 * 1.25 * (1 + l) + 0.05 * l : 0.0);
  };
  auto us_turns = [&](int i, double rounds) { return 4.0 + rounds * std::max(0.3 * p->pr[i].k_blocks, p->pr[i].f32 ? 1.5 : 0.8); };
  // (a tile of a pair, in blocks of the contraction, 0.3 us: its own, or what its store takes, which the next tile's MMAs don't hide,
  // and the accumulator's way out of the tensor core)
  auto pair_cost = [&](int i) { return p->pr[i].f32 ? 6 + std::max(p->pr[i].k_blocks, 3) : 3 + std::max(p->pr[i].k_blocks, 7); };
  plan->tile_n = 256;
  int lg[2] = {0, 0};
  bool in_turn = n_problems == 1;                            // the last problem's tiles in turn on the CTAs that there is room for
  if (n_problems == 1) {
    lg[0] = plan_split(t128[0], std::min(p->pr[0].M, 128), p->pr[0].k_blocks, 0.2, 1.25, 1.3, n_sms);
    if (lg[0] > 0 && !may_split(0, lg[0])) lg[0] = 0;
    if (lg[0] < 0 && p->pr[0].M > 128) {
      // More tiles than SMs: pairs, with tiles of 192 columns where their rounds end sooner (a forward product's only: columns of a weight that
      // lies by rows, 96 to a CTA; a block takes them 0.8 of the time), or single CTAs in turn.  Columns of 256 and 192, us: 1024 x 4096 -> 4096
      // 21.0 and 25.2, 8192 x 4096 -> 4096 116.2 and 121.9, 768 x 4096 -> 4096 20.0 and 17.1, 1280 x 4096 -> 4096 31.5 and 26.5.  The better pairs and single
      // CTAs: 1501 x 2000 -> 4176 22.1 and 28.3, 640 x 1024 -> 4096 9.2 and 10.2, 2048 x 512 -> 2048 9.6 and 8.5, 4096 x 256 -> 4096 15.0 and 13.2; the
      // weight's gradient of 64 x 4096 -> 4096 20.7 and 17.0, of 2048 x 2048 -> 2048 21.0 and 21.7.
      const Fp8Problem& q = p->pr[0];
      const int64_t t192 = (int64_t)((q.M + 255) / 256) * ((q.N + 191) / 192), pairs = n_sms / 2;
      double rounds = (double)((t256[0] + pairs - 1) / pairs) * pair_cost(0);
      const double r192 = (double)((t192 + pairs - 1) / pairs) * (3 + std::max(0.8 * q.k_blocks, 7.0));
      if (!q.a_mn && !q.b_mn && !q.f32 && r192 < rounds) { plan->tile_n = 192; t256[0] = t192; rounds = r192; }
      plan->pairs = 5.0 + 0.3 * rounds <= us_turns(0, (double)((t128[0] + n_sms - 1) / n_sms));
    }
    plan->cluster_log2 = std::max(0, lg[0]);
  } else {
    // The product with the longer contraction comes first and is split as far as that ends sooner, the other one's tiles take the SMs that
    // this leaves (or are split alike, where there is room for all): beside no clusters in turn, else a CTA each.  In us: what a stage, a
    // kernel's start and end, the exchange and a tile's store take; of clusters of four and eight the chip holds fewer CTAs.  192 x 256 -> 8192
    // (4 tiles of 64 blocks, 128 of two) 22.4 with no split, 17.7, 15.5 and 15.7 with 2, 4 and 8; 64 x 1024 -> 4096 (8 of 32, 256 of one) 14.0,
    // 11.8, 14.8, 17.3; 192 x 2048 -> 2048 (32 of 16, 256 of two) 11.8, a CTA for each tile 14.8, clusters of two 15.6.
    double best = 1e30;
    for (int l = 0; l <= 3 && (l == 0 || may_split(0, l)); ++l) {
      const int64_t room = l < 2 ? n_sms : l == 2 ? 128 : 120, left = room - (t128[0] << l);
      if (l > 0 && left <= 0) break;
      const bool turns = l == 0 && left >= n_sms / 4;
      const double rounds = (double)(left > 0 && (l > 0 || turns) ? (t128[1] + left - 1) / left : (t128[0] + t128[1] + room - 1) / room);
      const double alone = std::max(us(0, l), turns ? us_turns(1, rounds) : rounds * us(1, 0));
      const double alike = l > 0 && may_split(1, l) && (t128[0] + t128[1]) << l <= room ? std::max(us(0, l), us(1, l)) : 1e30;
      if (std::min(alone, alike) < best) {
        best = std::min(alone, alike);
        plan->cluster_log2 = lg[0] = l;
        lg[1] = alike < alone ? l : 0;
        in_turn = turns;
      }
    }
    if (t128[0] + t128[1] > 2 * n_sms) {
      // Pairs, a block takes one 0.3 us.  As above and on pairs: 333 x 2048 -> 2048 12.9 and 15.9, 100 x 768 -> 8192 17.7 and 27.9, 64 x 4096 -> 4096
      // 20.7 and 24.0; 512 x 4096 -> 1024 19.4 and 17.2, 2048 x 2048 -> 2048 37.7 and 27.9, 1 x 8192 -> 8192 83.9 and 71.9.  (One product after the other:
      // 21.3, 24.3, 30.6; 19.6, 32.6, 71.1.)
      const int64_t cost[2] = {pair_cost(0), pair_cost(1)};
      plan->pairs = 5.0 + 0.3 * plan_rounds(t256, cost, n_sms / 2, p) < best;
    }
  }
  for (int i = 0; i < n_problems; ++i) {
    Fp8Problem& q = p->pr[i];
    q.n_tiles = plan->pairs ? (q.N + plan->tile_n - 1) / plan->tile_n : (q.N + 127) / 128;
    p->tiles[i] = (int)(plan->pairs ? t256[i] : t128[i]);
    q.split_log2 = !plan->pairs && lg[i] == plan->cluster_log2 && lg[i] > 0 ? lg[i] : 0;
    if (plan->pairs) continue;
    p->ctas[i] = q.split_log2 ? p->tiles[i] << q.split_log2 : p->tiles[i];
    if (in_turn && i == n_problems - 1 && !q.split_log2) p->ctas[i] = std::min(p->tiles[i], n_sms - (i ? p->ctas[0] : 0));
    const int c = 1 << plan->cluster_log2;
    p->ctas[i] = (p->ctas[i] + c - 1) / c * c;             // (whole clusters of one problem)
  }
  if (plan->pairs) {
    const int64_t pairs = std::min<int64_t>(n_sms / 2, (int64_t)p->tiles[0] + p->tiles[1]);
    p->ctas[0] = (int)(2 * pairs);
    p->ctas[1] = n_problems == 2 ? (int)(2 * pairs) : 0;
    plan->grid = (int)(2 * pairs);
  }
  return QUADS_OK;
}

quads_status launch_fp8_linear(const Fp8LinearParams& p, const Fp8LinearMaps& m, const Fp8LinearPlan& plan, cudaStream_t st) {
  if (plan.pairs) {
    return plan.tile_n == 256 ? launch_pairs<256>(p, m, plan.grid, st) : launch_pairs<192>(p, m, plan.grid, st);
  }
  if (plan.quantize) return launch_wave<16, true>(p, m, plan.cluster_log2, st);
  if (plan.a_rows == 64) return launch_wave<64, false>(p, m, plan.cluster_log2, st);
  return launch_wave<128, false>(p, m, plan.cluster_log2, st);
}

}  // namespace quads
