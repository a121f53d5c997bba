// wdp_product.hip — matrix product of 8-bit operands with a scale for each block of 128 (include/wdp.h: wdp_product).
//
// c[i][j] = sum over blocks b of a_scale[i][b] b_scale[.][b] (a block's inner product): one matrix instruction
// 16 x 16 x 128 makes the inner products of a block, and one multiply-add an element adds them to the accumulators with
// the scales' product.  The instruction is fed b as its first operand and a as its second, so that a lane holds ONE row
// of a (one a_scale, and the block's scale product, per lane) and four adjacent columns of c (one store).
//
// The order of k inside a block is the same for both operands and otherwise free: a lane takes the 16-byte chunks
// g and g + 4 of its row (g = lane / 16).  In LDS a row is eight chunks; chunk c of row r lies at place c ^ (r / 2 % 8),
// which spreads the sixteen rows that a quarter of a wave reads over all banks.
#include "wdp_common.h"

namespace wdp {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

struct ProductArgs {
  const uint8_t *a, *b;
  const float *a_scale, *b_scale;
  void* c;
  int64_t a_stride, b_stride, c_stride, as_row, as_block, bs_row, bs_block;
  int32_t m, n, k, blocks;  // blocks of 128 along k
  int32_t m_tiles, n_tiles;
};


template <int FA, int FB> __device__ __forceinline__ f32x4 inner(i32x8 b, i32x8 a) {
  const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, zero, FB, FA, 0, 0, 0, 0);
}

__device__ __forceinline__ int place(int row, int chunk) { return row * 8 + (chunk ^ ((row >> 1) & 7)); }

// Chunk `chunk` (16 bytes) of a row's block; bytes from `left` on do not exist and read as zero.
__device__ __forceinline__ i32x4 load_chunk(const uint8_t* row, int64_t at, int left) {
  i32x4 v = {0, 0, 0, 0};
  if (left >= 16) {
    struct __attribute__((packed, aligned(1))) Raw {
      i32x4 v;
    };
    return reinterpret_cast<const Raw*>(row + at)->v;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (i < left) v[i >> 2] |= int(uint32_t(row[at + i]) << (8 * (i & 3)));
  return v;
}

template <typename C> __device__ __forceinline__ void store_c(const ProductArgs& p, int row, int col, f32x4 v) {
  C* c = static_cast<C*>(p.c) + int64_t(row) * p.c_stride + col;
  const float f[4] = {v[0], v[1], v[2], v[3]};
  store_some<C, 4>(c, p.n - col, f);
}

// A workgroup's tile of BM rows x BN columns, four waves of which each owns a part; the next block's chunks are
// requested into registers before this block is multiplied, and go to the other half of LDS behind it.
template <int FA, int FB, bool ROWS, typename C, int BM, int BN, int WAVES_M>
__global__ __launch_bounds__(256) void product_tile_kernel(ProductArgs p) {
  constexpr int WAVES_N = 4 / WAVES_M, TM = BM / WAVES_M / 16, TN = BN / WAVES_N / 16;
  constexpr int kA = BM * 8 / 256 ? BM * 8 / 256 : 1, kB = BN * 8 / 256;  // chunks a thread brings
  __shared__ i32x4 lds_a[2][BM * 8], lds_b[2][BN * 8];
  __shared__ __attribute__((aligned(16))) float scale_a[2][BM], scale_b[2][BN];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int64_t tile = blockIdx.x;
  const int m0 = int(tile / p.n_tiles) * BM, n0 = int(tile % p.n_tiles) * BN;
  const int wm = (wave % WAVES_M) * TM * 16, wn = (wave / WAVES_M) * TN * 16;
  const int r16 = lane & 15, g = lane >> 4;

  i32x4 next_a[kA], next_b[kB];
  float next_sa = 0.0f, next_sb = 0.0f;
  auto request = [&](int block) {
    const int k0 = block * WDP_BLOCK;
#pragma unroll
    for (int i = 0; i < kA; ++i) {
      const int e = t + 256 * i, row = e >> 3, chunk = e & 7;
      next_a[i] = i32x4{0, 0, 0, 0};
      if (e < BM * 8 && m0 + row < p.m) next_a[i] = load_chunk(p.a + int64_t(m0 + row) * p.a_stride, k0 + chunk * 16, p.k - k0 - chunk * 16);
    }
#pragma unroll
    for (int i = 0; i < kB; ++i) {
      const int e = t + 256 * i, row = e >> 3, chunk = e & 7;
      next_b[i] = i32x4{0, 0, 0, 0};
      if (n0 + row < p.n) next_b[i] = load_chunk(p.b + int64_t(n0 + row) * p.b_stride, k0 + chunk * 16, p.k - k0 - chunk * 16);
    }
    if (t < BM) next_sa = m0 + t < p.m ? p.a_scale[int64_t(m0 + t) * p.as_row + block * p.as_block] : 0.0f;
    if (t < BN) next_sb = n0 + t < p.n ? p.b_scale[int64_t(ROWS ? n0 + t : (n0 + t) / WDP_BLOCK) * p.bs_row + block * p.bs_block] : 0.0f;
  };
  auto stage = [&](int half) {
#pragma unroll
    for (int i = 0; i < kA; ++i) {
      const int e = t + 256 * i;
      if (e < BM * 8) lds_a[half][place(e >> 3, e & 7)] = next_a[i];
    }
#pragma unroll
    for (int i = 0; i < kB; ++i) {
      const int e = t + 256 * i;
      lds_b[half][place(e >> 3, e & 7)] = next_b[i];
    }
    if (t < BM) scale_a[half][t] = next_sa;
    if (t < BN) scale_b[half][t] = next_sb;
  };

  f32x4 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  request(0);
  stage(0);
  __syncthreads();
  for (int block = 0; block < p.blocks; ++block) {
    const int half = block & 1;
    const bool more = block + 1 < p.blocks;
    if (more) request(block + 1);
    i32x8 fa[TM];
    float sa[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int row = wm + i * 16 + r16;
      const i32x4 lo = lds_a[half][place(row, g)], hi = lds_a[half][place(row, g + 4)];
      fa[i] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      sa[i] = scale_a[half][row];
    }
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int row = wn + j * 16 + r16;
      const i32x4 lo = lds_b[half][place(row, g)], hi = lds_b[half][place(row, g + 4)];
      const i32x8 fb = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      const f32x4 sb = *reinterpret_cast<const f32x4*>(&scale_b[half][wn + j * 16 + g * 4]);
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const f32x4 part = inner<FA, FB>(fb, fa[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(part[e], sa[i] * sb[e], acc[i][j][e]);
      }
    }
    if (more) stage(half ^ 1);
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int row = m0 + wm + i * 16 + r16;
    if (row >= p.m) continue;
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int col = n0 + wn + j * 16 + g * 4;
      if (col < p.n) store_c<C>(p, row, col, acc[i][j]);
    }
  }
}

// (a launch takes up to 2^22 tiles: all sizes of a grid, and rows counted in 32 bits, stay far from their limits)
template <int FA, int FB, bool ROWS, typename C> void launch(ProductArgs p, hipStream_t stream) {
  const int64_t rows = p.m;
  p.n_tiles = (p.n + 127) / 128;
  const int64_t most = (int64_t(1) << 22) / p.n_tiles * 128;
  for (int64_t at = 0; at < rows; at += most) {
    ProductArgs q = p;
    q.a += at * p.a_stride;
    q.a_scale += at * p.as_row;
    q.c = static_cast<C*>(p.c) + at * p.c_stride;
    q.m = int32_t(rows - at < most ? rows - at : most);
    q.m_tiles = (q.m + 127) / 128;
    product_tile_kernel<FA, FB, ROWS, C, 128, 128, 2><<<dim3(unsigned(int64_t(q.m_tiles) * q.n_tiles)), dim3(256), 0, stream>>>(q);
  }
}
template <int FA, int FB, bool ROWS> void launch_c(const ProductArgs& p, int c_type, hipStream_t stream) {
  if (c_type == WDP_F32) launch<FA, FB, ROWS, float>(p, stream);
  else if (c_type == WDP_BF16) launch<FA, FB, ROWS, bf16>(p, stream);
  else launch<FA, FB, ROWS, f16>(p, stream);
}
template <int FA, int FB> void launch_rows(const ProductArgs& p, bool rows, int c_type, hipStream_t stream) {
  if (rows) launch_c<FA, FB, true>(p, c_type, stream);
  else launch_c<FA, FB, false>(p, c_type, stream);
}

int check(const wdp_product_config& c) {
  if (c.struct_size != sizeof(wdp_product_config)) return WD_E_CONFIG;
  if (!is_8bit(c.a_type) || !is_8bit(c.b_type) || !is_float_type(c.c_type) || (c.b_scale_rows != 1 && c.b_scale_rows != WDP_BLOCK)) return WD_E_CONFIG;
  if (c.m < 0 || c.m > 0x7FFFFFFF || c.n < 0 || c.n > (1 << 24) || c.k < 1 || c.k > (1 << 24)) return WD_E_CONFIG;
  const int64_t most = int64_t(1) << 40;
  if (c.m > 1 && (c.a_stride < c.k || c.a_stride > most || c.c_stride < c.n || c.c_stride > most)) return WD_E_CONFIG;
  if (c.n > 1 && (c.b_stride < c.k || c.b_stride > most)) return WD_E_CONFIG;
  if (c.a_scale_row_stride < 0 || c.a_scale_block_stride < 0 || c.b_scale_row_stride < 0 || c.b_scale_block_stride < 0) return WD_E_CONFIG;
  return WD_OK;
}

}  // namespace
}  // namespace wdp

extern "C" {

int wdp_product_workspace(const wdp_product_config* cfg, size_t* bytes) {
  if (!cfg || !bytes) return WD_E_NULL;
  const int rc = wdp::check(*cfg);
  if (rc != WD_OK) return rc;
  *bytes = 0;
  return WD_OK;
}

int wdp_product(const wdp_product_config* cfg, const wdp_product_buffers* b) {
  using namespace wdp;
  if (!cfg || !b) return WD_E_NULL;
  const int rc = check(*cfg);
  if (rc != WD_OK) return rc;
  if (cfg->m == 0 || cfg->n == 0) return WD_OK;
  if (!b->a || !b->a_scale || !b->b || !b->b_scale || !b->c) return WD_E_NULL;
  if (!aligned(b->a_scale, 4) || !aligned(b->b_scale, 4) || !aligned(b->c, size_of(cfg->c_type)) || !aligned(b->workspace, 256)) return WD_E_ALIGN;
  const ProductArgs p = {static_cast<const uint8_t*>(b->a), static_cast<const uint8_t*>(b->b), b->a_scale, b->b_scale, b->c, cfg->a_stride, cfg->b_stride,
                         cfg->c_stride, cfg->a_scale_row_stride, cfg->a_scale_block_stride, cfg->b_scale_row_stride, cfg->b_scale_block_stride,
                         int32_t(cfg->m), cfg->n, cfg->k, (cfg->k + WDP_BLOCK - 1) / WDP_BLOCK, 0, 0};
  const hipStream_t stream = static_cast<hipStream_t>(cfg->stream);
  const bool rows = cfg->b_scale_rows == 1;
  if (cfg->a_type == WDP_E4M3 && cfg->b_type == WDP_E4M3) launch_rows<0, 0>(p, rows, cfg->c_type, stream);
  else if (cfg->a_type == WDP_E4M3) launch_rows<0, 1>(p, rows, cfg->c_type, stream);
  else if (cfg->b_type == WDP_E4M3) launch_rows<1, 0>(p, rows, cfg->c_type, stream);
  else launch_rows<1, 1>(p, rows, cfg->c_type, stream);
  return launched();
}

}  // extern "C"
