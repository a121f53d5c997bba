// wdp_norm.hip — RMS norm with the residual's addition and an 8-bit output with scales, and its gradients
// (include/wdp.h: wdp_norm, wdp_norm_backward).
//
// Both directions move each element once and compute a handful of operations on it: memory bounds them, latency where
// there are few rows.  A row is held in registers by THREADS_PER_ROW lanes, eight adjacent elements a lane and chunk
// (one 16-byte access of bfloat16), so that its mean square (or the gradient's inner product) is known before anything
// is written and nothing is read twice.  Eight elements a lane make sixteen lanes a block of 128, whose maximum is
// found by four exchanges within a row of sixteen lanes.
#include "wdp_common.h"

namespace wdp {
namespace {

constexpr int kVec = 8;          // elements of a lane's chunk
constexpr int kMaxWidth = 32768; // 1024 threads x 4 chunks x 8

struct NormArgs {
  const void *x, *residual, *weight;
  void *h, *y;
  uint8_t* q;
  float *scale, *rstd;
  int64_t rows, x_stride, residual_stride, h_stride, y_stride, q_stride, scale_row, scale_block;
  int32_t width, q_type;
  int32_t run;  // rows that a workgroup takes one after the other: a power of two
  float eps, inv_width;
};

struct GradArgs {
  const void *dy, *dh, *h, *weight;
  const float* rstd;
  void* dx;
  float* partial;  // [gridDim.x][width], or NULL
  int64_t rows, dy_stride, dh_stride, h_stride, dx_stride;
  int32_t width;
  float inv_width;
};

// Sum over the lanes of a row.  Rows of up to 64 lanes stay within a wave; wider ones are a workgroup each and join
// their waves' sums in LDS.  Two sets of places in turn: one barrier a row keeps the next row's sums from
// overtaking readers of this one's.
template <int TPR> __device__ __forceinline__ float row_sum(float v, float (*places)[16], int turn) {
  if (TPR <= 64) return group_sum<TPR>(v);
  v = group_sum<64>(v);
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) places[turn][wave] = v;
  __syncthreads();
  float total = 0.0f;
#pragma unroll
  for (int i = 0; i < TPR / 64; ++i) total += places[turn][i];
  return total;
}

// Where a lane's chunk lies.  The chunk that the row ends in is moved back to end with it (rows of eight elements and
// more): one access like the others, its first `skip` elements are its neighbour's.  (Elements one by one would cost every
// wave of an odd width a second pass of loads: 33333 x 999 bfloat16 took 97 us forward and 172 backward that way.)
struct Span {
  int start, skip, count;  // count: elements that exist; 0: none
};
template <int TPR> __device__ __forceinline__ Span span_of(int width, int c) {
  const int col = (c * TPR + int(threadIdx.x % TPR)) * kVec, left = width - col;
  if (left >= kVec) return {col, 0, kVec};
  if (left <= 0) return {0, kVec, 0};
  return width >= kVec ? Span{width - kVec, kVec - left, kVec} : Span{0, 0, left};
}
// A chunk as it lies in memory: requested one row ahead of its use, where the registers hold a row more (1024 threads have
// 128 each).
template <int TPR, int C> constexpr bool kAhead = TPR < 1024 || C == 1;
template <typename T> struct Words {
  u32x4 w[sizeof(T) / 2];
};
template <typename T> __device__ __forceinline__ Words<T> request(const T* row, const Span& s) {
  Words<T> r;
  if (s.count == kVec) {
#pragma unroll
    for (int i = 0; i < int(sizeof(T) / 2); ++i) r.w[i] = load_raw<u32x4>(row + s.start + i * (16 / sizeof(T)));
  } else {  // (a row of fewer than eight elements)
    float v[kVec];
    load_some<T, kVec>(row + s.start, s.count, v);
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      if constexpr (sizeof(T) == 4) r.w[i / 4][i % 4] = __float_as_uint(v[i]);
      else if (i % 2 == 0) r.w[0][i / 2] = narrow<T>(v[i], v[i + 1]);
    }
  }
  return r;
}
template <typename T> __device__ __forceinline__ void values(const Words<T>& r, float v[kVec]) {
#pragma unroll
  for (int i = 0; i < kVec; i += sizeof(T) == 4 ? 1 : 2) {
    if constexpr (sizeof(T) == 4) v[i] = __uint_as_float(r.w[i / 4][i % 4]);
    else widen<T>(r.w[0][i / 2], v + i);
  }
}
template <typename W> __device__ __forceinline__ void load_weight(const void* weight, const Span& s, float w[kVec]) {
  if (weight) {
    load_some<W, kVec>(static_cast<const W*>(weight) + s.start, s.count, w);
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i) w[i] = 1.0f;
  }
}

template <typename T, typename W, int TPR, int C>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void norm_kernel(NormArgs a) {
  constexpr int kThreads = TPR > 256 ? TPR : 256, kRows = kThreads / TPR;
  __shared__ float places[2][16];
  const int lane = threadIdx.x % TPR;
  int turn = 0;
  float w[C][kVec];
  Span at[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    at[c] = span_of<TPR>(a.width, c);
    if (C <= 2 && at[c].count) load_weight<W>(a.weight, at[c], w[c]);
  }
  // A workgroup takes runs of 32 neighbouring rows (a whole line of scales and of rstd, four bytes a row) in turn with the
  // others, which together go through memory from front to back: runs of a thousand rows each took 509 us for
  // 2000000 x 256 without residual, single rounds of eight 940 with residual and scales, where runs of 32 take 428 and 767.
  const int run = a.run;
  const auto following = [&](int64_t row) {
    const int64_t next = row + kRows;
    return run == kRows || next % run < kRows ? next + int64_t(gridDim.x - 1) * run : next;
  };
  const T *x = static_cast<const T*>(a.x), *residual = static_cast<const T*>(a.residual);
  Words<T> next_x[C], next_r[C];
  const auto ahead = [&](int64_t row) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (!at[c].count) continue;
      next_x[c] = request(x + row * a.x_stride, at[c]);
      if (residual) next_r[c] = request(residual + row * a.residual_stride, at[c]);
    }
  };
  int64_t row = int64_t(blockIdx.x) * run + threadIdx.x / TPR;
  if (kAhead<TPR, C> && row < a.rows) ahead(row);
  for (int64_t next; row < a.rows; row = next) {
    next = following(row);
    if (!kAhead<TPR, C>) ahead(row);
    float v[C][kVec];
    float square = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) v[c][i] = 0.0f;
      if (!at[c].count) continue;
      values(next_x[c], v[c]);
      if (residual) {
        float r[kVec];
        values(next_r[c], r);
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[c][i] = to_float<T>(from_float<T>(v[c][i] + r[i]));  // the norm is that of h as it is stored
      }
#pragma unroll
      for (int i = 0; i < kVec; ++i) square = fmaf(i < at[c].skip ? 0.0f : v[c][i], v[c][i], square);
    }
    if (kAhead<TPR, C> && next < a.rows) ahead(next);
    const float rstd = 1.0f / sqrtf(row_sum<TPR>(square, places, turn) * a.inv_width + a.eps);
    turn ^= 1;
    if (a.rstd && lane == 0) a.rstd[row] = rstd;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      // (what a moved chunk writes of its neighbour's elements is what the neighbour writes)
      if (at[c].count && a.h) store_some<T, kVec>(static_cast<T*>(a.h) + row * a.h_stride + at[c].start, at[c].count, v[c]);
      if (C > 2 && at[c].count) load_weight<W>(a.weight, at[c], w[c]);
      float y[kVec];
      float most = 0.0f;
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        y[i] = i < at[c].count ? v[c][i] * rstd * w[c][i] : 0.0f;
        most = fmaxf(most, i < at[c].skip ? 0.0f : fabsf(y[i]));
      }
      if (at[c].count && a.y) store_some<T, kVec>(static_cast<T*>(a.y) + row * a.y_stride + at[c].start, at[c].count, y);
      if (a.q) {
        most = fmaxf(group_max<(TPR < 16 ? TPR : 16)>(most), kTiny);
        const float largest = a.q_type == WDP_E4M3 ? kLargestE4M3 : kLargestE5M2;
        const float scale = most / largest, inv = 1.0f / scale;
        if (at[c].count) {
          const uint32_t lo = to_codes(a.q_type, y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
          const uint32_t hi = to_codes(a.q_type, y[4] * inv, y[5] * inv, y[6] * inv, y[7] * inv);
          uint8_t* q = a.q + row * a.q_stride + at[c].start;
          if (at[c].count == kVec && at[c].skip == 0) {
            store_raw(q, u32x2{lo, hi});
          } else {  // the row's end: up to seven codes, in fours, twos and ones (the neighbour's block has another scale)
            uint64_t codes = (uint64_t(hi) << 32 | lo) >> (8 * at[c].skip);
            q += at[c].skip;
            const int n = at[c].count - at[c].skip;
            if (n & 4) store_raw(q, uint32_t(codes)), codes >>= 32, q += 4;
            if (n & 2) store_raw(q, uint16_t(codes)), codes >>= 16, q += 2;
            if (n & 1) *q = uint8_t(codes);
          }
          const int col = at[c].start + at[c].skip;
          if (col % WDP_BLOCK == 0) a.scale[row * a.scale_row + (col / WDP_BLOCK) * a.scale_block] = scale;
        }
      }
    }
  }
}

template <typename T, typename W, int TPR, int C>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void norm_grad_kernel(GradArgs a) {
  constexpr int kThreads = TPR > 256 ? TPR : 256, kRows = kThreads / TPR;
  __shared__ float places[2][16];
  int turn = 0;
  float w[C][kVec], dw[C][kVec];
  Span at[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    at[c] = span_of<TPR>(a.width, c);
#pragma unroll
    for (int i = 0; i < kVec; ++i) w[c][i] = dw[c][i] = 0.0f;
    if (at[c].count) load_weight<W>(a.weight, at[c], w[c]);
  }
  const T *from_dy = static_cast<const T*>(a.dy), *from_h = static_cast<const T*>(a.h), *from_dh = static_cast<const T*>(a.dh);
  Words<T> next_dy[C], next_h[C], next_dh[C];
  float next_rstd = 0.0f;
  const auto ahead = [&](int64_t row) {
    next_rstd = a.rstd[row];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (!at[c].count) continue;
      next_dy[c] = request(from_dy + row * a.dy_stride, at[c]);
      next_h[c] = request(from_h + row * a.h_stride, at[c]);
      if (kAhead<TPR, C> && from_dh) next_dh[c] = request(from_dh + row * a.dh_stride, at[c]);
    }
  };
  const int64_t step = int64_t(gridDim.x) * kRows;
  int64_t row = int64_t(blockIdx.x) * kRows + threadIdx.x / TPR;
  if (kAhead<TPR, C> && row < a.rows) ahead(row);
  for (; row < a.rows; row += step) {
    if (!kAhead<TPR, C>) ahead(row);
    float dy[C][kVec], xhat[C][kVec];
    Words<T> dh[C];
    float dot = 0.0f;
    const float rstd = next_rstd;
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) dy[c][i] = xhat[c][i] = 0.0f;
      if (!at[c].count) continue;
      values(next_dy[c], dy[c]);
      values(next_h[c], xhat[c]);
      if (kAhead<TPR, C> && from_dh) dh[c] = next_dh[c];
    }
    if (kAhead<TPR, C> && row + step < a.rows) ahead(row + step);
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        xhat[c][i] *= rstd;
        const float g = i < at[c].skip ? 0.0f : dy[c][i];
        dw[c][i] = fmaf(g, xhat[c][i], dw[c][i]);
        dot = fmaf(g * w[c][i], xhat[c][i], dot);
        dy[c][i] *= w[c][i];
      }
    }
    if (!a.dx) continue;
    const float mean = row_sum<TPR>(dot, places, turn) * a.inv_width;
    turn ^= 1;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (!at[c].count) continue;
      float dx[kVec], more[kVec];
#pragma unroll
      for (int i = 0; i < kVec; ++i) more[i] = 0.0f;
      if (from_dh) {
        if (!kAhead<TPR, C>) dh[c] = request(from_dh + row * a.dh_stride, at[c]);
        values(dh[c], more);
      }
#pragma unroll
      for (int i = 0; i < kVec; ++i) dx[i] = rstd * (dy[c][i] - xhat[c][i] * mean) + more[i];
      store_some<T, kVec>(static_cast<T*>(a.dx) + row * a.dx_stride + at[c].start, at[c].count, dx);
    }
  }
  if (!a.partial) return;
  // the workgroup's rows joined in LDS, chunk by chunk, in the order of its groups of lanes
  __shared__ float joined[kRows > 1 ? kThreads * kVec : 1];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if (kRows > 1) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kVec; ++i) joined[threadIdx.x * kVec + i] = dw[c][i];
      __syncthreads();
      if (threadIdx.x < TPR) {
        for (int g = 1; g < kRows; ++g)
#pragma unroll
          for (int i = 0; i < kVec; ++i) dw[c][i] += joined[(g * TPR + threadIdx.x) * kVec + i];
      }
    }
    if (threadIdx.x < TPR && at[c].count) {
#pragma unroll
      for (int i = 0; i < kVec; ++i)
        if (i >= at[c].skip && i < at[c].count) a.partial[int64_t(blockIdx.x) * a.width + at[c].start + i] = dw[c][i];
    }
  }
}

// dw from the workgroups' sums: 16 columns a workgroup, 64 threads a column, in a fixed order.
__global__ __launch_bounds__(1024) void norm_grad_join_kernel(const float* __restrict__ partial, int parts, int width, float* __restrict__ dw) {
  __shared__ float sums[64][17];
  const int x = threadIdx.x & 15, y = threadIdx.x >> 4, col = blockIdx.x * 16 + x;
  float sum = 0.0f;
  if (col < width) {
#pragma unroll 4
    for (int p = y; p < parts; p += 64) sum += partial[int64_t(p) * width + col];
  }
  sums[y][x] = sum;
  __syncthreads();
  if (y < 8) {
    sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += sums[y * 8 + i][x];
    sums[y * 8][x] = sum;
  }
  __syncthreads();
  if (y == 0 && col < width) {
    sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += sums[i * 8][x];
    dw[col] = sum;
  }
}

int rows_a_block(int width) { return width <= 32 ? 64 : width <= 64 ? 32 : width <= 128 ? 16 : width <= 256 ? 8 : width <= 1024 ? 4 : 1; }

int64_t grad_blocks(const wdp_norm_config& c) {
  const int64_t per = rows_a_block(c.width), all = (c.rows + per - 1) / per, most = c.width > 4096 ? 256 : 1024;
  return all < most ? all : most;
}

template <typename T, typename W> struct Norm {
  template <int TPR, int C> static void run(NormArgs a, hipStream_t stream) {
    constexpr int threads = TPR > 256 ? TPR : 256, per = threads / TPR;
    const int64_t most = 2048 * 256 / threads;
    a.run = per < 32 && TPR <= 64 && a.rows > 32 * most ? 32 : per;  // (few rows: one round of as many workgroups as there can be)
    const int64_t all = (a.rows + a.run - 1) / a.run;
    norm_kernel<T, W, TPR, C><<<dim3(unsigned(all < most ? all : most)), dim3(threads), 0, stream>>>(a);
  }
};
template <typename T, typename W> struct Grad {
  template <int TPR, int C> static void run(const GradArgs& a, unsigned blocks, hipStream_t stream) {
    norm_grad_kernel<T, W, TPR, C><<<dim3(blocks), dim3(TPR > 256 ? TPR : 256), 0, stream>>>(a);
  }
};

// Lanes a row by its width: as many as hold it with eight elements each, within a wave up to 1024 elements (no barrier).
template <template <typename, typename> class K, typename T, typename W, typename... Args> void by_width(int width, Args... args) {
  if (width <= 32) K<T, W>::template run<4, 1>(args...);
  else if (width <= 64) K<T, W>::template run<8, 1>(args...);
  else if (width <= 128) K<T, W>::template run<16, 1>(args...);
  else if (width <= 256) K<T, W>::template run<32, 1>(args...);
  else if (width <= 512) K<T, W>::template run<64, 1>(args...);
  else if (width <= 1024) K<T, W>::template run<64, 2>(args...);
  else if (width <= 2048) K<T, W>::template run<256, 1>(args...);
  else if (width <= 4096) K<T, W>::template run<256, 2>(args...);
  else if (width <= 8192) K<T, W>::template run<1024, 1>(args...);
  else if (width <= 16384) K<T, W>::template run<1024, 2>(args...);
  else K<T, W>::template run<1024, 4>(args...);
}
template <template <typename, typename> class K, typename... Args> void by_type(int type, int weight_type, int width, Args... args) {
  if (type == WDP_F32) by_width<K, float, float>(width, args...);
  else if (type == WDP_BF16 && weight_type == WDP_F32) by_width<K, bf16, float>(width, args...);
  else if (type == WDP_BF16) by_width<K, bf16, bf16>(width, args...);
  else if (weight_type == WDP_F32) by_width<K, f16, float>(width, args...);
  else by_width<K, f16, f16>(width, args...);
}

int check(const wdp_norm_config& c) {
  if (c.struct_size != sizeof(wdp_norm_config)) return WD_E_CONFIG;
  if (!is_float_type(c.type) || (c.weight_type != WDP_F32 && c.weight_type != c.type)) return WD_E_CONFIG;
  if (c.rows < 0 || c.rows > (int64_t(1) << 40) || c.width < 1) return WD_E_CONFIG;
  if (!(c.eps >= 0.0f) || !isfinite(c.eps)) return WD_E_CONFIG;
  if (c.width > kMaxWidth) return WD_E_UNSUPPORTED;
  return WD_OK;
}
bool stride_ok(const wdp_norm_config& c, int64_t stride) { return c.rows <= 1 || (stride >= c.width && stride <= (int64_t(1) << 40)); }

}  // namespace
}  // namespace wdp

extern "C" {

int wdp_norm(const wdp_norm_config* cfg, const wdp_norm_buffers* b) {
  using namespace wdp;
  if (!cfg || !b) return WD_E_NULL;
  const int rc = check(*cfg);
  if (rc != WD_OK) return rc;
  if (b->q && !is_8bit(cfg->q_type)) return WD_E_CONFIG;
  if (cfg->rows == 0) return WD_OK;
  if (!b->x || (!b->q != !b->scale) || !(b->h || b->y || b->q || b->rstd)) return WD_E_NULL;
  if (!stride_ok(*cfg, cfg->x_stride) || (b->residual && !stride_ok(*cfg, cfg->residual_stride)) || (b->h && !stride_ok(*cfg, cfg->h_stride)) ||
      (b->y && !stride_ok(*cfg, cfg->y_stride)) || (b->q && !stride_ok(*cfg, cfg->q_stride)))
    return WD_E_CONFIG;
  if (b->q && (cfg->scale_row_stride < 0 || cfg->scale_block_stride < 0)) return WD_E_CONFIG;
  if (cfg->rows > 1 && ((b->h && b->h == b->x && cfg->h_stride != cfg->x_stride) || (b->h && b->h == b->residual && cfg->h_stride != cfg->residual_stride)))
    return WD_E_CONFIG;
  const size_t e = size_of(cfg->type);
  if (!aligned(b->x, e) || !aligned(b->residual, e) || !aligned(b->h, e) || !aligned(b->y, e) || !aligned(b->weight, size_of(cfg->weight_type)) ||
      !aligned(b->scale, 4) || !aligned(b->rstd, 4))
    return WD_E_ALIGN;
  const NormArgs a = {b->x, b->residual, b->weight, b->h, b->y, static_cast<uint8_t*>(b->q), b->scale, b->rstd, cfg->rows, cfg->x_stride,
                      cfg->residual_stride, cfg->h_stride, cfg->y_stride, cfg->q_stride, cfg->scale_row_stride, cfg->scale_block_stride,
                      cfg->width, cfg->q_type, 0, cfg->eps, float(1.0 / cfg->width)};
  by_type<Norm>(cfg->type, cfg->weight_type, cfg->width, a, static_cast<hipStream_t>(cfg->stream));
  return launched();
}

int wdp_norm_backward_workspace(const wdp_norm_config* cfg, size_t* bytes) {
  using namespace wdp;
  if (!cfg || !bytes) return WD_E_NULL;
  const int rc = check(*cfg);
  if (rc != WD_OK) return rc;
  *bytes = size_t(grad_blocks(*cfg)) * size_t(cfg->width) * sizeof(float);
  return WD_OK;
}

int wdp_norm_backward(const wdp_norm_config* cfg, const wdp_norm_grad_buffers* b) {
  using namespace wdp;
  if (!cfg || !b) return WD_E_NULL;
  const int rc = check(*cfg);
  if (rc != WD_OK) return rc;
  if (!b->dx && !b->dw) return WD_E_NULL;
  if (cfg->rows > 0) {
    if (!b->dy || !b->h || !b->rstd || (b->dw && !b->workspace)) return WD_E_NULL;
    if (!stride_ok(*cfg, cfg->dy_stride) || !stride_ok(*cfg, cfg->h_stride) || (b->dh && !stride_ok(*cfg, cfg->dh_stride)) ||
        (b->dx && !stride_ok(*cfg, cfg->dx_stride)))
      return WD_E_CONFIG;
    if (cfg->rows > 1 && b->dx && ((b->dx == b->dy && cfg->dx_stride != cfg->dy_stride) || (b->dx == b->dh && cfg->dx_stride != cfg->dh_stride)))
      return WD_E_CONFIG;
    const size_t e = size_of(cfg->type);
    if (!aligned(b->dy, e) || !aligned(b->dh, e) || !aligned(b->h, e) || !aligned(b->dx, e) || !aligned(b->weight, size_of(cfg->weight_type)) ||
        !aligned(b->rstd, 4) || !aligned(b->dw, 4) || !aligned(b->workspace, 256))
      return WD_E_ALIGN;
  }
  const hipStream_t stream = static_cast<hipStream_t>(cfg->stream);
  const int64_t blocks = grad_blocks(*cfg);
  if (blocks) {
    const GradArgs a = {b->dy, b->dh, b->h, b->weight, b->rstd, b->dx, b->dw ? static_cast<float*>(b->workspace) : nullptr, cfg->rows,
                        cfg->dy_stride, cfg->dh_stride, cfg->h_stride, cfg->dx_stride, cfg->width, float(1.0 / cfg->width)};
    by_type<Grad>(cfg->type, cfg->weight_type, cfg->width, a, unsigned(blocks), stream);
    const int status = launched();
    if (status != WD_OK) return status;
  }
  if (b->dw) {  // (of no rows: zeros)
    norm_grad_join_kernel<<<dim3(unsigned((cfg->width + 15) / 16)), dim3(1024), 0, stream>>>(static_cast<const float*>(b->workspace), int(blocks), cfg->width, b->dw);
    return launched();
  }
  return WD_OK;
}

}  // extern "C"
