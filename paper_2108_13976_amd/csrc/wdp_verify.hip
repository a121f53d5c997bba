// wdp_verify.hip — drafted actions or tokens verified against the target's probabilities (include/wdp.h: wdp_verify).
//
// With drafts x_i from q_i, accepting x_i with probability min(1, p_i(x_i) / q_i(x_i)) and drawing from max(p_i - q_i, 0),
// normalised, at the first refusal gives tokens distributed as draws from p.  The test u q < p is a product of two
// floats (exact in float64) against a float; the draw compares float64 sums, whose order moves a border by 1e-16 of
// the row's sum, so that the kernels below, which sum in different orders, answer alike.
//
// Three forms by the vocabulary.  Few actions (a policy of Tag has five): a lane a sequence.  Rows that a workgroup
// holds in registers: a workgroup (or a wave) a sequence.  Longer rows: a workgroup a piece of 4096 elements sums it,
// a second launch finds the piece that holds the drawn token and goes through that one alone.
#include "wdp_common.h"

namespace wdp {
namespace {

constexpr int kPiece = 4096;   // elements that a workgroup of 256 sums in the form with two launches
constexpr int kMaxDrafts = 64; // one wave tests them
constexpr int kLaneVocab = 16; // largest vocabulary of the form with a lane a sequence

struct VerifyArgs {
  const void *target, *draft;
  const int32_t *drafts_in, *lengths;
  const float* u;
  int32_t *accepted, *tokens;
  double* sums;  // [batch][pieces][2]: of r, of max(p, 0)
  int64_t start, batch;  // sequences [start, batch) of this launch
  int64_t target_batch, target_row, draft_batch, draft_row;
  int32_t drafts, vocab, bonus, pieces;
};

__device__ __forceinline__ double positive(double v) { return v > 0.0 ? v : 0.0; }  // NaN is zero

template <typename T> __device__ __forceinline__ bool accepts(const VerifyArgs& a, int64_t s, int i, int x) {
  if (x < 0 || x >= a.vocab) return false;
  const double p = to_float(static_cast<const T*>(a.target)[s * a.target_batch + i * a.target_row + x]);
  const double q = to_float(static_cast<const T*>(a.draft)[s * a.draft_batch + i * a.draft_row + x]);
  return double(a.u[s * (a.drafts + 1) + i]) * q < p;
}

__device__ __forceinline__ int drafted(const VerifyArgs& a, int64_t s) {
  if (!a.lengths) return a.drafts;
  const int n = a.lengths[s];
  return n < 0 ? 0 : n > a.drafts ? a.drafts : n;
}

// How many drafts of sequence s are accepted, by one wave (all 64 lanes of it).
template <typename T> __device__ __forceinline__ int count_accepted(const VerifyArgs& a, int64_t s, int n) {
  const int i = threadIdx.x & 63;
  const bool ok = i < n && accepts<T>(a, s, i, a.drafts_in[s * a.drafts + i]);
  const uint64_t refused = ~__ballot(ok);
  return refused ? __builtin_ctzll(refused) : 64;
}

// Where the draw's row stands; q is NULL at the bonus row.  False: no draw.
template <typename T>
__device__ __forceinline__ bool draw_rows(const VerifyArgs& a, int64_t s, int accepted, int n, const T** p, const T** q) {
  const bool whole = accepted == n;
  if (whole && !a.bonus) return false;
  *p = static_cast<const T*>(a.target) + s * a.target_batch + accepted * a.target_row;
  *q = whole ? nullptr : static_cast<const T*>(a.draft) + s * a.draft_batch + accepted * a.draft_row;
  return true;
}

// The outputs of a sequence: drafts up to `accepted`, the drawn token (or -1), -1.  Lanes l, l + step, ...
__device__ __forceinline__ void write_tokens(const VerifyArgs& a, int64_t s, int accepted, int token, int l, int step) {
  const int slots = a.drafts + a.bonus;
  for (int i = l; i < slots; i += step)
    a.tokens[s * slots + i] = i < accepted ? a.drafts_in[s * a.drafts + i] : i == accepted ? token : -1;
  if (l == 0 && a.accepted) a.accepted[s] = accepted;
}

// ---- a lane a sequence ----------------------------------------------------------------------
template <typename T> __global__ __launch_bounds__(256) void verify_lane_kernel(VerifyArgs a) {
  const int64_t s = a.start + int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (s >= a.batch) return;
  const int n = drafted(a, s);
  int accepted = 0;
  while (accepted < n && accepts<T>(a, s, accepted, a.drafts_in[s * a.drafts + accepted])) ++accepted;
  const T *p, *q;
  int token = -1;
  if (draw_rows(a, s, accepted, n, &p, &q)) {
    double sum = 0.0, plain = 0.0;
    for (int j = 0; j < a.vocab; ++j) {
      const double v = to_float(p[j]);
      sum += positive(q ? v - double(to_float(q[j])) : v);
      plain += positive(v);
    }
    if (!(sum > 0.0)) q = nullptr, sum = plain;
    const double mark = double(a.u[s * (a.drafts + 1) + a.drafts]) * sum;
    double run = 0.0;
    token = a.vocab - 1;
    for (int j = 0; j < a.vocab; ++j) {
      const double v = to_float(p[j]), r = positive(q ? v - double(to_float(q[j])) : v);
      if (!(r > 0.0)) continue;
      run += r;
      token = j;
      if (run > mark) break;
    }
  }
  write_tokens(a, s, accepted, token, 0, 1);
}

// ---- a workgroup's search for the token within elements [at, at + 16 * threads) -----------------
// r[16]: the lane's adjacent elements; before: sum of everything in front of them.  Lanes' sums are scanned over the
// workgroup; the first element whose running sum passes the mark wins, else the last that is above zero.
constexpr int kEach = 16;

template <typename T>
__device__ __forceinline__ void load_rest(const T* p, const T* q, int first, int vocab, double r[kEach], double* plain) {
  *plain = 0.0;
#pragma unroll
  for (int h = 0; h < kEach; h += 8) {
    float pv[8], qv[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) pv[i] = qv[i] = 0.0f;
    if (first + h < vocab) {
      load_some<T, 8>(p + first + h, vocab - first - h, pv);
      if (q) load_some<T, 8>(q + first + h, vocab - first - h, qv);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      r[h + i] = positive(double(pv[i]) - double(qv[i]));
      *plain += positive(double(pv[i]));
    }
  }
}

__device__ __forceinline__ double shuffle_up(double v, int by) { return __shfl_up(v, by); }

// Inclusive scan over the workgroup's lanes; *total: the sum.  Two barriers (waves > 1).
template <int WAVES> __device__ __forceinline__ double scan(double v, double* places, double* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int by = 1; by < 64; by <<= 1) {
    const double left = shuffle_up(v, by);
    if (lane >= by) v += left;
  }
  if (WAVES == 1) {
    *total = __shfl(v, 63);
    return v;
  }
  __syncthreads();
  if (lane == 63) places[wave] = v;
  __syncthreads();
  double before = 0.0, all = 0.0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    if (w < wave) before += places[w];
    all += places[w];
  }
  *total = all;
  return v + before;
}

// The token among the workgroup's elements, from the running sum `behind` at the end of this lane's elements (own:
// their sum), the elements in front of the workgroup included in neither mark nor sums.  -1: nothing above zero.
template <int WAVES> __device__ __forceinline__ int find(const double r[kEach], double behind, double own, double mark, int first, int* best) {
  if (threadIdx.x == 0) best[0] = 0x7FFFFFFF, best[1] = -1;
  __syncthreads();
  double run = behind - own;
  int hit = 0x7FFFFFFF, last = -1;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    run += r[i];
    if (r[i] > 0.0) {
      last = first + i;
      if (run > mark && hit == 0x7FFFFFFF) hit = first + i;
    }
  }
  if (hit != 0x7FFFFFFF) atomicMin(&best[0], hit);
  if (last >= 0) atomicMax(&best[1], last);
  __syncthreads();
  return best[0] != 0x7FFFFFFF ? best[0] : best[1];
}

// ---- a workgroup (or wave) a sequence: the whole row in registers -------------------------------------
template <typename T, int WAVES> __global__ __launch_bounds__(64 * WAVES) void verify_row_kernel(VerifyArgs a) {
  __shared__ double places[WAVES];
  __shared__ int best[2];
  const int64_t s = a.start + blockIdx.x;
  const int n = drafted(a, s);
  const int accepted = count_accepted<T>(a, s, n);  // (each wave for itself)
  const T *p, *q;
  int token = -1;
  if (draw_rows(a, s, accepted, n, &p, &q)) {
    const int first = threadIdx.x * kEach;
    double r[kEach], plain, sum, own = 0.0;
    load_rest<T>(p, q, first, a.vocab, r, &plain);
#pragma unroll
    for (int i = 0; i < kEach; ++i) own += r[i];
    double behind = scan<WAVES>(own, places, &sum);
    if (!(sum > 0.0) && q) {  // nothing is left of p - q: from p itself
      load_rest<T>(p, static_cast<const T*>(nullptr), first, a.vocab, r, &own);
      behind = scan<WAVES>(own, places, &sum);
    }
    token = find<WAVES>(r, behind, own, double(a.u[s * (a.drafts + 1) + a.drafts]) * sum, first, best);
    if (token < 0) token = a.vocab - 1;
  }
  __syncthreads();
  write_tokens(a, s, accepted, token, threadIdx.x, 64 * WAVES);
}

// ---- long rows: sums of the pieces, then the search in one of them --------------------------------------
template <typename T> __global__ __launch_bounds__(256) void verify_sums_kernel(VerifyArgs a) {
  __shared__ double places[4];
  const int64_t s = a.start + blockIdx.y + int64_t(blockIdx.z) * 32768;
  if (s >= a.batch) return;
  const int n = drafted(a, s), accepted = count_accepted<T>(a, s, n);
  const T *p, *q;
  if (!draw_rows(a, s, accepted, n, &p, &q)) return;
  double r[kEach], plain, sum, all, own = 0.0;
  load_rest<T>(p, q, blockIdx.x * kPiece + threadIdx.x * kEach, a.vocab, r, &plain);
#pragma unroll
  for (int i = 0; i < kEach; ++i) own += r[i];
  scan<4>(own, places, &sum);
  scan<4>(plain, places, &all);
  if (threadIdx.x == 0) {
    a.sums[(s * a.pieces + blockIdx.x) * 2] = sum;
    a.sums[(s * a.pieces + blockIdx.x) * 2 + 1] = all;
  }
}

template <typename T> __global__ __launch_bounds__(256) void verify_find_kernel(VerifyArgs a) {
  __shared__ double places[4];
  __shared__ int best[2];
  const int64_t s = a.start + blockIdx.x;
  const int n = drafted(a, s), accepted = count_accepted<T>(a, s, n);
  const T *p, *q;
  int token = -1;
  if (draw_rows(a, s, accepted, n, &p, &q)) {
    // the row's sum, and the piece: every lane goes through the pieces' sums (the same order in all)
    const double* sums = a.sums + s * a.pieces * 2;
    double total = 0.0, plain = 0.0;
    for (int i = 0; i < a.pieces; ++i) total += sums[2 * i], plain += sums[2 * i + 1];
    const bool from_p = !(total > 0.0) && q;
    if (from_p) total = plain, q = nullptr;
    const double mark = double(a.u[s * (a.drafts + 1) + a.drafts]) * total;
    double run = 0.0, before = 0.0;
    int piece = -1;
    for (int i = 0; i < a.pieces; ++i) {
      const double v = sums[2 * i + (from_p ? 1 : 0)];
      if (!(v > 0.0)) continue;
      piece = i, before = run;
      run += v;
      if (run > mark) break;
    }
    if (piece >= 0) {
      const int first = piece * kPiece + threadIdx.x * kEach;
      double r[kEach], unused, all, own = 0.0;
      load_rest<T>(p, q, first, a.vocab, r, &unused);
#pragma unroll
      for (int i = 0; i < kEach; ++i) own += r[i];
      const double behind = scan<4>(own, places, &all) + before;
      token = find<4>(r, behind, own, mark, first, best);
    }
    if (token < 0) token = a.vocab - 1;
  }
  __syncthreads();
  write_tokens(a, s, accepted, token, threadIdx.x, 256);
}

// (a launch takes 2^22 sequences: all sizes of a grid stay far from their limits)
template <typename T> void launch(VerifyArgs a, hipStream_t stream) {
  const int64_t end = a.batch, most = int64_t(1) << 22;
  for (; a.start < end; a.start += most) {
    a.batch = end - a.start < most ? end : a.start + most;
    const unsigned count = unsigned(a.batch - a.start);
    if (a.vocab <= kLaneVocab) verify_lane_kernel<T><<<dim3((count + 255) / 256), 256, 0, stream>>>(a);
    else if (a.vocab <= 64 * kEach) verify_row_kernel<T, 1><<<dim3(count), 64, 0, stream>>>(a);
    else if (a.vocab <= kPiece) verify_row_kernel<T, 4><<<dim3(count), 256, 0, stream>>>(a);
    else {
      verify_sums_kernel<T><<<dim3(unsigned(a.pieces), count < 32768 ? count : 32768, (count + 32767) / 32768), 256, 0, stream>>>(a);
      verify_find_kernel<T><<<dim3(count), 256, 0, stream>>>(a);
    }
  }
}

int pieces_of(const wdp_verify_config& c) { return c.vocab <= kPiece ? 0 : (c.vocab + kPiece - 1) / kPiece; }

int check(const wdp_verify_config& c) {
  if (c.struct_size != sizeof(wdp_verify_config) || !is_float_type(c.type)) return WD_E_CONFIG;
  if (c.batch < 0 || c.batch > 0x7FFFFFFF || c.drafts < 0 || c.drafts > kMaxDrafts || c.vocab < 1 || c.vocab > (1 << 24)) return WD_E_CONFIG;
  if ((c.bonus != 0 && c.bonus != 1) || c.drafts + c.bonus < 1) return WD_E_CONFIG;
  const int64_t most = int64_t(1) << 40;
  if (c.drafts + c.bonus > 1 && (c.target_row_stride < c.vocab || c.target_row_stride > most)) return WD_E_CONFIG;
  if (c.drafts > 1 && (c.draft_row_stride < c.vocab || c.draft_row_stride > most)) return WD_E_CONFIG;
  if (c.batch > 1 && (c.target_batch_stride < 0 || c.target_batch_stride > most || c.draft_batch_stride < 0 || c.draft_batch_stride > most)) return WD_E_CONFIG;
  return WD_OK;
}

}  // namespace
}  // namespace wdp

extern "C" {

int wdp_verify_workspace(const wdp_verify_config* cfg, size_t* bytes) {
  if (!cfg || !bytes) return WD_E_NULL;
  const int rc = wdp::check(*cfg);
  if (rc != WD_OK) return rc;
  *bytes = size_t(cfg->batch) * size_t(wdp::pieces_of(*cfg)) * 2 * sizeof(double);
  return WD_OK;
}

int wdp_verify(const wdp_verify_config* cfg, const wdp_verify_buffers* b) {
  using namespace wdp;
  if (!cfg || !b) return WD_E_NULL;
  const int rc = check(*cfg);
  if (rc != WD_OK) return rc;
  if (cfg->batch == 0) return WD_OK;
  const int pieces = pieces_of(*cfg);
  if (!b->target || !b->u || !b->tokens || (cfg->drafts > 0 && (!b->draft_probs || !b->drafts_in)) || (pieces && !b->workspace)) return WD_E_NULL;
  if (cfg->bonus && b->tokens == b->drafts_in) return WD_E_CONFIG;
  const size_t e = size_of(cfg->type);
  if (!aligned(b->target, e) || !aligned(b->draft_probs, e) || !aligned(b->drafts_in, 4) || !aligned(b->lengths, 4) || !aligned(b->u, 4) ||
      !aligned(b->accepted, 4) || !aligned(b->tokens, 4) || !aligned(b->workspace, 256))
    return WD_E_ALIGN;
  const VerifyArgs a = {b->target, b->draft_probs, b->drafts_in, b->lengths, b->u, b->accepted, b->tokens, static_cast<double*>(b->workspace),
                        0, cfg->batch, cfg->target_batch_stride, cfg->target_row_stride, cfg->draft_batch_stride, cfg->draft_row_stride,
                        cfg->drafts, cfg->vocab, cfg->bonus, pieces};
  const hipStream_t stream = static_cast<hipStream_t>(cfg->stream);
  if (cfg->type == WDP_F32) launch<float>(a, stream);
  else if (cfg->type == WDP_BF16) launch<bf16>(a, stream);
  else launch<f16>(a, stream);
  return launched();
}

}  // extern "C"
