// wdp_verify.hip — drafted actions or tokens verified against the target's probabilities (include/wdp.h: wdp_verify).
//
// With drafts x_i from q_i, accepting x_i with probability min(1, p_i(x_i) / q_i(x_i)) and drawing from max(p_i - q_i, 0),
// normalised, at the first refusal gives tokens distributed as draws from p.  The test u q < p is a product of two
// floats (exact in float64) against a float; the draw compares float64 sums, whose order moves a border by 1e-16 of
// the row's sum, so that the kernels below, which sum in different orders, answer alike.
//
// Forms by the vocabulary.  Few actions (a policy of Tag has five): a lane a sequence, the row in its registers.  Up to
// 1024: sixteen lanes (256) or a wave a sequence, no barrier (50000 x 2 x 100: 24 us with a wave each, 13 with sixteen
// lanes).  Up to 4096: a workgroup.  Longer rows: a wave a piece of 1024 elements sums it, a second launch finds the piece
// that holds the drawn token and goes through that one alone.  Memory bounds the large batches (2000000 x 1 x 5: 24 us,
// 5.6 TB/s), the chain of dependent loads (drafts, their elements, the row, the token) the small ones (64 x 4 x 50000:
// 7.6 us and 4.6).
#include "wdp_common.h"

namespace wdp {
namespace {

constexpr int kRow = 4096;     // largest vocabulary that a workgroup of 256 holds in registers
constexpr int kPiece = 1024;   // elements that a wave sums in the form with two launches
constexpr int kMaxDrafts = 64;

struct VerifyArgs {
  const void *target, *draft;
  const int32_t *drafts_in, *lengths;
  const float* u;
  int32_t *accepted, *tokens;
  double* sums;  // [batch][pieces][2]: of r, of max(p, 0); behind them int32 [batch]: accepted
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
// ONE: one draft and no bonus row, so that both rows are known beforehand and the test takes its elements from them.
template <typename T, int MOST, bool ONE> __global__ __launch_bounds__(256) void verify_lane_kernel(VerifyArgs a) {
  const int64_t s = a.start + int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (s >= a.batch) return;
  const int n = drafted(a, s);
  float p[MOST], q[MOST];
  const auto load = [&](const T* from_p, const T* from_q) {
#pragma unroll
    for (int j = 0; j < MOST; ++j) {
      p[j] = j < a.vocab ? to_float(from_p[j]) : 0.0f;
      q[j] = j < a.vocab && from_q ? to_float(from_q[j]) : 0.0f;
    }
  };
  int accepted = 0, first = -1;
  bool draws;
  if (ONE) {
    first = a.drafts_in[s];
    const double u = a.u[2 * s];
    load(static_cast<const T*>(a.target) + s * a.target_batch, static_cast<const T*>(a.draft) + s * a.draft_batch);
    float px = 0.0f, qx = 1.0f;  // (a token out of range is refused)
#pragma unroll
    for (int j = 0; j < MOST; ++j)
      if (j == first && j < a.vocab) px = p[j], qx = q[j];
    accepted = n == 1 && first >= 0 && first < a.vocab && u * double(qx) < double(px);
    draws = accepted < n;
  } else {
    while (accepted < n && accepts<T>(a, s, accepted, a.drafts_in[s * a.drafts + accepted])) ++accepted;
    const T *from_p, *from_q;
    draws = draw_rows(a, s, accepted, n, &from_p, &from_q);
    if (draws) load(from_p, from_q);
  }
  int token = -1;
  if (draws) {
    double r[MOST], sum = 0.0;
#pragma unroll
    for (int j = 0; j < MOST; ++j) r[j] = positive(double(p[j]) - double(q[j])), sum += r[j];
    if (!(sum > 0.0)) {  // nothing is left of p - q: from p itself
      sum = 0.0;
#pragma unroll
      for (int j = 0; j < MOST; ++j) r[j] = positive(double(p[j])), sum += r[j];
    }
    const double mark = double(a.u[s * (a.drafts + 1) + a.drafts]) * sum;
    double run = 0.0;
    bool found = false;
    token = a.vocab - 1;
#pragma unroll
    for (int j = 0; j < MOST; ++j) {
      run += r[j];
      if (!found && r[j] > 0.0) token = j, found = run > mark;
    }
  }
  if (ONE) {
    a.tokens[s] = accepted ? first : token;
    if (a.accepted) a.accepted[s] = accepted;
  } else {
    write_tokens(a, s, accepted, token, 0, 1);
  }
}

// ---- a workgroup's search for the token within elements [at, at + 16 * threads) -----------------
// r: the lane's adjacent elements.  Lanes' sums are scanned over the workgroup; the first element whose running sum passes
// the mark wins, else the last that is above zero.
constexpr int kEach = 16;

template <typename T, int E>
__device__ __forceinline__ void load_rest(const T* p, const T* q, int first, int vocab, double r[E], double* plain) {
  constexpr int kStep = E < 8 ? E : 8;
  *plain = 0.0;
#pragma unroll
  for (int h = 0; h < E; h += kStep) {
    float pv[kStep], qv[kStep];
#pragma unroll
    for (int i = 0; i < kStep; ++i) pv[i] = qv[i] = 0.0f;
    if (first + h < vocab) {
      load_some<T, kStep>(p + first + h, vocab - first - h, pv);
      if (q) load_some<T, kStep>(q + first + h, vocab - first - h, qv);
    }
#pragma unroll
    for (int i = 0; i < kStep; ++i) {
      r[h + i] = positive(double(pv[i]) - double(qv[i]));
      *plain += positive(double(pv[i]));
    }
  }
}

// Inclusive scan over aligned groups of G = 16 or 64 lanes (all of them active): within a row of sixteen lanes by shifts
// that need no LDS, then the sums of the rows before.
template <int BY> __device__ __forceinline__ double from_left(double v) {  // zero where there is no such lane in the row
  const uint64_t bits = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, int(bits), 0x110 + BY, 0xF, 0xF, true);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, int(bits >> 32), 0x110 + BY, 0xF, 0xF, true);
  return __builtin_bit_cast(double, uint64_t(hi) << 32 | lo);
}
__device__ __forceinline__ double of_lane(double v, int lane) {
  const uint64_t bits = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_readlane(int(bits), lane), hi = __builtin_amdgcn_readlane(int(bits >> 32), lane);
  return __builtin_bit_cast(double, uint64_t(hi) << 32 | lo);
}
template <int G> __device__ __forceinline__ double group_scan(double v) {
  static_assert(G == 16 || G == 64, "a row of lanes, or the wave");
  v += from_left<1>(v);
  v += from_left<2>(v);
  v += from_left<4>(v);
  v += from_left<8>(v);
  if (G == 64) {
    const int row = (threadIdx.x >> 4) & 3;
    const double a = of_lane(v, 15), b = of_lane(v, 31), c = of_lane(v, 47);
    v += row == 0 ? 0.0 : row == 1 ? a : row == 2 ? a + b : a + b + c;
  }
  return v;
}
// The group's last lane's value, in all of them.
template <int G> __device__ __forceinline__ double last_of(double v) { return G == 64 ? of_lane(v, 63) : __shfl(v, G - 1, G); }

// The token among a group's elements r (E adjacent ones a lane, from `first` on), `run` being the sum of everything before
// the lane's: the first above zero whose running sum passes the mark, else the last above zero, else -1.
template <int G, int E, typename Votes> __device__ __forceinline__ int find_in_group(const double r[E], double run, double mark, int first, Votes votes) {
  int hit = -1, last = -1;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    run += r[i];
    if (r[i] > 0.0) {
      last = first + i;
      if (hit < 0 && run > mark) hit = first + i;
    }
  }
  const uint64_t hits = votes(hit >= 0), some = votes(last >= 0);
  if (hits) return __shfl(hit, __builtin_ctzll(hits), G);
  return some ? __shfl(last, 63 - __builtin_clzll(some), G) : -1;
}

// ---- G lanes a sequence, E adjacent elements of the row each -----------------------------------------
template <typename T, int G, int E> __global__ __launch_bounds__(256) void verify_group_kernel(VerifyArgs a) {
  const int64_t s = a.start + int64_t(blockIdx.x) * (256 / G) + threadIdx.x / G;
  if (s >= a.batch) return;
  const int lane = threadIdx.x & (G - 1), shift = threadIdx.x & 63 & ~(G - 1);
  const auto votes = [&](bool yes) { return (__ballot(yes) >> shift) & (~uint64_t(0) >> (64 - G)); };  // of the group
  const int n = drafted(a, s);
  int accepted = 0;
  for (int at = 0; at < n; at += G) {
    const bool ok = at + lane < n && accepts<T>(a, s, at + lane, a.drafts_in[s * a.drafts + at + lane]);
    const uint64_t refused = votes(!ok);
    accepted = at + (refused ? __builtin_ctzll(refused) : G);
    if (refused) break;
  }
  const T *p, *q;
  int token = -1;
  if (draw_rows(a, s, accepted, n, &p, &q)) {
    const int first = lane * E;
    double r[E], plain, own = 0.0;
    load_rest<T, E>(p, q, first, a.vocab, r, &plain);
#pragma unroll
    for (int i = 0; i < E; ++i) own += r[i];
    double behind = group_scan<G>(own), sum = last_of<G>(behind);
    if (!(sum > 0.0) && q) {  // nothing is left of p - q: from p itself
      load_rest<T, E>(p, static_cast<const T*>(nullptr), first, a.vocab, r, &own);
      behind = group_scan<G>(own), sum = last_of<G>(behind);
    }
    const double mark = double(a.u[s * (a.drafts + 1) + a.drafts]) * sum;
    token = find_in_group<G, E>(r, behind - own, mark, first, votes);
    if (token < 0) token = a.vocab - 1;
  }
  write_tokens(a, s, accepted, token, lane, G);
}

// Inclusive scan over the workgroup's lanes; *total: the sum.  Two barriers.
template <int WAVES> __device__ __forceinline__ double scan(double v, double* places, double* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  v = group_scan<64>(v);
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

// ---- a workgroup a sequence: the whole row in registers -------------------------------------
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
    load_rest<T, kEach>(p, q, first, a.vocab, r, &plain);
#pragma unroll
    for (int i = 0; i < kEach; ++i) own += r[i];
    double behind = scan<WAVES>(own, places, &sum);
    if (!(sum > 0.0) && q) {  // nothing is left of p - q: from p itself
      load_rest<T, kEach>(p, static_cast<const T*>(nullptr), first, a.vocab, r, &own);
      behind = scan<WAVES>(own, places, &sum);
    }
    token = find<WAVES>(r, behind, own, double(a.u[s * (a.drafts + 1) + a.drafts]) * sum, first, best);
    if (token < 0) token = a.vocab - 1;
  }
  __syncthreads();
  write_tokens(a, s, accepted, token, threadIdx.x, 64 * WAVES);
}

// ---- long rows: sums of the pieces, then the search in one of them --------------------------------------
__device__ __forceinline__ int32_t* counts(const VerifyArgs& a, int64_t all) { return reinterpret_cast<int32_t*>(a.sums + all * a.pieces * 2); }

template <typename T> __global__ __launch_bounds__(256) void verify_sums_kernel(VerifyArgs a, int64_t all) {
  const int64_t s = a.start + blockIdx.y + int64_t(blockIdx.z) * 32768;
  if (s >= a.batch) return;
  const int n = drafted(a, s), accepted = count_accepted<T>(a, s, n);
  if (blockIdx.x == 0 && threadIdx.x == 0) counts(a, all)[s] = accepted;
  const int piece = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  const T *p, *q;
  if (piece >= a.pieces || !draw_rows(a, s, accepted, n, &p, &q)) return;
  double r[kEach], plain, own = 0.0;
  load_rest<T, kEach>(p, q, piece * kPiece + lane * kEach, a.vocab, r, &plain);
#pragma unroll
  for (int i = 0; i < kEach; ++i) own += r[i];
  own = group_scan<64>(own), plain = group_scan<64>(plain);
  if (lane == 63) {
    a.sums[(s * a.pieces + piece) * 2] = own;
    a.sums[(s * a.pieces + piece) * 2 + 1] = plain;
  }
}

template <typename T> __global__ __launch_bounds__(64) void verify_find_kernel(VerifyArgs a, int64_t all) {
  const int64_t s = a.start + blockIdx.x;
  // everything that depends on nothing is asked for at once: the call's time is the chain of loads that do
  const int lane = threadIdx.x, slots = a.drafts + a.bonus;
  const double* sums = a.sums + s * a.pieces * 2;
  const double first_sum = lane < a.pieces ? sums[2 * lane] : 0.0, first_plain = lane < a.pieces ? sums[2 * lane + 1] : 0.0;
  const double u = a.u[s * (a.drafts + 1) + a.drafts];
  const int kept = lane < a.drafts ? a.drafts_in[s * a.drafts + lane] : -1;  // (at most 64)
  const int n = drafted(a, s), accepted = counts(a, all)[s];
  const T *p, *q;
  int token = -1;
  if (draw_rows(a, s, accepted, n, &p, &q)) {
    // the row's sum and the piece, by each wave for itself: 64 pieces at a time
    double total = first_sum;
    for (int at = 64; at < a.pieces; at += 64) total += at + lane < a.pieces ? sums[2 * (at + lane)] : 0.0;
    total = of_lane(group_scan<64>(total), 63);
    const bool from_p = !(total > 0.0) && q;
    if (from_p) {
      q = nullptr, total = first_plain;
      for (int at = 64; at < a.pieces; at += 64) total += at + lane < a.pieces ? sums[2 * (at + lane) + 1] : 0.0;
      total = of_lane(group_scan<64>(total), 63);
    }
    const double mark = u * total;
    double run = 0.0, before = 0.0;
    int piece = -1;
    for (int at = 0; at < a.pieces; at += 64) {
      double v = 0.0;
      if (at == 0) v = from_p ? first_plain : first_sum;
      else if (at + lane < a.pieces) v = sums[2 * (at + lane) + (from_p ? 1 : 0)];
      const double behind = run + group_scan<64>(v);
      const uint64_t some = __ballot(v > 0.0), hits = __ballot(v > 0.0 && behind > mark);
      if (hits || some) {
        const int l = hits ? __builtin_ctzll(hits) : 63 - __builtin_clzll(some);
        piece = at + l, before = of_lane(behind - v, l);
      }
      if (hits) break;
      run = of_lane(behind, 63);
    }
    if (piece >= 0) {
      const int first = piece * kPiece + lane * kEach;
      double r[kEach], unused, own = 0.0;
      load_rest<T, kEach>(p, q, first, a.vocab, r, &unused);
#pragma unroll
      for (int i = 0; i < kEach; ++i) own += r[i];
      const double behind = group_scan<64>(own) + before;
      token = find_in_group<64, kEach>(r, behind - own, mark, first, [](bool yes) { return uint64_t(__ballot(yes)); });
    }
    if (token < 0) token = a.vocab - 1;
  }
  // (65 slots at most: drafts and one more)
  for (int i = lane; i < slots; i += 64) a.tokens[s * slots + i] = i < accepted ? kept : i == accepted ? token : -1;
  if (lane == 0 && a.accepted) a.accepted[s] = accepted;
}

// (a launch takes 2^22 sequences: all sizes of a grid stay far from their limits)
template <typename T> int launch(VerifyArgs a, hipStream_t stream) {
  const int64_t end = a.batch, most = int64_t(1) << 22;
  for (; a.start < end; a.start += most) {
    a.batch = end - a.start < most ? end : a.start + most;
    const unsigned count = unsigned(a.batch - a.start);
    int status;
    const auto blocks = [&](unsigned each) { return dim3((count + each - 1) / each); };
    if (a.vocab <= 8 && a.drafts == 1 && !a.bonus) status = enqueue(verify_lane_kernel<T, 8, true>, blocks(256), 256, stream, a);
    else if (a.vocab <= 8) status = enqueue(verify_lane_kernel<T, 8, false>, blocks(256), 256, stream, a);
    else if (a.vocab <= 64) status = enqueue(verify_group_kernel<T, 16, 4>, blocks(16), 256, stream, a);
    else if (a.vocab <= 128) status = enqueue(verify_group_kernel<T, 16, 8>, blocks(16), 256, stream, a);
    else if (a.vocab <= 256) status = enqueue(verify_group_kernel<T, 16, 16>, blocks(16), 256, stream, a);
    else if (a.vocab <= 1024) status = enqueue(verify_group_kernel<T, 64, 16>, blocks(4), 256, stream, a);
    else if (a.vocab <= kRow) status = enqueue(verify_row_kernel<T, 4>, dim3(count), 256, stream, a);
    else {
      status = enqueue(verify_sums_kernel<T>, dim3(unsigned((a.pieces + 3) / 4), count < 32768 ? count : 32768, (count + 32767) / 32768), 256, stream, a, end);
      if (status == WD_OK) status = enqueue(verify_find_kernel<T>, dim3(count), 64, stream, a, end);
    }
    if (status != WD_OK) return status;
  }
  return WD_OK;
}

int pieces_of(const wdp_verify_config& c) { return c.vocab <= kRow ? 0 : (c.vocab + kPiece - 1) / kPiece; }

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
  const size_t pieces = size_t(wdp::pieces_of(*cfg));
  *bytes = pieces ? size_t(cfg->batch) * (pieces * 2 * sizeof(double) + sizeof(int32_t)) : 0;
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
  if (cfg->type == WDP_F32) return launch<float>(a, stream);
  return cfg->type == WDP_BF16 ? launch<bf16>(a, stream) : launch<f16>(a, stream);
}

}  // extern "C"
