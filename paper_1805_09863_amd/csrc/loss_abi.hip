// Host side of the output layer's losses: argument validation, the plan of a
// call and the entry points declared in include/kbest_loss.h.
#include <float.h>
#include <limits.h>
#include <math.h>

#include <algorithm>

#include "kb_status.hpp"
#include "kbest_loss.h"
#include "loss_common.hpp"

namespace kb {
hipError_t launch_loss_logits_bf16(int planes, int BN, const LossLogitsArgs& a, int blocks, hipStream_t st);
hipError_t launch_loss_logits_f32(int planes, int BN, const LossLogitsArgs& a, int blocks, hipStream_t st);
hipError_t launch_loss_dh_bf16(int BN, const LossGradArgs& a, hipStream_t st);
hipError_t launch_loss_dh_f32(int BN, const LossGradArgs& a, hipStream_t st);
hipError_t launch_loss_dw_bf16(int planes, int BNh, const LossGradArgs& a, hipStream_t st);
hipError_t launch_loss_dw_f32(int planes, int BNh, const LossGradArgs& a, hipStream_t st);
hipError_t launch_loss_both_bf16(int BN, const LossGradArgs& h, const LossGradArgs& w, hipStream_t st);
hipError_t launch_loss_both_f32(int BN, const LossGradArgs& h, const LossGradArgs& w, hipStream_t st);
}  // namespace kb

namespace {

using kb::aligned;
using kb::fail;
using kb::ok;

static_assert(kb::kLossMaxV == KB_LOSS_MAX_V && kb::kLossMaxK == KB_LOSS_MAX_K, "the same limits");

int up(int x, int a) { return (x + a - 1) / a * a; }

// Takes stretches of a workspace, each at a multiple of 256 bytes.
struct Space {
  size_t at = 0;
  size_t take(size_t bytes) {
    const size_t p = at;
    at = (at + bytes + 255) / 256 * 256;
    return p;
  }
};

struct Plan {
  bool bf16, few, direct;  // few: the few rows' kernels
  int planes, g_planes, z;  // bf16 pieces of the operands and of the dlogits, bytes of a value
  int N, H, V, K;
  int BN, R, WN, WTM, WTN;  // row tile, how many, and the wave's part
  int Hp, Hk, BNh;
  int BNd, Rd, two;         // dh: its row tile and how many; where second pieces of the dlogits lie (0: none)
  int dw_grid;
  int vt, words0, nb, grid;
  int piece;                // word tiles of a piece of the vocabulary
  int pieces;
  int dh_mt, dh_splits, dw_ntn, dw_splits;
  // workspace
  size_t count, map, inv, flag, token, part, known, offs, items, ph, b, wp, stat, sumx, xt, rowp, g, dbp, dh_part, dw_part;
  size_t stat_piece;        // values of one piece's statistics
  size_t bytes;
  bool both() const { return BN >= 192 && BNh == 256; }  // dh and dW in one launch
};

// The row tile with the least time for the logits: rounds of the card's workgroups times a tile's time, which is that of
// its stages (96 of float32, 512 states: 73 us for 256 rows, 60 for 192, 50 for 128, 38 for 64, 32 for 32; two workgroups
// of the last on a CU 44), so small problems take small tiles (a training pass of 163 x 512 x 4,384 in float32: 124 us in
// tiles of 32 rows, 251 in tiles of 256; bf16 6,852 x 512 x 2,000: 156 in tiles of 256, 179 in tiles of 128), and others
// those that leave least of the last round and the last tile empty (scored and trained: 640 x 512 x 30,000 in float32
// 608 in tiles of 192, 663 in tiles of 256; 570 x 1,024 x 50,000 in bf16 334, 372 and, in tiles of 128, 368; 180 x 1,024 x
// 60,000 175, 196 and 205).  How many of the rows count is not known here: the sum over all, nine tenths and eight tenths
// of them, as a batch's padding has it (1,111 x 512 x 32,000 in bf16: 226 in tiles of 192, 253 in tiles of 256; of 889
// rows that count 207 and 200).
int row_tile(int N, int vt) {
  int best = 32;
  long long least = LLONG_MAX;
  for (int BN : {32, 64, 128, 192, 256}) {
    long long all = 0;
    for (int tenths : {10, 9, 8}) {
      const int rows = (int)(((long long)N * tenths + 9) / 10);
      const long long cells = (long long)kb::loss_row_tiles(rows, BN) * vt;
      const int slots = BN == 32 ? 512 : 256;
      const int time = BN == 256 ? 73 : BN == 192 ? 60 : BN == 128 ? 50 : BN == 64 ? 38 : cells <= 256 ? 32 : 44;
      all += (cells + slots - 1) / slots * time;
    }
    if (all < least) best = BN, least = all;
    if (BN >= N) break;
  }
  return best;
}

// When the last of nh workgroups of lh stages each, and after them nw of lw, is done, with 256 at a time.
long long all_done(long long nh, long long lh, long long nw, long long lw) {
  const long long q = nh / 256, rest = nh % 256;
  auto fits = [&](long long t) {  // of the second kind, by then
    return std::max(0ll, (t - q * lh) / lw) * (256 - rest) + std::max(0ll, (t - (q + 1) * lh) / lw) * rest;
  };
  long long lo = q * lh + (rest > 0 ? lh : 0), hi = lo + (nw + 255) / 256 * lw;
  if (fits(lo) >= nw) return lo;
  while (lo + 1 < hi) {
    const long long t = (lo + hi) / 2;
    (fits(t) >= nw ? hi : lo) = t;
  }
  return hi;
}

struct Splits {
  int dh, dw;
  long long time;  // in stages of 32 steps
};

// dh and dW of a piece of `tiles` word tiles in one launch: stages of dh along the piece's words, of dW along the rows.
// Every workgroup about its share of all stages, and none of less than 16; dh's splits so that both are done soonest,
// whether each takes its share or the workgroups fill whole rounds of the card (640 x 512 x 30,000 in float32, row tiles
// of 256, a piece: 256 workgroups in 23 splits, 262 in 24; the training pass 654 us and 775).  A part's writing and
// reading costs the card 0.13 us, a sixth of a stage, and counts twice: a card that waits for its last workgroups clocks
// higher (4,096 x 1,024 x 50,000 in whole rounds of four splits 1,504 us, in shares of two 1,484).
Splits both_splits(const Plan& p, int tiles) {
  const long long st_h = (long long)tiles * (kb::kLossM / kb::kLossStage), st_w = up(p.N, kb::kLossStage) / kb::kLossStage;
  const long long n_h = (long long)p.Rd * p.dh_mt, n_w = (long long)tiles * p.dw_ntn;
  const int start = p.bf16 ? 6 : 1;  // a tile's start and end, in stages
  const long long share = std::max<long long>(16, (n_h * st_h + n_w * st_w) / 256);
  Splits s{1, (int)std::max<long long>(1, (st_w + share / 2) / share), LLONG_MAX};
  const long long nw = n_w * s.dw, lw = (st_w + s.dw - 1) / s.dw + start;
  for (int k = 0; k <= 3; ++k) {
    long long sh = k == 0 ? (st_h + share / 2) / share : (256 * k - nw) / n_h;
    sh = std::max<long long>(1, std::min<long long>(std::min(sh, st_h / 16), tiles));
    const long long time = all_done(n_h * sh, (st_h + sh - 1) / sh * p.BN / 256 + start, nw, lw) + n_h * sh / (p.bf16 ? 3 : 18);
    if (time < s.time) s.time = time, s.dh = (int)sh;
  }
  return s;
}

// The products' time with pieces of `piece` word tiles, in stages of a tile of 256 rows: rounds of the logits' tiles, whose
// epilogue takes 5 stages (13 with dlogits), the gradients' launch, and 6 for each launch.  Dlogits of more than 128 MB,
// half the last-level cache, cost 7% (8,192 x 1,024 x 90,000, the gradients: 11 pieces of 128 MB and 44 rounds of the
// logits' tiles 4,182 us, 2 pieces of 704 MB and 44 rounds 4,499, 6 of 236 MB and 48 rounds 4,596); rounds that are not
// full cost more (5,000 x 512 x 32,001: 3 pieces of 110 MB and 12 rounds 800 us, 2 of 165 MB and 10 rounds 611; the loss of
// 1,024 x 1,024 x 60,000 in float32: 3 pieces and 6 rounds 1,065, 2 and 4 rounds 769).
long long pieces_time(const Plan& p, int piece, bool grad, size_t bytes) {
  const int passes = p.bf16 ? 1 : 6;
  auto one = [&](int tiles) {
    const long long P = kb::loss_splits(p.grid, p.R, tiles), rounds = (tiles + P - 1) / P * ((p.R * P + p.grid - 1) / p.grid);
    long long t = rounds * (p.Hk / kb::kLossStage * passes + (grad ? 13 : 5)) * p.BN / 256 + 6;
    if (grad) t += (p.both() ? both_splits(p, tiles).time * passes : (long long)tiles * p.dh_mt) + 6;
    return t;
  };
  const int full = p.vt / piece, rest = p.vt % piece;
  const long long sum = full * one(piece) + (rest > 0 ? one(rest) : 0);
  return grad && bytes > (size_t)128 << 20 ? sum + sum * 7 / 100 : sum;
}

// A batch's tiles, pieces and splits are chosen as for the next step of rows: every number up to 16, multiples of 32 up
// to 2,048, from there 32 steps to each doubling.  Within a step the workspace only grows with the rows.
int plan_rows(int N) {
  if (N <= 16) return N;
  int q = 32;
  while (q * 64 < N) q *= 2;
  return up(N, q);
}
constexpr int kPlanSteps = 16 + 64 + 32 * 11;  // up to KB_LOSS_MAX_N = 2,048 x 2^11
int step_rows(int i) {
  if (i < 16) return i + 1;
  if (i < 80) return 32 * (i - 15);
  const int doubling = (i - 80) / 32;
  return (32 + (i - 80) % 32 + 1) * (64 << doubling);
}

// The plan of a call. `direct`: W is read where it lies; else its pieces are laid out first (float32 in bf16 pieces, odd
// sizes and addresses with zeros filled up).
Plan make_plan(int dtype, int N, int H, int V, int K, bool teacher, bool grad, bool w_aligned) {
  Plan p{};
  p.bf16 = dtype == KB_BF16;
  p.planes = p.bf16 ? 1 : 3;
  p.g_planes = !p.bf16 ? 3 : N <= 128 ? 2 : 1;
  p.z = p.bf16 ? 2 : 4;
  p.N = N, p.H = H, p.V = V, p.K = K;
  // Up to 16 rows of float32 are scored eight after eight: W read where it lies twice instead of laid out in pieces and
  // read six times (16 x 1,024 x 60,000: 116 us and 226, 16 x 256 x 8,000 23 and 31; 24 rows 180 and 227, 34 and 31).
  const bool halves = !p.bf16 && !grad && N > kb::kFewRows && N <= 2 * kb::kFewRows;
  p.few = kb::few_fits(p.bf16, halves ? kb::kFewRows : N, H, V);
  if (p.few) {
    Space s;
    p.grid = kb::few_grid(p.bf16, V);
    if (grad) {
      p.dh_part = s.take((size_t)p.grid * H * kb::few_held(N) * 4);
    } else {
      const size_t rows = std::min(N, kb::kFewRows);  // at a time
      p.stat = s.take(rows * p.grid * sizeof(float2));
      p.sumx = s.take(rows * p.grid * 4);
      p.xt = s.take(rows * K * 4);
    }
    p.bytes = s.at;
    return p;
  }
  p.vt = (V + kb::kLossM - 1) / kb::kLossM;
  p.BN = row_tile(plan_rows(N), p.vt);
  p.WN = p.BN >= 128 ? 2 : 1;
  p.WTM = kb::loss_wtm(p.BN);
  p.WTN = kb::loss_wtn(p.BN);
  p.BNh = p.BN <= 128 ? 64 : H > 128 ? 256 : 128;
  p.Hp = up(H, H > 128 ? 256 : 128);
  p.Hk = up(H, kb::kLossStage);
  p.words0 = p.vt * (kb::kLossM / p.WTM);
  p.nb = p.BN / p.WTN * p.words0 * kb::loss_blocks(p.BN);
  const bool shape = p.bf16 && H % kb::kLossStage == 0 && V % 8 == 0 && V >= kb::kLossM;
  p.direct = shape && w_aligned;
  auto set_rows = [&](int rows) {
    p.N = rows;
    p.R = kb::loss_row_tiles(rows, p.BN);
    p.grid = std::max(p.BN == 32 ? 512 : 256, p.R);
    // two pieces of the dlogits: rows of one tile of dh, the second ones behind all of the first
    p.two = p.g_planes == 2 ? p.R * p.BN : 0;
    p.BNd = p.two == 0 ? p.BN : p.two <= 32 ? 64 : p.two <= 64 ? 128 : 256;
    p.Rd = p.two == 0 ? p.R : 1;
  };
  set_rows(plan_rows(N));
  p.dh_mt = (H + kb::kLossM - 1) / kb::kLossM;
  p.dw_ntn = (H + p.BNh - 1) / p.BNh;

  // Pieces: as many as take the least time of those whose dlogits, and whose part of W that is laid out, have 64 to 256 MB.
  // (W at an odd address where its shape needs no laying out: small pieces of it, so that the workspace need not grow.)
  const size_t w_tile = (size_t)p.Hk * kb::kLossM * 2 * p.planes;
  size_t g_tile = (size_t)p.R * p.BN * kb::kLossM * 2 * p.g_planes;
  auto tiles_of = [&](size_t most) {
    size_t tiles = p.vt;
    if (!p.direct) tiles = std::min(tiles, std::max<size_t>(1, (shape ? most / 16 : most) / w_tile));
    if (grad) tiles = std::min(tiles, std::max<size_t>(1, most / g_tile));
    return (int)tiles;
  };
  const int fewest = (p.vt + tiles_of((size_t)256 << 20) - 1) / tiles_of((size_t)256 << 20);
  const int most = (p.vt + tiles_of((size_t)64 << 20) - 1) / tiles_of((size_t)64 << 20);
  p.piece = (p.vt + fewest - 1) / fewest;
  long long least = LLONG_MAX;
  for (int k = fewest; k <= most && fewest < most; ++k) {
    const int piece = (p.vt + k - 1) / k;
    const long long time = pieces_time(p, piece, grad, piece * ((grad ? g_tile : 0) + (p.direct ? 0 : w_tile)));
    if (time < least) p.piece = piece, least = time;
  }
  p.pieces = (p.vt + p.piece - 1) / p.piece;
  if (grad) {
    const long long st_w = up(p.N, kb::kLossStage) / kb::kLossStage, n_w = (long long)p.piece * p.dw_ntn;
    const long long n_h = (long long)p.Rd * p.dh_mt;
    if (p.both()) {
      const Splits both = both_splits(p, p.piece);
      p.dh_splits = both.dh, p.dw_splits = both.dw;
    } else {
      p.dh_splits = (int)std::max<long long>(1, std::min<long long>((p.BNd == 32 ? 512 : 256) / n_h, p.piece));
      p.dw_splits = (int)std::max<long long>(1, std::min<long long>(256 / n_w, st_w / 8));
    }
    // few stages a tile: a workgroup takes several tiles, the next one's loads under way while it writes one
    p.dw_grid = (int)(n_w * p.dw_splits);
    if (p.dw_splits == 1 && st_w * p.g_planes <= 16) p.dw_grid = std::min(p.dw_grid, p.BNh == 64 ? 512 : 256);
  }

  set_rows(N);
  g_tile = (size_t)p.R * p.BN * kb::kLossM * 2 * p.g_planes;
  Space s;
  p.count = s.take(4);
  p.map = s.take((size_t)N * 4);
  p.inv = s.take((size_t)N * 4);
  if (teacher) {
    p.flag = s.take(N);
    p.token = s.take((size_t)N * K * 4);
    p.part = s.take((size_t)N * K * 4);
    p.known = s.take((size_t)N * 4);
  }
  p.offs = s.take((size_t)p.R * (p.nb + 2) * 2);
  p.items = s.take((size_t)p.R * p.BN * K * sizeof(kb::LossItem));
  p.ph = s.take((size_t)p.planes * p.R * p.BN * p.Hp * 2);
  p.b = s.take((size_t)p.vt * kb::kLossM * 4);
  if (!p.direct) p.wp = s.take(p.piece * w_tile);
  if (!grad) {
    p.stat_piece = (size_t)p.grid * p.BN;
    p.stat = s.take(p.pieces * p.stat_piece * sizeof(float2));
    p.sumx = s.take(p.pieces * p.stat_piece * 4);
    p.xt = s.take((size_t)p.R * p.BN * K * 4);
  } else {
    p.rowp = s.take((size_t)p.R * p.BN * sizeof(float2));
    p.g = s.take(p.two == 0 ? p.piece * g_tile : (size_t)p.piece * kb::kLossM * 2 * p.BNd);
    p.dbp = s.take((size_t)p.R * p.WN * p.vt * kb::kLossM * 4);
    p.dh_part = s.take((size_t)p.dh_splits * p.Rd * p.dh_mt * kb::kLossM * p.BNd * 4);
    if (p.dw_splits > 1) p.dw_part = s.take((size_t)p.dw_splits * p.piece * p.dw_ntn * kb::kLossM * p.BNh * 4);
  }
  p.bytes = s.at;
  return p;
}

kb_status check_sizes(int dtype, int N, int H, int V, int K) {
  if (dtype != KB_F32 && dtype != KB_BF16) return fail(KB_ERR_INVALID_ARG, "unknown dtype %d", dtype);
  if (N < 0 || H < 1 || V < 1) return fail(KB_ERR_INVALID_ARG, "N = %d, H = %d, V = %d", N, H, V);
  if (K < 1 || K > KB_LOSS_MAX_K) return fail(KB_ERR_INVALID_ARG, "K = %d: 1 to %d", K, KB_LOSS_MAX_K);
  if (V > KB_LOSS_MAX_V || H > KB_LOSS_MAX_H || N > KB_LOSS_MAX_N || (long long)N * K > (1 << 30))
    return fail(KB_ERR_UNSUPPORTED, "N = %d, H = %d, V = %d, K = %d: beyond the limits", N, H, V, K);
  return KB_OK;
}

// What the largest of all batches of up to N rows takes, so that a workspace for a program's largest batch serves the
// smaller ones: pieces are chosen by their time, and 5,825 rows of 1,024 x 90,000 have larger ones than 8,192.  The steps
// that were worked out for the last layer are kept, by its sizes alone (all up to 8,192 rows of 1,024 x 90,000: 1.8 ms).
size_t workspace_bytes(int dtype, int N, int H, int V, int K, bool grad) {
  if (check_sizes(dtype, N, H, V, K) != KB_OK || N == 0) return 0;
  static thread_local struct {
    int dtype, H, V, K, grad, n;
    size_t most[kPlanSteps];
  } t = {};
  if (t.n == 0 || t.dtype != dtype || t.H != H || t.V != V || t.K != K || t.grad != grad)
    t.dtype = dtype, t.H = H, t.V = V, t.K = K, t.grad = grad, t.n = 0;
  int i = 0;
  while (step_rows(i) < N) ++i;
  for (; t.n <= i; ++t.n) {
    size_t most = t.n > 0 ? t.most[t.n - 1] : 0;
    for (bool at16 : {true, false}) most = std::max(most, make_plan(dtype, step_rows(t.n), H, V, K, true, grad, at16).bytes);
    t.most[t.n] = most;
  }
  return t.most[i];
}

// What the two losses have in common.
struct Call {
  int dtype, N, H, V, K;
  const void *h, *W;
  const float* b;
  const int32_t* token;
  const float* logit;  // null: targets
  float smoothing, temperature;
  float *loss, *lse;   // forward
  const float *lse_in, *grad;
  void *dh, *dW;
  float* db;
  void* ws;
  size_t ws_bytes;
  hipStream_t st;
};

// smoothing / V.  One that is 0 in float32 is the smallest value instead: it has no weight, but a word of b = -inf that the
// labels name takes the loss to +inf all the same (0 x -inf has no value).
float rest_of(const Call& c) {
  return c.smoothing > 0.f ? std::max(c.smoothing / (float)c.V, FLT_TRUE_MIN) : 0.f;
}

kb_status check_call(const Call& c, const Plan& p) {
  if (!c.h || !c.W || !c.b || !c.token) return fail(KB_ERR_INVALID_ARG, "null h, W, b or words");
  if (!aligned(c.h, p.z) || !aligned(c.W, p.z) || !aligned(c.b, 4) || !aligned(c.token, 4) || !aligned(c.logit, 4))
    return fail(KB_ERR_INVALID_ARG, "h, W, b or words not aligned to their type");
  if (!c.ws) return fail(KB_ERR_WORKSPACE, "workspace is null (%zu bytes needed)", p.bytes);
  if (!aligned(c.ws, 256)) return fail(KB_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (c.ws_bytes < p.bytes) return fail(KB_ERR_WORKSPACE, "workspace %zu bytes < %zu needed", c.ws_bytes, p.bytes);
  return KB_OK;
}

struct Work {
  kb::LossRows rows;
  char* ws;
  template <class X>
  X* at(size_t o) const {
    return reinterpret_cast<X*>(ws + o);
  }
};

#define KB_LAUNCH(what, call)                                                            \
  do {                                                                                   \
    const hipError_t e_ = (call);                                                        \
    if (e_ != hipSuccess) return fail(KB_ERR_HIP, what ": %s", hipGetErrorString(e_));   \
  } while (0)

kb::LossPackWArgs piece_pack(const Call& c, const Plan& p, const Work& w, int t0, int tiles) {
  const int Vc = tiles * kb::kLossM;
  return {c.W, c.H, c.V, t0 * kb::kLossM, Vc, p.Hk, w.at<uint16_t>(p.wp), (size_t)p.Hk * Vc};
}

// Rows that count, their states and entries, the bias and the first piece of W laid out.
kb_status prepare(const Call& c, const Plan& p, Work& w, bool grad) {
  w.ws = static_cast<char*>(c.ws);
  kb::LossRows& r = w.rows;
  r = {c.N, c.H, c.V, c.K, c.token, nullptr, 1.f - c.smoothing, nullptr, w.at<int32_t>(p.map), w.at<int32_t>(p.inv),
       w.at<int32_t>(p.count)};
  if (c.logit) {
    r.token = w.at<int32_t>(p.token);
    r.part = w.at<float>(p.part);
    r.flag = w.at<uint8_t>(p.flag);
    const kb::LossTeacherArgs t{c.N, c.K, c.V, c.token, c.logit, 1.f / c.temperature, w.at<int32_t>(p.token),
                                w.at<float>(p.part), w.at<float>(p.known), w.at<uint8_t>(p.flag)};
    KB_LAUNCH("teacher's rows", kb::launch_loss_teacher(t, c.st));
  }
  kb::LossPackArgs a{};
  a.rows = r;
  a.find_rows = kb::loss_finds_rows(c.N, p.nb);
  if (!a.find_rows) KB_LAUNCH("rows of a loss", kb::launch_loss_rows(r, c.st));
  a.h = c.h;
  a.ph = w.at<uint16_t>(p.ph);
  a.ph_plane = (size_t)p.R * p.BN * p.Hp;
  a.Hp = p.Hp;
  a.BN = p.BN;
  a.tiles = p.R;
  a.nb = p.nb;
  a.words0 = p.words0;
  a.offs = w.at<uint16_t>(p.offs);
  a.items = w.at<kb::LossItem>(p.items);
  a.b = c.b;
  a.bp = w.at<float>(p.b);
  a.Vp = p.vt * kb::kLossM;
  if (!p.direct) a.w = piece_pack(c, p, w, 0, p.piece);
  if (grad) {
    a.lse = c.lse_in;
    a.grad = c.grad;
    a.grad_scale = c.temperature;  // d loss / dx = T^2 (p - q) / T; 1 for targets
    a.rowp = w.at<float2>(p.rowp);
  }
  KB_LAUNCH("states of a loss", kb::launch_loss_pack(p.bf16, a, c.st));
  return KB_OK;
}

// Side W of a piece that starts at word tile t0 and has `tiles` of them: laid out if it has to be.
struct PieceW {
  const uint16_t* p;
  size_t plane;
  int ld, cols, rows;
};
kb_status piece_w(const Call& c, const Plan& p, const Work& w, int t0, int tiles, PieceW& out) {
  const int v0 = t0 * kb::kLossM;
  if (p.direct) {
    out = {static_cast<const uint16_t*>(c.W) + v0, 0, c.V, c.V - v0, c.H};
    return KB_OK;
  }
  const kb::LossPackWArgs a = piece_pack(c, p, w, t0, tiles);
  if (t0 > 0) KB_LAUNCH("weights of a loss", kb::launch_loss_pack_w(p.bf16, a, c.st));
  out = {a.out, a.plane, a.Vc, a.Vc, p.Hk};
  return KB_OK;
}

kb::LossLogitsArgs logits_args(const Call& c, const Plan& p, const Work& w, const PieceW& pw, int t0, int tiles) {
  kb::LossLogitsArgs a{};
  a.A = pw.p;
  a.a_plane = pw.plane;
  a.lda = pw.ld;
  a.a_cols = pw.cols;
  a.ph = w.at<uint16_t>(p.ph);
  a.ph_plane = (size_t)p.R * p.BN * p.Hp;
  a.Hp = p.Hp;
  a.Hk = p.Hk;
  a.b = w.at<float>(p.b) + (size_t)t0 * kb::kLossM;
  a.words = c.V - t0 * kb::kLossM;
  a.vt = tiles;
  a.count = w.rows.count;
  a.grid = p.grid;
  a.scale = kb::kL2E / c.temperature;
  a.offs = w.at<uint16_t>(p.offs);
  a.items = w.at<kb::LossItem>(p.items);
  a.nb = p.nb;
  a.words0 = p.words0;
  a.wt0 = t0 * (kb::kLossM / p.WTM);
  a.K = c.K;
  a.rest = rest_of(c);
  return a;
}

kb::LossFewArgs few_args(const Call& c, const Plan& p) {
  kb::LossFewArgs a{};
  a.N = c.N, a.H = c.H, a.V = c.V, a.K = c.K;
  a.h = c.h, a.W = c.W, a.b = c.b;
  a.token = c.token, a.logit = c.logit;
  a.inv_t = 1.f / c.temperature;
  a.t2 = c.temperature * c.temperature;
  a.target_part = 1.f - c.smoothing;
  a.rest = rest_of(c);
  a.grid = p.grid;
  return a;
}

kb_status few_forward(const Call& c, const Plan& p) {
  char* ws = static_cast<char*>(c.ws);
  kb::LossFewArgs a = few_args(c, p);
  a.stat = reinterpret_cast<float2*>(ws + p.stat);
  a.sumx = reinterpret_cast<float*>(ws + p.sumx);
  a.xt = reinterpret_cast<float*>(ws + p.xt);
  for (int r0 = 0; r0 < c.N; r0 += kb::kFewRows) {
    a.N = std::min(c.N - r0, kb::kFewRows);
    a.h = static_cast<const char*>(c.h) + (size_t)r0 * c.H * p.z;
    a.token = c.token + (size_t)r0 * c.K;
    a.logit = c.logit ? c.logit + (size_t)r0 * c.K : nullptr;
    a.loss = c.loss + r0;
    a.lse_out = c.lse + r0;
    KB_LAUNCH("logits of a loss", kb::launch_loss_few(p.bf16, false, a, c.st));
    KB_LAUNCH("losses", kb::launch_loss_few_finish(a, c.st));
  }
  return ok();
}

kb_status few_gradient(const Call& c, const Plan& p) {
  kb::LossFewArgs a = few_args(c, p);
  a.lse = c.lse_in;
  a.grad = c.grad;
  a.grad_scale = c.temperature;
  a.dh_part = c.dh ? reinterpret_cast<float*>(static_cast<char*>(c.ws) + p.dh_part) : nullptr;
  a.dh = c.dh;
  a.dW = c.dW;
  a.db = c.db;
  KB_LAUNCH("gradients of a loss", kb::launch_loss_few(p.bf16, true, a, c.st));
  if (c.dh) KB_LAUNCH("gradient of the states", kb::launch_loss_few_join(p.bf16, a, c.st));
  return ok();
}

kb_status forward(const Call& c) {
  const Plan p = make_plan(c.dtype, c.N, c.H, c.V, c.K, c.logit != nullptr, false, aligned(c.W, 16));
  kb_status s = check_call(c, p);
  if (s != KB_OK) return s;
  if (!c.loss || !c.lse) return fail(KB_ERR_INVALID_ARG, "null loss or lse");
  if (!aligned(c.loss, 4) || !aligned(c.lse, 4)) return fail(KB_ERR_INVALID_ARG, "loss or lse not aligned to their type");
  if (p.few) return few_forward(c, p);
  Work w;
  if ((s = prepare(c, p, w, false)) != KB_OK) return s;
  const bool smooth = c.smoothing > 0.f;
  for (int i = 0; i < p.pieces; ++i) {
    const int t0 = i * p.piece, tiles = std::min(p.piece, p.vt - t0);
    PieceW pw;
    if ((s = piece_w(c, p, w, t0, tiles, pw)) != KB_OK) return s;
    kb::LossLogitsArgs a = logits_args(c, p, w, pw, t0, tiles);
    a.stat = w.at<float2>(p.stat) + i * p.stat_piece;
    a.sumx = smooth ? w.at<float>(p.sumx) + i * p.stat_piece : nullptr;
    a.xt = w.at<float>(p.xt);
    KB_LAUNCH("logits of a loss", p.bf16 ? kb::launch_loss_logits_bf16(0, p.BN, a, p.grid, c.st)
                                         : kb::launch_loss_logits_f32(0, p.BN, a, p.grid, c.st));
  }
  kb::LossFinishArgs f{};
  f.rows = w.rows;
  f.stat = w.at<float2>(p.stat);
  f.sumx = smooth ? w.at<float>(p.sumx) : nullptr;
  f.stat_piece = p.stat_piece;
  f.pieces = p.pieces;
  f.vt_piece = p.piece;
  f.vt_last = p.vt - (p.pieces - 1) * p.piece;
  f.grid = p.grid;
  f.BN = p.BN;
  f.xt = w.at<float>(p.xt);
  f.known = c.logit ? w.at<float>(p.known) : nullptr;
  f.scale = kb::kL2E / c.temperature;
  f.inv_t = 1.f / c.temperature;
  f.rest = rest_of(c);
  f.t2 = c.temperature * c.temperature;
  f.loss = c.loss;
  f.lse = c.lse;
  KB_LAUNCH("losses", kb::launch_loss_finish(f, c.st));
  return ok();
}

kb_status gradient(const Call& c) {
  const Plan p = make_plan(c.dtype, c.N, c.H, c.V, c.K, c.logit != nullptr, true, aligned(c.W, 16));
  kb_status s = check_call(c, p);
  if (s != KB_OK) return s;
  if (!c.lse_in || !c.grad) return fail(KB_ERR_INVALID_ARG, "null lse or grad");
  if (!aligned(c.lse_in, 4) || !aligned(c.grad, 4))
    return fail(KB_ERR_INVALID_ARG, "lse or grad not aligned to their type");
  if (p.few) return few_gradient(c, p);
  Work w;
  if ((s = prepare(c, p, w, true)) != KB_OK) return s;
  const size_t rows = (size_t)p.R * p.BN;
  const int Vp = p.vt * kb::kLossM;
  for (int i = 0; i < p.pieces; ++i) {
    const int t0 = i * p.piece, tiles = std::min(p.piece, p.vt - t0), Vc = tiles * kb::kLossM;
    PieceW pw;
    if ((s = piece_w(c, p, w, t0, tiles, pw)) != KB_OK) return s;
    kb::LossLogitsArgs a = logits_args(c, p, w, pw, t0, tiles);
    if (!p.bf16) a.scale = 1.f / c.temperature;  // the difference from lse is taken first
    a.rowp = w.at<float2>(p.rowp);
    a.g = w.at<uint16_t>(p.g);
    a.g_plane = rows * Vc;
    a.gld = Vc;
    a.dbp = c.db ? w.at<float>(p.dbp) : nullptr;
    a.db_ld = Vp;
    a.db0 = t0 * kb::kLossM;
    KB_LAUNCH("logits of a loss", p.bf16 ? kb::launch_loss_logits_bf16(p.g_planes, p.BN, a, p.grid, c.st)
                                         : kb::launch_loss_logits_f32(p.g_planes, p.BN, a, p.grid, c.st));
    kb::LossGradArgs g{};
    g.W = pw.p;
    g.w_plane = pw.plane;
    g.ldw = pw.ld;
    g.w_rows = pw.rows;
    g.ph = a.ph;
    g.ph_plane = a.ph_plane;
    g.Hp = p.Hp;
    g.H = c.H;
    g.g = a.g;
    g.g_plane = a.g_plane;
    g.gld = Vc;
    g.vt = tiles;
    g.N = c.N;
    g.count = w.rows.count;
    g.V = c.V;
    kb::LossGradArgs gh = g, gw = g;
    gh.words = pw.cols;
    gh.splits = p.dh_splits;
    gh.mt = p.dh_mt;
    gh.two = p.two;
    gh.part = w.at<float>(p.dh_part);
    gh.add = i > 0;
    gw.words = c.V - t0 * kb::kLossM;
    gw.splits = p.dw_splits;
    gw.mt = tiles;
    gw.ntn = p.dw_ntn;
    gw.grid = std::min(p.dw_grid, gw.splits * gw.mt * gw.ntn);
    gw.part = p.dw_splits > 1 ? w.at<float>(p.dw_part) : nullptr;
    gw.out = static_cast<char*>(c.dW) + (size_t)t0 * kb::kLossM * p.z;
    if (c.dh && c.dW && p.both()) {
      KB_LAUNCH("gradients of a loss",
                p.bf16 ? kb::launch_loss_both_bf16(p.BN, gh, gw, c.st) : kb::launch_loss_both_f32(p.BN, gh, gw, c.st));
    } else {
      if (c.dh)
        KB_LAUNCH("gradient of the states",
                  p.bf16 ? kb::launch_loss_dh_bf16(p.BNd, gh, c.st) : kb::launch_loss_dh_f32(p.BNd, gh, c.st));
      if (c.dW)
        KB_LAUNCH("gradient of the weights",
                  p.bf16 ? kb::launch_loss_dw_bf16(p.g_planes, p.BNh, gw, c.st) : kb::launch_loss_dw_f32(p.g_planes, p.BNh, gw, c.st));
    }
    if (c.dW && gw.part) {
      const kb::LossJoinArgs j{gw.part, p.dw_splits, tiles, p.dw_ntn, p.BNh, c.H, std::min(gw.words, Vc), 0, nullptr,
                               nullptr, gw.out, c.V, 0};
      KB_LAUNCH("gradient of the weights", kb::launch_loss_join(p.bf16, j, kb::LossJoinMore{}, c.st));
    }
  }
  const kb::LossBiasArgs db{w.at<float>(p.dbp), p.WN, p.BN, Vp, w.rows.count, c.V, c.db};
  if (c.dh) {
    const kb::LossJoinArgs j{w.at<float>(p.dh_part), p.dh_splits, p.dh_mt, p.Rd, p.BNd, c.N, c.H, 1, w.rows.map,
                             w.rows.count, c.dh, c.H, p.two};
    KB_LAUNCH("gradient of the states", kb::launch_loss_join(p.bf16, j, kb::LossJoinMore{w.rows.inv, c.N, db, 0, 0}, c.st));
  } else if (c.db) {
    KB_LAUNCH("gradient of the bias", kb::launch_loss_db(db, c.st));
  }
  return ok();
}

kb_status run_gradient(const Call& c) {
  const int z = c.dtype == KB_BF16 ? 2 : 4;
  if (!c.dh && !c.dW && !c.db) return fail(KB_ERR_INVALID_ARG, "no gradient is asked for");
  if (!aligned(c.dh, z) || !aligned(c.dW, z) || !aligned(c.db, 4))
    return fail(KB_ERR_INVALID_ARG, "dh, dW or db not aligned to their type");
  if (c.N > 0) return gradient(c);
  if (c.dW) KB_LAUNCH("gradient of the weights", kb::launch_loss_zero(c.dW, (size_t)c.H * c.V * z, c.st));
  if (c.db) KB_LAUNCH("gradient of the bias", kb::launch_loss_zero(c.db, (size_t)c.V * 4, c.st));
  return ok();
}

kb_status check_smoothing(float s) {
  if (!(s >= 0.f && s < 1.f)) return fail(KB_ERR_INVALID_ARG, "smoothing = %g: 0 <= smoothing < 1", (double)s);
  return KB_OK;
}

kb_status check_temperature(float t) {
  // T^2 and 1 / T are finite and normal
  if (!(t >= 1e-6f && t <= 1e6f)) return fail(KB_ERR_INVALID_ARG, "temperature = %g: 1e-6 to 1e6", (double)t);
  return KB_OK;
}

}  // namespace

extern "C" {

size_t kb_loss_workspace_bytes(int dtype, int N, int H, int V, int K) { return workspace_bytes(dtype, N, H, V, K, false); }

size_t kb_loss_grad_workspace_bytes(int dtype, int N, int H, int V, int K) {
  return workspace_bytes(dtype, N, H, V, K, true);
}

kb_status kb_cross_entropy(int dtype, int N, int H, int V, const void* h, const void* W, const float* b,
                           const int32_t* target, float smoothing, float* loss, float* lse, void* workspace,
                           size_t workspace_bytes, void* stream) {
  kb_status s = check_sizes(dtype, N, H, V, 1);
  if (s != KB_OK || (s = check_smoothing(smoothing)) != KB_OK) return s;
  if (N == 0) return ok();
  Call c{dtype, N, H, V, 1, h, W, b, target};
  c.smoothing = smoothing;
  c.temperature = 1.f;
  c.loss = loss;
  c.lse = lse;
  c.ws = workspace;
  c.ws_bytes = workspace_bytes;
  c.st = reinterpret_cast<hipStream_t>(stream);
  return forward(c);
}

kb_status kb_cross_entropy_grad(int dtype, int N, int H, int V, const void* h, const void* W, const float* b,
                                const int32_t* target, float smoothing, const float* lse, const float* grad, void* dh,
                                void* dW, float* db, void* workspace, size_t workspace_bytes, void* stream) {
  kb_status s = check_sizes(dtype, N, H, V, 1);
  if (s != KB_OK || (s = check_smoothing(smoothing)) != KB_OK) return s;
  Call c{dtype, N, H, V, 1, h, W, b, target};
  c.smoothing = smoothing;
  c.temperature = 1.f;
  c.lse_in = lse;
  c.grad = grad;
  c.dh = dh;
  c.dW = dW;
  c.db = db;
  c.ws = workspace;
  c.ws_bytes = workspace_bytes;
  c.st = reinterpret_cast<hipStream_t>(stream);
  return run_gradient(c);
}

kb_status kb_distill(int dtype, int N, int H, int V, int K, const void* h, const void* W, const float* b,
                     const int32_t* token, const float* logit, float temperature, float* loss, float* lse,
                     void* workspace, size_t workspace_bytes, void* stream) {
  kb_status s = check_sizes(dtype, N, H, V, K);
  if (s != KB_OK || (s = check_temperature(temperature)) != KB_OK) return s;
  if (N == 0) return ok();
  if (!logit) return fail(KB_ERR_INVALID_ARG, "null logit");
  Call c{dtype, N, H, V, K, h, W, b, token, logit};
  c.temperature = temperature;
  c.loss = loss;
  c.lse = lse;
  c.ws = workspace;
  c.ws_bytes = workspace_bytes;
  c.st = reinterpret_cast<hipStream_t>(stream);
  return forward(c);
}

kb_status kb_distill_grad(int dtype, int N, int H, int V, int K, const void* h, const void* W, const float* b,
                          const int32_t* token, const float* logit, float temperature, const float* lse,
                          const float* grad, void* dh, void* dW, float* db, void* workspace, size_t workspace_bytes,
                          void* stream) {
  kb_status s = check_sizes(dtype, N, H, V, K);
  if (s != KB_OK || (s = check_temperature(temperature)) != KB_OK) return s;
  if (N > 0 && !logit) return fail(KB_ERR_INVALID_ARG, "null logit");
  Call c{dtype, N, H, V, K, h, W, b, token, logit};
  c.temperature = temperature;
  c.lse_in = lse;
  c.grad = grad;
  c.dh = dh;
  c.dW = dW;
  c.db = db;
  c.ws = workspace;
  c.ws_bytes = workspace_bytes;
  c.st = reinterpret_cast<hipStream_t>(stream);
  return run_gradient(c);
}

}  // extern "C"
