// The output layer's losses: argument blocks that the host side (loss_abi.hip)
// and the kernels share, and the tiles of the matrix products.
#pragma once

#include "kb_common.hpp"

namespace kb {

// A tile of a product: 256 x BN, four waves of MB x NB blocks of 32 x 32.  The M side lies along a lane's
// accumulators (four neighbours each), the N side along the lanes.
template <int MB_, int NB_, int WM_, int WN_>
struct LossTile {
  static constexpr int MB = MB_, NB = NB_, WM = WM_, WN = WN_;
  static constexpr int BM = 32 * MB * WM, BN = 32 * NB * WN;
  static constexpr int WTM = 32 * MB, WTN = 32 * NB;  // a wave's part of the tile
  static_assert(WM * WN == 4 && BM == 256, "four waves, 256 on the M side");
};
using LossT256 = LossTile<4, 4, 2, 2>;
using LossT192 = LossTile<4, 3, 2, 2>;
using LossT128 = LossTile<4, 2, 2, 2>;
using LossT64 = LossTile<2, 2, 4, 1>;
using LossT32 = LossTile<2, 1, 4, 1>;

constexpr int kLossM = 256;      // words (or states) of a tile's M side
constexpr int kLossStage = 32;   // contraction steps of a pipeline stage
constexpr int kLossMaxV = 1 << 18;
constexpr int kLossMaxK = 128;

// The wave's part of a tile with BN rows, for the lists of entries: its extent, and its blocks of 32 x 32 (a multiple of
// two, and at most sixteen).
__host__ __device__ inline int loss_wtm(int BN) { return BN >= 128 ? 128 : 64; }
__host__ __device__ inline int loss_wtn(int BN) { return BN >= 128 ? BN / 2 : BN; }
__host__ __device__ inline int loss_blocks(int BN) { return loss_wtm(BN) / 32 * (loss_wtn(BN) / 32); }

// Rows that count lie packed: `map` has the original row of each packed one, `inv` the packed row of each
// original one or -1, *count how many there are.
struct LossRows {
  int N, H, V, K;          // K: entries of a row (1: its target)
  const int32_t* token;    // N x K, outside [0, V): no entry
  const float* part;       // N x K: the part of the entry's word in the row's distribution; null: 1 - smoothing
  float target_part;       // 1 - smoothing
  const uint8_t* flag;     // N: the row has an entry (distillation); null: by its target
  int32_t* map;
  int32_t* inv;
  int32_t* count;
};

// An entry in the list of its block: where a wave holds its logit, and what goes with it.
struct alignas(8) LossItem {
  int32_t code;     // register << 8 | lane
  int32_t payload;  // forward: packed row * K + entry; gradient: its part of the row's distribution, as float32 bits
};

struct LossTeacherArgs {
  int N, K, V;
  const int32_t* token;
  const float* logit;
  float inv_t;
  int32_t* out_token;  // N x K: the entry's word, -1 where there is none or an earlier entry has the same word
  float* part;         // N x K: softmax over the row's words of logit / T
  float* known;        // N: sum of part * ln(part)
  uint8_t* flag;       // N
};

// A piece of W: words v0 .. v0 + Vc - 1 (those from V on as zeros), Hk rows (those from H on zeros).
struct LossPackWArgs {
  const void* W;
  int H, V, v0, Vc, Hk;
  uint16_t* out;       // planes x Hk x Vc bf16; null: none
  size_t plane;
};

struct LossPackArgs {
  LossRows rows;
  int find_rows;       // the map has not been made: every workgroup that needs it finds the rows that count by itself
  const void* h;
  uint16_t* ph;        // planes x rows x Hp bf16
  size_t ph_plane;     // values from one plane to the next
  int Hp, BN;
  // lists of entries by block of the waves' tiles
  int tiles, nb;       // row tiles (most), blocks of each
  int words0;          // wave tiles along the words
  uint16_t* offs;      // tiles x (nb + 2)
  LossItem* items;     // tiles x BN x K
  // gradient: what the rows' logits are turned into gradients with
  const float* lse;
  const float* grad;
  float grad_scale;
  float2* rowp;        // (log-sum-exp, gradient) of each packed row; null: forward
  const float* b;
  float* bp;           // the bias, -inf for the words that fill the last tile up
  int Vp;
  LossPackWArgs w;     // the first piece's
  int states_wg, bias_wg, w_wg;  // workgroups of each kind behind the `tiles` that make lists
};

// The logits' product: A words x states (states apart by lda), B packed rows.
struct LossLogitsArgs {
  const uint16_t* A;
  size_t a_plane;
  int lda, a_cols;       // columns there are (clamped to)
  const uint16_t* ph;
  size_t ph_plane;
  int Hp, Hk;            // row length of ph; states, a multiple of 32
  const float* b;        // bias of the piece's first word on
  int words;             // words of the piece that exist
  int vt;                // its word tiles
  const int32_t* count;
  int grid;              // workgroups that share the tiles
  float scale;           // log2(e) / T
  const uint16_t* offs;  // lists of entries
  const LossItem* items;
  int nb, words0, wt0;   // blocks of a row tile; wave tiles along the words, and of the words before this piece
  int K;
  // forward
  float2* stat;          // [packed row][split] (max, sum) of the piece
  float* sumx;           // the same: sum of logits; null: not wanted
  float* xt;             // packed row x K: the entries' logits
  // gradient
  const float2* rowp;
  float rest;            // smoothing / V
  uint16_t* g;           // planes x rows x gld
  size_t g_plane;
  int gld;
  float* dbp;            // (row tile x wave row) x db_ld: sums over the wave's rows; null: not wanted
  int db_ld, db0;
};

// Gradients: C = A B over a long axis.
struct LossGradArgs {
  const uint16_t* W;     // dh: states x words (words contiguous, ldw apart)
  size_t w_plane;
  int ldw, w_rows, words;
  const uint16_t* ph;    // dW: packed rows x states
  size_t ph_plane;
  int Hp, H;
  const uint16_t* g;     // packed rows x words of the piece
  size_t g_plane;
  int gld, vt;           // words of the piece with its last tile filled up, word tiles
  int N;
  const int32_t* count;
  int splits;            // of the long axis
  int mt, ntn;           // tiles along M and N (dh: states, rows; dW: words, states)
  int two;               // dh: the dlogits' second pieces are rows this far behind the first, all in one row tile; 0: none
  int grid;              // dW: workgroups
  float* part;           // [split][tile] in the order of the registers; null (dW): written to out
  int add;               // dh: added to what the pieces before have left
  void* out;             // dW
  int V;                 // row length of dW
};

struct LossJoinArgs {
  const float* part;
  int splits, mt, ntn, BNt;   // BNt: the tile's N side
  int rows, cols;             // extent of N and M sides
  int is_dh;
  const int32_t* map;
  const int32_t* count;
  void* out;
  int ld;
  int two;                    // dh: a row's second piece lies this many rows behind it; 0: there is one piece
};

// The bias' gradient from dbp (wave_rows rows for each row tile of BN).
struct LossBiasArgs {
  const float* dbp;
  int wave_rows, BN, ld;
  const int32_t* count;
  int V;
  float* db;                  // null: not wanted
};

// What the join of dh does besides: rows that do not count (of N; inv < 0), and the bias.
struct LossJoinMore {
  const int32_t* inv;         // null: none
  int N;
  LossBiasArgs db;
  int zero_wg, db_wg;         // workgroups (set by the launch)
};

struct LossFinishArgs {
  LossRows rows;
  const float2* stat;
  const float* sumx;
  size_t stat_piece;      // values of stat and sumx from one piece's to the next's
  int pieces;
  int vt_piece, vt_last;  // word tiles of each piece but the last, and of the last
  int grid, BN;
  const float* xt;
  const float* known;
  float scale, inv_t, rest, t2;
  float* loss;
  float* lse;
};

// A few rows (loss_few.hip).
constexpr int kFewRows = 8;
constexpr int kFewGrid = 512;   // workgroups at most

struct LossFewArgs {
  int N, H, V, K;
  const void* h;
  const void* W;
  const float* b;
  const int32_t* token;   // N x K: targets (K = 1) or the teacher's words
  const float* logit;     // the teacher's logits; null: targets
  float inv_t, t2;        // 1 / T, T^2
  float target_part;      // 1 - smoothing
  float rest;             // smoothing / V
  int grid;
  // forward
  float2* stat;           // row x grid: (max, sum)
  float* sumx;            // row x grid
  float* xt;              // row x K: the entries' logits
  float* loss;
  float* lse_out;
  // gradient
  const float* lse;
  const float* grad;
  float grad_scale;
  float* dh_part;         // grid x H x rows held; null: not wanted
  void* dh;
  void* dW;
  float* db;
};
int few_held(int N);                       // rows that a workgroup holds for N
bool few_fits(bool bf16, int N, int H, int V);  // the few rows' kernels take this size
int few_grid(bool bf16, int V);
hipError_t launch_loss_few(bool bf16, bool grad, const LossFewArgs& a, hipStream_t st);
hipError_t launch_loss_few_finish(const LossFewArgs& a, hipStream_t st);
hipError_t launch_loss_few_join(bool bf16, const LossFewArgs& a, hipStream_t st);

hipError_t launch_loss_teacher(const LossTeacherArgs& a, hipStream_t st);
hipError_t launch_loss_rows(const LossRows& a, hipStream_t st);
bool loss_finds_rows(int N, int nb);  // launch_loss_pack can do without launch_loss_rows
hipError_t launch_loss_pack(bool bf16, LossPackArgs a, hipStream_t st);
hipError_t launch_loss_pack_w(bool bf16, const LossPackWArgs& a, hipStream_t st);
hipError_t launch_loss_finish(const LossFinishArgs& a, hipStream_t st);
hipError_t launch_loss_join(bool bf16, const LossJoinArgs& a, LossJoinMore more, hipStream_t st);
hipError_t launch_loss_zero(void* p, size_t bytes, hipStream_t st);
hipError_t launch_loss_db(const LossBiasArgs& a, hipStream_t st);

// How the row tiles that exist share the workgroups: the same on the host's sizes, in the kernels and in the join.
__host__ __device__ inline int loss_row_tiles(int rows, int BN) { return (rows + BN - 1) / BN; }
__host__ __device__ inline int loss_splits(int grid, int row_tiles, int word_tiles) {
  int p = row_tiles > 0 ? grid / row_tiles : 1;
  p = p < 1 ? 1 : p;
  return p < word_tiles ? p : word_tiles;
}

}  // namespace kb
