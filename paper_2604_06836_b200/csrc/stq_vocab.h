// Internal interface between the host layer of the vocabulary cross entropy (stq_vocab_api.cu) and its kernels.
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace stq {

// Rows are compact: only tokens that count have one, in the tokens' order (`count` of them, known on the device alone).
// Without compaction every token has a row, and those that do not count get zeros.
struct VocabRows {
  const void* x;              // bf16 hidden states, a row each
  size_t ldx;
  uint32_t rows;              // rows of x that exist
  uint32_t most;              // rows at most, a multiple of 256 (of 128 for a single tile)
  const uint32_t* count;      // on the device, or null: `rows`
  const uint32_t* token;      // row -> token, or null: the same
  const int32_t* row;         // token -> row or -1, or null
  const float* scale;         // gradients: what they are multiplied with at the end (GatherArgs), on the device
};

// What the products of hidden states and the matrix need.
struct VocabArgs {
  VocabRows r;
  const void* w;              // bf16 [v][d]
  size_t ldw;
  const float* bias;          // [v], or null
  uint32_t v, d;
  const int64_t* target;      // of a token
  int64_t ignore;
  uint32_t t;
  int device;
};

// ---- rows (stq_vocab_scores.cu) ----------------------------------------------------------------------------------
// Tokens that count -> compact rows; rows up to `most` behind them are zero.
struct GatherArgs {
  const void* x;
  size_t ldx;
  uint32_t t, d, most;
  const int64_t* target;
  int64_t ignore;
  void* out;
  size_t ldo;
  uint32_t* count;
  uint32_t* token;
  int32_t* row;
  // Gradients: the largest |dloss| of the tokens that count (1 if that is 0 or infinite).  The gradients of the logits are formed for
  // dloss / scale: for a mean over tokens that is 1, and the 1 of p - 1 then has no rounding in bf16.
  const float* dloss;
  float* scale;
  bool aligned;               // (set by the launch) rows are whole 16-byte pieces
};
cudaError_t launch_vocab_gather(const GatherArgs& a, cudaStream_t stream);

// Tiles of the products: `cg` CTAs share 128 * cg rows and `wide` entries of the vocabulary.  The loss (planes = 0) takes any width that
// the matrix units do, the gradients whole panels (below), those in three parts narrow ones.  cost, if wanted: the time in clock cycles.
// chunk: how many stages of 64 columns are added up in the matrix unit.  It goes by the number of tokens alone: loss and gradients then round
// a logit in the same way, and a target's exp(z - lse) - 1 is as exact as lse.
struct VocabShape {
  int cg;
  uint32_t wide;
  uint32_t chunk;
};
VocabShape vocab_shape(uint32_t rows, uint32_t v, uint32_t d, int planes, int sms, double* cost = nullptr);

// Maxima and sums of exp of each row over parts of the vocabulary: part[i][row] for i < vocab_parts(), pitch `most`.
uint32_t vocab_parts(const VocabArgs& a, VocabShape s, uint32_t most, int sms);
// How many parts a tile makes of each of its rows, where there are more than 128 tokens.
uint32_t vocab_parts_of_tile(uint32_t d);
// (most: the one that the parts were counted for.)  chosen[row]: the logit of the row's target, if that is in the vocabulary.
cudaError_t launch_vocab_parts(const VocabArgs& a, VocabShape s, uint32_t most, float2* part, float* chosen, int sms, int* err,
                               cudaStream_t stream);
// loss and lse of all tokens from these.
cudaError_t launch_vocab_finish(const VocabArgs& a, const float2* part, uint32_t parts, const float* chosen, float* loss, float* lse, int sms,
                                cudaStream_t stream);

// Gradients of the logits of entries [v0, v1), divided by scale: `planes` bf16 numbers (1 or 3) whose sum they are.  They lie in panels
// of 64 entries, p[plane][(v - v0) / 64][row][(v - v0) % 64], `panels` to a plane and `most` rows to a panel, so that every box that is
// copied (64 entries, any rows) is one range of memory.  dbias: sums over 32 rows each, [most / 32] of pitch ldb, or null.
struct VocabGradOut {
  void* p;
  uint32_t panels;
  int planes;
  float* dbias;
  size_t ldb;
  const float* lse;
  const float* dloss;
};
cudaError_t launch_vocab_dlogits(const VocabArgs& a, VocabShape s, uint32_t v0, uint32_t v1, const VocabGradOut& o, int sms, int* err,
                                 cudaStream_t stream);

// ---- gradients (stq_vocab_grad.cu) ---------------------------------------------------------------------------------
// dw[v0 + i][:] = scale * sum over rows of p[row][i] x[row][:].  part: vocab_dw_partial() floats.
struct VocabDw {
  VocabRows r;
  const void* p;
  uint32_t panels;
  uint32_t cols, d;           // v1 - v0
  void* dw;                   // row v0
  size_t lddw;
  bool f32;
  int device;
};
size_t vocab_dw_partial(const VocabDw& a, int sms);
double vocab_dw_cost(const VocabDw& a, int sms);      // in clock cycles
cudaError_t launch_vocab_dw(const VocabDw& a, float* part, int sms, int* err, cudaStream_t stream);
// Adds shares of tiles up, if the plan has any.
cudaError_t launch_vocab_dw_join(const VocabDw& a, const float* part, int sms, cudaStream_t stream, int* launches);

// plane[row][:] (+)= sum over [v0, v0 + cols) of p[row][i] w[v0 + i][:], or segments of that sum (stq_vocab_ranges.h), a tile to each.
// All pieces but the last are equally long (`first` columns).
struct VocabDx {
  VocabRows r;
  const void* p;
  uint32_t panels;
  const void* w;              // row v0
  size_t ldw;
  uint32_t cols, d, first;
  bool begin;                 // the first piece
  bool beside;                // launched right after dw of the same piece
  float *plane, *segments;
  size_t ldd;                 // columns of the plane, a multiple of 32
  int device;
};
void vocab_dx_space(uint32_t most, uint32_t d, size_t ldd, int sms, size_t* plane, size_t* segments);      // floats that suffice
cudaError_t launch_vocab_dx(const VocabDx& a, int sms, int* err, cudaStream_t stream);
// dbias of `cols` entries from the sums over 32 rows each.
struct VocabDbias {
  const float* part;
  size_t ldb;
  uint32_t cols;
  float* out;
};
cudaError_t launch_vocab_dbias(const VocabDbias& a, const VocabRows& r, cudaStream_t stream);
// dx of all tokens (zero for those that do not count): scale times the plane or the sum of the segments.  With db, dbias too.
cudaError_t launch_vocab_dx_finish(const VocabDx& a, uint32_t t, void* dx, size_t lddx, const VocabDbias* db, int sms, cudaStream_t stream);

}  // namespace stq
