// Internal interface between the host side of the sequence operators (ops_api.hip) and their gfx950
// kernels.  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/evconv_ops.h"

namespace evk {

// Threads of one launch, at most: HIP counts them in 32 bits.
constexpr int64_t kMostThreads = (1ll << 32) - 1;

// Text of evconv_last_error(NULL) (evconv_api.hip).
void set_call_error(const char* text) noexcept;

// ---- gated delta rule ---------------------------------------------------------------------------
constexpr int kDeltaChunk = 64;       // tokens of a chunk
constexpr int kDeltaShortRagged = 4;  // sequences of up to so many tokens go token by token, at least, where lengths are their own (ops_api.hip)

struct DeltaParams {
  evconv_delta_args a;
  int share;        // value heads per key head
  int len;          // tokens of every sequence, or -1: seq_offsets
  int short_len;    // sequences of up to so many tokens go token by token
  int slots_total;  // chunk slots that the sequences have together, at most
  int dkp;          // d_k, rounded up to whole 32
  int vec;          // q, k rows may be read in 16-byte loads
  int vec_v;        // v rows too, and o rows written in 8-byte stores
  // workspace
  char* frag_k;     // per chunk slot and key head: K, Q and K' as matrix-core operands
  char* frag_t;     // per chunk slot and value head: T and P
  float* scal;      // per chunk slot and value head: kDeltaScalars
  int* slot_seq;    // per chunk slot: the sequence whose it is (seq_offsets only; anything where it is nobody's)
  int segs, seg_chunks;   // segments of a sequence (1: whole), chunks of one
  float *trans, *start0;  // what segments do to the state, the first one's start
};
// Sizes in the workspace, per chunk slot and head.
size_t delta_frag_k_bytes(int dtype, int dkp);
size_t delta_frag_t_bytes(int dtype);
constexpr int kDeltaScalars = 512;  // four factors of every token, the decay; up to whole 1 KB
// Threads of the largest launch of each way.
int64_t delta_steps_threads(const DeltaParams& p);
int64_t delta_chunks_threads(const DeltaParams& p);
int64_t delta_fused_threads(const DeltaParams& p);
void launch_delta_steps(const DeltaParams& p, hipStream_t s);
void launch_delta_chunks(const DeltaParams& p, hipStream_t s);
// chunks in one launch
bool delta_fused_supported(const DeltaParams& p);
// segments of long sequences, of either way
size_t plan_delta_segments(DeltaParams& p, bool fused);  // sets segs and seg_chunks; bytes of workspace
void place_delta_segments(DeltaParams& p, char* workspace);
void launch_delta_join(const DeltaParams& p, hipStream_t s);
void launch_delta_fused(const DeltaParams& p, hipStream_t s);

// ---- norms around a block, rows of 8-bit integers ------------------------------------------------
// vectors of eight that a row takes (the lanes of a group that it does not fill among them), at most
constexpr int kNormVectors = 2048;
int block_norm_vectors(const evconv_norm_args& a);
void launch_block_norm(const evconv_norm_args& a, bool vec, hipStream_t s);

// ---- product in 8-bit integers -------------------------------------------------------------------
void launch_quant_matmul(const evconv_quant_args& a, hipStream_t s);

// ---- paged cache ---------------------------------------------------------------------------------
// Channels of a head in the cache.
constexpr int cache_channels(int d) { return d <= 32 ? 32 : d <= 64 ? 64 : d <= 96 ? 96 : d <= 128 ? 128 : d <= 192 ? 192 : 256; }
void launch_cache_append(const evconv_append_args& a, bool vec, hipStream_t s);
void launch_cache_read(const evconv_read_args& a, hipStream_t s);

// How the rows of a call (tokens x query heads that share a key head) are dealt out over workgroups.
struct AttendWay {
  int64_t units;  // tiles of rows; 0: none goes this way
  int tiles;      // of a sequence of equal lengths (of a token with chosen pages), or -1
  int chunk;      // tokens that a workgroup looks at (with chosen pages: of their list)
  int splits;     // workgroups that share a row's tokens
};
constexpr int kFewRows = 16;                             // rows of a workgroup of the first way
constexpr int kPieceRowsBf16 = 128, kPieceRowsF32 = 64;  // of the second

struct AttendParams {
  evconv_attend_args a;
  int dp, log;      // padded channels, log2 of the page
  int share;        // query heads to a key head
  bool vec, vec_o;  // rows of q may be read in 16-byte loads, rows of o written four values at a time
  int64_t most;     // tokens of a sequence that are looked at, at most
  float scale2;     // scale * log2(e)
  AttendWay rows, pieces;
  int few;          // sequences of up to so many rows go the first way
  // workspace
  float* part;      // [splits][n_tokens * heads_q][dp] sums
  float* stat;      // [splits][n_tokens * heads_q][2] largest exponent, sum of weights
};
size_t plan_attend(AttendParams& p);  // bytes of workspace
void place_attend(AttendParams& p, char* workspace);
void launch_attend(const AttendParams& p, hipStream_t s);
void launch_attend_rows_bf16(const AttendParams& p, hipStream_t s);
void launch_attend_rows_fp4(const AttendParams& p, hipStream_t s);
void launch_attend_pieces_bf16(const AttendParams& p, hipStream_t s);
void launch_attend_pieces_fp4(const AttendParams& p, hipStream_t s);

struct SelectParams {
  evconv_select_args a;
  int dp, log, share;
  int64_t most;   // as above
  int pages;      // pages of a sequence at most, the row length of `score`
  int len;        // tokens of every sequence, or -1
  unsigned* score;  // workspace: [n_tokens][heads][pages], in the order of the scores
};
size_t plan_select(SelectParams& p);
void launch_select(const SelectParams& p, hipStream_t s);

}  // namespace evk
