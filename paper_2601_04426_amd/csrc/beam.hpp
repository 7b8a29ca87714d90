// Beam search under a grammar: launchers of the kernels in beam.hip, and what their host side (beam.cpp) shares with api.cpp.
#pragma once
#include <cmath>
#include <cstdint>
#include <mutex>

#include "../../include/xg2mask.h"
#include "device.hpp"

namespace xg2 {

// ---- selection ------------------------------------------------------------------------------------------------------
constexpr uint32_t kBeamsMost = 64, kBeamOutMost = 128;     // beams of a group; candidates chosen for one
constexpr int32_t kBeamVocabMost = 1 << 24;
constexpr uint32_t kBeamRowsMost = 1u << 20;
constexpr int kBeamPiece = 2048, kBeamBlock = 64;           // tokens that a wavefront takes; tokens that share a maximum
constexpr int kBeamPieceBlocks = kBeamPiece / kBeamBlock;
// Pieces of a row, counted from the 128-byte boundary at or before its begin, wherever that lies.
constexpr uint32_t beam_pieces(int32_t V, int32_t elem_bytes) { return ((uint32_t)V + 128u / (uint32_t)elem_bytes - 1 + kBeamPiece - 1) / kBeamPiece; }

struct BeamSelect {
    const void* logits; long long row_stride;               // elements
    const uint32_t* bitmask; long long bm_stride;           // null: everything is allowed
    const float* scores; const int32_t* finished;           // [rows]; finished may be null
    float4* stats;                                          // [rows * pieces]: of what counts in the softmax the maximum and the sum of exponentials relative
                                                            // to it, and the largest allowed logit
    float* block_max;                                       // [rows * pieces * kBeamPieceBlocks] largest allowed logit
    float* out_scores; int32_t* out_parents; int32_t* out_tokens; int32_t* out_finished;
    uint32_t groups, beams, n_out, pieces;
    int32_t V, eos_id;
    uint32_t over_all;                                      // the softmax goes over all tokens, not over the allowed ones
    uint32_t dtype;
    double near;                                            // scores of different rows closer than this are compared with sums in 64 bits
};
// How far the difference of two rows' scores may be off by their sums in 32 bits: twice what one sum may be off, relative to its value.
// A term 2^t, t = x log2(e) - c, is off by one unit of the exponential (2^-23), by the rounding of t (|t| 2^-24 ln 2 = (top - x) 2^-24)
// and by that of log2(e) to 32 bits, which is made good for the largest x and leaves (top - x) 0.23 2^-24; the mean of top - x over the
// probabilities is at most ln V.  Between a term and its piece's sum lie 11 additions of 2^-24 each.  (Pieces are joined in 64 bits.)
inline double beam_near(int32_t V) { return (1.23 * std::log((double)(V < 2 ? 2 : V)) + 2 + 11) / (1 << 23); }
void launch_beam_select(const BeamSelect& A, hipStream_t stream);

// ---- reordering -----------------------------------------------------------------------------------------------------
void launch_batch_reorder(const BatchDev& D, uint32_t beams, const int32_t* parents_dev, int32_t* status_dev, hipStream_t stream);

constexpr uint32_t kBeamPiecesMost = 1u << 23;              // pieces of a row of a buffer: a workgroup of 256 threads each at the least
struct BeamRows {
    uint8_t* data; const int32_t* parents;
    const int32_t* begin; const int32_t* end;               // [groups] positions, or null: all
    int64_t row_stride, outer_stride, piece_stride;         // bytes
    int64_t position_bytes;
    uint32_t groups, beams, outer, pieces, positions;
};
void launch_beam_reorder_rows(const BeamRows& A, hipStream_t stream);

struct BeamTrace {
    const int32_t* tokens; const int32_t* parents; int64_t step_stride;      // entries from one step to the next
    int32_t* out; int64_t out_stride; int32_t* lengths;
    uint32_t steps, groups, beams;
};
void launch_beam_backtrace(const BeamTrace& A, hipStream_t stream);

// ---- what api.cpp lends ---------------------------------------------------------------------------------------------
int32_t api_fail(int32_t code, const char* message);                         // sets the thread's error text
int32_t api_guarded(int32_t (*call)(void*), void* arg);                      // exceptions become status codes
void api_require_device();                                                   // throws without one
struct BatchView { std::unique_lock<std::mutex> lock; BatchDev dev; bool all_assigned; };
BatchView api_batch(xg2_batch* batch);

}  // namespace xg2
