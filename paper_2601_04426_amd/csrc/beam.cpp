// C ABI of beam search (see include/xg2mask.h): argument checks and launches.
#include <algorithm>
#include <string>

#include "beam.hpp"

using namespace xg2;

namespace {

template <typename F>
int32_t enter(F&& f) {
    return api_guarded([](void* p) { return (*static_cast<std::remove_reference_t<F>*>(p))(); }, &f);
}

int32_t launched() {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? XG2_OK : api_fail(XG2_EHIP, (std::string("kernel launch: ") + hipGetErrorString(e)).c_str());
}

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
size_t rounded(size_t n) { return (n + 255) & ~(size_t)255; }

struct Shape { size_t stats, blocks; uint32_t pieces; };
Shape select_shape(int32_t dtype, int32_t groups, int32_t beams, int32_t V) {
    const size_t rows = (size_t)groups * (size_t)beams;
    const uint32_t pieces = beam_pieces(V, dtype == XG2_F32 ? 4 : 2);
    return {rounded(rows * pieces * sizeof(float4)), rounded(rows * pieces * kBeamPieceBlocks * sizeof(float)), pieces};
}
const char* bad_shape(int32_t dtype, int32_t groups, int32_t beams, int32_t V, int32_t n_out) {
    if (dtype != XG2_F32 && dtype != XG2_BF16) return "unknown dtype";
    if (groups < 0 || beams < 1 || (uint32_t)beams > kBeamsMost) return "between 1 and 64 beams a group";
    if ((int64_t)groups * beams > (int64_t)kBeamRowsMost) return "more than 2^20 rows";
    if (V < 1 || V > kBeamVocabMost) return "between 1 and 2^24 tokens";
    if (n_out < 1 || (uint32_t)n_out > kBeamOutMost) return "between 1 and 128 candidates a group";
    return nullptr;
}
int32_t bad(const char* call, const char* what) { return api_fail(XG2_EINVAL, (std::string(call) + ": " + what).c_str()); }

}  // namespace

extern "C" {

int32_t xg2_beam_select_workspace(int32_t dtype, int32_t groups, int32_t beams, int32_t V, int32_t n_out, size_t* bytes) {
    return enter([&]() -> int32_t {
        if (!bytes) return bad("xg2_beam_select_workspace", "bad argument");
        if (const char* what = bad_shape(dtype, groups, beams, V, n_out)) return bad("xg2_beam_select_workspace", what);
        const Shape s = select_shape(dtype, groups, beams, V);
        *bytes = s.stats + s.blocks;
        return XG2_OK;
    });
}

int32_t xg2_beam_select(const void* logits_dev, int32_t dtype, int32_t groups, int32_t beams, int32_t V, int64_t row_stride_elems,
                        const int32_t* bitmask_dev, int64_t bm_row_stride_words, int32_t over, const float* scores_dev, const int32_t* finished_dev,
                        int32_t eos_id, int32_t n_out, float* out_scores_dev, int32_t* out_parents_dev, int32_t* out_tokens_dev,
                        int32_t* out_finished_dev, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
    return enter([&]() -> int32_t {
        const char* const me = "xg2_beam_select";
        if (const char* what = bad_shape(dtype, groups, beams, V, n_out)) return bad(me, what);
        if (over != XG2_OVER_ALLOWED && over != XG2_OVER_ALL) return bad(me, "the softmax goes over XG2_OVER_ALLOWED or XG2_OVER_ALL");
        if (groups == 0) return XG2_OK;
        if (!logits_dev || !scores_dev || !out_scores_dev || !out_parents_dev || !out_tokens_dev || !workspace_dev) return bad(me, "null buffer");
        if (row_stride_elems < V || (bitmask_dev && bm_row_stride_words < ((int64_t)V + 31) / 32)) return bad(me, "stride smaller than the row");
        if (!aligned(logits_dev, dtype == XG2_F32 ? 4 : 2) || !aligned(workspace_dev, 16)) return bad(me, "logits off a multiple of their type, or workspace off 16 bytes");
        if (!aligned(bitmask_dev, 4) || !aligned(scores_dev, 4) || !aligned(finished_dev, 4) || !aligned(out_scores_dev, 4) || !aligned(out_parents_dev, 4) ||
            !aligned(out_tokens_dev, 4) || !aligned(out_finished_dev, 4))
            return bad(me, "buffer of words off a multiple of 4 bytes");
        const Shape s = select_shape(dtype, groups, beams, V);
        if (workspace_bytes < s.stats + s.blocks) return bad(me, "workspace smaller than xg2_beam_select_workspace says");
        api_require_device();
        BeamSelect A{};
        A.logits = logits_dev; A.row_stride = row_stride_elems;
        A.bitmask = reinterpret_cast<const uint32_t*>(bitmask_dev); A.bm_stride = bm_row_stride_words;
        A.scores = scores_dev; A.finished = finished_dev;
        A.stats = static_cast<float4*>(workspace_dev);
        A.block_max = reinterpret_cast<float*>(static_cast<char*>(workspace_dev) + s.stats);
        A.out_scores = out_scores_dev; A.out_parents = out_parents_dev; A.out_tokens = out_tokens_dev; A.out_finished = out_finished_dev;
        A.groups = (uint32_t)groups; A.beams = (uint32_t)beams; A.n_out = (uint32_t)n_out; A.pieces = s.pieces;
        A.V = V; A.eos_id = eos_id; A.over_all = over == XG2_OVER_ALL; A.dtype = (uint32_t)dtype; A.near = beam_near(V);
        launch_beam_select(A, (hipStream_t)hip_stream);
        return launched();
    });
}

int32_t xg2_batch_reorder(xg2_batch* batch, int32_t beams, const int32_t* parents_dev, int32_t* status_dev, void* hip_stream) {
    return enter([&]() -> int32_t {
        const char* const me = "xg2_batch_reorder";
        if (!batch || !parents_dev || beams < 1 || (uint32_t)beams > kBeamsMost) return bad(me, "bad argument");
        if (!aligned(parents_dev, 4) || !aligned(status_dev, 4)) return bad(me, "buffer of words off a multiple of 4 bytes");
        BatchView b = api_batch(batch);
        if (b.dev.B % (uint32_t)beams != 0) return bad(me, "the number of slots is no multiple of the beams");
        if (!b.all_assigned) return bad(me, "every slot needs a cache first (xg2_batch_assign)");
        launch_batch_reorder(b.dev, (uint32_t)beams, parents_dev, status_dev, (hipStream_t)hip_stream);
        return launched();
    });
}

int32_t xg2_beam_reorder_rows(void* data_dev, int32_t groups, int32_t beams, const int32_t* parents_dev, int64_t row_stride, int32_t outer,
                              int64_t outer_stride, int32_t pieces, int64_t piece_stride, int32_t positions, int64_t position_bytes,
                              const int32_t* begin_dev, const int32_t* end_dev, void* hip_stream) {
    return enter([&]() -> int32_t {
        const char* const me = "xg2_beam_reorder_rows";
        if (groups < 0 || beams < 1 || (uint32_t)beams > kBeamsMost || outer < 0 || pieces < 0 || positions < 0 || position_bytes < 0) return bad(me, "bad argument");
        if ((int64_t)groups * beams > (int64_t)kBeamRowsMost) return bad(me, "more than 2^20 rows");
        if ((int64_t)outer * pieces > (int64_t)kBeamPiecesMost) return bad(me, "more than 2^23 pieces a row");
        if (groups == 0 || outer == 0 || pieces == 0 || positions == 0 || position_bytes == 0 || beams == 1) return XG2_OK;
        if (!data_dev || !parents_dev) return bad(me, "null buffer");
        if (!aligned(parents_dev, 4) || !aligned(begin_dev, 4) || !aligned(end_dev, 4)) return bad(me, "buffer of words off a multiple of 4 bytes");
        if (position_bytes > INT64_MAX / positions) return bad(me, "a piece of more than 2^63 - 1 bytes");
        const int64_t piece = (int64_t)positions * position_bytes;
        // rows, pieces and outer parts must not share bytes: a stride is at least a piece where there is more than one of its kind
        if (row_stride < piece || (pieces > 1 && piece_stride < piece) || (outer > 1 && outer_stride < piece)) return bad(me, "stride smaller than a piece");
        api_require_device();
        BeamRows A{};
        A.data = static_cast<uint8_t*>(data_dev); A.parents = parents_dev; A.begin = begin_dev; A.end = end_dev;
        A.row_stride = row_stride; A.outer_stride = outer > 1 ? outer_stride : 0; A.piece_stride = pieces > 1 ? piece_stride : 0;
        A.position_bytes = position_bytes;
        A.groups = (uint32_t)groups; A.beams = (uint32_t)beams; A.outer = (uint32_t)outer; A.pieces = (uint32_t)pieces; A.positions = (uint32_t)positions;
        launch_beam_reorder_rows(A, (hipStream_t)hip_stream);
        return launched();
    });
}

int32_t xg2_beam_backtrace(const int32_t* tokens_dev, const int32_t* parents_dev, int32_t steps, int64_t step_stride, int32_t groups, int32_t beams,
                           int32_t* out_tokens_dev, int64_t out_stride, int32_t* out_lengths_dev, void* hip_stream) {
    return enter([&]() -> int32_t {
        const char* const me = "xg2_beam_backtrace";
        if (steps < 0 || groups < 0 || beams < 1 || (uint32_t)beams > kBeamsMost) return bad(me, "bad argument");
        if ((int64_t)groups * beams > (int64_t)kBeamRowsMost) return bad(me, "more than 2^20 rows");
        if (groups == 0) return XG2_OK;
        if (steps > 0 && (!tokens_dev || !parents_dev || !out_tokens_dev)) return bad(me, "null buffer");
        if (steps > 0 && (step_stride < (int64_t)groups * beams || out_stride < steps)) return bad(me, "stride smaller than the row");
        if (!aligned(tokens_dev, 4) || !aligned(parents_dev, 4) || !aligned(out_tokens_dev, 4) || !aligned(out_lengths_dev, 4)) return bad(me, "buffer of words off a multiple of 4 bytes");
        if (steps == 0 && !out_lengths_dev) return XG2_OK;
        api_require_device();
        launch_beam_backtrace(BeamTrace{tokens_dev, parents_dev, step_stride, out_tokens_dev, out_stride, out_lengths_dev, (uint32_t)steps, (uint32_t)groups, (uint32_t)beams},
                              (hipStream_t)hip_stream);
        return launched();
    });
}

}  // extern "C"
