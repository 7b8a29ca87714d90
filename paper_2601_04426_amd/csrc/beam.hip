// gfx950 (CDNA4, wave64) kernels of beam search under a grammar:
//   k_beam_scan          one pass over the logits: sums of exponentials and the largest allowed logit of every block of tokens
//   k_beam_pick          the best candidates of a group, from the blocks that can hold them
//   k_batch_reorder      matcher slots take over the state of their parents
//   k_beam_reorder_rows  the same for rows of a caller's buffer, in place (k_beam_reorder_strips: more than 16 beams)
//   k_beam_backtrace     sequences from the steps' tokens and parents
#include <algorithm>
#include <cstddef>
#include <type_traits>

#include "beam.hpp"

namespace xg2 {
namespace {

constexpr float NINF = -__builtin_inff();

// Memory that is known to be device memory: a pointer out of a struct of arguments could be of any kind, and loads of that sort are waited
// for together with those of LDS.
#if defined(__HIP_DEVICE_COMPILE__)
#define XG2_GLOBAL __attribute__((address_space(1)))
#else
#define XG2_GLOBAL
#endif
template <class P> using Global = XG2_GLOBAL P*;

__device__ __forceinline__ uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }
__device__ __forceinline__ float lane_float(float v, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); }

// Sums and maxima over lanes: the partners within a row of 16 lanes, then the rows.  After the first four steps all lanes of a row have
// the row's value, after the next (lane 15 of a row to the row behind it) lanes 31 and 63 that of 32 lanes, after the last lane 63 that of all.
constexpr int DPP_SWAP1 = 0xB1, DPP_SWAP2 = 0x4E, DPP_HALF_MIRROR = 0x141, DPP_MIRROR = 0x140, DPP_ROW_BCAST15 = 0x142, DPP_ROW_BCAST31 = 0x143;
template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ float moved(float own, float v) { return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(own), __float_as_int(v), CTRL, ROWS, 0xF, false)); }
// The larger of two (three) numbers, of two with a quiet NaN the other.  A signalling NaN takes the number away, in v_max_f32 and in what the
// compiler makes of fmaxf, so who takes the maximum of values from memory looks for NaN among them.
__device__ __forceinline__ float larger(float a, float b) { float d; asm("v_max_f32 %0, %1, %2" : "=v"(d) : "v"(a), "v"(b)); return d; }
__device__ __forceinline__ float larger(float a, float b, float c) { float d; asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c)); return d; }
// Four values at a time, stage by stage, so that none is read across lanes within two instructions of being written (which the device does
// not wait for, and of which the compiler knows nothing here).
#if defined(__HIP_DEVICE_COMPILE__)
#define XG2_MAX4(HOW) "v_max_f32_dpp %0, %0, %0 " HOW "\n\tv_max_f32_dpp %1, %1, %1 " HOW "\n\tv_max_f32_dpp %2, %2, %2 " HOW "\n\tv_max_f32_dpp %3, %3, %3 " HOW "\n\t"
__device__ __forceinline__ void largest_of_8(float& a, float& b, float& c, float& d) {                                                      // all lanes
    asm volatile("s_nop 1\n\t" XG2_MAX4("quad_perm:[1,0,3,2] row_mask:0xf bank_mask:0xf") XG2_MAX4("quad_perm:[2,3,0,1] row_mask:0xf bank_mask:0xf")
                 XG2_MAX4("row_half_mirror row_mask:0xf bank_mask:0xf") "s_nop 1" : "+v"(a), "+v"(b), "+v"(c), "+v"(d));
}
__device__ __forceinline__ void largest_of_16(float& a, float& b, float& c, float& d) {                                                     // all lanes
    asm volatile("s_nop 1\n\t" XG2_MAX4("quad_perm:[1,0,3,2] row_mask:0xf bank_mask:0xf") XG2_MAX4("quad_perm:[2,3,0,1] row_mask:0xf bank_mask:0xf")
                 XG2_MAX4("row_half_mirror row_mask:0xf bank_mask:0xf") XG2_MAX4("row_mirror row_mask:0xf bank_mask:0xf") "s_nop 1" : "+v"(a), "+v"(b), "+v"(c), "+v"(d));
}
__device__ __forceinline__ float largest_of_64(float v) {                                                                                  // lane 63
    asm volatile("s_nop 1\n\tv_max_f32_dpp %0, %0, %0 quad_perm:[1,0,3,2] row_mask:0xf bank_mask:0xf\n\ts_nop 1\n\tv_max_f32_dpp %0, %0, %0 quad_perm:[2,3,0,1] row_mask:0xf bank_mask:0xf\n\t"
                 "s_nop 1\n\tv_max_f32_dpp %0, %0, %0 row_half_mirror row_mask:0xf bank_mask:0xf\n\ts_nop 1\n\tv_max_f32_dpp %0, %0, %0 row_mirror row_mask:0xf bank_mask:0xf\n\t"
                 "s_nop 1\n\tv_max_f32_dpp %0, %0, %0 row_bcast:15 row_mask:0xa bank_mask:0xf\n\ts_nop 1\n\tv_max_f32_dpp %0, %0, %0 row_bcast:31 row_mask:0xc bank_mask:0xf\n\ts_nop 1" : "+v"(v));
    return v;
}
#else
__device__ void largest_of_8(float&, float&, float&, float&) {}
__device__ void largest_of_16(float&, float&, float&, float&) {}
__device__ float largest_of_64(float v) { return v; }
#endif
__device__ __forceinline__ float sum_of_64(float v) {                                                                                      // lane 63
    v += moved<DPP_SWAP1>(v, v);
    v += moved<DPP_SWAP2>(v, v);
    v += moved<DPP_HALF_MIRROR>(v, v);
    v += moved<DPP_MIRROR>(v, v);
    v += moved<DPP_ROW_BCAST15, 0xA>(0.f, v);
    return v + moved<DPP_ROW_BCAST31, 0xC>(0.f, v);
}

// ---- selection ------------------------------------------------------------------------------------------------------
// score(row, token) = s_row - L_row + x, L_row = log of the sum of exp x over the tokens that count.  Chosen are the n best of all rows
// of a group.  A candidate among the n best lies in one of the n blocks (of kBeamBlock consecutive tokens) whose best tokens are the
// best, so one pass over the logits leaves two things of them: for every piece of kBeamPiece tokens the largest logit M that counts and
// the sum of exp(x - M), and for every block its largest allowed logit.  The second kernel has the rows' L from the first, takes the
// blocks whose best score is not below the n-th best of them, and looks at the tokens of these blocks only.
//
// The pass: a wavefront per piece, counted from the 128-byte boundary at or before the row's begin, so that all vectors are aligned
// whatever the row; 32 logits a lane in registers, all loaded before the first is used; under a mask one word of it a lane, vectors
// without an allowed token not loaded and pieces without one not looked at; where no mask word allows more than six tokens, each lane loads
// those of its word alone (4 rows of 32,000 tokens with two dozen allowed, us with the second kernel: vectors 10.6, up to three 10.1, up to
// six 9.6).  The piece's maximum goes into the exponents as it is (no
// running maximum, no second exponential).  Bound by memory and, over bfloat16, as much by instructions (8.5 a logit, one of them at a
// quarter rate: 47 us of issue for 1,024 rows of V = 151,936, 311 MB of logits and 19 of masks, which take 49 us, 6.7 TB/s, part of it from the
// last-level cache).  From memory alone, 2.49 GB without a mask: bfloat16 471 us, 5.3 TB/s, fp32 446 us, 5.6 TB/s.  256 rows fp32, masks of all kinds 14.4 us; 64 rows of V = 128,256 4.1; 4 rows of 32,000 with few tokens allowed 3.0.
constexpr int kScanWaves = 4, kScanFew = 6;
constexpr float LOG2E = 1.44269504088896340736f;
constexpr double LN2 = 0.693147180559945309417232;

typedef uint32_t Vec4 __attribute__((ext_vector_type(4)));
// vectors at any byte: the device takes them
typedef uint32_t Wide4 __attribute__((ext_vector_type(4), aligned(1)));
template <class E> struct Elem;
template <> struct Elem<float> {
    static constexpr int EPV = 4;
    static __device__ __forceinline__ float load(const float* p) { return *(Global<const float>)p; }
    static __device__ __forceinline__ void unpack(const Vec4& v, float* x) { _Pragma("unroll") for (int k = 0; k < 4; ++k) x[k] = __uint_as_float(v[k]); }
    // the vector at element e of the row, put together; what is not of the row is any of its logits
    static __device__ __forceinline__ Vec4 gather(const float* row, int e, int V) {
        Vec4 v;
        _Pragma("unroll") for (int k = 0; k < 4; ++k) v[k] = __float_as_uint(load(row + min(max(e + k, 0), V - 1)));
        return v;
    }
};
template <> struct Elem<uint16_t> {                                  // bfloat16
    static constexpr int EPV = 8;
    static __device__ __forceinline__ float load(const uint16_t* p) { return __uint_as_float((uint32_t)*(Global<const uint16_t>)p << 16); }
    static __device__ __forceinline__ void unpack(const Vec4& v, float* x) {
        _Pragma("unroll") for (int k = 0; k < 4; ++k) { x[2 * k] = __uint_as_float(v[k] << 16); x[2 * k + 1] = __uint_as_float(v[k] & 0xFFFF0000u); }
    }
    static __device__ __forceinline__ Vec4 gather(const uint16_t* row, int e, int V) {
        uint32_t x[8];
        _Pragma("unroll") for (int k = 0; k < 8; ++k) x[k] = *(Global<const uint16_t>)(row + min(max(e + k, 0), V - 1));
        return Vec4{x[0] | x[1] << 16, x[2] | x[3] << 16, x[4] | x[5] << 16, x[6] | x[7] << 16};
    }
};

// Whether a lane has a signalling NaN among its values.  A piece's sum is NaN if a term is, whereupon the choice looks through the row again;
// where no maximum is left to take a sum of, what counts may have fallen to a signalling NaN, and the sum has to say so too.
template <int N>
__device__ __forceinline__ bool signalling(const float (&x)[N]) {
    bool any = false;
    _Pragma("unroll") for (int i = 0; i < N; ++i) any |= __builtin_amdgcn_classf(x[i], 1);
    return any;
}
template <int M, int N>
__device__ __forceinline__ bool signalling(const float (&x)[M][N]) {
    bool any = false;
    _Pragma("unroll") for (int i = 0; i < M; ++i) any |= signalling(x[i]);
    return any;
}

__device__ __forceinline__ Vec4 stats_of(float top, float sum, float best) { return Vec4{__float_as_uint(top), __float_as_uint(sum), __float_as_uint(best), 0u}; }

// Elements of a row before the 128-byte boundary that its pieces and blocks are counted from.
template <class E> __device__ __forceinline__ int before_row(const E* row) { return (int)(reinterpret_cast<uintptr_t>(row) & 127) / (int)sizeof(E); }

// A row whose beam has ended or does not exist is not read.
__device__ __forceinline__ bool live_row(const float* scores, const int32_t* finished, uint32_t r) {
    const float s = ((Global<const float>)scores)[r];
    const int32_t ended = finished ? ((Global<const int32_t>)finished)[r] : 0;
    return ended == 0 && s > NINF && s < -NINF;
}

// WHICH: 0 no mask, 1 the softmax goes over the allowed tokens, 2 over all.
template <class E, int WHICH>
__global__ __launch_bounds__(64 * kScanWaves) void k_beam_scan(const uint32_t* bitmask, long long bm_stride, const float* scores, const int32_t* finished,
                                                                const void* logits, long long row_stride, uint32_t pieces, int V, BeamSelect A, uint32_t first_row) {
    // (the first 14 words of arguments are in registers when the kernel starts, a struct's are loaded)
    constexpr int EPV = Elem<E>::EPV, STEPS = kBeamPiece / 64 / EPV, VPW = 32 / EPV, LANES = kBeamBlock / EPV;   // vectors of a mask word, lanes of a block
    constexpr uint32_t ALL = (1u << EPV) - 1;
    const uint32_t r = first_row + blockIdx.y, lane = threadIdx.x & 63, piece = blockIdx.x * kScanWaves + uniform(threadIdx.x >> 6);
    if (piece >= pieces) return;
    const E* const row = static_cast<const E*>(logits) + (long long)r * row_stride;
    const int e0 = (int)piece * kBeamPiece - before_row(row);             
    const bool inner = e0 >= 0 && e0 + kBeamPiece <= V;
    // this lane's 32 tokens from e0 + 32 * lane on: which are in the row, and which of them are allowed
    const int first = e0 + 32 * (int)lane;
    uint32_t inside = ~0u;
    if (!inner) {
        if (first < 0) inside = first <= -32 ? 0 : ~0u << -first;
        if (first + 32 > V) inside &= first >= V ? 0 : ~0u >> (first + 32 - V);
    }
    uint32_t allowed = inside;
    if (WHICH != 0) {
        // (of words that are not the row's any: their tokens are not inside)
        const Global<const uint32_t> bm = (Global<const uint32_t>)(bitmask + (long long)r * bm_stride);
        const int at = first >> 5, last = (V - 1) >> 5;                              // (an arithmetic shift: rounds down)
        const uint32_t word = bm[min(max(at, 0), last)], next = bm[min(max(at + 1, 0), last)];
        allowed &= (uint32_t)(((uint64_t)next << 32 | word) >> (e0 & 31));
    }
    if (!live_row(scores, finished, r)) return;
    const uint32_t counted = WHICH == 1 ? allowed : inside;
    const Global<Vec4> stats = (Global<Vec4>)(A.stats + ((size_t)r * pieces + piece));
    const Global<float> block_max = (Global<float>)(A.block_max + ((size_t)r * pieces + piece) * kBeamPieceBlocks);
    if (WHICH == 1 && __ballot(counted != 0) == 0) {
        if (lane == 0) *stats = stats_of(NINF, 0.f, NINF);
        if (lane < kBeamPieceBlocks) block_max[lane] = NINF;                           // (a wavefront has as many lanes)
        return;
    }
    if (WHICH == 1 && __ballot(__popc(counted) > kScanFew) == 0) {
        // few tokens: each lane takes its own one by one, two lanes have a block (5 and 6 additions between a term and the sum)
        float x[kScanFew], own = NINF;
        uint32_t left = counted;
        _Pragma("unroll") for (int c = 0; c < kScanFew; ++c, left &= left - 1) {
            x[c] = NINF;
            if (left != 0) x[c] = Elem<E>::load(row + (first + __ffs((int)left) - 1));
        }
        _Pragma("unroll") for (int c = 0; c < kScanFew; ++c) own = fmaxf(own, x[c]);
        const float block = fmaxf(own, moved<DPP_SWAP1>(own, own)), all = lane_float(largest_of_64(own), 63);
        if (lane % 2 == 0) block_max[lane / 2] = block;
        float sum = 0;
        if (all > NINF) {
            const float c = larger(__fmul_rn(all, LOG2E), -3.4028234e38f);
            _Pragma("unroll") for (int i = 0; i < kScanFew; ++i) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], LOG2E, -c));
            sum = sum_of_64(sum);
        } else if (__ballot(signalling(x)) != 0) sum = __builtin_nanf("");
        if (lane == 63) *stats = stats_of(all, sum, all);
        return;
    }
    const E* const from = row + e0;
    const Global<const Vec4> vectors = (Global<const Vec4>)from;
    Vec4 raw[STEPS];
    uint32_t bits[STEPS];
    if (WHICH != 1 && inner) {
        _Pragma("unroll") for (int j = 0; j < STEPS; ++j) { bits[j] = ALL; raw[j] = vectors[j * 64 + (int)lane]; }
    } else {
        _Pragma("unroll") for (int j = 0; j < STEPS; ++j) bits[j] = ((uint32_t)__shfl((int)counted, (j * 64 + (int)lane) / VPW) >> ((int)lane % VPW * EPV)) & ALL;
        // A vector that the row shares with its neighbours lies between the buffer's first and last logit all the same, but for one at the
        // begin of the first row and one at the end of the last: these are put together from logits.
        const long long at = (long long)r * row_stride + e0, end = (long long)(A.groups * A.beams - 1) * row_stride + V;
        const bool apart = !inner && (at < 0 || at + kBeamPiece > end);
        unsigned long long open = 0;
        _Pragma("unroll") for (int j = 0; j < STEPS; ++j) {
            const int v = j * 64 + (int)lane;
            const bool whole = !apart || (at + v * EPV >= 0 && at + (v + 1) * EPV <= end);
            raw[j] = Vec4{0, 0, 0, 0};
            if (bits[j] != 0 && whole) raw[j] = vectors[v];
            if (apart) open |= __ballot(bits[j] != 0 && !whole);
        }
        if (open != 0) {
            _Pragma("unroll") for (int j = 0; j < STEPS; ++j) {
                const int v = j * 64 + (int)lane;
                if (bits[j] != 0 && !(at + v * EPV >= 0 && at + (v + 1) * EPV <= end)) raw[j] = Elem<E>::gather(row, e0 + v * EPV, V);
            }
        }
    }
    float x[STEPS][EPV], top = NINF, best[STEPS];
#pragma unroll
    for (int j = 0; j < STEPS; ++j) {
        Elem<E>::unpack(raw[j], x[j]);
        if (WHICH == 1 || !inner) {
            // (a bit spread over a word picks the logit or minus infinity)
            _Pragma("unroll") for (int c = 0; c < EPV; ++c) {
                const uint32_t m = (uint32_t)__builtin_amdgcn_sbfe((int)bits[j], c, 1);
                x[j][c] = __uint_as_float((__float_as_uint(x[j][c]) & m) | (__float_as_uint(NINF) & ~m));
            }
        }
        float m = larger(x[j][0], x[j][1], x[j][2]);
        if (EPV == 8) { m = larger(m, x[j][3], x[j][4]); m = larger(m, x[j][5], x[j][6]); }
        m = larger(m, x[j][EPV - 1]);
        if (WHICH == 2) top = larger(top, m);
        if (WHICH == 2) {
            const uint32_t ok = (uint32_t)__shfl((int)allowed, (j * 64 + (int)lane) / VPW) >> ((int)lane % VPW * EPV);
            float y[EPV];
            _Pragma("unroll") for (int c = 0; c < EPV; ++c) {
                const uint32_t w = (uint32_t)__builtin_amdgcn_sbfe((int)ok, c, 1);
                y[c] = __uint_as_float((__float_as_uint(x[j][c]) & w) | (__float_as_uint(NINF) & ~w));
            }
            m = larger(y[0], y[1], y[2]);
            if (EPV == 8) { m = larger(m, y[3], y[4]); m = larger(m, y[5], y[6]); }
            m = larger(m, y[EPV - 1]);
        }
        best[j] = m;
    }
    // the largest logit a lane has, then a block's maximum in all its lanes, of which the j-th writes that of step j
    float own = best[0];
    _Pragma("unroll") for (int j = 1; j < STEPS; ++j) own = larger(own, best[j]);
    if (EPV == 8) largest_of_8(best[0], best[1], best[2], best[3]);
    else { _Pragma("unroll") for (int j = 0; j < STEPS; j += 4) largest_of_16(best[j], best[j + 1], best[j + 2], best[j + 3]); }
    const uint32_t turn = lane % LANES;
    float written = best[0];
    _Pragma("unroll") for (int j = 1; j < STEPS; ++j) written = turn == (uint32_t)j ? best[j] : written;
    if (turn < STEPS) block_max[turn * (64 / LANES) + lane / LANES] = written;
    // the piece's largest allowed logit, and its largest that counts
    const float ok_max = lane_float(largest_of_64(own), 63), all = WHICH == 2 ? lane_float(largest_of_64(top), 63) : ok_max;
    float sum = 0;
    if (all > NINF) {
        const float c = larger(__fmul_rn(all, LOG2E), -3.4028234e38f);             // (finite, or minus infinity would come back as NaN)
        // (added up as a tree: 11 additions between a term and the sum, which is what its error is derived from)
        float part[STEPS * EPV];
        _Pragma("unroll") for (int i = 0; i < STEPS * EPV; ++i) part[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i / EPV][i % EPV], LOG2E, -c));
        _Pragma("unroll") for (int d = STEPS * EPV / 2; d > 0; d /= 2)
            _Pragma("unroll") for (int i = 0; i < d; ++i) part[i] += part[i + d];
        sum = sum_of_64(part[0]);
    } else if (__ballot(signalling(x)) != 0) sum = __builtin_nanf("");
    if (lane == 63) *stats = stats_of(all, sum, ok_max);
}

// ---- the best candidates of a group ---------------------------------------------------------------------------------
// One workgroup per group.  How near a score is to the best is measured in bins whose width grows with the distance (64 to an octave
// from 2^-6 on).  A count of the pieces' best scores gives the bin that the n-th best of them lies in: at least n candidates lie in it or
// below, so only pieces, in them blocks, in them tokens that do are looked at, which are few more than n as a rule.  Where they are not (fewer
// pieces than candidates, rows that differ much), blocks, and then tokens, are counted again.  16 lanes have a row's pieces.
// Bound by latency: a dozen dependent steps (rows' sums, count, pieces, blocks, tokens, places), three of them with a load from memory
// that other dies have written (about 1 us each).  us, kernel trace: 1 group of 4 beams, V = 32,000, 8 candidates 7.0; 16 of 4, V = 128,256,
// 8 candidates 8.8; 128 of 8, V = 151,936, 16 candidates 9.8; 8 of 32, V = 151,936, 64 candidates 12.7.  Both kernels in one launch, a workgroup
// for a group of up to 64 pieces, was slower when it was tried: 1 x 4 beams, V = 32,000 12.3 as two, 23.6 as one; 64 x 8, V = 4,000 13.9 and 21.6.
// What the pass left of a row's pieces stays in registers up to kPickHeld * 16 * kBeamPiece = 163,840 tokens; what is beyond is read again, one
// load at a time.  Calls over bfloat16 without a mask at V = 151,936 / 201,088 / 256,000 / 524,288, us: 1 group of 4 beams 11.6 / 14.1 / 14.4 / 22.2,
// 16 of 8 19.5 / 21.9 / 25.5 / 42.3, 4 of 32 21.0 / 24.8 / 27.9 / 47.6.
constexpr int kPickThreads = 1024, kPickMostWaves = kPickThreads / 64, kPickBins = 1024, kPickListed = 512, kPickElems = 1024, kPickHeld = 5;

constexpr uint32_t kRowShift = 26, kRowBits = (1u << kRowShift) - 1;
static_assert(kBeamsMost <= 1u << (32 - kRowShift) && ((uint64_t)kBeamVocabMost + 64 + kBeamPiece) / kBeamBlock <= kRowBits, "a row and its block fit a word");

enum RowState : uint32_t { ROW_NONE, ROW_LIVE, ROW_ENDED };
// A candidate: its score and its place in the order of rows and tokens, row << 32 | token + 1.
struct alignas(16) Candidate { double score; uint64_t at; };
struct PickShared {
    double base[kBeamsMost];                   // score of a token of the row: base + its logit (infinite: base, where the logit is +inf)
    float largest[kBeamsMost];                 // of the row's logits that count, from the first kernel
    uint32_t state[kBeamsMost];
    uint32_t infinite[kBeamsMost], exact[kBeamsMost], repair[kBeamsMost];
    double wave_top[kPickMostWaves];
    uint32_t bins[kPickBins];                  // bin b at (b % 16) * 64 + b / 16
    uint32_t pieces[kPickListed];              // row in the group << kRowShift | piece
    uint32_t blocks[kPickListed];              // row in the group << kRowShift | block
    uint32_t n_pieces, n_blocks, n_elems;
    Candidate found[kPickElems];
    float x[kPickElems];
    uint32_t place[kPickElems];
    uint16_t sorted[kPickElems];
    Candidate wave_best[kPickMostWaves];
};

// 2^t (down to -1000), and the natural logarithm of a sum of at least a half, to some 13 digits (what is added up has seven).
__device__ __forceinline__ double exp2_of(double t) {
    const double n = __builtin_rint(t), f = (t - n) * LN2;
    double p = 1.0 / 3628800;
    constexpr double C[] = {1.0 / 362880, 1.0 / 40320, 1.0 / 5040, 1.0 / 720, 1.0 / 120, 1.0 / 24, 1.0 / 6, 1.0 / 2, 1.0, 1.0};
    _Pragma("unroll") for (int i = 0; i < 10; ++i) p = __builtin_fma(p, f, C[i]);
    return __builtin_ldexp(p, (int)n);
}
__device__ __forceinline__ double log_of(double v) {
    const double y = (double)__builtin_amdgcn_logf((float)v), e = v * exp2_of(-y) - 1.0;      // (log2 in 32 bits, then what is missing)
    return y * LN2 + e - e * e * 0.5;
}
// a * b + c for a constant c that stays in its registers (the compiler's own choice adds to c in place, and copies it for every use).
__device__ __forceinline__ double fma_const(double a, double b, double c) {
#if defined(__HIP_DEVICE_COMPILE__)
    double d;
    asm("v_fma_f64 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
    return d;
#else
    return a * b + c;
#endif
}
// The sum of e^d over four d <= 0, each to the last bits of a double: side by side, since a step waits for the one before it and a
// workgroup has a wavefront or two on a unit.
__device__ __forceinline__ double sum_of_exps(const double (&x)[4]) {
    double n[4], f[4], p[4];
    _Pragma("unroll") for (int i = 0; i < 4; ++i) f[i] = __builtin_fmax(x[i], -1000.0);                 // (zero)
    _Pragma("unroll") for (int i = 0; i < 4; ++i) n[i] = __builtin_rint(f[i] * 1.4426950408889634073599);
    _Pragma("unroll") for (int i = 0; i < 4; ++i) f[i] = __builtin_fma(-n[i], 0.69314718055994528623, f[i]);
    _Pragma("unroll") for (int i = 0; i < 4; ++i) f[i] = __builtin_fma(-n[i], 2.3190468138462996e-17, f[i]);
    constexpr double C[] = {1.0 / 39916800, 1.0 / 3628800, 1.0 / 362880, 1.0 / 40320, 1.0 / 5040, 1.0 / 720, 1.0 / 120, 1.0 / 24, 1.0 / 6, 1.0 / 2, 1.0, 1.0};
    _Pragma("unroll") for (int i = 0; i < 4; ++i) p[i] = 1.0 / 479001600;                               // (|f| <= 0.35: the next term is 2^-52)
    _Pragma("unroll") for (int t = 0; t < 12; ++t) _Pragma("unroll") for (int i = 0; i < 4; ++i) p[i] = fma_const(p[i], f[i], C[t]);
    _Pragma("unroll") for (int i = 0; i < 4; ++i) p[i] = __builtin_ldexp(p[i], (int)n[i]);
    return (p[0] + p[1]) + (p[2] + p[3]);
}
// Over a row of 16 lanes, in all of them; and how many of the lanes' counts lie up to and with a lane.
template <int CTRL>
__device__ __forceinline__ double moved(double v) {
    const uint64_t u = (uint64_t)__double_as_longlong(v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp((int)u, (int)u, CTRL, 0xF, 0xF, false), hi = (uint32_t)__builtin_amdgcn_update_dpp((int)(u >> 32), (int)(u >> 32), CTRL, 0xF, 0xF, false);
    return __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
}
__device__ __forceinline__ double sum_of_16(double v) {
    v += moved<DPP_SWAP1>(v);
    v += moved<DPP_SWAP2>(v);
    v += moved<DPP_HALF_MIRROR>(v);
    return v + moved<DPP_MIRROR>(v);
}
__device__ __forceinline__ float largest_of_16(float v) {
    v = fmaxf(v, moved<DPP_SWAP1>(v, v));
    v = fmaxf(v, moved<DPP_SWAP2>(v, v));
    v = fmaxf(v, moved<DPP_HALF_MIRROR>(v, v));
    return fmaxf(v, moved<DPP_MIRROR>(v, v));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t shifted(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false); }
__device__ __forceinline__ uint32_t count_upto(uint32_t v) {
    v += shifted<0x111, 0xF>(v);                                     // from 1, 2, 4 and 8 lanes below in the row
    v += shifted<0x112, 0xF>(v);
    v += shifted<0x114, 0xF>(v);
    v += shifted<0x118, 0xF>(v);
    v += shifted<DPP_ROW_BCAST15, 0xA>(v);
    return v + shifted<DPP_ROW_BCAST31, 0xC>(v);
}

__device__ __forceinline__ uint32_t bin_of(double top, double score) {
    // (monotone: each step rounds one way for all; logits of 1e30 leave a score nothing of its beam's, and it can lie above the best)
    const float d = fmaxf((float)(top - score), 0.f) + 0.015625f;
    const uint32_t b = (__float_as_uint(d) >> 17) - (__float_as_uint(0.015625f) >> 17);
    return b < kPickBins - 1 ? b : kPickBins - 1;
}
// How far from the best the last score of a bin may lie (a bound).
__device__ __forceinline__ double reach_of(uint32_t bin) { return (double)__uint_as_float((bin + 1 + (__float_as_uint(0.015625f) >> 17)) << 17); }
__device__ __forceinline__ uint32_t bin_at(uint32_t b) { return b % 16 * 64 + b / 16; }
__device__ __forceinline__ double score_of(const PickShared& S, uint32_t k, float x) {
    return S.base[k] + (double)(S.infinite[k] ? (x == -NINF ? 0.f : NINF) : x);
}
__device__ __forceinline__ bool token_allowed(const BeamSelect& A, uint32_t r, long long t) {
    return !A.bitmask || ((((Global<const uint32_t>)A.bitmask)[(long long)r * A.bm_stride + (t >> 5)] >> (t & 31)) & 1u);
}
__device__ __forceinline__ uint64_t place_of(uint32_t row, long long token) { return (uint64_t)row << 32 | (uint64_t)(token + 1); }
// (no branch: three compares)
__device__ __forceinline__ bool before(const Candidate& a, const Candidate& b) { return (a.score > b.score) | ((a.score == b.score) & (a.at < b.at)); }

// 16 tokens of a row from t0 on: asked for, and taken when they are there: their logits, and which of them are in the row and, unless all
// are wanted, allowed.
template <class E>
struct Sixteen {
    static constexpr int EPV = Elem<E>::EPV, VECS = 16 / EPV;
    Vec4 raw[VECS];
    uint32_t word, next;
    __device__ __forceinline__ void ask(const BeamSelect& A, uint32_t r, int t0, bool all) {
        const E* const row = static_cast<const E*>(A.logits) + (long long)r * A.row_stride;
        word = next = ~0u;
        if (A.bitmask && !all) {
            const Global<const uint32_t> bm = (Global<const uint32_t>)(A.bitmask + (long long)r * A.bm_stride);
            const int at = t0 >> 5, last = (A.V - 1) >> 5;           // (an arithmetic shift: rounds down)
            word = bm[min(max(at, 0), last)];
            next = bm[min(max(at + 1, 0), last)];
        }
        if (t0 >= 0 && t0 + 16 <= A.V) { _Pragma("unroll") for (int v = 0; v < VECS; ++v) raw[v] = ((Global<const Wide4>)(row + t0))[v]; }
        else { _Pragma("unroll") for (int v = 0; v < VECS; ++v) raw[v] = Elem<E>::gather(row, t0 + v * EPV, A.V); }
    }
    __device__ __forceinline__ uint32_t take(int V, int t0, float* x) const {
        uint32_t ok = (uint32_t)(((uint64_t)next << 32 | word) >> (t0 & 31)) & 0xFFFF;
        if (t0 < 0) ok &= 0xFFFFu << min(-t0, 16);
        if (t0 + 16 > V) ok &= t0 < V ? 0xFFFFu >> (t0 + 16 - V) : 0u;
        _Pragma("unroll") for (int v = 0; v < VECS; ++v) Elem<E>::unpack(raw[v], x + v * EPV);
        return ok;
    }
};

// What is seldom called is no part of the kernel; it is handed the launch's own arguments and the place in LDS (a struct on the stack would be
// read from memory a word at a time, and LDS through flat instructions).
#if defined(__HIP_DEVICE_COMPILE__)
#define XG2_CONSTANT __attribute__((address_space(4)))
#define XG2_LDS __attribute__((address_space(3)))
#else
#define XG2_CONSTANT
#define XG2_LDS
#endif
typedef const XG2_CONSTANT BeamSelect* PickArgs;
typedef XG2_LDS PickShared* PickLds;
// k_beam_pick's arguments as they lie in memory, one behind the other at its type's alignment; the kernel's type is held against it below.
struct PickParams { const float4* all_stats; const float* scores; const int32_t* finished; uint32_t K, pieces, N; BeamSelect A; };
__device__ __forceinline__ PickArgs pick_args() {
#if defined(__HIP_DEVICE_COMPILE__)
    return (PickArgs)((const XG2_CONSTANT char*)__builtin_amdgcn_kernarg_segment_ptr() + offsetof(PickParams, A));
#else
    return nullptr;
#endif
}
__device__ __forceinline__ BeamSelect args_of(PickArgs p) {
    const uint64_t at = reinterpret_cast<uint64_t>(p);
    const PickArgs same = reinterpret_cast<PickArgs>((uint64_t)uniform((uint32_t)(at >> 32)) << 32 | uniform((uint32_t)at));
    BeamSelect A;
    __builtin_memcpy(&A, same, sizeof(A));
    return A;
}

// The row's sum in 64 bits; anew: also the maxima of its pieces and blocks without NaN (what the first kernel left of the row is not used).
template <class E>
__device__ __attribute__((noinline)) void repair_row(PickArgs args, PickLds lds, uint32_t group, uint32_t beam, bool anew) {
    const BeamSelect A = args_of(args);
    PickShared& S = *(PickShared*)lds;
    const uint32_t g = uniform(group), k = uniform(beam), r = g * A.beams + k, tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), waves = blockDim.x >> 6;
    const E* const row = static_cast<const E*>(A.logits) + (long long)r * A.row_stride;
    const int before = before_row(row);
    float top = NINF, x[16];
    const float score = ((Global<const float>)A.scores)[r];
    __syncthreads();                                                 // (S.wave_top has been read by all)
    if (anew) {
        // four lanes have a block, a wavefront in two turns a piece
        for (uint32_t p = wave; p < A.pieces; p += waves) {
            float piece_best = NINF;
            for (uint32_t b = lane >> 2; b < kBeamPieceBlocks; b += 16) {
                const int t0 = (int)p * kBeamPiece + (int)b * kBeamBlock + 16 * (int)(lane & 3) - before;
                Sixteen<E> T;
                T.ask(A, r, t0, false);
                const uint32_t ok = T.take(A.V, t0, x);
                T.word = T.next = ~0u;
                const uint32_t inside = T.take(A.V, t0, x);
                float best = NINF;
                _Pragma("unroll") for (int c = 0; c < 16; ++c) {
                    if ((ok >> c) & 1u) best = x[c] > best ? x[c] : best;                                    // (false for NaN)
                    if (((A.over_all ? inside : ok) >> c) & 1u) top = x[c] > top ? x[c] : top;
                }
                for (int d = 1; d < 4; d *= 2) { const float o = __shfl_xor(best, d); best = o > best ? o : best; }
                if ((lane & 3) == 0) ((Global<float>)A.block_max)[((size_t)r * A.pieces + p) * kBeamPieceBlocks + b] = best;
                piece_best = best > piece_best ? best : piece_best;
            }
            for (int d = 4; d < 64; d *= 2) { const float o = __shfl_xor(piece_best, d); piece_best = o > piece_best ? o : piece_best; }
            if (lane == 0) ((Global<float>)(A.stats + ((size_t)r * A.pieces + p)))[2] = piece_best;
        }
        for (int d = 1; d < 64; d *= 2) { const float o = __shfl_xor(top, d); top = o > top ? o : top; }
        if (lane == 0) S.wave_top[wave] = top;
        __syncthreads();
        for (uint32_t w = 0; w < waves; ++w) top = (float)S.wave_top[w] > top ? (float)S.wave_top[w] : top;
        __syncthreads();
    } else top = S.largest[k];
    // (counted from the row's begin, wherever it lies: rows that are alike have sums that are alike; the tokens of the next turn are on
    // their way)
    const bool infinite = top == -NINF;                              // (the tokens that have it count one, the others nothing)
    const double from = infinite ? 0.0 : (double)top;
    double sum = 0;
    const int step = 16 * (int)blockDim.x;
    Sixteen<E> one, two;
    int t0 = 16 * (int)tid;
    if (t0 < A.V) one.ask(A, r, t0, A.over_all);
    if (t0 + step < A.V) two.ask(A, r, t0 + step, A.over_all);
    for (; t0 < A.V; t0 += step) {
        const uint32_t counted = one.take(A.V, t0, x);
        one = two;
        if (t0 + 2 * step < A.V) two.ask(A, r, t0 + 2 * step, A.over_all);
        if (counted == 0) continue;
        if (infinite) { _Pragma("unroll") for (int c = 0; c < 16; ++c) x[c] = x[c] == -NINF ? 0.f : NINF; }
        _Pragma("unroll") for (int c = 0; c < 16; c += 4) {
            double d[4];
            _Pragma("unroll") for (int i = 0; i < 4; ++i) {
                // (a bit spread over a word picks the logit or minus infinity; what is NaN counts nothing, sum_of_exps sees to it)
                const uint32_t m = (uint32_t)__builtin_amdgcn_sbfe((int)counted, c + i, 1);
                d[i] = (double)__uint_as_float((__float_as_uint(x[c + i]) & m) | (__float_as_uint(NINF) & ~m)) - from;
            }
            sum += sum_of_exps(d);
        }
    }
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    if (lane == 0) S.wave_top[wave] = sum;
    __syncthreads();
    if (tid == 0) {
        double all = 0;
        for (uint32_t w = 0; w < waves; ++w) all += S.wave_top[w];
        S.exact[k] = 1;
        if (top == NINF) S.state[k] = ROW_NONE;
        else {
            S.infinite[k] = infinite;
            S.base[k] = (double)score - (log(all) + from);
        }
    }
    __threadfence_block();
    __syncthreads();
}

// The best of all threads' candidates, in all threads (at ~0: none).
__device__ Candidate best_of_all(PickShared& S, Candidate c) {
    for (int d = 1; d < 64; d *= 2) {
        const Candidate o{__shfl_xor(c.score, d), (uint64_t)__shfl_xor((unsigned long long)c.at, d)};
        if (o.at != ~0ull && (c.at == ~0ull || before(o, c))) c = o;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) S.wave_best[threadIdx.x >> 6] = c;
    __syncthreads();
    for (uint32_t w = 0; w < blockDim.x >> 6; ++w) {
        const Candidate o = S.wave_best[w];
        if (o.at != ~0ull && (c.at == ~0ull || before(o, c))) c = o;
    }
    return c;
}

__device__ __forceinline__ void write_choice(const BeamSelect& A, uint32_t g, uint32_t n, bool any, const Candidate& c) {
    const size_t at = (size_t)g * A.n_out + n;
    const int32_t token = any ? (int32_t)((uint32_t)c.at - 1u) : -1;
    A.out_scores[at] = any ? (float)c.score : NINF;
    A.out_parents[at] = any ? (int32_t)(g * A.beams + (uint32_t)(c.at >> 32)) : -1;
    A.out_tokens[at] = token;
    if (A.out_finished) A.out_finished[at] = token < 0 || token == A.eos_id;
}

// Too many are too much alike (logits that are all the same): all sums in 64 bits, then the best block n times, and the best candidate of
// these blocks n times, each the next one after the one before.
template <class E>
__device__ __attribute__((noinline)) void pick_one_by_one(PickArgs args, PickLds lds, uint32_t group) {
    const BeamSelect A = args_of(args);
    PickShared& S = *(PickShared*)lds;
    const uint32_t g = uniform(group), tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, waves = blockDim.x >> 6, K = A.beams, N = A.n_out, n_blocks = A.pieces * kBeamPieceBlocks;
    const double none = -(double)__builtin_inff();
    for (uint32_t k = 0; k < K; ++k) if (S.state[k] == ROW_LIVE && !S.exact[k]) repair_row<E>(args, lds, g, k, false);
    uint32_t n_found = 0;
    Candidate last{0, ~0ull};
    for (; n_found < N; ++n_found) {
        Candidate c{none, ~0ull};
        for (uint32_t k = wave; k < K; k += waves) {
            if (S.state[k] != ROW_LIVE) continue;
            for (uint32_t b = lane; b < n_blocks; b += 64) {
                const Candidate o{score_of(S, k, A.block_max[(size_t)(g * K + k) * n_blocks + b]), place_of(k, b)};
                if (o.score > none && (last.at == ~0ull || before(last, o)) && (c.at == ~0ull || before(o, c))) c = o;
            }
        }
        c = best_of_all(S, c);
        if (c.at == ~0ull) break;
        if (tid == 0) S.blocks[n_found] = (uint32_t)(c.at >> 32) << kRowShift | ((uint32_t)c.at - 1);
        last = c;
    }
    __syncthreads();
    last.at = ~0ull;
    for (uint32_t n = 0; n < N; ++n) {
        Candidate c{none, ~0ull};
        for (uint32_t i = wave; i < n_found; i += waves) {
            const uint32_t k = S.blocks[i] >> kRowShift, b = S.blocks[i] & kRowBits, r = g * K + k;
            const E* const row = static_cast<const E*>(A.logits) + (long long)r * A.row_stride;
            const long long t0 = (long long)b * kBeamBlock - before_row(row) + lane;
            for (int d = 0; d < kBeamBlock; d += 64) {
                const long long t = t0 + d;
                if (t < 0 || t >= A.V || !token_allowed(A, r, t)) continue;
                const Candidate o{score_of(S, k, Elem<E>::load(row + t)), place_of(k, t)};
                if (o.score > none && (last.at == ~0ull || before(last, o)) && (c.at == ~0ull || before(o, c))) c = o;
            }
        }
        if (tid < K && S.state[tid] == ROW_ENDED) {
            const Candidate o{S.base[tid], place_of(tid, -1)};
            if ((last.at == ~0ull || before(last, o)) && (c.at == ~0ull || before(o, c))) c = o;
        }
        c = best_of_all(S, c);
        if (tid == 0) write_choice(A, g, n, c.at != ~0ull, c);
        if (c.at == ~0ull) c = Candidate{none, ~0ull - 1};           // nothing comes after
        last = c;
    }
}

template <class E>
__global__ __launch_bounds__(kPickThreads) void k_beam_pick(const float4* all_stats, const float* scores, const int32_t* finished, uint32_t K, uint32_t pieces, uint32_t N, BeamSelect A) {
    __shared__ PickShared S;
    const PickArgs args = pick_args();
    const PickLds lds = (PickLds)&S;
    const uint32_t g = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), waves = blockDim.x >> 6;
    constexpr double none = -(double)__builtin_inff();
    // 16 lanes have a row.
    const uint32_t k = tid >> 4, part = tid & 15, r = g * K + k;
    const Global<const Vec4> stats = (Global<const Vec4>)(all_stats + (size_t)r * pieces);
    const bool mine = k < K;
    float s = NINF, best[kPickHeld];
    Vec4 held[kPickHeld];
    int32_t ended = 0;
    if (mine) {
        s = ((Global<const float>)scores)[r];
        if (finished) ended = ((Global<const int32_t>)finished)[r];
        _Pragma("unroll") for (int i = 0; i < kPickHeld; ++i) held[i] = stats[min(part + i * 16, pieces - 1)];
    }
    for (uint32_t i = tid; i < kPickBins; i += blockDim.x) S.bins[i] = 0;
    if (tid == 0) S.n_pieces = S.n_blocks = S.n_elems = 0;
    uint32_t state = !(s > NINF && s < -NINF) ? ROW_NONE : ended != 0 ? ROW_ENDED : ROW_LIVE, repair = 0;
    double base = s;
    float largest = NINF;
    if (state == ROW_LIVE) {
        float& m = largest;
        bool odd = false;
        auto look = [&](const Vec4& v) {
            const float x = __uint_as_float(v[0]), y = __uint_as_float(v[1]);
            odd |= x != x || y != y;
            m = x > m ? x : m;
        };
        _Pragma("unroll") for (int i = 0; i < kPickHeld; ++i) {
            if (part + i * 16 >= pieces) held[i] = stats_of(NINF, 0.f, NINF);
            look(held[i]);
            best[i] = __uint_as_float(held[i][2]);
        }
        for (uint32_t p = part + kPickHeld * 16; p < pieces; p += 16) look(stats[p]);
        m = largest_of_16(m);
        // a NaN or an infinity among what counts, or magnitudes that the sum's exponents cannot take or that leave a score no places behind
        // the point: from the logits again, by this workgroup alone, row after row (a call of 128 groups whose seven other beams have scores
        // of -1e9 697 us; of -1e5 66, of minus infinity 24)
        odd |= !(m < 1e6f) || (m > NINF && m < -1e6f) || !(s < 1e6f && s > -1e6f);
        repair = ((__ballot(odd) >> (lane & 48)) & 0xFFFF) != 0;
        // A piece's sum is of 2^(x * LOG2E - c), c = the rounded product of its maximum and LOG2E; LOG2E itself is off by `off`.
        const double off = (double)LOG2E - 1.4426950408889634073599, mc = (double)__fmul_rn(m, LOG2E) - (double)m * off;
        double sum = 0;
        auto add = [&](const Vec4& v) {
            const float x = __uint_as_float(v[0]);
            const double t = (double)__fmul_rn(x, LOG2E) - (double)x * off - mc;
            if (t > -200) sum += (double)__uint_as_float(v[1]) * exp2_of(t);
        };
        _Pragma("unroll") for (int i = 0; i < kPickHeld; ++i) if (i * 16u < pieces) add(held[i]);     // (the same in all lanes)
        for (uint32_t p = part + kPickHeld * 16; p < pieces; p += 16) add(stats[p]);
        sum = sum_of_16(sum);
        if (!repair) {
            if (m == NINF) state = ROW_NONE;
            else base -= log_of(sum) + mc * LN2;
        }
    }
    if (mine && part == 0) { S.state[k] = state; S.base[k] = base; S.infinite[k] = 0; S.exact[k] = state != ROW_LIVE; S.repair[k] = repair; S.largest[k] = largest; }
    // Distances are taken from the best candidate: the best beam's score would do while few candidates lie as far from it as the n-th, but
    // where a row's logits are nearly the same all tokens are as far from it (4 groups of 32 rows of 151,936 logits with a deviation of 0.3:
    // 4,631 us, from the best candidate 21; ordinary rows 0.1 to 0.4 us less).
    bool infinite = false;
    auto own_score = [&](float m) { return infinite ? (m == -NINF ? base : none) : base + (double)m; };
    auto find_top = [&] {
        double t = state == ROW_ENDED ? base : none;
        if (state == ROW_LIVE) {
            float m = NINF;
            _Pragma("unroll") for (int i = 0; i < kPickHeld; ++i) m = best[i] > m ? best[i] : m;
            for (uint32_t p = part + kPickHeld * 16; p < pieces; p += 16) { const float o = ((Global<const float>)(stats + p))[2]; m = o > m ? o : m; }
            m = largest_of_16(m);
            if (m > NINF) t = own_score(m);
        }
        double o = __shfl_xor(t, 16);
        t = o > t ? o : t;
        o = __shfl_xor(t, 32);
        t = o > t ? o : t;
        if (lane == 0) S.wave_top[wave] = t;
    };
    find_top();
    if (__syncthreads_or((int)repair)) {
        for (uint32_t q = 0; q < K; ++q) if (S.repair[q]) repair_row<E>(args, lds, g, q, true);
        if (repair) {
            state = S.state[k]; base = S.base[k]; infinite = S.infinite[k] != 0;
            _Pragma("unroll") for (int i = 0; i < kPickHeld; ++i) best[i] = part + i * 16 < pieces ? ((Global<const float>)(stats + part + i * 16))[2] : NINF;
        }
        find_top();
        __syncthreads();
    }
    double top = none;
    for (uint32_t w = 0; w < waves; ++w) top = S.wave_top[w] > top ? S.wave_top[w] : top;
    // how many pieces (and ended beams) have their best score in each bin
    uint32_t bin[kPickHeld];
    auto bin_if = [&](uint32_t row, float m) {
        const double v = score_of(S, row, m);
        return m > NINF && v > none ? bin_of(top, v) : (uint32_t)kPickBins;
    };
    auto count = [&](uint32_t b) { if (b < kPickBins) atomicAdd(&S.bins[bin_at(b)], 1u); };
    if (state == ROW_LIVE) {
        auto own_bin = [&](float m) { return m > NINF && own_score(m) > none ? bin_of(top, own_score(m)) : (uint32_t)kPickBins; };
        _Pragma("unroll") for (int i = 0; i < kPickHeld; ++i) { bin[i] = own_bin(best[i]); count(bin[i]); }
        for (uint32_t p = part + kPickHeld * 16; p < pieces; p += 16) count(own_bin(((Global<const float>)(stats + p))[2]));
    } else if (state == ROW_ENDED && part == 0) count(bin_of(top, base));
    __syncthreads();
    // The bin of the n-th best of what was counted (every wavefront for itself), one more: what lies within A.near of it; if fewer were counted, the last.
    auto bin_of_nth = [&] {
        uint32_t n[16], sum = 0;
        _Pragma("unroll") for (uint32_t i = 0; i < 16; ++i) { n[i] = S.bins[i * 64 + lane]; sum += n[i]; }
        const uint32_t upto = count_upto(sum);
        const unsigned long long reached = __ballot(upto >= N);
        if (reached == 0) return (uint32_t)kPickBins - 1;
        uint32_t at = upto - sum, b = 0;
        _Pragma("unroll") for (uint32_t i = 0; i < 16; ++i) { at += n[i]; b += at < N ? 1u : 0u; }
        return (uint32_t)min(__builtin_amdgcn_readlane((int)(lane * 16 + b + 1), __ffsll((long long)reached) - 1), kPickBins - 1);
    };
    auto count_anew = [&] {
        __syncthreads();
        for (uint32_t i = tid; i < kPickBins; i += blockDim.x) S.bins[i] = 0;
        if (tid == 0) S.n_blocks = 0;
        __syncthreads();
        if (state == ROW_ENDED && part == 0) count(bin_of(top, S.base[k]));
    };
    uint32_t last_bin = bin_of_nth();
    // the pieces that can hold one of the n best, of them the blocks, of them and the ended beams the candidates that can be one
    auto list_piece = [&](uint32_t p) { const uint32_t at = atomicAdd(&S.n_pieces, 1u); if (at < kPickListed) S.pieces[at] = k << kRowShift | p; };
    auto list_candidate = [&](double v, uint64_t at, float x) {
        const uint32_t i = atomicAdd(&S.n_elems, 1u);
        if (i < kPickElems) { S.found[i] = Candidate{v, at}; S.x[i] = x; }
    };
    if (state == ROW_LIVE) {
        _Pragma("unroll") for (int i = 0; i < kPickHeld; ++i) if (bin[i] <= last_bin) list_piece(part + i * 16);
        for (uint32_t p = part + kPickHeld * 16; p < pieces; p += 16) if (bin_if(k, ((Global<const float>)(stats + p))[2]) <= last_bin) list_piece(p);
    }
    __syncthreads();
    const uint32_t n_pieces = min(S.n_pieces, (uint32_t)kPickListed);
    auto each_block = [&](auto&& visit) {
        for (uint32_t i0 = tid; i0 < n_pieces * kBeamPieceBlocks; i0 += 4 * blockDim.x) {
            uint32_t at[4];                                          // (four loads before the first is used)
            float m[4];
            _Pragma("unroll") for (int q = 0; q < 4; ++q) {
                const uint32_t i = i0 + q * blockDim.x;
                m[q] = NINF;
                if (i >= n_pieces * kBeamPieceBlocks) continue;
                const uint32_t piece = S.pieces[i / kBeamPieceBlocks], row_k = piece >> kRowShift, block = (piece & kRowBits) * kBeamPieceBlocks + i % kBeamPieceBlocks;
                at[q] = row_k << kRowShift | block;
                m[q] = ((Global<const float>)A.block_max)[(size_t)(g * K + row_k) * pieces * kBeamPieceBlocks + block];
            }
            _Pragma("unroll") for (int q = 0; q < 4; ++q) if (m[q] > NINF) visit(at[q], bin_if(at[q] >> kRowShift, m[q]));
        }
    };
    for (bool counted = last_bin == kPickBins - 1;; counted = true) {
        if (counted) {
            count_anew();
            each_block([&](uint32_t, uint32_t b) { count(b); });
            __syncthreads();
            last_bin = min(last_bin, bin_of_nth());
        }
        each_block([&](uint32_t at, uint32_t b) {
            if (b > last_bin) return;
            const uint32_t n = atomicAdd(&S.n_blocks, 1u);
            if (n < kPickListed) S.blocks[n] = at;
        });
        __syncthreads();
        if (counted || S.n_blocks <= N + N / 2 + 16) break;
    }
    for (uint32_t i = tid; i < kPickElems; i += blockDim.x) S.place[i] = 0;
    // four lanes have a block, each of them 16 tokens
    const uint32_t listed_all = S.n_blocks, listed = min(listed_all, (uint32_t)kPickListed);
    auto each_token = [&](auto&& visit) {
        const double reach = last_bin < kPickBins - 1 ? top - reach_of(last_bin) : none;
        for (uint32_t i = tid >> 2; i < listed; i += blockDim.x >> 2) {
            const uint32_t block = S.blocks[i], row_k = block >> kRowShift, row_r = g * K + row_k;
            const int t0 = (int)((block & kRowBits) * kBeamBlock + 16 * (tid & 3)) - before_row(static_cast<const E*>(A.logits) + (long long)row_r * A.row_stride);
            float x[16];
            Sixteen<E> T;
            T.ask(A, row_r, t0, false);
            const uint32_t ok = T.take(A.V, t0, x);
            // a bound in 32 bits first, below what is sought by more than its own rounding (1e-6 of it) and that of the three sums in 64
            // bits behind it (half a place each, 2^-53 of a base that can be 1e14 times a logit: tokens that differ have one score then)
            const double base = S.base[row_k], least = reach - base;
            const float bound = (float)least - (__builtin_fabsf((float)least) * 1e-6f + 1e-3f + (float)__builtin_fabs(base) * 0x1p-50f);
            uint32_t hits = 0;
            _Pragma("unroll") for (int c = 0; c < 16; ++c) hits |= x[c] >= bound ? 1u << c : 0u;
            for (hits &= ok; hits != 0; hits &= hits - 1) {
                const int c = __ffs((int)hits) - 1;
                float v = x[0];
                _Pragma("unroll") for (int q = 1; q < 16; ++q) v = c == q ? x[q] : v;
                if (!(v > NINF)) continue;
                const double score = score_of(S, row_k, v);
                if (score > none) visit(score, row_k, t0 + c, v);
            }
        }
    };
    for (bool counted = last_bin == kPickBins - 1 && listed > 4;; counted = true) {
        if (counted) {
            count_anew();
            each_token([&](double score, uint32_t, int, float) { count(bin_of(top, score)); });
            __syncthreads();
            last_bin = min(last_bin, bin_of_nth());
            if (tid == 0) S.n_elems = 0;
            __syncthreads();
        }
        if (state == ROW_ENDED && part == 0) list_candidate(S.base[k], place_of(k, -1), 0.f);
        each_token([&](double score, uint32_t row_k, int t, float v) { if (bin_of(top, score) <= last_bin) list_candidate(score, place_of(row_k, t), v); });
        __syncthreads();
        if (counted || S.n_elems <= 2 * N + 64) break;
    }
    if (S.n_pieces > kPickListed || listed_all > kPickListed || S.n_elems > kPickElems) { pick_one_by_one<E>(args, lds, g); return; }
    const uint32_t R = S.n_elems;
    for (;;) {
        // A candidate's place is the number of candidates before it: a wavefront compares 64 candidates with its part of all.
        // (16 of all for each, so that a few candidates take four wavefronts and no division)
        const uint32_t sixteenths = (R + 15) / 16;
        for (uint32_t i = lane; i < (R + 63) / 64 * 64; i += 64) {
            const Candidate c = S.found[i < R ? i : 0];
            uint32_t n = 0;
            for (uint32_t q = wave; q < sixteenths; q += waves) {
                const uint32_t to = min(q * 16 + 16, R);
                _Pragma("unroll 8") for (uint32_t j = q * 16; j < to; ++j) { const Candidate o = S.found[j]; n += before(o, c) ? 1u : 0u; }
            }
            if (i < R && n != 0) atomicAdd(&S.place[i], n);
        }
        __syncthreads();
        for (uint32_t i = tid; i < R; i += blockDim.x) { S.sorted[S.place[i]] = (uint16_t)i; S.place[i] = 0; }
        if (tid < K) S.repair[tid] = 0;
        __syncthreads();
        // Neighbours of different rows that are too close for their sums, among the chosen and those that are as close to the last of
        // them: these rows' sums in 64 bits.  (Two that are close and not neighbours have neighbours of different rows between them.)
        int any = 0;
        for (uint32_t n = tid; n + 1 < R; n += blockDim.x) {
            const Candidate a = S.found[S.sorted[n]], b = S.found[S.sorted[n + 1]];
            const uint32_t ka = (uint32_t)(a.at >> 32), kb = (uint32_t)(b.at >> 32);
            if (ka == kb || (S.exact[ka] && S.exact[kb]) || a.score - b.score > A.near) continue;
            if (n + 1 <= N || !(S.found[S.sorted[N - 1]].score - b.score > A.near)) { S.repair[ka] = S.repair[kb] = 1; any = 1; }
        }
        if (!__syncthreads_or(any)) break;
        for (uint32_t q = 0; q < K; ++q) if (S.repair[q] && !S.exact[q]) repair_row<E>(args, lds, g, q, false);
        for (uint32_t i = tid; i < R; i += blockDim.x)
            if ((uint32_t)S.found[i].at != 0) S.found[i].score = score_of(S, (uint32_t)(S.found[i].at >> 32), S.x[i]);
        __syncthreads();
    }
    if (tid < N) write_choice(A, g, tid, tid < R, tid < R ? S.found[S.sorted[tid]] : Candidate{0, 0});
}

template <class... P> using Kernel = void(P...);
static_assert(std::is_same_v<decltype(k_beam_pick<float>), Kernel<decltype(PickParams::all_stats), decltype(PickParams::scores), decltype(PickParams::finished), decltype(PickParams::K),
                                                                  decltype(PickParams::pieces), decltype(PickParams::N), decltype(PickParams::A)>> &&
              std::is_standard_layout_v<PickParams>, "k_beam_pick finds its last argument at its place in PickParams");

// ---- matcher slots --------------------------------------------------------------------------------------------------
// One workgroup per group of beams, a wavefront for up to SLOTS of its slots.  A slot's context has two buffers, and nobody reads the one
// that is not its own state, so the parent's goes there at once; the slot's record and its frontier planes have one place, so these
// wait in registers (the record a word a lane) until all wavefronts of the group have read theirs.  Bound by latency: three loads in a row
// (parents, records, context), so the first 64 of everything in a context are asked for together, without waiting for the counts (a slot
// has room for that many and more), like the planes.  4 slots 2.2 us, 512 slots in groups of 8 4.0 (with records in LDS and contexts asked
// for after their counts 4.0 and 9.0).
constexpr uint32_t kRowWords = sizeof(FillRow) / 4;
static_assert(kRowWords <= 64 && offsetof(FillRow, front_off) == 0 && offsetof(FillRow, front_n) == 4 && offsetof(FillRow, item_off) == 8 && offsetof(FillRow, item_n) == 12 &&
              offsetof(FillRow, wait_base) == 16 && offsetof(FillRow, waitoff_off) == 20 && offsetof(FillRow, H) == 24 && offsetof(FillRow, pad) == 36 && offsetof(FillRow, n_wait) == 44,
              "k_batch_reorder has a record a word a lane");
template <int SLOTS>
__global__ __launch_bounds__(1024) void k_batch_reorder(const int32_t* parents, FillRow* rows, uint32_t K, BatchDev D, int32_t* status) {
    const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), waves = blockDim.x >> 6, first = blockIdx.x * K;
    uint64_t plane[SLOTS];
    uint32_t word[SLOTS];
    bool moves[SLOTS];
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) {
        const uint32_t k = wave + (uint32_t)j * waves, b = first + k;
        moves[j] = false;
        if (k >= K) continue;
        const int32_t p = (int32_t)uniform((uint32_t)((Global<const int32_t>)parents)[b]);
        const bool in_group = p >= 0 && (uint32_t)p >= first && (uint32_t)p < first + K;
        if (status && lane == 0) ((Global<int32_t>)status)[b] = in_group || p == -1 ? kAccOk : kAccInvalid;
        if (!in_group || (uint32_t)p == b) continue;
        moves[j] = true;
        const uint32_t own = ((Global<const uint32_t>)(rows + b))[offsetof(FillRow, pad) / 4], w = lane < kRowWords ? ((Global<const uint32_t>)(rows + p))[lane] : 0u;
        auto field = [&](uint32_t at) { return (uint32_t)__builtin_amdgcn_readlane((int)w, (int)at); };
        const uint32_t to = uniform(own) ^ 1u, item_n = field(3), H = field(6), n_wait = field(11);
        const Global<const uint32_t> items = (Global<const uint32_t>)(D.items + field(2)), off = (Global<const uint32_t>)(D.wait_off + field(5));
        const Global<const uint64_t> wait = (Global<const uint64_t>)(D.wait + field(4));
        const size_t slot = (size_t)to * D.B + b;
        const Global<uint32_t> items_out = (Global<uint32_t>)(D.items + slot * D.KI), off_out = (Global<uint32_t>)(D.wait_off + slot * (D.KH + 1));
        const Global<uint64_t> wait_out = (Global<uint64_t>)(D.wait + slot * D.KW);
        const uint32_t item0 = items[lane], off0 = off[lane];
        const uint64_t wait0 = wait[lane];
        plane[j] = lane < D.KF ? ((Global<const uint64_t>)D.front)[(size_t)field(0) + lane] : 0u;
        if (lane < item_n) items_out[lane] = item0;
        if (lane <= H) off_out[lane] = off0;
        if (lane < n_wait) wait_out[lane] = wait0;
        for (uint32_t i = lane + 64; i <= H; i += 64) off_out[i] = off[i];
        for (uint32_t i = lane + 64; i < n_wait; i += 64) wait_out[i] = wait[i];
        // the record as it will be: places of its own, the rest the parent's
        word[j] = w;
        if (lane == 0) word[j] = b * D.KF;
        if (lane == 2) word[j] = (uint32_t)(slot * D.KI);
        if (lane == 4) word[j] = (uint32_t)(slot * D.KW);
        if (lane == 5) word[j] = (uint32_t)(slot * (D.KH + 1));
        if (lane == offsetof(FillRow, pad) / 4) word[j] = to;
    }
    // (what was loaded is there before any wavefront stores)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) {
        if (!moves[j]) continue;
        const uint32_t b = first + wave + (uint32_t)j * waves, n = (uint32_t)__builtin_amdgcn_readlane((int)word[j], 1);
        if (lane < n) ((Global<uint64_t>)D.front)[(size_t)b * D.KF + lane] = plane[j];
        if (lane < kRowWords) ((Global<uint32_t>)(rows + b))[lane] = word[j];
    }
}

// ---- rows of a buffer -----------------------------------------------------------------------------------------------
// A thread has one column of all rows of a group: it loads what every row will hold there and then stores it, so nothing waits for
// anybody and no second buffer is needed.  Rows that keep their place are neither read (but as parents) nor written.  Bound by memory:
// 32 groups of 8 beams, 472 MB read and written 90 us, 5.2 TB/s, what a large copy reaches.
// TOGETHER columns of a thread, `apart` bytes from one to the next, of which `n` exist.  (from: lane k has the row that row k takes; the
// lane's rows are picked by constants.  What a row's number makes of its stride is worked out anew where it is used: kept for all rows
// it would not fit the scalar registers.)
template <class T, int MOST, int TOGETHER, bool PAST>
__device__ __forceinline__ void move_columns(uint8_t* at, int64_t apart, int n, int64_t row_stride, uint32_t from, uint64_t moves) {
    T v[TOGETHER][MOST];
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("" : "+s"(row_stride));
#endif
#pragma unroll
    for (int k = 0; k < MOST; ++k) {
        if (!((moves >> k) & 1)) continue;
        const uint8_t* const row = at + (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)from, k) * row_stride;
        _Pragma("unroll") for (int j = 0; j < TOGETHER; ++j)
            if (j < n) v[j][k] = PAST ? __builtin_nontemporal_load((Global<const T>)(row + j * apart)) : *(Global<const T>)(row + j * apart);
    }
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("" : "+s"(row_stride));
#endif
#pragma unroll
    for (int k = 0; k < MOST; ++k) {
        if (!((moves >> k) & 1)) continue;
        uint8_t* const row = at + (int64_t)k * row_stride;
        _Pragma("unroll") for (int j = 0; j < TOGETHER; ++j) {
            if (j >= n) continue;
            if (PAST) __builtin_nontemporal_store(v[j][k], (Global<T>)(row + j * apart));
            else *(Global<T>)(row + j * apart) = v[j][k];
        }
    }
}

template <class T, int MOST, int TOGETHER, bool PAST>
__global__ __launch_bounds__(256) void k_beam_reorder_rows(const int32_t* parents, const int32_t* begins, const int32_t* ends, uint32_t K, uint32_t splits, uint32_t positions, BeamRows A) {
    const uint32_t split = blockIdx.x % splits, unit = blockIdx.x / splits, g = blockIdx.y + blockIdx.z * 32768u, lane = threadIdx.x & 63;
    if (g >= A.groups) return;
    const int32_t p = lane < K ? ((Global<const int32_t>)parents)[g * K + lane] : -1;
    int64_t begin = begins ? ((Global<const int32_t>)begins)[g] : 0, end = ends ? ((Global<const int32_t>)ends)[g] : (int64_t)positions;
    begin = begin < 0 ? 0 : begin;
    end = end > (int64_t)positions ? (int64_t)positions : end;
    if (begin >= end) return;
    const uint32_t from = (uint32_t)p - g * K;
    const uint64_t moves = __ballot(p >= 0 && from < K && from != lane);
    if (moves == 0) return;
    uint8_t* const piece = A.data + (int64_t)(g * K) * A.row_stride + (int64_t)(unit / A.pieces) * A.outer_stride + (int64_t)(unit % A.pieces) * A.piece_stride
                           + begin * A.position_bytes;
    constexpr int64_t SIZE = sizeof(T);
    const int64_t bytes = (end - begin) * A.position_bytes, whole = bytes / SIZE;
    for (int64_t v = (int64_t)split * 256 * TOGETHER + threadIdx.x; v < whole; v += (int64_t)splits * 256 * TOGETHER) {
        const int64_t left = (whole - v + 255) / 256;
        move_columns<T, MOST, TOGETHER, PAST>(piece + v * SIZE, 256 * SIZE, left < TOGETHER ? (int)left : TOGETHER, A.row_stride, from, moves);
    }
    const int64_t rest = whole * SIZE + threadIdx.x;                 // (less than a vector)
    if (split == 0 && rest < bytes) move_columns<uint8_t, MOST, 1, false>(piece + rest, 0, 1, A.row_stride, from, moves);
}

// Many beams: a column of all rows no longer fits a thread's registers with loads of 16 bytes, so a workgroup has a strip of 256 bytes of
// all rows in LDS, loads it whole and then stores it.  TB/s as below with strips of 128 / 256 / 512 / 1,024 bytes: 17 beams 2.7 / 3.7 / 3.4 / 2.3,
// 32 beams 4.1 / 4.6 / 4.0 / 2.7, 64 beams 4.5 / 4.7 / 4.1 / 3.1.
constexpr int kStripVecs = 16, kStripRows = 16;                       // vectors of a strip; rows that the 256 threads have at a time
template <bool PAST>
__global__ __launch_bounds__(256) void k_beam_reorder_strips(const int32_t* parents, const int32_t* begins, const int32_t* ends, uint32_t K, uint32_t splits, uint32_t positions, BeamRows A) {
    constexpr int TURNS = kBeamsMost / kStripRows;
    __shared__ Vec4 strip[kBeamsMost][kStripVecs];
    const uint32_t split = blockIdx.x % splits, unit = blockIdx.x / splits, g = blockIdx.y + blockIdx.z * 32768u, lane = threadIdx.x & 63;
    if (g >= A.groups) return;
    const int32_t p = lane < K ? ((Global<const int32_t>)parents)[g * K + lane] : -1;
    int64_t begin = begins ? ((Global<const int32_t>)begins)[g] : 0, end = ends ? ((Global<const int32_t>)ends)[g] : (int64_t)positions;
    begin = begin < 0 ? 0 : begin;
    end = end > (int64_t)positions ? (int64_t)positions : end;
    if (begin >= end) return;
    const uint32_t from = (uint32_t)p - g * K;
    const bool moving = p >= 0 && from < K && from != lane;
    const uint64_t moves = __ballot(moving);
    if (moves == 0) return;
    uint64_t sources = 0;                                            // rows that a row takes
    for (uint32_t k = 0; k < K; ++k) sources |= __ballot(moving && from == k) != 0 ? 1ull << k : 0ull;
    uint8_t* const piece = A.data + (int64_t)(g * K) * A.row_stride + (int64_t)(unit / A.pieces) * A.outer_stride + (int64_t)(unit % A.pieces) * A.piece_stride
                           + begin * A.position_bytes;
    const int64_t bytes = (end - begin) * A.position_bytes, whole = bytes / 16;
    const uint32_t own = threadIdx.x % kStripVecs, first = threadIdx.x / kStripVecs;
    uint32_t takes[TURNS];                                           // the row that this thread's rows take
    _Pragma("unroll") for (int j = 0; j < TURNS; ++j) takes[j] = (uint32_t)__shfl((int)from, (int)(first + j * kStripRows));
    for (int64_t v0 = (int64_t)split * kStripVecs; v0 < whole; v0 += (int64_t)splits * kStripVecs) {
        const bool inside = v0 + own < whole;
        uint8_t* const at = piece + (v0 + own) * 16;
        Wide4 v[TURNS];
        _Pragma("unroll") for (int j = 0; j < TURNS; ++j) {
            const uint32_t k = first + j * kStripRows;
            if (!inside || !((sources >> k) & 1)) continue;
            const Global<const Wide4> place = (Global<const Wide4>)(at + (int64_t)k * A.row_stride);
            v[j] = PAST ? __builtin_nontemporal_load(place) : *place;
        }
        _Pragma("unroll") for (int j = 0; j < TURNS; ++j) {
            const uint32_t k = first + j * kStripRows;
            if (inside && ((sources >> k) & 1)) strip[k][own] = v[j];
        }
        __syncthreads();
        _Pragma("unroll") for (int j = 0; j < TURNS; ++j) {
            const uint32_t k = first + j * kStripRows;
            if (!inside || !((moves >> k) & 1)) continue;
            const Wide4 w = strip[takes[j]][own];
            const Global<Wide4> place = (Global<Wide4>)(at + (int64_t)k * A.row_stride);
            if (PAST) __builtin_nontemporal_store(w, place);
            else *place = w;
        }
        __syncthreads();
    }
    const int64_t rest = whole * 16 + threadIdx.x;                   // (less than a vector)
    if (split == 0 && rest < bytes) move_columns<uint8_t, kBeamsMost, 1, false>(piece + rest, 0, 1, A.row_stride, from, moves);
}

// ---- sequences ------------------------------------------------------------------------------------------------------
// A chain of as many look-ups as there are steps, one behind the other; but where the beams behind a segment of the steps come from
// before it does not hang on the other segments.  So the steps are cut into segments, each worked out by WIDTH lanes of a wavefront (a
// beam each): first every segment's map from the beams behind it to those before it, then the maps of all segments from each one on,
// put together two and two (in as many rounds as the number of segments has binary digits), then every segment again from the beams
// that the sequences enter it with, writing their tokens.  A step's parents are one load for all beams of a group, which waits for nothing;
// which of them a beam's is comes from the lane that holds it.  Segments of up to kTraceHeld steps are loaded once and kept in registers.
// Bound by latency (the loads, then some 30 exchanges of about 50 ns).  4 beams, 128 steps 4.8 us, 64 groups of 8 beams, 1,500 steps 9.4 us;
// a thread per sequence, step after step 22.4 and 537.
constexpr int kTraceThreads = 1024, kTraceHeld = 16;
template <int WIDTH>
__global__ __launch_bounds__(kTraceThreads) void k_beam_backtrace(BeamTrace A, uint32_t segments, uint32_t length) {
    constexpr uint32_t NONE = 255;
    __shared__ uint8_t maps[2][kTraceThreads];                       // [segment * WIDTH + beam behind it]: the beam before it
    __shared__ int32_t last[WIDTH];                                  // steps up to and with a sequence's last token
    // (groups that lie side by side share cache lines of a step: they go to one die, which every eighth workgroup does)
    const uint32_t g = blockIdx.x % 8 * ((A.groups + 7) / 8) + blockIdx.x / 8;
    if (g >= A.groups) return;
    const uint32_t K = A.beams, lane = threadIdx.x & 63, k = lane % WIDTH, base = lane - k, first = g * K, s = threadIdx.x / WIDTH;
    const uint32_t from = s * length, to = s < segments ? min(from + length, A.steps) : from;
    const bool mine = k < K;
    const uint32_t row = first + (mine ? k : 0);
    const Global<const int32_t> parents = (Global<const int32_t>)A.parents, tokens = (Global<const int32_t>)A.tokens;
    uint32_t beam[kTraceHeld];                                       // of the parent, NONE if it is not of the group
    int32_t token[kTraceHeld];
    // steps from the segment's end on, `done` of them already walked (the loops are the same in all lanes of a wavefront)
    auto load = [&](uint32_t done, bool with_tokens) {
        _Pragma("unroll") for (int i = 0; i < kTraceHeld; ++i) {
            if (from + done + i < to) {
                const int64_t t = (int64_t)(to - 1 - done - i) * A.step_stride + row;
                beam[i] = (uint32_t)parents[t] - first;
                if (with_tokens) token[i] = tokens[t];
            }
        }
    };
    auto step = [&](uint32_t at, uint32_t next) { return at >= K ? NONE : next < K ? next : NONE; };
    const bool held = length <= kTraceHeld;
    load(0, held);
    if (threadIdx.x < WIDTH) last[threadIdx.x] = 0;
    uint32_t at = mine ? k : NONE;
    for (uint32_t done = 0; done < length; done += kTraceHeld) {
        if (done != 0) load(done, false);
        _Pragma("unroll") for (int i = 0; i < kTraceHeld; ++i) {
            const uint32_t next = (uint32_t)__shfl((int)beam[i], (int)(base + at % WIDTH));
            if (from + done + i < to) at = step(at, next);
        }
    }
    maps[0][threadIdx.x] = (uint8_t)at;
    __syncthreads();
    // maps[s] becomes the map from the end of all steps to before segment s
    uint32_t turn = 0;
    for (uint32_t d = 1; d < segments; d *= 2) {
        if (s + d < segments) {
            const uint32_t behind = maps[turn][threadIdx.x + d * WIDTH];
            at = behind < K ? maps[turn][s * WIDTH + behind] : NONE;
        }
        turn ^= 1;
        maps[turn][threadIdx.x] = (uint8_t)at;
        __syncthreads();
    }
    at = !mine ? NONE : s + 1 < segments ? maps[turn][threadIdx.x + WIDTH] : k;
    int32_t end = 0;
    const Global<int32_t> out = (Global<int32_t>)(A.out + (int64_t)row * A.out_stride);
    for (uint32_t done = 0; done < length; done += kTraceHeld) {
        if (!held) load(done, true);
        _Pragma("unroll") for (int i = 0; i < kTraceHeld; ++i) {
            const int source = (int)(base + at % WIDTH);
            const uint32_t next = (uint32_t)__shfl((int)beam[i], source);
            const int32_t t = __shfl(token[i], source);
            token[i] = at < K ? t : -1;
            if (from + done + i < to) at = step(at, next);
        }
        if (!mine) continue;
        _Pragma("unroll") for (int i = 0; i < kTraceHeld; i += 4) {
            const uint32_t n = done + i;
            if (from + n + 3 < to) {
                *(Global<Wide4>)(out + (to - 4 - n)) = Wide4{(uint32_t)token[i + 3], (uint32_t)token[i + 2], (uint32_t)token[i + 1], (uint32_t)token[i]};
                _Pragma("unroll") for (int j = 0; j < 4; ++j) if (token[i + j] >= 0) end = max(end, (int32_t)(to - n - j));
            } else {
                _Pragma("unroll") for (int j = 0; j < 4; ++j) {
                    if (from + n + j >= to) continue;
                    out[to - 1 - n - j] = token[i + j];
                    if (token[i + j] >= 0) end = max(end, (int32_t)(to - n - j));
                }
            }
        }
    }
    if (end > 0) atomicMax(&last[k], end);
    __syncthreads();
    if (A.lengths && threadIdx.x < K) ((Global<int32_t>)A.lengths)[first + threadIdx.x] = last[threadIdx.x];
}

}  // namespace

template <class E>
static void launch_beam_select_as(const BeamSelect& A, hipStream_t stream) {
    const uint32_t rows = A.groups * A.beams;
    auto* const kernel = !A.bitmask ? k_beam_scan<E, 0> : A.over_all ? k_beam_scan<E, 2> : k_beam_scan<E, 1>;
    for (uint32_t first = 0; first < rows; first += 65535) {         // grid.y limit
        const uint32_t n = std::min<uint32_t>(65535, rows - first);
        hipLaunchKernelGGL(kernel, dim3((A.pieces + kScanWaves - 1) / kScanWaves, n), dim3(64 * kScanWaves), 0, stream, A.bitmask, A.bm_stride, A.scores, A.finished, A.logits, A.row_stride, A.pieces, A.V, A, first);
    }
    // 16 lanes for every row, four for every block that is looked at
    const uint32_t threads = std::min<uint32_t>(kPickThreads, std::max<uint32_t>(256, (std::max(16 * A.beams, 4 * (A.n_out + A.n_out / 4)) + 63) / 64 * 64));
    hipLaunchKernelGGL(k_beam_pick<E>, dim3(A.groups), dim3(threads), 0, stream, A.stats, A.scores, A.finished, A.beams, A.pieces, A.n_out, A);
}

void launch_beam_select(const BeamSelect& A, hipStream_t stream) {
    if (A.groups == 0) return;
    if (A.dtype == XG2_F32) launch_beam_select_as<float>(A, stream);
    else launch_beam_select_as<uint16_t>(A, stream);
}

void launch_batch_reorder(const BatchDev& D, uint32_t beams, const int32_t* parents_dev, int32_t* status_dev, hipStream_t stream) {
    static_assert(kSlotItems == 64 && kSlotSets + 1 >= 64 && kSlotWaits >= 64 && kSlotPlanes <= 64, "a wavefront asks for the first 64 of everything");
    if (D.B == 0) return;
    const dim3 grid(D.B / beams), block(64 * std::min<uint32_t>(beams, 16));
    if (beams <= 16) hipLaunchKernelGGL(k_batch_reorder<1>, grid, block, 0, stream, parents_dev, D.rows, beams, D, status_dev);
    else hipLaunchKernelGGL(k_batch_reorder<4>, grid, block, 0, stream, parents_dev, D.rows, beams, D, status_dev);
}

// Buffers beyond the last-level cache (256 MB) are moved past it: what is moved is not there when attention reads the whole buffer, moved or
// not.  Through the caches / past them, us, 8 beams, 64 pieces of 32 kB a row: 256 MB (below the line) 53.4 / 48.5, 320 MB 66.6 / 60.5,
// 512 MB 98.9 / 90.7; below the line what is left in the cache is worth more to the next reader.
// A piece is cut into at most 16 parts where there are many, or so many that there are 4,096 workgroups: a part beyond a group's window
// costs a workgroup that finds nothing to do (19 groups, 6 pieces of 313 kB, windows of a quarter, at most 64 / 16 / 8 parts: 16.0 / 13.1 / 13.4
// us; one piece of 100 MB a row, 16 / 64 / 4,096 parts: 806 / 219 / 46).
constexpr int64_t ROWS_PAST_BYTES = 256ll << 20;
constexpr uint32_t ROWS_SPLITS = 16, ROWS_GROUPS = 4096;

// A workgroup takes `vectors_each` vectors of `vector` bytes of a piece at a time.
template <class K>
static void launch_rows(const BeamRows& A, hipStream_t stream, int64_t vector, uint32_t vectors_each, K* near, K* past_caches) {
    const uint32_t units = A.outer * A.pieces;
    const int64_t piece = A.positions * A.position_bytes, vectors = piece / vector;
    const uint64_t all = (uint64_t)units * A.groups, most = std::max<uint64_t>(ROWS_SPLITS, ROWS_GROUPS / all);
    uint32_t splits = (uint32_t)std::min<uint64_t>((uint64_t)vectors / vectors_each + 1, most);
    splits = std::max<uint32_t>(1, std::min<uint32_t>(splits, (1u << 23) / units));            // (a grid has less than 2^32 threads)
    const bool past = (double)piece * (double)all * A.beams > (double)ROWS_PAST_BYTES;
    hipLaunchKernelGGL(past ? past_caches : near, dim3(units * splits, std::min<uint32_t>(A.groups, 32768), (A.groups + 32767) / 32768), dim3(256), 0, stream,
                       A.parents, A.begin, A.end, A.beams, splits, A.positions, A);
}

template <class T, int MOST, int TOGETHER>
static void launch_rows_as(const BeamRows& A, hipStream_t stream) {
    launch_rows(A, stream, sizeof(T), 256 * TOGETHER, k_beam_reorder_rows<T, MOST, TOGETHER, false>, k_beam_reorder_rows<T, MOST, TOGETHER, true>);
}

// What a thread holds of each row, and how many columns of it.  TB/s over 537 MB (rows of 256 positions of 128 bytes, moved bytes counted
// once read and once written), 2 / 4 / 8 / 16 / 17 / 32 / 33 / 64 beams: 16 bytes, one column 3.3 / 5.4 / 5.2 / 4.8 / - / 3.9 / - / -, two columns
// 4.8 / 5.1 / 5.0 (their registers cost wavefronts), 4 bytes - / - / - / - / 4.1 / 4.2 / 2.6 / 3.3, strips in LDS - / - / - / - / 3.7 / 4.6 / 4.5 / 4.7.
// (Columns of 4 bytes were a tenth faster at 17 beams; strips are all that is kept above 16, since they are the faster ones at 32 and above.)
void launch_beam_reorder_rows(const BeamRows& A, hipStream_t stream) {
    if (A.beams <= 2) launch_rows_as<Wide4, 2, 2>(A, stream);
    else if (A.beams <= 4) launch_rows_as<Wide4, 4, 1>(A, stream);
    else if (A.beams <= 8) launch_rows_as<Wide4, 8, 1>(A, stream);
    else if (A.beams <= 16) launch_rows_as<Wide4, 16, 1>(A, stream);
    else launch_rows(A, stream, 16, kStripVecs, k_beam_reorder_strips<false>, k_beam_reorder_strips<true>);
}

template <int WIDTH>
static void launch_backtrace_as(const BeamTrace& A, hipStream_t stream) {
    // as many segments as a workgroup has room for, of eight steps at the least
    constexpr uint32_t most = kTraceThreads / WIDTH;
    const uint32_t length = std::max<uint32_t>(8, (A.steps + most - 1) / most), segments = (A.steps + length - 1) / length;
    const uint32_t threads = std::max<uint32_t>(64, (segments * WIDTH + 63) / 64 * 64);
    hipLaunchKernelGGL(k_beam_backtrace<WIDTH>, dim3((A.groups + 7) / 8 * 8), dim3(threads), 0, stream, A, segments, length);
}

void launch_beam_backtrace(const BeamTrace& A, hipStream_t stream) {
    if (A.groups == 0) return;
    if (A.beams <= 4) launch_backtrace_as<4>(A, stream);
    else if (A.beams <= 8) launch_backtrace_as<8>(A, stream);
    else if (A.beams <= 16) launch_backtrace_as<16>(A, stream);
    else if (A.beams <= 32) launch_backtrace_as<32>(A, stream);
    else launch_backtrace_as<64>(A, stream);
}

}  // namespace xg2
