// gfx950 (CDNA4, wave64) kernels of beam search under a grammar:
//   k_beam_scan          one pass over the logits: sums of exponentials and the largest allowed logit of every block of tokens
//   k_beam_pick          the best candidates of a group, from the blocks that can hold them
//   k_batch_reorder      matcher slots take over the state of their parents
//   k_beam_reorder_rows  the same for rows of a caller's buffer, in place
//   k_beam_backtrace     sequences from the steps' tokens and parents
#include <algorithm>

#include "beam.hpp"

namespace xg2 {
namespace {

constexpr float NINF = -__builtin_inff();

__device__ __forceinline__ uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }

// ---- selection ------------------------------------------------------------------------------------------------------
// score(row, token) = s_row - L_row + x, L_row = log of the sum of exp x over the tokens that count.  Chosen are the n best of all rows
// of a group.  A candidate among the n best lies in one of the n blocks (of kBeamBlock consecutive tokens) whose best tokens are the
// best, so one pass over the logits leaves two things of them: for every piece of kBeamPiece tokens the largest logit M that counts and
// the sum of exp(x - M), and for every block its largest allowed logit.  The second kernel has the rows' L from the first, takes the
// blocks whose best score is not below the n-th best of them, and looks at the tokens of these blocks only.
constexpr int kScanWaves = 4;
constexpr float LOG2E = 1.44269504088896340736f;
constexpr double LN2 = 0.693147180559945309417232;

template <class E> struct Elem;
template <> struct Elem<float> {
    static constexpr int EPV = 4;
    static __device__ __forceinline__ float value(float e) { return e; }
    static __device__ __forceinline__ void unpack(const uint4& v, float* x) { x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w); }
};
struct Bf16 { uint16_t bits; };
template <> struct Elem<Bf16> {
    static constexpr int EPV = 8;
    static __device__ __forceinline__ float value(Bf16 e) { return __uint_as_float((uint32_t)e.bits << 16); }
    static __device__ __forceinline__ void unpack(const uint4& v, float* x) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        _Pragma("unroll") for (int k = 0; k < 4; ++k) { x[2 * k] = __uint_as_float(w[k] << 16); x[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u); }
    }
};

// The larger of two numbers; a NaN loses.
__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }

// Elements of a row before the 128-byte boundary that its pieces and blocks are counted from.
template <class E> __device__ __forceinline__ int before_row(const E* row) { return (int)(reinterpret_cast<uintptr_t>(row) & 127) / (int)sizeof(E); }

// A row whose beam has ended or does not exist is not read.
__device__ __forceinline__ bool live_row(const BeamSelect& A, uint32_t r) {
    const float s = A.scores[r];
    return !(A.finished && A.finished[r] != 0) && s > NINF && s < -NINF;
}

// WHICH: 0 no mask, 1 the softmax goes over the allowed tokens, 2 over all.
template <class E, int WHICH>
__global__ __launch_bounds__(64 * kScanWaves) void k_beam_scan(BeamSelect A, uint32_t first_row) {
    constexpr int EPV = Elem<E>::EPV, STEPS = kBeamPiece / 64 / EPV, LANES = kBeamBlock / EPV;   // lanes that share a block
    constexpr uint32_t ALL = (1u << EPV) - 1;
    const uint32_t r = first_row + blockIdx.y, lane = threadIdx.x & 63, piece = blockIdx.x * kScanWaves + uniform(threadIdx.x >> 6);
    if (piece >= A.pieces || !live_row(A, r)) return;
    const E* const row = static_cast<const E*>(A.logits) + (long long)r * A.row_stride;
    const int V = A.V;
    const long long e0 = (long long)piece * kBeamPiece - before_row(row);
    const bool inner = e0 >= 0 && e0 + kBeamPiece <= V;
    // this lane's 32 tokens from e0 + 32 * lane on: which are in the row, and which of them are allowed
    const long long first = e0 + 32 * (long long)lane;
    uint32_t inside = ~0u;
    if (!inner) {
        if (first < 0) inside = first <= -32 ? 0 : ~0u << -first;
        if (first + 32 > V) inside &= first >= V ? 0 : ~0u >> (first + 32 - V);
    }
    uint32_t allowed = inside;
    if (WHICH != 0) {
        const uint32_t* const bm = A.bitmask + (long long)r * A.bm_stride;
        const long long at = first >> 5, last = (V - 1) >> 5;       // (an arithmetic shift: rounds down)
        const int shift = (int)(e0 & 31);                            // (the same in all lanes)
        uint32_t word = at >= 0 && at <= last ? bm[at] : 0;
        if (shift != 0) {
            const uint32_t next = at + 1 >= 0 && at + 1 <= last ? bm[at + 1] : 0;
            word = (word >> shift) | (next << (32 - shift));
        }
        allowed &= word;
    }
    const uint32_t counted = WHICH == 1 ? allowed : inside;
    float2* const stats = A.stats + ((size_t)r * A.pieces + piece);
    float* const block_max = A.block_max + ((size_t)r * A.pieces + piece) * kBeamPieceBlocks;
    if (WHICH == 1 && __ballot(counted != 0) == 0) {
        if (lane == 0) *stats = make_float2(NINF, 0.f);
        if (lane < kBeamPieceBlocks) block_max[lane] = NINF;
        return;
    }
    const E* const from = row + e0;
    uint4 raw[STEPS];
    uint32_t bits[STEPS];
#pragma unroll
    for (int j = 0; j < STEPS; ++j) {
        const int v = j * 64 + (int)lane;
        bits[j] = ((uint32_t)__shfl((int)counted, v / (32 / EPV)) >> (v % (32 / EPV) * EPV)) & ALL;
        raw[j] = make_uint4(0, 0, 0, 0);
        const long long e = e0 + v * EPV;
        if (bits[j] != 0) {
            if (e >= 0 && e + EPV <= V) raw[j] = reinterpret_cast<const uint4*>(from)[v];
            else {                                                   // a vector that the row shares with its neighbours
                E part[EPV] = {};
                for (int c = 0; c < EPV; ++c) if (e + c >= 0 && e + c < V) part[c] = row[e + c];
                __builtin_memcpy(&raw[j], part, 16);
            }
        }
    }
    float x[STEPS][EPV], top = NINF;
#pragma unroll
    for (int j = 0; j < STEPS; ++j) {
        Elem<E>::unpack(raw[j], x[j]);
        _Pragma("unroll") for (int c = 0; c < EPV; ++c) if (!((bits[j] >> c) & 1)) x[j][c] = NINF;
        float m = NINF, best;
        _Pragma("unroll") for (int c = 0; c < EPV; ++c) m = larger(m, x[j][c]);
        top = larger(top, m);
        best = m;
        if (WHICH == 2) {
            const int v = j * 64 + (int)lane;
            const uint32_t ok = ((uint32_t)__shfl((int)allowed, v / (32 / EPV)) >> (v % (32 / EPV) * EPV)) & ALL;
            best = NINF;
            _Pragma("unroll") for (int c = 0; c < EPV; ++c) best = larger(best, (ok >> c) & 1 ? x[j][c] : NINF);
        }
        _Pragma("unroll") for (int d = 1; d < LANES; d *= 2) best = larger(best, __shfl_xor(best, d));
        if (lane % LANES == 0) block_max[j * (64 / LANES) + (int)lane / LANES] = best;
    }
    _Pragma("unroll") for (int d = 1; d < 64; d *= 2) top = larger(top, __shfl_xor(top, d));
    float sum = 0;
    if (top > NINF) {
        const float c = __fmul_rn(top, LOG2E);
        // (added up as a tree: 11 additions between a term and the sum, which is what its error is derived from)
        float part[STEPS * EPV];
        _Pragma("unroll") for (int i = 0; i < STEPS * EPV; ++i) part[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i / EPV][i % EPV], LOG2E, -c));
        _Pragma("unroll") for (int d = STEPS * EPV / 2; d > 0; d /= 2)
            _Pragma("unroll") for (int i = 0; i < d; ++i) part[i] += part[i + d];
        sum = part[0];
        _Pragma("unroll") for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    }
    if (lane == 0) *stats = make_float2(top, sum);
}

// ---- the best candidates of a group ---------------------------------------------------------------------------------
// One workgroup per group.  How near a score is to the best is measured in bins whose width grows with the distance (64 to an octave
// from 2^-6 on), so that one count over the blocks' best scores gives a line that at least n of them lie above and few more.
constexpr int kPickThreads = 1024, kPickBins = 1024, kPickBlocks = 1024, kPickElems = 2048;
enum RowState : uint32_t { ROW_NONE, ROW_LIVE, ROW_ENDED };
struct PickShared {
    double base[kBeamsMost];                   // score of a token of the row: base + its logit (infinite: base, where the logit is +inf)
    uint32_t state[kBeamsMost];
    uint32_t infinite[kBeamsMost], exact[kBeamsMost], repair[kBeamsMost];
    double near_top[kPickThreads / 64];
    uint32_t bins[kPickBins];
    uint32_t blocks[kPickBlocks];              // row in the group * blocks of a row + block
    uint32_t n_blocks, n_elems, last_bin, any, found;
    double score[kPickElems];
    float x[kPickElems];
    int32_t token[kPickElems];
    uint16_t row[kPickElems];
    uint16_t sorted[kPickElems];
    double r_score[kPickThreads / 64];
    uint32_t r_row[kPickThreads / 64];
    long long r_at[kPickThreads / 64];
};

__device__ __forceinline__ uint32_t bin_of(double top, double score) {
    const float d = (float)(top - score) + 0.015625f;                // (monotone: each step rounds one way for all)
    const uint32_t b = (__float_as_uint(d) >> 17) - (__float_as_uint(0.015625f) >> 17);
    return b < kPickBins - 1 ? b : kPickBins - 1;
}
__device__ __forceinline__ double score_of(const PickShared& S, uint32_t k, float x) {
    return S.base[k] + (double)(S.infinite[k] ? (x == -NINF ? 0.f : NINF) : x);
}
__device__ __forceinline__ bool token_allowed(const BeamSelect& A, uint32_t r, long long t) {
    return !A.bitmask || ((A.bitmask[(long long)r * A.bm_stride + (t >> 5)] >> (t & 31)) & 1u);
}

// The row's sum in 64 bits, and its blocks' maxima without NaN: what the first kernel left of the row is not used.
template <class E>
__device__ void repair_row(const BeamSelect& A, PickShared& S, uint32_t g, uint32_t k) {
    const uint32_t r = g * A.beams + k, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n_blocks = A.pieces * kBeamPieceBlocks;
    const E* const row = static_cast<const E*>(A.logits) + (long long)r * A.row_stride;
    const int before = before_row(row);
    float* const block_max = A.block_max + (size_t)r * n_blocks;
    float top = NINF;
    __syncthreads();                                                 // (S.near_top has been read by all)
    for (uint32_t b = wave; b < n_blocks; b += kPickThreads / 64) {
        float best = NINF;
        for (int c = 0; c < kBeamBlock; c += 64) {
            const long long t = (long long)b * kBeamBlock - before + c + lane;
            if (t < 0 || t >= A.V) continue;
            const float x = Elem<E>::value(row[t]);
            const bool ok = token_allowed(A, r, t);
            if (x != x) continue;
            if (ok) best = x > best ? x : best;
            if (ok || A.over_all) top = x > top ? x : top;
        }
        for (int d = 1; d < 64; d *= 2) { const float o = __shfl_xor(best, d); best = o > best ? o : best; }
        if (lane == 0) block_max[b] = best;
    }
    for (int d = 1; d < 64; d *= 2) { const float o = __shfl_xor(top, d); top = o > top ? o : top; }
    if (lane == 0) S.near_top[wave] = top;
    __syncthreads();
    for (int w = 0; w < kPickThreads / 64; ++w) top = (float)S.near_top[w] > top ? (float)S.near_top[w] : top;
    __syncthreads();
    double sum = 0;
    for (long long t = tid; t < A.V; t += kPickThreads) {
        const float x = Elem<E>::value(row[t]);
        if (x != x || x == NINF || !(A.over_all || token_allowed(A, r, t))) continue;
        if (top == -NINF) sum += x == top ? 1.0 : 0.0;
        else sum += exp((double)x - (double)top);
    }
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    if (lane == 0) S.near_top[wave] = sum;
    __syncthreads();
    if (tid == 0) {
        double total = 0;
        for (int w = 0; w < kPickThreads / 64; ++w) total += S.near_top[w];
        S.exact[k] = 1;
        if (top == NINF) S.state[k] = ROW_NONE;
        else {
            S.infinite[k] = top == -NINF;
            S.base[k] = (double)A.scores[r] - (log(total) + (top == -NINF ? 0.0 : (double)top));
        }
    }
    __threadfence_block();
    __syncthreads();
}

// Whether candidate a comes before candidate b.
__device__ __forceinline__ bool before(double sa, uint32_t ra, long long ta, double sb, uint32_t rb, long long tb) {
    return sa > sb || (sa == sb && (ra < rb || (ra == rb && ta < tb)));
}

// The best of all threads' candidates, in all threads (row ~0: none).
__device__ void best_of_all(PickShared& S, double& s, uint32_t& r, long long& t) {
    for (int d = 1; d < 64; d *= 2) {
        const double os = __shfl_xor(s, d);
        const uint32_t orow = (uint32_t)__shfl_xor((int)r, d);
        const long long ot = __shfl_xor(t, d);
        if (orow != ~0u && (r == ~0u || before(os, orow, ot, s, r, t))) { s = os; r = orow; t = ot; }
    }
    const uint32_t wave = threadIdx.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) { S.r_score[wave] = s; S.r_row[wave] = r; S.r_at[wave] = t; }
    __syncthreads();
    for (int w = 0; w < kPickThreads / 64; ++w)
        if (S.r_row[w] != ~0u && (r == ~0u || before(S.r_score[w], S.r_row[w], S.r_at[w], s, r, t))) { s = S.r_score[w]; r = S.r_row[w]; t = S.r_at[w]; }
}

__device__ __forceinline__ void write_choice(const BeamSelect& A, const PickShared& S, uint32_t g, uint32_t n, bool any, double s, uint32_t k, int32_t token) {
    const size_t at = (size_t)g * A.n_out + n;
    A.out_scores[at] = any ? (float)s : NINF;
    A.out_parents[at] = any ? (int32_t)(g * A.beams + k) : -1;
    A.out_tokens[at] = any ? token : -1;
    if (A.out_finished) A.out_finished[at] = !any || token < 0 || token == A.eos_id;
}

template <class E>
__global__ __launch_bounds__(kPickThreads) void k_beam_pick(BeamSelect A) {
    __shared__ PickShared S;
    const uint32_t g = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), K = A.beams, n_blocks = A.pieces * kBeamPieceBlocks, N = A.n_out;
    constexpr uint32_t WAVES = kPickThreads / 64;
    for (uint32_t i = tid; i < kPickBins; i += kPickThreads) S.bins[i] = 0;
    if (tid == 0) S.n_blocks = S.n_elems = S.any = S.found = 0;
    __syncthreads();
    // the rows' sums
    double top = -(double)__builtin_inff();                          // no score is above it
    for (uint32_t k = wave; k < K; k += WAVES) {
        const uint32_t r = g * K + k;
        const float s = A.scores[r];
        uint32_t state = !(s > NINF && s < -NINF) ? ROW_NONE : A.finished && A.finished[r] != 0 ? ROW_ENDED : ROW_LIVE, repair = 0;
        double base = s;
        if (state == ROW_LIVE) {
            const float2* const stats = A.stats + (size_t)r * A.pieces;
            float m = NINF;
            bool odd = false;
            for (uint32_t p = lane; p < A.pieces; p += 64) {
                const float2 v = stats[p];
                odd |= !(v.y < -NINF) || v.x != v.x || (v.x > NINF && !(v.x > -1e38f && v.x < 1e38f));
                m = v.x > m ? v.x : m;
            }
            for (int d = 1; d < 64; d *= 2) { const float o = __shfl_xor(m, d); m = o > m ? o : m; }
            // a NaN or an infinity among what counts, or magnitudes that the sum's exponents cannot take: from the logits again
            repair = __ballot(odd) != 0;
            if (repair) {}
            else if (m == NINF) state = ROW_NONE;
            else {
                // a piece's sum is of 2^(x * LOG2E - c), c = the rounded product of its maximum and LOG2E; LOG2E itself is off by `off`
                const double off = (double)LOG2E - 1.4426950408889634073599, mc = (double)__fmul_rn(m, LOG2E) - (double)m * off;
                double sum = 0;
                for (uint32_t p = lane; p < A.pieces; p += 64) {
                    const float2 v = stats[p];
                    if (v.x > NINF) sum += (double)v.y * exp2((double)__fmul_rn(v.x, LOG2E) - (double)v.x * off - mc);
                }
                for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
                base -= log(sum) + mc * LN2;
                top = base + m > top ? base + m : top;
            }
        } else if (state == ROW_ENDED) top = base > top ? base : top;
        if (lane == 0) {
            S.state[k] = state; S.base[k] = base; S.infinite[k] = 0; S.exact[k] = state != ROW_LIVE; S.repair[k] = repair;
            if (repair) S.any = 1;
        }
    }
    if (lane == 0) S.near_top[wave] = top;
    __syncthreads();
    for (uint32_t w = 0; w < WAVES; ++w) top = S.near_top[w] > top ? S.near_top[w] : top;
    if (S.any) {                                                     // (the same in all threads)
        for (uint32_t k = 0; k < K; ++k) {
            if (!S.repair[k]) continue;
            repair_row<E>(A, S, g, k);
            // (a bound: no logit of the row is above its largest)
            if (S.state[k] != ROW_LIVE) continue;
            float m = NINF;
            for (uint32_t b = lane; b < n_blocks; b += 64) { const float o = A.block_max[(size_t)(g * K + k) * n_blocks + b]; m = o > m ? o : m; }
            for (int d = 1; d < 64; d *= 2) { const float o = __shfl_xor(m, d); m = o > m ? o : m; }
            const double s = score_of(S, k, m);
            top = s > top ? s : top;
        }
        __syncthreads();
    }
    const uint32_t steps = (n_blocks + 63) / 64, units = K * steps;
    // how many blocks (and ended beams) have their best score in each bin
    for (uint32_t u = wave; u < units; u += WAVES) {
        const uint32_t k = u / steps, b = u % steps * 64 + lane;
        if (S.state[k] != ROW_LIVE || b >= n_blocks) continue;
        const double s = score_of(S, k, A.block_max[(size_t)(g * K + k) * n_blocks + b]);
        if (s > -(double)__builtin_inff()) atomicAdd(&S.bins[bin_of(top, s)], 1u);
    }
    if (tid < K && S.state[tid] == ROW_ENDED) atomicAdd(&S.bins[bin_of(top, S.base[tid])], 1u);
    __syncthreads();
    if (wave == 0) {
        constexpr uint32_t EACH = kPickBins / 64;
        uint32_t mine = 0;
        for (uint32_t i = 0; i < EACH; ++i) mine += S.bins[lane * EACH + i];
        uint32_t upto = mine;
        for (int d = 1; d < 64; d *= 2) { const uint32_t o = (uint32_t)__shfl_up((int)upto, d); if ((int)lane >= d) upto += o; }
        const unsigned long long reached = __ballot(upto >= N);
        if (reached == 0) { if (lane == 0) S.last_bin = kPickBins - 1; }
        else if ((int)lane == __ffsll((long long)reached) - 1) {
            uint32_t n = upto - mine, i = 0;
            for (; i < EACH; ++i) { n += S.bins[lane * EACH + i]; if (n >= N) break; }
            S.last_bin = lane * EACH + i + 1;                        // one bin more: what lies within A.near of the n-th best
        }
    }
    __syncthreads();
    const uint32_t last_bin = S.last_bin;
    // the blocks that can hold one of the n best, and of them and the ended beams the candidates that can be one
    for (uint32_t u = wave; u < units; u += WAVES) {
        const uint32_t k = u / steps, b = u % steps * 64 + lane;
        if (S.state[k] != ROW_LIVE || b >= n_blocks) continue;
        const double s = score_of(S, k, A.block_max[(size_t)(g * K + k) * n_blocks + b]);
        if (s > -(double)__builtin_inff() && bin_of(top, s) <= last_bin) {
            const uint32_t i = atomicAdd(&S.n_blocks, 1u);
            if (i < kPickBlocks) S.blocks[i] = k * n_blocks + b;
        }
    }
    if (tid < K && S.state[tid] == ROW_ENDED) {
        const uint32_t i = atomicAdd(&S.n_elems, 1u);
        S.score[i] = S.base[tid]; S.x[i] = 0.f; S.token[i] = -1; S.row[i] = (uint16_t)tid;
    }
    __syncthreads();
    const uint32_t listed = S.n_blocks < kPickBlocks ? S.n_blocks : kPickBlocks;
    for (uint32_t i = wave; i < listed; i += WAVES) {
        const uint32_t k = S.blocks[i] / n_blocks, b = S.blocks[i] % n_blocks, r = g * K + k;
        const E* const row = static_cast<const E*>(A.logits) + (long long)r * A.row_stride;
        const long long t0 = (long long)b * kBeamBlock - before_row(row) + lane;
        for (int c = 0; c < kBeamBlock; c += 64) {
            const long long t = t0 + c;
            if (t < 0 || t >= A.V || !token_allowed(A, r, t)) continue;
            const float x = Elem<E>::value(row[t]);
            const double s = score_of(S, k, x);
            if (!(s > -(double)__builtin_inff()) || bin_of(top, s) > last_bin) continue;
            const uint32_t at = atomicAdd(&S.n_elems, 1u);
            if (at < kPickElems) { S.score[at] = s; S.x[at] = x; S.token[at] = (int32_t)t; S.row[at] = (uint16_t)k; }
        }
    }
    __syncthreads();
    if (S.n_blocks <= kPickBlocks && S.n_elems <= kPickElems) {
        const uint32_t R = S.n_elems;
        for (;;) {
            // a candidate's place is the number of candidates before it
            for (uint32_t i = tid; i < R; i += kPickThreads) {
                const double s = S.score[i];
                const uint32_t k = S.row[i];
                const int32_t t = S.token[i];
                uint32_t place = 0;
                for (uint32_t j = 0; j < R; ++j) place += before(S.score[j], S.row[j], S.token[j], s, k, t) ? 1u : 0u;
                S.sorted[place] = (uint16_t)i;
            }
            if (tid < K) S.repair[tid] = 0;
            if (tid == 0) S.any = 0;
            __syncthreads();
            // Neighbours of different rows that are too close for their sums, among the chosen and those that are as close to the last
            // of them: these rows' sums in 64 bits.  (Two that are close and not neighbours have neighbours of different rows between them.)
            for (uint32_t n = tid; n + 1 < R; n += kPickThreads) {
                const uint32_t i = S.sorted[n], j = S.sorted[n + 1], ki = S.row[i], kj = S.row[j];
                if (ki == kj || (S.exact[ki] && S.exact[kj]) || S.score[i] - S.score[j] > A.near) continue;
                if (n + 1 <= N || !(S.score[S.sorted[N - 1]] - S.score[j] > A.near)) { S.repair[ki] = S.repair[kj] = 1; S.any = 1; }
            }
            __syncthreads();
            if (!S.any) break;
            for (uint32_t k = 0; k < K; ++k) if (S.repair[k] && !S.exact[k]) repair_row<E>(A, S, g, k);
            __syncthreads();
            for (uint32_t i = tid; i < R; i += kPickThreads) if (S.token[i] >= 0) S.score[i] = score_of(S, S.row[i], S.x[i]);
            __syncthreads();
        }
        if (tid < N) {
            const bool any = tid < R;
            const uint32_t i = any ? S.sorted[tid] : 0;
            write_choice(A, S, g, tid, any, any ? S.score[i] : 0, any ? S.row[i] : 0, any ? S.token[i] : -1);
        }
        return;
    }
    // Too many are too much alike (logits that are all the same): all sums in 64 bits, then the best block n times, and the best
    // candidate of these blocks n times, each the next one after the one before.
    for (uint32_t k = 0; k < K; ++k) if (S.state[k] == ROW_LIVE && !S.exact[k]) repair_row<E>(A, S, g, k);
    const double none = -(double)__builtin_inff();
    uint32_t n_found = 0;
    {
        double ls = 0;
        uint32_t lr = ~0u;
        long long lb = 0;
        while (n_found < N) {
            double s = none;
            uint32_t k1 = ~0u;
            long long b1 = 0;
            for (uint32_t u = wave; u < units; u += WAVES) {
                const uint32_t k = u / steps, b = u % steps * 64 + lane;
                if (S.state[k] != ROW_LIVE || b >= n_blocks) continue;
                const double v = score_of(S, k, A.block_max[(size_t)(g * K + k) * n_blocks + b]);
                if (!(v > none) || (lr != ~0u && !before(ls, lr, lb, v, k, b))) continue;
                if (k1 == ~0u || before(v, k, b, s, k1, b1)) { s = v; k1 = k; b1 = b; }
            }
            best_of_all(S, s, k1, b1);
            if (k1 == ~0u) break;
            if (tid == 0) S.blocks[n_found] = k1 * n_blocks + (uint32_t)b1;
            ++n_found;
            ls = s; lr = k1; lb = b1;
        }
    }
    __syncthreads();
    double ls = 0;
    uint32_t lr = ~0u;
    long long lt = 0;
    for (uint32_t n = 0; n < N; ++n) {
        double s = none;
        uint32_t k1 = ~0u;
        long long t1 = 0;
        for (uint32_t i = wave; i < n_found; i += WAVES) {
            const uint32_t k = S.blocks[i] / n_blocks, b = S.blocks[i] % n_blocks, r = g * K + k;
            const E* const row = static_cast<const E*>(A.logits) + (long long)r * A.row_stride;
            const long long t0 = (long long)b * kBeamBlock - before_row(row) + lane;
            for (int c = 0; c < kBeamBlock; c += 64) {
                const long long t = t0 + c;
                if (t < 0 || t >= A.V || !token_allowed(A, r, t)) continue;
                const double v = score_of(S, k, Elem<E>::value(row[t]));
                if (!(v > none) || (lr != ~0u && !before(ls, lr, lt, v, k, t))) continue;
                if (k1 == ~0u || before(v, k, t, s, k1, t1)) { s = v; k1 = k; t1 = t; }
            }
        }
        if (tid < K && S.state[tid] == ROW_ENDED) {
            const double v = S.base[tid];
            if ((lr == ~0u || before(ls, lr, lt, v, tid, -1)) && (k1 == ~0u || before(v, tid, -1, s, k1, t1))) { s = v; k1 = tid; t1 = -1; }
        }
        best_of_all(S, s, k1, t1);
        if (tid == 0) write_choice(A, S, g, n, k1 != ~0u, s, k1, (int32_t)t1);
        if (k1 != ~0u) { ls = s; lr = k1; lt = t1; }
        else { lr = K; ls = none; }                                  // nothing comes after
    }
}

// ---- matcher slots --------------------------------------------------------------------------------------------------
// One workgroup per group of beams, a wavefront for up to SLOTS of its slots.  A slot's context has two buffers, and nobody reads the one
// that is not its own state, so the parent's goes there at once; the slot's record and its frontier planes have one place, so these
// wait in registers until all wavefronts of the group have read theirs.
template <int SLOTS>
__global__ __launch_bounds__(1024) void k_batch_reorder(BatchDev D, uint32_t K, const int32_t* parents, int32_t* status) {
    const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), waves = blockDim.x >> 6, first = blockIdx.x * K;
    uint64_t plane[SLOTS];
    FillRow row[SLOTS];
    bool moved[SLOTS];
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) {
        const uint32_t k = wave + (uint32_t)j * waves, b = first + k;
        moved[j] = false;
        if (k >= K) continue;
        const int32_t p = parents[b];
        const bool in_group = p >= 0 && (uint32_t)p >= first && (uint32_t)p < first + K;
        if (status && lane == 0) status[b] = in_group || p == -1 ? kAccOk : kAccInvalid;
        if (!in_group || (uint32_t)p == b) continue;
        const uint32_t to = D.rows[b].pad[0] ^ 1u;
        const size_t slot = (size_t)to * D.B + b;
        FillRow r = D.rows[p];
        plane[j] = lane < r.front_n ? D.front[(size_t)r.front_off + lane] : 0;
        const uint32_t* const items = D.items + r.item_off;
        const uint32_t* const off = D.wait_off + r.waitoff_off;
        const uint2* const wait = D.wait + r.wait_base;
        for (uint32_t i = lane; i < r.item_n; i += 64) D.items[slot * D.KI + i] = items[i];
        for (uint32_t i = lane; i <= r.H; i += 64) D.wait_off[slot * (D.KH + 1) + i] = off[i];
        for (uint32_t i = lane; i < r.n_wait; i += 64) D.wait[slot * D.KW + i] = wait[i];
        r.front_off = b * D.KF;
        r.item_off = (uint32_t)(slot * D.KI); r.wait_base = (uint32_t)(slot * D.KW); r.waitoff_off = (uint32_t)(slot * (D.KH + 1));
        r.pad[0] = to;
        row[j] = r;
        moved[j] = true;
    }
    // (what was loaded is there before any wavefront stores)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) {
        if (!moved[j]) continue;
        const uint32_t b = first + wave + (uint32_t)j * waves;
        if (lane < row[j].front_n) D.front[(size_t)b * D.KF + lane] = plane[j];
        if (lane == 0) D.rows[b] = row[j];
    }
}

// ---- rows of a buffer -----------------------------------------------------------------------------------------------
// A thread has one column of all rows of a group: it loads what every row will hold there and then stores it, so nothing waits for
// anybody and no second buffer is needed.  Rows that keep their place are neither read (but as parents) nor written.
// (vectors at any byte: the device takes them, and a row's stride or a position's size need not be a multiple of anything)
typedef uint32_t Wide4 __attribute__((ext_vector_type(4), aligned(1)));
typedef uint32_t Wide2 __attribute__((ext_vector_type(2), aligned(1)));

template <class T, int MOST>
__device__ __forceinline__ void move_column(uint8_t* at, int64_t row_stride, const int32_t* from, uint64_t moves) {
    T v[MOST];
#pragma unroll
    for (int k = 0; k < MOST; ++k)
        if ((moves >> k) & 1) v[k] = *reinterpret_cast<const T*>(at + (int64_t)uniform((uint32_t)from[k]) * row_stride);
#pragma unroll
    for (int k = 0; k < MOST; ++k)
        if ((moves >> k) & 1) *reinterpret_cast<T*>(at + (int64_t)k * row_stride) = v[k];
}

template <class T, int MOST>
__global__ __launch_bounds__(256) void k_beam_reorder_rows(BeamRows A, uint32_t splits) {
    __shared__ int32_t from[kBeamsMost];
    __shared__ uint64_t moving;
    const uint32_t split = blockIdx.x % splits, unit = blockIdx.x / splits, g = blockIdx.y + blockIdx.z * 32768u, K = A.beams;
    if (g >= A.groups) return;
    if (threadIdx.x < 64) {
        const int32_t p = threadIdx.x < K ? A.parents[g * K + threadIdx.x] : -1, k = p >= 0 ? p - (int32_t)(g * K) : -1;
        const bool moves = k >= 0 && k < (int32_t)K && k != (int32_t)threadIdx.x;
        from[threadIdx.x] = moves ? k : 0;
        const uint64_t all = __ballot(moves);
        if (threadIdx.x == 0) moving = all;
    }
    __syncthreads();
    const uint64_t moves = (uint64_t)uniform((uint32_t)(moving >> 32)) << 32 | uniform((uint32_t)moving);
    if (moves == 0) return;
    int64_t begin = A.begin ? A.begin[g] : 0, end = A.end ? A.end[g] : (int64_t)A.positions;
    begin = begin < 0 ? 0 : begin;
    end = end > (int64_t)A.positions ? (int64_t)A.positions : end;
    if (begin >= end) return;
    uint8_t* const piece = A.data + (int64_t)(g * K) * A.row_stride + (int64_t)(unit / A.pieces) * A.outer_stride + (int64_t)(unit % A.pieces) * A.piece_stride
                           + begin * A.position_bytes;
    const int64_t bytes = (end - begin) * A.position_bytes, whole = bytes / (int64_t)sizeof(T);
    for (int64_t v = (int64_t)split * 256 + threadIdx.x; v < whole; v += (int64_t)splits * 256) move_column<T, MOST>(piece + v * (int64_t)sizeof(T), A.row_stride, from, moves);
    const int64_t rest = whole * (int64_t)sizeof(T) + threadIdx.x;   // (less than a vector)
    if (split == 0 && rest < bytes) move_column<uint8_t, MOST>(piece + rest, A.row_stride, from, moves);
}

// ---- sequences ------------------------------------------------------------------------------------------------------
// One thread per sequence, from the last step to the first.
__global__ __launch_bounds__(64) void k_beam_backtrace(BeamTrace A) {
    const uint32_t g = blockIdx.x, k = threadIdx.x;
    if (k >= A.beams) return;
    const uint32_t first = g * A.beams;
    int32_t* const out = A.out + (int64_t)(first + k) * A.out_stride;
    int32_t length = 0;
    int64_t row = first + k;
    for (int64_t t = (int64_t)A.steps - 1; t >= 0; --t) {
        int32_t token = -1;
        if (row >= 0) {
            token = A.tokens[t * A.step_stride + row];
            row = A.parents[t * A.step_stride + row];
            if (row < (int64_t)first || row >= (int64_t)first + A.beams) row = -1;
        }
        out[t] = token;
        if (token >= 0 && length == 0) length = (int32_t)t + 1;
    }
    if (A.lengths) A.lengths[first + k] = length;
}

}  // namespace

template <class E>
static void launch_beam_select_as(const BeamSelect& A, hipStream_t stream) {
    const uint32_t rows = A.groups * A.beams;
    auto* const kernel = !A.bitmask ? k_beam_scan<E, 0> : A.over_all ? k_beam_scan<E, 2> : k_beam_scan<E, 1>;
    for (uint32_t first = 0; first < rows; first += 65535) {         // grid.y limit
        const uint32_t n = std::min<uint32_t>(65535, rows - first);
        hipLaunchKernelGGL(kernel, dim3((A.pieces + kScanWaves - 1) / kScanWaves, n), dim3(64 * kScanWaves), 0, stream, A, first);
    }
    hipLaunchKernelGGL(k_beam_pick<E>, dim3(A.groups), dim3(kPickThreads), 0, stream, A);
}

void launch_beam_select(const BeamSelect& A, hipStream_t stream) {
    if (A.groups == 0) return;
    if (A.dtype == XG2_F32) launch_beam_select_as<float>(A, stream);
    else launch_beam_select_as<Bf16>(A, stream);
}

void launch_batch_reorder(const BatchDev& D, uint32_t beams, const int32_t* parents_dev, int32_t* status_dev, hipStream_t stream) {
    if (D.B == 0 || D.KF > 64) return;
    const dim3 grid(D.B / beams), block(64 * std::min<uint32_t>(beams, 16));
    if (beams <= 16) hipLaunchKernelGGL(k_batch_reorder<1>, grid, block, 0, stream, D, beams, parents_dev, status_dev);
    else hipLaunchKernelGGL(k_batch_reorder<4>, grid, block, 0, stream, D, beams, parents_dev, status_dev);
}

template <class T, int MOST>
static void launch_rows_as(const BeamRows& A, hipStream_t stream) {
    const uint32_t units = A.outer * A.pieces;
    const int64_t vectors = A.positions * A.position_bytes / (int64_t)sizeof(T);
    uint32_t splits = (uint32_t)std::min<int64_t>(vectors / 256 + 1, 64);
    splits = std::max<uint32_t>(1, std::min<uint32_t>(splits, 0x7FFFFFFFu / units));
    hipLaunchKernelGGL((k_beam_reorder_rows<T, MOST>), dim3(units * splits, std::min<uint32_t>(A.groups, 32768), (A.groups + 32767) / 32768), dim3(256), 0, stream, A, splits);
}

void launch_beam_reorder_rows(const BeamRows& A, hipStream_t stream) {
    // what a thread holds is a vector a row
    if (A.beams <= 4) launch_rows_as<Wide4, 4>(A, stream);
    else if (A.beams <= 8) launch_rows_as<Wide4, 8>(A, stream);
    else if (A.beams <= 16) launch_rows_as<Wide4, 16>(A, stream);
    else if (A.beams <= 32) launch_rows_as<Wide4, 32>(A, stream);
    else launch_rows_as<Wide2, 64>(A, stream);
}

void launch_beam_backtrace(const BeamTrace& A, hipStream_t stream) {
    if (A.groups == 0) return;
    hipLaunchKernelGGL(k_beam_backtrace, dim3(A.groups), dim3(64), 0, stream, A);
}

}  // namespace xg2
