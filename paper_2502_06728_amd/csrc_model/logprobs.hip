// Log probabilities of given tokens: log sum exp, entropy and the best tokens of every row of the logits, and
// the gradient of the logits.
//
// Forward.  A workgroup takes a piece of a row in one pass with the running maximum m, s = sum exp(z - m) and
// w = sum (z - m) exp(z - m), in fp32 and in units of log 2:
//     lse = m + log s        entropy = log s - w / s
// A lane's 32 values raise the maximum once, and their exponents are one fused multiply-add each, d = z / log 2 - c
// with c the product of the maximum as rounded: sums relative to c are exact in that respect, and are brought to
// the maximum itself at the end.  (Where the product leaves fp32's range, at a type's lowest value say, the lane
// takes its values once more and subtracts first.)
// Rows are cut into pieces where there are too few of them to fill the chip (a sampled token is one row); a
// second launch joins a row's pieces.  The best tokens: the K-th largest of the threads' maxima is a value
// that at least K elements reach, and seldom many more do; a second look at the piece lists those, and the
// list is ranked by (value, index), so that the order in which it was filled does not matter.  A piece where
// the list does not hold them (many equal values) is searched K times instead.
//
// Backward.  A stream: p = exp(z - m - log s) from the row's saved m and log s.
#include "device.hip.h"

namespace deto {
namespace model {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kLanes;
constexpr int kMaxTop = 32;
constexpr int kList = 1024;                    // listed candidates of a piece
constexpr int kMaxPieces = kList / kMaxTop;    // the join ranks kMaxTop of every piece in one list
static_assert(kMaxPieces <= kLanes, "a lane for each piece");
constexpr int64_t kPieceElems = kThreads * 8;  // least length of a piece: eight elements a lane
constexpr int64_t kFillWorkgroups = 1024;      // workgroups that fill the chip

// What a piece, or a part of one, has seen: m over the raw logits, a NaN if one was; s, w scaled (w in units of
// log 2).  m is -infinity before the first value above that.
struct Seen {
    float m, s, w;
};

// of piece p of row t in the workspace: [T][pieces] Seen, then [T][pieces][top] ranked candidates
struct Parts {
    Seen* seen;
    uint64_t* best;
    int pieces;
};

struct Forward {
    int64_t V, ld;
    const void* logits;
    float scale;         // of the logits
    float unit;          // scale / log 2
    const void* targets;
    int target_bytes;
    float* logp;
    float* lse;
    float* entropy;
    int top;
    int32_t* top_idx;
    float* top_logp;
    float* stats;
    Parts parts;
    int64_t piece;       // elements of a piece, a multiple of 8
};

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// the larger, a NaN if either is one
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }

__device__ __forceinline__ float wave_larger(float v) {
    v = larger(v, moved<0xB1>(v));
    v = larger(v, moved<0x4E>(v));
    v = larger(v, moved<0x141>(v));
    v = larger(v, moved<0x140>(v));
    return larger(larger(lane_value(v, 0), lane_value(v, 16)), larger(lane_value(v, 32), lane_value(v, 48)));
}

// d 2^d is 0 where 2^d is
constexpr float kFarBelow = -16384.f;
// products of the maximum that sums may be relative to
constexpr float kInRange = 1e30f;

// The same relative to m, which is not below r.m.  (m = -infinity stands for nothing above it: no difference is
// taken from it.)
__device__ __forceinline__ Seen relative_to(const Seen& r, float m, float unit) {
    const float ref = m == -__builtin_inff() ? 0.f : m;
    const float d = fmaxf((r.m - ref) * unit, kFarBelow), e = exp2_fast(d);
    return {m, r.s * e, (r.w + r.s * d) * e};
}

// All lanes of a wavefront as one, in every lane.
__device__ __forceinline__ Seen join_wave(Seen r, float unit) {
    r = relative_to(r, wave_larger(r.m), unit);
    return {r.m, wave_sum(r.s), wave_sum(r.w)};
}

// An order of all values, NaNs above everything, -0 and +0 the same: larger means earlier.  0 is no value, and
// no candidate is all ones.
constexpr uint32_t kNanKey = 0xFFFFFFFEu, kLowestKey = 0x007FFFFFu;      // of a NaN, of -infinity
__device__ __forceinline__ uint32_t order_key(float v) {
    const uint32_t b = f32_bits(v + 0.f);      // (-0 + 0 = +0)
    if (v != v) return kNanKey;
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) {
    if (k == kNanKey) return __builtin_nanf("");
    return bits_f32(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}
// value and index: larger values first, among equal ones lower indices
__device__ __forceinline__ uint64_t candidate(uint32_t key, uint32_t index) {
    return static_cast<uint64_t>(key) << 32 | static_cast<uint32_t>(~index);
}

__device__ __forceinline__ int64_t target_of(const void* targets, int bytes, int64_t t) {
    return bytes == 8 ? static_cast<const int64_t*>(targets)[t] : static_cast<const int32_t*>(targets)[t];
}

// A row's target and its logit (loaded early: two loads, one after the other)
struct Target {
    int64_t y;
    float z;
    bool scored;
};
template <int DT>
__device__ __forceinline__ Target load_target(const Forward& a, int64_t t) {
    const int64_t y = target_of(a.targets, a.target_bytes, t);
    const bool scored = y >= 0 && y < a.V;
    return {y, scored ? load1<DT>(a.logits, t * a.ld + y) : 0.f, scored};
}

__device__ __forceinline__ void write_row(const Forward& a, int64_t t, const Seen& r, const Target& y) {
    const float log_s = logf(r.s);
    const bool none = r.m == -__builtin_inff();       // -infinities throughout
    float logp = 0.f;
    if (y.scored) logp = none ? -__builtin_inff() : (y.z - r.m) * a.scale - log_s;
    a.logp[t] = logp;
    if (a.lse) a.lse[t] = none ? -__builtin_inff() : r.m * a.scale + log_s;
    if (a.entropy) a.entropy[t] = none ? 0.f : log_s - 0.69314718055994531f * (r.w / r.s);
    if (a.stats) {
        a.stats[2 * t] = r.m;
        a.stats[2 * t + 1] = none ? 0.f : log_s;
    }
}

__device__ __forceinline__ void write_best(const Forward& a, int64_t t, int rank, uint64_t c, float m,
                                           float log_s) {
    a.top_idx[t * a.top + rank] = static_cast<int32_t>(~static_cast<uint32_t>(c));
    if (!a.top_logp) return;
    const float v = key_value(static_cast<uint32_t>(c >> 32));
    a.top_logp[t * a.top + rank] =
        v == -__builtin_inff() && log_s == log_s ? v : (v - m) * a.scale - log_s;
}

// Vectors of eight that a lane takes at a time: 64 bytes.
template <int DT> constexpr int kVectors = DT == DETO_F32 ? 2 : 4;

template <int DT>
struct Taken {
    float v[kVectors<DT>][8];        // -infinity past the end
};

template <int DT>
struct Piece {
    const void* logits;
    int64_t row, first, end;
    __device__ __forceinline__ int64_t at(int64_t d, int i) const { return d + i * kThreads * 8; }
    __device__ __forceinline__ int count(int64_t d, int i) const {
        const int64_t left = end - at(d, i);
        return left >= 8 ? 8 : left > 0 ? static_cast<int>(left) : 0;
    }
    __device__ __forceinline__ void load(int64_t d, Raw8<DT> (&raw)[kVectors<DT>]) const {
#pragma unroll
        for (int i = 0; i < kVectors<DT>; ++i) raw[i] = load8<DT>(logits, row, at(d, i), count(d, i));
    }
    __device__ __forceinline__ void unpack(int64_t d, const Raw8<DT> (&raw)[kVectors<DT>], Taken<DT>& x) const {
#pragma unroll
        for (int i = 0; i < kVectors<DT>; ++i) {
            unpack8<DT>(raw[i], x.v[i]);
            const int n = count(d, i);
            if (n < 8) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j >= n) x.v[i][j] = -__builtin_inff();
            }
        }
    }
};

// r.s and r.w are relative to the product of r.m and unit as rounded.
template <int DT, bool ENTROPY>
__device__ __forceinline__ void see(Seen& r, const Taken<DT>& x, float unit) {
    float m = r.m;
#pragma unroll
    for (int i = 0; i < kVectors<DT>; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) m = larger(m, x.v[i][j]);
    const float c = fabsf(m * unit) <= kInRange ? m * unit : 0.f;     // (else the lane starts again at the end)
    const float d0 = fmaxf(r.m * unit - c, kFarBelow), e0 = exp2_fast(d0);
    float s = r.s * e0, w = (r.w + r.s * d0) * e0;
#pragma unroll
    for (int i = 0; i < kVectors<DT>; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float d = __builtin_fmaf(x.v[i][j], unit, -c);
            if constexpr (ENTROPY) d = fmaxf(d, kFarBelow);
            const float e = exp2_fast(d);
            s += e;
            if constexpr (ENTROPY) w = __builtin_fmaf(d, e, w);
        }
    r = {m, s, w};
}

// The whole workgroup's, in every thread.
__device__ __forceinline__ Seen join_workgroup(Seen r, float unit, Seen* lds) {
    r = join_wave(r, unit);
    if (threadIdx.x % kLanes == 0) lds[threadIdx.x / kLanes] = r;
    __syncthreads();
    float m = lds[0].m;
#pragma unroll
    for (int i = 1; i < kWaves; ++i) m = larger(m, lds[i].m);
    Seen all = {m, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        const Seen p = relative_to(lds[i], m, unit);
        all.s += p.s;
        all.w += p.w;
    }
    return all;
}

// The K-th largest of the workgroup's keys, down to its upper 16 bits, by bisection: counts of keys in each wavefront
// alone, which holds all of them.
__device__ __forceinline__ uint32_t kth_key(const uint32_t* lds_keys, int K) {
    uint32_t k[kWaves];
#pragma unroll
    for (int i = 0; i < kWaves; ++i) k[i] = lds_keys[i * kLanes + threadIdx.x % kLanes];
    uint32_t found = 0;
#pragma unroll
    for (int bit = 31; bit >= 16; --bit) {
        const uint32_t t = found | 1u << bit;
        int n = 0;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) n += __popcll(__ballot(k[i] >= t));
        if (n >= K) found = t;
    }
    return found;
}

// How many of the list's n candidates rank before c.  (The list is filled up with zeros to a multiple of 8.)
__device__ __forceinline__ int rank_of(const uint64_t* list, int n, uint64_t c) {
    int rank = 0;
    for (int j = 0; j < n; j += 8) {
#pragma unroll
        for (int k = 0; k < 8; ++k) rank += list[j + k] > c;
    }
    return rank;
}
__device__ __forceinline__ void fill_up(uint64_t* list, int n) {
    if (threadIdx.x < 8 && n + static_cast<int>(threadIdx.x) < (n + 7) / 8 * 8) list[n + threadIdx.x] = 0;
}

template <int DT, bool ENTROPY, bool TOP>
__global__ __launch_bounds__(kThreads) void logprobs_kernel(Forward a) {
    __shared__ Seen lds_seen[kWaves];
    const int64_t t = blockIdx.x / a.parts.pieces;
    const int piece = blockIdx.x % a.parts.pieces;
    const int64_t begin = piece * a.piece;
    const Piece<DT> p = {a.logits, t * a.ld, begin, begin + a.piece < a.V ? begin + a.piece : a.V};
    const bool whole = a.parts.pieces == 1;
    Target y = {};
    if (whole) y = load_target<DT>(a, t);
    constexpr int64_t kStep = kThreads * 8 * kVectors<DT>;
    const int64_t mine = p.first + 8 * threadIdx.x;
    Seen r = {-__builtin_inff(), 0.f, 0.f};
    Raw8<DT> raw[kVectors<DT>];
    Taken<DT> x;
    for (int64_t d = mine; d < p.end; d += kStep) {
        p.load(d, raw);
        p.unpack(d, raw, x);
        see<DT, ENTROPY>(r, x, a.unit);
    }
    {
        // from the rounded product to the maximum itself
        const float c = r.m * a.unit, off = __builtin_fmaf(r.m, a.unit, -c), e = exp2_fast(-off);
        if (fabsf(c) <= kInRange) {
            r = {r.m, r.s * e, (r.w - off * r.s) * e};
        } else if (r.m == r.m && r.m != -__builtin_inff()) {
            r.s = r.w = 0.f;
            for (int64_t d = mine; d < p.end; d += kStep) {
                p.load(d, raw);
                p.unpack(d, raw, x);
#pragma unroll
                for (int i = 0; i < kVectors<DT>; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float l = (x.v[i][j] - r.m) * a.unit, e1 = exp2_fast(l);
                        r.s += e1;
                        r.w += fmaxf(l, kFarBelow) * e1;
                    }
            }
        }
    }
    const uint32_t key = mine < p.end ? order_key(r.m) : 0u;
    r = join_workgroup(r, a.unit, lds_seen);
    if (threadIdx.x == 0) {
        if (whole) write_row(a, t, r, y);
        else a.parts.seen[blockIdx.x] = r;
    }
    if constexpr (TOP) {
        __shared__ uint32_t lds_keys[kThreads];
        __shared__ uint64_t list[kList + 8];
        __shared__ uint32_t listed;
        const float log_s = logf(r.s);
        uint64_t* part = a.parts.best + static_cast<int64_t>(blockIdx.x) * a.top;
        auto give = [&](int rank, uint64_t c) {
            if (whole) write_best(a, t, rank, c, r.m, log_s);
            else part[rank] = c;
        };
        lds_keys[threadIdx.x] = key;
        if (threadIdx.x == 0) listed = 0;
        __syncthreads();
        const uint32_t least = kth_key(lds_keys, a.top);
        // (0: fewer than `top` threads saw a value, all of them are listed; a NaN is not below anything)
        const float least_value = least > kLowestKey ? key_value(least) : -__builtin_inff();
        for (int64_t d = mine; d < p.end; d += kStep) {
            if (p.end - p.first > kStep) {       // (else the registers still hold the piece)
                p.load(d, raw);
                p.unpack(d, raw, x);
            }
#pragma unroll
            for (int i = 0; i < kVectors<DT>; ++i) {
                float m = x.v[i][0];
#pragma unroll
                for (int j = 1; j < 8; ++j) m = larger(m, x.v[i][j]);
                if (m < least_value) continue;
                const int n = p.count(d, i);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (j < n && !(x.v[i][j] < least_value)) {
                        const uint32_t at = atomicAdd(&listed, 1u);
                        if (at < kList)
                            list[at] = candidate(order_key(x.v[i][j]), static_cast<uint32_t>(p.at(d, i) + j));
                    }
                }
            }
        }
        __syncthreads();
        const int n = listed;
        if (n <= kList) {
            fill_up(list, n);
            __syncthreads();
            for (int i = threadIdx.x; i < n; i += kThreads) {
                const uint64_t c = list[i];
                const int rank = rank_of(list, n, c);
                if (rank < a.top) give(rank, c);
            }
            // a piece of fewer than `top` elements: the rest of its part is empty
            for (int i = n + threadIdx.x; i < a.top; i += kThreads) give(i, 0);
            return;
        }
        // Too many reach the threshold: one search for each place, each for the largest candidate below the
        // one before.
        uint64_t before = ~uint64_t{0};
        for (int rank = 0; rank < a.top; ++rank) {
            uint64_t best = 0;
            for (int64_t d = mine; d < p.end; d += kStep) {
                p.load(d, raw);
                p.unpack(d, raw, x);
#pragma unroll
                for (int i = 0; i < kVectors<DT>; ++i) {
                    const int n_there = p.count(d, i);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const uint64_t c = candidate(order_key(x.v[i][j]), static_cast<uint32_t>(p.at(d, i) + j));
                        if (j < n_there && c < before && c > best) best = c;
                    }
                }
            }
#pragma unroll
            for (int step = 1; step < kLanes; step <<= 1) {
                const uint64_t o = __shfl_xor(best, step);
                best = o > best ? o : best;
            }
            __syncthreads();               // the list's last readers are done
            if (threadIdx.x % kLanes == 0) list[threadIdx.x / kLanes] = best;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kWaves; ++i) best = list[i] > best ? list[i] : best;
            if (threadIdx.x == 0) give(rank, best);
            before = best;
        }
    }
}

// A workgroup per row: its pieces as one.  (Every wavefront joins the sums for itself: no barrier for those.)
template <int DT>
__global__ __launch_bounds__(kThreads) void logprobs_join_kernel(Forward a) {
    __shared__ uint64_t list[kList + 8];
    const int64_t t = blockIdx.x;
    const int pieces = a.parts.pieces, lane = threadIdx.x % kLanes;
    const Target y = load_target<DT>(a, t);
    Seen r = {-__builtin_inff(), 0.f, 0.f};
    if (lane < pieces) r = a.parts.seen[t * pieces + lane];
    const int n = pieces * a.top;           // at most kList
    const uint64_t* part = a.parts.best + t * n;
    for (int i = threadIdx.x; i < n; i += kThreads) list[i] = part[i];
    fill_up(list, n);
    r = join_wave(r, a.unit);
    if (threadIdx.x == 0) write_row(a, t, r, y);
    if (a.top == 0) return;
    __syncthreads();
    const float log_s = logf(r.s);
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const uint64_t c = list[i];
        const int rank = rank_of(list, n, c);
        if (rank < a.top && c) write_best(a, t, rank, c, r.m, log_s);
    }
}

struct Backward {
    int64_t V, ld, ld_out;
    const void* logits;
    void* dlogits;
    float scale, unit;
    const void* targets;
    int target_bytes;
    const float* stats;
    const float* entropy;
    const float* g_logp;
    const float* g_entropy;
    uint32_t pieces;     // workgroups of a row
};

constexpr int kBackwardVectors = 4;      // of eight elements, a lane
constexpr int64_t kBackwardElems = kThreads * 8 * kBackwardVectors;

template <int DT, bool ENTROPY>
__global__ __launch_bounds__(kThreads) void logprobs_backward_kernel(Backward a) {
    const int64_t t = blockIdx.x / a.pieces;
    const int64_t first = (blockIdx.x % a.pieces) * kBackwardElems + 8 * threadIdx.x;
    const float m = a.stats[2 * t], log_s = a.stats[2 * t + 1] * 1.4426950408889634f;
    const int64_t y = target_of(a.targets, a.target_bytes, t);
    const bool none = m == -__builtin_inff() && log_s == log_s;     // -infinities throughout
    const float g = a.g_logp && y >= 0 && y < a.V ? a.g_logp[t] * a.scale : 0.f;
    float ge = 0.f, h = 0.f;               // the entropy in units of log 2
    if constexpr (ENTROPY) {
        ge = a.g_entropy[t] * a.scale * 0.69314718055994531f;
        h = a.entropy[t] * 1.4426950408889634f;
    }
    Raw8<DT> raw[kBackwardVectors];
    int count[kBackwardVectors];
#pragma unroll
    for (int i = 0; i < kBackwardVectors; ++i) {
        const int64_t left = a.V - (first + i * kThreads * 8);
        count[i] = left >= 8 ? 8 : left > 0 ? static_cast<int>(left) : 0;
        raw[i] = load8<DT>(a.logits, t * a.ld, first + i * kThreads * 8, count[i]);
    }
#pragma unroll
    for (int i = 0; i < kBackwardVectors; ++i) {
        const int64_t d = first + i * kThreads * 8;
        float v[8];
        unpack8<DT>(raw[i], v);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float l = (v[j] - m) * a.unit - log_s;      // log2 p
            const float p = exp2_fast(l);
            float o = -g * p;
            if constexpr (ENTROPY) o -= ge * p * (fmaxf(l, -16384.f) + h);
            if (d + j == y) o += g;
            v[j] = none ? 0.f : o;
        }
        store8<DT>(a.dlogits, t * a.ld_out + d, v, count[i]);
    }
}

bool bad_shape(int64_t T, int64_t V, int top) {
    return T < 0 || V < 1 || V > 0x7FFFFFFF || top < 0 || top > kMaxTop || top > V;
}

// Pieces of a row: as many as fill the chip, each of kPieceElems elements at least.
int pieces_of(int64_t T, int64_t V) {
    const int64_t most = (V + kPieceElems - 1) / kPieceElems;
    int64_t want = T > 0 ? kFillWorkgroups / T : 1;
    if (want > most) want = most;
    if (want > kMaxPieces) want = kMaxPieces;
    return want < 1 ? 1 : static_cast<int>(want);
}

// Rows whose workgroups a launch can count (31 bits).
constexpr int64_t kMaxGrid = 0x7FFFFFFF;

}  // namespace
}  // namespace model
}  // namespace deto

using namespace deto::model;

extern "C" {

int64_t detonation_token_logprobs_workspace(int64_t T, int64_t V, int32_t top) {
    if (bad_shape(T, V, top)) return -1;
    const int64_t pieces = pieces_of(T, V);
    if (pieces == 1) return 0;
    return (T * pieces * static_cast<int64_t>(sizeof(Seen)) + 15) / 16 * 16 +
           T * pieces * top * static_cast<int64_t>(sizeof(uint64_t));
}

int detonation_token_logprobs(int64_t T, int64_t V, const deto_rows* logits, float logit_scale,
                              const void* targets, int target_bytes, float* logp, float* lse,
                              float* entropy, int32_t top, int32_t* top_idx, float* top_logp,
                              float* stats, void* workspace, void* stream) {
    if (bad_shape(T, V, top)) return DETO_ERR_BAD_CONFIG;
    if (!(logit_scale > 0.f) || !std::isfinite(logit_scale)) return DETO_ERR_BAD_CONFIG;
    if (target_bytes != 4 && target_bytes != 8) return DETO_ERR_BAD_CONFIG;
    if (T == 0) return DETO_OK;
    const int pieces = pieces_of(T, V);
    if (!here(logits) || !targets || !logp || (top && !top_idx) || (pieces > 1 && !workspace))
        return DETO_ERR_NULL;
    const int rc = check_rows(logits, T, V);
    if (rc) return rc;
    if (!is_aligned(targets, target_bytes) || !is_aligned(logp, 4) || !is_aligned(lse, 4) ||
        !is_aligned(entropy, 4) || !is_aligned(top_idx, 4) || !is_aligned(top_logp, 4) ||
        !is_aligned(stats, 4) || (pieces > 1 && !is_aligned(workspace, 16)))
        return DETO_ERR_ALIGN;
    if (T > kMaxGrid) return DETO_ERR_UNSUPPORTED;
    char* ws = static_cast<char*>(workspace);
    const int64_t seen_bytes = (T * pieces * static_cast<int64_t>(sizeof(Seen)) + 15) / 16 * 16;
    const int64_t piece = ((V + pieces - 1) / pieces + 7) / 8 * 8;
    const Forward a = {V, logits->ld, logits->data, logit_scale, logit_scale * 1.4426950408889634f,
                       targets, target_bytes, logp, lse, entropy, top, top_idx, top_logp, stats,
                       {reinterpret_cast<Seen*>(ws),
                        pieces > 1 ? reinterpret_cast<uint64_t*>(ws + seen_bytes) : nullptr, pieces},
                       piece};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const unsigned grid = static_cast<unsigned>(T * pieces);
    fresh();
    by_type(logits->dtype, [&](auto dt) {
        constexpr int DT = dt.value;
        if (top) {
            if (entropy) logprobs_kernel<DT, true, true><<<grid, kThreads, 0, st>>>(a);
            else logprobs_kernel<DT, false, true><<<grid, kThreads, 0, st>>>(a);
        } else {
            if (entropy) logprobs_kernel<DT, true, false><<<grid, kThreads, 0, st>>>(a);
            else logprobs_kernel<DT, false, false><<<grid, kThreads, 0, st>>>(a);
        }
        if (pieces > 1)
            logprobs_join_kernel<DT><<<static_cast<unsigned>(T), kThreads, 0, st>>>(a);
        return 0;
    });
    return enqueued();
}

int detonation_token_logprobs_backward(int64_t T, int64_t V, const deto_rows* logits,
                                       float logit_scale, const void* targets, int target_bytes,
                                       const float* stats, const float* entropy,
                                       const float* g_logp, const float* g_entropy,
                                       const deto_rows* dlogits, void* stream) {
    if (bad_shape(T, V, 0)) return DETO_ERR_BAD_CONFIG;
    if (!(logit_scale > 0.f) || !std::isfinite(logit_scale)) return DETO_ERR_BAD_CONFIG;
    if (target_bytes != 4 && target_bytes != 8) return DETO_ERR_BAD_CONFIG;
    if (T == 0) return DETO_OK;
    if (!here(logits) || !here(dlogits) || !targets || !stats || (!g_logp && !g_entropy) ||
        (g_entropy && !entropy))
        return DETO_ERR_NULL;
    const int rc = first_error(check_rows(logits, T, V), check_rows(dlogits, T, V));
    if (rc) return rc;
    if (dlogits->dtype != logits->dtype) return DETO_ERR_BAD_CONFIG;
    if (!is_aligned(targets, target_bytes) || !is_aligned(stats, 4) || !is_aligned(entropy, 4) ||
        !is_aligned(g_logp, 4) || !is_aligned(g_entropy, 4))
        return DETO_ERR_ALIGN;
    const int64_t pieces = (V + kBackwardElems - 1) / kBackwardElems;
    if (T > kMaxGrid / pieces) return DETO_ERR_UNSUPPORTED;
    const Backward a = {V, logits->ld, dlogits->ld, logits->data, dlogits->data, logit_scale,
                        logit_scale * 1.4426950408889634f, targets, target_bytes, stats, entropy,
                        g_logp, g_entropy, static_cast<uint32_t>(pieces)};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const unsigned grid = static_cast<unsigned>(T * pieces);
    fresh();
    by_type(logits->dtype, [&](auto dt) {
        constexpr int DT = dt.value;
        if (g_entropy) logprobs_backward_kernel<DT, true><<<grid, kThreads, 0, st>>>(a);
        else logprobs_backward_kernel<DT, false><<<grid, kThreads, 0, st>>>(a);
        return 0;
    });
    return enqueued();
}

}  // extern "C"
