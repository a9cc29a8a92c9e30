// Log probabilities of given tokens: log sum exp, entropy and the best tokens of every row of the logits, and
// the gradient of the logits.
//
// Forward.  A workgroup takes a piece of a row in one pass with the running maximum m, s = sum exp(z - m) and
// w = sum (z - m) exp(z - m), in fp32 and in units of log 2:
//     lse = m + log s        entropy = log s - w / s
// A lane's 32 values raise the maximum once, and their exponents are one fused multiply-add each, d = z / log 2 - c
// with c the product of the maximum as rounded: sums relative to c are exact in that respect, and the 32 values' are brought
// to the maximum itself.  (Where the product is large, so that its rounding is, the values are subtracted first: masks
// of -1e10 or a type's lowest value.)
// Rows are cut into pieces where there are too few of them to fill the chip (a sampled token is one row); a
// second launch joins a row's pieces.  The best tokens: the K-th largest of the threads' maxima is a value
// that at least K elements reach, and seldom many more do; a second look at the piece lists those, and the
// list is ranked by (value, index), so that the order in which it was filled does not matter.  A piece where
// the list does not hold them (many equal values) is searched K times instead.
//
// Backward.  A stream: p = exp(z - m - log s) from the row's saved m and log s.
//
// Measured (8,192 rows of 50,304 bf16): forward 162 us = 5.1 TB/s, about ten vector instructions a value behind the loads, 132
// without the entropy; backward 268 us = 6.1 TB/s, memory.  1,021 rows of 32,101 fp16 with the 20 best: 27 us, of which memory is 11: one round
// of workgroups, each a chain of first look, threshold, second look and ranking.
#include "device.hip.h"

namespace deto {
namespace model {
namespace {

constexpr int kThreads = 256;                  // of the join and of the backward pass
constexpr int kMaxTop = 32;
constexpr int kKeys = 256;                     // maxima of parts of a piece that the threshold is taken of
constexpr int kList = 1024;                    // listed candidates of a piece
constexpr int kMaxPieces = kList / kMaxTop;    // the join ranks kMaxTop of every piece in one list
static_assert(kMaxPieces <= kLanes, "a lane for each piece");
constexpr int64_t kPieceElems = 1 << 16;       // above a piece's length, if there are no more of them than
constexpr int64_t kFillWorkgroups = 512;       // fill the chip

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
    int64_t V, ld, row0;     // row0: of this launch
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
// Products of the maximum that values are fused with: up to here their rounding is 2^-4 at most.
constexpr float kInRange = 1 << 20;

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

template <int DT, int THREADS, bool ONCE>
struct Piece {
    const void* logits;
    int64_t row, first, end;
    __device__ __forceinline__ int64_t at(int64_t d, int i) const { return d + i * THREADS * 8; }
    __device__ __forceinline__ int count(int64_t d, int i) const {
        const int64_t left = end - at(d, i);
        return left >= 8 ? 8 : left > 0 ? static_cast<int>(left) : 0;
    }
    __device__ __forceinline__ void load(int64_t d, Raw8<DT> (&raw)[kVectors<DT>]) const {
#pragma unroll
        for (int i = 0; i < kVectors<DT>; ++i) raw[i] = load8<DT, ONCE>(logits, row, at(d, i), count(d, i));
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

// r and the lane's next values, relative to the larger maximum.
template <int DT, bool ENTROPY>
__device__ __forceinline__ void see(Seen& r, const Taken<DT>& x, float unit) {
    float m = r.m;
#pragma unroll
    for (int i = 0; i < kVectors<DT>; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) m = larger(m, x.v[i][j]);
    const Seen before = relative_to(r, m, unit);
    const float ref = m == -__builtin_inff() ? 0.f : m, c = ref * unit;
    float s = 0.f, w = 0.f;
    if (fabsf(c) <= kInRange) {
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
        // from the rounded product to the maximum itself
        const float off = __builtin_fmaf(ref, unit, -c), e = exp2_fast(-off);
        w = (w - off * s) * e;
        s *= e;
    } else {           // (an infinity or a NaN as well: its sums are NaNs)
#pragma unroll
        for (int i = 0; i < kVectors<DT>; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = (x.v[i][j] - ref) * unit, e = exp2_fast(d);
                s += e;
                if constexpr (ENTROPY) w = __builtin_fmaf(fmaxf(d, kFarBelow), e, w);
            }
    }
    r = {m, before.s + s, before.w + w};
}

// The whole workgroup's, in every thread.
template <int WAVES>
__device__ __forceinline__ Seen join_workgroup(Seen r, float unit, Seen* lds) {
    r = join_wave(r, unit);
    const int lane = threadIdx.x % kLanes;
    if (lane == 0) lds[threadIdx.x / kLanes] = r;
    __syncthreads();
    r = {-__builtin_inff(), 0.f, 0.f};
    if (lane < WAVES) r = lds[lane];
    return join_wave(r, unit);
}

// The K-th largest of kKeys keys, down to its upper 16 bits, by bisection: counts in one wavefront, which holds all.
__device__ __forceinline__ uint32_t kth_key(const uint32_t* lds_keys, int K) {
    uint32_t k[kKeys / kLanes];
#pragma unroll
    for (int i = 0; i < kKeys / kLanes; ++i) k[i] = lds_keys[i * kLanes + threadIdx.x % kLanes];
    uint32_t found = 0;
#pragma unroll
    for (int bit = 31; bit >= 16; --bit) {
        const uint32_t t = found | 1u << bit;
        int n = 0;
#pragma unroll
        for (int i = 0; i < kKeys / kLanes; ++i) n += __popcll(__ballot(k[i] >= t));
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

// Elements of a lane that stay in registers between the two looks at a piece: a second look at memory is what they
// save.
constexpr int kKept = 64;

template <int DT, bool ENTROPY, bool TOP, int THREADS, bool ONCE>
__global__ __launch_bounds__(THREADS) void logprobs_kernel(Forward a) {
    constexpr int kWaves = THREADS / kLanes, V8 = kVectors<DT>, kKeep = TOP && THREADS > 256 ? kKept / (8 * V8) : 1;
    __shared__ Seen lds_seen[kWaves];
    const int64_t t = a.row0 + blockIdx.x / a.parts.pieces;
    const int piece = blockIdx.x % a.parts.pieces;
    const int64_t begin = piece * a.piece;
    const Piece<DT, THREADS, ONCE> p = {a.logits, t * a.ld, begin, begin + a.piece < a.V ? begin + a.piece : a.V};
    const bool whole = a.parts.pieces == 1;
    Target y = {};
    if (whole) y = load_target<DT>(a, t);
    constexpr int64_t kStep = THREADS * 8 * V8;
    const int64_t mine = p.first + 8 * threadIdx.x;
    Seen r = {-__builtin_inff(), 0.f, 0.f};
    Raw8<DT> raw[kKeep][V8];
    Taken<DT> x;
    const bool kept = p.end - p.first <= kKeep * kStep;
    if constexpr (kKeep > 1) {
        // The first kKeep steps' loads go out together.
#pragma unroll
        for (int k = 0; k < kKeep; ++k)
            if (mine + k * kStep < p.end) p.load(mine + k * kStep, raw[k]);
#pragma unroll
        for (int k = 0; k < kKeep; ++k)
            if (mine + k * kStep < p.end) {
                p.unpack(mine + k * kStep, raw[k], x);
                see<DT, ENTROPY>(r, x, a.unit);
            }
        for (int64_t d = mine + kKeep * kStep; d < p.end; d += kStep) {
            Raw8<DT> more[V8];
            p.load(d, more);
            p.unpack(d, more, x);
            see<DT, ENTROPY>(r, x, a.unit);
        }
    } else {
        // A step's loads go out before the one before is summed.
        if (mine < p.end) p.load(mine, raw[0]);
        for (int64_t d = mine; d < p.end; d += kStep) {
            p.unpack(d, raw[0], x);
            if (d + kStep < p.end) p.load(d + kStep, raw[0]);
            see<DT, ENTROPY>(r, x, a.unit);
        }
    }
    uint32_t key = mine < p.end ? order_key(r.m) : 0u;
    r = join_workgroup<kWaves>(r, a.unit, lds_seen);
    if (threadIdx.x == 0) {
        if (whole) write_row(a, t, r, y);
        else a.parts.seen[blockIdx.x] = r;
    }
    if constexpr (TOP) {
        __shared__ uint32_t lds_keys[kKeys];
        __shared__ uint64_t list[kList + 8];
        __shared__ uint32_t listed, threshold;
        const float log_s = logf(r.s);
        uint64_t* part = a.parts.best + static_cast<int64_t>(blockIdx.x) * a.top;
        auto give = [&](int rank, uint64_t c) {
            if (whole) write_best(a, t, rank, c, r.m, log_s);
            else part[rank] = c;
        };
        // a key for each kShare neighbours
        constexpr int kShare = THREADS / kKeys;
#pragma unroll
        for (int step = 1; step < kShare; step <<= 1) {
            const uint32_t o = __shfl_xor(key, step);
            key = o > key ? o : key;
        }
        if (threadIdx.x % kShare == 0) lds_keys[threadIdx.x / kShare] = key;
        if (threadIdx.x == 0) listed = 0;
        __syncthreads();
        if (threadIdx.x < kLanes) {
            const uint32_t found = kth_key(lds_keys, a.top);
            if (threadIdx.x == 0) threshold = found;
        }
        __syncthreads();
        const uint32_t least = threshold;
        // (0: fewer than `top` threads saw a value, all of them are listed; a NaN is not below anything)
        const float least_value = least > kLowestKey ? key_value(least) : -__builtin_inff();
        auto look = [&](int64_t d) {
#pragma unroll
            for (int i = 0; i < V8; ++i) {
                const float(&v)[8] = x.v[i];
                float m = v[0];
#pragma unroll
                for (int j = 1; j < 8; ++j) m = larger(m, v[j]);
                if (m < least_value) continue;
                const int n = p.count(d, i);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (j < n && !(v[j] < least_value)) {
                        const uint32_t at = atomicAdd(&listed, 1u);
                        if (at < kList)
                            list[at] = candidate(order_key(v[j]), static_cast<uint32_t>(p.at(d, i) + j));
                    }
                }
            }
        };
        if (kKeep > 1 && kept) {
#pragma unroll
            for (int k = 0; k < kKeep; ++k)
                if (mine + k * kStep < p.end) {
                    p.unpack(mine + k * kStep, raw[k], x);
                    look(mine + k * kStep);
                }
        } else {
            if (mine < p.end) p.load(mine, raw[0]);
            for (int64_t d = mine; d < p.end; d += kStep) {
                p.unpack(d, raw[0], x);
                if (d + kStep < p.end) p.load(d + kStep, raw[0]);
                look(d);
            }
        }
        __syncthreads();
        const int n = listed;
        if (n <= kList) {
            fill_up(list, n);
            __syncthreads();
            for (int i = threadIdx.x; i < n; i += THREADS) {
                const uint64_t c = list[i];
                const int rank = rank_of(list, n, c);
                if (rank < a.top) give(rank, c);
            }
            // a piece of fewer than `top` elements: the rest of its part is empty
            for (int i = n + threadIdx.x; i < a.top; i += THREADS) give(i, 0);
            return;
        }
        // Too many reach the threshold: one search for each place, each for the largest candidate below the
        // one before.
        uint64_t before = ~uint64_t{0};
        for (int rank = 0; rank < a.top; ++rank) {
            uint64_t best = 0;
            for (int64_t d = mine; d < p.end; d += THREADS * 8) {
                const int n_there = p.count(d, 0);
                float v[8];
                unpack8<DT>(load8<DT>(a.logits, p.row, d, n_there), v);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint64_t c = candidate(order_key(v[j]), static_cast<uint32_t>(d + j));
                    if (j < n_there && c < before && c > best) best = c;
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
    int64_t V, ld, ld_out, row0;
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

template <int DT, bool ENTROPY, bool ONCE>
__global__ __launch_bounds__(kThreads) void logprobs_backward_kernel(Backward a) {
    const int64_t t = a.row0 + blockIdx.x / a.pieces;
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
        raw[i] = load8<DT, ONCE>(a.logits, t * a.ld, first + i * kThreads * 8, count[i]);
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
        store8<DT, ONCE>(a.dlogits, t * a.ld_out + d, v, count[i]);
    }
}

bool bad_shape(int64_t T, int64_t V, int top) {
    return T < 0 || V < 1 || V > 0x7FFFFFFF || top < 0 || top > kMaxTop || top > V;
}

// (scale / log 2 is a number)
bool bad_scale(float scale) { return !(scale > 0.f && scale <= 0x1p127f); }

// Few rows take a workgroup of 1,024 threads each (one row of 50,304 bf16 logits with its eight best: 25 pieces and
// their join 13 us, 1,024 threads 10 us: 3 of them the exponentials of one CU, the rest a chain of latencies).  Rows that are long even for those are cut in pieces.
constexpr int64_t kFewRows = 512;
constexpr int kThreadsFew = 1024, kThreadsMany = 256;

int pieces_of(int64_t T, int64_t V) {
    if (T >= kFewRows) return 1;
    int64_t want = V / kPieceElems + 1;
    if (T * want > kFillWorkgroups) want = kFillWorkgroups / T;
    if (want > kMaxPieces) want = kMaxPieces;
    return want < 1 ? 1 : static_cast<int>(want);
}

// Logits that the caches do not hold until the backward pass, nor their gradient until whoever takes that: loads and
// stores that leave no trace there are faster (8,192 x 50,304 bf16, forward and backward, us: 467, without 430).
bool streams(int64_t T, int64_t V, int dtype) { return T * V * type_size(dtype) > kCacheBytes / 2; }

// Workgroups that a call counts in 31 bits.
constexpr int64_t kMaxGrid = 0x7FFFFFFF;

// One launch for each run of rows, of `pieces` workgroups each, whose threads are fewer than the 2^32 that a launch may have:
// launch(first row, workgroups).
template <class F>
void for_rows(int64_t T, int64_t pieces, int threads, F launch) {
    const int64_t most = 0xFFFFFFFF / threads / pieces;
    for (int64_t t = 0; t < T; t += most) launch(t, static_cast<unsigned>((T - t < most ? T - t : most) * pieces));
}

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
    if (bad_scale(logit_scale)) return DETO_ERR_BAD_CONFIG;
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
    Forward a = {V, logits->ld, 0, logits->data, logit_scale, logit_scale * 1.4426950408889634f,
                       targets, target_bytes, logp, lse, entropy, top, top_idx, top_logp, stats,
                       {reinterpret_cast<Seen*>(ws),
                        pieces > 1 ? reinterpret_cast<uint64_t*>(ws + seen_bytes) : nullptr, pieces},
                       piece};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    fresh();
    const auto run = [&](auto dt, auto threads, auto once) {
        constexpr int DT = decltype(dt)::value, THREADS = decltype(threads)::value;
        constexpr bool ONCE = decltype(once)::value;
        for_rows(T, pieces, THREADS, [&](int64_t row0, unsigned grid) {      // (of several pieces: T is below kFewRows)
            a.row0 = row0;
            if (top) {      // (looks at the logits twice)
                if (entropy) logprobs_kernel<DT, true, true, THREADS, false><<<grid, THREADS, 0, st>>>(a);
                else logprobs_kernel<DT, false, true, THREADS, false><<<grid, THREADS, 0, st>>>(a);
            } else {
                if (entropy) logprobs_kernel<DT, true, false, THREADS, ONCE><<<grid, THREADS, 0, st>>>(a);
                else logprobs_kernel<DT, false, false, THREADS, ONCE><<<grid, THREADS, 0, st>>>(a);
            }
        });
    };
    by_type(logits->dtype, [&](auto dt) {
        if (T < kFewRows) run(dt, Type<kThreadsFew>{}, std::false_type{});
        else if (streams(T, V, logits->dtype)) run(dt, Type<kThreadsMany>{}, std::true_type{});
        else run(dt, Type<kThreadsMany>{}, std::false_type{});
        if (pieces > 1)
            logprobs_join_kernel<dt.value><<<static_cast<unsigned>(T), kThreads, 0, st>>>(a);
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
    if (bad_scale(logit_scale)) return DETO_ERR_BAD_CONFIG;
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
    Backward a = {V, logits->ld, dlogits->ld, 0, logits->data, dlogits->data, logit_scale,
                        logit_scale * 1.4426950408889634f, targets, target_bytes, stats, entropy,
                        g_logp, g_entropy, static_cast<uint32_t>(pieces)};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    fresh();
    by_type(logits->dtype, [&](auto dt) {
        constexpr int DT = dt.value;
        const auto run = [&](auto once) {
            constexpr bool ONCE = decltype(once)::value;
            for_rows(T, pieces, kThreads, [&](int64_t row0, unsigned grid) {
                a.row0 = row0;
                if (g_entropy) logprobs_backward_kernel<DT, true, ONCE><<<grid, kThreads, 0, st>>>(a);
                else logprobs_backward_kernel<DT, false, ONCE><<<grid, kThreads, 0, st>>>(a);
            });
        };
        if (streams(T, V, logits->dtype)) run(std::true_type{});
        else run(std::false_type{});
        return 0;
    });
    return enqueued();
}

}  // extern "C"
