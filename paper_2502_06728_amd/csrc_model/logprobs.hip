// Log probabilities of given tokens: log sum exp, entropy and the best tokens of every row of the logits, and
// the gradient of the logits.
//
// Forward.  A workgroup takes a piece of a row: one pass with the running maximum m, s = sum exp(z - m) and
// w = sum (z - m) exp(z - m), in fp32 and in units of log 2:
//     lse = m + log s        entropy = log s - w / s
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
constexpr int64_t kPieceElems = kThreads * 8;  // least length of a piece: eight elements a lane
constexpr int64_t kFillWorkgroups = 1024;      // workgroups that fill the chip

// What a piece, or a part of one, has seen: m over the raw logits; s, w scaled (w in units of log 2).  m is
// -infinity before the first value above that.
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

// a and b as one.  (m = -infinity stands for nothing above it: no difference is taken from it.)
__device__ __forceinline__ Seen join(const Seen& a, const Seen& b, float unit) {
    const float m = fmaxf(a.m, b.m);
    const float ref = m == -__builtin_inff() ? 0.f : m;
    const float da = fmaxf((a.m - ref) * unit, -16384.f), db = fmaxf((b.m - ref) * unit, -16384.f);
    const float ea = exp2_fast(da), eb = exp2_fast(db);
    return {m, a.s * ea + b.s * eb, (a.w + a.s * da) * ea + (b.w + b.s * db) * eb};
}

// An order of all values, NaNs above everything, -0 and +0 the same: larger means earlier.  0 is no value, and
// no candidate is all ones.
constexpr uint32_t kNanKey = 0xFFFFFFFEu;
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

template <int DT>
__device__ __forceinline__ void write_row(const Forward& a, int64_t t, const Seen& r) {
    const float log_s = logf(r.s);
    const bool none = r.m == -__builtin_inff() && r.s == 0.f;       // -infinities throughout
    const float top = r.m * a.scale;
    const int64_t y = target_of(a.targets, a.target_bytes, t);
    float logp = 0.f;
    if (y >= 0 && y < a.V) {
        const float z = load1<DT>(a.logits, t * a.ld + y);
        logp = none ? -__builtin_inff() : (z - r.m) * a.scale - log_s;
    }
    a.logp[t] = logp;
    if (a.lse) a.lse[t] = none ? -__builtin_inff() : top + log_s;
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

// (a NaN row's s is NaN: a NaN, or +infinity - +infinity)
template <int DT, bool ENTROPY>
__device__ __forceinline__ void see8(Seen& r, const float (&v)[8], float unit) {
    float m = r.m;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = fmaxf(m, v[j]);
    const float ref = m == -__builtin_inff() ? 0.f : m;
    const float d0 = fmaxf((r.m - ref) * unit, -16384.f), e0 = exp2_fast(d0);
    float s = r.s * e0, w = (r.w + r.s * d0) * e0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float d = (v[j] - ref) * unit, e = exp2_fast(d);
        s += e;
        if constexpr (ENTROPY) w += fmaxf(d, -16384.f) * e;
    }
    r = {m, s, w};
}

// The same over all threads of the workgroup, in every thread.
__device__ __forceinline__ Seen join_workgroup(Seen r, float unit, Seen* lds) {
#pragma unroll
    for (int step = 1; step < kLanes; step <<= 1)
        r = join(r, {__shfl_xor(r.m, step), __shfl_xor(r.s, step), __shfl_xor(r.w, step)}, unit);
    if (threadIdx.x % kLanes == 0) lds[threadIdx.x / kLanes] = r;
    __syncthreads();
    r = lds[0];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) r = join(r, lds[i], unit);
    return r;
}

template <int DT, bool ENTROPY, bool TOP>
__global__ __launch_bounds__(kThreads) void logprobs_kernel(Forward a) {
    __shared__ Seen lds_seen[kWaves];
    const int64_t t = blockIdx.x / a.parts.pieces;
    const int piece = blockIdx.x % a.parts.pieces;
    const int64_t first = piece * a.piece;
    const int64_t end = first + a.piece < a.V ? first + a.piece : a.V;
    const int64_t row = t * a.ld;
    Seen r = {-__builtin_inff(), 0.f, 0.f};
    uint32_t key = 0;                       // the thread's largest
    for (int64_t d = first + 8 * threadIdx.x; d < end; d += kThreads * 8) {
        const int count = end - d < 8 ? static_cast<int>(end - d) : 8;
        float v[8];
        unpack8<DT>(load8<DT>(a.logits, row, d, count), v);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (j >= count) v[j] = -__builtin_inff();
            else if constexpr (TOP) {
                const uint32_t k = order_key(v[j]);
                key = k > key ? k : key;
            }
        }
        see8<DT, ENTROPY>(r, v, a.unit);
    }
    r = join_workgroup(r, a.unit, lds_seen);
    const bool whole = a.parts.pieces == 1;
    if (threadIdx.x == 0) {
        if (whole) write_row<DT>(a, t, r);
        else a.parts.seen[blockIdx.x] = r;
    }
    if constexpr (TOP) {
        __shared__ uint32_t lds_keys[kThreads];
        __shared__ uint64_t list[kList];
        __shared__ uint32_t threshold, listed;
        const float log_s = logf(r.s);
        uint64_t* part = a.parts.best + static_cast<int64_t>(blockIdx.x) * a.top;
        auto give = [&](int rank, uint64_t c) {
            if (whole) write_best(a, t, rank, c, r.m, log_s);
            else part[rank] = c;
        };
        lds_keys[threadIdx.x] = key;
        if (threadIdx.x == 0) listed = 0;
        __syncthreads();
        int above = 0;                      // of the threads' keys, before this one's
        for (int i = 0; i < kThreads; ++i) {
            const uint32_t k = lds_keys[i];
            above += k > key || (k == key && i < static_cast<int>(threadIdx.x));
        }
        if (above == a.top - 1) threshold = key;
        __syncthreads();
        const uint32_t least = threshold ? threshold : 1u;   // 0: fewer than `top` threads saw a value
        for (int64_t d = first + 8 * threadIdx.x; d < end; d += kThreads * 8) {
            const int count = end - d < 8 ? static_cast<int>(end - d) : 8;
            float v[8];
            unpack8<DT>(load8<DT>(a.logits, row, d, count), v);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t k = order_key(v[j]);
                if (j < count && k >= least) {
                    const uint32_t at = atomicAdd(&listed, 1u);
                    if (at < kList) list[at] = candidate(k, static_cast<uint32_t>(d + j));
                }
            }
        }
        __syncthreads();
        const int n = listed;
        if (n <= kList) {
            for (int i = threadIdx.x; i < n; i += kThreads) {
                const uint64_t c = list[i];
                int rank = 0;
                for (int j = 0; j < n; ++j) rank += list[j] > c;
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
            for (int64_t d = first + 8 * threadIdx.x; d < end; d += kThreads * 8) {
                const int count = end - d < 8 ? static_cast<int>(end - d) : 8;
                float v[8];
                unpack8<DT>(load8<DT>(a.logits, row, d, count), v);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint64_t c = candidate(order_key(v[j]), static_cast<uint32_t>(d + j));
                    if (j < count && c < before && c > best) best = c;
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

// A workgroup per row: its pieces as one.
template <int DT>
__global__ __launch_bounds__(kThreads) void logprobs_join_kernel(Forward a) {
    __shared__ Seen lds_seen[kWaves];
    __shared__ uint64_t list[kList];
    const int64_t t = blockIdx.x;
    const int pieces = a.parts.pieces;
    Seen r = {-__builtin_inff(), 0.f, 0.f};
    for (int i = threadIdx.x; i < pieces; i += kThreads)
        r = join(r, a.parts.seen[t * pieces + i], a.unit);
    r = join_workgroup(r, a.unit, lds_seen);
    if (threadIdx.x == 0) write_row<DT>(a, t, r);
    if (a.top == 0) return;
    const int n = pieces * a.top;           // at most kList
    const uint64_t* part = a.parts.best + t * n;
    for (int i = threadIdx.x; i < n; i += kThreads) list[i] = part[i];
    __syncthreads();
    const float log_s = logf(r.s);
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const uint64_t c = list[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += list[j] > c;
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
