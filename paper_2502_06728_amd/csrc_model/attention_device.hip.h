// What the kernels of attention share: sequences and their tiles, matrices in LDS, the two products on the matrix cores.
//
// Every product is one of 32 x 32 blocks (a wavefront's instruction), in two forms:
//   rows    C[i][j] = sum_d A[i][d] B[j][d]     over features: scores, and dout . v.  A comes from LDS, B is in registers.
//   columns C[d][j] += sum_i A[i][d] W[i][j]    over rows i: what the scores weigh.  A comes from LDS turned, W are
//           results of the first form: a lane holds, of one column j = lane % 32, the rows
//           (r / 4) * 8 + (lane / 32) * 4 + r % 4 in its registers r = 0 ... 15.  The sum may take its rows in any order:
//           both operands take them in the one in which W already lies, so W never leaves its lanes.
// So a lane has one query (or, for the gradients of keys, one key) throughout: its maximum, sum and bounds are one
// register each.
#pragma once

#include "device.hip.h"

namespace deto {
namespace model {
namespace attention {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kSide = 32;               // of a block
constexpr int kCUs = 256;
constexpr float kLog2E = 1.44269504088896341f, kLn2 = 0.693147180559945309f;

// A head's features: rows of DP in LDS, of which products take the first DU (zeros behind the last feature).
template <int DT_, int DP_, int DU_>
struct Shape {
    static constexpr int DT = DT_, DP = DP_, DU = DU_;
    static constexpr int kElem = kSize<DT>;
    static constexpr int kRow = DP * kElem;             // bytes of a row in LDS
    static constexpr int kPieces = kRow / 16;           // of 16 bytes
    static constexpr int kOf = 16 / kElem;              // features of a piece
    static constexpr int kFrags = DU * kElem / 32;      // operands of the rows form: two pieces, one for each half of the lanes
    static constexpr int kBlocks = DU / kSide;          // blocks of features
};

// The wavefronts that a SIMD is given registers for (three with up to 64 features of 16 bits: four would spill).
template <class S> constexpr int kResident = S::DP == 64 && S::DT != DETO_F32 ? 3 : 2;
// Keys of a step of a walk over keys
template <class S, int W> constexpr int kKeys = S::DT == DETO_F32 || S::DP == 64 || W == 4 ? 32 : 64;

struct Matrix {
    char* data;
    int64_t ld;       // in bytes
};

struct Args {
    Matrix q, k, v, out, dout, dq, dk, dv;
    float* lse;
    float* stats;                        // [3, heads, Tq]: lse in powers of two (or a far base's power), dout . out, a far base's score
    const int32_t *q_starts, *k_starts;
    int64_t Tq, Tk, sequences;
    int32_t heads, kv_heads, group, head_dim, causal;
    float scale;
    uint32_t tiles;                      // of one head (with starts: at most), see Plan
    uint32_t per_sequence;               // tiles of one sequence, without starts
    float* parts;                        // [splits, heads * Tq, part_row(head_dim)], where a walk is cut into several
};

// A split's sums for a query are a row of floats: a head's features, in whole pieces of four.  Behind all of those the
// forward pass has three planes of splits * heads * Tq: bases (two) and sums of weights; the backward pass as many rows again, the
// sums of p k, and one plane, the sums of ds.
__host__ __device__ __forceinline__ int part_row(int head_dim) { return (head_dim + 3) / 4 * 4; }

// ---- sequences
struct Sequence {
    int64_t q0, k0;      // first rows
    int32_t Lq, Lk;
};

__device__ __forceinline__ int64_t clamped(int64_t at, int64_t T) { return at < 0 ? 0 : at < T ? at : T; }

__device__ __forceinline__ void span_of(const int32_t* starts, int64_t s, int64_t sequences, int64_t T, int64_t& first,
                                        int32_t& length) {
    if (starts) {
        first = clamped(starts[s], T);
        const int64_t end = clamped(starts[s + 1], T);
        length = end > first ? static_cast<int32_t>(end - first) : 0;
    } else {
        length = static_cast<int32_t>(T / sequences);
        first = s * length;
    }
}

// what is the same in all lanes, in a scalar register
__device__ __forceinline__ int32_t uniform(int32_t v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform(int64_t v) {
    const uint32_t lo = uniform(static_cast<int32_t>(v)), hi = uniform(static_cast<int32_t>(v >> 32));
    return static_cast<int64_t>(uint64_t{hi} << 32 | lo);
}

__device__ __forceinline__ Sequence sequence_of(const Args& a, int64_t s) {
    Sequence seq;
    span_of(a.q_starts, s, a.sequences, a.Tq, seq.q0, seq.Lq);
    span_of(a.k_starts, s, a.sequences, a.Tk, seq.k0, seq.Lk);
    return {uniform(seq.q0), uniform(seq.k0), uniform(seq.Lq), uniform(seq.Lk)};
}

// Tile number `id` of all packed sequences' rows, `size` rows a tile: its sequence, and which of that one's tiles it is.
// False where there are fewer.  The sequences' tiles are counted 64 at a time, a lane each.
__device__ __forceinline__ bool find_tile(const Args& a, const int32_t* starts, int64_t T, int size, uint32_t id,
                                          int64_t& s, int32_t& tile, int32_t& tiles) {
    const int lane = threadIdx.x % kLanes;
    int64_t before = 0;
    for (int64_t base = 0; base < a.sequences; base += kLanes) {
        int64_t first;
        int32_t length = 0;
        if (base + lane < a.sequences) span_of(starts, base + lane, a.sequences, T, first, length);
        const int32_t own = length / size + (length % size != 0);
        int64_t upto = own;
#pragma unroll
        for (int by = 1; by < kLanes; by *= 2) {
            const int64_t below = __shfl_up(upto, by);
            if (lane >= by) upto += below;
        }
        const uint64_t past = __ballot(before + upto > static_cast<int64_t>(id));
        if (past) {
            const int at = __builtin_ctzll(past);
            s = uniform(base + at);
            tile = uniform(static_cast<int32_t>(id - before - __shfl(upto - own, at)));
            tiles = uniform(__shfl(own, at));
            return true;
        }
        before += __shfl(upto, kLanes - 1);
    }
    return false;
}

// A workgroup's tile and head.  Workgroups go to the chip's eight parts in turn; heads are dealt out so that those in a
// row, which share keys, meet in one part, whose own cache then holds these for all of them.  Under a mask the longest
// tiles of all heads and of all sequences of one length come first (`last_first`: those are the last ones), so that no long
// one is left over at the end; packed sequences follow in their order, each one's longest tiles first.  Without a mask, a
// head's tiles follow each other.
struct Place {
    int64_t s;
    int32_t head, tile;
};
__device__ __forceinline__ bool place_of(const Args& a, const int32_t* starts, int64_t T, int size, int heads, bool last_first,
                                         Place& p) {
    const uint32_t rows = starts ? a.tiles : a.per_sequence;                 // of the grid: tiles of a column
    const uint32_t columns = starts ? heads : static_cast<uint32_t>(heads * a.sequences);
    uint32_t row, column;
    if (a.causal) {
        row = blockIdx.x / columns;
        column = blockIdx.x % columns;
        if (columns % 8 == 0) column = column % 8 * (columns / 8) + column / 8;
    } else {
        const uint32_t all = gridDim.x, part = blockIdx.x % 8, each = all / 8, more = all % 8;
        const uint32_t n = part * each + (part < more ? part : more) + blockIdx.x / 8;
        row = n % rows;
        column = n / rows;
    }
    int32_t tiles;
    if (starts) {
        p.head = column;
        if (!find_tile(a, starts, T, size, row, p.s, p.tile, tiles)) return false;
    } else {
        p.s = column / heads;
        p.head = column % heads;
        p.tile = row;
        tiles = rows;
    }
    if (last_first) p.tile = tiles - 1 - p.tile;
    return true;
}

// ---- matrices in LDS.  Four rows lie together, in blocks of 256 bytes: four pieces of each row side by side, in an
// order of their own for each of four such fours.  So the rows form (a piece of each of 16 rows) and the columns form
// (four pieces of four rows) both read 256 bytes of different banks, and a lane's places differ by constants but for two
// in each form.
template <class S>
__device__ __forceinline__ uint32_t place(int row, int piece) {
    return row / 4 * 4 * S::kRow + piece / 4 * 256 + row % 4 * 64 + ((piece ^ row / 4) & 3) * 16;
}

struct Places {
    uint32_t rows[2];       // of a lane's piece 0 and 2 (or 1 and 3) of its row: the others are 256 bytes apart
    uint32_t turned[2];     // of what it reads for the columns form in the first and the second eight rows
};
template <class S>
__device__ __forceinline__ Places places_of() {
    const int lane = threadIdx.x % kLanes, half = lane / kSide;
    Places p;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        p.rows[i] = place<S>(lane % kSide, 2 * i + half);
        if constexpr (S::DT == DETO_F32)
            p.turned[i] = place<S>(8 * i + 4 * half, lane % kSide / 4) + lane % 4 * 4;
        else        // sixteen lanes read four rows of sixteen features, four at a time, and get four rows of one feature
            p.turned[i] = place<S>(8 * i + 4 * half + lane % 16 / 4, lane / 16 % 2 * 2 + lane % 4 / 2) + lane % 2 * 8;
    }
    return p;
}

// piece `piece` of a row of D features: 16 bytes, zeros behind the last feature
// (WHOLE: there are no parts of a piece)
template <class S, bool WHOLE>
__device__ __forceinline__ u32x4 load_piece(const char* row, int piece, int D) {
    const int d = piece * S::kOf;
    u32x4 r = {0, 0, 0, 0};
    if constexpr (WHOLE) {
        const u32x4 v = *reinterpret_cast<const u32x4_any2*>(row + (d < D ? d : 0) * S::kElem);
        return d < D ? v : r;
    }
    if (d + S::kOf <= D) return *reinterpret_cast<const u32x4_any2*>(row + d * S::kElem);
    if (d >= D) return r;
    if constexpr (S::DT == DETO_F32) {
#pragma unroll
        for (int j = 0; j < 3; ++j)
            if (d + j < D) r[j] = reinterpret_cast<const uint32_t*>(row)[d + j];
    } else {
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (d + j < D) r[j / 2] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(row)[d + j]) << (16 * (j % 2));
    }
    return r;
}

// Rows into LDS by a workgroup of W wavefronts.  Rows that are missing at the end of a sequence are copies of the last
// one: what they are multiplied with is zero.
// DIRECT: heads of whole pieces at multiples of 4 bytes, from memory to LDS without a register: a wavefront's call writes
// 64 pieces in a row, so its lanes read the pieces that belong there (those behind the last feature stay as they are).
// begin() starts kCalls of these; who reads the rows waits until they have come (arrived()), and for the other wavefronts'
// (meet()).
// Otherwise through registers: begin() loads, end() stores.
template <class S, int ROWS, int W, bool DIRECT>
struct Rows {
    static constexpr int kThreads = W * kLanes, kUnits = DIRECT ? 1 : ROWS * S::kPieces / kThreads;
    static constexpr int kCalls = ROWS * S::kPieces / kThreads;
    static_assert(ROWS * S::kPieces % kThreads == 0, "");
    u32x4 r[kUnits];
    uint32_t off[DIRECT ? kCalls : 1];      // what a lane reads in each call, in bytes from the first row, if all rows are there

    // (the inverse of place)
    static __device__ __forceinline__ int row_of(int slot) { return slot / (4 * S::kPieces) * 4 + slot / 4 % 4; }
    static __device__ __forceinline__ int piece_of(int slot) {
        return slot / 16 % (S::kPieces / 4) * 4 + ((slot ^ slot / (4 * S::kPieces)) & 3);
    }
    __device__ __forceinline__ explicit Rows(int64_t ld) {
        if constexpr (DIRECT) {
#pragma unroll
            for (int i = 0; i < kCalls; ++i) {
                const int slot = threadIdx.x + i * kThreads;
                off[i] = static_cast<uint32_t>(row_of(slot)) * static_cast<uint32_t>(ld) + piece_of(slot) * 16;
            }
        }
    }

    // `have` (1 or more) rows from `at` on
    __device__ __forceinline__ void begin(char* lds, const char* at, int64_t ld, int have, int D) {
        if constexpr (DIRECT) {
            const int wave = uniform(static_cast<int32_t>(threadIdx.x / kLanes));
            const auto call = [&](int i, uint32_t from) {
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(at + from),
                                                 (__attribute__((address_space(3))) void*)(lds + (wave + i * W) * kLanes * 16), 16, 0, 0);
            };
            if (have == ROWS && D == S::DP) {
#pragma unroll
                for (int i = 0; i < kCalls; ++i) call(i, off[i]);
            } else {
#pragma unroll
                for (int i = 0; i < kCalls; ++i) {
                    const int slot = threadIdx.x + i * kThreads, row = row_of(slot), piece = piece_of(slot);
                    if (piece * S::kOf < D)
                        call(i, static_cast<uint32_t>(row < have ? row : have - 1) * static_cast<uint32_t>(ld) + piece * 16);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < kUnits; ++i) {
                const int unit = threadIdx.x + i * kThreads, row = unit / S::kPieces;
                r[i] = load_piece<S, false>(at + (row < have ? row : have - 1) * ld, unit % S::kPieces, D);
            }
        }
    }
    __device__ __forceinline__ void end(char* lds) {
        if constexpr (!DIRECT) {
#pragma unroll
            for (int i = 0; i < kUnits; ++i) {
                const int unit = threadIdx.x + i * kThreads;
                *reinterpret_cast<u32x4*>(lds + place<S>(unit / S::kPieces, unit % S::kPieces)) = r[i];
            }
        }
    }
};

// The forward walk has the rows of two steps in LDS, which it computes with, and asks for kLead - 2 steps more; staged
// through registers, one is in these.  In 16 bits these do not stay on their way for long: the compiler takes the turned reads
// of the columns form for reads of what the copies to LDS write, and waits for all of a wavefront's loads before the first of
// them in each step, here and in the walks of both gradients.  (fp32 has none of these reads, nor that wait.)
template <bool DIRECT> constexpr int kLead = DIRECT ? 3 : 2;
template <bool DIRECT> constexpr int kBuffers = kLead<DIRECT> + 1;

// Zeros behind the last feature, before the first begin().
template <class S, int W>
__device__ __forceinline__ void clear(char* lds, int bytes, int D) {
    if (D == S::DP) return;
    for (int at = threadIdx.x * 16; at < bytes; at += W * kLanes * 16) *reinterpret_cast<u32x4*>(lds + at) = {0, 0, 0, 0};
    __syncthreads();
}

// All of this wavefront's loads but the last N have come (they come in order).
template <int N>
__device__ __forceinline__ void arrived() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// ... but those of the last `more` (0 ... 3) runs of N
template <int N>
__device__ __forceinline__ void arrived_but(int more) {
    if (more >= 3) arrived<3 * N>();
    else if (more == 2) arrived<2 * N>();
    else if (more == 1) arrived<N>();
    else arrived<0>();
}
// A barrier that leaves loads on their way.
__device__ __forceinline__ void meet() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

template <class S>
__device__ __forceinline__ bool is_odd(uint32_t word, uint32_t& cleaned) {      // holds an infinity or a NaN
    cleaned = word;
    if constexpr (S::DT == DETO_F32) {
        if ((word & 0x7F800000u) == 0x7F800000u) cleaned = 0;
    } else {
        constexpr uint32_t kExponent = S::DT == DETO_BF16 ? 0x7F80u : 0x7C00u;
        if ((word & kExponent) == kExponent) cleaned &= 0xFFFF0000u;
        if ((word & kExponent << 16) == kExponent << 16) cleaned &= 0xFFFFu;
    }
    return cleaned != word;
}

// Takes infinities and NaNs out of rows in LDS, and says whether there were any: in a product whose other operand has
// zeros for what is masked, they would reach what does not see them.  What they give to what does see them is added in
// the end, by scalar products (see `add_odd`): it is rare, and the kernels' loops stay small.
template <class S, int ROWS, int W>
__device__ __forceinline__ void take_out_odd(char* lds, uint32_t* found) {
    constexpr int kThreads = W * kLanes;
#pragma unroll
    for (int i = 0; i < ROWS * S::kPieces / kThreads; ++i) {
        u32x4* const at = reinterpret_cast<u32x4*>(lds + (threadIdx.x + i * kThreads) * 16);
        u32x4 r = *at;
        bool any = false;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            uint32_t cleaned;
            const uint32_t word = r[w];
            any |= is_odd<S>(word, cleaned);
            r[w] = cleaned;
        }
        if (any) {
            *at = r;
            *found = 1;
        }
    }
}

// Says whether there are any, and leaves them: for rows that the scores are computed from as well.
template <class S, int ROWS, int W>
__device__ __forceinline__ void find_odd(const char* lds, uint32_t* found) {
    constexpr int kThreads = W * kLanes;
    // (an exponent of all ones, and nothing else, carries into the bit above it)
    constexpr uint32_t kExponent = S::DT == DETO_F32 ? 0x7F800000u : S::DT == DETO_BF16 ? 0x7F807F80u : 0x7C007C00u;
    constexpr uint32_t kLowest = S::DT == DETO_F32 ? 0x00800000u : S::DT == DETO_BF16 ? 0x00800080u : 0x04000400u;
    constexpr uint32_t kAbove = S::DT == DETO_F32 ? 0x80000000u : 0x80008000u;
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < ROWS * S::kPieces / kThreads; ++i) {
        const u32x4 r = *reinterpret_cast<const u32x4*>(lds + (threadIdx.x + i * kThreads) * 16);
#pragma unroll
        for (int w = 0; w < 4; ++w) any |= (r[w] & kExponent) + kLowest;
    }
    if (any & kAbove) *found = 1;
}

// whether a row in memory holds any (a wavefront's lanes look at its features together)
template <class S>
__device__ __forceinline__ bool row_is_odd(const char* row, int D) {
    bool any = false;
    for (int d = threadIdx.x % kLanes; d < D; d += kLanes) any |= !(fabsf(load1<S::DT>(row, d)) < __builtin_inff());
    return __any(any);
}

// the scalar product of two rows in memory
template <class S>
__device__ __forceinline__ float slow_dot(const char* x, const char* y, int D) {
    float sum = 0.f;
#pragma unroll 1
    for (int d = 0; d < D; ++d) sum = fmaf(load1<S::DT>(x, d), load1<S::DT>(y, d), sum);
    return sum;
}

// Adds what a row's infinities and NaNs give under a weight to a row of results that is in memory already (the halves of
// the lanes take turns at the features).
template <class S, int OUT = S::DT>
__device__ __forceinline__ void add_odd(void* to, const char* row, int D, float weight) {
#pragma unroll 1
    for (int d = threadIdx.x / kSide % 2; d < D; d += 2) {
        const float v = load1<S::DT>(row, d);
        if (!(fabsf(v) < __builtin_inff())) store1<OUT>(to, d, load1<OUT>(to, d) + weight * v);
    }
}
// this wavefront's stores are there for its loads
__device__ __forceinline__ void stored() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup"); }

// ---- the rows form
template <int DT>
__device__ __forceinline__ f32x16 multiply(const u32x4& a, const u32x4& b, f32x16 c) {
    if constexpr (DT == DETO_BF16)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else if constexpr (DT == DETO_F16)
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else {
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(bits_f32(a[j]), bits_f32(b[j]), c, 0, 0, 0);
        return c;
    }
}

// a lane's row of B; one that is missing is zeros
template <class S, bool WHOLE>
__device__ __forceinline__ void load_row(const char* row, bool there, int D, u32x4 (&f)[S::kFrags]) {
    const int half = (threadIdx.x / kSide) % 2;
#pragma unroll
    for (int m = 0; m < S::kFrags; ++m) {
        f[m] = load_piece<S, WHOLE>(row, 2 * m + half, D);
        if (!there) f[m] = {0, 0, 0, 0};
    }
}

// BLOCKS blocks of 32 rows of a matrix in LDS times the lane's row
template <class S, int BLOCKS>
__device__ __forceinline__ void rows_product(const char* lds, const Places& at, const u32x4 (&b)[S::kFrags], f32x16 (&c)[BLOCKS]) {
#pragma unroll
    for (int k = 0; k < BLOCKS; ++k) c[k] = f32x16{};
#pragma unroll
    for (int m = 0; m < S::kFrags; ++m)
#pragma unroll
        for (int k = 0; k < BLOCKS; ++k) {
            const u32x4 a = *reinterpret_cast<const u32x4*>(lds + at.rows[m % 2] + m / 2 * 256 + k * kSide * S::kRow);
            c[k] = multiply<S::DT>(a, b[m], c[k]);
        }
}

// a block of rows with the lane's row in LDS too, among the 32 at `b`
template <class S>
__device__ __forceinline__ f32x16 block_product(const char* lds, const Places& at, const char* b) {
    f32x16 c = {};
#pragma unroll
    for (int m = 0; m < S::kFrags; ++m) {
        const uint32_t from = at.rows[m % 2] + m / 2 * 256;
        c = multiply<S::DT>(*reinterpret_cast<const u32x4*>(lds + from), *reinterpret_cast<const u32x4*>(b + from), c);
    }
    return c;
}
template <class S>
__device__ __forceinline__ f32x16 block_product(const char* lds, const Places& at, const u32x4 (&b)[S::kFrags]) {
    f32x16 c[1];
    rows_product<S, 1>(lds, at, b, c);
    return c[0];
}

// ---- the columns form
typedef __attribute__((address_space(3))) s16x4* TurnedAt;

// W as the second operand: one of two runs of 16 rows, rounded
template <int DT>
__device__ __forceinline__ u32x4 operand(const f32x16& w, int run) {
    u32x4 r;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float lo = w[8 * run + 2 * j], hi = w[8 * run + 2 * j + 1];
        r[j] = DT == DETO_BF16 ? pack_bf16(lo, hi) : pack_f16(lo, hi);
    }
    return r;
}
// ... and what the rounding took away, rounded in its turn (of the number that was rounded: fused with the product that it
// may be, the difference would have bits that depend on the loop it stands in)
template <int DT>
__device__ __forceinline__ u32x4 operand_rest(const f32x16& w, int run, const u32x4& rounded) {
#pragma clang fp contract(off)
    u32x4 r;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t two = rounded[j];
        float lo = w[8 * run + 2 * j], hi = w[8 * run + 2 * j + 1];
        if constexpr (DT == DETO_BF16) {
            lo -= bits_f32(two << 16);
            hi -= bits_f32(two & 0xFFFF0000u);
            r[j] = pack_bf16(lo, hi);
        } else {
            const f16x2 h = __builtin_bit_cast(f16x2, two);
            lo -= static_cast<float>(h.x);
            hi -= static_cast<float>(h.y);
            r[j] = pack_f16(lo, hi);
        }
    }
    return r;
}

// C += A^T W and E += A^T V with the same 32 rows A in LDS (SECOND: otherwise C alone); TWICE: W to twice the bits; CLEAN:
// without A's infinities and NaNs
template <class S, bool TWICE, bool SECOND, bool CLEAN = false>
__device__ __forceinline__ void columns_products(const char* lds, const Places& at, const f32x16& w, const f32x16& v,
                                                 f32x16 (&c)[S::kBlocks], f32x16* e) {
    if constexpr (S::DT == DETO_F32) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
#pragma unroll
            for (int b = 0; b < S::kBlocks; ++b) {
                uint32_t word = *reinterpret_cast<const uint32_t*>(lds + at.turned[r / 4 % 2] + r / 8 * 16 * S::kRow + r % 4 * 64 + b * 512);
                if constexpr (CLEAN) is_odd<S>(word, word);
                const float a = bits_f32(word);
                c[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, w[r], c[b], 0, 0, 0);
                if constexpr (SECOND) e[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, v[r], e[b], 0, 0, 0);
            }
        }
    } else {
#pragma unroll
        for (int run = 0; run < 2; ++run) {
            const u32x4 own = operand<S::DT>(w, run);
            u32x4 rest, other;
            if constexpr (TWICE) rest = operand_rest<S::DT>(w, run, own);
            if constexpr (SECOND) other = operand<S::DT>(v, run);
#pragma unroll
            for (int b = 0; b < S::kBlocks; ++b) {
                u32x4 a;
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const s16x4 four = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (TurnedAt)(lds + at.turned[s] + run * 16 * S::kRow + b * 256));
                    const u32x2 words = __builtin_bit_cast(u32x2, four);
                    a[2 * s] = words[0];
                    a[2 * s + 1] = words[1];
                }
                if constexpr (CLEAN) {
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        uint32_t cleaned;
                        is_odd<S>(a[w], cleaned);
                        a[w] = cleaned;
                    }
                }
                c[b] = multiply<S::DT>(a, own, c[b]);
                if constexpr (TWICE) c[b] = multiply<S::DT>(a, rest, c[b]);
                if constexpr (SECOND) e[b] = multiply<S::DT>(a, other, e[b]);
            }
        }
    }
}
template <class S, bool TWICE = false>
__device__ __forceinline__ void columns_product(const char* lds, const Places& at, const f32x16& w, f32x16 (&c)[S::kBlocks]) {
    columns_products<S, TWICE, false>(lds, at, w, w, c, nullptr);
}

// ---- both halves' maximum and sum of a column
__device__ __forceinline__ float halves_max(float v) {
    const auto both = __builtin_amdgcn_permlane32_swap(f32_bits(v), f32_bits(v), false, false);
    return fmaxf(bits_f32(both[0]), bits_f32(both[1]));
}
__device__ __forceinline__ float halves_sum(float v) {
    const auto both = __builtin_amdgcn_permlane32_swap(f32_bits(v), f32_bits(v), false, false);
    return bits_f32(both[0]) + bits_f32(both[1]);
}

// Columns of C times a factor into the lanes' rows of a matrix, 16 bytes a lane: the two halves of the lanes, which hold
// four features each of every eight, exchange theirs for that.
template <class S>
__device__ __forceinline__ void store_block(const f32x16& c, int b, float factor, char* row, bool there, int D) {
    const int half = threadIdx.x / kSide % 2;
    if constexpr (S::DT == DETO_F32) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int d = b * kSide + 8 * g + 4 * half;
            u32x4 v;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = f32_bits(c[4 * g + j] * factor);
            if (there && d + 4 <= D) *reinterpret_cast<u32x4_any4*>(row + d * 4) = v;
            else if (there) {
#pragma unroll
                for (int j = 0; j < 3; ++j)
                    if (d + j < D) reinterpret_cast<uint32_t*>(row)[d + j] = v[j];
            }
        }
    } else {
#pragma unroll
        for (int g = 0; g < 4; g += 2) {
            uint32_t w[2][2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float lo = c[4 * (g + i) + 2 * j] * factor, hi = c[4 * (g + i) + 2 * j + 1] * factor;
                    w[i][j] = S::DT == DETO_BF16 ? pack_bf16(lo, hi) : pack_f16(lo, hi);
                }
            const auto x = __builtin_amdgcn_permlane32_swap(w[0][0], w[1][0], false, false);
            const auto y = __builtin_amdgcn_permlane32_swap(w[0][1], w[1][1], false, false);
            const u32x4 v = {x[0], y[0], x[1], y[1]};
            const int d = b * kSide + 8 * (g + half);
            if (there && d + 8 <= D) *reinterpret_cast<u32x4_any2*>(row + d * 2) = v;
            else if (there) {
#pragma unroll
                for (int j = 0; j < 7; ++j)
                    if (d + j < D) reinterpret_cast<uint16_t*>(row)[d + j] = static_cast<uint16_t>(v[j / 2] >> (16 * (j % 2)));
            }
        }
    }
}
template <class S>
__device__ __forceinline__ void store_columns(const f32x16 (&c)[S::kBlocks], float factor, char* row, bool there, int D) {
#pragma unroll
    for (int b = 0; b < S::kBlocks; ++b) store_block<S>(c[b], b, factor, row, there, D);
}

// the same as fp32 sums, as they are
template <class S>
__device__ __forceinline__ void store_part(const f32x16 (&c)[S::kBlocks], float* row, bool there, int D) {
    const int half = threadIdx.x / kSide % 2;
#pragma unroll
    for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int d = b * kSide + 8 * g + 4 * half;
            u32x4 v;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = f32_bits(c[b][4 * g + j]);
            if (there && d < D) *reinterpret_cast<u32x4*>(row + d) = v;
        }
}

__device__ __forceinline__ float power2(float x) { return __builtin_amdgcn_exp2f(x); }

// of scores, to powers of two
__device__ __forceinline__ float factor_of(float scale) { return fminf(scale * kLog2E, 3.402823466e38f); }

// What weights are relative to: that of score x is 2^((x - score) * factor - power).  Of scores in reach it is `power` alone:
// the difference to a rounded power is exact in one operation, and the rounding is the same for all weights.  Out of it a
// power would be rounded by more than a weight may be off by, up to all of its range, so there the scores are subtracted
// first.
constexpr float kReach = 1 << 20;
struct Base {
    float score, power;
    __device__ __forceinline__ bool far() const { return score != 0.f; }
    __device__ __forceinline__ float above(float x, float factor) const { return fmaf(x - score, factor, -power); }
    // how far this one is above another one, in powers of two
    __device__ __forceinline__ float over(const Base& other, float factor) const {
        return fmaf(score - other.score, factor, power - other.power);
    }
};
// the one under which this score weighs 2^up (-infinity stays a power: of nothing)
__device__ __forceinline__ Base base_of(float score, float factor, float up) {
    const float power = score * factor;
    const bool far = score > -__builtin_inff() && !(fabsf(power) < kReach);
    return {far ? score : 0.f, (far ? 0.f : power) - up};
}
__device__ __forceinline__ float log_sum(const Base& base, float total, float scale) {
    return total == 0.f ? -__builtin_inff() : fmaf(base.score, scale, (base.power + __builtin_amdgcn_logf(total)) * kLn2);
}

// ---- host side
int check(const deto_attention* cfg, int64_t Tq, int64_t Tk);
int check_matrix(const deto_attention* cfg, const deto_rows* m, int64_t T, int heads, int dtype);
Args args_of(const deto_attention* cfg, int64_t Tq, int64_t Tk, const deto_rows* q, const deto_rows* k, const deto_rows* v);

inline Matrix matrix_of(const deto_rows* m) {
    return {static_cast<char*>(m->data), m->ld * type_size(m->dtype)};
}

// Into how many parts the walks over keys are cut.  Where fewer workgroups than CUs would walk over many keys, a second
// launch that adds up what parts of 64 (fp32: 32) keys leave costs less than the rest of the walk.  (Sequences of equal
// length are assumed; the parts are equal shares of each tile's own walk, whatever its length.)  fp32 steps take longer: it
// is cut from 128 keys on, 16-bit types from 512 on.  Forward, in one part and in several: one query over 2,048 keys of 16
// heads of 128, bf16, 45 us and 12; 8 x 114 queries over 512 keys of 12 heads of 64, fp32, 48 and 42.
inline int splits_of(const deto_attention* cfg, int64_t Tq, int64_t Tk, bool f32) {
    if (!Tq || !Tk) return 1;
    const int64_t queried = cfg->sequences < Tq ? cfg->sequences : Tq;
    const int64_t groups = cfg->heads * ((Tq + 127) / 128 > queried ? (Tq + 127) / 128 : queried);
    const int64_t keys = Tk / (cfg->sequences < Tk ? cfg->sequences : Tk);
    if (groups >= kCUs || keys < (f32 ? 128 : 512)) return 1;
    int64_t n = (f32 ? 4 : 2) * kCUs / groups;
    n = n < keys / (f32 ? 32 : 64) ? n : keys / (f32 ? 32 : 64);
    return static_cast<int>(n < 32 ? n : 32);
}
inline int64_t stats_floats(const deto_attention* cfg, int64_t Tq) {        // of the backward pass, to whole pieces
    return (3 * cfg->heads * Tq + 3) / 4 * 4;
}
inline int64_t part_floats(const deto_attention* cfg, int64_t Tq, int splits) {
    return splits > 1 ? splits * cfg->heads * Tq * (2 * part_row(cfg->head_dim) + 2) : 0;
}

// Tiles of `size` rows of one head, into args; false where a launch cannot number those of all heads.
inline bool plan(Args& a, const int32_t* starts, int64_t T, int size, int heads) {
    int64_t tiles;
    if (starts) {
        tiles = T / size + (a.sequences < T ? a.sequences : T);
        a.per_sequence = 1;
    } else {
        const int64_t each = (T / a.sequences + size - 1) / size;
        tiles = each * a.sequences;
        a.per_sequence = static_cast<uint32_t>(each ? each : 1);
    }
    const bool fits = tiles * heads < (int64_t{1} << 22);          // (2^32 threads are the most of a launch)
    a.tiles = fits ? static_cast<uint32_t>(tiles) : 0;
    return fits;
}

// f(Shape, direct) for a head's features; `words`: every row of the matrices that are walked over starts at a multiple
// of 4 bytes
template <int DT, class F>
inline int by_shape(int head_dim, bool words, F f) {
    const auto by_way = [&](auto shape) {
        return words && head_dim % decltype(shape)::kOf == 0 ? f(shape, Type<1>{}) : f(shape, Type<0>{});
    };
    if (head_dim <= 32) return by_way(Shape<DT, 64, 32>{});
    if (head_dim <= 64) return by_way(Shape<DT, 64, 64>{});
    if (head_dim <= 96) return by_way(Shape<DT, 128, 96>{});
    return by_way(Shape<DT, 128, 128>{});
}
inline bool in_words(const Matrix& m) { return is_aligned(m.data, 4) && m.ld % 4 == 0 && m.ld < (int64_t{1} << 24); }

}  // namespace attention
}  // namespace model
}  // namespace deto
