// dw[n][k] = sum_t dy[t][n] x[t][k] with x in 8 bits: a linear layer's weight gradient on the matrix cores.
//
// Codes times a power of two are exact in bf16, so x enters the bf16 matrix instructions without a rounding.
// dy does too: bf16 as it is, fp16 as the sum of two bf16 numbers, fp32 as the sum of three (each takes the
// leading 8 bits of what is left).  Products are exact, sums fp32.
//
// Both operands have the sum's index t as their slow one, and a matrix instruction wants eight consecutive t of
// one n (or k) in a lane.  The turn happens on the way into LDS: a thread takes four rows of eight columns,
// packs pairs of rows (a byte permute for dy; for x the conversion from fp32 packs any two) and writes four t
// of each column.  LDS holds [column][64 t]; the 16-byte pieces of a column's 128 bytes are rotated by
// (column / 8) ^ column, so that neither the writes (columns eight apart) nor the reads (columns side by side)
// meet in a bank.
//
// Bound by the matrix cores for large products (8,192 x 2,048 x 8,192 bf16: 252 us = 1.09 PFLOP/s, where the library's
// largest bf16 products reach 1.25 and its product of this shape 0.94); few tiles are cut along t, in a workgroup or over
// several with a second launch to join them, always in the same order.
#include "device.hip.h"

namespace deto {
namespace model {
namespace {

constexpr int kBand = 4;                // tiles along n that share their part of x
constexpr int kDepth = 64;              // rows t of a step
constexpr int kRowBytes = kDepth * 2;   // of an LDS column

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// BM, BN: of a workgroup's tile; WM, WN: of a wavefront's part of it; GROUPS of wavefronts that take the tile's rows t
// in turns of their own and add up their sums at the end.
template <int BM_, int BN_, int WM_, int WN_, int GROUPS_ = 1>
struct Tile {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, GROUPS = GROUPS_;
    static constexpr int kGroup = (BM / WM) * (BN / WN) * kLanes, kThreads = kGroup * GROUPS;
    static_assert((kDepth / 4) * (BM / 8) % kGroup == 0 && (kDepth / 4) * (BN / 8) % kGroup == 0, "");
    static constexpr int kUnitsA = (kDepth / 4) * (BM / 8) / kGroup;
    static constexpr int kUnitsB = (kDepth / 4) * (BN / 8) / kGroup;
    static constexpr int step_lds(int terms) { return (BM * terms + BN) * kRowBytes; }
    // two buffers of a step; groups have one each, and their sums in the end
    static constexpr int lds(int terms) {
        const int steps = (GROUPS > 1 ? GROUPS : 2) * step_lds(terms), sums = GROUPS > 1 ? GROUPS * BM * BN * 4 : 0;
        return steps > sums ? steps : sums;
    }
};
using Large = Tile<256, 256, 128, 64>;
using Small = Tile<128, 128, 64, 64>;
using Grouped = Tile<64, 64, 64, 64, 4>;

struct Args {
    int64_t T, N, K;
    deto_rows dy, dw;
    deto_act8 x;
    int accumulate;
    int tiles_k;         // tiles along k
    int splits;
    int64_t span;        // rows t of a split, a multiple of kDepth
    float* parts;        // [split][N][K], if splits > 1
};

__device__ __forceinline__ uint32_t lds_at(int column, int t8) {     // byte offset of rows 8 t8 ... + 7
    return column * kRowBytes + (((t8 ^ (column >> 3) ^ column) & 7) << 4);
}

__device__ __forceinline__ uint32_t low_halves(uint32_t first, uint32_t second) {
    return __builtin_amdgcn_perm(second, first, 0x05040100u);
}
__device__ __forceinline__ uint32_t high_halves(uint32_t first, uint32_t second) {
    return __builtin_amdgcn_perm(second, first, 0x07060302u);
}

template <int DT> constexpr int kTerms = DT == DETO_BF16 ? 1 : DT == DETO_F16 ? 2 : 3;

template <int DT>
__device__ __forceinline__ float element(const Raw8<DT>& r, int j) {
    if constexpr (DT == DETO_F32) return bits_f32(j < 4 ? r.a[j & 3] : r.b[j & 3]);
    else {
        const uint32_t word = r.a[j / 2];
        const f16x2 h = __builtin_bit_cast(f16x2, word);
        return static_cast<float>(j % 2 ? h.y : h.x);
    }
}

// What is left of v above its leading 8 bits.  (An infinity is one term, a NaN stays one.)
__device__ __forceinline__ float rest(float v) {
    const float r = v - bits_f32(f32_bits(v) & 0xFFFF0000u);
    return fabsf(v) == __builtin_inff() ? 0.f : r;
}

template <int DT> struct UnitA { Raw8<DT> row[4]; };
struct UnitB { u32x2 codes[4]; uint32_t exps[4]; };

// ---- Loads of a step, without a branch, which would make each wait for the one before.
// NEAR: through buffers that end where the matrix does: rows past its end read as zeros without a comparison, a lane
// needs one offset, and columns past a row's end read whatever comes next (they add to columns of dw that are not
// written).  A buffer gives whole words at multiples of four bytes: rows have to start at those.
// REACH: rows past the end are the last row and columns past the end the last eight, put right when they are used.
// (4,096 x 2,048 x 2,048 bf16: NEAR 66 us, REACH 91.)
// FAR: the same with 64-bit places, for steps of more than 2^32 bytes, and for rows of fewer than eight columns.
enum Mode { kNear, kReach, kFar };
typedef __amdgpu_buffer_rsrc_t Rsrc;

// (The word that holds the last byte counts whole.  It is aligned: no access leaves the memory's last word.)
__device__ __forceinline__ Rsrc resource(const void* base, int64_t bytes, bool words = true) {
    const int n = bytes > 0x7FFFFFF0 ? 0x7FFFFFF0 : bytes > 0 ? static_cast<int>(bytes) : 0;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, words ? (n + 3) & ~3 : n, 0x00020000);
}

template <int DT, class TL, int MODE>
struct Loader {
    static constexpr bool REACH = MODE == kReach;
    const Args& a;
    int64_t n0, k0, end;
    __device__ __forceinline__ Loader(const Args& args, int64_t n, int64_t k, int64_t e)
        : a(args), n0(n), k0(k), end(e) {}

    // Units of eight columns and four rows: rows 4 (u / units a row) of the step.
    static __device__ __forceinline__ int unit(int i) { return threadIdx.x % TL::kGroup + i * TL::kGroup; }
    // the step's first row, and how many it has
    __device__ __forceinline__ int64_t from(int64_t t) const { return t < end ? t : end - 1; }
    __device__ __forceinline__ int rows(int64_t t) const {
        return end - t >= kDepth ? kDepth : end - t > 0 ? static_cast<int>(end - t) : 0;
    }
    static __device__ __forceinline__ int within(int row, int rows) { return row < rows ? row : rows > 0 ? rows - 1 : 0; }

    __device__ __forceinline__ void load_a(int64_t t, UnitA<DT> (&ua)[TL::kUnitsA]) const {
        if constexpr (MODE == kNear) {
            constexpr int kElem = kSize<DT>;
            const int ld = static_cast<int>(a.dy.ld) * kElem;
            const int64_t at = (t * a.dy.ld + n0) * kElem;
            const Rsrc rsrc = resource(static_cast<const char*>(a.dy.data) + at,
                                       ((end - 1) * a.dy.ld + a.N) * kElem - at);
#pragma unroll
            for (int i = 0; i < TL::kUnitsA; ++i) {
                const int off = unit(i) / (TL::BM / 8) * 4 * ld + unit(i) % (TL::BM / 8) * 8 * kElem;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    ua[i].row[r].a = __builtin_amdgcn_raw_buffer_load_b128(rsrc, off, r * ld, 0);
                    if constexpr (DT == DETO_F32)
                        ua[i].row[r].b = __builtin_amdgcn_raw_buffer_load_b128(rsrc, off + 16, r * ld, 0);
                }
            }
            return;
        }
        const int have = rows(t);
        const char* const base = static_cast<const char*>(a.dy.data) + from(t) * a.dy.ld * kSize<DT>;
#pragma unroll
        for (int i = 0; i < TL::kUnitsA; ++i) {
            const int64_t n = n0 + unit(i) % (TL::BM / 8) * 8;
            const int row = unit(i) / (TL::BM / 8) * 4;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int at = within(row + r, have);
                if constexpr (REACH) {
                    const uint32_t column = static_cast<uint32_t>(n < a.N - 8 ? n : a.N - 8);
                    const uint32_t off = (static_cast<uint32_t>(at) * static_cast<uint32_t>(a.dy.ld) + column) * kSize<DT>;
                    ua[i].row[r] = load8_whole<DT>(base + off);
                } else {
                    ua[i].row[r] = load8<DT>(base, at * a.dy.ld, n, n >= a.N ? 0 : a.N - n < 8 ? static_cast<int>(a.N - n) : 8);
                }
            }
        }
    }

    // Makes what units of rows t ... hold what was asked for.
    __device__ __forceinline__ void settle_a(int64_t t, UnitA<DT> (&ua)[TL::kUnitsA]) const {
        if constexpr (MODE == kNear) return;
        const int have = rows(t);
        if (have == kDepth && (!REACH || n0 + TL::BM <= a.N)) return;
#pragma unroll
        for (int i = 0; i < TL::kUnitsA; ++i) {
            const int64_t by = n0 + unit(i) % (TL::BM / 8) * 8 - (a.N - 8);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (REACH && by > 0 && by < 8) move_down<DT>(ua[i].row[r], static_cast<int>(by));
                if (unit(i) / (TL::BM / 8) * 4 + r >= have) ua[i].row[r] = {};
            }
        }
    }

    __device__ __forceinline__ void load_b(int64_t t, UnitB (&ub)[TL::kUnitsB]) const {
        if constexpr (MODE == kNear) {
            const int ldc = static_cast<int>(a.x.ld_codes), lde = static_cast<int>(a.x.ld_exps);
            const int64_t at_c = t * a.x.ld_codes + k0, at_e = t * a.x.ld_exps + k0 / DETO_ACT8_GROUP;
            const int64_t groups = (a.K + DETO_ACT8_GROUP - 1) / DETO_ACT8_GROUP;
            const Rsrc rc = resource(a.x.codes + at_c, (end - 1) * a.x.ld_codes + a.K - at_c);
            const Rsrc re = resource(a.x.exps + at_e, (end - 1) * a.x.ld_exps + groups - at_e, false);    // bytes
#pragma unroll
            for (int i = 0; i < TL::kUnitsB; ++i) {
                const int t4 = unit(i) / (TL::BN / 8) * 4, c8 = unit(i) % (TL::BN / 8);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    ub[i].codes[r] = __builtin_amdgcn_raw_buffer_load_b64(rc, t4 * ldc + c8 * 8, r * ldc, 0);
                    ub[i].exps[r] = __builtin_amdgcn_raw_buffer_load_b8(re, t4 * lde + c8 / 4, r * lde, 0);
                }
            }
            return;
        }
        const int have = rows(t);
        const int8_t* const codes = a.x.codes + from(t) * a.x.ld_codes;
        const uint8_t* const exps = a.x.exps + from(t) * a.x.ld_exps;
        const int last = static_cast<int>((a.K - 1) / DETO_ACT8_GROUP);
#pragma unroll
        for (int i = 0; i < TL::kUnitsB; ++i) {
            const int64_t k = k0 + unit(i) % (TL::BN / 8) * 8;
            const int row = unit(i) / (TL::BN / 8) * 4;
            const int group = k / DETO_ACT8_GROUP < last ? static_cast<int>(k / DETO_ACT8_GROUP) : last;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int at = within(row + r, have);
                if constexpr (REACH) {
                    const uint32_t column = static_cast<uint32_t>(k < a.K - 8 ? k : a.K - 8);
                    ub[i].codes[r] = *reinterpret_cast<const u32x2_any1*>(
                        codes + (static_cast<uint32_t>(at) * static_cast<uint32_t>(a.x.ld_codes) + column));
                    ub[i].exps[r] = exps[static_cast<uint32_t>(at) * static_cast<uint32_t>(a.x.ld_exps) + static_cast<uint32_t>(group)];
                } else {
                    ub[i].codes[r] = load_codes(codes + at * a.x.ld_codes, k, k >= a.K ? 0 : a.K - k < 8 ? static_cast<int>(a.K - k) : 8);
                    ub[i].exps[r] = exps[at * a.x.ld_exps + group];
                }
            }
        }
    }

    __device__ __forceinline__ void settle_b(int64_t t, UnitB (&ub)[TL::kUnitsB]) const {
        if constexpr (MODE == kNear) return;
        const int have = rows(t);
        if (have == kDepth && (!REACH || k0 + TL::BN <= a.K)) return;
#pragma unroll
        for (int i = 0; i < TL::kUnitsB; ++i) {
            const int64_t by = k0 + unit(i) % (TL::BN / 8) * 8 - (a.K - 8);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (REACH && by > 0 && by < 8)
                    ub[i].codes[r] = __builtin_bit_cast(u32x2, __builtin_bit_cast(uint64_t, ub[i].codes[r]) >> (8 * by));
                if (unit(i) / (TL::BN / 8) * 4 + r >= have) ub[i].exps[r] = 0u;
            }
        }
    }
};

// four rows (quarter tq of the step) of column `column`: 8 bytes
__device__ __forceinline__ void put4(char* lds, int column, int tq, uint32_t first, uint32_t second) {
    const u32x2 v = {first, second};
    *reinterpret_cast<u32x2*>(lds + lds_at(column, tq >> 1) + (tq & 1) * 8) = v;
}

// Quarter Q (two columns) of a unit of dy, in all its terms.
template <int DT, class TL, int Q>
__device__ __forceinline__ void store_a(const UnitA<DT>& u, char* lds, int column, int tq) {
    if constexpr (DT == DETO_BF16) {
        put4(lds, column + 2 * Q, tq, low_halves(u.row[0].a[Q], u.row[1].a[Q]),
             low_halves(u.row[2].a[Q], u.row[3].a[Q]));
        put4(lds, column + 2 * Q + 1, tq, high_halves(u.row[0].a[Q], u.row[1].a[Q]),
             high_halves(u.row[2].a[Q], u.row[3].a[Q]));
    } else {
#pragma unroll
        for (int j = 2 * Q; j < 2 * Q + 2; ++j) {
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = element<DT>(u.row[i], j);
#pragma unroll
            for (int term = 0; term < kTerms<DT>; ++term) {
                put4(lds + term * TL::BM * kRowBytes, column + j, tq,
                     high_halves(f32_bits(v[0]), f32_bits(v[1])), high_halves(f32_bits(v[2]), f32_bits(v[3])));
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = rest(v[i]);
            }
        }
    }
}

// Byte J of a word of codes as fp32.
template <int J>
__device__ __forceinline__ float code_value(uint32_t word) {
    float f;
    if constexpr (J == 0)
        asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_0" : "=v"(f) : "v"(word));
    else if constexpr (J == 1)
        asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1" : "=v"(f) : "v"(word));
    else if constexpr (J == 2)
        asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2" : "=v"(f) : "v"(word));
    else
        asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3" : "=v"(f) : "v"(word));
    return f;
}

// Column J of a unit of x.  (The lower halves of the values are zeros: bf16 holds them.)
template <int J>
__device__ __forceinline__ void store_b(const UnitB& u, const float (&scale)[4], char* lds, int column, int tq) {
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t word = u.codes[i][J / 4];
        v[i] = code_value<J % 4>(word) * scale[i];
    }
    put4(lds, column + J, tq, high_halves(f32_bits(v[0]), f32_bits(v[1])),
         high_halves(f32_bits(v[2]), f32_bits(v[3])));
}

// f(Type<0>) ... f(Type<N - 1>)
template <int N, class F>
__device__ __forceinline__ void each_of(F f) {
    if constexpr (N > 0) {
        each_of<N - 1>(f);
        f(Type<N - 1>{});
    }
}

// a workgroup's tile and split
struct Place {
    int64_t n0, k0, split;
};
template <class TL>
__device__ __forceinline__ Place place_of(const Args& a) {
    // Workgroups go to the chip's eight parts in turn: a part takes a run of tiles, four high, whose operands
    // its own cache then holds for all of them.
    const unsigned all = gridDim.x, part = blockIdx.x % 8, each = all / 8, more_parts = all % 8;
    const unsigned id = part * each + (part < more_parts ? part : more_parts) + blockIdx.x / 8;
    const int tiles = all / a.splits, split = id / tiles;
    const int tile = id % tiles, tiles_n = tiles / a.tiles_k;
    const int band = tile / (kBand * a.tiles_k), within = tile % (kBand * a.tiles_k);
    const int high = tiles_n - band * kBand < kBand ? tiles_n - band * kBand : kBand;
    return {static_cast<int64_t>(band * kBand + within % high) * TL::BM, static_cast<int64_t>(within / high) * TL::BN,
            split};
}

// where a split's sums go: to its part of the workspace, if there are several
__device__ __forceinline__ deto_rows output_of(const Args& a, int64_t split) {
    const deto_rows partial = {a.parts + split * a.N * a.K, a.K, DETO_F32, 0};
    return a.splits > 1 ? partial : a.dw;
}
template <class F>
__device__ __forceinline__ void by_output(const deto_rows& out, F f) {
    if (out.dtype == DETO_F32) f(Type<DETO_F32>{});
    else if (out.dtype == DETO_BF16) f(Type<DETO_BF16>{});
    else f(Type<DETO_F16>{});
}

// The 32 x 32 block at (n, k): lane l holds column l % 32, rows 8 (r / 4) + 4 (l / 32) + r % 4.
template <int OUT>
__device__ __forceinline__ void write_block(const Args& a, const deto_rows& out, bool add, int64_t n, int64_t k,
                                            const f32x16& v) {
    const int lane = threadIdx.x % kLanes;
    n += 4 * (lane / 32);
    k += lane % 32;
    if (k >= a.K) return;
    const int rows_left = a.N - n < 32 ? static_cast<int>(a.N - n) : 32;
    char* const at = static_cast<char*>(out.data) + (n * out.ld + k) * kSize<OUT>;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int down = 8 * (r / 4) + r % 4;
        if (down < rows_left) {
            char* const row = at + down * out.ld * kSize<OUT>;
            float s = v[r];
            if (add) s += load1<OUT>(row, 0);
            store1<OUT>(row, 0, s);
        }
    }
}

// What this wavefront wrote to LDS is there for its reads, and what it read is read: the compiler keeps the order, and
// LDS keeps that of one wavefront.
__device__ __forceinline__ void ordered() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

template <int DT, class TL, int MODE>
__global__ __launch_bounds__(TL::kThreads) void weight_grad_kernel(Args a) {
    extern __shared__ __align__(16) char lds[];
    constexpr int kTermsA = kTerms<DT>;
    constexpr int kBytesA = TL::BM * kRowBytes, kBuffer = (TL::BM * kTermsA + TL::BN) * kRowBytes;
    const Place at = place_of<TL>(a);
    const int64_t n0 = at.n0, k0 = at.k0, split = at.split;
    const int64_t t0 = split * a.span;
    const int64_t end = t0 + a.span < a.T ? t0 + a.span : a.T;
    const int lane = threadIdx.x % kLanes, wave = threadIdx.x / kLanes;
    const int wm = wave / (TL::BN / TL::WN) * TL::WM, wn = wave % (TL::BN / TL::WN) * TL::WN;

    f32x16 acc[TL::WM / 32][TL::WN / 32];
#pragma unroll
    for (int i = 0; i < TL::WM / 32; ++i)
#pragma unroll
        for (int j = 0; j < TL::WN / 32; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

    UnitA<DT> ua[TL::kUnitsA];
    UnitB ub[TL::kUnitsB];
    const Loader<DT, TL, MODE> loader(a, n0, k0, end);
    // (A's and B's units lie alike over their columns where the tile is square)
    auto place = [&](int i, int wide) { return loader.unit(i) % (wide / 8) * 8; };
    auto quarter = [&](int i, int wide) { return loader.unit(i) / (wide / 8); };
    auto put_a = [&](char* at, auto q) {
#pragma unroll
        for (int i = 0; i < TL::kUnitsA; ++i)
            store_a<DT, TL, q.value>(ua[i], at, place(i, TL::BM), quarter(i, TL::BM));
    };
    float scale[TL::kUnitsB][4];
    auto scales = [&] {
#pragma unroll
        for (int i = 0; i < TL::kUnitsB; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) scale[i][r] = act8_scale(ub[i].exps[r]);
    };
    auto put_b = [&](char* at, auto j) {
#pragma unroll
        for (int i = 0; i < TL::kUnitsB; ++i)
            store_b<j.value>(ub[i], scale[i], at + kTermsA * kBytesA, place(i, TL::BN), quarter(i, TL::BN));
    };
    // Where a lane's operands of 16 rows t are, from the first of a wavefront's 32-column blocks.  (A block further
    // flips the third bit of column / 8, which is that of rows 32 further.)
    uint32_t at_a[kDepth / 16], at_b[kDepth / 16];
#pragma unroll
    for (int s = 0; s < kDepth / 16; ++s) {
        at_a[s] = lds_at(wm + lane % 32, 2 * s + lane / 32);
        at_b[s] = lds_at(wn + lane % 32, 2 * s + lane / 32);
    }
    bf16x8 fa[2][kTermsA][TL::WM / 32], fb[2][TL::WN / 32];
    auto fetch = [&](const char* la, auto s) {
        constexpr int S = s.value;
        const char* lb = la + kTermsA * kBytesA;
#pragma unroll
        for (int j = 0; j < TL::WN / 32; ++j)
            fb[S % 2][j] = *reinterpret_cast<const bf16x8*>(lb + at_b[S ^ 2 * (j % 2)] + j * 32 * kRowBytes);
#pragma unroll
        for (int term = 0; term < kTermsA; ++term)
#pragma unroll
            for (int i = 0; i < TL::WM / 32; ++i)
                fa[S % 2][term][i] = *reinterpret_cast<const bf16x8*>(
                    la + term * kBytesA + at_a[S ^ 2 * (i % 2)] + i * 32 * kRowBytes);
    };
    // the products of rows 16 S ... + 15 of the step that use blocks I of n
    auto multiply = [&](auto s, auto block) {
        constexpr int S = s.value, I = block.value;
#pragma unroll
        for (int term = 0; term < kTermsA; ++term)
#pragma unroll
            for (int j = 0; j < TL::WN / 32; ++j)
                acc[I][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[S % 2][term][I], fb[S % 2][j], acc[I][j],
                                                                    0, 0, 0);
    };
    if (t0 < end) {
        loader.load_a(t0, ua);
        loader.load_b(t0, ub);
        loader.settle_a(t0, ua);
        loader.settle_b(t0, ub);
        scales();
        each_of<4>([&](auto q) { put_a(lds, q); });
        each_of<8>([&](auto j) { put_b(lds, j); });
        loader.load_a(t0 + kDepth, ua);
        loader.load_b(t0 + kDepth, ub);
    }
    __syncthreads();
    int buffer = 0;
    // While a step's products run from one buffer, the next step's rows, in registers, turn into the other, and
    // the ones after that are loaded as registers fall free.  (Rows past the end are zeros.)
    constexpr int kBlocks = TL::WM / 32;
    // (The quarters stay apart: scheduled over the whole step, products wait for operands.  4,096 x 2,048 x 2,048: 75 us.)
    auto fence = [] { __builtin_amdgcn_sched_barrier(0); };
    for (int64_t t = t0; t < end; t += kDepth) {
        const char* la = lds + buffer * kBuffer;
        buffer ^= 1;
        char* next = lds + buffer * kBuffer;
        fetch(la, Type<0>{});
        fetch(la, Type<1>{});
        loader.settle_a(t + kDepth, ua);
        each_of<kBlocks>([&](auto i) {
            multiply(Type<0>{}, i);
            each_of<4 / kBlocks>([&](auto q) { put_a(next, Type<i.value * (4 / kBlocks) + q.value>{}); });
        });
        fence();
        loader.load_a(t + 2 * kDepth, ua);
        loader.settle_b(t + kDepth, ub);
        scales();
        fetch(la, Type<2>{});
        each_of<kBlocks>([&](auto i) {
            multiply(Type<1>{}, i);
            each_of<4 / kBlocks>([&](auto q) { put_b(next, Type<i.value * (4 / kBlocks) + q.value>{}); });
        });
        fence();
        fetch(la, Type<3>{});
        each_of<kBlocks>([&](auto i) {
            multiply(Type<2>{}, i);
            each_of<4 / kBlocks>([&](auto q) { put_b(next, Type<4 + i.value * (4 / kBlocks) + q.value>{}); });
        });
        fence();
        loader.load_b(t + 2 * kDepth, ub);
        each_of<kBlocks>([&](auto i) { multiply(Type<3>{}, i); });
        __syncthreads();
    }
    const deto_rows out = output_of(a, split);
    const bool add = a.accumulate && a.splits == 1;
    auto write = [&](auto type) {
#pragma unroll
        for (int i = 0; i < TL::WM / 32; ++i)
#pragma unroll
            for (int j = 0; j < TL::WN / 32; ++j)
                write_block<decltype(type)::value>(a, out, add, n0 + wm + i * 32, k0 + wn + j * 32, acc[i][j]);
    };
    by_output(out, write);
}

// The same for products of few tiles: a wavefront takes a 64 x 64 tile by itself, four of them a quarter of the rows t
// each, and their sums meet in LDS.  (1,021 x 770 x 519 bf16, us: tiles of 128 split in workgroups and joined by a
// second launch 20, this 12.)  Wavefronts share nothing until then: what one writes to LDS only it reads, in order.
template <int DT, class TL, int MODE>
__global__ __launch_bounds__(TL::kThreads) void weight_grad_groups_kernel(Args a) {
    static_assert(TL::kGroup == kLanes && TL::GROUPS == 4 && TL::WM == 64 && TL::WN == 64, "a wavefront is a group");
    extern __shared__ __align__(16) char lds[];
    constexpr int kTermsA = kTerms<DT>, kBytesA = TL::BM * kRowBytes;
    const Place at = place_of<TL>(a);
    const int lane = threadIdx.x % kLanes, wave = threadIdx.x / kLanes;
    const int64_t t0 = at.split * a.span;
    const int64_t end = t0 + a.span < a.T ? t0 + a.span : a.T;
    const int64_t steps = (end - t0 + kDepth - 1) / kDepth, each = (steps + TL::GROUPS - 1) / TL::GROUPS;
    const int64_t first = t0 + wave * each * kDepth;
    const int64_t last = first + each * kDepth < end ? first + each * kDepth : end;
    f32x16 acc[2][2];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i / 2][i % 2][r] = 0.f;
    if (first < last) {
        UnitA<DT> ua[TL::kUnitsA];
        UnitB ub[TL::kUnitsB];
        const Loader<DT, TL, MODE> loader(a, at.n0, at.k0, last);
        char* const mine = lds + wave * TL::step_lds(kTermsA);
        loader.load_a(first, ua);
        loader.load_b(first, ub);
        for (int64_t t = first; t < last; t += kDepth) {
            loader.settle_a(t, ua);
            loader.settle_b(t, ub);
            ordered();                       // the step before is read
            each_of<4>([&](auto q) {
#pragma unroll
                for (int i = 0; i < TL::kUnitsA; ++i)
                    store_a<DT, TL, q.value>(ua[i], mine, loader.unit(i) % 8 * 8, loader.unit(i) / 8);
            });
#pragma unroll
            for (int i = 0; i < TL::kUnitsB; ++i) {
                float scale[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) scale[r] = act8_scale(ub[i].exps[r]);
                each_of<8>([&](auto j) {
                    store_b<j.value>(ub[i], scale, mine + kTermsA * kBytesA, loader.unit(i) % 8 * 8,
                                     loader.unit(i) / 8);
                });
            }
            ordered();
            if (t + kDepth < last) {
                loader.load_a(t + kDepth, ua);
                loader.load_b(t + kDepth, ub);
            }
#pragma unroll
            for (int s = 0; s < kDepth / 16; ++s) {
                const int t8 = 2 * s + lane / 32;
                bf16x8 fa[kTermsA][2], fb[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    fb[i] = *reinterpret_cast<const bf16x8*>(mine + kTermsA * kBytesA + lds_at(i * 32 + lane % 32, t8));
#pragma unroll
                    for (int term = 0; term < kTermsA; ++term)
                        fa[term][i] = *reinterpret_cast<const bf16x8*>(mine + term * kBytesA +
                                                                       lds_at(i * 32 + lane % 32, t8));
                }
#pragma unroll
                for (int term = 0; term < kTermsA; ++term)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        acc[i / 2][i % 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[term][i / 2], fb[i % 2],
                                                                                    acc[i / 2][i % 2], 0, 0, 0);
            }
        }
    }
    __syncthreads();                         // the steps' LDS is free
    float* const sums = reinterpret_cast<float*>(lds);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) sums[((wave * 4 + i) * 16 + r) * kLanes + lane] = acc[i / 2][i % 2][r];
    __syncthreads();
    f32x16 all;                              // a 32 x 32 block of the tile for each wavefront
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        float v[4];
#pragma unroll
        for (int g = 0; g < 4; ++g) v[g] = sums[((g * 4 + wave) * 16 + r) * kLanes + lane];
        all[r] = (v[0] + v[1]) + (v[2] + v[3]);
    }
    const deto_rows out = output_of(a, at.split);
    const bool add = a.accumulate && a.splits == 1;
    by_output(out, [&](auto type) {
        write_block<decltype(type)::value>(a, out, add, at.n0 + wave / 2 * 32, at.k0 + wave % 2 * 32, all);
    });
}

// Adds the splits' sums: a wavefront takes 256 columns of a row, a lane four, the loads of eight splits side by side.
constexpr int kJoinRows = 4;         // rows of a workgroup

template <int OUT>
__global__ __launch_bounds__(kJoinRows* kLanes) void weight_grad_join_kernel(Args a) {
    const int64_t k = (static_cast<int64_t>(blockIdx.x) * kLanes + threadIdx.x % kLanes) * 4;
    const int count = a.K - k >= 4 ? 4 : a.K - k > 0 ? static_cast<int>(a.K - k) : 0;
    if (count == 0) return;
    for (int64_t n = static_cast<int64_t>(blockIdx.y) * kJoinRows + threadIdx.x / kLanes; n < a.N;
         n += static_cast<int64_t>(gridDim.y) * kJoinRows) {
        float s[4] = {0.f, 0.f, 0.f, 0.f};
        const int64_t step = a.N * a.K;
        const float* at = a.parts + n * a.K + k;
        if (count == 4) {
            typedef float f32x4_any4 __attribute__((ext_vector_type(4), aligned(4)));
            for (int i = 0; i < a.splits; i += 8) {
                f32x4_any4 v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (i + j < a.splits) v[j] = *reinterpret_cast<const f32x4_any4*>(at + (i + j) * step);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (i + j < a.splits)
#pragma unroll
                        for (int c = 0; c < 4; ++c) s[c] += v[j][c];
            }
        } else {
            for (int i = 0; i < a.splits; ++i)
#pragma unroll
                for (int c = 0; c < 3; ++c)
                    if (c < count) s[c] += at[i * step + c];
        }
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (c < count) {
                if (a.accumulate) s[c] += load1<OUT>(a.dw.data, n * a.dw.ld + k + c);
                store1<OUT>(a.dw.data, n * a.dw.ld + k + c, s[c]);
            }
    }
}

bool bad_shape(int64_t T, int64_t N, int64_t K) {
    constexpr int64_t kMost = int64_t{1} << 30;
    return T < 0 || T > kMost || N < 1 || N > kMost || K < 1 || K > kMost || N > (int64_t{1} << 40) / K;
}

enum Kind { kLarge, kSmall, kGrouped };

struct Plan {
    int kind;
    int64_t tiles, tiles_k, splits, span;
    double us;
};

// The splits of T that take least time by what was measured (us): a step of 64 rows 0.95 in a workgroup of small tiles
// that has a CU to itself and 1.25 in one of two; 1.4 and 2.0 with two and three terms, which leave room for one; 1.9 in
// one of large tiles; 1.95 (2.7 in one workgroup of two), 2.8 and 4.0 in a wavefront of grouped ones, which share the
// steps between four; 5 to start and to write the tile; 3 for the second launch, which the splits' sums go to and come from at 3.5 TB/s.
Plan plan_with(int64_t T, int64_t N, int64_t K, int kind, int terms) {
    const int64_t b = kind == kLarge ? Large::BM : kind == kSmall ? Small::BM : Grouped::BM;
    Plan best = {};
    const int64_t tiles_k = (K + b - 1) / b, tiles = (N + b - 1) / b * tiles_k;
    const int64_t steps = T ? (T + kDepth - 1) / kDepth : 1;
    for (int64_t splits = 1; splits <= 32 && splits <= steps; ++splits) {
        const int64_t each = (steps + splits - 1) / splits;
        if (splits > 1 && each * (splits - 1) >= steps) continue;      // an empty split
        const int64_t slots = kind == kLarge || terms > 1 ? 256 : 512;
        const double step = kind == kLarge ? 1.9
                            : kind == kGrouped ? (terms == 2 ? 2.8 : terms == 3 ? 4.0 : tiles * splits > 256 ? 2.7 : 1.95)
                            : terms == 2 ? 1.4 : terms == 3 ? 2.0 : tiles * splits > 256 ? 1.25 : 0.95;
        const int64_t turns = kind == kGrouped ? (each + Grouped::GROUPS - 1) / Grouped::GROUPS : each;
        double us = static_cast<double>((tiles * splits + slots - 1) / slots) * (step * static_cast<double>(turns) + 5.0);
        if (splits > 1)
            us += 3.0 + 8.0 * static_cast<double>(splits) * static_cast<double>(N) * static_cast<double>(K) / 3.5e6;
        if (splits == 1 || us < best.us) best = {kind, tiles, tiles_k, splits, each * kDepth, us};
    }
    return best;
}

int mode_of(const Args& a) {
    const int64_t e = type_size(a.dy.dtype), row = a.dy.ld * e, least = int64_t{1} << 24, most = int64_t{1} << 25;
    if (row < least && a.x.ld_codes < least && a.x.ld_exps < least && row % 4 == 0 && a.x.ld_codes % 4 == 0 &&
        is_aligned(a.dy.data, 4) && is_aligned(a.x.codes, 4))
        return kNear;
    return row < most && a.x.ld_codes < most && a.x.ld_exps < most && a.N >= 8 && a.K >= 8 ? kReach : kFar;
}

// One term (bf16 dy) may take large tiles; far rows take small ones.
Plan plan_of(int64_t T, int64_t N, int64_t K, bool far, int terms) {
    Plan best = plan_with(T, N, K, kSmall, terms);
    if (far) return best;
    const Plan grouped = plan_with(T, N, K, kGrouped, terms);
    if (grouped.us < best.us) best = grouped;
    if (terms > 1) return best;
    const Plan large = plan_with(T, N, K, kLarge, 1);
    return large.us < best.us ? large : best;
}

}  // namespace
}  // namespace model
}  // namespace deto

using namespace deto::model;

extern "C" {

int64_t detonation_act8_weight_grad_workspace(int64_t T, int64_t N, int64_t K) {
    if (bad_shape(T, N, K)) return -1;
    int64_t most = 0;
    for (bool far : {true, false})
        for (int terms : {1, 2, 3}) {
            const Plan p = plan_of(T, N, K, far, terms);
            if (p.splits > 1 && p.splits > most) most = p.splits;
        }
    return most * N * K * static_cast<int64_t>(sizeof(float));
}

int detonation_act8_weight_grad(int64_t T, int64_t N, int64_t K, const deto_rows* dy,
                                const deto_act8* x8, const deto_rows* dw, int accumulate,
                                void* workspace, void* stream) {
    if (bad_shape(T, N, K)) return DETO_ERR_BAD_CONFIG;
    if (!here(dw) || (T && (!here(dy) || !here(x8)))) return DETO_ERR_NULL;
    const int rc = first_error(check_rows(dw, N, K), T ? check_rows(dy, T, N) : 0,
                               T ? check_act8(x8, T, K) : 0);
    if (rc) return rc;
    const int dtype = T ? dy->dtype : static_cast<int>(DETO_BF16);
    const deto_rows none = {};
    const deto_act8 none8 = {};
    Args a = {T, N, K, T ? *dy : none, *dw, T ? *x8 : none8, accumulate != 0, 0, 0, 0,
              static_cast<float*>(workspace)};
    if (T <= 1) {           // (a single row's distance to the next one says nothing)
        a.dy.ld = (N + 1) / 2 * 2;
        a.x.ld_codes = (K + 3) / 4 * 4;
        a.x.ld_exps = (K + DETO_ACT8_GROUP - 1) / DETO_ACT8_GROUP;
    }
    const int mode = T > 0 ? mode_of(a) : static_cast<int>(kNear);
    const Plan p = plan_of(T, N, K, mode == kFar, dtype == DETO_BF16 ? 1 : dtype == DETO_F16 ? 2 : 3);
    if (p.splits > 1 && !workspace) return DETO_ERR_NULL;
    if (p.splits > 1 && !is_aligned(workspace, 16)) return DETO_ERR_ALIGN;
    if (p.tiles > 0x7FFFFFFF / p.splits) return DETO_ERR_UNSUPPORTED;
    a.tiles_k = static_cast<int>(p.tiles_k);
    a.splits = static_cast<int>(p.splits);
    a.span = p.span;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const unsigned grid = static_cast<unsigned>(p.tiles * p.splits);
    fresh();
    if (p.kind == kLarge) {
        if (mode == kNear)
            weight_grad_kernel<DETO_BF16, Large, kNear><<<grid, Large::kThreads, Large::lds(1), st>>>(a);
        else
            weight_grad_kernel<DETO_BF16, Large, kReach><<<grid, Large::kThreads, Large::lds(1), st>>>(a);
    } else {
        by_type(dtype, [&](auto dt) {
            constexpr int DT = dt.value, kLds = Small::lds(kTerms<DT>), kLdsGrouped = Grouped::lds(kTerms<DT>);
            if (p.kind == kGrouped) {
                if (mode == kNear)
                    weight_grad_groups_kernel<DT, Grouped, kNear><<<grid, Grouped::kThreads, kLdsGrouped, st>>>(a);
                else
                    weight_grad_groups_kernel<DT, Grouped, kReach><<<grid, Grouped::kThreads, kLdsGrouped, st>>>(a);
            } else if (mode == kNear) {
                weight_grad_kernel<DT, Small, kNear><<<grid, Small::kThreads, kLds, st>>>(a);
            } else if (mode == kReach) {
                weight_grad_kernel<DT, Small, kReach><<<grid, Small::kThreads, kLds, st>>>(a);
            } else {
                weight_grad_kernel<DT, Small, kFar><<<grid, Small::kThreads, kLds, st>>>(a);
            }
            return 0;
        });
    }
    if (p.splits > 1) {
        const int64_t rows = (N + kJoinRows - 1) / kJoinRows;
        const dim3 join(static_cast<unsigned>((K + 4 * kLanes - 1) / (4 * kLanes)),
                        static_cast<unsigned>(rows < 65535 ? rows : 65535));
        by_type(dw->dtype, [&](auto dt) {
            weight_grad_join_kernel<dt.value><<<join, kJoinRows * kLanes, 0, st>>>(a);
            return 0;
        });
    }
    return enqueued();
}

}  // extern "C"
