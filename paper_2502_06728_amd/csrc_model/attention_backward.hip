// Gradients of attention, in two launches: those of queries, a workgroup for each 128 queries of a head that walks over
// the keys they see; then those of keys and values, a workgroup for each 128 or 256 keys that walks over the queries that
// see them, of all heads that share the keys.  The weights are computed again from lse in both: two of seven products,
// but every sum has one owner, who adds in a fixed order.  The first launch leaves dout . out of every query for the
// second.
//
// What bounds them: in 16 bits the wait for a step's own loads in its middle (see kLead of the forward walk), and two
// wavefronts a SIMD, whose matrix products, exponentials and LDS reads only partly share the time; sums of two gradients, or
// operands in two terms, fill the registers.  4 x 2,048 tokens of 16 heads of 128 under the mask, bf16: queries 156 us (880
// TFLOP/s in four products), keys 184 (745 in four); without what makes dout . out exact, queries 120.  64 x 197 tokens of 12
// heads of 64 in fp16: 40 and 48.  fp32, 8 x 114 queries over 512 keys: 35 + 11 (the join) and 44, chains of a few steps each.
#include "attention_device.hip.h"

namespace deto {
namespace model {
namespace attention {
namespace {

// ---- dq: the forward kernel's walk.
//
// `out` is rounded, and dout . out with it, by as much as 2^-9 of |dout| |out| in bf16: more than ds may be where a query
// sees few keys, or one outweighs the others.  What is missing is the sum of a query's ds, since its p are 1 together.  So
// the gradients of keys get the sum back with dout . out; those of queries take it times the sum of p k back in the end
// (MEAN: that sum takes as many registers as dq, and shares its reads of LDS).  TWICE: what ds loses by rounding is
// multiplied too.  Errors of dq in bf16, where rounding dq itself is 1.7e-3:
//                  neither   MEAN     TWICE    both
//   2,048 keys     2.7e-3    2.4e-3   2.2e-3   1.7e-3
//   2 keys         6.1e-3    2.4e-3   6.3e-3   1.7e-3
// 16-bit types take MEAN but for long walks over 128 features, whose registers it does not leave (4 x 2,048 tokens of 16
// heads, MEAN 189 us, TWICE 158, neither 120), fp32 where there are few keys; TWICE where there is time for it
// (8 x 114 queries of 12 heads over 512 keys, fp32: MEAN 46 us, without 36, errors 5.7e-7 both).
// Calls with fewer keys a sequence take MEAN.
template <int DT> constexpr int64_t kFewKeys = DT == DETO_F32 ? 128 : 512;
// In the others, queries of 16-bit types that see up to this many get the sum of ds from a walk in front, so that short
// sequences are no less exact beside long ones.  (Errors of a row of dq in bf16, weights from scores of a standard deviation
// of 1 and 2: of 2 keys 4.1e-3 and 5.8e-3 without, of 32 1.9e-3 and 2.7e-3, of 128 1.7e-3 and 2.3e-3, and 1.7e-3 with it for
// all.  In fp32 dout . out is off by its own roundings as much as by that of out.)
constexpr int kFewSeen = 128;
// rows of all heads, up to which there is time for it in both kernels: a row's error may stand out among few, and the chip
// is not full.  (16,384 rows of keys, 1 x 2,048 tokens of 32 heads over 8: 277 us without, 316 with it)
constexpr int64_t kFewRows = 32 * kCUs;

// A query's lse in powers of two; one that sees nothing gets weights of zero.
__device__ __forceinline__ float stored_lse(float lse) {
    return lse == -__builtin_inff() ? __builtin_inff() : lse * kLog2E;
}

// lse is as it was written, rounded in proportion to its size: above this, in powers of two, by as much as 2^-13 (weights are
// off by 1e-4 then, about what a score of that size is, whose product is rounded as well).  Such a query's largest score and
// its sum are taken again, in a walk of their own, and its base is both of them.
constexpr float kFarLse = 1024.f;

// the sum of the products of two rows, each half of the lanes holding its part of them
template <class S>
__device__ __forceinline__ float rows_dot(const u32x4 (&x)[S::kFrags], const u32x4 (&y)[S::kFrags]) {
    float sum = 0.f;
#pragma unroll
    for (int m = 0; m < S::kFrags; ++m)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if constexpr (S::DT == DETO_F32) {
                sum = fmaf(bits_f32(x[m][w]), bits_f32(y[m][w]), sum);
            } else if constexpr (S::DT == DETO_BF16) {
                sum = fmaf(bits_f32(x[m][w] << 16), bits_f32(y[m][w] << 16), sum);
                sum = fmaf(bits_f32(x[m][w] & 0xFFFF0000u), bits_f32(y[m][w] & 0xFFFF0000u), sum);
            } else {
                const uint32_t wx = x[m][w], wy = y[m][w];
                const f16x2 a = __builtin_bit_cast(f16x2, wx), b = __builtin_bit_cast(f16x2, wy);
                sum = fmaf(static_cast<float>(a.x), static_cast<float>(b.x), sum);
                sum = fmaf(static_cast<float>(a.y), static_cast<float>(b.y), sum);
            }
        }
    return halves_sum(sum);
}

// Steps that are asked for ahead of the one that is computed: three, where the workgroups that share a CU then have room in
// its LDS (two of four wavefronts, or one of eight); a step that goes through registers is the only one.
template <int W, int STEP, bool DIRECT>
constexpr int kAhead = !DIRECT ? 1 : STEP * 4 * (8 / W) <= 144 * 1024 ? 3 : 1;

template <class S, int W, bool MEAN, bool TWICE, bool DIRECT>
__global__ __launch_bounds__(W * kLanes) __attribute__((amdgpu_waves_per_eu(kResident<S>, kResident<S>))) void queries_kernel(Args a) {
    constexpr int BM = W * kSide, BN = kKeys<S, W>, kMatrix = BN * S::kRow, kStep = 2 * kMatrix;
    constexpr int AHEAD = kAhead<W, kStep, DIRECT>;
    extern __shared__ __align__(16) char lds[];          // AHEAD + 1 steps of keys and values
    __shared__ uint32_t odd;                             // infinities or NaNs among keys that not all queries see
    __shared__ uint32_t far[W];                          // queries of a wavefront with a far lse
    Place at;
    if (!place_of(a, a.q_starts, a.Tq, BM, a.heads, a.causal, at)) return;
    const Sequence seq = sequence_of(a, at.s);
    const int D = a.head_dim, lane = threadIdx.x % kLanes, half = lane / kSide, wave = uniform(static_cast<int32_t>(threadIdx.x / kLanes));
    const int i0 = at.tile * BM, w0 = i0 + wave * kSide, i = w0 + lane % kSide, last = seq.Lq - 1;
    const bool there = i <= last;

    const auto seen = [&](int n) {
        if (!a.causal) return seq.Lk;
        const int64_t upto = int64_t{n < last ? n : last} + seq.Lk - last;
        return static_cast<int>(upto < 0 ? 0 : upto);
    };
    const int upto = seen(i0 + BM - 1), wave_upto = w0 > last ? 0 : seen(w0 + kSide - 1);
    const int own = seen(i), all_steps = (upto + BN - 1) / BN, splits = gridDim.y, split = blockIdx.y;
    // of which this workgroup takes one part
    const int from = static_cast<int>(int64_t{all_steps} * split / splits), steps = static_cast<int>(int64_t{all_steps} * (split + 1) / splits);
    const int whole_steps = min(max(seen(i0) / BN, from), steps);

    const int64_t col = int64_t{at.head} * D * S::kElem, kv = int64_t{at.head / a.group} * D * S::kElem;
    const int64_t row = seq.q0 + (there ? i : last);
    const char* const keys = a.k.data + seq.k0 * a.k.ld + kv;
    const char* const values = a.v.data + seq.k0 * a.v.ld + kv;
    const char* const query = a.q.data + row * a.q.ld + col;
    const char* const grad = a.dout.data + row * a.dout.ld + col;

    Rows<S, BN, W, DIRECT> rk(a.k.ld), rv(a.v.ld);
    const auto buffer = [&](int step) { return lds + step % (AHEAD + 1) * kStep; };
    const auto begin = [&](int step) __attribute__((always_inline)) {
        const int have = seq.Lk - step * BN < BN ? seq.Lk - step * BN : BN;
        rk.begin(buffer(step), keys + int64_t{step} * BN * a.k.ld, a.k.ld, have, D);
        rv.begin(buffer(step) + kMatrix, values + int64_t{step} * BN * a.v.ld, a.v.ld, have, D);
    };
    const auto end = [&](int step) __attribute__((always_inline)) {
        rk.end(buffer(step));
        rv.end(buffer(step) + kMatrix);
    };
    // a walk's first steps on their way; the wait for one of its steps, and another one on its way
    const auto start = [&](int first, int to) __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < AHEAD; ++n)
            if (first + n < to) begin(first + n);
        if (first < to) end(first);
    };
    const auto arrive = [&](int step, int to) __attribute__((always_inline)) {
        if constexpr (DIRECT) arrived_but<2 * Rows<S, BN, W, DIRECT>::kCalls>(min(AHEAD - 1, to - 1 - step));
        meet();
        if (step + AHEAD < to) begin(step + AHEAD);
    };
    const auto leave = [&](int step, int to) __attribute__((always_inline)) {
        if (step + AHEAD < to) end(step + AHEAD);
    };
    // (a walk in front of the others, whatever part of the keys this workgroup takes: see below)
    const bool ahead = !MEAN && S::DT != DETO_F32 && seen(i0) <= kFewSeen;
    const int ahead_steps = min(all_steps, kFewSeen / BN), first_from = ahead ? 0 : from, first_to = ahead ? ahead_steps : steps;
    if (threadIdx.x == 0) odd = 0;
    if constexpr (DIRECT) clear<S, W>(lds, (AHEAD + 1) * kStep, D);
    start(first_from, first_to);

    const float factor = factor_of(a.scale);
    const Places places = places_of<S>();
    u32x4 q[S::kFrags], g[S::kFrags];
    load_row<S, DIRECT>(grad, there, D, g);
    load_row<S, DIRECT>(a.out.data + row * a.out.ld + col, there, D, q);
    const float lse = there ? a.lse[at.head * a.Tq + row] : -__builtin_inff();
    float delta = rows_dot<S>(g, q);
    load_row<S, DIRECT>(query, there, D, q);

    Base base = {0.f, stored_lse(lse)};
    const bool own_far = fabsf(base.power) > kFarLse && lse > -__builtin_inff();
    const uint64_t wave_far = __ballot(own_far);
    if (lane == 0) far[wave] = wave_far != 0;
    if (first_from < first_to) arrive(first_from, first_to);
    else meet();
    bool any_far = false;
#pragma unroll
    for (int w = 0; w < W; ++w) any_far |= uniform(static_cast<int32_t>(far[w])) != 0;
    if (any_far) {
        if constexpr (DIRECT) arrived<0>();
        meet();
        float top = -__builtin_inff(), sum = 0.f;
        start(0, all_steps);
        for (int step = 0; step < all_steps; ++step) {
            arrive(step, all_steps);
            if (step * BN < wave_upto) {
                const int left = own - step * BN - half * 4;
#pragma unroll 1
                for (int b = 0; b < BN / kSide; ++b) {
                    f32x16 x = block_product<S>(buffer(step) + b * kSide * S::kRow, places, q);
                    float most = -__builtin_inff();
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        if (b * kSide + (r / 4) * 8 + r % 4 >= left) x[r] = -__builtin_inff();
                        most = fmaxf(most, x[r]);
                    }
                    most = halves_max(most);
                    if (most > top) {
                        sum *= power2((top - most) * factor);
                        top = most;
                    }
#pragma unroll
                    for (int r = 0; r < 16; ++r) sum += top > -__builtin_inff() ? power2((x[r] - top) * factor) : 0.f;
                }
            }
            leave(step, all_steps);
        }
        sum = halves_sum(sum);
        if (own_far) base = {top, __builtin_amdgcn_logf(sum)};
        meet();
        start(first_from, first_to);
        if (first_from < first_to) arrive(first_from, first_to);
    }
    if (ahead) {
        // the sum of ds alone, in front of the walk that needs dout . out exact, of queries that see no other keys
        float rest = 0.f;
        for (int step = 0; step < ahead_steps; ++step) {
            if (step > 0) arrive(step, ahead_steps);
            if (step * BN < wave_upto) {
                const int left = own - step * BN - half * 4;
#pragma unroll 1
                for (int b = 0; b < BN / kSide; ++b) {
                    const char* const rows_k = buffer(step) + b * kSide * S::kRow;
                    const f32x16 x = block_product<S>(rows_k, places, q), dp = block_product<S>(rows_k + kMatrix, places, g);
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        rest += b * kSide + (r / 4) * 8 + r % 4 < left ? power2(base.above(x[r], factor)) * (dp[r] - delta) : 0.f;
                }
            }
            leave(step, ahead_steps);
        }
        rest = halves_sum(rest);
        if (own <= kFewSeen) delta += rest;
        meet();
        start(from, steps);
        if (from < steps) arrive(from, steps);
    }
    if (there && half == 0 && split == 0) {
        float* const stats = a.stats + at.head * a.Tq + row;
        const int64_t plane = a.heads * a.Tq;
        stats[0] = base.power;
        stats[plane] = delta;
        stats[2 * plane] = base.score;
    }
    f32x16 dq[S::kBlocks] = {}, mean[MEAN ? S::kBlocks : 1] = {};
    float rest = 0.f;

    const auto compute = [&](int step, auto masked, auto slow) __attribute__((always_inline)) {
        constexpr bool MASKED = masked.value != 0, SLOW = slow.value != 0;
        const char* const from = buffer(step);
        const int left = own - step * BN - half * 4;
#pragma unroll
        for (int b = 0; b < BN / kSide; ++b) {
            const char* const rows_k = from + b * kSide * S::kRow;
            f32x16 p = block_product<S>(rows_k, places, q), ds = block_product<S>(rows_k + kMatrix, places, g);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const bool shown = b * kSide + (r / 4) * 8 + r % 4 < left;
                p[r] = power2(SLOW ? base.above(p[r], factor) : fmaf(p[r], factor, -base.power));
                if (MASKED) p[r] = shown ? p[r] : 0.f;
                ds[r] = p[r] * (ds[r] - delta);
                if (MASKED) ds[r] = shown ? ds[r] : 0.f;
                rest += ds[r];
            }
            columns_products<S, TWICE, MEAN, SLOW>(rows_k, places, ds, p, dq, mean);
        }
    };

    // (loops of their own: a branch between the forms in one would keep a second set of sums.  The first step is there.)
    int step = from;
    if (!any_far) {
        for (; step < whole_steps; ++step) {
            if (step > from) arrive(step, steps);
            if (step * BN < wave_upto) compute(step, Type<0>{}, Type<0>{});
            leave(step, steps);
        }
        for (; step < steps; ++step) {
            if (step > from) arrive(step, steps);
            find_odd<S, BN, W>(buffer(step), &odd);
            meet();
            if (uniform(static_cast<int32_t>(odd))) break;
            if (step * BN < wave_upto) compute(step, Type<1>{}, Type<0>{});
            leave(step, steps);
        }
    }
    // From the first step on that has infinities or NaNs among the keys, the second product goes without them: its other
    // operand has zeros for what is masked, which they would pass by.  (The scores keep them: one that is -infinity is no
    // weight.)  What they give to the queries that see them is added behind the stores.  The same loop takes far queries.
    const int slow_from = step;
    for (; step < steps; ++step) {
        if (step > slow_from) arrive(step, steps);
        if (any_far) find_odd<S, BN, W>(buffer(step), &odd);
        if (step * BN < wave_upto) compute(step, Type<1>{}, Type<1>{});
        leave(step, steps);
    }
    if (any_far) meet();

    float* const part = a.parts + ((int64_t{split} * a.heads + at.head) * a.Tq + row) * part_row(D);
    rest = halves_sum(rest);
    // (the weight of a query's only key does not change; a NaN stays one)
    const bool alone = own <= 1 && fabsf(rest) < __builtin_inff();
#pragma unroll
    for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            if (MEAN && splits == 1) dq[b][r] -= rest * mean[MEAN ? b : 0][r];
            dq[b][r] = alone ? 0.f : dq[b][r];
            if (MEAN) mean[MEAN ? b : 0][r] = alone ? 0.f : mean[MEAN ? b : 0][r];
        }
    if (splits == 1) {
        store_columns<S>(dq, a.scale, a.dq.data + row * a.dq.ld + col, there, D);
        if (there && half == 0) a.stats[(a.heads + at.head) * a.Tq + row] = delta + rest;
    } else {
        store_part<S>(dq, part, there, D);
        if constexpr (MEAN) store_part<S>(mean, part + splits * a.heads * a.Tq * part_row(D), there, D);
        if (there && half == 0) a.parts[(2 * splits * part_row(D) + split) * a.heads * a.Tq + at.head * a.Tq + row] = rest;
    }
    if (steps > slow_from && odd) {
        stored();
        for (int j = slow_from * BN; j < min(wave_upto, steps * BN); ++j) {
            const char* const key = keys + j * a.k.ld;
            if (!row_is_odd<S>(key, D)) continue;
            const float p = power2(base.above(slow_dot<S>(query, key, D), factor));
            const float ds = p * (slow_dot<S>(grad, values + j * a.v.ld, D) - delta);
            if (!there || j >= own) continue;
            if (splits == 1) add_odd<S>(a.dq.data + row * a.dq.ld + col, key, D, ds * a.scale);
            else add_odd<S, DETO_F32>(part, key, D, ds);
        }
    }
}

// A tile's rows of dq out of what the splits left: a wavefront for each, its lanes two features each.
template <class S, int W, bool MEAN>
__global__ __launch_bounds__(W * kLanes) void join_kernel(Args a, int splits) {
    constexpr int BM = W * kSide;
    Place at;
    if (!place_of(a, a.q_starts, a.Tq, BM, a.heads, a.causal, at)) return;
    const Sequence seq = sequence_of(a, at.s);
    const int i = at.tile * BM + blockIdx.y * W + threadIdx.x / kLanes;
    if (i >= seq.Lq) return;
    const int D = a.head_dim, P = part_row(D), lane = threadIdx.x % kLanes;
    const int64_t rows = a.heads * a.Tq, row = at.head * a.Tq + seq.q0 + i;
    const float* const part = a.parts + row * P + 2 * (2 * lane < D ? lane : 0);
    f32x2 x = {0.f, 0.f}, mean = {0.f, 0.f};
#pragma unroll 8
    for (int s = 0; s < splits; ++s) {
        const f32x2 v = *reinterpret_cast<const f32x2*>(part + s * rows * P);
        x.x += v.x;
        x.y += v.y;
        if constexpr (MEAN) {
            const f32x2 m = *reinterpret_cast<const f32x2*>(part + (splits + s) * rows * P);
            mean.x += m.x;
            mean.y += m.y;
        }
    }
    const float rest = wave_sum(lane < splits ? a.parts[(2 * splits * P + lane) * rows + row] : 0.f);    // (at most 32)
    if constexpr (MEAN) {
        x.x -= rest * mean.x;
        x.y -= rest * mean.y;
    }
    if (lane == 0) a.stats[rows + row] += rest;
    char* const dq = a.dq.data + (seq.q0 + i) * a.dq.ld + int64_t{at.head} * D * S::kElem;
    if (2 * lane < D) store1<S::DT>(dq, 2 * lane, x.x * a.scale);
    if (2 * lane + 1 < D) store1<S::DT>(dq, 2 * lane + 1, x.y * a.scale);
}

// ---- dk, dv
constexpr int kQueries = kSide;       // of a step
// HEADS of the heads that share keys are taken at a time, by wavefronts of their own, which add up their sums in the end:
// so that a few long walks are cut where there are not many workgroups.  Their rows leave room for fewer steps ahead.
template <class S, int HEADS, bool DIRECT>
constexpr int kAheadOfKeys = !DIRECT || S::kRow > 256 || HEADS == 4 ? 1 : HEADS == 2 ? 2 : 3;
// Sums of fp32 take the registers of two wavefronts with 128 features; 16-bit values of 128 features stay in LDS, which
// leaves the registers that two wavefronts need beside keys and sums.
template <class S> constexpr int kResidentKeys = S::kRow > 256 ? 1 : 2;
template <class S> constexpr bool kValuesStay = S::kRow == 256 && S::DT != DETO_F32;

// fp32: after so many steps the sums go to the results, and start again from zero.  Added up in one run, those of 8 heads of
// 2,100 queries were off by 2.4e-6 (sums of a head's products by 1.2e-6).
constexpr int kSumSteps = 32;

template <class S>
__device__ __forceinline__ void add_columns(f32x16 (&c)[S::kBlocks], float factor, char* row, bool there, int D, bool more) {
    if (more) {
        const int half = threadIdx.x / kSide % 2;
        const float* const from = reinterpret_cast<const float*>(row);
#pragma unroll
        for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int d = b * kSide + r / 4 * 8 + 4 * half + r % 4;
                c[b][r] = c[b][r] * factor + (there && d < D ? from[d] : 0.f);
            }
        factor = 1.f;
    }
    store_columns<S>(c, factor, row, there, D);
#pragma unroll
    for (int b = 0; b < S::kBlocks; ++b) c[b] = f32x16{};
}

template <class S, int BLOCKS, int HEADS>
__device__ __forceinline__ void add_heads(char* lds, const f32x16 (&c)[S::kBlocks], int own_block, int own_head, float factor,
                                          char* row, bool there, int D) {
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    constexpr int kSums = S::kBlocks * 16 * kLanes * 4;              // bytes of a wavefront's
    const int lane = threadIdx.x % kLanes;
    f32x4* const own = reinterpret_cast<f32x4*>(lds + (own_head * BLOCKS + own_block) * kSums) + lane;
    __syncthreads();
#pragma unroll
    for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            own[(4 * b + g) * kLanes] = f32x4{c[b][4 * g], c[b][4 * g + 1], c[b][4 * g + 2], c[b][4 * g + 3]};
    __syncthreads();
#pragma unroll
    for (int n = 0; n < (S::kBlocks + HEADS - 1) / HEADS; ++n) {
        const int b = n * HEADS + own_head;
        if (b >= S::kBlocks) continue;
        f32x16 sum = {};
#pragma unroll
        for (int h = 0; h < HEADS; ++h) {
            const f32x4* const from = reinterpret_cast<const f32x4*>(lds + (h * BLOCKS + own_block) * kSums) + 4 * b * kLanes + lane;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 v = from[g * kLanes];
#pragma unroll
                for (int j = 0; j < 4; ++j) sum[4 * g + j] += v[j];
            }
        }
        store_block<S>(sum, b, factor, row, there, D);
    }
}

template <class S, int W, int HEADS, bool TWICE, bool DIRECT>
__global__ __launch_bounds__(W * kLanes) __attribute__((amdgpu_waves_per_eu(kResidentKeys<S>, kResidentKeys<S>))) void keys_kernel(Args a) {
    constexpr int BLOCKS = W / HEADS, BN = BLOCKS * kSide, BQ = kQueries, kMatrix = BQ * S::kRow, kStep = 2 * HEADS * kMatrix;
    constexpr bool STAY = kValuesStay<S>;
    constexpr int AHEAD = kAheadOfKeys<S, HEADS, DIRECT>;
    extern __shared__ __align__(16) char lds[];          // AHEAD + 1 steps of queries and gradients of outputs; values
    __shared__ __align__(16) float stats[AHEAD + 1][HEADS][2 * BQ];      // lse and delta
    __shared__ uint32_t odd;                             // infinities or NaNs among rows that do not see all keys
    __shared__ uint32_t far[W];                          // a far base among those that a wavefront has looked at
    Place at;
    if (!place_of(a, a.k_starts, a.Tk, BN, a.kv_heads, false, at)) return;
    const Sequence seq = sequence_of(a, at.s);
    const int D = a.head_dim, lane = threadIdx.x % kLanes, half = lane / kSide;
    const int wave = uniform(static_cast<int32_t>(threadIdx.x / kLanes)), own_block = wave % BLOCKS, own_head = wave / BLOCKS;
    const int j0 = at.tile * BN, j = j0 + own_block * kSide + lane % kSide;
    const int last = seq.Lk - 1;
    const bool there = j <= last;

    // the first query that sees key n
    const auto seen_from = [&](int n) {
        if (!a.causal) return 0;
        const int64_t from = int64_t{n < last ? n : last} - last - 1 + seq.Lq;
        return static_cast<int>(from < 0 ? 0 : from);
    };
    const int first_step = seen_from(j0) / BQ, steps = (seq.Lq + BQ - 1) / BQ - first_step;    // of a head
    const int all_from = seen_from(j0 + BN - 1);                 // from here on queries see all of these keys
    const int wave_from = j0 + own_block * kSide > last ? seq.Lq + BQ : seen_from(j0 + own_block * kSide), own = seen_from(j);
    const int total = steps * (a.group / HEADS);                 // those of the first heads, then of the next ones

    const int64_t kv = int64_t{at.head} * D * S::kElem, row = seq.k0 + (there ? j : last);
    const char* const key = a.k.data + row * a.k.ld + kv;
    const char* const value = a.v.data + row * a.v.ld + kv;

    Rows<S, BQ, W, DIRECT> rq(a.q.ld), rg(a.dout.ld);
    float stat[HEADS][2 * BQ / kLanes];
    // a step: of which heads, from which query on, and its buffer
    struct Step {
        int head, query, buffer;
    };
    const auto next = [&](Step s) __attribute__((always_inline)) {
        s.query += BQ;
        if (s.query >= seq.Lq) {
            s.query = first_step * BQ;
            s.head += HEADS;
        }
        s.buffer = s.buffer == AHEAD ? 0 : s.buffer + 1;
        return s;
    };
    const auto begin = [&](Step s) __attribute__((always_inline)) {
        char* const to = lds + s.buffer * kStep;
        const int have = seq.Lq - s.query < BQ ? seq.Lq - s.query : BQ;
        const int64_t first = seq.q0 + s.query;
#pragma unroll
        for (int h = 0; h < HEADS; ++h) {
            const int64_t col = int64_t{s.head + h} * D * S::kElem;
            rq.begin(to + 2 * h * kMatrix, a.q.data + first * a.q.ld + col, a.q.ld, have, D);
            rg.begin(to + (2 * h + 1) * kMatrix, a.dout.data + first * a.dout.ld + col, a.dout.ld, have, D);
            // lse and delta, 64 at a time, all wavefronts the same
#pragma unroll
            for (int c = 0; c < 2 * BQ / kLanes; ++c) {
                const int n = c * kLanes + lane, t = n % BQ;
                const float* const from =
                    a.stats + (int64_t{n / BQ} * a.heads + s.head + h) * a.Tq + first + (t < have ? t : have - 1);
                if constexpr (DIRECT)
                    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                                     (__attribute__((address_space(3))) void*)(stats[s.buffer][h] + c * kLanes),
                                                     4, 0, 0);
                else stat[h][c] = *from;
            }
        }
    };
    const auto end = [&](Step s) __attribute__((always_inline)) {
        char* const to = lds + s.buffer * kStep;
        rq.end(to);                                      // (one head at a time)
        rg.end(to + kMatrix);
        if constexpr (!DIRECT) {
#pragma unroll
            for (int c = 0; c < 2 * BQ / kLanes; ++c) stats[s.buffer][0][c * kLanes + lane] = stat[0][c];
        }
    };
    // Is any of the queries far?  The first ones are on their way together.
    constexpr int kLooks = 4, kThreads = W * kLanes;
    const int queries = seq.Lq - first_step * BQ, looks = queries * a.group;
    const auto look = [&](int n) __attribute__((always_inline)) {
        const int h = a.group == 1 ? 0 : n / queries;
        return a.stats[(2 * a.heads + at.head * a.group + h) * a.Tq + seq.q0 + first_step * BQ + n - h * queries];
    };
    float looked[kLooks] = {};
    if (looks > 0) {
#pragma unroll
        for (int n = 0; n < kLooks; ++n) looked[n] = look(min(static_cast<int>(threadIdx.x) + n * kThreads, looks - 1));
    }
    if (threadIdx.x == 0) odd = 0;
    if constexpr (DIRECT) clear<S, W>(lds, (AHEAD + 1) * kStep + (STAY ? BN * S::kRow : 0), D);
    if constexpr (STAY) {
        Rows<S, BN, W, DIRECT> rv(a.v.ld);
        rv.begin(lds + (AHEAD + 1) * kStep, a.v.data + (seq.k0 + j0) * a.v.ld + kv, a.v.ld, last - j0 < BN ? last - j0 + 1 : BN, D);
        rv.end(lds + (AHEAD + 1) * kStep);
    }
    Step now = {at.head * a.group, first_step * BQ, 0}, ahead = now;
#pragma unroll
    for (int n = 0; n < AHEAD; ++n)
        if (n < total) {
            begin(ahead);
            if constexpr (DIRECT) ahead = next(ahead);
        }
    if (total > 0 && !DIRECT) {
        end(ahead);
        ahead = next(ahead);
    }

    u32x4 k[S::kFrags], v[S::kFrags];
    load_row<S, DIRECT>(key, there, D, k);
    if constexpr (!STAY) load_row<S, DIRECT>(value, there, D, v);
    const float factor = factor_of(a.scale);
    f32x16 dk[S::kBlocks] = {}, dv[S::kBlocks] = {};

    const Places places = places_of<S>();
    const char* const own_values = lds + (AHEAD + 1) * kStep + own_block * kSide * S::kRow;
    const auto compute = [&](Step s, auto masked, auto slow) __attribute__((always_inline)) {
        constexpr bool MASKED = masked.value != 0, SLOW = slow.value != 0;
        const float* const scores = a.stats + (2 * a.heads + s.head + own_head) * a.Tq + seq.q0 + s.query;
        const char* const from = lds + s.buffer * kStep + 2 * own_head * kMatrix;
#pragma unroll
        for (int b = 0; b < BQ / kSide; ++b) {
            const int first = s.query + b * kSide + half * 4, upto = seq.Lq - first, own_from = own - first;
            const float* const stat = stats[s.buffer][own_head] + b * kSide + half * 4;
            const char *const rows_q = from + b * kSide * S::kRow, *const rows_g = rows_q + kMatrix;
            f32x16 p = block_product<S>(rows_q, places, k), ds;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int t = (r / 4) * 8 + r % 4;
                if constexpr (SLOW) p[r] -= scores[min(b * kSide + half * 4 + t, seq.Lq - s.query - 1)];
                p[r] = power2(fmaf(p[r], factor, -stat[t]));
                if (MASKED) p[r] = t >= own_from && t < upto ? p[r] : 0.f;
            }
            if constexpr (STAY) ds = block_product<S>(rows_g, places, own_values);
            else ds = block_product<S>(rows_g, places, v);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int t = (r / 4) * 8 + r % 4;
                ds[r] = p[r] * (ds[r] - stat[BQ + t]);
                if (MASKED) ds[r] = t >= own_from && t < upto ? ds[r] : 0.f;
            }
            columns_product<S, TWICE>(rows_g, places, p, dv);
            columns_product<S, TWICE>(rows_q, places, ds, dk);
        }
    };

    // steps of one form, as long as they are (loops of their own: a branch between the two in one would keep a second set
    // of sums; one for all steps where a query is far)
    const auto walk = [&](int& n, int upto, auto masked, auto slow) __attribute__((always_inline)) {
        constexpr bool MASKED = masked.value != 0, SLOW = slow.value != 0;
        while (n < upto) {
            const bool whole = now.query >= all_from && now.query + BQ <= seq.Lq;
            if (!SLOW && whole == MASKED) break;
            if constexpr (DIRECT) arrived_but<HEADS * (2 * Rows<S, BQ, W, DIRECT>::kCalls + 2 * BQ / kLanes)>(min(AHEAD - 1, total - 1 - n));
            meet();
            const bool more = n + AHEAD < total;
            if (more) begin(ahead);
            if (SLOW ? !whole : MASKED) {
                take_out_odd<S, 2 * HEADS * BQ, W>(lds + now.buffer * kStep, &odd);
                meet();
            }
            if (now.query + BQ > wave_from) compute(now, masked, slow);
            if (more) {
                end(ahead);
                ahead = next(ahead);
            }
            now = next(now);
            ++n;
        }
    };
    bool own_far = false;
#pragma unroll
    for (int n = 0; n < kLooks; ++n) own_far |= looked[n] != 0.f;
    for (int n = threadIdx.x + kLooks * kThreads; n < looks; n += kThreads) own_far |= look(n) != 0.f;
    const uint64_t wave_far = __ballot(own_far);
    if (lane == 0) far[wave] = wave_far != 0;
    meet();
    bool any_far = false;
#pragma unroll
    for (int w = 0; w < W; ++w) any_far |= uniform(static_cast<int32_t>(far[w])) != 0;

    char *const to_k = a.dk.data + row * a.dk.ld + kv, *const to_v = a.dv.data + row * a.dv.ld + kv;
    const auto all = [&](int& n, int upto) __attribute__((always_inline)) {
        if (any_far) walk(n, upto, Type<1>{}, Type<1>{});
        while (n < upto) {
            walk(n, upto, Type<0>{}, Type<0>{});
            walk(n, upto, Type<1>{}, Type<0>{});
        }
    };
    int n = 0;
    if constexpr (S::DT == DETO_F32) {
        do {
            const bool more = n > 0;
            all(n, min(total, n + kSumSteps));
            add_columns<S>(dk, a.scale, to_k, there, D, more);
            add_columns<S>(dv, 1.f, to_v, there, D, more);
        } while (n < total);
    } else {
        all(n, total);
    }
    if constexpr (S::DT == DETO_F32) {
        // (they are there)
    } else if constexpr (HEADS == 1) {
        store_columns<S>(dk, a.scale, to_k, there, D);
        store_columns<S>(dv, 1.f, to_v, there, D);
    } else {
        // a wavefront adds up the heads' sums of every HEADS-th block of features, in their order (in LDS, where the copy of
        // the values may still be on its way if no step has waited for it: a sequence may have no queries)
        if constexpr (DIRECT) arrived<0>();
        add_heads<S, BLOCKS, HEADS>(lds, dk, own_block, own_head, a.scale, to_k, there, D);
        add_heads<S, BLOCKS, HEADS>(lds, dv, own_block, own_head, 1.f, to_v, there, D);
    }
    if (total > 0 && odd) {
        if constexpr (HEADS == 1) {
            stored();
        } else {
            __syncthreads();
            if (own_head) return;
        }
        const int tail = seq.Lq / BQ * BQ;                  // steps that were masked: up to all_from, and a short last one
        for (int h = at.head * a.group; h < (at.head + 1) * a.group; ++h)
            for (int t = first_step * BQ; t < seq.Lq; ++t) {
                if (t >= (all_from + BQ - 1) / BQ * BQ && t < tail) t = tail;
                if (t >= seq.Lq) break;
                const int64_t at_t = seq.q0 + t, col = int64_t{h} * D * S::kElem;
                const char *const query = a.q.data + at_t * a.q.ld + col, *const grad = a.dout.data + at_t * a.dout.ld + col;
                const bool odd_q = row_is_odd<S>(query, D), odd_g = row_is_odd<S>(grad, D);
                if (!odd_q && !odd_g) continue;
                const Base base = {a.stats[(2 * a.heads + h) * a.Tq + at_t], a.stats[h * a.Tq + at_t]};
                const float p = power2(base.above(slow_dot<S>(query, key, D), factor));
                const float ds = p * (slow_dot<S>(grad, value, D) - a.stats[(a.heads + h) * a.Tq + at_t]);
                if (t < own || !there) continue;
                add_odd<S>(a.dv.data + row * a.dv.ld + kv, grad, D, p);
                add_odd<S>(a.dk.data + row * a.dk.ld + kv, query, D, ds * a.scale);
            }
    }
}

}  // namespace
}  // namespace attention
}  // namespace model
}  // namespace deto

using namespace deto::model;
using namespace deto::model::attention;

extern "C" {

int detonation_attention_backward(const deto_attention* cfg, int64_t Tq, int64_t Tk, const deto_rows* q,
                                  const deto_rows* k, const deto_rows* v, const deto_rows* out,
                                  const float* lse, const deto_rows* dout, const deto_rows* dq,
                                  const deto_rows* dk, const deto_rows* dv, void* workspace, void* stream) {
    int rc = check(cfg, Tq, Tk);
    if (rc) return rc;
    if (Tq == 0 && Tk == 0) return DETO_OK;
    const deto_rows* const any = Tq ? q : k;
    if (!here(any)) return DETO_ERR_NULL;
    const int H = cfg->heads, K = cfg->kv_heads, dtype = any->dtype;
    rc = first_error(check_matrix(cfg, q, Tq, H, dtype), check_matrix(cfg, k, Tk, K, dtype), check_matrix(cfg, v, Tk, K, dtype),
                     check_matrix(cfg, out, Tq, H, dtype), check_matrix(cfg, dout, Tq, H, dtype),
                     check_matrix(cfg, dq, Tq, H, dtype), check_matrix(cfg, dk, Tk, K, dtype),
                     check_matrix(cfg, dv, Tk, K, dtype));
    if (rc) return rc;
    if (Tq && (!lse || !workspace)) return DETO_ERR_NULL;
    if (!is_aligned(lse, 4) || !is_aligned(workspace, 16)) return DETO_ERR_ALIGN;
    Args a = args_of(cfg, Tq, Tk, q, k, v);
    a.lse = const_cast<float*>(lse);
    a.stats = static_cast<float*>(workspace);
    a.parts = a.stats + stats_floats(cfg, Tq);
    const int splits = splits_of(cfg, Tq, Tk, dtype == DETO_F32);
    if (Tq) {
        a.out = matrix_of(out);
        a.dout = matrix_of(dout);
        a.dq = matrix_of(dq);
    }
    if (Tk) {
        a.dk = matrix_of(dk);
        a.dv = matrix_of(dv);
    }
    const hipStream_t on = static_cast<hipStream_t>(stream);
    int planned = DETO_OK;
    bool launch = false;
    fresh();
    by_type(dtype, [&](auto dt) {
        return by_shape<dt.value>(cfg->head_dim, in_words(a.q) && in_words(a.k) && in_words(a.v) && in_words(a.dout),
                                  [&](auto shape, auto direct) {
            using S = decltype(shape);
            constexpr bool DIRECT = direct.value != 0;
            const auto queries = [&](auto waves, auto mean, auto twice) {
                constexpr int W = waves.value, kStep = 2 * kKeys<S, W> * S::kRow;
                constexpr bool MEAN = mean.value, TWICE = twice.value;
                if (!plan(a, cfg->q_starts, Tq, W * kSide, H)) return DETO_ERR_UNSUPPORTED;
                if (Tq && launch) {
                    const dim3 grid(a.tiles * H, splits);
                    queries_kernel<S, W, MEAN, TWICE, DIRECT><<<grid, W * kLanes, (kAhead<W, kStep, DIRECT> + 1) * kStep, on>>>(a);
                    if (splits > 1) join_kernel<S, W, MEAN><<<dim3(grid.x, kSide), W * kLanes, 0, on>>>(a, splits);
                }
                return DETO_OK;
            };
            const auto keys = [&](auto waves, auto heads, auto twice) {
                constexpr int W = waves.value, HEADS = heads.value, BN = W / HEADS * kSide, kStep = 2 * HEADS * kQueries * S::kRow;
                constexpr int kLds = (kAheadOfKeys<S, HEADS, DIRECT> + 1) * kStep + (kValuesStay<S> ? BN * S::kRow : 0);
                if (!plan(a, cfg->k_starts, Tk, BN, K)) return DETO_ERR_UNSUPPORTED;
                if (Tk && launch) keys_kernel<S, W, HEADS, twice.value, DIRECT><<<a.tiles * K, W * kLanes, kLds, on>>>(a);
                return DETO_OK;
            };
            constexpr bool kWide = S::DP == 128;
            const bool wide = kWide && Tq * H >= int64_t{256} * kCUs && Tq / cfg->sequences >= 2048;
            const auto by_waves = [&](auto mean, auto twice) {
                if constexpr (kWide) {
                    if (wide) return queries(Type<8>{}, mean, twice);
                }
                return queries(Type<4>{}, mean, twice);
            };
            const bool few = Tk / cfg->sequences < kFewKeys<S::DT>, spare = Tq * H <= kFewRows;
            const auto choose = [&]() -> int {
                int rc;
                if constexpr (S::DT == DETO_F32) {
                    rc = few ? queries(Type<4>{}, Type<1>{}, Type<0>{}) : by_waves(Type<0>{}, Type<0>{});
                } else if constexpr (S::DU == 128) {
                    rc = !few ? by_waves(Type<0>{}, Type<1>{}) : spare ? queries(Type<4>{}, Type<1>{}, Type<1>{})
                                                                       : queries(Type<4>{}, Type<1>{}, Type<0>{});
                } else {
                    rc = spare ? queries(Type<4>{}, Type<1>{}, Type<1>{}) : by_waves(Type<1>{}, Type<0>{});
                }
                if (rc) return rc;
                // (groups of four heads of 128, bf16, both passes of gradients, four and two heads at a time: 2 x 2,048 tokens of
                // 32 heads 375 us and 424, 1 x 4,200 706 and 808, 1 x 6,000 1,338 and 1,315, 1 x 8,100 2,198 and 2,045; 12 packed
                // sequences of up to 1,500, one at a time 520 us, two 399, four 445, the keys' kernel alone)
                const auto by_heads = [&](auto twice) {
                    if constexpr (kWide && kResidentKeys<S> == 2) {
                        if constexpr (DIRECT) {
                            if (Tk * K < int64_t{160} * kCUs && a.group % 4 == 0) return keys(Type<8>{}, Type<4>{}, twice);
                            if (Tk * K < int64_t{512} * kCUs && a.group % 2 == 0) return keys(Type<8>{}, Type<2>{}, twice);
                        }
                        if constexpr (!twice.value) {
                            if (Tk * K >= int64_t{256} * kCUs) return keys(Type<8>{}, Type<1>{}, twice);
                        }
                    }
                    return keys(Type<4>{}, Type<1>{}, twice);
                };
                if constexpr (S::DT != DETO_F32) {
                    if (Tk * K <= kFewRows) return by_heads(Type<1>{});
                }
                return by_heads(Type<0>{});
            };
            // (all of it is planned before any of it is launched)
            planned = choose();
            launch = true;
            return planned ? planned : choose();
        });
    });
    return planned ? planned : enqueued();
}

}  // extern "C"
