// softmax(scale q k^T) v and log sum exp, one pass over the keys.
//
// A workgroup takes 128 or 256 queries of a head, 32 a wavefront, and walks over the keys they see, 32 or 64 at a time in
// LDS.  A lane has one query: its base and sum are two registers, and its scores, as they come out of the first product,
// are the second product's operand.  A step's exponentials and second product share the time with the next step's scores.
//
// What bounds it: long sequences the matrix cores, at the chip's power (16,384 tokens of 16 heads of 128 under the mask,
// bf16: 1,040 us, 1.06 PFLOP/s, as the library's products of 8,192^3); 4 x 2,048 tokens (97 us, 0.71) the wait for loads in
// each step (see kLead) and the tiles' unequal lengths; 64 x 197 tokens of 12 heads of 64 (fp16, 27 us) that wait in walks of
// seven steps, the last one of five keys (all exponentials of the chip are some 4 us); few queries a chain of loads (one query
// over 2,048 keys of 16 heads: 7.6 us + 4.2 to join 16 parts, 45 in one part).  64 queries a wavefront (one wavefront a SIMD)
// took 205 us at 4 x 2,048.
#include "attention_device.hip.h"

namespace deto {
namespace model {
namespace attention {
namespace {

// Weights are powers of two of a score less the query's base.  The base is the largest score of the first keys, and it
// stays until a step's weights, which a lane adds up anyway, pass this: no step needs its scores' maximum, and the sums
// so far are seldom scaled down.  fp16 has numbers up to 65504, and few below 1: there the largest of the first keys weighs
// 2^7, so that all of a weight's bits stay down to 2^-21 of that, which thousands of other keys may add up to.  (At 2^10 scores
// of a standard deviation of 2 pass the limit so often that 64 x 197 tokens of 12 heads of 64 take 32 us in the place of 29.)
template <int DT> constexpr float kUp = DT == DETO_F16 ? 7.f : 0.f;
template <int DT> constexpr float kMost = DT == DETO_F16 ? 61440.f : 8192.f;

template <class S, int W, bool DIRECT>
__global__ __launch_bounds__(W * kLanes) __attribute__((amdgpu_waves_per_eu(kResident<S>, kResident<S>)))
void forward_kernel(Args a) {
    constexpr int BM = W * kSide, BN = kKeys<S, W>, kMatrix = BN * S::kRow, kStep = 2 * kMatrix;
    constexpr int LEAD = kLead<DIRECT>, NB = BN / kSide;
    extern __shared__ __align__(16) char lds[];          // steps of keys and values
    __shared__ uint32_t odd;                             // infinities or NaNs among values that not all queries see
    Place at;
    if (!place_of(a, a.q_starts, a.Tq, BM, a.heads, a.causal, at)) return;
    const Sequence seq = sequence_of(a, at.s);
    const int D = a.head_dim, lane = threadIdx.x % kLanes, half = lane / kSide;
    const int i0 = at.tile * BM, w0 = i0 + uniform(static_cast<int32_t>(threadIdx.x / kLanes)) * kSide, last = seq.Lq - 1;

    // keys that query n sees
    const auto seen = [&](int n) {
        if (!a.causal) return seq.Lk;
        const int64_t upto = int64_t{n < last ? n : last} + seq.Lk - last;
        return static_cast<int>(upto < 0 ? 0 : upto);
    };
    const int upto = seen(i0 + BM - 1), wave_upto = w0 > last ? 0 : seen(w0 + kSide - 1);    // by any of the workgroup's, the wavefront's
    const int all_steps = (upto + BN - 1) / BN, splits = gridDim.y, split = blockIdx.y;
    // of which this workgroup takes one part
    const int from = static_cast<int>(int64_t{all_steps} * split / splits), steps = static_cast<int>(int64_t{all_steps} * (split + 1) / splits);
    const int whole_steps = min(max(seen(i0) / BN, from), steps);

    const int64_t col = int64_t{at.head} * D * S::kElem, kv = int64_t{at.head / a.group} * D * S::kElem;
    const char* const keys = a.k.data + seq.k0 * a.k.ld + kv;
    const char* const values = a.v.data + seq.k0 * a.v.ld + kv;
    const char* const queries = a.q.data + seq.q0 * a.q.ld + col;

    Rows<S, BN, W, DIRECT> rk(a.k.ld), rv(a.v.ld);
    const auto buffer = [&](int step) { return lds + step % kBuffers<DIRECT> * kStep; };
    const auto begin = [&](int step) __attribute__((always_inline)) {
        const int have = seq.Lk - step * BN < BN ? seq.Lk - step * BN : BN;
        rk.begin(buffer(step), keys + int64_t{step} * BN * a.k.ld, a.k.ld, have, D);
        rv.begin(buffer(step) + kMatrix, values + int64_t{step} * BN * a.v.ld, a.v.ld, have, D);
    };
    const auto end = [&](int step) __attribute__((always_inline)) {
        rk.end(buffer(step));
        rv.end(buffer(step) + kMatrix);
    };
    if (threadIdx.x == 0) odd = 0;
    if constexpr (DIRECT) clear<S, W>(lds, kBuffers<DIRECT> * kStep, D);
#pragma unroll
    for (int n = 0; n < LEAD; ++n)
        if (from + n < steps) {
            begin(from + n);
            end(from + n);
        }

    const float factor = factor_of(a.scale);
    const int i = w0 + lane % kSide, own = seen(i);
    u32x4 q[S::kFrags];
    load_row<S, DIRECT>(queries + (i < last ? i : last) * a.q.ld, i <= last, D, q);
    Base base = {0.f, own > 0 ? -__builtin_inff() : 0.f};
    float l = 0.f, most = kMost<S::DT>;
    f32x16 o[S::kBlocks] = {};
    const Places places = places_of<S>();
    f32x16 x[NB];                                        // scores of a step, computed in the one before

    const auto hide = [&](int step) __attribute__((always_inline)) {
        const int left = own - step * BN - half * 4;            // of the keys that the query sees
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) x[b][r] = b * kSide + (r / 4) * 8 + r % 4 < left ? x[b][r] : -__builtin_inff();
    };
    // scores into weights, and their sum
    const auto weigh = [&](Base from) __attribute__((always_inline)) {
        float sum = 0.f;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                x[b][r] = power2(from.above(x[b][r], factor));
                sum += x[b][r];
            }
        return sum;
    };
    // the largest score
    const auto largest = [&]() __attribute__((always_inline)) {
        float top = -__builtin_inff();
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, x[b][r]);
        return halves_max(top);
    };
    // (a far base's weights are always taken the second way)
    const auto set = [&](Base to) __attribute__((always_inline)) {
        base = to;
        most = to.far() ? -1.f : kMost<S::DT>;
    };
    // weights of a step's scores, their products with its values, and the next step's scores (the last step's again
    // behind it: a branch here would keep the three from sharing the time)
    const auto compute = [&](int step, auto masked) __attribute__((always_inline)) {
        constexpr bool MASKED = masked.value != 0;
        f32x16 next[NB];
        if (MASKED) hide(step);
        rows_product<S, NB>(buffer(step + 1 < steps ? step + 1 : step), places, q, next);
        float sum = weigh({0.f, base.power});
        const uint64_t high = __ballot(!(sum <= most));          // (or no base yet)
        if (high) {
            rows_product<S, NB>(buffer(step), places, q, x);
            if (MASKED) hide(step);
            const float top = largest();
            // (a query's two lanes do the same, whatever the others do)
            if ((high | high << kSide | high >> kSide) >> lane & 1 && base.above(top, factor) > kUp<S::DT>) {
                const Base risen = base_of(top, factor, kUp<S::DT>);
                const float less = power2(base.over(risen, factor));
                set(risen);
                l *= less;
#pragma unroll
                for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[b][r] *= less;
            }
            sum = weigh({base.score, base.power > -__builtin_inff() ? base.power : 0.f});
        }
        l += sum;
#pragma unroll
        for (int b = 0; b < NB; ++b) columns_product<S>(buffer(step) + kMatrix + b * kSide * S::kRow, places, x[b], o);
#pragma unroll
        for (int b = 0; b < NB; ++b) x[b] = next[b];
    };

    constexpr int kLoads = 2 * Rows<S, BN, W, DIRECT>::kCalls;
    if (from < steps) {
        if constexpr (DIRECT) arrived_but<kLoads>(min(LEAD - 1, steps - 1 - from));
        meet();
        rows_product<S, NB>(buffer(from), places, q, x);
        const float top = largest();
        if (own > 0 && from < whole_steps) set(base_of(top, factor, kUp<S::DT>));           // (what is masked makes no base too low)
    }
    // (two loops: a branch between the two forms in one would keep a second set of sums)
    const auto walk = [&](int& step, int to, auto masked) __attribute__((always_inline)) {
        for (; step < to; ++step) {
            if constexpr (DIRECT) arrived_but<kLoads>(max(0, min(LEAD - 2, steps - 2 - step)));
            meet();
            if (step + LEAD < steps) begin(step + LEAD);
            if constexpr (masked.value != 0) {
                take_out_odd<S, BN, W>(buffer(step) + kMatrix, &odd);
                meet();
            }
            if (step * BN < wave_upto) compute(step, masked);
            if (step + LEAD < steps) end(step + LEAD);
        }
    };
    int step = from;
    walk(step, whole_steps, Type<0>{});
    walk(step, steps, Type<1>{});

    const float total = halves_sum(l), to_one = total == 0.f ? 0.f : 1.f / total;
    const bool there = i <= last;
    const int64_t row = seq.q0 + (there ? i : last);
    char* const out = a.out.data + row * a.out.ld + col;
    const int64_t rows = a.heads * a.Tq, of_part = split * rows + at.head * a.Tq + row;
    float* const part = a.parts + of_part * part_row(D);
    if (splits == 1) {
        store_columns<S>(o, to_one, out, there, D);
        if (a.lse && there && half == 0)
            a.lse[at.head * a.Tq + row] = log_sum(base, total, a.scale);
    } else {
        store_part<S>(o, part, there, D);
        if (there && half == 0) {
            float* const stats = a.parts + splits * rows * part_row(D) + of_part;
            stats[0] = base.score;
            stats[splits * rows] = base.power;
            stats[2 * splits * rows] = total;
        }
    }
    if (steps > whole_steps && odd) {
        stored();
        for (int j = whole_steps * BN; j < min(wave_upto, steps * BN); ++j) {
            const char* const value = values + j * a.v.ld;
            if (!row_is_odd<S>(value, D)) continue;
            const float weight = power2(base.above(slow_dot<S>(queries + (there ? i : last) * a.q.ld, keys + j * a.k.ld, D), factor));
            if (!there || j >= own) continue;
            if (splits == 1) add_odd<S>(out, value, D, weight * to_one);
            else add_odd<S, DETO_F32>(part, value, D, weight);
        }
    }
}

// Queries out of what the splits left of them: a wavefront for each of a tile, its lanes two features each.
constexpr int kJoinWaves = 4;

template <class S, int BM>
__global__ __launch_bounds__(kJoinWaves * kLanes) void join_kernel(Args a, int splits) {
    Place at;
    if (!place_of(a, a.q_starts, a.Tq, BM, a.heads, a.causal, at)) return;
    const Sequence seq = sequence_of(a, at.s);
    const int i = at.tile * BM + blockIdx.y * kJoinWaves + threadIdx.x / kLanes;
    if (i >= seq.Lq) return;
    const int D = a.head_dim, P = part_row(D), lane = threadIdx.x % kLanes;
    const int64_t rows = a.heads * a.Tq, row = at.head * a.Tq + seq.q0 + i;
    const float* const bases = a.parts + splits * rows * P + row;
    // a lane looks at one split's base and sum (there are at most 32)
    const bool own = lane < splits;
    const Base base = {own ? bases[lane * rows] : 0.f, own ? bases[(splits + lane) * rows] : -__builtin_inff()};
    const float sum = own ? bases[(2 * splits + lane) * rows] : 0.f, factor = factor_of(a.scale);
    // the highest one: by its power, and the far ones that are rounded to the same by their scores
    const float power = base.far() ? base.score * factor + base.power : base.power;
    float top = power;
#pragma unroll
    for (int by = 1; by < kLanes; by *= 2) top = fmaxf(top, __shfl_xor(top, by));
    Base highest = {0.f, top};
    if (!(fabsf(top) < kReach)) {
        float score = power == top && base.far() ? base.score : -__builtin_inff();
#pragma unroll
        for (int by = 1; by < kLanes; by *= 2) score = fmaxf(score, __shfl_xor(score, by));
        if (score > -__builtin_inff()) highest = {score, -kUp<S::DT>};
    }
    const float less = sum == 0.f ? 0.f : power2(base.over(highest, factor));          // (of a part that the query sees nothing of: 0)
    const float total = wave_sum(sum * less);
    const float* const part = a.parts + row * P + 2 * (2 * lane < D ? lane : 0);
    float x = 0.f, y = 0.f;
    constexpr int kOnce = 16;                                           // splits' loads in flight
    for (int first = 0; first < splits; first += kOnce) {
        f32x2 v[kOnce];
#pragma unroll
        for (int n = 0; n < kOnce; ++n) v[n] = *reinterpret_cast<const f32x2*>(part + min(first + n, splits - 1) * rows * P);
#pragma unroll
        for (int n = 0; n < kOnce; ++n) {
            const float w = __shfl(less, first + n);                    // (0 behind the last one)
            x += w == 0.f ? 0.f : v[n].x * w;
            y += w == 0.f ? 0.f : v[n].y * w;
        }
    }
    const float to_one = total == 0.f ? 0.f : 1.f / total;
    char* const out = a.out.data + (seq.q0 + i) * a.out.ld + int64_t{at.head} * D * S::kElem;
    if (2 * lane < D) store1<S::DT>(out, 2 * lane, x * to_one);
    if (2 * lane + 1 < D) store1<S::DT>(out, 2 * lane + 1, y * to_one);
    if (a.lse && lane == 0) a.lse[row] = log_sum(highest, total, a.scale);
}

}  // namespace

int check(const deto_attention* cfg, int64_t Tq, int64_t Tk) {
    if (!cfg) return DETO_ERR_NULL;
    constexpr int64_t kMostRows = (int64_t{1} << 31) - 512, kMostSequences = (int64_t{1} << 31) - 1;    // (a tile more is an int)
    if (Tq < 0 || Tk < 0 || Tq > kMostRows || Tk > kMostRows || cfg->sequences < 1 || cfg->sequences > kMostSequences)
        return DETO_ERR_BAD_CONFIG;
    if (cfg->heads < 1 || cfg->heads > 65536 || cfg->kv_heads < 1 || cfg->heads % cfg->kv_heads || cfg->head_dim < 1)
        return DETO_ERR_BAD_CONFIG;
    if ((cfg->causal != 0 && cfg->causal != 1) || cfg->reserved != 0) return DETO_ERR_BAD_CONFIG;
    if (!(cfg->scale > 0.f && cfg->scale < __builtin_inff())) return DETO_ERR_BAD_CONFIG;
    if ((!cfg->q_starts && Tq % cfg->sequences) || (!cfg->k_starts && Tk % cfg->sequences)) return DETO_ERR_BAD_CONFIG;
    if (!is_aligned(cfg->q_starts, 4) || !is_aligned(cfg->k_starts, 4)) return DETO_ERR_ALIGN;
    return cfg->head_dim > 128 ? DETO_ERR_UNSUPPORTED : DETO_OK;
}

int check_matrix(const deto_attention* cfg, const deto_rows* m, int64_t T, int heads, int dtype) {
    if (T == 0) return DETO_OK;
    if (!here(m)) return DETO_ERR_NULL;
    const int rc = check_rows(m, T, int64_t{heads} * cfg->head_dim);
    return rc ? rc : m->dtype != dtype ? DETO_ERR_BAD_CONFIG : DETO_OK;
}

Args args_of(const deto_attention* cfg, int64_t Tq, int64_t Tk, const deto_rows* q, const deto_rows* k, const deto_rows* v) {
    Args a = {};
    if (Tq) a.q = matrix_of(q);
    if (Tk) {
        a.k = matrix_of(k);
        a.v = matrix_of(v);
    }
    a.q_starts = cfg->q_starts;
    a.k_starts = cfg->k_starts;
    a.Tq = Tq;
    a.Tk = Tk;
    a.sequences = cfg->sequences;
    a.heads = cfg->heads;
    a.kv_heads = cfg->kv_heads;
    a.group = cfg->heads / cfg->kv_heads;
    a.head_dim = cfg->head_dim;
    a.causal = cfg->causal;
    a.scale = cfg->scale;
    return a;
}

}  // namespace attention
}  // namespace model
}  // namespace deto

using namespace deto::model;
using namespace deto::model::attention;

extern "C" {

int64_t detonation_attention_workspace(const deto_attention* cfg, int64_t Tq, int64_t Tk) {
    if (check(cfg, Tq, Tk) != DETO_OK) return -1;
    // (fp32 is cut into at least as many parts as the others)
    return (stats_floats(cfg, Tq) + part_floats(cfg, Tq, splits_of(cfg, Tq, Tk, true))) * static_cast<int64_t>(sizeof(float));
}

int detonation_attention_forward(const deto_attention* cfg, int64_t Tq, int64_t Tk, const deto_rows* q,
                                 const deto_rows* k, const deto_rows* v, const deto_rows* out,
                                 float* lse, void* workspace, void* stream) {
    int rc = check(cfg, Tq, Tk);
    if (rc) return rc;
    if (Tq == 0) return DETO_OK;
    if (!here(q)) return DETO_ERR_NULL;
    rc = first_error(check_matrix(cfg, q, Tq, cfg->heads, q->dtype), check_matrix(cfg, k, Tk, cfg->kv_heads, q->dtype),
                     check_matrix(cfg, v, Tk, cfg->kv_heads, q->dtype), check_matrix(cfg, out, Tq, cfg->heads, q->dtype));
    if (rc) return rc;
    if (!is_aligned(lse, 4)) return DETO_ERR_ALIGN;
    const int splits = splits_of(cfg, Tq, Tk, q->dtype == DETO_F32);
    if (splits > 1 && !workspace) return DETO_ERR_NULL;
    if (!is_aligned(workspace, 16)) return DETO_ERR_ALIGN;
    Args a = args_of(cfg, Tq, Tk, q, k, v);
    a.out = matrix_of(out);
    a.lse = lse;
    a.parts = static_cast<float*>(workspace);
    int planned = DETO_OK;
    // (bf16, 16 heads of 128 under the mask, eight wavefronts and four: 16 x 512 rows 52 us and 48, 8 x 1,024 65 and 64,
    // 5 x 1,536 78 and 80, 4 x 2,048 98 and 100, 2 x 4,096 157 and 171, 1 x 8,192 311 and 345; on half of the chip, 1 x 2,048,
    // 60 and 56.  The gradients of queries meet at the same place: 8 x 1,024 both 196, 2 x 4,096 516 and 529, with those of
    // keys.  64 features, 64 x 197 of 12 heads: 37 and 27)
    const bool wide = Tq * cfg->heads >= int64_t{256} * kCUs && Tq / cfg->sequences >= 2048;
    fresh();
    by_type(q->dtype, [&](auto dt) {
        return by_shape<dt.value>(cfg->head_dim, in_words(a.k) && in_words(a.v), [&](auto shape, auto direct) {
            using S = decltype(shape);
            const auto run = [&](auto waves) {
                constexpr int W = waves.value, BM = W * kSide, kStep = 2 * kKeys<S, W> * S::kRow;
                constexpr bool DIRECT = direct.value != 0;
                if (!plan(a, cfg->q_starts, Tq, BM, cfg->heads)) return planned = DETO_ERR_UNSUPPORTED;
                const hipStream_t on = static_cast<hipStream_t>(stream);
                const dim3 grid(a.tiles * cfg->heads, splits);
                forward_kernel<S, W, DIRECT><<<grid, W * kLanes, kBuffers<DIRECT> * kStep, on>>>(a);
                if (splits > 1) {
                    const unsigned of_tile = (min(int64_t{BM}, Tq) + kJoinWaves - 1) / kJoinWaves;
                    join_kernel<S, BM><<<dim3(grid.x, of_tile), kJoinWaves * kLanes, 0, on>>>(a, splits);
                }
                return planned = DETO_OK;
            };
            if constexpr (S::DP == 128) {
                if (wide) return run(Type<8>{});
            }
            return run(Type<4>{});
        });
    });
    if (planned) return planned;
    return enqueued();
}

}  // extern "C"
