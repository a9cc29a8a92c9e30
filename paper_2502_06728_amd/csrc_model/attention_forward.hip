// softmax(scale q k^T) v and log sum exp, one pass over the keys.
//
// A workgroup takes 128 queries of a head, 32 a wavefront, and walks over the keys they see, 64 (fp32: 32) at a time in
// LDS.  A lane has one query: its running maximum and sum are two registers, and its scores, as they come out of the
// first product, are the second product's operand.
#include "attention_device.hip.h"

namespace deto {
namespace model {
namespace attention {
namespace {

constexpr int kQueries = kWaves * kSide;    // of a workgroup
template <int DT> constexpr int kKeys = DT == DETO_F32 ? 32 : 64;      // of a step

// A query's maximum may lag behind by this much (in powers of two): its weights stay below 2^8, and the sums so far need
// not be scaled down for every new maximum.
constexpr float kLag = 8.f;

template <class S, bool WHOLE>
__global__ __launch_bounds__(kThreads, 2) void forward_kernel(Args a) {
    constexpr int DT = S::DT, BN = kKeys<DT>, kMatrix = BN * S::kRow;
    extern __shared__ __align__(16) char lds[];          // two buffers of keys and values
    __shared__ uint32_t bits[3][2];                      // rows of values that hold infinities
    const uint32_t id = number_in_part();
    const int h = id / a.tiles;
    int64_t s;
    int32_t tile, tiles;
    if (!find_tile(a, a.q_starts, a.Tq, kQueries, id % a.tiles, s, tile, tiles)) return;
    if (a.causal) tile = tiles - 1 - tile;               // long ones first
    const Sequence seq = sequence_of(a, s);
    const int D = a.head_dim, lane = threadIdx.x % kLanes, half = lane / kSide;
    const int i0 = tile * kQueries, w0 = i0 + threadIdx.x / kLanes * kSide, i = w0 + lane % kSide;
    const bool there = i < seq.Lq;

    // keys that query n sees
    const auto seen = [&](int n) {
        if (!a.causal) return seq.Lk;
        const int64_t upto = int64_t{n} + seq.Lk - seq.Lq + 1;
        return static_cast<int>(upto < 0 ? 0 : upto < seq.Lk ? upto : seq.Lk);
    };
    const int last = seq.Lq - 1;
    const int upto = seen(i0 + kQueries - 1 < last ? i0 + kQueries - 1 : last);       // by any of the workgroup's
    const int wave_upto = seen(w0 + kSide - 1 < last ? w0 + kSide - 1 : last);
    const int own = seen(i);
    const int steps = (upto + BN - 1) / BN, whole_steps = seen(i0) / BN;

    const int64_t kv = int64_t{h / a.group} * D * S::kElem;
    const char* const keys = a.k.data + seq.k0 * a.k.ld + kv;
    const char* const values = a.v.data + seq.k0 * a.v.ld + kv;
    u32x4 q[S::kFrags];
    load_row<S, WHOLE>(a.q.data + (seq.q0 + (there ? i : last)) * a.q.ld + int64_t{h} * D * S::kElem, there, D, q);

    const float factor = a.scale * kLog2E;       // of scores, to powers of two
    float m = -__builtin_inff(), base = 0.f, l = 0.f;
    f32x16 o[S::kBlocks] = {};

    if (threadIdx.x < 6) bits[threadIdx.x / 2][threadIdx.x % 2] = 0;
    __syncthreads();
    Stage<S, BN, WHOLE> sk, sv;
    const auto have = [&](int step) { return seq.Lk - step * BN < BN ? seq.Lk - step * BN : BN; };
    const auto load = [&](int step) {
        sk.load(keys + int64_t{step} * BN * a.k.ld, a.k.ld, have(step), D);
        sv.load(values + int64_t{step} * BN * a.v.ld, a.v.ld, have(step), D);
    };
    const auto store = [&](int step) {
        char* const at = lds + step % 2 * 2 * kMatrix;
        sk.template store<false>(at, have(step), nullptr);
        if (step >= whole_steps) sv.template store<true>(at + kMatrix, have(step), bits[step % 3]);
        else sv.template store<false>(at + kMatrix, have(step), nullptr);
    };
    const auto compute = [&](int step, auto masked) {
        constexpr bool MASKED = masked.value != 0;
        const char* const at = lds + step % 2 * 2 * kMatrix;
        f32x16 x[BN / kSide];
#pragma unroll
        for (int b = 0; b < BN / kSide; ++b) x[b] = rows_product<S>(at, b, q);
        const int left = own - step * BN - half * 4;         // of the keys that the query sees
        float top = -__builtin_inff();
#pragma unroll
        for (int b = 0; b < BN / kSide; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                if (MASKED) x[b][r] = b * kSide + (r / 4) * 8 + r % 4 < left ? x[b][r] : -__builtin_inff();
                top = fmaxf(top, x[b][r]);
            }
        top = halves_max(top);
        if (__any((top - m) * factor > kLag)) {
            m = fmaxf(m, top);
            const float before = base;
            base = m > -__builtin_inff() ? m * factor : 0.f;
            const float less = power2(before - base);
            l *= less;
#pragma unroll
            for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[b][r] *= less;
        }
        float sum = 0.f;
#pragma unroll
        for (int b = 0; b < BN / kSide; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                x[b][r] = power2(fmaf(x[b][r], factor, -base));
                sum += x[b][r];
            }
        l += sum;
#pragma unroll
        for (int b = 0; b < BN / kSide; ++b) {
            columns_product<S>(at + kMatrix, b, x[b], o);
            if (MASKED) {
                const uint32_t odd = bits[step % 3][b];
                if (odd)
                    add_infinities<S>(odd, values + (int64_t{step} * BN + b * kSide) * a.v.ld, a.v.ld, D, x[b],
                                      [&](int n) { return step * BN + b * kSide + n < own; }, o);
            }
        }
    };

    if (steps > 0) {
        load(0);
        store(0);
    }
    __syncthreads();
    for (int step = 0; step < steps; ++step) {
        if (threadIdx.x < 2) bits[(step + 2) % 3][threadIdx.x] = 0;
        if (step + 1 < steps) load(step + 1);
        if (step < whole_steps) compute(step, Type<0>{});
        else if (step * BN < wave_upto) compute(step, Type<1>{});
        if (step + 1 < steps) store(step + 1);
        __syncthreads();
    }

    l = halves_sum(l);
    const int64_t row = seq.q0 + i;
    store_columns<S>(o, l == 0.f ? 0.f : 1.f / l, a.out.data + row * a.out.ld + int64_t{h} * D * S::kElem, there, D);
    if (a.lse && there && half == 0)
        a.lse[h * a.Tq + row] = l == 0.f ? -__builtin_inff() : (base + __builtin_amdgcn_logf(l)) * kLn2;
}

}  // namespace

int check(const deto_attention* cfg, int64_t Tq, int64_t Tk) {
    if (!cfg) return DETO_ERR_NULL;
    constexpr int64_t kMost = (int64_t{1} << 31) - 1;
    if (Tq < 0 || Tk < 0 || Tq > kMost || Tk > kMost || cfg->sequences < 1 || cfg->sequences > kMost)
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
    return cfg->heads * Tq * static_cast<int64_t>(sizeof(float));
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
    (void)workspace;
    Args a = args_of(cfg, Tq, Tk, q, k, v);
    a.out = matrix_of(out);
    a.lse = lse;
    if (!plan(a, cfg->q_starts, Tq, kQueries, cfg->heads)) return DETO_ERR_UNSUPPORTED;
    fresh();
    by_type(q->dtype, [&](auto dt) {
        return by_shape<dt.value>(cfg->head_dim, [&](auto shape, auto whole) {
            using S = decltype(shape);
            forward_kernel<S, whole.value != 0><<<a.tiles * cfg->heads, kThreads, 4 * kKeys<S::DT> * S::kRow,
                                                  static_cast<hipStream_t>(stream)>>>(a);
            return 0;
        });
    });
    return enqueued();
}

}  // extern "C"
