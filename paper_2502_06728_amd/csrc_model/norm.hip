// x_out = x + scale * gate (.) post(f) and y = pre(x_out): the norm after a block, its gate, the residual
// sum and the norm before the next block in one pass over the rows, y also in 8 bits.
//
// Bound by memory: x and f are read once, x_out, y and the codes written once; a row stays in registers
// between its two norms.  LAYER takes its variance around the row's mean (two sums one after the other), so
// that a large mean costs no digits.
#include "norm_device.hip.h"

namespace deto {
namespace model {
namespace {

struct Args {
    deto_norm_residual cfg;
    int64_t T;
    int D;
    int64_t rows_per_team;
    deto_rows x, f, x_out, y;
    deto_act8 y8;
};

// v <- norm(v) * w + b, of a row of which this lane holds C vectors
template <class TM, int C>
__device__ __forceinline__ void normalise(TM& team, float (&v)[C][8], int kind, float eps,
                                          const void* w, const void* b, int dtype, int D) {
    const float inv_d = 1.f / static_cast<float>(D);
    if (kind == DETO_NORM_LAYER) {
        float s[1] = {0.f};
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) s[0] += v[c][j];
        team.sum(s);
        const float mean = s[0] * inv_d;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int n = TM::count(c, D);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[c][j] = j < n ? v[c][j] - mean : 0.f;
        }
    }
    float q[1] = {0.f};
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) q[0] += v[c][j] * v[c][j];
    team.sum(q);
    const float r = 1.f / sqrtf(q[0] * inv_d + eps);
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int d = TM::feature(c), n = TM::count(c, D);
        float p[8];
        if (w) load8_any(w, dtype, d, n, p);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[c][j] = v[c][j] * r * (w ? p[j] : 1.f);
        if (b) {
            load8_any(b, dtype, d, n, p);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[c][j] += p[j];
        }
    }
}

template <int XT, int FT, int W, int C>
__global__ __launch_bounds__((Team<W, C>::kThreadsWg)) void norm_residual_kernel(Args a) {
    using TM = Team<W, C>;
    __shared__ float lds[TM::kSlots];
    TM team(lds);
    const int D = a.D;
    const int64_t first = TM::index() * a.rows_per_team;
    const int64_t end = first + a.rows_per_team < a.T ? first + a.rows_per_team : a.T;
    const bool branch = a.f.data != nullptr;
    for (int64_t t = first; t < end; ++t) {
        Raw8<XT> rx[C];
        Raw8<FT> rf[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int d = TM::feature(c), n = TM::count(c, D);
            rx[c] = load8<XT>(a.x.data, t * a.x.ld + d, n);
            if (branch) rf[c] = load8<FT>(a.f.data, t * a.f.ld + d, n);
        }
        float v[C][8];
        if (branch) {
#pragma unroll
            for (int c = 0; c < C; ++c) unpack8<FT>(rf[c], v[c]);
            if (a.cfg.post != DETO_NORM_NONE)
                normalise(team, v, a.cfg.post, a.cfg.eps_post, a.cfg.w_post, a.cfg.b_post,
                          a.cfg.param_dtype, D);
            const int64_t gate_row = a.cfg.rows_per_gate ? t / a.cfg.rows_per_gate : 0;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int d = TM::feature(c), n = TM::count(c, D);
                float x[8], g[8];
                unpack8<XT>(rx[c], x);
                if (a.cfg.gate)
                    load8_any(a.cfg.gate, a.cfg.param_dtype, gate_row * a.cfg.ld_gate + d, n, g);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    v[c][j] = j < n ? x[j] + a.cfg.scale * (a.cfg.gate ? g[j] : 1.f) * v[c][j] : 0.f;
            }
        } else {
#pragma unroll
            for (int c = 0; c < C; ++c) unpack8<XT>(rx[c], v[c]);
        }
        if (a.x_out.data) {
#pragma unroll
            for (int c = 0; c < C; ++c)
                store8<XT>(a.x_out.data, t * a.x_out.ld + TM::feature(c), v[c], TM::count(c, D));
        }
        if (a.cfg.pre == DETO_NORM_NONE) continue;
        normalise(team, v, a.cfg.pre, a.cfg.eps_pre, a.cfg.w_pre, a.cfg.b_pre, a.cfg.param_dtype, D);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int d = TM::feature(c), n = TM::count(c, D);
            if (a.y.data) store8<FT>(a.y.data, t * a.y.ld + d, v[c], n);
            if (a.y8.codes) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[c][j] = j < n ? v[c][j] : 0.f;
                act8_put(a.y8, t, d, v[c], n);
            }
        }
    }
}

// Rows a team takes one after the other.
int64_t rows_per_team(int64_t T, int teams_wg) {
    const int64_t teams = int64_t{4096} * teams_wg;
    const int64_t rows = (T + teams - 1) / teams;
    return rows < 1 ? 1 : rows;
}

}  // namespace
}  // namespace model
}  // namespace deto

using namespace deto::model;

extern "C" int detonation_norm_residual(const deto_norm_residual* cfg, int64_t T, int64_t D,
                                        const deto_rows* x, const deto_rows* f,
                                        const deto_rows* x_out, const deto_rows* y,
                                        const deto_act8* y8, void* stream) {
    int rc = check_norm(cfg, T, D);
    if (rc || T == 0) return rc;
    const bool branch = here(f), pre = cfg->pre != DETO_NORM_NONE;
    if (!here(x) || (branch && !here(x_out)) || (pre && !here(y) && !here(y8))) return DETO_ERR_NULL;
    if ((!branch && (cfg->post != DETO_NORM_NONE || cfg->gate || here(x_out))) ||
        (!pre && (here(y) || here(y8))) || (!branch && !pre))
        return DETO_ERR_BAD_CONFIG;
    rc = first_error(check_rows(x, T, D), branch ? check_rows(f, T, D) : 0,
                     branch ? check_rows(x_out, T, D) : 0, here(y) ? check_rows(y, T, D) : 0,
                     here(y8) ? check_act8(y8, T, D) : 0);
    if (rc) return rc;
    // y has f's type; without f it may have any, without both it has x's
    const int ft = branch ? f->dtype : here(y) ? y->dtype : x->dtype;
    if ((branch && x_out->dtype != x->dtype) || (here(y) && y->dtype != ft) ||
        (x->dtype != ft && x->dtype != DETO_F32))
        return DETO_ERR_BAD_CONFIG;
    const deto_rows none = {};
    Args a = {*cfg, T, static_cast<int>(D), 0, *x, branch ? *f : none, branch ? *x_out : none,
              here(y) ? *y : none, here(y8) ? *y8 : deto_act8{}};
    fresh();
    by_width(D, [&](auto w, auto c) {
        using TM = Team<w.value, c.value>;
        a.rows_per_team = rows_per_team(T, TM::kTeamsWg);
        const int64_t teams = (T + a.rows_per_team - 1) / a.rows_per_team;
        const unsigned grid = static_cast<unsigned>((teams + TM::kTeamsWg - 1) / TM::kTeamsWg);
        by_types(x->dtype, ft, [&](auto xt, auto fty) {
            norm_residual_kernel<xt.value, fty.value, w.value, c.value>
                <<<grid, TM::kThreadsWg, 0, static_cast<hipStream_t>(stream)>>>(a);
            return 0;
        });
    });
    return enqueued();
}
