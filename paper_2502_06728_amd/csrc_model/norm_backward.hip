// Gradients of norm, gate and residual: both inputs, the gate, the norms' weights and biases.
//
// With n the normalised row, r its factor, a = dy (.) w, the gradient of a norm's input is
//     r (a - n mean(a n) [- mean(a) under LAYER])
// and those of its weight and bias are the sums over rows of dy (.) n and dy.  A team takes a run of rows, keeps
// the sums of its columns in registers and leaves them in the workspace; a second launch adds the teams'
// sums, always in the same order.  A run lies within one gate row (or holds whole ones, whose gradients the
// team then writes itself).
//
// Memory bounds it: x_out, f, dy, dx_out are read once, dx and df written once.  RMS takes two sums over the row one
// after the other: x^2, dy w x and f^2 together, then what df needs of G.  Measured (16,384 x 2,048, fp32 residual stream
// and bf16): 123 us = 4.9 TB/s and 7 us for the join: six streams, and two wavefronts a SIMD, since the columns' sums, the
// parameters and the next row take 150 registers.
#include "norm_device.hip.h"

namespace deto {
namespace model {
namespace {

enum { kWPre, kBPre, kWPost, kBPost, kGate, kSums };
enum { kWPostRms = 1, kGateRms, kSumsRms };      // where they are without biases

// How rows are dealt to teams: `gates` gate rows of `rows` rows each (one of all rows without
// rows_per_gate); every gate row is cut into `cuts` runs, or a team takes `group` whole ones.
struct Deal {
    int64_t T, rows, gates, cuts, run, group, teams;
};

struct Args {
    deto_norm_residual cfg;
    int D;
    Deal deal;
    deto_rows x, f, dy, dxo, dx, df;
    deto_norm_grads grads;
    bool once;           // dx and df are stored past the caches
    float* parts;        // [team][slot][D]
    int slot[kSums];     // of a sum in `parts`, -1: not wanted, or written by the team itself
    int slots;
};

template <int C>
__device__ __forceinline__ void clear(float (&v)[C][8]) {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[c][j] = 0.f;
}

// LAYER: one of the norms is one, or has a bias, or a bias's gradient is wanted.  (Without, the registers of the
// biases' sums are not held.)
template <int XT, int FT, int W, int C, int L, bool WHOLE, bool LAYER>
__global__ __launch_bounds__((Team<W, C, L, WHOLE>::kThreadsWg)) void norm_backward_kernel(Args a) {
    using TM = Team<W, C, L, WHOLE>;
    __shared__ float lds[TM::kSlots];
    TM team(lds);
    const int D = a.D;
    const float inv_d = 1.f / static_cast<float>(D);
    const Deal& deal = a.deal;
    const int64_t me = TM::index();
    if (me >= deal.teams) return;            // (teams of one wavefront only: no barriers)
    int64_t first, end;
    if (deal.group) {
        first = me * deal.group * deal.rows;
        end = first + deal.group * deal.rows;
    } else {
        const int64_t g = me / deal.cuts;
        first = g * deal.rows + me % deal.cuts * deal.run;
        end = first + deal.run;
        const int64_t last = (g + 1) * deal.rows;
        if (end > last) end = last;
    }
    if (end > deal.T) end = deal.T;
    const bool branch = a.f.data != nullptr, pre = a.cfg.pre != DETO_NORM_NONE,
               post = branch && a.cfg.post != DETO_NORM_NONE, through = a.dxo.data != nullptr;
    const bool pre_layer = LAYER && a.cfg.pre == DETO_NORM_LAYER, post_layer = LAYER && a.cfg.post == DETO_NORM_LAYER;

    Raw8<XT> rx[C], ro[C];
    Raw8<FT> rf[C], ry[C];
    auto load = [&](int64_t t) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (pre) {
                rx[c] = TM::template load<XT>(a.x.data, t * a.x.ld, c, D);
                ry[c] = TM::template load<FT>(a.dy.data, t * a.dy.ld, c, D);
            }
            if (through) ro[c] = TM::template load<XT>(a.dxo.data, t * a.dxo.ld, c, D);
            if (branch) rf[c] = TM::template load<FT>(a.f.data, t * a.f.ld, c, D);
        }
    };
#pragma unroll
    for (int c = 0; c < C; ++c) {
        rx[c] = ro[c] = {};
        rf[c] = ry[c] = {};
    }
    if (!TM::kLean && first < end) load(first);
    float w_pre[C][8], w_post[C][8], b_post[C][8], gate[C][8];
    auto param = [&](float (&v)[C][8], const void* at, int64_t row, float otherwise) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (at) TM::load_any(at, a.cfg.param_dtype, row, c, D, v[c]);
            else
#pragma unroll
                for (int j = 0; j < 8; ++j) v[c][j] = otherwise;
        }
    };
    auto params_of_pre = [&] { param(w_pre, pre ? a.cfg.w_pre : nullptr, 0, 1.f); };
    auto params_of_post = [&] {
        param(w_post, post ? a.cfg.w_post : nullptr, 0, 1.f);
        if constexpr (LAYER) param(b_post, post ? a.cfg.b_post : nullptr, 0, 0.f);
    };
    if constexpr (!TM::kLean) {
        params_of_pre();
        params_of_post();
    }
    float sums[LAYER ? kSums : kSumsRms][C][8];
    constexpr int kAtGate = LAYER ? kGate : kGateRms, kAtPost = LAYER ? kWPost : kWPostRms;
#pragma unroll
    for (int i = 0; i < (LAYER ? kSums : kSumsRms); ++i) clear(sums[i]);
    int64_t gate_row = -1;
    for (int64_t t = first; t < end; ++t) {
        float x[C][8], f[C][8], G[C][8], o[C][8];
        if constexpr (TM::kLean) load(t);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            TM::template unpack<XT>(rx[c], c, D, x[c]);
            TM::template unpack<XT>(ro[c], c, D, o[c]);
            TM::template unpack<FT>(ry[c], c, D, G[c]);
            TM::template unpack<FT>(rf[c], c, D, f[c]);
        }
        if constexpr (TM::kLean) params_of_pre();
        else if (t + 1 < end) load(t + 1);
        if (pre_layer || post_layer) {
            float s[2] = {0.f, 0.f};
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    s[0] += x[c][j];
                    s[1] += f[c][j];
                }
            team.sum(s);
            const float mx = pre_layer ? s[0] * inv_d : 0.f, mf = post_layer ? s[1] * inv_d : 0.f;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int n = TM::count(c, D);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    x[c][j] = j < n ? x[c][j] - mx : 0.f;
                    f[c][j] = j < n ? f[c][j] - mf : 0.f;
                }
            }
        }
        // x and f are centred; a = dy (.) w:  sum x^2, sum a x, sum f^2, sum a
        float s[LAYER ? 4 : 3];
#pragma unroll
        for (int i = 0; i < (LAYER ? 4 : 3); ++i) s[i] = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float dyw = G[c][j] * w_pre[c][j];
                s[0] += x[c][j] * x[c][j];
                s[1] += dyw * x[c][j];
                s[2] += f[c][j] * f[c][j];
                if constexpr (LAYER) s[3] += dyw;
            }
        team.sum(s);
        const float r = pre ? 1.f / sqrtf(s[0] * inv_d + a.cfg.eps_pre) : 0.f;
        const float m0 = r * r * (s[1] * inv_d);
        float m1 = 0.f;
        if constexpr (LAYER) m1 = pre_layer ? s[3] * inv_d : 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                sums[kWPre][c][j] += G[c][j] * (x[c][j] * r);
                if constexpr (LAYER) sums[kBPre][c][j] += G[c][j];
                G[c][j] = r * (G[c][j] * w_pre[c][j] - x[c][j] * m0 - m1) + o[c][j];
            }
            TM::template store<XT>(a.dx.data, t * a.dx.ld, c, D, G[c], a.once);
        }
        if (!branch) continue;
        const int64_t row = a.cfg.rows_per_gate ? t / a.cfg.rows_per_gate : 0;
        if constexpr (TM::kLean) params_of_post();
        if (TM::kLean || row != gate_row) {
            gate_row = row;
            param(gate, a.cfg.gate, row * a.cfg.ld_gate, 1.f);
        }
        const float rf_ = post ? 1.f / sqrtf(s[2] * inv_d + a.cfg.eps_post) : 1.f;
        float q[2] = {0.f, 0.f};
#pragma unroll
        for (int c = 0; c < C; ++c) {
            // (Past the row's end G is -r m1, and absent parameters are ones: it would reach the sums.  Without m1 it is
            // zero where a lane's vectors are whole or empty.)
            const int n = TM::count(c, D);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float v = f[c][j] * rf_;
                float u = v * w_post[c][j];
                if constexpr (LAYER) u += b_post[c][j];
                const float g = (WHOLE && !LAYER) || j < n ? a.cfg.scale * G[c][j] : 0.f;
                sums[kAtGate][c][j] += g * u;
                const float h = g * gate[c][j];
                sums[kAtPost][c][j] += h * v;
                if constexpr (LAYER) sums[kBPost][c][j] += h;
                G[c][j] = h * w_post[c][j];
                q[0] += G[c][j] * f[c][j];
                q[1] += G[c][j];
            }
        }
        if (post) {
            if constexpr (LAYER) team.sum(q);
            else team.sum(reinterpret_cast<float (&)[1]>(q));
            const float n0 = rf_ * rf_ * (q[0] * inv_d), n1 = post_layer ? q[1] * inv_d : 0.f;
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) G[c][j] = rf_ * (G[c][j] - f[c][j] * n0 - n1);
        }
#pragma unroll
        for (int c = 0; c < C; ++c) TM::template store<FT>(a.df.data, t * a.df.ld, c, D, G[c], a.once);
        // a gate row of this team's own ends
        if (deal.group && a.grads.gate && ((t + 1) % deal.rows == 0 || t + 1 == deal.T)) {
#pragma unroll
            for (int c = 0; c < C; ++c)
                TM::template store<DETO_F32>(a.grads.gate, t / deal.rows * D, c, D, sums[kAtGate][c]);
            clear(sums[kAtGate]);
        }
    }
    auto leave = [&](int which, const float (&v)[C][8]) {
        if (a.slot[which] < 0) return;
#pragma unroll
        for (int c = 0; c < C; ++c)
            TM::template store<DETO_F32>(a.parts, (me * a.slots + a.slot[which]) * D, c, D, v[c]);
    };
    leave(kWPre, sums[kWPre]);
    leave(kWPost, sums[kAtPost]);
    leave(kGate, sums[kAtGate]);
    if constexpr (LAYER) {
        leave(kBPre, sums[kBPre]);
        leave(kBPost, sums[kBPost]);
    }
}

// Adds the teams' sums of 16 columns: 64 lanes in turn for each, their loads side by side (24 MB of 1,024 teams'
// sums of 2,048 columns: 75 us with four lanes to a column, whose loads follow each other).  blockIdx.y is the output
// row: the weights' and biases' sums over all teams, then the gate's rows, each over the teams of its own.
constexpr int kJoinColumns = 16, kJoinThreads = 1024, kJoinLanes = kJoinThreads / kJoinColumns;

struct JoinArgs {
    const float* parts;
    int D, slots;
    int64_t teams;
    float* out[kSums];
    int slot[kSums];
    int outs;             // of the first four
    int64_t gate_teams;   // teams of a gate row
};

__global__ __launch_bounds__(kJoinThreads) void norm_join_kernel(JoinArgs a, int64_t y0) {
    __shared__ float lds[kJoinLanes][kJoinColumns + 1];
    const int c = threadIdx.x % kJoinColumns, lane = threadIdx.x / kJoinColumns;
    const int col = blockIdx.x * kJoinColumns + c;
    const int64_t y = y0 + blockIdx.y;
    const bool gate = y >= a.outs;
    const int i = gate ? kGate : static_cast<int>(y);
    const int64_t first = gate ? (y - a.outs) * a.gate_teams : 0;
    const int64_t end = gate ? first + a.gate_teams : a.teams;
    float s = 0.f;
    if (col < a.D) {
        const float* at = a.parts + static_cast<int64_t>(a.slot[i]) * a.D + col;
        const int64_t step = static_cast<int64_t>(a.slots) * a.D;
        int64_t t = first + lane;
        for (; t + 7 * kJoinLanes < end; t += 8 * kJoinLanes) {
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = at[(t + k * kJoinLanes) * step];
#pragma unroll
            for (int k = 0; k < 8; ++k) s += v[k];
        }
        for (; t < end; t += kJoinLanes) s += at[t * step];
    }
    lds[lane][c] = s;
    __syncthreads();
    for (int half = kJoinLanes / 2; half; half >>= 1) {
        if (lane < half) lds[lane][c] += lds[lane + half][c];
        __syncthreads();
    }
    if (lane == 0 && col < a.D) a.out[i][(gate ? (y - a.outs) * a.D : 0) + col] = lds[0][c];
}

// Teams that are wanted: two wavefronts a SIMD (a workgroup of sixteen: four).  What more of them would hide of memory's
// latency, their sums' way to the workspace and back costs again (16,384 x 2,048, fp32 and bf16, us: 1,024 teams 152, 768
// 128, 512 123; 8,192 x 4,096: 384 teams 142, 256 127).
int64_t wanted_teams(int64_t D) {
    int64_t teams = 0;
    by_width(D, [&](auto w, auto, auto l, auto) { teams = w.value >= 16 ? 256 : 2048 * (kLanes / l.value) / w.value; });
    return teams;
}

// A team takes two rows at least (1,379 x 771: one row 28 us, two 21, four 23).
Deal deal_rows(const deto_norm_residual* cfg, int64_t T, int64_t D) {
    int64_t most = wanted_teams(D);
    if (most > T / 2) most = T / 2 > 0 ? T / 2 : 1;
    Deal d = {};
    d.T = T;
    d.rows = cfg->rows_per_gate ? cfg->rows_per_gate : T;
    if (d.rows > T) d.rows = T;
    if (T == 0) {
        d.rows = 1;
        return d;
    }
    d.gates = (T + d.rows - 1) / d.rows;
    if (d.gates > most) {
        d.group = (d.gates + most - 1) / most;
        d.teams = (d.gates + d.group - 1) / d.group;
        return d;
    }
    d.cuts = most / d.gates;
    if (d.cuts > d.rows) d.cuts = d.rows;
    d.run = (d.rows + d.cuts - 1) / d.cuts;
    d.cuts = (d.rows + d.run - 1) / d.run;
    d.teams = d.gates * d.cuts;
    return d;
}

}  // namespace
}  // namespace model
}  // namespace deto

using namespace deto::model;

extern "C" {

int64_t detonation_norm_residual_workspace(const deto_norm_residual* cfg, int64_t T, int64_t D) {
    if (check_norm(cfg, T, D)) return -1;
    return deal_rows(cfg, T, D).teams * kSums * D * static_cast<int64_t>(sizeof(float));
}

int detonation_norm_residual_backward(const deto_norm_residual* cfg, int64_t T, int64_t D,
                                      const deto_rows* x_out, const deto_rows* f,
                                      const deto_rows* dy, const deto_rows* dx_out,
                                      const deto_rows* dx, const deto_rows* df,
                                      const deto_norm_grads* grads, void* workspace, void* stream) {
    int rc = check_norm(cfg, T, D);
    if (rc) return rc;
    const deto_norm_grads no_grads = {};
    const deto_norm_grads g = grads ? *grads : no_grads;
    const bool pre = cfg->pre != DETO_NORM_NONE, post = cfg->post != DETO_NORM_NONE;
    // (without rows there is nothing to tell a missing matrix from an empty one by)
    const bool branch = T ? here(f) : true;
    if (((g.w_pre || g.b_pre) && !pre) || ((g.w_post || g.b_post) && !(branch && post)) ||
        (g.gate && !(branch && cfg->gate)))
        return DETO_ERR_BAD_CONFIG;
    for (const float* p : {g.w_pre, g.b_pre, g.w_post, g.b_post, g.gate})
        if (!is_aligned(p, 4)) return DETO_ERR_ALIGN;
    Args a = {};
    if (T > 0) {
        if (!here(x_out) || !here(dx) || (pre && !here(dy)) || (branch && !here(df)))
            return DETO_ERR_NULL;
        if ((!pre && here(dy)) || (!branch && (post || cfg->gate || here(df))) || (!branch && !pre))
            return DETO_ERR_BAD_CONFIG;
        rc = first_error(check_rows(x_out, T, D), check_rows(dx, T, D), branch ? check_rows(f, T, D) : 0,
                         branch ? check_rows(df, T, D) : 0, pre ? check_rows(dy, T, D) : 0,
                         here(dx_out) ? check_rows(dx_out, T, D) : 0);
        if (rc) return rc;
        const int xt = x_out->dtype, ft = branch ? f->dtype : dy->dtype;
        if (dx->dtype != xt || (here(dx_out) && dx_out->dtype != xt) || (branch && df->dtype != ft) ||
            (pre && dy->dtype != ft) || (xt != ft && xt != DETO_F32))
            return DETO_ERR_BAD_CONFIG;
    }
    a.cfg = *cfg;
    // (16,384 x 2,048, us: all bf16 95, past the caches 79; with an fp32 residual stream, of which a lane's 16 bytes are
    // half of what lies together, 135 and 137)
    a.once = T > 0 && x_out->dtype != DETO_F32 && T * D * 2 >= kCacheBytes / 4;
    a.D = static_cast<int>(D);
    const bool layer = cfg->pre == DETO_NORM_LAYER || cfg->post == DETO_NORM_LAYER || cfg->b_post || g.b_pre ||
                       g.b_post;
    a.deal = deal_rows(cfg, T, D);
    a.grads = g;
    float* const outs[kSums] = {g.w_pre, g.b_pre, g.w_post, g.b_post, g.gate};
    JoinArgs j = {};
    for (int i = 0; i < kSums; ++i) {
        const bool wanted = outs[i] && !(i == kGate && a.deal.group);
        a.slot[i] = wanted ? a.slots++ : -1;
        if (!wanted) continue;
        const int at = i == kGate ? kGate : j.outs++;
        j.out[at] = outs[i];
        j.slot[at] = a.slot[i];
    }
    if (a.slots && a.deal.teams) {
        if (!workspace) return DETO_ERR_NULL;
        if (!is_aligned(workspace, 16)) return DETO_ERR_ALIGN;
    }
    if (T == 0 && a.slots == 0) return DETO_OK;
    a.parts = static_cast<float*>(workspace);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    fresh();
    if (T > 0) {
        const deto_rows none = {};
        a.x = *x_out;
        a.dx = *dx;
        a.f = branch ? *f : none;
        a.df = branch ? *df : none;
        a.dy = pre ? *dy : none;
        a.dxo = here(dx_out) ? *dx_out : none;
        by_width(D, [&](auto w, auto c, auto l, auto whole) {
            using TM = Team<w.value, c.value, l.value, whole.value>;
            const unsigned grid = static_cast<unsigned>((a.deal.teams + TM::kTeamsWg - 1) / TM::kTeamsWg);
            by_types(a.x.dtype, branch ? a.f.dtype : a.dy.dtype, [&](auto xt, auto ft) {
                if (layer)
                    norm_backward_kernel<xt.value, ft.value, w.value, c.value, l.value, whole.value, true>
                        <<<grid, TM::kThreadsWg, 0, st>>>(a);
                else
                    norm_backward_kernel<xt.value, ft.value, w.value, c.value, l.value, whole.value, false>
                        <<<grid, TM::kThreadsWg, 0, st>>>(a);
                return 0;
            });
        });
    }
    if (a.slots) {
        j.parts = a.parts;
        j.D = a.D;
        j.slots = a.slots;
        j.teams = a.deal.teams;
        j.gate_teams = a.deal.cuts;
        // without rows: one gate row without rows_per_gate, none with it
        const int64_t gates = a.slot[kGate] < 0 ? 0 : T ? a.deal.gates : cfg->rows_per_gate ? 0 : 1;
        const int64_t all = j.outs + gates;
        for (int64_t y0 = 0; y0 < all; y0 += 65535) {
            const unsigned rows = static_cast<unsigned>(all - y0 < 65535 ? all - y0 : 65535);
            const unsigned columns = static_cast<unsigned>((D + kJoinColumns - 1) / kJoinColumns);
            norm_join_kernel<<<dim3(columns, rows), kJoinThreads, 0, st>>>(j, y0);
        }
    }
    return enqueued();
}

}  // extern "C"
