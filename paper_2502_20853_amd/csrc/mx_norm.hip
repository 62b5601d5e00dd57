// Forward pass of the gated residual with norms, the launch shapes of both passes, and the end of the backward pass.
#include "mx_norm.hpp"

namespace mxl {

namespace {

__device__ __forceinline__ uint32_t codes4(const F8& f, bool floor_mode, uint32_t& byte)
{
    byte = mxd::scale_byte(mxd::quad_max(mxd::amax_bits8(f)), floor_mode);
    return mxd::rtn_codes8_f32(f.v, byte);
}

// Mean (0 for RMS) and reciprocal deviation of the team's row; columns past the row's end hold zeros.
template <int V, bool TAIL, typename R>
__device__ __forceinline__ float2 statistics(const R (&a)[V], Team& team, const NormArgs& g, const Place& at)
{
    float mean = 0.0f;
    if (g.layer) {
        float s = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const F8 f = widen(a[v]);
#pragma unroll
            for (int t = 0; t < 8; ++t) s += f.v[t];
        }
        team.sum<1>(&s);
        mean = s * g.inv_cols;
    }
    float q = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int n = (int)g.cols - (int)at.col(v);
        // whole vectors lie in the row or behind it, where they are zero and stay it
        const float m = v < V - 1 || n > 0 ? mean : 0.0f;
        const F8 f = widen(a[v]);
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            const float d = !TAIL || v < V - 1 || t < n ? f.v[t] - m : 0.0f;
            q = __builtin_fmaf(d, d, q);
        }
    }
    team.sum<1>(&q);
    // rounded as the formula is written, here and in h: with the hardware's reciprocal root and a fused multiply-add 26 % of an
    // FP32 stream differ in the last bit from that, and of 10 million values 11 fall into another 8-bit code; so 5 %, and 3
    return make_float2(mean, 1.0f / __builtin_sqrtf(q * g.inv_cols + g.eps));
}

// Forward pass.  A team walks over a run of rows and has the next row's loads in flight while it works on one.  With one
// vector a lane the parameters stay in registers, else they are read from LDS (in the widest rows those without room there from cache).  Between the
// loads of a row and its use the number of memory instructions is the same on every way through the loop (what there is
// no array for goes to an empty descriptor), so that the wait for them is not one for all of the stores behind them too.
template <typename XT, typename UT, int V, bool POST, bool GATE, bool EIGHT, RowEnd END>
__global__ __launch_bounds__(NORM_THREADS) void residual_norm_fwd_kernel(const NormArgs g)
{
    extern __shared__ float lds[];                                       // the parameters, where a lane has two or three vectors
    __shared__ TeamScratch scratch;
    constexpr bool TAIL = END != ROW_WHOLE;
    using Params = ParamLds<POST, GATE, true, false>;
    const uint32_t stride = g.layer ? Params::STRIDE : ParamLds<POST, GATE, false, false>::STRIDE;      // the biases come last
    const uint32_t team_in_block = threadIdx.x / g.lanes, lane = threadIdx.x % g.lanes;
    const uint32_t teams = blockDim.x / g.lanes;
    Team team{g.lanes, team_in_block * (g.lanes >> 6), &scratch};
    const uint32_t step = g.lanes * 8u, vectors = g.lanes * V;
    const bool post = POST && (!TAIL || g.post), gated = GATE && (!TAIL || g.gate != nullptr), gate_by_row = GATE && g.gate_by_row;

    // every g.teams-th row, so that the chip works in one window of the matrix at a time; with gate rows a run of rows, so that a
    // team's gate row rarely changes
    const bool runs = GATE && g.row_step == 1;
    const TeamRows own(runs, team_in_block, teams, g.lanes);
    const int64_t k0 = own.k0, k = own.k;
    const int64_t first = runs ? g.rows * k0 / g.teams : k0, begin = k >= g.teams ? first : runs ? g.rows * k / g.teams : k;
    const uint32_t count = k >= g.teams ? 0u : (uint32_t)(runs ? g.rows * (k + 1) / g.teams - begin : (g.rows - k + g.teams - 1) / g.teams);
    Place at{first, (uint32_t)(begin - first), lane * 8u, step, g.cols, g.pitch8, count > 0, back_of<END, V>(g.cols, lane * 8u, step)};
    Raw<XT> xn[V];
    Raw<UT> un[V];
    auto fetch = [&](const Place& at) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            xn[v] = load_vec<END, V, XT>(g.x, g.ldx, at, v);
            un[v] = load_vec<END, V, UT>(g.u, g.ldu, at, v);
        }
    };
    fetch(at);
    F8 held[PARAMS];
    auto each_param = [&](auto&& f) {
        f(P_PRE_WEIGHT);
        if (g.layer) f(P_PRE_BIAS);
        if (POST) f(P_POST_WEIGHT);
        if (POST && g.layer) f(P_POST_BIAS);
        if (GATE && !gate_by_row) f(P_GATE);
    };
    if constexpr (V == 1) {
        each_param([&](NormParam which) { held[which] = norm_param<TAIL>(g, which, at.col0); });
    } else if constexpr (V < 4) {
        each_param([&](NormParam which) {
            for (uint32_t c = threadIdx.x; c < vectors; c += blockDim.x) Params::put(lds, stride, which, c, norm_param<TAIL>(g, which, c * 8));
        });
        __syncthreads();
    } else {
        each_param([&](NormParam which) {
            if (g.plane[which] == ParamPlanes::NO_PLANE) return;
            for (uint32_t c = threadIdx.x; c < vectors; c += blockDim.x)
                ParamPlanes::put(lds, g.plane[which], vectors, c, param_is_bf16(g, which), norm_param<TAIL>(g, which, c * 8));
        });
        __syncthreads();
    }
    // the gate's row of the team's, and the place in its run
    int64_t gate_row = 0, in_run = 0;
    if (gate_by_row) {
        gate_row = at.row() / g.gate_run;
        in_run = at.row() - gate_row * g.gate_run;
    }
    float* own_gate = lds + vectors * stride + team_in_block * vectors * Params::GATE_STRIDE;     // a lane reads what it wrote
    auto gate_of_row = [&](int v) { return param8<TAIL>(g.gate, g.gate_bf16, gate_row * g.ld_gate + at.col(v), at.left(v), 0.0f); };
    auto take_gate = [&]() {
        if constexpr (V == 1) held[P_GATE] = gate_of_row(0);
        else if constexpr (V < 4) {
#pragma unroll
            for (int v = 0; v < V; ++v) Params::put(own_gate + (lane + v * g.lanes) * Params::GATE_STRIDE, gate_of_row(v));
        }
    };
    if (gate_by_row) take_gate();
    auto param = [&](NormParam which, int v) {
        if constexpr (V == 1) return held[which];
        else if constexpr (V < 4) {
            if (which == P_GATE && gate_by_row) return Params::get(own_gate + (lane + v * g.lanes) * Params::GATE_STRIDE);
            return Params::get(lds, stride, which, lane + v * g.lanes);
        } else {
            if (which == P_GATE && gate_by_row) return gate_of_row(v);
            if (g.plane[which] != ParamPlanes::NO_PLANE) return ParamPlanes::get(lds, g.plane[which], vectors, lane + v * g.lanes, param_is_bf16(g, which));
            return norm_param<TAIL>(g, which, at.col(v));
        }
    };

    for (uint32_t i = 0; i < (uint32_t)g.team_rows; ++i) {
        Raw<XT> h[V];
        Raw<UT> u[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            h[v] = xn[v];
            u[v] = un[v];
        }
        settle(u[V - 1], at.back);
        settle(h[V - 1], at.back);
        if (END == ROW_ENDS && g.in_place) {
            // the row's last eight elements may be another wave's to overwrite
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
        }
        forget();
        Place next = at;
        next.first += g.row_step;
        next.live = i + 1 < count;
        fetch(next);
        float2 su = make_float2(0.0f, 0.0f);
        if (post) su = statistics<V, TAIL>(u, team, g, at);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            renew(u[v]);
            renew(h[v]);
            F8 b = widen(u[v]);
            if (EIGHT) store_codes8<V>(g.u8, g.u8_scales, at, v, b);
            if (POST && post) {
                const F8 w = param(P_POST_WEIGHT, v);
#pragma unroll
                for (int t = 0; t < 8; ++t) b.v[t] = (b.v[t] - su.x) * su.y * w.v[t];
                if (g.layer) {
                    const F8 c = param(P_POST_BIAS, v);
#pragma unroll
                    for (int t = 0; t < 8; ++t) b.v[t] += c.v[t];
                }
            }
            if (GATE && gated) {
                const F8 gate = param(P_GATE, v);
#pragma unroll
                for (int t = 0; t < 8; ++t) b.v[t] *= gate.v[t];
            }
            const F8 x = widen(h[v]);
#pragma unroll
            for (int t = 0; t < 8; ++t) b.v[t] = g.rho * x.v[t] + g.sigma * b.v[t];
            narrow(b, h[v]);
            b = widen(h[v]);                                             // the stream as it is stored
            store_vec<END, V, XT>(g.h, g.ldh, at, v, b);
            if (EIGHT) store_codes8<V>(g.h8, g.h8_scales, at, v, b);
            if (V > 1) __builtin_amdgcn_sched_barrier(0);                // one vector at a time: registers are short
        }
        const float2 sh = statistics<V, TAIL>(h, team, g, at);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            renew(h[v]);
            const F8 w = param(P_PRE_WEIGHT, v);
            F8 y = widen(h[v]);
#pragma unroll
            for (int t = 0; t < 8; ++t) y.v[t] = (y.v[t] - sh.x) * sh.y;
            if (g.layer) {
                const F8 c = param(P_PRE_BIAS, v);
#pragma unroll
                for (int t = 0; t < 8; ++t) y.v[t] = __builtin_fmaf(y.v[t], w.v[t], c.v[t]);
            } else {
#pragma unroll
                for (int t = 0; t < 8; ++t) y.v[t] *= w.v[t];
            }
            if (g.y_codes != nullptr) {
                uint32_t byte;
                const uint32_t c = codes4(y, g.floor_mode, byte);
                const uint32_t groups = g.cols >> 5, in = at.in<V>(v, g.cols);
                __builtin_amdgcn_raw_buffer_store_b32(c, descriptor(g.y_codes, at.first * (g.cols >> 1)),
                                                      in ? at.behind * (g.cols >> 1) + (at.col0 >> 1) : OFF_END, v * step >> 1, 0);
                __builtin_amdgcn_raw_buffer_store_b8((uint8_t)byte, descriptor(g.y_scales, at.first * groups),
                                                     in && (lane & 3u) == 0 ? at.behind * groups + (at.col0 >> 5) : OFF_END, v * step >> 5, 0);
            } else {
                store_vec<END, V, UT>(g.y, g.ldy, at, v, y);
            }
            if (V > 1) __builtin_amdgcn_sched_barrier(0);
        }
        if (g.stats != nullptr && at.live && lane == 0) g.stats[at.row()] = make_float4(su.x, su.y, sh.x, sh.y);
        if (gate_by_row && ++in_run == g.gate_run) {
            in_run = 0;
            ++gate_row;
            at.live = next.live;                                         // its lanes in the row are the same
            take_gate();
        }
        at = next;
    }
}

struct NormFinishArgs {
    const float* partials;
    const float* gate_partials;
    void* out[SUMS];
    uint32_t parts, gate_parts, gate_rows, cols;
    uint32_t none;             // bit s: the call has no part of sum s, which is zero
    bool param_bf16, gate_bf16;
};

// Adds the workgroups' sums up: 32 columns a workgroup, its 32 parts of 32 lanes each take a run of the partial rows in
// order (8 of 256, loaded at once), and the runs are added in order.  Eight parts with runs of 32 to 64: 5 to 6.4 us, this: 4 to 4.8.
// Gate rows of no more than 32 parts: a row to each run.  Backward pass of 16384 x 1024 with 1024 gate rows of two parts: 44.7 us
// so, 111.6 with a workgroup for each; 256 rows of eight: 43.5 and 58.8.
constexpr uint32_t FINISH_RUNS = 32;
__host__ __device__ constexpr bool gate_row_a_run(uint32_t gate_rows, uint32_t gate_parts) { return gate_rows > 1 && gate_parts <= 32; }
__global__ __launch_bounds__(32 * FINISH_RUNS) void residual_norm_finish_kernel(const NormFinishArgs a)
{
    __shared__ float part[FINISH_RUNS][33];
    const uint32_t lc = threadIdx.x & 31u, p = threadIdx.x >> 5, blocks = (a.cols + 31u) / 32u;
    // the sums in order: first the four parameters (those wanted), then the gate's rows
    const uint32_t y = blockIdx.x / blocks, c = blockIdx.x % blocks * 32u + lc;
    const bool is_gate = y >= SUMS - 1;
    const uint32_t s = is_gate ? GATE_SUM : y >= GATE_SUM ? y + 1 : y;
    if (a.out[s] == nullptr) return;
    if (is_gate && gate_row_a_run(a.gate_rows, a.gate_parts)) {
        const uint32_t row = (y - (SUMS - 1)) * FINISH_RUNS + p;
        if (row >= a.gate_rows || c >= a.cols) return;
        const float* q = a.gate_partials + (int64_t)row * a.gate_parts * a.cols + c;
        float t = 0.0f;
        for (uint32_t b = 0; b < a.gate_parts; ++b) t += q[(int64_t)b * a.cols];
        const int64_t at = (int64_t)row * a.cols + c;
        if (a.gate_bf16) static_cast<__bf16*>(a.out[s])[at] = (__bf16)t;
        else             static_cast<float*>(a.out[s])[at] = t;
        return;
    }
    const uint32_t parts = is_gate ? a.gate_parts : (a.none >> s & 1u) ? 0u : a.parts;
    const float* from = is_gate ? a.gate_partials + (int64_t)(y - (SUMS - 1)) * parts * a.cols : a.partials + (int64_t)s * parts * a.cols;
    const uint32_t per = (parts + FINISH_RUNS - 1) / FINISH_RUNS, b0 = min(parts, p * per), b1 = min(parts, b0 + per);
    float t = 0.0f;
    if (c < a.cols) {
        const float* q = from + (int64_t)b0 * a.cols + c;
        uint32_t b = b0;
        for (; b + 8u <= b1; b += 8u, q += (int64_t)8 * a.cols) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = q[(int64_t)i * a.cols];
#pragma unroll
            for (int i = 0; i < 8; ++i) t += v[i];
        }
        for (; b < b1; ++b, q += a.cols) t += *q;
    }
    part[p][lc] = t;
    __syncthreads();
    if (p == 0 && c < a.cols) {
        float sum = part[0][lc];
#pragma unroll
        for (uint32_t i = 1; i < FINISH_RUNS; ++i) sum += part[i][lc];
        const int64_t at = (is_gate ? (int64_t)(y - (SUMS - 1)) * a.cols : 0) + c;
        if (is_gate ? a.gate_bf16 : a.param_bf16) static_cast<__bf16*>(a.out[s])[at] = (__bf16)sum;
        else                                      static_cast<float*>(a.out[s])[at] = sum;
    }
}

// Rows whose parameters do not fit in LDS one by one (ParamPlanes).  The forward kernel holds the next row beside this one, which with
// four vectors is more than a lane's registers: 20 to 356 bytes of scratch a lane in whole rows with a post-norm, about 1000 in odd ones.
TeamShape four_vectors(int64_t cols) { return {lanes_for((cols + 31) / 32), 4}; }

// The shape that wastes the fewest lanes, of those that keep a row in one wave if there is one.  50432 x 768 bf16, layer norms on
// both sides and a gate: three vectors of 32 lanes 56.7 us, two of 64, a quarter of them idle, 66.0; the RMS pre-norm alone 52.3
// and 52.8.  (In FP32 with few rows the second is up to 7 % ahead: 25216 x 384 41.4 and 38.8.)
TeamShape shape_for(int64_t cols, int most)
{
    const int64_t vectors = (cols + 7) / 8;
    TeamShape best{0, 0};
    int64_t slots = INT64_MAX;
    if (vectors <= 64 * most) {
        for (uint32_t lanes = 64; lanes >= 8; lanes /= 2) {
            const int v = (int)((vectors + lanes - 1) / lanes);
            if (v <= most && (int64_t)lanes * v < slots) { best = {lanes, v}; slots = (int64_t)lanes * v; }
        }
        return best;
    }
    for (int v = 2; v <= most; ++v) {
        const uint32_t lanes = lanes_for((vectors + v - 1) / v);
        const int held = (int)((vectors + lanes - 1) / lanes);              // only the last vector of a lane may lie behind the row
        if (lanes <= NORM_THREADS && (int64_t)lanes * held < slots) { best = {lanes, held}; slots = (int64_t)lanes * held; }
    }
    return best.v > 0 ? best : four_vectors(cols);
}

template <typename XT, typename UT>
hipError_t launch_fwd(const ResidualNormParams& p, hipStream_t st)
{
    const int64_t vectors = (p.cols + 7) / 8;
    // few rows, of which a unit has no more than four: a lane takes one vector, the latency of a row counts.  One row of 4096 with
    // both norms 3.7 us, by the other rule 4.5; 1000 rows 9.7 and 9.9; one row of 768 3.0 and 4.3, 1000 rows 4.4 and 4.9
    TeamShape s = p.rows <= 4 * UNITS && vectors <= NORM_THREADS ? TeamShape{lanes_for(vectors), 1} : shape_for(p.cols, 3);
    const bool gate_rows = p.gate != nullptr && p.gate_rows > 1;
    NormArgs g;
    uint32_t teams, grid;
    const RowEnd end = row_end(p.cols);
    bool far = false;
    size_t lds;
    for (;;) {
        const uint32_t most = far ? 1 : std::max(1u, NORM_THREADS / s.lanes);
        teams = whole_waves((uint32_t)std::min<int64_t>(most, std::max<int64_t>(1, (p.rows + UNITS - 1) / UNITS)), s.lanes);
        g = norm_args(p, s);
        // 8 waves on a unit, with one vector a lane 16.  8192 x 4096 bf16 with everything: 8 waves 51.9 us, 12 52.9, 16 58.8 (2048
        // columns 30.9, 31.0, 29.6).  One vector a lane, 50432 x 256: 8 waves 26.0 us, 16 24.6, 32 28.3 (FP32 44.7, 46.7, 48.1)
        const uint32_t per_unit = std::max(1u, (s.v == 1 ? 16u : 8u) * 64u / (teams * s.lanes));
        grid = (uint32_t)std::min<int64_t>((p.rows + teams - 1) / teams, (int64_t)UNITS * per_unit);
        g.teams = std::min<int64_t>(p.rows, (int64_t)grid * teams);
        g.team_rows = (p.rows + g.teams - 1) / g.teams;
        g.row_step = gate_rows ? 1 : g.teams;
        const int64_t span = rows_at_once(gate_rows, s.lanes, grid, teams, g.team_rows);
        if (!far && (!covers(p.x, p.x_bf16, p.ldx, span) || !covers(p.u, p.u_bf16, p.ldu, span) || !covers(p.h, p.x_bf16, p.ldh, span) ||
                     !covers(p.y, p.u_bf16, p.ldy, span))) {
            far = true;
            s = one_team(s, p.cols);
            continue;
        }
        lds = s.v == 1 ? 0 :
              s.v == 4 ? give_planes(g, s, {{P_PRE_WEIGHT, p.y || p.y_codes}, {P_POST_WEIGHT, p.post}, {P_GATE, p.gate && !gate_rows},
                                            {P_PRE_BIAS, p.layer && (p.y || p.y_codes)}, {P_POST_BIAS, p.layer && p.post}}) :
                         param_bytes(s, end, p.post, p.gate != nullptr, p.layer, false, gate_rows ? teams : 0);
        if (lds <= NORM_LDS_MAX) break;
        s = four_vectors(p.cols);
    }
    const uint32_t threads = teams * s.lanes;
    hipError_t e = hipSuccess;
    by_vectors(s.v, [&](auto v) {
        by_kind(end, p.post, p.gate != nullptr, [&](auto post, auto gate, auto ends) {
            auto run = [&](auto eight) {
                if constexpr (decltype(ends)::value != ROW_SHORT || decltype(v)::value == 1) e = start_norm(residual_norm_fwd_kernel<XT, UT, decltype(v)::value, decltype(post)::value, decltype(gate)::value,
                                                        decltype(eight)::value, decltype(ends)::value>, grid, threads, lds, st, g);
            };
            if constexpr (decltype(ends)::value != ROW_WHOLE) run(std::true_type{});
            else                                              by_flag(p.h8 != nullptr || p.u8 != nullptr, run);
        });
    });
    return e;
}

// Whether a backward kernel's parameters and its teams' gate rows fit in LDS.
bool fit_in_lds(int64_t cols, int64_t gate_rows, bool post, bool gate, bool layer)
{
    const TeamShape s = shape_for(cols, 2);
    return s.v < 4 && param_bytes(s, row_end(cols), post, gate, layer, true, gate_rows > 1 ? whole_waves(NORM_THREADS / s.lanes, s.lanes) : 0) <= NORM_LDS_MAX;
}

// Shape of a backward launch, the same for every type.  Up to two vectors a lane: with three the sums of all kinds do not fit in
// registers.  In halves the rows are read twice, which is ahead where one kernel would have to load a row for each of its steps:
// 2048 x 16384 bf16, RMS norms on both sides, gate, 8-bit checkpoints 277 us in one, 151 in halves; layer norms 467 and 162; the
// RMS pre-norm alone, of which one kernel would hold the sums, 87 and 104.  And where the teams' gate rows do not fit in LDS
// beside the parameters (8192 columns, the larger kinds).
struct BwdPlan {
    TeamShape shape;
    uint32_t teams_per_block, grid, strips;
    int64_t teams, pieces, team_rows;        // pieces 0: teams own whole gate rows
    bool halves;                             // rows first, then sums (strips of columns, a wave each)
};

// fits: the parameters fit in LDS (fit_in_lds).
// far_grid: the workgroups of a launch whose teams are one each (one_team), which takes no more workspace than the other; 0: not so.
BwdPlan plan_bwd(int64_t rows, int64_t cols, int64_t gate_rows, bool fits, uint32_t far_grid = 0)
{
    BwdPlan b{};
    b.shape = shape_for(cols, 2);
    b.halves = b.shape.v == 4 || !fits;
    if (b.halves) b.shape = {64, 1};
    b.strips = b.halves ? (uint32_t)((cols + 511) / 512) : 1;
    if (far_grid > 0) b.shape = one_team(b.shape, cols);
    const uint32_t lanes = b.shape.lanes, most = far_grid > 0 ? 1 : NORM_THREADS / lanes;
    const uint32_t grid = far_grid > 0 ? far_grid : UNITS / b.strips;                      // 8 waves on a unit: few sums to add up
    b.teams_per_block = (uint32_t)std::min<int64_t>(most, std::max<int64_t>(1, (rows + grid - 1) / grid));
    b.teams_per_block = whole_waves(b.teams_per_block, lanes);
    const int64_t teams = std::min<int64_t>(rows, (int64_t)grid * b.teams_per_block), run = rows / gate_rows;
    if (gate_rows == 1 || 2 * gate_rows <= teams) {
        b.pieces = std::min(run, teams / gate_rows);
        b.teams = gate_rows * b.pieces;
        b.team_rows = (run + b.pieces - 1) / b.pieces;
    } else {
        b.teams = gate_rows <= 2 * teams && far_grid == 0 ? gate_rows : teams;
        b.team_rows = (gate_rows + b.teams - 1) / b.teams * run;
    }
    b.grid = (uint32_t)((b.teams + b.teams_per_block - 1) / b.teams_per_block);
    return b;
}

}  // namespace

hipError_t launch_residual_norm_fwd(const ResidualNormParams& p, hipStream_t st)
{
    hipError_t e = hipSuccess;
    by_types(p.x_bf16, p.u_bf16, [&](auto xt, auto ut) { e = launch_fwd<decltype(xt), decltype(ut)>(p, st); });
    return e;
}

size_t residual_norm_workspace_bytes(int64_t rows, int64_t cols, int64_t gate_rows)
{
    size_t most = 0;
    // whether a call goes in halves may depend on its kind: enough for the largest kind and the smallest
    for (const bool fits : {fit_in_lds(cols, gate_rows, true, true, true), fit_in_lds(cols, gate_rows, false, gate_rows > 0, false)}) {
        const BwdPlan b = plan_bwd(rows, cols, std::max<int64_t>(1, gate_rows), fits);
        const int64_t gate = gate_rows > 1 ? (b.pieces > 0 ? b.teams : 0) : b.grid;
        most = std::max(most, (b.halves ? (size_t)rows * sizeof(float2) : 0) + ((size_t)SUMS * b.grid + (size_t)gate) * (size_t)cols * sizeof(float));
    }
    return most;
}

hipError_t launch_residual_norm_bwd(const ResidualNormParams& given, const ResidualNormGrads& d, hipStream_t st)
{
    ResidualNormParams p = given;
    const bool eight = p.h8 != nullptr || p.u8 != nullptr;
    if (d.dy == nullptr) {
        // nothing of the pre-norm's term is left: h reads as zero and its weight as one, so that a row of h that is not finite, or
        // such a weight, does not meet the zeros of dy; nor do the statistics, which a kernel with a post-norm masks, and another
        // does without
        p.h = p.h8 = p.h8_scales = nullptr;
        p.pre_weight = nullptr;
        if (!p.post) p.stats = nullptr;
    }
    const int64_t gate_rows = p.gate != nullptr ? p.gate_rows : 1;
    const bool fits = fit_in_lds(p.cols, gate_rows, p.post, p.gate != nullptr, p.layer);
    BwdPlan b = plan_bwd(p.rows, p.cols, gate_rows, fits);
    const int64_t span = rows_at_once(gate_rows > 1, b.shape.lanes, b.grid, b.teams_per_block, b.team_rows);
    if (!covers(d.dh, p.x_bf16, d.lddh, span) || !covers(d.dy, p.u_bf16, d.lddy, span) || !covers(d.dx, p.x_bf16, d.lddx, span) ||
        !covers(d.du, p.u_bf16, d.lddu, span) || (!eight && (!covers(p.h, p.x_bf16, p.ldh, span) || !covers(p.u, p.u_bf16, p.ldu, span))))
        b = plan_bwd(p.rows, p.cols, gate_rows, fits, b.grid);
    const RowEnd end = row_end(p.cols);
    const auto launch = p.layer ? launch_norm_bwd_layer : launch_norm_bwd_rms;
    NormGradArgs a{};
    a.f = norm_args(p, b.shape);
    a.dh = d.dh; a.dy = d.dy; a.dx = d.dx; a.du = d.du;
    a.lddh = d.lddh; a.lddy = d.lddy; a.lddx = d.lddx; a.lddu = d.lddu;
    a.means = static_cast<float2*>(d.workspace);
    a.partials = static_cast<float*>(d.workspace) + (b.halves ? 2 * p.rows : 0);
    a.gate_partials = a.partials + (int64_t)SUMS * b.grid * p.cols;
    a.dgate = d.dgate;
    a.gate_rows = gate_rows; a.pieces = b.pieces;
    a.want_gate = p.gate != nullptr && d.dgate != nullptr;
    NormFinishArgs f{};
    f.partials = a.partials; f.gate_partials = a.gate_partials;
    f.parts = b.grid; f.gate_parts = gate_rows > 1 ? (uint32_t)b.pieces : b.grid; f.cols = (uint32_t)p.cols;
    f.param_bf16 = p.param_bf16; f.gate_bf16 = p.gate_bf16;
    f.out[PRE_WEIGHT] = d.dpre_weight; f.out[PRE_BIAS] = d.dpre_bias; f.out[POST_WEIGHT] = d.dpost_weight; f.out[POST_BIAS] = d.dpost_bias;
    const bool part[] = {d.dy != nullptr, p.post, true, d.dy != nullptr && p.layer, p.post && p.layer};       // as NormSum
    for (int s = 0; s < SUMS; ++s) f.none |= part[s] ? 0u : 1u << s;
    f.out[GATE_SUM] = a.want_gate && b.pieces > 0 ? d.dgate : nullptr;
    f.gate_rows = (uint32_t)gate_rows;
    const uint32_t gates = !f.out[GATE_SUM] ? 0 : gate_row_a_run(f.gate_rows, f.gate_parts) ? (f.gate_rows + FINISH_RUNS - 1) / FINISH_RUNS : f.gate_rows;
    bool wanted = gates > 0;
    for (void* o : f.out) wanted = wanted || o != nullptr;

    hipError_t e = hipSuccess;
    if (b.halves) {
        const TeamShape s = four_vectors(p.cols);
        NormGradArgs r = a;
        r.f = norm_args(p, s);
        const uint32_t grid = (uint32_t)std::min<int64_t>(p.rows, UNITS);
        r.f.teams = r.f.row_step = grid;
        r.f.team_rows = (p.rows + grid - 1) / grid;
        const size_t lds = give_planes(r.f, s, {{P_PRE_WEIGHT, d.dy != nullptr}, {P_POST_WEIGHT, p.post}, {P_GATE, p.gate && gate_rows == 1}});
        e = launch(r, p.x_bf16, p.u_bf16, eight, end, s.v, BWD_ROWS, grid, s.lanes, lds, st);
        if (e != hipSuccess || (!wanted && !a.want_gate)) return e;
    }
    a.f.teams = b.teams; a.f.team_rows = b.team_rows; a.f.row_step = gate_rows > 1 ? 1 : b.teams;
    const uint32_t threads = b.teams_per_block * b.shape.lanes, width = b.shape.lanes * b.shape.v * 8;
    // the parameters, with the teams' gate rows; at the end the sums
    size_t lds = param_bytes(b.shape, end, p.post, p.gate != nullptr, p.layer, true, a.f.gate_by_row ? b.teams_per_block : 0);
    if (b.teams_per_block > 1) lds = std::max(lds, (size_t)b.teams_per_block * width * sizeof(float));
    e = launch(a, p.x_bf16, p.u_bf16, eight, end, b.shape.v, b.halves ? BWD_SUMS : BWD_ALL, dim3(b.grid, b.strips), threads, lds, st);
    if (e != hipSuccess || !wanted) return e;
    residual_norm_finish_kernel<<<(uint32_t)((p.cols + 31) / 32) * (SUMS - 1 + gates), 32 * FINISH_RUNS, 0, st>>>(f);
    return hipGetLastError();
}

}  // namespace mxl
