// Activations with 8-bit checkpoints of their input: a = act(p), or act(p1) . p2 of a matrix [p1 | p2]; the backward pass
// reads the checkpoint in place of p.  And the checkpoint codec by itself.
//
// All of them stream: a lane owns eight consecutive elements, four neighbouring lanes a group of 32, and every array is
// touched once, 16 bytes (8 of codes) a lane.  Bound by memory, GELU by the vector units as well (29 operations an element
// forward with the checkpoint; busy all of the time, so that its time follows the clock).  bf16 with checkpoints: GELU
// 50432 x 4096 187 us forward for 1039 MB and 194 backward, gated SiLU 16384 x (2 x 8192) 201 and 202 us for 1082 MB each; a
// large copy's 5.4 TB/s would take 192 and 200.  Packing 50432 x 1024 in bf16 28 us, unpacking 23.5 (the codes partly cached).
#include "mx_block.hpp"

#include <algorithm>

namespace mxl {

using namespace mxb;

namespace {

// Chunks of eight elements, `per_row` of them to a row of whole groups; chunk / per_row without a division: with
// magic = ceil(2^64 / per_row) the product's upper 64 bits are exact for every 32-bit chunk number.
struct Chunks {
    uint64_t magic;
    uint32_t per_row, count;
    __device__ __forceinline__ uint32_t row_of(uint32_t chunk) const
    {
        const uint64_t lo = (uint64_t)chunk * (uint32_t)magic, hi = (uint64_t)chunk * (uint32_t)(magic >> 32) + (lo >> 32);
        return (uint32_t)(hi >> 32);
    }
};

Chunks chunks_of(int64_t rows, int64_t cols)
{
    Chunks c{};
    c.per_row = (uint32_t)((cols + 31) / 32 * 4);
    c.count = (uint32_t)(rows * c.per_row);
    c.magic = ~0ull / c.per_row + 1;                     // per_row > 1
    return c;
}

struct ActArgs {
    const void* p;
    void* a;
    void* dp;
    uint8_t* a_codes;
    uint8_t* a_scales;
    uint8_t* p8;
    uint8_t* p8_scales;
    int64_t ldp, lda, lddp;
    Chunks chunks;
    uint32_t cols;
    bool floor_mode;
};

// act(x) and, where wanted, its derivative.
//   SiLU: x s, s = 1 / (1 + exp(-x));  derivative s (1 + x (1 - s)).
//   GELU: x Phi(x);  derivative Phi(x) + x phi(x).  With z = |x| / sqrt(2), Phi(-|x|) = erfc(z) / 2 = exp(-x^2 / 2) G(z) / 2,
//   G(z) = t P8(t - t0), t = 1 / (1 + z / 2): the fit of the scaled complementary error function that the products' GELU
//   stage uses (fit_gelu_erfcx.py); the exponential serves both Phi and phi.  Taking its argument in one rounding leaves
//   a relative error of 2^-24 x^2 / 2 in the tails, where the values are exp(-x^2 / 2).
template <bool SILU, bool SLOPE>
__device__ __forceinline__ float act(float x, float& slope)
{
    if (SILU) {
        const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * -1.442695041f));
        if (SLOPE) slope = s * __builtin_fmaf(x, 1.0f - s, 1.0f);
        return x * s;
    }
    constexpr float T0 = 0.5709219574928284f;
    constexpr float C[9] = {0.562385082244873f, 0.768385112285614f, 0.584431529045105f, 0.09252145141363144f, -0.20070798695087433f,
                            -0.058531392365694046f, 0.11107011884450912f, 0.014878340996801853f, -0.05936833471059799f};
    const float ax = __builtin_fabsf(x);
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(ax, 0.35355339059327376f, 1.0f));
    const float e = __builtin_amdgcn_exp2f(ax * ax * -0.72134752044f);
    const float w = t - T0;
    float g = __builtin_fmaf(C[8], w, C[7]);
#pragma unroll
    for (int k = 6; k >= 0; --k) g = __builtin_fmaf(g, w, C[k]);
    const float c = 0.5f * g * t * e;                    // Phi(-|x|)
    if (SLOPE) slope = __builtin_fmaf(x, e * 0.3989422804f, x >= 0.0f ? 1.0f - c : c);
    return __builtin_fmaf(-ax, c, __builtin_fmaxf(x, 0.0f));
}

constexpr uint32_t THREADS = 256;

// Chunks a lane works on, one workgroup's width apart; their loads go out together.  Gated SiLU backward, 16384 x 16384 bf16: two
// chunks 201 us, four 202, eight 210; packing 50432 x 1024: 26.6, 26.3, 25.6.
template <typename T> constexpr int CHUNKS = sizeof(T) == 2 ? 4 : 2;

template <typename T, bool SILU, bool GATED, bool TAIL>
__global__ __launch_bounds__(THREADS) void activation_fwd_kernel(const ActArgs g)
{
    constexpr int N = GATED ? CHUNKS<T> / 2 : CHUNKS<T>;
    constexpr int HALVES = GATED ? 2 : 1;
    const uint32_t base = blockIdx.x * (THREADS * N) + threadIdx.x;
    Raw<T> r[N][HALVES];
    uint32_t row[N], col[N];
    int n[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t chunk = base + i * THREADS;
        row[i] = g.chunks.row_of(chunk);
        col[i] = (chunk - row[i] * g.chunks.per_row) * 8u;
        n[i] = chunk < g.chunks.count ? (int)g.cols - (int)col[i] : 0;
        const T* p = static_cast<const T*>(g.p) + row[i] * g.ldp + col[i];
#pragma unroll
        for (int k = 0; k < HALVES; ++k) r[i][k] = load_raw<TAIL>(p + (k ? g.cols : 0), n[i]);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const bool live = base + i * THREADS < g.chunks.count;
        F8 f[HALVES], y;
#pragma unroll
        for (int k = 0; k < HALVES; ++k) f[k] = widen(r[i][k]);
        if (g.p8 != nullptr) {
#pragma unroll
            for (int k = 0; k < HALVES; ++k) {
                uint32_t byte;
                const Codes8 c = pack8(f[k], byte);
                if (live) {
                    const int64_t at = ((int64_t)row[i] * HALVES + k) * (g.chunks.per_row * 8u) + col[i];
                    *reinterpret_cast<uint2*>(g.p8 + at) = make_uint2(c.w[0], c.w[1]);
                    if ((threadIdx.x & 3u) == 0) g.p8_scales[at >> 5] = (uint8_t)byte;
                }
            }
        }
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            float slope;
            y.v[t] = act<SILU, false>(f[0].v[t], slope);
            if (GATED) y.v[t] *= f[HALVES - 1].v[t];
        }
        if (g.a_codes != nullptr) {
            const uint32_t byte = mxd::scale_byte(mxd::quad_max(mxd::amax_bits8(y)), g.floor_mode);
            const uint32_t c = mxd::rtn_codes8_f32(y.v, byte);
            if (live) {
                const int64_t at = (int64_t)row[i] * g.cols + col[i];        // whole groups only
                *reinterpret_cast<uint32_t*>(g.a_codes + (at >> 1)) = c;
                if ((threadIdx.x & 3u) == 0) g.a_scales[at >> 5] = (uint8_t)byte;
            }
        } else {
            store8<TAIL>(static_cast<T*>(g.a) + row[i] * g.lda + col[i], y, n[i]);
        }
    }
}

template <typename T, bool SILU, bool GATED, bool CKPT, bool TAIL>
__global__ __launch_bounds__(THREADS) void activation_bwd_kernel(const ActArgs g)
{
    constexpr int N = GATED ? CHUNKS<T> / 2 : CHUNKS<T>;
    constexpr int HALVES = GATED ? 2 : 1;
    const uint32_t base = blockIdx.x * (THREADS * N) + threadIdx.x;
    Raw<T> d[N], r[N][HALVES];
    Codes8 code[N][HALVES];
    uint32_t byte[N][HALVES], row[N], col[N];
    int n[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t chunk = base + i * THREADS;
        row[i] = g.chunks.row_of(chunk);
        col[i] = (chunk - row[i] * g.chunks.per_row) * 8u;
        n[i] = chunk < g.chunks.count ? (int)g.cols - (int)col[i] : 0;
        d[i] = load_raw<TAIL>(static_cast<const T*>(g.a) + row[i] * g.lda + col[i], n[i]);
#pragma unroll
        for (int k = 0; k < HALVES; ++k) {
            if (CKPT) {
                const int64_t at = ((int64_t)row[i] * HALVES + k) * (g.chunks.per_row * 8u) + col[i];
                code[i][k].w[0] = code[i][k].w[1] = byte[i][k] = 0;
                if (n[i] > 0) {
                    // read once: 128 MB of gradient 50.3 us with an ordinary load, 43.7 so; beyond the last-level cache the same
                    const u2_any c = __builtin_nontemporal_load(reinterpret_cast<const u2_any*>(g.p8 + at));
                    code[i][k].w[0] = c.x; code[i][k].w[1] = c.y;
                    byte[i][k] = g.p8_scales[at >> 5];
                }
            } else {
                r[i][k] = load_raw<TAIL>(static_cast<const T*>(g.p) + row[i] * g.ldp + col[i] + (k ? g.cols : 0), n[i]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        F8 f[HALVES], out[HALVES];
        const F8 da = widen(d[i]);
#pragma unroll
        for (int k = 0; k < HALVES; ++k) f[k] = CKPT ? unpack8(code[i][k], byte[i][k]) : widen(r[i][k]);
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            float slope;
            const float y = act<SILU, true>(f[0].v[t], slope);
            if (GATED) {
                out[0].v[t] = da.v[t] * f[HALVES - 1].v[t] * slope;
                out[HALVES - 1].v[t] = da.v[t] * y;
            } else {
                out[0].v[t] = da.v[t] * slope;
            }
        }
#pragma unroll
        for (int k = 0; k < HALVES; ++k) store8<TAIL>(static_cast<T*>(g.dp) + row[i] * g.lddp + col[i] + (k ? g.cols : 0), out[k], n[i]);
    }
}

struct CodecArgs {
    void* values;
    uint8_t* codes;
    uint8_t* scales;
    int64_t ld;
    Chunks chunks;
    uint32_t cols;
};

template <typename T, bool TAIL>
__global__ __launch_bounds__(THREADS) void checkpoint_pack_kernel(const CodecArgs g)
{
    constexpr int N = CHUNKS<T>;
    const uint32_t base = blockIdx.x * (THREADS * N) + threadIdx.x;
    Raw<T> r[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t chunk = base + i * THREADS, row = g.chunks.row_of(chunk), col = (chunk - row * g.chunks.per_row) * 8u;
        r[i] = load_raw<TAIL>(static_cast<const T*>(g.values) + row * g.ld + col, chunk < g.chunks.count ? (int)g.cols - (int)col : 0);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t chunk = base + i * THREADS;
        uint32_t byte;
        const Codes8 c = pack8(widen(r[i]), byte);
        if (chunk < g.chunks.count) {
            *reinterpret_cast<uint2*>(g.codes + (size_t)chunk * 8) = make_uint2(c.w[0], c.w[1]);
            if ((threadIdx.x & 3u) == 0) g.scales[chunk >> 2] = (uint8_t)byte;
        }
    }
}

template <typename T, bool TAIL>
__global__ __launch_bounds__(THREADS) void checkpoint_unpack_kernel(const CodecArgs g)
{
    constexpr int N = CHUNKS<T>;
    const uint32_t base = blockIdx.x * (THREADS * N) + threadIdx.x;
    Codes8 c[N];
    uint32_t byte[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t chunk = base + i * THREADS;
        c[i].w[0] = c[i].w[1] = byte[i] = 0;
        if (chunk < g.chunks.count) {
            const uint2 w = *reinterpret_cast<const uint2*>(g.codes + (size_t)chunk * 8);
            c[i].w[0] = w.x; c[i].w[1] = w.y;
            byte[i] = g.scales[chunk >> 2];
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t chunk = base + i * THREADS, row = g.chunks.row_of(chunk), col = (chunk - row * g.chunks.per_row) * 8u;
        store8<TAIL>(static_cast<T*>(g.values) + row * g.ld + col, unpack8(c[i], byte[i]), chunk < g.chunks.count ? (int)g.cols - (int)col : 0);
    }
}

uint32_t blocks_for(const Chunks& c, int per_lane)
{
    const uint64_t per = (uint64_t)THREADS * per_lane;
    return (uint32_t)((c.count + per - 1) / per);
}

ActArgs args_of(const ActivationParams& p)
{
    ActArgs g{};
    g.p = p.p; g.a = p.a; g.dp = p.dp; g.a_codes = p.a_codes; g.a_scales = p.a_scales; g.p8 = p.p8; g.p8_scales = p.p8_scales;
    g.ldp = p.ldp; g.lda = p.lda; g.lddp = p.lddp;
    g.chunks = chunks_of(p.rows, p.cols);
    g.cols = (uint32_t)p.cols;
    g.floor_mode = p.floor_mode;
    return g;
}

template <typename T, typename F>
void by_kind(bool silu, bool gated, F&& f)
{
    using std::bool_constant;
    if (silu) gated ? f(bool_constant<true>{}, bool_constant<true>{}) : f(bool_constant<true>{}, bool_constant<false>{});
    else      gated ? f(bool_constant<false>{}, bool_constant<true>{}) : f(bool_constant<false>{}, bool_constant<false>{});
}

template <typename T>
void launch_act(const ActivationParams& p, bool backward, hipStream_t st)
{
    const ActArgs g = args_of(p);
    by_kind<T>(p.silu, p.gated, [&](auto silu, auto gated) {
        const uint32_t blocks = blocks_for(g.chunks, decltype(gated)::value ? CHUNKS<T> / 2 : CHUNKS<T>);
        constexpr bool S = decltype(silu)::value, G = decltype(gated)::value;
        auto run = [&](auto kernel) { kernel<<<blocks, THREADS, 0, st>>>(g); };
        const bool tail = p.cols % 8 != 0;
        if (!backward)            tail ? run(activation_fwd_kernel<T, S, G, true>) : run(activation_fwd_kernel<T, S, G, false>);
        else if (p.p8 != nullptr) tail ? run(activation_bwd_kernel<T, S, G, true, true>) : run(activation_bwd_kernel<T, S, G, true, false>);
        else                      tail ? run(activation_bwd_kernel<T, S, G, false, true>) : run(activation_bwd_kernel<T, S, G, false, false>);
    });
}

CodecArgs args_of(const CheckpointParams& p)
{
    CodecArgs g{};
    g.values = p.values; g.codes = p.codes; g.scales = p.scales; g.ld = p.ld;
    g.chunks = chunks_of(p.rows, p.cols);
    g.cols = (uint32_t)p.cols;
    return g;
}

}  // namespace

hipError_t launch_activation_fwd(const ActivationParams& p, hipStream_t st)
{
    p.bf16 ? launch_act<uint16_t>(p, false, st) : launch_act<float>(p, false, st);
    return hipGetLastError();
}

hipError_t launch_activation_bwd(const ActivationParams& p, hipStream_t st)
{
    p.bf16 ? launch_act<uint16_t>(p, true, st) : launch_act<float>(p, true, st);
    return hipGetLastError();
}

template <typename T>
static void launch_codec(const CheckpointParams& p, bool pack, hipStream_t st)
{
    const CodecArgs g = args_of(p);
    auto run = [&](auto kernel) { kernel<<<blocks_for(g.chunks, CHUNKS<T>), THREADS, 0, st>>>(g); };
    const bool tail = p.cols % 8 != 0;
    if (pack) tail ? run(checkpoint_pack_kernel<T, true>) : run(checkpoint_pack_kernel<T, false>);
    else      tail ? run(checkpoint_unpack_kernel<T, true>) : run(checkpoint_unpack_kernel<T, false>);
}

hipError_t launch_checkpoint_pack(const CheckpointParams& p, hipStream_t st)
{
    p.bf16 ? launch_codec<uint16_t>(p, true, st) : launch_codec<float>(p, true, st);
    return hipGetLastError();
}

hipError_t launch_checkpoint_unpack(const CheckpointParams& p, hipStream_t st)
{
    p.bf16 ? launch_codec<uint16_t>(p, false, st) : launch_codec<float>(p, false, st);
    return hipGetLastError();
}

}  // namespace mxl
