// Gated residual with the norms on both sides of a block, and its backward pass: what their launches share.
//     v = post ? n(u; post_weight, post_bias) : u
//     h = rho x + sigma g . v                       stored in the stream's type
//     y = n(h; pre_weight, pre_bias)                of the stored h; in the branch's type, or as MXFP4 codes
// with n(a; w, b) = a r w, r = (mean a^2 + eps)^-1/2 (RMS), or (a - mu) r w + b, r = (var a + eps)^-1/2 (layer).
// Backward, with a^ the normalised input (a - mu) r:
//     b = dy pre_weight;        dh = dh_out + r_h (b - [mean b] - h^ mean(b h^));     dx = rho dh
//     dv = sigma g . dh;        c = dv post_weight;     du = r_u (c - [mean c] - u^ mean(c u^))
//     d_pre_weight = sum dy h^, d_pre_bias = sum dy, d_post_weight = sum dv u^, d_post_bias = sum dv,
//     d_gate = sum sigma dh . v        ([...]: layer only; the sums run over rows, for the gate over its rows)
//
// Both passes are bound by memory (8 to 12 bytes an element in bf16; 30 to 42 vector operations an element keep the vector
// units busy for half to two thirds of that time), so a row is read once: a team of lanes holds it in registers, V vectors of
// eight elements a lane, through both norms.  16384 x 4096 bf16, RMS norms on both sides, 8-bit checkpoints: 127 us forward for
// 675 MB and as much backward for 675 MB, 5.3 TB/s, which is a large copy's rate; 50432 x 768, layer norm, gate: 83 and 85 us for
// 391 and 394 MB; 25216 x 384 in FP32, layer norms on both sides, 128 gate rows: 43 and 58 us for 156 and 234 MB.
#pragma once
#include "mx_block.hpp"

#include <algorithm>
#include <initializer_list>
#include <utility>

namespace mxl {

using namespace mxb;

struct NormArgs {
    const void* x;
    const void* u;
    void* h;
    void* y;
    const void* pre_weight;
    const void* pre_bias;
    const void* post_weight;
    const void* post_bias;
    const void* gate;
    uint8_t* y_codes;
    uint8_t* y_scales;
    uint8_t* h8;
    uint8_t* h8_scales;
    uint8_t* u8;
    uint8_t* u8_scales;
    float4* stats;
    int64_t rows, ldx, ldu, ldh, ldy, ld_gate, gate_run;      // gate_run: rows of the stream that share a gate row
    int64_t teams, team_rows, row_step;                       // teams of the launch, the most rows that one has, from one to the next
    uint32_t cols, pitch8, lanes;
    float inv_cols, rho, sigma, eps;
    uint8_t plane[8];                                         // of the parameters in LDS (ParamPlanes)
    bool layer, post, param_bf16, gate_bf16, gate_by_row, floor_mode;
    bool in_place;                                            // h is x
};

struct NormGradArgs {
    NormArgs f;
    const void* dh;
    const void* dy;
    void* dx;
    void* du;
    int64_t lddh, lddy, lddx, lddu;
    float* partials;          // [SUMS][workgroups][cols]
    float* gate_partials;     // [gate rows x pieces][cols], or [workgroups][cols] for a gate of one row
    float2* means;            // of each row, between the two halves
    void* dgate;              // where whole gate rows belong to one team
    int64_t gate_rows, pieces;                                // pieces 0: teams own whole gate rows
    bool want_gate;
};

// What a backward kernel does: the whole pass, or for rows so wide that the sums and a row do not fit in registers its two halves: the
// gradients of the rows, and then (from the means of the rows that these leave) the sums, a strip of columns at a time.
enum BwdPart { BWD_ALL, BWD_ROWS, BWD_SUMS };

enum NormSum { PRE_WEIGHT, POST_WEIGHT, GATE_SUM, PRE_BIAS, POST_BIAS, SUMS };
enum NormParam { P_PRE_WEIGHT, P_POST_WEIGHT, P_GATE, P_PRE_BIAS, P_POST_BIAS, PARAMS };

constexpr uint32_t UNITS = 256;                          // compute units
// The largest workgroup: rows of 16384 at four vectors a lane, and one wave of eight that load while others compute.  With 256
// and twice the workgroups 16384 x 4096 takes 138 us instead of 128 forward, 4096 x 8192 52 instead of 47.6.
constexpr uint32_t NORM_THREADS = 512;
constexpr size_t NORM_LDS_MAX = 160 * 1024 - sizeof(TeamScratch);

// How many elements the row has from `col` on (not positive: none).
__device__ __forceinline__ int left(uint32_t cols, uint32_t col) { return (int)cols - (int)col; }

// The parameters in LDS: for each eight columns the eight values of every parameter one behind the other, and four words
// more, so that the 16-byte reads of neighbouring lanes fall into different banks.  A lane needs one address for all of them.
template <bool POST, bool GATE, bool LAYER, bool BACKWARD>
struct ParamLds {
    static constexpr uint32_t GATE_SLOT = 1 + POST, PRE_BIAS_SLOT = GATE_SLOT + GATE, POST_BIAS_SLOT = PRE_BIAS_SLOT + (LAYER && !BACKWARD);
    static constexpr uint32_t STRIDE = (POST_BIAS_SLOT + (LAYER && POST)) * 8 + 4;      // words from one eight columns to the next
    static constexpr uint32_t GATE_STRIDE = 12;                          // the same for a gate row of a team's own
    static constexpr uint32_t slot(NormParam p)
    {
        return p == P_PRE_WEIGHT ? 0 : p == P_POST_WEIGHT ? 1 : p == P_GATE ? GATE_SLOT : p == P_PRE_BIAS ? PRE_BIAS_SLOT : POST_BIAS_SLOT;
    }
    static __device__ __forceinline__ void put(float* lds, uint32_t stride, NormParam p, uint32_t vector, const F8& f)
    {
        put(lds + vector * stride + slot(p) * 8, f);
    }
    static __device__ __forceinline__ F8 get(const float* lds, uint32_t stride, NormParam p, uint32_t vector) { return get(lds + vector * stride + slot(p) * 8); }
    static __device__ __forceinline__ void put(float* at, const F8& f)
    {
        float4* to = reinterpret_cast<float4*>(at);
        to[0] = make_float4(f.v[0], f.v[1], f.v[2], f.v[3]);
        to[1] = make_float4(f.v[4], f.v[5], f.v[6], f.v[7]);
    }
    static __device__ __forceinline__ F8 get(const float* at)
    {
        const float4* from = reinterpret_cast<const float4*>(at);
        const float4 lo = from[0], hi = from[1];
        return F8{{lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w}};
    }
};

// The same for rows so wide that they do not fit in that form: a plane of 16 bytes for each eight columns where a parameter is
// bfloat16, two where it is FP32, for as many as there is room for.  The rest are read from cache (NO_PLANE).
struct ParamPlanes {
    static constexpr uint8_t NO_PLANE = 0xFF;
    static __device__ __forceinline__ void put(float* lds, uint32_t plane, uint32_t vectors, uint32_t vector, bool bf16, const F8& f)
    {
        uint4* to = reinterpret_cast<uint4*>(lds) + plane * vectors + vector;
        if (bf16) {
            RawBf16 r;
            narrow(f, r);                                                // exact: it came from there
            to[0] = make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]);
        } else {
            to[0] = make_uint4(__float_as_uint(f.v[0]), __float_as_uint(f.v[1]), __float_as_uint(f.v[2]), __float_as_uint(f.v[3]));
            to[vectors] = make_uint4(__float_as_uint(f.v[4]), __float_as_uint(f.v[5]), __float_as_uint(f.v[6]), __float_as_uint(f.v[7]));
        }
    }
    static __device__ __forceinline__ F8 get(const float* lds, uint32_t plane, uint32_t vectors, uint32_t vector, bool bf16)
    {
        const uint4* from = reinterpret_cast<const uint4*>(lds) + plane * vectors + vector;
        const uint4 a = from[0];
        if (bf16) return widen(RawBf16{{a.x, a.y, a.z, a.w}});
        const uint4 b = from[vectors];
        return F8{{__uint_as_float(a.x), __uint_as_float(a.y), __uint_as_float(a.z), __uint_as_float(a.w),
                   __uint_as_float(b.x), __uint_as_float(b.y), __uint_as_float(b.z), __uint_as_float(b.w)}};
    }
};

__device__ __forceinline__ bool param_is_bf16(const NormArgs& g, NormParam which) { return which == P_GATE ? g.gate_bf16 : g.param_bf16; }

// A parameter's eight values from `col` on, from memory.
template <bool TAIL>
__device__ __forceinline__ F8 norm_param(const NormArgs& g, int which, uint32_t col)
{
    const int n = left(g.cols, col);
    switch (which) {
        case P_PRE_WEIGHT:  return param8<TAIL>(g.pre_weight, g.param_bf16, col, n, 1.0f);
        case P_POST_WEIGHT: return param8<TAIL>(g.post_weight, g.param_bf16, col, n, 1.0f);
        case P_PRE_BIAS:    return param8<TAIL>(g.pre_bias, g.param_bf16, col, n, 0.0f);
        case P_POST_BIAS:   return param8<TAIL>(g.post_bias, g.param_bf16, col, n, 0.0f);
        default:            return param8<TAIL>(g.gate, g.gate_bf16, col, n, 1.0f);
    }
}

// ---- a team's rows of a matrix ---------------------------------------------------------------------
// Rows at any alignment, through a buffer descriptor that starts at a row which is the same for the whole workgroup: the
// descriptor moves on by scalar instructions, a lane's offset from there never changes, and a lane without work has one beyond
// the descriptor's end, where the hardware returns zero and drops stores.  That saves the address arithmetic and its registers,
// and every branch.  A matrix that there is not (null) reads as zero and takes no stores.
// How a row ends: with whole vectors; inside one (ROW_ENDS: its lane loads the row's last eight elements and moves them down,
// and stores what it has in three pieces; nothing of that is a branch around a load, which would be waited for at once: 9850 rows
// of 1001 in bf16 take 32.7 us with one, 28.3 with all rows by address); or in its first vector (ROW_SHORT: by address).
enum RowEnd { ROW_WHOLE, ROW_ENDS, ROW_SHORT };
constexpr uint32_t OFF_END = 0x80000000u;                // beyond the end of every descriptor
constexpr int64_t OFF_MAX = 0x7FFFFFF0;                  // what one covers: a workgroup's rows have to fit

typedef uint32_t u4_vec __attribute__((ext_vector_type(4)));
typedef uint32_t u2_vec __attribute__((ext_vector_type(2)));

__device__ __forceinline__ __amdgpu_buffer_rsrc_t descriptor(const void* base, int64_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(base)) + bytes, (short)0, base == nullptr ? 0 : (int)OFF_MAX, 0x00020000);
}

constexpr int NT = 2;                                    // the nontemporal bit: loads that are not repeated soon, and 8-bit checkpoints

__device__ __forceinline__ RawBf16 buffer_load_raw(__amdgpu_buffer_rsrc_t r, uint32_t off, uint32_t step, uint16_t)
{
    const u4_vec a = __builtin_amdgcn_raw_buffer_load_b128(r, off, step, NT);
    return RawBf16{{a.x, a.y, a.z, a.w}};
}
__device__ __forceinline__ F8 buffer_load_raw(__amdgpu_buffer_rsrc_t r, uint32_t off, uint32_t step, float)
{
    const u4_vec a = __builtin_amdgcn_raw_buffer_load_b128(r, off, step, NT), b = __builtin_amdgcn_raw_buffer_load_b128(r, off + 16u, step, NT);
    return F8{{__uint_as_float(a.x), __uint_as_float(a.y), __uint_as_float(a.z), __uint_as_float(a.w),
               __uint_as_float(b.x), __uint_as_float(b.y), __uint_as_float(b.z), __uint_as_float(b.w)}};
}
// The step is added to the lane's offset: a 16-byte store with its offset in a scalar register reads its data late enough that an
// instruction right behind it, which the compiler takes to be safe there, has overwritten it (the first word of 16 lanes at a
// time); without one the compiler keeps the distance.
__device__ __forceinline__ void buffer_store_raw(__amdgpu_buffer_rsrc_t r, uint32_t off, uint32_t step, const RawBf16& v)
{
    __builtin_amdgcn_raw_buffer_store_b128(u4_vec{v.w[0], v.w[1], v.w[2], v.w[3]}, r, off + step, 0, 0);
}
__device__ __forceinline__ void buffer_store_raw(__amdgpu_buffer_rsrc_t r, uint32_t off, uint32_t step, const F8& v)
{
    const float* f = v.v;
    __builtin_amdgcn_raw_buffer_store_b128(u4_vec{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])}, r, off + step, 0, 0);
    __builtin_amdgcn_raw_buffer_store_b128(u4_vec{__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7])}, r, off + step + 16u, 0, 0);
}

// Where a lane of a team is: the workgroup's row `first`, and the team's so many rows behind it; both move on together.
struct Place {
    int64_t first;
    uint32_t behind;
    uint32_t col0, step;     // the lane's first column, columns from one of its vectors to the next
    uint32_t cols, pitch8;
    uint32_t live;           // whether the team has a row
    uint32_t back;           // by how much the lane's last vector begins before its column (ROW_ENDS)
    __device__ __forceinline__ int64_t row() const { return first + behind; }
    __device__ __forceinline__ uint32_t col(int v) const { return col0 + v * step; }
    __device__ __forceinline__ int left(int v) const { return live != 0 ? (int)cols - (int)col(v) : 0; }
    // Only the last of a lane's vectors can lie behind the row's end.
    template <int V> __device__ __forceinline__ bool in(int v, uint32_t end) const { return live != 0 && (v < V - 1 || col(v) < end); }
};

// Which of the launch's teams this one is, k, and which the workgroup's first, k0.  In order; but where a wave has several rows
// and they are not runs, the waves of a workgroup are a launch's width apart, so that the last rows, of which not every team has
// one, are spread over all units: 12608 x 768 in FP32 38.8 us in order, 34.7 so (pre-norm alone), 25216 x 384 40.2 and 35.6, in
// bf16 20.2 and 19.5.  With a row or less to a wave 9850 x 1001 in bf16, whose neighbouring rows share lines, takes 26.2 and 28.8.
struct TeamRows {
    int64_t k0, k;
    static __host__ __device__ __forceinline__ bool spread(bool runs, uint32_t lanes) { return !runs && lanes < 64u; }
    __device__ __forceinline__ TeamRows(bool runs, uint32_t team_in_block, uint32_t teams, uint32_t lanes)
    {
        const bool apart = spread(runs, lanes);
        const uint32_t per = apart ? 64u / lanes : teams;                 // of a wave
        k0 = (int64_t)blockIdx.x * per;
        k = k0 + (apart ? team_in_block / per * (gridDim.x * per) + team_in_block % per : team_in_block);
    }
};

template <RowEnd END, int V>
__device__ __forceinline__ uint32_t back_of(uint32_t cols, uint32_t col0, uint32_t step)
{
    const int n = left(cols, col0 + (V - 1) * step);
    return END == ROW_ENDS && n > 0 && n < 8 ? 8u - n : 0u;
}

template <RowEnd END, int V, typename T>
__device__ __forceinline__ Raw<T> load_vec(const void* base, int64_t ld, const Place& at, int v)
{
    if constexpr (END == ROW_SHORT) return load_raw<true>(static_cast<const T*>(base) + at.row() * ld + at.col(v), base == nullptr ? 0 : at.left(v));
    const __amdgpu_buffer_rsrc_t r = descriptor(base, at.first * ld * (int64_t)sizeof(T));
    const bool in = at.in<V>(v, at.cols);
    if (END == ROW_ENDS && v == V - 1) return buffer_load_raw(r, in ? (at.behind * (uint32_t)ld + at.col(v) - at.back) * sizeof(T) : OFF_END, 0, T{});
    return buffer_load_raw(r, in ? (at.behind * (uint32_t)ld + at.col0) * sizeof(T) : OFF_END, v * at.step * sizeof(T), T{});
}

// What load_vec gave for a lane's last vector, moved down to where it belongs; zeros come in behind it.
__device__ __forceinline__ void settle(RawBf16& r, uint32_t back)
{
    if (back == 0) return;
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = back & 1 ? __builtin_amdgcn_alignbit(i < 3 ? r.w[i + 1] : 0u, r.w[i], 16) : r.w[i];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = back & 2 ? (i < 3 ? w[i + 1] : 0u) : w[i];
#pragma unroll
    for (int i = 0; i < 4; ++i) r.w[i] = back & 4 ? (i < 2 ? w[i + 2] : 0u) : w[i];
}
__device__ __forceinline__ void settle(F8& r, uint32_t back)
{
    if (back == 0) return;
    float w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = back & 1 ? (i < 7 ? r.v[i + 1] : 0.0f) : r.v[i];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = back & 2 ? (i < 6 ? w[i + 2] : 0.0f) : w[i];
#pragma unroll
    for (int i = 0; i < 8; ++i) r.v[i] = back & 4 ? (i < 4 ? w[i + 4] : 0.0f) : w[i];
}

// The first n of eight elements, n < 8 (others: none), in pieces of four, two and one.
__device__ __forceinline__ void buffer_store_end(__amdgpu_buffer_rsrc_t r, uint32_t off, const RawBf16& v, int n)
{
    const bool some = n > 0 && n < 8, four = n & 4, two = n & 2;
    const uint32_t a = four ? v.w[2] : v.w[0], b = four ? v.w[3] : v.w[1];
    __builtin_amdgcn_raw_buffer_store_b64(u2_vec{v.w[0], v.w[1]}, r, some && four ? off : OFF_END, 0, 0);
    __builtin_amdgcn_raw_buffer_store_b32(a, r, some && two ? off + (n & 4) * 2u : OFF_END, 0, 0);
    __builtin_amdgcn_raw_buffer_store_b16((uint16_t)(two ? b : a), r, some && (n & 1) ? off + (n & 6) * 2u : OFF_END, 0, 0);
}
__device__ __forceinline__ void buffer_store_end(__amdgpu_buffer_rsrc_t r, uint32_t off, const F8& v, int n)
{
    const bool some = n > 0 && n < 8, four = n & 4, two = n & 2;
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(v.v[i]);
    const uint32_t a = four ? w[4] : w[0], b = four ? w[5] : w[1], c = four ? w[6] : w[2];
    __builtin_amdgcn_raw_buffer_store_b128(u4_vec{w[0], w[1], w[2], w[3]}, r, some && four ? off : OFF_END, 0, 0);
    __builtin_amdgcn_raw_buffer_store_b64(u2_vec{a, b}, r, some && two ? off + (n & 4) * 4u : OFF_END, 0, 0);
    __builtin_amdgcn_raw_buffer_store_b32(two ? c : a, r, some && (n & 1) ? off + (n & 6) * 4u : OFF_END, 0, 0);
}

template <RowEnd END, int V, typename T>
__device__ __forceinline__ void store_vec(void* base, int64_t ld, const Place& at, int v, const F8& f)
{
    Raw<T> raw;
    narrow(f, raw);
    if constexpr (END == ROW_SHORT) {
        store_raw<true>(static_cast<T*>(base) + at.row() * ld + at.col(v), raw, base == nullptr ? 0 : at.left(v));
        return;
    }
    const __amdgpu_buffer_rsrc_t r = descriptor(base, at.first * ld * (int64_t)sizeof(T));
    const uint32_t off = (at.behind * (uint32_t)ld + at.col0) * sizeof(T), step = v * at.step * sizeof(T);
    const bool ends = END == ROW_ENDS && v == V - 1;
    buffer_store_raw(r, (ends ? at.left(v) >= 8 : at.in<V>(v, at.cols)) ? off : OFF_END, step, raw);
    if (ends) buffer_store_end(r, off + step, raw, at.left(v));
}

// 8-bit codes and scale bytes; their rows are whole groups, so they always go through descriptors.
template <int V>
__device__ __forceinline__ void store_codes8(uint8_t* codes, uint8_t* scales, const Place& at, int v, const F8& f)
{
    uint32_t byte;
    const Codes8 c = pack8(f, byte);
    const bool in = at.in<V>(v, at.pitch8);
    const uint32_t groups = at.pitch8 >> 5;
    __builtin_amdgcn_raw_buffer_store_b64(u2_vec{c.w[0], c.w[1]}, descriptor(codes, at.first * at.pitch8), in ? at.behind * at.pitch8 + at.col0 : OFF_END, v * at.step, NT);
    __builtin_amdgcn_raw_buffer_store_b8((uint8_t)byte, descriptor(scales, at.first * groups),
                                         in && (at.col0 & 31u) == 0 ? at.behind * groups + (at.col0 >> 5) : OFF_END, v * at.step >> 5, 0);
}

template <int V>
__device__ __forceinline__ Codes8 load_codes8(const uint8_t* codes, const uint8_t* scales, const Place& at, int v, uint32_t& byte)
{
    const bool in = at.in<V>(v, at.pitch8);
    const uint32_t groups = at.pitch8 >> 5;
    const u2_vec c = __builtin_amdgcn_raw_buffer_load_b64(descriptor(codes, at.first * at.pitch8), in ? at.behind * at.pitch8 + at.col0 : OFF_END, v * at.step, NT);
    byte = __builtin_amdgcn_raw_buffer_load_b8(descriptor(scales, at.first * groups), in ? at.behind * groups + (at.col0 >> 5) : OFF_END, v * at.step >> 5, 0);
    return Codes8{{c.x, c.y}};
}

// The value is used from here on as it stands in its registers: what was computed from it before is computed again, not kept.
__device__ __forceinline__ void renew(RawBf16& r) { asm volatile("" : "+v"(r.w[0]), "+v"(r.w[1]), "+v"(r.w[2]), "+v"(r.w[3])); }
__device__ __forceinline__ void renew(F8& r)
{
    asm volatile("" : "+v"(r.v[0]), "+v"(r.v[1]), "+v"(r.v[2]), "+v"(r.v[3]), "+v"(r.v[4]), "+v"(r.v[5]), "+v"(r.v[6]), "+v"(r.v[7]));
}
__device__ __forceinline__ void renew(Codes8& c) { asm volatile("" : "+v"(c.w[0]), "+v"(c.w[1])); }

// What was loaded before is loaded again behind this, not kept: registers are short, and parameters near.
__device__ __forceinline__ void forget() { asm volatile("" ::: "memory"); }

// Lanes and vectors a lane of a team.
struct TeamShape {
    uint32_t lanes;
    int v;
};

inline uint32_t lanes_for(int64_t vectors)
{
    for (uint32_t l = 8; l < 64; l *= 2)
        if (vectors <= l) return l;
    return (uint32_t)((vectors + 63) / 64 * 64);
}

// Teams of a workgroup, raised to whole waves.
inline uint32_t whole_waves(uint32_t teams, uint32_t lanes)
{
    const uint32_t per = lanes < 64 ? 64 / lanes : 1;
    return (teams + per - 1) / per * per;
}

inline NormArgs norm_args(const ResidualNormParams& p, const TeamShape& shape)
{
    NormArgs g{};
    g.x = p.x; g.u = p.u; g.h = p.h; g.y = p.y;
    g.pre_weight = p.pre_weight; g.pre_bias = p.pre_bias; g.post_weight = p.post_weight; g.post_bias = p.post_bias; g.gate = p.gate;
    g.y_codes = p.y_codes; g.y_scales = p.y_scales;
    g.h8 = p.h8; g.h8_scales = p.h8_scales; g.u8 = p.u8; g.u8_scales = p.u8_scales;
    g.stats = reinterpret_cast<float4*>(p.stats);
    g.rows = p.rows; g.ldx = p.ldx; g.ldu = p.ldu; g.ldh = p.ldh; g.ldy = p.ldy; g.ld_gate = p.ld_gate;
    g.gate_run = p.gate != nullptr && p.gate_rows > 0 ? p.rows / p.gate_rows : p.rows;
    g.gate_by_row = p.gate != nullptr && p.gate_rows > 1;
    g.cols = (uint32_t)p.cols; g.pitch8 = (uint32_t)((p.cols + 31) / 32 * 32);
    g.lanes = shape.lanes;
    g.inv_cols = (float)(1.0 / (double)p.cols);
    g.rho = p.residual_scale; g.sigma = p.branch_scale; g.eps = p.eps;
    g.layer = p.layer; g.post = p.post;
    g.in_place = p.h != nullptr && p.h == p.x;
    g.param_bf16 = p.param_bf16; g.gate_bf16 = p.gate_bf16; g.floor_mode = p.floor_mode;
    return g;
}

// Calls f with the element types of the stream and the branch.
template <typename F>
void by_types(bool x_bf16, bool u_bf16, F&& f)
{
    if (x_bf16) f(uint16_t{}, uint16_t{});
    else if (u_bf16) f(float{}, uint16_t{});
    else f(float{}, float{});
}

// Calls f with a truth value, with what a kernel is compiled for (post-norm, gate, how rows end), or with a number of vectors, as types.
template <typename F>
void by_flag(bool a, F&& f) { a ? f(std::true_type{}) : f(std::false_type{}); }
inline RowEnd row_end(int64_t cols) { return cols < 8 ? ROW_SHORT : cols % 8 != 0 ? ROW_ENDS : ROW_WHOLE; }
template <RowEnd END> using Ends = std::integral_constant<RowEnd, END>;
template <typename F>
void by_kind(RowEnd end, bool post, bool gate, F&& f)
{
    using Y = std::true_type;
    using N = std::false_type;
    // rows that do not end with a whole vector have one kernel for all kinds
    if (end == ROW_SHORT)     f(Y{}, Y{}, Ends<ROW_SHORT>{});
    else if (end == ROW_ENDS) f(Y{}, Y{}, Ends<ROW_ENDS>{});
    else if (post)            gate ? f(Y{}, Y{}, Ends<ROW_WHOLE>{}) : f(Y{}, N{}, Ends<ROW_WHOLE>{});
    else                      gate ? f(N{}, Y{}, Ends<ROW_WHOLE>{}) : f(N{}, N{}, Ends<ROW_WHOLE>{});
}
template <typename F>
void by_vectors(int v, F&& f)
{
    if (v == 1)      f(std::integral_constant<int, 1>{});
    else if (v == 2) f(std::integral_constant<int, 2>{});
    else if (v == 3) f(std::integral_constant<int, 3>{});
    else             f(std::integral_constant<int, 4>{});
}

// Whether one descriptor covers so many rows of a matrix.
inline bool covers(const void* p, bool bf16, int64_t ld, int64_t rows)
{
    return p == nullptr || rows <= OFF_MAX / (bf16 ? 2 : 4) / std::max<int64_t>(1, ld) - 1;
}

// The rows that a workgroup's teams reach over at a time.
inline int64_t rows_at_once(bool runs, uint32_t lanes, uint32_t grid, uint32_t teams, int64_t team_rows)
{
    return TeamRows::spread(runs, lanes) ? (int64_t)grid * teams : (teams + 1) * (runs ? team_rows : 1);
}

// Where rows lie so far apart that one does not cover those of a workgroup, each team is a workgroup of its own.
inline TeamShape one_team(const TeamShape& s, int64_t cols) { return s.lanes >= 64 ? s : TeamShape{64, (int)((cols + 511) / 512)}; }

// Bytes of LDS that the parameters of a kernel take (the ParamLds of its kind), and gate rows of the teams' own.
inline size_t param_bytes(const TeamShape& s, RowEnd end, bool post, bool gate, bool layer, bool backward, uint32_t own_gates)
{
    size_t words = 0;
    by_kind(end, post, gate, [&](auto p, auto g, auto) {
        by_flag(layer, [&](auto l) {
            by_flag(backward, [&](auto b) { words = ParamLds<decltype(p)::value, decltype(g)::value, decltype(l)::value, decltype(b)::value>::STRIDE; });
        });
    });
    return (words + (size_t)own_gates * 12) * s.lanes * s.v * sizeof(float);
}

// Gives planes to the parameters that a kernel reads, in the order of `wanted`, and returns their bytes.
inline size_t give_planes(NormArgs& g, const TeamShape& s, std::initializer_list<std::pair<NormParam, bool>> wanted)
{
    const size_t bytes = (size_t)s.lanes * s.v * 16;
    size_t planes = 0;
    for (uint8_t& p : g.plane) p = ParamPlanes::NO_PLANE;
    for (const auto& [which, there] : wanted) {
        const size_t n = (which == P_GATE ? g.gate_bf16 : g.param_bf16) ? 1 : 2;
        if (!there || (planes + n) * bytes > NORM_LDS_MAX) continue;
        g.plane[which] = (uint8_t)planes;
        planes += n;
    }
    return planes * bytes;
}

// Starts a kernel with `lds` bytes, asking for more than a kernel may have by itself where need be.
template <typename K, typename A>
hipError_t start_norm(K kernel, dim3 grid, uint32_t threads, size_t lds, hipStream_t st, const A& args)
{
    if (lds > 65536 - sizeof(TeamScratch)) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    kernel<<<grid, threads, lds, st>>>(args);
    return hipGetLastError();
}

// The backward kernels by norm (a file each).
hipError_t launch_norm_bwd_rms(const NormGradArgs& a, bool x_bf16, bool u_bf16, bool eight, RowEnd end, int v, BwdPart part, dim3 grid, uint32_t threads, size_t lds, hipStream_t st);
hipError_t launch_norm_bwd_layer(const NormGradArgs& a, bool x_bf16, bool u_bf16, bool eight, RowEnd end, int v, BwdPart part, dim3 grid, uint32_t threads, size_t lds, hipStream_t st);

}  // namespace mxl
