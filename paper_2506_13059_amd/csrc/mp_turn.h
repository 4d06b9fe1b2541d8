// Turning rows to their positions: device code of mp_rotary.hip and mp_norm_rotary.hip, which say what is computed.
#pragma once
#include "mp_device.h"
#include "mp_paged.h"

namespace mp {

namespace {

constexpr double kTurn = 0.15915494309189533577;      // 1 / (2 pi)

__device__ __forceinline__ float2 cos_sin(double position, double freq, float amplitude)
{
    double turns = position * freq * kTurn;
    turns -= __builtin_rint(turns);
    float s, c;
    sincospif(2.f * (float)turns, &s, &c);
    return make_float2(c * amplitude, s * amplitude);
}

// What a lane needs to turn its dims [8 c, 8 c + 8) of a row, c = lane & 15.
struct Turn {
    float cs[8], sn[8];          // of its dims (interleaved: of its pairs, twice each); sn with the sign of the partner's share
    int partner;                 // half layout: lane of the row with the partner dims
    int n;                       // how many of the dims are turned
};

// table: cosine and sine of every pair, in LDS
__device__ __forceinline__ Turn load_turn(const float2* table, const Rotation& rot)
{
    Turn t;
    const int c = threadIdx.x & 15, half = rot.rot_dim >> 1;
    t.partner = c;
    t.n = min(max(rot.rot_dim - 8 * c, 0), 8);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int d = 8 * c + i;
        const bool in = d < rot.rot_dim;
        const int pair = rot.interleaved ? d >> 1 : d < half ? d : d - half;
        const bool first = rot.interleaved ? (d & 1) == 0 : d < half;
        const float2 v = in ? table[pair] : make_float2(1.f, 0.f);
        t.cs[i] = v.x;
        t.sn[i] = first ? -v.y : v.y;
    }
    if (!rot.interleaved && 8 * c < rot.rot_dim) t.partner = 8 * c < half ? c + (half >> 3) : c - (half >> 3);
    return t;
}

__device__ __forceinline__ void unpack(const uint4& w, float (&x)[8])
{
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = bf16lo_to_f32(u[i]);
        x[2 * i + 1] = bf16hi_to_f32(u[i]);
    }
}

__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    return (uint32_t)f32_to_bf16_rne(a) | ((uint32_t)f32_to_bf16_rne(b) << 16);
}

// The partner elements of a lane's eight.  All 64 lanes take part.
__device__ __forceinline__ void partners(const uint4& w, const Turn& t, const Rotation& rot, float (&y)[8])
{
    if (rot.interleaved) {
        float x[8];
        unpack(w, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = x[i ^ 1];
        return;
    }
    const int row = threadIdx.x & 48;
    if ((rot.rot_dim & 15) == 0) {
        uint4 p;
        p.x = __shfl(w.x, row + t.partner, 64);
        p.y = __shfl(w.y, row + t.partner, 64);
        p.z = __shfl(w.z, row + t.partner, 64);
        p.w = __shfl(w.w, row + t.partner, 64);
        unpack(p, y);
        return;
    }
    // (a half of the pairs that is no multiple of eight dims: element by element)
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
    const int c = threadIdx.x & 15, half = rot.rot_dim >> 1;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int d = 8 * c + i;
        const int e = d >= rot.rot_dim ? d : d < half ? d + half : d - half;
        uint32_t word[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) word[k] = __shfl(u[k], row + (e >> 3), 64);
        const uint32_t v = (e & 4) ? ((e & 2) ? word[3] : word[2]) : ((e & 2) ? word[1] : word[0]);
        y[i] = (e & 1) ? bf16hi_to_f32(v) : bf16lo_to_f32(v);
    }
}

// (dims that are not turned keep their bits: no 0 * inf, and no NaN made another one)
__device__ __forceinline__ uint4 turned(const uint4& w, const float (&y)[8], const Turn& t)
{
    float x[8];
    unpack(w, x);
    uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {        // (rot_dim is even: both dims of a word, or neither)
        const uint32_t r = pack2(fmaf(y[2 * i], t.sn[2 * i], x[2 * i] * t.cs[2 * i]), fmaf(y[2 * i + 1], t.sn[2 * i + 1], x[2 * i + 1] * t.cs[2 * i + 1]));
        u[i] = 2 * i < t.n ? r : u[i];
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
}

// Cosines and sines of one position for a wave, in its part of LDS.
__device__ __forceinline__ void fill_table(float2* table, const Rotation& rot, int position)
{
    const int lane = threadIdx.x & 63;
    if (lane < (rot.rot_dim >> 1)) table[lane] = cos_sin(position, rot.freqs[lane], rot.amplitude);
    wave_lds_sync();
}

constexpr int kWaves = 4;
constexpr int kDeep = 4;           // groups of four rows whose loads are on their way together

// kOnce: the results are more than the caches hold by the time someone wants them, and go past them (non-temporal).
template <bool kOnce>
__device__ __forceinline__ void store16(uint4* p, const uint4& v)
{
    if constexpr (kOnce) store_once(p, v);
    else *p = v;
}

// Rows a wave takes of a token's `total`: four where there are few tokens (a wave's rows follow one another), all where the chip is full
// of waves anyway and the angles of a token are worth working out once.
int rows_of_a_wave(int n_tokens, int total)
{
    int rows = 4;
    while (rows < total && (long long)n_tokens * ((total + rows - 1) / rows) > 8192) rows *= 2;
    return rows;
}

// Results of more than 64 MiB go past the caches.  Us with and without, the same tensors again and again: five prompts' append (486 MB moved) 76 and 100, gather with lookup keys
// (336 MB) 57 and 77, (2.7 GB) 499 and 519; a prompt's queries (84 MB written) 28.4 and 28.9.
bool past_caches(long long rows) { return rows * 256 > 64ll << 20; }

}  // namespace
}  // namespace mp
