// Rotary positions, and the paged cache of keys and values: append (with rotation of the keys) and read back.
//
// All three are bound by HBM (by a launch and a memory latency or two for the tokens of one decode step): every element is read and
// written once, in 16-byte accesses where its neighbours are in the same thread.  Measured: rotary 8192 tokens of 40 bf16 heads of 128, 30 us,
// 5.6 TB/s; append 4096 tokens of 8 heads of 128 from bf16 to fp8, 10 us, 2.5 TB/s, and 16384 of them read back, 23 us, 4.4 TB/s; a decode
// step (16 tokens, 8 heads, int8, keys rotated) 4.9 us, 16 tokens read back 4.6 us; 5 tokens rotated 3.5 us.
#include <math.h>

#include "attn_internal.h"

namespace mmoe {

// Eight consecutive elements as fp32.
template <bool F32>
__device__ __forceinline__ void load8(const char* p, float* x)
{
    if constexpr (F32) {
        const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
    } else {
        const u32x4 a = *(const u32x4*)p;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[2 * i] = bf16_lo(a[i]), x[2 * i + 1] = bf16_hi(a[i]);
    }
}
template <bool F32>
__device__ __forceinline__ void store8(char* p, const float* x)
{
    if constexpr (F32) {
        *(f32x4*)p = f32x4{x[0], x[1], x[2], x[3]};
        *(f32x4*)(p + 16) = f32x4{x[4], x[5], x[6], x[7]};
    } else {
        *(u32x4*)p = u32x4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
    }
}

// A unit is 16 elements of a head: two runs of 8.  Units below rot/16 hold 8 pairs: runs 8u and rot/2 + 8u (halves), or the 16
// elements from 16u on (neighbours); the units behind them are the elements that are copied.
struct UnitPlace {
    int a, b;  // first elements of the runs
};
template <bool HALVES>
__device__ __forceinline__ UnitPlace unit_place(int u, int rot)
{
    if (HALVES && u < rot / 16) return {8 * u, rot / 2 + 8 * u};
    return {16 * u, 16 * u + 8};
}

// (The angle's error is 2^-26 turn, the rounding to fp32, at any position, and 2^-55 of a turn for each position, the steps': a product in fp32 would
// be off by whole turns from 2^24 on.)
// Cosine and sine of pairs 8u .. 8u+7 at a position, times m.  steps: turns per position in units of 2^-64; the product's
// overflow is whole turns.  The upper 32 bits, as a signed number, are the angle in [-1/2, 1/2) turn.
__device__ __forceinline__ void turn_of(const uint64_t* __restrict__ steps, int pos, float m, float sign, float* c, float* s)
{
#pragma clang fp contract(off)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint64_t turns = steps[i] * (uint64_t)(int64_t)pos;
        const float half_turns = (float)(int32_t)(turns >> 32) * 0x1p-31f;
        float sn, cs;
        sincospif(half_turns, &sn, &cs);
        c[i] = cs * m;
        s[i] = sn * (m * sign);
    }
}

template <bool HALVES>
__device__ __forceinline__ void rotate(float* x, const float* c, const float* s)
{
#pragma clang fp contract(off)  // the same bits from every kernel that rotates
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int p = HALVES ? i : 2 * i, q = HALVES ? 8 + i : 2 * i + 1;
        const float a = x[p], b = x[q];
        x[p] = __builtin_fmaf(a, c[i], -(b * s[i]));
        x[q] = __builtin_fmaf(a, s[i], b * c[i]);
    }
}

// A wavefront takes a share of the heads of one token.  Lane l holds unit l mod U of head l / U, then of the heads that follow in
// steps of what the wavefronts of the token cover, so its sines are made once.
template <bool F32, bool HALVES>
__global__ __launch_bounds__(256) void rotary_kernel(const char* X, const int32_t* __restrict__ pos, const uint64_t* __restrict__ steps,
                                                     char* Y, int T, int heads, int D, int rot, int waves, float m, float sign,
                                                     int64_t xt, int64_t xh, int64_t yt, int64_t yh, bool in_place)
{
    constexpr int kEsz = F32 ? 4 : 2;
    const int64_t wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int t = (int)(wave / waves), part = (int)(wave % waves);
    if (t >= T) return;
    const int lane = threadIdx.x & 63, U = D / 16, across = 64 / U;
    if (lane >= across * U) return;
    const int u = lane % U;
    const bool turns = u < rot / 16;
    if (!turns && in_place) return;
    float c[8], s[8];
    if (turns) turn_of(steps + 8 * u, pos[t], m, sign, c, s);
    const UnitPlace at = unit_place<HALVES>(u, rot);
    for (int h = part * across + lane / U; h < heads; h += waves * across) {
        const char* x = X + (t * xt + h * xh) * kEsz;
        char* y = Y + (t * yt + h * yh) * kEsz;
        float v[16];
        load8<F32>(x + at.a * kEsz, v);
        load8<F32>(x + at.b * kEsz, v + 8);
        if (turns) rotate<HALVES>(v, c, s);
        store8<F32>(y + at.a * kEsz, v);
        store8<F32>(y + at.b * kEsz, v + 8);
    }
}

int launch_rotary(const mmoe_rotary_shape& s, const void* X, const int32_t* pos, const uint64_t* steps, void* Y, hipStream_t st)
{
    const int across = 64 / (s.head_dim / 16);
    const int most = (s.heads + across - 1) / across;
    // About 4096 wavefronts: fewer leave compute units idle, more make the same sines again.  us, with one to a token, this rule, one to every
    // `across` heads (48 heads of 128): 64 tokens 5.4, 3.5, 3.5; 512 6.2, 5.3, 5.3; 1024 6.8, 6.9, 7.9; 2048 10.1, 9.9, 12.4; 8192 33.3, 33.3, 37.3.
    const int waves = s.T * (int64_t)most <= 4096 ? most : s.T < 4096 ? 4096 / s.T : 1;
    const int64_t xh = s.x_head ? s.x_head : s.head_dim, xt = s.x_token ? s.x_token : (int64_t)s.heads * s.head_dim;
    const int64_t yh = s.y_head ? s.y_head : s.head_dim, yt = s.y_token ? s.y_token : (int64_t)s.heads * s.head_dim;
    const dim3 grid((unsigned)(((int64_t)s.T * waves + 3) / 4)), block(256);
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, block, 0, st, (const char*)X, pos, steps, (char*)Y, s.T, s.heads, s.head_dim, s.rot, waves,
                           s.magnitude, s.transpose ? -1.0f : 1.0f, xt, xh, yt, yh, X == Y && xt == yt && xh == yh);
    };
    const bool halves = s.layout == MMOE_ROTARY_HALVES;
    if (s.dtype == MMOE_F32) halves ? go(rotary_kernel<true, true>) : go(rotary_kernel<true, false>);
    else halves ? go(rotary_kernel<false, true>) : go(rotary_kernel<false, false>);
    return launch_status();
}

// ---- cache --------------------------------------------------------------------------------------------
// What a page holds (the layout is in mmoe.h).  E elements to a piece of 16 bytes.
template <int FORMAT, bool F32>
struct Kept {
    static constexpr bool kPlain = FORMAT == MMOE_CACHE_PLAIN;
    static constexpr int kBytes = kPlain ? (F32 ? 4 : 2) : 1;  // of an element
    static constexpr int E = 16 / kBytes;
    __device__ static int k_at(int r, int d, int D) { return ((((r >> 4) * (D / (4 * E)) + d / (4 * E)) * 64) + (d % (4 * E)) / E * 16 + (r & 15)) * E + d % E; }
    __device__ static int v_at(int r, int d)
    {
        const int j = (r >> 4) * 4 + (r & 3);
        return (((d >> 4) * (16 / E) + j / E) * 64 + ((r & 15) >> 2) * 16 + (d & 15)) * E + j % E;
    }
};

constexpr float kTop[3] = {0.0f, 127.0f, 448.0f};
constexpr float kLeast = 0x1p-100f;

// Code of one value (bits), and of a code the value.
template <int FORMAT>
__device__ __forceinline__ uint32_t code_of(float x)
{
    if constexpr (FORMAT == MMOE_CACHE_INT8) return (uint32_t)((int)rintf(x) + 128) & 0xFF;
    else return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x, x, 0, false) & 0xFF;
}
template <int FORMAT>
__device__ __forceinline__ float value_of(uint32_t code)
{
    if constexpr (FORMAT == MMOE_CACHE_INT8) return (float)((int)code - 128);
    else return __builtin_amdgcn_cvt_f32_fp8((int)code, 0);
}

struct AppendArgs {
    const char *K, *V;
    const int32_t* places;
    const int32_t* pos;
    const uint64_t* steps;
    char *k, *v;
    float *k_scale, *v_scale;
    int64_t kt, kh, vt, vh;  // strides
    int T, heads, rot;
    int64_t n_places;
    float m, sign;
};

// A head's 8-bit scale is amax / 127 (448), found between its lanes; a value in fp32 times top / amax is rounded once, to the code.
// A workgroup appends 16 tokens of one head (a value piece holds 16 tokens: fewer would write it twice, more leave compute units
// idle): thread (matrix, token, unit) has 16 elements.  Keys go out from there, two runs of 8 each in one piece; values, whose pieces
// hold several tokens, through LDS, where four tokens in consecutive places become one store.
// ROTATE: 0 no, 1 halves, 2 neighbours.
template <int FORMAT, bool F32, int ROTATE, int D>
__global__ __launch_bounds__(2 * D) void append_kernel(AppendArgs g)
{
    using P = Kept<FORMAT, F32>;
    constexpr int kEsz = F32 ? 4 : 2, kTok = 16;
    constexpr int U = D / 16, kThreads = 2 * kTok * U;
    const int tid = threadIdx.x;
    __shared__ __attribute__((aligned(16))) char codes[kTok * D * P::kBytes];  // [kTok][D] of V
    __shared__ int place[kTok];
    const int t0 = blockIdx.x * kTok, h = blockIdx.y;
    const int which = tid / (kTok * U), tok = tid / U % kTok, u = tid % U;  // which: 0 keys, 1 values
    const int t = min(t0 + tok, g.T - 1);
    const char* src = which ? g.V + (t * g.vt + h * g.vh) * kEsz : g.K + (t * g.kt + h * g.kh) * kEsz;
    const bool turns = ROTATE && which == 0 && u < g.rot / 16;
    const UnitPlace at = ROTATE == 1 && which == 0 ? unit_place<true>(u, g.rot) : unit_place<false>(u, g.rot);
    float x[16];
    load8<F32>(src + at.a * kEsz, x);
    load8<F32>(src + at.b * kEsz, x + 8);
    int p = t0 + tok < g.T ? g.places[t] : -1;
    if (p >= g.n_places) p = -1;
    if (u == 0 && which == 0) place[tok] = p;
    if (turns) {
        float c[8], s[8];
        turn_of(g.steps + 8 * u, g.pos[t], g.m, g.sign, c, s);
        rotate<ROTATE == 1>(x, c, s);
        if constexpr (!F32) {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = bf16_bits_to_f32(f32_to_bf16_bits(x[i]));
        }
    }
    uint32_t code[16];
    if constexpr (!P::kPlain) {
        float a = 0.0f;
        bool odd = false;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            a = fmaxf(a, fabsf(x[i]));
            odd = odd || !(fabsf(x[i]) < INFINITY);
        }
        // over the head's U lanes
        if (odd) a = INFINITY;
        a = fmaxf(a, lane_xor<1>(a));
        a = fmaxf(a, lane_xor<2>(a));
        if constexpr (U >= 8) a = fmaxf(a, lane_xor<4>(a));
        if constexpr (U >= 16) a = fmaxf(a, lane_xor<8>(a));
        const bool fine = a < INFINITY && a >= kLeast;
        const float inv = fine ? kTop[FORMAT] / a : 0.0f;
        const float scale = a < INFINITY ? (fine ? a * (float)(1.0 / (double)kTop[FORMAT]) : 0.0f) : NAN;
#pragma unroll
        for (int i = 0; i < 16; ++i) code[i] = code_of<FORMAT>(fine ? x[i] * inv : 0.0f);
        if (u == 0 && p >= 0) (which ? g.v_scale : g.k_scale)[((int64_t)(p / kPage) * g.heads + h) * kPage + p % kPage] = scale;
    }
    const int64_t block = (int64_t)kPage * D;
    if (which == 0) {
        if (p >= 0) {
            char* k = g.k + ((int64_t)(p / kPage) * g.heads + h) * block * P::kBytes;
            if constexpr (!P::kPlain && ROTATE != 1) {  // 16 codes in a row are a piece
                u32x4 piece;
#pragma unroll
                for (int i = 0; i < 4; ++i) piece[i] = code[4 * i] | code[4 * i + 1] << 8 | code[4 * i + 2] << 16 | code[4 * i + 3] << 24;
                *(u32x4*)(k + (int64_t)P::k_at(p % kPage, 16 * u, D)) = piece;
            } else
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int d = half ? at.b : at.a;
                char* dst = k + (int64_t)P::k_at(p % kPage, d, D) * P::kBytes;
                const float* v = x + 8 * half;
                if constexpr (P::kPlain && F32) {
                    *(f32x4*)dst = f32x4{v[0], v[1], v[2], v[3]};
                    *(f32x4*)(k + (int64_t)P::k_at(p % kPage, d + 4, D) * 4) = f32x4{v[4], v[5], v[6], v[7]};
                } else if constexpr (P::kPlain) {
                    store8<false>(dst, v);
                } else {
                    const uint32_t* q = code + 8 * half;
                    *(u32x2*)dst = u32x2{q[0] | q[1] << 8 | q[2] << 16 | q[3] << 24, q[4] | q[5] << 8 | q[6] << 16 | q[7] << 24};
                }
            }
        }
    } else {
        char* row = codes + (tok * D + 16 * u) * P::kBytes;
        if constexpr (P::kPlain) {
            store8<F32>(row, x);
            store8<F32>(row + 8 * kEsz, x + 8);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                ((uint32_t*)row)[i] = code[4 * i] | code[4 * i + 1] << 8 | code[4 * i + 2] << 16 | code[4 * i + 3] << 24;
        }
    }
    __syncthreads();
    // Four tokens that stand in consecutive places, the first in a multiple of four, are one store for each element; they start at the
    // first token's distance from such a place.
    const int shift = -place[0] & 3;
    for (int i = tid; i < (kTok / 4 + 1) * D; i += kThreads) {
        const int d = i % D, first = (i / D - 1) * 4 + shift;  // token of the group's first place; the group may begin before the tile
        const int next = D * P::kBytes;
        const char* from = codes + (first * D + d) * P::kBytes;
        auto dst = [&](int q) { return g.v + (((int64_t)(q / kPage) * g.heads + h) * block + P::v_at(q % kPage, d)) * P::kBytes; };
        bool whole = first >= 0 && first + 3 < kTok && place[first] >= 0 && (place[first] & 3) == 0;
        if (whole)
#pragma unroll
            for (int j = 1; j < 4; ++j) whole = whole && place[first + j] == place[first] + j;
        if (whole) {
            char* to = dst(place[first]);
            if constexpr (P::kBytes == 1) {
                auto at8 = [&](int j) { return (uint32_t) * (const uint8_t*)(from + j * next); };
                *(uint32_t*)to = at8(0) | at8(1) << 8 | at8(2) << 16 | at8(3) << 24;
            } else if constexpr (P::kBytes == 2) {
                auto at16 = [&](int j) { return (uint32_t) * (const uint16_t*)(from + j * next); };
                *(u32x2*)to = u32x2{at16(0) | at16(1) << 16, at16(2) | at16(3) << 16};
            } else {
                auto at32 = [&](int j) { return *(const uint32_t*)(from + j * next); };
                *(u32x4*)to = u32x4{at32(0), at32(1), at32(2), at32(3)};
            }
        } else {
            for (int j = max(0, -first); j < 4 && first + j < kTok; ++j) {
                if (place[first + j] < 0) continue;
                char* to = dst(place[first + j]);
                if constexpr (P::kBytes == 1) *to = from[j * next];
                else if constexpr (P::kBytes == 2) *(uint16_t*)to = *(const uint16_t*)(from + j * next);
                else *(uint32_t*)to = *(const uint32_t*)(from + j * next);
            }
        }
    }
}

template <int FORMAT, bool F32, int D>
static void append_wide(const mmoe_rotary_shape* rotary, const AppendArgs& g, hipStream_t st)
{
    const dim3 grid((g.T + 15) / 16, g.heads), block(2 * D);
    if (!rotary) hipLaunchKernelGGL((append_kernel<FORMAT, F32, 0, D>), grid, block, 0, st, g);
    else if (rotary->layout == MMOE_ROTARY_HALVES) hipLaunchKernelGGL((append_kernel<FORMAT, F32, 1, D>), grid, block, 0, st, g);
    else hipLaunchKernelGGL((append_kernel<FORMAT, F32, 2, D>), grid, block, 0, st, g);
}

template <int FORMAT, bool F32>
static void append(int D, const mmoe_rotary_shape* rotary, const AppendArgs& g, hipStream_t st)
{
    if (D == 64) append_wide<FORMAT, F32, 64>(rotary, g, st);
    else if (D == 128) append_wide<FORMAT, F32, 128>(rotary, g, st);
    else append_wide<FORMAT, F32, 256>(rotary, g, st);
}

int launch_cache_append(const mmoe_cache_shape& s, const mmoe_cache_rows& rows, const void* K, const void* V, const int32_t* places,
                        const mmoe_rotary_shape* rotary, const int32_t* pos, const uint64_t* steps, const mmoe_cache& cache,
                        hipStream_t st)
{
    const int64_t hd = s.head_dim, td = (int64_t)s.kv_heads * s.head_dim;
    AppendArgs g = {(const char*)K, (const char*)V, places, pos, steps, (char*)cache.k, (char*)cache.v, cache.k_scale, cache.v_scale,
                    rows.k_token ? rows.k_token : td, rows.k_head ? rows.k_head : hd, rows.v_token ? rows.v_token : td,
                    rows.v_head ? rows.v_head : hd, rows.T, s.kv_heads, rotary ? rotary->rot : 0,
                    (int64_t)s.n_pages * kPage, rotary ? rotary->magnitude : 1.0f, rotary && rotary->transpose ? -1.0f : 1.0f};
    const bool f32 = s.dtype == MMOE_F32;
    switch (s.format) {
        case MMOE_CACHE_PLAIN: f32 ? append<MMOE_CACHE_PLAIN, true>(s.head_dim, rotary, g, st) : append<MMOE_CACHE_PLAIN, false>(s.head_dim, rotary, g, st); break;
        case MMOE_CACHE_INT8: f32 ? append<MMOE_CACHE_INT8, true>(s.head_dim, rotary, g, st) : append<MMOE_CACHE_INT8, false>(s.head_dim, rotary, g, st); break;
        default: f32 ? append<MMOE_CACHE_FP8, true>(s.head_dim, rotary, g, st) : append<MMOE_CACHE_FP8, false>(s.head_dim, rotary, g, st); break;
    }
    return launch_status();
}

// A wavefront reads the keys or the values of one head and of `rows` (64, 16 or 4) of the listed places back.  The first of them is
// chosen so that, where the list starts with a run of places, a wavefront's are one page's.
template <int FORMAT, bool F32, int D>
__global__ __launch_bounds__(256) void read_kernel(const char* __restrict__ k, const char* __restrict__ v, const float* __restrict__ ks,
                                                   const float* __restrict__ vs, const int32_t* __restrict__ places,
                                                   char* __restrict__ K, char* __restrict__ V, int R, int heads, int64_t n_places,
                                                   int rows)
{
    using P = Kept<FORMAT, F32>;
    constexpr int kEsz = F32 ? 4 : 2, E = P::E;
    constexpr int DG = D == 64 || F32 ? 4 : 8;  // elements of a row that a lane stores at once: 16 bytes (8 for heads of 64)
    const int lane = threadIdx.x & 63;
    const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int which = (int)(item & 1), h = (int)((item >> 1) % heads);
    const int64_t tile = (item >> 1) / heads;
    const int64_t r0 = tile * rows - (places[0] & (rows - 1));  // first row of the list; rows before 0 and from R on are not there
    if (r0 >= R) return;  // uniform
    const int64_t mine = r0 + lane;
    const bool listed = lane < rows && mine >= 0 && mine < R;
    int p = listed ? places[mine] : -1;
    if (p >= n_places || p < 0) p = -1;
    const uint64_t all = __ballot(listed);
    // values as fp32 from a piece
    auto value = [&](const u32x4& x, int i) {
        if constexpr (P::kPlain && F32) return __uint_as_float(x[i]);
        else if constexpr (P::kPlain) return i & 1 ? bf16_hi(x[i / 2]) : bf16_lo(x[i / 2]);
        else return value_of<FORMAT>((x[i / 4] >> (i % 4 * 8)) & 0xFF);
    };
    if (which == 0) {
        // 16 rows by 4 units of 16 elements at a time: pieces of adjacent rows are neighbours
        constexpr int U = D / 16;
        for (int part = 0; part < 4; ++part) {
            if (!(all >> (part * 16) & 0xFFFF)) continue;  // uniform
            const int row = part * 16 + (lane & 15);
            const int64_t r = r0 + row;
            const int q = __shfl(p, row);
            const bool there = row < rows && r >= 0 && r < R;
            const int64_t ph = (int64_t)(max(q, 0) / kPage) * heads + h;
            const char* base = k + ph * kPage * D * P::kBytes;
            float scale = 1.0f;
            if constexpr (!P::kPlain) scale = q >= 0 ? ks[ph * kPage + q % kPage] : 0.0f;
            for (int u = lane >> 4; u < U; u += 4) {
                float x[16];
#pragma unroll
                for (int i = 0; i < 16 / E; ++i) {
                    const u32x4 piece = *(const u32x4*)(base + (int64_t)P::k_at(max(q, 0) % kPage, 16 * u + i * E, D) * P::kBytes);
#pragma unroll
                    for (int j = 0; j < E; ++j) x[i * E + j] = q >= 0 ? value(piece, j) * scale : 0.0f;
                }
                if (there) {
                    char* out = K + ((r * heads + h) * D + 16 * u) * kEsz;
                    store8<F32>(out, x);
                    store8<F32>(out + 8 * kEsz, x + 8);
                }
            }
        }
        return;
    }
    // Values: runs of places on one page, each read as whole pieces.  Lane (g, c) has the rows 16 q + 4 g + e of the page and D/16
    // elements.
    const int before = __shfl_up(p, 1);
    uint64_t starts = __ballot(listed && (lane == 0 || p < 0 || p != before + 1 || (p & (kPage - 1)) == 0 || mine == 0));
    const int g = lane & 3, c = lane >> 2;
    constexpr int n = D / 16;
    while (starts) {
        const int first = __ffsll((unsigned long long)starts) - 1;
        starts &= starts - 1;
        const int next = starts ? __ffsll((unsigned long long)starts) - 1 : 64 - __clzll((long long)all);
        const int place = __shfl(p, first);                    // uniform
        const int begin = place & (kPage - 1), count = next - first;  // rows begin .. of the page are rows first .. of the tile
        const int64_t ph = (int64_t)(max(place, 0) / kPage) * heads + h;
        const char* base = v + ph * kPage * D * P::kBytes;
        char* out = V + ((r0 + first - begin) * heads + h) * D * kEsz;  // of the page's row 0
        if (place < 0) {
            for (int i = lane; i < count * D; i += 64) {
                char* to = V + (((r0 + first + i / D) * heads + h) * D + i % D) * kEsz;
                if (F32) *(float*)to = 0.0f;
                else *(uint16_t*)to = 0;
            }
            continue;
        }
        f32x4 scale[4];
        if constexpr (!P::kPlain)
#pragma unroll
            for (int q = 0; q < 4; ++q) scale[q] = *(const f32x4*)(vs + ph * kPage + q * 16 + g * 4);
        for (int d0 = c * n; d0 < (c + 1) * n; d0 += DG) {  // DG elements of 16 rows
            u32x4 piece[DG][16 / E];
#pragma unroll
            for (int i = 0; i < DG; ++i)
#pragma unroll
                for (int j = 0; j < 16 / E; ++j)
                    piece[i][j] = *(const u32x4*)(base + ((((int64_t)(d0 + i) >> 4) * (16 / E) + j) * 64 + g * 16 + ((d0 + i) & 15)) * 16);
            each<16>([&](auto atc) {
                constexpr int at = decltype(atc)::value, q = at / 4, e = at % 4;
                const int row = q * 16 + g * 4 + e;
                if (row < begin || row >= begin + count) return;
                float x[DG];
                each<DG>([&](auto i) {
                    x[decltype(i)::value] = value(piece[decltype(i)::value][at / E], at % E);
                    if constexpr (!P::kPlain) x[decltype(i)::value] *= scale[q][e];
                });
                char* to = out + ((int64_t)row * heads * D + d0) * kEsz;
                if constexpr (DG == 8) store8<F32>(to, x);
                else if constexpr (F32) *(f32x4*)to = f32x4{x[0], x[1], x[2], x[3]};
                else *(u32x2*)to = u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
            });
        }
    }
}

template <int FORMAT, bool F32>
static void read_back(const mmoe_cache_shape& s, const mmoe_cache& c, int R, const int32_t* places, void* K, void* V, hipStream_t st)
{
    // Rows to a wavefront: few of a short list, so that its wavefronts wait at the same time.  us, 8 heads of 128 int8, a run of places | places
    // apart, with 64, 16 and 4 rows: 64 listed 5.6, 3.9, 3.9 | 51, 15, 5.8; 256 7.0, 4.1, 4.1 | 52, 15, 5.8; 1024 7.5, 4.6, 7.6 | 59, 19, 14;
    // 4096 9.0, 9.2, 21 | 62, 41, 40; 16384 22.8, 26.1, 72.7 | 195, 187, 175.
    const int64_t all = (int64_t)R * s.kv_heads;
    const int rows = all <= 2048 ? 4 : all <= 16384 ? 16 : 64;
    const int64_t items = ((int64_t)(R + rows - 1) / rows + 1) * s.kv_heads * 2;
    const dim3 grid((unsigned)((items + 3) / 4)), block(256);
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, block, 0, st, (const char*)c.k, (const char*)c.v, c.k_scale, c.v_scale, places, (char*)K, (char*)V,
                           R, s.kv_heads, (int64_t)s.n_pages * kPage, rows);
    };
    if (s.head_dim == 64) go(read_kernel<FORMAT, F32, 64>);
    else if (s.head_dim == 128) go(read_kernel<FORMAT, F32, 128>);
    else go(read_kernel<FORMAT, F32, 256>);
}

int launch_cache_read(const mmoe_cache_shape& s, const mmoe_cache& c, int R, const int32_t* places, void* K, void* V, hipStream_t st)
{
    const bool f32 = s.dtype == MMOE_F32;
    auto go = [&](auto read) { read(s, c, R, places, K, V, st); };
    switch (s.format) {
        case MMOE_CACHE_PLAIN: f32 ? go(read_back<MMOE_CACHE_PLAIN, true>) : go(read_back<MMOE_CACHE_PLAIN, false>); break;
        case MMOE_CACHE_INT8: f32 ? go(read_back<MMOE_CACHE_INT8, true>) : go(read_back<MMOE_CACHE_INT8, false>); break;
        default: f32 ? go(read_back<MMOE_CACHE_FP8, true>) : go(read_back<MMOE_CACHE_FP8, false>); break;
    }
    return launch_status();
}

}  // namespace mmoe
