// Attention of drafted tokens over the paged cache: out[t,h] = sum_j softmax_j(scale <Q[t,h], K[j]>) V[j], in one pass over
// the keys with the running maximum m and sum l of the softmax: at a step with scores s, m' = max(m, s),
// O <- O 2^(m - m') + sum 2^(s - m') V, l likewise (everything in base 2; the scores carry log2 e).
//
// A column is a (token, query head) pair of one request and key head: all that read the same keys.  A wavefront holds 16 NC
// columns.  Keys are the row operand of the first product, so a lane has four consecutive keys of a column per tile of 16, which
// is, with the order in which pages keep values, its part of the column operand of the second: probabilities go
// from one product to the other inside a lane, and keys and values from memory straight into operand registers, 1 KB an
// instruction, no LDS and no barrier in the loop.
#include <math.h>

#include "attn_internal.h"

namespace mmoe {

enum { kBf16 = 0, kInt8 = 1, kFp8 = 2, kF32 = 3 };  // what pages hold

struct AttendArgs {
    const char* Q;
    const int32_t *starts, *ctx;
    const uint64_t* tree;
    const int32_t* pages;
    const char *k, *v;
    const float *k_scale, *v_scale;
    char* out;
    float* lse;
    float* part_o;   // [nsplit][T * heads][D]
    float* part_ml;  // [nsplit][T * heads][2]
    int64_t qt, qh, ot, oh;
    int T, B, heads, kv_heads, G, max_pages, max_drafts, mask_words, n_pages;
    int groups, nsplit, chunk;  // column groups; splits of the keys, pages of each
    float scale;
};

template <int KIND>
__device__ __forceinline__ f32x4 mma_kind(u32x4 a, u32x4 b, f32x4 c)
{
    if constexpr (KIND == kF32) return mma<true>(a, b, c);
    else if constexpr (KIND == kBf16) return mma<false>(a, b, c);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Four codes as fp16.  Int8: 0x6400 | (code + 128) is 1024 + 128 + code; fp8 has an instruction.
template <int KIND>
__device__ __forceinline__ u32x2 widen(uint32_t x)
{
    if constexpr (KIND == kInt8) {
        const f16x2 bias = {(_Float16)1152.0f, (_Float16)1152.0f};
        const f16x2 a = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, x, 0x04010400u)) - bias;
        const f16x2 b = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, x, 0x04030402u)) - bias;
        return u32x2{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
    } else {
        return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 1.0f, false)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 1.0f, true))};
    }
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    const f16x2 h = {(_Float16)lo, (_Float16)hi};
    return __builtin_bit_cast(uint32_t, h);
}

__device__ __forceinline__ float max_groups(float x)  // over the four lane groups
{
    x = fmaxf(x, lane_xor<16>(x));
    return fmaxf(x, lane_xor<32>(x));
}
__device__ __forceinline__ float sum_groups(float x)
{
    x += lane_xor<16>(x);
    return x + lane_xor<32>(x);
}

// 2^x; -infinity gives 0.
__device__ __forceinline__ float pow2(float x) { return __builtin_amdgcn_exp2f(x); }

constexpr int kLiftBits = 14;  // fp16 probabilities are up to 2^14 times their share, which keeps small ones out of the subnormal range

template <int D, int KIND, int NC>
struct AttendPlan {
    static constexpr int kBytes = KIND == kF32 ? 4 : KIND == kBf16 ? 2 : 1;
    static constexpr int E = 16 / kBytes;
    static constexpr bool kCodes = KIND == kInt8 || KIND == kFp8;
    // tiles of 16 keys to a step: a page, or the part of it whose pieces fill the registers
    static constexpr int KT = kCodes ? 4 : D * kBytes <= 256 ? 4 : D * kBytes <= 512 ? 2 : 1;
    static constexpr int NKS = D / (4 * E);            // pieces of a key row that a lane holds
    static constexpr int NV = KT * 4 / E == 0 ? 1 : KT * 4 / E;  // value pieces to 16 elements of a step
    static constexpr int QS = KIND == kF32 ? D / 16 : D / 32;    // query pieces
    static constexpr int DT = D / 16;
};

template <int D, int KIND, int NC, bool COLS>
__global__ __launch_bounds__(256, NC == 1 && D <= 128 ? 2 : 1) void attend_kernel(AttendArgs g)
{
    using L = AttendPlan<D, KIND, NC>;
    constexpr int KT = L::KT, NKS = L::NKS, NV = L::NV, QS = L::QS, DT = L::DT, E = L::E, kSteps = 4 / KT;
    constexpr bool kCodes = L::kCodes;
    constexpr int kEsz = KIND == kF32 ? 4 : 2;  // of Q and out
    const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    int id = blockIdx.x;
    const int cg = id % g.groups;
    id /= g.groups;
    const int h = id % g.kv_heads;
    id /= g.kv_heads;
    const int b = id % g.B, split = id / g.B;
    const int start = g.starts[b], n = min(min(g.starts[b + 1], g.T) - start, g.max_drafts), ctx = g.ctx[b];
    const int C = n * g.G;
    constexpr int kWide = COLS ? 64 * NC : 16 * NC;
    if (start < 0 || cg * kWide >= C || ctx < 0) return;  // uniform
    const int total = (int)min((int64_t)ctx + n, (int64_t)g.max_pages * kPage);
    const int all_pages = (total + kPage - 1) / kPage;
    const int active = min(g.nsplit, max(1, (all_pages + g.chunk - 1) / g.chunk));
    if (split >= active) return;
    const int col0 = cg * kWide + (COLS ? wave * 16 * NC : 0);

    // what the last column of these sees at most
    const int last_token = min(C - 1, cg * kWide + kWide - 1) / g.G;
    const int limit = g.tree ? total : (int)min((int64_t)total, (int64_t)ctx + last_token + 1);
    const int step0 = split * g.chunk * kSteps;
    const int step1 = min(split == active - 1 ? all_pages * kSteps : (split + 1) * g.chunk * kSteps, (limit + 16 * KT - 1) / (16 * KT));

    // ---- queries ----
    u32x4 q[NC][QS];
    float mult[NC];  // of the scores
    int token[NC];   // of the request; n where the column is none
#pragma unroll
    for (int ct = 0; ct < NC; ++ct) {
        const int c = col0 + ct * 16 + lr;
        const bool there = c < C;
        token[ct] = there ? c / g.G : n;
        const char* src = g.Q + ((int64_t)(start + (there ? c / g.G : 0)) * g.qt + (int64_t)(h * g.G + (there ? c % g.G : 0)) * g.qh) * kEsz;
        mult[ct] = g.scale * 1.44269504088896340736f;
#pragma unroll
        for (int s = 0; s < QS; ++s) {
            // codes: two instructions of 32 share a piece of 16 codes
            const int d = kCodes ? (s >> 1) * 64 + lg * 16 + (s & 1) * 8 : s * (KIND == kF32 ? 16 : 32) + lg * (KIND == kF32 ? 4 : 8);
            q[ct][s] = there ? *(const u32x4*)(src + d * kEsz) : u32x4{0, 0, 0, 0};
        }
        if constexpr (kCodes) {  // to fp16, by a power of two that puts the largest at 2^12
            float a = 0.0f;
#pragma unroll
            for (int s = 0; s < QS; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i) a = fmaxf(a, fmaxf(fabsf(bf16_lo(q[ct][s][i])), fabsf(bf16_hi(q[ct][s][i]))));
            a = max_groups(a);
            const int e = a > 0.0f && a < INFINITY ? min(100, 12 - (int)((__float_as_uint(a) >> 23) - 127)) : 0;
            const float up = ldexpf(1.0f, e);
            mult[ct] *= ldexpf(1.0f, -e);
#pragma unroll
            for (int s = 0; s < QS; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i) q[ct][s][i] = pack_f16(bf16_lo(q[ct][s][i]) * up, bf16_hi(q[ct][s][i]) * up);
        }
    }

    f32x4 o[NC][DT];
    float m[NC], l[NC];
#pragma unroll
    for (int ct = 0; ct < NC; ++ct) {
        m[ct] = -INFINITY;
        l[ct] = 0.0f;  // this lane's keys only, until the end
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[ct][dt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    int lift = -126;  // o holds 2^(kLiftBits - lift) times its value (codes): lift is the largest exponent of a value scale so far

    constexpr int64_t kBlock = (int64_t)kPage * D * L::kBytes;
    const int32_t* table = g.pages + (int64_t)b * g.max_pages;
    auto block_of = [&](int step) {  // page and head; negative where there is no such page
        const int p = __builtin_amdgcn_readfirstlane(table[step / kSteps]);
        return (unsigned)p < (unsigned)g.n_pages ? (int64_t)p * g.kv_heads + h : (int64_t)-1;
    };
    u32x4 kf[KT][NKS], vf[DT][NV];
    auto load_k = [&](int64_t block, int step) {
        const char* src = g.k + block * kBlock + (step % kSteps) * (KT * NKS * 1024) + lane * 16;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int s = 0; s < NKS; ++s) kf[kt][s] = *(const u32x4*)(src + (kt * NKS + s) * 1024);
    };
    auto load_v = [&](int64_t block, int step) {
        const char* src = g.v + block * kBlock + (step % kSteps) * (NV * 1024) + lane * 16;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int i = 0; i < NV; ++i) vf[dt][i] = *(const u32x4*)(src + (dt * (16 / E) + i) * 1024);
    };

    // One step: keys 16 KT step .. of the request.  TAIL: not all of them are committed keys.
    auto work = [&](auto tailc, int64_t block, int step, auto&& between) {
        constexpr bool TAIL = decltype(tailc)::value;
        const int key0 = step * 16 * KT;
        f32x4 s[NC][KT];
#pragma unroll
        for (int ct = 0; ct < NC; ++ct)
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) s[ct][kt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int i = 0; i < NKS; ++i) {
                if constexpr (kCodes) {
                    const u32x2 a = widen<KIND>(kf[kt][i][0]), c = widen<KIND>(kf[kt][i][1]);
                    const u32x2 d = widen<KIND>(kf[kt][i][2]), e = widen<KIND>(kf[kt][i][3]);
                    const u32x4 lo = {a[0], a[1], c[0], c[1]}, hi = {d[0], d[1], e[0], e[1]};
#pragma unroll
                    for (int ct = 0; ct < NC; ++ct) {
                        s[ct][kt] = mma_kind<KIND>(lo, q[ct][2 * i], s[ct][kt]);
                        s[ct][kt] = mma_kind<KIND>(hi, q[ct][2 * i + 1], s[ct][kt]);
                    }
                } else {
#pragma unroll
                    for (int ct = 0; ct < NC; ++ct) s[ct][kt] = mma_kind<KIND>(kf[kt][i], q[ct][i], s[ct][kt]);
                }
            }
        between();
        f32x4 ks[KT], vs[KT];
        if constexpr (kCodes) {
            const int64_t at = block * kPage + lg * 4;
            float most = 0.0f;
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
                ks[kt] = *(const f32x4*)(g.k_scale + at + kt * 16);
                vs[kt] = *(const f32x4*)(g.v_scale + at + kt * 16);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (TAIL && key0 + kt * 16 + lg * 4 + e >= total) vs[kt][e] = 0.0f;
                    most = fmaxf(most, vs[kt][e]);
                }
            }
            most = max_groups(most);
            // exponent above the largest: scale * 2^-here < 1
            const int here = __builtin_amdgcn_readfirstlane((int)(__float_as_uint(most) >> 23) - 126);
            const int next = max(lift, min(here, 127));
            if (next != lift) {
                const float down = ldexpf(1.0f, max(lift - next, -140));
#pragma unroll
                for (int ct = 0; ct < NC; ++ct)
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) o[ct][dt] *= down;
                lift = next;
            }
            const float up = ldexpf(1.0f, kLiftBits - lift);
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) vs[kt] *= up;
        }
        u32x4 p[NC][KT * 4 / (KIND == kF32 ? 4 : 8)];
        u32x4 seen_p[NC][KT * 4 / (KIND == kF32 ? 4 : 8)];  // 1 where the column sees the key (tail of plain pages)
#pragma unroll
        for (int ct = 0; ct < NC; ++ct) {
            uint64_t vis = ~(uint64_t)0;  // keys of the page that the column sees
            if constexpr (TAIL) {
                const int page0 = key0 & ~(kPage - 1), d0 = page0 - ctx;  // first key of the page, as a drafted token
                const int i = token[ct];
                auto committed_and = [&](uint64_t drafted) {  // bits of the page below ctx, and above them those given from bit max(0,-d0) on
                    return d0 >= 0 ? drafted : d0 <= -kPage ? ~(uint64_t)0 : (((uint64_t)1 << -d0) - 1) | drafted << -d0;
                };
                const int from = max(d0, 0);  // first drafted token of the page
                uint64_t bits = 0;
                if (i < n && from < n) {
                    if (g.tree) {
                        const uint64_t* row = g.tree + (int64_t)(start + i) * g.mask_words;
                        const int w = from >> 6, r = from & 63;
                        if (w < g.mask_words) bits = row[w] >> r;
                        if (r && w + 1 < g.mask_words) bits |= row[w + 1] << (64 - r);
                    } else {
                        const int c = i + 1 - from;
                        bits = c <= 0 ? 0 : c >= 64 ? ~(uint64_t)0 : ((uint64_t)1 << c) - 1;
                    }
                    if (n - from < 64) bits &= ((uint64_t)1 << (n - from)) - 1;
                }
                vis = committed_and(bits);
                if (total - page0 < 64) vis &= total > page0 ? ((uint64_t)1 << (total - page0)) - 1 : 0;
                if (i >= n) vis = 0;
                vis >>= key0 - page0;
            }
            auto sees = [&](int kt, int e) { return !TAIL || (vis >> (kt * 16 + lg * 4 + e) & 1); };
            float top = m[ct];
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float x = s[ct][kt][e] * mult[ct];
                    if constexpr (kCodes) x *= ks[kt][e];
                    if (!sees(kt, e)) x = -INFINITY;
                    s[ct][kt][e] = x;
                    top = fmaxf(top, x);
                }
            top = max_groups(top);
            const float base = top == -INFINITY ? 0.0f : top;
            const float alpha = pow2(m[ct] - base);
            m[ct] = top;
            float sum = 0.0f;
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = pow2(s[ct][kt][e] - base);
                    sum += x;
                    s[ct][kt][e] = kCodes ? (sees(kt, e) ? x * vs[kt][e] : 0.0f) : x;
                }
            l[ct] = l[ct] * alpha + sum;
            if (__any(alpha != 1.0f)) {
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) o[ct][dt] *= alpha;
            }
            // tiles to operand pieces: 16-bit ones hold two tiles' keys
            if constexpr (KIND == kF32) {
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) p[ct][kt] = __builtin_bit_cast(u32x4, s[ct][kt]);
            } else {
#pragma unroll
                for (int i = 0; i < KT / 2; ++i)
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const f32x4& x = s[ct][2 * i + w / 2];
                        p[ct][i][w] = kCodes ? pack_f16(x[(w & 1) * 2], x[(w & 1) * 2 + 1]) : pack_bf16(x[(w & 1) * 2], x[(w & 1) * 2 + 1]);
                    }
            }
            if constexpr (TAIL && !kCodes) {
                if constexpr (KIND == kF32) {
#pragma unroll
                    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) seen_p[ct][kt][e] = sees(kt, e) ? 0x3F800000u : 0u;
                } else {
#pragma unroll
                    for (int i = 0; i < KT / 2; ++i)
#pragma unroll
                        for (int w = 0; w < 4; ++w)
                            seen_p[ct][i][w] = (sees(2 * i + w / 2, (w & 1) * 2) ? 0x3F80u : 0u) | (sees(2 * i + w / 2, (w & 1) * 2 + 1) ? 0x3F800000u : 0u);
                }
            }
        }
        // Values of rows past the end may be anything: zeros.  (Int8 codes are finite whatever they are.)
        auto row_there = [&](int kt, int e) { return key0 + kt * 16 + lg * 4 + e < total; };
        bool odd = false;  // a value that is not finite, of a key that some columns may not see
        if constexpr (TAIL && !kCodes) {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        uint32_t x = vf[dt][i][w];
                        if constexpr (KIND == kF32) {
                            if (!row_there(i, w)) x = 0;
                            odd = odd || (x & 0x7F800000u) == 0x7F800000u;
                        } else {
                            if (!row_there(2 * i + w / 2, (w & 1) * 2)) x &= 0xFFFF0000u;
                            if (!row_there(2 * i + w / 2, (w & 1) * 2 + 1)) x &= 0xFFFFu;
                            odd = odd || (x & 0x7F80u) == 0x7F80u || (x & 0x7F800000u) == 0x7F800000u;
                        }
                        vf[dt][i][w] = x;
                    }
            // 0 times what is not finite would reach columns that do not see the key: such values are taken out, and
            // counted per kind with the columns that do see them.
            if (__any(odd)) {
                for (int kind = 0; kind < 3; ++kind) {  // +infinity, -infinity, NaN
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) {
                        f32x4 count[NC];
#pragma unroll
                        for (int ct = 0; ct < NC; ++ct) count[ct] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                        for (int i = 0; i < NV; ++i) {
                            u32x4 mark;
#pragma unroll
                            for (int w = 0; w < 4; ++w) {
                                auto is = [&](uint32_t bits) {  // fp32 bits
                                    return kind == 0 ? bits == 0x7F800000u : kind == 1 ? bits == 0xFF800000u : (bits & 0x7FFFFFFFu) > 0x7F800000u;
                                };
                                const uint32_t x = vf[dt][i][w];
                                if constexpr (KIND == kF32) mark[w] = is(x) ? 0x3F800000u : 0u;
                                else mark[w] = (is(x << 16) ? 0x3F80u : 0u) | (is(x & 0xFFFF0000u) ? 0x3F800000u : 0u);
                            }
#pragma unroll
                            for (int ct = 0; ct < NC; ++ct) count[ct] = mma_kind<KIND>(mark, seen_p[ct][i], count[ct]);
                        }
#pragma unroll
                        for (int ct = 0; ct < NC; ++ct)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (count[ct][e] > 0.0f) o[ct][dt][e] += kind == 0 ? INFINITY : kind == 1 ? -INFINITY : NAN;
                    }
                }
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                    for (int i = 0; i < NV; ++i)
#pragma unroll
                        for (int w = 0; w < 4; ++w) {
                            uint32_t x = vf[dt][i][w];
                            if constexpr (KIND == kF32) {
                                if ((x & 0x7F800000u) == 0x7F800000u) x = 0;
                            } else {
                                if ((x & 0x7F80u) == 0x7F80u) x &= 0xFFFF0000u;
                                if ((x & 0x7F800000u) == 0x7F800000u) x &= 0xFFFFu;
                            }
                            vf[dt][i][w] = x;
                        }
            }
        }
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
            if constexpr (kCodes) {
                u32x4 x = vf[dt][0];
                if constexpr (TAIL && KIND == kFp8) {  // codes of rows past the end may be NaN
#pragma unroll
                    for (int w = 0; w < 4; ++w)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (!row_there(w, e)) x[w] &= ~(0xFFu << 8 * e);
                }
                const u32x2 a = widen<KIND>(x[0]), c = widen<KIND>(x[1]), d = widen<KIND>(x[2]), e = widen<KIND>(x[3]);
                const u32x4 lo = {a[0], a[1], c[0], c[1]}, hi = {d[0], d[1], e[0], e[1]};
#pragma unroll
                for (int ct = 0; ct < NC; ++ct) {
                    o[ct][dt] = mma_kind<KIND>(lo, p[ct][0], o[ct][dt]);
                    o[ct][dt] = mma_kind<KIND>(hi, p[ct][1], o[ct][dt]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int ct = 0; ct < NC; ++ct) o[ct][dt] = mma_kind<KIND>(vf[dt][i], p[ct][i], o[ct][dt]);
            }
        }
    };

    constexpr int kStride = COLS ? 1 : 4;
    int step = step0 + (COLS ? 0 : wave);
    if (step < step1 && (!COLS || col0 < C)) {  // uniform over the wavefront
        int64_t block = block_of(step);
        if (block >= 0) load_k(block, step);
        while (step < step1) {
            const int next = step + kStride;
            int64_t next_block = -1;
            if (next < step1) next_block = block_of(next);
            auto ahead = [&]() {
                if (next_block >= 0) load_k(next_block, next);
            };
            if (block >= 0) {
                load_v(block, step);
                if ((step + 1) * 16 * KT > ctx) work(std::true_type{}, block, step, ahead);
                else work(std::false_type{}, block, step, ahead);
            } else {
                ahead();
            }
            step = next;
            block = next_block;
        }
    }

    // ---- results ----
    if constexpr (kCodes) {
        const float down = ldexpf(1.0f, max(lift - kLiftBits, -140));
#pragma unroll
        for (int ct = 0; ct < NC; ++ct)
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[ct][dt] *= down;
    }
#pragma unroll
    for (int ct = 0; ct < NC; ++ct) l[ct] = sum_groups(l[ct]);

    const bool direct = g.nsplit == 1;
    auto put = [&](int c, int d, f32x4 x, float total_l) {  // four consecutive elements of column c
        const int64_t t = start + c / g.G, head = h * g.G + c % g.G;
        if (!direct) {
            *(f32x4*)(g.part_o + (((int64_t)split * g.T + t) * g.heads + head) * D + d) = x;
            return;
        }
        const float r = total_l != 0.0f ? 1.0f / total_l : 0.0f;
        char* dst = g.out + (t * g.ot + head * g.oh + d) * kEsz;
        if constexpr (KIND == kF32) *(f32x4*)dst = x * r;
        else *(u32x2*)dst = u32x2{pack_bf16(x[0] * r, x[1] * r), pack_bf16(x[2] * r, x[3] * r)};
    };
    auto put_sums = [&](int c, float mm, float ll) {
        const int64_t t = start + c / g.G, head = h * g.G + c % g.G;
        if (!direct) {
            float* ml = g.part_ml + (((int64_t)split * g.T + t) * g.heads + head) * 2;
            ml[0] = mm;
            ml[1] = ll;
        } else if (g.lse) {
            g.lse[t * g.heads + head] = ll == 0.0f ? -INFINITY : (mm + __log2f(ll)) * 0.693147180559945309417f;
        }
    };
    if constexpr (COLS) {
#pragma unroll
        for (int ct = 0; ct < NC; ++ct) {
            const int c = col0 + ct * 16 + lr;
            if (c >= C) continue;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) put(c, dt * 16 + lg * 4, o[ct][dt], l[ct]);
            if (lg == 0) put_sums(c, m[ct], l[ct]);
        }
    } else {
        // The four wavefronts had different keys: join them, 32 elements of the columns at a time.
        constexpr int kRow = 36;
        __shared__ __attribute__((aligned(16))) float sums[4][16 * NC][kRow];
        __shared__ float mls[4][16 * NC][2];
#pragma unroll
        for (int ct = 0; ct < NC; ++ct)
            if (lg == 0) {
                mls[wave][ct * 16 + lr][0] = m[ct];
                mls[wave][ct * 16 + lr][1] = l[ct];
            }
        __syncthreads();
        float factor[NC];
#pragma unroll
        for (int ct = 0; ct < NC; ++ct) {
            const int c = ct * 16 + lr;
            const float top = fmaxf(fmaxf(mls[0][c][0], mls[1][c][0]), fmaxf(mls[2][c][0], mls[3][c][0]));
            factor[ct] = pow2(m[ct] - (top == -INFINITY ? 0.0f : top));
        }
        auto joined = [&](int c, float& top) {
            top = fmaxf(fmaxf(mls[0][c][0], mls[1][c][0]), fmaxf(mls[2][c][0], mls[3][c][0]));
            const float base = top == -INFINITY ? 0.0f : top;
            float ll = 0.0f;
#pragma unroll
            for (int w = 0; w < 4; ++w) ll += mls[w][c][1] * pow2(mls[w][c][0] - base);
            return ll;
        };
#pragma unroll
        for (int pass = 0; pass < D / 32; ++pass) {
#pragma unroll
            for (int ct = 0; ct < NC; ++ct)
#pragma unroll
                for (int i = 0; i < 2; ++i) *(f32x4*)&sums[wave][ct * 16 + lr][i * 16 + lg * 4] = o[ct][pass * 2 + i] * factor[ct];
            __syncthreads();
            for (int i = tid; i < 16 * NC * 8; i += 256) {
                const int c = i / 8, d = i % 8 * 4;
                if (col0 + c < C) {
                    f32x4 x = *(f32x4*)&sums[0][c][d];
#pragma unroll
                    for (int w = 1; w < 4; ++w) x += *(f32x4*)&sums[w][c][d];
                    float top;
                    put(col0 + c, pass * 32 + d, x, joined(c, top));
                }
            }
            __syncthreads();
        }
        if (tid < 16 * NC && col0 + tid < C) {
            float top;
            const float ll = joined(tid, top);
            put_sums(col0 + tid, top, ll);
        }
    }
}

// Joins the splits of a request's keys: a wavefront takes a (token, head).
template <int D, bool F32>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs g)
{
    const int per = (min(g.max_drafts, g.T) * g.heads + 3) / 4, b = blockIdx.x / per;
    const int start = g.starts[b], n = min(min(g.starts[b + 1], g.T) - start, g.max_drafts), ctx = g.ctx[b];
    const int row = blockIdx.x % per * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;  // token of the request, head
    if (start < 0 || ctx < 0 || row >= n * g.heads) return;
    const int64_t t = start + row / g.heads, head = row % g.heads;
    const int total = (int)min((int64_t)ctx + n, (int64_t)g.max_pages * kPage);
    const int active = min(g.nsplit, max(1, ((total + kPage - 1) / kPage + g.chunk - 1) / g.chunk));
    const int64_t at = t * g.heads + head, all = (int64_t)g.T * g.heads;
    float top = -INFINITY;
    for (int s = lane; s < active; s += 64) top = fmaxf(top, g.part_ml[(s * all + at) * 2]);
#define MMOE_JOIN(OFF) top = fmaxf(top, lane_xor<OFF>(top))
    MMOE_JOIN(1); MMOE_JOIN(2); MMOE_JOIN(4); MMOE_JOIN(8); MMOE_JOIN(16); MMOE_JOIN(32);
#undef MMOE_JOIN
    const float base = top == -INFINITY ? 0.0f : top;
    constexpr int kPer = D / 64;
    float x[kPer], l = 0.0f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) x[i] = 0.0f;
    for (int s = 0; s < active; ++s) {
        const float w = pow2(g.part_ml[(s * all + at) * 2] - base);
        l += w * g.part_ml[(s * all + at) * 2 + 1];
#pragma unroll
        for (int i = 0; i < kPer; ++i) x[i] += w * g.part_o[(s * all + at) * D + i * 64 + lane];
    }
    const float r = l != 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int64_t dst = t * g.ot + head * g.oh + i * 64 + lane;
        if (F32) ((float*)g.out)[dst] = x[i] * r;
        else ((uint16_t*)g.out)[dst] = f32_to_bf16_bits(x[i] * r);
    }
    if (lane == 0 && g.lse) g.lse[at] = l == 0.0f ? -INFINITY : (top + __log2f(l)) * 0.693147180559945309417f;
}

// How a call is shared out: columns to a wavefront, whether the wavefronts of a workgroup take different columns or
// different keys, and splits of the keys.
struct Shares {
    int nc, groups, chunk, nsplit;
    bool cols;
};
static Shares shares(const mmoe_attend_shape& s)
{
    Shares r;
    const int G = s.heads / s.cache.kv_heads, most = s.cache.head_dim > 128 ? 2 : 4;
    const int64_t C = (int64_t)(s.max_drafts < s.T ? s.max_drafts : s.T) * G;
    r.cols = C > 16 * most;
    const int64_t per = r.cols ? (C + 3) / 4 : C;
    r.nc = per <= 16 ? 1 : per <= 32 || most == 2 ? 2 : 4;
    const int wide = 16 * r.nc * (r.cols ? 4 : 1);
    r.groups = (int)((C + wide - 1) / wide);
    int64_t longest = s.max_keys ? s.max_keys : (int64_t)s.max_pages * kPage;
    if (longest > (int64_t)s.max_pages * kPage) longest = (int64_t)s.max_pages * kPage;
    const int64_t all = s.sum_keys ? s.sum_keys : (int64_t)s.n_requests * longest;
    const int64_t pages = all / kPage + s.n_requests, most_pages = (longest + kPage - 1) / kPage;
    const int64_t target = r.nc == 1 ? 1024 : 512;
    int64_t chunk = (pages * s.cache.kv_heads * r.groups + target - 1) / target;
    if (chunk < 16) chunk = 16;
    int64_t n = (most_pages + chunk - 1) / chunk;
    if (n > 256) n = 256, chunk = (most_pages + n - 1) / n;
    if (n < 1) n = 1;
    r.chunk = (int)chunk;
    r.nsplit = (int)n;
    return r;
}

// Whether the grids' sizes fit.
bool attend_fits(const mmoe_attend_shape& s)
{
    const Shares r = shares(s);
    const int64_t drafts = s.max_drafts < s.T ? s.max_drafts : s.T, most = ((int64_t)1 << 31) - 1;
    return drafts * s.heads < most && (drafts * s.heads + 3) / 4 * s.n_requests <= most &&
           (int64_t)r.groups * s.cache.kv_heads * s.n_requests <= most / r.nsplit;
}

size_t attend_ws_bytes(const mmoe_attend_shape& s)
{
    const Shares r = shares(s);
    if (r.nsplit == 1) return 256;
    const size_t rows = (size_t)r.nsplit * s.T * s.heads;
    return align256(rows * s.cache.head_dim * 4) + align256(rows * 8);
}

template <int D, int KIND>
static void attend(const Shares& r, const AttendArgs& g, hipStream_t st)
{
    const dim3 grid((unsigned)((int64_t)r.groups * g.kv_heads * g.B * r.nsplit)), block(256);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, st, g); };
    if (r.cols) {
        if (r.nc == 1) go(attend_kernel<D, KIND, 1, true>);
        else if (r.nc == 2) go(attend_kernel<D, KIND, 2, true>);
        else if constexpr (D <= 128) go(attend_kernel<D, KIND, 4, true>);
    } else {
        if (r.nc == 1) go(attend_kernel<D, KIND, 1, false>);
        else if (r.nc == 2) go(attend_kernel<D, KIND, 2, false>);
        else if constexpr (D <= 128) go(attend_kernel<D, KIND, 4, false>);
    }
    if (r.nsplit > 1) {
        const int drafts = g.max_drafts < g.T ? g.max_drafts : g.T;
        hipLaunchKernelGGL((attend_join_kernel<D, KIND == kF32>), dim3((unsigned)(((int64_t)drafts * g.heads + 3) / 4 * g.B)), block, 0, st, g);
    }
}

template <int KIND>
static void attend(int D, const Shares& r, const AttendArgs& g, hipStream_t st)
{
    if (D == 64) attend<64, KIND>(r, g, st);
    else if (D == 128) attend<128, KIND>(r, g, st);
    else attend<256, KIND>(r, g, st);
}

int launch_attend(const mmoe_attend_shape& s, const void* Q, const int32_t* starts, const int32_t* ctx, const uint64_t* tree,
                  const int32_t* pages, const mmoe_cache& c, void* out, float* lse, void* ws, hipStream_t st)
{
    const Shares r = shares(s);
    const int64_t D = s.cache.head_dim;
    const size_t rows = (size_t)r.nsplit * s.T * s.heads;
    AttendArgs g = {(const char*)Q, starts, ctx, tree, pages, (const char*)c.k, (const char*)c.v, c.k_scale, c.v_scale, (char*)out, lse,
                    (float*)ws, (float*)((char*)ws + align256(rows * D * 4)),
                    s.q_token ? s.q_token : s.heads * D, s.q_head ? s.q_head : D, s.o_token ? s.o_token : s.heads * D,
                    s.o_head ? s.o_head : D, s.T, s.n_requests, s.heads, s.cache.kv_heads, s.heads / s.cache.kv_heads, s.max_pages,
                    s.max_drafts, s.mask_words, s.cache.n_pages, r.groups, r.nsplit, r.chunk, s.scale};
    if (s.cache.format == MMOE_CACHE_INT8) attend<kInt8>((int)D, r, g, st);
    else if (s.cache.format == MMOE_CACHE_FP8) attend<kFp8>((int)D, r, g, st);
    else if (s.cache.dtype == MMOE_F32) attend<kF32>((int)D, r, g, st);
    else attend<kBf16>((int)D, r, g, st);
    return launch_status();
}

}  // namespace mmoe
