// The attention kernel's template: one translation unit for each kind of page (attend_*.hip).
//
// out[t,h] = sum_j softmax_j(scale <Q[t,h], K[j]>) V[j], in one pass over the keys with a reference m for the exponents and the
// sum l: O holds sum 2^(s_j - m) V_j, and where a step's largest score exceeds m by more than kSlack, m becomes that score and O and
// l are scaled (everything in base 2: the scores carry log2 e).  Over 8-bit pages m follows the products of probabilities and value scales
// that the column sees in the same way, by column: what a row that is hidden or all but improbable holds takes no bits from the others.
//
// A column is a (token, query head) pair of one request and key head: all that read the same keys.  A wavefront holds 16 NC
// columns.  Keys are the row operand of the first product, so a lane has four consecutive keys of a column per tile of 16, which
// is, with the order in which pages keep values, its part of the column operand of the second: probabilities go
// from one product to the other inside a lane, and keys and values from memory straight into operand registers, 1 KB an
// instruction, no LDS and no barrier in the loop.  Queries of more than 16 columns stand in LDS in operand order.
//
// Bound by the cache's bytes up to 32 columns (8 requests of 60000 fp8 keys, 32 heads on 8 of 128: single tokens 185 us, 5.5 TB/s; 8 tokens
// each 199 us, 5.1 TB/s), then more and more by vector instructions (16 tokens, 64 columns: 4.6 TB/s), fp32 by its matrix rate, few keys by
// latency (4 requests of up to 700: 9.8 us).  8-bit codes widen to fp16, which holds them exactly; their key scales multiply scores and
// their value scales probabilities, so pages are never written out in 16 bits.
//
// Roundings below 32 bits: probabilities to bf16 or, with their value's scale, fp16, the operand type of the second product (8 and
// 11 bits of numbers that are summed, fp16 to 2^-30 of the largest; the sum l has them in fp32); with codes queries to fp16 too, scaled by a power of two (exact but for
// elements under 2^-26 of the head's largest); out once.
#pragma once
#include <math.h>

#include "attn_internal.h"

namespace mmoe {

enum { kBf16 = 0, kInt8 = 1, kFp8 = 2, kF32 = 3 };  // what pages hold

// How a call is shared out: 16-column tiles to a wavefront; sets of columns to a workgroup's four wavefronts, which take different
// keys within a set; groups of columns; and workgroups for each key head and column group: one for each request (shares 0), or
// `shares` ones that take equal parts of all requests' pages one after the other.
struct Shares {
    int nc, sets, groups, shares;
};
constexpr int kMaxShared = 2048;  // requests whose pages are shared out

// The request's drafted tokens, its keys, and their pages.
struct Request {
    int start, n, ctx, total, pages;
};
template <typename G>
__device__ __forceinline__ Request request_of(const G& g, int b)
{
    Request r;
    r.start = g.starts[b];
    r.n = min(min(g.starts[b + 1], g.T) - r.start, g.max_drafts);
    r.ctx = g.ctx[b];
    if (r.start < 0 || r.ctx < 0) r.n = 0;
    r.total = r.n > 0 ? (int)min((int64_t)r.ctx + r.n, (int64_t)g.max_pages * kPage) : 0;
    r.pages = (r.total + kPage - 1) / kPage;
    return r;
}
// Shares of `pages` pages: the first `more` of them have each + 1.
struct Cut {
    int each, more;
    __device__ Cut(int pages, int shares) : each(pages / shares), more(pages % shares) {}
    __device__ int start(int w) const { return w * each + min(w, more); }
    __device__ int of(int page) const
    {
        const int lead = more * (each + 1);
        return page < lead ? page / (each + 1) : more + (page - lead) / each;
    }
};

struct AttendArgs {
    const char* Q;
    const int32_t *starts, *ctx;
    const uint64_t* tree;
    const int32_t* pages;
    const char *k, *v;
    const float *k_scale, *v_scale;
    char* out;
    float* lse;
    // a share's part of a request that it does not have all of, [shares][2][kv_heads][columns]: 0 the share's first, 1 its last
    float* part_o;   // [D]
    float* part_ml;  // [2]
    int64_t qt, qh, ot, oh;
    int T, B, heads, kv_heads, G, max_pages, max_drafts, mask_words, n_pages;
    int groups, shares, columns;  // column groups; see Shares; columns of a request at most
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

__device__ __forceinline__ void in_agprs(f32x4& x) { asm volatile("" : "+a"(x)); }

// What is worked out of it in a rare branch is not worked out ahead of the branch.
template <typename T>
__device__ __forceinline__ void only_here(T& x) { asm volatile("" : "+v"(x)); }

// 2^x; -infinity gives 0.
__device__ __forceinline__ float pow2(float x) { return __builtin_amdgcn_exp2f(x); }

// Probabilities are up to 2^8: scores that rise slowly then leave O and l as they are.  (Random keys: level, 202 us with, 199 without;
// the scaling of 64 registers where every step has a new maximum is what it spares.)
constexpr float kSlack = 8.0f;
// Over codes the reference follows the products of probabilities and value scales, which go into fp16: a column's largest one is under 2^7 when it is
// found and may rise to 2^15, which keeps small ones out of the subnormal range.  Rows that the column does not see have no part in it.
// Scales that are not zero are 2^-109 at least, so l could leave fp32: probabilities are 2^60 to 2^-90 of the reference at their peak, and what that
// leaves of the lift is kept apart, by column.
constexpr float kLiftBits = 7.0f, kTopBits = 15.0f, kMostBits = 100.0f;

template <int D, int KIND, int NC>
struct AttendPlan {
    static constexpr int kBytes = KIND == kF32 ? 4 : KIND == kBf16 ? 2 : 1;
    static constexpr int E = 16 / kBytes;
    static constexpr bool kCodes = KIND == kInt8 || KIND == kFp8;
    // tiles of 16 keys to a step: 16 KB of keys and values for heads of 128
    static constexpr int KT = kCodes ? 4 : D * kBytes <= 128 ? 4 : D * kBytes <= 256 || KIND == kBf16 ? 2 : 1;
    static constexpr int NKS = D / (4 * E);            // pieces of a key row that a lane holds
    static constexpr int NV = KT * 4 / E == 0 ? 1 : KT * 4 / E;  // value pieces to 16 elements of a step
    static constexpr int QS = KIND == kF32 ? D / 16 : D / 32;    // query pieces
    static constexpr int DT = D / 16;
    static constexpr bool kLdsQ = NC > 1;
};

// Waves to a SIMD: two where the accumulators and the operands in flight leave half of the registers.
template <int D, int KIND, int NC>
constexpr int attend_waves() { return (NC == 1 && D <= 128) || (NC == 2 && D <= 128) ? 2 : 1; }

template <int D, int KIND, int NC, int CW>
__global__ __launch_bounds__(256, (attend_waves<D, KIND, NC>())) void attend_kernel(AttendArgs g)
{
    using L = AttendPlan<D, KIND, NC>;
    constexpr int KT = L::KT, NKS = L::NKS, NV = L::NV, QS = L::QS, DT = L::DT, E = L::E, kSteps = 4 / KT;
    constexpr int NP = KT * 4 / (KIND == kF32 ? 4 : 8);  // operand pieces of the probabilities
    constexpr bool kCodes = L::kCodes;
    constexpr int kEsz = KIND == kF32 ? 4 : 2;  // of Q and out
    // What follows from the lane is worked out where it is used: hoisted out of the loops, it would push operands out of registers.
    auto fresh = [](int x) {
        asm volatile("" : "+v"(x));
        return x;
    };
    int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    // column groups of the same keys on one XCD (workgroup id mod 8)
    int id = blockIdx.x / 8;
    const int cg = id % g.groups;
    id = id / g.groups * 8 + blockIdx.x % 8;
    const int h = id % g.kv_heads;
    id /= g.kv_heads;
    const int share = id;
    if (share >= (g.shares ? g.shares : g.B)) return;  // uniform

    // CW sets of columns, each for KW wavefronts that share its queries and take different keys
    constexpr int KW = 4 / CW, kWide = CW * 16 * NC;
    constexpr int kQBytes = L::kLdsQ ? CW * NC * QS * 1024 : 16;
    constexpr int kRow = 36, kSumBytes = KW == 1 ? 16 : 2 * KW * kWide * kRow * 4;
    const int set = wave % CW, turn = wave / CW;
    __shared__ __attribute__((aligned(16))) char lds[kQBytes > kSumBytes ? kQBytes : kSumBytes];  // queries, and at the end the join's sums
    __shared__ float mls[KW == 1 ? 1 : KW][kWide][2];
    __shared__ int first_page[kMaxShared + 1];  // of each request among all pages (fewer than 2^30, or there are no shares)

    int at = 0, until = 1;  // pages of the share
    int b = share;
    if (g.shares) {
        // prefix sums over the requests: a thread has a run of them
        __shared__ int wave_sum[4];
        const int per = (g.B + 255) / 256;
        int sum = 0;
        for (int i = tid * per; i < min((tid + 1) * per, g.B); ++i) sum += request_of(g, i).pages;
        int before = sum;
#pragma unroll
        for (int off = 1; off < 64; off *= 2) {
            const int up = __shfl_up(before, off);
            if (lane >= off) before += up;
        }
        if (lane == 63) wave_sum[wave] = before;
        __syncthreads();
        int all = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if (w < wave) before += wave_sum[w];
            all += wave_sum[w];
        }
        before -= sum;
        for (int i = tid * per; i < min((tid + 1) * per, g.B); ++i) {
            first_page[i] = before;
            before += request_of(g, i).pages;
        }
        if (tid == 0) first_page[g.B] = all;
        __syncthreads();
        const Cut cut(all, g.shares);
        at = cut.start(share);
        until = cut.start(share + 1);
        if (at >= until) return;  // uniform
        int lo = 0, hi = g.B;  // the request with page `at`: the last one that starts there or before, if it has pages
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (first_page[mid] <= at) lo = mid;
            else hi = mid;
        }
        b = __builtin_amdgcn_readfirstlane(lo);
    }
    const int share_at = at;
  for (; at < until; ++b) {  // requests of the share
    tid = fresh(threadIdx.x), lane = tid & 63, lr = lane & 15, lg = lane >> 4;
    const Request r = request_of(g, b);
    const int start = r.start, n = r.n, ctx = r.ctx, total = r.total, C = n * g.G;
    // pages of the request that are the share's; `slot`: where its part goes, -1 if it is all of the request
    int page0 = 0, page1 = r.pages, slot = -1;
    if (g.shares) {
        const int first = __builtin_amdgcn_readfirstlane(first_page[b]);
        page0 = at - first;
        page1 = min(until - first, r.pages);
        if (page0 > 0 || page1 < r.pages) slot = at == share_at ? 0 : 1;
        at = first + page1;
    } else {
        at = until;
    }
    if (cg * kWide >= C) continue;  // uniform
    const int col0 = cg * kWide + set * 16 * NC;

    // what the last column of these sees at most
    const int last_token = min(C - 1, cg * kWide + kWide - 1) / g.G;
    const int limit = g.tree ? total : (int)min((int64_t)total, (int64_t)ctx + last_token + 1);
    const int step0 = page0 * kSteps;
    const int step1 = min(page1 * kSteps, (limit + 16 * KT - 1) / (16 * KT));

    constexpr int64_t kBlock = (int64_t)kPage * D * L::kBytes;
    // (constant address space: scalar loads, which the counts of the vector loads in flight do not see)
    const auto* table = (const __attribute__((address_space(4))) int32_t*)(g.pages + (int64_t)b * g.max_pages);
    // Page and head of a step.  A page number outside the cache is page 0 with `hole` set: its keys are not seen.
    auto page_of = [&](int step) { return __builtin_amdgcn_readfirstlane(table[step / kSteps]); };
    auto block_of = [&](int page) { return (int64_t)((unsigned)page < (unsigned)g.n_pages ? page : 0) * g.kv_heads + h; };
    u32x4 kf[KT][NKS], vf[DT][NV];
    f32x4 ks[KT], vs[KT];
    auto load_k = [&](int64_t block, int step) {
        const char* src = g.k + block * kBlock + (step % kSteps) * (KT * NKS * 1024) + lane * 16;
        each<KT * NKS>([&](auto x) {
            constexpr int i = decltype(x)::value;
            kf[i / NKS][i % NKS] = *(const u32x4*)(src + i * 1024);
        });
    };
    auto load_ks = [&](int64_t block) {
        if constexpr (kCodes)
            each<KT>([&](auto x) { ks[decltype(x)::value] = *(const f32x4*)(g.k_scale + block * kPage + lg * 4 + decltype(x)::value * 16); });
    };
    auto load_v = [&](int64_t block, int step, auto dtc) {
        constexpr int dt = decltype(dtc)::value;
        const char* src = g.v + block * kBlock + (step % kSteps) * (NV * 1024) + lane * 16;
        each<NV>([&](auto x) { vf[dt][decltype(x)::value] = *(const u32x4*)(src + (dt * (16 / E) + decltype(x)::value) * 1024); });
    };
    auto load_vs = [&](int64_t block) {
        if constexpr (kCodes)
            each<KT>([&](auto x) { vs[decltype(x)::value] = *(const f32x4*)(g.v_scale + block * kPage + lg * 4 + decltype(x)::value * 16); });
    };
    constexpr int kStride = KW;
    // Two wavefronts to a SIMD and two tiles: no registers for values and scales ahead of their use, the other wavefront covers them.  (All ahead:
    // 8 tokens, fp8, 8 requests of 60000 202 -> 221 us, 32 of 4000 67 -> 80.)
    constexpr bool kLate = attend_waves<D, KIND, NC>() == 2 && NC == 2 && D == 128;
    int step = step0 + turn;
    const bool works = step < step1 && col0 < C;  // uniform over the wavefront
    int page = 0;
    if (works) {
        page = page_of(step);
        const int64_t block = block_of(page);
        load_k(block, step);
        if constexpr (!kLate) {
            load_ks(block);
            load_vs(block);
            each<DT>([&](auto dt) { load_v(block, step, dt); });
        }
    }

    // ---- queries ----
    if constexpr (L::kLdsQ || KW > 1) __syncthreads();  // the request before is done with the LDS
    char* const lds_q = lds + set * NC * QS * 1024 + lane * 16;
    u32x4 q_reg[L::kLdsQ ? 1 : QS];
    float mult[NC];  // of the scores, in base 2; positive
    int token[NC];   // of the request; n where the column is none
    uint64_t word[NC];  // first 64 bits of the token's row of the tree
    each<NC>([&](auto ctc) {
        constexpr int ct = decltype(ctc)::value;
        const int c = col0 + ct * 16 + lr;
        const bool there = c < C && g.scale != 0.0f;
        token[ct] = c < C ? c / g.G : n;
        word[ct] = g.tree && c < C ? g.tree[(int64_t)(start + token[ct]) * g.mask_words] : 0;
        const char* src = g.Q + ((int64_t)(start + (there ? c / g.G : 0)) * g.qt + (int64_t)(h * g.G + (there ? c % g.G : 0)) * g.qh) * kEsz;
        mult[ct] = g.scale != 0.0f ? fabsf(g.scale) * 1.44269504088896340736f : 1.0f;
        const uint32_t sign = g.scale < 0.0f ? (KIND == kF32 ? 0x80000000u : 0x80008000u) : 0u;
        u32x4 q[QS];
        each<QS>([&](auto x) {
            constexpr int i = decltype(x)::value;
            // codes: two instructions of 32 share a piece of 16 codes
            const int d = kCodes ? (i >> 1) * 64 + lg * 16 + (i & 1) * 8 : i * (KIND == kF32 ? 16 : 32) + lg * (KIND == kF32 ? 4 : 8);
            q[i] = there ? *(const u32x4*)(src + d * kEsz) ^ sign : u32x4{0, 0, 0, 0};
        });
        if constexpr (kCodes) {  // to fp16, by a power of two that puts the largest at 2^12
            float a = 0.0f;
            each<QS * 4>([&](auto x) {
                const uint32_t w = q[decltype(x)::value / 4][decltype(x)::value % 4];
                a = fmaxf(a, fmaxf(fabsf(bf16_lo(w)), fabsf(bf16_hi(w))));
            });
            a = max_groups(a);
            const int e = a > 0.0f && a < INFINITY ? min(100, 12 - (int)((__float_as_uint(a) >> 23) - 127)) : 0;
            const float up = ldexpf(1.0f, e);
            mult[ct] *= ldexpf(1.0f, -e);
            each<QS * 4>([&](auto x) {
                constexpr int i = decltype(x)::value / 4, w = decltype(x)::value % 4;
                q[i][w] = pack_f16(bf16_lo(q[i][w]) * up, bf16_hi(q[i][w]) * up);
            });
        }
        each<QS>([&](auto x) {
            constexpr int i = decltype(x)::value;
            if constexpr (!L::kLdsQ) q_reg[i] = q[i];
            else if (turn == ct % KW) *(u32x4*)(lds_q + (ct * QS + i) * 1024) = q[i];
        });
    });
    if constexpr (L::kLdsQ) __syncthreads();
    auto query = [&](int ct, int i) -> u32x4 {
        if constexpr (L::kLdsQ) return *(const u32x4*)(lds_q + (ct * QS + i) * 1024);
        else return q_reg[i];
    };

    f32x4 o[NC][DT];
    float m[NC], l[NC];
    each<NC>([&](auto ct) {
        m[decltype(ct)::value] = -INFINITY;
        l[decltype(ct)::value] = 0.0f;  // this lane's keys only, until the end
        each<DT>([&](auto dt) { o[decltype(ct)::value][decltype(dt)::value] = f32x4{0.0f, 0.0f, 0.0f, 0.0f}; });
    });
    float apart[NC];  // codes: o holds 2^apart times what the reference says
    each<NC>([&](auto ct) { apart[decltype(ct)::value] = 0.0f; });
    bool aparts = false;  // one of them is not zero

    // Accumulators are read by vector instructions in rare branches only: they stay in AGPRs around them.
    auto pin = [&](int ct) {
        if constexpr (attend_waves<D, KIND, NC>() == 1)
            each<DT>([&](auto dt) { in_agprs(o[ct][decltype(dt)::value]); });
    };
    auto fragments = [&](const u32x4& x, u32x4& lo, u32x4& hi) {  // 16 codes as two operands
        const u32x2 a = widen<KIND>(x[0]), c = widen<KIND>(x[1]), d = widen<KIND>(x[2]), e = widen<KIND>(x[3]);
        lo = u32x4{a[0], a[1], c[0], c[1]};
        hi = u32x4{d[0], d[1], e[0], e[1]};
    };

    while (works && step < step1) {
        const int next = step + kStride;
        const bool more = next < step1;
        // What is loaded ahead is loaded in every iteration, the last one's own step again: behind a branch the waits could not count.
        const int next_page = page_of(more ? next : step);
        const int64_t next_block = block_of(next_page);
        const int ahead = more ? next : step;
        const bool hole = (unsigned)page >= (unsigned)g.n_pages;
        const bool tail = hole || (step + 1) * 16 * KT > ctx;  // not all of the step's keys are committed ones
        const int key0 = step * 16 * KT;
        const int there = hole ? 0 : total;  // keys from here on are not seen by anybody
        const int left = there - key0 - lg * 4;  // those of them from the lane's first key on

        if constexpr (kLate) load_ks(block_of(page));
        f32x4 s[NC][KT];
        each<NC * KT>([&](auto x) { s[decltype(x)::value / KT][decltype(x)::value % KT] = f32x4{0.0f, 0.0f, 0.0f, 0.0f}; });
        u32x4 q_now[NC], q_next[NC];
        each<NC>([&](auto ct) { q_next[decltype(ct)::value] = query(decltype(ct)::value, 0); });
        each<QS>([&](auto xc) {
            constexpr int i = decltype(xc)::value;
            each<NC>([&](auto ctc) {
                constexpr int ct = decltype(ctc)::value;
                q_now[ct] = q_next[ct];
                if constexpr (i + 1 < QS) q_next[ct] = query(ct, i + 1);
            });
            u32x4 key[KT];  // operands of this part of the heads
            each<KT>([&](auto ktc) {
                constexpr int kt = decltype(ktc)::value;
                if constexpr (kCodes) {
                    const u32x2 a = widen<KIND>(kf[kt][i / 2][i % 2 * 2]), c = widen<KIND>(kf[kt][i / 2][i % 2 * 2 + 1]);
                    key[kt] = u32x4{a[0], a[1], c[0], c[1]};
                } else {
                    key[kt] = kf[kt][i];
                }
            });
            each<NC>([&](auto ctc) {
                constexpr int ct = decltype(ctc)::value;
                each<KT>([&](auto ktc) {
                    constexpr int kt = decltype(ktc)::value;
                    s[ct][kt] = mma_kind<KIND>(key[kt], q_now[ct], s[ct][kt]);
                });
            });
            if constexpr (NC > 1) __builtin_amdgcn_sched_barrier(0);  // (the compiler would fetch all queries first)
        });
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (kLate) {
            const int64_t block = block_of(page);
            load_vs(block);
            each<DT>([&](auto dt) { load_v(block, step, dt); });
            __builtin_amdgcn_sched_barrier(0);
        }
        float room = 0.0f;  // codes: bits by which a probability may exceed the reference, whichever value it goes with
        if constexpr (kCodes) {
            each<KT>([&](auto ktc) {
                constexpr int kt = decltype(ktc)::value;
                each<NC>([&](auto ct) { s[decltype(ct)::value][kt] *= ks[kt]; });
            });
            if (tail)  // scales of rows past the end may be anything
                each<KT * 4>([&](auto x) {
                    constexpr int kt = decltype(x)::value / 4, e = decltype(x)::value % 4;
                    if (kt * 16 + e >= left) vs[kt][e] = 0.0f;
                });
            float most = 0.0f;
            each<KT * 4>([&](auto x) { most = fmaxf(most, vs[decltype(x)::value / 4][decltype(x)::value % 4]); });
            most = max_groups(most);
            room = most > 0.0f ? kTopBits - (float)__builtin_amdgcn_frexp_expf(most) : kMostBits;  // (the scale is under 2^frexp)
        }
        load_k(next_block, ahead);
        if constexpr (!kLate) load_ks(next_block);
        __builtin_amdgcn_sched_barrier(0);

        u32x4 p[NC][NP];
        uint64_t vis[NC];  // keys of the step that the column sees, from the lane's first on
        each<NC>([&](auto ctc) {
            constexpr int ct = decltype(ctc)::value;
            vis[ct] = ~(uint64_t)0;
            if (tail) {
                const int page0 = key0 & ~(kPage - 1), d0 = page0 - ctx;  // first key of the page, as a drafted token
                const int i = token[ct], from = max(d0, 0);               // first drafted token of the page
                uint64_t bits = 0;
                if (i < n && from < n) {
                    if (g.tree) {
                        const uint64_t* row = g.tree + (int64_t)(start + i) * g.mask_words;
                        const int w = from >> 6, r = from & 63;
                        if (w == 0) bits = word[ct] >> r;
                        else if (w < g.mask_words) bits = row[w] >> r;
                        if (r && w + 1 < g.mask_words) bits |= row[w + 1] << (64 - r);
                    } else {
                        const int c = i + 1 - from;
                        bits = c <= 0 ? 0 : c >= 64 ? ~(uint64_t)0 : ((uint64_t)1 << c) - 1;
                    }
                    if (n - from < 64) bits &= ((uint64_t)1 << (n - from)) - 1;
                }
                // below them the committed keys
                uint64_t v = d0 >= 0 ? bits : d0 <= -kPage ? ~(uint64_t)0 : (((uint64_t)1 << -d0) - 1) | bits << -d0;
                if (there - page0 < 64) v &= there > page0 ? ((uint64_t)1 << (there - page0)) - 1 : 0;
                if (i >= n) v = 0;
                vis[ct] = v >> (key0 - page0 + lg * 4);
                each<KT * 4>([&](auto x) {
                    constexpr int kt = decltype(x)::value / 4, e = decltype(x)::value % 4;
                    if (!(vis[ct] & (uint64_t)1 << (kt * 16 + e))) s[ct][kt][e] = -INFINITY;
                });
            }
            float top = -INFINITY;
            each<KT * 4>([&](auto x) { top = fmaxf(top, s[ct][decltype(x)::value / 4][decltype(x)::value % 4]); });
            const float score = max_groups(top);
            top = score * mult[ct];
            pin(ct);
            if constexpr (kCodes) {
                // (never where top is -infinity; not top - m: far off, its rounding is many bits that the exponents do not have)
                if (__any(__builtin_fmaf(score, mult[ct], -m[ct]) > fminf(room - apart[ct], kMostBits))) {
                    each<KT>([&](auto kt) { only_here(s[ct][decltype(kt)::value]), only_here(vs[decltype(kt)::value]); });
                    const float from = fmaxf(m[ct], top), gap = from - m[ct];  // (infinite where there was nothing so far, NaN where there still is not)
                    float most = -INFINITY;  // log2 of the largest product that the column sees: a scale's bits are 2^23 (log2 + 127) less 0 to 0.09
                    each<KT * 4>([&](auto x) {
                        constexpr int kt = decltype(x)::value / 4, e = decltype(x)::value % 4;
                        most = fmaxf(most, __builtin_fmaf((float)__float_as_uint(vs[kt][e]), 0x1p-23f, __builtin_fmaf(s[ct][kt][e], mult[ct], -from)));
                    });
                    most = max_groups(most) - 126.9f + apart[ct];
                    const float peak = fmaxf(__log2f(max_groups(l[ct])) - gap, __builtin_fmaf(score, mult[ct], -from));  // of the probabilities, or of l's parts
                    const bool stay = !(most + gap > kTopBits || peak + gap > 90.0f);  // a row was in doubt that the column sees with a small product, or not
                    const float by = most + gap > kTopBits ? most - kLiftBits : -gap;  // that the reference should be above `from`
                    float up = fminf(fmaxf(by, peak - 90.0f), peak + 60.0f);
                    if (!(fabsf(from) < 0x1p20f)) up = 0.0f;  // (so far off, references are not so near one another)
                    m[ct] = stay ? m[ct] : from + up;
                    up = m[ct] - from;
                    const float rest = !stay && fabsf(up - by) > 1.0f ? fminf(apart[ct] + (up - by), 115.0f - fmaxf(peak - up, 0.0f)) : apart[ct];
                    const float f = stay ? 1.0f : pow2(rest - apart[ct] - up - gap);
                    each<DT>([&](auto dt) { o[ct][decltype(dt)::value] *= f; });
                    l[ct] *= stay ? 1.0f : pow2(-up - gap);
                    apart[ct] = rest;
                    aparts = aparts || __any(rest != 0.0f);
                    pin(ct);
                }
            } else if (__any(top - m[ct] > kSlack)) {  // (never where top is -infinity)
                const float up = fmaxf(m[ct], top), alpha = pow2(m[ct] - (up == -INFINITY ? 0.0f : up));
                m[ct] = up;
                l[ct] *= alpha;
                each<DT>([&](auto dt) { o[ct][decltype(dt)::value] *= alpha; });
                pin(ct);
            }
            const float base = m[ct] == -INFINITY ? 0.0f : m[ct];
            float sum = 0.0f;
            each<KT * 4>([&](auto x) {
                constexpr int kt = decltype(x)::value / 4, e = decltype(x)::value % 4;
                s[ct][kt][e] = pow2(__builtin_fmaf(s[ct][kt][e], mult[ct], -base));
                sum += s[ct][kt][e];
            });
            if constexpr (kCodes) {
                each<KT>([&](auto kt) { s[ct][decltype(kt)::value] *= vs[decltype(kt)::value]; });
                if (tail || aparts) {
                    const float f = pow2(apart[ct]);
                    uint64_t seen = vis[ct];
                    only_here(seen);
                    each<KT * 4>([&](auto x) {  // (0 times a scale may be NaN)
                        constexpr int kt = decltype(x)::value / 4, e = decltype(x)::value % 4;
                        s[ct][kt][e] = seen & (uint64_t)1 << (kt * 16 + e) ? s[ct][kt][e] * f : 0.0f;
                    });
                }
            }
            l[ct] += sum;
            // tiles to operand pieces: 16-bit ones hold two tiles' keys
            if constexpr (KIND == kF32) {
                each<KT>([&](auto kt) { p[ct][decltype(kt)::value] = __builtin_bit_cast(u32x4, s[ct][decltype(kt)::value]); });
            } else {
                each<NP * 4>([&](auto x) {
                    constexpr int i = decltype(x)::value / 4, w = decltype(x)::value % 4;
                    const float lo = s[ct][2 * i + w / 2][(w & 1) * 2], hi = s[ct][2 * i + w / 2][(w & 1) * 2 + 1];
                    p[ct][i][w] = kCodes ? pack_f16(lo, hi) : pack_bf16(lo, hi);
                });
            }
            __builtin_amdgcn_sched_barrier(0);
        });

        each<NC>([&](auto ct) { pin(decltype(ct)::value); });
        if (tail) {
            // Values of rows past the end may be anything: zeros.  (Int8 codes are finite whatever they are.)  Piece word w of
            // 16-bit kinds holds keys 2 (w%2), +1 of the group in tile 2i + w/2; of 8-bit ones the four keys of tile w.
            auto row_there = [&](int kt, int e) { return kt * 16 + e < left; };
            bool odd = false;  // a value that is not finite, of a key that some columns may not see
            each<DT * NV * 4>([&](auto xc) {
                constexpr int x = decltype(xc)::value, dt = x / (NV * 4), i = x / 4 % NV, w = x % 4;
                uint32_t y = vf[dt][i][w];
                if constexpr (KIND == kF32) {
                    if (!row_there(i, w)) y = 0;
                    odd = odd || (y & 0x7F800000u) == 0x7F800000u;
                } else if constexpr (KIND == kBf16) {
                    if (!row_there(2 * i + w / 2, (w & 1) * 2)) y &= 0xFFFF0000u;
                    if (!row_there(2 * i + w / 2, (w & 1) * 2 + 1)) y &= 0xFFFFu;
                    odd = odd || (y & 0x7F80u) == 0x7F80u || (y & 0x7F800000u) == 0x7F800000u;
                } else if constexpr (KIND == kFp8) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (!row_there(w, e)) y &= ~(0xFFu << 8 * e);
                }
                vf[dt][i][w] = y;
                if constexpr (x % (NV * 4) == NV * 4 - 1) __builtin_amdgcn_sched_barrier(0);
            });
            // 0 times what is not finite would reach columns that do not see the key: such values are taken out, and
            // counted per kind with the columns that do see them.
            if constexpr (!kCodes) {
                if (__any(odd)) {
                    for (int kind = 0; kind < 3; ++kind) {  // +infinity, -infinity, NaN
                        auto is = [&](uint32_t bits) {      // fp32 bits
                            return kind == 0 ? bits == 0x7F800000u : kind == 1 ? bits == 0xFF800000u : (bits & 0x7FFFFFFFu) > 0x7F800000u;
                        };
                        each<DT * NC>([&](auto xc) {
                            constexpr int dt = decltype(xc)::value / NC, ct = decltype(xc)::value % NC;
                            f32x4 count = {0.0f, 0.0f, 0.0f, 0.0f};
                            each<NV>([&](auto ic) {
                                constexpr int i = decltype(ic)::value;
                                u32x4 mark, seen;
                                each<4>([&](auto wc) {
                                    constexpr int w = decltype(wc)::value;
                                    auto sees = [&](int kt, int e) { return (vis[ct] & (uint64_t)1 << (kt * 16 + e)) != 0; };
                                    const uint32_t y = vf[dt][i][w];
                                    if constexpr (KIND == kF32) {
                                        mark[w] = is(y) ? 0x3F800000u : 0u;
                                        seen[w] = sees(i, w) ? 0x3F800000u : 0u;
                                    } else {
                                        mark[w] = (is(y << 16) ? 0x3F80u : 0u) | (is(y & 0xFFFF0000u) ? 0x3F800000u : 0u);
                                        seen[w] = (sees(2 * i + w / 2, (w & 1) * 2) ? 0x3F80u : 0u) |
                                                  (sees(2 * i + w / 2, (w & 1) * 2 + 1) ? 0x3F800000u : 0u);
                                    }
                                });
                                count = mma_kind<KIND>(mark, seen, count);
                            });
                            f32x4 add;
                            each<4>([&](auto e) {
                                const float special = kind == 0 ? INFINITY : kind == 1 ? -INFINITY : NAN;
                                add[decltype(e)::value] = count[decltype(e)::value] > 0.0f ? special : 0.0f;
                            });
                            o[ct][dt] += add;
                            if constexpr (attend_waves<D, KIND, NC>() == 1) in_agprs(o[ct][dt]);
                            __builtin_amdgcn_sched_barrier(0);
                        });
                    }
                    each<DT * NV * 4>([&](auto xc) {
                        constexpr int x = decltype(xc)::value, dt = x / (NV * 4), i = x / 4 % NV, w = x % 4;
                        uint32_t y = vf[dt][i][w];
                        if constexpr (KIND == kF32) {
                            if ((y & 0x7F800000u) == 0x7F800000u) y = 0;
                        } else {
                            if ((y & 0x7F80u) == 0x7F80u) y &= 0xFFFF0000u;
                            if ((y & 0x7F800000u) == 0x7F800000u) y &= 0xFFFFu;
                        }
                        vf[dt][i][w] = y;
                    });
                }
            }
            each<NC>([&](auto ct) { pin(decltype(ct)::value); });
        }
        if constexpr (!kLate) load_vs(next_block);
        each<DT>([&](auto dtc) {
            constexpr int dt = decltype(dtc)::value;
            if constexpr (kCodes) {
                u32x4 lo, hi;
                fragments(vf[dt][0], lo, hi);
                each<NC>([&](auto ct) { o[decltype(ct)::value][dt] = mma_kind<KIND>(lo, p[decltype(ct)::value][0], o[decltype(ct)::value][dt]); });
                each<NC>([&](auto ct) { o[decltype(ct)::value][dt] = mma_kind<KIND>(hi, p[decltype(ct)::value][1], o[decltype(ct)::value][dt]); });
            } else {
                each<NV>([&](auto ic) {
                    constexpr int i = decltype(ic)::value;
                    each<NC>([&](auto ct) { o[decltype(ct)::value][dt] = mma_kind<KIND>(vf[dt][i], p[decltype(ct)::value][i], o[decltype(ct)::value][dt]); });
                });
            }
        });
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (!kLate) each<DT>([&](auto dt) { load_v(next_block, ahead, dt); });
        __builtin_amdgcn_sched_barrier(0);
        step = next;
        page = next_page;
    }

    // ---- results ----
    tid = fresh(threadIdx.x), lane = tid & 63, lr = lane & 15, lg = lane >> 4;
#pragma unroll
    for (int ct = 0; ct < NC; ++ct) l[ct] = sum_groups(l[ct]);
    if constexpr (kCodes) {  // the reference to where l is between 1/2 and 1
#pragma unroll
        for (int ct = 0; ct < NC; ++ct) {
            const int bits = __builtin_amdgcn_frexp_expf(l[ct]);
            const float down = ldexpf(pow2(-apart[ct]), -bits);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[ct][dt] *= down;
            l[ct] = ldexpf(l[ct], -bits);
            m[ct] += (float)bits;
        }
    }

    const bool direct = slot < 0;
    const int64_t part = (((int64_t)share * 2 + slot) * g.kv_heads + h) * g.columns;
    // Four consecutive elements of column c, whose token and head have their place in `to`.
    auto put = [&](int c, int64_t to, int d, f32x4 x) {
        if (!direct) *(f32x4*)(g.part_o + (part + c) * D + d) = x;
        else if constexpr (KIND == kF32) *(f32x4*)(g.out + (to + d) * kEsz) = x;
        else *(u32x2*)(g.out + (to + d) * kEsz) = u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
    };
    auto place = [&](int c) { return (int64_t)(start + c / g.G) * g.ot + (int64_t)(h * g.G + c % g.G) * g.oh; };
    auto put_sums = [&](int c, float mm, float ll) {
        if (!direct) {
            float* ml = g.part_ml + (part + c) * 2;
            ml[0] = mm;
            ml[1] = ll;
        } else if (g.lse) {
            g.lse[(int64_t)(start + c / g.G) * g.heads + h * g.G + c % g.G] = ll == 0.0f ? -INFINITY : (mm + __log2f(ll)) * 0.693147180559945309417f;
        }
    };
    auto share_of = [&](float ll) { return !direct ? 1.0f : ll != 0.0f ? 1.0f / ll : 0.0f; };  // partial results stay sums
    if constexpr (KW == 1) {
        each<NC>([&](auto ctc) {
            constexpr int ct = decltype(ctc)::value;
            const int c = col0 + ct * 16 + lr;
            if (c < C) {
                const int64_t to = place(c);
                const float f = share_of(l[ct]);
                each<DT>([&](auto dt) { put(c, to, decltype(dt)::value * 16 + lg * 4, o[ct][decltype(dt)::value] * f); });
                if (lg == 0) put_sums(c, m[ct], l[ct]);
            }
        });
    } else {
        // Wavefronts with the same columns had different keys: join them, 32 elements of the columns at a time, in two buffers in turn.
        float(*sums)[KW][kWide][kRow] = (float(*)[KW][kWide][kRow])lds;
        const int first = cg * kWide;  // column of the workgroup
        each<NC>([&](auto ctc) {
            constexpr int ct = decltype(ctc)::value;
            if (lg == 0) {
                mls[turn][set * 16 * NC + ct * 16 + lr][0] = m[ct];
                mls[turn][set * 16 * NC + ct * 16 + lr][1] = l[ct];
            }
        });
        __syncthreads();
        if (tid < kWide) {
            float top = -INFINITY, ll = 0.0f, f[KW];
#pragma unroll
            for (int w = 0; w < KW; ++w) top = fmaxf(top, mls[w][tid][0]);
#pragma unroll
            for (int w = 0; w < KW; ++w) {
                f[w] = pow2(mls[w][tid][0] - (top == -INFINITY ? 0.0f : top));
                ll += mls[w][tid][1] * f[w];
            }
#pragma unroll
            for (int w = 0; w < KW; ++w) mls[w][tid][0] = f[w] * share_of(ll);
            if (first + tid < C) put_sums(first + tid, top, ll);
        }
        __syncthreads();
        constexpr int kPer = (kWide * 8 + 255) / 256;  // of a thread: four elements of a column
        int64_t to[kPer];
        each<kPer>([&](auto x) {
            const int c = (tid + decltype(x)::value * 256) / 8;
            to[decltype(x)::value] = place(min(first + c, C - 1));
        });
        float f[NC];
        each<NC>([&](auto ct) { f[decltype(ct)::value] = mls[turn][set * 16 * NC + decltype(ct)::value * 16 + lr][0]; });
        each<D / 32>([&](auto passc) {
            constexpr int pass = decltype(passc)::value, buf = pass & 1;
            each<NC * 2>([&](auto x) {
                constexpr int ct = decltype(x)::value / 2, i = decltype(x)::value % 2;
                *(f32x4*)&sums[buf][turn][set * 16 * NC + ct * 16 + lr][i * 16 + lg * 4] = o[ct][pass * 2 + i] * f[ct];
            });
            __syncthreads();
            each<kPer>([&](auto xc) {
                const int i = tid + decltype(xc)::value * 256, c = i / 8, d = i % 8 * 4;
                if (c < kWide && first + c < C) {
                    f32x4 x = *(f32x4*)&sums[buf][0][c][d];
#pragma unroll
                    for (int w = 1; w < KW; ++w) x += *(f32x4*)&sums[buf][w][c][d];
                    put(first + c, to[decltype(xc)::value], pass * 32 + d, x);
                }
            });
        });
    }
  }
}

template <int D, int KIND>
static void attend_wide(const Shares& r, const AttendArgs& g, hipStream_t st)
{
    const int64_t sets = ((int64_t)g.kv_heads * (r.shares ? r.shares : g.B) + 7) / 8 * 8;
    const dim3 grid((unsigned)(sets * r.groups)), block(256);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, st, g); };
    if (r.sets == 1) {
        if (r.nc == 1) go(attend_kernel<D, KIND, 1, 1>);
        else if (r.nc == 2) go(attend_kernel<D, KIND, 2, 1>);
        else if constexpr (D <= 128) go(attend_kernel<D, KIND, 3, 1>);
    } else r.sets == 2 ? go(attend_kernel<D, KIND, 2, 2>) : go(attend_kernel<D, KIND, 2, 4>);
}

template <int KIND>
static void attend_kind(int D, const Shares& r, const AttendArgs& g, hipStream_t st)
{
    if (D == 64) attend_wide<64, KIND>(r, g, st);
    else if (D == 128) attend_wide<128, KIND>(r, g, st);
    else attend_wide<256, KIND>(r, g, st);
}

void attend_bf16(int D, const Shares& r, const AttendArgs& g, hipStream_t st);
void attend_int8(int D, const Shares& r, const AttendArgs& g, hipStream_t st);
void attend_fp8(int D, const Shares& r, const AttendArgs& g, hipStream_t st);
void attend_f32(int D, const Shares& r, const AttendArgs& g, hipStream_t st);

}  // namespace mmoe
