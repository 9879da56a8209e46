// Projection shared by the variants with each token's low-rank adapter beside it:
//   Y[t] = X[t] W + scale[a] (X[t] A[a]) B[a],  a = aid[t].
//
// The adapters' two products are thin: they ride on the large one.  U = scale X A is made by a kernel of its own (or beside the large
// product, where that is cut into parts), and U B is added to the accumulators of X W.  Prefill is bound by the matrix cores
// (8192 x 4096 x 6144 bf16, 2 adapters of rank 32: 345 us, 1.2 PFLOP/s; 321 without adapters, a library product alone 302 to 320), fp32 by
// its matrix rate (4096 cubed 918 us, 150 TFLOP/s), few tokens by the weights they read (64 x 4096 x 6144, 48 adapters:
// 21 us, 3.2 TB/s over both launches) and by the launches (3 tokens: 4.8 + 4.0 us).
#include "attn_internal.h"

namespace mmoe {

// ---- packing, once --------------------------------------------------------------------------------
// in [S, K, N] -> pieces [S][Np/16][Kp/c][64][16 bytes], zeros beyond K and N.  A thread gathers a piece.
template <typename T>
__global__ __launch_bounds__(256) void pack_pieces_kernel(const T* __restrict__ in, u32x4* __restrict__ out, int K, int N, int Kp,
                                                          int Np, int64_t pieces)
{
    constexpr int E = 16 / sizeof(T);
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= pieces) return;
    const int lane = id & 63;
    const int64_t frag = id >> 6;
    const int nk = Kp / (4 * E);
    const int k0 = (int)(frag % nk) * 4 * E + (lane >> 4) * E;
    const int64_t row = frag / nk * 16 + (lane & 15);  // over all S matrices of Np rows
    const int64_t s = row / Np;
    const int n = (int)(row % Np);
    union {
        T e[E];
        u32x4 v;
    } p;
#pragma unroll
    for (int j = 0; j < E; ++j) p.e[j] = k0 + j < K && n < N ? in[(s * K + k0 + j) * N + n] : (T)0;
    out[id] = p.v;
}

int launch_pack_pieces(const void* in, void* out, int S, int K, int N, int Kp, int Np, int dtype, hipStream_t st)
{
    const int64_t pieces = (int64_t)S * Kp * Np * (int64_t)elem_size(dtype) / 16;
    const dim3 grid((unsigned)((pieces + 255) / 256)), block(256);
    if (dtype == MMOE_BF16)
        hipLaunchKernelGGL(pack_pieces_kernel<uint16_t>, grid, block, 0, st, (const uint16_t*)in, (u32x4*)out, K, N, Kp, Np, pieces);
    else
        hipLaunchKernelGGL(pack_pieces_kernel<float>, grid, block, 0, st, (const float*)in, (u32x4*)out, K, N, Kp, Np, pieces);
    return launch_status();
}

// ---- U = scale (X A) ----------------------------------------------------------------------------------
// With bf16 storage U is kept as two bf16 parts, its first 8 bits and what they leave, [T][2][Rp]: the second product runs
// on the bf16 instruction with 16 bits of U, so the adapter adds no error of its own to the rounding of Y.  Both parts have the sign of U and neither
// is zero or infinite where U is not (down to 2^-110), so that an infinity in B gives one of its sign, not NaN.
//
// A workgroup takes the tokens of one adapter among a chunk of the batch, 32 at a time; its four wavefronts a quarter of K each.
// (32 tokens fill two columns' tiles: fewer read the adapter more often, more leave compute units idle.  8192 tokens of 4096, 2 adapters: 26 us,
// 2.6 TB/s: four rounds of loads, each a memory latency.)
// A token is read once and an adapter once for each chunk that has tokens of it.  Adapters are numbered by `group`: their own
// number, or, where they are more than the tokens of a chunk, that of the chunk's first token that uses it.
struct ShrinkArgs {
    const char *X, *Ap;
    const int32_t* aid;
    const float* scale;
    char* U;
    int64_t ldx;
    int T, K, R, Rp, n;
    int chunk;        // tokens
    int groups;       // of a chunk
    int pairs;        // of blocks of 16 ranks: a workgroup takes one
    int turns;        // workgroups that take 32 tokens of an adapter and chunk in turn
    bool by_token;    // groups are tokens (chunks of up to kScan)
};
constexpr int kScan = 512;  // tokens looked through at once
struct TokenList {
    int list[kScan];
    int counts[4];
};
struct ShrinkLds {
    float part[4][32][33];
    TokenList tokens;
};

// The tokens t0 .. t0 + count - 1 (at most kScan) with adapter a, ascending, to `list`; returns how many.  a = n stands for none.
__device__ __forceinline__ int tokens_of(const int32_t* aid, int t0, int count, int a, int n, TokenList& l)
{
    constexpr int kPer = kScan / 256;  // runs of 64 tokens of a wavefront
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint64_t who[kPer];
    bool mine[kPer];
    int have = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int at = (wave * kPer + i) * 64 + lane;
        const int x = n && at < count ? aid[t0 + at] : -1;
        mine[i] = at < count && ((unsigned)x < (unsigned)n ? x == a : a == n);
        who[i] = __ballot(mine[i]);
        have += __popcll(who[i]);
    }
    if (lane == 0) l.counts[wave] = have;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (w < wave) before += l.counts[w];
        all += l.counts[w];
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        if (mine[i]) l.list[before + __popcll(who[i] & (((uint64_t)1 << lane) - 1))] = t0 + (wave * kPer + i) * 64 + lane;
        before += __popcll(who[i]);
    }
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(all);
}

// The adapter of a group (n: none), or -1 if the group has no tokens to look for.
__device__ __forceinline__ int adapter_of(const int32_t* aid, int t0, int count, int group, bool by_token, int n)
{
    if (!by_token) return group;
    if (group >= count) return -1;
    const int x = aid[t0 + group], a = (unsigned)x < (unsigned)n ? x : n;
    bool first = true;  // of the tokens with this adapter
    for (int i = threadIdx.x & 63; i < group; i += 64) {
        const int y = aid[t0 + i];
        if (((unsigned)y < (unsigned)n ? y : n) == a) first = false;
    }
    return __all(first) ? a : -1;
}

// v = hi + lo, 2^-16 of v apart at most; hi is cut, not rounded: rounded, it would be infinite above bf16's largest number.
__device__ __forceinline__ void split_bf16(float v, uint16_t& hi, uint16_t& lo)
{
    const uint32_t bits = __float_as_uint(v);
    hi = (uint16_t)(bits >> 16);
    const float left = v - bf16_bits_to_f32(hi);
    lo = f32_to_bf16_bits(left);
    if (left == 0.0f && fabsf(v) >= 0x1p-110f) lo = (uint16_t)((hi & 0x8000) | 0x0080);  // 2^-126
    if (!(fabsf(v) < INFINITY)) lo = fabsf(v) == INFINITY ? hi : (uint16_t)0;            // NaN: the first part's
}

template <bool F32, int RB>
__device__ __forceinline__ void shrink_tiles(const ShrinkArgs& g, ShrinkLds& lds, int a, int rb0, int cols, int at, int count)
{
    constexpr int kEsz = F32 ? 4 : 2, kParts = F32 ? 1 : 2;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lr = lane & 15, lg = lane >> 4;
    const int slices = g.K * kEsz / 64, per = slices / 4;  // 64 bytes of a row each
    const char* x[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) x[j] = g.X + (int64_t)lds.tokens.list[at + min(j * 16 + lr, count - 1)] * g.ldx * kEsz + wave * per * 64 + lg * 16;
    const char* w = g.Ap + (((int64_t)a * (g.Rp / 16) + rb0) * slices + wave * per) * 1024 + lane * 16;
    f32x4 acc[RB][2];
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const bool two = count > 16;  // uniform
    auto slice = [&](auto qc, int s) {  // slices s .. s + Q - 1, their loads together
        constexpr int Q = decltype(qc)::value;
        u32x4 xf[Q][2], wf[Q][RB];
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            xf[q][0] = *(const u32x4*)(x[0] + (s + q) * 64);
            if (two) xf[q][1] = *(const u32x4*)(x[1] + (s + q) * 64);
#pragma unroll
            for (int i = 0; i < RB; ++i) wf[q][i] = *(const u32x4*)(w + ((int64_t)i * slices + s + q) * 1024);
        }
#pragma unroll
        for (int q = 0; q < Q; ++q)
#pragma unroll
            for (int i = 0; i < RB; ++i) {
                acc[i][0] = mma<F32>(wf[q][i], xf[q][0], acc[i][0]);
                if (two) acc[i][1] = mma<F32>(wf[q][i], xf[q][1], acc[i][1]);
            }
    };
    int s = 0;
    for (; s + 8 <= per; s += 8) slice(std::integral_constant<int, 8>{}, s);
    if (s + 4 <= per) slice(std::integral_constant<int, 4>{}, s), s += 4;
    if (s < per) slice(std::integral_constant<int, 2>{}, s);  // (K is a multiple of 256, eight slices: per is even)
    __syncthreads();  // the sums of the tiles before have been read
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) lds.part[wave][i * 16 + lg * 4 + e][j * 16 + lr] = acc[i][j][e];
    __syncthreads();
    const float f = g.scale[a];
    // cols: those of U from rb0 on; the padding's are zeros (not the sums of padded A's zeros, which an infinite X makes NaN)
    const int ranks = min(g.R - rb0 * 16, RB * 16);
    for (int i = tid; i < count * cols; i += 256) {
        const int tok = i / cols, r = i % cols;
        const float v = r < ranks ? (lds.part[0][r][tok] + lds.part[1][r][tok] + (lds.part[2][r][tok] + lds.part[3][r][tok])) * f : 0.0f;
        const int64_t to = (int64_t)lds.tokens.list[at + tok] * g.Rp * kParts + rb0 * 16 + r;
        if (F32) {
            ((float*)g.U)[to] = v;
        } else {
            uint16_t hi, lo;
            split_bf16(v, hi, lo);
            ((uint16_t*)g.U)[to] = hi;
            ((uint16_t*)g.U)[to + g.Rp] = lo;
        }
    }
}

template <bool F32>
__device__ __forceinline__ void shrink_body(const ShrinkArgs& g, ShrinkLds& lds, int group, int chunk, int rb, int turn)
{
    const int t0 = chunk * g.chunk, t1 = min(t0 + g.chunk, g.T);
    const int a = adapter_of(g.aid, t0, t1 - t0, group, g.by_token, g.n);
    if (a < 0 || a >= g.n) return;  // uniform
    const int real = (g.R + 15) / 16;                            // blocks of 16 that hold ranks; this workgroup's are rb and rb + 1
    const int cols = rb + 2 < real ? 32 : g.Rp - rb * 16;
    for (int t = t0; t < t1; t += kScan) {
        __syncthreads();  // the list before has been used
        const int count = tokens_of(g.aid, t, min(kScan, t1 - t), a, g.n, lds.tokens);
        for (int at = turn * 32; at < count; at += g.turns * 32)
            if (rb + 1 < real) shrink_tiles<F32, 2>(g, lds, a, rb, cols, at, min(32, count - at));
            else shrink_tiles<F32, 1>(g, lds, a, rb, cols, at, min(32, count - at));
    }
}

template <bool F32>
__global__ __launch_bounds__(256) void shrink_kernel(ShrinkArgs g)
{
    __shared__ ShrinkLds lds;
    shrink_body<F32>(g, lds, blockIdx.y, blockIdx.x, blockIdx.z % g.pairs * 2, blockIdx.z / g.pairs);
}

// ---- Y = X W + U B -----------------------------------------------------------------------------------
struct ProjectArgs {
    const char *X, *Wp, *Bp, *U;
    char* Y;
    float* part;         // not null: [splits][T][N] parts of X W, which another kernel adds up and the adapters to them
    const int32_t* aid;
    int64_t ldx, ldy;
    int T, K, N, R, Rp, n;
    int tiles_m, tiles_n, splits;
};

typedef __attribute__((address_space(3))) void* lds_ptr;

// Tile: 32 WM tokens x 32 WN features by four wavefronts, two by two, each 16 WM x 16 WN: weights are the row operand, tokens the
// column one.  A step is 64 bytes of a row: 32 k (16 of fp32).
//
// Both operands go from memory to LDS without passing registers (global_load_lds, 1 KB an instruction) into a ring of
// kStages steps, in the order in which lanes hold them: LDS reads are 1 KB in a row, without conflicts.  Iteration t
//   waits until its fragments (read from LDS during t - 1) are in registers and its share of step t + 1's copies has landed;
//   passes the barrier: then step t + 1 is whole, and nobody reads the stage of step t any more;
//   multiplies step t, reads step t + 1's fragments, and copies step t + kStages into the stage of t.
// The copies are in assembly and nothing else in the loop is a vector memory instruction, so the waits that
// order them can count: kStages - 2 steps' copies may be in flight at a barrier.  What a step takes: at project_plan.
template <int WM, int WN>
struct TileLds {
    static constexpr int kStep = (WM + WN) * 2048;  // bytes of a step: 2 WM token fragments, then 2 WN of weights
    // steps in the ring: four, but 128 x 256 leaves room for two workgroups (with two 29.5 -> 36.4 us at 2000 x 1024 x 4096; eight of
    // 64 x 128 fetch more than a short k has: 64 x 256 x 65536 in 21.2 us, with four 16.7)
    static constexpr int kStages = WM == 4 && WN == 8 ? 3 : 4;
    __attribute__((aligned(1024))) char ring[kStages * kStep];
    uint32_t used[kMaxAdapters / 32];
    uint32_t odd[4][kMaxAdapters / 32];  // adapters with infinities or NaN among a wavefront's features
};

// Adds to a wavefront's part of Y what the adapters in `odd` give: 64 bytes of rank at a time, those that are not finite.
// Tokens t0 .., blocks of 16 features from f0 on.
template <bool F32, int WM, int WN>
__device__ __forceinline__ void add_odd(const ProjectArgs& g, const uint32_t* odd, int t0, int f0)
{
    constexpr int kEsz = F32 ? 4 : 2, kParts = F32 ? 1 : 2;
    int lane = threadIdx.x & 63;
    asm("" : "+v"(lane));  // nothing of this is worked out ahead
    const int lr = lane & 15, lg = lane >> 4, rs = g.Rp * kEsz / 64;
    __threadfence_block();  // other lanes wrote Y
    for (int word = 0; word < (g.n + 31) / 32; ++word)
        for (uint32_t bits = __builtin_amdgcn_readfirstlane(odd[word]); bits; bits &= bits - 1) {
            const int a = word * 32 + __ffs(bits) - 1;
            const char* b = g.Bp + ((int64_t)a * (g.N / 16) + f0) * rs * 1024 + lane * 16;
#pragma unroll 1
            for (int x = 0; x < WM * WN; ++x) {
                const int j = x / WN, i = x % WN, t = min(t0 + j * 16 + lr, g.T - 1);
                f32x4 own = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
                for (int s = 0; s < rs; ++s) {
                    f32x4 zero = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                    for (int o = 0; o < WN; ++o) zero = mma<F32>(*(const u32x4*)(b + ((int64_t)o * rs + s) * 1024), u32x4{0, 0, 0, 0}, zero);
                    if (!__any(zero[0] + zero[1] + zero[2] + zero[3] != 0.0f)) continue;  // is in Y
                    const char* u = g.U + (int64_t)t * kParts * g.Rp * kEsz + s * 64 + lg * 16;
                    for (int p = 0; p < kParts; ++p)
                        own = mma<F32>(*(const u32x4*)(b + ((int64_t)i * rs + s) * 1024), *(const u32x4*)(u + p * g.Rp * kEsz), own);
                }
                if (t0 + j * 16 + lr < g.T && g.aid[t] == a)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int64_t at = t * g.ldy + (f0 + i) * 16 + lg * 4 + e;
                        if (F32) ((float*)g.Y)[at] += own[e];
                        else ((uint16_t*)g.Y)[at] = f32_to_bf16_bits(bf16_bits_to_f32(((uint16_t*)g.Y)[at]) + own[e]);
                    }
            }
        }
}

template <bool F32, int WM, int WN>
__device__ __forceinline__ void tile_body(const ProjectArgs& g, TileLds<WM, WN>& shared, int block, int blocks)
{
    constexpr int kEsz = F32 ? 4 : 2, kParts = F32 ? 1 : 2;
    constexpr int kStages = TileLds<WM, WN>::kStages, kStep = TileLds<WM, WN>::kStep;
    constexpr int kCopies = (WM + WN) / 2;                  // of a wavefront and step
    static_assert(WM % 2 == 0 && WN % 2 == 0, "copies are shared out evenly");
    char* const lds = shared.ring;
    uint32_t* const used = shared.used;

    // XCD x (workgroup id mod 8) takes a run of tiles: eight feature tiles of a token tile, then the next token tile.
    const int all = g.tiles_m * g.tiles_n * g.splits, per = blocks / 8;
    int tile = block % 8 * per + block / 8;
    if (tile >= all) return;  // uniform
    const int split = tile % g.splits;
    tile /= g.splits;
    const int band = tile / (g.tiles_m * 8), in_band = tile % (g.tiles_m * 8), wide = min(8, g.tiles_n - band * 8);
    const int tm = in_band / wide, tn = band * 8 + in_band % wide;
    const int t0 = tm * 32 * WM, f0 = tn * 2 * WN;  // first token, first block of 16 features

    const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave & 1, wn = wave >> 1;
    const int slices = g.K * kEsz / 64;
    const int k0 = (int)((int64_t)(slices / 8) * split / g.splits) * 8, k1 = (int)((int64_t)(slices / 8) * (split + 1) / g.splits) * 8;
    const int last = k1 - k0 - 1;

    // copy i of this wavefront: token fragments wave*WM/2 + i, then weight fragments wave*WN/2 + i - WM/2
    uint32_t x_off[WM / 2];
    const char* x_base = g.X + (int64_t)t0 * g.ldx * kEsz + (int64_t)k0 * 64;
#pragma unroll
    for (int i = 0; i < WM / 2; ++i) {
        const int row = min((wave * (WM / 2) + i) * 16 + lr, g.T - 1 - t0);
        x_off[i] = (uint32_t)(row * g.ldx * kEsz) + lg * 16;
    }
    const char* w_base = g.Wp + ((int64_t)(f0 + wave * (WN / 2)) * slices + k0) * 1024;
    const uint32_t w_off = lane * 16;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr)lds;
    auto copy = [&](int step, int stage, int i) {  // stage: byte offset in the ring
        const int at = min(step, last);
        const bool tokens = i < WM / 2;
        const char* base = tokens ? x_base + (int64_t)at * 64 : w_base + ((int64_t)(i - WM / 2) * slices + at) * 1024;
        const uint32_t off = tokens ? x_off[tokens ? i : 0] : w_off;
        const uint32_t dst = lds0 + stage + (tokens ? wave * (WM / 2) + i : 2 * WM + wave * (WN / 2) + i - WM / 2) * 1024;
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(off), "s"(base), "s"(dst) : "m0", "memory");
    };

    f32x4 acc[WM][WN];
#pragma unroll
    for (int j = 0; j < WM; ++j)
#pragma unroll
        for (int i = 0; i < WN; ++i) acc[j][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    // accumulators stay in AGPRs: the instruction is written out
    auto multiply = [&](f32x4& c, const u32x4& w, const u32x4& x) {
        if constexpr (F32) {
#pragma unroll
            for (int e = 0; e < 4; ++e) asm volatile("v_mfma_f32_16x16x4_f32 %0, %1, %2, %0" : "+a"(c) : "v"(w[e]), "v"(x[e]));
        } else {
            asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(w), "v"(x));
        }
    };

    u32x4 frag[2][WM + WN];
    const char* const lds_x = lds + wm * WM * 1024 + lane * 16;
    const char* const lds_w = lds + (2 * WM + wn * WN) * 1024 + lane * 16;
    auto read = [&](int set, int stage, int i) {
        frag[set][i] = *(const u32x4*)(i < WM ? lds_x + stage + i * 1024 : lds_w + stage + (i - WM) * 1024);
    };
    auto arrived = [](const u32x4& f) { asm volatile("" ::"v"(f)); };
    if (g.n && !g.part) {  // adapters of the tile's tokens
        if (tid < kMaxAdapters / 32) used[tid] = 0;
        if (lane < kMaxAdapters / 32) shared.odd[wave][lane] = 0;
        __syncthreads();
        for (int t = t0 + tid; t < min(t0 + 32 * WM, g.T); t += 256) {
            const int a = g.aid[t];
            if ((unsigned)a < (unsigned)g.n) atomicOr(&used[a >> 5], 1u << (a & 31));
        }
        __syncthreads();
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int s = 0; s < kStages; ++s)
#pragma unroll
        for (int i = 0; i < kCopies; ++i) copy(s, s * kStep, i);
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((kStages - 1) * kCopies) : "memory");
#pragma unroll
    for (int i = 0; i < WM + WN; ++i) read(0, 0, i);

    int stage = 0;
    for (int t = 0; t <= last; t += 2) {  // (an even number of steps: eight slices to 256 k)
        each<2>([&](auto uc) {
            const int next = stage == (kStages - 1) * kStep ? 0 : stage + kStep;
            constexpr int u = decltype(uc)::value, set = u, kUnits = WM * WN, kReads = WM + WN;
            each<kReads>([&](auto i) { arrived(frag[set][decltype(i)::value]); });
            asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((kStages - 2) * kCopies) : "memory");
            __builtin_amdgcn_sched_barrier(0);
            each<kUnits>([&](auto xc) {
                constexpr int x = decltype(xc)::value;
                multiply(acc[x % WM][x / WM], frag[set][WM + x / WM], frag[set][x % WM]);
                // reads in the first half, copies in the second
                each<kReads>([&](auto ic) {
                    constexpr int i = decltype(ic)::value;
                    if constexpr (i * (kUnits / 2) / kReads == x) read(set ^ 1, next, i);
                });
                each<kCopies>([&](auto ic) {
                    constexpr int i = decltype(ic)::value;
                    if constexpr (kUnits / 2 + i * (kUnits / 2) / kCopies == x) copy(t + u + kStages, stage, i);
                });
                __builtin_amdgcn_sched_barrier(0);
            });
            stage = next;
        });
    }
    asm volatile("s_waitcnt vmcnt(0)\n\ts_nop 15\n\ts_nop 15" ::: "memory");  // no copy is on its way when the workgroup ends

    // Adapters that the tile's tokens use, one by one: tokens of other adapters with zeros, fragments without any not at all.  A token's
    // U is its own adapter's, read once; the weights of the next adapter are on their way while this one's are multiplied.
    // Zeros keep other tokens apart where the weights are finite; 64 bytes of rank that are not are left for the end (`odd`).
    bool odd = false;
    if (g.n && !g.part) {
        const int rs = g.Rp * kEsz / 64;
        int mine[WM];
#pragma unroll
        for (int j = 0; j < WM; ++j) mine[j] = g.aid[min(t0 + (wm * WM + j) * 16 + lr, g.T - 1)];
        for (int s = 0; s < rs; ++s) {
            u32x4 uf[WM][kParts], wf[WN], ahead[WN];
#pragma unroll
            for (int j = 0; j < WM; ++j)
#pragma unroll
                for (int p = 0; p < kParts; ++p)
                    uf[j][p] = *(const u32x4*)(g.U + ((int64_t)min(t0 + (wm * WM + j) * 16 + lr, g.T - 1) * kParts + p) * g.Rp * kEsz + s * 64 + lg * 16);
            int word = 0;
            uint32_t bits = __builtin_amdgcn_readfirstlane(used[0]);
            auto next = [&]() {  // of the tile's adapters; -1: no more
                while (!bits && ++word < (g.n + 31) / 32) bits = __builtin_amdgcn_readfirstlane(used[word]);
                if (!bits) return -1;
                const int a = word * 32 + __ffs(bits) - 1;
                bits &= bits - 1;
                return a;
            };
            auto fetch = [&](int a) {
                const char* b = g.Bp + (((int64_t)max(a, 0) * (g.N / 16) + f0 + wn * WN) * rs + s) * 1024 + lane * 16;
                each<WN>([&](auto i) { ahead[decltype(i)::value] = *(const u32x4*)(b + (int64_t)decltype(i)::value * rs * 1024); });
            };
            int a = next();
            if (a >= 0) fetch(a);
            while (a >= 0) {
                each<WN>([&](auto i) { wf[decltype(i)::value] = ahead[decltype(i)::value]; });
                f32x4 zero = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                each<WN>([&](auto i) { zero = mma<F32>(wf[decltype(i)::value], u32x4{0, 0, 0, 0}, zero); });
                const int then = next();
                fetch(then);
                if (__any(zero[0] + zero[1] + zero[2] + zero[3] != 0.0f)) {
                    if (lane == 0) shared.odd[wave][a >> 5] |= 1u << (a & 31);
                    odd = true;
                    a = then;
                    continue;
                }
                each<WM>([&](auto jc) {
                    constexpr int j = decltype(jc)::value;
                    if (!__any(mine[j] == a)) return;  // uniform
                    u32x4 u[kParts];
#pragma unroll
                    for (int p = 0; p < kParts; ++p) u[p] = mine[j] == a ? uf[j][p] : u32x4{0, 0, 0, 0};
                    // (by the builtin: between branches the compiler has to know which registers a matrix instruction still writes)
                    each<kParts * WN>([&](auto xc) {
                        constexpr int i = decltype(xc)::value % WN, p = decltype(xc)::value / WN;
                        acc[j][i] = mma<F32>(wf[i], u[p], acc[j][i]);
                    });
                });
                a = then;
            }
        }
        asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
    }
#pragma unroll
    for (int j = 0; j < WM; ++j)
#pragma unroll
        for (int i = 0; i < WN; ++i) asm volatile("" : "+a"(acc[j][i]));

    // A lane has four consecutive features of a token in each block.  bf16: two blocks are packed and exchanged between neighbouring
    // lane groups, after which lane group lg holds features 8 (lg/2) .. +7 of block lg%2.
#pragma unroll
    for (int j = 0; j < WM; ++j) {
        const int t = t0 + (wm * WM + j) * 16 + lr;
        if (g.part) {
            float* y = g.part + ((int64_t)split * g.T + t) * g.N + (f0 + wn * WN) * 16 + lg * 4;
            if (t < g.T)
#pragma unroll
                for (int i = 0; i < WN; ++i) *(f32x4*)(y + i * 16) = acc[j][i];
        } else if constexpr (F32) {
            float* y = (float*)g.Y + t * g.ldy + (f0 + wn * WN) * 16 + lg * 4;
            if (t < g.T)
#pragma unroll
                for (int i = 0; i < WN; ++i) *(f32x4*)(y + i * 16) = acc[j][i];
        } else {
            uint16_t* y = (uint16_t*)g.Y + t * g.ldy + (f0 + wn * WN) * 16 + (lg & 1) * 16 + (lg >> 1) * 8;
#pragma unroll
            for (int p = 0; p < WN / 2; ++p) {
                const f32x4 a = acc[j][2 * p], c = acc[j][2 * p + 1];
                const u32x2 s0 = __builtin_amdgcn_permlane16_swap(pack_bf16(a[0], a[1]), pack_bf16(c[0], c[1]), false, false);
                const u32x2 s1 = __builtin_amdgcn_permlane16_swap(pack_bf16(a[2], a[3]), pack_bf16(c[2], c[3]), false, false);
                if (t < g.T) *(u32x4*)(y + p * 32) = u32x4{s0[0], s1[0], s0[1], s1[1]};
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    if (odd) add_odd<F32, WM, WN>(g, shared.odd[wave], t0 + wm * WM * 16, f0 + wn * WN);
}

template <bool F32, int WM, int WN>
__global__ __launch_bounds__(256, WM * WN > 32 || WM == 2 ? 1 : 2) void project_tile_kernel(ProjectArgs g)
{
    __shared__ TileLds<WM, WN> lds;
    tile_body<F32, WM, WN>(g, lds, blockIdx.x, gridDim.x);
}

// Few tokens: the parts of X W, and U beside them in the same launch.
template <bool F32, int WM, int WN>
__global__ __launch_bounds__(256, WM * WN > 32 || WM == 2 ? 1 : 2) void project_parts_kernel(ProjectArgs g, ShrinkArgs u, int tiles)
{
    __shared__ union {
        TileLds<WM, WN> tile;
        ShrinkLds shrink;
    } lds;
    if ((int)blockIdx.x < tiles) tile_body<F32, WM, WN>(g, lds.tile, blockIdx.x, tiles);
    else {
        const int id = blockIdx.x - tiles, pair = id % u.pairs, turn = id / u.pairs % u.turns, of = id / (u.pairs * u.turns);
        shrink_body<F32>(u, lds.shrink, of % u.groups, of / u.groups, pair * 2, turn);
    }
}

// Few tokens: Y = the parts of X W, in their order, + U B.  A workgroup takes tokens of one adapter (or of none) among kScan, 16 of
// every `sixteens` times 16, and 256 features, 64 to a wavefront.  Bound by the latency of a chain (tokens, their list, parts), so parts
// are loaded four at a time, and few tokens by the B of their adapters (64 tokens of 6144, 48 adapters of rank 16, four parts: 7.6 us).
template <bool F32>
__global__ __launch_bounds__(256) void project_join_kernel(ProjectArgs g, bool by_token, int sixteens)
{
    constexpr int kEsz = F32 ? 4 : 2, kParts = F32 ? 1 : 2;
    __shared__ TokenList tokens;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lr = lane & 15, lg = lane >> 4;
    const int t0 = blockIdx.z / sixteens * kScan, some = min(kScan, g.T - t0);
    const int a = adapter_of(g.aid, t0, some, blockIdx.y, by_token, g.n);
    if (a < 0) return;  // uniform
    const int count = tokens_of(g.aid, t0, some, a, g.n, tokens);
    const int nb = (blockIdx.x * 4 + wave) * 4, rs = a < g.n ? g.Rp * kEsz / 64 : 0;
    const char* b = g.Bp + ((int64_t)a * (g.N / 16) + nb) * rs * 1024 + lane * 16;
    for (int at = blockIdx.z % sixteens * 16; at < count; at += sixteens * 16) {
        const int64_t t = tokens.list[min(at + lr, count - 1)];
        const float* part = g.part + t * g.N + nb * 16 + lg * 4;
        const char* u = g.U + t * kParts * g.Rp * kEsz + lg * 16;
        u32x4 uf[kParts], wf[4];
        auto fetch = [&](int s) {
#pragma unroll
            for (int p = 0; p < kParts; ++p) uf[p] = *(const u32x4*)(u + p * g.Rp * kEsz + s * 64);
            const bool ranks = (s * 4 + lg) * (16 / kEsz) < g.R;  // the padding's are zeros, and not read
#pragma unroll
            for (int i = 0; i < 4; ++i) wf[i] = ranks ? *(const u32x4*)(b + ((int64_t)i * rs + s) * 1024) : u32x4{0, 0, 0, 0};
        };
        if (rs) fetch(0);
        f32x4 acc[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        auto add = [&](auto qc, int s) {  // parts s .. s + Q - 1, their loads together
            constexpr int Q = decltype(qc)::value;
            f32x4 x[Q][4];
#pragma unroll
            for (int q = 0; q < Q; ++q)
#pragma unroll
                for (int i = 0; i < 4; ++i) x[q][i] = *(const f32x4*)(part + (int64_t)(s + q) * g.T * g.N + i * 16);
#pragma unroll
            for (int q = 0; q < Q; ++q)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[i] += x[q][i];
        };
        int s = 0;
        for (; s + 4 <= g.splits; s += 4) add(std::integral_constant<int, 4>{}, s);
        if (s + 2 <= g.splits) add(std::integral_constant<int, 2>{}, s), s += 2;
        if (s < g.splits) add(std::integral_constant<int, 1>{}, s);
        for (int s = 0; s < rs; ++s) {
            if (s) fetch(s);
#pragma unroll
            for (int p = 0; p < kParts; ++p)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[i] = mma<F32>(wf[i], uf[p], acc[i]);
        }
        if (at + lr < count)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                char* y = g.Y + (t * g.ldy + (nb + i) * 16 + lg * 4) * kEsz;
                if (F32) *(f32x4*)y = acc[i];
                else *(u32x2*)y = u32x2{pack_bf16(acc[i][0], acc[i][1]), pack_bf16(acc[i][2], acc[i][3])};
            }
    }
}

// Few tokens run in two launches: parts of X W beside U, then their join with U B.  More in two as well: U, then tiles
// that add U B themselves.  (Parts still pay at 2800 tokens: 2813 x 4096 x 4864, 16 adapters of 64 140 us in one part, 154 whole; their
// workspace ends at kFewTokens.)
constexpr int kFewTokens = 4096;
// One workgroup for all tokens of an adapter in a look is no choice: 512 x 4096 x 512, one adapter, 25 -> 162 us; 4096 x 4096 x 256 39 -> 194.
static int shrink_chunk(int n, int most) { return 32 * n < most ? 32 * n : most; }
struct ProjectPlan {
    int wm, wn, splits;
    bool few;
};

// The plan with the least estimated time, in cycles.  The constants are fitted to 1200 measured times, every tile and number of parts at
// 44 shapes (1 to 5000 tokens, 256 to 4096 k, both types); at 28 others the plan is within 3 % of the best on average, 14 % at most.  One size
// does not fit all: us of 8x8, 4x8, 4x4 and 2x4, whole and in parts (the plan's first), 64 x 4096 x 6144 with 48 adapters 2x4/4 21.5,
// 4x4/4 21.7, 4x8/8 25.7, 2x4/0 45.9; 2000 x 4096 x 4096 4x8/0 76, 4x4/0 97, 8x8/0 102, 8x8/2 97; 8192 x 4096 x 6144
// 8x8/0 345, 4x8/0 378, 4x4/0 501, 2x4/0 600.
static ProjectPlan project_plan(const mmoe_project_shape& s)
{
    struct Tile {
        int wm, wn;
        double alone, two, ends;  // cycles of a step, alone on its compute unit; of two beside one another; of a tile's beginning and end
    };
    static const Tile tiles[] = {{8, 8, 1430.0, 0.0, 13500.0}, {4, 8, 880.0, 1640.0, 10200.0}, {4, 4, 600.0, 1340.0, 5900.0}, {2, 4, 400.0, 850.0, 5500.0}};
    // a launch more; bytes of parts a cycle; a part of the join; a round of making U; an adapter of a tile, and
    // 64 bytes of its rank (12 adapters of 128, 2034 x 1792 x 4608: 129 us whole, 93 with the adapters in the join; of 16 71 either way)
    constexpr double kLaunch = 6700.0, kBytes = 1680.0, kPart = 800.0, kRound = 12500.0, kAdapter = 300.0, kRanks = 2500.0;
    const bool f32 = s.dtype == MMOE_F32;
    const int slices = s.d_in / (f32 ? 16 : 32), ranks = s.n_adapters ? padded_rank(s) / (f32 ? 16 : 32) : 0;
    const int T = (s.T + 31) / 32 * 32, most = s.T > kFewTokens ? 0 : s.d_in / 256 < 16 ? s.d_in / 256 : 16;
    const int chunk = s.n_adapters ? shrink_chunk(s.n_adapters, kScan) : kScan;
    ProjectPlan best = {8, 8, 1, false};
    double least = 1e30;
    for (const Tile& t : tiles) {
        const int64_t n = (int64_t)((T + 32 * t.wm - 1) / (32 * t.wm)) * (s.d_out / (32 * t.wn));
        const double matrix = f32 ? t.wm * t.wn * 135.0 : 0.0;  // fp32 is bound by its matrix rate
        for (int splits = 0; splits <= most; ++splits) {        // 0: not in parts
            const int64_t wgs = splits ? n * splits : n, room = t.two > 0.0 ? 512 : 256, full = wgs / room, rest = wgs % room;
            // beside the parts run the workgroups that make U: a round of their own where the last one has no room for them, and a tile
            // shares its compute unit with one of them where it has
            const int64_t beside = splits && s.n_adapters ? (s.n_adapters < T ? s.n_adapters : T) * ((T + chunk - 1) / chunk) * ((s.rank + 31) / 32) : 0;
            const double steps = (double)slices / (splits ? splits : 1);
            const double alone = (t.alone > matrix ? t.alone : matrix) * steps + t.ends;
            const double two = (t.two > 2.0 * matrix ? t.two : 2.0 * matrix) * steps + t.ends;
            double time = full * (room == 512 ? two : alone);
            if (rest) time += room == 512 && rest + beside > 256 ? two : alone;
            if (beside && (rest ? rest : room) + beside > room) time += kRound * (((rest ? rest : room) + beside - 1) / room);
            if (splits) time += kLaunch + kPart * splits + (1.7 * splits + 1.0) * T * s.d_out * 4.0 / kBytes;
            else if (s.n_adapters) time += 2.0 * kLaunch + (kAdapter + kRanks * ranks) * (s.n_adapters < 32 * t.wm ? s.n_adapters : 32 * t.wm);
            if (time < least) least = time, best = {t.wm, t.wn, splits ? splits : 1, splits > 0};
        }
    }
    return best;
}

static size_t u_bytes(const mmoe_project_shape& s) { return s.n_adapters ? align256((size_t)s.T * padded_rank(s) * 4) : 0; }  // fp32 or two bf16 parts

static size_t part_bytes(const mmoe_project_shape& s)
{
    const ProjectPlan p = project_plan(s);
    return p.few ? align256((size_t)p.splits * s.T * s.d_out * 4) : 0;
}

// What a call of this shape uses.
size_t project_need(const mmoe_project_shape& s) { return u_bytes(s) + part_bytes(s); }

// The most that one of up to this many tokens does: parts are of kFewTokens tokens at most and of 256 k at least.
size_t project_ws_bytes(const mmoe_project_shape& s)
{
    size_t most = 0;
    for (int T = 32;; T += 32) {  // the plan is the same within 32 tokens
        mmoe_project_shape q = s;
        q.T = T < s.T ? T : s.T;
        const size_t b = part_bytes(q);
        if (b > most) most = b;
        if (T >= s.T || T >= kFewTokens) break;
    }
    return u_bytes(s) + most;
}

template <bool F32>
static void project(const mmoe_project_shape& s, const void* X, const int32_t* aid, const void* Wp, const void* Ap, const void* Bp,
                    const float* scale, void* Y, void* ws, hipStream_t st)
{
    const int64_t ldx = s.ldx ? s.ldx : s.d_in, ldy = s.ldy ? s.ldy : s.d_out;
    const int n = s.n_adapters, rp = n ? padded_rank(s) : 0;
    const ProjectPlan p = project_plan(s);
    ProjectArgs g = {(const char*)X, (const char*)Wp, (const char*)Bp, (const char*)ws, (char*)Y, p.few ? (float*)((char*)ws + u_bytes(s)) : nullptr, aid,
                     ldx, ldy, s.T, s.d_in, s.d_out, s.rank, rp, n, (s.T + 32 * p.wm - 1) / (32 * p.wm), s.d_out / (32 * p.wn), p.splits};
    ShrinkArgs u = {(const char*)X, (const char*)Ap, aid, scale, (char*)ws, ldx, s.T, s.d_in, s.rank, rp, n, s.T, n, (s.rank + 31) / 32, 1, false};
    const int tiles = (g.tiles_m * g.tiles_n * g.splits + 7) / 8 * 8;
    const dim3 block(256);
    if (p.few) {
        const int chunk = s.T < kScan ? s.T : kScan, chunks = (s.T + kScan - 1) / kScan;
        const bool by_token = n + 1 > chunk;
        u.by_token = by_token;
        // U: about 32 tokens of an adapter to a workgroup, so that it is done before the tiles are
        u.chunk = by_token ? chunk : shrink_chunk(n, chunk);
        u.groups = by_token ? chunk : n;
        // (two, where few adapters leave them room beside the tiles: us with one and two, 200 x 2048 x 2048, 3 adapters 20.6, 18.7, in blocks
        // 24.7, 19.5; 400, 8 20.1, 19.4; but 2000 x 4096 x 1024, 16 adapters 41, 47, in blocks 64, 61)
        if (!by_token && u.chunk >= 64 && n <= 8) u.turns = 2;
        const dim3 grid(tiles + (n ? u.groups * u.pairs * u.turns * ((s.T + u.chunk - 1) / u.chunk) : 0));
        auto parts = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, st, g, u, tiles); };
        if (p.wm == 8) parts(project_parts_kernel<F32, 8, 8>);
        else if (p.wn == 8) parts(project_parts_kernel<F32, 4, 8>);
        else if (p.wm == 4) parts(project_parts_kernel<F32, 4, 4>);
        else parts(project_parts_kernel<F32, 2, 4>);
        // twice as many workgroups to an adapter as its even share of the tokens has sixteens (200 x 2048 x 2048 18.7 -> 17.2; 4000 x 1024 x 1024, 32
        // adapters in blocks 52.4 -> 48.7)
        const int groups = by_token ? chunk : n + 1, most = (chunk + 15) / 16,
                  even = (chunk + 16 * groups - 1) / (16 * groups), sixteens = 2 * even < most ? 2 * even : most;
        hipLaunchKernelGGL(project_join_kernel<F32>, dim3(s.d_out / 256, groups, chunks * sixteens), block, 0, st, g, by_token, sixteens);
        return;
    }
    if (n) {
        // about 512 workgroups: chunks of 32 tokens and more.  (One chunk: 8192 x 4096 x 6144, 2 adapters 330 -> 1717 us, 32 adapters 401 -> 512.)
        const int chunks = n >= 512 ? 1 : 512 / n;
        u.chunk = (s.T + chunks - 1) / chunks;
        if (u.chunk < 32) u.chunk = 32;
        // An adapter's tokens may follow one another and be most of a chunk: up to four workgroups to them.  (8192 x 4096 x 1024, us with one and
        // four: 32 adapters in blocks 152, 100, in turns of chance 105, 105; 8 in blocks 112, 92.  Over two looks the looking costs more: 20000
        // tokens, 500 adapters 66, 129.)
        u.turns = u.chunk > 2 * kScan ? 1 : u.chunk < 128 ? u.chunk / 32 : 4;
        hipLaunchKernelGGL(shrink_kernel<F32>, dim3((s.T + u.chunk - 1) / u.chunk, n, u.pairs * u.turns), block, 0, st, u);
    }
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(tiles), block, 0, st, g); };
    if (p.wm == 8) go(project_tile_kernel<F32, 8, 8>);
    else if (p.wn == 8) go(project_tile_kernel<F32, 4, 8>);
    else if (p.wm == 4) go(project_tile_kernel<F32, 4, 4>);
    else go(project_tile_kernel<F32, 2, 4>);
}

int launch_project(const mmoe_project_shape& s, const void* X, const int32_t* aid, const void* Wp, const void* Ap, const void* Bp,
                   const float* scale, void* Y, void* ws, hipStream_t st)
{
    if (s.dtype == MMOE_F32) project<true>(s, X, aid, Wp, Ap, Bp, scale, Y, ws, st);
    else project<false>(s, X, aid, Wp, Ap, Bp, scale, Y, ws, st);
    return launch_status();
}

}  // namespace mmoe
