// Projection shared by the variants with each token's low-rank adapter beside it:
//   Y[t] = X[t] W + scale[a] (X[t] A[a]) B[a],  a = aid[t].
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
// With bf16 storage U is kept as two bf16 parts, the value rounded and what that leaves, [T][2][Rp]: the second product runs
// on the bf16 instruction with 16 bits of U, so the adapter adds no error of its own to the rounding of Y.
// A workgroup takes 16 tokens; its four wavefronts a quarter of K each.  For every adapter among the tokens all 16 are
// multiplied, and the tokens whose adapter it is keep the result.
template <bool F32>
__global__ __launch_bounds__(256) void shrink_kernel(const char* __restrict__ X, int64_t ldx, const int32_t* __restrict__ aid,
                                                     const char* __restrict__ Ap, const float* __restrict__ scale,
                                                     char* __restrict__ U, int T, int K, int Rp, int n)
{
    constexpr int kEsz = F32 ? 4 : 2, kParts = F32 ? 1 : 2;
    __shared__ float part[4][16][17];
    __shared__ int of[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, lr = lane & 15, lg = lane >> 4;
    const int t0 = blockIdx.x * 16;
    if (tid < 16) {
        const int a = t0 + tid < T ? aid[t0 + tid] : -1;
        of[tid] = (unsigned)a < (unsigned)n ? a : -1;
    }
    __syncthreads();
    const int slices = K * kEsz / 64, per = slices / 4;  // 64 bytes of a row each
    const char* x = X + (int64_t)min(t0 + lr, T - 1) * ldx * kEsz + wave * per * 64 + lg * 16;
    for (int i = 0; i < 16; ++i) {
        const int a = of[i];
        bool first = a >= 0;
        for (int j = 0; j < i; ++j) first = first && of[j] != a;
        if (!first) continue;  // uniform
        for (int rb = 0; rb < Rp / 16; ++rb) {
            f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
            const char* w = Ap + (((int64_t)a * (Rp / 16) + rb) * slices + wave * per) * 1024 + lane * 16;
#pragma unroll 4
            for (int s = 0; s < per; ++s)
                acc = mma<F32>(*(const u32x4*)(w + (int64_t)s * 1024), *(const u32x4*)(x + s * 64), acc);
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 4; ++e) part[wave][lg * 4 + e][lr] = acc[e];
            __syncthreads();
            const int tok = tid >> 4, r = tid & 15;
            if (of[tok] == a) {
                const float v = (part[0][r][tok] + part[1][r][tok] + (part[2][r][tok] + part[3][r][tok])) * scale[a];
                const int64_t at = (int64_t)(t0 + tok) * Rp * kParts + rb * 16 + r;
                if (F32) {
                    ((float*)U)[at] = v;
                } else {
                    const uint16_t hi = f32_to_bf16_bits(v);
                    ((uint16_t*)U)[at] = hi;
                    ((uint16_t*)U)[at + Rp] = f32_to_bf16_bits(v - bf16_bits_to_f32(hi));
                }
            }
        }
    }
}

// ---- Y = X W + U B -----------------------------------------------------------------------------------
struct ProjectArgs {
    const char *X, *Wp, *Bp, *U;
    char* Y;
    float* part;         // [splits][T][N] where the reduction is split
    const int32_t* aid;
    int64_t ldx, ldy;
    int T, K, N, Rp, n;
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
// order them can count: kStages - 2 steps' copies may be in flight at a barrier.
template <bool F32, int WM, int WN>
__global__ __launch_bounds__(256, WM * WN > 16 ? 1 : 2) void project_tile_kernel(ProjectArgs g)
{
    constexpr int kEsz = F32 ? 4 : 2, kParts = F32 ? 1 : 2;
    constexpr int kStages = 4, kStep = (WM + WN) * 2048;    // bytes of a step: 2 WM token fragments, then 2 WN of weights
    constexpr int kCopies = (WM + WN) / 2;                  // of a wavefront and step
    static_assert(WM % 2 == 0 && WN % 2 == 0, "copies are shared out evenly");
    __shared__ __attribute__((aligned(1024))) char lds[kStages * kStep];
    __shared__ uint32_t used[kMaxAdapters / 32];

    // XCD x (workgroup id mod 8) takes a run of tiles: eight feature tiles of a token tile, then the next token tile.
    const int all = g.tiles_m * g.tiles_n * g.splits, per = gridDim.x / 8;
    int tile = blockIdx.x % 8 * per + blockIdx.x / 8;
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
    auto copy = [&](int step, int stage, int i) {
        const int at = min(step, last);
        const bool tokens = i < WM / 2;
        const char* base = tokens ? x_base + (int64_t)at * 64 : w_base + ((int64_t)(i - WM / 2) * slices + at) * 1024;
        const uint32_t off = tokens ? x_off[tokens ? i : 0] : w_off;
        const uint32_t dst = lds0 + stage * kStep + (tokens ? wave * (WM / 2) + i : 2 * WM + wave * (WN / 2) + i - WM / 2) * 1024;
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
    auto read = [&](int set, int stage, int i) {
        const int at = i < WM ? wm * WM + i : 2 * WM + wn * WN + i - WM;
        frag[set][i] = *(const u32x4*)(lds + stage * kStep + at * 1024 + lane * 16);
    };
    auto arrived = [](const u32x4& f) { asm volatile("" ::"v"(f)); };
    if (g.n) {  // adapters of the tile's tokens
        if (tid < kMaxAdapters / 32) used[tid] = 0;
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
        for (int i = 0; i < kCopies; ++i) copy(s, s, i);
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((kStages - 1) * kCopies) : "memory");
#pragma unroll
    for (int i = 0; i < WM + WN; ++i) read(0, 0, i);

    for (int t = 0; t <= last; t += kStages) {
        each<kStages>([&](auto uc) {
            constexpr int u = decltype(uc)::value, set = u & 1, kUnits = WM * WN, kReads = WM + WN;
            each<kReads>([&](auto i) { arrived(frag[set][decltype(i)::value]); });
            asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((kStages - 2) * kCopies) : "memory");
            __builtin_amdgcn_sched_barrier(0);
            each<kUnits>([&](auto xc) {
                constexpr int x = decltype(xc)::value;
                multiply(acc[x % WM][x / WM], frag[set][WM + x / WM], frag[set][x % WM]);
                // reads in the first half, copies in the second
                each<kReads>([&](auto ic) {
                    constexpr int i = decltype(ic)::value;
                    if constexpr (i * (kUnits / 2) / kReads == x) read(set ^ 1, (u + 1) % kStages, i);
                });
                each<kCopies>([&](auto ic) {
                    constexpr int i = decltype(ic)::value;
                    if constexpr (kUnits / 2 + i * (kUnits / 2) / kCopies == x) copy(t + u + kStages, u, i);
                });
                __builtin_amdgcn_sched_barrier(0);
            });
        });
    }
    asm volatile("s_waitcnt vmcnt(0)\n\ts_nop 15\n\ts_nop 15" ::: "memory");  // no copy is on its way when the workgroup ends

    // adapters that the tile's tokens use, one by one; tokens of other adapters with zeros
    if (g.n && split == 0) {
        const int rs = g.Rp * kEsz / 64;
        int mine[WM];
        const char* u[WM];
#pragma unroll
        for (int j = 0; j < WM; ++j) {
            const int t = min(t0 + (wm * WM + j) * 16 + lr, g.T - 1);
            mine[j] = g.aid[t];
            u[j] = g.U + (int64_t)t * kParts * g.Rp * kEsz + lg * 16;
        }
        for (int word = 0; word < (g.n + 31) / 32; ++word) {
            uint32_t bits = __builtin_amdgcn_readfirstlane(used[word]);
            while (bits) {
                const int a = word * 32 + __ffs(bits) - 1;
                bits &= bits - 1;
                const char* b = g.Bp + ((int64_t)a * (g.N / 16) + f0 + wn * WN) * rs * 1024 + lane * 16;
                for (int s = 0; s < rs; ++s) {
                    u32x4 wf[WN], uf[WM][kParts];
#pragma unroll
                    for (int i = 0; i < WN; ++i) wf[i] = *(const u32x4*)(b + ((int64_t)i * rs + s) * 1024);
#pragma unroll
                    for (int j = 0; j < WM; ++j)
#pragma unroll
                        for (int p = 0; p < kParts; ++p)
                            uf[j][p] = mine[j] == a ? *(const u32x4*)(u[j] + p * g.Rp * kEsz + s * 64) : u32x4{0, 0, 0, 0};
                    // a vector instruction's result needs its time before a matrix instruction that the compiler does not see reads it
                    asm volatile("s_nop 7" ::: "memory");
                    each<kParts * WM * WN>([&](auto xc) {
                        constexpr int x = decltype(xc)::value, j = x % WM, i = x / WM % WN, p = x / (WM * WN);
                        multiply(acc[j][i], wf[i], uf[j][p]);
                    });
                }
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
        if (g.splits > 1) {
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
}

// Y = the sum of the splits' parts, in their order.
template <bool F32>
__global__ __launch_bounds__(256) void project_sum_kernel(const float* __restrict__ part, char* __restrict__ Y, int64_t ldy, int T, int N,
                                                          int splits)
{
    const int64_t id = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4, all = (int64_t)T * N;
    if (id >= all) return;
    f32x4 v = *(const f32x4*)(part + id);
    for (int s = 1; s < splits; ++s) v += *(const f32x4*)(part + s * all + id);
    const int64_t at = id / N * ldy + id % N;
    if (F32) *(f32x4*)((float*)Y + at) = v;
    else *(u32x2*)((uint16_t*)Y + at) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
}

// Tile and splits of the reduction.
struct ProjectPlan {
    int wm, wn, splits;
};
static ProjectPlan project_plan(const mmoe_project_shape& s)
{
    ProjectPlan p;
    auto tiles = [&](int wm, int wn) { return (int64_t)((s.T + 32 * wm - 1) / (32 * wm)) * (s.d_out / (32 * wn)); };
    if (tiles(8, 8) >= 200) p = {8, 8, 1};
    else if (s.T > 64) p = {4, 4, 1};
    else p = {2, 4, 1};
    const int64_t n = tiles(p.wm, p.wn);
    const int most = s.d_in / 512 > 0 ? s.d_in / 512 : 1;
    if (p.wm < 8)
        while (p.splits < most && n * p.splits < 256) ++p.splits;
    return p;
}

static size_t u_bytes(const mmoe_project_shape& s) { return s.n_adapters ? align256((size_t)s.T * padded_rank(s) * 4) : 0; }  // fp32 or two bf16 parts

static size_t part_bytes(const mmoe_project_shape& s)
{
    const ProjectPlan p = project_plan(s);
    return p.splits > 1 ? align256((size_t)p.splits * s.T * s.d_out * 4) : 0;
}

// What a call of this shape uses.
size_t project_need(const mmoe_project_shape& s) { return u_bytes(s) + part_bytes(s); }

// The most that one of up to this many tokens does.
size_t project_ws_bytes(const mmoe_project_shape& s)
{
    size_t most = 0;
    for (int T = 64;; T += 64) {  // the plan is the same within 64 tokens
        mmoe_project_shape q = s;
        q.T = T < s.T ? T : s.T;
        const size_t b = part_bytes(q);
        if (b > most) most = b;
        if (T >= s.T || T >= 16384) break;  // from there on there are 256 tiles of 128 tokens for any d_out
    }
    return u_bytes(s) + most;
}

template <bool F32>
static void project(const mmoe_project_shape& s, const void* X, const int32_t* aid, const void* Wp, const void* Ap, const void* Bp,
                    const float* scale, void* Y, void* ws, hipStream_t st)
{
    const int64_t ldx = s.ldx ? s.ldx : s.d_in, ldy = s.ldy ? s.ldy : s.d_out;
    const int n = s.n_adapters, rp = n ? padded_rank(s) : 0;
    if (n)
        hipLaunchKernelGGL(shrink_kernel<F32>, dim3((s.T + 15) / 16), dim3(256), 0, st, (const char*)X, ldx, aid, (const char*)Ap, scale,
                           (char*)ws, s.T, s.d_in, rp, n);
    const ProjectPlan p = project_plan(s);
    ProjectArgs g = {(const char*)X, (const char*)Wp, (const char*)Bp, (const char*)ws, (char*)Y, (float*)((char*)ws + u_bytes(s)), aid, ldx, ldy,
                     s.T, s.d_in, s.d_out, rp, n, (s.T + 32 * p.wm - 1) / (32 * p.wm), s.d_out / (32 * p.wn), p.splits};
    const dim3 grid((g.tiles_m * g.tiles_n * g.splits + 7) / 8 * 8), block(256);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, st, g); };
    if (p.wm == 8) go(project_tile_kernel<F32, 8, 8>);
    else if (p.wm == 4) go(project_tile_kernel<F32, 4, 4>);
    else go(project_tile_kernel<F32, 2, 4>);
    if (p.splits > 1)
        hipLaunchKernelGGL(project_sum_kernel<F32>, dim3((unsigned)(((int64_t)s.T * s.d_out / 4 + 255) / 256)), block, 0, st, g.part, (char*)Y, ldy,
                           s.T, s.d_out, p.splits);
}

int launch_project(const mmoe_project_shape& s, const void* X, const int32_t* aid, const void* Wp, const void* Ap, const void* Bp,
                   const float* scale, void* Y, void* ws, hipStream_t st)
{
    if (s.dtype == MMOE_F32) project<true>(s, X, aid, Wp, Ap, Bp, scale, Y, ws, st);
    else project<false>(s, X, aid, Wp, Ap, Bp, scale, Y, ws, st);
    return launch_status();
}

}  // namespace mmoe
