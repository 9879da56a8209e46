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
// A wavefront computes 64 tokens x 16 features; weights are the row operand.  After X W, the adapters that the
// 64 tokens use are added one by one, tokens of other adapters with a U of zero.
template <bool F32>
__global__ __launch_bounds__(256) void project_kernel(const char* __restrict__ X, int64_t ldx, const int32_t* __restrict__ aid,
                                                      const char* __restrict__ Wp, const char* __restrict__ Bp,
                                                      const char* __restrict__ U, char* __restrict__ Y, int64_t ldy, int T, int K,
                                                      int N, int Rp, int n)
{
    constexpr int kEsz = F32 ? 4 : 2, kParts = F32 ? 1 : 2, NT = 4;
    __shared__ uint32_t used[kMaxAdapters / 32];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, lr = lane & 15, lg = lane >> 4;
    const int t0 = blockIdx.y * 64, nb = blockIdx.x * 4 + wave;
    if (n) {
        if (tid < kMaxAdapters / 32) used[tid] = 0;
        __syncthreads();
        if (tid < 64 && t0 + tid < T) {
            const int a = aid[t0 + tid];
            if ((unsigned)a < (unsigned)n) atomicOr(&used[a >> 5], 1u << (a & 31));
        }
        __syncthreads();
    }
    const int slices = K * kEsz / 64;
    const char* x[NT];
    int mine[NT];
    f32x4 acc[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int t = min(t0 + j * 16 + lr, T - 1);
        x[j] = X + (int64_t)t * ldx * kEsz + lg * 16;
        mine[j] = n ? aid[t] : -1;
        acc[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    const char* w = Wp + (int64_t)nb * slices * 1024 + lane * 16;
#pragma unroll 4
    for (int s = 0; s < slices; ++s) {
        const u32x4 wf = *(const u32x4*)(w + (int64_t)s * 1024);
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[j] = mma<F32>(wf, *(const u32x4*)(x[j] + s * 64), acc[j]);
    }
    const int rs = Rp * kEsz / 64;
    for (int word = 0; word < (n + 31) / 32; ++word) {
        uint32_t bits = used[word];
        while (bits) {
            const int a = word * 32 + __ffs(bits) - 1;
            bits &= bits - 1;
            const char* b = Bp + ((int64_t)a * (N / 16) + nb) * rs * 1024 + lane * 16;
            for (int s = 0; s < rs; ++s) {
                const u32x4 wf = *(const u32x4*)(b + s * 1024);
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int part = 0; part < kParts; ++part) {
                        u32x4 u = {0, 0, 0, 0};
                        if (mine[j] == a)
                            u = *(const u32x4*)(U + ((int64_t)min(t0 + j * 16 + lr, T - 1) * kParts + part) * Rp * kEsz + s * 64 + lg * 16);
                        acc[j] = mma<F32>(wf, u, acc[j]);
                    }
            }
        }
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int t = t0 + j * 16 + lr;
        if (t >= T) continue;
        char* y = Y + ((int64_t)t * ldy + nb * 16 + lg * 4) * kEsz;
        if (F32) *(f32x4*)y = acc[j];
        else *(u32x2*)y = u32x2{pack_bf16(acc[j][0], acc[j][1]), pack_bf16(acc[j][2], acc[j][3])};
    }
}

size_t project_ws_bytes(const mmoe_project_shape& s)
{
    return s.n_adapters ? align256((size_t)s.T * padded_rank(s) * 4) : 0;  // U, in fp32 or two bf16 parts
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
    hipLaunchKernelGGL(project_kernel<F32>, dim3(s.d_out / 64, (s.T + 63) / 64), dim3(256), 0, st, (const char*)X, ldx, aid,
                       (const char*)Wp, (const char*)Bp, (const char*)ws, (char*)Y, ldy, s.T, s.d_in, s.d_out, rp, n);
}

int launch_project(const mmoe_project_shape& s, const void* X, const int32_t* aid, const void* Wp, const void* Ap, const void* Bp,
                   const float* scale, void* Y, void* ws, hipStream_t st)
{
    if (s.dtype == MMOE_F32) project<true>(s, X, aid, Wp, Ap, Bp, scale, Y, ws, st);
    else project<false>(s, X, aid, Wp, Ap, Bp, scale, Y, ws, st);
    return launch_status();
}

}  // namespace mmoe
