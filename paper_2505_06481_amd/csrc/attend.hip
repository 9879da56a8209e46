// Attention of drafted tokens over the paged cache: how a call is shared out, and the join of split keys.  The kernel is in
// attend_kernel.h.
#include "attend_kernel.h"

namespace mmoe {

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

static Shares shares(const mmoe_attend_shape& s)
{
    Shares r;
    const int G = s.heads / s.cache.kv_heads, most = s.cache.head_dim > 128 ? 2 : 4;
    const int64_t C = (int64_t)(s.max_drafts < s.T ? s.max_drafts : s.T) * G;
    r.cols = C > 16 * most;
    const int64_t per = r.cols ? (C + 3) / 4 : C;
    r.nc = !r.cols && per <= 16 ? 1 : per <= 32 || most == 2 ? 2 : 4;
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
           ((int64_t)s.cache.kv_heads * s.n_requests + 8) * r.groups <= most / r.nsplit;
}

size_t attend_ws_bytes(const mmoe_attend_shape& s)
{
    const Shares r = shares(s);
    if (r.nsplit == 1) return 256;
    const size_t rows = (size_t)r.nsplit * s.T * s.heads;
    return align256(rows * s.cache.head_dim * 4) + align256(rows * 8);
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
    const bool f32 = s.cache.dtype == MMOE_F32;
    (s.cache.format == MMOE_CACHE_INT8 ? attend_int8 : s.cache.format == MMOE_CACHE_FP8 ? attend_fp8 : f32 ? attend_f32 : attend_bf16)((int)D, r, g, st);
    if (r.nsplit > 1) {
        const int64_t drafts = s.max_drafts < s.T ? s.max_drafts : s.T;
        const dim3 grid((unsigned)((drafts * s.heads + 3) / 4 * s.n_requests)), block(256);
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, st, g); };
        if (D == 64) f32 ? go(attend_join_kernel<64, true>) : go(attend_join_kernel<64, false>);
        else if (D == 128) f32 ? go(attend_join_kernel<128, true>) : go(attend_join_kernel<128, false>);
        else f32 ? go(attend_join_kernel<256, true>) : go(attend_join_kernel<256, false>);
    }
    return launch_status();
}

}  // namespace mmoe
