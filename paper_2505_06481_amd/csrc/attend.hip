// Attention of drafted tokens over the paged cache: how a call is shared out, and the join of split keys.  The kernel is in
// attend_kernel.h.
#include "attend_kernel.h"

namespace mmoe {

constexpr int kLeastPages = 16;   // of a share
constexpr int kMaxShares = 4096;

// Joins the parts of a request that several shares have: a wavefront takes a (token, head).
template <int D, bool F32>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs g)
{
    __shared__ int sums[256][2];
    const int tid = threadIdx.x, per = (min(g.max_drafts, g.T) * g.heads + 3) / 4, b = blockIdx.x / per;
    const Request r = request_of(g, b);
    const int row = blockIdx.x % per * 4 + (tid >> 6), lane = tid & 63;  // token of the request, head
    if (blockIdx.x % per * 4 >= r.n * g.heads) return;  // uniform
    int before = 0, all = 0;
    for (int i = tid; i < g.B; i += 256) {
        const int pages = request_of(g, i).pages;
        all += pages;
        if (i < b) before += pages;
    }
#define MMOE_JOIN(OFF) all += lane_xor<OFF>(all), before += lane_xor<OFF>(before)
    MMOE_JOIN(1); MMOE_JOIN(2); MMOE_JOIN(4); MMOE_JOIN(8); MMOE_JOIN(16); MMOE_JOIN(32);
#undef MMOE_JOIN
    if (lane == 0) sums[tid >> 6][0] = all, sums[tid >> 6][1] = before;
    __syncthreads();
    const int P = sums[0][0] + sums[1][0] + sums[2][0] + sums[3][0], p0 = sums[0][1] + sums[1][1] + sums[2][1] + sums[3][1];
    if (row >= r.n * g.heads || !r.pages) return;
    // shares of the request's first and last page
    const Cut cut(P, g.shares);
    const int w0 = cut.of(p0), w1 = cut.of(p0 + r.pages - 1);
    if (w0 == w1) return;  // written by the share that has it all
    const int64_t t = r.start + row / g.heads;
    const int head = row % g.heads, h = head / g.G, c = row / g.heads * g.G + head % g.G;
    auto part = [&](int w) {
        const int slot = w == w0 && cut.start(w) < p0 ? 1 : 0;
        return (((int64_t)w * 2 + slot) * g.kv_heads + h) * g.columns + c;
    };
    float top = -INFINITY;
    for (int w = w0 + lane; w <= w1; w += 64)
        top = fmaxf(top, g.part_ml[part(w) * 2]);
#define MMOE_JOIN(OFF) top = fmaxf(top, lane_xor<OFF>(top))
    MMOE_JOIN(1); MMOE_JOIN(2); MMOE_JOIN(4); MMOE_JOIN(8); MMOE_JOIN(16); MMOE_JOIN(32);
#undef MMOE_JOIN
    const float base = top == -INFINITY ? 0.0f : top;
    constexpr int kPer = D / 64;
    float x[kPer], l = 0.0f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) x[i] = 0.0f;
#pragma unroll 4
    for (int w = w0; w <= w1; ++w) {
        const int64_t at = part(w);
        const float f = pow2(g.part_ml[at * 2] - base);
        l += f * g.part_ml[at * 2 + 1];
#pragma unroll
        for (int i = 0; i < kPer; ++i) x[i] += f * g.part_o[at * D + i * 64 + lane];
    }
    const float inv = l != 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int64_t dst = t * g.ot + head * g.oh + i * 64 + lane;
        if (F32) ((float*)g.out)[dst] = x[i] * inv;
        else ((uint16_t*)g.out)[dst] = f32_to_bf16_bits(x[i] * inv);
    }
    if (lane == 0 && g.lse) g.lse[t * g.heads + head] = l == 0.0f ? -INFINITY : (top + __log2f(l)) * 0.693147180559945309417f;
}

static Shares shares_of(const mmoe_attend_shape& s)
{
    Shares r;
    const int G = s.heads / s.cache.kv_heads, most = s.cache.head_dim > 128 ? 2 : 4;
    const int64_t C = (int64_t)(s.max_drafts < s.T ? s.max_drafts : s.T) * G;
    r.cols = C > 16 * most;
    const int64_t per = r.cols ? (C + 3) / 4 : C;
    r.nc = !r.cols && per <= 16 ? 1 : per <= 32 || most == 2 ? 2 : !r.cols && per <= 48 ? 3 : 4;
    const int wide = 16 * r.nc * (r.cols ? 4 : 1);
    r.groups = (int)((C + wide - 1) / wide);
    const int64_t cap = (int64_t)s.max_pages * kPage;
    const int64_t longest = s.max_keys && s.max_keys < cap ? s.max_keys : cap;
    const int64_t sum = s.sum_keys ? s.sum_keys : (int64_t)s.n_requests * longest;
    const int64_t pages = sum / kPage + s.n_requests, most_pages = (longest + kPage - 1) / kPage;
    // workgroups that are resident at once, for each key head and column group
    const int64_t room = 256 * (r.nc == 1 && s.cache.head_dim <= 128 ? 2 : 1), heads = (int64_t)s.cache.kv_heads * r.groups;
    int64_t w = room / heads;
    if (w < s.n_requests) w = s.n_requests;
    if (w > pages / kLeastPages) w = pages / kLeastPages;
    if (w > kMaxShares) w = kMaxShares;
    // One workgroup to a request where the longest request is not what the call would wait for.
    const int64_t rounds = (s.n_requests * heads + room - 1) / room;
    const bool even = most_pages <= kLeastPages || most_pages * room <= pages * heads + (rounds > 1 ? pages * heads / 4 : 0);
    r.shares = even || s.n_requests > kMaxShared || w <= 1 || s.n_requests * (int64_t)s.max_pages >= (int64_t)1 << 30 ? 0 : (int)w;
    return r;
}

// Whether the grids' sizes fit.
bool attend_fits(const mmoe_attend_shape& s)
{
    const Shares r = shares_of(s);
    const int64_t drafts = s.max_drafts < s.T ? s.max_drafts : s.T, most = ((int64_t)1 << 31) - 1;
    return drafts * s.heads < most && (drafts * s.heads + 3) / 4 * s.n_requests <= most &&
           ((int64_t)s.cache.kv_heads * (r.shares ? r.shares : s.n_requests) + 8) * r.groups <= most;
}

// Columns of a request at most, and rows of partial results.
static int64_t columns_of(const mmoe_attend_shape& s) { return (int64_t)(s.max_drafts < s.T ? s.max_drafts : s.T) * (s.heads / s.cache.kv_heads); }
static size_t part_rows(const mmoe_attend_shape& s, const Shares& r) { return (size_t)r.shares * 2 * s.cache.kv_heads * columns_of(s); }

size_t attend_ws_bytes(const mmoe_attend_shape& s)
{
    const size_t rows = part_rows(s, shares_of(s));
    return 256 + align256(rows * s.cache.head_dim * 4) + align256(rows * 8);
}

int launch_attend(const mmoe_attend_shape& s, const void* Q, const int32_t* starts, const int32_t* ctx, const uint64_t* tree,
                  const int32_t* pages, const mmoe_cache& c, void* out, float* lse, void* ws, hipStream_t st)
{
    const Shares r = shares_of(s);
    const int64_t D = s.cache.head_dim;
    AttendArgs g = {(const char*)Q, starts, ctx, tree, pages, (const char*)c.k, (const char*)c.v, c.k_scale, c.v_scale, (char*)out, lse,
                    (float*)ws, (float*)((char*)ws + align256(part_rows(s, r) * D * 4)),
                    s.q_token ? s.q_token : s.heads * D, s.q_head ? s.q_head : D, s.o_token ? s.o_token : s.heads * D,
                    s.o_head ? s.o_head : D, s.T, s.n_requests, s.heads, s.cache.kv_heads, s.heads / s.cache.kv_heads, s.max_pages,
                    s.max_drafts, s.mask_words, s.cache.n_pages, r.groups, r.shares, (int)columns_of(s), s.scale};
    const bool f32 = s.cache.dtype == MMOE_F32;
    (s.cache.format == MMOE_CACHE_INT8 ? attend_int8 : s.cache.format == MMOE_CACHE_FP8 ? attend_fp8 : f32 ? attend_f32 : attend_bf16)((int)D, r, g, st);
    if (r.shares) {
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
