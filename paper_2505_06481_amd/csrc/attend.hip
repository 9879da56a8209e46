// Attention of drafted tokens over the paged cache: how a call is shared out, and the join of split keys.  The kernel is in
// attend_kernel.h.
#include "attend_kernel.h"

namespace mmoe {

constexpr int kMaxShares = 4096;
constexpr int64_t kMostGroups = ((int64_t)1 << 24) - 1;  // workgroups of 256: a launch has fewer than 2^32 threads
constexpr int kMostShared = 1024;  // workgroups of a call whose pages are shared out: two rounds (of 27000 plans 38 would have more); bounds the workspace
constexpr int kManyParts = 8;  // of a request on average: four wavefronts join them (us, 32 heads, attention with the join by one wavefront and by four:
                              // 1 request of 60000 keys 37, 31; 4 of 8000 28.2, 26.8; but 8 tokens of 32 requests 67, 76; 512 of 3 242, 299)

// out = sum 2^(m_w - m) O_w / sum 2^(m_w - m) l_w over the shares w that have keys of the row, in their order.  Parts were written just
// before: 32 requests of 12 tokens, 19 MB of parts, 9.4 us, 2.0 TB/s.
// Joins the parts of a request that several shares have: WPR wavefronts take a (token, head), each every WPR-th part.
template <int D, bool F32, int WPR>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs g)
{
    __shared__ int sums[4][2];
    __shared__ float parts[WPR == 1 ? 1 : 4][D + 1];
    constexpr int kRows = 4 / WPR;  // of a workgroup
    const int tid = threadIdx.x, per = (min(g.max_drafts, g.T) * g.heads + kRows - 1) / kRows, b = blockIdx.x / per;
    const int lane = tid & 63, wave = tid >> 6, mine = wave % WPR;
    const Request r = request_of(g, b);
    const int rows = r.n * g.heads, row0 = blockIdx.x % per * kRows;
    if (row0 >= rows || !r.pages) return;              // uniform
    const int row = min(row0 + wave / WPR, rows - 1);  // token of the request, head; the last one again where there are no more
    int before = 0, all = 0;
    for (int i = tid; i < g.B; i += 256) {
        const int pages = request_of(g, i).pages;
        all += pages;
        if (i < b) before += pages;
    }
#define MMOE_JOIN(OFF) all += lane_xor<OFF>(all), before += lane_xor<OFF>(before)
    MMOE_JOIN(1); MMOE_JOIN(2); MMOE_JOIN(4); MMOE_JOIN(8); MMOE_JOIN(16); MMOE_JOIN(32);
#undef MMOE_JOIN
    if (lane == 0) sums[wave][0] = all, sums[wave][1] = before;
    __syncthreads();
    const int P = sums[0][0] + sums[1][0] + sums[2][0] + sums[3][0], p0 = sums[0][1] + sums[1][1] + sums[2][1] + sums[3][1];
    // shares of the request's first and last page
    const Cut cut(P, g.shares);
    const int w0 = cut.of(p0), w1 = cut.of(p0 + r.pages - 1);
    if (w0 == w1) return;  // written by the share that has it all
    const int64_t t = r.start + row / g.heads;
    const int head = row % g.heads, h = head / g.G, c = row / g.heads * g.G + head % g.G;
    const int slot0 = cut.start(w0) < p0 ? 1 : 0;
    auto part = [&](int w) { return (((int64_t)w * 2 + (w == w0 ? slot0 : 0)) * g.kv_heads + h) * g.columns + c; };
    float top = -INFINITY;
    for (int w = w0 + lane; w <= w1; w += 64) top = fmaxf(top, g.part_ml[part(w) * 2]);
#define MMOE_JOIN(OFF) top = fmaxf(top, lane_xor<OFF>(top))
    MMOE_JOIN(1); MMOE_JOIN(2); MMOE_JOIN(4); MMOE_JOIN(8); MMOE_JOIN(16); MMOE_JOIN(32);
#undef MMOE_JOIN
    const float base = top == -INFINITY ? 0.0f : top;
    constexpr int kPer = D / 64;
    float x[kPer], l = 0.0f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) x[i] = 0.0f;
#pragma unroll 4
    for (int w = w0 + mine; w <= w1; w += WPR) {
        const int64_t at = part(w);
        const float f = pow2(g.part_ml[at * 2] - base);
        l += f * g.part_ml[at * 2 + 1];
#pragma unroll
        for (int i = 0; i < kPer; ++i) x[i] += f * g.part_o[at * D + i * 64 + lane];
    }
    if constexpr (WPR > 1) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) parts[wave][i * 64 + lane] = x[i];
        if (lane == 0) parts[wave][D] = l;
        __syncthreads();
        if (mine) return;
#pragma unroll
        for (int v = 1; v < WPR; ++v) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) x[i] += parts[wave + v][i * 64 + lane];
            l += parts[wave + v][D];
        }
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

// The shares with the least estimated time for `sets` sets of columns at most.
static double shares_for(const mmoe_attend_shape& s, int sets, bool three, Shares& r)  // three: tiles to a wavefront
{
    const int G = s.heads / s.cache.kv_heads;
    const int64_t C = (int64_t)(s.max_drafts < s.T ? s.max_drafts : s.T) * G;
    const int64_t cap = (int64_t)s.max_pages * kPage;
    const int64_t longest = s.max_keys && s.max_keys < cap ? s.max_keys : cap;
    const int64_t sum = s.sum_keys ? s.sum_keys : (int64_t)s.n_requests * longest;
    const int64_t pages = sum / kPage + s.n_requests, most_pages = (longest + kPage - 1) / kPage;
    r.nc = C <= 16 ? 1 : three ? 3 : 2;
    r.sets = C <= 32 || three ? 1 : C <= 64 ? 2 : sets;
    const int wide = 16 * r.nc * r.sets;
    r.groups = (int)((C + wide - 1) / wide);
    // Estimated cycles, fitted to 800 measured times (90 calls of 1 to 100 requests, equal or 2 % to all of the longest, each with up to ten
    // numbers of shares; the choice is within 4 % of the best on average, 30 % at most): a page to a wavefront, which is its requests' latency
    // and the work on NC tiles, or its part of the memory's rate where that is more; a request that a workgroup takes up; the join, by parts
    // and their bytes.  Wavefronts with different keys take pages at once.  us, without shares : with the best number, 32 heads on 8 of
    // 128: 1 request of 8000 keys bf16 38 : 15; 8 of 1200 to 60000 fp8 448 : 117; 6 of 1500, 40 tokens, fp32 69 : 31; but 32 of 80 to 4000, int8 45 : 56;
    // 64 of 80 to 4000, bf16 103 : 112.
    const double wide_heads = s.cache.head_dim / 128.0;
    const bool codes = s.cache.format != MMOE_CACHE_PLAIN, f32 = s.cache.dtype == MMOE_F32;
    const double alone = !three ? 1.0 : codes ? 0.8 : f32 ? 0.7 : 0.9;  // a lone wavefront's page
    const double page = alone * ((codes ? 2200.0 : f32 ? 2550.0 : 2100.0) * (0.6 + 0.4 * wide_heads) + (codes ? 1260.0 : f32 ? 10500.0 : 740.0) * r.nc * wide_heads);
    const double kRequest = three ? 15600.0 : 7800.0;
    constexpr double kJoin = 18800.0, kJoinPart = 73.0, kJoinByte = 1.47e-3, kRate = 3070.0;  // (bytes a cycle)
    const int64_t room = s.cache.head_dim <= 128 && !three ? 512 : 256, heads = (int64_t)s.cache.kv_heads * r.groups;
    const int kept = s.cache.head_dim * (codes ? 1 : (int)elem_size(s.cache.dtype));
    const double bytes = 2.0 * kPage * (kept + (codes ? 4 : 0));                                      // of a page
    const double steps = codes || kept <= 128 ? 1.0 : kept <= 256 || !f32 ? 2.0 : 4.0;                // to a page
    auto work = [&](double n, double one) { return ceil(n * steps * r.sets / 4.0) * one / steps; };  // n pages
    const double even = fmax(work((double)pages * heads / room, page), (double)pages * s.cache.kv_heads * bytes / kRate);  // all of it, spread evenly
    double least = kRequest * ((s.n_requests * heads + room - 1) / room) + fmax(work((double)most_pages, page), even);
    r.shares = 0;
    const int64_t rows = C / G * s.heads;  // of a request: the join's grid
    if (s.n_requests <= kMaxShared && s.n_requests * (int64_t)s.max_pages < (int64_t)1 << 30 && rows * s.n_requests <= kMostGroups) {
        // rounds of resident workgroups, or shares of a few pages
        const int64_t tries[] = {room / heads, 2 * room / heads, 3 * room / heads, 4 * room / heads, pages, pages / 2, pages / 4, pages / 8, pages / 16, pages / 32};
        for (int64_t w : tries) {
            if (w < 2 || w > kMaxShares || w > pages || w * heads > kMostShared) continue;
            const double each = (double)pages / w, taken = 1.0 + (double)s.n_requests / w;  // pages, requests of a share
            const double active = fmin((double)w * heads, (double)room) / r.groups;
            const double one = fmax(page, bytes * active * 4.0 / r.sets / kRate);
            const double parts = fmin(2.0 * w, (double)(w + s.n_requests)) * heads * fmin((double)C, (double)wide) * s.cache.head_dim * 4.0;
            const double time = (double)((w * heads + room - 1) / room) * (taken * (work(each / taken, one) + kRequest)) + kJoin + kJoinPart * w / s.n_requests + kJoinByte * parts;
            if (time < least) least = time, r.shares = (int)w;
        }
    }
    return least;
}

// 32 columns to a wavefront leave room for a second one on its SIMD, whose vector instructions run under the first one's matrix instructions.
// 33 to 48 columns are two sets of them, or three tiles to a lone wavefront, which reads and converts the keys once.  us, two sets : three
// tiles, 32 heads on 8 of 128: 32 requests of 12 tokens over 3000 keys int8 62 : 49, 8 over 60000 fp8 225 : 200, 28 over 1000 fp32 100 : 76; but
// 64 over 700 fp8 31 : 45, 11 of 10 over 2900 int8 40 : 46, 32 over 3000 bf16 79 : 81.  (64 columns so: 60000, fp8 233 : 224, bf16 205 : 228.)
// More than 64 columns: four sets read a page once for 128, two sets and more groups spread few requests over more compute units.  us, four : two: 2
// requests of 100 tokens over 500 keys, heads of 256 51 : 34; 28 of 50 over 400, fp32 64 : 53; 8 of 128 over 1000, int8 47 : 42; but 64 of 32 over 500 40 : 48.
static Shares shares_of(const mmoe_attend_shape& s)
{
    Shares r, other;
    double least = shares_for(s, 2, false, r);
    auto also = [&](int sets, bool three) {
        const double time = shares_for(s, sets, three, other);
        if (time < least) least = time, r = other;
    };
    also(4, false);
    const int64_t C = (int64_t)(s.max_drafts < s.T ? s.max_drafts : s.T) * (s.heads / s.cache.kv_heads);
    if (C > 32 && C <= 48 && s.cache.head_dim <= 128) also(1, true);
    return r;
}

// Whether the grid's size fits.
bool attend_fits(const mmoe_attend_shape& s)
{
    const Shares r = shares_of(s);
    return ((int64_t)s.cache.kv_heads * (r.shares ? r.shares : s.n_requests) + 7) / 8 * 8 * r.groups <= kMostGroups;
}

// Columns of a request at most, and rows of partial results.
static int64_t columns_of(const mmoe_attend_shape& s) { return (int64_t)(s.max_drafts < s.T ? s.max_drafts : s.T) * (s.heads / s.cache.kv_heads); }
static size_t part_rows(const mmoe_attend_shape& s, const Shares& r) { return (size_t)r.shares * 2 * s.cache.kv_heads * columns_of(s); }

static size_t parts_bytes(const mmoe_attend_shape& s, size_t rows) { return 256 + align256(rows * s.cache.head_dim * 4) + align256(rows * 8); }

// What a call of this shape uses.
size_t attend_need(const mmoe_attend_shape& s) { return parts_bytes(s, part_rows(s, shares_of(s))); }

// The most that one of up to these requests, tokens, drafts, pages and keys does: fewer requests may have more shares.  A workgroup of a share has
// 2 * 128 rows of parts at most, and a share is a page or more.
size_t attend_ws_bytes(const mmoe_attend_shape& s)
{
    const int64_t cap = (int64_t)s.max_pages * kPage, most = (int64_t)s.n_requests * cap, C = columns_of(s);
    const int64_t pages = (s.sum_keys ? s.sum_keys : most) / kPage + s.n_requests;
    const int64_t by_shares = 2 * kMostShared * (C < 128 ? C : 128), by_pages = 2 * (pages < kMaxShares ? pages : kMaxShares) * s.cache.kv_heads * C;
    return parts_bytes(s, (size_t)(by_shares < by_pages ? by_shares : by_pages));
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
        auto go = [&](auto kernel, int rows) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)((drafts * s.heads + rows - 1) / rows * s.n_requests)), dim3(256), 0, st, g);
        };
        auto wide = [&](auto d, auto f) {
            constexpr int kD = decltype(d)::value;
            constexpr bool kF = decltype(f)::value;
            if (r.shares >= kManyParts * (int64_t)s.n_requests) go(attend_join_kernel<kD, kF, 4>, 1);
            else go(attend_join_kernel<kD, kF, 1>, 4);
        };
        auto typed = [&](auto d) { f32 ? wide(d, std::true_type{}) : wide(d, std::false_type{}); };
        if (D == 64) typed(std::integral_constant<int, 64>{});
        else if (D == 128) typed(std::integral_constant<int, 128>{});
        else typed(std::integral_constant<int, 256>{});
    }
    return launch_status();
}

}  // namespace mmoe
