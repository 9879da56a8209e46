// C-ABI entry points of the attention half: argument checks; the work is in project.hip, rotary_cache.hip and attend.hip.
#include <math.h>

#include "attn_internal.h"

namespace mmoe {

static inline bool misaligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

// A stride in elements: 0 (dense), or at least `least` and whole pieces of 16 bytes.
static bool bad_stride(int64_t stride, int64_t least, int dtype)
{
    return stride != 0 && (stride < least || stride > (int64_t)1 << 40 || (stride * (int64_t)elem_size(dtype)) % 16 != 0);
}

// Strides of [T, heads, D].  Either may be the outer one: the larger has to step over what the smaller spans.
static bool bad_strides(int64_t token, int64_t head, int64_t T, int64_t heads, int64_t D, int dtype)
{
    if (bad_stride(token, D, dtype) || bad_stride(head, D, dtype)) return true;
    const int64_t h = head ? head : D, t = token ? token : heads * D;
    return !(t >= (heads - 1) * h + D || h >= (T - 1) * t + D);
}

int check_project(const mmoe_project_shape* s)
{
    if (!s) return MMOE_ERR_NULL;
    if (s->T <= 0 || s->d_in <= 0 || s->d_out <= 0 || s->n_adapters < 0) return MMOE_ERR_DIM;
    if (s->dtype != MMOE_F32 && s->dtype != MMOE_BF16) return MMOE_ERR_DTYPE;
    if (s->d_in % 256 || s->d_out % 256) return MMOE_ERR_MULTIPLE;
    if (s->n_adapters && s->rank <= 0) return MMOE_ERR_DIM;
    if (s->d_in > 65536 || s->d_out > 262144 || s->n_adapters > kMaxAdapters || (s->n_adapters && s->rank > kMaxRank) ||
        s->T > (1 << 24) || (int64_t)s->T * s->d_out >= (int64_t)1 << 40 || s->ldx > kMaxRow || s->ldy > kMaxRow)
        return MMOE_ERR_LIMIT;
    if (bad_stride(s->ldx, s->d_in, s->dtype) || bad_stride(s->ldy, s->d_out, s->dtype)) return MMOE_ERR_STRIDE;
    return MMOE_OK;
}

int check_rotary(const mmoe_rotary_shape* s)
{
    if (!s) return MMOE_ERR_NULL;
    if (s->T <= 0 || s->heads <= 0) return MMOE_ERR_DIM;
    if (s->dtype != MMOE_F32 && s->dtype != MMOE_BF16) return MMOE_ERR_DTYPE;
    if (s->layout != MMOE_ROTARY_HALVES && s->layout != MMOE_ROTARY_NEIGHBOURS) return MMOE_ERR_FORMAT;
    if (s->transpose != 0 && s->transpose != 1) return MMOE_ERR_FORMAT;
    if (s->head_dim <= 0 || s->head_dim > 512 || s->head_dim % 16 || s->rot <= 0 || s->rot > s->head_dim || s->rot % 16)
        return MMOE_ERR_HEAD;
    if (s->heads > 65536 || s->T > (1 << 24)) return MMOE_ERR_LIMIT;
    if (bad_strides(s->x_token, s->x_head, s->T, s->heads, s->head_dim, s->dtype) ||
        bad_strides(s->y_token, s->y_head, s->T, s->heads, s->head_dim, s->dtype))
        return MMOE_ERR_STRIDE;
    return MMOE_OK;
}

int check_cache(const mmoe_cache_shape* s)
{
    if (!s) return MMOE_ERR_NULL;
    if (s->n_pages <= 0 || s->kv_heads <= 0) return MMOE_ERR_DIM;
    if (s->dtype != MMOE_F32 && s->dtype != MMOE_BF16) return MMOE_ERR_DTYPE;
    if (s->format != MMOE_CACHE_PLAIN && s->format != MMOE_CACHE_INT8 && s->format != MMOE_CACHE_FP8) return MMOE_ERR_FORMAT;
    if (s->head_dim != 64 && s->head_dim != 128 && s->head_dim != 256) return MMOE_ERR_HEAD;
    if (s->n_pages > (1 << 25) || s->kv_heads > 1024) return MMOE_ERR_LIMIT;  // places are int32
    return MMOE_OK;
}

static int check_cache_pointers(const mmoe_cache_shape& s, const mmoe_cache* c)
{
    if (!c || !c->k || !c->v) return MMOE_ERR_NULL;
    if (s.format != MMOE_CACHE_PLAIN && (!c->k_scale || !c->v_scale)) return MMOE_ERR_NULL;
    if (misaligned(c->k, 16) || misaligned(c->v, 16) || misaligned(c->k_scale, 16) || misaligned(c->v_scale, 16)) return MMOE_ERR_ALIGN;
    return MMOE_OK;
}

int check_attend(const mmoe_attend_shape* s)
{
    if (!s) return MMOE_ERR_NULL;
    if (int rc = check_cache(&s->cache)) return rc;
    if (s->T <= 0 || s->n_requests <= 0 || s->heads <= 0 || s->max_pages <= 0 || s->max_drafts <= 0 || s->mask_words < 0 ||
        s->max_keys < 0 || s->sum_keys < 0)
        return MMOE_ERR_DIM;
    if (s->cache.format != MMOE_CACHE_PLAIN && s->cache.dtype != MMOE_BF16) return MMOE_ERR_FORMAT;
    if (s->heads % s->cache.kv_heads || s->heads / s->cache.kv_heads > 64) return MMOE_ERR_HEAD;
    if (s->max_pages > (1 << 24) || s->n_requests > (1 << 20) || s->T > (1 << 24) || s->heads > 65536) return MMOE_ERR_LIMIT;
    if (!(fabsf(s->scale) <= 1e30f)) return MMOE_ERR_LIMIT;
    const int D = s->cache.head_dim, dt = s->cache.dtype;
    if (bad_strides(s->q_token, s->q_head, s->T, s->heads, D, dt) || bad_strides(s->o_token, s->o_head, s->T, s->heads, D, dt))
        return MMOE_ERR_STRIDE;
    return attend_fits(*s) ? MMOE_OK : MMOE_ERR_LIMIT;
}

// Turns per position of every pair, in double precision.
static void rotary_frequencies(int rot, double base, int scaling, double factor, double original, double* f, double* magnitude)
{
    const double turn = 2.0 * M_PI;
    *magnitude = 1.0;
    if (scaling == MMOE_SCALE_BASE && rot > 2) base *= pow(factor, rot / (rot - 2.0));
    double lo = 0.0, hi = 0.0;
    if (scaling == MMOE_SCALE_RAMP) {
        auto pair_of = [&](double turns) { return rot * log(original / (turns * turn)) / (2.0 * log(base)); };
        lo = fmax(floor(pair_of(32.0)), 0.0);
        hi = fmin(ceil(pair_of(1.0)), rot - 1.0);
        *magnitude = 0.1 * log(factor) + 1.0;
    }
    for (int i = 0; i < rot / 2; ++i) {
        const double own = pow(base, -2.0 * i / rot);
        double keep = 1.0;
        if (scaling == MMOE_SCALE_LINEAR) keep = 0.0;
        if (scaling == MMOE_SCALE_RAMP) keep = 1.0 - fmin(1.0, fmax(0.0, (i - lo) / fmax(hi - lo, 1e-3)));
        if (scaling == MMOE_SCALE_BANDS) keep = fmin(1.0, fmax(0.0, (original * own / turn - 1.0) / 3.0));
        f[i] = (own * keep + own / factor * (1.0 - keep)) / turn;
    }
}

}  // namespace mmoe

using namespace mmoe;

extern "C" {

size_t mmoe_project_workspace_bytes(const mmoe_project_shape* shape)
{
    return check_project(shape) == MMOE_OK ? project_ws_bytes(*shape) : 0;
}

size_t mmoe_project_packed_rank(const mmoe_project_shape* shape)
{
    return check_project(shape) == MMOE_OK && shape->n_adapters ? (size_t)padded_rank(*shape) : 0;
}

int mmoe_pack_projection(const mmoe_project_shape* shape, const void* W, void* Wp, void* stream)
{
    if (int rc = check_project(shape)) return rc;
    if (!W || !Wp) return MMOE_ERR_NULL;
    if (misaligned(W, 16) || misaligned(Wp, 16)) return MMOE_ERR_ALIGN;
    return launch_pack_pieces(W, Wp, 1, shape->d_in, shape->d_out, shape->d_in, shape->d_out, shape->dtype, (hipStream_t)stream);
}

int mmoe_pack_adapters(const mmoe_project_shape* shape, const void* A, const void* B, void* Ap, void* Bp, void* stream)
{
    if (int rc = check_project(shape)) return rc;
    if (!shape->n_adapters) return MMOE_ERR_DIM;
    if (!A || !B || !Ap || !Bp) return MMOE_ERR_NULL;
    if (misaligned(A, 4) || misaligned(B, 4) || misaligned(Ap, 16) || misaligned(Bp, 16)) return MMOE_ERR_ALIGN;
    const int rp = padded_rank(*shape);
    if (int rc = launch_pack_pieces(A, Ap, shape->n_adapters, shape->d_in, shape->rank, shape->d_in, rp, shape->dtype, (hipStream_t)stream))
        return rc;
    return launch_pack_pieces(B, Bp, shape->n_adapters, shape->rank, shape->d_out, rp, shape->d_out, shape->dtype, (hipStream_t)stream);
}

int mmoe_project(const mmoe_project_shape* shape, const void* X, const int32_t* aid, const void* Wp, const void* Ap, const void* Bp,
                 const float* scale, void* Y, void* ws, size_t ws_bytes, void* stream)
{
    if (int rc = check_project(shape)) return rc;
    if (!X || !Wp || !Y) return MMOE_ERR_NULL;
    if (shape->n_adapters && (!aid || !Ap || !Bp || !scale)) return MMOE_ERR_NULL;
    const size_t need = project_need(*shape);
    if (need && (!ws || ws_bytes < need)) return MMOE_ERR_WORKSPACE;
    if (misaligned(X, 16) || misaligned(Wp, 16) || misaligned(Y, 16) || misaligned(Ap, 16) || misaligned(Bp, 16) ||
        misaligned(aid, 4) || misaligned(scale, 4) || misaligned(ws, 256))
        return MMOE_ERR_ALIGN;
    return launch_project(*shape, X, aid, Wp, Ap, Bp, scale, Y, ws, (hipStream_t)stream);
}

int mmoe_rotary_steps(int32_t rot, double base, int32_t scaling, double factor, int32_t original, uint64_t* steps, float* magnitude)
{
    if (!steps || !magnitude) return MMOE_ERR_NULL;
    if (rot <= 0 || rot > 512 || rot % 16) return MMOE_ERR_HEAD;
    if (scaling < MMOE_SCALE_NONE || scaling > MMOE_SCALE_BANDS) return MMOE_ERR_FORMAT;
    if (!(base > 1.0 && base < 1e12)) return MMOE_ERR_LIMIT;
    if (scaling != MMOE_SCALE_NONE && !(factor >= 1.0 && factor < 1e6)) return MMOE_ERR_LIMIT;
    if (scaling >= MMOE_SCALE_RAMP && original <= 0) return MMOE_ERR_DIM;
    double f[256], m;
    rotary_frequencies(rot, base, scaling, scaling == MMOE_SCALE_NONE ? 1.0 : factor, original, f, &m);
    for (int i = 0; i < rot / 2; ++i) steps[i] = (uint64_t)ldexp(f[i], 64);  // f < 1/6 turn; below 2^53 units the fraction is cut
    *magnitude = (float)m;
    return MMOE_OK;
}

int mmoe_rotary(const mmoe_rotary_shape* shape, const void* X, const int32_t* pos, const uint64_t* steps, void* Y, void* stream)
{
    if (int rc = check_rotary(shape)) return rc;
    if (!X || !pos || !steps || !Y) return MMOE_ERR_NULL;
    if (misaligned(X, 16) || misaligned(Y, 16) || misaligned(pos, 4) || misaligned(steps, 8)) return MMOE_ERR_ALIGN;
    return launch_rotary(*shape, X, pos, steps, Y, (hipStream_t)stream);
}

size_t mmoe_cache_bytes(const mmoe_cache_shape* shape, size_t* scale_bytes)
{
    if (scale_bytes) *scale_bytes = 0;
    if (check_cache(shape) != MMOE_OK) return 0;
    const size_t rows = (size_t)shape->n_pages * shape->kv_heads * kPage;
    if (shape->format == MMOE_CACHE_PLAIN) return rows * shape->head_dim * elem_size(shape->dtype);
    if (scale_bytes) *scale_bytes = rows * sizeof(float);
    return rows * shape->head_dim;
}

int mmoe_cache_append(const mmoe_cache_shape* shape, const mmoe_cache_rows* rows, const void* K, const void* V, const int32_t* places,
                      const mmoe_rotary_shape* rotary, const int32_t* pos, const uint64_t* steps, const mmoe_cache* cache, void* stream)
{
    if (int rc = check_cache(shape)) return rc;
    if (!rows || !K || !V || !places) return MMOE_ERR_NULL;
    if (rows->T <= 0) return MMOE_ERR_DIM;
    if (rows->T > (1 << 24)) return MMOE_ERR_LIMIT;
    if (bad_strides(rows->k_token, rows->k_head, rows->T, shape->kv_heads, shape->head_dim, shape->dtype) ||
        bad_strides(rows->v_token, rows->v_head, rows->T, shape->kv_heads, shape->head_dim, shape->dtype))
        return MMOE_ERR_STRIDE;
    if (rotary) {
        mmoe_rotary_shape r = *rotary;
        r.T = r.heads = 1;
        r.x_token = r.x_head = r.y_token = r.y_head = 0;
        if (int rc = check_rotary(&r)) return rc;
        if (r.head_dim != shape->head_dim) return MMOE_ERR_HEAD;
        if (r.dtype != shape->dtype) return MMOE_ERR_DTYPE;
        if (!pos || !steps) return MMOE_ERR_NULL;
        if (misaligned(pos, 4) || misaligned(steps, 8)) return MMOE_ERR_ALIGN;
    }
    if (int rc = check_cache_pointers(*shape, cache)) return rc;
    if (misaligned(K, 16) || misaligned(V, 16) || misaligned(places, 4)) return MMOE_ERR_ALIGN;
    return launch_cache_append(*shape, *rows, K, V, places, rotary, pos, steps, *cache, (hipStream_t)stream);
}

int mmoe_cache_read(const mmoe_cache_shape* shape, const mmoe_cache* cache, int32_t R, const int32_t* places, void* K, void* V,
                    void* stream)
{
    if (int rc = check_cache(shape)) return rc;
    if (R <= 0) return MMOE_ERR_DIM;
    if (R > (1 << 28)) return MMOE_ERR_LIMIT;
    if (!places || !K || !V) return MMOE_ERR_NULL;
    if (int rc = check_cache_pointers(*shape, cache)) return rc;
    if (misaligned(K, 16) || misaligned(V, 16) || misaligned(places, 4)) return MMOE_ERR_ALIGN;
    return launch_cache_read(*shape, *cache, R, places, K, V, (hipStream_t)stream);
}

size_t mmoe_attend_workspace_bytes(const mmoe_attend_shape* shape)
{
    return check_attend(shape) == MMOE_OK ? attend_ws_bytes(*shape) : 0;
}

int mmoe_attend(const mmoe_attend_shape* shape, const void* Q, const int32_t* starts, const int32_t* ctx, const uint64_t* tree,
                const int32_t* pages, const mmoe_cache* cache, void* out, float* lse, void* ws, size_t ws_bytes, void* stream)
{
    if (int rc = check_attend(shape)) return rc;
    if (!Q || !starts || !ctx || !pages || !out) return MMOE_ERR_NULL;
    if (tree && shape->mask_words <= 0) return MMOE_ERR_DIM;
    if (int rc = check_cache_pointers(shape->cache, cache)) return rc;
    if (!ws || ws_bytes < attend_need(*shape)) return MMOE_ERR_WORKSPACE;
    if (misaligned(Q, 16) || misaligned(out, 16) || misaligned(starts, 4) || misaligned(ctx, 4) || misaligned(pages, 4) ||
        misaligned(tree, 8) || misaligned(lse, 4) || misaligned(ws, 256))
        return MMOE_ERR_ALIGN;
    return launch_attend(*shape, Q, starts, ctx, tree, pages, *cache, out, lse, ws, (hipStream_t)stream);
}

}  // extern "C"
