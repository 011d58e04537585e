// C-ABI layer of the reader operators: argument checks, scratch and launches.  See include/w2v.h.
#include <cmath>
#include <cstring>

#include "w2v_handle.h"
#include "w2v_reader.h"

using namespace w2v;

namespace {

bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

int32_t launched(w2v_handle *h, int k, const char *what)
{
    if (k < 0) return fail(h, W2V_ERR_CUDA, what, cudaGetLastError());
    h->launches += (uint64_t)k;
    return W2V_OK;
}

int32_t check_norm(w2v_handle *h, uint64_t rows, uint32_t d, uint32_t x_type, uint32_t y_type)
{
    if (d < 1 || d > kNormMaxD) return fail(h, W2V_ERR_ARG, "d must be in 1..8192");
    if (rows >= (1ull << 40)) return fail(h, W2V_ERR_ARG, "rows must be below 2^40");
    if (x_type > kF16 || y_type > kF16) return fail(h, W2V_ERR_ARG, "types must be W2V_TYPE_F32, W2V_TYPE_BF16 or W2V_TYPE_F16");
    if (x_type != y_type && x_type != kF32) return fail(h, W2V_ERR_ARG, "y must have the type of x unless x is W2V_TYPE_F32");
    return W2V_OK;
}

// Do two arrays at one address have their rows at the same places?  (Otherwise rows lie over others that are not read yet.)
bool same_rows(uint64_t rows, uint32_t a_type, uint64_t a_stride, uint32_t b_type, uint64_t b_stride)
{
    return a_type == b_type && (rows < 2 || a_stride == b_stride);
}

// First distances of a side's n buckets: n/2 buckets of one distance each, then bucket n/2 + k starts at
// ceil(e (reach/e)^(k/(n-e))), e = n/2.  The last bit of the power is forgiven (1e-12), so that a power
// that is a whole number counts as that number.
void bucket_starts(uint32_t n, uint32_t reach, int32_t *start)
{
    const uint32_t e = n / 2;
    for (uint32_t i = 0; i < e; ++i) start[i] = (int32_t)i;
    for (uint32_t k = 0; e + k < n; ++k) {
        const long double x = (long double)e * powl((long double)reach / (long double)e, (long double)k / (long double)(n - e));
        start[e + k] = (int32_t)ceill(x * (1.0L - 1e-12L));
    }
}

int32_t check_buckets(w2v_handle *h, uint32_t buckets, uint32_t reach, uint32_t two_sided)
{
    if (two_sided > 1) return fail(h, W2V_ERR_ARG, "two_sided must be 0 or 1");
    if (buckets < 2 || buckets > kMaxBuckets) return fail(h, W2V_ERR_ARG, "buckets must be 0 or in 2..64");
    if (two_sided && (buckets < 4 || buckets % 2)) return fail(h, W2V_ERR_ARG, "two-sided buckets must be an even number of at least 4");
    const uint32_t n = two_sided ? buckets / 2 : buckets;
    if (reach <= n / 2 || reach > kMaxReach) return fail(h, W2V_ERR_ARG, "reach must be above half of a side's buckets and at most 1024");
    return W2V_OK;
}

int32_t check_window(w2v_handle *h, const w2v_window *w, const float *bias, BucketStarts *b)
{
    if (!w) return fail(h, W2V_ERR_ARG, "the window description is NULL");
    if (w->type != kBF16 && w->type != kF16) return fail(h, W2V_ERR_ARG, "type must be W2V_TYPE_BF16 or W2V_TYPE_F16");
    if (w->heads < 1 || w->heads > 1024 || w->kv_heads < 1 || w->heads % w->kv_heads)
        return fail(h, W2V_ERR_ARG, "heads must be in 1..1024 and a multiple of kv_heads");
    if (w->head_dim < 8 || w->head_dim > kMaxHeadDim || w->head_dim % 8)
        return fail(h, W2V_ERR_ARG, "head_dim must be a multiple of 8 in 8..128");
    if (w->left >= (1u << 30) || w->right >= (1u << 30)) return fail(h, W2V_ERR_ARG, "left and right must be below 2^30");
    if (w->sinks > kMaxSinks) return fail(h, W2V_ERR_ARG, "sinks must be at most 64");
    if (!(w->scale > 0.f) || std::isinf(w->scale)) return fail(h, W2V_ERR_ARG, "scale must be positive and finite");
    if (!aligned(bias, 4)) return fail(h, W2V_ERR_ARG, "bias must be aligned to its elements");
    std::memset(b, 0, sizeof(*b));
    if (w->buckets) {
        const int32_t rc = check_buckets(h, w->buckets, w->reach, w->two_sided);
        if (rc != W2V_OK) return rc;
        if (!bias) return fail(h, W2V_ERR_ARG, "bias is NULL but buckets is not 0");
        b->n = w->two_sided ? w->buckets / 2 : w->buckets;
        b->two_sided = w->two_sided;
        bucket_starts(b->n, w->reach, b->start);
    } else if (bias) {
        return fail(h, W2V_ERR_ARG, "bias given but buckets is 0");
    }
    return W2V_OK;
}

// One [n][heads][dim] operand: 16-byte accesses need aligned rows.
int32_t check_rows(w2v_handle *h, const void *p, uint64_t stride, uint64_t width, const char *what)
{
    if (!p) return fail(h, W2V_ERR_ARG, what);
    if (!aligned(p, 16) || stride % 8 || stride < width || stride >= (1ull << 32)) return fail(h, W2V_ERR_ARG, what);
    return W2V_OK;
}

int32_t fill_attend(w2v_handle *h, const w2v_window *w, uint64_t n, const int32_t *spans, const float *bias, AttendParams *p)
{
    std::memset(p, 0, sizeof(*p));
    const int32_t rc = check_window(h, w, bias, &p->b);
    if (rc != W2V_OK) return rc;
    if (n >= (1ull << 31) - 256) return fail(h, W2V_ERR_ARG, "n must be below 2^31 - 256");
    if (n && (!spans || !aligned(spans, 8))) return fail(h, W2V_ERR_ARG, "spans must be 8-byte aligned and not NULL");
    if (((n + kAttendTile - 1) / kAttendTile) * w->heads >= (1ull << 31)) return fail(h, W2V_ERR_ARG, "n times heads must be below 2^38");
    p->spans = reinterpret_cast<const int2 *>(spans);
    p->bias = bias;
    p->n = (int64_t)n;
    p->heads = w->heads; p->kv_heads = w->kv_heads; p->dim = w->head_dim;
    p->left = (int32_t)w->left; p->right = (int32_t)w->right; p->sinks = (int32_t)w->sinks;
    p->scale = w->scale;
    return W2V_OK;
}

}  // namespace

extern "C" {

int32_t w2v_layer_norm(w2v_handle *h, uint64_t rows, uint32_t d, const void *x, uint64_t x_stride, uint32_t x_type,
                       const float *gamma, const float *beta, float eps, void *y, uint64_t y_stride, uint32_t y_type,
                       float *mean, float *rstd)
{
    if (!h) return W2V_ERR_ARG;
    int32_t rc = check_norm(h, rows, d, x_type, y_type);
    if (rc != W2V_OK) return rc;
    if (!gamma || !beta || (rows && (!x || !y))) return fail(h, W2V_ERR_ARG, "x, y, gamma or beta is NULL");
    if (x_stride < d || y_stride < d) return fail(h, W2V_ERR_ARG, "strides must be at least d");
    if (!aligned(x, type_size(x_type)) || !aligned(y, type_size(y_type)) || !aligned(gamma, 4) || !aligned(beta, 4) || !aligned(mean, 4) || !aligned(rstd, 4))
        return fail(h, W2V_ERR_ARG, "x, y, gamma, beta, mean and rstd must be aligned to their elements");
    if (rows && x == y && !same_rows(rows, x_type, x_stride, y_type, y_stride))
        return fail(h, W2V_ERR_ARG, "y may be x only with the same type and stride");
    if (!(eps >= 0.f) || std::isinf(eps)) return fail(h, W2V_ERR_ARG, "eps must be finite and not negative");
    DeviceGuard g(h->device);
    NormParams p;
    std::memset(&p, 0, sizeof(p));
    p.x = x; p.y = y; p.gamma = gamma; p.beta = beta; p.mean = mean; p.rstd = rstd;
    p.rows = rows; p.ldx = x_stride; p.ldy = y_stride; p.d = d; p.eps = eps;
    if ((rc = ensure_error_word(h)) != W2V_OK) return rc;
    return launched(h, launch_norm(p, x_type, y_type, h->tc_error, h->sms, h->stream), "layer norm launch");
}

int32_t w2v_layer_norm_backward(w2v_handle *h, uint64_t rows, uint32_t d, const void *dy, uint64_t dy_stride, uint32_t y_type,
                                const void *x, uint64_t x_stride, uint32_t x_type, const float *gamma, const float *mean,
                                const float *rstd, void *dx, uint64_t dx_stride, float *dgamma, float *dbeta)
{
    if (!h) return W2V_ERR_ARG;
    int32_t rc = check_norm(h, rows, d, x_type, y_type);
    if (rc != W2V_OK) return rc;
    if (!gamma || !dgamma || !dbeta || (rows && (!x || !dy || !dx || !mean || !rstd)))
        return fail(h, W2V_ERR_ARG, "x, dy, dx, gamma, mean, rstd, dgamma or dbeta is NULL");
    if (x_stride < d || dy_stride < d || dx_stride < d) return fail(h, W2V_ERR_ARG, "strides must be at least d");
    if (!aligned(x, type_size(x_type)) || !aligned(dx, type_size(x_type)) || !aligned(dy, type_size(y_type)) || !aligned(gamma, 4) ||
        !aligned(dgamma, 4) || !aligned(dbeta, 4) || !aligned(mean, 4) || !aligned(rstd, 4))
        return fail(h, W2V_ERR_ARG, "arrays must be aligned to their elements");
    if (rows && ((dx == dy && !same_rows(rows, x_type, dx_stride, y_type, dy_stride)) || (dx == x && !same_rows(rows, x_type, dx_stride, x_type, x_stride))))
        return fail(h, W2V_ERR_ARG, "dx may be dy or x only with the same type and stride");
    DeviceGuard g(h->device);
    NormParams p;
    std::memset(&p, 0, sizeof(p));
    p.x = x; p.dy = dy; p.dx = dx; p.gamma = gamma;
    p.mean = const_cast<float *>(mean); p.rstd = const_cast<float *>(rstd);
    p.rows = rows; p.ldx = x_stride; p.ldy = dy_stride; p.ld_dx = dx_stride; p.d = d;
    const uint32_t blocks = norm_backward_blocks(rows, d, h->sms);
    if ((rc = ensure_error_word(h)) != W2V_OK) return rc;
    if ((rc = grow(h, &h->reader_ws, &h->reader_ws_cap, (uint64_t)blocks * 2 * d * sizeof(float) + 16, true)) != W2V_OK) return rc;
    p.part = reinterpret_cast<float *>(h->reader_ws);
    return launched(h, launch_norm_backward(p, x_type, y_type, dgamma, dbeta, blocks, h->tc_error, h->sms, h->stream), "layer norm backward launch");
}

int32_t w2v_sentence_spans(w2v_handle *h, const int32_t *tokens, uint64_t n, int32_t *spans)
{
    if (!h) return W2V_ERR_ARG;
    if (n >= (1ull << 31) - 256) return fail(h, W2V_ERR_ARG, "n must be below 2^31 - 256");
    if (n && (!tokens || !spans || !aligned(spans, 8) || !aligned(tokens, 4)))
        return fail(h, W2V_ERR_ARG, "tokens or spans is NULL, or spans is not 8-byte aligned");
    DeviceGuard g(h->device);
    const int32_t rc = grow(h, &h->reader_ws, &h->reader_ws_cap, spans_tiles(n) * 8 + 16, true);
    if (rc != W2V_OK) return rc;
    return launched(h, launch_spans(tokens, n, (uint32_t)h->vocab, reinterpret_cast<int32_t *>(h->reader_ws),
                                    reinterpret_cast<int2 *>(spans), h->stream), "sentence spans launch");
}

int32_t w2v_bucket_starts(uint32_t buckets, uint32_t reach, uint32_t two_sided, int32_t *starts)
{
    if (!starts || check_buckets(nullptr, buckets, reach, two_sided) != W2V_OK) return W2V_ERR_ARG;
    bucket_starts(two_sided ? buckets / 2 : buckets, reach, starts);
    return W2V_OK;
}

int32_t w2v_attend(w2v_handle *h, const w2v_window *w, uint64_t n, const int32_t *spans, const void *q, uint64_t q_stride,
                   const void *k, uint64_t k_stride, const void *v, uint64_t v_stride, const float *bias, void *o,
                   uint64_t o_stride, float *lse)
{
    if (!h) return W2V_ERR_ARG;
    AttendParams p;
    int32_t rc = fill_attend(h, w, n, spans, bias, &p);
    if (rc != W2V_OK) return rc;
    if (n == 0) return W2V_OK;
    const uint64_t wq = (uint64_t)w->heads * w->head_dim, wk = (uint64_t)w->kv_heads * w->head_dim;
    const char *bad = "q, k, v and o must be 16-byte aligned, with strides that are multiples of 8 and hold every head";
    if ((rc = check_rows(h, q, q_stride, wq, bad)) != W2V_OK || (rc = check_rows(h, k, k_stride, wk, bad)) != W2V_OK ||
        (rc = check_rows(h, v, v_stride, wk, bad)) != W2V_OK || (rc = check_rows(h, o, o_stride, wq, bad)) != W2V_OK)
        return rc;
    if (!aligned(lse, 4)) return fail(h, W2V_ERR_ARG, "lse must be aligned to its elements");
    DeviceGuard g(h->device);
    if ((rc = ensure_error_word(h)) != W2V_OK) return rc;
    p.q = q; p.k = k; p.v = v; p.out = o; p.lse = lse;
    p.ldq = q_stride; p.ldk = k_stride; p.ldv = v_stride; p.ldo = o_stride;
    return launched(h, launch_attend(p, w->type, h->tc_error, h->sms, h->stream), "attention launch");
}

int32_t w2v_attend_backward(w2v_handle *h, const w2v_window *w, uint64_t n, const int32_t *spans, const void *q, uint64_t q_stride,
                            const void *k, uint64_t k_stride, const void *v, uint64_t v_stride, const float *bias, const void *o,
                            uint64_t o_stride, const float *lse, const void *d_o, uint64_t do_stride, void *dq,
                            uint64_t dq_stride, void *dk, uint64_t dk_stride, void *dv, uint64_t dv_stride, float *dbias)
{
    if (!h) return W2V_ERR_ARG;
    AttendParams p;
    int32_t rc = fill_attend(h, w, n, spans, bias, &p);
    if (rc != W2V_OK) return rc;
    if (!aligned(lse, 4) || !aligned(dbias, 4)) return fail(h, W2V_ERR_ARG, "lse and dbias must be aligned to their elements");
    if (dbias && !w->buckets) return fail(h, W2V_ERR_ARG, "dbias given but buckets is 0");
    const uint64_t wq = (uint64_t)w->heads * w->head_dim, wk = (uint64_t)w->kv_heads * w->head_dim;
    const char *bad = "q, k, v, o, d_o, dq, dk and dv must be 16-byte aligned, with strides that are multiples of 8 and hold every head";
    if (n) {
        if ((rc = check_rows(h, q, q_stride, wq, bad)) != W2V_OK || (rc = check_rows(h, k, k_stride, wk, bad)) != W2V_OK ||
            (rc = check_rows(h, v, v_stride, wk, bad)) != W2V_OK || (rc = check_rows(h, o, o_stride, wq, bad)) != W2V_OK ||
            (rc = check_rows(h, d_o, do_stride, wq, bad)) != W2V_OK || (rc = check_rows(h, dq, dq_stride, wq, bad)) != W2V_OK ||
            (rc = check_rows(h, dk, dk_stride, wk, bad)) != W2V_OK || (rc = check_rows(h, dv, dv_stride, wk, bad)) != W2V_OK)
            return rc;
        if (!lse) return fail(h, W2V_ERR_ARG, "lse is NULL");
    }
    DeviceGuard g(h->device);
    if ((rc = ensure_error_word(h)) != W2V_OK) return rc;
    p.q = q; p.k = k; p.v = v; p.o = o; p.d_o = d_o; p.lse = const_cast<float *>(lse);
    p.dq = dq; p.dk = dk; p.dv = dv; p.dbias = dbias;
    p.ldq = q_stride; p.ldk = k_stride; p.ldv = v_stride; p.ldo = o_stride; p.ld_do = do_stride;
    p.ld_dq = dq_stride; p.ld_dk = dk_stride; p.ld_dv = dv_stride;
    if ((rc = grow(h, &h->reader_ws, &h->reader_ws_cap, attend_backward_ws(p, dbias != nullptr), true)) != W2V_OK) return rc;
    return launched(h, launch_attend_backward(p, w->type, h->reader_ws, h->tc_error, h->sms, h->stream), "attention backward launch");
}

int32_t w2v_attend_token(w2v_handle *h, const w2v_window *w, uint32_t batch, const int32_t *pos, const void *q, const void *k,
                         const void *v, void *cache_k, void *cache_v, uint64_t places, const float *bias, void *o)
{
    if (!h) return W2V_ERR_ARG;
    TokenParams p;
    std::memset(&p, 0, sizeof(p));
    const int32_t rc = check_window(h, w, bias, &p.b);
    if (rc != W2V_OK) return rc;
    if (w->right || (w->buckets && w->two_sided)) return fail(h, W2V_ERR_ARG, "a new token sees nothing after it: right and two_sided must be 0");
    if (places < (uint64_t)w->sinks + w->left + 1 || places >= (1ull << 31))
        return fail(h, W2V_ERR_ARG, "places must be at least sinks + left + 1 and below 2^31");
    if (batch >= (1u << 20)) return fail(h, W2V_ERR_ARG, "batch must be below 2^20");
    if (batch == 0) return W2V_OK;
    if (!pos || !q || !k || !v || !cache_k || !cache_v || !o) return fail(h, W2V_ERR_ARG, "an array is NULL");
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(cache_k, 16) || !aligned(cache_v, 16) || !aligned(o, 16))
        return fail(h, W2V_ERR_ARG, "q, k, v, the cache and o must be 16-byte aligned");
    if (!aligned(pos, 4)) return fail(h, W2V_ERR_ARG, "pos must be aligned to its elements");
    DeviceGuard g(h->device);
    p.q = q; p.k = k; p.v = v; p.ck = cache_k; p.cv = cache_v; p.out = o; p.pos = pos; p.bias = bias; p.places = places;
    p.batch = batch; p.heads = w->heads; p.kv_heads = w->kv_heads; p.dim = w->head_dim;
    p.left = (int32_t)w->left; p.sinks = (int32_t)w->sinks; p.scale = w->scale;
    return launched(h, launch_attend_token(p, w->type, h->sms, h->stream), "single-token attention launch");
}

static int32_t check_fourbit(w2v_handle *h, uint64_t rows, uint32_t d, uint32_t group, const void *packed, const void *scales)
{
    if (d < 1 || d > 16384) return fail(h, W2V_ERR_ARG, "d must be in 1..16384");
    if (group != 32 && group != 64 && group != 128) return fail(h, W2V_ERR_ARG, "group must be 32, 64 or 128");
    if (rows >= (1ull << 31)) return fail(h, W2V_ERR_ARG, "rows must be below 2^31");
    if (rows && (!packed || !scales || !aligned(packed, 16) || !aligned(scales, 2)))
        return fail(h, W2V_ERR_ARG, "packed must be 16-byte aligned, and neither packed nor scales NULL");
    return W2V_OK;
}

int32_t w2v_fourbit_pack(w2v_handle *h, const float *rows, uint64_t n, uint32_t d, uint64_t row_stride, uint32_t group,
                         uint8_t *packed, void *scales)
{
    if (!h) return W2V_ERR_ARG;
    const int32_t rc = check_fourbit(h, n, d, group, packed, scales);
    if (rc != W2V_OK) return rc;
    if (n && (!rows || !aligned(rows, 4))) return fail(h, W2V_ERR_ARG, "rows is NULL or misaligned");
    if (row_stride < d) return fail(h, W2V_ERR_ARG, "row_stride must be at least d");
    DeviceGuard g(h->device);
    return launched(h, launch_fourbit_pack(rows, n, d, row_stride, group, packed, scales, h->sms, h->stream), "4-bit pack launch");
}

int32_t w2v_fourbit_scores(w2v_handle *h, const float *x, uint32_t m, uint64_t x_stride, const uint8_t *packed, const void *scales,
                           uint64_t rows, uint32_t d, uint32_t group, float *out, uint64_t out_stride)
{
    if (!h) return W2V_ERR_ARG;
    const int32_t rc = check_fourbit(h, rows, d, group, packed, scales);
    if (rc != W2V_OK) return rc;
    if (m > 8) return fail(h, W2V_ERR_ARG, "m must be at most 8");
    if (m == 0 || rows == 0) return W2V_OK;
    if (!x || !out || !aligned(x, 4) || !aligned(out, 4)) return fail(h, W2V_ERR_ARG, "x or out is NULL or misaligned");
    if (x_stride < d || out_stride < rows) return fail(h, W2V_ERR_ARG, "x_stride must be at least d and out_stride at least rows");
    DeviceGuard g(h->device);
    return launched(h, launch_fourbit_scores(x, m, x_stride, packed, scales, rows, d, group, out, out_stride, h->sms, h->stream),
                    "4-bit product launch");
}

}  // extern "C"
