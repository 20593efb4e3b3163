// Host side of the norms and the paged cache of include/cascade_kv.h: checks of arguments and the launches of every call.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>

#include <new>

#include "paged.h"
#include "structure.h"

using namespace ckv;

namespace {

constexpr int kTextBytes = 240;
constexpr int kMaxCallTokens = 1 << 20;      // a launch has a workgroup of up to 1024 threads per token, and 2^32 threads at most
constexpr int kMaxHeads = 1024;
thread_local char g_paged_init_error[kTextBytes] = "";

// Calls of a context launch on its device, whichever is current.
struct OnDevice {
    int before = -1;
    hipError_t err = hipSuccess;
    explicit OnDevice(int device)
    {
        int now = 0;
        err = hipGetDevice(&now);
        if (err == hipSuccess && now != device) {
            err = hipSetDevice(device);
            if (err == hipSuccess) before = now;
        }
    }
    ~OnDevice() { if (before >= 0) (void)hipSetDevice(before); }
};

bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

}  // namespace

struct cascade_paged_ctx {
    PagedGeom g;
    int dtype, elem, max_seqs, device;
    void* scratch;
    char err[kTextBytes];
};

static int fail(cascade_paged_ctx* ctx, int code, const char* format, ...)
{
    va_list args;
    va_start(args, format);
    vsnprintf(ctx ? ctx->err : g_paged_init_error, kTextBytes, format, args);
    va_end(args);
    return code;
}

static int launched(cascade_paged_ctx* ctx, const char* who)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? CASCADE_OK : fail(ctx, CASCADE_E_HIP, "%s: %s", who, hipGetErrorString(e));
}

// Fills everything of g that follows from the configuration.
static int check_paged_config(const cascade_paged_config* c, PagedGeom& g)
{
    const char* who = "cascade_paged_config";
    if (c->n_q_heads < 1 || c->n_kv_heads < 1 || c->n_q_heads > kMaxHeads || c->n_q_heads % c->n_kv_heads)
        return fail(nullptr, CASCADE_E_INVALID_CONFIG, "%s: n_q_heads must be a multiple of n_kv_heads, both 1 to %d", who, kMaxHeads);
    if (c->dtype != CASCADE_F32 && c->dtype != CASCADE_BF16) return fail(nullptr, CASCADE_E_UNSUPPORTED, "%s: dtype must be CASCADE_F32 or CASCADE_BF16", who);
    if (c->head_dim != 64 && c->head_dim != 128) return fail(nullptr, CASCADE_E_UNSUPPORTED, "%s: head_dim must be 64 or 128", who);
    if (c->page_size < kGroupTokens || c->page_size > 65536 || c->page_size % kGroupTokens)
        return fail(nullptr, CASCADE_E_INVALID_CONFIG, "%s: page_size must be a multiple of %d, at most 65536", who, kGroupTokens);
    if (c->max_seqs < 1 || c->max_seqs > 65535) return fail(nullptr, CASCADE_E_INVALID_CONFIG, "%s: max_seqs must be 1 to 65535", who);
    if (!(c->softmax_scale >= 0.f) || !isfinite(c->softmax_scale)) return fail(nullptr, CASCADE_E_INVALID_CONFIG, "%s: softmax_scale must be finite and not negative", who);
    if (c->window < 0) return fail(nullptr, CASCADE_E_INVALID_CONFIG, "%s: window must not be negative", who);
    g.Hq = c->n_q_heads;
    g.Hkv = c->n_kv_heads;
    g.G = g.Hq / g.Hkv;
    g.d = c->head_dim;
    g.page_size = c->page_size;
    g.groups = c->page_size / kGroupTokens;
    g.group_bytes = paged_group_bytes(g.d);
    // page numbers are 32-bit, places of groups in units of 128 bytes as well: 2^39 bytes, more than a device has
    if (c->n_pages < 1 || c->n_pages > 0x7FFFFFFF || c->n_pages > (1ll << 39) / ((int64_t)g.Hkv * g.groups * g.group_bytes))
        return fail(nullptr, CASCADE_E_INVALID_CONFIG, "%s: n_pages out of range", who);
    g.n_pages = c->n_pages;
    g.scale = c->softmax_scale == 0.f ? 1.f / sqrtf((float)g.d) : c->softmax_scale;
    g.window = c->window;
    g.pages = nullptr;
    g.rope = nullptr;
    g.rope_positions = 0;
    return CASCADE_OK;
}

extern "C" size_t cascade_rope_table_bytes(int64_t n_positions, int32_t head_dim)
{
    if (n_positions < 1 || n_positions > (1ll << 31) || head_dim < 2 || head_dim > 256 || head_dim % 2) return 0;
    return rope_pair_table_bytes(n_positions, head_dim);
}

// The calls without a context leave their text where cascade_last_error(NULL) finds it.
static int fail_without_context(int code, const char* text)
{
    try {
        set_init_error(text);
    } catch (...) {      // no memory for the text
    }
    return code;
}
#define CKV_REFUSE(code, text) return fail_without_context(code, text)

extern "C" int cascade_rope_table(void* dev_rope, size_t bytes, int64_t n_positions, int32_t head_dim, double base, void* stream)
{
    if (!dev_rope) CKV_REFUSE(CASCADE_E_NULL_ARG, "cascade_rope_table: NULL table");
    const size_t need = cascade_rope_table_bytes(n_positions, head_dim);
    if (need == 0) CKV_REFUSE(CASCADE_E_BAD_ARG, "cascade_rope_table: n_positions must be 1 to 2^31, head_dim even and 2 to 256");
    if (!(base > 0.0) || !isfinite(base)) CKV_REFUSE(CASCADE_E_BAD_ARG, "cascade_rope_table: base must be finite and above 0");
    if (!aligned(dev_rope, 16)) CKV_REFUSE(CASCADE_E_BAD_ARG, "cascade_rope_table: the table must be 16-byte aligned");
    if (bytes < need) CKV_REFUSE(CASCADE_E_WORKSPACE_TOO_SMALL, "cascade_rope_table: buffer smaller than cascade_rope_table_bytes");
    launch_rope_pair_table((double2*)dev_rope, n_positions, head_dim, base, (hipStream_t)stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) CKV_REFUSE(CASCADE_E_HIP, hipGetErrorString(e));
    return CASCADE_OK;
}

extern "C" int cascade_norm_rope(const cascade_norm_rope_args* args, void* stream)
{
    if (!args) CKV_REFUSE(CASCADE_E_NULL_ARG, "cascade_norm_rope: NULL arguments");
    const cascade_norm_rope_args& x = *args;
    if (x.dtype != CASCADE_F32 && x.dtype != CASCADE_BF16) CKV_REFUSE(CASCADE_E_UNSUPPORTED, "cascade_norm_rope: dtype must be CASCADE_F32 or CASCADE_BF16");
    if (x.head_dim < 2 || x.head_dim > 256 || x.head_dim % 2) CKV_REFUSE(CASCADE_E_UNSUPPORTED, "cascade_norm_rope: head_dim must be even, 2 to 256");
    if (x.n_tokens < 0 || x.n_tokens > kMaxCallTokens) CKV_REFUSE(CASCADE_E_BAD_ARG, "cascade_norm_rope: n_tokens must be 0 to 2^20");
    if (x.n_q_heads < 0 || x.n_k_heads < 0 || x.n_q_heads > kMaxHeads || x.n_k_heads > kMaxHeads) CKV_REFUSE(CASCADE_E_BAD_ARG, "cascade_norm_rope: heads must be 0 to 1024");
    if ((x.norm != 0 && x.norm != 1) || x.reserved != 0) CKV_REFUSE(CASCADE_E_BAD_ARG, "cascade_norm_rope: norm must be 0 or 1, reserved 0");
    if (x.norm && !(x.eps >= 0.f && isfinite(x.eps))) CKV_REFUSE(CASCADE_E_BAD_ARG, "cascade_norm_rope: eps must be finite and not negative");
    if (x.n_tokens == 0 || x.n_q_heads + x.n_k_heads == 0) return CASCADE_OK;
    if ((x.n_q_heads && (!x.dev_q || !x.dev_q_out)) || (x.n_k_heads && (!x.dev_k || !x.dev_k_out))) CKV_REFUSE(CASCADE_E_NULL_ARG, "cascade_norm_rope: NULL input or output");
    if (x.dev_positions && !x.dev_rope) CKV_REFUSE(CASCADE_E_NULL_ARG, "cascade_norm_rope: positions need a rotation table");
    if (x.dev_positions && (x.rope_positions < 1 || x.rope_positions > (1ll << 31) || !aligned(x.dev_rope, 16) || !aligned(x.dev_positions, 4)))
        CKV_REFUSE(CASCADE_E_BAD_ARG, "cascade_norm_rope: rope_positions out of range, or positions or table not aligned");
    const int elem = x.dtype == CASCADE_BF16 ? 2 : 4;
    NormRope a;
    a.d = x.head_dim;
    a.n_tokens = x.n_tokens;
    a.Hq = x.n_q_heads;
    a.Hk = x.n_k_heads;
    a.norm = x.norm;
    a.eps = x.eps;
    a.q = x.dev_q;
    a.k = x.dev_k;
    a.q_out = x.dev_q_out;
    a.k_out = x.dev_k_out;
    a.q_weight = x.norm ? x.dev_q_weight : nullptr;
    a.k_weight = x.norm ? x.dev_k_weight : nullptr;
    a.positions = x.dev_positions;
    a.rope = (const double2*)x.dev_rope;
    a.rope_positions = x.rope_positions;
    a.vectors = x.head_dim % 16 == 0;
    const int64_t q_row = (int64_t)x.n_q_heads * x.head_dim, k_row = (int64_t)x.n_k_heads * x.head_dim;
    const struct { int64_t given; int64_t row; const void* p; int64_t* to; int heads; } rows[4] = {
        {x.q_stride, q_row, x.dev_q, &a.q_stride, x.n_q_heads}, {x.k_stride, k_row, x.dev_k, &a.k_stride, x.n_k_heads},
        {x.q_out_stride, q_row, x.dev_q_out, &a.q_out_stride, x.n_q_heads}, {x.k_out_stride, k_row, x.dev_k_out, &a.k_out_stride, x.n_k_heads}};
    for (const auto& r : rows) {
        *r.to = r.given ? r.given : r.row;
        if (!r.heads) continue;
        if (*r.to < r.row || *r.to > (1ll << 40)) CKV_REFUSE(CASCADE_E_BAD_ARG, "cascade_norm_rope: a stride is below heads * head_dim, or out of range");
        if (!aligned(r.p, elem)) CKV_REFUSE(CASCADE_E_BAD_ARG, "cascade_norm_rope: an array is not aligned to its elements");
        a.vectors = a.vectors && aligned(r.p, 16) && *r.to * elem % 16 == 0;
    }
    if ((x.n_q_heads && x.dev_q == x.dev_q_out && a.q_stride != a.q_out_stride) || (x.n_k_heads && x.dev_k == x.dev_k_out && a.k_stride != a.k_out_stride))
        CKV_REFUSE(CASCADE_E_BAD_ARG, "cascade_norm_rope: an output over its input needs the same stride");
    if (!aligned(a.q_weight, elem) || !aligned(a.k_weight, elem)) CKV_REFUSE(CASCADE_E_BAD_ARG, "cascade_norm_rope: a weight is not aligned to its elements");
    a.vectors = a.vectors && aligned(a.q_weight, 16) && aligned(a.k_weight, 16);
    launch_norm_rope(a, x.dtype, (hipStream_t)stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) CKV_REFUSE(CASCADE_E_HIP, hipGetErrorString(e));
    return CASCADE_OK;
}

extern "C" size_t cascade_paged_page_bytes(const cascade_paged_config* cfg)
{
    PagedGeom g;
    if (!cfg || check_paged_config(cfg, g) != CASCADE_OK) return 0;
    return (size_t)g.Hkv * g.groups * g.group_bytes;
}

extern "C" size_t cascade_paged_workspace_bytes(const cascade_paged_config* cfg)
{
    PagedGeom g;
    if (!cfg || check_paged_config(cfg, g) != CASCADE_OK) return 0;
    return paged_scratch_bytes(g);
}

extern "C" int cascade_paged_init(const cascade_paged_config* cfg, void* dev_pages, void* dev_workspace, size_t workspace_bytes,
                                  const void* dev_rope, int64_t rope_positions, cascade_paged_ctx** out_ctx)
{
    if (out_ctx) *out_ctx = nullptr;
    if (!cfg || !dev_pages || !dev_workspace || !out_ctx) return fail(nullptr, CASCADE_E_NULL_ARG, "cascade_paged_init: NULL argument");
    PagedGeom g;
    const int rc = check_paged_config(cfg, g);
    if (rc != CASCADE_OK) return rc;
    if (!aligned(dev_pages, 128)) return fail(nullptr, CASCADE_E_BAD_ARG, "cascade_paged_init: pages must be 128-byte aligned");
    if (!aligned(dev_workspace, 256)) return fail(nullptr, CASCADE_E_BAD_ARG, "cascade_paged_init: workspace must be 256-byte aligned");
    if (workspace_bytes < paged_scratch_bytes(g)) return fail(nullptr, CASCADE_E_WORKSPACE_TOO_SMALL, "cascade_paged_init: workspace too small");
    if (dev_rope && (rope_positions < 1 || rope_positions > (1ll << 31) || !aligned(dev_rope, 16)))
        return fail(nullptr, CASCADE_E_BAD_ARG, "cascade_paged_init: rope_positions out of range, or the table not 16-byte aligned");
    int device = 0;
    const hipError_t e = hipGetDevice(&device);
    if (e == hipErrorNoDevice) device = -1;      // a context for checks of arguments: every launch is refused
    else if (e != hipSuccess) return fail(nullptr, CASCADE_E_HIP, "cascade_paged_init: %s", hipGetErrorString(e));
    cascade_paged_ctx* ctx = new (std::nothrow) cascade_paged_ctx;
    if (!ctx) return fail(nullptr, CASCADE_E_INTERNAL, "cascade_paged_init: out of host memory");
    g.pages = (uint8_t*)dev_pages;
    g.rope = (const double2*)dev_rope;
    g.rope_positions = dev_rope ? rope_positions : 0;
    ctx->g = g;
    ctx->dtype = cfg->dtype;
    ctx->elem = cfg->dtype == CASCADE_BF16 ? 2 : 4;
    ctx->max_seqs = cfg->max_seqs;
    ctx->device = device;
    ctx->scratch = dev_workspace;
    ctx->err[0] = 0;
    *out_ctx = ctx;
    return CASCADE_OK;
}

extern "C" void cascade_paged_destroy(cascade_paged_ctx* ctx) { delete ctx; }

extern "C" const char* cascade_paged_last_error(const cascade_paged_ctx* ctx) { return ctx ? ctx->err : g_paged_init_error; }

// Checks what all calls have in common; n is what is left to do (0: nothing).
static int check_batch(cascade_paged_ctx* ctx, const char* who, const cascade_paged_batch* x, PagedBatch& b, int& n)
{
    n = 0;
    if (!x) return fail(ctx, CASCADE_E_NULL_ARG, "%s: NULL batch", who);
    if (x->n_seqs < 0 || x->n_seqs > ctx->max_seqs) return fail(ctx, CASCADE_E_BAD_ARG, "%s: n_seqs must be 0 to max_seqs", who);
    if (x->n_tokens < 0 || x->n_tokens > kMaxCallTokens) return fail(ctx, CASCADE_E_BAD_ARG, "%s: n_tokens must be 0 to 2^20", who);
    if (x->max_new < 0 || x->max_length < 0 || x->max_length > 0x7FFFFFFF - kMaxCallTokens)
        return fail(ctx, CASCADE_E_BAD_ARG, "%s: max_new and max_length must not be negative, max_length at most 2^31 - 2^20", who);
    if (x->table_stride < 0) return fail(ctx, CASCADE_E_BAD_ARG, "%s: table_stride must not be negative", who);
    b.n_seqs = x->n_seqs;
    b.n_tokens = x->n_tokens;
    b.max_new = x->max_new < x->n_tokens ? x->max_new : x->n_tokens;
    b.max_length = x->max_length;
    b.lengths = x->dev_lengths;
    b.offsets = x->dev_new_offsets;
    b.table = x->dev_page_table;
    b.table_stride = x->table_stride;
    if (b.n_seqs == 0 || b.max_new == 0) return CASCADE_OK;
    // workgroups of up to 512 threads, and 2^32 threads at most in a launch: one per KV head and group of 32 tokens (two of a sequence may be begun) and one per
    // token (append), or one per KV head and block of 128 rows (one of a sequence may be begun)
    const int64_t n_groups = b.n_tokens / kGroupTokens + 2 * (int64_t)b.n_seqs;
    if (n_groups * ctx->g.Hkv + b.n_tokens > (1 << 22) || (int64_t)b.n_tokens * ctx->g.Hq / 128 + (int64_t)b.n_seqs * ctx->g.Hkv > (1 << 22))
        return fail(ctx, CASCADE_E_BAD_ARG, "%s: too many tokens or sequences for one call", who);
    if (!b.lengths || !b.offsets || (!b.table && b.table_stride)) return fail(ctx, CASCADE_E_NULL_ARG, "%s: NULL array in the batch", who);
    if (!aligned(b.lengths, 4) || !aligned(b.offsets, 4) || !aligned(b.table, 4)) return fail(ctx, CASCADE_E_BAD_ARG, "%s: the batch's arrays must be 4-byte aligned", who);
    n = b.n_tokens;
    return CASCADE_OK;
}

// A token array: fills in the stride that 0 stands for.
static int check_rows(cascade_paged_ctx* ctx, const char* who, const char* name, const void* p, int heads, int64_t given, int64_t& stride)
{
    if (!p) return fail(ctx, CASCADE_E_NULL_ARG, "%s: NULL %s", who, name);
    const int64_t row = (int64_t)heads * ctx->g.d;
    stride = given ? given : row;
    if (stride < row || stride > (1ll << 40)) return fail(ctx, CASCADE_E_BAD_ARG, "%s: the stride of %s is below heads * head_dim, or out of range", who, name);
    if (!aligned(p, 16) || stride * ctx->elem % 16) return fail(ctx, CASCADE_E_BAD_ARG, "%s: rows of %s must be 16-byte aligned", who, name);
    return CASCADE_OK;
}

extern "C" int cascade_paged_append(cascade_paged_ctx* ctx, const cascade_paged_batch* batch, const void* dev_k, int64_t k_stride, const void* dev_v,
                                    int64_t v_stride, const void* dev_q, int64_t q_stride, void* dev_q_out, void* stream)
{
    const char* who = "cascade_paged_append";
    if (!ctx) return fail(nullptr, CASCADE_E_NULL_ARG, "%s: NULL context", who);
    PagedBatch b;
    PagedRows x = {dev_k, dev_v, dev_q, dev_q_out, 0, 0, 0};
    int n, rc = check_batch(ctx, who, batch, b, n);
    if (rc != CASCADE_OK) return rc;
    if (dev_q && !ctx->g.rope) return fail(ctx, CASCADE_E_BAD_ARG, "%s: queries are rotated by a context with a rotation table", who);
    if (n == 0) return CASCADE_OK;
    if ((rc = check_rows(ctx, who, "k", dev_k, ctx->g.Hkv, k_stride, x.k_stride)) != CASCADE_OK) return rc;
    if ((rc = check_rows(ctx, who, "v", dev_v, ctx->g.Hkv, v_stride, x.v_stride)) != CASCADE_OK) return rc;
    if (dev_q) {
        int64_t whole;
        if ((rc = check_rows(ctx, who, "q", dev_q, ctx->g.Hq, q_stride, x.q_stride)) != CASCADE_OK) return rc;
        if ((rc = check_rows(ctx, who, "q_out", dev_q_out, ctx->g.Hq, 0, whole)) != CASCADE_OK) return rc;
        if (dev_q == dev_q_out && x.q_stride != whole) return fail(ctx, CASCADE_E_BAD_ARG, "%s: q_out over q needs contiguous queries", who);
    }
    if (ctx->g.rope && b.max_length > ctx->g.rope_positions) return fail(ctx, CASCADE_E_BAD_ARG, "%s: max_length is behind the rotation table", who);
    OnDevice on(ctx->device);
    if (on.err != hipSuccess) return fail(ctx, CASCADE_E_HIP, "%s: %s", who, hipGetErrorString(on.err));
    launch_paged_append(ctx->g, b, x, ctx->dtype, (hipStream_t)stream);
    return launched(ctx, who);
}

extern "C" int cascade_paged_attend(cascade_paged_ctx* ctx, const cascade_paged_batch* batch, const void* dev_q, int64_t q_stride, void* dev_out, void* stream)
{
    const char* who = "cascade_paged_attend";
    if (!ctx) return fail(nullptr, CASCADE_E_NULL_ARG, "%s: NULL context", who);
    PagedBatch b;
    int n, rc = check_batch(ctx, who, batch, b, n);
    if (rc != CASCADE_OK) return rc;
    if (n == 0) return CASCADE_OK;
    int64_t stride, whole;
    if ((rc = check_rows(ctx, who, "q", dev_q, ctx->g.Hq, q_stride, stride)) != CASCADE_OK) return rc;
    if ((rc = check_rows(ctx, who, "out", dev_out, ctx->g.Hq, 0, whole)) != CASCADE_OK) return rc;
    if (dev_q == dev_out) return fail(ctx, CASCADE_E_BAD_ARG, "%s: out must not be q", who);
    OnDevice on(ctx->device);
    if (on.err != hipSuccess) return fail(ctx, CASCADE_E_HIP, "%s: %s", who, hipGetErrorString(on.err));
    launch_paged_attend(ctx->g, b, dev_q, stride, dev_out, ctx->scratch, ctx->dtype, (hipStream_t)stream);
    return launched(ctx, who);
}

extern "C" int cascade_paged_read(cascade_paged_ctx* ctx, const cascade_paged_batch* batch, void* dev_k_out, void* dev_v_out, void* stream)
{
    const char* who = "cascade_paged_read";
    if (!ctx) return fail(nullptr, CASCADE_E_NULL_ARG, "%s: NULL context", who);
    PagedBatch b;
    int n, rc = check_batch(ctx, who, batch, b, n);
    if (rc != CASCADE_OK) return rc;
    if (n == 0 || (!dev_k_out && !dev_v_out)) return CASCADE_OK;
    if (!aligned(dev_k_out, 16) || !aligned(dev_v_out, 16)) return fail(ctx, CASCADE_E_BAD_ARG, "%s: outputs must be 16-byte aligned", who);
    OnDevice on(ctx->device);
    if (on.err != hipSuccess) return fail(ctx, CASCADE_E_HIP, "%s: %s", who, hipGetErrorString(on.err));
    launch_paged_read(ctx->g, b, dev_k_out, dev_v_out, ctx->dtype, (hipStream_t)stream);
    return launched(ctx, who);
}
