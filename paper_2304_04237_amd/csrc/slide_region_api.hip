// C ABI of region selection, region attention and dropout: argument validation on the host, then the kernels' launches.
// Declarations and contracts: include/slide_attn.h.
#include "slide_attn.h"
#include "slide_region.h"

using slide::region::Args;
using slide::region::LOG2E;

static bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

static bool make_map(int H, int W, int h, int w, const int* size, slide::region::Map& m)
{
    if (H < 1 || W < 1 || h < 1 || w < 1) return false;
    if ((long long)H * W >= 1ll << 29) return false;                    // (regions * places stay below 2^31)
    h = std::min(h, H); w = std::min(w, W);
    const int across = (W + w - 1) / w, down = (H + h - 1) / h;
    m = slide::region::Map{H, W, h, w, across, across * down, h * w, size, slide::region::Div::by(across), slide::region::Div::by(w)};
    return (long long)across * down * h * w < 1ll << 31;
}

static bool make_random(float p, unsigned long long seed, unsigned int offset, const long long* offset_device, slide::region::Random& r)
{
    if (!(p >= 0.0f && p < 1.0f)) return false;
    const uint32_t t = (uint32_t)std::lrint((double)p * 65536.0);
    if (t >= 65536) return false;
    r = slide::region::Random{(uint32_t)seed, (uint32_t)(seed >> 32), offset, offset_device, t, (float)(65536.0 / (65536 - t))};
    return true;
}

// pixels of a map do not overlap, and offsets stay far below 63 bits
static bool strides_fit(long long pixel, long long image, int channels, const slide::region::Map& m)
{
    const bool one = m.H == 1 && m.W == 1;
    return (one ? pixel >= 0 : pixel >= channels) && pixel < 1ll << 31 && image >= 0 && image < 1ll << 45;
}

// Validates a problem and fills in what the kernels take; SLIDE_OK or the first thing that is wrong.
static int check(const slide_region_problem* p, int call, Args& a)
{
    if (!p) return SLIDE_ERR_NULL;
    if (p->dtype != SLIDE_F32 && p->dtype != SLIDE_BF16) return SLIDE_ERR_DTYPE;
    if (p->B < 1 || p->heads < 1 || p->kv_heads < 1 || p->heads % p->kv_heads != 0) return SLIDE_ERR_SHAPE;
    // (as the library's other calls; products of these and head sizes stay ints)
    if (p->B > 65535 || p->heads > 65535 || (long long)p->B * p->kv_heads > 65535) return SLIDE_ERR_SHAPE;
    if (p->head_dim < 1 || p->head_dim > 128 || p->topk < 1 || p->topk > 1024) return SLIDE_ERR_SHAPE;
    a = Args{};
    a.B = p->B; a.heads = p->heads; a.kv = p->kv_heads; a.g = p->heads / p->kv_heads;
    a.d = p->head_dim; a.T = p->topk; a.dtype = p->dtype;
    if (!make_map(p->q_h, p->q_w, p->q_region_h, p->q_region_w, p->q_size, a.qm) ||
        !make_map(p->k_h, p->k_w, p->k_region_h, p->k_region_w, p->k_size, a.km)) return SLIDE_ERR_SHAPE;
    const long long rows = (long long)a.qm.places * a.g;
    if (rows * a.qm.regions >= 1ll << 30) return SLIDE_ERR_SHAPE;       // (the dropout counter's second word; rows of a share)
    a.R = (int)rows;
    a.quads = (a.km.places + 3) / 4; a.pairs = (a.R + 1) / 2;
    a.by_g = slide::region::Div::by(a.g); a.by_slots = slide::region::Div::by(4 * a.quads);
    if (4ll * a.quads * a.T >= (1ll << 31) - 256) return SLIDE_ERR_SHAPE;        // (slots of a group, and some past its end)
    // waves of one launch: every 32 rows of a group, every 32 places of a region of keys
    if ((long long)a.B * a.kv * a.qm.regions * ((a.R + 31) / 32) >= 1ll << 24 ||
        (long long)a.B * a.kv * a.km.regions * ((a.km.places + 31) / 32) >= 1ll << 24) return SLIDE_ERR_SHAPE;
    if ((long long)a.quads * a.km.regions >= 1ll << 32) return SLIDE_ERR_SHAPE;
    if ((long long)a.qm.regions * a.T >= 1ll << 30) return SLIDE_ERR_SHAPE;
    if (!strides_fit(p->q_pixel, p->q_image, p->heads * p->head_dim, a.qm) || !strides_fit(p->k_pixel, p->k_image, p->kv_heads * p->head_dim, a.km))
        return SLIDE_ERR_SHAPE;
    if (call == SLIDE_REGION_SELECT) {
        if (a.km.regions > 16384) return SLIDE_ERR_SHAPE;
    } else {
        if (!strides_fit(p->v_pixel, p->v_image, p->kv_heads * p->head_dim, a.km)) return SLIDE_ERR_SHAPE;
        if (!(p->scale >= 0.0f) || std::isinf(p->scale)) return SLIDE_ERR_SHAPE;
        if (!make_random(p->dropout, p->seed, p->offset, p->offset_device, a.rnd)) return SLIDE_ERR_SHAPE;
        // what the kernels multiply by: an infinity would make a NaN of every zero
        if (std::isinf(p->scale * LOG2E) || (call == SLIDE_REGION_BWD && std::isinf(p->scale * a.rnd.scale))) return SLIDE_ERR_SHAPE;
        if (!aligned(p->offset_device, 8)) return SLIDE_ERR_ALIGN;
    }
    if (!aligned(p->q_size, 4) || !aligned(p->k_size, 4)) return SLIDE_ERR_ALIGN;
    a.qs = {p->q_pixel, p->q_image}; a.ks = {p->k_pixel, p->k_image}; a.vs = {p->v_pixel, p->v_image};
    a.os = {(long long)p->heads * p->head_dim, (long long)p->q_h * p->q_w * p->heads * p->head_dim};
    a.hd = a.dl = a.d;
    a.scale = p->scale > 0.0f ? p->scale : 1.0f / sqrtf((float)p->head_dim);
    return SLIDE_OK;
}

static size_t workspace_bytes_of(const Args& a, int call)
{
    return call == SLIDE_REGION_SELECT ? slide::region::select_workspace_bytes(a)
         : call == SLIDE_REGION_FWD ? slide::region::fwd_workspace_bytes(a) : slide::region::bwd_workspace_bytes(a);
}

// The pointers of a call: none missing, aligned to their elements; the workspace.
static int check_pointers(const Args& a, int call, std::initializer_list<const void*> activations, const void* index,
                          const void* lse, const void* workspace, size_t workspace_bytes)
{
    for (const void* p : activations)
        if (!p) return SLIDE_ERR_NULL;
    if (!index) return SLIDE_ERR_NULL;
    for (const void* p : activations)
        if (!aligned(p, a.dtype == SLIDE_F32 ? 4 : 2)) return SLIDE_ERR_ALIGN;
    if (!aligned(index, 4) || !aligned(lse, 4)) return SLIDE_ERR_ALIGN;
    const size_t need = workspace_bytes_of(a, call);
    if (need && (!workspace || workspace_bytes < need)) return SLIDE_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return SLIDE_ERR_ALIGN;
    return SLIDE_OK;
}

extern "C" size_t slide_region_workspace_bytes(const slide_region_problem* p, int call)
{
    Args a;
    if (call < SLIDE_REGION_SELECT || call > SLIDE_REGION_BWD || check(p, call, a) != SLIDE_OK) return 0;
    return workspace_bytes_of(a, call);
}

extern "C" int slide_region_select(const slide_region_problem* p, const void* q, const void* k, int* index,
                                   void* workspace, size_t workspace_bytes, void* stream)
{
    Args a;
    int st = check(p, SLIDE_REGION_SELECT, a);
    if (st != SLIDE_OK) return st;
    st = check_pointers(a, SLIDE_REGION_SELECT, {q, k}, index, nullptr, workspace, workspace_bytes);
    if (st != SLIDE_OK) return st;
    a.q = q; a.k = k;
    return slide::region::launch_select(a, index, workspace, (hipStream_t)stream) == hipSuccess ? SLIDE_OK : SLIDE_ERR_HIP;
}

extern "C" int slide_region_attn_fwd(const slide_region_problem* p, const void* q, const void* k, const void* v, const int* index,
                                     void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream)
{
    Args a;
    int st = check(p, SLIDE_REGION_FWD, a);
    if (st != SLIDE_OK) return st;
    st = check_pointers(a, SLIDE_REGION_FWD, {q, k, v, out}, index, lse, workspace, workspace_bytes);
    if (st != SLIDE_OK) return st;
    a.q = q; a.k = k; a.v = v; a.index = index;
    return slide::region::launch_fwd(a, out, lse, workspace, (hipStream_t)stream) == hipSuccess ? SLIDE_OK : SLIDE_ERR_HIP;
}

extern "C" int slide_region_attn_bwd(const slide_region_problem* p, const void* dout, const void* q, const void* k, const void* v,
                                     const int* index, const void* out, const float* lse, void* dq, void* dk, void* dv,
                                     void* workspace, size_t workspace_bytes, void* stream)
{
    Args a;
    int st = check(p, SLIDE_REGION_BWD, a);
    if (st != SLIDE_OK) return st;
    if (!lse) return SLIDE_ERR_NULL;
    st = check_pointers(a, SLIDE_REGION_BWD, {dout, q, k, v, out, dq, dk, dv}, index, lse, workspace, workspace_bytes);
    if (st != SLIDE_OK) return st;
    a.q = q; a.k = k; a.v = v; a.index = index;
    return slide::region::launch_bwd(a, dout, out, lse, dq, dk, dv, workspace, (hipStream_t)stream) == hipSuccess ? SLIDE_OK : SLIDE_ERR_HIP;
}

static int dropout(const void* x, const void* residual, void* y, long long n, int dtype, float p,
                   unsigned long long seed, unsigned int offset, const long long* offset_device, void* stream)
{
    if (dtype != SLIDE_F32 && dtype != SLIDE_BF16) return SLIDE_ERR_DTYPE;
    slide::region::Random r;
    if (n < 1 || n >= 1ll << 34 || !make_random(p, seed, offset, offset_device, r)) return SLIDE_ERR_SHAPE;
    if (!x || !y) return SLIDE_ERR_NULL;
    const size_t esz = dtype == SLIDE_F32 ? 4 : 2;
    if (!aligned(x, esz) || !aligned(residual, esz) || !aligned(y, esz) || !aligned(offset_device, 8)) return SLIDE_ERR_ALIGN;
    return slide::region::launch_dropout(x, residual, y, n, dtype, r, (hipStream_t)stream) == hipSuccess ? SLIDE_OK : SLIDE_ERR_HIP;
}

extern "C" int slide_dropout_fwd(const void* x, const void* residual, void* y, long long n, int dtype, float p,
                                 unsigned long long seed, unsigned int offset, const long long* offset_device, void* stream)
{
    return dropout(x, residual, y, n, dtype, p, seed, offset, offset_device, stream);
}

extern "C" int slide_dropout_bwd(const void* dout, void* dx, long long n, int dtype, float p,
                                 unsigned long long seed, unsigned int offset, const long long* offset_device, void* stream)
{
    return dropout(dout, nullptr, dx, n, dtype, p, seed, offset, offset_device, stream);
}
