// C ABI of libvarrate: validation, sizing, workspace carving and kernel dispatch.
// Every check runs on the host before anything is enqueued; no entry point synchronises or
// allocates device memory.  The one piece of state kept across calls is the per (kernel,
// device) record of raised dynamic-LDS limits (ensure_lds_limit, under a lock).
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <cmath>

#include <map>
#include <mutex>
#include <string>
#include <utility>

#include "vr_internal.h"
#include "vr_pages.h"

using namespace vr;

namespace vr {

hipError_t ensure_lds_limit(const void* fn, size_t bytes) {
    static std::mutex mu;
    static std::map<std::pair<const void*, int>, size_t> raised;
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    try {                                                  // nothing is thrown through a C entry
        std::lock_guard<std::mutex> lock(mu);
        size_t& have = raised[{fn, dev}];
        if (bytes <= have) return hipSuccess;
        e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
        if (e == hipSuccess) have = bytes;
    } catch (...) {
        return hipErrorOutOfMemory;
    }
    return e;
}

}  // namespace vr

namespace {

thread_local std::string g_err;

int fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
int fail(int code, const char* fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    try {
        g_err = buf;
    } catch (...) {                                        // no memory for the text: the code stands
    }
    return code;
}

int hip_status(hipError_t e, const char* what) {
    if (e == hipSuccess) return VARRATE_OK;
    return fail(VARRATE_EHIP, "%s: %s", what, hipGetErrorString(e));
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }


int check_shape_only(const varrate_shape* sh) {
    if (!sh) return fail(VARRATE_EINVAL, "shape is NULL");
    if (sh->d != VARRATE_HEAD_DIM) return fail(VARRATE_EUNSUPPORTED, "head dim %d != 128", sh->d);
    if (sh->G < 1 || sh->H < 1) return fail(VARRATE_EINVAL, "G=%d H=%d must be >= 1", sh->G, sh->H);
    if (sh->H % sh->G != 0) return fail(VARRATE_EUNSUPPORTED, "H=%d is not a multiple of G=%d", sh->H, sh->G);
    if (sh->w < 1) return fail(VARRATE_EINVAL, "window w=%d must be >= 1", sh->w);
    if (sh->n <= sh->w) return fail(VARRATE_EBUDGET, "n=%lld leaves no coded tokens (w=%d)", (long long)sh->n, sh->w);
    if (sh->r_min < 0 || sh->r_min > VARRATE_HEAD_DIM)
        return fail(VARRATE_EINVAL, "r_min=%d outside [0, 128]", sh->r_min);
    if (sh->kappa_pct < 1 || sh->kappa_pct > 100) return fail(VARRATE_EINVAL, "kappa_pct=%d outside [1, 100]", sh->kappa_pct);
    if (sh->dtype != VARRATE_BF16 && sh->dtype != VARRATE_F32) return fail(VARRATE_EINVAL, "unknown dtype %d", sh->dtype);
    if ((int64_t)(sh->H / sh->G) * sh->w > 256)
        return fail(VARRATE_EUNSUPPORTED, "(H/G) * w = %lld window rows per KV head exceeds 256",
                    (long long)(sh->H / sh->G) * sh->w);
    if (sh->n - sh->w > MAX_CODED)
        return fail(VARRATE_EUNSUPPORTED, "N=%lld coded tokens exceeds %lld", (long long)(sh->n - sh->w), (long long)MAX_CODED);
    if (sh->anchor_stride != 0) {
        if (sh->anchor_stride < 2 || sh->anchor_stride > 4096)
            return fail(VARRATE_EINVAL, "anchor_stride=%d outside {0} or [2, 4096]", sh->anchor_stride);
        if (sh->dtype != VARRATE_BF16) return fail(VARRATE_EUNSUPPORTED, "the residual codec needs a bf16 layer");
        if (anchor_count(*sh) > 65535) return fail(VARRATE_EUNSUPPORTED, "more than 65535 anchors");
        if (anchor_count(*sh) < 4) return fail(VARRATE_EBUDGET, "fewer than 4 anchors");
        if (coded_count(*sh) < 1) return fail(VARRATE_EBUDGET, "no coded tokens between the anchors");
    }
    if (sh->rope != 0) {
        if (sh->rope != 1) return fail(VARRATE_EINVAL, "rope=%d outside {0, 1}", sh->rope);
        if (sh->anchor_stride != 0) return fail(VARRATE_EUNSUPPORTED, "rotary keys with anchors");
        for (int i = 0; i < VARRATE_HEAD_DIM / 2; ++i)
            if (!(sh->rope_theta[i] >= 0.f) || !std::isfinite(sh->rope_theta[i]))
                return fail(VARRATE_EINVAL, "rope_theta[%d] is negative or not finite", i);
    }
    return VARRATE_OK;
}

int check_shape(const varrate_shape* sh) {
    int rc = check_shape_only(sh);
    if (rc) return rc;
    const int64_t B = coded_budget(*sh);
    const int64_t N = coded_count(*sh);
    if (N * sh->r_min > B || B > N * VARRATE_HEAD_DIM)
        return fail(VARRATE_EBUDGET, "budget B=%lld infeasible for N=%lld, r_min=%d, R=128", (long long)B,
                    (long long)N, sh->r_min);
    return VARRATE_OK;
}

// shared cross-head basis: R rows, joint budget
int64_t joint_budget(const varrate_shape& sh) {
    return varrate_coded_budget(sh.n, 2 * sh.G * VARRATE_HEAD_DIM, sh.w, sh.kappa_pct);
}

int check_joint(const varrate_shape* sh, int R) {
    int rc = check_shape_only(sh);
    if (rc) return rc;
    if (sh->rope || sh->anchor_stride)
        return fail(VARRATE_EUNSUPPORTED, "the shared basis takes position-free keys and no anchors");
    const int Dz = 2 * sh->G * VARRATE_HEAD_DIM;
    if (R < 256 || R > 1024 || R % 256 != 0 || R > Dz)
        return fail(VARRATE_EUNSUPPORTED, "R=%d: need a multiple of 256 in [256, min(1024, 2 G d = %d)]", R, Dz);
    if (sh->r_min > R) return fail(VARRATE_EINVAL, "r_min=%d exceeds R=%d", sh->r_min, R);
    const int64_t B = joint_budget(*sh);
    const int64_t N = sh->n - sh->w;
    if (N * sh->r_min > B || B > N * R)
        return fail(VARRATE_EBUDGET, "joint budget B=%lld infeasible for N=%lld, r_min=%d, R=%d", (long long)B,
                    (long long)N, sh->r_min, R);
    if (B + VARRATE_JOINT_PAD > (int64_t)UINT32_MAX)
        return fail(VARRATE_EUNSUPPORTED, "joint budget B=%lld exceeds 32-bit offsets", (long long)B);
    return VARRATE_OK;
}

int check_jcache(const varrate_shape* sh, const varrate_jcache* c) {
    if (!c) return fail(VARRATE_EINVAL, "jcache is NULL");
    int rc = check_joint(sh, c->R);
    if (rc) return rc;
    if (!c->coef || !c->rank || !c->offset || !c->chunk_off || !c->k_exact || !c->v_exact)
        return fail(VARRATE_EINVAL, "jcache has a NULL buffer");
    if (!aligned16(c->coef) || !aligned16(c->k_exact) || !aligned16(c->v_exact))
        return fail(VARRATE_EINVAL, "jcache buffers must be 16-byte aligned");
    if (c->coef_stride < joint_budget(*sh) + VARRATE_JOINT_PAD)
        return fail(VARRATE_EINVAL, "coef_stride %lld < B + %d", (long long)c->coef_stride, VARRATE_JOINT_PAD);
    if (c->cap < sh->w || c->cap > 8192) return fail(VARRATE_EINVAL, "exact capacity %lld outside [w, 8192]",
                                                     (long long)c->cap);
    return VARRATE_OK;
}

int check_cache(const varrate_shape* sh, const varrate_cache* c, bool need_layout) {
    if (!c) return fail(VARRATE_EINVAL, "cache is NULL");
    const int64_t B = coded_budget(*sh);
    if (sh->anchor_stride != 0 && (!c->k_anchor || !c->v_anchor || !c->snn || !c->inv_off || !c->inv_pos ||
                                   !c->piece_off || !c->piece_anchor))
        return fail(VARRATE_EINVAL, "cache has a NULL anchor buffer");
    if (sh->anchor_stride != 0 && (!aligned16(c->k_anchor) || !aligned16(c->v_anchor)))
        return fail(VARRATE_EINVAL, "anchor buffers must be 16-byte aligned");
    if (!c->coef_k || !c->coef_v || !c->rank || !c->chunk_off || !c->k_exact || !c->v_exact ||
        (need_layout && (!c->srank || !c->sidx)))
        return fail(VARRATE_EINVAL, "cache has a NULL buffer");
    if (!aligned16(c->coef_k) || !aligned16(c->coef_v) || !aligned16(c->k_exact) || !aligned16(c->v_exact))
        return fail(VARRATE_EINVAL, "cache buffers must be 16-byte aligned");
    const int64_t N = coded_count(*sh);
    const int64_t need = B + (int64_t)8 * VARRATE_CHUNK * ((N + VARRATE_CHUNK - 1) / VARRATE_CHUNK) + VARRATE_COEF_PAD;
    if (c->coef_stride < need || (c->coef_stride % 8) != 0)
        return fail(VARRATE_EINVAL, "coef_stride=%lld must be a multiple of 8 and >= %lld (B + 2048 per chunk + %d)",
                    (long long)c->coef_stride, (long long)need, VARRATE_COEF_PAD);
    if (c->cap < sh->w) return fail(VARRATE_EINVAL, "exact capacity %lld < w=%d", (long long)c->cap, sh->w);
    return VARRATE_OK;
}

size_t compress_ws_base(const varrate_shape& sh) {
    const int64_t N = sh.n - sh.w;
    return align256(salience_ws_bytes(sh)) + align256(allocate_ws_bytes(sh)) + align256((size_t)N * 4);
}

// rotary keys: the un-rotated copy of K [n][G][d] follows the other buffers
size_t compress_ws(const varrate_shape& sh) {
    if (sh.anchor_stride != 0) return anchor_ws_bytes(sh);
    const size_t es = sh.dtype == VARRATE_BF16 ? 2 : 4;
    return compress_ws_base(sh) + (sh.rope ? align256((size_t)sh.n * sh.G * VARRATE_HEAD_DIM * es) : 0);
}

// Eq. (6) projection; with rotary keys, of the keys turned back to pre-RoPE (Algorithm 1,
// first step) in the workspace
// chunk_sizes: as launch_project's (NULL: the cache's chunk table is already scanned)
hipError_t project_keys(const varrate_shape& sh, const void* K, const void* V, const float* PK,
                        const float* PV, varrate_cache& c, uint8_t* ws, hipStream_t st,
                        const uint32_t* chunk_sizes = nullptr) {
    if (!sh.rope) return launch_project(sh, K, V, PK, PV, c, st, chunk_sizes);
    void* Kr = ws + compress_ws_base(sh);
    hipError_t e = launch_rope_unrotate(sh, K, Kr, st);
    if (e != hipSuccess) return e;
    return launch_project(sh, Kr, V, PK, PV, c, st, chunk_sizes);
}

}  // namespace

extern "C" {

const char* varrate_status_string(int s) {
    switch (s) {
        case VARRATE_OK: return "ok";
        case VARRATE_EINVAL: return "invalid argument";
        case VARRATE_EBUDGET: return "infeasible budget";
        case VARRATE_EUNSUPPORTED: return "unsupported shape";
        case VARRATE_EHIP: return "HIP runtime error";
        default: return "unknown status";
    }
}

const char* varrate_last_error(void) { return g_err.c_str(); }

int varrate_version(void) { return 1; }

int varrate_read_probe(const void* src, size_t bytes, uint32_t* sink, void* stream) {
    if (!src || !sink || !aligned16(src) || bytes == 0 || bytes % 16 != 0)
        return fail(VARRATE_EINVAL, "read probe: src and sink non-NULL, src 16-byte aligned, bytes a positive "
                                    "multiple of 16");
    return hip_status(launch_read_probe(src, bytes, sink, (hipStream_t)stream), "read probe launch");
}

int64_t varrate_coded_budget(int64_t n, int32_t d, int32_t w, int32_t kappa_pct) {
    return ((int64_t)kappa_pct * n * d) / 100 - (int64_t)w * d;
}

int varrate_cache_bytes(const varrate_shape* sh, int64_t cap, varrate_cache_bytes_t* out) {
    int rc = check_shape(sh);
    if (rc) return rc;
    if (!out) return fail(VARRATE_EINVAL, "out is NULL");
    if (cap < sh->w) return fail(VARRATE_EINVAL, "exact capacity %lld < w=%d", (long long)cap, sh->w);
    const size_t es = sh->dtype == VARRATE_BF16 ? 2 : 4;
    out->N = coded_count(*sh);
    out->B = coded_budget(*sh);
    out->na = anchor_count(*sh);
    out->k_anchor = out->v_anchor = (size_t)out->na * sh->G * VARRATE_HEAD_DIM * es;
    out->snn = out->na ? (size_t)out->N * 4 * 2 : 0;
    out->inv_off = out->na ? (size_t)(out->na + 1) * 4 : 0;
    out->inv_pos = out->na ? (size_t)out->N * 4 * 4 : 0;
    out->piece_off = out->inv_off;
    out->piece_anchor = out->na ? (size_t)(out->N * 4 / 64 + out->na) * 2 : 0;
    out->n_chunks = (out->N + VARRATE_CHUNK - 1) / VARRATE_CHUNK;
    // tile rectangles: a chunk's 16 tiles take at most its ranks + 16 x 128 elements
    const int64_t bound = out->B + (int64_t)8 * VARRATE_CHUNK * out->n_chunks;
    out->coef_stride = ((bound + VARRATE_COEF_PAD + 63) / 64) * 64;
    out->coef_k = out->coef_v = (size_t)sh->G * out->coef_stride * es;
    out->rank = out->srank = (size_t)((out->N + 63) / 64) * 64;   // padded for 16-byte loads
    out->sidx = (size_t)out->N * 4;
    out->chunk_off = (size_t)(out->n_chunks + 1) * 4;
    out->k_exact = out->v_exact = (size_t)sh->G * cap * VARRATE_HEAD_DIM * es;
    return VARRATE_OK;
}

size_t varrate_compress_workspace_bytes(const varrate_shape* sh) {
    if (check_shape(sh)) return 0;
    return compress_ws(*sh);
}

size_t varrate_decode_workspace_bytes(const varrate_shape* sh, int32_t S, int32_t Q) {
    if (check_shape(sh) || S < 1 || Q < 1) return 0;
    return decode_ws_bytes(*sh, S, Q);
}

static int ws_check(void* ws, size_t have, size_t need) {
    if (!ws) return fail(VARRATE_EINVAL, "workspace is NULL");
    if (!aligned16(ws)) return fail(VARRATE_EINVAL, "workspace must be 16-byte aligned");
    if (have < need) return fail(VARRATE_EINVAL, "workspace %zu bytes < required %zu", have, need);
    return VARRATE_OK;
}

int varrate_salience(const varrate_shape* sh, const void* K, const void* Qw, float* sbar, void* ws,
                     size_t ws_bytes, void* stream) {
    int rc = check_shape(sh);
    if (rc) return rc;
    if (!K || !Qw || !sbar) return fail(VARRATE_EINVAL, "K, Qw and sbar must be non-NULL");
    if (!aligned16(K) || !aligned16(Qw)) return fail(VARRATE_EINVAL, "K and Qw must be 16-byte aligned");
    if ((rc = ws_check(ws, ws_bytes, compress_ws(*sh)))) return rc;
    return hip_status(launch_salience(*sh, K, Qw, sbar, (uint8_t*)ws, (hipStream_t)stream), "salience launch");
}

int varrate_allocate(const varrate_shape* sh, const float* sbar, varrate_cache* c, void* ws,
                     size_t ws_bytes, void* stream) {
    int rc = check_shape(sh);
    if (rc) return rc;
    if (sh->anchor_stride) return fail(VARRATE_EUNSUPPORTED, "residual codec: use varrate_anchor_encode");
    if ((rc = check_cache(sh, c, false))) return rc;
    if (!sbar) return fail(VARRATE_EINVAL, "sbar is NULL");
    if ((rc = ws_check(ws, ws_bytes, compress_ws(*sh)))) return rc;
    c->N = sh->n - sh->w;
    c->B = varrate_coded_budget(sh->n, sh->d, sh->w, sh->kappa_pct);
    uint8_t* w8 = (uint8_t*)ws + align256(salience_ws_bytes(*sh));
    return hip_status(launch_allocate(*sh, sbar, *c, w8, (hipStream_t)stream), "allocate launch");
}

int varrate_project(const varrate_shape* sh, const void* K, const void* V, const float* PK,
                    const float* PV, varrate_cache* c, void* ws, size_t ws_bytes, void* stream) {
    int rc = check_shape(sh);
    if (rc) return rc;
    if (sh->anchor_stride) return fail(VARRATE_EUNSUPPORTED, "residual codec: use varrate_anchor_encode");
    if ((rc = check_cache(sh, c, true))) return rc;
    if (!K || !V || !PK || !PV) return fail(VARRATE_EINVAL, "K, V, P_K and P_V must be non-NULL");
    if (!aligned16(K) || !aligned16(V) || !aligned16(PK) || !aligned16(PV))
        return fail(VARRATE_EINVAL, "K, V, P_K, P_V must be 16-byte aligned");
    if ((rc = ws_check(ws, ws_bytes, compress_ws(*sh)))) return rc;
    c->N = sh->n - sh->w;
    c->B = varrate_coded_budget(sh->n, sh->d, sh->w, sh->kappa_pct);
    hipStream_t st = (hipStream_t)stream;
    rc = hip_status(project_keys(*sh, K, V, PK, PV, *c, (uint8_t*)ws, st), "project launch");
    if (rc) return rc;
    c->n_exact = sh->w;
    return VARRATE_OK;
}

int varrate_compress(const varrate_shape* sh, const void* K, const void* V, const void* Qw,
                     const float* PK, const float* PV, varrate_cache* c, float* sbar_out, void* ws,
                     size_t ws_bytes, void* stream) {
    int rc = check_shape(sh);
    if (rc) return rc;
    if ((rc = check_cache(sh, c, true))) return rc;
    if (!K || !V || !Qw || !PK || !PV) return fail(VARRATE_EINVAL, "inputs must be non-NULL");
    if ((rc = ws_check(ws, ws_bytes, compress_ws(*sh)))) return rc;
    if (!aligned16(K) || !aligned16(V) || !aligned16(Qw) || !aligned16(PK) || !aligned16(PV))
        return fail(VARRATE_EINVAL, "K, V, Qw, P_K, P_V must be 16-byte aligned");
    if (sh->anchor_stride) {
        // residual codec: salience over the whole prefix (pooled), anchor search, encode
        hipStream_t st = (hipStream_t)stream;
        const AnchorWs w = anchor_ws(*sh, (uint8_t*)ws);
        float* sb = sbar_out ? sbar_out : w.sbar;
        if ((rc = hip_status(launch_salience(*sh, K, Qw, sb, w.sal, st, true), "salience launch"))) return rc;
        if ((rc = hip_status(launch_anchor_search(*sh, K, V, w.nn, w, st), "anchor search launch"))) return rc;
        c->N = coded_count(*sh);
        c->B = coded_budget(*sh);
        c->na = anchor_count(*sh);
        if ((rc = hip_status(launch_anchor_encode(*sh, K, V, sb, w.nn, PK, PV, *c, w, st), "anchor encode launch")))
            return rc;
        c->n_exact = sh->w;
        return VARRATE_OK;
    }
    float* sbar = sbar_out;
    if (!sbar) {
        sbar = (float*)((uint8_t*)ws + align256(salience_ws_bytes(*sh)) + align256(allocate_ws_bytes(*sh)));
    }
    // salience passes, then the allocation's first pass pools sbar from the column sums
    // itself (the separate pooling launch is skipped), then the rest of the allocation and
    // the projection, which scans the chunk sizes into the chunk table itself (the
    // allocation's scan launch is skipped): the same results as the three entry points in turn
    hipStream_t st = (hipStream_t)stream;
    uint8_t* w0 = (uint8_t*)ws;
    if ((rc = hip_status(launch_salience(*sh, K, Qw, sbar, w0, st, false), "salience launch"))) return rc;
    c->N = sh->n - sh->w;
    c->B = varrate_coded_budget(sh->n, sh->d, sh->w, sh->kappa_pct);
    uint8_t* w8 = w0 + align256(salience_ws_bytes(*sh));
    const uint32_t* csz = nullptr;
    if ((rc = hip_status(launch_allocate(*sh, sbar, *c, w8, st, salience_part(*sh, w0), &csz), "allocate launch")))
        return rc;
    if ((rc = hip_status(project_keys(*sh, K, V, PK, PV, *c, w0, st, csz), "project launch"))) return rc;
    c->n_exact = sh->w;
    return VARRATE_OK;
}

int varrate_anchor_search(const varrate_shape* sh, const void* K, const void* V, uint16_t* nn, void* ws,
                          size_t ws_bytes, void* stream) {
    int rc = check_shape(sh);
    if (rc) return rc;
    if (!sh->anchor_stride) return fail(VARRATE_EINVAL, "anchor_stride is 0");
    if (!K || !V || !nn) return fail(VARRATE_EINVAL, "K, V and nn must be non-NULL");
    if (!aligned16(K) || !aligned16(V)) return fail(VARRATE_EINVAL, "K and V must be 16-byte aligned");
    if ((rc = ws_check(ws, ws_bytes, compress_ws(*sh)))) return rc;
    const AnchorWs w = anchor_ws(*sh, (uint8_t*)ws);
    return hip_status(launch_anchor_search(*sh, K, V, nn, w, (hipStream_t)stream), "anchor search launch");
}

int varrate_anchor_encode(const varrate_shape* sh, const void* K, const void* V, const float* sbar, const uint16_t* nn,
                          const float* PK, const float* PV, varrate_cache* c, void* ws, size_t ws_bytes, void* stream) {
    int rc = check_shape(sh);
    if (rc) return rc;
    if (!sh->anchor_stride) return fail(VARRATE_EINVAL, "anchor_stride is 0");
    if ((rc = check_cache(sh, c, true))) return rc;
    if (!K || !V || !sbar || !nn || !PK || !PV) return fail(VARRATE_EINVAL, "inputs must be non-NULL");
    if (!aligned16(K) || !aligned16(V) || !aligned16(PK) || !aligned16(PV))
        return fail(VARRATE_EINVAL, "K, V, P_K, P_V must be 16-byte aligned");
    if ((rc = ws_check(ws, ws_bytes, compress_ws(*sh)))) return rc;
    const AnchorWs w = anchor_ws(*sh, (uint8_t*)ws);
    c->N = coded_count(*sh);
    c->B = coded_budget(*sh);
    c->na = anchor_count(*sh);
    if ((rc = hip_status(launch_anchor_encode(*sh, K, V, sbar, nn, PK, PV, *c, w, (hipStream_t)stream),
                         "anchor encode launch")))
        return rc;
    c->n_exact = sh->w;
    return VARRATE_OK;
}

int varrate_append_exact(const varrate_shape* sh, varrate_cache* c, const void* k_new, const void* v_new,
                         void* stream) {
    int rc = check_shape(sh);
    if (rc) return rc;
    if ((rc = check_cache(sh, c, false))) return rc;
    if (!k_new || !v_new) return fail(VARRATE_EINVAL, "k_new and v_new must be non-NULL");
    if (c->n_exact >= c->cap) return fail(VARRATE_EINVAL, "exact capacity %lld is full", (long long)c->cap);
    const size_t es = sh->dtype == VARRATE_BF16 ? 2 : 4;
    const size_t row = VARRATE_HEAD_DIM * es;
    hipStream_t st = (hipStream_t)stream;
    for (int kv = 0; kv < 2; ++kv) {
        uint8_t* dst = (uint8_t*)(kv ? c->v_exact : c->k_exact) + (size_t)c->n_exact * row;
        const void* src = kv ? v_new : k_new;
        hipError_t e = hipMemcpy2DAsync(dst, (size_t)c->cap * row, src, row, row, sh->G,
                                        hipMemcpyDeviceToDevice, st);
        if ((rc = hip_status(e, "append copy"))) return rc;
    }
    c->n_exact += 1;
    return VARRATE_OK;
}

static int check_decode(const varrate_shape* sh, const varrate_cache* caches, int32_t S, const void* q,
                        int32_t Q, const float* PK, const float* PV, void* out) {
    int rc = check_shape(sh);
    if (rc) return rc;
    if (!caches || S < 1 || S > VARRATE_MAX_SEQS) return fail(VARRATE_EINVAL, "S=%d outside [1, %d]", S, VARRATE_MAX_SEQS);
    if (Q < 1 || (int64_t)Q * (sh->H / sh->G) > VARRATE_MAX_QROWS)
        return fail(VARRATE_EUNSUPPORTED, "Q=%d query rows per KV head exceed %d", Q, VARRATE_MAX_QROWS);
    if (!q || !out || !PK || !PV) return fail(VARRATE_EINVAL, "q, out, P_K, P_V must be non-NULL");
    if (!aligned16(q) || !aligned16(PK) || !aligned16(PV))
        return fail(VARRATE_EINVAL, "q, P_K, P_V must be 16-byte aligned");
    for (int s = 0; s < S; ++s) {
        if ((rc = check_cache(sh, &caches[s], true))) return rc;
        if (caches[s].N != coded_count(*sh)) return fail(VARRATE_EINVAL, "cache %d was not compressed with this shape", s);
        if (caches[s].n_exact < 0 || caches[s].n_exact > caches[s].cap)
            return fail(VARRATE_EINVAL, "cache %d has n_exact outside [0, cap]", s);
        if (caches[s].coef_stride != caches[0].coef_stride || caches[s].cap != caches[0].cap)
            return fail(VARRATE_EINVAL, "caches must share coef_stride and cap");
    }
    if (!decode_supported(*sh, S, Q))
        return fail(VARRATE_EUNSUPPORTED, "S * G * ceil(Q H/G / 16) exceeds 16384 merge slots");
    return VARRATE_OK;
}

int varrate_decode_attn(const varrate_shape* sh, const varrate_cache* caches, int32_t S, const void* q,
                        int32_t Q, const float* PK, const float* PV, void* out, void* ws, size_t ws_bytes,
                        void* stream) {
    int rc = check_decode(sh, caches, S, q, Q, PK, PV, out);
    if (rc) return rc;
    if ((rc = ws_check(ws, ws_bytes, decode_ws_bytes(*sh, S, Q)))) return rc;
    return hip_status(launch_decode(*sh, caches, S, q, Q, PK, PV, out, (uint8_t*)ws, (hipStream_t)stream),
                      "decode launch");
}

int varrate_qcache_bytes(const varrate_shape* sh, int32_t bits, int64_t* q_stride, size_t* qchunk_off_bytes) {
    int rc = check_shape(sh);
    if (rc) return rc;
    if (bits != 3 && bits != 4 && bits != 8) return fail(VARRATE_EUNSUPPORTED, "bits=%d not in {3, 4, 8}", bits);
    if (!q_stride || !qchunk_off_bytes) return fail(VARRATE_EINVAL, "outputs must be non-NULL");
    const int64_t N = coded_count(*sh);
    *q_stride = (int64_t)qcache_stride(*sh, bits);
    *qchunk_off_bytes = (size_t)((N + VARRATE_CHUNK - 1) / VARRATE_CHUNK + 1) * 4;
    return VARRATE_OK;
}

static int check_qcache(const varrate_shape* sh, const varrate_qcache* q) {
    if (!q) return fail(VARRATE_EINVAL, "qcache is NULL");
    if (sh->dtype != VARRATE_BF16) return fail(VARRATE_EUNSUPPORTED, "quantised coefficients need a bf16 layer");
    if (q->bits != 3 && q->bits != 4 && q->bits != 8)
        return fail(VARRATE_EUNSUPPORTED, "bits=%d not in {3, 4, 8}", q->bits);
    if (!q->code_k || !q->code_v || !q->qchunk_off) return fail(VARRATE_EINVAL, "qcache has a NULL buffer");
    if (!aligned16(q->code_k) || !aligned16(q->code_v)) return fail(VARRATE_EINVAL, "code buffers must be 16-byte aligned");
    const int64_t need = (int64_t)qcache_stride(*sh, q->bits);
    if (q->q_stride < need || (q->q_stride % 16) != 0)
        return fail(VARRATE_EINVAL, "q_stride=%lld must be a multiple of 16 and >= %lld", (long long)q->q_stride,
                    (long long)need);
    return VARRATE_OK;
}

int varrate_quantize(const varrate_shape* sh, const varrate_cache* c, varrate_qcache* q, void* stream) {
    int rc = check_shape(sh);
    if (rc) return rc;
    if (sh->rope) return fail(VARRATE_EUNSUPPORTED, "quantised coefficients of rotary keys");
    if ((rc = check_cache(sh, c, true))) return rc;
    if ((rc = check_qcache(sh, q))) return rc;
    return hip_status(launch_quantize(*sh, *c, *q, (hipStream_t)stream), "quantize launch");
}

int varrate_decode_attn_q(const varrate_shape* sh, const varrate_cache* caches, const varrate_qcache* qcaches,
                          int32_t S, const void* q, int32_t Q, const float* PK, const float* PV, void* out,
                          void* ws, size_t ws_bytes, void* stream) {
    int rc = check_decode(sh, caches, S, q, Q, PK, PV, out);
    if (rc) return rc;
    if (sh->rope) return fail(VARRATE_EUNSUPPORTED, "quantised coefficients of rotary keys");
    if (!qcaches) return fail(VARRATE_EINVAL, "qcaches is NULL");
    for (int s = 0; s < S; ++s) {
        if ((rc = check_qcache(sh, &qcaches[s]))) return rc;
        if (qcaches[s].bits != qcaches[0].bits || qcaches[s].q_stride != qcaches[0].q_stride)
            return fail(VARRATE_EINVAL, "qcaches must share bits and q_stride");
    }
    if ((rc = ws_check(ws, ws_bytes, decode_ws_bytes(*sh, S, Q)))) return rc;
    return hip_status(launch_decode(*sh, caches, S, q, Q, PK, PV, out, (uint8_t*)ws, (hipStream_t)stream, false,
                                    qcaches),
                      "decode launch");
}

int varrate_jcache_bytes(const varrate_shape* sh, int32_t R, int64_t cap, varrate_jcache_bytes_t* out) {
    int rc = check_joint(sh, R);
    if (rc) return rc;
    if (!out) return fail(VARRATE_EINVAL, "out is NULL");
    if (cap < sh->w || cap > 8192) return fail(VARRATE_EINVAL, "exact capacity %lld outside [w, 8192]", (long long)cap);
    const size_t es = sh->dtype == VARRATE_BF16 ? 2 : 4;
    out->N = sh->n - sh->w;
    out->B = joint_budget(*sh);
    out->n_chunks = (out->N + VARRATE_CHUNK - 1) / VARRATE_CHUNK;
    out->coef_stride = ((out->B + VARRATE_JOINT_PAD + 63) / 64) * 64;
    out->coef = (size_t)out->coef_stride * es;
    out->rank = (size_t)((out->N + 31) / 32) * 64;
    out->offset = (size_t)(out->N + 1) * 4;
    out->chunk_off = (size_t)(out->n_chunks + 1) * 4;
    out->k_exact = out->v_exact = (size_t)sh->G * cap * VARRATE_HEAD_DIM * es;
    return VARRATE_OK;
}

size_t varrate_joint_compress_workspace_bytes(const varrate_shape* sh, int32_t R) {
    if (check_joint(sh, R)) return 0;
    return compress_ws_base(*sh) + joint_project_ws_bytes(*sh, R);
}

size_t varrate_joint_decode_workspace_bytes(const varrate_shape* sh, int32_t R, int32_t S, int32_t Q) {
    if (check_joint(sh, R) || S < 1 || Q < 1 || (int64_t)Q * sh->H > 32) return 0;
    return joint_decode_ws_bytes(*sh, R, S, Q);
}

int varrate_joint_compress(const varrate_shape* sh, const void* K, const void* V, const void* Qw, const float* W,
                           varrate_jcache* c, float* sbar_out, void* ws, size_t ws_bytes, void* stream) {
    int rc = check_jcache(sh, c);
    if (rc) return rc;
    if (!K || !V || !Qw || !W) return fail(VARRATE_EINVAL, "inputs must be non-NULL");
    if (!aligned16(K) || !aligned16(V) || !aligned16(Qw) || !aligned16(W))
        return fail(VARRATE_EINVAL, "K, V, Qw, W must be 16-byte aligned");
    if ((rc = ws_check(ws, ws_bytes, varrate_joint_compress_workspace_bytes(sh, c->R)))) return rc;
    hipStream_t st = (hipStream_t)stream;
    uint8_t* w0 = (uint8_t*)ws;
    uint8_t* wp = w0 + compress_ws_base(*sh);
    float* sbar = sbar_out ? sbar_out
                           : (float*)(w0 + align256(salience_ws_bytes(*sh)) + align256(allocate_ws_bytes(*sh)));
    c->N = sh->n - sh->w;
    c->B = joint_budget(*sh);
    if ((rc = hip_status(launch_salience(*sh, K, Qw, sbar, w0, st, false), "salience launch"))) return rc;
    uint8_t* w8 = w0 + align256(salience_ws_bytes(*sh));
    if ((rc = hip_status(launch_allocate_joint(*sh, c->R, c->B, sbar, c->rank, c->offset, c->chunk_off, w8, st,
                                               salience_part(*sh, w0), joint_lists(*sh, c->R, wp)),
                         "allocate launch")))
        return rc;
    if ((rc = hip_status(launch_joint_project(*sh, c->R, K, V, W, *c, wp, st), "project launch"))) return rc;
    c->n_exact = sh->w;
    return VARRATE_OK;
}

int varrate_joint_decode_attn(const varrate_shape* sh, const varrate_jcache* caches, int32_t S, const void* q,
                              int32_t Q, const float* W, void* out, void* ws, size_t ws_bytes, void* stream) {
    if (!caches || S < 1 || S > VARRATE_MAX_SEQS) return fail(VARRATE_EINVAL, "S=%d outside [1, %d]", S, VARRATE_MAX_SEQS);
    int rc;
    for (int s = 0; s < S; ++s) {
        if ((rc = check_jcache(sh, &caches[s]))) return rc;
        if (caches[s].N != sh->n - sh->w || caches[s].R != caches[0].R || caches[s].cap != caches[0].cap)
            return fail(VARRATE_EINVAL, "jcache %d does not match the shape, R or cap of jcache 0", s);
        if (caches[s].n_exact < 1 || caches[s].n_exact > caches[s].cap)
            return fail(VARRATE_EINVAL, "jcache %d has n_exact outside [1, cap]", s);
    }
    if (Q < 1 || (int64_t)Q * sh->H > 32) return fail(VARRATE_EUNSUPPORTED, "Q H = %lld query rows exceed 32",
                                                      (long long)Q * sh->H);
    if (!q || !out || !W) return fail(VARRATE_EINVAL, "q, out and W must be non-NULL");
    if (!aligned16(q) || !aligned16(W)) return fail(VARRATE_EINVAL, "q and W must be 16-byte aligned");
    if ((rc = ws_check(ws, ws_bytes, joint_decode_ws_bytes(*sh, caches[0].R, S, Q)))) return rc;
    return hip_status(launch_joint_decode(*sh, caches[0].R, caches, S, q, Q, W, out, (uint8_t*)ws,
                                          (hipStream_t)stream),
                      "joint decode launch");
}

int varrate_joint_append_exact(const varrate_shape* sh, varrate_jcache* c, const void* k_new, const void* v_new,
                               void* stream) {
    int rc = check_jcache(sh, c);
    if (rc) return rc;
    if (!k_new || !v_new) return fail(VARRATE_EINVAL, "k_new and v_new must be non-NULL");
    if (c->n_exact >= c->cap) return fail(VARRATE_EINVAL, "exact capacity %lld is full", (long long)c->cap);
    const size_t es = sh->dtype == VARRATE_BF16 ? 2 : 4;
    const size_t row = VARRATE_HEAD_DIM * es;
    hipStream_t st = (hipStream_t)stream;
    for (int kv = 0; kv < 2; ++kv) {
        uint8_t* dst = (uint8_t*)(kv ? c->v_exact : c->k_exact) + (size_t)c->n_exact * row;
        const void* src = kv ? v_new : k_new;
        hipError_t e = hipMemcpy2DAsync(dst, (size_t)c->cap * row, src, row, row, sh->G, hipMemcpyDeviceToDevice, st);
        if ((rc = hip_status(e, "append copy"))) return rc;
    }
    c->n_exact += 1;
    return VARRATE_OK;
}

size_t varrate_decode_scratch_need(const varrate_shape* sh, int32_t S, int32_t Q) {
    if (check_shape(sh) || S < 1 || S > VARRATE_MAX_SEQS || Q < 1 ||
        (int64_t)Q * (sh->H / sh->G) > VARRATE_MAX_QROWS)
        return 0;
    return decode_group_bytes(*sh, S, Q);
}

int varrate_decode_attn_noalloc(const varrate_shape* sh, const varrate_cache* caches, int32_t S, const void* q,
                                int32_t Q, const float* PK, const float* PV, void* out, void* stream) {
    int rc = check_decode(sh, caches, S, q, Q, PK, PV, out);
    if (rc) return rc;
    if (sh->anchor_stride || sh->rope)
        return fail(VARRATE_EUNSUPPORTED, "the residual codec's and rotary keys' decode need a workspace "
                                          "(varrate_decode_attn)");
    const size_t need = decode_group_bytes(*sh, S, Q);
    if (need > (size_t)VARRATE_DECODE_SCRATCH_BYTES)
        return fail(VARRATE_EUNSUPPORTED,
                    "this decode needs %zu bytes of partial records, more than the fixed %zu-byte scratch; "
                    "call varrate_decode_attn with a workspace instead",
                    need, (size_t)VARRATE_DECODE_SCRATCH_BYTES);
    uint8_t* scratch = nullptr;
    if ((rc = hip_status(decode_scratch(&scratch), "decode scratch lookup"))) return rc;
    return hip_status(launch_decode(*sh, caches, S, q, Q, PK, PV, out, scratch, (hipStream_t)stream, true),
                      "decode launch");
}

// ---- paged cache ------------------------------------------------------------------------------

static int check_dtype(int dtype) {
    if (dtype != VARRATE_BF16 && dtype != VARRATE_F32) return fail(VARRATE_EINVAL, "unknown dtype %d", dtype);
    return VARRATE_OK;
}

static int check_pages(const varrate_pages* pg) {
    if (!pg) return fail(VARRATE_EINVAL, "pages is NULL");
    if (pg->d != VARRATE_HEAD_DIM) return fail(VARRATE_EUNSUPPORTED, "head dim %d != 128", pg->d);
    int rc = check_dtype(pg->dtype);
    if (rc) return rc;
    if (pg->G < 1 || pg->G > 1024) return fail(VARRATE_EINVAL, "G=%d outside [1, 1024]", pg->G);
    if (pg->page < PAGE_MIN || pg->page > PAGE_MAX || (pg->page & (pg->page - 1)) != 0)
        return fail(VARRATE_EUNSUPPORTED, "page=%d: need a power of two in [16, 256]", pg->page);
    if (pg->n_pages < 1 || pg->n_pages > INT32_MAX)
        return fail(VARRATE_EINVAL, "n_pages=%lld outside [1, 2^31 - 1]", (long long)pg->n_pages);
    if (!pg->k || !pg->v) return fail(VARRATE_EINVAL, "pages has a NULL buffer");
    if (!aligned16(pg->k) || !aligned16(pg->v)) return fail(VARRATE_EINVAL, "page buffers must be 16-byte aligned");
    return VARRATE_OK;
}

static int check_width(int32_t width, int32_t page) {
    if (width < 1 || (int64_t)width * page > ((int64_t)1 << 30))
        return fail(VARRATE_EINVAL, "table width %d outside [1, 2^30 / page]", width);
    return VARRATE_OK;
}

static int check_batch(const varrate_batch* b, int32_t page) {
    if (!b) return fail(VARRATE_EINVAL, "batch is NULL");
    if (!b->table || !b->kv_len || !b->q_start) return fail(VARRATE_EINVAL, "batch has a NULL array");
    if (((uintptr_t)b->table | (uintptr_t)b->kv_len | (uintptr_t)b->q_start) & 3u)
        return fail(VARRATE_EINVAL, "batch arrays must be 4-byte aligned");
    if (b->S < 1 || b->S > 65536) return fail(VARRATE_EINVAL, "S=%d outside [1, 65536]", b->S);
    if (b->T < 0) return fail(VARRATE_EINVAL, "T=%lld is negative", (long long)b->T);
    int rc = check_width(b->width, page);
    if (rc) return rc;
    if (b->table_stride < 0) return fail(VARRATE_EINVAL, "table_stride=%lld is negative", (long long)b->table_stride);
    return VARRATE_OK;
}

// rows [T][heads][128] with `stride` elements between tokens; outputs must not overlap themselves
static int check_rows(const void* p, int64_t stride, int64_t T, int32_t heads, int dtype, bool out, const char* name) {
    if (!p) return fail(VARRATE_EINVAL, "%s is NULL", name);
    const int per16 = dtype == VARRATE_BF16 ? 8 : 4;
    if (!aligned16(p) || stride % per16 != 0)
        return fail(VARRATE_EINVAL, "%s must be 16-byte aligned, its tokens %d elements or a multiple apart", name, per16);
    if (stride < 0 || (out && T > 1 && stride < (int64_t)heads * VARRATE_HEAD_DIM))
        return fail(VARRATE_EINVAL, "%s: %lld elements between tokens", name, (long long)stride);
    return VARRATE_OK;
}

// 32-bit row numbers
static int check_rows_total(int64_t T, int64_t heads) {
    if (T > ((int64_t)1 << 30) / heads)
        return fail(VARRATE_EUNSUPPORTED, "T=%lld tokens of %lld heads exceed 2^30 rows", (long long)T, (long long)heads);
    return VARRATE_OK;
}

int varrate_norm_rotate(int32_t dtype, int64_t T, const void* q, int64_t q_stride, int32_t H, const void* k,
                        int64_t k_stride, int32_t G, const int32_t* pos, const float* theta, const float* wq,
                        int64_t wq_stride, const float* wk, int64_t wk_stride, float eps, void* q_out,
                        int64_t q_out_stride, void* k_out, int64_t k_out_stride, void* stream) {
    int rc = check_dtype(dtype);
    if (rc) return rc;
    if (T < 0) return fail(VARRATE_EINVAL, "T=%lld is negative", (long long)T);
    if (H < 0 || G < 0 || H + (int64_t)G < 1 || H > 65536 || G > 65536)
        return fail(VARRATE_EINVAL, "H=%d G=%d: need one head at least, 65536 at most", H, G);
    if ((rc = check_rows_total(T, (int64_t)H + G))) return rc;
    if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(VARRATE_EINVAL, "eps is negative or not finite");
    if (theta && !pos) return fail(VARRATE_EINVAL, "rotation needs pos");
    if (((uintptr_t)theta | (uintptr_t)pos) & 3u) return fail(VARRATE_EINVAL, "theta and pos must be 4-byte aligned");
    for (int side = 0; side < 2; ++side) {
        const float* w = side ? wk : wq;
        const int64_t ws = side ? wk_stride : wq_stride;
        if (w && (!aligned16(w) || (ws != 0 && ws != VARRATE_HEAD_DIM)))
            return fail(VARRATE_EINVAL, "%s must be 16-byte aligned, its heads 0 or 128 elements apart", side ? "wk" : "wq");
    }
    if (T == 0) return VARRATE_OK;
    if (H && ((rc = check_rows(q, q_stride, T, H, dtype, false, "q")) ||
              (rc = check_rows(q_out, q_out_stride, T, H, dtype, true, "q_out")))) return rc;
    if (G && ((rc = check_rows(k, k_stride, T, G, dtype, false, "k")) ||
              (rc = check_rows(k_out, k_out_stride, T, G, dtype, true, "k_out")))) return rc;
    if (H && q == q_out && q_stride != q_out_stride && T > 1) return fail(VARRATE_EINVAL, "q_out is q with another stride");
    if (G && k == k_out && k_stride != k_out_stride && T > 1) return fail(VARRATE_EINVAL, "k_out is k with another stride");
    const NormRotate n = {q, k, q_out, k_out, q_stride, k_stride, q_out_stride, k_out_stride, wq_stride, wk_stride,
                          pos, theta, wq, wk, eps, T, H, G};
    return hip_status(launch_norm_rotate(dtype, n, (hipStream_t)stream), "norm and rotation launch");
}

int varrate_paged_append(const varrate_pages* pg, const varrate_batch* b, const void* k_new, int64_t k_stride,
                         const void* v_new, int64_t v_stride, const float* theta, void* stream) {
    int rc = check_pages(pg);
    if (rc || (rc = check_batch(b, pg->page)) || (rc = check_rows_total(b->T, 2 * pg->G))) return rc;
    if ((uintptr_t)theta & 3u) return fail(VARRATE_EINVAL, "theta must be 4-byte aligned");
    if (b->T == 0) return VARRATE_OK;
    if ((rc = check_rows(k_new, k_stride, b->T, pg->G, pg->dtype, false, "k_new")) ||
        (rc = check_rows(v_new, v_stride, b->T, pg->G, pg->dtype, false, "v_new"))) return rc;
    return hip_status(launch_paged_append(*pg, *b, k_new, k_stride, v_new, v_stride, theta, (hipStream_t)stream),
                      "paged append launch");
}

static int check_paged_heads(const varrate_pages* pg, const varrate_batch* b, int32_t H) {
    int rc = check_pages(pg);
    if (rc || (rc = check_batch(b, pg->page))) return rc;
    if (H < 1) return fail(VARRATE_EINVAL, "H=%d must be >= 1", H);
    if (H % pg->G != 0) return fail(VARRATE_EUNSUPPORTED, "H=%d is not a multiple of G=%d", H, pg->G);
    return check_rows_total(b->T, H);
}

size_t varrate_paged_attn_workspace_bytes(const varrate_pages* pg, const varrate_batch* b, int32_t H) {
    if (check_paged_heads(pg, b, H) || b->T == 0) return 0;
    return paged_attn_ws_bytes(b->T, b->S, pg->G, H, pg->dtype, (int64_t)b->width * pg->page);
}

int varrate_paged_attn(const varrate_pages* pg, const varrate_batch* b, const void* q, int64_t q_stride, int32_t H,
                       int32_t causal, int32_t window, float scale, void* out, int64_t out_stride, void* ws,
                       size_t ws_bytes, void* stream) {
    int rc = check_paged_heads(pg, b, H);
    if (rc) return rc;
    if (causal != 0 && causal != 1) return fail(VARRATE_EINVAL, "causal=%d outside {0, 1}", causal);
    if (window < 0 || window > (1 << 30)) return fail(VARRATE_EINVAL, "window=%d outside [0, 2^30]", window);
    if (window && !causal) return fail(VARRATE_EUNSUPPORTED, "a window without causal order");
    if (!(scale >= 0x1p-100f && scale <= 0x1p100f)) return fail(VARRATE_EINVAL, "scale outside [2^-100, 2^100]");
    if (b->T == 0) return VARRATE_OK;
    if ((rc = check_rows(q, q_stride, b->T, H, pg->dtype, false, "q")) ||
        (rc = check_rows(out, out_stride, b->T, H, pg->dtype, true, "out"))) return rc;
    if (q == out) return fail(VARRATE_EINVAL, "out is q");
    const size_t need = paged_attn_ws_bytes(b->T, b->S, pg->G, H, pg->dtype, (int64_t)b->width * pg->page);
    if (need && (rc = ws_check(ws, ws_bytes, need))) return rc;
    return hip_status(launch_paged_attn(*pg, *b, q, q_stride, H, causal, window, scale, out, out_stride, ws,
                                        (hipStream_t)stream),
                      "paged attention launch");
}

int varrate_paged_gather(const varrate_pages* pg, const int32_t* table, int32_t width, int64_t n, void* K, void* V,
                         void* stream) {
    int rc = check_pages(pg);
    if (rc || (rc = check_width(width, pg->page))) return rc;
    if (!table || ((uintptr_t)table & 3u)) return fail(VARRATE_EINVAL, "table must be non-NULL and 4-byte aligned");
    if (n < 0 || n > (int64_t)width * pg->page)
        return fail(VARRATE_EINVAL, "n=%lld outside [0, width page = %lld]", (long long)n, (long long)width * pg->page);
    if (n == 0) return VARRATE_OK;
    if (!K || !V || !aligned16(K) || !aligned16(V)) return fail(VARRATE_EINVAL, "K and V must be non-NULL and 16-byte aligned");
    return hip_status(launch_paged_gather(*pg, table, n, K, V, (hipStream_t)stream), "paged gather launch");
}

// ---- paged cache of 8-bit codes -----------------------------------------------------------------

static int check_pages8(const varrate_pages8* pg) {
    if (!pg) return fail(VARRATE_EINVAL, "pages is NULL");
    if (pg->d != VARRATE_HEAD_DIM) return fail(VARRATE_EUNSUPPORTED, "head dim %d != 128", pg->d);
    if (pg->G < 1 || pg->G > 1024) return fail(VARRATE_EINVAL, "G=%d outside [1, 1024]", pg->G);
    if (pg->page < VARRATE_BLOCK8 || pg->page > PAGE_MAX || (pg->page & (pg->page - 1)) != 0)
        return fail(VARRATE_EUNSUPPORTED, "page=%d: need a power of two in [32, 256]", pg->page);
    if (pg->n_pages < 1 || pg->n_pages > INT32_MAX)
        return fail(VARRATE_EINVAL, "n_pages=%lld outside [1, 2^31 - 1]", (long long)pg->n_pages);
    if (pg->reserved != 0) return fail(VARRATE_EINVAL, "reserved must be 0");
    if (!pg->k || !pg->v || !pg->k_scale || !pg->v_scale) return fail(VARRATE_EINVAL, "pages has a NULL buffer");
    if (!aligned16(pg->k) || !aligned16(pg->v)) return fail(VARRATE_EINVAL, "page buffers must be 16-byte aligned");
    return VARRATE_OK;
}

static int check_paged8(const varrate_pages8* pg, const varrate_batch* b, int32_t dtype) {
    int rc = check_pages8(pg);
    if (rc || (rc = check_batch(b, pg->page))) return rc;
    return check_dtype(dtype);
}

static int check_paged8_heads(const varrate_pages8* pg, const varrate_batch* b, int32_t dtype, int32_t H) {
    int rc = check_paged8(pg, b, dtype);
    if (rc) return rc;
    if (H < 1) return fail(VARRATE_EINVAL, "H=%d must be >= 1", H);
    if (H % pg->G != 0) return fail(VARRATE_EUNSUPPORTED, "H=%d is not a multiple of G=%d", H, pg->G);
    return check_rows_total(b->T, H);
}

static int check_attn_options(int32_t causal, int32_t window, float scale) {
    if (causal != 0 && causal != 1) return fail(VARRATE_EINVAL, "causal=%d outside {0, 1}", causal);
    if (window < 0 || window > (1 << 30)) return fail(VARRATE_EINVAL, "window=%d outside [0, 2^30]", window);
    if (window && !causal) return fail(VARRATE_EUNSUPPORTED, "a window without causal order");
    if (!(scale >= 0x1p-100f && scale <= 0x1p100f)) return fail(VARRATE_EINVAL, "scale outside [2^-100, 2^100]");
    return VARRATE_OK;
}

static int check_words(const void* p, bool needed, const char* name) {
    if ((needed && !p) || ((uintptr_t)p & 3u))
        return fail(VARRATE_EINVAL, "%s must be%s 4-byte aligned", name, needed ? " non-NULL and" : "");
    return VARRATE_OK;
}

int varrate_paged8_append(const varrate_pages8* pg, const varrate_batch* b, int32_t dtype, const void* k_new, int64_t k_stride,
                          const void* v_new, int64_t v_stride, void* stream) {
    int rc = check_paged8(pg, b, dtype);
    if (rc || (rc = check_rows_total(b->T, 2 * pg->G))) return rc;
    if (b->T == 0) return VARRATE_OK;
    if ((rc = check_rows(k_new, k_stride, b->T, pg->G, dtype, false, "k_new")) ||
        (rc = check_rows(v_new, v_stride, b->T, pg->G, dtype, false, "v_new"))) return rc;
    return hip_status(launch_paged8_append(*pg, *b, dtype, k_new, k_stride, v_new, v_stride, (hipStream_t)stream),
                      "8-bit paged append launch");
}

size_t varrate_paged8_attn_workspace_bytes(const varrate_pages8* pg, const varrate_batch* b, int32_t dtype, int32_t H) {
    if (check_paged8_heads(pg, b, dtype, H) || b->T == 0) return 0;
    return paged8_attn_ws_bytes(b->T, b->S, pg->G, H, dtype, (int64_t)b->width * pg->page);
}

int varrate_paged8_attn(const varrate_pages8* pg, const varrate_batch* b, int32_t dtype, const void* q, int64_t q_stride,
                        int32_t H, int32_t causal, int32_t window, float scale, void* out, int64_t out_stride, float* lse,
                        void* ws, size_t ws_bytes, void* stream) {
    int rc = check_paged8_heads(pg, b, dtype, H);
    if (rc || (rc = check_attn_options(causal, window, scale)) || (rc = check_words(lse, false, "lse"))) return rc;
    if (b->T == 0) return VARRATE_OK;
    if ((rc = check_rows(q, q_stride, b->T, H, dtype, false, "q")) ||
        (rc = check_rows(out, out_stride, b->T, H, dtype, true, "out"))) return rc;
    if (q == out) return fail(VARRATE_EINVAL, "out is q");
    const size_t need = paged8_attn_ws_bytes(b->T, b->S, pg->G, H, dtype, (int64_t)b->width * pg->page);
    if (need && (rc = ws_check(ws, ws_bytes, need))) return rc;
    return hip_status(launch_paged8_attn(*pg, *b, dtype, q, q_stride, H, causal, window, scale, out, out_stride, lse, ws,
                                         (hipStream_t)stream),
                      "8-bit paged attention launch");
}

int varrate_paged8_mass(const varrate_pages8* pg, const varrate_batch* b, int32_t dtype, const void* q, int64_t q_stride,
                        int32_t H, int32_t causal, int32_t window, float scale, const float* lse, const float* mass, float* out,
                        int64_t L, void* stream) {
    int rc = check_paged8_heads(pg, b, dtype, H);
    if (rc || (rc = check_attn_options(causal, window, scale))) return rc;
    if (L < 1 || L > (1 << 30)) return fail(VARRATE_EINVAL, "L=%lld outside [1, 2^30]", (long long)L);
    if ((rc = check_words(mass, true, "mass")) || (rc = check_words(out, true, "out"))) return rc;
    if (b->T && ((rc = check_rows(q, q_stride, b->T, H, dtype, false, "q")) || (rc = check_words(lse, true, "lse")))) return rc;
    return hip_status(launch_paged8_mass(*pg, *b, dtype, q, q_stride, H, causal, window, scale, lse, mass, out, L,
                                         (hipStream_t)stream),
                      "8-bit paged attention mass launch");
}

int varrate_paged8_evict(const varrate_pages8* pg, const int32_t* table, int64_t table_stride, int32_t width,
                         const int32_t* kv_len, int32_t S, const float* mass, int64_t L, int64_t keep, int64_t first,
                         int64_t recent, const int32_t* into, int64_t into_stride, int32_t into_width, int32_t* index,
                         float* mass_out, int32_t* len_out, void* stream) {
    int rc = check_pages8(pg);
    if (rc || (rc = check_width(width, pg->page)) || (rc = check_width(into_width, pg->page))) return rc;
    if (S < 1 || S > 65536) return fail(VARRATE_EINVAL, "S=%d outside [1, 65536]", S);
    if (table_stride < 0 || into_stride < 0) return fail(VARRATE_EINVAL, "a table stride is negative");
    if (L < 1 || L > (1 << 30)) return fail(VARRATE_EINVAL, "L=%lld outside [1, 2^30]", (long long)L);
    if (keep < 1 || keep > (int64_t)into_width * pg->page)
        return fail(VARRATE_EINVAL, "keep=%lld outside [1, %lld], what a row of into holds", (long long)keep,
                    (long long)into_width * pg->page);
    if (first < 0 || recent < 0 || first > keep || recent > keep - first)
        return fail(VARRATE_EINVAL, "first=%lld and recent=%lld: together 0 .. keep", (long long)first, (long long)recent);
    if ((rc = check_words(table, true, "table")) || (rc = check_words(into, true, "into")) ||
        (rc = check_words(kv_len, true, "kv_len")) || (rc = check_words(mass, true, "mass")) ||
        (rc = check_words(index, true, "index")) || (rc = check_words(mass_out, true, "mass_out")) ||
        (rc = check_words(len_out, true, "len_out"))) return rc;
    if (mass_out == mass || len_out == kv_len) return fail(VARRATE_EINVAL, "an output is an input");
    const Evict8Args e = {table, into, kv_len, table_stride, into_stride, mass, index, mass_out, len_out, L, keep, first, recent, S,
                          width};
    return hip_status(launch_paged8_evict(*pg, e, (hipStream_t)stream), "8-bit paged eviction launch");
}

int varrate_paged8_gather(const varrate_pages8* pg, const int32_t* table, int32_t width, int64_t n, int32_t dtype, void* K,
                          void* V, void* stream) {
    int rc = check_pages8(pg);
    if (rc || (rc = check_width(width, pg->page)) || (rc = check_dtype(dtype)) || (rc = check_words(table, true, "table"))) return rc;
    if (n < 0 || n > (int64_t)width * pg->page)
        return fail(VARRATE_EINVAL, "n=%lld outside [0, width page = %lld]", (long long)n, (long long)width * pg->page);
    if (n == 0) return VARRATE_OK;
    if (!K || !V || !aligned16(K) || !aligned16(V)) return fail(VARRATE_EINVAL, "K and V must be non-NULL and 16-byte aligned");
    return hip_status(launch_paged8_gather(*pg, table, n, dtype, K, V, (hipStream_t)stream), "8-bit paged gather launch");
}

}  // extern "C"
