// C ABI of librhymeflow.so: argument validation, kernel-argument packing and
// launch on the caller's stream. Every check runs before the first HIP call.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include "rf_cross_plan.h"
#include "rf_internal.h"
#include "rf_linear_plan.h"

namespace {

thread_local char g_err[512] = "";

int fail(int status, const char *fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof g_err, fmt, ap);
    va_end(ap);
    return status;
}

int ok() {
    g_err[0] = '\0';
    return RF_OK;
}

bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Byte counts are 64-bit: sizes whose product (computed in double) passes this
// are rejected before any of it is formed in integers.
constexpr double kMaxBytes = 4.0e18;

// Half-open byte ranges [a, a+na) and [b, b+nb) intersect.
bool overlaps(const void *a, int64_t na, const void *b, int64_t nb) {
    const uintptr_t pa = reinterpret_cast<uintptr_t>(a);
    const uintptr_t pb = reinterpret_cast<uintptr_t>(b);
    return pa < pb + static_cast<uintptr_t>(nb) && pb < pa + static_cast<uintptr_t>(na);
}

int launched(hipError_t e, const char *what) {
    if (e != hipSuccess)
        return fail(RF_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
    return ok();
}

// Strictly increasing ids in [0, T), copied into dst.
int check_id_list(const int32_t *ids, int32_t M, int32_t T, int32_t *dst, const char *what) {
    if (!ids) return fail(RF_ERR_INVALID_ARG, "%s: id list is NULL", what);
    if (M <= 0) return fail(RF_ERR_INVALID_ARG, "%s: M = %d must be positive", what, M);
    if (T <= 0) return fail(RF_ERR_INVALID_ARG, "%s: T = %d must be positive", what, T);
    if (T > RF_MAX_FRAMES)
        return fail(RF_ERR_RANGE, "%s: T = %d exceeds %d frames", what, T, RF_MAX_FRAMES);
    if (M > T) return fail(RF_ERR_RANGE, "%s: M = %d exceeds T = %d", what, M, T);
    for (int32_t i = 0; i < M; ++i) {
        if (ids[i] < 0 || ids[i] >= T)
            return fail(RF_ERR_RANGE, "%s: id %d at position %d outside [0, %d)", what, ids[i], i, T);
        if (i > 0 && ids[i] <= ids[i - 1])
            return fail(RF_ERR_INVALID_ARG, "%s: ids not strictly increasing at position %d", what, i);
        dst[i] = ids[i];
    }
    return RF_OK;
}

}  // namespace

extern "C" {

const char *rf_status_string(int status) {
    switch (status) {
        case RF_OK: return "RF_OK";
        case RF_ERR_INVALID_ARG: return "RF_ERR_INVALID_ARG";
        case RF_ERR_UNSUPPORTED: return "RF_ERR_UNSUPPORTED";
        case RF_ERR_RANGE: return "RF_ERR_RANGE";
        case RF_ERR_HIP: return "RF_ERR_HIP";
        default: return "RF_UNKNOWN_STATUS";
    }
}

const char *rf_last_error(void) { return g_err; }

int rf_abi_version(void) { return RF_ABI_VERSION; }

int rf_select_keyframes(const int32_t *frame_ids, int32_t n_ids, int32_t T, uint32_t flags,
                        int32_t *keyframe_ids_out, int32_t *num_keyframes_out,
                        uint8_t *keyframe_mask_out) {
    if (!keyframe_ids_out || !num_keyframes_out)
        return fail(RF_ERR_INVALID_ARG, "rf_select_keyframes: NULL output");
    if (n_ids < 0) return fail(RF_ERR_INVALID_ARG, "rf_select_keyframes: n_ids < 0");
    if (n_ids > 0 && !frame_ids)
        return fail(RF_ERR_INVALID_ARG, "rf_select_keyframes: frame_ids is NULL");
    if (T <= 0 || T > RF_MAX_FRAMES)
        return fail(RF_ERR_RANGE, "rf_select_keyframes: T = %d outside 1..%d", T, RF_MAX_FRAMES);
    if (flags & ~RF_SEL_NO_FORCE_FIRST)
        return fail(RF_ERR_INVALID_ARG, "rf_select_keyframes: unknown flags 0x%x", flags);
    uint8_t member[RF_MAX_FRAMES] = {0};
    for (int32_t i = 0; i < n_ids; ++i) {
        if (frame_ids[i] < 0 || frame_ids[i] >= T)
            return fail(RF_ERR_RANGE, "rf_select_keyframes: id %d outside [0, %d)", frame_ids[i], T);
        member[frame_ids[i]] = 1;
    }
    if (!(flags & RF_SEL_NO_FORCE_FIRST)) member[0] = 1;  // the first frame anchors the video
    int32_t n = 0;
    for (int32_t f = 0; f < T; ++f) n += member[f];
    if (n == 0) return fail(RF_ERR_INVALID_ARG, "rf_select_keyframes: empty keyframe set");
    n = 0;
    for (int32_t f = 0; f < T; ++f)
        if (member[f]) keyframe_ids_out[n++] = f;
    *num_keyframes_out = n;
    if (keyframe_mask_out)
        for (int32_t f = 0; f < T; ++f) keyframe_mask_out[f] = member[f];
    return ok();
}

int rf_keyframes_stride(int32_t T, int32_t k, int32_t *ids_out, int32_t *n_out) {
    if (!ids_out || !n_out) return fail(RF_ERR_INVALID_ARG, "rf_keyframes_stride: NULL output");
    if (k <= 0) return fail(RF_ERR_INVALID_ARG, "rf_keyframes_stride: k = %d must be positive", k);
    if (T <= 0 || T > RF_MAX_FRAMES)
        return fail(RF_ERR_RANGE, "rf_keyframes_stride: T = %d outside 1..%d", T, RF_MAX_FRAMES);
    int32_t n = 0;
    for (int32_t f = 0; f < T; f += k) ids_out[n++] = f;
    *n_out = n;
    return ok();
}

int rf_keyframes_uniform(int32_t T, int32_t M, int32_t *ids_out, int32_t *n_out) {
    if (!ids_out || !n_out) return fail(RF_ERR_INVALID_ARG, "rf_keyframes_uniform: NULL output");
    if (T <= 0 || T > RF_MAX_FRAMES)
        return fail(RF_ERR_RANGE, "rf_keyframes_uniform: T = %d outside 1..%d", T, RF_MAX_FRAMES);
    if (M <= 0 || M > T)
        return fail(RF_ERR_RANGE, "rf_keyframes_uniform: M = %d outside 1..%d", M, T);
    if (M == 1) {
        ids_out[0] = 0;
        *n_out = 1;
        return ok();
    }
    // nearest integer to i*(T-1)/(M-1), halves rounded up: floor((2i(T-1) + (M-1)) / (2(M-1)))
    for (int32_t i = 0; i < M; ++i) {
        const int64_t num = 2LL * i * (T - 1) + (M - 1);
        ids_out[i] = static_cast<int32_t>(num / (2LL * (M - 1)));
    }
    *n_out = M;
    return ok();
}

int rf_project_latents(const void *latents, void *out, const double timesteps[3],
                       const uint8_t *keyframe_mask, int32_t B, int32_t C, int32_t T,
                       int32_t Hl, int32_t Wl, int32_t dtype, void *stream) {
    const char *fn = "rf_project_latents";
    if (!latents || !out || !timesteps || !keyframe_mask)
        return fail(RF_ERR_INVALID_ARG, "%s: NULL argument", fn);
    if (B <= 0 || C <= 0 || T <= 0 || Hl <= 0 || Wl <= 0)
        return fail(RF_ERR_INVALID_ARG, "%s: sizes must be positive (B=%d C=%d T=%d Hl=%d Wl=%d)",
                    fn, B, C, T, Hl, Wl);
    if (T > RF_MAX_FRAMES) return fail(RF_ERR_RANGE, "%s: T = %d exceeds %d", fn, T, RF_MAX_FRAMES);
    if (dtype != RF_F32 && dtype != RF_BF16)
        return fail(RF_ERR_UNSUPPORTED, "%s: unknown dtype %d", fn, dtype);
    if (static_cast<double>(B) * 2.0 * C * T * Hl * Wl * 4.0 > kMaxBytes)
        return fail(RF_ERR_RANGE, "%s: sizes overflow 64-bit byte counts", fn);
    const double t_start = timesteps[0], t_end = timesteps[1], tau = timesteps[2];
    if (!isfinite(t_start) || !isfinite(t_end) || !isfinite(tau))
        return fail(RF_ERR_INVALID_ARG, "%s: timesteps must be finite", fn);
    if (!aligned16(latents) || !aligned16(out))
        return fail(RF_ERR_UNSUPPORTED, "%s: pointers must be 16-byte aligned", fn);

    const int64_t elem = dtype == RF_F32 ? 4 : 2;
    const int64_t plane = static_cast<int64_t>(Hl) * Wl;
    const int64_t slot_bytes = static_cast<int64_t>(C) * T * plane * elem;
    const int64_t lat_bytes = static_cast<int64_t>(B) * 2 * slot_bytes;
    const int64_t out_bytes = static_cast<int64_t>(B) * slot_bytes;
    const char *slot1 = static_cast<const char *>(latents) + slot_bytes;
    int skip_keyframes = 0;
    if (B == 1 && out == slot1) {
        skip_keyframes = 1;  // out is slot 1 itself: keyframe planes already hold their state
    } else if (overlaps(latents, lat_bytes, out, out_bytes)) {
        return fail(RF_ERR_INVALID_ARG, "%s: out overlaps latents (only out == slot 1 with B == 1 is allowed)", fn);
    }

    rf::ProjParams p{};
    p.latents = latents;
    p.out = out;
    p.plane = plane;
    p.B = B;
    p.C = C;
    p.T = T;
    p.dtype = dtype;
    p.skip_keyframes = skip_keyframes;
    // Eq. (3): alpha = (t_start - tau) / (t_start - t_end), in double, kept in
    // [0, 1]; equal endpoints (both snapshots the same state) give 1.
    double alpha = 1.0;
    if (t_start != t_end) {
        alpha = (t_start - tau) / (t_start - t_end);
        alpha = alpha < 0.0 ? 0.0 : (alpha > 1.0 ? 1.0 : alpha);
    }
    p.alpha = static_cast<float>(alpha);
    for (int32_t f = 0; f < T; ++f) p.is_key[f] = keyframe_mask[f] ? 1 : 0;
    return launched(rf::launch_projection(p, static_cast<hipStream_t>(stream)), fn);
}

// Shared validation and launch of the two attention entry points.
// Bytes of split-tail workspace a bf16 attention of these sizes uses on a device
// of `cus` compute units (0 for fp32 or when nothing is split); the sizes must
// already be valid.
static int64_t attention_ws_need(int32_t M, int32_t n_kv, int32_t T, int64_t N, int32_t heads, int32_t head_dim,
                                 int32_t dtype, int32_t cus) {
    if (dtype != RF_BF16) return 0;
    return rf::attention_split(static_cast<int64_t>(M) * N, heads, head_dim, N, N * T, n_kv, cus).ws_bytes;
}

// The current device's geometry, as an rf_status.
static int query_geometry(rf::DeviceGeometry *geo, const char *fn) {
    const hipError_t e = rf::device_geometry(geo);
    if (e != hipSuccess)
        return fail(RF_ERR_HIP, "%s: cannot query the current device: %s", fn, hipGetErrorString(e));
    return RF_OK;
}

// The cache form of an attention call: the cached frames' projected states at
// t_skip replace their keys and values (already validated).
struct CacheForm {
    const rf_rolling_cache *cache;
    const void *store;
    double t_skip;
};

static double cache_alpha(const rf_rolling_cache &c, int32_t f, double t_skip);

// use_scratch: the split tail takes the library's static scratch (the
// allocation-free entry point) instead of a caller workspace.
static int attention_call(const void *q, const void *k, const void *v, void *out, const int32_t *q_ids,
                          int32_t M, const int32_t *kv_ids, int32_t Mkv, int32_t T, int32_t H, int32_t W,
                          int32_t heads, int32_t head_dim, int32_t dtype, void *ws, int64_t ws_bytes,
                          void *stream, const char *fn, bool use_scratch = false,
                          const CacheForm *cf = nullptr) {
    if (!q || !k || !v || !out) return fail(RF_ERR_INVALID_ARG, "%s: NULL tensor", fn);
    if (H <= 0 || W <= 0 || heads <= 0 || head_dim <= 0)
        return fail(RF_ERR_INVALID_ARG, "%s: sizes must be positive (H=%d W=%d heads=%d head_dim=%d)",
                    fn, H, W, heads, head_dim);
    if (static_cast<double>(H) * W * (T > 0 ? T : 1) * heads * head_dim * 4.0 > kMaxBytes)
        return fail(RF_ERR_RANGE, "%s: sizes overflow 64-bit byte counts (T=%d H=%d W=%d heads=%d head_dim=%d)",
                    fn, T, H, W, heads, head_dim);
    rf::AttnParams p{};
    int rc = check_id_list(q_ids, M, T, p.kf, fn);
    if (rc != RF_OK) return rc;
    int32_t kvf[RF_MAX_FRAMES];
    if (kv_ids) {
        rc = check_id_list(kv_ids, Mkv, T, kvf, fn);
        if (rc != RF_OK) return rc;
    }
    if (head_dim != 64 && head_dim != 128)
        return fail(RF_ERR_UNSUPPORTED, "%s: head_dim %d not in {64, 128}", fn, head_dim);
    if (dtype != RF_BF16 && dtype != RF_F32)
        return fail(RF_ERR_UNSUPPORTED, "%s: unknown dtype %d", fn, dtype);
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out))
        return fail(RF_ERR_UNSUPPORTED, "%s: pointers must be 16-byte aligned", fn);

    const int64_t N = static_cast<int64_t>(H) * W;
    const int64_t S = N * T;
    const int64_t row = static_cast<int64_t>(heads) * head_dim * (dtype == RF_F32 ? 4 : 2);
    const int64_t in_bytes = S * row;
    const int64_t out_bytes = N * M * row;
    if (overlaps(out, out_bytes, q, in_bytes) || overlaps(out, out_bytes, k, in_bytes) ||
        overlaps(out, out_bytes, v, in_bytes))
        return fail(RF_ERR_INVALID_ARG, "%s: out overlaps q, k or v", fn);
    const int32_t n_kv = (kv_ids && Mkv < T) ? Mkv : 0;
    if (cf) {
        const rf_rolling_cache &c = *cf->cache;
        const int64_t store_bytes = 2 * static_cast<int64_t>(c.n_cached) * c.frame_bytes;
        if (overlaps(out, out_bytes, cf->store, store_bytes))
            return fail(RF_ERR_INVALID_ARG, "%s: out overlaps the cache store", fn);
        p.cache_form = 1;
        p.store = cf->store;
        for (int32_t f = 0; f < T; ++f) {
            p.cslot[f] = -1;
            p.calpha[f] = 0.0f;
            if (c.after_slot[f] >= 0) {
                p.cslot[f] = static_cast<int32_t>(c.before_slot[f]) | (static_cast<int32_t>(c.after_slot[f]) << 16);
                p.calpha[f] = static_cast<float>(cache_alpha(c, f, cf->t_skip));
            }
        }
    }
    if (ws) {
        if (ws_bytes < 0) return fail(RF_ERR_INVALID_ARG, "%s: workspace_bytes < 0", fn);
        if (!aligned16(ws)) return fail(RF_ERR_UNSUPPORTED, "%s: workspace must be 16-byte aligned", fn);
        if (ws_bytes > 0 && (overlaps(ws, ws_bytes, q, in_bytes) || overlaps(ws, ws_bytes, k, in_bytes) ||
                             overlaps(ws, ws_bytes, v, in_bytes) || overlaps(ws, ws_bytes, out, out_bytes)))
            return fail(RF_ERR_INVALID_ARG, "%s: workspace overlaps q, k, v or out", fn);
    }
    // every argument is valid: the split plan and tile order follow the device
    rc = query_geometry(&p.geo, fn);
    if (rc != RF_OK) return rc;
    p.split_keys = use_scratch || ws != nullptr;
    if (use_scratch) {
        const int64_t need = attention_ws_need(M, n_kv, T, N, heads, head_dim, dtype, p.geo.cus);
        if (need > rf::kAttentionScratchBytes)
            return fail(RF_ERR_RANGE,
                        "%s: the split-key tail needs %lld bytes of scratch on %d compute units, the static "
                        "scratch holds %lld (rf_keyframe_attention_ws takes a workspace of any size)",
                        fn, static_cast<long long>(need), p.geo.cus,
                        static_cast<long long>(rf::kAttentionScratchBytes));
        if (need > 0) {
            const hipError_t e = rf::attention_scratch(&p.ws);
            if (e != hipSuccess)
                return fail(RF_ERR_HIP, "%s: cannot look up the static scratch: %s", fn, hipGetErrorString(e));
            p.ws_bytes = rf::kAttentionScratchBytes;
        }
    } else if (ws) {
        const int64_t need = attention_ws_need(M, n_kv, T, N, heads, head_dim, dtype, p.geo.cus);
        if (ws_bytes < need)
            return fail(RF_ERR_INVALID_ARG, "%s: workspace of %lld bytes, %lld needed on %d compute units", fn,
                        static_cast<long long>(ws_bytes), static_cast<long long>(need), p.geo.cus);
        p.ws = need > 0 ? ws : nullptr;
        p.ws_bytes = ws_bytes;
    }

    p.q = q;
    p.k = k;
    p.v = v;
    p.out = out;
    p.S = S;
    p.N = N;
    p.M = M;
    p.heads = heads;
    p.head_dim = head_dim;
    p.dtype = dtype;
    // every frame listed: the unmasked kernel
    p.n_kv = n_kv;
    for (int32_t i = 0; i < p.n_kv; ++i) p.kvf[i] = kvf[i];
    return launched(rf::launch_attention(p, static_cast<hipStream_t>(stream)), fn);
}

int rf_keyframe_attention(const void *q, const void *k, const void *v, void *out,
                          const int32_t *keyframe_ids, int32_t M, int32_t T, int32_t H,
                          int32_t W, int32_t heads, int32_t head_dim, int32_t dtype,
                          void *stream) {
    return attention_call(q, k, v, out, keyframe_ids, M, nullptr, 0, T, H, W, heads, head_dim, dtype,
                          nullptr, 0, stream, "rf_keyframe_attention");
}

int rf_keyframe_attention_ws(const void *q, const void *k, const void *v, void *out,
                             const int32_t *keyframe_ids, int32_t M, int32_t T, int32_t H, int32_t W,
                             int32_t heads, int32_t head_dim, int32_t dtype, void *workspace,
                             int64_t workspace_bytes, void *stream) {
    const char *fn = "rf_keyframe_attention_ws";
    if (!workspace) return fail(RF_ERR_INVALID_ARG, "%s: NULL workspace", fn);
    return attention_call(q, k, v, out, keyframe_ids, M, nullptr, 0, T, H, W, heads, head_dim, dtype,
                          workspace, workspace_bytes, stream, fn);
}

int rf_keyframe_attention_noalloc(const void *q, const void *k, const void *v, void *out,
                                  const int32_t *keyframe_ids, int32_t M, int32_t T, int32_t H, int32_t W,
                                  int32_t heads, int32_t head_dim, int32_t dtype, void *stream) {
    return attention_call(q, k, v, out, keyframe_ids, M, nullptr, 0, T, H, W, heads, head_dim, dtype, nullptr, 0,
                          stream, "rf_keyframe_attention_noalloc", true);
}

int rf_frame_attention(const void *q, const void *k, const void *v, void *out,
                       const int32_t *q_frames, int32_t Mq, const int32_t *kv_frames, int32_t Mkv,
                       int32_t T, int32_t H, int32_t W, int32_t heads, int32_t head_dim,
                       int32_t dtype, void *workspace, int64_t workspace_bytes, void *stream) {
    const char *fn = "rf_frame_attention";
    if (!kv_frames) return fail(RF_ERR_INVALID_ARG, "%s: kv_frames is NULL", fn);
    return attention_call(q, k, v, out, q_frames, Mq, kv_frames, Mkv, T, H, W, heads, head_dim, dtype,
                          workspace, workspace_bytes, stream, fn);
}

// Sizes of an attention plan query, and the compute units it is planned for
// (0: the current device's, which needs a device query).
static int plan_args(int32_t M, int32_t Mkv, int32_t T, int32_t H, int32_t W, int32_t heads, int32_t head_dim,
                     int32_t dtype, int32_t compute_units, int32_t *cus, const char *fn) {
    if (H <= 0 || W <= 0 || heads <= 0 || T <= 0 || M <= 0 || Mkv <= 0)
        return fail(RF_ERR_INVALID_ARG, "%s: sizes must be positive", fn);
    if (T > RF_MAX_FRAMES) return fail(RF_ERR_RANGE, "%s: T = %d exceeds %d", fn, T, RF_MAX_FRAMES);
    if (M > T || Mkv > T) return fail(RF_ERR_RANGE, "%s: M = %d or Mkv = %d exceeds T = %d", fn, M, Mkv, T);
    if (head_dim != 64 && head_dim != 128)
        return fail(RF_ERR_UNSUPPORTED, "%s: head_dim %d not in {64, 128}", fn, head_dim);
    if (dtype != RF_BF16 && dtype != RF_F32) return fail(RF_ERR_UNSUPPORTED, "%s: unknown dtype %d", fn, dtype);
    if (static_cast<double>(H) * W * T * heads * head_dim * 4.0 > kMaxBytes)
        return fail(RF_ERR_RANGE, "%s: sizes overflow 64-bit byte counts", fn);
    if (compute_units < 0 || compute_units > RF_MAX_COMPUTE_UNITS)
        return fail(RF_ERR_RANGE, "%s: compute_units = %d outside 0..%d", fn, compute_units, RF_MAX_COMPUTE_UNITS);
    if (compute_units > 0) {
        *cus = compute_units;
        return RF_OK;
    }
    rf::DeviceGeometry geo;
    const int rc = query_geometry(&geo, fn);
    if (rc != RF_OK) return rc;
    *cus = geo.cus;
    return RF_OK;
}

int rf_attention_workspace(int32_t M, int32_t Mkv, int32_t T, int32_t H, int32_t W, int32_t heads,
                           int32_t head_dim, int32_t dtype, int32_t compute_units, int64_t *bytes_out) {
    const char *fn = "rf_attention_workspace";
    if (!bytes_out) return fail(RF_ERR_INVALID_ARG, "%s: NULL output", fn);
    int32_t cus = 0;
    const int rc = plan_args(M, Mkv, T, H, W, heads, head_dim, dtype, compute_units, &cus, fn);
    if (rc != RF_OK) return rc;
    *bytes_out = attention_ws_need(M, Mkv < T ? Mkv : 0, T, static_cast<int64_t>(H) * W, heads, head_dim, dtype,
                                   cus);
    return ok();
}

int rf_attention_plan(int32_t M, int32_t Mkv, int32_t T, int32_t H, int32_t W, int32_t heads, int32_t head_dim,
                      int32_t dtype, int32_t compute_units, rf_attention_split *plan_out) {
    const char *fn = "rf_attention_plan";
    if (!plan_out) return fail(RF_ERR_INVALID_ARG, "%s: NULL output", fn);
    int32_t cus = 0;
    const int rc = plan_args(M, Mkv, T, H, W, heads, head_dim, dtype, compute_units, &cus, fn);
    if (rc != RF_OK) return rc;
    const int64_t N = static_cast<int64_t>(H) * W;
    rf_attention_split out;
    memset(&out, 0, sizeof out);
    out.compute_units = cus;
    rf::AttnSplit sp{};
    if (dtype == RF_BF16) {
        sp = rf::attention_split(static_cast<int64_t>(M) * N, heads, head_dim, N, N * T, Mkv < T ? Mkv : 0, cus);
        out.tiles = sp.n_tiles;
        out.whole_tiles = sp.n_direct;
        out.tail_tiles = sp.n_tail;
        out.parts = static_cast<int32_t>(sp.split);
        out.key_tiles_per_part = static_cast<int32_t>(sp.kv_per_split);
        out.workspace_bytes = sp.ws_bytes;
    }
    rf::AttnParams p{};
    p.S = N * T;
    p.N = N;
    p.M = M;
    p.heads = heads;
    p.head_dim = head_dim;
    p.dtype = dtype;
    p.n_kv = Mkv < T ? Mkv : 0;
    for (int32_t i = 0; i < p.n_kv; ++i) p.kvf[i] = i;
    p.geo.cus = cus;
    out.shared_keys = rf::attention_shares_keys(p, sp) ? 1 : 0;
    *plan_out = out;
    return ok();
}

static int frame_copy(const void *src, void *dst, const int32_t *frame_ids, int32_t M, int32_t T,
                      int64_t rows_per_frame, int64_t row_bytes, void *stream, int scatter,
                      const char *fn) {
    if (!src || !dst) return fail(RF_ERR_INVALID_ARG, "%s: NULL buffer", fn);
    if (rows_per_frame <= 0 || row_bytes <= 0)
        return fail(RF_ERR_INVALID_ARG, "%s: rows_per_frame and row_bytes must be positive", fn);
    if (static_cast<double>(rows_per_frame) * static_cast<double>(row_bytes) * RF_MAX_FRAMES > kMaxBytes)
        return fail(RF_ERR_RANGE, "%s: rows_per_frame x row_bytes overflows 64-bit byte counts", fn);
    rf::FrameCopyParams p{};
    int32_t ids[RF_MAX_FRAMES];
    const int rc = check_id_list(frame_ids, M, T, ids, fn);
    if (rc != RF_OK) return rc;
    if (row_bytes % 16 != 0)
        return fail(RF_ERR_UNSUPPORTED, "%s: row_bytes %lld not a multiple of 16", fn,
                    static_cast<long long>(row_bytes));
    if (!aligned16(src) || !aligned16(dst))
        return fail(RF_ERR_UNSUPPORTED, "%s: pointers must be 16-byte aligned", fn);
    const int64_t frame_bytes = rows_per_frame * row_bytes;
    const int64_t full = frame_bytes * T, compact = frame_bytes * M;
    if (overlaps(src, scatter ? compact : full, dst, scatter ? full : compact))
        return fail(RF_ERR_INVALID_ARG, "%s: source and destination overlap", fn);
    p.src = src;
    p.dst = dst;
    p.frame_bytes = frame_bytes;
    p.M = M;
    for (int32_t m = 0; m < M; ++m) {
        p.src_idx[m] = scatter ? m : ids[m];
        p.dst_idx[m] = scatter ? ids[m] : m;
    }
    return launched(rf::launch_frame_copy(p, static_cast<hipStream_t>(stream)), fn);
}

int rf_gather_frames(const void *src_full, void *dst_compact, const int32_t *frame_ids, int32_t M,
                     int32_t T, int64_t rows_per_frame, int64_t row_bytes, void *stream) {
    return frame_copy(src_full, dst_compact, frame_ids, M, T, rows_per_frame, row_bytes, stream, 0,
                      "rf_gather_frames");
}

int rf_scatter_frames(const void *src_compact, void *dst_full, const int32_t *frame_ids, int32_t M,
                      int32_t T, int64_t rows_per_frame, int64_t row_bytes, void *stream) {
    return frame_copy(src_compact, dst_full, frame_ids, M, T, rows_per_frame, row_bytes, stream, 1,
                      "rf_scatter_frames");
}

int rf_frame_similarity_workspace(int32_t B, int32_t C, int32_t T, int32_t H, int32_t W,
                                  int64_t *bytes_out) {
    const char *fn = "rf_frame_similarity_workspace";
    if (!bytes_out) return fail(RF_ERR_INVALID_ARG, "%s: NULL output", fn);
    if (B <= 0 || C <= 0 || T <= 0 || H <= 0 || W <= 0)
        return fail(RF_ERR_INVALID_ARG, "%s: sizes must be positive (B=%d C=%d T=%d H=%d W=%d)",
                    fn, B, C, T, H, W);
    if (T > RF_MAX_FRAMES) return fail(RF_ERR_RANGE, "%s: T = %d exceeds %d", fn, T, RF_MAX_FRAMES);
    const rf::SimGeometry g = rf::similarity_geometry(B, C, T, static_cast<int64_t>(H) * W);
    if (static_cast<double>(B) * static_cast<double>(g.n_runs) * g.NBP * 128.0 > kMaxBytes ||
        static_cast<double>(C) * H * W * T * B > kMaxBytes)
        return fail(RF_ERR_RANGE, "%s: workspace size overflows", fn);
    *bytes_out = g.workspace_bytes;
    return ok();
}

int rf_frame_similarity(const void *latents, double *sim_out, void *workspace,
                        int64_t workspace_bytes, int32_t B, int32_t C, int32_t T, int32_t H,
                        int32_t W, int32_t dtype, void *stream) {
    const char *fn = "rf_frame_similarity";
    if (!latents || !sim_out || !workspace) return fail(RF_ERR_INVALID_ARG, "%s: NULL argument", fn);
    int64_t need = 0;
    const int rc = rf_frame_similarity_workspace(B, C, T, H, W, &need);
    if (rc != RF_OK) return rc;
    if (dtype != RF_F32 && dtype != RF_BF16)
        return fail(RF_ERR_UNSUPPORTED, "%s: unknown dtype %d", fn, dtype);
    if (!aligned16(latents) || !aligned16(workspace) || (reinterpret_cast<uintptr_t>(sim_out) & 7u))
        return fail(RF_ERR_UNSUPPORTED, "%s: latents/workspace must be 16-byte and sim_out 8-byte aligned", fn);
    if (workspace_bytes < need)
        return fail(RF_ERR_INVALID_ARG, "%s: workspace of %lld bytes, %lld needed", fn,
                    static_cast<long long>(workspace_bytes), static_cast<long long>(need));
    const int64_t plane = static_cast<int64_t>(H) * W;
    const int64_t lat_bytes = static_cast<int64_t>(B) * C * T * plane * (dtype == RF_F32 ? 4 : 2);
    const int64_t sim_bytes = static_cast<int64_t>(B) * T * T * 8;
    if (overlaps(sim_out, sim_bytes, latents, lat_bytes) || overlaps(sim_out, sim_bytes, workspace, need) ||
        overlaps(workspace, need, latents, lat_bytes))
        return fail(RF_ERR_INVALID_ARG, "%s: latents, sim_out and workspace must not overlap", fn);
    rf::SimParams p{};
    p.latents = latents;
    p.sim = sim_out;
    p.workspace = static_cast<double *>(workspace);
    p.plane = plane;
    p.B = B;
    p.C = C;
    p.T = T;
    p.dtype = dtype;
    return launched(rf::launch_similarity(p, static_cast<hipStream_t>(stream)), fn);
}

int rf_select_keyframes_adaptive(const double *sim, int32_t T, double tau, int32_t M, double dtau,
                                 double delta_up, double delta_down, uint32_t flags,
                                 int32_t *keyframe_ids_out, int32_t *num_keyframes_out,
                                 uint8_t *keyframe_mask_out) {
    const char *fn = "rf_select_keyframes_adaptive";
    if (!sim || !keyframe_ids_out || !num_keyframes_out)
        return fail(RF_ERR_INVALID_ARG, "%s: NULL argument", fn);
    if (T <= 0 || T > RF_MAX_FRAMES) return fail(RF_ERR_RANGE, "%s: T = %d outside 1..%d", fn, T, RF_MAX_FRAMES);
    if (M <= 0 || M > T) return fail(RF_ERR_RANGE, "%s: M = %d outside 1..%d", fn, M, T);
    if (!isfinite(tau) || !isfinite(dtau) || !isfinite(delta_up) || !isfinite(delta_down))
        return fail(RF_ERR_INVALID_ARG, "%s: tau, dtau, delta_up and delta_down must be finite", fn);
    if (flags & ~RF_SEL_INTENT_SIGN) return fail(RF_ERR_INVALID_ARG, "%s: unknown flags 0x%x", fn, flags);
    const bool intent = (flags & RF_SEL_INTENT_SIGN) != 0;
    // Alg. 1: the first frame seeds the set; expected interval L_avg = T / M.
    const double l_avg = static_cast<double>(T) / static_cast<double>(M);
    int32_t n = 0, last = 0;
    keyframe_ids_out[n++] = 0;
    for (int32_t i = 1; i < T && n < M; ++i) {
        // Eq. (1): compare with the most recent keyframe, strictly below the threshold
        if (sim[static_cast<int64_t>(i) * T + last] < tau) {
            const double gap = static_cast<double>(i - last);
            if (gap >= l_avg + delta_up)
                tau = intent ? tau + dtau : tau - dtau;
            else if (gap <= l_avg - delta_down)
                tau = intent ? tau - dtau : tau + dtau;
            keyframe_ids_out[n++] = i;
            last = i;
        }
    }
    *num_keyframes_out = n;
    if (keyframe_mask_out) {
        for (int32_t f = 0; f < T; ++f) keyframe_mask_out[f] = 0;
        for (int32_t m = 0; m < n; ++m) keyframe_mask_out[keyframe_ids_out[m]] = 1;
    }
    return ok();
}

// ---------------------------------------------------------------------------
// Rolling cache (App. B.2)
// ---------------------------------------------------------------------------

static const uint32_t kCacheMagic = 0x52464331u;
static const double kHiddenEps = 1e-8;

static int64_t elem_bytes(int32_t dtype) { return dtype == RF_F32 ? 4 : 2; }

static int cache_store_bytes(int32_t n_cached, int64_t rows_per_frame, int32_t hidden, int32_t dtype,
                             int64_t *bytes_out, const char *fn) {
    if (n_cached <= 0 || rows_per_frame <= 0 || hidden <= 0)
        return fail(RF_ERR_INVALID_ARG, "%s: sizes must be positive", fn);
    if (n_cached > RF_MAX_FRAMES)
        return fail(RF_ERR_RANGE, "%s: n_cached = %d exceeds %d", fn, n_cached, RF_MAX_FRAMES);
    if (dtype != RF_F32 && dtype != RF_BF16) return fail(RF_ERR_UNSUPPORTED, "%s: unknown dtype %d", fn, dtype);
    if (static_cast<double>(rows_per_frame) * hidden * elem_bytes(dtype) * 2.0 * n_cached * RF_MAX_FRAMES > kMaxBytes)
        return fail(RF_ERR_RANGE, "%s: size overflows", fn);
    *bytes_out = 2 * static_cast<int64_t>(n_cached) * rows_per_frame * hidden * elem_bytes(dtype);
    return RF_OK;
}

int rf_cache_store_bytes(int32_t n_cached, int64_t rows_per_frame, int32_t hidden, int32_t dtype,
                         int64_t *bytes_out) {
    const char *fn = "rf_cache_store_bytes";
    if (!bytes_out) return fail(RF_ERR_INVALID_ARG, "%s: NULL output", fn);
    const int rc = cache_store_bytes(n_cached, rows_per_frame, hidden, dtype, bytes_out, fn);
    return rc == RF_OK ? ok() : rc;
}

// An initialised cache struct whose sizes and slot indices are consistent.
static int check_cache(const rf_rolling_cache *c, const char *fn) {
    if (!c) return fail(RF_ERR_INVALID_ARG, "%s: NULL cache", fn);
    if (c->magic != kCacheMagic) return fail(RF_ERR_INVALID_ARG, "%s: cache not initialised by rf_cache_init", fn);
    if (c->T <= 0 || c->T > RF_MAX_FRAMES || c->n_cached <= 0 || c->n_cached > c->T ||
        c->rows_per_frame <= 0 || c->hidden <= 0 || (c->dtype != RF_F32 && c->dtype != RF_BF16) ||
        static_cast<double>(c->rows_per_frame) * c->hidden * 4.0 * 2.0 * RF_MAX_FRAMES > kMaxBytes ||
        c->frame_bytes != c->rows_per_frame * c->hidden * elem_bytes(c->dtype))
        return fail(RF_ERR_INVALID_ARG, "%s: cache struct is inconsistent", fn);
    for (int32_t f = 0; f < c->T; ++f) {
        const int b = c->before_slot[f], a = c->after_slot[f];
        if (b < 0 && a < 0) continue;
        if (b < 0 || a < 0 || b >= 2 * c->n_cached || a >= 2 * c->n_cached || (b >> 1) != (a >> 1))
            return fail(RF_ERR_INVALID_ARG, "%s: cache struct has bad slots for frame %d", fn, f);
        if (!isfinite(c->t_before[f]) || !isfinite(c->t_after[f]) || !(c->t_after[f] <= c->t_before[f]))
            return fail(RF_ERR_INVALID_ARG, "%s: cache struct has bad timesteps for frame %d", fn, f);
    }
    return RF_OK;
}

// The listed frames (NULL: every cached frame), strictly increasing and cached.
static int cache_frames(const rf_rolling_cache *c, const int32_t *frames, int32_t n, int32_t *out,
                        int32_t *n_out, const char *fn) {
    if (!frames) {
        int32_t k = 0;
        for (int32_t f = 0; f < c->T; ++f)
            if (c->after_slot[f] >= 0) out[k++] = f;
        *n_out = k;
        return RF_OK;
    }
    if (n <= 0 || n > c->T) return fail(RF_ERR_INVALID_ARG, "%s: n = %d outside 1..%d", fn, n, c->T);
    for (int32_t i = 0; i < n; ++i) {
        if (frames[i] < 0 || frames[i] >= c->T)
            return fail(RF_ERR_RANGE, "%s: frame %d outside [0, %d)", fn, frames[i], c->T);
        if (i > 0 && frames[i] <= frames[i - 1])
            return fail(RF_ERR_INVALID_ARG, "%s: frames not strictly increasing at position %d", fn, i);
        if (c->after_slot[frames[i]] < 0) return fail(RF_ERR_INVALID_ARG, "%s: frame %d is not cached", fn, frames[i]);
        out[i] = frames[i];
    }
    *n_out = n;
    return RF_OK;
}

// Copies the rows of each listed frame of h_full into its after slot.
static int store_after(const rf_rolling_cache &c, void *store, const void *h_full, const int32_t *fr,
                       int32_t n, void *stream, const char *fn) {
    if (!store) return fail(RF_ERR_INVALID_ARG, "%s: NULL store", fn);
    if (!aligned16(store) || !aligned16(h_full))
        return fail(RF_ERR_UNSUPPORTED, "%s: store and h_full must be 16-byte aligned", fn);
    const int64_t store_bytes = 2 * static_cast<int64_t>(c.n_cached) * c.frame_bytes;
    if (overlaps(store, store_bytes, h_full, c.frame_bytes * c.T))
        return fail(RF_ERR_INVALID_ARG, "%s: store overlaps h_full", fn);
    rf::FrameCopyParams p{};
    p.src = h_full;
    p.dst = store;
    p.frame_bytes = c.frame_bytes;
    p.M = n;
    for (int32_t i = 0; i < n; ++i) {
        p.src_idx[i] = fr[i];
        p.dst_idx[i] = c.after_slot[fr[i]];
    }
    return launched(rf::launch_frame_copy(p, static_cast<hipStream_t>(stream)), fn);
}

int rf_cache_init(rf_rolling_cache *cache, void *store, const void *h_full, const int32_t *frames,
                  int32_t n, int32_t T, int64_t rows_per_frame, int32_t hidden, int32_t dtype,
                  double t_w, void *stream) {
    const char *fn = "rf_cache_init";
    if (!cache) return fail(RF_ERR_INVALID_ARG, "%s: NULL cache", fn);
    int32_t ids[RF_MAX_FRAMES];
    int rc = check_id_list(frames, n, T, ids, fn);
    if (rc != RF_OK) return rc;
    int64_t need = 0;
    rc = cache_store_bytes(n, rows_per_frame, hidden, dtype, &need, fn);
    if (rc != RF_OK) return rc;
    if ((static_cast<int64_t>(hidden) * elem_bytes(dtype)) % 16 != 0)
        return fail(RF_ERR_UNSUPPORTED, "%s: a row of %d elements is not a multiple of 16 bytes", fn, hidden);
    if (!isfinite(t_w)) return fail(RF_ERR_INVALID_ARG, "%s: t_w must be finite", fn);
    if (h_full && !store) return fail(RF_ERR_INVALID_ARG, "%s: NULL store", fn);

    rf_rolling_cache c;
    memset(&c, 0, sizeof c);
    c.T = T;
    c.n_cached = n;
    c.rows_per_frame = rows_per_frame;
    c.hidden = hidden;
    c.dtype = dtype;
    c.frame_bytes = rows_per_frame * hidden * elem_bytes(dtype);
    c.magic = kCacheMagic;
    for (int32_t f = 0; f < RF_MAX_FRAMES; ++f) {
        c.before_slot[f] = c.after_slot[f] = -1;
        c.t_before[f] = c.t_after[f] = 0.0;
    }
    // h_before = h_after = the state at t_w: both indices name slot 2i
    for (int32_t i = 0; i < n; ++i) {
        c.before_slot[ids[i]] = c.after_slot[ids[i]] = static_cast<int16_t>(2 * i);
        c.t_before[ids[i]] = c.t_after[ids[i]] = t_w;
    }
    if (h_full) {
        rc = store_after(c, store, h_full, ids, n, stream, fn);
        if (rc != RF_OK) return rc;
    }
    *cache = c;
    return ok();
}

int rf_cache_shift_store(rf_rolling_cache *cache, void *store, const void *h_full, const int32_t *frames,
                         int32_t n, double t_denoise, void *stream) {
    const char *fn = "rf_cache_shift_store";
    int rc = check_cache(cache, fn);
    if (rc != RF_OK) return rc;
    int32_t fr[RF_MAX_FRAMES], k = 0;
    rc = cache_frames(cache, frames, n, fr, &k, fn);
    if (rc != RF_OK) return rc;
    if (!isfinite(t_denoise)) return fail(RF_ERR_INVALID_ARG, "%s: t_denoise must be finite", fn);
    for (int32_t i = 0; i < k; ++i)
        if (!(t_denoise < cache->t_after[fr[i]]))
            return fail(RF_ERR_INVALID_ARG, "%s: t_denoise %g is not below t_after %g of frame %d", fn,
                        t_denoise, cache->t_after[fr[i]], fr[i]);
    rf_rolling_cache c = *cache;
    for (int32_t i = 0; i < k; ++i) {
        const int32_t f = fr[i];
        // h_before <- h_after, t_before <- t_after; h_after goes to the other slot of the pair
        c.before_slot[f] = c.after_slot[f];
        c.t_before[f] = c.t_after[f];
        c.after_slot[f] = static_cast<int16_t>(c.before_slot[f] ^ 1);
        c.t_after[f] = t_denoise;
    }
    if (h_full) {
        rc = store_after(c, store, h_full, fr, k, stream, fn);
        if (rc != RF_OK) return rc;
    }
    *cache = c;
    return ok();
}

// App. B.2's weight with its epsilon, clamped to [0, 1].
static double cache_alpha(const rf_rolling_cache &c, int32_t f, double t_skip) {
    const double a = (c.t_before[f] - t_skip) / (c.t_before[f] - c.t_after[f] + kHiddenEps);
    return a < 0.0 ? 0.0 : (a > 1.0 ? 1.0 : a);
}

int rf_cache_alpha(const rf_rolling_cache *cache, int32_t frame, double t_skip, double *alpha_out) {
    const char *fn = "rf_cache_alpha";
    int rc = check_cache(cache, fn);
    if (rc != RF_OK) return rc;
    if (!alpha_out) return fail(RF_ERR_INVALID_ARG, "%s: NULL output", fn);
    if (frame < 0 || frame >= cache->T) return fail(RF_ERR_RANGE, "%s: frame %d outside [0, %d)", fn, frame, cache->T);
    if (cache->after_slot[frame] < 0) return fail(RF_ERR_INVALID_ARG, "%s: frame %d is not cached", fn, frame);
    if (!isfinite(t_skip)) return fail(RF_ERR_INVALID_ARG, "%s: t_skip must be finite", fn);
    *alpha_out = cache_alpha(*cache, frame, t_skip);
    return ok();
}

int rf_cache_project_kv(const rf_rolling_cache *cache, const void *store, void *k, void *v,
                        const int32_t *frames, int32_t n, double t_skip, void *stream) {
    const char *fn = "rf_cache_project_kv";
    int rc = check_cache(cache, fn);
    if (rc != RF_OK) return rc;
    if (!store || !k || !v) return fail(RF_ERR_INVALID_ARG, "%s: NULL buffer", fn);
    int32_t fr[RF_MAX_FRAMES], cnt = 0;
    rc = cache_frames(cache, frames, n, fr, &cnt, fn);
    if (rc != RF_OK) return rc;
    if (!isfinite(t_skip)) return fail(RF_ERR_INVALID_ARG, "%s: t_skip must be finite", fn);
    if (!aligned16(store) || !aligned16(k) || !aligned16(v))
        return fail(RF_ERR_UNSUPPORTED, "%s: pointers must be 16-byte aligned", fn);
    const int64_t store_bytes = 2 * static_cast<int64_t>(cache->n_cached) * cache->frame_bytes;
    const int64_t kv_bytes = cache->frame_bytes * cache->T;
    if (overlaps(k, kv_bytes, v, kv_bytes) || overlaps(k, kv_bytes, store, store_bytes) ||
        overlaps(v, kv_bytes, store, store_bytes))
        return fail(RF_ERR_INVALID_ARG, "%s: k, v and store must not overlap", fn);
    rf::CacheProjParams p{};
    p.store = store;
    p.k = k;
    p.v = v;
    p.frame_bytes = cache->frame_bytes;
    p.n = cnt;
    p.dtype = cache->dtype;
    for (int32_t i = 0; i < cnt; ++i) {
        const int32_t f = fr[i];
        p.before[i] = cache->before_slot[f];
        p.after[i] = cache->after_slot[f];
        p.dst[i] = static_cast<uint8_t>(f);
        p.alpha[i] = static_cast<float>(cache_alpha(*cache, f, t_skip));
    }
    return launched(rf::launch_cache_projection(p, static_cast<hipStream_t>(stream)), fn);
}

int rf_keyframe_attention_cached(const void *q, const void *k, const void *v, void *out,
                                 const int32_t *keyframe_ids, int32_t M, int32_t T, int32_t H, int32_t W,
                                 int32_t heads, int32_t head_dim, int32_t dtype, const rf_rolling_cache *cache,
                                 const void *store, double t_skip, void *workspace, int64_t workspace_bytes,
                                 void *stream) {
    const char *fn = "rf_keyframe_attention_cached";
    int rc = check_cache(cache, fn);
    if (rc != RF_OK) return rc;
    if (!store) return fail(RF_ERR_INVALID_ARG, "%s: NULL store", fn);
    if (!aligned16(store)) return fail(RF_ERR_UNSUPPORTED, "%s: store must be 16-byte aligned", fn);
    if (!isfinite(t_skip)) return fail(RF_ERR_INVALID_ARG, "%s: t_skip must be finite", fn);
    if (dtype != RF_BF16)
        return fail(RF_ERR_UNSUPPORTED, "%s: the projected keys and values are formed in bf16 attention only", fn);
    if (cache->T != T || H <= 0 || W <= 0 || cache->rows_per_frame != static_cast<int64_t>(H) * W ||
        heads <= 0 || head_dim <= 0 || cache->hidden != static_cast<int64_t>(heads) * head_dim ||
        cache->dtype != dtype)
        return fail(RF_ERR_INVALID_ARG,
                    "%s: the cache (T=%d, %lld rows of %d, dtype %d) does not match the attention "
                    "(T=%d, %d x %d rows of %d x %d, dtype %d)", fn, cache->T,
                    static_cast<long long>(cache->rows_per_frame), cache->hidden, cache->dtype, T, H, W, heads,
                    head_dim, dtype);
    if (!workspace) return fail(RF_ERR_INVALID_ARG, "%s: NULL workspace", fn);
    const CacheForm cf{cache, store, t_skip};
    return attention_call(q, k, v, out, keyframe_ids, M, nullptr, 0, T, H, W, heads, head_dim, dtype, workspace,
                          workspace_bytes, stream, fn, false, &cf);
}

// ---------------------------------------------------------------------------
// Progressive asynchronous schedule (Eq. 2, Alg. 2)
// ---------------------------------------------------------------------------

int rf_async_schedule(int32_t T, int32_t T_w, int32_t T_mid, int32_t n_small, int32_t n_large,
                      rf_step_plan *plan_out, int32_t *n_rhythmic_out, int32_t *n_skipped_out) {
    const char *fn = "rf_async_schedule";
    if (!plan_out) return fail(RF_ERR_INVALID_ARG, "%s: NULL plan", fn);
    if (T < 1 || T > (1 << 20)) return fail(RF_ERR_RANGE, "%s: T = %d outside 1..%d", fn, T, 1 << 20);
    if (T_w < 0 || T_w > T) return fail(RF_ERR_RANGE, "%s: T_w = %d outside 0..T", fn, T_w);
    if (T_mid < 0 || T_mid > T) return fail(RF_ERR_RANGE, "%s: T_mid = %d outside 0..T", fn, T_mid);
    if (n_small < 1 || n_large < 1)
        return fail(RF_ERR_INVALID_ARG, "%s: strides must be >= 1 (n_small=%d n_large=%d)", fn, n_small, n_large);
    int32_t state = T;   // the non-keyframes' state time
    int32_t left = -1;   // the time of their last update
    int32_t n_rp = 0, n_sk = 0;
    for (int32_t t = T, i = 0; t >= 1; --t, ++i) {
        rf_step_plan p;
        p.t = t;
        p.nonkey_to = p.t_start = p.t_end = -1;
        p.alpha = 0.0;
        if (t > T - T_w) {  // synchronous warm-up
            p.phase = RF_STEP_WARMUP;
            p.n_skip = 1;
            p.nonkey_to = state = t - 1;
        } else {
            p.n_skip = t > T_mid ? n_small : n_large;   // Eq. (2)
            if (state == t) {  // the non-keyframes are at t: a Rhythmic Point
                p.phase = RF_STEP_RHYTHMIC;
                p.nonkey_to = t - p.n_skip > 0 ? t - p.n_skip : 0;
                left = t;
                state = p.nonkey_to;
                ++n_rp;
            } else {           // skipped: project on the interval [state, left]
                p.phase = RF_STEP_SKIP;
                p.t_start = left;
                p.t_end = state;
                p.alpha = static_cast<double>(left - t) / static_cast<double>(left - state);
                ++n_sk;
            }
        }
        plan_out[i] = p;
    }
    if (n_rhythmic_out) *n_rhythmic_out = n_rp;
    if (n_skipped_out) *n_skipped_out = n_sk;
    return ok();
}

// --- a block's operators around the attention ---

static_assert(RF_MAX_FRAMES <= 256, "a frame index is a byte");
static void row_frames(const int32_t *ids, int32_t M, bool in_full, bool out_full, rf::RowFrames *f) {
    for (int32_t m = 0; m < M; ++m) f->frame[m] = static_cast<uint8_t>(ids[m]);
    f->in_full = in_full;
    f->out_full = out_full;
}

static int64_t abs_diff(uintptr_t a, uintptr_t b) { return static_cast<int64_t>(a > b ? a - b : b - a); }

// Two sets of rows of a_row and b_row bytes, `stride` bytes apart each, share memory.
// With one stride for both, rows may interleave (views of one buffer).
static bool rows_overlap(const void *a, int64_t a_rows, int64_t a_stride, int64_t a_row, const void *b,
                         int64_t b_rows, int64_t b_stride, int64_t b_row) {
    if (!overlaps(a, (a_rows - 1) * a_stride + a_row, b, (b_rows - 1) * b_stride + b_row)) return false;
    if (a_stride != b_stride) return true;
    const uintptr_t pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b);
    const int64_t off = abs_diff(pa, pb) % a_stride;   // of the later set's rows after the earlier one's
    const int64_t first = pa <= pb ? a_row : b_row, second = pa <= pb ? b_row : a_row;
    return off < first || off + second > a_stride;
}

static int rotary_call(const void *q, void *q_out, const void *k, void *k_out, const int32_t *frame_ids, int32_t M,
                       int32_t T, int32_t H, int32_t W, int32_t q_heads, int32_t k_heads, int32_t head_dim,
                       const rf_rotary_axes *axes, const int64_t (&strides)[4], uint32_t flags, int32_t dtype,
                       void *stream, const char *fn) {
    if (!q || !q_out || !axes || (k && !k_out)) return fail(RF_ERR_INVALID_ARG, "%s: NULL argument", fn);
    const uint32_t known = RF_ROWS_IN_FULL | RF_ROWS_OUT_FULL | RF_ROTARY_HALVES | RF_ROTARY_INVERSE;
    if (flags & ~known) return fail(RF_ERR_INVALID_ARG, "%s: unknown flags 0x%x", fn, flags);
    if (H <= 0 || W <= 0 || q_heads <= 0 || (k && k_heads <= 0) || head_dim <= 0)
        return fail(RF_ERR_INVALID_ARG, "%s: sizes must be positive (H=%d W=%d q_heads=%d k_heads=%d head_dim=%d)", fn,
                    H, W, q_heads, k_heads, head_dim);
    if (q_heads > 65535 || (k && k_heads > 65535))
        return fail(RF_ERR_RANGE, "%s: more than 65535 heads", fn);
    if (H > 65536 || W > 65536) return fail(RF_ERR_RANGE, "%s: H = %d or W = %d exceeds 65536", fn, H, W);
    if (static_cast<double>(H) * W > 67108864.0) return fail(RF_ERR_RANGE, "%s: more than 2^26 tokens a frame", fn);
    int32_t ids[RF_MAX_FRAMES];
    const int rc = check_id_list(frame_ids, M, T, ids, fn);
    if (rc != RF_OK) return rc;
    int64_t R = 0;
    for (int a = 0; a < 3; ++a) {
        if (axes->dims[a] < 0 || (axes->dims[a] & 1))
            return fail(RF_ERR_INVALID_ARG, "%s: axis %d turns %d dimensions (even, not negative)", fn, a, axes->dims[a]);
        if (!(axes->theta[a] >= 1.0) || !isfinite(axes->theta[a]))
            return fail(RF_ERR_INVALID_ARG, "%s: axis %d: theta must be finite and at least 1", fn, a);
        if (!isfinite(axes->origin[a]) || !isfinite(axes->step[a]))
            return fail(RF_ERR_INVALID_ARG, "%s: axis %d: origin and step must be finite", fn, a);
        if (fabs(axes->origin[a]) + 65536.0 * fabs(axes->step[a]) > 2147483648.0)
            return fail(RF_ERR_RANGE, "%s: axis %d: positions pass 2^31", fn, a);
        R += axes->dims[a];
    }
    if (R < 2 || R > head_dim)
        return fail(RF_ERR_INVALID_ARG, "%s: the axes turn %lld dimensions, a head has %d", fn,
                    static_cast<long long>(R), head_dim);
    if (head_dim % 8 != 0 || head_dim > 2 * rf::kMaxRotaryPairs)
        return fail(RF_ERR_UNSUPPORTED, "%s: head_dim %d is no multiple of 8 up to %d", fn, head_dim,
                    2 * rf::kMaxRotaryPairs);
    if ((flags & RF_ROTARY_HALVES) && R % 16 != 0)
        return fail(RF_ERR_UNSUPPORTED, "%s: halves of %lld dimensions (a multiple of 16)", fn,
                    static_cast<long long>(R));
    if (dtype != RF_BF16 && dtype != RF_F32) return fail(RF_ERR_UNSUPPORTED, "%s: unknown dtype %d", fn, dtype);
    const int64_t esize = dtype == RF_F32 ? 4 : 2;
    const int64_t N = static_cast<int64_t>(H) * W;
    const bool in_full = (flags & RF_ROWS_IN_FULL) != 0 || M == T, out_full = (flags & RF_ROWS_OUT_FULL) != 0 || M == T;
    const int64_t in_rows = N * (in_full ? T : M), out_rows = N * (out_full ? T : M);
    const int64_t heads[2] = {q_heads, k ? k_heads : 0};
    const void *in[2] = {q, k};
    void *out[2] = {q_out, k_out};
    rf::RotaryParams p{};
    int64_t row[2], is[2], os[2];
    for (int t = 0; t < (k ? 2 : 1); ++t) {
        const int64_t width = heads[t] * head_dim;
        is[t] = strides[2 * t] == 0 ? width : strides[2 * t];
        os[t] = strides[2 * t + 1] == 0 ? width : strides[2 * t + 1];
        if (is[t] < width || os[t] < width)
            return fail(RF_ERR_INVALID_ARG, "%s: a row stride is below the row's %lld elements", fn,
                        static_cast<long long>(width));
        if (static_cast<double>(N) * T * static_cast<double>(is[t]) * 4.0 > kMaxBytes ||
            static_cast<double>(N) * T * static_cast<double>(os[t]) * 4.0 > kMaxBytes)
            return fail(RF_ERR_RANGE, "%s: sizes overflow 64-bit byte counts", fn);
        if (!aligned16(in[t]) || !aligned16(out[t]) || (is[t] * esize) % 16 != 0 || (os[t] * esize) % 16 != 0)
            return fail(RF_ERR_UNSUPPORTED, "%s: pointers and row strides must be multiples of 16 bytes", fn);
        row[t] = width * esize;
        is[t] *= esize;
        os[t] *= esize;
        p.x[t] = in[t];
        p.y[t] = out[t];
        p.x_stride[t] = is[t] / esize;
        p.y_stride[t] = os[t] / esize;
        p.heads[t] = static_cast<int32_t>(heads[t]);
    }
    for (int t = 0; t < (k ? 2 : 1); ++t)
        for (int u = 0; u < (k ? 2 : 1); ++u) {
            const bool in_place = t == u && in[u] == out[t] && is[u] == os[t] && in_full == out_full;
            if (!in_place && rows_overlap(out[t], out_rows, os[t], row[t], in[u], in_rows, is[u], row[u]))
                return fail(RF_ERR_INVALID_ARG, "%s: an output overlaps an input", fn);
        }
    if (k && rows_overlap(q_out, out_rows, os[0], row[0], k_out, out_rows, os[1], row[1]))
        return fail(RF_ERR_INVALID_ARG, "%s: q_out overlaps k_out", fn);
    p.head_dim = head_dim;
    p.dtype = dtype;
    p.M = M;
    p.H = H;
    p.W = W;
    p.halves = (flags & RF_ROTARY_HALVES) != 0;
    p.pairs = static_cast<int32_t>(R / 2);
    p.pair_end[0] = axes->dims[0] / 2;
    p.pair_end[1] = (axes->dims[0] + axes->dims[1]) / 2;
    int32_t pair = 0;
    for (int a = 0; a < 3; ++a) {
        p.origin[a] = axes->origin[a];
        p.step[a] = axes->step[a];
        // theta^(-2j/dims) by multiplication: with 64-bit mantissas 128 of them stay right to a double's last place
        const long double ratio = axes->dims[a] > 0 ? powl(axes->theta[a], -2.0L / axes->dims[a]) : 1.0L;
        long double turns = ((flags & RF_ROTARY_INVERSE) ? -0.5L : 0.5L) / 3.14159265358979323846264338328L;
        for (int32_t j = 0; j < axes->dims[a] / 2; ++j, turns *= ratio) p.turns[pair++] = static_cast<double>(turns);
    }
    row_frames(ids, M, in_full, out_full, &p.frames);
    return launched(rf::launch_rotary(p, static_cast<hipStream_t>(stream)), fn);
}

int rf_rotary(const void *q, void *q_out, const void *k, void *k_out, const int32_t *frame_ids, int32_t M,
              int32_t T, int32_t H, int32_t W, int32_t q_heads, int32_t k_heads, int32_t head_dim,
              const rf_rotary_axes *axes, int64_t q_stride, int64_t q_out_stride, int64_t k_stride,
              int64_t k_out_stride, uint32_t flags, int32_t dtype, void *stream) {
    const int64_t strides[4] = {q_stride, q_out_stride, k_stride, k_out_stride};
    return rotary_call(q, q_out, k, k_out, frame_ids, M, T, H, W, q_heads, k_heads, head_dim, axes, strides, flags,
                       dtype, stream, "rf_rotary");
}

// Sizes common to a cross attention and its workspace query.
static int cross_sizes(int32_t B, int32_t Lq, int32_t Lk, int32_t heads, int32_t kv_heads, int32_t head_dim,
                       int32_t dtype, const char *fn) {
    if (B <= 0 || Lq <= 0 || Lk <= 0 || heads <= 0 || kv_heads <= 0)
        return fail(RF_ERR_INVALID_ARG, "%s: sizes must be positive (B=%d Lq=%d Lk=%d heads=%d kv_heads=%d)", fn, B,
                    Lq, Lk, heads, kv_heads);
    if (heads % kv_heads != 0)
        return fail(RF_ERR_INVALID_ARG, "%s: %d heads are no multiple of %d key heads", fn, heads, kv_heads);
    if (head_dim != 64 && head_dim != 128)
        return fail(RF_ERR_UNSUPPORTED, "%s: head_dim %d not in {64, 128}", fn, head_dim);
    if (dtype != RF_BF16 && dtype != RF_F32) return fail(RF_ERR_UNSUPPORTED, "%s: unknown dtype %d", fn, dtype);
    if (static_cast<double>(B) * Lq * heads * head_dim * 4.0 > kMaxBytes ||
        static_cast<double>(B) * Lk * kv_heads * head_dim * 4.0 > kMaxBytes)
        return fail(RF_ERR_RANGE, "%s: sizes overflow 64-bit byte counts", fn);
    if (Lk > (1 << 30)) return fail(RF_ERR_RANGE, "%s: Lk = %d exceeds 2^30", fn, Lk);
    if (static_cast<double>((static_cast<int64_t>(Lq) + 31) / 32) * B * heads > 16777216.0)
        return fail(RF_ERR_RANGE, "%s: more than 2^24 tiles of 32 queries", fn);
    if (!rf::cross_whole_fits(B, static_cast<int64_t>(heads / kv_heads) * Lq, kv_heads, dtype))
        return fail(RF_ERR_RANGE, "%s: more than 2^24 - 64 tiles of 128 queries in fp32", fn);
    return RF_OK;
}

// The compute units an operator's workspace is planned for (0: the current device's).
static int plan_units(int32_t compute_units, int32_t *cus, const char *fn) {
    if (compute_units < 0 || compute_units > RF_MAX_COMPUTE_UNITS)
        return fail(RF_ERR_RANGE, "%s: compute_units = %d outside 0..%d", fn, compute_units, RF_MAX_COMPUTE_UNITS);
    *cus = compute_units;
    if (compute_units > 0) return RF_OK;
    rf::DeviceGeometry geo;
    const int rc = query_geometry(&geo, fn);
    if (rc == RF_OK) *cus = geo.cus;
    return rc;
}

int rf_cross_attention_workspace(int32_t B, int32_t Lq, int32_t Lk, int32_t heads, int32_t kv_heads,
                                 int32_t head_dim, int32_t dtype, int32_t compute_units, int64_t *bytes_out) {
    const char *fn = "rf_cross_attention_workspace";
    if (!bytes_out) return fail(RF_ERR_INVALID_ARG, "%s: NULL output", fn);
    int rc = cross_sizes(B, Lq, Lk, heads, kv_heads, head_dim, dtype, fn);
    if (rc != RF_OK) return rc;
    int32_t cus = 0;
    rc = plan_units(compute_units, &cus, fn);
    if (rc != RF_OK) return rc;
    *bytes_out = rf::cross_workspace(B, Lq, Lk, heads, kv_heads, head_dim, dtype, cus);
    return ok();
}

// Bytes from the first to behind the last element of a [B][L][heads][head_dim]
// tensor of these strides (elements), or -1 where that passes kMaxBytes.
static int64_t strided_bytes(const int64_t (&st)[3], int64_t B, int64_t L, int64_t heads, int64_t d, int64_t esize) {
    const double top = (static_cast<double>(B - 1) * st[0] + static_cast<double>(L - 1) * st[1] +
                        static_cast<double>(heads - 1) * st[2] + d) * esize;
    if (top > kMaxBytes) return -1;
    return ((B - 1) * st[0] + (L - 1) * st[1] + (heads - 1) * st[2] + d) * esize;
}

// No element of a tensor of these strides lies in another's place: taken from the
// shortest stride up, each passes everything that the ones before span.
static bool distinct(const int64_t (&st)[3], int64_t B, int64_t L, int64_t heads, int64_t d) {
    const int64_t n[3] = {B, L, heads};
    bool used[3] = {n[0] == 1, n[1] == 1, n[2] == 1};
    double span = static_cast<double>(d);
    for (int i = 0; i < 3; ++i) {
        int at = -1;
        for (int j = 0; j < 3; ++j)
            if (!used[j] && (at < 0 || st[j] < st[at])) at = j;
        if (at < 0) break;
        if (static_cast<double>(st[at]) < span) return false;
        span += static_cast<double>(st[at]) * static_cast<double>(n[at] - 1);
        used[at] = true;
    }
    return true;
}

int rf_cross_attention(const void *q, const void *k, const void *v, void *out, const int32_t *kv_lengths,
                       const uint8_t *key_mask, int32_t B, int32_t Lq, int32_t Lk, int32_t heads,
                       int32_t kv_heads, int32_t head_dim, const rf_cross_layout *layout, int32_t dtype,
                       void *workspace, int64_t workspace_bytes, void *stream) {
    const char *fn = "rf_cross_attention";
    if (!q || !k || !v || !out) return fail(RF_ERR_INVALID_ARG, "%s: NULL tensor", fn);
    int rc = cross_sizes(B, Lq, Lk, heads, kv_heads, head_dim, dtype, fn);
    if (rc != RF_OK) return rc;
    rf::CrossParams p{};
    const int64_t esize = dtype == RF_F32 ? 4 : 2;
    const int64_t qrow = static_cast<int64_t>(heads) * head_dim, krow = static_cast<int64_t>(kv_heads) * head_dim;
    const rf_cross_layout plain = {{Lq * qrow, qrow, head_dim}, {Lk * krow, krow, head_dim},
                                   {Lk * krow, krow, head_dim}, {Lq * qrow, qrow, head_dim}};
    const rf_cross_layout &l = layout ? *layout : plain;
    const int64_t *const sets[4] = {l.q, l.k, l.v, l.out};
    int64_t *const dst[4] = {p.qs, p.ks, p.vs, p.os};
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 3; ++j) {
            if (sets[i][j] < 0) return fail(RF_ERR_INVALID_ARG, "%s: negative stride", fn);
            if (static_cast<double>(sets[i][j]) * 4.0 > kMaxBytes) return fail(RF_ERR_RANGE, "%s: a stride overflows", fn);
            if (sets[i][j] * esize % 16 != 0)
                return fail(RF_ERR_UNSUPPORTED, "%s: strides must be multiples of 16 bytes", fn);
            dst[i][j] = sets[i][j];
        }
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out))
        return fail(RF_ERR_UNSUPPORTED, "%s: pointers must be 16-byte aligned", fn);
    if (reinterpret_cast<uintptr_t>(kv_lengths) & 3u)
        return fail(RF_ERR_UNSUPPORTED, "%s: kv_lengths must be 4-byte aligned", fn);
    // (keys past a tile's last valid one lie past its memory: tokens do not overlap)
    if (Lk == 1) p.ks[1] = p.vs[1] = head_dim;
    if (p.ks[1] < head_dim || p.vs[1] < head_dim)
        return fail(RF_ERR_INVALID_ARG, "%s: a token stride of k or v is below head_dim", fn);
    // (byte offsets inside a tile of keys are 32-bit)
    if (p.ks[1] * esize >= (1 << 24) || p.vs[1] * esize >= (1 << 24))
        return fail(RF_ERR_UNSUPPORTED, "%s: a token stride of k or v reaches 16 MB", fn);
    if (!distinct(p.os, B, Lq, heads, head_dim))
        return fail(RF_ERR_INVALID_ARG, "%s: out's strides put elements into one place", fn);
    const int64_t qb = strided_bytes(p.qs, B, Lq, heads, head_dim, esize);
    const int64_t kb = strided_bytes(p.ks, B, Lk, kv_heads, head_dim, esize);
    const int64_t vb = strided_bytes(p.vs, B, Lk, kv_heads, head_dim, esize);
    const int64_t ob = strided_bytes(p.os, B, Lq, heads, head_dim, esize);
    if (qb < 0 || kb < 0 || vb < 0 || ob < 0) return fail(RF_ERR_RANGE, "%s: strides overflow 64-bit byte counts", fn);
    const int64_t mask_bytes = static_cast<int64_t>(B) * Lk;
    if (overlaps(out, ob, q, qb) || overlaps(out, ob, k, kb) || overlaps(out, ob, v, vb) ||
        (kv_lengths && overlaps(out, ob, kv_lengths, 4 * static_cast<int64_t>(B))) ||
        (key_mask && overlaps(out, ob, key_mask, mask_bytes)))
        return fail(RF_ERR_INVALID_ARG, "%s: out overlaps an input", fn);
    if (workspace) {
        if (workspace_bytes < 0) return fail(RF_ERR_INVALID_ARG, "%s: workspace_bytes < 0", fn);
        if (!aligned16(workspace)) return fail(RF_ERR_UNSUPPORTED, "%s: workspace must be 16-byte aligned", fn);
        const int64_t wb = workspace_bytes;
        if (wb > 0 && (overlaps(workspace, wb, q, qb) || overlaps(workspace, wb, k, kb) ||
                       overlaps(workspace, wb, v, vb) || overlaps(workspace, wb, out, ob) ||
                       (kv_lengths && overlaps(workspace, wb, kv_lengths, 4 * static_cast<int64_t>(B))) ||
                       (key_mask && overlaps(workspace, wb, key_mask, mask_bytes))))
            return fail(RF_ERR_INVALID_ARG, "%s: workspace overlaps a tensor", fn);
    }
    rc = query_geometry(&p.geo, fn);
    if (rc != RF_OK) return rc;
    if (workspace) {
        const int64_t need = rf::cross_workspace(B, Lq, Lk, heads, kv_heads, head_dim, dtype, p.geo.cus);
        if (workspace_bytes < need)
            return fail(RF_ERR_INVALID_ARG, "%s: workspace of %lld bytes, %lld needed on %d compute units", fn,
                        static_cast<long long>(workspace_bytes), static_cast<long long>(need), p.geo.cus);
        p.ws = need > 0 ? workspace : nullptr;
    }
    p.q = q;
    p.k = k;
    p.v = v;
    p.out = out;
    p.kv_lengths = kv_lengths;
    p.key_mask = key_mask;
    p.B = B;
    p.Lq = Lq;
    p.Lk = Lk;
    p.heads = heads;
    p.kv_heads = kv_heads;
    p.head_dim = head_dim;
    p.dtype = dtype;
    return launched(rf::launch_cross(p, static_cast<hipStream_t>(stream)), fn);
}

// Sizes common to a matrix product and its workspace query.
static int linear_sizes(int32_t M, int64_t N, int32_t K, int32_t n_out, int32_t dtype, const char *fn) {
    if (M <= 0 || N <= 0 || K <= 0 || n_out <= 0)
        return fail(RF_ERR_INVALID_ARG, "%s: sizes must be positive (M=%d rows_per_frame=%lld in=%d out=%d)", fn, M,
                    static_cast<long long>(N), K, n_out);
    if (static_cast<double>(M) * static_cast<double>(N) > 2147483647.0)
        return fail(RF_ERR_RANGE, "%s: %d frames of %lld rows exceed 2^31 - 1 rows", fn, M, static_cast<long long>(N));
    if (dtype != RF_BF16 && dtype != RF_F32) return fail(RF_ERR_UNSUPPORTED, "%s: unknown dtype %d", fn, dtype);
    const int32_t vec = dtype == RF_F32 ? 4 : 8;
    if (K % vec != 0 || n_out % vec != 0)
        return fail(RF_ERR_UNSUPPORTED, "%s: %d in_features or %d out_features make no rows of 16-byte multiples", fn,
                    K, n_out);
    // (byte offsets inside a tile of 256 rows are 32-bit)
    if (K >= (1 << 23) / (dtype == RF_F32 ? 4 : 2))
        return fail(RF_ERR_UNSUPPORTED, "%s: rows of in_features = %d reach 8 MB", fn, K);
    return RF_OK;
}

// Those of a product of 8-bit integers.
static int linear_i8_sizes(int32_t M, int64_t N, int32_t K, int32_t n_out, int32_t dtype, const char *fn) {
    if (M <= 0 || N <= 0 || K <= 0 || n_out <= 0)
        return fail(RF_ERR_INVALID_ARG, "%s: sizes must be positive (M=%d rows_per_frame=%lld in=%d out=%d)", fn, M,
                    static_cast<long long>(N), K, n_out);
    if (static_cast<double>(M) * static_cast<double>(N) > 2147483647.0)
        return fail(RF_ERR_RANGE, "%s: %d frames of %lld rows exceed 2^31 - 1 rows", fn, M, static_cast<long long>(N));
    if (dtype != RF_BF16 && dtype != RF_F32) return fail(RF_ERR_UNSUPPORTED, "%s: unknown dtype %d", fn, dtype);
    // (a sum's terms are 2^14 at most: 2^16 of them stay in 32 bits)
    static_assert(RF_I8_FEATURES * int64_t(128) * 128 < INT32_MAX, "sums of 8-bit products fit");
    if (K % 16 != 0 || K > RF_I8_FEATURES)
        return fail(RF_ERR_UNSUPPORTED, "%s: %d in_features are no multiple of 16 up to %d", fn, K, RF_I8_FEATURES);
    if (n_out % (dtype == RF_F32 ? 4 : 8) != 0)
        return fail(RF_ERR_UNSUPPORTED, "%s: %d out_features make no rows of 16-byte multiples", fn, n_out);
    return RF_OK;
}

int rf_frame_linear_workspace(int32_t M, int64_t rows_per_frame, int32_t in_features, int32_t out_features,
                              int32_t dtype, int32_t compute_units, int64_t *bytes_out) {
    const char *fn = "rf_frame_linear_workspace";
    if (!bytes_out) return fail(RF_ERR_INVALID_ARG, "%s: NULL output", fn);
    int rc = linear_sizes(M, rows_per_frame, in_features, out_features, dtype, fn);
    if (rc != RF_OK) return rc;
    int32_t cus = 0;
    rc = plan_units(compute_units, &cus, fn);
    if (rc != RF_OK) return rc;
    *bytes_out = rf::linear_workspace(M * rows_per_frame, in_features, out_features, dtype, cus);
    return ok();
}

// What a matrix product reads; with i8 set x and weight are int8 and have scales.
struct LinearIn {
    const void *x, *weight, *bias, *gate, *residual;
    bool i8;
    const float *x_scale, *w_scale;
};

static int linear_call(const LinearIn &in, void *y, const int32_t *frame_ids, int32_t M, int32_t T,
                       int64_t rows_per_frame, int32_t in_features, int32_t out_features, int32_t activation,
                       uint32_t flags, int32_t dtype, void *workspace, int64_t workspace_bytes, void *stream,
                       const char *fn) {
    if (!in.x || !in.weight || !y || (in.i8 && (!in.x_scale || !in.w_scale)))
        return fail(RF_ERR_INVALID_ARG, "%s: NULL tensor", fn);
    if (flags & ~(RF_ROWS_IN_FULL | RF_ROWS_OUT_FULL | RF_GATE_PER_FRAME))
        return fail(RF_ERR_INVALID_ARG, "%s: unknown flags 0x%x", fn, flags);
    if ((flags & RF_GATE_PER_FRAME) && !in.gate) return fail(RF_ERR_INVALID_ARG, "%s: a gate per frame needs a gate", fn);
    if (activation < RF_ACT_NONE || activation > RF_ACT_SILU)
        return fail(RF_ERR_INVALID_ARG, "%s: unknown activation %d", fn, activation);
    int32_t ids[RF_MAX_FRAMES];
    int rc = check_id_list(frame_ids, M, T, ids, fn);
    if (rc != RF_OK) return rc;
    rc = in.i8 ? linear_i8_sizes(M, rows_per_frame, in_features, out_features, dtype, fn)
               : linear_sizes(M, rows_per_frame, in_features, out_features, dtype, fn);
    if (rc != RF_OK) return rc;
    if (static_cast<double>(T) * static_cast<double>(rows_per_frame) * (in_features > out_features ? in_features : out_features) * 4.0 >
        kMaxBytes)
        return fail(RF_ERR_RANGE, "%s: sizes overflow 64-bit byte counts", fn);
    if (!aligned16(in.x) || !aligned16(in.weight) || !aligned16(y) || !aligned16(in.bias) || !aligned16(in.gate) ||
        !aligned16(in.residual) || !aligned16(in.w_scale))
        return fail(RF_ERR_UNSUPPORTED, "%s: pointers must be 16-byte aligned", fn);
    if (!aligned4(in.x_scale)) return fail(RF_ERR_UNSUPPORTED, "%s: x_scale must be 4-byte aligned", fn);
    const int64_t esize = dtype == RF_F32 ? 4 : 2, in_size = in.i8 ? 1 : esize;
    const int64_t in_rows = rows_per_frame * ((flags & RF_ROWS_IN_FULL) ? T : M);
    const int64_t out_rows = rows_per_frame * ((flags & RF_ROWS_OUT_FULL) ? T : M);
    const int64_t out_row = out_features * esize;
    struct Range {
        const void *p;
        int64_t n;
    };
    const Range ins[7] = {{in.x, in_rows * in_features * in_size},
                          {in.weight, static_cast<int64_t>(out_features) * in_features * in_size},
                          {in.bias, out_row},
                          {in.gate, out_row * ((flags & RF_GATE_PER_FRAME) ? T : 1)},
                          {in.residual == y ? nullptr : in.residual, out_rows * out_row},
                          {in.x_scale, in_rows * 4},
                          {in.w_scale, static_cast<int64_t>(out_features) * 4}};
    for (const Range &r : ins)
        if (r.p && overlaps(y, out_rows * out_row, r.p, r.n))
            return fail(RF_ERR_INVALID_ARG, "%s: y overlaps an input", fn);
    if (workspace) {
        if (workspace_bytes < 0) return fail(RF_ERR_INVALID_ARG, "%s: workspace_bytes < 0", fn);
        if (!aligned16(workspace)) return fail(RF_ERR_UNSUPPORTED, "%s: workspace must be 16-byte aligned", fn);
        if (workspace_bytes > 0) {
            bool hit = overlaps(workspace, workspace_bytes, y, out_rows * out_row);
            for (const Range &r : ins) hit = hit || (r.p && overlaps(workspace, workspace_bytes, r.p, r.n));
            if (hit) return fail(RF_ERR_INVALID_ARG, "%s: workspace overlaps a tensor", fn);
        }
    }
    if (!rf::linear_whole_fits(M * rows_per_frame, out_features))
        return fail(RF_ERR_RANGE, "%s: more than 2^24 - 64 tiles of 128 rows and 128 features", fn);
    rf::LinearParams p{};
    rc = query_geometry(&p.geo, fn);
    if (rc != RF_OK) return rc;
    if (workspace) {
        const int64_t need = in.i8 ? rf::linear_i8_workspace(M * rows_per_frame, in_features, out_features, dtype, p.geo.cus)
                                   : rf::linear_workspace(M * rows_per_frame, in_features, out_features, dtype, p.geo.cus);
        if (workspace_bytes < need)
            return fail(RF_ERR_INVALID_ARG, "%s: workspace of %lld bytes, %lld needed on %d compute units", fn,
                        static_cast<long long>(workspace_bytes), static_cast<long long>(need), p.geo.cus);
        p.ws = need > 0 ? workspace : nullptr;
    }
    p.x = in.x;
    p.weight = in.weight;
    p.bias = in.bias;
    p.gate = in.gate;
    p.residual = in.residual;
    p.y = y;
    p.N = rows_per_frame;
    p.M = M;
    p.K = in_features;
    p.n_out = out_features;
    p.activation = activation;
    p.dtype = dtype;
    p.gate_rows = (flags & RF_GATE_PER_FRAME) != 0;
    row_frames(ids, M, (flags & RF_ROWS_IN_FULL) != 0, (flags & RF_ROWS_OUT_FULL) != 0, &p.frames);
    hipStream_t hs = static_cast<hipStream_t>(stream);
    return launched(in.i8 ? rf::launch_linear_i8(p, in.x_scale, in.w_scale, hs) : rf::launch_linear(p, hs), fn);
}

int rf_frame_linear(const void *x, const void *weight, const void *bias, const void *gate, const void *residual,
                    void *y, const int32_t *frame_ids, int32_t M, int32_t T, int64_t rows_per_frame,
                    int32_t in_features, int32_t out_features, int32_t activation, uint32_t flags, int32_t dtype,
                    void *workspace, int64_t workspace_bytes, void *stream) {
    const LinearIn in = {x, weight, bias, gate, residual, false, nullptr, nullptr};
    return linear_call(in, y, frame_ids, M, T, rows_per_frame, in_features, out_features, activation, flags, dtype,
                       workspace, workspace_bytes, stream, "rf_frame_linear");
}

int rf_frame_linear_i8_workspace(int32_t M, int64_t rows_per_frame, int32_t in_features, int32_t out_features,
                                 int32_t dtype, int32_t compute_units, int64_t *bytes_out) {
    const char *fn = "rf_frame_linear_i8_workspace";
    if (!bytes_out) return fail(RF_ERR_INVALID_ARG, "%s: NULL output", fn);
    int rc = linear_i8_sizes(M, rows_per_frame, in_features, out_features, dtype, fn);
    if (rc != RF_OK) return rc;
    int32_t cus = 0;
    rc = plan_units(compute_units, &cus, fn);
    if (rc != RF_OK) return rc;
    *bytes_out = rf::linear_i8_workspace(M * rows_per_frame, in_features, out_features, dtype, cus);
    return ok();
}

int rf_frame_linear_i8(const int8_t *x, const float *x_scale, const int8_t *weight, const float *weight_scale,
                       const void *bias, const void *gate, const void *residual, void *y, const int32_t *frame_ids,
                       int32_t M, int32_t T, int64_t rows_per_frame, int32_t in_features, int32_t out_features,
                       int32_t activation, uint32_t flags, int32_t dtype, void *workspace, int64_t workspace_bytes,
                       void *stream) {
    const LinearIn in = {x, weight, bias, gate, residual, true, x_scale, weight_scale};
    return linear_call(in, y, frame_ids, M, T, rows_per_frame, in_features, out_features, activation, flags, dtype,
                       workspace, workspace_bytes, stream, "rf_frame_linear_i8");
}

int rf_frame_quantize(const void *x, int8_t *q, float *scale, const int32_t *frame_ids, int32_t M, int32_t T,
                      int64_t rows_per_frame, int32_t features, int64_t x_stride, uint32_t flags, int32_t dtype,
                      void *stream) {
    const char *fn = "rf_frame_quantize";
    if (!x || !q || !scale) return fail(RF_ERR_INVALID_ARG, "%s: NULL tensor", fn);
    if (flags & ~(RF_ROWS_IN_FULL | RF_ROWS_OUT_FULL)) return fail(RF_ERR_INVALID_ARG, "%s: unknown flags 0x%x", fn, flags);
    int32_t ids[RF_MAX_FRAMES];
    int rc = check_id_list(frame_ids, M, T, ids, fn);
    if (rc != RF_OK) return rc;
    if (rows_per_frame <= 0 || features <= 0)
        return fail(RF_ERR_INVALID_ARG, "%s: sizes must be positive (rows_per_frame=%lld features=%d)", fn,
                    static_cast<long long>(rows_per_frame), features);
    if (static_cast<double>(M) * static_cast<double>(rows_per_frame) > 2147483647.0)
        return fail(RF_ERR_RANGE, "%s: more than 2^31 - 1 rows", fn);
    if (dtype != RF_BF16 && dtype != RF_F32) return fail(RF_ERR_UNSUPPORTED, "%s: unknown dtype %d", fn, dtype);
    if (features % 16 != 0 || features > RF_I8_FEATURES)
        return fail(RF_ERR_UNSUPPORTED, "%s: %d features are no multiple of 16 up to %d", fn, features, RF_I8_FEATURES);
    const int64_t esize = dtype == RF_F32 ? 4 : 2, stride = x_stride == 0 ? features : x_stride;
    if (stride < features)
        return fail(RF_ERR_INVALID_ARG, "%s: x_stride is below the row's %d elements", fn, features);
    if (static_cast<double>(T) * static_cast<double>(rows_per_frame) * static_cast<double>(stride) * 4.0 > kMaxBytes)
        return fail(RF_ERR_RANGE, "%s: sizes overflow 64-bit byte counts", fn);
    if (!aligned16(x) || !aligned16(q) || (stride * esize) % 16 != 0)
        return fail(RF_ERR_UNSUPPORTED, "%s: x, q and the row stride must be multiples of 16 bytes", fn);
    if (!aligned4(scale)) return fail(RF_ERR_UNSUPPORTED, "%s: scale must be 4-byte aligned", fn);
    const int64_t in_rows = rows_per_frame * ((flags & RF_ROWS_IN_FULL) ? T : M);
    const int64_t out_rows = rows_per_frame * ((flags & RF_ROWS_OUT_FULL) ? T : M);
    const int64_t in_bytes = ((in_rows - 1) * stride + features) * esize;
    if (overlaps(q, out_rows * features, x, in_bytes) || overlaps(scale, out_rows * 4, x, in_bytes) ||
        overlaps(scale, out_rows * 4, q, out_rows * features))
        return fail(RF_ERR_INVALID_ARG, "%s: an output overlaps a tensor", fn);
    rf::QuantizeParams p{};
    p.x = x;
    p.q = q;
    p.scale = scale;
    p.N = rows_per_frame;
    p.x_stride = stride;
    p.M = M;
    p.K = features;
    p.dtype = dtype;
    row_frames(ids, M, (flags & RF_ROWS_IN_FULL) != 0, (flags & RF_ROWS_OUT_FULL) != 0, &p.frames);
    return launched(rf::launch_quantize(p, static_cast<hipStream_t>(stream)), fn);
}

// Sizes common to a group norm and its workspace query.
static int norm_sizes(int32_t M, int64_t N, int32_t C, int32_t groups, int32_t together, bool rows8, int32_t dtype,
                      const char *fn) {
    if (M <= 0 || N <= 0 || C <= 0 || groups <= 0 || together <= 0)
        return fail(RF_ERR_INVALID_ARG, "%s: sizes must be positive (M=%d rows_per_frame=%lld channels=%d groups=%d "
                    "frames_together=%d)", fn, M, static_cast<long long>(N), C, groups, together);
    if (M > RF_MAX_FRAMES) return fail(RF_ERR_RANGE, "%s: M = %d exceeds %d frames", fn, M, RF_MAX_FRAMES);
    if (static_cast<double>(M) * static_cast<double>(N) > 2147483647.0)
        return fail(RF_ERR_RANGE, "%s: more than 2^31 - 1 rows", fn);
    if (dtype != RF_BF16 && dtype != RF_F32) return fail(RF_ERR_UNSUPPORTED, "%s: unknown dtype %d", fn, dtype);
    const int32_t vec = rows8 ? 16 : dtype == RF_F32 ? 4 : 8;
    if (C % vec != 0 || C > RF_NORM_CHANNELS)
        return fail(RF_ERR_UNSUPPORTED, "%s: %d channels are no multiple of %d up to %d", fn, C, vec, RF_NORM_CHANNELS);
    if (C % groups != 0) return fail(RF_ERR_INVALID_ARG, "%s: %d groups do not divide %d channels", fn, groups, C);
    if (M % together != 0)
        return fail(RF_ERR_INVALID_ARG, "%s: frames_together = %d does not divide %d frames", fn, together, M);
    return RF_OK;
}

int rf_frame_group_norm_workspace(int32_t M, int64_t rows_per_frame, int32_t channels, int32_t groups,
                                  int32_t frames_together, int32_t rows_8bit, int32_t dtype, int32_t compute_units,
                                  int64_t *bytes_out) {
    const char *fn = "rf_frame_group_norm_workspace";
    if (!bytes_out) return fail(RF_ERR_INVALID_ARG, "%s: NULL output", fn);
    int rc = norm_sizes(M, rows_per_frame, channels, groups, frames_together, rows_8bit != 0, dtype, fn);
    if (rc != RF_OK) return rc;
    int32_t cus = 0;
    rc = plan_units(compute_units, &cus, fn);
    if (rc != RF_OK) return rc;
    *bytes_out = rf::norm_workspace(M, rows_per_frame, channels, groups, frames_together, rows_8bit != 0, dtype, cus);
    return ok();
}

int rf_frame_group_norm(const void *x, const void *weight, const void *bias, void *y, float *y_scale,
                        const int32_t *frame_ids, int32_t M, int32_t T, int64_t rows_per_frame, int32_t channels,
                        int32_t groups, int32_t frames_together, double eps, int32_t activation, int64_t x_stride,
                        int64_t y_stride, uint32_t flags, int32_t dtype, void *workspace, int64_t workspace_bytes,
                        void *stream) {
    const char *fn = "rf_frame_group_norm";
    if (!x || !y) return fail(RF_ERR_INVALID_ARG, "%s: NULL tensor", fn);
    if (flags & ~(RF_ROWS_IN_FULL | RF_ROWS_OUT_FULL | RF_AFFINE_PER_FRAME))
        return fail(RF_ERR_INVALID_ARG, "%s: unknown flags 0x%x", fn, flags);
    if ((flags & RF_AFFINE_PER_FRAME) && !weight && !bias)
        return fail(RF_ERR_INVALID_ARG, "%s: a weight and bias per frame need one of them", fn);
    if (activation < RF_ACT_NONE || activation > RF_ACT_SILU)
        return fail(RF_ERR_INVALID_ARG, "%s: unknown activation %d", fn, activation);
    if (!(eps >= 1e-30 && eps <= 1e30)) return fail(RF_ERR_INVALID_ARG, "%s: eps outside 1e-30..1e30", fn);
    int32_t ids[RF_MAX_FRAMES];
    int rc = check_id_list(frame_ids, M, T, ids, fn);
    if (rc != RF_OK) return rc;
    const bool rows8 = y_scale != nullptr;
    rc = norm_sizes(M, rows_per_frame, channels, groups, frames_together, rows8, dtype, fn);
    if (rc != RF_OK) return rc;
    const int64_t N = rows_per_frame, C = channels, esize = dtype == RF_F32 ? 4 : 2, out_size = rows8 ? 1 : esize;
    const int64_t xs = x_stride == 0 ? C : x_stride, ys = y_stride == 0 ? C : y_stride;
    if (xs < C || ys < C) return fail(RF_ERR_INVALID_ARG, "%s: a row stride is below the row's %d elements", fn, channels);
    if (rows8 && ys != C) return fail(RF_ERR_INVALID_ARG, "%s: rows in 8 bits are contiguous", fn);
    if (static_cast<double>(T) * static_cast<double>(N) * static_cast<double>(xs > ys ? xs : ys) * 4.0 > kMaxBytes)
        return fail(RF_ERR_RANGE, "%s: sizes overflow 64-bit byte counts", fn);
    if (!aligned16(x) || !aligned16(y) || !aligned16(weight) || !aligned16(bias) || (xs * esize) % 16 != 0 ||
        (ys * out_size) % 16 != 0)
        return fail(RF_ERR_UNSUPPORTED, "%s: pointers and row strides must be multiples of 16 bytes", fn);
    if (!aligned4(y_scale)) return fail(RF_ERR_UNSUPPORTED, "%s: y_scale must be 4-byte aligned", fn);
    const bool in_full = (flags & RF_ROWS_IN_FULL) != 0 || M == T, out_full = (flags & RF_ROWS_OUT_FULL) != 0 || M == T;
    const int64_t in_rows = N * (in_full ? T : M), out_rows = N * (out_full ? T : M);
    const bool in_place = !rows8 && y == x && xs == ys && in_full == out_full;
    if (!in_place && rows_overlap(y, out_rows, ys * out_size, C * out_size, x, in_rows, xs * esize, C * esize))
        return fail(RF_ERR_INVALID_ARG, "%s: y overlaps x", fn);
    const int64_t in_bytes = ((in_rows - 1) * xs + C) * esize, out_bytes = ((out_rows - 1) * ys + C) * out_size;
    const int64_t affine = C * esize * ((flags & RF_AFFINE_PER_FRAME) ? T : 1);
    if ((weight && overlaps(y, out_bytes, weight, affine)) || (bias && overlaps(y, out_bytes, bias, affine)))
        return fail(RF_ERR_INVALID_ARG, "%s: y overlaps an input", fn);
    if (rows8 && (overlaps(y_scale, out_rows * 4, x, in_bytes) || overlaps(y_scale, out_rows * 4, y, out_bytes) ||
                  (weight && overlaps(y_scale, out_rows * 4, weight, affine)) ||
                  (bias && overlaps(y_scale, out_rows * 4, bias, affine))))
        return fail(RF_ERR_INVALID_ARG, "%s: y_scale overlaps a tensor", fn);
    if (workspace) {
        if (workspace_bytes < 0) return fail(RF_ERR_INVALID_ARG, "%s: workspace_bytes < 0", fn);
        if (!aligned16(workspace)) return fail(RF_ERR_UNSUPPORTED, "%s: workspace must be 16-byte aligned", fn);
        if (workspace_bytes > 0 &&
            (overlaps(workspace, workspace_bytes, x, in_bytes) || overlaps(workspace, workspace_bytes, y, out_bytes) ||
             (weight && overlaps(workspace, workspace_bytes, weight, affine)) ||
             (bias && overlaps(workspace, workspace_bytes, bias, affine)) ||
             (rows8 && overlaps(workspace, workspace_bytes, y_scale, out_rows * 4))))
            return fail(RF_ERR_INVALID_ARG, "%s: workspace overlaps a tensor", fn);
    }
    rf::NormParams p{};
    rc = query_geometry(&p.geo, fn);
    if (rc != RF_OK) return rc;
    const int64_t need = rf::norm_workspace(M, N, channels, groups, frames_together, rows8, dtype, p.geo.cus);
    if (need > 0 && (!workspace || workspace_bytes < need))
        return fail(RF_ERR_INVALID_ARG, "%s: workspace of %lld bytes, %lld needed on %d compute units", fn,
                    static_cast<long long>(workspace ? workspace_bytes : 0), static_cast<long long>(need), p.geo.cus);
    p.x = x;
    p.weight = weight;
    p.bias = bias;
    p.y = y;
    p.y_scale = y_scale;
    p.N = N;
    p.x_stride = xs;
    p.y_stride = ys;
    p.eps = eps;
    p.M = M;
    p.C = channels;
    p.groups = groups;
    p.together = frames_together;
    p.activation = activation;
    p.dtype = dtype;
    p.affine_rows = (flags & RF_AFFINE_PER_FRAME) != 0;
    p.ws = workspace;
    row_frames(ids, M, in_full, out_full, &p.frames);
    return launched(rf::launch_norm(p, static_cast<hipStream_t>(stream)), fn);
}

int rf_probe_mfma_bf16(const void *operands, int32_t workgroups, int32_t rounds, float *sink, void *stream) {
    const char *fn = "rf_probe_mfma_bf16";
    if (!operands || !sink) return fail(RF_ERR_INVALID_ARG, "%s: NULL argument", fn);
    if (workgroups < 1 || workgroups > (1 << 20) || rounds < 1 || rounds > (1 << 22))
        return fail(RF_ERR_RANGE, "%s: workgroups %d (1..2^20) or rounds %d (1..2^22) out of range", fn,
                    workgroups, rounds);
    if (!aligned16(operands) || (reinterpret_cast<uintptr_t>(sink) & 3u))
        return fail(RF_ERR_UNSUPPORTED, "%s: operands must be 16-byte and sink 4-byte aligned", fn);
    return launched(rf::launch_mfma_probe(operands, workgroups, rounds, sink, static_cast<hipStream_t>(stream)),
                    fn);
}

int rf_probe_lds_read(int32_t workgroups, int32_t rounds, int32_t width, uint32_t *sink, uint64_t *ticks,
                      void *stream) {
    const char *fn = "rf_probe_lds_read";
    if (!sink) return fail(RF_ERR_INVALID_ARG, "%s: NULL sink", fn);
    if (width != 16 && width != 8) return fail(RF_ERR_INVALID_ARG, "%s: width %d is not 16 or 8", fn, width);
    if (workgroups < 1 || workgroups > (1 << 20) || rounds < 1 || rounds > (1 << 22))
        return fail(RF_ERR_RANGE, "%s: workgroups %d (1..2^20) or rounds %d (1..2^22) out of range", fn,
                    workgroups, rounds);
    if ((reinterpret_cast<uintptr_t>(sink) & 3u) || (reinterpret_cast<uintptr_t>(ticks) & 7u))
        return fail(RF_ERR_UNSUPPORTED, "%s: sink must be 4-byte and ticks 8-byte aligned", fn);
    return launched(
        rf::launch_lds_read_probe(workgroups, rounds, width, sink, ticks, static_cast<hipStream_t>(stream)), fn);
}

int rf_probe_hbm_read(const void *src, int64_t bytes, int32_t workgroups, uint32_t *sink, void *stream) {
    const char *fn = "rf_probe_hbm_read";
    if (!src || !sink) return fail(RF_ERR_INVALID_ARG, "%s: NULL argument", fn);
    if (bytes < 16 || bytes % 16 != 0)
        return fail(RF_ERR_INVALID_ARG, "%s: bytes = %lld must be a positive multiple of 16", fn,
                    static_cast<long long>(bytes));
    if (workgroups < 1 || workgroups > (1 << 20))
        return fail(RF_ERR_RANGE, "%s: workgroups %d out of range (1..2^20)", fn, workgroups);
    if (!aligned16(src) || (reinterpret_cast<uintptr_t>(sink) & 3u))
        return fail(RF_ERR_UNSUPPORTED, "%s: src must be 16-byte and sink 4-byte aligned", fn);
    return launched(rf::launch_hbm_read_probe(src, bytes, workgroups, sink, static_cast<hipStream_t>(stream)), fn);
}

}  // extern "C"
