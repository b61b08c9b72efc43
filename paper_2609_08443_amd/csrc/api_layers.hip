// Host side of the C ABI (include/sa_sketch.h): the attention over recent histories.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "recent_attn.h"
#include "sa_internal.h"

namespace {

using sa::api_fail;

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
sa_status hip_fail(hipError_t e, const char* what) { return api_fail(SA_ERR_HIP, "%s: %s", what, hipGetErrorString(e)); }

// ---------------------------------------------------------------- attention over recent histories
struct AttnPlan {
    bool wide = false;
    sa::attn::RowsShape shape;
    int64_t tiles = 0;
    int32_t grid = 1;
    size_t off_recs = 0, off_prefix = 0, off_parts = 0, off_delta = 0, total = 0;
};

AttnPlan plan_attn(const sa_recent_attn& a, bool bwd) {
    AttnPlan p;
    const bool bf = a.dtype == SA_BF16;
    const int64_t g = a.h / a.hk, rows = a.N * g;
    // tiles of 128 rows where users have that many on average
    p.wide = rows > 48 * a.B;
    p.shape = sa::attn::rows_shape(bf, a.d, p.wide, bwd);
    p.tiles = rows / p.shape.bq + a.B + 1;
    // no more workgroups than units of work
    const double most = (double)p.tiles * a.hk * std::max<int64_t>(1, (a.T + p.shape.unit - 1) / p.shape.unit);
    p.grid = (int32_t)std::min<double>(most, (double)sa::device_cus() * p.shape.per_cu);
    size_t off = 0;
    auto carve = [&](size_t bytes) {
        const size_t o = off;
        off = align_up(off + bytes, 256);
        return o;
    };
    p.off_recs = carve(sizeof(sa::attn::TileRec) * (size_t)p.tiles);
    p.off_prefix = carve(sizeof(int64_t) * ((size_t)p.tiles + 1));
    p.off_parts = carve(sizeof(float) * 2 * (size_t)p.grid * p.shape.bq * (a.d + 2));
    if (bwd) p.off_delta = carve(sizeof(float) * (size_t)a.N * a.h);
    p.total = off;
    return p;
}

sa_status check_attn_sizes(const sa_recent_attn* a) {
    if (!a) return api_fail(SA_ERR_INVALID_ARG, "null pointer argument");
    if (a->dtype != SA_BF16 && a->dtype != SA_FP32) return api_fail(SA_ERR_INVALID_ARG, "unknown dtype %d", (int)a->dtype);
    if (a->B < 0 || a->T < 0 || a->N < 0 || a->h < 1 || a->hk < 1 || a->d < 1 || a->window < 0)
        return api_fail(SA_ERR_INVALID_ARG, "bad sizes B=%lld T=%lld N=%lld h=%d hk=%d d=%d window=%d", (long long)a->B,
                        (long long)a->T, (long long)a->N, a->h, a->hk, a->d, a->window);
    if (a->h % a->hk != 0) return api_fail(SA_ERR_INVALID_ARG, "h=%d is not a multiple of hk=%d", a->h, a->hk);
    if (!(std::isfinite(a->scale) && a->scale > 0.f)) return api_fail(SA_ERR_INVALID_ARG, "scale must be finite and > 0");
    if (!(std::isfinite(a->cap) && a->cap >= 0.f)) return api_fail(SA_ERR_INVALID_ARG, "cap must be finite and >= 0");
    if (a->d != 64 && a->d != 128) return api_fail(SA_ERR_UNSUPPORTED, "d must be 64 or 128 (got %d)", a->d);
    constexpr int64_t k31 = int64_t(1) << 31;
    if (a->h > 65536) return api_fail(SA_ERR_UNSUPPORTED, "h must be <= 65536 (got %d)", a->h);
    if (a->T >= k31 || a->N >= k31 || a->N * a->h >= k31 || a->B >= k31 - 1 || a->B + a->T / 128 + 1 >= k31)
        return api_fail(SA_ERR_UNSUPPORTED, "sizes beyond the supported range");
    return SA_OK;
}

// a stride pair of [., heads, d], with those of a packed tensor for 0
sa_status check_strides(const char* name, int64_t* row, int64_t* head, int32_t heads, int32_t d, bool bf) {
    if (*head == 0) *head = d;
    if (*row == 0) *row = (int64_t)heads * d;
    const int64_t step = bf ? 8 : 4;
    if (*row < 0 || *head < 0 || *row % step != 0 || *head % step != 0)
        return api_fail(SA_ERR_INVALID_ARG, "the strides of %s must be multiples of 16 bytes", name);
    // (rows of a tile and heads are addressed in 32 bits)
    if (*row >= (int64_t(1) << 24) || *head * heads >= (int64_t(1) << 24))
        return api_fail(SA_ERR_UNSUPPORTED, "the strides of %s must span less than 2^24 elements", name);
    return SA_OK;
}

sa_status attn_view(const sa_recent_attn& a, sa::attn::View* v) {
    const bool bf = a.dtype == SA_BF16;
    *v = {a.q, a.K, a.V, a.offsets, a.targets, a.ends, a.slopes, a.B, a.T, a.N, a.h, a.hk, a.h / a.hk, a.window, a.scale,
          a.cap, a.q_stride, a.q_head_stride, a.k_stride, a.k_head_stride, a.v_stride, a.v_head_stride};
    sa_status st = check_strides("q", &v->q_t, &v->q_h, a.h, a.d, bf);
    if (st == SA_OK) st = check_strides("K", &v->k_t, &v->k_h, a.hk, a.d, bf);
    if (st == SA_OK) st = check_strides("V", &v->v_t, &v->v_h, a.hk, a.d, bf);
    if (st != SA_OK) return st;
    if (!a.offsets || !a.targets || (a.N > 0 && !a.q) || (a.T > 0 && (!a.K || !a.V)))
        return api_fail(SA_ERR_INVALID_ARG, "null pointer argument");
    if (!aligned16(a.q) || !aligned16(a.K) || !aligned16(a.V) || !aligned16(a.offsets) || !aligned16(a.targets) ||
        !aligned16(a.ends) || !aligned16(a.slopes))
        return api_fail(SA_ERR_INVALID_ARG, "tensor arguments must be 16-byte aligned");
    return SA_OK;
}

sa_status check_workspace(const void* workspace, size_t bytes, size_t need) {
    if (!workspace || bytes < need)
        return api_fail(SA_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, workspace ? bytes : (size_t)0);
    if (!aligned16(workspace)) return api_fail(SA_ERR_WORKSPACE, "workspace must be 16-byte aligned");
    return SA_OK;
}

sa::attn::RowsArgs rows_args(const sa::attn::View& v, const AttnPlan& p, uint8_t* ws) {
    sa::attn::RowsArgs f{};
    f.a = v;
    f.p = {reinterpret_cast<const sa::attn::TileRec*>(ws + p.off_recs), reinterpret_cast<const int64_t*>(ws + p.off_prefix),
           p.tiles, 1};
    f.parts = reinterpret_cast<float*>(ws + p.off_parts);
    f.grid = p.grid;
    return f;
}

hipError_t run_rows(const sa::attn::RowsArgs& f, const AttnPlan& p, const sa_recent_attn& a, bool bwd, uint8_t* ws,
                    hipStream_t stream) {
    const bool bf = a.dtype == SA_BF16;
    hipError_t e;
    {
        sa::ProfScope ps("recent_attn_plan", stream);
        e = sa::attn::launch_plan(f.a, p.shape, p.tiles, reinterpret_cast<sa::attn::TileRec*>(ws + p.off_recs),
                                  reinterpret_cast<int64_t*>(ws + p.off_prefix), stream);
    }
    if (e == hipSuccess) {
        sa::ProfScope ps(bwd ? "recent_attn_dq" : "recent_attn_fwd", stream);
        e = bwd ? sa::attn::launch_rows_dq(f, bf, a.d, p.wide, stream) : sa::attn::launch_rows_fwd(f, bf, a.d, p.wide, stream);
    }
    if (e == hipSuccess) {
        sa::ProfScope ps("recent_attn_join", stream);
        e = sa::attn::launch_join(f, bf, a.d, p.shape.bq, bwd, stream);
    }
    return e;
}

}  // namespace

extern "C" {

size_t sa_recent_attn_fwd_workspace_size(const sa_recent_attn* a) {
    return check_attn_sizes(a) == SA_OK ? plan_attn(*a, false).total : 0;
}

sa_status sa_recent_attn_fwd(const sa_recent_attn* a, void* out, float* lse, void* workspace, size_t workspace_bytes,
                             void* stream_) {
    sa::api_clear();
    sa_status st = check_attn_sizes(a);
    if (st != SA_OK) return st;
    if (a->N == 0) return SA_OK;
    sa::attn::View v;
    st = attn_view(*a, &v);
    if (st != SA_OK) return st;
    if (!out) return api_fail(SA_ERR_INVALID_ARG, "null pointer argument");
    if (!aligned16(out) || !aligned16(lse)) return api_fail(SA_ERR_INVALID_ARG, "tensor arguments must be 16-byte aligned");
    const AttnPlan p = plan_attn(*a, false);
    st = check_workspace(workspace, workspace_bytes, p.total);
    if (st != SA_OK) return st;
    uint8_t* ws = reinterpret_cast<uint8_t*>(workspace);
    hipStream_t stream = reinterpret_cast<hipStream_t>(stream_);
    sa::attn::RowsArgs f = rows_args(v, p, ws);
    f.out = out;
    f.lse = lse;
    const hipError_t e = run_rows(f, p, *a, false, ws, stream);
    if (e != hipSuccess) return hip_fail(e, "recent attention launch");
    return SA_OK;
}

size_t sa_recent_attn_bwd_workspace_size(const sa_recent_attn* a) {
    return check_attn_sizes(a) == SA_OK ? plan_attn(*a, true).total : 0;
}

sa_status sa_recent_attn_bwd(const sa_recent_attn* a, const void* out, const float* lse, const void* dout,
                             const sa_recent_attn_grads* grads, void* workspace, size_t workspace_bytes, void* stream_) {
    sa::api_clear();
    sa_status st = check_attn_sizes(a);
    if (st != SA_OK) return st;
    if (a->N == 0 && a->T == 0) return SA_OK;
    sa::attn::View v;
    st = attn_view(*a, &v);
    if (st != SA_OK) return st;
    if (!grads) return api_fail(SA_ERR_INVALID_ARG, "null pointer argument");
    sa_recent_attn_grads gr = *grads;
    const bool bf = a->dtype == SA_BF16;
    st = check_strides("dq", &gr.dq_stride, &gr.dq_head_stride, a->h, a->d, bf);
    if (st == SA_OK) st = check_strides("dK", &gr.dk_stride, &gr.dk_head_stride, a->hk, a->d, bf);
    if (st == SA_OK) st = check_strides("dV", &gr.dv_stride, &gr.dv_head_stride, a->hk, a->d, bf);
    if (st != SA_OK) return st;
    if ((a->N > 0 && (!out || !lse || !dout || !gr.dq)) || (a->T > 0 && (!gr.dK || !gr.dV)))
        return api_fail(SA_ERR_INVALID_ARG, "null pointer argument");
    if (!aligned16(out) || !aligned16(lse) || !aligned16(dout) || !aligned16(gr.dq) || !aligned16(gr.dK) || !aligned16(gr.dV))
        return api_fail(SA_ERR_INVALID_ARG, "tensor arguments must be 16-byte aligned");
    const AttnPlan p = plan_attn(*a, true);
    st = check_workspace(workspace, workspace_bytes, p.total);
    if (st != SA_OK) return st;
    uint8_t* ws = reinterpret_cast<uint8_t*>(workspace);
    hipStream_t stream = reinterpret_cast<hipStream_t>(stream_);
    float* delta = reinterpret_cast<float*>(ws + p.off_delta);
    hipError_t e = hipSuccess;
    if (a->N > 0) {
        sa::attn::RowsArgs f = rows_args(v, p, ws);
        f.out = gr.dq;
        f.dq_t = gr.dq_stride;
        f.dq_h = gr.dq_head_stride;
        f.lse = const_cast<float*>(lse);
        f.o = out;
        f.dout = dout;
        f.delta = delta;
        e = run_rows(f, p, *a, true, ws, stream);
    }
    if (e == hipSuccess && a->T > 0) {
        sa::ProfScope ps("recent_attn_keys", stream);
        sa::attn::KeysArgs f{v, dout, lse, delta, gr.dK, gr.dV, gr.dk_stride, gr.dk_head_stride, gr.dv_stride,
                             gr.dv_head_stride, sa::attn::key_tiles(a->B, a->T)};
        e = sa::attn::launch_keys(f, bf, a->d, stream);
    }
    if (e != hipSuccess) return hip_fail(e, "recent attention backward launch");
    return SA_OK;
}

}  // extern "C"
