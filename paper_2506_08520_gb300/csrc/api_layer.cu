// C entries of the operators around a language-model layer's attention: argument checks and dispatch.
// Declarations and the full contract are in include/nystra.h.
#include <limits.h>
#include <math.h>

#include <algorithm>
#include <initializer_list>

#include "checks.cuh"
#include "layer.cuh"
#include "nystra.h"

namespace {

using namespace nystra_host;
using nystra::LinArgs;
using nystra::LinRole;
using nystra::Strided;

bool dtype_ok(int dtype) { return dtype == NYSTRA_F32 || dtype == NYSTRA_BF16 || dtype == NYSTRA_F16; }
bool aligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// Sizes of the norm's calls.  Columns, and a partial row's 2 C sums, are indexed with 32 bits.
bool norm_sizes(long long rows, int C) { return rows >= 0 && C >= 0 && C <= NYSTRA_LAYER_NORM_MAX_C; }

// Memory from a tensor's first to behind its last element.
struct Span {
    const void* p;
    size_t bytes;
    bool meets(const Span& o) const { return p && o.p && bytes && o.bytes && overlaps2(p, bytes, o.p, o.bytes); }
};

// A tensor of `axes` strided axes and d adjacent features.
struct Tensor {
    const void* p;
    long long stride[3] = {0, 0, 0};
    long long size[3] = {1, 1, 1};
    int axes, d;
    size_t es;

    Tensor(const void* p_, const long long* s, std::initializer_list<long long> sizes, int d_, size_t es_)
        : p(p_), axes((int)sizes.size()), d(d_), es(es_) {
        int i = 0;
        for (long long z : sizes) {
            size[i] = z;
            stride[i] = s ? s[i] : 0;
            ++i;
        }
    }
    // The furthest element, or -1 where it is out of a 62-bit range or a stride is negative.
    long long last() const {
        __int128 at = d - 1;
        for (int i = 0; i < axes; ++i) {
            if (stride[i] < 0) return -1;
            at += (__int128)(size[i] - 1) * stride[i];
        }
        return at < ((__int128)1 << 60) ? (long long)at : -1;
    }
    bool ok() const { return p && aligned(p, es) && last() >= 0; }
    Span span() const { return {p, (size_t)(last() + 1) * es}; }
    // Every element has a place of its own: with the axes in order of their
    // strides, each steps over all that the smaller ones reach.
    bool apart() const {
        int order[3] = {0, 1, 2};
        std::sort(order, order + axes, [&](int a, int b) { return stride[a] < stride[b]; });
        __int128 reach = d;
        for (int i = 0; i < axes; ++i) {
            const int x = order[i];
            if (size[x] < 2) continue;
            if (stride[x] < reach) return false;
            reach += (__int128)(size[x] - 1) * stride[x];
        }
        return true;
    }
    bool same(const Tensor& o) const {
        if (p != o.p) return false;
        for (int i = 0; i < axes; ++i)
            if (size[i] > 1 && stride[i] != o.stride[i]) return false;
        return true;
    }
    Strided strided() const { return {stride[0], stride[1], stride[2]}; }
};

// Whether two tensors [n, heads, N, d] of one type are known to share no element.  By the axes in the order
// of their strides: what the inner ones reach is an interval of its own in either tensor, and each outer
// axis, which steps alike in both, steps over the two intervals and all that the axes inside it reach.  With
// every axis inside, that is two tensors one behind the other; with the heads inside, slices of a fused
// projection.
bool disjoint(const Tensor& a, const Tensor& b) {
    const __int128 off = ((__int128)(intptr_t)b.p - (intptr_t)a.p) / (long long)a.es;
    long long step[2][3];
    for (int i = 0; i < 3; ++i) {  // an axis of one element steps like the other tensor's
        step[0][i] = a.size[i] > 1 ? a.stride[i] : b.size[i] > 1 ? b.stride[i] : 0;
        step[1][i] = b.size[i] > 1 ? b.stride[i] : step[0][i];
    }
    int order[3] = {0, 1, 2};
    std::sort(order, order + 3, [&](int x, int y) {
        return std::max(step[0][x], step[1][x]) < std::max(step[0][y], step[1][y]);
    });
    for (int inner = 0; inner <= 3; ++inner) {
        __int128 ra = a.d, rb = b.d;
        for (int i = 0; i < inner; ++i) {
            const int x = order[i];
            ra += (__int128)(a.size[x] - 1) * step[0][x];
            rb += (__int128)(b.size[x] - 1) * step[1][x];
        }
        bool ok = off >= ra || -off >= rb;
        __int128 reach = off >= 0 ? std::max(ra, off + rb) : std::max(rb, ra - off);
        for (int i = inner; i < 3; ++i) {
            const int x = order[i];
            const long long most = std::max(a.size[x], b.size[x]);
            if (most < 2) continue;
            ok = ok && step[0][x] == step[1][x] && step[0][x] >= reach;
            reach += (__int128)(most - 1) * step[0][x];
        }
        if (ok) return true;
    }
    return false;
}

Span flat(const void* p, size_t bytes) { return {p, p ? bytes : 0}; }

bool any_meet(const Span& out, std::initializer_list<Span> others) {
    for (const Span& o : others)
        if (out.meets(o)) return true;
    return false;
}

int done(cudaError_t e) { return e == cudaSuccess ? NYSTRA_OK : fail_cuda(e); }

// Sizes of the linear-attention calls.  Units and segments index grids and 32-bit registers.
bool linear_sizes(int n, int heads, int N, int d_k, int d_v) {
    return n >= 0 && heads >= 0 && N >= 0 && N <= NYSTRA_LINEAR_MAX_N && d_k >= 1 && d_k <= NYSTRA_LINEAR_MAX_D &&
           d_v >= 1 && d_v <= NYSTRA_LINEAR_MAX_D && (long long)n * heads <= (1 << 24);
}

LinArgs linear_args(int roles, int n, int heads, int N, int d_k, int d_v, int dtype) {
    LinArgs a{};
    a.roles = roles;
    a.n = n;
    a.heads = heads;
    a.N = N;
    for (int i = 0; i < roles; ++i) {  // transposed states (dq, dk) swap the two
        a.role[i].db = roles == 3 && i < 2 ? d_v : d_k;
        a.role[i].dc = roles == 3 && i < 2 ? d_k : d_v;
    }
    linear_plan(a, dtype);
    return a;
}

// Whether to run in segments: with the workspace, or not at all.
int use_workspace(LinArgs& a, void* workspace, long long bytes) {
    const long long need = linear_workspace_bytes(a);
    if (!workspace) {
        a.segs = 1;
        a.seg_len = a.N;
        return NYSTRA_OK;
    }
    if (bytes < need || !aligned16(workspace)) return NYSTRA_EINVAL;
    a.ws = static_cast<float*>(workspace);
    return NYSTRA_OK;
}

void set_role(LinRole& r, const Tensor& a, const Tensor& b, const Tensor& c, const Tensor& out) {
    r.a = a.p;
    r.b = b.p;
    r.c = c.p;
    r.out = const_cast<void*>(out.p);
    r.sa = a.strided();
    r.sb = b.strided();
    r.sc = c.strided();
    r.so = out.strided();
}

}  // namespace

extern "C" {

int nystra_layer_norm(const void* x, long long x_stride, const void* weight, const void* bias, void* y,
                      long long y_stride, float* mean, float* rstd, long long rows, int C, float eps, int dtype,
                      int w_dtype, void* stream) {
    if (!dtype_ok(dtype) || (w_dtype != NYSTRA_F32 && w_dtype != dtype)) return NYSTRA_EDTYPE;
    if (!norm_sizes(rows, C) || !(eps >= 0.f) || !isfinite(eps)) return NYSTRA_EINVAL;
    if (rows == 0 || C == 0) return NYSTRA_OK;
    const size_t es = elem_size(dtype), ws = elem_size(w_dtype);
    const Tensor tx(x, &x_stride, {rows}, C, es), ty(y, &y_stride, {rows}, C, es);
    if (!tx.ok() || !ty.ok() || !ty.apart()) return NYSTRA_EINVAL;
    if (!aligned(weight, ws) || !aligned(bias, ws) || !aligned(mean, 4) || !aligned(rstd, 4)) return NYSTRA_EINVAL;
    const Span sx = tx.span(), sy = ty.span(), sw = flat(weight, C * ws), sb = flat(bias, C * ws),
               sm = flat(mean, rows * 4), sr = flat(rstd, rows * 4);
    if ((sy.meets(sx) && !ty.same(tx)) || any_meet(sy, {sw, sb, sm, sr}) || any_meet(sm, {sx, sw, sb, sr}) ||
        any_meet(sr, {sx, sw, sb}))
        return NYSTRA_EINVAL;
    if (!device_ok()) return NYSTRA_EDEVICE;
    return done(launch_layer_norm(x, x_stride, weight, bias, y, y_stride, mean, rstd, rows, C, eps, dtype,
                                  w_dtype == NYSTRA_F32, (cudaStream_t)stream));
}

long long nystra_layer_norm_workspace(long long rows, int C) {
    if (!norm_sizes(rows, C)) return NYSTRA_EINVAL;
    return (long long)layer_norm_parts(rows, C) * 2 * C * 4;
}

int nystra_layer_norm_backward(const void* dy, long long dy_stride, const void* x, long long x_stride,
                               const float* mean, const float* rstd, const void* weight, void* dx, long long dx_stride,
                               void* dweight, void* dbias, long long rows, int C, int dtype, int w_dtype,
                               void* workspace, long long workspace_bytes, void* stream) {
    if (!dtype_ok(dtype) || (w_dtype != NYSTRA_F32 && w_dtype != dtype)) return NYSTRA_EDTYPE;
    if (!norm_sizes(rows, C)) return NYSTRA_EINVAL;
    if (C == 0) return NYSTRA_OK;
    const size_t es = elem_size(dtype), ws = elem_size(w_dtype);
    if (!aligned(weight, ws) || !aligned(dweight, ws) || !aligned(dbias, ws)) return NYSTRA_EINVAL;
    const bool wanted = dweight || dbias;
    if (rows == 0 && !wanted) return NYSTRA_OK;
    const long long need = wanted ? nystra_layer_norm_workspace(rows, C) : 0;
    if (wanted && (!workspace || !aligned16(workspace) || workspace_bytes < need)) return NYSTRA_EINVAL;
    const Span sw = flat(weight, C * ws), gw = flat(dweight, C * ws), gb = flat(dbias, C * ws),
               sp = flat(wanted ? workspace : nullptr, (size_t)need);
    if (any_meet(gw, {sw, gb, sp}) || any_meet(gb, {sw, sp}) || any_meet(sp, {sw})) return NYSTRA_EINVAL;
    if (rows > 0) {
        const Tensor td(dy, &dy_stride, {rows}, C, es), tx(x, &x_stride, {rows}, C, es), to(dx, &dx_stride, {rows}, C, es);
        if (!td.ok() || !tx.ok() || !to.ok() || !to.apart()) return NYSTRA_EINVAL;
        if (!mean || !rstd || !aligned(mean, 4) || !aligned(rstd, 4)) return NYSTRA_EINVAL;
        const Span sd = td.span(), sx = tx.span(), so = to.span(), sm = flat(mean, rows * 4), sr = flat(rstd, rows * 4);
        if ((so.meets(sd) && !to.same(td)) || (so.meets(sx) && !to.same(tx)) || any_meet(so, {sw, gw, gb, sp, sm, sr}))
            return NYSTRA_EINVAL;
        for (const Span& o : {gw, gb, sp})
            if (any_meet(o, {sd, sx, sm, sr})) return NYSTRA_EINVAL;
    }
    if (!device_ok()) return NYSTRA_EDEVICE;
    return done(launch_layer_norm_backward(dy, dy_stride, x, x_stride, mean, rstd, weight, dx, dx_stride, dweight,
                                           dbias, rows, C, dtype, w_dtype == NYSTRA_F32,
                                           static_cast<float*>(workspace), (cudaStream_t)stream));
}

int nystra_rotary(const void* q, const long long* q_strides, void* q_out, const long long* q_out_strides, int q_heads,
                  const void* k, const long long* k_strides, void* k_out, const long long* k_out_strides, int k_heads,
                  const double* inv_freq, int rotary_dim, const void* positions, int positions_bits,
                  long long positions_stride, float amplitude, int n, int N, int d, int layout, int inverse, int dtype,
                  void* stream) {
    if (!dtype_ok(dtype)) return NYSTRA_EDTYPE;
    if (n < 0 || N < 0 || q_heads < 0 || k_heads < 0 || d < 1 || d > NYSTRA_ROTARY_MAX_D) return NYSTRA_EINVAL;
    if (rotary_dim < 0 || rotary_dim > d || rotary_dim % 2 != 0) return NYSTRA_EINVAL;
    if (layout != NYSTRA_ROTARY_HALF && layout != NYSTRA_ROTARY_INTERLEAVED) return NYSTRA_EINVAL;
    if ((inverse != 0 && inverse != 1) || !isfinite(amplitude)) return NYSTRA_EINVAL;
    if (q_heads > 1 << 16 || k_heads > 1 << 16) return NYSTRA_EINVAL;
    if (n == 0 || N == 0 || q_heads + k_heads == 0) return NYSTRA_OK;
    if (rotary_dim > 0 && (!inv_freq || !aligned(inv_freq, 8))) return NYSTRA_EINVAL;
    if (positions && ((positions_bits != 32 && positions_bits != 64) || !aligned(positions, positions_bits / 8) ||
                      positions_stride < 0))
        return NYSTRA_EINVAL;
    const size_t es = elem_size(dtype);
    const Tensor x[2] = {Tensor(q, q_strides, {n, q_heads, N}, d, es), Tensor(k, k_strides, {n, k_heads, N}, d, es)};
    const Tensor y[2] = {Tensor(q_out, q_out_strides, {n, q_heads, N}, d, es),
                         Tensor(k_out, k_out_strides, {n, k_heads, N}, d, es)};
    const int heads[2] = {q_heads, k_heads};
    const long long* const strides[4] = {q_strides, q_out_strides, k_strides, k_out_strides};
    const Span table = flat(inv_freq, (size_t)rotary_dim / 2 * 8);
    Span pos = flat(nullptr, 0);
    if (positions) {
        const Tensor t(positions, &positions_stride, {n}, N, (size_t)positions_bits / 8);
        if (t.last() < 0) return NYSTRA_EINVAL;
        pos = t.span();
    }
    bool in_place[2] = {false, false};
    for (int i = 0; i < 2; ++i) {
        if (heads[i] == 0) continue;
        if (!strides[2 * i] || !strides[2 * i + 1]) return NYSTRA_EINVAL;
        if (!x[i].ok() || !y[i].ok() || !y[i].apart()) return NYSTRA_EINVAL;
        in_place[i] = y[i].same(x[i]);
        const Span s = y[i].span();
        if ((!in_place[i] && s.meets(x[i].span())) || any_meet(s, {table, pos})) return NYSTRA_EINVAL;
    }
    if (q_heads && k_heads) {  // in place, q and k may be interleaved slices of one buffer
        if ((in_place[0] || in_place[1]) && !disjoint(x[0], x[1])) return NYSTRA_EINVAL;
        if (!(in_place[0] && in_place[1]) && y[0].span().meets(y[1].span())) return NYSTRA_EINVAL;
        if (!in_place[0] && y[0].span().meets(x[1].span())) return NYSTRA_EINVAL;
        if (!in_place[1] && y[1].span().meets(x[0].span())) return NYSTRA_EINVAL;
    }
    if (!device_ok()) return NYSTRA_EDEVICE;
    RotaryTensor t[2];
    for (int i = 0; i < 2; ++i)
        t[i] = {x[i].p, const_cast<void*>(y[i].p), x[i].strided(), y[i].strided(), heads[i]};
    return done(launch_rotary(t[0], t[1], inv_freq, rotary_dim, positions, positions_bits == 32, positions_stride,
                              amplitude, n, N, d, layout, inverse != 0, dtype, (cudaStream_t)stream));
}

long long nystra_linear_attention_workspace(int n, int heads, int N, int d_k, int d_v, int dtype, int backward) {
    if (!linear_sizes(n, heads, N, d_k, d_v) || !dtype_ok(dtype)) return NYSTRA_EINVAL;
    if ((long long)n * heads == 0 || N == 0) return 0;
    return linear_workspace_bytes(linear_args(backward ? 3 : 1, n, heads, N, d_k, d_v, dtype));
}

int nystra_linear_attention(const void* q, const long long* q_strides, const void* k, const long long* k_strides,
                            const void* v, const long long* v_strides, void* out, const long long* out_strides,
                            const float* log_decay, const int* lengths, const float* state_in, float* state_out,
                            float scale, int n, int heads, int N, int d_k, int d_v, int dtype, void* workspace,
                            long long workspace_bytes, void* stream) {
    if (!dtype_ok(dtype)) return NYSTRA_EDTYPE;
    if (!linear_sizes(n, heads, N, d_k, d_v) || !isfinite(scale)) return NYSTRA_EINVAL;
    const long long units = (long long)n * heads;
    if (units == 0 || (N == 0 && !state_out)) return NYSTRA_OK;
    const size_t es = elem_size(dtype), state_bytes = (size_t)units * d_k * d_v * 4;
    if (!log_decay || !aligned(log_decay, 4) || !aligned(lengths, 4) || !aligned(state_in, 4) || !aligned(state_out, 4))
        return NYSTRA_EINVAL;
    const Tensor tq(q, q_strides, {n, heads, N}, d_k, es), tk(k, k_strides, {n, heads, N}, d_k, es),
        tv(v, v_strides, {n, heads, N}, d_v, es), to(out, out_strides, {n, heads, N}, d_v, es);
    LinArgs a = linear_args(1, n, heads, N, d_k, d_v, dtype);
    const int rc = use_workspace(a, workspace, workspace_bytes);
    if (rc != NYSTRA_OK) return rc;
    const Span si = flat(state_in, state_bytes), so = flat(state_out, state_bytes), sl = flat(log_decay, heads * 4),
               sn = flat(lengths, n * 4), sp = flat(workspace, a.segs > 1 ? (size_t)linear_workspace_bytes(a) : 0);
    if ((so.meets(si) && state_out != state_in) || any_meet(so, {sl, sn, sp}) || any_meet(sp, {si, sl, sn}))
        return NYSTRA_EINVAL;
    if (N > 0) {
        if (!q_strides || !k_strides || !v_strides || !out_strides) return NYSTRA_EINVAL;
        if (!tq.ok() || !tk.ok() || !tv.ok() || !to.ok() || !to.apart()) return NYSTRA_EINVAL;
        const Span s = to.span();
        if (any_meet(s, {tq.span(), tk.span(), tv.span(), si, so, sl, sn, sp})) return NYSTRA_EINVAL;
        for (const Span& o : {so, sp})
            if (any_meet(o, {tq.span(), tk.span(), tv.span()})) return NYSTRA_EINVAL;
    }
    if (!device_ok()) return NYSTRA_EDEVICE;
    a.log_decay = log_decay;
    a.lengths = lengths;
    LinRole& r = a.role[0];
    set_role(r, tq, tk, tv, to);
    r.s_in = state_in;
    r.s_out = state_out;
    r.s_scale = 1.f;
    r.o_scale = scale;
    return done(launch_linear(a, dtype, (cudaStream_t)stream));
}

int nystra_linear_attention_backward(const void* dout, const long long* dout_strides, const void* q,
                                     const long long* q_strides, const void* k, const long long* k_strides,
                                     const void* v, const long long* v_strides, const float* log_decay,
                                     const int* lengths, const float* state_in, const float* dstate_out, void* dq,
                                     const long long* dq_strides, void* dk, const long long* dk_strides, void* dv,
                                     const long long* dv_strides, float* dstate_in, float scale, int n, int heads,
                                     int N, int d_k, int d_v, int dtype, void* workspace, long long workspace_bytes,
                                     void* stream) {
    if (!dtype_ok(dtype)) return NYSTRA_EDTYPE;
    if (!linear_sizes(n, heads, N, d_k, d_v) || !isfinite(scale)) return NYSTRA_EINVAL;
    const long long units = (long long)n * heads;
    if (units == 0 || (N == 0 && !dstate_in)) return NYSTRA_OK;
    const size_t es = elem_size(dtype), state_bytes = (size_t)units * d_k * d_v * 4;
    if (!log_decay || !aligned(log_decay, 4) || !aligned(lengths, 4)) return NYSTRA_EINVAL;
    if (!aligned(state_in, 4) || !aligned(dstate_out, 4) || !aligned(dstate_in, 4)) return NYSTRA_EINVAL;
    const Tensor in[4] = {Tensor(dout, dout_strides, {n, heads, N}, d_v, es), Tensor(q, q_strides, {n, heads, N}, d_k, es),
                          Tensor(k, k_strides, {n, heads, N}, d_k, es), Tensor(v, v_strides, {n, heads, N}, d_v, es)};
    const Tensor out[3] = {Tensor(dq, dq_strides, {n, heads, N}, d_k, es), Tensor(dk, dk_strides, {n, heads, N}, d_k, es),
                           Tensor(dv, dv_strides, {n, heads, N}, d_v, es)};
    LinArgs a = linear_args(3, n, heads, N, d_k, d_v, dtype);
    const int rc = use_workspace(a, workspace, workspace_bytes);
    if (rc != NYSTRA_OK) return rc;
    const Span si = flat(state_in, state_bytes), sd = flat(dstate_out, state_bytes), so = flat(dstate_in, state_bytes),
               sl = flat(log_decay, heads * 4), sn = flat(lengths, n * 4),
               sp = flat(workspace, a.segs > 1 ? (size_t)linear_workspace_bytes(a) : 0);
    // dk also starts from dstate_out, so dv's pass must not write dstate_in over it.
    if (any_meet(so, {si, sd, sl, sn, sp}) || any_meet(sp, {si, sd, sl, sn})) return NYSTRA_EINVAL;
    if (N > 0) {
        for (const long long* s : {dout_strides, q_strides, k_strides, v_strides, dq_strides, dk_strides, dv_strides})
            if (!s) return NYSTRA_EINVAL;
        for (const Tensor& t : in)
            if (!t.ok() || so.meets(t.span()) || sp.meets(t.span())) return NYSTRA_EINVAL;
        for (int i = 0; i < 3; ++i) {
            if (!out[i].ok() || !out[i].apart()) return NYSTRA_EINVAL;
            const Span s = out[i].span();
            for (const Tensor& t : in)
                if (s.meets(t.span())) return NYSTRA_EINVAL;
            for (int j = 0; j < i; ++j)
                if (s.meets(out[j].span())) return NYSTRA_EINVAL;
            if (any_meet(s, {si, sd, so, sl, sn, sp})) return NYSTRA_EINVAL;
        }
    }
    if (!device_ok()) return NYSTRA_EDEVICE;
    a.log_decay = log_decay;
    a.lengths = lengths;
    const Tensor &tdo = in[0], &tq = in[1], &tk = in[2], &tv = in[3];
    LinRole& rq = a.role[0];
    set_role(rq, tdo, tv, tk, out[0]);
    rq.s_in = state_in;
    rq.transposed = 1;
    rq.s_scale = 1.f;
    rq.o_scale = scale;
    LinRole& rk = a.role[1];
    set_role(rk, tv, tdo, tq, out[1]);
    rk.s_in = dstate_out;
    rk.transposed = 1;
    rk.backward = 1;
    rk.s_scale = scale;
    rk.o_scale = 1.f;
    LinRole& rv = a.role[2];
    set_role(rv, tk, tq, tdo, out[2]);
    rv.s_in = dstate_out;
    rv.s_out = dstate_in;
    rv.backward = 1;
    rv.s_scale = scale;
    rv.o_scale = 1.f;
    return done(launch_linear(a, dtype, (cudaStream_t)stream));
}

int nystra_linear_attention_step(const void* q, const long long* q_strides, const void* k, const long long* k_strides,
                                 const void* v, const long long* v_strides, void* out, const long long* out_strides,
                                 const float* log_decay, const float* state_in, float* state_out, float scale, int n,
                                 int heads, int d_k, int d_v, int dtype, void* stream) {
    if (!dtype_ok(dtype)) return NYSTRA_EDTYPE;
    if (!linear_sizes(n, heads, 1, d_k, d_v) || !isfinite(scale)) return NYSTRA_EINVAL;
    const long long units = (long long)n * heads;
    if (units == 0) return NYSTRA_OK;
    if (!q_strides || !k_strides || !v_strides || !out_strides) return NYSTRA_EINVAL;
    const size_t es = elem_size(dtype), state_bytes = (size_t)units * d_k * d_v * 4;
    const Tensor tq(q, q_strides, {n, heads}, d_k, es), tk(k, k_strides, {n, heads}, d_k, es),
        tv(v, v_strides, {n, heads}, d_v, es), to(out, out_strides, {n, heads}, d_v, es);
    if (!tq.ok() || !tk.ok() || !tv.ok() || !to.ok() || !to.apart()) return NYSTRA_EINVAL;
    if (!log_decay || !state_out || !aligned(log_decay, 4) || !aligned(state_in, 4) || !aligned(state_out, 4))
        return NYSTRA_EINVAL;
    const Span s = to.span(), si = flat(state_in, state_bytes), so = flat(state_out, state_bytes),
               sl = flat(log_decay, heads * 4);
    if ((so.meets(si) && state_out != state_in) || any_meet(s, {tq.span(), tk.span(), tv.span(), si, so, sl}) ||
        any_meet(so, {tq.span(), tk.span(), tv.span(), sl}))
        return NYSTRA_EINVAL;
    if (!device_ok()) return NYSTRA_EDEVICE;
    return done(launch_linear_step(q, q_strides, k, k_strides, v, v_strides, out, out_strides, log_decay, state_in,
                                   state_out, scale, n, heads, d_k, d_v, dtype, (cudaStream_t)stream));
}

}  // extern "C"
