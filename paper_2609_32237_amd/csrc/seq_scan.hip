// seq_scan.hip -- the gated linear recurrence h += q (c - h) along the tokens,
// q = rate s(r), c = s(g) x, and its gradient.
#include <hip/hip_runtime.h>

#include "seq_device.hpp"
#include "seq_host.hpp"

namespace mi355seq {
namespace {

constexpr int kChunk = SEQ_SCAN_CHUNK;

struct ScanArgs {
    int64_t batch, len, channels;
    const void *x, *r, *g, *dy;
    void *y, *dx, *dr, *dg;
    int64_t xb, xt, rb, rt, gb, gt, yb, yt, dyb, dyt, dxb, dxt, drb, drt, dgb, dgt;
    const float *rate, *state, *dstate_out;
    const int32_t *lengths;
    float *state_out, *saved, *dstate, *drate, *partial;
};

__device__ __forceinline__ int64_t valid_tokens(const ScanArgs &a, int64_t b) {
    if (!a.lengths) return a.len;
    const int64_t n = a.lengths[b];
    return n < 0 ? 0 : n > a.len ? a.len : n;
}

// One thread per sequence and channel, token after token.
template <typename E>
__global__ void __launch_bounds__(256) scan_forward(ScanArgs a) {
    using T = typename E::T;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= a.batch * a.channels) return;
    const int64_t b = i / a.channels, d = i % a.channels, n = valid_tokens(a, b);
    const int64_t chunks = (a.len + kChunk - 1) / kChunk;
    const T *x = (const T *)a.x + b * a.xb + d, *r = (const T *)a.r + b * a.rb + d, *g = (const T *)a.g + b * a.gb + d;
    T *y = (T *)a.y + b * a.yb + d;
    const float rate = a.rate[d];
    float h = a.state ? a.state[i] : 0.0f;
    for (int64_t t = 0; t < a.len; ++t) {
        if (a.saved && t % kChunk == 0) a.saved[(b * chunks + t / kChunk) * a.channels + d] = h;
        float out = 0.0f;
        if (t < n) {
            const float q = rate * sigmoid(E::to_f(r[t * a.rt]));
            const float c = sigmoid(E::to_f(g[t * a.gt])) * E::to_f(x[t * a.xt]);
            h = fmaf(q, c - h, h);
            out = h;
        }
        y[t * a.yt] = E::of_f(out);
    }
    if (a.state_out) a.state_out[i] = h;
}

// One thread per sequence and channel, chunk after chunk from the last; the
// states of a chunk are computed again from the saved one.
template <typename E>
__global__ void __launch_bounds__(256) scan_backward(ScanArgs a) {
    using T = typename E::T;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= a.batch * a.channels) return;
    const int64_t b = i / a.channels, d = i % a.channels, n = valid_tokens(a, b);
    const int64_t chunks = (a.len + kChunk - 1) / kChunk;
    const T *x = (const T *)a.x + b * a.xb + d, *r = (const T *)a.r + b * a.rb + d, *g = (const T *)a.g + b * a.gb + d;
    const T *dy = (const T *)a.dy + b * a.dyb + d;
    T *dx = (T *)a.dx + b * a.dxb + d, *dr = (T *)a.dr + b * a.drb + d, *dg = (T *)a.dg + b * a.dgb + d;
    const float rate = a.rate[d];
    float k = a.dstate_out ? a.dstate_out[i] : 0.0f, drate = 0.0f;
    for (int64_t j = chunks - 1; j >= 0; --j) {
        float h[kChunk + 1];
        h[0] = a.saved[(b * chunks + j) * a.channels + d];
#pragma unroll
        for (int s = 0; s < kChunk; ++s) {
            const int64_t t = j * kChunk + s;
            h[s + 1] = h[s];
            if (t < n) {
                const float q = rate * sigmoid(E::to_f(r[t * a.rt]));
                const float c = sigmoid(E::to_f(g[t * a.gt])) * E::to_f(x[t * a.xt]);
                h[s + 1] = fmaf(q, c - h[s], h[s]);
            }
        }
#pragma unroll
        for (int s = kChunk - 1; s >= 0; --s) {
            const int64_t t = j * kChunk + s;
            if (t < a.len) {
                float ox = 0.0f, orr = 0.0f, og = 0.0f;
                if (t < n) {
                    const float sr = sigmoid(E::to_f(r[t * a.rt])), sg = sigmoid(E::to_f(g[t * a.gt]));
                    const float xv = E::to_f(x[t * a.xt]), q = rate * sr;
                    const float dh = E::to_f(dy[t * a.dyt]) + k;
                    const float e = dh * (sg * xv - h[s]);
                    drate = fmaf(e, sr, drate);
                    orr = e * q * (1.0f - sr);
                    ox = dh * q * sg;
                    og = ox * xv * (1.0f - sg);
                    k = fmaf(-q, dh, dh);
                }
                dx[t * a.dxt] = E::of_f(ox);
                dr[t * a.drt] = E::of_f(orr);
                dg[t * a.dgt] = E::of_f(og);
            }
        }
    }
    if (a.dstate) a.dstate[i] = k;
    a.partial[i] = drate;
}

// drate of a channel: the partial sums in their order.
__global__ void __launch_bounds__(256) scan_sum_rate(const float *partial, int64_t rows, int64_t channels, float *drate) {
    const int64_t d = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (d >= channels) return;
    float s = 0.0f;
    for (int64_t k = 0; k < rows; ++k) s += partial[k * channels + d];
    drate[d] = s;
}

bool sizes_ok(int64_t batch, int64_t len, int64_t channels) { return batch >= 0 && len >= 0 && channels >= 1; }
bool sizes_supported(int64_t batch, int64_t len, int64_t channels) {
    if (batch > kMaxSize || len > kMaxSize || channels > kMaxSize) return false;
    const __int128 n = (__int128)batch * (len > 0 ? len : 1) * channels;
    return n <= kMaxElements && ceil_div(batch * channels, 256) <= kMaxSize;
}

const void *forward_kernel(int type) {
    return type == SEQ_FP32 ? (const void *)scan_forward<F32>
                            : type == SEQ_FP16 ? (const void *)scan_forward<F16> : (const void *)scan_forward<BF16>;
}
const void *backward_kernel(int type) {
    return type == SEQ_FP32 ? (const void *)scan_backward<F32>
                            : type == SEQ_FP16 ? (const void *)scan_backward<F16> : (const void *)scan_backward<BF16>;
}

}  // namespace
}  // namespace mi355seq

using namespace mi355seq;

extern "C" {

size_t seq_scan_saved_bytes(int64_t batch, int64_t len, int64_t channels) {
    if (!sizes_ok(batch, len, channels) || !sizes_supported(batch, len, channels)) return 0;
    return (size_t)(batch * ceil_div(len, kChunk) * channels) * sizeof(float);
}

size_t seq_scan_workspace_bytes(int64_t batch, int64_t len, int64_t channels, int type, int backward) {
    if (!sizes_ok(batch, len, channels) || !sizes_supported(batch, len, channels) || !known_type(type)) return 0;
    return backward ? up16((size_t)(batch * channels) * sizeof(float)) : 0;
}

int seq_scan_forward(int64_t batch, int64_t len, int64_t channels, int type, const void *x, const void *r,
                     const void *g, const int64_t *strides, const float *rate, const float *state,
                     const int32_t *lengths, void *y, float *state_out, float *saved, void *workspace,
                     hipStream_t stream) {
    if (!sizes_ok(batch, len, channels) || !known_type(type)) return SEQ_EINVAL;
    if (!sizes_supported(batch, len, channels)) return SEQ_EUNSUPPORTED;
    const int64_t elements = batch * len * channels, states = batch * channels;
    if (states == 0) return SEQ_OK;
    if (!rate || (elements && (!x || !r || !g || !y))) return SEQ_EINVAL;
    const Grid grid{batch, len, channels, element_bytes(type)};
    Rows in[3] = {{x, 0, 0}, {r, 0, 0}, {g, 0, 0}}, out{y, 0, 0};
    for (int i = 0; i < 3; ++i) {
        in[i].so = strides ? strides[2 * i] : len * channels;
        in[i].si = strides ? strides[2 * i + 1] : channels;
    }
    out.so = strides ? strides[6] : len * channels;
    out.si = strides ? strides[7] : channels;
    for (const Rows &v : in)
        if (!strides_in_range(v)) return SEQ_EINVAL;
    if (!strides_in_range(out)) return SEQ_EINVAL;
    for (const void *p : {x, r, g, (const void *)y})
        if (misaligned(p, grid.bytes)) return SEQ_EALIGN;
    for (const void *p : {(const void *)rate, (const void *)state, (const void *)lengths, (const void *)state_out, (const void *)saved})
        if (misaligned(p, 4)) return SEQ_EALIGN;
    if (elements) {
        if (!rows_apart(out, grid)) return SEQ_EINVAL;
        for (const Rows &v : in)
            if (!same_rows(v, out, grid) && may_share(v, out, grid)) return SEQ_EINVAL;
    }
    const size_t state_bytes = (size_t)states * 4, saved_bytes = seq_scan_saved_bytes(batch, len, channels);
    if (state_out != state && ranges_share(state, state_bytes, state_out, state_bytes)) return SEQ_EINVAL;
    if (ranges_share(saved, saved_bytes, state, state_bytes) || ranges_share(saved, saved_bytes, state_out, state_bytes))
        return SEQ_EINVAL;
    const size_t need = seq_scan_workspace_bytes(batch, len, channels, type, 0);
    if (need && !workspace) return SEQ_EINVAL;
    if (misaligned(workspace, 16)) return SEQ_EALIGN;

    ScanArgs a{};
    a.batch = batch, a.len = len, a.channels = channels;
    a.x = x, a.r = r, a.g = g, a.y = y;
    a.xb = in[0].so, a.xt = in[0].si, a.rb = in[1].so, a.rt = in[1].si, a.gb = in[2].so, a.gt = in[2].si;
    a.yb = out.so, a.yt = out.si;
    a.rate = rate, a.state = state, a.lengths = lengths, a.state_out = state_out, a.saved = saved;
    void *args[] = {&a};
    return launch(forward_kernel(type), dim3((unsigned)ceil_div(states, 256)), dim3(256), args, 0, stream);
}

int seq_scan_backward(int64_t batch, int64_t len, int64_t channels, int type, const void *dy, const void *x,
                      const void *r, const void *g, const int64_t *strides, const float *rate, const float *saved,
                      const int32_t *lengths, const float *dstate_out, void *dx, void *dr, void *dg, float *drate,
                      float *dstate, void *workspace, hipStream_t stream) {
    if (!sizes_ok(batch, len, channels) || !known_type(type)) return SEQ_EINVAL;
    if (!sizes_supported(batch, len, channels)) return SEQ_EUNSUPPORTED;
    const int64_t elements = batch * len * channels, states = batch * channels;
    if (!rate || !drate || (elements && (!dy || !x || !r || !g || !dx || !dr || !dg || !saved))) return SEQ_EINVAL;
    const Grid grid{batch, len, channels, element_bytes(type)};
    Rows v[7] = {{dy, 0, 0}, {x, 0, 0}, {r, 0, 0}, {g, 0, 0}, {dx, 0, 0}, {dr, 0, 0}, {dg, 0, 0}};
    for (int i = 0; i < 7; ++i) {
        v[i].so = strides ? strides[2 * i] : len * channels;
        v[i].si = strides ? strides[2 * i + 1] : channels;
        if (!strides_in_range(v[i])) return SEQ_EINVAL;
    }
    for (const Rows &w : v)
        if (misaligned(w.p, grid.bytes)) return SEQ_EALIGN;
    for (const void *p : {(const void *)rate, (const void *)saved, (const void *)lengths, (const void *)dstate_out, (const void *)drate, (const void *)dstate})
        if (misaligned(p, 4)) return SEQ_EALIGN;
    if (elements) {
        for (int i = 4; i < 7; ++i) {
            if (!rows_apart(v[i], grid)) return SEQ_EINVAL;
            for (int j = 0; j < i; ++j) {
                const bool own = (i == 4 && j == 0) || (i == 5 && j == 2) || (i == 6 && j == 3);
                if (own && same_rows(v[i], v[j], grid)) continue;
                if (may_share(v[i], v[j], grid)) return SEQ_EINVAL;
            }
        }
    }
    const size_t state_bytes = (size_t)states * 4;
    if (dstate != dstate_out && ranges_share(dstate, state_bytes, dstate_out, state_bytes)) return SEQ_EINVAL;
    if (ranges_share(drate, (size_t)channels * 4, rate, (size_t)channels * 4)) return SEQ_EINVAL;
    const size_t need = seq_scan_workspace_bytes(batch, len, channels, type, 1);
    if (need && !workspace) return SEQ_EINVAL;
    if (misaligned(workspace, 16)) return SEQ_EALIGN;

    ScanArgs a{};
    a.batch = batch, a.len = len, a.channels = channels;
    a.dy = dy, a.x = x, a.r = r, a.g = g, a.dx = dx, a.dr = dr, a.dg = dg;
    a.dyb = v[0].so, a.dyt = v[0].si, a.xb = v[1].so, a.xt = v[1].si, a.rb = v[2].so, a.rt = v[2].si;
    a.gb = v[3].so, a.gt = v[3].si, a.dxb = v[4].so, a.dxt = v[4].si, a.drb = v[5].so, a.drt = v[5].si;
    a.dgb = v[6].so, a.dgt = v[6].si;
    a.rate = rate, a.saved = const_cast<float *>(saved), a.lengths = lengths, a.dstate_out = dstate_out;
    a.drate = drate, a.dstate = dstate, a.partial = (float *)workspace;
    if (states) {
        void *args[] = {&a};
        const int rc = launch(backward_kernel(type), dim3((unsigned)ceil_div(states, 256)), dim3(256), args, 0, stream);
        if (rc != SEQ_OK) return rc;
    }
    const float *partial = a.partial;
    void *args[] = {&partial, &batch, &channels, &drate};
    return launch((const void *)scan_sum_rate, dim3((unsigned)ceil_div(channels, 256)), dim3(256), args, 0, stream);
}

const char *seq_strerror(int code) {
    switch (code) {
        case SEQ_OK: return "success";
        case SEQ_EINVAL: return "invalid argument";
        case SEQ_EUNSUPPORTED: return "size not supported";
        case SEQ_EALIGN: return "pointer not aligned";
        case SEQ_EHIP: return "HIP runtime error";
        default: return "unknown error code";
    }
}

}  // extern "C"
