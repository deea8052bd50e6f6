// seq_norm.hip -- the norms before and after a block with its gate and scaled
// residual, and their gradient.
#include <hip/hip_runtime.h>

#include "seq_device.hpp"
#include "seq_host.hpp"

namespace mi355seq {
namespace {

constexpr int kThreads = 256;
constexpr int64_t kMaxChannels = 65536;
constexpr int kRowGroups = 64;  // partial sums of each column

struct NormArgs {
    int64_t rows;
    int channels;
    float eps, inv_channels;
    const void *x, *y, *z, *dout, *dnormed;
    void *out, *normed, *dx, *dy, *dz;
    int64_t xs, ys, zs, outs, normeds, douts, dnormeds, dxs, dys, dzs;
    const float *post, *scale, *pre;
    float *stats, *mean, *partial, *dpost, *dscale, *dpre;
};

__device__ __forceinline__ float block_sum(float v) {
    __shared__ float part[kThreads / kWave];
#pragma unroll
    for (int m = kWave / 2; m > 0; m /= 2) v += __shfl_xor(v, m);
    __syncthreads();
    if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = v;
    __syncthreads();
    float s = 0.0f;
    for (int w = 0; w < kThreads / kWave; ++w) s += part[w];
    return s;
}

// scale * post of one channel
__device__ __forceinline__ float weight(const NormArgs &a, int d) { return a.post[d] * (a.scale ? a.scale[d] : 1.0f); }

// v - vh mean(v vh) of a row vh of norm 1 - eps i^2: with one channel it is
// v eps i^2, of which the difference of two FP32 values would leave nothing.
// So there the factor is that and the mean is 0.
__device__ __forceinline__ float one_channel(const NormArgs &a, float i) { return a.channels == 1 ? a.eps * i * i : 1.0f; }

template <typename E>
struct Row {
    using T = typename E::T;
    const NormArgs &a;
    int64_t row;
    __device__ float at(const void *p, int64_t stride, int d) const { return E::to_f(((const T *)p)[row * stride + d]); }
    __device__ void put(void *p, int64_t stride, int d, float v) const { ((T *)p)[row * stride + d] = E::of_f(v); }
    __device__ float gate(int d, float *slope) const {
        if (!a.z) {
            *slope = 0.0f;
            return 1.0f;
        }
        const float z = at(a.z, a.zs, d), s = sigmoid(z), g = z * s;
        *slope = fmaf(g, 1.0f - s, s);
        return g;
    }
    __device__ float o(int d, float iy) const {
        float v = at(a.x, a.xs, d), slope;
        if (a.y) v = fmaf(weight(a, d) * gate(d, &slope), at(a.y, a.ys, d) * iy, v);
        return v;
    }
    // the gradient that reaches o
    __device__ float t(int d, float iy, float io, float mean) const {
        float v = a.dout ? at(a.dout, a.douts, d) : 0.0f;
        if (a.pre) v += io * (at(a.dnormed, a.dnormeds, d) * a.pre[d] * one_channel(a, io) - o(d, iy) * io * mean);
        return v;
    }
};

template <typename E>
__global__ void __launch_bounds__(kThreads) norm_forward(NormArgs a) {
    const Row<E> row{a, blockIdx.x};
    float iy = 0.0f, io = 0.0f;
    if (a.y) {
        float s = 0.0f;
        for (int d = threadIdx.x; d < a.channels; d += kThreads) {
            const float v = row.at(a.y, a.ys, d);
            s = fmaf(v, v, s);
        }
        iy = 1.0f / sqrtf(fmaf(block_sum(s), a.inv_channels, a.eps));
    }
    if (a.pre) {
        float s = 0.0f;
        for (int d = threadIdx.x; d < a.channels; d += kThreads) {
            const float v = row.o(d, iy);
            s = fmaf(v, v, s);
        }
        io = 1.0f / sqrtf(fmaf(block_sum(s), a.inv_channels, a.eps));
    }
    for (int d = threadIdx.x; d < a.channels; d += kThreads) {
        const float o = row.o(d, iy);
        if (a.out) row.put(a.out, a.outs, d, o);
        if (a.pre) row.put(a.normed, a.normeds, d, o * io * a.pre[d]);
    }
    if (a.stats && threadIdx.x < 2) a.stats[2 * row.row + threadIdx.x] = threadIdx.x ? io : iy;
}

// mean(v oh) of each row
template <typename E>
__global__ void __launch_bounds__(kThreads) norm_row_mean(NormArgs a) {
    const Row<E> row{a, blockIdx.x};
    const float iy = a.stats[2 * row.row], io = a.stats[2 * row.row + 1];
    float s = 0.0f;
    for (int d = threadIdx.x; d < a.channels; d += kThreads)
        s = fmaf(row.at(a.dnormed, a.dnormeds, d) * a.pre[d], row.o(d, iy) * io, s);
    s = block_sum(s);
    if (threadIdx.x == 0) a.mean[row.row] = a.channels == 1 ? 0.0f : s * a.inv_channels;
}

// partial sums of the weights' gradients over a group of rows
template <typename E>
__global__ void __launch_bounds__(kThreads) norm_columns(NormArgs a) {
    const int d = blockIdx.x * kThreads + threadIdx.x;
    if (d >= a.channels) return;
    float p = 0.0f, dpre = 0.0f;
    for (int64_t k = blockIdx.y; k < a.rows; k += gridDim.y) {
        const Row<E> row{a, k};
        const float iy = a.stats[2 * k], io = a.stats[2 * k + 1];
        float slope;
        if (a.y) p = fmaf(row.t(d, iy, io, a.pre ? a.mean[k] : 0.0f) * row.gate(d, &slope), row.at(a.y, a.ys, d) * iy, p);
        if (a.pre) dpre = fmaf(row.at(a.dnormed, a.dnormeds, d), row.o(d, iy) * io, dpre);
    }
    a.partial[(2 * (int64_t)blockIdx.y) * a.channels + d] = p;
    a.partial[(2 * (int64_t)blockIdx.y + 1) * a.channels + d] = dpre;
}

__global__ void __launch_bounds__(kThreads) norm_sum_columns(NormArgs a, int groups) {
    const int d = blockIdx.x * kThreads + threadIdx.x;
    if (d >= a.channels) return;
    float p = 0.0f, dpre = 0.0f;
    for (int k = 0; k < groups; ++k) {
        p += a.partial[(2 * (int64_t)k) * a.channels + d];
        dpre += a.partial[(2 * (int64_t)k + 1) * a.channels + d];
    }
    if (a.dpost) a.dpost[d] = p * (a.scale ? a.scale[d] : 1.0f);
    if (a.dscale) a.dscale[d] = p * a.post[d];
    if (a.dpre) a.dpre[d] = dpre;
}

template <typename E>
__global__ void __launch_bounds__(kThreads) norm_backward(NormArgs a) {
    const Row<E> row{a, blockIdx.x};
    const float iy = a.stats[2 * row.row], io = a.stats[2 * row.row + 1], mean = a.pre ? a.mean[row.row] : 0.0f;
    float s = 0.0f, slope;
    if (a.y) {
        for (int d = threadIdx.x; d < a.channels; d += kThreads)
            s = fmaf(row.t(d, iy, io, mean) * weight(a, d) * row.gate(d, &slope), row.at(a.y, a.ys, d) * iy, s);
        s = a.channels == 1 ? 0.0f : block_sum(s) * a.inv_channels;
    }
    for (int d = threadIdx.x; d < a.channels; d += kThreads) {
        const float t = row.t(d, iy, io, mean);
        if (a.y) {
            const float m = row.at(a.y, a.ys, d) * iy, tw = t * weight(a, d);
            const float dy = iy * (tw * row.gate(d, &slope) * one_channel(a, iy) - m * s);
            if (a.z) row.put(a.dz, a.dzs, d, tw * m * slope);
            row.put(a.dy, a.dys, d, dy);
        }
        row.put(a.dx, a.dxs, d, t);
    }
}

#define KERNEL_OF(type, name) \
    ((type) == SEQ_FP32 ? (const void *)name<F32> : (type) == SEQ_FP16 ? (const void *)name<F16> : (const void *)name<BF16>)

bool sizes_ok(int64_t rows, int64_t channels) { return rows >= 0 && channels >= 1; }
bool sizes_supported(int64_t rows, int64_t channels) { return rows <= kMaxSize && channels <= kMaxChannels; }

}  // namespace
}  // namespace mi355seq

using namespace mi355seq;

extern "C" {

int seq_norm_forward(int64_t rows, int64_t channels, int type, const void *x, const void *y, const void *z,
                     const int64_t *strides, const float *post, const float *scale, const float *pre, float eps,
                     void *out, void *normed, float *stats, hipStream_t stream) {
    if (!sizes_ok(rows, channels) || !known_type(type) || !(eps > 0.0f)) return SEQ_EINVAL;
    if (!sizes_supported(rows, channels)) return SEQ_EUNSUPPORTED;
    if (rows == 0) return SEQ_OK;
    if ((y == nullptr) != (post == nullptr) || (y == nullptr) != (out == nullptr)) return SEQ_EINVAL;
    if (!y && (z || scale)) return SEQ_EINVAL;
    if ((pre == nullptr) != (normed == nullptr)) return SEQ_EINVAL;
    if (!x || (!y && !pre)) return SEQ_EINVAL;
    const Grid grid{1, rows, channels, element_bytes(type)};
    Rows v[5] = {{x, 0, 0}, {y, 0, 0}, {z, 0, 0}, {out, 0, 0}, {normed, 0, 0}};
    for (int i = 0; i < 5; ++i) {
        v[i].si = strides ? strides[i] : channels;
        if (!strides_in_range(v[i])) return SEQ_EINVAL;
        if (misaligned(v[i].p, grid.bytes)) return SEQ_EALIGN;
    }
    for (const void *p : {(const void *)post, (const void *)scale, (const void *)pre, (const void *)stats})
        if (misaligned(p, 4)) return SEQ_EALIGN;
    for (int i = 3; i < 5; ++i) {
        if (v[i].p && !rows_apart(v[i], grid)) return SEQ_EINVAL;
        for (int j = 0; j < i; ++j) {
            const bool own = (i == 3 && j == 0) || (i == 4 && (j == 1 || j == 2));
            if (own && same_rows(v[i], v[j], grid)) continue;
            if (may_share(v[i], v[j], grid)) return SEQ_EINVAL;
        }
    }
    NormArgs a{};
    a.rows = rows, a.channels = (int)channels, a.eps = eps, a.inv_channels = 1.0f / (float)channels;
    a.x = x, a.y = y, a.z = z, a.out = out, a.normed = normed;
    a.xs = v[0].si, a.ys = v[1].si, a.zs = v[2].si, a.outs = v[3].si, a.normeds = v[4].si;
    a.post = post, a.scale = scale, a.pre = pre, a.stats = stats;
    void *args[] = {&a};
    return launch(KERNEL_OF(type, norm_forward), dim3((unsigned)rows), dim3(kThreads), args, 0, stream);
}

size_t seq_norm_workspace_bytes(int64_t rows, int64_t channels, int type) {
    if (!sizes_ok(rows, channels) || !sizes_supported(rows, channels) || !known_type(type)) return 0;
    return up16((size_t)rows * 4) + up16((size_t)(2 * kRowGroups) * (size_t)channels * 4);
}

int seq_norm_backward(int64_t rows, int64_t channels, int type, const void *dout, const void *dnormed,
                      const void *x, const void *y, const void *z, const int64_t *strides, const float *post,
                      const float *scale, const float *pre, float eps, const float *stats, void *dx, void *dy,
                      void *dz, float *dpost, float *dscale, float *dpre, void *workspace, hipStream_t stream) {
    if (!sizes_ok(rows, channels) || !known_type(type) || !(eps > 0.0f)) return SEQ_EINVAL;
    if (!sizes_supported(rows, channels)) return SEQ_EUNSUPPORTED;
    if ((post == nullptr) != (dpost == nullptr) || (scale == nullptr) != (dscale == nullptr) ||
        (pre == nullptr) != (dpre == nullptr) || (scale && !post))
        return SEQ_EINVAL;
    if (rows) {  // tensors without elements have no address
        if ((y == nullptr) != (post == nullptr) || (y == nullptr) != (dy == nullptr)) return SEQ_EINVAL;
        if ((z == nullptr) != (dz == nullptr) || (!y && z)) return SEQ_EINVAL;
        if ((pre == nullptr) != (dnormed == nullptr)) return SEQ_EINVAL;
        if (!x || !dx || !stats || !workspace || (!y && !pre)) return SEQ_EINVAL;
    }
    const Grid grid{1, rows, channels, element_bytes(type)};
    Rows v[8] = {{dout, 0, 0}, {dnormed, 0, 0}, {x, 0, 0}, {y, 0, 0}, {z, 0, 0}, {dx, 0, 0}, {dy, 0, 0}, {dz, 0, 0}};
    for (int i = 0; i < 8; ++i) {
        v[i].si = strides ? strides[i] : channels;
        if (!strides_in_range(v[i])) return SEQ_EINVAL;
        if (misaligned(v[i].p, grid.bytes)) return SEQ_EALIGN;
    }
    for (const void *p : {(const void *)post, (const void *)scale, (const void *)pre, (const void *)stats,
                          (const void *)dpost, (const void *)dscale, (const void *)dpre})
        if (misaligned(p, 4)) return SEQ_EALIGN;
    if (misaligned(workspace, 16)) return SEQ_EALIGN;
    for (int i = 5; i < 8; ++i) {
        if (v[i].p && !rows_apart(v[i], grid)) return SEQ_EINVAL;
        for (int j = 0; j < i; ++j) {
            const bool own = (i == 5 && (j == 0 || j == 2)) || (i == 6 && (j == 1 || j == 3)) || (i == 7 && j == 4);
            if (own && same_rows(v[i], v[j], grid)) continue;
            if (may_share(v[i], v[j], grid)) return SEQ_EINVAL;
        }
    }
    NormArgs a{};
    a.rows = rows, a.channels = (int)channels, a.eps = eps, a.inv_channels = 1.0f / (float)channels;
    a.dout = dout, a.dnormed = dnormed, a.x = x, a.y = y, a.z = z, a.dx = dx, a.dy = dy, a.dz = dz;
    a.douts = v[0].si, a.dnormeds = v[1].si, a.xs = v[2].si, a.ys = v[3].si, a.zs = v[4].si;
    a.dxs = v[5].si, a.dys = v[6].si, a.dzs = v[7].si;
    a.post = post, a.scale = scale, a.pre = pre, a.stats = const_cast<float *>(stats);
    a.mean = (float *)workspace, a.partial = (float *)((char *)workspace + up16((size_t)rows * 4));
    a.dpost = dpost, a.dscale = dscale, a.dpre = dpre;
    int groups = rows ? kRowGroups : 0;
    void *args[] = {&a, &groups};
    const dim3 block(kThreads);
    const unsigned columns = (unsigned)ceil_div(channels, kThreads);
    int rc = SEQ_OK;
    if (rows && pre) rc = launch(KERNEL_OF(type, norm_row_mean), dim3((unsigned)rows), block, args, 0, stream);
    if (rc == SEQ_OK && rows) rc = launch(KERNEL_OF(type, norm_columns), dim3(columns, kRowGroups), block, args, 0, stream);
    if (rc == SEQ_OK) rc = launch((const void *)norm_sum_columns, dim3(columns), block, args, 0, stream);
    if (rc == SEQ_OK && rows) rc = launch(KERNEL_OF(type, norm_backward), dim3((unsigned)rows), block, args, 0, stream);
    return rc;
}

}  // extern "C"
