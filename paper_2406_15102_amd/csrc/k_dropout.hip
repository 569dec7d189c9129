// Dropout from the counter stream, with the residual added on the way: y = r + keep(i) x / (1 - p).
// The backward pass is the same map of the gradient without a residual: nothing is kept of the forward pass.
// Bound by memory: 2 or 3 tensors once.  A word of the stream serves two elements, and the four words of a lane's vector share a
// product (rand_words<4>): about 12 issue slots an element with the selection and the conversion.
#include "around_device.hpp"

namespace hlq {

// U vectors of 8 elements to a lane, 256 lanes' vectors side by side; the loads of all U go out before the first is used.
template <typename T, bool RES, int U>
__global__ __launch_bounds__(256) void k_dropout(const T *x, const T *r, int64_t n, DropRule d, T *y)
{
    const int64_t base = (static_cast<int64_t>(blockIdx.x) * U * 256 + threadIdx.x) * 8;
    const float factor = d.below ? d.scale : 1.0f;
    Raw<T, 8> a[U], b[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t i = base + u * 2048;
        if (i + 8 <= n) {
            a[u].load(x + i);
            if (RES) b[u].load(r + i);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t i = base + u * 2048;
        float v[8], q[8];
        if (i + 8 <= n) {
            if (d.below) drop_raw(a[u], static_cast<uint32_t>(i >> 1), d);
            a[u].widen(v);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= factor;
            if (RES) {
                b[u].widen(q);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += q[e];
            }
            a[u].pack(v);
            a[u].store(y + i);
        } else {
            for (int64_t k = i; k < n; ++k) {          // at most seven, in one lane of the grid
                Raw<T, 1> one;
                one.load(x + k);
                if (d.below) drop_raw(one, k, d);
                one.widen(v);
                v[0] *= factor;
                if (RES) v[0] += load_one(r + k);
                store_one(y + k, v[0]);
            }
        }
    }
}

template <typename T, bool RES>
static hipError_t go(const T *x, const T *r, int64_t n, const DropRule &d, T *y, hipStream_t st)
{
    constexpr int64_t per = 256 * 8;
    if (n >= int64_t(1) << 22)
        k_dropout<T, RES, 2><<<static_cast<unsigned>((n + 2 * per - 1) / (2 * per)), 256, 0, st>>>(x, r, n, d, y);
    else
        k_dropout<T, RES, 1><<<static_cast<unsigned>((n + per - 1) / per), 256, 0, st>>>(x, r, n, d, y);
    return hipGetLastError();
}

hipError_t launch_dropout(const void *x, const void *r, int64_t n, bool is_f32, const DropRule &d, void *y, hipStream_t st)
{
    if (is_f32)
        return r ? go<float, true>(static_cast<const float *>(x), static_cast<const float *>(r), n, d, static_cast<float *>(y), st)
                 : go<float, false>(static_cast<const float *>(x), nullptr, n, d, static_cast<float *>(y), st);
    return r ? go<bf16_t, true>(static_cast<const bf16_t *>(x), static_cast<const bf16_t *>(r), n, d, static_cast<bf16_t *>(y), st)
             : go<bf16_t, false>(static_cast<const bf16_t *>(x), nullptr, n, d, static_cast<bf16_t *>(y), st);
}

}  // namespace hlq
