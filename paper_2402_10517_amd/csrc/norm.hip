// The norms around a block of a decoder layer, fused with the block's gate, scale and residual.
//
// A workgroup holds a row in registers, `PER` chunks of 8 columns per thread: each input is read and each output written once, and the norm after the
// residual needs no second pass over memory. Bound by HBM; a single row by its launch, its loads and a reduction per norm.
#include "decode_device.h"

namespace apgemv {

namespace {

struct NormArgs {
    const _Float16 *x, *gate;
    const void *residual;
    void *residual_out;
    _Float16 *out;
    int64_t x_stride, gate_stride, residual_stride, residual_out_stride, out_stride;
    const _Float16 *weight, *bias, *post_weight, *post_bias;
    int64_t tokens;
    int columns, post, centred;
    float scale, eps;
};

constexpr int kEach = 8; // adjacent columns of a chunk

// 8 adjacent values, kept as words so that halves stay packed.  Rows start at any element: 16-byte accesses that ask for the element's alignment only.
template <class T> struct Eight {
    typedef T values_t __attribute__((ext_vector_type(kEach)));
    struct __attribute__((packed, aligned(sizeof(T)))) Place {
        values_t x;
    };
    values_t x;
    __device__ float operator[](int i) const { return (float)x[i]; }
};

// The chunk at column c of a row; 0 where there are no such columns
template <bool TAIL, class T> __device__ __forceinline__ Eight<T> load(const T *row, int c, int columns)
{
    typedef Eight<T> E;
    if (!TAIL || c + kEach <= columns) return E{reinterpret_cast<const typename E::Place *>(row + c)->x};
    E e{};
    for (int i = 0; i < kEach - 1; ++i)
        if (c + i < columns) e.x[i] = row[c + i];
    return e;
}

template <bool TAIL, class T> __device__ __forceinline__ void store(T *row, int c, int columns, const Eight<T> &e)
{
    if (!TAIL || c + kEach <= columns) {
        reinterpret_cast<typename Eight<T>::Place *>(row + c)->x = e.x;
        return;
    }
    for (int i = 0; i < kEach - 1; ++i)
        if (c + i < columns) row[c + i] = e.x[i];
}

// The sum over the workgroup, the same bits in all threads.  `place` alternates, so that one barrier is enough.
__device__ __forceinline__ double block_sum(double x, double *place)
{
    for (int m = 1; m < 64; m <<= 1) x += __shfl_xor(x, m);
    if (blockDim.x == 64) return x;
    if ((threadIdx.x & 63) == 0) place[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0;
    for (int w = 0; w < (int)(blockDim.x >> 6); ++w) x += place[w];
    return x;
}

// The square of a sum's range: sums of squares beyond it are taken again of values times 2^-64 or 2^64
constexpr float kLeastSum = 0x1p-80f, kMostSum = 0x1p120f;

// TAIL: the last chunk of a row is not whole
template <class R, int PER, bool POST, bool CENTRED, bool TAIL> __global__ __launch_bounds__(1024) void norm_kernel(const NormArgs a)
{
    __shared__ double places[2][16];
    constexpr bool LATE = PER >= 4; // registers do not hold all of a wide row's inputs
    int turn = 0;
    const auto sum = [&](double x) { return block_sum(x, places[turn++ & 1]); };
    const int columns = a.columns, first = threadIdx.x * kEach, step = blockDim.x * kEach;
    for (int64_t row = blockIdx.x; row < a.tokens; row += gridDim.x) {
        float v[PER][kEach]; // 0 in columns that do not exist
        // columns from chunk p on; asked for anew in each place, as the compiler would keep a mask per column in scalar registers that it does not have
        const auto left = [&](int p) {
            int n = columns - (first + p * step);
            asm("" : "+v"(n));
            return n;
        };
        // normalises v: sums of up to 8 (the mean) or 32 values in binary32, of those in binary64.  The mean may be far above the differences from it: 48 bits.
        const auto norm = [&](const _Float16 *weight, const _Float16 *bias) {
            if constexpr (CENTRED) {
                double s = 0;
#pragma unroll
                for (int p = 0; p < PER; ++p)
                    s += (double)(((v[p][0] + v[p][1]) + (v[p][2] + v[p][3])) + ((v[p][4] + v[p][5]) + (v[p][6] + v[p][7])));
                const double mean = sum(s) / columns;
                const float high = (float)mean, low = (float)(mean - (double)high);
#pragma unroll
                for (int p = 0; p < PER; ++p) {
                    const int n = TAIL ? left(p) : left(p) > 0 ? kEach : 0;
#pragma unroll
                    for (int i = 0; i < kEach; ++i) v[p][i] = i < n ? (v[p][i] - high) - low : 0.0f;
                }
            }
            const auto squares = [&](float by) {
                float s = 0;
#pragma unroll
                for (int p = 0; p < PER; ++p)
#pragma unroll
                    for (int i = 0; i < kEach; ++i) s = __builtin_fmaf(v[p][i] * by, v[p][i] * by, s);
                return sum((double)s);
            };
            double mean = squares(1.0f);
            if (mean > (double)kMostSum) mean = squares(0x1p-64f) * 0x1p128;
            else if (mean < (double)kLeastSum) mean = squares(0x1p64f) * 0x1p-128;
            const double inverse = 1.0 / sqrt(mean / columns + (double)a.eps);
            // as two factors, of which neither leaves binary32 where their product does not
            const float f = (float)__builtin_sqrt(inverse);
            const float g = f > 0 ? (float)(inverse / (double)f) : 0.0f; // of a row with an infinity 0: its finite values become 0
#pragma unroll
            for (int p = 0; p < PER; ++p) {
                const int c = first + p * step;
                if (c < columns) {
                    Eight<_Float16> w, b;
#pragma unroll
                    for (int i = 0; i < kEach; ++i) w.x[i] = (_Float16)1, b.x[i] = (_Float16)0;
                    if (weight) w = load<TAIL>(weight, c, columns);
                    if (bias) b = load<TAIL>(bias, c, columns);
#pragma unroll
                    for (int i = 0; i < kEach; ++i) v[p][i] = __builtin_fmaf(v[p][i] * f * g, w[i], b[i]);
                }
            }
        };
        const R *from = static_cast<const R *>(a.residual) + row * a.residual_stride;
        R *const to = static_cast<R *>(a.residual_out) + row * a.residual_out_stride;
        Eight<R> r[PER];
        Eight<_Float16> x[PER], g[PER];
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            const int c = first + p * step;
            if (c < columns) {
                if (a.x) x[p] = load<TAIL>(a.x + row * a.x_stride, c, columns);
                if (!LATE && a.residual) r[p] = load<TAIL>(from, c, columns);
                if (!LATE && a.gate) g[p] = load<TAIL>(a.gate + row * a.gate_stride, c, columns);
            }
        }
        if (a.x) {
#pragma unroll
            for (int p = 0; p < PER; ++p) {
                const bool there = left(p) > 0;
#pragma unroll
                for (int i = 0; i < kEach; ++i) v[p][i] = there ? x[p][i] : 0.0f;
            }
            if constexpr (POST) norm(a.post_weight, a.post_bias);
        }
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            const int c = first + p * step;
            if (c < columns) {
                if (LATE && a.residual) r[p] = load<TAIL>(from, c, columns);
                if (LATE && a.gate) g[p] = load<TAIL>(a.gate + row * a.gate_stride, c, columns);
                Eight<R> y;
                const int n = TAIL ? left(p) : left(p) > 0 ? kEach : 0;
#pragma unroll
                for (int i = 0; i < kEach; ++i) {
                    const float gated = a.gate ? v[p][i] * g[p][i] : v[p][i];
                    y.x[i] = !a.x ? r[p].x[i] : (R)(a.residual ? __builtin_fmaf(a.scale, gated, r[p][i]) : a.scale * gated);
                    v[p][i] = i < n ? (float)y.x[i] : 0.0f;
                }
                if (a.residual_out) store<TAIL>(to, c, columns, y);
            } else {
#pragma unroll
                for (int i = 0; i < kEach; ++i) v[p][i] = 0;
            }
        }
        if (!a.out) continue;
        norm(a.weight, a.bias);
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            const int c = first + p * step;
            if (c < columns) {
                Eight<_Float16> y;
#pragma unroll
                for (int i = 0; i < kEach; ++i) y.x[i] = (_Float16)v[p][i];
                store<TAIL>(a.out + row * a.out_stride, c, columns, y);
            }
        }
    }
}

template <class R, int PER, bool TAIL> void launch(const NormArgs &k, int threads, hipStream_t stream)
{
    const dim3 grid((unsigned)(k.tokens < 1 << 20 ? k.tokens : 1 << 20));
    if (k.post) {
        if (k.centred) norm_kernel<R, PER, true, true, TAIL><<<grid, threads, 0, stream>>>(k);
        else norm_kernel<R, PER, true, false, TAIL><<<grid, threads, 0, stream>>>(k);
    } else {
        if (k.centred) norm_kernel<R, PER, false, true, TAIL><<<grid, threads, 0, stream>>>(k);
        else norm_kernel<R, PER, false, false, TAIL><<<grid, threads, 0, stream>>>(k);
    }
}

template <class R, bool TAIL> void launch(const NormArgs &k, hipStream_t stream)
{
    const int chunks = (k.columns + kEach - 1) / kEach;
    const auto threads = [&](int per) { return (chunks + 64 * per - 1) / (64 * per) * 64; };
    if (chunks <= 1024) launch<R, 1, TAIL>(k, threads(1), stream);
    else if (chunks <= 2048) launch<R, 2, TAIL>(k, threads(2), stream);
    else launch<R, 4, TAIL>(k, threads(4), stream);
}

template <class R> void launch(const NormArgs &k, hipStream_t stream)
{
    if (k.columns % kEach) launch<R, true>(k, stream);
    else launch<R, false>(k, stream);
}

} // namespace

hipError_t launch_norm(const ap_normed &a, hipStream_t stream)
{
    NormArgs k;
    k.x = static_cast<const _Float16 *>(a.x.data), k.gate = a.x.data ? static_cast<const _Float16 *>(a.gate.data) : nullptr;
    k.residual = a.residual.data;
    k.residual_out = const_cast<void *>(a.residual_out.data);
    k.out = static_cast<_Float16 *>(const_cast<void *>(a.out.data));
    k.x_stride = a.x.stride, k.gate_stride = a.gate.stride, k.residual_stride = a.residual.stride, k.residual_out_stride = a.residual_out.stride,
    k.out_stride = a.out.stride;
    k.weight = static_cast<const _Float16 *>(a.weight), k.bias = static_cast<const _Float16 *>(a.bias);
    k.post_weight = static_cast<const _Float16 *>(a.post_weight), k.post_bias = static_cast<const _Float16 *>(a.post_bias);
    k.tokens = a.tokens, k.columns = (int)a.columns, k.post = a.post, k.centred = a.centred;
    k.scale = a.scale, k.eps = a.eps;
    if (a.half) launch<_Float16>(k, stream);
    else launch<float>(k, stream);
    return hipGetLastError();
}

} // namespace apgemv
