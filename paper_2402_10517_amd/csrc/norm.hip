// The norms around a block of a decoder layer, fused with the block's gate, scale and residual.
//
// r = residual + scale * gate * norm(x) (the norm of the block's output only with `post`), out = norm(r); norm(v) = weight * (v - mean) / sqrt(mean square + eps) + bias.
//
// A workgroup holds a row in registers, `PER` chunks of 8 columns per thread: each input is read and each output written once, and the norm after the
// residual needs no second pass over memory.  Large ones are bound by HBM: 8192 x 8192 with a post norm, a gate per value and a binary32 residual 172 us (940 MB, 5.5 TB/s),
// with no post norm, binary16, 95 us (537 MB, 5.7 TB/s).  Smaller ones are bound by what a row does one after the other, of which a CU has two or three at a time: loads
// from HBM, two sums over the workgroup for a centred norm and one for another, weights from the L2, stores.  1531 x 5121 centred with a post norm 25.5 us (63 MB, 2.5 TB/s), 30 with
// inputs from HBM, of which the rows' odd starts are 5.  One row of 4096: 4.4 us, a launch that does nothing 3.5.
#include <type_traits>

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
    double each; // 1 / columns
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

// x of the lane that a data-parallel primitive names, 0 without one
template <int CTRL, int ROWS> __device__ __forceinline__ double moved(double x)
{
    const uint64_t bits = __builtin_bit_cast(uint64_t, x);
    const uint32_t low = __builtin_amdgcn_update_dpp(0, (int)bits, CTRL, ROWS, 0xf, true), high = __builtin_amdgcn_update_dpp(0, (int)(bits >> 32), CTRL, ROWS, 0xf, true);
    return __builtin_bit_cast(double, (uint64_t)high << 32 | low);
}

__device__ __forceinline__ double from_lane(double x, int lane)
{
    const uint64_t bits = __builtin_bit_cast(uint64_t, x);
    const uint32_t low = __builtin_amdgcn_readlane((int)bits, lane), high = __builtin_amdgcn_readlane((int)(bits >> 32), lane);
    return __builtin_bit_cast(double, (uint64_t)high << 32 | low);
}

// The sum over the workgroup, the same bits in all threads.  `place` alternates, so that one barrier is enough.
template <int WAVES> __device__ __forceinline__ double block_sum(double x, double *place)
{
    x += moved<0x111, 0xf>(x); // row_shr:1, 2, 4, 8: lane 15 of each row has the row's
    x += moved<0x112, 0xf>(x);
    x += moved<0x114, 0xf>(x);
    x += moved<0x118, 0xf>(x);
    x += moved<0x142, 0xa>(x); // row_bcast:15, 31: lane 63 has all
    x += moved<0x143, 0xc>(x);
    const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
    if (waves == 1) return from_lane(x, 63);
    if (lane == 63) place[threadIdx.x >> 6] = x;
    __syncthreads();
    const int of = lane & (WAVES - 1);
    x = of < waves ? place[of] : 0;
    x += moved<0x111, 0xf>(x);
    x += moved<0x112, 0xf>(x);
    if constexpr (WAVES > 4) x += moved<0x114, 0xf>(x);
    if constexpr (WAVES > 8) x += moved<0x118, 0xf>(x);
    return from_lane(x, WAVES - 1);
}

// Sums of squares outside these are taken again of values times 2^-70 or 2^100: a thread's 32 then add up to 2^121 at most, or are 2^-98 each at least, subnormal values' too
constexpr float kLeastSum = 0x1p-80f, kMostSum = 0x1p120f;

// TAIL: the last chunk of a row is not whole.  CENTRED by itself, as what large rows of it need costs the others registers (two workgroups of 1024 threads on a CU leave each 62
// vector and 80 scalar ones): 8192 x 8192, binary32 residual, post norm 152 us, 166 with a branch.
template <class R, int THREADS, int PER, bool TAIL, bool CENTRED> __global__ __launch_bounds__(THREADS) void norm_kernel(const NormArgs a)
{
    __shared__ double places[2][16];
    constexpr bool LATE = THREADS * PER > 2048; // registers do not hold all of a wide row's inputs
    int turn = 0;
    const auto sum = [&](double x) { return block_sum<THREADS / 64>(x, places[turn++ & 1]); };
    const int columns = a.columns, first = threadIdx.x * kEach, step = blockDim.x * kEach;
    for (int64_t row = blockIdx.x; row < a.tokens; row += gridDim.x) {
        float v[PER][kEach]; // 0 in columns that do not exist
        // columns from chunk p on; asked for anew in each place, as the compiler would keep a mask per column in scalar registers that it does not have
        const auto left = [&](int p) {
            int n = columns - (first + p * step);
            asm("" : "+v"(n));
            return n;
        };
        // 0 in the columns that chunk p does not have
        const auto cut = [&](int p) {
            int n = left(p);
            if (n >= (TAIL ? kEach : 1)) return;
            asm volatile("" : "+v"(n)); // stays a branch
#pragma unroll
            for (int i = 0; i < kEach; ++i) v[p][i] = TAIL && i < n ? v[p][i] : 0.0f;
        };
        // normalises v: sums of up to 8 (the mean) or 32 values in binary32, of those in binary64.  The mean may be far above the differences from it: 48 bits.
        // large: values may be of any size; else they have been rounded to binary16
        const auto norm = [&](const _Float16 *weight, const _Float16 *bias, auto large) {
            asm("" : "+s"(weight), "+s"(bias)); // not in registers for the next row
            float part = 1.0f;
            if constexpr (CENTRED) {
                const auto values = [&](float by) {
                    double s = 0;
#pragma unroll
                    for (int p = 0; p < PER; ++p) {
                        const auto x = [&](int i) { return v[p][i] * by; };
                        s += (double)(((x(0) + x(1)) + (x(2) + x(3))) + ((x(4) + x(5)) + (x(6) + x(7))));
                    }
                    return sum(s);
                };
                double mean = values(1.0f);
                if (large() && !(__builtin_fabs(mean) < (double)INFINITY)) mean = values(0x1p-8f) * 0x1p8; // eight values may add up to more than binary32 holds
                mean *= a.each;
                float high = (float)mean, low = (float)(mean - (double)high);
                if (large()) { // and a difference may be more where the mean is not below the greatest's last place: a quarter of all of them then
                    part = __builtin_fabsf(high) < 0x1p100f ? 1.0f : 0.25f;
                    high *= part, low *= part;
                }
#pragma unroll
                for (int p = 0; p < PER; ++p) {
#pragma unroll
                    for (int i = 0; i < kEach; ++i) v[p][i] = (large() ? __builtin_fmaf(v[p][i], part, -high) : v[p][i] - high) - low;
                    cut(p);
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
            float s = 0;
#pragma unroll
            for (int p = 0; p < PER; ++p)
#pragma unroll
                for (int i = 0; i < kEach; ++i) s = __builtin_fmaf(v[p][i], v[p][i], s);
            double mean = sum((double)s);
            if (mean > (double)kMostSum) mean = squares(0x1p-70f) * 0x1p140;
            else if (mean < (double)kLeastSum) mean = squares(0x1p100f) * 0x1p-200;
            mean = mean * a.each + (double)(CENTRED && large() ? a.eps * part * part : a.eps);
            // 1 / sqrt as two factors, an inverse root (to 1 ulp) and a power of two, which comes first: values times it are 2^8 at most.  The root is of 1/4 .. 1, or of less where
            // the power would leave binary32 (rows of subnormal values, without eps).  Of a row with an infinity both are 0 and its finite values become 0.
            const int half = (__builtin_amdgcn_frexp_exp(mean) + 1) >> 1, power = half > -126 ? half : -126;
            const bool finite = mean < (double)INFINITY;
            const float f = finite ? __builtin_amdgcn_rsqf((float)__builtin_ldexp(mean, -2 * power)) : mean == (double)INFINITY ? 0.0f : NAN;
            const float g = finite ? __builtin_ldexpf(1.0f, -power) : 0.0f;
#pragma unroll
            for (int p = 0; p < PER; ++p) {
                const int c = first + p * step;
                if (c < columns) {
                    if (LATE) asm volatile("" ::: "memory");
                    Eight<_Float16> w, b;
#pragma unroll
                    for (int i = 0; i < kEach; ++i) w.x[i] = (_Float16)1, b.x[i] = (_Float16)0;
                    if (weight) w = load<TAIL>(weight, c, columns);
                    if (bias) b = load<TAIL>(bias, c, columns);
#pragma unroll
                    for (int i = 0; i < kEach; ++i) v[p][i] = __builtin_fmaf(v[p][i] * g * f, w[i], b[i]);
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
            if (a.post) norm(a.post_weight, a.post_bias, std::false_type{});
        }
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            const int c = first + p * step;
            if (c < columns) {
                if (LATE) asm volatile("" ::: "memory"); // a chunk's after the one before
                if (LATE && a.residual) r[p] = load<TAIL>(from, c, columns);
                if (LATE && a.gate) g[p] = load<TAIL>(a.gate + row * a.gate_stride, c, columns);
                Eight<R> y;
#pragma unroll
                for (int i = 0; i < kEach; ++i) {
                    const float gated = a.gate ? v[p][i] * g[p][i] : v[p][i];
                    y.x[i] = !a.x ? r[p].x[i] : (R)(a.residual ? __builtin_fmaf(a.scale, gated, r[p][i]) : a.scale * gated);
                    v[p][i] = (float)y.x[i];
                }
                if (a.residual_out) store<TAIL>(to, c, columns, y);
            }
            cut(p);
        }
        if (!a.out) continue;
        norm(a.weight, a.bias, std::bool_constant<sizeof(R) == 4>{});
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

template <class R, bool TAIL, bool CENTRED> void launch(const NormArgs &k, hipStream_t stream)
{
    const int chunks = (k.columns + kEach - 1) / kEach;
    const dim3 grid((unsigned)(k.tokens < 1 << 20 ? k.tokens : 1 << 20));
    const auto threads = [&](int per) { return (chunks + 64 * per - 1) / (64 * per) * 64; };
    // A chunk per thread up to 8192 columns, as a row's time is that of its loads, sums and stores one after the other; of more rows than CUs with a binary16 residual two
    // (three workgroups of 8192 columns on a CU) where a row has more sums or its last chunk takes registers.  us with one / two, binary16 residual: 8192 x 8190 159 / 127,
    // centred with a post norm 225 / 144, 300 x 6201 8.4 / 7.0; 8192 x 8192 centred with a post norm 123 / 119, centred 104 / 105, 2000 x 6144 centred with a post norm
    // 24.7 / 23.8; where it stays one: 256 x 8192 5.3 / 5.4, 1024 x 8192 12.7 / 13.7, 8192 x 8192 95 / 100, with a post norm 105 / 111, 4096 x 4096 22.1 / 22.9; binary32
    // residual, 8192 x 8192 141 / 148, with a post norm and a gate 171 / 179.
    if (chunks <= 256) norm_kernel<R, 256, 1, TAIL, CENTRED><<<grid, threads(1), 0, stream>>>(k);
    else if (sizeof(R) == 2 && (TAIL || CENTRED) && chunks > 512 && chunks <= 1024 && k.tokens > 256) norm_kernel<R, 512, 2, TAIL, CENTRED><<<grid, threads(2), 0, stream>>>(k);
    else if (chunks <= 1024) norm_kernel<R, 1024, 1, TAIL, CENTRED><<<grid, threads(1), 0, stream>>>(k);
    else if (chunks <= 2048) norm_kernel<R, 1024, 2, TAIL, CENTRED><<<grid, threads(2), 0, stream>>>(k);
    else norm_kernel<R, 1024, 4, TAIL, CENTRED><<<grid, threads(4), 0, stream>>>(k);
}

template <class R> void launch(const NormArgs &k, hipStream_t stream)
{
    if (k.columns % kEach) k.centred ? launch<R, true, true>(k, stream) : launch<R, true, false>(k, stream);
    else k.centred ? launch<R, false, true>(k, stream) : launch<R, false, false>(k, stream);
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
    k.scale = a.scale, k.eps = a.eps, k.each = 1.0 / (double)(a.columns > 0 ? a.columns : 1);
    if (a.half) launch<_Float16>(k, stream);
    else launch<float>(k, stream);
    return hipGetLastError();
}

} // namespace apgemv
