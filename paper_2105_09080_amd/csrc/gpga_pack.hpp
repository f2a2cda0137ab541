// Rows of fp32, bf16 or fp16 as rows of halves for gpga_product.hpp, by one wavefront each: the row is read twice, the second time
// from the caches.
#pragma once

#include "gpga_product.hpp"
#include "gpga_rows.hpp"

__device__ __forceinline__ float max_nan(float a, float b) { return a > b || a != a ? a : b; }  // NaN if either is

struct RowStat {
    float down;       // inverse of the row's scale
    float norm, sum;  // of the scaled values: root of the sum of squares, sum of magnitudes
};

template <typename E>
__device__ __forceinline__ float row_max(const typename E::mem* row, int32_t cols) {
    float m = 0.f;
    for (int32_t c = (int32_t)(threadIdx.x & (kWave - 1)) * kOct; c < cols; c += kWave * kOct) {
        float v[kOct];
        piece_read<kOct, E>(row, c, cols, v);
#pragma unroll
        for (int j = 0; j < kOct; ++j) m = max_nan(m, fabsf(v[j]));
    }
    return wave_all<kWave>(m, max_nan);
}

// `cols` values, of which fold(column, eight values) makes others, times the row's scale (or `given`, where that is not `own`), into `cols2` halves and
// as many in the second plane; zeros behind the values.  A fold sees columns up to `cols2`.
struct NoFold {
    __device__ __forceinline__ void operator()(int32_t, float*) const {}
};
template <typename E, int Planes, typename Fold = NoFold>
__device__ __forceinline__ RowStat pack_row(const typename E::mem* row, int32_t cols, int32_t cols2, bool own, Scale given, half_t* to, int64_t plane,
                                            Fold&& fold = {}) {
    const int32_t lane = (int32_t)(threadIdx.x & (kWave - 1));
    auto read = [&](int32_t c, float* v) {
        if (c < cols) {
            piece_read<kOct, E>(row, c, cols, v);
            fold(c, v);
        } else {
#pragma unroll
            for (int j = 0; j < kOct; ++j) v[j] = 0.f;
        }
    };
    Scale s;
    if (!own) {
        s = given;
    } else {
        float m = 0.f;
        for (int32_t c = lane * kOct; c < cols; c += kWave * kOct) {
            float v[kOct];
            read(c, v);
#pragma unroll
            for (int j = 0; j < kOct; ++j) m = max_nan(m, fabsf(v[j]));
        }
        s = scale_for(wave_all<kWave>(m, max_nan));
    }
    float squares = 0.f, sum = 0.f;
    for (int32_t c = lane * kOct; c < cols2; c += kWave * kOct) {
        float v[kOct];
        read(c, v);
        half8 hi, lo;
#pragma unroll
        for (int j = 0; j < kOct; ++j) {
            const float w = v[j] * s.up;
            half_t h, l;
            split(w, &h, &l);
            hi[j] = h;
            lo[j] = l;
            squares += w * w;
            sum += fabsf(w);
        }
        *reinterpret_cast<half8*>(to + c) = hi;
        if constexpr (Planes == 2) *reinterpret_cast<half8*>(to + plane + c) = lo;
    }
    return {s.down, sqrtf(wave_sum<kWave>(squares)), wave_sum<kWave>(sum)};
}

// e, a whole number in -126 .. 126, with the row's norm below 2^e; -infinity for a row of zeros, NaN for one with an infinity or NaN.
__device__ __forceinline__ float norm_exponent(const RowStat& r) {
    if (r.down == 0.f) return -INFINITY;
    if (r.down != r.down) return NAN;
    const int e = (int)(__float_as_uint(r.norm * 1.0001f) >> 23) - 126 + (int)(__float_as_uint(r.down) >> 23) - 127;
    return (float)min(max(e, -126), 126);
}
// 2^e for -126 <= e <= 127; 0 for -infinity (and 2^-e for `e` negated: 0 as well), NaN for NaN.
__device__ __forceinline__ float power_of_two(float e) {
    if (e != e) return NAN;
    return fabsf(e) == INFINITY ? 0.f : __uint_as_float((uint32_t)(127 + (int)e) << 23);
}
