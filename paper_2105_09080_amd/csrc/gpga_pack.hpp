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

// `cols` values, times fold[column] if there is one, times the row's scale (or `given`, where that is not `own`), into `cols2` halves and as many in the
// second plane; zeros behind the values.
template <typename E, int Planes>
__device__ __forceinline__ RowStat pack_row(const typename E::mem* row, int32_t cols, int32_t cols2, const float* fold, bool own, Scale given, half_t* to,
                                            int64_t plane) {
    const int32_t lane = (int32_t)(threadIdx.x & (kWave - 1));
    auto read = [&](int32_t c, float* v) {
        if (c < cols) {
            piece_read<kOct, E>(row, c, cols, v);
            if (fold) {
#pragma unroll
                for (int j = 0; j < kOct; ++j) v[j] *= fold[c + j];  // padded like the row of halves
            }
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
            hi[j] = (half_t)w;
            lo[j] = (half_t)(w - (float)hi[j]);
            squares += w * w;
            sum += fabsf(w);
        }
        *reinterpret_cast<half8*>(to + c) = hi;
        if constexpr (Planes == 2) *reinterpret_cast<half8*>(to + plane + c) = lo;
    }
    return {s.down, sqrtf(wave_sum<kWave>(squares)), wave_sum<kWave>(sum)};
}
