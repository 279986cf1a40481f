// Four-bit weights on the host: the stored form of a row, and rounding to nearest onto the grid.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "qmoe.h"

namespace {

constexpr int kMaxRows = 1 << 24, kMaxCols = 1 << 20;

size_t row_bytes(int cols) { return (size_t)64 * (((size_t)cols + 127) / 128); }

// Where column c's four bits stand in a row, in halves of bytes.
inline size_t place(int c)
{
    const int in = c % 128, s = in / 32, i = in % 32 / 8, j = in % 8;
    return (size_t)(c / 128) * 128 + 8 * (size_t)(4 * i + s) + 4 * (size_t)(j % 2) + (size_t)(j / 2);
}
inline void put(uint8_t *row, int c, int v)
{
    const size_t p = place(c);
    row[p / 2] = (uint8_t)(row[p / 2] | v << (4 * (p % 2)));
}

uint16_t half_bits(float f)  // f >= 0 and below 65520; to nearest even
{
    uint32_t u;
    std::memcpy(&u, &f, 4);
    if (u < 0x38800000u) return (uint16_t)std::nearbyintf(f * 16777216.0f);  // below 2^-14: units of 2^-24
    u += 0xFFFu + ((u >> 13) & 1u);
    return (uint16_t)((u >> 13) - (112u << 10));
}
float half_value(uint16_t h)
{
    if (h < 0x400) return (float)h * 5.9604644775390625e-8f;
    const uint32_t u = ((uint32_t)h << 13) + (112u << 23);
    float f;
    std::memcpy(&f, &u, 4);
    return f;
}

bool shape_ok(int rows, int cols) { return rows >= 1 && cols >= 1; }

}  // namespace

extern "C" {

size_t qmoe_int4_row_bytes(int cols) { return cols < 1 ? 0 : row_bytes(cols); }

qmoe_status qmoe_int4_pack_host(const uint8_t *values, int rows, int cols, uint8_t *weights)
{
    if (!values || !weights || !shape_ok(rows, cols)) return QMOE_E_INVALID_ARG;
    if (rows > kMaxRows || cols > kMaxCols) return QMOE_E_LIMIT;
    const size_t rb = row_bytes(cols);
    for (int r = 0; r < rows; r++) {
        const uint8_t *v = values + (size_t)r * cols;
        uint8_t *row = weights + (size_t)r * rb;
        std::memset(row, 0, rb);
        for (int c = 0; c < cols; c++) {
            if (v[c] > 15) return QMOE_E_BAD_SYMBOL;
            put(row, c, v[c]);
        }
    }
    return QMOE_OK;
}

qmoe_status qmoe_int4_unpack_host(const uint8_t *weights, int rows, int cols, uint8_t *values)
{
    if (!values || !weights || !shape_ok(rows, cols)) return QMOE_E_INVALID_ARG;
    if (rows > kMaxRows || cols > kMaxCols) return QMOE_E_LIMIT;
    const size_t rb = row_bytes(cols);
    for (int r = 0; r < rows; r++)
        for (int c = 0; c < cols; c++) {
            const size_t p = place(c);
            values[(size_t)r * cols + c] = (uint8_t)(weights[(size_t)r * rb + p / 2] >> (4 * (p % 2)) & 15);
        }
    return QMOE_OK;
}

qmoe_status qmoe_int4_quantize_host(const float *w, int rows, int cols, int group, uint8_t *weights, uint16_t *scale_f16,
                                    uint8_t *zero)
{
    if (!w || !weights || !scale_f16 || !shape_ok(rows, cols) || (group != 32 && group != 64 && (group < 1 || group % 128)))
        return QMOE_E_INVALID_ARG;
    if (rows > kMaxRows || cols > kMaxCols) return QMOE_E_LIMIT;
    const size_t rb = row_bytes(cols), groups = ((size_t)cols + group - 1) / group;
    for (int r = 0; r < rows; r++) {
        const float *v = w + (size_t)r * cols;
        uint8_t *row = weights + (size_t)r * rb;
        std::memset(row, 0, rb);
        for (size_t g = 0; g < groups; g++) {
            const int c0 = (int)(g * group), c1 = (int)std::min<long long>(cols, (long long)c0 + group);
            float lo = 0.0f, hi = 0.0f;
            for (int c = c0; c < c1; c++) {
                if (!std::isfinite(v[c])) return QMOE_E_INVALID_ARG;
                lo = std::min(lo, v[c]);
                hi = std::max(hi, v[c]);
            }
            const double want = zero ? ((double)hi - lo) / 15.0 : (double)std::max(hi, -lo) / 7.0;
            if (!(want < 65520.0)) return QMOE_E_LIMIT;
            const uint16_t bits = half_bits((float)want);
            if (bits > 0x7BFF) return QMOE_E_LIMIT;
            const float s = half_value(bits);
            int z = 8;
            if (zero && s > 0.0f) z = (int)std::min(15.0f, std::max(0.0f, std::nearbyintf(-lo / s)));
            for (int c = c0; c < c1; c++) {
                float q = (float)z;
                if (s > 0.0f) q = std::min(15.0f, std::max(0.0f, std::nearbyintf(v[c] / s) + (float)z));
                put(row, c, (int)q);
            }
            scale_f16[(size_t)r * groups + g] = bits;
            if (zero) zero[(size_t)r * groups + g] = (uint8_t)z;
        }
    }
    return QMOE_OK;
}

}  // extern "C"
