// k_rope.hip -- rotary positions: the table of cosines and sines, and the rotation of activations.
//
// Pair i of a head's first rot columns is turned by the angle position * f_i (a 2 x 2 rotation, times the table's
// magnitude); its transpose, with -sin, is the gradient.  Both are bound by reading x and writing y.
#include "kv.hpp"
#include "launch.hpp"

namespace lacache {

__global__ __launch_bounds__(256) void k_rope_table(float2* __restrict__ table, int64_t first, int64_t n, int half,
                                                    double base, double factor, double original, double low,
                                                    double high, double magnitude) {
    const int64_t total = n * half, step = (int64_t)gridDim.x * 256;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += step) {
        const int64_t row = i / half;
        const int j = (int)(i - row * half);
        const double f = exp2(-log2(base) * (double)j / (double)half);
        const double turns = original * f * 0.15915494309189535;  // 1 / (2 pi)
        double g = (turns - low) / (high - low);
        g = g < 0.0 ? 0.0 : g > 1.0 ? 1.0 : g;
        const double angle = (double)(first + row) * ((1.0 - g) * f / factor + g * f);
        table[i] = make_float2((float)(magnitude * cos(angle)), (float)(magnitude * sin(angle)));
    }
}

// One element a thread, whatever the strides and alignment.
__global__ __launch_bounds__(256) void k_rope_any(const void* x, void* y, int dtype, int64_t rows, int H, int d,
                                                  int64_t x_row, int64_t x_head, int64_t y_row, int64_t y_head,
                                                  const int32_t* __restrict__ pos, RopeArgs rope, bool backward) {
    // a pair, or a column that stays, is one item: y may be x
    const int half = rope.rot / 2, items = d - half;
    const int64_t total = rows * H * items, step = (int64_t)gridDim.x * 256;
    for (int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x; n < total; n += step) {
        const int64_t r = n / items / H;
        const int i = (int)(n % items), h = (int)(n / items % H);
        const int64_t xi = r * x_row + h * x_head, yi = r * y_row + h * y_head;
        auto get = [&](int c) {
            return dtype == 0 ? ((const float*)x)[xi + c] : bf16_to_f32(((const uint16_t*)x)[xi + c]);
        };
        auto put = [&](int c, float v) {
            if (dtype == 0) ((float*)y)[yi + c] = v;
            else ((uint16_t*)y)[yi + c] = f32_to_bf16(v);
        };
        if (i >= half) {
            put(i + half, get(i + half));
            continue;
        }
        int64_t p = pos[r];
        p = p < 0 ? 0 : p >= rope.n_pos ? rope.n_pos - 1 : p;
        const float2 cs = ((const float2*)rope.table)[p * half + i];
        const int ca = rope.pairs ? 2 * i : i, cb = rope.pairs ? 2 * i + 1 : i + half;
        float a = get(ca), b = get(cb);
        turn(a, b, cs.x, backward ? -cs.y : cs.y);
        put(ca, a);
        put(cb, b);
    }
}

hipError_t launch_rope_table(float* table, int64_t first, int64_t n, int rot, double base, double factor,
                             double original, double low, double high, double magnitude, hipStream_t s) {
    if (n <= 0) return hipSuccess;
    k_rope_table<<<dim3((unsigned)grid_blocks((n * (rot / 2) + 255) / 256)), dim3(256), 0, s>>>(
        (float2*)table, first, n, rot / 2, base, factor, original, low, high, magnitude);
    return hipGetLastError();
}

hipError_t launch_rope(const void* x, void* y, int dtype, int64_t rows, int H, int d, int64_t x_row, int64_t x_head,
                       int64_t y_row, int64_t y_head, const int32_t* pos, const RopeArgs& rope, bool backward,
                       hipStream_t s) {
    if (rows <= 0) return hipSuccess;
    const int64_t items = rows * H * (d - rope.rot / 2);
    k_rope_any<<<dim3((unsigned)grid_blocks((items + 255) / 256)), dim3(256), 0, s>>>(
        x, y, dtype, rows, H, d, x_row, x_head, y_row, y_head, pos, rope, backward);
    return hipGetLastError();
}

}  // namespace lacache
