// k_rope.hip -- rotary positions: the table of cosines and sines, and the rotation of activations.
//
// Pair i of a head's first rot columns is turned by the angle position * f_i (a 2 x 2 rotation, times the table's
// magnitude); its transpose, with -sin, is the gradient.  Both are bound by reading x and writing y: a thread turns eight or
// sixteen columns, 16 bytes a lane, so that all of a head's pairs are loaded once whatever the layout.  8192 x 32 x 128 float32,
// half of the columns turned: 51 us, 5.2 TB/s (a large copy 4.8); 64 x 40 x 128 bfloat16: 3.1 us, the launch.  Where the pairs do not
// come in whole eights a thread turns one: 8192 x 32 x 80 bfloat16, 40 columns in halves 60 us, 1.4 TB/s (pairs 17 us).  The table
// is bound by cosines and sines in double: 131,072 x 64 pairs 75 us.
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

// A thread an item (turn_item) of a head of a row.
template <bool F32, int BY>
__global__ __launch_bounds__(256) void k_rope(const char* x, char* y, int64_t rows, int H, int d, int64_t x_row,
                                              int64_t x_head, int64_t y_row, int64_t y_head,
                                              const int32_t* __restrict__ pos, RopeArgs rope, float sign) {
    constexpr int ESZ = F32 ? 4 : 2;
    const int items = turn_items(d, rope.rot, BY);
    const uint32_t of_row = (uint32_t)(H * items);
    const int64_t total = rows * of_row, step = (int64_t)gridDim.x * 256;
    for (int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x; n < total; n += step) {
        const int64_t r = (total >> 32) == 0 ? (int64_t)((uint32_t)n / of_row) : n / of_row;
        const uint32_t in_row = (uint32_t)(n - r * of_row);
        const int h = (int)(in_row / (uint32_t)items), i = (int)(in_row - h * items);
        turn_item<F32, BY>(x + (r * x_row + h * x_head) * ESZ, y + (r * y_row + h * y_head) * ESZ, d, rope,
                           table_row(rope, pos[r]), i, sign);
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
    const TurnBy by = turn_by(d, rope);
    const int64_t items = rows * H * turn_items(d, rope.rot, by);
    const dim3 grid((unsigned)grid_blocks((items + 255) / 256)), block(256);
    const float sign = backward ? -1.0f : 1.0f;
    auto go = [&](auto f32, auto how) {
        k_rope<decltype(f32)::value, decltype(how)::value><<<grid, block, 0, s>>>(
            (const char*)x, (char*)y, rows, H, d, x_row, x_head, y_row, y_head, pos, rope, sign);
    };
    auto pick = [&](auto f32) {
        if (by == kTurnHalves) go(f32, std::integral_constant<int, kTurnHalves>{});
        else if (by == kTurnPairs) go(f32, std::integral_constant<int, kTurnPairs>{});
        else go(f32, std::integral_constant<int, kTurnOne>{});
    };
    if (dtype == 0) pick(std::true_type{});
    else pick(std::false_type{});
    return hipGetLastError();
}

}  // namespace lacache
