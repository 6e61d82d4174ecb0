// Which tiles a product is cut into, and how often its sum.  Plain host arithmetic.
#pragma once
#include <stdint.h>

namespace am_host {

constexpr uint32_t kComputeUnits = 256;      // of an MI355X

struct ProductPlan {
    uint32_t tile;         // 256, 128 or 64: both sides
    uint32_t splits;       // workgroups that share a tile's sum
    uint32_t split_k;      // of k for each, a multiple of a step
};

// Time of a product by the rounds its workgroups take: a round lasts as long as its steps, `resident` workgroups a compute unit at a
// time, and a sum that is split costs its parts' way through memory and a launch.
inline ProductPlan product_plan(bool bf16, uint64_t replicas, uint64_t m, uint64_t n, uint64_t k)
{
    struct Shape { uint32_t tile, resident; double step_us, fixed_us; };
    static const Shape shapes_bf16[] = {{256, 1, 1.25, 3.0}, {128, 2, 0.65, 2.0}, {64, 4, 0.45, 1.5}};
    static const Shape shapes_f32[] = {{128, 2, 4.6, 2.0}, {64, 4, 2.4, 1.5}};
    const Shape *shapes = bf16 ? shapes_bf16 : shapes_f32;
    const int count = bf16 ? 3 : 2;
    const uint64_t step = bf16 ? 64 : 32, steps = (k + step - 1) / step;
    ProductPlan best = {64, 1, (uint32_t)(steps * step)};
    double best_us = -1.;
    for (int i = 0; i < count; ++i) {
        const Shape &s = shapes[i];
        const uint64_t tiles = ((m + s.tile - 1) / s.tile) * ((n + s.tile - 1) / s.tile) * replicas;
        for (uint64_t splits = 1; splits <= 32 && splits <= steps; splits = splits < 4 ? splits + 1 : splits * 2) {
            const uint64_t each = (steps + splits - 1) / splits, used = (steps + each - 1) / each;
            const uint64_t slots = (uint64_t)kComputeUnits * s.resident, rounds = (tiles * used + slots - 1) / slots;
            double us = (double)rounds * ((double)each * s.step_us + s.fixed_us);
            if (used > 1) us += 4. + (double)(used + 1) * 4. * (double)(replicas * m) * (double)n / 4e6;
            if (best_us < 0. || us < best_us) { best_us = us; best = {s.tile, (uint32_t)used, (uint32_t)(each * step)}; }
        }
    }
    return best;
}

// Rows for each workgroup of the column sums: some 2048 workgroups, 64 rows at least.
inline void column_parts(uint64_t replicas, uint64_t m, uint64_t n, uint32_t *rows_per_part, uint32_t *parts)
{
    const uint64_t across = ((n + 255) / 256) * replicas;
    uint64_t want = across >= 2048 ? 1 : 2048 / across;
    uint64_t rows = (m + want - 1) / want;
    rows = rows < 64 ? 64 : rows;
    if ((m + rows - 1) / rows > 65535) rows = (m + 65534) / 65535;
    *rows_per_part = (uint32_t)rows;
    *parts = (uint32_t)((m + rows - 1) / rows);
}

}  // namespace am_host
