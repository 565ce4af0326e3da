// The projections' tile kernels on rows that are gathered by expert, for the mixture of experts.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace gdn {
namespace linear {

// An entry of the tile table: a tile of rows of expert `expert`, whose `tiles` entries begin at entry `first`.
struct ExpertTile { int32_t expert, first, tiles, rows; };       // rows: of the whole expert

struct ExpertProduct {
    const void* x;                 // bf16, rows of K
    int64_t ldx;
    int32_t x_rows;                // rows of x; x_rows ldx 2 < 2^31
    int32_t div;                   // a listed row v is row v / div of x
    const void* w;                 // bf16, per expert [n_w][K]: N rows, or with `gated` N of the gate and N of up
    bool gated;
    int32_t act;
    const float* weights;          // by listed row: a factor on the outputs (with `gated`)
    void* y;                       // row v of y for a listed row v, N apart: bf16 with `gated`, else fp32
    const int32_t* list;           // [expert][list_stride]
    int32_t list_stride;
    const ExpertTile* table;       // device
    const int32_t* n_tiles;        // device: entries of the table
    int32_t most_tiles;            // at most so many, by the host's count
    int32_t N, K;
};

// Rows of a tile in tile shape `shape` (as gdn_linear_tune's numbers: 0, 2 or 3).
int expert_tile_rows(int shape);
// The estimated time of a product of so many row tiles with weights of so many rows, by the rounds over the chip.
double expert_product_us(int shape, int64_t row_tiles, int64_t rows_w, int32_t K);
hipError_t launch_expert_product(const ExpertProduct& p, int shape, hipStream_t stream);

}  // namespace linear
}  // namespace gdn
