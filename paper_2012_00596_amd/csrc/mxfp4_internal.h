// Linear layers in microscaled 4-bit floats: the packed handle, its device format and the kernels' argument blocks.
//
// Operand images.  The matrix instruction 32 x 32 x 64 takes per lane 32 consecutive elements of a row (16 bytes, one block) and the
// block's scale byte: lane 32 h + r holds row r, elements 32 h .. 32 h + 31 of a 64-element step.  An image is the 1 KB that the 64 lanes
// hold, in their order.  Steps are counted from the row's start, an even number of them, filled up with zero codes and zero scales.
//   weights:      64 outputs a group; image ((group * steps + step) * 2 + j), row r = output 64 group + 2 r + j
//   activations:  32 rows a tile; image (tile * steps + step), row r = row 32 tile + r of the batch
// Scales: four steps' bytes of a lane in one word, byte s of word [(group * quads + step / 4) * 2 + j][lane] (activations: [tile * quads
// + step / 4][lane]) for step 4 (step / 4) + s.
#pragma once
#include <cstddef>
#include <cstdint>
#include <vector>

#include "npas_internal.h"

struct npas_mxfp4 {
    int dtype = 0, OUT = 0, IN = 0;
    int blocks = 0, steps = 0, quads = 0, groups = 0; // blocks of 32, steps of 64 (even) and runs of four steps in a row; groups of 64 outputs
    std::vector<uint8_t> codes, scales;               // canonical: [OUT][16 blocks], [OUT][blocks]
    int device = -1;
    void *blob = nullptr;
    size_t bytes = 0;
    const void *images = nullptr;
    const uint32_t *image_scales = nullptr;
};

namespace npas {

struct QuantizeArgs {
    const void *x;
    uint8_t *codes, *scales; // canonical rows; or images of activations and their scale words
    int64_t x_stride;
    int rows, K, blocks, steps, quads;
    WideDiv by_blocks; // canonical rows: of a slab of rows, see row_slab
    int slab;
};

struct DequantizeArgs {
    const uint8_t *codes, *scales;
    void *y;
    int rows, K, blocks;
    WideDiv by_blocks;
    int slab;
};

struct FcMxArgs {
    const void *x; // rows as they are, for launches that quantise them themselves
    int64_t x_stride;
    const void *x_images;
    const uint32_t *x_scales;
    const void *w_images;
    const uint32_t *w_scales;
    const float *bias;
    void *y;
    int B, IN, OUT, blocks, steps, quads, groups, tiles, act;
};

int launch_mxfp4_quantize(int dt, const QuantizeArgs &a, void *stream);
int launch_mxfp4_quantize_images(int dt, const QuantizeArgs &a, void *stream);
int launch_mxfp4_dequantize(int dt, const DequantizeArgs &a, void *stream);
bool fc_mxfp4_quantises(int B, int steps, int groups); // the product's launch takes its rows as they are
int launch_fc_mxfp4(int dt, const FcMxArgs &a, void *stream);

} // namespace npas
