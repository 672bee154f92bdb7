// tensor_map.cuh -- host side: tensor maps with 128-byte swizzle.
#pragma once

#include <cuda.h>

#include "encoder.cuh"

namespace sieve {
namespace enc {

sieve_status encode_map(CUtensorMap *map, CUtensorMapDataType type, int rank, const void *base, const cuuint64_t *dims,
                        const cuuint64_t *strides, const cuuint32_t *box);

// a map of [rows][width], rows `stride` elements apart, boxes of 128 bytes x
// `box_rows`; base 16-byte aligned, width and stride multiples of 16 bytes
sieve_status make_matrix_map(CUtensorMap *map, int dtype, const void *base, int64_t rows, int64_t width,
                             int64_t stride, int box_rows);

}  // namespace enc
}  // namespace sieve
