// Dropout with a counter-based generator (philox.h).  The pass is a copy with eight
// values a lane: bf16 moves 32 bytes and takes one evaluation of the generator.
#include "lm_internal.h"
#include "philox.h"
#include "row_io.h"

namespace dyad {

namespace {

constexpr int kThreads = 256;

template <class T>
__global__ void __launch_bounds__(kThreads) dropout_kernel(const T *x, T *y, int64_t rows, int n, int octets, DropArgs d) {
    const uint64_t offset = drop_offset(d);
    const int64_t total = rows * octets;
    for (int64_t o = (int64_t)blockIdx.x * kThreads + threadIdx.x; o < total; o += (int64_t)gridDim.x * kThreads) {
        const int64_t row = total >> 32 ? o / octets : (int64_t)((uint32_t)o / (uint32_t)octets);
        const int c = (int)(o - row * octets) * 8;
        float v[8];
        load_cols(x + row * n, c, n, v);
        apply_drop(v, keep_bits(philox(d.seed, offset, (uint64_t)o), d.thr), d.scale);
        store_cols<true>(y + row * n, c, n, v);
    }
}

}  // namespace

hipError_t launch_dropout(int64_t rows, int64_t cols, int dtype, const void *x, const DropArgs &d, void *y, hipStream_t s) {
    const int octets = (int)((cols + 7) / 8);
    const int64_t blocks = (rows * octets + kThreads - 1) / kThreads;
    const unsigned grid = (unsigned)(blocks < 8192 ? blocks : 8192);
    if (dtype == kBF16)
        dropout_kernel<<<grid, kThreads, 0, s>>>(static_cast<const uint16_t *>(x), static_cast<uint16_t *>(y), rows,
                                                 (int)cols, octets, d);
    else
        dropout_kernel<<<grid, kThreads, 0, s>>>(static_cast<const float *>(x), static_cast<float *>(y), rows, (int)cols,
                                                 octets, d);
    return hipGetLastError();
}

}  // namespace dyad
