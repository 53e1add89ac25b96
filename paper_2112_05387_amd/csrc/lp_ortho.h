// Launch descriptors of the orthogonalisation by Newton-Schulz products (lp_ortho.hip).
#pragma once
#include <hip/hip_runtime.h>

#include "lp_gemm.h"

namespace lp {

// One tensor.  Matrices are worked on with their shorter side as rows (tall ones are transposed on the way in and out).
struct NsProb {
    const void* src;                    // the matrix, or null: it is the momentum of an update
    void* out;                          // orthogonalised matrix (src != null), or the parameters
    const float* grad; float *vel, *master;
    long ld_src, ld_out;
    char *x0, *x1, *s, *b;              // X before and after a step, X X^T, the polynomial in it
    int rows, cols, r, c, ldr, ldc;     // as stored; shorter and longer side; elements of a row of S, B and of X: 32 of the first
                                        // plane, the same 32 of the second, and so on, zeros behind the last
    int src_low, out_low;               // bf16
    int plain;                          // updated without orthogonalisation
    float lr, shrink;                   // the step taken, what is left of the parameters (1 - lr * weight decay)
    int vec, vec_out;                   // 16-byte accesses to what is read (grad, vel or src), to rows of out and master
};

// First block of every tensor in the launches over elements, over 64 x 64 pieces, over tiles of r x r and of r x c; behind
// the last tensor the number of blocks.  All of it lies in device memory: `table` ints [4][n + 1], then the tensors.
struct NsArgs {
    const int* start;                   // of this launch
    const int* start_norm;
    const NsProb* p;
    double* norm;                       // sums of squares, one a block of the launch over elements
    int n, total;
    float momentum, wd, rest_lr;
    int nesterov;
    int odd, last;                      // step: which of x0 / x1 it reads; its result is the answer
};

struct NsChunk { unsigned* dst; int words; unsigned w[960]; };

constexpr int kNsElems = 4096;          // elements of a block of the launch over elements

// Tiles of a step (i: longer side, j: shorter side) and of the symmetric products, and the tile that is fastest for `tiles(cfg)` of them
enum NsTile { NT_256 = 0, NT_256x320, NT_128, NT_64, NT_COUNT };
void ns_tile_size(int cfg, int* bi, int* bj);
double ns_tile_time(int cfg, long tiles);
hipError_t launch_ns_put(const NsChunk& c, hipStream_t s);
hipError_t launch_ns_norm(const NsArgs& a, hipStream_t s);
hipError_t launch_ns_split(const NsArgs& a, hipStream_t s);
hipError_t launch_ns_gram(const NsArgs& a, int cfg, hipStream_t s);
hipError_t launch_ns_poly(const NsArgs& a, int cfg, hipStream_t s);
hipError_t launch_ns_step(const NsArgs& a, int cfg, hipStream_t s);

}  // namespace lp
