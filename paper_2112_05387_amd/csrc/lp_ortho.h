// Launch descriptors of the orthogonalisation by Newton-Schulz products (lp_ortho.hip).
#pragma once
#include <hip/hip_runtime.h>

#include "lp_gemm.h"

namespace lp {

enum NsFlag { NS_SRC_LOW = 1, NS_OUT_LOW = 2,      // bf16
              NS_PLAIN = 4,                         // updated without orthogonalisation
              NS_VEC = 8, NS_VEC_OUT = 16 };        // 16-byte accesses to what is read (grad, vel or src), to rows of out and master

// One tensor.  Matrices are worked on with their shorter side as rows (tall ones are transposed on the way in and out).
struct NsProb {
    const void* src;                    // the matrix, or null: it is the momentum of an update
    void* out;                          // orthogonalised matrix (src != null), or the parameters
    const float* grad; float *vel, *master;
    char* work;                         // X before and after a step, X X^T, the polynomial in it: see NsWork
    long ld_src, ld_out;
    int rows, cols;                     // as stored
    float lr, shrink;                   // the step taken, what is left of the parameters (1 - lr * weight decay)
    int flags, pad_;
};

// What follows from the sizes: shorter and longer side; elements of a row of S, B and of X (32 of the first plane, the same 32 of the
// second, and so on, zeros behind the last); bytes of X and of S.
struct NsWork {
    int r, c, ldr, ldc;
    size_t x, s;
    __host__ __device__ __forceinline__ NsWork(int rows, int cols) {
        r = rows < cols ? rows : cols; c = rows < cols ? cols : rows;
        ldr = (r + 31) / 32 * 64; ldc = (c + 31) / 32 * 64;
        x = ((size_t)r * ldc * 2 + 255) / 256 * 256; s = ((size_t)r * ldr * 2 + 255) / 256 * 256;
    }
    __host__ __device__ __forceinline__ size_t bytes() const { return 2 * x + 2 * s; }
    // The Gram matrix is a long sum, and little else happens to the matrix: added up by the matrix cores, which cut every addend to the sum's
    // last bit, it is what the result is off by (64 x 5000 2.4 times, 64 x 50000 5 times as far as the same products in fp32; 640 x 5760 0.7 times).
    // It is added up in parts then (0.8 and 0.7 times); 191 and 1258 us for the five steps became 199 and 1326.
    __host__ __device__ __forceinline__ bool thin() const { return c / 16 >= r; }
};
constexpr int kNsPart = 8;              // k-tiles (of 32) of such a part

// First block of every tensor in the launches: of the small matrices and the tensors that are none; over the elements of the others, over
// their 64 x 64 pieces, over tiles of r x r and of r x c.  Behind the last tensor the number of blocks.  All of it lies in device
// memory: ints [kNsLaunches][n + 1], then the tensors.
constexpr int kNsLaunches = 5;
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

// The same for the tensors of an update, whose pointers are offsets in a few buffers: words of the buffers of every set (params, grads,
// velocity, master), then records.  A record: rows, cols, flags | set << 8, offset in params (two words), in the others (two), first
// block of launch 0; and where matrices are worked on in memory (`full`) offset of the work (two), first blocks of launches 1 to 4.
constexpr int kNsSetWords = 8, kNsRecord = 8, kNsRecordFull = 14;
struct NsPack {
    int* table; NsProb* probs; char* work;
    int n, first, count, sets, full;
    float lr, shrink;
    int total[kNsLaunches];
    unsigned w[960];
};

constexpr int kNsElems = 4096;          // elements of a block of the launches over elements

// Small matrices: one workgroup each, in LDS from the first step to the last.  Bytes it takes, 0: does not fit.
constexpr size_t kNsSmallLds = 160 * 1024;
__host__ __device__ inline size_t ns_small_lds(int rows, int cols) {
    const int r = rows < cols ? rows : cols, c = rows < cols ? cols : rows;
    if (r > 64) return 0;
    const size_t need = r > 32 ? (size_t)64 * ((c + 63) / 64 * 256) + 16384 : (size_t)32 * ((c + 63) / 64 * 256) + 12288;
    return need <= kNsSmallLds ? need : 0;
}

// Tiles of a step (i: longer side, j: shorter side) and of the symmetric products, and the tile that is fastest for `tiles(cfg)` of them
enum NsTile { NT_256 = 0, NT_256x320, NT_128, NT_64, NT_COUNT };
void ns_tile_size(int cfg, int* bi, int* bj);
double ns_tile_time(int cfg, long tiles);
hipError_t launch_ns_put(const NsChunk& c, hipStream_t s);
hipError_t launch_ns_pack(const NsPack& c, hipStream_t s);
hipError_t launch_ns_small(const NsArgs& a, int steps, size_t lds, hipStream_t s);
hipError_t launch_ns_norm(const NsArgs& a, hipStream_t s);
hipError_t launch_ns_split(const NsArgs& a, hipStream_t s);
hipError_t launch_ns_gram(const NsArgs& a, int cfg, hipStream_t s);
hipError_t launch_ns_poly(const NsArgs& a, int cfg, hipStream_t s);
hipError_t launch_ns_step(const NsArgs& a, int cfg, hipStream_t s);

}  // namespace lp
