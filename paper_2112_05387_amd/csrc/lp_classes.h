// Launch descriptors of the linear classifier's cross-entropy (lp_classes.hip).
#pragma once
#include <hip/hip_runtime.h>

#include "lp_gemm.h"

namespace lp {

// rows of `cols` elements, ld apart, to rows of `width`; rows 0: nothing
struct CePack { const void* src; void* dst; long ld; int rows, cols, width, blocks; };

// l = X W^T over one piece of the classes (rows i: classes v0 .. v0 + V - 1, columns j: samples)
struct CeLogits {
    GemmOperand w, x;
    GemmPairs pairs;
    int K, kchunk;                      // channels, and how many of them a slice has
    int V, N, v0, V_all;
    int tiles_i, tiles_j, band;
    const float* bias;                  // of the piece, or null
    unsigned long long* mask; int* count;    // probabilities: which rows count, and how many do, are found beside them
    int* ticket;                        // statistics, partial logits: set to zero for the kernel behind, or null
    float2* partial; int parts;         // statistics: [N][parts] (maximum, sum) without the label's class
    float* own;                         // statistics: the label's logit of every row that has one
    float* slices; size_t slice;        // partial logits: [slices][N][ldv]
    int ldv, ldp;                       // classes of a row of slices / prob, a multiple of 8 (three planes: 32); elements of a row of prob
    const float* lse; const int* labels;
    char* prob; size_t pplane;          // probabilities: three planes of bf16 [N][ldv], or beside each other [N][ldp]
    float* colsum; int ld_colsum;       // their sums over the samples of every wave's tile, or null
    float* others;                      // their sums over the classes of every wave's tile but the label's, [N][parts], or null
    const float* dlabel;                // the label's p - 1 where p > 1/2, or null: left at zero
};
struct CeLabel {
    int N, V, parts, ldp;
    const int* labels;
    const float* others;
    unsigned short* prob; size_t pplane;
    float* dlabel;                      // -sum of the others where p > 1/2, or zero
};
struct CeRows {
    int N, V;
    const int* labels;
    const float* bias;
    const float2* partial; int parts; const float* own;
    const float* slices; size_t slice; int nslices, ldv;
    float *lse, *row_loss, *loss;
    float* bsum; int* bcnt;             // of every workgroup
    int* ticket;                        // workgroups that are done, zero before; or null: somebody else adds up
    unsigned long long* mask; int* count;
};
// out[j][i] (+)= sum_k a[k][i] * b[..]; i channels, j samples or classes
struct CeGrad {
    GemmOperand a, b;
    GemmPairs pairs;
    int K, kchunk, I, J;
    int tiles_i, tiles_j, band;
    float* out; size_t slice; int ldo;
    int vec, add;                       // 16-byte stores (I a multiple of four then); add to what is there
    const int* count; float scale;      // scaled by scale / count, or not
    const unsigned long long* mask;
    // the gradient itself instead of a partial result: its rows (with a class, or zero), type, 16-byte (bf16: 8-byte) stores
    void* last; long ldlast; int C, low, vec_last, V_all; const int* labels;
};
struct CeSum { const float* part; size_t slice; int nslices, ldp; void* out; size_t ldo; int rows, cols, parts_log; };
struct CeFinish {
    CeSum x, w;
    int blocks_x, blocks_w, blocks_b;
    const int* labels; const int* count; float scale;
    int N, V, V_all;                    // V: classes of the bias here
    const float* colsum; int parts, ld_colsum;
    const float* dlabel;                // what the labels' classes have besides, or null
    const unsigned short* prob; size_t pplane; int beside, ldp;
    float* dbias;
};

// Small problems, straight from the caller's operands (lp_classes_direct.hip)
struct CeDirect {
    int N, C, V;
    const void *x, *w; long ldx, ldw;
    int vec;                            // rows of the weights can be read 16 bytes at a time
    const float* bias; const int* labels;
    float *lse_out, *row_loss, *loss, *bsum; int* bcnt;      // forward
    const float* lse; float scale; float* d;                // backward: d [N][V] between its two kernels
    void* dx; long lddx; float *dw, *dbias;
};
int ce_direct_waves(int N, int C, int V);
hipError_t launch_ce_direct_forward(const CeDirect& a, int dtype, int waves, hipStream_t s);
hipError_t launch_ce_direct_backward(const CeDirect& a, int dtype, int waves, hipStream_t s);
hipError_t launch_ce_total(const float* sums, const int* counts, int n, float* loss, hipStream_t s);

// tiles: 0 256 x 256, 1 128 x 128, 2 64 x 64, 3 128 x 32 (few samples); of three planes 4 128 x 128, 5 64 x 64; waves along either side
void ce_tile_size(int cfg, int* bi, int* bj, int* wi, int* wj);
double ce_tile_time(int cfg, long blocks, int ktiles);
hipError_t launch_ce_pack(CePack x, CePack w, int dtype, hipStream_t s);
hipError_t launch_ce_stats(const CeLogits& a, int cfg, hipStream_t s);
hipError_t launch_ce_prob_tiles(const CeLogits& a, int cfg, hipStream_t s);
hipError_t launch_ce_sums(const CeLogits& a, int cfg, hipStream_t s);
hipError_t launch_ce_label(const CeLabel& a, bool beside, hipStream_t s);
hipError_t launch_ce_others(const CeLabel& a, bool first, hipStream_t s);
hipError_t launch_ce_slices(const CeLogits& a, int slices, int cfg, hipStream_t s);
hipError_t launch_ce_rows(const CeRows& a, hipStream_t s);
hipError_t launch_ce_prob(const CeRows& a, unsigned short* prob, size_t pplane, int ldp, bool beside, hipStream_t s);
hipError_t launch_ce_dx(const CeGrad& a, int slices, int cfg, hipStream_t s);
hipError_t launch_ce_dw(const CeGrad& a, int slices, int cfg, hipStream_t s);
hipError_t launch_ce_finish(const CeFinish& a, int dtype, hipStream_t s);
hipError_t launch_ce_zero(float* p, size_t n, hipStream_t s);

}  // namespace lp
