// Softmax cross-entropy of a linear classifier over many classes (gfx950), logits never handed out:
//
//   l_nv = sum_c x_nc w_vc + b_v,   lse_n = log sum_v exp l_nv,   loss_n = lse_n - l_n,y(n)
//   d_nv = (exp(l_nv - lse_n) - [v = y(n)]) / count,   dX = d W,   dW = d^T X,   db_v = sum_n d_nv
//
// Products on the matrix cores, each with what follows it as its epilogue.  Forward: l = X W^T, of which a workgroup keeps the
// maximum and the sum of exponentials of its classes for every row (the statistics of all tiles are joined by a small kernel; the label's
// class is kept apart until then).  Backward: the same product once more, whose epilogue turns a tile into
// probabilities; they go to memory, all at once or piece of the classes by piece, and are read from there by the two gradient products.
// Keeping the logits would save one product (of seven in bf16: dW takes three, dX two) and cost 4 bytes a logit.
//
// Precision.  bf16: products of bf16 are exact, sums are fp32.  The probabilities are kept as three bf16 (24 bits), all of which dW and
// the bias read, which are fp32 (with two dW is off by 1.8e-6, with three by the 2e-7 of its sums).  dX, rounded to bf16 itself,
// reads two: sum_v d_nv is zero, so what the rows of W have in common cancels in dX, and with one part of 8 bits it does not (64 x 256
// -> 4000 with 0.5 added to every weight: 8e-3 off instead of 1.7e-3).
// fp32: every operand as three bf16 (24 bits) that lie beside each other, six of the nine products (the others are below 2^-25).
// 73623 classes x 8716 rows of 633 channels: a product in 4.2 ms, 195 TFLOP/s of fp32; the card's fp32 matrix product reaches 151.
//
// Of a row that is all but certain p - 1 has lost what tells p from one (lse is fp32: 33 x 2026 -> 234 with a loss of 7e-4, dW off by 4.7e-4,
// some p above one).  There d is minus the sum of the other classes' p, which the tiles yield beside their probabilities: the label's own is
// filled in by a small kernel behind them, or, where the classes come in pieces, known from a pass over all pieces ahead of them.
//
// Rows whose label is no class (ignored): probability zero in the epilogue by selection, and their features count as zero in
// dW whatever they hold (a bit a row, read by the loads): no infinity or NaN in them reaches a sum.
//
// Few tiles (small mini-batches, few classes) are cut along the reduction, partial results in fp32, and joined by the kernel
// that needs all of a row anyway (softmax) or by the one that rounds (gradients); no atomics, the order of every sum is fixed.
#include "lp_classes.h"

#include <algorithm>

#include "lp_gemm.h"
#include "lp_kernels.h"

namespace lp {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kInf = __builtin_inff();

__device__ __forceinline__ float bf16_up(unsigned bits) { return __uint_as_float(bits << 16); }
// nearest bf16 of a finite value stays finite: the last step up to infinity would leave a rest that is none
__device__ __forceinline__ unsigned bf16_part(float x) {
    const unsigned b = float_to_bf16_bits(x);
    return (b & 0x7fffu) == 0x7f80u && (__float_as_uint(x) & 0x7fffffffu) < 0x7f800000u ? __float_as_uint(x) >> 16 : b;
}
// x as a sum of NP bf16; infinities and NaN in the first alone
template <int NP> __device__ __forceinline__ void split_bf16(float x, unsigned (&b)[NP]) {
    b[0] = bf16_part(x);
    const bool fin = (b[0] & 0x7f80u) != 0x7f80u;
#pragma unroll
    for (int p = 1; p < NP; ++p) {
        x -= bf16_up(b[p - 1]);
        b[p] = fin ? float_to_bf16_bits(x) : 0u;
    }
}

// Element c of plane k in a row of three planes: they lie beside each other, 32 of each in turn, or `plane` elements apart
template <bool BESIDE> __device__ __forceinline__ size_t plane_at(int c, int k, size_t plane) {
    if constexpr (BESIDE) return (size_t)(c >> 5) * 96 + k * 32 + (c & 31);
    else return k * plane + c;
}

// ---------------------------------------------------------------------------------------------------------------------------------
// Operands in the form the products want: rows of `width` elements a plane (a multiple of 8, of 32 in three planes), zeros behind the last
// ---------------------------------------------------------------------------------------------------------------------------------
template <class T, int NP> __global__ __launch_bounds__(256) void ce_pack_kernel(const CePack x, const CePack w) {
    const bool first = (int)blockIdx.x < x.blocks;
    const CePack& a = first ? x : w;
    const T* const src = reinterpret_cast<const T*>(a.src);
    unsigned short* const dst = reinterpret_cast<unsigned short*>(a.dst);
    constexpr int E = 4;                                          // elements of a thread: its loads lie beside its neighbours'
    const int cpr = a.width / E;
    const size_t n = (size_t)a.rows * cpr;
    const bool vec = a.ld % E == 0;                               // (the first row is aligned)
    for (size_t t = (size_t)(blockIdx.x - (first ? 0 : x.blocks)) * 256 + threadIdx.x; t < n; t += (size_t)a.blocks * 256) {
        const int r = (int)(t / cpr), c = (int)(t - (size_t)r * cpr) * E;
        const T* s = src + (size_t)r * a.ld + c;
        unsigned short out[NP][E];
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int e = 0; e < E; ++e) out[0][e] = c + e < a.cols ? reinterpret_cast<const unsigned short*>(s)[e] : 0;
        } else {
            f32x4 v = {0.f, 0.f, 0.f, 0.f};
            if (vec && c + E <= a.cols) v = *reinterpret_cast<const f32x4*>(s);
            else
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (c + e < a.cols) v[e] = s[e];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                unsigned b[NP];
                split_bf16<NP>(v[e], b);
#pragma unroll
                for (int p = 0; p < NP; ++p) out[p][e] = (unsigned short)b[p];
            }
        }
#pragma unroll
        for (int p = 0; p < NP; ++p)
            *reinterpret_cast<u32x2*>(dst + (size_t)r * (NP * a.width) + (NP == 3 ? plane_at<true>(c, p, 0) : c)) = u32x2{out[p][0] | ((unsigned)out[p][1] << 16), out[p][2] | ((unsigned)out[p][3] << 16)};
    }
}

__device__ __forceinline__ bool is_class(int y, int V) { return (unsigned)y < (unsigned)V; }

// bit n & 63 of word n >> 6: row n counts; and how many do.  By one workgroup, beside those that form the probabilities.
__device__ __forceinline__ void ce_labels(const int* __restrict__ labels, int N, int V, unsigned long long* __restrict__ mask, int* __restrict__ count, int* s) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, nw = blockDim.x >> 6;
    int c = 0;
    for (int n0 = wave * 64; n0 < N; n0 += 64 * nw) {
        const int n = n0 + lane;
        const unsigned long long m = __ballot(n < N && is_class(labels[n < N ? n : 0], V));
        c += __popcll(m);
        if (lane == 0) mask[n0 >> 6] = m;
    }
    if (lane == 0) s[wave] = c;
    __syncthreads();
    if (threadIdx.x == 0) {
        int t = 0;
        for (int i = 0; i < nw; ++i) t += s[i];
        *count = t;
    }
}

// ---------------------------------------------------------------------------------------------------------------------------------
// l = X W^T: rows i are classes, columns j are samples, so that a lane has four consecutive classes of one sample and the
// statistics of a sample are sums inside a lane and over two lanes
// ---------------------------------------------------------------------------------------------------------------------------------
enum LogitsMode { LM_STATS, LM_PROB, LM_SLICE, LM_SUM };

// parts of 32 samples' probabilities that fit into LDS for all waves at once
template <class T> constexpr int prob_parts() { return 3 * T::NW * 32 * (T::TI * 2 + 16) <= 160 * 1024 ? 3 : 2; }

template <class T, int MODE, int WAVES> __global__ __launch_bounds__(T::NT, WAVES) void ce_logits_kernel(const CeLogits a) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    if constexpr (MODE == LM_PROB)
        if ((int)blockIdx.x == a.tiles_i * a.tiles_j) { ce_labels(a.labels, a.N, a.V_all, a.mask, a.count, reinterpret_cast<int*>(smem)); return; }
    int ti, tj;
    gemm_tile_of(blockIdx.x, a.tiles_i * a.tiles_j, a.tiles_i, a.tiles_j, a.band, ti, tj);
    const int i0 = ti * T::BI, j0 = tj * T::BJ;
    typename T::Acc acc;
#pragma unroll
    for (int i = 0; i < T::TI / 32; ++i)
#pragma unroll
        for (int j = 0; j < T::TJ / 32; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    if ((MODE == LM_STATS || MODE == LM_SLICE) && a.ticket && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *a.ticket = 0;
    const int kb = blockIdx.y * a.kchunk;
    T::run(a.w, a.x, a.pairs, i0, j0, kb, min(a.K, kb + a.kchunk), (GemmMask)nullptr, smem, acc);

    if (T::idle()) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wi = wave / (T::BJ / T::TJ), wj = wave % (T::BJ / T::TJ);
    const int lr = lane & 31, h = lane >> 5;
    const int ib = i0 + wi * T::TI, jb = j0 + wj * T::TJ;      // first class of the piece, first sample of this wave
    constexpr int FI = T::TI / 32, FJ = T::TJ / 32;

    if constexpr (MODE == LM_SLICE) {
        float* const out = a.slices + (size_t)blockIdx.y * a.slice;
#pragma unroll
        for (int j = 0; j < FJ; ++j) {
            const int n = jb + j * 32 + lr;
            if (n >= a.N) continue;
#pragma unroll
            for (int i = 0; i < FI; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int v = ib + i * 32 + 8 * q + 4 * h;
                    if (v < a.ldv) *reinterpret_cast<f32x4*>(out + (size_t)n * a.ldv + v) = f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                }
        }
        return;
    }
    // with the bias; classes beyond the last: minus infinity
    const bool ragged = i0 + T::BI > a.V;
#pragma unroll
    for (int i = 0; i < FI; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int v = ib + i * 32 + T::row(r, lane);
            const float b = a.bias ? a.bias[min(v, a.V - 1)] : 0.f;
#pragma unroll
            for (int j = 0; j < FJ; ++j) {
                acc[i][j][r] += b;
                if (ragged && v >= a.V) acc[i][j][r] = -kInf;
            }
        }
    if constexpr (MODE == LM_STATS) {
#pragma unroll
        for (int j = 0; j < FJ; ++j) {
            const int n = jb + j * 32 + lr;
            // the label's logit is handed on and left out here, by the lane that has it (few waves have one): what the other classes
            // have beside it is then never the difference of two numbers that are nearly one
            const int y = n < a.N ? a.labels[n] : -1, at = is_class(y, a.V) ? y - ib - 4 * h : -1;
            if (__any(at >= 0 && at < T::TI)) {
#pragma unroll
                for (int i = 0; i < FI; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (at == i * 32 + 8 * (r >> 2) + (r & 3)) { a.own[n] = acc[i][j][r]; acc[i][j][r] = -kInf; }
            }
            float m = -kInf;
#pragma unroll
            for (int i = 0; i < FI; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) m = fmaxf(m, acc[i][j][r]);
            m = fmaxf(m, __shfl_xor(m, 32));
            const float m0 = m == -kInf ? 0.f : m;              // nothing but minus infinity: a sum of zero
            float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < FI; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r & 3] += __builtin_amdgcn_exp2f((acc[i][j][r] - m0) * kLog2e);
            float t = (s[0] + s[1]) + (s[2] + s[3]);
            t += __shfl_xor(t, 32);
            if (h == 0 && n < a.N) a.partial[(size_t)n * a.parts + ti * (T::BI / T::TI) + wi] = make_float2(m, t);
        }
    } else {
        // probabilities: 32 samples of the wave at a time through LDS, from where they go out as 16-byte pieces of rows; as many of
        // their parts at once as LDS holds, what is left of a probability stays in its accumulator
        constexpr int NP = 3, PITCH = T::TI * 2 + 16, EP = 32 * PITCH, CPR = T::TI / 8, RPL = 64 / CPR, AT_ONCE = prob_parts<T>();
        constexpr int UNROLL = FI > 2 ? 1 : 8;                     // (256 x 256: the addresses of all rows do not fit into the registers beside the accumulators)
        unsigned char* const E0 = smem + wave * (AT_ONCE * EP);
        const int c = lane % CPR, jr = lane / CPR;
        float cs[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) cs[e] = 0.f;
#pragma unroll
        for (int j = 0; j < FJ; ++j) {
            const int n = jb + j * 32 + lr;
            const int y = n < a.N ? a.labels[n] : -1;
            const bool valid = is_class(y, a.V_all);
            const float lse = n < a.N ? a.lse[n] : 0.f;
            // the label's class, where this lane has it
            const int at = valid ? y - a.v0 - ib - 4 * h : -1;
            const bool here = __any(at >= 0 && at < T::TI);
            float own = 0.f, s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < FI; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][j][r] = valid ? __builtin_amdgcn_exp2f((acc[i][j][r] - lse) * kLog2e) : 0.f;
            if (here) {
#pragma unroll
                for (int i = 0; i < FI; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (at == i * 32 + 8 * (r >> 2) + (r & 3)) { own = acc[i][j][r]; acc[i][j][r] = 0.f; }
            }
            if (a.others) {
#pragma unroll
                for (int i = 0; i < FI; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[r & 3] += acc[i][j][r];
                float t = (s[0] + s[1]) + (s[2] + s[3]);
                t += __shfl_xor(t, 32);
                if (h == 0 && n < a.N) a.others[(size_t)n * a.parts + ti * (T::BI / T::TI) + wi] = t;
            }
            if constexpr (MODE == LM_SUM) continue;
            if (here) {
                // p - 1; where p is near one the difference has lost what tells them apart, and minus the sum of the others stands in for it, now
                // (dlabel) or as soon as it is known
                const float d = own > 0.5f ? (a.dlabel && at >= 0 && at < T::TI ? a.dlabel[n] : 0.f) : own - 1.f;
#pragma unroll
                for (int i = 0; i < FI; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (at == i * 32 + 8 * (r >> 2) + (r & 3)) acc[i][j][r] = d;
            }
#pragma unroll
            for (int k0 = 0; k0 < NP; k0 += AT_ONCE) {
#pragma unroll
                for (int i = 0; i < FI; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        unsigned char* const d = E0 + lr * PITCH + (i * 32 + 8 * q + 4 * h) * 2;
                        float p[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) p[e] = acc[i][j][4 * q + e];
#pragma unroll
                        for (int k = k0; k < NP && k < k0 + AT_ONCE; ++k) {
                            const unsigned lo = pack_bf16x2(p[0], p[1]), hi = pack_bf16x2(p[2], p[3]);
                            *reinterpret_cast<u32x2*>(d + (k - k0) * EP) = u32x2{lo, hi};
                            p[0] -= __uint_as_float(lo << 16); p[1] -= __uint_as_float(lo & 0xffff0000u);
                            p[2] -= __uint_as_float(hi << 16); p[3] -= __uint_as_float(hi & 0xffff0000u);
                        }
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][j][4 * q + e] = p[e];
                    }
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                __builtin_amdgcn_s_waitcnt(0xc07f);
                const int v = ib + c * 8;
#pragma unroll UNROLL
                for (int t = 0; t < 32 / RPL; ++t) {
                    const int row = t * RPL + jr, no = jb + j * 32 + row;
#pragma unroll
                    for (int k = k0; k < NP && k < k0 + AT_ONCE; ++k) {
                        const u32x4 w = *reinterpret_cast<const u32x4*>(E0 + (k - k0) * EP + row * PITCH + c * 16);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            cs[2 * e] += __uint_as_float(w[e] << 16);
                            cs[2 * e + 1] += __uint_as_float(w[e] & 0xffff0000u);
                        }
                        if (no < a.N && v < a.ldv) *reinterpret_cast<u32x4*>(a.prob + ((size_t)no * a.ldp + plane_at<T::TRIPLE>(v, k, a.pplane / 2)) * 2) = w;
                    }
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
                __builtin_amdgcn_s_waitcnt(0xc07f);              // read before the next ones overwrite it
            }
        }
        if (MODE == LM_PROB && a.colsum) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll
                for (int o = CPR; o < 64; o <<= 1) cs[e] += __shfl_xor(cs[e], o);
            const int v = ib + c * 8;
            if (jr == 0 && v < a.ld_colsum) {
                float* const d = a.colsum + (size_t)(tj * (T::BJ / T::TJ) + wj) * a.ld_colsum + v;
                *reinterpret_cast<f32x4*>(d) = f32x4{cs[0], cs[1], cs[2], cs[3]};
                *reinterpret_cast<f32x4*>(d + 4) = f32x4{cs[4], cs[5], cs[6], cs[7]};
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------------------------------------------
// The end of the forward pass.  (m, s) of the tiles (or the partial logits themselves), all of it without the label's class, and the
// label's logit to lse, the row's loss and every workgroup's sum of them; a last small kernel (or the only workgroup) adds those up.  WPR waves a row: one, or four where rows
// are few or their logits come in slices.
// ---------------------------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void join(float& m, float& s, float m2, float s2) {
    const float t = fmaxf(m, m2), t0 = t == -kInf ? 0.f : t;
    s = s * __builtin_amdgcn_exp2f((m - t0) * kLog2e) + s2 * __builtin_amdgcn_exp2f((m2 - t0) * kLog2e);
    m = t;
}

// sums of the slices of two logits, eight slices requested at once
__device__ __forceinline__ float2 sliced(const float* p, size_t slice, int n) {
    float2 l = make_float2(0.f, 0.f);
    int k = 0;
    for (; k + 8 <= n; k += 8) {
        float2 t[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) t[q] = *reinterpret_cast<const float2*>(p + (k + q) * slice);
#pragma unroll
        for (int q = 0; q < 8; ++q) { l.x += t[q].x; l.y += t[q].y; }
    }
    for (; k < n; ++k) { const float2 t = *reinterpret_cast<const float2*>(p + k * slice); l.x += t.x; l.y += t.y; }
    return l;
}

// sum of n losses and number of rows, by a workgroup of 256.  AGENT: of values that other workgroups of the same launch have stored
template <bool AGENT> __device__ __forceinline__ void ce_total(const float* sums, const int* counts, int n, float* loss) {
    __shared__ double s_t[4];
    __shared__ int s_c[4];
    const int tid = threadIdx.x;
    double t = 0.0;
    int c = 0;
#pragma unroll 4
    for (int b = tid; b < n; b += 256) {
        t += AGENT ? __hip_atomic_load(sums + b, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : sums[b];
        c += AGENT ? __hip_atomic_load(counts + b, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : counts[b];
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { t += __shfl_xor(t, o); c += __shfl_xor(c, o); }
    if ((tid & 63) == 0) { s_t[tid >> 6] = t; s_c[tid >> 6] = c; }
    __syncthreads();
    if (tid == 0) {
        const int all = s_c[0] + s_c[1] + s_c[2] + s_c[3];
        *loss = (float)(((s_t[0] + s_t[1]) + (s_t[2] + s_t[3])) / (double)(all > 1 ? all : 1));
    }
}
__global__ __launch_bounds__(256) void ce_total_kernel(const float* sums, const int* counts, int n, float* loss) { ce_total<false>(sums, counts, n, loss); }

template <bool SLICES, int WPR> __global__ __launch_bounds__(256) void ce_rows_kernel(const CeRows a) {
    __shared__ float s_m[4], s_s[4], s_own[4], s_loss[4];
    __shared__ int s_cnt[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = blockIdx.x * (4 / WPR) + wave / WPR;
    const int part = wave % WPR, l0 = part * 64 + lane;
    constexpr int STEP = 64 * WPR;
    float loss = 0.f, m = -kInf, s = 0.f, own = 0.f;
    int y = -1;
    bool valid = false;
    if (n < a.N) {
        y = a.labels[n];
        valid = is_class(y, a.V);
        if constexpr (SLICES) {
            const float* const row = a.slices + (size_t)n * a.ldv;
            for (int v = 2 * l0; v < a.V; v += 2 * STEP) {
                float2 l = sliced(row + v, a.slice, a.nslices);
                if (a.bias) { l.x += a.bias[v]; l.y += v + 1 < a.V ? a.bias[v + 1] : 0.f; }
                if (v == y) own = l.x;
                else join(m, s, l.x, 1.f);
                if (v + 1 == y) own = l.y;
                else if (v + 1 < a.V) join(m, s, l.y, 1.f);
            }
        } else {
            const float2* const row = a.partial + (size_t)n * a.parts;
            int t = l0;
            for (; t + 3 * STEP < a.parts; t += 4 * STEP) {
                float2 v[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) v[q] = row[t + q * STEP];
#pragma unroll
                for (int q = 0; q < 4; ++q) join(m, s, v[q].x, v[q].y);
            }
            for (; t < a.parts; t += STEP) { const float2 v = row[t]; join(m, s, v.x, v.y); }
            if (valid && l0 == 0) own = a.own[n];
        }
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const float m2 = __shfl_xor(m, o), s2 = __shfl_xor(s, o);
            join(m, s, m2, s2);
            own += __shfl_xor(own, o);
        }
    }
    if constexpr (WPR == 4) {
        if (lane == 0) { s_m[wave] = m; s_s[wave] = s; s_own[wave] = own; }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if (w == 0) { m = s_m[0]; s = s_s[0]; own = s_own[0]; }
            else { join(m, s, s_m[w], s_s[w]); own += s_own[w]; }
        }
    }
    if (n < a.N && part == 0) {
        const float mo = m, so = s;                              // of the other classes, where there is a label
        if (valid) join(m, s, own, 1.f);
        const float ls = __builtin_amdgcn_logf(s) * kLn2, lse = m + ls;      // (log2)
        // Of a row that is all but certain the logits cancel first, and what the other classes have is not added to one: its loss is
        // never negative and has all its digits.  (Classes at the type's lowest value have logits that only differences can hold.)
        if (!valid) loss = 0.f;
        else if (lse != lse) loss = lse;
        else if (mo - own < 5.f) loss = log1pf(so * __builtin_amdgcn_exp2f((mo - own) * kLog2e));
        else loss = (m - own) + ls;
        if (lane == 0) {
            a.lse[n] = lse;
            if (a.row_loss) a.row_loss[n] = loss;
        }
    }
    if (lane == 0) { s_loss[wave] = loss; s_cnt[wave] = part == 0 && valid ? 1 : 0; }
    __syncthreads();
    const float sum = (s_loss[0] + s_loss[1]) + (s_loss[2] + s_loss[3]);
    const int cnt = s_cnt[0] + s_cnt[1] + s_cnt[2] + s_cnt[3];
    if (!a.ticket) {
        if (tid == 0) { a.bsum[blockIdx.x] = sum; a.bcnt[blockIdx.x] = cnt; }
        return;
    }
    // Few workgroups: the one that finishes last adds up.  It is found by a count of those that have stored, whose order is of no account
    // to the sums.  Stores and loads of these values go past the L2 of their own die, and a store has arrived before it is counted.
    __shared__ int s_last;
    if (tid == 0) {
        __hip_atomic_store(a.bsum + blockIdx.x, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(a.bcnt + blockIdx.x, cnt, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        s_last = __hip_atomic_fetch_add(a.ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
    }
    __syncthreads();
    if (s_last) ce_total<true>(a.bsum, a.bcnt, gridDim.x, a.loss);
}

// Behind the tiles' sums of the probabilities of all classes but the label's, a wave a row: the label's own where p > 1/2 (what the tiles left
// at zero; any other is -1/2 or below) goes into the parts, and to dlabel for the bias.
template <bool BESIDE> __global__ __launch_bounds__(256) void ce_label_kernel(const CeLabel a) {
    const int n = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (n >= a.N) return;
    const int y = a.labels[n];
    unsigned short* const row = a.prob + (size_t)n * a.ldp;
    const bool left = is_class(y, a.V) && (row[plane_at<BESIDE>(is_class(y, a.V) ? y : 0, 0, a.pplane / 2)] & 0x7fffu) == 0;
    float t = 0.f;
    if (left) {
#pragma unroll 4
        for (int k = lane; k < a.parts; k += 64) t += a.others[(size_t)n * a.parts + k];
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) t += __shfl_xor(t, o);
    }
    if (lane == 0) a.dlabel[n] = -t;
    if (!left || lane != 0) return;
    unsigned b[3];
    split_bf16<3>(-t, b);
#pragma unroll
    for (int k = 0; k < 3; ++k) row[plane_at<BESIDE>(y, k, a.pplane / 2)] = (unsigned short)b[k];
}
// Where the classes come in pieces: minus the sum over all of them, piece by piece, ahead of the probabilities
__global__ __launch_bounds__(256) void ce_others_kernel(const CeLabel a, bool first) {
    const int n = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (n >= a.N) return;
    float t = 0.f;
#pragma unroll 4
    for (int k = lane; k < a.parts; k += 64) t += a.others[(size_t)n * a.parts + k];
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) t += __shfl_xor(t, o);
    if (lane == 0) a.dlabel[n] = (first ? 0.f : a.dlabel[n]) - t;
}

// Probabilities from partial logits (few tiles): a workgroup a row
template <bool BESIDE> __global__ __launch_bounds__(256) void ce_prob_kernel(const CeRows a, unsigned short* __restrict__ prob, size_t pplane, int ldp) {
    constexpr int NP = 3;
    __shared__ int s_cnt[4];
    const int n = blockIdx.x;
    if (n == a.N) { ce_labels(a.labels, a.N, a.V, a.mask, a.count, s_cnt); return; }
    const int y = a.labels[n];
    const bool valid = is_class(y, a.V);
    const float lse = a.lse[n];
    const float* const row = a.slices + (size_t)n * a.ldv;
    // the label's p - 1, where p is near one, as minus the sum of the others: 1 - p would lose what tells them apart
    __shared__ float s_others[4];
    float others = 0.f, mine[2] = {0.f, 0.f};
    int at = -1;                                                  // this thread has the label's pair
    auto store = [&](int v, const float (&p)[2]) __attribute__((always_inline)) {
        unsigned b[2][NP];
#pragma unroll
        for (int e = 0; e < 2; ++e) split_bf16<NP>(p[e], b[e]);
#pragma unroll
        for (int k = 0; k < NP; ++k) *reinterpret_cast<unsigned*>(prob + (size_t)n * ldp + plane_at<BESIDE>(v, k, pplane / 2)) = b[0][k] | (b[1][k] << 16);
    };
    for (int v = threadIdx.x * 2; v < a.ldv; v += 512) {
        const float2 l = sliced(row + v, a.slice, a.nslices);
        float p[2] = {0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 2; ++e)
            if (valid && v + e < a.V) {
                p[e] = __builtin_amdgcn_exp2f(((e ? l.y : l.x) + (a.bias ? a.bias[v + e] : 0.f) - lse) * kLog2e);
                if (v + e != y) others += p[e];
            }
        if (valid && (v == y || v + 1 == y)) { at = v; mine[0] = p[0]; mine[1] = p[1]; }
        else store(v, p);
    }
    if (!valid) return;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) others += __shfl_xor(others, o);
    if ((threadIdx.x & 63) == 0) s_others[threadIdx.x >> 6] = others;
    __syncthreads();
    if (at < 0) return;
    others = (s_others[0] + s_others[1]) + (s_others[2] + s_others[3]);
    float& p = y == at ? mine[0] : mine[1];
    p = p > 0.5f ? -others : p - 1.f;
    store(at, mine);
}

// ---------------------------------------------------------------------------------------------------------------------------------
// The two gradient products: rows i are channels, columns j are samples (dX) or classes (dW)
// ---------------------------------------------------------------------------------------------------------------------------------
template <class T, int WAVES> __global__ __launch_bounds__(T::NT, WAVES) void ce_grad_kernel(const CeGrad a) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    int ti, tj;
    gemm_tile_of(blockIdx.x, a.tiles_i * a.tiles_j, a.tiles_i, a.tiles_j, a.band, ti, tj);
    const int i0 = ti * T::BI, j0 = tj * T::BJ;
    typename T::Acc acc;
#pragma unroll
    for (int i = 0; i < T::TI / 32; ++i)
#pragma unroll
        for (int j = 0; j < T::TJ / 32; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    const int kb = blockIdx.y * a.kchunk;
    T::run(a.a, a.b, a.pairs, i0, j0, kb, min(a.K, kb + a.kchunk), (GemmMask)a.mask, smem, acc);

    if (T::idle()) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wi = wave / (T::BJ / T::TJ), wj = wave % (T::BJ / T::TJ);
    const int lr = lane & 31, h = lane >> 5;
    const float g = a.count ? a.scale / (float)max(*a.count, 1) : 1.f;
    float* const out = a.out + (size_t)blockIdx.y * a.slice;
    if (a.last) {  // dX itself
#pragma unroll
        for (int j = 0; j < T::TJ / 32; ++j) {
            const int n = j0 + wj * T::TJ + j * 32 + lr;
            if (n >= a.J) continue;
            const bool live = is_class(a.labels[n], a.V_all);
#pragma unroll
            for (int i = 0; i < T::TI / 32; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int c = i0 + wi * T::TI + i * 32 + 8 * q + 4 * h;
                    if (c >= a.C) continue;
                    f32x4 v = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                    if (a.add) v += *reinterpret_cast<const f32x4*>(out + (size_t)n * a.ldo + c);
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = live ? v[e] * g : 0.f;
                    if (a.low) {
                        unsigned short* const d = reinterpret_cast<unsigned short*>(a.last) + (size_t)n * a.ldlast + c;
                        if (a.vec_last) *reinterpret_cast<u32x2*>(d) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
                        else
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (c + e < a.C) d[e] = float_to_bf16_bits(v[e]);
                    } else {
                        float* const d = reinterpret_cast<float*>(a.last) + (size_t)n * a.ldlast + c;
                        if (a.vec_last) *reinterpret_cast<f32x4*>(d) = v;
                        else
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (c + e < a.C) d[e] = v[e];
                    }
                }
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < T::TJ / 32; ++j) {
        const int col = j0 + wj * T::TJ + j * 32 + lr;
        if (col >= a.J) continue;
#pragma unroll
        for (int i = 0; i < T::TI / 32; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int c = i0 + wi * T::TI + i * 32 + 8 * q + 4 * h;
                float* const d = out + (size_t)col * a.ldo + c;
                f32x4 v = {acc[i][j][4 * q] * g, acc[i][j][4 * q + 1] * g, acc[i][j][4 * q + 2] * g, acc[i][j][4 * q + 3] * g};
                if (a.vec) {
                    if (c < a.I) {
                        if (a.add) v += *reinterpret_cast<const f32x4*>(d);
                        *reinterpret_cast<f32x4*>(d) = v;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (c + e < a.I) d[e] = v[e];
                }
            }
    }
}

// Sums of the partial results, scaled, rounded to the type of the gradient; rows without a class are zero.  And the bias.
template <class T> __global__ __launch_bounds__(256) void ce_finish_kernel(const CeFinish a) {
    const float g = a.scale / (float)max(*a.count, 1);
    const int b = blockIdx.x;
    if (b < a.blocks_x + a.blocks_w) {
        const bool x = b < a.blocks_x;
        const CeSum& s = x ? a.x : a.w;
        // vectors by 64 >> lg lanes of a wave, their slices in 1 << lg parts
        const int lg = s.parts_log, lane = threadIdx.x & 63, span = 64 >> lg, part = lane >> (6 - lg);
        const size_t wave = (size_t)(x ? b : b - a.blocks_x) * 4 + (threadIdx.x >> 6), stride = (size_t)(x ? a.blocks_x : a.blocks_w) * 4 * span;
        const int vpr = (s.cols + 3) >> 2;
        const size_t n = (size_t)s.rows * vpr;
        for (size_t base = wave * span; base < n; base += stride) {      // (the whole wave together)
            const size_t t = min(base + (lane & (span - 1)), n - 1);
            const int r = (int)(t / vpr), c = (int)(t - (size_t)r * vpr) * 4;
            const float* const p = s.part + (size_t)r * s.ldp + c;
            f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
            for (int k = part; k < s.nslices; k += 1 << lg) v += *reinterpret_cast<const f32x4*>(p + k * s.slice);
            for (int o = span; o < 64; o <<= 1)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += __shfl_xor(v[e], o);
            if (base + lane >= n || part != 0) continue;
            const bool live = !x || is_class(a.labels[r], a.V_all);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = live ? v[e] * g : 0.f;
            if (x) {
                T* const d = reinterpret_cast<T*>(s.out) + (size_t)r * s.ldo + c;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (c + e < s.cols) d[e] = from_float<T>(v[e]);
            } else {
                float* const d = reinterpret_cast<float*>(s.out) + (size_t)r * s.ldo + c;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (c + e < s.cols) d[e] = v[e];
            }
        }
        return;
    }
    if (a.colsum) {  // bias from the tiles' sums: 32 classes a workgroup, eight groups of threads a part of the tiles each
        __shared__ float s_b[8][32];
        extern __shared__ float s_l[];                            // [32][257]: every thread's sums of the label's share, of the rows it has
        const int col = threadIdx.x & 31, grp = threadIdx.x >> 5, v0 = (b - a.blocks_x - a.blocks_w) * 32, v = v0 + col;
        float t = 0.f;
        if (a.dlabel) {
            constexpr int PITCH = 257;
            float* const mine = s_l + threadIdx.x;
#pragma unroll
            for (int k = 0; k < 32; ++k) mine[k * PITCH] = 0.f;
            constexpr int R = 16;                                 // rows whose loads are under way together
            for (int n0 = threadIdx.x; n0 < a.N; n0 += 256 * R) {
                int y[R];
                float d[R];
#pragma unroll
                for (int q = 0; q < R; ++q) {
                    const int n = min(n0 + q * 256, a.N - 1);
                    y[q] = a.labels[n];
                    d[q] = a.dlabel[n];
                }
#pragma unroll
                for (int q = 0; q < R; ++q) {
                    const unsigned k = (unsigned)(y[q] - v0);
                    if (n0 + q * 256 < a.N && k < 32u) mine[k * PITCH] += d[q];
                }
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < 32; ++k) t += s_l[col * PITCH + grp * 32 + k];
        }
        if (v < a.V) {
#pragma unroll 8
            for (int k = grp; k < a.parts; k += 8) t += a.colsum[(size_t)k * a.ld_colsum + v];
        }
        s_b[grp][col] = t;
        __syncthreads();
        if (grp == 0 && v < a.V) {
            for (int k = 1; k < 8; ++k) t += s_b[k][col];
            a.dbias[v] = t * g;
        }
        return;
    }
    // bias from the planes of P: eight classes a workgroup, a thread reads them in 16 bytes and takes every 256th row (3399 rows of
    // 22 classes in three planes: 32 classes a workgroup and an element a load, 1300 loads in a chain, took 300 us).  P's rows are padded
    // to whole eight classes.
    __shared__ float s_p[4][8];
    const int v0 = (b - a.blocks_x - a.blocks_w) * 8;
    float t[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < 3; ++p) {
        const unsigned short* const q = a.prob + (a.beside ? plane_at<true>(v0, p, 0) : plane_at<false>(v0, p, a.pplane / 2));
#pragma unroll 4
        for (int n = threadIdx.x; n < a.N; n += 256) {
            const u32x4 u = *reinterpret_cast<const u32x4*>(q + (size_t)n * a.ldp);
#pragma unroll
            for (int e = 0; e < 4; ++e) { t[2 * e] += __uint_as_float(u[e] << 16); t[2 * e + 1] += __uint_as_float(u[e] & 0xffff0000u); }
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) t[e] += __shfl_xor(t[e], o);
        if ((threadIdx.x & 63) == 0) s_p[threadIdx.x >> 6][e] = t[e];
    }
    __syncthreads();
    if (threadIdx.x < 8 && v0 + (int)threadIdx.x < a.V) {
        float u = 0.f;
        for (int w = 0; w < 4; ++w) u += s_p[w][threadIdx.x];
        a.dbias[v0 + threadIdx.x] = u * g;
    }
}

__global__ __launch_bounds__(256) void ce_zero_kernel(float* p, size_t n) {
    for (size_t t = (size_t)blockIdx.x * 256 + threadIdx.x; t < n; t += (size_t)gridDim.x * 256) p[t] = 0.f;
}

// tiles: big and middle (one workgroup a compute unit), small (two), few samples
template <bool AKR, bool BKR, bool M> using TBig = GemmTile<bf16_t, AKR, BKR, 2, 4, 4, 2, 2, M>;
template <bool AKR, bool BKR, bool M> using TMid = GemmTile<bf16_t, AKR, BKR, 2, 2, 2, 2, 4, M>;
template <bool AKR, bool BKR, bool M> using TSmall = GemmTile<bf16_t, AKR, BKR, 2, 2, 1, 1, 4, M>;
template <bool AKR, bool BKR, bool M> using TFew = GemmTile<bf16_t, AKR, BKR, 4, 1, 1, 1, 3, M>;
// ... of three planes
template <bool AKR, bool BKR, bool M> using TMid3 = GemmTile<bf16_t, AKR, BKR, 2, 2, 2, 2, 3, M, 3>;
template <bool AKR, bool BKR, bool M> using TSmall3 = GemmTile<bf16_t, AKR, BKR, 2, 2, 1, 1, 3, M, 3>;

template <class K, class A> hipError_t launch(K kernel, OncePerDevice& once, dim3 grid, int threads, int lds, hipStream_t s, const A& args) {
    if (const hipError_t e = raise_lds_limit(once, {(const void*)kernel}, lds); e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, grid, dim3(threads), lds, s, args);
    return hipGetLastError();
}

template <class T, int MODE, int WAVES> hipError_t launch_logits_t(const CeLogits& a, int slices, hipStream_t s) {
    static OncePerDevice once;
    constexpr int EP = MODE == LM_PROB ? T::NW * prob_parts<T>() * 32 * (T::TI * 2 + 16) : 0;
    return launch(ce_logits_kernel<T, MODE, WAVES>, once, dim3(a.tiles_i * a.tiles_j + (MODE == LM_PROB ? 1 : 0), slices), T::NT, std::max(T::LDS, EP), s, a);
}
template <class T, int WAVES> hipError_t launch_grad_t(const CeGrad& a, int slices, hipStream_t s) {
    static OncePerDevice once;
    return launch(ce_grad_kernel<T, WAVES>, once, dim3(a.tiles_i * a.tiles_j, slices), T::NT, T::LDS, s, a);
}

}  // namespace

// Time of a product cut into `blocks` workgroups of `ktiles` k-tiles each, microseconds: rounds of as many as run at once, a k-tile of a
// full chip and of a nearly empty one as measured (256 x 256 1.95 and 1.4 us, 128 x 128 0.52 and 0.36, 64 x 64 0.43 and 0.27, 128 x 32
// 0.40 and 0.25; of three planes, 32 k, 128 x 128 1.13 and 0.95, 64 x 64 0.7 to 0.85 and 0.4), and what a workgroup does besides.
double ce_tile_time(int cfg, long blocks, int ktiles) {
    static const struct { int slots; double some, full, rest; } t[6] = {{256, 1.4, 1.95, 6.0}, {256, 0.36, 0.52, 4.0}, {512, 0.27, 0.43, 3.0},
                                                                        {512, 0.25, 0.40, 3.0}, {256, 0.95, 1.13, 5.0}, {512, 0.4, 0.75, 4.0}};
    const long rounds = blocks / t[cfg].slots, over = blocks - rounds * t[cfg].slots;
    const double last = t[cfg].some + (t[cfg].full - t[cfg].some) * (double)over / t[cfg].slots;
    return (double)rounds * (t[cfg].rest + ktiles * t[cfg].full) + (over ? t[cfg].rest + ktiles * last : 0.0);
}

void ce_tile_size(int cfg, int* bi, int* bj, int* wi, int* wj) {
    static const int d[6][4] = {{256, 256, 2, 4}, {128, 128, 2, 2}, {64, 64, 2, 2}, {128, 32, 4, 1}, {128, 128, 2, 2}, {64, 64, 2, 2}};
    *bi = d[cfg][0]; *bj = d[cfg][1]; *wi = d[cfg][2]; *wj = d[cfg][3];
}

hipError_t launch_ce_pack(CePack x, CePack w, int dtype, hipStream_t s) {
    for (CePack* a : {&x, &w}) a->blocks = (int)std::min<size_t>(((size_t)a->rows * (a->width / 4) + 255) / 256, 1u << 16);
    const dim3 grid(x.blocks + w.blocks);
    if (grid.x == 0) return hipSuccess;
    if (dtype == 1) hipLaunchKernelGGL((ce_pack_kernel<bf16_t, 1>), grid, dim3(256), 0, s, x, w);
    else hipLaunchKernelGGL((ce_pack_kernel<float, 3>), grid, dim3(256), 0, s, x, w);
    return hipGetLastError();
}
hipError_t launch_ce_stats(const CeLogits& a, int cfg, hipStream_t s) {
    switch (cfg) {
        case 0: return launch_logits_t<TBig<false, false, false>, LM_STATS, 2>(a, 1, s);
        case 1: return launch_logits_t<TMid<false, false, false>, LM_STATS, 2>(a, 1, s);
        case 2: return launch_logits_t<TSmall<false, false, false>, LM_STATS, 2>(a, 1, s);
        case 3: return launch_logits_t<TFew<false, false, false>, LM_STATS, 2>(a, 1, s);
        case 4: return launch_logits_t<TMid3<false, false, false>, LM_STATS, 2>(a, 1, s);
        default: return launch_logits_t<TSmall3<false, false, false>, LM_STATS, 2>(a, 1, s);
    }
}
hipError_t launch_ce_prob_tiles(const CeLogits& a, int cfg, hipStream_t s) {
    switch (cfg) {
        case 0: return launch_logits_t<TBig<false, false, false>, LM_PROB, 2>(a, 1, s);
        case 1: return launch_logits_t<TMid<false, false, false>, LM_PROB, 2>(a, 1, s);
        case 2: return launch_logits_t<TSmall<false, false, false>, LM_PROB, 2>(a, 1, s);
        case 3: return launch_logits_t<TFew<false, false, false>, LM_PROB, 2>(a, 1, s);
        case 4: return launch_logits_t<TMid3<false, false, false>, LM_PROB, 2>(a, 1, s);
        default: return launch_logits_t<TSmall3<false, false, false>, LM_PROB, 2>(a, 1, s);
    }
}
hipError_t launch_ce_sums(const CeLogits& a, int cfg, hipStream_t s) {
    switch (cfg) {
        case 0: return launch_logits_t<TBig<false, false, false>, LM_SUM, 2>(a, 1, s);
        case 1: return launch_logits_t<TMid<false, false, false>, LM_SUM, 2>(a, 1, s);
        case 2: return launch_logits_t<TSmall<false, false, false>, LM_SUM, 2>(a, 1, s);
        case 3: return launch_logits_t<TFew<false, false, false>, LM_SUM, 2>(a, 1, s);
        case 4: return launch_logits_t<TMid3<false, false, false>, LM_SUM, 2>(a, 1, s);
        default: return launch_logits_t<TSmall3<false, false, false>, LM_SUM, 2>(a, 1, s);
    }
}
hipError_t launch_ce_label(const CeLabel& a, bool beside, hipStream_t s) {
    if (beside) hipLaunchKernelGGL(ce_label_kernel<true>, dim3((a.N + 3) / 4), dim3(256), 0, s, a);
    else hipLaunchKernelGGL(ce_label_kernel<false>, dim3((a.N + 3) / 4), dim3(256), 0, s, a);
    return hipGetLastError();
}
hipError_t launch_ce_others(const CeLabel& a, bool first, hipStream_t s) {
    hipLaunchKernelGGL(ce_others_kernel, dim3((a.N + 3) / 4), dim3(256), 0, s, a, first);
    return hipGetLastError();
}
hipError_t launch_ce_slices(const CeLogits& a, int slices, int cfg, hipStream_t s) {
    switch (cfg) {
        case 2: return launch_logits_t<TSmall<false, false, false>, LM_SLICE, 2>(a, slices, s);
        case 3: return launch_logits_t<TFew<false, false, false>, LM_SLICE, 2>(a, slices, s);
        default: return launch_logits_t<TSmall3<false, false, false>, LM_SLICE, 2>(a, slices, s);
    }
}
hipError_t launch_ce_rows(const CeRows& a, hipStream_t s) {
    // (a wave a row 9 us for 8192 rows of 256 parts and for 10000 of 172; four waves a row 5 for 777)
    const bool wide = a.slices || a.N < 2048;
    const int blocks = wide ? a.N : (a.N + 3) / 4;
    // counting workgroups costs 12 ns each (64 rows: 6.3 us against 5.6 and 1.7 of a launch for the sum; 777: 13.8 against 5.1 and 4.6)
    CeRows r = a;
    if (blocks > 128) r.ticket = nullptr;
    if (a.slices) hipLaunchKernelGGL((ce_rows_kernel<true, 4>), dim3(blocks), dim3(256), 0, s, r);
    else if (wide) hipLaunchKernelGGL((ce_rows_kernel<false, 4>), dim3(blocks), dim3(256), 0, s, r);
    else hipLaunchKernelGGL((ce_rows_kernel<false, 1>), dim3(blocks), dim3(256), 0, s, r);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess || r.ticket) return e;
    return launch_ce_total(a.bsum, a.bcnt, blocks, a.loss, s);
}
hipError_t launch_ce_total(const float* sums, const int* counts, int n, float* loss, hipStream_t s) {
    hipLaunchKernelGGL(ce_total_kernel, dim3(1), dim3(256), 0, s, sums, counts, n, loss);
    return hipGetLastError();
}
hipError_t launch_ce_prob(const CeRows& a, unsigned short* prob, size_t pplane, int ldp, bool beside, hipStream_t s) {
    if (!beside) hipLaunchKernelGGL(ce_prob_kernel<false>, dim3(a.N + 1), dim3(256), 0, s, a, prob, pplane, ldp);
    else hipLaunchKernelGGL(ce_prob_kernel<true>, dim3(a.N + 1), dim3(256), 0, s, a, prob, pplane, ldp);
    return hipGetLastError();
}
hipError_t launch_ce_dx(const CeGrad& a, int slices, int cfg, hipStream_t s) {
    switch (cfg) {
        case 0: return launch_grad_t<TBig<true, false, false>, 2>(a, slices, s);
        case 1: return launch_grad_t<TMid<true, false, false>, 2>(a, slices, s);
        case 2: return launch_grad_t<TSmall<true, false, false>, 2>(a, slices, s);
        case 3: return launch_grad_t<TFew<true, false, false>, 2>(a, slices, s);
        case 4: return launch_grad_t<TMid3<true, false, false>, 2>(a, slices, s);
        default: return launch_grad_t<TSmall3<true, false, false>, 2>(a, slices, s);
    }
}
hipError_t launch_ce_dw(const CeGrad& a, int slices, int cfg, hipStream_t s) {
    switch (cfg) {
        case 0: return launch_grad_t<TBig<true, true, true>, 2>(a, slices, s);
        case 1: return launch_grad_t<TMid<true, true, true>, 2>(a, slices, s);
        case 2: return launch_grad_t<TSmall<true, true, true>, 2>(a, slices, s);
        case 4: return launch_grad_t<TMid3<true, true, true>, 2>(a, slices, s);
        default: return launch_grad_t<TSmall3<true, true, true>, 2>(a, slices, s);
    }
}
hipError_t launch_ce_finish(const CeFinish& a, int dtype, hipStream_t s) {
    const int blocks = a.blocks_x + a.blocks_w + a.blocks_b;
    if (blocks == 0) return hipSuccess;
    const int lds = a.blocks_b && a.dlabel ? 32 * 257 * (int)sizeof(float) : 0;
    if (dtype == 1) hipLaunchKernelGGL(ce_finish_kernel<bf16_t>, dim3(blocks), dim3(256), lds, s, a);
    else hipLaunchKernelGGL(ce_finish_kernel<float>, dim3(blocks), dim3(256), lds, s, a);
    return hipGetLastError();
}
hipError_t launch_ce_zero(float* p, size_t n, hipStream_t s) {
    if (n == 0) return hipSuccess;
    hipLaunchKernelGGL(ce_zero_kernel, dim3((unsigned)std::min<size_t>((n + 255) / 256, 4096)), dim3(256), 0, s, p, n);
    return hipGetLastError();
}

}  // namespace lp
