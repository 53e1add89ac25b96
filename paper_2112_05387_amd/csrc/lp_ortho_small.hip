// Orthogonalisation of small matrices, from the momentum to the updated parameters in one workgroup (gfx950).
//
// The products of a matrix of at most 64 rows (a filter of a narrow network: 64 x 576) are a few microseconds of work and fifteen
// launches of it.  Here a workgroup of eight waves keeps X in LDS, both parts (147 KB of the 160), and S and B in the 16 KB beside
// it, in turn; what a product yields stays in registers until everybody has read what it replaces.  Precision and scales are
// those of the large matrices' products.  A step of 64 x 576 is 14 MFLOP in three products of fp16 parts and 7.5 us, of which the LDS reads
// of two products on the same 147 KB and the exchange of S and B between the waves are most; the three launches it replaces take 20.
// The whole matrix, read, five steps and written: 60 us, an update of 55 of them and 110 vectors 76.
//
// X lies in LDS as rows of 128-byte groups, 32 first parts and the same 32 second parts, S and B as rows of two groups.  The 16-byte
// chunks of every 256 bytes trade places by the row, F(row) = 4 (row & 3) + (row >> 2 & 3): 16 rows of a chunk lie on all banks (fragments
// with k along the row), and so do the two 32-byte pairs of four rows (transposing reads).
//
// The same launch updates the tensors that are no matrices, 4096 elements a workgroup.
#include <algorithm>

#include "lp_kernels.h"
#include "lp_ortho_dev.h"

namespace lp {
namespace {

constexpr int kThreads = 512;
typedef __attribute__((address_space(3))) void* lds_ptr_t;
typedef __attribute__((ext_vector_type(4))) short s16x4;

__device__ __forceinline__ int swap16(int row) { return ((row & 3) << 2) | ((row >> 2) & 3); }
// byte of 16-byte chunk q of a row
__device__ __forceinline__ int chunk_at(int row, int pitch, int q) { return row * pitch + ((q ^ swap16(row)) << 4); }

__device__ __forceinline__ u32x4 frag(const unsigned char* m, int row, int pitch, int q) { return *reinterpret_cast<const u32x4*>(m + chunk_at(row, pitch, q)); }
__device__ __forceinline__ u32x2 frag_tr(const unsigned char* m, int row, int pitch, int q, int sub) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(lds_ptr_t)const_cast<unsigned char*>(m + chunk_at(row, pitch, q) + sub)));
}
// the three products, each to a sum of its own: a chain through one would wait for every product's end
struct Sums { f32x16 lh, hl, hh; };
__device__ __forceinline__ void clear(f32x16& s) {
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.f;
}
__device__ __forceinline__ void clear(Sums& s) { clear(s.lh); clear(s.hl); clear(s.hh); }
__device__ __forceinline__ void three(const u32x4& ah, const u32x4& al, const u32x4& bh, const u32x4& bl, Sums& s) {
    Mma<f16_t, 32>::run(al, bh, s.lh);
    Mma<f16_t, 32>::run(ah, bl, s.hl);
    Mma<f16_t, 32>::run(ah, bh, s.hh);
}
__device__ __forceinline__ f32x16 total(const Sums& s) {
    f32x16 t;
#pragma unroll
    for (int e = 0; e < 16; ++e) t[e] = (s.lh[e] + s.hl[e]) + s.hh[e];
    return t;
}
// four consecutive values of a row, from column i on (a multiple of four), in two parts
__device__ __forceinline__ void put4(unsigned char* m, int row, int pitch, int i, const float (&v)[4]) {
    unsigned h0, h1, l0, l1;
    split_f16x2(v[0], v[1], h0, l0);
    split_f16x2(v[2], v[3], h1, l1);
    const int q = (i >> 5) * 8 + ((i & 31) >> 3), sub = (i & 7) * 2;
    *reinterpret_cast<u32x2*>(m + chunk_at(row, pitch, q) + sub) = u32x2{h0, h1};
    *reinterpret_cast<u32x2*>(m + chunk_at(row, pitch, q + 4) + sub) = u32x2{l0, l1};
}
__device__ __forceinline__ void get4(const unsigned char* m, int row, int pitch, int i, float (&v)[4]) {
    const int q = (i >> 5) * 8 + ((i & 31) >> 3), sub = (i & 7) * 2;
    const u32x2 h = *reinterpret_cast<const u32x2*>(m + chunk_at(row, pitch, q) + sub), l = *reinterpret_cast<const u32x2*>(m + chunk_at(row, pitch, q + 4) + sub);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = f16_up((h[e >> 1] >> (16 * (e & 1))) & 0xffffu) + f16_up((l[e >> 1] >> (16 * (e & 1))) & 0xffffu);
}

// NJ: 32-row tiles of X (one or two); NI: tiles of its columns a wave has at most (LDS holds 1152 columns of one, 576 of two)
template <int NJ, int NI> __device__ void small_matrix(const NsArgs& a, const NsProb& P, int steps, unsigned char* smem) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lr = lane & 31, kg = lane >> 5;
    const int rows = P.rows, cols = P.cols;
    const bool tall = rows > cols;
    const int r = tall ? cols : rows, c = tall ? rows : cols, c64 = (c + 63) >> 6 << 6, pitch = c64 * 4, ntile = c64 >> 5;
    constexpr int R = NJ * 32;
    unsigned char *const X = smem, *const S = smem + R * pitch;
    constexpr int SP = 256;

    // ---- the matrix, as fp32 where its two parts will lie; the momentum on the way; the sum of squares
    if (r != R || c != c64) {
        for (int i = tid * 16; i < R * pitch; i += kThreads * 16) *reinterpret_cast<u32x4*>(X + i) = u32x4{0u, 0u, 0u, 0u};
        __syncthreads();
    }
    const int numel = rows * cols;
    const float per_col = 1.f / (float)cols;
    double sum = 0.0;
    auto put = [&](int row, int col, float u) __attribute__((always_inline)) {
        const int xr = tall ? col : row, xc = tall ? row : col;
        *reinterpret_cast<float*>(X + chunk_at(xr, pitch, xc >> 2) + (xc & 3) * 4) = u;
        sum += (double)u * u;
    };
    auto row_of = [&](int e) __attribute__((always_inline)) {         // e / cols for e < 2^16
        const int row = (int)((float)e * per_col);
        return row + ((row + 1) * cols <= e ? 1 : 0) - (row * cols > e ? 1 : 0);
    };
    auto momentum = [&](float g, float& v) __attribute__((always_inline)) {
        v = fmaf(a.momentum, v, g);
        return a.nesterov ? fmaf(a.momentum, v, g) : v;
    };
    const int src_low = P.flags & NS_SRC_LOW;
    if ((P.flags & NS_VEC) && cols % 4 == 0) {
        constexpr int U = 4;
        for (int e0 = tid * 4; e0 < numel; e0 += kThreads * 4 * U) {
            f32x4 g[U], v[U];
#pragma unroll
            for (int q = 0; q < U; ++q) {
                const int e = e0 + q * kThreads * 4;
                if (e >= numel) continue;
                if (!P.src) { g[q] = *reinterpret_cast<const f32x4*>(P.grad + e); v[q] = *reinterpret_cast<const f32x4*>(P.vel + e); }
                else if (src_low) {
                    const u32x2 w = *reinterpret_cast<const u32x2*>(reinterpret_cast<const unsigned short*>(P.src) + e);
                    g[q] = f32x4{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xffff0000u), __uint_as_float(w[1] << 16), __uint_as_float(w[1] & 0xffff0000u)};
                } else g[q] = *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(P.src) + e);
            }
#pragma unroll
            for (int q = 0; q < U; ++q) {
                const int e = e0 + q * kThreads * 4;
                if (e >= numel) continue;
                const int row = row_of(e), col = e - row * cols;
                f32x4 u = g[q];
                if (!P.src) {
#pragma unroll
                    for (int t = 0; t < 4; ++t) { float vt = v[q][t]; u[t] = momentum(g[q][t], vt); v[q][t] = vt; }
                    *reinterpret_cast<f32x4*>(P.vel + e) = v[q];
                }
                if (!tall) {
                    *reinterpret_cast<f32x4*>(X + chunk_at(row, pitch, col >> 2)) = u;
#pragma unroll
                    for (int t = 0; t < 4; ++t) sum += (double)u[t] * u[t];
                } else {
#pragma unroll
                    for (int t = 0; t < 4; ++t) put(row, col + t, u[t]);
                }
            }
        }
    } else {
        // eight elements a thread and trip, all loads first
        constexpr int U = 8;
        for (int e0 = tid; e0 < numel; e0 += kThreads * U) {
            float g[U], v[U];
            auto from = [&](int q) __attribute__((always_inline)) {
                const int e = min(e0 + q * kThreads, numel - 1), row = row_of(e);
                return (size_t)row * P.ld_src + (e - row * cols);
            };
            if (P.src && src_low) {
#pragma unroll
                for (int q = 0; q < U; ++q) g[q] = bf16_bits_to_float(reinterpret_cast<const unsigned short*>(P.src)[from(q)]);
            } else if (P.src) {
#pragma unroll
                for (int q = 0; q < U; ++q) g[q] = reinterpret_cast<const float*>(P.src)[from(q)];
            } else {
#pragma unroll
                for (int q = 0; q < U; ++q) {
                    const int e = min(e0 + q * kThreads, numel - 1);
                    g[q] = P.grad[e]; v[q] = P.vel[e];
                }
            }
#pragma unroll
            for (int q = 0; q < U; ++q) {
                const int e = e0 + q * kThreads;
                if (e >= numel) continue;
                const int row = row_of(e), col = e - row * cols;
                if (P.src) put(row, col, g[q]);
                else { float vt = v[q]; put(row, col, momentum(g[q], vt)); P.vel[e] = vt; }
            }
        }
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
    double* const part = reinterpret_cast<double*>(S);
    if (lane == 0) part[wave] = sum;
    __syncthreads();
    sum = 0.0;
#pragma unroll
    for (int w = 0; w < 8; ++w) sum += part[w];
    const double norm = sqrt(sum);
    const float inv = (float)((double)kScaleX / (norm < 1e-7 ? 1e-7 : norm));
    // 256 bytes of a row by half a wave: 64 values read, their parts written in their place
    {
        const int h = lane & 31, k = (2 * h) & 31;
        for (int row = wave * 2 + (lane >> 5); row < R; row += 16)
#pragma unroll 4
            for (int q0 = 0; q0 < c64 / 4; q0 += 16) {
                const float2 u = *reinterpret_cast<const float2*>(X + chunk_at(row, pitch, q0 + (h >> 1)) + (h & 1) * 8);
                unsigned hi, lo;
                split_f16x2(u.x * inv, u.y * inv, hi, lo);
                const int q = q0 + (h >> 4) * 8 + (k >> 3);
                *reinterpret_cast<unsigned*>(X + chunk_at(row, pitch, q) + (k & 7) * 2) = hi;
                *reinterpret_cast<unsigned*>(X + chunk_at(row, pitch, q + 4) + (k & 7) * 2) = lo;
            }
    }
    __syncthreads();

    constexpr int NT = NJ * NJ, PARTS = NJ == 2 ? 2 : 4;             // tiles of S, waves that share one
    const int t = wave % NT, ti = t / NJ, tj = t % NJ, kpart = wave / NT;
    f32x16 acc[NI][NJ];
    for (int step = 0; step < steps; ++step) {
        // ---- S = X X^T: a tile a wave, its k-steps in PARTS parts, joined through LDS
        Sums sums;
        clear(sums);
#pragma unroll 2
        for (int ks = kpart; kpart < PARTS && ks < c64 / 16; ks += PARTS) {
            const int q = (ks >> 1) * 8 + (ks & 1) * 2 + kg;
            const u32x4 bh = frag(X, tj * 32 + lr, pitch, q), bl = frag(X, tj * 32 + lr, pitch, q + 4);
            u32x4 ah = bh, al = bl;
            if (ti != tj) { ah = frag(X, ti * 32 + lr, pitch, q); al = frag(X, ti * 32 + lr, pitch, q + 4); }
            three(ah, al, bh, bl, sums);
        }
        f32x16 s = total(sums);
        float* const scratch = reinterpret_cast<float*>(S);
        if (kpart > 0 && kpart < PARTS) {
#pragma unroll
            for (int e = 0; e < 16; ++e) scratch[((t * (PARTS - 1) + kpart - 1) * 16 + e) * 64 + lane] = s[e];
        }
        __syncthreads();
        if (kpart == 0) {
#pragma unroll
            for (int p = 0; p < PARTS - 1; ++p)
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] += scratch[((t * (PARTS - 1) + p) * 16 + e) * 64 + lane];
        }
        __syncthreads();
        if (kpart == 0) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = s[4 * q + e] * (kScaleS / (kScaleX * kScaleX));
                put4(S, tj * 32 + lr, SP, ti * 32 + 8 * q + 4 * kg, v);
            }
        }
        __syncthreads();
        // ---- B = a I + b S + c S S in the place of S
        if (kpart == 0) {
            clear(sums);
#pragma unroll
            for (int ks = 0; ks < 2 * NJ; ++ks) {
                const int q = (ks >> 1) * 8 + (ks & 1) * 2 + kg;
                three(frag(S, ti * 32 + lr, SP, q), frag(S, ti * 32 + lr, SP, q + 4), frag(S, tj * 32 + lr, SP, q), frag(S, tj * 32 + lr, SP, q + 4), sums);
            }
            s = total(sums);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int i = ti * 32 + 8 * q + 4 * kg, j = tj * 32 + lr;
                float v[4];
                get4(S, j, SP, i, v);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[4 * q + e] = fmaf(kB * (kScaleB / kScaleS), v[e], s[4 * q + e] * (kC * kScaleB / (kScaleS * kScaleS)));
                    if (i + e == j) s[4 * q + e] += kA * kScaleB;
                }
            }
        }
        __syncthreads();
        if (kpart == 0) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float v[4] = {s[4 * q], s[4 * q + 1], s[4 * q + 2], s[4 * q + 3]};
                put4(S, tj * 32 + lr, SP, ti * 32 + 8 * q + 4 * kg, v);
            }
        }
        __syncthreads();
        // ---- B X: rows i are columns of X, tiles wave, wave + 8, ...
#pragma unroll
        for (int n = 0; n < NI; ++n)
#pragma unroll
            for (int j = 0; j < NJ; ++j) clear(acc[n][j]);
#pragma unroll
        for (int ks = 0; ks < 2 * NJ; ++ks) {
            u32x4 bh[NJ], bl[NJ];
            const int q = (ks >> 1) * 8 + (ks & 1) * 2 + kg;
#pragma unroll
            for (int j = 0; j < NJ; ++j) { bh[j] = frag(S, j * 32 + lr, SP, q); bl[j] = frag(S, j * 32 + lr, SP, q + 4); }
            const int lq = lane & 15, row = 16 * ks + 8 * kg + (lq >> 2), qt = 2 * ((lane >> 4) & 1) + ((lq & 3) >> 1), sub = 8 * (lq & 1);
#pragma unroll
            for (int n = 0; n < NI; ++n) {
                const int it = wave + 8 * n;
                if (it >= ntile) continue;
                const u32x2 h0 = frag_tr(X, row, pitch, it * 8 + qt, sub), h1 = frag_tr(X, row + 4, pitch, it * 8 + qt, sub);
                const u32x2 l0 = frag_tr(X, row, pitch, it * 8 + qt + 4, sub), l1 = frag_tr(X, row + 4, pitch, it * 8 + qt + 4, sub);
                const u32x4 ah = {h0[0], h0[1], h1[0], h1[1]}, al = {l0[0], l0[1], l1[0], l1[1]};
#pragma unroll
                for (int p = 0; p < 3; ++p)
#pragma unroll
                    for (int j = 0; j < NJ; ++j) Mma<f16_t, 32>::run(p == 0 ? al : ah, p == 1 ? bl[j] : bh[j], acc[n][j]);
            }
        }
        if (step + 1 == steps) break;
        __syncthreads();
#pragma unroll
        for (int n = 0; n < NI; ++n) {
            const int it = wave + 8 * n;
            if (it >= ntile) continue;
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = acc[n][j][4 * q + e] * (1.f / kScaleB);
                    put4(X, j * 32 + lr, pitch, it * 32 + 8 * q + 4 * kg, v);
                }
        }
        __syncthreads();
    }
    // ---- the answer: stored, or taken as the step of the parameters
    const int out_low = P.flags & NS_OUT_LOW;
    constexpr float back = 1.f / (kScaleB * kScaleX);
#pragma unroll
    for (int n = 0; n < NI; ++n) {
        const int it = wave + 8 * n;
        if (it >= ntile) continue;
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            const int jj = j * 32 + lr;
            if (jj >= r) continue;
            if ((P.flags & NS_VEC_OUT) && !tall) {
                f32x4 old[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int i = it * 32 + 8 * q + 4 * kg;
                    const size_t e = (size_t)jj * P.ld_out + i;
                    if (P.src || i >= c) continue;
                    if (P.master) old[q] = *reinterpret_cast<const f32x4*>(P.master + e);
                    else if (out_low) {
                        const u32x2 w = *reinterpret_cast<const u32x2*>(reinterpret_cast<const unsigned short*>(P.out) + e);
                        old[q] = f32x4{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xffff0000u), __uint_as_float(w[1] << 16), __uint_as_float(w[1] & 0xffff0000u)};
                    } else old[q] = *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(P.out) + e);
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int i = it * 32 + 8 * q + 4 * kg;
                    const size_t e = (size_t)jj * P.ld_out + i;
                    if (i >= c) continue;
                    f32x4 o;
#pragma unroll
                    for (int t2 = 0; t2 < 4; ++t2) o[t2] = acc[n][j][4 * q + t2] * back;
                    if (!P.src) {
#pragma unroll
                        for (int t2 = 0; t2 < 4; ++t2) o[t2] = fmaf(-P.lr, o[t2], old[q][t2] * P.shrink);
                        if (P.master) *reinterpret_cast<f32x4*>(P.master + e) = o;
                    }
                    if (out_low) *reinterpret_cast<u32x2*>(reinterpret_cast<unsigned short*>(P.out) + e) = u32x2{pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])};
                    else *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(P.out) + e) = o;
                }
            } else {
#pragma unroll
                for (int e16 = 0; e16 < 16; ++e16) {
                    const int i = it * 32 + acc_row<32>(e16, lane);
                    if (i >= c) continue;
                    const size_t e = tall ? (size_t)i * P.ld_out + jj : (size_t)jj * P.ld_out + i;
                    const float o = acc[n][j][e16] * back;
                    if (P.src) store_low(P.out, out_low, e, o);
                    else {
                        const float was = P.master ? P.master[e] : load_low(P.out, out_low, e);
                        const float w = fmaf(-P.lr, o, was * P.shrink);
                        if (P.master) P.master[e] = w;
                        store_low(P.out, out_low, e, w);
                    }
                }
            }
        }
    }
}

// 4096 elements of a tensor that is updated by its momentum alone
__device__ __forceinline__ void plain_update(const NsArgs& a, const NsProb& P, int block) {
    const size_t numel = (size_t)P.rows * P.cols, base = (size_t)block * kNsElems;
    const int out_low = P.flags & NS_OUT_LOW;
    constexpr int U = kNsElems / kThreads;
    float g[U], v[U], w[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const size_t e = base + (size_t)i * kThreads + threadIdx.x;
        if (e >= numel) continue;
        g[i] = P.grad[e]; v[i] = P.vel[e];
        w[i] = P.master ? P.master[e] : load_low(P.out, out_low, e);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const size_t e = base + (size_t)i * kThreads + threadIdx.x;
        if (e >= numel) continue;
        v[i] = fmaf(a.momentum, v[i], fmaf(a.wd, w[i], g[i]));
        w[i] = fmaf(-a.rest_lr, v[i], w[i]);
        P.vel[e] = v[i];
        if (P.master) P.master[e] = w[i];
        store_low(P.out, out_low, e, w[i]);
    }
}

__global__ __launch_bounds__(kThreads) void ns_small_kernel(const NsArgs a, int steps) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    const int pi = ns_find(a.start, a.n, blockIdx.x);
    const NsProb& P = a.p[pi];
    if (P.flags & NS_PLAIN) plain_update(a, P, blockIdx.x - a.start[pi]);
    else if (min(P.rows, P.cols) > 32) small_matrix<2, 3>(a, P, steps, smem);
    else small_matrix<1, 5>(a, P, steps, smem);
}

// what LDS holds, the waves' registers hold too
static_assert(32 * (5 * 8 * 32 + 64) * 4 + 12288 > kNsSmallLds && 64 * (3 * 8 * 32 + 64) * 4 + 16384 > kNsSmallLds, "columns of a small matrix");

}  // namespace

hipError_t launch_ns_small(const NsArgs& a, int steps, size_t lds, hipStream_t s) {
    if (a.total <= 0) return hipSuccess;
    static OncePerDevice once;
    if (const hipError_t e = raise_lds_limit(once, {(const void*)ns_small_kernel}, (int)kNsSmallLds); e != hipSuccess) return e;
    hipLaunchKernelGGL(ns_small_kernel, dim3(a.total), dim3(kThreads), lds, s, a, steps);
    return hipGetLastError();
}

}  // namespace lp
