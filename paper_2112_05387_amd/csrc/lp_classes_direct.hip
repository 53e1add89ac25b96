// Cross-entropy of a linear classifier, small problems (gfx950): sums in fp32 without the matrix cores.
//
// A few hundred rows against a few hundred classes are less work than the launches of the tiled products are apart: laying out the
// operands, products, softmax and sums were eleven kernels of 3 to 8 us each, behind which the host stood for 70 us.  Here two kernels make
// the forward pass (a workgroup a row; the sum of the losses) and two the backward pass (a workgroup a row: the probabilities again
// and dX; a workgroup four classes: dW and the bias), straight from the operands, whatever their strides.
// Every row reads all of the weights from L2, so what bounds these kernels is how long a chain of such reads is: a lane has a class,
// the waves of a row have a part of the channels each; for the gradients a group of threads has the channels and a part of
// the classes or rows.  The rule that sends a problem here (ce_direct_waves) bounds the chains.  Loss and
// gradients in fp32, host and all, tiled and here: 256 x 16 -> 10 67 and 38 us, 212 x 277 -> 112 70 and 42, 2 x 19 -> 2485 73 and 50; bf16
// 911 x 28 -> 541 71 and 41.
#include <algorithm>

#include "lp_classes.h"
#include "lp_kernels.h"

namespace lp {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f, kInf = __builtin_inff();

__device__ __forceinline__ bool is_class(int y, int V) { return (unsigned)y < (unsigned)V; }
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o);
    return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) v = fmaxf(v, __shfl_xor(v, o));
    return v;
}
// eight channels from p on
template <class T> __device__ __forceinline__ void eight(const T* p, bool vec, float (&f)[8]) {
    if (vec) {
        if constexpr (sizeof(T) == 2) {
            const u32x4 v = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
            for (int e = 0; e < 4; ++e) { f[2 * e] = __uint_as_float(v[e] << 16); f[2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u); }
        } else {
            const f32x4 v = *reinterpret_cast<const f32x4*>(p), w = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) { f[e] = v[e]; f[4 + e] = w[e]; }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = to_float(p[e]);
    }
}

// All logits of row n to s_l[V], by NW waves: their channels in parts, a class a lane.  s_x: C floats, s_p: NW * V
template <class T, int NW> __device__ __forceinline__ void row_logits(const CeDirect& a, int n, float* s_x, float* s_p, float* s_l) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const T* const x = reinterpret_cast<const T*>(a.x) + (size_t)n * a.ldx;
    for (int c = tid; c < a.C; c += NW * 64) s_x[c] = to_float(x[c]);
    __syncthreads();
    const int part = ((a.C + NW - 1) / NW + 7) & ~7, c0 = min(wave * part, a.C), c1 = min(c0 + part, a.C);
    for (int v = lane; v < a.V; v += 64) {
        const T* const w = reinterpret_cast<const T*>(a.w) + (size_t)v * a.ldw;
        float l[2] = {0.f, 0.f};
        int c = c0;
#pragma unroll 4
        for (; c + 8 <= c1; c += 8) {
            float f[8];
            eight(w + c, a.vec, f);
#pragma unroll
            for (int e = 0; e < 8; ++e) l[e & 1] = fmaf(s_x[c + e], f[e], l[e & 1]);
        }
        for (; c < c1; ++c) l[0] = fmaf(s_x[c], to_float(w[c]), l[0]);
        s_p[wave * a.V + v] = l[0] + l[1];
    }
    __syncthreads();
    for (int v = tid; v < a.V; v += NW * 64) {
        float l = s_p[v];
        for (int w = 1; w < NW; ++w) l += s_p[w * a.V + v];
        s_l[v] = l + (a.bias ? a.bias[v] : 0.f);
    }
    __syncthreads();
}

// NW waves a row
template <class T, int NW> __global__ __launch_bounds__(NW * 64) void ce_direct_forward_kernel(const CeDirect a) {
    extern __shared__ float smem[];
    __shared__ float s_r[NW];
    float *const s_x = smem, *const s_l = s_x + a.C, *const s_p = s_l + a.V;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = blockIdx.x, y = a.labels[n];
    row_logits<T, NW>(a, n, s_x, s_p, s_l);
    float m = -kInf;
    for (int v = tid; v < a.V; v += NW * 64) m = fmaxf(m, s_l[v]);
    m = wave_max(m);
    if (lane == 0) s_r[wave] = m;
    __syncthreads();
    for (int w = 0; w < NW; ++w) m = fmaxf(m, s_r[w]);
    __syncthreads();
    const float m0 = m == -kInf ? 0.f : m;
    float s = 0.f;                                               // of the classes but the label's
    for (int v = tid; v < a.V; v += NW * 64) s += v == y ? 0.f : __builtin_amdgcn_exp2f((s_l[v] - m0) * kLog2e);
    s = wave_sum(s);
    if (lane == 0) s_r[wave] = s;
    __syncthreads();
    if (tid != 0) return;
    s = 0.f;
    for (int w = 0; w < NW; ++w) s += s_r[w];
    const bool valid = is_class(y, a.V);
    const float own = valid ? s_l[y] : -kInf, all = s + __builtin_amdgcn_exp2f((own - m0) * kLog2e);
    const float ls = __builtin_amdgcn_logf(all) * kLn2, lse = m + ls;
    // of a row that is all but certain the logits cancel first, and what the other classes have is not added to one
    const float loss = !valid ? 0.f : m - own < 5.f ? log1pf(s * __builtin_amdgcn_exp2f((m - own) * kLog2e)) : (m - own) + ls;
    a.lse_out[n] = lse;
    if (a.row_loss) a.row_loss[n] = loss;
    a.bsum[n] = loss;
    a.bcnt[n] = valid ? 1 : 0;
    if (gridDim.x == 1) *a.loss = loss;
}

// number of rows that count, by a whole workgroup
__device__ __forceinline__ int count_rows(const CeDirect& a, int* s) {
    int c = 0;
    for (int n = threadIdx.x; n < a.N; n += blockDim.x) c += is_class(a.labels[n], a.V) ? 1 : 0;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) c += __shfl_xor(c, o);
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = c;
    __syncthreads();
    c = 0;
    for (int w = 0; w < (int)(blockDim.x >> 6); ++w) c += s[w];
    return max(c, 1);
}

// a row: d = (p - [label]) scale / count to memory and to LDS, dX = d W
template <class T, int NW> __global__ __launch_bounds__(NW * 64) void ce_direct_rows_kernel(const CeDirect a, int cw_log) {
    extern __shared__ float smem[];
    __shared__ int s_c[NW];
    __shared__ float s_o[NW];
    float *const s_x = smem, *const s_l = s_x + a.C, *const s_p = s_l + a.V;
    const int tid = threadIdx.x, n = blockIdx.x, y = a.labels[n];
    const bool valid = is_class(y, a.V);
    const float g = a.scale / (float)count_rows(a, s_c);
    if (valid) {
        row_logits<T, NW>(a, n, s_x, s_p, s_l);
        // the label's p - 1, where p is near one, as minus the sum of the others: 1 - p would lose what tells them apart
        const float shift = a.lse[n];
        float others = 0.f;
        for (int v = tid; v < a.V; v += NW * 64) {
            const float p = __builtin_amdgcn_exp2f((s_l[v] - shift) * kLog2e);
            if (v != y) { others += p; a.d[(size_t)n * a.V + v] = p * g; }
            s_l[v] = v != y ? p * g : p;
        }
        others = wave_sum(others);
        if ((tid & 63) == 0) s_o[tid >> 6] = others;
        __syncthreads();
        if (tid == 0) {
            others = 0.f;
            for (int w = 0; w < NW; ++w) others += s_o[w];
            const float p = s_l[y], d = (p > 0.5f ? -others : p - 1.f) * g;
            s_l[y] = d;
            a.d[(size_t)n * a.V + y] = d;
        }
    } else {
        for (int v = tid; v < a.V; v += NW * 64) a.d[(size_t)n * a.V + v] = 0.f;
    }
    if (!a.dx) return;
    __syncthreads();
    // channels by 2^cw_log threads at a time, the classes in as many parts as there are such groups
    const int cw = 1 << cw_log, col = tid & (cw - 1), grp = tid >> cw_log, groups = (NW * 64) >> cw_log;
    T* const dx = reinterpret_cast<T*>(a.dx) + (size_t)n * a.lddx;
    for (int c0 = 0; c0 < a.C; c0 += cw) {
        const int c = c0 + col;
        float t = 0.f;
        if (valid) {
            const T* const w = reinterpret_cast<const T*>(a.w) + min(c, a.C - 1);
#pragma unroll 8
            for (int v = grp; v < a.V; v += groups) t = fmaf(s_l[v], to_float(w[(size_t)v * a.ldw]), t);
        }
        s_p[tid] = t;
        __syncthreads();
        if (grp == 0 && c < a.C) {
            for (int k = 1; k < groups; ++k) t += s_p[(k << cw_log) + col];
            dx[c] = from_float<T>(t);
        }
        __syncthreads();
    }
}

// four classes of up to 256 channels: dW = d^T X over the rows that count, in 1024 / CW groups of rows; the first also dbias.  What
// bounds it are round trips to d, which other dies' workgroups have just written: eight rows' loads are under way, none behind a branch
// (212 x 277 -> 112 by 256 threads with four rows under way: 60 us).
template <class T> __global__ __launch_bounds__(1024) void ce_direct_weights_kernel(const CeDirect a, int cw_log) {
    __shared__ float s_t[4][1024];
    constexpr int R = 8;
    const int v0 = blockIdx.x * 4, cw = 1 << cw_log, col = threadIdx.x & (cw - 1), grp = threadIdx.x >> cw_log, groups = 1024 >> cw_log;
    const int c = blockIdx.y * cw + col;
    float t[4] = {0.f, 0.f, 0.f, 0.f}, b[4] = {0.f, 0.f, 0.f, 0.f};
    const T* const x = reinterpret_cast<const T*>(a.x) + min(c, a.C - 1);
    for (int n0 = grp; n0 < a.N; n0 += R * groups) {
        float xv[R], d[R][4];
        int y[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int n = min(n0 + r * groups, a.N - 1);
            y[r] = a.labels[n];
            xv[r] = to_float(x[(size_t)n * a.ldx]);
#pragma unroll
            for (int i = 0; i < 4; ++i) d[r][i] = a.d[(size_t)n * a.V + min(v0 + i, a.V - 1)];
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const bool valid = n0 + r * groups < a.N && is_class(y[r], a.V);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                t[i] = valid ? fmaf(d[r][i], xv[r], t[i]) : t[i];
                b[i] += valid ? d[r][i] : 0.f;
            }
        }
    }
    for (int pass = 0; pass < 2; ++pass) {
        if (pass == 1 && (!a.dbias || blockIdx.y != 0)) return;
        if (pass == 0 && !a.dw) continue;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) s_t[i][threadIdx.x] = pass ? b[i] : t[i];
        __syncthreads();
        for (int half = groups >> 1; half > 0; half >>= 1) {
            if (grp < half)
#pragma unroll
                for (int i = 0; i < 4; ++i) s_t[i][threadIdx.x] += s_t[i][threadIdx.x + (half << cw_log)];
            __syncthreads();
        }
        if (grp == 0) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (v0 + i >= a.V) continue;
                if (pass == 0) { if (c < a.C) a.dw[(size_t)(v0 + i) * a.C + c] = s_t[i][col]; }
                else if (col == 0) a.dbias[v0 + i] = s_t[i][0];
            }
        }
    }
}

// threads that take the channels together: a power of two, from 4 to `most`
int channel_threads_log(int C, int most_log) {
    int lg = 2;
    while ((1 << lg) < C && lg < most_log) ++lg;
    return lg;
}
size_t row_lds(const CeDirect& a, int waves) { return ((size_t)a.C + a.V + std::max(waves * a.V, waves * 64)) * sizeof(float); }

template <class T> hipError_t forward(const CeDirect& a, int waves, hipStream_t s) {
    if (waves == 16) hipLaunchKernelGGL((ce_direct_forward_kernel<T, 16>), dim3(a.N), dim3(1024), row_lds(a, waves), s, a);
    else hipLaunchKernelGGL((ce_direct_forward_kernel<T, 4>), dim3(a.N), dim3(256), row_lds(a, waves), s, a);
    return hipGetLastError();
}
template <class T> hipError_t backward(const CeDirect& a, int waves, hipStream_t s) {
    const int lx = channel_threads_log(a.C, waves == 16 ? 10 : 8), lw = channel_threads_log(a.C, 8);
    if (waves == 16) hipLaunchKernelGGL((ce_direct_rows_kernel<T, 16>), dim3(a.N), dim3(1024), row_lds(a, waves), s, a, lx);
    else hipLaunchKernelGGL((ce_direct_rows_kernel<T, 4>), dim3(a.N), dim3(256), row_lds(a, waves), s, a, lx);
    if (hipError_t e = hipGetLastError(); e != hipSuccess || (!a.dw && !a.dbias)) return e;
    hipLaunchKernelGGL(ce_direct_weights_kernel<T>, dim3((a.V + 3) / 4, (a.C + (1 << lw) - 1) >> lw), dim3(1024), 0, s, a, lw);
    return hipGetLastError();
}

}  // namespace

// Waves a row, 0: not a problem for these kernels.  A read of L2 in a chain is worth some 75 clocks with eight under way, and eight of
// d's some 2400; the chains of a row (its logits, then dX) and of a class (dW) may take 20000 clocks each, all rows together not more
// than 2^24 products, and a row's logits have to fit into the 64 KB of LDS that need no leave.
int ce_direct_waves(int N, int C, int V) {
    if (N < 1 || N > 1024 || (size_t)N * V * C > ((size_t)1 << 24)) return 0;
    const int lw = channel_threads_log(C, 8);
    if ((N + 8 * (1024 >> lw) - 1) / (8 * (1024 >> lw)) * 2400 > 20000) return 0;
    for (const int nw : {4, 16}) {
        const int lx = channel_threads_log(C, nw == 16 ? 10 : 8), groups = (nw * 64) >> lx;
        const long logits = (long)((V + 63) / 64) * (((C + nw - 1) / nw + 7) / 8 * 75 + 300);
        const long dx = (long)((V + groups - 1) / groups) * 75 * ((C + (1 << lx) - 1) >> lx);
        if (((size_t)C + (size_t)V * (nw + 1)) * 4 <= 60000 && logits + dx <= 20000 && (nw == 4 || N <= 256)) return nw;
    }
    return 0;
}
hipError_t launch_ce_direct_forward(const CeDirect& a, int dtype, int waves, hipStream_t s) {
    hipError_t e = dtype == 1 ? forward<bf16_t>(a, waves, s) : forward<float>(a, waves, s);
    if (e == hipSuccess && a.N > 1) e = launch_ce_total(a.bsum, a.bcnt, a.N, a.loss, s);
    return e;
}
hipError_t launch_ce_direct_backward(const CeDirect& a, int dtype, int waves, hipStream_t s) {
    return dtype == 1 ? backward<bf16_t>(a, waves, s) : backward<float>(a, waves, s);
}

}  // namespace lp
