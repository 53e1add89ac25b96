// Orthogonalisation of matrices by Newton-Schulz products, and the parameter update that takes it as its direction (gfx950):
//
//   X <- U / |U|;   five times:  S = X X^T,  B = a I + b S + c S S,  X <- B X
//
// drives every singular value of U towards one (the odd polynomial a x + b x^3 + c x^5 of each, with the coefficients below, stays
// within 0.7 .. 1.2 from the fifth step on).  Products with the shorter side r as rows: 2 r^2 (2 c + r) multiplications a step.
//
// Precision.  The small singular values grow by a = 3.4 a step, 480 times in five, and so does every rounding in their
// directions.  In bf16 the result of a random matrix is off by 1 %, of one of low rank by half; with 11 bits (one fp16) by 0.15 %
// and 6 %.  Here every operand is a sum of two fp16 (22 bits; the entries are bounded by 1.21, S by 1.5, B by 3.5, so powers of
// two that keep the second part above the subnormal numbers are fixed), and a product takes three of the four: off by 7e-7 and
// 2e-5 of it, as fp32 arithmetic is (1.5e-6, 3e-5).
//
// All tensors of an update go through the same launches: one over the elements (momentum, sums of squares, and the whole update
// of the tensors that are not matrices), one that scales, splits and turns tall matrices, and three products a step.
#include "lp_ortho.h"

#include <algorithm>

#include "lp_gemm.h"
#include "lp_kernels.h"
#include "lp_ortho_dev.h"

namespace lp {
namespace {

// (the arguments lie in host memory: one round trip for all of them)
__global__ __launch_bounds__(1024) void ns_put_kernel(const NsChunk c) {
    static_assert(sizeof(c.w) / 4 <= 1024, "a word a thread");
    if ((int)threadIdx.x < c.words) c.dst[threadIdx.x] = c.w[threadIdx.x];
}

// (3.8 KB of arguments: 4.6 us; a network of 55 filters and 110 vectors of batch norms: 18 KB as they are, 5 as records)
__global__ __launch_bounds__(1024) void ns_pack_kernel(const NsPack c) {
    static_assert(sizeof(c.w) / 4 <= 1024, "a word a thread");
    __shared__ unsigned w[1024];
    const int rec = c.full ? kNsRecordFull : kNsRecord, words = c.sets * kNsSetWords + c.count * rec, i = threadIdx.x;
    if (i < words) w[i] = c.w[i];
    __syncthreads();
    if (c.first == 0 && i < kNsLaunches) c.table[i * (c.n + 1) + c.n] = c.total[i];
    if (i >= c.count) return;
    const unsigned* const r = w + c.sets * kNsSetWords + i * rec;
    const unsigned* const b = w + (r[2] >> 8) * kNsSetWords;
    auto wide = [](const unsigned* p) __attribute__((always_inline)) { return (unsigned long long)p[0] | (unsigned long long)p[1] << 32; };
    const unsigned long long po = wide(r + 3), go = wide(r + 5);
    NsProb p;
    p.src = nullptr;
    p.out = reinterpret_cast<void*>(wide(b) + po);
    p.grad = reinterpret_cast<const float*>(wide(b + 2) + go);
    p.vel = reinterpret_cast<float*>(wide(b + 4) + go);
    p.master = wide(b + 6) ? reinterpret_cast<float*>(wide(b + 6) + go) : nullptr;
    p.work = c.full ? c.work + wide(r + 8) : nullptr;
    p.rows = (int)r[0]; p.cols = (int)r[1];
    p.ld_src = 0; p.ld_out = p.cols;
    p.lr = (float)((double)c.lr * sqrt(fmax(1.0, (double)p.rows / p.cols)));
    p.shrink = c.shrink;
    p.flags = (int)(r[2] & 255u); p.pad_ = 0;
    const int t = c.first + i;
    c.probs[t] = p;
    c.table[t] = (int)r[7];
    if (c.full)
        for (int k = 1; k < kNsLaunches; ++k) c.table[k * (c.n + 1) + t] = (int)r[9 + k];
}

// Elements: momentum of the matrices and their sums of squares
__global__ __launch_bounds__(256) void ns_norm_kernel(const NsArgs a) {
    const int pi = ns_find(a.start, a.n, blockIdx.x);
    const NsProb& P = a.p[pi];
    const size_t numel = (size_t)P.rows * P.cols, base = (size_t)(blockIdx.x - a.start[pi]) * kNsElems;
    const int tid = threadIdx.x;
    double sum = 0.0;
    auto element = [&](size_t e, float g, float v) __attribute__((always_inline)) {
        v = fmaf(a.momentum, v, g);
        P.vel[e] = v;
        const float u = a.nesterov ? fmaf(a.momentum, v, g) : v;
        sum += (double)u * u;
    };
    constexpr int U = kNsElems / 1024;
    const int src_low = P.flags & NS_SRC_LOW;
    if (P.flags & NS_VEC) {
        // four elements a thread and trip, all loads first
        f32x4 g[U], v[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const size_t e = base + (size_t)(i * 256 + tid) * 4;
            g[i] = f32x4{0.f, 0.f, 0.f, 0.f}; v[i] = g[i];
            if (e + 4 > numel) continue;
            if (P.src) {
                if (src_low) {
                    const u32x2 w = *reinterpret_cast<const u32x2*>(reinterpret_cast<const unsigned short*>(P.src) + e);
                    g[i] = f32x4{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xffff0000u), __uint_as_float(w[1] << 16), __uint_as_float(w[1] & 0xffff0000u)};
                } else g[i] = *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(P.src) + e);
            } else {
                g[i] = *reinterpret_cast<const f32x4*>(P.grad + e);
                v[i] = *reinterpret_cast<const f32x4*>(P.vel + e);
            }
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const size_t e = base + (size_t)(i * 256 + tid) * 4;
            if (e + 4 <= numel) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float u = g[i][q];
                    if (!P.src) {
                        v[i][q] = fmaf(a.momentum, v[i][q], g[i][q]);
                        u = a.nesterov ? fmaf(a.momentum, v[i][q], g[i][q]) : v[i][q];
                    }
                    sum += (double)u * u;
                }
                if (!P.src) *reinterpret_cast<f32x4*>(P.vel + e) = v[i];
            } else {
                for (size_t t = e; t < numel; ++t) {
                    if (P.src) { const float u = load_low(P.src, src_low, t); sum += (double)u * u; }
                    else element(t, P.grad[t], P.vel[t]);
                }
            }
        }
    } else if (P.src) {
        for (int i = tid; i < kNsElems; i += 256) {
            const size_t e = base + i;
            if (e >= numel) break;
            const size_t row = e / P.cols;
            const float u = load_low(P.src, src_low, row * P.ld_src + (e - row * P.cols));
            sum += (double)u * u;
        }
    } else {
        for (int i = tid; i < kNsElems; i += 256) {
            const size_t e = base + i;
            if (e >= numel) break;
            element(e, P.grad[e], P.vel[e]);
        }
    }
    __shared__ double s[4];
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
    if ((tid & 63) == 0) s[tid >> 6] = sum;
    __syncthreads();
    if (tid == 0) a.norm[blockIdx.x] = (s[0] + s[1]) + (s[2] + s[3]);
}

// 64 x 64 pieces of U / |U| into the planes of X, turned where the matrix is tall
__global__ __launch_bounds__(256) void ns_split_kernel(const NsArgs a) {
    __shared__ float t[64][65];
    __shared__ double s[4];
    const int pi = ns_find(a.start, a.n, blockIdx.x);
    const NsProb& P = a.p[pi];
    const int tid = threadIdx.x;
    const int local = blockIdx.x - a.start[pi], pc = (P.cols + 63) >> 6;
    const int r0 = local / pc * 64, c0 = (local - local / pc * pc) * 64;
    const int col = tid & 63, c = c0 + col;
    // the elements and the sums of squares under way together
    float u[16], g[16];
    auto place = [&](int k, long ld) __attribute__((always_inline)) { return (size_t)min(r0 + (tid >> 6) + 4 * k, P.rows - 1) * ld + min(c, P.cols - 1); };
    if (P.src && (P.flags & NS_SRC_LOW)) {
#pragma unroll
        for (int k = 0; k < 16; ++k) u[k] = bf16_bits_to_float(reinterpret_cast<const unsigned short*>(P.src)[place(k, P.ld_src)]);
    } else if (P.src) {
#pragma unroll
        for (int k = 0; k < 16; ++k) u[k] = reinterpret_cast<const float*>(P.src)[place(k, P.ld_src)];
    } else {
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            u[k] = P.vel[place(k, P.cols)];
            g[k] = a.nesterov ? P.grad[place(k, P.cols)] : 0.f;
        }
    }
    const int b0 = a.start_norm[pi], b1 = a.start_norm[pi + 1];
    double sum = 0.0;
#pragma unroll 4
    for (int b = b0 + tid; b < b1; b += 256) sum += a.norm[b];
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
    if ((tid & 63) == 0) s[tid >> 6] = sum;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        const int row = (tid >> 6) + 4 * k;
        const float w = P.src || !a.nesterov ? u[k] : fmaf(a.momentum, u[k], g[k]);
        t[row][col] = r0 + row < P.rows && c < P.cols ? w : 0.f;
    }
    __syncthreads();
    const double norm = sqrt((s[0] + s[1]) + (s[2] + s[3]));
    const float inv = (float)((double)kScaleX / (norm < 1e-7 ? 1e-7 : norm));
    const bool tall = P.rows > P.cols;
    // the piece as rows of X: row x0 + i, columns y0 + 2 j, y0 + 2 j + 1
    const int x0 = tall ? c0 : r0, y0 = tall ? r0 : c0;
    const NsWork W(P.rows, P.cols);
    unsigned* const out = reinterpret_cast<unsigned*>(P.work);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int i = (tid >> 5) + 8 * k, j = 2 * (tid & 31);
        if (x0 + i < W.r && 2 * (y0 + j) < W.ldc) {
            const float u0 = (tall ? t[j][i] : t[i][j]) * inv, u1 = (tall ? t[j + 1][i] : t[i][j + 1]) * inv;
            const size_t at = ((size_t)(x0 + i) * W.ldc + (y0 + j) / 32 * 64 + (j & 31)) >> 1;
            split_f16x2(u0, u1, out[at], out[at + 16]);
        }
    }
}

enum NsMode { NS_GRAM, NS_POLY, NS_STEP, NS_LAST };

// A piece of O, 32 rows of 32 W columns as they are stored: what it is the step of is requested before its values lie in LDS.
template <int W> struct NsOld { f32x4 w[4 * W]; };         // (bf16: two words of each)
template <int W> __device__ __forceinline__ void ns_request(const NsProb& P, NsOld<W>& old, int row0, int col0, int lane) {
    if (P.src || !(P.flags & NS_VEC_OUT)) return;
    const int col = min(col0 + 4 * (lane & (8 * W - 1)), P.cols - 4);       // (rows and columns beyond the last: read, not used)
#pragma unroll
    for (int k = 0; k < 4 * W; ++k) {
        const size_t e = (size_t)min(row0 + lane / (8 * W) + 8 / W * k, P.rows - 1) * P.ld_out + col;
        if (P.master) old.w[k] = *reinterpret_cast<const f32x4*>(P.master + e);
        else if (P.flags & NS_OUT_LOW) {
            const u32x2 b = *reinterpret_cast<const u32x2*>(reinterpret_cast<const unsigned short*>(P.out) + e);
            old.w[k][0] = __uint_as_float(b[0]); old.w[k][1] = __uint_as_float(b[1]);
        }
        else old.w[k] = *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(P.out) + e);
    }
}
// ... in LDS, element (m, l) at E[m * step + l * next]: stored, or taken as the step of the parameters
template <int W> __device__ __forceinline__ void ns_answer(const NsProb& P, const NsOld<W>& old, const float* E, int step, int next, int row0, int col0, int lane) {
    const int out_low = P.flags & NS_OUT_LOW;
    if (P.flags & NS_VEC_OUT) {
        const int l0 = 4 * (lane & (8 * W - 1)), col = col0 + l0;
        if (col >= P.cols) return;
#pragma unroll
        for (int k = 0; k < 4 * W; ++k) {
            const int m = lane / (8 * W) + 8 / W * k;
            f32x4 o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = E[m * step + (l0 + e) * next];
            if (!P.src) {
                f32x4 w = old.w[k];
                if (!P.master && out_low) {
                    const unsigned b0 = __float_as_uint(w[0]), b1 = __float_as_uint(w[1]);
                    w = f32x4{__uint_as_float(b0 << 16), __uint_as_float(b0 & 0xffff0000u), __uint_as_float(b1 << 16), __uint_as_float(b1 & 0xffff0000u)};
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = fmaf(-P.lr, o[e], w[e] * P.shrink);
            }
            if (row0 + m >= P.rows) continue;
            const size_t e = (size_t)(row0 + m) * P.ld_out + col;
            if (P.master) *reinterpret_cast<f32x4*>(P.master + e) = o;
            if (out_low) *reinterpret_cast<u32x2*>(reinterpret_cast<unsigned short*>(P.out) + e) = u32x2{pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])};
            else *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(P.out) + e) = o;
        }
        return;
    }
    const int l = lane & (32 * W - 1), col = col0 + l;
    if (col >= P.cols) return;
#pragma unroll 4
    for (int m = lane / (32 * W); m < 32; m += 2 / W) {
        if (row0 + m >= P.rows) break;
        const float o = E[m * step + l * next];
        const size_t e = (size_t)(row0 + m) * P.ld_out + col;
        if (P.src) store_low(P.out, out_low, e, o);
        else {
            const float was = P.master ? P.master[e] : load_low(P.out, out_low, e);
            const float w = fmaf(-P.lr, o, was * P.shrink);
            if (P.master) P.master[e] = w;
            store_low(P.out, out_low, e, w);
        }
    }
}

// a 32 x 32 piece in LDS, rows of 32 first and 32 second parts (128 bytes, a pitch of 144), to rows row0.. of `out`
constexpr int kPiecePitch = 144, kPiece = 32 * kPiecePitch;
__device__ __forceinline__ void ns_piece_out(const unsigned char* E, char* out, int ld, int row0, int rows, int col0, int lane) {
    if (2 * col0 >= ld) return;
    const int m0 = lane >> 3, c = lane & 7;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int m = m0 + 8 * k;
        const u32x4 v = *reinterpret_cast<const u32x4*>(E + m * kPiecePitch + c * 16);
        if (row0 + m < rows) *reinterpret_cast<u32x4*>(out + ((size_t)(row0 + m) * ld + 2 * col0) * 2 + c * 16) = v;
    }
}

template <class T, int MODE> __global__ __launch_bounds__(T::NT, 2) void ns_gemm_kernel(const NsArgs a) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    const int x = blockIdx.x & 7, per = a.total >> 3, rem = a.total & 7;
    const int t = x * per + (x < rem ? x : rem) + (blockIdx.x >> 3);       // consecutive tiles to one XCD
    const int pi = ns_find(a.start, a.n, t);
    const NsProb& P = a.p[pi];
    const NsWork W(P.rows, P.cols);
    const int local = t - a.start[pi], r = W.r, ldr = W.ldr, ldc = W.ldc;
    char* const Xs[2] = {P.work, P.work + W.x};
    char *const S = P.work + 2 * W.x, *const B = S + W.s;
    constexpr bool STEP = MODE == NS_STEP || MODE == NS_LAST;
    int ti, tj;
    if constexpr (STEP) {
        const int ti_n = (W.c + T::BI - 1) / T::BI, tj_n = (r + T::BJ - 1) / T::BJ;
        const int band = min(8, tj_n), full = band * ti_n, bd = local / full, w = min(band, tj_n - bd * band), in = local - bd * full;
        ti = in / w; tj = bd * band + in - ti * w;
    } else {                                                      // symmetric: the tiles with ti <= tj, and what they mirror
        tj = (int)((sqrtf(8.f * (float)local + 1.f) - 1.f) * 0.5f);
        while (tj * (tj + 1) / 2 > local) --tj;
        while ((tj + 1) * (tj + 2) / 2 <= local) ++tj;
        ti = local - tj * (tj + 1) / 2;
    }
    const int i0 = ti * T::BI, j0 = tj * T::BJ;
    char* const X = Xs[a.odd];
    const GemmOperand ox = {X, 0, ldc, STEP ? ldc : r}, os = {S, 0, ldr, r}, ob = {B, 0, ldr, r};
    const GemmPairs one = {1, 0, 0};
    typename T::Acc acc;
#pragma unroll
    for (int i = 0; i < T::TI / 32; ++i)
#pragma unroll
        for (int j = 0; j < T::TJ / 32; ++j)
#pragma unroll
            for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.f;
    if constexpr (MODE == NS_GRAM) T::run(ox, ox, one, i0, j0, 0, W.c, (GemmMask)nullptr, smem, acc, W.thin() ? kNsPart : 0);
    else if constexpr (MODE == NS_POLY) T::run(os, os, one, i0, j0, 0, r, (GemmMask)nullptr, smem, acc);
    else T::run(ox, ob, one, i0, j0, 0, r, (GemmMask)nullptr, smem, acc);

    if (T::idle()) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wi = wave / (T::BJ / T::TJ), wj = wave % (T::BJ / T::TJ);
    const int lr = lane & 31, h = lane >> 5;
    const int ib = i0 + wi * T::TI, jb = j0 + wj * T::TJ;
    constexpr int FI = T::TI / 32, FJ = T::TJ / 32;

    if constexpr (MODE == NS_LAST) {
        // the answer through LDS, so that both orientations go out along rows: two micro-tiles side by side at a time (256 bytes of a row)
        // where there are two, and what later ones are the step of under way as far as the registers go.  (Last step of the wide network's
        // update 260 us, of the ImageNet-sized one's 186; 128 bytes of a row and one piece ahead: 296 and 223.  The step alone: 135 and 106.)
        constexpr float back = 1.f / (kScaleB * kScaleX);
        auto all = [&](auto tall_c, auto w_c) __attribute__((always_inline)) {
            constexpr bool TALL = decltype(tall_c)::value;
            constexpr int W = decltype(w_c)::value, N = FI * FJ / W, DEEP = FI * FJ > 8 ? (W > 1 ? 1 : 3) : W > 1 ? 2 : 4;
            constexpr int PITCH = TALL ? 33 : 32 * W + 1;
            float* const E = reinterpret_cast<float*>(smem) + wave * (32 * 33 * W);
            // piece n: micro-tiles (i, j) and the next along the rows of what is stored
            auto at_i = [](int n) { return TALL ? n % FI : n % (FI / W) * W; };
            auto at_j = [](int n) { return TALL ? n / FI * W : n / (FI / W); };
            NsOld<W> old[DEEP];
            auto request = [&](int n) __attribute__((always_inline)) {
                const int ip = ib + at_i(n) * 32, jp = jb + at_j(n) * 32;
                ns_request<W>(P, old[n % DEEP], TALL ? ip : jp, TALL ? jp : ip, lane);
            };
#pragma unroll
            for (int n = 0; n < DEEP - 1 && n < N; ++n) request(n);
#pragma unroll
            for (int n = 0; n < N; ++n) {
                if (n + DEEP - 1 < N) request(n + DEEP - 1);
#pragma unroll
                for (int w = 0; w < W; ++w)
#pragma unroll
                    for (int q = 0; q < 16; ++q)
                        E[((TALL ? w * 32 : 0) + lr) * PITCH + (TALL ? 0 : w * 32) + T::row(q, lane)] = acc[at_i(n) + (TALL ? 0 : w)][at_j(n) + (TALL ? w : 0)][q] * back;
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                __builtin_amdgcn_s_waitcnt(0xc07f);
                const int ip = ib + at_i(n) * 32, jp = jb + at_j(n) * 32;
                ns_answer<W>(P, old[n % DEEP], E, TALL ? 1 : PITCH, TALL ? PITCH : 1, TALL ? ip : jp, TALL ? jp : ip, lane);
                __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
                __builtin_amdgcn_s_waitcnt(0xc07f);
            }
        };
        static_assert(T::NW * 2 * 32 * 33 * 4 <= T::LDS, "two micro-tiles of every wave");
        if (P.rows > P.cols) all(std::true_type(), std::integral_constant<int, FJ % 2 == 0 ? 2 : 1>());
        else all(std::false_type(), std::integral_constant<int, FI % 2 == 0 ? 2 : 1>());
        return;
    }
    // the two parts of the result, 32 x 32 at a time through LDS, from where they go out as whole cache lines
    constexpr float scale = MODE == NS_GRAM ? kScaleS / (kScaleX * kScaleX) : MODE == NS_POLY ? kC * kScaleB / (kScaleS * kScaleS) : 1.f / kScaleB;
    char* const out = MODE == NS_GRAM ? S : MODE == NS_POLY ? B : Xs[a.odd ^ 1];
    const int ldo = STEP ? ldc : ldr;
    unsigned char* const E = smem + wave * kPiece;
#pragma unroll
    for (int j = 0; j < FJ; ++j)
#pragma unroll
        for (int i = 0; i < FI; ++i) {
            const int jj = jb + j * 32 + lr, jp = jb + j * 32, ip = ib + i * 32;
            unsigned hb[8], lb[8];                              // pairs along i
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int ii = ip + 8 * q + 4 * h;
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = acc[i][j][4 * q + e] * scale;
                if constexpr (MODE == NS_POLY) {
                    if (jj < r && 2 * ip < ldr) {
                        const char* const sp = S + ((size_t)jj * ldr + 2 * ip + (ii - ip)) * 2;
                        const u32x2 s0 = *reinterpret_cast<const u32x2*>(sp), s1 = *reinterpret_cast<const u32x2*>(sp + 64);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float sv = f16_up((s0[e >> 1] >> (16 * (e & 1))) & 0xffffu) + f16_up((s1[e >> 1] >> (16 * (e & 1))) & 0xffffu);
                            v[e] = fmaf(kB * (kScaleB / kScaleS), sv, v[e]);
                            if (ii + e == jj) v[e] += kA * kScaleB;
                        }
                    }
                }
                split_f16x2(v[0], v[1], hb[2 * q], lb[2 * q]);
                split_f16x2(v[2], v[3], hb[2 * q + 1], lb[2 * q + 1]);
                unsigned char* const d = E + lr * kPiecePitch + (8 * q + 4 * h) * 2;
                *reinterpret_cast<u32x2*>(d) = u32x2{hb[2 * q], hb[2 * q + 1]};
                *reinterpret_cast<u32x2*>(d + 64) = u32x2{lb[2 * q], lb[2 * q + 1]};
            }
            auto visible = [] { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); __builtin_amdgcn_s_waitcnt(0xc07f); };
            visible();
            ns_piece_out(E, out, ldo, jp, r, ip, lane);
            visible();
            if (!STEP && ti != tj) {
#pragma unroll
                for (int q = 0; q < 16; ++q) {
                    unsigned short* const d = reinterpret_cast<unsigned short*>(E + T::row(q, lane) * kPiecePitch + lr * 2);
                    d[0] = (unsigned short)(hb[q >> 1] >> (16 * (q & 1)));
                    d[32] = (unsigned short)(lb[q >> 1] >> (16 * (q & 1)));
                }
                visible();
                ns_piece_out(E, out, ldo, ip, r, jp, lane);
                visible();
            }
        }
}

template <bool AKR> using NBig = GemmTile<f16_t, AKR, false, 2, 4, 4, 2, 2, false, 2>;
template <bool AKR> using NWide = GemmTile<f16_t, AKR, false, 4, 2, 2, 5, 2, false, 2>;
template <bool AKR, int MODE> using NMid = GemmTile<f16_t, AKR, false, 2, 2, 2, 2, 4, false, 2, MODE == NS_GRAM>;
template <bool AKR, int MODE> using NSmall = GemmTile<f16_t, AKR, false, 2, 2, 1, 1, 4, false, 2, MODE == NS_GRAM>;

template <class T, int MODE> hipError_t launch_gemm(const NsArgs& a, hipStream_t s) {
    static OncePerDevice once;
    constexpr int lds = T::LDS;
    static_assert(T::NW * kPiece <= lds, "the way out fits into the stages");
    auto k = ns_gemm_kernel<T, MODE>;
    if (const hipError_t e = raise_lds_limit(once, {(const void*)k}, lds); e != hipSuccess) return e;
    hipLaunchKernelGGL(k, dim3(a.total), dim3(T::NT), lds, s, a);
    return hipGetLastError();
}
template <bool AKR, int MODE> hipError_t launch_mode(const NsArgs& a, int cfg, hipStream_t s) {
    if (a.total <= 0) return hipSuccess;
    if constexpr (AKR)
        if (cfg == NT_256x320) return launch_gemm<NWide<AKR>, MODE>(a, s);
    switch (cfg) {
        case NT_256: return launch_gemm<NBig<AKR>, MODE>(a, s);
        case NT_128: return launch_gemm<NMid<AKR, MODE>, MODE>(a, s);
        default: return launch_gemm<NSmall<AKR, MODE>, MODE>(a, s);
    }
}

}  // namespace

void ns_tile_size(int cfg, int* bi, int* bj) {
    static const int d[NT_COUNT][2] = {{256, 256}, {256, 320}, {128, 128}, {64, 64}};
    *bi = d[cfg][0]; *bj = d[cfg][1];
}

// Time of `tiles` tiles, in microseconds at 8192 k: the rounds that fill the chip (`slots` workgroups at once), and the last one by how
// full it is.  Measured: 256 x 256 430 a round, 256 x 320 530, 128 x 128 118 (64 tiles) to 173, 64 x 64 67 (256 tiles) to 227 (1024).
double ns_tile_time(int cfg, long tiles) {
    static const struct { int slots; double some, full; } t[NT_COUNT] = {{256, 330, 430}, {256, 410, 530}, {256, 100, 173}, {512, 30, 115}};
    const long rounds = tiles / t[cfg].slots, rest = tiles - rounds * t[cfg].slots;
    return (double)rounds * t[cfg].full + (rest ? t[cfg].some + (t[cfg].full - t[cfg].some) * (double)rest / t[cfg].slots : 0.0);
}

hipError_t launch_ns_put(const NsChunk& c, hipStream_t s) {
    hipLaunchKernelGGL(ns_put_kernel, dim3(1), dim3(1024), 0, s, c);
    return hipGetLastError();
}
hipError_t launch_ns_pack(const NsPack& c, hipStream_t s) {
    hipLaunchKernelGGL(ns_pack_kernel, dim3(1), dim3(1024), 0, s, c);
    return hipGetLastError();
}
hipError_t launch_ns_norm(const NsArgs& a, hipStream_t s) {
    if (a.total <= 0) return hipSuccess;
    hipLaunchKernelGGL(ns_norm_kernel, dim3(a.total), dim3(256), 0, s, a);
    return hipGetLastError();
}
hipError_t launch_ns_split(const NsArgs& a, hipStream_t s) {
    if (a.total <= 0) return hipSuccess;
    hipLaunchKernelGGL(ns_split_kernel, dim3(a.total), dim3(256), 0, s, a);
    return hipGetLastError();
}
hipError_t launch_ns_gram(const NsArgs& a, int cfg, hipStream_t s) { return launch_mode<false, NS_GRAM>(a, cfg, s); }
hipError_t launch_ns_poly(const NsArgs& a, int cfg, hipStream_t s) { return launch_mode<false, NS_POLY>(a, cfg, s); }
hipError_t launch_ns_step(const NsArgs& a, int cfg, hipStream_t s) { return a.last ? launch_mode<true, NS_LAST>(a, cfg, s) : launch_mode<true, NS_STEP>(a, cfg, s); }

}  // namespace lp
