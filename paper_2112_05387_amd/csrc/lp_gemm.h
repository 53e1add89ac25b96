// Matrix product of 16-bit operands, one output tile per workgroup (gfx950):
//
//   D[i][j] = sum over pairs (a, b) of planes, sum over k of A_a[i, k] * B_b[j, k]        (fp32 sums)
//
// Values that need more than the 8 or 11 bits of a 16-bit float are kept as a sum of planes (x = x0 + x1 [+ x2], each the
// rounded rest of the ones before), and a product is the sum over those pairs of planes that matter; the pairs lie one after
// the other along the reduction, so the kernel below is the same for one product and for six.
//
// An operand lies in memory with k contiguous (KR = false: rows i, pitch ld) or with its rows along k (KR = true: rows k, the
// index i contiguous).  Both come into LDS by direct loads of 1 KiB a wave, as they lie, and leave it as fragments of
// v_mfma_f32_32x32x16: the former by 16-byte reads, the latter by transposing reads (ds_read_b64_tr_b16: 16 lanes read four
// k of 16 rows and get four k of one row each).  So no operand is ever laid out anew for the other direction of a product.
//
// DUAL: both operands are sums of two planes that lie beside each other, 32 k of the first and the same 32 of the second in 128
// bytes, and a k-tile of 64 elements is 32 k of either.  From the fragments of two planes come three products (the
// fourth, of the two rests, is below the precision): half as much again for the same loads and LDS reads.
//
// A k-tile is 64 elements long (128-byte rows: whole cache lines) and its loads are spread between the products of the one before
// it.  Four waves (tiles of 128 and less, two workgroups a compute unit): one barrier a k-tile, ahead of the products of its last
// 16 k, both frees its stage and shows the next.  Eight waves (256 x 256, one workgroup): two groups that take turns.
// What bounds it: power.  8192 x 8192 x 4096 in bf16 1105 (k contiguous), 1220 (one operand with rows along k), 1240 TFLOP/s
// (both), DUAL 1440 of its three products, at 1.6 to 1.9 GHz; without the loads 1270 to 1570, the matrix cores busy for 85 % of
// the clocks.  All eight waves in step, as the four are: 1013, 1128, 1203, 1370; a quarter as many waves of 128 x 128 each,
// a third fewer LDS reads: 5 % less than that; fragments two k-steps ahead: the same.
// Rows are unpadded; their 16-byte chunks (KR: 32-byte pairs) trade places so that a read touches every bank once:
//   KR = false  chunk c of row r at c ^ (r >> 1 & 7)
//   KR = true   pair p of row k at p ^ 2 (k & 3) (rows of 256 bytes or more), p ^ 2 (k >> 1 & 1) (128 bytes), p (64 bytes)
// Ragged edges, tails of k and rows that are to count as zero are out-of-range buffer offsets, which read as zeros.
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

#include "lp_mma.h"

namespace lp {

struct GemmOperand {
    const char* base;      // plane 0, element (0, 0); 16-byte aligned
    size_t plane;          // bytes from a plane to the next
    int ld;                // elements from a row to the next, a multiple of 8
    int extent;            // rows i (KR = false), or columns i in a row, a multiple of 8 (KR = true)
};

// pairs of planes, four bits each, first pair lowest: A's plane and B's plane of pair s
struct GemmPairs { int n; unsigned a, b; };

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
struct f16_t { unsigned short v; };   // storage-only half
template <> struct Mma<f16_t, 32> {
    __device__ static __forceinline__ void run(const u32x4& a, const u32x4& b, f32x16& c) {
        c = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
};

typedef __attribute__((address_space(3))) void* gemm_lds_t;
typedef const __attribute__((address_space(4))) unsigned long long* GemmMask;      // read by scalar loads
typedef __attribute__((ext_vector_type(4))) short gemm_s16x4;

template <class E, bool AKR, bool BKR, int WI, int WJ, int FI, int FJ, int STAGES, bool MASKED = false, bool DUAL = false, bool LOADERS = false> struct GemmTile {
    static constexpr int BK = 64, NW = WI * WJ, NT = NW * 64 * (LOADERS ? 2 : 1);
    static constexpr int TI = FI * 32, TJ = FJ * 32, BI = WI * TI, BJ = WJ * TJ;
    static constexpr int A_BYTES = BI * BK * 2, STAGE = (BI + BJ) * BK * 2, LDS = STAGES * STAGE;
    static constexpr int NSA = BI / 8 / NW, NSB = BJ / 8 / NW, NL = NSA + NSB;      // wave-loads of a k-tile
    static constexpr int KS = BK / 16;
    static constexpr int PL = DUAL ? 2 : 1, KT = BK / PL;           // planes beside each other; k of a k-tile
    static constexpr bool TURNS = NW == 8;                          // two waves a SIMD, one of either group (see run)
    static_assert(NW % 2 == 0 && NSA * NW * 8 == BI && NSB * NW * 8 == BJ, "every wave loads the same number of slabs");
    typedef f32x16 Acc[FI][FJ];

    static constexpr unsigned kOOB = 0x80000000u;       // beyond any buffer of 2^31 - 1 bytes
    template <int N> __device__ static __forceinline__ void wait_vmcnt() {
        __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
    }
    __device__ static __forceinline__ __amdgpu_buffer_rsrc_t rsrc(const char* p) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p), 0, 0x7fffffff, 0x00020000);
    }

    // KR: the places of a row's 32-byte pairs
    template <int B> __device__ static __forceinline__ int swap(int k) { return B * PL >= 128 ? (k & 3) << 1 : B * PL == 64 ? ((k >> 1) & 1) << 1 : 0; }

    // One operand's loads: lane's offset in a slab, and what it has to compare with at the edges.
    template <bool KR, int B, int NS> struct Loader {
        static constexpr int RB = B * PL * 2, RPS = KR ? 1024 / RB : 8; // KR: bytes of a row of the stage; rows of a slab
        const char* base; size_t plane; int ldb;        // bytes of a row of the operand
        unsigned voff; int row, chunk, last;            // row: this lane's in slab 0; last: rows that exist from row 0 of the tile on
        int step;                                       // bytes between the slabs of a wave

        __device__ __forceinline__ void init(const GemmOperand& o, int x0, int lane, int wave) {
            ldb = o.ld * 2; plane = o.plane;
            if constexpr (!KR) {
                const int pos = lane & 7;
                chunk = pos ^ (4 * (wave & 1) + (lane >> 4));
                row = wave * 8 + (lane >> 3);
                base = o.base + (size_t)x0 * ldb;
                last = o.extent - x0;
                voff = (unsigned)(row * ldb + chunk * 16);
            } else {
                constexpr int CPR = RB / 16;
                const int sub = lane / CPR, pos = lane % CPR;
                row = wave * RPS + sub;
                const int f = swap<B>(row);
                const int col = x0 * PL + (((pos >> 1) ^ f) << 4) + (pos & 1) * 8;
                base = o.base; chunk = 0; last = 0;
                voff = col < o.extent ? (unsigned)(row * ldb + col * 2) : kOOB;
            }
            step = NW * RPS * ldb;
        }
        // load i of the k-tile that starts at k (krem: k that are left), of the plane at `p`
        __device__ __forceinline__ unsigned offset(int i, int krem, unsigned long long mask) const {
            if constexpr (!KR) return row + i * (NW * RPS) < last && (DUAL ? 0 : chunk * 8) < krem ? voff : kOOB;
            else {
                const int k = row + i * (NW * RPS);
                bool ok = k < krem;
                if constexpr (MASKED) ok = ok && ((mask >> k) & 1ull);
                return ok ? voff : kOOB;
            }
        }
        __device__ __forceinline__ const char* at(int p, int k) const {
            return base + (size_t)p * plane + (KR ? (size_t)k * ldb : (size_t)k * 2 * PL);
        }
    };

    // Fragments are read by inline assembly and waited for explicitly: in front of the built-in of the transposing read the compiler
    // waits for every load to LDS that is under way.  Nothing may touch a fragment between read() and arrived(), which is
    // where its value becomes usable; no fragment is under way where control flow joins.
    template <bool KR, int B, int F> struct Reader {
        static constexpr int RB = B * PL * 2;
        unsigned addr[KR ? F : KS];
        u32x4 whole[2 * PL][KR ? 1 : F];               // DUAL: [k-step][plane]
        u32x2 half[2 * PL][KR ? F : 1][2];

        __device__ __forceinline__ void init(int w, int lane, unsigned lds0) {
            if constexpr (!KR) {
                const int r = lane & 31, sw = (r >> 1) & 7;
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) addr[ks] = lds0 + (w * F * 32 + r) * (BK * 2) + (((2 * ks + (lane >> 5)) ^ sw) << 4);
            } else {
                const int lq = lane & 15, k = 8 * (lane >> 5) + (lq >> 2);
                const int f = swap<B>(k);
#pragma unroll
                for (int m = 0; m < F; ++m) addr[m] = lds0 + k * RB + (((2 * PL * (w * F + m) + ((lane >> 4) & 1)) ^ f) << 5) + 8 * (lq & 3);
            }
        }
        // the fragments of k-step S of the stage that starts at byte `st` (DUAL: S = 2 * plane + k-step of the k-tile's two)
        template <int S, int M = 0> __device__ __forceinline__ void read(unsigned st) {
            constexpr int slot = DUAL ? 2 * (S & 1) + (S >> 1) : S & 1;      // [k-step][plane], or two k-steps
            if constexpr (M < F) {
                if constexpr (!KR) asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(whole[slot][M]) : "v"(addr[S] + st), "i"(M * 32 * BK * 2));
                else {
                    constexpr int off = (DUAL ? S & 1 : S) * 16 * RB;
                    const unsigned a = (DUAL && S >= 2 ? addr[M] ^ 64u : addr[M]) + st;      // the second plane: two pairs on
                    asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(half[slot][M][0]) : "v"(a), "i"(off));
                    asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(half[slot][M][1]) : "v"(a), "i"(off + 4 * RB));
                }
                read<S, M + 1>(st);
            }
        }
        __device__ __forceinline__ void arrived(int slot) {
#pragma unroll
            for (int m = 0; m < F; ++m) {
                if constexpr (!KR) asm volatile("" : "+v"(whole[slot][m]));
                else asm volatile("" : "+v"(half[slot][m][0]), "+v"(half[slot][m][1]));
            }
        }
        __device__ __forceinline__ u32x4 get(int slot, int m) const {
            if constexpr (!KR) return whole[slot][m];
            else return u32x4{half[slot][m][0][0], half[slot][m][0][1], half[slot][m][1][0], half[slot][m][1][1]};
        }
    };

    // waves that have no share of the result
    __device__ static __forceinline__ bool idle() { return LOADERS && (int)threadIdx.x >= NW * 64; }

    // Adds to acc the products of rows i0.. of A and j0.. of B over k in [kb, ke), kb a multiple of 64.  (DUAL: one pair, and operands
    // with k contiguous are zero behind ke up to a multiple of 32.)  mask (MASKED): bit k & 63
    // of word k >> 6 is set where A's row k counts.  Ends with every load landed and all waves past their last LDS read.
    __device__ static __forceinline__ void run(const GemmOperand& A, const GemmOperand& B, const GemmPairs& pairs, int i0, int j0, int kb, int ke,
                                               GemmMask mask, unsigned char* smem, Acc& acc) {
        const int tid = threadIdx.x, lane = tid & 63, number = __builtin_amdgcn_readfirstlane(tid >> 6);
        const bool loader = LOADERS && number >= NW;
        const int wave = loader ? number - NW : number;
        const int nkt = (ke - kb + KT - 1) / KT, total = ke > kb ? nkt * pairs.n : 0;
        if (total <= 0) return;
        Loader<AKR, BI, NSA> la;
        Loader<BKR, BJ, NSB> lb;
        la.init(A, i0, lane, wave);
        lb.init(B, j0, lane, wave);
        const unsigned lds0 = (unsigned)(uintptr_t)(gemm_lds_t)smem;
        Reader<AKR, BI, FI> ra;
        Reader<BKR, BJ, FJ> rb;
        ra.init(wave / WJ, lane, lds0);
        rb.init(wave % WJ, lane, lds0 + A_BYTES);

        int seg = 0, kt = 0, issued = 0, t_krem = 0;
        unsigned long long t_mask = 0, ahead = 0;              // ahead: of the k-tile behind, loaded where nothing waits for it
        const char *pa = nullptr, *pb = nullptr;
        unsigned char* t_dst = smem;
        // the k-tile that is loaded next; past the end nothing is left of k and everything reads as zero
        auto tile_begin = [&](int st) __attribute__((always_inline)) {
            const int k = kb + kt * KT;
            t_krem = issued < total ? ke - k : 0;
            pa = la.at((pairs.a >> (4 * seg)) & 15, k);
            pb = lb.at((pairs.b >> (4 * seg)) & 15, k);
            if constexpr (MASKED) t_mask = TURNS ? ahead : mask[min(k, ke - 1) >> 6];
            t_dst = smem + st * STAGE + wave * 1024;
            ++issued;
            if (++kt == nkt) { kt = 0; if (seg + 1 < pairs.n) ++seg; }
        };
        auto mask_ahead = [&] __attribute__((always_inline)) {
            if constexpr (MASKED && TURNS) ahead = mask[min(kb + kt * KT, ke - 1) >> 6];
        };
        auto issue_one = [&](int i) __attribute__((always_inline)) {
            if (i < NSA)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc(pa), (gemm_lds_t)(t_dst + i * (NW * 1024)), 16, (int)la.offset(i, t_krem, t_mask), i * la.step, 0, 0);
            else if (i < NL)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc(pb), (gemm_lds_t)(t_dst + A_BYTES + (i - NSA) * (NW * 1024)), 16,
                                                         (int)lb.offset(i - NSA, t_krem, ~0ull), (i - NSA) * lb.step, 0, 0);
        };
        auto arrived = [&](int slot) __attribute__((always_inline)) {
            __builtin_amdgcn_s_waitcnt(0xc07f);                // lgkmcnt(0)
#pragma unroll
            for (int p = 0; p < PL; ++p) {
                ra.arrived(PL * slot + p);
                rb.arrived(PL * slot + p);
            }
        };
        constexpr int NM = FI * FJ, NP = DUAL ? 3 * NM : NM;   // products of a phase (a k-step) = places for loads
        // The loads of a k-tile are issued between the products behind the barrier that frees its stage.  Two stages: as early as
        // they go, one or more a place, as they have to land within the k-tile; more stages: evenly over a whole k-tile.
        constexpr int PHASES = DUAL ? 2 : KS, PLACES = STAGES == 2 ? (NL < 2 * NP ? NL : 2 * NP) : PHASES * NP;
        // DUAL: the small terms first
        auto products = [&](int slot, int first, bool issue) __attribute__((always_inline)) {
#pragma unroll
            for (int p = 0; p < NP / NM; ++p)
#pragma unroll
                for (int i = 0; i < FI; ++i)
#pragma unroll
                    for (int j = 0; j < FJ; ++j) {
                        if constexpr (DUAL) Mma<E, 32>::run(ra.get(2 * slot + (p == 0), i), rb.get(2 * slot + (p == 1), j), acc[i][j]);
                        else Mma<E, 32>::run(ra.get(slot, i), rb.get(slot, j), acc[i][j]);
                        if (issue) {
#pragma unroll
                            for (int q = 0; q < NL; ++q)
                                if (q * PLACES / NL == first + p * NM + i * FJ + j) issue_one(q);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
        };
        if (!LOADERS || loader) {
#pragma unroll
            for (int s = 0; s < (TURNS ? 1 : STAGES); ++s) {
                mask_ahead();
                tile_begin(s);
#pragma unroll
                for (int i = 0; i < NL; ++i) issue_one(i);
            }
            if constexpr (TURNS) mask_ahead();
            wait_vmcnt<TURNS ? 0 : (STAGES - 1) * NL>();
        }
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        auto barrier = [&] __attribute__((always_inline)) {
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
        };
        const std::integral_constant<int, 0> k0;
        const std::integral_constant<int, 1> k1;
        const std::integral_constant<int, 2> k2;
        const std::integral_constant<int, 3> k3;
        if constexpr (TURNS) {
            // Two groups of four waves, one of each on a SIMD, take turns: one multiplies half a k-tile while the other fetches its
            // fragments and issues loads.  The second group runs one barrier behind.
            static_assert(STAGES == 2 && NL - NL / 2 <= (DUAL ? 3 : 2) * NM / 2, "the stage that is not read is loaded");
            const bool second = wave >= NW / 2;
            auto fetch = [&](auto half, unsigned stage) __attribute__((always_inline)) {
                constexpr int H = decltype(half)::value, S0 = DUAL ? H : 2 * H, S1 = DUAL ? H + 2 : 2 * H + 1;
                ra.template read<S0>(stage); rb.template read<S0>(stage);
                ra.template read<S1>(stage); rb.template read<S1>(stage);
            };
            auto fetched = [&](auto half) __attribute__((always_inline)) {
                constexpr int H = decltype(half)::value, S0 = DUAL ? 2 * H : 0;
                __builtin_amdgcn_s_waitcnt(0xc07f);            // lgkmcnt(0)
                ra.arrived(S0); rb.arrived(S0);
                ra.arrived(S0 + 1); rb.arrived(S0 + 1);
            };
            // half a k-tile of products; the first half's with the later loads, one at every second product
            auto multiply = [&](auto half) __attribute__((always_inline)) {
                constexpr int H = decltype(half)::value;
                __builtin_amdgcn_s_setprio(1);
#pragma unroll
                for (int p = 0; p < (DUAL ? 3 : 2); ++p)
#pragma unroll
                    for (int i = 0; i < FI; ++i)
#pragma unroll
                        for (int j = 0; j < FJ; ++j) {
                            const int n = (p * FI + i) * FJ + j;
                            if constexpr (DUAL) Mma<E, 32>::run(ra.get(2 * H + (p == 0), i), rb.get(2 * H + (p == 1), j), acc[i][j]);
                            else Mma<E, 32>::run(ra.get(p, i), rb.get(p, j), acc[i][j]);
                            if (H == 0 && n % 2 == 0 && NL / 2 + n / 2 < NL) issue_one(NL / 2 + n / 2);
                            __builtin_amdgcn_sched_barrier(0);
                        }
                __builtin_amdgcn_s_setprio(0);
            };
            if (second) barrier();
            unsigned st = 0;
            int sn = 0;
            for (int t = 0; t < total; ++t) {
                fetch(k0, st);
                tile_begin(sn ^ 1);                            // k-tile t + 1, where both groups have read all of k-tile t - 1
#pragma unroll
                for (int i = 0; i < NL / 2; ++i) issue_one(i);
                fetched(k0);
                barrier();
                mask_ahead();
                multiply(k0);
                barrier();
                fetch(k1, st);
                fetched(k1);
                if (second) wait_vmcnt<0>();                   // k-tile t + 1 has landed ahead of the barrier behind which the first group
                barrier();                                     // reads it: the second group fetches in front of that one, the first multiplies
                multiply(k1);
                if (!second) wait_vmcnt<0>();
                barrier();
                sn ^= 1;
                st = (unsigned)(sn * STAGE);
            }
            if (!second) barrier();
        } else if (loader) {
            // A wave that issues a load stands still for some 30 clocks, and where it is the only one of its SIMD the matrix core does so
            // too: here the loads have waves of their own.
            int sn = 0;
            for (int t = 0; t < total; ++t) {
                wait_vmcnt<(STAGES - 2) * NL>();               // k-tile t + 1 landed
                barrier();                                     // ... and k-tile t is read
                tile_begin(sn);
#pragma unroll
                for (int i = 0; i < NL; ++i) issue_one(i);
                if (++sn == STAGES) sn = 0;
            }
        } else {
            auto read = [&](auto k, unsigned stage) __attribute__((always_inline)) {
                constexpr int S = decltype(k)::value;
                ra.template read<S>(stage); rb.template read<S>(stage);
                if constexpr (DUAL) { ra.template read<S + 2>(stage); rb.template read<S + 2>(stage); }
            };
            read(k0, 0);
            arrived(0);
            unsigned st = 0;
            int sn = 0;
            for (int t = 0; t < total; ++t) {
                read(k1, st);
                __builtin_amdgcn_sched_barrier(0);
                // (in the first iteration all of the stages' loads are under way)
                products(0, NP, !LOADERS && t > 0);
                arrived(1);
                if constexpr (!DUAL) {
                    read(k2, st);
                    __builtin_amdgcn_sched_barrier(0);
                    products(1, 2 * NP, !LOADERS && t > 0);
                    arrived(0);
                    read(k3, st);
                    __builtin_amdgcn_sched_barrier(0);
                    products(0, 3 * NP, !LOADERS && t > 0);
                    arrived(1);
                }                                              // this wave has read all of its stage
                if constexpr (!LOADERS) wait_vmcnt<(STAGES - 2) * NL>();      // k-tile t + 1 landed (this wave's share)
                asm volatile("" ::: "memory");
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
                const int freed = sn;
                if (++sn == STAGES) sn = 0;
                st = (unsigned)(sn * STAGE);
                read(k0, st);                                      // (behind the last k-tile: zeros, not used)
                if constexpr (!LOADERS) tile_begin(freed);
                __builtin_amdgcn_sched_barrier(0);
                products(1, 0, !LOADERS);
                arrived(0);
            }
#pragma unroll
            for (int q = 0; q < NL; ++q)                       // what would have been issued in the next iteration: zeros
                if (!LOADERS && q * PLACES / NL >= NP) issue_one(q);
        }
        wait_vmcnt<0>();
        asm volatile("" ::: "memory");
        __syncthreads();
    }

    // index of accumulator register r inside its micro-tile: column j is lane & 31
    __device__ static __forceinline__ int row(int r, int lane) { return acc_row<32>(r, lane); }
};

// Which tile a workgroup of a product of ti x tj tiles has.  The hardware deals consecutive workgroups to the 8 XCDs in turn, each
// with an L2 of its own: an XCD gets consecutive tiles, and those go through bands of `band` tiles along j, so that the 32 that run
// at once on its compute units share rows of both operands.
__device__ __forceinline__ void gemm_tile_of(int block, int total, int ti, int tj, int band, int& i, int& j) {
    const int x = block & 7, per = total >> 3, rem = total & 7;
    const int t = x * per + (x < rem ? x : rem) + (block >> 3);
    const int full = band * ti, b = t / full, w = min(band, tj - b * band), in = t - b * full;
    i = in / w;
    j = b * band + in - i * w;
}

}  // namespace lp
