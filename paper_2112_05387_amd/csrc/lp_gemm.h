// Matrix product of 16-bit operands, one output tile per workgroup (gfx950):
//
//   D[i][j] = sum over pairs (a, b) of planes, sum over k of A_a[i, k] * B_b[j, k]        (fp32 sums)
//
// Values that need more than the 8 or 11 bits of a 16-bit float are kept as a sum of planes (x = x0 + x1 [+ x2], each the
// rounded rest of the ones before), and a product is the sum over those pairs of planes that matter.  Planes that lie apart: the pairs
// lie one after the other along the reduction, so the kernel is the same for one product and for several.
//
// An operand lies in memory with k contiguous (KR = false: rows i, pitch ld) or with its rows along k (KR = true: rows k, the
// index i contiguous).  Both come into LDS by direct loads of 1 KiB a wave, as they lie, and leave it as fragments of
// v_mfma_f32_32x32x16: the former by 16-byte reads, the latter by transposing reads (ds_read_b64_tr_b16: 16 lanes read four
// k of 16 rows and get four k of one row each).  So no operand is ever laid out anew for the other direction of a product.
//
// PL = 2 (DUAL), 3 (TRIPLE): both operands are sums of planes that lie beside each other, 32 elements of the first, the same 32 of the
// second [and of the third] in 128 [192] bytes, and a k-tile is 32 k of all.  From the fragments of two planes come three products, of
// three planes six (the others are below the precision): half as much again, or twice as much, for the same loads and LDS reads.
//
// A k-tile is 128 (192) bytes of a row long.  Eight waves (256 x 256 and 256 x 320, one workgroup a compute unit) are two groups that
// take turns, the loads of the next k-tile between their products.  Four waves (tiles of 128 and less) have four more beside them
// that only load; one barrier a k-tile, ahead of the products of its last 16 k, both frees its stage and shows the next.
// What bounds it: power, and the loads.  8192 x 8192 x 4096 in bf16 1105 (k contiguous), 1220 (one operand with rows along k), 1240
// TFLOP/s (both), DUAL 1440 of its three products, at 1.6 to 1.9 GHz, the matrix cores busy for 60 to 70 % of the clocks; without the
// loads 1270 to 1570 and 85 %.  All eight waves in step: 1013, 1128, 1203, 1370; half as many waves of 128 x 128 each, a third fewer LDS
// reads: 5 % less than that; fragments two k-steps ahead: the same.  DUAL in tiles of 128 x 128 over 8192, 64 and 256
// workgroups: 145 and 186 us without loading waves, 118 and 173 with.  TRIPLE: 73623 x 8716 over 633 1170 TFLOP/s of its six
// products, with the planes apart in 256 x 256 tiles 810; 230 workgroups of 128 x 128 over 1781 64 us, with planes apart 116.
// Rows are unpadded; their 16-byte chunks (KR: 32-byte pairs) trade places so that a read touches every bank once:
//   KR = false  chunk c of row r at c ^ (r >> 1 & 7)
//   KR = true   pair p of row k at p ^ 2 (k & 3) (rows of 256, 512 or 768 bytes), p ^ 2 (k >> 1 & 1) (128, 384 bytes), p (64 bytes)
//   TRIPLE, KR = false  chunk c of a plane of row r at c ^ (r >> 2 & 3)
// Ragged edges, tails of k and rows that are to count as zero are out-of-range buffer offsets, which read as zeros.
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>
#include <utility>

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

template <class E, bool AKR, bool BKR, int WI, int WJ, int FI, int FJ, int STAGES, bool MASKED = false, int PL = 1, bool PARTS = false> struct GemmTile {
    static constexpr int NW = WI * WJ;
    static constexpr bool TURNS = NW == 8, LOADERS = !TURNS;        // two waves a SIMD, one of either group; as many waves again that load (see run)
    static constexpr int NT = NW * 64 * (LOADERS ? 2 : 1);
    static constexpr int TI = FI * 32, TJ = FJ * 32, BI = WI * TI, BJ = WJ * TJ;
    static constexpr bool DUAL = PL == 2, TRIPLE = PL == 3;         // planes beside each other
    static constexpr int KT = PL == 1 ? 64 : 32, KS = KT / 16, RK = KT * PL * 2;    // k of a k-tile; bytes of a row (k contiguous)
    static constexpr int A_BYTES = BI * RK, STAGE = (BI + BJ) * RK, LDS = STAGES * STAGE;
    static constexpr int NSA = A_BYTES / 1024 / NW, NSB = (STAGE - A_BYTES) / 1024 / NW, NL = NSA + NSB;      // wave-loads of a k-tile
    static_assert(NW % 2 == 0 && NSA * NW * 1024 == A_BYTES && NL * NW * 1024 == STAGE, "every wave loads the same number of slabs");
    static_assert(TURNS || NW == 4, "one or two multiplying waves a SIMD");
    static_assert(!TRIPLE || (LOADERS && NSA % 3 == 0 && NSB % 3 == 0), "loads of three slabs, by waves of their own");
    static_assert(!PARTS || LOADERS, "registers for a second sum");
    typedef f32x16 Acc[FI][FJ];

    static constexpr unsigned kOOB = 0x80000000u;       // beyond any buffer of 2^31 - 1 bytes
    template <int N> __device__ static __forceinline__ void wait_vmcnt() {
        __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
    }
    __device__ static __forceinline__ __amdgpu_buffer_rsrc_t rsrc(const char* p) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p), 0, 0x7fffffff, 0x00020000);
    }

    // KR: the places of a row's 32-byte pairs
    template <int B> __device__ static __forceinline__ int swap(int k) {
        static_assert(!TRIPLE || B == 64 || B == 128, "rows of 384 or 768 bytes");
        constexpr int W = TRIPLE ? B : B * PL;
        return W >= 128 ? (k & 3) << 1 : W == 64 ? ((k >> 1) & 1) << 1 : 0;
    }

    // One operand's loads: lane's offset in a slab, and what it has to compare with at the edges.
    template <bool KR, int B, int NS> struct Loader {
        static constexpr int RB = KR ? B * PL * 2 : RK;                 // bytes of a row of the stage
        // a wave's slabs: every NW-th; TRIPLE, where only three of them are whole rows: consecutive ones, PERIOD = 3
        static constexpr int PERIOD = TRIPLE ? 3 : 1, RPP = PERIOD * 1024 / RB, RSTEP = TRIPLE ? RPP : NW * RPP;
        const char* base; size_t plane; int ldb;        // bytes of a row of the operand
        unsigned voff[PERIOD]; int row[PERIOD], chunk, last;      // row: this lane's in slab 0; last: rows that exist from row 0 of the tile on
        int step;                                       // bytes between the slabs (periods) of a wave

        __device__ __forceinline__ void init(const GemmOperand& o, int x0, int lane, int wave) {
            ldb = o.ld * 2; plane = o.plane;
            if constexpr (TRIPLE) {
                constexpr int CPR = RB / 16;
                chunk = 0;
                base = KR ? o.base : o.base + (size_t)x0 * ldb;
                last = KR ? 0 : o.extent - x0;
#pragma unroll
                for (int b = 0; b < 3; ++b) {
                    const int q = b * 64 + lane, pos = q % CPR;
                    row[b] = wave * (NS / 3) * RPP + q / CPR;
                    if constexpr (!KR) voff[b] = (unsigned)(row[b] * ldb + (pos ^ ((row[b] >> 2) & 3)) * 16);
                    else {
                        const int col = x0 * 3 + (((pos >> 1) ^ swap<B>(row[b])) << 4) + (pos & 1) * 8;
                        voff[b] = col < o.extent ? (unsigned)(row[b] * ldb + col * 2) : kOOB;
                    }
                }
            } else if constexpr (!KR) {
                const int pos = lane & 7;
                chunk = pos ^ (4 * (wave & 1) + (lane >> 4));
                row[0] = wave * 8 + (lane >> 3);
                base = o.base + (size_t)x0 * ldb;
                last = o.extent - x0;
                voff[0] = (unsigned)(row[0] * ldb + chunk * 16);
            } else {
                constexpr int CPR = RB / 16;
                const int sub = lane / CPR, pos = lane % CPR;
                row[0] = wave * RPP + sub;
                const int f = swap<B>(row[0]);
                const int col = x0 * PL + (((pos >> 1) ^ f) << 4) + (pos & 1) * 8;
                base = o.base; chunk = 0; last = 0;
                voff[0] = col < o.extent ? (unsigned)(row[0] * ldb + col * 2) : kOOB;
            }
            step = RSTEP * ldb;
        }
        // load i of the k-tile that starts at k (krem: k that are left), of the plane at `p`
        __device__ __forceinline__ unsigned offset(int i, int krem, unsigned long long mask) const {
            const int b = i % PERIOD, r = row[b] + i / PERIOD * RSTEP;
            if constexpr (!KR) return r < last && (PL > 1 ? 0 : chunk * 8) < krem ? voff[b] : kOOB;
            else {
                bool ok = r < krem;
                if constexpr (MASKED) ok = ok && ((mask >> r) & 1ull);
                return ok ? voff[b] : kOOB;
            }
        }
        __device__ __forceinline__ int behind(int i) const { return i / PERIOD * step; }
        // where slab i of wave `wave` goes
        __device__ static __forceinline__ int place(int wave, int i) { return (TRIPLE ? wave * NS + i : i * NW + wave) * 1024; }
        __device__ __forceinline__ const char* at(int p, int k) const {
            return base + (size_t)p * plane + (KR ? (size_t)k * ldb : (size_t)k * 2 * PL);
        }
    };

    // Fragments are read by inline assembly and waited for explicitly: in front of the built-in of the transposing read the compiler
    // waits for every load to LDS that is under way.  Nothing may touch a fragment between read() and arrived(), which is
    // where its value becomes usable; no fragment is under way where control flow joins.
    template <bool KR, int B, int F> struct Reader {
        static constexpr int RB = B * PL * 2;
        unsigned addr[KR ? (TRIPLE ? 3 * F : F) : TRIPLE ? 2 : 4];
        u32x4 whole[2 * PL][KR ? 1 : F];               // several planes: [k-step][plane]
        u32x2 half[2 * PL][KR ? F : 1][2];

        __device__ __forceinline__ void init(int w, int lane, unsigned lds0) {
            if constexpr (!KR) {
                const int r = lane & 31, sw = TRIPLE ? (r >> 2) & 3 : (r >> 1) & 7;
#pragma unroll
                for (int ks = 0; ks < (TRIPLE ? 2 : 4); ++ks) addr[ks] = lds0 + (w * F * 32 + r) * RK + (((2 * ks + (lane >> 5)) ^ sw) << 4);
            } else {
                const int lq = lane & 15, k = 8 * (lane >> 5) + (lq >> 2);
                const int f = swap<B>(k);
#pragma unroll
                for (int m = 0; m < F; ++m)
#pragma unroll
                    for (int p = 0; p < (TRIPLE ? 3 : 1); ++p)
                        addr[TRIPLE ? 3 * m + p : m] = lds0 + k * RB + (((2 * PL * (w * F + m) + 2 * p + ((lane >> 4) & 1)) ^ f) << 5) + 8 * (lq & 3);
            }
        }
        // the fragments of k-step S of the stage that starts at byte `st` (several planes: S = 2 * plane + k-step of the k-tile's two)
        template <int S, int M> __device__ __forceinline__ void read_one(unsigned st) {
            constexpr int slot = PL > 1 ? PL * (S & 1) + (S >> 1) : S & 1;   // [k-step][plane], or two k-steps
            if constexpr (!KR)
                asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(whole[slot][M]) : "v"(addr[TRIPLE ? S & 1 : S] + st), "i"(M * 32 * RK + (TRIPLE ? S / 2 * 64 : 0)));
            else {
                constexpr int off = (PL > 1 ? S & 1 : S) * 16 * RB;
                // DUAL: the second plane two pairs on
                const unsigned a = (TRIPLE ? addr[3 * M + S / 2] : DUAL && S >= 2 ? addr[M] ^ 64u : addr[M]) + st;
                asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(half[slot][M][0]) : "v"(a), "i"(off));
                asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(half[slot][M][1]) : "v"(a), "i"(off + 4 * RB));
            }
        }
        template <int S, int M = 0> __device__ __forceinline__ void read(unsigned st) {
            if constexpr (M < F) {
                read_one<S, M>(st);
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

    // f of every constant of a list
    template <class F, int... Q> __device__ static __forceinline__ void each(std::integer_sequence<int, Q...>, F f) { (f(std::integral_constant<int, Q>()), ...); }

    // waves that have no share of the result
    __device__ static __forceinline__ bool idle() { return LOADERS && (int)threadIdx.x >= NW * 64; }

    // Adds to acc the products of rows i0.. of A and j0.. of B over k in [kb, ke), kb a multiple of 64.  (Several planes: one pair, and operands
    // with k contiguous are zero behind ke up to a multiple of 32.)  mask (MASKED): bit k & 63
    // of word k >> 6 is set where A's row k counts.  Ends with every load landed and all waves past their last LDS read.
    // PARTS: every `every` k-tiles (0: never) acc is added to a sum of its own and starts from zero again, as a product that is added to a
    // long sum is cut to that sum's last bit.
    __device__ static __forceinline__ void run(const GemmOperand& A, const GemmOperand& B, const GemmPairs& pairs, int i0, int j0, int kb, int ke,
                                               GemmMask mask, unsigned char* smem, Acc& acc, int every = 0) {
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
            if constexpr (MASKED) t_mask = TURNS ? ahead : mask[min(k, ke - 1) >> 6] >> (k & 63);
            t_dst = smem + st * STAGE;
            ++issued;
            if (++kt == nkt) { kt = 0; if (seg + 1 < pairs.n) ++seg; }
        };
        auto mask_ahead = [&] __attribute__((always_inline)) {
            if constexpr (MASKED && TURNS) ahead = mask[min(kb + kt * KT, ke - 1) >> 6];
        };
        auto issue_one = [&](int i) __attribute__((always_inline)) {
            if (i < NSA)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc(pa), (gemm_lds_t)(t_dst + la.place(wave, i)), 16, (int)la.offset(i, t_krem, t_mask), la.behind(i), 0, 0);
            else if (i < NL)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc(pb), (gemm_lds_t)(t_dst + A_BYTES + lb.place(wave, i - NSA)), 16,
                                                         (int)lb.offset(i - NSA, t_krem, ~0ull), lb.behind(i - NSA), 0, 0);
        };
        auto arrived = [&](int slot) __attribute__((always_inline)) {
            __builtin_amdgcn_s_waitcnt(0xc07f);                // lgkmcnt(0)
#pragma unroll
            for (int p = 0; p < PL; ++p) {
                ra.arrived(PL * slot + p);
                rb.arrived(PL * slot + p);
            }
        };
        constexpr int NM = FI * FJ, NP = TRIPLE ? 6 * NM : DUAL ? 3 * NM : NM;   // products of a k-step
        // Several planes: the small terms first.  `ahead_of(n)` comes ahead of product n.
        auto products = [&](int slot, auto ahead_of) __attribute__((always_inline)) {
#pragma unroll
            for (int p = 0; p < NP / NM; ++p) {
                constexpr int pair_a[6] = {2, 0, 1, 1, 0, 0}, pair_b[6] = {0, 2, 1, 0, 1, 0};
#pragma unroll
                for (int i = 0; i < FI; ++i)
#pragma unroll
                    for (int j = 0; j < FJ; ++j) {
                        ahead_of(p * NM + i * FJ + j);
                        __builtin_amdgcn_sched_barrier(0);
                        if constexpr (TRIPLE) Mma<E, 32>::run(ra.get(3 * slot + pair_a[p], i), rb.get(3 * slot + pair_b[p], j), acc[i][j]);
                        else if constexpr (DUAL) Mma<E, 32>::run(ra.get(2 * slot + (p == 0), i), rb.get(2 * slot + (p == 1), j), acc[i][j]);
                        else Mma<E, 32>::run(ra.get(slot, i), rb.get(slot, j), acc[i][j]);
                        __builtin_amdgcn_sched_barrier(0);
                    }
            }
        };
        if (TURNS || loader) {
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
            // The fragments of the next k-step.  A wave that issues an LDS read stands still for a while, and it is the only one of its SIMD
            // that multiplies: where there are half as many products again as reads, the reads are spread over the first two thirds of
            // them (128 x 128, two planes: 201 workgroups over 5760 115 -> 105 us; three, rows along k: 510 -> 440).  Where there are fewer
            // (one plane, or 64 x 64) that is up to 10 % slower than reading ahead of the products, three planes one at a time.
            constexpr int NR = PL * (FI + FJ), SPAN = NP * 2 / 3;
            constexpr bool BETWEEN = 2 * NP >= 3 * NR;
            auto fragment = [&](auto k, auto q, unsigned stage) __attribute__((always_inline)) {
                constexpr int S = decltype(k)::value + 2 * (decltype(q)::value / (FI + FJ)), M = decltype(q)::value % (FI + FJ);
                if constexpr (M < FI) ra.template read_one<S, M>(stage);
                else rb.template read_one<S, M - FI>(stage);
            };
            auto step = [&](auto k, unsigned stage, int slot) __attribute__((always_inline)) {
                products(slot, [&](int n) __attribute__((always_inline)) {
                    each(std::make_integer_sequence<int, NR>(), [&](auto q) __attribute__((always_inline)) {
                        constexpr int Q = decltype(q)::value;
                        if (n == (BETWEEN ? Q * SPAN / NR + 1 : TRIPLE ? Q / (FI + FJ) * NM : 0)) fragment(k, q, stage);
                    });
                });
                arrived(slot ^ 1);
            };
            each(std::make_integer_sequence<int, NR>(), [&](auto q) __attribute__((always_inline)) { fragment(k0, q, 0u); });
            arrived(0);
            unsigned st = 0;
            int sn = 0, left = every;
            Acc whole;
            auto join = [&](bool last) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < FI; ++i)
#pragma unroll
                    for (int j = 0; j < FJ; ++j)
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            whole[i][j][e] += acc[i][j][e];
                            acc[i][j][e] = last ? whole[i][j][e] : 0.f;
                        }
            };
            if constexpr (PARTS) {
#pragma unroll
                for (int i = 0; i < FI; ++i)
#pragma unroll
                    for (int j = 0; j < FJ; ++j)
#pragma unroll
                        for (int e = 0; e < 16; ++e) whole[i][j][e] = 0.f;
            }
            for (int t = 0; t < total; ++t) {
                step(k1, st, 0);
                if constexpr (PL == 1) {
                    step(k2, st, 1);
                    step(k3, st, 0);
                }                                              // this wave has read all of its stage
                asm volatile("" ::: "memory");
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
                if (++sn == STAGES) sn = 0;
                st = (unsigned)(sn * STAGE);
                step(k0, st, 1);                               // (behind the last k-tile it reads zeros, not used)
                if constexpr (PARTS)
                    if (--left == 0) { join(false); left = every; }
            }
            if constexpr (PARTS) join(true);
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
