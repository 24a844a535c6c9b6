// Matrix product of two block-scaled 8-bit operands,
//   out[m, n] = sum_b 2^(ea[b, m] + eb[b, n] - 254) sum_{k in block b} a[m, k] b[n, k],
// both with the contraction innermost.  v_mfma_scale_f32_16x16x128 multiplies 16 rows by 16 columns over a whole block of 128
// and takes the exponents as operands, so the sum over blocks stays in one fp32 accumulator.  With lane l, lo = l % 16, hi = l / 16:
//   A, B operand: lane holds 32 bytes of row lo; which of the block's bytes only has to be the same on both sides, as all
//                 lanes of a row pass the same exponent: chunks hi and hi + 4 of the block's eight 16-byte chunks
//   C: lane holds C[4 hi + r][lo] in register r
// Row lo of fragment i of a group of 64 rows is row 4 lo + i: the exponents of a lane's four fragments are then one 32-bit word,
// of which the instruction picks byte i, and a lane's results for four fragments of b are four neighbouring columns of out.
//
// That instruction adds its 128 products in groups of eight, aligned to the group's largest: what lies 14 binary places below is
// lost (measured: 2^16 + 2^3 is exact inside a group, 2^16 + 2^2 gives 2^16; between groups and into the accumulator the sums are
// those of fp32).  N(0, 1) operands come out 1.5e-5 off, a hundredth of a bf16 result's rounding, so results in bf16 are made this way.
// Results in fp32 are sums in fp32 throughout: their operands are widened to bf16, which holds every 8-bit value times
// its scale exactly while that stays in bf16's range, and multiplied by v_mfma_f32_16x16x32_bf16, at half the rate.
#include "attn_common.h"
#include "fp8_matmul_ways.h"
#include "sp_common.h"

namespace {

using sp::f32x4;
using sp::u32x2;
using sp::u32x4;
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

struct MatmulArgs {
    const uint8_t* a; const uint8_t* a_scale;
    const uint8_t* b; const uint8_t* b_scale;
    void* out;
    uint32_t M, N, K;          // below 2^31; 32 bits, as the scalar unit compares no more
    uint32_t a_pitch, b_pitch; // of the scales: M, N rounded up to 16
    bool accumulate;           // fp32 results only
};

// Eight 8-bit values over their scale (bytes 8 PART .. 8 PART + 7 of a lane's 32, scale exponent in byte I of a word) as bf16.
template <bool E5M2, int I, int PART>
__device__ __forceinline__ sp::bf16x8 widen(const i32x8& v, int exponents) {
    const float scale = __builtin_bit_cast(float, (((uint32_t)exponents >> (8 * I)) & 255u) << 23);
    sp::bf16x8 r;
    sp::static_for<0, 4>([&](auto h) {
        sp::bf16x2 p;
        if constexpr (E5M2) p = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(v[2 * PART + h / 2], scale, h % 2 == 1);
        else p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * PART + h / 2], scale, h % 2 == 1);
        r[2 * h] = p[0];
        r[2 * h + 1] = p[1];
    });
    return r;
}

// acc += the product of a fragment of a, exponents in byte I of ea, and one of b, in byte J of eb, with the accumulator held in place in
// the accumulation registers (the compiler moves it about in a kernel that fills the register file).  The compiler does not know that
// this is a matrix instruction: operands come from LDS reads, whose waits it places, and the results are read only behind
// matrix_results().
template <bool E5M2, int I, int J>
__device__ __forceinline__ void multiply_in_place(f32x4& acc, const i32x8& a, const i32x8& b, int ea, int eb) {
    asm volatile(SP_MFMA_PRE "v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[%5,%6,0] op_sel_hi:[%7,%8,0] cbsz:%9" SP_MFMA_POST
                 : "+a"(acc)
                 : "v"(a), "v"(b), "v"(ea), "v"(eb), "n"(I & 1), "n"(J & 1), "n"(I >> 1), "n"(J >> 1), "n"(E5M2 ? 1 : 0));
}
// zeros, likewise in place: the smallest matrix instruction, of zeros
__device__ __forceinline__ void clear_in_place(f32x4& acc, const u32x2& zeros) {
    asm volatile(SP_MFMA_PRE "v_mfma_f32_4x4x4_16b_bf16 %0, %1, %1, 0" SP_MFMA_POST : "+a"(acc) : "v"(zeros));
}
// Nothing but the accumulators themselves keeps a read of them behind the wait, so the statements behind it hand each one on, and
// nothing is scheduled across them (without either, copies for a store's operand went in front of the wait).
template <int NA, int NB>
__device__ __forceinline__ void matrix_results(f32x4 (&acc)[NA][NB]) {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 15\n\ts_nop 7" ::: "memory");
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) asm volatile("" : "+a"(acc[i][j]));
    __builtin_amdgcn_sched_barrier(0);
}

__device__ __forceinline__ i32x8 join(const u32x4& lo, const u32x4& hi) {
    i32x8 r;
#pragma unroll
    for (int e = 0; e < 4; ++e) { r[e] = (int)lo[e]; r[4 + e] = (int)hi[e]; }
    return r;
}

// four neighbouring results of row m from column n on, fp32 and bf16 (two in a word)
__device__ __forceinline__ void store4(const MatmulArgs& p, uint32_t m, uint32_t n, f32x4 v) {
    if (m >= p.M || n >= p.N) return;
    float* const o = (float*)p.out + ((size_t)m * p.N + n);
    if (p.N % 4 == 0) {
        f32x4* const whole = reinterpret_cast<f32x4*>(o);
        *whole = p.accumulate ? *whole + v : v;
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (n + e < p.N) o[e] = p.accumulate ? o[e] + v[e] : v[e];
}
__device__ __forceinline__ void store4(const MatmulArgs& p, uint32_t m, uint32_t n, u32x2 v) {
    if (m >= p.M || n >= p.N) return;
    uint16_t* const o = (uint16_t*)p.out + ((size_t)m * p.N + n);
    if (p.N % 4 == 0) {
        *reinterpret_cast<u32x2*>(o) = v;
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (n + e < p.N) o[e] = (uint16_t)(v[e / 2] >> (e % 2 * 16));
}

// ------------------------------------------------------------------ tiles through LDS
// A workgroup of WR x WC waves makes TM x TN results, each wave 64 GM x 64 GN of them.  Per block of 128 the tile's rows of a and
// of b and the exponents that each wave needs are copied into one of STAGES stages of LDS.
//
// LDS row of row 64 g + 4 lo + i of the tile: 64 g + 16 i + lo, so that the 16 lanes that read a fragment read neighbouring LDS
// rows; the 16-byte chunk c of LDS row s lies at chunk position c ^ (s/2 % 8), which puts the same chunk of 16 neighbouring rows
// on all 64 banks.
template <int GM, int GN, int WR, int WC>
struct Tile {
    static constexpr int kWaves = WR * WC, kCols = WC, kM = 64 * GM * WR, kN = 64 * GN * WC;
    static constexpr int kCopies = (kM + kN) / 8 / kWaves;  // of 1024 bytes (8 rows) per wave and stage, the exponents' not counted
    static constexpr int kA = 0, kB = kM * 128, kScale = kB + kN * 128, kStage = kScale + kWaves * 256;
    static_assert(kWaves % 2 == 0 && (kM / 8) % kWaves == 0 && (kN / 8) % kWaves == 0 && 16 * (GM + GN) <= 64, "");
};

// Raw buffers of 32-bit format: loads beyond the end give zeros and stores there are dropped, so rows behind the matrix's last
// need no care.
constexpr int kRawBuffer = 0x00020000;
// up to `most` rows of `pitch` bytes from row0 on
__device__ __forceinline__ i32x4 rows_from(const uint8_t* base, uint32_t row0, uint32_t rows, uint32_t most, uint32_t pitch) {
    const uint64_t at = (uint64_t)base + (uint64_t)row0 * pitch;
    return i32x4{(int)(uint32_t)at, (int)(uint32_t)(at >> 32), (int)((rows - row0 < most ? rows - row0 : most) * pitch), kRawBuffer};
}

// 1024 bytes from memory to LDS, 16 per lane from its offset plus `scalar` in the resource to `to` + 16 * lane; and 256, 4 per lane from
// its address.  Issued as assembly: the compiler would wait for every copy under way before any read of LDS, as it cannot tell the
// stages apart.  No register waits for a copy, so nothing is hidden from it but LDS, whose order the kernels' own waits and
// barriers give, and what it may do to m0 and to the scalar operands just before, which a test reads from its output.
__device__ __forceinline__ void copy_16(uint32_t to, const i32x4& from, int off, int scalar) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(to), "v"(off), "s"(from), "s"(scalar) : "memory");
}
__device__ __forceinline__ void copy_4(uint32_t to, const uint8_t* from) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(to), "v"(from) : "memory");
}

// A wave's share of the copies: copy j brings the eight LDS rows of number wave + kWaves * j in a's, then b's part of the stage.
// What differs from lane to lane is one 32-bit offset per copy, the same in a and in b, and the block's is scalar.
template <typename T, int GM, int GN>
struct Copier {
    static constexpr int kPerA = T::kM / 8 / T::kWaves, kPerB = T::kN / 8 / T::kWaves;
    i32x4 a, b;           // buffer resources: the tile's rows
    int off[kPerA > kPerB ? kPerA : kPerB];  // of this lane's 16 bytes from the tile's first row, block 0
    int block_off;        // of the block to be copied
    const uint8_t* scale; // this lane's exponents of it
    uint32_t scale_step;
    int wave, lane;

    __device__ __forceinline__ Copier(const MatmulArgs& p, int wave_, int lane_) : wave(wave_), lane(lane_) {
        sp::static_for<0, (kPerA > kPerB ? kPerA : kPerB)>([&](auto j) {
            const int s = 8 * (wave + T::kWaves * j) + (lane >> 3), chunk = (lane & 7) ^ ((s >> 1) & 7);
            off[j] = (64 * (s >> 6) + 4 * (s & 15) + ((s >> 4) & 3)) * (int)p.K + 16 * chunk;
        });
    }
    // the first block of the tile at m0, n0
    __device__ __forceinline__ void tile(const MatmulArgs& p, uint32_t m0, uint32_t n0) {
        a = rows_from(p.a, m0, p.M, T::kM, p.K);
        b = rows_from(p.b, n0, p.N, T::kN, p.K);
        block_off = 0;
        // lanes 0 .. 16 GM - 1: words of a's exponents, the next 16 GN: of b's; the rest repeat the last
        const int w = lane < 16 * (GM + GN) ? lane : 16 * (GM + GN) - 1;
        const bool of_a = w < 16 * GM;
        const uint32_t row = of_a ? m0 + 64 * GM * (wave / T::kCols) + 4 * w : n0 + 64 * GN * (wave % T::kCols) + 4 * (w - 16 * GM);
        const uint32_t pitch = of_a ? p.a_pitch : p.b_pitch;
        scale = (of_a ? p.a_scale : p.b_scale) + (row < pitch ? row : 0);
        scale_step = pitch;
    }
    // copy J (of kCopies + 1) of the block to the stage at this LDS address
    template <int J>
    __device__ __forceinline__ void copy(uint32_t stage) const {
        if constexpr (J == T::kCopies) {
            copy_4(stage + T::kScale + wave * 256, scale);
        } else {
            constexpr bool is_a = J < kPerA;
            constexpr int j = is_a ? J : J - kPerA;
            const uint32_t to = stage + (is_a ? T::kA : T::kB) + (wave + T::kWaves * j) * 1024;
            copy_16(to, is_a ? a : b, off[j], block_off);
        }
    }
    // the next block, or one of zeros if there is none (its exponents are the last block's)
    __device__ __forceinline__ void next(bool more = true) {
        block_off += 128;
        scale += more ? scale_step : 0;
        a[2] = more ? a[2] : 0;
        b[2] = more ? b[2] : 0;
    }
};

// tiles in the order workgroups take them: workgroups go to the eight XCDs in turn, so each XCD gets a run of tiles, and a run
// walks kBand tile rows together, so that the tiles that an XCD works on at a time share rows of a and of b in its L2
constexpr uint32_t kBand = 8;
__device__ __forceinline__ void tile_of(uint32_t wg, uint32_t mt, uint32_t nt, uint32_t& tm, uint32_t& tn) {
    const uint32_t n = mt * nt, xcd = wg & 7, each = n >> 3, extra = n & 7;
    const uint32_t t = xcd * each + (xcd < extra ? xcd : extra) + (wg >> 3);
    const uint32_t band = t / (kBand * nt), in = t - band * kBand * nt;
    const uint32_t rows = mt - band * kBand < kBand ? mt - band * kBand : kBand;
    tn = in / rows;
    tm = band * kBand + in - tn * rows;
}

template <int N>
__device__ __forceinline__ void wait_copies_and_meet() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

__device__ __forceinline__ i32x8 fragment(const uint8_t* rows, int at) {
    return join(*reinterpret_cast<const u32x4*>(rows + at), *reinterpret_cast<const u32x4*>(rows + (at ^ 64)));
}

// Results in fp32: 64 x 64 per wave, two workgroups per compute unit.  The widened operands go to the matrix instruction as they are
// made, and the products, twice as long as those in 8 bits, cover the copies of the next block and the other workgroup's reads.
// What the results are added to is read under the last block's products; behind them, where all workgroups come at about the same
// time, reads and stores took turns (28672 x 4096 x 512 297 against 208 us, 6144 x 4096 x 4096 194 / 184).
// Bound by the conversions, a quarter of the vector unit's rate: twice the cycles of the products, on the other unit.  28672 x 4096 x
// 16384 3110 us, 1240 TFLOP/s, where the library's product of bf16 operands, which has nothing to convert, takes 2370; 6144 x 4096 x 4096
// 182 and 152.  Waves of 128 x 64, which convert three quarters of it, were slower with two workgroups of one stage (spills) and 3 to
// 6 % faster as a pipeline with one workgroup a unit (6144 x 4096 x 4096 170 -> 165 us); that pipeline is not here.
template <bool E5M2>
__global__ __launch_bounds__(256, 2) void matmul_f32_kernel(MatmulArgs p, uint32_t mt, uint32_t nt) {
    typedef Tile<1, 1, 2, 2> T;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * T::kStage];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lo = lane & 15, hi = lane >> 4;
    const int wr = wave >> 1, wc = wave & 1;
    uint32_t tm, tn;
    tile_of(blockIdx.x, mt, nt, tm, tn);
    const uint32_t m0 = tm * T::kM, n0 = tn * T::kN;
    Copier<T, 1, 1> from(p, wave, lane);
    from.tile(p, m0, n0);
    f32x4 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int blocks = (int)(p.K / 128);
    const uint32_t base = sp::lds_addr(lds);
    auto copy_all = [&](uint32_t stage) __attribute__((always_inline)) {
        sp::static_for<0, T::kCopies + 1>([&](auto j) { from.template copy<j>(base + stage); });
    };
    if (blocks > 0) copy_all(0);
    const int at = lo * 128 + ((hi ^ (lo >> 1)) << 4);
    f32x4 old[4][4];
    const bool add = p.accumulate && p.N % 4 == 0;
    auto read_old = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const uint32_t m = m0 + wr * 64 + 4 * (4 * hi + r) + i, n = n0 + wc * 64 + 4 * lo;
                old[i][r] = m < p.M && n < p.N ? *reinterpret_cast<const f32x4*>((const float*)p.out + ((size_t)m * p.N + n)) : f32x4{0.f, 0.f, 0.f, 0.f};
            }
    };
    uint32_t cur = 0;
    for (int kb = 0; kb < blocks; ++kb) {
        from.next(kb + 1 < blocks);
        wait_copies_and_meet<0>();
        if (add && kb + 1 == blocks) read_old();
        if (kb + 1 < blocks) copy_all(T::kStage - cur);
        const uint8_t* st = lds + cur;
        const int ea = *reinterpret_cast<const int*>(st + T::kScale + wave * 256 + lo * 4);
        const int eb = *reinterpret_cast<const int*>(st + T::kScale + wave * 256 + 64 + lo * 4);
        i32x8 fa[4], fb[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            fa[i] = fragment(st + T::kA + wr * 8192 + i * 2048, at);
            fb[i] = fragment(st + T::kB + wc * 8192 + i * 2048, at);
        }
        sp::static_for<0, 4>([&](auto part) {
            sp::bf16x8 wa[4], wb[4];
            sp::static_for<0, 4>([&](auto i) {
                wa[i] = widen<E5M2, i, part>(fa[i], ea);
                wb[i] = widen<false, i, part>(fb[i], eb);
            });
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wa[i], wb[j], acc[i][j], 0, 0, 0);
        });
        cur = T::kStage - cur;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const uint32_t m = m0 + wr * 64 + 4 * (4 * hi + r) + i, n = n0 + wc * 64 + 4 * lo;
            const f32x4 v = {acc[i][0][r], acc[i][1][r], acc[i][2][r], acc[i][3][r]};
            if (add && blocks > 0) {
                if (m < p.M && n < p.N) *reinterpret_cast<f32x4*>((float*)p.out + ((size_t)m * p.N + n)) = old[i][r] + v;
            } else {
                store4(p, m, n, v);
            }
        }
}

// 64 GM x 64 GN results per wave as a software pipeline over the blocks: while the products of a fragment of a run, the fragment
// after the next is read; all fragments of b are held, in two sets.  A stage has been read through when the second last fragment of
// a is multiplied: there the waves meet, copies start into it, spread over the products, and the next block's fragments are read
// under the last products.
// A workgroup takes tiles wg, wg + gridDim.x, ... and the pipeline runs through: the copies go on with the next tile's blocks, and
// its first fragments are in registers when the results of the last are stored.  Steps come in pairs, one for either set; an odd
// number of blocks is filled up with one of zeros.  K > 0.
// 16384 x 28672 x 4096 in tiles of 256 x 256: 1387 us, 2780 TFLOP/s, the library's product with one scale, in turn on the same card, 1268;
// 8192^3 347 and 339, 4096 x 6144 x 4096 84 and 86.  The matrix unit is busy 0.73 of the cycles, the rest goes where the waves meet.  Power
// sets the clock, so the card and the operands' values do the rest: the first takes 1340 to 1430 us.  256 x 128 1597 us, 128 x 128 2070
// (256 x 256 1336 in that run): 48 and 32 KB of copies for a half and a quarter of the products.
// SPLIT: a tile's blocks are shared out among `splits` workgroups, `per` blocks each (the last may have fewer), whose sums go in fp32
// to the workspace [splits][M][N rounded up to 4]; add_splits_kernel adds them in order.
// workgroups per compute unit, by the 160 KiB of LDS
constexpr int pipe_groups(int GM, int GN, int STAGES) { return STAGES * ((GM + GN) * 2 * 64 * 128 + 1024) <= 80 * 1024 ? 2 : 1; }
template <int GM, int GN, int STAGES, bool E5M2, bool SPLIT>
__global__ __launch_bounds__(256, pipe_groups(GM, GN, STAGES)) void matmul_pipe_kernel(MatmulArgs p, uint32_t mt, uint32_t nt, uint32_t splits, uint32_t per) {
    typedef Tile<GM, GN, 2, 2> T;
    constexpr int NA = 4 * GM, NB = 4 * GN, kMeet = (NA - 2) * NB;
    // Copies of the block STAGES - 1 ahead: the first kEarly behind the meeting point of a step, the rest in the first products of
    // the next step, one every other product; then the copier moves on.
    constexpr int kEarly = GM * GN == 1 ? 5 : NB, kLate = T::kCopies + 1 - kEarly;
    static_assert(2 * kLate <= kMeet && kEarly <= 2 * NB && (STAGES - 1) * (T::kCopies + 1) < 64, "");
    __shared__ __attribute__((aligned(1024))) uint8_t lds[STAGES * T::kStage];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lo = lane & 15, hi = lane >> 4;
    const int wr = wave >> 1, wc = wave & 1;
    const uint32_t whole = mt * nt, tiles = SPLIT ? whole * splits : whole;
    const int all_blocks = (int)(p.K / 128), most = SPLIT ? (int)per : all_blocks, pairs = (most + 1) / 2;
    int blocks = all_blocks;  // of the copier's tile
    const int at = lo * 128 + ((hi ^ (lo >> 1)) << 4);
    const uint32_t base = sp::lds_addr(lds);

    Copier<T, GM, GN> from(p, wave, lane);
    auto go_to_tile = [&](uint32_t t) __attribute__((always_inline)) {
        uint32_t tm, tn;
        tile_of(SPLIT ? t % whole : t, mt, nt, tm, tn);
        from.tile(p, tm * T::kM, tn * T::kN);
        if constexpr (SPLIT) {
            const int first = (int)(t / whole * per);
            blocks = all_blocks - first < (int)per ? all_blocks - first : (int)per;
            from.block_off = first * 128;
            from.scale += (size_t)first * from.scale_step;
        }
    };

    f32x4 acc[NA][NB];
    auto clear = [&]() __attribute__((always_inline)) {
        const u32x2 zeros = {0u, 0u};
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) clear_in_place(acc[i][j], zeros);
    };
    i32x8 fa[4], fb[2][NB];
    int ea[2][GM], eb[2][GN];
    auto read_a = [&](uint32_t stage, auto i) __attribute__((always_inline)) {
        fa[i % 4] = fragment(lds + stage + T::kA + wr * GM * 8192 + i * 2048, at);
    };
    auto read_b = [&](auto set, uint32_t stage, auto j) __attribute__((always_inline)) {
        fb[set][j] = fragment(lds + stage + T::kB + wc * GN * 8192 + j * 2048, at);
    };
    auto read_scales = [&](auto set, uint32_t stage) __attribute__((always_inline)) {
        const uint8_t* s = lds + stage + T::kScale + wave * 256 + lo * 4;
#pragma unroll
        for (int g = 0; g < GM; ++g) ea[set][g] = *reinterpret_cast<const int*>(s + 64 * g);
#pragma unroll
        for (int g = 0; g < GN; ++g) eb[set][g] = *reinterpret_cast<const int*>(s + 64 * GM + 64 * g);
    };
    // stages (bytes from the first): of this block, of the next, of the one whose copies are under way
    uint32_t cur = 0, next = T::kStage, under_way = (STAGES - 1) * T::kStage;
    auto step = [&](auto set, auto move_on) __attribute__((always_inline)) {
        constexpr int S = set;
        const uint32_t s_cur = STAGES == 2 ? S * T::kStage : cur, s_next = STAGES == 2 ? (1 - S) * T::kStage : next,
                       s_late = STAGES == 2 ? (1 - S) * T::kStage : under_way;
        sp::static_for<0, NA * NB>([&](auto slot) {
            constexpr int i = slot / NB, j = slot % NB, past = slot - kMeet;
            if constexpr (past < 0 && j == 0) read_a(s_cur, sp::Int<i + 2>{});
            if constexpr (slot % 2 == 1 && slot / 2 < kLate) from.template copy<kEarly + slot / 2>(base + s_late);
            if constexpr (slot == 2 * kLate) move_on();
            if constexpr (past == 0) {
                wait_copies_and_meet<(STAGES - 2) * (T::kCopies + 1)>();
                read_scales(sp::Int<1 - S>{}, s_next);
            }
            if constexpr (past >= 0) {
                if constexpr (past % 2 == 0) read_b(sp::Int<1 - S>{}, s_next, sp::Int<past / 2>{});
                if constexpr (past == 3 || past == 7) read_a(s_next, sp::Int<past / 4>{});
                if constexpr (kEarly == NB ? past % 2 == 1 : past < kEarly) from.template copy<kEarly == NB ? past / 2 : past>(base + s_cur);
            }
            multiply_in_place<E5M2, i % 4, j % 4>(acc[i][j], fa[i % 4], fb[S][j], ea[S][i / 4], eb[S][j / 4]);
            __builtin_amdgcn_sched_barrier(0);
        });
        if constexpr (STAGES > 2) {
            under_way = cur;
            cur = next;
            next = next == (STAGES - 1) * T::kStage ? 0 : next + T::kStage;
        }
    };
    auto finish = [&](uint32_t tile) __attribute__((always_inline)) {
        uint32_t tm, tn;
        tile_of(SPLIT ? tile % whole : tile, mt, nt, tm, tn);
        const uint32_t m0 = tm * T::kM, n0 = tn * T::kN;
        const uint32_t rows = p.M - m0 < T::kM ? p.M - m0 : T::kM;
        if constexpr (SPLIT) {  // columns up to the pitch, a multiple of 4, hold zeros' sums
            const uint32_t pitch = (p.N + 3) / 4 * 4;
            const __amdgpu_buffer_rsrc_t out = __builtin_amdgcn_make_buffer_rsrc(
                (float*)p.out + ((size_t)(tile / whole) * p.M + m0) * pitch + n0, 0, (int)(4 * (rows * pitch - n0)), kRawBuffer);
            matrix_results(acc);
            sp::static_for<0, GN>([&](auto h) {
                const int c = 64 * GN * wc + 4 * lo + 64 * h;
                const int off = n0 + c < pitch ? 4 * ((64 * GM * wr + 16 * hi) * (int)pitch + c) : (int)0x80000000;
                sp::static_for<0, 16 * GM>([&](auto k) {
                    constexpr int g = k / 16, i = k / 4 % 4, r = k % 4;
                    const f32x4* v = acc[4 * g + i] + 4 * h;
                    const f32x4 four = {v[0][r], v[1][r], v[2][r], v[3][r]};
                    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, four), out, off, 4 * (64 * g + 4 * r + i) * (int)pitch, 0);
                });
            });
            return;
        }
        const __amdgpu_buffer_rsrc_t out =
            __builtin_amdgcn_make_buffer_rsrc((uint16_t*)p.out + ((size_t)m0 * p.N + n0), 0, (int)(2 * (rows * p.N - n0)), kRawBuffer);
        const int pitch = 2 * (int)p.N, col = 64 * GN * wc + 4 * lo;
        // columns behind the last: an offset beyond the resource
        auto at_column = [&](int c) __attribute__((always_inline)) {
            return n0 + c < p.N ? (64 * GM * wr + 16 * hi) * pitch + 2 * c : (int)0x80000000;
        };
        matrix_results(acc);
        sp::static_for<0, GN>([&](auto h) {
            const int off = at_column(col + 64 * h);
            const int one[3] = {at_column(col + 64 * h + 1), at_column(col + 64 * h + 2), at_column(col + 64 * h + 3)};
            sp::static_for<0, 16 * GM>([&](auto k) {
                constexpr int g = k / 16, i = k / 4 % 4, r = k % 4;
                const f32x4 *v = acc[4 * g + i] + 4 * h;
                const u32x2 two = {sp::pack_bf16(v[0][r], v[1][r]), sp::pack_bf16(v[2][r], v[3][r])};
                const int row = (64 * g + 4 * r + i) * pitch;
                if (p.N % 4 == 0) {
                    __builtin_amdgcn_raw_buffer_store_b64(two, out, off, row, 0);
                } else {  // rows begin anywhere
                    __builtin_amdgcn_raw_buffer_store_b16((uint16_t)two[0], out, off, row, 0);
                    __builtin_amdgcn_raw_buffer_store_b16((uint16_t)(two[0] >> 16), out, one[0], row, 0);
                    __builtin_amdgcn_raw_buffer_store_b16((uint16_t)two[1], out, one[1], row, 0);
                    __builtin_amdgcn_raw_buffer_store_b16((uint16_t)(two[1] >> 16), out, one[2], row, 0);
                }
            });
        });
    };

    // The copier runs STAGES blocks ahead of the products, in the tile after this one towards the end; behind the last tile it brings
    // that one again, so that every step waits for the same number.
    uint32_t tile = blockIdx.x;
    uint32_t ahead_tile = tile;  // the copier's
    int ahead = 0;               // and its block, of 2 * pairs
    auto move_on = [&]() __attribute__((always_inline)) {
        ++ahead;
        from.next(ahead < blocks);
    };
    auto to_next_tile = [&]() __attribute__((always_inline)) {
        ahead_tile = ahead_tile + gridDim.x < tiles ? ahead_tile + gridDim.x : ahead_tile;
        ahead = 0;
        go_to_tile(ahead_tile);
    };
    auto move_on_or_to_next = [&]() __attribute__((always_inline)) {
        if (ahead + 1 < 2 * pairs) move_on();
        else to_next_tile();
    };
    go_to_tile(tile);
    sp::static_for<0, STAGES - 1>([&](auto s) {
        sp::static_for<0, T::kCopies + 1>([&](auto j) { from.template copy<j>(base + s * T::kStage); });
        move_on_or_to_next();
    });
    sp::static_for<0, kEarly>([&](auto j) { from.template copy<j>(base + (STAGES - 1) * T::kStage); });
    wait_copies_and_meet<(STAGES - 2) * (T::kCopies + 1) + kEarly>();
    read_scales(sp::Int<0>{}, 0);
    sp::static_for<0, NB>([&](auto j) { read_b(sp::Int<0>{}, 0, j); });
    read_a(0, sp::Int<0>{});
    read_a(0, sp::Int<1>{});
    for (;;) {
        clear();
        for (int pair = 1; pair < pairs; ++pair) {
            if constexpr (STAGES == 2) {  // the copier is two blocks ahead: in this tile up to the last pair
                step(sp::Int<0>{}, move_on);
                step(sp::Int<1>{}, move_on);
            } else {
                step(sp::Int<0>{}, move_on_or_to_next);
                step(sp::Int<1>{}, move_on_or_to_next);
            }
        }
        if constexpr (STAGES == 2) {
            step(sp::Int<0>{}, to_next_tile);
            step(sp::Int<1>{}, move_on);
        } else {
            step(sp::Int<0>{}, move_on_or_to_next);
            step(sp::Int<1>{}, move_on_or_to_next);
        }
        finish(tile);
        tile += gridDim.x;
        if (tile >= tiles) break;
    }
    sp::wait_vmem();  // no copy is under way when the workgroup's LDS is given back
}

// out = the sums of `splits` [M][pitch] in fp32, in order, as bf16: four columns a thread
__global__ __launch_bounds__(256) void add_splits_kernel(MatmulArgs p, const float* __restrict__ sums, uint32_t splits) {
    const uint32_t pitch = (p.N + 3) / 4 * 4, at = blockIdx.x * 256 + threadIdx.x, m = at / (pitch / 4), n = (at - m * (pitch / 4)) * 4;
    if (m >= p.M) return;
    const float* from = sums + (size_t)m * pitch + n;
    f32x4 v = *reinterpret_cast<const f32x4*>(from);
#pragma unroll 4
    for (uint32_t s = 1; s < splits; ++s) v += *reinterpret_cast<const f32x4*>(from + (size_t)s * p.M * pitch);
    store4(p, m, n, u32x2{sp::pack_bf16(v[0], v[1]), sp::pack_bf16(v[2], v[3])});
}

// ------------------------------------------------------------------ few rows of a
// Workgroup (x, y) takes rows 16 MB x, ... of a and the y-th range of `groups` groups of 16 rows of b, NB at a time, and its waves share
// out the blocks: wave w takes w, w + WAVES, ..., so that the workgroup reads whole runs of b's rows and every byte of b once.  Each
// wave copies its blocks into STAGES stages of LDS of its own, as above but with row lo of a group in LDS row lo, and goes straight on to its blocks of
// the next groups: waves wait for each other only where their sums are added, in order, kPiece fragments at a time.
// b is the first operand of the products here: a lane's four results are neighbouring columns.  Those of kHeld rounds in bf16 wait in
// LDS and leave in runs of 32 kHeld NB bytes; 32 NB at a time, between the reads, they cost more than their bytes (16 x 57344 x 8192, 16 x
// 16 at a time, 104 against 93 us, without any store 86).
// One row is bound by memory: 57344 x 8192 83 us, b at 5.7 TB/s.  With more rows the copies of a come to it, of which every workgroup
// needs all: 32 x 8192 x 28672 55 us, 128 x 6144 x 4096 14, at 45 to 50 bytes a ns in each compute unit.  b straight into
// registers, a ring shared by the workgroup (waves side by side on b's rows) and a wave of its own for the results were no faster.
template <int MB, int NB, int WAVES, int STAGES, bool E5M2, bool F32>
__global__ __launch_bounds__(64 * WAVES) void matmul_few_kernel(MatmulArgs p, uint32_t groups) {
    constexpr int kCopies = 2 * (NB + MB), kStage = (NB + MB) * 2048 + 256, kPiece = NB * MB < 4 ? NB * MB : 4,
                  kHeld = NB * MB < 16 ? 16 / (NB * MB) : 1;
    static_assert((STAGES - 1) * (kCopies + 1) < 64 && NB + MB <= 16 && NB * MB % kPiece == 0, "");
    __shared__ __attribute__((aligned(1024))) uint8_t lds[WAVES * STAGES * kStage];
    __shared__ f32x4 part[WAVES][kPiece][64];
    __shared__ u32x2 held[F32 ? 1 : kHeld * NB * MB][64];
    const int lane = threadIdx.x & 63, lo = lane & 15, hi = lane >> 4;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t first = blockIdx.y * groups * 16, m0 = blockIdx.x * 16 * MB, blocks = p.K / 128;
    const uint32_t end = p.N - first < groups * 16 ? p.N : first + groups * 16;  // of the range of b's rows
    const uint32_t mine = wave < blocks ? (blocks - wave + WAVES - 1) / WAVES : 0;
    uint8_t* const ring = lds + wave * STAGES * kStage;
    const uint32_t base = sp::lds_addr(ring);

    int off[2 * (NB > MB ? NB : MB)];
#pragma unroll
    for (int d = 0; d < 2 * (NB > MB ? NB : MB); ++d) {
        const int s = 8 * d + (lane >> 3);
        off[d] = s * (int)p.K + 16 * ((lane & 7) ^ ((s >> 1) & 7));
    }
    // the copier: at block `ahead` of this wave's, of the rows of b from `ahead_n` on.  Exponents: lanes 0 .. 4 NB - 1 bring words of
    // b's, the next 4 MB of a's; the rest repeat the last.  Behind the last rows it brings zeros.
    uint32_t ahead = 0, ahead_n = first;
    int block_off;
    i32x4 a, b;
    const uint8_t* scale;
    const int w = lane < 4 * (NB + MB) ? lane : 4 * (NB + MB) - 1;
    const uint32_t pitch = w < 4 * NB ? p.b_pitch : p.a_pitch;
    auto go_to_rows = [&]() __attribute__((always_inline)) {
        a = rows_from(p.a, m0, p.M, 16 * MB, p.K);
        b = rows_from(p.b, ahead_n, end, 16 * NB, p.K);
        block_off = wave * 128;
        const uint32_t row = w < 4 * NB ? ahead_n + 4 * w : m0 + 4 * (w - 4 * NB);
        scale = (w < 4 * NB ? p.b_scale : p.a_scale) + (row < pitch ? row : 0) + (size_t)wave * pitch;
    };
    auto copy = [&](uint32_t stage) __attribute__((always_inline)) {
        sp::static_for<0, kCopies>([&](auto d) {
            if constexpr (d < 2 * NB) copy_16(stage + d * 1024, b, off[d], block_off);
            else copy_16(stage + d * 1024, a, off[d - 2 * NB], block_off);
        });
        copy_4(stage + kCopies * 1024, scale);
        if (++ahead < mine) {
            block_off += 128 * WAVES;
            scale += (size_t)pitch * WAVES;
        } else if (ahead_n + 16 * NB < end) {
            ahead = 0;
            ahead_n += 16 * NB;
            go_to_rows();
        } else {
            a[2] = b[2] = 0;
        }
    };
    const int at = lo * 128 + ((hi ^ (lo >> 1)) << 4);
    uint32_t cur = 0, rounds = 0;  // the stage to read; rounds in `held`
    if (mine > 0) {
        go_to_rows();
        for (int s = 0; s < STAGES; ++s) copy(base + s * kStage);
    }
    for (uint32_t n0 = first; n0 < end; n0 += 16 * NB) {
        f32x4 acc[NB][MB];
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int j = 0; j < MB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (uint32_t k = 0; k < mine; ++k) {
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"((STAGES - 1) * (kCopies + 1)) : "memory");
            const uint8_t* st = ring + cur * kStage;
            i32x8 fb[NB], fa[MB];
            int eb[NB], ea[MB];
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                fb[i] = fragment(st + i * 2048, at);
                eb[i] = st[kCopies * 1024 + 16 * i + lo];
            }
#pragma unroll
            for (int j = 0; j < MB; ++j) {
                fa[j] = fragment(st + (NB + j) * 2048, at);
                ea[j] = st[kCopies * 1024 + 16 * (NB + j) + lo];
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            copy(base + cur * kStage);
            if constexpr (F32) {
                sp::static_for<0, 4>([&](auto eighth) {
                    sp::bf16x8 wa[MB];
#pragma unroll
                    for (int j = 0; j < MB; ++j) wa[j] = widen<E5M2, 0, eighth>(fa[j], ea[j]);
#pragma unroll
                    for (int i = 0; i < NB; ++i) {
                        const sp::bf16x8 wb = widen<false, 0, eighth>(fb[i], eb[i]);
#pragma unroll
                        for (int j = 0; j < MB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb, wa[j], acc[i][j], 0, 0, 0);
                    }
                });
            } else {
#pragma unroll
                for (int i = 0; i < NB; ++i)
#pragma unroll
                    for (int j = 0; j < MB; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[i], fa[j], acc[i][j], 0, E5M2 ? 1 : 0, 0, eb[i], 0, ea[j]);
            }
            cur = cur + 1 == STAGES ? 0 : cur + 1;
        }
        sp::static_for<0, NB * MB / kPiece>([&](auto piece) {
            sp::static_for<0, kPiece>([&](auto f) { part[wave][f][lane] = acc[(piece * kPiece + f) / MB][(piece * kPiece + f) % MB]; });
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            for (int t = threadIdx.x; t < kPiece * 64; t += 64 * WAVES) {
                const int f = t / 64, l = t % 64, whole = piece * kPiece + f;
                f32x4 v = part[0][f][l];
#pragma unroll
                for (int x = 1; x < WAVES; ++x) v += part[x][f][l];
                if constexpr (F32) {
                    const uint32_t n = n0 + 16 * (whole / MB) + 4 * (l / 16);
                    if (n < end) store4(p, m0 + 16 * (whole % MB) + l % 16, n, v);
                } else {
                    held[rounds * NB * MB + whole][l] = u32x2{sp::pack_bf16(v[0], v[1]), sp::pack_bf16(v[2], v[3])};
                }
            }
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        });
        if constexpr (!F32) {
            if (++rounds == kHeld || n0 + 16 * NB >= end) {
                const uint32_t words = 4 * NB * rounds, from = n0 + 16 * NB - 4 * words;  // words of a row, its first column
                for (uint32_t e = threadIdx.x; e < 16 * MB * words; e += 64 * WAVES) {
                    const uint32_t row = e / words, c = e - row * words, n = from + 4 * c;
                    if (n < end) store4(p, m0 + row, n, held[c / 4 * MB + row / 16][c % 4 * 16 + row % 16]);
                }
                rounds = 0;  // the next round's are written behind its barrier
            }
        }
    }
    sp::wait_vmem();  // no copy is under way when the workgroup's LDS is given back
}

// ------------------------------------------------------------------ launches
using namespace sp::ways;

template <int WAY, bool E5M2, bool F32>
bool launch_few(const MatmulArgs& p, hipStream_t st) {
    const FewGrid g = few_grid(WAY, p.M, p.N);
    if (!sp::launchable(g.x, 64 * kFewWaves[WAY])) return false;
    hipLaunchKernelGGL((matmul_few_kernel<kFewMB[WAY], kFewNB[WAY], kFewWaves[WAY], kFewStages[WAY], E5M2, F32>), dim3((unsigned)g.x, (unsigned)g.y),
                       dim3(64 * kFewWaves[WAY]), 0, st, p, (uint32_t)g.groups);
    return true;
}
template <int WAY, bool E5M2>
bool launch_pipe(const MatmulArgs& p, hipStream_t st) {
    const int64_t mt = parts(p.M, 128 * kPipeGM[WAY]), nt = parts(p.N, 128 * kPipeGN[WAY]);
    if (mt * nt > 0x7fffffff) return false;
    hipLaunchKernelGGL((matmul_pipe_kernel<kPipeGM[WAY], kPipeGN[WAY], kPipeStages[WAY], E5M2, false>), dim3((unsigned)(mt * nt < kUnits ? mt * nt : kUnits)),
                       dim3(256), 0, st, p, (uint32_t)mt, (uint32_t)nt, 1u, 0u);
    return true;
}
template <bool E5M2>
void launch_split(MatmulArgs p, const Split& s, float* sums, hipStream_t st) {
    const uint32_t mt = (uint32_t)parts(p.M, 128), nt = (uint32_t)parts(p.N, 128), tiles = mt * nt * (uint32_t)s.splits;
    void* const out = p.out;
    p.out = sums;
    hipLaunchKernelGGL((matmul_pipe_kernel<1, 1, kPipeStages[0], E5M2, true>), dim3(tiles < kUnits ? tiles : (unsigned)kUnits), dim3(256), 0, st, p, mt, nt,
                       (uint32_t)s.splits, (uint32_t)s.per);
    p.out = out;
    hipLaunchKernelGGL(add_splits_kernel, dim3((unsigned)parts((int64_t)p.M * ((p.N + 3) / 4), 256)), dim3(256), 0, st, p, sums, (uint32_t)s.splits);
}
template <bool E5M2, bool F32>
bool launch_way(int way, const MatmulArgs& p, hipStream_t st) {
    if (way == 0) return launch_few<0, E5M2, F32>(p, st);
    if (way == 1) return launch_few<1, E5M2, F32>(p, st);
    if (way == 2) return launch_few<2, E5M2, F32>(p, st);
    if (way == 3) return launch_few<3, E5M2, F32>(p, st);
    if (way == 4) return launch_few<4, E5M2, F32>(p, st);
    if (way == 5) return launch_few<5, E5M2, F32>(p, st);
    if constexpr (F32) {
        const int64_t mt = parts(p.M, 128), nt = parts(p.N, 128);
        if (!sp::launchable(mt * nt, 256)) return false;
        hipLaunchKernelGGL((matmul_f32_kernel<E5M2>), dim3((unsigned)(mt * nt)), dim3(256), 0, st, p, (uint32_t)mt, (uint32_t)nt);
        return true;
    } else {
        if (way == kFew) return launch_pipe<0, E5M2>(p, st);
        if (way == kFew + 1) return launch_pipe<1, E5M2>(p, st);
        return launch_pipe<2, E5M2>(p, st);
    }
}

}  // namespace

namespace sp {

size_t fp8_matmul_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    const Split s = which_split(M, N, K);
    return s.splits > 1 ? (size_t)s.splits * (size_t)M * (size_t)((N + 3) / 4 * 4) * sizeof(float) : 0;
}

sp_status launch_fp8_matmul_split(const void* a, const void* a_scale, const void* b, const void* b_scale, void* out, float* sums,
                                  int64_t M, int64_t N, int64_t K, bool a_e5m2, hipStream_t st) {
    const Split s = which_split(M, N, K);
    if (s.splits <= 1) return launch_fp8_matmul(a, a_scale, b, b_scale, out, M, N, K, a_e5m2, false, false, st);
    const MatmulArgs p{(const uint8_t*)a, (const uint8_t*)a_scale, (const uint8_t*)b, (const uint8_t*)b_scale, out,
                       (uint32_t)M, (uint32_t)N, (uint32_t)K, (uint32_t)((M + 15) / 16 * 16), (uint32_t)((N + 15) / 16 * 16), false};
    if (a_e5m2) launch_split<true>(p, s, sums, st);
    else launch_split<false>(p, s, sums, st);
    return launch_status();
}

sp_status launch_fp8_matmul(const void* a, const void* a_scale, const void* b, const void* b_scale, void* out, int64_t M, int64_t N,
                            int64_t K, bool a_e5m2, bool f32, bool accumulate, hipStream_t st) {
    const MatmulArgs p{(const uint8_t*)a, (const uint8_t*)a_scale, (const uint8_t*)b, (const uint8_t*)b_scale, out,
                       (uint32_t)M, (uint32_t)N, (uint32_t)K, (uint32_t)((M + 15) / 16 * 16), (uint32_t)((N + 15) / 16 * 16), accumulate};
    const int way = which_way(M, N, K, f32);
    if (K == 0) {  // nothing is read: nothing is added, or zeros by as many launches as the rows need
        if (accumulate) return SP_OK;
        constexpr int64_t kMost = (int64_t)1 << 26;
        bool fits = true;
        for (int64_t m = 0; m < M && fits; m += kMost) {
            MatmulArgs part = p;
            part.out = (char*)out + (size_t)m * (size_t)N * (f32 ? 4 : 2);
            part.M = (uint32_t)(M - m < kMost ? M - m : kMost);
            fits = f32 ? launch_way<false, true>(way, part, st) : launch_way<false, false>(way, part, st);
        }
        return fits ? launch_status() : SP_ERR_SHAPE;
    }
    const bool fits = a_e5m2 ? (f32 ? launch_way<true, true>(way, p, st) : launch_way<true, false>(way, p, st))
                             : (f32 ? launch_way<false, true>(way, p, st) : launch_way<false, false>(way, p, st));
    return fits ? launch_status() : SP_ERR_SHAPE;
}

}  // namespace sp
