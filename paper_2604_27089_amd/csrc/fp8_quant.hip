// Operands of the block-scaled 8-bit products: the residual RMS norm whose output leaves in 8 bits, and the conversion of a
// bf16 tensor by rows, by columns or both.  Everything streams: each element is read once, each result written once.
#include "fp8_common.h"
#include "sp_common.h"

namespace {

using namespace sp::stream;
using namespace sp::fp8;
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Largest finite magnitude of eight values; those that are not finite become quiet NaN.
__device__ __forceinline__ uint32_t largest_finite(float (&f)[8]) {
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t m = magnitude(f[e]);
        if (m < kInf) most = umax(most, m);
        else f[e] = __builtin_nanf("");
    }
    return most;
}

// bf16(a + b)
__device__ __forceinline__ u32x4 add8(const u32x4& a, const u32x4& b) {
    float f[8], g[8];
    widen(a, f);
    widen(b, g);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] += g[e];
    return narrow(f);
}
__device__ __forceinline__ float squares(const u32x4& x) {
    float f[8], s = 0.f;
    widen(x, f);
#pragma unroll
    for (int e = 0; e < 8; ++e) s += f[e] * f[e];
    return s;
}
// x * r * w (zeros where not `in`) as e4m3, with the exponent of the block that the 16 neighbouring lanes hold
__device__ __forceinline__ uint32_t convert8(const u32x4& x, const u32x4& w, float r, bool in, u32x2& bytes) {
    float f[8], g[8];
    widen(x, f);
    widen(w, g);
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        f[e] = in ? f[e] * r * g[e] : 0.f;
        most = umax(most, magnitude(f[e]));
    }
    if (__any(most >= kInf)) most = largest_finite(f);
    const uint32_t ex = scale_exponent<false>(max_of_16(most));
    bytes = u32x2{pack4<false>(f[0], f[1], f[2], f[3], ex), pack4<false>(f[4], f[5], f[6], f[7], ex)};
    return ex;
}

// ------------------------------------------------------------------ residual RMS norm, forward
//   h = bf16(x + res),  rstd = 1/sqrt(mean_c h^2 + eps),  y = h * rstd * w in fp32,  (q, scale) = y in blocks of 128 columns
// A workgroup per row, which stays in registers between the sum of squares and the conversion: thread t owns the 8-column vectors
// number t, t + THREADS, ... (NVT of them), so a block is 16 neighbouring lanes, and the sum goes over the waves through LDS.  h may be x
// or res: a thread reads a vector before it writes it, and no other thread uses it (those behind the row's end read the last vector, maybe
// after that write, and drop it).
// A wave per row took longer throughout (one row of 4096 5.7 against 3.5 us, 1031 x 5120 10.4 / 5.9, 16384 x 4096 86.7 / 82.4): a row's
// loads are four times as deep then, and few rows leave most of the chip idle.  16384 x 4096: 470 MB at 6.0 TB/s (79 us).
// Rows lie over two dimensions of the grid, kRowsX in the first: a launch has less than 2^32 threads in a dimension.
constexpr int64_t kRowsX = (int64_t)1 << 22;
template <int NVT, int THREADS, bool RES>
__global__ __launch_bounds__(THREADS) void rmsnorm_fp8_kernel(const __bf16* x, const __bf16* res, const __bf16* __restrict__ w,
                                                             __bf16* h, uint8_t* __restrict__ q, uint8_t* __restrict__ q_scale,
                                                             float* __restrict__ rstd, int64_t T, int32_t C, int64_t scale_pitch,
                                                             float eps) {
    __shared__ float sums[THREADS / 64];
    const int64_t row = blockIdx.x + blockIdx.y * kRowsX;
    const int32_t Cp = (C + kBlock - 1) / kBlock * kBlock;
    if (row >= T) {  // entries behind the last row, up to a multiple of 16
        if (row < scale_pitch)
            for (int b = threadIdx.x; b < Cp / kBlock; b += THREADS) q_scale[b * scale_pitch + row] = 1;
        return;
    }
    u32x4 xv[NVT], wv[NVT];
#pragma unroll
    for (int j = 0; j < NVT; ++j) {
        const int c0 = (j * THREADS + (int)threadIdx.x) * 8, at = c0 < C ? c0 : C - 8;
        xv[j] = ld16(x + row * C + at);
        wv[j] = *reinterpret_cast<const u32x4*>(w + at);
    }
    if constexpr (RES) {
        u32x4 rv[NVT];
#pragma unroll
        for (int j = 0; j < NVT; ++j) {
            const int c0 = (j * THREADS + (int)threadIdx.x) * 8;
            rv[j] = ld16(res + row * C + (c0 < C ? c0 : C - 8));
        }
#pragma unroll
        for (int j = 0; j < NVT; ++j) {
            const int c0 = (j * THREADS + (int)threadIdx.x) * 8;
            xv[j] = add8(xv[j], rv[j]);
            if (c0 < C) st16(h + row * C + c0, xv[j]);
        }
    }
    float ss = 0.f;
#pragma unroll
    for (int j = 0; j < NVT; ++j) ss += (j * THREADS + (int)threadIdx.x) * 8 < C ? squares(xv[j]) : 0.f;
    ss = wave_sum(ss);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = ss;
    __syncthreads();
    ss = sums[0];
#pragma unroll
    for (int i = 1; i < THREADS / 64; ++i) ss += sums[i];
    const float r = 1.0f / sqrtf(ss / (float)C + eps);
    if (threadIdx.x == 0) rstd[row] = r;
#pragma unroll
    for (int j = 0; j < NVT; ++j) {
        const int c0 = (j * THREADS + (int)threadIdx.x) * 8;
        u32x2 bytes;
        const uint32_t ex = convert8(xv[j], wv[j], r, c0 < C, bytes);
        if (c0 < Cp) {
            __builtin_nontemporal_store(bytes, reinterpret_cast<u32x2*>(q + row * Cp + c0));
            if ((threadIdx.x & 15) == 0) q_scale[c0 / kBlock * scale_pitch + row] = (uint8_t)ex;
        }
    }
}

// ------------------------------------------------------------------ conversion by rows and by columns
// A workgroup takes a tile of 128 rows by 128 columns: a block of the row side for each row, one of the column side for each
// column.  Thread (rg, cv) owns rows 8 rg .. 8 rg + 7 of the 8-column vector cv and keeps them in registers for both sides.
//   rows: the 16 threads of a row are neighbouring lanes; 8 bytes per thread and row.
//   columns: the largest magnitude of a column goes over the four rg of a wave by lane exchange and over the four waves through
//     LDS; the bytes are transposed through LDS, 8 at a time since a thread's rows are consecutive, and leave 128 bytes a column.
// bf16 is compared two at a time and converted as it is, about three vector instructions per element for both sides (fourteen when
// every element went through fp32: 210 us on 16384 x 14336 both ways).  With rstd and w given, the element is x * rstd * w in fp32,
// the norm's output in the forward's own order of operations.
// Elements that are not finite are looked for once per thread and made quiet NaN with no magnitude.
template <bool ROWS, bool COLS, bool NORM, bool E5M2>
__global__ __launch_bounds__(256) void quant_kernel(const __bf16* __restrict__ x, const float* __restrict__ rstd,
                                                   const __bf16* __restrict__ w, uint8_t* __restrict__ q,
                                                   uint8_t* __restrict__ q_scale, uint8_t* __restrict__ qt,
                                                   uint8_t* __restrict__ qt_scale, int64_t T, int32_t C, int64_t q_pitch,
                                                   int64_t t_pitch, int32_t col_blocks) {
    __shared__ __attribute__((aligned(16))) uint32_t part[4][kBlock];  // largest magnitudes of the columns, by wave (fp32 bits)
    __shared__ __attribute__((aligned(16))) uint8_t tile[COLS ? kBlock * kBlock : 16];
    const int tid = threadIdx.x, cv = tid & 15, rg = tid >> 4, wave = tid >> 6;
    // Order of the tiles: by rows alone along the rows; otherwise down bands of kBand tiles, so that what is written of a column at a
    // time lies together.  16384 x 14336, columns alone 164 us along the rows, 132 in bands of 32; both sides 193 and 184; rows alone
    // 123 and 133.
    constexpr uint32_t kBand = COLS ? 32 : 1;
    const uint32_t row_blocks = (uint32_t)((T + kBlock - 1) / kBlock), band = blockIdx.x / (kBand * col_blocks);
    const uint32_t in = blockIdx.x - band * kBand * col_blocks, height = row_blocks - band * kBand < kBand ? row_blocks - band * kBand : kBand;
    const int32_t cb = (int32_t)(in / height);
    const int64_t tb = band * kBand + (in - cb * height);
    const int64_t t0 = tb * kBlock + rg * 8;
    const int32_t c0 = cb * kBlock + cv * 8;
    const int32_t Cp = col_blocks * kBlock;
    u32x4 xv[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int64_t t = t0 + j < T ? t0 + j : T - 1;
        xv[j] = ld16(x + t * C + (c0 < C ? c0 : C - 8));
    }
    if (t0 + 8 > T || c0 >= C) {  // beyond the edges come zeros
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (t0 + j >= T || c0 >= C) xv[j] = u32x4{0, 0, 0, 0};
    }
    float v[NORM ? 8 : 1][8];
    uint32_t row_most[8], col_most[8];  // fp32 bits
    if constexpr (NORM) {
        float wf[8];
        widen(*reinterpret_cast<const u32x4*>(w + (c0 < C ? c0 : C - 8)), wf);
        float row[8], col[8], all = 0.f;  // a maximum passes over NaN, which needs no more care: it stays NaN
#pragma unroll
        for (int e = 0; e < 8; ++e) col[e] = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float r = rstd[t0 + j < T ? t0 + j : T - 1];
            const bool inside = t0 + j < T && c0 < C;
            widen(xv[j], v[j]);
            row[j] = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[j][e] = inside ? v[j][e] * r * wf[e] : 0.f;  // a zero of x against a rstd that is not finite
                if constexpr (ROWS) row[j] = fmaxf(row[j], fabsf(v[j][e]));
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
#pragma unroll
            for (int j = 0; j < 8; ++j) col[e] = fmaxf(col[e], fabsf(v[j][e]));
            all = fmaxf(all, col[e]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            row_most[e] = ROWS ? magnitude(row[e]) : 0u;
            col_most[e] = magnitude(col[e]);
        }
        if (__any(magnitude(all) >= kInf)) {
#pragma unroll
            for (int e = 0; e < 8; ++e) col_most[e] = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                row_most[j] = largest_finite(v[j]);
#pragma unroll
                for (int e = 0; e < 8; ++e) col_most[e] = umax(col_most[e], magnitude(v[j][e]) < kInf ? magnitude(v[j][e]) : 0u);
            }
        }
    } else {
        u16x2 rows2[8], cols2[4];
        auto compare = [&](auto mag) __attribute__((always_inline)) {
#pragma unroll
            for (int d = 0; d < 4; ++d) cols2[d] = mag(xv[0][d]);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const u16x2 m[4] = {mag(xv[j][0]), mag(xv[j][1]), mag(xv[j][2]), mag(xv[j][3])};
                rows2[j] = max2(max2(m[0], m[1]), max2(m[2], m[3]));
#pragma unroll
                for (int d = 0; d < 4; ++d) cols2[d] = max2(cols2[d], m[d]);
            }
        };
        compare([](uint32_t word) __attribute__((always_inline)) { return magnitude2(word); });
        const u16x2 all = max2(max2(cols2[0], cols2[1]), max2(cols2[2], cols2[3]));
        if (__any(all[0] >= kInf >> 16 || all[1] >= kInf >> 16)) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    const u16x2 m = magnitude2(xv[j][d]);
                    if (m[0] >= kInf >> 16) xv[j][d] = (xv[j][d] & 0xffff0000u) | 0x7fc0u;
                    if (m[1] >= kInf >> 16) xv[j][d] = (xv[j][d] & 0xffffu) | 0x7fc00000u;
                }
            compare([](uint32_t word) __attribute__((always_inline)) {
                u16x2 m = magnitude2(word);
                m[0] = m[0] < kInf >> 16 ? m[0] : 0;
                m[1] = m[1] < kInf >> 16 ? m[1] : 0;
                return m;
            });
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) row_most[j] = (uint32_t)(rows2[j][0] > rows2[j][1] ? rows2[j][0] : rows2[j][1]) << 16;
#pragma unroll
        for (int e = 0; e < 8; ++e) col_most[e] = (uint32_t)cols2[e / 2][e % 2] << 16;
    }
    if constexpr (ROWS) {
        uint32_t row_exp[2] = {0, 0};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t ex = scale_exponent<E5M2>(max_of_16(row_most[j]));
            row_exp[j / 4] |= ex << (8 * (j % 4));
            u32x2 bytes;
            if constexpr (NORM) bytes = u32x2{pack4<E5M2>(v[j][0], v[j][1], v[j][2], v[j][3], ex), pack4<E5M2>(v[j][4], v[j][5], v[j][6], v[j][7], ex)};
            else bytes = u32x2{pack4<E5M2>(xv[j][0], xv[j][1], ex), pack4<E5M2>(xv[j][2], xv[j][3], ex)};
            if (t0 + j < T) __builtin_nontemporal_store(bytes, reinterpret_cast<u32x2*>(q + (t0 + j) * Cp + c0));
        }
        if (cv == 0 && t0 < q_pitch) *reinterpret_cast<uint2*>(q_scale + cb * q_pitch + t0) = uint2{row_exp[0], row_exp[1]};
    }
    if constexpr (COLS) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            col_most[e] = umax(col_most[e], __shfl_xor(col_most[e], 16, 64));
            col_most[e] = umax(col_most[e], __shfl_xor(col_most[e], 32, 64));
        }
        if ((tid & 63) < 16) {
            *reinterpret_cast<u32x4*>(&part[wave][cv * 8]) = u32x4{col_most[0], col_most[1], col_most[2], col_most[3]};
            *reinterpret_cast<u32x4*>(&part[wave][cv * 8 + 4]) = u32x4{col_most[4], col_most[5], col_most[6], col_most[7]};
        }
        __syncthreads();
        uint32_t col_exp[2] = {0, 0};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int c = cv * 8 + e;
            const uint32_t ex = scale_exponent<E5M2>(umax(umax(part[0][c], part[1][c]), umax(part[2][c], part[3][c])));
            col_exp[e / 4] |= ex << (8 * (e % 4));
            uint2 bytes;
            if constexpr (NORM) {
                bytes = uint2{pack4<E5M2>(v[0][e], v[1][e], v[2][e], v[3][e], ex), pack4<E5M2>(v[4][e], v[5][e], v[6][e], v[7][e], ex)};
            } else {  // the column's halves of two rows' words, side by side
                uint32_t two[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) two[j] = __builtin_amdgcn_perm(xv[2 * j + 1][e / 2], xv[2 * j][e / 2], e % 2 ? 0x07060302u : 0x05040100u);
                bytes = uint2{pack4<E5M2>(two[0], two[1], ex), pack4<E5M2>(two[2], two[3], ex)};
            }
            // 16-byte chunk rg/2 of column c lies at chunk position (rg/2) ^ (cv % 8), so that the 16 columns that a store
            // instruction writes fall on different banks
            *reinterpret_cast<uint2*>(tile + c * kBlock + ((rg / 2) ^ (cv & 7)) * 16 + (rg & 1) * 8) = bytes;
        }
        if (rg == 0 && c0 < t_pitch) *reinterpret_cast<uint2*>(qt_scale + tb * t_pitch + c0) = uint2{col_exp[0], col_exp[1]};
        __syncthreads();
        const int64_t Tp = (T + kBlock - 1) / kBlock * kBlock;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = (tid + 256 * i) / 8, chunk = tid & 7;
            if (cb * kBlock + c < C)
                st16(qt + (int64_t)(cb * kBlock + c) * Tp + tb * kBlock + chunk * 16, *reinterpret_cast<const u32x4*>(tile + c * kBlock + (chunk ^ (c / 8 & 7)) * 16));
        }
    }
}

inline int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

}  // namespace

namespace sp {

sp_status launch_rmsnorm_fp8_fwd(const void* x, const void* res, const void* w, void* h, void* q, void* q_scale, float* rstd,
                                 int64_t T, int32_t C, float eps, hipStream_t st) {
    const int64_t pitch = up(T, 16);
    const int vectors = (int)(up(C, kBlock) / 8);
    const dim3 grid((unsigned)(pitch < kRowsX ? pitch : kRowsX), (unsigned)((pitch + kRowsX - 1) / kRowsX));
#define SP_NORM_(NVT, N, RES) hipLaunchKernelGGL((rmsnorm_fp8_kernel<NVT, N, RES>), grid, dim3(N), 0, st, (const __bf16*)x, (const __bf16*)res, (const __bf16*)w, (__bf16*)h, (uint8_t*)q, (uint8_t*)q_scale, rstd, T, C, pitch, eps)
#define SP_NORM(NVT, N) do { if (res) SP_NORM_(NVT, N, true); else SP_NORM_(NVT, N, false); } while (0)
    // two vectors per thread at most: 16384 x 8192 with 512 threads 163 us, with 256 164 (64 x 8192 4.3 / 4.8); 16384 x 4096 with 256 82,
    // with 512 83, with 128 84.  No more waves than the row fills: 16384 x 5120 without a residual with 320 threads 50, with 512 56;
    // 1031 x 5120 5.9 / 6.7, where 512 leave 1024 rows at a time
    if (vectors <= 256) SP_NORM(1, 256); else if (vectors <= 512) SP_NORM(2, 256); else if (vectors <= 640) SP_NORM(2, 320);
    else if (vectors <= 768) SP_NORM(2, 384); else if (vectors <= 896) SP_NORM(2, 448); else SP_NORM(2, 512);
#undef SP_NORM
#undef SP_NORM_
    return launch_status();
}

sp_status launch_fp8_quant(const void* x, const float* rstd, const void* w, void* q, void* q_scale, void* qt, void* qt_scale,
                           int64_t T, int32_t C, bool e5m2, hipStream_t st) {
    const int64_t cbs = up(C, kBlock) / kBlock, tiles = cbs * (up(T, kBlock) / kBlock);
    if (!launchable(tiles, 256)) return SP_ERR_SHAPE;
    const dim3 grid((unsigned)tiles), block(256);
#define SP_QUANT_(R, CO, N, E) hipLaunchKernelGGL((quant_kernel<R, CO, N, E>), grid, block, 0, st, (const __bf16*)x, rstd, (const __bf16*)w, (uint8_t*)q, (uint8_t*)q_scale, (uint8_t*)qt, (uint8_t*)qt_scale, T, C, up(T, 16), up(C, 16), (int32_t)cbs)
#define SP_QUANT(R, CO) do { if (w) { if (e5m2) SP_QUANT_(R, CO, true, true); else SP_QUANT_(R, CO, true, false); } \
                             else { if (e5m2) SP_QUANT_(R, CO, false, true); else SP_QUANT_(R, CO, false, false); } } while (0)
    if (q && qt) SP_QUANT(true, true); else if (q) SP_QUANT(true, false); else SP_QUANT(false, true);
#undef SP_QUANT
#undef SP_QUANT_
    return launch_status();
}

}  // namespace sp
