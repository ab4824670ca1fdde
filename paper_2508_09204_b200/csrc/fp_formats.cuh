// Floating-point experts: microscaled 4-bit formats (MXFP4, NVFP4) and plain bf16.
//
// A 4-bit number is e2m1 (0, .5, 1, 1.5, 2, 3, 4, 6 and a sign bit); 32 (MXFP4) or 16 (NVFP4) consecutive k share a scale, a
// power of two (E8M0) or an e4m3 number; an NVFP4 row has an fp32 scale of its own on top.  See moqe.h for the arithmetic.
//
// Every rounding here is that of an exact real quotient.  MXFP4 divides by a power of two.  NVFP4 divides by an e4m3 number.  For a
// source of bf16 a quotient that is not half way between two numbers is at least 2^-9 of its size away from there: a product with a
// reciprocal that is a little too large, cut to 12 bits, is the half way mark where the quotient is, and on the quotient's side of it
// elsewhere.  For fp32 the nearest quotient beside a mark is more than half a unit of the mark's last place away from it, so that a
// correctly rounded one would never meet a mark wrongly; the one worked out here is a unit off at most, but not shown to be correctly
// rounded, so that on a mark the sign of the remainder decides (nv_quotient).
//
// Packed layout, the same for experts and for a call's token rows: k-blocks of 128 bytes a row (256 codes or 64 bf16), in which a
// row's eight 16-byte chunks are permuted by the 128-byte swizzle (chunk c of row r at place c ^ (r & 7)), eight rows to 1024
// bytes: what the tensor cores read K-major, so that a bulk copy without a tensor map brings an operand tile.  Scales stand in
// the order that tensor memory wants, 512 bytes for 128 rows x 4 scales: row r, scale j at (r % 32) * 16 + (r / 32) * 4 + j.
//   expert : tile (nt, kb) = 128 channels: 16 KB codes, then their scales (MXFP4 1 KB, NVFP4 2 KB); tiles ordered [nt][kb],
//            one bulk copy each.  Then NVFP4's channel scales, fp32 [Np].  Rows and k behind the matrix are zeros.
//   tokens : the rows of an expert start at a multiple of 16 rows (`pad0`); codes [kb][row / 8][1024 bytes], so that the
//            rows of any tile are one piece; scales [kb][tile][one or two blocks of 1 or 2 KB]; row scales fp32.
#pragma once
#include "common.cuh"

struct moqe_fp_expert {
    int N, K, format;             // as given by the caller
    int Np, KB;                   // channels padded to 128; k-blocks
    int device;
    bool pooled;
    uint8_t* tiles;
    float* outer;                 // NVFP4: [Np], behind the tiles
    size_t tiles_alloc, outer_alloc;
};

namespace moqe {

constexpr int FP_MAX_K = 1 << 24, FP_MAX_N = 1 << 30;      // (indices within a row and numbers of rows are 32-bit)
__host__ __device__ inline int fp_block(int format) { return format == MOQE_FP_MXFP4 ? 32 : 16; }       // k that share a scale
__host__ __device__ inline int fp_kbk(int format) { return format == MOQE_FP_BF16 ? 64 : 256; }         // k of a k-block
__host__ __device__ inline int fp_sf_bytes(int format) { return format == MOQE_FP_MXFP4 ? 1024 : format == MOQE_FP_NVFP4 ? 2048 : 0; }   // scales of 128 rows, a k-block
__host__ __device__ inline int fp_tile_stride(int format) { return 16384 + fp_sf_bytes(format); }
__host__ __device__ inline int fp_kblocks(int K, int format) { const int b = fp_kbk(format); return (K + b - 1) / b; }

// Where one row of a packed matrix lies.
struct PackedRow {
    uint8_t* codes; size_t codes_kb;      // first k-block's 128 bytes of the row; from k-block to k-block
    uint8_t* sf; size_t sf_kb;            // first scale of the row; from k-block to k-block
    int r7;                               // row % 8
    __device__ __forceinline__ uint8_t* chunk(int kb, int c) const { return codes + kb * codes_kb + ((c ^ r7) << 4); }
    __device__ __forceinline__ uint8_t* scale(int kb, int b) const { return sf + kb * sf_kb + ((b >> 2) << 9) + (b & 3); }
};
__device__ __forceinline__ PackedRow expert_row(uint8_t* tiles, int KB, int format, int n) {
    const int stride = fp_tile_stride(format), r = n & 127;
    uint8_t* t = tiles + (size_t)(n >> 7) * KB * stride;
    return {t + (r >> 3) * 1024 + (r & 7) * 128, (size_t)stride, t + 16384 + (r & 31) * 16 + (r >> 5) * 4, (size_t)stride, r & 7};
}
__device__ __forceinline__ float rcp_approx(float s) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s)); return r; }
// a / b for 0 <= a, 0 < b (a 32-bit division takes far longer; the quotient is a few units off at most)
__device__ __forceinline__ int div_small(int a, int b) {
    int q = (int)((float)a * rcp_approx((float)b));
    while ((q + 1) * b <= a) ++q;
    while (q * b > a) --q;
    return q;
}
// The token tiles of an expert's n rows: as few as TN tokens allow, of equal size (a multiple of 16), because a tile of 16 tokens costs
// two thirds of one of 256.
struct TokenTiles { int tiles, rows; };
__device__ __forceinline__ TokenTiles token_tiles(int n, int TN) {
    const int t = (n + TN - 1) >> (31 - __clz(TN));       // (TN: a power of two)
    return {t, t > 1 ? (div_small(n + t - 1, t) + 15) & ~15 : TN};
}
// row i of a segment of `pad` rows; scales in blocks of 128 rows, as many to a tile as TN tokens need
__device__ __forceinline__ PackedRow token_row(uint8_t* codes, uint8_t* sf, int format, int i, int pad, const TokenTiles& t, int TN) {
    const int sfb = fp_sf_bytes(format), bpt = TN > 128 ? 2 : 1, tile = t.tiles > 1 ? div_small(i, t.rows) : 0, in = i - tile * t.rows, r = in & 127;
    return {codes + (size_t)(i >> 3) * 1024 + (i & 7) * 128, (size_t)pad * 128,
            sf + (size_t)(tile * bpt + (in >> 7)) * sfb + (r & 31) * 16 + (r >> 5) * 4, (size_t)(t.tiles * bpt) * sfb, i & 7};
}

__device__ __forceinline__ float pow2_field(int field) { return __int_as_float(field << 23); }   // 2^(field - 127), 1 <= field <= 254
__device__ __forceinline__ float e8m0_value(uint32_t b) { return b == 0 ? __int_as_float(0x00400000) : b == 255 ? __int_as_float(0x7FC00000) : pow2_field((int)b); }
__device__ __forceinline__ float e4m3_value(uint32_t b) {       // 0 <= b <= 127
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)b));
    return __low2float(*reinterpret_cast<const __half2*>(&h));
}

// eight e2m1 codes, the first in the lowest nibble; to nearest, ties to the even code, beyond 6 to 6
__device__ __forceinline__ uint32_t e2m1_x8(const float* v) {
    uint32_t d;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(d) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return d;
}
// what eight codes stand for
__device__ __forceinline__ void e2m1_values(uint32_t codes, float (&v)[8]) {
    uint32_t h[4];
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\tcvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(codes));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
        v[2 * i] = f.x; v[2 * i + 1] = f.y;
    }
}
// a * b to odd: of the two fp32 numbers around a product that fp32 does not hold, the one whose last bit is set.  Rounded to bf16 after
// that it is the product rounded once (an fp32 nearest to it can be half way between two bf16 numbers where the product is not).
__device__ __forceinline__ float mul_to_odd(float a, float b) {
    const float below = __fmul_rd(a, b), above = __fmul_ru(a, b);
    return __float_as_uint(below) & 1u ? below : above;
}
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// nearest e4m3 number's byte, 0 <= v <= 448
__device__ __forceinline__ uint32_t e4m3_byte(float v) {
    uint16_t d;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(d) : "f"(0.f), "f"(v));
    return d & 0xFFu;
}

// y / s for s > 0, one of the two fp32 numbers around it, and itself where that is one; 1 / s to an unit or two of the last place in rs
// (one step of Markstein's correction).  fp32 sources: moved off a border by a unit of the last place where it is not there exactly,
// as the remainder's sign says.
template <bool FP32>
__device__ __forceinline__ float nv_quotient(float y, float s, float rs) {
    const float q0 = y * rs;
    const float q = __fmaf_rn(__fmaf_rn(-q0, s, y), rs, q0);
    if constexpr (FP32) {
        const float rem = __fmaf_rn(-q, s, y);
        const int bits = __float_as_int(q);
        if ((bits & 0xFFFFF) == 0 && rem != 0.f) return __int_as_float(bits + (rem > 0.f ? 1 : -1));
    }
    return q;
}

// Scale and codes of 16 consecutive k of a row.  `amax`: the largest magnitude of the numbers that share the scale (a NaN if there is
// one among them); `row_field`: NVFP4's row scale is 2^(row_field - 127).  -> the scale's byte; the codes, the first in the lowest nibble.
template <int FORMAT, bool FP32>
__device__ __forceinline__ uint32_t encode16(const float (&x)[16], float amax, int row_field, uint32_t (&codes)[2]) {
    const uint32_t top = __float_as_uint(amax);
    if (top >= 0x7F800000u) {                               // an infinity or a NaN: the block is a NaN
        codes[0] = codes[1] = 0;
        return FORMAT == MOQE_FP_MXFP4 ? 255u : 127u;
    }
    float q[16];
    uint32_t byte;
    if constexpr (FORMAT == MOQE_FP_MXFP4) {
        byte = (uint32_t)max((int)(top >> 23) - 2, 0);
        const float inv = pow2_field(254 - (int)byte);
#pragma unroll
        for (int i = 0; i < 16; ++i) q[i] = x[i] * inv;
    } else {
        const float inv = pow2_field(254 - row_field);
        byte = e4m3_byte(nv_quotient<false>(amax * inv, 6.0f, 1.0f / 6.0f));
        const float s = e4m3_value(byte);
        const float rs = byte ? rcp_approx(s) : 0.f;
        if constexpr (FP32) {
#pragma unroll
            for (int i = 0; i < 16; ++i) q[i] = copysignf(nv_quotient<true>(fabsf(x[i]) * inv, s, rs), x[i]);
        } else {
            float k = rs * 0x1.000008p0f * inv;                 // (a factor of 1 + 2^-21)
#pragma unroll
            for (int i = 0; i < 16; ++i) q[i] = x[i];
            if (row_field < 32) {                               // (a row of tiny numbers, for which k could be infinite)
                k = rs * 0x1.000008p0f * pow2_field(190 - row_field);
#pragma unroll
                for (int i = 0; i < 16; ++i) q[i] *= 0x1p64f;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) q[i] = __uint_as_float(__float_as_uint(q[i] * k) & 0xFFFFF000u);
        }
    }
    codes[0] = e2m1_x8(q);
    codes[1] = e2m1_x8(q + 8);
    return byte;
}
// NVFP4: the row scale's exponent field for the bits of the row's largest finite magnitude
__device__ __forceinline__ int nv_row_field(uint32_t amax) { return amax == 0 ? 127 : max((int)(amax >> 23) - 10, 1); }

// Rows are taken in chunks of 16 consecutive k, neighbouring lanes neighbouring chunks; two lanes agree on a scale of MXFP4.  (With
// eight to a chunk the shared work of a block, its scale and the addresses, made 16384 x 11008 take 161 instead of 130 us.)  A thread
// holds CHUNKS of them, all loaded before the first is used: two where rows are few and a row's latency counts, more where there
// are many, so that what a block does once for a row weighs less.
struct Raw32 { uint32_t w[8]; };
// 32 bytes, of which `have` (0, 16 or all) are read; `wide`: from a 32-byte boundary
__device__ __forceinline__ void load32(const void* p, int have, bool wide, Raw32& r) {
    if (wide && have >= 32) {
        asm volatile("ld.global.nc.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]), "=r"(r.w[4]), "=r"(r.w[5]), "=r"(r.w[6]), "=r"(r.w[7]) : "l"(p));
        return;
    }
    const uint4 z = make_uint4(0, 0, 0, 0), *q = reinterpret_cast<const uint4*>(p);
    const uint4 a = have > 0 ? __ldg(q) : z, b = have > 16 ? __ldg(q + 1) : z;
    r.w[0] = a.x; r.w[1] = a.y; r.w[2] = a.z; r.w[3] = a.w; r.w[4] = b.x; r.w[5] = b.y; r.w[6] = b.z; r.w[7] = b.w;
}
__device__ __forceinline__ void store32(void* p, int have, bool wide, const Raw32& r) {
    if (wide && have >= 32) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                     ::"l"(p), "r"(r.w[0]), "r"(r.w[1]), "r"(r.w[2]), "r"(r.w[3]), "r"(r.w[4]), "r"(r.w[5]), "r"(r.w[6]), "r"(r.w[7]) : "memory");
        return;
    }
    uint4* q = reinterpret_cast<uint4*>(p);
    if (have > 0) q[0] = make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]);
    if (have > 16) q[1] = make_uint4(r.w[4], r.w[5], r.w[6], r.w[7]);
}
// 16 numbers of a row, zeros behind its end (K is a multiple of 8)
struct RawBf16 { Raw32 r; };
struct RawF32 { Raw32 a, b; };
__device__ __forceinline__ void load16(const __nv_bfloat16* row, int k, int K, bool wide, RawBf16& raw) { load32(row + k, (K - k) * 2, wide, raw.r); }
__device__ __forceinline__ void load16(const float* row, int k, int K, bool wide, RawF32& raw) {
    load32(row + k, (K - k) * 4, wide, raw.a);
    load32(row + k + 8, (K - k - 8) * 4, wide, raw.b);
}
__device__ __forceinline__ void widen(const RawBf16& raw, float (&x)[16]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) { x[2 * i] = __uint_as_float(raw.r.w[i] << 16); x[2 * i + 1] = __uint_as_float(raw.r.w[i] & 0xFFFF0000u); }
}
__device__ __forceinline__ void widen(const RawF32& raw, float (&x)[16]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) { x[i] = __uint_as_float(raw.a.w[i]); x[8 + i] = __uint_as_float(raw.b.w[i]); }
}
// the largest magnitude; a NaN if there is one
__device__ __forceinline__ float max_abs3(float a, float b, float c) { float d; asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c)); return d; }
__device__ __forceinline__ float amax16(const float (&x)[16]) {
    float m = max_abs3(x[0], x[1], x[2]);
#pragma unroll
    for (int i = 3; i < 15; i += 2) m = max_abs3(m, x[i], x[i + 1]);
    return max_abs3(m, x[15], x[15]);
}
// the same of 16 numbers as they were loaded
__device__ __forceinline__ float raw_amax(const RawF32& raw) { float x[16]; widen(raw, x); return amax16(x); }
// (magnitudes of pairs; the signs that come out are of no use)
__device__ __forceinline__ uint32_t max_abs_bf16x2(uint32_t a, uint32_t b) { uint32_t d; asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b)); return d; }
__device__ __forceinline__ float larger_half(uint32_t two) { const float lo = __uint_as_float(two << 16), hi = __uint_as_float(two & 0xFFFF0000u); return max_abs3(lo, hi, hi); }
__device__ __forceinline__ float raw_amax(const RawBf16& raw) {
    uint32_t m = raw.r.w[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) m = max_abs_bf16x2(m, raw.r.w[i]);
    return larger_half(m);
}
// ... of those that are finite; a: of all
template <class Raw>
__device__ __forceinline__ uint32_t finite_amax(const Raw& raw, float a) {
    uint32_t m = __float_as_uint(a);
    if (m >= 0x7F800000u) {
        float x[16];
        widen(raw, x);
        m = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) { const uint32_t b = __float_as_uint(x[i]) & 0x7FFFFFFFu; m = max(m, b < 0x7F800000u ? b : 0u); }
    }
    return m;
}
// the largest value of all threads of the block (a multiple of 32 threads); `buf`: 32 words
__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t* buf) {
    v = __reduce_max_sync(0xFFFFFFFFu, v);
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    v = threadIdx.x % 32 < blockDim.x / 32 ? buf[threadIdx.x & 31] : 0u;
    return __reduce_max_sync(0xFFFFFFFFu, v);
}

// One row by `nt` threads, a whole block or one of its warps (then `tid` is the lane): every chunk of the `padded` k is encoded and
// handed to `sink(k, chunk, byte, codes, field)`, `chunk` its number among the thread's, by all lanes of its warp together; NVFP4's row scale comes first (from registers where the row fits into them, else the row is read twice).
// `wide`: rows begin on 32-byte boundaries.
template <class T> struct RawOf { typedef RawBf16 type; };
template <> struct RawOf<float> { typedef RawF32 type; };
template <int FORMAT, int CHUNKS, class T, class Sink>
__device__ __forceinline__ void encode_row(const T* row, int have, int padded, bool wide, int tid, int nt, uint32_t* buf, float* outer, Sink sink) {
    constexpr bool FP32 = sizeof(T) == 4;
    const int span = nt * 16 * CHUNKS, parts = (padded + span - 1) / span, k0 = tid * 16, step = nt * 16;
    typename RawOf<T>::type raw[CHUNKS];
    float most[CHUNKS];
    int field = 127;
    if constexpr (FORMAT == MOQE_FP_NVFP4) {
        uint32_t m = 0;
        for (int part = 0; part < parts; ++part) {
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) load16(row, part * span + k0 + i * step, have, wide, raw[i]);
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) { most[i] = raw_amax(raw[i]); m = max(m, finite_amax(raw[i], most[i])); }
        }
        field = nv_row_field(nt == 32 ? __reduce_max_sync(0xFFFFFFFFu, m) : block_max(m, buf));
        if (outer && tid == 0) *outer = pow2_field(field);
    }
    for (int part = 0; part < parts; ++part) {
        if (FORMAT != MOQE_FP_NVFP4 || parts > 1) {
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) load16(row, part * span + k0 + i * step, have, wide, raw[i]);
        }
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) {
            const int k = part * span + k0 + i * step;
            if (k - (int)(threadIdx.x & 31) * 16 >= padded) break;         // (the whole warp)
            float x[16];
            widen(raw[i], x);
            float a = FORMAT == MOQE_FP_NVFP4 ? parts > 1 ? raw_amax(raw[i]) : most[i] : amax16(x);
            uint32_t codes[2];
            if constexpr (FORMAT == MOQE_FP_MXFP4) { const float b = __shfl_xor_sync(0xFFFFFFFFu, a, 1); a = max_abs3(a, b, b); }
            const uint32_t byte = encode16<FORMAT, FP32>(x, a, field, codes);
            sink(k, part * CHUNKS + i, byte, codes, field);
        }
    }
}
// Threads that take a row, so that the row fits into their registers if it can; rows of a block: four where a warp is enough.
inline int row_threads(int K, int chunks) {
    const int t = ((K + 15) / 16 + chunks - 1) / chunks;
    return t >= 512 ? 512 : (t + 31) / 32 * 32;
}
constexpr int ROWS_OF_WARPS = 4;
struct RowLaunch { int blocks, threads; };
inline RowLaunch row_launch(int rows, int K, int chunks) {
    const int t = row_threads(K, chunks);
    return t > 32 ? RowLaunch{rows, t} : RowLaunch{rows / ROWS_OF_WARPS + (rows % ROWS_OF_WARPS != 0), 32 * ROWS_OF_WARPS};   // (any int of rows)
}
// which row this thread works on, as which of how many threads
struct RowPlace { int row, tid, nt; };
__device__ __forceinline__ RowPlace row_place(bool warps) {
    if (warps) return {(int)(blockIdx.x * ROWS_OF_WARPS + (threadIdx.x >> 5)), (int)(threadIdx.x & 31), 32};
    return {(int)blockIdx.x, (int)threadIdx.x, (int)blockDim.x};
}
// ... into a packed row, of which a thread has every nt-th chunk, the same place in some k-blocks: four scales to a store.  (All lanes of
// a warp; `padded` is a multiple of 256, so half warps are there as a whole.)
struct PackedLane { uint8_t *code, *scale; size_t code_step, scale_step; };
template <int FORMAT>
__device__ __forceinline__ PackedLane packed_lane(const PackedRow& out, int tid, int nt) {
    const int kb = tid >> 4, in = tid & 15;                               // (nt is a multiple of 32)
    return {out.chunk(kb, in >> 1) + (in & 1) * 8, out.scale(kb, FORMAT == MOQE_FP_MXFP4 ? in >> 1 : in), (nt >> 4) * out.codes_kb, (nt >> 4) * out.sf_kb};
}
template <int FORMAT>
__device__ __forceinline__ void put_packed(const PackedLane& out, int chunk, bool inside, uint32_t byte, const uint32_t (&codes)[2]) {
    constexpr int LANES = FORMAT == MOQE_FP_MXFP4 ? 2 : 1;                 // of a block
    uint32_t w = byte | __shfl_down_sync(0xFFFFFFFFu, byte, LANES) << 8;
    w |= __shfl_down_sync(0xFFFFFFFFu, w, 2 * LANES) << 16;
    if (!inside) return;
    *reinterpret_cast<uint2*>(out.code + chunk * out.code_step) = make_uint2(codes[0], codes[1]);
    if ((threadIdx.x & (4 * LANES - 1)) == 0) *reinterpret_cast<uint32_t*>(out.scale + chunk * out.scale_step) = w;
}

// a call's kernels run on the current device, and read an expert where it was built
inline moqe_status fp_on_current_device(const moqe_fp_expert* e) {
    int now = 0;
    if (cudaGetDevice(&now) != cudaSuccess) { cudaGetLastError(); return MOQE_ERR_CUDA; }
    return now == e->device ? MOQE_OK : MOQE_ERR_MISMATCH;
}

// quantize.cu: device memory of experts (a pool of the library's)
void* expert_malloc(size_t bytes, int device, cudaStream_t st, bool& pooled);
bool expert_free(void* p, bool pooled, int device);

// fp_rows.cu: the token rows of a sorted batch in their experts' formats
struct FpTokens {
    uint8_t *codes, *sf; float* outer;    // regions of the workspace
    size_t row_bytes, block_sf;           // room for a row's codes, and for a block of scales: the largest of the call's formats
    int TN;                               // most tokens of a tile
};
struct FpExperts { uint8_t format[MOQE_MAX_EXPERTS]; };
moqe_status launch_fp_tokens(const void* X, const int32_t* perm, const int32_t* offsets, int M, int K, int E, const FpExperts& formats,
                             const FpTokens& tokens, uint32_t* counters, int n_counters, cudaStream_t st);

// fp_gemm.cu
moqe_status launch_fp_gemm(const moqe_fp_expert* const* ex, int E, int M, const int32_t* perm, const int32_t* offsets, const FpTokens& tokens,
                           uint32_t* counters, void* partials, void* Y, cudaStream_t st);
int fp_gemm_counters();
size_t fp_gemm_partial_bytes(int M);

// fp_gemv.cu: batches of one row, or a few of a small layer
bool fp_gemv_supported(const moqe_fp_expert* const* ex, int E, int M);
moqe_status launch_fp_gemv(const void* X, int M, const int32_t* perm, const int32_t* offsets, const moqe_fp_expert* const* ex, int E, void* Y, cudaStream_t st);

}  // namespace moqe
