// Routed product of floating-point experts for one row (a single sequence's decode step), and for a few of a small layer: one launch, a
// row's weights read once.
//
//   Y[perm[j]][n] = bf16( o_x o_w[n] sum_b sx[b] sw[n][b] sum_{k in b} cx[k] cw[n][k] )
//
// 4.25 or 4.5 bits a weight have to come from HBM, but latency counts as much: the row's place, its numbers and their quantization come
// one after the other before the first weight is multiplied.  The tensor-core kernel needs the row quantized by a kernel before
// it, splits few tiles along k and adds parked sums up, which is most of its time here.  So a block of 4 to 16 warps takes 32
// channels and all of k: nothing is added up outside the block, and every block quantizes the row for itself while its first
// weights are on their way.  A row in a chain of calls, experts in turn so that weights come from HBM, us (the bytes' time; the
// tensor-core kernel): 11008 k -> 4096 MXFP4 9.1 (3.7; 13.7), NVFP4 10.1 (3.9; 14.7), bf16 17.0 (13.9; 23.6); 4096 k -> 4096 5.6 (1.4;
// 10.3), 6.1 (1.5; 10.5), 8.4 (5.2; 15.3); 4096 k -> 11008 10.6 (3.7; 11.3), 11.5 (3.9; 11.5), 18.7 (13.9; 25.2).  The same expert again and
// again, its weights in L2: 11008 k -> 4096 8.2, 8.8, 11.4.
//
// A 4-bit number doubled is a whole number, {0, 1, 2, 3, 4, 6, 8, 12} and a sign, so that the products of a block of codes are
// summed exactly in integers, four to an instruction; the two scales and the row scales are applied in fp32.  One byte permutation looks
// up four numbers: a selector nibble is a code, and its top bit, the sign, makes the looked-up byte's sign bit fill the result, which is
// zero for this table; so the codes give the positive numbers, the codes with inverted signs the negative ones (5.5 integer
// instructions for four codes, about what HBM leaves time for).
#include "fp_formats.cuh"

namespace moqe {
namespace {

constexpr int GEMV_WARPS = 16, GEMV_THREADS = 32 * GEMV_WARPS;      // at most, of a block
constexpr int GEMV_SMEM_MAX = 96 * 1024;

struct GemvExpert { uint8_t* tiles; const float* outer; int format, KB; };
struct GemvParams {
    GemvExpert ex[MOQE_MAX_EXPERTS];
    const __nv_bfloat16* X;
    const int32_t *perm, *offsets;
    __nv_bfloat16* Y;
    int K, N, E;
    bool wide;
};

constexpr uint32_t TWICE_LO = 0x03020100u, TWICE_HI = 0x0C080604u;                       // e2m1 magnitudes, doubled
__device__ __forceinline__ uint32_t look_up(uint32_t codes) {                              // codes in the low 16 bits
    uint32_t d;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(d) : "r"(TWICE_LO), "r"(TWICE_HI), "r"(codes));
    return d;
}
__device__ __forceinline__ uint4 load_weights(const uint8_t* p) {                          // (nobody else of this SM reads them)
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
// sum of eight codes' doubled numbers times eight small integers (signed bytes)
__device__ __forceinline__ int dot8(uint32_t codes, uint32_t a0, uint32_t a1, int acc) {
    const uint32_t flipped = codes ^ 0x88888888u;
    int pos = __dp4a((int)look_up(codes), (int)a0, acc), neg = __dp4a((int)look_up(flipped), (int)a0, 0);
    pos = __dp4a((int)look_up(codes >> 16), (int)a1, pos);
    neg = __dp4a((int)look_up(flipped >> 16), (int)a1, neg);
    return pos - neg;
}

// What a lane reads of a k-block: of 4 x 8 channels (8 apart in each of the tile's quarters) the 16-byte chunks of two rows of each
// eight, and the scales of these two rows in all quarters.
struct GemvBlock { uint4 w[4][2]; uint4 sf[2]; };
template <int FORMAT>
__device__ __forceinline__ void load_block(const uint8_t* tile, int q, int lane, GemvBlock& b) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int row = (lane >> 3) + 4 * h, c = (lane & 7) ^ row;
#pragma unroll
        for (int j = 0; j < 4; ++j) b.w[j][h] = load_weights(tile + (4 * j + q) * 1024 + h * 512 + lane * 16);
        if constexpr (FORMAT != MOQE_FP_BF16)
            b.sf[h] = __ldg(reinterpret_cast<const uint4*>(tile + 16384 + (FORMAT == MOQE_FP_MXFP4 ? c >> 2 : c >> 1) * 512 + (8 * q + row) * 16));
    }
}
// what the two scales in the low 16 bits stand for
__device__ __forceinline__ float2 e4m3_pair(uint32_t two) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)(two & 0x7F7Fu)));
    return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
// (a product of two scales that fp32 does not hold may still meet a sum of zero)
__device__ __forceinline__ float finite_or_nan(float s) { float d; asm("min.NaN.f32 %0, %1, 0f7F7FFFFF;" : "=f"(d) : "f"(s)); return d; }
__device__ __forceinline__ uint32_t word_of(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// act: the row as signed bytes (4-bit formats: doubled numbers) or bf16, 256 or 128 bytes a k-block; sx: its blocks' scales
template <int FORMAT>
__device__ __forceinline__ void add_block(const GemvBlock& b, const unsigned char* act, const float* sx, int kb, int lane, float (&acc)[4][2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int c = (lane & 7) ^ ((lane >> 3) + 4 * h);
        if constexpr (FORMAT == MOQE_FP_BF16) {
            const uint4 a = *reinterpret_cast<const uint4*>(act + kb * 128 + c * 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t x = word_of(a, i);
                const float x0 = __uint_as_float(x << 16), x1 = __uint_as_float(x & 0xFFFF0000u);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t w = word_of(b.w[j][h], i);
                    acc[j][h] = fmaf(__uint_as_float(w << 16), x0, acc[j][h]);
                    acc[j][h] = fmaf(__uint_as_float(w & 0xFFFF0000u), x1, acc[j][h]);
                }
            }
        } else {
            const float s1 = FORMAT == MOQE_FP_MXFP4 ? sx[kb * 8 + c] : 0.f;
            const float2 s2 = FORMAT == MOQE_FP_MXFP4 ? make_float2(0.f, 0.f) : *reinterpret_cast<const float2*>(sx + kb * 16 + 2 * c);
            const uint4 a0 = *reinterpret_cast<const uint4*>(act + kb * 256 + c * 32), a1 = *reinterpret_cast<const uint4*>(act + kb * 256 + c * 32 + 16);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint4 w = b.w[j][h];
                const uint32_t s = word_of(b.sf[h], j);
                if constexpr (FORMAT == MOQE_FP_MXFP4) {
                    const int sum = dot8(w.x, a0.x, a0.y, dot8(w.y, a0.z, a0.w, dot8(w.z, a1.x, a1.y, dot8(w.w, a1.z, a1.w, 0))));
                    acc[j][h] = fmaf((float)sum, finite_or_nan(e8m0_value((s >> (8 * (c & 3))) & 255u) * s1), acc[j][h]);
                } else {
                    const int lo = dot8(w.x, a0.x, a0.y, dot8(w.y, a0.z, a0.w, 0)), hi = dot8(w.z, a1.x, a1.y, dot8(w.w, a1.z, a1.w, 0));
                    const float2 sw = e4m3_pair(s >> (16 * (c & 1)));
                    acc[j][h] = fmaf((float)lo, sw.x * s2.x, acc[j][h]);
                    acc[j][h] = fmaf((float)hi, sw.y * s2.y, acc[j][h]);
                }
            }
        }
    }
}

template <int FORMAT>
__device__ __forceinline__ void gemv(const GemvParams& p, const GemvExpert& x, int from, unsigned char* smem, uint32_t* buf, float (*sums)[32]) {
    const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5, lane = threadIdx.x & 31, nt = blockIdx.x >> 2, q = blockIdx.x & 3;
    constexpr int STRIDE = FORMAT == MOQE_FP_BF16 ? 16384 : FORMAT == MOQE_FP_MXFP4 ? 17408 : 18432;
    const uint8_t* tile = x.tiles + (size_t)nt * x.KB * STRIDE;
    GemvBlock b;
    if (warp < x.KB) load_block<FORMAT>(tile + (size_t)warp * STRIDE, q, lane, b);       // (on its way while the row is quantized)
    const __nv_bfloat16* row = p.X + (size_t)from * p.K;
    float* sx = reinterpret_cast<float*>(smem + x.KB * 256);
    float ox = 1.f;
    if constexpr (FORMAT == MOQE_FP_BF16) {
        for (int c = threadIdx.x; c < x.KB * 8; c += blockDim.x)
            reinterpret_cast<uint4*>(smem)[c] = c * 8 < p.K ? *reinterpret_cast<const uint4*>(row + c * 8) : make_uint4(0, 0, 0, 0);
    } else {
        int f = 127;
        encode_row<FORMAT, 3>(row, p.K, x.KB * 256, p.wide, (int)threadIdx.x, (int)blockDim.x, buf, nullptr, [&](int k, int, uint32_t byte, const uint32_t (&c)[2], int field) {
            f = field;
            if (k >= x.KB * 256) return;
            uint32_t o[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t four = i & 1 ? c[i >> 1] >> 16 : c[i >> 1];
                o[i] = __vsub4(look_up(four), look_up(four ^ 0x8888u));
            }
            *reinterpret_cast<uint4*>(smem + k) = make_uint4(o[0], o[1], o[2], o[3]);
            if (FORMAT == MOQE_FP_NVFP4) sx[k >> 4] = e4m3_value(byte);
            else if ((k & 16) == 0) sx[k >> 5] = 0.25f * e8m0_value(byte);                 // (both factors are doubled)
        });
        ox = pow2_field(f);
    }
    __syncthreads();
    float acc[4][2] = {};
    for (int kb = warp; kb < x.KB; kb += warps) {
        GemvBlock next;
        if (kb + warps < x.KB) load_block<FORMAT>(tile + (size_t)(kb + warps) * STRIDE, q, lane, next);
        add_block<FORMAT>(b, smem, sx, kb, lane, acc);
        b = next;
    }
    // eight lanes share a channel, then the warps
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int d = 1; d < 8; d <<= 1) acc[j][h] += __shfl_xor_sync(0xFFFFFFFFu, acc[j][h], d);
            if ((lane & 7) == 0) sums[warp][8 * j + 4 * h + (lane >> 3)] = acc[j][h];
        }
    __syncthreads();
    if (threadIdx.x < 32) {
        float s = 0.f;
        for (int w = 0; w < warps; ++w) s += sums[w][threadIdx.x];
        const int n = nt * 128 + 32 * (threadIdx.x >> 3) + 8 * q + (threadIdx.x & 7);
        if (n < p.N) {
            if constexpr (FORMAT == MOQE_FP_NVFP4) s *= 0.25f;                           // (both factors are doubled)
            if constexpr (FORMAT == MOQE_FP_NVFP4) s = s * x.outer[n] * ox;
            p.Y[(size_t)from * p.N + n] = __float2bfloat16_rn(s);
        }
    }
}

__global__ void __launch_bounds__(GEMV_THREADS, 1) fp_gemv_kernel(const __grid_constant__ GemvParams p) {
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ uint32_t buf[32];
    __shared__ float sums[GEMV_WARPS][32];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    // the row's expert: whose segment holds its place, if any does
    const int lane = threadIdx.x & 31, at = min(lane, p.E - 1), place = blockIdx.y, from = p.perm[place];
    const uint32_t mine = __ballot_sync(0xFFFFFFFFu, lane < p.E && p.offsets[at] <= place && p.offsets[at + 1] > place);
    if (mine == 0) return;
    const GemvExpert& x = p.ex[__ffs(mine) - 1];
    if (x.format == MOQE_FP_MXFP4) gemv<MOQE_FP_MXFP4>(p, x, from, smem, buf, sums);
    else if (x.format == MOQE_FP_NVFP4) gemv<MOQE_FP_NVFP4>(p, x, from, smem, buf, sums);
    else gemv<MOQE_FP_BF16>(p, x, from, smem, buf, sums);
}

size_t gemv_smem(const moqe_fp_expert* const* ex, int E) {
    size_t most = 0;
    for (int e = 0; e < E; ++e) {
        const size_t s = (size_t)ex[e]->KB * (ex[e]->format == MOQE_FP_BF16 ? 128 : ex[e]->format == MOQE_FP_MXFP4 ? 256 + 32 : 256 + 64);
        most = s > most ? s : most;
    }
    return most;
}

}  // namespace

// One row; or rows that a block each for 32 channels takes less time for than the 4 us that the tensor-core kernel and the one before it
// need to get going.  A block costs as much as 530 k of its channels.  This kernel / the other, us:
//   4096 x 4096  4-bit: 1 row 4.6 / 10.4, 2 rows 7.1 / 10.3, 3 rows 10.7 / 10.3;  with a bf16 expert: 2 rows 10 / 18
//   1024 x 1024  4-bit: 4 rows 3.9 / 7.5, 16 rows 5.1 / 7.5, 32 rows 7.5 / 7.5;  with a bf16 expert: 16 rows 4.7 / 9.8
//   512 x 512    4-bit: 64 rows 6.2 / 6.7, 128 rows 11.2 / 7.1;   11008 x 4096, 2 rows: 14.7 / 10.5
bool fp_gemv_supported(const moqe_fp_expert* const* ex, int E, int M) {
    if (gemv_smem(ex, E) > (size_t)GEMV_SMEM_MAX) return false;
    return M == 1 || (long long)M * ex[0]->Np * (ex[0]->K + 530ll) <= 49000000;
}

moqe_status launch_fp_gemv(const void* X, int M, const int32_t* perm, const int32_t* offsets, const moqe_fp_expert* const* ex, int E, void* Y, cudaStream_t st) {
    GemvParams p = {};
    for (int e = 0; e < E; ++e) p.ex[e] = {ex[e]->tiles, ex[e]->outer, ex[e]->format, ex[e]->KB};
    p.X = (const __nv_bfloat16*)X; p.perm = perm; p.offsets = offsets; p.Y = (__nv_bfloat16*)Y;
    p.K = ex[0]->K; p.N = ex[0]->N; p.E = E;
    p.wide = p.K % 16 == 0 && (uintptr_t)X % 32 == 0;
    static std::atomic<unsigned long long> attr{0};
    if (!ensure_dynamic_smem((const void*)fp_gemv_kernel, GEMV_SMEM_MAX, attr)) { cudaGetLastError(); return MOQE_ERR_CUDA; }
    cudaLaunchConfig_t cfg = {};
    // all blocks at once, if they are not too many: 4, 2 or 1 to an SM (344 blocks of 16 warps, three after one another on an SM: 16.3 us
    // for 11008 channels x 4096 k, with 4 warps 11.3)
    const int blocks = ex[0]->Np / 32 * M, sms = device_sm_count(), warps = blocks <= sms ? GEMV_WARPS : blocks <= 2 * sms ? 8 : 4;
    cfg.gridDim = dim3(ex[0]->Np / 32, M); cfg.blockDim = dim3(32 * warps); cfg.dynamicSmemBytes = gemv_smem(ex, E); cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at; cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, fp_gemv_kernel, p) != cudaSuccess) { cudaGetLastError(); return MOQE_ERR_CUDA; }
    count_launch();
    return MOQE_OK;
}

}  // namespace moqe
