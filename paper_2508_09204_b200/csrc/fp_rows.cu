// Rows of activations in the microscaled 4-bit formats: canonical arrays for the caller (moqe_fp4_quantize_rows), and the packed
// token rows of a routed product.  One block a row; a thread takes 16 consecutive k at a time.  Bound by HBM: 2 bytes a number are
// read, half a byte and the scales written.
#include "fp_formats.cuh"

namespace moqe {
namespace {

// NVFP4's row scale: needs the whole row before the first block can be rounded; the second pass finds the row in L1 or L2.
template <class T>
__device__ __forceinline__ int row_field_of(const T* row, int K, uint32_t* buf) {
    uint32_t m = 0;
    for (int k = threadIdx.x * 16; k < K; k += blockDim.x * 16) {
        float x[16];
        load16(row, k, K, x);
        m = max(m, finite_amax16(x));
    }
    return nv_row_field(block_max(m, buf));
}

template <int FORMAT>
__global__ void fp4_rows_kernel(const __nv_bfloat16* __restrict__ X, int K, uint8_t* codes, uint8_t* scales, float* outer, __nv_bfloat16* values) {
    __shared__ uint32_t buf[32];
    const size_t m = blockIdx.x;
    const __nv_bfloat16* row = X + m * K;
    const int blocks = (K + fp_block(FORMAT) - 1) / fp_block(FORMAT);
    int field = 127;
    if constexpr (FORMAT == MOQE_FP_NVFP4) {
        field = row_field_of(row, K, buf);
        if (outer && threadIdx.x == 0) outer[m] = pow2_field(field);
    }
    for (int k0 = 0; k0 < K; k0 += blockDim.x * 16) {
        const int k = k0 + threadIdx.x * 16;
        float x[16];
        load16(row, k, K, x);
        uint32_t a = amax16(x), c[2];
        if constexpr (FORMAT == MOQE_FP_MXFP4) a = max(a, __shfl_xor_sync(0xFFFFFFFFu, a, 1));
        const uint32_t byte = encode16<FORMAT, false>(x, a, field, c);
        if (k >= K) continue;
        if (codes) {
            uint32_t* out = reinterpret_cast<uint32_t*>(codes + m * (K / 2) + k / 2);
            out[0] = c[0];
            if (k + 8 < K) out[1] = c[1];
        }
        if (scales && (FORMAT == MOQE_FP_NVFP4 || k % 32 == 0)) scales[m * blocks + k / fp_block(FORMAT)] = (uint8_t)byte;
        if (values) {
            const float s = FORMAT == MOQE_FP_MXFP4 ? e8m0_value(byte) : e4m3_value(byte), o = pow2_field(field);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (k + 8 * h >= K) break;
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t two = c[h] >> (8 * i);
                    const __nv_bfloat162 v = __floats2bfloat162_rn(e2m1_value(two & 15u) * s * o, e2m1_value((two >> 4) & 15u) * s * o);
                    w[i] = *reinterpret_cast<const uint32_t*>(&v);
                }
                *reinterpret_cast<uint4*>(values + m * K + k + 8 * h) = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    }
}

template <int FORMAT>
__device__ __forceinline__ void pack_row(const __nv_bfloat16* row, int K, const PackedRow& out, float* outer, uint32_t* buf) {
    int field = 127;
    if constexpr (FORMAT == MOQE_FP_NVFP4) {
        field = row_field_of(row, K, buf);
        if (threadIdx.x == 0) *outer = pow2_field(field);
    }
    const int padded = fp_kblocks(K, FORMAT) * 256;
    for (int k0 = 0; k0 < padded; k0 += blockDim.x * 16) {
        const int k = k0 + threadIdx.x * 16;
        float x[16];
        load16(row, k, K, x);
        uint32_t a = amax16(x), c[2];
        if constexpr (FORMAT == MOQE_FP_MXFP4) a = max(a, __shfl_xor_sync(0xFFFFFFFFu, a, 1));
        const uint32_t byte = encode16<FORMAT, false>(x, a, field, c);
        if (k >= padded) continue;
        const int kb = k >> 8, u = (k >> 4) & 15;
        *reinterpret_cast<uint2*>(out.chunk(kb, u >> 1) + 8 * (u & 1)) = make_uint2(c[0], c[1]);
        if (FORMAT == MOQE_FP_NVFP4) *out.scale(kb, u) = (uint8_t)byte;
        else if (!(u & 1)) *out.scale(kb, u >> 1) = (uint8_t)byte;
    }
}

struct TokenParams {
    const __nv_bfloat16* X;
    const int32_t *perm, *offsets;
    int K, E;
    FpTokens t;
    uint32_t* counters;
    int n_counters;
    FpExperts formats;
};

// One block a place j of the sorted order.  The row goes to its place in its expert's segment; segments start at multiples of 128
// rows.  Places outside [offsets[0], offsets[E]) are nobody's.
__global__ void fp_tokens_kernel(const __grid_constant__ TokenParams p) {
    __shared__ uint32_t buf[32];
    // the product behind this kernel may read the offset table before this kernel has ended, so nothing is let go before the wait
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int j = blockIdx.x;
    for (int i = j * blockDim.x + threadIdx.x; i < p.n_counters; i += gridDim.x * blockDim.x) p.counters[i] = 0;
    const int lane = threadIdx.x & 31;
    const int lo = lane < p.E ? p.offsets[lane] : 0x7FFFFFFF, hi = lane < p.E ? p.offsets[lane + 1] : 0x7FFFFFFF;
    const int pad = lane < p.E ? (hi - lo + 127) & ~127 : 0;
    const uint32_t mine = __ballot_sync(0xFFFFFFFFu, j >= lo && j < hi);
    if (mine == 0) return;
    const int e = __ffs(mine) - 1;
    const size_t pad0 = __reduce_add_sync(0xFFFFFFFFu, lane < e ? pad : 0);
    const int i = j - __shfl_sync(0xFFFFFFFFu, lo, e), seg = __shfl_sync(0xFFFFFFFFu, pad, e);
    const int format = p.formats.format[e];
    const __nv_bfloat16* row = p.X + (size_t)p.perm[j] * p.K;
    const int KB = fp_kblocks(p.K, format);
    const PackedRow out = token_row(p.t.codes + pad0 * p.t.row_bytes, p.t.sf + (pad0 >> p.t.sf_shift) * p.t.block_sf, format, i, seg, p.t.sf_shift);
    if (format == MOQE_FP_MXFP4) pack_row<MOQE_FP_MXFP4>(row, p.K, out, nullptr, buf);
    else if (format == MOQE_FP_NVFP4) pack_row<MOQE_FP_NVFP4>(row, p.K, out, p.t.outer + pad0 + i, buf);
    else {
        for (int c = threadIdx.x; c < KB * 8; c += blockDim.x) {
            const uint4 v = c * 8 < p.K ? *reinterpret_cast<const uint4*>(row + c * 8) : make_uint4(0, 0, 0, 0);
            *reinterpret_cast<uint4*>(out.chunk(c >> 3, c & 7)) = v;
        }
    }
}

int row_threads(int K) { return K >= 4096 ? 256 : K >= 2048 ? 128 : K >= 1024 ? 64 : 32; }

}  // namespace

moqe_status launch_fp_tokens(const void* X, const int32_t* perm, const int32_t* offsets, int M, int K, int E, const FpExperts& formats,
                             const FpTokens& tokens, uint32_t* counters, int n_counters, cudaStream_t st) {
    TokenParams p = {(const __nv_bfloat16*)X, perm, offsets, K, E, tokens, counters, n_counters, formats};
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(M); cfg.blockDim = dim3(row_threads(K)); cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at; cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, fp_tokens_kernel, p) != cudaSuccess) { cudaGetLastError(); return MOQE_ERR_CUDA; }
    count_launch();
    return MOQE_OK;
}

}  // namespace moqe

using namespace moqe;

extern "C" moqe_status moqe_fp4_quantize_rows(const void* X_bf16, int M, int K, int format, uint8_t* codes, uint8_t* scales, float* outer,
                                              void* values_bf16, void* stream) {
    if (M < 0 || K <= 0) return MOQE_ERR_SHAPE;
    if ((format != MOQE_FP_MXFP4 && format != MOQE_FP_NVFP4) || K % 8 != 0) return MOQE_ERR_UNSUPPORTED;
    if (M == 0) return MOQE_OK;
    if (!X_bf16) return MOQE_ERR_NULL;
    if ((uintptr_t)X_bf16 % 16 || (uintptr_t)values_bf16 % 16 || (uintptr_t)codes % 16 || (uintptr_t)outer % 4) return MOQE_ERR_UNSUPPORTED;
    const auto kernel = format == MOQE_FP_MXFP4 ? fp4_rows_kernel<MOQE_FP_MXFP4> : fp4_rows_kernel<MOQE_FP_NVFP4>;
    kernel<<<M, row_threads(K), 0, (cudaStream_t)stream>>>((const __nv_bfloat16*)X_bf16, K, codes, scales, outer, (__nv_bfloat16*)values_bf16);
    count_launch();
    return cuda_ok(cudaGetLastError());
}
