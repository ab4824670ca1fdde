// Rows of activations in the microscaled 4-bit formats: canonical arrays for the caller (moqe_fp4_quantize_rows), and the packed
// token rows of a routed product.  One block or warp a row (see encode_row).  Bound by HBM: 2 bytes a number are
// read, half a byte and the scales written.
#include "fp_formats.cuh"

namespace moqe {
namespace {

// (Held to 64 registers, a few of which NVFP4 with four chunks spills, more rows are under way on an SM: 16384 x 11008 NVFP4 116 -> 95 us, with
// values 154 -> 135, MXFP4 74.6 -> 70.8 and 120.8 -> 122.9.)
template <int FORMAT, int CHUNKS>
__global__ void __maxnreg__(64) fp4_rows_kernel(const __nv_bfloat16* __restrict__ X, int M, int K, bool wide, bool warps, uint8_t* codes, uint8_t* scales, float* outer, __nv_bfloat16* values) {
    __shared__ uint32_t buf[32];
    const RowPlace at = row_place(warps);
    if (at.row >= M) return;
    const size_t m = at.row;
    const int blocks = (K + fp_block(FORMAT) - 1) / fp_block(FORMAT);
    encode_row<FORMAT, CHUNKS>(X + m * K, K, K, wide, at.tid, at.nt, buf, outer ? outer + m : nullptr, [&](int k, uint32_t byte, const uint32_t (&c)[2], int field) {
        if (k >= K) return;
        if (codes) {
            uint32_t* to = reinterpret_cast<uint32_t*>(codes + m * (K / 2) + k / 2);
            if (wide) *reinterpret_cast<uint2*>(to) = make_uint2(c[0], c[1]);
            else { to[0] = c[0]; if (k + 8 < K) to[1] = c[1]; }
        }
        if (scales && (FORMAT == MOQE_FP_NVFP4 || k % 32 == 0)) scales[m * blocks + k / fp_block(FORMAT)] = (uint8_t)byte;
        if (values) {
            const float s = FORMAT == MOQE_FP_MXFP4 ? e8m0_value(byte) : e4m3_value(byte), o = pow2_field(field);
            Raw32 r;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float v[8];
                e2m1_values(c[h], v);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    r.w[4 * h + i] = FORMAT == MOQE_FP_MXFP4 ? pack_bf16x2(v[2 * i] * s, v[2 * i + 1] * s) : pack_bf16x2(v[2 * i] * s * o, v[2 * i + 1] * s * o);
            }
            store32(values + m * K + k, (K - k) * 2, wide, r);
        }
    });
}

template <int FORMAT, int CHUNKS>
__device__ __forceinline__ void pack_row(const __nv_bfloat16* row, int K, bool wide, const RowPlace& at, const PackedRow& out, float* outer, uint32_t* buf) {
    const int padded = fp_kblocks(K, FORMAT) * 256;
    encode_row<FORMAT, CHUNKS>(row, K, padded, wide, at.tid, at.nt, buf, outer, [&](int k, uint32_t byte, const uint32_t (&c)[2], int) { put_packed<FORMAT>(out, k, padded, byte, c); });
}

struct TokenParams {
    const __nv_bfloat16* X;
    const int32_t *perm, *offsets;
    int M, K, E;
    bool wide, warps;
    FpTokens t;
    uint32_t* counters;
    int n_counters;
    FpExperts formats;
};

// One block, or one warp of it, a place j of the sorted order.  The row goes to its place in its expert's segment; segments start at
// multiples of 16 rows.  Places outside [offsets[0], offsets[E]) are nobody's.  (94 registers; held to 64 or 72 it spills, and 4160 rows of
// 18944 k in NVFP4 take 13 us longer.)
template <int CHUNKS>
__global__ void fp_tokens_kernel(const __grid_constant__ TokenParams p) {
    __shared__ uint32_t buf[32];
    // the product behind this kernel may read the offset table before this kernel has ended, so nothing is let go before the wait
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const RowPlace at = row_place(p.warps);
    const int j = at.row;
    for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < p.n_counters; i += gridDim.x * blockDim.x) p.counters[i] = 0;
    if (j >= p.M) return;
    const int lane = threadIdx.x & 31, from = p.perm[j];
    const int lo = lane < p.E ? p.offsets[lane] : 0x7FFFFFFF, hi = lane < p.E ? p.offsets[lane + 1] : 0x7FFFFFFF;
    const int n = lane < p.E ? hi - lo : 0, pad = (n + 15) & ~15, blocks = (n + p.t.TN - 1) / p.t.TN * (p.t.TN > 128 ? 2 : 1);
    const uint32_t mine = __ballot_sync(0xFFFFFFFFu, j >= lo && j < hi);
    if (mine == 0) return;
    const int e = __ffs(mine) - 1;
    const size_t pad0 = __reduce_add_sync(0xFFFFFFFFu, lane < e ? pad : 0), blk0 = __reduce_add_sync(0xFFFFFFFFu, lane < e ? blocks : 0);
    const int i = j - __shfl_sync(0xFFFFFFFFu, lo, e), seg = __shfl_sync(0xFFFFFFFFu, pad, e);
    const int format = p.formats.format[e];
    const __nv_bfloat16* row = p.X + (size_t)from * p.K;
    const int KB = fp_kblocks(p.K, format);
    const PackedRow out = token_row(p.t.codes + pad0 * p.t.row_bytes, p.t.sf + blk0 * p.t.block_sf, format, i, seg, token_tiles(__shfl_sync(0xFFFFFFFFu, n, e), p.t.TN), p.t.TN);
    if (format == MOQE_FP_MXFP4) pack_row<MOQE_FP_MXFP4, CHUNKS>(row, p.K, p.wide, at, out, nullptr, buf);
    else if (format == MOQE_FP_NVFP4) pack_row<MOQE_FP_NVFP4, CHUNKS>(row, p.K, p.wide, at, out, p.t.outer + pad0 + i, buf);
    else {
        for (int c0 = at.tid; c0 < KB * 4; c0 += at.nt * CHUNKS) {
            RawBf16 raw[CHUNKS];
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) load16(row, (c0 + i * at.nt) * 16, p.K, p.wide, raw[i]);
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) {
                const int c = 2 * (c0 + i * at.nt);
                const uint32_t* w = raw[i].r.w;
                if (c >= KB * 8) break;
                *reinterpret_cast<uint4*>(out.chunk(c >> 3, c & 7)) = make_uint4(w[0], w[1], w[2], w[3]);
                *reinterpret_cast<uint4*>(out.chunk(c >> 3, (c & 7) + 1)) = make_uint4(w[4], w[5], w[6], w[7]);
            }
        }
    }
}

int row_chunks(int M) { return M < 1024 ? 2 : 4; }

}  // namespace

moqe_status launch_fp_tokens(const void* X, const int32_t* perm, const int32_t* offsets, int M, int K, int E, const FpExperts& formats,
                             const FpTokens& tokens, uint32_t* counters, int n_counters, cudaStream_t st) {
    const bool wide = K % 16 == 0 && (uintptr_t)X % 32 == 0;
    TokenParams p = {(const __nv_bfloat16*)X, perm, offsets, M, K, E, wide, row_threads(K, row_chunks(M)) == 32, tokens, counters, n_counters, formats};
    cudaLaunchConfig_t cfg = {};
    const RowLaunch l = row_launch(M, K, row_chunks(M));
    cfg.gridDim = dim3(l.blocks); cfg.blockDim = dim3(l.threads); cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at; cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, row_chunks(M) == 2 ? fp_tokens_kernel<2> : fp_tokens_kernel<4>, p) != cudaSuccess) { cudaGetLastError(); return MOQE_ERR_CUDA; }
    count_launch();
    return MOQE_OK;
}

}  // namespace moqe

using namespace moqe;

extern "C" moqe_status moqe_fp4_quantize_rows(const void* X_bf16, int M, int K, int format, uint8_t* codes, uint8_t* scales, float* outer,
                                              void* values_bf16, void* stream) {
    if (M < 0 || K <= 0) return MOQE_ERR_SHAPE;
    if ((format != MOQE_FP_MXFP4 && format != MOQE_FP_NVFP4) || K % 8 != 0 || K > FP_MAX_K) return MOQE_ERR_UNSUPPORTED;
    if (M == 0) return MOQE_OK;
    if (!X_bf16) return MOQE_ERR_NULL;
    if ((uintptr_t)X_bf16 % 16 || (uintptr_t)values_bf16 % 16 || (uintptr_t)codes % 16 || (uintptr_t)outer % 4) return MOQE_ERR_UNSUPPORTED;
    const bool wide = K % 16 == 0 && (uintptr_t)X_bf16 % 32 == 0 && (uintptr_t)values_bf16 % 32 == 0;
    const int chunks = row_chunks(M);
    const auto kernel = format == MOQE_FP_MXFP4 ? (chunks == 2 ? fp4_rows_kernel<MOQE_FP_MXFP4, 2> : fp4_rows_kernel<MOQE_FP_MXFP4, 4>)
                                                : (chunks == 2 ? fp4_rows_kernel<MOQE_FP_NVFP4, 2> : fp4_rows_kernel<MOQE_FP_NVFP4, 4>);
    const RowLaunch l = row_launch(M, K, chunks);
    kernel<<<l.blocks, l.threads, 0, (cudaStream_t)stream>>>((const __nv_bfloat16*)X_bf16, M, K, wide, row_threads(K, chunks) == 32, codes, scales, outer, (__nv_bfloat16*)values_bf16);
    count_launch();
    return cuda_ok(cudaGetLastError());
}
