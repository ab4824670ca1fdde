// Floating-point experts: built from fp32 weights, imported from and exported to canonical arrays.  One block or warp
// a channel (see encode_row).
#include <new>

#include "fp_formats.cuh"

namespace moqe {
namespace {

// (64 registers, of which NVFP4 spills two: 3584 x 18944 NVFP4 145 -> 98 us, 11008 x 4096 49 -> 45.)
template <int FORMAT>
__global__ void __maxnreg__(64) fp_build_kernel(const float* __restrict__ W, int N, int K, int KB, bool wide, bool warps, uint8_t* tiles, float* outer) {
    __shared__ uint32_t buf[32];
    const RowPlace at = row_place(warps);                  // (channels are a multiple of a block's)
    const int n = at.row, padded = KB * fp_kbk(FORMAT);
    const PackedRow out = expert_row(tiles, KB, FORMAT, n);
    const float* row = W + (size_t)n * K;
    const int have = n < N ? K : 0;                         // channels behind the last are zeros
    if constexpr (FORMAT == MOQE_FP_BF16) {
        for (int k = at.tid * 16; k < padded; k += at.nt * 16) {
            RawF32 raw;
            load16(row, k, have, wide, raw);
            float x[16];
            widen(raw, x);
#pragma unroll
            for (int h = 0; h < 2; ++h)
                *reinterpret_cast<uint4*>(out.chunk(k >> 6, ((k >> 3) & 7) + h)) =
                    make_uint4(bf16_pair(x[8 * h], x[8 * h + 1]), bf16_pair(x[8 * h + 2], x[8 * h + 3]), bf16_pair(x[8 * h + 4], x[8 * h + 5]), bf16_pair(x[8 * h + 6], x[8 * h + 7]));
        }
    } else {
        const PackedLane to = packed_lane<FORMAT>(out, at.tid, at.nt);
        encode_row<FORMAT, 2>(row, have, padded, wide, at.tid, at.nt, buf, outer ? outer + n : nullptr,
                              [&](int k, int chunk, uint32_t byte, const uint32_t (&c)[2], int) { put_packed<FORMAT>(to, chunk, k < padded, byte, c); });
    }
}

// canonical arrays -> packed
template <int FORMAT>
__global__ void fp_import_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, const float* __restrict__ outer_in,
                                 const __nv_bfloat16* __restrict__ values, int N, int K, int KB, uint8_t* tiles, float* outer) {
    const int n = blockIdx.x, padded = KB * fp_kbk(FORMAT), have = n < N ? K : 0;
    const PackedRow out = expert_row(tiles, KB, FORMAT, n);
    if (FORMAT == MOQE_FP_NVFP4 && threadIdx.x == 0) outer[n] = n < N ? (outer_in ? outer_in[n] : 1.f) : 0.f;
    const int size = fp_block(FORMAT), blocks = (K + size - 1) / size;
    for (int k = threadIdx.x * 8; k < padded; k += blockDim.x * 8) {
        if constexpr (FORMAT == MOQE_FP_BF16) {
            const uint4 v = k < have ? *reinterpret_cast<const uint4*>(values + (size_t)n * K + k) : make_uint4(0, 0, 0, 0);
            *reinterpret_cast<uint4*>(out.chunk(k >> 6, (k >> 3) & 7)) = v;
        } else {
            const uint32_t v = k < have ? *reinterpret_cast<const uint32_t*>(codes + (size_t)n * (K / 2) + k / 2) : 0u;
            *reinterpret_cast<uint32_t*>(out.chunk(k >> 8, (k >> 5) & 7) + ((k >> 1) & 15)) = v;
            if (k % size == 0) {
                uint32_t b = k < have ? scales[(size_t)n * blocks + k / size] : 0u;
                *out.scale(k >> 8, (k & 255) / size) = (uint8_t)(FORMAT == MOQE_FP_NVFP4 ? b & 0x7Fu : b);
            }
        }
    }
}

// packed -> canonical arrays; a thread takes 16 consecutive k at a time.  `wide`: their rows lie on 8-byte (codes) and 32-byte boundaries
template <int FORMAT>
__global__ void fp_export_kernel(uint8_t* tiles, const float* outer, int K, int KB, bool wide, uint8_t* codes, uint8_t* scales, float* outer_out,
                                 __nv_bfloat16* values) {
    const int n = blockIdx.x;
    const PackedRow in = expert_row(tiles, KB, FORMAT, n);
    float o = 1.f;
    if constexpr (FORMAT == MOQE_FP_NVFP4) {
        o = outer[n];
        if (outer_out && threadIdx.x == 0) outer_out[n] = o;
    }
    // (a row scale that is a power of two, as of rows quantized here: every product is exact)
    const bool plain = (__float_as_uint(o) & 0x7FFFFFu) == 0;
    const auto scaled = [&](float a, float b) {
        if constexpr (FORMAT != MOQE_FP_NVFP4) return bf16_pair(a, b);
        return plain ? bf16_pair(a * o, b * o) : bf16_pair(mul_to_odd(a, o), mul_to_odd(b, o));
    };
    const int blocks = (K + fp_block(FORMAT) - 1) / fp_block(FORMAT);
    for (int k = threadIdx.x * 16; k < K; k += blockDim.x * 16) {
        Raw32 r;
        if constexpr (FORMAT == MOQE_FP_BF16) {
            const uint4 a = *reinterpret_cast<const uint4*>(in.chunk(k >> 6, (k >> 3) & 7)), b = *reinterpret_cast<const uint4*>(in.chunk(k >> 6, ((k >> 3) & 7) + 1));
            r.w[0] = a.x; r.w[1] = a.y; r.w[2] = a.z; r.w[3] = a.w; r.w[4] = b.x; r.w[5] = b.y; r.w[6] = b.z; r.w[7] = b.w;
        } else {
            const uint2 c = *reinterpret_cast<const uint2*>(in.chunk(k >> 8, (k >> 5) & 7) + ((k >> 1) & 8));
            const uint32_t byte = *in.scale(k >> 8, (k & 255) / fp_block(FORMAT));
            if (codes) {
                uint32_t* to = reinterpret_cast<uint32_t*>(codes + (size_t)n * (K / 2) + k / 2);
                if (wide) *reinterpret_cast<uint2*>(to) = c;
                else { to[0] = c.x; if (k + 8 < K) to[1] = c.y; }
            }
            if (scales && k % fp_block(FORMAT) == 0) scales[(size_t)n * blocks + k / fp_block(FORMAT)] = (uint8_t)byte;
            if (!values) continue;
            const float s = FORMAT == MOQE_FP_MXFP4 ? e8m0_value(byte) : e4m3_value(byte);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float v[8];
                e2m1_values(h ? c.y : c.x, v);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    r.w[4 * h + i] = scaled(v[2 * i] * s, v[2 * i + 1] * s);
            }
        }
        if (values) store32(values + (size_t)n * K + k, (K - k) * 2, wide, r);
    }
}

moqe_status fp_check(int N, int K, int format) {
    if (N <= 0 || K <= 0) return MOQE_ERR_SHAPE;
    if (format < MOQE_FP_MXFP4 || format > MOQE_FP_BF16 || K % 8 != 0 || K > FP_MAX_K || N > FP_MAX_N) return MOQE_ERR_UNSUPPORTED;
    return MOQE_OK;
}

moqe_status fp_alloc(int N, int K, int format, cudaStream_t st, moqe_fp_expert** out) {
    moqe_fp_expert* e = new (std::nothrow) moqe_fp_expert();
    if (!e) return MOQE_ERR_ALLOC;
    e->N = N; e->K = K; e->format = format;
    e->Np = (N + 127) / 128 * 128;
    e->KB = fp_kblocks(K, format);
    if (cudaGetDevice(&e->device) != cudaSuccess) { cudaGetLastError(); delete e; return MOQE_ERR_CUDA; }
    e->tiles_alloc = (size_t)(e->Np / 128) * e->KB * fp_tile_stride(format);
    e->outer_alloc = format == MOQE_FP_NVFP4 ? (size_t)e->Np * 4 : 0;
    e->tiles = (uint8_t*)expert_malloc(e->tiles_alloc + e->outer_alloc, e->device, st, e->pooled);
    if (!e->tiles) { delete e; return MOQE_ERR_ALLOC; }
    e->outer = e->outer_alloc ? (float*)(e->tiles + e->tiles_alloc) : nullptr;
    *out = e;
    return MOQE_OK;
}

int channel_threads(int K, int step) { return K >= 256 * step ? 256 : K >= 128 * step ? 128 : 64; }

}  // namespace
}  // namespace moqe

using namespace moqe;

extern "C" moqe_status moqe_fp_quantize(const float* W, int N, int K, int format, void* stream, moqe_fp_expert** out) {
    if (!W || !out) return MOQE_ERR_NULL;
    moqe_status s = fp_check(N, K, format);
    if (s != MOQE_OK) return s;
    if ((uintptr_t)W % 16) return MOQE_ERR_UNSUPPORTED;
    cudaStream_t st = (cudaStream_t)stream;
    moqe_fp_expert* e = nullptr;
    if ((s = fp_alloc(N, K, format, st, &e)) != MOQE_OK) return s;
    const auto kernel = format == MOQE_FP_MXFP4 ? fp_build_kernel<MOQE_FP_MXFP4> : format == MOQE_FP_NVFP4 ? fp_build_kernel<MOQE_FP_NVFP4> : fp_build_kernel<MOQE_FP_BF16>;
    const RowLaunch l = row_launch(e->Np, K, 2);
    kernel<<<l.blocks, l.threads, 0, st>>>(W, N, K, e->KB, (uintptr_t)W % 32 == 0, row_threads(K, 2) == 32, e->tiles, e->outer);
    count_launch();
    if (cudaGetLastError() != cudaSuccess) { moqe_fp_expert_destroy(e); return MOQE_ERR_CUDA; }
    *out = e;
    return MOQE_OK;
}

extern "C" moqe_status moqe_fp_expert_import(int N, int K, int format, const uint8_t* codes, const uint8_t* scales, const float* outer,
                                             const void* values_bf16, void* stream, moqe_fp_expert** out) {
    if (!out) return MOQE_ERR_NULL;
    moqe_status s = fp_check(N, K, format);
    if (s != MOQE_OK) return s;
    if (format == MOQE_FP_BF16 ? !values_bf16 : !codes || !scales) return MOQE_ERR_NULL;
    if (format == MOQE_FP_BF16 ? (uintptr_t)values_bf16 % 16 : (uintptr_t)codes % 4 || (uintptr_t)outer % 4) return MOQE_ERR_UNSUPPORTED;
    cudaStream_t st = (cudaStream_t)stream;
    moqe_fp_expert* e = nullptr;
    if ((s = fp_alloc(N, K, format, st, &e)) != MOQE_OK) return s;
    const auto kernel = format == MOQE_FP_MXFP4 ? fp_import_kernel<MOQE_FP_MXFP4> : format == MOQE_FP_NVFP4 ? fp_import_kernel<MOQE_FP_NVFP4> : fp_import_kernel<MOQE_FP_BF16>;
    kernel<<<e->Np, channel_threads(K, 8), 0, st>>>(codes, scales, outer, (const __nv_bfloat16*)values_bf16, N, K, e->KB, e->tiles, e->outer);
    count_launch();
    if (cudaGetLastError() != cudaSuccess) { moqe_fp_expert_destroy(e); return MOQE_ERR_CUDA; }
    *out = e;
    return MOQE_OK;
}

extern "C" moqe_status moqe_fp_expert_export(const moqe_fp_expert* e, uint8_t* codes, uint8_t* scales, float* outer, void* values_bf16, void* stream) {
    if (!e) return MOQE_ERR_NULL;
    if ((uintptr_t)codes % 4 || (uintptr_t)outer % 4 || (uintptr_t)values_bf16 % 16) return MOQE_ERR_UNSUPPORTED;
    if (e->format == MOQE_FP_BF16 ? codes || scales || outer : e->format == MOQE_FP_MXFP4 && outer) return MOQE_ERR_UNSUPPORTED;
    if (!codes && !scales && !outer && !values_bf16) return MOQE_OK;
    const moqe_status here = fp_on_current_device(e);
    if (here != MOQE_OK) return here;
    cudaStream_t st = (cudaStream_t)stream;
    const auto kernel = e->format == MOQE_FP_MXFP4 ? fp_export_kernel<MOQE_FP_MXFP4> : e->format == MOQE_FP_NVFP4 ? fp_export_kernel<MOQE_FP_NVFP4> : fp_export_kernel<MOQE_FP_BF16>;
    const bool wide = e->K % 16 == 0 && (uintptr_t)codes % 8 == 0 && (uintptr_t)values_bf16 % 32 == 0;
    kernel<<<e->N, channel_threads(e->K, 16), 0, st>>>(e->tiles, e->outer, e->K, e->KB, wide, codes, scales, outer, (__nv_bfloat16*)values_bf16);
    count_launch();
    return cuda_ok(cudaGetLastError());
}

extern "C" moqe_status moqe_fp_expert_info(const moqe_fp_expert* e, int* N, int* K, int* format, size_t* code_bytes, size_t* meta_bytes,
                                           size_t* alloc_bytes) {
    if (!e) return MOQE_ERR_NULL;
    const bool four = e->format != MOQE_FP_BF16;
    const int size = fp_block(e->format);
    if (N) *N = e->N;
    if (K) *K = e->K;
    if (format) *format = e->format;
    if (code_bytes) *code_bytes = four ? (size_t)e->N * e->K / 2 : (size_t)e->N * e->K * 2;
    if (meta_bytes) *meta_bytes = four ? (size_t)e->N * ((e->K + size - 1) / size) + (e->format == MOQE_FP_NVFP4 ? (size_t)e->N * 4 : 0) : 0;
    if (alloc_bytes) *alloc_bytes = e->tiles_alloc + e->outer_alloc;
    return MOQE_OK;
}

extern "C" moqe_status moqe_fp_expert_destroy(moqe_fp_expert* e) {
    if (!e) return MOQE_ERR_NULL;
    const bool ok = expert_free(e->tiles, e->pooled, e->device);
    delete e;
    return ok ? MOQE_OK : MOQE_ERR_CUDA;
}
