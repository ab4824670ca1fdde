// Rows of activations in the microscaled 4-bit formats: canonical arrays for the caller (moqe_fp4_quantize_rows), and the packed
// token rows of a routed product.  One block or warp a row (see encode_row), or a ring of rows in shared memory.  Bound by HBM: 2 bytes a number are
// read, half a byte and the scales written.
#include "fp_formats.cuh"
#include "ptx.cuh"

namespace moqe {
namespace {

// (Held to 64 registers, of which both formats spill a few with four chunks (24 and 56 bytes stored), more rows are under way on an SM: 16384 x
// 11008 NVFP4 116 -> 95 us, with values 154 -> 135, MXFP4 74.6 -> 70.8 and 120.8 -> 122.9.)
template <int FORMAT, int CHUNKS>
__global__ void __maxnreg__(64) fp4_rows_kernel(const __nv_bfloat16* __restrict__ X, int M, int K, bool wide, bool warps, uint8_t* codes, uint8_t* scales, float* outer, __nv_bfloat16* values) {
    __shared__ uint32_t buf[32];
    const RowPlace at = row_place(warps);
    if (at.row >= M) return;
    const size_t m = at.row;
    const int blocks = (K + fp_block(FORMAT) - 1) / fp_block(FORMAT);
    encode_row<FORMAT, CHUNKS>(X + m * K, K, K, wide, at.tid, at.nt, buf, outer ? outer + m : nullptr, [&](int k, int, uint32_t byte, const uint32_t (&c)[2], int field) {
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
                    r.w[4 * h + i] = FORMAT == MOQE_FP_MXFP4 ? bf16_pair(v[2 * i] * s, v[2 * i + 1] * s) : bf16_pair(v[2 * i] * s * o, v[2 * i + 1] * s * o);
            }
            store32(values + m * K + k, (K - k) * 2, wide, r);
        }
    });
}

template <int FORMAT, int CHUNKS>
__device__ __forceinline__ void pack_row(const __nv_bfloat16* row, int K, bool wide, const RowPlace& at, const PackedRow& out, float* outer, uint32_t* buf) {
    const int padded = fp_kblocks(K, FORMAT) * 256;
    const PackedLane to = packed_lane<FORMAT>(out, at.tid, at.nt);
    encode_row<FORMAT, CHUNKS>(row, K, padded, wide, at.tid, at.nt, buf, outer,
                               [&](int k, int chunk, uint32_t byte, const uint32_t (&c)[2], int) { put_packed<FORMAT>(to, chunk, k < padded, byte, c); });
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

// Where the row at place j of the sorted order goes: its expert's segment, which starts at a multiple of 16 rows.  Every lane holds an
// expert's part of the offset table.
struct TokenSegments {
    int lo, hi, pad, pad0, blk0;
    TokenTiles tiles;
    __device__ __forceinline__ void load(const TokenParams& p, int lane) {
        const bool is = lane < p.E;
        lo = is ? p.offsets[lane] : 0x7FFFFFFF;
        hi = is ? p.offsets[lane + 1] : 0x7FFFFFFF;
        const int n = hi - lo;
        tiles = token_tiles(n, p.t.TN);
        pad = (n + 15) & ~15;
        const int blocks = tiles.tiles * (p.t.TN > 128 ? 2 : 1);
        pad0 = pad;
        blk0 = blocks;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int a = __shfl_up_sync(0xFFFFFFFFu, pad0, d), b = __shfl_up_sync(0xFFFFFFFFu, blk0, d);
            if (lane >= d) { pad0 += a; blk0 += b; }
        }
        pad0 -= pad;
        blk0 -= blocks;
    }
    // (all lanes of a warp; false: nobody's)
    __device__ __forceinline__ bool place(const TokenParams& p, int j, int& format, PackedRow& out, float*& outer) const {
        const uint32_t mine = __ballot_sync(0xFFFFFFFFu, j >= lo && j < hi);
        if (mine == 0) return false;
        const int e = __ffs(mine) - 1, i = j - __shfl_sync(0xFFFFFFFFu, lo, e);
        const size_t row0 = __shfl_sync(0xFFFFFFFFu, pad0, e), block0 = __shfl_sync(0xFFFFFFFFu, blk0, e);
        const TokenTiles t = {__shfl_sync(0xFFFFFFFFu, tiles.tiles, e), __shfl_sync(0xFFFFFFFFu, tiles.rows, e)};
        format = p.formats.format[e];
        out = token_row(p.t.codes + row0 * p.t.row_bytes, p.t.sf + block0 * p.t.block_sf, format, i, __shfl_sync(0xFFFFFFFFu, pad, e), t, p.t.TN);
        outer = p.t.outer + row0 + i;
        return true;
    }
};

// Few rows, or very long ones: a block, or one warp of it, a place j.  (The other kernel, which comes to its first row later but to the
// next ones sooner, takes over at 9 million numbers.  Both with a product of 1024 channels in MXFP4 behind them, rows not in L2, this
// kernel / the other, us: 1953 rows of 512 k 10.1 / 10.5, 976 x 1024 8.8 / 9.4, 488 x 4096 11.7 / 12.0; 18554 x 512 31.0 / 28.0, 4638 x 2048
// 21.5 / 20.6, 2319 x 4096 21.2 / 19.5, 501 x 18944 30.1 / 25.1.  They really cross at 4 to 6 million, for the longest rows at 2, so that
// between there and 9 million this kernel is the slower one: 16384 x 512 29.3 / 26.2, 1025 x 8192 23.5 / 22.1, 443 x 18944 27.7 / 23.7 (NVFP4
// 31.8 / 25.4), 105 x 18944 19.6 / 17.8.)
__global__ void fp_tokens_kernel(const __grid_constant__ TokenParams p) {
    __shared__ uint32_t buf[32];
    // the product behind this kernel may read the offset table before this kernel has ended, so nothing is let go before the wait
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const RowPlace at = row_place(p.warps);
    const int j = at.row, lane = threadIdx.x & 31;
    for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < p.n_counters; i += gridDim.x * blockDim.x) p.counters[i] = 0;
    if (j >= p.M) return;
    const int from = p.perm[j];
    TokenSegments seg;
    seg.load(p, lane);
    int format;
    PackedRow out;
    float* outer;
    if (!seg.place(p, j, format, out, outer)) return;
    const __nv_bfloat16* row = p.X + (size_t)from * p.K;
    if (format == MOQE_FP_MXFP4) pack_row<MOQE_FP_MXFP4, 2>(row, p.K, p.wide, at, out, nullptr, buf);
    else if (format == MOQE_FP_NVFP4) pack_row<MOQE_FP_NVFP4, 2>(row, p.K, p.wide, at, out, outer, buf);
    else {
        const int KB = fp_kblocks(p.K, format);
        for (int c0 = at.tid; c0 < KB * 4; c0 += at.nt * 2) {
            RawBf16 raw[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) load16(row, (c0 + i * at.nt) * 16, p.K, p.wide, raw[i]);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int c = 2 * (c0 + i * at.nt);
                const uint32_t* w = raw[i].r.w;
                if (c >= KB * 8) break;
                *reinterpret_cast<uint4*>(out.chunk(c >> 3, c & 7)) = make_uint4(w[0], w[1], w[2], w[3]);
                *reinterpret_cast<uint4*>(out.chunk(c >> 3, (c & 7) + 1)) = make_uint4(w[4], w[5], w[6], w[7]);
            }
        }
    }
}

// 16 numbers of a row in shared memory, zeros behind its end
__device__ __forceinline__ void read16(const unsigned char* row, int k, int K, RawBf16& raw) {
    const uint4 z = make_uint4(0, 0, 0, 0), *q = reinterpret_cast<const uint4*>(row + k * 2);
    const uint4 a = k < K ? q[0] : z, b = k + 8 < K ? q[1] : z;
    raw.r.w[0] = a.x; raw.r.w[1] = a.y; raw.r.w[2] = a.z; raw.r.w[3] = a.w;
    raw.r.w[4] = b.x; raw.r.w[5] = b.y; raw.r.w[6] = b.z; raw.r.w[7] = b.w;
}
// A token row in shared memory into its place, by the whole block.
template <int FORMAT>
__device__ __forceinline__ void pack_ring_row(const unsigned char* row, int K, const PackedRow& out, float* outer, uint32_t* buf) {
    const int tid = threadIdx.x, nt = blockDim.x, lane = tid & 31, padded = fp_kblocks(K, FORMAT) * fp_kbk(FORMAT);
    int field = 127;
    if constexpr (FORMAT == MOQE_FP_NVFP4) {
        uint32_t two = 0;
        for (int k = tid * 8; k < K; k += nt * 8) {
            const uint4 v = *reinterpret_cast<const uint4*>(row + k * 2);
            two = max_abs_bf16x2(max_abs_bf16x2(max_abs_bf16x2(max_abs_bf16x2(two, v.x), v.y), v.z), v.w);
        }
        uint32_t m = __float_as_uint(larger_half(two));
        if (m >= 0x7F800000u) {                                // (infinities and NaN do not count)
            m = 0;
            for (int k = tid * 8; k < K; k += nt * 8)
                for (int i = 0; i < 8; ++i) {
                    const uint32_t b = (uint32_t)(*reinterpret_cast<const uint16_t*>(row + (k + i) * 2) & 0x7FFFu) << 16;
                    m = max(m, b < 0x7F800000u ? b : 0u);
                }
        }
        field = nv_row_field(block_max(m, buf));
        if (tid == 0) *outer = pow2_field(field);
    }
    const PackedLane to = packed_lane<FORMAT>(out, tid, nt);
#pragma unroll 1
    for (int k = tid * 16, chunk = 0; k - lane * 16 < padded; k += nt * 16, ++chunk) {
        RawBf16 raw;
        read16(row, k, K, raw);
        if constexpr (FORMAT == MOQE_FP_BF16) {
            if (k >= padded) continue;
            const uint32_t* w = raw.r.w;
            *reinterpret_cast<uint4*>(out.chunk(k >> 6, (k >> 3) & 7)) = make_uint4(w[0], w[1], w[2], w[3]);
            *reinterpret_cast<uint4*>(out.chunk(k >> 6, ((k >> 3) & 7) + 1)) = make_uint4(w[4], w[5], w[6], w[7]);
        } else {
            float x[16];
            widen(raw, x);
            float a = FORMAT == MOQE_FP_NVFP4 ? raw_amax(raw) : amax16(x);
            uint32_t codes[2];
            if constexpr (FORMAT == MOQE_FP_MXFP4) { const float b = __shfl_xor_sync(0xFFFFFFFFu, a, 1); a = max_abs3(a, b, b); }
            const uint32_t byte = encode16<FORMAT, false>(x, a, field, codes);
            put_packed<FORMAT>(to, chunk, k < padded, byte, codes);
        }
    }
}
// Many rows: as many blocks as there is room for, each with a ring of rows that bulk copies bring to shared memory, a place after
// another.  A block that takes its row from global memory has its loads under way in the L1 cache, of which next to nothing is left
// on an SM set up for the product's shared memory, and this kernel's first blocks run beside the last of a product (4160 rows of 18944 k in
// NVFP4 with a product behind them 104 -> 86 us; alone 64 -> 53).  What is left is instructions: two thirds of the issue slots, 250 for 32 x 16
// numbers, of which a row's own cost 50.  16384 rows of 4096 k: MXFP4 36 us, NVFP4 47, for 26 of HBM.
constexpr int RING_MAX_STAGES = 4, RING_MAX_K = 32768;     // (two rows of 64 KB)
__global__ void __maxnreg__(64) fp_tokens_ring_kernel(const __grid_constant__ TokenParams p, int stages, int stride, int* status) {
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ uint32_t buf[32];
    __shared__ unsigned long long full[RING_MAX_STAGES];
    __shared__ int aborted;
    const int lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < stages; ++i) mbar_init(smem_u32(full) + 8 * i, 1);
        aborted = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    // (as above)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int end = p.offsets[p.E], bytes = p.K * 2, step = gridDim.x;
    int j = p.offsets[0] + blockIdx.x;
    auto fetch = [&](int place, int from, int stage) {         // (one thread)
        if (place >= end) return;
        mbar_expect_tx(smem_u32(full) + 8 * stage, bytes);
        bulk_load(smem_u32(ring) + stage * stride, p.X + (size_t)from * p.K, bytes, smem_u32(full) + 8 * stage);
    };
    int from = 0;                                               // of the next row to fetch
    if (threadIdx.x == 0) {
        int first[RING_MAX_STAGES];
#pragma unroll
        for (int i = 0; i < RING_MAX_STAGES; ++i) first[i] = j + i * step < end ? p.perm[j + i * step] : 0;
        if (j + stages * step < end) from = p.perm[j + stages * step];
#pragma unroll
        for (int i = 0; i < RING_MAX_STAGES; ++i)
            if (i < stages) fetch(j + i * step, first[i], i);
    }
    for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < p.n_counters; i += gridDim.x * blockDim.x) p.counters[i] = 0;
    TokenSegments seg;
    seg.load(p, lane);
    bool ok = true;
    for (int stage = 0, phase = 0; j < end; j += step) {
        int format;
        PackedRow out;
        float* outer;
        const bool have = seg.place(p, j, format, out, outer);
        ok = mbar_wait_short(smem_u32(full) + 8 * stage, phase, &aborted, status);
        const unsigned char* row = ring + stage * stride;
        if (have) {
            if (format == MOQE_FP_MXFP4) pack_ring_row<MOQE_FP_MXFP4>(row, p.K, out, outer, buf);
            else if (format == MOQE_FP_NVFP4) pack_ring_row<MOQE_FP_NVFP4>(row, p.K, out, outer, buf);
            else pack_ring_row<MOQE_FP_BF16>(row, p.K, out, outer, buf);
        }
        if (!(ok = __syncthreads_and(ok))) break;               // the row has been read: its stage may be filled again
        if (threadIdx.x == 0) {
            fetch(j + stages * step, from, stage);
            if (j + (stages + 1) * step < end) from = p.perm[j + (stages + 1) * step];
        }
        if (++stage == stages) { stage = 0; phase ^= 1; }
    }
    if (!ok) {                                                  // (copies under way land first)
        const unsigned long long t0 = global_ns();
        while (global_ns() - t0 < 200000ull) __nanosleep(1000);
        __syncthreads();
    }
}

// Four chunks to a thread from 1024 rows on.  Two / four, with values, rows not in L2, us.  NVFP4: 16384 x 11008 175 / 130, 4096 x 18944
// 86 / 62, 1024 x 11008 12.6 / 11.4; 16 x 4096 2.3 / 3.2, 512 x 4096 3.9 / 4.7.  What short rows pay: 1024 x 4096 5.2 / 6.5, 2048 x 4096 8.2 / 8.8, 16384
// x 512 9.2 / 11.0.  MXFP4 gains from 18944 k only (4096 rows 62 / 57; 16384 x 11008 124 / 125) and pays up to 14 % below (1024 x 4096 4.6 / 5.2).
int row_chunks(int M) { return M < 1024 ? 2 : 4; }

}  // namespace

moqe_status launch_fp_tokens(const void* X, const int32_t* perm, const int32_t* offsets, int M, int K, int E, const FpExperts& formats,
                             const FpTokens& tokens, uint32_t* counters, int n_counters, cudaStream_t st) {
    const bool wide = K % 16 == 0 && (uintptr_t)X % 32 == 0;
    TokenParams p = {(const __nv_bfloat16*)X, perm, offsets, M, K, E, wide, row_threads(K, 2) == 32, tokens, counters, n_counters, formats};
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at; cfg.numAttrs = 1; cfg.stream = st;
    const int stride = (K * 2 + 127) / 128 * 128, stages = K <= 2048 ? 4 : 2;
    cudaError_t err;
    if ((long long)M * K < 9000000 || K > RING_MAX_K) {
        const RowLaunch l = row_launch(M, K, 2);
        cfg.gridDim = dim3(l.blocks); cfg.blockDim = dim3(l.threads);
        err = cudaLaunchKernelEx(&cfg, fp_tokens_kernel, p);
    } else {
        static std::atomic<unsigned long long> attr{0};
        if (!ensure_dynamic_smem((const void*)fp_tokens_ring_kernel, RING_MAX_K * 4, attr)) { cudaGetLastError(); return MOQE_ERR_CUDA; }
        int* status = device_status_word();
        if (!status) return MOQE_ERR_ALLOC;
        const int threads = row_threads(K, 4), by_threads = 1024 / threads, by_smem = 228 * 1024 / (stages * stride + 1344), each = by_threads < by_smem ? by_threads : by_smem;
        const int room = device_sm_count() * (each > 32 ? 32 : each);
        cfg.gridDim = dim3(M < room ? M : room); cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = stages * stride;
        err = cudaLaunchKernelEx(&cfg, fp_tokens_ring_kernel, p, stages, stride, status);
    }
    if (err != cudaSuccess) { cudaGetLastError(); return MOQE_ERR_CUDA; }
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
