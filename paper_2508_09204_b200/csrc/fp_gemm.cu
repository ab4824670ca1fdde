// Routed product of floating-point experts: grouped by expert, ragged, any mixture of MXFP4, NVFP4 and bf16 in one call.
//
//   Y[perm[j]][n] = bf16( o_x[j] o_w[n] sum_k x[j][k] w_e[n][k] ),  e = the expert whose segment holds j
//
// 128 channels are the rows of an MMA (TMEM lanes), up to 128 tokens its columns, so that single tokens and prompts are the same
// code: only the columns shrink.  The tensor cores multiply the 4-bit codes and their block scales as they are
// (tcgen05.mma kind::mxf4nvf4, 64 k to an instruction); bf16 experts use kind::f16 with 16 k.  Either way an instruction takes
// 32 bytes of a row, so a k-block of 128 bytes a row is four instructions of about the same duration, whatever the format, and is
// the unit that work is split by.
//
// One CTA to an SM.  Warp 4 (one lane) fills a ring of stages with bulk copies (weights with their scales: one copy; token rows:
// one; their scales: one), warp 5 (one elected lane) copies scales to tensor memory and issues the MMAs into one of two
// accumulators, warps 0-3 read the other one, a thread a channel, scale, round and store.  Work: whole tiles dealt out in turn where
// there are plenty; else the tiles' k-blocks in one sequence, an equal share to every CTA ("stream-K").  A warp that holds part
// of a tile parks its fp32 sums and counts itself in; the last one adds them up in the order of the CTAs, so that a call gives
// the same bits every time.  Nobody waits for another CTA.
//
// Every mbarrier wait is bounded; on expiry the CTA raises its abort flag, latches MOQE_ERR_TIMEOUT, lets copies in flight land,
// frees its tensor memory and returns.
#include "fp_formats.cuh"
#include "tc_ptx.cuh"

namespace moqe {
namespace {

constexpr int FP_TN = 128;                       // most tokens of a tile
constexpr int FP_THREADS = 192;
constexpr int FP_MAX_STAGES = 12;
constexpr int FP_RING_BYTES = 216 * 1024;
constexpr int FP_SMEM = FP_RING_BYTES + 1024;
constexpr int FP_SF_COLS = 32;                   // tensor-memory columns of a k-block's scales: weights' 16, tokens' 16
constexpr int FP_SF_COL0 = 2 * FP_TN;            // two of them behind the accumulators

struct FpGemmExpert { const uint8_t* tiles; const float* outer; int format, KB; };
struct FpGemmParams {
    FpGemmExpert ex[MOQE_MAX_EXPERTS];
    const int32_t *perm, *offsets;
    FpTokens t;
    uint32_t* counters;          // [CTA][warp], zero on entry
    float* partials;             // [CTA][2][TN][128]
    __nv_bfloat16* Y;
    int* status;
    int E, N, NT, TN;            // channel tiles; tokens of a tile
    int stages, stage_bytes, b_off, sfb_off;
};

struct FpSched {
    int off[MOQE_MAX_EXPERTS + 1], tile0[MOQE_MAX_EXPERTS + 1], unit0[MOQE_MAX_EXPERTS + 1];
    int KB[MOQE_MAX_EXPERTS], pad0[MOQE_MAX_EXPERTS];
    int E, G, split;             // G: CTAs that share the split
    uint32_t tmem;
    int abort;
};

// k-blocks [kb0, kb1) of channel tile nt of the tokens [i0, i0 + rows) of expert e
struct FpPiece { int e, nt, i0, rows, kb0, kb1, KB; };

// what one CTA does, piece after piece; every role walks it for itself
struct FpWalk {
    int e, t, u, ue;
    __device__ __forceinline__ void start(const FpSched& s) {
        e = 0;
        const int c = blockIdx.x, U = s.unit0[s.E];
        t = c;
        u = ue = 0;
        if (s.split && c < s.G) { u = (int)((long long)c * U / s.G); ue = (int)((long long)(c + 1) * U / s.G); }
    }
    __device__ __forceinline__ bool next(const FpSched& s, const FpGemmParams& p, FpPiece& pc) {
        int tile;
        if (s.split) {
            if (u >= ue) return false;
            while (u >= s.unit0[e + 1]) ++e;
            const int v = u - s.unit0[e], KB = s.KB[e];
            tile = v / KB;
            pc.kb0 = v - tile * KB;
            pc.kb1 = min(KB, pc.kb0 + ue - u);
            u += pc.kb1 - pc.kb0;
        } else {
            if (t >= s.tile0[s.E]) return false;
            while (t >= s.tile0[e + 1]) ++e;
            tile = t - s.tile0[e];
            pc.kb0 = 0;
            pc.kb1 = s.KB[e];
            t += gridDim.x;
        }
        const int tt = tile / p.NT;
        pc.e = e;
        pc.KB = s.KB[e];
        pc.nt = tile - tt * p.NT;
        pc.i0 = tt * p.TN;
        pc.rows = min(p.TN, s.off[e + 1] - s.off[e] - pc.i0);
        return true;
    }
};

// ---------------------------------------------------------------------------- PTX of the block-scaled forms
// 128 rows x 4 scales, 512 bytes of shared memory, to four columns of tensor memory (32 lanes, repeated for every quarter)
__device__ __forceinline__ void tmem_copy_scales(uint32_t taddr, uint32_t smem_addr) {
    const uint64_t desc = (uint64_t)((smem_addr >> 4) & 0x3FFFu) | (8ull << 32) | (1ull << 46);    // rows of 16 bytes, eight to 128 bytes
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
template <int FORMAT>
__device__ __forceinline__ void umma_fp4(uint32_t d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
    if constexpr (FORMAT == MOQE_FP_MXFP4)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
            ::"r"(d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
            ::"r"(d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
}
// e2m1 x e2m1 -> fp32, both K-major, M = 128, N = n; scales E8M0 (bit 23) or e4m3; `id`: which of a column's four scales come first
__device__ __forceinline__ uint32_t idesc_fp4(int n, bool e8m0, uint32_t id) {
    return (id << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)e8m0 << 23) | ((128u >> 4) << 24) | (id << 29);
}

// the MMAs of one k-block; sf: its tensor-memory columns
template <int FORMAT>
__device__ __forceinline__ void issue_kblock(uint32_t d, uint32_t a, uint32_t sfa, uint32_t b, uint32_t sfb, uint32_t sf, int n, int steps, bool first) {
    const uint64_t ad = umma_desc_sw128(a), bd = umma_desc_sw128(b);
    if constexpr (FORMAT == MOQE_FP_BF16) {
        const uint32_t id = umma_idesc(n);
#pragma unroll
        for (int s = 0; s < 4; ++s)
            if (s < steps) umma_bf16(d, ad + 2 * s, bd + 2 * s, id, first && s == 0 ? 0u : 1u);
    } else {
        constexpr int GROUPS = FORMAT == MOQE_FP_MXFP4 ? 2 : 4;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            tmem_copy_scales(sf + 4 * g, sfa + 512 * g);
            tmem_copy_scales(sf + 16 + 4 * g, sfb + 512 * g);
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int g = FORMAT == MOQE_FP_MXFP4 ? s >> 1 : s;
            const uint32_t id = idesc_fp4(n, FORMAT == MOQE_FP_MXFP4, FORMAT == MOQE_FP_MXFP4 ? (s & 1) * 2 : 0);
            if (s < steps) umma_fp4<FORMAT>(d, ad + 2 * s, bd + 2 * s, id, sf + 4 * g, sf + 16 + 4 * g, first && s == 0 ? 0u : 1u);
        }
    }
}

__device__ __forceinline__ uint32_t count_in(uint32_t* p) {
    uint32_t old;
    asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(old) : "l"(p) : "memory");
    return old;
}

// 32 tokens' sums of this lane's channel -> Y.  Lanes of a pair swap halves, so that each stores two channels of every other token.
// (N is even and the pair's first channel n & ~1 too.)
__device__ __forceinline__ void store_columns(const FpGemmParams& p, const float (&v)[32], int to, int cols, int n, int lane) {
    const int odd = lane & 1;
    __nv_bfloat16* y = p.Y + (n & ~1);
#pragma unroll
    for (int c = 0; c < 32; c += 2) {
        const float give = odd ? v[c] : v[c + 1], keep = odd ? v[c + 1] : v[c];
        const float got = __shfl_xor_sync(0xFFFFFFFFu, give, 1);
        const int row = __shfl_sync(0xFFFFFFFFu, to, c + odd);
        const __nv_bfloat162 h = odd ? __floats2bfloat162_rn(got, keep) : __floats2bfloat162_rn(keep, got);
        if (c + odd < cols && n < p.N) *reinterpret_cast<__nv_bfloat162*>(y + (size_t)row * p.N) = h;
    }
}

__global__ void __launch_bounds__(FP_THREADS, 1) fp_gemm_kernel(const __grid_constant__ FpGemmParams p) {
    extern __shared__ unsigned char smem_raw[];
    __shared__ FpSched sh;
    __shared__ unsigned long long bars[2 * FP_MAX_STAGES + 4];
    const uint32_t ring0 = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t bar_full = smem_u32(bars), bar_empty = bar_full + 8 * FP_MAX_STAGES;
    const uint32_t bar_accfull = bar_empty + 8 * FP_MAX_STAGES, bar_accempty = bar_accfull + 16;

    if (threadIdx.x == 0) {
        for (int i = 0; i < p.stages; ++i) { mbar_init(bar_full + 8 * i, 1); mbar_init(bar_empty + 8 * i, 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(bar_accfull + 8 * i, 1); mbar_init(bar_accempty + 8 * i, 128); }
        sh.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 5) tmem_alloc(smem_u32(&sh.tmem), 512);
    if (warp == 4) {
        // the schedule, from the sort's offset table (the kernel before this one waited for it before it let this one start)
        const bool is = lane < p.E;
        const int lo = is ? __ldcg(p.offsets + lane) : 0, hi = is ? __ldcg(p.offsets + lane + 1) : 0;
        const int rows = hi - lo, KB = is ? p.ex[lane].KB : 1;
        const int tiles = (rows + p.TN - 1) / p.TN * p.NT;
        int pad = (rows + 127) & ~127, tsum = tiles, usum = tiles * KB, psum = pad;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int a = __shfl_up_sync(0xFFFFFFFFu, tsum, d), b = __shfl_up_sync(0xFFFFFFFFu, usum, d), c = __shfl_up_sync(0xFFFFFFFFu, psum, d);
            if (lane >= d) { tsum += a; usum += b; psum += c; }
        }
        if (is) {
            sh.off[lane] = lo; sh.KB[lane] = KB; sh.pad0[lane] = psum - pad;
            sh.tile0[lane] = tsum - tiles; sh.unit0[lane] = usum - tiles * KB;
            if (lane == p.E - 1) { sh.off[p.E] = hi; sh.tile0[p.E] = tsum; sh.unit0[p.E] = usum; }
        }
        const int T = __shfl_sync(0xFFFFFFFFu, tsum, 31), U = __shfl_sync(0xFFFFFFFFu, usum, 31);
        if (lane == 0) {
            sh.E = p.E;
            sh.split = T < 2 * (int)gridDim.x;
            sh.G = max(1, min((int)gridDim.x, U / 4));
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem;

    if (warp == 4) {
        // ---------------- producer ----------------
        if (lane == 0) {
            FpWalk walk;
            FpPiece pc;
            Ring ring;
            bool ok = true;
            // The weights of the first stages are fetched while the kernel before is still writing the token rows.
            auto weights = [&](const FpPiece& q, int kb, int st) {
                const int format = p.ex[q.e].format, sfb = fp_sf_bytes(format), n16 = (q.rows + 15) & ~15;
                const int stride = fp_tile_stride(format);
                const uint32_t full = bar_full + 8 * st;
                mbar_expect_tx(full, (uint32_t)(stride + n16 * 128 + sfb));
                bulk_load(ring0 + st * p.stage_bytes, p.ex[q.e].tiles + ((size_t)q.nt * q.KB + kb) * stride, stride, full);
            };
            auto tokens = [&](const FpPiece& q, int kb, int st) {
                const int format = p.ex[q.e].format, sfb = fp_sf_bytes(format), n16 = (q.rows + 15) & ~15;
                const uint32_t full = bar_full + 8 * st, base = ring0 + st * p.stage_bytes;
                const size_t pad0 = sh.pad0[q.e];
                const int seg = (sh.off[q.e + 1] - sh.off[q.e] + 127) & ~127;
                const uint8_t* codes = p.t.codes + pad0 * p.t.row_bytes + ((size_t)kb * seg + q.i0) * 128;
                bulk_load(base + p.b_off, codes, n16 * 128, full);
                if (sfb) bulk_load(base + p.sfb_off, p.t.sf + (pad0 >> 7) * p.t.block_sf + ((size_t)(q.i0 >> 7) * q.KB + kb) * sfb, sfb, full);
            };
            walk.start(sh);
            int ahead = 0;
            while (ahead < p.stages && walk.next(sh, p, pc))
                for (int kb = pc.kb0; kb < pc.kb1 && ahead < p.stages; ++kb, ++ahead) weights(pc, kb, ahead);
            asm volatile("griddepcontrol.wait;" ::: "memory");
            asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
            asm volatile("fence.proxy.async;" ::: "memory");
            int done = 0;
            walk.start(sh);
            while (ok && walk.next(sh, p, pc)) {
                for (int kb = pc.kb0; kb < pc.kb1; ++kb, ++done) {
                    if (done >= ahead) {
                        if (!(ok = mbar_wait_short(bar_empty + 8 * ring.stage, ring.phase ^ 1u, &sh.abort, p.status))) break;
                        weights(pc, kb, ring.stage);
                    }
                    tokens(pc, kb, ring.stage);
                    ring.advance(p.stages);
                }
            }
        }
        __syncwarp();
    } else if (warp == 5) {
        // ---------------- MMA issuer: the whole warp walks, one elected lane issues ----------------
        FpWalk walk;
        FpPiece pc;
        Ring ring;
        bool ok = true;
        uint32_t uses = 0, kbs = 0;
        int last_stage = 0, last2_stage = 0;
        uint32_t last_phase = 0, last2_phase = 0;
        walk.start(sh);
        while (ok && walk.next(sh, p, pc)) {
            const int buf = uses & 1;
            const int format = p.ex[pc.e].format, n = (pc.rows + 15) & ~15;
            const uint32_t d = tmem + buf * FP_TN;
            if (!(ok = __all_sync(0xFFFFFFFFu, mbar_wait_short(bar_accempty + 8 * buf, ((uses >> 1) & 1u) ^ 1u, &sh.abort, p.status)))) break;
            for (int kb = pc.kb0; kb < pc.kb1; ++kb, ++kbs) {
                // The scales' columns alternate: those of two k-blocks ago must have been multiplied.
                if (format != MOQE_FP_BF16 && kbs >= 2) ok = mbar_wait_short(bar_empty + 8 * last2_stage, last2_phase, &sh.abort, p.status);
                ok = ok && mbar_wait_short(bar_full + 8 * ring.stage, ring.phase, &sh.abort, p.status);
                if (!(ok = __all_sync(0xFFFFFFFFu, ok))) break;
                tc_fence_after();
                const uint32_t a = ring0 + ring.stage * p.stage_bytes, b = a + p.b_off, sfb = a + p.sfb_off, sf = tmem + FP_SF_COL0 + (kbs & 1u) * FP_SF_COLS;
                if (elect_one()) {
                    if (format == MOQE_FP_MXFP4) issue_kblock<MOQE_FP_MXFP4>(d, a, a + 16384, b, sfb, sf, n, 4, kb == pc.kb0);
                    else if (format == MOQE_FP_NVFP4) issue_kblock<MOQE_FP_NVFP4>(d, a, a + 16384, b, sfb, sf, n, 4, kb == pc.kb0);
                    else issue_kblock<MOQE_FP_BF16>(d, a, 0, b, 0, 0, n, 4, kb == pc.kb0);
                    umma_commit(bar_empty + 8 * ring.stage);
                    if (kb + 1 == pc.kb1) umma_commit(bar_accfull + 8 * buf);
                }
                __syncwarp();
                last2_stage = last_stage; last2_phase = last_phase;
                last_stage = ring.stage; last_phase = ring.phase;
                ring.advance(p.stages);
            }
            ++uses;
        }
    } else {
        // ---------------- epilogue: thread = channel = TMEM lane ----------------
        asm volatile("griddepcontrol.wait;" ::: "memory");
        FpWalk walk;
        FpPiece pc;
        bool ok = true;
        uint32_t uses = 0;
        walk.start(sh);
        while (ok && walk.next(sh, p, pc)) {
            const int buf = uses & 1;
            const int j0 = sh.off[pc.e] + pc.i0, n = pc.nt * 128 + warp * 32 + lane;
            const float* ow = p.ex[pc.e].outer;
            const float* ox = p.t.outer + sh.pad0[pc.e] + pc.i0;
            const float w = ow ? ow[n] : 1.f;
            if (!(ok = __all_sync(0xFFFFFFFFu, mbar_wait_short(bar_accfull + 8 * buf, (uses >> 1) & 1u, &sh.abort, p.status)))) break;
            tc_fence_after();
            const uint32_t acc = tmem + ((uint32_t)(warp * 32) << 16) + buf * FP_TN;
            const bool whole = pc.kb0 == 0 && pc.kb1 == pc.KB;
            int c0 = blockIdx.x, c1 = blockIdx.x;
            bool finish = true;
            if (!whole) {
                // the CTAs that share this tile
                const long long U = sh.unit0[sh.E], G = sh.G;
                const long long first = walk.u - pc.kb1, last = first + pc.KB - 1;
                c0 = (int)(((first + 1) * G - 1) / U);
                c1 = (int)(((last + 1) * G - 1) / U);
                float* slot = p.partials + ((size_t)blockIdx.x * 2 + (pc.kb0 == 0 ? 1 : 0)) * p.TN * 128 + warp * 32 + lane;
                for (int c = 0; c < pc.rows; c += 32) {
                    uint32_t v[32];
                    tmem_ld32(acc + c, v);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (c + i < pc.rows) __stcg(slot + (c + i) * 128, __uint_as_float(v[i]));
                }
                __syncwarp();
                uint32_t old = 0;
                if (lane == 0) { __threadfence(); old = count_in(p.counters + c0 * 4 + warp); __threadfence(); }
                old = __shfl_sync(0xFFFFFFFFu, old, 0);
                finish = (int)old == c1 - c0;
            }
            if (finish) {
                for (int c = 0; c < pc.rows; c += 32) {
                    float f[32];
                    if (whole) {
                        uint32_t v[32];
                        tmem_ld32(acc + c, v);
                        tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < 32; ++i) f[i] = __uint_as_float(v[i]);
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i) f[i] = 0.f;
                        for (int q = c0; q <= c1; ++q) {
                            const float* slot = p.partials + ((size_t)q * 2 + (q == c0 ? 1 : 0)) * p.TN * 128 + warp * 32 + lane;
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                if (c + i < pc.rows) f[i] += __ldcg(slot + (c + i) * 128);
                        }
                    }
                    const int cols = pc.rows - c;
                    const int to = lane < cols ? p.perm[j0 + c + lane] : 0;
                    if (ow) {
                        const float x = lane < cols ? ox[c + lane] : 0.f;
#pragma unroll
                        for (int i = 0; i < 32; ++i) f[i] *= w * __shfl_sync(0xFFFFFFFFu, x, i);
                    }
                    store_columns(p, f, to, cols, n, lane);
                }
            }
            tc_fence_before();
            mbar_arrive(bar_accempty + 8 * buf);
            ++uses;
        }
    }

    // ---------------- teardown ----------------
    tc_fence_before();
    __syncthreads();
    if (sh.abort) {
        const unsigned long long t0 = global_ns();
        while (global_ns() - t0 < 200000ull) __nanosleep(1000);
        __syncthreads();
    }
    if (warp == 5) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

int tile_tokens(int M) { return M <= 16 ? 16 : M <= 32 ? 32 : M <= 64 ? 64 : 128; }

size_t al256(size_t x) { return (x + 255) / 256 * 256; }

struct FpLayout { size_t perm, offsets, sort, counters, codes, sf, outer, partials, total, row_bytes, block_sf; };

FpLayout fp_layout(int M, const moqe_fp_expert* const* ex, int E) {
    FpLayout w = {};
    for (int e = 0; e < E; ++e) {
        const size_t rb = (size_t)ex[e]->KB * 128, sb = (size_t)ex[e]->KB * fp_sf_bytes(ex[e]->format);
        w.row_bytes = rb > w.row_bytes ? rb : w.row_bytes;
        w.block_sf = sb > w.block_sf ? sb : w.block_sf;
    }
    // every expert's segment is filled up to 128 rows
    const size_t blocks = ((size_t)M + 127ull * (size_t)(M < E ? M : E)) / 128;
    size_t off = 0;
    w.perm = off;     off += al256((size_t)M * 4 + 16);
    w.offsets = off;  off += al256((MOQE_MAX_EXPERTS + 2) * 4);
    w.sort = off;     off += al256(sort_workspace_bytes(M, E));
    w.counters = off; off += al256((size_t)fp_gemm_counters() * 4);
    w.codes = off;    off += al256(blocks * 128 * w.row_bytes);
    w.sf = off;       off += al256(blocks * w.block_sf);
    w.outer = off;    off += al256(blocks * 128 * 4);
    w.partials = off; off += al256(fp_gemm_partial_bytes(M));
    w.total = off;
    return w;
}

moqe_status fp_args(const void* X, const void* rows, const void* offsets, int M, const moqe_fp_expert* const* ex, int E, const void* Y,
                    const void* workspace, size_t workspace_bytes, FpLayout& w) {
    if (!ex) return MOQE_ERR_NULL;
    if (E <= 0 || M < 0) return MOQE_ERR_SHAPE;
    if (E > MOQE_MAX_EXPERTS) return MOQE_ERR_UNSUPPORTED;
    for (int e = 0; e < E; ++e)
        if (!ex[e]) return MOQE_ERR_NULL;
    for (int e = 1; e < E; ++e)
        if (ex[e]->N != ex[0]->N || ex[e]->K != ex[0]->K) return MOQE_ERR_MISMATCH;
    if (M == 0) return MOQE_OK;
    if (!X || !rows || !offsets || !Y) return MOQE_ERR_NULL;
    if (ex[0]->N % 8 != 0 || (uintptr_t)X % 16 || (uintptr_t)Y % 16) return MOQE_ERR_UNSUPPORTED;
    w = fp_layout(M, ex, E);
    if (!workspace || workspace_bytes < w.total || (uintptr_t)workspace % 256) return MOQE_ERR_WORKSPACE;
    return MOQE_OK;
}

moqe_status fp_run(const void* X, const int32_t* perm, const int32_t* offsets, int M, const moqe_fp_expert* const* ex, int E, void* Y,
                   char* base, const FpLayout& w, cudaStream_t st) {
    FpTokens t = {(uint8_t*)base + w.codes, (uint8_t*)base + w.sf, (float*)(base + w.outer), w.row_bytes, w.block_sf};
    FpExperts formats;
    for (int e = 0; e < E; ++e) formats.format[e] = (uint8_t)ex[e]->format;
    uint32_t* counters = (uint32_t*)(base + w.counters);
    const moqe_status s = launch_fp_tokens(X, perm, offsets, M, ex[0]->K, E, formats, t, counters, fp_gemm_counters(), st);
    if (s != MOQE_OK) return s;
    return launch_fp_gemm(ex, E, M, perm, offsets, t, counters, base + w.partials, Y, st);
}

}  // namespace

int fp_gemm_counters() { return device_sm_count() * 4; }
size_t fp_gemm_partial_bytes(int M) { return (size_t)device_sm_count() * 2 * tile_tokens(M) * 128 * 4; }

moqe_status launch_fp_gemm(const moqe_fp_expert* const* ex, int E, int M, const int32_t* perm, const int32_t* offsets, const FpTokens& tokens,
                           uint32_t* counters, void* partials, void* Y, cudaStream_t st) {
    FpGemmParams p = {};
    int sf = 0;
    for (int e = 0; e < E; ++e) {
        p.ex[e] = {ex[e]->tiles, ex[e]->outer, ex[e]->format, ex[e]->KB};
        const int b = fp_sf_bytes(ex[e]->format);
        sf = b > sf ? b : sf;
    }
    p.perm = perm; p.offsets = offsets; p.t = tokens; p.counters = counters; p.partials = (float*)partials; p.Y = (__nv_bfloat16*)Y;
    p.status = device_status_word();
    if (!p.status) return MOQE_ERR_ALLOC;
    p.E = E; p.N = ex[0]->N; p.NT = ex[0]->Np / 128; p.TN = tile_tokens(M);
    // a stage: weights, their scales, token rows (from a multiple of 1024), their scales
    p.b_off = 16384 + sf;
    p.sfb_off = p.b_off + p.TN * 128;
    p.stage_bytes = (p.sfb_off + sf + 1023) & ~1023;
    p.stages = FP_RING_BYTES / p.stage_bytes;
    if (p.stages > FP_MAX_STAGES) p.stages = FP_MAX_STAGES;
    static std::atomic<unsigned long long> attr{0};
    if (!ensure_dynamic_smem((const void*)fp_gemm_kernel, FP_SMEM, attr)) { cudaGetLastError(); return MOQE_ERR_CUDA; }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(device_sm_count()); cfg.blockDim = dim3(FP_THREADS); cfg.dynamicSmemBytes = FP_SMEM; cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at; cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, fp_gemm_kernel, p) != cudaSuccess) { cudaGetLastError(); return MOQE_ERR_CUDA; }
    count_launch();
    return MOQE_OK;
}

}  // namespace moqe

using namespace moqe;

extern "C" size_t moqe_routed_fpgemm_workspace(int M, const moqe_fp_expert* const* h_experts, int E) {
    if (M < 0 || !h_experts || E <= 0 || E > MOQE_MAX_EXPERTS) return 0;
    for (int e = 0; e < E; ++e)
        if (!h_experts[e]) return 0;
    return fp_layout(M, h_experts, E).total;
}

extern "C" moqe_status moqe_routed_fpgemm_sorted(const void* X_bf16, const int32_t* perm, const int32_t* offsets, int M,
                                                 const moqe_fp_expert* const* h_experts, int E, void* Y_bf16, void* workspace,
                                                 size_t workspace_bytes, void* stream) {
    FpLayout w;
    const moqe_status s = fp_args(X_bf16, perm, offsets, M, h_experts, E, Y_bf16, workspace, workspace_bytes, w);
    if (s != MOQE_OK || M == 0) return s;
    return fp_run(X_bf16, perm, offsets, M, h_experts, E, Y_bf16, (char*)workspace, w, (cudaStream_t)stream);
}

extern "C" moqe_status moqe_routed_fpgemm(const void* X_bf16, const int32_t* row_ids, int M, const moqe_fp_expert* const* h_experts, int E,
                                          void* Y_bf16, void* workspace, size_t workspace_bytes, void* stream) {
    FpLayout w;
    moqe_status s = fp_args(X_bf16, row_ids, row_ids, M, h_experts, E, Y_bf16, workspace, workspace_bytes, w);
    if (s != MOQE_OK || M == 0) return s;
    char* base = (char*)workspace;
    int32_t *perm = (int32_t*)(base + w.perm), *offsets = (int32_t*)(base + w.offsets);
    s = launch_sort(row_ids, M, E, perm, offsets, base + w.sort, w.counters - w.sort, nullptr, 0, Y_bf16, h_experts[0]->N, (cudaStream_t)stream);
    if (s != MOQE_OK) return s;
    return fp_run(X_bf16, perm, offsets, M, h_experts, E, Y_bf16, base, w, (cudaStream_t)stream);
}
