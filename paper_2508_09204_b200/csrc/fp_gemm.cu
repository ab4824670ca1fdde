// Routed product of floating-point experts: grouped by expert, ragged, any mixture of MXFP4, NVFP4 and bf16 in one call.
//
//   Y[perm[j]][n] = bf16( o_x[j] o_w[n] sum_k x[j][k] w_e[n][k] ),  e = the expert whose segment holds j
//
// 128 channels (two SMs: 256) are the rows of an MMA (TMEM lanes), up to 128 (256) tokens its columns, so that a few tokens and prompts
// are the same code: only the columns shrink.  The tensor cores multiply the 4-bit codes and their block scales as they are
// (tcgen05.mma kind::mxf4nvf4, 64 k to an instruction); bf16 experts use kind::f16 with 16 k.  Either way an instruction takes
// 32 bytes of a row, so a k-block of 128 bytes a row is four instructions of about the same duration, whatever the format, and is
// the unit that work is split by.
//
// One CTA to an SM; a worker is a CTA or a pair.  Two warps (one lane each) fill a ring of stages with bulk copies: weights with their
// scales (one copy), which do not wait for the kernel that quantizes the rows; token rows and their scales (two).  One warp (one elected
// lane) copies scales to tensor memory and issues the MMAs into one of two accumulators; eight warps read the other one, 32 channels
// x twice 32 tokens each at a time, scale, round, turn them round with matrix stores and write 64 bytes a token.  Work: whole tiles
// dealt out in turn where there are plenty; else, and for what is left over, the tiles' k-blocks in one sequence, an equal share to
// every worker.  A warp that holds part of a tile parks its fp32 sums and counts itself in; the last one adds them up in the
// order of the workers, so that a call gives the same bits every time.  Nobody waits for another worker.
//
// Bound by HBM up to some 100 rows an expert (16 rows, 4096 -> 11008, three formats: 139.9 MB in 27.2 us with the kernel before it,
// 79 % of the copy rate), by the tensor cores beyond (8192 x 4096 x 4096: bf16 180 us, 1527 TFLOP/s; MXFP4 60.5 us, 4540; NVFP4 65.1 us,
// 4220).  A 4-bit k-block of a pair takes 512 cycles at the least; a turn of the issuing warp is about as long with NVFP4 (12
// copies of scales and 4 MMAs: 580 cycles), and the first k-blocks of a tile wait until half of the last accumulator has been read (1600
// of a tile's 9800 cycles at k = 4096).
//
// Every mbarrier wait is bounded; on expiry the CTA raises its abort flag, latches MOQE_ERR_TIMEOUT, lets copies in flight land,
// frees its tensor memory and returns.
#include "fp_formats.cuh"
#include "tc_ptx.cuh"

namespace moqe {
namespace {

// Of a k-block.  (16 rows x 4096 -> 11008, equal costs: bf16 tiles were done after 22, 4-bit ones after 27 us.  Whole calls with 4, 5 and 6 to
// 4: four experts 38.9, 35.6 and 35.3, three experts 28.8, 29.0 and 29.8; 40 x 11008 -> 4096, three 35.0, 33.0 and 33.6; 777 x 2056 -> 1000, four 19.1,
// 14.8 and 14.8; 4160 x 18944 -> 3584, two 286, 286 and 300, three 264, 273 and 272; others within 2 %.)
constexpr int FP_COST_4BIT = 5, FP_COST_BF16 = 4;
constexpr int FP_BAND = 8;                       // token tiles that are gone through together (see FpWalk)
constexpr int FP_EPI_WARPS = 8;
constexpr int FP_WEIGHTS_WARP = FP_EPI_WARPS, FP_MMA_WARP = FP_EPI_WARPS + 1, FP_TOKENS_WARP = FP_EPI_WARPS + 2;
constexpr int FP_THREADS = 32 * (FP_EPI_WARPS + 3);
constexpr int FP_MAX_STAGES = 8;
constexpr int FP_RING_BYTES = 200 * 1024;
constexpr int FP_BOX = 32 * 64;                  // 32 tokens x 32 channels of bf16, an epilogue warp's
constexpr int FP_SMEM = FP_RING_BYTES + FP_EPI_WARPS * FP_BOX + 1024;

// CG: SMs to a tile.  Tensor memory: two accumulators, then as many sets of scales as the ring has stages (a set: the weights'
// columns, four to 128 k (MXFP4) or 64 k (NVFP4), then the tokens', four or eight).  A pair's accumulators of 256 columns leave too
// little room for that: the second one begins half way through the first, and whoever reads an accumulator reads the shared half
// first; and there are two sets for NVFP4.
template <int CG> struct FpCfg {
    static constexpr int ACC1 = 128;                 // column of the second accumulator
    static constexpr int SF0 = 128 * (CG + 1);       // column of the scales
};

struct FpGemmExpert { const uint8_t* tiles; const float* outer; int format, KB; };
struct FpGemmParams {
    FpGemmExpert ex[MOQE_MAX_EXPERTS];
    const int32_t *perm, *offsets;
    FpTokens t;
    uint32_t* counters;          // [CTA][warp], zero on entry
    uint4* partials;             // [CTA][2][TN / 4][128]: four tokens' fp32 sums of a channel
    __nv_bfloat16* Y;
    int* status;
    int E, N, NT, TN;            // NT: tiles of 128 channels; TN: tokens of a tile
    int sf;                      // bytes of a tile's scales in a stage: the most of the call's formats
    int split_cost, least_share;     // what splitting costs, and the least share of a worker, in k-blocks
};

struct FpSched {
    // by place in the order of work: bf16 experts first, whose tiles are four times as deep, then the 4-bit ones
    int order[MOQE_MAX_EXPERTS], tile0[MOQE_MAX_EXPERTS + 1], unit0[MOQE_MAX_EXPERTS + 1], KB[MOQE_MAX_EXPERTS], cost[MOQE_MAX_EXPERTS], tts[MOQE_MAX_EXPERTS];
    int off[MOQE_MAX_EXPERTS + 1], pad0[MOQE_MAX_EXPERTS], blk0[MOQE_MAX_EXPERTS], rpt[MOQE_MAX_EXPERTS];      // by expert: rows, padded rows and blocks of scales before it, rows of a token tile
    int stages, stage_bytes, sfb_off;       // of the ring, which the largest token tile of the call decides
    int W, NT, all_deep;         // workers (CTAs or pairs); channel tiles of a worker; tiles of bf16 experts
    int deep, light;             // tiles dealt out whole: of bf16 experts; of 4-bit ones, behind all of those
    int late, extra;             // workers from `late` on, who have a deep tile less, have `extra` rounds of light ones before the others
    int u0, G, q, r, more;       // what costs from u0 on in shares for G workers: q G + r in equal ones, `more` for each from `late` on
    uint32_t tmem;
    int abort;
    // Where worker w's share begins (u0 and the end of everything for w = 0 and G): a k-block belongs to the share that its start
    // is in.
    __device__ __forceinline__ int cut(int w) const { return u0 + w * q + div_small(w * r, G) + max(0, w - late) * more; }
};

// k-blocks [kb0, kb1) of channel tile nt of the tokens [i0, i0 + rows) of expert e; at: its place in the order; tile: the expert's
struct FpPiece { int e, nt, tt, i0, rows, kb0, kb1, KB, at, tile; };

// tokens [i0, i0 + rows) and channel tile of an expert's tile: bands of FP_BAND token tiles, in a band channel tile by channel tile
__device__ __forceinline__ void place_tile(const FpSched& s, FpPiece& pc) {
    const int band = div_small(pc.tile, FP_BAND * s.NT), in = pc.tile - band * FP_BAND * s.NT, deep = min(FP_BAND, s.tts[pc.at] - band * FP_BAND);
    pc.e = s.order[pc.at];
    pc.nt = div_small(in, deep);
    pc.tt = band * FP_BAND + in - pc.nt * deep;
    pc.i0 = pc.tt * s.rpt[pc.e];
    pc.rows = min(s.rpt[pc.e], s.off[pc.e + 1] - s.off[pc.e] - pc.i0);
}

// What one worker does, piece after piece; every role walks it for itself.  Bands of tiles make the workers of a moment share both
// token and weight tiles in L2.  Whole tiles go to the workers in turn; the rest are one sequence of k-blocks, cut into shares of
// equal cost (a 4-bit k-block brings scales, and its tiles are short).
struct FpWalk {
    int at, w, phase, t, u, ue;
    __device__ __forceinline__ void start(const FpSched& s, int worker) {
        at = phase = 0;
        t = w = worker;
        u = ue = 0;
        if (w < s.G) { u = s.cut(w); ue = s.cut(w + 1); }
    }
    __device__ __forceinline__ bool next(const FpSched& s, const FpGemmParams& p, FpPiece& pc) {
        if (phase == 0 && t >= s.deep) { phase = 1; t = w >= s.late ? w - s.late : s.light; }
        if (phase == 1 && t >= min(s.light, s.extra * (s.W - s.late))) { phase = 2; t = s.extra * (s.W - s.late) + w; }
        if (phase == 2 && t >= s.light) phase = 3;
        if (phase < 3) {
            const int tile = phase == 0 ? t : s.all_deep + t;
            while (tile >= s.tile0[at + 1]) ++at;
            pc.tile = tile - s.tile0[at];
            pc.KB = s.KB[at];
            pc.kb0 = 0;
            pc.kb1 = pc.KB;
            t += phase == 1 ? s.W - s.late : s.W;
        } else {
            // (u, ue: in costs; the k-blocks that begin in [u, ue))
            int c, v, end;
            for (;;) {
                if (u >= ue) return false;
                while (u >= s.unit0[at + 1]) ++at;
                const int to = min(ue, s.unit0[at + 1]);
                c = s.cost[at];
                v = div_small(u - s.unit0[at] + c - 1, c);
                end = div_small(to - s.unit0[at] + c - 1, c);
                if (v < end) break;
                u = to;
            }
            pc.KB = s.KB[at];
            pc.tile = div_small(v, pc.KB);
            pc.kb0 = v - pc.tile * pc.KB;
            pc.kb1 = min(pc.KB, pc.kb0 + end - v);
            u = s.unit0[at] + (pc.tile * pc.KB + pc.kb1) * c;
        }
        pc.at = at;
        place_tile(s, pc);
        return true;
    }
};

// ---------------------------------------------------------------------------- PTX of the block-scaled and two-SM forms
template <int CG>
__device__ __forceinline__ void fp_tmem_alloc(uint32_t smem_dst) {
    if constexpr (CG == 1) tmem_alloc(smem_dst, 512);
    else {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_dst) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
}
template <int CG>
__device__ __forceinline__ void fp_tmem_dealloc(uint32_t taddr) {
    if constexpr (CG == 1) tmem_dealloc(taddr, 512);
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(taddr) : "memory");
}
// 128 rows x 4 scales, 512 bytes of shared memory, to four columns of tensor memory (32 lanes, repeated for every quarter); in both
// CTAs of a pair, each from its own shared memory
template <int CG>
__device__ __forceinline__ void tmem_copy_scales(uint32_t taddr, uint64_t desc) {
    if constexpr (CG == 1) asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
    else asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
#define MOQE_UMMA_FP4(GROUP, VEC)                                                                                              \
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"                                                             \
                 "tcgen05.mma.cta_group::" GROUP ".kind::mxf4nvf4.block_scale.scale_vec::" VEC " [%0], %1, %2, %3, [%4], [%5], p;\n\t}" \
                 ::"r"(d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory")
template <int CG, int FORMAT>
__device__ __forceinline__ void umma_fp4(uint32_t d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
    if constexpr (FORMAT == MOQE_FP_MXFP4) {
        if constexpr (CG == 1) MOQE_UMMA_FP4("1", "2X"); else MOQE_UMMA_FP4("2", "2X");
    } else {
        if constexpr (CG == 1) MOQE_UMMA_FP4("1", "4X"); else MOQE_UMMA_FP4("2", "4X");
    }
}
#undef MOQE_UMMA_FP4
template <int CG>
__device__ __forceinline__ void fp_umma_bf16(uint32_t d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    if constexpr (CG == 1) umma_bf16(d, adesc, bdesc, idesc, accumulate);
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
// arrives at the barrier (of both CTAs) when every MMA issued so far is done
template <int CG>
__device__ __forceinline__ void fp_commit(uint32_t bar) {
    if constexpr (CG == 1) umma_commit(bar);
    else {
        const uint16_t both = 3;
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"(both) : "memory");
    }
}
// e2m1 x e2m1 -> fp32, both K-major, M = 128 CG, N = n; scales E8M0 (bit 23) or e4m3; `id`: which of a column's four scales come first
template <int CG>
__device__ __forceinline__ uint32_t idesc_fp4(int n, bool e8m0, uint32_t id) {
    return (id << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)e8m0 << 23) | ((128u * CG >> 4) << 24) | (id << 29);
}
template <int CG>
__device__ __forceinline__ uint32_t idesc_bf16(int n) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((128u * CG >> 4) << 24);
}

// Two barriers' bounded wait: both tries are on their way before the first is looked at.
__device__ __forceinline__ bool mbar_wait_two(uint32_t bar0, uint32_t parity0, uint32_t bar1, uint32_t parity1, volatile int* abort_flag, int* status) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 q, [%3], %4;\n\t"
        "and.pred p, p, q;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(bar0), "r"(parity0), "r"(bar1), "r"(parity1) : "memory");
    if (ok) return true;
    bool got = mbar_wait_short(bar0, parity0, abort_flag, status);
    got &= mbar_wait_short(bar1, parity1, abort_flag, status);
    return got;
}

// The issuing warp's state, and the k-blocks of one piece.  A turn of the loop costs its instructions' latencies (waits, the elected
// lane's branch, operands moved to the uniform datapath), so it holds nothing that can be worked out before it.  One SM's tiles
// are small: two k-blocks to a turn there.  A pair multiplies 256 tokens in 512 cycles or more, and would rather have its stages back.
// A wait that runs out is looked at after the piece: what is issued until then stays in bounds, and no later wait takes long.
struct FpStages { int stages, bytes, b_off, sfb_off; };
struct FpIssue {
    Ring ring, last;             // the next stage; the last one (issued before it)
    Ring behind;                 // the stage whose k-block had the next set of scales
    int format, set, fresh;      // of the scales in tensor memory: their format, the next set of columns, sets that nobody has had yet
    bool ok;
};
template <int CG, int FORMAT>
__device__ __forceinline__ void issue_kblock(uint32_t d, uint32_t a, uint32_t b_off, uint32_t sfb_off, uint32_t sf, uint32_t id0, int n, bool first) {
    constexpr int GROUPS = FORMAT == MOQE_FP_MXFP4 ? 2 : 4;
    constexpr uint32_t GROUP = CG == 2 ? 8 : 4;                                             // columns of a group of the tokens' scales
    constexpr uint32_t SECOND = (2u << 4) | (2u << 29);                                     // the second pair of a column's scales
    const uint64_t ad = umma_desc_sw128(0) + (a >> 4), bd = ad + (b_off >> 4);
    if constexpr (FORMAT == MOQE_FP_BF16) {
#pragma unroll
        for (int s = 0; s < 4; ++s) fp_umma_bf16<CG>(d, ad + 2 * s, bd + 2 * s, id0, first && s == 0 ? 0u : 1u);
    } else {
        // scales: rows of 16 bytes, eight to 128 bytes
        const uint64_t sd = ((8ull << 32) | (1ull << 46)) + ((a + 16384) >> 4), td = ((8ull << 32) | (1ull << 46)) + ((a + sfb_off) >> 4);
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            tmem_copy_scales<CG>(sf + 4 * g, sd + 32 * g);
            tmem_copy_scales<CG>(sf + 4 * GROUPS + GROUP * g, td + 32 * g);
            if (CG == 2 && n > 128) tmem_copy_scales<CG>(sf + 4 * GROUPS + GROUP * g + 4, td + 32 * (GROUPS + g));
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int g = FORMAT == MOQE_FP_MXFP4 ? s >> 1 : s;
            umma_fp4<CG, FORMAT>(d, ad + 2 * s, bd + 2 * s, FORMAT == MOQE_FP_MXFP4 && (s & 1) ? id0 | SECOND : id0, sf + 4 * g,
                                 sf + 4 * GROUPS + GROUP * g, first && s == 0 ? 0u : 1u);
        }
    }
}
template <int CG, int FORMAT>
__device__ __forceinline__ void issue_piece(FpIssue& q, const FpGemmParams& p, const FpStages& st, uint32_t ring0, uint32_t bar_full, uint32_t bar_empty, uint32_t d,
                                            uint32_t sf0, int n, int kblocks, uint32_t accfull, volatile int* abort_flag) {
    constexpr uint32_t SET = (FORMAT == MOQE_FP_MXFP4 ? 2 : 4) * (CG == 2 ? 12 : 8);        // columns of a set
    // With as many sets as stages, a stage that has been filled again frees its set.  A pair has room for two of NVFP4's.
    constexpr bool SCARCE = CG == 2 && FORMAT == MOQE_FP_NVFP4;
    constexpr int TURN = CG == 2 ? 1 : 2;
    const int sets = SCARCE ? 2 : st.stages;
    const uint32_t id0 = FORMAT == MOQE_FP_BF16 ? idesc_bf16<CG>(n) : idesc_fp4<CG>(n, FORMAT == MOQE_FP_MXFP4, 0);
    if (FORMAT != MOQE_FP_BF16 && q.format != FORMAT) {
        // sets of another size, or none for a while: everything before must have been multiplied
        if (q.format != 0) q.ok &= mbar_wait_short(bar_empty + 8 * q.last.stage, q.last.phase, abort_flag, p.status);
        q.set = 0;
        q.fresh = sets;
        q.behind = q.ring;
    }
    q.format = FORMAT;
    for (int k = 0; k < kblocks; k += TURN) {
        const Ring r0 = q.ring;
        Ring r1 = r0;
        r1.advance(st.stages);
        const bool two = TURN == 2 && k + 1 < kblocks;
        const uint32_t full0 = bar_full + 8 * r0.stage, full1 = bar_full + 8 * r1.stage;
        if constexpr (SCARCE) {
            if (q.fresh > 0) --q.fresh;
            else { q.ok &= mbar_wait_short(bar_empty + 8 * q.behind.stage, q.behind.phase, abort_flag, p.status); q.behind.advance(st.stages); }
        }
        q.ok &= two ? mbar_wait_two(full0, r0.phase, full1, r1.phase, abort_flag, p.status) : mbar_wait_short(full0, r0.phase, abort_flag, p.status);
        __syncwarp();
        tc_fence_after();
        const uint32_t a0 = ring0 + r0.stage * st.bytes, a1 = ring0 + r1.stage * st.bytes;
        const int set1 = q.set + 1 >= sets ? 0 : q.set + 1;
        if (elect_one()) {
            issue_kblock<CG, FORMAT>(d, a0, st.b_off, st.sfb_off, sf0 + q.set * SET, id0, n, k == 0);
            fp_commit<CG>(bar_empty + 8 * r0.stage);
            if (two) {
                issue_kblock<CG, FORMAT>(d, a1, st.b_off, st.sfb_off, sf0 + set1 * SET, id0, n, false);
                fp_commit<CG>(bar_empty + 8 * r1.stage);
            }
            if (k + TURN >= kblocks) fp_commit<CG>(accfull);
        }
        __syncwarp();
        q.last = two ? r1 : r0;
        q.ring = q.last;
        q.ring.advance(st.stages);
        q.set = !two ? set1 : set1 + 1 == sets ? 0 : set1 + 1;
    }
}

__device__ __forceinline__ uint32_t count_in(uint32_t* p) {
    uint32_t old;
    asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(old) : "l"(p) : "memory");
    return old;
}
__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t of_leader(uint32_t addr) {       // the same place in the pair's first CTA
    uint32_t d;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(d) : "r"(addr));
    return d;
}
__device__ __forceinline__ void leader_arrive(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}

// An epilogue warp holds 32 channels x 32 tokens of sums as the 16-row shape of tensor-memory loads gives them: token block j (eight
// tokens), channel half h: v[16 h + 4 j + {0, 1}] = channel 16 h + lane / 4, tokens 8 j + 2 (lane % 4) + {0, 1}; + {2, 3}: channel + 8.
// So pairs of tokens are packed in a thread, and a transposing matrix store puts eight channels of a token side by side.
__device__ __forceinline__ void tmem_ld_16x256(uint32_t taddr, uint32_t* v) {
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
          "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(taddr) : "memory");
}
// Scaled (by channel, w, and token, x of token `lane`) and rounded: o[4 j + b] = tokens 8 j + 2 (lane % 4) + {0, 1} of channel 8 b + lane / 4.
__device__ __forceinline__ void pack_block(const uint32_t* v, bool scaled, const float (&w)[4], float x, int lane, uint32_t* o) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float x0 = 1.f, x1 = 1.f;
        if (scaled) { x0 = __shfl_sync(0xFFFFFFFFu, x, 8 * j + 2 * (lane & 3)); x1 = __shfl_sync(0xFFFFFFFFu, x, 8 * j + 2 * (lane & 3) + 1); }
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            float lo = __uint_as_float(v[16 * (b >> 1) + 4 * j + 2 * (b & 1)]), hi = __uint_as_float(v[16 * (b >> 1) + 4 * j + 2 * (b & 1) + 1]);
            if (scaled) { lo = lo * w[b] * x0; hi = hi * w[b] * x1; }
            o[4 * j + b] = bf16_pair(lo, hi);
        }
    }
}
// `cols` tokens of them -> Y, through the warp's box of shared memory (64 bytes a token; chunks permuted so that neither side has
// bank conflicts).  to: the row of Y of token `lane`; n0: the first channel.  (N is a multiple of 8, so a 16-byte chunk is there or not.)
__device__ __forceinline__ void store_block(const FpGemmParams& p, const uint32_t* o, uint32_t box, int to, int cols, int n0, int lane) {
    const uint32_t put = box + (lane & 7) * 64 + (((lane >> 3) ^ ((lane >> 1) & 3)) << 4);
#pragma unroll
    for (int j = 0; j < 4; ++j)
        asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};"
                     ::"r"(put + j * 512), "r"(o[4 * j]), "r"(o[4 * j + 1]), "r"(o[4 * j + 2]), "r"(o[4 * j + 3]) : "memory");
    __syncwarp();
    const int tok = lane >> 2, chunk = lane & 3, n = n0 + chunk * 8;
    const uint32_t get = box + tok * 64 + ((chunk ^ ((tok >> 1) & 3)) << 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint4 q;
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "r"(get + i * 512));
        const int row = __shfl_sync(0xFFFFFFFFu, to, tok + 8 * i);
        if (tok + 8 * i < cols && n < p.N) *reinterpret_cast<uint4*>(p.Y + (size_t)row * p.N + n) = q;
    }
    __syncwarp();
}

template <int CG>
__global__ void __launch_bounds__(FP_THREADS, 1) fp_gemm_kernel(const __grid_constant__ FpGemmParams p) {
    using L = FpCfg<CG>;
    extern __shared__ unsigned char smem_raw[];
    __shared__ FpSched sh;
    __shared__ unsigned long long bars[2 * FP_MAX_STAGES + 4];
    const uint32_t ring0 = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = CG == 2 ? cluster_rank() : 0u;
    const int worker = blockIdx.x / CG;
    const uint32_t bar_full = smem_u32(bars), bar_empty = bar_full + 8 * FP_MAX_STAGES;
    const uint32_t bar_accfull = bar_empty + 8 * FP_MAX_STAGES, bar_accempty = bar_accfull + 16;

    if (threadIdx.x == FP_WEIGHTS_WARP * 32) {
        // (weights and tokens arrive on their own; a pair's first CTA issues the MMAs: its full barriers take an arrival for the other CTA, too)
        for (int i = 0; i < FP_MAX_STAGES; ++i) { mbar_init(bar_full + 8 * i, CG == 2 && rank == 0 ? 3 : 2); mbar_init(bar_empty + 8 * i, 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(bar_accfull + 8 * i, 1); mbar_init(bar_accempty + 8 * i, FP_EPI_WARPS * CG); }
        sh.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == FP_MMA_WARP) fp_tmem_alloc<CG>(smem_u32(&sh.tmem));
    if (warp == FP_WEIGHTS_WARP) {
        // the schedule, from the sort's offset table (the kernel before this one waited for it before it let this one start)
        {
            const bool is = lane < p.E, deep = is && p.ex[lane].format == MOQE_FP_BF16;
            const int lo = is ? __ldcg(p.offsets + lane) : 0, hi = is ? __ldcg(p.offsets + lane + 1) : 0;
            const uint32_t bf = __ballot_sync(0xFFFFFFFFu, deep), four = __ballot_sync(0xFFFFFFFFu, is && !deep), below = (1u << lane) - 1u;
            const TokenTiles t = token_tiles(hi - lo, p.TN);
            const int pad = (hi - lo + 15) & ~15, most = __reduce_max_sync(0xFFFFFFFFu, t.tiles > 1 ? t.rows : pad), blocks = t.tiles * (p.TN > 128 ? 2 : 1);
            int psum = pad, bsum = blocks;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int c = __shfl_up_sync(0xFFFFFFFFu, psum, d), b = __shfl_up_sync(0xFFFFFFFFu, bsum, d);
                if (lane >= d) { psum += c; bsum += b; }
            }
            if (is) {
                sh.off[lane] = lo;
                sh.pad0[lane] = psum - pad;
                sh.blk0[lane] = bsum - blocks;
                sh.rpt[lane] = t.rows;
                if (lane == p.E - 1) {
                    sh.off[p.E] = hi;
                    // A stage: weights, their scales, token rows (from a multiple of 1024), their scales; as many as fit, and as there is
                    // room for sets of scales.  (Sized for 128 tokens where a call's largest tile has 48, 18944 channels x 3584 k of two
                    // formats take 21.8 instead of 20.8 us; 512 rows of three, 4096 x 4096, 28.6 for 25.1.)
                    const int at = 16384 + p.sf + most / CG * 128, bytes = (at + (most > 128 ? 2 : 1) * p.sf + 1023) & ~1023;
                    sh.sfb_off = at;
                    sh.stage_bytes = bytes;
                    sh.stages = min(FP_RING_BYTES / bytes, CG == 2 && p.sf ? 5 : 8);
                }
                sh.order[deep ? __popc(bf & below) : __popc(bf) + __popc(four & below)] = lane;
            }
        }
        __syncwarp();
        {
            const bool is = lane < p.E;
            const int e = is ? sh.order[lane] : 0, rows = is ? sh.off[e + 1] - sh.off[e] : 0, KB = is ? p.ex[e].KB : 1, NT = (p.NT + CG - 1) / CG;
            const int tts = token_tiles(rows, p.TN).tiles, tiles = tts * NT, cost = is && p.ex[e].format == MOQE_FP_BF16 ? FP_COST_BF16 : FP_COST_4BIT, units = tiles * KB * cost;
            int tsum = tiles, usum = units;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int a = __shfl_up_sync(0xFFFFFFFFu, tsum, d), b = __shfl_up_sync(0xFFFFFFFFu, usum, d);
                if (lane >= d) { tsum += a; usum += b; }
            }
            if (is) {
                sh.tile0[lane] = tsum - tiles; sh.unit0[lane] = usum - units; sh.KB[lane] = KB; sh.cost[lane] = cost; sh.tts[lane] = tts;
                if (lane == p.E - 1) { sh.tile0[p.E] = tsum; sh.unit0[p.E] = usum; }
            }
            // There are tiles of two costs: Tb deep ones (bf16) and Tl light ones.  Dealt out whole, their workers go through the same k
            // together and find half of what they need in L2; a worker without the last round's deep tile gets as many light ones
            // more as make up for it.  If that leaves too many without work, what does not fill a round of whole tiles, at least a
            // tile for each, is cut into shares that make up for a deep tile less (a pair's 18944 k, 70 bf16 and 210 4-bit tiles on
            // 74 workers: 303 us, 369 with shares of all but two rounds of 4-bit tiles).
            const bool is_deep = is && p.ex[e].format == MOQE_FP_BF16;
            const int T = __shfl_sync(0xFFFFFFFFu, tsum, 31), U = __shfl_sync(0xFFFFFFFFu, usum, 31), W = (int)gridDim.x / CG;
            const int Tb = __reduce_add_sync(0xFFFFFFFFu, is_deep ? tiles : 0), Tl = T - Tb, rb = div_small(Tb, W), b = Tb - rb * W, even = div_small(U, W);
            const int cb = __reduce_max_sync(0xFFFFFFFFu, is_deep && tiles ? KB * cost : 0), cl = __reduce_max_sync(0xFFFFFFFFu, is && !is_deep && tiles ? KB * cost : 0);
            const int split = p.split_cost * FP_COST_BF16;
            // all whole, `lane` rounds of light tiles for everybody: how many more for those without the last deep one, and how long it takes
            const int few = b ? (rb + 1) * cb : 0, short_of = max(0, Tl - lane * W), rounds = div_small(short_of + W - b - 1, W - b);
            const int takes = max(few + (b ? lane * cl : 0), rb * cb + (lane + rounds) * cl);
            const int best = __reduce_min_sync(0xFFFFFFFFu, takes), who = __ffs(__ballot_sync(0xFFFFFFFFu, takes == best)) - 1;
            const int extra_best = __shfl_sync(0xFFFFFFFFu, rounds, who);
            if (lane == 0) {
                int whole = 0, extra = 0, late = 0, more = 0, R = U, G;
                if (T > 0 && best <= even + split) { whole = T; extra = extra_best; late = b; R = 0; }
                for (int n = div_small(T, W); whole == 0 && n > 0; --n) {
                    const int deep = min(Tb, n * W), rest = U - deep * cb - (n * W - deep) * cl;
                    const bool uneven = deep < n * W && b > 0;                  // workers from b on have had a deep tile less
                    const int d = uneven ? cb - cl : 0;
                    if (rest >= W * (cl ? cl : cb) && rest - (W - b) * d >= W * 4 * FP_COST_4BIT) { whole = n * W; R = rest; late = uneven ? b : 0; extra = uneven; more = d; }
                }
                G = whole ? W : max(max(1, min(T, W)), min(W, div_small(R, p.least_share * FP_COST_BF16)));
                // few tiles, all alike: the same number of workers for each, so that nobody has the ends of two, if that is not much longer
                if (whole == 0 && T > 0 && (Tb == 0 || Tb == T) && T <= G && div_small(max(cb, cl), div_small(G, T)) <= div_small(R, G) + split) G = div_small(G, T) * T;
                if (R == 0) G = 0;
                sh.W = W; sh.NT = NT; sh.all_deep = Tb; sh.deep = min(Tb, whole); sh.light = whole - sh.deep; sh.late = late; sh.extra = extra; sh.more = more;
                sh.u0 = sh.deep * cb + sh.light * cl; sh.G = G;
                R -= max(0, G - late) * more;
                sh.q = G ? div_small(R, G) : 0; sh.r = G ? R - sh.q * G : 0;
            }
        }
    }
    // The weights' warp, which has set up all but tensor memory, goes ahead: it has nothing to do with the other CTA.
    tc_fence_before();
    __syncwarp();
    if (warp == FP_WEIGHTS_WARP) asm volatile("bar.arrive 1, %0;" ::"n"(FP_THREADS) : "memory");
    else asm volatile("bar.sync 1, %0;" ::"n"(FP_THREADS) : "memory");
    if constexpr (CG == 2) {
        asm volatile("barrier.cluster.arrive.release;" ::: "memory");
        if (warp != FP_WEIGHTS_WARP) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    }
    tc_fence_after();
    const uint32_t tmem = warp == FP_WEIGHTS_WARP ? 0u : sh.tmem;
    const FpStages st = {sh.stages, sh.stage_bytes, 16384 + p.sf, sh.sfb_off};

    if (warp == FP_WEIGHTS_WARP) {
        // ---------------- weights and their scales ----------------
        if (lane == 0) {
            FpWalk walk;
            FpPiece pc;
            Ring ring;
            bool ok = true;
            walk.start(sh, worker);
            while (ok && walk.next(sh, p, pc)) {
                const FpGemmExpert& x = p.ex[pc.e];
                const uint32_t stride = fp_tile_stride(x.format);
                const uint8_t* src = x.tiles + ((size_t)min(pc.nt * CG + (int)rank, p.NT - 1) * pc.KB + pc.kb0) * stride;
                for (int k = pc.kb1 - pc.kb0; k > 0; --k, src += stride) {
                    if (!(ok = mbar_wait_short(bar_empty + 8 * ring.stage, ring.phase ^ 1u, &sh.abort, p.status))) break;
                    mbar_expect_tx(bar_full + 8 * ring.stage, stride);
                    bulk_load(ring0 + ring.stage * st.bytes, src, stride, bar_full + 8 * ring.stage);
                    ring.advance(st.stages);
                }
            }
            // (the last stages are handed back by arrivals from the tensor cores, a pair's second CTA's from the first: they land here)
            for (int i = 0; ok && i < st.stages; ++i, ring.advance(st.stages)) ok = mbar_wait_short(bar_empty + 8 * ring.stage, ring.phase ^ 1u, &sh.abort, p.status);
        }
        __syncwarp();
        if constexpr (CG == 2) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    } else if (warp == FP_TOKENS_WARP) {
        // ---------------- token rows (of a pair, each CTA's half) and their scales ----------------
        if (lane == 0) {
            FpWalk walk;
            FpPiece pc;
            Ring ring;
            walk.start(sh, worker);
            bool ok = walk.next(sh, p, pc);
            asm volatile("griddepcontrol.wait;" ::: "memory");
            asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
            for (; ok; ok = ok && walk.next(sh, p, pc)) {
                const int sfb = fp_sf_bytes(p.ex[pc.e].format), n = (pc.rows + 15) & ~15, bpt = p.TN > 128 ? 2 : 1;
                const size_t pad0 = sh.pad0[pc.e], seg = (sh.off[pc.e + 1] - sh.off[pc.e] + 15) & ~15;
                const uint32_t bytes = n / CG * 128, sbytes = n > 128 ? 2 * sfb : sfb;
                const size_t step = seg * 128, sstep = (size_t)(sh.tts[pc.at] * bpt) * sfb;
                const uint8_t* src = p.t.codes + pad0 * p.t.row_bytes + pc.kb0 * step + (size_t)(pc.i0 + rank * (n / 2)) * 128;
                const uint8_t* ssrc = p.t.sf + sh.blk0[pc.e] * p.t.block_sf + pc.kb0 * sstep + (size_t)(pc.tt * bpt) * sfb;
                for (int k = pc.kb1 - pc.kb0; k > 0; --k, src += step, ssrc += sstep) {
                    if (!(ok = mbar_wait_short(bar_empty + 8 * ring.stage, ring.phase ^ 1u, &sh.abort, p.status))) break;
                    const uint32_t full = bar_full + 8 * ring.stage, base = ring0 + ring.stage * st.bytes;
                    mbar_expect_tx(full, bytes + sbytes);
                    bulk_load(base + st.b_off, src, bytes, full);
                    if (sbytes) bulk_load(base + st.sfb_off, ssrc, sbytes, full);
                    ring.advance(st.stages);
                }
            }
        }
        __syncwarp();
    } else if (warp == FP_MMA_WARP && rank == 0) {
        // ---------------- MMA issuer: the whole warp walks, one elected lane issues ----------------
        FpWalk walk;
        FpPiece pc;
        FpIssue q;
        q.format = 0; q.set = 0; q.fresh = 0; q.ok = true;
        uint32_t uses = 0;
        const uint32_t sf0 = tmem + L::SF0;
        walk.start(sh, worker);
        while (q.ok && walk.next(sh, p, pc)) {
            const int buf = uses & 1, format = p.ex[pc.e].format, n = (pc.rows + 15) & ~15;
            // one SM: the accumulator of two tiles ago has been read; a pair: what this one shares with the last has
            const uint32_t before = CG == 2 ? uses + 1 : uses, d = tmem + buf * L::ACC1, accfull = bar_accfull + 8 * buf;
            q.ok = mbar_wait_short(bar_accempty + 8 * (before & 1), ((before >> 1) & 1u) ^ 1u, &sh.abort, p.status);
            if (format == MOQE_FP_MXFP4) issue_piece<CG, MOQE_FP_MXFP4>(q, p, st, ring0, bar_full, bar_empty, d, sf0, n, pc.kb1 - pc.kb0, accfull, &sh.abort);
            else if (format == MOQE_FP_NVFP4) issue_piece<CG, MOQE_FP_NVFP4>(q, p, st, ring0, bar_full, bar_empty, d, sf0, n, pc.kb1 - pc.kb0, accfull, &sh.abort);
            else issue_piece<CG, MOQE_FP_BF16>(q, p, st, ring0, bar_full, bar_empty, d, sf0, n, pc.kb1 - pc.kb0, accfull, &sh.abort);
            q.ok = __all_sync(0xFFFFFFFFu, q.ok);
            ++uses;
        }
    } else if (warp == FP_MMA_WARP) {
        // ---------------- a pair's second CTA: tells the first when its half of a stage has landed ----------------
        if (lane == 0) {
            FpWalk walk;
            FpPiece pc;
            Ring ring;
            bool ok = true;
            const uint32_t to = of_leader(bar_full);
            walk.start(sh, worker);
            while (ok && walk.next(sh, p, pc)) {
                for (int kb = pc.kb0; kb < pc.kb1; ++kb) {
                    if (!(ok = mbar_wait_short(bar_full + 8 * ring.stage, ring.phase, &sh.abort, p.status))) break;
                    leader_arrive(to + 8 * ring.stage);
                    ring.advance(st.stages);
                }
            }
        }
        __syncwarp();
    } else {
        // ---------------- epilogue: two warps to a quarter of the channels (TMEM lanes), every other 32 tokens each ----------------
        asm volatile("griddepcontrol.wait;" ::: "memory");
        const int quarter = warp & 3, half = warp >> 2;
        const uint32_t box = ring0 + FP_RING_BYTES + warp * FP_BOX;
        const uint32_t accempty = CG == 2 ? of_leader(bar_accempty) : bar_accempty;
        FpWalk walk;
        FpPiece pc;
        bool ok = true;
        uint32_t uses = 0;
        int owed = 0, owed_at[2], owed_tile[2], owed_w[2];  // tiles that this warp has to add up (its worker shares two at most)
        walk.start(sh, worker);
        while (ok && walk.next(sh, p, pc)) {
            const int buf = uses & 1;
            const int j0 = sh.off[pc.e] + pc.i0, n0 = (pc.nt * CG + (int)rank) * 128 + quarter * 32;
            const float* ow = p.ex[pc.e].outer;
            const float* ox = p.t.outer + sh.pad0[pc.e] + pc.i0;
            float w[4];                                      // channel scales of this lane's rows
#pragma unroll
            for (int i = 0; i < 4; ++i) { const int n = n0 + (lane >> 2) + 8 * i; w[i] = ow && n < p.N ? ow[n] : 1.f; }
            // where this lane's share of the tokens goes, and their scales: fetched while the tile is multiplied
            int to[CG][2];
            float sx[CG][2];
#pragma unroll
            for (int g = 0; g < CG; ++g)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int c = g * 128 + h * 64 + half * 32 + lane;
                    to[g][h] = c < pc.rows ? p.perm[j0 + c] : 0;
                    sx[g][h] = ow && c < pc.rows ? ox[c] : 1.f;
                }
            if (!(ok = __all_sync(0xFFFFFFFFu, mbar_wait_short(bar_accfull + 8 * buf, (uses >> 1) & 1u, &sh.abort, p.status)))) break;
            tc_fence_after();
            const uint32_t acc = tmem + ((uint32_t)(quarter * 32) << 16) + buf * L::ACC1;
            const bool whole = pc.kb0 == 0 && pc.kb1 == pc.KB;
            // parked sums: a CTA has a place for its last piece (the start of a tile) and one for its first
            auto slot_of = [&](int w, bool starts) { return p.partials + ((size_t)(w * CG + rank) * 2 + (starts ? 1 : 0)) * p.TN * 32 + quarter * 32 + lane; };
            uint4* slot = slot_of(worker, pc.kb0 == 0);
            uint32_t o[16];                                  // 32 tokens, rounded
#pragma unroll
            for (int g = 0; g < CG; ++g) {
                // a pair's first turn: the half that the accumulators share, columns 128.. of the first, 0.. of the second
                const bool upper = CG == 2 && (g ^ buf ^ 1);
                const int c = (upper ? 128 : 0) + half * 32, cols = pc.rows - c;        // 32 tokens, and 32 more 64 on
                uint32_t v[64];
                if (cols > 0) { tmem_ld_16x256(acc + c, v); tmem_ld_16x256(acc + (16u << 16) + c, v + 16); }
                if (cols > 64) { tmem_ld_16x256(acc + c + 64, v + 32); tmem_ld_16x256(acc + (16u << 16) + c + 64, v + 48); }
                tmem_ld_wait();
                if (g == 0) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) { if constexpr (CG == 2) leader_arrive(accempty + 8 * buf); else mbar_arrive(accempty + 8 * buf); }
                }
                if (whole) {
                    if (cols > 0) {
                        pack_block(v, ow != nullptr, w, upper ? sx[CG - 1][0] : sx[0][0], lane, o);
                        store_block(p, o, box, upper ? to[CG - 1][0] : to[0][0], cols, n0, lane);
                    }
                    if (cols > 64) {
                        pack_block(v + 32, ow != nullptr, w, upper ? sx[CG - 1][1] : sx[0][1], lane, o);
                        store_block(p, o, box, upper ? to[CG - 1][1] : to[0][1], cols - 64, n0, lane);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {           // (token block i / 2, channel half i % 2)
                        const int r = 32 * (i >> 3) + 16 * (i & 1) + 4 * ((i >> 1) & 3), at = 8 * ((i >> 1) & 3) + 64 * (i >> 3);
                        if (at < cols) __stcg(slot + ((c + at) >> 3) * 256 + (i & 1) * 128, make_uint4(v[r], v[r + 1], v[r + 2], v[r + 3]));
                    }
                }
            }
            if (!whole) {
                // The workers that share this tile: those whose shares its first and its last k-block begin in.  (The release that
                // counts this warp in publishes what it has parked; whoever is last has acquired the others'.)
                const int c = sh.cost[pc.at], s0 = sh.unit0[pc.at] + pc.tile * pc.KB * c, s1 = s0 + (pc.KB - 1) * c;
                const float per = (float)sh.G / (float)max(1, sh.unit0[p.E] - sh.u0);
                int w0 = min(sh.G - 1, (int)((float)(s0 - sh.u0) * per)), w1 = min(sh.G - 1, (int)((float)(s1 - sh.u0) * per));
                while (sh.cut(w0) > s0) --w0;
                while (w0 + 1 < sh.G && sh.cut(w0 + 1) <= s0) ++w0;
                while (sh.cut(w1) > s1) --w1;
                while (w1 + 1 < sh.G && sh.cut(w1 + 1) <= s1) ++w1;
                __syncwarp();
                uint32_t old = 0;
                if (lane == 0) old = count_in(p.counters + (w0 * CG + rank) * FP_EPI_WARPS + warp);
                old = __shfl_sync(0xFFFFFFFFu, old, 0);
                __syncwarp();                                // (the lane that has acquired them, then the lanes that read: a shuffle orders no memory)
                // the adding up waits until this worker's other pieces are parked: somebody may be waiting for those
                if ((int)old == w1 - w0) {
                    if (owed == 0) { owed_at[0] = pc.at; owed_tile[0] = pc.tile; owed_w[0] = w0 | w1 << 16; }
                    else { owed_at[1] = pc.at; owed_tile[1] = pc.tile; owed_w[1] = w0 | w1 << 16; }
                    ++owed;
                }
            }
            ++uses;
        }
#pragma unroll 1
        for (int k = 0; ok && k < owed; ++k) {
            pc.at = k ? owed_at[1] : owed_at[0];
            pc.tile = k ? owed_tile[1] : owed_tile[0];
            const int w01 = k ? owed_w[1] : owed_w[0], w0 = w01 & 0xFFFF, w1 = w01 >> 16;
            place_tile(sh, pc);
            const int j0 = sh.off[pc.e] + pc.i0, n0 = (pc.nt * CG + (int)rank) * 128 + quarter * 32;
            const float* ow = p.ex[pc.e].outer;
            const float* ox = p.t.outer + sh.pad0[pc.e] + pc.i0;
            float w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) { const int n = n0 + (lane >> 2) + 8 * i; w[i] = ow && n < p.N ? ow[n] : 1.f; }
#pragma unroll 1
            for (int g = 0; g < 2 * CG; ++g) {
                const int c = (g >> 1) * 128 + half * 32 + (g & 1) * 64, cols = pc.rows - c;
                if (cols <= 0) continue;
                const int to = lane < cols ? p.perm[j0 + c + lane] : 0;
                const float x = ow && lane < cols ? ox[c + lane] : 1.f;
                auto parked = [&](int q) { return p.partials + ((size_t)(q * CG + rank) * 2 + (q == w0 ? 1 : 0)) * p.TN * 32 + (c >> 3) * 256 + quarter * 32 + lane; };
                uint32_t f[32], o[16];
#pragma unroll
                for (int i = 0; i < 32; ++i) f[i] = 0;
                auto add = [&](int r, const uint4& a) {
                    f[r] = __float_as_uint(__uint_as_float(f[r]) + __uint_as_float(a.x)); f[r + 1] = __float_as_uint(__uint_as_float(f[r + 1]) + __uint_as_float(a.y));
                    f[r + 2] = __float_as_uint(__uint_as_float(f[r + 2]) + __uint_as_float(a.z)); f[r + 3] = __float_as_uint(__uint_as_float(f[r + 3]) + __uint_as_float(a.w));
                };
                // several workers' sums on their way at a time, added in the workers' order: four of 16 tokens, two of 32
                if (cols <= 16) {
                    for (int q = w0; q <= w1; q += 4) {
                        uint4 a[4][4];
#pragma unroll
                        for (int j = 0; j < 4; ++j)
#pragma unroll
                            for (int i = 0; i < 4; ++i) a[j][i] = q + j <= w1 && 8 * (i >> 1) < cols ? __ldcg(parked(q + j) + i * 128) : make_uint4(0, 0, 0, 0);
#pragma unroll
                        for (int j = 0; j < 4; ++j)
#pragma unroll
                            for (int i = 0; i < 4; ++i) add(16 * (i & 1) + 4 * (i >> 1), a[j][i]);
                    }
                } else {
                    for (int q = w0; q <= w1; q += 2) {
                        uint4 a[2][8];
#pragma unroll
                        for (int j = 0; j < 2; ++j)
#pragma unroll
                            for (int i = 0; i < 8; ++i) a[j][i] = q + j <= w1 && 8 * (i >> 1) < cols ? __ldcg(parked(q + j) + i * 128) : make_uint4(0, 0, 0, 0);
#pragma unroll
                        for (int j = 0; j < 2; ++j)
#pragma unroll
                            for (int i = 0; i < 8; ++i) add(16 * (i & 1) + 4 * (i >> 1), a[j][i]);
                    }
                }
                pack_block(f, ow != nullptr, w, x, lane, o);
                store_block(p, o, box, to, cols, n0, lane);
            }
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
    if constexpr (CG == 2) cluster_sync();                 // (the other CTA's copies, MMAs and arrivals are done too)
    if (warp == FP_MMA_WARP) {
        __syncwarp();
        tc_fence_after();
        fp_tmem_dealloc<CG>(tmem);
    }
}

// Tokens of a tile, and whether two SMs share it.  Up to 64 rows a tile is as narrow as the batch.  A pair reads weights and tokens half as
// often, but its tiles are four times as large: it gets them if there are at least half as many of them as pairs (4096 -> 4096: 2048 rows
// MXFP4 28.2 us, with one SM to a tile 35.1, 600 rows 15.3 and 17.6, 8192 rows bf16 238 and 312; 4096 -> 1024, 2048 rows in NVFP4 and bf16
// 38.3 with pairs, 34.0 without).  One SM's tiles take 64 tokens instead of 128 where the larger ones would leave SMs without and a call
// has both kinds of experts, bf16 ones four times as deep (777 rows, 2056 -> 1000, three formats: 16.5 us, with 128 tokens 20.7;
// 4-bit experts only 12.5 and 11.9, bf16 only 19.8 and 19.4 (512 channels of 3584 k)).  Three formats, rows spread evenly, weights not in L2,
// 64 / 128: 200 x 2056 -> 1000 14.8 / 16.9, 512 x 3584 -> 512 17.8 / 18.6, 1000 x 3584 -> 512 20.9 / 23.5, 500 x 2048 -> 2048 14.4 / 19.3, 256 x 4096 -> 4096
// 21.7 / 23.6; the slower choice for many rows of a long k: 1500 x 8200 -> 520 33.7 / 32.4, over two formats and skewed 40.3 / 36.9.
struct FpTile { int TN; bool pair; };
FpTile pick_tile(int M, const moqe_fp_expert* const* ex, int E) {
    if (M <= 64) return {M <= 16 ? 16 : M <= 32 ? 32 : 64, false};
    const long long workers = device_sm_count(), NT = ex[0]->Np / 128;
    if (M > 128 && 4 * ((NT + 1) / 2) * ((M + 255ll) / 256) >= workers) return {256, true};
    int deep = 0;
    for (int e = 0; e < E; ++e) deep += ex[e]->format == MOQE_FP_BF16;
    return {M <= 128 || deep == 0 || deep == E || 2 * NT * ((M + 127ll) / 128) >= workers ? 128 : 64, false};
}

// The schedule counts costs in 32 bits.
bool fp_schedulable(int M, const moqe_fp_expert* const* ex, int E) {
    if (M > 1 << 30) return false;
    long long deepest = 0;
    for (int e = 0; e < E; ++e) {
        const long long cost = (long long)ex[e]->KB * (ex[e]->format == MOQE_FP_BF16 ? FP_COST_BF16 : FP_COST_4BIT);
        deepest = cost > deepest ? cost : deepest;
    }
    const FpTile t = pick_tile(M, ex, E);
    const long long tiles = ((long long)M / t.TN + E) * (t.pair ? (ex[0]->Np / 128 + 1) / 2 : ex[0]->Np / 128);
    return tiles <= (1ll << 30) / deepest;
}

size_t al256(size_t x) { return (x + 255) / 256 * 256; }

struct FpLayout { size_t perm, offsets, sort, counters, codes, sf, outer, partials, total, row_bytes, block_sf; };

FpLayout fp_layout(int M, const moqe_fp_expert* const* ex, int E) {
    FpLayout w = {};
    for (int e = 0; e < E; ++e) {
        const size_t rb = (size_t)ex[e]->KB * 128, sb = (size_t)ex[e]->KB * fp_sf_bytes(ex[e]->format);
        w.row_bytes = rb > w.row_bytes ? rb : w.row_bytes;
        w.block_sf = sb > w.block_sf ? sb : w.block_sf;
    }
    // Every expert's segment is filled up to 16 rows, its last tile's scales to a block or two.  (Whatever the tile, there are no more
    // blocks than these: a workspace for many rows serves fewer ones.)
    const size_t some = M < E ? M : E, rows = (size_t)M + 15 * some, blocks = (size_t)M / 64 + 2 * some + 1;
    size_t off = 0;
    w.perm = off;     off += al256((size_t)M * 4 + 16);
    w.offsets = off;  off += al256((MOQE_MAX_EXPERTS + 2) * 4);
    w.sort = off;     off += al256(sort_workspace_bytes(M, E));
    w.counters = off; off += al256((size_t)fp_gemm_counters() * 4);
    w.codes = off;    off += al256(rows * w.row_bytes);
    w.sf = off;       off += al256(blocks * w.block_sf);
    w.outer = off;    off += al256(rows * 4);
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
        if (ex[e]->N != ex[0]->N || ex[e]->K != ex[0]->K || ex[e]->device != ex[0]->device) return MOQE_ERR_MISMATCH;
    if (M == 0) return MOQE_OK;
    if (!X || !rows || !offsets || !Y) return MOQE_ERR_NULL;
    const moqe_status here = fp_on_current_device(ex[0]);
    if (here != MOQE_OK) return here;
    if (ex[0]->N % 8 != 0 || (uintptr_t)X % 16 || (uintptr_t)Y % 16 || !fp_schedulable(M, ex, E)) return MOQE_ERR_UNSUPPORTED;
    w = fp_layout(M, ex, E);
    if (!workspace || workspace_bytes < w.total || (uintptr_t)workspace % 256) return MOQE_ERR_WORKSPACE;
    return MOQE_OK;
}

moqe_status fp_run(const void* X, const int32_t* perm, const int32_t* offsets, int M, const moqe_fp_expert* const* ex, int E, void* Y,
                   char* base, const FpLayout& w, cudaStream_t st) {
    if (fp_gemv_supported(ex, E, M)) return launch_fp_gemv(X, M, perm, offsets, ex, E, Y, st);
    FpTokens t = {(uint8_t*)base + w.codes, (uint8_t*)base + w.sf, (float*)(base + w.outer), w.row_bytes, w.block_sf, pick_tile(M, ex, E).TN};
    FpExperts formats;
    for (int e = 0; e < E; ++e) formats.format[e] = (uint8_t)ex[e]->format;
    uint32_t* counters = (uint32_t*)(base + w.counters);
    const moqe_status s = launch_fp_tokens(X, perm, offsets, M, ex[0]->K, E, formats, t, counters, fp_gemm_counters(), st);
    if (s != MOQE_OK) return s;
    return launch_fp_gemm(ex, E, M, perm, offsets, t, counters, base + w.partials, Y, st);
}

}  // namespace

int fp_gemm_counters() { return device_sm_count() * FP_EPI_WARPS; }
size_t fp_gemm_partial_bytes(int M) { return (size_t)device_sm_count() * 2 * (M <= 16 ? 16 : M <= 32 ? 32 : M <= 64 ? 64 : M <= 128 ? 128 : 256) * 128 * 4; }

moqe_status launch_fp_gemm(const moqe_fp_expert* const* ex, int E, int M, const int32_t* perm, const int32_t* offsets, const FpTokens& tokens,
                           uint32_t* counters, void* partials, void* Y, cudaStream_t st) {
    FpGemmParams p = {};
    int sf = 0;
    for (int e = 0; e < E; ++e) {
        p.ex[e] = {ex[e]->tiles, ex[e]->outer, ex[e]->format, ex[e]->KB};
        const int b = fp_sf_bytes(ex[e]->format);
        sf = b > sf ? b : sf;
    }
    p.perm = perm; p.offsets = offsets; p.t = tokens; p.counters = counters; p.partials = (uint4*)partials; p.Y = (__nv_bfloat16*)Y;
    p.status = device_status_word();
    if (!p.status) return MOQE_ERR_ALLOC;
    p.E = E; p.N = ex[0]->N; p.NT = ex[0]->Np / 128;
    const FpTile tile = pick_tile(M, ex, E);
    const bool pair = tile.pair;
    p.TN = tile.TN;
    p.sf = sf;
    static_assert(FP_RING_BYTES / (16384 + 1024) >= 8 && FP_MAX_STAGES >= 8, "the ring's stages");
    // One SM's sums are parked and added up in some 20 k-blocks' time, a pair's (four times as many) in 36.  With 6 and 18 instead:
    // 48 rows of NVFP4, 4096 -> 11008, 18.9 us for 12.5; 512 rows in three formats 32 for 28.5; 4160 rows of 3584 -> 18944 295 for 285;
    // 2048 rows of bf16 62 for 59.
    p.split_cost = pair ? 36 : 20;
    p.least_share = pair ? 24 : 12;
    static std::atomic<unsigned long long> attr[2] = {};
    const auto kernel = pair ? fp_gemm_kernel<2> : fp_gemm_kernel<1>;
    if (!ensure_dynamic_smem((const void*)kernel, FP_SMEM, attr[pair])) { cudaGetLastError(); return MOQE_ERR_CUDA; }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(pair ? device_sm_count() & ~1 : device_sm_count()); cfg.blockDim = dim3(FP_THREADS); cfg.dynamicSmemBytes = FP_SMEM; cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = 2; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
    cfg.attrs = at; cfg.numAttrs = pair ? 2 : 1;
    if (cudaLaunchKernelEx(&cfg, kernel, p) != cudaSuccess) { cudaGetLastError(); return MOQE_ERR_CUDA; }
    count_launch();
    return MOQE_OK;
}

}  // namespace moqe

using namespace moqe;

extern "C" size_t moqe_routed_fpgemm_workspace(int M, const moqe_fp_expert* const* h_experts, int E) {
    if (M < 0 || !h_experts || E <= 0 || E > MOQE_MAX_EXPERTS) return 0;
    for (int e = 0; e < E; ++e)
        if (!h_experts[e]) return 0;
    return fp_schedulable(M, h_experts, E) ? fp_layout(M, h_experts, E).total : 0;
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
