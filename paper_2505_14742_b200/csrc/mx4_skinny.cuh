// The skinny products of the 4-bit layer's adapters (one side r <= 64 columns wide), each in one launch:
//   kSkinnyDown : T = X A, and in the same pass over X its MXFP4 codes and scales      kSkinnyParts : G = s dY B^T
//   kSkinnyFold : dA = X^T G (G in bf16 parts, added up)                                kSkinnyTurned : dB = (s dY^T T)^T
//
// A CTA has 128 output rows and a slice of the contraction, which arrives by TMA in stages of 64 elements; the slices of a row
// tile form a cluster: their shares are left in shared memory and added up in rank order through it, so neither partial sums in
// HBM nor a second launch are needed.  Bound by HBM: the long operand once (measured, cold: G and dB over 8192 x 11008 37 and 36 us,
// 4.9 TB/s; T with the codes over 8192 x 4096 25 us, where three launches took 40).  The quantization rides along: a stage of X
// is 128 rows x 64 columns, which eight warps quantize out of the same shared memory (a thread has one block of 32 columns); two
// such groups take turns (8192 x 11008 49 us, 8192 x 4096 20 us with the operands partly in L2; one group 0.7 us more).
//
// A tcgen05.mma loses up to one unit in the last place of its running sum, always towards zero, so the error of a chain of n
// grows like n.  The MMAs of a tile therefore go round robin to as many accumulators as tensor memory holds (up to sixteen; dA has three
// parts of G beside one another, which leaves 8, 4 and 2 of them for r = 16, 32 and 64), added up in fp32 at the end.  Where that still makes chains of more than
// kSkChain, the accumulators are two sets: one is drained into fp32 registers while the other is filled.  dA of 8192 tokens x 11008, error over
// norm, operands of both signs / all positive: r = 16 6e-7 / 7e-7, r = 64 7e-7 / 9e-7 (in one set 1.1e-6 / 1.6e-6 and 4.6e-6 / 1.0e-5,
// growing with the tokens; the backward without dX 1 us less of 68 and of 82).
#pragma once

#include "mx4_gemm.cuh"

namespace quaff {

constexpr int kSkGroup = 8, kSkWarps = 2 * kSkGroup, kSkThreads = 64 + kSkWarps * 32;
template <int MODE> struct SkinnyCfg {
    static constexpr int kCols = MODE == kSkinnyFold ? 192 : 64;                            // columns at most (dA: three parts of G)
    static constexpr int kStageBytes = 16384 + kCols / 64 * kAtomBytes;                     // 128 rows x 64; the short operand
    static constexpr int kStages = MODE == kSkinnyFold ? 5 : 8;
    static constexpr bool kAMn = MODE >= kSkinnyFold, kBMn = MODE != kSkinnyParts;          // operands whose rows are the contraction
    static_assert(kStages * kStageBytes >= 128 * kCols * 4, "a share takes the stages' place");
};
constexpr int kSkChain = 32;               // MMAs that one accumulator adds up at most
struct SkinnySmem {
    uint64_t full[8], empty[8];
    uint64_t acc_full[2], acc_free[2];     // a set of accumulators is complete; is drained
    uint32_t tmem_base;
    AbortCtl abort;
};
template <int MODE> constexpr size_t skinny_smem() { return 1024 + (size_t)SkinnyCfg<MODE>::kStages * SkinnyCfg<MODE>::kStageBytes + sizeof(SkinnySmem); }

__device__ __forceinline__ float4 ld_share(uint32_t at, int rank, int ranks, const unsigned char* smem_dyn, uint32_t raw) {
    return ranks > 1 ? ld_cluster_f4(mapa_shared(at, rank)) : *reinterpret_cast<const float4*>(smem_dyn + (at - raw));
}

// (p has to be a __grid_constant__ parameter of the kernel, or part of one: it holds tensor maps)
template <int MODE>
__device__ __forceinline__ void mx4_skinny_body(const SkinnyParams& p, int block) {
    using Cfg = SkinnyCfg<MODE>;
    constexpr int kStages = Cfg::kStages, kStageBytes = Cfg::kStageBytes;
    extern __shared__ unsigned char smem_dyn[];
    const uint32_t raw = smem_u32(smem_dyn);
    const uint32_t base = (raw + 1023u) & ~1023u;
    unsigned char* stages = smem_dyn + (base - raw);
    SkinnySmem* sm = reinterpret_cast<SkinnySmem*>(stages + (size_t)kStages * kStageBytes);
    volatile AbortCtl* abort_flag = &sm->abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = p.ranks > 1 ? (int)cluster_ctarank() : 0;
    const int m0 = block / p.ranks * 128;
    const int s0 = rank * p.per, count = max(0, min(p.per, p.nst - s0));
    const uint32_t full0 = smem_u32(&sm->full[0]), empty0 = smem_u32(&sm->empty[0]);
    const uint32_t acc_full0 = smem_u32(&sm->acc_full[0]), acc_free0 = smem_u32(&sm->acc_free[0]);
    // one set of p.rot accumulators for all stages, or sets of half as many for `chunk` stages each
    const bool one_set = 4 * p.per <= kSkChain * p.rot;
    const int rot = one_set ? p.rot : p.rot / 2, chunk = one_set ? p.per : kSkChain / 4 * rot;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) { mbar_init(full0 + 8u * s, 1); mbar_init(empty0 + 8u * s, MODE == kSkinnyDown ? 1 + kSkGroup : 1); }
        for (int h = 0; h < 2; ++h) { mbar_init(acc_full0 + 8u * h, 1); mbar_init(acc_free0 + 8u * h, kSkWarps); }
        sm->abort.flag = 0;
        sm->abort.peer = 0;
        fence_barrier_init();
    }
    if (warp == 1) {
        tmem_alloc<1>(smem_u32(&sm->tmem_base), 512);
        tmem_relinquish<1>();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sm->tmem_base;
    pdl_wait();
    pdl_launch_dependents();      // only now: what starts early behind this kernel may rely on all work in front of it

    if (warp == 0) {
        if (elect_one()) {
            for (int i = 0; i < count; ++i) {
                const uint32_t s = (uint32_t)(i % kStages), dst = base + s * kStageBytes, bar = full0 + 8u * s;
                if (i >= kStages && !mbar_wait(empty0 + 8u * s, (uint32_t)(i / kStages - 1) & 1u, abort_flag)) break;
                const int k = (s0 + i) * 64;
                mbar_arrive_expect_tx(bar, p.tx_bytes);
                if (Cfg::kAMn) {       // boxes of 64 contraction rows x 64 output rows
                    tma_load_2d<1>(dst, &p.map_a, m0, k, bar);
                    tma_load_2d<1>(dst + kAtomBytes, &p.map_a, m0 + 64, k, bar);
                } else {
                    tma_load_2d<1>(dst, &p.map_a, k, m0, bar);
                }
                if (Cfg::kBMn) for (int x = 0; x * 64 < p.cols; ++x) tma_load_2d<1>(dst + 16384 + x * kAtomBytes, &p.map_b, 64 * x, k, bar);
                else tma_load_2d<1>(dst + 16384, &p.map_b, k, 0, bar);
            }
        }
    } else if (warp == 1) {
        if (elect_one()) {
            const uint32_t idesc = umma_idesc(kCFmtF32, kFmtBF16, 128, 0) | ((uint32_t)(p.cols >> 3) << 17) | (Cfg::kAMn ? 1u << 15 : 0u) | (Cfg::kBMn ? 1u << 16 : 0u);
            constexpr uint32_t a_lbo = Cfg::kAMn ? (uint32_t)(kAtomBytes >> 4) << 16 : 1u << 16, a_adv = Cfg::kAMn ? 128u : 2u;
            constexpr uint32_t b_lbo = Cfg::kBMn ? (uint32_t)(kAtomBytes >> 4) << 16 : 1u << 16, b_adv = Cfg::kBMn ? 128u : 2u;
            int set = 0, at = 0;           // sets filled so far; stages of the present one
            for (int i = 0; i < count; ++i) {
                const uint32_t s = (uint32_t)(i % kStages), half = (uint32_t)set & 1u;
                if (at == 0 && set >= 2 && !mbar_wait(acc_free0 + 8u * half, (uint32_t)(set / 2 - 1) & 1u, abort_flag)) break;
                if (!mbar_wait(full0 + 8u * s, (uint32_t)(i / kStages) & 1u, abort_flag)) break;
                tc_fence_after();
                const uint32_t s_lo = ((base + s * kStageBytes) & 0x3FFFFu) >> 4;
                const uint32_t a_lo = s_lo | a_lbo, b_lo = (s_lo + (16384u >> 4)) | b_lbo;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int n = 4 * at + k;
                    umma_f16<1>(tmem + (half * rot + (n & (rot - 1))) * p.cols, make_desc(a_lo + k * a_adv, kDescHi), make_desc(b_lo + k * b_adv, kDescHi), idesc, n >= rot);
                }
                umma_commit<1>(empty0 + 8u * s);
                if (++at == chunk || i == count - 1) {
                    umma_commit<1>(acc_full0 + 8u * half);
                    ++set;
                    at = 0;
                }
            }
        }
    } else {
        // (quantization: warps 2..9 take the even stages, 10..17 the odd ones, four of each the first block of a stage, four the
        // second;) row = lane quarter, as TMEM wants it below
        const int q = warp & 3, row = q * 32 + lane, quad = (warp - 2) >> 2, half = quad & 1;
        const int m = m0 + row;
        bool ok = true;
        // this thread's columns of its row: sixteen of every 64
        float sum[Cfg::kCols / 64][16];
#pragma unroll
        for (int c = 0; c < Cfg::kCols / 64; ++c)
#pragma unroll
            for (int j = 0; j < 16; ++j) sum[c][j] = 0.0f;
        int drained = 0;
        auto drain = [&]() {
            const uint32_t half = (uint32_t)drained & 1u;
            if (!mbar_wait(acc_full0 + 8u * half, (uint32_t)(drained / 2) & 1u, abort_flag)) return false;
            tc_fence_after();
            const int used = min(rot, 4 * (count - drained * chunk));
#pragma unroll
            for (int c = 0; c < Cfg::kCols / 64; ++c) {
                const int cc = c * 64 + quad * 16;
                for (int a = 0; a < used && cc < p.cols; ++a) {
                    uint32_t t[16];
                    tmem_ld_32x16(tmem + ((uint32_t)(q * 32) << 16) + (half * rot + a) * p.cols + cc, t);
                    tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 16; ++j) sum[c][j] += __uint_as_float(t[j]);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(acc_free0 + 8u * half);
            ++drained;
            return true;
        };
        for (int i = quad >> 1; MODE == kSkinnyDown && i < count; i += 2) {
            // (a set whose stages are quantized; its MMAs wait for nothing else)
            while (ok && drained < i / chunk) ok = drain();
            if (!ok) break;
            const uint32_t s = (uint32_t)(i % kStages);
            if (!mbar_wait(full0 + 8u * s, (uint32_t)(i / kStages) & 1u, abort_flag)) { ok = false; break; }
            const unsigned char* src = stages + (size_t)s * kStageBytes + row * 128;
            uint4 v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = *reinterpret_cast<const uint4*>(src + (((half * 4 + j) ^ (row & 7)) * 16));
            uint32_t c[4], byte;
            mx4_quantize_block(v, c, byte);
            // Hand the stage back once its words are in registers.  The arrival does not wait for loads that are still on their way, not
            // even those of its own warp, so it is made to depend on them: no scale byte has bit 8.
            const uint32_t seen = __reduce_or_sync(0xFFFFFFFFu, byte) >> 8;
            if (lane == 0) mbar_arrive(empty0 + 8u * (s + seen));
            const int block = (s0 + i) * 2 + half;
            if (m < p.M && block * 32 < p.K) *reinterpret_cast<uint4*>(p.codes + (int64_t)m * p.ldc + block * 16) = make_uint4(c[0], c[1], c[2], c[3]);
            uint8_t* sc = p.scales + mx4_scale_offset(m, block, p.ktiles);
            *sc = (uint8_t)byte;                                  // rows and columns beyond the matrix are zeros: byte 0
            if (s0 + i == p.nst - 1 && (p.nst & 1)) sc[2] = 0;    // the other half of the last scale tile
        }
        while (ok && drained * chunk < count) ok = drain();
        if (MODE == kSkinnyDown) named_bar_sync(1, kSkWarps * 32);      // nobody reads a stage any more
        if (ok) {
            float* share = reinterpret_cast<float*>(stages) + row * p.cols;
#pragma unroll
            for (int c = 0; c < Cfg::kCols / 64; ++c) {
                const int cc = c * 64 + quad * 16;
                if (cc >= p.cols) continue;
#pragma unroll
                for (int j = 0; j < 16; j += 4) *reinterpret_cast<float4*>(share + cc + j) = make_float4(sum[c][j], sum[c][j + 1], sum[c][j + 2], sum[c][j + 3]);
            }
        }
    }

    tc_fence_before();
    __syncthreads();
    if (p.ranks > 1) cluster_sync();
    if (!abort_flag->flag) {
        // this rank's rows, eight columns per thread; consecutive threads take consecutive columns, or rows where those are
        // neighbours in the result
        const int per_rank = (128 + p.ranks - 1) / p.ranks, lo = rank * per_rank, rows = min(min(per_rank, 128 - lo), p.M - m0 - lo);
        const int groups = p.rp >> 3;
        for (int i = (int)threadIdx.x; i < rows * groups; i += kSkThreads) {
            const int row = lo + (MODE == kSkinnyTurned ? i % rows : i / groups), j = (MODE == kSkinnyTurned ? i / rows : i % groups) * 8;
            const int64_t m = m0 + row;
            float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            for (int n = p.cols / p.rp - 1; n >= 0; --n) {            // (parts of G: the small ones first)
                const uint32_t at = base + (uint32_t)(row * p.cols + n * p.rp + j) * 4u;
                float h[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll 4
                for (int q = 0; q < p.ranks; ++q) {
                    const float4 a = ld_share(at, q, p.ranks, smem_dyn, raw), b = ld_share(at + 16, q, p.ranks, smem_dyn, raw);
                    h[0] += a.x; h[1] += a.y; h[2] += a.z; h[3] += a.w;
                    h[4] += b.x; h[5] += b.y; h[6] += b.z; h[7] += b.w;
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += h[e];
            }
            if (MODE == kSkinnyFold) {
                if (j >= p.r) continue;
                float4* d = reinterpret_cast<float4*>(p.f32_out + m * p.r + j);
                float4 a = make_float4(v[0], v[1], v[2], v[3]), b = make_float4(v[4], v[5], v[6], v[7]);
                if (p.accumulate) {
                    const float4 c = d[0], e = d[1];
                    a.x += c.x; a.y += c.y; a.z += c.z; a.w += c.w;
                    b.x += e.x; b.y += e.y; b.z += e.z; b.w += e.w;
                }
                d[0] = a;
                d[1] = b;
            } else if (MODE == kSkinnyTurned) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (j + e < p.r) {
                        float* d = p.f32_out + (int64_t)(j + e) * p.M + m;
                        *d = p.accumulate ? *d + p.scale * v[e] : p.scale * v[e];
                    }
            } else {
                if (p.bf16_out && j < p.r) {
                    const float s = p.bf16_scale;
                    *reinterpret_cast<uint4*>(p.bf16_out + m * p.r + j) =
                        make_uint4(pack_bf16x2(s * v[0], s * v[1]), pack_bf16x2(s * v[2], s * v[3]), pack_bf16x2(s * v[4], s * v[5]), pack_bf16x2(s * v[6], s * v[7]));
                }
                // the parts: the rounding, the rounding of what that leaves, and so on (8 bits each); columns beyond r are zero
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = __fmul_rn(p.scale, v[e]);
                uint16_t* t = p.parts_out + m * p.parts * p.rp + j;
                for (int n = 0; n < p.parts; ++n, t += p.rp) {
                    uint32_t w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t lo = bf16_part(v[2 * e]);
                        w[e] = lo | bf16_part(v[2 * e + 1]) << 16;
                    }
                    *reinterpret_cast<uint4*>(t) = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
        }
    }
    if (abort_flag->flag) {
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);   // let copies in flight land before the CTA retires
        if (threadIdx.x == 0 && p.status) atomicExch(p.status, (int)QUAFF_ERR_TIMEOUT);
    }
    __syncthreads();
    if (p.ranks > 1) cluster_sync();       // shares stay until every rank has read them
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc<1>(tmem, 512);
    }
}
template <int MODE>
__global__ void __launch_bounds__(kSkThreads, 1) mx4_skinny_kernel(const __grid_constant__ SkinnyParams p) {
    mx4_skinny_body<MODE>(p, (int)blockIdx.x);
}

}  // namespace quaff
