// The MXFP4 product for few tokens: Y = Xd Wd^T (+ s T B) where 256 x 256 tiles would leave most SMs idle.
//
// The time is that of reading W once, so the contraction is cut over a cluster of up to eight CTAs and the tile is turned
// round: the 128 accumulator rows (lanes of TMEM) are rows of W, its columns are tokens, as many as there are (a multiple of
// 16, up to 128).  A token's outputs then lie along the lanes, so partial sums go to shared memory and results to Y in whole
// lines.  Every CTA leaves its partial tile in shared memory; after a cluster barrier rank q adds up tokens q, q + ranks, ... of all
// of them in rank order (no atomics) and stores them.
//
// Measured, 4096 x 4096: 1 token 5.5 us (8.9 MB of weight: 1.4 us at the measured HBM rate, the rest is the latency of launch, TMEM,
// first copies, cluster barrier), 16 tokens 5.7, 128 tokens 9.7; with 256 x 256 tiles 11.0 to 11.7.
//
//   warp 0 : TMA producer    warp 1 : TMEM, scale copies, tcgen05.mma (one CTA)    warps 2..5 : epilogue
//
// FUSED (up to 16 tokens): the whole layer in this one launch.  X arrives in bf16 beside W, the epilogue warps quantize it into the
// stage's operand (a thread has one block of 32 columns) while the tensor core multiplies it with A (turned round too: the
// accumulator rows are ranks of A); every row tile repeats that, which costs A from L2 once more per tile.  The shares of T are added up
// like those of Y, and s T B is added in fp32, the column of B fetched into registers while the tensor core works.  What it saves is
// the launch in front: through 4096 x 4096 with everything in L2, 1 token, r = 16: 8.6 us instead of 8.9, and 10.4 us of host time instead of 12.6; 16 tokens,
// r = 64: 11.0 instead of 15.2.  The dispatch in mx4.cu has more sizes, with weights from HBM.
//
// Not fused, but behind a kernel that makes codes, scales and s T and lets this one start early (mx4_prep_kernel, mx4_skinny), the
// producer fetches W ahead of griddepcontrol.wait: W was complete before that kernel passed its own.
#pragma once

#include "mx4_gemm.cuh"

namespace quaff {

constexpr int kMsTokens = 128;                                                       // token tile at most
constexpr int kMsThreads = 192, kMsMaxStages = 6, kMsFusedTokens = 16;
template <bool FUSED> struct MsCfg {
    static constexpr int kTokens = FUSED ? kMsFusedTokens : kMsTokens;
    static constexpr int kX = 16384, kSf = kX + kTokens * 128;                       // W | X codes | scales of W, of X | X in bf16 | A
    static constexpr int kRaw = kSf + 2048, kA = kRaw + 4 * 2048;
    static constexpr int kStageBytes = FUSED ? kA + 4 * kAtomBytes : kRaw;
    static constexpr int kStages = FUSED ? 3 : kMsMaxStages;
    static constexpr int kPartFloats = kTokens * 128 + (FUSED ? 64 * kMsFusedTokens : 0);      // shares of Y, of T
    static_assert(kStages * kStageBytes >= (kPartFloats + (FUSED ? kMsFusedTokens * 64 : 0)) * 4, "the shares (and T) take the stages' place");
};
// TMEM: the accumulator, (FUSED) eight of T with 16 columns, the scale slots
constexpr int kMsTCol = 16, kMsTRot = 8, kMsSfCol = 160, kMsSfSlot = 16, kMsSfSlots = 4, kMsTmemCols = 256;
constexpr uint32_t kMsIdesc = (1u << 7) | (1u << 10) | (1u << 23) | ((128u >> 4) << 24);      // + N, scale selectors

struct Mx4SmallParams {
    CUtensorMap map_w, map_x, map_sw, map_sx;
    CUtensorMap map_t, map_b;
    int ktiles, sw_tiles, sx_tiles;
    int nblk, nmma_last, per;        // stages of the contraction; of a rank
    int rp, lora_parts;
    int M, N, nt, row_tiles, ranks;
    int early_w;
    // FUSED
    CUtensorMap map_raw, map_a;      // X [M][K], A [K][r]
    const uint16_t* B;
    uint16_t* T;
    int r;
    float scale;
    void* Y;
    int64_t ldy;
    int y_f32;
    int32_t* status;
};
struct MsSmem {
    uint64_t full[kMsMaxStages], empty[kMsMaxStages], quantized[kMsMaxStages], acc_full;
    uint32_t tmem_base;
    AbortCtl abort;
};
template <bool FUSED> constexpr size_t ms_smem() { return 1024 + (size_t)MsCfg<FUSED>::kStages * MsCfg<FUSED>::kStageBytes + sizeof(MsSmem); }

__device__ __forceinline__ void umma_mxf4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void tmem_cp_scales(uint32_t taddr, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}

template <bool FUSED>
__global__ void __launch_bounds__(kMsThreads, 1) mx4_small_kernel(const __grid_constant__ Mx4SmallParams p) {
    using Cfg = MsCfg<FUSED>;
    constexpr int kMsStages = Cfg::kStages, kMsStageBytes = Cfg::kStageBytes;
    extern __shared__ unsigned char smem_dyn[];
    const uint32_t raw = smem_u32(smem_dyn);
    const uint32_t base = (raw + 1023u) & ~1023u;
    MsSmem* sm = reinterpret_cast<MsSmem*>(smem_dyn + (base - raw) + (size_t)kMsStages * kMsStageBytes);
    volatile AbortCtl* abort_flag = &sm->abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = p.ranks > 1 ? (int)cluster_ctarank() : 0;
    const int unit = (int)blockIdx.x / p.ranks;
    const int n0 = unit % p.row_tiles * 128, t0 = unit / p.row_tiles * p.nt;
    const int b0 = rank * p.per, b1 = min(b0 + p.per, p.nblk);       // every rank has one stage at least
    const int lora = !FUSED && rank == 0 ? p.lora_parts : 0;
    const uint32_t full0 = smem_u32(&sm->full[0]), empty0 = smem_u32(&sm->empty[0]), acc_full = smem_u32(&sm->acc_full);
    const uint32_t quant0 = smem_u32(&sm->quantized[0]);
    if (threadIdx.x == 0) {
        for (int s = 0; s < kMsStages; ++s) { mbar_init(full0 + 8u * s, 1); mbar_init(empty0 + 8u * s, 1); mbar_init(quant0 + 8u * s, 4); }
        mbar_init(acc_full, 1);
        sm->abort.flag = 0;
        sm->abort.peer = 0;
        fence_barrier_init();
    }
    if (warp == 1) {
        tmem_alloc<1>(smem_u32(&sm->tmem_base), kMsTmemCols);
        tmem_relinquish<1>();
    }
    pdl_launch_dependents();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sm->tmem_base;
    const uint32_t x_bytes = (uint32_t)p.nt * 128u;
    const int row_of = (int)threadIdx.x - 64;      // epilogue threads: the output column of their own
    uint32_t b2[FUSED ? 32 : 1];

    if (warp == 0) {
        if (elect_one()) {
            const int sw = min(n0 >> 7, p.sw_tiles - 1) * p.ktiles * 4, sx = min(t0 >> 7, p.sx_tiles - 1) * p.ktiles * 4;
            auto load_w = [&](int i) {           // stage of the rank's i-th block
                const uint32_t s = (uint32_t)(i % kMsStages), dst = base + s * kMsStageBytes, bar = full0 + 8u * s;
                mbar_arrive_expect_tx(bar, FUSED ? 16384u + 1024u + 4u * 2048u + (p.r ? 4u * kAtomBytes : 0u) : 16384u + x_bytes + 2048u);
                tma_load_2d<1>(dst, &p.map_w, (b0 + i) * 128, n0, bar);
                tma_load_2d<1>(dst + Cfg::kSf, &p.map_sw, 0, sw + (b0 + i) * 8, bar);
            };
            auto load_x = [&](int i) {
                const uint32_t s = (uint32_t)(i % kMsStages), dst = base + s * kMsStageBytes, bar = full0 + 8u * s;
                if (FUSED) {
                    for (int u = 0; u < 4; ++u) tma_load_2d<1>(dst + Cfg::kRaw + u * 2048, &p.map_raw, (b0 + i) * 256 + 64 * u, 0, bar);
                    if (p.r) for (int u = 0; u < 4; ++u) tma_load_2d<1>(dst + Cfg::kA + u * kAtomBytes, &p.map_a, 0, (b0 + i) * 256 + 64 * u, bar);
                } else {
                    tma_load_2d<1>(dst + Cfg::kX, &p.map_x, (b0 + i) * 128, t0, bar);
                    tma_load_2d<1>(dst + Cfg::kSf + 1024, &p.map_sx, 0, sx + (b0 + i) * 8, bar);
                }
            };
            const int nb = b1 - b0, ahead = min(nb, kMsStages);
            if (!p.early_w) pdl_wait();
            for (int i = 0; i < ahead; ++i) load_w(i);
            if (p.early_w) pdl_wait();
            for (int i = 0; i < ahead; ++i) load_x(i);
            bool ok = true;
            for (int i = ahead; i < nb + lora && ok; ++i) {
                const uint32_t s = (uint32_t)(i % kMsStages);
                if (i >= kMsStages && !mbar_wait(empty0 + 8u * s, (uint32_t)(i / kMsStages - 1) & 1u, abort_flag)) { ok = false; break; }
                if (i < nb) {
                    load_w(i);
                    load_x(i);
                } else {                         // LoRA: B [r][N] (rows = contraction), a part of s T
                    const uint32_t dst = base + s * kMsStageBytes, bar = full0 + 8u * s;
                    mbar_arrive_expect_tx(bar, 2u * (uint32_t)p.rp * 128u + x_bytes);
                    tma_load_2d<1>(dst, &p.map_b, n0, 0, bar);
                    tma_load_2d<1>(dst + kAtomBytes, &p.map_b, n0 + 64, 0, bar);
                    tma_load_2d<1>(dst + Cfg::kX, &p.map_t, (i - nb) * p.rp, t0, bar);
                }
            }
        }
    } else if (warp == 1) {
        if (elect_one()) {
            bool ok = true;
            const int nb = b1 - b0;
            uint32_t accumulate = 0;
            const uint32_t idn = (uint32_t)(p.nt >> 3) << 17;
            for (int i = 0; i < nb + lora && ok; ++i) {
                const uint32_t s = (uint32_t)(i % kMsStages);
                if (!mbar_wait(full0 + 8u * s, (uint32_t)(i / kMsStages) & 1u, abort_flag)) { ok = false; break; }
                const uint32_t s_lo = ((base + s * kMsStageBytes) & 0x3FFFFu) >> 4;
                const uint32_t x_lo = (s_lo + ((uint32_t)Cfg::kX >> 4)) | (1u << 16);
                if (FUSED) {
                    tc_fence_after();
                    if (p.r) {                   // T: A (MN-major, 64 ranks; its leading offset of 0 repeats them in the other 64 rows) times X in bf16
                        const uint32_t idt = umma_idesc(kCFmtF32, kFmtBF16, 128, 16) | (1u << 15);
#pragma unroll
                        for (int u = 0; u < 4; ++u)
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const int n = 16 * i + 4 * u + k;
                                const uint32_t a_lo = s_lo + ((uint32_t)(Cfg::kA + u * kAtomBytes) >> 4);
                                const uint32_t r_lo = (s_lo + ((uint32_t)(Cfg::kRaw + u * 2048) >> 4)) | (1u << 16);
                                umma_f16<1>(tmem + kMsTCol + (uint32_t)(n % kMsTRot) * 16u, make_desc(a_lo + k * 128, kDescHi), make_desc(r_lo + k * 2, kDescHi), idt,
                                            n >= kMsTRot);
                            }
                    }
                    if (!mbar_wait(quant0 + 8u * s, (uint32_t)(i / kMsStages) & 1u, abort_flag)) { ok = false; break; }
                }
                if (i < nb) {
                    const uint32_t slot = (uint32_t)i % kMsSfSlots, sfa = tmem + kMsSfCol + slot * kMsSfSlot, sfb = sfa + 8;
                    // the MMAs that read this scale slot are done (with three stages the refilled stage has said so)
                    if (i >= kMsSfSlots && kMsSfSlots < kMsStages) {
                        const int j = i - kMsSfSlots;
                        if (!mbar_wait(empty0 + 8u * (uint32_t)(j % kMsStages), (uint32_t)(j / kMsStages) & 1u, abort_flag)) { ok = false; break; }
                    }
                    tc_fence_after();
                    const uint32_t sf_lo = s_lo + ((uint32_t)Cfg::kSf >> 4);
#pragma unroll
                    for (int kt = 0; kt < 2; ++kt) {
                        tmem_cp_scales(sfa + kt * 4, make_desc(sf_lo + kt * 32, kMxSfDescHi));
                        tmem_cp_scales(sfb + kt * 4, make_desc(sf_lo + 64 + kt * 32, kMxSfDescHi));
                    }
                    const int nmma = b0 + i == p.nblk - 1 ? p.nmma_last : 4;
                    const uint32_t w_lo = s_lo | (1u << 16);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (k < nmma) {
                            const uint32_t id = kMsIdesc | idn | ((uint32_t)(k & 1) << 30) | ((uint32_t)(k & 1) << 5);
                            umma_mxf4(tmem, make_desc(w_lo + k * 2, kDescHi), make_desc(x_lo + k * 2, kDescHi), id, sfa + (k >> 1) * 4, sfb + (k >> 1) * 4,
                                      accumulate);
                            accumulate = 1;
                        }
                } else {
                    tc_fence_after();
                    const uint32_t idl = umma_idesc(kCFmtF32, kFmtBF16, 128, 0) | idn | (1u << 15);      // A (LoRA B) is MN-major
                    const uint32_t w_lo = s_lo | ((uint32_t)(kAtomBytes >> 4) << 16);
                    for (int k = 0; k < p.rp / 16; ++k) umma_f16<1>(tmem, make_desc(w_lo + k * 128, kDescHi), make_desc(x_lo + k * 2, kDescHi), idl, 1);
                }
                umma_commit<1>(empty0 + 8u * s);
            }
            if (ok) umma_commit<1>(acc_full);
        }
    } else {
        const int q = warp & 3, row = q * 32 + lane;
        if (FUSED) {
            // thread = token, one of a stage's eight blocks
            const int t = row & 15, bq = row >> 4;
            bool ok = true;
            for (int i = 0; i < b1 - b0 && ok; ++i) {
                const uint32_t s = (uint32_t)(i % kMsStages);
                if (!mbar_wait(full0 + 8u * s, (uint32_t)(i / kMsStages) & 1u, abort_flag)) { ok = false; break; }
                unsigned char* st = smem_dyn + (base - raw) + (size_t)s * kMsStageBytes;
                const unsigned char* src = st + Cfg::kRaw + (bq >> 1) * 2048 + t * 128;
                uint4 v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = *reinterpret_cast<const uint4*>(src + ((((bq & 1) * 4 + j) ^ (t & 7)) * 16));
                uint32_t c[4], byte;
                mx4_quantize_block(v, c, byte);
                *reinterpret_cast<uint4*>(st + Cfg::kX + t * 128 + ((bq ^ (t & 7)) * 16)) = make_uint4(c[0], c[1], c[2], c[3]);
                st[Cfg::kSf + 1024 + (bq >> 2) * 512 + t * 16 + (bq & 3)] = (uint8_t)byte;
                fence_proxy_async();             // the tensor core reads them
                __syncwarp();
                if (lane == 0) mbar_arrive(quant0 + 8u * s);
            }
            pdl_wait();
            // this thread's column of B, on its way while the tensor core works: two ranks per register
            const bool in = n0 + row_of < p.N;
#pragma unroll
            for (int j = 0; j < 32; ++j)
                if (2 * j < p.r && in)
                    b2[j] = (uint32_t)__ldg(p.B + (int64_t)(2 * j) * p.N + n0 + row_of) | (uint32_t)__ldg(p.B + (int64_t)(2 * j + 1) * p.N + n0 + row_of) << 16;
        }
        if (mbar_wait(acc_full, 0, abort_flag)) {
            tc_fence_after();
            float* part = reinterpret_cast<float*>(smem_dyn + (base - raw));
            if (FUSED && p.r && q < 2) {         // T: the lane's rank, sixteen tokens
                float sum[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) sum[j] = 0.0f;
#pragma unroll 1
                for (int a = 0; a < kMsTRot; ++a) {
                    uint32_t r[16];
                    tmem_ld_32x16(tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(kMsTCol + a * 16), r);
                    tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 16; ++j) sum[j] += __uint_as_float(r[j]);
                }
#pragma unroll
                for (int j = 0; j < 16; ++j) part[Cfg::kTokens * 128 + row * 16 + j] = sum[j];
            }
            for (int c = 0; c < p.nt; c += 16) {
                uint32_t r[16];
                tmem_ld_32x16(tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)c, r);
                tmem_ld_wait();
#pragma unroll
                for (int j = 0; j < 16; ++j) part[(c + j) * 128 + row] = __uint_as_float(r[j]);
            }
        }
        if (!FUSED) pdl_wait();          // Y may belong to work in front of this kernel until here
    }

    tc_fence_before();
    __syncthreads();
    if (p.ranks > 1) cluster_sync();
    if (FUSED && warp >= 2 && !abort_flag->flag) {
        // this rank's tokens, a thread per output column; their T first, put together from the ranks' shares
        const int tokens = p.M > rank ? (p.M - rank + p.ranks - 1) / p.ranks : 0;
        float* sum_t = reinterpret_cast<float*>(smem_dyn + (base - raw)) + Cfg::kPartFloats;      // [token][64]
        if (p.r) {
            for (int i = row_of; i < tokens * 64; i += 128) {
                const int j = i & 63, token = rank + (i >> 6) * p.ranks;
                const uint32_t at = base + (uint32_t)(Cfg::kTokens * 128 + j * 16 + token) * 4u;
                float v[8], s = 0.0f;
#pragma unroll
                for (int r = 0; r < 8; ++r)
                    if (r < p.ranks) v[r] = p.ranks > 1 ? __uint_as_float(ld_cluster_u32(mapa_shared(at, r))) : *reinterpret_cast<const float*>(smem_dyn + (at - raw));
#pragma unroll
                for (int r = 0; r < 8; ++r) if (r < p.ranks) s += v[r];
                sum_t[i] = s;
                if (n0 == 0 && j < p.r) p.T[(int64_t)token * p.r + j] = (uint16_t)(pack_bf16x2(s, 0.0f) & 0xFFFFu);
            }
            named_bar_sync(1, 128);
        }
        for (int i = 0; i < tokens; ++i) {
            const int token = rank + i * p.ranks;
            const uint32_t at = base + (uint32_t)(token * 128 + row_of) * 4u;
            float v[8], y = 0.0f, l0 = 0.0f, l1 = 0.0f;
#pragma unroll
            for (int r = 0; r < 8; ++r)
                if (r < p.ranks) v[r] = p.ranks > 1 ? __uint_as_float(ld_cluster_u32(mapa_shared(at, r))) : *reinterpret_cast<const float*>(smem_dyn + (at - raw));
#pragma unroll
            for (int r = 0; r < 8; ++r) if (r < p.ranks) y += v[r];
#pragma unroll
            for (int j = 0; j < 32; ++j)
                if (2 * j < p.r) {
                    const float2 tj = *reinterpret_cast<const float2*>(sum_t + i * 64 + 2 * j);
                    l0 = fmaf(tj.x, bf16_lo(b2[j]), l0);
                    l1 = fmaf(tj.y, bf16_hi(b2[j]), l1);
                }
            if (p.r) y = fmaf(p.scale, l0 + l1, y);
            if (n0 + row_of < p.N) {
                const int64_t o = (int64_t)token * p.ldy + n0 + row_of;
                if (p.y_f32) reinterpret_cast<float*>(p.Y)[o] = y;
                else reinterpret_cast<uint16_t*>(p.Y)[o] = (uint16_t)(pack_bf16x2(y, 0.0f) & 0xFFFFu);
            }
        }
    }
    if (!FUSED && warp >= 2 && !abort_flag->flag) {
        // a warp takes a token, a lane four outputs; four tokens' loads are in flight at a time
        const int tokens = min(p.nt, p.M - t0), n = n0 + 4 * lane;
        const bool vec = (p.ldy & 3) == 0 && n + 4 <= p.N;
        const int step = 4 * p.ranks;
        for (int t = rank + (warp - 2) * p.ranks; t < tokens; t += 4 * step) {
            float4 y[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) y[u] = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int r = 0; r < p.ranks; ++r) {
                float4 v[4];
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (t + u * step < tokens) {
                        const uint32_t at = base + (uint32_t)((t + u * step) * 128 + 4 * lane) * 4u;
                        v[u] = p.ranks > 1 ? ld_cluster_f4(mapa_shared(at, r)) : *reinterpret_cast<const float4*>(smem_dyn + (at - raw));
                    }
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (t + u * step < tokens) { y[u].x += v[u].x; y[u].y += v[u].y; y[u].z += v[u].z; y[u].w += v[u].w; }
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (t + u * step >= tokens) continue;
                const int64_t o = (int64_t)(t0 + t + u * step) * p.ldy + n;
                const float e[4] = {y[u].x, y[u].y, y[u].z, y[u].w};
                const uint32_t lo = pack_bf16x2(e[0], e[1]), hi = pack_bf16x2(e[2], e[3]);
                if (p.y_f32) {
                    float* out = reinterpret_cast<float*>(p.Y) + o;
                    if (vec) *reinterpret_cast<float4*>(out) = y[u];
                    else
#pragma unroll
                        for (int j = 0; j < 4; ++j) if (n + j < p.N) out[j] = e[j];
                } else {
                    uint16_t* out = reinterpret_cast<uint16_t*>(p.Y) + o;
                    if (vec) *reinterpret_cast<uint2*>(out) = make_uint2(lo, hi);
                    else
#pragma unroll
                        for (int j = 0; j < 4; ++j) if (n + j < p.N) out[j] = (uint16_t)((j < 2 ? lo : hi) >> ((j & 1) * 16));
                }
            }
        }
    }
    if (abort_flag->flag) {
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);   // let copies in flight land before the CTA retires
        if (threadIdx.x == 0 && p.status) atomicExch(p.status, (int)QUAFF_ERR_TIMEOUT);
        __syncthreads();
    }
    __syncwarp();
    if (p.ranks > 1) cluster_sync();       // partial tiles stay until every rank has read them
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc<1>(tmem, kMsTmemCols);
    }
}

}  // namespace quaff
