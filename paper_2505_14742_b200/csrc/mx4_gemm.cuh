// Y = Xd Wd^T (+ s T B) with both operands in MXFP4: persistent, warp-specialised tcgen05 kernel on CTA pairs.
//
//   warp 0      : TMA producer - code tiles, scale tiles, and the two LoRA operands, into a ring of stages
//   warp 1      : TMEM allocation; MMA issue (the leader's elected lane, for the pair)
//   warp 6      : block scales, shared memory -> TMEM, up to four stages ahead (the leader's elected lane, for the pair)
//   warps 2..5  : epilogue - tcgen05.ld, conversion, stores
//
// The block scales are applied inside the tensor core (kind::mxf4, block_scale, 32 elements per scale), products and sums
// are exact fp4 x fp4 times a power of two, accumulated in fp32.  The accumulator therefore IS the result, and the LoRA
// term joins it as further kind::f16 MMAs on the same accumulator: s T (fp32) is handed over as bf16 parts, its rounding and
// what that leaves - two for a bf16 result (17 bits), three for an f32 one.
//
// A tile is 256 rows x 256 columns of a CTA pair.  One stage is 256 elements of the contraction (128 bytes per row): A
// 16 KB, this CTA's half of B 16 KB, the scales of its 128 rows of A 1 KB, the scales of ALL 256 rows of B 2 KB (each SM
// of a pair scales its own accumulator rows, so both hold every scale of B).
//
// TMEM (512 columns): two accumulators of 256 columns that share 96 of them - columns [0,256) and [160,416) - and four
// slots of 24 columns for the scales of a stage.  The epilogue drains the half with the shared columns first, after which
// the tensor pipe may begin the next tile while the other half is still being stored.  A scale slot is rewritten only when the
// MMAs that read it have completed (the commit that frees their smem stage tells).  A warp of its own copies the scales: with
// that between its MMAs the issuing thread left the pipe empty (8192 x 11008 x 4096 143 us; 132 with the copying warp).
// A stage is back 1.7 us after its MMAs, so the ring's depth counts: 4 stages 143 us, 5 132, 6 126 (for them the epilogue has one
// buffer per warp).
//
// Bound by the tensor pipe (an MMA of 256 x 256 x 64 takes 128 clocks at best, about 160 here) and, under load, by the power cap:
// with operands of zeros the first of these takes 10 us less.  Measured: 8192 x 11008 x 4096 125 us = 5.9 PFLOP/s, 0.90 of
// four times the measured bf16 rate; 8192 x 4096 x 11008 (a 180 MB result) 139 us; 4096 x 4096 x 4096 31 to 34.  With 16-byte
// stores from registers the second took 40 us more, with the halves drained 64 columns at a time 11 us more.
//
// The epilogue stages 32 rows x 128 bytes per warp in shared memory and stores them by TMA (whole lines); where Y's pitch
// does not allow that, and in the last columns where N does not fill 16 bytes (a tiled store writes whole 16-byte
// pieces), the warp stores row by row.
#pragma once

#include "mx4.cuh"
#include "umma_gemm.cuh"

namespace quaff {

constexpr int kMxTileM = 256, kMxTileN = 256;
constexpr int kMxABytes = 128 * 128, kMxBBytes = 128 * 128, kMxSfBytes = 3 * 1024;     // per CTA and stage
constexpr int kMxStageBytes = kMxABytes + kMxBBytes + kMxSfBytes;
constexpr int kMxStages = 6;
constexpr int kMxThreads = 224;
constexpr int kMxAccStep = 160;            // second accumulator's first column: 96 columns shared
constexpr int kMxSfCol = 416, kMxSfSlot = 24, kMxSfSlots = 4;
constexpr int kMxOutBytes = 4 * 4096;      // a buffer of 32 rows x 128 bytes per epilogue warp

struct Mx4GemmParams {
    CUtensorMap map_a, map_b;      // codes [rows][bytes]
    CUtensorMap map_sa, map_sb;    // scale tiles as rows of 128 bytes
    CUtensorMap map_y;             // boxes of 32 rows x 128 bytes
    CUtensorMap map_t, map_bt;     // LoRA: [M][parts rp] (s T in bf16 parts), B [r][N]
    int ktiles;                    // scale tiles per row band
    int sa_tiles, sb_tiles;        // row bands of the two scale arrays
    int nblk, nmma_last;           // stages of 256 elements; MMAs (64 elements) of the last one
    int rp;                        // LoRA rank rounded up to 16
    int lora_parts;                // bf16 parts of s T: stages of the LoRA term, 0: none
    int M, N, tiles_m, tiles_n, band_m;
    void* Y;
    int64_t ldy;
    int y_f32;
    int tma_cols;                  // boxes that end at or before this column are stored by TMA (0: none)
    int32_t* status;
};

struct Mx4Smem {
    uint64_t full[kMxStages], empty[kMxStages];
    uint64_t scales[kMxSfSlots];   // a slot's scales are in TMEM
    uint64_t acc_full;       // a tile's accumulator is complete
    uint64_t acc_shared;     // its 96 shared columns are drained (with the rest of their half)
    uint64_t acc_empty;      // all of it is drained
    uint32_t tmem_base;
    AbortCtl abort;
};
constexpr size_t kMxSmemBytes = (size_t)kMxStages * kMxStageBytes + kMxOutBytes + sizeof(Mx4Smem);
static_assert(kMxSmemBytes <= 232448, "a CTA has 227 KB");

// A position in the ring of stages
struct MxRing {
    uint32_t stage = 0, phase = 0;
    __device__ __forceinline__ void next(uint32_t n = 1) {
        stage += n;
        if (stage >= kMxStages) { stage -= kMxStages; phase ^= 1u; }       // n <= kMxStages
    }
};
// 2-D tiled store from shared memory; out-of-range rows and columns of the box are dropped
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* m, int x, int y, uint32_t smem_src) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];"
                 ::"l"(reinterpret_cast<uint64_t>(m)), "r"(x), "r"(y), "r"(smem_src)
                 : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void bulk_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void st_shared_v4(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// Instruction descriptor of kind::mxf4: e2m1 x e2m1, e8m0 scales, M = 256; the two scale-byte selectors are added per MMA
constexpr uint32_t kMxIdesc = (1u << 7) | (1u << 10) | ((uint32_t)(kMxTileN >> 3) << 17) | (1u << 23) | ((uint32_t)(kMxTileM >> 4) << 24);

__device__ __forceinline__ void umma_mxf4_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
        : "memory");
}
// 32 rows x 16 bytes of shared memory -> 4 TMEM columns, repeated in the four lane quarters, in both CTAs of the pair
__device__ __forceinline__ void tmem_cp_scales_pair(uint32_t taddr, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
// ... and their completion, on a barrier of this CTA
__device__ __forceinline__ void tmem_cp_commit_pair(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// descriptor of a 512-byte scale tile: no swizzle, groups of 8 rows x 16 bytes are 128 bytes apart
constexpr uint32_t kMxSfDescHi = (128u >> 4) | (1u << 14);

template <typename E> __device__ __forceinline__ uint32_t ld_shared_element(uint32_t addr) {
    uint32_t v;
    if (sizeof(E) == 4) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    else asm volatile("{\n\t.reg .u16 h;\n\tld.shared.u16 h, [%1];\n\tcvt.u32.u16 %0, h;\n\t}" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
// Up to 32 rows x 128 bytes out of a buffer with 128-byte swizzle, at any pitch: a store instruction covers neighbouring columns of
// a row, eight rows are on their way at a time.
template <typename E> __device__ __forceinline__ void mx4_store_columns(uint32_t buf, E* y, int64_t ldy, int rows, int cols, int lane) {
#pragma unroll 1
    for (int x = lane; x < cols; x += 32) {
        const int byte = x * (int)sizeof(E);
        uint32_t at[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) at[e] = buf + (uint32_t)(e * 128 + ((byte >> 4) ^ e) * 16 + (byte & 15));
        E* d = y + x;
#pragma unroll 1
        for (int r = 0; r < rows; r += 8) {
            uint32_t v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e] = ld_shared_element<E>(at[e]);
                at[e] += 1024;
            }
            if (r + 8 <= rows) {
#pragma unroll
                for (int e = 0; e < 8; ++e, d += ldy) *d = (E)v[e];
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e, d += ldy) if (r + e < rows) *d = (E)v[e];
            }
        }
    }
}

__global__ void __launch_bounds__(kMxThreads, 1) mx4_gemm_kernel(const __grid_constant__ Mx4GemmParams p) {
    extern __shared__ __align__(1024) unsigned char smem_dyn[];
    const uint32_t raw = smem_u32(smem_dyn), base = raw;
    if (base & 1023u) {                    // swizzled tiles need it, and six stages leave no room to round up
        if (threadIdx.x == 0 && p.status) atomicExch(p.status, (int)QUAFF_ERR_ALIGNMENT);
        return;
    }
    const uint32_t out_base = base + kMxStages * kMxStageBytes;
    Mx4Smem* sm = reinterpret_cast<Mx4Smem*>(smem_dyn + (out_base - raw) + kMxOutBytes);
    volatile AbortCtl* abort_flag = &sm->abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int unit = (int)(blockIdx.x >> 1), nunits = (int)(gridDim.x >> 1);
    const int ntiles = p.tiles_m * p.tiles_n;
    const uint32_t full0 = smem_u32(&sm->full[0]), empty0 = smem_u32(&sm->empty[0]);
    const uint32_t acc_full = smem_u32(&sm->acc_full), acc_shared = smem_u32(&sm->acc_shared), acc_empty = smem_u32(&sm->acc_empty);
    const uint32_t scales0 = smem_u32(&sm->scales[0]);
    const uint32_t lead_full0 = mapa_shared(full0, 0);
    const uint32_t lead_shared = mapa_shared(acc_shared, 0), lead_empty = mapa_shared(acc_empty, 0);

    if (threadIdx.x == 0) {
        for (int s = 0; s < kMxStages; ++s) { mbar_init(full0 + 8u * s, 1); mbar_init(empty0 + 8u * s, 1); }
        for (int s = 0; s < kMxSfSlots; ++s) mbar_init(scales0 + 8u * s, 1);
        mbar_init(acc_full, 1);
        mbar_init(acc_shared, 8);
        mbar_init(acc_empty, 8);
        sm->abort.flag = 0;
        sm->abort.peer = mapa_shared(smem_u32(&sm->abort.flag), rank ^ 1u);
        fence_barrier_init();
    }
    if (warp == 1) {
        tmem_alloc<2>(smem_u32(&sm->tmem_base), 512);
        tmem_relinquish<2>();
    }
    pdl_launch_dependents();
    tc_fence_before();
    __syncthreads();
    cluster_sync();
    tc_fence_after();
    const uint32_t tmem = sm->tmem_base;
    pdl_wait();

    if (warp == 0) {
        if (elect_one()) {
            prefetch_tmap(&p.map_a); prefetch_tmap(&p.map_b); prefetch_tmap(&p.map_sa); prefetch_tmap(&p.map_sb);
            MxRing ring;
            bool ok = true;
            for (int tile = unit; tile < ntiles && ok; tile += nunits) {
                int tm, tn;
                tile_coords(tile, p.tiles_m, p.tiles_n, p.band_m, tm, tn);
                const int m0 = tm * kMxTileM + (int)rank * 128, n0 = tn * kMxTileN + (int)rank * 128;
                // a band beyond the matrix takes the last band's scales: its rows are zero codes and are not stored
                const int sa = min(m0 >> 7, p.sa_tiles - 1) * p.ktiles * 4;
                const int sb0 = min(tn * 2, p.sb_tiles - 1) * p.ktiles * 4, sb1 = min(tn * 2 + 1, p.sb_tiles - 1) * p.ktiles * 4;
                for (int b = 0; b < p.nblk; ++b) {
                    if (!mbar_wait(empty0 + 8u * ring.stage, ring.phase ^ 1u, abort_flag)) { ok = false; break; }
                    const uint32_t bar = lead_full0 + 8u * ring.stage, dst = base + ring.stage * kMxStageBytes;
                    if (rank == 0) mbar_arrive_expect_tx(full0 + 8u * ring.stage, 2u * kMxStageBytes);
                    tma_load_2d<2>(dst, &p.map_a, b * 128, m0, bar);
                    tma_load_2d<2>(dst + kMxABytes, &p.map_b, b * 128, n0, bar);
                    const uint32_t sf = dst + kMxABytes + kMxBBytes;
                    tma_load_2d<2>(sf, &p.map_sa, 0, sa + b * 8, bar);
                    tma_load_2d<2>(sf + 1024, &p.map_sb, 0, sb0 + b * 8, bar);
                    tma_load_2d<2>(sf + 2048, &p.map_sb, 0, sb1 + b * 8, bar);
                    ring.next();
                }
                for (int l = 0; l < p.lora_parts && ok; ++l) {
                    if (!mbar_wait(empty0 + 8u * ring.stage, ring.phase ^ 1u, abort_flag)) { ok = false; break; }
                    const uint32_t bar = lead_full0 + 8u * ring.stage, dst = base + ring.stage * kMxStageBytes;
                    const uint32_t box = (uint32_t)p.rp * 128u;
                    if (rank == 0) mbar_arrive_expect_tx(full0 + 8u * ring.stage, 2u * (kMxABytes + 2u * box));
                    tma_load_2d<2>(dst, &p.map_t, l * p.rp, m0, bar);
                    tma_load_2d<2>(dst + kMxABytes, &p.map_bt, n0, 0, bar);
                    tma_load_2d<2>(dst + kMxABytes + kAtomBytes, &p.map_bt, n0 + 64, 0, bar);
                    ring.next();
                }
            }
        }
    } else if (warp == 1) {
        if (rank == 0 && elect_one()) {
            MxRing ring;
            uint32_t n = 0;                // block-scaled stages so far
            bool ok = true;
            int t = 0;
            for (int tile = unit; tile < ntiles && ok; tile += nunits, ++t) {
                const uint32_t acc = tmem + (uint32_t)((t & 1) * kMxAccStep);
                // tile t overwrites the columns it shares with tile t - 1, and others that tile t - 2 has given back before
                // tile t - 1's accumulator was handed to the epilogue (below)
                if (t > 0 && !mbar_wait(acc_shared, (uint32_t)((t - 1) & 1), abort_flag)) break;
                uint32_t accumulate = 0;
                for (int b = 0; b < p.nblk; ++b) {
                    const uint32_t slot = n % kMxSfSlots;
                    const uint32_t sfa = tmem + kMxSfCol + slot * kMxSfSlot, sfb = sfa + 8;
                    const uint32_t s_lo = ((base + ring.stage * kMxStageBytes) & 0x3FFFFu) >> 4;
                    const uint32_t a_lo = s_lo | (1u << 16), b_lo = (s_lo + (kMxABytes >> 4)) | (1u << 16);
                    const int nmma = b == p.nblk - 1 ? p.nmma_last : 4;
                    if (!mbar_wait(full0 + 8u * ring.stage, ring.phase, abort_flag) || !mbar_wait(scales0 + 8u * slot, (n / kMxSfSlots) & 1u, abort_flag)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (k < nmma) {      // scale bytes 0,1 (even k) or 2,3 (odd k) of the word of the 128-element tile
                            const uint32_t id = kMxIdesc | ((uint32_t)(k & 1) << 30) | ((uint32_t)(k & 1) << 5);
                            umma_mxf4_pair(acc, make_desc(a_lo + k * 2, kDescHi), make_desc(b_lo + k * 2, kDescHi), id, sfa + (k >> 1) * 4,
                                           sfb + (k >> 1) * 8, accumulate);
                            accumulate = 1;
                        }
                    umma_commit<2>(empty0 + 8u * ring.stage);
                    ring.next();
                    ++n;
                }
                if (!ok) break;
                const uint32_t idl = umma_idesc(kCFmtF32, kFmtBF16, kMxTileM, kMxTileN) | (1u << 16);     // B is MN-major
                for (int l = 0; l < p.lora_parts; ++l) {
                    if (!mbar_wait(full0 + 8u * ring.stage, ring.phase, abort_flag)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t s_lo = ((base + ring.stage * kMxStageBytes) & 0x3FFFFu) >> 4;
                    const uint32_t a_lo = s_lo | (1u << 16), b_lo = (s_lo + (kMxABytes >> 4)) | ((uint32_t)(kAtomBytes >> 4) << 16);
                    for (int k = 0; k < p.rp / 16; ++k)
                        umma_f16<2>(acc, make_desc(a_lo + k * 2, kDescHi), make_desc(b_lo + k * 128, kDescHi), idl, 1);
                    umma_commit<2>(empty0 + 8u * ring.stage);
                    ring.next();
                }
                // the epilogue takes one tile after the other, so waiting here costs it nothing
                if (!ok || (t > 0 && !mbar_wait(acc_empty, (uint32_t)((t - 1) & 1), abort_flag))) break;
                umma_commit<2>(acc_full);
            }
        }
    } else if (warp == 6) {
        // scales: shared memory -> their slot of TMEM, up to four stages ahead of the MMAs
        if (rank == 0 && elect_one()) {
            MxRing ring, old;                    // the stage whose scales come next; the block-scaled stage four before it
            uint32_t pos = 0, old_pos = 0, n = 0;
            int old_b = 0;
            bool ok = true;
            for (int tile = unit; tile < ntiles && ok; tile += nunits) {
                for (int b = 0; b < p.nblk; ++b) {
                    // Two things have to be over.  The MMAs that read this slot: their commit freed their stage, or, a full round of the ring
                    // later, the stage of the position one round before this one.  And that position itself, which may be a stage of the adapters
                    // that this warp passes over: until it is filled and used, the parity of its barrier is the one waited for below, and the
                    // wait would end before the copies of this position have landed.  (Neither barrier can be two phases off: what this
                    // warp saw filled last had waited for every position up to ten before this one, and nothing from here on is used without its scales.)
                    if (n >= kMxSfSlots && pos - old_pos < kMxStages) {
                        if (!mbar_wait(empty0 + 8u * old.stage, old.phase, abort_flag)) { ok = false; break; }
                    } else if (pos >= kMxStages) {
                        if (!mbar_wait(empty0 + 8u * ring.stage, ring.phase ^ 1u, abort_flag)) { ok = false; break; }
                    }
                    if (n >= kMxSfSlots) {
                        uint32_t step = 1;
                        if (++old_b == p.nblk) { old_b = 0; step += (uint32_t)p.lora_parts; }
                        old.next(step);
                        old_pos += step;
                    }
                    if (!mbar_wait(full0 + 8u * ring.stage, ring.phase, abort_flag)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t sf_lo = (((base + ring.stage * kMxStageBytes) & 0x3FFFFu) >> 4) + ((kMxABytes + kMxBBytes) >> 4);
                    const uint32_t slot = n % kMxSfSlots, sfa = tmem + kMxSfCol + slot * kMxSfSlot, sfb = sfa + 8;
#pragma unroll
                    for (int kt = 0; kt < 2; ++kt) {     // 128 elements of the contraction: 4 columns of A scales, 8 of B scales
                        tmem_cp_scales_pair(sfa + kt * 4, make_desc(sf_lo + kt * 32, kMxSfDescHi));
                        tmem_cp_scales_pair(sfb + kt * 8, make_desc(sf_lo + 64 + kt * 32, kMxSfDescHi));
                        tmem_cp_scales_pair(sfb + kt * 8 + 4, make_desc(sf_lo + 128 + kt * 32, kMxSfDescHi));
                    }
                    tmem_cp_commit_pair(scales0 + 8u * slot);
                    ring.next();
                    ++pos;
                    ++n;
                }
                ring.next((uint32_t)p.lora_parts);
                pos += (uint32_t)p.lora_parts;
            }
        }
    } else {
        const int q = warp & 3;
        const uint32_t s = out_base + (uint32_t)q * 4096u;            // this warp's store buffer
        const int width = p.y_f32 ? 32 : 64;                          // columns of 128 bytes
        int t = 0;
        for (int tile = unit; tile < ntiles; tile += nunits, ++t) {
            int tm, tn;
            tile_coords(tile, p.tiles_m, p.tiles_n, p.band_m, tm, tn);
            const int mw = tm * kMxTileM + (int)rank * 128 + q * 32, n0 = tn * kMxTileN;
            if (!mbar_wait(acc_full, (uint32_t)(t & 1), abort_flag)) break;
            tc_fence_after();
            const uint32_t lane_addr = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)((t & 1) * kMxAccStep);
            // 128 bytes of every row of this warp: w of lane = row, columns nc .. nc + width
            auto store = [&](int nc, const uint32_t (&w)[32]) {
                const bool whole = nc + width <= p.tma_cols;
                if (lane == 0) bulk_wait_read<0>();                   // the last store has read the buffer
                __syncwarp();
#pragma unroll
                for (int j = 0; j < 8; ++j)                           // 128-byte swizzle, as the store's tensor map has it
                    st_shared_v4(s + (uint32_t)lane * 128u + (uint32_t)((j ^ (lane & 7)) * 16), w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
                if (whole) {
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) {
                        tma_store_2d(&p.map_y, nc, mw, s);
                        bulk_commit();
                    }
                } else {
                    __syncwarp();
                    const int cols = min(width, p.N - nc), rows = min(32, p.M - mw);
                    if (p.y_f32) mx4_store_columns<uint32_t>(s, reinterpret_cast<uint32_t*>(p.Y) + (int64_t)mw * p.ldy + nc, p.ldy, rows, cols, lane);
                    else mx4_store_columns<uint16_t>(s, reinterpret_cast<uint16_t*>(p.Y) + (int64_t)mw * p.ldy + nc, p.ldy, rows, cols, lane);
                    __syncwarp();
                }
            };
            // The half that holds the shared columns first - the upper one of the first accumulator, the lower one of the second -
            // all of it into registers: the tensor pipe waits for no more than that.
#pragma unroll 1
            for (int half = 0; half < 2; ++half) {
                const int col = ((t & 1) ^ half) ? 0 : 128;
                const bool live = n0 + col < p.N && mw < p.M;         // uniform across the warp
                uint32_t r[4][32];
                if (live) {
#pragma unroll
                    for (int h = 0; h < 4; ++h) tmem_ld_32x32(lane_addr + (uint32_t)(col + 32 * h), r[h]);
                    tmem_ld_wait();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(half ? lead_empty : lead_shared);
                if (!live) continue;
                if (p.y_f32) {
#pragma unroll
                    for (int h = 0; h < 4; ++h) if (n0 + col + 32 * h < p.N) store(n0 + col + 32 * h, r[h]);
                } else {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t w[32];
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            w[j] = pack_bf16x2(__uint_as_float(r[2 * h + j / 16][2 * (j % 16)]), __uint_as_float(r[2 * h + j / 16][2 * (j % 16) + 1]));
                        if (n0 + col + 64 * h < p.N) store(n0 + col + 64 * h, w);
                    }
                }
            }
        }
        if (lane == 0) bulk_wait_all();
    }

    tc_fence_before();
    __syncthreads();
    if (abort_flag->flag) {
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);   // let copies in flight land before the CTA retires
        if (threadIdx.x == 0 && p.status) atomicExch(p.status, (int)QUAFF_ERR_TIMEOUT);
        __syncthreads();
    }
    cluster_sync();       // neither CTA of the pair may retire while its partner still uses its memory or barriers
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc<2>(tmem, 512);
    }
}

}  // namespace quaff
