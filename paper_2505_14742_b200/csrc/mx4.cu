// MXFP4: quantization, its inverse, and the product of two MXFP4 operands (with a LoRA term).
#include <string.h>

#include <mutex>

#include "mx4_skinny.cuh"
#include "mx4_small.cuh"

namespace quaff {

// ------------------------------------------------------------------ quantization and back
// Both kernels move 2.53 bytes per element and are bound by HBM.  A scale tile holds the four blocks of rows i, i + 32,
// i + 64, i + 96 in 16 consecutive bytes, so that is the work of sixteen lanes: four rows x 128 columns, a lane has eight
// columns of each row.  That makes four independent 128-bit loads (bf16) per thread, one 32-bit store of codes per row, and
// one 128-bit store of scales per sixteen lanes; two such groups of a warp take neighbouring columns.
// Measured at 8192 x 11008: quantize 41 us from bf16 (5.6 TB/s), 59 us from f32 (6.9 TB/s), back to bf16 36 us (6.4 TB/s);
// with one row per thread (one load in flight, 4-byte scale stores) 75 and 53 us.
constexpr int kMxqThreads = 256;

struct Mx4Item { int row0, kt, l; bool in; };      // first row, scale tile, lane of the group
__device__ __forceinline__ Mx4Item mx4_item(int ktiles, int band, int item) {      // item: of 32 row groups x pairs of scale tiles, a warp each
    const int pairs = (ktiles + 1) >> 1;
    Mx4Item it;
    const int i = item / pairs;
    it.kt = 2 * (item - i * pairs) + ((threadIdx.x >> 4) & 1);
    it.l = threadIdx.x & 15;
    it.row0 = band * kMx4TileRows + i;
    it.in = i < 32 && it.kt < ktiles;
    return it;
}
__device__ __forceinline__ Mx4Item mx4_item(int ktiles) {
    return mx4_item(ktiles, (int)blockIdx.y, blockIdx.x * (kMxqThreads / 32) + (threadIdx.x >> 5));
}
static dim3 mx4_grid(int rows, int ktiles) {
    return dim3((unsigned)ceil_div(32 * ((ktiles + 1) / 2), kMxqThreads / 32), (unsigned)mx4_row_tiles(rows));
}

template <bool F32>
__global__ void __launch_bounds__(kMxqThreads) mx4_quantize_kernel(const void* __restrict__ X, int64_t ldx, int M, int K, int ktiles,
                                                                 uint8_t* __restrict__ codes, int64_t ldc, uint8_t* __restrict__ scales) {
    pdl_launch_dependents();
    pdl_wait();
    const Mx4Item it = mx4_item(ktiles);
    const int k0 = it.kt * 128 + it.l * 8;
    constexpr int kWords = F32 ? 8 : 4;
    uint32_t raw[4][kWords];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int row = it.row0 + 32 * j;
#pragma unroll
        for (int e = 0; e < kWords; ++e) raw[j][e] = 0;
        if (it.in && row < M && k0 < K) {
            if (F32) {
                const uint32_t* src = reinterpret_cast<const uint32_t*>(X) + (int64_t)row * ldx + k0;
                if (k0 + 8 <= K) {
                    const uint4 a = __ldg(reinterpret_cast<const uint4*>(src)), b = __ldg(reinterpret_cast<const uint4*>(src) + 1);
                    raw[j][0] = a.x; raw[j][1] = a.y; raw[j][2] = a.z; raw[j][3] = a.w;
                    raw[j][kWords - 4] = b.x; raw[j][kWords - 3] = b.y; raw[j][kWords - 2] = b.z; raw[j][kWords - 1] = b.w;
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) if (k0 + e < K) raw[j][e % kWords] = __ldg(src + e);
                }
            } else {
                const uint16_t* src = reinterpret_cast<const uint16_t*>(X) + (int64_t)row * ldx + k0;
                if (k0 + 8 <= K) {
                    const uint4 a = __ldg(reinterpret_cast<const uint4*>(src));
                    raw[j][0] = a.x; raw[j][1] = a.y; raw[j][2] = a.z; raw[j][3] = a.w;
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) if (k0 + e < K) raw[j][e >> 1] |= (uint32_t)__ldg(src + e) << ((e & 1) * 16);
                }
            }
        }
    }
    uint32_t word[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        // the block's largest magnitude, on bit patterns (ordered like the values): its exponent field is exact for any input
        uint32_t top;
        if (F32) {
            top = 0;
#pragma unroll
            for (int e = 0; e < kWords; ++e) top = max(top, raw[j][e] & 0x7FFFFFFFu);
            top >>= 23;
        } else {
            uint32_t m2 = 0;
#pragma unroll
            for (int e = 0; e < kWords; ++e) m2 = __vmaxu2(m2, raw[j][e] & 0x7FFF7FFFu);
            top = max(m2 & 0xFFFFu, m2 >> 16) >> 7;
        }
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
        const uint32_t byte = mx4_scale_of(top);
        const float inv = mx4_inv_scale(byte);
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = F32 ? __uint_as_float(raw[j][e % kWords]) : ((e & 1) ? bf16_hi(raw[j][(e >> 1) % kWords]) : bf16_lo(raw[j][(e >> 1) % kWords]));
            v[e] = __fmul_rn(x, inv);
        }
        uint32_t c = mx4_pack8(v);
        if (byte == 255u) c = 0;                                  // infinity or NaN times 0 above
        const int row = it.row0 + 32 * j;
        if (it.in && row < M && (k0 & ~31) < K)                   // every block that holds a column is written whole
            *reinterpret_cast<uint32_t*>(codes + (int64_t)row * ldc + (k0 >> 1)) = c;
        // the four blocks' scale bytes -> one word (lanes 0, 4, 8, 12 of the group)
        uint32_t w = byte << ((it.l >> 2) * 8);
        w |= __shfl_xor_sync(0xFFFFFFFFu, w, 4);
        w |= __shfl_xor_sync(0xFFFFFFFFu, w, 8);
        word[j] = w;
    }
    if (it.in && it.l == 0) *reinterpret_cast<uint4*>(scales + mx4_scale_offset(it.row0, it.kt * 4, ktiles)) = make_uint4(word[0], word[1], word[2], word[3]);
}

quaff_status_t mx4_quantize_launch(const void* X, int x_dtype, int64_t ldx, int M, int K, uint8_t* codes, int64_t ldc, uint8_t* scales,
                                   cudaStream_t st) {
    const int ktiles = mx4_ktiles(K);      // rows and blocks of padding too: their scales are written
    const dim3 grid = mx4_grid(M, ktiles);
    if (x_dtype == QUAFF_F32) launch_pdl(mx4_quantize_kernel<true>, grid, dim3(kMxqThreads), 0, st, 1, X, ldx, M, K, ktiles, codes, ldc, scales);
    else launch_pdl(mx4_quantize_kernel<false>, grid, dim3(kMxqThreads), 0, st, 1, X, ldx, M, K, ktiles, codes, ldc, scales);
    return launch_status();
}

// Back to bf16 (exact: two significant bits times a power of two)
__device__ __forceinline__ void mx4_dequantize_item(const Mx4Item& it, const uint8_t* __restrict__ codes, int64_t ldc, const uint8_t* __restrict__ scales,
                                                    int M, int K, int ktiles, uint16_t* __restrict__ out, int64_t ldo) {
    const int k0 = it.kt * 128 + it.l * 8;
    if (!it.in || k0 >= K) return;
    uint32_t c[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
        c[j] = it.row0 + 32 * j < M ? __ldg(reinterpret_cast<const uint32_t*>(codes + (int64_t)(it.row0 + 32 * j) * ldc + (k0 >> 1))) : 0u;
    const uint4 sw = __ldg(reinterpret_cast<const uint4*>(scales + mx4_scale_offset(it.row0, it.kt * 4, ktiles)));
    const uint32_t word[4] = {sw.x, sw.y, sw.z, sw.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int row = it.row0 + 32 * j;
        const float s = mx4_scale_value((word[j] >> ((it.l >> 2) * 8)) & 255u);
        uint32_t h[4], w[4];
        mx4_unpack8(c[j], h);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&h[e]));
            w[e] = pack_bf16x2(__fmul_rn(v.x, s), __fmul_rn(v.y, s));
        }
        uint16_t* dst = out + (int64_t)row * ldo + k0;
        if (row < M) {
            if (k0 + 8 <= K) *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
            else
                for (int e = 0; e < 8; ++e) if (k0 + e < K) dst[e] = (uint16_t)(w[e >> 1] >> ((e & 1) * 16));
        }
    }
}
__global__ void __launch_bounds__(kMxqThreads) mx4_dequantize_kernel(const uint8_t* __restrict__ codes, int64_t ldc, const uint8_t* __restrict__ scales,
                                                                   int M, int K, int ktiles, uint16_t* __restrict__ out, int64_t ldo) {
    pdl_launch_dependents();
    pdl_wait();
    mx4_dequantize_item(mx4_item(ktiles), codes, ldc, scales, M, K, ktiles, out, ldo);
}

quaff_status_t mx4_dequantize_launch(const uint8_t* codes, int64_t ldc, const uint8_t* scales, int M, int K, uint16_t* out, int64_t ldo,
                                     cudaStream_t st) {
    const int ktiles = mx4_ktiles(K);
    launch_pdl(mx4_dequantize_kernel, mx4_grid(M, ktiles), dim3(kMxqThreads), 0, st, 1, codes, ldc, scales, M, K, ktiles, out, ldo);
    return launch_status();
}

// ------------------------------------------------------------------ product
// ---- few tokens: codes, scales, T and the parts of s T in one launch
// A cluster of eight CTAs per token, each with an eighth of the columns (whole scale tiles): the columns are quantized and kept
// in shared memory as floats for their share of x A, the shares are added up through distributed shared memory in rank
// order.  A is read once per token (from L2), so this is for few of them; what it saves is two launches.
constexpr int kPrepThreads = 256, kPrepCtas = 8, kPrepSlice = 4096;      // columns of a CTA at most
struct Mx4PrepParams {
    const uint16_t* X;
    int64_t ldx;
    int M, K, ktiles, slice;
    uint8_t* codes;
    int64_t ldc;
    uint8_t* scales;
    const uint16_t* A;
    int r, rp, parts;
    float scale;
    uint16_t *T, *Tp;
};
__global__ void __launch_bounds__(kPrepThreads) mx4_prep_kernel(const Mx4PrepParams p) {
    __shared__ float xs[kPrepSlice];
    __shared__ float red[kPrepThreads * 8];
    __shared__ float sums[64];
    pdl_wait();
    pdl_launch_dependents();      // only now: what starts early behind this kernel may rely on all work in front of it
    const int rank = (int)cluster_ctarank(), row = (int)blockIdx.x / kPrepCtas, tid = threadIdx.x;
    const int k_begin = rank * p.slice, n = max(0, min(p.slice, p.K - k_begin));
    const int tiles_end = max(0, min(p.slice, p.ktiles * 128 - k_begin));          // to the end of the last scale tile
    // x A takes eight columns of A per thread, rows dealt over the threads; the first rows are on their way during the quantization
    const int g = max(p.r >> 3, 1), lanes = kPrepThreads / g, kk = tid / g, j8 = tid - kk * g;
    const uint4* a = reinterpret_cast<const uint4*>(p.A + (int64_t)(k_begin + kk) * p.r) + j8;
    uint4 ahead[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) ahead[i] = p.r && kk < lanes && kk + i * lanes < n ? __ldg(a + (int64_t)i * lanes * g) : make_uint4(0, 0, 0, 0);
    for (int c0 = tid * 8; c0 - (tid & 31) * 8 < tiles_end; c0 += kPrepThreads * 8) {
        const int k0 = k_begin + c0;
        float v[8];
        uint32_t m2 = 0;
        uint32_t raw[4] = {0, 0, 0, 0};
        if (c0 < tiles_end && k0 < p.K) {
            const uint16_t* src = p.X + (int64_t)row * p.ldx + k0;
            if (k0 + 8 <= p.K) {
                const uint4 a = __ldg(reinterpret_cast<const uint4*>(src));
                raw[0] = a.x; raw[1] = a.y; raw[2] = a.z; raw[3] = a.w;
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) if (k0 + e < p.K) raw[e >> 1] |= (uint32_t)__ldg(src + e) << ((e & 1) * 16);
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            m2 = __vmaxu2(m2, raw[e] & 0x7FFF7FFFu);
            v[2 * e] = bf16_lo(raw[e]);
            v[2 * e + 1] = bf16_hi(raw[e]);
            if (c0 < tiles_end) { xs[c0 + 2 * e] = v[2 * e]; xs[c0 + 2 * e + 1] = v[2 * e + 1]; }
        }
        uint32_t top = max(m2 & 0xFFFFu, m2 >> 16) >> 7;
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
        const uint32_t byte = mx4_scale_of(top);
        const float inv = mx4_inv_scale(byte);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __fmul_rn(v[e], inv);
        uint32_t c = mx4_pack8(v);
        if (byte == 255u) c = 0;
        if (c0 < tiles_end && (k0 & ~31) < p.K) *reinterpret_cast<uint32_t*>(p.codes + (int64_t)row * p.ldc + (k0 >> 1)) = c;
        uint32_t w = byte << (((tid >> 2) & 3) * 8);
        w |= __shfl_xor_sync(0xFFFFFFFFu, w, 4);
        w |= __shfl_xor_sync(0xFFFFFFFFu, w, 8);
        if ((tid & 15) == 0 && c0 < tiles_end) *reinterpret_cast<uint32_t*>(p.scales + mx4_scale_offset(row, k0 >> 5, p.ktiles)) = w;
    }
    if (p.r == 0) return;         // the same for all CTAs
    __syncthreads();
    float acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (kk < lanes) {
        auto add = [&](float x, const uint4& w) {
            acc[0] = fmaf(x, bf16_lo(w.x), acc[0]); acc[1] = fmaf(x, bf16_hi(w.x), acc[1]);
            acc[2] = fmaf(x, bf16_lo(w.y), acc[2]); acc[3] = fmaf(x, bf16_hi(w.y), acc[3]);
            acc[4] = fmaf(x, bf16_lo(w.z), acc[4]); acc[5] = fmaf(x, bf16_hi(w.z), acc[5]);
            acc[6] = fmaf(x, bf16_lo(w.w), acc[6]); acc[7] = fmaf(x, bf16_hi(w.w), acc[7]);
        };
#pragma unroll
        for (int i = 0; i < 4; ++i) if (kk + i * lanes < n) add(xs[kk + i * lanes], ahead[i]);
#pragma unroll 4
        for (int k = kk + 4 * lanes; k < n; k += lanes) add(xs[k], __ldg(a + (int64_t)(k - kk) * g));
#pragma unroll
        for (int e = 0; e < 8; ++e) red[kk * p.r + j8 * 8 + e] = acc[e];
    }
    __syncthreads();
    const int groups = kPrepThreads / p.r, gj = tid / p.r, j = tid - gj * p.r;     // rows of `red` in `groups` interleaved sets
    float s = 0.0f;
    if (gj < groups) for (int i = gj; i < lanes; i += groups) s += red[i * p.r + j];
    __syncthreads();
    if (gj < groups) red[gj * p.r + j] = s;
    __syncthreads();
    if (tid < p.r) {
        s = 0.0f;
        for (int i = 0; i < groups; ++i) s += red[i * p.r + tid];
        sums[tid] = s;
    }
    __syncwarp();
    cluster_sync();
    if (rank == 0 && tid < p.rp) {
        float v = 0.0f;
        if (tid < p.r) {
            for (int q = 0; q < kPrepCtas; ++q) v += __uint_as_float(ld_cluster_u32(mapa_shared(smem_u32(&sums[tid]), q)));
            p.T[(int64_t)row * p.r + tid] = (uint16_t)(pack_bf16x2(v, 0.0f) & 0xFFFFu);
        }
        v = __fmul_rn(p.scale, v);
        for (int i = 0; i < p.parts; ++i) p.Tp[((int64_t)row * p.parts + i) * p.rp + tid] = (uint16_t)bf16_part(v);
    }
    __syncwarp();
    cluster_sync();               // the partners' sums stay until they are read
}
// Up to here the one launch of a cluster per token is the faster way; A is read M times.  The whole layer, 4096 x 4096, r = 16:
// 1 token 8.8 us, 32 tokens 11.4; 33 tokens through the pass over row tiles 14.4.
static bool mx4_use_prep(int M, int K, int r) { return (int64_t)M * max(r, 8) <= 512 && K <= kPrepCtas * kPrepSlice; }
static quaff_status_t launch_mx4_prep(const uint16_t* X, int64_t ldx, int M, int K, uint8_t* codes, int64_t ldc, uint8_t* scales, const uint16_t* A, int r,
                                      int parts, float scale, uint16_t* T, uint16_t* Tp, cudaStream_t st) {
    const int slice = (ceil_div(K, kPrepCtas) + 127) / 128 * 128;
    const Mx4PrepParams p = {X, ldx, M, K, mx4_ktiles(K), slice, codes, ldc, scales, A, r, (r + 15) / 16 * 16, parts, scale, T, Tp};
    launch_pdl(mx4_prep_kernel, dim3((unsigned)M * kPrepCtas), dim3(kPrepThreads), 0, st, kPrepCtas, p);
    return launch_status();
}

// ---- the two product kernels
struct Mx4Operands {
    int M, K, N;
    const uint8_t* Xc; int64_t ldxc; const uint8_t* Xs;
    const uint8_t* Wc; int64_t ldwc; const uint8_t* Ws;
    const uint16_t* Tp; const quaff_bf16* B; int r, parts;      // LoRA: s T in bf16 parts, B; r = 0: none
    void* Y; int y_dtype; int64_t ldy;
    int32_t* status;
};

// What the device can hold at once: clusters of 1 .. 8 CTAs of the small kernel and of the skinny products, CTA pairs of the large one.  (A GPC takes whole
// clusters only: of 148 SMs, clusters of eight reach fewer than 128.)
struct Mx4Device {
    std::once_flag once;
    bool ok = false;
    int clusters[9], skinny[9], pairs;
};
__global__ void mx4_front_kernel(const __grid_constant__ Mx4FrontParams p);
template <int MODE> static bool skinny_attr() {
    return cudaFuncSetAttribute(mx4_skinny_kernel<MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)skinny_smem<MODE>()) == cudaSuccess;
}
static Mx4Device* mx4_device() {
    static Mx4Device per_dev[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return nullptr;
    Mx4Device& d = per_dev[dev];
    std::call_once(d.once, [&d] {
        d.ok = cudaFuncSetAttribute(mx4_gemm_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMxSmemBytes) == cudaSuccess &&
               cudaFuncSetAttribute(mx4_front_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)skinny_smem<kSkinnyParts>()) == cudaSuccess &&
               skinny_attr<kSkinnyDown>() && skinny_attr<kSkinnyParts>() && skinny_attr<kSkinnyFold>() && skinny_attr<kSkinnyTurned>() &&
               cudaFuncSetAttribute(mx4_small_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)ms_smem<false>()) == cudaSuccess &&
               cudaFuncSetAttribute(mx4_small_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)ms_smem<true>()) == cudaSuccess;
        auto fits = [](auto kernel, int cluster, int threads, size_t smem) {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3((unsigned)(sm_count() / cluster * cluster));
            cfg.blockDim = dim3((unsigned)threads);
            cfg.dynamicSmemBytes = smem;
            cudaLaunchAttribute attr;
            attr.id = cudaLaunchAttributeClusterDimension;
            attr.val.clusterDim.x = (unsigned)cluster; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
            cfg.attrs = &attr;
            cfg.numAttrs = 1;
            int n = 0;
            if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n <= 0) { cudaGetLastError(); n = 1; }
            return min(n, max(1, sm_count() / cluster));
        };
        d.clusters[0] = d.skinny[0] = 0;
        d.clusters[1] = d.skinny[1] = sm_count();
        for (int c = 2; c <= 8; ++c) {
            d.clusters[c] = fits(mx4_small_kernel<false>, c, kMsThreads, ms_smem<false>());
            d.skinny[c] = fits(mx4_skinny_kernel<kSkinnyFold>, c, kSkThreads, skinny_smem<kSkinnyFold>());      // (the modes differ little in size)
        }
        d.pairs = fits(mx4_gemm_kernel, 2, kMxThreads, kMxSmemBytes);
    });
    return d.ok ? &d : nullptr;
}

// ---- the skinny products
quaff_status_t mx4_skinny_prepare(SkinnyParams& p, int mode, const void* A, int64_t lda, const void* B, int64_t ldb, int rows, int kc, int r, int cols,
                                  int32_t* status) {
    const Mx4Device* d = mx4_device();
    if (!d) return QUAFF_ERR_CUDA;
    memset(&p, 0, sizeof(p));
    const bool a_mn = mode >= kSkinnyFold, b_mn = mode != kSkinnyParts;
    p.r = r;
    p.rp = (r + 15) / 16 * 16;
    p.cols = (cols + 15) / 16 * 16;
    quaff_status_t rc = a_mn ? make_tmap_2d(&p.map_a, A, 2, kc, rows, lda, 64, 64) : make_tmap_2d(&p.map_a, A, 2, rows, kc, lda, 128, 64);
    if (rc != QUAFF_OK) return rc;
    rc = b_mn ? make_tmap_2d(&p.map_b, B, 2, kc, cols, ldb, 64, 64) : make_tmap_2d(&p.map_b, B, 2, cols, kc, ldb, p.cols, 64);
    if (rc != QUAFF_OK) return rc;
    p.tx_bytes = 16384u + (b_mn ? (uint32_t)ceil_div(p.cols, 64) * kAtomBytes : (uint32_t)p.cols * 128u);
    p.M = rows;
    p.nst = ceil_div(kc, 64);
    // as many slices of a row tile as run in one wave, four stages each at least
    const int tiles = ceil_div(rows, 128);
    int ranks = 1;
    for (int c = 2; c <= 8 && p.nst >= 4 * c; ++c) if (tiles <= d->skinny[c]) ranks = c;
    p.per = ceil_div(p.nst, ranks);
    p.ranks = ceil_div(p.nst, p.per);
    p.rot = 16;
    while (p.rot * p.cols > 512) p.rot /= 2;
    p.status = status;
    return QUAFF_OK;
}
template <int MODE> static void skinny_go(const SkinnyParams& p, cudaStream_t st) {
    launch_pdl(mx4_skinny_kernel<MODE>, dim3((unsigned)(ceil_div(p.M, 128) * p.ranks)), dim3(kSkThreads), skinny_smem<MODE>(), st, p.ranks, p);
}
quaff_status_t mx4_skinny_launch(const SkinnyParams& p, int mode, cudaStream_t st) {
    if (mode == kSkinnyDown) skinny_go<kSkinnyDown>(p, st);
    else if (mode == kSkinnyParts) skinny_go<kSkinnyParts>(p, st);
    else if (mode == kSkinnyFold) skinny_go<kSkinnyFold>(p, st);
    else skinny_go<kSkinnyTurned>(p, st);
    return launch_status();
}

// ---- what the backward needs first, in one launch: G, dB and the expanded weight, each with CTAs of its own
__global__ void __launch_bounds__(kSkThreads, 1) mx4_front_kernel(const __grid_constant__ Mx4FrontParams p) {
    const int block = (int)blockIdx.x;
    if (block < p.g_ctas) {
        mx4_skinny_body<kSkinnyParts>(p.g, block);
    } else if (block < p.g_ctas + p.db_ctas) {
        mx4_skinny_body<kSkinnyTurned>(p.db, block - p.g_ctas);
    } else {
        pdl_wait();
        pdl_launch_dependents();
        const int band = 32 * ((p.ktiles + 1) >> 1), warps = kSkThreads / 32;        // items of 128 rows
        for (int w = (block - p.g_ctas - p.db_ctas) * warps + (threadIdx.x >> 5); w < p.items; w += p.w_ctas * warps)
            mx4_dequantize_item(mx4_item(p.ktiles, w / band, w % band), p.codes, p.ldc, p.scales, p.N, p.K, p.ktiles, p.out, p.ldo);
    }
}
// CTAs of the three parts (and the slices of G's and dB's contractions) if all of them run in one wave, with two to kFrontStages
// stages per slice and at most kFrontItems items of the weight per warp; false if not.  Measured, us back to back (on the device), backward
// of tokens x columns x rows of W, one launch / three on three streams: 515 x 1000 x 1544, r = 8 24.9 / 28.5 (20.2 / 20.1); 1 x 1024 x 1024
// 27.2 / 36.1 (13.0 / 11.8); 1024 x 2048 x 2048 32.9 / 36.9 (30.4 / 28.5); 3000 x 4096 x 2048 61.2 / 67.8 (57.9 / 64.6); 512 x 2048 x 4096
// 33.4 / 37.1 (28.3 / 26.6).  Longer slices keep too few CTAs at work: 8192 x 1024 x 1024 (128 stages) 62.0 / 46.3 (58.6 / 41.1).  So the rule is for
// calls from the host, which it makes 4 to 9 us cheaper; in a captured step it costs up to 2 us.  It does not ask whether the stream is being captured:
// the slices, and with them the last bits of G and dB, would then differ between a call and its graph.
constexpr int kFrontItems = 8, kFrontStages = 48;
bool mx4_front_prepare(Mx4FrontParams& p, int M, bool want_db) {
    const Mx4Device* d = mx4_device();
    if (!d) return false;
    // The choice takes all three parts into account, wanted or not: which results are asked for does not change their bits.
    const int64_t all = (int64_t)32 * ((p.ktiles + 1) / 2) * mx4_row_tiles(p.N);
    if (all > (int64_t)kFrontItems * (kSkThreads / 32) * d->skinny[1]) return false;
    const int items = p.items = (int)all;
    const int g = ceil_div(M, 128), db = ceil_div(p.N, 128), g_nst = ceil_div(p.N, 64), db_nst = ceil_div(M, 64);
    int ranks = 0;
    for (int c = 1; c <= 8; ++c) {
        const int w = ceil_div(items, kSkThreads / 32 * kFrontItems * c);       // clusters of c CTAs
        if (g + db + w > d->skinny[c] || max(g_nst, db_nst) > kFrontStages * c) continue;
        if (c > 1 && min(g_nst, db_nst) < 2 * c) continue;
        ranks = c;
    }
    if (!ranks) return false;
    p.ranks = p.g.ranks = p.db.ranks = ranks;
    p.g.per = ceil_div(g_nst, ranks);
    p.db.per = ceil_div(db_nst, ranks);
    p.g_ctas = g * ranks;
    p.db_ctas = want_db ? db * ranks : 0;
    p.w_ctas = p.out ? min(d->skinny[ranks] - g - db, ceil_div(items, kSkThreads / 32 * ranks)) * ranks : 0;
    return true;
}
quaff_status_t mx4_front_launch(const Mx4FrontParams& p, cudaStream_t st) {
    launch_pdl(mx4_front_kernel, dim3((unsigned)(p.g_ctas + p.db_ctas + p.w_ctas)), dim3(kSkThreads), skinny_smem<kSkinnyParts>(), st, p.ranks, p);
    return launch_status();
}

// 128 x 128 tiles turned round, the contraction cut over a cluster, where that fills the SMs in one wave; else 256 x 256
// tiles of CTA pairs.  Measured, small / large tiles in us (tokens x columns x rows of W): 16 x 4096 x 4096 5.8 / 9.6,
// 64 x 11008 x 4096 9.9 / 17.6, 64 x 4096 x 18000 10.7 / 11.1, 256 x 11008 x 4096 15.4 / 18.4, 384 x 16384 x 2048 18.3 / 24.4.  From 65 tokens on
// the partial tiles are large, and a short contraction or a single rank does not pay for them: 127 x 1024 x 4096 8.5 / 7.1,
// 127 x 4096 x 11008 12.3 / 11.5, 384 x 11008 x 4096 21.4 / 19.1.  Over one wave the small tiles pay up to 32 tokens: 1 x 4096 x 32000
// 15.4 / 20.9, 32 x 4096 x 32000 16.8 / 19.7, 48 x 1024 x 32000 9.9 / 9.9, 64 x 4096 x 32000 19.2 / 17.0.
static int mx4_token_tile(int M) { return M >= kMsTokens ? kMsTokens : (M + 15) / 16 * 16; }
// k-blocks of a rank of the small kernel, 0: the large one
static int mx4_small_plan(const Mx4Device* d, int M, int N, int nblk) {
    const int64_t tiles = (int64_t)ceil_div(N, 128) * ceil_div(M, mx4_token_tile(M));
    int ranks = 1;
    for (int c = 2; c <= min(8, nblk); ++c) if (tiles <= d->clusters[c]) ranks = c;
    if (M > kMsTokens / 2 && (ranks == 1 || nblk < 16)) return 0;
    if (M > kMsTokens / 4 && tiles > d->clusters[1]) return 0;
    return ceil_div(nblk, ranks);
}

struct Mx4Launch { bool small; Mx4GemmParams big; Mx4SmallParams few; };
static quaff_status_t mx4_product_prepare(Mx4Launch& l, const Mx4Operands& o, bool after_prep) {
    const Mx4Device* dev = mx4_device();
    if (!dev) return QUAFF_ERR_CUDA;
    const uint64_t cols = (uint64_t)mx4_row_bytes(o.K);
    const int nblk = ceil_div(o.K, 256), nmma_last = ceil_div(o.K - (nblk - 1) * 256, 64), rp = (o.r + 15) / 16 * 16;
    quaff_status_t rc;
    const int per = mx4_small_plan(dev, o.M, o.N, nblk);
    l.small = per > 0;
    if (l.small) {
        Mx4SmallParams& p = l.few;
        memset(&p, 0, sizeof(p));
        p.nt = mx4_token_tile(o.M);
        p.row_tiles = ceil_div(o.N, 128);
        p.per = per;
        p.ranks = ceil_div(nblk, p.per);
        if ((rc = make_tmap_2d(&p.map_w, o.Wc, 1, o.N, cols, o.ldwc, 128, 128)) != QUAFF_OK) return rc;
        if ((rc = make_tmap_2d(&p.map_x, o.Xc, 1, o.M, cols, o.ldxc, p.nt, 128)) != QUAFF_OK) return rc;
        if ((rc = make_tmap_rows128(&p.map_sw, o.Ws, mx4_scale_bytes(o.N, o.K), 8)) != QUAFF_OK) return rc;
        if ((rc = make_tmap_rows128(&p.map_sx, o.Xs, mx4_scale_bytes(o.M, o.K), 8)) != QUAFF_OK) return rc;
        if (o.r > 0) {
            p.rp = rp;
            p.lora_parts = o.parts;
            if ((rc = make_tmap_2d(&p.map_t, o.Tp, 2, o.M, o.parts * rp, o.parts * rp, p.nt, 64)) != QUAFF_OK) return rc;
            if ((rc = make_tmap_2d(&p.map_b, o.B, 2, o.r, o.N, o.N, rp, 64)) != QUAFF_OK) return rc;
        }
        p.ktiles = mx4_ktiles(o.K);
        p.sw_tiles = mx4_row_tiles(o.N);
        p.sx_tiles = mx4_row_tiles(o.M);
        p.nblk = nblk;
        p.nmma_last = nmma_last;
        p.M = o.M; p.N = o.N;
        p.early_w = after_prep;
        p.Y = o.Y; p.ldy = o.ldy; p.y_f32 = o.y_dtype == QUAFF_F32;
        p.status = o.status;
        return QUAFF_OK;
    }
    Mx4GemmParams& p = l.big;
    memset(&p, 0, sizeof(p));
    if ((rc = make_tmap_2d(&p.map_a, o.Xc, 1, o.M, cols, o.ldxc, 128, 128)) != QUAFF_OK) return rc;
    if ((rc = make_tmap_2d(&p.map_b, o.Wc, 1, o.N, cols, o.ldwc, 128, 128)) != QUAFF_OK) return rc;
    if ((rc = make_tmap_rows128(&p.map_sa, o.Xs, mx4_scale_bytes(o.M, o.K), 8)) != QUAFF_OK) return rc;
    if ((rc = make_tmap_rows128(&p.map_sb, o.Ws, mx4_scale_bytes(o.N, o.K), 8)) != QUAFF_OK) return rc;
    if (o.r > 0) {
        p.rp = rp;
        p.lora_parts = o.parts;
        if ((rc = make_tmap_2d(&p.map_t, o.Tp, 2, o.M, o.parts * rp, o.parts * rp, 128, 64)) != QUAFF_OK) return rc;
        if ((rc = make_tmap_2d(&p.map_bt, o.B, 2, o.r, o.N, o.N, rp, 64)) != QUAFF_OK) return rc;
    }
    // whole-line stores need 16-byte aligned rows
    const int esz = o.y_dtype == QUAFF_F32 ? 4 : 2;
    if ((o.ldy * esz) % 16 == 0) {
        p.tma_cols = (o.N * (int64_t)esz) % 16 == 0 ? (int)round_up(o.N, 128 / esz) : o.N;
        if ((rc = make_tmap_out(&p.map_y, o.Y, esz, o.M, o.N, o.ldy)) != QUAFF_OK) return rc;
    }
    p.ktiles = mx4_ktiles(o.K);
    p.sa_tiles = mx4_row_tiles(o.M);
    p.sb_tiles = mx4_row_tiles(o.N);
    p.nblk = nblk;
    p.nmma_last = nmma_last;
    p.M = o.M; p.N = o.N;
    p.tiles_m = ceil_div(o.M, kMxTileM); p.tiles_n = ceil_div(o.N, kMxTileN);
    // row tiles per band of the tile order: a band of X stays in L2 while the column tiles sweep over it
    const size_t band = (40u << 20) / max((size_t)1, (size_t)kMxTileM * (size_t)cols);
    p.band_m = min(max((int)min(band, (size_t)1 << 20), max(1, ceil_div(148 / 2, p.tiles_n))), p.tiles_m);
    p.Y = o.Y; p.ldy = o.ldy; p.y_f32 = o.y_dtype == QUAFF_F32;
    p.status = o.status;
    return QUAFF_OK;
}

static quaff_status_t mx4_product_launch(const Mx4Launch& l, cudaStream_t st) {
    if (l.small) {
        const Mx4SmallParams& p = l.few;
        launch_pdl(mx4_small_kernel<false>, dim3((unsigned)(p.ranks * p.row_tiles * ceil_div(p.M, p.nt))), dim3(kMsThreads), ms_smem<false>(), st, p.ranks, p);
    } else {
        const int units = min(l.big.tiles_m * l.big.tiles_n, mx4_device()->pairs);
        launch_pdl(mx4_gemm_kernel, dim3(units * 2), dim3(kMxThreads), kMxSmemBytes, st, 2, l.big);
    }
    return launch_status();
}

// workspace of quaff_mx4_linear_fwd: the activations' codes and scales, s T in up to three parts
struct Mx4FwdWorkspace { size_t off_c, off_s, off_t, total; int64_t ldc; };
static Mx4FwdWorkspace mx4_fwd_workspace(int M, int K, int r) {
    Mx4FwdWorkspace w;
    w.ldc = mx4_row_bytes(K);
    size_t off = 0;
    w.off_c = off;    off += round_up((size_t)M * (size_t)w.ldc, 256);
    w.off_s = off;    off += round_up(mx4_scale_bytes(M, K), 256);
    w.off_t = off;    off += round_up((size_t)M * 3 * ((r + 15) / 16 * 16) * 2, 256);
    w.total = off;
    return w;
}
size_t mx4_fwd_workspace_bytes(int M, int K, int r) { return M < 0 || K <= 0 || r < 0 ? 0 : mx4_fwd_workspace(M, K, r).total; }

}  // namespace quaff

using namespace quaff;

extern "C" size_t quaff_mx4_scale_bytes(int rows, int K) { return rows <= 0 || K <= 0 ? 0 : mx4_scale_bytes(rows, K); }

extern "C" quaff_status_t quaff_mx4_quantize(const void* X, int x_dtype, int64_t ldx, int M, int K, uint8_t* codes, int64_t ldc, uint8_t* scales,
                                             quaff_stream_t stream) {
    QUAFF_RETURN_IF(M < 0 || K <= 0 || (M > 0 && (!X || !codes || !scales)) || ldx < K, QUAFF_ERR_INVALID_ARG);
    QUAFF_RETURN_IF(x_dtype != QUAFF_BF16 && x_dtype != QUAFF_F32, QUAFF_ERR_INVALID_ARG);
    QUAFF_RETURN_IF(ldc < mx4_row_bytes(K), QUAFF_ERR_INVALID_ARG);
    QUAFF_RETURN_IF(mx4_row_tiles(M) > 65535 || K > (1 << 28), QUAFF_ERR_UNSUPPORTED_SHAPE);      // launch grid
    QUAFF_RETURN_IF(!aligned16(X) || (ldx % (x_dtype == QUAFF_F32 ? 4 : 8)) || !aligned16(codes) || !aligned16(scales) || (ldc % 16), QUAFF_ERR_ALIGNMENT);
    if (M == 0) return QUAFF_OK;
    return mx4_quantize_launch(X, x_dtype, ldx, M, K, codes, ldc, scales, (cudaStream_t)stream);
}

extern "C" quaff_status_t quaff_mx4_dequantize(const uint8_t* codes, int64_t ldc, const uint8_t* scales, int M, int K, quaff_bf16* out, int64_t ldo,
                                               quaff_stream_t stream) {
    QUAFF_RETURN_IF(M < 0 || K <= 0 || (M > 0 && (!codes || !scales || !out)) || ldo < K || ldc < mx4_row_bytes(K), QUAFF_ERR_INVALID_ARG);
    QUAFF_RETURN_IF(mx4_row_tiles(M) > 65535 || K > (1 << 28), QUAFF_ERR_UNSUPPORTED_SHAPE);      // launch grid
    QUAFF_RETURN_IF(!aligned16(codes) || !aligned16(scales) || !aligned16(out) || (ldc % 16) || (ldo % 8), QUAFF_ERR_ALIGNMENT);
    if (M == 0) return QUAFF_OK;
    return mx4_dequantize_launch(codes, ldc, scales, M, K, out, ldo, (cudaStream_t)stream);
}

extern "C" quaff_status_t quaff_mx4_matmul(int M, int K, int N, const uint8_t* Xc, int64_t ldxc, const uint8_t* Xs, const uint8_t* Wc, int64_t ldwc,
                                           const uint8_t* Ws, void* Y, int y_dtype, int64_t ldy, int32_t* status_opt, void* /*ws*/, size_t /*ws_bytes*/,
                                           quaff_stream_t stream) {
    QUAFF_RETURN_IF(M < 0 || K <= 0 || N <= 0 || (M > 0 && (!Xc || !Xs || !Y)) || !Wc || !Ws || ldy < N, QUAFF_ERR_INVALID_ARG);
    QUAFF_RETURN_IF(ldxc < mx4_row_bytes(K) || ldwc < mx4_row_bytes(K), QUAFF_ERR_INVALID_ARG);
    QUAFF_RETURN_IF(y_dtype != QUAFF_BF16 && y_dtype != QUAFF_F32, QUAFF_ERR_INVALID_ARG);
    QUAFF_RETURN_IF(!aligned16(Xc) || !aligned16(Xs) || !aligned16(Wc) || !aligned16(Ws) || !aligned16(Y) || (ldxc % 16) || (ldwc % 16), QUAFF_ERR_ALIGNMENT);
    if (M == 0) return QUAFF_OK;
    Mx4Launch l;
    const Mx4Operands o = {M, K, N, Xc, ldxc, Xs, Wc, ldwc, Ws, nullptr, nullptr, 0, 0, Y, y_dtype, ldy, status_opt};
    const quaff_status_t rc = mx4_product_prepare(l, o, false);
    return rc != QUAFF_OK ? rc : mx4_product_launch(l, (cudaStream_t)stream);
}

extern "C" quaff_status_t quaff_mx4_linear_fwd(int M, int K, int N, const quaff_bf16* X, int64_t ldx, const uint8_t* Wc, int64_t ldwc, const uint8_t* Ws,
                                               const quaff_bf16* A, const quaff_bf16* B, int r, float lora_scale, quaff_bf16* T_out, void* Y,
                                               int y_dtype, int64_t ldy, int32_t* status_opt, void* ws, size_t ws_bytes, quaff_stream_t stream) {
    QUAFF_RETURN_IF(M < 0 || K <= 0 || N <= 0 || r < 0 || (M > 0 && (!X || !Y)) || !Wc || !Ws || ldx < K || ldy < N, QUAFF_ERR_INVALID_ARG);
    QUAFF_RETURN_IF(ldwc < mx4_row_bytes(K), QUAFF_ERR_INVALID_ARG);
    QUAFF_RETURN_IF(r > 0 && (!A || !B || (M > 0 && !T_out)), QUAFF_ERR_INVALID_ARG);
    QUAFF_RETURN_IF(y_dtype != QUAFF_BF16 && y_dtype != QUAFF_F32, QUAFF_ERR_INVALID_ARG);
    QUAFF_RETURN_IF((r % 8) || r > 64 || (r > 0 && ((K % 8) || (N % 8))), QUAFF_ERR_UNSUPPORTED_SHAPE);
    QUAFF_RETURN_IF(mx4_row_tiles(M) > 65535 || K > (1 << 28), QUAFF_ERR_UNSUPPORTED_SHAPE);      // launch grid
    QUAFF_RETURN_IF(!aligned16(X) || (ldx % 8) || !aligned16(Wc) || !aligned16(Ws) || (ldwc % 16) || !aligned16(Y), QUAFF_ERR_ALIGNMENT);
    QUAFF_RETURN_IF(r > 0 && (!aligned16(A) || !aligned16(B) || !aligned16(T_out)), QUAFF_ERR_ALIGNMENT);
    const Mx4FwdWorkspace w = mx4_fwd_workspace(M, K, r);
    QUAFF_RETURN_IF(M > 0 && (!ws || !aligned16(ws) || ws_bytes < w.total), QUAFF_ERR_WORKSPACE_TOO_SMALL);
    if (M == 0) return QUAFF_OK;
    cudaStream_t st = (cudaStream_t)stream;
    uint8_t* base = reinterpret_cast<uint8_t*>(ws);
    uint8_t *Xc = base + w.off_c, *Xs = base + w.off_s;
    uint16_t* Tp = reinterpret_cast<uint16_t*>(base + w.off_t);
    const int parts = y_dtype == QUAFF_F32 ? 3 : 2;
    const Mx4Device* d = mx4_device();
    if (!d) return QUAFF_ERR_CUDA;
    // Up to 16 tokens, and row tiles few enough for clusters of four: everything in one launch, each row tile quantizing X and
    // multiplying it with A for itself.  More row tiles mean longer shares of K per CTA, and A comes from L2 once per tile: then two launches
    // are better.  One / two launches, us on the device with weights that have left L2 (tokens, K -> N, r): 1, 1024 -> 1024, 16 6.0 / 7.0; 1, 11008 -> 1024, 16
    // 9.7 / 12.5; 16, 11008 -> 1024, 64 12.1 / 22.1; 1, 4096 -> 4096, 16 10.5 / 9.3; 16, 4096 -> 4096, 64 13.8 / 15.9; 1, 8192 -> 4096, 16 13.3 / 12.3; 1, 8192 -> 4096, 64
    // 14.5 / 16.7; 1, 11008 -> 4096, 16 14.7 / 15.4; 16, 11008 -> 4096, 16 16.7 / 16.3; 16, 11008 -> 4096, 64 18.1 / 24.3.  Where one launch loses on the device
    // (r = 16, N = 4096, by 1.2 at most, with no order in K) it saves 2 to 3 us of the host's time; warm: 1, 4096 -> 8192, 16 11.4 / 9.0; 16, 4096 -> 11008, 64 20.7 / 16.7.
    if (M <= kMsFusedTokens && ceil_div(N, 128) <= d->clusters[4]) {
        Mx4SmallParams p;
        memset(&p, 0, sizeof(p));
        quaff_status_t rc;
        if ((rc = make_tmap_2d(&p.map_w, Wc, 1, N, (uint64_t)mx4_row_bytes(K), ldwc, 128, 128)) != QUAFF_OK) return rc;
        if ((rc = make_tmap_rows128(&p.map_sw, Ws, mx4_scale_bytes(N, K), 8)) != QUAFF_OK) return rc;
        if ((rc = make_tmap_2d(&p.map_raw, X, 2, M, K, ldx, kMsFusedTokens, 64)) != QUAFF_OK) return rc;
        if (r > 0 && (rc = make_tmap_2d(&p.map_a, A, 2, K, r, r, 64, 64)) != QUAFF_OK) return rc;
        p.nblk = ceil_div(K, 256);
        p.nmma_last = ceil_div(K - (p.nblk - 1) * 256, 64);
        p.per = mx4_small_plan(d, M, N, p.nblk);
        p.ranks = ceil_div(p.nblk, p.per);
        p.ktiles = mx4_ktiles(K);
        p.sw_tiles = mx4_row_tiles(N);
        p.sx_tiles = 1;
        p.M = M; p.N = N; p.nt = kMsFusedTokens;
        p.row_tiles = ceil_div(N, 128);
        p.B = B; p.T = T_out; p.r = r; p.scale = lora_scale;
        p.Y = Y; p.ldy = ldy; p.y_f32 = y_dtype == QUAFF_F32;
        p.status = status_opt;
        launch_pdl(mx4_small_kernel<true>, dim3((unsigned)(p.ranks * p.row_tiles)), dim3(kMsThreads), ms_smem<true>(), st, p.ranks, p);
        return launch_status();
    }
    // what makes the product's operands: one launch either way (few tokens: a cluster per token; else a pass over row tiles), and
    // both let the product fetch W early; without adapters the plain quantization for many tokens
    const bool prep = mx4_use_prep(M, K, r), down = !prep && r > 0;
    Mx4Launch l;
    SkinnyParams sp;
    const Mx4Operands o = {M, K, N, Xc, w.ldc, Xs, Wc, ldwc, Ws, Tp, B, r, parts, Y, y_dtype, ldy, status_opt};
    quaff_status_t rc = mx4_product_prepare(l, o, prep || down);
    if (rc != QUAFF_OK) return rc;
    if (down) {
        if ((rc = mx4_skinny_prepare(sp, kSkinnyDown, X, ldx, A, r, M, K, r, r, status_opt)) != QUAFF_OK) return rc;
        sp.bf16_out = T_out; sp.bf16_scale = 1.0f;
        sp.parts_out = Tp; sp.parts = parts; sp.scale = lora_scale;
        sp.K = K; sp.ktiles = mx4_ktiles(K);
        sp.codes = Xc; sp.ldc = w.ldc; sp.scales = Xs;
    }
    if (prep) rc = launch_mx4_prep(X, ldx, M, K, Xc, w.ldc, Xs, A, r, parts, lora_scale, T_out, Tp, st);
    else if (down) rc = mx4_skinny_launch(sp, kSkinnyDown, st);
    else rc = mx4_quantize_launch(X, QUAFF_BF16, ldx, M, K, Xc, w.ldc, Xs, st);
    return rc != QUAFF_OK ? rc : mx4_product_launch(l, st);
}
