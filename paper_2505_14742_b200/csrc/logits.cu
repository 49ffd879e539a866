// Kernels over rows of logits: the k largest of a teacher's row with its log-sum-exp, and the distillation loss of a
// student's row against such a list with the gradient of its logits.
//
// Both read a row from HBM once.  A row belongs to one CTA or to a cluster of up to eight, each of which holds a slice in
// shared memory; a thread copies (cp.async) the 16-byte words that only it works on later, so the first pass over a slice
// needs no barrier and the next row's words can be fetched into the place of those it is done with.  The CTAs are
// persistent (three per SM) for that.  Per-slice maxima, sums and lists are combined through distributed shared memory.
#include <float.h>
#include <math.h>

#include <atomic>

#include "common.cuh"

namespace quaff {

// What a thread does once per row (reductions, the list) costs as much as its share of a row: 256 threads with sixteen words
// each of a 64 KB slice; three CTAs per SM overlap their copies, sums and stores.  Measured: top 64 of 4096 x 32000 bf16
// 85 us (3.1 TB/s; without the log-sum-exp 64), distillation of 8192 x 32000 bf16 226 us (4.6 TB/s read and written).  Both are bound
// by instruction issue and the exponential unit (57 % of either at 24 warps per SM), not by HBM.
constexpr int kLgThreads = 256;
constexpr int kLgWarps = kLgThreads / 32;
constexpr int kLgMaxK = 256;                 // list length limit of both operators
// Lists longer than this: one threshold for a cluster.  Separate / together, us, f32: 8 x 128000 k = 20 9.9 / 11.0, k = 64 13.5 / 11.7;
// 33 x 50000 k = 20 10.1 / 12.2, k = 100 22.6 / 12.7, k = 256 49.6 / 13.7.
constexpr int kLgTogether = 32;
constexpr int kLgMaxCluster = 8;
static_assert(kLgMaxK <= kLgThreads, "a thread per entry of a list");
constexpr int kLgSliceMax = 192 * 1024;      // bytes of a row that one CTA may hold
constexpr int kLgSmemMax = 232448;           // dynamic shared memory of a CTA on sm_100
constexpr int kLgSmemSm = 233472;            // shared memory of an SM, of which every CTA takes 1 KB for the system
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(reinterpret_cast<uint64_t>(src)) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
// 2^x; results below 2^-126 become 0: they are shares of a sum of at least 1
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float ld_cluster_f32(uint32_t addr) { return __uint_as_float(ld_cluster_u32(addr)); }
__device__ __forceinline__ unsigned long long ld_cluster_u64(uint32_t addr) {
    unsigned long long v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(addr) : "memory");
    return v;
}

template <typename T> struct Row;
template <> struct Row<uint16_t> {            // bf16 bits
    static constexpr int kVec = 8;
    static constexpr uint16_t kMinusInf = 0xFF80u;
    static constexpr uint32_t kMinusInfWord = 0xFF80FF80u;
    static __device__ __forceinline__ float at(const uint16_t* p, int i) { return bf16_bits_to_f32(p[i]); }
    static __device__ __forceinline__ void elements(const uint4& a, float (&v)[8]) {
        v[0] = bf16_lo(a.x); v[1] = bf16_hi(a.x); v[2] = bf16_lo(a.y); v[3] = bf16_hi(a.y);
        v[4] = bf16_lo(a.z); v[5] = bf16_hi(a.z); v[6] = bf16_lo(a.w); v[7] = bf16_hi(a.w);
    }
    static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {      // NaN is skipped
        uint32_t m;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
        return m;
    }
    static __device__ __forceinline__ float2 block_max(const uint4 (&a)[4]) {      // of its first and its last two words
        uint32_t m[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) m[j] = max2(max2(a[j].x, a[j].y), max2(a[j].z, a[j].w));
        m[0] = max2(m[0], m[1]);
        m[2] = max2(m[2], m[3]);
        return make_float2(fmaxf(bf16_lo(m[0]), bf16_hi(m[0])), fmaxf(bf16_lo(m[2]), bf16_hi(m[2])));
    }
    static __device__ __forceinline__ uint4 pack(const float (&v)[8]) {
        return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
    }
    static __device__ __forceinline__ uint16_t one(float x) { return (uint16_t)(pack_bf16x2(x, 0.0f) & 0xFFFFu); }
};
template <> struct Row<float> {
    static constexpr int kVec = 4;
    static constexpr float kMinusInf = -INFINITY;
    static constexpr uint32_t kMinusInfWord = 0xFF800000u;
    static __device__ __forceinline__ float at(const float* p, int i) { return p[i]; }
    static __device__ __forceinline__ void elements(const uint4& a, float (&v)[4]) {
        v[0] = __uint_as_float(a.x); v[1] = __uint_as_float(a.y); v[2] = __uint_as_float(a.z); v[3] = __uint_as_float(a.w);
    }
    static __device__ __forceinline__ float2 block_max(const uint4 (&a)[4]) {
        float m[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            m[j] = fmaxf(fmaxf(__uint_as_float(a[j].x), __uint_as_float(a[j].y)), fmaxf(__uint_as_float(a[j].z), __uint_as_float(a[j].w)));
        return make_float2(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
    }
    static __device__ __forceinline__ uint4 pack(const float (&v)[4]) {
        return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    }
    static __device__ __forceinline__ float one(float x) { return x; }
};

// This CTA's slice of a row of V elements: [begin, begin + n); slices start at multiples of 8 elements
struct Slice { int begin, n; };
template <typename T>
__device__ __forceinline__ Slice slice_of(int V, int rank, int csize) {
    const int per = ((V + csize - 1) / csize + 7) & ~7;
    Slice s;
    s.begin = min(rank * per, V);
    s.n = min(per, V - s.begin);
    return s;
}
// A thread works in blocks of four words (word tid + (4 b + j) threads is the j-th of its block b): the bookkeeping per block,
// not per element, is what keeps the instruction count down.  The slice's place in shared memory is whole blocks long; what
// lies beyond the slice holds -inf from the start and is never written again.
__host__ __device__ __forceinline__ int blocks_of(int words) { return (words + 4 * kLgThreads - 1) / (4 * kLgThreads); }
template <typename T>
__device__ __forceinline__ void block_load(const T* row, int b, uint4 (&a)[4]) {
    const uint4* p = reinterpret_cast<const uint4*>(row) + threadIdx.x + b * 4 * kLgThreads;
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] = p[j * kLgThreads];
}
template <typename T>
__device__ __forceinline__ void pad_slice(T* row, int words) {
    const uint4 none = make_uint4(Row<T>::kMinusInfWord, Row<T>::kMinusInfWord, Row<T>::kMinusInfWord, Row<T>::kMinusInfWord);
    for (int i = words + (int)threadIdx.x; i < blocks_of(words) * 4 * kLgThreads; i += kLgThreads) reinterpret_cast<uint4*>(row)[i] = none;
}
// Starts the copy of this thread's words of block b.  Elements that do not fill a word are stored by the thread that owns it.
template <typename T>
__device__ __forceinline__ void block_fetch(T* row, const T* __restrict__ src, int n, int b) {
    constexpr int W = Row<T>::kVec;
    const int full = n / W, i = (int)threadIdx.x + b * 4 * kLgThreads;
    const uint32_t to = smem_u32(row) + (uint32_t)i * 16u;
    const T* from = src + (int64_t)i * W;
    if ((b + 1) * 4 * kLgThreads <= full) {
#pragma unroll
        for (int j = 0; j < 4; ++j) cp_async16(to + j * kLgThreads * 16u, from + j * kLgThreads * W);
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) if (i + j * kLgThreads < full) cp_async16(to + j * kLgThreads * 16u, from + j * kLgThreads * W);
    if (full * W < n && (int)threadIdx.x == full % kLgThreads && b == full / (4 * kLgThreads))
        for (int e = 0; e < W; ++e) row[full * W + e] = full * W + e < n ? src[full * W + e] : Row<T>::kMinusInf;
}
// The blocks of a slice travel in four groups: f(block) for the blocks of each group, then done(); or each group as soon
// as it has arrived
template <typename F, typename G>
__device__ __forceinline__ void in_groups(int nb, F f, G done) {
    const int quarter = (nb + 3) / 4;
    int b = 0;
#pragma unroll 1
    for (int g = 1; g <= 4; ++g) {
#pragma unroll 1
        for (const int end = min(g * quarter, nb); b < end; ++b) f(b);
        done();
    }
}
template <typename F>
__device__ __forceinline__ void as_they_arrive(int nb, F f) {
    const int quarter = (nb + 3) / 4;
    int b = 0;
#pragma unroll 1
    for (int g = 1; g <= 4; ++g) {        // (one copy of f in the code: a row's work must stay in the instruction cache)
        if (g == 1) cp_async_wait<3>();
        else if (g == 2) cp_async_wait<2>();
        else if (g == 3) cp_async_wait<1>();
        else cp_async_wait<0>();
#pragma unroll 1
        for (const int end = min(g * quarter, nb); b < end; ++b) f(b);
    }
}

// ------------------------------------------------------------------ exponentials relative to a maximum
// 2^((z - max) c1).  The many terms are taken as 2^(z c1 - shift), shift = max c1 rounded: one fused multiply-add, two elements
// per instruction; what the rounding of the shift adds to every exponent alike is taken out of their sum.  That is up to 2^-25 of the shift, so
// it has to stay small: from |max c1| = 2^31 on (finite masks fill the words) floats next to the maximum are 128 and more apart
// in the exponent, and all but the maximum itself vanish; a power of two that keeps the product exact stands in for c1.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack2(float a, float b) {
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2(f32x2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
struct Base {              // a maximum as the exponentials take it
    float m, mul, shift;   // the maximum (0 in place of an infinity), c1 or what stands in for it, m mul
    __device__ __forceinline__ void set(float mx, float c1) {
        m = fabsf(mx) == INFINITY ? 0.0f : mx;
        mul = c1;
        shift = m * c1;
        if (!(fabsf(shift) < 0x1p31f)) {
            mul = __uint_as_float(((127u + 31u + 127u) << 23) - (__float_as_uint(m) & 0x7F800000u));      // 2^31 / 2^exponent (that of m is -96 at least: c1 < 2^127)
            shift = m * mul;
        }
    }
    __device__ __forceinline__ float log2_of(float z, float c1) const { return (z - m) * c1; }
    // what brings exps() to 2^((z - m) c1)
    __device__ __forceinline__ float unfix() const { return ex2(-fmaf(m, mul, -shift)); }
    // exponentials of a block's elements, as pairs handed to f(pair, word, pair of the word)
    template <typename T, typename F> __device__ __forceinline__ void exps(const uint4 (&a)[4], F f) const {
        const f32x2 cc = pack2(mul, mul), nn = pack2(-shift, -shift);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float v[Row<T>::kVec];
            Row<T>::elements(a[j], v);
#pragma unroll
            for (int e = 0; e < Row<T>::kVec; e += 2) {
                float x, y;
                unpack2(fma2(pack2(v[e], v[e + 1]), cc, nn), x, y);
                f(pack2(ex2(x), ex2(y)), j, e / 2);
            }
        }
    }
    // log2 of what brings sums relative to this base to another one
    __device__ __forceinline__ float to(const Base& b, float c1) const { return (m - b.m) * c1; }
};
// A thread's running maximum and sum of exponentials; the maximum moves rarely after the first words
struct RunSum {
    float mx = -INFINITY;
    f32x2 s = 0ull;
    Base b = {0.0f, 1.0f, 0.0f};
    template <typename T> __device__ __forceinline__ void add(const uint4 (&a)[4], float top, float c1) {
        if (top > mx) {
            Base n;
            n.set(top, c1);
            // (nothing finite so far: the sum is 0, or NaN)
            const float f = mx == -INFINITY ? 0.0f : ex2(b.mul == c1 && n.mul == c1 ? b.shift - n.shift : (b.m - n.m) * c1);
            s = mul2(s, pack2(f, f));
            mx = top;
            b = n;
        }
        f32x2 t[4] = {0ull, 0ull, 0ull, 0ull};
        b.exps<T>(a, [&](f32x2 e, int j, int) { t[j] = add2(t[j], e); });
        s = add2(s, add2(add2(t[0], t[1]), add2(t[2], t[3])));
    }
    __device__ __forceinline__ float sum() const {
        float x, y;
        unpack2(s, x, y);
        return (x + y) * b.unfix();
    }
};

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    return v;
}
template <typename F> __device__ __forceinline__ F warp_sum(F v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}
// ... over kLgWarps values, one per lane modulo kLgWarps: the result in every lane
__device__ __forceinline__ float slots_max(float v) {
#pragma unroll
    for (int o = kLgWarps / 2; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    return v;
}
template <typename F> __device__ __forceinline__ F slots_sum(F v) {
#pragma unroll
    for (int o = kLgWarps / 2; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}
// A sum relative to its maximum mx, brought to another base
__device__ __forceinline__ float at_base(float mx, float s, const Base& b, float c1) {
    Base o;
    o.set(mx, c1);
    return s == 0.0f ? 0.0f : s * ex2(o.to(b, c1));
}
// Maxima and sums of a warp's lanes -> the warp's maximum, and the sum relative to it
__device__ __forceinline__ float2 warp_run(float mx, float s, float c1) {
    const float wm = warp_max(mx);
    Base b;
    b.set(wm, c1);
    return make_float2(wm, warp_sum(at_base(mx, s, b, c1)));
}

// ==================================================================================== distillation
// With z' = z / tau, q = softmax(z'), the listed probabilities p_j, P = sum p_j and the teacher's remaining mass
// R = max(0, 1 - P) (0 when the list is renormalised), r = the student's mass on the unlisted tokens, c = P + R:
//   loss = w tau^2 [ sum_j p_j (log p_j - log q_j) + R (log R - log r) ]
//   dz_v = w tau (c q_v - p_v)      v listed,      w tau (c q_v - R q_v / r)      otherwise
// A byte per word of the slice marks the listed elements while the row is on its way; the first pass, which follows the
// copy group by group, leaves them out of the sum over the unlisted and sets them to -inf, so r is a sum of its own
// and not a difference of two sums that may cancel.  It may be less than 2^-126 (a student that is sure of the list; a finite mask on all others), its
// logarithm and the shares q_v / r are not.  So the unlisted have a maximum of their own, mu; where it is far below mx, that over all, their exponentials are
// relative to it: with su = the sum of exp(z'_v - mu) and S the sum of exp(z'_v - mx) over all,
//   log r = mu - mx + log su - log S,      q_v / r = exp(z'_v - mu) / su,      q_v = exp(z'_v - mu) exp(mu - mx) / S:
// one exponential per token either way.
// R is a difference, by definition: the listed probabilities and their sum are
// taken in 64 bits when the list comes with a log-sum-exp (one exponential per listed token; in 32 bits R would be known to
// about 1e-6 absolute, and R / r, the whole gradient of the unlisted tokens, only as well as that over r).  The log-sum-exp itself has 32
// bits and the error of its sums: where everything visible is listed, R is that error or 0, r is 0, and R log(R / r) would be infinite for about
// every second row.  Up to 2^-16 + 2^-20 |lse| (what quaff_topk_logits is held to) such an R counts as 0.
struct DistillSmem {
    float4 warps[kLgWarps];            // maximum and sum of each warp: of the unlisted, of the listed
    float2 lists[kLgWarps];            // maximum and sum of the teacher's list
    double mass[kLgWarps];             // sum of the listed probabilities
    float loss[kLgWarps];
    alignas(16) float part[4];         // this CTA's maximum and sum of the unlisted, of the listed
    float2 base;                       // what the sums are relative to
    float total;                       // its share of the loss
};
struct DistillParams {
    const void* Z;
    int64_t ldz;
    int M, V, k;
    const float* t_val;
    const int32_t* t_idx;
    const float* t_lse;
    float inv_tau, tau;
    double inv_tau64;
    const float* row_w;
    float* loss;
    void* dZ;
    int64_t lddz;
};

// Thread j < k has entry j of the list.  What a row needs besides its logits is fetched ahead of the copies of whole rows,
// behind which it would queue: weight, list and log-sum-exp two rows ahead, the student's logits at the list one.
struct DistillRow {
    float w, t, lse, z;
    int at;              // listed token, -1: none
};

template <typename T>
__global__ void __launch_bounds__(kLgThreads, 3) distill_kernel(const DistillParams p, int csize) {
    constexpr int W = Row<T>::kVec;
    extern __shared__ __align__(16) unsigned char smem_dyn[];
    DistillSmem* sm = reinterpret_cast<DistillSmem*>(smem_dyn);
    T* row = reinterpret_cast<T*>(smem_dyn + ((sizeof(DistillSmem) + 15) / 16) * 16);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = csize > 1 ? (int)cluster_ctarank() : 0;
    const int stride = (int)gridDim.x / csize;
    const Slice s = slice_of<T>(p.V, rank, csize);
    const int words = (s.n + W - 1) / W, nb = blocks_of(words);
    uint32_t* marks = reinterpret_cast<uint32_t*>(row + (size_t)nb * 4 * kLgThreads * W);      // a byte per word, the four of a block in one word
    for (int b = 0; b < nb; ++b) marks[b * kLgThreads + tid] = 0;
    pad_slice(row, words);
    const float c1 = p.inv_tau * kLog2e;
    pdl_launch_dependents();
    pdl_wait();

    auto src = [&](int m) { return reinterpret_cast<const T*>(p.Z) + (int64_t)m * p.ldz + s.begin; };
    auto dst = [&](int m) { return reinterpret_cast<T*>(p.dZ) + (int64_t)m * p.lddz + s.begin; };
    auto mine = [&](const DistillRow& r) { return r.at >= s.begin && r.at < s.begin + s.n; };
    auto zero_row = [&](int m) {
        if (p.dZ) {
            T* d = dst(m);
            for (int i = tid; i < s.n / W; i += kLgThreads) *reinterpret_cast<uint4*>(d + (int64_t)i * W) = make_uint4(0, 0, 0, 0);
            if (tid < s.n % W) d[s.n / W * W + tid] = 0;
        }
        if (rank == 0 && tid == 0) p.loss[m] = 0.0f;
    };
    auto fetch = [&](int m, DistillRow& r) {
        r.w = 1.0f;
        r.t = r.z = -INFINITY;
        r.at = -1;
        r.lse = 0.0f;
        if (m >= p.M) return;
        if (p.row_w) r.w = p.row_w[m];
        if (p.t_lse) r.lse = p.t_lse[m];
        if (tid < p.k) { r.at = p.t_idx[(int64_t)m * p.k + tid]; r.t = p.t_val[(int64_t)m * p.k + tid]; }
    };
    // the row from m on that has a weight (the same for all threads of the cluster), its list checked, its listed logits on the way
    auto settle = [&](int m, DistillRow& r) {
        while (m < p.M && r.w == 0.0f) {
            zero_row(m);
            m += stride;
            fetch(m, r);
        }
        if (!(r.at >= 0 && r.at < p.V && r.t > -INFINITY)) r.at = -1;
        if (m < p.M && mine(r)) r.z = Row<T>::at(src(m), r.at - s.begin);
        return m;
    };

    DistillRow cur, nxt;
    int m = (int)blockIdx.x / csize;
    fetch(m, cur);
    m = settle(m, cur);
    fetch(m + stride, nxt);
    if (m < p.M) in_groups(nb, [&](int b) { block_fetch<T>(row, src(m), s.n, b); }, [] { cp_async_commit(); });
    int last = -1;                        // the row whose loss waits in sm->loss
    __syncthreads();                      // the marks are clear
    while (m < p.M) {
        if (mine(cur)) {
            const int j = cur.at - s.begin, word = j / W;
            atomicOr(&marks[word / (4 * kLgThreads) * kLgThreads + word % kLgThreads], (1u << (j % W)) << (word / kLgThreads % 4 * 8));
        }
        __syncthreads();
        if (csize == 1 && tid == 0 && last >= 0) {
            float l = 0.0f;
            for (int i = 0; i < kLgWarps; ++i) l += sm->loss[i];
            p.loss[last] = l;
        }
        // one pass over this thread's own words as they arrive; without a gradient they are then free for the next row
        RunSum run;
        as_they_arrive(nb, [&](int bl) {
            uint32_t out = marks[bl * kLgThreads + tid];
            if (out) {
                marks[bl * kLgThreads + tid] = 0;
                for (; out; out &= out - 1) {
                    const int j = __ffs(out) - 1;
                    row[(tid + (4 * bl + (j >> 3)) * kLgThreads) * W + (j & 7)] = Row<T>::kMinusInf;
                }
            }
            uint4 a[4];
            block_load(row, bl, a);
            const float2 top = Row<T>::block_max(a);
            run.add<T>(a, fmaxf(top.x, top.y), c1);
        });
        // this warp's share: unlisted, listed, the teacher's list
        const bool listed = cur.at >= 0;
        float logp = -INFINITY, prob = 0.0f;
        {
            const float2 u = warp_run(run.mx, run.sum(), c1);
            float2 l = make_float2(-INFINITY, 0.0f), ts = l;
            double mass = 0.0;
            if (warp * 32 < p.k) {
                l = warp_run(cur.z, cur.z == -INFINITY ? 0.0f : cur.z - cur.z + 1.0f, c1);      // (NaN for +inf)
                if (p.t_lse) {
                    if (listed) {
                        const double lp = (double)cur.t * p.inv_tau64 - (double)cur.lse;
                        mass = exp(lp);
                        logp = (float)lp;
                        prob = (float)mass;
                    }
                    mass = warp_sum(mass);
                } else {
                    ts = warp_run(listed ? cur.t : -INFINITY, listed ? 1.0f : 0.0f, c1);
                }
            }
            if (lane == 0) {
                sm->warps[warp] = make_float4(u.x, u.y, l.x, l.y);
                sm->lists[warp] = ts;
                sm->mass[warp] = mass;
            }
        }
        __syncthreads();
        const int next = settle(m + stride, nxt);
        DistillRow after;
        fetch(next + stride, after);
        // the row's maxima and sums, of the unlisted (relative to `bu`) and of all (to `b`), in every thread
        float mu, su, ml, sl, c = 1.0f, R = 0.0f, logP = 0.0f;
        bool dead = false;
        Base b, bu;
        auto bases = [&]() {
            b.set(fmaxf(mu, ml), c1);
            bu.set(mu, c1);
            if (bu.to(b, c1) > -60.0f) bu = b;                   // (then r is an ordinary number, and more exact without a factor for the whole row)
        };
        {
            const float4 u = sm->warps[lane % kLgWarps];
            mu = slots_max(u.x);
            ml = slots_max(u.z);
            bases();
            su = slots_sum(at_base(u.x, u.y, bu, c1));
            sl = slots_sum(at_base(u.z, u.w, b, c1));
            if (p.t_lse) {
                // NaN stays NaN, from the list or (an empty list of a teacher row with a NaN) from the log-sum-exp alone
                const double P = slots_sum(sm->mass[lane % kLgWarps]) + (isnan(cur.lse) ? (double)cur.lse : 0.0);
                R = P < 1.0 ? (float)(1.0 - P) : (P >= 1.0 ? 0.0f : NAN);
                c = P < 1.0 ? 1.0f : (float)P;
            } else {
                const float2 l = sm->lists[lane % kLgWarps];
                const float tm = slots_max(l.x);
                Base tb;
                tb.set(tm, c1);
                const float sum = slots_sum(at_base(l.x, l.y, tb, c1));
                logP = logf(sum);
                dead = tm == -INFINITY;                          // nothing listed
                if (tm == INFINITY) c = logP = NAN;              // a listed value of +inf: inf / inf
                if (listed) { logp = (cur.t - tb.m) * p.inv_tau - logP; prob = ex2((cur.t - tb.m) * c1) / sum; }      // (that of the largest has no error of ex2)
            }
        }
        if (csize > 1) {
            if (tid == 0) {
                *reinterpret_cast<float4*>(sm->part) = make_float4(mu, su, ml, sl);
                sm->base = make_float2(bu.m, b.m);
            }
            cluster_sync();
            const uint32_t a = mapa_shared(smem_u32(&sm->part[0]), lane < csize ? lane : 0), ab = mapa_shared(smem_u32(&sm->base), lane < csize ? lane : 0);
            float4 u = make_float4(-INFINITY, 0.0f, -INFINITY, 0.0f);
            if (lane < csize) u = ld_cluster_f4(a);
            mu = warp_max(u.x);
            ml = warp_max(u.z);
            bases();
            su = warp_sum(at_base(ld_cluster_f32(ab), u.y, bu, c1));
            sl = warp_sum(at_base(ld_cluster_f32(ab + 4), u.w, b, c1));
        }
        const float dm = bu.m - b.m, gap = dm == 0.0f ? 1.0f : ex2(dm * c1);
        float S = (su == 0.0f ? 0.0f : su * gap) + sl;
        if (S == INFINITY) S = NAN;                              // a logit of +inf
        dead = dead || S == 0.0f;                                // or no logit above -inf: nothing to learn
        // No unlisted token is visible to the student, and what the teacher left is within what its log-sum-exp can tell: all is listed
        if (su == 0.0f && R < 1.0f && R <= fmaf(0x1p-20f, fabsf(cur.lse), 0x1p-16f)) { c -= R; R = 0.0f; }
        const float wt = cur.w * p.tau, f = wt / S;
        if (p.dZ) {
            const float co1 = (su == 0.0f ? 0.0f : wt * (c * gap / S - R / su)) * bu.unfix();
            const f32x2 co = pack2(co1, co1);
            const int full = s.n / W;
            T* d = dst(m);
            const T* from = src(next);
            in_groups(nb, [&](int bl) {
                uint4 a[4];
                block_load(row, bl, a);
                float g[4][W];
                if (!dead) bu.exps<T>(a, [&](f32x2 e, int j, int h) { unpack2(mul2(e, co), g[j][2 * h], g[j][2 * h + 1]); });
                else
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int e = 0; e < W; ++e) g[j][e] = 0.0f;
                const int i = tid + bl * 4 * kLgThreads;
                uint4* to = reinterpret_cast<uint4*>(d) + i;
                if ((bl + 1) * 4 * kLgThreads <= full) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) to[j * kLgThreads] = Row<T>::pack(g[j]);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (i + j * kLgThreads < full) to[j * kLgThreads] = Row<T>::pack(g[j]);
                        else if (i + j * kLgThreads < words) {   // the elements that do not fill a word
#pragma unroll
                            for (int e = 0; e < W; ++e) if (full * W + e < s.n) d[full * W + e] = Row<T>::one(g[j][e]);
                        }
                    }
                }
                if (next < p.M) block_fetch<T>(row, from, s.n, bl);
            }, [] { cp_async_commit(); });
            __syncthreads();                                     // the listed entries overwrite what the words' owners stored
            if (mine(cur) && !dead) d[cur.at - s.begin] = Row<T>::one(f * c * ex2(b.log2_of(cur.z, c1)) - wt * prob);
        } else {
            const T* from = src(next);
            in_groups(nb, [&](int bl) { if (next < p.M) block_fetch<T>(row, from, s.n, bl); }, [] { cp_async_commit(); });
        }
        // the loss: this warp's terms, the rest's in thread 0; logarithms times tau, as the logits are (a finite mask over a tau below 1 is
        // beyond the floats, its term of the loss need not be)
        const float logS = p.tau * logf(S);
        float part = 0.0f;
        if (warp * 32 < p.k) {
            if (!dead && mine(cur) && !(prob <= 0.0f)) part = wt * prob * (p.tau * logp - ((cur.z - b.m) - logS));
            part = warp_sum(part);
        }
        if (rank == 0 && tid == 0 && !dead && !(R <= 0.0f)) {
            part += wt * R * (p.tau * logf(R) - (dm == 0.0f ? p.tau * logf(su / S) : dm + p.tau * logf(su) - logS));
        }
        if (lane == 0) sm->loss[warp] = part;
        if (csize > 1) {
            __syncthreads();
            if (tid == 0) {
                float l = 0.0f;
                for (int i = 0; i < kLgWarps; ++i) l += sm->loss[i];
                sm->total = l;
            }
            cluster_sync();
            if (rank == 0 && tid == 0) {
                float l = 0.0f;
                for (int r = 0; r < csize; ++r) l += ld_cluster_f32(mapa_shared(smem_u32(&sm->total), r));
                p.loss[m] = l;
            }
        }
        last = m;
        m = next;
        cur = nxt;
        nxt = after;
    }
    __syncthreads();
    if (csize == 1 && tid == 0 && last >= 0) {
        float l = 0.0f;
        for (int i = 0; i < kLgWarps; ++i) l += sm->loss[i];
        p.loss[last] = l;
    }
    if (csize > 1) cluster_sync();                               // rank 0 may still be reading its partners' parts
}

// ==================================================================================== top logits
// Every thread keeps the maximum of its words; groups of threads are joined until there are at least 2 k groups (or as
// many groups as threads).  The k-th largest of the group maxima is at most the k-th largest element, so the elements
// that reach it hold the whole list and, as a rule, few others: they are collected and put in order by counting, for
// each, how many come before it (larger, or equal with a lower index).  A slice of ties that overflows the candidate
// buffer is decided exactly instead, by bisection on the key and then on the index.
struct TopkSmem {                         // behind it: this CTA's k largest in order (8 bytes each), the candidates, the slice, bmax
    float gmax[2 * kLgThreads];           // group maxima; later the blocks that reach the threshold (16 bits each)
    float2 warps[kLgWarps];               // maximum and sum of each warp
    float joined[kLgThreads];             // group maxima as the other CTAs of the cluster read them
    float part[2];                        // maximum, sum
    int have;                             // entries of this CTA's list
    int count, hits;
    uint32_t thr;
};
struct TopkParams {
    const void* Z;
    int64_t ldz;
    int M, V, k;
    int cap;             // entries of the candidate buffer: at least cluster size x k
    float inv_tau;
    float* val;
    int32_t* idx;
    float* lse;
};

// Order of the values as unsigned integers; -0 and +0 are equal, -inf and NaN lowest (never listed: key 0)
__device__ __forceinline__ uint32_t logit_key(float z) {
    if (!(z > -INFINITY)) return 0u;
    const uint32_t u = __float_as_uint(z + 0.0f);
    return (u >> 31) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float key_logit(uint32_t k) { return __uint_as_float((k >> 31) ? (k & 0x7FFFFFFFu) : ~k); }

__device__ __forceinline__ int cta_count(int v, int* counter) {     // sum over the CTA, in every thread
    v = __reduce_add_sync(0xFFFFFFFFu, v);
    __syncthreads();
    if (threadIdx.x == 0) *counter = 0;
    __syncthreads();
    if ((threadIdx.x & 31) == 0 && v) atomicAdd(counter, v);
    __syncthreads();
    return *counter;
}

// Number of entries above c among `len` descending ones (distinct; padded with zeros)
__device__ __forceinline__ int count_above(const unsigned long long* run, int len, unsigned long long c) {
    int pos = 0;
    for (int step = 1 << (31 - __clz(len)); step; step >>= 1)
        if (pos + step <= len && run[pos + step - 1] > c) pos += step;
    return pos;
}
// cand[0..n) (distinct, n <= cap, cap a multiple of 32) -> out[rank] for the first k of the descending order; returns
// min(n, k).  Warps sort runs of 32 in registers; an entry's rank is its place in its run and what the other runs hold above it.
__device__ __forceinline__ int rank_select(unsigned long long* cand, int n, int k, unsigned long long* out) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, runs = (n + 31) >> 5;
    for (int r = warp; r < runs; r += kLgWarps) {
        unsigned long long c = r * 32 + lane < n ? cand[r * 32 + lane] : 0ull;
#pragma unroll
        for (int size = 2; size <= 32; size *= 2)
#pragma unroll
            for (int o = size / 2; o > 0; o /= 2) {
                const unsigned long long other = __shfl_xor_sync(0xFFFFFFFFu, c, o);
                const bool keep_max = ((lane & o) == 0) == ((lane & size) == 0 || size == 32);
                c = (c > other) == keep_max ? c : other;
            }
        cand[r * 32 + lane] = c;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kLgThreads) {
        const unsigned long long c = cand[i];
        int before = i & 31;
        for (int r = 0; r < runs; ++r)
            if (r != i >> 5) {
                const unsigned long long* run = cand + r * 32;
                int pos = 0;
#pragma unroll
                for (int step = 16; step; step >>= 1) if (run[pos + step - 1] > c) pos += step;
                before += pos + (run[pos] > c);
            }
        if (before < k) out[before] = c;
    }
    return min(n, k);
}

// Largest 16-bit key that at least k of a warp's NK x 32 keys reach (0: fewer than k)
template <int NK>
__device__ __forceinline__ uint32_t kth_key16(const uint32_t (&key)[NK], int k) {
    uint32_t thr = 0;
#pragma unroll 1
    for (int b = 14; b >= 0; b -= 2) {
        int n1 = 0, n2 = 0, n3 = 0;
        const uint32_t c1 = thr | (1u << b), c2 = thr | (2u << b), c3 = thr | (3u << b);
#pragma unroll
        for (int i = 0; i < NK; ++i) { n1 += key[i] >= c1; n2 += key[i] >= c2; n3 += key[i] >= c3; }
        n1 = __reduce_add_sync(0xFFFFFFFFu, n1 | (n2 << 16));      // at most 512 each
        n3 = __reduce_add_sync(0xFFFFFFFFu, n3);
        n2 = n1 >> 16;
        n1 &= 0xFFFF;
        thr = n3 >= k ? c3 : (n2 >= k ? c2 : (n1 >= k ? c1 : thr));
    }
    return thr;
}

template <typename T>
__global__ void __launch_bounds__(kLgThreads, 3) topk_logits_kernel(const TopkParams p, int csize) {
    constexpr int W = Row<T>::kVec;
    extern __shared__ __align__(16) unsigned char smem_dyn[];
    TopkSmem* sm = reinterpret_cast<TopkSmem*>(smem_dyn);
    // the candidates: key of the value in the upper half, ~index in the lower
    unsigned long long* list = reinterpret_cast<unsigned long long*>(smem_dyn + ((sizeof(TopkSmem) + 15) / 16) * 16);
    unsigned long long* cand = list + ((p.k + 1) & ~1);
    T* row = reinterpret_cast<T*>(cand + p.cap);
    const int rank = csize > 1 ? (int)cluster_ctarank() : 0;
    const int stride = (int)gridDim.x / csize;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const Slice s = slice_of<T>(p.V, rank, csize);
    const int words = (s.n + W - 1) / W, nb = blocks_of(words);
    uint16_t* bmax = reinterpret_cast<uint16_t*>(row + (size_t)nb * 4 * kLgThreads * W);      // key of every block's maximum, upper half
    pad_slice(row, words);
    const float c1 = p.inv_tau * kLog2e;
    if (tid == 0) sm->count = sm->hits = 0;
    pdl_launch_dependents();
    pdl_wait();
    auto fetch = [&](int m) {
        const T* src = reinterpret_cast<const T*>(p.Z) + (int64_t)m * p.ldz + s.begin;
        in_groups(nb, [&](int b) { if (m < p.M) block_fetch<T>(row, src, s.n, b); }, [] { cp_async_commit(); });
    };
    auto put = [&](int m, int i, unsigned long long c) {            // an entry, 0: none
        p.val[(int64_t)m * p.k + i] = c ? key_logit((uint32_t)(c >> 32)) : -INFINITY;
        p.idx[(int64_t)m * p.k + i] = c ? (int32_t)~(uint32_t)c : -1;
    };
    // A cluster takes its threshold from all its group maxima, so that the lists of its CTAs are k entries together and not each; it
    // has to meet once more for that.
    const bool together = csize > 1 && p.k > kLgTogether;
    fetch((int)blockIdx.x / csize);
#pragma unroll 1
    for (int m = (int)blockIdx.x / csize; m < p.M; m += stride) {
        // maximum and sum of this thread's own words as they arrive
        RunSum run;
        float g0 = -INFINITY, g1 = -INFINITY;      // of the first and the last two words of the blocks
        as_they_arrive(nb, [&](int bl) {
            uint4 a[4];
            block_load(row, bl, a);
            const float2 half = Row<T>::block_max(a);
            const float top = fmaxf(half.x, half.y);
            bmax[bl * kLgThreads + tid] = (uint16_t)(logit_key(top) >> 16);
            if (p.lse) run.add<T>(a, top, c1);
            else run.mx = fmaxf(run.mx, top);
            g0 = fmaxf(g0, half.x);
            g1 = fmaxf(g1, half.y);
        });
        *reinterpret_cast<float2*>(&sm->gmax[2 * tid]) = make_float2(g0, g1);
        {
            const float2 u = warp_run(run.mx, run.sum(), c1);
            if (lane == 0) sm->warps[warp] = u;
        }
        __syncthreads();
        if (together) {
            const int per = 2 * kLgThreads / csize;
            if (tid < per) {
                float g = sm->gmax[tid * csize];
                for (int i = 1; i < csize; ++i) g = fmaxf(g, sm->gmax[tid * csize + i]);
                sm->joined[tid] = g;
            }
            cluster_sync();
        }
        // k-th largest group maximum on the upper 16 bits of the key (a lower bound, exact for bf16), two bits at a time.  A
        // group is half the words of a thread, or all words of two threads when that still leaves 2 k groups.
        if (tid < 32) {
            constexpr int G = 2 * kLgThreads / 32;
            uint32_t thr = 0;
            if (together) {
                const int per = 2 * kLgThreads / csize;
                uint32_t key[G];
#pragma unroll
                for (int i = 0; i < G; ++i) {
                    const int g = i * 32 + lane;
                    key[i] = logit_key(ld_cluster_f32(mapa_shared(smem_u32(&sm->joined[g % per]), g / per))) >> 16;
                }
                thr = kth_key16(key, p.k);
            } else if (2 * p.k <= kLgThreads / 2) {
                uint32_t key[G / 4];
#pragma unroll
                for (int i = 0; i < G / 4; ++i) {
                    const float4 g = *reinterpret_cast<const float4*>(&sm->gmax[(i * 32 + lane) * 4]);
                    key[i] = logit_key(fmaxf(fmaxf(g.x, g.y), fmaxf(g.z, g.w))) >> 16;
                }
                thr = kth_key16(key, p.k);
            } else {
                uint32_t key[G];
#pragma unroll
                for (int i = 0; i < G; ++i) key[i] = logit_key(sm->gmax[i * 32 + lane]) >> 16;
                thr = kth_key16(key, p.k);
            }
            if (lane == 0) sm->thr = thr << 16;
        }
        __syncthreads();
        const uint32_t thr = max(sm->thr, 1u);
        const float tz = thr == 1u ? -FLT_MAX : key_logit(thr);      // thr = 1 (fewer than k groups hold anything): all visible elements
        // the blocks that reach it, then their words, one per lane
        constexpr int kHits = 4 * kLgThreads;
        const uint32_t lowest = max(thr >> 16, 0x0080u);      // (the key of the lowest finite value is 0x00800000)
        uint16_t* hit = reinterpret_cast<uint16_t*>(sm->gmax);
        for (int i = tid; i < nb * kLgThreads; i += kLgThreads)
            if (bmax[i] >= lowest) {
                const int at = atomicAdd(&sm->hits, 1);
                if (at < kHits) hit[at] = (uint16_t)i;
            }
        __syncthreads();
        const int hits = sm->hits;
        for (int i = tid; i < min(hits, kHits) * 4; i += kLgThreads) {
            const int h = hit[i >> 2], wd = h % kLgThreads + (h / kLgThreads * 4 + (i & 3)) * kLgThreads;
            if (wd >= words) continue;
            float v[W];
            Row<T>::elements(reinterpret_cast<const uint4*>(row)[wd], v);
            uint32_t in = 0;
#pragma unroll
            for (int e = 0; e < W; ++e) in |= (v[e] >= tz ? 1u : 0u) << e;
            for (; in; in &= in - 1) {
                const int j = wd * W + __ffs(in) - 1;
                const int at = atomicAdd(&sm->count, 1);
                if (at < p.cap) cand[at] = ((unsigned long long)logit_key(Row<T>::at(row, j)) << 32) | (uint32_t)~(s.begin + j);
            }
        }
        Base b;
        float mx, total;
        {
            const float2 u = sm->warps[lane % kLgWarps];
            mx = slots_max(u.x);
            b.set(mx, c1);
            total = slots_sum(at_base(u.x, u.y, b, c1));
        }
        __syncthreads();
        int n = sm->count;
        if (n > p.cap || hits > kHits) {
            // too many candidates (ties): exact key of the k-th element, then the lowest indices among its equals
            const int kk = p.k;                    // fewer than the elements above -inf
            uint32_t kth = 0;
            for (int b = 31; b >= 0; --b) {
                const uint32_t c = kth | (1u << b);
                int cnt = 0;
                for (int i = tid; i < words; i += kLgThreads)
                    for (int e = 0; e < W; ++e) cnt += logit_key(Row<T>::at(row, i * W + e)) >= c;
                if (cta_count(cnt, &sm->count) >= kk) kth = c;
            }
            int above = 0;
            for (int i = tid; i < words; i += kLgThreads)
                for (int e = 0; e < W; ++e) above += logit_key(Row<T>::at(row, i * W + e)) > kth;
            const int need = kk - cta_count(above, &sm->count);
            int last = -1;                         // largest index such that fewer than `need` equals lie at or below it
            for (int b = 30; b >= 0; --b) {
                const int c = last + (1 << b);     // (last + 1) | bit, minus 1
                if (c < last || c >= s.n) continue;
                int cnt = 0;
                for (int i = tid; i < words; i += kLgThreads)
                    for (int e = 0; e < W; ++e) cnt += i * W + e <= c && logit_key(Row<T>::at(row, i * W + e)) == kth;
                if (cta_count(cnt, &sm->count) < need) last = c;
            }
            __syncthreads();
            if (tid == 0) sm->count = 0;
            __syncthreads();
            for (int i = tid; i < words; i += kLgThreads)
                for (int e = 0; e < W; ++e) {
                    const int j = i * W + e;
                    const uint32_t key = logit_key(Row<T>::at(row, j));
                    if (key > kth || (key == kth && j <= last + 1)) {
                        const int at = atomicAdd(&sm->count, 1);
                        if (at < p.cap) cand[at] = ((unsigned long long)key << 32) | (uint32_t)~(s.begin + j);
                    }
                }
            __syncthreads();
            n = min(sm->count, p.cap);
        }
        fetch(m + stride);                     // nobody reads this row's slice any more
        const int have = rank_select(cand, n, p.k, list);
        if (!together) for (int i = have + tid; i < p.k; i += kLgThreads) list[i] = 0ull;
        if (tid == 0) { sm->part[0] = mx; sm->part[1] = total; sm->have = have; sm->hits = 0; }
        if (csize > 1) {
            cluster_sync();
            const uint32_t other = mapa_shared(smem_u32(&sm->part[0]), lane < csize ? lane : 0);
            const float pm = rank == 0 && lane < csize ? ld_cluster_f32(other) : -INFINITY, ps = rank == 0 && lane < csize ? ld_cluster_f32(other + 4) : 0.0f;
            if (together) {
                // every CTA takes a copy of all lists and finds the places of its own entries
                const int length = lane < csize ? (int)ld_cluster_u32(mapa_shared(smem_u32(&sm->have), lane)) : 0;
#pragma unroll
                for (int r = 0; r < kLgMaxCluster; ++r) {
                    const int len = __shfl_sync(0xFFFFFFFFu, length, r);
                    if (tid < len) cand[r * p.k + tid] = ld_cluster_u64(mapa_shared(smem_u32(list), r) + 8u * tid);
                }
                __syncthreads();
                if (warp * 32 < have) {
                    const unsigned long long c = tid < have ? cand[rank * p.k + tid] : 0ull;
                    int before = tid;
                    for (int r = 0; r < csize; ++r) {
                        const int len = __shfl_sync(0xFFFFFFFFu, length, r);
                        if (r != rank && len) before += count_above(cand + r * p.k, len, c);
                    }
                    if (tid < have && before < p.k) put(m, before, c);
                }
                const int all = __reduce_add_sync(0xFFFFFFFFu, length);
                if (rank == 0 && tid >= all && tid < p.k) put(m, tid, 0ull);
            } else if (rank == 0) {
                // every CTA's list, k entries each (cap holds cluster size x k); the place of its own is cleared for the result
                for (int i = tid; i < csize * p.k; i += kLgThreads) {
                    const int r = i / p.k, j = i - r * p.k;
                    cand[i] = ld_cluster_u64(mapa_shared(smem_u32(list), r) + 8u * j);
                    if (r == 0) list[j] = 0ull;
                }
                __syncthreads();
                for (int i = tid; i < csize * p.k; i += kLgThreads) {
                    const unsigned long long c = cand[i];
                    if (c == 0ull) continue;
                    const int own = i / p.k;
                    int before = i - own * p.k;
                    for (int r = 0; r < csize; ++r)
                        if (r != own) before += count_above(cand + r * p.k, p.k, c);
                    if (before < p.k) list[before] = c;
                }
            }
            if (rank == 0) {
                b.set(warp_max(pm), c1);
                total = warp_sum(at_base(pm, ps, b, c1));
            }
        }
        __syncthreads();
        if (tid == 0) sm->count = 0;
        if (rank == 0) {
            if (!together) for (int i = tid; i < p.k; i += kLgThreads) put(m, i, list[i]);
            if (p.lse && tid == 0) p.lse[m] = b.m * p.inv_tau + logf(total);
        }
        // lists and parts stay until all have read them; where the cluster meets for its threshold that says so
        if (csize > 1 && !(together && m + stride < p.M)) cluster_sync();
    }
}

// ==================================================================================== host
// CTAs per row.  One CTA per row is the least work; a row is cut when its slice would leave no room for three CTAs on the SM
// (copies, sums and stores of different rows then overlap), or when there are too few rows to fill the SMs.
static int row_cluster(int M, int V, int esz) {
    int c = 1;
    while (c < kLgMaxCluster && (int64_t)V * esz > (int64_t)c * 64 * 1024) c *= 2;
    while (c < kLgMaxCluster && (int64_t)M * c * 2 <= 2 * 148 && V / (2 * c) >= 4096) c *= 2;
    return c;
}
// ... and the bytes of a slice, in whole blocks, with its marks (4 bytes per block and thread) or maxima (2)
static size_t slice_bytes(int V, int c, int esz, int per_block) {
    const size_t row = ((size_t)((V + c - 1) / c + 7) / 8 * 8) * esz;
    return (size_t)blocks_of((int)(row / 16)) * kLgThreads * (4 * 16 + per_block);
}

template <typename P>
static quaff_status_t launch_rows(void (*kernel)(const P, int), const P& p, int M, int V, int esz, size_t fixed, int per_block, int slot, cudaStream_t st) {
    static std::atomic<bool> configured[4][64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return QUAFF_ERR_CUDA;
    if (!configured[slot][dev].load()) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kLgSmemMax) != cudaSuccess) return QUAFF_ERR_CUDA;
        configured[slot][dev].store(true);
    }
    const int c = row_cluster(M, V, esz);
    const size_t smem = fixed + slice_bytes(V, c, esz, per_block);
    const int per_sm = max(1, min(3, (int)(kLgSmemSm / (smem + 1024))));       // (three CTAs' registers fill an SM)
    const int64_t groups = min((int64_t)M, max((int64_t)1, (int64_t)sm_count() * per_sm / c));
    launch_pdl(kernel, dim3((unsigned)(groups * c)), dim3(kLgThreads), smem, st, c, p, c);
    return launch_status();
}

}  // namespace quaff

using namespace quaff;

extern "C" quaff_status_t quaff_topk_logits(const void* Z, int z_dtype, int64_t ldz, int M, int V, int k, float temperature, float* val, int32_t* idx,
                                            float* lse_opt, quaff_stream_t stream) {
    QUAFF_RETURN_IF(M < 0 || V <= 0 || k <= 0 || (M > 0 && (!Z || !val || !idx)) || ldz < V, QUAFF_ERR_INVALID_ARG);
    QUAFF_RETURN_IF(z_dtype != QUAFF_BF16 && z_dtype != QUAFF_F32, QUAFF_ERR_INVALID_ARG);
    QUAFF_RETURN_IF(!(temperature >= FLT_MIN) || isinf(temperature), QUAFF_ERR_INVALID_ARG);      // (1 / temperature and that times log2 e are floats)
    const int esz = z_dtype == QUAFF_F32 ? 4 : 2;
    QUAFF_RETURN_IF(k > kLgMaxK || (int64_t)V * esz > (int64_t)kLgMaxCluster * (kLgSliceMax - 64) || M > (1 << 27), QUAFF_ERR_UNSUPPORTED_SHAPE);
    QUAFF_RETURN_IF(!aligned16(Z) || (ldz * esz) % 16, QUAFF_ERR_ALIGNMENT);
    if (M == 0) return QUAFF_OK;
    // candidates: as a rule k and a few (at most about 1.4 k with 2 k groups); clusters gather their lists in the same place
    const int cap = (int)round_up((size_t)max(max(512, 4 * k), row_cluster(M, V, esz) * k), 32);
    const TopkParams p = {Z, ldz, M, V, k, cap, 1.0f / temperature, val, idx, lse_opt};
    const size_t fixed = (sizeof(TopkSmem) + 15) / 16 * 16 + ((size_t)((k + 1) & ~1) + cap) * 8;
    if (esz == 4) return launch_rows(topk_logits_kernel<float>, p, M, V, esz, fixed, 2, 0, (cudaStream_t)stream);
    return launch_rows(topk_logits_kernel<uint16_t>, p, M, V, esz, fixed, 2, 1, (cudaStream_t)stream);
}

extern "C" quaff_status_t quaff_distill_topk(const void* Z, int z_dtype, int64_t ldz, int M, int V, const float* t_val, const int32_t* t_idx, int k,
                                             const float* t_lse_opt, float temperature, const float* row_w_opt, float* loss, void* dZ_opt,
                                             int64_t lddz, quaff_stream_t stream) {
    QUAFF_RETURN_IF(M < 0 || V <= 0 || k <= 0 || ldz < V || (dZ_opt && lddz < V), QUAFF_ERR_INVALID_ARG);
    QUAFF_RETURN_IF(M > 0 && (!Z || !t_val || !t_idx || !loss), QUAFF_ERR_INVALID_ARG);
    QUAFF_RETURN_IF(z_dtype != QUAFF_BF16 && z_dtype != QUAFF_F32, QUAFF_ERR_INVALID_ARG);
    QUAFF_RETURN_IF(!(temperature >= FLT_MIN) || isinf(temperature), QUAFF_ERR_INVALID_ARG);      // (1 / temperature and that times log2 e are floats)
    const int esz = z_dtype == QUAFF_F32 ? 4 : 2;
    QUAFF_RETURN_IF(k > kLgMaxK || (int64_t)V * esz > (int64_t)kLgMaxCluster * (kLgSliceMax - 64) || M > (1 << 27), QUAFF_ERR_UNSUPPORTED_SHAPE);
    QUAFF_RETURN_IF(!aligned16(Z) || (ldz * esz) % 16 || (dZ_opt && (!aligned16(dZ_opt) || (lddz * esz) % 16)), QUAFF_ERR_ALIGNMENT);
    if (M == 0) return QUAFF_OK;
    const DistillParams p = {Z, ldz, M, V, k, t_val, t_idx, t_lse_opt, 1.0f / temperature, temperature, 1.0 / (double)temperature, row_w_opt, loss, dZ_opt, lddz};
    const size_t fixed = (sizeof(DistillSmem) + 15) / 16 * 16;
    if (esz == 4) return launch_rows(distill_kernel<float>, p, M, V, esz, fixed, 4, 2, (cudaStream_t)stream);
    return launch_rows(distill_kernel<uint16_t>, p, M, V, esz, fixed, 4, 3, (cudaStream_t)stream);
}
