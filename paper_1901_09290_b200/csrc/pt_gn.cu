// Group normalisation + residual add + activation on ragged channel counts and groups, channels last, forward and backward. NHWC bf16
// activations with channel pitch ld, fp32 statistics and parameters. Per image n and group g of m = H*W*|g| values:
//   forward : mean, rstd = 1/sqrt(var + eps), z = gamma*(x - mean)*rstd + beta (+ residual), y = act(z)
//   backward: dz = dy*act'(z), A = sum gamma*dz, B = sum gamma*dz*xhat, dx = rstd*(gamma*dz - A/m - xhat*B/m)
// Both directions need an image's sums before its first result, and are bound by memory: the aim is to read an image once.
//
// A unit of work is an image, or a slab of its channels (whole groups, whole 16-byte vectors) where that fills the device better. A thread-
// block cluster owns a unit; each of its blocks owns a run of consecutive pixels, and a thread of a block a 16-byte vector column and every so
// many-th pixel. Threads bring in what they will use themselves, by asynchronous copies into places of their own in shared memory, a ring of
// batches of a few pixels: there is nobody to wait for but one's own copies. A thread walks its pixels forwards for the sums; the blocks of
// the cluster exchange the groups' sums through distributed shared memory; and it walks the pixels BACKWARDS for the results: the last
// batches of the first walk are still in the ring, and the others were read last and are the likeliest to be in L2. Batches that the second
// walk is done with make room for the cluster's next unit. No atomics: sums in a fixed order (run-to-run identical). The forward pass's
// statistics are means and squares about the mean from a thread's first few pixels on, joined in 64 bits; the backward pass's sums are fp32
// in short chains. Two blocks of 256 threads share an SM, with up to 128 registers a thread: a thread's 40 to 48 constants (five or six per
// channel) and two or four pixels.
//
// Measured (B200; in brackets the bytes that have to move, at the copy rate of 6.56 TB/s, over the time): 64x28x28x371 with ReLU and a
// residual forward 27.7 us (0.61), backward 54.1 (0.52); 64x56x56x256 with SiLU forward 53.3 (0.59), with the checkpoint 63.3 (0.62),
// backward 83.8 (0.56), from the checkpoint and with y again 110.5 (0.50); with ReLU 47.7, 59.5, 79.2 and 92.2. The backward pass of
// 64x56x56x256 with SiLU reads 366 MB from DRAM where 206 would do: all images are in work at once, and the rings hold 19 of those 206 MB.
// It issues in 53 % of the cycles, DRAM is busy in 63 %; both passes of 64x28x28x371 with a residual issue in 34 and 46 % and keep DRAM busy
// in 37 and 51 %, waiting for loads and at barriers. The small ones are a row of latencies: launch, first load, sums, exchange, and for the
// backward pass a second launch for dgamma and dbeta.
//   (The first form had a producer warp and bulk copies of whole chunks of pixels. One thread issues such a copy every 0.3 to 0.5 us, which
// with two or three tensors was the bound: 150 to 260 us for the backward pass at 64x28x28x371 with a residual, by the chunk's size.
// Fewer images at a time, in rounds that fit L2, cost about 4.5 us a round and do not pay; nor do eviction hints on the copies.)
#include "pt_internal.h"
#include "pt_act.cuh"
#include "pt_sm100_ptx.cuh"

namespace {

constexpr int kGnThreads = 256;              // most threads of a block
constexpr int kGnTable = 256;                // most groups of a table
constexpr int kGnMaxLd = 2048;
constexpr int kGnMaxN = 1 << 24;             // most images: units, and steps behind the last one, are counted in 32 bits
constexpr int kGnMaxCluster = 16;
constexpr int kGnExchange = 1024;            // most entries (blocks of the cluster x groups) of one exchange buffer
constexpr int kGnSlabs = 32;                 // most slabs of channels
constexpr int kGnChain = 32;                 // units whose sums for dgamma and dbeta are added up in fp32

enum { kGnFwd = 0, kGnFwdPack = 1, kGnBwd = 2, kGnBwdPacked = 3 };

__host__ __device__ constexpr bool gn_bwd(int mode) { return mode >= kGnBwd; }
// Bytes of a thread's place for one pixel: the vectors of x (or codes and the word that holds the scale byte), dy and the residual.
__host__ __device__ constexpr int gn_slot(int mode, bool res) { return (mode == kGnBwdPacked ? 12 : 16) + (gn_bwd(mode) ? 16 : 0) + (gn_bwd(mode) && res ? 16 : 0); }
// Pixels of a thread's batch: four in the forward pass (28 us at 64x28x28x371 with a residual, 32 with two); the backward pass, which has
// twice the constants, is as fast with two.
__host__ __device__ constexpr int gn_rows(int mode) { return gn_bwd(mode) ? 2 : 4; }
// Batches of a thread's ring: what two blocks to an SM have room for.
__host__ __device__ constexpr int gn_batches(int mode, bool res) { return 290 / (gn_rows(mode) * gn_slot(mode, res)); }
// Words of a thread's place for its sums: eight pairs, and in the forward pass eight bf16 and a count besides. Odd, so that 32 places share no bank.
__host__ __device__ constexpr int gn_red(int mode) { return gn_bwd(mode) ? 17 : 21; }
__host__ __device__ constexpr int gn_ring(int mode, bool res) { return gn_rows(mode) * gn_batches(mode, res) * gn_slot(mode, res); }
constexpr int kGnBlocks = 2;                 // blocks of an SM: while one exchanges its sums, the other one moves data
constexpr size_t kGnSmem = 113 * 1024, kGnSmemMost = 226 * 1024;     // shared memory of a block: two on an SM, one

struct GnP {
    int N, HW, C, ld, LV, ldq, nb, G, cg;        // (cg: channels of a group without a table)
    int slabs, gs;               // slabs of channels, most groups of one; a unit of work is an image's slab
    int w, rl, ppb, threads;     // lanes of a checkpoint's block, lanes of a pixel, pixels the threads cover at a time, threads
    int gl, gc;                  // lanes that add up a group, and those of them that take different channels (as powers of two)
    int cl, clusters, share;     // blocks of a cluster, clusters, pixels of a block
    int step_n, step_s;          // a cluster's next unit: images and slabs further on
    int table;
    unsigned sm_gid, sm_gam, sm_bet, sm_grp, sm_red, sm_xch, sm_acc, sm_ring;
    float eps;
    uint16_t slab_v[kGnSlabs + 1], slab_g[kGnSlabs + 1];         // first vector and first group of each slab
    uint16_t begin[kGnTable + 1];
};

struct GnArgs {
    const uint4 *x, *res, *dy;
    const uint8_t *codes_in, *scales_in;
    const float *gamma, *beta, *mean, *rstd;
    float *save_mean, *save_rstd;
    uint4 *y, *dx, *dres;
    uint8_t *codes, *scales;
    float *rows;                 // backward: [blocks][2][ld] sums of dz and dz * xhat over a block's units
    double *wide;                // [blocks][2][ld] those of all but its last few units
    float *dgamma, *dbeta;
};

__device__ __forceinline__ int group_begin(const GnP &p, int g) { return p.table ? p.begin[g] : g * p.cg; }

// ---- pairs of fp32 values in one 64-bit register: one instruction adds or multiplies both
struct f2 { unsigned long long v; };
__device__ __forceinline__ f2 mk2(float a, float b) { f2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void un2(f2 x, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x.v)); }
__device__ __forceinline__ f2 add2(f2 a, f2 b) { f2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ f2 mul2(f2 a, f2 b) { f2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) { f2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v)); return r; }
// two bf16 as fp32
__device__ __forceinline__ f2 from_bf(uint32_t w) { return mk2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ uint32_t to_bf(f2 x)
{
    float a, b;
    un2(x, a, b);
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ float bf_half(uint32_t w, int i) { return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16); }
// 1/x to some 46 bits, from fp32's by a Newton step.
__device__ __forceinline__ double inverse(double x) { const double r = (double)(1.f / (float)x); return r * fma(-x, r, 2.0); }

// A group's sums, by direction: fp32 in the backward pass; the forward pass takes a variance from them, for which they are kept in 64 bits.
template <bool BWD> struct GnSums { typedef float T; typedef float2 T2; };
template <> struct GnSums<false> { typedef double T; typedef double2 T2; };

__device__ __forceinline__ float ex2(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ float rcp(float x) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }

// SiLU works on w = -z * log2(e), which costs nothing: the factor is in the constants that give z. sigmoid(z) = 1/(1 + 2^w), 2 ulp and
// |z| * 2^-24 off. One reciprocal serves a pair, 1/a = b/(a*b): the special-function units take 8 cycles for an instruction of a warp, and
// with two exponentials and two reciprocals per pair, twice in the backward pass, they were the bound at 64x56x56x256 (46 us of their time
// alone; 35 with one reciprocal). 2^w stops at 2^60, so that a*b is finite: below z = -41.6 the sigmoid stays 1e-18, and z*sigmoid(z) is
// 1e-9 at most where |z| < 2^30. A residual, which may be of the type's lowest value, is taken as -2^20 at least (a clamp of w itself took
// 12 % longer). A NaN stays in w and leaves its neighbour in the pair alone.
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
__device__ __forceinline__ f2 sigmoid_w(f2 w, f2 &e)                       // e: 2^w, so that 1 - sigmoid is e * sigmoid
{
    float a, b;
    un2(w, a, b);
    e = mk2(fminf(ex2(a), 1.152921504606846976e18f), fminf(ex2(b), 1.152921504606846976e18f));
    un2(add2(e, mk2(1.f, 1.f)), a, b);
    const float r = rcp(a * b);
    return mk2(r * b, r * a);
}
__device__ __forceinline__ f2 silu_residual(uint32_t w)
{
    const uint32_t low = 0xc980c980u;                                    // -2^20, twice
    const __nv_bfloat162 h = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162 *>(&w), *reinterpret_cast<const __nv_bfloat162 *>(&low));
    return from_bf(*reinterpret_cast<const uint32_t *>(&h));
}

template <int ACT>
__device__ __forceinline__ f2 activate2(f2 z)
{
    if (ACT == PT_ACT_NONE) return z;
    if (ACT == PT_ACT_SILU) {                                            // (of w)
        f2 e;
        return mul2(mul2(z, mk2(-kLn2, -kLn2)), sigmoid_w(z, e));
    }
    float a, b;
    un2(z, a, b);
    return mk2(a > 0.f ? a : (a != a ? a : 0.f), b > 0.f ? b : (b != b ? b : 0.f));
}

// Two values into the shared memory of another block of the cluster, visible there behind the cluster's barrier.
__device__ __forceinline__ void st_cluster_2f(uint32_t addr, float a, float b)
{
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(addr), "f"(a), "f"(b) : "memory");
}
__device__ __forceinline__ void st_cluster_2f(uint32_t addr, double a, double b)
{
    asm volatile("st.shared::cluster.v2.f64 [%0], {%1, %2};" ::"r"(addr), "d"(a), "d"(b) : "memory");
}
// The two halves of sm100::cluster_barrier. (Shared memory of another block may be written once that block has started.)
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// Asynchronous copies of a thread, in groups; waiting for all but the last `PENDING` groups.
__device__ __forceinline__ void copy16(uint32_t dst, const void *src) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void copy8(uint32_t dst, const void *src) { asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void copy4(uint32_t dst, const void *src) { asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int PENDING>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(PENDING) : "memory"); }

// The largest bf16 <= v (its bits): x > v exactly where x > that, for every bf16 x.
__device__ __forceinline__ uint32_t bf16_floor(float v)
{
    const uint32_t u = __float_as_uint(v);
    if ((u & 0x7fffffffu) > 0x7f800000u) return 0x7fc0u;                 // NaN: no x is above it
    return (u >> 31) ? ((u + 0xffffu) >> 16) : (u >> 16);                // (towards -inf: a negative one's magnitude rounds up)
}

__device__ __forceinline__ double exact_z(double x, float mean, float rstd, float gamma, float beta) { return (x - (double)mean) * (double)rstd * (double)gamma + (double)beta; }

// ReLU without a residual: z = s*(x - mean) + beta > 0, s = gamma*rstd, for bf16 x, as sg ^ x > th. For s > 0 that is x > mean - beta/s, for
// s < 0 -x > -(mean - beta/s), for s = 0 a constant. What fp32 leaves uncertain of the limit hardly ever lies about a bf16 value; where it
// does, or is out of range, z at the bf16 values themselves decides, in 64 bits. (A limit in 64 bits would not: beta may be lost beside the
// mean.) z rises with sg ^ x, so that a bisection finds the last value without z > 0: of the bf16 values in their order, number_of, between
// lo, which is such a value, and hi, which is none unless it is infinity.
__device__ __forceinline__ uint32_t number_of(uint32_t bits) { return bits & 0x8000u ? ~bits & 0xffffu : bits | 0x8000u; }
constexpr uint32_t kLowest = 0x7fu, kHighest = 0xff80u;                  // -inf and inf
__device__ __noinline__ uint32_t relu_limit_exact(float mean, float rstd, float gamma, float beta, uint32_t lo, uint32_t hi)     // th, and sg above it
{
    const double sd = (double)gamma * (double)rstd;
    if (sd == 0.0) return beta > 0.f ? 0xff80u : 0x7f80u;
    const uint32_t flip = sd < 0.0 ? 0x8000u : 0u;
    const auto bits_of = [](uint32_t i) { return i & 0x8000u ? i ^ 0x8000u : ~i & 0xffffu; };
    const auto above = [&](uint32_t i) { return exact_z((double)__uint_as_float((bits_of(i) ^ flip) << 16), mean, rstd, gamma, beta) > 0.0; };
    if (hi == kHighest && !above(hi)) lo = hi;                           // (statistics that are NaN)
    while (lo + 1u < hi) {
        const uint32_t mid = (lo + hi) >> 1;
        if (above(mid)) hi = mid;
        else lo = mid;
    }
    return bits_of(lo) | flip << 16;
}
__device__ __forceinline__ void relu_limit(float mean, float rstd, float gamma, float beta, uint32_t &th, uint32_t &sg)
{
    const float s = gamma * rstd, q = __fdividef(beta, s), lim = s < 0.f ? q - mean : mean - q, off = 1e-6f * (fabsf(mean) + fabsf(q));
    const bool in_range = fabsf(lim) > 1e-30f && fabsf(lim) < 1e30f && fabsf(s) > 1e-30f && fabsf(s) < 1e30f;
    sg = s < 0.f ? 0x8000u : 0u;
    th = bf16_floor(lim - off);
    const uint32_t up = bf16_floor(lim + off);
    if (th != up || !in_range) {
        th = relu_limit_exact(mean, rstd, gamma, beta, in_range ? number_of(th) : kLowest, in_range ? number_of(up) + 1u : kHighest);
        sg = th >> 16;
        th &= 0xffffu;
    }
}

// Which of two neighbouring values (bf16 halves of x) have z = gamma*xhat + beta + residual > 0, in 64 bits. Rarely called: fp32 decides
// everywhere but next to 0.
__device__ __noinline__ uint32_t exact_mask(uint32_t x, uint32_t r, int c, const uint16_t *gid, const float *grp, int G, const float *gam, const float *bet)
{
    uint32_t m = 0u;
    for (int h = 0; h < 2; ++h) {
        const int g = gid[c + h];
        const double xv = (double)__uint_as_float(h ? x & 0xffff0000u : x << 16), rv = (double)__uint_as_float(h ? r & 0xffff0000u : r << 16);
        if (exact_z(xv, grp[g], grp[G + g], gam[c + h], bet[c + h]) + rv > 0.0) m |= h ? 0xffff0000u : 0xffffu;
    }
    return m;
}

// A block's sums on to its own in 64 bits; the first time they are what those hold. Out of line: rarely called.
__device__ __noinline__ void empty_sums(double *wide, float *acc, int n, bool first)
{
    double *row = wide + (size_t)blockIdx.x * n;
    for (int e = threadIdx.x; e < n; e += blockDim.x) {
        row[e] = (first ? 0.0 : row[e]) + (double)acc[e];
        acc[e] = 0.f;
    }
}

// Eight restored values as pairs (act8::decode8), and two of them as bf16, in which they are exact: their upper halves.
__device__ __forceinline__ void decode8(const uint2 &q, uint32_t byte, f2 (&x)[4])
{
    const float s = act8::scale_of(byte);
    const f2 bias = mk2(-8388736.f, -8388736.f), ss = mk2(s, s);
    const uint32_t a = q.x ^ 0x80808080u, b = q.y ^ 0x80808080u;
    x[0] = mk2(__uint_as_float(__byte_perm(a, 0x4b000000u, 0x7440)), __uint_as_float(__byte_perm(a, 0x4b000000u, 0x7441)));
    x[1] = mk2(__uint_as_float(__byte_perm(a, 0x4b000000u, 0x7442)), __uint_as_float(__byte_perm(a, 0x4b000000u, 0x7443)));
    x[2] = mk2(__uint_as_float(__byte_perm(b, 0x4b000000u, 0x7440)), __uint_as_float(__byte_perm(b, 0x4b000000u, 0x7441)));
    x[3] = mk2(__uint_as_float(__byte_perm(b, 0x4b000000u, 0x7442)), __uint_as_float(__byte_perm(b, 0x4b000000u, 0x7443)));
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = mul2(add2(x[i], bias), ss);
}
__device__ __forceinline__ uint32_t exact_bf(f2 x)
{
    float a, b;
    un2(x, a, b);
    return __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632);
}

// What a thread reads of one pixel: its vector of x (or of codes, with the block's scale byte), of dy and of the residual.
struct Raw {
    uint4 x, dy, res;
    uint2 q;
    uint32_t byte;
};

template <int MODE, int ACT, bool RES>
__global__ void __launch_bounds__(kGnThreads, kGnBlocks) gn_kernel(const __grid_constant__ GnP p, const GnArgs a)
{
    constexpr bool BWD = gn_bwd(MODE), PACK = MODE == kGnFwdPack, PACKED = MODE == kGnBwdPacked;
    constexpr int B = gn_batches(MODE, RES), U = gn_rows(MODE), kRed = gn_red(MODE);
    typedef typename GnSums<BWD>::T Sum;
    typedef typename GnSums<BWD>::T2 Sum2;
    // the ring's parts, [B][U][threads] each: x or codes, dy, residual, scale words
    constexpr uint32_t kXs = PACKED ? 8 : 16, kRowX = kGnThreads * kXs, kRow = kGnThreads * 16, kRowS = kGnThreads * 4, kPlace = U * kRow;
    constexpr uint32_t kDy = B * U * kRowX, kRes = kDy + (BWD ? B * U * kRow : 0), kSc = kRes + (BWD && RES ? B * U * kRow : 0);
    extern __shared__ __align__(128) uint8_t smem[];
    uint16_t *gid = reinterpret_cast<uint16_t *>(smem + p.sm_gid);       // [ld] group of a channel
    float *gam = reinterpret_cast<float *>(smem + p.sm_gam), *bet = reinterpret_cast<float *>(smem + p.sm_bet);      // [ld]
    float *grps = reinterpret_cast<float *>(smem + p.sm_grp);            // [2][2][G] of alternating images: mean and rstd (backward)
    float *out = grps + 4 * p.G;                                         // [2][G] rstd and mean (forward), the group's terms of dx (backward)
    float *red = reinterpret_cast<float *>(smem + p.sm_red);             // [threads][kRed]
    Sum2 *xch = reinterpret_cast<Sum2 *>(smem + p.sm_xch);               // [2][cl][gs], of alternating images; one without clusters
    float *acc = reinterpret_cast<float *>(smem + p.sm_acc);             // [2][ld] sums of dz and dz * xhat over the block's last units
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31, warps = p.threads >> 5;
    const int rank = (int)(blockIdx.x % p.cl), cluster = (int)(blockIdx.x / p.cl);
    const int first = rank * p.share, mine = p.HW - first < p.share ? (p.HW - first > 0 ? p.HW - first : 0) : p.share;
    const int step = U * p.ppb, full = mine / step, NB = full * step < mine ? full + 1 : full;     // pixels of a batch; whole batches, and all
    const int pr0 = t / p.rl, cv0 = t - pr0 * p.rl, pr = pr0 < p.ppb ? pr0 : 0;
    const uint8_t *mine_x = smem + p.sm_ring + t * kXs, *mine_v = smem + p.sm_ring + t * 16, *mine_s = smem + p.sm_ring + kSc + t * 4;
    const uint32_t to_x = sm100::smem_u32(mine_x), to_v = sm100::smem_u32(mine_v), to_s = sm100::smem_u32(mine_s);
    if (p.cl > 1) cluster_arrive();                                      // (waited for before the first exchange)
    for (int g = t; g < p.G; g += p.threads)
        for (int c = group_begin(p, g), e = group_begin(p, g + 1); c < e; ++c) gid[c] = (uint16_t)g;
    for (int c = p.C + t; c < p.ld; c += p.threads) gid[c] = (uint16_t)(p.G - 1);
    sm100::grid_dependency_wait();
    sm100::grid_launch_dependents();
    // Offsets in bytes from an image's first pixel of this block: 32 bits, added to addresses that all threads share.
    const uint32_t row = (uint32_t)p.ld * 2u, step_v = (uint32_t)step * row, step_q = (uint32_t)step * (uint32_t)p.ldq, step_s = (uint32_t)step * (uint32_t)p.nb;
    const uint32_t row_u = (uint32_t)p.ppb * row, row_q = (uint32_t)p.ppb * (uint32_t)p.ldq, row_s = (uint32_t)p.ppb * (uint32_t)p.nb;   // from one of a thread's pixels to the next
    const auto bytes = [](const void *q) { return reinterpret_cast<const uint8_t *>(q); };
    // A unit's tensors from the block's first pixel and the slab's first channel on, and the thread's vector there. Threads without a vector
    // of their own (t >= rl * ppb, lanes behind a narrower slab or that fill up a checkpoint's block) read vector 0 and store nothing. Vectors
    // of pad lanes only are read and come out as zeros; their codes, which there are none of, are read as vector 0's.
    struct Pos { uint32_t v, q, s; };                                    // offsets of a thread's first pixel of a batch: vectors, codes, scales
    struct Src {
        const uint8_t *x, *dy, *res, *q, *s;
        Pos at;                                                          // of batch 0
    };
    const auto moved = [&](const Pos &o, int b) { return Pos{o.v + (uint32_t)b * step_v, o.q + (uint32_t)b * step_q, o.s + (uint32_t)b * step_s}; };
    const auto source = [&](int n, int sl) {
        Src g{};
        const int v0 = p.slab_v[sl], nv = p.slab_v[sl + 1] - v0;
        const size_t pix = (size_t)n * p.HW + first;
        const int cv = pr0 < p.ppb && cv0 < nv ? cv0 : 0, cq = (v0 + cv) * 8 < p.C ? cv : 0;
        if (PACKED) {
            g.q = a.codes_in + pix * p.ldq + v0 * 8; g.s = a.scales_in + pix * p.nb + (v0 >> 2);
            g.at.q = (uint32_t)pr * (uint32_t)p.ldq + (uint32_t)cq * 8u; g.at.s = (uint32_t)pr * (uint32_t)p.nb + ((uint32_t)cq >> 2);
        } else {
            g.x = bytes(a.x) + pix * row + v0 * 16;
        }
        if (BWD) g.dy = bytes(a.dy) + pix * row + v0 * 16;
        if (RES) g.res = bytes(a.res) + pix * row + v0 * 16;
        g.at.v = (uint32_t)pr * row + (uint32_t)cv * 16u;
        return g;
    };
    // A batch into the ring's place s (in bytes of the vectors' part); `all`: the thread has all of its pixels, else those of the last batch.
    const int tail = mine - full * step - pr;                            // pixel u of the last batch is there if u * ppb < tail
    const auto bring = [&](const Src &g, const Pos &o, uint32_t s, bool all) {
        const auto one = [&](int u) {
            if (PACKED) {
                copy8(to_x + s / 2 + (uint32_t)u * kRowX, g.q + (o.q + (uint32_t)u * row_q));
                copy4(to_s + s / 4 + (uint32_t)u * kRowS, reinterpret_cast<const void *>(reinterpret_cast<uintptr_t>(g.s + (o.s + (uint32_t)u * row_s)) & ~(uintptr_t)3));
            } else {
                copy16(to_v + s + (uint32_t)u * kRow, g.x + (o.v + (uint32_t)u * row_u));
            }
            if (BWD) copy16(to_v + kDy + s + (uint32_t)u * kRow, g.dy + (o.v + (uint32_t)u * row_u));
            if (BWD && RES) copy16(to_v + kRes + s + (uint32_t)u * kRow, g.res + (o.v + (uint32_t)u * row_u));
        };
        if (all) {
#pragma unroll
            for (int u = 0; u < U; ++u) one(u);
        } else {
#pragma unroll 1
            for (int u = 0; u * p.ppb < tail && u < U; ++u) one(u);
        }
    };
    // (these loads first: behind the ring's copies they would wait for those)
    const bool ahead = BWD && p.gs <= p.threads;                         // a unit's statistics are fetched before they are needed
    float next_mean = 0.f, next_rstd = 0.f;
    const auto fetch_stats = [&](int n, int sl) {
        const int g = p.slab_g[sl] + t;
        if (ahead && g < p.slab_g[sl + 1]) {
            next_mean = a.mean[(size_t)n * p.G + g];
            next_rstd = a.rstd[(size_t)n * p.G + g];
        }
    };
    int n = p.slabs == 1 ? cluster : cluster / p.slabs, sl = cluster - n * p.slabs;      // the unit: image and slab
    fetch_stats(n, sl);
    // (A pad lane's z must not be near 0, see gradient: its beta is 1.) Every load comes before the ring's copies, behind which it would wait
    // for them all (10 us where the device has started everywhere at once); the first is stored behind them, its latency is theirs.
    const float gam0 = t < p.C ? a.gamma[t] : 0.f, bet0 = t < p.C ? a.beta[t] : 1.f;
    for (int c = p.threads + t; c < p.ld; c += p.threads) {
        gam[c] = c < p.C ? a.gamma[c] : 0.f;
        bet[c] = c < p.C ? a.beta[c] : 1.f;
    }
    Src src = source(n, sl);
    __syncthreads();                                                     // (every warp's loads are on their way)
    // (as much as keeps the memory busy until the first unit's constants are there; more would hold its threads up at the first barrier, copies being
    // accepted at the rate at which the memory serves them)
    constexpr int kFirst = 128 / (U * gn_slot(MODE, RES)) < 1 ? 1 : 128 / (U * gn_slot(MODE, RES)) < B ? 128 / (U * gn_slot(MODE, RES)) : B;
#pragma unroll 1
    for (int b = 0; b < kFirst; ++b) {
        if (b < NB) bring(src, moved(src.at, b), (uint32_t)b * kPlace, b < full);
        copy_commit();
    }
    if (t < p.ld) { gam[t] = gam0; bet[t] = bet0; }
    if (BWD)
        for (int c = t; c < 2 * p.ld; c += p.threads) acc[c] = 0.f;
    int dir = 0, it = 0;
    const float inv_hw = 1.f / (float)p.HW;
    const int whole = p.HW / p.share;                                    // blocks with all their pixels
    const float rest = (float)(p.HW - whole * p.share);                  // pixels of the one behind them
    while (n < p.N) {
        if (BWD && it > 0 && it % kGnChain == 0) {                       // (here: at the loop's end it would cost registers)
            __syncthreads();
            empty_sums(a.wide, acc, 2 * p.ld, it == kGnChain);
        }
        int next_n = n + p.step_n, next_s = sl + p.step_s;
        if (next_s >= p.slabs) { next_s -= p.slabs; next_n += 1; }
        const bool more = next_n < p.N;
        const int v0 = p.slab_v[sl], nv = p.slab_v[sl + 1] - v0, gb = p.slab_g[sl], ge = p.slab_g[sl + 1];
        const bool lane_ok = pr0 < p.ppb && cv0 < nv;
        const int cv = v0 + (lane_ok ? cv0 : 0), c0 = cv * 8;           // the thread's vector and its first channel
        const bool has = c0 < p.C;                                       // it holds channels, not pad lanes only
        const uint4 keep = act8::keep_bits(c0, p.C);
        const size_t base = (size_t)n * p.HW + first;                    // the block's first pixel
        // (so that a batch of the first walk always has B - 1 groups behind it when it is waited for)
        if (it > 0)
            for (int b = NB; b < B; ++b) copy_commit();
        // ---- what the first walk needs of every group: the statistics (backward)
        float *grp = grps + (it & 1) * 2 * p.G;
        if (BWD && ahead) {
            if (gb + t < ge) { grp[gb + t] = next_mean; grp[p.G + gb + t] = next_rstd; }
        } else if (BWD) {
            for (int g = gb + t; g < ge; g += p.threads) {
                grp[g] = a.mean[(size_t)n * p.G + g];
                grp[p.G + g] = a.rstd[(size_t)n * p.G + g];
            }
        }
        if (BWD) __syncthreads();
        // the thread's constants, backward: minus the mean, gamma*rstd, beta, and the ReLU's limits as bf16: without a residual, z > 0 exactly
        // where x ^ sgn > thr. Forward: minus the pivots, at first the values of the thread's first pixel.
        f2 nm[4], k[4], kz[4], be[4];                                    // (kz: k, or for SiLU what gives w)
        uint32_t thr[4], sgn[4];
        float be_max = 1e-30f;                                           // (z so small that bf16 might not hold it is decided there too)
        int taken = 0;                                                   // pixels that the thread's statistics hold (forward)
        int extra = 0;                                                   // the thread's pixels of the last, partial batch
        if (!BWD) {
#pragma unroll
            for (int u = 0; u < U; ++u) extra += u * p.ppb < tail;
            if (it == 0) copy_wait<kFirst - 1>();
            else copy_wait<B - 1>();
            uint4 v = make_uint4(0u, 0u, 0u, 0u);
            if (full + extra > 0) v = *reinterpret_cast<const uint4 *>(mine_v + (dir ? (B - 1) * kPlace : 0u));
            nm[0] = from_bf(v.x ^ 0x80008000u); nm[1] = from_bf(v.y ^ 0x80008000u); nm[2] = from_bf(v.z ^ 0x80008000u); nm[3] = from_bf(v.w ^ 0x80008000u);
        } else {
            float m[8], kk[8], b[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int c = c0 + j, g = gid[c];
                m[j] = -grp[g];
                kk[j] = gam[c] * grp[p.G + g];
                b[j] = bet[c];
                be_max = fmaxf(be_max, 1e-6f * fabsf(b[j]));
                if (ACT == PT_ACT_SILU) b[j] *= -kLog2e;
                if (ACT == PT_ACT_RELU && !RES) {
                    uint32_t th, sg;
                    relu_limit(grp[g], grp[p.G + g], gam[c], bet[c], th, sg);
                    thr[j >> 1] = j & 1 ? thr[j >> 1] | th << 16 : th;
                    sgn[j >> 1] = j & 1 ? sgn[j >> 1] | sg << 16 : sg;
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                nm[i] = mk2(m[2 * i], m[2 * i + 1]);
                k[i] = mk2(kk[2 * i], kk[2 * i + 1]);
                kz[i] = ACT == PT_ACT_SILU ? mul2(k[i], mk2(-kLog2e, -kLog2e)) : k[i];
                be[i] = mk2(b[2 * i], b[2 * i + 1]);
            }
        }
        // pixel u of a batch at the ring's place s; os: the thread's place in the scales
        const uint32_t s_base = PACKED ? (uint32_t)(reinterpret_cast<uintptr_t>(src.s) & 3u) : 0u;
        const auto fetch = [&](Raw &w, uint32_t os, uint32_t s, int u) {
            if (PACKED) {
                w.q = *reinterpret_cast<const uint2 *>(mine_x + s / 2 + (uint32_t)u * kRowX);
                w.byte = *reinterpret_cast<const uint32_t *>(mine_s + s / 4 + (uint32_t)u * kRowS) >> (((s_base + os + (uint32_t)u * row_s) & 3u) * 8u) & 0xffu;
            } else {
                w.x = *reinterpret_cast<const uint4 *>(mine_v + s + (uint32_t)u * kRow);
            }
            if (BWD) w.dy = *reinterpret_cast<const uint4 *>(mine_v + kDy + s + (uint32_t)u * kRow);
            if (BWD && RES) w.res = *reinterpret_cast<const uint4 *>(mine_v + kRes + s + (uint32_t)u * kRow);
        };
        const auto values = [&](Raw &w, f2 (&x)[4]) {                   // x as fp32 pairs (and, from codes, as bf16 words)
            if (PACKED) {
                decode8(w.q, w.byte, x);
                if (ACT == PT_ACT_RELU) w.x = make_uint4(exact_bf(x[0]), exact_bf(x[1]), exact_bf(x[2]), exact_bf(x[3]));
            } else {
                x[0] = from_bf(w.x.x); x[1] = from_bf(w.x.y); x[2] = from_bf(w.x.z); x[3] = from_bf(w.x.w);
            }
        };
        // dz: in place of dy's words where it is dy's bits under a mask, and as pairs. d: x - mean.
        const auto gradient = [&](Raw &w, const f2 (&d)[4], f2 (&z)[4], f2 (&dz)[4], bool want_z) {
            uint32_t *g = reinterpret_cast<uint32_t *>(&w.dy);
            const uint32_t *xb = reinterpret_cast<const uint32_t *>(&w.x), *rb = reinterpret_cast<const uint32_t *>(&w.res);
            if (ACT == PT_ACT_SILU || want_z || (ACT == PT_ACT_RELU && RES))
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    z[i] = fma2(d[i], kz[i], be[i]);
                    if (RES) z[i] = ACT == PT_ACT_SILU ? fma2(silu_residual(rb[i]), mk2(-kLog2e, -kLog2e), z[i]) : add2(z[i], from_bf(rb[i]));
                }
            if (ACT == PT_ACT_RELU && !RES) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t u = xb[i] ^ sgn[i];
                    g[i] &= __hgt2_mask(*reinterpret_cast<const __nv_bfloat162 *>(&u), *reinterpret_cast<const __nv_bfloat162 *>(&thr[i]));
                }
            }
            if (ACT == PT_ACT_RELU && RES) {
                // Where z is near 0, fp32 leaves it wrong by less than 2^-22 of |residual| + |beta|: there 64 bits decide. One test for the eight
                // values, the least |z| against the largest |residual| and |beta|: it is passed a few times in a hundred thousand.
                float zz[8], low = INFINITY;
                __nv_bfloat162 top = __float2bfloat162_rn(0.f);          // (a NaN, in a pad lane too, leaves the others' maximum alone)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    un2(z[i], zz[2 * i], zz[2 * i + 1]);
                    low = fminf(low, fminf(fabsf(zz[2 * i]), fabsf(zz[2 * i + 1])));
                    top = __hmax2(top, __habs2(*reinterpret_cast<const __nv_bfloat162 *>(&rb[i])));
                }
                const float rmax = fmaxf(__low2float(top), __high2float(top));
                if (low <= fmaf(rmax, 1e-6f, be_max)) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        // (gamma = 0, a pruned channel's or a pad lane's: z = beta + residual, of the right sign in fp32)
                        const bool near0 = gam[c0 + 2 * i] != 0.f && fabsf(zz[2 * i]) <= fmaf(fabsf(__uint_as_float(rb[i] << 16)), 1e-6f, be_max);
                        const bool near1 = gam[c0 + 2 * i + 1] != 0.f && fabsf(zz[2 * i + 1]) <= fmaf(fabsf(__uint_as_float(rb[i] & 0xffff0000u)), 1e-6f, be_max);
                        uint32_t m = (zz[2 * i] > 0.f ? 0xffffu : 0u) | (zz[2 * i + 1] > 0.f ? 0xffff0000u : 0u);
                        if (near0 || near1) m = exact_mask(xb[i], rb[i], c0 + 2 * i, gid, grp, p.G, gam, bet);
                        g[i] &= m;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {                        // (the sign is that of z as bf16)
                        const uint32_t u = to_bf(z[i]), zero = 0u;
                        g[i] &= __hgt2_mask(*reinterpret_cast<const __nv_bfloat162 *>(&u), *reinterpret_cast<const __nv_bfloat162 *>(&zero));
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                dz[i] = from_bf(g[i]);
                if (ACT == PT_ACT_SILU) {
                    // act' = s + z*s*(1 - s) = s * (1 - w * ln 2 * (e * s)): 1 - s by itself is a step of s wrong, and times a large z anything
                    f2 e;
                    const f2 s = sigmoid_w(z[i], e);
                    dz[i] = mul2(mul2(dz[i], s), fma2(z[i], mul2(mul2(e, s), mk2(-kLn2, -kLn2)), mk2(1.f, 1.f)));
                }
            }
        };

        if (it == 0)
#pragma unroll 1
            for (int b = kFirst; b < B; ++b) {
                if (b < NB) bring(src, moved(src.at, b), (uint32_t)b * kPlace, b < full);
                copy_commit();
            }
        // ---- first walk: sums of x - pivot and its square, or of dz and dz * (x - mean)
        f2 s0[4], s1[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) s0[i] = s1[i] = mk2(0.f, 0.f);
        const auto count = [&](Raw &w) {
            f2 x[4], z[4], dz[4];
            values(w, x);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = add2(x[i], nm[i]);
            if (BWD) gradient(w, x, z, dz, false);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f2 d = BWD ? dz[i] : x[i];
                s0[i] = add2(s0[i], d);
                s1[i] = fma2(d, x[i], s1[i]);
            }
        };
        // A thread's chains of additions stay short. Backward: every 64 rows the sums go to the thread's place in shared memory.
        // Forward: one-pass sums about a pivot lose a variance that is small beside the square of what the pivot is off by, and a first pixel
        // may be nothing like the rest (a border, a mask). So the thread keeps, for each channel, its pixels' mean, as a pivot of bf16 plus an
        // offset of fp32, and the sum of squares about that mean; a run's sums are joined to them, and the next run is taken about the new mean.
        // The runs end behind 4 and every 16 batches: what an odd first pixel leaves in the pivot falls as the pixels grow in number.
        bool flushed = false;
        const auto flush = [&](int batches) {
            float *o = red + t * kRed;
            if (!BWD) {
                const int now = (batches < full ? batches : full) * U + (batches > full ? extra : 0), run = now - taken;
                if (run > 0) {
                    const float inv = 1.f / (float)run;
                    float w = 1.f, w2 = 0.f;
                    if (taken > 0) { w = (float)run / (float)now; w2 = (float)taken * w; }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float sum[2], sq[2], off[2];
                        un2(s0[i], sum[0], sum[1]);
                        un2(s1[i], sq[0], sq[1]);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const int j = 2 * i + h;
                            const float d = sum[h] * inv;
                            sq[h] = fmaf(-sum[h], d, sq[h]);
                            sq[h] = sq[h] < 0.f ? 0.f : sq[h];           // (a NaN stays)
                            off[h] = d;
                            if (taken > 0) {
                                const float was = o[j], apart = d - was;
                                sq[h] = fmaf(apart * apart, w2, sq[h] + o[8 + j]);
                                off[h] = fmaf(apart, w, was);
                            }
                            o[8 + j] = sq[h];
                        }
                        if (batches < NB) {                              // the pivot of the next run
                            float q[2];
                            un2(nm[i], q[0], q[1]);                      // (minus the last one)
                            const uint32_t word = to_bf(mk2(off[0] - q[0], off[1] - q[1]));
                            nm[i] = from_bf(word ^ 0x80008000u);
#pragma unroll
                            for (int h = 0; h < 2; ++h) off[h] -= bf_half(word, h) + q[h];
                        }
                        o[2 * i] = off[0];
                        o[2 * i + 1] = off[1];
                    }
                    taken = now;
                } else if (now == 0) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) o[j] = 0.f;
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float u[4];
                    un2(s0[i], u[0], u[1]);
                    un2(s1[i], u[2], u[3]);
                    o[2 * i] = flushed ? o[2 * i] + u[0] : u[0];
                    o[2 * i + 1] = flushed ? o[2 * i + 1] + u[1] : u[1];
                    o[8 + 2 * i] = flushed ? o[8 + 2 * i] + u[2] : u[2];
                    o[9 + 2 * i] = flushed ? o[9 + 2 * i] + u[3] : u[3];
                }
                flushed = true;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) s0[i] = s1[i] = mk2(0.f, 0.f);
        };
        // the ring's places in the order of the walk, and where they begin and end
        const uint32_t s_first = dir ? (B - 1) * kPlace : 0u, s_last = dir ? 0u : (B - 1) * kPlace, s_step = dir ? 0u - kPlace : kPlace;
        const uint4 keep_own = lane_ok ? keep : make_uint4(0u, 0u, 0u, 0u);
        uint32_t s = s_first;
        Pos here = src.at, then = moved(src.at, B);
        int b = 0;
        do {
          for (const int end = min(BWD ? b + 64 / U : b == 0 ? 4 : (b & ~15) + 16, NB); b < end; ++b) {
            copy_wait<B - 1>();
            const bool all = b < full;
            if (PACK) {                                                  // (whole warps: the lanes of a checkpoint's block exchange)
                uint8_t *gq = a.codes + base * p.ldq + (size_t)b * step_q, *gs = a.scales + base * p.nb + (size_t)b * step_s;
                const auto store = [&](const Raw &w, uint32_t byte, int u) {
                    if (lane_ok && has) {
                        *reinterpret_cast<uint2 *>(gq + ((uint32_t)pr * (uint32_t)p.ldq + (uint32_t)c0 + (uint32_t)u * row_q)) = act8::encode8(w.x, byte);
                        if ((cv & 3) == 0) gs[(uint32_t)pr * (uint32_t)p.nb + (uint32_t)(cv >> 2) + (uint32_t)u * row_s] = (uint8_t)byte;
                    }
                };
                if (all) {
                    Raw w[U];
                    uint32_t top[U];
#pragma unroll
                    for (int u = 0; u < U; ++u) fetch(w[u], here.s, s, u);
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        count(w[u]);
                        w[u].x = act8::and4(w[u].x, keep_own);
                        top[u] = act8::amax8(w[u].x);
                    }
#pragma unroll
                    for (int u = 0; u < U; ++u) top[u] = act8::scale_byte(act8::block_max(top[u], p.w));
#pragma unroll
                    for (int u = 0; u < U; ++u) store(w[u], top[u], u);
                } else {
#pragma unroll 1
                    for (int u = 0; u < U; ++u) {
                        const bool ok = u * p.ppb < tail;
                        Raw w;
                        w.x = make_uint4(0u, 0u, 0u, 0u);
                        if (ok) {
                            fetch(w, here.s, s, u);
                            count(w);
                        }
                        w.x = act8::and4(w.x, keep_own);
                        const uint32_t byte = act8::scale_byte(act8::block_max(act8::amax8(w.x), p.w));
                        if (ok) store(w, byte, u);
                    }
                }
            } else if (all) {                                            // a batch at a time, its loads first
                Raw w[U];
#pragma unroll
                for (int u = 0; u < U; ++u) fetch(w[u], here.s, s, u);
#pragma unroll
                for (int u = 0; u < U; ++u) count(w[u]);
            } else {                                                     // (one copy of the code: a small image is one such batch)
#pragma unroll 1
                for (int u = 0; u * p.ppb < tail && u < U; ++u) {
                    Raw w;
                    fetch(w, here.s, s, u);
                    count(w);
                }
            }
            if (b + B < NB) bring(src, then, s, b + B < full);           // (the last B batches stay for the second walk)
            copy_commit();
            then = moved(then, 1);
            here = moved(here, 1);
            s = s == s_last ? s_first : s + s_step;
          }
          flush(b);
        } while (b < NB);
        if (!BWD) {                                                      // the pivots, behind offsets and squares, and the number of pixels
#pragma unroll
            for (int i = 0; i < 4; ++i) reinterpret_cast<uint32_t *>(red)[t * kRed + 16 + i] = to_bf(nm[i]) ^ 0x80008000u;
            red[t * kRed + 20] = (float)taken;
        }
        // ---- a group's sums over the threads' rows and its channels
        __syncthreads();
        if (p.cl > 1 && it == 0) cluster_wait();
        {
            // a group's lanes: gc of them take its channels, the others more of the threads' rows
            const int gl = 1 << p.gl, gc = 1 << p.gc, per = 32 >> p.gl, l = lane & (gl - 1), lc = l & (gc - 1), lr = l >> p.gc, nr = gl >> p.gc, buf = p.cl > 1 ? it & 1 : 0;
            for (int g0 = gb + warp * per; g0 < ge; g0 += warps * per) {
                const int g = g0 + (lane >> p.gl);
                const int b = g < ge ? group_begin(p, g) : 0, e = g < ge ? group_begin(p, g + 1) : 0;
                Sum f0 = 0, f1 = 0, one = 0;
                if (!BWD && g < ge && mine > 0) one = inverse((double)mine * (double)(e - b));
                float ref = 0.f, ref_off = 0.f;
                if (BWD) {
                    for (int c = b + lc; c < e; c += gc) {
                        const float *src = red + (lr * p.rl + (c >> 3) - v0) * kRed + (c & 7);
                        float w0 = 0.f, w1 = 0.f;
#pragma unroll 4
                        for (int r = lr; r < p.ppb; r += nr, src += nr * p.rl * kRed) { w0 += src[0]; w1 += src[8]; }
                        f0 += gam[c] * w0;
                        f1 += gam[c] * w1;
                    }
                } else {
                    // The threads' means as differences from that of the group's first thread and channel, which may be far from the others:
                    // sums about it in 64 bits.
                    const auto pivot = [&](const float *place, int c) { return bf_half(reinterpret_cast<const uint32_t *>(place)[16 + ((c & 7) >> 1)], c); };
                    if (g < ge) {
                        const float *first_place = red + ((b >> 3) - v0) * kRed;
                        ref = pivot(first_place, b);
                        ref_off = first_place[b & 7];
                    }
                    float m2 = 0.f;
                    for (int c = b + lc; c < e; c += gc) {
                        const float *src = red + (lr * p.rl + (c >> 3) - v0) * kRed;
#pragma unroll 4
                        for (int r = lr; r < p.ppb; r += nr, src += nr * p.rl * kRed) {
                            const Sum d = (Sum)((pivot(src, c) - ref) + (src[c & 7] - ref_off)), dn = d * (Sum)src[20];
                            m2 += src[8 + (c & 7)];
                            f0 += dn;
                            f1 += dn * d;
                        }
                    }
                    f1 += (Sum)m2;
                }
                for (int o = gl >> 1; o; o >>= 1) {
                    f0 += __shfl_xor_sync(0xffffffffu, f0, o);
                    f1 += __shfl_xor_sync(0xffffffffu, f1, o);
                }
                if (!BWD) {                                              // the block's mean and sum of squares about it
                    const Sum d = f0 * one;
                    f1 -= f0 * d;
                    f1 = f1 < 0 ? 0 : f1;
                    f0 = (Sum)ref + (Sum)ref_off + d;
                }
                if (g < ge)
                    for (int r = l; r < p.cl; r += gl) {
                        Sum2 *to = xch + (buf * p.cl + rank) * p.gs + (g - gb);
                        if (p.cl == 1) { to->x = f0; to->y = f1; }
                        else st_cluster_2f(sm100::map_to_rank(sm100::smem_u32(to), (uint32_t)r), f0, f1);
                    }
            }
            // (divided before the wait)
            const int own_g = gb + t;
            const Sum inv_n = BWD ? 0 : inverse(p.HW);
            const float im0 = own_g < ge ? inv_hw / (float)(group_begin(p, own_g + 1) - group_begin(p, own_g)) : 0.f;
            if (p.cl > 1) sm100::cluster_barrier();
            else __syncthreads();
            // ---- the image's values from those of the cluster's blocks, in order
            for (int g = own_g; g < ge; g += p.threads) {
                const Sum2 *v = xch + buf * p.cl * p.gs + (g - gb);
                const int size = group_begin(p, g + 1) - group_begin(p, g);
                const float im = g == own_g ? im0 : inv_hw / (float)size;
                if (BWD) {
                    float e0 = 0.f, e1 = 0.f;
                    for (int r = 0; r < p.cl; ++r) { e0 += v[r * p.gs].x; e1 += v[r * p.gs].y; }
                    const float rs = grp[p.G + g], t1 = -(rs * (rs * (rs * (e1 * im))));     // (rs^3 by itself may not be an fp32 number)
                    out[g] = -(rs * e0 * im);
                    out[p.G + g] = t1;
                } else {
                    // All blocks but the last have `share` pixels (those behind the last have none). Means are averaged as differences from the
                    // first block's, and the squares of what the blocks' means differ by belong to the variance.
                    const Sum ref = v[0].x;
                    Sum d = 0, sq = 0, spread = 0;
                    for (int r = 0; r < whole; ++r) {
                        const Sum o = v[r * p.gs].x - ref;
                        d += o; spread += o * o; sq += v[r * p.gs].y;
                    }
                    d *= p.share; spread *= p.share;
                    if (rest > 0.f) {
                        const Sum o = v[whole * p.gs].x - ref, n = o * rest;
                        d += n; spread += n * o; sq += v[whole * p.gs].y;
                    }
                    spread -= d * d * inv_n;
                    d *= inv_n;
                    // (squares that fp32 does not hold are an infinity or a NaN by now, and no variance)
                    const float var = (float)((spread * size + sq) * (Sum)im);
                    const float fm = (float)(ref + d), fr = var < INFINITY ? 1.f / sqrtf(var + p.eps) : __uint_as_float(0x7fc00000u);
                    out[g] = fr;
                    out[p.G + g] = fm;
                    if (rank == 0) {
                        a.save_mean[(size_t)n * p.G + g] = fm;
                        a.save_rstd[(size_t)n * p.G + g] = fr;
                    }
                }
            }
        }
        __syncthreads();
        // The second walk's constants: forward, minus the mean, gamma*rstd and beta; backward, the group's terms of dx. (About x - mean: folded
        // into z = x*k + (beta - mean*k) they would save an addition, and lose z where the variance is far below the mean's square: of a
        // constant group of 1000, with rstd = 316 from eps, 0.02.)
        f2 c1[4], c2[4];
        {
            float u[8], v[8], m[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int c = c0 + j, g = gid[c];
                u[j] = out[g];
                v[j] = out[p.G + g];
                if (!BWD) {
                    m[j] = -v[j];
                    u[j] *= ACT == PT_ACT_SILU ? -kLog2e * gam[c] : gam[c];
                    v[j] = ACT == PT_ACT_SILU ? -kLog2e * bet[c] : bet[c];
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                c1[i] = mk2(u[2 * i], u[2 * i + 1]);
                c2[i] = mk2(v[2 * i], v[2 * i + 1]);
                if (!BWD) nm[i] = mk2(m[2 * i], m[2 * i + 1]);
            }
        }
        if (more) fetch_stats(next_n, next_s);
        // ---- second walk, backwards: the results
        const bool want_y = !BWD || (PACKED && a.y);
        // the unit's first pixel in dx, dresidual and y
        const size_t unit_v = base * row + (size_t)v0 * 16;
        uint8_t *const gx = reinterpret_cast<uint8_t *>(a.dx) + unit_v, *const gr = reinterpret_cast<uint8_t *>(a.dres) + unit_v, *const gy = reinterpret_cast<uint8_t *>(a.y) + unit_v;
        const auto result = [&](Raw &w, uint32_t at) {
            f2 x[4], z[4], dz[4];
            uint4 o;
            uint32_t *ow = reinterpret_cast<uint32_t *>(&o);
            values(w, x);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = add2(x[i], nm[i]);
            if (!BWD) {
                const uint32_t *rb = reinterpret_cast<const uint32_t *>(&w.res);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    f2 y = fma2(x[i], c1[i], c2[i]);
                    if (RES) y = ACT == PT_ACT_SILU ? fma2(silu_residual(rb[i]), mk2(-kLog2e, -kLog2e), y) : add2(y, from_bf(rb[i]));
                    ow[i] = to_bf(activate2<ACT>(y));
                }
                if (lane_ok) *reinterpret_cast<uint4 *>(gy + at) = act8::and4(o, keep);
            } else {
                gradient(w, x, z, dz, want_y);
#pragma unroll
                for (int i = 0; i < 4; ++i) ow[i] = to_bf(fma2(k[i], dz[i], fma2(x[i], c2[i], c1[i])));
                if (lane_ok) *reinterpret_cast<uint4 *>(gx + at) = act8::and4(o, keep);
                if (a.dres) {
                    if (ACT == PT_ACT_SILU) w.dy = make_uint4(to_bf(dz[0]), to_bf(dz[1]), to_bf(dz[2]), to_bf(dz[3]));
                    if (lane_ok) *reinterpret_cast<uint4 *>(gr + at) = act8::and4(w.dy, keep);
                }
                if (want_y) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) ow[i] = to_bf(activate2<ACT>(z[i]));
                    if (lane_ok) *reinterpret_cast<uint4 *>(gy + at) = act8::and4(o, keep);
                }
            }
        };
        Raw ahead_w[U];                                                  // forward: the residual, a batch ahead
        here = moved(src.at, NB - 1);
        const uint8_t *const res_v = RES ? src.res : nullptr;
        const auto residual = [&](uint32_t at, bool all) {
            if (!BWD && RES)
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (all || u * p.ppb < tail) ahead_w[u].res = *reinterpret_cast<const uint4 *>(res_v + (at + (uint32_t)u * row_u));
        };
        if (NB > 0) residual(here.v, NB == full);
        const int kept = NB < B ? NB : B;
        for (int b = NB - 1; b >= 0; --b) {
            s = s == s_first ? s_last : s - s_step;
            copy_wait<B - 1>();
            Raw w[U];
            if (!BWD && RES) {
#pragma unroll
                for (int u = 0; u < U; ++u) w[u].res = ahead_w[u].res;
                if (b > 0) residual(here.v - step_v, true);
            }
            if (b < full) {
#pragma unroll
                for (int u = 0; u < U; ++u) fetch(w[u], here.s, s, u);
#pragma unroll
                for (int u = 0; u < U; ++u) result(w[u], here.v + (uint32_t)u * row_u);
            } else {
#pragma unroll 1
                for (int u = 0; u * p.ppb < tail && u < U; ++u) {
                    Raw v;
                    if (!BWD && RES) v.res = *reinterpret_cast<const uint4 *>(res_v + (here.v + (uint32_t)u * row_u));
                    fetch(v, here.s, s, u);
                    result(v, here.v + (uint32_t)u * row_u);
                }
            }
            // the place takes an earlier batch, or one of the cluster's next unit: its first goes to the place that is free first
            if (b >= B) {
                bring(src, moved(here, -B), s, true);
            } else if (more) {
                const int m = kept - 1 - b;
                if (m == 0) src = source(next_n, next_s);
                bring(src, moved(src.at, m), (uint32_t)(dir ? m : B - 1 - m) * kPlace, m < full);
            }
            copy_commit();
            here = moved(here, -1);
        }
        if (BWD)                                                         // the images' sums of dz and dz * xhat, a channel's
            for (int c = v0 * 8 + t; c < min(p.C, (v0 + nv) * 8); c += p.threads) {
                const float *src = red + ((c >> 3) - v0) * kRed + (c & 7);
                float w0 = 0.f, w1 = 0.f, u0 = 0.f, u1 = 0.f;
                int r = 0;
                for (; r + 1 < p.ppb; r += 2, src += 2 * p.rl * kRed) {
                    w0 += src[0]; w1 += src[8];
                    u0 += src[p.rl * kRed]; u1 += src[p.rl * kRed + 8];
                }
                if (r < p.ppb) { w0 += src[0]; w1 += src[8]; }
                acc[c] += w0 + u0;
                acc[p.ld + c] += (w1 + u1) * grp[p.G + gid[c]];
            }
        n = next_n; sl = next_s; dir ^= 1; ++it;
    }
    // ---- the block's row of sums
    if (BWD) {
        __syncthreads();
        const size_t own = (size_t)blockIdx.x * 2 * p.ld;
        for (int e = t; e < 2 * p.ld; e += p.threads) {
            const int s = e >= p.ld, c = e - s * p.ld;
            const float v = it > kGnChain ? (float)(a.wide[own + e] + (double)acc[e]) : acc[e];
            if (gridDim.x > 1) a.rows[own + e] = v;
            else if (c < p.C) (s ? a.dgamma : a.dbeta)[c] = v;
        }
    }
}

// dgamma, dbeta: the blocks' rows. A block owns 32 columns; a warp adds every 32nd row of them, all loads before the first addition, then
// a column's 32 sums: a fixed order, chains of at most ten. (In 64 bits the backward pass of 64x14x14x931 from a checkpoint takes 43.7 us
// for 43.3.) Plain loads: the rows are still being written when this kernel starts, so they are not read-only for all of its life.
__global__ void __launch_bounds__(1024) gn_finish_kernel(const float *rows, int n, int C, int ld, float *dgamma, float *dbeta)
{
    __shared__ float part[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, e = blockIdx.x * 32 + lane;
    sm100::grid_dependency_wait();
    sm100::grid_launch_dependents();
    const float *src = rows + e;
    const size_t pitch = (size_t)2 * ld;
    float v = 0.f;
    for (int r0 = warp; r0 < n; r0 += 10 * 32) {                         // (296 rows are one round)
        float x[10];
#pragma unroll
        for (int i = 0; i < 10; ++i) x[i] = e < 2 * ld && r0 + 32 * i < n ? src[(r0 + 32 * i) * pitch] : 0.f;
#pragma unroll
        for (int i = 0; i < 10; ++i) v += x[i];
    }
    part[warp][lane] = v;
    __syncthreads();
    v = part[lane][warp];
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    const int f = blockIdx.x * 32 + warp, s = f >= ld, c = f - s * ld;
    if (lane == 0 && f < 2 * ld && c < C) (s ? dgamma : dbeta)[c] = v;
}

typedef void (*GnKernel)(GnP, GnArgs);

template <int MODE>
GnKernel gn_pick(int act, bool res)
{
    switch (act) {
    case PT_ACT_NONE: return res ? gn_kernel<MODE, PT_ACT_NONE, true> : gn_kernel<MODE, PT_ACT_NONE, false>;
    case PT_ACT_RELU: return res ? gn_kernel<MODE, PT_ACT_RELU, true> : gn_kernel<MODE, PT_ACT_RELU, false>;
    default: return res ? gn_kernel<MODE, PT_ACT_SILU, true> : gn_kernel<MODE, PT_ACT_SILU, false>;
    }
}

GnKernel gn_kernel_of(int mode, int act, bool res)
{
    switch (mode) {
    case kGnFwd: return gn_pick<kGnFwd>(act, res);
    case kGnFwdPack: return gn_pick<kGnFwdPack>(act, res);
    case kGnBwd: return gn_pick<kGnBwd>(act, res);
    default: return gn_pick<kGnBwdPacked>(act, res);
    }
}

pt_status gn_params(const pt_ctx *c, const pt_gn_desc *d, bool codes, GnP *p)
{
    if (!c || !d) return PT_ERR_INVALID_ARG;
    if (d->N < 1 || d->H < 1 || d->W < 1 || d->C < 1 || d->ld < d->C || (d->ld & 7)) return PT_ERR_INVALID_ARG;
    if (d->groups < 1 || d->groups > d->C || !(d->eps >= 0.f) || d->act < PT_ACT_NONE || d->act > PT_ACT_SILU) return PT_ERR_INVALID_ARG;
    if (codes && (d->ldq < d->C || (d->ldq & 7))) return PT_ERR_INVALID_ARG;
    memset(p, 0, sizeof(*p));
    const int32_t *b = d->group_begin;
    if (b) {
        if (b[0] != 0 || b[d->groups] != d->C) return PT_ERR_INVALID_ARG;
        for (int g = 0; g < d->groups; ++g) {
            if (b[g] < 0 || b[g + 1] <= b[g] || b[g + 1] > d->C) return PT_ERR_INVALID_ARG;
            if ((long long)b[g] * d->groups != (long long)g * d->C) p->table = 1;
        }
    } else if (d->C % d->groups) {
        return PT_ERR_INVALID_ARG;
    }
    if (d->N > kGnMaxN || d->ld > kGnMaxLd || (p->table && d->groups > kGnTable)) return PT_ERR_UNSUPPORTED;
    const long long hw = (long long)d->H * d->W;
    // (offsets in an image have 32 bits; first the pixels alone, so that the products have fewer than 64)
    if (hw >= 0x80000000ll || hw * d->ld * 2 >= 0x100000000ll || (codes && hw * d->ldq >= 0x100000000ll)) return PT_ERR_UNSUPPORTED;
    if (p->table)
        for (int g = 0; g <= d->groups; ++g) p->begin[g] = (uint16_t)b[g];
    p->N = d->N; p->HW = (int)hw; p->C = d->C; p->ld = d->ld; p->LV = d->ld / 8; p->ldq = d->ldq; p->nb = pt_ceil_div(d->C, act8::kBlock);
    p->G = d->groups; p->cg = d->C / d->groups; p->eps = d->eps;
    p->w = p->LV >= 3 ? 4 : p->LV;
    return PT_OK;
}

int gn_begin(const GnP &p, int g) { return p.table ? p.begin[g] : g * (p.C / p.G); }

// Cuts the channels into about `want` slabs of whole groups and whole vectors (whole blocks of 32 channels where there is a checkpoint).
void gn_slabs(GnP *p, int want, bool blocks)
{
    const int align = blocks ? act8::kBlock : 8;
    p->slabs = 1;
    p->gs = 0;
    int last = 0;
    const auto cut = [&](int v, int g) {
        p->slab_v[p->slabs] = (uint16_t)v; p->slab_g[p->slabs] = (uint16_t)g;
        p->gs = p->gs > g - last ? p->gs : g - last;
        last = g;
    };
    p->slab_v[0] = p->slab_g[0] = 0;
    for (int g = 1; g < p->G && p->slabs < want; ++g) {
        const int c = gn_begin(*p, g);
        // the first boundary at or behind the place of the next cut
        if (c % align == 0 && (long long)c * want >= (long long)p->slabs * p->C) { cut(c / 8, g); p->slabs += 1; }
    }
    cut(p->LV, p->G);
    p->rl = 0;
    for (int s = 0; s < p->slabs; ++s) {
        const int w = p->slab_v[s + 1] - p->slab_v[s];
        p->rl = p->rl > w ? p->rl : w;
    }
}

// The launch shape for clusters of cl blocks: how the threads cover a slab's pixels, and the shared memory's parts. Returns its bytes.
size_t gn_shape(GnP *p, int mode, bool res, int cl)
{
    p->cl = cl;
    p->share = pt_ceil_div(p->HW, cl);
    if (mode == kGnFwdPack) p->rl = pt_ceil_div(p->rl, p->w) * p->w;
    p->ppb = kGnThreads / p->rl;
    if (p->ppb > p->share) p->ppb = p->share;
    p->threads = (p->rl * p->ppb + 31) / 32 * 32;
    // lanes of a group: as many as there are for it; as many of them for its channels as it has
    int most = 1;
    for (int g = 0; g < p->G; g += p->table ? 1 : p->G) most = most > gn_begin(*p, g + 1) - gn_begin(*p, g) ? most : gn_begin(*p, g + 1) - gn_begin(*p, g);
    p->gl = p->gc = 0;
    while (p->gl < 5 && (2 << p->gl) * p->gs <= p->threads && (1 << p->gl) < most * p->ppb) p->gl += 1;
    while (p->gc < p->gl && (1 << p->gc) < most) p->gc += 1;
    size_t at = 0;
    const auto part = [&](unsigned *off, size_t bytes) { *off = (unsigned)at; at += pt_align_up(bytes, 16); };
    part(&p->sm_ring, (size_t)kGnThreads * gn_ring(mode, res));
    part(&p->sm_gid, (size_t)p->ld * 2);
    part(&p->sm_gam, (size_t)p->ld * 4);
    part(&p->sm_bet, (size_t)p->ld * 4);
    part(&p->sm_grp, (size_t)p->G * 6 * 4);
    part(&p->sm_red, (size_t)p->threads * gn_red(mode) * 4);
    part(&p->sm_xch, (size_t)(cl > 1 ? 2 : 1) * cl * p->gs * (gn_bwd(mode) ? 8 : 16));
    part(&p->sm_acc, gn_bwd(mode) ? (size_t)2 * p->ld * 4 : 0);
    return at;
}

bool aligned16(const void *q) { return ((uintptr_t)q & 15) == 0; }

struct GnPlan {
    GnP key, p;                  // what gn_params gave, and with the launch shape
    int mode;                    // the kernel's number
    size_t smem;
};
typedef std::unordered_multimap<uint64_t, GnPlan> GnPlans;

void gn_config(cudaLaunchConfig_t *cfg, cudaLaunchAttribute (&attr)[2], int clusters, int cl, int threads, size_t smem, cudaStream_t st)
{
    memset(cfg, 0, sizeof(*cfg));
    memset(attr, 0, sizeof(attr));
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cl; attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg->gridDim = dim3((unsigned)(clusters * cl)); cfg->blockDim = dim3((unsigned)threads); cfg->dynamicSmemBytes = smem; cfg->stream = st;
    cfg->attrs = attr;
    cfg->numAttrs = cl > 1 ? 2 : 1;
}

// Clusters of cl blocks that the device holds at once, with shared memory for two blocks on an SM or for one.
pt_status gn_fit(pt_ctx *c, GnKernel kernel, int index, int cl, bool two, int *n)
{
    int &known = c->gn_fit[index][cl][two ? 1 : 0];
    if (!known) {
        cudaLaunchConfig_t cfg;
        cudaLaunchAttribute attr[2];
        int m = 0;
        gn_config(&cfg, attr, 1, cl, kGnThreads, two ? kGnSmem : kGnSmemMost, nullptr);
        cfg.numAttrs = 2;
        PT_CUDA_OK(cudaOccupancyMaxActiveClusters(&m, (const void *)kernel, &cfg));
        known = m + 1;
    }
    *n = known - 1;
    return PT_OK;
}

// The slabs and the cluster size of the least estimated time. A unit of work costs a block about 4.5 us whatever it holds (loads, barriers,
// exchange, all in a row), so that one unit per block is best nearly everywhere, and `row` per row of its threads: 0.25 to 0.55 by direction
// and checkpoint, 0.1 more with a residual, 1.8 times that where two blocks share an SM (backward 64x56x56x256: 0.47 us a row alone, 0.85
// together). 1.25 for slabs of less than 64 bytes a pixel, 0.7 for a cluster's exchange and 1.0 for a second block's start are guesses that
// put close candidates in order, not measurements by themselves; bytes are not in it. Microseconds by clusters of 1, 2, 4, 8, 16 blocks:
// 180, 97, 87, 96, 116 for the backward pass at 64x56x56x256 with SiLU (taken: four slabs without clusters, 84), 47.4, 32.6, 27.8, 36.6, 53.8
// for the forward pass at 64x28x28x371 with a residual; 95, 51, 28, 17, 11 at 2x112x112x64 with SiLU, where four slabs and 9 blocks take
// 8.1. Of thirteen shapes swept this way it took the best, or within 1 %, for eight, and lost 4 to 13 % at the others: 64x56x56x256 with ReLU
// backward 79.0 (two slabs and 8 blocks 71.3), forward 48.0 (46.0); 2x112x112x64 9.0 (8.0); 128x32x32x16 forward and back from its checkpoint
// 21.1 (clusters of two 19.9); 8x16x16x27 4.7 (4.4).
pt_status gn_plan(pt_ctx *c, GnKernel kernel, int index, int mode, bool res, GnPlan *plan)
{
    const bool blocks = mode == kGnFwdPack || mode == kGnBwdPacked;
    const double row = (mode == kGnFwd ? 0.25 : mode == kGnFwdPack ? 0.4 : mode == kGnBwd ? 0.45 : 0.55) + (res ? 0.1 : 0.0);
    double best = 1e30;
    int last = 0;
    for (int want = 1; want <= kGnSlabs && want <= plan->key.G; ++want) {
        GnP q = plan->key;
        gn_slabs(&q, want, blocks);
        if (q.slabs == last) continue;
        last = q.slabs;
        if (q.slabs > 1 && q.rl < 2) break;                              // (a slab of 16 bytes a pixel would read every sector twice)
        for (int cl = 1; cl <= kGnMaxCluster; ++cl) {
            if (cl > 1 && (cl > q.HW || cl * q.gs > kGnExchange)) break;
            GnP r = q;
            const size_t smem = gn_shape(&r, mode, res, cl);
            if (smem > kGnSmemMost) continue;
            int n = 0;
            const pt_status s = gn_fit(c, kernel, index, cl, smem <= kGnSmem, &n);
            if (s != PT_OK) return s;
            if (n < 1) continue;
            const int most = (smem <= kGnSmem ? kGnBlocks : 1) * c->sm_count / cl, units = q.N * q.slabs;
            n = n < most ? n : most;
            r.clusters = n < units ? n : units;
            r.step_n = r.clusters / r.slabs; r.step_s = r.clusters % r.slabs;
            const bool shared = r.clusters * cl > c->sm_count;
            const double rows = (double)pt_ceil_div(r.share, r.ppb) * r.threads / kGnThreads, narrow = q.rl < 4 && q.slabs > 1 ? 1.25 : 1.0;
            const double us = pt_ceil_div(units, r.clusters) * (4.5 + rows * row * narrow * (shared ? 1.8 : 1.0)) + (cl > 1 ? 0.7 : 0.0) + (shared ? 1.0 : 0.0);
            if (us < best) { best = us; plan->p = r; plan->smem = smem; }
        }
    }
    return best < 1e30 ? PT_OK : PT_ERR_UNSUPPORTED;
}

// The plan of a shape: those met so far are kept, choosing one walks a few hundred candidates.
pt_status gn_plan_of(pt_ctx *c, GnKernel kernel, int index, int mode, bool res, const GnP &key, GnPlan *plan)
{
    uint64_t h = (uint64_t)index, w;
    for (size_t k = 0; k + 8 <= sizeof(GnP); k += 8) {
        memcpy(&w, reinterpret_cast<const char *>(&key) + k, 8);
        h = (h ^ w) * 0x9e3779b97f4a7c15ull;
        h ^= h >> 29;
    }
    std::lock_guard<std::mutex> lock(c->gn_mutex);
    GnPlans *known = static_cast<GnPlans *>(c->gn_plans.get());
    if (known) {
        const auto range = known->equal_range(h);
        for (auto it = range.first; it != range.second; ++it)
            if (it->second.mode == index && memcmp(&it->second.key, &key, sizeof(GnP)) == 0) {
                *plan = it->second;
                return PT_OK;
            }
    }
    memset(plan, 0, sizeof(*plan));
    memcpy(&plan->key, &key, sizeof(GnP));
    plan->mode = index;
    const pt_status r = gn_plan(c, kernel, index, mode, res, plan);
    if (r != PT_OK) return r;
    try {
        if (!known) {
            c->gn_plans = std::make_shared<GnPlans>();
            known = static_cast<GnPlans *>(c->gn_plans.get());
        }
        if (known->size() >= pt_ctx::kGnPlans) known->clear();
        known->emplace(h, *plan);
    } catch (const std::bad_alloc &) {                           // (no room: the plan is chosen again next time)
    }
    return PT_OK;
}

pt_status launch_gn(pt_ctx *c, const GnP &key, const GnArgs &a, int mode, int act, cudaStream_t st)
{
    const bool res = a.res != nullptr;
    const GnKernel kernel = gn_kernel_of(mode, act, res);
    const int index = (mode * 3 + act) * 2 + (res ? 1 : 0);
    if (!(c->gn_attr_done & (1u << index))) {
        PT_CUDA_OK(cudaFuncSetAttribute((const void *)kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kGnSmemMost));
        PT_CUDA_OK(cudaFuncSetAttribute((const void *)kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
        c->gn_attr_done |= 1u << index;
    }
    GnPlan plan;
    const pt_status r = gn_plan_of(c, kernel, index, mode, res, key, &plan);
    if (r != PT_OK) return r;
    const GnP &p = plan.p;
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[2];
    gn_config(&cfg, attr, p.clusters, p.cl, p.threads, plan.smem, st);
    PT_CUDA_OK(cudaLaunchKernelEx(&cfg, kernel, p, a));
    c->launches += 1;
    if (mode >= kGnBwd && p.clusters * p.cl > 1) {
        PT_CUDA_OK(pt_launch_pdl(gn_finish_kernel, dim3((unsigned)pt_ceil_div(2 * p.ld, 32)), dim3(1024), 0, st, (const float *)a.rows, p.clusters * p.cl, p.C,
                                 p.ld, a.dgamma, a.dbeta));
        c->launches += 1;
    }
    return PT_OK;
}

// Sums of dz and dz * xhat in the workspace: a row per block.
size_t gn_sums(const pt_ctx *c, const GnP &p) { return (size_t)c->sm_count * kGnBlocks * 2 * p.ld; }

}  // namespace

extern "C" size_t pt_gn_workspace_bytes(const pt_ctx *c, const pt_gn_desc *d)
{
    GnP p;
    if (gn_params(c, d, false, &p) != PT_OK) return 0;
    return gn_sums(c, p) * (sizeof(double) + sizeof(float));
}

extern "C" pt_status pt_gn_act_fwd(pt_ctx *c, const pt_gn_desc *d, const void *x, const void *residual, const float *gamma, const float *beta,
                                   float *save_mean, float *save_rstd, void *y, void *codes, void *scales, void *stream)
{
    GnP p;
    pt_status r = gn_params(c, d, codes != nullptr, &p);
    if (r != PT_OK) return r;
    if (!pt_on_device(c) || !x || !gamma || !beta || !save_mean || !save_rstd || !y || (codes == nullptr) != (scales == nullptr)) return PT_ERR_INVALID_ARG;
    if (!aligned16(x) || !aligned16(residual) || !aligned16(y) || !aligned16(codes) || !aligned16(scales)) return PT_ERR_INVALID_ARG;
    GnArgs a{};
    a.x = (const uint4 *)x; a.res = (const uint4 *)residual; a.gamma = gamma; a.beta = beta; a.save_mean = save_mean; a.save_rstd = save_rstd;
    a.y = (uint4 *)y; a.codes = (uint8_t *)codes; a.scales = (uint8_t *)scales;
    return launch_gn(c, p, a, codes ? kGnFwdPack : kGnFwd, d->act, (cudaStream_t)stream);
}

extern "C" pt_status pt_gn_act_bwd(pt_ctx *c, const pt_gn_desc *d, const void *x, const void *residual, const void *dy, const float *gamma,
                                   const float *beta, const float *save_mean, const float *save_rstd, void *dx, void *dresidual, float *dgamma,
                                   float *dbeta, void *ws, size_t ws_bytes, void *stream)
{
    GnP p;
    pt_status r = gn_params(c, d, false, &p);
    if (r != PT_OK) return r;
    if (!pt_on_device(c) || !x || !dy || !gamma || !beta || !save_mean || !save_rstd || !dx || !dgamma || !dbeta) return PT_ERR_INVALID_ARG;
    if (!aligned16(x) || !aligned16(residual) || !aligned16(dy) || !aligned16(dx) || !aligned16(dresidual)) return PT_ERR_INVALID_ARG;
    if (!ws || !aligned16(ws) || ws_bytes < pt_gn_workspace_bytes(c, d)) return PT_ERR_WORKSPACE;
    GnArgs a{};
    a.x = (const uint4 *)x; a.res = (const uint4 *)residual; a.dy = (const uint4 *)dy; a.gamma = gamma; a.beta = beta; a.mean = save_mean;
    a.rstd = save_rstd; a.dx = (uint4 *)dx; a.dres = (uint4 *)dresidual;
    a.wide = (double *)ws; a.rows = (float *)(a.wide + gn_sums(c, p)); a.dgamma = dgamma; a.dbeta = dbeta;
    return launch_gn(c, p, a, kGnBwd, d->act, (cudaStream_t)stream);
}

extern "C" pt_status pt_gn_act_bwd_packed(pt_ctx *c, const pt_gn_desc *d, const void *codes, const void *scales, const void *residual,
                                          const void *dy, const float *gamma, const float *beta, const float *save_mean, const float *save_rstd,
                                          void *dx, void *dresidual, float *dgamma, float *dbeta, void *y, void *ws, size_t ws_bytes, void *stream)
{
    GnP p;
    pt_status r = gn_params(c, d, true, &p);
    if (r != PT_OK) return r;
    if (!pt_on_device(c) || !codes || !scales || !dy || !gamma || !beta || !save_mean || !save_rstd || !dx || !dgamma || !dbeta) return PT_ERR_INVALID_ARG;
    if (!aligned16(codes) || !aligned16(scales) || !aligned16(residual) || !aligned16(dy) || !aligned16(dx) || !aligned16(dresidual) || !aligned16(y))
        return PT_ERR_INVALID_ARG;
    if (!ws || !aligned16(ws) || ws_bytes < pt_gn_workspace_bytes(c, d)) return PT_ERR_WORKSPACE;
    GnArgs a{};
    a.codes_in = (const uint8_t *)codes; a.scales_in = (const uint8_t *)scales; a.res = (const uint4 *)residual; a.dy = (const uint4 *)dy;
    a.gamma = gamma; a.beta = beta; a.mean = save_mean; a.rstd = save_rstd; a.dx = (uint4 *)dx; a.dres = (uint4 *)dresidual; a.y = (uint4 *)y;
    a.wide = (double *)ws; a.rows = (float *)(a.wide + gn_sums(c, p)); a.dgamma = dgamma; a.dbeta = dbeta;
    return launch_gn(c, p, a, kGnBwdPacked, d->act, (cudaStream_t)stream);
}
