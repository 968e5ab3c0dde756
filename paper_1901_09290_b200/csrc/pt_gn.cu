// Group normalisation + residual add + activation on ragged channel counts and groups, channels last, forward and backward. NHWC bf16
// activations with channel pitch ld, fp32 statistics and parameters. Per image n and group g of m = H*W*|g| values:
//   forward : mean, rstd = 1/sqrt(var + eps), z = gamma*(x - mean)*rstd + beta (+ residual), y = act(z)
//   backward: dz = dy*act'(z), A = sum gamma*dz, B = sum gamma*dz*xhat, dx = rstd*(gamma*dz - A/m - xhat*B/m)
// Both directions need an image's sums before its first result, and are bound by HBM: the aim is to read an image once.
//
// A thread-block cluster owns an image; each of its blocks owns a run of consecutive pixels, and a thread of a block a 16-byte vector
// column and every so many-th pixel. Threads bring in what they will use themselves, by asynchronous copies into places of their own in
// shared memory, a ring of batches of two pixels: there is nobody to wait for but one's own copies. A thread walks its pixels forwards for
// the sums; the blocks of the cluster exchange the groups' sums through distributed shared memory; and it walks the pixels BACKWARDS for
// the results: the last batches of the first walk are still in the ring, all of them where the image fits the cluster, and the others
// were read recently enough to be in L2. Batches that the second walk is done with make room for the next image of the cluster.
// No atomics: sums in a fixed order (run-to-run identical).
//   (The first form had a producer warp and bulk copies of whole chunks of pixels. One thread issues such a copy every 0.3 to 0.5 us, which
// with two or three tensors was the bound: 150 to 260 us for the backward pass at 64x28x28x371 with a residual, by the chunk's size.)
#include "pt_internal.h"
#include "pt_act.cuh"
#include "pt_sm100_ptx.cuh"

namespace {

constexpr int kGnThreads = 256;              // most consumer threads of a block (a producer warp follows them)
constexpr int kGnTable = 256;                // most groups of a table
constexpr int kGnMaxLd = 2048;
constexpr int kGnMaxCluster = 16;
constexpr int kGnExchange = 512;             // most entries (blocks of the cluster x groups) of one exchange buffer
constexpr int kGnRows = 2;                   // pixels of a thread's batch

enum { kGnFwd = 0, kGnFwdPack = 1, kGnBwd = 2, kGnBwdPacked = 3 };

__host__ __device__ constexpr bool gn_bwd(int mode) { return mode >= kGnBwd; }
// Bytes of a thread's place for one pixel: the vectors of x (or codes and the word that holds the scale byte), dy and the residual.
__host__ __device__ constexpr int gn_slot(int mode, bool res) { return (mode == kGnBwdPacked ? 12 : 16) + (gn_bwd(mode) ? 16 : 0) + (gn_bwd(mode) && res ? 16 : 0); }
// Batches of a thread's ring: what two blocks to an SM have room for.
__host__ __device__ constexpr int gn_batches(int mode, bool res) { return 280 / (kGnRows * gn_slot(mode, res)); }
constexpr int kGnBlocks = 2;                 // blocks of an SM: while one exchanges its sums, the other one moves data

struct GnP {
    int N, HW, C, ld, LV, ldq, nb, G;
    int w, rl, ppb, threads;     // lanes of a checkpoint's block, lanes of a pixel, pixels the threads cover at a time, threads
    int gl, gc;                  // lanes that add up a group, and those of them that take different channels
    int cl, clusters, share;     // blocks of a cluster, clusters, pixels of a block
    int table;
    unsigned sm_gid, sm_gam, sm_bet, sm_grp, sm_red, sm_xch, sm_acc, sm_ring;
    float eps;
    uint16_t begin[kGnTable + 1];
};

struct GnArgs {
    const uint4 *x, *res, *dy;
    const uint8_t *codes_in, *scales_in;
    const float *gamma, *beta, *mean, *rstd;
    float *save_mean, *save_rstd;
    uint4 *y, *dx, *dres;
    uint8_t *codes, *scales;
    double *rows;                // backward: [clusters][2][ld] sums of dz and dz * xhat over a cluster's images
    float *dgamma, *dbeta;
};

__device__ __forceinline__ int group_begin(const GnP &p, int g) { return p.table ? p.begin[g] : g * (p.C / p.G); }

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

__device__ __forceinline__ float ex2(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ float rcp(float x) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }

// SiLU works on w = -z * log2(e), which costs nothing: the factor is in the constants that give z. sigmoid(z) = 1/(1 + 2^w), 2 ulp and
// |z| * 2^-24 off. One reciprocal serves a pair, 1/a = b/(a*b): the special-function units take 8 cycles for an instruction of a warp, and
// with two exponentials and two reciprocals per pair, twice in the backward pass, they were the bound at 64x56x56x256 (46 us of their time
// alone; 35 with one reciprocal). 2^w stops at 2^60, a sigmoid of 1e-18, so that a*b is finite. (A NaN does not come through: the
// result is only ever multiplied by w.)
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
__device__ __forceinline__ f2 sigmoid_w(f2 w)
{
    float a, b;
    un2(w, a, b);
    un2(add2(mk2(ex2(fminf(a, 60.f)), ex2(fminf(b, 60.f))), mk2(1.f, 1.f)), a, b);
    const float r = rcp(a * b);
    return mk2(r * b, r * a);
}

template <int ACT>
__device__ __forceinline__ f2 activate2(f2 z)
{
    if (ACT == PT_ACT_NONE) return z;
    if (ACT == PT_ACT_SILU) return mul2(mul2(z, mk2(-kLn2, -kLn2)), sigmoid_w(z));       // (of w)
    float a, b;
    un2(z, a, b);
    return mk2(a > 0.f ? a : (a != a ? a : 0.f), b > 0.f ? b : (b != b ? b : 0.f));
}

// Two fp64 values into the shared memory of another block of the cluster, visible there behind the cluster's barrier.
__device__ __forceinline__ void st_cluster_2d(uint32_t addr, double a, double b)
{
    asm volatile("st.shared::cluster.v2.f64 [%0], {%1, %2};" ::"r"(addr), "d"(a), "d"(b) : "memory");
}
__device__ __forceinline__ double ld_cluster_d(uint32_t addr)
{
    double v;
    asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(addr) : "memory");
    return v;
}
// Asynchronous copies of a thread, in groups; waiting for all but the last `PENDING` groups.
__device__ __forceinline__ void copy16(uint32_t dst, const void *src) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void copy8(uint32_t dst, const void *src) { asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void copy4(uint32_t dst, const void *src) { asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int PENDING>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(PENDING) : "memory"); }

// The largest bf16 <= v (its bits): x > v exactly where x > that, for every bf16 x.
__device__ __forceinline__ uint32_t bf16_floor(double v)
{
    const uint32_t u = __float_as_uint(__double2float_rd(v));
    if ((u & 0x7fffffffu) > 0x7f800000u) return 0x7fc0u;                 // NaN: no x is above it
    return (u >> 31) ? ((u + 0xffffu) >> 16) : (u >> 16);                // (towards -inf: a negative one's magnitude rounds up)
}

// Which of two neighbouring values (bf16 halves of x) have z = gamma*xhat + beta + residual > 0, in 64 bits. Rarely called: fp32 decides
// everywhere but next to 0.
__device__ __noinline__ uint32_t exact_mask(uint32_t x, uint32_t r, int c, const uint16_t *gid, const float *grp, int G, const float *gam, const float *bet)
{
    uint32_t m = 0u;
    for (int h = 0; h < 2; ++h) {
        const int g = gid[c + h];
        const double xv = (double)__uint_as_float(h ? x & 0xffff0000u : x << 16), rv = (double)__uint_as_float(h ? r & 0xffff0000u : r << 16);
        if ((xv - (double)grp[g]) * (double)grp[G + g] * (double)gam[c + h] + (double)bet[c + h] + rv > 0.0) m |= h ? 0xffff0000u : 0xffffu;
    }
    return m;
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
    constexpr int B = gn_batches(MODE, RES), U = kGnRows;
    // the ring's parts, [B][U][threads] each: x or codes, dy, residual, scale words
    constexpr uint32_t kXs = PACKED ? 8 : 16, kRowX = kGnThreads * kXs, kRow = kGnThreads * 16, kRowS = kGnThreads * 4;
    constexpr uint32_t kDy = B * U * kRowX, kRes = kDy + (BWD ? B * U * kRow : 0), kSc = kRes + (BWD && RES ? B * U * kRow : 0);
    extern __shared__ __align__(128) uint8_t smem[];
    uint16_t *gid = reinterpret_cast<uint16_t *>(smem + p.sm_gid);       // [ld] group of a channel
    float *gam = reinterpret_cast<float *>(smem + p.sm_gam), *bet = reinterpret_cast<float *>(smem + p.sm_bet);      // [ld]
    float *grps = reinterpret_cast<float *>(smem + p.sm_grp);            // [2][2][G] of alternating images: mean and rstd (backward), pivot
    float *out = grps + 4 * p.G;                                         // [2][G] rstd and mean (forward), the group's terms of dx (backward)
    float *red = reinterpret_cast<float *>(smem + p.sm_red);             // [threads][17]
    double2 *xch = reinterpret_cast<double2 *>(smem + p.sm_xch);         // [2][cl][G]
    double *acc = reinterpret_cast<double *>(smem + p.sm_acc);           // [2][ld]
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31, warps = p.threads >> 5;
    const int rank = (int)(blockIdx.x % p.cl), cluster = (int)(blockIdx.x / p.cl);
    const int first = rank * p.share, mine = p.HW - first < p.share ? (p.HW - first > 0 ? p.HW - first : 0) : p.share;
    const int step = U * p.ppb, NB = (mine + step - 1) / step;           // pixels and number of the block's batches
    // Threads without a vector of their own (t >= rl * ppb, or lanes that only fill up a checkpoint's block) do what thread 0 does and store
    // nothing. Vectors of pad lanes only are read and come out as zeros; their codes, which there are none of, are read as vector 0's.
    int pr = t / p.rl, cv = t - pr * p.rl;
    const bool lane_ok = pr < p.ppb && cv < p.LV;
    if (!lane_ok) pr = cv = 0;
    const int c0 = cv * 8;
    const bool has = c0 < p.C;                                           // the vector holds channels, not pad lanes only
    const uint4 keep = act8::keep_bits(c0, p.C);
    const uint8_t *mine_x = smem + p.sm_ring + t * kXs, *mine_v = smem + p.sm_ring + t * 16, *mine_s = smem + p.sm_ring + kSc + t * 4;
    const uint32_t to_x = sm100::smem_u32(mine_x), to_v = sm100::smem_u32(mine_v), to_s = sm100::smem_u32(mine_s);
    for (int g = t; g < p.G; g += p.threads)
        for (int c = group_begin(p, g), e = group_begin(p, g + 1); c < e; ++c) gid[c] = (uint16_t)g;
    for (int c = p.C + t; c < p.ld; c += p.threads) gid[c] = (uint16_t)(p.G - 1);
    sm100::grid_dependency_wait();
    sm100::grid_launch_dependents();
    // Offsets in bytes from an image's first pixel of this block: 32 bits, added to addresses that all threads share.
    const uint32_t row = (uint32_t)p.ld * 2u, step_v = (uint32_t)step * row, step_q = (uint32_t)(step * p.ldq), step_s = (uint32_t)(step * p.nb);
    uint32_t off[U], off_q[U], off_s[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t r = (uint32_t)(pr + u * p.ppb);
        off[u] = r * row + (uint32_t)cv * 16u;
        off_q[u] = r * (uint32_t)p.ldq + (has ? (uint32_t)c0 : 0u);
        off_s[u] = r * (uint32_t)p.nb + (has ? (uint32_t)(cv >> 2) : 0u);
    }
    const auto bytes = [](const void *q) { return reinterpret_cast<const uint8_t *>(q); };
    struct Src { const uint8_t *x, *dy, *res, *q, *s; };                 // an image's tensors from the block's first pixel on
    const auto source = [&](int n) {
        Src g{};
        const size_t pix = (size_t)n * p.HW + first;
        if (PACKED) { g.q = a.codes_in + pix * p.ldq; g.s = a.scales_in + pix * p.nb; }
        else g.x = bytes(a.x) + pix * row;
        if (BWD) g.dy = bytes(a.dy) + pix * row;
        if (RES) g.res = bytes(a.res) + pix * row;
        return g;
    };
    // batch b of an image into the ring's place s (a multiple of U)
    const auto bring = [&](const Src &g, int b, int s) {
        const uint32_t bv = (uint32_t)b * step_v, bq = (uint32_t)b * step_q, bs = (uint32_t)b * step_s;
        const auto one = [&](int u) {
            if (PACKED) {
                copy8(to_x + (uint32_t)(s + u) * kRowX, g.q + (bq + off_q[u]));
                copy4(to_s + (uint32_t)(s + u) * kRowS, reinterpret_cast<const void *>(reinterpret_cast<uintptr_t>(g.s + (bs + off_s[u])) & ~(uintptr_t)3));
            } else {
                copy16(to_x + (uint32_t)(s + u) * kRowX, g.x + (bv + off[u]));
            }
            if (BWD) copy16(to_v + kDy + (uint32_t)(s + u) * kRow, g.dy + (bv + off[u]));
            if (BWD && RES) copy16(to_v + kRes + (uint32_t)(s + u) * kRow, g.res + (bv + off[u]));
        };
        if ((b + 1) * step <= mine) {
#pragma unroll
            for (int u = 0; u < U; ++u) one(u);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (b * step + u * p.ppb + pr < mine) one(u);
        }
    };
    // (these loads first: behind the ring's copies they would wait for those)
    const bool ahead = BWD && p.G <= p.threads;                          // an image's statistics are fetched before they are needed
    float next_mean = 0.f, next_rstd = 0.f;
    if (ahead && t < p.G) {
        next_mean = a.mean[(size_t)cluster * p.G + t];
        next_rstd = a.rstd[(size_t)cluster * p.G + t];
    }
    for (int c = t; c < p.ld; c += p.threads) {
        gam[c] = c < p.C ? a.gamma[c] : 0.f;
        bet[c] = c < p.C ? a.beta[c] : 1.f;                              // (a pad lane's z must not be near 0, see gradient)
        if (BWD) acc[c] = acc[p.ld + c] = 0.0;
    }
    Src src = source(cluster);
#pragma unroll 1
    for (int b = 0; b < B; ++b) {
        if (b < NB) bring(src, b, b * U);
        copy_commit();
    }
    int dir = 0, it = 0;
    const double inv_hw = 1.0 / (double)p.HW;
    const int whole = p.HW / p.share;                                    // blocks with all their pixels
    const double rest = (double)(p.HW - whole * p.share);                // pixels of the one behind them
    for (int n = cluster; n < p.N; n += p.clusters, dir ^= 1, ++it) {
        const size_t base = (size_t)n * p.HW + first;                    // the block's first pixel
        const Src next = source(n + p.clusters < p.N ? n + p.clusters : n);
        // (so that a batch of the first walk always has B - 1 groups behind it when it is waited for)
        if (it > 0)
            for (int b = NB; b < B; ++b) copy_commit();
        // ---- what the first walk needs of every group: the statistics (backward), or a value near its mean (forward)
        float *grp = grps + (it & 1) * 2 * p.G;
        if (BWD && ahead) {
            if (t < p.G) { grp[t] = next_mean; grp[p.G + t] = next_rstd; }
        } else if (BWD) {
            for (int g = t; g < p.G; g += p.threads) {
                grp[g] = a.mean[(size_t)n * p.G + g];
                grp[p.G + g] = a.rstd[(size_t)n * p.G + g];
            }
        } else {
            copy_wait<B - 1>();
            __syncthreads();
            // the average over the group's channels of the block's first pixels: as near the mean as a few values tell
            const int rows = min(min(4, p.ppb), mine), per = 32 / p.gl, l = lane & (p.gl - 1);
            const uint8_t *px = smem + p.sm_ring + (dir ? (B - 1) * U * kRowX : 0u);
            for (int g0 = warp * per; g0 < p.G; g0 += warps * per) {
                const int g = g0 + lane / p.gl;
                const int b = g < p.G ? group_begin(p, g) : 0, e = g < p.G ? group_begin(p, g + 1) : 0;
                float v = 0.f;
                for (int c = b + l; c < e; c += p.gl)
                    for (int r = 0; r < rows; ++r)
                        v += __bfloat162float(*reinterpret_cast<const __nv_bfloat16 *>(px + (size_t)(r * p.rl + (c >> 3)) * 16 + (c & 7) * 2));
                for (int o = p.gl >> 1; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
                if (l == 0 && g < p.G) grp[g] = rows > 0 ? v / (float)(rows * (e - b)) : 0.f;
            }
        }
        __syncthreads();
        // the thread's constants: minus the mean (or pivot), and in the backward pass gamma*rstd, beta, and the ReLU's limits as bf16: without
        // a residual, z > 0 exactly where x ^ sgn > thr
        f2 nm[4], k[4], kz[4], be[4];                                    // (kz: k, or for SiLU what gives w)
        uint32_t thr[4], sgn[4];
        float be_max = 1e-30f;                                           // (z so small that bf16 might not hold it is decided there too)
        {
            float m[8], kk[8], b[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int c = c0 + j, g = gid[c];
                m[j] = -grp[g];
                if (BWD) {
                    kk[j] = gam[c] * grp[p.G + g];
                    b[j] = bet[c];
                    be_max = fmaxf(be_max, 1e-6f * fabsf(b[j]));
                    if (ACT == PT_ACT_SILU) b[j] *= -kLog2e;
                }
                if (BWD && ACT == PT_ACT_RELU && !RES) {
                    // z = s*(x - mean) + beta > 0  <=>  x > mean - beta/s (s > 0), -x > -(mean - beta/s) (s < 0); a constant for s = 0
                    const double s = (double)gam[c] * (double)grp[p.G + g], bj = (double)bet[c];
                    const double lim = s == 0.0 ? (bj > 0.0 ? -INFINITY : INFINITY) : (double)grp[g] - bj / s;
                    const uint32_t th = bf16_floor(s < 0.0 ? -lim : lim), sg = s < 0.0 ? 0x8000u : 0u;
                    thr[j >> 1] = j & 1 ? thr[j >> 1] | th << 16 : th;
                    sgn[j >> 1] = j & 1 ? sgn[j >> 1] | sg << 16 : sg;
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                nm[i] = mk2(m[2 * i], m[2 * i + 1]);
                if (BWD) {
                    k[i] = mk2(kk[2 * i], kk[2 * i + 1]);
                    kz[i] = ACT == PT_ACT_SILU ? mul2(k[i], mk2(-kLog2e, -kLog2e)) : k[i];
                    be[i] = mk2(b[2 * i], b[2 * i + 1]);
                }
            }
        }
        // pixel u of a batch, at the ring's place s; bs: the batch's offset in the scales
        const uint32_t s_base = PACKED ? (uint32_t)(base * p.nb) : 0u;   // (the buffer starts on a word)
        const auto fetch = [&](Raw &w, uint32_t bs, int s, int u) {
            if (PACKED) {
                w.q = *reinterpret_cast<const uint2 *>(mine_x + (uint32_t)(s + u) * kRowX);
                const uint32_t sc = s_base + bs + off_s[u];
                w.byte = *reinterpret_cast<const uint32_t *>(mine_s + (uint32_t)(s + u) * kRowS) >> ((sc & 3u) * 8u) & 0xffu;
            } else {
                w.x = *reinterpret_cast<const uint4 *>(mine_x + (uint32_t)(s + u) * kRowX);
            }
            if (BWD) w.dy = *reinterpret_cast<const uint4 *>(mine_v + kDy + (uint32_t)(s + u) * kRow);
            if (BWD && RES) w.res = *reinterpret_cast<const uint4 *>(mine_v + kRes + (uint32_t)(s + u) * kRow);
        };
        const auto values = [&](Raw &w, f2 (&x)[4]) {                   // x as fp32 pairs (and, from codes, as bf16 words)
            if (PACKED) {
                decode8(w.q, w.byte, x);
                if (ACT == PT_ACT_RELU) w.x = make_uint4(exact_bf(x[0]), exact_bf(x[1]), exact_bf(x[2]), exact_bf(x[3]));
            } else {
                x[0] = from_bf(w.x.x); x[1] = from_bf(w.x.y); x[2] = from_bf(w.x.z); x[3] = from_bf(w.x.w);
            }
        };
        // dz: in place of dy's words where it is dy's bits under a mask, and as pairs. d = x - mean.
        const auto gradient = [&](Raw &w, const f2 (&d)[4], f2 (&z)[4], f2 (&dz)[4], bool want_z) {
            uint32_t *g = reinterpret_cast<uint32_t *>(&w.dy);
            const uint32_t *xb = reinterpret_cast<const uint32_t *>(&w.x), *rb = reinterpret_cast<const uint32_t *>(&w.res);
            if (ACT == PT_ACT_SILU || want_z || (ACT == PT_ACT_RELU && RES))
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    z[i] = fma2(d[i], kz[i], be[i]);
                    if (RES) z[i] = ACT == PT_ACT_SILU ? fma2(from_bf(rb[i]), mk2(-kLog2e, -kLog2e), z[i]) : add2(z[i], from_bf(rb[i]));
                }
            if (ACT == PT_ACT_RELU && !RES) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t u = xb[i] ^ sgn[i];
                    g[i] &= __hgt2_mask(*reinterpret_cast<const __nv_bfloat162 *>(&u), *reinterpret_cast<const __nv_bfloat162 *>(&thr[i]));
                }
            }
            if (ACT == PT_ACT_RELU && RES) {
                // Where z is near 0, fp32 leaves it wrong by less than 2^-22 of |beta| + |residual|: there 64 bits decide. One test for the
                // eight values, the least |z| against the largest |residual|: it is passed a few times in a hundred thousand.
                float zz[8], low = INFINITY;
                uint32_t top = 0u;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    un2(z[i], zz[2 * i], zz[2 * i + 1]);
                    low = fminf(low, fminf(fabsf(zz[2 * i]), fabsf(zz[2 * i + 1])));
                    top = __vmaxu2(top, rb[i] & 0x7fff7fffu);
                }
                const float rmax = fmaxf(__uint_as_float(top << 16), __uint_as_float(top & 0xffff0000u));
                if (low <= fmaf(rmax, 1e-6f, be_max)) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        // (gamma = 0, a pruned channel's or a pad lane's: z = beta + residual, of the right sign in fp32)
                        float k0, k1, b0, b1;
                        un2(k[i], k0, k1);
                        un2(be[i], b0, b1);
                        const bool near0 = k0 != 0.f && fabsf(zz[2 * i]) <= 1e-6f * (fabsf(__uint_as_float(rb[i] << 16)) + fabsf(b0));
                        const bool near1 = k1 != 0.f && fabsf(zz[2 * i + 1]) <= 1e-6f * (fabsf(__uint_as_float(rb[i] & 0xffff0000u)) + fabsf(b1));
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
                if (ACT == PT_ACT_SILU) {                                // act' = s + z*s*(1 - s) = s * (1 + w * ln 2 * (s - 1))
                    const f2 s = sigmoid_w(z[i]);
                    dz[i] = mul2(mul2(dz[i], s), fma2(z[i], fma2(s, mk2(kLn2, kLn2), mk2(-kLn2, -kLn2)), mk2(1.f, 1.f)));
                }
            }
        };

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
        // a thread's chains of additions stay short: every 64 rows they go to its place in shared memory
        bool flushed = false;
        const auto flush = [&]() {
            float *o = red + t * 17;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float u[4];
                un2(s0[i], u[0], u[1]);
                un2(s1[i], u[2], u[3]);
                o[2 * i] = flushed ? o[2 * i] + u[0] : u[0];
                o[2 * i + 1] = flushed ? o[2 * i + 1] + u[1] : u[1];
                o[8 + 2 * i] = flushed ? o[8 + 2 * i] + u[2] : u[2];
                o[9 + 2 * i] = flushed ? o[9 + 2 * i] + u[3] : u[3];
                s0[i] = s1[i] = mk2(0.f, 0.f);
            }
            flushed = true;
        };
        // the ring's places in the order of the walk, and where they begin and end
        const int s_first = dir ? (B - 1) * U : 0, s_last = dir ? 0 : (B - 1) * U, s_step = dir ? -U : U;
        int s = s_first;
        for (int b = 0; b < NB; ++b) {
            copy_wait<B - 1>();
            const int left = mine - b * step - pr;                       // pixel u is there if u * ppb < left
            const uint32_t bs = (uint32_t)b * step_s;
            if (PACK) {                                                  // (whole warps: the lanes of a checkpoint's block exchange)
                uint8_t *gq = a.codes + base * p.ldq, *gs = a.scales + base * p.nb;
                const uint32_t bq = (uint32_t)b * step_q;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const bool ok = u * p.ppb < left;
                    Raw w;
                    w.x = make_uint4(0u, 0u, 0u, 0u);
                    if (ok) {
                        fetch(w, bs, s, u);
                        count(w);
                    }
                    w.x = act8::and4(w.x, keep);
                    if (!lane_ok) w.x = make_uint4(0u, 0u, 0u, 0u);
                    const uint32_t byte = act8::scale_byte(act8::block_max(act8::amax8(w.x), p.w));
                    if (ok && lane_ok && has) {
                        *reinterpret_cast<uint2 *>(gq + (bq + off_q[u])) = act8::encode8(w.x, byte);
                        if ((cv & 3) == 0) gs[bs + off_s[u]] = (uint8_t)byte;
                    }
                }
            } else if ((b + 1) * step <= mine) {                         // two pixels at a time, their loads first
                Raw w[U];
#pragma unroll
                for (int u = 0; u < U; ++u) fetch(w[u], bs, s, u);
#pragma unroll
                for (int u = 0; u < U; ++u) count(w[u]);
            } else {
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (u * p.ppb < left) {
                        Raw w;
                        fetch(w, bs, s, u);
                        count(w);
                    }
            }
            if (b + B < NB) bring(src, b + B, s);                        // (the last B batches stay for the second walk)
            copy_commit();
            if ((b & 31) == 31 || b == NB - 1) flush();
            s = s == s_last ? s_first : s + s_step;
        }
        if (NB == 0) flush();
        // ---- a group's sums over the threads' rows and its channels
        __syncthreads();
        {
            // a group's lanes: gc of them take its channels, the others more of the threads' rows
            const int per = 32 / p.gl, l = lane & (p.gl - 1), lc = l & (p.gc - 1), lr = l / p.gc, nr = p.gl / p.gc, buf = it & 1;
            for (int g0 = warp * per; g0 < p.G; g0 += warps * per) {
                const int g = g0 + lane / p.gl;
                const int b = g < p.G ? group_begin(p, g) : 0, e = g < p.G ? group_begin(p, g + 1) : 0;
                float f0 = 0.f, f1 = 0.f;
                for (int c = b + lc; c < e; c += p.gc) {
                    const float *src = red + (lr * p.rl + (c >> 3)) * 17 + (c & 7);
                    float w0 = 0.f, w1 = 0.f;
#pragma unroll 4
                    for (int r = lr; r < p.ppb; r += nr, src += nr * p.rl * 17) { w0 += src[0]; w1 += src[8]; }
                    const float f = BWD ? gam[c] : 1.f;
                    f0 = fmaf(f, w0, f0);
                    f1 = fmaf(f, w1, f1);
                }
                for (int o = p.gl >> 1; o; o >>= 1) {
                    f0 += __shfl_xor_sync(0xffffffffu, f0, o);
                    f1 += __shfl_xor_sync(0xffffffffu, f1, o);
                }
                double v0 = (double)f0, v1 = (double)f1;
                if (!BWD) {                                              // the block's mean and sum of squares about it
                    const double cnt = (double)mine * (double)(e - b), d = cnt > 0.0 ? v0 / cnt : 0.0;
                    v1 = v1 - v0 * d;
                    v0 = g < p.G && mine > 0 ? (double)grp[g] + d : 0.0;
                    if (v1 < 0.0) v1 = 0.0;
                }
                if (g < p.G)
                    for (int r = l; r < p.cl; r += p.gl) {
                        double2 *to = xch + ((size_t)buf * p.cl + rank) * p.G + g;
                        if (p.cl == 1) *to = make_double2(v0, v1);
                        else st_cluster_2d(sm100::map_to_rank(sm100::smem_u32(to), (uint32_t)r), v0, v1);
                    }
            }
            if (p.cl > 1) sm100::cluster_barrier();
            else __syncthreads();
            // ---- the image's values from those of the cluster's blocks, in order
            for (int g = t; g < p.G; g += p.threads) {
                const double2 *v = xch + (size_t)buf * p.cl * p.G + g;
                const int size = group_begin(p, g + 1) - group_begin(p, g);
                const double m = (double)p.HW * (double)size;
                double v0 = 0.0, v1 = 0.0;
                if (BWD) {
                    for (int r = 0; r < p.cl; ++r) { v0 += v[(size_t)r * p.G].x; v1 += v[(size_t)r * p.G].y; }
                    const double rs = (double)grp[p.G + g], im = 1.0 / m;
                    const double t1 = -(rs * rs * rs * v1 * im);
                    out[g] = (float)(-(rs * v0 * im) - t1 * (double)grp[g]);
                    out[p.G + g] = (float)t1;
                } else {
                    // all blocks but the last have `share` pixels (those behind the last have none, and sent zeros)
                    for (int r = 0; r < whole; ++r) v0 += v[(size_t)r * p.G].x;
                    const double last = rest > 0.0 ? v[(size_t)whole * p.G].x : 0.0;
                    v0 = (v0 * (double)p.share + last * rest) * inv_hw;
                    double spread = 0.0;
                    for (int r = 0; r < whole; ++r) {
                        const double d = v[(size_t)r * p.G].x - v0;
                        spread += d * d;
                        v1 += v[(size_t)r * p.G].y;
                    }
                    spread = spread * (double)p.share + (last - v0) * (last - v0) * rest;
                    if (rest > 0.0) v1 += v[(size_t)whole * p.G].y;
                    v1 += spread * (double)size;
                    const float fm = (float)v0, fr = (float)rsqrt(v1 / m + (double)p.eps);
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
        // The second walk's constants, about x itself: forward, z = x*c1 + c2; backward, z = x*kz + be and the group's terms of dx,
        // x*c2 + c1. (What x - mean would keep of the last bits is lost in the rounding to bf16: with a mean of r standard deviations z is off by
        // r * 2^-23, and bf16 values of one mean and 2^-8 of it apart have r < 2^8 or so.)
        f2 c1[4], c2[4];
        {
            float u[8], v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int c = c0 + j, g = gid[c];
                u[j] = out[g];
                v[j] = out[p.G + g];
                if (!BWD) {
                    const float mean = v[j];
                    u[j] *= gam[c];
                    v[j] = fmaf(-mean, u[j], bet[c]);
                    if (ACT == PT_ACT_SILU) { u[j] *= -kLog2e; v[j] *= -kLog2e; }
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                c1[i] = mk2(u[2 * i], u[2 * i + 1]);
                c2[i] = mk2(v[2 * i], v[2 * i + 1]);
                if (BWD && !(ACT == PT_ACT_RELU && RES)) be[i] = fma2(nm[i], kz[i], be[i]);
            }
        }
        if (ahead && t < p.G && n + p.clusters < p.N) {
            next_mean = a.mean[(size_t)(n + p.clusters) * p.G + t];
            next_rstd = a.rstd[(size_t)(n + p.clusters) * p.G + t];
        }
        // ---- second walk, backwards: the results
        const bool want_y = !BWD || (PACKED && a.y);
        // gx, gr, gy: the batch's first pixel in dx, dresidual and y
        const auto result = [&](Raw &w, uint8_t *gx, uint8_t *gr, uint8_t *gy, uint32_t at) {
            f2 x[4], z[4], dz[4];
            uint4 o;
            uint32_t *ow = reinterpret_cast<uint32_t *>(&o);
            values(w, x);
            if (!BWD) {
                const uint32_t *rb = reinterpret_cast<const uint32_t *>(&w.res);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    f2 y = fma2(x[i], c1[i], c2[i]);
                    if (RES) y = ACT == PT_ACT_SILU ? fma2(from_bf(rb[i]), mk2(-kLog2e, -kLog2e), y) : add2(y, from_bf(rb[i]));
                    ow[i] = to_bf(activate2<ACT>(y));
                }
                if (lane_ok) *reinterpret_cast<uint4 *>(gy + at) = act8::and4(o, keep);
            } else {
                f2 d[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) d[i] = ACT == PT_ACT_RELU && RES ? add2(x[i], nm[i]) : x[i];
                gradient(w, d, z, dz, want_y);
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
        const auto residual = [&](int b) {
            if (!BWD && RES && b >= 0) {
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (b * step + u * p.ppb + pr < mine) ahead_w[u].res = *reinterpret_cast<const uint4 *>(src.res + ((uint32_t)b * step_v + off[u]));
            }
        };
        residual(NB - 1);
        const int kept = NB < B ? NB : B;
        uint8_t *gx = reinterpret_cast<uint8_t *>(a.dx) + base * row, *gr = reinterpret_cast<uint8_t *>(a.dres) + base * row, *gy = reinterpret_cast<uint8_t *>(a.y) + base * row;
        for (int b = NB - 1; b >= 0; --b) {
            s = s == s_first ? s_last : s - s_step;
            copy_wait<B - 1>();
            const int left = mine - b * step - pr;
            const uint32_t bv = (uint32_t)b * step_v, bs = (uint32_t)b * step_s;
            Raw w[U];
            if (!BWD && RES) {
#pragma unroll
                for (int u = 0; u < U; ++u) w[u].res = ahead_w[u].res;
                residual(b - 1);
            }
            if ((b + 1) * step <= mine) {
#pragma unroll
                for (int u = 0; u < U; ++u) fetch(w[u], bs, s, u);
#pragma unroll
                for (int u = 0; u < U; ++u) result(w[u], gx, gr, gy, bv + off[u]);
            } else {
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (u * p.ppb < left) {
                        fetch(w[u], bs, s, u);
                        result(w[u], gx, gr, gy, bv + off[u]);
                    }
            }
            // the place takes an earlier batch, or one of the cluster's next image: its first goes to the place that is free first
            if (b >= B) bring(src, b - B, s);
            else if (n + p.clusters < p.N) bring(next, kept - 1 - b, dir ? (kept - 1 - b) * U : (B - kept + b) * U);
            copy_commit();
        }
        src = next;
        if (BWD)                                                         // the images' sums of dz and dz * xhat, a channel's
            for (int c = t; c < p.C; c += p.threads) {
                const float *src = red + (c >> 3) * 17 + (c & 7);
                float v0 = 0.f, v1 = 0.f, u0 = 0.f, u1 = 0.f;
                int r = 0;
                for (; r + 1 < p.ppb; r += 2, src += 2 * p.rl * 17) {
                    v0 += src[0]; v1 += src[8];
                    u0 += src[p.rl * 17]; u1 += src[p.rl * 17 + 8];
                }
                if (r < p.ppb) { v0 += src[0]; v1 += src[8]; }
                acc[c] += (double)v0 + (double)u0;
                acc[p.ld + c] += ((double)v1 + (double)u1) * (double)grp[p.G + gid[c]];
            }
    }
    // ---- the cluster's sums over its images
    if (BWD) {
        if (p.cl > 1) sm100::cluster_barrier();
        else __syncthreads();
        const int per = (2 * p.ld + p.cl - 1) / p.cl;
        for (int e = rank * per + t; e < min(2 * p.ld, (rank + 1) * per); e += p.threads) {
            double v = 0.0;
            if (p.cl == 1) v = acc[e];
            else
                for (int r = 0; r < p.cl; ++r) v += ld_cluster_d(sm100::map_to_rank(sm100::smem_u32(acc + e), (uint32_t)r));
            const int s = e >= p.ld, c = e - s * p.ld;
            if (p.clusters > 1) a.rows[(size_t)cluster * 2 * p.ld + e] = v;
            else if (c < p.C) (s ? a.dgamma : a.dbeta)[c] = (float)v;
        }
    }
    if (p.cl > 1) sm100::cluster_barrier();
}

// dgamma, dbeta: the clusters' rows. A block owns 32 columns; its warps take every 32nd row each, then one thread per column adds the
// warps' sums: a fixed order, fp64.
__global__ void __launch_bounds__(1024) gn_finish_kernel(const double *rows, int n, int C, int ld, float *dgamma, float *dbeta)
{
    __shared__ double part[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, e = blockIdx.x * 32 + lane;
    sm100::grid_dependency_wait();
    sm100::grid_launch_dependents();
    double v = 0.0;
    if (e < 2 * ld)
        for (int r = warp; r < n; r += 32) v += rows[(size_t)r * 2 * ld + e];
    part[warp][lane] = v;
    __syncthreads();
    if (warp == 0 && e < 2 * ld) {
        v = 0.0;
        for (int k = 0; k < 32; ++k) v += part[k][lane];
        const int s = e >= ld, c = e - s * ld;
        if (c < C) (s ? dgamma : dbeta)[c] = (float)v;
    }
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
    if (d->ld > kGnMaxLd || (p->table && d->groups > kGnTable)) return PT_ERR_UNSUPPORTED;
    const long long hw = (long long)d->H * d->W;
    if (hw * d->ld * 2 >= 0x100000000ll || (codes && hw * d->ldq >= 0x100000000ll)) return PT_ERR_UNSUPPORTED;    // (offsets in an image have 32 bits)
    if (p->table)
        for (int g = 0; g <= d->groups; ++g) p->begin[g] = (uint16_t)b[g];
    p->N = d->N; p->HW = (int)hw; p->C = d->C; p->ld = d->ld; p->LV = d->ld / 8; p->ldq = d->ldq; p->nb = pt_ceil_div(d->C, act8::kBlock);
    p->G = d->groups; p->eps = d->eps;
    p->w = p->LV >= 3 ? 4 : p->LV;
    return PT_OK;
}

// The launch shape for clusters of cl blocks: how the threads cover a pixel row, and the shared memory's parts. Returns its bytes.
size_t gn_shape(GnP *p, int mode, bool res, int cl)
{
    p->cl = cl;
    p->share = pt_ceil_div(p->HW, cl);
    p->rl = mode == kGnFwdPack ? pt_ceil_div(p->LV, p->w) * p->w : p->LV;
    p->ppb = kGnThreads / p->rl;
    if (p->ppb > p->share) p->ppb = p->share;
    p->threads = (p->rl * p->ppb + 31) / 32 * 32;
    // lanes of a group: as many as there are for it; as many of them for its channels as it has
    int most = pt_ceil_div(p->C, p->G);
    if (p->table)
        for (int g = 0; g < p->G; ++g) most = most > p->begin[g + 1] - p->begin[g] ? most : p->begin[g + 1] - p->begin[g];
    p->gl = 1;
    while (p->gl < 32 && 2 * p->gl * p->G <= p->threads && p->gl < most * p->ppb) p->gl *= 2;
    p->gc = 1;
    while (p->gc < p->gl && p->gc < most) p->gc *= 2;
    size_t at = 0;
    const auto part = [&](unsigned *off, size_t bytes) { *off = (unsigned)at; at += pt_align_up(bytes, 16); };
    part(&p->sm_ring, (size_t)kGnThreads * kGnRows * gn_batches(mode, res) * gn_slot(mode, res));
    part(&p->sm_gid, (size_t)p->ld * 2);
    part(&p->sm_gam, (size_t)p->ld * 4);
    part(&p->sm_bet, (size_t)p->ld * 4);
    part(&p->sm_grp, (size_t)p->G * 6 * 4);
    part(&p->sm_red, (size_t)p->threads * 17 * 4);
    part(&p->sm_xch, (size_t)2 * cl * p->G * 16);
    part(&p->sm_acc, gn_bwd(mode) ? (size_t)2 * p->ld * 8 : 0);
    return at;
}

bool aligned16(const void *q) { return ((uintptr_t)q & 15) == 0; }

pt_status launch_gn(pt_ctx *c, GnP p, GnArgs a, int mode, int act, cudaStream_t st)
{
    const bool res = a.res != nullptr;
    const GnKernel kernel = gn_kernel_of(mode, act, res);
    const unsigned bit = 1u << ((mode * 3 + act) * 2 + (res ? 1 : 0));
    if (!(c->gn_attr_done & bit)) {
        PT_CUDA_OK(cudaFuncSetAttribute((const void *)kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 225 * 1024));
        PT_CUDA_OK(cudaFuncSetAttribute((const void *)kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
        c->gn_attr_done |= bit;
    }
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[2];
    memset(&cfg, 0, sizeof(cfg));
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.stream = st;
    cfg.attrs = attr;
    // the cluster size of the least estimated time
    double best = 1e30;
    int best_cl = 0, best_n = 0;
    for (int cl = 1; cl <= kGnMaxCluster; cl *= 2) {
        if (cl > 1 && (cl > p.HW || cl * p.G > kGnExchange)) break;
        GnP q = p;
        const size_t smem = gn_shape(&q, mode, res, cl);
        if (smem > 225 * 1024) continue;
        cfg.gridDim = dim3((unsigned)cl); cfg.blockDim = dim3((unsigned)q.threads); cfg.dynamicSmemBytes = smem;
        attr[1].val.clusterDim.x = (unsigned)cl;
        cfg.numAttrs = 2;
        int n = 0;
        if (cl > 1) {
            PT_CUDA_OK(cudaOccupancyMaxActiveClusters(&n, (const void *)kernel, &cfg));
        } else {
            PT_CUDA_OK(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, (const void *)kernel, (int)cfg.blockDim.x, smem));
            n *= c->sm_count;
        }
        if (n < 1) continue;
        if (n > kGnBlocks * c->sm_count) n = kGnBlocks * c->sm_count;
        const int clusters = n < p.N ? n : p.N, waves = pt_ceil_div(p.N, clusters);
        const double slot = gn_slot(mode, res), in = (double)q.share * p.LV * slot, ring = (double)kGnThreads * kGnRows * gn_batches(mode, res) * slot;
        const double bytes = in + 2.0 * q.share * p.ld + 0.5 * (in > ring ? in - ring : 0.0);
        double rate = 6500e3 / (clusters * cl);                   // bytes per microsecond and block
        if (rate > 60e3) rate = 60e3;
        const double us = waves * (bytes / rate + 2.0 + (cl > 1 ? 0.5 : 0.0));
        if (us < best) { best = us; best_cl = cl; best_n = clusters; }
    }
    if (!best_cl) return PT_ERR_UNSUPPORTED;
    const size_t smem = gn_shape(&p, mode, res, best_cl);
    p.clusters = best_n;
    cfg.gridDim = dim3((unsigned)(p.clusters * p.cl)); cfg.blockDim = dim3((unsigned)p.threads); cfg.dynamicSmemBytes = smem;
    attr[1].val.clusterDim.x = (unsigned)p.cl;
    cfg.numAttrs = p.cl > 1 ? 2 : 1;
    PT_CUDA_OK(cudaLaunchKernelEx(&cfg, kernel, p, a));
    c->launches += 1;
    if (mode >= kGnBwd && p.clusters > 1) {
        PT_CUDA_OK(pt_launch_pdl(gn_finish_kernel, dim3((unsigned)pt_ceil_div(2 * p.ld, 32)), dim3(1024), 0, st, (const double *)a.rows, p.clusters, p.C,
                                 p.ld, a.dgamma, a.dbeta));
        c->launches += 1;
    }
    return PT_OK;
}

}  // namespace

extern "C" size_t pt_gn_workspace_bytes(const pt_ctx *c, const pt_gn_desc *d)
{
    GnP p;
    if (gn_params(c, d, false, &p) != PT_OK) return 0;
    // a row of sums per cluster: no more than there are images, or blocks on the device
    const size_t most = (size_t)c->sm_count * 2;
    return ((size_t)p.N < most ? (size_t)p.N : most) * 2 * p.ld * sizeof(double);
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
    a.rows = (double *)ws; a.dgamma = dgamma; a.dbeta = dbeta;
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
    a.rows = (double *)ws; a.dgamma = dgamma; a.dbeta = dbeta;
    return launch_gn(c, p, a, kGnBwdPacked, d->act, (cudaStream_t)stream);
}
