// Group normalisation + residual add + activation on ragged channel counts and groups, channels last, forward and backward. NHWC bf16
// activations with channel pitch ld, fp32 statistics and parameters. Per image n and group g of m = H*W*|g| values:
//   forward : mean, rstd = 1/sqrt(var + eps), z = gamma*(x - mean)*rstd + beta (+ residual), y = act(z)
//   backward: dz = dy*act'(z), A = sum gamma*dz, B = sum gamma*dz*xhat, dx = rstd*(gamma*dz - A/m - xhat*B/m)
// A thread block per image reads its pixels twice, once for the sums and once for the results. No atomics: sums in a fixed order.
#include "pt_internal.h"
#include "pt_act.cuh"

namespace {

constexpr int kGnThreads = 256;
constexpr int kGnTable = 256;                // most groups of a table
constexpr int kGnMaxLd = 2048;

struct GnP {
    int N, HW, C, ld, LV, ldq, nb, G;
    int w, rl, ppb;              // lanes of a checkpoint's block, lanes of a pixel, pixels the threads cover at a time
    int act, table;
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
    float *rows;                 // backward: [N][2][ld] sums of dz and dz * xhat
};

__device__ __forceinline__ int group_begin(const GnP &p, int g) { return p.table ? p.begin[g] : g * (p.C / p.G); }

__device__ __forceinline__ float sigmoid(float z) { return __fdividef(1.f, 1.f + __expf(-z)); }

__device__ __forceinline__ float activate(float z, int act)
{
    if (act == PT_ACT_RELU) return z > 0.f ? z : (z != z ? z : 0.f);
    return act == PT_ACT_SILU ? z * sigmoid(z) : z;
}

// z > 0, decided in 64 bits where fp32 might be wrong about it.
__device__ __forceinline__ bool positive(float x, float mean, float rstd, float gamma, float beta, float r)
{
    const float u = (x - mean) * (gamma * rstd), z = u + beta + r;
    if (fabsf(z) > 1e-5f * (fabsf(u) + fabsf(r))) return z > 0.f;
    return ((double)x - (double)mean) * (double)rstd * (double)gamma + (double)beta + (double)r > 0.0;
}

template <bool BWD>
__global__ void __launch_bounds__(kGnThreads) gn_kernel(const __grid_constant__ GnP p, const GnArgs a)
{
    extern __shared__ float sm[];
    float *red = sm;                                     // [threads][16]
    double *chan = reinterpret_cast<double *>(sm + kGnThreads * 16);     // [2][ld]
    float *g0 = reinterpret_cast<float *>(chan + 2 * p.ld), *g1 = g0 + p.ld, *g2 = g1 + p.ld, *g3 = g2 + p.ld;       // per channel, from its group
    const int t = threadIdx.x, pr = t / p.rl, cv = t - pr * p.rl, n = blockIdx.x;
    const bool lane_ok = pr < p.ppb && cv < p.LV;
    const size_t base = (size_t)n * p.HW;
    const int c0 = cv * 8;
    const uint4 keep = act8::keep_bits(c0, p.C);
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
    if (BWD) {
        for (int g = t; g < p.G; g += kGnThreads)
            for (int c = group_begin(p, g); c < group_begin(p, g + 1); ++c) {
                g0[c] = a.mean[(size_t)n * p.G + g];
                g1[c] = a.rstd[(size_t)n * p.G + g];
            }
    } else {
        for (int g = t; g < p.G; g += kGnThreads) {      // pivot: the group's first value in the image
            const float v = __bfloat162float(reinterpret_cast<const __nv_bfloat16 *>(a.x)[base * p.ld + group_begin(p, g)]);
            for (int c = group_begin(p, g); c < group_begin(p, g + 1); ++c) g0[c] = v;
        }
    }
    __syncthreads();
    float s0[8], s1[8], k0[8], k1[8], gam[8], bet[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const bool ok = lane_ok && c0 + j < p.C;
        s0[j] = s1[j] = 0.f;
        k0[j] = ok ? g0[c0 + j] : 0.f;
        k1[j] = ok && BWD ? g1[c0 + j] : 0.f;
        gam[j] = ok ? a.gamma[c0 + j] : 0.f;
        bet[j] = ok ? a.beta[c0 + j] : 0.f;
    }
    const auto load_x = [&](size_t pix, float (&f)[8]) {
        if (BWD && a.codes_in) act8::decode8(*reinterpret_cast<const uint2 *>(a.codes_in + pix * p.ldq + c0), a.scales_in[pix * p.nb + (cv >> 2)], f);
        else act8::unpack8(a.x[pix * (p.ld / 8) + cv], f);
    };
    const auto load_dz = [&](size_t pix, const float (&x)[8], float (&dz)[8], float (&z)[8]) {
        float r[8];
        act8::unpack8(a.dy[pix * (p.ld / 8) + cv], dz);
        if (a.res) act8::unpack8(a.res[pix * (p.ld / 8) + cv], r);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float rj = a.res ? r[j] : 0.f;
            z[j] = fmaf(x[j] - k0[j], gam[j] * k1[j], bet[j]) + rj;
            if (p.act == PT_ACT_RELU) dz[j] = positive(x[j], k0[j], k1[j], gam[j], bet[j], rj) ? dz[j] : 0.f;
            if (p.act == PT_ACT_SILU) { const float s = sigmoid(z[j]); dz[j] *= fmaf(z[j] * s, 1.f - s, s); }
        }
    };
    for (int q0 = 0; q0 < p.HW; q0 += p.ppb) {
        const int q = q0 + pr;
        const bool ok = lane_ok && q < p.HW;
        const size_t pix = base + q;
        float x[8];
        if (BWD) {
            if (!ok || c0 >= p.C) continue;
            float dz[8], z[8];
            load_x(pix, x);
            load_dz(pix, x, dz, z);
#pragma unroll
            for (int j = 0; j < 8; ++j) { s0[j] += dz[j]; s1[j] = fmaf(dz[j], x[j] - k0[j], s1[j]); }
        } else {
            const uint4 v = ok ? a.x[pix * (p.ld / 8) + cv] : zero;
            act8::unpack8(v, x);
            if (ok)
#pragma unroll
                for (int j = 0; j < 8; ++j) { const float d = x[j] - k0[j]; s0[j] += d; s1[j] = fmaf(d, d, s1[j]); }
            if (a.codes) {
                const uint4 m = act8::and4(v, keep);
                const uint32_t byte = act8::scale_byte(act8::block_max(act8::amax8(m), p.w));
                if (ok && c0 < p.C) {
                    *reinterpret_cast<uint2 *>(a.codes + pix * p.ldq + c0) = act8::encode8(m, byte);
                    if ((cv & 3) == 0) a.scales[pix * p.nb + (cv >> 2)] = (uint8_t)byte;
                }
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) { red[t * 16 + j] = s0[j]; red[t * 16 + 8 + j] = s1[j]; }
    __syncthreads();
    for (int e = t; e < 2 * p.C; e += kGnThreads) {
        const int s = e >= p.C, c = e - s * p.C;
        double v = 0.0;
        for (int r = 0; r < p.ppb; ++r) v += (double)red[(r * p.rl + (c >> 3)) * 16 + s * 8 + (c & 7)];
        if (BWD && s) v *= (double)g1[c];
        chan[s * p.ld + c] = v;
        if (BWD) a.rows[((size_t)n * 2 + s) * p.ld + c] = (float)v;
    }
    __syncthreads();
    for (int g = t; g < p.G; g += kGnThreads) {
        const int b = group_begin(p, g), e = group_begin(p, g + 1);
        const double m = (double)p.HW * (double)(e - b);
        double v0 = 0.0, v1 = 0.0;
        for (int c = b; c < e; ++c) {
            const double f = BWD ? (double)a.gamma[c] : 1.0;
            v0 += f * chan[c];
            v1 += f * chan[p.ld + c];
        }
        float f0, f1;
        if (BWD) {
            const double r = (double)g1[b];
            f0 = (float)(r * v0 / m);
            f1 = (float)(r * r * v1 / m);
        } else {
            const double d = v0 / m;
            double var = v1 / m - d * d;
            if (var < 0.0) var = 0.0;
            f0 = (float)((double)g0[b] + d);
            f1 = (float)(1.0 / sqrt(var + (double)p.eps));
            a.save_mean[(size_t)n * p.G + g] = f0;
            a.save_rstd[(size_t)n * p.G + g] = f1;
        }
        for (int c = b; c < e; ++c) { g2[c] = f0; g3[c] = f1; }
    }
    __syncthreads();
    float k2[8], k3[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const bool ok = lane_ok && c0 + j < p.C;
        k2[j] = ok ? g2[c0 + j] : 0.f;
        k3[j] = ok ? g3[c0 + j] : 0.f;
    }
    if (!lane_ok) return;
    for (int q = pr; q < p.HW; q += p.ppb) {
        const size_t pix = base + q, at = pix * (p.ld / 8) + cv;
        float x[8], o[8];
        if (c0 >= p.C) {                                 // vectors of pad lanes only
            if (BWD) { a.dx[at] = zero; if (a.dres) a.dres[at] = zero; }
            if (a.y) a.y[at] = zero;
            continue;
        }
        load_x(pix, x);
        if (!BWD) {
            float r[8];
            if (a.res) act8::unpack8(a.res[at], r);
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = activate(fmaf(x[j] - k2[j], gam[j] * k3[j], bet[j]) + (a.res ? r[j] : 0.f), p.act);
            a.y[at] = act8::and4(act8::pack8(o), keep);
        } else {
            float dz[8], z[8];
            load_dz(pix, x, dz, z);
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = fmaf(gam[j] * k1[j], dz[j], -fmaf(x[j] - k0[j], k3[j], k2[j]));
            a.dx[at] = act8::and4(act8::pack8(o), keep);
            if (a.dres) a.dres[at] = act8::and4(act8::pack8(dz), keep);
            if (a.y) {
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = activate(z[j], p.act);
                a.y[at] = act8::and4(act8::pack8(o), keep);
            }
        }
    }
}

// dgamma, dbeta: the images' rows in order, in fp64.
__global__ void gn_finish_kernel(const float *rows, int n, int C, int ld, float *dgamma, float *dbeta)
{
    const int e = blockIdx.x * blockDim.x + threadIdx.x, s = e >= C, c = e - s * C;
    if (e >= 2 * C) return;
    double v = 0.0;
    for (int r = 0; r < n; ++r) v += (double)rows[((size_t)r * 2 + s) * ld + c];
    (s ? dgamma : dbeta)[c] = (float)v;
}

pt_status gn_params(const pt_ctx *c, const pt_gn_desc *d, bool codes, GnP *p)
{
    if (!c || !d) return PT_ERR_INVALID_ARG;
    if (d->N < 1 || d->H < 1 || d->W < 1 || d->C < 1 || d->ld < d->C || (d->ld & 7)) return PT_ERR_INVALID_ARG;
    if (d->groups < 1 || d->groups > d->C || !(d->eps >= 0.f) || d->act < PT_ACT_NONE || d->act > PT_ACT_SILU) return PT_ERR_INVALID_ARG;
    if (codes && (d->ldq < d->C || (d->ldq & 7))) return PT_ERR_INVALID_ARG;
    p->table = 0;
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
    if (hw > 0x7fffffffll) return PT_ERR_UNSUPPORTED;
    if (p->table)
        for (int g = 0; g <= d->groups; ++g) p->begin[g] = (uint16_t)b[g];
    p->N = d->N; p->HW = (int)hw; p->C = d->C; p->ld = d->ld; p->LV = d->ld / 8; p->ldq = d->ldq; p->nb = pt_ceil_div(d->C, act8::kBlock);
    p->G = d->groups; p->act = d->act; p->eps = d->eps;
    p->w = p->LV >= 3 ? 4 : p->LV;
    p->rl = pt_ceil_div(p->LV, p->w) * p->w;
    p->ppb = kGnThreads / p->rl;
    return PT_OK;
}

size_t gn_smem(const GnP &p) { return kGnThreads * 16 * sizeof(float) + 2 * (size_t)p.ld * sizeof(double) + 4 * (size_t)p.ld * sizeof(float); }

bool aligned16(const void *q) { return ((uintptr_t)q & 15) == 0; }

template <bool BWD>
pt_status launch_gn(pt_ctx *c, const GnP &p, const GnArgs &a, cudaStream_t st)
{
    PT_CUDA_OK(cudaFuncSetAttribute(gn_kernel<BWD>, cudaFuncAttributeMaxDynamicSharedMemorySize, 100 * 1024));
    gn_kernel<BWD><<<p.N, kGnThreads, gn_smem(p), st>>>(p, a);
    c->launches += 1;
    PT_CUDA_OK(cudaGetLastError());
    return PT_OK;
}

pt_status gn_backward(pt_ctx *c, const GnP &p, GnArgs &a, float *dgamma, float *dbeta, void *ws, cudaStream_t st)
{
    a.rows = (float *)ws;
    pt_status r = launch_gn<true>(c, p, a, st);
    if (r != PT_OK) return r;
    gn_finish_kernel<<<pt_ceil_div(2 * p.C, 128), 128, 0, st>>>(a.rows, p.N, p.C, p.ld, dgamma, dbeta);
    c->launches += 1;
    PT_CUDA_OK(cudaGetLastError());
    return PT_OK;
}

}  // namespace

extern "C" size_t pt_gn_workspace_bytes(const pt_ctx *c, const pt_gn_desc *d)
{
    GnP p;
    if (gn_params(c, d, false, &p) != PT_OK) return 0;
    return (size_t)p.N * 2 * p.ld * sizeof(float);
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
    return launch_gn<false>(c, p, a, (cudaStream_t)stream);
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
    return gn_backward(c, p, a, dgamma, dbeta, ws, (cudaStream_t)stream);
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
    return gn_backward(c, p, a, dgamma, dbeta, ws, (cudaStream_t)stream);
}
