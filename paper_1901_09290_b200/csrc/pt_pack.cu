// 8-bit activation checkpoints of whole tensors: bf16 [npix][ld] -> codes int8 [npix][ldq] and scale bytes [npix][ceil(C / 32)], and back.
// Bound by memory: 3 + 1/32 bytes per value in either direction. A thread owns a 16-byte vector of a pixel; the (at most four) neighbouring
// lanes of a block find its largest magnitude by shuffles.
#include "pt_internal.h"
#include "pt_act.cuh"

namespace {

constexpr int kPackThreads = 256;

struct PackP {
    long long npix;
    int C, ld, ldq, LV, nb;
    int w, rl, rows;            // lanes of a block (1, 2 or 4), lanes of a pixel (LV rounded up to w), pixels a thread block covers at a time
};

__global__ void __launch_bounds__(kPackThreads) pack_kernel(const PackP p, const uint4 *x, uint8_t *codes, uint8_t *scales)
{
    const int t = threadIdx.x, pr = t / p.rl, cv = t - pr * p.rl;
    const bool lane_ok = pr < p.rows && cv < p.LV;
    const uint4 keep = act8::keep_bits(cv * 8, p.C);
    for (long long p0 = (long long)blockIdx.x * p.rows; p0 < p.npix; p0 += (long long)gridDim.x * p.rows) {
        const long long pix = p0 + pr;
        const bool ok = lane_ok && pix < p.npix;
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (ok) v = act8::and4(x[pix * (p.ld / 8) + cv], keep);
        const uint32_t byte = act8::scale_byte(act8::block_max(act8::amax8(v), p.w));
        if (ok) {
            *reinterpret_cast<uint2 *>(codes + pix * p.ldq + cv * 8) = act8::encode8(v, byte);
            if ((cv & 3) == 0) scales[pix * p.nb + (cv >> 2)] = (uint8_t)byte;
        }
    }
}

__global__ void __launch_bounds__(kPackThreads) unpack_kernel(const PackP p, const uint8_t *codes, const uint8_t *scales, uint4 *x)
{
    const int t = threadIdx.x, out_lv = p.ld / 8;
    const long long n = p.npix * out_lv;
    for (long long i = (long long)blockIdx.x * kPackThreads + t; i < n; i += (long long)gridDim.x * kPackThreads) {
        const long long pix = i / out_lv;
        const int cv = (int)(i - pix * out_lv);
        uint4 o = make_uint4(0u, 0u, 0u, 0u);
        if (cv < p.LV) {
            float f[8];
            act8::decode8(*reinterpret_cast<const uint2 *>(codes + pix * p.ldq + cv * 8), scales[pix * p.nb + (cv >> 2)], f);
            o = act8::and4(act8::pack8(f), act8::keep_bits(cv * 8, p.C));
        }
        x[i] = o;
    }
}

pt_status pack_params(const pt_ctx *c, const pt_pack_desc *d, const void *x, const void *codes, const void *scales, PackP *p)
{
    if (!c || !d || !x || !codes || !scales) return PT_ERR_INVALID_ARG;
    if (d->npix < 0 || d->C < 1 || d->ld < d->C || (d->ld & 7) || d->ldq < d->C || (d->ldq & 7)) return PT_ERR_INVALID_ARG;
    if (((uintptr_t)x | (uintptr_t)codes | (uintptr_t)scales) & 15) return PT_ERR_INVALID_ARG;
    if (!pt_on_device(c)) return PT_ERR_INVALID_ARG;
    if (d->ld > 2048) return PT_ERR_UNSUPPORTED;
    p->npix = d->npix; p->C = d->C; p->ld = d->ld; p->ldq = d->ldq;
    p->LV = (d->C + 7) / 8; p->nb = pt_ceil_div(d->C, act8::kBlock);
    p->w = p->LV >= 3 ? 4 : p->LV;
    p->rl = pt_ceil_div(p->LV, p->w) * p->w;
    p->rows = kPackThreads / p->rl;
    return PT_OK;
}

}  // namespace

extern "C" size_t pt_act_scale_bytes(int64_t npix, int32_t C)
{
    if (npix < 0 || C < 1) return 0;
    return pt_align_up((size_t)npix * (size_t)((C + act8::kBlock - 1) / act8::kBlock), 16);
}

extern "C" pt_status pt_act_pack(pt_ctx *c, const pt_pack_desc *d, const void *x, void *codes, void *scales, void *stream)
{
    PackP p;
    const pt_status r = pack_params(c, d, x, codes, scales, &p);
    if (r != PT_OK) return r;
    if (p.npix == 0) return PT_OK;
    const long long need = (p.npix + p.rows - 1) / p.rows, most = (long long)c->sm_count * 8;
    pack_kernel<<<(unsigned)(need < most ? need : most), kPackThreads, 0, (cudaStream_t)stream>>>(p, (const uint4 *)x, (uint8_t *)codes, (uint8_t *)scales);
    c->launches += 1;
    PT_CUDA_OK(cudaGetLastError());
    return PT_OK;
}

extern "C" pt_status pt_act_unpack(pt_ctx *c, const pt_pack_desc *d, const void *codes, const void *scales, void *x, void *stream)
{
    PackP p;
    const pt_status r = pack_params(c, d, x, codes, scales, &p);
    if (r != PT_OK) return r;
    if (p.npix == 0) return PT_OK;
    const long long need = (p.npix * (p.ld / 8) + kPackThreads - 1) / kPackThreads, most = (long long)c->sm_count * 8;
    unpack_kernel<<<(unsigned)(need < most ? need : most), kPackThreads, 0, (cudaStream_t)stream>>>(p, (const uint8_t *)codes, (const uint8_t *)scales, (uint4 *)x);
    c->launches += 1;
    PT_CUDA_OK(cudaGetLastError());
    return PT_OK;
}
