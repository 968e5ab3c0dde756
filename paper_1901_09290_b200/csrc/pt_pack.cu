// 8-bit activation checkpoints of whole tensors: bf16 [npix][ld] -> codes int8 [npix][ldq] and scale bytes [npix][ceil(C / 32)], and back.
// Bound by memory: 3 + 1/32 bytes per value in either direction. A thread owns a 16-byte vector column and every so many-th pixel, four of
// them at a time, all loads before the first use: the pair of passes takes 53.8 us at 64x56x56x256 (5.8 TB/s, 0.88 of the copy rate), and took
// 73 with one at a time, what was in flight being the bound. The (at most four) neighbouring lanes of a block find its largest magnitude by shuffles.
#include "pt_internal.h"
#include "pt_act.cuh"
#include "pt_sm100_ptx.cuh"

namespace {

constexpr int kPackThreads = 256;
constexpr long long kMaxPixels = 1ll << 40;      // more than any memory holds: products with pitches stay within 64 bits
constexpr int kPackBlocks = 6;      // thread blocks of an SM at a time

struct PackP {
    long long npix;
    int C, ld, ldq, LV, nb;
    int w, rl, rows;            // lanes of a block (1, 2 or 4), lanes of a pixel, pixels a thread block covers at a time
};

// PACK: x -> codes, scales; otherwise back, with zeros for the pad lanes (every vector of a pixel has a lane then).
// U: pixels of a thread at a time.
template <bool PACK, int U>
__global__ void __launch_bounds__(kPackThreads, kPackBlocks) pack_kernel(const PackP p, uint8_t *x, uint8_t *codes, uint8_t *scales)
{
    const int t = threadIdx.x, pr = t / p.rl, cv = t - pr * p.rl;
    const bool has = pr < p.rows && cv < p.LV, pad = !PACK && pr < p.rows && cv < p.ld / 8;
    const uint4 keep = act8::keep_bits(cv * 8, p.C), zero = make_uint4(0u, 0u, 0u, 0u);
    const int step = U * p.rows;
    uint32_t ox[U], oq[U], os[U];                                // (a thread block's pixels at a time: less than 4 GB, see launch_pack)
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t r = (uint32_t)(pr + u * p.rows);
        ox[u] = r * (uint32_t)p.ld * 2u + (uint32_t)cv * 16u;
        oq[u] = r * (uint32_t)p.ldq + (uint32_t)cv * 8u;
        os[u] = r * (uint32_t)p.nb + (uint32_t)(cv >> 2);
    }
    sm100::grid_dependency_wait();
    sm100::grid_launch_dependents();
    for (long long p0 = (long long)blockIdx.x * step; p0 < p.npix; p0 += (long long)gridDim.x * step) {
        uint8_t *gx = x + p0 * p.ld * 2, *gq = codes + p0 * p.ldq, *gs = scales + p0 * p.nb;
        const int left = p.npix - p0 < step ? (int)(p.npix - p0) : step;
        if (PACK) {
            uint4 v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = has && pr + u * p.rows < left ? *reinterpret_cast<const uint4 *>(gx + ox[u]) : zero;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                v[u] = act8::and4(v[u], keep);
                const uint32_t byte = act8::scale_byte(act8::block_max(act8::amax8(v[u]), p.w));
                if (has && pr + u * p.rows < left) {
                    *reinterpret_cast<uint2 *>(gq + oq[u]) = act8::encode8(v[u], byte);
                    if ((cv & 3) == 0) gs[os[u]] = (uint8_t)byte;
                }
            }
        } else {
            uint2 q[U];
            uint32_t b[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool ok = has && pr + u * p.rows < left;
                q[u] = ok ? *reinterpret_cast<const uint2 *>(gq + oq[u]) : make_uint2(0u, 0u);
                b[u] = ok ? gs[os[u]] : 0u;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float f[8];
                act8::decode8(q[u], b[u], f);
                if (pad && pr + u * p.rows < left) *reinterpret_cast<uint4 *>(gx + ox[u]) = act8::and4(act8::pack8(f), keep);
            }
        }
    }
}

template <bool PACK>
pt_status launch_pack(pt_ctx *c, PackP p, void *x, void *codes, void *scales, cudaStream_t st)
{
    if (p.npix == 0) return PT_OK;
    p.rl = PACK ? pt_ceil_div(p.LV, p.w) * p.w : p.ld / 8;
    p.rows = kPackThreads / p.rl;
    // Offsets within a thread block's pixels have 32 bits: where codes lie megabytes apart a block takes fewer pixels, so that rows * ldq is
    // below 2^32. (Four of them at a time only where that holds for all four. Pitches of bf16 are far below.)
    if ((long long)p.rows * p.ldq > 0xffffffffll) p.rows = (int)(0xffffffffll / p.ldq);
    // Blocks of a few rounds each, four to a place on an SM: both passes at 64x56x56x256 take 56.5 us with one round of blocks that share
    // everything, 53.8 with four, 57.3 with a block for every four pixels a thread. Small tensors: a pixel at a time, spread over more blocks
    // (128x8x8x41: 3.8 us where four at a time took 4.7).
    const long long most = (long long)c->sm_count * kPackBlocks * 4, one = (p.npix + p.rows - 1) / p.rows;
    const bool four = one >= most && 4ll * p.rows * p.ldq <= 0xffffffffll;
    const long long need = four ? (one + 3) / 4 : one;
    PT_CUDA_OK(pt_launch_pdl(four ? pack_kernel<PACK, 4> : pack_kernel<PACK, 1>, dim3((unsigned)(need < most ? need : most)), dim3(kPackThreads), 0, st, p,
                             (uint8_t *)x, (uint8_t *)codes, (uint8_t *)scales));
    c->launches += 1;
    PT_CUDA_OK(cudaGetLastError());
    return PT_OK;
}

pt_status pack_params(const pt_ctx *c, const pt_pack_desc *d, const void *x, const void *codes, const void *scales, PackP *p)
{
    if (!c || !d || !x || !codes || !scales) return PT_ERR_INVALID_ARG;
    if (d->npix < 0 || d->C < 1 || d->ld < d->C || (d->ld & 7) || d->ldq < d->C || (d->ldq & 7)) return PT_ERR_INVALID_ARG;
    if (((uintptr_t)x | (uintptr_t)codes | (uintptr_t)scales) & 15) return PT_ERR_INVALID_ARG;
    if (!pt_on_device(c)) return PT_ERR_INVALID_ARG;
    if (d->ld > 2048 || d->npix > kMaxPixels) return PT_ERR_UNSUPPORTED;
    p->npix = d->npix; p->C = d->C; p->ld = d->ld; p->ldq = d->ldq;
    p->LV = (d->C + 7) / 8; p->nb = pt_ceil_div(d->C, act8::kBlock);
    p->w = p->LV >= 3 ? 4 : p->LV;
    return PT_OK;
}

}  // namespace

extern "C" size_t pt_act_scale_bytes(int64_t npix, int32_t C)
{
    if (npix < 0 || npix > kMaxPixels || C < 1 || C > 2048) return 0;
    return pt_align_up((size_t)npix * (size_t)pt_ceil_div(C, act8::kBlock), 16);
}

extern "C" pt_status pt_act_pack(pt_ctx *c, const pt_pack_desc *d, const void *x, void *codes, void *scales, void *stream)
{
    PackP p;
    const pt_status r = pack_params(c, d, x, codes, scales, &p);
    return r != PT_OK ? r : launch_pack<true>(c, p, const_cast<void *>(x), codes, scales, (cudaStream_t)stream);
}

extern "C" pt_status pt_act_unpack(pt_ctx *c, const pt_pack_desc *d, const void *codes, const void *scales, void *x, void *stream)
{
    PackP p;
    const pt_status r = pack_params(c, d, x, codes, scales, &p);
    return r != PT_OK ? r : launch_pack<false>(c, p, x, const_cast<void *>(codes), const_cast<void *>(scales), (cudaStream_t)stream);
}
