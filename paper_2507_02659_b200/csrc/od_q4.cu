// An output layer with 4-bit weights, for a few tokens, and the way of a gradient back through it:
//   w[v,h] = s[v, h / G] (u[v,h] - 8),   y[n,v] = sum_h x[n,h] w[v,h],   dx[n,h] = sum_v dy[n,v] w[v,h].
// Codes u are 4 bits (column 2i in the low half of byte i of a row), scales s are bf16. Products and sums are fp32.
#include "od_common.cuh"

namespace {

constexpr int TOKENS = 8;                                  // of a block

template <typename T> __device__ __forceinline__ float to_float(T v);
template <> __device__ __forceinline__ float to_float<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_float<unsigned short>(unsigned short v) { return __uint_as_float((uint32_t)v << 16); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ unsigned short from_float<unsigned short>(float v)
{
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(0.f), "f"(v));
    return (unsigned short)d;
}

// a warp to a row of the weights
template <typename X, typename Y>
__global__ void od_q4_kernel(int N, int V, int H, int log_g, const X *x, int64_t xs, const uint8_t *codes, const unsigned short *scales,
                             Y *y, int64_t ys)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x & 31, v = blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5), n0 = blockIdx.y * TOKENS;
    if (v >= V) return;
    float acc[TOKENS] = {};
    for (int i = lane; i < H / 2; i += 32) {
        const uint8_t q = codes[(size_t)v * (H / 2) + i];
        const float s = to_float(scales[(size_t)v * (H >> log_g) + (2 * i >> log_g)]);
        const float lo = s * (float)((q & 15) - 8), hi = s * (float)((q >> 4) - 8);
#pragma unroll
        for (int t = 0; t < TOKENS; ++t)
            if (n0 + t < N) acc[t] += lo * to_float(x[(n0 + t) * xs + 2 * i]) + hi * to_float(x[(n0 + t) * xs + 2 * i + 1]);
    }
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) {
#pragma unroll
        for (int o = 16; o; o >>= 1) acc[t] += __shfl_xor_sync(0xFFFFFFFFu, acc[t], o);
        if (lane == 0 && n0 + t < N) y[(n0 + t) * ys + v] = from_float<Y>(acc[t]);
    }
}

// a thread to two columns of the weights
template <typename X, typename Y>
__global__ void od_q4_grad_kernel(int N, int V, int H, int log_g, const X *dy, int64_t ds, const uint8_t *codes,
                                  const unsigned short *scales, Y *dx, int64_t xs)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int i = blockIdx.x * blockDim.x + threadIdx.x, n0 = blockIdx.y * TOKENS;
    if (i >= H / 2) return;
    float lo[TOKENS] = {}, hi[TOKENS] = {};
    for (int v = 0; v < V; ++v) {
        const uint8_t q = codes[(size_t)v * (H / 2) + i];
        const float s = to_float(scales[(size_t)v * (H >> log_g) + (2 * i >> log_g)]);
#pragma unroll
        for (int t = 0; t < TOKENS; ++t) {
            if (n0 + t >= N) continue;
            const float g = s * to_float(dy[(n0 + t) * ds + v]);
            lo[t] += g * (float)((q & 15) - 8);
            hi[t] += g * (float)((q >> 4) - 8);
        }
    }
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) {
        if (n0 + t >= N) break;
        dx[(n0 + t) * xs + 2 * i] = from_float<Y>(lo[t]);
        dx[(n0 + t) * xs + 2 * i + 1] = from_float<Y>(hi[t]);
    }
}

template <typename X, typename Y>
cudaError_t launch(bool backward, int32_t N, int32_t V, int32_t H, int log_g, const void *a, int64_t as, const void *codes,
                   const void *scales, void *b, int64_t bs, bool pdl, cudaStream_t s)
{
    cudaLaunchConfig_t cfg = {};
    const unsigned tiles = (unsigned)((N + TOKENS - 1) / TOKENS);
    cfg.blockDim = dim3(128);
    cfg.gridDim = backward ? dim3((unsigned)((H / 2 + 127) / 128), tiles) : dim3((unsigned)((V + 3) / 4), tiles);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = pdl ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, backward ? od_q4_grad_kernel<X, Y> : od_q4_kernel<X, Y>, (int)N, (int)V, (int)H, log_g, (const X *)a, as,
                              (const uint8_t *)codes, (const unsigned short *)scales, (Y *)b, bs);
}

}  // namespace

cudaError_t od_launch_q4(const od_ctx *c, bool backward, int32_t N, int32_t V, int32_t H, int32_t G, const void *a, int32_t a_dtype,
                         int64_t as, const void *codes, const void *scales, void *b, int32_t b_dtype, int64_t bs, cudaStream_t s)
{
    const int log_g = G == 32 ? 5 : G == 64 ? 6 : 7;
    const bool pdl = c->opt_pdl != 0;
    typedef unsigned short bf16;
    if (a_dtype == OD_BF16)
        return b_dtype == OD_BF16 ? launch<bf16, bf16>(backward, N, V, H, log_g, a, as, codes, scales, b, bs, pdl, s)
                                  : launch<bf16, float>(backward, N, V, H, log_g, a, as, codes, scales, b, bs, pdl, s);
    return b_dtype == OD_BF16 ? launch<float, bf16>(backward, N, V, H, log_g, a, as, codes, scales, b, bs, pdl, s)
                              : launch<float, float>(backward, N, V, H, log_g, a, as, codes, scales, b, bs, pdl, s);
}
