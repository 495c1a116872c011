// An output layer with 4-bit weights, for a few tokens, and the way of a gradient back through it:
//   w[v,h] = s[v, h / G] (u[v,h] - 8),   y[n,v] = sum_h x[n,h] w[v,h],   dx[n,h] = sum_v dy[n,v] w[v,h].
// Codes u are 4 bits (column 2i in the low half of byte i of a row), scales s are bf16.
//
// Both products run on the tensor pipe as mma.m16n8k16 with the codes as the first operand and eight tokens as the
// second. A code is exact in bf16, and so is an input: a bf16 one as it is, an fp32 one as the sum of three bf16 pieces
// (24 bits = 8 + 8 + 8), the product of a bf16 gradient and a bf16 scale as that of two. So the only roundings are those
// of fp32 sums (and of an fp32 gradient times its scale). The scale of a group belongs to a row of the weights: forward
// it multiplies the group's sum, backward, where rows are summed over, the gradient.
//
// For a few tokens the codes are all there is to move, and unpacking them is what competes with that. Forward, of bf16 inputs,
// nothing is subtracted from a code and nothing or'ed to it: with no more than eight bits set a bf16 number is its bits times 2^-133 (in
// the first binade too), so two masks, a shift and two masks make eight codes u, half of them as 16 u, ready for the tensor
// pipe. The inputs are scaled by a power of two so that products are in fp32's range, and divided by 16 where they meet a
// 16 u. The 8 is taken off in what a group's sum begins at, -8 times the sum of its inputs, which is exact for inputs of 8 bits that
// are not too far apart. (Eight tokens through 128256 x 4096, bf16 results: 52 us, and 62 with u - 8 as ordinary bf16 numbers.) What that
// costs is digits where inputs have one sign or a few of them stand out, as sums run through numbers many times the result: against 64 bits
// 0.9e-6 of the result's norm for inputs of one sign through 4096 columns in groups of 128 (plain fp32 sums 1.5e-7), 1.4e-6 for 16384.
// For fp32 inputs such a beginning is rounded itself (2e-5 for equal ones, 1.6e-6 for one sign): their codes are made u - 8, as
// ordinary numbers, and a group's sums begin at zero (1e-7, where plain fp32 sums are 4e-7 off). Beside three pieces that costs little (8 tokens
// through 32000 x 2048: 17.4 us for 16.5, 6 through 128256 x 1024 30.1 for 28.3).
// Operands go from registers into mma.sync: for tcgen05 they would be written to shared memory and read there at two
// bytes a weight, 29 us of its bandwidth for 128256 x 2048 by arithmetic, whose codes HBM brings in 21. That speaks against it for 8
// tokens; for 16 and more, where these kernels take 63 us and more backward, it does not, and tcgen05 has not been tried.
//
// A warp streams its own codes through a ring in shared memory (cp.async, 2 KB stages), so that no block barrier holds it
// up: without the arithmetic the forward kernel reads 6.2 TB/s. Sixteen-byte pieces are placed so that the words of a
// fragment lie in different banks.
//
// Measured (us; codes and scales / HBM's rate): forward 8 tokens, 128256 x 4096 in groups of 128: 52 (42), and 60 in a long
// run, under the power cap; backward 8 positions, 128256 x 2048: 44 (21), 16: 63, 24: 85, 32: 105, with fp32 results 47, 71, 103 and 115. No
// unit is full (ncu, 8 tokens): forward shared memory's data path is busiest, 67 %, as a warp reads 512 bytes of fragments for every 256
// of codes, then issue 60 %, the masks' pipe 56 %, the tensor pipe 30 %; backward issue 61 %, the masks' pipe 56 %, the tensor pipe 37 %.
#include <float.h>

#include <mutex>

#include "od_common.cuh"

namespace {

constexpr int F_WARPS = 16, F_THREADS = 32 * F_WARPS;
constexpr int ROWS = 16;                                   // of a matrix instruction
constexpr int COLS = 128;                                  // backward: of a warp, four blocks of 32
// Backward: warps of a block, by eights of tokens. A warp's sums are 32 numbers of a lane for every eight tokens: with fewer warps
// codes are unpacked for more tokens at once. (128256 x 2048, us to bf16 results: 16 tokens by 16 / 12 / 8 warps 69 / 63 / 68; 24 by 8 / 10
// 85 / 98, and 113 as 16 and then 8; 32 by 8 / 10 105 / 136; 8 by 16 / 12 45 / 46.)
constexpr int G_WARPS[5] = {0, 16, 12, 8, 8};
constexpr int G_RING = 3;                                  // backward: stages of a warp
constexpr int WIDE = 8;                                    // forward: blocks of 32 columns to a stage
constexpr int WIDE_STAGE = ROWS * WIDE * 16;              // bytes

struct Q4Args {
    const void *in;                                        // x or dy
    int64_t in_stride;
    const uint8_t *codes;
    const unsigned short *scales;
    void *out;
    int64_t out_stride;
    int32_t N, V, H, in_f32, out_f32;
    int32_t wide_scales;                                   // the scales of a stage's row are one aligned word
    uint32_t bf16_128;                                     // see unpack
    int32_t k_split;                                       // forward: warps to the same rows
    int32_t split, col_warps;                              // backward: blocks on the same columns, warps side by side
    int32_t cluster;                                       // the blocks on the same columns are one
    int32_t first_token;
    float *parts;                                          // the context's scratch
};

__device__ __forceinline__ void cp16(uint32_t to, const void *from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint32_t lds32(uint32_t at)
{
    return *(const uint32_t *)__cvta_shared_to_generic(at);
}
__device__ __forceinline__ uint4 lds128(uint32_t at)
{
    return *(const uint4 *)__cvta_shared_to_generic(at);
}
__device__ __forceinline__ uint64_t f2_mul(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ float load_cluster(const float *p, uint32_t rank)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(od_cluster_address(p, rank)) : "memory");
    return v;
}
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_of(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)   // from zero
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t halves(uint32_t a, uint32_t b, uint32_t pick)
{
    return __byte_perm(a, b, pick);
}
constexpr uint32_t CODE = 0x000F000Fu, CODE16 = 0x00F000F0u;
// Codes I and I + 4 of a word, less 8, as a pair of bf16: 128 + u has u in its last bits. (bf16_128, a pair of 128, is an
// argument of the kernel: a mask and an or with two constants that the compiler knows are two instructions, with one in a
// register they are one.)
template <int I>
__device__ __forceinline__ uint32_t unpack(uint32_t w, uint32_t bf16_128)
{
    uint32_t m, d;
    asm("lop3.b32 %0, %1, 0x000F000F, %2, 0xEA;" : "=r"(m) : "r"(w >> 4 * I), "r"(bf16_128));
    asm("sub.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(m), "r"(0x43084308u));
    return d;
}
constexpr uint32_t LOW = 0x5410, HIGH = 0x7632;            // both low halves, both high halves

// P pieces of a pair as bf16 pairs: the leading 8 bits of what is left, which are cut off it
template <int P>
__device__ __forceinline__ void pieces(float a, float b, uint32_t (&out)[P])
{
    out[0] = halves(__float_as_uint(a), __float_as_uint(b), HIGH);
#pragma unroll
    for (int p = 1; p < P; ++p) {
        a -= __uint_as_float(__float_as_uint(a) & 0xFFFF0000u);
        b -= __uint_as_float(__float_as_uint(b) & 0xFFFF0000u);
        out[p] = halves(__float_as_uint(a), __float_as_uint(b), HIGH);
    }
}

__device__ __forceinline__ void store(const Q4Args &A, int n, int i, float v)
{
    if (A.out_f32) {
        ((float *)A.out)[(size_t)n * A.out_stride + i] = v;
    } else {
        uint32_t d;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(0.f), "f"(v));
        ((unsigned short *)A.out)[(size_t)n * A.out_stride + i] = (unsigned short)d;
    }
}

// The scales of a stage's columns in one row of the weights, raw: 4 / GB of them in the first halves of two words.
template <int GB>
struct Scales {
    uint32_t w[GB == 1 ? 2 : 1];
    // at: the row's first scale of the stage; n: how many of them there are
    __device__ __forceinline__ void load(const unsigned short *at, int n, bool wide)
    {
        if (GB == 4) {
            w[0] = __ldg(at);
        } else if (wide) {
            if constexpr (GB == 1) {
                const uint2 v = __ldg((const uint2 *)at);
                w[0] = v.x; w[1] = v.y;
            } else {
                w[0] = __ldg((const uint32_t *)at);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4 / GB; i += 2) {
                const uint32_t lo = i < n ? __ldg(at + i) : 0u, hi = i + 1 < n ? __ldg(at + i + 1) : 0u;
                w[i / 2] = lo | hi << 16;
            }
        }
    }
    __device__ __forceinline__ float get(int i) const { return i & 1 ? od_bf16_hi(w[i >> 1]) : od_bf16_lo(w[i >> 1]); }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (auto &x : w) x = 0;
    }
};

// ---- forward: 16 rows of the weights to a warp, all columns -------------------------------------
//
// A word of a row is eight columns: a stage's block of 32 columns is four words, one to each of the four lanes that share
// a row of the fragment, and codes i and i + 4 of the word are its pairs. The lanes' inputs are the same eight columns of
// a token. XS: a block of threads keeps its tokens' inputs in shared memory as the words of the fragments, 16 bytes to a
// lane; where they do not fit, they are read and cut again for every 16 rows.

// The scale of a token whose largest magnitude has these bits is 2^(CODES + k). Codes are 2^-CODES of themselves (of fp32 inputs
// they are themselves), and k is 0 or, for products in fp32's range, -27 where that is from 2^-8 up to 2^20, as it is nearly
// always; for others (all of zeros too) it brings the largest to 2^-7. An input keeps all its digits down to 2^-90 of its token's
// largest.
template <bool F32> constexpr int CODES = F32 ? 0 : 133;
__device__ __forceinline__ bool usual(uint32_t largest) { return largest >= (127u - 8 << 23) && largest < (127u + 20 << 23); }
template <bool F32>
__device__ __forceinline__ int scale_of_token(uint32_t largest) { return CODES<F32> + (usual(largest) ? F32 ? 0 : -27 : 120 - (int)(largest >> 23)); }
// eight columns of a token (columns 8t .. 8t + 7 of a block) by this; a token with infinities or NaN is zero here
template <bool F32>
struct Token {
    float up, up2;                                         // the scale is their product
    __device__ __forceinline__ Token(uint32_t largest)
    {
        const int k = largest < 0x7F800000u ? scale_of_token<F32>(largest) : 0, h = k / 2;
        up = largest < 0x7F800000u ? __int_as_float((127 + h) << 23) : 0.f;
        up2 = __int_as_float((127 + k - h) << 23);
    }
};
// sums of a token back to its units
template <bool F32>
__device__ __forceinline__ float scaled_back(float v, uint32_t largest)
{
    const int k = CODES<F32> - scale_of_token<F32>(largest), h = k / 2;
    return v * __int_as_float((127 + h) << 23) * __int_as_float((127 + k - h) << 23);
}
template <bool F32>
__device__ __forceinline__ void load_columns(const void *at, bool has, float (&x)[8])
{
    if constexpr (F32) {
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f), w = v;
        if (has) { v = __ldg((const float4 *)at); w = __ldg((const float4 *)at + 1); }
        x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w; x[4] = w.x; x[5] = w.y; x[6] = w.z; x[7] = w.w;
    } else {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (has) v = __ldg((const uint4 *)at);
        x[0] = od_bf16_lo(v.x); x[1] = od_bf16_hi(v.x); x[2] = od_bf16_lo(v.y); x[3] = od_bf16_hi(v.y);
        x[4] = od_bf16_lo(v.z); x[5] = od_bf16_hi(v.z); x[6] = od_bf16_lo(v.w); x[7] = od_bf16_hi(v.w);
    }
}
// and the words of a lane's fragments
template <int P>
__device__ __forceinline__ void cut_columns(float (&x)[8], const Token<P == 3> &k, uint32_t (&b)[P][4])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x[i] *= k.up;
        x[i] = k.up == 0.f ? 0.f : x[i] * k.up2;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float f = P == 1 && i & 1 ? 0.0625f : 1.f;   // (meets 16 u)
        uint32_t c[P];
        pieces<P>(x[i] * f, x[i + 4] * f, c);
#pragma unroll
        for (int p = 0; p < P; ++p) b[p][i] = c[p];
    }
}

// one result as it is defined: of tokens that hold an infinity or NaN
template <bool F32>
__device__ __noinline__ float one_logit(const Q4Args &A, int n, int v, int G)
{
    float total = 0.f;
    for (int h = 0; h < A.H; h += G) {
        float sum = 0.f;
        for (int i = h; i < h + G; ++i) {
            const float x = F32 ? ((const float *)A.in)[(size_t)n * A.in_stride + i]
                                : __uint_as_float((uint32_t)((const unsigned short *)A.in)[(size_t)n * A.in_stride + i] << 16);
            sum += x * (float)((A.codes[((size_t)v * A.H + i) / 2] >> (i & 1) * 4 & 15) - 8);
        }
        total += __uint_as_float((uint32_t)A.scales[((size_t)v * A.H + h) / G] << 16) * sum;
    }
    return total;
}

template <int P, int NT, int GB, bool XS, int RING>
__global__ void __launch_bounds__(F_THREADS, 1) od_q4_kernel(const Q4Args A)
{
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ uint32_t largest_of[8 * NT];                // bits of the tokens' largest magnitudes
    constexpr bool F32 = P == 3;
    constexpr int IN_BYTES = F32 ? 4 : 2;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0);    // (known to be the same in the warp's lanes)
    const int H = A.H, V = A.V, blocks = H / 32, stages = (blocks + WIDE - 1) / WIDE, n_groups = blocks / GB;
    const int n0 = blockIdx.y * (8 * NT);
    // k_split warps to the same rows, each a share of the stages
    const int ks = A.k_split, sub = warp % ks, groups = F_WARPS / ks;
    const int first = stages * sub / ks, last = stages * (sub + 1) / ks;
    const int units = (V + ROWS - 1) / ROWS, step = gridDim.x * groups, begin = blockIdx.x + warp / ks * gridDim.x;
    unsigned char *const mine = smem + warp * (RING * WIDE_STAGE);
    const size_t row_bytes = (size_t)H / 2;

    // fetching: this lane copies pieces lane % 4 and 4 + lane % 4 of rows lane / 4 and 8 + lane / 4
    int fu = begin, fs = first, slot_f = 0;
    const uint32_t put = (uint32_t)__cvta_generic_to_shared(mine) + (lane >> 2) * 128 + ((t ^ (lane >> 2)) << 4);
    const uint8_t *f0 = nullptr, *f1 = nullptr;
    auto fetch = [&]() {
        if (fu < units) {
            if (fs == first) {
                const int r = fu * ROWS + (lane >> 2);
                f0 = A.codes + min(r, V - 1) * row_bytes + first * (16 * WIDE) + t * 16;
                f1 = A.codes + min(r + 8, V - 1) * row_bytes + first * (16 * WIDE) + t * 16;
            }
            const uint32_t to = put + slot_f;
            if (fs * WIDE + t < blocks) { cp16(to, f0); cp16(to + 8 * 128, f1); }
            if (fs * WIDE + 4 + t < blocks) { cp16(to ^ 64, f0 + 64); cp16((to ^ 64) + 8 * 128, f1 + 64); }
            f0 += 16 * WIDE; f1 += 16 * WIDE;
            if (++fs == last) { fs = first; fu += step; }
        }
        cp_commit();
        slot_f = slot_f + WIDE_STAGE == RING * WIDE_STAGE ? 0 : slot_f + WIDE_STAGE;
    };
#pragma unroll
    for (int i = 0; i < RING - 1; ++i) fetch();

    // [group][8 tokens to a part]: what the group's sums begin at; [block of 32 columns][part][piece][lane]: the fragments
    float *const starts = (float *)(smem + F_WARPS * RING * WIDE_STAGE);
    unsigned char *const inputs = (unsigned char *)(starts + (F32 ? 0 : n_groups * 8 * NT));
    auto prepare = [&](bool all_usual) {
        for (int i = warp; i < n_groups * NT; i += F_WARPS) {
            const int q = i % NT, n = n0 + q * 8 + g;
            const Token<F32> k(all_usual ? 127u << 23 : largest_of[q * 8 + g]);
            float start = 0.f;
            uint32_t m = 0;
#pragma unroll
            for (int j = 0; j < GB; ++j) {
                const int blk = i / NT * GB + j;
                float x[8];
                load_columns<F32>((const char *)A.in + ((int64_t)n * A.in_stride + blk * 32 + t * 8) * IN_BYTES, n < A.N, x);
                if (all_usual)
#pragma unroll
                    for (int c = 0; c < 8; ++c) m = max(m, __float_as_uint(x[c]) & 0x7FFFFFFFu);
                uint32_t b[P][4];
                cut_columns<P>(x, k, b);
                if (!F32)
#pragma unroll
                    for (int c = 0; c < 8; ++c) start = fmaf(x[c], -0x1p-126f * 0.0625f, start);   // -8 times 2^-133
                if constexpr (XS)
#pragma unroll
                    for (int p = 0; p < P; ++p) ((uint4 *)inputs)[((blk * NT + q) * P + p) * 32 + lane] = make_uint4(b[p][0], b[p][1], b[p][2], b[p][3]);
            }
            if (!F32) {
                start += __shfl_xor_sync(0xFFFFFFFFu, start, 1);
                start += __shfl_xor_sync(0xFFFFFFFFu, start, 2);
                if (t == 0) starts[i * 8 + g] = start;
            }
            if (all_usual) {
                m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
                m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
                if (t == 0) atomicMax(&largest_of[q * 8 + g], m);
            }
        }
    };
    if (threadIdx.x < 8 * NT) largest_of[threadIdx.x] = 0;
    __syncthreads();
    prepare(true);
    // (a token of zeros is as good with any scale)
    __syncthreads();
    if (__syncthreads_or(threadIdx.x < 8 * NT && largest_of[threadIdx.x] != 0 && !usual(largest_of[threadIdx.x]))) prepare(false);
    auto largest = [&](int n) { return largest_of[n]; };
    const char *x_at[NT];
    if constexpr (!XS)
#pragma unroll
        for (int q = 0; q < NT; ++q)
            x_at[q] = (const char *)A.in + ((int64_t)min(n0 + q * 8 + g, A.N - 1) * A.in_stride + t * 8) * IN_BYTES;

    const uint32_t get = (uint32_t)__cvta_generic_to_shared(mine) + g * 128 + (g << 4) + t * 4;   // this lane's first word of the first slot
    int slot = 0;
    Scales<GB> next0[2], next1[2];
    const unsigned short *e0, *e1;                         // the next stage's scales
    auto aim_scales = [&](int u) {
        const int r = u * ROWS + g;
        e0 = A.scales + (size_t)min(r, V - 1) * n_groups + first * (WIDE / GB);
        e1 = A.scales + (size_t)min(r + 8, V - 1) * n_groups + first * (WIDE / GB);
    };
    auto load_scales = [&](int s) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int left = n_groups - (s * WIDE + 4 * i) / GB;
            if (i == 0 || left > 0) {
                next0[i].load(e0 + 4 / GB * i, left, A.wide_scales);
                next1[i].load(e1 + 4 / GB * i, left, A.wide_scales);
            }
        }
        e0 += WIDE / GB; e1 += WIDE / GB;
    };
    int u = begin;
    if (u < units) { aim_scales(u); load_scales(first); }
    float4 *const parts = (float4 *)(inputs + (XS ? H * 16 * NT * P : 0)) + lane;      // [warp][8 tokens][lane]
    __syncthreads();
    for (; u < units; u += step) {
        float total[NT][4] = {};
        uint32_t xs = (uint32_t)__cvta_generic_to_shared(inputs) + lane * 16 + first * (WIDE * NT * P * 512);
        const float2 *begin_at = (const float2 *)starts + first * (WIDE / GB) * NT * 4 + t;
        for (int s = first; s < last; ++s) {
            const Scales<GB> s0[2] = {next0[0], next0[1]}, s1[2] = {next1[0], next1[1]};
            if (s + 1 < last) load_scales(s + 1);
            else if (u + step < units) { aim_scales(u + step); load_scales(first); }
            cp_wait<RING - 2>();
            __syncwarp();
            fetch();
            // (of pieces the small ones in a chain of their own: the tensor pipe cuts what it adds to 2^-23 of the largest)
            float sum[NT][4], small[NT][4];
            auto block = [&](int j) {
                uint32_t b[NT][P][4];
#pragma unroll
                for (int q = 0; q < NT; ++q) {
                    if constexpr (XS) {
#pragma unroll
                        for (int p = 0; p < P; ++p) {
                            const uint4 v = lds128(xs + ((j * NT + q) * P + p) * 512);
                            b[q][p][0] = v.x; b[q][p][1] = v.y; b[q][p][2] = v.z; b[q][p][3] = v.w;
                        }
                    } else {
                        float x[8];
                        load_columns<F32>(x_at[q] + (size_t)(s * WIDE + j) * 32 * IN_BYTES, n0 + q * 8 + g < A.N, x);
                        cut_columns<P>(x, Token<F32>(largest(q * 8 + g)), b[q]);
                    }
                    if (j % GB == 0) {
                        const float2 v = F32 ? make_float2(0.f, 0.f) : begin_at[(j / GB * NT + q) * 4];
                        sum[q][0] = sum[q][2] = v.x; sum[q][1] = sum[q][3] = v.y;
                        if (P > 1) small[q][0] = small[q][1] = small[q][2] = small[q][3] = 0.f;
                    }
                }
                const uint32_t w0 = lds32((get + slot) ^ (j << 4)), w1 = lds32(((get + slot) ^ (j << 4)) + 8 * 128);
                const uint32_t v0 = w0 >> 8, v1 = w1 >> 8, k = A.bf16_128;
                uint32_t a0[4] = {w0 & CODE, w1 & CODE, w0 & CODE16, w1 & CODE16};
                uint32_t a1[4] = {v0 & CODE, v1 & CODE, v0 & CODE16, v1 & CODE16};
                if (F32) {
                    a0[0] = unpack<0>(w0, k); a0[1] = unpack<0>(w1, k); a0[2] = unpack<1>(w0, k); a0[3] = unpack<1>(w1, k);
                    a1[0] = unpack<2>(w0, k); a1[1] = unpack<2>(w1, k); a1[2] = unpack<3>(w0, k); a1[3] = unpack<3>(w1, k);
                }
#pragma unroll
                for (int q = 0; q < NT; ++q) {
#pragma unroll
                    for (int p = 0; p < P; ++p) {
                        mma(p == 0 ? sum[q] : small[q], a0, b[q][p][0], b[q][p][1]);
                        mma(p == 0 ? sum[q] : small[q], a1, b[q][p][2], b[q][p][3]);
                    }
                    if (P > 1 && j % GB == GB - 1)
#pragma unroll
                        for (int k = 0; k < 4; ++k) sum[q][k] += small[q][k];
                    if (j % GB == GB - 1) {
                        const float c0 = s0[j / 4].get(j % 4 / GB), c1 = s1[j / 4].get(j % 4 / GB);
                        total[q][0] = fmaf(c0, sum[q][0], total[q][0]); total[q][1] = fmaf(c0, sum[q][1], total[q][1]);
                        total[q][2] = fmaf(c1, sum[q][2], total[q][2]); total[q][3] = fmaf(c1, sum[q][3], total[q][3]);
                    }
                }
            };
            if (s * WIDE + WIDE <= blocks) {
#pragma unroll
                for (int j = 0; j < WIDE; ++j) block(j);
            } else {
#pragma unroll
                for (int j = 0; j < WIDE - 1; ++j)
                    if (s * WIDE + j < blocks) block(j);
            }
            xs += WIDE * NT * P * 512;
            begin_at += WIDE / GB * NT * 4;
            slot = slot + WIDE_STAGE == RING * WIDE_STAGE ? 0 : slot + WIDE_STAGE;
        }
        if (ks > 1) {
            if (sub > 0) {
#pragma unroll
                for (int q = 0; q < NT; ++q)
                    parts[(warp * NT + q) * 32] = make_float4(total[q][0], total[q][1], total[q][2], total[q][3]);
            }
            asm volatile("bar.sync %0, %1;" ::"r"(1 + warp / ks), "r"(32 * ks) : "memory");
            if (sub == 0) {
                for (int w = 1; w < ks; ++w)
#pragma unroll
                    for (int q = 0; q < NT; ++q) {
                        const float4 v = parts[((warp + w) * NT + q) * 32];
                        total[q][0] += v.x; total[q][1] += v.y; total[q][2] += v.z; total[q][3] += v.w;
                    }
            }
            asm volatile("bar.sync %0, %1;" ::"r"(1 + warp / ks), "r"(32 * ks) : "memory");
            if (sub > 0) continue;
        }
#pragma unroll
        for (int q = 0; q < NT; ++q)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int m = q * 8 + 2 * t + (k & 1), n = n0 + m, v = u * ROWS + g + (k >> 1) * 8;
                if (n >= A.N || v >= V) continue;
                const uint32_t l = largest(m);
                store(A, n, v, l < 0x7F800000u ? scaled_back<F32>(total[q][k], l) : one_logit<F32>(A, n, v, 32 * GB));
            }
    }
    cp_wait<0>();
}

// ---- backward: 128 columns to a warp, every so many-th 32 rows ----------------------------------
//
// Rows are summed over: two of them are the pair of an operand, four columns in a row are a half word. The tokens' side is
// made anew for each group: gradient times scale, in pieces. The codes are brought to u - 8 here, as ordinary bf16 numbers
// (two shifts or masks more and a subtraction for two codes: 44 us for 41 with eight positions). Gradients have mostly one sign (a softmax but
// for one large entry), and where sums of them with 0 to 15 were taken the tensor pipe's cuts were 1e-5 of the result; with
// numbers below bf16's normal ones, which the pipe lines up as if their leading bits were there, 1e-6; so they are 4e-7, and
// of fp32 results 2e-7 (EXACT below), where plain fp32 sums are 5e-7 off.
// Warps side by side share rows (a block reads up to 256 bytes in a row). Those on the same columns are summed at the end,
// and so are the blocks on the same columns, both in a fixed order: through a cluster's shared memory, or, as clusters do not
// fill the device, by a second kernel from the context's scratch. That takes 4 us, a cluster's barriers one.
constexpr int G_ROWS = 32;                                 // of a stage
constexpr int G_CODES = G_ROWS * COLS / 2;                 // bytes

__device__ __forceinline__ void cp16_part(uint32_t to, const void *from, int bytes)    // the rest is zeros
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}

template <int P, int NT> constexpr int g_stage = G_CODES + 8 * NT * G_ROWS * (P == 3 ? 4 : 2);
template <int P, int NT, int GB> constexpr int g_warp = G_RING * g_stage<P, NT> + 2 * G_ROWS * (4 / GB) * 4;

// EXACT, for fp32 results: the tensor pipe cuts what it adds to its accumulators (to 2^-23 of the largest), so what it adds up in a
// stage begins at zero and is then added to the sums in fp32 as such, which rounds (128256 x 1824, 28 positions: 2e-6 of the
// result otherwise, where plain fp32 sums are 7e-7 off). For bf16 results it is left out: 20 % of the time with 24 positions, for cuts that add up
// to 3e-5 of the result at most (152064 x 16384, 24 or 32 positions: all rows to eight warps), where its rounding is 2e-3.
template <int P, int NT, int GB, bool EXACT, int WARPS>
__global__ void __launch_bounds__(32 * WARPS, 1) od_q4_grad_kernel(const Q4Args A)
{
    extern __shared__ __align__(128) unsigned char smem[];
    constexpr bool F32 = P == 3;
    constexpr int THREADS = 32 * WARPS;
    constexpr int ESZ = F32 ? 4 : 2, GROUPS = 4 / GB, PIECES = G_ROWS * ESZ / 16, STAGE = g_stage<P, NT>;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0);
    const int H = A.H, V = A.V, cw = A.col_warps, split = A.split;
    const int rank = blockIdx.x % split, tile = blockIdx.x / split;
    const int col = (tile * cw + warp % cw) * COLS, here = max(0, min(4, (H - col) / 32)), n_groups = H / (32 * GB);
    const int slabs = split * (WARPS / cw), slab = rank * (WARPS / cw) + warp / cw;
    const int steps = here > 0 ? (V - 1) / G_ROWS + 1 : 0, n0 = A.first_token;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * g_warp<P, NT, GB>;
    float *const scale_of = (float *)(smem + warp * g_warp<P, NT, GB> + G_RING * STAGE);   // [2][row][group]
    const size_t row_bytes = (size_t)H / 2;

    // fetching: this lane copies piece lane % 4 of rows lane / 4 + 8 i, and pieces of the tokens' rows
    int fs = slab, slot_f = 0;
    const uint32_t put = ring + (lane >> 2) * 64 + ((t ^ (lane >> 4)) << 4);
    const uint8_t *const from = A.codes + (size_t)col / 2 + t * 16;
    const uint8_t *code_at = from + (size_t)(slab * G_ROWS + (lane >> 2)) * row_bytes;
    const size_t code_step = (size_t)slabs * G_ROWS * row_bytes, eight = 8 * row_bytes;
    constexpr int ITEMS = 8 * NT * PIECES / 32;            // pieces of tokens of a lane: of tokens 32 / PIECES apart
    const int n_at = lane / PIECES, c_at = lane % PIECES;
    const uint32_t put_d = ring + G_CODES + n_at * (PIECES * 16) + ((c_at ^ (F32 ? (n_at & 1) << 2 : (n_at >> 1 & 1) << 1)) << 4);
    const char *d_at = (const char *)A.in + ((int64_t)(n0 + n_at) * A.in_stride + slab * G_ROWS + c_at * (16 / ESZ)) * ESZ;
    const int64_t d_step = (int64_t)slabs * G_ROWS * ESZ, d_token = 32 / PIECES * A.in_stride * ESZ;
    const int whole = V / G_ROWS;                          // stages of no row behind the last
    int size[ITEMS];                                       // (nothing is read of a token that there is not: zeros)
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) size[i] = n0 + n_at + i * (32 / PIECES) < A.N ? 16 : 0;
    auto fetch = [&]() {
        if (fs < steps) {
            const uint32_t to = put + slot_f, to_d = put_d + slot_f;
            if (fs < whole) {
                if (t < here) {                            // (rows 8 on: the piece's place has another bit)
                    cp16(to, code_at);
                    cp16((to + 8 * 64) ^ 32, code_at + eight);
                    cp16(to + 16 * 64, code_at + 2 * eight);
                    cp16((to + 24 * 64) ^ 32, code_at + 3 * eight);
                }
#pragma unroll
                for (int i = 0; i < ITEMS; ++i) cp16_part(to_d + i * 512, size[i] ? d_at + i * d_token : A.in, size[i]);
            } else {
                const int bytes = max(0, min(16 / ESZ, V - (fs * G_ROWS + c_at * (16 / ESZ)))) * ESZ;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (t < here) cp16((to + i * 8 * 64) ^ (i & 1 ? 32 : 0), from + (size_t)min(fs * G_ROWS + (lane >> 2) + 8 * i, V - 1) * row_bytes);
#pragma unroll
                for (int i = 0; i < ITEMS; ++i) cp16_part(to_d + i * 512, size[i] && bytes ? d_at + i * d_token : A.in, min(size[i], bytes));
            }
            fs += slabs;
            code_at += code_step;
            d_at += d_step;
        }
        cp_commit();
        slot_f = slot_f + STAGE == G_RING * STAGE ? 0 : slot_f + STAGE;
    };
#pragma unroll
    for (int i = 0; i < G_RING - 1; ++i) fetch();

    // the scales of row `lane` of a stage
    Scales<GB> raw;
    auto load_scales = [&](int s) {
        const int r = s * G_ROWS + lane, i = col / (32 * GB);
        if (r < V) raw.load(A.scales + (size_t)r * n_groups + i, n_groups - i, A.wide_scales);
        else raw.clear();                                  // (zero times a gradient of zero)
    };
    // A lane's words: rows 4t .. 4t + 3; of a group of 64 or more word g of two blocks, of one of 32 a half of word g / 2 of
    // a block. (Pieces of these rows are placed by t.)
    constexpr bool PAIRS = GB > 1;
    const uint32_t get = ring + 4 * t * 64 + (PAIRS ? g & 3 : g >> 1) * 4, pick = g & 1 ? HIGH : LOW;
    const uint32_t get_d = ring + G_CODES + g * (PIECES * 16) + (F32 ? (t ^ (g & 1) << 2) << 4 : (g >> 1 & 1) << 5 | t << 3);
    float acc[8][NT][4] = {};
    int slot = 0, flip = 0;
    if (slab < steps) load_scales(slab);
    for (int s = slab; s < steps; s += slabs) {
#pragma unroll
        for (int i = 0; i < GROUPS; ++i) scale_of[(flip * G_ROWS + lane) * GROUPS + i] = raw.get(i);
        if (s + slabs < steps) load_scales(s + slabs);
        cp_wait<G_RING - 2>();
        __syncwarp();
        fetch();
        // of eight tokens both halves of the rows side by side, for what can run at the same time; of more registers lack
        constexpr int SIDE = NT == 1 ? 2 : 1;
#pragma unroll
        for (int base = 0; base < 2; base += SIDE) {
            float d[SIDE][NT][4], e[SIDE][4][GROUPS];
#pragma unroll
            for (int half = 0; half < SIDE; ++half) {
#pragma unroll
                for (int q = 0; q < NT; ++q) {
                    const uint32_t at = get_d + slot + q * 8 * (PIECES * 16);
                    if constexpr (F32) {
                        const uint4 v = lds128(at ^ ((base + half) << 6));
                        d[half][q][0] = __uint_as_float(v.x); d[half][q][1] = __uint_as_float(v.y);
                        d[half][q][2] = __uint_as_float(v.z); d[half][q][3] = __uint_as_float(v.w);
                    } else {
                        const uint2 v = *(const uint2 *)__cvta_shared_to_generic(at ^ ((base + half) << 5));
                        d[half][q][0] = od_bf16_lo(v.x); d[half][q][1] = od_bf16_hi(v.x);
                        d[half][q][2] = od_bf16_lo(v.y); d[half][q][3] = od_bf16_hi(v.y);
                    }
                }
                float flat[4 * GROUPS];                        // [row][group]
#pragma unroll
                for (int k = 0; k < GROUPS; ++k)
                    *(float4 *)(flat + 4 * k) = *(const float4 *)(scale_of + (flip * G_ROWS + (base + half) * 16 + 4 * t) * GROUPS + 4 * k);
#pragma unroll
                for (int k = 0; k < 4 * GROUPS; ++k) e[half][k / GROUPS][k % GROUPS] = flat[k];
            }
#pragma unroll
            for (int i = 0; i < GROUPS; ++i) {
                if (i * GB >= here) break;
                uint64_t z[SIDE][NT][2];                          // pairs of rows
                float m = 0.f;
#pragma unroll
                for (int half = 0; half < SIDE; ++half)
#pragma unroll
                    for (int q = 0; q < NT; ++q)
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            z[half][q][k] = f2_mul(f2_pack(d[half][q][2 * k], d[half][q][2 * k + 1]), f2_pack(e[half][2 * k][i], e[half][2 * k + 1][i]));
                            float lo, hi;
                            f2_unpack(z[half][q][k], lo, hi);
                            m = fmaxf(fmaxf(m, fabsf(lo)), fabsf(hi));
                        }
                const bool guard = __any_sync(0xFFFFFFFFu, m == INFINITY);
                uint32_t b[SIDE][NT][2][P];
#pragma unroll
                for (int half = 0; half < SIDE; ++half)
#pragma unroll
                    for (int q = 0; q < NT; ++q)
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            uint64_t rest = z[half][q][k];
#pragma unroll
                            for (int p = 0; p < P; ++p) {
                                float lo, hi;
                                f2_unpack(rest, lo, hi);
                                b[half][q][k][p] = halves(__float_as_uint(lo), __float_as_uint(hi), HIGH);
                                if (p + 1 < P)
                                    rest = f2_fma(f2_pack(__uint_as_float(__float_as_uint(lo) & 0xFFFF0000u), __uint_as_float(__float_as_uint(hi) & 0xFFFF0000u)),
                                                  f2_pack(-1.f, -1.f), rest);
                                if (p + 1 < P && guard) {  // (all of an infinity is in its first piece)
                                    float u, v;
                                    f2_unpack(rest, u, v);
                                    rest = f2_pack(fabsf(lo) == INFINITY ? 0.f : u, fabsf(hi) == INFINITY ? 0.f : v);
                                }
                            }
                        }
                // four codes of a lane in each of four rows, of both halves: two columns of two sums
                auto product = [&](const uint32_t (&w01)[SIDE], const uint32_t (&w23)[SIDE], int c) {
                    const uint32_t k = A.bf16_128;
#pragma unroll
                    for (int upper = 0; upper < 2; ++upper) {
                        float sum[NT][4];
#pragma unroll
                        for (int half = 0; half < SIDE; ++half) {
                            uint32_t a[4];
                            if (upper) { a[0] = unpack<2>(w01[half], k); a[1] = unpack<3>(w01[half], k); a[2] = unpack<2>(w23[half], k); a[3] = unpack<3>(w23[half], k); }
                            else { a[0] = unpack<0>(w01[half], k); a[1] = unpack<1>(w01[half], k); a[2] = unpack<0>(w23[half], k); a[3] = unpack<1>(w23[half], k); }
#pragma unroll
                            for (int p = 0; p < P; ++p)
#pragma unroll
                                for (int q = 0; q < NT; ++q) {
                                    if (!EXACT) mma(acc[c + upper][q], a, b[half][q][0][p], b[half][q][1][p]);
                                    else if (half == 0 && p == 0) mma_of(sum[q], a, b[half][q][0][p], b[half][q][1][p]);
                                    else mma(sum[q], a, b[half][q][0][p], b[half][q][1][p]);
                                }
                        }
                        if (EXACT)
#pragma unroll
                            for (int q = 0; q < NT; ++q)
#pragma unroll
                                for (int e = 0; e < 4; e += 2) {
                                    float (&to)[4] = acc[c + upper][q];
                                    f2_unpack(f2_add(f2_pack(to[e], to[e + 1]), f2_pack(sum[q][e], sum[q][e + 1])), to[e], to[e + 1]);
                                }
                    }
                };
#pragma unroll
                for (int j = i * GB; j < (i + 1) * GB; j += PAIRS ? 2 : 1) {
                    uint32_t low01[SIDE], low23[SIDE], high01[SIDE], high23[SIDE];
#pragma unroll
                    for (int half = 0; half < SIDE; ++half) {
                        const uint32_t at = get + slot + (base + half) * 16 * 64 + ((PAIRS ? (j + (g >> 2)) ^ t : j ^ t) << 4);
                        const uint32_t w0 = lds32(at), w1 = lds32(at + 64), w2 = lds32(at + 128), w3 = lds32(at + 192);
                        low01[half] = halves(w0, w1, PAIRS ? LOW : pick); low23[half] = halves(w2, w3, PAIRS ? LOW : pick);
                        if (PAIRS) { high01[half] = halves(w0, w1, HIGH); high23[half] = halves(w2, w3, HIGH); }
                    }
                    product(low01, low23, 2 * j);
                    if constexpr (PAIRS) product(high01, high23, 2 * j + 2);
                }
            }
        }
        slot = slot + STAGE == G_RING * STAGE ? 0 : slot + STAGE;
        flip ^= 1;
    }
    cp_wait<0>();
    __syncthreads();                                       // the rings are free

    // [warp][token][column]; the warps on the same columns are summed into the first of them
    constexpr int PART = 8 * NT * COLS;                    // numbers of a warp
    float *const part = (float *)smem;
#pragma unroll
    for (int c = 0; c < 8; ++c)
#pragma unroll
        for (int q = 0; q < NT; ++q)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int column = PAIRS ? c / 4 * 64 + 8 * g + c % 4 * 2 : c / 2 * 32 + 4 * g + c % 2 * 2;
                *(float2 *)(part + warp * PART + (q * 8 + 2 * t + k) * COLS + column) = make_float2(acc[c][q][k], acc[c][q][k + 2]);
            }
    __syncthreads();
    for (int i = threadIdx.x; i < cw * PART; i += THREADS) {
        float v = part[i];
        for (int w = cw; w < WARPS; w += cw) v += part[w * PART + i];
        const int n = n0 + i % PART / COLS, h = (tile * cw + i / PART) * COLS + i % COLS;
        if (A.cluster) part[i] = v;
        else if (split > 1) A.parts[(size_t)blockIdx.x * (cw * PART) + i] = v;
        else if (n < A.N && h < H) store(A, n, h, v);
    }
    if (!A.cluster) return;
    __syncthreads();
    od_cluster_arrive(); od_cluster_wait();
    // each block has a share of the cluster's columns
    for (int i = cw * PART * rank / split + threadIdx.x; i < cw * PART * (rank + 1) / split; i += THREADS) {
        const int n = n0 + i % PART / COLS, h = (tile * cw + i / PART) * COLS + i % COLS;
        float v = 0.f;
#pragma unroll 4
        for (int r = 0; r < split; ++r) v += load_cluster(part + i, r);
        if (n < A.N && h < H) store(A, n, h, v);
    }
    od_cluster_arrive(); od_cluster_wait();                // (nobody leaves while another reads)
}

// The blocks on the same columns: [tile][split][warp side by side][token][column]. A block of threads has 32 numbers,
// each by eight threads that have every eighth part, and adds theirs in order.
constexpr int JOIN = 8;
__global__ void __launch_bounds__(32 * JOIN) od_q4_join_kernel(const Q4Args A, int tokens)
{
    __shared__ float sums[JOIN][32];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int h = blockIdx.x * 32 + threadIdx.x, n = blockIdx.y;               // (H is a multiple of 32)
    const int size = A.col_warps * tokens * COLS, tile = h / (A.col_warps * COLS);
    const float *p = A.parts + (size_t)tile * A.split * size + (h / COLS % A.col_warps * tokens + n) * COLS + h % COLS;
    float v = 0.f;
#pragma unroll 8
    for (int k = threadIdx.y; k < A.split; k += JOIN) v += p[(size_t)k * size];
    sums[threadIdx.y][threadIdx.x] = v;
    __syncthreads();
    if (threadIdx.y > 0) return;
#pragma unroll
    for (int k = 1; k < JOIN; ++k) v += sums[k][threadIdx.x];
    store(A, A.first_token + n, h, v);
}

template <int NT> constexpr int part_bytes = F_WARPS * NT * 512;
template <int P, int NT, int GB, int WARPS> constexpr int grad_bytes = WARPS * (g_warp<P, NT, GB> > 8 * NT * COLS * 4 ? g_warp<P, NT, GB> : 8 * NT * COLS * 4);

typedef void (*Kernel)(Q4Args);
struct Variant { Kernel kernel; int smem, tokens, threads; };

// Forward: 8, 16 or 32 tokens to a block, the most (and no more than there are) whose inputs fit into shared memory
// beside the rings; where those of 8 do not, they stay in global memory. Backward: 8, 16, 24 or 32.
// The ring of a warp has three stages, or two where the tokens' fragments fit with two only (16 tokens of 4096 columns,
// 32000 rows: 24 us, and 34 eight at a time).
constexpr int SMEM_MOST = 226 * 1024;                      // (and a little of fixed size)
template <int P, int NT, int GB, bool XS>
Variant forward_kernel(int32_t H)
{
    const int rest = part_bytes<NT> + (P == 3 ? 0 : H / GB * NT) + (XS ? H * 16 * NT * P : 0), stage = F_WARPS * WIDE_STAGE;
    if (!XS || rest + 3 * stage <= SMEM_MOST) return {od_q4_kernel<P, NT, GB, XS, 3>, rest + 3 * stage, 8 * NT, F_THREADS};
    return {od_q4_kernel<P, NT, GB, XS, XS ? 2 : 3>, rest + 2 * stage, 8 * NT, F_THREADS};
}
template <int GB>
Variant forward_of(bool f32, int N, int32_t H)
{
    Variant v = f32 ? (N > 8 ? forward_kernel<3, 2, GB, true>(H) : forward_kernel<3, 1, GB, true>(H)) : N > 16 ? forward_kernel<1, 4, GB, true>(H)
              : N > 8 ? forward_kernel<1, 2, GB, true>(H) : forward_kernel<1, 1, GB, true>(H);
    if (v.smem > SMEM_MOST && !f32 && N > 16) v = forward_kernel<1, 2, GB, true>(H);
    if (v.smem > SMEM_MOST) v = f32 ? forward_kernel<3, 1, GB, true>(H) : forward_kernel<1, 1, GB, true>(H);
    if (v.smem <= SMEM_MOST) return v;
    return f32 ? forward_kernel<3, 1, GB, false>(H) : forward_kernel<1, 1, GB, false>(H);
}
template <int P, int NT, int GB, bool EXACT>
Variant backward_for()
{
    constexpr int W = G_WARPS[NT];
    return {od_q4_grad_kernel<P, NT, GB, EXACT, W>, grad_bytes<P, NT, GB, W>, 8 * NT, 32 * W};
}
template <int P, int GB, bool EXACT>
Variant backward_kernel(int N)
{
    return N <= 8 ? backward_for<P, 1, GB, EXACT>() : N <= 16 ? backward_for<P, 2, GB, EXACT>()
         : N <= 24 ? backward_for<P, 3, GB, EXACT>() : backward_for<P, 4, GB, EXACT>();
}
template <int GB>
Variant backward_of(bool f32, bool exact, int N)
{
    if (exact) return f32 ? backward_kernel<3, GB, true>(N) : backward_kernel<2, GB, true>(N);
    return f32 ? backward_kernel<3, GB, false>(N) : backward_kernel<2, GB, false>(N);
}
Variant variant(bool backward, int32_t G, bool f32, bool out_f32, int N, int32_t H)
{
    if (backward) return G == 32 ? backward_of<1>(f32, out_f32, N) : G == 64 ? backward_of<2>(f32, out_f32, N) : backward_of<4>(f32, out_f32, N);
    return G == 32 ? forward_of<1>(f32, N, H) : G == 64 ? forward_of<2>(f32, N, H) : forward_of<4>(f32, N, H);
}

template <typename K, typename... A>
cudaError_t launch(K kernel, dim3 grid, dim3 threads, int smem, int cluster, bool pdl, cudaStream_t s, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid; cfg.blockDim = threads;
    cfg.dynamicSmemBytes = smem; cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)cluster; attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = pdl ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace

// What a kernel needs is set when a context launches it for the first time, and what the gradient asks of the device when it is
// called first: for all 84 kernels it took 23 ms in every process's first od_create, of those too that have no such layer. (Neither
// allocates or waits: also while a stream is captured. Two threads may call at once.)
namespace {

std::mutex &first_calls() { static std::mutex m; return m; }

bool limits_set(const od_ctx *c, const void *kernel)
{
    for (const void *const &k : c->q4_kernels) {
        const void *const known = __atomic_load_n(&k, __ATOMIC_ACQUIRE);
        if (known == kernel) return true;
        if (!known) break;
    }
    return false;
}

cudaError_t set_limits(od_ctx *c, const void *kernel, bool backward)
{
    if (limits_set(c, kernel)) return cudaSuccess;
    std::lock_guard<std::mutex> lock(first_calls());
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_MOST);
    if (e == cudaSuccess && backward) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    for (const void *&k : c->q4_kernels) {
        if (k == kernel) break;
        if (k) continue;
        __atomic_store_n(&k, kernel, __ATOMIC_RELEASE);
        break;
    }
    return cudaSuccess;
}

// q4_clusters[n]: clusters of n blocks of the gradient that are resident at a time, by the variant with the most shared memory
// (each fills a multiprocessor)
cudaError_t ask_for_clusters(od_ctx *c)
{
    if (__atomic_load_n(&c->q4_clusters_known, __ATOMIC_ACQUIRE)) return cudaSuccess;
    const Variant v = variant(true, 32, true, true, 8, 128);
    const cudaError_t e = set_limits(c, (const void *)v.kernel, true);
    if (e != cudaSuccess) return e;
    std::lock_guard<std::mutex> lock(first_calls());
    if (c->q4_clusters_known) return cudaSuccess;
    for (int n = 0; n <= OD_Q4_MAX_SPLIT; ++n) {
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = (unsigned)n; attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cfg.gridDim = dim3((unsigned)n); cfg.blockDim = dim3(v.threads); cfg.dynamicSmemBytes = v.smem;
        cfg.attrs = attr; cfg.numAttrs = 1;
        int here = 0;
        if (n < 2 || cudaOccupancyMaxActiveClusters(&here, (const void *)v.kernel, &cfg) != cudaSuccess) {
            cudaGetLastError();
            here = 0;
        }
        c->q4_clusters[n] = here;
    }
    __atomic_store_n(&c->q4_clusters_known, true, __ATOMIC_RELEASE);
    return cudaSuccess;
}

}  // namespace

cudaError_t od_launch_q4(od_ctx *c, bool backward, int32_t N, int32_t V, int32_t H, int32_t G, const void *a, int32_t a_dtype,
                         int64_t as, const void *codes, const void *scales, void *b, int32_t b_dtype, int64_t bs, cudaStream_t s)
{
    const bool f32 = a_dtype == OD_F32, pdl = c->opt_pdl != 0;
    const int32_t sms = c->sm_count;
    Q4Args args = {a, as, (const uint8_t *)codes, (const unsigned short *)scales, b, bs, N, V, H, f32, b_dtype == OD_F32,
                   H % COLS == 0 && ((uintptr_t)scales & 7u) == 0, 0x43004300u, 1, 1, 1, 0, 0, c->d_q4_parts};
    if (!backward) {
        const Variant v = variant(false, G, f32, false, N, H);
        const cudaError_t ready = set_limits(c, (const void *)v.kernel, false);
        if (ready != cudaSuccess) return ready;
        const int64_t units = ((int64_t)V + ROWS - 1) / ROWS, blocks = units < sms ? units : sms;
        // Warps to the same 16 rows (1, 2, 4), by the time of a warp's turns: its stages, and for the sums to be joined as much as
        // one stage more, or of four warps three. (us, 1 / 2 / 4: 8 tokens through 128256 x 4096 59 / 52 / 57, 2000 x 4096
        // 10.9 / 8.1 / 6.7, 4 through 152064 x 2048 34 / 36 / 43, 8 through 64000 x 1024 12.7 / 12.7 / 16.9.)
        const int64_t each = (units + blocks - 1) / blocks, stages = (H + 32 * WIDE - 1) / (32 * WIDE);
        int64_t best = INT64_MAX;
        for (int32_t ks = 1; ks <= 4 && ks <= stages; ks *= 2) {
            const int64_t cost = (each * ks + F_WARPS - 1) / F_WARPS * ((stages + ks - 1) / ks + ks - 1);
            if (cost < best) { best = cost; args.k_split = ks; }
        }
        return launch(v.kernel, dim3((unsigned)blocks, (unsigned)((N + v.tokens - 1) / v.tokens)), F_THREADS, v.smem, 1, pdl, s, args);
    }
    cudaError_t e = ask_for_clusters(c);
    if (e != cudaSuccess) return e;
    // 32 tokens at a time, then what is left: the scratch is for one time
    for (int32_t n = 0; n < N;) {
        const Variant v = variant(true, G, f32, b_dtype == OD_F32, N - n, H);
        e = set_limits(c, (const void *)v.kernel, true);
        if (e != cudaSuccess) return e;
        // Warps side by side (4, 2, 1), blocks on the same columns (as many as there are multiprocessors for, or a cluster of
        // any size) and how these are joined, by the time that it takes in twentieths of a us, as measured with 16 warps (in proportion to them it chose no better): a stage of a warp 13, and
        // for every eight tokens 13, 6 for each group of its columns but one and 6 if they are fp32; the join 80, a cluster 20.
        // Of equal ones the widest rows.
        const int64_t steps = ((int64_t)V + G_ROWS - 1) / G_ROWS, stage = 13 + v.tokens / 8 * (13 + 6 * (128 / G - 1) + 6 * f32);
        int64_t best = INT64_MAX, blocks = 0;
        const int warps = v.threads / 32;
        auto offer = [&](int32_t cw, int64_t split, int64_t rounds, int64_t join, bool cluster) {
            const int64_t slabs = split * (warps / cw), cost = rounds * ((steps + slabs - 1) / slabs) * stage + join;
            if (cost >= best) return;
            best = cost; blocks = (H + cw * COLS - 1) / (cw * COLS) * split;
            args.col_warps = cw; args.split = (int32_t)split; args.cluster = cluster;
        };
        for (int32_t cw = 4 * 8 / v.tokens; cw >= 1; cw /= 2) {
            const int64_t tiles = (H + cw * COLS - 1) / (cw * COLS), deep = warps / cw, most = (steps + deep - 1) / deep;
            const int64_t split = tiles > sms ? 1 : sms / tiles < most ? sms / tiles : most;
            offer(cw, split, (tiles * split + sms - 1) / sms, split > 1 ? 80 : 0, false);
            for (int32_t k = 2; k <= OD_Q4_MAX_SPLIT && k <= most; ++k)
                if (c->q4_clusters[k] > 0) offer(cw, k, (tiles + c->q4_clusters[k] - 1) / c->q4_clusters[k], 20, true);
        }
        args.first_token = n;
        e = launch(v.kernel, dim3((unsigned)blocks), v.threads, v.smem, args.cluster ? args.split : 1, pdl, s, args);
        if (e == cudaSuccess && args.split > 1 && !args.cluster)
            e = launch(od_q4_join_kernel, dim3((unsigned)(H / 32), (unsigned)(N - n < v.tokens ? N - n : v.tokens)), dim3(32, JOIN), 0, 1, pdl, s, args, v.tokens);
        if (e != cudaSuccess) return e;
        n += v.tokens;
    }
    return cudaSuccess;
}
