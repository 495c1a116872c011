// Scores of tokens from logit rows, and their gradient. For a row x of V logits at temperature T, with
// M = max x, e_j = exp((x_j - M) / T), S = sum e, p = e / S:
//   log probability   ln p_t = (x_t - M) / T - ln S
//   entropy           H = ln S - (1 / S) sum_j e_j (x_j - M) / T
//   alternatives      the n largest logits, equal ones by the lower id
//   gradient          d/dx_j = (1/T) (sum_i g_i [j == id_i] - p_j (G + g_H (ln p_j + H))),  G = sum_i g_i,
//                     i over the given token and the listed alternatives
// Everything is held in fp32. Differences from the running maximum are formed before they are scaled: x T^-1 may
// overflow (a mask of the type's lowest value) or lose the digits that the exponential is made of, x - M does not.
//
// Forward: one pass. A block of 128 or 256 threads (or a cluster of them: one contiguous slice of the row to each) keeps, per
// thread, the maximum, the sum of e and the sum of e (x - M), raised to a new maximum once per four 16-byte loads.
// The alternatives cost next to nothing in that pass: the largest logits of 32 groups of threads are 32 different
// elements, so the n-th largest of them is a bound that at least n elements of the slice reach and few more do. Threads leave
// the maximum of every four loads in shared memory: only loads whose maximum reaches the bound are looked at again (from L2,
// all of them at once), and what reaches the bound is ranked by counting. Where too much reaches it (many equal logits, or many of
// the largest in one thread's elements) each warp goes through its share of the slice again and keeps a sorted list. And where one token has nearly
// all of the mass, what its thread has read is summed again without it.
//
// Backward: elementwise, one read and one write; the given token and the alternatives are written over the dense
// values of their chunk behind a block barrier.
//
// Measured (us; HBM's rate for the bytes): scores of 4608 rows of 152064 bf16 logits with one alternative 242 (213), without
// 226; 96 rows of 128256 with 20 16 (3.8: launch, a row's chain of barriers, its alternatives); gradient of 448 rows of 128256,
// 256 of which count, 32 (27). The large ones are at HBM's rate but for a row's end, the small ones at their chain.
#include <float.h>

#include "od_common.cuh"

namespace {

constexpr int THREADS = 256;                               // (of the scores' blocks also half as many)
constexpr int WARPS = THREADS / 32;
constexpr int U = 4;                                       // 16-byte loads of a thread in flight
constexpr int MAX_SPLIT = 8;                               // blocks of a row (a portable cluster)
constexpr int CAP = 512;                                   // candidates that are ranked by counting
constexpr int GRAD_TURNS = 8;
constexpr int SLOTS = 32;                                  // maxima that a thread leaves
constexpr int AGAIN = 256;                                 // of them that are looked at again
constexpr float LEAST = -150.f;                            // exp2 of it is zero
constexpr float LN2 = 0.69314718055994531f, LOG2E = 1.4426950408889634f;
static_assert(WARPS * OD_MAX_TOP <= CAP, "a list from every warp fits");

struct ScoreArgs {
    const char *logits;
    int64_t row_bytes, seq_bytes;
    int32_t R, V, n_top, split;                            // blocks of a row
    const int32_t *ids, *n_rows;
    const float *temperature;
    float *logprob, *entropy, *row_max, *row_sum, *top_logprobs;
    int32_t *top_ids;
    uint32_t *flags;
};

__device__ __forceinline__ uint4 ld_stream(const void *p)
{
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ uint64_t f2_mul(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint32_t bf16x2_max(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

template <int DTYPE> constexpr int VEC = DTYPE == OD_BF16 ? 8 : 4;
template <int DTYPE> constexpr uint32_t NONE = DTYPE == OD_BF16 ? 0xFF80FF80u : 0xFF800000u;   // -inf

template <int DTYPE>
__device__ __forceinline__ float element(const uint4 &v, int k)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    if (DTYPE == OD_F32) return __uint_as_float(w[k]);
    return k & 1 ? od_bf16_hi(w[k >> 1]) : od_bf16_lo(w[k >> 1]);
}

// vector i of a row: whole ones as they lie; of a last one that the row ends in, what is there and -inf.
// READ_ONLY: the kernel does not write the row
template <int DTYPE, bool READ_ONLY = true>
__device__ __forceinline__ uint4 load_vec(const char *row, int i, int V)
{
    if (i < V / VEC<DTYPE>) return READ_ONLY ? ld_stream(row + (size_t)i * 16) : __ldcs((const uint4 *)(row + (size_t)i * 16));
    uint32_t w[4] = {NONE<DTYPE>, NONE<DTYPE>, NONE<DTYPE>, NONE<DTYPE>};
#pragma unroll
    for (int k = 0; k < VEC<DTYPE>; ++k) {
        const int j = i * VEC<DTYPE> + k;
        if (j >= V) continue;
        if (DTYPE == OD_F32) w[k] = __ldcs((const uint32_t *)row + j);
        else w[k >> 1] = (w[k >> 1] & (k & 1 ? 0xFFFFu : 0xFFFF0000u)) | (uint32_t)__ldcs((const unsigned short *)row + j) << (k & 1 ? 16 : 0);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// c = the largest logit so far (at least -FLT_MAX), s = sum of exp2((x - c) scale), a = sum of those times (x - c) scale
struct Sums {
    float c, s, a;
    __device__ __forceinline__ void raise(float to, float scale)
    {
        const float cn = fmaxf(c, to), d = fmaxf((c - cn) * scale, LEAST), f = od_ex2(d);
        a = (a + s * d) * f;
        s *= f;
        c = cn;
    }
};

__device__ __forceinline__ void absorb_pair(uint64_t &s2, uint64_t &a2, float lo, float hi, uint64_t nc2, uint64_t scale2)
{
    float d0, d1;
    f2_unpack(f2_mul(f2_add(f2_pack(lo, hi), nc2), scale2), d0, d1);
    const uint64_t e2 = f2_pack(od_ex2(d0), od_ex2(d1));
    s2 = f2_add(s2, e2);
    // (an exponential of -inf is zero, and so is its product with what is clamped here; NaN is in e)
    a2 = f2_fma(e2, f2_pack(fmaxf(d0, LEAST), fmaxf(d1, LEAST)), a2);
}

template <int DTYPE>
__device__ __forceinline__ float absorb(Sums &t, const uint4 (&x)[U], float scale)
{
    float gm;
    if (DTYPE == OD_BF16) {
        uint32_t g = NONE<DTYPE>;
#pragma unroll
        for (int u = 0; u < U; ++u) g = bf16x2_max(bf16x2_max(bf16x2_max(g, x[u].x), bf16x2_max(x[u].y, x[u].z)), x[u].w);
        gm = fmaxf(od_bf16_lo(g), od_bf16_hi(g));
    } else {
        gm = -INFINITY;
#pragma unroll
        for (int u = 0; u < U; ++u)
            gm = fmaxf(gm, fmaxf(fmaxf(__uint_as_float(x[u].x), __uint_as_float(x[u].y)),
                                 fmaxf(__uint_as_float(x[u].z), __uint_as_float(x[u].w))));
    }
    t.raise(gm, scale);
    const uint64_t nc2 = f2_pack(-t.c, -t.c), scale2 = f2_pack(scale, scale);
    uint64_t s0 = 0, s1 = 0, a0 = 0, a1 = 0;               // pairs of zeros
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int k = 0; k < VEC<DTYPE>; k += 4) {
            absorb_pair(s0, a0, element<DTYPE>(x[u], k), element<DTYPE>(x[u], k + 1), nc2, scale2);
            absorb_pair(s1, a1, element<DTYPE>(x[u], k + 2), element<DTYPE>(x[u], k + 3), nc2, scale2);
        }
    }
    float p, q;
    f2_unpack(f2_add(s0, s1), p, q);
    t.s += p + q;
    f2_unpack(f2_add(a0, a1), p, q);
    t.a += p + q;
    return gm;
}

// The order of the alternatives, by logit and then by the lower id, as one number: the larger comes first. 0 is none.
typedef unsigned long long Key;
__device__ __forceinline__ Key key_of(float v, int i)
{
    const uint32_t b = __float_as_uint(v + 0.f);           // (-0 is 0)
    return (Key)(b ^ ((int32_t)b < 0 ? 0xFFFFFFFFu : 0x80000000u)) << 32 | (0xFFFFFFFFu - (uint32_t)i);
}
__device__ __forceinline__ float logit_of(Key k)
{
    const uint32_t o = (uint32_t)(k >> 32);
    return __uint_as_float(o ^ ((int32_t)o < 0 ? 0x80000000u : 0xFFFFFFFFu));
}
__device__ __forceinline__ int id_of(Key k) { return (int)(0xFFFFFFFFu - (uint32_t)k); }

// how many of count keys (a multiple of four, a 16-byte aligned place in shared memory) come in front of k
__device__ __forceinline__ int keys_in_front(const Key *keys, int count, Key k)
{
    int rank = 0;
#pragma unroll 2
    for (int i = 0; i < count; i += 4) {
        const ulonglong2 a = *(const ulonglong2 *)(keys + i), b = *(const ulonglong2 *)(keys + i + 2);
        rank += (a.x > k) + (a.y > k) + (b.x > k) + (b.y > k);
    }
    return rank;
}

// Sorted list of the best in a warp's lanes, lane 0 first; the same k in every lane goes in at its place.
__device__ __forceinline__ void list_insert(Key &l, Key k, int lane)
{
    const int at = __popc(__ballot_sync(0xFFFFFFFFu, l > k));
    const Key up = __shfl_up_sync(0xFFFFFFFFu, l, 1);
    if (lane > at) l = up;
    if (lane == at) l = k;
}

__device__ __forceinline__ void store_cluster(float *p, uint32_t rank, float v)
{
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(od_cluster_address(p, rank)), "f"(v) : "memory");
}
__device__ __forceinline__ void store_cluster(int *p, uint32_t rank, int v)
{
    asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(od_cluster_address(p, rank)), "r"(v) : "memory");
}
__device__ __forceinline__ void store_cluster(Key *p, uint32_t rank, Key v)
{
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(od_cluster_address(p, rank)), "l"(v) : "memory");
}

// over a warp: the largest c, and the sums at it
__device__ __forceinline__ Sums warp_total(Sums t, float scale)
{
    float g = t.c;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) g = fmaxf(g, __shfl_xor_sync(0xFFFFFFFFu, g, o));
    t.raise(g, scale);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        t.s += __shfl_xor_sync(0xFFFFFFFFu, t.s, o);
        t.a += __shfl_xor_sync(0xFFFFFFFFu, t.a, o);
    }
    return t;
}

// (a temperature whose reciprocal overflows is none)
__device__ __forceinline__ bool usable(float T) { return T > 0.f && T < INFINITY && LOG2E / T < INFINITY; }

template <int DTYPE, bool TOP, int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) od_score_kernel(const ScoreArgs A)
{
    constexpr int WARPS = THREADS / 32, GROUP = THREADS / 32;  // threads to one of 32 groups
    __shared__ float group_max[32];
    __shared__ Sums warp_sums[WARPS], block_sums[MAX_SPLIT];
    __shared__ float block_ones[MAX_SPLIT], peak_rest;
    __shared__ int peak_warp;
    // candidates, and the best of all blocks of the row; maxima, and those that reach the bound (slot << 8 | thread)
    __shared__ __align__(16) Key cand[TOP ? CAP : 1], best[TOP ? MAX_SPLIT * OD_MAX_TOP : 1];
    __shared__ float maxima[TOP ? SLOTS : 1][THREADS];
    __shared__ unsigned short again[TOP ? AGAIN : 1];
    __shared__ int n_again, filled_of[MAX_SPLIT];          // (alternatives of each block)
    __shared__ int n_cand;

    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t split = A.split, part = blockIdx.x % split;
    const int64_t r = blockIdx.x / split;
    const int32_t b = (int32_t)(r / A.R), rr = (int32_t)(r % A.R);
    // (asked for at once; the blocks of a cluster leave together)
    const int live = A.n_rows ? A.n_rows[b] : A.R;
    const float T = A.temperature ? A.temperature[b] : 1.f;
    const int id = A.ids ? A.ids[r] : -1;
    if (rr >= live) return;
    const char *row = A.logits + b * A.seq_bytes + rr * A.row_bytes;
    const int V = A.V, n = A.n_top;
    const uint32_t bad_id = id < -1 || id >= V ? OD_LF_BAD_ID : 0u;
    // the slice of this block, by vectors
    const int nvec = (V - 1) / VEC<DTYPE> + 1;
    const int lo = (int)((int64_t)nvec * part / split), hi = (int)((int64_t)nvec * (part + 1) / split);
    const uint4 none = make_uint4(NONE<DTYPE>, NONE<DTYPE>, NONE<DTYPE>, NONE<DTYPE>);
    // turns of the loop to a slot: 2^per
    const int turns = (hi - lo + U * THREADS - 1) / (U * THREADS);
    int per = 0;
    while (turns > SLOTS << per) ++per;
    Sums t = {-FLT_MAX, 0.f, 0.f};
    uint4 x[U], y[U];
    // turns whose loads are all whole vectors of this block's slice
    const int whole = max(0, min(hi, V / VEC<DTYPE>) - lo) / (U * THREADS);
    const char *next = row + (size_t)(lo + tid) * 16;
    auto load = [&](uint4 (&v)[U], int turn) {
        if (turn < whole) {
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = ld_stream(next + u * THREADS * 16);
            next += U * THREADS * 16;
        } else {
            const int i = lo + tid + turn * (U * THREADS);
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = i + u * THREADS < hi ? load_vec<DTYPE>(row, i + u * THREADS, V) : none;
        }
    };
    load(x, 0);
    if (!usable(T)) {
        if (part == 0) {
            if (tid == 0) {
                A.row_max[r] = A.row_sum[r] = 0.f;
                if (A.logprob) A.logprob[r] = 0.f;
                if (A.entropy) A.entropy[r] = 0.f;
                if (A.flags) A.flags[r] = OD_LF_BAD_TEMPERATURE | bad_id;
            }
            if (TOP && tid < n) { A.top_ids[r * n + tid] = -1; A.top_logprobs[r * n + tid] = -INFINITY; }
        }
        return;
    }
    if (TOP) {
        for (int i = tid; i < CAP; i += THREADS) cand[i] = 0;
        if (tid == 0) n_cand = n_again = 0;
    }
    if (split > 1) od_cluster_arrive_relaxed();            // waited for before this block writes into another
    const float scale = LOG2E / T;
    float x_t = 0.f;                                       // requested early, by the thread that uses it
    if (tid == 0 && part == 0 && id >= 0 && id < V) x_t = od_load_logit<DTYPE>(row, id);

    auto take = [&](const uint4 (&v)[U], int turn) {
        float m = absorb<DTYPE>(t, v, scale);
        if (TOP) {
            float &most = maxima[turn >> per][tid];
            if (turn & (1 << per) - 1) m = fmaxf(m, most);
            most = m;
        }
    };
    for (int k = 0; k < turns; k += 2) {
        if (k + 1 < turns) load(y, k + 1);
        take(x, k);
        if (k + 1 == turns) break;
        if (k + 2 < turns) load(x, k + 2);
        take(y, k + 1);
    }
    if (TOP) {
        float g = t.c;
#pragma unroll
        for (int o = 1; o < GROUP; o <<= 1) g = fmaxf(g, __shfl_xor_sync(0xFFFFFFFFu, g, o));
        if (tid % GROUP == 0) group_max[tid / GROUP] = g;
    }
    const Sums w = warp_total(t, scale);
    if (lane == 0) warp_sums[warp] = w;
    __syncthreads();
    const Sums nothing = {-FLT_MAX, 0.f, 0.f};
    Sums of_warp = lane < WARPS ? warp_sums[lane] : nothing, all = warp_total(of_warp, scale);
    // Where the largest logit has nearly all of the mass, what the others have is what the entropy and its log probability
    // are made of, and behind the largest one's 1 its digits are lost: the thread that has read that one is summed again
    // without it, and ones + s is the sum from here on. (Its warp's sum goes to a place of its own: other warps may still
    // be reading warp_sums, by which all of them decide the same.)
    const bool peaked = all.s >= 1.f && all.s < 1.0625f;
    if (peaked) {
        const unsigned has = __ballot_sync(0xFFFFFFFFu, t.c == all.c && t.s >= 1.f);
        if (has) {                                         // (one lane of one warp)
            float rest = 0.f;
            for (int i = lo + warp * 32 + __ffs(has) - 1 + lane * THREADS; i < hi; i += 32 * THREADS) {
                const uint4 v = load_vec<DTYPE>(row, i, V);
#pragma unroll
                for (int k = 0; k < VEC<DTYPE>; ++k) {
                    const float e = element<DTYPE>(v, k);
                    if (e < all.c) rest += od_ex2((e - all.c) * scale);
                }
            }
            if (!(has >> lane & 1)) {
                Sums mine = t;
                mine.raise(all.c, scale);
                rest += mine.s;
            }
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) rest += __shfl_xor_sync(0xFFFFFFFFu, rest, o);
            if (lane == 0) { peak_rest = rest; peak_warp = warp; }
        }
        __syncthreads();
        if (lane == peak_warp) of_warp.s = peak_rest;
        all = warp_total(of_warp, scale);
    }
    if (TOP) {
        // the bound: the largest logit of the group that has n - 1 others in front of it
        const float g = group_max[lane];
        int rank = 0;
#pragma unroll
        for (int k = 0; k < 32; ++k) rank += group_max[k] > g || (group_max[k] == g && k < lane);
        const float bound = __shfl_sync(0xFFFFFFFFu, g, __ffs(__ballot_sync(0xFFFFFFFFu, rank == n - 1)) - 1);
        // by whole warps: a place for what reaches the bound (which is at least -FLT_MAX) in N vectors of each lane
        auto offer = [&](const uint4 *x, const int *at, int N) {
            int here = 0;
#pragma unroll
            for (int u = 0; u < N; ++u)
#pragma unroll
                for (int k = 0; k < VEC<DTYPE>; ++k) here += element<DTYPE>(x[u], k) >= bound;
            int before = here;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(0xFFFFFFFFu, before, o);
                if (lane >= o) before += v;
            }
            const int sum = __shfl_sync(0xFFFFFFFFu, before, 31);
            if (sum == 0) return;
            int place = 0;
            if (lane == 0) place = atomicAdd(&n_cand, sum);
            place = __shfl_sync(0xFFFFFFFFu, place, 0) + before - here;
            if (here)
#pragma unroll
                for (int u = 0; u < N; ++u)
#pragma unroll
                    for (int k = 0; k < VEC<DTYPE>; ++k) {
                        const float v = element<DTYPE>(x[u], k);
                        if (v < bound || v != v) continue;
                        if (place < CAP) cand[place] = key_of(v, at[u] * VEC<DTYPE> + k);
                        ++place;
                    }
        };
        if (turns <= 1) {                                  // all that a thread has read is still in its registers
            int at[U];
#pragma unroll
            for (int u = 0; u < U; ++u) at[u] = lo + tid + u * THREADS;
            offer(x, at, U);
        } else {
            if (t.c >= bound)
                for (int k = 0; k <= (turns - 1) >> per; ++k)
                    if (maxima[k][tid] >= bound) {
                        const int at = atomicAdd(&n_again, 1);
                        if (at < AGAIN) again[at] = (unsigned short)(k << 8 | tid);
                    }
            __syncthreads();
            if (n_again > AGAIN) {
                if (tid == 0) n_cand = CAP + 1;
            } else {
                const int each = U << per;                 // vectors of a slot
                for (int j0 = 0; j0 < n_again * each; j0 += THREADS) {
                    const int j = j0 + tid;
                    int i = hi;
                    if (j < n_again * each) {
                        const int what = again[j / each];
                        i = lo + (what & 255) + ((what >> 8) * each + j % each) * THREADS;
                    }
                    const uint4 v = i < hi ? load_vec<DTYPE>(row, i, V) : none;
                    offer(&v, &i, 1);
                }
            }
        }
        __syncthreads();
        int count = n_cand;
        if (count > CAP) {
            // many equal logits, or many of the largest in one thread: each warp lists the best of its elements
            // instead, in the order of their ids, so that of equal ones the first n are all that goes in
            __syncthreads();
            Key l = 0;
            for (int i0 = lo + warp * 32; i0 < hi; i0 += THREADS) {
                const int i = i0 + lane;
                const uint4 v = i < hi ? load_vec<DTYPE>(row, i, V) : none;
                const Key last = __shfl_sync(0xFFFFFFFFu, l, n - 1);
#pragma unroll
                for (int k = 0; k < VEC<DTYPE>; ++k) {
                    const Key mine = key_of(element<DTYPE>(v, k), i * VEC<DTYPE> + k);
                    unsigned in = __ballot_sync(0xFFFFFFFFu, element<DTYPE>(v, k) >= bound && mine > last);
                    for (; in; in &= in - 1) list_insert(l, __shfl_sync(0xFFFFFFFFu, mine, __ffs(in) - 1), lane);
                }
            }
            if (lane < n) cand[warp * n + lane] = l;
            __syncthreads();
            count = WARPS * n;
        }
        if (split > 1) od_cluster_wait();
        for (int j = tid; j < count; j += THREADS) {       // rank by counting (behind the last is none)
            const Key k = cand[j];
            const int rank = keys_in_front(cand, (count + 3) & ~3, k);
            if (k && rank < n) store_cluster(best + part * n + rank, 0, k);
        }
        if (tid < n && tid >= count) store_cluster(best + part * n + tid, 0, (Key)0);
        if (tid == 0) store_cluster(filled_of + part, 0, min(count, n));
    } else if (split > 1) {
        od_cluster_wait();
    }
    // the parts of the row to its cluster's first block
    if (tid < 3) store_cluster((float *)(block_sums + part) + tid, 0, tid == 0 ? all.c : tid == 1 ? all.s : all.a);
    if (tid == 3) store_cluster(block_ones + part, 0, peaked ? 1.f : 0.f);
    od_cluster_arrive();
    if (part != 0) return;                                 // (nobody writes into this block)
    od_cluster_wait();
    float ones = 0.f;
    {
        Sums of = nothing;
        if (lane < (int)split) { of = block_sums[lane]; ones = block_ones[lane]; }
        float c = of.c;
#pragma unroll
        for (int o = 1; o < MAX_SPLIT; o <<= 1) c = fmaxf(c, __shfl_xor_sync(0xFFFFFFFFu, c, o));
        c = __shfl_sync(0xFFFFFFFFu, c, 0);
        if (of.c < c) { of.s += ones; ones = 0.f; }        // (a one of another largest logit is none of the row's)
        all = warp_total(of, scale);
#pragma unroll
        for (int o = 1; o < MAX_SPLIT; o <<= 1) ones += __shfl_xor_sync(0xFFFFFFFFu, ones, o);
        ones = __shfl_sync(0xFFFFFFFFu, ones, 0);
    }
    const float rest = all.s;
    all.s += ones;
    const bool finite = all.s == all.s, empty = all.s == 0.f;
    const float nan = __int_as_float(0x7FFFFFFF), ln_s = ones == 1.f ? log1pf(rest) : logf(all.s);
    if (tid == 0) {
        A.row_max[r] = !finite ? nan : empty ? -INFINITY : all.c;
        A.row_sum[r] = all.s;
        float lp = 0.f;
        if (id >= 0 && id < V) lp = empty ? -INFINITY : (x_t - all.c) / T - ln_s;
        if (id >= 0 && id < V && !finite) lp = nan;
        if (A.logprob) A.logprob[r] = lp;
        if (A.entropy) A.entropy[r] = empty ? 0.f : ln_s - LN2 * (all.a / all.s);
        if (A.flags) A.flags[r] = (finite ? 0u : OD_LF_NONFINITE) | (empty ? OD_LF_NO_MASS : 0u) | bad_id;
    }
    if (TOP) {
        if (!finite) {
            if (tid < n) { A.top_ids[r * n + tid] = -1; A.top_logprobs[r * n + tid] = nan; }
            return;
        }
        // the blocks' lists are in order: a key's place is the sum of its places in all of them
        for (int j = tid; j < (int)split * n; j += THREADS) {
            const Key k = best[j];
            int at[MAX_SPLIT] = {};
#pragma unroll
            for (int o = OD_MAX_TOP; o > 0; o >>= 1) {
                if (o > n) continue;
#pragma unroll
                for (int p = 0; p < MAX_SPLIT; ++p)
                    if (p < (int)split && at[p] + o <= n && best[p * n + at[p] + o - 1] > k) at[p] += o;
            }
            int rank = 0;
#pragma unroll
            for (int p = 0; p < MAX_SPLIT; ++p) rank += at[p];
            if (k && rank < n) {
                A.top_ids[r * n + rank] = id_of(k);
                A.top_logprobs[r * n + rank] = (logit_of(k) - all.c) / T - ln_s;
            }
        }
        int filled = 0;
        for (int p = 0; p < (int)split; ++p) filled += filled_of[p];
        if (tid < n && tid >= filled) { A.top_ids[r * n + tid] = -1; A.top_logprobs[r * n + tid] = -INFINITY; }
    }
}

// ---- the gradient ------------------------------------------------------------------------------

struct ScoreGradArgs {
    const char *logits;
    int64_t row_bytes, seq_bytes;
    char *grad;
    int64_t grad_row_bytes, grad_seq_bytes;
    int32_t R, V, n_top, chunks, turns;                    // blocks of a row, loads of U vectors of a thread
    const int32_t *ids, *n_rows, *top_ids;
    const float *temperature, *row_max, *row_sum, *entropy, *g_logprob, *g_entropy, *g_top;
};


__device__ __forceinline__ uint32_t bf16x2(float lo, float hi)
{
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
template <int DTYPE>
__device__ __forceinline__ void store_element(char *row, int j, float v)
{
    if (DTYPE == OD_F32) ((float *)row)[j] = v;
    else ((unsigned short *)row)[j] = (unsigned short)bf16x2(v, 0.f);
}
template <int DTYPE>
__device__ __forceinline__ void store_whole(char *at, const float (&v)[VEC<DTYPE>])
{
    uint4 o;
    if constexpr (DTYPE == OD_F32)
        o = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    else
        o = make_uint4(bf16x2(v[0], v[1]), bf16x2(v[2], v[3]), bf16x2(v[4], v[5]), bf16x2(v[6], v[7]));
    *(uint4 *)at = o;
}
template <int DTYPE>
__device__ __forceinline__ void store_vec(char *row, int i, int V, const float (&v)[VEC<DTYPE>])
{
    if (i < V / VEC<DTYPE>) {
        store_whole<DTYPE>(row + (size_t)i * 16, v);
        return;
    }
#pragma unroll
    for (int k = 0; k < VEC<DTYPE>; ++k)
        if (i * VEC<DTYPE> + k < V) store_element<DTYPE>(row, i * VEC<DTYPE> + k, v[k]);
}

// grad may be the logits themselves: an element is written by the thread that has read it, the given ones behind a
// barrier from logits that were read in front of it.
template <int DTYPE, bool ENTROPY>
__global__ void __launch_bounds__(THREADS) od_score_grad_kernel(const ScoreGradArgs A)
{
    constexpr int GIVEN = OD_MAX_TOP + 1;
    __shared__ int given_id[GIVEN];
    __shared__ float given_g[GIVEN];

    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int tid = threadIdx.x, lane = tid & 31;
    const int64_t r = blockIdx.x / A.chunks;
    const int chunk = blockIdx.x % A.chunks, V = A.V, n = A.n_top;
    const int32_t b = (int32_t)(r / A.R), rr = (int32_t)(r % A.R);
    const char *row = A.logits + b * A.seq_bytes + rr * A.row_bytes;
    char *out = A.grad + b * A.grad_seq_bytes + rr * A.grad_row_bytes;
    const int nvec = (V - 1) / VEC<DTYPE> + 1, per_block = A.turns * (U * THREADS), lo = chunk * per_block, hi = min(nvec, lo + per_block);
    // (all that is asked for at once: none of it hangs on another)
    const int live = A.n_rows ? A.n_rows[b] : A.R;
    const float T = A.temperature ? A.temperature[b] : 1.f, S = A.row_sum[r], M = A.row_max[r];
    const float g_h = ENTROPY ? A.g_entropy[r] : 0.f, H = ENTROPY ? A.entropy[r] : 0.f;
    int id = A.ids && A.g_logprob ? A.ids[r] : -1, top = -1;
    float g_id = A.ids && A.g_logprob ? A.g_logprob[r] : 0.f, g = 0.f;
    if (A.g_top && lane < n) { top = A.top_ids[r * n + lane]; g = A.g_top[r * n + lane]; }
    auto zeros = [&]() {
        const float zero[VEC<DTYPE>] = {};
        for (int i = lo + tid; i < hi; i += THREADS) store_vec<DTYPE>(out, i, V, zero);
    };
    if (rr >= live) { zeros(); return; }
    const int whole = max(0, min(hi, V / VEC<DTYPE>) - lo) / (U * THREADS), turns = (hi - lo + U * THREADS - 1) / (U * THREADS);
    auto load = [&](uint4 (&v)[U], int turn) {
        const int i = lo + turn * (U * THREADS) + tid;
        if (turn < whole) {
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = __ldcs((const uint4 *)(row + (size_t)i * 16) + u * THREADS);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * THREADS < hi) v[u] = load_vec<DTYPE, false>(row, i + u * THREADS, V);
        }
    };
    uint4 x[U], y[U];
    load(x, 0);
    if (!usable(T) || S == 0.f) { zeros(); return; }

    // every warp sums the weights itself, in the same order
    const float ln_s = logf(S), scale = LOG2E / T;
    if (id < 0 || id >= V) { id = -1; g_id = 0.f; }
    if (top < 0 || top >= V) { top = -1; g = 0.f; }
    float G = g;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) G += __shfl_xor_sync(0xFFFFFFFFu, G, o);
    G += g_id;
    // the alternatives and behind them the given id
    if (tid < n) { given_id[tid] = top; given_g[tid] = g; }
    if (tid == 0) { given_id[n] = id; given_g[n] = g_id; }
    __syncthreads();
    const float per = -1.f / (S * T);
    const float c0 = per * (G + (ENTROPY ? g_h * (H - ln_s) : 0.f)), c1 = per * g_h * LN2;

    // the value of a given id in this chunk: it is written by the first entry that names it, with the sum of their weights
    int write = -1;
    float value = 0.f;
    if (tid <= n) {
        const int j = given_id[tid], i = j / VEC<DTYPE>;
        if (j >= 0 && i >= lo && i < hi) {
            float sum = 0.f;
            bool first = true;
            for (int k = 0; k <= n; ++k)
                if (given_id[k] == j) { sum += given_g[k]; first = first && k >= tid; }
            if (first) {
                const float xj = DTYPE == OD_F32 ? __ldcs((const float *)row + j) : __uint_as_float((uint32_t)__ldcs((const unsigned short *)row + j) << 16);
                const float d = (xj - M) * scale;
                value = od_ex2(d) * (ENTROPY ? c0 + c1 * fmaxf(d, LEAST) : c0) + sum / T;
                write = j;
            }
        }
    }
    // (in front of every store: they may be to the logits that were read above)
    __syncthreads();
    const uint64_t nm2 = f2_pack(-M, -M), scale2 = f2_pack(scale, scale), c02 = f2_pack(c0, c0), c12 = f2_pack(c1, c1);
    auto put = [&](const uint4 (&v)[U], int turn) {
        const int i = lo + turn * (U * THREADS) + tid;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (turn >= whole && i + u * THREADS >= hi) break;
            float w[VEC<DTYPE>];
#pragma unroll
            for (int k = 0; k < VEC<DTYPE>; k += 2) {
                float d0, d1;
                f2_unpack(f2_mul(f2_add(f2_pack(element<DTYPE>(v[u], k), element<DTYPE>(v[u], k + 1)), nm2), scale2), d0, d1);
                const uint64_t e2 = f2_pack(od_ex2(d0), od_ex2(d1));
                f2_unpack(f2_mul(e2, ENTROPY ? f2_fma(f2_pack(fmaxf(d0, LEAST), fmaxf(d1, LEAST)), c12, c02) : c02), w[k], w[k + 1]);
            }
            if (turn < whole) store_whole<DTYPE>(out + ((size_t)i + u * THREADS) * 16, w);
            else store_vec<DTYPE>(out, i + u * THREADS, V, w);
        }
    };
    // (in place too: a thread has read what it writes, and what it reads ahead is its own)
    for (int k = 0; k < turns; k += 2) {
        if (k + 1 < turns) load(y, k + 1);
        put(x, k);
        if (k + 1 == turns) break;
        if (k + 2 < turns) load(x, k + 2);
        put(y, k + 1);
    }
    __syncthreads();
    if (write >= 0) store_element<DTYPE>(out, write, value);
}

template <typename K, typename A>
cudaError_t launch(K kernel, unsigned blocks, unsigned cluster, bool pdl, const A &args, cudaStream_t s, unsigned threads = THREADS)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks); cfg.blockDim = dim3(threads);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cluster; attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = pdl ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, args);
}

}  // namespace

cudaError_t od_launch_score(const od_ctx *c, int32_t B, int32_t R, int32_t V, const void *logits, int32_t dtype, int64_t row_stride,
                            int64_t seq_stride, const int32_t *ids, const int32_t *n_rows, const float *temperature, int32_t n_top,
                            float *logprob, float *entropy, float *row_max, float *row_sum, int32_t *top_ids, float *top_logprobs,
                            uint32_t *flags, cudaStream_t s)
{
    const int64_t esz = dtype == OD_BF16 ? 2 : 4, rows = (int64_t)B * R;
    // Blocks of a row: one for many rows, up to 8 where there are few (of ragged ones half count, about): at most seven for two
    // multiprocessors, and none of a slice below 14 KB. (us with 20 alternatives, 1 / 2 / 4 / 8 blocks a row: one row of
    // 152064 bf16 logits 21 / 14 / 11 / 10, 96 rows of 128256 19 / 16 / 16 / 21, 448 rows 39 / 40 / 48 / 70, 4608 rows of
    // 152064 290 / 345 / 461 / 738.)
    const int64_t count = n_rows ? (rows + 1) / 2 : rows;
    int32_t split = 1;
    while (split < MAX_SPLIT && count * split * 4 <= 7 * c->sm_count && (int64_t)V * esz / (split * 2) >= 14 * 1024) split *= 2;
    const ScoreArgs a = {(const char *)logits, row_stride * esz, seq_stride * esz, R, V, n_top, split, ids, n_rows, temperature,
                         logprob, entropy, row_max, row_sum, top_logprobs, top_ids, flags};
    const unsigned blocks = (unsigned)(rows * split);
    const bool pdl = c->opt_pdl != 0;
    // Threads of a block that has a row alone: half as many where rows are short or more than are resident at a time, so that
    // more rows are, and one's end lies under others' loads. (us with one alternative, 256 / 128 threads: 2200 rows of 32000
    // bf16 logits 49 / 42, 4608 of 152064 258 / 242, 1000 of 4000 17 / 11; but 448 of 128256 34 / 37.)
    const bool half = split == 1 && (rows > 4 * c->sm_count || (int64_t)V * esz <= 96 * 1024);
    const auto of = [&](auto whole_block, auto half_block) {
        return half ? launch(half_block, blocks, 1, pdl, a, s, THREADS / 2) : launch(whole_block, blocks, split, pdl, a, s);
    };
    if (dtype == OD_BF16)
        return n_top ? of(od_score_kernel<OD_BF16, true, THREADS>, od_score_kernel<OD_BF16, true, THREADS / 2>)
                     : of(od_score_kernel<OD_BF16, false, THREADS>, od_score_kernel<OD_BF16, false, THREADS / 2>);
    return n_top ? of(od_score_kernel<OD_F32, true, THREADS>, od_score_kernel<OD_F32, true, THREADS / 2>)
                 : of(od_score_kernel<OD_F32, false, THREADS>, od_score_kernel<OD_F32, false, THREADS / 2>);
}

// Loads of a thread: up to 8, as long as there are eight blocks for every multiprocessor
static int32_t grad_turns(int64_t rows, int32_t nvec, int32_t sms)
{
    int32_t turns = 1;
    while (turns < GRAD_TURNS && rows * nvec / (U * THREADS * 2 * turns) >= 8 * (int64_t)sms) turns *= 2;
    return turns;
}

int64_t od_score_grad_blocks(int64_t rows, int32_t V, int32_t dtype, int32_t sms)
{
    const int32_t nvec = dtype == OD_BF16 ? (V - 1) / VEC<OD_BF16> + 1 : (V - 1) / VEC<OD_F32> + 1;
    const int32_t chunk = U * THREADS * grad_turns(rows, nvec, sms);
    return rows * ((nvec + chunk - 1) / chunk);
}

cudaError_t od_launch_score_grad(const od_ctx *c, int32_t B, int32_t R, int32_t V, const void *logits, int32_t dtype, int64_t row_stride,
                                 int64_t seq_stride, const int32_t *ids, const int32_t *n_rows, const float *temperature,
                                 const float *row_max, const float *row_sum, const float *entropy, int32_t n_top,
                                 const int32_t *top_ids, const float *g_logprob, const float *g_entropy, const float *g_top, void *grad,
                                 int64_t grad_row_stride, int64_t grad_seq_stride, cudaStream_t s)
{
    const int64_t esz = dtype == OD_BF16 ? 2 : 4, rows = (int64_t)B * R, blocks = od_score_grad_blocks(rows, V, dtype, c->sm_count);
    const int32_t nvec = (int32_t)(((int64_t)V * esz + 15) / 16);
    const ScoreGradArgs a = {(const char *)logits, row_stride * esz, seq_stride * esz, (char *)grad, grad_row_stride * esz,
                             grad_seq_stride * esz, R, V, n_top, (int32_t)(blocks / rows), grad_turns(rows, nvec, c->sm_count), ids,
                             n_rows, top_ids, temperature, row_max, row_sum, entropy, g_logprob, g_entropy, g_top};
    const bool pdl = c->opt_pdl != 0;
    if (dtype == OD_BF16)
        return g_entropy ? launch(od_score_grad_kernel<OD_BF16, true>, (unsigned)blocks, 1, pdl, a, s) : launch(od_score_grad_kernel<OD_BF16, false>, (unsigned)blocks, 1, pdl, a, s);
    return g_entropy ? launch(od_score_grad_kernel<OD_F32, true>, (unsigned)blocks, 1, pdl, a, s) : launch(od_score_grad_kernel<OD_F32, false>, (unsigned)blocks, 1, pdl, a, s);
}
