// What a row of logits says about a token: its log probability, the row's entropy, the largest log probabilities with their
// places; one pass over the logits, nothing of the size of the row written.
//
// A CTA (or each of the CTAs of a cluster, for a part of a row) takes its values from global memory once, into shared memory as
// they come; on the way a thread keeps its maximum m, the sum S of e^(x-m) and, for the entropy, the sum T of e^(x-m) (x-m).
// H = log S - T / S.  (x - m is exact for the largest, so that a token without alternatives has log probability and entropy zero.)
// Memory bounds many rows (one exponential and eight instructions a value are close behind), the chain of steps a few.
//
// The largest `top` of a part: of each warp the q-th largest of its threads' maxima, the least of these over the warps: q times the
// warps threads reach it, so that at least `top` values do, and hardly more than a hundred.  They are listed, and each finds its
// place by counting those before it.  Where more values reach the bound than the list holds (many equal ones), the top-th value
// is searched bit by bit.  Equal values count in the order of their places throughout: a value and its place are one number.
#include <cuda_bf16.h>

#include "spqt_common.cuh"
#include "spqt_gemv_device.cuh"
#include "spqt_kv.cuh"

namespace spqt {

constexpr int kMaxTop = 32, kMaxVocab = 1 << 20;
constexpr int kLogThreads = 512, kLogWarps = kLogThreads / 32;
constexpr int kMaxLogCtas = 8;          // of a cluster
constexpr int kLogList = 1536;          // values that may reach the bound
constexpr size_t kLogKeep = 98304;      // bytes of a part that shared memory keeps; larger ones are read again

struct LogArgs {
    const void* logits;
    long long row_stride;
    const int32_t* tokens;
    float *logprob, *entropy, *top_logprob;
    int32_t* top_index;
    int vocab, top, part, keep;         // part: values of a CTA; keep: they stay in shared memory
};

constexpr float kLog2e = 1.4426950408889634f;

// Whole numbers in the order of the values, not-a-number above all, zeros of both signs alike, 0 below all; behind them the place,
// lower ones larger.
__device__ __forceinline__ unsigned value_bits(float f)
{
    if (f != f) return 0xffffffffu;
    const unsigned u = __float_as_uint(f + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(unsigned k)
{
    return k == 0xffffffffu ? __int_as_float(0x7fffffff) : __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}
__device__ __forceinline__ unsigned long long key_of(float f, int place) { return (unsigned long long)value_bits(f) << 32 | (unsigned)(0x7fffffff - place); }
__device__ __forceinline__ int place_of(unsigned long long key) { return 0x7fffffff - (int)(unsigned)key; }

__device__ __forceinline__ float exp_of(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x * kLog2e));
    return y;
}

struct Sums {
    float m, s, t;                      // m = -infinity: nothing summed
};
__device__ __forceinline__ void move_to(Sums& a, float m)   // to a maximum not below its own
{
    if (a.m == m) return;
    const float d = a.m - m, f = exp_of(d);
    a.t = a.s == 0.0f ? 0.0f : fmaf(a.s, d, a.t) * f;
    a.s *= f;
    a.m = m;
}
__device__ __forceinline__ Sums joined(Sums a, Sums b)
{
    const float m = fmaxf(a.m, b.m);
    move_to(a, m);
    move_to(b, m);
    return {m, a.s + b.s, a.t + b.t};
}
__device__ __forceinline__ Sums shuffled(const Sums& a, int o)
{
    return {__shfl_xor_sync(0xffffffffu, a.m, o), __shfl_xor_sync(0xffffffffu, a.s, o), __shfl_xor_sync(0xffffffffu, a.t, o)};
}

template <class T>
struct Vec {                            // 16 bytes of values
    static constexpr int N = 16 / (int)sizeof(T);
    float x[N];
    __device__ __forceinline__ explicit Vec(const uint4& w)
    {
        const unsigned u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 4) {
                x[i] = __uint_as_float(u[i]);
            } else if constexpr (std::is_same<T, __half>::value) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
                x[2 * i] = f.x, x[2 * i + 1] = f.y;
            } else {
                x[2 * i] = __uint_as_float(u[i] << 16), x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
            }
        }
    }
};

struct LogShared {
    Sums sums[kLogWarps];
    Sums parts[kMaxLogCtas];                            // of the cluster's CTAs (in the first one's memory)
    unsigned long long best[kMaxLogCtas * kMaxTop];     // their largest, in order
    unsigned long long mine[kMaxTop];
    unsigned long long list[kLogList];
    unsigned bound[kLogWarps];
    int count, votes[2];
    float odd[16];                                      // values in front of the first whole 16 bytes and behind the last
};

// Shared memory of the cluster's first CTA at the address of this CTA's `p`.
__device__ __forceinline__ unsigned in_first_cta(const void* p) { return cluster_map(smem_u32(p), 0); }

template <class T, bool CLUSTER>
__global__ void __launch_bounds__(kLogThreads) token_logprobs_kernel(const LogArgs a)
{
    extern __shared__ __align__(16) unsigned char s_vals[];   // the part's whole 16 bytes
    __shared__ LogShared sh;
    constexpr int V = Vec<T>::N;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int ctas = CLUSTER ? (int)gridDim.x : 1, rank = CLUSTER ? (int)blockIdx.x : 0, r = CLUSTER ? (int)blockIdx.y : (int)blockIdx.x;
    const int first = rank * a.part, n = max(0, min(a.part, a.vocab - first));
    if (CLUSTER) cluster_arrive();
    if (tid == 0) sh.count = 0;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const T* const whole_row = static_cast<const T*>(a.logits) + (long long)r * a.row_stride;
    const T* const row = whole_row + first;
    const int token = a.tokens && rank == 0 && tid == 0 ? (int)ld_global_u32(a.tokens + r) : -1;
    const bool wanted = (unsigned)token < (unsigned)a.vocab;
    const float chosen = wanted ? (float)whole_row[token] : 0.0f;

    // ---- one pass
    Sums sum = {-INFINITY, 0.0f, 0.0f};
    float largest = -INFINITY;          // (not-a-number is not seen here: the value is one that some value reaches; and it makes the sums not-a-number)
    const bool entropy = a.entropy != nullptr;
    auto add = [&](const float* x, auto count) {
        constexpr int N = decltype(count)::value;
        float m = x[0];
#pragma unroll
        for (int i = 1; i < N; ++i) m = fmaxf(m, x[i]);
        if (m > largest) {
            largest = m;
            move_to(sum, m);
        }
        const float base = sum.m == -INFINITY ? 0.0f : sum.m;
        float s = 0.0f, t = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float d = x[i] - base, e = exp_of(d);
            s += e;
            if (entropy) t = fmaf(e, fmaxf(d, -1e30f), t);      // (-infinity: 0, not 0 times infinity)
        }
        sum.s += s;
        sum.t += t;
    };
    const int head = min(n, (int)((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / (int)sizeof(T));
    const int vecs = (n - head) / V, odd = n - vecs * V;        // odd ones: the head, then the tail; V - 1 of each at most
    auto place_of_odd = [&](int i) { return i < head ? i : vecs * V + i; };
    if (tid < odd) {
        const float x = (float)row[place_of_odd(tid)];
        sh.odd[tid] = x;
        add(&x, std::integral_constant<int, 1>());
    }
    constexpr int kU = 4;
#pragma unroll 1
    for (int i0 = tid; i0 < vecs; i0 += kLogThreads * kU) {
        uint4 w[kU];
#pragma unroll
        for (int u = 0; u < kU; ++u) w[u] = ld_global_v4_if(i0 + u * kLogThreads < vecs, row + head + (size_t)(i0 + u * kLogThreads) * V);
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const int i = i0 + u * kLogThreads;
            if (i < vecs) {
                if (a.keep) *reinterpret_cast<uint4*>(s_vals + (size_t)i * 16) = w[u];
                const Vec<T> v(w[u]);
                add(v.x, std::integral_constant<int, V>());
            }
        }
    }
    Sums all = sum;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) all = joined(all, shuffled(all, o));
    if (lane == 0) sh.sums[warp] = all;

    // ---- the largest values
    if (a.top > 0) {
        const int full = min(kLogWarps, vecs / 32);            // warps all of whose threads have values
        unsigned mine = value_bits(largest), bound = 0u;
        if (warp < full)
            for (int q = (a.top + full - 1) / full; q > 0; --q) {
                bound = __reduce_max_sync(0xffffffffu, mine);
                const unsigned who = __ballot_sync(0xffffffffu, mine == bound);
                if (lane == __ffs(who) - 1) mine = 0u;
            }
        if (lane == 0) sh.bound[warp] = warp < full ? bound : 0xffffffffu;
        __syncthreads();
        unsigned least = full == 0 || full * 32 < a.top ? 0u : sh.bound[lane % kLogWarps];
        least = __reduce_min_sync(0xffffffffu, least);
        // each value of the part with its place; `f` is called by all threads the same number of times
        auto each = [&](auto f) {
            if (tid < odd) f(key_of(sh.odd[tid], place_of_odd(tid)));
#pragma unroll 1
            for (int i = tid; i < vecs; i += kLogThreads) {
                const uint4 w = a.keep ? *reinterpret_cast<const uint4*>(s_vals + (size_t)i * 16) : ld_global_v4(row + head + (size_t)i * V);
                const Vec<T> v(w);
#pragma unroll
                for (int e = 0; e < V; ++e) f(key_of(v.x[e], head + i * V + e));
            }
        };
        unsigned long long from = (unsigned long long)least << 32;
        each([&](unsigned long long k) {
            if (k >= from) {
                const int at = atomicAdd(&sh.count, 1);
                if (at < kLogList) sh.list[at] = k;
            }
        });
        __syncthreads();
        int listed = sh.count;
        if (listed > kLogList) {                                // the top-th largest key, bit by bit
            from = 0ull;
#pragma unroll 1
            for (int bit = 63; bit >= 0; --bit) {
                const unsigned long long trial = from | 1ull << bit;
                int c = 0;
                each([&](unsigned long long k) { c += k >= trial; });
                c = __reduce_add_sync(0xffffffffu, c);
                if (tid < 2) sh.votes[tid] = 0;
                __syncthreads();
                if (lane == 0) atomicAdd(&sh.votes[0], c);
                __syncthreads();
                if (sh.votes[0] >= a.top) from = trial;
                __syncthreads();
            }
            if (tid == 0) sh.count = 0;
            __syncthreads();
            each([&](unsigned long long k) {
                if (k >= from) sh.list[atomicAdd(&sh.count, 1)] = k;    // (keys are distinct: these are `top`, or all of the part)
            });
            __syncthreads();
            listed = sh.count;
        }
        if (tid < a.top) sh.mine[tid] = 0ull;                   // (a part may have fewer)
        __syncthreads();
        for (int i = tid; i < listed; i += kLogThreads) {
            const unsigned long long k = sh.list[i];
            int before = 0;
            for (int j = 0; j < listed; ++j) before += sh.list[j] > k;
            if (before < a.top) sh.mine[before] = k;
        }
    }
    __syncthreads();
    Sums part = sh.sums[lane % kLogWarps];
#pragma unroll
    for (int o = kLogWarps / 2; o > 0; o >>= 1) part = joined(part, shuffled(part, o));

    // ---- the parts of a row, in the cluster's first CTA
    if (CLUSTER) {
        cluster_wait();                                         // (all CTAs have begun)
        if (warp == 0) {
            if (lane == 0) {
                const unsigned to = in_first_cta(&sh.parts[rank]);
                asm volatile("st.shared::cluster.f32 [%0], %1;\n\tst.shared::cluster.f32 [%0+4], %2;\n\tst.shared::cluster.f32 [%0+8], %3;" ::"r"(to),
                             "f"(part.m), "f"(part.s), "f"(part.t)
                             : "memory");
            }
            if (lane < a.top) {
                const unsigned long long k = sh.mine[lane];     // (places of the whole row)
                const unsigned long long whole = k == 0ull ? 0ull : k - (unsigned)first;
                asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(in_first_cta(&sh.best[rank * a.top + lane])), "l"(whole) : "memory");
            }
        }
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        if (rank != 0) return;
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        part = lane < ctas ? sh.parts[lane] : Sums{-INFINITY, 0.0f, 0.0f};
#pragma unroll
        for (int o = kMaxLogCtas / 2; o > 0; o >>= 1) part = joined(part, shuffled(part, o));
    }
    // (of a row without a finite value m is infinite: not-a-number.  In a row of the cluster the lanes from 8 on have joined nothing)
    const float m = __shfl_sync(0xffffffffu, part.m, 0), s = __shfl_sync(0xffffffffu, part.s, 0), t = __shfl_sync(0xffffffffu, part.t, 0);
    const bool none = !(fabsf(m) < INFINITY) || s != s;
    const float nan = __int_as_float(0x7fffffff), logsum = logf(s);
    if (tid == 0) {
        if (a.logprob) a.logprob[r] = none || !wanted ? nan : (chosen - m) - logsum;
        if (a.entropy) a.entropy[r] = none ? nan : logsum - t / s;
    }
    auto put = [&](int i, unsigned long long k) {
        a.top_index[(size_t)r * a.top + i] = place_of(k);
        a.top_logprob[(size_t)r * a.top + i] = none ? nan : (value_of((unsigned)(k >> 32)) - m) - logsum;
    };
    if (!CLUSTER) {
        if (tid < a.top) put(tid, sh.mine[tid]);
    } else {
        const int keys = ctas * a.top;
        if (tid < keys) {
            const unsigned long long k = sh.best[tid];
            int before = 0;
            for (int j = 0; j < keys; ++j) before += sh.best[j] > k;
            if (k != 0ull && before < a.top) put(before, k);
        }
    }
}

template <class T>
cudaError_t launch_logprobs(LogArgs a, int rows, cudaStream_t s)
{
    // CTAs per row: enough for a part to stay in shared memory; more while there are fewer CTAs than two per SM and a thread would
    // still have a vector of each part.
    const int sms = sm_count();
    if (sms <= 0) return cudaErrorInvalidDevice;
    constexpr int V = Vec<T>::N;
    int ctas = 1;
    auto part_of = [&](int c) { return ((a.vocab + c - 1) / c + V - 1) / V * V; };
    while (ctas < kMaxLogCtas && ((size_t)part_of(ctas) * sizeof(T) > kLogKeep || ((long long)rows * ctas < 2 * sms && part_of(2 * ctas) >= kLogThreads * V))) ctas *= 2;
    a.part = part_of(ctas);
    const size_t bytes = (size_t)a.part * sizeof(T);
    a.keep = a.top > 0 && bytes <= kLogKeep;
    const size_t smem = a.keep ? bytes : 0;
    static thread_local int allowed_dev = -1;
    int dev = 0;
    cudaError_t err = cudaGetDevice(&dev);
    if (err != cudaSuccess) return err;
    if (allowed_dev != dev) {
        err = cudaFuncSetAttribute(token_logprobs_kernel<T, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kLogKeep);
        if (err == cudaSuccess) err = cudaFuncSetAttribute(token_logprobs_kernel<T, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kLogKeep);
        if (err != cudaSuccess) return err;
        allowed_dev = dev;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(kLogThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ctas;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = g_no_pdl ? attr + 1 : attr;
    cfg.numAttrs = (g_no_pdl ? 0 : 1) + (ctas > 1 ? 1 : 0);
    if (ctas == 1) {
        cfg.gridDim = dim3(rows);
        err = cudaLaunchKernelEx(&cfg, token_logprobs_kernel<T, false>, a);
        if (err == cudaSuccess) count_launch();
        return err;
    }
    // (rows are the grid's second dimension: 65535 at a time)
    for (int r0 = 0; r0 < rows && err == cudaSuccess; r0 += 65535) {
        const int some = rows - r0 < 65535 ? rows - r0 : 65535;
        LogArgs b = a;
        b.logits = static_cast<const T*>(a.logits) + (long long)r0 * a.row_stride;
        if (a.tokens) b.tokens = a.tokens + r0;
        if (a.logprob) b.logprob = a.logprob + r0;
        if (a.entropy) b.entropy = a.entropy + r0;
        if (a.top > 0) b.top_logprob = a.top_logprob + (size_t)r0 * a.top, b.top_index = a.top_index + (size_t)r0 * a.top;
        cfg.gridDim = dim3(ctas, some);
        err = cudaLaunchKernelEx(&cfg, token_logprobs_kernel<T, true>, b);
        if (err == cudaSuccess) count_launch();
    }
    return err;
}

}  // namespace spqt

extern "C" spqt_status spqt_token_logprobs(const void* logits, int dtype, int rows, int vocab, long long row_stride, const int32_t* tokens, int top,
                                           float* logprob, float* entropy, float* top_logprob, int32_t* top_index, void* stream)
{
    using namespace spqt;
    if (rows < 0 || vocab < 1 || top < 0 || top > vocab || row_stride < vocab) return SPQT_ERR_INVALID_ARG;
    if (dtype != SPQT_LOGITS_FP16 && dtype != SPQT_LOGITS_BF16 && dtype != SPQT_LOGITS_FP32) return SPQT_ERR_UNSUPPORTED;
    if (top > kMaxTop || vocab > kMaxVocab) return SPQT_ERR_UNSUPPORTED;
    if (rows == 0) return SPQT_OK;
    if (!logits || (tokens && !logprob) || (!tokens && logprob) || (top > 0 && (!top_logprob || !top_index))) return SPQT_ERR_INVALID_ARG;
    const size_t size = dtype == SPQT_LOGITS_FP32 ? 4 : 2;
    if (!aligned(logits, size) || !aligned(tokens, 4) || !aligned(logprob, 4) || !aligned(entropy, 4) || !aligned(top_logprob, 4) || !aligned(top_index, 4))
        return SPQT_ERR_ALIGNMENT;
    const LogArgs a = {logits, row_stride, tokens, logprob, entropy, top_logprob, top_index, vocab, top, 0, 0};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return launched(dtype == SPQT_LOGITS_FP16   ? launch_logprobs<__half>(a, rows, s)
                    : dtype == SPQT_LOGITS_BF16 ? launch_logprobs<__nv_bfloat16>(a, rows, s)
                                                : launch_logprobs<float>(a, rows, s));
}
