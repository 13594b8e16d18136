// What a row of logits says about a token: its log probability, the row's entropy, the largest log probabilities with their
// places; one pass over the logits, nothing of the size of the row written.
//
// A row is read once, by a CTA, by the CTAs of a cluster (few rows: a part each) or by a warp (short rows).  On the way a thread keeps
// its maximum m, the sum S of e^(x-m) and, for the entropy, the sum T of e^(x-m) (x-m).  H = log S - T / S.  (x - m is exact for the
// largest, so that a token without alternatives has log probability and entropy zero.)  Memory bounds many rows, with the
// instructions close behind (an exponential and five more a value, two values an instruction where there is one for two), the
// chain of steps a few.
//
// The largest `top` of a part: every warp names the largest few of its threads' maxima, and the top-th largest of those named is a
// bound that `top` values or more reach, hardly more in most rows.  Only the threads that reach it have their values looked at again;
// these are listed, and each finds its place by counting those before it.  Where more reach the bound than the list holds, those above
// it are listed and the first of those equal to it; where too many are above it, the top-th value is searched bit by bit.  Equal values count in the order of their places throughout: a value
// and its place are one number.
#include <cuda_bf16.h>

#include "spqt_common.cuh"
#include "spqt_gemv_device.cuh"
#include "spqt_kv.cuh"

namespace spqt {

constexpr int kMaxTop = 32, kMaxVocab = 1 << 20;
constexpr int kMaxLogCtas = 8;          // of a cluster
constexpr int kNamed = 64;              // maxima that the warps name: 4 of each, or more of fewer warps
constexpr int kLogList = 1536;          // values that may reach the bound

struct LogArgs {
    const void* logits;
    long long row_stride;
    const int32_t* tokens;
    float *logprob, *entropy, *top_logprob;
    int32_t* top_index;
    int vocab, top, part;               // part: values of a CTA of a cluster
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

__device__ __forceinline__ float exp2_of(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float exp_of(float x) { return exp2_of(x * kLog2e); }

struct Sums {
    float m, s, t;                      // m = -infinity: nothing summed
};
__device__ __forceinline__ void move_to(Sums& a, float m)   // to a maximum not below its own
{
    if (a.m == m) return;
    const float d = a.m - m, f = exp_of(d);
    // (f = 0: nothing summed, or nothing is left of the sums; s * d, with masks of the type's lowest value, may then be infinite)
    a.t = f == 0.0f ? 0.0f : fmaf(a.s, d, a.t) * f;
    a.s *= f;
    a.m = m;
}
// over the lanes of a warp (in all of them)
__device__ __forceinline__ Sums joined(Sums a)
{
    float m = a.m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    move_to(a, m);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        a.s += __shfl_xor_sync(0xffffffffu, a.s, o);
        a.t += __shfl_xor_sync(0xffffffffu, a.t, o);
    }
    return a;
}

// x - base in fp32 of two values of a word (exact where it counts: x near base)
__device__ __forceinline__ unsigned long long less_base(unsigned w, float base, __half)
{
    float lo, hi;
    asm("{\n\t.reg .f16 a, b;\n\tmov.b32 {a, b}, %2;\n\tadd.rn.f32.f16 %0, a, %3;\n\tadd.rn.f32.f16 %1, b, %3;\n\t}" : "=f"(lo), "=f"(hi) : "r"(w), "f"(-base));
    return pack2(lo, hi);
}
__device__ __forceinline__ unsigned long long less_base(unsigned w, float base, __nv_bfloat16)
{
    return fadd2(pack2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)), pack2(-base, -base));
}

// 16 bytes of values.
template <class T>
struct Vec {
    static constexpr int N = 16 / (int)sizeof(T), P = N / 2;   // P pairs
    uint4 w;
    __device__ __forceinline__ explicit Vec(const uint4& v) : w(v) {}
    __device__ __forceinline__ unsigned word(int i) const { return i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w; }
    __device__ __forceinline__ void pair(int i, float& lo, float& hi) const
    {
        if constexpr (sizeof(T) == 4) {
            lo = __uint_as_float(word(2 * i)), hi = __uint_as_float(word(2 * i + 1));
        } else if constexpr (std::is_same<T, __half>::value) {
            const unsigned u = word(i);
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u));
            lo = f.x, hi = f.y;
        } else {
            lo = __uint_as_float(word(i) << 16), hi = __uint_as_float(word(i) & 0xffff0000u);
        }
    }
    __device__ __forceinline__ unsigned long long less(int i, float base) const
    {
        if constexpr (sizeof(T) == 4) return fadd2(pack2(__uint_as_float(word(2 * i)), __uint_as_float(word(2 * i + 1))), pack2(-base, -base));
        else return less_base(word(i), base, T());
    }
    // the larger of two words' values each, not-a-number left out, and the largest of a word
    static __device__ __forceinline__ unsigned larger(unsigned a, unsigned b)
    {
        if constexpr (sizeof(T) == 4) {
            return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
        } else if constexpr (std::is_same<T, __half>::value) {
            const __half2 m = __hmax2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
            return *reinterpret_cast<const unsigned*>(&m);
        } else {
            const __nv_bfloat162 m = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
            return *reinterpret_cast<const unsigned*>(&m);
        }
    }
    static __device__ __forceinline__ float largest_of(unsigned a)
    {
        if constexpr (sizeof(T) == 4) {
            return __uint_as_float(a);
        } else if constexpr (std::is_same<T, __half>::value) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&a));
            return fmaxf(f.x, f.y);
        } else {
            return fmaxf(__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u));
        }
    }
    __device__ __forceinline__ unsigned larger() const { return larger(larger(w.x, w.y), larger(w.z, w.w)); }
    __device__ __forceinline__ float top() const { return largest_of(larger()); }
};

// Sum of e^d d, d = x - base, of 16 bytes of values, -infinity adding nothing.  (A call, since the values in earnest seldom need it.)
template <class T>
__device__ __noinline__ float without_infinities(uint4 w, float base)
{
    const Vec<T> v(w);
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < Vec<T>::P; ++i) {
        float lo, hi;
        v.pair(i, lo, hi);
        t = fmaf(exp_of(lo - base), fmaxf(lo - base, -1e30f), t);
        t = fmaf(exp_of(hi - base), fmaxf(hi - base, -1e30f), t);
    }
    return t;
}

constexpr int kSlots = 8;

// What a team of threads (a warp, or a CTA) shares.  Two of what the first warp may still read, or set, when the others are at the
// next row.
template <int NW, int LIST>
struct LogShared {
    uint4 named[kNamed / 4];
    unsigned long long list[LIST];
    unsigned long long mine[kMaxTop];                   // the largest, in order
    Sums sums[2][NW];
    int listed[2], reached[2], votes;
    float odd[16];                                      // values in front of the first whole 16 bytes and behind the last
    float tops[kSlots][32 * NW];                        // the largest of a thread's vectors, those of a few rounds in a slot
    unsigned short who[kSlots * 32 * NW];               // slots (times the threads) and threads whose largest reaches the bound
};
struct LogClusterShared {                               // (in the first CTA's memory)
    Sums parts[kMaxLogCtas];
    unsigned long long best[kMaxLogCtas * kMaxTop];
};

// Shared memory of the cluster's first CTA at the address of this CTA's `p`.
__device__ __forceinline__ unsigned in_first_cta(const void* p) { return cluster_map(smem_u32(p), 0); }

// A row of a type's values from `first` on: the odd ones in front, whole 16 bytes, the odd ones behind.
template <class T>
struct LogPart {
    static constexpr int V = Vec<T>::N;
    const T* row;
    int head, vecs, odd;
    __device__ __forceinline__ LogPart(const T* p, int n) : row(p)
    {
        head = min(n, (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / (int)sizeof(T));
        vecs = (n - head) / V;
        odd = n - vecs * V;
    }
    __device__ __forceinline__ int place_of_odd(int i) const { return i < head ? i : vecs * V + i; }
    __device__ __forceinline__ const void* vec(int i) const { return row + head + (size_t)i * V; }
};

constexpr int kVecs = 4;                // vectors of a thread on their way at a time: a round

// TEAM threads for a part: 32 or 128 (several teams in the CTA) or the whole CTA.
template <class T, int TEAM, int LIST>
struct LogTeam {
    static constexpr int NW = TEAM / 32, V = Vec<T>::N;
    LogShared<NW, LIST>& sh;
    const LogArgs& a;
    int tid, lane, warp;                // in the team
    int turn;                           // 0, 1, 0, ... row after row
    Sums sum;
    float largest;                      // (not-a-number is not seen here: some value reaches it; and it makes the sums not-a-number)
    int slot_shift;                     // log2 of the rounds of a slot
    float slot_top;

    static __device__ __forceinline__ void sync()
    {
        if constexpr (TEAM == 32) __syncwarp();
        else if constexpr (TEAM == 128) asm volatile("bar.sync %0, 128;" ::"r"((int)threadIdx.x / 128 + 1) : "memory");
        else __syncthreads();
    }
    __device__ __forceinline__ void load(uint4* w, const LogPart<T>& p, int i0) const
    {
#pragma unroll
        for (int u = 0; u < kVecs; ++u) w[u] = ld_global_v4_if(i0 + u * TEAM < p.vecs, p.vec(i0 + u * TEAM));
    }
    // a new maximum, if it is one; what is subtracted
    __device__ __forceinline__ float reach(float m)
    {
        if (m > largest) {
            largest = m;
            move_to(sum, m);
        }
        return sum.m == -INFINITY ? 0.0f : sum.m;
    }
    __device__ __forceinline__ void begin(const LogPart<T>& p)
    {
        sum = {-INFINITY, 0.0f, 0.0f};
        largest = slot_top = -INFINITY;
        const int rounds = (p.vecs + TEAM * kVecs - 1) / (TEAM * kVecs);
        slot_shift = rounds <= kSlots ? 0 : 32 - __clz((rounds - 1) / kSlots);
        if (tid < p.odd) {
            const float x = (float)p.row[p.place_of_odd(tid)];
            sh.odd[tid] = x;
            const float d = x - reach(x), e = exp_of(d);
            sum.s += e;
            sum.t = fmaf(e, fmaxf(d, -1e30f), sum.t);           // (-infinity: 0, not 0 times infinity)
        }
        if (tid == 0) sh.listed[turn] = sh.reached[turn] = 0;
    }
    // a round's vectors, the first at i0 (of all threads at `round` * TEAM * kVecs)
    __device__ __forceinline__ void add(const uint4* w, const LogPart<T>& p, int i0, int round)
    {
        if ((round + 1) * (TEAM * kVecs) <= p.vecs) add_some<true>(w, p, i0);
        else add_some<false>(w, p, i0);
        if (a.top > 0 && (((round + 1) & ((1 << slot_shift) - 1)) == 0 || (round + 1) * (TEAM * kVecs) >= p.vecs)) {
            sh.tops[round >> slot_shift][tid] = slot_top;
            slot_top = -INFINITY;
        }
    }
    template <bool ALL>
    __device__ __forceinline__ void add_some(const uint4* w, const LogPart<T>& p, int i0)
    {
        const bool entropy = a.entropy != nullptr;
        float top = -INFINITY;
        if (ALL) {
            unsigned m = Vec<T>(w[0]).larger();
#pragma unroll
            for (int u = 1; u < kVecs; ++u) m = Vec<T>::larger(m, Vec<T>(w[u]).larger());
            top = fmaxf(top, Vec<T>::largest_of(m));
        } else {
#pragma unroll
            for (int u = 0; u < kVecs; ++u)
                if (i0 + u * TEAM < p.vecs) top = fmaxf(top, Vec<T>(w[u]).top());
        }
        slot_top = fmaxf(slot_top, top);
        const float base = reach(top);
        unsigned long long s = 0ull, t = 0ull;
        float lo, hi;
#pragma unroll
        for (int u = 0; u < kVecs; ++u)
            if (ALL || i0 + u * TEAM < p.vecs) {
                const Vec<T> v(w[u]);
#pragma unroll
                for (int i = 0; i < Vec<T>::P; ++i) {
                    const unsigned long long d = v.less(i, base);
                    unpack2(fmul2(d, pack2(kLog2e, kLog2e)), lo, hi);
                    const unsigned long long e = pack2(exp2_of(lo), exp2_of(hi));
                    s = fadd2(s, e);
                    if (entropy) t = fma2(e, d, t);
                }
            }
        unpack2(s, lo, hi);
        sum.s += lo + hi;
        unpack2(t, lo, hi);
        float both = lo + hi;
        if (both != both) {                                     // 0 times infinity, unless it is not-a-number in earnest
            both = 0.0f;
#pragma unroll
            for (int u = 0; u < kVecs; ++u)
                if (ALL || i0 + u * TEAM < p.vecs) both += without_infinities<T>(w[u], base);
        }
        sum.t += both;
    }
    __device__ __forceinline__ void put(unsigned long long k)
    {
        const int at = atomicAdd(&sh.listed[turn], 1);
        if (at < LIST) sh.list[at] = k;
    }
    static __device__ __forceinline__ bool overfull(const int& count) { return *reinterpret_cast<volatile const int*>(&count) > LIST; }
    // More values reach the bound than the list holds.  In a row whose other values are masked most of them are the bound itself: the
    // values above it are listed, and of those equal to it the first `top` of each warp's share of the part, of which the first of all
    // are some.  (Where too many are above it the list is left overfull.)  A call, with few arguments:
    // the team's own registers are those of the rows.  8 x 128256 with all but 50 values masked 190 us when the
    // top-th key was searched for at once, 2048 x 32000 with all but 10, top 20, 7.8 ms.
    static __device__ __noinline__ void list_beside_equal(LogShared<NW, LIST>& sh, const T* row, int n, int tid, int turn, int top, float floor)
    {
        const LogPart<T> p(row, n);
        const int lane = tid & 31, warp = tid >> 5;
        int& count = sh.listed[turn];
        auto put = [&](unsigned long long k) {
            const int at = atomicAdd(&count, 1);
            if (at < LIST) sh.list[at] = k;
        };
        if (tid < p.odd && !(sh.odd[tid] < floor)) put(key_of(sh.odd[tid], p.place_of_odd(tid)));
        float lo, hi;
#pragma unroll 1
        for (int i = tid; i < p.vecs && !overfull(count); i += TEAM) {
            const Vec<T> w(ld_global_v4(p.vec(i)));
#pragma unroll
            for (int e = 0; e < Vec<T>::P; ++e) {
                w.pair(e, lo, hi);
                if (!(lo <= floor)) put(key_of(lo, p.head + i * V + 2 * e));        // (not-a-number is above)
                if (!(hi <= floor)) put(key_of(hi, p.head + i * V + 2 * e + 1));
            }
        }
        sync();
        const bool room = count + NW * top <= LIST;
        sync();
        if (!room) {
            if (tid == 0) count = LIST + 1;
            return;
        }
        const int share = (p.vecs + NW - 1) / NW, end = min(p.vecs, (warp + 1) * share);
        int found = 0;
#pragma unroll 1
        for (int i0 = warp * share; i0 < end && found < top; i0 += 32) {
            const int i = i0 + lane;
            unsigned same = 0u;                                 // which of the vector's values
            if (i < end) {
                const Vec<T> w(ld_global_v4(p.vec(i)));
#pragma unroll
                for (int e = 0; e < Vec<T>::P; ++e) {
                    w.pair(e, lo, hi);
                    same |= (lo == floor ? 1u : 0u) << (2 * e) | (hi == floor ? 2u : 0u) << (2 * e);
                }
            }
            const int mine = __popc(same);
            int until = mine;                                   // in this lane and those before it
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, until, o);
                if (lane >= o) until += v;
            }
            for (int at = found + until - mine; same != 0u && at < top; same &= same - 1u, ++at) put(key_of(floor, p.head + i * V + __ffs(same) - 1));
            found += __shfl_sync(0xffffffffu, until, 31);
        }
    }
    // The sums of the warps and, in order, the part's `top` largest keys (places within the part), for the first warp.
    __device__ __forceinline__ void finish(const LogPart<T>& p)
    {
        constexpr int kEach = NW == 1 ? 0 : 32 / NW > 4 ? 32 / NW : 4;   // that a warp names at least
        const int full = min(NW, p.vecs / 32);                  // warps all of whose threads have values
        const int each = full == 0 ? 0 : max(kEach, (a.top + full - 1) / full);
        unsigned least = 0u;
        if (a.top > 0) {
            unsigned mine = value_bits(largest);
            unsigned* const named = reinterpret_cast<unsigned*>(sh.named);
            for (int q = 0; q < each && warp < full; ++q) {
                const unsigned best = __reduce_max_sync(0xffffffffu, mine);
                const unsigned who = __ballot_sync(0xffffffffu, mine == best);
                if (lane == __ffs(who) - 1) mine = 0u;
                if (NW == 1) least = best;                      // (the last one stands)
                else if (lane == 0) named[warp * each + q] = best;
            }
            if (NW > 1 && tid < kNamed && tid >= full * each) named[tid] = 0u;
        }
        const Sums all = joined(sum);
        if (lane == 0) sh.sums[turn][warp] = all;
        sync();
        if (a.top == 0) return;
        if (NW > 1) {                                           // the top-th of those named, by every warp for itself
            constexpr int kTwo = NW * kEach > 32 ? 2 : 1;
            const unsigned* const named = reinterpret_cast<const unsigned*>(sh.named);
            if (full * each <= 32 * kTwo) {
                unsigned v[kTwo];
                int before[kTwo];
#pragma unroll
                for (int h = 0; h < kTwo; ++h) v[h] = named[h * 32 + lane], before[h] = 0;
#pragma unroll
                for (int j = 0; j < 8 * kTwo; ++j) {
                    const uint4 o = sh.named[j];
#pragma unroll
                    for (int h = 0; h < kTwo; ++h) before[h] += (o.x > v[h]) + (o.y > v[h]) + (o.z > v[h]) + (o.w > v[h]);
                }
                // (of equal ones any: the least of those with fewer than `top` before them)
#pragma unroll
                for (int h = 0; h < kTwo; ++h) {
                    const unsigned k = __reduce_min_sync(0xffffffffu, before[h] < a.top ? v[h] : 0xffffffffu);
                    least = h == 0 ? k : min(least, k);
                }
            } else {                                            // few warps with values, which name up to 32 each: the least of all
                least = 0xffffffffu;
                for (int j = lane; j < full * each; j += 32) least = min(least, named[j]);
                least = __reduce_min_sync(0xffffffffu, least);
            }
        }
        const float floor = least == 0u ? -INFINITY : value_of(least);
        const int rounds = (p.vecs + TEAM * kVecs - 1) / (TEAM * kVecs);
        // the slots whose largest reaches the bound, or of threads who have met not-a-number; their vectors, by all threads
        const bool strange = sum.s != sum.s;
        if (value_bits(largest) >= least || strange)
            for (int k = 0; k << slot_shift < rounds; ++k)
                if (strange || sh.tops[k][tid] >= floor) sh.who[atomicAdd(&sh.reached[turn], 1)] = (unsigned short)(k * TEAM + tid);
        sync();
        const int shift = slot_shift + 2, pairs = sh.reached[turn] << shift;
        static_assert(kVecs == 4, "vectors of a round: two bits");
        for (int x = tid; x < pairs; x += TEAM) {
            const int k = sh.who[x >> shift], v = x & ((1 << shift) - 1);
            const int i = ((k / TEAM << slot_shift) + (v >> 2)) * (TEAM * kVecs) + (v & 3) * TEAM + k % TEAM;
            if (i >= p.vecs) continue;
            if (pairs > LIST / 2 && overfull(sh.listed[turn])) break;   // (they are looked at anew below; few pairs are through sooner)
            const Vec<T> w(ld_global_v4(p.vec(i)));
            float lo, hi, any = 0.0f;
#pragma unroll
            for (int e = 0; e < Vec<T>::P; ++e) {
                w.pair(e, lo, hi);
                any += lo + hi;                                 // (not-a-number if one of them is)
            }
            if (w.top() >= floor || any != any) {
#pragma unroll
                for (int e = 0; e < Vec<T>::P; ++e) {
                    w.pair(e, lo, hi);
                    if (!(lo < floor)) put(key_of(lo, p.head + i * V + 2 * e));
                    if (!(hi < floor)) put(key_of(hi, p.head + i * V + 2 * e + 1));
                }
            }
        }
        if (tid < p.odd && !(sh.odd[tid] < floor)) put(key_of(sh.odd[tid], p.place_of_odd(tid)));
        sync();
        int listed = sh.listed[turn];
        if (listed > LIST && least != 0u) {                    // (every warp has the same bound)
            sync();
            if (tid == 0) sh.listed[turn] = 0;
            sync();
            list_beside_equal(sh, p.row, p.odd + p.vecs * V, tid, turn, a.top, floor);
            sync();
            listed = sh.listed[turn];
        }
        if (listed > LIST) {                                    // the top-th largest key, bit by bit
            // each value of the part with its place
            auto each_key = [&](auto f) {
                if (tid < p.odd) f(key_of(sh.odd[tid], p.place_of_odd(tid)));
#pragma unroll 1
                for (int i = tid; i < p.vecs * V; i += TEAM) f(key_of((float)p.row[p.head + i], p.head + i));
            };
            unsigned long long from = 0ull;
#pragma unroll 1
            for (int bit = 63; bit >= 0; --bit) {
                const unsigned long long trial = from | 1ull << bit;
                int c = 0;
                each_key([&](unsigned long long k) { c += k >= trial; });
                c = __reduce_add_sync(0xffffffffu, c);
                sync();
                if (tid == 0) sh.votes = 0;
                sync();
                if (lane == 0) atomicAdd(&sh.votes, c);
                sync();
                if (sh.votes >= a.top) from = trial;
            }
            sync();
            if (tid == 0) sh.listed[turn] = 0;
            sync();
            each_key([&](unsigned long long k) {
                if (k >= from) put(k);                          // (keys are distinct: these are `top`, or all of the part)
            });
            sync();
            listed = sh.listed[turn];
        }
        const bool many = NW > 1 && listed > 128;               // then all threads look for the places, else the first warp alone
        if (warp > 0 && !many) return;
        if (tid < a.top && listed < a.top) sh.mine[tid] = 0ull;
        if (many) sync();
        else __syncwarp();
        for (int i = tid; i < listed; i += many ? TEAM : 32) {
            const unsigned long long k = sh.list[i];
            int before = 0;
            for (int j = 0; j < listed; ++j) before += sh.list[j] > k;
            if (before < a.top) sh.mine[before] = k;
        }
        if (many) sync();
        else __syncwarp();
    }
    __device__ __forceinline__ Sums all_sums() const { return joined(lane < NW ? sh.sums[turn][lane] : Sums{-INFINITY, 0.0f, 0.0f}); }
};

// The row's answers from its sums, by the threads that have a key or are the first.
struct LogAnswer {
    const LogArgs& a;
    size_t r;
    float m, logsum, mean;
    bool none;
    __device__ __forceinline__ LogAnswer(const LogArgs& args, size_t row, const Sums& x)
        : a(args), r(row), m(x.m), logsum(logf(x.s)), mean(x.t / x.s),
          none(!(fabsf(x.m) < INFINITY) || x.s != x.s)          // (a row of -infinity alone, or with not-a-number or +infinity)
    {
    }
    static __device__ __forceinline__ float nan() { return __int_as_float(0x7fffffff); }
    __device__ __forceinline__ void scalars(bool wanted, float chosen) const
    {
        if (a.logprob) a.logprob[r] = none || !wanted ? nan() : (chosen - m) - logsum;
        if (a.entropy) a.entropy[r] = none ? nan() : logsum - mean;
    }
    __device__ __forceinline__ void place(int i, unsigned long long k) const
    {
        a.top_index[r * a.top + i] = place_of(k);
        a.top_logprob[r * a.top + i] = none ? nan() : (value_of((unsigned)(k >> 32)) - m) - logsum;
    }
};

// Rows one after the other, a team of threads each: the values of the next 4 vectors of a thread, be they of the next row, are on
// their way while those before are added or the row is finished.
template <class T, int TEAM>
__global__ void __launch_bounds__(256, 4) token_logprobs_rows_kernel(const LogArgs a, unsigned rows)
{
    constexpr int kTeams = 256 / TEAM, kList = TEAM == 32 ? 256 : TEAM == 128 ? 1024 : kLogList;
    __shared__ LogShared<TEAM / 32, kList> shared[kTeams];
    const int which = threadIdx.x / TEAM, tid = threadIdx.x % TEAM;
    LogTeam<T, TEAM, kList> team = {shared[which], a, tid, (int)threadIdx.x & 31, tid >> 5, 0, {}, 0.0f, 0, 0.0f};
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const T* const logits = static_cast<const T*>(a.logits);
    uint4 w[kVecs];
    // (unsigned: a row number plus a step passes 2^31 where there are nearly so many rows)
    unsigned r = blockIdx.x * kTeams + which;
    const unsigned step = gridDim.x * kTeams;
    if (r < rows) team.load(w, LogPart<T>(logits + (long long)r * a.row_stride, a.vocab), tid);
    for (; r < rows; r += step) {
        const LogPart<T> part(logits + (long long)r * a.row_stride, a.vocab);
        const int token = a.tokens && tid == 0 ? (int)ld_global_u32(a.tokens + r) : -1;
        const bool wanted = (unsigned)token < (unsigned)a.vocab;
        const float chosen = wanted ? (float)part.row[token] : 0.0f;
        team.begin(part);
        for (int i0 = 0; i0 == 0 || i0 < part.vecs; i0 += TEAM * kVecs) {
            uint4 next[kVecs];
            if (i0 + TEAM * kVecs < part.vecs) team.load(next, part, i0 + TEAM * kVecs + tid);
            else if (r + step < rows) team.load(next, LogPart<T>(logits + (long long)(r + step) * a.row_stride, a.vocab), tid);
            team.add(w, part, i0 + tid, i0 / (TEAM * kVecs));
#pragma unroll
            for (int u = 0; u < kVecs; ++u) w[u] = next[u];
        }
        team.finish(part);
        if (team.warp == 0) {
            const LogAnswer answer(a, r, team.all_sums());
            if (tid == 0) answer.scalars(wanted, chosen);
            if (tid < a.top) answer.place(tid, team.sh.mine[tid]);
            __syncwarp();
        }
        team.turn ^= 1;
    }
}

// A row for the CTAs of a cluster, a part each, which meet in the first one.
constexpr int kPartThreads = 512;
template <class T>
__global__ void __launch_bounds__(kPartThreads, 2) token_logprobs_parts_kernel(const LogArgs a)
{
    __shared__ LogShared<kPartThreads / 32, kLogList> shared;
    __shared__ LogClusterShared meet;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    LogTeam<T, kPartThreads, kLogList> team = {shared, a, tid, lane, warp, 0, {}, 0.0f, 0, 0.0f};
    const int ctas = (int)gridDim.x, rank = (int)blockIdx.x, r = (int)blockIdx.y;
    const int first = rank * a.part, n = max(0, min(a.part, a.vocab - first));
    cluster_arrive();
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const T* const row = static_cast<const T*>(a.logits) + (long long)r * a.row_stride;
    const int token = a.tokens && rank == 0 && tid == 0 ? (int)ld_global_u32(a.tokens + r) : -1;
    const LogPart<T> part(row + first, n);
    uint4 w[kVecs];
    team.load(w, part, tid);
    team.begin(part);
    for (int i0 = 0; i0 < part.vecs;) {
        team.add(w, part, i0 + tid, i0 / (kPartThreads * kVecs));
        i0 += kPartThreads * kVecs;
        if (i0 < part.vecs) team.load(w, part, i0 + tid);
    }
    const bool wanted = (unsigned)token < (unsigned)a.vocab;
    const float chosen = wanted ? (float)row[token] : 0.0f;
    team.finish(part);
    cluster_wait();                                             // (all CTAs have begun)
    if (warp == 0) {
        const Sums mine = team.all_sums();
        if (lane == 0) {
            const unsigned to = in_first_cta(&meet.parts[rank]);
            asm volatile("st.shared::cluster.f32 [%0], %1;\n\tst.shared::cluster.f32 [%0+4], %2;\n\tst.shared::cluster.f32 [%0+8], %3;" ::"r"(to), "f"(mine.m),
                         "f"(mine.s), "f"(mine.t)
                         : "memory");
        }
        if (lane < a.top) {
            const unsigned long long k = shared.mine[lane];     // (places of the whole row)
            const unsigned long long whole = k == 0ull ? 0ull : k - (unsigned)first;
            asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(in_first_cta(&meet.best[rank * a.top + lane])), "l"(whole) : "memory");
        }
    }
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    if (rank != 0) return;                                      // (the first CTA stays until all have sent)
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    const LogAnswer answer(a, r, joined(lane < ctas ? meet.parts[lane] : Sums{-INFINITY, 0.0f, 0.0f}));
    if (tid == 0) answer.scalars(wanted, chosen);
    const int keys = ctas * a.top;
    if (tid < keys) {
        const unsigned long long k = meet.best[tid];
        int before = 0;
        for (int j = 0; j < keys; ++j) before += meet.best[j] > k;
        if (k != 0ull && before < a.top) answer.place(before, k);
    }
}

template <class T>
cudaError_t launch_logprobs(LogArgs a, int rows, cudaStream_t s)
{
    const int sms = sm_count();
    if (sms <= 0) return cudaErrorInvalidDevice;
    constexpr int V = Vec<T>::N;
    // CTAs per row: more while there are fewer CTAs than two per SM and a thread would still have a vector of each part.
    int ctas = 1;
    auto part_of = [&](int c) { return ((a.vocab + c - 1) / c + V - 1) / V * V; };
    while (ctas < kMaxLogCtas && (long long)rows * ctas < 2 * sms && part_of(2 * ctas) >= kPartThreads * V) ctas *= 2;
    if (ctas == 1) {
        auto rows_by = [&](auto kernel, int team) {
            const int teams = 256 / team, grid = (rows - 1) / teams + 1;
            return launch_overlapping(kernel, dim3(grid < 4 * sms ? grid : 4 * sms), 256, 0, s, a, rows);
        };
        // fp16, a warp / 128 threads a row, top 5 and top 20: 1000 x 2000 5.6 / 7.1 and 9.1 / 7.7 us; 4000 x 2000 9.6 / 23.1 and 15.7 / 25.0;
        // 1000 x 4000 9.7 / 7.9 and 11.2 / 8.4; 2000 x 8000 16.1 / 16.7 and 21.3 / 18.3; 4096 x 8000 24.0 / 31.7 and 30.1 / 34.7.
        // 128 / 256 threads, top 20: 2048 x 32000 38.3 / 46.2; 512 x 128256 37.9 / 34.7
        if (a.vocab <= 2048 || (a.vocab <= 8192 && rows >= 16 * sms)) return rows_by(token_logprobs_rows_kernel<T, 32>, 32);
        if ((size_t)a.vocab * sizeof(T) <= 65536) return rows_by(token_logprobs_rows_kernel<T, 128>, 128);
        return rows_by(token_logprobs_rows_kernel<T, 256>, 256);
    }
    a.part = part_of(ctas);
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(kPartThreads);
    cfg.gridDim = dim3(ctas, rows);                             // (fewer rows than two per SM)
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ctas;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = g_no_pdl ? attr + 1 : attr;
    cfg.numAttrs = g_no_pdl ? 1 : 2;
    const cudaError_t err = cudaLaunchKernelEx(&cfg, token_logprobs_parts_kernel<T>, a);
    if (err == cudaSuccess) count_launch();
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
    const LogArgs a = {logits, row_stride, tokens, logprob, entropy, top_logprob, top_index, vocab, top, 0};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return launched(dtype == SPQT_LOGITS_FP16   ? launch_logprobs<__half>(a, rows, s)
                    : dtype == SPQT_LOGITS_BF16 ? launch_logprobs<__nv_bfloat16>(a, rows, s)
                                                : launch_logprobs<float>(a, rows, s));
}
