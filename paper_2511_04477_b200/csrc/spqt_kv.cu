// The 8-bit cache but for the attention over it: new tokens (with the rounding of blocks that become full), the cache as fp16,
// and the eviction of blocks.
#include <cuda_fp8.h>

#include "spqt_common.cuh"
#include "spqt_gemv_device.cuh"
#include "spqt_kv.cuh"

namespace spqt {

// ---------------------------------------------------------------- eight values to codes and back

// x / s rounded to the nearest whole number, ties to even, in one rounding: q is the whole number next to x * (1/s), which is off
// by one at most where x/s is within 2^-16 of a tie; x - q*s is exact (|q| < 2^7 times 24 bits of s, of which x is a neighbour),
// and says on which side of the tie x/s lies.
__device__ __forceinline__ unsigned to_int8(float x, float s, float inv)
{
    constexpr float kMagic = 12582912.0f;   // 1.5 * 2^23: its sum's last bits are the whole number
    float t = fmaf(x, inv, kMagic);
    const float r = fmaf(-(t - kMagic), s, x);
    const float a = 2.0f * fabsf(r);
    if (a >= s && (a > s || (__float_as_uint(t) & 1u))) t += copysignf(1.0f, r);
    return __float_as_uint(t) & 0xffu;
}

// x / s in fp32 with its last bit set where the quotient is not exact: a second rounding to few bits then gives what one rounding
// of the exact quotient gives.  q is x/s to the last place or next to it, and the sign of x - q*s (exact in an FMA) says between
// which two neighbours x/s lies.
__device__ __forceinline__ float quotient_to_odd(float x, float s, float inv)
{
    const float q0 = x * inv;
    const float q = fmaf(fmaf(-q0, s, x), inv, q0);
    const float r = fmaf(-q, s, x);
    const unsigned bits = __float_as_uint(q);
    const unsigned over = (__float_as_uint(r) ^ bits) >> 31;     // |q| > |x/s|
    return __uint_as_float((r == 0.0f ? bits : (bits - over) | 1u) | (__float_as_uint(x) & 0x80000000u));   // (-0 / s is -0)
}

template <int FMT>
__device__ __noinline__ uint2 to_codes_exactly(uint4 h, float s, float inv)
{
    const __half2* p = reinterpret_cast<const __half2*>(&h);
    unsigned w[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(p[i]);
        unsigned pair;
        if (FMT == SPQT_KV_INT8)
            pair = to_int8(f.x, s, inv) | to_int8(f.y, s, inv) << 8;
        else
            pair = __nv_cvt_float2_to_fp8x2(make_float2(quotient_to_odd(f.x, s, inv), quotient_to_odd(f.y, s, inv)), __NV_SATFINITE, __NV_E4M3);
        w[i >> 1] |= pair << (16 * (i & 1));
    }
    return make_uint2(w[0], w[1]);
}

// Eight values.  x * (1/s) in fp32, within 2^-23 of x/s relative to it, rounds as x/s does unless a tie lies that near: where one of
// the eight is near a tie the exact steps above are taken for them, which happens for one in hundreds (they are 30 instructions
// a value, these 6: a prompt's 30 million values 34 us with them alone).
template <int FMT>
__device__ __forceinline__ uint2 to_codes(const uint4& h, float s, float inv)
{
    const unsigned u[4] = {h.x, h.y, h.z, h.w};
    unsigned w[2];
    bool near = false;
    if (FMT == SPQT_KV_INT8) {
        constexpr float kMagic = 12582912.0f;   // 1.5 * 2^23: its sum's last bits are the whole number
        const unsigned long long i2 = pack2(inv, inv), s2 = pack2(-s, -s), m2 = pack2(kMagic, kMagic), n2 = pack2(-kMagic, -kMagic);
        float far = 0.0f;
        unsigned t[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
            const unsigned long long x = pack2(f.x, f.y);
            const unsigned long long q = fma2(x, i2, m2), r = fma2(fadd2(q, n2), s2, x);   // r, what is left of x, is exact
            float lo, hi;
            unpack2(r, lo, hi);
            far = fmaxf(far, fmaxf(fabsf(lo), fabsf(hi)));
            unpack2(q, lo, hi);
            t[2 * i] = __float_as_uint(lo), t[2 * i + 1] = __float_as_uint(hi);
        }
        near = far >= s * 0.49993896484375f;    // 1/2 - 2^-14
#pragma unroll
        for (int i = 0; i < 2; ++i)
            w[i] = __byte_perm(__byte_perm(t[4 * i], t[4 * i + 1], 0x0040), __byte_perm(t[4 * i + 2], t[4 * i + 3], 0x0040), 0x5410);
    } else {
        const unsigned long long i2 = pack2(inv, inv);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            unsigned pair[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[2 * i + k]));
                float lo, hi;
                unpack2(fmul2(pack2(f.x, f.y), i2), lo, hi);
                pair[k] = __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
                // a tie has 1000... behind the three bits that stay; below 2^-6 fewer stay, and zero is no tie
                const unsigned a = __float_as_uint(lo) & 0x7fffffffu, b = __float_as_uint(hi) & 0x7fffffffu;
                near = near || ((a + 0x80008u) & 0xfffffu) < 0x11u || ((b + 0x80008u) & 0xfffffu) < 0x11u || a - 1u < 0x3c800000u - 1u || b - 1u < 0x3c800000u - 1u;
            }
            w[i] = pair[0] | pair[1] << 16;
        }
    }
    return near ? to_codes_exactly<FMT>(h, s, inv) : make_uint2(w[0], w[1]);
}

// Eight codes times their scale, rounded to fp16.
template <int FMT>
__device__ __forceinline__ uint4 from_codes(const uint2& w, float s)
{
    const unsigned long long s2 = pack2(s, s);
    unsigned h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float2 f;
        if (FMT == SPQT_KV_INT8) {              // code + 128 under the exponent of 1024: 1152 + code
            const unsigned v = __byte_perm((i < 2 ? w.x : w.y) ^ 0x80808080u, 0x64646464u, i & 1 ? 0x4342 : 0x4140);
            f = __half22float2(__hsub2(*reinterpret_cast<const __half2*>(&v), __half2half2(__ushort_as_half(0x6480))));
        } else {
            f = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)((i < 2 ? w.x : w.y) >> (16 * (i & 1)) & 0xffffu), __NV_E4M3)));
        }
        float lo, hi;
        unpack2(fmul2(pack2(f.x, f.y), s2), lo, hi);
        const __half2 r = __floats2half2_rn(lo, hi);
        h[i] = *reinterpret_cast<const unsigned*>(&r);
    }
    return make_uint4(h[0], h[1], h[2], h[3]);
}

// ---------------------------------------------------------------- new tokens

// A CTA works on one touched block of one stream: its first half of threads on the keys, the second on the values, a thread on up
// to PPT 16-byte pieces of the block's rows, which stay in registers between the maximum and the rounding, so that every row is
// read once.  Memory is what bounds a prompt: 4 bytes read and 2 written per value pair; heads of a block of tokens are neighbours
// in the grid, since their rows are neighbours in memory.
struct AppendArgs {
    spqt_kv_cache c;
    const __half *k, *v;
    int tokens;
    long long batch_stride, token_stride;
    const int32_t* counts;
    int32_t* length_out;
    int* status;
};

template <int FMT, int D, int PPT, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 256 ? 6 : 1) kv_append_kernel(const AppendArgs a)
{
    __shared__ unsigned s_max[32];
    const spqt_kv_cache& c = a.c;
    const int tid = threadIdx.x, half = blockDim.x >> 1, warp = tid >> 5;
    const int h = blockIdx.x, j = blockIdx.y, b = blockIdx.z;
    const int stream = b * c.kv_heads + h, bt = c.block_tokens;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    const int held = (int)ld_global_u32(c.length + stream);
    int count = a.counts ? (int)ld_global_u32(a.counts + b) : a.tokens;
    const int n = length_or_none(held, c, a.status);
    if (count < 0 || count > a.tokens) {
        refuse(a.status);
        count = 0;
    }
    const int shift = 31 - __clz(bt), first = n >> shift, before = n & (bt - 1);
    const long long end = (long long)n + count;
    const int total = before + count;               // rows from the beginning of block `first` on
    const int touched = (total + bt - 1) >> shift, closed = total >> shift;
    const bool values = tid >= half;
    const int t = values ? tid - half : tid;
    const __half* const fresh = (values ? a.v : a.k) + (long long)b * a.batch_stride + (long long)h * D;
    __half* const tail = static_cast<__half*>(values ? c.v_tail : c.k_tail) + (size_t)stream * bt * D;
    constexpr int kRow = D / 8;                     // pieces of a row
    const int r0 = t / kRow, col = t % kRow * 8, step = half / kRow;   // a thread's pieces lie `step` rows apart (half is a multiple of kRow)
    // (the rows are on their way while the table is looked at)
    uint4 x[PPT];
    const __half* src = fresh + (long long)(j * bt + r0 - before) * a.token_stride + col;
#pragma unroll
    for (int i = 0; i < PPT; ++i) {
        const int r = r0 + i * step;
        x[i] = ld_global_v4_if(j < closed && r < bt, j * bt + r < before ? tail + r * D + col : src);
        src += step * a.token_stride;
    }
    bool fine = held == n && end <= (long long)c.table_width * bt;
    const int32_t* const row = c.table + (size_t)stream * c.table_width + first;
    if (count > 0) {                                // every CTA of the stream comes to the same verdict
        bool bad = false;
        if (fine)
            for (int i = tid; i < touched; i += blockDim.x) bad = bad || (unsigned)row[i] >= (unsigned)c.blocks;
        fine = !__syncthreads_or(bad) && fine;
        if (!fine) refuse(a.status);
    }
    if (!fine || count == 0) {
        if (j == 0 && tid == 0 && a.length_out) a.length_out[stream] = held;
        return;
    }
    if (j >= touched) return;
    const size_t block = (size_t)row[j];

    if (c.weight) {
        const int from = j == 0 ? before : 0, to = min(bt, total - j * bt);
        for (int i = from + tid; i < to; i += blockDim.x) c.weight[block * bt + i] = 0.0f;
    }
    if (j < closed) {
        unsigned top = 0u;
#pragma unroll
        for (int i = 0; i < PPT; ++i) {
            // (magnitudes of fp16 in the order of their bits, not-a-number above infinity)
            top = __vmaxu2(top, __vmaxu2(__vmaxu2(x[i].x & 0x7fff7fffu, x[i].y & 0x7fff7fffu), __vmaxu2(x[i].z & 0x7fff7fffu, x[i].w & 0x7fff7fffu)));
        }
        top = __reduce_max_sync(0xffffffffu, max(top & 0xffffu, top >> 16));
        if ((tid & 31) == 0) s_max[warp] = top;
        __syncthreads();
        const int w0 = values ? half >> 5 : 0;
        for (int w = 0; w < half >> 5; ++w) top = max(top, s_max[w0 + w]);
        const bool poisoned = top >= 0x7c00u;
        const float amax = __half2float(__ushort_as_half((unsigned short)top));
        // amax / 127 or 448, correctly rounded: the quotient by the reciprocal, and what it leaves (every fp16 value has been tried)
        constexpr float kMost = FMT == SPQT_KV_INT8 ? 127.0f : 448.0f, kInv = 1.0f / kMost;
        const float q = amax * kInv, exact = fmaf(fmaf(-q, kMost, amax), kInv, q);
        const float s = poisoned ? __int_as_float(0x7fffffff) : exact;
        const float inv = s > 0.0f ? __fdividef(1.0f, s) : 0.0f;
        uint2* const dst = reinterpret_cast<uint2*>(static_cast<unsigned char*>(values ? c.v_codes : c.k_codes) + block * bt * D);
#pragma unroll
        for (int i = 0; i < PPT; ++i)
            if (r0 + i * step < bt) dst[i * half + t] = poisoned ? make_uint2(0u, 0u) : to_codes<FMT>(x[i], s, inv);
        if (t == 0) (values ? c.v_scale : c.k_scale)[block] = s;
    }
    if (j != 0) return;
    // The CTA that has read the tail is the one that writes it, behind its last read.
    __syncthreads();
    const int base = closed * bt;                   // the first row of the block that stays open
    const int from = closed > 0 ? 0 : before, rows = total - base;
    for (int p = from * kRow + t; p < rows * kRow; p += half)
        *reinterpret_cast<uint4*>(tail + p * 8) = ld_global_v4(fresh + (long long)(base + p / kRow - before) * a.token_stride + p % kRow * 8);
    if (tid == 0 && a.length_out) a.length_out[stream] = (int)end;
}

// Lengths in place of the old ones, behind a kernel several of whose CTAs read the old one.
__global__ void kv_lengths_kernel(const int32_t* from, int32_t* to, int n)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i < n) to[i] = from[i];
}

template <int FMT, int D>
cudaError_t launch_append(const AppendArgs& a, cudaStream_t s)
{
    const int bt = a.c.block_tokens, pieces = bt * D / 8;
    // (blocks behind the table's last are refused by the first CTA of the stream)
    const int touched = (int)(((long long)a.tokens + 2 * bt - 2) / bt), most = a.c.table_width;
    const dim3 grid((unsigned)a.c.kv_heads, (unsigned)(touched < most ? touched : most), (unsigned)a.c.batch);
    // threads for one of k and v: a multiple of a warp and of a row's pieces
    constexpr int kUnit = D == 96 ? 96 : 32;
    if constexpr (D == 256) {                       // (blocks of 128 tokens: eight pieces a thread)
        if (pieces > 2048) return launch_overlapping(kv_append_kernel<FMT, D, 8, 1024>, grid, 1024, 0, s, a);
    }
    const int half = (pieces / 4 + kUnit - 1) / kUnit * kUnit;
    if (half <= 128) return launch_overlapping(kv_append_kernel<FMT, D, 4, 256>, grid, 2 * half, 0, s, a);
    return launch_overlapping(kv_append_kernel<FMT, D, 4, 1024>, grid, 2 * half, 0, s, a);
}

// ---------------------------------------------------------------- the cache as fp16

struct ReadArgs {
    spqt_kv_cache c;
    const int32_t* length;
    __half *k, *v;
    int tokens;
    long long batch_stride, token_stride, head_stride;
    int* status;
};

constexpr int kReadTokens = 16, kReadWarps = 8;   // of a warp: a part of one block of a stream; of a CTA

// A warp turns sixteen tokens of a stream, a piece of one block or of the tail; the warps of the heads of the same tokens are
// neighbours, since their rows are neighbours in the output.
template <int FMT, int D>
__global__ void __launch_bounds__(kReadWarps * 32) kv_read_kernel(const ReadArgs a)
{
    const spqt_kv_cache& c = a.c;
    constexpr int kRow = D / 8, N = kReadTokens * kRow / 32;   // pieces of eight values: of a row, of a lane
    const int lane = threadIdx.x & 31, w = blockIdx.x * kReadWarps + (threadIdx.x >> 5), b = blockIdx.y;
    const int h = w % c.kv_heads, t0 = w / c.kv_heads * kReadTokens, bt = c.block_tokens, shift = 31 - __clz(bt), j = t0 >> shift;
    const int stream = b * c.kv_heads + h;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (t0 >= a.tokens) return;
    // (t0 < a.tokens <= table_width * bt: the entry is there, whatever it holds)
    const unsigned block = (unsigned)c.table[(size_t)stream * c.table_width + j];
    const int n = length_or_none(a.length[stream], c, a.status), last = min(n, a.tokens);
    if (t0 >= last) return;
    long long to = (long long)b * a.batch_stride + (long long)h * a.head_stride;
    uint4 k[N], v[N];
    if (t0 < n >> shift << shift) {
        const bool known = block < (unsigned)c.blocks;
        const size_t id = known ? block : 0u, at = ((id << shift) + (t0 & (bt - 1))) * D + lane * 8;
        uint2 kc[N], vc[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            kc[i] = *reinterpret_cast<const uint2*>(static_cast<const unsigned char*>(c.k_codes) + at + i * 256);
            vc[i] = *reinterpret_cast<const uint2*>(static_cast<const unsigned char*>(c.v_codes) + at + i * 256);
        }
        float ks = c.k_scale[id], vs = c.v_scale[id];
        if (!known) {
            refuse(a.status);
            ks = vs = __int_as_float(0x7fffffff);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int p = i * 32 + lane, t = t0 + p / kRow;
            if (t >= last) continue;
            const long long at = to + (long long)t * a.token_stride + p % kRow * 8;
            *reinterpret_cast<uint4*>(a.k + at) = from_codes<FMT>(kc[i], ks);
            *reinterpret_cast<uint4*>(a.v + at) = from_codes<FMT>(vc[i], vs);
        }
    } else {
        const size_t at = (((size_t)stream << shift) + (t0 & (bt - 1))) * D + lane * 8;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            k[i] = *reinterpret_cast<const uint4*>(static_cast<const __half*>(c.k_tail) + at + i * 256);
            v[i] = *reinterpret_cast<const uint4*>(static_cast<const __half*>(c.v_tail) + at + i * 256);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int p = i * 32 + lane, t = t0 + p / kRow;
            if (t >= last) continue;
            const long long at = to + (long long)t * a.token_stride + p % kRow * 8;
            *reinterpret_cast<uint4*>(a.k + at) = k[i];
            *reinterpret_cast<uint4*>(a.v + at) = v[i];
        }
    }
}

// ---------------------------------------------------------------- eviction

constexpr int kMostEvictWarps = 32;
constexpr int kOwnKeys = 16;      // keys of a lane, where one warp or four look for the bound
constexpr int kBoundWarps = 4;    // (128 threads are the fewest of a CTA)

struct EvictArgs {
    spqt_kv_cache c;
    int keep, first, recent;
    int32_t *table_out, *length_out;
    int* status;
};

// Whole numbers in the order of fp32 values, not-a-number above all, zeros of both signs alike.
__device__ __forceinline__ unsigned ordered(float f)
{
    if (f != f) return 0xffffffffu;
    const unsigned u = __float_as_uint(f + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Sums over 2^k neighbouring lanes of N values each: lanes exchange halves of what they still have, then (one value left) add.  A lane's
// result is of value `which`.
template <int N, int LANES>
__device__ __forceinline__ double sums_over(const double* v, int lane, int bit, int* which)
{
    if constexpr (LANES == 1) {
        return v[0];
    } else if constexpr (N > 1) {
        const bool upper = (lane & bit) != 0;
        double w[N / 2];
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const double keep = upper ? v[i + N / 2] : v[i], send = upper ? v[i] : v[i + N / 2];
            w[i] = keep + __shfl_xor_sync(0xffffffffu, send, bit);
        }
        if (upper) *which += N / 2;
        return sums_over<N / 2, LANES / 2>(w, lane, bit << 1, which);
    } else {
        const double w = v[0] + __shfl_xor_sync(0xffffffffu, v[0], bit);
        return sums_over<1, LANES / 2>(&w, lane, bit << 1, which);
    }
}

// How many of the CTA's values are true, and how many are in threads before this one (in thread order).
__device__ __forceinline__ int count_before(bool v, int* s_warps, int* all)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const unsigned mask = __ballot_sync(0xffffffffu, v);
    __syncthreads();                        // (s_warps may still be read)
    if (lane == 0) s_warps[warp] = __popc(mask);
    __syncthreads();
    const int mine = lane < warps ? s_warps[lane] : 0;
    *all = __reduce_add_sync(0xffffffffu, mine);
    return __reduce_add_sync(0xffffffffu, lane < warp ? mine : 0) + __popc(mask & ((1u << lane) - 1u));
}

// The m-th largest of `count` keys, by WARPS warps (0: by the whole CTA) which call this together: the keys' bits from the top, two a
// step, since three counts take hardly longer than one.  `key`: it; `equal`: how many of the keys equal to it are among the m;
// `exactly`: all are.  A thread keeps up to KEYS keys in registers, or (KEYS 0) reads them anew for each step.
template <int KEYS, int WARPS>
__device__ __forceinline__ void find_bound(const unsigned* keys, int count, int m, int4 (*s_count)[kMostEvictWarps], unsigned* key, int* equal, bool* exactly)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int warps = WARPS ? WARPS : blockDim.x >> 5, threads = warps * 32;
    unsigned k[KEYS ? KEYS : 1];
    if constexpr (KEYS > 0) {
#pragma unroll
        for (int i = 0; i < KEYS; ++i) k[i] = i * threads + tid < count ? keys[i * threads + tid] : 0u;   // (0 reaches no trial)
    }
    const int mine = (count + threads - 1) / threads;
    int parity = 0;
    auto reach = [&](unsigned t1, unsigned t2, unsigned t3) {
        int3 c = make_int3(0, 0, 0);
        if constexpr (KEYS > 0) {
#pragma unroll
            for (int i = 0; i < KEYS; i += 4) {
                if (i >= mine) break;
#pragma unroll
                for (int e = 0; e < 4; ++e) c.x += k[i + e] >= t1, c.y += k[i + e] >= t2, c.z += k[i + e] >= t3;
            }
        } else {
            for (int j = tid; j < count; j += threads) {
                const unsigned v = keys[j];
                c.x += v >= t1, c.y += v >= t2, c.z += v >= t3;
            }
        }
        c.x = __reduce_add_sync(0xffffffffu, c.x), c.y = __reduce_add_sync(0xffffffffu, c.y), c.z = __reduce_add_sync(0xffffffffu, c.z);
        if constexpr (WARPS != 1) {
            parity ^= 1;                    // (counts of the step before may still be read)
            if (lane == 0) s_count[parity][warp] = make_int4(c.x, c.y, c.z, 0);
            if constexpr (WARPS) asm volatile("bar.sync 1, %0;" ::"n"(WARPS * 32) : "memory");
            else __syncthreads();
            const int4 part = lane < warps ? s_count[parity][lane] : make_int4(0, 0, 0, 0);
            c.x = __reduce_add_sync(0xffffffffu, part.x), c.y = __reduce_add_sync(0xffffffffu, part.y), c.z = __reduce_add_sync(0xffffffffu, part.z);
        }
        return c;
    };
    *key = 0u, *equal = m, *exactly = false;
    for (int bit = 30; bit >= 0 && !*exactly; bit -= 2) {
        const unsigned t1 = *key | 1u << bit, t2 = *key | 2u << bit, t3 = *key | 3u << bit;
        const int3 c = reach(t1, t2, t3);
        *key = c.z >= m ? t3 : c.y >= m ? t2 : c.x >= m ? t1 : *key;
        *exactly = c.z == m || c.y == m || c.x == m;
    }
    if (!*exactly && *key != 0xffffffffu) *equal = m - reach(*key + 1u, 0xffffffffu, 0xffffffffu).x;
}

// One CTA per stream: the blocks' sums as ordered whole numbers in shared memory beside the row of the table; the m-th largest by
// find_bound; then one pass in order.  The weights are read once, all loads of a row of up to 32 K tokens in flight together; the
// rest is a chain of steps.  Up to 512 keys are one warp's, up to 2048 four warps', which meet at a barrier of their own: sixteen
// times 32768 tokens 8.0 us (one warp with 1024 keys 11.5, two with 512 each 8.5, eight with 128 each 8.2; a barrier of the CTA for
// every bit 13.8), one of 4100 tokens 4.7.
template <int BT>
__global__ void __launch_bounds__(1024) kv_evict_kernel(const EvictArgs a)
{
    extern __shared__ unsigned s_dyn[];     // keys [table_width], then the row of the table [table_width]
    __shared__ int s_warps[kMostEvictWarps], s_found[3];
    __shared__ int4 s_count[2][kMostEvictWarps];
    const spqt_kv_cache& c = a.c;
    const int stream = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x;
    constexpr int bt = BT, shift = BT == 16 ? 4 : BT == 32 ? 5 : BT == 64 ? 6 : 7;
    const int width = c.table_width;
    unsigned* const s_key = s_dyn;
    int* const s_row = reinterpret_cast<int*>(s_dyn + width);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int held = (int)ld_global_u32(c.length + stream);
    const int32_t* const row = c.table + (size_t)stream * width;
    int32_t* const row_out = (a.table_out ? a.table_out : c.table) + (size_t)stream * width;
    int32_t* const length_out = (a.length_out ? a.length_out : c.length) + stream;
    for (int i = tid; i < width; i += threads) s_row[i] = row[i];
    const int n = length_or_none(held, c, a.status);
    const int closed = n >> shift;
    __syncthreads();                        // (also: every thread has the length)
    if (closed <= a.keep) {
        if (row_out != row)
            for (int i = tid; i < width; i += threads) row_out[i] = s_row[i];
        if (tid == 0) *length_out = held;
        return;
    }
    // sums: bt / 4 lanes a block, four weights a lane, in fp64 (the order of the sum is then of no consequence to the rounded one
    // but in one case of 2^29).  A lane has N blocks, so that the lanes of a block can share the additions.
    constexpr int kLanes = BT / 4, kAtOnce = 32 / kLanes, N = kLanes < 8 ? kLanes : 8;
    const int sub = lane / kLanes, l = lane % kLanes, turn = (threads >> 5) * kAtOnce;
    for (int j0 = warp * kAtOnce; j0 < closed; j0 += turn * N) {       // (short rows: a block or few for every warp)
        float4 w[N];
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int j = j0 + u * turn + sub;
            const unsigned id = j < closed ? (unsigned)s_row[j] : 0xffffffffu;
            w[u] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (id < (unsigned)c.blocks) w[u] = *reinterpret_cast<const float4*>(c.weight + ((size_t)id << shift) + 4 * l);
        }
        double v[N];
#pragma unroll
        for (int u = 0; u < N; ++u) {
            v[u] = 0.0;
            if (j0 + u * turn < closed) v[u] = ((double)w[u].x + w[u].y) + ((double)w[u].z + w[u].w);
        }
        int u = 0;
        const double sum = sums_over<N, kLanes>(v, lane, 1, &u);
        const int j = j0 + u * turn + sub;
        if (j < closed && l < N) {           // (lanes beyond have the same sums again)
            const bool known = (unsigned)s_row[j] < (unsigned)c.blocks;
            s_key[j] = known ? ordered((float)sum) : 0u;               // (what no block stands behind leaves first)
            if (!known) refuse(a.status);
        }
    }
    __syncthreads();
    // the m-th largest key among the blocks that are not protected
    const int lo = a.first, hi = closed - a.recent, m = a.keep - a.first - a.recent;
    unsigned key = 0u;                      // its bits so far
    int equal = m;                          // of the keys equal to it only the first so many stay
    bool exactly = false;                   // m keys reach it, so that all that do stay
    if (m > 0) {
        const int count = hi - lo;
        if (count <= 32 * kOwnKeys) {
            if (warp == 0) find_bound<kOwnKeys, 1>(s_key + lo, count, m, s_count, &key, &equal, &exactly);
        } else if (count <= 32 * kOwnKeys * kBoundWarps) {
            if (warp < kBoundWarps) find_bound<kOwnKeys, kBoundWarps>(s_key + lo, count, m, s_count, &key, &equal, &exactly);
        } else {
            find_bound<0, 0>(s_key + lo, count, m, s_count, &key, &equal, &exactly);
        }
        if (tid == 0) s_found[0] = (int)key, s_found[1] = equal, s_found[2] = exactly;
        __syncthreads();
        key = (unsigned)s_found[0], equal = s_found[1], exactly = s_found[2] != 0;
    }
    // in order: blocks that stay to the front, the open one, those that leave, the rest where it was
    const int some = n & (bt - 1) ? 1 : 0;
    int stay = 0, leave = a.keep + some;    // places
    for (int j0 = 0; j0 < closed; j0 += threads) {
        const int j = j0 + tid;
        const bool in = j >= lo && j < hi;
        const unsigned k = in ? s_key[j] : 0u;
        int all;
        bool keeps = j < closed && (!in || (m > 0 && k >= key));
        if (!exactly) {
            const bool same = in && m > 0 && k == key;
            const int rank = count_before(same, s_warps, &all);
            keeps = keeps && !(same && rank >= equal);
            equal -= all;
        }
        const int place = count_before(keeps, s_warps, &all);
        if (j < closed) row_out[keeps ? stay + place : leave + tid - place] = s_row[j];
        stay += all;
        leave += min(threads, closed - j0) - all;
    }
    if (some && tid == 0) row_out[a.keep] = s_row[closed];
    if (row_out != row)
        for (int i = closed + some + tid; i < width; i += threads) row_out[i] = s_row[i];
    if (tid == 0) *length_out = a.keep * bt + (n & (bt - 1));
}

}  // namespace spqt

// Calls `f` with the cache's format and row size as constants.
#define SPQT_KV_DISPATCH(c, f)                                                            \
    ((c).format == SPQT_KV_INT8 ? ((c).head_dim == 64    ? f(SPQT_KV_INT8, 64)            \
                                   : (c).head_dim == 96  ? f(SPQT_KV_INT8, 96)            \
                                   : (c).head_dim == 128 ? f(SPQT_KV_INT8, 128)           \
                                                         : f(SPQT_KV_INT8, 256))          \
                                : ((c).head_dim == 64    ? f(SPQT_KV_E4M3, 64)            \
                                   : (c).head_dim == 96  ? f(SPQT_KV_E4M3, 96)            \
                                   : (c).head_dim == 128 ? f(SPQT_KV_E4M3, 128)           \
                                                         : f(SPQT_KV_E4M3, 256)))

extern "C" {

spqt_status spqt_kv_append(const spqt_kv_cache* cache, const void* k, const void* v, int tokens, long long batch_stride, long long token_stride,
                           const int32_t* counts, int32_t* length_out, void* workspace, size_t workspace_bytes, void* stream)
{
    using namespace spqt;
    spqt_status st = check_cache(cache);
    if (st != SPQT_OK) return st;
    if (!k || !v || tokens < 1 || batch_stride < 0 || token_stride < 0) return SPQT_ERR_INVALID_ARG;
    if (!aligned(k, 16) || !aligned(v, 16) || batch_stride % 8 || token_stride % 8 || !aligned(counts, 4) || !aligned(length_out, 4)) return SPQT_ERR_ALIGNMENT;
    if (tokens > (1 << 28)) return SPQT_ERR_UNSUPPORTED;
    st = check_kv_workspace(workspace, workspace_bytes, kKvScratch + kv_lengths_bytes(*cache));
    if (st != SPQT_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    AppendArgs a = {*cache, static_cast<const __half*>(k), static_cast<const __half*>(v), tokens, batch_stride, token_stride, counts,
                    length_out ? length_out : cache->length, static_cast<int*>(status_word(workspace))};
    // Lengths are written in place at once where one CTA per stream reads them (a single token); else by way of the workspace.
    const bool indirect = a.length_out == cache->length && tokens > 1;
    if (indirect) a.length_out = reinterpret_cast<int32_t*>(static_cast<unsigned char*>(workspace) + kKvScratch);
#define SPQT_F(F, D) launch_append<F, D>(a, s)
    cudaError_t err = SPQT_KV_DISPATCH(*cache, SPQT_F);
#undef SPQT_F
    if (err == cudaSuccess && indirect) {
        const int n = cache->batch * cache->kv_heads;
        err = launch_overlapping(kv_lengths_kernel, dim3((n + 255) / 256), 256, 0, s, a.length_out, cache->length, n);
    }
    return launched(err);
}

spqt_status spqt_kv_read(const spqt_kv_cache* cache, const int32_t* length, void* k, void* v, int tokens, long long batch_stride, long long token_stride,
                         long long head_stride, void* workspace, size_t workspace_bytes, void* stream)
{
    using namespace spqt;
    spqt_status st = check_cache(cache);
    if (st != SPQT_OK) return st;
    if (!k || !v || tokens < 1 || batch_stride < 0 || token_stride < 0 || head_stride < 0) return SPQT_ERR_INVALID_ARG;
    if (!aligned(k, 16) || !aligned(v, 16) || batch_stride % 8 || token_stride % 8 || head_stride % 8 || !aligned(length, 4)) return SPQT_ERR_ALIGNMENT;
    st = check_kv_workspace(workspace, workspace_bytes, kKvHeader);
    if (st != SPQT_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int most = cache->table_width * cache->block_tokens;
    if (tokens > most) tokens = most;
    RowStride strides[] = {{batch_stride, cache->batch}, {token_stride, tokens}, {head_stride, cache->kv_heads}};
    const long long apart = (static_cast<const char*>(k) - static_cast<const char*>(v)) / 2;
    if (!rows_apart(cache->head_dim, strides) || (apart < cache->head_dim && -apart < cache->head_dim)) return SPQT_ERR_INVALID_ARG;
    const ReadArgs a = {*cache, length ? length : cache->length, static_cast<__half*>(k), static_cast<__half*>(v), tokens, batch_stride, token_stride,
                        head_stride, static_cast<int*>(status_word(workspace))};
    // (warps: at most 2^17 pieces of a row of the table times 2^14 streams)
    const long long warps = (long long)((tokens + kReadTokens - 1) / kReadTokens) * cache->kv_heads;
    const dim3 grid((unsigned)((warps + kReadWarps - 1) / kReadWarps), (unsigned)cache->batch);
#define SPQT_F(F, D) launch_overlapping(kv_read_kernel<F, D>, grid, kReadWarps * 32, 0, s, a)
    const cudaError_t err = SPQT_KV_DISPATCH(*cache, SPQT_F);
#undef SPQT_F
    return launched(err);
}

spqt_status spqt_kv_evict(const spqt_kv_cache* cache, int keep, int first, int recent, int32_t* table_out, int32_t* length_out, void* workspace,
                          size_t workspace_bytes, void* stream)
{
    using namespace spqt;
    spqt_status st = check_cache(cache);
    if (st != SPQT_OK) return st;
    if (!cache->weight || keep < 0 || first < 0 || recent < 0 || (long long)first + recent > keep) return SPQT_ERR_INVALID_ARG;
    if (!aligned(table_out, 4) || !aligned(length_out, 4)) return SPQT_ERR_ALIGNMENT;
    st = check_kv_workspace(workspace, workspace_bytes, kKvHeader);
    if (st != SPQT_OK) return st;
    const size_t smem = (size_t)cache->table_width * 8;
    static thread_local int allowed_dev = -1;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return launched(cudaErrorInvalidDevice);
    if (smem > 40 * 1024 && allowed_dev != dev) {   // (48 KB with the kernel's own need no leave)
        for (auto kernel : {kv_evict_kernel<16>, kv_evict_kernel<32>, kv_evict_kernel<64>, kv_evict_kernel<128>}) {
            const cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxTableWidth * 8);
            if (err != cudaSuccess) return launched(err);
        }
        allowed_dev = dev;
    }
    const EvictArgs a = {*cache, keep, first, recent, table_out, length_out, static_cast<int*>(status_word(workspace))};
    // a thread per block of a row, and some more for the loads of short ones
    const int threads = cache->table_width <= 128 ? 128 : cache->table_width <= 512 ? 512 : 1024;
    const auto kernel = cache->block_tokens == 16 ? kv_evict_kernel<16> : cache->block_tokens == 32 ? kv_evict_kernel<32> : cache->block_tokens == 64 ? kv_evict_kernel<64> : kv_evict_kernel<128>;
    return launched(launch_overlapping(kernel, dim3(cache->batch * cache->kv_heads), threads, smem, static_cast<cudaStream_t>(stream), a));
}

spqt_status spqt_kv_status(const void* workspace, int* status_host, void* stream)
{
    if (!workspace || !status_host) return SPQT_ERR_INVALID_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const void* const word = static_cast<const unsigned char*>(workspace) + spqt::kStatusOffset;
    if (cudaMemcpyAsync(status_host, word, sizeof(int), cudaMemcpyDeviceToHost, s) != cudaSuccess || cudaStreamSynchronize(s) != cudaSuccess)
        return spqt::launched(cudaErrorUnknown);
    return *status_host == 0 ? SPQT_OK : SPQT_ERR_INVALID_ARG;
}

}  // extern "C"
