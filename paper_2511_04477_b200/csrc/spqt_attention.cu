// Attention of a step's queries over the 8-bit cache.
//
// out = sum_t p_t v_t with p = softmax_t(scale * <q, k_t>), k and v = code * scale of their block.  What bounds it is the codes,
// 2 * head_dim bytes a token, read once: the query heads of a kv head and the queries of a step are rows of one product.
//
// The product runs transposed on mma.sync.m16n8k16: A is the codes, 16 tokens (or 16 dimensions of v) an instruction, B the
// queries (or the probabilities), eight rows; with few rows the tensor cores are there for their operand format, and the other
// orientation would fill its 16 rows with nothing.  An 8-bit code becomes an exact fp16 value in registers (a byte permutation and a
// subtraction, or one conversion from e4m3), and with four to sixteen rows that is most of a tile's instructions (of 780 with four
// rows 32 are products), tensor pipe 17 % at most.  tcgen05 would not change that: its A may come from tensor memory, which takes
// the widened values from registers, 16 bits each, on top.  Scales stay outside of the product: a block's k scale multiplies its scores,
// its v scale the probabilities.
//
// Probabilities are needed in fp16: p = 2^(s + e - M + 10), s the score in powers of two, 2^e the power of two in the v scale, M the
// largest s + e when it was last looked at, which is when one exceeds it by 4: lanes need not ask one another for the largest of a
// tile.  p then lies in 0 .. 2^14, and what 16 bits cannot hold of it (2^-11) enters as a second fp16 value: with up to four rows in
// the columns that they leave free, else in a second instruction.  Without it the result is 1.4 times as far from the exact one,
// as far as its own rounding to fp16 takes it.  Sums are fp32 and know nothing of v's scales.
//
// Work: the tiles (32 tokens) of all segments (a stream, or sixteen of its rows where it has more) are laid end to end, each
// segment with some room in front for what it costs beside its tiles, and cut into equal parts, one per CTA; the warps of a CTA take
// its tiles in turn, each with a ring of tiles on their way (cp.async, so that a block number is all that is needed ahead).  A segment
// that lies within one CTA is finished there; of the others the CTA that comes last adds the parts, in the order of the CTAs.  Where
// weights are accumulated, a second kernel turns the scores that the first one left into probabilities.  Few segments of caches that
// hold little go the other way (cluster_of): a cluster of CTAs each, whose sums meet through its shared memory, weights included.
#include <cuda_fp8.h>

#include "spqt_common.cuh"
#include "spqt_gemv_device.cuh"
#include "spqt_mma.cuh"
#include "spqt_kv.cuh"

namespace spqt {

constexpr int kTile = 32;               // tokens of a tile of codes; half as many of the block that is not full
// Tiles that a segment costs beside its own.  With 0 / 6 / 12 / 20: 160 streams of up to 2047 tokens 34.6 / 26.5 / 24.8 / 23.0 us, 4001
// tokens of eight streams 18.5 / 11.5 / 11.5 / 11.4, ten streams of five queries in two row groups 39.8 / 38.3 / 36.8 / 39.6.
constexpr int kRoom = 16;
constexpr int kMaxAttnCtas = 160;       // parts at most
constexpr int kMostCluster = 16, kPortableCluster = 8;   // CTAs of a cluster at most; of one that every device has
constexpr int kLengthCache = 1024;      // streams whose lengths a CTA keeps in shared memory
constexpr float kUp = 10.0f;            // p of the largest score is 2^kUp, when M is set
constexpr float kSlack = 4.0f;          // and 2^(kUp + kSlack) before M is set anew

struct AttnArgs {
    spqt_kv_cache c;
    const __half* q;
    long long q_batch, q_token;
    __half* out;
    long long out_batch, out_token;
    int group, queries, rows;           // rows = group * queries of a stream, row i * group + g
    int row_groups;                     // of ROWS rows
    int shift;                          // log2 of the tokens of a block
    int accumulate;
    int most_tiles;                     // that a segment may have
    int cluster;                        // CTAs of a cluster, where a cluster takes each segment
    unsigned cluster_inv;               // 2^32 / cluster rounded up (cluster 1: 0)
    float scale_log2;
    int* status;
    int* begin;                         // workspace: the place of every segment's first tile, behind them the sum of tiles and rooms
    int* arrived;                       // parts that are there, of every segment; zero between calls
    float2* ml;                         // parts: (M, l) of every row
    float* o;                           // parts: sums of every row, not divided yet
    float2* lse;                        // segments: M - kUp and 1 / l of every row
    int4* tiles;                        // places: what tile it is, see TileNote
    float* scores;                      // places: [kTile][ROWS], in powers of two
};

template <int D, int ROWS>
struct AttnShape {
    static constexpr int kWarps = D == 256 ? 4 : 8;
    static constexpr int kTileBytes = 2 * kTile * D;
    static constexpr int kStages = D == 64 ? 4 : D == 96 ? 3 : D == 128 ? 2 : ROWS == 16 ? 2 : 3;
    static constexpr int kCols = ROWS == 16 ? 2 : 1;             // sets of eight columns
    static constexpr int kStride = D + 4;                        // of a row of sums in shared memory: 8 bytes a lane without conflicts
    static constexpr int kRing = kWarps * kStages * kTileBytes, kDynamic = kRing + kMaxAttnCtas * ROWS * 8;
    static constexpr int kStatic = kLengthCache * 4 + kWarps * kStages * 16 + (kWarps + 2) * ROWS * 8 + kWarps / 2 * ROWS * kStride * 4 + 512;
    static_assert(kStatic <= 48 * 1024 && kDynamic + kStatic + 1024 <= 227 * 1024, "shared memory of a CTA");
};

// Tokens of a stream's full blocks, and its tiles: those by 32 tokens, then the open block's by 16.
__device__ __forceinline__ int full_tokens(int n, int shift) { return n >> shift << shift; }
__device__ __forceinline__ int code_tiles(int n, int shift) { return (full_tokens(n, shift) + kTile - 1) / kTile; }
__device__ __forceinline__ int tiles_of(int n, int shift) { return code_tiles(n, shift) + (n - full_tokens(n, shift) + 15) / 16; }

__device__ __forceinline__ int places_of(int tiles) { return tiles == 0 ? 0 : kRoom + tiles; }

// CTAs that work: one for each segment (`busy` have tiles) where these are so short that to add parts would take longer than to
// have all the tiles (eight streams of 512 tokens 7.5 us with one, 8.1 with two; of 768 9.0 and 8.2), else not more than leave a tile for every warp.  A CTA's places
// begin at total * i / ctas.  (In fp64: the products are exact, and a quotient that is no whole number is 1/ctas or more from one.)
constexpr int kWhole = 20;
__device__ __forceinline__ int working_ctas(int total, int busy, int warps, int most)
{
    return min(max(total <= (kRoom + kWhole) * busy ? busy : (total + warps - 1) / warps, 1), most);
}
__device__ __forceinline__ int begin_of(int cta, int total, int ctas) { return (int)((double)total * cta / ctas); }
__device__ __forceinline__ int owner_of(int place, int total, int ctas) { return (int)(((double)(place + 1LL) * ctas - 1.0) / total); }

// What the second kernel has to know of a tile: its segment (-1: a place without a tile), the blocks of its halves, their rows and tokens.
__device__ __forceinline__ int4 tile_note(int seg, int id0, int id1, int row0, int row1, int count0, int count1)
{
    return make_int4(seg, id0, id1, row0 | row1 << 8 | count0 << 16 | count1 << 24);
}

__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Four codes of a register as fp16: bytes (0, 1) and (2, 3), or (0, 2) and (1, 3).
template <int FMT, bool SPREAD>
__device__ __forceinline__ void widen(unsigned w, unsigned& x, unsigned& y)
{
    if (FMT == SPQT_KV_INT8) {
        const unsigned u = w ^ 0x80808080u;              // code + 128 under the exponent of 1024: 1152 + code
        const __half2 bias = __half2half2(__ushort_as_half(0x6480));
        unsigned a = __byte_perm(u, 0x64646464u, SPREAD ? 0x4240 : 0x4140), b = __byte_perm(u, 0x64646464u, SPREAD ? 0x4341 : 0x4342);
        const __half2 ha = __hsub2(*reinterpret_cast<__half2*>(&a), bias), hb = __hsub2(*reinterpret_cast<__half2*>(&b), bias);
        x = *reinterpret_cast<const unsigned*>(&ha);
        y = *reinterpret_cast<const unsigned*>(&hb);
    } else {
        const unsigned u = SPREAD ? __byte_perm(w, 0u, 0x3120) : w;
        asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\tcvt.rn.f16x2.e4m3x2 %1, hi;\n\t}" : "=r"(x), "=r"(y) : "r"(u));
    }
}

__device__ __forceinline__ void ldsm_x4(unsigned addr, unsigned* r)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ unsigned transposed(unsigned v)
{
    unsigned r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ unsigned halves(float a, float b)
{
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const unsigned*>(&h);
}
// 16 bytes, or zeros where `bytes` is 0
__device__ __forceinline__ void cp_async_16_of(unsigned dst, const void* src, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_scale(unsigned dst, const void* src)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}

// Where a 16-byte piece of a row of N lies in a tile: as in memory, so that the pieces of neighbouring lanes of a copy lie within the
// same 128 bytes (a copy whose lanes write 32 places takes 32 turns: the whole call 100 instead of 56 us with 131072 tokens), but
// exchanged among them by the row, so that the same piece of eight rows, which ldmatrix reads at once, lies in eight places.
template <int N>
__device__ __forceinline__ unsigned place_of(int row, int piece)
{
    const int turn = N % 8 == 0 ? row & 7 : N % 4 == 0 ? row >> 1 & 3 : row >> 2 & 1;
    if (N % 8 == 0) return (unsigned)(row * N * 16 + (((piece & 7) ^ turn) + (piece & ~7)) * 16);
    return (unsigned)((row * N + piece) ^ turn) * 16;
}

// 8 bytes and 16 of the shared memory of another CTA of the cluster
__device__ __forceinline__ float2 ld_cluster_f32x2(unsigned addr)
{
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float4 ld_cluster_f32x4(unsigned addr)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ unsigned cluster_rank()
{
    unsigned r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_arrive_release() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }

// MOST > 0: a segment for each cluster of up to MOST CTAs instead of parts of all of them; the CTAs' sums meet through shared memory, and
// the weights are added here as well.  No CTA leaves early: the others may read its shared memory.
template <int FMT, int D, int ROWS, int MOST>
__global__ void __launch_bounds__(AttnShape<D, ROWS>::kWarps * 32, 1) kv_attention_kernel(const AttnArgs a, int streams)
{
    using S = AttnShape<D, ROWS>;
    constexpr bool CLUSTER = MOST > 0;
    constexpr int NW = S::kWarps, STAGES = S::kStages, NC = S::kCols, CH = D / 16;
    extern __shared__ __align__(128) unsigned char s_ring[];                 // [NW][STAGES][kTileBytes], then s_part
    __shared__ int s_len[kLengthCache];
    __shared__ int s_scan[NW], s_busy[NW], s_start[2];
    __shared__ __align__(16) float s_scale[NW][STAGES][4];                   // k scale of the halves, v scale of the halves
    __shared__ float2 s_ml[NW][ROWS], s_cta[ROWS], s_lse[ROWS];
    __shared__ __align__(16) float s_o[NW / 2][ROWS][S::kStride];
    float2(*const s_part)[ROWS] = reinterpret_cast<float2(*)[ROWS]>(s_ring + NW * STAGES * S::kTileBytes);   // (M, l) of the parts of a segment
    const spqt_kv_cache& c = a.c;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, cc = lane & 3;
    const int shift = a.shift;
    const unsigned ring = smem_u32(s_ring) + warp * STAGES * S::kTileBytes;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    // ---- which tiles are this CTA's
    const int cta = blockIdx.x, segments = streams * a.row_groups;
    int t0, t1, seg0, begin0, n0, tiles0, total = 0, ctas = 0;
    auto length_of = [&](int st) { return st < kLengthCache ? s_len[st] : length_or_none((int)ld_global_u32(c.length + st), c, a.status); };
    if constexpr (CLUSTER) {
        const int rank = (int)cluster_rank();
        asm("mov.u32 %0, %%clusterid.x;" : "=r"(seg0));
        n0 = length_or_none((int)ld_global_u32(c.length + seg0 / a.row_groups), c, a.status);
        tiles0 = tiles_of(n0, shift);
        begin0 = 0;
        t0 = (int)__umulhi((unsigned)(tiles0 * rank), a.cluster_inv);       // tiles0 * rank / cluster (2^15 at most, so exact)
        t1 = (int)__umulhi((unsigned)(tiles0 * (rank + 1)), a.cluster_inv);
        if (a.cluster == 1) t1 = tiles0;
    } else {
    const int per = (streams + NW * 32 - 1) / (NW * 32);
    int mine = 0, busy = 0;
    for (int i = 0; i < per; ++i) {
        const int st = tid * per + i;
        if (st < streams) {
            const int n = length_or_none((int)ld_global_u32(c.length + st), c, a.status);
            if (st < kLengthCache) s_len[st] = n;
            mine += places_of(tiles_of(n, shift)) * a.row_groups;
            busy += n > 0;
        }
    }
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
    }
    busy = __reduce_add_sync(0xffffffffu, busy);
    if (lane == 31) s_scan[warp] = incl, s_busy[warp] = busy;
    __syncthreads();
    int base = incl - mine;
    busy = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        base += w < warp ? s_scan[w] : 0;
        total += s_scan[w];
        busy += s_busy[w];
    }
    ctas = working_ctas(total, busy * a.row_groups, NW, gridDim.x);
    if (a.accumulate && cta == 0) {           // for the second kernel
        if (tid == 0) a.begin[streams * a.row_groups] = total;
        for (int st = tid * per, at = base; st < min(streams, (tid + 1) * per); ++st) {
            const int k = places_of(tiles_of(length_of(st), shift));
            for (int r = 0; r < a.row_groups; ++r, at += k) a.begin[st * a.row_groups + r] = at + kRoom;
        }
    }
    for (int st = cta; st < streams; st += gridDim.x) {   // queries that see nothing
        if (length_of(st) != 0) continue;
        const int b = st / c.kv_heads, h = st % c.kv_heads;
        for (int i = tid; i < a.rows * (D / 8); i += NW * 32) {
            const int r = i / (D / 8), qi = r / a.group;
            __half* const to = a.out + (long long)b * a.out_batch + (long long)qi * a.out_token + ((long long)h * a.group + (r - qi * a.group)) * D + i % (D / 8) * 8;
            *reinterpret_cast<uint4*>(to) = make_uint4(0u, 0u, 0u, 0u);
        }
    }
    if (total == 0 || cta >= ctas) return;
    t0 = begin_of(cta, total, ctas), t1 = begin_of(cta + 1, total, ctas);
    if (t0 >= base && t0 < base + mine) {
        // (bounded here and below, should lengths change while the kernel runs)
        int st = tid * per, at = base;
        for (; st + 1 < streams; ++st) {
            const int k = places_of(tiles_of(length_of(st), shift)) * a.row_groups;
            if (t0 < at + k) break;
            at += k;
        }
        s_start[0] = st;
        s_start[1] = at;
    }
    __syncthreads();
    const int stream0 = s_start[0];
    n0 = length_of(stream0), tiles0 = tiles_of(n0, shift);
    if (tiles0 == 0) return;
    const int rg0 = min((t0 - s_start[1]) / places_of(tiles0), a.row_groups - 1);
    seg0 = stream0 * a.row_groups + rg0, begin0 = s_start[1] + rg0 * places_of(tiles0) + kRoom;
    }
    // (of a cluster: places of its own for the scores)
    float* const scores = a.scores + (CLUSTER ? (size_t)seg0 * a.most_tiles * (kTile * ROWS) : 0);

    // ---- the tiles ahead: a walk over this warp's tiles that knows the segment of each; first the block numbers, one tile later
    // the copies.  (Of a segment's tiles in the part the first is the first warp's.)
    constexpr int kNoTile = 0x7fffffff;
    int w_seg = seg0, w_begin = begin0, w_n = n0, w_end = begin0 + tiles0, w_tile = max(t0, begin0) + warp;
    auto seek = [&]() {                       // the next segment with a tile for this warp, where this one has no more
        while (w_tile >= min(w_end, t1)) {
            if (CLUSTER || w_end >= t1) {
                w_tile = kNoTile;
                return;
            }
            if (++w_seg >= segments) {
                w_tile = kNoTile;
                return;
            }
            w_n = length_of(w_seg / a.row_groups);
            const int k = tiles_of(w_n, shift);
            if (k == 0) continue;
            w_begin = w_end + kRoom;
            w_end = w_begin + k;
            if (w_begin >= t1) {
                w_tile = kNoTile;
                return;
            }
            w_tile = w_begin + warp;
        }
    };
    seek();
    // the tile whose block numbers are on their way (lane u: half u)
    int p_tile = w_tile, p_seg = 0, p_local = 0, p_n = 0, p_id = 0;
    auto look_up = [&]() {
        p_tile = w_tile;
        if (w_tile != kNoTile) {
            p_seg = w_seg;
            p_local = w_tile - w_begin;
            p_n = w_n;
            const int full = full_tokens(w_n, shift), tail = p_local - (full + kTile - 1) / kTile;
            const int token = tail < 0 ? p_local * kTile + (lane & 1) * 16 : full + tail * 16;
            p_id = token < (tail < 0 ? full : !CLUSTER && a.accumulate ? w_n : 0) ? (int)ld_global_u32(c.table + (size_t)(w_seg / a.row_groups) * c.table_width + (token >> shift)) : 0;
            w_tile += NW;
            if (w_tile >= w_end) seek();
            else if (w_tile >= t1) w_tile = kNoTile;
        }
    };
    // A lane's pieces of a half tile of codes; those of eight rows and more apart lie as far apart.
    constexpr int kDistinct = CH == 4 ? 1 : CH == 8 ? 2 : CH == 16 ? 4 : D / 32;
    unsigned place[kDistinct];
#pragma unroll
    for (int i = 0; i < kDistinct; ++i) place[i] = place_of<CH>((i * 32 + lane) / CH, (i * 32 + lane) % CH);
    auto copy = [&](int stage) {
        if (p_tile == kNoTile) return;
        const unsigned dst = ring + stage * S::kTileBytes;
        const int full = full_tokens(p_n, shift), tail = p_local - (full + kTile - 1) / kTile;
        const bool known = (unsigned)p_id < (unsigned)c.blocks;
        if (!known) refuse(a.status);
        if (!CLUSTER && a.accumulate) {
            const int id1 = __shfl_sync(0xffffffffu, p_id, 1), mask = (1 << shift) - 1, there = tail < 0 ? full : p_n;
            const int token = tail < 0 ? p_local * kTile : full + tail * 16;
            if (lane == 0)
                a.tiles[p_tile] = tile_note(p_seg, p_id, id1, token & mask, (token + 16) & mask, known ? min(16, there - token) : 0,
                                            tail < 0 && (unsigned)id1 < (unsigned)c.blocks ? max(0, min(16, there - token - 16)) : 0);
        }
        if (tail < 0) {
            const int id = known ? p_id : 0;
            if (lane < 4) {
                // (lanes 0 and 1: k of the halves, 2 and 3: v of the halves; lane & 1 is the half whose number the lane holds)
                const unsigned at = smem_u32(&s_scale[warp][stage][0]) + lane * 4;
                if (known) cp_async_scale(at, (lane < 2 ? c.k_scale : c.v_scale) + id);
                else sts_u32(at, 0x7fffffffu);
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int token = p_local * kTile + u * 16;
                const int bytes = u == 0 || token < full ? 16 : 0;
                const size_t from = (((size_t)(unsigned)__shfl_sync(0xffffffffu, id, u) << shift) + (token & ((1 << shift) - 1))) * D + lane * 16;
                const unsigned char* const k = static_cast<const unsigned char*>(c.k_codes) + from;
                const unsigned char* const v = static_cast<const unsigned char*>(c.v_codes) + from;
#pragma unroll
                for (int i = 0; i < D / 32; ++i) {
                    const unsigned to = dst + place[i % kDistinct] + (unsigned)(i / kDistinct * kDistinct * 512 + u * 16 * D);
                    cp_async_16_of(to, k + i * 512, bytes);
                    cp_async_16_of(to + kTile * D, v + i * 512, bytes);
                }
            }
        } else {
            const int r0 = tail * 16;
            const size_t from = (((size_t)(p_seg / a.row_groups) << shift) + r0) * D;
            const __half* const k = static_cast<const __half*>(c.k_tail) + from + lane * 8;
            const __half* const v = static_cast<const __half*>(c.v_tail) + from + lane * 8;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                const int p = i * 32 + lane, r = p / (D / 8), ch = p % (D / 8);
                const unsigned to = dst + place_of<2 * CH>(r, ch);
                const int bytes = full + r0 + r < p_n ? 16 : 0;
                cp_async_16_of(to, k + i * 256, bytes);
                cp_async_16_of(to + kTile * D, v + i * 256, bytes);
            }
        }
    };
    look_up();
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) {
        copy(i);
        cp_async_commit();
        look_up();
    }

    // ---- segment after segment
    int stage = 0, seg = seg0, begin = begin0, n = n0;
    unsigned qf[NC][CH][2];
    // Queries: column g of set s is row row0 + 8s + g of its stream (with four rows twice the same four); a lane's dimensions of a
    // chunk of 16 are 4cc .. 4cc + 3, as its bytes of the codes are.
    auto load_queries = [&]() {
        const int stream = seg / a.row_groups, row0 = seg % a.row_groups * ROWS, b = stream / c.kv_heads, h = stream % c.kv_heads;
#pragma unroll
        for (int s = 0; s < NC; ++s) {
            const int r = row0 + s * 8 + (ROWS == 4 ? g & 3 : g), i = r / a.group;
            const __half* const q = a.q + (long long)b * a.q_batch + (long long)i * a.q_token + ((long long)h * a.group + (r - i * a.group)) * D + 4 * cc;
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                uint2 v = make_uint2(0u, 0u);
                if (r < a.rows) v = *reinterpret_cast<const uint2*>(q + j * 16);
                qf[s][j][0] = v.x;
                qf[s][j][1] = v.y;
            }
        }
    };
    load_queries();
    for (bool once = true; CLUSTER ? once : begin < t1; once = false) {
        const int tiles = tiles_of(n, shift), end = begin + tiles;
        const int stream = seg / a.row_groups, row0 = seg % a.row_groups * ROWS;
        const int b = stream / c.kv_heads, h = stream % c.kv_heads;
        if (!CLUSTER && a.accumulate && begin >= t0 && tid < kRoom) a.tiles[begin - kRoom + tid] = tile_note(-1, 0, 0, 0, 0, 0, 0);
        int lim[NC][2];                       // tokens that the rows of this lane's columns see
#pragma unroll
        for (int s = 0; s < NC; ++s)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int rc = row0 + s * 8 + (ROWS == 4 ? (2 * cc + e) & 3 : 2 * cc + e);
                lim[s][e] = rc < a.rows ? n - a.queries + 1 + rc / a.group : n;
            }
        const int full = full_tokens(n, shift), nt = (full + kTile - 1) / kTile;
        const int clean = max(0, min(full, n - a.queries + 1)) / kTile;   // tiles of whose tokens all are there and all rows see all
        float o[CH][NC][4];
        float M[NC][2], less[NC][2], l[NC][2];   // less: M - kUp, finite
#pragma unroll
        for (int s = 0; s < NC; ++s) {
            M[s][0] = M[s][1] = -INFINITY;
            less[s][0] = less[s][1] = 0.0f;
            l[s][0] = l[s][1] = 0.0f;
#pragma unroll
            for (int d = 0; d < CH; ++d) o[d][s][0] = o[d][s][1] = o[d][s][2] = o[d][s][3] = 0.0f;
        }
        const int stop = min(end, t1);
        for (int tile = max(t0, begin) + warp; tile < stop; tile += NW) {
            cp_async_wait<STAGES - 2>();
            __syncwarp();
            {
                const int ahead = stage == 0 ? STAGES - 1 : stage - 1;
                copy(ahead);
                cp_async_commit();
                look_up();
            }
            const unsigned at = ring + stage * S::kTileBytes;
            const int local = tile - begin;
            const bool codes = local < nt;
            const int token0 = codes ? local * kTile : full + (local - nt) * 16;
            float x[NC][2][4];                // scores: half u, (token g, column 2cc), (g, 2cc+1), (g+8, 2cc), (g+8, 2cc+1)
            float ks[2] = {1.0f, 1.0f}, vs[2] = {1.0f, 1.0f};
#pragma unroll
            for (int s = 0; s < NC; ++s)
#pragma unroll
                for (int u = 0; u < 2; ++u) x[s][u][0] = x[s][u][1] = x[s][u][2] = x[s][u][3] = 0.0f;
            if (codes) {
                const float4 sc = *reinterpret_cast<const float4*>(&s_scale[warp][stage][0]);
                ks[0] = sc.x, vs[0] = sc.z;
                if (token0 + 16 < full) ks[1] = sc.y, vs[1] = sc.w;
#pragma unroll
                for (int j = 0; j < CH; ++j) {
                    unsigned r[4], f[4][2];
                    ldsm_x4(at + place_of<CH>(lane, j), r);
#pragma unroll
                    for (int m = 0; m < 4; ++m) widen<FMT, false>(r[m], f[m][0], f[m][1]);
#pragma unroll
                    for (int s = 0; s < NC; ++s) {
                        mma_16816(x[s][0], f[0][0], f[1][0], f[0][1], f[1][1], qf[s][j][0], qf[s][j][1]);
                        mma_16816(x[s][1], f[2][0], f[3][0], f[2][1], f[3][1], qf[s][j][0], qf[s][j][1]);
                    }
                }
            } else {
#pragma unroll
                for (int j = 0; j < CH; ++j) {
                    const int ch = 2 * j + (cc >> 1);
                    const uint2 r0 = lds_v2(at + place_of<2 * CH>(g, ch) + (cc & 1) * 8);
                    const uint2 r1 = lds_v2(at + place_of<2 * CH>(g + 8, ch) + (cc & 1) * 8);
#pragma unroll
                    for (int s = 0; s < NC; ++s) mma_16816(x[s][0], r0.x, r1.x, r0.y, r1.y, qf[s][j][0], qf[s][j][1]);
                }
            }
            // scores in powers of two, with the v scale as 2^ve * vf (one that is zero, below the normal numbers or not finite: ve = 0)
            float ve[2], vf[2], down[2];
            bool plain = true;
            if (a.accumulate) {
                float* const to = scores + (size_t)tile * (kTile * ROWS);
                if (ROWS >= 8 || cc < 2) {
#pragma unroll
                    for (int s = 0; s < NC; ++s)
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            const float f = ks[u] * a.scale_log2;
                            float v[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) v[e] = token0 + u * 16 + (e >> 1) * 8 + g < lim[s][e & 1] ? x[s][u][e] * f : -INFINITY;
                            *reinterpret_cast<float2*>(to + (u * 16 + g) * ROWS + s * 8 + 2 * cc) = make_float2(v[0], v[1]);
                            *reinterpret_cast<float2*>(to + (u * 16 + g + 8) * ROWS + s * 8 + 2 * cc) = make_float2(v[2], v[3]);
                        }
                }
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const unsigned bits = __float_as_uint(vs[u]), ex = bits >> 23 & 0xffu;
                const bool p = ex != 0u && ex != 0xffu;
                plain = plain && p;
                ve[u] = p ? (float)((int)ex - 127) : 0.0f;
                vf[u] = p ? __uint_as_float((bits & 0x807fffffu) | 0x3f800000u) : vs[u];
                down[u] = p ? __uint_as_float((254u - ex) << 23) : 1.0f;      // 2^-ve
                const float f = ks[u] * a.scale_log2;
#pragma unroll
                for (int s = 0; s < NC; ++s)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[s][u][e] = fmaf(x[s][u][e], f, ve[u]);
            }
            if (local >= clean) {
                // (a half tile behind the last full block counts for the next kind of tile)
                const int there = codes ? full : n;
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int token = token0 + u * 16 + (e >> 1) * 8 + g;
                        const bool in = token < there && (codes || u == 0);
#pragma unroll
                        for (int s = 0; s < NC; ++s)
                            if (!in || token >= lim[s][e & 1]) x[s][u][e] = -INFINITY;
                    }
            }
            unsigned ph[NC][2][2], pl[NC][2][2];
            float top[NC][2];
            bool above = false;
#pragma unroll
            for (int s = 0; s < NC; ++s)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    top[s][e] = fmaxf(fmaxf(x[s][0][e], x[s][0][e + 2]), fmaxf(x[s][1][e], x[s][1][e + 2]));
                    above = above || top[s][e] > M[s][e] + kSlack;
                }
            if (__any_sync(0xffffffffu, above)) {
                float alpha[NC][2];
#pragma unroll
                for (int s = 0; s < NC; ++s)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float m = top[s][e];
                        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
                        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
                        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
                        m = fmaxf(m, M[s][e]);
                        alpha[s][e] = m == M[s][e] ? 1.0f : exp2_fast(M[s][e] - m);
                        M[s][e] = m;
                        less[s][e] = m == -INFINITY ? 0.0f : m - kUp;
                        l[s][e] *= alpha[s][e];
                    }
#pragma unroll
                for (int d = 0; d < CH; ++d)
#pragma unroll
                    for (int s = 0; s < NC; ++s)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[d][s][e] *= alpha[s][e & 1];
            }
#pragma unroll
            for (int s = 0; s < NC; ++s)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    float w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float p = exp2_fast(x[s][u][e] - less[s][e & 1]);
                        l[s][e & 1] = fmaf(p, down[u], l[s][e & 1]);
                        w[e] = p * vf[u];
                    }
                    if (!plain) {             // (what is not seen is nothing, whatever its block's scale)
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[e] = x[s][u][e] == -INFINITY ? 0.0f : w[e];
                    }
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const unsigned hi = halves(w[2 * k], w[2 * k + 1]);
                        const float2 back = __half22float2(*reinterpret_cast<const __half2*>(&hi));
                        const unsigned lo = halves(w[2 * k] - back.x, w[2 * k + 1] - back.y);
                        if (ROWS == 4) {
                            ph[s][u][k] = transposed(cc < 2 ? hi : lo);
                        } else {
                            ph[s][u][k] = transposed(hi);
                            pl[s][u][k] = transposed(lo);
                        }
                    }
                }
            if (codes) {
#pragma unroll
                for (int d = 0; d < CH; ++d) {
                    unsigned r[4], f[4][2];
                    ldsm_x4_trans(at + kTile * D + place_of<CH>(lane, d), r);
#pragma unroll
                    for (int m = 0; m < 4; ++m) widen<FMT, true>(r[m], f[m][0], f[m][1]);
#pragma unroll
                    for (int s = 0; s < NC; ++s) {
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            mma_16816(o[d][s], f[2 * u][0], f[2 * u][1], f[2 * u + 1][0], f[2 * u + 1][1], ph[s][u][0], ph[s][u][1]);
                            if (ROWS > 4) mma_16816(o[d][s], f[2 * u][0], f[2 * u][1], f[2 * u + 1][0], f[2 * u + 1][1], pl[s][u][0], pl[s][u][1]);
                        }
                    }
                }
            } else {
#pragma unroll
                for (int d = 0; d < CH; ++d) {
                    const int ch = 2 * d + (g >> 2);
                    unsigned w[4];
                    bool odd = false;             // values that are not finite: out of the product, and to the rows that see them
                    auto word = [&](int token) { return lds_u32(at + kTile * D + place_of<2 * CH>(token, ch) + (g & 3) * 4); };
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        w[k] = word(2 * cc + (k & 1) + (k >> 1) * 8);
                        const bool o0 = (w[k] & 0x7c00u) == 0x7c00u, o1 = (w[k] & 0x7c000000u) == 0x7c000000u;
                        odd = odd || o0 || o1;
                        w[k] &= (o0 ? 0u : 0xffffu) | (o1 ? 0u : 0xffff0000u);
                    }
                    const unsigned a0 = __byte_perm(w[0], w[1], 0x5410), a1 = __byte_perm(w[0], w[1], 0x7632);
                    const unsigned a2 = __byte_perm(w[2], w[3], 0x5410), a3 = __byte_perm(w[2], w[3], 0x7632);
#pragma unroll
                    for (int s = 0; s < NC; ++s) {
                        mma_16816(o[d][s], a0, a1, a2, a3, ph[s][0][0], ph[s][0][1]);
                        if (ROWS > 4) mma_16816(o[d][s], a0, a1, a2, a3, pl[s][0][0], pl[s][0][1]);
                    }
                    if (__any_sync(0xffffffffu, odd)) {
#pragma unroll 1
                        for (int k = 0; k < 16 && token0 + k < n; ++k) {
                            const unsigned v = word(k);
                            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&v));
                            const bool o0 = (v & 0x7c00u) == 0x7c00u, o1 = (v & 0x7c000000u) == 0x7c000000u;
#pragma unroll
                            for (int s = 0; s < NC; ++s)
#pragma unroll
                                for (int e = 0; e < 2; ++e)
                                    if (token0 + k < lim[s][e]) {
                                        if (o0) o[d][s][e] += f.x;
                                        if (o1) o[d][s][e + 2] += f.y;
                                    }
                        }
                    }
                }
            }
            stage = stage + 1 == STAGES ? 0 : stage + 1;
        }

        // ---- the next segment, whose queries are on their way while this one is finished
        const int this_seg = seg, this_begin = begin;
        if constexpr (!CLUSTER) {
        begin = end;
        do {
            n = ++seg < segments && begin + kRoom < t1 ? length_of(seg / a.row_groups) : 1;
        } while (n == 0);
        begin = seg < segments ? begin + kRoom : t1;
        if (begin < t1) load_queries();
        }

        // ---- the warps' sums: to the CTA's largest M, then by way of shared memory, half the warps at a time
#pragma unroll
        for (int s = 0; s < NC; ++s)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                l[s][e] += __shfl_xor_sync(0xffffffffu, l[s][e], 4);
                l[s][e] += __shfl_xor_sync(0xffffffffu, l[s][e], 8);
                l[s][e] += __shfl_xor_sync(0xffffffffu, l[s][e], 16);
                const int r = s * 8 + 2 * cc + e;
                if (g == 0 && r < ROWS) s_ml[warp][r] = make_float2(M[s][e], l[s][e]);
            }
        if (ROWS == 4) {                      // the columns of what 16 bits did not hold
#pragma unroll
            for (int d = 0; d < CH; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[d][0][e] += __shfl_xor_sync(0xffffffffu, o[d][0][e], 2);
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < NC; ++s) {
            float f[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = s * 8 + 2 * cc + e;
                float m = -INFINITY;
#pragma unroll
                for (int w = 0; w < NW; ++w) m = fmaxf(m, s_ml[w][r % ROWS].x);
                f[e] = M[s][e] == m ? 1.0f : exp2_fast(M[s][e] - m);
            }
#pragma unroll
            for (int d = 0; d < CH; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[d][s][e] *= f[e & 1];
        }
        const bool writes = ROWS >= 8 || cc < 2;
        auto put = [&](float(*to)[S::kStride], bool add) {
            if (!writes) return;
#pragma unroll
            for (int s = 0; s < NC; ++s)
#pragma unroll
                for (int d = 0; d < CH; ++d)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float2* const p = reinterpret_cast<float2*>(&to[s * 8 + 2 * cc + e][d * 16 + 2 * g]);
                        float2 v = make_float2(o[d][s][e], o[d][s][e + 2]);
                        if (add) {
                            const float2 w = *p;
                            v.x += w.x;
                            v.y += w.y;
                        }
                        *p = v;
                    }
        };
        if (warp >= NW / 2) put(s_o[warp - NW / 2], false);
        __syncthreads();
        if (warp < NW / 2) put(s_o[warp], true);
        __syncthreads();
        const bool whole = !CLUSTER && this_begin >= t0 && end <= t1;
        const size_t part = (size_t)cta + this_seg;
        auto answer = [&](int r, int d, float m, float sum, const float4& v) {   // four dimensions of a row
            const int rr = row0 + r, qi = rr / a.group;
            const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;           // (a row that sees nothing: zeros)
            __half* const to = a.out + (long long)b * a.out_batch + (long long)qi * a.out_token + ((long long)h * a.group + (rr - qi * a.group)) * D + d;
            *reinterpret_cast<uint2*>(to) = make_uint2(halves(v.x * inv, v.y * inv), halves(v.z * inv, v.w * inv));
            if (!CLUSTER && a.accumulate && d == 0) a.lse[(size_t)this_seg * ROWS + r] = make_float2(m == -INFINITY ? 0.0f : m - kUp, inv);
        };
        for (int i = tid; i < ROWS * (D / 4); i += NW * 32) {
            const int r = i / (D / 4), d = i % (D / 4) * 4;
            if (row0 + r >= a.rows) continue;
            float m = -INFINITY, sum = 0.0f;
#pragma unroll
            for (int w = 0; w < NW; ++w) m = fmaxf(m, s_ml[w][r].x);
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float2 v = s_ml[w][r];
                sum += v.x == m ? v.y : v.y * exp2_fast(v.x - m);
            }
            float4 v = *reinterpret_cast<const float4*>(&s_o[0][r][d]);
#pragma unroll
            for (int w = 1; w < NW / 2; ++w) {
                const float4 k = *reinterpret_cast<const float4*>(&s_o[w][r][d]);
                v.x += k.x, v.y += k.y, v.z += k.z, v.w += k.w;
            }
            if constexpr (CLUSTER) {          // (each of these values has been read by this thread alone)
                *reinterpret_cast<float4*>(&s_o[0][r][d]) = v;
                if (d == 0) s_cta[r] = make_float2(m, sum);
            } else if (whole) {
                answer(r, d, m, sum, v);
            } else {
                *reinterpret_cast<float4*>(a.o + (part * ROWS + r) * D + d) = v;
                if (d == 0) a.ml[part * ROWS + r] = make_float2(m, sum);
            }
        }
        if constexpr (CLUSTER) {
            // ---- the CTAs' sums: each CTA finishes its share of the rows' dimensions
            cluster_arrive_release();
            cluster_wait();
            constexpr int kItems = ROWS * (D / 4);
            const int rank = (int)cluster_rank(), share = (int)__umulhi((unsigned)(kItems + a.cluster - 1), a.cluster_inv) + (a.cluster == 1 ? kItems : 0);
            // the CTAs' (M, l) of a row, their largest M and the sum.  (Places behind the last CTA read its values again, which count as
            // none: a branch for each of them takes 1.1 us.)
            auto joined = [&](int r, float2* x, float* most) {
                float m = -INFINITY, sum = 0.0f;
#pragma unroll
                for (int k = 0; k < MOST; ++k) {
                    x[k] = ld_cluster_f32x2(cluster_map(smem_u32(&s_cta[r]), min(k, a.cluster - 1)));
                    if (k >= a.cluster) x[k] = make_float2(-INFINITY, 0.0f);
                }
#pragma unroll
                for (int k = 0; k < MOST; ++k) m = fmaxf(m, x[k].x);
#pragma unroll
                for (int k = 0; k < MOST; ++k) sum += x[k].x == m ? x[k].y : x[k].y * exp2_fast(x[k].x - m);
                *most = m;
                return sum;
            };
            float2 x[MOST > 0 ? MOST : 1];
            float m;
            for (int i = rank * share + tid; i < min(kItems, (rank + 1) * share); i += NW * 32) {
                const int r = i / (D / 4), d = i % (D / 4) * 4;
                float4 y[MOST > 0 ? MOST : 1], v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int k = 0; k < MOST; ++k) y[k] = ld_cluster_f32x4(cluster_map(smem_u32(&s_o[0][r][d]), min(k, a.cluster - 1)));
                const float sum = joined(r, x, &m);
#pragma unroll
                for (int k = 0; k < MOST; ++k) {
                    const float f = x[k].x == m ? 1.0f : exp2_fast(x[k].x - m);
                    const bool in = k < a.cluster;
                    v.x = fmaf(in ? y[k].x : 0.0f, f, v.x), v.y = fmaf(in ? y[k].y : 0.0f, f, v.y);
                    v.z = fmaf(in ? y[k].z : 0.0f, f, v.z), v.w = fmaf(in ? y[k].w : 0.0f, f, v.w);
                }
                if (row0 + r < a.rows) answer(r, d, m, sum, v);
            }
            const int r = tid - (NW * 32 - ROWS);             // (threads that have no share where there are any)
            if (a.accumulate && r >= 0) {
                const float sum = joined(r, x, &m);
                s_lse[r] = make_float2(m == -INFINITY ? 0.0f : m - kUp, sum == 0.0f ? 0.0f : 1.0f / sum);
            }
            __syncthreads();
            cluster_arrive_release();
            if (a.accumulate) {
                // ---- weights of this warp's tiles, a lane per token; two tiles at a time
                const int32_t* const row = c.table + (size_t)stream * c.table_width;
                for (int x0 = t0 + warp; x0 < t1; x0 += 2 * NW) {
                    unsigned block[2];
                    int token[2];
                    bool there[2];
                    float sum[2], old[2];
                    float4 e[2][ROWS / 4];
                    float* to[2];
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int local = x0 + u * NW;
                        const bool codes = local < nt;
                        token[u] = (codes ? local * kTile : full + (local - nt) * 16) + lane;
                        there[u] = local < t1 && token[u] < (codes ? full : n) && (codes || lane < 16);
                        block[u] = there[u] ? (unsigned)row[token[u] >> shift] : 0u;
                        const float4* const from = reinterpret_cast<const float4*>(scores + ((size_t)local * kTile + lane) * ROWS);
#pragma unroll
                        for (int q = 0; q < ROWS / 4; ++q)
                            if (there[u] && 4 * q < a.rows) e[u][q] = from[q];
                    }
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        if (there[u] && block[u] >= (unsigned)c.blocks) {
                            refuse(a.status);
                            there[u] = false;
                        }
                        to[u] = c.weight + ((size_t)block[u] << shift) + (token[u] & ((1 << shift) - 1));
                        old[u] = there[u] ? *to[u] : 0.0f;
                    }
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        sum[u] = 0.0f;
                        if (!there[u]) continue;
#pragma unroll
                        for (int q = 0; q < ROWS / 4; ++q) {
                            if (4 * q >= a.rows) continue;
                            const float v[4] = {e[u][q].x, e[u][q].y, e[u][q].z, e[u][q].w};
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                if (4 * q + k < a.rows) sum[u] = fmaf(exp2_fast(v[k] - s_lse[4 * q + k].x), s_lse[4 * q + k].y, sum[u]);
                        }
                        *to[u] = old[u] + sum[u];
                    }
                }
            }
            cluster_wait();                   // (nobody reads this CTA's shared memory any more)
        } else {
        __syncthreads();
        if (!whole) {
            // ---- a segment that several CTAs share: the last of them adds the parts
            const int c0 = owner_of(this_begin, total, ctas), c1 = owner_of(end - 1, total, ctas);
            if (tid == 0) {
                // (the parts, which the barrier has brought behind this thread, before the count; the count before the others' parts)
                int before;
                asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(before) : "l"(a.arrived + this_seg) : "memory");
                s_start[0] = before == c1 - c0;
            }
            __syncthreads();
            if (s_start[0]) {
                if (tid == 0) a.arrived[this_seg] = 0;
                // a thread has four dimensions of a row, of every kSplit-th part; the first kAhead are on their way beside the parts' (M, l)
                constexpr int kItems = ROWS * (D / 4), kSplit = NW * 32 / kItems < 1 ? 1 : NW * 32 / kItems, kAhead = 6;
                for (int i = tid; i < (c1 - c0 + 1) * ROWS; i += NW * 32)
                    s_part[i / ROWS][i % ROWS] = __ldcg(a.ml + ((size_t)c0 + i / ROWS + this_seg) * ROWS + i % ROWS);
                auto sums_of = [&](int i, int k) {   // of part k
                    return __ldcg(reinterpret_cast<const float4*>(a.o + (((size_t)k + this_seg) * ROWS + i % kItems / (D / 4)) * D + i % (D / 4) * 4));
                };
                float4 ahead[kAhead];
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    const int at = c0 + tid / kItems + k * kSplit;
                    ahead[k] = tid < kItems * kSplit && at <= c1 ? sums_of(tid, at) : make_float4(0.f, 0.f, 0.f, 0.f);
                }
                __syncthreads();
                for (int i = tid; i < kItems * kSplit; i += NW * 32) {
                    const int r = i % kItems / (D / 4), d = i % (D / 4) * 4, first = c0 + i / kItems;
                    if (row0 + r < a.rows) {
                        float m = -INFINITY, sum = 0.0f;
                        for (int k = 0; k <= c1 - c0; ++k) m = fmaxf(m, s_part[k][r].x);
                        for (int k = 0; k <= c1 - c0; ++k) {
                            const float2 x = s_part[k][r];
                            sum += x.x == m ? x.y : x.y * exp2_fast(x.x - m);
                        }
                        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
                        auto add = [&](int k, const float4& y) {
                            const float x = s_part[k - c0][r].x, f = x == m ? 1.0f : exp2_fast(x - m);
                            v.x = fmaf(y.x, f, v.x), v.y = fmaf(y.y, f, v.y), v.z = fmaf(y.z, f, v.z), v.w = fmaf(y.w, f, v.w);
                        };
                        int k = first;
                        if (i == tid) {
#pragma unroll
                            for (int u = 0; u < kAhead; ++u)
                                if (first + u * kSplit <= c1) add(first + u * kSplit, ahead[u]);
                            k += kAhead * kSplit;
                        }
#pragma unroll 1
                        for (; ROWS <= 8 && k + 7 * kSplit <= c1; k += 8 * kSplit) {   // (sixteen rows have no registers left)
                            float4 y[8];
#pragma unroll
                            for (int u = 0; u < 8; ++u) y[u] = sums_of(i, k + u * kSplit);
#pragma unroll
                            for (int u = 0; u < 8; ++u) add(k + u * kSplit, y[u]);
                        }
#pragma unroll 4
                        for (; k <= c1; k += kSplit) add(k, sums_of(i, k));
                        if (kSplit == 1) {
                            answer(r, d, m, sum, v);
                        } else {
                            *reinterpret_cast<float4*>(&s_o[i / kItems][r][d]) = v;
                            if (d == 0 && i < kItems) s_ml[0][r] = make_float2(m, sum);
                        }
                    }
                }
                if (kSplit > 1) {
                    __syncthreads();
                    for (int i = tid; i < kItems; i += NW * 32) {
                        const int r = i / (D / 4), d = i % (D / 4) * 4;
                        if (row0 + r < a.rows) {
                            float4 v = *reinterpret_cast<const float4*>(&s_o[0][r][d]);
#pragma unroll
                            for (int k = 1; k < kSplit; ++k) {
                                const float4 y = *reinterpret_cast<const float4*>(&s_o[k][r][d]);
                                v.x += y.x, v.y += y.y, v.z += y.z, v.w += y.w;
                            }
                            answer(r, d, s_ml[0][r].x, s_ml[0][r].y, v);
                        }
                    }
                }
                __syncthreads();
            }
        }
        }
    }
    cp_async_wait<0>();
}

// ---------------------------------------------------------------- weights

constexpr int kNoteWarps = 8;

// The probabilities that a tile's tokens have received, a lane per token and a warp for a few places at a time: their notes, then
// scores, sums and weights are on their way together.
template <int ROWS>
__global__ void __launch_bounds__(kNoteWarps * 32, ROWS == 16 ? 2 : 4) kv_weights_kernel(const AttnArgs a, int segments)
{
    // places at a time, four rows each.  (Eight sequences of 8192 tokens, eight rows: two at a time on four CTAs an SM 43.4 us with the
    // attention, four on two 44.6; four rows 41.5 and 42.3; sixteen rows spill with four CTAs, 38.5 against 35.2)
    constexpr int N = 2, Q = ROWS / 4;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, shift = a.shift;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int total = (int)ld_global_u32(a.begin + segments);
    for (int x0 = (blockIdx.x * kNoteWarps + warp) * N; x0 < total; x0 += gridDim.x * kNoteWarps * N) {
        int seg[N];
        float* to[N];
        float sum[N], old[N];
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int4 t = x0 + u < total ? a.tiles[x0 + u] : make_int4(-1, 0, 0, 0);
            const int half = lane >> 4, row = t.w >> (8 * half) & 0xff, count = t.w >> (16 + 8 * half) & 0xff;
            // (a stream's first row group stands for all)
            seg[u] = t.x >= 0 && t.x % a.row_groups == 0 && (lane & 15) < count ? t.x : -1;
            to[u] = a.c.weight + ((size_t)(unsigned)(half ? t.z : t.y) << shift) + row + (lane & 15);
            sum[u] = 0.0f;
        }
#pragma unroll
        for (int u = 0; u < N; ++u) old[u] = seg[u] >= 0 ? *to[u] : 0.0f;
        for (int rg = 0; rg < a.row_groups; ++rg) {
            const int rows = min(ROWS, a.rows - rg * ROWS);
            float4 s[N][Q];
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const int sg = max(seg[u], 0), x = rg == 0 ? x0 + u : x0 + u - a.begin[sg] + a.begin[sg + rg];
                const float4* const from = reinterpret_cast<const float4*>(a.scores + ((size_t)(seg[u] < 0 ? 0 : x) * kTile + lane) * ROWS);
#pragma unroll
                for (int q = 0; q < Q; ++q)
                    if (seg[u] >= 0 && 4 * q < rows) s[u][q] = from[q];
            }
            // (the sums of a segment's rows: those of the place before them in most cases)
            float4 l[2 * Q];
            auto load_sums = [&](int sg) {
                const float4* const lse = reinterpret_cast<const float4*>(a.lse + (size_t)(sg + rg) * ROWS);
#pragma unroll
                for (int q = 0; q < 2 * Q; ++q) l[q] = lse[q];
            };
            int have = max(seg[N - 1], 0);
            load_sums(have);
#pragma unroll
            for (int u = 0; u < N; ++u) {
                if (seg[u] < 0) continue;
                if (seg[u] != have) load_sums(have = seg[u]);
#pragma unroll
                for (int q = 0; q < Q; ++q) {
                    if (4 * q >= rows) continue;
                    const float4 e = s[u][q], l0 = l[2 * q], l1 = l[2 * q + 1];
                    sum[u] = fmaf(exp2_fast(e.x - l0.x), l0.y, sum[u]);
                    if (4 * q + 1 < rows) sum[u] = fmaf(exp2_fast(e.y - l0.z), l0.w, sum[u]);
                    if (4 * q + 2 < rows) sum[u] = fmaf(exp2_fast(e.z - l1.x), l1.y, sum[u]);
                    if (4 * q + 3 < rows) sum[u] = fmaf(exp2_fast(e.w - l1.z), l1.w, sum[u]);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < N; ++u)
            if (seg[u] >= 0) *to[u] = old[u] + sum[u];
    }
}

// ---------------------------------------------------------------- host

// Rows that go through the product together.  Few streams are cut into many parts, whose sums one CTA adds: sixteen rows of one
// stream of 65536 tokens by eight 20.0 us, by sixteen 45.1; of sixteen streams of 8192 19.3 and 19.8, of 32 31.1 and 26.5.
inline int rows_of(int rows, long long streams) { return rows <= 4 ? 4 : rows <= 8 || streams <= 16 ? 8 : 16; }

struct AttnWorkspace {
    size_t arrived, begin, ml, o, lse, tiles, scores, bytes;   // (what stays zero between calls at a place that depends on nothing)
};

constexpr int kMoreTiles = 8;           // tiles of 16 tokens of a block of 128, the largest
inline int most_tiles(const spqt_kv_cache& c) { return (c.table_width * c.block_tokens + kTile - 1) / kTile + kMoreTiles; }
static_assert((long long)kMaxStreams * (kMaxTableWidth * 128 / kTile + kMoreTiles + kRoom) <= 0x7fffffffLL, "a tile's number in 31 bits, whatever the cache");

// false where there are more segments than counts of parts
inline bool attention_workspace(const spqt_kv_cache& c, int group, int queries, AttnWorkspace* w)
{
    const long long streams = (long long)c.batch * c.kv_heads;
    const int rows = group * queries, R = rows_of(rows, streams), groups = (rows + R - 1) / R;
    const long long segments = streams * groups;
    if (segments > kMaxStreams) return false;
    const long long tiles = segments * (most_tiles(c) + kRoom);
    auto up = [](size_t v) { return (v + 255) / 256 * 256; };
    size_t at = kKvHeader;
    w->arrived = at, at += (size_t)kMaxStreams * 4;
    w->begin = at, at += up(((size_t)segments + 1) * 4);
    const size_t parts = (size_t)(kMaxAttnCtas + segments);
    w->ml = at, at += up(parts * R * 8);
    w->o = at, at += up(parts * R * c.head_dim * 4);
    w->lse = w->tiles = w->scores = at;
    if (c.weight) {
        at += up((size_t)segments * R * 8);
        w->tiles = at, at += up((size_t)tiles * 16);
        w->scores = at, at += up((size_t)tiles * kTile * R * 4);
    }
    w->bytes = at;
    return true;
}

// CTAs of the clusters that take a segment each, 0: the work is divided among all CTAs instead.  `most`: clusters of so many CTAs that
// fit (of 16: 7, 10: 11, 8: 15, 6: 22, 4: 33 on the GPU that the figures are of); the segments have to fit all.
//   A cluster has none of the fixed cost of the division, of parts by way of global memory and of a kernel for the weights, but fewer
// SMs.  Eight heads of 1 / 2 / 5 / 8 / 12 sequences of 1000 tokens by clusters 5.8 / 6.1 / 7.3 / 8.1 / 10.5 us, otherwise 8.6 / 8.9 / 10.5 /
// 13.1 / 15.5; eight sequences with weights 9.3 against 16.1; four sequences of 2000, twelve rows, 9.7 against 15.2; four heads of 16000
// 10.2 against 11.7.  Five tiles a warp at most: the lengths are on the device, so that what the table can hold stands for them, and
// where one stream alone has them all, the other SMs wait (12 us, when 9 would do).
//   Of the sizes that fit, the smallest that saves the warps a tile, but 8, or 4 for few tiles, where the warps share a scheduler less
// (two heads of 1000 tokens by 4 6.1 us, by 8 5.5; eight of 40 5.3 and 5.6).
inline int cluster_of(const AttnArgs& a, int warps, int segments, const int* most)
{
    if (a.accumulate && a.row_groups > 1) return 0;
    const int tiles = a.most_tiles - kMoreTiles;
    int cl = kMostCluster;
    while (cl > 0 && most[cl] < segments) --cl;
    if (cl == 0 || tiles > 5 * warps * cl) return 0;
    const int each = (tiles + warps * cl - 1) / (warps * cl), fewest = (tiles + warps * each - 1) / (warps * each), least = tiles > 2 * warps ? 8 : 4;
    return fewest > least ? fewest : cl < least ? cl : least;
}

template <int FMT, int D, int ROWS, int MOST>
cudaError_t launch_clusters(const AttnArgs& a, int segments, bool prepare, cudaLaunchConfig_t cfg, cudaLaunchAttribute* attr, int* most)
{
    const auto kernel = kv_attention_kernel<FMT, D, ROWS, MOST>;
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    if (prepare) {                          // most[cl]: clusters of so many CTAs that fit, for the sizes that are this kernel's
        cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)cfg.dynamicSmemBytes);
        if (err == cudaSuccess && MOST > kPortableCluster) err = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (err != cudaSuccess) return err;
        cfg.numAttrs = 1;
        for (int cl = MOST == 4 ? 1 : MOST / 2 + 1; cl <= MOST; ++cl) {
            attr[0].val.clusterDim.x = cl;
            cfg.gridDim = dim3((unsigned)cl);
            if (cudaOccupancyMaxActiveClusters(&most[cl], kernel, &cfg) != cudaSuccess) {
                (void)cudaGetLastError();
                most[cl] = 0;
            }
        }
        return cudaSuccess;
    }
    attr[0].val.clusterDim.x = a.cluster;
    cfg.gridDim = dim3((unsigned)(segments * a.cluster));
    cfg.numAttrs = g_no_pdl ? 1 : 2;
    const cudaError_t err = cudaLaunchKernelEx(&cfg, kernel, a, a.c.batch * a.c.kv_heads);
    if (err == cudaSuccess) count_launch();
    return err;
}

// *taken: whether the call went by clusters.
template <int FMT, int D, int ROWS>
cudaError_t try_clusters(AttnArgs a, int segments, cudaStream_t s, bool* taken)
{
    using S = AttnShape<D, ROWS>;
    static thread_local int prepared_dev = -1, most[kMostCluster + 1];
    int dev = 0;
    cudaError_t err = cudaGetDevice(&dev);
    if (err != cudaSuccess) return err;
    cudaLaunchAttribute attr[2];
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(S::kWarps * 32);
    cfg.dynamicSmemBytes = S::kRing;
    cfg.stream = s;
    constexpr bool kLarge = ROWS < 16;      // (sixteen rows are for more streams than there are clusters of more than 8)
    if (prepared_dev != dev) {
        err = launch_clusters<FMT, D, ROWS, 4>(a, segments, true, cfg, attr, most);
        if (err == cudaSuccess) err = launch_clusters<FMT, D, ROWS, 8>(a, segments, true, cfg, attr, most);
        if constexpr (kLarge)
            if (err == cudaSuccess) err = launch_clusters<FMT, D, ROWS, 16>(a, segments, true, cfg, attr, most);
        if (err != cudaSuccess) return err;
        prepared_dev = dev;
    }
    a.cluster = cluster_of(a, S::kWarps, segments, most);
    *taken = a.cluster > 0;
    if (!*taken) return cudaSuccess;
    a.cluster_inv = a.cluster == 1 ? 0u : (unsigned)(((1ULL << 32) + a.cluster - 1) / a.cluster);
    if constexpr (kLarge)
        if (a.cluster > 8) return launch_clusters<FMT, D, ROWS, 16>(a, segments, false, cfg, attr, most);
    return a.cluster > 4 ? launch_clusters<FMT, D, ROWS, 8>(a, segments, false, cfg, attr, most) : launch_clusters<FMT, D, ROWS, 4>(a, segments, false, cfg, attr, most);
}

template <int FMT, int D, int ROWS>
cudaError_t launch_attention(const AttnArgs& a, cudaStream_t s)
{
    using S = AttnShape<D, ROWS>;
    const int streams = a.c.batch * a.c.kv_heads, segments = streams * a.row_groups;
    bool taken = false;
    cudaError_t err = try_clusters<FMT, D, ROWS>(a, segments, s, &taken);
    if (err != cudaSuccess || taken) return err;
    static thread_local int allowed_dev = -1;
    int dev = 0;
    err = cudaGetDevice(&dev);
    if (err != cudaSuccess) return err;
    if (allowed_dev != dev) {
        err = cudaFuncSetAttribute(kv_attention_kernel<FMT, D, ROWS, 0>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kDynamic);
        if (err != cudaSuccess) return err;
        allowed_dev = dev;
    }
    const int sms = sm_count();
    if (sms <= 0) return cudaErrorInvalidDevice;
    const int parts = sms < kMaxAttnCtas ? sms : kMaxAttnCtas;
    err = launch_overlapping(kv_attention_kernel<FMT, D, ROWS, 0>, dim3(parts), S::kWarps * 32, S::kDynamic, s, a, streams);
    if (err != cudaSuccess) return err;
    return a.accumulate ? launch_overlapping(kv_weights_kernel<ROWS>, dim3(4 * sms), kNoteWarps * 32, 0, s, a, segments) : cudaSuccess;
}

template <int FMT, int D>
cudaError_t launch_rows(const AttnArgs& a, cudaStream_t s)
{
    const int r = rows_of(a.rows, (long long)a.c.batch * a.c.kv_heads);
    return r == 4 ? launch_attention<FMT, D, 4>(a, s) : r == 8 ? launch_attention<FMT, D, 8>(a, s) : launch_attention<FMT, D, 16>(a, s);
}

template <int FMT>
cudaError_t launch_dim(const AttnArgs& a, cudaStream_t s)
{
    switch (a.c.head_dim) {
        case 64: return launch_rows<FMT, 64>(a, s);
        case 96: return launch_rows<FMT, 96>(a, s);
        case 128: return launch_rows<FMT, 128>(a, s);
        default: return launch_rows<FMT, 256>(a, s);
    }
}

static spqt_status check_rows(const spqt_kv_cache* cache, int q_heads, int queries, AttnWorkspace* w)
{
    spqt_status st = check_cache(cache);
    if (st != SPQT_OK) return st;
    if (q_heads <= 0 || queries <= 0) return SPQT_ERR_INVALID_ARG;
    if (q_heads % cache->kv_heads || q_heads / cache->kv_heads > 64 || queries > 16) return SPQT_ERR_UNSUPPORTED;
    return attention_workspace(*cache, q_heads / cache->kv_heads, queries, w) ? SPQT_OK : SPQT_ERR_UNSUPPORTED;
}

}  // namespace spqt

extern "C" {

spqt_status spqt_kv_workspace(const spqt_kv_cache* cache, int q_heads, int queries, size_t* bytes)
{
    spqt::AttnWorkspace w;
    if (!bytes) return SPQT_ERR_INVALID_ARG;
    spqt_status st = spqt::check_rows(cache, q_heads, queries, &w);
    if (st != SPQT_OK) return st;
    // (fewer queries may take the rows in other groups)
    size_t most = w.bytes;
    for (int q = 1; q < queries; ++q) {
        st = spqt::check_rows(cache, q_heads, q, &w);
        if (st == SPQT_OK && w.bytes > most) most = w.bytes;
    }
    *bytes = most;
    return SPQT_OK;
}

spqt_status spqt_kv_attention(const spqt_kv_cache* cache, const void* q, long long q_batch_stride, long long q_token_stride, int q_heads, int queries,
                              float scale, int accumulate, void* out, long long out_batch_stride, long long out_token_stride, void* workspace,
                              size_t workspace_bytes, void* stream)
{
    using namespace spqt;
    AttnWorkspace w;
    spqt_status st = check_rows(cache, q_heads, queries, &w);
    if (st != SPQT_OK) return st;
    if (!q || !out || (accumulate && !cache->weight) || q_batch_stride < 0 || q_token_stride < 0 || out_batch_stride < 0 || out_token_stride < 0)
        return SPQT_ERR_INVALID_ARG;
    if (!aligned(q, 16) || !aligned(out, 16) || q_batch_stride % 8 || q_token_stride % 8 || out_batch_stride % 8 || out_token_stride % 8) return SPQT_ERR_ALIGNMENT;
    st = check_kv_workspace(workspace, workspace_bytes, accumulate ? w.bytes : w.lse);
    if (st != SPQT_OK) return st;
    RowStride strides[] = {{out_batch_stride, cache->batch}, {out_token_stride, queries}};
    if (!rows_apart((long long)q_heads * cache->head_dim, strides)) return SPQT_ERR_INVALID_ARG;
    unsigned char* const ws = static_cast<unsigned char*>(workspace);
    const int group = q_heads / cache->kv_heads, rows = group * queries, R = rows_of(rows, (long long)cache->batch * cache->kv_heads);
    const AttnArgs a = {*cache, static_cast<const __half*>(q), q_batch_stride, q_token_stride, static_cast<__half*>(out), out_batch_stride, out_token_stride,
                        group, queries, rows, (rows + R - 1) / R, 31 - __builtin_clz((unsigned)cache->block_tokens), accumulate ? 1 : 0, most_tiles(*cache), 0, 0u, scale * 1.4426950408889634f, static_cast<int*>(status_word(workspace)),
                        reinterpret_cast<int*>(ws + w.begin), reinterpret_cast<int*>(ws + w.arrived), reinterpret_cast<float2*>(ws + w.ml),
                        reinterpret_cast<float*>(ws + w.o), reinterpret_cast<float2*>(ws + w.lse), reinterpret_cast<int4*>(ws + w.tiles),
                        reinterpret_cast<float*>(ws + w.scores)};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return launched(cache->format == SPQT_KV_INT8 ? launch_dim<SPQT_KV_INT8>(a, s) : launch_dim<SPQT_KV_E4M3>(a, s));
}

}  // extern "C"
