// Attention of a chunk of new tokens over the mixed-format paged cache (mkv_chunk_attention).
//
// Row i of request b is its position p = seq_lens[b] - n_b + i (n_b new tokens, cached already).  For every query head
//   s_t = scale q . k_t for t <= p,   out = sum_t exp(s_t) v_t / sum_t exp(s_t),
// over the FP8 and Stale pages of the request's table row under one softmax (Section 3.3), each page read in its own
// format (Section 4.1).  Stale keys stay in the rotated domain: s_t = scale q' . c_t g_t with q' = d^-1/2 H (sigma . q).
//
// Mapping to the hardware
//   * The rows of a tile are (token, query head) pairs of one KV head, 128 per tensor-memory accumulator: a query group
//     shares every unpacked key and value.  A block takes two such row tiles at d = 128 and one at d = 256 (the output
//     accumulators, 256 columns, and two score buffers of 128 columns fill tensor memory) and walks tiles of 128 keys.
//     Where a unit fills one of two row tiles, the key tiles go by turns to both accumulators (8 requests of 5 rows over 16K
//     tokens, d = 128: 89 us with one, 77 by turns).
//   * Each key tile holds pages of one format (chunk_plan_kernel sorts a row's pages by format), so that the products
//     take one query: the rotated one for Stale tiles, then the plain one, written over it, for FP8 tiles.
//   * Pages are unpacked once per block to fp16 in shared memory, K-major with the 128-byte swizzle, by eight warps
//     (e4m3 -> fp16 is exact; Stale keys are level * g, values code * scale + zero, each rounded to fp16: 2^-12 of an
//     element on average, as the probabilities' rounding and far below the output's bf16.  The decode kernels, whose output is
//     fp32, keep such factors apart).  A lane of the packed fragment order holds scattered dims (keys) and tokens (values): the
//     order of the contraction is free, so query dims and key rows are permuted such that every lane's share is one 16-byte
//     store without bank conflicts.
//   * One warp issues the products S = Q K^T (both operands in shared memory) and O += P V (P in tensor memory, over
//     the scores it came from), the scores of the tile after next before the softmax of this one has finished.
//   * A softmax thread owns a row (its tensor-memory lane): no exchange between threads.  The reference of the
//     exponentials is raised only when 32 of them sum to more than 2^15, which keeps P within fp16 and rescaling of O rare;
//     it is set 7 below the maximum, so that probabilities down to 2^-31 of the largest are not flushed.
//   * (unit, key tiles) pairs are cut evenly over the SMs; a unit that several blocks share leaves fp32 partials
//     (m, l, O) in the workspace and chunk_merge_kernel joins them (Eq. softmax-merge), in the order of the blocks.
//
// What bounds it (B200; measured with the arenas in HBM, rates are of the visible pairs' 4 d flops): no unit of the SM, but the
// chains between the roles.
//   * Long chunks, d = 256 (2,048 rows of 24 heads over 57K tokens, format 2): 3.06 to 3.1 ms by the clock that the power cap leaves,
//     0.95 PFLOP/s, 57 % of what a large bf16 matrix product reaches here.  On a case of the same kind the tensor pipe is active in 50 % of
//     the cycles, the data path of shared memory in 53 % (ncu's figure, without the products' operand reads), issue slots in 50 %.  Keys and
//     values have one stage each: a product waits for two unpacking warps a scheduler, they for it.  Unpacking left out, it would be
//     2.3 ms; every row tile unpacks every key tile again (96 times a KV head here).
//   * d = 128 (1,000 rows of 32 heads over 16K tokens, twice): 0.75 ms, 0.73 PFLOP/s; tensor pipe 36 %, issue slots 47 %.  The softmax,
//     chains of two warps a scheduler beside two unpacking ones: a step of 32 columns costs some 240 cycles whatever it does (steps of 16:
//     0.98 ms; of 64: registers).  Spilled registers count: 104 for a softmax thread 0.85 ms, 112 0.74 (in one run).  Score buffers of 64
//     columns, four of them, hide the wait for the scores and lose more in steps (0.9 ms for 0.8); two threads to a row, the softmax fully
//     unrolled and unpacking split by keys and values were slower, too.
//   * Prompts (3 x 4,097 rows, d = 256): 0.74 ms, half of the rate: a unit's query, masks and epilogue cost as much as four to five key
//     tiles, of 17 on average (with six of them in the cut and one price for all tiles 6 % more, with two 27 %).
//   * A few rows per request: latency.  4 rows over 4,092 tokens: 30 us in three launches: plan 4, the scan's start (share, query, first
//     keys) 6, then the largest share's key tiles (four, by turns to two accumulators), partials and merge 7, the launches.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math_constants.h>
#include <mutex>

#include "mkv_internal.cuh"
#include "tensor_ptx.cuh"

namespace mkv {
namespace chunk {

constexpr int kMaxBlocks = 160;              // of the scan's grid: sizes the partials
constexpr int kKeys = 128;                   // keys of a tile: eight runs of 16 tokens
// The cut's prices: of a key tile, of one in a unit that fills one of two row tiles, and of a unit besides (query, epilogue).
// Measured: 3.0, 1.8 and 12 - 20 us at d = 128, 2.25 and 9.5 at d = 256.
constexpr int kTileCost = 5, kHalfTileCost = 3, kUnitCost = 24;
// Of a block: two key tiles, or three to four where a unit fills one of two row tiles; smaller shares cost more in partials than
// they save.  (Longer than any tile: every block of a unit then begins one.)
constexpr int kLeastShare = 2 * kTileCost;
constexpr float kShift = 7.f;                // see above: the reference lies so far below the maximum when it is set
constexpr float kMostSum = 32768.f;          // of the probabilities of a step, so of any of them: fp16 holds them
constexpr int kNoPos = 0x7fffffff;

template <int N>
struct Int { static constexpr int value = N; };

// What chunk_plan_kernel leaves of a request.  Runs are of 16 tokens.
struct Request {
    int n_new, row0, len;
    int n_stale, n_fp8;          // runs in the two lists
    int stale_end;               // runs of the row up to the last Stale page
    int exact;                   // every page of the row is in a list
    int pad;
    long long cost;              // of one KV head: its units'
};
struct Merge {
    int b, h, rt, last;          // unit, last block that has a part of it; b < 0: nothing to merge
    int first_slot, pad[3];
};

struct Params {
    const uint8_t *fp8, *tq3;
    int fp8_pages, tq3_pages, hkv, group, tiles;
    SigmaBits sigma;
    float sc2;                   // |scale| log2 e
    int negative;                // scale < 0: the queries change their sign
    float k_scale, v_scale;      // of FP8 pages
    int ke, ve;                  // exponents of the units 2^ke, 2^ve in which Stale keys and values are held as fp16
    const __nv_bfloat16* q;
    long long q_stride;          // elements from a token to the next
    int n_rows;
    const int32_t *starts, *bt, *lens;
    const uint8_t* tags;
    int B, max_pages;
    __nv_bfloat16* out;
    float* lse;
    Request* req;
    int2* list;                  // [B][max_pages] (logical page, id): Stale pages from the front, FP8 pages from the back
    float* part_o;               // [2 * blocks][rows][D]
    float2* part_ml;             // [2 * blocks][rows] (reference, sum)
    Merge* merge;
    uint32_t* status;
    unsigned long long wait_ns;
};

// mbarriers (index); phases are counted by the waiting side
enum {
    kKFull = 0, kKEmpty = 2, kVFull = 4, kVEmpty = 6,           // [stage]
    kSFull = 8, kPFull = 10,                                    // [score buffer]
    kPvDone = 12,                                               // [row tile]
    kQFull = 14, kFacRead = 15, kDrained = 16,
    kOutput = 17,                                               // [row tile] the last product of a segment
    kJoin = 19, kJoined = 23,                                   // [warp of a softmax group] rows handed over, and taken
    kBars = 27
};

// ---- the units --------------------------------------------------------------------------------------
struct Unit { int stale_tiles, fp8_tiles, n_fp8; };

// (of any length up to 2^31 - 1)
__device__ __forceinline__ int runs_of(int len) { return ((len - 1) >> 4) + 1; }

// key tiles of the rows [rt * ROWS, (rt + 1) * ROWS) of a request
template <int ROWS>
__device__ __forceinline__ Unit unit_of(const Request& r, int group, int rt)
{
    const int last = (min(r.n_new * group, (rt + 1) * ROWS) - 1) / group;
    const int p = r.len - r.n_new + last;                       // the last position that a row sees
    Unit u = {0, 0, 0};
    if (p < 0) return u;
    const int run = p >> 4, runs = runs_of(r.len);
    // FP8 runs behind the last row's position are left out where they are the row's last runs; elsewhere the masks do it
    u.n_fp8 = r.exact && r.stale_end <= run + 1 ? r.n_fp8 - (runs - 1 - run) : r.n_fp8;
    u.stale_tiles = (r.n_stale + 7) >> 3;
    u.fp8_tiles = (u.n_fp8 + 7) >> 3;
    return u;
}

template <int ROWS>
__device__ __forceinline__ int row_tiles_of(const Request& r, int group, int rt) { return min(ROWS / 128, (r.n_new * group - rt * ROWS + 127) / 128); }
template <int ROWS>
__device__ __forceinline__ int tile_cost(const Request& r, int group, int rt)
{
    return row_tiles_of<ROWS>(r, group, rt) * 128 == ROWS ? kTileCost : kHalfTileCost;
}
template <int ROWS>
__device__ __forceinline__ int unit_cost(const Request& r, int group, int rt)
{
    const Unit u = unit_of<ROWS>(r, group, rt);
    return kUnitCost + (u.stale_tiles + u.fp8_tiles) * tile_cost<ROWS>(r, group, rt);
}

struct Segment {
    Request r;
    Unit u;
    int b, h, rt, nt;            // nt: row tiles that hold rows
    int t0, t1;                  // key tiles of this block, Stale ones first
    int slot;                    // of the partial, or -1 where the block has the whole unit
    bool first_part;
    int last_block;
};

// A block's share [p0, p1) of the units laid end to end (shared memory), and where its first unit's request begins.
struct Share {
    long long p0, p1, per, request_start;
    int request;
};

// Walks the units that a block's share meets; every warp does so by itself, with its place and its present segment in shared
// memory (registers are what the roles are short of).
struct Walk {
    Segment s;
    long long at;
    int b, h, rt;

    // To the unit where the share begins (the whole warp, 32 units at a time).
    template <int ROWS>
    __device__ __forceinline__ void open(const Params& P, const Share* share, int lane)
    {
        const Request r = P.req[share->request];
        const long long skip = (share->p0 - share->request_start) / r.cost;      // KV heads before the first unit
        const int n_rt = (r.n_new * P.group + ROWS - 1) / ROWS;
        long long pos = share->request_start + skip * r.cost;
        int first = 0;
        for (; first < n_rt; first += 32) {
            const int c = first + lane < n_rt ? unit_cost<ROWS>(r, P.group, first + lane) : 0;
            long long sum = c;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long a = __shfl_up_sync(0xffffffffu, sum, o);
                if (lane >= o) sum += a;
            }
            const uint32_t m = __ballot_sync(0xffffffffu, pos + sum > share->p0);
            if (m) {
                const int src = __ffs(m) - 1;
                first += src;
                pos += __shfl_sync(0xffffffffu, sum - c, src);
                break;
            }
            pos += __shfl_sync(0xffffffffu, sum, 31);
        }
        if (lane == 0) {
            b = share->request;
            h = (int)skip;
            rt = first;
            at = pos;
        }
        __syncwarp();
    }
    template <int ROWS>
    __device__ __forceinline__ bool next(const Params& P, const Share* share)
    {
        const long long p0 = share->p0, p1 = share->p1;
        while (at < p1 && b < P.B) {
            s.r = P.req[b];
            const int n_rt = (s.r.n_new * P.group + ROWS - 1) / ROWS;
            if (n_rt == 0) {
                ++b;
                continue;
            }
            s.u = unit_of<ROWS>(s.r, P.group, rt);
            const int n = s.u.stale_tiles + s.u.fp8_tiles;
            const long long start = at, first = at + kUnitCost;
            s.b = b; s.h = h; s.rt = rt;
            s.nt = row_tiles_of<ROWS>(s.r, P.group, rt);
            const int price = tile_cost<ROWS>(s.r, P.group, rt), all = n * price;
            at = first + all;
            if (++rt == n_rt) {
                rt = 0;
                if (++h == P.hkv) {
                    h = 0;
                    ++b;
                }
            }
            // a tile is the block's in whose share it begins (a share is longer than any tile)
            s.t0 = ((int)min((long long)all, max(0ll, p0 - first)) + price - 1) / price;
            s.t1 = ((int)min((long long)all, max(0ll, p1 - first)) + price - 1) / price;
            if (s.t1 > s.t0 || (n == 0 && start >= p0)) {
                const bool whole = s.t0 == 0 && s.t1 == n;
                s.slot = whole ? -1 : 2 * (int)blockIdx.x + (start >= p0 ? 1 : 0);
                s.first_part = !whole && s.t0 == 0;
                s.last_block = n > 0 ? (int)((first + (n - 1) * price) / share->per) : (int)blockIdx.x;
                return true;
            }
        }
        return false;
    }
};

template <int D>
struct Geo {
    static constexpr int NT = D == 128 ? 2 : 1;                 // row tiles of a block
    static constexpr int ROWS = 128 * NT;
    static constexpr int COLS = 32;                             // score columns of a softmax step (registers)
    static constexpr int STAGES = D == 128 ? 2 : 1;             // key tiles, and value tiles, in shared memory
    static constexpr int Q_TILE = 128 * D * 2, K_TILE = kKeys * D * 2, V_TILE = K_TILE;
    static constexpr int SOFT_WARPS = 4 * NT, UNPACK_WARPS = 8;
    static constexpr int MMA_WARP = SOFT_WARPS + UNPACK_WARPS, THREADS = 32 * (MMA_WARP + 4);
    // registers: of the launch, and of the softmax, unpacking and product warps afterwards (the sums agree)
    static constexpr int REGS = D == 128 ? 96 : 128;
    static constexpr int SOFT_REGS = D == 128 ? 112 : 128, UNPACK_REGS = D == 128 ? 104 : 152, MMA_REGS = D == 128 ? 48 : 80;
    static_assert(SOFT_WARPS * SOFT_REGS + UNPACK_WARPS * UNPACK_REGS + 4 * MMA_REGS <= (MMA_WARP + 4) * REGS, "register split");
    static constexpr int OFF_Q = 0, OFF_K = OFF_Q + NT * Q_TILE, OFF_V = OFF_K + STAGES * K_TILE;
    static constexpr int OFF_FAC = OFF_V + STAGES * V_TILE;     // factor of every row's scores
    static constexpr int OFF_NAN = OFF_FAC + ROWS * 4;          // 64-bit word per channel, see note_nan
    static constexpr int OFF_PAIR = OFF_NAN + D * 8;            // 16 bytes a row: what the second of two softmax groups hands over
    static constexpr int OFF_BAR = OFF_PAIR + (NT == 2 ? 128 * 16 : 0);
    static constexpr int OFF_MISC = OFF_BAR + 256;
    static constexpr int OFF_WALK = OFF_MISC + 128;             // a Walk per warp
    static constexpr int SMEM = OFF_WALK + 32 * (int)sizeof(Walk) + 1024;           // the tiles start on a 1,024-byte boundary
    static_assert(SMEM <= 232448, "shared memory of a block");
};

// ---- plan -------------------------------------------------------------------------------------------
// One block per request: the row's pages by format, in order, and what the cut needs to know.  Bound by latency (a scan
// of the row's tags, 4,096 pages at a time).
constexpr int kPlanThreads = 256, kPlanPer = 16;

template <int ROWS>
__global__ void __launch_bounds__(kPlanThreads) chunk_plan_kernel(const Params P)
{
    __shared__ int warp_sum[2][kPlanThreads / 32];
    __shared__ int bad_s, stale_end_s, open_s;                  // open: the last page is an FP8 one
    __shared__ long long cost_s;
    pdl_begin();
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int T = P.tiles * kPage;
    if (tid == 0) { bad_s = 0; stale_end_s = 0; open_s = 0; cost_s = 0; }
    int len = P.lens[b];
    const int first = P.starts[b], last = P.starts[b + 1];
    uint32_t flags = 0;
    if ((long long)len > (long long)P.max_pages * T) { flags = kStBounds; len = P.max_pages * T; }
    if (len < 0) len = 0;
    int n_new = last - first;
    if (first < 0 || last > P.n_rows || n_new < 0) { flags = kStBounds; n_new = 0; }
    const int pages = n_new > 0 && len > 0 ? (len - 1) / T + 1 : 0;
    const int32_t* ids = P.bt + (size_t)b * P.max_pages;
    const uint8_t* tags = P.tags + (size_t)b * P.max_pages;
    int2* list = P.list + (size_t)b * P.max_pages;
    int n_stale = 0, n_fp8 = 0;                                 // pages listed so far
    __syncthreads();
    for (int base = 0; base < pages; base += kPlanThreads * kPlanPer) {
        const int p0 = base + tid * kPlanPer;
        int id[kPlanPer], tag_of[kPlanPer];
        uint32_t stale = 0, fp8 = 0;
#pragma unroll
        for (int i = 0; i < kPlanPer; ++i) {                    // (all at once: no load waits for another)
            const int p = min(p0 + i, pages - 1);
            tag_of[i] = tags[p];
            id[i] = ids[p];
        }
#pragma unroll
        for (int i = 0; i < kPlanPer; ++i) {
            const int p = p0 + i, tag = tag_of[i];
            if (p >= pages) continue;
            const bool is_stale = tag == MKV_TAG_STALE;
            const bool ok = is_stale ? id[i] >= 0 && id[i] < P.tq3_pages && (long long)(p + 1) * T <= len
                                     : tag <= MKV_TAG_ANCHOR && id[i] >= 0 && id[i] < P.fp8_pages;
            if (!ok) flags |= kStBounds;                        // never dereferenced
            else if (is_stale) stale |= 1u << i;
            else fp8 |= 1u << i;
        }
        const int c3 = __popc(stale), c8 = __popc(fp8);
        int s3 = c3, s8 = c8;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int a = __shfl_up_sync(0xffffffffu, s3, o), c = __shfl_up_sync(0xffffffffu, s8, o);
            if (lane >= o) { s3 += a; s8 += c; }
        }
        if (lane == 31) { warp_sum[0][warp] = s3; warp_sum[1][warp] = s8; }
        __syncthreads();
        int at3 = n_stale + s3 - c3, at8 = n_fp8 + s8 - c8;
#pragma unroll
        for (int w = 0; w < kPlanThreads / 32; ++w) {
            if (w < warp) { at3 += warp_sum[0][w]; at8 += warp_sum[1][w]; }
            n_stale += warp_sum[0][w];
            n_fp8 += warp_sum[1][w];
        }
#pragma unroll
        for (int i = 0; i < kPlanPer; ++i) {
            if (stale >> i & 1) list[at3++] = make_int2(p0 + i, id[i]);
            else if (fp8 >> i & 1) list[P.max_pages - 1 - at8++] = make_int2(p0 + i, id[i]);
        }
        if (pages - 1 - p0 >= 0 && pages - 1 - p0 < kPlanPer && (fp8 >> (pages - 1 - p0) & 1)) open_s = 1;
        if (stale) atomicMax(&stale_end_s, (p0 + 32 - __clz(stale)) * P.tiles);
        __syncthreads();
    }
    if (flags) {
        bad_s = 1;
        atomicOr(P.status, flags);
    }
    __syncthreads();
    Request r;
    r.n_new = n_new; r.row0 = first; r.len = len; r.pad = 0;
    r.n_stale = n_stale * P.tiles;
    r.n_fp8 = n_fp8 * P.tiles;
    // an open last page counts its filled runs (an open page is FP8, or it is in no list)
    r.exact = !bad_s;
    if (open_s)
        r.n_fp8 -= P.tiles - ((len - (pages - 1) * T + kPage - 1) / kPage);
    r.stale_end = stale_end_s;
    const int n_rt = (n_new * P.group + ROWS - 1) / ROWS;
    long long cost = 0;
    for (int rt = tid; rt < n_rt; rt += kPlanThreads) cost += unit_cost<ROWS>(r, P.group, rt);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) cost += __shfl_xor_sync(0xffffffffu, cost, o);
    if (lane == 0 && cost) atomicAdd(reinterpret_cast<unsigned long long*>(&cost_s), (unsigned long long)cost);
    __syncthreads();
    if (tid == 0) {
        r.cost = cost_s;
        P.req[b] = r;
    }
}

// ---- shared-memory operands and tensor-memory access ----------------------------------------------------
// K-major operand with the 128-byte swizzle: rows of 64 fp16, eight rows 1,024 bytes; the 16-byte chunk c of row r sits
// at chunk c ^ (r mod 8).  Successive 64-element atoms are a whole operand column apart.
__device__ __forceinline__ uint64_t operand_desc(uint32_t saddr)
{
    return (uint64_t)((saddr >> 4) & 0x3FFF) | ((uint64_t)1 << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) |
           ((uint64_t)2 << 61);
}
__device__ __forceinline__ uint32_t chunk_at(int row, int c) { return (uint32_t)(row * 128 + ((c ^ (row & 7)) << 4)); }
__host__ __device__ constexpr uint32_t idesc(int n) { return (1u << 4) | (uint32_t)(n >> 3) << 17 | (uint32_t)(128 >> 4) << 24; }   // f16 x f16 -> f32, M 128

__device__ __forceinline__ void sts128(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void sts64(uint32_t addr, uint32_t a, uint32_t b)
{
    asm volatile("st.shared.v2.u32 [%0], {%1,%2};" ::"r"(addr), "r"(a), "r"(b) : "memory");
}
__device__ __forceinline__ void sts32(uint32_t addr, uint32_t a) { asm volatile("st.shared.u32 [%0], %1;" ::"r"(addr), "r"(a) : "memory"); }

// Products are issued by a whole warp in step, one elected lane of it taking effect: descriptors and addresses then live in
// uniform registers.  (Issued from a lane's own branch every operand is moved there first, 190 cycles a product.)
__device__ __forceinline__ void issue_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t id, uint32_t accumulate)
{
    asm volatile("{\n .reg .pred p, e;\n elect.sync _|e, 0xffffffff;\n setp.ne.b32 p, %4, 0;\n"
                 " @e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d), "l"(a), "l"(b), "r"(id), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void issue_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t id, uint32_t accumulate)
{
    asm volatile("{\n .reg .pred p, e;\n elect.sync _|e, 0xffffffff;\n setp.ne.b32 p, %4, 0;\n"
                 " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
                 ::"r"(d), "r"(a), "l"(b), "r"(id), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void issue_commit(uint32_t bar)
{
    asm volatile("{\n .reg .pred e;\n elect.sync _|e, 0xffffffff;\n"
                 " @e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(bar) : "memory");
}
// a value that is the same in every lane, in a uniform register
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __reduce_max_sync(0xffffffffu, x); }
// 32 columns of the thread's tensor-memory lane
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float (&r)[32])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,"
                 "%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]),
                   "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]), "=f"(r[16]),
                   "=f"(r[17]), "=f"(r[18]), "=f"(r[19]), "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]), "=f"(r[24]),
                   "=f"(r[25]), "=f"(r[26]), "=f"(r[27]), "=f"(r[28]), "=f"(r[29]), "=f"(r[30]), "=f"(r[31])
                 : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const float (&r)[32])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,"
                 "%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
                 ::"r"(taddr), "f"(r[0]), "f"(r[1]), "f"(r[2]), "f"(r[3]), "f"(r[4]), "f"(r[5]), "f"(r[6]), "f"(r[7]), "f"(r[8]),
                   "f"(r[9]), "f"(r[10]), "f"(r[11]), "f"(r[12]), "f"(r[13]), "f"(r[14]), "f"(r[15]), "f"(r[16]), "f"(r[17]),
                   "f"(r[18]), "f"(r[19]), "f"(r[20]), "f"(r[21]), "f"(r[22]), "f"(r[23]), "f"(r[24]), "f"(r[25]), "f"(r[26]),
                   "f"(r[27]), "f"(r[28]), "f"(r[29]), "f"(r[30]), "f"(r[31]) : "memory");
}
__device__ __forceinline__ void tmem_ld8_u32(uint32_t taddr, uint32_t (&r)[8])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_ld_n(uint32_t taddr, float (&r)[32]) { tmem_ld32(taddr, r); }
__device__ __forceinline__ void tmem_ld_n(uint32_t taddr, float (&r)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]),
                   "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15])
                 : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st_n(uint32_t taddr, const uint32_t (&r)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
                   "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tmem_st_n(uint32_t taddr, const uint32_t (&r)[8])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
// two fp32 operations in one instruction
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(reinterpret_cast<unsigned long long&>(r))
        : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)), "l"(reinterpret_cast<unsigned long long&>(c)));
    return r;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<unsigned long long&>(r))
        : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)));
    return r;
}
// fast_exp2 that stays in its place among its like (a lone warp on a scheduler, d = 256, then runs its exponentials in one sweep;
// with two warps, d = 128, the compiler's order is as fast and takes fewer registers)
__device__ __forceinline__ float exp2_in_order(float x)
{
    float r;
    asm volatile("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ uint32_t hmul2_u32(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ __half2 as_half2(uint32_t x) { return *reinterpret_cast<const __half2*>(&x); }
__device__ __forceinline__ uint32_t as_u32(__half2 x) { return *reinterpret_cast<const uint32_t*>(&x); }
__device__ __forceinline__ uint4 ldg128(const void* p)          // coherent: pages may have been written by the kernel before
{
    uint4 v;
    asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ uint2 ldg64(const void* p)
{
    uint2 v;
    asm volatile("ld.global.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
    return v;
}
__device__ __forceinline__ uint32_t ldg16(const void* p)
{
    uint16_t v;
    asm volatile("ld.global.u16 %0, [%1];" : "=h"(v) : "l"(p));
    return v;
}
__device__ __forceinline__ uint32_t ldg32(const void* p)
{
    uint32_t v;
    asm volatile("ld.global.u32 %0, [%1];" : "=r"(v) : "l"(p));
    return v;
}

// four key levels of record format 2 from four nibbles (the fp16 levels 3400, 3A00, 3D80, 4080 | sign)
__device__ __forceinline__ void key_lut4_v2(uint32_t sel, uint32_t& r0, uint32_t& r1)
{
    const uint32_t hi = prmt(0x403D3A34u, 0xC0BDBAB4u, sel);
    const uint32_t lo = prmt(0x80800000u, 0x80800000u, sel);
    r0 = prmt(lo, hi, 0x5140u);
    r1 = prmt(lo, hi, 0x7362u);
}

// Key row of token t of the run e in a tile: FP8 tiles keep the order; Stale tiles follow the lanes of the value codes,
// which hold tokens 2q, 2q + 1, 2q + 8, 2q + 9 of a run: two runs' shares are one 16-byte chunk, chunk 2q + (pair mod 2).
__device__ __forceinline__ int stale_row(int e, int t)
{
    return 64 * (e >> 2) + 8 * (2 * ((t & 7) >> 1) + ((e >> 1) & 1)) + 4 * (e & 1) + 2 * (t >> 3) + (t & 1);
}
// So key row n is token 2 (n / 16 mod 4) + 8 (n / 2 mod 2) + n mod 2 of run 4 (n / 64) + 2 (n / 8 mod 2) + n / 4 mod 2.

// A run of 16 tokens in a list of pages; moves on by a key tile (eight runs).
struct Cursor {
    int page, sub, left;                      // page of the list, run within it, runs from here to the end of the list

    __device__ __forceinline__ void open(int run, int n, int tiles)
    {
        page = run / tiles;
        sub = run - page * tiles;
        left = n - run;
    }
    __device__ __forceinline__ void next(int tiles)
    {
        left -= 8;
        if (tiles == 1) page += 8;
        else {
            sub += 8;
            if (sub >= tiles) {
                const int q = sub / tiles;
                page += q;
                sub -= q * tiles;
            }
        }
    }
};

// ---- scan -------------------------------------------------------------------------------------------
template <int D, int FMT>
__global__ void __launch_bounds__(Geo<D>::THREADS, 1) chunk_scan_kernel(const Params P)
{
    using G = Geo<D>;
    using namespace tm;
    constexpr int NT = G::NT, ROWS = G::ROWS, COLS = G::COLS;
    constexpr uint32_t FULL = 0xffffffffu;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_at = smem_u32(smem_raw), sb = (raw_at + 1023) & ~1023u;
    uint8_t* smem = smem_raw + (sb - raw_at);
    float* fac_s = reinterpret_cast<float*>(smem + G::OFF_FAC);
    unsigned long long* nan_s = reinterpret_cast<unsigned long long*>(smem + G::OFF_NAN);
    const uint32_t failed_at = sb + G::OFF_MISC;                 // word: a wait has given up
    uint32_t* tmem_s = reinterpret_cast<uint32_t*>(smem + G::OFF_MISC + 4);
    constexpr int kFinished = 16 + (int)sizeof(Share);           // word per softmax warp: the last segment that it is done with
    static_assert(kFinished % 4 == 0 && kFinished + 4 * G::SOFT_WARPS <= 128, "words behind the share");
    const uint32_t finished_at = sb + G::OFF_MISC + kFinished;
    volatile uint32_t* noted_s = reinterpret_cast<volatile uint32_t*>(smem + G::OFF_MISC + 8);    // segment of the latest note
    Share* share = reinterpret_cast<Share*>(smem + G::OFF_MISC + 16);
    // (the warp's number as a uniform value: whole-warp branches are then known as such)
    const int tid = threadIdx.x, warp = (int)uniform((uint32_t)tid >> 5), lane = tid & 31;
    auto bar = [&](int i) -> uint32_t { return sb + G::OFF_BAR + 8 * i; };

    if (tid == 0) {
        for (int i = 0; i < kBars; ++i) {
            int count = 1;
            if ((i >= kKFull && i < kKEmpty) || (i >= kVFull && i < kVEmpty) || i == kQFull) count = G::UNPACK_WARPS;
            else if (i >= kPFull && i < kPvDone) count = 4;
            else if (i == kFacRead) count = G::SOFT_WARPS;
            mbar_init(bar(i), count);
        }
        sts32(failed_at, 0);
        *noted_s = 0;
        for (int w = 0; w < G::SOFT_WARPS; ++w) sts32(finished_at + 4 * w, 0);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    for (int i = tid; i < D; i += G::THREADS) nan_s[i] = 0;
    pdl_wait();
    // ---- the block's share: [p0, p1) of the units laid end to end
    if (warp == 0) {
        long long total = 0;
        for (int i = lane; i < P.B; i += 32) total += P.req[i].cost;
        total *= P.hkv;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(FULL, total, o);
        const long long per = max((total + gridDim.x - 1) / gridDim.x, (long long)kLeastShare);
        const long long p0 = per * blockIdx.x;
        long long before = 0, at = 0;
        int found = -1;
        for (int i0 = 0; i0 < P.B && p0 < total && found < 0; i0 += 32) {
            const long long c = i0 + lane < P.B ? P.req[i0 + lane].cost * P.hkv : 0;
            long long s = c;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long a = __shfl_up_sync(FULL, s, o);
                if (lane >= o) s += a;
            }
            const uint32_t m = __ballot_sync(FULL, before + s > p0);
            if (m) {
                const int src = __ffs(m) - 1;
                found = i0 + src;
                at = before + __shfl_sync(FULL, s - c, src);
            }
            before += __shfl_sync(FULL, s, 31);
        }
        if (lane == 0) {
            share->request = found;
            share->request_start = at;
            share->p0 = p0;
            share->p1 = min(total, p0 + per);
            share->per = per;
        }
    }
    __syncthreads();
    if (tid == 0) P.merge[blockIdx.x].b = -1;
    if (share->request < 0) return;                                          // nothing to do (and nothing allocated yet)
    if (warp == G::MMA_WARP) tmem_alloc(smem_u32(tmem_s), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tb = *tmem_s;
    constexpr uint32_t kColS = NT * D;                           // O: NT x D columns, then two score buffers
    Walk* walk = reinterpret_cast<Walk*>(smem + G::OFF_WALK) + warp;
    const Segment& s = walk->s;
    walk->open<ROWS>(P, share, lane);
    auto next_segment = [&]() -> bool {
        __syncwarp();                                            // the segment before is no longer looked at
        bool more = false;
        if (lane == 0) more = walk->next<ROWS>(P, share);
        __syncwarp();
        return __any_sync(FULL, more);
    };

    // Bounded by wall time: a wait that gives up flags the pool and lets every later wait of the block pass.  Polls are few
    // instructions, since they take issue slots from the working warps.
    // The whole warp waits, and is in step again afterwards (what follows may be an instruction of the whole warp).
    auto wait = [&](int i, uint32_t parity) {
        const uint32_t a = bar(i);
        if (!mbar_try_wait(a, parity)) {
            unsigned long long t0 = 0, t1;
            for (int polls = 1; !mbar_try_wait(a, parity); ++polls) {
                __nanosleep(20);
                if (polls & 63) continue;
                if (lds32(failed_at)) break;
                asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t1));
                if (t0 == 0) t0 = t1;
                if (t1 - t0 > P.wait_ns) {
                    sts32(failed_at, 1);
                    atomicOr(P.status, kStTimeout);
                }
            }
        }
        __syncwarp();
    };

    if (warp >= G::MMA_WARP) {
        // ================= products =================
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(G::MMA_REGS));
        if (warp == G::MMA_WARP) {
            constexpr uint32_t kTb = 0;                          // the whole of tensor memory is this block's
            uint32_t job = 0, tile = 0, fills = 0;               // scores, key tiles and queries so far
            while (next_segment()) {
                const int nt = (int)uniform(s.nt), n = (int)uniform(s.t1 - s.t0) * nt;
                const int turn = (int)uniform(max(s.u.stale_tiles - s.t0, 0));        // key tile of the segment that starts the FP8 ones
                // job i of the segment: key tile t0 + i / nt, row tile i % nt; its scores are issued two jobs ahead.  With one row
                // tile where there is room for two, the key tiles go by turns to two accumulators (and softmax groups).
                const bool by_turns = NT == 2 && nt == 1;
                // limit 0 (diagnostic): the first look comes while the query's loads are in flight
                if (P.wait_ns == 0 && fills == 0 && n > 0 && !mbar_test_wait(bar(kQFull), 0)) {
                    sts32(failed_at, 1);
                    atomicOr(P.status, kStTimeout);
                }
                for (int i = -2; i < n; ++i) {
                    if (i >= 0) {
                        const uint32_t j = nt == 2 ? i >> 1 : i, t = NT == 2 ? i & 1 : 0;
                        const uint32_t at = tile + j, st = at % G::STAGES, buf = (job + i) & 1;
                        if (t == 0 || by_turns) wait(kVFull + st, (at / G::STAGES) & 1);
                        wait(kPFull + buf, ((job + i) >> 1) & 1);
                        tc_fence_after();
                        const uint64_t v = operand_desc(sb + G::OFF_V + st * G::V_TILE);
                        const uint32_t o = kTb + t * D, p = kTb + kColS + kKeys * buf;
#pragma unroll
                        for (int kk = 0; kk < kKeys / 16; ++kk)
                            issue_ts(o, p + 8 * kk, v + (((kk >> 2) * (D * 128) + (kk & 3) * 32) >> 4), idesc(D), kk > 0 ? 1u : (i >= NT ? 1u : 0u));
                        issue_commit(bar(kPvDone + t));
                        if (i + NT >= n) issue_commit(bar(kOutput + t));
                        if (by_turns || (int)t == nt - 1) issue_commit(bar(kVEmpty + st));
                    }
                    if (i + 2 < n) {
                        const uint32_t i2 = i + 2, j = nt == 2 ? i2 >> 1 : i2, t = NT == 2 && !by_turns ? i2 & 1 : 0;
                        const uint32_t at = tile + j, st = at % G::STAGES, buf = (job + i2) & 1;
                        if (t == 0) {
                            if (j == 0 || (int)j == turn) wait(kQFull, fills++ & 1);
                            wait(kKFull + st, (at / G::STAGES) & 1);
                            tc_fence_after();
                        }
                        const uint64_t a = operand_desc(sb + G::OFF_Q + t * G::Q_TILE), k = operand_desc(sb + G::OFF_K + st * G::K_TILE);
                        const uint32_t d = kTb + kColS + kKeys * buf;
#pragma unroll
                        for (int kk = 0; kk < D / 16; ++kk) {
                            const uint64_t step = ((kk >> 2) * (128 * 128) + (kk & 3) * 32) >> 4;
                            issue_ss(d, a + step, k + step, idesc(kKeys), kk > 0);
                        }
                        issue_commit(bar(kSFull + buf));
                        if ((int)t == nt - 1) issue_commit(bar(kKEmpty + st));
                    }
                }
                job = uniform(job + n);
                tile = uniform(tile + n / nt);
            }
            // tensor memory is given back when nothing writes it any more (also after a wait that gave up; bounded again)
            issue_commit(bar(kDrained));
            unsigned long long t0, t1;
            asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t0));
            while (!mbar_try_wait(bar(kDrained), 0)) {
                asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t1));
                if (t1 - t0 > 20000000ull) {
                    atomicOr(P.status, kStTimeout);
                    break;
                }
            }
        }
        __syncwarp();
    } else if (warp >= G::SOFT_WARPS) {
        // ================= queries and unpacking =================
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(G::UNPACK_REGS));
        const int w = warp - G::SOFT_WARPS, g = lane >> 2, tq = lane & 3;
        const uint32_t ku = (uint32_t)(15 - P.ke) << 10, vu = (uint32_t)(15 - P.ve) << 10;     // 2^-ke, 2^-ve as fp16
        const uint32_t k_unit = ku | ku << 16, v_unit = vu | vu << 16;
        uint32_t k_tile = 0, v_tile = 0, fills = 0, segments = 0;   // key tiles and value tiles unpacked so far
        auto arrive = [&](int i) {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(i));
        };
        while (next_segment()) {
            ++segments;
            const int first_pos = s.r.len - s.r.n_new + s.rt * ROWS / P.group;        // of the unit's first row
            const int rows = min(ROWS, s.r.n_new * P.group - s.rt * ROWS);
            const int2* list = P.list + (size_t)s.b * P.max_pages;
            const size_t page8 = fp8_page_bytes(D, P.tiles), page3 = tq3_page_bytes(D, P.tiles);
            const uint32_t stride8 = (uint32_t)(P.hkv * page8), stride3 = (uint32_t)(P.hkv * page3);     // of a page (launch checks)
            const uint8_t* base8 = P.fp8 + s.h * page8;
            const uint8_t* base3 = P.tq3 + s.h * page3;

            // ---- queries of one format: a warp per row, a lane D / 32 dims
            auto fill_query = [&](bool stale, uint32_t tiles) {  // tiles: key tiles whose products take the query before
                if (tiles > 0) wait(kKEmpty + (tiles - 1) % G::STAGES, ((tiles - 1) / G::STAGES) & 1);
                if (fills > 0) wait(kFacRead, (fills - 1) & 1);
                ++fills;
                constexpr int N = D / 32;
                // (rows behind the last one stay what they are: a row of a product sees no other)
                for (int r0 = w * 4; r0 < ((rows + 31) & ~31); r0 += 4 * G::UNPACK_WARPS) {
                    uint32_t raw[4][N / 2];
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const int r = r0 + u, row = s.rt * ROWS + r, tok = row / P.group;
#pragma unroll
                        for (int i = 0; i < N / 2; ++i) raw[u][i] = 0;
                        if (r < rows) {
                            const __nv_bfloat16* src = P.q + (size_t)(s.r.row0 + tok) * P.q_stride +
                                                       (size_t)(s.h * P.group + row - tok * P.group) * D + lane * N;
                            if constexpr (N == 8) {
                                const uint4 v = ldg128(src);
                                raw[u][0] = v.x; raw[u][1] = v.y; raw[u][2] = v.z; raw[u][3] = v.w;
                            } else {
                                const uint2 v = ldg64(src);
                                raw[u][0] = v.x; raw[u][1] = v.y;
                            }
                        }
                    }
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const int r = r0 + u;
                        float x[N];
#pragma unroll
                        for (int i = 0; i < N / 2; ++i) {
                            x[2 * i] = __uint_as_float(raw[u][i] << 16);
                            x[2 * i + 1] = __uint_as_float(raw[u][i] & 0xffff0000u);
                        }
                        if (stale) {
#pragma unroll
                            for (int i = 0; i < N; ++i) {
                                const int dim = lane * N + i;
                                if ((P.sigma.w[dim >> 5] >> (dim & 31)) & 1u) x[i] = -x[i];
                            }
#pragma unroll
                            for (int hh = 1; hh < N; hh <<= 1)
#pragma unroll
                                for (int i = 0; i < N; ++i)
                                    if ((i & hh) == 0) {
                                        const float p = x[i], q = x[i + hh];
                                        x[i] = p + q;
                                        x[i + hh] = p - q;
                                    }
#pragma unroll
                            for (int m = 1; m < 32; m <<= 1)
#pragma unroll
                                for (int i = 0; i < N; ++i) {
                                    const float o = __shfl_xor_sync(FULL, x[i], m);
                                    x[i] = (lane & m) ? o - x[i] : x[i] + o;
                                }
                            const float rs = D == 256 ? 0.0625f : 0.08838834764831845f;        // d^-1/2
#pragma unroll
                            for (int i = 0; i < N; ++i) x[i] *= rs;
                        }
                        // a power of two brings the largest element to [1/2, 1): exact for the plain query
                        float big = 0.f;
#pragma unroll
                        for (int i = 0; i < N; ++i) big = fmaxf(big, fabsf(x[i]));
#pragma unroll
                        for (int m = 16; m > 0; m >>= 1) big = fmaxf(big, __shfl_xor_sync(FULL, big, m));
                        // (within [1/4, 4) at the ends of fp32's range; zeros and infinities stay what they are)
                        const int e = min(max((int)(__float_as_uint(big) >> 23) - 126, -126), 126);
                        const float down = __uint_as_float((uint32_t)(127 - e) << 23), up = __uint_as_float((uint32_t)(127 + e) << 23);
                        const float sg = P.negative ? -down : down;
                        uint32_t h2[N / 2];
#pragma unroll
                        for (int i = 0; i < N / 2; ++i) h2[i] = pack_f16x2(x[2 * i] * sg, x[2 * i + 1] * sg);
                        if (lane == 0)
                            fac_s[r] = fmaxf(P.sc2 * up * (stale ? __uint_as_float((uint32_t)(127 + P.ke) << 23) : P.k_scale), 1e-30f);
                        const uint32_t row_at = sb + G::OFF_Q + (r >> 7) * G::Q_TILE;
                        const int rr = r & 127, d0 = lane * N;
                        if (!stale) {
                            const uint32_t a = row_at + (d0 >> 6) * (128 * 128) + chunk_at(rr, (d0 & 63) >> 3);
                            if constexpr (N == 8) sts128(a, h2[0], h2[1], h2[2], h2[3]);
                            else sts64(a + (d0 & 7) * 2, h2[0], h2[1]);
                        } else if constexpr (FMT == 2) {
                            // dims 4 q .. 4 q + 3 (+ 16) of a 32-dim step: chunk 2 q + step, elements 4 (k / 16) ..
#pragma unroll
                            for (int i = 0; i < N; i += 4) {
                                const int dim = d0 + i, k = dim & 31;
                                const int c = 2 * ((k & 15) >> 2) + ((dim >> 5) & 1);
                                sts64(row_at + (dim >> 6) * (128 * 128) + chunk_at(rr, c) + 8 * (k >> 4), h2[i / 2], h2[i / 2 + 1]);
                            }
                        } else {
                            // dims 2 q, 2 q + 1 (+ 8) of a 16-dim block: chunk 2 q + (block / 2 mod 2), elements 4 (block mod 2) ..
#pragma unroll
                            for (int i = 0; i < N; i += 2) {
                                const int dim = d0 + i, sl = dim & 15, kb = (dim >> 4) & 3;
                                const int c = 2 * ((sl & 7) >> 1) + (kb >> 1);
                                sts32(row_at + (dim >> 6) * (128 * 128) + chunk_at(rr, c) + 8 * (kb & 1) + 4 * (sl >> 3), h2[i / 2]);
                            }
                        }
                    }
                }
                arrive(kQFull);
            };

            // An FP8 value that is NaN is as a rule seen by every row of the tile (0 x NaN).  In a tile with masked places
            // its bytes are cleared and the channel's first such position is noted; the epilogue gives NaN to the rows
            // from there on.  The note carries the segment, and the epilogue of the segment before is waited for.
            auto note_nan = [&](uint4 (&x)[16 * D / 512], int pos) {
                // (Words, not a barrier: the roles may be several segments apart.  One of each warp, not their sum: warps without
                // rows are done with a segment at once, and with one or two key tiles also with the next.)
                auto finished = [&] {
                    bool all = true;
#pragma unroll
                    for (int k = 0; k < G::SOFT_WARPS; ++k) all &= lds32(finished_at + 4 * k) + 1 >= segments;
                    return all;
                };
                unsigned long long t0, t1;
                asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t0));
                while (!finished() && !lds32(failed_at)) {
                    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t1));
                    if (t1 - t0 > P.wait_ns) {
                        sts32(failed_at, 1);
                        atomicOr(P.status, kStTimeout);
                    }
                }
#pragma unroll
                for (int i = 0; i < 16 * D / 512; ++i) {
                    uint32_t* word = reinterpret_cast<uint32_t*>(&x[i]);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const uint32_t bad = __vcmpeq4(word[q] & 0x7f7f7f7fu, 0x7f7f7f7fu);
                        if (!bad) continue;
                        const int at = pos + 4 * q + ((__ffs(bad) - 1) >> 3);
                        atomicMax(&nan_s[i * 32 + lane], (unsigned long long)segments << 32 | (uint32_t)(kNoPos - at));
                        *noted_s = segments;
                        word[q] &= ~bad;
                    }
                }
            };

            const int cut = s.u.stale_tiles, len = s.r.len;
            if (s.t0 < cut) {
                // ---- Stale tiles.  Keys: a warp per run.  Values: two warps for two runs (whose shares make up 16-byte
                // chunks), half of the channels each.
                constexpr int KW = 3 * D / 64, BLOCKS = D / 32;  // packed key words of a lane, 16-channel blocks of a warp
                const int n_tiles = min(s.t1, cut), half = w & 1;
                // Ids of the runs to load next, looked up a tile ahead.  Nothing here may look at what a load brings: that
                // would hold the warp until it is there.  So runs behind the list's end load its last page, and are cleared
                // where they are unpacked.
                const int last_page = (s.r.n_stale + P.tiles - 1) / P.tiles - 1;
                Cursor kc, vc;
                int k_id, v_id[2], k_live, v_live;               // live: runs that the loaded words hold
                kc.open(s.t0 * 8 + w, s.r.n_stale, P.tiles);
                vc.open(s.t0 * 8 + (w & ~1), s.r.n_stale, P.tiles);
                auto look_keys = [&] { k_id = (int)ldg32(&list[min(kc.page, last_page)].y); };
                auto look_values = [&] {                         // a run and the one behind it
                    v_id[0] = (int)ldg32(&list[min(vc.page, last_page)].y);
                    v_id[1] = (int)ldg32(&list[min(vc.page + (vc.sub + 1 == P.tiles ? 1 : 0), last_page)].y);
                };
                look_keys();
                look_values();
                uint32_t kw[KW], gw[2], vw[2][KW / 2 + (KW / 2 & 1)], mw[2][BLOCKS][2];
                auto load_keys = [&] {                           // of the tile that kc is at, which moves on
                    const uint8_t* r = base3 + (unsigned long long)(uint32_t)k_id * stride3 + kc.sub * (uint32_t)(12 * D + 32);
#pragma unroll
                    for (int c = 0; c < KW / 4; ++c) {
                        const uint4 v = ldg128(r + c * 512 + lane * 16);
                        kw[4 * c] = v.x; kw[4 * c + 1] = v.y; kw[4 * c + 2] = v.z; kw[4 * c + 3] = v.w;
                    }
                    if constexpr (KW % 4 != 0) {
                        const uint2 v = ldg64(r + (KW / 4) * 512 + lane * 8);
                        kw[KW - 2] = v.x; kw[KW - 1] = v.y;
                    }
                    gw[0] = ldg16(r + 12 * D + 2 * g);           // g of tokens g and g + 8
                    gw[1] = ldg16(r + 12 * D + 2 * g + 16);
                    k_live = kc.left;
                    kc.next(P.tiles);
                    look_keys();
                };
                auto load_values = [&] {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint8_t* page = base3 + (unsigned long long)(uint32_t)v_id[e] * stride3;
                        const int sub = e == 0 ? vc.sub : vc.sub + 1 == P.tiles ? 0 : vc.sub + 1;
                        const uint8_t* at = page + sub * (uint32_t)(12 * D + 32) + 6 * D + lane * 16;
                        if constexpr (D == 256) {                // words 0-5 or 6-11 of the lane
                            if (half == 0) {
                                const uint4 a = ldg128(at);
                                const uint2 c = ldg64(at + 512);
                                vw[e][0] = a.x; vw[e][1] = a.y; vw[e][2] = a.z; vw[e][3] = a.w; vw[e][4] = c.x; vw[e][5] = c.y;
                            } else {
                                const uint2 a = ldg64(at + 512 + 8);
                                const uint4 c = ldg128(at + 1024);
                                vw[e][0] = a.x; vw[e][1] = a.y; vw[e][2] = c.x; vw[e][3] = c.y; vw[e][4] = c.z; vw[e][5] = c.w;
                            }
                        } else {                                 // words 0-2 or 3-5
                            if (half == 0) {
                                const uint4 a = ldg128(at);
                                vw[e][0] = a.x; vw[e][1] = a.y; vw[e][2] = a.z;
                            } else {
                                vw[e][0] = ldg32(at + 12);
                                const uint2 c = ldg64(at + 512 - lane * 8);
                                vw[e][1] = c.x; vw[e][2] = c.y;
                            }
                        }
                        // scale / zero of the warp's block pairs: (sc g, sc g+8), (zp g, zp g+8), twice
                        const uint8_t* meta = page + P.tiles * (uint32_t)(12 * D + 32) + half * (D / 64) * 128 + g * 16;
#pragma unroll
                        for (int i = 0; i < BLOCKS / 2; ++i) {
                            const uint4 m = ldg128(meta + i * 128);
                            mw[e][2 * i][0] = m.x; mw[e][2 * i][1] = m.y; mw[e][2 * i + 1][0] = m.z; mw[e][2 * i + 1][1] = m.w;
                        }
                    }
                    v_live = vc.left;
                    vc.next(P.tiles);
                    look_values();
                };
                auto put_keys = [&] {
                    const uint32_t st = k_tile % G::STAGES;
                    if (k_tile >= G::STAGES) wait(kKEmpty + st, (k_tile / G::STAGES & 1) ^ 1);
                    const uint32_t k_at = sb + G::OFF_K + st * G::K_TILE;
                    const int n0 = stale_row(w, g), n1 = stale_row(w, g + 8);
                    const uint32_t g0 = k_live > 0 ? hmul2_u32(prmt(gw[0], gw[0], 0x1010u), k_unit) : 0u;        // no run: zeros
                    const uint32_t g1 = k_live > 0 ? hmul2_u32(prmt(gw[1], gw[1], 0x1010u), k_unit) : 0u;
#pragma unroll
                    for (int j = 0; j < D / 64; ++j) {
                        const uint32_t A = kw[3 * j], Bw = kw[3 * j + 1], Cw = kw[3 * j + 2];
                        uint32_t sel[4];
                        sel[0] = A & 0x77777777u;
                        sel[1] = Bw & 0x77777777u;
                        sel[2] = lop3_and_or(A >> 1, 0x44444444u, Cw & 0x33333333u);
                        sel[3] = lop3_and_or(Bw >> 1, 0x44444444u, (Cw >> 2) & 0x33333333u);
                        const uint32_t at = k_at + j * (kKeys * 128);
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            uint32_t lo[4], hi[4];               // chunk of token g, of token g + 8
                            if constexpr (FMT == 2) {
                                key_lut4_v2(sel[2 * c], lo[0], lo[1]);
                                key_lut4_v2(sel[2 * c] >> 16, lo[2], lo[3]);
                                key_lut4_v2(sel[2 * c + 1], hi[0], hi[1]);
                                key_lut4_v2(sel[2 * c + 1] >> 16, hi[2], hi[3]);
                            } else {
                                key_lut4(sel[2 * c], lo[0], hi[0]);
                                key_lut4(sel[2 * c] >> 16, lo[1], hi[1]);
                                key_lut4(sel[2 * c + 1], lo[2], hi[2]);
                                key_lut4(sel[2 * c + 1] >> 16, lo[3], hi[3]);
                            }
                            sts128(at + chunk_at(n0, 2 * tq + c), hmul2_u32(lo[0], g0), hmul2_u32(lo[1], g0), hmul2_u32(lo[2], g0), hmul2_u32(lo[3], g0));
                            sts128(at + chunk_at(n1, 2 * tq + c), hmul2_u32(hi[0], g1), hmul2_u32(hi[1], g1), hmul2_u32(hi[2], g1), hmul2_u32(hi[3], g1));
                        }
                    }
                    arrive(kKFull + st);
                    ++k_tile;
                };
                auto put_values = [&] {
                    if (v_live < 2) {                            // no second run, or none: scale and zero of 0
#pragma unroll
                        for (int i = 0; i < BLOCKS; ++i) {
                            mw[1][i][0] = mw[1][i][1] = 0;
                            if (v_live < 1) mw[0][i][0] = mw[0][i][1] = 0;
                        }
                    }
                    if (P.ve != 0) {
#pragma unroll
                        for (int e = 0; e < 2; ++e)
#pragma unroll
                            for (int i = 0; i < BLOCKS; ++i) {
                                mw[e][i][0] = hmul2_u32(mw[e][i][0], v_unit);
                                mw[e][i][1] = hmul2_u32(mw[e][i][1], v_unit);
                            }
                    }
                    const uint32_t st = v_tile % G::STAGES;
                    if (v_tile >= G::STAGES) wait(kVEmpty + st, (v_tile / G::STAGES & 1) ^ 1);
                    const int c = 2 * tq + ((w >> 1) & 1), ch0 = half * (D / 2) + g;
                    const uint32_t v_at = sb + G::OFF_V + st * G::V_TILE + (w >> 2) * (D * 128) + chunk_at(ch0, c);
#pragma unroll
                    for (int j = 0; j < D / 128; ++j) {          // 64 channels: four blocks of 16
                        uint32_t X[2][2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            X[e][0] = prmt(vw[e][3 * j], vw[e][3 * j + 1], 0x6341u);
                            X[e][1] = prmt(vw[e][3 * j + 1], vw[e][3 * j + 2], 0x6341u);
                        }
                        auto put_block = [&](auto block) {       // rows g and g + 8
                            constexpr int B4 = decltype(block)::value;
                            const int i = 4 * j + B4;
                            uint32_t o[2][4];                    // run e: row g (tokens low, high), row g + 8 (low, high)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                uint32_t a[4];
                                value_operands<B4>(a, vw[e][3 * j], vw[e][3 * j + 1], vw[e][3 * j + 2], X[e][B4 >> 1]);
                                const __half2 sc = as_half2(mw[e][i][0]), zp = as_half2(mw[e][i][1]);
                                o[e][0] = as_u32(__hfma2(as_half2(a[0]), __low2half2(sc), __low2half2(zp)));
                                o[e][1] = as_u32(__hfma2(as_half2(a[2]), __low2half2(sc), __low2half2(zp)));
                                o[e][2] = as_u32(__hfma2(as_half2(a[1]), __high2half2(sc), __high2half2(zp)));
                                o[e][3] = as_u32(__hfma2(as_half2(a[3]), __high2half2(sc), __high2half2(zp)));
                            }
                            sts128(v_at + i * 2048, o[0][0], o[0][1], o[1][0], o[1][1]);
                            sts128(v_at + i * 2048 + 1024, o[0][2], o[0][3], o[1][2], o[1][3]);
                        };
                        put_block(Int<0>{});
                        put_block(Int<1>{});
                        put_block(Int<2>{});
                        put_block(Int<3>{});
                    }
                    arrive(kVFull + st);
                    ++v_tile;
                };
                load_keys();
                load_values();
                {                                                // the first keys need not wait for the query's turn
                    const uint32_t before = k_tile;
                    put_keys();
                    load_keys();
                    fill_query(true, before);
                }
                for (int t = n_tiles - s.t0; t > 0; --t) {
                    if (t > 1) {
                        put_keys();
                        load_keys();
                    }
                    put_values();
                    load_values();
                }
            }
            if (s.t1 > cut) {
                // ---- FP8 tiles: a warp per run
                constexpr int N = 16 * D / 512;                  // 16-byte loads of a lane for a run's keys, or values
                const int t_first = max(s.t0, cut);
                // the run to load next (keys), looked up a tile ahead as above, and that of the tile before it (values)
                const int last_page = (s.u.n_fp8 + P.tiles - 1) / P.tiles - 1;
                Cursor kc;
                uint2 k_page, v_page = make_uint2(0, 0);
                int k_sub, v_sub = 0, k_left, v_left = 0;
                kc.open((t_first - cut) * 8 + w, s.u.n_fp8, P.tiles);
                auto look = [&] {
                    k_page = ldg64(&list[P.max_pages - 1 - min(kc.page, last_page)]);
                    k_sub = kc.left > 0 ? kc.sub : 0;
                    k_left = kc.left;
                };
                look();
                uint4 kr[N], vr[N];
                int v_lp, v_at_sub, v_live;                      // of the run whose values are loaded
                auto load = [&](uint4 (&x)[N], uint32_t id, int sub, int off) {
                    const uint8_t* rec = base8 + (unsigned long long)id * stride8 + sub * (uint32_t)(32 * D) + off;
#pragma unroll
                    for (int i = 0; i < N; ++i) x[i] = ldg128(rec + i * 512);
                };
                // eight lanes take 64 dims of two keys: their 16-byte stores meet every bank once
                const int k_tok = (D == 128 ? 2 * (lane >> 4) : 0) + ((lane >> 2) & 1), k_atom = D == 128 ? (lane >> 3) & 1 : lane >> 3;
                auto load_keys = [&] { load(kr, k_page.y, k_sub, k_tok * D + k_atom * 64 + (lane & 3) * 16); };
                auto load_values = [&] {
                    load(vr, v_page.y, v_sub, 16 * D + lane * 16);
                    v_lp = (int)v_page.x;
                    v_at_sub = v_sub;
                    v_live = v_left;
                };
                auto move_on = [&] {
                    v_page = k_page;
                    v_sub = k_sub;
                    v_left = k_left;
                    kc.next(P.tiles);
                    look();
                };
                auto put_keys = [&] {
                    const uint32_t st = k_tile % G::STAGES;
                    if (k_tile >= G::STAGES) wait(kKEmpty + st, (k_tile / G::STAGES & 1) ^ 1);
                    const uint32_t k_at = sb + G::OFF_K + st * G::K_TILE;
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const int row = 16 * w + k_tok + i * (512 / D), c = 2 * (lane & 3);
                        const uint32_t x[4] = {kr[i].x, kr[i].y, kr[i].z, kr[i].w};
                        uint32_t o[8];
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            o[2 * q] = e4m3x2_to_f16x2((uint16_t)(x[q] & 0xffffu));
                            o[2 * q + 1] = e4m3x2_to_f16x2((uint16_t)(x[q] >> 16));
                        }
                        const uint32_t at = k_at + k_atom * (kKeys * 128);
                        sts128(at + chunk_at(row, c), o[0], o[1], o[2], o[3]);
                        sts128(at + chunk_at(row, c + 1), o[4], o[5], o[6], o[7]);
                    }
                    arrive(kKFull + st);
                    ++k_tile;
                };
                auto put_values = [&] {
                    const uint32_t st = v_tile % G::STAGES;
                    if (v_tile >= G::STAGES) wait(kVEmpty + st, (v_tile / G::STAGES & 1) ^ 1);
                    const int v_pos = (v_lp * P.tiles + v_at_sub) * kPage, left = v_live > 0 ? len - v_pos : 0;   // tokens that exist
                    if (left < kPage) {                          // what no token fills may be anything
#pragma unroll
                        for (int i = 0; i < N; ++i) {
                            uint32_t* word = reinterpret_cast<uint32_t*>(&vr[i]);
#pragma unroll
                            for (int q = 0; q < 4; ++q) {
                                const int keep = left - 4 * q;
                                word[q] &= keep >= 4 ? FULL : keep <= 0 ? 0u : (1u << (8 * keep)) - 1u;
                            }
                        }
                    }
                    if (left > 0 && v_pos + kPage - 1 > first_pos) {                  // some row does not see the whole run
                        uint32_t bad = 0;
#pragma unroll
                        for (int i = 0; i < N; ++i) {
                            const uint32_t x[4] = {vr[i].x, vr[i].y, vr[i].z, vr[i].w};
#pragma unroll
                            for (int q = 0; q < 4; ++q) bad |= __vcmpeq4(x[q] & 0x7f7f7f7fu, 0x7f7f7f7fu);
                        }
                        if (bad) note_nan(vr, v_pos);
                        __syncwarp();
                    }
                    const uint32_t v_at = sb + G::OFF_V + st * G::V_TILE + (w >> 2) * (D * 128);
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const int ch = i * 32 + lane, c = 2 * (w & 3);
                        const uint32_t x[4] = {vr[i].x, vr[i].y, vr[i].z, vr[i].w};
                        uint32_t o[8];
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            o[2 * q] = e4m3x2_to_f16x2((uint16_t)(x[q] & 0xffffu));
                            o[2 * q + 1] = e4m3x2_to_f16x2((uint16_t)(x[q] >> 16));
                        }
                        sts128(v_at + chunk_at(ch, c), o[0], o[1], o[2], o[3]);
                        sts128(v_at + chunk_at(ch, c + 1), o[4], o[5], o[6], o[7]);
                    }
                    arrive(kVFull + st);
                    ++v_tile;
                };
                load_keys();
                move_on();
                load_values();
                {                                                // the first keys need not wait for the query's turn
                    const uint32_t before = k_tile;
                    put_keys();
                    load_keys();
                    fill_query(false, before);
                }
                for (int t = s.t1 - t_first; t > 0; --t) {
                    move_on();
                    if (t > 1) {
                        put_keys();
                        load_keys();
                    }
                    put_values();
                    load_values();
                }
            }
        }
    } else {
        // ================= softmax and output =================
        if constexpr (G::SOFT_REGS > G::REGS) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(G::SOFT_REGS));
        const int t = warp >> 2;                                 // row tile
        const uint32_t my_lanes = (uint32_t)(32 * (warp & 3)) << 16;
        const int my_row = t * 128 + (warp & 3) * 32 + lane;     // within the unit
        const uint32_t col_o = tb + my_lanes + t * D;
        uint32_t job = 0, fills = 0, done = 0, outputs = 0, joins = 0, segments = 0;   // done, outputs: value products, segments with any, on this row tile
        auto warp_arrive = [&](int i) {
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(i));
        };
        while (next_segment()) {
            // the output so far times f (a factor of the row), once the products issued so far are done.  (The product before
            // the last is: the scores looked at were issued behind it.  So the barrier's parity is the last one's.)
            auto scale_output = [&](float f) {
                wait(kPvDone + t, (done - 1) & 1);
                tc_fence_after();
#pragma unroll 1
                for (int c = 0; c < D / 8; ++c) {
                    uint32_t y[8];
                    tmem_ld8_u32(col_o + 8 * c, y);
                    tmem_wait_ld();
#pragma unroll
                    for (int k = 0; k < 8; ++k) y[k] = __float_as_uint(__uint_as_float(y[k]) * f);
                    tmem_st_n(col_o + 8 * c, y);
                }
                tmem_wait_st();                                  // (it may be scaled again in the same tile)
            };
            ++segments;
            // one row tile where there is room for two: both groups take its rows, and the key tiles by turns
            const bool by_turns = NT == 2 && s.nt == 1;
            const int in_unit = my_row - (by_turns ? t * 128 : 0), row = s.rt * ROWS + in_unit, n_rows = s.r.n_new * P.group;
            const bool live = row < n_rows, warp_live = row - lane < n_rows;
            const int tok = row / P.group, head = s.h * P.group + row - tok * P.group;
            const int qpos = s.r.len - s.r.n_new + tok;
            const int first_pos = s.r.len - s.r.n_new + (s.rt * ROWS + (by_turns ? 0 : t * 128)) / P.group;
            const int2* list = P.list + (size_t)s.b * P.max_pages;
            const int cut = s.u.stale_tiles, runs = runs_of(s.r.len);
            const bool ordinary = s.r.exact && s.r.stale_end * kPage <= first_pos + 1;     // every Stale page lies before the first row
            float ref = -CUDART_INF_F, sum = 0.f, fac = 0.f;
            int n_done = 0;                                      // key tiles of this segment so far
            bool in_stale = false;                               // the last one was a Stale tile
            const int t0 = s.t0, t1 = s.t1, nt = s.nt, n_stale = s.r.n_stale, n_fp8 = s.u.n_fp8, all_fp8 = s.r.n_fp8;
            for (int kt = t0; kt < t1; ++kt) {
                const bool stale = kt < cut;
                if (kt == t0 || kt == cut) {
                    wait(kQFull, fills++ & 1);
                    fac = fac_s[in_unit];
                    warp_arrive(kFacRead);
                }
                if (by_turns ? ((kt - t0) & 1) != t : t >= nt) continue;
                // from the Stale values' unit to the FP8 values'
                const bool turn = !stale && in_stale && n_done > 0 && P.v_scale != __uint_as_float((uint32_t)(127 + P.ve) << 23);
                in_stale = stale;
                const uint32_t i = by_turns ? job + (uint32_t)(kt - t0) : job + (uint32_t)(kt - t0) * nt + t, buf = i & 1;
                wait(kSFull + buf, (i >> 1) & 1);
                tc_fence_after();
                const uint32_t col_s = tb + my_lanes + kColS + kKeys * buf;
                if (warp_live) {
                    // masks are looked at where the tile is not full, or its last run passes the first row's position
                    const int n_in = min(8, (stale ? n_stale : n_fp8) - (stale ? kt : kt - cut) * 8);
                    bool masked = n_in < 8 || !ordinary;
                    if (!masked && !stale) masked = (runs - all_fp8 + (kt - cut) * 8 + 7) * kPage + kPage - 1 > first_pos;
                    if (masked) {                                // what the row does not see becomes -inf in tensor memory
#pragma unroll 1
                        for (int c = 0; c < 4; ++c) {
                            int seen[4];                         // tokens that the row sees of the runs in these 32 columns
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const int e = stale ? 4 * (c >> 1) + k : 2 * c + (k & 1);
                                seen[k] = 0;
                                if (e < n_in) {
                                    const int run = (stale ? kt : kt - cut) * 8 + e, pg = run / P.tiles, sub = run - pg * P.tiles;
                                    const int lp = list[stale ? pg : P.max_pages - 1 - pg].x;
                                    seen[k] = qpos - (lp * P.tiles + sub) * kPage + 1;
                                }
                            }
                            float x[32];
                            tmem_ld32(col_s + 32 * c, x);
                            tmem_wait_ld();
                            const int t_add = 4 * (c & 1);
#pragma unroll
                            for (int k = 0; k < 32; ++k) {
                                const int lim = stale ? seen[2 * ((k >> 3) & 1) + ((k >> 2) & 1)] : seen[k >> 4];
                                const int tk = stale ? t_add + 2 * (k >> 4) + (k & 1) + 8 * ((k >> 1) & 1) : k & 15;
                                if (tk >= lim) x[k] = -CUDART_INF_F;
                            }
                            tmem_st32(col_s + 32 * c, x);
                        }
                        tmem_wait_st();
                    }
                    const float2 fac2 = make_float2(fac, fac);
                    if (turn) scale_output(__uint_as_float((uint32_t)(127 + P.ve) << 23) / P.v_scale);
                    // Exponentials against the reference so far.  Their sum shows where one has grown too large for fp16 (as a rule
                    // only in a unit's first tile): the reference is then raised by whole powers of two, what was summed or stored
                    // before is scaled down, and the columns are taken again.  (Exactly, but for probabilities that leave fp16's normal
                    // numbers: 2^-25 or less each time, where the row's largest is 2^6 or more.)
#pragma unroll 1
                    for (int c = 0; c < kKeys / COLS; ++c) {
                        float part;
                        uint32_t h2[COLS / 2];
#pragma unroll 1
                        for (bool again = false;; again = true) {
                            float x[COLS];
                            tmem_ld_n(col_s + COLS * c, x);
                            tmem_wait_ld();
                            if (again) {
                                tmem_wait_st();                  // the probabilities of the columns before these are read again
                                float mx = x[0];
#pragma unroll
                                for (int k = 1; k < COLS; ++k) mx = fmaxf(mx, x[k]);
                                mx *= fac;
                                const bool raise = (part > kMostSum || ref == -CUDART_INF_F) && mx > ref + kShift;
                                float up = 0.f;                  // octaves
                                if (raise) {
                                    up = ceilf(mx - kShift - ref);               // infinite where there was none
                                    ref = ref == -CUDART_INF_F ? mx - kShift : ref + up;
                                }
                                const float f = exp2f(-up);
                                sum *= f;
                                if (n_done > 0) scale_output(f);
#pragma unroll 1
                                for (int p = 0; p < c * COLS / 16; ++p) {    // the probabilities of the columns before these
                                    uint32_t y[8];
                                    tmem_ld8_u32(col_s + 8 * p, y);
                                    tmem_wait_ld();
#pragma unroll
                                    for (int k = 0; k < 8; ++k) {            // (by an fp32 factor: fp16 has no 2^-25, but 2^15 times that)
                                        const float2 e = half2_to_float2(y[k]);
                                        y[k] = pack_f16x2(e.x * f, e.y * f);
                                    }
                                    tmem_st_n(col_s + 8 * p, y);
                                }
                            }
                            const float base = ref == -CUDART_INF_F ? 0.f : ref;
                            const float2 base2 = make_float2(-base, -base);
                            float2 s2[4];
                            if constexpr (D == 256) {            // one warp a scheduler: in sweeps, no pair waits for its own steps
#pragma unroll
                                for (int k = 0; k < COLS; k += 2) {
                                    const float2 e = fma2(make_float2(x[k], x[k + 1]), fac2, base2);
                                    x[k] = e.x;
                                    x[k + 1] = e.y;
                                }
#pragma unroll
                                for (int k = 0; k < COLS; ++k) x[k] = exp2_in_order(x[k]);
                            }
#pragma unroll
                            for (int k = 0; k < COLS / 2; ++k) {
                                float2 e = make_float2(x[2 * k], x[2 * k + 1]);
                                if constexpr (D == 128) {
                                    e = fma2(e, fac2, base2);
                                    e.x = fast_exp2(e.x);
                                    e.y = fast_exp2(e.y);
                                }
                                s2[k & 3] = k < 4 ? e : add2(s2[k & 3], e);
                                h2[k] = pack_f16x2(e.x, e.y);
                            }
                            s2[0] = add2(add2(s2[0], s2[1]), add2(s2[2], s2[3]));
                            part = s2[0].x + s2[0].y;
                            if (again || !__any_sync(FULL, part > kMostSum || ref == -CUDART_INF_F)) break;
                        }
                        sum += part;
                        tmem_st_n(col_s + COLS / 2 * c, h2);
                    }
                    tmem_wait_st();
                }
                tc_fence_before();
                warp_arrive(kPFull + buf);
                ++done;
                ++n_done;
            }
            job += (uint32_t)(s.t1 - s.t0) * s.nt;
            if (n_done > 0) ++outputs;
            if ((by_turns || t < s.nt) && warp_live) {
                if (n_done > 0) {
                    wait(kOutput + t, (outputs - 1) & 1);
                    tc_fence_after();
                }
                // by turns: the first group joins both (the second one's reference, sum and unit come through shared memory; its
                // accumulator has the same lanes)
                float join = 0.f;                                // factor of the second accumulator
                int n_join = 0;                                  // key tiles in it (of the whole warp: it decides on loads)
                bool joins_in = false;                           // the row sees any of them
                float unit = in_stale ? __uint_as_float((uint32_t)(127 + P.ve) << 23) : P.v_scale;    // of the accumulator: the last tile's
                if (by_turns) {
                    const uint32_t at = sb + G::OFF_PAIR + 16 * in_unit;
                    if (t == 1) {
                        sts128(at, __float_as_uint(ref), __float_as_uint(sum), __float_as_uint(unit), 0);
                        tc_fence_before();
                        warp_arrive(kJoin + (warp & 3));
                    } else {
                        wait(kJoin + (warp & 3), joins & 1);
                        tc_fence_after();
                        n_join = (t1 - t0) >> 1;
                        const uint4 o = lds128(at);
                        const float ref1 = __uint_as_float(o.x), sum1 = __uint_as_float(o.y), to = fmaxf(ref, ref1);
                        const float f0 = ref == -CUDART_INF_F ? sum : exp2f(ref - to);       // no maximum: nothing, or NaN
                        const float f1 = ref1 == -CUDART_INF_F ? sum1 : exp2f(ref1 - to);
                        sum = sum * f0 + sum1 * f1;
                        unit *= f0;
                        join = f1 * __uint_as_float(o.z);
                        joins_in = f1 != 0.f || ref1 != -CUDART_INF_F;
                        ref = to;
                    }
                }
                if (t == 0 || !by_turns) {                       // this group writes the rows
                    const bool none = sum == 0.f, noted = *noted_s == segments;
                    const float f = s.slot >= 0 ? unit : none ? 0.f : unit / sum, f1 = s.slot >= 0 ? join : none ? 0.f : join / sum;
                    const size_t orow = (size_t)(s.r.row0 + tok) * (P.hkv * P.group) + head;
                    const size_t prow = (size_t)max(s.slot, 0) * ROWS + in_unit;
#pragma unroll 1
                    for (int ch = 0; ch < D; ch += 16) {
                        float x[16], y[16];
                        if (n_done > 0) tmem_ld_n(col_o + ch, x);
                        if (NT == 2 && n_join > 0) tmem_ld_n(col_o + D + ch, y);
                        tmem_wait_ld();
#pragma unroll
                        for (int k = 0; k < 16; ++k) {
                            x[k] = none || n_done == 0 ? 0.f : x[k] * f;
                            if (NT == 2 && n_join > 0) x[k] = joins_in ? fmaf(y[k], f1, x[k]) : x[k];
                        }
                        if (noted) {
#pragma unroll
                            for (int k = 0; k < 16; ++k) {
                                const unsigned long long note = nan_s[ch + k];
                                if ((uint32_t)(note >> 32) == segments && kNoPos - (int)(uint32_t)note <= qpos) x[k] = CUDART_NAN_F;
                            }
                        }
                        if (live && s.slot >= 0) {
                            float4* dst = reinterpret_cast<float4*>(P.part_o + prow * D + ch);
#pragma unroll
                            for (int k = 0; k < 4; ++k) dst[k] = make_float4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]);
                        } else if (live) {
                            uint4* dst = reinterpret_cast<uint4*>(P.out + orow * D + ch);
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                uint32_t o[4];
#pragma unroll
                                for (int q = 0; q < 4; ++q) {
                                    const __nv_bfloat162 p2 = __floats2bfloat162_rn(x[8 * k + 2 * q], x[8 * k + 2 * q + 1]);
                                    o[q] = *reinterpret_cast<const uint32_t*>(&p2);
                                }
                                dst[k] = make_uint4(o[0], o[1], o[2], o[3]);
                            }
                        }
                        __syncwarp();
                    }
                    if (live) {
                        if (s.slot >= 0) P.part_ml[prow] = make_float2(ref, sum);
                        else if (P.lse) P.lse[orow] = none ? -CUDART_INF_F : (ref + log2f(sum)) * 0.6931471805599453f;
                    }
                }
                tc_fence_before();
                if (by_turns) {                                  // the second accumulator has been read
                    if (t == 0) warp_arrive(kJoined + (warp & 3));
                    else wait(kJoined + (warp & 3), joins & 1);
                    ++joins;
                }
            }
            if (s.first_part && tid == 0) {
                Merge m = {};
                m.b = s.b; m.h = s.h; m.rt = s.rt; m.last = s.last_block; m.first_slot = s.slot;
                P.merge[blockIdx.x] = m;
            }
            __threadfence_block();
            __syncwarp();
            if (lane == 0) sts32(finished_at + 4 * warp, segments);
        }
    }
    __syncthreads();
    pdl_let_next_start();
    tc_fence_after();
    if (warp == G::MMA_WARP) tmem_dealloc(tb, 512);
}

// ---- merge ------------------------------------------------------------------------------------------
// Rows of the units that several blocks share: a warp per row, parts in the order of their blocks.
template <int D, int ROWS>
__global__ void __launch_bounds__(256) chunk_merge_kernel(const Params P)
{
    pdl_begin();
    const Merge m = P.merge[blockIdx.x];
    if (m.b < 0) return;
    const Request r = P.req[m.b];
    const int lane = threadIdx.x & 31, in_unit = blockIdx.y * 8 + (threadIdx.x >> 5), row = m.rt * ROWS + in_unit;
    if (row >= r.n_new * P.group) return;
    const int parts = m.last - (int)blockIdx.x + 1;
    auto slot = [&](int i) { return (size_t)(i == 0 ? m.first_slot : 2 * (blockIdx.x + i)) * ROWS + in_unit; };
    float ref = -CUDART_INF_F;
    for (int i = lane; i < parts; i += 32) ref = fmaxf(ref, P.part_ml[slot(i)].x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ref = fmaxf(ref, __shfl_xor_sync(0xffffffffu, ref, o));
    constexpr int N = D / 128;                                   // float4 of a lane
    float4 acc[N];
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < N; ++k) acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int i = 0; i < parts; ++i) {
        const float2 ml = P.part_ml[slot(i)];
        const float f = ml.x == -CUDART_INF_F ? (ml.y == 0.f ? 0.f : ml.y) : exp2f(ml.x - ref);   // a part with NaN scores only has no maximum
        sum = fmaf(ml.y, f, sum);
        const float4* src = reinterpret_cast<const float4*>(P.part_o + slot(i) * D);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float4 v = src[lane + 32 * k];
            acc[k].x = fmaf(v.x, f, acc[k].x);
            acc[k].y = fmaf(v.y, f, acc[k].y);
            acc[k].z = fmaf(v.z, f, acc[k].z);
            acc[k].w = fmaf(v.w, f, acc[k].w);
        }
    }
    const int tok = row / P.group, head = m.h * P.group + row - tok * P.group;
    const size_t orow = (size_t)(r.row0 + tok) * (P.hkv * P.group) + head;
    const float f = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const __nv_bfloat162 a = __floats2bfloat162_rn(acc[k].x * f, acc[k].y * f), c = __floats2bfloat162_rn(acc[k].z * f, acc[k].w * f);
        reinterpret_cast<uint2*>(P.out + orow * D)[lane + 32 * k] =
            make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&c));
    }
    if (lane == 0 && P.lse) P.lse[orow] = sum == 0.f ? -CUDART_INF_F : (ref + log2f(sum)) * 0.6931471805599453f;
}

static size_t up(size_t x) { return (x + 255) / 256 * 256; }

struct Layout { size_t req, merge, ml, o, list, bytes; };
static Layout layout_of(int d, int B, int max_pages)
{
    const size_t rows = d == 128 ? Geo<128>::ROWS : Geo<256>::ROWS;
    Layout l;
    l.req = 0;
    l.merge = up(l.req + sizeof(Request) * (size_t)B);
    l.ml = up(l.merge + sizeof(Merge) * kMaxBlocks);
    l.o = up(l.ml + sizeof(float2) * 2 * kMaxBlocks * rows);
    l.list = up(l.o + sizeof(float) * 2 * kMaxBlocks * rows * d);
    l.bytes = up(l.list + sizeof(int2) * (size_t)B * max_pages);
    return l;
}

template <int D, int FMT>
static int32_t launch(const Params& P, int device, int sms, cudaStream_t s)
{
    using G = Geo<D>;
    // once per device: the kernel's shared memory, and a check that the warps' shares of the registers add up to the launch's (a
    // build that takes fewer would wait for the rest for ever; build.py refuses it first)
    static std::mutex mu;
    static unsigned long long ready = 0;                         // a bit per device
    {
        std::lock_guard<std::mutex> lk(mu);
        if (device < 0 || device >= 64) {
            set_last_error("chunk attention: device index beyond the 64 this library keeps launch state for");
            return MKV_E_INVALID;
        }
        if (!(ready >> device & 1)) {
            cudaFuncAttributes attr;
            MKV_CUDA(cudaFuncGetAttributes(&attr, chunk_scan_kernel<D, FMT>));
            if (attr.numRegs != G::REGS) {
                set_last_error("chunk attention: the kernel was built with another number of registers than its warps share out");
                return MKV_E_CUDA;
            }
            MKV_CUDA(cudaFuncSetAttribute(chunk_scan_kernel<D, FMT>, cudaFuncAttributeMaxDynamicSharedMemorySize, G::SMEM));
            ready |= 1ull << device;
        }
    }
    if ((unsigned long long)P.hkv * fp8_page_bytes(D, P.tiles) >> 32) {
        set_last_error("chunk attention: a page of all KV heads has 4 GB or more");
        return MKV_E_INVALID;
    }
    const int blocks = sms < kMaxBlocks ? sms : kMaxBlocks;
    MKV_CUDA(launch_pdl(chunk_plan_kernel<G::ROWS>, dim3(P.B), kPlanThreads, 0, 1, s, P));
    MKV_CUDA(launch_pdl(chunk_scan_kernel<D, FMT>, dim3(blocks), G::THREADS, G::SMEM, 1, s, P));
    MKV_CUDA(launch_pdl(chunk_merge_kernel<D, G::ROWS>, dim3(blocks, G::ROWS / 8), 256, 0, 1, s, P));
    MKV_CUDA(cudaGetLastError());
    return MKV_OK;
}

}  // namespace chunk

size_t chunk_ws_bytes(int d, int B, int max_pages) { return chunk::layout_of(d, B, max_pages).bytes; }

int32_t launch_chunk_attention(mkv_pool* p, const void* q, int64_t q_stride, int n_rows, const int32_t* starts, const int32_t* bt,
                               const uint8_t* tags, const int32_t* lens, int B, int max_pages, float scale, void* out, float* lse,
                               void* ws, cudaStream_t s)
{
    using namespace chunk;
    Params P = {};
    P.fp8 = p->fp8; P.tq3 = p->tq3;
    P.fp8_pages = p->cfg.fp8_pages; P.tq3_pages = p->cfg.tq3_pages;
    P.hkv = p->hkv; P.group = p->group; P.tiles = p->tiles;
    P.sigma = p->sigma;
    P.sc2 = (scale < 0.f ? -scale : scale) * kLog2e;
    P.negative = scale < 0.f;
    P.k_scale = p->cfg.k_scale; P.v_scale = p->cfg.v_scale;
    // Demote writes numbers of at most 448 times the pool's scales: units of their size keep fp16 from overflow
    auto unit = [](float x) {
        int e;
        frexpf(x, &e);
        return e - 1 < -14 ? -14 : e - 1 > 14 ? 14 : e - 1;
    };
    P.ke = unit(P.k_scale); P.ve = unit(P.v_scale);
    P.q = static_cast<const __nv_bfloat16*>(q);
    P.q_stride = q_stride;
    P.n_rows = n_rows;
    P.starts = starts; P.bt = bt; P.lens = lens; P.tags = tags;
    P.B = B; P.max_pages = max_pages;
    P.out = static_cast<__nv_bfloat16*>(out);
    P.lse = lse;
    const Layout l = layout_of(p->d, B, max_pages);
    uint8_t* w = static_cast<uint8_t*>(ws);
    P.req = reinterpret_cast<Request*>(w + l.req);
    P.merge = reinterpret_cast<Merge*>(w + l.merge);
    P.part_ml = reinterpret_cast<float2*>(w + l.ml);
    P.part_o = reinterpret_cast<float*>(w + l.o);
    P.list = reinterpret_cast<int2*>(w + l.list);
    P.status = p->status_dev;
    P.wait_ns = p->wait_ns;
    const int sms = p->dev.sm_count;
    if (p->d == 128) return p->fmt == 2 ? launch<128, 2>(P, p->device, sms, s) : launch<128, 1>(P, p->device, sms, s);
    return p->fmt == 2 ? launch<256, 2>(P, p->device, sms, s) : launch<256, 1>(P, p->device, sms, s);
}

}  // namespace mkv
