// Attention of one decode step over the cache, and over shared prefixes.
//
// Mathematics.  With logits x_n = scale * q . k_n a set N of rows is summarised by
//       m = a bound near max x_n (base-2 exponents),  l = sum 2^(x_n - m),  o = sum 2^(x_n - m) v_n,
// and two summaries merge by bringing both to the larger m and adding.  out = o / l, so the rows of a unit may be cut
// anywhere: over the warps of a block, over blocks, over a prefix and a sequence's own rows.
//
// What bounds it.  2 x 128 cached values are read for 4 * 128 * G flops: the kernel is bound by HBM.  Every cached row is
// read once, with 16-byte asynchronous copies into a ring of two 8 KB stages that each warp keeps for itself; the copies run
// one step ahead, across the units of a block's share.  128 KB in flight per multiprocessor measured best: 192 KB cost 5 %.
//
// Work split.  All units of a call (sequence x KV head [x tile of query rows]) are laid end to end on a line, each as many
// steps long as it has tiles of rows plus a fixed number that stands for its own cost (queries, joining, output), and
// every block takes an equal share of that line, which begins and ends anywhere inside a unit.  (Shares per warp instead
// of per block measured 10 % slower on long units: 1,184 streams of 4 KB against 296 of 16 KB, and four times the parts.)
// A unit that lies in one share is finished there; the parts of the others go to the workspace, one slot for a block's
// first unit and one for its last, and k_attend_merge joins them in a fixed order.  The lengths are on the device only,
// so every block finds its share by a sum over them.
#pragma once
#include <cuda_bf16.h>

#include "tri_score_tma.cuh"
#include "tri_step.cuh"

namespace tri {

constexpr int kAttWarps = 4, kAttThreads = 32 * kAttWarps, kAttBlocksPerSM = 2;
constexpr int kAttStages = 2, kAttStageBytes = 8192;             // K and V of 16 bf16 or 32 e4m3 rows (three stages: 5 % slower)
constexpr int kAttRingBytes = kAttWarps * kAttStages * kAttStageBytes;
template <bool KEY8> constexpr int kAttRows = KEY8 ? 32 : 16;    // rows of a warp's step; a tile is one step of all warps
constexpr int kAttUnitCost = 2;                                  // a unit's own cost, in tiles
// Few units with room for few rows go to clusters of 8 blocks, one unit each, in one launch: for one sequence of 8 heads
// 5.2 against 7.9 us at 600 rows, 6.9 against 9.0 at 2,176, equal at 4,352, 13.4 against 11.4 at 8,192, where cutting the
// unit over the whole GPU wins.  (The lengths are on the device: the rule goes by the view's capacity.)
constexpr int kAttCluster = 8, kAttClusterRows = 4352;
constexpr int kAttRowPitch = kHeadDim + 4;                       // floats per row of a part: 128 sums, m, l, two unused
// A weight is 2^(x - m).  The bound m is raised, to kAttBelow under the largest logit, when one passes it by kAttAbove.  As
// bf16 a weight has the range of fp32.  An f16 ends at 2^16 and 2^-24, and a million rows each 2^-26 of the largest are mass:
// the largest weight is kept in [2^11, 2^15], so that what falls below the format is 2^-36 of it.
template <bool F16> constexpr float kAttAbove = F16 ? 15.0f : 8.0f;
template <bool F16> constexpr float kAttBelow = F16 ? 11.0f : 0.0f;

struct AttendParams {
    View src;
    int32_t layer, nseq, H, G;                            // nseq: sequences (or prefixes) of src
    int32_t spt;                                          // prefixes: sequences per tile of query rows; own rows: 0
    int32_t S;                                            // sequences of the call
    int32_t box_rows;                                     // k_attend_prefix: rows per copied box
    int32_t under;                                        // launched behind a pass over prefixes
    const int32_t *unit_lens;                             // [nseq][H] of this layer or NULL
    const float *k_scale, *v_scale;                       // [H] of this layer or NULL
    const int32_t *group_start;                           // [nseq + 1], prefixes only
    const char *q;
    int64_t q_seq, q_head;
    char *out;
    int64_t out_seq, out_head;
    float *lse;
    float scale;                                          // times log2 e
    int32_t finish;                                       // units that lie in one block are written to out
    float *slots;                                         // [blocks][2][rows][kAttRowPitch] parts of cut units
    float *whole;                                         // [S][H][G][kAttRowPitch] summaries of uncut units (finish == 0)
    int2 *rec;                                            // per unit: slot of its first part, number of parts
    int32_t *device_status;
};

__device__ __forceinline__ int att_len(const AttendParams &p, int seq, int h)
{
    const int n = ld_here(p.unit_lens ? p.unit_lens + (int64_t)seq * p.H + h : p.src.seq_lens + seq);
    return min(max(n, 0), p.src.n_max);
}
// Sequences [first, first + count) of a group.  (STRONG: before the kernel has waited, see ld_relaxed.)
template <bool STRONG = false>
__device__ __forceinline__ int2 att_group(const int32_t *start, int S, int g)
{
    const int a0 = STRONG ? ld_relaxed(start + g) : ld_here(start + g), b0 = STRONG ? ld_relaxed(start + g + 1) : ld_here(start + g + 1);
    const int a = min(max(a0, 0), S), b = min(max(b0, 0), S);
    return make_int2(a, max(b - a, 0));
}
// Whether a group ends before it begins.  Boundaries outside [0, S] count as the nearest bound here, too: a group that descends
// out there only is an empty one.
__device__ __forceinline__ bool att_descends(const int32_t *start, int S, int g)
{
    return min(max(start[g], 0), S) > min(max(start[g + 1], 0), S);
}
// r / d for r < 256, 0 < d <= 16, with inv = 65536 / d + 1: the product's error r * d / 65536 never reaches the next integer.
__device__ __forceinline__ int att_small_div(int r, int inv) { return (r * inv) >> 16; }
__device__ __forceinline__ int att_row_tiles(const AttendParams &p, int seq)
{
    if (p.spt == 0) return 1;
    return (att_group(p.group_start, p.S, seq).y + p.spt - 1) / p.spt;
}
// The last group that starts at or before a sequence (0 if none does); the warp's lanes look at 32 starts at a time.
template <bool STRONG = false>
__device__ __forceinline__ int att_group_of(const int32_t *start, int groups, int seq, int lane)
{
    int g = -1;
    for (int b = 0; b < groups; b += 32) {
        const int32_t *at = start + min(b + lane, groups - 1);
        g += __popc(__ballot_sync(0xffffffffu, b + lane < groups && (STRONG ? ld_relaxed(at) : ld_here(at)) <= seq));
    }
    return max(g, 0);
}
// Index of tile `rt` of group g in units before the head is added: the tiles of ascending groups never collide, and no
// index reaches P + S / spt + 1 whatever group_start holds.
__device__ __forceinline__ int att_tile_index(int g, int first, int spt, int rt) { return g + first / spt + rt; }

// 16 bytes (or zeros, bytes = 0) with an L2 policy.
__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, uint32_t bytes, uint64_t policy)
{
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2, %3;\n" ::"r"(dst), "l"(src), "r"(bytes), "l"(policy) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;\n" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;\n" ::"n"(N) : "memory"); }
__device__ __forceinline__ void ldmatrix_x4_t(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];\n"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void mma_bf16_16816_acc(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                                   uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <bool F16>
__device__ __forceinline__ void mma16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    if (F16) mma_f16_16816(d, a0, a1, a2, a3, b0, b1);
    else mma_bf16_16816_acc(d, a0, a1, a2, a3, b0, b1);
}
// (lower, upper) as a 16-bit pair, and what the rounding left over as a second pair.
template <bool F16>
__device__ __forceinline__ void split16(float lower, float upper, uint32_t &hi, uint32_t &lo)
{
    if (F16) {
        asm("cvt.rn.f16x2.f32 %0, %1, %2;\n" : "=r"(hi) : "f"(upper), "f"(lower));
        const float rl = lower - f16_value(hi & 0xffffu), ru = upper - f16_value(hi >> 16);
        asm("cvt.rn.f16x2.f32 %0, %1, %2;\n" : "=r"(lo) : "f"(ru), "f"(rl));
    } else {
        hi = cvt_bf16x2(upper, lower);
        lo = cvt_bf16x2(upper - bf16_hi(hi), lower - bf16_lo(hi));
    }
}
// An 8 x 8 matrix of 16-bit values held as a fragment (row lane / 4, columns 2 (lane % 4), + 1), transposed.
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x)
{
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
    return y;
}

// The share of one block: where it begins on the line and which unit lies there.  (The host refuses calls whose line
// could pass 2^31 steps.)
struct AttShare {
    int total, t0, t1;                // steps of the call; this block's [t0, t1)
    int each, longer;                 // steps per share; the first `longer` shares have one more
    int shares;                       // blocks that get steps
    int seq, h, start;                // the unit at t0 and its first step (all of its row tiles)
};
// Where a block stands on the line, and what it finds there: tiles [ka, kb) of one unit and tile of query rows.
struct AttCursor { int seq, h, rt, start; };
struct AttJob {
    int seq, h, len, kt, ka, kb;      // tiles [ka, kb) of the unit's kt
    int first_seq, nrows;             // query rows: G of each sequence from first_seq on (prefixes), or of seq
    int rec;                          // index of the unit's record
    int rows0;                        // step of the unit's first tile
    bool begins, complete;            // the unit's first step is here (its part goes to the last slot); all tiles are here
    bool of_prefix;                   // in a cluster: rows of the sequence's prefix, not its own
};

// The share of this block.  Where the heads of a sequence have equal lengths the sums run over sequences only.  Groups that
// descend, and so overlap, could make the line longer than the host has checked: no block gets a share then.
template <int TILE, int COST>
__device__ __forceinline__ AttShare att_share(const AttendParams &p)
{
    __shared__ int part_s[32], found_s[3];
    const int tid = threadIdx.x, nth = blockDim.x, lane = tid & 31, warp = tid >> 5;
    const bool by_head = p.unit_lens != nullptr;
    const int n = by_head ? p.nseq * p.H : p.nseq, heads = by_head ? 1 : p.H;
    const int per = n <= nth ? 1 : (n + nth - 1) / nth;
    const int a = min(tid * per, n), b = min(a + per, n);
    // steps of entry x, one head.  Where the pass does not wait for its predecessor the thread's first length is acquired; with
    // the barrier below every other load of the block follows thread 0's.
    auto cost = [&](int x) -> int {
        const int32_t *at = (by_head ? p.unit_lens : p.src.seq_lens) + x;
        const int len = p.under && x == a ? ld_acquire(at) : ld_here(at);
        const int kt = (int)(((uint32_t)min(max(len, 0), p.src.n_max) + TILE - 1) / TILE);
        return (kt + COST) * (p.spt ? att_row_tiles(p, by_head ? x / p.H : x) : 1);
    };
    int sum = 0, c0 = 0, descends = 0;
    for (int x = a; x < b; ++x) {
        c0 = cost(x);
        sum += c0 * heads;
        if (p.spt) {
            const int g = by_head ? x / p.H : x;
            descends |= att_descends(p.group_start, p.S, g);
        }
    }
    int incl = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += o;
    }
    if (lane == 31) part_s[warp] = incl;
    descends = __syncthreads_or(descends);
    int before = 0, total = 0;
    for (int w = 0; w < nth / 32; ++w) {
        if (w < warp) before += part_s[w];
        total += part_s[w];
    }
    if (descends) total = 0;
    AttShare r;
    r.total = total;
    r.shares = min(max(total, 1), (int)gridDim.x);
    r.each = (int)((uint32_t)total / (uint32_t)r.shares);
    r.longer = total - r.each * r.shares;
    const int worker = (int)blockIdx.x;
    const bool have = worker < r.shares && total > 0;
    r.t0 = have ? worker * r.each + min(worker, r.longer) : total;
    r.t1 = have ? r.t0 + r.each + (worker < r.longer ? 1 : 0) : total;
    int at = before + incl - sum;                         // this thread's entries: steps [at, at + sum)
    if (r.t0 >= at && r.t0 < at + sum) {
        for (int x = a; x < b; ++x) {
            const int c = per == 1 ? c0 : cost(x);
            if (r.t0 < at + c * heads) {
                const int skip = by_head ? 0 : (int)((uint32_t)(r.t0 - at) / (uint32_t)c);
                found_s[0] = by_head ? x / p.H : x;
                found_s[1] = by_head ? x % p.H : skip;
                found_s[2] = at + skip * c;
                break;
            }
            at += c * heads;
        }
    }
    __syncthreads();
    r.seq = have ? found_s[0] : p.nseq;
    r.h = have ? found_s[1] : 0;
    r.start = have ? found_s[2] : total;
    return r;
}

// Which block holds step t of the line.
__device__ __forceinline__ int att_block_of(const AttShare &r, int t)
{
    const int split = r.longer * (r.each + 1);
    return t < split ? (int)((uint32_t)t / (uint32_t)(r.each + 1)) : r.longer + (int)((uint32_t)(t - split) / (uint32_t)r.each);
}

// The record of a unit, made by the block that holds its first step: slot of its first part, number of parts.
__device__ __forceinline__ int2 att_record(const AttShare &sh, const AttJob &j)
{
    if (j.kt == 0) return make_int2(0, 0);
    const int here = (int)blockIdx.x;
    if (j.complete) return make_int2(2 * here, 1);
    const int first = j.rows0 < sh.t1 ? here : att_block_of(sh, j.rows0);
    return make_int2(2 * first + (first == here ? 1 : 0), att_block_of(sh, j.rows0 + j.kt - 1) - first + 1);
}

// The next unit of a share; false at its end.  Units without rows come too, and units of which the share holds only the
// steps that stand for their own cost (kb <= ka).
template <int TILE, int COST>
__device__ __forceinline__ bool att_next(const AttendParams &p, const AttShare &sh, AttCursor &c, AttJob &j)
{
    while (c.start < sh.t1 && c.seq < p.nseq) {
        j.seq = c.seq; j.h = c.h;
        j.len = att_len(p, j.seq, j.h);
        j.kt = (int)(((uint32_t)j.len + TILE - 1) / TILE);
        const int c1 = j.kt + COST, rt = c.rt;
        int2 grp = make_int2(j.seq, 1);
        int rts = 1;
        if (p.spt) { grp = att_group(p.group_start, p.S, j.seq); rts = (grp.y + p.spt - 1) / p.spt; }
        const int js = c.start, rows0 = js + COST, je = js + c1;             // the steps of this tile of query rows
        if (rt < rts) c.start += c1;
        if (++c.rt >= rts) {
            c.rt = 0;
            if (++c.h == p.H) { c.h = 0; ++c.seq; }
        }
        if (rt >= rts || je <= sh.t0) continue;
        j.first_seq = grp.x + rt * p.spt;
        j.nrows = p.spt ? min(p.spt, grp.y - rt * p.spt) * p.G : p.G;
        j.rec = p.spt ? att_tile_index(j.seq, grp.x, p.spt, rt) * p.H + j.h : j.seq * p.H + j.h;
        j.ka = max(sh.t0 - rows0, 0);
        j.kb = min(max(sh.t1 - rows0, 0), j.kt);
        j.begins = js >= sh.t0;
        j.complete = j.ka == 0 && j.kb == j.kt;
        j.rows0 = rows0;
        return true;
    }
    return false;
}

// KEY8: e4m3 rows, widened exactly to f16 (the queries are brought to f16 by a power of two per row).
// RT = 8: at most 8 query rows.  bf16: they are rows of A; the rest of the rounded weights rides in the upper 8 rows of the
// 16-row MMA, for free.  e4m3, where widening leaves less room for waiting: the products are formed transposed (TR), keys and
// dimensions as the 16 rows of A, the query rows as the 8 columns.  Logits then take half the MMAs, the sums half the
// registers, and the rest of the weights a second MMA: 64 x 8 units of 0..4K rows 63.4 us against 67.9.  (16-row steps at
// 4 blocks per multiprocessor 65.2, 32-row steps at 3 blocks 63.1; the copies alone 58.)
// RT = 16: up to 16 query rows are rows of A; the rest of the weights takes a second MMA.
// CL > 0: a cluster of CL blocks takes one unit, cuts it evenly, and joins its parts through distributed shared memory: one
// launch and no workspace where there are few short units.  `pre` (pre.nseq > 0): the prefixes; a unit is then the rows of
// its sequence's prefix, if it has one, and its own.
template <bool KEY8, int RT, int CL>
__device__ __forceinline__ void attend_block(const AttendParams &p, const AttendParams &pre)
{
    constexpr bool TR = KEY8 && RT == 8;
    constexpr int ST = kAttStages, ROWS = kAttRows<KEY8>, NK = ROWS / 16, TILE = kAttWarps * ROWS;
    constexpr int kRowBytes = KEY8 ? 128 : 256, kHalf = ROWS * kRowBytes;                             // K | V
    constexpr int kChunks = kRowBytes / 16, kCopies = ROWS * kChunks / 32;
    constexpr int NR = TR ? 2 : RT / 8;                   // query rows per thread
    extern __shared__ __align__(128) uint8_t dyn[];
    __shared__ float2 stat[kAttWarps][RT];
    __shared__ __align__(16) float part[CL ? RT : 1][kAttRowPitch];      // this block's sums, and (m, l)

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g8 = lane >> 2, t4 = lane & 3;
    const uint32_t ring = smem_u32(dyn) + warp * (ST * kAttStageBytes);
    // 16-byte chunk c of row r lies at chunk c ^ (r & 7) of its 128 bytes; as stages are multiples of 128 bytes, the chunk's
    // number can be xor-ed into a lane's address.  Matrices of one load: keys as (8 keys, 2 chunks), values as (16 keys, 2 chunks)
    const int krow = KEY8 ? (lane & 15) : (lane & 7) + ((lane & 16) >> 1), vrow = lane & 15;
    const uint32_t klane = krow * kRowBytes + ((((KEY8 ? lane >> 4 : (lane >> 3) & 1) ^ krow) & 7) << 4);
    const uint32_t vlane = vrow * kRowBytes + ((((lane >> 4) ^ vrow) & 7) << 4);
    // Set up under the kernel before it in the stream and waits for it here, except behind a pass over prefixes, whose blocks
    // this pass's may follow one by one: that pass is waited for at the end, and att_share's first load orders the others.
    if (!p.under) grid_dependency_wait();
    grid_dependents_launch();
    auto params_of = [&](const AttJob &u) -> const AttendParams & {
        if constexpr (CL == 0) return p;
        else return u.of_prefix ? pre : p;
    };
    AttShare sh = {};
    int rank = 0, group = -1;                             // in a cluster: this block's number, the sequence's prefix
    if constexpr (CL == 0) {
        sh = att_share<TILE, kAttUnitCost>(p);
        if ((int)blockIdx.x >= sh.shares) return;
    } else {
        asm volatile("mov.u32 %0, %%cluster_ctarank;\n" : "=r"(rank));
        sh.seq = (int)blockIdx.x / CL / p.H; sh.h = (int)blockIdx.x / CL - sh.seq * p.H;
        if (tid < RT) { part[CL ? tid : 0][kHeadDim] = -INFINITY; part[CL ? tid : 0][kHeadDim + 1] = 0.f; }      // no rows so far
        if (pre.nseq > 0) {
            group = att_group_of(pre.group_start, pre.nseq, sh.seq, lane);
            const int2 g = att_group(pre.group_start, pre.S, group);
            if (sh.seq < g.x || sh.seq >= g.x + g.y) group = -1;
            if (blockIdx.x == 0 && p.device_status)
                for (int i = tid; i < pre.nseq; i += kAttThreads)
                    if (att_descends(pre.group_start, pre.S, i)) atomicExch(p.device_status, (int)TRI_ERR_DEVICE_CHECK);
        }
    }
    auto next_unit = [&](AttCursor &c, AttJob &u) -> bool {
        if constexpr (CL == 0) {
            return att_next<TILE, kAttUnitCost>(p, sh, c, u);
        } else {
            if (c.rt == 0 && group < 0) c.rt = 1;
            if (c.rt > 1) return false;
            u.of_prefix = c.rt++ == 0;
            u.seq = u.of_prefix ? group : c.seq; u.h = c.h; u.nrows = p.G; u.first_seq = c.seq;
            u.len = att_len(params_of(u), u.seq, c.h);
            u.kt = (int)(((uint32_t)u.len + TILE - 1) / TILE);
            u.ka = rank * u.kt / CL; u.kb = (rank + 1) * u.kt / CL;
            u.begins = u.complete = false;
            return true;
        }
    };

    // ---------------- copies: a cursor of their own, ST - 1 steps ahead ----------------
    AttCursor pc = {sh.seq, sh.h, 0, sh.start};
    AttJob pj = {};
    int pit = 0, pstage = 0, page[NK], slot[NK];          // next step; page and first slot of its 16-row halves
    uint32_t bad = 0;                                     // bits 2 i, 2 i + 1: these 16 rows of stage i are absent
    bool more = true;
    int64_t unit_base = 0;                                // first row of the unit; of page 0, where rows are paged
    // own rows are read once in a step: first to leave L2 (3 % faster on long batches); a prefix's tiles of query rows share them
    uint64_t policy;
    if (p.spt) asm("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;\n" : "=l"(policy));
    else asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;\n" : "=l"(policy));
    int64_t step_row = 0;                                 // elements between rows
    auto advance = [&]() {                                // to the next step, its pages looked up before they are needed
        if (pit == pj.kb) {
            do more = next_unit(pc, pj); while (more && pj.kb <= pj.ka);
            pit = pj.ka;
            const AttendParams &a = params_of(pj);
            step_row = a.src.paged ? a.src.stride_slot : a.src.stride_tok;
            unit_base = (int64_t)a.layer * a.src.stride_layer + (int64_t)pj.h * a.src.stride_head +
                        (a.src.paged ? 0 : (int64_t)pj.seq * a.src.stride_seq);
        }
        const AttendParams &a = params_of(pj);
        if (more && a.src.paged) {
#pragma unroll
            for (int half = 0; half < NK; ++half) {
                const uint32_t r = (uint32_t)pit * TILE + warp * ROWS + 16 * half;
                const uint32_t pg = a.src.page_shift >= 0 ? r >> a.src.page_shift : r / (uint32_t)a.src.page_size;
                page[half] = r < (uint32_t)pj.len ? ld_here(a.src.page_table + (int64_t)pj.seq * a.src.max_pages_per_seq + pg) : 0;
                slot[half] = (int)(r - pg * (uint32_t)a.src.page_size);
            }
        }
    };
    auto issue = [&]() {
        if (more) {
            const View &src = params_of(pj).src;
            const uint32_t dst = ring + pstage * kAttStageBytes;
            constexpr int es = KEY8 ? 1 : 2;
            const int c = lane % kChunks, r0 = lane / kChunks;
            uint32_t miss = 0;
#pragma unroll
            for (int half = 0; half < NK; ++half) {       // 16 rows each: they lie in one page
                const uint32_t r = (uint32_t)pit * TILE + warp * ROWS + 16 * half;
                int have = r < (uint32_t)pj.len ? min(pj.len - (int)r, 16) : 0;
                int64_t base = unit_base;
                if (src.paged) {
                    base += (int64_t)page[half] * src.stride_page + (int64_t)slot[half] * step_row;
                    if (have && src.n_pages > 0 && (uint32_t)page[half] >= (uint32_t)src.n_pages) {
                        have = 0;
                        miss |= 1u << half;
                        if (lane == 0 && p.device_status) atomicExch(p.device_status, (int)TRI_ERR_DEVICE_CHECK);
                    }
                } else {
                    base += (int64_t)r * step_row;
                }
                int64_t from = (base + r0 * step_row) * es + 16 * c;
                const uint32_t to = dst + (16 * half + r0) * kRowBytes;
                constexpr int kRowsAtOnce = 32 / kChunks;
                if (have == 16) {
#pragma unroll
                    for (int i = 0; i < kCopies / NK; ++i) {
                        const uint32_t off = i * kRowsAtOnce * kRowBytes + (((c & 8) | ((c ^ (i * kRowsAtOnce + r0)) & 7)) << 4);
                        cp_async16(to + off, src.k + from, 16u, policy);
                        cp_async16(to + kHalf + off, src.v + from, 16u, policy);
                        from += kRowsAtOnce * step_row * es;
                    }
                } else {
                    // rows behind the length (or absent ones) arrive as zeros and are not read
#pragma unroll 1
                    for (int i = 0; i < kCopies / NK; ++i) {
                        const int rr = i * kRowsAtOnce + r0;
                        const bool there = rr < have;
                        const int64_t at = there ? from : 16 * c;
                        const uint32_t off = i * kRowsAtOnce * kRowBytes + (((c & 8) | ((c ^ rr) & 7)) << 4);
                        cp_async16(to + off, src.k + at, there ? 16u : 0u, policy);
                        cp_async16(to + kHalf + off, src.v + at, there ? 16u : 0u, policy);
                        from += kRowsAtOnce * step_row * es;
                    }
                }
            }
            bad = (bad & ~(3u << (2 * pstage))) | (miss << (2 * pstage));
            ++pit;
            advance();
        }
        pstage = pstage + 1 == ST ? 0 : pstage + 1;
        cp_commit();
    };
    advance();

    AttCursor cur = {sh.seq, sh.h, 0, sh.start};
    AttJob j = {};
    uint32_t qa[8][4];
    const int inv_g = 65536 / p.G + 1;
    float mul[NR], k_scale = 1.f;                         // logit in base-2 units per accumulator unit
    float o[TR ? 8 : 16][4], m[NR], l[NR];
    int it = 0, stage = 0, ahead = ST - 1;
    for (;;) {
        // the stage of the step before: read, or used and released in joining a unit
        issue();
        if (ahead > 0) { --ahead; continue; }
        if (it == j.kb) {
            // ---------------- the next unit ----------------
            bool rows = false;
            while (!rows && next_unit(cur, j)) {
                if (j.begins && tid == 0) p.rec[j.rec] = att_record(sh, j);
                rows = j.kb > j.ka;
                if (j.kt == 0 && j.begins && p.finish)    // no rows: zeros
                    for (int i = tid; i < p.G * 16; i += kAttThreads) {
                        const int hq = j.h * p.G + (i >> 4);
                        *reinterpret_cast<uint4 *>(p.out + ((int64_t)j.seq * p.out_seq + (int64_t)hq * p.out_head) * 2 + 16 * (i & 15)) =
                            make_uint4(0u, 0u, 0u, 0u);
                        if (p.lse && (i & 15) == 0) p.lse[(int64_t)j.seq * p.H * p.G + hq] = -INFINITY;
                    }
            }
            if (!rows) break;
            it = j.ka;
            // ---------------- query rows as the A operand ----------------
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = g8 + 8 * i;
                const bool have = r < j.nrows && (RT == 16 || i == 0);
                const char *qr = nullptr;
                if (have) {
                    const int sr = p.spt ? att_small_div(r, inv_g) : 0, sq = j.first_seq + sr, gg = r - sr * p.G;
                    qr = p.q + ((int64_t)sq * p.q_seq + (int64_t)(j.h * p.G + gg) * p.q_head) * 2;
                }
                float amax = 0.f;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    // slots 2 t4, 2 t4 + 1 and 2 t4 + 8, + 9 of step k: dims 16 k + slot, for 8-bit keys dims 16 k + 4 t4 + 0..3
                    const int d0 = 16 * k + (KEY8 ? 4 * t4 : 2 * t4), d1 = KEY8 ? d0 + 2 : d0 + 8;
                    qa[k][i] = have ? *reinterpret_cast<const uint32_t *>(qr + 2 * d0) : 0u;
                    qa[k][i + 2] = have ? *reinterpret_cast<const uint32_t *>(qr + 2 * d1) : 0u;
                    if (KEY8) {
                        amax = fmaxf(amax, fmaxf(fmaxf(fabsf(bf16_lo(qa[k][i])), fabsf(bf16_hi(qa[k][i]))),
                                                 fmaxf(fabsf(bf16_lo(qa[k][i + 2])), fabsf(bf16_hi(qa[k][i + 2])))));
                    }
                }
                float back = 1.f;
                if (KEY8) {
                    // f16 holds 11 bits down to 2^-14: with the row's largest entry brought to [1, 2) a bf16 entry is exact
                    // unless it is 2^14 times smaller than that one
                    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
                    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
                    int e = (int)((__float_as_uint(amax) >> 23) & 255u) - 127;
                    e = min(max(e, -126), 126);
                    if (amax == 0.f) e = 0;
                    const float by = __uint_as_float((uint32_t)(127 - e) << 23);
                    back = __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
                    for (int k = 0; k < 8; ++k)
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const uint32_t w = qa[k][i + 2 * x];
                            qa[k][i + 2 * x] = f16_bits(bf16_lo(w) * by) | (f16_bits(bf16_hi(w) * by) << 16);
                        }
                }
                if (TR) {
                    if (i == 0)
#pragma unroll
                        for (int x = 0; x < NR; ++x) mul[x] = p.scale * __shfl_sync(0xffffffffu, back, (2 * t4 + x) * 4);
                } else if (i < NR) {
                    mul[i % NR] = p.scale * back;
                }
            }
#pragma unroll
            for (int i = 0; i < (TR ? 8 : 16); ++i) { o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f; }
#pragma unroll
            for (int i = 0; i < NR; ++i) { m[i] = -INFINITY; l[i] = 0.f; }
            k_scale = params_of(j).k_scale ? params_of(j).k_scale[j.h] : 1.f;
#pragma unroll
            for (int i = 0; i < NR; ++i) mul[i] *= k_scale;
        }

        // ---------------- one step ----------------
        cp_wait<ST - 1>();
        __syncwarp();
        const uint32_t r0 = (uint32_t)it * TILE + warp * ROWS;
        const int have = r0 < (uint32_t)j.len ? min(j.len - (int)r0, ROWS) : 0;
        const uint32_t miss = (bad >> (2 * stage)) & 3u;
        const bool cut = have < ROWS || miss;
        const uint32_t kb_s = ring + stage * kAttStageBytes, vb_s = kb_s + kHalf;
        if constexpr (TR) {
            // logits transposed: 16 keys x 8 query rows per accumulator (x 2: even and odd steps of 16 dims, shorter chains); the
            // thread holds keys g8, g8 + 8 of query rows 2 t4, 2 t4 + 1
            float w[NK][4];
#pragma unroll
            for (int kg = 0; kg < NK; ++kg) {
                float odd[4] = {0.f, 0.f, 0.f, 0.f};
                w[kg][0] = w[kg][1] = w[kg][2] = w[kg][3] = 0.f;
#pragma unroll
                for (int k = 0; k < 8; k += 2) {
                    uint32_t f[4], a[8];
                    ldmatrix_x4(f, (kb_s + klane + 16 * kg * 128) ^ (k << 4));
#pragma unroll
                    for (int x = 0; x < 4; ++x) e4m3x4_to_f16x2(f[x], a[2 * x], a[2 * x + 1]);
                    mma16<true>(w[kg], a[0], a[2], a[1], a[3], qa[k][0], qa[k][2]);
                    mma16<true>(odd, a[4], a[6], a[5], a[7], qa[k + 1][0], qa[k + 1][2]);
                }
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    w[kg][x] = (w[kg][x] + odd[x]) * mul[x & 1];
                    if (cut && (16 * kg + g8 + 8 * (x >> 1) >= have || ((miss >> kg) & 1u))) w[kg][x] = -INFINITY;
                }
            }
            // the bound is looked at by a vote and searched for only when it has to be raised
            float mx[NR];
            bool raise = false;
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                mx[i] = fmaxf(w[0][i], w[0][i + 2]);
#pragma unroll
                for (int kg = 1; kg < NK; ++kg) mx[i] = fmaxf(mx[i], fmaxf(w[kg][i], w[kg][i + 2]));
                raise = raise || mx[i] > m[i] + kAttAbove<KEY8>;
            }
            if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
                for (int i = 0; i < NR; ++i) {
                    mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 4));
                    mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 8));
                    mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 16));
                    if (mx[i] > m[i] + kAttAbove<KEY8>) {
                        mx[i] -= kAttBelow<KEY8>;
                        const float by = ex2(m[i] - mx[i]);          // 0 where there was no bound yet
                        m[i] = mx[i];
                        l[i] *= by;
#pragma unroll
                        for (int n = 0; n < 8; ++n) { o[n][i] *= by; o[n][i + 2] *= by; }
                    }
                }
            }
            // weights, and transposed into the B operand: 16 keys x 8 query rows
            uint32_t ph[NK][2], pl[NK][2];
#pragma unroll
            for (int kg = 0; kg < NK; ++kg) {
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    w[kg][x] = ex2(w[kg][x] - (m[x & 1] == -INFINITY ? 0.f : m[x & 1]));
                    l[x & 1] += w[kg][x];
                }
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    split16<true>(w[kg][2 * x], w[kg][2 * x + 1], ph[kg][x], pl[kg][x]);
                    ph[kg][x] = transpose8x8(ph[kg][x]);
                    pl[kg][x] = transpose8x8(pl[kg][x]);
                }
            }
#pragma unroll
            for (int kg = 0; kg < NK; ++kg)
#pragma unroll
                for (int ch = 0; ch < 8; ch += 2) {
                    uint32_t f[4];
                    ldmatrix_x4_t(f, (vb_s + vlane + 16 * kg * 128) ^ (ch << 4));
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        // bytes of a word: key 2 t4 dims (2 g8, 2 g8 + 1), key 2 t4 + 1 the same dims; even dims are rows 0..7
                        uint32_t e0, d0, e1, d1;
                        e4m3x4_to_f16x2(__byte_perm(f[2 * x], 0, 0x3120), e0, d0);
                        e4m3x4_to_f16x2(__byte_perm(f[2 * x + 1], 0, 0x3120), e1, d1);
                        mma16<true>(o[ch + x], e0, d0, e1, d1, ph[kg][0], ph[kg][1]);
                        mma16<true>(o[ch + x], e0, d0, e1, d1, pl[kg][0], pl[kg][1]);
                    }
                }
        } else {
            // logits: 8 rows x 8 keys per accumulator (x 2: even and odd steps of 16 dims apart, shorter chains)
            float sc[2 * NK][4];
            if (KEY8) {
#pragma unroll
                for (int x = 0; x < 2 * NK; ++x) sc[x][0] = sc[x][1] = sc[x][2] = sc[x][3] = 0.f;
#pragma unroll
                for (int k = 0; k < 8; k += 2)
#pragma unroll
                    for (int kg = 0; kg < NK; ++kg) {
                        uint32_t f[4];
                        ldmatrix_x4(f, (kb_s + klane + 16 * kg * 128) ^ (k << 4));
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            uint32_t b0, b1;
                            e4m3x4_to_f16x2(f[x], b0, b1);
                            const int kk = k + (x >> 1);
                            mma16<true>(sc[2 * kg + (x & 1)], qa[kk][0], qa[kk][1], qa[kk][2], qa[kk][3], b0, b1);
                        }
                    }
            } else {
                float sd[2][4];
#pragma unroll
                for (int x = 0; x < 2; ++x) { sc[x][0] = sc[x][1] = sc[x][2] = sc[x][3] = 0.f; sd[x][0] = sd[x][1] = sd[x][2] = sd[x][3] = 0.f; }
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    uint32_t f[4];
                    ldmatrix_x4(f, (kb_s + klane + (k >> 2) * 128) ^ ((2 * k & 7) << 4));
                    mma16<false>(k & 1 ? sd[0] : sc[0], qa[k][0], qa[k][1], qa[k][2], qa[k][3], f[0], f[1]);
                    mma16<false>(k & 1 ? sd[1] : sc[1], qa[k][0], qa[k][1], qa[k][2], qa[k][3], f[2], f[3]);
                }
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int y = 0; y < 4; ++y) sc[x][y] += sd[x][y];
            }
            // running bound and weights; the thread holds keys 8 x + 2 t4, + 1 of row g8 (+ 8)
            float w[NR][4 * NK];
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                float mx = -INFINITY;
#pragma unroll
                for (int x = 0; x < 4 * NK; ++x) {
                    w[i][x] = sc[x >> 1][2 * i + (x & 1)] * mul[i];
                    if (cut) {
                        const int key = 8 * (x >> 1) + 2 * t4 + (x & 1);
                        if (key >= have || ((miss >> (x >> 2)) & 1u)) w[i][x] = -INFINITY;
                    }
                    mx = fmaxf(mx, w[i][x]);
                }
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
                const bool raise = mx > m[i] + kAttAbove<KEY8> || (m[i] == -INFINITY && mx > m[i]);
                if (__any_sync(0xffffffffu, raise)) {
                    mx -= kAttBelow<KEY8>;
                    const float by = raise ? ex2(m[i] - mx) : 1.f;       // 0 where there was no bound yet
                    if (raise) m[i] = mx;
                    l[i] *= by;
#pragma unroll
                    for (int n = 0; n < 16; ++n) {
                        o[n][2 * i] *= by; o[n][2 * i + 1] *= by;
                        if (RT == 8) { o[n][2] *= by; o[n][3] *= by; }
                    }
                }
                const float ref = m[i] == -INFINITY ? 0.f : m[i];
#pragma unroll
                for (int x = 0; x < 4 * NK; ++x) {
                    w[i][x] = ex2(w[i][x] - ref);
                    l[i] += w[i][x];
                }
            }
#pragma unroll
            for (int kg = 0; kg < NK; ++kg) {
                uint32_t ph[NR][2], pl[NR][2];
#pragma unroll
                for (int i = 0; i < NR; ++i) {
                    split16<KEY8>(w[i][4 * kg], w[i][4 * kg + 1], ph[i][0], pl[i][0]);
                    split16<KEY8>(w[i][4 * kg + 2], w[i][4 * kg + 3], ph[i][1], pl[i][1]);
                }
                auto pv = [&](float (&acc)[4], uint32_t b0, uint32_t b1) {
                    if (RT == 8) {
                        mma16<KEY8>(acc, ph[0][0], pl[0][0], ph[0][1], pl[0][1], b0, b1);
                    } else {
                        mma16<KEY8>(acc, ph[0][0], ph[NR - 1][0], ph[0][1], ph[NR - 1][1], b0, b1);
                        mma16<KEY8>(acc, pl[0][0], pl[NR - 1][0], pl[0][1], pl[NR - 1][1], b0, b1);
                    }
                };
                if (KEY8) {
#pragma unroll
                    for (int ch = 0; ch < 8; ch += 2) {
                        uint32_t f[4];
                        ldmatrix_x4_t(f, (vb_s + vlane + 16 * kg * 128) ^ (ch << 4));
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            // bytes of a word: key 2 t4 dims (2 g8, 2 g8 + 1), key 2 t4 + 1 the same dims
                            uint32_t e0, d0, e1, d1;
                            e4m3x4_to_f16x2(__byte_perm(f[2 * x], 0, 0x3120), e0, d0);
                            e4m3x4_to_f16x2(__byte_perm(f[2 * x + 1], 0, 0x3120), e1, d1);
                            pv(o[2 * (ch + x)], e0, e1);
                            pv(o[2 * (ch + x) + 1], d0, d1);
                        }
                    }
                } else {
#pragma unroll
                    for (int n = 0; n < 16; n += 2) {
                        uint32_t f[4];
                        ldmatrix_x4_t(f, (vb_s + vlane + (n >> 3) * 128) ^ ((n & 7) << 4));
                        pv(o[n], f[0], f[1]);
                        pv(o[n + 1], f[2], f[3]);
                    }
                }
            }
        }
        __syncwarp();
        uint8_t *used = dyn + (warp * ST + stage) * kAttStageBytes;
        stage = stage + 1 == ST ? 0 : stage + 1;
        if (++it < j.kb) continue;
        float vs = params_of(j).v_scale ? params_of(j).v_scale[j.h] : 1.f;
        if constexpr (CL > 0) {
            // the prefix's rows are through: the sequence's own go on with the same sums, in units of their own scales
            const float k_before = k_scale, v_before = vs;
            bool own = false;
            while (!own && next_unit(cur, j)) own = j.kb > j.ka;
            if (own) {
                it = j.ka;
                k_scale = params_of(j).k_scale ? params_of(j).k_scale[j.h] : 1.f;
                vs = params_of(j).v_scale ? params_of(j).v_scale[j.h] : 1.f;
                const float k_by = k_scale / k_before, v_by = v_before / vs;
#pragma unroll
                for (int i = 0; i < NR; ++i) mul[i] *= k_by;
#pragma unroll
                for (int n = 0; n < (TR ? 8 : 16); ++n)
#pragma unroll
                    for (int x = 0; x < 4; ++x) o[n][x] *= v_by;
                continue;
            }
        }

        // ---------------- the unit's rows of this share are through: join the warps ----------------
        // each leaves its sums in the stage it has just read, fragment by fragment, and takes a quarter of the dims of all
        if constexpr (TR) {
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                l[i] += __shfl_xor_sync(0xffffffffu, l[i], 4);
                l[i] += __shfl_xor_sync(0xffffffffu, l[i], 8);
                l[i] += __shfl_xor_sync(0xffffffffu, l[i], 16);
                if (g8 == 0) stat[warp][2 * t4 + i] = make_float2(m[i], l[i]);
            }
#pragma unroll
            for (int n = 0; n < 8; ++n) *reinterpret_cast<float4 *>(used + n * 512 + lane * 16) = make_float4(o[n][0], o[n][1], o[n][2], o[n][3]);
        } else {
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
                l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
                if (t4 == 0) stat[warp][g8 + 8 * i] = make_float2(m[i], l[i]);
#pragma unroll
                for (int n = 0; n < 16; n += 2) {
                    float y[4];
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        y[x] = o[n + (x >> 1)][2 * i + (x & 1)] + (RT == 8 ? o[n + (x >> 1)][2 + (x & 1)] : 0.f);
                    *reinterpret_cast<float4 *>(used + (i * 8 + n / 2) * 512 + lane * 16) = make_float4(y[0], y[1], y[2], y[3]);
                }
            }
        }
        __syncthreads();
        const bool final = j.complete && p.finish;
        if constexpr (TR) {
            float4 y[2];                                   // dims 16 n + 2 g8, + 1 of query rows 2 t4, + 1, for n = 2 warp, + 1
            y[0] = y[1] = make_float4(0.f, 0.f, 0.f, 0.f);
            float mm[NR], ll[NR], st[kAttWarps][NR];
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                mm[i] = -INFINITY; ll[i] = 0.f;
#pragma unroll
                for (int w2 = 0; w2 < kAttWarps; ++w2) mm[i] = fmaxf(mm[i], stat[w2][2 * t4 + i].x);
#pragma unroll
                for (int w2 = 0; w2 < kAttWarps; ++w2) {
                    const float2 ml = stat[w2][2 * t4 + i];
                    st[w2][i] = ml.x == -INFINITY ? 0.f : ex2(ml.x - mm[i]);
                    ll[i] += ml.y * st[w2][i];
                }
            }
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int w2 = 0; w2 < kAttWarps; ++w2) {
                    const float4 z = *reinterpret_cast<const float4 *>(used + (w2 - warp) * (ST * kAttStageBytes) + (2 * warp + x) * 512 + lane * 16);
                    y[x].x += z.x * st[w2][0]; y[x].y += z.y * st[w2][1]; y[x].z += z.z * st[w2][0]; y[x].w += z.w * st[w2][1];
                }
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                const int r = 2 * t4 + i;
                if (r >= j.nrows) continue;
                const float by = final ? (ll[i] == 0.f ? 0.f : vs / ll[i]) : vs;
                const int hq = j.h * p.G + r;
                char *out = p.out + ((int64_t)j.first_seq * p.out_seq + (int64_t)hq * p.out_head) * 2;
                float *to = CL ? part[CL ? r : 0]
                               : (j.complete ? p.whole + ((int64_t)j.first_seq * p.H * p.G + hq) * kAttRowPitch
                                             : p.slots + (((int64_t)blockIdx.x * 2 + (j.begins ? 1 : 0)) * RT + r) * kAttRowPitch);
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int d = 16 * (2 * warp + x) + 2 * g8;
                    const float lower = (i ? y[x].y : y[x].x) * by, upper = (i ? y[x].w : y[x].z) * by;
                    if (final) *reinterpret_cast<uint32_t *>(out + 2 * d) = cvt_bf16x2(upper, lower);
                    else *reinterpret_cast<float2 *>(to + d) = make_float2(lower, upper);
                }
                if (warp == 0 && g8 == 0) {
                    if (!final) *reinterpret_cast<float2 *>(to + kHeadDim) = make_float2(mm[i], ll[i]);
                    else if (p.lse) p.lse[(int64_t)j.first_seq * p.H * p.G + hq] = ll[i] == 0.f ? -INFINITY : (mm[i] + log2f(ll[i])) * 0.69314718f;
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                const int r = g8 + 8 * i;
                float2 st[kAttWarps];
                float mm = -INFINITY, ll = 0.f;
#pragma unroll
                for (int w2 = 0; w2 < kAttWarps; ++w2) { st[w2] = stat[w2][r]; mm = fmaxf(mm, st[w2].x); }
#pragma unroll
                for (int w2 = 0; w2 < kAttWarps; ++w2) {
                    st[w2].x = st[w2].x == -INFINITY ? 0.f : ex2(st[w2].x - mm);
                    ll += st[w2].y * st[w2].x;
                }
                const float by = final ? (ll == 0.f ? 0.f : vs / ll) : vs;
                const int sr = p.spt ? att_small_div(r, inv_g) : 0, sq = j.first_seq + sr, hq = j.h * p.G + r - sr * p.G;
                char *out = p.out + ((int64_t)sq * p.out_seq + (int64_t)hq * p.out_head) * 2;
                float *to = CL ? part[CL ? r : 0]
                               : (j.complete ? p.whole + ((int64_t)sq * p.H * p.G + hq) * kAttRowPitch
                                             : p.slots + (((int64_t)blockIdx.x * 2 + (j.begins ? 1 : 0)) * RT + r) * kAttRowPitch);
#pragma unroll
                for (int q2 = 0; q2 < 2; ++q2) {
                    const int q = 2 * warp + q2;               // fragments 2 q, 2 q + 1
                    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                    for (int w2 = 0; w2 < kAttWarps; ++w2) {
                        const float4 x = *reinterpret_cast<const float4 *>(used + (w2 - warp) * (ST * kAttStageBytes) + (i * 8 + q) * 512 + lane * 16);
                        y.x += x.x * st[w2].x; y.y += x.y * st[w2].x; y.z += x.z * st[w2].x; y.w += x.w * st[w2].x;
                    }
                    y.x *= by; y.y *= by; y.z *= by; y.w *= by;
                    if (r >= j.nrows) continue;
                    if (KEY8) {                                // dims 16 q + 4 t4 + 0..3: even ones from fragment 2 q, odd ones from 2 q + 1
                        const int d = 16 * q + 4 * t4;
                        if (final) *reinterpret_cast<uint2 *>(out + 2 * d) = make_uint2(cvt_bf16x2(y.z, y.x), cvt_bf16x2(y.w, y.y));
                        else *reinterpret_cast<float4 *>(to + d) = make_float4(y.x, y.z, y.y, y.w);
                    } else {                                   // dims 16 q + 2 t4 + 0, 1 and 8 further on
                        const int d = 16 * q + 2 * t4;
                        if (final) {
                            *reinterpret_cast<uint32_t *>(out + 2 * d) = cvt_bf16x2(y.y, y.x);
                            *reinterpret_cast<uint32_t *>(out + 2 * d + 16) = cvt_bf16x2(y.w, y.z);
                        } else {
                            *reinterpret_cast<float2 *>(to + d) = make_float2(y.x, y.y);
                            *reinterpret_cast<float2 *>(to + d + 8) = make_float2(y.z, y.w);
                        }
                    }
                }
                if (warp == 0 && t4 == 0 && r < j.nrows) {
                    if (!final) *reinterpret_cast<float2 *>(to + kHeadDim) = make_float2(mm, ll);
                    else if (p.lse) p.lse[(int64_t)sq * p.H * p.G + hq] = ll == 0.f ? -INFINITY : (mm + log2f(ll)) * 0.69314718f;
                }
            }
        }
        if constexpr (CL > 0) break;                       // (j may be an empty job by now)
        __syncthreads();                                   // the stages may be refilled
    }
    cp_wait<0>();
    if constexpr (CL > 0) {
        // every block of the cluster joins 128 / CL dims of all rows
        constexpr int DIMS = kHeadDim / (CL ? CL : 1);
        asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;\n" ::: "memory");
        for (int i = tid; i < p.G * DIMS; i += kAttThreads) {
            const int r = i / DIMS, d = rank * DIMS + i % DIMS;
            float x[CL], pm[CL], pl[CL], mm = -INFINITY;
#pragma unroll
            for (int b = 0; b < CL; ++b) {
                const uint32_t row = smem_u32(part[r]);
                uint32_t peer;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(peer) : "r"(row), "r"(b));
                asm volatile("ld.shared::cluster.f32 %0, [%1];\n" : "=f"(x[b]) : "r"(peer + 4 * d));
                asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];\n" : "=f"(pm[b]), "=f"(pl[b]) : "r"(peer + 4 * kHeadDim));
                mm = fmaxf(mm, pm[b]);
            }
            float y = 0.f, ll = 0.f;
#pragma unroll
            for (int b = 0; b < CL; ++b) {
                if (pm[b] == -INFINITY && !(pl[b] != pl[b])) continue;         // no rows there (a NaN sum stays)
                const float by = pm[b] == -INFINITY ? 1.f : ex2(pm[b] - mm);
                y += x[b] * by;
                ll += pl[b] * by;
            }
            const int hq = sh.h * p.G + r;
            *reinterpret_cast<__nv_bfloat16 *>(p.out + ((int64_t)sh.seq * p.out_seq + (int64_t)hq * p.out_head) * 2 + 2 * d) =
                __float2bfloat16_rn(ll == 0.f ? 0.f : y / ll);
            if (p.lse && d == 0) p.lse[(int64_t)sh.seq * p.H * p.G + hq] = ll == 0.f ? -INFINITY : (mm + log2f(ll)) * 0.69314718f;
        }
        asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;\n" ::: "memory");   // peers have read
    }
    if (p.under) grid_dependency_wait();                  // not through before the pass over prefixes is
}

template <bool KEY8, int RT>
__global__ void __launch_bounds__(kAttThreads, kAttBlocksPerSM) k_attend(const __grid_constant__ AttendParams p)
{
    attend_block<KEY8, RT, 0>(p, p);
}
template <bool KEY8, int RT>
__global__ void __launch_bounds__(kAttThreads, kAttBlocksPerSM)
k_attend_cluster(const __grid_constant__ AttendParams p, const __grid_constant__ AttendParams pre)
{
    attend_block<KEY8, RT, kAttCluster>(p, pre);
}

// ----------------------------------------------------------------------------------------------
// Joins the parts of every (sequence, KV head): those of its own rows and those of its prefix.
// ----------------------------------------------------------------------------------------------
struct AttendPass {                // where a pass left its parts
    const int2 *rec;
    const float *slots, *whole;
    int32_t blocks;                // of the pass
    int32_t rows;                  // query rows per slot; 128: the sums of 4 dims of all rows, the next 4 dims, .., (m, l) of all rows
    int32_t spt;                   // prefixes: sequences per tile
};

struct MergeParams {
    AttendPass own, pre;           // pre.rec == NULL: no prefixes
    int32_t S, P, H, G;
    int32_t rows;                  // query rows per block: G or 1
    const int32_t *group_start;
    char *out;
    int64_t out_seq, out_head;
    float *lse;
    int32_t *device_status;
};

constexpr int kMergeTile = 128;     // query rows per slot of k_attend_prefix, see AttendPass::rows

// A block joins `rows` query rows of one (sequence, KV head): all G, or one where there are too few units to fill the GPU.
// 16 / rows warps per row take its parts four at a time, each lane four sums, and are joined through shared memory.  Bound
// by the latency of a chain of three L2 reads (record; parts; nothing more for up to 4 parts per warp).
// The kernel is launched while the pass before it still runs (programmatic dependent launch) and waits for it here.
constexpr int kMergeWarps = 16, kMergeThreads = 32 * kMergeWarps;

__global__ void __launch_bounds__(kMergeThreads) k_attend_merge(const MergeParams p)
{
    __shared__ float4 red[kMergeWarps][32];
    __shared__ float2 red_ml[kMergeWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int per = p.G / p.rows, unit = blockIdx.x / per, s = unit / p.H, h = unit - s * p.H;
    // the sequence's group, before the passes are waited for: they began behind whatever wrote group_start (see ld_relaxed)
    int pre_rec = -1, row0 = 0;
    if (p.pre.rec) {
        const int lo = att_group_of<true>(p.group_start, p.P, s, lane);
        const int2 g = att_group<true>(p.group_start, p.S, lo);
        if (s >= g.x && s < g.x + g.y) {
            const int rt = (s - g.x) / p.pre.spt;
            pre_rec = att_tile_index(lo, g.x, p.pre.spt, rt) * p.H + h;
            row0 = (s - g.x - rt * p.pre.spt) * p.G;
        }
    }
    grid_dependency_wait();
    grid_dependents_launch();
    if (p.pre.rec && blockIdx.x == 0 && p.device_status)
        for (int i = threadIdx.x; i < p.P; i += kMergeThreads)
            if (att_descends(p.group_start, p.S, i)) atomicExch(p.device_status, (int)TRI_ERR_DEVICE_CHECK);
    const int2 own = p.own.rec[unit];
    if (!p.pre.rec && own.y < 2) return;                                     // finished by its block
    int2 pre = pre_rec >= 0 ? p.pre.rec[pre_rec] : make_int2(0, 0);
    // groups that descend have no records: whatever lies there names no slot outside the workspace
    if ((uint32_t)pre.y > (uint32_t)p.pre.blocks || (uint32_t)(pre.x >> 1) > (uint32_t)(p.pre.blocks - pre.y)) pre = make_int2(0, 0);
    const int parts = own.y + pre.y;
    const int wpr = kMergeWarps / p.rows, r = warp / wpr, sub = warp - r * wpr, g = ((int)blockIdx.x - unit * per) * p.rows + r;
    const bool active = r < p.rows;
    const int64_t hq = (int64_t)h * p.G + g;
    // part i: the own rows' parts in ascending order, then the prefix's; its row, and where its (m, l) lie
    const bool tiled = p.pre.rows == kMergeTile && pre.y > 1;
    auto at = [&](int i, const float2 *&ml) -> const float * {
        const bool is_own = i < own.y;
        const AttendPass &a = is_own ? p.own : p.pre;
        const int2 rc = is_own ? own : pre;
        const int k = is_own ? i : i - own.y, row = is_own ? g : row0 + g;
        const float *src;
        if (rc.y == 1) {
            src = a.whole + ((int64_t)s * p.H * p.G + hq) * kAttRowPitch;
        } else {
            src = a.slots + (int64_t)(k == 0 ? rc.x : (rc.x & ~1) + 2 * k) * a.rows * kAttRowPitch;
            if (!is_own && tiled) {
                ml = reinterpret_cast<const float2 *>(src + kMergeTile * kHeadDim) + row;
                return src + 4 * row;
            }
            src += row * kAttRowPitch;
        }
        ml = reinterpret_cast<const float2 *>(src + kHeadDim);
        return src;
    };
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
    float mm = -INFINITY, ll = 0.f;
    auto add = [&](float2 ml, float4 x) {                                    // one more summary
        const float top = fmaxf(mm, ml.x);
        const float old = mm == -INFINITY ? 0.f : ex2(mm - top), by = ml.x == -INFINITY ? 0.f : ex2(ml.x - top);
        mm = top;
        ll = ll * old + ml.y * by;
        a.x = a.x * old + x.x * by; a.y = a.y * old + x.y * by; a.z = a.z * old + x.z * by; a.w = a.w * old + x.w * by;
    };
    if (active) {
        for (int b = sub; b < parts; b += 4 * wpr) {
            float2 ml[4];
            float4 x[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int i = b + k * wpr;
                ml[k] = make_float2(-INFINITY, 0.f);
                x[k] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (i < parts) {
                    const float2 *mlp;
                    const float *src = at(i, mlp);
                    ml[k] = *mlp;
                    x[k] = *reinterpret_cast<const float4 *>(src + lane * (tiled && i >= own.y ? 4 * kMergeTile : 4));
                }
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) add(ml[k], x[k]);
        }
        red[warp][lane] = a;
        if (lane == 0) red_ml[warp] = make_float2(mm, ll);
    }
    __syncthreads();
    if (!active || sub != 0) return;
    for (int w = 1; w < wpr; ++w) add(red_ml[warp + w], red[warp + w][lane]);
    const float inv = ll == 0.f ? 0.f : 1.f / ll;
    *reinterpret_cast<uint2 *>(p.out + ((int64_t)s * p.out_seq + hq * p.out_head) * 2 + 8 * lane) =
        make_uint2(cvt_bf16x2(a.y * inv, a.x * inv), cvt_bf16x2(a.w * inv, a.z * inv));
    if (p.lse && lane == 0) p.lse[(int64_t)s * p.H * p.G + hq] = ll == 0.f ? -INFINITY : (mm + log2f(ll)) * 0.69314718f;
}

}  // namespace tri
