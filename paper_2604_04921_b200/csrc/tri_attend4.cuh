// Attention of one decode step over a 4-bit cache (tri_row4.cuh).
//
// Mathematics.  As in tri_attend.cuh, with k_n = s_ng (u - 8) + c_ng for the codes u of group g (32 components), and v_n likewise:
//       q . k_n  = sum_g s_ng (sum_d q_d u_nd - 8 Q_g) + sum_g c_ng Q_g,      Q_g = sum of q over group g
//       sum_n p_n v_n = sum_n (p_n s_ng) u + sum_n p_n (c_ng - 8 s_ng)
// so that the matrix instructions work on codes, and scales and centres are applied per row and group:
//   logits   keys are the 16 rows of A, 8 query rows the columns of B.  A nibble in 16 bits of its own is the f16 value u 2^-24, or
//            u 2^-20 where it lies four bits further up: 5 integer instructions make operands of 8 codes (as bf16, with 128 or-ed in,
//            7; as e4m3, whose matrix instructions sm_100a makes of conversions and f16 ones, 3 and 20 conversions).  A query row is
//            brought to [2^14, 2^15) by a power of two and goes in as f16, a sixteenth of it where the codes are 16 times as large: a
//            bf16 value is exact unless it is 2^28 times smaller than the row's largest.  Centres, and the 8 that each code is too
//            large by, go through one matrix instruction more: c_ng against Q_g and s_ng against -8 Q_g, both in two bf16 parts, that
//            is to 2^-16.
//   sums     the 16 rows of A are components, its 16 columns cached rows, operands likewise: A's upper 8 rows carry 16 times the lower
//            ones.  They sum p_n s_ng u; the 8 goes with the centres, sum_n p_n (c_ng - 8 s_ng).  The matrix instructions truncate, so
//            that sums of positive terms drift by some 2^-25 per instruction, against which a difference of the two would not last:
//            every 16 steps the accumulators go to sums in shared memory.  (8 taken off in the accumulators, by a matrix of constants,
//            takes 41.5 us where this takes 39.6.)  The weights p_n s_ng are rounded once to f16: the bound on the logits that p is
//            taken against goes by the largest scale of the rows so far, too, so that they use f16's range from 2^15 down.  The
//            centres are summed in fp32.
//
// What bounds it.  160 bytes per row and head: at HBM speed a multiprocessor gets 16 rows every 60 ns, in which 316 warp instructions
// have to be issued.  131,072 rows of 8 heads, G = 4: 40.0 us, 4.2 TB/s (0.65 of the copy rate).  No unit is full: issue slots 0.54,
// ALU 0.51, tensor pipe 0.23, HBM 0.5.  What is waited for is the chain within a step (scales to shared memory and back, matrix
// instructions, the vote, exponentials, transposes, matrix instructions), which the 3 warps that a scheduler has do not cover; fixed
// latency is the first of the stalls.  (Shifts as multiplications on the other pipe: 41.5 us; four blocks per multiprocessor spill; widening to tensor
// memory for tcgen05.mma, whose instructions then cost nothing: 55 us, the widening of a row per thread takes longer.)
// Copies are 16-byte asynchronous ones into a ring of stages that each warp keeps for itself; a stage is 32 rows of K and of V (bulk
// copies per warp: 44 us).  Work split, records and parts are those of tri_attend.cuh.
#pragma once
#include "tri_attend.cuh"
#include "tri_row4.cuh"

namespace tri {

constexpr int kA4Warps = kAttWarps, kA4Threads = 32 * kA4Warps, kA4Rows = 32, kA4Stages = 2;      // (one step ahead)
constexpr int kA4Half = kA4Rows * kRow4Bytes, kA4StageBytes = 2 * kA4Half;                  // K | V
constexpr int kA4ScaleBytes = kA4Rows * 48;                      // scales of K, scales and centres of V in fp32
constexpr int kA4SumSteps = 16;                                  // steps between two additions to the sums in shared memory
template <int RT> constexpr int kA4SumBytes = (RT == 16 ? 2 : 1) * 8 * 512;
template <int RT> constexpr int kA4WarpBytes = kA4Stages * kA4StageBytes + kA4ScaleBytes + kA4SumBytes<RT>;
template <int RT> constexpr int kA4RingBytes = kA4Warps * kA4WarpBytes<RT>;
constexpr int kA4Tile = kA4Warps * kA4Rows;
constexpr int kA4UnitCost = 2;                                   // a unit's own cost, in tiles
// Units that go to a cluster each, as in tri_attend.cuh, have up to so many rows, by query rows (one sequence of 8 heads, cluster against
// the whole GPU: G = 4, 600 rows 4.7 / 8.4 us, 4,352 8.5 / 10.4, 8,192 11.0 / 11.8, 12,288 14.6 / 13.3; G = 16, 600 rows 7.6 / 10.7, 2,176
// 10.6 / 11.8, 3,584 11.3 / 12.1, 4,352 12.8 / 12.2).
constexpr int kA4ClusterRows = 8192, kA4ClusterRowsWide = 3584;  // up to 8 query rows, more
template <int RT> constexpr int kA4BlocksPerSM = RT <= 8 ? 3 : 2;
constexpr float kA4NoBound = -3e38f;                             // below every logit; finite, so that 2^(-infinity - m) is 0
constexpr uint32_t kLow = 0x000f000fu, kHigh = 0x00f000f0u;     // nibbles that are pairs of f16 values u 2^-24, u 2^-20
static_assert(kA4StageBytes >= 8 * 512, "the sums of a warp fit into a stage");

__device__ __forceinline__ void mma_bf16_16816_new(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};\n"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ void mma_f16_16816_new(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};\n"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t cvt_f16x2(float upper, float lower)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;\n" : "=r"(r) : "f"(upper), "f"(lower));
    return r;
}
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;\n" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint4 lds128(uint32_t at)
{
    uint4 r;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];\n" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(at) : "memory");
    return r;
}
__device__ __forceinline__ float4 lds_f4(uint32_t at)
{
    const uint4 x = lds128(at);
    return make_float4(__uint_as_float(x.x), __uint_as_float(x.y), __uint_as_float(x.z), __uint_as_float(x.w));
}
__device__ __forceinline__ void sts128(uint32_t at, float a, float b, float c, float d)
{
    asm volatile("st.shared.v4.f32 [%0], {%1,%2,%3,%4};\n" ::"r"(at), "f"(a), "f"(b), "f"(c), "f"(d) : "memory");
}
__device__ __forceinline__ uint2 lds64(uint32_t at)
{
    uint2 r;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];\n" : "=r"(r.x), "=r"(r.y) : "r"(at) : "memory");
    return r;
}
__device__ __forceinline__ float2 lds_f2(uint32_t at)
{
    const uint2 x = lds64(at);
    return make_float2(__uint_as_float(x.x), __uint_as_float(x.y));
}
__device__ __forceinline__ uint32_t lds32(uint32_t at)
{
    uint32_t r;
    asm volatile("ld.shared.u32 %0, [%1];\n" : "=r"(r) : "r"(at) : "memory");
    return r;
}
// Group g of four values in the order of groups 0, 2, 1, 3.
__device__ __forceinline__ float pick(const float4 &x, int g) { return g == 0 ? x.x : (g == 2 ? x.y : (g == 1 ? x.z : x.w)); }
__device__ __forceinline__ uint32_t pick(const uint4 &x, int i) { return i == 0 ? x.x : (i == 1 ? x.y : (i == 2 ? x.z : x.w)); }

// RT: query rows, up to 4, 8 or 16 (two column tiles).  RT = 4: the other 4 columns hold the same rows again; then the weights of
// two groups go into one operand, half of the columns each, and their sums into those columns of each group's accumulators.
// CL > 0: a cluster of CL blocks takes one unit, as in tri_attend.cuh.
template <int RT, int CL>
__device__ __forceinline__ void attend4_block(const AttendParams &p)
{
    constexpr int CT = RT == 16 ? 2 : 1, COLS = 8 * CT, GP = RT == 4 ? 2 : 4, ST = kA4Stages, ROWS = kA4Rows, NK = 2, TILE = kA4Tile;
    static_assert(ROWS == 16 * NK, "two tiles of 16 cached rows per step");
    extern __shared__ __align__(128) uint8_t dyn[];
    __shared__ float2 stat[kA4Warps][COLS];
    __shared__ __align__(16) float part[CL ? COLS : 1][kAttRowPitch];      // this block's sums, and (m, l)

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g8 = lane >> 2, t4 = lane & 3;
    const uint32_t ring = smem_u32(dyn) + warp * kA4WarpBytes<RT>, scales = ring + ST * kA4StageBytes;
    float4 *sums = reinterpret_cast<float4 *>(dyn + warp * kA4WarpBytes<RT> + ST * kA4StageBytes + kA4ScaleBytes) + lane;      // 32 apart
    // Cached row of row i of a matrix tile of keys: i / 2 + 4 (i % 2) of 8 (the second 8 rows 8 further on).  Rows 4 apart are 64 bytes
    // apart in the banks: two rows' 64 bytes of codes, one load's phase, take all of them.  The sums over cached rows then take
    // columns 2 t4, 2 t4 + 1 of A from rows t4, t4 + 4.
    const int row_k = (g8 >> 1) + 4 * (g8 & 1);
    const uint32_t klane = row_k * kRow4Bytes, vlane = t4 * kRow4Bytes + 16 * (g8 >> 1);
    const int odd_cols = RT == 4 ? t4 >> 1 : 0;           // RT = 4: which group of a pair this lane's columns are for
    const uint32_t half = g8 & 1 ? 0x7632u : 0x5410u;     // which half of a word of V holds this lane's components
    grid_dependency_wait();
    grid_dependents_launch();
    AttShare sh = {};
    int rank = 0;
    if constexpr (CL == 0) {
        sh = att_share<TILE, kA4UnitCost>(p);
        if ((int)blockIdx.x >= sh.shares) return;
    } else {
        asm volatile("mov.u32 %0, %%cluster_ctarank;\n" : "=r"(rank));
        sh.seq = (int)blockIdx.x / CL / p.H; sh.h = (int)blockIdx.x / CL - sh.seq * p.H;
        if (tid < COLS) { part[CL ? tid : 0][kHeadDim] = -INFINITY; part[CL ? tid : 0][kHeadDim + 1] = 0.f; }      // no rows so far
    }
    // ---------------- the walk over the share's units, one step ahead of the sums ----------------
    AttCursor cursor = {sh.seq, sh.h, 0, sh.start};
    AttJob u = {};                                        // the unit that is being copied
    // To the next unit with rows; units without rows, and those of which the share holds only their own cost, are settled here.
    auto walk = [&]() -> bool {
        if constexpr (CL == 0) {
            while (att_next<TILE, kA4UnitCost>(p, sh, cursor, u)) {
                if (u.begins && tid == 0) p.rec[u.rec] = att_record(sh, u);
                if (u.kt == 0 && u.begins)                // no rows: zeros
                    for (int i = tid; i < p.G * 16; i += kA4Threads) {
                        const int hq = u.h * p.G + (i >> 4);
                        *reinterpret_cast<uint4 *>(p.out + ((int64_t)u.seq * p.out_seq + (int64_t)hq * p.out_head) * 2 + 16 * (i & 15)) =
                            make_uint4(0u, 0u, 0u, 0u);
                        if (p.lse && (i & 15) == 0) p.lse[(int64_t)u.seq * p.H * p.G + hq] = -INFINITY;
                    }
                if (u.kb > u.ka) return true;
            }
            return false;
        } else {
            if (cursor.rt++ > 0) return false;
            u.seq = cursor.seq; u.h = cursor.h;
            u.len = att_len(p, u.seq, u.h);
            u.kt = (int)(((uint32_t)u.len + TILE - 1) / TILE);
            u.ka = rank * u.kt / CL; u.kb = (rank + 1) * u.kt / CL;
            u.begins = u.complete = false;
            return u.kb > u.ka;
        }
    };

    // ---------------- copies ----------------
    int next = 0, stage = 0, page[NK] = {}, slot[NK] = {};        // next step to copy; page and first slot of its 16-row halves
    uint32_t bad = 0;                                     // bits 2 i, 2 i + 1: these 16 rows of stage i are absent
    int64_t unit_base = 0;                                // first row of the unit; of page 0, where rows are paged
    uint64_t policy;                                      // rows are read once in a step: first to leave L2
    asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;\n" : "=l"(policy));
    const uint32_t step_row = (uint32_t)(p.src.paged ? p.src.stride_slot : p.src.stride_tok);      // bytes between rows (the host checks)
    auto look_up = [&]() {                                // pages of the next step
        if (!p.src.paged) return;
#pragma unroll
        for (int x = 0; x < NK; ++x) {
            const uint32_t r = (uint32_t)next * TILE + warp * ROWS + 16 * x;
            const uint32_t pg = p.src.page_shift >= 0 ? r >> p.src.page_shift : r / (uint32_t)p.src.page_size;
            page[x] = r < (uint32_t)u.len ? ld_here(p.src.page_table + (int64_t)u.seq * p.src.max_pages_per_seq + pg) : 0;
            slot[x] = (int)(r - pg * (uint32_t)p.src.page_size);
        }
    };
    auto begin_unit = [&]() {
        next = u.ka;
        unit_base = (int64_t)p.layer * p.src.stride_layer + (int64_t)u.h * p.src.stride_head + (p.src.paged ? 0 : (int64_t)u.seq * p.src.stride_seq);
        look_up();
    };
    auto issue = [&](int to) {                            // the next step into stage `to`
        const uint32_t dst = ring + to * kA4StageBytes + 16 * lane;
        const uint32_t r = (uint32_t)next * TILE + warp * ROWS;
        const int rows = r < (uint32_t)u.len ? min(u.len - (int)r, ROWS) : 0;
        int have[NK] = {min(rows, 16), max(rows - 16, 0)};
        int64_t base[NK];
        uint32_t miss = 0;
        if (p.src.paged) {
#pragma unroll
            for (int x = 0; x < NK; ++x) {                // 16 rows each: they lie in one page
                base[x] = unit_base + (int64_t)page[x] * p.src.stride_page + (int64_t)((uint64_t)(uint32_t)slot[x] * step_row);
                if (have[x] && p.src.n_pages > 0 && (uint32_t)page[x] >= (uint32_t)p.src.n_pages) {
                    have[x] = 0;
                    miss |= 1u << x;
                    if (lane == 0 && p.device_status) atomicExch(p.device_status, (int)TRI_ERR_DEVICE_CHECK);
                }
            }
        } else {
            base[0] = unit_base + (int64_t)((uint64_t)r * step_row);
            base[1] = base[0] + (int64_t)((uint64_t)16 * step_row);
        }
        // The 160 pieces of a stage's keys, 5 per row, go to the lanes in turn; where rows lie side by side, as they do in the
        // stage, a piece's place in the copy is its place in the source.
        if (rows == ROWS && miss == 0 && step_row == kRow4Bytes) {
            const char *k0 = p.src.k + (base[0] + 16 * lane), *v0 = p.src.v + (base[0] + 16 * lane);
            if (base[1] == base[0] + 16 * kRow4Bytes) {
#pragma unroll
                for (int i = 0; i < 5; ++i) {
                    cp_async16(dst + 512 * i, k0 + 512 * i, 16u, policy);
                    cp_async16(dst + kA4Half + 512 * i, v0 + 512 * i, 16u, policy);
                }
            } else {
                const char *k1 = p.src.k + (base[1] + (16 * lane - 16 * kRow4Bytes)), *v1 = p.src.v + (base[1] + (16 * lane - 16 * kRow4Bytes));
#pragma unroll
                for (int i = 0; i < 5; ++i) {             // (piece 80 is the second half's first)
                    const bool second = i == 2 ? lane >= 16 : i > 2;
                    cp_async16(dst + 512 * i, (second ? k1 : k0) + 512 * i, 16u, policy);
                    cp_async16(dst + kA4Half + 512 * i, (second ? v1 : v0) + 512 * i, 16u, policy);
                }
            }
        } else {
            // rows behind the length (or absent ones) arrive as zeros and are not read
#pragma unroll 1
            for (int i = 0; i < 5; ++i) {
                const int piece = 32 * i + lane, row = piece / 5, col = piece - 5 * row, x = row >> 4;
                const bool there = (row & 15) < (x == 0 ? have[0] : have[1]);
                const int64_t at = there ? (x == 0 ? base[0] : base[1]) + (int64_t)((uint64_t)(uint32_t)(row & 15) * step_row) + 16 * col : 0;
                cp_async16(dst + 512 * i, p.src.k + at, there ? 16u : 0u, policy);
                cp_async16(dst + kA4Half + 512 * i, p.src.v + at, there ? 16u : 0u, policy);
            }
        }
        bad = (bad & ~(3u << (2 * to))) | (miss << (2 * to));
        if (++next < u.kb) look_up();
    };
    bool more = walk();
    if (more) { begin_unit(); issue(0); }
    cp_commit();

    struct { int seq, h, len, it, kb; bool begins, complete; } j = {};      // the unit that is being summed
    uint32_t q[CT][4][4];                                 // components 32 g + 8 t4 .. + 7 of query row g8 (+ 8 ct)
    float mul[CT][2];                                     // logit in base-2 units per accumulator unit, query rows 2 t4, 2 t4 + 1
    uint32_t qsum[CT][2];                                 // Q and -8 Q in two bf16 parts, B operand of centres and scales
    float o[CT][4][2][4], oc[CT][GP][2], m[CT][2], l[CT][2];
    float top = 0.f, above = 0.f;                         // largest size of values so far, a power of two; 15 less its exponent
    bool summed = false;                                  // whether there are sums in shared memory
    auto to_sums = [&]() {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                float (&a)[4] = o[ct][x >> 1][x & 1];
                float4 y = make_float4(a[0], a[1], a[2], a[3]);
                if (summed) {
                    const float4 z = sums[32 * (8 * ct + x)];
                    y.x += z.x; y.y += z.y; y.z += z.z; y.w += z.w;
                }
                sums[32 * (8 * ct + x)] = y;
                a[0] = a[1] = a[2] = a[3] = 0.f;
            }
        summed = true;
    };
    for (;;) {
        if (j.it == j.kb) {
            // ---------------- the next unit: the one whose first step has been copied ----------------
            if (!more) break;
            j = {u.seq, u.h, u.len, u.ka, u.kb, u.begins, u.complete};
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                const int r = (RT == 4 ? g8 & 3 : g8) + 8 * ct;
                const char *qr = p.q + ((int64_t)j.seq * p.q_seq + (int64_t)(j.h * p.G + r) * p.q_head) * 2 + 16 * t4;
                float x[4][8], amax = 0.f, sum[4];
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const uint4 raw = r < p.G ? *reinterpret_cast<const uint4 *>(qr + 64 * g) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        x[g][2 * i] = bf16_lo(pick(raw, i)); x[g][2 * i + 1] = bf16_hi(pick(raw, i));
                        amax = fmaxf(amax, fmaxf(fabsf(x[g][2 * i]), fabsf(x[g][2 * i + 1])));
                    }
                }
                amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
                amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
                const int e = min(max((int)(__float_as_uint(amax) >> 23) - 127, -113), 127);
                const float by = __uint_as_float((uint32_t)(141 - e) << 23), back = p.scale * 0x1p10f * __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
                for (int g = 0; g < 4; ++g) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[g][i] *= by;
                    // (i odd: against codes 16 times as large)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float part = i & 1 ? 0.0625f : 1.f;
                        q[ct][g][i] = cvt_f16x2(x[g][2 * i + 1] * part, x[g][2 * i] * part);
                    }
                    sum[g] = ((x[g][0] + x[g][1]) + (x[g][2] + x[g][3])) + ((x[g][4] + x[g][5]) + (x[g][6] + x[g][7]));
                    sum[g] += __shfl_xor_sync(0xffffffffu, sum[g], 1);
                    sum[g] += __shfl_xor_sync(0xffffffffu, sum[g], 2);
                    sum[g] *= 0x1p-24f;                    // in units of the accumulators of codes u 2^-24
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) mul[ct][i] = __shfl_sync(0xffffffffu, back, (2 * t4 + i) * 4);
                // slots 2 t4, 2 t4 + 1 of the first 8: Q of groups (0, 1), (2, 3), the high parts, then the low ones; of the second 8
                // -8 Q likewise
                const float a = t4 & 1 ? sum[2] : sum[0], b = t4 & 1 ? sum[3] : sum[1];
                const uint32_t hi = cvt_bf16x2(b, a), lo = cvt_bf16x2(b - bf16_hi(hi), a - bf16_lo(hi)), part8 = t4 < 2 ? hi : lo;
                qsum[ct][0] = part8;
                qsum[ct][1] = cvt_bf16x2(-8.f * bf16_hi(part8), -8.f * bf16_lo(part8));
#pragma unroll
                for (int g = 0; g < 4; ++g) {
#pragma unroll
                    for (int y = 0; y < 2; ++y) o[ct][g][y][0] = o[ct][g][y][1] = o[ct][g][y][2] = o[ct][g][y][3] = 0.f;
                    oc[ct][g % GP][0] = oc[ct][g % GP][1] = 0.f;
                }
                m[ct][0] = m[ct][1] = kA4NoBound;
                l[ct][0] = l[ct][1] = 0.f;
            }
            summed = false;
            top = 0x1p-81f; above = kAttAbove<true> + 81.f;
        }
        // the other stage has been read, or used and released in joining a unit
        if (more && next == u.kb) {
            more = walk();
            if (more) begin_unit();
        }
        if (more) issue(stage ^ 1);
        cp_commit();

        // ---------------- one step ----------------
        cp_wait<ST - 1>();
        __syncwarp();
        const uint32_t r0 = (uint32_t)j.it * TILE + warp * ROWS;
        const int have = r0 < (uint32_t)j.len ? min(j.len - (int)r0, ROWS) : 0;
        const uint32_t miss = (bad >> (2 * stage)) & 3u;
        const bool cut = have < ROWS || miss;
        const uint32_t kb_s = ring + stage * kA4StageBytes, vb_s = kb_s + kA4Half;
        // a lane widens the scales (of groups 0, 2, 1, 3) and centres (of V: c - 8 s) of one row for all
        const uint4 k_par = lds128(kb_s + lane * kRow4Bytes + kRow4Scales), v_par = lds128(vb_s + lane * kRow4Bytes + kRow4Scales);
        const uint32_t row48 = scales + lane * 48;
        sts128(row48, bf16_lo(k_par.x), bf16_lo(k_par.y), bf16_hi(k_par.x), bf16_hi(k_par.y));
        sts128(row48 + 16, bf16_lo(v_par.x), bf16_lo(v_par.y), bf16_hi(v_par.x), bf16_hi(v_par.y));
        sts128(row48 + 32, fmaf(-8.f, bf16_lo(v_par.x), bf16_lo(v_par.z)), fmaf(-8.f, bf16_lo(v_par.y), bf16_lo(v_par.w)),
               fmaf(-8.f, bf16_hi(v_par.x), bf16_hi(v_par.z)), fmaf(-8.f, bf16_hi(v_par.y), bf16_hi(v_par.w)));
        const uint32_t s_max = max_bf16x2(v_par.x, v_par.y), c_max = max_bf16x2(v_par.z & 0x7fff7fffu, v_par.w & 0x7fff7fffu);
        __syncwarp();
        // logits: 16 cached rows x 8 query rows; the thread holds rows g8, g8 + 8 of the tile for query rows 2 t4, 2 t4 + 1
        float w[CT][NK][4];
#pragma unroll
        for (int kg = 0; kg < NK; ++kg) {
            const uint32_t at = kb_s + klane + 16 * kg * kRow4Bytes;
            const uint4 ka = lds128(at + 16 * t4), kb = lds128(at + 8 * kRow4Bytes + 16 * t4);
            const uint32_t wide = scales + row_k * 48 + 16 * kg * 48;
            const float4 sa = lds_f4(wide), sb = lds_f4(wide + 8 * 48);
            const uint32_t ca = lds32(at + kRow4Centres + 4 * (t4 & 1)), cb = lds32(at + 8 * kRow4Bytes + kRow4Centres + 4 * (t4 & 1));
            const uint32_t da = lds32(at + kRow4Scales + 4 * (t4 & 1)), db = lds32(at + 8 * kRow4Bytes + kRow4Scales + 4 * (t4 & 1));
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) mma_bf16_16816_new(w[ct][kg], ca, cb, da, db, qsum[ct][0], qsum[ct][1]);
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const uint32_t xa = pick(ka, g), xb = pick(kb, g);
                const uint32_t xa8 = xa >> 8, xb8 = xb >> 8;
                const float s0 = pick(sa, g), s1 = pick(sb, g);
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    float acc[4];
                    mma_f16_16816_new(acc, xa & kLow, xb & kLow, xa & kHigh, xb & kHigh, q[ct][g][0], q[ct][g][1]);
                    mma_f16_16816(acc, xa8 & kLow, xb8 & kLow, xa8 & kHigh, xb8 & kHigh, q[ct][g][2], q[ct][g][3]);
                    w[ct][kg][0] = fmaf(s0, acc[0], w[ct][kg][0]); w[ct][kg][1] = fmaf(s0, acc[1], w[ct][kg][1]);
                    w[ct][kg][2] = fmaf(s1, acc[2], w[ct][kg][2]); w[ct][kg][3] = fmaf(s1, acc[3], w[ct][kg][3]);
                }
            }
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int x = 0; x < 4; ++x) w[ct][kg][x] *= mul[ct][x & 1];
        }
        if (cut) {
#pragma unroll
            for (int kg = 0; kg < NK; ++kg)
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    if (16 * kg + row_k + 8 * (x >> 1) >= have || ((miss >> kg) & 1u))
#pragma unroll
                        for (int ct = 0; ct < CT; ++ct) w[ct][kg][x] = -INFINITY;
        }
        // The bound m on the logits, and `top` on the sizes of values: scales, and centres by 2^-30 (weights times centres stay below
        // 2^45).  m keeps weights times top in [2^11, 2^15] where they are largest.  Both are looked at by a vote and searched for only
        // when one has to be raised.  m is a whole number, so that top's exponent goes into it and out of it (at the join) exactly.
        float mx[CT][2], sm = fmaxf(fmaxf(bf16_lo(s_max), bf16_hi(s_max)), fmaxf(bf16_lo(c_max), bf16_hi(c_max)) * 0x1p-30f);
        bool raise = sm > top;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                mx[ct][i] = fmaxf(fmaxf(w[ct][0][i], w[ct][0][i + 2]), fmaxf(w[ct][NK - 1][i], w[ct][NK - 1][i + 2]));
                raise = raise || mx[ct][i] > m[ct][i] + above;
            }
        if (__any_sync(0xffffffffu, raise)) {
            if (summed) {                                 // (the sums are scaled below as what they were: accumulators)
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int x = 0; x < 8; ++x) {
                        const float4 z = sums[32 * (8 * ct + x)];
                        float (&a)[4] = o[ct][x >> 1][x & 1];
                        a[0] += z.x; a[1] += z.y; a[2] += z.z; a[3] += z.w;
                    }
                summed = false;
            }
#pragma unroll
            for (int d = 1; d < 32; d *= 2) sm = fmaxf(sm, __shfl_xor_sync(0xffffffffu, sm, d));
            if (sm > top) {                               // (all lanes alike)
                const int e = (int)min(__float_as_uint(sm) >> 23, 252u) - 126;
                top = __uint_as_float((uint32_t)(e + 127) << 23);
                above = kAttAbove<true> - (float)e;
            }
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
#pragma unroll
                    for (int d = 4; d < 32; d *= 2) mx[ct][i] = fmaxf(mx[ct][i], __shfl_xor_sync(0xffffffffu, mx[ct][i], d));
                    // the largest logit so far is at most m + above as it was, that is as far above m as the weights may reach
                    float to = m[ct][i];
                    if (mx[ct][i] > m[ct][i] + above) to = floorf(mx[ct][i] - above + (kAttAbove<true> - kAttBelow<true>));
                    // Two factors: where top rises from next to nothing to 2^100, rows that weigh as much as the new one are brought
                    // down by more than 2^126, which one factor would flush to 0.  (0 where there was no bound yet.)
                    const float down = m[ct][i] - to, part = fmaxf(down, -100.f), by = ex2(part), rest = ex2(down - part);
                    m[ct][i] = to;
                    l[ct][i] = l[ct][i] * by * rest;
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        if (g < GP) oc[ct][g][i] = oc[ct][g][i] * by * rest;
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            o[ct][g][y][i] = o[ct][g][y][i] * by * rest;
                            o[ct][g][y][i + 2] = o[ct][g][y][i + 2] * by * rest;
                        }
                    }
                }
        }
#pragma unroll
        for (int kg = 0; kg < NK; ++kg) {
            // weights, times scales, and transposed into the B operand: 16 cached rows x 8 query rows for each group
            uint32_t pw[CT][GP][2];
            float4 vs[2], vc[2];                          // scales and centres of rows g8, g8 + 8 of the tile; RT = 4: of two groups
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const uint32_t wide = scales + row_k * 48 + (16 * kg + 8 * x) * 48;
                if constexpr (RT == 4) {
                    const float2 a = lds_f2(wide + 16 + 8 * odd_cols), b = lds_f2(wide + 32 + 8 * odd_cols);
                    vs[x] = make_float4(a.x, a.y, 0.f, 0.f); vc[x] = make_float4(b.x, b.y, 0.f, 0.f);
                } else {
                    vs[x] = lds_f4(wide + 16); vc[x] = lds_f4(wide + 32);
                }
            }
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                float e[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    e[x] = ex2(w[ct][kg][x] - m[ct][x & 1]);
                    l[ct][x & 1] += e[x];
                }
#pragma unroll
                for (int g = 0; g < GP; ++g)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const float c = RT == 4 ? (g ? vc[x].y : vc[x].x) : pick(vc[x], g), s = RT == 4 ? (g ? vs[x].y : vs[x].x) : pick(vs[x], g);
                        oc[ct][g][0] = fmaf(e[2 * x], c, oc[ct][g][0]);
                        oc[ct][g][1] = fmaf(e[2 * x + 1], c, oc[ct][g][1]);
                        pw[ct][g][x] = transpose8x8(cvt_f16x2(e[2 * x + 1] * s, e[2 * x] * s));
                    }
            }
            const uint32_t at = vb_s + vlane + 16 * kg * kRow4Bytes;
            const uint4 v0 = lds128(at), v1 = lds128(at + 4 * kRow4Bytes), v2 = lds128(at + 8 * kRow4Bytes), v3 = lds128(at + 12 * kRow4Bytes);
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                // four components of rows (t4, t4 + 4) and of rows (t4 + 8, t4 + 12)
                const uint32_t xa = __byte_perm(pick(v0, g), pick(v1, g), half), xb = __byte_perm(pick(v2, g), pick(v3, g), half);
                const uint32_t xa8 = xa >> 8, xb8 = xb >> 8;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    mma_f16_16816(o[ct][g][0], xa & kLow, xa & kHigh, xb & kLow, xb & kHigh, pw[ct][g * GP / 4][0], pw[ct][g * GP / 4][1]);
                    mma_f16_16816(o[ct][g][1], xa8 & kLow, xa8 & kHigh, xb8 & kLow, xb8 & kHigh, pw[ct][g * GP / 4][0], pw[ct][g * GP / 4][1]);
                }
            }
        }
        __syncwarp();
        uint8_t *used = dyn + warp * kA4WarpBytes<RT> + stage * kA4StageBytes;
        stage ^= 1;
        if (++j.it < j.kb) {
            if (j.it % kA4SumSteps == 0) to_sums();
            continue;
        }
        if (summed) to_sums();

        // ---------------- the unit's rows of this share are through: join the warps ----------------
        // per 8 query rows: each leaves its sums in the stage it has just read, fragment by fragment, and takes a group of all.
        // Whoever joins parts multiplies them by 2^(difference of their bounds), which has to be one of logits alone: top, of which
        // every warp has its own, leaves the bound here.  (2^-20: 2^31 weights of 2^15 times values of 2^100 stay in fp32's range.)
        const bool final = j.complete && p.finish;
        const float unit = top * 0x1p-20f, shift = above - kAttAbove<true> + 20.f;      // 2^(shift) = 1 / unit
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
                for (int d = 4; d < 32; d *= 2) {
                    l[ct][i] += __shfl_xor_sync(0xffffffffu, l[ct][i], d);
#pragma unroll
                    for (int g = 0; g < GP; ++g) oc[ct][g][i] += __shfl_xor_sync(0xffffffffu, oc[ct][g][i], d);
                }
                if (g8 == 0) stat[warp][8 * ct + 2 * t4 + i] = make_float2(m[ct][i] + shift, l[ct][i] * unit);
            }
#pragma unroll
            for (int g = 0; g < 4; ++g)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    if (summed) {
                        const float4 z = sums[32 * (8 * ct + 2 * g + y)];
                        o[ct][g][y][0] = z.x; o[ct][g][y][1] = z.y; o[ct][g][y][2] = z.z; o[ct][g][y][3] = z.w;
                    }
                    *reinterpret_cast<float4 *>(used + (2 * g + y) * 512 + lane * 16) =
                        make_float4(fmaf(o[ct][g][y][0], 0x1p24f, oc[ct][g * GP / 4][0]) * unit, fmaf(o[ct][g][y][1], 0x1p24f, oc[ct][g * GP / 4][1]) * unit,
                                    fmaf(o[ct][g][y][2], 0x1p20f, oc[ct][g * GP / 4][0]) * unit, fmaf(o[ct][g][y][3], 0x1p20f, oc[ct][g * GP / 4][1]) * unit);
                }
            __syncthreads();
            const int from = RT == 4 ? 4 * g8 + (t4 & 1) + 2 * (warp & 1) : lane;          // (RT = 4: where the group's columns are)
            // components 32 warp + 8 (g8 / 2) + g8 % 2 + 0, 2, 4, 6 of query rows 2 t4, 2 t4 + 1 (+ 8 ct)
            float mm[2], ll[2], by[kA4Warps][2], z[2][4];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                mm[i] = -INFINITY; ll[i] = 0.f;
                z[i][0] = z[i][1] = z[i][2] = z[i][3] = 0.f;
#pragma unroll
                for (int w2 = 0; w2 < kA4Warps; ++w2) mm[i] = fmaxf(mm[i], stat[w2][8 * ct + 2 * t4 + i].x);
#pragma unroll
                for (int w2 = 0; w2 < kA4Warps; ++w2) {
                    const float2 ml = stat[w2][8 * ct + 2 * t4 + i];
                    by[w2][i] = ex2(ml.x - mm[i]);
                    ll[i] += ml.y * by[w2][i];
                }
            }
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int w2 = 0; w2 < kA4Warps; ++w2) {
                    const float4 x = *reinterpret_cast<const float4 *>(used + (w2 - warp) * kA4WarpBytes<RT> + (2 * warp + y) * 512 + from * 16);
                    z[0][2 * y] += x.x * by[w2][0]; z[1][2 * y] += x.y * by[w2][1];
                    z[0][2 * y + 1] += x.z * by[w2][0]; z[1][2 * y + 1] += x.w * by[w2][1];
                }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                // the pair of lanes with odd and even components swaps halves: four neighbours each
                const bool odd = g8 & 1;
                const float g0 = __shfl_xor_sync(0xffffffffu, odd ? z[i][0] : z[i][2], 4), g1 = __shfl_xor_sync(0xffffffffu, odd ? z[i][1] : z[i][3], 4);
                const float n = final ? (ll[i] == 0.f ? 0.f : 1.f / ll[i]) : 1.f;
                const float y0 = (odd ? g0 : z[i][0]) * n, y1 = (odd ? z[i][2] : g0) * n, y2 = (odd ? g1 : z[i][1]) * n, y3 = (odd ? z[i][3] : g1) * n;
                const int r = 8 * ct + 2 * t4 + i, d = 32 * warp + 8 * (g8 >> 1) + 4 * (g8 & 1);
                if (r >= p.G) continue;
                const int hq = j.h * p.G + r;
                float *to = CL ? part[CL ? r : 0] : p.slots + (((int64_t)blockIdx.x * 2 + (j.begins ? 1 : 0)) * COLS + r) * kAttRowPitch;
                if (final) *reinterpret_cast<uint2 *>(p.out + ((int64_t)j.seq * p.out_seq + (int64_t)hq * p.out_head) * 2 + 2 * d) = make_uint2(cvt_bf16x2(y1, y0), cvt_bf16x2(y3, y2));
                else *reinterpret_cast<float4 *>(to + d) = make_float4(y0, y1, y2, y3);
                if (warp == 0 && g8 == 0) {
                    if (!final) *reinterpret_cast<float2 *>(to + kHeadDim) = make_float2(mm[i], ll[i]);
                    else if (p.lse) p.lse[(int64_t)j.seq * p.H * p.G + hq] = ll[i] == 0.f ? -INFINITY : (mm[i] + log2f(ll[i])) * 0.69314718f;
                }
            }
            if (CL == 0 || ct + 1 < CT) __syncthreads();   // the stages may be refilled
        }
        if constexpr (CL > 0) break;
    }
    cp_wait<0>();
    if constexpr (CL > 0) {
        // every block of the cluster joins 128 / CL dims of all rows
        constexpr int DIMS = kHeadDim / (CL ? CL : 1);
        asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;\n" ::: "memory");
        for (int i = tid; i < p.G * DIMS; i += kA4Threads) {
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
}

template <int RT>
__global__ void __launch_bounds__(kA4Threads, kA4BlocksPerSM<RT>) k_attend4(const __grid_constant__ AttendParams p)
{
    attend4_block<RT, 0>(p);
}
template <int RT>
__global__ void __launch_bounds__(kA4Threads, 2) k_attend4_cluster(const __grid_constant__ AttendParams p)
{
    attend4_block<RT, kAttCluster>(p);
}

}  // namespace tri
