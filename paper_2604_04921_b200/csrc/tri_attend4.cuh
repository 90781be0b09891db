// Attention of one decode step over a 4-bit cache (tri_row4.cuh).
//
// Mathematics.  As in tri_attend.cuh, with k_n = s_ng (u - 8) + c_ng for the codes u of group g (32 components), and v_n likewise:
//       q . k_n  = sum_g s_ng (sum_d q_d u_nd - 8 Q_g) + sum_g c_ng Q_g,      Q_g = sum of q over group g
//       sum_n p_n v_n = sum_n (p_n s_ng) (u - 8) + sum_n p_n c_ng
// so that the matrix instructions work on codes, and scales and centres are applied per row and group:
//   logits   keys are the 16 rows of A, 8 query rows the columns of B.  A nibble or-ed under 0x4300 is the bf16 value 128 + u: 7
//            integer instructions widen 8 codes, and the 128 + 8 is taken off by the accumulator's initial value, -136 Q_g.  (136 Q_g
//            is rounded at 2^-24 of itself: some 2^-19 of the products' own sum.)  The queries are used as they are.  The centres take
//            one matrix instruction more, bf16 against Q in three bf16 parts.
//   sums     the 16 rows of A are components, its 16 columns cached rows.  A nibble or-ed under 0x6400 is the f16 value 1024 + u (16 u
//            where it lies four bits further up, which saves the shift), and one f16 multiply-add makes u - 8 of it, exactly.  The
//            weights p_n s_ng 2^-E are rounded once to f16; E keeps the largest scale of the rows so far below 1, and p is kept as in
//            tri_attend.cuh, so that they use f16's range from 2^15 down.  The centres are summed in fp32.
//
// What bounds it.  160 bytes per row and head: at HBM speed a multiprocessor gets 16 rows every 60 ns, and the instructions that turn
// 16 x 256 codes into operands have to fit in there.  Copies are 16-byte asynchronous ones into a ring of stages that each warp keeps
// for itself; a stage is 32 rows of K and of V.  Work split, records and parts are those of tri_attend.cuh.
#pragma once
#include "tri_attend.cuh"
#include "tri_row4.cuh"

namespace tri {

constexpr int kA4Warps = kAttWarps, kA4Threads = 32 * kA4Warps, kA4Rows = 32, kA4Stages = 2;
constexpr int kA4Half = kA4Rows * kRow4Bytes, kA4StageBytes = 2 * kA4Half;                  // K | V
constexpr int kA4RingBytes = kA4Warps * kA4Stages * kA4StageBytes;
constexpr int kA4Tile = kA4Warps * kA4Rows;
constexpr int kA4UnitCost = 2;                                   // a unit's own cost, in tiles
template <int RT> constexpr int kA4BlocksPerSM = RT == 8 ? 4 : 2;
static_assert(kA4StageBytes >= 8 * 512, "the sums of a warp fit into a stage");

__device__ __forceinline__ void mma_bf16_from(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1,
                                              float c0, float c1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%10,%11};\n"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1));
}
// (w & mask) | bits, one instruction
template <uint32_t MASK, uint32_t BITS>
__device__ __forceinline__ uint32_t nibbles(uint32_t w)
{
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;\n" : "=r"(r) : "r"(w), "n"(MASK), "r"(BITS));
    return r;
}
__device__ __forceinline__ uint32_t sub_f16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("sub.rn.f16x2 %0, %1, %2;\n" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t fma_f16x2(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;\n" : "=r"(r) : "r"(a), "r"(b), "r"(c));
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
__device__ __forceinline__ uint2 lds64(uint32_t at)
{
    uint2 r;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];\n" : "=r"(r.x), "=r"(r.y) : "r"(at) : "memory");
    return r;
}
__device__ __forceinline__ uint32_t lds32(uint32_t at)
{
    uint32_t r;
    asm volatile("ld.shared.u32 %0, [%1];\n" : "=r"(r) : "r"(at) : "memory");
    return r;
}
__device__ __forceinline__ uint32_t pick(const uint4 &x, int i) { return i == 0 ? x.x : (i == 1 ? x.y : (i == 2 ? x.z : x.w)); }

// RT: query rows, 8 or up to 16 (two column tiles).  CL > 0: a cluster of CL blocks takes one unit, as in tri_attend.cuh.
template <int RT, int CL>
__device__ __forceinline__ void attend4_block(const AttendParams &p)
{
    constexpr int CT = RT / 8, ST = kA4Stages, ROWS = kA4Rows, NK = ROWS / 16, TILE = kA4Tile;
    extern __shared__ __align__(128) uint8_t dyn[];
    __shared__ float2 stat[kA4Warps][RT];
    __shared__ __align__(16) float part[CL ? RT : 1][kAttRowPitch];      // this block's sums, and (m, l)

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g8 = lane >> 2, t4 = lane & 3;
    const uint32_t ring = smem_u32(dyn) + warp * (ST * kA4StageBytes);
    // Cached row of row i of a matrix tile of keys: i / 2 + 4 (i % 2) of 8 (the second 8 rows 8 further on).  Rows 4 apart are 64 bytes
    // apart in the banks: two rows' 64 bytes of codes, one load's phase, take all of them.  The sums over cached rows then take
    // columns 2 t4, 2 t4 + 1 of A from rows t4, t4 + 4.
    const int row_k = (g8 >> 1) + 4 * (g8 & 1);
    const uint32_t klane = row_k * kRow4Bytes, vlane = t4 * kRow4Bytes + 16 * (g8 >> 1);
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
        if (tid < RT) { part[CL ? tid : 0][kHeadDim] = -INFINITY; part[CL ? tid : 0][kHeadDim + 1] = 0.f; }      // no rows so far
    }
    auto next_unit = [&](AttCursor &c, AttJob &u) -> bool {
        if constexpr (CL == 0) {
            return att_next<TILE, kA4UnitCost>(p, sh, c, u);
        } else {
            if (c.rt++ > 0) return false;
            u.seq = c.seq; u.h = c.h; u.nrows = p.G; u.first_seq = c.seq;
            u.len = att_len(p, u.seq, c.h);
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
    uint64_t policy;                                      // rows are read once in a step: first to leave L2
    asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;\n" : "=l"(policy));
    const uint32_t step_row = (uint32_t)(p.src.paged ? p.src.stride_slot : p.src.stride_tok);      // bytes between rows (the host checks)
    auto advance = [&]() {                                // to the next step, its pages looked up before they are needed
        if (pit == pj.kb) {
            do more = next_unit(pc, pj); while (more && pj.kb <= pj.ka);
            pit = pj.ka;
            unit_base = (int64_t)p.layer * p.src.stride_layer + (int64_t)pj.h * p.src.stride_head +
                        (p.src.paged ? 0 : (int64_t)pj.seq * p.src.stride_seq);
        }
        if (more && p.src.paged) {
#pragma unroll
            for (int x = 0; x < NK; ++x) {
                const uint32_t r = (uint32_t)pit * TILE + warp * ROWS + 16 * x;
                const uint32_t pg = p.src.page_shift >= 0 ? r >> p.src.page_shift : r / (uint32_t)p.src.page_size;
                page[x] = r < (uint32_t)pj.len ? ld_here(p.src.page_table + (int64_t)pj.seq * p.src.max_pages_per_seq + pg) : 0;
                slot[x] = (int)(r - pg * (uint32_t)p.src.page_size);
            }
        }
    };
    auto issue = [&]() {
        if (more) {
            const uint32_t dst = ring + pstage * kA4StageBytes + 16 * lane;
            int64_t base[NK];
            int have[NK];
            uint32_t miss = 0;
#pragma unroll
            for (int x = 0; x < NK; ++x) {                // 16 rows each: they lie in one page
                const uint32_t r = (uint32_t)pit * TILE + warp * ROWS + 16 * x;
                have[x] = r < (uint32_t)pj.len ? min(pj.len - (int)r, 16) : 0;
                base[x] = unit_base;
                if (p.src.paged) {
                    base[x] += (int64_t)page[x] * p.src.stride_page + (int64_t)slot[x] * p.src.stride_slot;
                    if (have[x] && p.src.n_pages > 0 && (uint32_t)page[x] >= (uint32_t)p.src.n_pages) {
                        have[x] = 0;
                        miss |= 1u << x;
                        if (lane == 0 && p.device_status) atomicExch(p.device_status, (int)TRI_ERR_DEVICE_CHECK);
                    }
                } else {
                    base[x] += (int64_t)r * p.src.stride_tok;
                }
            }
            // the 160 pieces of a stage's keys, 5 per row, go to the lanes in turn; rows behind the length (or absent ones)
            // arrive as zeros and are not read
#pragma unroll
            for (int i = 0; i < 5; ++i) {
                const int piece = 32 * i + lane, row = piece / 5, col = piece - 5 * row, x = row >> 4;
                const bool there = (row & 15) < have[x == 0 ? 0 : NK - 1];
                const int64_t at = there ? (x == 0 ? base[0] : base[NK - 1]) + (int64_t)((uint64_t)(uint32_t)(row & 15) * step_row) + 16 * col : 0;
                cp_async16(dst + 512 * i, p.src.k + at, there ? 16u : 0u, policy);
                cp_async16(dst + kA4Half + 512 * i, p.src.v + at, there ? 16u : 0u, policy);
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
    uint4 q[CT][4];                                       // components 32 g + 8 t4 .. + 7 of query row g8 (+ 8 ct)
    uint32_t qsum[CT][2];                                 // Q in three bf16 parts, the B operand of the centres
    float from[CT][4][2];                                 // -136 Q_g of query rows 2 t4, 2 t4 + 1
    float o[CT][4][2][4], oc[CT][4][2], m[CT][2], l[CT][2];
    float top = 0.f, down = 1.f;                          // 2^E, no scale of V so far is above it; 2^-E
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
                if (j.kt == 0 && j.begins)                // no rows: zeros
                    for (int i = tid; i < p.G * 16; i += kA4Threads) {
                        const int hq = j.h * p.G + (i >> 4);
                        *reinterpret_cast<uint4 *>(p.out + ((int64_t)j.seq * p.out_seq + (int64_t)hq * p.out_head) * 2 + 16 * (i & 15)) =
                            make_uint4(0u, 0u, 0u, 0u);
                        if (p.lse && (i & 15) == 0) p.lse[(int64_t)j.seq * p.H * p.G + hq] = -INFINITY;
                    }
            }
            if (!rows) break;
            it = j.ka;
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                const int r = g8 + 8 * ct;
                const char *qr = p.q + ((int64_t)j.seq * p.q_seq + (int64_t)(j.h * p.G + r) * p.q_head) * 2 + 16 * t4;
                float sum[4];
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    q[ct][g] = r < p.G ? *reinterpret_cast<const uint4 *>(qr + 64 * g) : make_uint4(0u, 0u, 0u, 0u);
                    const uint4 x = q[ct][g];
                    sum[g] = ((bf16_lo(x.x) + bf16_hi(x.x)) + (bf16_lo(x.y) + bf16_hi(x.y))) + ((bf16_lo(x.z) + bf16_hi(x.z)) + (bf16_lo(x.w) + bf16_hi(x.w)));
                    sum[g] += __shfl_xor_sync(0xffffffffu, sum[g], 1);
                    sum[g] += __shfl_xor_sync(0xffffffffu, sum[g], 2);
#pragma unroll
                    for (int x2 = 0; x2 < 2; ++x2) from[ct][g][x2] = -136.f * __shfl_sync(0xffffffffu, sum[g], (2 * t4 + x2) * 4);
                }
                // slots 2 t4, 2 t4 + 1 of the first 8: groups (0, 1), (2, 3), their high parts, then their middle ones; of the second
                // 8 the low parts, then nothing
                const float a = t4 & 1 ? sum[2] : sum[0], b = t4 & 1 ? sum[3] : sum[1];
                const uint32_t hi = cvt_bf16x2(b, a);
                const float a1 = a - bf16_lo(hi), b1 = b - bf16_hi(hi);
                const uint32_t mid = cvt_bf16x2(b1, a1);
                qsum[ct][0] = t4 < 2 ? hi : mid;
                qsum[ct][1] = t4 < 2 ? cvt_bf16x2(b1 - bf16_hi(mid), a1 - bf16_lo(mid)) : 0u;
#pragma unroll
                for (int g = 0; g < 4; ++g) {
#pragma unroll
                    for (int y = 0; y < 2; ++y) o[ct][g][y][0] = o[ct][g][y][1] = o[ct][g][y][2] = o[ct][g][y][3] = 0.f;
                    oc[ct][g][0] = oc[ct][g][1] = 0.f;
                }
                m[ct][0] = m[ct][1] = -INFINITY;
                l[ct][0] = l[ct][1] = 0.f;
            }
            top = 0.f; down = 1.f;
        }

        // ---------------- one step ----------------
        cp_wait<ST - 1>();
        __syncwarp();
        const uint32_t r0 = (uint32_t)it * TILE + warp * ROWS;
        const int have = r0 < (uint32_t)j.len ? min(j.len - (int)r0, ROWS) : 0;
        const uint32_t miss = (bad >> (2 * stage)) & 3u;
        const bool cut = have < ROWS || miss;
        const uint32_t kb_s = ring + stage * kA4StageBytes, vb_s = kb_s + kA4Half;
        // logits: 16 cached rows x 8 query rows; the thread holds rows g8, g8 + 8 of the tile for query rows 2 t4, 2 t4 + 1
        float w[CT][NK][4];
#pragma unroll
        for (int kg = 0; kg < NK; ++kg) {
            const uint32_t at = kb_s + klane + 16 * kg * kRow4Bytes;
            const uint4 ka = lds128(at + 16 * t4), kb = lds128(at + 8 * kRow4Bytes + 16 * t4);
            const uint2 sa = lds64(at + kRow4Scales), sb = lds64(at + 8 * kRow4Bytes + kRow4Scales);
            const uint32_t ca = lds32(at + kRow4Centres + 4 * (t4 & 1)), cb = lds32(at + 8 * kRow4Bytes + kRow4Centres + 4 * (t4 & 1));
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) mma_bf16_from(w[ct][kg], ca, cb, ca, cb, qsum[ct][0], qsum[ct][1], 0.f, 0.f);
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const uint32_t xa = pick(ka, g), xb = pick(kb, g);
                uint32_t a[4], b[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    a[i] = nibbles<0x000f000fu, 0x43004300u>(xa >> 4 * i);
                    b[i] = nibbles<0x000f000fu, 0x43004300u>(xb >> 4 * i);
                }
                const float s0 = g & 1 ? bf16_hi(g < 2 ? sa.x : sa.y) : bf16_lo(g < 2 ? sa.x : sa.y);
                const float s1 = g & 1 ? bf16_hi(g < 2 ? sb.x : sb.y) : bf16_lo(g < 2 ? sb.x : sb.y);
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    float acc[4];
                    mma_bf16_from(acc, a[0], b[0], a[1], b[1], q[ct][g].x, q[ct][g].y, from[ct][g][0], from[ct][g][1]);
                    mma_bf16_16816_acc(acc, a[2], b[2], a[3], b[3], q[ct][g].z, q[ct][g].w);
                    w[ct][kg][0] = fmaf(s0, acc[0], w[ct][kg][0]); w[ct][kg][1] = fmaf(s0, acc[1], w[ct][kg][1]);
                    w[ct][kg][2] = fmaf(s1, acc[2], w[ct][kg][2]); w[ct][kg][3] = fmaf(s1, acc[3], w[ct][kg][3]);
                }
            }
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    w[ct][kg][x] *= p.scale;
                    if (cut && (16 * kg + row_k + 8 * (x >> 1) >= have || ((miss >> kg) & 1u))) w[ct][kg][x] = -INFINITY;
                }
        }
        // the bounds of weights and scales are looked at by a vote and searched for only when one has to be raised
        uint2 vs[NK][2], vc[NK][2];                       // scales and centres of rows g8, g8 + 8 of V
        uint32_t smax = 0;
#pragma unroll
        for (int kg = 0; kg < NK; ++kg)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const uint32_t at = vb_s + klane + (16 * kg + 8 * x) * kRow4Bytes;
                vs[kg][x] = lds64(at + kRow4Scales);
                vc[kg][x] = lds64(at + kRow4Centres);
                smax = max_bf16x2(smax, max_bf16x2(vs[kg][x].x, vs[kg][x].y));
            }
        float mx[CT][2], sm = fmaxf(bf16_lo(smax), bf16_hi(smax));
        bool raise = sm > top;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                mx[ct][i] = fmaxf(fmaxf(w[ct][0][i], w[ct][0][i + 2]), fmaxf(w[ct][NK - 1][i], w[ct][NK - 1][i + 2]));
                raise = raise || mx[ct][i] > m[ct][i] + kAttAbove<true>;
            }
        if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
            for (int d = 4; d < 32; d *= 2) sm = fmaxf(sm, __shfl_xor_sync(0xffffffffu, sm, d));
            float by_s = 1.f;
            if (sm > top) {                               // (all lanes alike)
                // the power of two above it; scales are 0 or at least 2^-126 and below 2^126
                const uint32_t e = min(__float_as_uint(sm) >> 23, 252u) + 1;
                const float up = __uint_as_float(e << 23);
                by_s = top * __uint_as_float((254u - e) << 23);
                top = up;
                down = __uint_as_float((254u - e) << 23);
            }
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
#pragma unroll
                    for (int d = 4; d < 32; d *= 2) mx[ct][i] = fmaxf(mx[ct][i], __shfl_xor_sync(0xffffffffu, mx[ct][i], d));
                    float by = 1.f;
                    if (mx[ct][i] > m[ct][i] + kAttAbove<true>) {
                        mx[ct][i] -= kAttBelow<true>;
                        by = ex2(m[ct][i] - mx[ct][i]);           // 0 where there was no bound yet
                        m[ct][i] = mx[ct][i];
                        l[ct][i] *= by;
                    }
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        oc[ct][g][i] *= by;
#pragma unroll
                        for (int y = 0; y < 2; ++y) { o[ct][g][y][i] *= by * by_s; o[ct][g][y][i + 2] *= by * by_s; }
                    }
                }
        }
#pragma unroll
        for (int kg = 0; kg < NK; ++kg) {
            // weights, times scales, and transposed into the B operand: 16 cached rows x 8 query rows for each group
            uint32_t pw[CT][4][2];
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                float e[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    e[x] = ex2(w[ct][kg][x] - (m[ct][x & 1] == -INFINITY ? 0.f : m[ct][x & 1]));
                    l[ct][x & 1] += e[x];
                }
#pragma unroll
                for (int g = 0; g < 4; ++g)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const uint32_t s2 = g < 2 ? vs[kg][x].x : vs[kg][x].y, c2 = g < 2 ? vc[kg][x].x : vc[kg][x].y;
                        const float c = g & 1 ? bf16_hi(c2) : bf16_lo(c2);
                        const float s = (g & 1 ? bf16_hi(s2) : bf16_lo(s2)) * down;
                        oc[ct][g][0] = fmaf(e[2 * x], c, oc[ct][g][0]);
                        oc[ct][g][1] = fmaf(e[2 * x + 1], c, oc[ct][g][1]);
                        uint32_t h2;
                        asm("cvt.rn.f16x2.f32 %0, %1, %2;\n" : "=r"(h2) : "f"(e[2 * x + 1] * s), "f"(e[2 * x] * s));
                        pw[ct][g][x] = transpose8x8(h2);
                    }
            }
            const uint32_t at = vb_s + vlane + 16 * kg * kRow4Bytes;
            const uint4 v0 = lds128(at), v1 = lds128(at + 4 * kRow4Bytes), v2 = lds128(at + 8 * kRow4Bytes), v3 = lds128(at + 12 * kRow4Bytes);
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                // four components of rows (t4, t4 + 4) and of rows (t4 + 8, t4 + 12)
                const uint32_t u = __byte_perm(pick(v0, g), pick(v1, g), half), x = __byte_perm(pick(v2, g), pick(v3, g), half);
                const uint32_t u8 = u >> 8, x8 = x >> 8;
                const uint32_t a0 = sub_f16x2(nibbles<0x000f000fu, 0x64006400u>(u), 0x64086408u);                         // 1032
                const uint32_t a1 = fma_f16x2(nibbles<0x00f000f0u, 0x64006400u>(u), 0x2c002c00u, 0xd480d480u);            // 1/16, -72
                const uint32_t a2 = sub_f16x2(nibbles<0x000f000fu, 0x64006400u>(x), 0x64086408u);
                const uint32_t a3 = fma_f16x2(nibbles<0x00f000f0u, 0x64006400u>(x), 0x2c002c00u, 0xd480d480u);
                const uint32_t b0 = sub_f16x2(nibbles<0x000f000fu, 0x64006400u>(u8), 0x64086408u);
                const uint32_t b1 = fma_f16x2(nibbles<0x00f000f0u, 0x64006400u>(u8), 0x2c002c00u, 0xd480d480u);
                const uint32_t b2 = sub_f16x2(nibbles<0x000f000fu, 0x64006400u>(x8), 0x64086408u);
                const uint32_t b3 = fma_f16x2(nibbles<0x00f000f0u, 0x64006400u>(x8), 0x2c002c00u, 0xd480d480u);
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    mma_f16_16816(o[ct][g][0], a0, a1, a2, a3, pw[ct][g][0], pw[ct][g][1]);
                    mma_f16_16816(o[ct][g][1], b0, b1, b2, b3, pw[ct][g][0], pw[ct][g][1]);
                }
            }
        }
        __syncwarp();
        uint8_t *used = dyn + (warp * ST + stage) * kA4StageBytes;
        stage = stage + 1 == ST ? 0 : stage + 1;
        if (++it < j.kb) continue;

        // ---------------- the unit's rows of this share are through: join the warps ----------------
        // per 8 query rows: each leaves its sums in the stage it has just read, fragment by fragment, and takes a group of all
        const bool final = j.complete && p.finish;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
                for (int d = 4; d < 32; d *= 2) {
                    l[ct][i] += __shfl_xor_sync(0xffffffffu, l[ct][i], d);
#pragma unroll
                    for (int g = 0; g < 4; ++g) oc[ct][g][i] += __shfl_xor_sync(0xffffffffu, oc[ct][g][i], d);
                }
                if (g8 == 0) stat[warp][8 * ct + 2 * t4 + i] = make_float2(m[ct][i], l[ct][i]);
            }
#pragma unroll
            for (int g = 0; g < 4; ++g)
#pragma unroll
                for (int y = 0; y < 2; ++y)
                    *reinterpret_cast<float4 *>(used + (2 * g + y) * 512 + lane * 16) =
                        make_float4(fmaf(o[ct][g][y][0], top, oc[ct][g][0]), fmaf(o[ct][g][y][1], top, oc[ct][g][1]),
                                    fmaf(o[ct][g][y][2], top, oc[ct][g][0]), fmaf(o[ct][g][y][3], top, oc[ct][g][1]));
            __syncthreads();
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
                    by[w2][i] = ml.x == -INFINITY ? 0.f : ex2(ml.x - mm[i]);
                    ll[i] += ml.y * by[w2][i];
                }
            }
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int w2 = 0; w2 < kA4Warps; ++w2) {
                    const float4 x = *reinterpret_cast<const float4 *>(used + (w2 - warp) * (ST * kA4StageBytes) + (2 * warp + y) * 512 + lane * 16);
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
                float *to = CL ? part[CL ? r : 0] : p.slots + (((int64_t)blockIdx.x * 2 + (j.begins ? 1 : 0)) * RT + r) * kAttRowPitch;
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
