// Attention of many query rows over a shared prefix on the 5th-generation tensor cores (bf16 rows).
//
// A prefix that n sequences share meets n * G query rows per KV head: up to 128 of them are one M = 128 tile, so every
// cached row fetched from memory serves all of them.  Per tile of 128 cached rows:
//   producer warp    bulk-tensor copies of the K and V rows (boxes of 16 rows x 64 dims, 128-byte swizzle) into rings of
//                    three stages each; K is the K-major, V the N-major B operand as they lie
//   MMA warp         S = Q K^T (8 MMAs 128 x 128 x 16) into tensor memory, and one tile later O += P V with P taken from
//                    tensor memory: the bf16 weights and, in a second sweep, the bf16 of what that rounding left over
//   2 x 4 warps      softmax: each group of four takes every other tile with statistics and an accumulator O of its own
//                    (two independent streams, so the groups never wait for each other); a thread owns one query row,
//                    reads its 128 logits, raises its bound m only when a logit passes it by 2^8 (then O is rescaled in
//                    tensor memory), and writes the weights over the logits
// Tensor memory: S/P of both streams (2 x 128 columns) and O of both (2 x 128), all of its 512 columns.
// At the end of a unit's share the streams are joined and the part goes to the workspace, as in k_attend.
//
// What bounds it: with up to 128 rows per prefix, HBM (64 KB per 1.5 us and SM); the MMAs of a tile take 1536 cycles, the
// exponentials 1024, against about 2800 cycles for its rows.  With more rows the tiles of one prefix share its rows
// through L2 and the MMAs bound it.
//
// Every wait is bounded; one that runs out sets TRI_ERR_TIMEOUT, all roles leave their loops and the tensor memory is
// released at the common exit.
#pragma once
#include "tri_attend.cuh"
#include "tri_score_umma.cuh"

namespace tri {

constexpr int kPTile = 128;                               // cached rows per tile, query rows per tile
constexpr int kPStages = 3;
constexpr int kPBlock = kPTile * 128;                     // 128 rows x 64 bf16, one swizzled block
constexpr int kPTileBytes = 2 * kPBlock;                  // dims 0..63 | dims 64..127
constexpr int kPSoftWarps = 8;
constexpr int kPThreads = (kPSoftWarps + 2) * 32;
constexpr int kPDynSmem = (1 + 2 * kPStages) * kPTileBytes + 1024;      // Q, K ring, V ring

// V as the B operand: N (dims) contiguous, 64-element chunks one block apart, groups of 8 cached rows 1024 bytes apart.
__device__ __forceinline__ uint64_t tc_desc_sw128_n(uint32_t smem_addr)
{
    return (uint64_t)((smem_addr >> 4) & 0x3fffu) | ((uint64_t)(kPBlock >> 4) << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ void tc_ld32(uint32_t taddr, uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,"
        "%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr));
}
__device__ __forceinline__ void tc_ld16(uint32_t taddr, uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr));
}
__device__ __forceinline__ void tc_st16(uint32_t taddr, const uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};\n" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tc_ld2(uint32_t taddr, uint32_t (&r)[2])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x2.b32 {%0,%1}, [%2];\n" : "=r"(r[0]), "=r"(r[1]) : "r"(taddr));
}
__device__ __forceinline__ void tc_st2(uint32_t taddr, float a, float b)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x2.b32 [%0], {%1,%2};\n" ::"r"(taddr), "f"(a), "f"(b) : "memory");
}
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory"); }
// Registers a tensor-memory load fills may be read only behind the wait: this keeps the compiler from moving a use before it.
template <int N>
__device__ __forceinline__ void tc_loaded(uint32_t (&r)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+r"(r[i]));
}
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;\n" ::: "memory"); }

struct PrefixBars {
    uint64_t kfull[kPStages], kempty[kPStages], vfull[kPStages], vempty[kPStages];
    uint64_t sfull[2], pready[2], pvdone[2], q, ml;
};

__global__ void __launch_bounds__(kPThreads, 1)
k_attend_prefix(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap, const AttendParams p)
{
    extern __shared__ uint8_t dyn[];
    __shared__ __align__(8) PrefixBars bars;
    __shared__ uint32_t tmem_base_s;
    __shared__ volatile int gave_up;
    __shared__ uint32_t absent[kPStages];                  // per stage: boxes of 16 rows whose page id is out of range

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const AttShare sh = att_share(p, kPTile);
    if ((int)blockIdx.x >= sh.blocks) return;

    const uint32_t base = (smem_u32(dyn) + 1023u) & ~1023u;
    const uint32_t sm_q = base, sm_k = base + kPTileBytes, sm_v = sm_k + kPStages * kPTileBytes;
    uint8_t *gq = dyn + (base - smem_u32(dyn)), *gv = gq + (1 + kPStages) * kPTileBytes;
    const uint32_t b_kfull = smem_u32(bars.kfull), b_kempty = smem_u32(bars.kempty), b_vfull = smem_u32(bars.vfull),
                   b_vempty = smem_u32(bars.vempty), b_sfull = smem_u32(bars.sfull), b_pready = smem_u32(bars.pready),
                   b_pvdone = smem_u32(bars.pvdone), b_q = smem_u32(&bars.q), b_ml = smem_u32(&bars.ml);
    if (tid == 0) {
        for (int i = 0; i < kPStages; ++i) {
            mbar_init(b_kfull + 8 * i, 1); mbar_init(b_kempty + 8 * i, 1);
            mbar_init(b_vfull + 8 * i, 1); mbar_init(b_vempty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(b_sfull + 8 * i, 1);
            mbar_init(b_pready + 8 * i, kPSoftWarps / 2);
            mbar_init(b_pvdone + 8 * i, 1);
        }
        mbar_init(b_q, kPSoftWarps);
        mbar_init(b_ml, kPSoftWarps);
        gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    if (warp == kPSoftWarps + 1) {                         // the MMA warp owns the tensor-memory allocation
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(&tmem_base_s)), "r"(512)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_base_s;
    // columns: S/P of stream w at 128 w (weights: 64 columns, their rest: 64), O of stream w at 256 + 128 w

    AttCursor cur = {sh.unit, 0, sh.start};
    AttJob j;
    int done = 0;                                          // tiles of all earlier units of this block

    if (warp == kPSoftWarps) {
        // ---------------- producer: lane = (matrix, box of 16 rows, half) is 2 x 16 x 1: K on lanes 0..15, V on 16..31 ----------
        const int sub = (lane & 15) >> 1, half = lane & 1;
        const bool is_v = lane >= 16;
        while (!gave_up && att_next(p, sh, kPTile, cur, j)) {
            const int n = j.kb - j.ka;
            auto locate = [&](int t, int &c1, int &c3) -> bool {          // false: the box's page id is out of range
                const int64_t row = (int64_t)(j.ka + t) * kPTile + sub * kTileKeys;
                c1 = (int)row; c3 = j.seq;
                if (!p.src.paged || t >= n || row >= j.len) return true;
                const int pg = p.src.page_shift >= 0 ? (int)row >> p.src.page_shift : (int)row / p.src.page_size;
                c3 = __ldg(p.src.page_table + (int64_t)j.seq * p.src.max_pages_per_seq + pg);
                c1 = (int)row - pg * p.src.page_size;
                return p.src.n_pages <= 0 || (c3 >= 0 && c3 < p.src.n_pages);
            };
            int c1 = 0, c3 = 0;
            bool ok = locate(0, c1, c3);
            for (int t = 0; t < n; ++t) {
                const int i = done + t, st = i % kPStages;
                const uint32_t par = ((i / kPStages) - 1) & 1;
                const int64_t row0 = (int64_t)(j.ka + t) * kPTile;
                const int nsub = (int)min((int64_t)(kPTile / kTileKeys), (j.len - row0 + kTileKeys - 1) / kTileKeys);
                const uint32_t bad = __ballot_sync(0xffffffffu, !ok && sub < nsub && half == 0 && !is_v);
                uint32_t mask = 0;
                for (int x = 0; x < kPTile / kTileKeys; ++x) mask |= ((bad >> (2 * x)) & 1u) << x;
                if (mask && lane == 0 && p.device_status) atomicExch(p.device_status, (int)TRI_ERR_DEVICE_CHECK);
                const uint32_t bytes = (uint32_t)(nsub - __popc(mask)) * kTileBytes;
                const bool mine = sub < nsub && ok;
                // K first: its stage frees as soon as the logits of three tiles before are done
                bool w = i < kPStages || mbar_wait_parked<20>(b_kempty + 8 * st, par);
                if (!__all_sync(0xffffffffu, w)) { gave_up = 1; break; }
                if (lane == 0) mbar_expect_tx(b_kfull + 8 * st, bytes);
                __syncwarp();
                if (!is_v && mine)
                    tma_load_5d(sm_k + st * kPTileBytes + half * kPBlock + sub * (kTileKeys * 128), &kmap, b_kfull + 8 * st,
                                half * (kHeadDim / 2), c1, j.h, c3, p.layer);
                w = i < kPStages || mbar_wait_parked<20>(b_vempty + 8 * st, par);
                if (!__all_sync(0xffffffffu, w)) { gave_up = 1; break; }
                if (lane == 0) { absent[st] = mask; mbar_expect_tx(b_vfull + 8 * st, bytes); }
                __syncwarp();
                if (is_v && mine)
                    tma_load_5d(sm_v + st * kPTileBytes + half * kPBlock + sub * (kTileKeys * 128), &vmap, b_vfull + 8 * st,
                                half * (kHeadDim / 2), c1, j.h, c3, p.layer);
                ok = locate(t + 1, c1, c3);
            }
            done += n;
        }
    } else if (warp == kPSoftWarps + 1) {
        // ---------------- MMA issue ----------------
        constexpr uint32_t idesc_qk = tc_idesc_bf16(kPTile);                     // both operands K-major
        constexpr uint32_t idesc_pv = tc_idesc_bf16(kHeadDim) | (1u << 16);      // B (the values) N-major
        int units = 0, cnt[2] = {0, 0};                    // tiles each stream had in earlier units
        while (!gave_up && att_next(p, sh, kPTile, cur, j)) {
            const int n = j.kb - j.ka;
            if (n == 0) continue;
            bool ok = __all_sync(0xffffffffu, mbar_wait_bounded(b_q, units & 1));
            for (int t = -1; t < n && ok; ++t) {
                if (t + 1 < n) {
                    // logits of tile t + 1; their columns were last read by the MMAs of tile t - 1, issued before these
                    const int i = done + t + 1, st = i % kPStages;
                    ok = __all_sync(0xffffffffu, mbar_wait_bounded(b_kfull + 8 * st, (i / kPStages) & 1));
                    if (!ok) break;
                    tc_fence_after();
                    if (lane == 0) {
                        const uint32_t ka = sm_k + st * kPTileBytes, acc = tmem + 128 * ((t + 1) & 1);
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            tc_mma_bf16(acc, tc_desc_sw128(sm_q + (k >> 2) * kPBlock + (k & 3) * 32),
                                        tc_desc_sw128(ka + (k >> 2) * kPBlock + (k & 3) * 32), idesc_qk, k > 0);
                        tc_commit(b_kempty + 8 * st);
                        tc_commit(b_sfull + 8 * ((t + 1) & 1));
                    }
                    __syncwarp();
                }
                if (t < 0) continue;
                // weights of tile t times its values
                const int i = done + t, st = i % kPStages, w = t & 1;
                ok = mbar_wait_bounded(b_vfull + 8 * st, (i / kPStages) & 1) &&
                     mbar_wait_bounded(b_pready + 8 * w, (cnt[w] + (t >> 1)) & 1);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                if (lane == 0) {
                    const uint32_t va = sm_v + st * kPTileBytes, acc = tmem + 256 + 128 * w, pw = tmem + 128 * w;
#pragma unroll
                    for (int k = 0; k < 16; ++k)           // 8 steps of 16 rows with the weights, 8 with their rest
                        tc_mma_bf16_ts(acc, pw + 32 * ((k & 7) >> 1) + 8 * (k & 1) + 2 * (k & 8), tc_desc_sw128_n(va + (k & 7) * 2048), idesc_pv, t >= 2 || k > 0);
                    tc_commit(b_vempty + 8 * st);
                    tc_commit(b_pvdone + 8 * w);
                }
                __syncwarp();
            }
            done += n;
            cnt[0] += (n + 1) >> 1;
            cnt[1] += n >> 1;
            ++units;
            if (!ok) { gave_up = 1; break; }
        }
    } else {
        // ---------------- softmax: stream w takes tiles w, w + 2, ..; this thread owns query row `row` of its stream ----------
        const int w = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16, t_s = tmem + lane_base + 128 * w, t_o = tmem + lane_base + 256;
        const uint32_t flip = p.scale < 0.f ? 0x80008000u : 0u;            // a negative scale goes into the queries' signs
        const bool check_pages = p.src.paged && p.src.n_pages > 0;
        int units = 0, cnt[2] = {0, 0};
        while (!gave_up && att_next(p, sh, kPTile, cur, j)) {
            if (j.begins && tid == 0) p.rec[j.rec] = j.record;
            const int n = j.kb - j.ka;
            if (n == 0) continue;
            for (int i = tid; i < kPTile * 16; i += kPSoftWarps * 32) {
                const int r = i >> 4, c = i & 15;
                uint4 x = make_uint4(0u, 0u, 0u, 0u);
                if (r < j.nrows) {
                    const int sq = j.first_seq + r / p.G, g = r % p.G;
                    x = *reinterpret_cast<const uint4 *>(p.q + ((int64_t)sq * p.q_seq + (int64_t)(j.h * p.G + g) * p.q_head) * 2 + 16 * c);
                    x.x ^= flip; x.y ^= flip; x.z ^= flip; x.w ^= flip;
                }
                *reinterpret_cast<uint4 *>(gq + (c >> 3) * kPBlock + sw128(r, c & 7)) = x;
            }
            asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
            tc_fence_before();                             // the last unit's accumulators have been read
            __syncwarp();
            if (lane == 0) mbar_arrive(b_q);

            // base-2 logit = accumulator * mul (not 0: a masked logit is -infinity)
            const float mul = fmaxf(fabsf(p.scale) * (p.k_scale ? __ldg(p.k_scale + j.h) : 1.f), 1.17549435e-38f);
            float m = -INFINITY, l = 0.f;
            bool ok = true;
            for (int t = w; t < n; t += 2) {
                const int i = done + t, st = i % kPStages;
                const int64_t left = j.len - (int64_t)(j.ka + t) * kPTile;
                const int have = left < kPTile ? (int)left : kPTile;
                ok = mbar_wait_bounded(b_sfull + 8 * w, (cnt[w] + (t >> 1)) & 1);
                if (have < kPTile || check_pages) ok = ok && mbar_wait_bounded(b_vfull + 8 * st, (i / kPStages) & 1);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                const uint32_t miss = check_pages ? absent[st] : 0u;
                tc_fence_after();
                if (have < kPTile || miss) {
                    // rows behind the length or of absent pages: no weight, and zeros for values (they may hold anything)
                    if (row >= have || ((miss >> (row >> 4)) & 1u)) {
#pragma unroll
                        for (int c = 0; c < 16; ++c)
                            *reinterpret_cast<uint4 *>(gv + st * kPTileBytes + (c >> 3) * kPBlock + row * 128 + (c & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                    }
                    asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
                }
                // 32 logits of the row at a time: the maximum over all four chunks first, the last two stay in registers
                auto chunk = [&](int c, uint32_t (&r)[32]) {
                    tc_wait_ld();
                    tc_loaded(r);
                    if (have < kPTile || miss) {
#pragma unroll
                        for (int x = 0; x < 32; ++x)
                            if (32 * c + x >= have || ((miss >> (2 * c + (x >> 4))) & 1u)) r[x] = 0xff800000u;
                    }
                };
                auto largest = [&](const uint32_t (&r)[32], float top) {
#pragma unroll
                    for (int x = 0; x < 32; ++x) top = fmaxf(top, __uint_as_float(r[x]));
                    return top;
                };
                uint32_t sa[32], sb[32];
                tc_ld32(t_s, sa);
                tc_ld32(t_s + 32, sb);
                chunk(0, sa);
                float top = largest(sa, -INFINITY);
                tc_ld32(t_s + 64, sa);
                tc_loaded(sb);
                if (have < kPTile || miss) chunk(1, sb);
                top = largest(sb, top);
                tc_ld32(t_s + 96, sb);
                chunk(2, sa);
                top = largest(sa, top);
                tc_loaded(sb);
                if (have < kPTile || miss) chunk(3, sb);
                top = largest(sb, top);
                top *= mul;
                const bool raise = top > m + kAttLazy || (m == -INFINITY && top > m);
                if (__any_sync(0xffffffffu, raise)) {
                    const float by = raise ? ex2(m - top) : 1.f;
                    if (raise) m = top;
                    l *= by;
                    if (t >= 2) {                          // an accumulator exists: wait until it rests, then rescale it
                        ok = __all_sync(0xffffffffu, mbar_wait_bounded(b_pvdone + 8 * w, (cnt[w] + (t >> 1) - 1) & 1));
                        if (!ok) break;
                        tc_fence_after();
#pragma unroll 1
                        for (int c = 0; c < 8; ++c) {
                            uint32_t o[16];
                            tc_ld16(t_o + 128 * w + 16 * c, o);
                            tc_wait_ld();
                            tc_loaded(o);
#pragma unroll
                            for (int x = 0; x < 16; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * by);
                            tc_st16(t_o + 128 * w + 16 * c, o);
                        }
                    }
                }
                const float ref = m == -INFINITY ? 0.f : m;
                auto emit = [&](int c, const uint32_t (&r)[32]) {       // weights over the logits: 16 columns of bf16 pairs, 16 of their rest
                    uint32_t hi[16], lo[16];
#pragma unroll
                    for (int x = 0; x < 16; ++x) {
                        const float a = ex2(fmaf(__uint_as_float(r[2 * x]), mul, -ref));
                        const float b = ex2(fmaf(__uint_as_float(r[2 * x + 1]), mul, -ref));
                        l += a + b;
                        split16<false>(a, b, hi[x], lo[x]);
                    }
                    tc_st16(t_s + 32 * c, hi);
                    tc_st16(t_s + 32 * c + 16, lo);
                };
                emit(2, sa);
                tc_ld32(t_s, sa);
                emit(3, sb);
                tc_ld32(t_s + 32, sb);
                chunk(0, sa);
                emit(0, sa);
                tc_loaded(sb);
                if (have < kPTile || miss) chunk(1, sb);
                emit(1, sb);
                tc_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(b_pready + 8 * w);
            }
            done += n;
            cnt[0] += (n + 1) >> 1;
            cnt[1] += n >> 1;
            // ---------------- join the two streams ----------------
            // own stream first: the MMAs complete in order, so the other's barrier is then at most one phase behind its last
            // (a parity wait cannot tell a phase from the one two before it)
            for (int x = 0; x < 2 && ok; ++x) {
                const int y = x == 0 ? w : 1 - w;
                if (y == 0 || n >= 2) ok = mbar_wait_bounded(b_pvdone + 8 * y, (cnt[y] - 1) & 1);
            }
            // (the columns of S and P are idle until the next unit's queries are announced: m and l pass through them)
            ok = __all_sync(0xffffffffu, ok);
            if (ok) {
                tc_fence_after();
                tc_st2(t_s, m, l);
                tc_wait_st();
                tc_fence_before();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(b_ml);
            ok = __all_sync(0xffffffffu, ok && mbar_wait_bounded(b_ml, units & 1));
            if (!ok) { gave_up = 1; break; }
            tc_fence_after();
            uint32_t s0[2], s1[2];
            tc_ld2(tmem + lane_base, s0);
            tc_ld2(tmem + lane_base + 128, s1);
            tc_wait_ld();
            tc_loaded(s0);
            tc_loaded(s1);
            const float m0 = __uint_as_float(s0[0]), m1 = __uint_as_float(s1[0]), mm = fmaxf(m0, m1);
            const float f0 = m0 == -INFINITY ? 0.f : ex2(m0 - mm), f1 = m1 == -INFINITY ? 0.f : ex2(m1 - mm);
            const bool mine = row < j.nrows;
            const int sq = j.first_seq + (mine ? row : 0) / p.G, hq = j.h * p.G + row % p.G;
            float *to = j.complete ? p.whole + ((int64_t)sq * p.H * p.G + hq) * kAttRowPitch
                                   : p.slots + (((int64_t)blockIdx.x * 2 + (j.begins ? 1 : 0)) * kPTile + row) * kAttRowPitch;
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {                  // this group's half of the dims, 16 at a time
                uint32_t a[16], b[16];
                tc_ld16(t_o + 64 * w + 16 * c, a);
                if (n >= 2) tc_ld16(t_o + 128 + 64 * w + 16 * c, b);
                tc_wait_ld();
                tc_loaded(a);
                if (n >= 2) tc_loaded(b);
                float y[16];
#pragma unroll
                for (int x = 0; x < 16; ++x) y[x] = __uint_as_float(a[x]) * f0 + (n >= 2 ? __uint_as_float(b[x]) * f1 : 0.f);
                if (mine) {
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        *reinterpret_cast<float4 *>(to + 64 * w + 16 * c + 4 * x) = make_float4(y[4 * x], y[4 * x + 1], y[4 * x + 2], y[4 * x + 3]);
                }
            }
            if (mine && w == 0) *reinterpret_cast<float2 *>(to + kHeadDim) = make_float2(mm, __uint_as_float(s0[1]) * f0 + __uint_as_float(s1[1]) * f1);
            ++units;
        }
    }

    tc_fence_before();
    __syncthreads();
    if (gave_up) {
        // a wait ran out: report it, and give copies still in flight one more bounded chance to land before the block exits
        if (tid == 0 && p.device_status) atomicExch(p.device_status, (int)TRI_ERR_TIMEOUT);
        if (warp == kPSoftWarps)
            for (int i = 0; i < 2 * kPStages; ++i) {
                (void)mbar_wait_parked(b_kfull + 8 * (i % kPStages), (i / kPStages) & 1);
                (void)mbar_wait_parked(b_vfull + 8 * (i % kPStages), (i / kPStages) & 1);
            }
    }
    if (warp == kPSoftWarps + 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(512) : "memory");
    }
}

}  // namespace tri
