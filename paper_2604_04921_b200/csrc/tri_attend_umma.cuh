// Attention of many query rows over a shared prefix on the 5th-generation tensor cores.
//
// A prefix that n sequences share meets n * G query rows per KV head: up to 128 of them are one M = 128 tile, so every
// cached row fetched from memory serves all of them.  Per tile of 128 cached rows:
//   producer warps   bulk-tensor copies of the K and V rows (boxes of 16..128 rows x 64 dims, 128-byte swizzle) into rings
//                    of three stages each; K is the K-major, V the N-major B operand as they lie
//   MMA warp         S = Q K^T (8 MMAs 128 x 128 x 16) into tensor memory, and one tile later O += P V with P taken from
//                    tensor memory, bf16
//   2 x 4 warps      softmax: each group of four takes every other tile with statistics and an accumulator O of its own
//                    (two independent streams, so the groups never wait for each other); a thread owns one query row,
//                    reads its 128 logits, raises its bound m only when a weight would pass 2^8 (then O is rescaled in
//                    tensor memory), and writes the weights over the logits
// Tensor memory: S/P of both streams (2 x 128 columns) and O of both (2 x 128), all of its 512 columns.
// 8-bit rows: the producers' two warps per matrix widen the raw e4m3 rows to f16 on their way into the operand stages, and
// the MMAs are f16 (queries scaled to f16 by a power of two per row, weights with 11 bits).
// At the end of a unit's share the streams are joined and the part goes to the workspace, as in k_attend.
//
// What bounds it: with up to 128 query rows per prefix, HBM: a tile's 64 KB take about 2800 cycles per multiprocessor, its
// MMAs 1024 (as issued, one by one, 1600), the exponentials 1024.  One prefix of 256K rows, 128 query rows per head: 6.7 TB/s.
// With more query rows the tiles of one prefix share its rows through L2 and the issue of the MMAs bounds it.  Start, drain
// and join cost about 15 us, which is what counts on short prefixes.
// 8-bit rows are half the bytes but take as long (whole calls: 32 sequences on 32K rows 69.8 us, bf16 68.1; 64 on six prompts
// 113.9, bf16 109.4): HBM does not bound them.  Not taken apart; the two converting warps per matrix stand between the copies
// and the MMAs, and the MMAs as issued alone need more than the rows' 1400 cycles.
//
// Weights are rounded once, to bf16 (8-bit rows: f16), and the sum that divides is that of the rounded ones, which cancels the
// part of the error that all rows share.  Error of the outputs against 64 bits, relative, where one rounding of the output makes
// 1.65e-3: 1.68e-3 for values around a common centre of half their spread, 2.2e-3 to 2.4e-3 for values without one (1.8e-3 to
// 2.0e-3 where few rows have the weight); 8-bit rows 1.67e-3.  The rest of a weight in a second MMA would take this off; it made
// the MMAs 25 % longer.
//
// Every wait is bounded; one that runs out sets TRI_ERR_TIMEOUT, all roles leave their loops and the tensor memory is
// released at the common exit.
#pragma once
#include "tri_attend.cuh"
#include "tri_score_umma.cuh"

namespace tri {

constexpr int kPTile = 128;                               // cached rows per tile, query rows per tile
constexpr int kPHalf = 64;                                // the weights of a tile are handed over in two halves, so that MMAs and softmax overlap
template <bool KEY8> constexpr int kPStages = KEY8 ? 2 : 3;     // operand stages of K and of V
constexpr int kPUnitCost = 2;                             // a unit's own cost, in tiles
static_assert(kPTile == kMergeTile, "slots are laid out for the joining kernel");
constexpr int kPBlock = kPTile * 128;                     // 128 rows x 64 bf16, one swizzled block
constexpr int kPTileBytes = 2 * kPBlock;                  // dims 0..63 | dims 64..127
constexpr int kPSoftWarps = 8;
template <bool KEY8> constexpr int kPMoveWarps = KEY8 ? 4 : 2;    // producers (8 bits: and converters) of K, of V; then the MMA warp
template <bool KEY8> constexpr int kPThreads = (kPSoftWarps + kPMoveWarps<KEY8> + 1) * 32;
constexpr int kPRawBytes = kPTile * 128;                  // 128 rows of 128 e4m3 values
constexpr int kPDynSmem = 7 * kPTileBytes + 1024;         // Q, K and V stages; 8 bits: two stages of raw rows each in place of one of them

// V as the B operand: N (dims) contiguous, 64-element chunks one block apart, groups of 8 cached rows 1024 bytes apart.
__device__ __forceinline__ uint64_t tc_desc_sw128_n(uint32_t smem_addr)
{
    return (uint64_t)((smem_addr >> 4) & 0x3fffu) | ((uint64_t)(kPBlock >> 4) << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ void tc_ld64(uint32_t taddr, uint32_t (&r)[64])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x64.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,"
        "%24,%25,%26,%27,%28,%29,%30,%31,%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,"
        "%48,%49,%50,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63}, [%64];\n"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]),
          "=r"(r[32]), "=r"(r[33]), "=r"(r[34]), "=r"(r[35]), "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]),
          "=r"(r[40]), "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]), "=r"(r[45]), "=r"(r[46]), "=r"(r[47]),
          "=r"(r[48]), "=r"(r[49]), "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]), "=r"(r[54]), "=r"(r[55]),
          "=r"(r[56]), "=r"(r[57]), "=r"(r[58]), "=r"(r[59]), "=r"(r[60]), "=r"(r[61]), "=r"(r[62]), "=r"(r[63])
        : "r"(taddr));
}
__device__ __forceinline__ void tc_st64(uint32_t taddr, const uint32_t (&r)[64])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x64.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,"
        "%24,%25,%26,%27,%28,%29,%30,%31,%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,"
        "%47,%48,%49,%50,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63,%64};\n" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
        "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
        "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]),
        "r"(r[32]), "r"(r[33]), "r"(r[34]), "r"(r[35]), "r"(r[36]), "r"(r[37]), "r"(r[38]), "r"(r[39]),
        "r"(r[40]), "r"(r[41]), "r"(r[42]), "r"(r[43]), "r"(r[44]), "r"(r[45]), "r"(r[46]), "r"(r[47]),
        "r"(r[48]), "r"(r[49]), "r"(r[50]), "r"(r[51]), "r"(r[52]), "r"(r[53]), "r"(r[54]), "r"(r[55]),
        "r"(r[56]), "r"(r[57]), "r"(r[58]), "r"(r[59]), "r"(r[60]), "r"(r[61]), "r"(r[62]), "r"(r[63])
        : "memory");
}
// Two fp32 operations in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 d;
    asm("{\n.reg .b64 a, b, c, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmov.b64 c, {%6, %7};\nfma.rn.f32x2 d, a, b, c;\n"
        "mov.b64 {%0, %1}, d;\n}\n" : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 d;
    asm("{\n.reg .b64 a, b, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nadd.rn.f32x2 d, a, b;\nmov.b64 {%0, %1}, d;\n}\n"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
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
__device__ __forceinline__ void tc_ld4(uint32_t taddr, uint32_t (&r)[4])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0,%1,%2,%3}, [%4];\n" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(taddr));
}
__device__ __forceinline__ void tc_st4f(uint32_t taddr, float a, float b, float c)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1,%2,%3,%3};\n" ::"r"(taddr), "f"(a), "f"(b), "f"(c) : "memory");
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
    uint64_t kfull[3], kempty[3], vfull[3], vempty[3];
    uint64_t sfull[2], pready[4], q, ml;                  // per stream; per (stream, half of a tile's rows); block
    uint64_t rawfull[4], rawfree[4];                      // 8 bits: two stages of raw K, two of raw V
};
// Instruction descriptor of an f16 or bf16 MMA with M = 128, both operands K-major.
__host__ __device__ constexpr uint32_t tc_idesc_16(bool f16, int ncol) { return f16 ? tc_idesc_bf16(ncol) & ~((1u << 7) | (1u << 10)) : tc_idesc_bf16(ncol); }

template <bool KEY8>
__global__ void __launch_bounds__(kPThreads<KEY8>, 1)
k_attend_prefix(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap, const AttendParams p)
{
    extern __shared__ uint8_t dyn[];
    __shared__ __align__(8) PrefixBars bars;
    __shared__ uint32_t tmem_base_s;
    __shared__ volatile int gave_up;
    __shared__ uint32_t absent[3], absent_raw[2];          // per stage: groups of 16 rows whose page id is out of range
    __shared__ float qscale_s[KEY8 ? kPTile : 1];          // 8 bits: power of two a query row was divided by
    constexpr int ST = kPStages<KEY8>, kMmaWarp = kPSoftWarps + kPMoveWarps<KEY8>;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    grid_dependency_wait();                                // set up under the kernel before it in the stream
    grid_dependents_launch();                              // the pass over the sequences' own rows may start as blocks leave
    const uint32_t base = (smem_u32(dyn) + 1023u) & ~1023u;
    const uint32_t sm_q = base, sm_k = base + kPTileBytes, sm_v = sm_k + ST * kPTileBytes;
    uint8_t *gq = dyn + (base - smem_u32(dyn)), *gv = gq + (1 + ST) * kPTileBytes;
    const uint32_t b_kfull = smem_u32(bars.kfull), b_kempty = smem_u32(bars.kempty), b_vfull = smem_u32(bars.vfull),
                   b_vempty = smem_u32(bars.vempty), b_sfull = smem_u32(bars.sfull), b_pready = smem_u32(bars.pready),
                   b_q = smem_u32(&bars.q), b_ml = smem_u32(&bars.ml);
    if (tid == 0) {
        for (int i = 0; i < ST; ++i) {
            mbar_init(b_kfull + 8 * i, KEY8 ? 2 : 1); mbar_init(b_kempty + 8 * i, 1);       // filled by a copy, or by two converter warps
            mbar_init(b_vfull + 8 * i, KEY8 ? 2 : 1); mbar_init(b_vempty + 8 * i, 1);
        }
        if (KEY8)
            for (int i = 0; i < 4; ++i) { mbar_init(smem_u32(&bars.rawfull[i]), 1); mbar_init(smem_u32(&bars.rawfree[i]), 2); }
        for (int i = 0; i < 2; ++i) mbar_init(b_sfull + 8 * i, 1);
        for (int i = 0; i < 4; ++i) mbar_init(b_pready + 8 * i, kPSoftWarps / 2);
        mbar_init(b_q, kPSoftWarps);
        mbar_init(b_ml, kPSoftWarps);
        gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    // (the barriers are set up before its synchronisations, so that the producers may begin behind it)
    const AttShare sh = att_share<kPTile, kPUnitCost>(p);
    if ((int)blockIdx.x >= sh.shares || sh.total == 0) return;

    if (warp == kMmaWarp) {                                // the MMA warp owns the tensor-memory allocation
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(&tmem_base_s)), "r"(512)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    }
    AttCursor cur = {sh.seq, sh.h, 0, sh.start};
    AttJob j;
    int done = 0;                                          // tiles of all earlier units of this block
    const int inv_g = 65536 / p.G + 1;
    auto query_row = [&](const AttJob &u, int r) -> const char * {
        const int sr = att_small_div(r, inv_g);
        return p.q + ((int64_t)(u.first_seq + sr) * p.q_seq + (int64_t)(u.h * p.G + r - sr * p.G) * p.q_head) * 2;
    };
    // a unit's queries into L2, one 128-byte line per thread of the softmax warps: asked for behind 200 KB of copies in flight
    // they would take microseconds
    auto prefetch_queries = [&](const AttJob &u) {
        if ((tid >> 1) < u.nrows) asm volatile("prefetch.global.L2 [%0];\n" ::"l"(query_row(u, tid >> 1) + (tid & 1) * 128));
    };
    // the next unit of the share that has rows here; `records`: of those passed over or found, where they begin here
    auto next_rows = [&](bool records) -> bool {
        while (att_next<kPTile, kPUnitCost>(p, sh, cur, j)) {
            if (records && j.begins) p.rec[j.rec] = att_record(sh, j);
            if (j.kb > j.ka) return true;
        }
        return false;
    };
    bool more = false;
    if (warp < kPSoftWarps) {
        more = next_rows(tid == 0);
        if (more) prefetch_queries(j);
    }
    // tensor memory is there; the producers have no part in it and are at work
    if (warp < kPSoftWarps || warp == kMmaWarp) {
        tc_fence_before();
        asm volatile("bar.sync 2, %0;\n" ::"n"(32 * (kPSoftWarps + 1)) : "memory");
        tc_fence_after();
    }
    const uint32_t tmem = tmem_base_s;
    // columns: S of stream w at 128 w, P of its halves in the first 32 columns of either half, O of stream w at 256 + 128 w

    if (KEY8 && warp >= kPSoftWarps && warp < kMmaWarp) {
        // ---------------- 8 bits: two warps for K, two for V; the first of a pair issues the copies of raw rows two tiles ahead,
        // each widens half of a tile's rows to f16 into the operand's stage (rows behind the length or absent become zeros) ----
        const bool is_v = warp >= kPSoftWarps + 2, lead = ((warp - kPSoftWarps) & 1) == 0;
        const uint32_t b_full = is_v ? b_vfull : b_kfull, b_empty = is_v ? b_vempty : b_kempty;
        const uint32_t b_raw = smem_u32(&bars.rawfull[is_v ? 2 : 0]), b_free = smem_u32(&bars.rawfree[is_v ? 2 : 0]);
        uint8_t *g_raw = gq + (1 + 2 * ST) * kPTileBytes + (is_v ? 2 * kPRawBytes : 0), *g_out = gq + (1 + (is_v ? ST : 0)) * kPTileBytes;
        const uint32_t raw = smem_u32(g_raw);
        const CUtensorMap *map = is_v ? &vmap : &kmap;
        const int box = p.box_rows, boxes = kPTile / box;
        AttCursor ahead = cur;
        AttJob a;                                          // the unit whose rows are being asked for
        int at = 0, asked = 0;
        auto next_asked = [&]() -> bool {
            while (att_next<kPTile, kPUnitCost>(p, sh, ahead, a))
                if (a.kb > a.ka) return true;
            return false;
        };
        bool open = lead && next_asked();
        auto ask = [&]() -> bool {                         // raw rows of the share's next tile
            if (!open) return true;
            const int st = asked & 1;
            if (asked >= 2 && !__all_sync(0xffffffffu, mbar_wait_parked<20>(b_free + 8 * st, ((asked >> 1) - 1) & 1))) return false;
            const int64_t row = (int64_t)(a.ka + at) * kPTile + lane * box, left = a.len - (int64_t)(a.ka + at) * kPTile;
            const int nsub = left >= kPTile ? boxes : (int)((left + box - 1) / box);
            int c1 = (int)row, c3 = a.seq;
            bool ok = true;
            if (p.src.paged && lane < nsub) {
                const int pg = p.src.page_shift >= 0 ? (int)row >> p.src.page_shift : (int)row / p.src.page_size;
                c3 = ld_here(p.src.page_table + (int64_t)a.seq * p.src.max_pages_per_seq + pg);
                c1 = (int)row - pg * p.src.page_size;
                ok = p.src.n_pages <= 0 || (c3 >= 0 && c3 < p.src.n_pages);
            }
            const uint32_t bad = __ballot_sync(0xffffffffu, !ok);
            if (lane == 0) {
                uint32_t mask = 0;
                if (bad) {
                    for (int x = 0; x < kPTile / kTileKeys; ++x) mask |= ((bad >> (x * kTileKeys / box)) & 1u) << x;
                    if (!is_v && p.device_status) atomicExch(p.device_status, (int)TRI_ERR_DEVICE_CHECK);
                }
                if (is_v) absent_raw[st] = mask;
                mbar_expect_tx(b_raw + 8 * st, (uint32_t)(nsub - __popc(bad)) * box * 128);
            }
            __syncwarp();
            if (lane < nsub && ok) tma_load_5d(raw + st * kPRawBytes + lane * box * 128, map, b_raw + 8 * st, 0, c1, a.h, c3, p.layer);
            ++asked;
            if (++at == a.kb - a.ka) { at = 0; open = next_asked(); }
            return true;
        };
        bool ok = ask() && ask();
        while (ok && !gave_up && next_rows(false)) {
            const int n = j.kb - j.ka;
            for (int t = 0; t < n; ++t) {
                const int i = done + t, st = i & 1;
                ok = mbar_wait_parked<20>(b_raw + 8 * st, (i >> 1) & 1) && (i < 2 || mbar_wait_parked<20>(b_empty + 8 * st, ((i >> 1) - 1) & 1));
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                const int64_t left = j.len - (int64_t)(j.ka + t) * kPTile;
                const int have = left < kPTile ? (int)left : kPTile;
                const uint32_t miss = is_v ? absent_raw[st] : 0u;
                const bool cut = is_v && (have < kPTile || miss);
                if (is_v && lead && lane == 0) absent[st] = miss;
                const uint8_t *src = g_raw + st * kPRawBytes;
                uint8_t *dst = g_out + st * kPTileBytes;
                // lane = (row of four, 16 values): 512 contiguous bytes in, four wavefronts per store out
                const int c = lane & 7, first = (lead ? 0 : 64) + (lane >> 3);
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    uint4 x[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const int r = first + 4 * (8 * b + k);
                        x[k] = *reinterpret_cast<const uint4 *>(src + r * 128 + ((c ^ (r & 7)) << 4));
                    }
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const int r = first + 4 * (8 * b + k);
                        uint4 lo, hi;
                        e4m3x4_to_f16x2(x[k].x, lo.x, lo.y);
                        e4m3x4_to_f16x2(x[k].y, lo.z, lo.w);
                        e4m3x4_to_f16x2(x[k].z, hi.x, hi.y);
                        e4m3x4_to_f16x2(x[k].w, hi.z, hi.w);
                        if (cut && (r >= have || ((miss >> (r >> 4)) & 1u))) { lo = make_uint4(0u, 0u, 0u, 0u); hi = lo; }
                        uint8_t *to = dst + (c >> 2) * kPBlock;
                        *reinterpret_cast<uint4 *>(to + sw128(r, 2 * c & 7)) = lo;
                        *reinterpret_cast<uint4 *>(to + sw128(r, (2 * c + 1) & 7)) = hi;
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
                __syncwarp();
                if (lane == 0) { mbar_arrive(b_full + 8 * st); mbar_arrive(b_free + 8 * st); }
                ok = ask();
                if (!ok) break;
            }
            done += n;
        }
        if (!ok) gave_up = 1;
    } else if (!KEY8 && warp >= kPSoftWarps && warp < kMmaWarp) {
        // ---------------- bf16 producers: one warp for K, one for V, lane = (box, half of the dims) ----------------
        // (one warp for both: its copies, 32 for 16-row boxes, are issued one by one and held a paged prefix back)
        // a box is `box` rows high: 128 where rows are contiguous, else the largest power of two up to 128 that divides a page
        const bool is_v = warp != kPSoftWarps;
        const CUtensorMap *map = is_v ? &vmap : &kmap;
        const uint32_t b_full = is_v ? b_vfull : b_kfull, b_empty = is_v ? b_vempty : b_kempty, ring = is_v ? sm_v : sm_k;
        const int box = p.box_rows, sub = lane >> 1, half = lane & 1, boxes = kPTile / box;
        while (!gave_up && next_rows(false)) {
            const int n = j.kb - j.ka;
            auto locate = [&](int t, int &c1, int &c3) -> bool {          // false: the box's page id is out of range
                const int64_t row = (int64_t)(j.ka + t) * kPTile + sub * box;
                c1 = (int)row; c3 = j.seq;
                if (!p.src.paged || t >= n || sub >= boxes || row >= j.len) return true;
                const int pg = p.src.page_shift >= 0 ? (int)row >> p.src.page_shift : (int)row / p.src.page_size;
                c3 = ld_here(p.src.page_table + (int64_t)j.seq * p.src.max_pages_per_seq + pg);
                c1 = (int)row - pg * p.src.page_size;
                return p.src.n_pages <= 0 || (c3 >= 0 && c3 < p.src.n_pages);
            };
            int c1 = 0, c3 = 0;
            bool ok = locate(0, c1, c3);
            for (int t = 0; t < n; ++t) {
                const int i = done + t, st = i % ST;
                const uint32_t par = ((i / ST) - 1) & 1;
                const int64_t left = j.len - (int64_t)(j.ka + t) * kPTile;
                const int nsub = left >= kPTile ? boxes : (int)((left + box - 1) / box);
                const uint32_t bad = __ballot_sync(0xffffffffu, !ok && sub < nsub && half == 0);
                uint32_t mask = 0;                         // of 16-row groups
                if (bad) {
                    for (int x = 0; x < kPTile / kTileKeys; ++x) mask |= ((bad >> (2 * (x * kTileKeys / box))) & 1u) << x;
                    if (lane == 0 && !is_v && p.device_status) atomicExch(p.device_status, (int)TRI_ERR_DEVICE_CHECK);
                }
                const uint32_t bytes = (uint32_t)(nsub - __popc(bad)) * box * (kHeadDim * 2);
                const bool w = i < ST || mbar_wait_parked<20>(b_empty + 8 * st, par);
                if (!__all_sync(0xffffffffu, w)) { gave_up = 1; break; }
                if (lane == 0) {
                    if (is_v) absent[st] = mask;
                    mbar_expect_tx(b_full + 8 * st, bytes);
                }
                __syncwarp();
                if (sub < nsub && ok)
                    tma_load_5d(ring + st * kPTileBytes + half * kPBlock + sub * box * 128, map, b_full + 8 * st, half * (kHeadDim / 2), c1, j.h,
                                c3, p.layer);
                ok = locate(t + 1, c1, c3);
            }
            done += n;
        }
    } else if (warp == kMmaWarp) {
        // ---------------- MMA issue ----------------
        constexpr uint32_t idesc_qk = tc_idesc_16(KEY8, kPTile);                 // both operands K-major
        constexpr uint32_t idesc_pv = tc_idesc_16(KEY8, kHeadDim) | (1u << 16);  // B (the values) N-major
        int units = 0, cnt[2] = {0, 0};                    // tiles each stream had in earlier units (phases of pready)
        while (!gave_up && next_rows(false)) {
            const int n = j.kb - j.ka;
            bool ok = __all_sync(0xffffffffu, mbar_wait_bounded(b_q, units & 1));
            // logits of tile t: into the columns whose weights the MMAs issued before have used up.  As MMAs complete in order,
            // sfull says that the stream's accumulator rests, too; behind the stream's last tile it says nothing else
            auto logits = [&](int t) -> bool {
                const int i = done + t, st = i % ST;
                if (!__all_sync(0xffffffffu, mbar_wait_bounded(b_kfull + 8 * st, (i / ST) & 1))) return false;
                tc_fence_after();
                if (lane == 0) {
                    const uint32_t ka = sm_k + st * kPTileBytes, acc = tmem + 128 * (t & 1);
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        tc_mma_bf16(acc, tc_desc_sw128(sm_q + (k >> 2) * kPBlock + (k & 3) * 32),
                                    tc_desc_sw128(ka + (k >> 2) * kPBlock + (k & 3) * 32), idesc_qk, k > 0);
                    tc_commit(b_sfull + 8 * (t & 1));
                    tc_commit(b_kempty + 8 * st);
                }
                __syncwarp();
                return true;
            };
            for (int t = 0; t < 2 && t < n && ok; ++t) ok = logits(t);
            for (int t = 0; t < n && ok; ++t) {
                // weights of tile t times its values, the upper half of its rows first (as the softmax delivers them), then
                // the logits of the stream's next tile
                const int i = done + t, st = i % ST, w = t & 1;
                ok = mbar_wait_bounded(b_vfull + 8 * st, (i / ST) & 1);
                for (int x = 1; x >= 0; --x) {
                    ok = __all_sync(0xffffffffu, ok && mbar_wait_bounded(b_pready + 8 * (2 * w + x), (cnt[w] + (t >> 1)) & 1));
                    if (!ok) break;
                    tc_fence_after();
                    if (lane == 0) {
                        const uint32_t va = sm_v + st * kPTileBytes + x * (kPHalf * 128), acc = tmem + 256 + 128 * w, pw = tmem + 128 * w + kPHalf * x;
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            tc_mma_bf16_ts(acc, pw + 8 * k, tc_desc_sw128_n(va + k * 2048), idesc_pv, t >= 2 || x == 0 || k > 0);
                        if (x == 0) tc_commit(b_vempty + 8 * st);
                        if (x == 0 && t + 2 >= n) tc_commit(b_sfull + 8 * w);
                    }
                    __syncwarp();
                }
                if (ok && t + 2 < n) ok = logits(t + 2);
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
        const bool check_pages = p.src.paged && p.src.n_pages > 0;
        int units = 0, phase[2] = {0, 0};                  // phases of sfull: one per tile, one more behind a unit's last
        const uint32_t flip = p.scale < 0.f ? 0x80008000u : 0u;            // a negative scale goes into the queries' signs
        while (!gave_up && more) {
            const AttJob u = j;                            // (j runs ahead to the unit behind it)
            const int n = u.kb - u.ka;
            constexpr int NQ = KEY8 ? 4 : 8;               // 16 bytes of 8 rows per thread, NQ rows at a time
#pragma unroll 1
            for (int q0 = 0; q0 < 8; q0 += NQ) {
                uint4 q[NQ];
#pragma unroll
                for (int i = 0; i < NQ; ++i) {
                    const int r = (tid >> 4) + 16 * (q0 + i);
                    q[i] = r < u.nrows ? *reinterpret_cast<const uint4 *>(query_row(u, r) + 16 * (tid & 15)) : make_uint4(0u, 0u, 0u, 0u);
                }
#pragma unroll
                for (int i = 0; i < NQ; ++i) {
                    const int r = (tid >> 4) + 16 * (q0 + i), c = tid & 15;
                    uint32_t x[4] = {q[i].x ^ flip, q[i].y ^ flip, q[i].z ^ flip, q[i].w ^ flip};
                    if (KEY8) {
                        // to f16, the row's largest entry brought to [1, 2) (see k_attend)
                        float amax = 0.f;
#pragma unroll
                        for (int y = 0; y < 4; ++y) amax = fmaxf(amax, fmaxf(fabsf(bf16_lo(x[y])), fabsf(bf16_hi(x[y]))));
#pragma unroll
                        for (int d = 1; d < 16; d <<= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, d));
                        int e = min(max((int)((__float_as_uint(amax) >> 23) & 255u) - 127, -126), 126);
                        if (amax == 0.f) e = 0;
                        const float by = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
                        for (int y = 0; y < 4; ++y) x[y] = f16_bits(bf16_lo(x[y]) * by) | (f16_bits(bf16_hi(x[y]) * by) << 16);
                        if (c == 0) qscale_s[KEY8 ? r : 0] = __uint_as_float((uint32_t)(127 + e) << 23);
                    }
                    *reinterpret_cast<uint4 *>(gq + (c >> 3) * kPBlock + sw128(r, c & 7)) = make_uint4(x[0], x[1], x[2], x[3]);
                }
            }
            asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
            tc_fence_before();                             // the last unit's accumulators have been read
            __syncwarp();
            if (lane == 0) mbar_arrive(b_q);
            more = next_rows(tid == 0);
            if (more) prefetch_queries(j);

            // base-2 logit = accumulator * mul (not 0: a masked logit is -infinity)
            bool ok = true;
            float mul = fabsf(p.scale) * (p.k_scale ? p.k_scale[u.h] : 1.f);
            if (KEY8) {
                ok = __all_sync(0xffffffffu, mbar_wait_bounded(b_q, units & 1));        // the other warps' rows and scales, too
                mul *= qscale_s[KEY8 ? row : 0];
            }
            mul = fmaxf(mul, 1.17549435e-38f);
            const float2 mul2 = make_float2(mul, mul);
            float m = -INFINITY;
            // sums of the weights (even and odd rows) as they are, for the row's statistics, and as they enter the MMAs: o is
            // divided by the latter, so that the roundings all but cancel
            float2 l = make_float2(0.f, 0.f), lr = make_float2(0.f, 0.f);
#pragma unroll 1
            for (int t = w; t < n && ok; t += 2) {
                const int i = done + t, st = i % ST;
                const int64_t left = u.len - (int64_t)(u.ka + t) * kPTile;
                const bool cut = left < kPTile;
                ok = mbar_wait_bounded(b_sfull + 8 * w, (phase[w] + (t >> 1)) & 1);
                if (cut || check_pages) ok = ok && mbar_wait_bounded(b_vfull + 8 * st, (i / ST) & 1);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                const uint32_t miss = check_pages ? absent[st] : 0u;
                const int have = cut ? (int)left : kPTile;
                uint32_t s[kPHalf];
                float top = -INFINITY;
                // the row's largest logit: the lower half is read again below, the upper half stays in registers
#pragma unroll 1
                for (int x = 0; x < 2; ++x) {
                    tc_ld64(t_s + kPHalf * x, s);
                    tc_wait_ld();
                    tc_loaded(s);
                    if (cut || miss) {
                        const int first = kPHalf * x;
#pragma unroll
                        for (int y = 0; y < kPHalf; ++y)
                            if (first + y >= have || ((miss >> (4 * x + (y >> 4))) & 1u)) s[y] = 0xff800000u;
                        if (x == 0) tc_st64(t_s, s);
                    }
                    float a = fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1])), b = fmaxf(__uint_as_float(s[2]), __uint_as_float(s[3]));
#pragma unroll
                    for (int y = 4; y < kPHalf; y += 4) {
                        a = fmaxf(a, fmaxf(__uint_as_float(s[y]), __uint_as_float(s[y + 1])));
                        b = fmaxf(b, fmaxf(__uint_as_float(s[y + 2]), __uint_as_float(s[y + 3])));
                    }
                    top = fmaxf(top, fmaxf(a, b));
                }
                if (cut || miss) {
                    // rows behind the length or of absent pages: no weight, and zeros for values (they may hold anything)
                    // (8 bits: the converters have seen to the values' rows)
                    if (!KEY8 && (row >= have || ((miss >> (row >> 4)) & 1u))) {
#pragma unroll
                        for (int c = 0; c < 16; ++c)
                            *reinterpret_cast<uint4 *>(gv + st * kPTileBytes + (c >> 3) * kPBlock + row * 128 + (c & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                    }
                    asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
                    tc_wait_st();
                }
                top *= mul;
                const bool raise = top > m + kAttAbove<KEY8> || (m == -INFINITY && top > m);
                if (__any_sync(0xffffffffu, raise)) {
                    top -= kAttBelow<KEY8>;
                    const float by = raise ? ex2(m - top) : 1.f;
                    if (raise) m = top;
                    l.x *= by; l.y *= by; lr.x *= by; lr.y *= by;
                    if (t >= 2) {                          // an accumulator exists, and rests
#pragma unroll 1
                        for (int c = 0; c < 8; ++c) {
                            uint32_t o[16];
                            tc_ld16(t_o + 128 * w + 16 * c, o);
                            tc_wait_ld();
                            tc_loaded(o);
#pragma unroll
                            for (int y = 0; y < 16; ++y) o[y] = __float_as_uint(__uint_as_float(o[y]) * by);
                            tc_st16(t_o + 128 * w + 16 * c, o);
                        }
                    }
                }
                const float ref = m == -INFINITY ? 0.f : m;
                const float2 ref2 = make_float2(-ref, -ref);
#pragma unroll 1
                for (int x = 1; x >= 0; --x) {
                    // weights over the logits of this half, 32 columns of bf16 pairs
#pragma unroll
                    for (int c = 0; c < kPHalf / 32; ++c) {
                        uint32_t hi[16];
#pragma unroll
                        for (int y = 0; y < 16; ++y) {
                            float2 e = fma2(make_float2(__uint_as_float(s[32 * c + 2 * y]), __uint_as_float(s[32 * c + 2 * y + 1])), mul2, ref2);
                            e.x = ex2(e.x);
                            e.y = ex2(e.y);
                            l = add2(l, e);
                            if (KEY8) {                    // 11 bits in f16
                                asm("cvt.rn.f16x2.f32 %0, %1, %2;\n" : "=r"(hi[y]) : "f"(e.y), "f"(e.x));
                            } else {
                                hi[y] = cvt_bf16x2(e.y, e.x);
                                lr = add2(lr, make_float2(bf16_lo(hi[y]), bf16_hi(hi[y])));
                            }
                        }
                        tc_st16(t_s + kPHalf * x + 16 * c, hi);
                    }
                    if (x == 1) {
                        tc_ld64(t_s, s);
                        tc_wait_ld();
                        tc_loaded(s);
                    }
                    tc_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(b_pready + 8 * (2 * w + x));
                }
            }
            done += n;
            phase[0] += ((n + 1) >> 1) + 1;
            phase[1] += n >= 2 ? (n >> 1) + 1 : 0;
            // ---------------- join the two streams ----------------
            // own stream first: a parity wait cannot tell a phase from the one two before it, and as the MMAs complete in
            // order, the other stream's barrier is then at most its last phase behind
            for (int z = 0; z < 2 && ok; ++z) {
                const int y = z == 0 ? w : 1 - w;
                if (y == 0 || n >= 2) ok = mbar_wait_bounded(b_sfull + 8 * y, (phase[y] - 1) & 1);
            }
            // (the columns of S and P are idle until the next unit's queries are announced: m, l and l / lr pass through them)
            ok = __all_sync(0xffffffffu, ok);
            if (ok) {
                tc_fence_after();
                tc_st4f(t_s, m, l.x + l.y, !KEY8 && lr.x + lr.y > 0.f ? (l.x + l.y) / (lr.x + lr.y) : 1.f);
                tc_wait_st();
                tc_fence_before();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(b_ml);
            ok = __all_sync(0xffffffffu, ok && mbar_wait_bounded(b_ml, units & 1));
            if (!ok) { gave_up = 1; break; }
            tc_fence_after();
            uint32_t s0[4], s1[4];
            tc_ld4(tmem + lane_base, s0);
            tc_ld4(tmem + lane_base + 128, s1);
            tc_wait_ld();
            tc_loaded(s0);
            tc_loaded(s1);
            const float m0 = __uint_as_float(s0[0]), m1 = __uint_as_float(s1[0]), mm = fmaxf(m0, m1);
            const float e0 = m0 == -INFINITY ? 0.f : ex2(m0 - mm), e1 = m1 == -INFINITY ? 0.f : ex2(m1 - mm);
            const float vs = p.v_scale ? p.v_scale[u.h] : 1.f;
            const float f0 = e0 * __uint_as_float(s0[2]) * vs, f1 = e1 * __uint_as_float(s1[2]) * vs;
            const bool mine = row < u.nrows;
            const int sr = att_small_div(row, inv_g), sq = u.first_seq + sr, hq = u.h * p.G + row - sr * p.G;
            // slots hold four dims of all rows, then the next four: a warp writes 512 bytes in a row
            float *to = u.complete ? p.whole + ((int64_t)(mine ? sq : 0) * p.H * p.G + hq) * kAttRowPitch
                                   : p.slots + ((int64_t)blockIdx.x * 2 + (u.begins ? 1 : 0)) * kPTile * kAttRowPitch + 4 * row;
            const int quad = u.complete ? 4 : 4 * kPTile;
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
                        *reinterpret_cast<float4 *>(to + (16 * w + 4 * c + x) * quad) = make_float4(y[4 * x], y[4 * x + 1], y[4 * x + 2], y[4 * x + 3]);
                }
            }
            if (mine && w == 0)
                *reinterpret_cast<float2 *>(u.complete ? to + kHeadDim : to - 4 * row + kPTile * kHeadDim + 2 * row) =
                    make_float2(mm, __uint_as_float(s0[1]) * e0 + __uint_as_float(s1[1]) * e1);
            ++units;
        }
    }

    tc_fence_before();
    __syncthreads();
    if (gave_up) {
        // a wait ran out: report it, and give copies still in flight one more bounded chance to land before the block exits
        if (tid == 0 && p.device_status) atomicExch(p.device_status, (int)TRI_ERR_TIMEOUT);
        if (warp == kPSoftWarps || warp == kPSoftWarps + 1)
            for (int i = 0; i < 2 * ST; ++i) {
                const uint32_t full = KEY8 ? smem_u32(&bars.rawfull[warp == kPSoftWarps ? 0 : 2]) : (warp == kPSoftWarps ? b_kfull : b_vfull);
                (void)mbar_wait_parked(full + 8 * (i % ST), (i / ST) & 1);
            }
    }
    if (warp == kMmaWarp) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(512) : "memory");
    }
}

}  // namespace tri
