// Appending a step's keys and values to a 4-bit cache: rotated as in tri_append.cuh, then quantised (tri_row4.cuh).
//
// Mathematics.  A group's range lo, hi gives c = bf16((8 hi + 7 lo) / 15) and s = the smallest bf16 not below (hi - c) / 7 and
// (c - lo) / 8, so that -8 .. 7 steps of s from c cover the range: no component is off by more than s / 2.
// fp32 does for nearly all rows.  A rotated key is off by a few steps of fp32, which matters where a quotient lies at the border of
// two codes, or c or s at the border of two bf16 numbers: such rows (8 of 1,000) are put on a list and done again in fp64, so that a
// row is what the definition says, not what the rounding of its rotation made of it.
//
// What bounds it.  Every byte of k, v, q is read once and every row written once; quantising costs some 200 instructions per lane
// and row beside 75 for a rotated query row.  16,384 tokens of 8 + 8 + 32 bf16 rows: 72 us, 4.9 TB/s (0.77 of the copy rate), issue
// slots in use 0.59 of the time; 64 sequences of one token 4 us, launch and the latency of fp64 sines.  Work split as in
// tri_append.cuh: eight lanes own a row, 16 components each; a block covers TT tokens of one sequence.
#pragma once
#include "tri_append.cuh"
#include "tri_row4.cuh"

namespace tri {

constexpr int kAppend4List = 32;      // rows that a block does again; where more are in doubt it does all of them again

// The 16 components of a lane as the two parts of its 8 bands, bands j and j + 1 side by side.
struct Bands { f32x2 re[4], im[4]; };
template <int KIND, bool SPLIT>
__device__ __forceinline__ void widen_bands(const Raw16<KIND> &raw, Bands &x)
{
    float y[16];
    widen16<KIND>(raw, y);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x.re[i] = SPLIT ? pair_of(y[2 * i], y[2 * i + 1]) : pair_of(y[4 * i], y[4 * i + 2]);
        x.im[i] = SPLIT ? pair_of(y[8 + 2 * i], y[9 + 2 * i]) : pair_of(y[4 * i + 1], y[4 * i + 3]);
    }
}
// Cosines and sines of a lane's bands.
struct Turns { f32x2 c[4], s[4]; };
__device__ __forceinline__ void load_turns(const float *cosines, const float *sines, int c, Turns &t)
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float4 a = *reinterpret_cast<const float4 *>(cosines + 8 * c + 4 * i), b = *reinterpret_cast<const float4 *>(sines + 8 * c + 4 * i);
        t.c[2 * i] = pair_of(a.x, a.y); t.c[2 * i + 1] = pair_of(a.z, a.w);
        t.s[2 * i] = pair_of(b.x, b.y); t.s[2 * i + 1] = pair_of(b.z, b.w);
    }
}
// Sine and cosine of position `at` of a band with w turns per position, in fp64.
__device__ __forceinline__ void turn_fp64(double at, double2 w, double &sn, double &cn)
{
    const double hi = at * w.x;
    sincospi(2.0 * ((hi - rint(hi)) + fma(at, w.y, fma(at, w.x, -hi))), &sn, &cn);
}
__device__ __forceinline__ void rotate_bands(Bands &x, const Turns &t)
{
    const f32x2 minus = pair_of(-1.f, -1.f);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x2 re = x.re[i], im = x.im[i];
        x.re[i] = fma2(t.c[i], re, mul2(mul2(t.s[i], im), minus));
        x.im[i] = fma2(t.s[i], re, mul2(t.c[i], im));
    }
}
template <bool SPLIT>
__device__ __forceinline__ void store_bands(char *row, int c, const Bands &x)
{
    float y[16];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        parts_of(x.re[i], y[SPLIT ? 2 * i : 4 * i], y[SPLIT ? 2 * i + 1 : 4 * i + 2]);
        parts_of(x.im[i], y[SPLIT ? 8 + 2 * i : 4 * i + 1], y[SPLIT ? 9 + 2 * i : 4 * i + 3]);
    }
    store16<2, SPLIT>(row, c, y);
}

// What a lane has of a row: half of group c / 2 (SPLIT: quarters of groups c / 4 and c / 4 + 2).
template <bool SPLIT> struct Row4Lane {
    static constexpr int NG = SPLIT ? 2 : 1, EL = 16 / NG;        // groups of the lane, its components of each
    float s[NG], m[NG];
    uint32_t w[2];
};
template <bool SPLIT>
__device__ __forceinline__ void store_row4(char *row, int c, const Row4Lane<SPLIT> &r)
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {                            // a word each: group g, unit t
        const int g = SPLIT ? (c >> 2) + 2 * i : c >> 1, t = SPLIT ? c & 3 : 2 * (c & 1) + i;
        *reinterpret_cast<uint32_t *>(row + 16 * t + 4 * g) = r.w[i];
        if (t == 0) {
            *reinterpret_cast<uint16_t *>(row + kRow4Scales + 2 * g) = (uint16_t)(__float_as_uint(r.s[SPLIT ? i : 0]) >> 16);
            *reinterpret_cast<uint16_t *>(row + kRow4Centres + 2 * g) = (uint16_t)(__float_as_uint(r.m[SPLIT ? i : 0]) >> 16);
        }
    }
}
// The lanes of a row, `lanes`, find the ranges of its groups together.  ROTATED: the values are a few steps of fp32 off; returns
// whether that may have changed a scale, a centre or a code (a quotient within 2^-16 of the border of two).
template <bool SPLIT, bool ROTATED>
__device__ __forceinline__ bool quantise_row4(const Bands &x, uint32_t lanes, Row4Lane<SPLIT> &r)
{
    constexpr int NG = Row4Lane<SPLIT>::NG;
    bool doubt = false;
    float off = 0.f, lo[2], hi[2], inv[NG];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const f32x2 *y = j ? x.im : x.re;
        float a, b;
        parts_of(y[0], a, b);
        lo[j] = min_nan(a, b); hi[j] = max_nan(a, b);
#pragma unroll
        for (int i = 1; i < 4; ++i) {
            parts_of(y[i], a, b);
            lo[j] = min_nan(lo[j], a, b); hi[j] = max_nan(hi[j], a, b);
        }
    }
    if (!SPLIT) { lo[0] = min_nan(lo[0], lo[1]); hi[0] = max_nan(hi[0], hi[1]); }
#pragma unroll
    for (int j = 0; j < NG; ++j) {
#pragma unroll
        for (int d = 1; d < (SPLIT ? 4 : 2); d *= 2) {
            lo[j] = min_nan(lo[j], __shfl_xor_sync(lanes, lo[j], d));
            hi[j] = max_nan(hi[j], __shfl_xor_sync(lanes, hi[j], d));
        }
        doubt = row4_group(lo[j], hi[j], r.s[j], r.m[j]) || doubt;
        inv[j] = __frcp_rn(r.s[j] > 0.f ? r.s[j] : 1.f);
    }
    r.w[0] = r.w[1] = 0u - kRow4Bias;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t a, b, d, e;
        row4_codes<!ROTATED>(x.re[i], r.s[0], inv[0], r.m[0], off, a, b);
        row4_codes<!ROTATED>(x.im[i], r.s[NG - 1], inv[NG - 1], r.m[NG - 1], off, d, e);
        if (SPLIT) {                                         // components 2 i, 2 i + 1 of either word
            r.w[0] += (a << 4 * i) + (b << 4 * (i + 4));
            r.w[1] += (d << 4 * i) + (e << 4 * (i + 4));
        } else {                                             // bands 2 i, 2 i + 1: components 4 i, 4 i + 2 and the ones behind them
            const int k = 2 * (i & 1);
            r.w[i >> 1] += (a << 4 * k) + (b << 4 * (k + 1)) + (d << 4 * (k + 4)) + (e << 4 * (k + 5));
        }
    }
    return ROTATED && (doubt || off > 0.5f - 0x1p-16f);
}
// A row of keys from what it came as, in fp64.  TURNED: `turn` holds the cosines and sines of the position, else turns per position.
template <int KIND, bool SPLIT, bool TURNED>
__device__ __forceinline__ void row4_fp64(const char *from, char *to, int c, double at, const double2 *turn, uint32_t lanes)
{
    constexpr int NG = Row4Lane<SPLIT>::NG, EL = Row4Lane<SPLIT>::EL;
    Raw16<KIND> raw;
    load16<KIND, SPLIT>(from, c, raw);
    float in[16];
    widen16<KIND>(raw, in);
    Row4Lane<SPLIT> r;
    double x[16];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const double2 w = turn[8 * c + j];
        double sn = w.y, cn = w.x;
        if (!TURNED) turn_fp64(at, w, sn, cn);
        const int ir = SPLIT ? j : 2 * j, ii = SPLIT ? j + 8 : 2 * j + 1;
        x[ir] = cn * in[ir] - sn * in[ii];
        x[ii] = sn * in[ir] + cn * in[ii];
    }
#pragma unroll
    for (int j = 0; j < NG; ++j) {
        double lo = x[EL * j], hi = lo;
        bool nan = false;                                    // (fmin and fmax pass over them)
#pragma unroll
        for (int i = 0; i < EL; ++i) {
            lo = fmin(lo, x[EL * j + i]); hi = fmax(hi, x[EL * j + i]);
            nan = nan || x[EL * j + i] != x[EL * j + i];
        }
        for (int d = 1; d < 32 / EL; d *= 2) {
            lo = fmin(lo, __shfl_xor_sync(lanes, lo, d));
            hi = fmax(hi, __shfl_xor_sync(lanes, hi, d));
            nan = __shfl_xor_sync(lanes, (int)nan, d) || nan;
        }
        float m = bf16_lo(cvt_bf16x2(0.f, (float)((8.0 * hi + 7.0 * lo) / 15.0)));
        const double below = __dsub_ru((double)m, lo);
        const float need = __double2float_ru(fmax(__ddiv_ru(__dsub_ru(hi, (double)m), 7.0), below * 0.125));      // (upwards, as in row4_group)
        const uint32_t up = max((__float_as_uint(need) + 0xffffu) & 0xffff0000u, 0x00800000u);
        float s = need > 0.f ? __uint_as_float(up) : 0.f;
        if (nan || !(fabsf((float)below) < INFINITY)) { m = __uint_as_float(0x7fc00000u); s = 0.f; }
        r.m[j] = m; r.s[j] = s;
        const double by = s > 0.f ? (double)s : 1.0;
#pragma unroll
        for (int i = 0; i < EL / 8; ++i) {
            uint32_t word = 0;
#pragma unroll
            for (int d = 0; d < 8; ++d) {
                const double q = rint((x[EL * j + 8 * i + d] - (double)m) / by);
                word |= (uint32_t)(int)(fmin(fmax(q, -8.0), 7.0) + 8.0) << 4 * ((d >> 1) + 4 * (d & 1));
            }
            r.w[j * (EL / 8) + i] = word;
        }
    }
    store_row4<SPLIT>(to, c, r);
}

template <int KIND, bool SPLIT>
__device__ __noinline__ void redo_row4(const char *from, char *to, int c, double at, const double2 *turn, uint32_t lanes)
{
    row4_fp64<KIND, SPLIT, false>(from, to, c, at, turn, lanes);
}

// A single token per sequence: latency is all that counts, and a row of some block is always in doubt.  Its keys go through fp64 at
// once, whose sines take a microsecond, beside the values, each on lanes of their own.
template <int KIND, bool SPLIT>
__global__ void __launch_bounds__(kAppendThreads) k_append4_one(const AppendParams p, int roles)
{
    constexpr int kGroups = kAppendThreads / 8, in_es = KIND == 0 ? 2 : 4, UQ = 2;
    __shared__ __align__(16) float cos_s[kBands], sin_s[kBands];
    __shared__ double2 turn_s[kBands];
    const int tid = threadIdx.x, c = tid & 7, grp = tid >> 3;
    const uint32_t lanes = 0xffu << (tid & 24);
    const int s = roles == 2 ? blockIdx.x >> 1 : blockIdx.x;
    const bool do_kv = roles == 1 || (blockIdx.x & 1) == 0, do_q = p.q && (roles == 1 || (blockIdx.x & 1));
    grid_dependency_wait();
    grid_dependents_launch();
    const int n_new = append_count(p, s);
    if (do_kv && tid == 0 && p.device_status && p.n_new) {
        const int raw = p.n_new[s];
        if (raw < 0 || raw > p.T) atomicExch(p.device_status, (int)TRI_ERR_DEVICE_CHECK);
    }
    if (n_new > 0) {
        const int64_t at = p.pos ? p.pos[s] : (int64_t)append_len(p, s, 0);
        const char *q = p.q + s * p.qs_seq * in_es, *k = p.k + s * p.ks_seq * in_es, *v = p.v + s * p.vs_seq * in_es;
        const int nq = do_q ? p.H * p.G : 0;
        Raw16<KIND> rq[UQ];                                   // queries are loaded one turn ahead, the first ones before the sines
#pragma unroll
        for (int u = 0; u < UQ; ++u)
            if (grp + u * kGroups < nq) load16<KIND, SPLIT>(q + (grp + u * kGroups) * p.qs_head * in_es, c, rq[u]);
        if (tid < kBands) {
            double sn, cn;
            turn_fp64((double)at, p.turn[tid], sn, cn);
            turn_s[tid] = make_double2(cn, sn);
            cos_s[tid] = (float)cn; sin_s[tid] = (float)sn;
        }
        __syncthreads();
        const bool pos_ok = at >= 0 && at <= 0x7fffffff;
        if (do_kv && tid == 0 && !pos_ok && p.device_status) atomicExch(p.device_status, (int)TRI_ERR_DEVICE_CHECK);
        if (pos_ok && do_kv) {
            const int rows = p.v ? 2 * p.H : p.H;
            for (int r = grp; r < rows; r += kGroups) {
                const bool is_k = r < p.H;
                const int h = is_k ? r : r - p.H;
                const int64_t slot = append_len(p, s, h);
                const int64_t off = slot < p.dst.n_max ? step_row_offset(p.dst, p.layer, s, h, (int)slot) : -1;
                if (off == -1) {                              // (offsets are multiples of 16)
                    if (p.device_status) atomicExch(p.device_status, (int)TRI_ERR_DEVICE_CHECK);
                    continue;
                }
                if (is_k) {
                    row4_fp64<KIND, SPLIT, true>(k + h * p.ks_head * in_es, p.dst.k + off, c, 0.0, turn_s, lanes);
                    if (c == 0 && p.dst.positions)
                        p.dst.positions[(((int64_t)p.layer * p.S + s) * p.H + h) * p.dst.n_max + slot] = (int32_t)at;
                } else {
                    Raw16<KIND> raw;
                    load16<KIND, SPLIT>(v + h * p.vs_head * in_es, c, raw);
                    Bands x;
                    Row4Lane<SPLIT> row;
                    widen_bands<KIND, SPLIT>(raw, x);
                    quantise_row4<SPLIT, false>(x, lanes, row);
                    store_row4<SPLIT>(p.dst.v + off, c, row);
                }
            }
        }
        if (pos_ok && nq) {
            Turns turns;
            load_turns(cos_s, sin_s, c, turns);
            char *q_out = p.q_out + s * p.qo_seq * 2;
            for (int r0 = grp; r0 < nq; r0 += UQ * kGroups) {
#pragma unroll
                for (int u = 0; u < UQ; ++u) {
                    const int r = r0 + u * kGroups, next = r + UQ * kGroups;
                    if (r >= nq) break;
                    Bands x;
                    widen_bands<KIND, SPLIT>(rq[u], x);
                    if (next < nq) load16<KIND, SPLIT>(q + next * p.qs_head * in_es, c, rq[u]);
                    rotate_bands(x, turns);
                    store_bands<SPLIT>(q_out + r * p.qo_head * 2, c, x);
                }
            }
        }
    }
    if (p.new_lens && do_kv) {                                // this block is the only reader of the lengths (see the launch)
        __syncthreads();
        const int n = p.unit_lens ? p.H : 1;
        for (int h = tid; h < n; h += kAppendThreads) {
            const int64_t len = (int64_t)append_len(p, s, h) + n_new;
            p.new_lens[(int64_t)s * n + h] = (int32_t)(len < p.dst.n_max ? len : p.dst.n_max);
        }
    }
}

// KIND: input 0 bf16, 1 fp32.  TT: tokens per block.  roles = 2: of two blocks of the same tokens the first takes keys and values, the
// second the queries, so that a multiprocessor has both kinds of work, one bound by instructions and the other by memory, at any time.
// (bf16: 64 registers spill 84 to 144 bytes; three blocks of 80, without spills, take as long: 88.8 against 88.3 us for 16,384 tokens
// with the read back, 43.5 against 43.3 for ragged pieces.)
template <int KIND, bool SPLIT, int TT>
__global__ void __launch_bounds__(kAppendThreads, KIND == 0 ? 4 : 2) k_append4(const AppendParams p, int roles)
{
    constexpr int kGroups = kAppendThreads / 8 / TT;          // row groups (of 8 lanes) per token
    constexpr int in_es = KIND == 0 ? 2 : 4, UQ = 2;      // (UQ: query rows in flight per lane)
    __shared__ __align__(16) float cos_s[TT][kBands], sin_s[TT][kBands];
    __shared__ int again_n;
    __shared__ int2 again_s[kAppend4List];                    // token, head

    const int tid = threadIdx.x, c = tid & 7;
    const uint32_t lanes = 0xffu << (tid & 24);
    const int tile = roles == 2 ? blockIdx.x >> 1 : blockIdx.x;
    const bool do_kv = roles == 1 || (blockIdx.x & 1) == 0, do_q = p.q && (roles == 1 || (blockIdx.x & 1));
    const int s = tile / p.ntiles, t0 = (tile - s * p.ntiles) * TT;
    grid_dependency_wait();
    grid_dependents_launch();
    const int n_new = append_count(p, s);
    const bool first = t0 == 0 && do_kv;
    if (first && tid == 0 && p.device_status && p.n_new) {
        const int raw = p.n_new[s];
        if (raw < 0 || raw > p.T) atomicExch(p.device_status, (int)TRI_ERR_DEVICE_CHECK);
    }
    if (t0 < n_new) {
        const int tt = tid / (8 * kGroups), grp = (tid >> 3) % kGroups, t = t0 + tt;
        const char *k = p.k + (s * p.ks_seq + t * p.ks_tok) * in_es, *v = p.v + (s * p.vs_seq + t * p.vs_tok) * in_es;
        // rows are loaded one turn ahead, those of the first heads before the sines
        Raw16<KIND> rk, rv;
        if (do_kv && t < n_new && grp < p.H) {
            load16<KIND, SPLIT>(k + grp * p.ks_head * in_es, c, rk);
            if (p.v) load16<KIND, SPLIT>(v + grp * p.vs_head * in_es, c, rv);
        }
        const int64_t p0 = p.pos ? p.pos[s] : (int64_t)append_len(p, s, 0);
        if (tid == 0) again_n = 0;
        for (int i = tid; i < TT * kBands; i += kAppendThreads) {
            const int f = i & (kBands - 1);
            const double2 w = p.turn[f];
            const double at = (double)(p0 + t0 + (i >> 6));
            const double hi = at * w.x;
            const double fr = (hi - rint(hi)) + fma(at, w.y, fma(at, w.x, -hi));     // turns, in about [-1/2, 1/2]
            const float fh = (float)fr;
            const float d = 6.2831853f * (float)(fr - (double)fh);                   // angle the fp32 turn leaves over
            float sn, cn;
            sincospif(2.0f * fh, &sn, &cn);
            cos_s[i >> 6][f] = fmaf(-d, sn, cn); sin_s[i >> 6][f] = fmaf(d, cn, sn);
        }
        __syncthreads();
        const int64_t at = p0 + t;
        const bool pos_ok = at >= 0 && at <= 0x7fffffff;
        if (do_kv && t < n_new && !pos_ok && p.device_status) atomicExch(p.device_status, (int)TRI_ERR_DEVICE_CHECK);
        // where the row of a token and head goes: its slot and its offset in the cache, -1 for none
        auto place = [&](int token, int h, int64_t &slot) -> int64_t {
            slot = (int64_t)append_len(p, s, h) + token;
            return slot < p.dst.n_max ? step_row_offset(p.dst, p.layer, s, h, (int)slot) : -1;
        };
        if (t < n_new && pos_ok) {
            Turns turns;
            load_turns(cos_s[tt], sin_s[tt], c, turns);
            if (do_kv) {
                int64_t slot = 0, off0 = -1;                  // head 0's row, when all heads have the same length
                if (!p.unit_lens) off0 = place(t, 0, slot);
                for (int h = grp; h < p.H; h += kGroups) {
                    int64_t off = off0 == -1 ? -1 : off0 + h * p.dst.stride_head;
                    if (p.unit_lens) off = place(t, h, slot);
                    const int next = h + kGroups;
                    Bands x;
                    Row4Lane<SPLIT> row;
                    widen_bands<KIND, SPLIT>(rk, x);
                    if (next < p.H) load16<KIND, SPLIT>(k + next * p.ks_head * in_es, c, rk);
                    rotate_bands(x, turns);
                    const bool doubt = __any_sync(lanes, quantise_row4<SPLIT, true>(x, lanes, row));
                    if (off != -1) store_row4<SPLIT>(p.dst.k + off, c, row);
                    if (p.v) {
                        widen_bands<KIND, SPLIT>(rv, x);
                        if (next < p.H) load16<KIND, SPLIT>(v + next * p.vs_head * in_es, c, rv);
                        quantise_row4<SPLIT, false>(x, lanes, row);
                        if (off != -1) store_row4<SPLIT>(p.dst.v + off, c, row);
                    }
                    if (off == -1) {                          // (offsets are multiples of 16)
                        if (p.device_status) atomicExch(p.device_status, (int)TRI_ERR_DEVICE_CHECK);
                        continue;
                    }
                    if (doubt && c == 0) {
                        const int i = atomicAdd(&again_n, 1);
                        if (i < kAppend4List) again_s[i] = make_int2(t, h);
                    }
                    if (c == 0 && p.dst.positions)
                        p.dst.positions[(((int64_t)p.layer * p.S + s) * p.H + h) * p.dst.n_max + slot] = (int32_t)at;
                }
            }
            if (do_q) {
                const int nq = p.H * p.G;
                const char *q = p.q + (s * p.qs_seq + t * p.qs_tok) * in_es;
                char *q_out = p.q_out + (s * p.qo_seq + t * p.qo_tok) * 2;
                Raw16<KIND> rq[UQ];
#pragma unroll
                for (int u = 0; u < UQ; ++u)
                    if (grp + u * kGroups < nq) load16<KIND, SPLIT>(q + (grp + u * kGroups) * p.qs_head * in_es, c, rq[u]);
                for (int r0 = grp; r0 < nq; r0 += UQ * kGroups) {
#pragma unroll
                    for (int u = 0; u < UQ; ++u) {
                        const int r = r0 + u * kGroups, next = r + UQ * kGroups;
                        if (r >= nq) break;
                        Bands x;
                        widen_bands<KIND, SPLIT>(rq[u], x);
                        if (next < nq) load16<KIND, SPLIT>(q + next * p.qs_head * in_es, c, rq[u]);
                        rotate_bands(x, turns);
                        store_bands<SPLIT>(q_out + r * p.qo_head * 2, c, x);
                    }
                }
            }
        }
        __syncthreads();
        // rows in doubt again, or all rows where the list is too short for them
        const bool all = again_n > kAppend4List;
        const int n = all ? min(TT, n_new - t0) * p.H : again_n;
        for (int i = tid >> 3; i < n; i += kAppendThreads / 8) {
            const int2 it = all ? make_int2(t0 + i / p.H, i % p.H) : again_s[i];
            int64_t slot;
            const int64_t off = p0 + it.x > 0x7fffffff || p0 + it.x < 0 ? -1 : place(it.x, it.y, slot);
            if (off != -1) redo_row4<KIND, SPLIT>(p.k + (s * p.ks_seq + it.x * p.ks_tok + it.y * p.ks_head) * in_es, p.dst.k + off, c, (double)(p0 + it.x), p.turn, lanes);
        }
    }
    // lengths into another array, or by the block that covers its whole sequence, their only reader, after its last read
    if (p.new_lens && first) {
        __syncthreads();
        const int n = p.unit_lens ? p.H : 1;
        for (int h = tid; h < n; h += kAppendThreads) {
            const int64_t len = (int64_t)append_len(p, s, h) + n_new;
            p.new_lens[(int64_t)s * n + h] = (int32_t)(len < p.dst.n_max ? len : p.dst.n_max);
        }
    }
}

}  // namespace tri
