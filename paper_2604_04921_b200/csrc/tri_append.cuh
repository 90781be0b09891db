// Appending a step's keys and values to the cache, keys and queries rotated to their positions on the way.
//
// Mathematics.  Band f of a row (x_re, x_im) at position p becomes (x_re + i x_im) e^{i omega_f p} (Section 2.1).  The
// angle is taken in turns, p * omega_f / 2 pi with the factor split into two doubles.  The factor is formed in the host's long
// double: with 64 bits of mantissa the turn's fraction is good to 3e-11 at p = 2^31 (worst of bases 1e4 .. 1e7 against 60 digits),
// far below fp32.  Its fp32 value and the rest of it give cos and sin to about one unit in the last place.
// The rotation itself is fp32 (2 multiplications, 2 FMAs per pair) and the result is rounded once to the cache's format.
//
// Shape of the work.  Pure streaming: every byte of k, v, q is read once and every cache row written once, so the kernel
// is bound by memory, or by launch latency for a single token.  Eight lanes own one row of 128 components, 16
// components (8 bands) each: whole 32-byte sectors on both sides.  A block covers TT tokens of one sequence and all of
// its rows (H keys, H values, H * G queries), so that the sines and cosines of a token are formed once, by one thread per
// band, and used from registers for every head.
#pragma once
#include "tri_score_tma.cuh"
#include "tri_step.cuh"

namespace tri {

constexpr int kAppendThreads = 256;
// Tokens per block when a call brings several.  (2 to 7 tokens leave places of a block idle: 64 sequences take 5.2 to 5.7 us in
// bf16 and 8.3 to 8.5 in e4m3, back to back, where one token takes 3.0 and 3.9 with a block of its own; fewer places were not
// measured.)
constexpr int kAppendTokens = 8;

struct AppendParams {
    View dst;
    int32_t layer, S, H, G, T, ntiles;
    const int32_t *unit_lens;                    // [S][H] of this layer or NULL
    const float *k_scale, *v_scale;              // [H] of this layer or NULL
    const char *k, *v, *q;
    char *q_out;
    int64_t ks_seq, ks_tok, ks_head, vs_seq, vs_tok, vs_head, qs_seq, qs_tok, qs_head, qo_seq, qo_tok, qo_head;
    const int32_t *n_new;
    const int64_t *pos;
    const double2 *turn;                         // [64] omega_f / 2 pi as hi + lo
    int32_t *new_lens;                           // NULL where k_append_lens writes them
    int32_t *device_status;
};

__device__ __forceinline__ int append_len(const AppendParams &p, int s, int h)
{
    const int n = p.unit_lens ? p.unit_lens[(int64_t)s * p.H + h] : p.dst.seq_lens[s];
    return min(max(n, 0), p.dst.n_max);
}
__device__ __forceinline__ int append_count(const AppendParams &p, int s)
{
    return p.n_new ? min(max(p.n_new[s], 0), p.T) : p.T;
}

// The 16 components a lane owns of a row.  SPLIT: components 8c..8c+7 and 64+8c..64+8c+7 (the two halves of 8 bands in the
// half-split layout), else 16c..16c+15.
template <int KIND> struct Raw16 { uint4 v[KIND == 0 ? 2 : 4]; };
template <int KIND, bool SPLIT>
__device__ __forceinline__ void load16(const char *row, int c, Raw16<KIND> &x)
{
    const int first = SPLIT ? 8 * c : 16 * c, second = SPLIT ? 64 + 8 * c : 16 * c + 8;
    if constexpr (KIND == 0) {
        x.v[0] = *reinterpret_cast<const uint4 *>(row + 2 * first);
        x.v[1] = *reinterpret_cast<const uint4 *>(row + 2 * second);
    } else {
        x.v[0] = *reinterpret_cast<const uint4 *>(row + 4 * first);
        x.v[1] = *reinterpret_cast<const uint4 *>(row + 4 * first + 16);
        x.v[2] = *reinterpret_cast<const uint4 *>(row + 4 * second);
        x.v[3] = *reinterpret_cast<const uint4 *>(row + 4 * second + 16);
    }
}
template <int KIND>
__device__ __forceinline__ void widen16(const Raw16<KIND> &r, float (&x)[16])
{
#pragma unroll
    for (int i = 0; i < (KIND == 0 ? 2 : 4); ++i) {
        const uint32_t w[4] = {r.v[i].x, r.v[i].y, r.v[i].z, r.v[i].w};
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            if constexpr (KIND == 0) { x[8 * i + 2 * y] = bf16_lo(w[y]); x[8 * i + 2 * y + 1] = bf16_hi(w[y]); }
            else x[4 * i + y] = __uint_as_float(w[y]);
        }
    }
}

// Four fp32 values as e4m3 bytes, to nearest even, saturating at +-448 (NaN stays NaN).
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d)
{
    uint32_t r;
    asm("{\n.reg .b16 l, h;\ncvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\ncvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n"
        "mov.b32 %0, {l, h};\n}\n" : "=r"(r) : "f"(a), "f"(b), "f"(c), "f"(d));
    return r;
}

// Stores the 16 components to a row of bytes per element ES: 2 = bf16, 1 = e4m3, 4 = fp32.
template <int ES, bool SPLIT>
__device__ __forceinline__ void store16(char *row, int c, const float (&x)[16])
{
    const int first = SPLIT ? 8 * c : 16 * c, second = SPLIT ? 64 + 8 * c : 16 * c + 8;
    if (ES == 2) {
        *reinterpret_cast<uint4 *>(row + 2 * first) =
            make_uint4(cvt_bf16x2(x[1], x[0]), cvt_bf16x2(x[3], x[2]), cvt_bf16x2(x[5], x[4]), cvt_bf16x2(x[7], x[6]));
        *reinterpret_cast<uint4 *>(row + 2 * second) =
            make_uint4(cvt_bf16x2(x[9], x[8]), cvt_bf16x2(x[11], x[10]), cvt_bf16x2(x[13], x[12]), cvt_bf16x2(x[15], x[14]));
    } else if (ES == 1) {
        *reinterpret_cast<uint2 *>(row + first) = make_uint2(e4m3x4(x[0], x[1], x[2], x[3]), e4m3x4(x[4], x[5], x[6], x[7]));
        *reinterpret_cast<uint2 *>(row + second) = make_uint2(e4m3x4(x[8], x[9], x[10], x[11]), e4m3x4(x[12], x[13], x[14], x[15]));
    } else {
        *reinterpret_cast<float4 *>(row + 4 * first) = make_float4(x[0], x[1], x[2], x[3]);
        *reinterpret_cast<float4 *>(row + 4 * first + 16) = make_float4(x[4], x[5], x[6], x[7]);
        *reinterpret_cast<float4 *>(row + 4 * second) = make_float4(x[8], x[9], x[10], x[11]);
        *reinterpret_cast<float4 *>(row + 4 * second + 16) = make_float4(x[12], x[13], x[14], x[15]);
    }
}

// Bands 8c .. 8c+7 of the 16 components: pair j is (x[2j], x[2j+1]) interleaved, (x[j], x[j+8]) half-split.
template <bool SPLIT>
__device__ __forceinline__ void rotate16(float (&x)[16], const float2 (&cs)[8])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int ir = SPLIT ? j : 2 * j, ii = SPLIT ? j + 8 : 2 * j + 1;
        const float re = x[ir], im = x[ii];
        x[ir] = fmaf(cs[j].x, re, -(cs[j].y * im));
        x[ii] = fmaf(cs[j].y, re, cs[j].x * im);
    }
}

// KIND: input 0 bf16, 1 fp32.  KK: the cache's k_kind.  TT: tokens per block.
template <int KIND, int KK, bool SPLIT, int TT>
__global__ void __launch_bounds__(kAppendThreads) k_append(const AppendParams p)
{
    constexpr int kES = KK == 1 ? 4 : (KK == 3 ? 1 : 2), vES = KK == 3 ? 1 : 2;
    constexpr bool kRotateKeys = KK == 0 || KK == 3;
    constexpr int kGroups = kAppendThreads / 8 / TT;          // row groups (of 8 lanes) per token
    __shared__ float2 cs_s[TT][kBands];

    const int tid = threadIdx.x, c = tid & 7;
    const int s = blockIdx.x / p.ntiles, t0 = (blockIdx.x - s * p.ntiles) * TT;
    grid_dependency_wait();                                   // set up under the kernel before it in the stream, as the next is under this one
    grid_dependents_launch();
    const int n_new = append_count(p, s);
    const bool first = t0 == 0;
    if (first && tid == 0 && p.device_status && p.n_new) {
        const int raw = p.n_new[s];
        if (raw < 0 || raw > p.T) atomicExch(p.device_status, (int)TRI_ERR_DEVICE_CHECK);
    }
    if (t0 < n_new) {
        const int64_t p0 = p.pos ? p.pos[s] : (int64_t)append_len(p, s, 0);
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
            cs_s[i >> 6][f] = make_float2(fmaf(-d, sn, cn), fmaf(d, cn, sn));
        }
        __syncthreads();
        const int tt = tid / (8 * kGroups), grp = (tid >> 3) % kGroups, t = t0 + tt;
        const int64_t at = p0 + t;
        const bool pos_ok = at >= 0 && at <= 0x7fffffff;
        if (t < n_new && !pos_ok && p.device_status) atomicExch(p.device_status, (int)TRI_ERR_DEVICE_CHECK);
        if (t < n_new && pos_ok) {
            constexpr int in_es = KIND == 0 ? 2 : 4, U = KIND == 0 ? 6 : 2;      // rows in flight per lane (2: 18 % slower, 4: 3 %)
            const int kv = p.v ? 2 * p.H : p.H;               // rows: H keys, H values, then the queries
            const int rows = kv + (p.q ? p.H * p.G : 0);
            // where head 0's row goes when all heads have the same length
            int64_t slot0 = 0, off0 = -1;
            if (!p.unit_lens) {
                slot0 = (int64_t)append_len(p, s, 0) + t;
                if (slot0 < p.dst.n_max) off0 = step_row_offset(p.dst, p.layer, s, 0, (int)slot0);
            }
            float2 cs[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) cs[j] = cs_s[tt][8 * c + j];
            const char *q = p.q + (s * p.qs_seq + t * p.qs_tok) * in_es, *k = p.k + (s * p.ks_seq + t * p.ks_tok) * in_es,
                       *v = p.v + (s * p.vs_seq + t * p.vs_tok) * in_es;
            for (int r0 = grp; r0 < rows; r0 += U * kGroups) {
                Raw16<KIND> raw[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int r = r0 + u * kGroups;
                    if (r >= rows) break;
                    const char *src = r < p.H ? k + r * p.ks_head * in_es : (r < kv ? v + (r - p.H) * p.vs_head * in_es : q + (r - kv) * p.qs_head * in_es);
                    load16<KIND, SPLIT>(src, c, raw[u]);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int r = r0 + u * kGroups;
                    if (r >= rows) break;
                    float x[16];
                    widen16<KIND>(raw[u], x);
                    if (r >= kv) {
                        rotate16<SPLIT>(x, cs);
                        store16<2, SPLIT>(p.q_out + (s * p.qo_seq + t * p.qo_tok + (r - kv) * p.qo_head) * 2, c, x);
                        continue;
                    }
                    const bool is_k = r < p.H;
                    const int h = is_k ? r : r - p.H;
                    int64_t slot = slot0, off = off0 == -1 ? -1 : off0 + h * p.dst.stride_head;
                    if (p.unit_lens) {
                        slot = (int64_t)append_len(p, s, h) + t;
                        off = slot < p.dst.n_max ? step_row_offset(p.dst, p.layer, s, h, (int)slot) : -1;
                    }
                    if (off == -1) {                          // (offsets are multiples of 8 elements)
                        if (p.device_status) atomicExch(p.device_status, (int)TRI_ERR_DEVICE_CHECK);
                        continue;
                    }
                    if (is_k && kRotateKeys) rotate16<SPLIT>(x, cs);
                    if (KK == 3) {
                        const float *sc = is_k ? p.k_scale : p.v_scale;
                        if (sc) {
                            const float scale = sc[h];
#pragma unroll
                            for (int i = 0; i < 16; ++i) x[i] = __fdiv_rn(x[i], scale);
                        }
                    }
                    if (is_k) store16<kES, SPLIT>(p.dst.k + off * kES, c, x);
                    else store16<vES, SPLIT>(p.dst.v + off * vES, c, x);
                    if (is_k && c == 0 && p.dst.positions)
                        p.dst.positions[(((int64_t)p.layer * p.S + s) * p.H + h) * p.dst.n_max + slot] = (int32_t)at;
                }
            }
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

// Lengths in place after an append whose blocks share sequences: a launch of its own, set up under the one that reads them.
__global__ void __launch_bounds__(256) k_append_lens(const AppendParams p)
{
    grid_dependency_wait();
    grid_dependents_launch();
    const int n = p.unit_lens ? p.H : 1;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (int64_t)p.S * n) return;
    const int s = (int)(i / n);
    const int64_t len = (int64_t)append_len(p, s, (int)(i - (int64_t)s * n)) + append_count(p, s);
    p.new_lens[i] = (int32_t)(len < p.dst.n_max ? len : p.dst.n_max);
}

}  // namespace tri
