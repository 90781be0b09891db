// Reading cached rows back, in any format of a cache.
//
// Pure streaming: a row is read once (80 bytes in 4 bits, 128 in e4m3, 256 in bf16) and written once (256 or 512 bytes), so the
// kernel is bound by the writes: 16 sequences of 8 heads, up to 8,192 rows in 4 bits to bf16, 413 MB, take 70 us, 5.9 TB/s (0.91 of
// the copy rate).  Eight lanes own a row, 16 components each, and store them as two (bf16) or four (fp32) runs of 16
// bytes; a thread has the keys and the values of kReadRows rows in flight before it stores the first.  A block covers kReadTile
// rows: neighbouring tokens of one head, or, where a call reads few tokens, those of several heads.
#pragma once
#include "tri_append.cuh"
#include "tri_row4.cuh"
#include "tri_step.cuh"

namespace tri {

constexpr int kReadThreads = 256, kReadRows = 2, kReadTile = kReadThreads / 8 * kReadRows;

struct ReadParams {
    View src;
    int32_t layer, S, H, T;
    int32_t tok_shift;                           // a block covers 2^tok_shift tokens of kReadTile >> tok_shift heads
    int32_t tiles_t, tiles_h;
    const int32_t *unit_lens;                    // [S][H] of this layer or NULL
    const float *k_scale, *v_scale;              // [H] of this layer or NULL
    char *k, *v;
    int64_t ks_seq, ks_tok, ks_head, vs_seq, vs_tok, vs_head;
    const int32_t *first;
    int32_t *device_status;
};

// What a lane loads of a row in format F (a view's k_kind), and the 16 components it then has: 8 from `at`, 8 from `at + gap`.
template <int F> struct ReadRaw { Raw16<F == 1 ? 1 : 0> r; };
template <> struct ReadRaw<3> { uint4 r; };
template <> struct ReadRaw<5> { uint2 codes; uint32_t s, c; };

template <int F>
__device__ __forceinline__ void read_load(const char *row, int c, ReadRaw<F> &x)
{
    if constexpr (F == 5) {                                  // unit c / 2, words of groups 2 (c % 2), + 1
        x.codes = *reinterpret_cast<const uint2 *>(row + 8 * c);
        x.s = *reinterpret_cast<const uint32_t *>(row + kRow4Scales + 4 * (c & 1));
        x.c = *reinterpret_cast<const uint32_t *>(row + kRow4Centres + 4 * (c & 1));
    } else if constexpr (F == 3) {
        x.r = *reinterpret_cast<const uint4 *>(row + 16 * c);
    } else {
        load16<F == 1 ? 1 : 0, false>(row, c, x.r);
    }
}
template <int F>
__device__ __forceinline__ void read_widen(const ReadRaw<F> &raw, float scale, float (&x)[16])
{
    if constexpr (F == 5) {
        row4_values(raw.codes.x, bf16_lo(raw.s), bf16_lo(raw.c), x);
        row4_values(raw.codes.y, bf16_hi(raw.s), bf16_hi(raw.c), x + 8);
    } else if constexpr (F == 3) {
        const uint32_t w[4] = {raw.r.x, raw.r.y, raw.r.z, raw.r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t a, b;
            e4m3x4_to_f16x2(w[i], a, b);
            x[4 * i] = f16_value(a & 0xffffu) * scale; x[4 * i + 1] = f16_value(a >> 16) * scale;
            x[4 * i + 2] = f16_value(b & 0xffffu) * scale; x[4 * i + 3] = f16_value(b >> 16) * scale;
        }
    } else {
        widen16<F == 1 ? 1 : 0>(raw.r, x);
    }
}
// Components at .. at + 7 and at + gap .. + 7 to a row of elements of OS bytes.
template <int F, int OS>
__device__ __forceinline__ void read_store(char *row, int c, const float (&x)[16])
{
    const int at = F == 5 ? 64 * (c & 1) + 8 * (c >> 1) : 16 * c, gap = F == 5 ? 32 : 8;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float *y = x + 8 * i;
        char *to = row + (at + gap * i) * OS;
        if (OS == 2) {
            *reinterpret_cast<uint4 *>(to) = make_uint4(cvt_bf16x2(y[1], y[0]), cvt_bf16x2(y[3], y[2]), cvt_bf16x2(y[5], y[4]), cvt_bf16x2(y[7], y[6]));
        } else {
            *reinterpret_cast<float4 *>(to) = make_float4(y[0], y[1], y[2], y[3]);
            *reinterpret_cast<float4 *>(to + 16) = make_float4(y[4], y[5], y[6], y[7]);
        }
    }
}

// A loaded row to elements of OS bytes.
template <int F, int OS>
__device__ __forceinline__ void read_put(char *row, int c, const ReadRaw<F> &raw, float scale)
{
    if constexpr (F == 5 && OS == 2) {
        char *to = row + (64 * (c & 1) + 8 * (c >> 1)) * 2;
        *reinterpret_cast<uint4 *>(to) = row4_bf16(raw.codes.x, __byte_perm(raw.s, 0, 0x1010), __byte_perm(raw.c, 0, 0x1010));
        *reinterpret_cast<uint4 *>(to + 64) = row4_bf16(raw.codes.y, __byte_perm(raw.s, 0, 0x3232), __byte_perm(raw.c, 0, 0x3232));
    } else {
        float x[16];
        read_widen<F>(raw, scale, x);
        read_store<F, OS>(row, c, x);
    }
}

// KK: the cache's k_kind.  OS: bytes per element of the outputs.
template <int KK, int OS>
__global__ void __launch_bounds__(kReadThreads) k_read(const ReadParams p)
{
    constexpr int VK = KK == 3 || KK == 5 ? KK : 0, U = kReadRows;
    constexpr int kES = KK == 1 ? 4 : (KK == 3 || KK == 5 ? 1 : 2), vES = VK == 0 ? 2 : 1;
    grid_dependency_wait();
    grid_dependents_launch();
    const int tid = threadIdx.x, c = tid & 7, grp = tid >> 3;
    const int tile = blockIdx.x % p.tiles_t, rest = blockIdx.x / p.tiles_t, s = rest / p.tiles_h;
    const int t_block = tile << p.tok_shift, h_block = (rest - s * p.tiles_h) * (kReadTile >> p.tok_shift);
    const int first = p.first ? max(ld_here(p.first + s), 0) : 0;
    int64_t off[U];                                       // of the row in the cache; -1: none
    ReadRaw<KK> rk[U];
    ReadRaw<VK> rv[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i = grp + u * (kReadThreads / 8), t = t_block + (i & ((1 << p.tok_shift) - 1)), h = h_block + (i >> p.tok_shift);
        off[u] = -1;
        if (h >= p.H || t >= p.T) continue;
        const int len = min(ld_here(p.unit_lens ? p.unit_lens + (int64_t)s * p.H + h : p.src.seq_lens + s), p.src.n_max);
        const int64_t slot = (int64_t)first + t;
        if (slot >= len) continue;
        off[u] = step_row_offset(p.src, p.layer, s, h, (int)slot);
        if (off[u] == -1) {
            if (p.device_status) atomicExch(p.device_status, (int)TRI_ERR_DEVICE_CHECK);
            continue;
        }
        if (p.k) read_load<KK>(p.src.k + off[u] * kES, c, rk[u]);
        if (p.v) read_load<VK>(p.src.v + off[u] * vES, c, rv[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (off[u] == -1) continue;
        const int i = grp + u * (kReadThreads / 8), t = t_block + (i & ((1 << p.tok_shift) - 1)), h = h_block + (i >> p.tok_shift);
        if (p.k) read_put<KK, OS>(p.k + (s * p.ks_seq + t * p.ks_tok + h * p.ks_head) * OS, c, rk[u], p.k_scale ? p.k_scale[h] : 1.f);
        if (p.v) read_put<VK, OS>(p.v + (s * p.vs_seq + t * p.vs_tok + h * p.vs_head) * OS, c, rv[u], p.v_scale ? p.v_scale[h] : 1.f);
    }
}

}  // namespace tri
