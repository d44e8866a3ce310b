// Causal attention of fp32 tokens over fp32 keys and values, tiles of 64 rows: the transposed
// products of attn_tile.hip on the 16x16x4 fp32 MFMA, whose products and sums are fp32
// throughout.  A wave owns 16 rows.  Lane group g takes elements 4g..4g+3 of every 16 of the
// head dimension (one 16-byte read feeds four MFMAs), and an accumulator's register i holds key
// 4g + i, which makes it the B operand of the i-th product with V^T.  The matrix rate of fp32
// bounds it (a sixteenth of bf16's).
#include "attn_device.h"

namespace lkv {

namespace {
constexpr int NW = 4, BM = ATTN_ROWS_F32, BN = 32;
static_assert(BM == 16 * NW, "a wave owns 16 rows");
}  // namespace

template <int D, bool PAGED>
__global__ __launch_bounds__(64 * NW) void attn_f32_kernel(AttnArgs p) {
    constexpr int NT = BN / 16, ND = D / 16, LD = D + 4;  // LDS rows padded by one 16-byte chunk
    __shared__ __align__(16) float sk[BN * LD], sv[BN * LD];
    __shared__ int s_end[NW];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int col = lane & 15, g = lane >> 4;

    int b = blockIdx.x;
    const int hk = b % p.h_kv;
    b /= p.h_kv;
    const int split = PAGED ? b % p.splits : 0;
    const int u = PAGED ? b / p.splits : b;
    const AttnUnit w = attn_unit<BM>(p.cu, p.n_req, p.n_tok, p.group, u, lane);
    if (w.r < 0) return;
    const int len = PAGED ? attn_len(p.pg, w.r) : w.n;
    const AttnRow row = attn_row<PAGED>(p, w, w.row0 + 16 * wave + col, hk, len);
    const int sees = row.kind == ROW_SEES ? row.pos + 1 : 0;
    const int wave_end = wave_max_int(sees);
    const int wave_all = wave_min_int(row.kind == ROW_SEES ? sees : 0x7fffffff);
    if (lane == 0) s_end[wave] = wave_end;
    __syncthreads();
    int end = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) end = max(end, s_end[i]);
    const KeyRange range = key_range<BN>(end, PAGED ? p.splits : 1, split);

    f32x4 qf[D / 16];
#pragma unroll
    for (int s = 0; s < D / 16; ++s) qf[s] = zero4();
    if (row.kind != ROW_NONE) {
        const float* q = reinterpret_cast<const float*>(p.q) + row.tok * p.q_stride + (int64_t)row.head * D;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) qf[s] = *reinterpret_cast<const f32x4*>(q + 16 * s + 4 * g);
    }
    f32x4 ot[ND];
#pragma unroll
    for (int t = 0; t < ND; ++t) ot[t] = zero4();
    float m = -INFINITY, l = 0.f;
    bool bad_page = false;
    const int my_pos = row.kind == ROW_SEES ? row.pos : 0x7fffffff;

    for (int j0 = range.from; j0 < range.to; j0 += BN) {
        bool bad_v = false;
        __syncthreads();
        for (int x = tid; x < BN * (D / 4); x += 64 * NW) {
            const int r = x / (D / 4), c = x % (D / 4);
            const int j = min(j0 + r, end - 1);  // rows past the last key seen repeat it
            const float *k, *v;
            if (!PAGED) {
                k = reinterpret_cast<const float*>(p.k) + (w.t0 + j) * p.k_stride + (int64_t)hk * D;
                v = reinterpret_cast<const float*>(p.v) + (w.t0 + j) * p.v_stride + (int64_t)hk * D;
            } else {
                int page = p.pg.table[(int64_t)w.r * p.pg.max_pages + (j >> p.pg.page_shift)];
                const bool ok = page >= 0 && page < p.pg.n_page;
                bad_page |= !ok;
                page = ok ? page : 0;
                const int64_t at = (((int64_t)page * p.h_kv + hk) << p.pg.page_shift) + (j & ((1 << p.pg.page_shift) - 1));
                k = reinterpret_cast<const float*>(p.pg.k) + at * D;
                v = reinterpret_cast<const float*>(p.pg.v) + at * D;
            }
            const f32x4 kc = *reinterpret_cast<const f32x4*>(k + 4 * c), vc = *reinterpret_cast<const f32x4*>(v + 4 * c);
            const u32x4 bits = __builtin_bit_cast(u32x4, vc);
#pragma unroll
            for (int i = 0; i < 4; ++i) bad_v |= (bits[i] & 0x7f800000u) == 0x7f800000u;
            *reinterpret_cast<f32x4*>(sk + r * LD + 4 * c) = kc;
            *reinterpret_cast<f32x4*>(sv + r * LD + 4 * c) = vc;
        }
        const bool masked = j0 + BN > wave_all;
        bad_v = __syncthreads_or(bad_v);
        if (j0 >= wave_end) continue;

        f32x4 st[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            st[t] = zero4();
#pragma unroll
            for (int s = 0; s < D / 16; ++s) {
                const f32x4 kf = lds4f(sk + (16 * t + col) * LD + 16 * s + 4 * g);
#pragma unroll
                for (int i = 0; i < 4; ++i) st[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[i], qf[s][i], st[t], 0, 0, 0);
            }
        }
        float top = -INFINITY;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (masked && j0 + 16 * t + 4 * g + i > my_pos) st[t][i] = -INFINITY;
                top = fmaxf(top, st[t][i]);
            }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float m_new = fmaxf(m, top * p.scale_log2);
        const float m_use = m_new == -INFINITY ? 0.f : m_new;
        const float scale = __builtin_amdgcn_exp2f(m - m_use);
        m = m_new;
        l *= scale;
#pragma unroll
        for (int t = 0; t < ND; ++t) ot[t] *= scale;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                st[t][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[t][i], p.scale_log2, -m_use));
                l += st[t][i];
            }
#pragma unroll
        for (int d = 0; d < ND; ++d) {
            f32x4 count = zero4();
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v = sv[(16 * t + 4 * g + i) * LD + 16 * d + col];
                    if (masked && bad_v) {  // as in attn_tile.hip
                        const bool bad = (__builtin_bit_cast(uint32_t, v) & 0x7f800000u) == 0x7f800000u;
                        const float seen = j0 + 16 * t + 4 * g + i <= my_pos ? 1.f : 0.f;
                        count = __builtin_amdgcn_mfma_f32_16x16x4f32(bad ? 1.f : 0.f, seen, count, 0, 0, 0);
                        v = bad ? 0.f : v;
                    }
                    ot[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, st[t][i], ot[d], 0, 0, 0);
                }
            if (masked && bad_v)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (count[i] > 0.f) ot[d][i] = NAN;
        }
    }
    if (PAGED && __syncthreads_or(bad_page)) l = NAN;
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (row.kind == ROW_NONE) return;
    if (PAGED && p.splits > 1) {
        const int64_t at = (int64_t)split * p.n_tok * p.h_q + row.tok * p.h_q + row.head;
        if (row.kind == ROW_NAN) l = NAN;
        if (row.kind == ROW_ZERO) l = 0.f, m = -INFINITY;
        if (g == 0) {
            p.part_ml[2 * at] = m;
            p.part_ml[2 * at + 1] = l;
        }
        if (l == 0.f) return;
#pragma unroll
        for (int t = 0; t < ND; ++t) *reinterpret_cast<f32x4*>(p.part_o + at * D + 16 * t + 4 * g) = ot[t];
        return;
    }
    float inv = l == 0.f ? 0.f : 1.f / l;
    if (row.kind == ROW_NAN) inv = NAN;
    const bool zero = row.kind == ROW_ZERO || l == 0.f;
    float* o = reinterpret_cast<float*>(p.o) + (row.tok * p.h_q + row.head) * D;
#pragma unroll
    for (int t = 0; t < ND; ++t) *reinterpret_cast<f32x4*>(o + 16 * t + 4 * g) = zero ? zero4() : ot[t] * inv;
}

hipError_t launch_attn_f32(int d, bool paged, const AttnArgs& a, hipStream_t st) {
    const dim3 grid((unsigned)((int64_t)a.n_units * a.h_kv * (paged ? a.splits : 1))), block(64 * NW);
    if (d == 64 && paged) hipLaunchKernelGGL((attn_f32_kernel<64, true>), grid, block, 0, st, a);
    else if (d == 64) hipLaunchKernelGGL((attn_f32_kernel<64, false>), grid, block, 0, st, a);
    else if (d == 128 && paged) hipLaunchKernelGGL((attn_f32_kernel<128, true>), grid, block, 0, st, a);
    else if (d == 128) hipLaunchKernelGGL((attn_f32_kernel<128, false>), grid, block, 0, st, a);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

// Join of the key ranges' results: with m = max m_s, o = sum 2^(m_s - m) o_s / sum 2^(m_s - m) l_s.
// A workgroup joins one row: every wave forms all weights, a part per lane, and adds a quarter of
// the parts, whose loads do not wait for each other; the quarters meet in LDS.  Short chains of
// loads are what counts here: a decoding call waits for it.
constexpr int JOIN_PARTS = 128;
template <int D, typename T>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs p) {
    constexpr int E = D / 64;  // elements of a lane
    __shared__ float so[3][D];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t rows = p.n_tok * p.h_q, at = blockIdx.x;
    const int64_t tok = at / p.h_q;
    if (tok < clamp_tok(p.cu[0], 0, p.n_tok) || tok >= clamp_tok(p.cu[p.n_req], 0, p.n_tok)) return;
    float ms[JOIN_PARTS / 64], ls[JOIN_PARTS / 64], m = -INFINITY;
#pragma unroll
    for (int i = 0; i < JOIN_PARTS / 64; ++i) {
        const int s = lane + 64 * i;
        const bool in = s < p.splits;
        ms[i] = in ? p.part_ml[2 * (s * rows + at)] : -INFINITY;
        ls[i] = in ? p.part_ml[2 * (s * rows + at) + 1] : 0.f;
        m = fmaxf(m, ms[i]);
    }
    for (int i = 1; i < 64; i <<= 1) m = fmaxf(m, __shfl_xor(m, i));
    const float m_use = m == -INFINITY ? 0.f : m;
    float f[JOIN_PARTS / 64], l = 0.f;
#pragma unroll
    for (int i = 0; i < JOIN_PARTS / 64; ++i) {
        f[i] = ls[i] == 0.f ? 0.f : __builtin_amdgcn_exp2f(ms[i] - m_use);
        l += f[i] * ls[i];
    }
    for (int i = 1; i < 64; i <<= 1) l += __shfl_xor(l, i);
    float o[E];
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.f;
    const float* part = p.part_o + at * D + E * lane;
#pragma unroll
    for (int i = 0; i < JOIN_PARTS / 64; ++i) {
        const int to = min(64 * (i + 1), p.splits);
        for (int s0 = 64 * i + wave; s0 < to; s0 += 32) {
            float y[8][E];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int s = min(s0 + 4 * k, to - 1);
#pragma unroll
                for (int e = 0; e < E; ++e) y[k][e] = part[s * rows * D + e];
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int s = s0 + 4 * k;
                const float w = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f[i]), s & 63));
#pragma unroll
                for (int e = 0; e < E; ++e) o[e] += s < to && w != 0.f ? w * y[k][e] : 0.f;  // parts without keys are not written
            }
        }
    }
    if (wave > 0)
#pragma unroll
        for (int e = 0; e < E; ++e) so[wave - 1][E * lane + e] = o[e];
    __syncthreads();
    if (wave > 0) return;
    const float inv = 1.f / l;
    T* out = reinterpret_cast<T*>(p.o) + at * D + E * lane;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int x = E * lane + e;
        out[e] = (T)(l == 0.f ? 0.f : (o[e] + so[0][x] + so[1][x] + so[2][x]) * inv);
    }
}

hipError_t launch_attn_join(int d, bool f32, const AttnArgs& a, hipStream_t st) {
    const dim3 grid((unsigned)(a.n_tok * a.h_q)), block(256);
    if (d == 64 && f32) hipLaunchKernelGGL((attn_join_kernel<64, float>), grid, block, 0, st, a);
    else if (d == 64) hipLaunchKernelGGL((attn_join_kernel<64, bf16>), grid, block, 0, st, a);
    else if (d == 128 && f32) hipLaunchKernelGGL((attn_join_kernel<128, float>), grid, block, 0, st, a);
    else if (d == 128) hipLaunchKernelGGL((attn_join_kernel<128, bf16>), grid, block, 0, st, a);
    else if (d == 256 && !f32) hipLaunchKernelGGL((attn_join_kernel<256, bf16>), grid, block, 0, st, a);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

}  // namespace lkv
