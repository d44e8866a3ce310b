// Causal attention of fp32 tokens over fp32 keys and values, tiles of 32 rows: the transposed
// products of attn_tile.hip on the 16x16x4 fp32 MFMA, whose products and sums are fp32
// throughout.  Lane group g takes elements 4g..4g+3 of every 16 of the head dimension (one 16-byte
// read feeds four MFMAs), and an accumulator's register i holds key 4g + i, which makes it the B
// operand of the i-th product with V^T.  Two waves share 16 rows, each with half of every tile of 64
// keys and a softmax of its own, joined at the end: the calls are small, and the chain of tiles
// bounds them before the matrix rate of fp32 does (four sequences of 100 to 700 tokens, 8 heads of 64:
// 36 us; with one wave per 16 rows and no tile ahead 64).  The next tile is loaded into registers
// while one is worked on.
#include "attn_device.h"

namespace lkv {

namespace {
constexpr int NW = 4, BM = ATTN_ROWS_F32, BN = 64, HN = BN / 2;  // HN: keys of a wave
static_assert(BM == 8 * NW, "two waves own 16 rows");
}  // namespace

template <int D, bool PAGED>
__global__ __launch_bounds__(64 * NW) void attn_f32_kernel(AttnArgs p) {
    constexpr int NT = HN / 16, ND = D / 16, LD = D + 4;  // LDS rows padded by one 16-byte chunk
    constexpr int PER = BN * (D / 4) / (64 * NW);
    __shared__ __align__(16) float sk[BN * LD], sv[BN * LD];
    __shared__ int s_end[NW];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int col = lane & 15, g = lane >> 4, half = wave >> 1;  // of the keys

    int b = blockIdx.x;
    const int hk = b % p.h_kv;
    b /= p.h_kv;
    const int split = PAGED ? b % p.splits : 0;
    const int u = PAGED ? b / p.splits : b;
    const AttnUnit w = attn_unit<BM>(p, u, lane);
    if (w.r < 0) return;
    const int len = PAGED ? attn_len(p.pg, w.r) : w.n;
    const AttnRow row = attn_row<PAGED>(p, w, w.row0 + 16 * (wave & 1) + col, hk, len);
    const int sees = row.kind == ROW_SEES ? row.pos + 1 : 0;
    const int wave_end = wave_max_int(sees);
    const int wave_all = wave_min_int(row.kind == ROW_SEES ? sees : 0x7fffffff);
    if (lane == 0) s_end[wave] = wave_end;
    __syncthreads();
    int end = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) end = max(end, s_end[i]);
    const KeyRange range = key_range<BN>(end, PAGED ? p.splits : 1, split);

    f32x4 kr[PER], vr[PER];
    bool bad_page = false;
    auto load = [&](int j0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int x = tid + i * 64 * NW, r = x / (D / 4), c = x % (D / 4);
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
            kr[i] = *reinterpret_cast<const f32x4*>(k + 4 * c);
            vr[i] = *reinterpret_cast<const f32x4*>(v + 4 * c);
        }
    };
    if (range.from < range.to) load(range.from);

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
    const int my_pos = row.kind == ROW_SEES ? row.pos : 0x7fffffff;

    for (int tile = range.from; tile < range.to; tile += BN) {
        bool bad_v = false;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int x = tid + i * 64 * NW, r = x / (D / 4), c = x % (D / 4);
            const u32x4 bits = __builtin_bit_cast(u32x4, vr[i]);
#pragma unroll
            for (int e = 0; e < 4; ++e) bad_v |= (bits[e] & 0x7f800000u) == 0x7f800000u;
            *reinterpret_cast<f32x4*>(sk + r * LD + 4 * c) = kr[i];
            *reinterpret_cast<f32x4*>(sv + r * LD + 4 * c) = vr[i];
        }
        bad_v = __syncthreads_or(bad_v);
        if (tile + BN < range.to) load(tile + BN);
        const int j0 = tile + HN * half;  // the wave's first key
        const bool masked = j0 + HN > wave_all;
        if (j0 >= wave_end) continue;
        const float *kt = sk + HN * half * LD, *vt = sv + HN * half * LD;

        f32x4 st[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            st[t] = zero4();
#pragma unroll
            for (int s = 0; s < D / 16; ++s) {
                const f32x4 kf = lds4f(kt + (16 * t + col) * LD + 16 * s + 4 * g);
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
                    float v = vt[(16 * t + 4 * g + i) * LD + 16 * d + col];
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

    // join of the two halves
    __shared__ float s_m[2][16], s_l[2][16];
    __syncthreads();
    float* so = sk + (wave & 1) * 16 * LD;
    if (half == 1) {
        if (g == 0) s_m[wave & 1][col] = m, s_l[wave & 1][col] = l;
#pragma unroll
        for (int t = 0; t < ND; ++t) *reinterpret_cast<f32x4*>(so + col * LD + 16 * t + 4 * g) = ot[t];
    }
    __syncthreads();
    if (half == 1 || row.kind == ROW_NONE) return;
    const float m2 = s_m[wave & 1][col], m_all = fmaxf(m, m2), m_use = m_all == -INFINITY ? 0.f : m_all;
    const float f1 = __builtin_amdgcn_exp2f(m - m_use), f2 = __builtin_amdgcn_exp2f(m2 - m_use);
    l = f1 * l + f2 * s_l[wave & 1][col];
#pragma unroll
    for (int t = 0; t < ND; ++t) ot[t] = f1 * ot[t] + f2 * *reinterpret_cast<const f32x4*>(so + col * LD + 16 * t + 4 * g);
    if (row.kind == ROW_NAN) l = NAN;
    if (row.kind == ROW_ZERO) l = 0.f;
    if (PAGED && p.splits > 1) {
        const int64_t at = (int64_t)split * p.n_tok * p.h_q + row.tok * p.h_q + row.head;
        const float stored = part_sum(l, row, range);
        if (g == 0) {
            p.part_ml[2 * at] = row.kind == ROW_ZERO ? -INFINITY : m_all;
            p.part_ml[2 * at + 1] = stored;
        }
        if (stored == 0.f) return;
#pragma unroll
        for (int t = 0; t < ND; ++t) *reinterpret_cast<f32x4*>(p.part_o + at * D + 16 * t + 4 * g) = ot[t];
        return;
    }
    const float inv = l == 0.f ? 1.f : 1.f / l;  // as in attn_tile.hip
    float* o = reinterpret_cast<float*>(p.o) + (row.tok * p.h_q + row.head) * D;
#pragma unroll
    for (int t = 0; t < ND; ++t) *reinterpret_cast<f32x4*>(o + 16 * t + 4 * g) = row.kind == ROW_ZERO ? zero4() : ot[t] * inv;
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

}  // namespace lkv
