// Causal attention of bf16 tokens, tiles of 128 rows (see attn_device.h for the rows).
//
// One pass over the keys with the running maximum and sum of the softmax.  A wave owns 32 rows
// and works on transposed tiles: S^T = K Q^T and O^T = V^T P^T, both with the 32x32x16 bf16
// MFMA.  In an accumulator of S^T lane l holds one row's scores (column l % 32) of 16 keys, so
// the softmax reduces within the lane and once between the wave's halves, and the same
// registers, rounded to bf16, are the B operand of the second product: an accumulator's
// registers 8s..8s+7 hold keys 16s + 4h + (0..3) and 16s + 8 + 4h + (0..3) in half h, and V^T's
// fragment is read from LDS with transposing reads of just those keys.
//
// The scores, the softmax's statistics and O are fp32; the probabilities are rounded to bf16
// for the product (2^-9 of each, below the outputs' own rounding).
#include "attn_device.h"

namespace lkv {

namespace {

constexpr int NW = 4;            // waves
constexpr int BM = ATTN_ROWS;    // rows
static_assert(BM == 32 * NW, "a wave owns 32 rows");

// Position of 16-byte chunk c of row r in a tile of bf16 rows in LDS (in chunks).  K fragments
// are read as one chunk of 32 consecutive rows, V fragments as 4 adjacent chunks of 4 rows, twice:
// the chunks of a row are permuted so that either touches every bank equally.
template <int D>
__device__ __forceinline__ int k_chunk(int r, int c) {
    constexpr int C = D / 8;
    const int f = C >= 16 ? r & 15 : (r >> 1) & 7;
    return r * C + (c ^ f);
}
template <int D>
__device__ __forceinline__ int v_chunk(int r, int c) {
    constexpr int C = D / 8;
    const int f = C >= 16 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
    return r * C + (c ^ f);
}

// any bf16 of the four words infinite or NaN
__device__ __forceinline__ bool any_nonfinite(u32x4 x) {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bad |= (x[i] & 0x7f80u) == 0x7f80u;
        bad |= (x[i] & 0x7f800000u) == 0x7f800000u;
    }
    return bad;
}

typedef __attribute__((address_space(3))) lds_i16x4 lds_tr_t;
__device__ __forceinline__ bf16x4 tr_read(const u32x4* lds, int chunk, int half8) {
    const char* a = reinterpret_cast<const char*>(lds) + chunk * 16 + half8 * 8;
    return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr_t*)(a)));
}

}  // namespace

template <int D, int KIND, bool PAGED>
__global__ __launch_bounds__(64 * NW, 2) void attn_tile_kernel(AttnArgs p) {
    constexpr int BN = D == 256 ? 32 : 64;  // keys of a tile
    constexpr int NT = BN / 32, NS = D / 16, ND = D / 32, C = D / 8;
    constexpr int CHUNKS = BN * C, PER = CHUNKS / (64 * NW);
    __shared__ u32x4 sk[CHUNKS], sv[CHUNKS];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int col = lane & 31, h = lane >> 5;

    int b = blockIdx.x;
    const int hk = b % p.h_kv;
    b /= p.h_kv;
    const int split = PAGED ? b % p.splits : 0;
    const int u = PAGED ? b / p.splits : b;
    const AttnUnit w = attn_unit<BM>(p.cu, p.n_req, p.n_tok, p.group, u, lane);
    if (w.r < 0) return;
    const int len = PAGED ? attn_len(p.pg, w.r) : w.n;
    const AttnRow row = attn_row<PAGED>(p, w, w.row0 + 32 * wave + col, hk, len);

    // last key that the wave and the workgroup see, first key that some row of the wave does not
    __shared__ int s_end[NW];
    const int sees = row.kind == ROW_SEES ? row.pos + 1 : 0;
    const int wave_end = wave_max_int(sees);
    const int wave_all = wave_min_int(row.kind == ROW_SEES ? sees : 0x7fffffff);
    if (lane == 0) s_end[wave] = wave_end;
    __syncthreads();
    int end = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) end = max(end, s_end[i]);
    const KeyRange range = key_range<BN>(end, PAGED ? p.splits : 1, split);

    bf16x8 qf[NS];
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[s] = bf16x8{};
    if (row.kind != ROW_NONE) {
        const bf16* q = reinterpret_cast<const bf16*>(p.q) + row.tok * p.q_stride + (int64_t)row.head * D;
#pragma unroll
        for (int s = 0; s < NS; ++s) qf[s] = *reinterpret_cast<const bf16x8*>(q + 16 * s + 8 * h);
    }

    f32x16 ot[ND];
#pragma unroll
    for (int t = 0; t < ND; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) ot[t][i] = 0.f;
    float m = -INFINITY, l = 0.f;  // running maximum (scaled, base 2) and this half's sum
    bool bad_page = false;
    const int my_pos = row.kind == ROW_SEES ? row.pos : 0x7fffffff;

    for (int j0 = range.from; j0 < range.to; j0 += BN) {
        // stage K and V; rows past the last key seen repeat it
        bool bad_v = false;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int x = tid + i * 64 * NW, r = x / C, c = x % C;
            const int j = min(j0 + r, end - 1);
            u32x4 kc, vc;
            if (!PAGED) {
                kc = *reinterpret_cast<const u32x4*>(reinterpret_cast<const bf16*>(p.k) + (w.t0 + j) * p.k_stride +
                                                     (int64_t)hk * D + 8 * c);
                vc = *reinterpret_cast<const u32x4*>(reinterpret_cast<const bf16*>(p.v) + (w.t0 + j) * p.v_stride +
                                                     (int64_t)hk * D + 8 * c);
            } else {
                int page = p.pg.table[(int64_t)w.r * p.pg.max_pages + (j >> p.pg.page_shift)];
                const bool ok = page >= 0 && page < p.pg.n_page;
                bad_page |= !ok;
                page = ok ? page : 0;
                const int64_t at = (((int64_t)page * p.h_kv + hk) << p.pg.page_shift) + (j & ((1 << p.pg.page_shift) - 1));
                if (KIND == KV_E4M3) {
                    const u32x2 k8 = *reinterpret_cast<const u32x2*>(reinterpret_cast<const uint8_t*>(p.pg.k) + at * D + 8 * c);
                    const u32x2 v8 = *reinterpret_cast<const u32x2*>(reinterpret_cast<const uint8_t*>(p.pg.v) + at * D + 8 * c);
                    const float ks = exp_scale(p.pg.k_exp[at]), vs = exp_scale(p.pg.v_exp[at]);
                    kc = u32x4{e4m3_pair(k8[0], ks, false), e4m3_pair(k8[0], ks, true), e4m3_pair(k8[1], ks, false),
                               e4m3_pair(k8[1], ks, true)};
                    vc = u32x4{e4m3_pair(v8[0], vs, false), e4m3_pair(v8[0], vs, true), e4m3_pair(v8[1], vs, false),
                               e4m3_pair(v8[1], vs, true)};
                } else {
                    kc = *reinterpret_cast<const u32x4*>(reinterpret_cast<const bf16*>(p.pg.k) + at * D + 8 * c);
                    vc = *reinterpret_cast<const u32x4*>(reinterpret_cast<const bf16*>(p.pg.v) + at * D + 8 * c);
                }
            }
            bad_v |= any_nonfinite(vc);
            sk[k_chunk<D>(r, c)] = kc;
            sv[v_chunk<D>(r, c)] = vc;
        }
        const bool masked = j0 + BN > wave_all;
        bad_v = __syncthreads_or(bad_v);
        if (j0 >= wave_end) continue;

        f32x16 st[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int i = 0; i < 16; ++i) st[t][i] = 0.f;
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                const bf16x8 kf = __builtin_bit_cast(bf16x8, sk[k_chunk<D>(32 * t + col, 2 * s + h)]);
                st[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[s], st[t], 0, 0, 0);
            }
        }
        if (masked) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (j0 + 32 * t + 8 * (i >> 2) + 4 * h + (i & 3) > my_pos) st[t][i] = -INFINITY;
        }
        float top = -INFINITY;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, st[t][i]);
        top = fmaxf(top, __shfl_xor(top, 32));
        const float m_new = fmaxf(m, top * p.scale_log2);
        const float m_use = m_new == -INFINITY ? 0.f : m_new;  // only scores of -inf so far
        const float scale = __builtin_amdgcn_exp2f(m - m_use);
        m = m_new;
        l *= scale;
#pragma unroll
        for (int t = 0; t < ND; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) ot[t][i] *= scale;
        bf16x8 pf[2 * NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(st[t][i], p.scale_log2, -m_use));
                l += e;
                st[t][i] = e;
            }
#pragma unroll
            for (int s = 0; s < 2; ++s)
                pf[2 * t + s] = __builtin_bit_cast(
                    bf16x8, u32x4{pack_bf16x2(st[t][8 * s], st[t][8 * s + 1]), pack_bf16x2(st[t][8 * s + 2], st[t][8 * s + 3]),
                                  pack_bf16x2(st[t][8 * s + 4], st[t][8 * s + 5]), pack_bf16x2(st[t][8 * s + 6], st[t][8 * s + 7])});
        }
        // V^T fragments: lane i of a group of 16 addresses key i / 4, columns 4 (i % 4) of its 16
        const int i16 = lane & 15, vr = 4 * h + (i16 >> 2), vc = 2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1), v8 = i16 & 1;
        auto v_frag = [&](int t, int s) {
            const bf16x4 a = tr_read(sv, v_chunk<D>(16 * s + vr, 4 * t + vc), v8);
            const bf16x4 c = tr_read(sv, v_chunk<D>(16 * s + 8 + vr, 4 * t + vc), v8);
            return __builtin_shufflevector(a, c, 0, 1, 2, 3, 4, 5, 6, 7);
        };
        if (masked && bad_v) {
            // Some value is infinite or NaN, and 0 * NaN would carry it to rows that do not see it:
            // such values count as zeros, and a second product counts those that a row sees
            bf16x8 seen[2 * NT];
#pragma unroll
            for (int s = 0; s < 2 * NT; ++s)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    seen[s][e] = (bf16)(j0 + 16 * s + 8 * (e >> 2) + 4 * h + (e & 3) <= my_pos ? 1.f : 0.f);
#pragma unroll
            for (int t = 0; t < ND; ++t) {
                f32x16 count;
#pragma unroll
                for (int i = 0; i < 16; ++i) count[i] = 0.f;
#pragma unroll
                for (int s = 0; s < 2 * NT; ++s) {
                    bf16x8 vf = v_frag(t, s), nf;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const bool bad = (__builtin_bit_cast(uint16_t, (bf16)vf[e]) & 0x7f80) == 0x7f80;
                        nf[e] = (bf16)(bad ? 1.f : 0.f);
                        vf[e] = bad ? (bf16)0.f : vf[e];
                    }
                    ot[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[s], ot[t], 0, 0, 0);
                    count = __builtin_amdgcn_mfma_f32_32x32x16_bf16(nf, seen[s], count, 0, 0, 0);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (count[i] > 0.f) ot[t][i] = NAN;
            }
        } else {
#pragma unroll
            for (int t = 0; t < ND; ++t)
#pragma unroll
                for (int s = 0; s < 2 * NT; ++s) ot[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_frag(t, s), pf[s], ot[t], 0, 0, 0);
        }
    }
    if (PAGED && __syncthreads_or(bad_page)) l = NAN;  // an invalid page was read
    l += __shfl_xor(l, 32);
    if (row.kind == ROW_NONE) return;
    if (PAGED && p.splits > 1) {
        const int64_t at = (int64_t)split * p.n_tok * p.h_q + row.tok * p.h_q + row.head;
        if (row.kind == ROW_NAN) l = NAN;
        if (row.kind == ROW_ZERO) l = 0.f, m = -INFINITY;
        if (h == 0) {
            p.part_ml[2 * at] = m;
            p.part_ml[2 * at + 1] = l;
        }
        if (l == 0.f) return;  // not read
#pragma unroll
        for (int t = 0; t < ND; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<f32x4*>(p.part_o + at * D + 32 * t + 8 * i + 4 * h) =
                    f32x4{ot[t][4 * i], ot[t][4 * i + 1], ot[t][4 * i + 2], ot[t][4 * i + 3]};
        return;
    }
    float inv = l == 0.f ? 0.f : 1.f / l;
    if (row.kind == ROW_NAN) inv = NAN;
    const bool zero = row.kind == ROW_ZERO || l == 0.f;
    bf16* o = reinterpret_cast<bf16*>(p.o) + (row.tok * p.h_q + row.head) * D;
#pragma unroll
    for (int t = 0; t < ND; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x4 y = f32x4{ot[t][4 * i], ot[t][4 * i + 1], ot[t][4 * i + 2], ot[t][4 * i + 3]} * inv;
            *reinterpret_cast<bf16x4*>(o + 32 * t + 8 * i + 4 * h) = zero ? zero_bf16x4() : to_bf16(y);
        }
}

template <int D>
static hipError_t launch_d(int kind, bool paged, const AttnArgs& a, hipStream_t st) {
    const dim3 grid((unsigned)((int64_t)a.n_units * a.h_kv * (paged ? a.splits : 1))), block(64 * NW);
    if (!paged) hipLaunchKernelGGL((attn_tile_kernel<D, KV_BF16, false>), grid, block, 0, st, a);
    else if (kind == KV_E4M3) hipLaunchKernelGGL((attn_tile_kernel<D, KV_E4M3, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((attn_tile_kernel<D, KV_BF16, true>), grid, block, 0, st, a);
    return hipGetLastError();
}

hipError_t launch_attn(int d, int kind, bool paged, const AttnArgs& a, hipStream_t st) {
    switch (d) {
        case 64: return launch_d<64>(kind, paged, a, st);
        case 128: return launch_d<128>(kind, paged, a, st);
        case 256: return launch_d<256>(kind, paged, a, st);
    }
    return hipErrorInvalidValue;
}

}  // namespace lkv
