// Attention of few rows per request over a paged cache (decoding, drafted tokens): bound by
// reading the cache once, from HBM.
//
// A workgroup works on 16 or 32 rows (see attn_device.h) and a part of the keys.  Its four waves
// take slices of keys in turn and keep a softmax and an output of their own, joined at the end
// through LDS, so there is no barrier on the way: a wave sends for its next slice as soon as the
// last one has come, then works on that.  The products are those of attn_tile.hip on the 16x16x32
// MFMA: S^T = K Q^T with K's fragments loaded straight into registers, O^T = V^T P^T with V's
// fragments read transposed from LDS, where bf16 rows land directly and e4m3 rows as bf16.
// 8 KB of keys and as much of values are in flight per wave with bf16, half with e4m3: 5.4 to 5.7 TB/s
// on 32 contexts of 8K (8 key/value heads of 128: 188 us in bf16, 100 in e4m3).  The registers hold one
// slice, refilled as the products free it, and so two workgroups fit on a CU (one with 32 rows of 256).
#include "attn_device.h"

namespace lkv {

namespace {

#define INLINE __attribute__((always_inline))

constexpr int NW = 4;  // waves

// Position of 16-byte chunk c of row r (in chunks): a transposing read takes two adjacent chunks of 16 rows
template <int D>
__device__ __forceinline__ int v_chunk(int r, int c) {
    constexpr int C = D / 8;
    const int f = C >= 16 ? ((r & 7) << 1) : ((r >> 1) & 3) << 1;
    return r * C + (c ^ f);
}

}  // namespace

template <int D, bool E4M3, int RT>
__global__ __launch_bounds__(64 * NW, D * RT == 512 ? 1 : 2) void attn_few_kernel(AttnArgs p) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, g = lane >> 4;
    constexpr int SL = 4096 / D;           // keys of a slice
    constexpr int KT = SL / 16;            // key tiles
    constexpr int PT = (KT + 1) / 2;       // their pairs, the contraction of one product with the values
    constexpr int NS = D / 32, ND = D / 16, C = D / 8, BM = 16 * RT;
    constexpr int VB = SL * C;             // chunks of a slice's values in LDS
    constexpr int U = E4M3 ? D / 16 : C;   // 16-byte pieces of a stored row
    constexpr int KL = NS * KT / (E4M3 ? 2 : 1), VL = SL * U / 64;  // loads per lane and slice
    constexpr int WB = (E4M3 ? 1 : 2) * VB;                         // a wave's chunks
    constexpr int LD = D + 4;                                       // row of the final join, in floats
    constexpr int JB = NW * 16 * LD / 4;
    __shared__ __align__(1024) u32x4 smem[NW * WB > JB ? NW * WB : JB];
    u32x4* const sv = smem + wave * WB;

    int b = blockIdx.x;
    const int hk = b % p.h_kv;
    b /= p.h_kv;
    const int split = b % p.splits, u = b / p.splits;
    const AttnUnit w = attn_unit<BM>(p, u, lane);
    if (w.r < 0) return;
    const int len = attn_len(p.pg, w.r);
    AttnRow row[RT];
    int my_pos[RT], end = 0, all = 0x7fffffff;
#pragma unroll
    for (int n = 0; n < RT; ++n) {
        row[n] = attn_row<true>(p, w, w.row0 + 16 * n + col, hk, len);
        const bool sees = row[n].kind == ROW_SEES;
        my_pos[n] = sees ? row[n].pos : 0x7fffffff;
        end = max(end, sees ? row[n].pos + 1 : 0);
        all = min(all, sees ? row[n].pos + 1 : 0x7fffffff);
    }
    end = wave_max_int(end);  // every wave has the same rows
    all = wave_min_int(all);
    const KeyRange range = key_range<SL * NW>(end, p.splits, split);
    const int slices = (range.to - range.from + SL - 1) / SL;
    auto start = [&](int j) INLINE { return range.from + j * SL; };

    // Key k of a 32-wide product: lane group g holds 8 elements.  bf16: 32 s + 8 g ..; e4m3, where a
    // 16-byte load covers two products: 64 (s / 2) + 16 g + 8 (s % 2) ..; q alike.
    bf16x8 qf[RT][NS];
#pragma unroll
    for (int n = 0; n < RT; ++n) {
        const bf16* q = reinterpret_cast<const bf16*>(p.q) + row[n].tok * p.q_stride + (int64_t)row[n].head * D;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const int e = E4M3 ? 64 * (s / 2) + 16 * g + 8 * (s % 2) : 32 * s + 8 * g;
            qf[n][s] = row[n].kind == ROW_NONE ? bf16x8{} : *reinterpret_cast<const bf16x8*>(q + e);
        }
    }
    f32x4 ot[RT][ND];
    float m[RT], l[RT];
#pragma unroll
    for (int n = 0; n < RT; ++n) {
        m[n] = -INFINITY, l[n] = 0.f;
#pragma unroll
        for (int t = 0; t < ND; ++t) ot[n][t] = zero4();
    }

    // Loads of slice j, whose page ids `ids` holds.  Keys past the last one seen repeat it.
    u32x4 kr[KL], vr[E4M3 ? VL : 1];
    uint8_t ke[E4M3 ? KT : 1], ve[E4M3 ? VL : 1];
    const int mask = (1 << p.pg.page_shift) - 1;
    constexpr int EB = E4M3 ? 1 : 2;
    bool bad_page = false;
    auto load_ids = [&](int j) INLINE {
        const int key = min(start(j) + 16 * (lane & (KT - 1)), end - 1);
        return p.pg.table[(int64_t)w.r * p.pg.max_pages + (key >> p.pg.page_shift)];
    };
    auto page_row = [&](int ids, int t) INLINE {  // pool row of the first token of the page of key tile t
        int page = __builtin_amdgcn_readlane(ids, t);
        const bool ok = (uint32_t)page < (uint32_t)p.pg.n_page;
        bad_page |= !ok;
        return ((int64_t)(ok ? page : 0) * p.h_kv + hk) << p.pg.page_shift;
    };
    auto fetch_values = [&](int j, int ids, int buf) INLINE {
        // piece x of the slice is piece x % U of row x / U; the 64 of a load are in one key tile
#pragma unroll
        for (int i = 0; i < VL; ++i) {
            const int r = (lane + 64 * i) / U, c = (lane + 64 * i) % U;
            const int64_t first = page_row(ids, 64 * i / U / 16);
            const int slot = min(start(j) + r, end - 1) & mask;
            const char* src = reinterpret_cast<const char*>(p.pg.v) + first * (D * EB);
            if constexpr (E4M3) {
                vr[i] = *reinterpret_cast<const u32x4*>(src + (uint32_t)(slot * U + c) * 16);
                ve[i] = p.pg.v_exp[first + slot];
            } else {
                typedef __attribute__((address_space(1))) const void global_t;
                typedef __attribute__((address_space(3))) void lds_t;
                const int piece = v_chunk<D>(r, c) - r * C;
                __builtin_amdgcn_global_load_lds((global_t*)(src + (uint32_t)(slot * U + piece) * 16),
                                                 (lds_t*)(sv + buf * VB + 64 * i), 16, 0, 0);
            }
        }
    };
    auto fetch_keys = [&](int j, int ids) INLINE {
#pragma unroll
        for (int t = 0; t < KT; ++t) {
            const int64_t first = page_row(ids, t);
            const int slot = min(start(j) + 16 * t + col, end - 1) & mask;
            const char* src = reinterpret_cast<const char*>(p.pg.k) + first * (D * EB);
            if constexpr (E4M3) ke[t] = p.pg.k_exp[first + slot];
#pragma unroll
            for (int s = 0; s < KL / KT; ++s)
                kr[t * (KL / KT) + s] = *reinterpret_cast<const u32x4*>(src + (uint32_t)(slot * U + 4 * s + g) * 16);
        }
    };

    const uint32_t v_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)(const char*)sv;
    // V^T fragment: lane i of group g addresses key 4 g + i / 4, columns 4 (i % 4) of its 16
    const int vrow = 4 * g + (col >> 2), vcol = (col & 3) >> 1;
    typedef __attribute__((address_space(3))) lds_i16x4 lds_tr_t;
    auto tr_read = [&](int t, int d, int buf) INLINE {  // keys of tile t, columns 16 d ..
        const uint32_t at = v_at + (E4M3 ? 0 : buf * VB * 16) + 16 * v_chunk<D>(16 * t + vrow, 2 * d + vcol) + 8 * (col & 1);
        return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr_t*)(uintptr_t)at));
    };

    // A masked slice whose values are not all finite: 0 * NaN would carry them to rows that do not see
    // them.  They are counted among those that a row sees, whose output becomes NaN, and cleared.
    auto check_values = [&](int j, int buf) INLINE {
        wave_lds_sync();
        u32x4* const x = sv + (E4M3 ? 0 : buf * VB);
        bool bad = false;
#pragma unroll
        for (int i = 0; i < VB / 64; ++i) bad |= nonfinite_bits(x[64 * i + lane]) != 0;
        if (!__any(bad)) return;
        u32x4 old[VB / 64];
#pragma unroll
        for (int i = 0; i < VB / 64; ++i) {
            old[i] = x[64 * i + lane];
            x[64 * i + lane] = one_bits(nonfinite_bits(old[i]));
        }
        wave_lds_sync();
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int t = 0; t < PT; ++t) {
                __builtin_amdgcn_sched_barrier(0);
                const bf16x4 v0 = tr_read(2 * t, d, buf), v1 = 2 * t + 1 < KT ? tr_read(2 * t + 1, d, buf) : zero_bf16x4();
#pragma unroll
                for (int n = 0; n < RT; ++n) {
                    bf16x4 s0, s1;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s0[e] = (bf16)(start(j) + 32 * t + 4 * g + e <= my_pos[n] ? 1.f : 0.f);
                        s1[e] = (bf16)(start(j) + 32 * t + 16 + 4 * g + e <= my_pos[n] ? 1.f : 0.f);
                    }
                    const f32x4 count = mma32(v0, v1, s0, s1, zero4());
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (count[i] > 0.f) ot[n][d][i] = NAN;
                }
            }
        wave_lds_sync();
#pragma unroll
        for (int i = 0; i < VB / 64; ++i) x[64 * i + lane] = clear_bits(old[i], nonfinite_bits(old[i]));
        wave_lds_sync();
    };
    // Slice j, which has come; slice j + NW, if there is one, is sent for as its registers become free.
    auto work = [&](int j, int buf, int next) INLINE {
        const bool more = j + NW < slices;
        if constexpr (E4M3) {
#pragma unroll
            for (int i = 0; i < VL; ++i) {
                const int r = (lane + 64 * i) / U, c = (lane + 64 * i) % U;
                const float s = exp_scale(ve[i]);
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    sv[v_chunk<D>(r, 2 * c + e)] =
                        u32x4{e4m3_pair(vr[i][2 * e], s, false), e4m3_pair(vr[i][2 * e], s, true),
                              e4m3_pair(vr[i][2 * e + 1], s, false), e4m3_pair(vr[i][2 * e + 1], s, true)};
            }
        }
        if (more) fetch_values(j + NW, next, buf ^ 1);
        const bool masked = start(j) + SL > all;
        if (masked) check_values(j, buf);
        f32x4 st[RT][KT];
#pragma unroll
        for (int t = 0; t < KT; ++t) {
#pragma unroll
            for (int n = 0; n < RT; ++n) st[n][t] = zero4();
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                bf16x8 kf;
                if constexpr (E4M3) {
                    const u32x4 y = kr[t * (KL / KT) + s / 2];
                    const float e = exp_scale(ke[t]);
                    const uint32_t a = y[2 * (s % 2)], c = y[2 * (s % 2) + 1];
                    kf = __builtin_bit_cast(bf16x8, u32x4{e4m3_pair(a, e, false), e4m3_pair(a, e, true), e4m3_pair(c, e, false),
                                                          e4m3_pair(c, e, true)});
                } else {
                    kf = __builtin_bit_cast(bf16x8, kr[t * NS + s]);
                }
#pragma unroll
                for (int n = 0; n < RT; ++n) st[n][t] = mma32(kf, qf[n][s], st[n][t]);
            }
        }
        if (more) fetch_keys(j + NW, next);
        bf16x4 pf[RT][2 * PT];
#pragma unroll
        for (int n = 0; n < RT; ++n) {
            float top = -INFINITY;
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (masked && start(j) + 16 * t + 4 * g + i > my_pos[n]) st[n][t][i] = -INFINITY;
                    // rows that are not stored see repeated keys, which no maximum needs
                    top = fmaxf(top, st[n][t][i]);
                }
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32)) * p.scale_log2;
            if (__any(!(top <= m[n] + 8.f))) {  // as in attn_tile.hip
                const float m_new = top > m[n] + 8.f ? top : m[n];
                const float scale = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[n] - m_new);
                m[n] = m_new;
                l[n] *= scale;
#pragma unroll
                for (int d = 0; d < ND; ++d) ot[n][d] *= scale;
            }
            const float m_use = m[n] == -INFINITY ? 0.f : m[n];
#pragma unroll
            for (int t = 0; t < KT; ++t) {
#pragma unroll
                for (int i = 0; i < 4; ++i) st[n][t][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[n][t][i], p.scale_log2, -m_use));
                pf[n][t] = to_bf16(st[n][t]);
                const f32x4 r = to_f32(pf[n][t]);
                l[n] += (r[0] + r[1]) + (r[2] + r[3]);
            }
            if (KT % 2) pf[n][KT] = zero_bf16x4();
        }
        if constexpr (E4M3) wave_lds_sync();
#pragma unroll
        for (int d = 0; d < ND; ++d) {
            if (d % 4 == 0) __builtin_amdgcn_sched_barrier(0);  // fragments of four products at a time: registers
#pragma unroll
            for (int t = 0; t < PT; ++t) {
                const bf16x4 v0 = tr_read(2 * t, d, buf), v1 = 2 * t + 1 < KT ? tr_read(2 * t + 1, d, buf) : zero_bf16x4();
                const bf16x8 vf = __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
                for (int n = 0; n < RT; ++n)
                    ot[n][d] = mma32(vf, pf[n][2 * t], pf[n][2 * t + 1], ot[n][d]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (E4M3) wave_lds_sync();
    };

    // Slices wave, wave + NW, ..
    auto arrive = [&]() INLINE { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); };
    if (wave < slices) {
        int next = load_ids(wave);
        fetch_values(wave, next, 0);
        fetch_keys(wave, next);
        next = load_ids(wave + NW);
        int buf = 0;
        for (int j = wave; j < slices; j += NW) {
            arrive();
            const int ids = next;
            next = load_ids(j + 2 * NW);
            work(j, buf, ids);
            buf ^= 1;
        }
    }
    if (bad_page) {
#pragma unroll
        for (int n = 0; n < RT; ++n) l[n] = NAN;
    }

    // Join of the waves, one row tile at a time, in the order of the waves; thread (row, part of D)
    __shared__ float s_m[NW][16], s_l[NW][16];
    float* so = reinterpret_cast<float*>(smem);  // [NW][16][LD]
    const int jr = tid >> 4, jc = tid & 15;  // row of the join, its lane
#pragma unroll
    for (int n = 0; n < RT; ++n) {
        __syncthreads();
        float sum = l[n] + __shfl_xor(l[n], 16);
        sum += __shfl_xor(sum, 32);
        if (g == 0) s_m[wave][col] = m[n], s_l[wave][col] = sum;
#pragma unroll
        for (int d = 0; d < ND; ++d) *reinterpret_cast<f32x4*>(so + (wave * 16 + col) * LD + 16 * d + 4 * g) = ot[n][d];
        __syncthreads();
        const AttnRow x = attn_row<true>(p, w, w.row0 + 16 * n + jr, hk, len);
        if (x.kind == ROW_NONE) continue;
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < NW; ++i) top = fmaxf(top, s_m[i][jr]);
        const float m_use = top == -INFINITY ? 0.f : top;
        float total = 0.f, f[NW];
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            f[i] = __builtin_amdgcn_exp2f(s_m[i][jr] - m_use);
            total += f[i] * s_l[i][jr];
        }
        if (x.kind == ROW_NAN) total = NAN;
        if (x.kind == ROW_ZERO) total = 0.f, top = -INFINITY;
        const int64_t at = x.tok * p.h_q + x.head, pat = (int64_t)split * p.n_tok * p.h_q + at;
        if (p.splits > 1) {
            const float stored = part_sum(total, x, range);
            if (jc == 0) {
                p.part_ml[2 * pat] = top;
                p.part_ml[2 * pat + 1] = stored;
            }
            if (stored == 0.f) continue;
        }
        const float inv = total == 0.f ? 1.f : 1.f / total;  // as in attn_tile.hip
#pragma unroll
        for (int e = 0; e < D / 64; ++e) {
            f32x4 y = zero4();
#pragma unroll
            for (int i = 0; i < NW; ++i) y += f[i] * *reinterpret_cast<const f32x4*>(so + (i * 16 + jr) * LD + 64 * e + 4 * jc);
            if (p.splits > 1) *reinterpret_cast<f32x4*>(p.part_o + pat * D + 64 * e + 4 * jc) = y;
            else
                *reinterpret_cast<bf16x4*>(reinterpret_cast<bf16*>(p.o) + at * D + 64 * e + 4 * jc) =
                    x.kind == ROW_ZERO ? zero_bf16x4() : to_bf16(y * inv);
        }
    }
}


template <int D, int RT>
static hipError_t launch_few_d(bool e4m3, const AttnArgs& a, hipStream_t st) {
    const dim3 grid((unsigned)((int64_t)a.n_units * a.h_kv * a.splits)), block(64 * NW);
    if (e4m3) hipLaunchKernelGGL((attn_few_kernel<D, true, RT>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((attn_few_kernel<D, false, RT>), grid, block, 0, st, a);
    return hipGetLastError();
}

hipError_t launch_attn_few(int d, int kind, int rows, const AttnArgs& a, hipStream_t st) {
    const bool e4m3 = kind == KV_E4M3;
    switch (d) {
        case 64: return rows == 16 ? launch_few_d<64, 1>(e4m3, a, st) : launch_few_d<64, 2>(e4m3, a, st);
        case 128: return rows == 16 ? launch_few_d<128, 1>(e4m3, a, st) : launch_few_d<128, 2>(e4m3, a, st);
        case 256: return rows == 16 ? launch_few_d<256, 1>(e4m3, a, st) : launch_few_d<256, 2>(e4m3, a, st);
    }
    return hipErrorInvalidValue;
}

}  // namespace lkv
