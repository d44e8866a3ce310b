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

// Eight bf16: bit i for an infinite or NaN element, the elements of set bits cleared, ones for set bits
__device__ __forceinline__ uint32_t nonfinite_bits(u32x4 x) {
    uint32_t b = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        b |= (x[i] & 0x7f80u) == 0x7f80u ? 1u << (2 * i) : 0u;
        b |= (x[i] & 0x7f800000u) == 0x7f800000u ? 2u << (2 * i) : 0u;
    }
    return b;
}
__device__ __forceinline__ u32x4 clear_bits(u32x4 x, uint32_t b) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] &= ((b >> (2 * i)) & 1 ? 0u : 0xffffu) | ((b >> (2 * i)) & 2 ? 0u : 0xffff0000u);
    return x;
}
__device__ __forceinline__ u32x4 one_bits(uint32_t b) {
    u32x4 x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = ((b >> (2 * i)) & 1 ? 0x3f80u : 0u) | ((b >> (2 * i)) & 2 ? 0x3f800000u : 0u);
    return x;
}

// Reads at byte offsets in LDS
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef __attribute__((address_space(3))) lds_i16x4 lds_tr_t;
__device__ __forceinline__ uint32_t lds_offset(const void* p) {
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)(p);
}
__device__ __forceinline__ bf16x8 frag_read(uint32_t at) {
    return __builtin_bit_cast(bf16x8, *(lds_u32x4*)(uintptr_t)at);
}
__device__ __forceinline__ bf16x4 tr_read(uint32_t at) {
    return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr_t*)(uintptr_t)at));
}

}  // namespace

// Staging of key tiles: thread's 16-byte pieces of the K and V rows, K and V alike.  Rows past the last
// key seen repeat it.  bf16 rows go from memory straight to LDS (a wave's 64 pieces land in
// consecutive chunks, so each lane fetches the piece that belongs to its chunk); e4m3 rows pass
// through registers, where they become bf16.
template <int D, int KIND, bool PAGED, int BN>
struct Stage {
    static constexpr int C = D / 8;                       // chunks of a bf16 row
    static constexpr int U = KIND == KV_E4M3 ? D / 16 : C;  // pieces of a stored row
    static constexpr int PER = BN * U / (64 * NW);
    static constexpr int EB = KIND == KV_E4M3 ? 1 : 2;
    static_assert(64 / U <= 16, "a wave's rows of one piece are in one page");
    const AttnArgs& p;
    const AttnUnit& w;
    int hk, end, tid, lane, wave;
    int k_off[PER], v_off[PER];  // bytes from the tile's (its page's) first row, full tiles
    int ids, ids_next;           // lane i: page of keys 16 i .. of the next tile, and of the one behind it
    u32x4 kr[PER], vr[PER];      // e4m3 pieces on their way
    float ks[PER], vs[PER];
    bool bad_page = false;

    __device__ __forceinline__ Stage(const AttnArgs& p_, const AttnUnit& w_, int hk_, int end_, int tid_)
        : p(p_), w(w_), hk(hk_), end(end_), tid(tid_), lane(tid_ & 63), wave(__builtin_amdgcn_readfirstlane(tid_ >> 6)) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int r = row(i);
            if (PAGED) {
                const int slot = r & ((1 << p.pg.page_shift) - 1);
                k_off[i] = (slot * U + piece(i, false)) * 16;
                v_off[i] = (slot * U + piece(i, true)) * 16;
            } else {
                k_off[i] = r * (int)p.k_stride * 2 + piece(i, false) * 16;
                v_off[i] = r * (int)p.v_stride * 2 + piece(i, true) * 16;
            }
        }
    }
    __device__ __forceinline__ int row(int i) const { return (tid + i * 64 * NW) / U; }
    // the piece of its row that this thread fetches
    __device__ __forceinline__ int piece(int i, bool v) const {
        const int x = tid + i * 64 * NW, r = x / U, c = x % U;
        if (KIND == KV_E4M3) return c;
        return (v ? v_chunk<D>(r, c) : k_chunk<D>(r, c)) - r * C;  // the permutation is its own inverse
    }
    // page ids of the tile at j0
    __device__ __forceinline__ int load_ids(int j0) const {
        if (!PAGED) return 0;
        const int j = min(j0 + 16 * (lane & (BN / 16 - 1)), end - 1);
        return p.pg.table[(int64_t)w.r * p.pg.max_pages + (j >> p.pg.page_shift)];
    }
    __device__ __forceinline__ void begin(int j0) {
        ids = load_ids(j0);
        ids_next = load_ids(j0 + BN);
    }
    __device__ __forceinline__ const char* at(const void* base, int64_t row, int64_t bytes) const {
        return reinterpret_cast<const char*>(base) + row * bytes;
    }
    // starts the fetch of the tile at j0
    __device__ __forceinline__ void fetch(int j0, u32x4* sk, u32x4* sv) {
        const bool full = j0 + BN <= end;
        const int mask = (1 << p.pg.page_shift) - 1;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const char *kb, *vb;
            int ko = k_off[i], vo = v_off[i];
            int64_t first = 0;
            if (PAGED) {
                const int r0 = (wave * 64 + i * 64 * NW) / U;  // the wave's first row: its rows are in one page
                int page = __builtin_amdgcn_readlane(ids, r0 / 16);
                const bool ok = (uint32_t)page < (uint32_t)p.pg.n_page;
                bad_page |= !ok;
                page = ok ? page : 0;
                first = ((int64_t)page * p.h_kv + hk) << p.pg.page_shift;
                if (full) {
                    first += j0 & mask;
                } else {
                    const int move = (min(j0 + row(i), end - 1) & mask) - (row(i) & mask);
                    ko += move * U * 16;
                    vo += move * U * 16;
                }
                kb = at(p.pg.k, first, U * 16);
                vb = at(p.pg.v, first, U * 16);
            } else {
                kb = at(p.k, (w.t0 + j0) * p.k_stride + (int64_t)hk * D, 2);
                vb = at(p.v, (w.t0 + j0) * p.v_stride + (int64_t)hk * D, 2);
                if (!full) {
                    const int move = min(row(i), end - 1 - j0) - row(i);
                    ko += move * (int)p.k_stride * 2;
                    vo += move * (int)p.v_stride * 2;
                }
            }
            if constexpr (KIND == KV_E4M3) {
                kr[i] = *reinterpret_cast<const u32x4*>(kb + (uint32_t)ko);
                vr[i] = *reinterpret_cast<const u32x4*>(vb + (uint32_t)vo);
                ks[i] = exp_scale(p.pg.k_exp[first + (uint32_t)ko / (16 * U)]);
                vs[i] = exp_scale(p.pg.v_exp[first + (uint32_t)vo / (16 * U)]);
            } else {
                typedef __attribute__((address_space(1))) const void global_t;
                typedef __attribute__((address_space(3))) void lds_t;
                const int x = wave * 64 + i * 64 * NW;
                __builtin_amdgcn_global_load_lds((global_t*)(kb + (uint32_t)ko), (lds_t*)(sk + x), 16, 0, 0);
                __builtin_amdgcn_global_load_lds((global_t*)(vb + (uint32_t)vo), (lds_t*)(sv + x), 16, 0, 0);
            }
        }
        ids = ids_next;
        ids_next = load_ids(j0 + 2 * BN);
    }
    // e4m3: the fetched tile into LDS
    __device__ __forceinline__ void commit(u32x4* sk, u32x4* sv) {
        if constexpr (KIND == KV_E4M3) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int x = tid + i * 64 * NW, r = x / U, c = x % U;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    sk[k_chunk<D>(r, 2 * c + e)] =
                        u32x4{e4m3_pair(kr[i][2 * e], ks[i], false), e4m3_pair(kr[i][2 * e], ks[i], true),
                              e4m3_pair(kr[i][2 * e + 1], ks[i], false), e4m3_pair(kr[i][2 * e + 1], ks[i], true)};
                    sv[v_chunk<D>(r, 2 * c + e)] =
                        u32x4{e4m3_pair(vr[i][2 * e], vs[i], false), e4m3_pair(vr[i][2 * e], vs[i], true),
                              e4m3_pair(vr[i][2 * e + 1], vs[i], false), e4m3_pair(vr[i][2 * e + 1], vs[i], true)};
                }
            }
        }
    }
};

template <int D, int KIND, bool PAGED>
__global__ __launch_bounds__(64 * NW, 2) void attn_tile_kernel(AttnArgs p) {
    constexpr int BN = D == 256 ? 32 : 64;  // keys of a tile
    constexpr int NT = BN / 32, NS = D / 16, ND = D / 32, C = D / 8;
    constexpr int CHUNKS = BN * C;
    __shared__ __align__(512) u32x4 sk[2 * CHUNKS], sv[2 * CHUNKS];  // the fragments' offsets are combined by exclusive or
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

    // keys that some row of the workgroup sees, that all of its rows see, and that some row of the wave sees
    __shared__ int s_end[NW], s_all[NW];
    const int sees = row.kind == ROW_SEES ? row.pos + 1 : 0;
    const int wave_end = wave_max_int(sees);
    const int wave_all = wave_min_int(row.kind == ROW_SEES ? sees : 0x7fffffff);
    if (lane == 0) s_end[wave] = wave_end, s_all[wave] = wave_all;
    __syncthreads();
    int end = 0, all = 0x7fffffff;
#pragma unroll
    for (int i = 0; i < NW; ++i) end = max(end, s_end[i]), all = min(all, s_all[i]);
    end = __builtin_amdgcn_readfirstlane(end);
    all = __builtin_amdgcn_readfirstlane(all);
    const KeyRange range = key_range<BN>(end, PAGED ? p.splits : 1, split);

    Stage<D, KIND, PAGED, BN> stage(p, w, hk, end, tid);
    if (range.from < range.to) {
        stage.begin(range.from);
        stage.fetch(range.from, sk, sv);
    }

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
    float m = -INFINITY, l = 0.f;  // running maximum (scaled, base 2; see below) and this half's sum
    const int my_pos = row.kind == ROW_SEES ? row.pos : 0x7fffffff;
    stage.commit(sk, sv);

    // Byte offsets of the lane's fragments; the chunks' permutation is an exclusive or, so the others are
    // one operation away.  V^T fragments: lane i of a group of 16 addresses key i / 4, columns 4 (i % 4)
    // of its 16.
    const int i16 = lane & 15, vrow = 4 * h + (i16 >> 2), vcol = 2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1);
    const uint32_t k_at = lds_offset(sk) + 16 * k_chunk<D>(col, h);
    const uint32_t v_at = lds_offset(sv) + 16 * v_chunk<D>(vrow, vcol) + 8 * (i16 & 1);
    constexpr int ROW = 2 * D;  // bytes
    auto k_frag = [&](uint32_t at, int t, int s) { return frag_read((at ^ (32 * s & 255 & (ROW - 1))) + 32 * t * ROW + (32 * s & ~255 & (ROW - 1))); };
    auto v_frag = [&](uint32_t at, int t, int s) {
        const uint32_t x = (at ^ (64 * t & 255 & (ROW - 1))) + (64 * t & ~255 & (ROW - 1)) + 16 * s * ROW;
        const bf16x4 a = tr_read(x), c = tr_read((x ^ 32) + 8 * ROW);
        return __builtin_shufflevector(a, c, 0, 1, 2, 3, 4, 5, 6, 7);
    };

    auto tile = [&](auto masked_c, int j0, int buf) {
        constexpr bool MASKED = decltype(masked_c)::value;
        const uint32_t ck = k_at + buf * CHUNKS * 16, cv = v_at + buf * CHUNKS * 16;
        f32x16 st[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int i = 0; i < 16; ++i) st[t][i] = 0.f;
#pragma unroll
            for (int s = 0; s < NS; ++s) st[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_frag(ck, t, s), qf[s], st[t], 0, 0, 0);
        }
        if (MASKED) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (j0 + 32 * t + 8 * (i >> 2) + 4 * h + (i & 3) > my_pos) st[t][i] = -INFINITY;
        }
        float top = st[0][0];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, st[t][i]);
        top = fmaxf(top, __shfl_xor(top, 32)) * p.scale_log2;
        // m need not be the maximum itself, only near it: it follows when it is exceeded by more than 8
        // (probabilities up to 2^8), which after the first tiles is rare, and else O stays as it is
        if (__any(!(top <= m + 8.f))) {
            const float m_new = fmaxf(m, top);
            const float scale = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
            m = m_new;
            l *= scale;
#pragma unroll
            for (int t = 0; t < ND; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) ot[t][i] *= scale;
        }
        const float m_use = m == -INFINITY ? 0.f : m;  // only scores of -inf so far
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            bf16x8 pf[2];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(st[t][i], p.scale_log2, -m_use));
                l += e;
                st[t][i] = e;
            }
#pragma unroll
            for (int s = 0; s < 2; ++s)
                pf[s] = __builtin_bit_cast(
                    bf16x8, u32x4{pack_bf16x2(st[t][8 * s], st[t][8 * s + 1]), pack_bf16x2(st[t][8 * s + 2], st[t][8 * s + 3]),
                                  pack_bf16x2(st[t][8 * s + 4], st[t][8 * s + 5]), pack_bf16x2(st[t][8 * s + 6], st[t][8 * s + 7])});
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int d = 0; d < ND; ++d)
                    ot[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_frag(cv, d, 2 * t + s), pf[s], ot[d], 0, 0, 0);
        }
    };

    // Two buffers: one tile is fetched while the one before it is worked on, with one barrier per tile.
    // Tiles that every row of the workgroup sees whole come first, without masks.
    int j0 = range.from, buf = 0;
    auto arrive = [&]() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
    for (; j0 < range.to && j0 + BN <= all; j0 += BN, buf ^= 1) {
        arrive();
        const bool more = j0 + BN < range.to;
        if (more) stage.fetch(j0 + BN, sk + (buf ^ 1) * CHUNKS, sv + (buf ^ 1) * CHUNKS);
        tile(std::false_type(), j0, buf);
        if (more) stage.commit(sk + (buf ^ 1) * CHUNKS, sv + (buf ^ 1) * CHUNKS);
    }
    // A masked tile whose values are not all finite: 0 * NaN would carry them to rows that do not see
    // them, so they count as zeros, and a second product counts those that a row sees.
    __shared__ int s_bad[2];
    for (; j0 < range.to; j0 += BN, buf ^= 1) {
        if (tid == 0) s_bad[buf] = 0;
        arrive();
        const bool more = j0 + BN < range.to;
        if (more) stage.fetch(j0 + BN, sk + (buf ^ 1) * CHUNKS, sv + (buf ^ 1) * CHUNKS);
        uint32_t bad = 0;  // 8 bits for each of the thread's chunks
        static_assert(CHUNKS == 4 * 64 * NW || CHUNKS == 2 * 64 * NW, "chunks of a thread");
#pragma unroll
        for (int i = 0; i < CHUNKS / (64 * NW); ++i) {
            u32x4& c = sv[buf * CHUNKS + tid + i * 64 * NW];
            const uint32_t b = nonfinite_bits(c);
            if (b) c = clear_bits(c, b);
            bad |= b << (8 * i);
        }
        if (bad) s_bad[buf] = 1;
        lds_barrier();
        if (j0 < wave_end) tile(std::true_type(), j0, buf);
        if (s_bad[buf]) {
            lds_barrier();
#pragma unroll
            for (int i = 0; i < CHUNKS / (64 * NW); ++i) sv[buf * CHUNKS + tid + i * 64 * NW] = one_bits(bad >> (8 * i));
            lds_barrier();
#pragma unroll
            for (int d = 0; d < ND; ++d) {
                f32x16 count;
#pragma unroll
                for (int i = 0; i < 16; ++i) count[i] = 0.f;
#pragma unroll 1
                for (int s = 0; s < 2 * NT; ++s) {
                    bf16x8 seen;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        seen[e] = (bf16)(j0 + 16 * s + 8 * (e >> 2) + 4 * h + (e & 3) <= my_pos ? 1.f : 0.f);
                    count = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_frag(v_at + buf * CHUNKS * 16, d, s), seen, count, 0, 0, 0);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (count[i] > 0.f) ot[d][i] = NAN;
            }
        }
        if (more) stage.commit(sk + (buf ^ 1) * CHUNKS, sv + (buf ^ 1) * CHUNKS);
    }
    const bool bad_page = stage.bad_page;
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
