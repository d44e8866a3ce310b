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
// for the product (2^-8 of each at most, as the outputs are).
//
// Power bounds the large calls (two workgroups per CU: the clock falls to 2.0 GHz with the matrix
// cores half busy): a 32K prompt of 32/8 heads of 128 takes 8.3 ms on new inputs, 1.06 PFLOP/s (8.2 on
// inputs at rest in the caches; up to 9.0 on other cards and under the profiler), an 8K prompt of
// 16/2 heads of 256 0.57 ms, 0.97 PFLOP/s (0.52; 0.60).  Measured beside it and not better: the
// next tile's scores formed in between softmax and product (8.3 ms), eight waves that share a tile
// (8.4), three waves per SIMD on tiles of 32 keys (8.2; 32 ragged blocks 490 against 460 us), keys
// staged through registers (8.0 with eight waves, but paged keys 6.2 against 4.7 ms), 64 rows per
// wave with one wave per SIMD (9.4 and more: each fragment read serves two products, but nothing
// hides the LDS and barrier waits).
#include <algorithm>

#include "attn_device.h"

namespace lkv {

namespace {

#define INLINE __attribute__((always_inline))  // lambdas over register arrays

constexpr int NW = 4;  // waves

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

// Maximum and sum over the wave's two halves
__device__ __forceinline__ float half_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}
__device__ __forceinline__ float half_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
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

// Staging of one side's tiles (keys, or values): the thread's 16-byte pieces of the rows.  Rows past the
// last key seen repeat it.  bf16 rows go from memory straight to LDS (a wave's 64 pieces land in
// consecutive chunks, so each lane fetches the piece that belongs to its chunk); e4m3 rows pass
// through registers, where they become bf16.
template <int D, int KIND, bool PAGED, int BN, int STEP, bool V>
struct Stage {
    static constexpr int C = D / 8;                         // chunks of a bf16 row
    static constexpr int U = KIND == KV_E4M3 ? D / 16 : C;  // pieces of a stored row
    static constexpr int PER = BN * U / (64 * NW);
    static_assert(64 / U <= 16, "a wave's rows of one piece are in one page");
    const AttnArgs& p;
    const AttnUnit& w;
    const char* base;  // the pool; packed sequences: the next tile's first row
    int64_t stride;    // elements between rows, packed sequences
    int hk, end, tid, lane, wave;
    int off[PER];  // bytes from the tile's (its page's) first row, full tiles
    u32x4 r[PER];  // e4m3 pieces on their way, and their rows' scales: not touched before commit
    uint8_t exps[PER];
    uint32_t put;  // e4m3: byte offset of the thread's first chunk in a buffer
    bool bad_page = false;

    __device__ __forceinline__ Stage(const AttnArgs& p_, const AttnUnit& w_, int hk_, int end_, int tid_)
        : p(p_), w(w_), base(reinterpret_cast<const char*>(PAGED ? (V ? p_.pg.v : p_.pg.k) : (V ? p_.v : p_.k))),
          stride(V ? p_.v_stride : p_.k_stride), hk(hk_), end(end_), tid(tid_), lane(tid_ & 63), wave(__builtin_amdgcn_readfirstlane(tid_ >> 6)) {
        put = 16 * (V ? v_chunk<D>(tid / U, 2 * (tid % U)) : k_chunk<D>(tid / U, 2 * (tid % U)));
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int x = tid + i * 64 * NW, row = x / U, c = x % U;
            // the permutation of a row's chunks is its own inverse
            const int piece = KIND == KV_E4M3 ? c : (V ? v_chunk<D>(row, c) : k_chunk<D>(row, c)) - row * C;
            off[i] = PAGED ? ((row & ((1 << p.pg.page_shift) - 1)) * U + piece) * 16 : row * (int)stride * 2 + piece * 16;
        }
    }
    __device__ __forceinline__ int row(int i) const { return (tid + i * 64 * NW) / U; }
    __device__ __forceinline__ void begin(int j0) {
        if (!PAGED) base += ((w.t0 + j0) * stride + (int64_t)hk * D) * 2;
    }
    // starts the fetch of the tile at j0; tiles are fetched in order.  ids: lane i has the page of keys 16 i ..
    __device__ __forceinline__ void fetch(int j0, u32x4* lds, int ids) {
        const bool full = j0 + BN <= end;
        const int mask = (1 << p.pg.page_shift) - 1;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            int o = off[i];
            int64_t first = 0;
            const char* b = base;
            if (PAGED) {
                const int r0 = (wave * 64 + i * 64 * NW) / U;  // the wave's first row: its rows are in one page
                int page = __builtin_amdgcn_readlane(ids, r0 / 16);
                const bool ok = (uint32_t)page < (uint32_t)p.pg.n_page;
                bad_page |= !ok;
                page = ok ? page : 0;
                first = ((int64_t)page * p.h_kv + hk) << p.pg.page_shift;
                if (full) first += j0 & mask;
                else o += ((min(j0 + row(i), end - 1) & mask) - (row(i) & mask)) * U * 16;
                b += first * (U * 16);
            } else {
                if (!full) o += (min(row(i), end - 1 - j0) - row(i)) * (int)stride * 2;
            }
            if constexpr (KIND == KV_E4M3) {
                r[i] = *reinterpret_cast<const u32x4*>(b + (uint32_t)o);
                exps[i] = (V ? p.pg.v_exp : p.pg.k_exp)[first + (uint32_t)o / (16 * U)];
            } else {
                typedef __attribute__((address_space(1))) const void global_t;
                typedef __attribute__((address_space(3))) void lds_t;
                __builtin_amdgcn_global_load_lds((global_t*)(b + (uint32_t)o), (lds_t*)(lds + wave * 64 + i * 64 * NW), 16, 0, 0);
            }
        }
        if (!PAGED) base += STEP * stride * 2;
    }
    // e4m3: the fetched tile into the buffer at byte offset `lds`.  The thread's pieces are a multiple of 16
    // rows apart, where the chunks' permutation repeats.
    __device__ __forceinline__ void commit(uint32_t lds) {
        if constexpr (KIND == KV_E4M3) {
            static_assert(PER == 1 || 64 * NW / U % 16 == 0, "rows of a thread's pieces");
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const float scale = exp_scale(exps[i]);
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    *(lds_u32x4*)(uintptr_t)(((lds + put) ^ (16 * e)) + i * (64 * NW / U) * 2 * D) =
                        u32x4{e4m3_pair(r[i][2 * e], scale, false), e4m3_pair(r[i][2 * e], scale, true),
                              e4m3_pair(r[i][2 * e + 1], scale, false), e4m3_pair(r[i][2 * e + 1], scale, true)};
            }
        }
    }
};

// KG = 2: two groups of NW waves work on the same rows, each on every other tile of keys with buffers, a
// softmax and an output of its own, joined at the end: where a call has few workgroups, the longest
// one's chain of tiles is its time.
template <int D, int KIND, bool PAGED, int KG>
__global__ __launch_bounds__(64 * NW * KG, 2) void attn_tile_kernel(AttnArgs p) {
    constexpr int BN = D == 256 ? 32 : 64;  // keys of a tile
    constexpr int NT = BN / 32, NS = D / 16, ND = D / 32, C = D / 8;
    constexpr int CHUNKS = BN * C, BM = ATTN_ROWS, STEP = KG * BN;  // STEP: keys of a round
    static_assert(BM == 32 * NW, "a wave owns 32 rows");
    __shared__ __align__(512) u32x4 smem[KG * 4 * CHUNKS];  // the fragments' offsets are combined by exclusive or
    const int kg = KG == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / (64 * NW));
    const int tid = threadIdx.x % (64 * NW), lane = tid & 63, wave = tid >> 6;  // in the group
    u32x4 *const sk = smem + kg * 4 * CHUNKS, *const sv = sk + 2 * CHUNKS;
    const int col = lane & 31, h = lane >> 5;

    int b = blockIdx.x;
    const int hk = b % p.h_kv;
    b /= p.h_kv;
    const int split = PAGED ? b % p.splits : 0;
    const int u = PAGED ? b / p.splits : b;
    const AttnUnit w = attn_unit<BM>(p, u, lane);
    if (w.r < 0) return;
    const int len = PAGED ? attn_len(p.pg, w.r) : w.n;
    // The lane's row; at d = 256, short of registers, formed again after the unmasked tiles, not held over them
    auto my_row = [&]() INLINE {
        int c = col;
        if (D == 256) asm volatile("" : "+v"(c));
        return attn_row<PAGED>(p, w, w.row0 + 32 * wave + c, hk, len);
    };
    const AttnRow first_row = my_row();
    const bool sees = first_row.kind == ROW_SEES;
    // keys that some row of the workgroup sees, and that all of its rows see
    __shared__ int s_end[NW], s_all[NW];
    int end = wave_max_int(sees ? first_row.pos + 1 : 0), all = wave_min_int(sees ? first_row.pos + 1 : 0x7fffffff);
    if (lane == 0) s_end[wave] = end, s_all[wave] = all;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NW; ++i) end = max(end, s_end[i]), all = min(all, s_all[i]);
    end = __builtin_amdgcn_readfirstlane(end);
    all = __builtin_amdgcn_readfirstlane(all);
    const KeyRange range = key_range<BN>(end, PAGED ? p.splits : 1, split);

    Stage<D, KIND, PAGED, BN, STEP, false> keys(p, w, hk, end, tid);
    Stage<D, KIND, PAGED, BN, STEP, true> vals(p, w, hk, end, tid);
    const int tiles = (range.to - range.from + STEP - 1) / STEP;  // of each group
    const int clear = min(max(all - range.from, 0) / STEP, tiles);  // that every row of the workgroup sees whole
    auto start = [&](int j) INLINE { return range.from + j * STEP + kg * BN; };
    // The second group's last tile may lie past the keys: its values are zeros, its scores masked
    auto exists = [&](int j) INLINE { return j < tiles && (KG == 1 || start(j) < end); };
    int b0 = 0, b1 = CHUNKS * 16;  // buffers of the tile at hand and of the next one
    auto k_buf = [&](int o) INLINE { return reinterpret_cast<u32x4*>(reinterpret_cast<char*>(sk) + o); };
    auto v_buf = [&](int o) INLINE { return reinterpret_cast<u32x4*>(reinterpret_cast<char*>(sv) + o); };
    auto load_ids = [&](int j0) INLINE {
        if (!PAGED) return 0;
        const int j = min(j0 + 16 * (lane & (BN / 16 - 1)), end - 1);
        return p.pg.table[(int64_t)w.r * p.pg.max_pages + (j >> p.pg.page_shift)];
    };
    int ids = 0;  // pages of the next tile to fetch
    if (exists(0)) {
        ids = load_ids(start(0));
        keys.begin(start(0));
        vals.begin(start(0));
        keys.fetch(start(0), sk, ids);
        vals.fetch(start(0), sv, ids);
        ids = load_ids(start(1));
    }

    // At d = 256 registers are short by a few fragments of Q: those are read from LDS each time.  (Spilled ones
    // would be worse than their number: a load from scratch waits for the next tile's loads before it.)
    constexpr int QL = D == 256 ? 3 : 0;
    __shared__ u32x4 sq[QL > 0 ? NW * QL * 64 : 1];
    const uint32_t q_at = lds_offset(sq) + 16 * (wave * QL * 64 + lane);
    bf16x8 qf[NS];
    const bf16* q = reinterpret_cast<const bf16*>(p.q) + first_row.tok * p.q_stride + (int64_t)first_row.head * D;
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[s] = first_row.kind == ROW_NONE ? bf16x8{} : *reinterpret_cast<const bf16x8*>(q + 16 * s + 8 * h);
#pragma unroll
    for (int s = 0; s < QL; ++s) sq[wave * QL * 64 + s * 64 + lane] = __builtin_bit_cast(u32x4, qf[s]);
    f32x16 ot[ND];
#pragma unroll
    for (int t = 0; t < ND; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) ot[t][i] = 0.f;
    float m = -INFINITY, l = 0.f;  // reference of the exponents (base 2, see below) and this half's sum
    if (exists(0)) {
        keys.commit(lds_offset(sk));
        vals.commit(lds_offset(sv));
    }

    // Byte offsets of the lane's fragments; the chunks' permutation is an exclusive or, so the others are
    // one operation away.  V^T fragments: lane i of a group of 16 addresses key i / 4, columns 4 (i % 4)
    // of its 16.
    const int i16 = lane & 15, vrow = 4 * h + (i16 >> 2), vcol = 2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1);
    const uint32_t k_at = lds_offset(sk) + 16 * k_chunk<D>(col, h);
    const uint32_t v_at = lds_offset(sv) + 16 * v_chunk<D>(vrow, vcol) + 8 * (i16 & 1);
    constexpr int ROW = 2 * D;  // bytes
    auto k_frag = [&](uint32_t at, int t, int s) INLINE { return frag_read((at ^ (32 * s & 255 & (ROW - 1))) + 32 * t * ROW + (32 * s & ~255 & (ROW - 1))); };
    auto v_frag = [&](uint32_t at, int t, int s) INLINE {
        const uint32_t x = at ^ (64 * t & 255 & (ROW - 1)), y = (64 * t & ~255 & (ROW - 1)) + 16 * s * ROW;
        const bf16x4 a = tr_read(x + y), c = tr_read((x ^ 32) + y + 8 * ROW);
        return __builtin_shufflevector(a, c, 0, 1, 2, 3, 4, 5, 6, 7);
    };

    int my_pos = 0;  // set for the masked tiles
    // Tile j, whose keys and values are in the buffers at b0; the next one's are sent for.
    auto tile = [&](bool masked, int j) INLINE {
        const bool more = exists(j + 1);
        if (more) {
            keys.fetch(start(j + 1), k_buf(b1), ids);
            if (KIND != KV_E4M3) {
                vals.fetch(start(j + 1), v_buf(b1), ids);
                ids = load_ids(start(j + 2));
            }
        }
        f32x16 st[NT];
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int i = 0; i < 16; ++i) st[t][i] = 0.f;
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                // Q's fragments in LDS are the wave's own
                const bf16x8 y = s < QL ? frag_read(q_at + 1024 * s) : qf[s];
                st[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_frag(k_at + b0, t, s), y, st[t], 0, 0, 0);
            }
        }
        __builtin_amdgcn_s_setprio(0);
        if (masked) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (start(j) + 32 * t + 8 * (e >> 2) + 4 * h + (e & 3) > my_pos) st[t][e] = -INFINITY;
        }
        // The reference m need not be the maximum, only near it: it follows when it is exceeded by more
        // than 8 (probabilities up to 2^8), which after the first tiles is rare, and else O stays as it is.
        float top = st[0][0];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, st[t][e]);
        top = half_max(top) * p.scale_log2;
        if (__any(!(top <= m + 8.f))) {
            const float m_new = top > m + 8.f ? top : m;  // by the row's own scores alone
            const float scale = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
            m = m_new;
            l *= scale;
#pragma unroll
            for (int t = 0; t < ND; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) ot[t][e] *= scale;
        }
        if (more) {
            keys.commit(lds_offset(sk) + b1);
            if (KIND == KV_E4M3) {  // through the registers that the keys left
                vals.fetch(start(j + 1), v_buf(b1), ids);
                ids = load_ids(start(j + 2));
            }
        }
        const float m_use = m == -INFINITY ? 0.f : m;  // only scores of -inf so far
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            bf16x8 pf[2];
#pragma unroll
            for (int i = 0; i < 16; ++i) st[t][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[t][i], p.scale_log2, -m_use));
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                u32x4 x;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[i] = pack_bf16x2(st[t][8 * s + 2 * i], st[t][8 * s + 2 * i + 1]);
                    // the sum is of the rounded probabilities, as the product's is
                    const bf16x2 ones{(bf16)1.f, (bf16)1.f};
                    l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, (uint32_t)x[i]), ones, l, false);
                }
                pf[s] = __builtin_bit_cast(bf16x8, x);
            }
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int d = 0; d < ND; ++d)
                    ot[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_frag(v_at + b0, d, 2 * t + s), pf[s], ot[d], 0, 0, 0);
        }
        if (more) vals.commit(lds_offset(sv) + b1);
        const int x = b0;
        b0 = b1, b1 = x;
    };

    auto arrive = [&]() INLINE { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
    __shared__ int s_bad[2];
    // A masked tile whose values are not all finite: 0 * NaN would carry them to rows that do not see
    // them.  A product of its own counts such values among those that a row sees, whose output
    // becomes NaN, and they are zeros from then on.
    auto check_values = [&](int j) INLINE {
        bool bad = false;
        if (!exists(j))
            for (int x = tid; x < CHUNKS; x += 64 * NW) v_buf(b0)[x] = u32x4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < CHUNKS / (64 * NW); ++i) bad |= nonfinite_bits(v_buf(b0)[tid + i * 64 * NW]) != 0;
        if (bad) s_bad[j & 1] = 1;
        lds_barrier();
        if (s_bad[j & 1] == 0) return;
        for (int x = tid; x < CHUNKS; x += 64 * NW) {
            const u32x4 c = v_buf(b0)[x];
            const uint32_t bits = nonfinite_bits(c);
            v_buf(b0)[x] = clear_bits(c, bits);
            v_buf(b1)[x] = one_bits(bits);  // free until the next tile is sent for
        }
        lds_barrier();
#pragma unroll
        for (int d = 0; d < ND; ++d) {
            __builtin_amdgcn_sched_barrier(0);
            f32x16 count;
#pragma unroll
            for (int i = 0; i < 16; ++i) count[i] = 0.f;
#pragma unroll 1
            for (int s = 0; s < 2 * NT; ++s) {
                bf16x8 seen;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    seen[e] = (bf16)(start(j) + 16 * s + 8 * (e >> 2) + 4 * h + (e & 3) <= my_pos ? 1.f : 0.f);
                count = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_frag(v_at + b1, d, s), seen, count, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (count[i] > 0.f) ot[d][i] = NAN;
        }
        lds_barrier();
    };
    // Two buffers, one barrier per tile.  Tiles that every row sees whole come first, without masks.
    int j = 0;
    for (; j < clear; ++j) {
        arrive();
        tile(false, j);
    }
    const AttnRow row = my_row();
    my_pos = row.kind == ROW_SEES ? row.pos : 0x7fffffff;
    for (; j < tiles; ++j) {
        if (threadIdx.x == 0) s_bad[j & 1] = 0;
        arrive();
        check_values(j);
        tile(true, j);
    }
    if constexpr (KG == 2) {  // the second group's results, through LDS, lane by lane
        float* const so = reinterpret_cast<float*>(smem) + (wave * ND * 4 * 64 + lane) * 4;
        __shared__ float s_m[64 * NW], s_l[64 * NW];
        __syncthreads();
        if (kg == 1) {
            s_m[tid] = m, s_l[tid] = l;
#pragma unroll
            for (int t = 0; t < ND; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *reinterpret_cast<f32x4*>(so + (4 * t + i) * 256) =
                        f32x4{ot[t][4 * i], ot[t][4 * i + 1], ot[t][4 * i + 2], ot[t][4 * i + 3]};
        }
        __syncthreads();
        if (kg == 1) return;
        const float top = fmaxf(m, s_m[tid]), m_use = top == -INFINITY ? 0.f : top;
        const float f0 = __builtin_amdgcn_exp2f(m - m_use), f1 = __builtin_amdgcn_exp2f(s_m[tid] - m_use);
        l = f0 * l + f1 * s_l[tid];
#pragma unroll
        for (int t = 0; t < ND; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x4 x = *reinterpret_cast<const f32x4*>(so + (4 * t + i) * 256);
#pragma unroll
                for (int e = 0; e < 4; ++e) ot[t][4 * i + e] = f0 * ot[t][4 * i + e] + f1 * x[e];
            }
    }
    const bool lost = PAGED && __syncthreads_or(keys.bad_page || vals.bad_page);  // an invalid page was read
    if (row.kind == ROW_NONE) return;
    const float sum = row.kind == ROW_ZERO ? 0.f : lost || row.kind == ROW_NAN ? NAN : half_sum(l);
    if (PAGED && p.splits > 1) {
        const int64_t at = (int64_t)split * p.n_tok * p.h_q + row.tok * p.h_q + row.head;
        const float stored = part_sum(sum, row, range);
        if (h == 0) {
            p.part_ml[2 * at] = row.kind == ROW_ZERO ? -INFINITY : m;
            p.part_ml[2 * at + 1] = stored;
        }
        if (stored == 0.f) return;  // not read
#pragma unroll
        for (int t = 0; t < ND; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<f32x4*>(p.part_o + at * D + 32 * t + 8 * i + 4 * h) =
                    f32x4{ot[t][4 * i], ot[t][4 * i + 1], ot[t][4 * i + 2], ot[t][4 * i + 3]};
        return;
    }
    // Two groups of four of the lane's values, exchanged between the halves, make 16 adjacent bytes.  Where all
    // scores are -inf the sum is 0 and O as it stands the result: 0, or NaN where a value is not finite.
    const float inv = sum == 0.f ? 1.f : 1.f / sum;
    bf16* o = reinterpret_cast<bf16*>(p.o) + (row.tok * p.h_q + row.head) * D;
#pragma unroll
    for (int t = 0; t < ND; ++t)
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
            u32x4 y;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int a = 4 * i + 2 * e, c = a + 4;
                const auto r = __builtin_amdgcn_permlane32_swap(pack_bf16x2(ot[t][a] * inv, ot[t][a + 1] * inv),
                                                                pack_bf16x2(ot[t][c] * inv, ot[t][c + 1] * inv), false, false);
                y[e] = r[0], y[2 + e] = r[1];
            }
            if (row.kind == ROW_ZERO) y = u32x4{0, 0, 0, 0};
            *reinterpret_cast<u32x4*>(o + 32 * t + 8 * i + 8 * h) = y;
        }
}

template <int D>
static hipError_t launch_d(int kind, bool paged, const AttnArgs& a, hipStream_t st) {
    const int64_t wgs = (int64_t)a.n_units * a.h_kv * (paged ? a.splits : 1);
    const dim3 grid((unsigned)wgs), block(64 * NW);
    // Two groups where the launch does not fill the GPU with workgroups, two a CU, and the chains are
    // long (a prompt of 4096, 8 heads of 128: 87 -> 66 us; 2048, 16/2 heads of 256: 117 -> 74; filled, or
    // short, the join and the rounds in step cost more: 16384, 8 heads of 128, 553 -> 607; four of
    // 300, 32/8 heads of 128, 15 -> 21).  The limit is a line under the measured borders, alike for the
    // three d: 512 tokens gain at 256 workgroups (d = 128: 17.8 -> 16.7 us) and lose at 320 (20.8 -> 22.2),
    // 768 even out at 384 (26.0, 25.5), 1024 gain at 384 (32.6 -> 30.4) and not at 512 (33.2, 33.7), 2048
    // and more gain up to 512 (58.6 -> 51.1) and lose at 640 (62.3 -> 72.1).  Paged calls split their
    // keys over workgroups instead.
    const int64_t mean = a.n_tok / a.n_req;
    const bool two = !paged && mean >= 512 && wgs <= std::min<int64_t>(512, mean * 3 / 8);
    if (two) hipLaunchKernelGGL((attn_tile_kernel<D, KV_BF16, false, 2>), grid, dim3(128 * NW), 0, st, a);
    else if (!paged) hipLaunchKernelGGL((attn_tile_kernel<D, KV_BF16, false, 1>), grid, block, 0, st, a);
    else if (kind == KV_E4M3) hipLaunchKernelGGL((attn_tile_kernel<D, KV_E4M3, true, 1>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((attn_tile_kernel<D, KV_BF16, true, 1>), grid, block, 0, st, a);
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
