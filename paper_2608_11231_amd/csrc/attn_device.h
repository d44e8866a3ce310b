// Pieces shared by the attention kernels.
//
// Row (token i of a request, query head) with position p attends to the keys j <= p of its
// request: s_j = scale q.k_j, o = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m), m = max_j s_j.
// The key/value head of a group of query heads is shared, so the rows of one (request,
// key/value head) are its tokens times the heads of the group, row = token * group + head: a
// tile of rows covers few tokens, which leaves little of it masked, and reads each key once for
// all heads of the group.
#pragma once
#include "attn_kernels.h"

namespace lkv {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ int64_t clamp_tok(int64_t x, int64_t lo, int64_t hi) { return x < lo ? lo : (x > hi ? hi : x); }

// A workgroup's rows: tokens t0 .. t0 + n of request r, rows row0 .. of its n * group.
struct AttnUnit {
    int r;  // -1: nothing to do
    int64_t t0;
    int n;
    int64_t row0;
};

// Unit u -> (request, row tile).  Every request's last tile, which sees the most keys, comes
// first, as unit u = request, found without looking at the other requests (decoding has only
// these); then the other tiles request by request, from the last on, found by a scan over the
// requests' tile counts.  The host knows only n_tok, so it launches n_req + (n_tok * group - 1) /
// BM units, which bounds the number of tiles; the surplus leaves at once, and so do the units of
// requests that another launch of the call takes.
template <int BM>
__device__ __forceinline__ AttnUnit attn_unit(const AttnArgs& p, int u, int lane) {
    AttnUnit w{-1, 0, 0, 0};
    auto tokens = [&](int r, int64_t& t0) {  // 0 for requests that are not the launch's
        t0 = clamp_tok(p.cu[r], 0, p.n_tok);
        const int n = (int)(clamp_tok(p.cu[r + 1], t0, p.n_tok) - t0);
        const int64_t rows = (int64_t)n * p.group;
        return rows >= p.rows_from && rows <= p.rows_to ? n : 0;
    };
    if (u < p.n_req) {
        w.n = tokens(u, w.t0);
        const int64_t rows = (int64_t)w.n * p.group;
        if (rows == 0) return w;
        w.r = u;
        w.row0 = (rows - 1) / BM * BM;
        return w;
    }
    int left = u - p.n_req;
    for (int r0 = 0; r0 < p.n_req; r0 += 64) {
        const int r = r0 + lane;
        int64_t t0 = 0;
        const int n = r < p.n_req ? tokens(r, t0) : 0;
        const int more = n > 0 ? (int)(((int64_t)n * p.group - 1) / BM) : 0;
        const int incl = wave_incl_scan_int(more);
        const int all = __builtin_amdgcn_readlane(incl, 63);
        if (left < all) {
            const uint64_t after = __ballot(incl > left);
            const int l = __builtin_amdgcn_readfirstlane((int)__builtin_ctzll(after));
            w.r = r0 + l;
            w.n = __builtin_amdgcn_readlane(n, l);
            w.t0 = __builtin_amdgcn_readlane((int)t0, l);  // n_tok is below 2^31
            const int m = __builtin_amdgcn_readlane(more, l);
            const int before = __builtin_amdgcn_readlane(incl, l) - m;
            w.row0 = (int64_t)(m - 1 - (left - before)) * BM;
            return w;
        }
        left -= all;
    }
    return w;
}

// Keys that a request's tokens may see
__device__ __forceinline__ int attn_len(const PagesArgs& pg, int r) {
    const int64_t most = (int64_t)pg.max_pages << pg.page_shift;
    return (int)clamp_tok(pg.len[r], 0, most);
}

// What a row of the tile is.  Only ROW_SEES rows count for the keys that the tile reads and for
// its masks; the others run along unmasked and are replaced when they are stored.
enum { ROW_SEES = 0, ROW_ZERO = 1, ROW_NAN = 2, ROW_NONE = 3 };
struct AttnRow {
    int kind;
    int pos;  // last key seen
    int64_t tok;
    int head;  // query head
};
template <bool PAGED>
__device__ __forceinline__ AttnRow attn_row(const AttnArgs& p, const AttnUnit& w, int64_t row, int hk, int len) {
    AttnRow x{ROW_NONE, -1, 0, 0};
    if (row >= (int64_t)w.n * p.group) return x;
    const int i = (int)((uint32_t)row / (uint32_t)p.group);
    x.tok = w.t0 + i;
    x.head = hk * p.group + (int)((uint32_t)row - (uint32_t)i * (uint32_t)p.group);
    if (!PAGED) {
        x.kind = ROW_SEES;
        x.pos = i;
    } else if (p.pos) {
        x.pos = p.pos[x.tok];
        x.kind = x.pos >= 0 && x.pos < len ? ROW_SEES : ROW_NAN;
    } else {
        x.pos = len - w.n + i;
        x.kind = x.pos >= 0 ? ROW_SEES : ROW_ZERO;
    }
    return x;
}

__device__ __forceinline__ int wave_min_int(int x) {  // of values >= 0
    return 0x7fffffff - wave_max_int(0x7fffffff - x);
}

// The key range [from, to) of part s of `splits`: whole tiles of BN keys, evenly
struct KeyRange {
    int from, to;
};
template <int BN>
__device__ __forceinline__ KeyRange key_range(int end, int splits, int s) {
    const int tiles = (end + BN - 1) / BN;
    const int per = (tiles + splits - 1) / splits;
    const int64_t a = (int64_t)s * per * BN, b = a + (int64_t)per * BN;
    return KeyRange{(int)(a < end ? a : end), (int)(b < end ? b : end)};
}

// A row's sum as stored for the join.  0 says that the row sees no key of the part and that its o is not
// written.  A row whose seen scores are all -inf has a sum of 0 too (and the reference -inf, so no weight),
// but its o counts: NaN where a value is not finite, else 0.
__device__ __forceinline__ float part_sum(float sum, const AttnRow& x, const KeyRange& range) {
    return sum == 0.f && x.kind == ROW_SEES && x.pos >= range.from ? 1.f : sum;
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

// e4m3 pairs -> bf16 pairs times 2^e, exact; scale holds the power of two
__device__ __forceinline__ uint32_t e4m3_pair(uint32_t x, float scale, bool hi) {
    const bf16x2 y = hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, true)
                        : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, false);
    return __builtin_bit_cast(uint32_t, y);
}
__device__ __forceinline__ float exp_scale(uint8_t b) { return __builtin_bit_cast(float, (uint32_t)b << 23); }

}  // namespace lkv
