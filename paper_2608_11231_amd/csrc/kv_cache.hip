// Write and read of the paged key/value cache.
//
// One wave moves one token's k and v rows, in chunks of 16 elements per lane (16 bytes of e4m3).
// The rows are read once and written once; both are bound by HBM for many tokens and by latency
// for few, so the wave finds its request with one pass of ballots over the offsets.
//
// e4m3 rows carry one power-of-two scale per (token, head).  A power of two costs a
// floating-point code no precision, the scaling is exact, and so is the value read back: 4
// significant bits times 2^e is a bf16 value.
#include "attn_device.h"

namespace lkv {

namespace {

struct KvSlot {
    int r;           // -1: token outside every request
    int64_t row;     // pool row of head 0: (page * h_kv << shift) + slot; -1: no such position or page
    bool duplicate;  // the next token of the request has the same position
};

// The request of token j is r with cu[r] <= j < cu[r + 1]; offsets are clamped to [0, n_tok].
__device__ __forceinline__ KvSlot kv_slot(const KvArgs& p, int64_t j, int lane) {
    KvSlot s{-1, -1, false};
    int count = 0;  // offsets <= j
    for (int r0 = 0; r0 <= p.n_req; r0 += 64) {
        const int r = r0 + lane;
        const bool before = r <= p.n_req && clamp_tok(p.cu[r], 0, p.n_tok) <= j;
        count += __builtin_popcountll(__ballot(before));
    }
    const int r = count - 1;
    if (r < 0 || r >= p.n_req) return s;
    const int64_t t0 = clamp_tok(p.cu[r], 0, p.n_tok), t1 = clamp_tok(p.cu[r + 1], t0, p.n_tok);
    if (j < t0 || j >= t1) return s;
    s.r = r;
    const int len = attn_len(p.pg, r);
    const int64_t pos = p.pos ? p.pos[j] : len - (t1 - j);
    s.duplicate = p.pos && j + 1 < t1 && p.pos[j + 1] == pos;
    if (pos < 0 || pos >= len) return s;
    const int page = p.pg.table[(int64_t)r * p.pg.max_pages + (pos >> p.pg.page_shift)];
    if (page < 0 || page >= p.pg.n_page) return s;
    s.row = (((int64_t)page * p.h_kv) << p.pg.page_shift) + (pos & ((1 << p.pg.page_shift) - 1));
    return s;
}

// 16 bf16 elements, widened
struct Vals {
    float x[16];
};
__device__ __forceinline__ Vals load16(const bf16* s) {
    Vals v;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const u32x4 b = reinterpret_cast<const u32x4*>(s)[i];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v.x[8 * i + 2 * e] = __builtin_bit_cast(float, b[e] << 16);
            v.x[8 * i + 2 * e + 1] = __builtin_bit_cast(float, b[e] & 0xffff0000u);
        }
    }
    return v;
}

// Scale byte of a row whose largest finite magnitude is amax: 127 + the least e in [-100, 120]
// with amax <= 448 * 2^e (448 = 1.75 * 2^8 is e4m3's largest)
__device__ __forceinline__ uint32_t scale_byte(float amax) {
    const uint32_t u = __builtin_bit_cast(uint32_t, amax);
    const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    return (uint32_t)(127 + min(max(e, -100), 120));
}

template <typename T, bool E4M3>
__device__ __forceinline__ void write_row(const KvArgs& p, const T* src, void* pages, uint8_t* exps, int64_t row, int lane,
                                          bool active, int per_head, int c) {
    // lanes of one head are adjacent, per_head of them (a power of two)
    if constexpr (!E4M3) {
        if (!active) return;
        const u32x4* s = reinterpret_cast<const u32x4*>(src);
        u32x4* d = reinterpret_cast<u32x4*>(reinterpret_cast<T*>(pages) + row * p.d + 16 * c);
#pragma unroll
        for (int i = 0; i < (int)sizeof(T); ++i) d[i] = s[i];
        return;
    } else {
    Vals v = {};
    if (active) v = load16(src);
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float a = __builtin_fabsf(v.x[i]);
        amax = a < INFINITY ? fmaxf(amax, a) : amax;  // infinities and NaN do not count and become NaN
    }
    for (int i = 1; i < per_head; i <<= 1) amax = fmaxf(amax, __shfl_xor(amax, i));
    const uint32_t byte = scale_byte(amax);
    const float inv = exp_scale((uint8_t)(254 - byte));  // 2^-e, exact
    u32x4 out;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float x = v.x[4 * i + e];
            y[e] = __builtin_fabsf(x) < INFINITY ? x * inv : NAN;
        }
        int word = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
        word = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], word, true);
        out[i] = (uint32_t)word;
    }
    if (!active) return;
    *reinterpret_cast<u32x4*>(reinterpret_cast<uint8_t*>(pages) + row * p.d + 16 * c) = out;
    if (c == 0) exps[row] = (uint8_t)byte;
    }
}

template <typename T, bool E4M3>
__device__ __forceinline__ void read_row(const KvArgs& p, T* dst, const void* pages, const uint8_t* exps, int64_t row, int c) {
    u32x4* d = reinterpret_cast<u32x4*>(dst);
    if (row < 0) {
        const uint32_t nan = sizeof(T) == 2 ? 0x7fc07fc0u : 0x7fc00000u;
#pragma unroll
        for (int i = 0; i < (int)sizeof(T); ++i) d[i] = u32x4{nan, nan, nan, nan};
    } else if constexpr (!E4M3) {
        const u32x4* s = reinterpret_cast<const u32x4*>(reinterpret_cast<const T*>(pages) + row * p.d + 16 * c);
#pragma unroll
        for (int i = 0; i < (int)sizeof(T); ++i) d[i] = s[i];
    } else {
        const u32x4 b = *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint8_t*>(pages) + row * p.d + 16 * c);
        const float s = exp_scale(exps[row]);
#pragma unroll
        for (int i = 0; i < 2; ++i)
            d[i] = u32x4{e4m3_pair(b[2 * i], s, false), e4m3_pair(b[2 * i], s, true), e4m3_pair(b[2 * i + 1], s, false),
                         e4m3_pair(b[2 * i + 1], s, true)};
    }
}

}  // namespace

template <typename T, bool E4M3, bool WRITE>
__global__ __launch_bounds__(256) void kv_move_kernel(KvArgs p) {
    const int lane = threadIdx.x & 63;
    const int64_t j = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (j >= p.n_tok) return;
    const KvSlot s = kv_slot(p, j, lane);
    if (s.r < 0) return;
    // of neighbours with one position the last is written
    if (WRITE && (s.row < 0 || s.duplicate)) return;
    const int per_head = p.d / 16, units = p.h_kv * per_head;
    for (int u0 = 0; u0 < units; u0 += 64) {
        const int u = u0 + lane, hk = u / per_head, c = u % per_head;
        const bool active = u < units;
        const int64_t row = s.row + ((int64_t)hk << p.pg.page_shift);
        T* k = reinterpret_cast<T*>(p.k) + j * p.k_stride + (int64_t)16 * u;
        T* v = reinterpret_cast<T*>(p.v) + j * p.v_stride + (int64_t)16 * u;
        if (WRITE) {
            write_row<T, E4M3>(p, k, p.pg.k, p.pg.k_exp, row, lane, active, per_head, c);
            write_row<T, E4M3>(p, v, p.pg.v, p.pg.v_exp, row, lane, active, per_head, c);
        } else if (active) {
            read_row<T, E4M3>(p, k, p.pg.k, p.pg.k_exp, s.row < 0 ? -1 : row, c);
            read_row<T, E4M3>(p, v, p.pg.v, p.pg.v_exp, s.row < 0 ? -1 : row, c);
        }
    }
}

template <bool WRITE>
static hipError_t launch_kv_move(const KvArgs& a, hipStream_t st) {
    const dim3 grid((unsigned)((a.n_tok + 3) / 4));
    if (a.kind == KV_F32) hipLaunchKernelGGL((kv_move_kernel<float, false, WRITE>), grid, dim3(256), 0, st, a);
    else if (a.kind == KV_BF16) hipLaunchKernelGGL((kv_move_kernel<bf16, false, WRITE>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((kv_move_kernel<bf16, true, WRITE>), grid, dim3(256), 0, st, a);
    return hipGetLastError();
}
hipError_t launch_kv_write(const KvArgs& a, hipStream_t st) { return launch_kv_move<true>(a, st); }
hipError_t launch_kv_read(const KvArgs& a, hipStream_t st) { return launch_kv_move<false>(a, st); }

}  // namespace lkv
