// Write and read of the paged key/value cache.
//
// G lanes move one token, its k and v rows in chunks of 16 elements per lane (16 bytes of e4m3): a
// wave, or a half or a quarter of one where the token has no more chunks than that.
// Small calls are latency: the token's slot is a chain of loads (offsets, position and length,
// page), which starts after the rows to write have been sent for.  Large ones are HBM traffic, each
// row read once and written once: 32768 tokens of 8 heads of 128 in bf16, written and read back,
// 117 us on new inputs, 4.6 TB/s (side by side on one card 110, and with four such tokens one after the
// other in a wave 119).
//
// e4m3 rows carry one power-of-two scale per (token, head).  A power of two costs a
// floating-point code no precision, the scaling is exact, and so is the value read back: 4
// significant bits times 2^e is a bf16 value.  At the largest scale, 2^120, codes stop at 240: the next,
// 256 * 2^120, is past bf16's range, and the largest values would come back infinite.
#include "attn_device.h"

namespace lkv {

namespace {

// Where a token's rows are: pool row of head 0, (page * h_kv << shift) + slot
constexpr int64_t NO_PLACE = -1;    // a position or page that does not exist
constexpr int64_t NO_REQUEST = -2;  // a token outside every request, or (write) one that a later token replaces
// The request of token j is r with cu[r] <= j < cu[r + 1], offsets clamped to [0, n_tok]: r + 1 is the
// number of offsets <= j, counted by the G lanes that have j.
template <bool WRITE, int G>
__device__ __forceinline__ int64_t kv_row(const KvArgs& p, int64_t j, int lane) {
    int count = 0;
    for (int r0 = 0; r0 <= p.n_req; r0 += G) {
        const int i = r0 + lane % G;
        uint64_t before = __ballot(i <= p.n_req && clamp_tok(p.cu[i], 0, p.n_tok) <= j);
        if (G < 64) before = (before >> (lane / G * G)) & ((1ull << (G & 63)) - 1);
        count += __builtin_popcountll(before);
    }
    const int r = count - 1;
    if (r < 0 || r >= p.n_req) return NO_REQUEST;
    const int64_t t0 = clamp_tok(p.cu[r], 0, p.n_tok), t1 = clamp_tok(p.cu[r + 1], t0, p.n_tok);
    const int len = attn_len(p.pg, r);
    if (j < t0 || j >= t1) return NO_REQUEST;
    const int64_t pos = p.pos ? p.pos[j] : len - (t1 - j);
    if (WRITE && p.pos && j + 1 < t1 && p.pos[j + 1] == pos) return NO_REQUEST;  // of such neighbours the last is written
    if (pos < 0 || pos >= len) return NO_PLACE;
    const int page = p.pg.table[(int64_t)r * p.pg.max_pages + (pos >> p.pg.page_shift)];
    if (page < 0 || page >= p.pg.n_page) return NO_PLACE;
    return (((int64_t)page * p.h_kv) << p.pg.page_shift) + (pos & ((1 << p.pg.page_shift) - 1));
}

// 16 elements as they lie in memory
template <typename T>
struct Raw {
    u32x4 x[sizeof(T)];
};
template <typename T>
__device__ __forceinline__ Raw<T> load_raw(const void* s) {
    Raw<T> r;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) r.x[i] = reinterpret_cast<const u32x4*>(s)[i];
    return r;
}
template <typename T>
__device__ __forceinline__ void store_raw(void* d, const Raw<T>& r) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) reinterpret_cast<u32x4*>(d)[i] = r.x[i];
}

// Scale byte of a row whose largest finite magnitude is amax: 127 + the least e in [-100, 120]
// with amax <= 448 * 2^e (448 = 1.75 * 2^8 is e4m3's largest)
__device__ __forceinline__ uint32_t scale_byte(float amax) {
    const uint32_t u = __builtin_bit_cast(uint32_t, amax);
    const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    return (uint32_t)(127 + min(max(e, -100), 120));
}

// Maximum over groups of 4, 8 or 16 adjacent lanes, in registers: neighbours, pairs, then mirrored halves
__device__ __forceinline__ float group_max(float x, int lanes) {
    x = fmaxf(x, dpp_mov<0xb1, 0xf, false>(x));   // quad_perm 1 0 3 2
    x = fmaxf(x, dpp_mov<0x4e, 0xf, false>(x));   // quad_perm 2 3 0 1
    if (lanes >= 8) x = fmaxf(x, dpp_mov<0x141, 0xf, false>(x));   // row_half_mirror
    if (lanes >= 16) x = fmaxf(x, dpp_mov<0x140, 0xf, false>(x));  // row_mirror
    return x;
}

// Codes of 16 bf16 and the scale byte of their row, which the per_head lanes of a head (adjacent, a power
// of two) hold between them
__device__ __forceinline__ u32x4 encode(const Raw<bf16>& r, int per_head, uint32_t& byte) {
    float x[16], amax = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t b = r.x[i / 4][i % 4];
        x[2 * i] = __builtin_bit_cast(float, b << 16);
        x[2 * i + 1] = __builtin_bit_cast(float, b & 0xffff0000u);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float a = __builtin_fabsf(x[i]);
        amax = a < INFINITY ? fmaxf(amax, a) : amax;  // infinities and NaN do not count and become NaN
    }
    amax = group_max(amax, per_head);
    byte = scale_byte(amax);
    const float inv = exp_scale((uint8_t)(254 - byte));  // 2^-e, exact
    const float most = byte == 127 + 120 ? 240.f : 448.f;
    u32x4 out;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = __builtin_fabsf(x[4 * i + e]) < INFINITY ? __builtin_amdgcn_fmed3f(x[4 * i + e] * inv, -most, most) : NAN;
        int word = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
        word = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], word, true);
        out[i] = (uint32_t)word;
    }
    return out;
}
__device__ __forceinline__ Raw<bf16> decode(u32x4 b, uint8_t byte) {
    const float s = exp_scale(byte);
    Raw<bf16> r;
#pragma unroll
    for (int i = 0; i < 2; ++i)
        r.x[i] = u32x4{e4m3_pair(b[2 * i], s, false), e4m3_pair(b[2 * i], s, true), e4m3_pair(b[2 * i + 1], s, false),
                       e4m3_pair(b[2 * i + 1], s, true)};
    return r;
}

}  // namespace

// T: element of the tokens (and of pages that are not e4m3)
template <typename T, bool E4M3, int G>
__global__ __launch_bounds__(256) void kv_write_kernel(KvArgs p) {
    const int lane = threadIdx.x & 63, gl = lane % G;
    const int64_t j = ((int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * (64 / G) + (G < 64 ? lane / G : 0);
    if (j >= p.n_tok) return;
    const int per_head = p.d / 16, units = p.h_kv * per_head;
    const T* ks = reinterpret_cast<const T*>(p.k) + j * p.k_stride;
    const T* vs = reinterpret_cast<const T*>(p.v) + j * p.v_stride;
    Raw<T> k = {}, v = {};
    if (gl < units) k = load_raw<T>(ks + 16 * gl), v = load_raw<T>(vs + 16 * gl);
    const int64_t first = kv_row<true, G>(p, j, lane);
    if (first < 0) return;
    for (int u0 = 0; u0 < units; u0 += G) {
        const int u = u0 + gl, hk = u / per_head, c = u % per_head;
        if (u0 > 0 && u < units) k = load_raw<T>(ks + 16 * u), v = load_raw<T>(vs + 16 * u);
        const int64_t row = first + ((int64_t)hk << p.pg.page_shift);
        if constexpr (E4M3) {
            uint32_t kb, vb;
            const u32x4 kc = encode(k, per_head, kb), vc = encode(v, per_head, vb);
            if (u >= units) continue;
            *reinterpret_cast<u32x4*>(reinterpret_cast<uint8_t*>(p.pg.k) + row * p.d + 16 * c) = kc;
            *reinterpret_cast<u32x4*>(reinterpret_cast<uint8_t*>(p.pg.v) + row * p.d + 16 * c) = vc;
            if (c == 0) p.pg.k_exp[row] = (uint8_t)kb, p.pg.v_exp[row] = (uint8_t)vb;
        } else if (u < units) {
            store_raw(reinterpret_cast<T*>(p.pg.k) + row * p.d + 16 * c, k);
            store_raw(reinterpret_cast<T*>(p.pg.v) + row * p.d + 16 * c, v);
        }
    }
}

template <typename T, bool E4M3, int G>
__global__ __launch_bounds__(256) void kv_read_kernel(KvArgs p) {
    const int lane = threadIdx.x & 63, gl = lane % G;
    const int64_t j = ((int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * (64 / G) + (G < 64 ? lane / G : 0);
    if (j >= p.n_tok) return;
    const int per_head = p.d / 16, units = p.h_kv * per_head;
    const int64_t first = kv_row<false, G>(p, j, lane);
    if (first == NO_REQUEST) return;
    for (int u = gl; u < units; u += G) {
        const int hk = u / per_head, c = u % per_head;
        const int64_t row = first + ((int64_t)hk << p.pg.page_shift);
        Raw<T> k, v;
        if (first == NO_PLACE) {
            const uint32_t nan = sizeof(T) == 2 ? 0x7fc07fc0u : 0x7fc00000u;
#pragma unroll
            for (int i = 0; i < (int)sizeof(T); ++i) k.x[i] = v.x[i] = u32x4{nan, nan, nan, nan};
        } else if constexpr (E4M3) {
            const u32x4 kc = *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint8_t*>(p.pg.k) + row * p.d + 16 * c);
            const u32x4 vc = *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint8_t*>(p.pg.v) + row * p.d + 16 * c);
            const uint8_t kb = p.pg.k_exp[row], vb = p.pg.v_exp[row];
            k = decode(kc, kb), v = decode(vc, vb);
        } else {
            k = load_raw<T>(reinterpret_cast<const T*>(p.pg.k) + row * p.d + 16 * c);
            v = load_raw<T>(reinterpret_cast<const T*>(p.pg.v) + row * p.d + 16 * c);
        }
        store_raw(reinterpret_cast<T*>(p.k) + j * p.k_stride + (int64_t)16 * u, k);
        store_raw(reinterpret_cast<T*>(p.v) + j * p.v_stride + (int64_t)16 * u, v);
    }
}

template <typename T, bool E4M3, int G>
static hipError_t launch_kv_g(const KvArgs& a, bool write, hipStream_t st) {
    constexpr int PER = 256 / G;  // tokens of a workgroup
    const dim3 grid((unsigned)((a.n_tok + PER - 1) / PER)), block(256);
    if (write) hipLaunchKernelGGL((kv_write_kernel<T, E4M3, G>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((kv_read_kernel<T, E4M3, G>), grid, block, 0, st, a);
    return hipGetLastError();
}
template <typename T, bool E4M3>
static hipError_t launch_kv(const KvArgs& a, bool write, hipStream_t st) {
    // Lanes per token: 131072 tokens of one head of 128 are written in 23 us in bf16 and 31 in e4m3, where
    // idle lanes cost as much as busy ones; by a wave each 42 and 91.  Between 16 and 32 chunks only
    // e4m3 gains (4 heads of 128: 101 -> 86 us; bf16 101 -> 103).
    const int units = a.h_kv * a.d / 16;
    if (units <= 16) return launch_kv_g<T, E4M3, 16>(a, write, st);
    if constexpr (E4M3)
        if (units <= 32) return launch_kv_g<T, E4M3, 32>(a, write, st);
    return launch_kv_g<T, E4M3, 64>(a, write, st);
}
static hipError_t launch_kv_kind(const KvArgs& a, bool write, hipStream_t st) {
    switch (a.kind) {
        case KV_F32: return launch_kv<float, false>(a, write, st);
        case KV_BF16: return launch_kv<bf16, false>(a, write, st);
        case KV_E4M3: return launch_kv<bf16, true>(a, write, st);
    }
    return hipErrorInvalidValue;
}
hipError_t launch_kv_write(const KvArgs& a, hipStream_t st) { return launch_kv_kind(a, true, st); }
hipError_t launch_kv_read(const KvArgs& a, hipStream_t st) { return launch_kv_kind(a, false, st); }

}  // namespace lkv
