#include "attn_device.h"

namespace lkv {

// Join of the key ranges' results: with m = max m_s, o = sum 2^(m_s - m) o_s / sum 2^(m_s - m) l_s.
// A part in which the row sees no key has l_s = 0 and no o_s; every other one counts, also where its
// weight underflows to 0, since 0 times a value that is not finite is NaN (see part_sum).
// A workgroup joins one row: every wave forms all weights, a part per lane, and adds a quarter of
// the parts, whose loads do not wait for each other; the quarters meet in LDS.  Short chains of
// loads are what counts here: a decoding call waits for it (four contexts of 8K in 16 parts: 28 us
// with the attention; 49 with one wave that walks the parts).
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
    uint64_t written[JOIN_PARTS / 64];
#pragma unroll
    for (int i = 0; i < JOIN_PARTS / 64; ++i) {
        written[i] = __ballot(ls[i] != 0.f);
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
                for (int e = 0; e < E; ++e) o[e] += s < to && (written[i] >> (s & 63)) & 1 ? w * y[k][e] : 0.f;
            }
        }
    }
    if (wave > 0)
#pragma unroll
        for (int e = 0; e < E; ++e) so[wave - 1][E * lane + e] = o[e];
    __syncthreads();
    if (wave > 0) return;
    const float inv = l == 0.f ? 1.f : 1.f / l;
    T* out = reinterpret_cast<T*>(p.o) + at * D + E * lane;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int x = E * lane + e;
        out[e] = (T)((o[e] + so[0][x] + so[1][x] + so[2][x]) * inv);
    }
}

// The same with a wave per row, whose loads of four parts are on their way with those of the weights.
template <int D, typename T>
__global__ __launch_bounds__(256) void attn_join_rows_kernel(AttnArgs p) {
    constexpr int E = D / 64;  // elements of a lane
    const int lane = threadIdx.x & 63;
    const int64_t rows = p.n_tok * p.h_q, at = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (at >= rows) return;
    const int64_t tok = at / p.h_q;
    if (tok < clamp_tok(p.cu[0], 0, p.n_tok) || tok >= clamp_tok(p.cu[p.n_req], 0, p.n_tok)) return;
    const float* part = p.part_o + at * D + E * lane;
    const bool in = lane < p.splits;
    float m = in ? p.part_ml[2 * (lane * rows + at)] : -INFINITY, l = in ? p.part_ml[2 * (lane * rows + at) + 1] : 0.f;
    float y[4][E], o[E];
    auto load = [&](int s0) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e) y[k][e] = part[min(s0 + k, p.splits - 1) * rows * D + e];
    };
    load(0);
    float top = m;
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) top = fmaxf(top, __shfl_xor(top, i));
    const float f = l == 0.f ? 0.f : __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.f : top));
    const uint64_t written = __ballot(l != 0.f);  // no bits past the last part
    l *= f;
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) l += __shfl_xor(l, i);
    l = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, l)));
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.f;
    for (int s0 = 0; s0 < p.splits; s0 += 4) {
        if (s0 > 0) load(s0);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float w = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f), s0 + k));
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] += (written >> (s0 + k)) & 1 ? w * y[k][e] : 0.f;
        }
    }
    const float inv = l == 0.f ? 1.f : 1.f / l;
    T* out = reinterpret_cast<T*>(p.o) + at * D + E * lane;
#pragma unroll
    for (int e = 0; e < E; ++e) out[e] = (T)(o[e] * inv);
}

template <int D, typename T>
static void launch_join(const AttnArgs& a, hipStream_t st) {
    const int64_t rows = a.n_tok * a.h_q;
    // A wave per row where the parts are few or the rows fill the GPU (two chunks of 512 tokens, 16/2 heads
    // of 256 in e4m3, 4 parts: 299 -> 282 us with the attention; 128 tokens over 8K, 32/8 heads of 128, 16
    // parts: 44 -> 39), a workgroup where they are many and the rows few (one token over 32K, 64 parts:
    // 20 us against 23).
    if (a.splits <= 8 || (a.splits <= 64 && rows >= 1024)) hipLaunchKernelGGL((attn_join_rows_kernel<D, T>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((attn_join_kernel<D, T>), dim3((unsigned)rows), dim3(256), 0, st, a);
}

hipError_t launch_attn_join(int d, bool f32, const AttnArgs& a, hipStream_t st) {
    if (d == 64 && f32) launch_join<64, float>(a, st);
    else if (d == 64) launch_join<64, bf16>(a, st);
    else if (d == 128 && f32) launch_join<128, float>(a, st);
    else if (d == 128) launch_join<128, bf16>(a, st);
    else if (d == 256 && !f32) launch_join<256, bf16>(a, st);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

}  // namespace lkv
