// Attention of drafted trees over a paged cache.
//
// With s_p = scale q.k_p over the places p that a token sees, out = sum_p e^{s_p - m} v_p / sum_p e^{s_p - m} for any m; m is the
// running maximum of the scores so far, and sums made under an older one are scaled by e^{m_old - m_new}: one pass over the keys and values.
#include "cache.hpp"
#include "device_utils.hpp"

namespace slimspec {
namespace {

template <bool F16> __device__ __forceinline__ float value_of(uint16_t b)
{
    if constexpr (F16) return (float)__builtin_bit_cast(_Float16, b);
    else return bf16_to_float(b);
}
template <bool F16> __device__ __forceinline__ uint16_t bits_of(float x)
{
    if constexpr (F16) return __builtin_bit_cast(uint16_t, (_Float16)x);
    else return __builtin_bit_cast(uint16_t, (__bf16)x);
}

// One wavefront per (token, query head): 64 places at a time, a lane scores one place and then owns four channels of the output.
template <bool F16>
__global__ __launch_bounds__(64) void tree_attention_kernel(CacheView c, int layer, TreeCall call, BatchView b)
{
    __shared__ float weight[64];
    __shared__ int64_t at[64];
    const int token = blockIdx.x, head = blockIdx.y, lane = threadIdx.x;
    int found = -1;
    for (int i = 0; i < b.n; i += 64) {
        const uint64_t hit = __ballot(i + lane < b.n && b.first[min(i + lane, b.n - 1)] <= token && token < b.first[min(i + lane, b.n - 1) + 1]);
        if (hit) found = i + __ffsll((unsigned long long)hit) - 1;
    }
    if (found < 0) return;
    const Sequence q = sequence_of(c, b, found);
    if (!q.valid) return;
    const int t = token - q.first;
    const int64_t base = (int64_t)layer * c.layer_stride + (head / (call.q_heads / c.heads)) * c.head_stride;
    const uint16_t *qr = call.q + token * call.q_token_stride + head * call.q_head_stride;
    float m = kNegInf, l = 0.f, o[4] = {};
    for (int p0 = 0; p0 < q.len + q.tokens; p0 += 64) {
        const int p = p0 + lane, j = p - q.len;
        bool seen = p < q.len + q.tokens;
        if (seen && j >= 0) seen = call.mask ? j < 64 * call.mask_words && (call.mask[(int64_t)token * call.mask_words + (j >> 6)] >> (j & 63) & 1) : j <= t;
        float s = kNegInf;
        at[lane] = -1;
        if (seen) {
            const int page = page_of(c, q.slot, p);
            if (page >= 0) {
                const int64_t e = base + page * c.page_stride + (p & ((1 << c.page_shift) - 1)) * c.place_stride;
                float sum = 0.f;
                for (int i = 0; i < c.head_dim; ++i) sum += value_of<F16>(qr[i]) * value_of<F16>(c.k[e + i]);
                s = sum * call.scale;
                at[lane] = e;
            }
        }
        const float top = fmaxf(m, wave_max(s));
        const float w = at[lane] >= 0 ? fast_exp(s - top) : 0.f;
        const float old = m == top ? 1.f : fast_exp(m - top);
        weight[lane] = w;
        __syncthreads();
        l = l * old + wave_sum(w);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] *= old;
        for (int x = 0; x < 64; ++x) {
            if (at[x] < 0) continue;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (lane + 64 * i < c.head_dim) o[i] += weight[x] * value_of<F16>(c.v[at[x] + lane + 64 * i]);
        }
        m = top;
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (lane + 64 * i < c.head_dim)
            call.out[token * call.out_token_stride + head * call.out_head_stride + lane + 64 * i] = bits_of<F16>(l > 0.f ? o[i] / l : l);
    if (call.lse && lane == 0) call.lse[(int64_t)token * call.q_heads + head] = l > 0.f ? m + fast_log(l) : (l == 0.f ? kNegInf : l);
}

}  // namespace

size_t tree_attention_workspace_bytes(int n, int tokens, int q_heads, int heads, int head_dim)
{
    (void)n; (void)tokens; (void)q_heads; (void)heads; (void)head_dim;
    return 256;
}

hipError_t launch_tree_attention(const CacheView &c, int layer, const TreeCall &call, const BatchView &b, void *workspace, hipStream_t st)
{
    (void)workspace;
    const dim3 grid((unsigned)b.tokens, (unsigned)call.q_heads);
    if (call.f16) tree_attention_kernel<true><<<grid, 64, 0, st>>>(c, layer, call, b);
    else tree_attention_kernel<false><<<grid, 64, 0, st>>>(c, layer, call, b);
    return hipGetLastError();
}

}  // namespace slimspec
