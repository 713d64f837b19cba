// Attention of a batch of prompts.
#include <hip/hip_runtime.h>

#include "device_util.h"
#include "kernels_attention.h"
#include "launch.h"

// ---------------------------------------------------------------------------
// Any layout, dtype and head_dim: a wavefront per query and head.  Keys in steps of 64, one a lane for the scores; then lanes
// are dims, and the softmax weights go round by shuffles.  Keys that the query does not see are not read.
namespace {
template <typename T>
__global__ __launch_bounds__(256) void attention_general_kernel(attention_args a)
{
    const int64_t id = blockIdx.x;
    const attention_tile t = a.tiles[id / a.num_heads];
    const int head = (int)(id % a.num_heads), lane = threadIdx.x & 63, D = a.head_dim;
    const T* const kb = static_cast<const T*>(a.k) + (int64_t)t.kv_row0 * a.ldk + (int64_t)(head / a.group) * D;
    const T* const vb = static_cast<const T*>(a.v) + (int64_t)t.kv_row0 * a.ldv + (int64_t)(head / a.group) * D;
    for (int i = threadIdx.x >> 6; i < t.rows; i += 4) {
        const T* const q = static_cast<const T*>(a.q) + (int64_t)(t.q_row0 + i) * a.ldq + (int64_t)head * D;
        const int sees = max(0, min(t.num_kv, t.ahead + i + 1));
        float o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
        for (int j0 = 0; j0 < sees; j0 += 64) {
            const int n = min(64, sees - j0);
            float x = -INFINITY;
            if (lane < n) {
                const T* const k = kb + (int64_t)(j0 + lane) * a.ldk;
                float s = 0.f;
                for (int d = 0; d < D; ++d) s += elem<T>::load(q + d) * elem<T>::load(k + d);
                x = s * a.scale;
            }
            float mx = x;
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor(mx, off, 64));
            mx = fmaxf(m, mx);
            const float ref = mx == -INFINITY ? 0.f : mx, alpha = m == -INFINITY ? 0.f : expf(m - ref);
            const float p = lane < n ? expf(x - ref) : 0.f;
            m = mx;
            l = l * alpha + wave_sum(p);
#pragma unroll
            for (int c = 0; c < 4; ++c) o[c] *= alpha;
            for (int j = 0; j < n; ++j) {
                const float pj = __shfl(p, j, 64);
                const T* const v = vb + (int64_t)(j0 + j) * a.ldv;
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (lane + 64 * c < D) o[c] += pj * elem<T>::load(v + lane + 64 * c);
            }
        }
        T* const out = static_cast<T*>(a.o) + (int64_t)(t.q_row0 + i) * a.ldo + (int64_t)head * D;
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (lane + 64 * c < D) elem<T>::store(out + lane + 64 * c, l == 0.f ? 0.f : o[c] / l);
    }
}
}  // namespace

hipError_t launch_attention_general(const attention_args& a, int32_t dtype, hipStream_t stream)
{
    const dim3 grid((uint32_t)((int64_t)a.num_tiles * a.num_heads));
    if (dtype == LORA_F32)
        LORA_LAUNCH(LORA_K_ATTENTION_GENERAL, (attention_general_kernel<float>), grid, dim3(256), 0, stream, a);
    else
        LORA_LAUNCH(LORA_K_ATTENTION_GENERAL, (attention_general_kernel<bf16_t>), grid, dim3(256), 0, stream, a);
    return hipGetLastError();
}
