// Decode step over a paged key/value cache: one query token per sequence.
#include <math.h>

#include "common.cuh"
#include "paged.cuh"

namespace tilemix {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct PagedDecodeParams {
    PagedCache c;
    int Hq, R;                      // query heads, query heads per KV head
    float scale_log2;
    const uint8_t* q;
    uint8_t* out;
    int64_t qs[2], os[2];           // bytes: (batch, head)
    float* lse;
};

// Plain form: one CTA per query head, a warp takes every fourth key, its lanes the head dimension.
template <class T, int D, bool INT8>
__global__ void __launch_bounds__(128)
paged_decode_kernel(const PagedDecodeParams prm) {
    constexpr int E = D / 32;
    const PagedCache& c = prm.c;
    const int b = blockIdx.y, hq = blockIdx.x, hk = hq / prm.R, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int len = paged_len(c, b);
    auto value = [](const uint8_t* p, int e) {
        if constexpr (INT8) return static_cast<float>(reinterpret_cast<const int8_t*>(p)[e]);
        else return static_cast<float>(reinterpret_cast<const T*>(p)[e]);
    };
    constexpr int kBytes = INT8 ? 1 : 2;
    float q[E], o[E], m = -INFINITY, z = 0.f;
    const T* qrow = reinterpret_cast<const T*>(prm.q + b * prm.qs[0] + hq * prm.qs[1]);
    for (int i = 0; i < E; ++i) { q[i] = static_cast<float>(qrow[lane + 32 * i]); o[i] = 0.f; }
    for (int pos = warp; pos < len; pos += 4) {
        const int page = paged_page(c, b, pos);
        if (page < 0) continue;
        const int at = pos & ((1 << c.page_shift) - 1);
        const uint8_t* k = c.k_pool + kBytes * (page * c.ks[0] + hk * c.ks[1] + at * c.ks[2]);
        const uint8_t* v = c.v_pool + kBytes * (page * c.vs[0] + hk * c.vs[1] + at * c.vs[2]);
        const int64_t so = ((static_cast<int64_t>(page) * c.Hk + hk) << c.page_shift) + at;
        float s = 0.f;
        for (int i = 0; i < E; ++i) s += q[i] * value(k, lane + 32 * i);
        for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
        s *= prm.scale_log2;
        if (INT8) s *= c.k_scale[so];
        const float m_new = fmaxf(m, s), use = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = exp2f(m - use), p = exp2f(s - use);
        z = z * alpha + p;
        const float pv = INT8 ? p * c.v_scale[so] : p;
        for (int i = 0; i < E; ++i) o[i] = o[i] * alpha + pv * value(v, lane + 32 * i);
        m = m_new;
    }
    __shared__ float ms[4], zs[4], os[4][D];
    for (int i = 0; i < E; ++i) os[warp][lane + 32 * i] = o[i];
    if (lane == 0) { ms[warp] = m; zs[warp] = z; }
    __syncthreads();
    if (threadIdx.x >= D) return;
    m = fmaxf(fmaxf(ms[0], ms[1]), fmaxf(ms[2], ms[3]));
    const float use = m == -INFINITY ? 0.f : m;
    float sum = 0.f;
    z = 0.f;
    for (int w = 0; w < 4; ++w) { const float a = exp2f(ms[w] - use); z += zs[w] * a; sum += os[w][threadIdx.x] * a; }
    reinterpret_cast<T*>(prm.out + b * prm.os[0] + hq * prm.os[1])[threadIdx.x] = static_cast<T>(z == 0.f ? 0.f : sum / z);
    if (threadIdx.x == 0 && prm.lse != nullptr) prm.lse[static_cast<int64_t>(b) * prm.Hq + hq] = z == 0.f ? -INFINITY : (m + log2f(z)) * kLn2;
}

using DecodeKernel = void (*)(const PagedDecodeParams);

template <class T>
DecodeKernel pick(int d, bool int8) {
    if (d == 128) return int8 ? paged_decode_kernel<T, 128, true> : paged_decode_kernel<T, 128, false>;
    return int8 ? paged_decode_kernel<T, 64, true> : paged_decode_kernel<T, 64, false>;
}

constexpr size_t kWorkspace = 256;

int resolve_decode(const tilemix_paged_t* p, int heads_q, PagedCache* c) {
    const int rc = resolve_paged(p, c);
    if (rc) return rc;
    if (heads_q <= 0 || heads_q % p->heads_kv != 0 || p->batch > 65535) return TILEMIX_ERR_SHAPE;
    return TILEMIX_OK;
}

int row_strides(const int64_t* in, int B, int H, int d, bool output, int64_t out[2]) {
    const int64_t size[2] = {B, H}, dense[2] = {static_cast<int64_t>(H) * d, d};
    for (int i = 0; i < 2; ++i) {
        const int64_t s = in != nullptr ? in[i] : dense[i];
        if (s < 0 || s > (int64_t{1} << 40) || (output && size[i] > 1 && s < d)) return TILEMIX_ERR_SHAPE;
        if (size[i] > 1 && s * 2 % 16 != 0) return TILEMIX_ERR_ALIGN;
        out[i] = size[i] == 1 ? 0 : 2 * s;
    }
    return TILEMIX_OK;
}

}  // namespace
}  // namespace tilemix

using namespace tilemix;

extern "C" {

size_t tilemix_paged_decode_workspace_size(const tilemix_paged_t* p, int32_t heads_q) {
    PagedCache c;
    return resolve_decode(p, heads_q, &c) ? 0 : kWorkspace;
}

int tilemix_paged_decode(const tilemix_paged_t* p, int32_t heads_q, float softmax_scale, const void* q, const int64_t* q_stride,
                         void* out, const int64_t* out_stride, float* lse, void* workspace, size_t workspace_bytes,
                         void* stream) {
    PagedDecodeParams prm{};
    int rc = resolve_decode(p, heads_q, &prm.c);
    if (rc) return rc;
    if (!q || !out || !workspace) return TILEMIX_ERR_NULL;
    if (!aligned16(q) || !aligned16(out) || !aligned16(workspace)) return TILEMIX_ERR_ALIGN;
    if ((rc = row_strides(q_stride, p->batch, heads_q, p->head_dim, false, prm.qs))) return rc;
    if ((rc = row_strides(out_stride, p->batch, heads_q, p->head_dim, true, prm.os))) return rc;
    if (workspace_bytes < kWorkspace) return TILEMIX_ERR_WORKSPACE;
    prm.Hq = heads_q; prm.R = heads_q / p->heads_kv;
    prm.scale_log2 = (softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf(static_cast<float>(p->head_dim))) * kLog2e;
    prm.q = static_cast<const uint8_t*>(q);
    prm.out = static_cast<uint8_t*>(out);
    prm.lse = lse;
    const bool int8 = p->cache_type == TILEMIX_CACHE_INT8;
    const DecodeKernel kernel = p->act_type == TILEMIX_TYPE_FP16 ? pick<__half>(p->head_dim, int8) : pick<__nv_bfloat16>(p->head_dim, int8);
    kernel<<<dim3(heads_q, p->batch), 128, 0, static_cast<cudaStream_t>(stream)>>>(prm);
    g_launch_count.fetch_add(1);
    return static_cast<int>(cudaGetLastError());
}

}  // extern "C"
