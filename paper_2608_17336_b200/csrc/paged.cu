// Paged key/value cache: the checks of its description, writing new tokens (quantised where the cache is INT8) and reading
// contexts back.  Both kernels move bytes: a row of head_dim values of one (token, head) is taken by d / 16 lanes, K and V
// together.
#include <algorithm>
#include <type_traits>

#include "common.cuh"
#include "paged.cuh"
#include "ptx_sm100.cuh"
#include "quant8.cuh"

namespace tilemix {

namespace {

// Element strides of a tensor of `n` axes; an axis of one entry may carry any stride, and gets that of a row.  Checked: 16-byte
// multiples, and that no two rows overlap (sorted by stride, each axis steps over the extent of those below it).
int checked_strides(const int64_t* in, const int64_t* size, int n, int d, int elem_bytes, int64_t* out) {
    int order[3] = {0, 1, 2};
    for (int i = 0; i < n; ++i) {
        out[i] = size[i] == 1 ? d : in[i];
        if (out[i] < d) return TILEMIX_ERR_SHAPE;
        if (out[i] > (int64_t{1} << 40) / elem_bytes - 16) return TILEMIX_ERR_SHAPE;     // (what a tensor map can hold)
        if (out[i] * elem_bytes % 16 != 0) return TILEMIX_ERR_ALIGN;
    }
    std::sort(order, order + n, [&](int a, int b) { return out[a] < out[b]; });
    __int128 extent = d;
    for (int i = 0; i < n; ++i) {
        const int a = order[i];
        if (size[a] == 1) continue;
        if (out[a] < extent) return TILEMIX_ERR_SHAPE;
        extent += static_cast<__int128>(out[a]) * (size[a] - 1);
    }
    return TILEMIX_OK;
}

bool all_zero3(const int64_t s[3]) { return s[0] == 0 && s[1] == 0 && s[2] == 0; }
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

}  // namespace

int resolve_paged(const tilemix_paged_t* p, PagedCache* c) {
    if (p == nullptr) return TILEMIX_ERR_NULL;
    if (p->batch <= 0 || p->heads_kv <= 0 || p->head_dim <= 0 || p->page_size <= 0 || p->n_pages <= 0 || p->max_pages <= 0)
        return TILEMIX_ERR_SHAPE;
    if ((p->head_dim != 64 && p->head_dim != 128) || (p->act_type != TILEMIX_TYPE_FP16 && p->act_type != TILEMIX_TYPE_BF16) ||
        (p->cache_type != TILEMIX_CACHE_16BIT && p->cache_type != TILEMIX_CACHE_INT8))
        return TILEMIX_ERR_UNSUPPORTED;
    int shift = 4;
    while (shift < 8 && (1 << shift) != p->page_size) ++shift;
    if ((1 << shift) != p->page_size) return TILEMIX_ERR_UNSUPPORTED;
    const int64_t capacity = static_cast<int64_t>(p->max_pages) << shift;
    if (capacity > (int64_t{1} << 30)) return TILEMIX_ERR_SHAPE;                         // positions are 32-bit
    if (p->table_stride != 0 && p->table_stride < p->max_pages && p->batch > 1) return TILEMIX_ERR_SHAPE;
    const bool int8 = p->cache_type == TILEMIX_CACHE_INT8;
    c->B = p->batch; c->Hk = p->heads_kv; c->d = p->head_dim; c->page_shift = shift;
    c->n_pages = p->n_pages; c->max_pages = p->max_pages; c->capacity = static_cast<int>(capacity);
    c->table_stride = p->table_stride != 0 && p->batch > 1 ? p->table_stride : p->max_pages;
    const int64_t size[3] = {p->n_pages, p->heads_kv, p->page_size};
    const int64_t dense[3] = {static_cast<int64_t>(p->heads_kv) * p->page_size * p->head_dim,
                              static_cast<int64_t>(p->page_size) * p->head_dim, p->head_dim};
    int rc;
    if ((rc = checked_strides(all_zero3(p->k_stride) ? dense : p->k_stride, size, 3, p->head_dim, int8 ? 1 : 2, c->ks))) return rc;
    if ((rc = checked_strides(all_zero3(p->v_stride) ? dense : p->v_stride, size, 3, p->head_dim, int8 ? 1 : 2, c->vs))) return rc;
    if (!p->k_pool || !p->v_pool || !p->block_table || !p->cache_len || (int8 && (!p->k_scale || !p->v_scale))) return TILEMIX_ERR_NULL;
    if (!aligned16(p->k_pool) || !aligned16(p->v_pool) || !aligned4(p->block_table) || !aligned4(p->cache_len) ||
        (int8 && (!aligned16(p->k_scale) || !aligned16(p->v_scale))))
        return TILEMIX_ERR_ALIGN;
    c->k_pool = static_cast<uint8_t*>(p->k_pool); c->v_pool = static_cast<uint8_t*>(p->v_pool);
    c->k_scale = int8 ? p->k_scale : nullptr; c->v_scale = int8 ? p->v_scale : nullptr;
    c->table = p->block_table; c->cache_len = p->cache_len;
    return TILEMIX_OK;
}

namespace {

// A lane takes kPieces pieces of eight values, 16 bytes of the 16-bit side, of one row; neighbouring lanes neighbouring pieces,
// so that every access of a warp is whole sectors.  One, two and four of them: read-back of 24 K tokens, 8 heads of 128, INT8
// 33.2 / 27.3 / 27.2 us, of 16 ragged BF16 contexts, heads of 64 79.9 / 72.3 / 76.5, 64 new tokens appended and read back
// 5.1 / 5.6 / 6.6; two rows of two pieces 28.4 / 72.6 / 7.8.  Blocks of 512 threads: 28.4, 72.3, 6.4.
constexpr int kMoveThreads = 128, kPieces = 2;

struct MoveParams {
    PagedCache c;
    int rows;                       // (token, head) pairs
    const int32_t* cu;              // packed tokens: first row of each sequence; nullptr: see the kernels
    const int32_t* start;           // gather: first token of each sequence, or nullptr
    int out_rows;                   // gather, dense: rows of a sequence
    uint8_t* k;                     // the 16-bit side
    uint8_t* v;
    int64_t k_st[3], v_st[3];       // bytes: (batch, head, token)
};

// Sequence that owns the packed row t: the number of sequences that end at or before it (B if none owns it).  A whole warp
// with one t: 32 ends at a time, whose loads do not wait for one another as those of a binary search would.
__device__ __forceinline__ int owner_of(const int32_t* __restrict__ cu, int B, int t) {
    const int lane = threadIdx.x & 31;
    int n = 0;
    for (int b = 0; b < B; b += 32) {
        const bool before = b + lane < B && cu[b + lane + 1] <= t;
        const int here = __popc(__ballot_sync(0xffffffffu, before));
        n += here;
        if (here < 32) break;
    }
    return n;
}

// The quantiser of one row, in the lanes that hold it: codes of this lane's values, and the scale.
// delta = RN(max|x| / 127), x8 = RN_int(RN(x / delta)).  The maximum is taken over the bit patterns, which order like the
// magnitudes and put infinities and NaN on top.  quant_scale's one-FMA form of the rounded quotient was derived for binary16;
// it holds for bfloat16 too: its ratios of 8-bit integers stay further from the half-integers than those of 11-bit ones, and
// the exact half-integers are the same two kinds.  It needs delta and 1 / delta to be normal numbers, hence the division for
// rows whose maximum is below 2^-100 (bfloat16 only).
__device__ __forceinline__ uint2 quant8_bf16(const uint4& x, const QuantScale& s, bool divide) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t code[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = act_to_float2(w[i], __nv_bfloat16());
        if (divide) {
            code[2 * i] = max(-127, min(127, __float2int_rn(__fdiv_rn(f.x, s.delta))));
            code[2 * i + 1] = max(-127, min(127, __float2int_rn(__fdiv_rn(f.y, s.delta))));
        } else {
            const float2 r2 = make_float2(s.r, s.r), magic = make_float2(12582912.f, 12582912.f);
            float2 y = __ffma2_rn(f, r2, magic);
            if (s.refine) {
                const float2 q = __fmul2_rn(f, r2);
                y = __fadd2_rn(__ffma2_rn(__ffma2_rn(make_float2(-s.delta, -s.delta), q, f), r2, q), magic);
            }
            code[2 * i] = __float_as_uint(y.x); code[2 * i + 1] = __float_as_uint(y.y);
        }
    }
    const uint32_t p0 = __byte_perm(code[0], code[1], 0x0040), p1 = __byte_perm(code[2], code[3], 0x0040);
    const uint32_t p2 = __byte_perm(code[4], code[5], 0x0040), p3 = __byte_perm(code[6], code[7], 0x0040);
    return make_uint2(__byte_perm(p0, p1, 0x5410), __byte_perm(p2, p3, 0x5410));
}
template <class T, int LANES, int P>
__device__ __forceinline__ float quantise_row(const uint4 (&x)[P], uint2 (&code)[P]) {
    constexpr bool BF16 = std::is_same<T, __nv_bfloat16>::value;
    uint32_t m2 = 0u;
#pragma unroll
    for (int i = 0; i < P; ++i)
        m2 = __vmaxu2(m2, __vmaxu2(__vmaxu2(habs2_bits(x[i].x), habs2_bits(x[i].y)), __vmaxu2(habs2_bits(x[i].z), habs2_bits(x[i].w))));
    uint32_t m = max(m2 & 0xffffu, m2 >> 16);
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    const bool odd = m >= (BF16 ? 0x7f80u : 0x7c00u);
    if (odd || m == 0u) {
#pragma unroll
        for (int i = 0; i < P; ++i) code[i] = make_uint2(0u, 0u);
        return odd ? __int_as_float(0x7fc00000) : 0.f;
    }
    const float amax = BF16 ? __uint_as_float(m << 16) : __half2float(__ushort_as_half(static_cast<unsigned short>(m)));
    const bool tiny = BF16 && amax < 7.888609052210118e-31f;
    QuantScale s;
    if (tiny) { s.delta = __fdiv_rn(amax, 127.f); s.r = 0.f; s.refine = false; }
    else s = quant_scale(amax);
#pragma unroll
    for (int i = 0; i < P; ++i) {
        if constexpr (BF16) code[i] = quant8_bf16(x[i], s, tiny);
        else code[i] = quant8(x[i], s);
    }
    return s.delta;
}

// The values that eight codes stand for: FP32 products, rounded.  A byte x + 128 under 0x4b0000 is the float 2^23 + x + 128.
// (The conversion instruction has a quarter of the rate.)
template <class T>
__device__ __forceinline__ uint4 dequantise8(const uint2& code, float delta) {
    const float2 off = make_float2(-8388736.f, -8388736.f), d2 = make_float2(delta, delta);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t biased = (i < 2 ? code.x : code.y) ^ 0x80808080u;
        const float2 f = make_float2(__uint_as_float(__byte_perm(biased, 0x4b000000u, i & 1 ? 0x7652 : 0x7650)),
                                     __uint_as_float(__byte_perm(biased, 0x4b000000u, i & 1 ? 0x7653 : 0x7651)));
        const float2 v = __fmul2_rn(__fadd2_rn(f, off), d2);
        w[i] = act_pack2(v.x, v.y, T());
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// New rows into the cache.  Row = (token, head), heads innermost, as the inputs lie.
template <class T, int D, bool INT8>
__global__ void __launch_bounds__(kMoveThreads)
paged_append_kernel(const MoveParams prm) {
    constexpr int P = kPieces, LANES = D / 8 / P, ROWS = kMoveThreads / LANES;
    const PagedCache& c = prm.c;
    const int row = blockIdx.x * ROWS + threadIdx.x / LANES, part = threadIdx.x % LANES;
    const int t = row / c.Hk, head = row - t * c.Hk;
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    int b = t, n_new = 1, i = 0;
    if (prm.cu != nullptr) {
        // the sequence of the warp's first row; a warp's rows are few tokens, so the others are at most a step or two on
        b = owner_of(prm.cu, c.B, __shfl_sync(0xffffffffu, t, 0));
        while (b < c.B && prm.cu[b + 1] <= t) ++b;
        if (b < c.B) {
            i = t - prm.cu[b];
            n_new = prm.cu[b + 1] - prm.cu[b];
        }
    }
    int page = -1, at = 0;
    uint4 k[P], v[P];
#pragma unroll
    for (int p = 0; p < P; ++p) k[p] = v[p] = make_uint4(0u, 0u, 0u, 0u);
    if (row < prm.rows && b < c.B && i >= 0) {
        const uint4* kf = reinterpret_cast<const uint4*>(prm.k + t * prm.k_st[2] + head * prm.k_st[1]) + part;
        const uint4* vf = reinterpret_cast<const uint4*>(prm.v + t * prm.v_st[2] + head * prm.v_st[1]) + part;
#pragma unroll
        for (int p = 0; p < P; ++p) { k[p] = __ldcs(kf + p * LANES); v[p] = __ldcs(vf + p * LANES); }
        const int64_t place = static_cast<int64_t>(c.cache_len[b]) - n_new + i;      // (not clamped: a token past the table has no place)
        const int pos = place >= 0 && place < c.capacity ? static_cast<int>(place) : -1;
        if (pos >= 0) page = paged_page(c, b, pos);
        at = pos & ((1 << c.page_shift) - 1);
    }
    const int64_t ko = page * c.ks[0] + head * c.ks[1] + at * c.ks[2], vo = page * c.vs[0] + head * c.vs[1] + at * c.vs[2];
    if constexpr (INT8) {
        uint2 k8[P], v8[P];
        const float dk = quantise_row<T, LANES>(k, k8), dv = quantise_row<T, LANES>(v, v8);
        if (page < 0) return;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            reinterpret_cast<uint2*>(c.k_pool + ko)[part + p * LANES] = k8[p];
            reinterpret_cast<uint2*>(c.v_pool + vo)[part + p * LANES] = v8[p];
        }
        if (part == 0) {
            const int64_t so = ((static_cast<int64_t>(page) * c.Hk + head) << c.page_shift) + at;
            c.k_scale[so] = dk;
            c.v_scale[so] = dv;
        }
    } else {
        if (page < 0) return;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            reinterpret_cast<uint4*>(c.k_pool + 2 * ko)[part + p * LANES] = k[p];
            reinterpret_cast<uint4*>(c.v_pool + 2 * vo)[part + p * LANES] = v[p];
        }
    }
}

// Rows of the cache out.  Packed outputs: row = (token, head), heads innermost; dense ones: (sequence, head, token).
// (The pools are read past L1: the kernel in front may have written them, and nothing is read twice.)
template <class T, int D, bool INT8>
__global__ void __launch_bounds__(kMoveThreads)
paged_gather_kernel(const MoveParams prm) {
    constexpr int P = kPieces, LANES = D / 8 / P, ROWS = kMoveThreads / LANES;
    const PagedCache& c = prm.c;
    const int row = blockIdx.x * ROWS + threadIdx.x / LANES, part = threadIdx.x % LANES;
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    int b, head, i, dst;            // dst: token of the output (packed), or i
    if (prm.cu != nullptr) {
        const int t = row / c.Hk;
        head = row - t * c.Hk;
        b = owner_of(prm.cu, c.B, __shfl_sync(0xffffffffu, t, 0));
        while (b < c.B && prm.cu[b + 1] <= t) ++b;
        i = b < c.B ? t - prm.cu[b] : -1;
        dst = t;
    } else {
        const int bh = row / prm.out_rows;
        i = dst = row - bh * prm.out_rows;
        b = bh / c.Hk;
        head = bh - b * c.Hk;
    }
    if (row >= prm.rows || b >= c.B || i < 0) return;
    const int len = paged_len(c, b), first = prm.start != nullptr ? max(prm.start[b], 0) : 0;
    if (i >= len - first) return;
    const int pos = first + i, page = paged_page(c, b, pos);
    uint4 k[P], v[P];
#pragma unroll
    for (int p = 0; p < P; ++p) k[p] = v[p] = make_uint4(0u, 0u, 0u, 0u);
    if (page >= 0) {
        const int at = pos & ((1 << c.page_shift) - 1);
        const int64_t ko = page * c.ks[0] + head * c.ks[1] + at * c.ks[2], vo = page * c.vs[0] + head * c.vs[1] + at * c.vs[2];
        if constexpr (INT8) {
            const int64_t so = ((static_cast<int64_t>(page) * c.Hk + head) << c.page_shift) + at;
            uint2 k8[P], v8[P];
#pragma unroll
            for (int p = 0; p < P; ++p) {
                k8[p] = __ldcg(reinterpret_cast<const uint2*>(c.k_pool + ko) + part + p * LANES);
                v8[p] = __ldcg(reinterpret_cast<const uint2*>(c.v_pool + vo) + part + p * LANES);
            }
            const float dk = __ldcg(c.k_scale + so), dv = __ldcg(c.v_scale + so);
#pragma unroll
            for (int p = 0; p < P; ++p) { k[p] = dequantise8<T>(k8[p], dk); v[p] = dequantise8<T>(v8[p], dv); }
        } else {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                k[p] = __ldcg(reinterpret_cast<const uint4*>(c.k_pool + 2 * ko) + part + p * LANES);
                v[p] = __ldcg(reinterpret_cast<const uint4*>(c.v_pool + 2 * vo) + part + p * LANES);
            }
        }
    }
    const int64_t batch = prm.cu != nullptr ? 0 : b;
    uint4* kt = reinterpret_cast<uint4*>(prm.k + batch * prm.k_st[0] + head * prm.k_st[1] + dst * prm.k_st[2]) + part;
    uint4* vt = reinterpret_cast<uint4*>(prm.v + batch * prm.v_st[0] + head * prm.v_st[1] + dst * prm.v_st[2]) + part;
#pragma unroll
    for (int p = 0; p < P; ++p) { __stcs(kt + p * LANES, k[p]); __stcs(vt + p * LANES, v[p]); }
}

// (a 16-bit cache is copied, whatever its type; programmatic dependent launch: the launch overlaps the kernel in front, whose
// end both kernels wait for)
template <bool APPEND, class T, int D>
int launch_move(bool int8, const MoveParams& prm, cudaStream_t stream) {
    void (*kernel)(const MoveParams);
    if constexpr (APPEND) kernel = int8 ? paged_append_kernel<T, D, true> : paged_append_kernel<__half, D, false>;
    else kernel = int8 ? paged_gather_kernel<T, D, true> : paged_gather_kernel<__half, D, false>;
    constexpr int kRows = kMoveThreads / (D / 8 / kPieces);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(ceil_div(prm.rows, kRows))); cfg.blockDim = dim3(kMoveThreads); cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, prm);
    g_launch_count.fetch_add(1);
    return static_cast<int>(e);
}
template <bool APPEND>
int launch_move(const tilemix_paged_t* p, const MoveParams& prm, cudaStream_t stream) {
    const bool int8 = p->cache_type == TILEMIX_CACHE_INT8;
    if (p->act_type == TILEMIX_TYPE_FP16)
        return p->head_dim == 128 ? launch_move<APPEND, __half, 128>(int8, prm, stream) : launch_move<APPEND, __half, 64>(int8, prm, stream);
    return p->head_dim == 128 ? launch_move<APPEND, __nv_bfloat16, 128>(int8, prm, stream) : launch_move<APPEND, __nv_bfloat16, 64>(int8, prm, stream);
}

// Byte strides (batch, head, token) of the 16-bit side.  Only outputs must not overlap themselves.
int side_strides(const int64_t* in, const int64_t dense[3], const int64_t size[3], int d, bool output, int64_t out[3]) {
    int64_t st[3];
    const int64_t* s = in != nullptr ? in : dense;
    if (output) {
        const int rc = checked_strides(s, size, 3, d, 2, st);
        if (rc) return rc;
    } else {
        for (int i = 0; i < 3; ++i) {
            st[i] = size[i] == 1 ? 0 : s[i];
            if (st[i] < 0 || st[i] > (int64_t{1} << 40)) return TILEMIX_ERR_SHAPE;
            if (st[i] * 2 % 16 != 0) return TILEMIX_ERR_ALIGN;
        }
    }
    for (int i = 0; i < 3; ++i) out[i] = 2 * st[i];
    return TILEMIX_OK;
}

}  // namespace
}  // namespace tilemix

using namespace tilemix;

extern "C" {

int tilemix_paged_append(const tilemix_paged_t* p, int32_t n_tokens, const void* k_new, const int64_t* k_new_stride,
                         const void* v_new, const int64_t* v_new_stride, const int32_t* cu_new, void* stream) {
    MoveParams prm{};
    int rc = resolve_paged(p, &prm.c);
    if (rc) return rc;
    if (n_tokens < 0 || (cu_new == nullptr && n_tokens != p->batch)) return TILEMIX_ERR_SHAPE;
    if (static_cast<int64_t>(n_tokens) * p->heads_kv > (int64_t{1} << 30)) return TILEMIX_ERR_SHAPE;
    if (n_tokens == 0) return TILEMIX_OK;
    if (!k_new || !v_new) return TILEMIX_ERR_NULL;
    if (!aligned16(k_new) || !aligned16(v_new) || !aligned4(cu_new)) return TILEMIX_ERR_ALIGN;
    const int64_t size[3] = {1, p->heads_kv, n_tokens};
    const int64_t dense[3] = {0, p->head_dim, static_cast<int64_t>(p->heads_kv) * p->head_dim};
    int64_t ks[3] = {0, 0, 0}, vs[3] = {0, 0, 0};
    if (k_new_stride) { ks[1] = k_new_stride[1]; ks[2] = k_new_stride[0]; }
    if (v_new_stride) { vs[1] = v_new_stride[1]; vs[2] = v_new_stride[0]; }
    if ((rc = side_strides(k_new_stride ? ks : nullptr, dense, size, p->head_dim, false, prm.k_st))) return rc;
    if ((rc = side_strides(v_new_stride ? vs : nullptr, dense, size, p->head_dim, false, prm.v_st))) return rc;
    prm.rows = n_tokens * p->heads_kv;
    prm.cu = cu_new;
    prm.k = static_cast<uint8_t*>(const_cast<void*>(k_new));
    prm.v = static_cast<uint8_t*>(const_cast<void*>(v_new));
    return launch_move<true>(p, prm, static_cast<cudaStream_t>(stream));
}

int tilemix_paged_gather(const tilemix_paged_t* p, const int32_t* start, const int32_t* cu_out, int32_t out_rows, void* k_out,
                         const int64_t* k_out_stride, void* v_out, const int64_t* v_out_stride, void* stream) {
    MoveParams prm{};
    int rc = resolve_paged(p, &prm.c);
    if (rc) return rc;
    if (out_rows < 0) return TILEMIX_ERR_SHAPE;
    const int64_t tokens = cu_out != nullptr ? out_rows : static_cast<int64_t>(out_rows) * p->batch;
    if (tokens > (int64_t{1} << 30) || tokens * p->heads_kv > (int64_t{1} << 30)) return TILEMIX_ERR_SHAPE;
    if (out_rows == 0) return TILEMIX_OK;
    if (!k_out || !v_out) return TILEMIX_ERR_NULL;
    if (!aligned16(k_out) || !aligned16(v_out) || !aligned4(cu_out) || !aligned4(start)) return TILEMIX_ERR_ALIGN;
    const int64_t rows = out_rows, d = p->head_dim, h = p->heads_kv;
    const int64_t size[3] = {cu_out != nullptr ? 1 : p->batch, h, rows};
    const int64_t dense[3] = {h * rows * d, cu_out != nullptr ? d : rows * d, cu_out != nullptr ? h * d : d};
    if ((rc = side_strides(k_out_stride, dense, size, p->head_dim, true, prm.k_st))) return rc;
    if ((rc = side_strides(v_out_stride, dense, size, p->head_dim, true, prm.v_st))) return rc;
    prm.rows = static_cast<int>(tokens * h);
    prm.cu = cu_out;
    prm.start = start;
    prm.out_rows = out_rows;
    prm.k = static_cast<uint8_t*>(k_out);
    prm.v = static_cast<uint8_t*>(v_out);
    return launch_move<false>(p, prm, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
