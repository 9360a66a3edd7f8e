// Decode step over a paged key/value cache: one query token per sequence.
//
// HBM-bound: a cached (token, KV head) is 4 d bytes (16-bit cache) or 2 (d + 4) (INT8 codes and scales), read once, and serves
// the R = H_q / H_k query heads of its group with 4 R d multiply-adds, far below the tensor cores' rate for R <= 16.  Hence
// warp-level MMAs: their operands pass through registers, where INT8 codes become FP16 and where a key past the end is masked,
// at the cost of ~17 instructions a token (INT8, d = 128) where HBM leaves an SM ~43 issue slots a token.
//
// Layout of the work.  A warp owns a ring of three stages, starts its own copies and takes CHUNKS of 16 to 64 keys, which one
// TMA box a page brings in, swizzled; no warp waits for another but at the end of a row.  Four or eight warps are a CTA, two
// CTAs share an SM: 192 KB are on the way.  (A warp of its own for the copies of all could not start them fast
// enough: four small ones a chunk, 8 x 32K keys of 128 in INT8 129 us, 101 so.)  Neighbouring chunks, one for each warp, are a UNIT; the units of all
// (sequence, KV head) rows, one row behind the other, are dealt out to the CTAs in equal runs, so that a batch of unequal
// lengths keeps every SM busy to the end.  A CTA finds its run from the lengths, which only the device knows.  Rows inside
// its run it finishes itself; of a row that it shares with its neighbours it leaves a partial result (m, z, O) to the joining
// kernel.  The copies run on across rows.
//
// Products.  S^T = K Q^T with the KEYS as the 16 rows of the MMA and eight query heads as its columns, then O^T = V^T P^T with
// the head dimension as the rows: nothing of a 16-row operand is wasted on absent query heads, and O^T takes D / 32 * 8
// registers for eight heads.  The score fragment (rows keys, columns queries) becomes the right operand of the second product by
// transposing its 8x8 blocks (movmatrix).
//
// INT8 codes become FP16 exactly: byte x + 128 under the exponent byte 0x64 is 1024 + (x + 128), less 1152.  The contraction
// index may be permuted as long as both operands agree, so a lane takes whole 16-byte pieces of a row; the keys of a block are
// permuted (key_of_row) so that those loads, of the keys and of the values, touch every bank once.
#include <math.h>

#include <type_traits>

#include "common.cuh"
#include "paged.cuh"
#include "ptx_sm100.cuh"
#include "softmax_tile.cuh"

namespace tilemix {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kStages = 3, kRingBytes = 96 * 1024;
constexpr int kCtasPerSm = 2, kSms = 148;

struct PagedDecodeParams {
    PagedCache c;
    int Hq, R;                      // query heads, query heads per KV head
    int groups, HG;                 // groups of up to 8 NB query heads per KV head; rows of a sequence (Hk * groups)
    float scale_log2;
    const uint8_t* q;
    uint8_t* out;
    int64_t qs[2], os[2];           // bytes: (batch, head)
    float* lse;
    int4* join;                     // [CTAs]: what the joining kernel has to do, see there
    float4* part_o;                 // [2 CTAs][D / 16][NB][32 lanes]: accumulator fragments
    float2* part_mz;                // [2 CTAs][8 NB]: maximum (log2 domain) and sum
    unsigned long long wait_limit_ns;
    int drop_chunk;                 // testing aid: every warp leaves out the copies of its chunk of this number (-1: none)
};

template <class T, int D, bool INT8, int NB>
struct Cfg {
    static constexpr int kElt = INT8 ? 1 : 2;
    // Warps at the products.  The INT8 form is bound by issue slots and latencies, not by bytes, unless many warps share them
    // (8 x 32K keys, d = 128: four a CTA 135 us, eight 101); sixteen query heads need the registers of four.
    static constexpr int W = INT8 && NB == 1 ? 8 : 4;
    static constexpr int kThreads = 32 * W;
    static constexpr int kStageBytes = kRingBytes / (W * kStages);
    static constexpr int CH = kStageBytes / (2 * D * kElt);         // keys of a chunk
    static constexpr int kChShift = CH == 16 ? 4 : CH == 32 ? 5 : 6;
    static_assert(CH == 1 << kChShift, "chunks are whole boxes");
    static constexpr int MB = CH / 16;                              // blocks of 16 keys
    static constexpr int kUnit = CH * W;
    static constexpr int kVOff = CH * D * kElt;                     // values behind the keys of a stage
    static constexpr int kBoxCols = INT8 ? 1 : D / 64;              // boxes side by side in a row of 16-bit values
    static constexpr int kScaleBytes = INT8 ? W * kStages * CH * 8 : 0;
    static constexpr int kSmemBytes = kRingBytes + kScaleBytes + 1024;
    static constexpr int kFrag = (D / 16) * NB * 32;                // float4 fragments of a row's O
    // The probabilities are carried 2^14 times as large in FP16, so that what the rounding loses is below 2^-28 of the
    // largest instead of 2^-14.  bfloat16 has FP32's exponents.  The running maximum is moved only when a score exceeds it by
    // more than kLine (log2 units): 2^(14 + 1.5) fits FP16, and a chunk whose maximum need not be known costs no shuffles.
    static constexpr bool kHalfP = INT8 || std::is_same<T, __half>::value;
    static constexpr float kOff = kHalfP ? 14.f : 0.f;
    static constexpr float kUnOff = kHalfP ? 6.103515625e-5f : 1.f;
    static constexpr float kLine = kHalfP ? 1.5f : 8.f;
    static_assert(kFrag * 16 <= kStageBytes, "a row's O of one warp fits the stage that the warp has just read");
};
constexpr float kNoMax = -1e38f;        // running maximum before the first key (finite: nothing is subtracted from an infinity)

// ---------------------------------------------------------------------------------------------------- warp-level pieces
template <bool BF16>
__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (BF16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
template <bool TRANS>
__device__ __forceinline__ void ldmatrix_x4(uint32_t (&r)[4], uint32_t addr) {
    if constexpr (TRANS)
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
    else
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t addr) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr) : "memory");
    return v;
}
// Bytes 0, 1 (HI = false) or 2, 3 of a word of codes + 128 as an FP16 pair.
template <bool HI>
__device__ __forceinline__ uint32_t codes_to_half2(uint32_t biased) {
    const uint32_t m = __byte_perm(biased, 0x64646464u, HI ? 0x4342u : 0x4140u);
    const __half2 h = __hsub2(*reinterpret_cast<const __half2*>(&m), __floats2half2_rn(1152.f, 1152.f));
    return *reinterpret_cast<const uint32_t*>(&h);
}

// Key of a block of eight that row r of an INT8 fragment holds.
template <int D>
__device__ __forceinline__ constexpr int key_of_row(int r) {
    return D == 128 ? ((r & 1) ? r ^ 4 : r) : r ^ ((r >> 1) & 1);
}
// Byte offset of the 16-byte piece `piece` of a row of codes, as the TMA swizzle places it (128- or 64-byte rows).
template <int D>
__device__ __forceinline__ uint32_t code_piece(int row, int piece) {
    return D == 128 ? row * 128 + ((piece ^ (row & 7)) << 4) : row * 64 + ((piece ^ ((row >> 1) & 3)) << 4);
}
// ... of a row of 16-bit values: pieces 0-7 and 8-15 are boxes of their own, CH rows of 128 bytes.
template <int CH>
__device__ __forceinline__ uint32_t value_piece(int row, int piece) {
    return (piece >> 3) * (CH * 128) + row * 128 + (((piece & 7) ^ (row & 7)) << 4);
}

// ---------------------------------------------------------------------------------------------------- the work list
// Place in the list of units: rows (b, h) of n_units units, h = KV head * groups + group of query heads.
struct Cursor {
    int b, h, unit, n_units, len, left;      // left: units from here to the end of the CTA's run
};
__device__ __forceinline__ void next_row(Cursor& c, const PagedDecodeParams& prm, int unit_keys) {
    c.unit = 0;
    if (++c.h == prm.HG) {
        c.h = 0;
        do {
            if (++c.b >= prm.c.B) {          // (only if a length changed meanwhile)
                c.left = 0;
                return;
            }
            c.len = paged_len(prm.c, c.b);
            c.n_units = (c.len + unit_keys - 1) / unit_keys;
        } while (c.n_units == 0);
    }
}
__device__ __forceinline__ void next_unit(Cursor& c, const PagedDecodeParams& prm, int unit_keys) {
    --c.left;
    if (++c.unit == c.n_units && c.left > 0) next_row(c, prm, unit_keys);
}

// The run of CTA `cta` of `ctas`: [cta U / n, (cta + 1) U / n) of the U units, n = min(ctas, U).  Whole warps, every one alike.
__device__ __forceinline__ Cursor find_run(const PagedDecodeParams& prm, int unit_keys, int cta, int ctas, int* total, int* used) {
    const int lane = threadIdx.x & 31, B = prm.c.B;
    auto units_of = [&](int b) { return b < B ? (paged_len(prm.c, b) + unit_keys - 1) / unit_keys : 0; };
    int sum = 0;
    for (int b = lane; b < B; b += 32) sum += units_of(b);
    const int U = __reduce_add_sync(0xffffffffu, sum) * prm.HG, n = min(ctas, U);
    *total = U; *used = n;
    Cursor c{};
    if (cta >= n) return c;
    const int first = static_cast<int>(static_cast<int64_t>(cta) * U / n);
    c.left = static_cast<int>(static_cast<int64_t>(cta + 1) * U / n) - first;
    int before = 0;                          // units of the sequences before the 32 in hand
    for (int b0 = 0; b0 < B; b0 += 32) {
        const int mine = units_of(b0 + lane) * prm.HG;
        int upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += x;
        }
        const uint32_t past = __ballot_sync(0xffffffffu, before + upto > first);
        if (past != 0u) {
            const int l = __ffs(past) - 1;
            c.b = b0 + l;
            c.n_units = __shfl_sync(0xffffffffu, mine, l) / prm.HG;
            const int at = first - before - (__shfl_sync(0xffffffffu, upto, l) - c.n_units * prm.HG);
            c.h = at / c.n_units;
            c.unit = at - c.h * c.n_units;
            c.len = paged_len(prm.c, c.b);
            return c;
        }
        before += __shfl_sync(0xffffffffu, upto, 31);
    }
    c.left = 0;
    return c;
}

// ---------------------------------------------------------------------------------------------------- results
// Fragment (md, lane) of O^T: x, y = row d0 of query columns 2 t, 2 t + 1; z, w = row d1; (d0, d1) = (16 md + g, + 8), of an
// INT8 cache (D / 8 g + 2 md, + 1).
__device__ __forceinline__ uint8_t* out_row(const PagedDecodeParams& prm, int b, int h, int width, int n) {
    const int hk = h / prm.groups, first = (h - hk * prm.groups) * width;
    return first + n < prm.R ? prm.out + b * prm.os[0] + (static_cast<int64_t>(hk) * prm.R + first + n) * prm.os[1] : nullptr;
}

// Writes the normalised fragment of query columns 2 t, 2 t + 1 of block nb, and the row's lse with fragment 0.
template <class T, int D, bool INT8, int NB>
__device__ __forceinline__ void write_out(const PagedDecodeParams& prm, int b, int h, int md, int nb, int lane, const float4& o,
                                          const float (&m)[2], const float (&z)[2]) {
    const int g = lane >> 2, t = lane & 3;
    const float v[2][2] = {{o.x, o.z}, {o.y, o.w}};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int n = 8 * nb + 2 * t + i;
        uint8_t* dst = out_row(prm, b, h, 8 * NB, n);
        if (dst == nullptr) continue;
        const bool empty = z[i] == 0.f;
        const uint32_t two = act_pack2(empty ? 0.f : v[i][0] / z[i], empty ? 0.f : v[i][1] / z[i], T());
        if constexpr (INT8) {
            reinterpret_cast<uint32_t*>(dst)[(D / 16) * g + md] = two;
        } else {
            reinterpret_cast<uint16_t*>(dst)[16 * md + g] = static_cast<uint16_t>(two);
            reinterpret_cast<uint16_t*>(dst)[16 * md + g + 8] = static_cast<uint16_t>(two >> 16);
        }
        if (md == 0 && g == 0 && prm.lse != nullptr) {
            const int hk = h / prm.groups;
            prm.lse[static_cast<int64_t>(b) * prm.Hq + hk * prm.R + (h - hk * prm.groups) * 8 * NB + n] =
                empty ? -INFINITY : (m[i] + log2f(z[i])) * kLn2;
        }
    }
}

// ---------------------------------------------------------------------------------------------------- the step
template <class T, int D, bool INT8, int NB>
__global__ void __launch_bounds__(Cfg<T, D, INT8, NB>::kThreads, kCtasPerSm)
paged_decode_kernel(const PagedDecodeParams prm, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
    using C = Cfg<T, D, INT8, NB>;
    constexpr int CH = C::CH, MB = C::MB, W = C::W, kStageBytes = C::kStageBytes;
    constexpr bool BF16 = !C::kHalfP;
    extern __shared__ uint8_t smem[];
    __shared__ __align__(8) uint64_t full_bar[W][kStages];
    __shared__ uint32_t hole_s[W][kStages];                          // bit 4 i: the 16 keys i of the chunk lie in a hole
    __shared__ float m_s[W][8 * NB], z_s[W][8 * NB], v_ref_s[W];
    __shared__ int held_s[W];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    uint8_t* ring = smem + ((1024u - (ptx::smem_u32(smem) & 1023u)) & 1023u);      // (the swizzle's pattern repeats every 1 KB)
    const PagedCache& c = prm.c;

    if (lane == 0) {
        // (arrivals: the lane that announces the bytes of the boxes, and every lane with its part of the scales)
        for (int i = 0; i < kStages; ++i) ptx::mbar_init(ptx::smem_u32(&full_bar[warp][i]), INT8 ? 33 : 1);
        ptx::fence_mbar_init();
        ptx::tma_prefetch_desc(&k_map);
        ptx::tma_prefetch_desc(&v_map);
    }
    __syncwarp();
    ptx::griddep_wait();                     // the cache, the lengths and the queries may be the work of the kernel before
    ptx::griddep_launch_dependents();

    int total, used;
    const int cta = blockIdx.x;
    Cursor cc = find_run(prm, C::kUnit, cta, gridDim.x, &total, &used);

    // ---- copies.  `prepare` finds this warp's next chunk and looks its pages up, every lane that of four of its keys;
    // `fire` starts its copies into the stage behind the one filled last.
    const int box_shift = min(c.page_shift, C::kChShift), page_mask = (1 << c.page_shift) - 1;
    const uint32_t ring_u32 = ptx::smem_u32(ring) + warp * (kStages * kStageBytes);
    const uint32_t scale_u32 = ptx::smem_u32(ring) + kRingBytes + warp * (kStages * CH * 8);
    constexpr int kQuads = CH / 4;
    const int quad = 4 * (lane & (kQuads - 1));
    Cursor ic = cc;
    int issued = 0, fill = 0, next_start = 0, next_len = 0, next_hk = 0, next_page = -1;
    bool next_there = false;
    auto prepare = [&]() {
        next_there = false;
        while (ic.left > 0) {
            next_start = (ic.unit * W + warp) * CH;
            if (next_start < ic.len) {
                next_there = true;
                break;
            }
            next_unit(ic, prm, C::kUnit);
        }
        if (!next_there) return;
        next_len = ic.len;
        next_hk = prm.groups == 1 ? ic.h : ic.h / prm.groups;
        next_page = next_start + quad < next_len ? paged_page(c, ic.b, next_start + quad) : -1;
        next_unit(ic, prm, C::kUnit);
    };
    auto fire = [&]() {
        if (!next_there) return;
        const uint32_t bar = ptx::smem_u32(&full_bar[warp][fill]);
        const uint32_t holes = __ballot_sync(0xffffffffu, next_page < 0 && next_start + quad < next_len);
        if (lane == 0) hole_s[warp][fill] = holes;
        if (issued != prm.drop_chunk) {
            const int boxes = (min(CH, next_len - next_start) + (1 << box_shift) - 1) >> box_shift, row = next_start & page_mask;
            if (lane == 0) ptx::mbar_arrive_expect_tx(bar, (boxes << box_shift) * (2 * D * C::kElt));
            const uint32_t dst = ring_u32 + fill * kStageBytes;
#pragma unroll
            for (int i = 0; i < CH / 16; ++i) {
                if (i >= boxes) break;
                // (a hole's box lies outside the map: zeros arrive, nothing is read; more boxes than one: whole pages)
                const int page = __shfl_sync(0xffffffffu, next_page, i << (box_shift - 2));
                const uint32_t to = dst + (i << box_shift) * (INT8 ? D : 128);
#pragma unroll
                for (int col = 0; col < C::kBoxCols; ++col) {
                    ptx::tma_load_4d_elect(to + col * (CH * 128), &k_map, bar, col * 64, i == 0 ? row : 0, next_hk, page);
                    ptx::tma_load_4d_elect(to + col * (CH * 128) + C::kVOff, &v_map, bar, col * 64, i == 0 ? row : 0, next_hk, page);
                }
            }
            if constexpr (INT8) {
                if (lane < 2 * kQuads) {
                    const float* from = lane < kQuads ? c.k_scale : c.v_scale;
                    const int64_t at = ((static_cast<int64_t>(next_page) * c.Hk + next_hk) << c.page_shift) + ((next_start + quad) & page_mask);
                    ptx::cp_async_16(scale_u32 + fill * (CH * 8) + lane * 16, from + (next_page >= 0 ? at : 0), next_page >= 0);
                }
                ptx::cp_async_arrive(bar);
            }
        }
        ++issued;
        if (++fill == kStages) fill = 0;
        prepare();
    };
    // Bounded wait for the chunk in `stage`.
    auto landed = [&](int stage, uint32_t phase) -> bool {
        const uint32_t bar = ptx::smem_u32(&full_bar[warp][stage]);
        if (ptx::mbar_try_wait(bar, phase)) return true;
        const uint64_t begin = ptx::globaltimer_ns();
        uint32_t spins = 0;
        while (!ptx::mbar_try_wait(bar, phase))
            if ((++spins & 63u) == 0u && ptx::globaltimer_ns() - begin > prm.wait_limit_ns) return false;
        return true;
    };
    prepare();
#pragma unroll 1
    for (int i = 0; i < kStages; ++i) fire();

    // ==================================================================== products
    // What the joining kernel finds for this CTA: the first CTA that begins inside a row joins that row.
    if (tid == 0) {
        int4 job = make_int4(-1, 0, 0, 0);
        if (cc.left > 0 && cc.unit > 0) {
            const int first = static_cast<int>(static_cast<int64_t>(cta) * total / used);
            const int before = static_cast<int>(static_cast<int64_t>(cta - 1) * total / used);
            if (before <= first - cc.unit) {
                const int64_t end = static_cast<int64_t>(first) - cc.unit + cc.n_units;         // of the row
                const int last = static_cast<int>((end * used - 1) / total);                    // CTA with the row's last unit
                // sequence, row, the slot of the part in front, parts of this CTA and those behind it
                job = make_int4(cc.b, cc.h, 2 * (cta - 1) + (before == first - cc.unit ? 0 : 1), last - cta + 1);
            }
        }
        prm.join[cta] = job;
    }
    // sequences without a key
    for (int b = cta; b < c.B; b += gridDim.x) {
        if (paged_len(c, b) > 0) continue;
        for (int i = tid; i < prm.Hq * (D / 8); i += 32 * W) {
            const int hq = i / (D / 8);
            reinterpret_cast<uint4*>(prm.out + b * prm.os[0] + hq * prm.os[1])[i - hq * (D / 8)] = make_uint4(0u, 0u, 0u, 0u);
        }
        if (prm.lse != nullptr)
            for (int hq = tid; hq < prm.Hq; hq += 32 * W) prm.lse[static_cast<int64_t>(b) * prm.Hq + hq] = -INFINITY;
    }

    const float* scale_ring = reinterpret_cast<const float*>(ring + kRingBytes) + warp * (kStages * CH * 2);
    int stage = 0, taken = 0;
    uint32_t phase = 0u;
    bool failed = false, first_segment = true;      // failed: a wait ran out; no more copies, the rows from here on are NaN
#pragma unroll 1
    while (cc.left > 0) {
        // ------------------------------------------------ a row, or this CTA's part of it
        const int u_end = min(cc.n_units, cc.unit + cc.left);
        const int hk = cc.h / prm.groups, q_first = (cc.h - hk * prm.groups) * 8 * NB;

        // ---- query fragments: the right operand (columns = heads g of the block), and what a score is multiplied by
        uint32_t qf[NB][D / 16][2];
        float q_mul[NB][2];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const bool on = q_first + 8 * nb + g < prm.R;
            const uint8_t* row = prm.q + cc.b * prm.qs[0] + (static_cast<int64_t>(hk) * prm.R + q_first + 8 * nb + g) * prm.qs[1];
            q_mul[nb][0] = q_mul[nb][1] = prm.scale_log2;
            if constexpr (INT8) {
                // fragment 4 j + w holds features 16 (t + 4 j) + 4 w .. + 3, as the codes come
#pragma unroll
                for (int j = 0; j < D / 64; ++j)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        uint4 x = make_uint4(0u, 0u, 0u, 0u);
                        if (on) x = __ldcg(reinterpret_cast<const uint4*>(row + 32 * (t + 4 * j)) + i);
                        qf[nb][4 * j + 2 * i][0] = x.x; qf[nb][4 * j + 2 * i][1] = x.y;
                        qf[nb][4 * j + 2 * i + 1][0] = x.z; qf[nb][4 * j + 2 * i + 1][1] = x.w;
                    }
                if constexpr (std::is_same<T, __nv_bfloat16>::value) {
                    // bfloat16 queries as FP16: multiplied by the power of two that brings the row's largest value to
                    // [2^13, 2^14); eight mantissa bits fit, and what becomes subnormal is below 2^-27 of the largest
                    uint32_t top = 0u;
#pragma unroll
                    for (int i = 0; i < D / 16; ++i)
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const uint32_t a = qf[nb][i][k] & 0x7fff7fffu;
                            top = max(top, max(a & 0xffffu, a >> 16));
                        }
                    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
                    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
                    const uint32_t e = top == 0u ? 140u : max(top >> 7, 14u);
                    const float up = __uint_as_float((267u - e) << 23), down = __uint_as_float((e - 13u) << 23);
#pragma unroll
                    for (int i = 0; i < D / 16; ++i)
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const float2 f = act_to_float2(qf[nb][i][k], __nv_bfloat16());
                            qf[nb][i][k] = act_pack2(f.x * up, f.y * up, __half());
                        }
                    q_mul[nb][0] *= __shfl_sync(0xffffffffu, down, 8 * t);
                    q_mul[nb][1] *= __shfl_sync(0xffffffffu, down, 8 * t + 4);
                }
            } else {
#pragma unroll
                for (int i = 0; i < D / 16; ++i)
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        qf[nb][i][k] = on ? __ldcg(reinterpret_cast<const uint32_t*>(row + 32 * i + 16 * k) + t) : 0u;
            }
        }

        float m_run[NB][2], z[NB][2], acc[D / 16][NB][4];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            m_run[nb][0] = m_run[nb][1] = kNoMax;
            z[nb][0] = z[nb][1] = 0.f;
#pragma unroll
            for (int md = 0; md < D / 16; ++md) acc[md][nb][0] = acc[md][nb][1] = acc[md][nb][2] = acc[md][nb][3] = 0.f;
        }
        // INT8: the scale of a value is folded into its probability relative to v_ref, a power of two at or above every
        // scale so far; O~ is in units of it.
        float v_ref = 7.888609052210118e-31f;                 // 2^-100
        const int end = min(cc.len, u_end * C::kUnit);        // keys of this segment
        bool any = false;
        int held = 0;

#pragma unroll 1
        for (int start = (cc.unit * W + warp) * CH; start < end; start += C::kUnit) {
            if (!failed && !landed(stage, phase)) failed = true;
            if (failed) break;
            any = true;
            const uint32_t kst = ring_u32 + stage * kStageBytes, vst = kst + C::kVOff;
            const int live = min(CH, cc.len - start);         // keys of the chunk
            const uint32_t holes = hole_s[warp][stage];
            const bool partial = live < CH || holes != 0u;
            // ---- S^T: sc[mb][nb] = (row g, columns 2 t, 2 t + 1), (row g + 8, the same)
            float sc[MB][NB][4], v_mul[MB][2];
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) sc[mb][nb][0] = sc[mb][nb][1] = sc[mb][nb][2] = sc[mb][nb][3] = 0.f;
                if constexpr (INT8) {
                    const int r0 = 16 * mb + key_of_row<D>(g);
#pragma unroll
                    for (int j = 0; j < D / 64; ++j) {
                        const uint4 xa = lds128(kst + code_piece<D>(r0, t + 4 * j)), xb = lds128(kst + code_piece<D>(r0 + 8, t + 4 * j));
                        const uint32_t wa[4] = {xa.x, xa.y, xa.z, xa.w}, wb[4] = {xb.x, xb.y, xb.z, xb.w};
#pragma unroll
                        for (int w = 0; w < 4; ++w) {
                            const uint32_t ua = wa[w] ^ 0x80808080u, ub = wb[w] ^ 0x80808080u;
                            const uint32_t a0 = codes_to_half2<false>(ua), a2 = codes_to_half2<true>(ua);
                            const uint32_t a1 = codes_to_half2<false>(ub), a3 = codes_to_half2<true>(ub);
#pragma unroll
                            for (int nb = 0; nb < NB; ++nb)
                                mma_16816<false>(sc[mb][nb], a0, a1, a2, a3, qf[nb][4 * j + w][0], qf[nb][4 * j + w][1]);
                        }
                    }
                    const float* sk = scale_ring + stage * (CH * 2) + r0;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float dk = sk[8 * i];
                        v_mul[mb][i] = sk[CH + 8 * i];
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb) { sc[mb][nb][2 * i] *= dk; sc[mb][nb][2 * i + 1] *= dk; }
                    }
                } else {
                    const int row = 16 * mb + (lane & 15), piece = lane >> 4;
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) {
                        uint32_t a[4];
                        ldmatrix_x4<false>(a, kst + value_piece<CH>(row, 2 * i + piece));
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb) mma_16816<BF16>(sc[mb][nb], a[0], a[1], a[2], a[3], qf[nb][i][0], qf[nb][i][1]);
                    }
                }
            }
            // ---- keys past the end and in holes do not exist, whatever lies in their rows
            if (partial) {
#pragma unroll
                for (int mb = 0; mb < MB; ++mb) {
                    const bool hole = (holes >> (4 * mb)) & 1u;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int key = 16 * mb + 8 * i + (INT8 ? key_of_row<D>(g) : g);
                        if (key < live && !hole) continue;
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb) sc[mb][nb][2 * i] = sc[mb][nb][2 * i + 1] = -INFINITY;
                        v_mul[mb][i] = 0.f;
                    }
                }
                if constexpr (!INT8) {
                    // (0 times a NaN is one)
                    for (int i = lane; i < (CH - live) * (D / 8); i += 32) {
                        const int row = live + i / (D / 8), piece = i & (D / 8 - 1);
                        asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(vst + value_piece<CH>(row, piece)), "r"(0u) : "memory");
                    }
                    ptx::fence_proxy_async_smem();
                    __syncwarp();
                }
            }
            // ---- exponents, relative to the running maximum; it moves when one of them passes the line
            float top = -INFINITY;
            auto exponents = [&](float (&e)[MB][NB][4]) {
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                        for (int k = 0; k < 4; ++k) e[mb][nb][k] = fmaf(sc[mb][nb][k], q_mul[nb][k & 1], C::kOff - m_run[nb][k & 1]);
            };
            float e[MB][NB][4];
            exponents(e);
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) top = fmax3(fmax3(top, e[mb][nb][0], e[mb][nb][1]), e[mb][nb][2], e[mb][nb][3]);
            bool past = top > C::kOff + C::kLine;
            if constexpr (INT8) {
                float v_top = fmaxf(v_mul[0][0], v_mul[0][1]);
#pragma unroll
                for (int mb = 1; mb < MB; ++mb) v_top = fmax3(v_top, v_mul[mb][0], v_mul[mb][1]);
                past = past || v_top > v_ref;
            }
            if (__any_sync(0xffffffffu, past)) {
                float alpha[NB][2];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        float x = fmaxf(sc[0][nb][k], sc[0][nb][2 + k]);
#pragma unroll
                        for (int mb = 1; mb < MB; ++mb) x = fmax3(x, sc[mb][nb][k], sc[mb][nb][2 + k]);
                        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
                        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
                        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
                        const float m_new = fmaxf(m_run[nb][k], x * q_mul[nb][k]);
                        alpha[nb][k] = exp2f(m_run[nb][k] - m_new);
                        m_run[nb][k] = m_new;
                        z[nb][k] *= alpha[nb][k];
                    }
                if constexpr (INT8) {
                    uint32_t dv = 0u;
#pragma unroll
                    for (int mb = 0; mb < MB; ++mb) dv = max(dv, max(__float_as_uint(fabsf(v_mul[mb][0])), __float_as_uint(fabsf(v_mul[mb][1]))));
                    dv = __reduce_max_sync(0xffffffffu, dv);
                    const uint32_t want = (min(dv, 0x7e800000u) + 0x7fffffu) & 0x7f800000u, have = __float_as_uint(v_ref);
                    if (want > have) {          // (the same in the whole warp)
                        const float back = __uint_as_float(have) * __uint_as_float(0x7f000000u - want);
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb) { alpha[nb][0] *= back; alpha[nb][1] *= back; }
                        v_ref = __uint_as_float(want);
                    }
                }
#pragma unroll
                for (int md = 0; md < D / 16; ++md)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        acc[md][nb][0] *= alpha[nb][0]; acc[md][nb][1] *= alpha[nb][1];
                        acc[md][nb][2] *= alpha[nb][0]; acc[md][nb][3] *= alpha[nb][1];
                    }
                exponents(e);
            }
            const float inv = __uint_as_float(0x7f000000u - __float_as_uint(v_ref));
            // ---- probabilities, and O^T += V^T P^T block by block
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
                uint32_t p0[NB], p1[NB];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    float p[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        p[k] = fast_exp2(e[mb][nb][k]);
                        z[nb][k & 1] += p[k];
                        if constexpr (INT8) p[k] *= v_mul[mb][k >> 1] * inv;
                    }
                    using P = typename std::conditional<C::kHalfP, __half, __nv_bfloat16>::type;
                    p0[nb] = transpose_8x8(act_pack2(p[0], p[1], P()));
                    p1[nb] = transpose_8x8(act_pack2(p[2], p[3], P()));
                }
                if constexpr (INT8) {
                    // keys of columns 2 t, 2 t + 1 (and + 8) of V^T: four rows, of which this lane takes D / 8 columns
                    const int r0 = 16 * mb + key_of_row<D>(2 * t), r1 = 16 * mb + key_of_row<D>(2 * t + 1);
                    uint32_t x[4][D / 32];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int row = (i & 1 ? r1 : r0) + (i >> 1) * 8;
                        if constexpr (D == 128) {
                            const uint4 v = lds128(vst + code_piece<D>(row, g));
                            x[i][0] = v.x; x[i][1] = v.y; x[i][2] = v.z; x[i][3] = v.w;
                        } else {
                            const uint2 v = lds64(vst + code_piece<D>(row, g >> 1) + 8 * (g & 1));
                            x[i][0] = v.x; x[i][1] = v.y;
                        }
                    }
#pragma unroll
                    for (int w = 0; w < D / 32; ++w) {
                        const uint32_t u0 = x[0][w] ^ 0x80808080u, u1 = x[1][w] ^ 0x80808080u;
                        const uint32_t u2 = x[2][w] ^ 0x80808080u, u3 = x[3][w] ^ 0x80808080u;
                        const uint32_t lo01 = __byte_perm(u0, u1, 0x5140), hi01 = __byte_perm(u0, u1, 0x7362);
                        const uint32_t lo23 = __byte_perm(u2, u3, 0x5140), hi23 = __byte_perm(u2, u3, 0x7362);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint32_t a01 = h ? hi01 : lo01, a23 = h ? hi23 : lo23;
                            const uint32_t a0 = codes_to_half2<false>(a01), a1 = codes_to_half2<true>(a01);
                            const uint32_t a2 = codes_to_half2<false>(a23), a3 = codes_to_half2<true>(a23);
#pragma unroll
                            for (int nb = 0; nb < NB; ++nb) mma_16816<false>(acc[2 * w + h][nb], a0, a1, a2, a3, p0[nb], p1[nb]);
                        }
                    }
                } else {
                    const int row = 16 * mb + (lane & 7) + 8 * (lane >> 4), piece = (lane >> 3) & 1;
#pragma unroll
                    for (int md = 0; md < D / 16; ++md) {
                        uint32_t a[4];
                        ldmatrix_x4<true>(a, vst + value_piece<CH>(row, 2 * md + piece));
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb) mma_16816<BF16>(acc[md][nb], a[0], a[1], a[2], a[3], p0[nb], p1[nb]);
                    }
                }
            }
            held = stage;
            if (++stage == kStages) { stage = 0; phase ^= 1u; }
            ++taken;
            __syncwarp();                    // every lane is done with the stage; the segment's last one is kept for the merge
            if (start + C::kUnit < end) fire();
        }

        // ------------------------------------------------ the warps' results of the segment, merged in the stages read last
        // (every warp holds the same places of O^T; a warp without a chunk here has no stage to itself: its place is not read)
        float4* mine = reinterpret_cast<float4*>(ring + (warp * kStages + held) * kStageBytes);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                if (failed) z[nb][k] = NAN;
                z[nb][k] += __shfl_xor_sync(0xffffffffu, z[nb][k], 4);
                z[nb][k] += __shfl_xor_sync(0xffffffffu, z[nb][k], 8);
                z[nb][k] += __shfl_xor_sync(0xffffffffu, z[nb][k], 16);
                if (g == 0) { m_s[warp][8 * nb + 2 * t + k] = m_run[nb][k]; z_s[warp][8 * nb + 2 * t + k] = z[nb][k]; }
            }
            if (any && !failed)
#pragma unroll
                for (int md = 0; md < D / 16; ++md)
                    mine[(md * NB + nb) * 32 + lane] = make_float4(acc[md][nb][0], acc[md][nb][1], acc[md][nb][2], acc[md][nb][3]);
        }
        if (lane == 0) {
            v_ref_s[warp] = any && !failed ? (INT8 ? v_ref : 1.f) : -1.f;
            held_s[warp] = held;
        }
        __syncthreads();
        {
            const bool whole = cc.unit == 0 && u_end == cc.n_units;
            const int slot = 2 * cta + (first_segment ? 0 : 1);
#pragma unroll 1
            for (int i = warp; i < (D / 16) * NB; i += W) {
                const int md = i / NB, nb = i - md * NB;
                float m[2], zz[2], wgt[W][2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int n = 8 * nb + 2 * t + k;
                    m[k] = m_s[0][n];
#pragma unroll
                    for (int w = 1; w < W; ++w) m[k] = fmaxf(m[k], m_s[w][n]);
                    zz[k] = 0.f;
#pragma unroll
                    for (int w = 0; w < W; ++w) {
                        const float f = exp2f(m_s[w][n] - m[k]) * C::kUnOff;
                        zz[k] += z_s[w][n] * f;
                        wgt[w][k] = f * v_ref_s[w];
                    }
                }
                float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    if (v_ref_s[w] < 0.f) continue;
                    const float4 x = reinterpret_cast<const float4*>(ring + (w * kStages + held_s[w]) * kStageBytes)[i * 32 + lane];
                    o.x += x.x * wgt[w][0]; o.y += x.y * wgt[w][1]; o.z += x.z * wgt[w][0]; o.w += x.w * wgt[w][1];
                }
                if (whole) write_out<T, D, INT8, NB>(prm, cc.b, cc.h, md, nb, lane, o, m, zz);
                else prm.part_o[static_cast<int64_t>(slot) * C::kFrag + i * 32 + lane] = o;
                if (!whole && md == 0 && g == 0)
                    *reinterpret_cast<float4*>(prm.part_mz + slot * (8 * NB) + 8 * nb + 2 * t) = make_float4(m[0], zz[0], m[1], zz[1]);
            }
        }
        ptx::fence_proxy_async_smem();       // the stages go back to the copies
        __syncthreads();
        if (any && !failed) fire();
        first_segment = false;
        cc.left -= u_end - cc.unit;
        if (cc.left > 0) next_row(cc, prm, C::kUnit);
    }
    if (failed) {
        // the copies that are still on the way land before the shared memory is given back
        for (int i = taken; i < issued; ++i) {
            if (i == prm.drop_chunk) continue;
            for (int spin = 0; spin < (1 << 16); ++spin)
                if (ptx::mbar_try_wait(ptx::smem_u32(&full_bar[warp][i % kStages]), (i / kStages) & 1)) break;
        }
        ptx::cp_async_wait_all();
    }
}

// Joins the parts of a row that several CTAs shared: job (b, h, s, n) of the CTA blockIdx.x names slot s and, of that CTA and
// the n - 1 behind it, their first slots.  Block y takes rows md = y of the fragments; its warps take the parts in turn and
// several at a time (what bounds it is the round trips), then merge in shared memory.
constexpr int kJoinWarps = 8, kJoinAtOnce = 4;
template <class T, int D, bool INT8, int NB>
__global__ void __launch_bounds__(32 * kJoinWarps)
paged_join_kernel(const PagedDecodeParams prm) {
    __shared__ float4 o_s[kJoinWarps][NB][32];
    __shared__ float2 mz_s[kJoinWarps][NB][32][2];
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    using C = Cfg<T, D, INT8, NB>;
    const int4 job = __ldcg(prm.join + blockIdx.x);
    if (job.x < 0) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, t = lane & 3, md = blockIdx.y, parts = job.w + 1;
    float4 o[NB];
    float m[NB][2], z[NB][2];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        o[nb] = make_float4(0.f, 0.f, 0.f, 0.f);
        m[nb][0] = m[nb][1] = kNoMax;
        z[nb][0] = z[nb][1] = 0.f;
    }
    auto add = [&](int nb, const float4& x, const float2 (&mz)[2]) {
        float back[2], fore[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const float top = fmaxf(m[nb][k], mz[k].x);
            back[k] = exp2f(m[nb][k] - top);
            fore[k] = exp2f(mz[k].x - top);
            z[nb][k] = z[nb][k] * back[k] + mz[k].y * fore[k];
            m[nb][k] = top;
        }
        o[nb].x = o[nb].x * back[0] + x.x * fore[0]; o[nb].y = o[nb].y * back[1] + x.y * fore[1];
        o[nb].z = o[nb].z * back[0] + x.z * fore[0]; o[nb].w = o[nb].w * back[1] + x.w * fore[1];
    };
    for (int i0 = warp; i0 < parts; i0 += kJoinWarps * kJoinAtOnce) {
        float4 x[kJoinAtOnce][NB];
        float2 mz[kJoinAtOnce][NB][2];
#pragma unroll
        for (int j = 0; j < kJoinAtOnce; ++j) {
            const int i = i0 + j * kJoinWarps;
            if (i >= parts) continue;
            const int64_t slot = i == 0 ? job.z : 2 * (static_cast<int>(blockIdx.x) + i - 1);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                x[j][nb] = __ldcg(prm.part_o + slot * C::kFrag + (md * NB + nb) * 32 + lane);
                const float4 two = __ldcg(reinterpret_cast<const float4*>(prm.part_mz + slot * (8 * NB) + 8 * nb + 2 * t));
                mz[j][nb][0] = make_float2(two.x, two.y);
                mz[j][nb][1] = make_float2(two.z, two.w);
            }
        }
#pragma unroll
        for (int j = 0; j < kJoinAtOnce; ++j)
            if (i0 + j * kJoinWarps < parts)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) add(nb, x[j][nb], mz[j][nb]);
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        o_s[warp][nb][lane] = o[nb];
        mz_s[warp][nb][lane][0] = make_float2(m[nb][0], z[nb][0]);
        mz_s[warp][nb][lane][1] = make_float2(m[nb][1], z[nb][1]);
    }
    __syncthreads();
    if (warp >= NB) return;
    const int nb = warp;
    o[0] = o_s[0][nb][lane];
#pragma unroll
    for (int k = 0; k < 2; ++k) { m[0][k] = mz_s[0][nb][lane][k].x; z[0][k] = mz_s[0][nb][lane][k].y; }
    for (int w = 1; w < min(kJoinWarps, parts); ++w) add(0, o_s[w][nb][lane], mz_s[w][nb][lane]);
    write_out<T, D, INT8, NB>(prm, job.x, job.y, md, nb, lane, o[0], m[0], z[0]);
}

// ---------------------------------------------------------------------------------------------------- host

struct Plan {
    int NB, groups, HG, unit, ctas, splits;      // splits: whether a row can have more units than one
    size_t join_bytes, mz_bytes, total;
};

int resolve_decode(const tilemix_paged_t* p, int heads_q, PagedCache* c, Plan* plan) {
    const int rc = resolve_paged(p, c);
    if (rc) return rc;
    if (heads_q <= 0 || heads_q % p->heads_kv != 0) return TILEMIX_ERR_SHAPE;
    const int R = heads_q / p->heads_kv;
    plan->NB = R > 8 ? 2 : 1;
    plan->groups = static_cast<int>(ceil_div(R, 8 * plan->NB));
    plan->unit = kRingBytes / kStages / (2 * p->head_dim * (p->cache_type == TILEMIX_CACHE_INT8 ? 1 : 2));    // Cfg::kUnit
    const int64_t rows = static_cast<int64_t>(p->heads_kv) * plan->groups;
    const int64_t units = rows * p->batch * ceil_div(c->capacity, plan->unit);
    if (rows > (1 << 24) || units > (int64_t{1} << 30) || static_cast<int64_t>(p->batch) * heads_q > (int64_t{1} << 30)) return TILEMIX_ERR_SHAPE;
    plan->HG = static_cast<int>(rows);
    plan->ctas = static_cast<int>(units < kCtasPerSm * kSms ? units : kCtasPerSm * kSms);
    plan->splits = c->capacity > plan->unit;
    plan->join_bytes = (plan->ctas * sizeof(int4) + 255) / 256 * 256;
    plan->mz_bytes = (static_cast<size_t>(plan->ctas) * 2 * 8 * plan->NB * sizeof(float2) + 255) / 256 * 256;
    plan->total = plan->join_bytes + plan->mz_bytes + static_cast<size_t>(plan->ctas) * 2 * p->head_dim * 8 * plan->NB * sizeof(float);
    return TILEMIX_OK;
}

int row_strides(const int64_t* in, int B, int H, int d, bool output, int64_t out[2]) {
    const int64_t size[2] = {B, H}, dense[2] = {static_cast<int64_t>(H) * d, d};
    for (int i = 0; i < 2; ++i) {
        const int64_t s = in != nullptr ? in[i] : dense[i];
        if (size[i] > 1 && (s < 0 || s > (int64_t{1} << 40) || (output && s < d))) return TILEMIX_ERR_SHAPE;
        if (size[i] > 1 && s * 2 % 16 != 0) return TILEMIX_ERR_ALIGN;
        out[i] = size[i] == 1 ? 0 : 2 * s;
    }
    if (output && B > 1 && H > 1) {       // rows that overlap
        const int64_t a = out[0] < out[1] ? out[0] : out[1], z = out[0] < out[1] ? out[1] : out[0];
        const int64_t n = out[0] < out[1] ? B : H;
        if (z < a * (n - 1) + 2 * d) return TILEMIX_ERR_SHAPE;
    }
    return TILEMIX_OK;
}

template <class T, int D, bool INT8, int NB>
int launch(const PagedDecodeParams& prm, const Plan& plan, cudaStream_t stream) {
    using C = Cfg<T, D, INT8, NB>;
    const PagedCache& c = prm.c;
    static_assert(C::kUnit == kRingBytes / kStages / (2 * D * C::kElt), "see resolve_decode");
    CUtensorMap km, vm;
    const int page = 1 << c.page_shift, box_rows = page < C::CH ? page : C::CH;
    int rc;
    if ((rc = encode_pool_map(&km, c.k_pool, C::kElt, D, page, c.Hk, c.n_pages, c.ks, box_rows))) return rc;
    if ((rc = encode_pool_map(&vm, c.v_pool, C::kElt, D, page, c.Hk, c.n_pages, c.vs, box_rows))) return rc;
    auto kernel = paged_decode_kernel<T, D, INT8, NB>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmemBytes);
    if (e != cudaSuccess) return static_cast<int>(e);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(plan.ctas); cfg.blockDim = dim3(C::kThreads); cfg.dynamicSmemBytes = C::kSmemBytes; cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, kernel, prm, km, vm);
    g_launch_count.fetch_add(1);
    if (e != cudaSuccess || !plan.splits) return static_cast<int>(e);
    cfg.gridDim = dim3(plan.ctas, D / 16); cfg.blockDim = dim3(32 * kJoinWarps); cfg.dynamicSmemBytes = 0;
    e = cudaLaunchKernelEx(&cfg, paged_join_kernel<T, D, INT8, NB>, prm);
    g_launch_count.fetch_add(1);
    return static_cast<int>(e);
}

using Launch = int (*)(const PagedDecodeParams&, const Plan&, cudaStream_t);
template <class T, int D>
Launch pick(bool int8, int NB) {
    if (int8) return NB == 1 ? launch<T, D, true, 1> : launch<T, D, true, 2>;
    return NB == 1 ? launch<T, D, false, 1> : launch<T, D, false, 2>;
}

}  // namespace
}  // namespace tilemix

using namespace tilemix;

extern "C" {

size_t tilemix_paged_decode_workspace_size(const tilemix_paged_t* p, int32_t heads_q) {
    PagedCache c;
    Plan plan;
    return resolve_decode(p, heads_q, &c, &plan) ? 0 : plan.total;
}

int tilemix_paged_decode(const tilemix_paged_t* p, int32_t heads_q, float softmax_scale, const void* q, const int64_t* q_stride,
                         void* out, const int64_t* out_stride, float* lse, void* workspace, size_t workspace_bytes,
                         void* stream) {
    PagedDecodeParams prm{};
    Plan plan;
    int rc = resolve_decode(p, heads_q, &prm.c, &plan);
    if (rc) return rc;
    if (!q || !out || !workspace) return TILEMIX_ERR_NULL;
    if (!aligned16(q) || !aligned16(out) || !aligned16(workspace)) return TILEMIX_ERR_ALIGN;
    if ((rc = row_strides(q_stride, p->batch, heads_q, p->head_dim, false, prm.qs))) return rc;
    if ((rc = row_strides(out_stride, p->batch, heads_q, p->head_dim, true, prm.os))) return rc;
    if (workspace_bytes < plan.total) return TILEMIX_ERR_WORKSPACE;
    prm.Hq = heads_q; prm.R = heads_q / p->heads_kv; prm.groups = plan.groups; prm.HG = plan.HG;
    prm.scale_log2 = (softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf(static_cast<float>(p->head_dim))) * kLog2e;
    prm.q = static_cast<const uint8_t*>(q);
    prm.out = static_cast<uint8_t*>(out);
    prm.lse = lse;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    prm.join = reinterpret_cast<int4*>(ws);
    prm.part_mz = reinterpret_cast<float2*>(ws + plan.join_bytes);
    prm.part_o = reinterpret_cast<float4*>(ws + plan.join_bytes + plan.mz_bytes);
    prm.wait_limit_ns = g_wait_limit_ns.load();
    prm.drop_chunk = g_test_drop.load() == 2 ? 1 : -1;
    const bool int8 = p->cache_type == TILEMIX_CACHE_INT8;
    Launch go;
    if (p->act_type == TILEMIX_TYPE_FP16) go = p->head_dim == 128 ? pick<__half, 128>(int8, plan.NB) : pick<__half, 64>(int8, plan.NB);
    else go = p->head_dim == 128 ? pick<__nv_bfloat16, 128>(int8, plan.NB) : pick<__nv_bfloat16, 64>(int8, plan.NB);
    return go(prm, plan, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
