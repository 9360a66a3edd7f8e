// Decode step over a paged key/value cache: one query token per sequence.
//
// HBM-bound: a cached (token, KV head) is 4 d bytes (16-bit cache) or 2 (d + 4) (INT8 codes and scales), read once, and serves
// the R = H_q / H_k query heads of its group with 4 R d multiply-adds, far below the tensor cores' rate for R <= 16.  Hence
// warp-level MMAs: their operands pass through registers, where INT8 codes become FP16 and where a key past the end is masked,
// at the cost of ~25 instructions a token (INT8, d = 128) where HBM leaves an SM ~43 issue slots a token.  16 x 32K keys of 128,
// four KV heads, BF16: 159 us, 6.5 TB/s; 8 x 32K, eight KV heads, INT8: 91 us, 6.1 TB/s, 107 at the clock that the power cap
// leaves after half a second; one sequence of 500 keys 7.1 us, of which the step's latencies are 4 and the joining kernel's 2.
//
// Layout of the work.  A warp owns a ring of stages, starts its own copies and takes CHUNKS of 16 to 64 keys, which one TMA box
// a page brings in, swizzled; no warp waits for another but at the end of a row.  Four warps are a CTA, three CTAs share an SM
// (two with more than eight query heads): 192 KB are on the way.  (A warp of its own for the copies of all could not start them
// fast enough: four small ones a chunk, 8 x 32K keys of 128 in INT8 129 us, 101 so.)  Neighbouring chunks, one for each warp,
// are a UNIT; the units of all (sequence, KV head) rows, one row behind the other, are dealt out to the CTAs in equal runs, so
// that a batch of unequal lengths keeps every SM busy to the end.  A CTA finds its run from the lengths, which only the device
// knows.  Rows inside its run it finishes itself; of a row that it shares with its neighbours it leaves a partial result
// (m, z, O) to the joining kernel.  The copies run on across rows.
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
constexpr int kSms = 148;

struct PagedDecodeParams {
    PagedCache c;
    int Hq, R;                      // query heads, query heads per KV head
    int wave, jobs, workers;        // CTAs that run at the same time; jobs of the joining kernel; workers that there may be
    int groups, HG;                 // groups of up to 8 NB query heads per KV head; rows of a sequence (Hk * groups)
    float scale_log2;
    const uint8_t* q;
    uint8_t* out;
    int64_t qs[2], os[2];           // bytes: (batch, head)
    float* lse;
    int jobs_by_row;                // 1: a job of the joining kernel for every row, 0: for every worker that there may be
    int4* join;                     // [jobs]
    float4* part_o;                 // [2 workers][NB][D / 16][32 lanes]: accumulator fragments
    float2* part_mz;                // [2 workers][8 NB]: maximum (log2 domain) and sum
    unsigned long long wait_limit_ns;
    int drop_chunk;                 // testing aid: every warp leaves out the copies of its chunk of this number (-1: none)
    int skew, skew_copies;          // testing aid: odd warps take every length for that much shorter; the copies, later rows' for that much longer
};

// Length of sequence b.  Every warp reads the lengths for itself, some of them twice; one that changes while the call runs can
// leave the warps of a CTA, or a warp's copies and its products, with different ideas of what there is to do.  Hence every wait
// for another warp is bounded as those for copies are, what one warp hands to another is in bounds whatever it holds, and no
// CTA ends with copies on the way.
__device__ __forceinline__ int length_of(const PagedDecodeParams& prm, int b) {
    return max(paged_len(prm.c, b) - ((threadIdx.x & 32) != 0 ? prm.skew : 0), 0);
}

// The pools as tensor maps: boxes of a chunk, or of a page if that is smaller, and boxes of 16 tokens for smaller chunks.
struct PoolMaps {
    CUtensorMap k, v, k16, v16;
};

template <class T, int D, bool INT8, int NB>
struct Cfg {
    static constexpr int kElt = INT8 ? 1 : 2;
    // Warps of a CTA, stages of their rings, CTAs of an SM.  The INT8 form is bound by issue slots before bytes unless the cost of
    // a chunk (its copies, its wait, the look at the maxima) is spread over 32 keys: eight warps with chunks of 16 keys need 495
    // instructions for 16 keys, four with 32 need 349.  Sixteen query heads take the registers of a third CTA.  (us, three
    // CTAs of two stages and two of three: 64 ragged FP16 contexts, heads of 64 96 / 100, 64 short ones of 128 35 / 39, 16 x 32K
    // BF16 equal; 256 short INT8 ones 25 / 36.)
    static constexpr int W = 4;
    static constexpr int kStages = NB == 1 ? 2 : 3;
    static constexpr int kCtasPerSm = NB == 1 ? 3 : 2;
    static constexpr int kStageBytes = 8192;
    static constexpr int kRingBytes = W * kStages * kStageBytes;
    static constexpr int kMinTeam = 2;                              // see find_work
    static constexpr int kThreads = 32 * W;
    static constexpr int CH = kStageBytes / (2 * D * kElt);         // keys of a chunk
    static constexpr int kChShift = CH == 16 ? 4 : CH == 32 ? 5 : 6;
    static_assert(CH == 1 << kChShift, "chunks are whole boxes");
    static constexpr int MB = CH / 16;                              // blocks of 16 keys
    static constexpr int kVOff = CH * D * kElt;                     // values behind the keys of a stage
    static constexpr int kBoxCols = INT8 ? 1 : D / 64;              // boxes side by side in a row of 16-bit values
    static constexpr int kScaleBytes = INT8 ? W * kStages * CH * 8 : 0;
    static constexpr int kSmemBytes = kRingBytes + kScaleBytes + 1024;
    static constexpr int kFrag = (D / 16) * 32;                     // float4 fragments of a row's O, eight query heads
    // The probabilities are carried 2^14 times as large in FP16, so that what the rounding loses is below 2^-28 of the
    // largest instead of 2^-14.  bfloat16 has FP32's exponents.  The running maximum is moved only when a score exceeds it by
    // more than kLine (log2 units): 2^(14 + 1.5) fits FP16, and a chunk whose maximum need not be known costs no shuffles.
    static constexpr bool kHalfP = INT8 || std::is_same<T, __half>::value;
    static constexpr float kOff = kHalfP ? 14.f : 0.f;
    static constexpr float kUnOff = kHalfP ? 6.103515625e-5f : 1.f;
    static constexpr float kLine = kHalfP ? 1.5f : 8.f;
    // bfloat16 queries over INT8 codes are multiplied by a power of two of their row (see the segment's start)
    static constexpr bool kScaledQ = INT8 && std::is_same<T, __nv_bfloat16>::value;
    // A probability goes to the tensor cores as two 16-bit numbers, what the first leaves out being the second, so that the
    // error of an output is that of its own rounding (one number: 1.4 times that).  Every key's does, so that what a row is
    // rounded by does not depend on the rows beside it, which have a say in how chunks are cut.  bfloat16 outputs over an INT8
    // cache: one FP16 number, which has three bits more than the output.  (us, two numbers and one: 8 x 32K INT8
    // 97.9 / 97.6, at the clock that the power cap leaves 102.6 / 95.5, 32 x 4K 39.2 / 36.8, 64 x 500 26.7 / 25.0, 256 short, heads of
    // 64 24.2 / 23.4.)
    static constexpr bool kTwoHalves = !kScaledQ;
    // Blocks that a warp takes together, where a chunk has them whole: what does not depend on their number is done once for two.
    // (us together and one by one: 64 ragged FP16 steps, heads of 64 97 / 98, 8 x 32K INT8, heads of 64 51.7 / 55.3, 16 x 8K
    // 32.8 / 34.9, 256 short ones 24.7 / 25.8, 16 x 4K INT8, sixteen query heads 28.2 / 29.2.)  Heads of 128 over INT8 with
    // probabilities as two numbers: one by one, which needs no registers beyond those of three CTAs an SM (2 x 32K 35.5 / 33.9,
    // 1 x 8000 12.5 / 11.8, 32 x 100 12.5 / 11.2, 32 x 4K 40.1 / 39.1, 8 x 32K 97.0 / 91.2, but 105.1 / 106.9 at the clock that the
    // power cap leaves after half a second).
    static constexpr int kTogether = MB == 1 || (INT8 && D == 128 && NB == 1 && kTwoHalves) ? 1 : 2;
    static_assert(kFrag * 16 <= kStageBytes, "a row's O of one warp fits the stage that the warp has just read");
};
constexpr float kNoMax = -3.4028234663852886e38f;        // running maximum before the first key (finite: nothing is subtracted from an infinity)
// Scores are FP32 numbers, log2 units, once they are scaled; what is exponentiated is their difference to a whole number.  Up to
// this size a whole number and kOff add up exactly; from here on the maximum is a whole number by itself and kOff is left out,
// so that the exponent of the largest key is 0 whatever the scores' size (kOff less a maximum above 2^25 is rounded, by 2 and more:
// a probability beyond FP16's range, or none at all).
constexpr float kExact = 8388608.f;     // 2^23

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
    int b, h, unit, n_units, len, left;      // left: places from here to the end of the worker's run
};
__device__ __forceinline__ void next_row(Cursor& c, const PagedDecodeParams& prm, int unit_shift, int longer) {
    c.unit = 0;
    if (++c.h == prm.HG) {
        c.h = 0;
        do {
            if (++c.b >= prm.c.B) {          // (only if a length changed meanwhile)
                c.left = 0;
                return;
            }
            c.len = min(max(__shfl_sync(0xffffffffu, length_of(prm, c.b), 0) + longer, 0), prm.c.capacity);
            c.n_units = (c.len + (1 << unit_shift) - 1) >> unit_shift;
        } while (c.n_units == 0);
    }
}

// What a warp has to do: a run of places in the list of rows.  A worker is a team of the CTA's warps: all of them, or, where there are rows enough for more workers
// and the rows are short (fewer than kShortRow chunks a warp of the team on average), half of them.  Chunks are CH keys, or
// fewer where there would be fewer units than CTAs.  A unit is a chunk for each warp of the team; the U units go to n workers in
// shares of U / n or one more (and a long share to two workers, see below).
struct Work {
    Cursor at;
    int team_shift, chunk_shift, worker;
    int base, longer;                        // units of a share; the first `longer` shares have one more
    int pieces_shift, small;                 // 0: a share is one worker's; 1: two workers', the second one's are its last `small` units
    int extra;                               // units that a row counts as beyond its own, behind them

    __device__ __forceinline__ int share_first(int i) const { return i * base + min(i, longer); }
    __device__ __forceinline__ int units_of(int w) const {
        if (w & pieces_shift) return small;
        return base + ((w >> pieces_shift) < longer ? 1 : 0) - small;
    }
    __device__ __forceinline__ int first_of(int w) const {
        const int i = w >> pieces_shift;
        return w & pieces_shift ? share_first(i + 1) - small : share_first(i);
    }
    __device__ __forceinline__ int worker_of(int unit) const {
        const int split = longer * (base + 1), i = unit < split ? unit / (base + 1) : longer + (unit - split) / base;
        return (i << pieces_shift) + (pieces_shift != 0 && unit >= share_first(i + 1) - small ? 1 : 0);
    }
};
// (fewer than 4, 8, 16: 64 x 500 BF16 31.7 / 32.0 / 33.0 us, 32 x 2K INT8, one query head a KV head, heads of 64
// 25.9 / 25.0 / 25.2)
constexpr int kShortRow = 8;
// SMs do not get the same share of the memory's bandwidth (equal shares of 8 x 32K keys end after 70 to 92 us, in the order of
// their SMs' clusters).  Of long shares of a 16-bit cache the last eighth is a worker of its own, which goes to the SM that is
// done first: blocks behind the first wave.  (us without and with: 64 ragged FP16 steps, heads of 64 97.4 / 92.8, 16 x 32K BF16
// 161.2 / 159.7; a block's entry costs as much as that gains where shares are short, 16 x 4K BF16, sixteen query heads
// 37.1 / 42.9, and in the INT8 form, 8 x 32K 93.2 / 97.0.)
constexpr int kLongShare = 32;
// The start of a row and its merge cost a worker as much as some blocks of 16 keys; unless shares are short, a row counts as
// that many more, or the workers with the most rows end last.  (us with 0, 2, 4, 6 blocks: 64 x 500 BF16 35.4 / 32.0 / 31.9 /
// 31.9, 200 x 300 BF16, heads of 64 22.7 / 19.5 / 19.2 / 19.4, 256 short INT8, heads of 64 24.5 / 24.5 / 23.3 / 23.3, 32 x 4K
// INT8 37.2 / 36.8 / 36.8 / 37.7.  Where a worker has no more units than two rows' extra ones, a row would be dealt to fewer
// workers than there are: counted always and by that rule, 1 x 500 INT8 7.8 / 6.9, 1 x 2000 FP16 10.2 / 10.1; but 1 x 8000 INT8
// 12.0 / 12.5, 16 x 1K 17.0 / 18.3.)
constexpr int kRowBlocks = 4;
template <int W, int CH_SHIFT, int MIN_TEAM, int WAVE, bool PIECES>
__device__ __forceinline__ Work find_work(const PagedDecodeParams& prm) {
    static_assert(W == 4 && MIN_TEAM == 2, "teams of four or two warps");
    constexpr int kTeamShift = 2, kMinShift = 1;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, B = prm.c.B, ctas = prm.wave;
    // (the lengths of the first 256 sequences stay in registers: the loads wait for memory once)
    constexpr int kKept = 8;
    int kept[kKept];
#pragma unroll
    for (int i = 0; i < kKept; ++i) kept[i] = lane + 32 * i < B ? length_of(prm, lane + 32 * i) : 0;
    // sum of f(length) over the sequences, of this lane
    auto sum_of = [&](auto f) {
        int sum = 0;
#pragma unroll
        for (int i = 0; i < kKept; ++i) sum += f(kept[i]);
        for (int b = 32 * kKept + lane; b < B; b += 32) sum += f(length_of(prm, b));
        return sum;
    };
    const int blocks = __reduce_add_sync(0xffffffffu, sum_of([](int len) { return (len + 15) >> 4; })) * prm.HG;     // of 16 keys
    const int rows = __reduce_add_sync(0xffffffffu, sum_of([](int len) { return len > 0 ? 1 : 0; })) * prm.HG;
    Work w{};
    w.team_shift = kTeamShift; w.chunk_shift = CH_SHIFT;
    while (w.chunk_shift > 4 && (blocks >> (w.chunk_shift - 4 + kTeamShift)) < ctas) --w.chunk_shift;
    while (w.team_shift > kMinShift && rows >= (WAVE << (kTeamShift - w.team_shift)) &&
           (blocks >> (w.chunk_shift - 4 + w.team_shift)) < kShortRow * rows)
        --w.team_shift;
    const int unit_shift = w.chunk_shift + w.team_shift;
    auto units_of = [&](int len) { return (len + (1 << unit_shift) - 1) >> unit_shift; };
    int U = __reduce_add_sync(0xffffffffu, sum_of(units_of)) * prm.HG;
    const int most = ctas << (kTeamShift - w.team_shift), n = min(most, U), extra = kRowBlocks << 4 >> w.chunk_shift;
    if (U > 2 * extra * most) {
        w.extra = extra;
        U += extra * rows;
    }
    if (n > 0) { w.base = U / n; w.longer = U - w.base * n; }
    const int block = blockIdx.x;
    if (PIECES && gridDim.x > ctas && w.team_shift == kTeamShift && w.base >= kLongShare) {
        w.pieces_shift = 1;
        w.small = w.base >> 3;
        w.worker = block < ctas ? 2 * block : 2 * (block - ctas) + 1;
    } else {
        w.worker = block < ctas ? (block << (kTeamShift - w.team_shift)) + (warp >> w.team_shift) : 0x40000000;
        if (w.worker >= n) return w;
    }
    Cursor& c = w.at;
    const int first = w.first_of(w.worker);
    int before = 0;                          // places of the sequences before the 32 in hand
    auto among = [&](int b0, int len) -> bool {
        const int mine = len > 0 ? units_of(len) + w.extra : 0, all = __reduce_add_sync(0xffffffffu, mine) * prm.HG;
        if (before + all <= first) {
            before += all;
            return false;
        }
        int upto = mine * prm.HG;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += x;
        }
        const int l = __ffs(__ballot_sync(0xffffffffu, before + upto > first)) - 1;
        c.b = b0 + l;
        const int places = __shfl_sync(0xffffffffu, mine, l);
        c.n_units = places - w.extra;
        c.len = __shfl_sync(0xffffffffu, len, l);
        const int at = first - before - (__shfl_sync(0xffffffffu, upto, l) - places * prm.HG);
        c.h = at / places;
        c.unit = at - c.h * places;
        c.left = w.units_of(w.worker);
        return true;
    };
#pragma unroll
    for (int i = 0; i < kKept; ++i)
        if (32 * i < B && among(32 * i, kept[i])) return w;
    for (int b0 = 32 * kKept; b0 < B; b0 += 32)
        if (among(b0, b0 + lane < B ? length_of(prm, b0 + lane) : 0)) return w;
    return w;
}

// ---------------------------------------------------------------------------------------------------- results
// Where the rows of query columns 2 t, 2 t + 1 of block nb go, and what their sums are divided by.  Fragment (md, lane) of O^T
// is (d0, column 2 t), (d0, 2 t + 1), (d1, 2 t), (d1, 2 t + 1) with (d0, d1) = (16 md + g, + 8), of an INT8 cache
// (D / 8 g + 2 md, + 1).
template <class T, int D, bool INT8>
struct OutRows {
    uint8_t* dst[2];                // nullptr: there is no such query head
    float inv[2];

    __device__ __forceinline__ OutRows(const PagedDecodeParams& prm, int b, int h, int width, int nb, int lane) {
        const int hk = prm.groups == 1 ? h : h / prm.groups, n = (h - hk * prm.groups) * width + 8 * nb + 2 * (lane & 3);
        uint8_t* row = prm.out + b * prm.os[0] + (static_cast<int64_t>(hk) * prm.R + n) * prm.os[1];
        dst[0] = n < prm.R ? row : nullptr;
        dst[1] = n + 1 < prm.R ? row + prm.os[1] : nullptr;
        head = static_cast<int64_t>(b) * prm.Hq + hk * prm.R + n;
    }
    // Sums of the columns; the lse of their rows by the lanes of `write_lse`.
    __device__ __forceinline__ void sums(const PagedDecodeParams& prm, const float (&m)[2], const float (&z)[2], bool write_lse) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const bool empty = z[i] == 0.f;              // (not if it is a NaN)
            inv[i] = empty ? 0.f : __fdividef(1.f, z[i]);
            if (write_lse && dst[i] != nullptr && prm.lse != nullptr) prm.lse[head + i] = empty ? -INFINITY : (m[i] + log2f(z[i])) * kLn2;
        }
    }
    __device__ __forceinline__ void store(int md, int lane, const float4& o) const {
        const int g = lane >> 2;
        const float v[2][2] = {{o.x, o.z}, {o.y, o.w}};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (dst[i] == nullptr) continue;
            const uint32_t two = act_pack2(v[i][0] * inv[i], v[i][1] * inv[i], T());
            if constexpr (INT8) {
                reinterpret_cast<uint32_t*>(dst[i])[(D / 16) * g + md] = two;
            } else {
                reinterpret_cast<uint16_t*>(dst[i])[16 * md + g] = static_cast<uint16_t>(two);
                reinterpret_cast<uint16_t*>(dst[i])[16 * md + g + 8] = static_cast<uint16_t>(two >> 16);
            }
        }
    }

private:
    int64_t head;
};

// ---------------------------------------------------------------------------------------------------- the step
template <class T, int D, bool INT8, int NB>
__global__ void __launch_bounds__(Cfg<T, D, INT8, NB>::kThreads, Cfg<T, D, INT8, NB>::kCtasPerSm)
paged_decode_kernel(const PagedDecodeParams prm, const __grid_constant__ PoolMaps maps) {
    using C = Cfg<T, D, INT8, NB>;
    constexpr int CH = C::CH, MB = C::MB, W = C::W, kStages = C::kStages, kStageBytes = C::kStageBytes;
    constexpr bool BF16 = !C::kHalfP;
    extern __shared__ uint8_t smem[];
    __shared__ __align__(8) uint64_t full_bar[W][kStages], team_bar[1 + W / C::kMinTeam];     // team_bar[0]: of all warps
    __shared__ uint32_t hole_s[W][kStages];                          // bit 4 i: the 16 keys i of the chunk lie in a hole
    __shared__ __align__(8) float m_s[W][8 * NB], z_s[W][8 * NB];
    __shared__ float v_ref_s[W];
    __shared__ int held_s[W];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    uint8_t* ring = smem + ((1024u - (ptx::smem_u32(smem) & 1023u)) & 1023u);      // (the swizzle's pattern repeats every 1 KB)
    const PagedCache& c = prm.c;

    if (lane == 0) {
        held_s[warp] = 0;                    // (read by the other warps of a team, should a wait for this one run out)
        v_ref_s[warp] = -1.f;
        if (warp == 0)
            for (int i = 0; i < 1 + W / C::kMinTeam; ++i) ptx::mbar_init(ptx::smem_u32(&team_bar[i]), i == 0 ? W : C::kMinTeam);
        // (arrivals: the lane that announces the bytes of the boxes, and every lane with its part of the scales)
        for (int i = 0; i < kStages; ++i) ptx::mbar_init(ptx::smem_u32(&full_bar[warp][i]), INT8 ? 33 : 1);
        ptx::fence_mbar_init();
    }
    __syncthreads();
    ptx::griddep_wait();                     // the cache, the lengths and the queries may be the work of the kernel before
    ptx::griddep_launch_dependents();

    const Work work = find_work<W, C::kChShift, C::kMinTeam, C::kCtasPerSm * kSms, !INT8>(prm);
    const int team = 1 << work.team_shift, member = warp & (team - 1), team_no = warp >> work.team_shift;
    const int chunk_shift = work.chunk_shift, chunk = 1 << chunk_shift, unit_shift = chunk_shift + work.team_shift, unit_keys = 1 << unit_shift;
    Cursor cc = work.at;

    // Bounded wait; the verdict is the warp's (a copy may land for some lanes as others give up, and what follows takes the whole
    // warp).
    auto passed = [&](uint32_t bar, uint32_t phase, uint64_t limit_ns) -> bool {
        if (__all_sync(0xffffffffu, ptx::mbar_try_wait(bar, phase))) return true;
        const uint64_t begin = ptx::globaltimer_ns();
        uint32_t spins = 0;
        while (!__all_sync(0xffffffffu, ptx::mbar_try_wait(bar, phase)))
            if ((++spins & 63u) == 0u && __any_sync(0xffffffffu, ptx::globaltimer_ns() - begin > limit_ns)) return false;
        return true;
    };
    bool failed = false, lost = false;              // a wait ran out: no more copies, the rows from here on are NaN; lost: one for the team
    // Barrier of the team.  (Its limit leaves the others time to give up a copy of theirs.)
    uint32_t team_phase = 0u;
    auto team_sync = [&]() {
        __syncwarp();
        if (lost) return;
        const uint32_t bar = ptx::smem_u32(&team_bar[team == W ? 0 : 1 + team_no]);
        if (lane == 0) ptx::mbar_arrive(bar);
        if (passed(bar, team_phase, 4 * prm.wait_limit_ns + 50000000u)) team_phase ^= 1u;
        else failed = lost = true;
    };

    // Query fragments of a row, as they lie in memory: the right operand (columns = heads g of the block).  INT8: fragment
    // 4 j + w holds features 16 (t + 4 j) + 4 w .. + 3, as the codes come.
    uint32_t qf[NB][D / 16][2];
    auto fetch_q = [&](const Cursor& at) {
        const int hk = prm.groups == 1 ? at.h : at.h / prm.groups, first = (at.h - hk * prm.groups) * 8 * NB;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const bool on = first + 8 * nb + g < prm.R;
            const uint8_t* row = prm.q + at.b * prm.qs[0] + (static_cast<int64_t>(hk) * prm.R + first + 8 * nb + g) * prm.qs[1];
            if constexpr (INT8) {
#pragma unroll
                for (int j = 0; j < D / 64; ++j)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        uint4 x = make_uint4(0u, 0u, 0u, 0u);
                        if (on) x = __ldcg(reinterpret_cast<const uint4*>(row + 32 * (t + 4 * j)) + i);
                        qf[nb][4 * j + 2 * i][0] = x.x; qf[nb][4 * j + 2 * i][1] = x.y;
                        qf[nb][4 * j + 2 * i + 1][0] = x.z; qf[nb][4 * j + 2 * i + 1][1] = x.w;
                    }
            } else {
#pragma unroll
                for (int i = 0; i < D / 16; ++i)
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        qf[nb][i][k] = on ? __ldcg(reinterpret_cast<const uint32_t*>(row + 32 * i + 16 * k) + t) : 0u;
            }
        }
    };
    if (cc.left > 0) fetch_q(cc);

    // ---- copies.  `prepare` finds this warp's next chunk and looks its pages up, every lane that of four of its keys;
    // `fire` starts its copies into the stage behind the one filled last.
    const CUtensorMap* const k_map = chunk_shift < C::kChShift ? &maps.k16 : &maps.k;
    const CUtensorMap* const v_map = chunk_shift < C::kChShift ? &maps.v16 : &maps.v;
    const int box_shift = chunk_shift < C::kChShift ? 4 : min(c.page_shift, chunk_shift), page_mask = (1 << c.page_shift) - 1;
    const uint32_t ring_u32 = ptx::smem_u32(ring) + warp * (kStages * kStageBytes);
    constexpr int kQuads = CH / 4;
    const int quad = 4 * (lane & (kQuads - 1));
    const uint32_t scale_u32 = ptx::smem_u32(ring) + C::kRingBytes + warp * (kStages * CH * 8) + 16 * lane;
    const int page_rows = c.Hk << c.page_shift;               // scales of a page
    Cursor ic = cc;                                           // the row of the next chunk
    int issued = 0, fill = 0, next_start = 0, next_end = 0, next_hk = 0, next_page = -1;   // next_end: of this worker's keys of the row
    const int32_t* next_table = nullptr;
    const float* next_scale = nullptr;                        // this lane's: of K or of V, of the row's head
    auto enter_row = [&]() {
        const int u_end = min(ic.n_units, ic.unit + ic.left);
        next_start = (ic.unit << unit_shift) + (member << chunk_shift);
        next_end = min(ic.len, u_end << unit_shift);
        ic.left -= u_end - ic.unit + work.extra;
        next_hk = prm.groups == 1 ? ic.h : ic.h / prm.groups;
        next_table = c.table + ic.b * c.table_stride;
        if constexpr (INT8) next_scale = (lane < kQuads ? c.k_scale : c.v_scale) + (static_cast<int64_t>(next_hk) << c.page_shift);
    };
    auto prepare = [&]() {
        while (next_start >= next_end && ic.left > 0) {
            next_row(ic, prm, unit_shift, prm.skew_copies);
            if (ic.left > 0) enter_row();
        }
        if (next_start >= next_end) return;
        const int pos = next_start + quad;
        next_page = -1;
        if (quad < chunk && pos < ic.len) next_page = next_table[pos >> c.page_shift];
        if (static_cast<unsigned>(next_page) >= static_cast<unsigned>(c.n_pages)) next_page = -1;
    };
    auto fire = [&]() {
        if (next_start >= next_end) return;
        const uint32_t bar = ptx::smem_u32(&full_bar[warp][fill]);
        const uint32_t holes = __ballot_sync(0xffffffffu, next_page < 0 && quad < chunk && next_start + quad < ic.len);
        if (lane == 0) hole_s[warp][fill] = holes;
        if (issued != prm.drop_chunk) {
            const int boxes = (min(chunk, ic.len - next_start) + (1 << box_shift) - 1) >> box_shift, row = next_start & page_mask;
            if (lane == 0) ptx::mbar_arrive_expect_tx(bar, (boxes << box_shift) * (2 * D * C::kElt));
            const uint32_t dst = ring_u32 + fill * kStageBytes;
#pragma unroll
            for (int i = 0; i < CH / 16; ++i) {
                if (i >= boxes) break;
                // (a hole's box lies outside the map: zeros arrive, nothing is read)
                const int page = __shfl_sync(0xffffffffu, next_page, i << (box_shift - 2));
                const uint32_t to = dst + (i << box_shift) * (INT8 ? D : 128);
#pragma unroll
                for (int col = 0; col < C::kBoxCols; ++col)
                    ptx::tma_load_pair_4d(to + col * (CH * 128), to + col * (CH * 128) + C::kVOff, k_map, v_map, bar, col * 64, (row + (i << box_shift)) & page_mask, next_hk, page);
            }
            if constexpr (INT8) {
                if (lane < 2 * kQuads)
                    ptx::cp_async_16(scale_u32 + fill * (CH * 8), next_scale + static_cast<int64_t>(max(next_page, 0)) * page_rows + ((next_start + quad) & page_mask),
                                     next_page >= 0);
                ptx::cp_async_arrive(bar);
            }
        }
        ++issued;
        if (++fill == kStages) fill = 0;
        next_start += unit_keys;
        prepare();
    };
    if (ic.left > 0) {
        enter_row();
        prepare();
    }
#pragma unroll 1
    for (int i = 0; i < kStages; ++i) fire();

    // ==================================================================== products
    // What the joining kernel finds: the first worker that begins inside a row has that row joined.
    if (member == 0 && lane == 0) {
        const int worker = work.worker;
        int4 job = make_int4(-1, 0, 0, 0);
        if (cc.left > 0 && cc.unit > 0 && cc.unit < cc.n_units) {
            const int row_first = work.first_of(worker) - cc.unit, before = work.first_of(worker - 1);
            if (before <= row_first) {
                const int last = work.worker_of(row_first + cc.n_units - 1);
                // row, the slot of the part in front, and the workers whose first slots hold the others
                job = make_int4(cc.b * prm.HG + cc.h, 2 * (worker - 1) + (before >= row_first - work.extra ? 0 : 1), worker, last - worker + 1);
            }
        }
        // (by worker: a job each; teams that there are not, and blocks without work, write theirs too)
        const int at = work.pieces_shift != 0 ? work.worker : static_cast<int>(blockIdx.x) * (W / C::kMinTeam) + team_no;
        if (prm.jobs_by_row) {
            if (job.x >= 0) prm.join[job.x] = job;
        } else if (at < prm.jobs) {
            prm.join[at] = job;
        }
    }
    if (!prm.jobs_by_row && work.pieces_shift == 0 && tid >= W / team && tid < W / C::kMinTeam) {
        const int at = static_cast<int>(blockIdx.x) * (W / C::kMinTeam) + tid;
        if (at < prm.jobs) prm.join[at] = make_int4(-1, 0, 0, 0);
    }
    // sequences without a key
    for (int b = blockIdx.x; b < c.B; b += gridDim.x) {
        if (paged_len(c, b) > 0) continue;
        for (int i = tid; i < prm.Hq * (D / 8); i += 32 * W) {
            const int hq = i / (D / 8);
            reinterpret_cast<uint4*>(prm.out + b * prm.os[0] + hq * prm.os[1])[i - hq * (D / 8)] = make_uint4(0u, 0u, 0u, 0u);
        }
        if (prm.lse != nullptr)
            for (int hq = tid; hq < prm.Hq; hq += 32 * W) prm.lse[static_cast<int64_t>(b) * prm.Hq + hq] = -INFINITY;
        if (prm.jobs_by_row)
            for (int h = tid; h < prm.HG; h += 32 * W) prm.join[b * prm.HG + h] = make_int4(-1, 0, 0, 0);
    }

    const float* const scale_ring = reinterpret_cast<const float*>(ring + C::kRingBytes) + warp * (kStages * CH * 2);
    // Where this lane's pieces of a stage lie.  INT8: rows key_of_row(g) of the keys, key_of_row(2 t) and (2 t + 1) of the
    // values; the other rows of a block are 8 or 16 rows, the other half of a row of 128 is bit 6 away.
    const int k_row = key_of_row<D>(g), v_row0 = key_of_row<D>(2 * t), v_row1 = key_of_row<D>(2 * t + 1);
    const uint8_t* const stages = ring + warp * (kStages * kStageBytes);
    const uint32_t k_at = code_piece<D>(k_row, t);
    const uint32_t v_at0 = C::kVOff + (D == 128 ? code_piece<D>(v_row0, g) : code_piece<D>(v_row0, g >> 1) + 8 * (g & 1));
    const uint32_t v_at1 = C::kVOff + (D == 128 ? code_piece<D>(v_row1, g) : code_piece<D>(v_row1, g >> 1) + 8 * (g & 1));
    int stage = 0, taken = 0;
    uint32_t phase = 0u;
    bool first_segment = true;
#pragma unroll 1
    while (cc.left > 0) {
        // ------------------------------------------------ a row, or this worker's part of it
        const int u_end = min(cc.n_units, cc.unit + cc.left);
        [[maybe_unused]] float q_mul[NB][2];                  // what a score is multiplied by yet: a power of two
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            if constexpr (C::kScaledQ) {
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
                q_mul[nb][0] = __shfl_sync(0xffffffffu, down, 8 * t);
                q_mul[nb][1] = __shfl_sync(0xffffffffu, down, 8 * t + 4);
            }
        }

        // sub = kOff less the running maximum, which is rounded up to a whole number: what has been summed is brought to another
        // maximum exactly, and an exponent, below 16, is rounded by 2^-21 at most.  (Above kExact: see there.)
        float sub[NB][2], z[NB][2], acc[D / 16][NB][4];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            sub[nb][0] = sub[nb][1] = C::kOff - kNoMax;
            z[nb][0] = z[nb][1] = 0.f;
#pragma unroll
            for (int md = 0; md < D / 16; ++md) acc[md][nb][0] = acc[md][nb][1] = acc[md][nb][2] = acc[md][nb][3] = 0.f;
        }
        // INT8: the scale of a value is folded into its probability relative to v_ref, a power of two at or above every
        // scale so far; O~ is in units of it.
        float v_ref = 7.888609052210118e-31f;                 // 2^-100
        const int end = min(cc.len, u_end << unit_shift);       // keys of this segment
        bool any = false;
        int held = 0;

#pragma unroll 1
        for (int start = (cc.unit << unit_shift) + (member << chunk_shift); start < end; start += unit_keys) {
            if (!failed && !passed(ptx::smem_u32(&full_bar[warp][stage]), phase, prm.wait_limit_ns)) failed = true;
            if (failed) break;
            any = true;
            const int live = min(chunk, cc.len - start);      // keys of the chunk
            const uint32_t holes = hole_s[warp][stage];
            // `first_mb`: block of 16 keys; BLOCKS of them together, PART: keys of it may not exist
            auto attend = [&](auto blocks, auto part, int first_mb) {
                constexpr int BLOCKS = decltype(blocks)::value;
                constexpr bool PART = decltype(part)::value;
                constexpr bool TWO_P = C::kTwoHalves;
                [[maybe_unused]] const uint32_t kst = ring_u32 + stage * kStageBytes + first_mb * (16 * (INT8 ? D : 128)), vst = kst + C::kVOff;
                [[maybe_unused]] const uint8_t* const st = stages + stage * kStageBytes + first_mb * (16 * (INT8 ? D : 128));
                // ---- S^T: sc[mb][nb] = (row g, columns 2 t, 2 t + 1), (row g + 8, the same).  A block alone sums its even and its
                // odd steps apart: the chain of MMAs that wait for one another is half as long.
                constexpr bool TWO = BLOCKS * NB == 1;
                [[maybe_unused]] float sc[BLOCKS][NB][4], v_mul[BLOCKS][2], odd[BLOCKS][NB][4];
#pragma unroll
                for (int mb = 0; mb < BLOCKS; ++mb)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                        for (int k = 0; k < 4; ++k) sc[mb][nb][k] = odd[mb][nb][k] = 0.f;
#pragma unroll
                for (int mb = 0; mb < BLOCKS; ++mb) {
                    if constexpr (INT8) {
#pragma unroll
                        for (int j = 0; j < D / 64; ++j) {
                            const uint8_t* const at = st + (k_at ^ (64 * j)) + 16 * mb * D;
                            const uint4 xa = *reinterpret_cast<const uint4*>(at), xb = *reinterpret_cast<const uint4*>(at + 8 * D);
                            const uint32_t wa[4] = {xa.x, xa.y, xa.z, xa.w}, wb[4] = {xb.x, xb.y, xb.z, xb.w};
#pragma unroll
                            for (int w = 0; w < 4; ++w) {
                                const uint32_t ua = wa[w] ^ 0x80808080u, ub = wb[w] ^ 0x80808080u;
                                const uint32_t a0 = codes_to_half2<false>(ua), a2 = codes_to_half2<true>(ua);
                                const uint32_t a1 = codes_to_half2<false>(ub), a3 = codes_to_half2<true>(ub);
#pragma unroll
                                for (int nb = 0; nb < NB; ++nb)
                                    mma_16816<false>(TWO && (w & 1) ? odd[mb][nb] : sc[mb][nb], a0, a1, a2, a3, qf[nb][4 * j + w][0], qf[nb][4 * j + w][1]);
                            }
                        }
                    } else {
                        const int row = 16 * mb + (lane & 15), piece = lane >> 4;
#pragma unroll
                        for (int i = 0; i < D / 16; ++i) {
                            uint32_t a[4];
                            ldmatrix_x4<false>(a, kst + value_piece<CH>(row, 2 * i + piece));
#pragma unroll
                            for (int nb = 0; nb < NB; ++nb)
                                mma_16816<BF16>(TWO && (i & 1) ? odd[mb][nb] : sc[mb][nb], a[0], a[1], a[2], a[3], qf[nb][i][0], qf[nb][i][1]);
                        }
                    }
                }
                [[maybe_unused]] const float* const sk = scale_ring + stage * (CH * 2) + 16 * first_mb + k_row;
#pragma unroll
                for (int mb = 0; mb < BLOCKS; ++mb)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        // (the scale is part of the score before the maximum is taken: equal keys have equal scores, and the
                        // largest one's exponent is what the maximum says.  As a factor of the exponent's multiply-add, its
                        // rounding would be a difference between the two, as large as the scores.)
                        float mul = prm.scale_log2;
                        if constexpr (INT8) { mul *= sk[16 * mb + 8 * i]; v_mul[mb][i] = sk[CH + 16 * mb + 8 * i]; }
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                if constexpr (TWO) sc[mb][nb][2 * i + k] += odd[mb][nb][2 * i + k];
                                sc[mb][nb][2 * i + k] *= mul;
                            }
                    }
                // ---- keys past the end and in holes do not exist, whatever lies in their rows
                if constexpr (PART) {
                    const bool hole = (holes >> (4 * first_mb)) & 1u;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        if (16 * first_mb + 8 * i + (INT8 ? k_row : g) < live && !hole) continue;
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb) sc[0][nb][2 * i] = sc[0][nb][2 * i + 1] = -INFINITY;
                        v_mul[0][i] = 0.f;
                    }
                    if constexpr (!INT8) {
                        const int left = live - 16 * first_mb;          // (0 times a NaN is one)
                        if (left < 16) {
                            for (int i = lane; i < (16 - left) * (D / 8); i += 32) {
                                const int row = left + i / (D / 8), piece = i & (D / 8 - 1);
                                asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(vst + value_piece<CH>(row, piece)), "r"(0u) : "memory");
                            }
                            ptx::fence_proxy_async_smem();
                            __syncwarp();
                        }
                    }
                }
                // ---- exponents, relative to the running maximum; it moves when one of them passes the line
                float top = -INFINITY;
                float e[BLOCKS][NB][4];
                auto exponents = [&]() {
#pragma unroll
                    for (int mb = 0; mb < BLOCKS; ++mb)
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                if constexpr (C::kScaledQ) e[mb][nb][k] = fmaf(sc[mb][nb][k], q_mul[nb][k & 1], sub[nb][k & 1]);
                                else e[mb][nb][k] = sc[mb][nb][k] + sub[nb][k & 1];
                            }
                };
                exponents();
#pragma unroll
                for (int mb = 0; mb < BLOCKS; ++mb)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) top = fmax3(fmax3(top, e[mb][nb][0], e[mb][nb][1]), e[mb][nb][2], e[mb][nb][3]);
                bool past = top > C::kOff + C::kLine;
                if constexpr (INT8) {
                    float v_top = fmaxf(v_mul[0][0], v_mul[0][1]);
#pragma unroll
                    for (int mb = 1; mb < BLOCKS; ++mb) v_top = fmax3(v_top, v_mul[mb][0], v_mul[mb][1]);
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
                            for (int mb = 1; mb < BLOCKS; ++mb) x = fmax3(x, sc[mb][nb][k], sc[mb][nb][2 + k]);
                            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
                            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
                            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
                            if constexpr (C::kScaledQ) x *= q_mul[nb][k];
                            x = ceilf(x);
                            const float s_new = fminf(sub[nb][k], (fabsf(x) < kExact ? C::kOff : 0.f) - x);
                            alpha[nb][k] = fast_exp2(s_new - sub[nb][k]);
                            sub[nb][k] = s_new;
                            z[nb][k] *= alpha[nb][k];
                        }
                    if constexpr (INT8) {
                        uint32_t dv = 0u;
#pragma unroll
                        for (int mb = 0; mb < BLOCKS; ++mb) dv = max(dv, max(__float_as_uint(fabsf(v_mul[mb][0])), __float_as_uint(fabsf(v_mul[mb][1]))));
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
                    exponents();
                }
                const float inv = __uint_as_float(0x7f000000u - __float_as_uint(v_ref));
                // ---- probabilities, and O^T += V^T P^T block by block
#pragma unroll
                for (int mb = 0; mb < BLOCKS; ++mb) {
                    [[maybe_unused]] uint32_t p0[NB], p1[NB], r0[NB], r1[NB];
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
                        const uint32_t h0 = act_pack2(p[0], p[1], P()), h1 = act_pack2(p[2], p[3], P());
                        p0[nb] = transpose_8x8(h0);
                        p1[nb] = transpose_8x8(h1);
                        if constexpr (TWO_P) {
                            const float2 f0 = act_to_float2(h0, P()), f1 = act_to_float2(h1, P());
                            r0[nb] = transpose_8x8(act_pack2(p[0] - f0.x, p[1] - f0.y, P()));
                            r1[nb] = transpose_8x8(act_pack2(p[2] - f1.x, p[3] - f1.y, P()));
                        }
                    }
                    if constexpr (INT8) {
                        // keys of columns 2 t, 2 t + 1 (and + 8) of V^T: four rows, of which this lane takes D / 8 columns
                        uint32_t x[4][D / 32];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint8_t* const at = st + (i & 1 ? v_at1 : v_at0) + (16 * mb + 8 * (i >> 1)) * D;
                            if constexpr (D == 128) {
                                const uint4 v = *reinterpret_cast<const uint4*>(at);
                                x[i][0] = v.x; x[i][1] = v.y; x[i][2] = v.z; x[i][3] = v.w;
                            } else {
                                const uint2 v = *reinterpret_cast<const uint2*>(at);
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
                                for (int nb = 0; nb < NB; ++nb) {
                                    mma_16816<false>(acc[2 * w + h][nb], a0, a1, a2, a3, p0[nb], p1[nb]);
                                    if constexpr (TWO_P) mma_16816<false>(acc[2 * w + h][nb], a0, a1, a2, a3, r0[nb], r1[nb]);
                                }
                            }
                        }
                    } else {
                        const int row = 16 * mb + (lane & 7) + 8 * (lane >> 4), piece = (lane >> 3) & 1;
#pragma unroll
                        for (int md = 0; md < D / 16; ++md) {
                            uint32_t a[4];
                            ldmatrix_x4<true>(a, vst + value_piece<CH>(row, 2 * md + piece));
#pragma unroll
                            for (int nb = 0; nb < NB; ++nb) {
                                mma_16816<BF16>(acc[md][nb], a[0], a[1], a[2], a[3], p0[nb], p1[nb]);
                                if constexpr (TWO_P) mma_16816<BF16>(acc[md][nb], a[0], a[1], a[2], a[3], r0[nb], r1[nb]);
                            }
                        }
                    }
                }
            };
            if (C::kTogether > 1 && live == CH && holes == 0u)
#pragma unroll 1
                for (int mb = 0; mb < MB; mb += C::kTogether) attend(std::integral_constant<int, C::kTogether>(), std::false_type(), mb);
            else
#pragma unroll 1
                for (int mb = 0; 16 * mb < live; ++mb) attend(std::integral_constant<int, 1>(), std::true_type(), mb);
            held = stage;
            if (++stage == kStages) { stage = 0; phase ^= 1u; }
            ++taken;
            __syncwarp();                    // every lane is done with the stage; the segment's last one is kept for the merge
            if (start + unit_keys < end) fire();
        }

        // ------------------------------------------------ the warps' results of the segment, merged in the stages read last
        // (every warp holds the same places of O^T; a warp without a chunk here has no stage to itself: its place is not read)
        const bool none = cc.unit >= cc.n_units, whole = cc.unit == 0 && u_end == cc.n_units;
        const int slot = 2 * work.worker + (first_segment ? 0 : 1), b = cc.b, h = cc.h;
        if (whole && prm.jobs_by_row && member == 0 && lane == 0) prm.join[b * prm.HG + h] = make_int4(-1, 0, 0, 0);
        first_segment = first_segment && none;
        cc.left -= u_end - cc.unit + work.extra;
        if (cc.left > 0) {
            next_row(cc, prm, unit_shift, 0);
            if (cc.left > 0) fetch_q(cc);                     // (on the way during the merge)
        }
        if (none) continue;                                   // (a run that begins behind the units of a row)
        float4* mine = reinterpret_cast<float4*>(ring + (warp * kStages + held) * kStageBytes);
        if (lane == 0) {
            v_ref_s[warp] = any && !failed ? (INT8 ? v_ref : 1.f) : -1.f;
            held_s[warp] = held;
        }
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                if (failed) z[nb][k] = NAN;
                z[nb][k] += __shfl_xor_sync(0xffffffffu, z[nb][k], 4);
                z[nb][k] += __shfl_xor_sync(0xffffffffu, z[nb][k], 8);
                z[nb][k] += __shfl_xor_sync(0xffffffffu, z[nb][k], 16);
                if (g == 0) { m_s[warp][8 * nb + 2 * t + k] = C::kOff - sub[nb][k]; z_s[warp][8 * nb + 2 * t + k] = z[nb][k]; }
            }
            if (any && !failed)
#pragma unroll
                for (int md = 0; md < D / 16; ++md)
                    mine[md * 32 + lane] = make_float4(acc[md][nb][0], acc[md][nb][1], acc[md][nb][2], acc[md][nb][3]);
            team_sync();
            // (all loads first: what this costs is latency)
            const int n = 8 * nb + 2 * t;
            float2 mw[W], zw[W];
            float refs[W], m[2] = {kNoMax, kNoMax}, zz[2] = {0.f, 0.f};
            const float4* frags[W];
#pragma unroll
            for (int w = 0; w < W; ++w) {
                mw[w] = *reinterpret_cast<const float2*>(&m_s[w][n]);
                zw[w] = *reinterpret_cast<const float2*>(&z_s[w][n]);
                refs[w] = (w >> work.team_shift) == team_no ? v_ref_s[w] : -1.f;
                if ((w >> work.team_shift) != team_no) { mw[w] = make_float2(kNoMax, kNoMax); zw[w] = make_float2(0.f, 0.f); }
                frags[w] = reinterpret_cast<const float4*>(ring + (w * kStages + held_s[w]) * kStageBytes) + lane;
                m[0] = fmaxf(m[0], mw[w].x); m[1] = fmaxf(m[1], mw[w].y);
            }
#pragma unroll
            for (int w = 0; w < W; ++w) {                     // (the maxima are whole numbers)
                mw[w] = make_float2(fast_exp2(mw[w].x - m[0]) * C::kUnOff, fast_exp2(mw[w].y - m[1]) * C::kUnOff);
                zz[0] += zw[w].x * mw[w].x; zz[1] += zw[w].y * mw[w].y;
                mw[w].x *= refs[w]; mw[w].y *= refs[w];
            }
            if (lost) zz[0] = zz[1] = NAN;
            constexpr int kMost = D / 16 / C::kMinTeam;
            float4 o[kMost];
#pragma unroll
            for (int i = 0; i < kMost; ++i) {
                const int md = member + i * team;
                o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (md >= D / 16) continue;
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    if (refs[w] < 0.f) continue;
                    const float4 x = frags[w][md * 32];
                    o[i].x += x.x * mw[w].x; o[i].y += x.y * mw[w].y; o[i].z += x.z * mw[w].x; o[i].w += x.w * mw[w].y;
                }
            }
            if (whole) {
                OutRows<T, D, INT8> rows(prm, b, h, 8 * NB, nb, lane);
                rows.sums(prm, m, zz, member == 0 && g == 0);
#pragma unroll
                for (int i = 0; i < kMost; ++i)
                    if (member + i * team < D / 16) rows.store(member + i * team, lane, o[i]);
            } else {
                float4* part = prm.part_o + (static_cast<int64_t>(slot) * NB + nb) * C::kFrag + lane;
#pragma unroll
                for (int i = 0; i < kMost; ++i)
                    if (member + i * team < D / 16) part[(member + i * team) * 32] = o[i];
                if (member == 0 && g == 0) *reinterpret_cast<float4*>(prm.part_mz + slot * (8 * NB) + n) = make_float4(m[0], zz[0], m[1], zz[1]);
            }
            if (nb == NB - 1) ptx::fence_proxy_async_smem();  // the stages go back to the copies
            team_sync();
        }
        if (any && !failed) fire();
    }
    if (taken < issued) {
        // a wait ran out: the copies that are still on the way land before the shared memory is given back
        for (int i = taken; i < issued; ++i) {
            if (i == prm.drop_chunk) continue;
            for (int spin = 0; spin < (1 << 16); ++spin)
                if (ptx::mbar_try_wait(ptx::smem_u32(&full_bar[warp][i % kStages]), (i / kStages) & 1)) break;
        }
        ptx::cp_async_wait_all();
    }
}

// Joins the parts of the rows that several workers shared.  A job (row, s, w, n) names slot s and the first slots of n workers
// from w on.  (A kernel of its own, whose launch overlaps the step: the last CTA of a row joining it at its end, found by a
// counter or by words that the others set, waits for fences and atomics longer than a grid does for its predecessor: measured
// together, one sequence of 500 keys 6.6 us so, 11.0 and 9.0 that way, 8 x 32 K 98, 104, 104.)  What bounds it is the round trips: the parts
// are loaded kJoinAtOnce at a time.  A row of up to twice as many has a warp for every fragment; the parts of others are shared
// out over the warps, fragment by fragment (by a block each where rows are few).
constexpr int kJoinAtOnce = 8;
struct Part {
    float4 o, mz;                   // sums; maximum and sum of column 2 t, of column 2 t + 1
};
// (maxima are whole numbers, so the weights are exact)
template <int N>
__device__ __forceinline__ Part join_parts(const Part (&p)[N]) {
    Part r;
    r.mz = make_float4(kNoMax, 0.f, kNoMax, 0.f);
    r.o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < N; ++i) { r.mz.x = fmaxf(r.mz.x, p[i].mz.x); r.mz.z = fmaxf(r.mz.z, p[i].mz.z); }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float f0 = fast_exp2(p[i].mz.x - r.mz.x), f1 = fast_exp2(p[i].mz.z - r.mz.z);
        r.mz.y += p[i].mz.y * f0; r.mz.w += p[i].mz.w * f1;
        r.o.x += p[i].o.x * f0; r.o.y += p[i].o.y * f1; r.o.z += p[i].o.z * f0; r.o.w += p[i].o.w * f1;
    }
    return r;
}
template <class T, int D, bool INT8, int NB, int WARPS>
__global__ void __launch_bounds__(32 * WARPS)
paged_join_kernel(const PagedDecodeParams prm) {
    using C = Cfg<T, D, INT8, NB>;
    __shared__ Part part_s[WARPS][32];
    ptx::griddep_wait();
    ptx::griddep_launch_dependents();
    const int4 job = __ldcg(prm.join + blockIdx.x);
    // (a job that no part of the step wrote, see length_of, is what the workspace held)
    if (static_cast<unsigned>(job.x) >= static_cast<unsigned>(prm.c.B * prm.HG) || static_cast<unsigned>(job.w) > static_cast<unsigned>(prm.workers) ||
        static_cast<unsigned>(job.z) > static_cast<unsigned>(prm.workers - job.w) || static_cast<unsigned>(job.y) >= 2u * prm.workers)
        return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, t = lane & 3, parts = job.w + 1;
    constexpr int F = (D / 16) * NB;
    const int f_begin = blockIdx.y * F / gridDim.y, f_end = (blockIdx.y + 1) * F / gridDim.y;
    // parts first, first + step, ... of fragment f = nb D / 16 + md
    auto take = [&](int f, int first, int step) -> Part {
        const int nb = f / (D / 16);
        Part sum;
        for (int i0 = first;; i0 += step * kJoinAtOnce) {
            Part p[kJoinAtOnce + 1];
#pragma unroll
            for (int j = 0; j < kJoinAtOnce; ++j) {
                const int i = i0 + j * step;
                p[j].mz = make_float4(kNoMax, 0.f, kNoMax, 0.f);
                p[j].o = make_float4(0.f, 0.f, 0.f, 0.f);
                if (i >= parts) continue;
                const int64_t slot = i == 0 ? job.y : 2 * (job.z + i - 1);
                p[j].o = __ldcg(prm.part_o + slot * (NB * C::kFrag) + f * 32 + lane);
                p[j].mz = __ldcg(reinterpret_cast<const float4*>(prm.part_mz + slot * (8 * NB) + 8 * nb + 2 * t));
            }
            if (i0 == first) { p[kJoinAtOnce].o = make_float4(0.f, 0.f, 0.f, 0.f); p[kJoinAtOnce].mz = make_float4(kNoMax, 0.f, kNoMax, 0.f); }
            else p[kJoinAtOnce] = sum;
            sum = join_parts(p);
            if (i0 + step * kJoinAtOnce >= parts) return sum;
        }
    };
    const int b = job.x / prm.HG, h = job.x - b * prm.HG;
    auto finish = [&](int f, const Part& p) {
        const int nb = f / (D / 16), md = f % (D / 16);
        OutRows<T, D, INT8> rows(prm, b, h, 8 * NB, nb, lane);
        const float m[2] = {p.mz.x, p.mz.z}, z[2] = {p.mz.y, p.mz.w};
        rows.sums(prm, m, z, md == 0 && lane < 4);
        rows.store(md, lane, p.o);
    };
    if (parts <= 2 * kJoinAtOnce) {
        for (int f = f_begin + warp; f < f_end; f += WARPS) finish(f, take(f, 0, 1));
        return;
    }
    for (int f = f_begin; f < f_end; ++f) {
        part_s[warp][lane] = take(f, warp, WARPS);
        __syncthreads();
        if (warp == 0) {
            Part p[WARPS];
#pragma unroll
            for (int w = 0; w < WARPS; ++w) p[w] = part_s[w][lane];
            finish(f, join_parts(p));
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------------------------------- host

// Shape of a launch by instance: what resolve_decode has to know of Cfg.
struct Plan {
    int NB, groups, HG, wave, ctas, jobs, splits;      // splits: whether a row can have more units than one
    int workers;                                 // workers that there may be
    size_t join_bytes, mz_bytes, total;
};

int resolve_decode(const tilemix_paged_t* p, int heads_q, PagedCache* c, Plan* plan) {
    const int rc = resolve_paged(p, c);
    if (rc) return rc;
    if (heads_q <= 0 || heads_q % p->heads_kv != 0) return TILEMIX_ERR_SHAPE;
    const int R = heads_q / p->heads_kv;
    // Eight query heads of a KV head share a read of the cache, or sixteen (two rows of eight instead: 1 x 128K keys, sixteen
    // heads 27.4 -> 31.5 us, 16 x 4K INT8 27.3 -> 32.6, BF16 37.0 -> 47.4).
    plan->NB = R > 8 ? 2 : 1;
    plan->groups = static_cast<int>(ceil_div(R, 8 * plan->NB));
    int W, ch, min_team, wave;
    auto shape = [&](auto cfg) {
        using C = decltype(cfg);
        W = C::W; ch = C::CH; min_team = C::kMinTeam; wave = C::kCtasPerSm * kSms;
    };
    const bool int8 = p->cache_type == TILEMIX_CACHE_INT8;
    if (p->head_dim == 128) {
        if (int8) { if (plan->NB == 1) shape(Cfg<__half, 128, true, 1>()); else shape(Cfg<__half, 128, true, 2>()); }
        else { if (plan->NB == 1) shape(Cfg<__half, 128, false, 1>()); else shape(Cfg<__half, 128, false, 2>()); }
    } else {
        if (int8) { if (plan->NB == 1) shape(Cfg<__half, 64, true, 1>()); else shape(Cfg<__half, 64, true, 2>()); }
        else { if (plan->NB == 1) shape(Cfg<__half, 64, false, 1>()); else shape(Cfg<__half, 64, false, 2>()); }
    }
    const int64_t rows_each = static_cast<int64_t>(p->heads_kv) * plan->groups;
    if (rows_each > (1 << 22)) return TILEMIX_ERR_SHAPE;
    const int64_t rows = rows_each * p->batch;
    if (rows > (1 << 28) || rows * ceil_div(c->capacity, 16) > (int64_t{1} << 30)) return TILEMIX_ERR_SHAPE;   // (units are counted in 32 bits)
    if (static_cast<int64_t>(p->batch) * heads_q > (int64_t{1} << 30)) return TILEMIX_ERR_SHAPE;
    plan->HG = static_cast<int>(rows_each);
    const int64_t units = rows * ceil_div(c->capacity, 16 * W);       // (the kernel makes chunks as small as 16 keys)
    plan->wave = static_cast<int>(units < wave ? units : wave);
    // blocks behind the first wave, see find_work (which sees the lengths: where shares are short, they return at once)
    const bool pieces = !int8 && rows * (c->capacity / (ch * W)) >= static_cast<int64_t>(kLongShare) * wave;
    plan->ctas = pieces ? 2 * wave : plan->wave;
    plan->splits = c->capacity > 16 * min_team;
    plan->workers = plan->wave * (W / min_team);         // (at least as many as CTAs)
    plan->jobs = static_cast<int>(rows < plan->workers ? rows : plan->workers);
    plan->join_bytes = (plan->jobs * sizeof(int4) + 255) / 256 * 256;
    plan->mz_bytes = (static_cast<size_t>(plan->workers) * 2 * 8 * plan->NB * sizeof(float2) + 255) / 256 * 256;
    plan->total = plan->join_bytes + plan->mz_bytes + static_cast<size_t>(plan->workers) * 2 * p->head_dim * 8 * plan->NB * sizeof(float);
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
    PoolMaps maps;
    const int page = 1 << c.page_shift, box_rows = page < C::CH ? page : C::CH;
    int rc;
    if ((rc = encode_pool_map(&maps.k, c.k_pool, C::kElt, D, page, c.Hk, c.n_pages, c.ks, box_rows))) return rc;
    if ((rc = encode_pool_map(&maps.v, c.v_pool, C::kElt, D, page, c.Hk, c.n_pages, c.vs, box_rows))) return rc;
    maps.k16 = maps.k; maps.v16 = maps.v;
    if (box_rows > 16) {
        if ((rc = encode_pool_map(&maps.k16, c.k_pool, C::kElt, D, page, c.Hk, c.n_pages, c.ks, 16))) return rc;
        if ((rc = encode_pool_map(&maps.v16, c.v_pool, C::kElt, D, page, c.Hk, c.n_pages, c.vs, 16))) return rc;
    }
    auto kernel = paged_decode_kernel<T, D, INT8, NB>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmemBytes);
    if (e != cudaSuccess) return static_cast<int>(e);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(plan.ctas); cfg.blockDim = dim3(C::kThreads); cfg.dynamicSmemBytes = C::kSmemBytes; cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, kernel, prm, maps);
    g_launch_count.fetch_add(1);
    if (e != cudaSuccess || !plan.splits) return static_cast<int>(e);
    // few rows: many parts each, a block of sixteen warps for a fragment; otherwise the parts of a row go at once, to the
    // warps of two blocks (64 rows of seven parts: 1.5 us so, 7 in large blocks, which an SM holds one of).  (Whole calls, us,
    // large blocks up to 55 rows (36 with sixteen query heads) / never / up to 110 (73): 1 x 128K INT8, 2 rows 27.1 / 45.1 / 27.2,
    // 1 x 8000, 8 rows 12.5 / 17.8 / 12.5, 2 x 32K, 16 rows 35.3 / 37.3 / 35.3, 4 x 20K BF16, 32 rows 62.4 / 61.2 / 62.3, 4 x 2K,
    // 32 rows 14.1 / 12.1 / 14.1, 8 x 32K, 64 rows 97.2 / 97.3 / 101.7, 12 x 2K FP16, 96 rows 24.9 / 24.9 / 31.3.)
    const bool few = prm.jobs_by_row && static_cast<int64_t>(plan.jobs) * kJoinAtOnce < plan.wave;
    constexpr int kFew = 16, kMany = 4, F = (D / 16) * NB;
    cfg.gridDim = dim3(plan.jobs, few ? F : F / kMany); cfg.blockDim = dim3(32 * (few ? kFew : kMany)); cfg.dynamicSmemBytes = 0;
    e = few ? cudaLaunchKernelEx(&cfg, paged_join_kernel<T, D, INT8, NB, kFew>, prm) : cudaLaunchKernelEx(&cfg, paged_join_kernel<T, D, INT8, NB, kMany>, prm);
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
    if (!aligned16(q) || !aligned16(out) || !aligned16(workspace) || (reinterpret_cast<uintptr_t>(lse) & 3u) != 0) return TILEMIX_ERR_ALIGN;
    if ((rc = row_strides(q_stride, p->batch, heads_q, p->head_dim, false, prm.qs))) return rc;
    if ((rc = row_strides(out_stride, p->batch, heads_q, p->head_dim, true, prm.os))) return rc;
    if (workspace_bytes < plan.total) return TILEMIX_ERR_WORKSPACE;
    prm.wave = plan.wave; prm.jobs = plan.jobs; prm.workers = plan.workers;
    prm.Hq = heads_q; prm.R = heads_q / p->heads_kv; prm.groups = plan.groups; prm.HG = plan.HG;
    prm.scale_log2 = (softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf(static_cast<float>(p->head_dim))) * kLog2e;
    prm.q = static_cast<const uint8_t*>(q);
    prm.out = static_cast<uint8_t*>(out);
    prm.lse = lse;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    prm.join = reinterpret_cast<int4*>(ws);
    prm.part_mz = reinterpret_cast<float2*>(ws + plan.join_bytes);
    prm.part_o = reinterpret_cast<float4*>(ws + plan.join_bytes + plan.mz_bytes);
    prm.jobs_by_row = static_cast<int64_t>(plan.HG) * p->batch <= plan.workers ? 1 : 0;
    prm.wait_limit_ns = g_wait_limit_ns.load();
    const int drop = g_test_drop.load();
    prm.drop_chunk = drop == 2 ? 1 : -1;
    prm.skew = drop == 4 ? 16 : drop == 5 ? 4096 : 0;
    prm.skew_copies = drop == 6 ? 4096 : drop == 7 ? -4096 : 0;
    const bool int8 = p->cache_type == TILEMIX_CACHE_INT8;
    Launch go;
    if (p->act_type == TILEMIX_TYPE_FP16) go = p->head_dim == 128 ? pick<__half, 128>(int8, plan.NB) : pick<__half, 64>(int8, plan.NB);
    else go = p->head_dim == 128 ? pick<__nv_bfloat16, 128>(int8, plan.NB) : pick<__nv_bfloat16, 64>(int8, plan.NB);
    return go(prm, plan, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
