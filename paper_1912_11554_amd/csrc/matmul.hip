// Matrix products of the token-model operators on the matrix cores, with their
// epilogues; the pass over a gradient's inputs before them.
//
// C(m, n) = sum over the terms of sum_k A(m, k) B(n, k).  A workgroup has a
// BM x BN tile of C, its waves WR x WC rectangles of it, each as 16 x 16
// blocks of v_mfma_f32_16x16x32_bf16 (lane l gives A[l % 16][8 (l / 16) + i],
// i < 8, likewise B, and holds D[4 (l / 16) + i][l % 16], i < 4).  B goes in as
// the instruction's first factor, so a lane holds four consecutive columns of
// one row of C.
//
// bf16 operands: 64 k of both at a time lie in one of two LDS stages, copied
// there straight from memory, 16 bytes a lane, while the other stage is
// multiplied.  fp32 operands and rows off the 16-byte grid go through registers.
#include "token.h"
#include "token_device.h"

namespace nuts {
namespace token {
namespace {

struct KernelArgs {
    int64_t M, N;
    int K;
    int steps;        // stages of one term
    int nterms;
    int small_stages; // so many stages at the start are of terms of corrections
    int tiles_m, tiles_n;
    int slices;       // the stages of all terms in so many runs (split sums)
    int64_t ldp;
    float* partials;  // [set][slice][gated 2][M][ldp], with slices > 1
    Term terms[2][kMaxTerms];
    Epilogue epi[2];
};
// The arguments are read where they lie: an index into a copy of the terms
// would put the copy into scratch memory.
typedef __attribute__((address_space(4))) const KernelArgs ConstArgs;
__device__ __forceinline__ const ConstArgs& const_args() { return *(ConstArgs*)__builtin_amdgcn_kernarg_segment_ptr(); }

// (field by field: a copy through a generic pointer would be vector loads, made
// again after every store)
__device__ __forceinline__ Epilogue epilogue_of(const ConstArgs& p, int set)
{
    const __attribute__((address_space(4))) Epilogue& q = p.epi[set];
    return {q.out, q.ldo, q.bias, q.res, q.ldr, q.pre, q.act, q.dtype};
}

// ---------------------------------------------------------------------------
// Copies to LDS.  The destination is the wave's LDS address in m0 plus 16 bytes
// a lane; the address is a uniform base plus 32 bits a lane.  Issued without
// the compiler's knowledge: meet() publishes them.  (Five wait states lie between a vector instruction that writes a
// scalar register, which may just have reloaded the address, and a memory
// instruction that reads it.)
__device__ __forceinline__ void copy16(uint32_t lds_at, const char* base, uint32_t offset)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2"
                 :
                 : "s"(lds_at), "v"(offset), "s"(base)
                 : "memory");
}
// This wave's copies have landed and its reads of LDS are done; so are all of the
// workgroup's.
__device__ __forceinline__ void meet() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
__device__ __forceinline__ uint32_t lds_address(const void* p)
{
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p;
}

// A stage's operand in LDS: R rows by KS k of bf16.
//
// k contiguous: KS / 8 slots of 16 bytes a row; slot s of row r holds the row's
// k-chunk s ^ swap(r): a read of one chunk of 16 rows then touches each of the
// 64 banks once per 16 lanes.
//
// Rows contiguous: 2 R bytes a k.  The 32-byte unit u of k holds unit
// u ^ swap(k): the transposing read of 16 rows at 16 k (four k in each of four
// groups) touches each bank twice per 64 lanes, the least there is.
template <int R, int KS, bool ROWS>
struct Tile {
    static constexpr int kBytes = R * KS * 2;
    static constexpr int kPer = ROWS ? R / 8 : KS / 8;  // 16-byte pieces of a k (of a row)
    static_assert(kPer >= (ROWS ? 8 : 4), "the swaps stay inside a k (a row)");

    __device__ __forceinline__ static int swap(int at)
    {
        if constexpr (ROWS && kPer >= 16) {
            return (at & 3) | ((at >> 1) & 4);
        } else if constexpr (ROWS) {  // (two k in 256 bytes: four units each)
            return ((at >> 1) & 1) | ((at >> 2) & 2);
        } else {
            const int rr = (at & 15) / (16 / kPer), middle = ((at >> 2) ^ (at >> 3)) & 1;  // (rows 4 .. 11)
            return (((rr & (kPer / 2 - 1)) << 1) | (rr / (kPer / 2))) ^ middle;
        }
    }
    // What slot s of k (of row) `at` holds, in pieces; its own inverse.
    __device__ __forceinline__ static int piece(int at, int s)
    {
        if constexpr (ROWS) return (((s >> 1) ^ swap(at)) << 1) | (s & 1);
        else return s ^ swap(at);
    }

    // The 16 x 32 block of rows r0 .. and k = 32 kk .. as a factor of the instruction.
    __device__ __forceinline__ static v8bf fragment(const char* tile, int r0, int kk, int lane)
    {
        if constexpr (ROWS) {
            typedef int16_t v4i16 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) v4i16 lds_v4;
            const int i = lane & 15, k = kk * 32 + 8 * (lane >> 4) + (i >> 2);
            // (k and k + 4 have one swap)
            const uint32_t at = lds_address(tile) + k * (R * 2) + (((r0 >> 4) ^ swap(k)) << 5) + (i & 3) * 8;
            union {
                v4i16 h[2];
                v8bf v;
            } u;
            u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4*)(uintptr_t)at);
            u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4*)(uintptr_t)(at + 4 * (R * 2)));
            return u.v;
        } else {
            const int r = r0 + (lane & 15), chunk = kk * 4 + (lane >> 4);
            return *(const v8bf*)(tile + r * (KS * 2) + (piece(r, chunk) << 4));
        }
    }
};
// Gated: G rows of the second operand's tile are a wave's, half of them the first
// factor's, half the second's for the same columns of the output: row `at` is
// this column of the tile's, of the second factor if at & G / 2.
template <int G>
__device__ __forceinline__ int gated_row(int at)
{
    return (at / G) * (G / 2) + at % (G / 2);
}

// A sum of corrections, held to the finite range.  Where a factor is infinite
// or a product leaves the fp32 range, the leading products (at least 64 times
// the corrections) hold the infinity or NaN that the fp32 product has, and the
// corrections hold inf - inf and inf * 0: a NaN becomes -2^122 here, which no
// infinity and no NaN notices, nor in the sum of kMaxSlices slices.  Corrections are
// the lower parts of fp32 factors and the terms of a bf16 dz's second part.
__device__ __forceinline__ v4f finite(v4f c)
{
    constexpr float big = 0x1p122f;
#pragma unroll
    for (int r = 0; r < 4; ++r) c[r] = __builtin_amdgcn_fmed3f(c[r], -big, big);
    return c;
}

// W consecutive elements (4 or 8) of an array of either type, `count` of them
// there.
template <int W>
__device__ __forceinline__ void load_run(const void* base, int dtype, int64_t at, int count, float (&v)[W])
{
    const char* p = (const char*)base + at * (dtype == NUTS_BF16 ? 2 : 4);
    if (count == W && dtype == NUTS_F32) {
#pragma unroll
        for (int i = 0; i < W; i += 4) {
            const v4u t = load16(p + i * 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i + j] = __uint_as_float(t[j]);
        }
    } else if (count == W && W == 8) {
        float t[8];
        unpack<__bf16>(load16(p), t);
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = t[i];
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = i < count ? load_as_f32(p, dtype, i) : 0.0f;
    }
}
template <int W>
__device__ __forceinline__ void store_run(void* base, int dtype, int64_t at, int count, const float (&v)[W])
{
    char* p = (char*)base + at * (dtype == NUTS_BF16 ? 2 : 4);
    if (count == W && dtype == NUTS_F32) {
#pragma unroll
        for (int i = 0; i < W; i += 4)
            store16(p + i * 4, v4u{__float_as_uint(v[i]), __float_as_uint(v[i + 1]), __float_as_uint(v[i + 2]),
                                   __float_as_uint(v[i + 3])});
    } else if (count == W && W == 8) {
        float t[8];
#pragma unroll
        for (int i = 0; i < W; ++i) t[i] = v[i];
        store16(p, pack<__bf16>(t));
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i)
            if (i < count) store_f32(p, dtype, i, v[i]);
    }
}

// The outputs n .. n + W - 1 of row m.
template <bool GATED, int W>
__device__ __forceinline__ void finish(const Epilogue& e, int64_t M, int64_t N, int64_t m, int64_t n, float (&z)[W],
                                       const float (&u)[W])
{
    const int count = N - n < W ? (int)(N - n) : W;
    if (e.bias) {
        float b[W];
        load_run<W>(e.bias, e.dtype, n, count, b);
#pragma unroll
        for (int i = 0; i < W; ++i) z[i] += b[i];
    }
    if (e.pre) {
        store_run<W>(e.pre, NUTS_F32, m * N + n, count, z);
        if constexpr (GATED) store_run<W>(e.pre, NUTS_F32, (M + m) * N + n, count, u);
    }
    if (e.act != NUTS_ACT_NONE) {
#pragma unroll
        for (int i = 0; i < W; ++i) z[i] = activate(z[i], e.act);
    }
    if constexpr (GATED) {
#pragma unroll
        for (int i = 0; i < W; ++i) z[i] *= u[i];
    }
    if (e.res) {
        float r[W];
        load_run<W>(e.res, e.dtype, m * e.ldr + n, count, r);
#pragma unroll
        for (int i = 0; i < W; ++i) z[i] += r[i];
    }
    store_run<W>(e.out, e.dtype, m * e.ldo + n, count, z);
}

// A wave's rectangle of C through LDS, AT blocks of 16 rows at a time: a lane
// there gets eight consecutive columns, so rows leave in runs of 64 bytes and
// more.  The blocks move down the registers as they are done, which keeps one
// copy of this code.  Chunk c (four floats) of row r lies at c ^ r: 16 rows at one
// column touch all banks.
template <int FN, int AT>
constexpr int kOutBytes = AT * 16 * FN * 16 * 4;
template <int FM, int FN, int AT, bool GATED>
__device__ __forceinline__ void write_out(const ConstArgs& p, int set, int64_t m0, int64_t n0, int lane, char* rows,
                                          v4f (&acc)[FM][FN])
{
    constexpr int kCols = GATED ? FN * 8 : FN * 16, kRuns = kCols / 8;  // of a row of the output
    constexpr int kAtOnce = 64 / kRuns;                                 // rows of a wave's store
    static_assert(FM % AT == 0 && AT * 16 % kAtOnce == 0, "whole passes");
    const Epilogue e = epilogue_of(p, set);
    const int64_t M = p.M, N = p.N, ldp = p.ldp, plane = M * ldp;
    float* part = nullptr;
    if (p.slices > 1) part = p.partials + ((int64_t)set * p.slices + blockIdx.y) * (GATED ? 2 : 1) * plane;
    auto place = [&](int r, int c) -> v4f* { return (v4f*)(rows + r * (FN * 64) + ((c ^ (r & (FN * 4 - 1))) << 4)); };
    const int c = lane % kRuns * 8;
    const int64_t n = n0 + c;
#pragma nounroll
    for (int i = 0; i < FM; i += AT) {
#pragma unroll
        for (int k = 0; k < AT; ++k)
#pragma unroll
            for (int j = 0; j < FN; ++j) *place(k * 16 + (lane & 15), j * 4 + (lane >> 4)) = acc[k][j];
        wave_sync();
#pragma nounroll
        for (int r = lane / kRuns; r < AT * 16; r += kAtOnce) {
            const int64_t m = m0 + i * 16 + r;
            if (m >= M || n >= N) continue;
            float z[8], u[8];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const v4f a = *place(r, c / 4 + q);
                v4f b = {0.0f, 0.0f, 0.0f, 0.0f};
                if constexpr (GATED) b = *place(r, kCols / 4 + c / 4 + q);
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    z[q * 4 + t] = a[t];
                    u[q * 4 + t] = b[t];
                }
            }
            if (part) {
                // (rows are padded to whole quads)
                const int count = ldp - n < 8 ? (int)(ldp - n) : 8;
                store_run<8>(part, NUTS_F32, m * ldp + n, count, z);
                if constexpr (GATED) store_run<8>(part, NUTS_F32, plane + m * ldp + n, count, u);
            } else {
                finish<GATED, 8>(e, M, N, m, n, z, u);
            }
        }
        wave_sync();
#pragma unroll
        for (int k = 0; k + AT < FM; ++k)
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[k][j] = acc[k + AT][j];
    }
}

// Tile of workgroup `id`: the eight XCDs take workgroups in turn, so XCD x gets
// the x-th eighth of the tiles, in columns of `kBand` tile rows: the tiles that
// run on it together share their operands in its L2.
constexpr int kBand = 8;
__device__ __forceinline__ void tile_of(int id, int tiles_m, int tiles_n, int* tm, int* tn)
{
    const int total = tiles_m * tiles_n;
    const int each = total / 8, more = total % 8;
    const int x = id % 8, at = id / 8;
    int t = x * each + (x < more ? x : more) + at;
    const int band = t / (kBand * tiles_n);
    const int first = band * kBand;
    const int height = tiles_m - first < kBand ? tiles_m - first : kBand;
    t -= first * tiles_n;
    *tm = first + t % height;
    *tn = t / height;
}

// This workgroup's stages of all terms.
struct Run {
    int from, to;
};
__device__ __forceinline__ Run run_of(const ConstArgs& p)
{
    const int64_t all = (int64_t)p.steps * p.nterms;
    return {(int)(all * blockIdx.y / p.slices), (int)(all * (blockIdx.y + 1) / p.slices)};
}
// The run's stage, counted from one, after which its sums are of corrections alone and
// done with them (0: it has none).
__device__ __forceinline__ int small_end(const ConstArgs& p, Run run)
{
    const int end = p.small_stages < run.to ? p.small_stages : run.to;
    return end > run.from ? end - run.from : 0;
}

// ---------------------------------------------------------------------------
// bf16 operands of 16-byte aligned rows of a whole multiple of 8 elements,
// copied as they lie.
//
// 2 M N K operations on matrix cores.  A 256 x 256 tile by 8 waves (128 x 64 each,
// 128 fp32 sums a lane) takes 64 KB for 64 k; the copies alone need 0.95 us a stage,
// the reads of LDS alone 0.42, the products without copies 0.8 to 0.9: the copies
// bound it, then the clock that the products leave.  Normally distributed inputs, on
// several cards: 8192 x 2048 x 8192 274 to 286 us (1.00 to 0.96 PFLOP/s), its gradients
// 288 to 296 and 267 to 270 us; the gated pair 8192 x 24,576 x 4096 1340 to 1400 us
// (1.23 to 1.18); gradients of 4096 x 8192 x 4096, two terms or two sets of two parts,
// 906 to 914 and 944 to 950 us (1.21 and 1.16).  The epilogue adds 8 us for each
// round of tiles, the rate at which memory takes the results.  128 x 128 and 64 x 64
// tiles are for products with few tiles.
// Tried, and slower or equal: 32 k a stage with three to five stages (7 to 10%
// slower), four waves of 128 x 128 (10%), copies spread over the groups or staggered by
// wave (within 3%), two groups of waves taking copies and products in turn (equal),
// copies through registers (half the speed), other wave priorities (equal).
template <int BM, int BN, int WR, int WC, bool AROWS, bool BROWS, bool GATED>
__global__ __launch_bounds__(64 * WR * WC, 2) void product_kernel(KernelArgs)
{
    constexpr int T = 64 * WR * WC;
    constexpr int FM = BM / WR / 16, FN = BN / WC / 16;
    using TA = Tile<BM, kStep, AROWS>;
    using TB = Tile<BN, kStep, BROWS>;
    constexpr int AT = FM < 4 ? FM : 4;  // blocks of a pass through LDS at the end
    constexpr int G = BN / WC;  // columns of a wave (gated: half of them of each factor)
    constexpr int kStageBytes = TA::kBytes + TB::kBytes;
    constexpr int kPassesA = TA::kBytes / (T * 16), kPassesB = TB::kBytes / (T * 16);
    constexpr int kRowsA = T / TA::kPer, kRowsB = T / TB::kPer;  // k or rows of a pass
    __shared__ __attribute__((aligned(1024))) char lds[2 * kStageBytes];
    static_assert(WR * WC * kOutBytes<FN, AT> <= 2 * kStageBytes, "the results pass through the stages' memory");

    const ConstArgs& p = const_args();
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wr = wave / WC, wc = wave % WC;
    const int set = blockIdx.z;
    int tm, tn;
    tile_of(blockIdx.x, p.tiles_m, p.tiles_n, &tm, &tn);
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * (GATED ? BN / 2 : BN);
    const Run run = run_of(p);

    v4f acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

    // Byte offset of this lane's piece in pass i from the operand's tile.
    auto offset_a = [&](int i, int64_t ld) -> uint32_t {
        const int at = i * kRowsA + tid / TA::kPer, piece = TA::piece(at, tid % TA::kPer);
        if constexpr (AROWS) {
            const int64_t last = (p.M + 7) / 8 - 1 - m0 / 8;
            return (uint32_t)(at * ld * 2 + (piece < last ? piece : last) * 16);
        } else {
            const int64_t r = m0 + at < p.M ? at : p.M - 1 - m0;
            return (uint32_t)(r * ld * 2 + piece * 16);
        }
    };
    auto offset_b = [&](int i, int64_t ld) -> uint32_t {
        const int at = i * kRowsB + tid / TB::kPer, piece = TB::piece(at, tid % TB::kPer);
        if constexpr (BROWS) {
            const int64_t last = (p.N + 7) / 8 - 1 - n0 / 8;
            return (uint32_t)(at * ld * 2 + (piece < last ? piece : last) * 16);
        } else {
            int64_t r = GATED ? gated_row<G>(at) : at;
            if (n0 + r >= p.N) r = p.N - 1 - n0;
            return (uint32_t)(r * ld * 2 + piece * 16);
        }
    };
    // First k of this lane's piece in pass i.
    auto k_a = [&](int i) {
        const int at = i * kRowsA + tid / TA::kPer;
        return AROWS ? at : 8 * TA::piece(at, tid % TA::kPer);
    };
    auto k_b = [&](int i) {
        const int at = i * kRowsB + tid / TB::kPer;
        return BROWS ? at : 8 * TB::piece(at, tid % TB::kPer);
    };
    // Gated: whether the rows that this wave copies in pass i are the second
    // factor's.
    auto second = [&](int i) -> bool {
        return GATED && __builtin_amdgcn_readfirstlane((i * kRowsB + tid / TB::kPer) & (G / 2));
    };

    // Copies the next stage of the run into LDS stage b.
    const uint32_t lds0 = lds_address(lds);
    int term = run.from < run.to ? run.from / p.steps : 0, step = run.from - term * p.steps;
    uint32_t aoff[kPassesA], boff[kPassesB];
    auto ldb = [&](int t, int i) { return second(i) ? p.terms[set][t].ldb2 : p.terms[set][t].ldb; };
    auto offsets = [&]() {
#pragma unroll
        for (int i = 0; i < kPassesA; ++i) aoff[i] = offset_a(i, p.terms[set][term].lda);
#pragma unroll
        for (int i = 0; i < kPassesB; ++i) boff[i] = offset_b(i, ldb(term, i));
    };
    auto copy_stage = [&](int b) {
        const __attribute__((address_space(4))) Term& q = p.terms[set][term];
        const int64_t k0 = (int64_t)step * kStep;
        const char* abase = (const char*)q.a + 2 * (AROWS ? k0 * q.lda + m0 : m0 * q.lda + k0);
        auto bbase = [&](int i) {
            const int64_t ld = ldb(term, i);
            return (const char*)(second(i) ? q.b2 : q.b) + 2 * (BROWS ? k0 * ld + n0 : n0 * ld + k0);
        };
        const int left = p.K - (int)k0;
        if (left >= kStep) {
            const uint32_t at = lds0 + b * kStageBytes + wave * 1024;
#pragma unroll
            for (int i = 0; i < kPassesA; ++i)
                copy16(__builtin_amdgcn_readfirstlane(at + i * T * 16), abase, aoff[i]);
#pragma unroll
            for (int i = 0; i < kPassesB; ++i)
                copy16(__builtin_amdgcn_readfirstlane(at + TA::kBytes + i * T * 16), bbase(i), boff[i]);
        } else {
            // the last k of a term: zeros past them
            char* dst = lds + b * kStageBytes + tid * 16;
            for (int i = 0; i < kPassesA; ++i) {
                v4u v = {0, 0, 0, 0};
                if (k_a(i) < left) v = *(const v4u*)(abase + offset_a(i, q.lda));
                *(v4u*)(dst + i * T * 16) = v;
            }
            for (int i = 0; i < kPassesB; ++i) {
                v4u v = {0, 0, 0, 0};
                if (k_b(i) < left) v = *(const v4u*)(bbase(i) + offset_b(i, ldb(term, i)));
                *(v4u*)(dst + TA::kBytes + i * T * 16) = v;
            }
        }
        if (++step == p.steps && term + 1 < p.nterms) {
            step = 0;
            ++term;
            offsets();
        }
    };

    // A stage is kGroups groups of FN products, (k half, block row) in turn.  A
    // group reads the factor that the group kAhead later takes, so that products
    // do not wait for LDS.  kAhead groups before the stage's end all of its
    // factors are in registers: there the waves meet, the next stage's copies have
    // landed, the one after it may be copied over this one, and the reads go on
    // in the next.
    constexpr int kGroups = 2 * FM, kAhead = FM > 2 ? 3 : 2, kRing = 4;
    static_assert(kGroups % kRing == 0 && kAhead < kRing, "the ring goes round a whole number of times a stage");
    static_assert(kStep == 64 && kGroups - kAhead >= FM, "the first half's columns are done with when the waves meet");
    v8bf fa[kRing], fb[2][FN];
    const int stages = run.to - run.from, small = small_end(p, run);
    if (stages > 0) {
        offsets();
        copy_stage(0);
        meet();
        if (stages > 1) copy_stage(1);
#pragma unroll
        for (int j = 0; j < FN; ++j) fb[0][j] = TB::fragment(lds + TA::kBytes, (wc * FN + j) * 16, 0, lane);
#pragma unroll
        for (int g = 0; g < kAhead; ++g) fa[g] = TA::fragment(lds, (wr * FM + g % FM) * 16, g / FM, lane);
    }
    for (int s = 0; s < stages; ++s) {
        const char* here = lds + (s & 1) * kStageBytes;
        const char* next = lds + (~s & 1) * kStageBytes;
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            constexpr int kMeet = kGroups - kAhead;
            const int kk = g / FM, ahead = (g + kAhead) % kGroups;
            if (g == kMeet && s + 1 < stages) {
                meet();
                if (s + 2 < stages) copy_stage(s & 1);
            }
            const char* from = g < kMeet ? here : next;
            // the second half's columns in its first groups, the next stage's with
            // its first rows
            if (g < FN && FM >= FN) {
                fb[1][g] = TB::fragment(here + TA::kBytes, (wc * FN + g) * 16, 1, lane);
            } else if (FM < FN && g < FM) {
#pragma unroll
                for (int j = g * FN / FM; j < (g + 1) * FN / FM; ++j)
                    fb[1][j] = TB::fragment(here + TA::kBytes, (wc * FN + j) * 16, 1, lane);
            }
            if (g >= kMeet && g < kMeet + 2) {
#pragma unroll
                for (int j = (g - kMeet) * FN / 2; j < (g - kMeet + 1) * FN / 2; ++j)
                    fb[0][j] = TB::fragment(next + TA::kBytes, (wc * FN + j) * 16, 0, lane);
            }
            fa[ahead % kRing] = TA::fragment(from, (wr * FM + ahead % FM) * 16, ahead / FM, lane);
#pragma unroll
            for (int j = 0; j < FN; ++j)
                acc[g % FM][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[kk][j], fa[g % kRing], acc[g % FM][j], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (s + 1 == small) {
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[i][j] = finite(acc[i][j]);
        }
    }
    __syncthreads();
    write_out<FM, FN, AT, GATED>(p, set, m0 + wr * FM * 16, n0 + wc * (GATED ? G / 2 : G), lane,
                                 lds + wave * kOutBytes<FN, AT>, acc);
}

// ---------------------------------------------------------------------------
// Operands of any alignment, fp32 or bf16, through registers.  An fp32 value
// goes into LDS as its three bf16 parts, and six products of them (those of
// relative size 2^-22 and below are left out) make the fp32 product: the
// leading ones in sums of their own, the other five in the corrections.
// Four waves have B / 2 x B / 2 of C each.
//
// fp32 in six bf16 products has a sixth of their rate at most, still above the fp32
// instructions': 4096^3 630 to 730 us (189 to 219 TFLOP/s; a library's fp32
// product 137), 8192 x 8192 x 4096 2.5 ms (217).  Cutting the parts (vector
// instructions) and the three parts' way through LDS bound it with the products.
// Small products wait: 1000 x 1027 x 513 21 us for 2.5 us of products at the bf16 rate,
// one 64 x 64 tile a unit and a chain of load, cut, LDS and product each 32 k; three
// stages are on their way to registers there.  Waves in groups of two or four that
// share out a small tile's k gained 12% at most and were not kept.
template <typename T>
constexpr int kStagedStep = sizeof(T) == 4 ? 32 : 64;

template <typename T, int B, bool AROWS, bool BROWS, bool GATED>
__global__ __launch_bounds__(256, B > 64 ? 2 : 3) void staged_kernel(KernelArgs)
{
    constexpr int KS = kStagedStep<T>, PARTS = sizeof(T) == 4 ? 3 : 1;
    constexpr int F = B / 32;  // 16 x 16 blocks of a wave, each way
    constexpr int AHEAD = B > 64 ? 1 : PARTS == 3 ? 3 : 2;  // stages on their way to registers
    using TA = Tile<B, KS, AROWS>;
    using TB = Tile<B, KS, BROWS>;
    constexpr int kPasses = B * KS / 8 / 256;
    __shared__ __attribute__((aligned(1024))) char lds[PARTS * (TA::kBytes + TB::kBytes)];
    static_assert(4 * kOutBytes<F, 2> <= (int)sizeof lds, "the results pass through the stage's memory");
    char* const lds_b = lds + PARTS * TA::kBytes;

    const ConstArgs& p = const_args();
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wr = wave / 2, wc = wave % 2;
    const int set = blockIdx.z;
    int tm, tn;
    tile_of(blockIdx.x, p.tiles_m, p.tiles_n, &tm, &tn);
    const int64_t m0 = (int64_t)tm * B, n0 = (int64_t)tn * (GATED ? B / 2 : B);
    const Run run = run_of(p);

    v4f acc[F][F], corr[PARTS == 3 ? F : 1][F];
#pragma unroll
    for (int i = 0; i < F; ++i) {
#pragma unroll
        for (int j = 0; j < F; ++j) {
            acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
            if (PARTS == 3) corr[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        }
    }

    struct Piece {
        alignas(16) T v[8];
    };
    Piece pieces[AHEAD][2][kPasses];
    // Eight elements from q, the first `count` of them there (any number), zeros
    // else.
    auto guarded = [&](const T* q, int64_t count, Piece& out) {
#pragma unroll
        for (int i = 0; i < 8; ++i) out.v[i] = i < count ? q[i] : (T)0.0f;
    };
    auto whole = [&](const char* base, uint32_t offset, Piece& out) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) * 8; i += 16) *(v4u*)((char*)out.v + i) = load16(base + offset + i);
    };
    // This lane's piece in pass i: its row (k contiguous, rows past the last repeat
    // it) or columns (rows contiguous, `cut` of which are there), and its byte offset
    // from the tile at the stage's first k.
    int term = 0, step = 0;
    uint32_t offa[kPasses], offb[kPasses];
    auto at_a = [&](int i) { return (i * 256 + tid) / TA::kPer; };
    auto at_b = [&](int i) { return (i * 256 + tid) / TB::kPer; };
    const int slot_a = tid % TA::kPer, slot_b = tid % TB::kPer;
    const int64_t cut_a = p.M - m0 - slot_a * 8, cut_b = p.N - n0 - slot_b * 8;
    auto second = [&](int i) { return GATED && (at_b(i) & (B / 4)); };
    auto row_a = [&](int i) -> int64_t { return m0 + at_a(i) < p.M ? at_a(i) : p.M - 1 - m0; };
    auto row_b = [&](int i) -> int64_t {
        const int64_t r = GATED ? gated_row<B / 2>(at_b(i)) : at_b(i);
        return n0 + r < p.N ? r : p.N - 1 - n0;
    };
    auto offsets = [&]() {
        const __attribute__((address_space(4))) Term& q = p.terms[set][term];
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            offa[i] = (uint32_t)((AROWS ? at_a(i) * q.lda + slot_a * 8 : row_a(i) * q.lda + slot_a * 8) * sizeof(T));
            const int64_t ldb = second(i) ? q.ldb2 : q.ldb;
            offb[i] = (uint32_t)((BROWS ? at_b(i) * ldb + slot_b * 8 : row_b(i) * ldb + slot_b * 8) * sizeof(T));
        }
    };
    if (run.from < run.to) {
        term = run.from / p.steps;
        step = run.from - term * p.steps;
        offsets();
    }
    // Takes the run's next stage on its way to registers.
    auto fetch_stage = [&](Piece (&two)[2][kPasses]) {
        const __attribute__((address_space(4))) Term& q = p.terms[set][term];
        const int64_t k0 = (int64_t)step * KS, left = p.K - k0;
        const char* a = (const char*)q.a + sizeof(T) * (AROWS ? k0 * q.lda + m0 : m0 * q.lda + k0);
        const char* b = (const char*)q.b + sizeof(T) * (BROWS ? k0 * q.ldb + n0 : n0 * q.ldb + k0);
        const char* b2 = GATED ? (const char*)q.b2 + sizeof(T) * (n0 * q.ldb2 + k0) : nullptr;
        if (left >= KS) {
#pragma unroll
            for (int i = 0; i < kPasses; ++i) {
                if (AROWS && cut_a < 8) guarded((const T*)(a + offa[i]), cut_a, two[0][i]);
                else whole(a, offa[i], two[0][i]);
            }
#pragma unroll
            for (int i = 0; i < kPasses; ++i) {
                if (BROWS && cut_b < 8) guarded((const T*)(b + offb[i]), cut_b, two[1][i]);
                else if (GATED) whole(second(i) ? b2 : b, offb[i], two[1][i]);
                else whole(b, offb[i], two[1][i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kPasses; ++i) {
                guarded((const T*)(a + offa[i]), AROWS ? (at_a(i) < left ? cut_a : 0) : left - slot_a * 8, two[0][i]);
                guarded((const T*)((second(i) ? b2 : b) + offb[i]),
                        BROWS ? (at_b(i) < left ? cut_b : 0) : left - slot_b * 8, two[1][i]);
            }
        }
        if (++step == p.steps && term + 1 < p.nterms) {
            step = 0;
            ++term;
            offsets();
        }
    };
    auto put = [&](char* tile, int bytes, const Piece& v, uint32_t at) {
        if constexpr (PARTS == 1) {
            *(v4u*)(tile + at) = *(const v4u*)v.v;
        } else {
            v4u part[3];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t two[3];
                parts3(v.v[2 * i], v.v[2 * i + 1], two);
#pragma unroll
                for (int q = 0; q < 3; ++q) part[q][i] = two[q];
            }
#pragma unroll
            for (int q = 0; q < 3; ++q) *(v4u*)(tile + q * bytes + at) = part[q];
        }
    };
    auto put_stage = [&](const Piece (&two)[2][kPasses]) {
        const Piece(&pa)[kPasses] = two[0], (&pb)[kPasses] = two[1];
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            const int at = (i * 256 + tid) / TA::kPer, slot = tid % TA::kPer;
            put(lds, TA::kBytes, pa[i], (at * TA::kPer + TA::piece(at, slot)) * 16);
        }
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            const int at = (i * 256 + tid) / TB::kPer, slot = tid % TB::kPer;
            put(lds_b, TB::kBytes, pb[i], (at * TB::kPer + TB::piece(at, slot)) * 16);
        }
    };

#pragma unroll
    for (int h = 0; h < AHEAD; ++h)
        if (run.from + h < run.to) fetch_stage(pieces[h]);
    const int small = small_end(p, run);
    for (int s = run.from; s < run.to; s += AHEAD) {
#pragma unroll
        for (int h = 0; h < AHEAD; ++h) {
            if (s + h >= run.to) break;
            put_stage(pieces[h]);
            __syncthreads();
            if (s + h + AHEAD < run.to) fetch_stage(pieces[h]);
#pragma unroll
            for (int kk = 0; kk < KS / 32; ++kk) {
                v8bf fb[F][PARTS];
#pragma unroll
                for (int j = 0; j < F; ++j)
#pragma unroll
                    for (int q = 0; q < PARTS; ++q)
                        fb[j][q] = TB::fragment(lds_b + q * TB::kBytes, (wc * F + j) * 16, kk, lane);
#pragma unroll
                for (int i = 0; i < F; ++i) {
                    v8bf fa[PARTS];
#pragma unroll
                    for (int q = 0; q < PARTS; ++q) fa[q] = TA::fragment(lds + q * TA::kBytes, (wr * F + i) * 16, kk, lane);
#pragma unroll
                    for (int j = 0; j < F; ++j) {
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[j][0], fa[0], acc[i][j], 0, 0, 0);
                        if constexpr (PARTS == 3) {
                            constexpr int order[5][2] = {{2, 0}, {1, 1}, {0, 2}, {1, 0}, {0, 1}};
#pragma unroll
                            for (int q = 0; q < 5; ++q)
                                corr[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[j][order[q][0]], fa[order[q][1]],
                                                                                     corr[i][j], 0, 0, 0);
                        }
                    }
                }
            }
            if (PARTS == 1 && s + h + 1 - run.from == small) {
#pragma unroll
                for (int i = 0; i < F; ++i)
#pragma unroll
                    for (int j = 0; j < F; ++j) acc[i][j] = finite(acc[i][j]);
            }
            __syncthreads();
        }
    }
    if constexpr (PARTS == 3) {
#pragma unroll
        for (int i = 0; i < F; ++i)
#pragma unroll
            for (int j = 0; j < F; ++j) acc[i][j] += finite(corr[i][j]);
    }
    write_out<F, F, 2, GATED>(p, set, m0 + wr * (B / 2), n0 + wc * (GATED ? B / 4 : B / 2), lane,
                              lds + wave * kOutBytes<F, 2>, acc);
}

// Sums of the slices in their order, and the epilogue.  Latency: four slices of 777 x
// 640 5 us.
template <bool GATED>
__global__ __launch_bounds__(256) void join_kernel(KernelArgs)
{
    const ConstArgs& p = const_args();
    const int set = blockIdx.z;
    const Epilogue e = epilogue_of(p, set);
    const int64_t quads = p.ldp / 4, plane = p.M * p.ldp, each = plane * (GATED ? 2 : 1);
    const float* part = p.partials + (int64_t)set * p.slices * each;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < p.M * quads; at += (int64_t)gridDim.x * 256) {
        const int64_t m = at / quads, n = at % quads * 4;
        const float* q = part + at * 4;
        v4f z = {0, 0, 0, 0}, u = {0, 0, 0, 0};
        for (int s = 0; s < p.slices; ++s, q += each) {
            z += *(const v4f*)q;
            if constexpr (GATED) u += *(const v4f*)(q + plane);
        }
        float zz[4], uu[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            zz[i] = z[i];
            uu[i] = u[i];
        }
        finish<GATED, 4>(e, p.M, p.N, m, n, zz, uu);
    }
}

template <int B, bool GATED, typename F>
hipError_t launch_tiles(KernelArgs& a, int sets, int threads, hipStream_t stream, F* kernel)
{
    constexpr int OUT_N = GATED ? B / 2 : B;
    a.tiles_m = (int)((a.M + B - 1) / B);
    a.tiles_n = (int)((a.N + OUT_N - 1) / OUT_N);
    const dim3 grid((unsigned)(a.tiles_m * (int64_t)a.tiles_n), (unsigned)a.slices, (unsigned)sets);
    kernel<<<grid, threads, 0, stream>>>(a);
    return hipGetLastError();
}
template <int B, int WR, int WC>
hipError_t launch_direct(const Product& p, KernelArgs& a, hipStream_t stream)
{
    constexpr int T = 64 * WR * WC;
    if (p.gated) return launch_tiles<B, true>(a, p.sets, T, stream, product_kernel<B, B, WR, WC, false, false, true>);
    if (p.a_rows) return launch_tiles<B, false>(a, p.sets, T, stream, product_kernel<B, B, WR, WC, true, true, false>);
    if (p.b_rows) return launch_tiles<B, false>(a, p.sets, T, stream, product_kernel<B, B, WR, WC, false, true, false>);
    return launch_tiles<B, false>(a, p.sets, T, stream, product_kernel<B, B, WR, WC, false, false, false>);
}
template <typename T, int B>
hipError_t launch_staged(const Product& p, KernelArgs& a, hipStream_t stream)
{
    if (p.gated) return launch_tiles<B, true>(a, p.sets, 256, stream, staged_kernel<T, B, false, false, true>);
    if (p.a_rows) return launch_tiles<B, false>(a, p.sets, 256, stream, staged_kernel<T, B, true, true, false>);
    if (p.b_rows) return launch_tiles<B, false>(a, p.sets, 256, stream, staged_kernel<T, B, false, true, false>);
    return launch_tiles<B, false>(a, p.sets, 256, stream, staged_kernel<T, B, false, false, false>);
}

}  // namespace

size_t product_workspace(const Product& p, int num_cu)
{
    const Plan plan = plan_product(p, num_cu);
    return plan.slices == 1 ? 0 : (size_t)p.M * up(p.N, 4) * (p.gated ? 2 : 1) * plan.slices * p.sets * sizeof(float);
}

hipError_t launch_product(const Product& p, float* partials, int num_cu, hipStream_t stream)
{
    if (p.M == 0 || p.N == 0) return hipSuccess;
    const Plan plan = plan_product(p, num_cu);
    KernelArgs a{};
    a.M = p.M;
    a.N = p.N;
    a.K = (int)p.K;
    a.steps = (int)steps_of(p);
    a.nterms = p.nterms;
    a.small_stages = p.small_terms * a.steps;
    a.slices = plan.slices;
    a.ldp = up(p.N, 4);
    a.partials = partials;
    for (int s = 0; s < p.sets; ++s) {
        for (int t = 0; t < p.nterms; ++t) a.terms[s][t] = p.terms[s][t];
        a.epi[s] = p.epi[s];
    }
    hipError_t e;
    if (!p.staged)
        e = plan.tile == 256   ? launch_direct<256, 2, 4>(p, a, stream)
            : plan.tile == 128 ? launch_direct<128, 2, 2>(p, a, stream)
                               : launch_direct<64, 2, 2>(p, a, stream);
    else if (p.dtype == NUTS_F32)
        e = plan.tile == 128 ? launch_staged<float, 128>(p, a, stream) : launch_staged<float, 64>(p, a, stream);
    else
        e = plan.tile == 128 ? launch_staged<__bf16, 128>(p, a, stream) : launch_staged<__bf16, 64>(p, a, stream);
    if (e != hipSuccess || plan.slices == 1) return e;
    const int64_t quads = p.M * (a.ldp / 4);
    const dim3 grid(groups_of((quads + 255) / 256), 1, (unsigned)p.sets);
    if (p.gated) join_kernel<true><<<grid, 256, 0, stream>>>(a);
    else join_kernel<false><<<grid, 256, 0, stream>>>(a);
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// A few rows.  A workgroup has 16 rows of w; its waves share K out among them,
// kFewAhead loads of 16 bytes a lane in flight (a load: 32 k of 16 rows in bf16,
// 16 k in fp32).  Products on the matrix cores (16x16x32 bf16; 16x16x4 fp32, a
// lane's four consecutive k in four instructions), the waves' blocks summed
// through LDS in their order.  Rows past the matrix's end repeat its last one:
// a row of a factor reaches its own row of the block alone.
//
// Bound by the one read of w: one row by 4096 x 4096 bf16 9.2 us (33.5 MB, 3.6 TB/s, with
// 3 to 4 us of launch and first loads), four rows by the gated block's 2 x 8192 x 4096
// 25 us (5.4 TB/s), fp32 one row by 16,384 x 4096 53 us (5.1).  Eight loads in flight a
// lane gained nothing over four.
namespace {

constexpr int kFewAhead = 4;

template <typename T>
__device__ __forceinline__ v4f few_mfma(v4u w, v4u x, v4f c)
{
    if constexpr (sizeof(T) == 2) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, w), __builtin_bit_cast(v8bf, x), c, 0, 0, 0);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[i]), __uint_as_float(x[i]), c, 0, 0, 0);
        return c;
    }
}

// Elements k .. of a row, zeros from K on.
template <typename T>
__device__ __forceinline__ v4u load_end(const T* row, int64_t k, int64_t K)
{
    constexpr int n = 16 / sizeof(T);
    if (k + n <= K) return load16(row + k);
    alignas(16) T t[n];
#pragma unroll
    for (int i = 0; i < n; ++i) t[i] = k + i < K ? row[k + i] : (T)0.0f;
    return *(const v4u*)t;
}

// TILES blocks of 16 rows of x.
template <typename T, bool GATED, int TILES, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void few_rows_kernel(FewRows p)
{
    constexpr int n = 16 / sizeof(T), U = kFewAhead;
    __shared__ v4f part[GATED ? 2 : 1][TILES][WAVES][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t n0 = (int64_t)blockIdx.x * 16;
    const int r = lane & 15, g = lane >> 4;
    const int64_t wrow = n0 + r < p.N ? n0 + r : p.N - 1;
    const T* w = (const T*)p.w + wrow * p.ldw + g * n;
    const T* w2 = GATED ? (const T*)p.w2 + wrow * p.ldw2 + g * n : nullptr;
    const T* x[TILES];
    v4f z[TILES], u[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        const int64_t row = t * 16 + r < p.M ? t * 16 + r : p.M - 1;
        x[t] = (const T*)p.x + row * p.ldx + g * n;
        z[t] = u[t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    }
    const int64_t step = WAVES * U * 4 * n;
    int64_t k = wave * (U * 4 * n);
    for (; k + U * 4 * n <= p.K; k += step) {
        v4u a[U], b[TILES][U], c[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            a[i] = load16(w + k + i * 4 * n);
            if constexpr (GATED) c[i] = load16(w2 + k + i * 4 * n);
        }
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int i = 0; i < U; ++i) b[t][i] = load16(x[t] + k + i * 4 * n);
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
#pragma unroll
            for (int i = 0; i < U; ++i) {
                z[t] = few_mfma<T>(a[i], b[t][i], z[t]);
                if constexpr (GATED) u[t] = few_mfma<T>(c[i], b[t][i], u[t]);
            }
        }
    }
    for (const int64_t end = k + U * 4 * n; k < p.K && k < end; k += 4 * n) {
        const int64_t left = p.K - g * n;
        const v4u a = load_end(w, k, left);
        v4u c = {0, 0, 0, 0};
        if constexpr (GATED) c = load_end(w2, k, left);
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            const v4u b = load_end(x[t], k, left);
            z[t] = few_mfma<T>(a, b, z[t]);
            if constexpr (GATED) u[t] = few_mfma<T>(c, b, u[t]);
        }
    }
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        part[0][t][wave][lane] = z[t];
        if constexpr (GATED) part[1][t][wave][lane] = u[t];
    }
    __syncthreads();
    // wave t: the waves' sums of tile t
    if (wave >= TILES) return;
    v4f zs = {0, 0, 0, 0}, us = {0, 0, 0, 0};
#pragma unroll
    for (int v = 0; v < WAVES; ++v) {
        zs += part[0][wave][v][lane];
        if constexpr (GATED) us += part[1][wave][v][lane];
    }
    const int64_t m = wave * 16 + (lane & 15), nn = n0 + 4 * (lane >> 4);
    if (m < p.M && nn < p.N) {
        float zz[4], uu[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            zz[i] = zs[i];
            uu[i] = us[i];
        }
        finish<GATED, 4>(p.epi, p.M, p.N, m, nn, zz, uu);
    }
}

template <typename T, bool GATED>
void run_few_rows(const FewRows& p, hipStream_t stream)
{
    const unsigned grid = (unsigned)((p.N + 15) / 16);  // (N is below 2^23, as the stride of y)
    // 16 waves have the loads in flight that 8 with two factors have (bf16, one row by
    // 4096 x 4096: 9.5 us, 11.4 with 8 waves; gated, 4 by 14,336 x 4096: 46.7 us
    // with 8, 48.1 with 16)
    if (p.M <= 16) {
        constexpr int waves = GATED ? 8 : 16;
        few_rows_kernel<T, GATED, 1, waves><<<grid, waves * 64, 0, stream>>>(p);
    } else if (p.M <= 32) {
        few_rows_kernel<T, GATED, 2, 8><<<grid, 512, 0, stream>>>(p);
    } else {
        few_rows_kernel<T, GATED, 4, 8><<<grid, 512, 0, stream>>>(p);
    }
}

}  // namespace

hipError_t launch_few_rows(const FewRows& p, hipStream_t stream)
{
    if (p.M == 0 || p.N == 0) return hipSuccess;
    if (p.epi.dtype == NUTS_BF16) p.gated ? run_few_rows<__bf16, true>(p, stream) : run_few_rows<__bf16, false>(p, stream);
    else p.gated ? run_few_rows<float, true>(p, stream) : run_few_rows<float, false>(p, stream);
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// The pass before a gradient's products.  A workgroup has ROWS rows of 64
// x 8 columns: 4 waves take ROWS / 4 rows each, all of them in flight, a
// lane eight columns; with dbias, sums over its rows by wave, then over the
// waves, and a second kernel adds the workgroups' sums.  Bound by memory: the gated
// block's 4096 x 8192 bf16 (dy, both fp32 pre-activations, dg and du in two parts: 604 MB)
// 117 to 122 us (5.0 to 5.2 TB/s); sums alone of 8192 x 2048 bf16 12 and 5 us.
namespace {

// Rows of a workgroup: four, a row a wave; sixteen with sums, a quarter of them to
// add again, where there are elements for it.  silu and dbias alone, bf16 (us,
// sixteen in parentheses): 1024 x 1024 6.7 (7.5), 777 x 3592 8.7 (9.0), 2048 x 2048 11.0
// (9.5), 8192 x 4096 47 (40).  With dx after it and no dbias, one part: 8192 x 4096 60
// (66), the gated block's 110 (117).
int64_t slope_rows(int64_t M, int64_t N, bool sums) { return sums && M * N >= (int64_t)1 << 22 ? 16 : 4; }

// (Past one row of the grid the work goes on in the next: a loop over it costs 7%, this 2.)
template <int ROWS, bool GATED>
__global__ __launch_bounds__(256) void slope_kernel(Slope s, int64_t stripes, int64_t all)
{
    constexpr int kEach = ROWS / 4;
    __shared__ float sum[4][64][9];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t b = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (b >= all) return;
    const int64_t stripe = b % stripes, block = b / stripes;
    const int64_t c = (stripe * 64 + lane) * 8;
    const int64_t r0 = block * ROWS + wave * kEach;
    const int count = s.N - c < 8 ? (int)(s.N - c) : 8;  // (none below 1)
    float total[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    float dz[kEach][8], z[kEach][8], u[kEach][8];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        if (r0 + i < s.M && count > 0) {
            load_run<8>(s.dy, s.dtype, (r0 + i) * s.lddy + c, count, dz[i]);
            if (s.pre) {
                load_run<8>(s.pre, NUTS_F32, (r0 + i) * s.N + c, count, z[i]);
                if constexpr (GATED) load_run<8>(s.pre, NUTS_F32, (s.M + r0 + i) * s.N + c, count, u[i]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        if (r0 + i >= s.M || count <= 0) continue;
        float du[8];
        if (s.pre) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float a, slope;
                activate_slope(z[i][j], s.act, &a, &slope);
                if constexpr (GATED) {
                    du[j] = dz[i][j] * a;
                    dz[i][j] *= u[i][j] * slope;
                } else {
                    dz[i][j] *= slope;
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) total[j] += dz[i][j];
        if (s.dz) {
            const int64_t at = (r0 + i) * s.ld + c;
            store_run<8>(s.dz, s.dtype, at, count, dz[i]);
            if constexpr (GATED) store_run<8>(s.dz2, s.dtype, at, count, du);
            if (s.rest) {
                // what rounding took off, as a second matrix (nothing of an infinity)
                auto off = [](float v) {
                    const float head = (float)(__bf16)v;
                    return fabsf(head) == __builtin_inff() ? 0.0f : v - head;
                };
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    dz[i][j] = off(dz[i][j]);
                    if constexpr (GATED) du[j] = off(du[j]);
                }
                store_run<8>(s.dz, s.dtype, s.rest + at, count, dz[i]);
                if constexpr (GATED) store_run<8>(s.dz2, s.dtype, s.rest + at, count, du);
            }
        }
    }
    if (!s.dbias) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[wave][lane][j] = total[j];
    __syncthreads();
    for (int t = threadIdx.x; t < 512; t += 256) {
        const int64_t n = stripe * 512 + t;
        if (n >= s.N) continue;
        const int l = t / 8, j = t % 8;
        s.sums[block * s.N + n] = (sum[0][l][j] + sum[1][l][j]) + (sum[2][l][j] + sum[3][l][j]);
    }
}

// 64 columns a workgroup; its 16 waves take the rows in turn.
__global__ __launch_bounds__(1024) void bias_kernel(const float* sums, int64_t blocks, int64_t N, void* dbias, int dtype)
{
    __shared__ float part[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int64_t n0 = (int64_t)blockIdx.x * 64; n0 < N; n0 += (int64_t)gridDim.x * 64) {
        const int64_t n = n0 + lane;
        float t = 0.0f;
        if (n < N) {
#pragma unroll 4
            for (int64_t b = wave; b < blocks; b += 16) t += sums[b * N + n];
        }
        part[wave][lane] = t;
        __syncthreads();
        if (wave == 0 && n < N) {
#pragma unroll
            for (int w = 1; w < 16; ++w) t += part[w][lane];
            store_f32(dbias, dtype, n, t);
        }
        __syncthreads();
    }
}

}  // namespace

size_t slope_sums_bytes(int64_t M, int64_t N)
{
    const int64_t rows = slope_rows(M, N, true);
    return (size_t)((M + rows - 1) / rows) * N * sizeof(float);
}

hipError_t launch_slope(const Slope& s, hipStream_t stream)
{
    const int64_t rows = slope_rows(s.M, s.N, s.dbias);
    const int64_t stripes = (s.N + 511) / 512, blocks = (s.M + rows - 1) / rows;
    if (const int64_t all = stripes * blocks) {
        const unsigned row = groups_of(all);
        const dim3 grid(row, (unsigned)((all + row - 1) / row));
        auto go = [&](auto* k) { k<<<grid, 256, 0, stream>>>(s, stripes, all); };
        s.gated ? go(slope_kernel<4, true>) : rows == 4 ? go(slope_kernel<4, false>) : go(slope_kernel<16, false>);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    if (s.dbias && s.N) {
        bias_kernel<<<groups_of((s.N + 63) / 64, 1024), 1024, 0, stream>>>(s.sums, blocks, s.N, s.dbias, s.dtype);
        return hipGetLastError();
    }
    return hipSuccess;
}

}  // namespace token
}  // namespace nuts
