// Embedding of tokens and the gradient of its table.
//
// Both move memory and compute next to nothing.  The gradient sorts the
// positions by token (a stable radix sort, least digit first: the order of a
// token's positions, and so its sum, is fixed), sums runs of equal tokens in
// chunks of sorted positions, so that a token that fills half a batch is read by the
// whole device, and joins the chunks' sums while it writes the table: a token's in
// the threads of its row, one after the other.
#include "token.h"
#include "token_device.h"

namespace nuts {
namespace token {
namespace {

// A run of W elements of a row: 16 bytes, or one element where a row is shorter
// than that.  The last run of a row ends with the row and so overlaps the one
// before it; both compute and write the same values there.
template <typename T, int W>
struct Run {
    v4u raw;
    __device__ __forceinline__ void load(const T* p)
    {
        if constexpr (W == 1) raw[0] = __float_as_uint(to_f32(*p));
        else raw = load16(p);
    }
    __device__ __forceinline__ void values(float (&v)[W]) const
    {
        if constexpr (W == 1) v[0] = __uint_as_float(raw[0]);
        else unpack<T>(raw, v);
    }
    template <bool PAST>
    __device__ __forceinline__ static void store(T* p, const float (&v)[W])
    {
        if constexpr (W == 1) *p = from_f32<T>(v[0]);
        else store16<PAST>(p, pack<T>(v));
    }
};

// Workgroups of 256 threads as `tx` runs of a row by 256 / tx rows.
struct Shape {
    int tx;        // a power of two, 8 .. 256
    int width;     // elements of a run
    int64_t cols;  // workgroups along a row
};
Shape row_shape(int64_t D, int dtype)
{
    const int width = D * (int64_t)type_bytes(dtype) < 16 ? 1 : 16 / (int)type_bytes(dtype);
    const int64_t runs = (D + width - 1) / width;
    int tx = 8;
    while (tx < 256 && tx < runs) tx *= 2;
    return {tx, width, (runs + tx - 1) / tx};
}
// Column of this thread's run in block column `col`, or -1.
template <int W>
__device__ __forceinline__ int64_t run_column(int64_t col, int tx, int64_t D)
{
    const int64_t c = (col * tx + threadIdx.x % tx) * W;
    return c >= D ? -1 : c + W <= D ? c : D - W;
}

// out_i = scale table[id_i].  Bound by memory: N (or the distinct tokens') rows
// read, N written.  A thread has 16 bytes of EACH rows, all of them in flight:
// four where there are rows for it.  32,768 rows of 4096 bf16 77 us (537 MB: 7.0 TB/s, a
// part of it read from caches), 8 rows 3.4 us.
template <typename T, int W, int EACH, bool PAST>
__global__ __launch_bounds__(256) void embedding_kernel(nuts_embedding_args a, int tx, int64_t cols, int64_t blocks)
{
    const int per = 256 / tx;
    for (int64_t b = blockIdx.x; b < blocks; b += gridDim.x) {
        const int64_t i0 = b / cols * (EACH * per) + threadIdx.x / tx, c = run_column<W>(b % cols, tx, a.D);
        if (c < 0) continue;
        int64_t id[EACH];
        Run<T, W> run[EACH];
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            const int64_t i = i0 + j * per;
            id[j] = i < a.N ? a.ids[i] : -1;
        }
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            run[j].raw = v4u{0, 0, 0, 0};
            if (id[j] >= 0 && id[j] < a.V) run[j].load((const T*)a.table + id[j] * a.ld_table + c);
        }
        const float scale = (float)a.scale;
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            const int64_t i = i0 + j * per;
            if (i >= a.N) continue;
            const bool there = id[j] >= 0 && id[j] < a.V;  // (0 scale may be -0, and infinities are the table's)
            float v[W];
            run[j].values(v);
#pragma unroll
            for (int e = 0; e < W; ++e) v[e] = there ? v[e] * scale : 0.0f;
            Run<T, W>::template store<PAST>((T*)a.out + i * a.ld_out + c, v);
        }
    }
}

// ---------------------------------------------------------------------------
// Sort.  A key is the token, or V for a position without one; the value is the
// position.

__device__ __forceinline__ uint32_t key_of(const int64_t* ids, int64_t i, int64_t V)
{
    const int64_t id = ids[i];
    return id >= 0 && id < V ? (uint32_t)id : (uint32_t)V;
}

constexpr int kDigitBits = 9;  // at most

// Lanes of the wave (among `live`) whose digit is this lane's.
struct Same {
    uint32_t lo, hi;
    __device__ __forceinline__ uint32_t before() const
    {
        return __builtin_amdgcn_mbcnt_hi(hi, __builtin_amdgcn_mbcnt_lo(lo, 0));
    }
    __device__ __forceinline__ uint32_t count() const { return __popc(lo) + __popc(hi); }
};
__device__ __forceinline__ Same same_digit(uint32_t digit, int bits, uint64_t live)
{
    uint32_t lo = (uint32_t)live, hi = (uint32_t)(live >> 32);
#pragma unroll
    for (int b = 0; b < kDigitBits; ++b) {
        if (b >= bits) break;
        const int mine = (int)(digit << (31 - b)) >> 31;  // all ones if bit b is set
        const uint64_t v = __ballot(mine);
        lo &= ~((uint32_t)v ^ mine);
        hi &= ~((uint32_t)(v >> 32) ^ mine);
    }
    return {lo, hi};
}

// Positions that one workgroup sorts in LDS: one launch for four or more.  A table's
// gradient of 30,000 rows: 500 positions 21 us (27 by the passes of many
// workgroups), 2000 28 (34), 4000 33 (35), 8000 41 (36).
constexpr int kSmallSort = 4096;
constexpr int kSmallWaves = 16;
constexpr int kSmallBits = 8;

struct Sorted {
    uint32_t* key;   // [N]
    uint32_t* at;    // [N]
    int32_t* first;  // [V]: first sorted position of a token, -1 where it has none
    int32_t* last;   // [V]: one past its last
};

// Workgroup 0 sorts; the others mark every token absent.  A radix sort of 8 bits a
// pass: a wave counts its own run's digits, the counts are summed in (digit, wave)
// order, and a wave's lanes take their places in order of the run: lanes with one
// digit find each other by a ballot a bit.  Bound by the latency of the chain of
// LDS accesses: 1000, 2000 and 4000 positions of 20,011 tokens take 6, 8 and 12 us.
__global__ __launch_bounds__(64 * kSmallWaves) void small_sort_kernel(const int64_t* ids, int N, int64_t V, int bits,
                                                                      Sorted out)
{
    if (blockIdx.x > 0) {
        const int64_t n = (int64_t)(gridDim.x - 1) * blockDim.x;
        for (int64_t v = (int64_t)(blockIdx.x - 1) * blockDim.x + threadIdx.x; v < V; v += n) out.first[v] = -1;
        return;
    }
    extern __shared__ uint32_t mem[];
    __shared__ uint32_t count[1 << kSmallBits][kSmallWaves];  // by digit, then wave
    __shared__ uint32_t wave_sum[kSmallWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int per = ((N + kSmallWaves - 1) / kSmallWaves + 63) / 64 * 64;  // of a wave, in rounds of 64
    const int padded = per * kSmallWaves;
    uint32_t *key = mem, *at = mem + padded;
    // the wave's run, 64 positions a round, in registers
    constexpr int kRounds = kSmallSort / (64 * kSmallWaves);
    const int w0 = wave * per, w1 = w0 + per < N ? w0 + per : N;
    uint32_t k[kRounds], a[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int i = w0 + r * 64 + lane;
        k[r] = i < w1 && r * 64 < per ? key_of(ids, i, V) : 0;
        a[r] = i;
    }
    for (int shift = 0; shift < bits; shift += kSmallBits) {
        for (int i = tid; i < (1 << kSmallBits) * kSmallWaves; i += blockDim.x) (&count[0][0])[i] = 0;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kRounds; ++r)
            if (r * 64 < per && w0 + r * 64 + lane < w1)
                atomicAdd(&count[(k[r] >> shift) & ((1 << kSmallBits) - 1)][wave], 1u);
        __syncthreads();
        // exclusive sums over the counts in (digit, wave) order: four a thread
        uint32_t* flat = &count[0][0];
        uint32_t c[4], sum = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            c[i] = flat[tid * 4 + i];
            sum += c[i];
        }
        uint32_t run = sum;
#pragma unroll
        for (int o = 1; o < 64; o *= 2) {
            const uint32_t v = __shfl_up(run, o);
            if (lane >= o) run += v;
        }
        if (lane == 63) wave_sum[wave] = run;
        __syncthreads();
        run -= sum;
#pragma unroll
        for (int w = 0; w < kSmallWaves; ++w) run += w < wave ? wave_sum[w] : 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            flat[tid * 4 + i] = run;
            run += c[i];
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            if (r * 64 >= per) break;
            const bool in = w0 + r * 64 + lane < w1;
            const uint32_t d = (k[r] >> shift) & ((1 << kSmallBits) - 1);
            const Same m = same_digit(d, kSmallBits, __ballot(in));
            const uint32_t base = in ? count[d][wave] : 0, before = m.before();
            wave_sync();
            if (in) {
                key[base + before] = k[r];
                at[base + before] = a[r];
                if (before == 0) count[d][wave] = base + m.count();
            }
            wave_sync();
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            const int i = w0 + r * 64 + lane;
            if (r * 64 < per && i < w1) {
                k[r] = key[i];
                a[r] = at[i];
            }
        }
    }
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int i = w0 + r * 64 + lane;
        if (r * 64 < per && i < w1) {
            out.key[i] = k[r];
            out.at[i] = a[r];
        }
    }
}
static_assert((1 << kSmallBits) * kSmallWaves == 4 * 64 * kSmallWaves, "four counts a thread");

// Many positions: workgroups of consecutive positions, a pass a digit of up to
// 9 bits: counts, then every workgroup's place for each digit from all counts.
// Bound by latency (32,768 positions move 2 MB a pass): a pass takes 5 us of
// counting, with marking 64,000 tokens absent in the first, and 7 us of placing, of
// which reading the other workgroups' counts is the most.  256 workgroups at most keep
// those counts few; digits of 9 bits sort 64,000 tokens in two passes.
constexpr int kSortGroups = 256;
constexpr int kSortWaves = 8;

struct SortPass {
    const int64_t* ids;       // the first pass reads the tokens
    const uint32_t *key, *at; // later ones the last pass's output
    uint32_t *key_out, *at_out;
    uint32_t* counts;         // [groups][1 << bits]
    int32_t* first;           // first pass: marked -1
    int64_t N, V;
    int64_t each;             // positions of a workgroup (a multiple of 64 * kSortWaves)
    int shift, bits;
};

__global__ __launch_bounds__(64 * kSortWaves) void count_kernel(SortPass p)
{
    __shared__ uint32_t count[1 << kDigitBits];
    for (int i = threadIdx.x; i < 1 << p.bits; i += blockDim.x) count[i] = 0;
    if (p.ids) {
        for (int64_t v = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; v < p.V; v += (int64_t)gridDim.x * blockDim.x)
            p.first[v] = -1;
    }
    __syncthreads();
    const int64_t b0 = blockIdx.x * p.each, b1 = b0 + p.each < p.N ? b0 + p.each : p.N;
    for (int64_t i = b0 + threadIdx.x; i < b1; i += blockDim.x) {
        const uint32_t k = p.ids ? key_of(p.ids, i, p.V) : p.key[i];
        atomicAdd(&count[(k >> p.shift) & ((1u << p.bits) - 1)], 1u);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 1 << p.bits; i += blockDim.x)
        p.counts[((int64_t)blockIdx.x << p.bits) + i] = count[i];
}

__global__ __launch_bounds__(64 * kSortWaves) void place_kernel(SortPass p)
{
    __shared__ uint32_t base[1 << kDigitBits];
    __shared__ uint32_t count[kSortWaves][1 << kDigitBits];
    __shared__ uint32_t wave_sum[kSortWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int bins = 1 << p.bits;
    // this workgroup's first place for digit `tid`: all smaller digits', and
    // its own digit's of earlier workgroups
    uint32_t before = 0, total = 0;
    if (tid < bins) {
        for (int g0 = 0; g0 < (int)gridDim.x; g0 += 16) {
            uint32_t c[16];
#pragma unroll
            for (int i = 0; i < 16; ++i)
                c[i] = g0 + i < (int)gridDim.x ? p.counts[((int64_t)(g0 + i) << p.bits) + tid] : 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                total += c[i];
                if (g0 + i < (int)blockIdx.x) before += c[i];
            }
        }
    }
    uint32_t run = total;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const uint32_t v = __shfl_up(run, o);
        if (lane >= o) run += v;
    }
    if (lane == 63) wave_sum[wave] = run;
    __syncthreads();
    run -= total;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) run += w < wave ? wave_sum[w] : 0;
    if (tid < bins) base[tid] = run + before;
    const int64_t b0 = blockIdx.x * p.each, b1 = b0 + p.each < p.N ? b0 + p.each : p.N;
    for (int64_t i = b0; i < b1; i += 64 * kSortWaves) {
        for (int j = tid; j < kSortWaves * bins; j += blockDim.x) count[j >> p.bits][j & (bins - 1)] = 0;
        __syncthreads();
        const bool in = i + tid < b1;
        uint32_t k = 0, a = 0;
        if (in) {
            k = p.ids ? key_of(p.ids, i + tid, p.V) : p.key[i + tid];
            a = p.ids ? (uint32_t)(i + tid) : p.at[i + tid];
        }
        const uint32_t d = (k >> p.shift) & (bins - 1);
        const Same m = same_digit(d, p.bits, __ballot(in));
        const uint32_t before = m.before();
        if (in && before == 0) count[wave][d] = m.count();
        __syncthreads();
        if (in) {
            uint32_t to = base[d] + before;
            for (int w = 0; w < wave; ++w) to += count[w][d];
            p.key_out[to] = k;
            p.at_out[to] = a;
        }
        __syncthreads();
        if (tid < bins) {
            uint32_t c = 0;
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) c += count[w][tid];
            base[tid] += c;
        }
        __syncthreads();
    }
}
static_assert(64 * kSortWaves >= 1 << kDigitBits, "a thread a digit");

// ---------------------------------------------------------------------------
// Sums.  A chunk is kChunk sorted positions.  A token whose positions lie in one
// chunk is finished there; otherwise each of its chunks keeps a partial row: the
// one that it begins in in slot 1, those that it comes from before in slot 0.
// Sums are fp32 in order of the positions, scaled and rounded once.
// Bound by memory: N rows read, the distinct tokens' rows written here and the
// others' zeros by the second kernel.  32,768 rows of 4096 bf16 to 64,000: 86 us (268 MB
// read in rows anywhere) and 68 us (6.3 TB/s of stores).
constexpr int kChunk = 32;
constexpr int kAhead = 8;  // rows in flight

template <typename T, int W, bool PAST>
__device__ __forceinline__ void chunk_sum(const nuts_embedding_grad_args& a, const Sorted& s, float* partial,
                                          int64_t chunk, int64_t c)
{
    const int64_t i0 = chunk * kChunk, i1 = i0 + kChunk < a.N ? i0 + kChunk : a.N;
    if (i0 >= a.N || c < 0) return;
    const uint32_t V = (uint32_t)a.V;
    uint32_t token = s.key[i0];
    if (token == V) return;  // (positions without a token are the last)
    const uint32_t open = i0 > 0 && s.key[i0 - 1] == token ? token : V;  // comes from the chunk before
    const uint32_t next = i1 < a.N ? s.key[i1] : V;
    const float scale = (float)a.scale;
    float sum[W];
#pragma unroll
    for (int e = 0; e < W; ++e) sum[e] = 0.0f;
    auto finish = [&](uint32_t t, bool last) {
        const bool from_before = t == open, goes_on = last && t == next;
        if (!from_before && !goes_on) {
            float v[W];
#pragma unroll
            for (int e = 0; e < W; ++e) v[e] = sum[e] * scale;
            Run<T, W>::template store<PAST>((T*)a.dtable + (int64_t)t * a.ld_dtable + c, v);
            return;
        }
        // (a run that comes from before and goes on lies in slot 0)
        float* p = partial + (2 * chunk + (from_before ? 0 : 1)) * a.D + c;
        if constexpr (W == 1) {
            *p = sum[0];
        } else {
#pragma unroll
            for (int e = 0; e < W; e += 4)
                store16(p + e, v4u{__float_as_uint(sum[e]), __float_as_uint(sum[e + 1]), __float_as_uint(sum[e + 2]),
                                   __float_as_uint(sum[e + 3])});
        }
    };
    const bool marks = c == 0;
    if (marks && token != open) s.first[token] = (int32_t)i0;
    for (int64_t i = i0; i < i1 && token != V; i += kAhead) {
        Run<T, W> row[kAhead];
        uint32_t key[kAhead], at[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int64_t k = i + j < i1 ? i + j : i1 - 1;
            key[j] = s.key[k];
            at[j] = s.at[k];
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (i + j >= i1) key[j] = V;
            if (key[j] != V) row[j].load((const T*)a.dout + (int64_t)at[j] * a.ld_dout + c);
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (i + j >= i1 || token == V) continue;
            if (key[j] != token) {
                finish(token, false);
                if (marks) {
                    s.last[token] = (int32_t)(i + j);
                    if (key[j] != V) s.first[key[j]] = (int32_t)(i + j);
                }
                token = key[j];
#pragma unroll
                for (int e = 0; e < W; ++e) sum[e] = 0.0f;
            }
            if (token != V) {
                float v[W];
                row[j].values(v);
#pragma unroll
                for (int e = 0; e < W; ++e) sum[e] += v[e];
            }
        }
    }
    if (token != V) {
        finish(token, true);
        if (marks && token != next) s.last[token] = (int32_t)i1;
    }
}

template <typename T, int W, bool PAST>
__global__ __launch_bounds__(256) void chunk_sum_kernel(nuts_embedding_grad_args a, Sorted s, float* partial, int tx,
                                                        int64_t cols, int64_t blocks)
{
    for (int64_t b = blockIdx.x; b < blocks; b += gridDim.x)
        chunk_sum<T, W, PAST>(a, s, partial, b / cols * (256 / tx) + threadIdx.x / tx, run_column<W>(b % cols, tx, a.D));
}

// The rows of tokens that no chunk finished: zeros, or the partial rows' sum.  A token
// of n positions is a chain of n / 32 additions here: 65,536 positions of 100 tokens,
// 1024 bf16 wide, take 133 us where a third of them hold one token, 53 us where all
// are as frequent.
constexpr int kTableRows = 4;  // of a thread
template <typename T, int W, bool PAST>
__global__ __launch_bounds__(256) void table_kernel(nuts_embedding_grad_args a, Sorted s, const float* partial, int tx,
                                                    int64_t cols, int64_t blocks)
{
    const int per = 256 / tx;
    for (int64_t b = blockIdx.x; b < blocks; b += gridDim.x) {
        const int64_t v0 = b / cols * (kTableRows * per) + threadIdx.x / tx, c = run_column<W>(b % cols, tx, a.D);
        if (c < 0) continue;
        int32_t first[kTableRows];
#pragma unroll
        for (int j = 0; j < kTableRows; ++j) first[j] = v0 + j * per < a.V ? s.first[v0 + j * per] : 0;
#pragma unroll
        for (int j = 0; j < kTableRows; ++j) {
            const int64_t v = v0 + j * per;
            if (v >= a.V) continue;
            float sum[W];
#pragma unroll
            for (int e = 0; e < W; ++e) sum[e] = 0.0f;
            if (first[j] >= 0) {
                const int64_t c0 = first[j] / kChunk, c1 = (s.last[v] - 1) / kChunk;
                if (c0 == c1) continue;
#pragma unroll 4
                for (int64_t k = c0; k <= c1; ++k) {
                    const float* p = partial + (2 * k + (k == c0 ? 1 : 0)) * a.D + c;
                    if constexpr (W == 1) {
                        sum[0] += *p;
                    } else {
#pragma unroll
                        for (int e = 0; e < W; e += 4) {
                            const v4u q = load16(p + e);
#pragma unroll
                            for (int i = 0; i < 4; ++i) sum[e + i] += __uint_as_float(q[i]);
                        }
                    }
                }
#pragma unroll
                for (int e = 0; e < W; ++e) sum[e] *= (float)a.scale;
            }
            Run<T, W>::template store<PAST>((T*)a.dtable + v * a.ld_dtable + c, sum);
        }
    }
}

int64_t align256(int64_t n) { return (n + 255) & ~(int64_t)255; }

struct GradSpace {
    int64_t key[2], at[2], counts, first, last, partial, bytes;
};
GradSpace grad_space(const nuts_embedding_grad_args& a)
{
    GradSpace g{};
    int64_t n = 0;
    auto take = [&](int64_t bytes) {
        const int64_t at = n;
        n += align256(bytes);
        return at;
    };
    const bool small = a.N <= kSmallSort;
    for (int i = 0; i < (small ? 1 : 2); ++i) {
        g.key[i] = take(a.N * 4);
        g.at[i] = take(a.N * 4);
    }
    if (!small) g.counts = take((int64_t)kSortGroups * (1 << kDigitBits) * 4);
    g.first = take(a.V * 4);
    g.last = take(a.V * 4);
    g.partial = take((a.N + kChunk - 1) / kChunk * 2 * a.D * 4);
    g.bytes = n;
    return g;
}

}  // namespace

namespace {
// Outputs of 128 MB and more, in rows on 16-byte boundaries, are stored past the
// caches: a table's gradient of 64,000 x 4096 bf16 from 32,768 rows 170 us (209
// through them), those rows' lookup 76 us (86); 20,011 x 1001 fp32, off the
// boundaries, 50 us (45).
bool past_caches(const void* out, int64_t rows, int64_t D, int64_t ld, int dtype)
{
    const int64_t bytes = (int64_t)type_bytes(dtype);
    return (uintptr_t)out % 16 == 0 && ld * bytes % 16 == 0 && D * bytes % 16 == 0 && rows * D * bytes >= (int64_t)1 << 27;
}

template <typename T, int W>
void run_embedding(const nuts_embedding_args& a, const Shape& s, hipStream_t stream)
{
    // four rows a thread where there are rows for it (bf16, D = 1024: 512 rows 2.7 us
    // one a thread, 3.6 us four; 2048 rows 3.6 and 4.0; 8192 rows 7.5 and 7.0; 32,768 x
    // 4096 99 and 78)
    const int64_t rows = 256 / s.tx, blocks = (a.N + rows - 1) / rows * s.cols;
    const int64_t fewer = (a.N + 4 * rows - 1) / (4 * rows) * s.cols;
    if (blocks <= 2048)
        embedding_kernel<T, W, 1, false><<<groups_of(blocks), 256, 0, stream>>>(a, s.tx, s.cols, blocks);
    else if (W > 1 && past_caches(a.out, a.N, a.D, a.ld_out, a.dtype))
        embedding_kernel<T, W, 4, (W > 1)><<<groups_of(fewer), 256, 0, stream>>>(a, s.tx, s.cols, fewer);
    else
        embedding_kernel<T, W, 4, false><<<groups_of(fewer), 256, 0, stream>>>(a, s.tx, s.cols, fewer);
}
template <typename T, int W, bool PAST>
hipError_t run_sums(const nuts_embedding_grad_args& a, const Sorted& s, float* partial, const Shape& sh,
                    hipStream_t stream)
{
    const int64_t rows = 256 / sh.tx, chunks = (a.N + kChunk - 1) / kChunk;
    const int64_t sums = (chunks + rows - 1) / rows * sh.cols;
    const int64_t table = (a.V + kTableRows * rows - 1) / (kTableRows * rows) * sh.cols;
    if (sums) chunk_sum_kernel<T, W, PAST><<<groups_of(sums), 256, 0, stream>>>(a, s, partial, sh.tx, sh.cols, sums);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    table_kernel<T, W, PAST><<<groups_of(table), 256, 0, stream>>>(a, s, partial, sh.tx, sh.cols, table);
    return hipGetLastError();
}
template <typename T>
hipError_t run_sums(const nuts_embedding_grad_args& a, const Sorted& s, float* partial, hipStream_t stream)
{
    constexpr int W = 16 / sizeof(T);
    const Shape sh = row_shape(a.D, a.dtype);
    if (sh.width == 1) return run_sums<T, 1, false>(a, s, partial, sh, stream);
    if (past_caches(a.dtable, a.V, a.D, a.ld_dtable, a.dtype)) return run_sums<T, W, true>(a, s, partial, sh, stream);
    return run_sums<T, W, false>(a, s, partial, sh, stream);
}
}  // namespace

hipError_t launch_embedding(const nuts_embedding_args& a, hipStream_t stream)
{
    if (a.N == 0 || a.D == 0) return hipSuccess;
    const Shape s = row_shape(a.D, a.dtype);
    if (a.dtype == NUTS_BF16) s.width == 1 ? run_embedding<__bf16, 1>(a, s, stream) : run_embedding<__bf16, 8>(a, s, stream);
    else s.width == 1 ? run_embedding<float, 1>(a, s, stream) : run_embedding<float, 4>(a, s, stream);
    return hipGetLastError();
}

size_t embedding_grad_workspace(const nuts_embedding_grad_args& a) { return (size_t)grad_space(a).bytes; }

hipError_t launch_embedding_grad(const nuts_embedding_grad_args& a, void* workspace, hipStream_t stream)
{
    if (a.V == 0 || a.D == 0) return hipSuccess;
    const GradSpace g = grad_space(a);
    char* ws = (char*)workspace;
    uint32_t* key[2] = {(uint32_t*)(ws + g.key[0]), (uint32_t*)(ws + g.key[1])};
    uint32_t* at[2] = {(uint32_t*)(ws + g.at[0]), (uint32_t*)(ws + g.at[1])};
    Sorted s{key[0], at[0], (int32_t*)(ws + g.first), (int32_t*)(ws + g.last)};
    float* partial = (float*)(ws + g.partial);
    int bits = 1;
    while (((int64_t)1 << bits) <= a.V) ++bits;  // keys are 0 .. V
    if (a.N <= kSmallSort) {
        const int per = (int)up(up(a.N, kSmallWaves) / kSmallWaves, 64);
        const size_t lds = (size_t)per * kSmallWaves * 2 * sizeof(uint32_t);
        const int64_t fill = (a.V + 4095) / 4096;
        small_sort_kernel<<<(unsigned)(1 + (fill < 256 ? fill : 256)), 64 * kSmallWaves, lds, stream>>>(
            a.ids, (int)a.N, a.V, bits, s);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    } else {
        const int passes = (bits + kDigitBits - 1) / kDigitBits;
        const int digit = (bits + passes - 1) / passes;
        const int64_t round = 64 * kSortWaves;
        const int64_t each = up((a.N + kSortGroups - 1) / kSortGroups, round);
        const unsigned groups = (unsigned)((a.N + each - 1) / each);
        SortPass p{};
        p.N = a.N;
        p.V = a.V;
        p.each = each;
        p.counts = (uint32_t*)(ws + g.counts);
        p.first = s.first;
        p.bits = digit;
        for (int i = 0; i < passes; ++i) {
            p.ids = i == 0 ? a.ids : nullptr;
            p.key = key[(i + 1) & 1];
            p.at = at[(i + 1) & 1];
            p.key_out = key[i & 1];
            p.at_out = at[i & 1];
            p.shift = i * digit;
            count_kernel<<<groups, 64 * kSortWaves, 0, stream>>>(p);
            if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
            place_kernel<<<groups, 64 * kSortWaves, 0, stream>>>(p);
            if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        }
        s.key = key[(passes - 1) & 1];
        s.at = at[(passes - 1) & 1];
    }
    return a.dtype == NUTS_BF16 ? run_sums<__bf16>(a, s, partial, stream) : run_sums<float>(a, s, partial, stream);
}

}  // namespace token
}  // namespace nuts
