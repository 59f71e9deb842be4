// Host-side launchers of the token-model operators and the plain structs they
// share with the C-ABI layer.  Every launcher enqueues on `stream` and returns
// the HIP status; arguments are validated by the caller.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/nuts_token.h"

namespace nuts {
namespace token {

inline size_t type_bytes(int dtype) { return dtype == NUTS_BF16 ? 2 : 4; }
// Workgroups of a launch: 2^30 threads at most (a grid holds fewer than 2^32), each
// workgroup takes further blocks of the work in turn.
inline unsigned groups_of(int64_t blocks, int threads = 256)
{
    const int64_t most = ((int64_t)1 << 30) / threads;
    return (unsigned)(blocks < most ? blocks : most);
}
inline int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// ---------------------------------------------------------------------------
// Matrix products C[M][N] = sum_k A(m, k) B(n, k) on the matrix cores,
// accumulated in fp32.  An operand is stored with k contiguous (A[m][k]) or with
// its rows contiguous (A[k][m]).  The sum runs over up to four terms (two for
// the sum of two products, twice as many for a factor in two parts), each over K.
struct Term {
    const void* a;
    const void* b;
    const void* b2;  // gated: the second factor's rows (else unused)
    int64_t lda, ldb, ldb2;
};
constexpr int kMaxTerms = 4;

// What happens to the sums.
struct Epilogue {
    void* out;
    int64_t ldo;
    const void* bias;  // [N] or null
    const void* res;   // or null
    int64_t ldr;
    float* pre;        // [M][N] (gated: [2][M][N]) or null
    int act;
    int dtype;
};

struct Product {
    int64_t M, N, K;  // N: columns of the output (gated: of the gated output)
    int dtype;
    bool staged;      // through registers: fp32, or bf16 operands off the 16-byte grid
    bool a_rows;      // A is stored [k][m]
    bool b_rows;      // B is stored [k][n] (with a_rows, always)
    bool gated;       // two sums per output: act(A B^T) (A B2^T)
    int nterms;
    int small_terms;  // so many terms at the start are corrections of the others
    int sets;         // products of one shape in one launch: set s has terms[s]
    Term terms[2][kMaxTerms];
    Epilogue epi[2];
};
constexpr int kStep = 64;  // k of a stage (32 for fp32)
constexpr int kMaxSlices = 32;

// Tiles and slices.  A unit has places for one workgroup of 256 x 256 tiles, two
// of 128 x 128, four of 64 x 64.  The largest tile that fills three quarters of
// the places is taken, the sum in slices where there are fewer tiles than places.
// The slices' sums are written, read and added, 7 us at 1000 x 1027 and 14 us at 777
// x 3592: a slice has 512 k at least (256 of the small tiles'), and small tiles one
// for each unit are not sliced.  fp32 at 1000 x 1027 x 513: 22 us in 64 x 64 tiles, 24
// in two slices, 28 in 128 x 128 tiles and two slices; 777 x 3592 x 640: 34, 44 and 41
// us; 777 x 640 x 3592: 94 us whole, 48 in four slices, 64 in 128 x 128 tiles and four.
struct Plan {
    int tile, slices;
};
inline int64_t steps_of(const Product& p)
{
    const int ks = p.dtype == NUTS_F32 ? 32 : kStep;
    return (p.K + ks - 1) / ks;
}
inline Plan plan_product(const Product& p, int num_cu)
{
    for (int tile = p.staged ? 128 : 256;; tile /= 2) {
        const int64_t tiles = ((p.M + tile - 1) / tile) * ((p.N * (p.gated ? 2 : 1) + tile - 1) / tile) * p.sets;
        const int64_t places = (int64_t)num_cu * (tile == 256 ? 1 : tile == 128 ? 2 : 4);
        int64_t s = tile == 256 || tiles >= (tile == 64 ? num_cu : places) ? 1 : places / tiles;
        const int64_t most = p.K * p.nterms / (tile == 64 ? 256 : 512);
        if (s > most) s = most;
        if (s > kMaxSlices) s = kMaxSlices;
        if (s < 1) s = 1;
        if (tile == 64 || tiles * s >= places * 3 / 4) return {tile, (int)s};
    }
}

// fp32 partial sums that the product needs (bytes), by its sizes alone.
size_t product_workspace(const Product& p, int num_cu);
hipError_t launch_product(const Product& p, float* partials, int num_cu, hipStream_t stream);

// A few rows: x [M][K] against w (and w2: gated) [N][K], read once in its own type
// and alignment.  16 rows at any size, up to 64 where the product is small: every
// workgroup reads all of x, which tiles of the product do not.  bf16 (us, in
// parentheses as tiles): 5 x 4096 x 1024 4.6 (9.3), 5 x 8192 x 4096 16 (22), 16 x 16,384
// x 4096 37 (34); 32 x 2048 x 2048 8.3 (11.3), 32 x 2048 x 8192 25 (22), 32 x 50,000 x
// 1024 44 (35); 64 x 4096 x 1024 7.9 (11.5), 64 x 2048 x 2048 12 (12), 64 x 16,384
// x 4096 85 (38).  fp32: 16 x 8192 x 4096 38 (58), 64 x 4096 x 1024 14 (17), 64 x 2048 x
// 2048 22 (17).
inline bool few_rows(int64_t M, int64_t N, int64_t K)
{
    return M <= 16 || (M <= 64 && M * K <= 65536 && N <= 8192);
}
struct FewRows {
    bool gated;
    int64_t M, N, K;
    const void* x;
    int64_t ldx;
    const void* w;
    int64_t ldw;
    const void* w2;
    int64_t ldw2;
    Epilogue epi;
};
hipError_t launch_few_rows(const FewRows& p, hipStream_t stream);

// dz = dy act'(pre) of the linear layer, or dg and du of the gated block, in
// the inputs' type, and the sums of dz over the rows.
struct Slope {
    int64_t M, N;
    const void* dy;
    int64_t lddy;
    const float* pre;   // [M][N], gated [2][M][N]; null: the identity
    int act;
    int dtype;
    bool gated;
    void* dz;           // [M][N], row stride ld (gated: dg); null: the sums alone
    void* dz2;          // gated: du
    int64_t rest;       // bf16: where the matrix of what rounding took off lies (elements on); 0: none
    int64_t ld;
    void* dbias;        // [N] or null
    float* sums;        // slope_sums_bytes(M, N), with dbias
};
size_t slope_sums_bytes(int64_t M, int64_t N);
hipError_t launch_slope(const Slope& s, hipStream_t stream);

// ---------------------------------------------------------------------------
hipError_t launch_embedding(const nuts_embedding_args& a, hipStream_t stream);

size_t embedding_grad_workspace(const nuts_embedding_grad_args& a);
hipError_t launch_embedding_grad(const nuts_embedding_grad_args& a, void* workspace, hipStream_t stream);

hipError_t launch_categorical(const nuts_categorical_args& a, hipStream_t stream);

}  // namespace token
}  // namespace nuts
