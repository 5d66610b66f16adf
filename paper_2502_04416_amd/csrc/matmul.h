// Products of the training operators (ffn.hip, head_loss.hip): C = A * B with what each operator does to the result while it is in
// registers.  Host interface; the kernels are in matmul_device.h.
#pragma once
#include <hip/hip_runtime.h>

#include "cmoe_internal.h"

namespace cmoe {

// An operand "by rows" has K along its rows (A [m, k], B [n, k]); "by columns" K runs down its columns (A [k, m], B [k, n]).
enum Product {
  PRODUCT_GATED,    // A by rows, B and B2 by columns: G = A B, U = A B2; c = silu(G) U, c2 = G, c3 = U (c2, c3 may be null)
  PRODUCT_DOWN,     // A by rows, B by columns: c = e1 + A B (e1 may be null)
  PRODUCT_DGATED,   // A, B by rows: from dH = A B^T, G = e1, U = e2: c = dG, c2 = dU
  PRODUCT_DX,       // A, B by rows, K in two parts: c = e1 + A B^T + A2 B2^T (e1 may be null)
  PRODUCT_DW,       // A, B by columns: c = alpha A^T B, and c2 = alpha A^T B2 where c2 is given (alpha times factor[0], where that is given)
  PRODUCT_LSE,      // A, B by rows: per row and column range the largest logit and the sum of exponentials; the target's logit
  PRODUCT_DLOGITS,  // A, B by rows: c = row weight * (exp(A B^T - lse) - [target])
  PRODUCT_DHEAD,    // A by rows, B by columns: acc (+)= A B over the pieces of a vocabulary, c = alpha * acc with the last one (factor as above)
};

// PRODUCT_LSE and PRODUCT_DLOGITS have to agree to the bit: 1 - p of a likely target is a difference of both.  The ring's tiles sum in one
// order, those for any operand in another, and so does every K split: both passes go by the same plan, for every piece of a vocabulary, which is a
// function of the sizes alone.  (bf16 operands that the ring can read where they are need no copies and take the ring in any case: x and the weight have to
// be at the same alignment in both passes, as the same tensors are.)
struct LogitsPlan {
  bool in_place;             // of operands that the ring cannot read where they are: no copies
  int k_split;               // of all tiles
};

struct MatArgs {
  const void *a, *a2, *b, *b2;
  int64_t lda, ldb;          // elements from one row of memory to the next (of both parts)
  int m, n, k;               // the result is [m, n]; k: of each part
  // what of an operand may be read where that is more or less than its part in the result: rows or columns of A (m_a >= m: padding, in
  // any state), of B (n_b <= n: zeros behind it), and B's K (k_b <= k: zeros behind it; A has zeros there itself)
  int m_a, n_b, k_b;
  int64_t a_plane, b_plane;  // elements from one plane of a copied fp32 operand to the next
  void *c, *c2, *c3;
  const void *e1, *e2;
  int64_t ldc;               // of c, c2, c3, e1 and e2
  float alpha;
  const float* factor;       // of alpha, on the device, or null: 1
  // head
  float* acc;                // [m, n]
  int first, last;           // pieces of the vocabulary
  int col0;                  // vocabulary index of column 0
  int vocab;
  const int32_t* ids;        // [m]
  const float* lse;          // [m]
  const float* dloss;        // [m] or null
  LogitsPlan logits;
  float2* part;              // [column ranges][m]
  float* picked;             // [m]
  // Tiles are numbered over both results (zs of them); from tile `full` on, each is split into k_split parts of K, whose sums go to slab
  // [tile][part][bm][bn] (both halves of a gated tile side by side), and a finishing kernel adds them in order.
  int zs, full, k_split, bm, bn;
  float* slab;
};

// The plan for the logits of m tokens of width k over n entries; for the two products of logits, below, of any piece of them.
LogitsPlan logits_plan(int dtype, int64_t m, int64_t n, int64_t k);
// Bytes of workspace, for copies of operands and slabs of a K split, that a product may ask for, whatever its operands' alignment.
size_t matmul_workspace_bytes(Product kind, int dtype, int64_t m, int64_t n, int64_t k, const LogitsPlan* plan = nullptr);
// Column ranges that PRODUCT_LSE may write: rows of `part`, whatever its operands' alignment.
int64_t lse_ranges(int dtype, int64_t m, int64_t n, int64_t k, const LogitsPlan& plan);
// Enqueues the product; m_a, n_b and k_b count as m, n and k where they are 0.  Workspace: 16-byte aligned.  *ranges, of PRODUCT_LSE: how many
// ranges have been written.
hipError_t matmul(Product kind, int dtype, MatArgs p, void* workspace, size_t workspace_bytes, hipStream_t s, int* ranges = nullptr);

}  // namespace cmoe
