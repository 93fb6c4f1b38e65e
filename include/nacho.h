/*
 * nacho.h -- C ABI of the MI355X (gfx950) library for provably load-balanced
 * partitioning of sparse tensor algebra and the partitioned kernels it balances.
 *
 * The operations follow the paper "Partitioning Unstructured Sparse Tensor
 * Algebra for Load-Balanced Parallel Execution":
 *   - nacho_partition : Section 3.2, Algorithm 1 (hierarchical search) with the
 *                       non-zero-count cost functions of Section 4.2.2, stored
 *                       in position space (Section 4.2, 4.2.3);
 *   - nacho_spmv/spmm : the compute kernel of Section 4.4 for y_i = A_ij x_j and
 *                       C_ik = A_ij B_jk (cost scaled by the broadcast extent,
 *                       Section 4.2.2, second listing);
 *   - nacho_spadd_k   : partition -> assembly (count) -> prefix sum -> compute
 *                       (Section 4.3, 4.4, pipeline of Figure 7(a)) for the
 *                       k-operand union of sparse vectors, CSR, DCSR or COO
 *                       matrices (Section 2.1, 2.2);
 *   - nacho_spmul_k   : the same pipeline for the k-operand intersection with
 *                       products (Section 2.1); DCSR operands intersect on the
 *                       outer level and take the recursive partitioning of
 *                       Section 3.3 (Algorithm 2);
 *   - nacho_validate  : debug aid, checks the preconditions below on the device;
 *   - nacho_distill, nacho_route, nacho_experts, nacho_combine, each with its
 *                       gradient: operators that train models, around the sparse
 *                       matrices which training makes (their own conventions below).
 *
 * Conventions that hold for every entry point
 *   * Descriptor structs (nacho_tensor, nacho_parts, nacho_sparse_out) live in
 *     HOST memory and are read during the call only.
 *   * Every array pointer inside them, and every `void*`/typed array argument
 *     that is not explicitly marked "host", is a DEVICE pointer owned by the
 *     caller.  The library allocates and frees nothing; scratch memory comes
 *     from the `ws` argument, sized by nacho_workspace_bytes().
 *   * A call only enqueues kernels on `hip_stream` (a hipStream_t passed as
 *     void*; NULL is the default stream) and returns without synchronising
 *     (nacho_workspace_parts, which launches nothing, reads one word back for a
 *     DCSR product and waits for it).
 *   * Indices and positions are int32; costs are int64.  Preconditions (not
 *     checked): coordinates sorted and unique inside each segment, `pos`
 *     non-decreasing with pos[0] = 0, sum of the operands' nnz < 2^31, all
 *     operands of one call share the same level kinds and extents.
 *   * `crd`, `val` and dense operand arrays must be 16-byte aligned (dense arrays of
 *     the operators that train models: to their elements).
 *   * The return value is a status code.  Argument errors are detected on the
 *     host before anything is launched (nothing is written then); a failed HIP
 *     launch maps to NACHO_ERR_HIP.
 *   * Calls that share a workspace or an output must not overlap in time.
 */
#ifndef NACHO_H
#define NACHO_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    NACHO_OK = 0,
    NACHO_ERR_INVALID_ARG = -1, /* null pointer, bad count, misaligned array, mismatched operands */
    NACHO_ERR_UNSUPPORTED = -2, /* level formats / operand count outside what is implemented      */
    NACHO_ERR_WORKSPACE = -3,   /* ws_bytes smaller than nacho_workspace_bytes() reports           */
    NACHO_ERR_CAPACITY = -4,    /* sparse output larger than the caller's capacity                 */
    NACHO_ERR_HIP = -5,         /* a HIP call failed                                               */
    NACHO_ERR_TOO_LARGE = -6    /* nacho_spmv_static: the call needs more than the built-in scratch */
} nacho_status;

/* F32 and F64: sparse algebra.  F32, BF16 and F16: the operators that train models (nacho_distill and below). */
typedef enum { NACHO_F32 = 0, NACHO_F64 = 1, NACHO_BF16 = 2, NACHO_F16 = 3 } nacho_dtype;
typedef enum { NACHO_DENSE = 0, NACHO_COMPRESSED = 1, NACHO_NONUNIQUE = 2, NACHO_SINGLETON = 3 } nacho_level_kind;
typedef enum {
    NACHO_OP_PARTITION = 0, NACHO_OP_SPMV = 1, NACHO_OP_SPMM = 2, NACHO_OP_SPADD = 3, NACHO_OP_SPMUL = 4
} nacho_op;

#define NACHO_MAX_OPERANDS 8
#define NACHO_MAX_LEVELS 3

/* One level of a tensor's coordinate hierarchy (Section 4.2.1).
 *   DENSE:      every coordinate in [0, extent) is present; pos, crd are NULL.
 *   COMPRESSED: pos[parent] .. pos[parent+1] delimit the sorted coordinates
 *               crd[] stored below `parent` (a top level has one parent, so
 *               pos has 2 entries).  `count` is the number of entries of crd.
 *   NONUNIQUE:  a top compressed level whose sorted coordinates may repeat, one
 *               entry per stored non-zero (the row level of a coordinate list);
 *               crd[count]; pos is not read.
 *   SINGLETON:  one coordinate per entry of the level above: crd[count], the
 *               same count (the column level of a coordinate list).            */
typedef struct {
    int32_t kind;       /* nacho_level_kind                                    */
    int64_t extent;     /* N_m, at most 2^31 - 1                               */
    const int32_t *pos; /* device, [parents + 1]                               */
    const int32_t *crd; /* device, [count]                                     */
    int64_t count;      /* stored coordinates at this level (COMPRESSED only)  */
} nacho_level;

/* A sparse operand.  Supported shapes:
 *   sparse vector  nlevels = 1  {COMPRESSED}
 *   CSR            nlevels = 2  {DENSE, COMPRESSED}
 *   DCSR           nlevels = 2  {COMPRESSED, COMPRESSED}
 *   CSF            nlevels = 3  {COMPRESSED, COMPRESSED, COMPRESSED}: third-order
 *                  tensors (nacho_partition and nacho_spadd_k)
 *   COO            nlevels = 2  {NONUNIQUE, SINGLETON}: entries sorted by (row,
 *                  column), no pair twice (nacho_partition, nacho_spadd_k,
 *                  nacho_spmul_k)
 * `val` (device, one value per innermost coordinate) may be NULL for
 * nacho_partition. */
typedef struct {
    int32_t nlevels;
    nacho_level lvl[NACHO_MAX_LEVELS];
    const void *val;
} nacho_tensor;

/* Stored result of the search (Section 4.2.3: the positions found by the
 * search are kept for the assembly and compute stages).  P partitions have
 * P + 1 boundaries; boundary 0 is the origin, boundary P the end of the
 * iteration space, and partition p spans boundaries p .. p+1.
 *   coord[b*d + m]          coordinate x_m of boundary b
 *   posn[(b*k + t)*d + m]   for operand t: position of the first level-m entry
 *                           that is not before the boundary (DENSE level: x_m)
 *   cost[b]                 C(x) of boundary b = work strictly before it      */
typedef struct {
    int32_t k, d;
    int64_t P;
    int32_t *coord; /* device, [(P+1) * d]     */
    int32_t *posn;  /* device, [(P+1) * k * d] */
    int64_t *cost;  /* device, [P+1]           */
} nacho_parts;

/* Caller-allocated sparse result of nacho_spadd_k, in the operands' format.
 *   vector: crd1[cap_nnz], val[cap_nnz]; pos1[2] = {0, nnz}
 *   CSR:    pos1[n_rows+1], crd1[cap_nnz], val[cap_nnz]
 *   DCSR:   pos0[2] = {0, rows}, crd0[cap_rows], pos1[cap_rows+1], crd1, val
 *   COO:    crd0[cap_nnz] (rows), crd1[cap_nnz] (columns), val[cap_nnz];
 *           pos1[2] = {0, nnz}; cap_rows is not used
 *   CSF (third order, three compressed levels): pos0[2] = {0, slices},
 *           crd0[cap_rows] (i), pos1[cap_rows+1], crd1[cap_fibres] (j),
 *           pos2[cap_fibres+1], crd2[cap_nnz] (k), val[cap_nnz]
 * counts[0] = stored rows (DCSR; n_rows for CSR; 1 for a vector), counts[1] =
 * nnz; for CSF counts = {slices, fibres, nnz}.  counts always has room for
 * three words.  pos2, crd2 and cap_fibres are read for CSF only.  *status is
 * set to NACHO_OK, or to NACHO_ERR_CAPACITY when cap_rows, cap_fibres or
 * cap_nnz is too small (then nothing is written beyond the capacities; counts
 * still hold the required sizes).  The sums of the operands' counts are always
 * sufficient capacities. */
typedef struct {
    int32_t *pos0;
    int32_t *crd0;
    int32_t *pos1;
    int32_t *crd1;
    void *val;
    int64_t cap_rows, cap_nnz;
    int64_t *counts; /* device, [3] */
    int32_t *status; /* device, [1] */
    int32_t *pos2;   /* CSF only */
    int32_t *crd2;   /* CSF only */
    int64_t cap_fibres;
} nacho_sparse_out;

/* Library version (major*10000 + minor*100 + patch) and a static string for a status. */
int32_t nacho_version(void);
const char *nacho_status_string(int32_t status);

/* Number of partitions a fused call uses for these operands (host descriptors;
 * only counts/extents are read) when the caller asks for `P` (0 = automatic).
 * Fused calls never use fewer partitions than needed for one partition's work
 * to fit the staging buffer of its wavefront (SpMV, SpMM) or workgroup (SpAdd,
 * SpMul), so the result is >= P.  For a DCSR product it is an upper bound (the
 * count depends on the rows the operands share).  `n_dense`: SpMM's dense
 * extent (0 otherwise).  For SpMM with P = 0 it is the count of a call whose
 * workspace has the size that nacho_workspace_bytes reports for the same
 * arguments; with a smaller one (sized for another n_dense) the call may use
 * fewer, longer partitions, and nacho_workspace_parts answers for the buffer.
 * Returns 0 on bad input. */
int64_t nacho_num_partitions(int32_t op, const nacho_tensor *ops, int32_t k, int32_t dtype,
                             int64_t n_dense, int64_t P);

/* Bytes of device workspace `op` needs for these operands (host descriptors;
 * only counts/extents are read).  `P` as passed to the call (0 = automatic),
 * `n_dense` = columns of B for SpMM (0 otherwise).  NACHO_OP_SPADD sizes
 * nacho_spadd_k, NACHO_OP_SPMUL nacho_spmul_k.  What it reports for a sum, for a
 * product (not of DCSR operands) or for SpMV with P = 0 also serves calls of the
 * same format, number of operands and value type with fewer entries.  SpMM keeps
 * a row of up to 256 columns of C per partition; large calls with P = 0 are cut
 * into up to eight times as many partitions as small ones, as long as these rows
 * take no more than 512 MiB. */
int32_t nacho_workspace_bytes(int32_t op, const nacho_tensor *ops, int32_t k, int32_t dtype,
                              int64_t n_dense, int64_t P, size_t *bytes);

/*
 * Algorithm 1 for all P+1 boundaries of a P-way partition, one independent
 * search per interior boundary (Section 3.2; Section 4.2.3).
 *   ops[k]        coiterated operands (1 <= k <= NACHO_MAX_OPERANDS)
 *   cost_scale    >= 1; every stored non-zero costs this much (the extent of a
 *                 broadcast dense inner loop, Section 4.2.2).  Queries are then
 *                 interpreted in scaled units and boundaries never fall inside
 *                 the dense loop: the boundary of query Q is that of
 *                 floor(Q / cost_scale) in unscaled units.
 *   P             number of partitions (>= 1)
 *   queries       device int64[P+1] or NULL.  NULL: Q_p = floor(p*Q_total/P).
 *                 Entries 0 and P are ignored (origin / end); an interior
 *                 query >= Q_total yields the end boundary.
 *   out           coord/posn/cost arrays of the sizes documented above
 * Errors: INVALID_ARG (null/size/kind), UNSUPPORTED (format), WORKSPACE, HIP.
 */
int32_t nacho_partition(const nacho_tensor *ops, int32_t k, int64_t cost_scale, int64_t P,
                        const int64_t *queries, const nacho_parts *out,
                        void *ws, size_t ws_bytes, void *hip_stream);

/*
 * nacho_partition for ONE CSR operand whose positions are 64-bit: operands of
 * 2^31 stored non-zeros or more, which the int32 descriptors above cannot
 * describe (Section 4.2.2's CSR cost functions, C_i(x) = pos[x] and the count
 * of the row's entries before a column; equal-share queries
 * Q_p = floor(p * nnz / P)).
 *   pos     device int64[n_rows + 1], non-decreasing, pos[0] = 0, pos[n_rows] = nnz
 *   crd     device int32[nnz], 16-byte aligned
 *   coord   device int32[(P+1) * 2]   (row, column) of every boundary
 *   posn    device int64[(P+1) * 2]   (row, position of the first entry not
 *           before the boundary)
 *   cost    device int64[P+1]
 * Rows and columns stay below 2^31.  Enqueues only.  Errors: INVALID_ARG, HIP.
 */
int32_t nacho_partition_csr64(const int64_t *pos, const int32_t *crd, int64_t n_rows, int64_t n_cols, int64_t nnz,
                              int64_t P, int32_t *coord, int64_t *posn, int64_t *cost, void *hip_stream);

/*
 * Where a fused call keeps its stored partitions (Section 4.2.3: the positions
 * found by the search are kept for the assembly and compute stages).  Fills
 * `parts` (host struct) with the number of partitions the fused call `op` uses
 * for these operands and with DEVICE pointers into the workspace `ws` the call
 * was (or will be) given; the table is valid once that call has run.  Nothing
 * is launched.  One case waits: for nacho_spmul_k on DCSR operands the number of
 * partitions is a result of the call's own kernels; it is read back on
 * `hip_stream` (the stream that call was enqueued on) and the function returns
 * once the stream has reached that point.  `hip_stream` is not used otherwise.  `grain` (host, may be NULL) receives G when the call uses the
 * fixed-grain queries Q_p = min(p*G, Q_total) (SpMV and SpMM with P = 0; G is
 * in scaled units, a multiple of n_dense for SpMM), 0 when it uses
 * Q_p = floor(p*Q_total/P).  Arguments as for nacho_workspace_bytes.
 */
int32_t nacho_workspace_parts(int32_t op, const nacho_tensor *ops, int32_t k, int32_t dtype,
                              int64_t n_dense, int64_t P, void *ws, size_t ws_bytes,
                              nacho_parts *parts /* host */, int64_t *grain /* host */, void *hip_stream);

/*
 * y = A x with A in CSR (Section 4.2.2 uses this expression for the broadcast
 * rule; the cost of a partition is its number of stored non-zeros of A, the
 * dense x is only located into).  One wavefront executes one partition; a row
 * split across partitions is completed by a deterministic carry fix-up pass.
 *   A      CSR, val of type `dtype`;  x[n_cols], y[n_rows] of type `dtype`
 *   P      0 = automatic, else the minimum number of partitions
 * Every y[i] is written (exactly 0 for an empty row).
 */
int32_t nacho_spmv(const nacho_tensor *A, const void *x, void *y, int32_t dtype, int64_t P,
                   void *ws, size_t ws_bytes, void *hip_stream);

/*
 * Row-aware cost (a variant; Section 4.2.2 remarks that the non-zero count only
 * approximates the run time, and a partition of 512 one-entry rows does more
 * than one of a single 512-entry row).  Every row of A costs `row_cost` units
 * (0 .. 64) on top of its stored non-zeros, charged in front of its first
 * column: C_i(r) = pos[r] + row_cost * r, C_j(x | r) = (x > 0 ? row_cost : 0) +
 * entries of row r with column < x -- monotone and hierarchically consistent
 * (Section 3.1), so Algorithm 1 applies unchanged; a boundary may fall at
 * (r, 0), also in an empty row.  row_cost = 0 is the paper's cost.
 *   nacho_partition_rowcost   boundaries of one CSR operand, queries
 *                             floor(p * total / P) with total = nnz + row_cost * rows;
 *                             `out` as for nacho_partition (k = 1, d = 2)
 *   nacho_spmv_rowcost        y = A x on those partitions; uses
 *                             nacho_rowcost_partitions(A, dtype, row_cost, P)
 *                             partitions (at least P, and enough that a
 *                             partition's cost fits one wavefront) and needs the
 *                             workspace nacho_workspace_bytes reports for
 *                             NACHO_OP_SPMV with that partition count
 * Errors as for nacho_partition / nacho_spmv.
 */
int64_t nacho_rowcost_partitions(const nacho_tensor *A, int32_t dtype, int64_t row_cost, int64_t P);
int32_t nacho_partition_rowcost(const nacho_tensor *A, int64_t row_cost, int64_t P, const nacho_parts *out,
                                void *hip_stream);
int32_t nacho_spmv_rowcost(const nacho_tensor *A, const void *x, void *y, int32_t dtype, int64_t row_cost,
                           int64_t P, void *ws, size_t ws_bytes, void *hip_stream);

/*
 * nacho_spmv without a partition pass (a P-free, fused search-in-execute form):
 * there is no partition table; every wavefront of the executing kernel finds its
 * own two boundaries -- Algorithm 1 for one CSR operand with the fixed-grain
 * queries Q_b = min(b * G, nnz), G non-zeros a wavefront, i.e. the row with
 * pos[r] <= Q_b < pos[r+1] by a 64-ary search over pos -- and y is cleared by a
 * small fill kernel first.  Same partitions, same arithmetic and the same result
 * as nacho_spmv with P = 0; it trades the partition kernel's one pass over pos
 * for two searches per wavefront (a measured variant, not the default).
 * Workspace: nacho_workspace_bytes(NACHO_OP_SPMV, ..., P = 0).
 */
int32_t nacho_spmv_fused(const nacho_tensor *A, const void *x, void *y, int32_t dtype, void *ws, size_t ws_bytes,
                         void *hip_stream);

/*
 * nacho_spadd_k on sparse vectors without a partition pass (the fused
 * search-in-execute form of the merge path; the paper's partitions "computed in
 * parallel" with the kernel they balance, Sections 1 and 2.1): every workgroup
 * of the merge kernel searches its own two boundaries with Algorithm 1
 * (Section 3.2; wavefront 0 the lower one, wavefront 1 the upper one, equal-share
 * queries Q_p = floor(p Q* / P)) and stores them in the partition table of the
 * workspace, which nacho_workspace_parts returns as after nacho_spadd_k; two
 * small fill kernels clear the prefix-sum state and the status word first.  Same
 * partitions, same result arrays, counts and status as nacho_spadd_k; other
 * formats: NACHO_ERR_UNSUPPORTED.  A measured variant, not the default: a
 * boundary search is as long as a workgroup's whole merge, and here every
 * workgroup waits for two of them.  Workspace: nacho_workspace_bytes(NACHO_OP_SPADD, ...).
 */
int32_t nacho_spadd_fused(const nacho_tensor *ops, int32_t k, int32_t dtype, int64_t P, const nacho_sparse_out *out,
                          void *ws, size_t ws_bytes, void *hip_stream);

/*
 * nacho_spmv for callers that cannot allocate device memory or pass a workspace
 * (code under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc).  Same operation, arguments, results and status codes as nacho_spmv,
 * but the partition table and the carries live in a scratch array that is part of
 * the library's code object (one copy per GPU, nacho_static_scratch_bytes() bytes,
 * held until the process ends) instead of a caller's workspace.  The call
 * allocates and frees nothing and only enqueues.  A matrix whose partitions do
 * not fit that array (about 36 bytes per partition, i.e. per 512 non-zeros --
 * per 1024 of a large fp32 matrix with long rows --, or per requested partition
 * when P is given) is refused with
 * NACHO_ERR_TOO_LARGE before anything is launched.  All calls on one GPU share
 * the array: two calls that overlap in time on one GPU (different streams or
 * threads) race; calls on one stream are ordered and safe.  The first call on a
 * device looks the array's address up (hipGetSymbolAddress), once.
 */
int32_t nacho_spmv_static(const nacho_tensor *A, const void *x, void *y, int32_t dtype, int64_t P,
                          void *hip_stream);
size_t nacho_static_scratch_bytes(void);

/*
 * C = A B with A in CSR and B, C dense row-major (loop order i -> j -> k, dense
 * k innermost; cost of a stored non-zero = n, the broadcast extent).
 *   B[n_cols(A) x n] leading dimension ldb,  C[n_rows(A) x n] leading dimension
 *   ldc (elements); n >= 1.  The executing kernel covers 256 columns at a time
 *   (64 in a workspace sized for no more): a wider B goes through it in
 *   stretches over the same partitions (A is then read once per stretch).
 *   Any workspace sized for A, the dtype and P serves, whatever n_dense it was
 *   sized for: a large call with P = 0 that does not fit its short
 *   partitions into it runs with longer ones, and slower.
 */
int32_t nacho_spmm(const nacho_tensor *A, const void *B, int64_t n, int64_t ldb,
                   void *C, int64_t ldc, int32_t dtype, int64_t P,
                   void *ws, size_t ws_bytes, void *hip_stream);

/*
 * Z = sum_t ops[t]: the union of k sparse vectors, CSR, DCSR or COO matrices
 * or third-order CSF tensors with sorted output coordinates; coinciding values
 * are added in operand order.  Two kernels: the partition search, then one
 * merge kernel whose workgroup p stages, merges, assembles and writes
 * partition p.
 *
 * Where workgroup p writes depends on what the workgroups before it emit, and
 * it learns that inside the kernel: every workgroup publishes its counts in
 * the workspace and reads those of its predecessors, polling a bounded number
 * of times for the ones not there yet.  This relies on the GPU starting the
 * workgroups of a launch in the order of their indices, so that a workgroup
 * only ever waits for workgroups that are already running or done; HIP does
 * not promise that order, every AMD GPU so far keeps it.  Should a wait run
 * out all the same (about 2^14 polls of a few hundred nanoseconds each), the
 * workgroup writes nothing and *status becomes NACHO_ERR_HIP: the output is
 * then incomplete and the call must be repeated.  Among several conditions the
 * gravest (lowest) status wins.
 */
int32_t nacho_spadd_k(const nacho_tensor *ops, int32_t k, int32_t dtype, int64_t P,
                      const nacho_sparse_out *out, void *ws, size_t ws_bytes, void *hip_stream);

/*
 * Z = prod_t ops[t] over the INTERSECTION of the operands' stored coordinates:
 * the k-way product of sparse vectors (the three-finger loop of Section 2.1,
 * z_i = a_i b_i c_i) or the Hadamard product of k CSR matrices.  The
 * intersection is on the innermost level, so the partitions are those of
 * Algorithm 1 on the operands' non-zero counts, exactly as for nacho_spadd_k
 * (Section 3.3: only an outer intersection needs the recursive partitioning);
 * an entry is emitted when all k operands store its coordinate, its value is
 * the product in operand order.  Same arguments, output layout, status and
 * capacity rules as nacho_spadd_k (min_t nnz_t is always a sufficient cap_nnz).
 *
 * DCSR operands intersect on the OUTER level as well, and rows that not every
 * operand stores are skipped with everything below them, so the plain non-zero
 * count is the wrong cost.  The call then follows the recursive partitioning of
 * Section 3.3 (Algorithm 2): a first, separately partitioned loop intersects
 * the operands' row coordinates and memoises, for the i'-th row all operands
 * store, T[i'] = the number of entries the operands store in it; the prefix sum
 * T' is the remapped cost function C'_i(x) = T'[x]; Algorithm 1 on the
 * remapped nest (i' over the intersected rows, then the columns) gives the
 * partitions of the product.  A row of the result is stored only when it holds
 * an entry (min_t rows_t is always a sufficient cap_rows).  The stored
 * partitions (nacho_workspace_parts with NACHO_OP_SPMUL, after the call) are
 * those of the remapped nest, a CSR-like space: coord = (i', j), posn[..][0] =
 * i', posn[..][1] = the number of entries the operand stores in the
 * intersected rows before the boundary.  Workspace: nacho_workspace_bytes with
 * NACHO_OP_SPMUL.  Like every other call this one only enqueues: the size of the
 * remapped space stays on the device, the kernels after the row loop are launched
 * for upper bounds (the sizes the workspace is carved for) and read the real
 * sizes there.
 */
int32_t nacho_spmul_k(const nacho_tensor *ops, int32_t k, int32_t dtype, int64_t P,
                      const nacho_sparse_out *out, void *ws, size_t ws_bytes, void *hip_stream);

/*
 * Operators that train models, around the sparse matrices which training makes:
 * a teacher's top logits, the routing of tokens to experts.  Dense arrays are
 * row-major with a leading dimension in elements, of F32, BF16 or F16, aligned to
 * their elements (16 bytes and leading dimensions that are multiples of 16 bytes
 * are fastest); sums, softmax statistics and losses are held in 32 bits, results of
 * 16 bits are rounded once.  Matrices may have up to 2^31 - 1 rows and more than
 * 2^31 elements.  Outputs must not overlap inputs.
 *
 * nacho_distill: the distillation loss of every row against a teacher's top logits.
 *   teacher     CSR [n_rows x vocabulary], values F32: the logits stored for a row,
 *               columns as in every CSR operand; a row may store none
 *   logits      the student's, [n_rows x vocabulary], leading dimension ldl
 *   weight      device float[n_rows], a factor of every row, or NULL for ones
 *   temperature tau, 1e-30 .. 1e18 (of higher ones the square is no 32-bit number)
 * With p the softmax of a row's stored teacher logits / tau (the others have no
 * share) and q the softmax of all its student logits / tau,
 *   loss[i] = weight[i] tau^2 sum_j p_j (log p_j - log q_j)
 *   lse[i]  = log sum_v exp(z_v / tau)
 *   grad    = weight[i] tau (q - p), the gradient of the sum of all losses, leading
 *             dimension ldg; NULL: not wanted
 * Rows of weight 0 and rows without a teacher's logit above -inf have loss, lse and
 * gradient 0, whatever their logits hold.  Student logits of -inf have q = 0
 * (a loss of +inf where the teacher gives them a share).  A row with nothing but
 * -inf, or with a NaN, has no distribution: NaN.
 * The loss is a difference of sums held in 32 bits, right to about 2^-20 of their
 * size, weight[i] tau^2 (1 + log n_cols + the logits' spread / tau): its last digits
 * where a teacher stores a small part of the vocabulary.  Of one that stores nearly
 * all of it, p and q are nearly alike at a high temperature and little of the loss is
 * left (32000 columns, all stored: off by 1e-4 of it at tau = 20, 3e-3 at 100, a third
 * at 1000).  grad has no difference but q - p itself.
 * Workspace: nacho_distill_workspace_bytes (may be 0: then ws may be NULL).
 *
 * nacho_distill_grad: grad alone, from the logits and the lse of an earlier
 * nacho_distill on the same operands and temperature; weight then is the factor of
 * the loss times the gradient that arrives at it.  lse has 32 bits: q is off by a
 * factor of exp(|lse| 2^-23), no matter for logits / tau up to thousands.
 */
int32_t nacho_distill_workspace_bytes(int64_t n_rows, int64_t n_cols, int32_t dtype, size_t *bytes);
int32_t nacho_distill(const nacho_tensor *teacher, const void *logits, int64_t ldl, int32_t dtype,
                      const float *weight, float temperature, float *loss, float *lse, void *grad, int64_t ldg,
                      void *ws, size_t ws_bytes, void *hip_stream);
int32_t nacho_distill_grad(const nacho_tensor *teacher, const void *logits, int64_t ldl, int32_t dtype,
                           const float *weight, float temperature, const float *lse, void *grad, int64_t ldg,
                           void *hip_stream);

/*
 * nacho_xent: the softmax cross entropy of rows against a large vocabulary, from the
 * rows and the vocabulary's weights; the logits are never stored.
 *   x       [n_rows x inner], head [vocabulary x inner], of one type
 *   label   device integers [n_rows] of label_bytes (4 or 8) each
 *   weight  device float[n_rows], a factor of every row, or NULL for ones
 * With z_iv the product of x[i] and head[v], summed in 32 bits,
 *   lse[i]  = log sum_v exp(z_iv)
 *   loss[i] = weight[i] (lse[i] - z_i,label[i])
 * Rows whose label lies outside the vocabulary (a negative one: a position that is not
 * to be learned) and rows of weight 0 have loss, lse and gradients 0, whatever they
 * hold; they are not computed.  A logit of -inf is a probability of 0 (the loss of a
 * row whose label has it is infinite); a row with a NaN or +inf among its logits, or
 * with nothing but -inf, has no distribution: NaN.  Gradients are what their formulas
 * give: an infinite weight times a probability of 0 is a NaN in that column of grad_x.
 * nacho_xent_grad: from the lse of an earlier nacho_xent on the same operands
 *   g_iv      = weight[i] (exp(z_iv - lse[i]) - [v = label[i]]), rounded to the type for
 *               the products (of f16 after multiplication by a power of two, which the
 *               results are divided by: small probabilities do not vanish)
 *   grad_x    = g head, grad_head = g^T x, each NULL where it is not wanted
 * weight then is the factor of the loss times the gradient that arrives at it.  A NaN
 * in a row that counts is one in all of grad_head.
 * Room: the loss takes 8 bytes for every row and 128 words of the vocabulary (64 of
 * floats, 32 where a call of floats has few tiles; of up to 16 rows, for at most 1024
 * parts of it).  The gradients take g of a piece of the vocabulary, 256 MiB or 256 words
 * of it (which is more of over 524288 rows of 16 bits, 262144 of floats); and, with
 * grad_x, sums in 32 bits for every stretch of a piece, 256 MiB or rows x inner of them
 * where that is more (inner in whole eights).  Either call keeps lists of under 40 bytes
 * a row beside that, and the copies below.
 * Limits: vocabulary, inner < 2^24, and the products of every two of n_rows,
 * vocabulary and inner < 2^42.  Workspaces: nacho_xent_workspace_bytes,
 * nacho_xent_grad_workspace_bytes, of the layer with the arrays that it will have (384
 * rows and more of 16 bits that do not start at multiples of 16 bytes are copied so that
 * they do: the rows, and 256 MiB of the vocabulary's at a time).
 */
typedef struct {
    int64_t n_rows, vocabulary, inner;
    const void *x;
    int64_t ldx;
    const void *head;
    int64_t ldh;
    const void *label;
    const float *weight;
    int32_t label_bytes, dtype;
} nacho_xent_layer;
int32_t nacho_xent_workspace_bytes(const nacho_xent_layer *layer, size_t *bytes);
int32_t nacho_xent(const nacho_xent_layer *layer, float *loss, float *lse, void *ws, size_t ws_bytes, void *hip_stream);
int32_t nacho_xent_grad_workspace_bytes(const nacho_xent_layer *layer, size_t *bytes);
int32_t nacho_xent_grad(const nacho_xent_layer *layer, const float *lse, void *grad_x, int64_t ldgx, void *grad_head, int64_t ldgh,
                        void *ws, size_t ws_bytes, void *hip_stream);

/*
 * nacho_route: the routing matrix of a mixture of experts.  Every token goes to the
 * top_k experts with the largest logits (ties: the lowest index; a logit of -inf or
 * NaN is never chosen, so a token may store fewer), and the matrix comes in the two
 * compressed forms its users read, all arrays on the device:
 *   by tokens   CSR [n_tokens x n_experts]: pos[n_tokens+1], expert (columns,
 *               ascending), gate (values)
 *   by experts  its transpose's pattern: expert_pos[n_experts+1], token (ascending
 *               for every expert); slot[i] is the place there of entry i
 * expert, gate, slot and token have room for n_tokens * top_k entries; places behind
 * the last entry get expert, slot and token -1 and gate 0.
 *   gate     the softmax of all the token's logits at the chosen experts; `normalise`
 *            divides them by their sum
 *   counts   [n_experts] entries of every expert
 *   lse      [n_tokens] log of the sum of exponentials of the token's logits
 *   balance  [1] n_experts * sum_e f_e P_e, f_e the expert's share of all entries, P_e
 *            the mean of its softmax over the tokens that store an entry
 *   routed   [1] the number of these tokens
 * Tokens whose byte in `keep` (device, may be NULL) is 0 store nothing and have lse 0;
 * their logits are not read.  So has a token whose logits are all -inf.  A NaN among
 * a token's logits makes its gates, its lse and the balance loss NaN.
 * Limits: n_experts <= 1024, top_k <= min(32, n_experts), n_tokens * top_k < 2^31.
 * Workspace: nacho_route_workspace_bytes.
 *
 * nacho_route_grad: the logits' gradient from that of the gates (grad_gate, by the
 * entries' order; NULL: none) plus `balance` times that of the balance loss (in which
 * the counts are constants), from the arrays that nacho_route left.
 */
typedef struct {
    int32_t *pos, *expert;
    float *gate;
    int32_t *slot, *expert_pos, *token, *counts;
    float *lse, *balance;
    int32_t *routed;
} nacho_routing;
int32_t nacho_route_workspace_bytes(int64_t n_tokens, int64_t n_experts, int32_t top_k, size_t *bytes);
int32_t nacho_route(const void *logits, int64_t ldl, int64_t n_tokens, int64_t n_experts, int32_t dtype,
                    int32_t top_k, int32_t normalise, const uint8_t *keep, const nacho_routing *out,
                    void *ws, size_t ws_bytes, void *hip_stream);
int32_t nacho_route_grad(const void *logits, int64_t ldl, int64_t n_tokens, int64_t n_experts, int32_t dtype,
                         int32_t top_k, int32_t normalise, const nacho_routing *routing, const float *grad_gate,
                         float balance, void *grad, int64_t ldg, void *hip_stream);

/*
 * nacho_experts: one dense layer of a mixture of experts.  The slots (rows) of expert
 * e are expert_pos[e] .. expert_pos[e+1], of any number, as nacho_route leaves them:
 *   y[s] = act(x[token[s]] w[e]^T + bias[e])   for every slot s of expert e
 *   expert_pos  device int32[n_experts+1], from 0, never decreasing, at most n_slots
 *   token       device int32[n_slots], rows of x; NULL: slot s reads row s
 *   x           [n_tokens x inner], leading dimension ldx
 *   w           [n_experts][outer x inner], leading dimension ldw, experts w_stride
 *               elements apart
 *   bias        [n_experts][outer], experts bias_stride apart, or NULL
 *   act         nacho_act; gelu is x Phi(x) with the error function
 *   y           [n_slots x outer]; slots from expert_pos[n_experts] on are not written
 *   pre         [n_slots x outer] or NULL: the rows before the activation, which the
 *               way back needs unless act is NACHO_ACT_NONE
 * All of one type; products are summed in 32 bits and rounded once.
 *
 * nacho_experts_grad: from grad_y [n_slots x outer], with z the rows before the
 * activation (taken from pre, so rounded to the type) and g_s = grad_y[s] act'(z_s),
 * rounded to the type for the products, which the matrix units take it in, and not
 * for the sums of grad_bias,
 *   grad_x[s]    = g_s w[e]             [n_slots x inner], by slots: nacho_combine
 *                                       without gates sums them by tokens
 *   grad_w[e]    = sum_s g_s^T x[token[s]]
 *   grad_bias[e] = sum_s g_s
 * each NULL where it is not wanted (w, or x and token, may then be NULL); experts
 * without a slot get 0.  pre may be NULL with NACHO_ACT_NONE.
 * Workspace: nacho_experts_workspace_bytes (may be 0: then ws may be NULL).
 * Limits: n_experts <= 65536; inner, outer < 2^24.
 */
typedef enum { NACHO_ACT_NONE = 0, NACHO_ACT_RELU = 1, NACHO_ACT_GELU = 2, NACHO_ACT_SILU = 3 } nacho_act;
typedef struct {
    const int32_t *expert_pos, *token;
    int64_t n_experts, n_slots, n_tokens, inner, outer;
    const void *x;
    int64_t ldx;
    const void *w;
    int64_t ldw, w_stride;
    const void *bias;
    int64_t bias_stride;
    int32_t act, dtype;
} nacho_experts_layer;
int32_t nacho_experts_workspace_bytes(const nacho_experts_layer *layer, size_t *bytes);
int32_t nacho_experts(const nacho_experts_layer *layer, void *y, int64_t ldy, void *pre, int64_t ldpre,
                      void *hip_stream);
int32_t nacho_experts_grad(const nacho_experts_layer *layer, const void *grad_y, int64_t ldgy, const void *pre,
                           int64_t ldpre, void *grad_x, int64_t ldgx, void *grad_w, int64_t ldgw, int64_t gw_stride,
                           void *grad_bias, int64_t gb_stride, void *ws, size_t ws_bytes, void *hip_stream);

/*
 * nacho_experts_step: a whole layer of a mixture of experts for a few tokens, as a
 * program that answers needs it (nacho_route, nacho_experts twice and nacho_combine
 * in one call, for up to 64 tokens):
 *   out[t] = residual[t] + sum_i g_i (down[e_i] h_i + down.bias[e_i])   over the top_k
 *            experts e_i of token t, chosen and weighted as by nacho_route (keep,
 *            normalise, ties, -inf and NaN as there; a token that chooses nothing
 *            gets its residual, or 0)
 *   h_i    = act(up[e_i] x[t] + up.bias[e_i]), or, where gate.w is given,
 *            act(gate[e_i] x[t] + gate.bias[e_i]) (up[e_i] x[t] + up.bias[e_i]);
 *            rounded to the type
 *   logits   [n_tokens x n_experts], the router's
 *   x        [n_tokens x inner]
 *   up, gate [n_experts][hidden x inner], down [n_experts][outer x hidden]: w of a
 *            leading dimension ld, experts `stride` elements apart; bias, or NULL, of
 *            experts bias_stride apart
 *   residual [n_tokens x outer], or NULL; out may be residual itself (same leading
 *            dimension)
 * All of one type; sums, gates and the weighted sum are held in 32 bits, out is rounded
 * once.  Weights of experts that no token chose are not read.  (Arrays of 16 bits should
 * start at multiples of 4 bytes: where x, up, gate or down starts at an odd element, all
 * of them are read element by element, two to five times as slowly.)
 * Limits: n_tokens <= 64, n_experts <= 1024, top_k <= min(32, n_experts); inner, hidden,
 * outer < 2^24.  Workspace: nacho_experts_step_workspace_bytes.
 */
typedef struct {
    const void *w;
    int64_t ld, stride;
    const void *bias;
    int64_t bias_stride;
} nacho_dense;
typedef struct {
    int64_t n_tokens, n_experts, inner, hidden, outer;
    const void *logits;
    int64_t ldl;
    const uint8_t *keep;
    const void *x;
    int64_t ldx;
    nacho_dense up, gate, down;
    const void *residual;
    int64_t ldr;
    void *out;
    int64_t ldo;
    int32_t top_k, normalise, act, dtype;
} nacho_experts_step_layer;
int32_t nacho_experts_step_workspace_bytes(const nacho_experts_step_layer *layer, size_t *bytes);
int32_t nacho_experts_step(const nacho_experts_step_layer *layer, void *ws, size_t ws_bytes, void *hip_stream);

/*
 * nacho_keep8: rows kept for the way back in 8 bits, to be restored or read where the
 * other rows are.  Every 32 columns of a row (the last ones may be fewer) share a step,
 * 2^(e - 127), with e = floor(log2 of their largest magnitude) + 121, at least 0:
 *   code      [n_rows x n] int8, leading dimension ldc: the nearest whole number of
 *             steps, ties to even, -127 .. 127
 *   exponent  [n_rows x ceil(n / 32)] bytes, leading dimension lde: e
 * A value is off by half a step, a 128th of the largest of its 32 at most (by one step
 * next to that one, where it has more than 127.5).  32 columns with a NaN or an
 * infinity among them have e = 255, and are restored as NaN.
 * nacho_restore8: the values that rows in 8 bits stand for, in a type; exact in BF16,
 * and in F16 and F32 where these have the value.
 *
 * nacho_experts_keep8: nacho_experts with the rows before the activation left in 8 bits
 * (from their sums in 32 bits).
 * nacho_experts_keep8_grad: nacho_experts_grad with x, pre or both of them from rows in
 * 8 bits (kept_x, kept_pre; NULL: those of layer and pre are read, as there): the
 * gradients are those at what the codes stand for.  (relu's slope is 0 at a row that was
 * kept as 0, up to half a step above it.)
 * Workspace: nacho_experts_keep8_workspace_bytes (may be 0: then ws may be NULL).
 */
typedef struct {
    int8_t *code;
    int64_t ldc;
    uint8_t *exponent;
    int64_t lde;
} nacho_kept;
int32_t nacho_keep8(const void *x, int64_t ldx, int64_t n_rows, int64_t n, int32_t dtype, const nacho_kept *kept, void *hip_stream);
int32_t nacho_restore8(const nacho_kept *kept, int64_t n_rows, int64_t n, int32_t dtype, void *out, int64_t ldo, void *hip_stream);
int32_t nacho_experts_keep8(const nacho_experts_layer *layer, void *y, int64_t ldy, const nacho_kept *pre, void *hip_stream);
int32_t nacho_experts_keep8_workspace_bytes(const nacho_experts_layer *layer, size_t *bytes);
int32_t nacho_experts_keep8_grad(const nacho_experts_layer *layer, const nacho_kept *kept_x, const void *grad_y, int64_t ldgy,
                                 const void *pre, int64_t ldpre, const nacho_kept *kept_pre, void *grad_x, int64_t ldgx, void *grad_w,
                                 int64_t ldgw, int64_t gw_stride, void *grad_bias, int64_t gb_stride, void *ws, size_t ws_bytes,
                                 void *hip_stream);

/*
 * nacho_combine: for every token the weighted sum of its experts' rows,
 *   out[t] = residual[t] + sum_i val_i y[crd_i]   over the entries i of row t of
 *   routing   CSR [n_tokens x n_slots]: crd the slots, values F32 the gates (val
 *             NULL: ones); in the arrays of nacho_routing pos, slot and gate.  Its
 *             count is an upper bound, as many as pos[n_tokens] are read
 *   y         [n_slots x n], residual (may be NULL), out [n_tokens x n], row-major
 * Tokens without an entry get their residual, or 0.  out may be residual itself
 * (same leading dimension), for sums in place.
 *
 * nacho_combine_grad: from grad_out [n_tokens x n]
 *   grad_y[crd_i] = val_i grad_out[t]        (NULL: not wanted; slots of no entry
 *                                             are not written; no slot may be in two)
 *   grad_val[i]   = sum_c grad_out[t, c] y[crd_i, c]   (float, NULL: not wanted,
 *                                             then y may be NULL; places behind the
 *                                             last entry are not written)
 */
int32_t nacho_combine(const nacho_tensor *routing, const void *y, int64_t ldy, int64_t n, int32_t dtype,
                      const void *residual, int64_t ldr, void *out, int64_t ldo, void *hip_stream);
int32_t nacho_combine_grad(const nacho_tensor *routing, const void *y, int64_t ldy, int64_t n, int32_t dtype,
                           const void *grad_out, int64_t ldg, void *grad_y, int64_t ldgy, float *grad_val,
                           void *hip_stream);

/*
 * Debug aid, not part of the hot path: checks on the device the preconditions
 * that the other entry points rely on without looking -- pos arrays start at 0,
 * never decrease and end at the level's count; coordinates lie inside the
 * extents and ascend strictly inside every segment (coordinate lists: the
 * (row, column) pairs ascend strictly).  Enqueues only.  *status (device)
 * becomes NACHO_OK or NACHO_ERR_INVALID_ARG; info (device int64[3], may be
 * NULL) = {operand, level, position} of one violation, {-1, -1, -1} if none.
 * The return value covers what the host can see (null pointers, kinds, counts).
 */
int32_t nacho_validate(const nacho_tensor *ops, int32_t k, int32_t *status /* device */,
                       int64_t *info /* device */, void *hip_stream);

/*
 * Machine ceilings for benchmarks (not part of the hot path): kernels of known
 * traffic, timed by the caller on the same GPU in the same run.  Enqueues only.
 *   NACHO_PROBE_READ    reads `bytes` of src once (dst: 8 writable device bytes)
 *   NACHO_PROBE_COPY    copies `bytes` from src to dst
 *   NACHO_PROBE_GATHER  `gathers` independent 8-byte loads at pseudo-random places
 *                       of the first `bytes` of src (dst: 8 writable device bytes):
 *                       what a row-major CSR SpMV does to x per stored non-zero
 * src, dst: device, 16-byte aligned; bytes >= 16.
 */
typedef enum { NACHO_PROBE_READ = 0, NACHO_PROBE_COPY = 1, NACHO_PROBE_GATHER = 2 } nacho_probe_kind;
int32_t nacho_probe(int32_t kind, void *dst, const void *src, size_t bytes, int64_t gathers, void *hip_stream);

/*
 * Per-wavefront measurements (not part of the hot path; benchmarks and tests of
 * the load balance use it).  Only the instrumented build of the library
 * (libnacho_instr.so, the same sources compiled with -DNACHO_INSTRUMENT) records
 * anything; the ordinary build returns NACHO_ERR_UNSUPPORTED.  After
 * nacho_instrument(records, capacity), wavefront i of every launch of an
 * executing kernel (SpMV, SpMM: workgroup i; the merge kernel: workgroup i / 8,
 * wavefront i % 8) overwrites record i < capacity of the caller's DEVICE buffer
 * when it ends; records = NULL switches the log off.  A record is
 * nacho_instrument_record_bytes() = 40 bytes:
 *   uint64 t_begin, t_end   constant 100 MHz counter, comparable across the chip
 *   uint64 cycles           shader clock cycles between the two
 *   uint32 items, rows      stored non-zeros (merge kernel: merged places) and rows
 *                           (merge kernel: output rows started) the wavefront worked on
 *   uint32 hw_id, xcc_id    where it ran (HW_ID and XCC_ID hardware registers)
 */
int32_t nacho_instrument(void *records /* device */, int64_t capacity);
int32_t nacho_instrument_record_bytes(void);
/* Instrumented build: from now on the wait of this workgroup of the row loop of a DCSR product counts as run out (-1:
 * none), for tests of what such a call leaves. */
int32_t nacho_instrument_wait(int64_t workgroup);
/* Wavefronts per workgroup (= per partition) of the merge kernel of nacho_spadd_k / nacho_spmul_k. */
int32_t nacho_merge_wavefronts(void);

/*
 * Per-kernel timing for benchmarks (not part of the hot path).  While enabled,
 * every fused call brackets each of its kernels with HIP events on the call's
 * stream.  nacho_profile_read synchronises on those events and returns the
 * number of kernels of the last call; ms[i] and names[i] (static strings,
 * host) are filled for i < min(n, max_n).
 */
int32_t nacho_profile_enable(int32_t on);
int32_t nacho_profile_read(float *ms /* host */, const char **names /* host */, int32_t max_n);

#ifdef __cplusplus
}
#endif
#endif /* NACHO_H */
