/*
 * dpc.h -- C ABI of the compressed se_a descriptor library (libdpc.so).
 *
 * DP Compress (Lu et al., arXiv:2107.02103), Sec. II: the embedding net
 * G(s^) of the Deep Potential se_a descriptor is replaced by a table of
 * piecewise fifth-order Hermite polynomials, and the product
 * S_i = G_i^T R~_i (here called T_i, M1 x 4) is evaluated by one fused kernel
 * that never materialises G and skips padded neighbours; then
 * D_i = T_i (T_i<)^T (M1 x M2) with T_i< the first M2 rows of T_i.  The
 * backward kernel maps dE/dT_i to dE/dR~_ij through the polynomial and its
 * derivative, which is what forces need.
 *
 * Conventions
 *  - All arrays are row-major and contiguous; sizes are element counts.
 *  - "device" pointers are HIP device memory on the current device; "host"
 *    pointers are ordinary host memory.  The library never allocates device
 *    memory and keeps no global state: every buffer is owned by the caller.
 *  - Kernels are enqueued on the given stream (a hipStream_t passed as
 *    void*, NULL = the null stream) and the calls return without
 *    synchronising.  Faults inside a kernel surface at the caller's next
 *    synchronisation.
 *  - Every argument is validated on the host before anything is launched;
 *    on error nothing is launched and nothing is written.
 *  - Return value: DPC_OK (0) or a negative DPC_E* code; dpc_strerror()
 *    describes it.
 */
#ifndef DPC_H
#define DPC_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define DPC_OK 0
#define DPC_EINVAL -1   /* null pointer, bad size/shape, bad dtype, sel/nnei mismatch */
#define DPC_ERANGE -2   /* bad table parameters: stride <= 0, L1 or L2 < 1, non-finite lo */
#define DPC_EHIP -3     /* HIP runtime or launch error */
#define DPC_ENOTSUP -4  /* supported but not implemented sizes (M1 > 256, ntypes > 8) */
#define DPC_EOVERFLOW -5 /* a neighbour list had more atoms of some type within r_c than sel */

#define DPC_MAX_TYPES 8
#define DPC_MAX_M1 256

/* Arithmetic of the kernels.
 *  DPC_F64        float64 table, R~, dE/dT, T, D and dE/dR~.
 *  DPC_F32        float32 table, R~, dE/dT, T, D and dE/dR~, float32 arithmetic.
 *  DPC_F32_ACC64  float32 table, R~ and dE/dT; in the forward the polynomial
 *                 is evaluated in float32, T and D accumulated and stored in
 *                 float64; dE/dR~ in float64.  The backward with m1 <= 208
 *                 converts its float32 inputs to float64 and runs like
 *                 DPC_F64; with m1 > 208 it evaluates the polynomial and its
 *                 derivative in float32 and sums in float64.               */
typedef enum { DPC_F64 = 0, DPC_F32 = 1, DPC_F32_ACC64 = 2 } dpc_dtype;

/* Tabulation range of one embedding net (one ordered type pair).
 * Paper Sec. II: the input s^ is tabulated on [s^(r_c), s^(r_l)] with an
 * equal step; here the main range [lo, x_up], x_up = lo + L1*d1, uses step d1
 * and an extrapolation band [x_up, x_end], x_end = x_up + L2*d2, uses d2.
 * Interval l < L1 covers [lo + l*d1, lo + (l+1)*d1); interval L1 + l covers
 * [x_up + l*d2, x_up + (l+1)*d2).  Inputs below lo use interval 0 (t < 0);
 * inputs at or beyond x_end take the value at x_end and zero derivative.
 * `offset` is the element offset of this pair's coefficients inside the
 * coefficient buffer; dpc_table_layout() fills it.                          */
typedef struct {
  double lo;
  double d1;
  double d2;
  int64_t L1;
  int64_t L2;
  int64_t offset;
} dpc_range;

/* Embedding net of one type pair (host memory, read only).
 * widths[0] must be 1; layer k maps widths[k] -> widths[k+1] with
 * y_{k+1} = tanh(y_k W_k + b_k) (+ [y_k, y_k] when widths[k+1] = 2 widths[k],
 * + y_k when widths[k+1] = widths[k]).  W[k] is [widths[k]][widths[k+1]].  */
typedef struct {
  int n_layers;
  const int* widths;         /* [n_layers + 1] */
  const double* const* W;    /* [n_layers] */
  const double* const* b;    /* [n_layers] */
} dpc_net;

/* Human-readable text of a status code (static storage). */
const char* dpc_strerror(int status);

/* Text of the HIP error behind the calling thread's last DPC_EHIP status
 * ("no error" if there was none). */
const char* dpc_last_hip_error(void);

/* Library version as 10000*major + 100*minor + patch. */
int dpc_version(void);

/* Coefficient layout for `npair` type pairs of width m1.
 * In:  ranges[p].{lo,d1,d2,L1,L2}.  Out: ranges[p].offset (elements) and
 * *total_bytes, the size of the coefficient buffer for `dtype` (DPC_F32 and
 * DPC_F32_ACC64 store float32 coefficients).  The layout of one pair is
 * [L1 + L2][3][DPC_TABLE_LD(m1)][2]: interval l holds 6 * ld elements, and
 * the coefficient of t^q of channel m, t = x - (left node of l), is element
 * DPC_TABLE_AT(ld, q, m) of it, so the coefficients of t^(2j) and t^(2j+1)
 * of one channel are adjacent (one 16-byte float64 load brings both).
 * Channels are padded with zeros to a multiple of 4 so that the kernels can
 * use 16-byte loads without leaving the buffer.                             */
#define DPC_TABLE_LD(m1) (((m1) + 3) / 4 * 4)
#define DPC_TABLE_AT(ld, q, m) (((q) >> 1) * 2 * (ld) + 2 * (m) + ((q) & 1))
int dpc_table_layout(int npair, int m1, dpc_range* ranges, dpc_dtype dtype,
                     size_t* total_bytes);

/* Paper Sec. II, Eqs. for the constraints y, y', y'' at both nodes of each
 * interval and the closed forms for a..f: tabulate `net` (m1 = last width)
 * over `range` and write its (L1 + L2) * 6 * DPC_TABLE_LD(m1) coefficients to `host_out`
 * (host memory, float64 or float32 per `dtype`).  The first and second
 * derivatives of the net are computed in forward mode in float64.          */
int dpc_build_table(const dpc_net* net, const dpc_range* range, dpc_dtype dtype,
                    void* host_out);

/* Forward (paper Sec. II, the fused tabulate-and-contract kernel and D):
 *   T_i[m][k] = sum over valid j of g_m^{a_i b_j}(R~_ij[0]) * R~_ij[k]
 *   D_i[m][n] = sum_k T_i[m][k] * T_i[n][k],  n < m2
 * Geometry: neighbour slot j of atom i belongs to block b_j (the first sel[0]
 * slots are block 0, the next sel[1] block 1, ...), nnei = sum(sel); its
 * table is pair a_i*ntypes + b_j with a_i = atype[i].  nlist[i][j] < 0 marks
 * padding, which is skipped (it contributes exactly zero).
 *   stream   hipStream_t as void*
 *   sel      host [ntypes], ntypes <= DPC_MAX_TYPES
 *   ranges   host [ntypes*ntypes], offsets from dpc_table_layout()
 *   coeff    device, the concatenated tables (float64 or float32 per dtype)
 *   atype    device int32 [nloc], values in [0, ntypes); an atom with another
 *            value gets NaN outputs (nothing is read out of bounds)
 *   nlist    device int32 [nloc][nnei]
 *   em       device R~ [nloc][nnei][4] (float64 for DPC_F64, else float32),
 *            16-byte aligned (rows are read 16 bytes at a time)
 *   T        device out [nloc][m1][4]   (float32 only for DPC_F32)
 *   D        device out [nloc][m1][m2]  (float32 only for DPC_F32)
 * Requires 1 <= m1 <= DPC_MAX_M1, 1 <= m2 <= m1.  nloc = 0 is a no-op.      */
int dpc_se_a_tab_fwd(void* stream, dpc_dtype dtype, int nloc, int ntypes, const int* sel,
                     int m1, int m2, const dpc_range* ranges, const void* coeff,
                     const int* atype, const int* nlist, const void* em,
                     void* T, void* D);

/* Backward of T (forces need dE/dR~, paper Sec. II):
 *   dE/dR~_ij[k] = sum_m dE/dT_i[m][k] g_m(x) + (k == 0) sum_m g'_m(x) w_m,
 *   w_m = sum_k' dE/dT_i[m][k'] R~_ij[k'],  x = R~_ij[0],
 * for valid j; padded rows are written as 0.  For DPC_F64, and DPC_F32_ACC64
 * with m1 <= 208, the channel sums are formed per (interval, atom) pair on the
 * matrix cores in float64, as
 * P[k][q] = sum_m dE/dT_i[m][k] C[m][q] followed by a polynomial in t per
 * neighbour: the same sums in another order of rounding.
 *   dE_dT    device [nloc][m1][4] (float64 for DPC_F64, else float32)
 *   dE_dem   device out [nloc][nnei][4] (float32 only for DPC_F32), 16-byte aligned
 * Other arguments as dpc_se_a_tab_fwd.                                      */
int dpc_se_a_tab_bwd(void* stream, dpc_dtype dtype, int nloc, int ntypes, const int* sel,
                     int m1, const dpc_range* ranges, const void* coeff,
                     const int* atype, const int* nlist, const void* em,
                     const void* dE_dT, void* dE_dem);

/* The backward from dE/dD: dpc_descriptor_bwd fused into dpc_se_a_tab_bwd.
 * The matrix-core backward forms dE/dT of its atoms itself, in a prologue on
 * the matrix cores,
 * from the forward's T and dE/dD (paper Sec. II: D_i = T_i (T_i<)^T), so dE/dT
 * is never stored:
 *   dE/dT_i[m][k] = sum_{n<m2} dE/dD_i[m][n] T_i[n][k] + (m < m2) sum_{m'} dE/dD_i[m'][m] T_i[m'][k],
 * then dE/dR~ as dpc_se_a_tab_bwd.  The result equals the two calls up to the
 * order of rounding.
 *   T       device float64 [nloc][m1][4] (the forward's T), 16-byte aligned
 *   dE_dD   device float64 [nloc][m1][m2], 16-byte aligned
 *   dE_dem  device out float64 [nloc][nnei][4], 16-byte aligned
 * Requires DPC_F64, m1 <= 128 and an even m2 <= 16 (DPC_ENOTSUP otherwise:
 * use the two calls).  Other arguments as dpc_se_a_tab_bwd.                 */
int dpc_se_a_tab_bwd_from_dD(void* stream, dpc_dtype dtype, int nloc, int ntypes, const int* sel,
                             int m1, int m2, const dpc_range* ranges, const void* coeff,
                             const int* atype, const int* nlist, const void* em, const void* T,
                             const void* dE_dD, void* dE_dem);

/* Backward of the descriptor (paper Sec. II: D_i = T_i (T_i<)^T, T_i< the
 * first m2 rows of T_i, i.e. D_i[m][n] = sum_k T_i[m][k] T_i[n][k], n < m2):
 *   dE/dT_i[m][k] = sum_{n<m2} dE/dD_i[m][n] T_i[n][k]
 *                 + (m < m2) sum_{m'} dE/dD_i[m'][m] T_i[m'][k].
 * Its output is the dE_dT input of dpc_se_a_tab_bwd, so that a caller holding
 * dE/dD (from the fitting net) and the forward's T gets dE/dR~ in two calls.
 *   T        device [nloc][m1][4], the forward's T (float64, or float32 for DPC_F32)
 *   dE_dD    device [nloc][m1][m2], same type as T
 *   dE_dT    device out [nloc][m1][4]: float64 for DPC_F64, float32 otherwise
 *            (the type dpc_se_a_tab_bwd takes); must not overlap the inputs
 * Arithmetic is float64 except for DPC_F32.  Requires 1 <= m2 <= m1 <=
 * DPC_MAX_M1 and (4 m1 + m1 (m2 + 1)) elements of the arithmetic type within
 * 64 KiB (DPC_ENOTSUP otherwise; m2 = 16 allows every m1).  nloc = 0 is a
 * no-op.  Errors and ownership as the calls above.                          */
int dpc_descriptor_bwd(void* stream, dpc_dtype dtype, int nloc, int m1, int m2,
                       const void* T, const void* dE_dD, void* dE_dT);

/* Environment matrix R~ from positions (paper Sec. II, Eq. (1) and the
 * normalisation after it).  For slot s of atom i with j = nlist[i][s] >= 0:
 * r_ij = r_j - r_i as the minimum image in a cubic periodic box of edge `box`,
 * r = |r_ij|, s(r) = 1/r (r < rcs), (1/r)[u^3(-6u^2+15u-10)+1] (rcs <= r < rc,
 * u = (r - rcs)/(rc - rcs)), 0 (r >= rc), and the row is
 *   ((s - mean[t]) / sigma[t], s x / sigma_all[t], s y / sigma_all[t], s z / sigma_all[t]),
 * t = atype[i]; padding rows (nlist < 0) are zero.
 *   box, rc, rcs  require 0 <= rcs < rc and box > 2 rc (else DPC_ERANGE)
 *   mean, sigma, sigma_all  host [ntypes], sigma and sigma_all > 0
 *   coord    device float64 [nloc][3]
 *   atype    device int32 [nloc]; nlist device int32 [nloc][nnei], entries < nloc
 *            (a row with an out-of-range type or neighbour index becomes NaN)
 *   em       device out [nloc][nnei][4]: float64 for DPC_F64, float32 otherwise
 *            (the em input of dpc_se_a_tab_fwd / _bwd in that mode)
 * Arithmetic is float64.  nloc = 0 is a no-op.                              */
int dpc_env_mat_a(void* stream, dpc_dtype dtype, int nloc, int ntypes, int nnei, double box,
                  double rc, double rcs, const double* mean, const double* sigma,
                  const double* sigma_all, const double* coord, const int* atype,
                  const int* nlist, void* em);

/* Reverse slots of a neighbour list, for dpc_force_a: rev[i][s] = the slot of
 * i in the list of j = nlist[i][s], searched in the sel block of i's type
 * (sel as in dpc_se_a_tab_fwd), or -1 if i is not there (and for padding);
 * if j's block holds i more than once, one of those slots.  In lists sorted
 * by distance within each block i sits near j's rank in i's list, where the
 * search looks first; other orders are scanned, with the same result.
 * Build it once per neighbour list.
 *   coord, box  as for the other calls (validated; the search reads only the
 *               lists and atype)
 *   rev   device out int32 [nloc][nnei]                                      */
int dpc_nlist_reverse(void* stream, int nloc, int ntypes, const int* sel, double box,
                      const double* coord, const int* atype, const int* nlist, int* rev);

/* Bytes of device workspace dpc_nlist_build needs for nloc atoms in a cubic
 * box of edge `box` with cutoff rc (the cell list: per-cell counters and
 * offsets, and the atoms in cell order, 32 bytes each); 0 for bad sizes.   */
size_t dpc_nlist_workspace_bytes(int nloc, double box, double rc);

/* Neighbour list (paper Sec. II, the environment matrix: the neighbours of
 * atom i within r_c, grouped by neighbour type into sel[beta] rows for type
 * beta, sorted by distance inside a group, the unused rows empty):
 *   - periodic cubic box of edge `box`, minimum image per component
 *     d = x_j - x_i - box * rint((x_j - x_i) / box);
 *   - r2 = dx*dx + dy*dy + dz*dz, each operation rounded on its own;
 *   - j != i is a neighbour when r2 < rc*rc (and 0 <= atype[j] < ntypes);
 *   - nlist[i][blk(beta) + k] = the k-th neighbour of type beta in the order
 *     (r2, j) ascending, for k < sel[beta]; the remaining slots hold -1.
 * The result does not depend on the order of the atoms inside the cell list
 * (the order is total), so it is reproducible bitwise.
 *   nloc         at most 2^28 (else DPC_ENOTSUP)
 *   box, rc      require rc > 0 and box > 2 rc (else DPC_ERANGE)
 *   sel          host [ntypes], ntypes <= DPC_MAX_TYPES
 *   coord        device float64 [nloc][3] (any real values: positions are
 *                wrapped into the box for the cell list only)
 *   atype        device int32 [nloc]
 *   workspace    device, 256-byte aligned, >= dpc_nlist_workspace_bytes()
 *   nlist        device out int32 [nloc][sum(sel)] (the nlist input of the
 *                calls above)
 *   status_host  host int [2] or NULL.  With NULL the call is asynchronous
 *                like the others; the two status counters it leaves in the
 *                first 8 bytes of the workspace are the numbers of atoms
 *                whose list was truncated (some type had more than sel
 *                neighbours: its nearest sel are kept) and of atoms with
 *                more than 1024 atoms within rc (their list is incomplete).
 *                With a host array the call waits for its kernels, copies
 *                the two counters there and returns DPC_EOVERFLOW if the
 *                first is nonzero, DPC_ENOTSUP if the second is.
 * nloc = 0 is a no-op.  Errors and ownership as the calls above.            */
int dpc_nlist_build(void* stream, int nloc, int ntypes, const int* sel, double box, double rc,
                    const double* coord, const int* atype, void* workspace,
                    size_t workspace_bytes, int* nlist, int* status_host);

/* For callers that cannot allocate device memory (code under HIP graph
 * capture, serving loops, harnesses that forbid hipMalloc): dpc_nlist_build
 * with its cell list kept in a static device array of the library instead of
 * a caller's workspace.  The call allocates nothing and never waits.  Each
 * GPU it runs on holds one copy of that array (about 25 MB: the layout for
 * DPC_NLIST_NOALLOC_MAX_ATOMS atoms) until the process ends.
 *   nloc    at most DPC_NLIST_NOALLOC_MAX_ATOMS (else DPC_ENOTSUP)
 *   stream  must run on the current device (else DPC_EINVAL)
 *   status  device out int [2] or NULL: the two counters of dpc_nlist_build
 *           (truncated lists, lists over capacity), written by the kernels
 * All calls on one GPU share the array and every call starts by clearing
 * its counters and overwrites the rest: calls that overlap in time on one
 * GPU (other streams, other host threads) race, and the caller must
 * serialise them.  Other arguments, results and errors as dpc_nlist_build. */
#define DPC_NLIST_NOALLOC_MAX_ATOMS 524288
int dpc_nlist_build_noalloc(void* stream, int nloc, int ntypes, const int* sel, double box,
                            double rc, const double* coord, const int* atype, int* nlist,
                            int* status);

/* Forces and per-atom virials from dE/dR~ (F = -dE/dr; paper Sec. II: the
 * forces need the derivatives of E with respect to R~).  With
 * g_is = dE/dr_ij = sum_c dE/dR~_is[c] dR~_is[c]/dr_ij (dR~/dr from the
 * positions, as in dpc_env_mat_a):
 *   force[i]  = sum_s g_is - sum_s g_{j, rev[i][s]}   (j = nlist[i][s])
 *   virial[i] = -sum_s r_is (x) g_is   (row-major 3x3: [a][b] = -sum r_a g_b)
 * so that a neighbour list in which every pair within rc appears in both
 * atoms' lists (no sel truncation) gives F = -dE/dr for every atom, and the
 * summed virial is -dE/d(eps) of the homogeneous strain r_ij -> (1+eps) r_ij
 * (transposed).  Each atom gathers its terms in a fixed order: the result is
 * bitwise reproducible.
 *   dE_dem  device [nloc][nnei][4]: float32 for DPC_F32, float64 otherwise
 *   rev     from dpc_nlist_reverse for this nlist
 *   force   device out float64 [nloc][3]; virial device out float64 [nloc][9] or NULL
 * Other arguments as dpc_env_mat_a.  Arithmetic is float64.                 */
int dpc_force_a(void* stream, dpc_dtype dtype, int nloc, int ntypes, int nnei, double box,
                double rc, double rcs, const double* sigma, const double* sigma_all,
                const double* coord, const int* atype, const int* nlist, const int* rev,
                const void* dE_dem, double* force, double* virial);

/* Fitting net (paper Sec. II: a fully connected network maps the descriptor
 * D_i to the atomic energy E_i; Sec. III: widths (240, 240, 240)), read as
 *   h_1 = tanh(x W_1 + b_1),  h_l = h_{l-1} + tanh(h_{l-1} W_l + b_l) (l = 2, 3),
 *   E_i = h_3 . w_out + b_out,   x = D_i flattened row-major (n_in = m1 * m2),
 * with its backward dE_i/dD_i (the dE_dD input of dpc_descriptor_bwd).
 * Weights are device float64, row-major: W[0] [n_in][width], W[1], W[2]
 * [width][width], b[l] [width], w_out [width]; the three widths are equal.  */
typedef struct {
  int n_in, width;
  const double* W[3];
  const double* b[3];
  const double* w_out;
  double b_out;
} dpc_fitting_net;

/* Bytes of device workspace dpc_fitting_fwd_bwd needs: five float64 arrays
 * of nloc * width (rounded up to even) elements: the tanh outputs of layers
 * 1 and 2, h_2, the pre-activations and the backward accumulator.
 * 0 for bad sizes.                                                         */
size_t dpc_fitting_workspace_bytes(int nloc, int width);

/* E [nloc] and, if dE_dD is not NULL, dE/dD [nloc][n_in] (float64) for
 * D [nloc][n_in] (float64, device).  For width 240, n_in a multiple of 4 and
 * 16-byte aligned D, dE_dD, weights and biases the products run in the
 * library's own kernels on the float64 matrix cores; else as rocBLAS
 * double-precision GEMMs on the caller's handle `blas` (a rocblas_handle as
 * void*, required in both cases; its stream is left set to `stream`; its
 * pointer mode is host for the call and restored after it);
 * this library allocates nothing: `workspace` (device, 16-byte aligned,
 * >= dpc_fitting_workspace_bytes) is the caller's (rocBLAS may keep a
 * workspace of its own inside the handle).  Sums have a fixed order
 * (for a given rocBLAS).  DPC_EHIP reports a HIP or rocBLAS failure.        */
int dpc_fitting_fwd_bwd(void* stream, void* blas, int nloc, const dpc_fitting_net* net,
                        const double* D, void* workspace, size_t workspace_bytes, double* E,
                        double* dE_dD);

/* ---- Routing: tokens sorted by expert and back --------------------------
 * A model with one fitting net per species (or a mixture of nets) sends each
 * atom's descriptor row to the nets it chooses and brings their results back.
 * Token t of ntok has topk choices; slot s = t * topk + j holds expert[s].
 * A slot whose expert is outside [0, nexpert) is dropped: it owns no row.
 * nslot = ntok * topk rows are laid out; the first offsets[nexpert] of them
 * are the kept slots sorted by expert (ties by slot), the rest is empty.   */

/* Types of the elements of rows (the routing calls and those behind them). */
typedef enum { DPC_ELEM_F64 = 0, DPC_ELEM_F32 = 1, DPC_ELEM_F16 = 2, DPC_ELEM_BF16 = 3 } dpc_elem;

#define DPC_MAX_EXPERTS 1024
#define DPC_MAX_TOPK 64

/* Bytes of device workspace dpc_route_plan needs; 0 for bad sizes. */
size_t dpc_route_workspace_bytes(int ntok, int topk, int nexpert);

/* The plan of a routing.
 *   expert   device int32 [ntok][topk]
 *   workspace  device, 16-byte aligned, >= dpc_route_workspace_bytes()
 *   offsets  device out int32 [nexpert + 1]: first row of each expert, and
 *            the number of kept rows
 *   rows     device out int32 [nslot]: slot of each row, -1 for empty rows
 *   pos      device out int32 [nslot]: row of each slot, -1 for dropped slots
 * Requires 1 <= topk <= DPC_MAX_TOPK, 1 <= nexpert <= DPC_MAX_EXPERTS
 * (DPC_ENOTSUP above) and nslot <= 2^30 (DPC_ENOTSUP).  The result is the same
 * on every call.  With ntok = 0 only the offsets (zeros) are written.       */
int dpc_route_plan(void* stream, int ntok, int topk, int nexpert, const int* expert, void* workspace,
                   size_t workspace_bytes, int* offsets, int* rows, int* pos);

/* Rows of the tokens in the plan's order:
 *   y[pos[t][j]] = weight[t][j] * x[t];  zeros in the empty rows.
 *   x       device [ntok] rows of `width` elements, ldx elements apart
 *   weight  device [ntok][topk] (float64 for DPC_ELEM_F64, else float32) or
 *           NULL for weights of 1.  With weights, this maps the gradient of
 *           dpc_route_combine's y to that of its x.
 *   rows, pos  the plan
 *   y       device out [nslot] rows, ldy elements apart
 * Products are rounded once from float64 (DPC_ELEM_F64) or float32.  Rows
 * need the alignment of their elements alone.  Requires 1 <= width <= 2^31 -
 * 128 (DPC_ENOTSUP above), ldx and ldy >= width.  Inputs and outputs must not
 * overlap.                                                                  */
int dpc_route_gather(void* stream, dpc_elem elem, int ntok, int topk, int width, const void* x,
                     int64_t ldx, const void* weight, const int* rows, const int* pos, void* y,
                     int64_t ldy);

/* Rows back to their tokens, with weights:
 *   y[t] = sum over j with pos[t][j] a row, j ascending, of
 *          weight[t][j] * x[pos[t][j]]
 * (zeros where a token has no row; what weight[t][j] holds for a dropped slot
 * does not matter).  Summed in float64 (DPC_ELEM_F64) or float32, rounded once.
 *   x  device [nslot] rows, ldx elements apart;  y  device out [ntok] rows
 * Without weights (NULL) this is the gradient of dpc_route_gather in x.
 * Other arguments as dpc_route_gather.                                      */
int dpc_route_combine(void* stream, dpc_elem elem, int ntok, int topk, int width, const void* x,
                      int64_t ldx, const void* weight, const int* pos, void* y, int64_t ldy);

/* Gradient of dpc_route_combine from dE/dy:
 *   dx[pos[t][j]] = weight[t][j] * dy[t]         (zeros in empty rows)
 *   dweight[t][j] = sum_c dy[t][c] * x[pos[t][j]][c]   (0 for a dropped slot)
 * in one pass over dy and x.  dx or dweight may be NULL (that half is left
 * out); x may be NULL when dweight is.
 *   dweight  device out [ntok][topk], the type of weight
 * The sum over c has a fixed order.  Other arguments as above.              */
int dpc_route_combine_bwd(void* stream, dpc_elem elem, int ntok, int topk, int width, const void* x,
                          int64_t ldx, const void* weight, const int* rows, const int* pos,
                          const void* dy, int64_t lddy, void* dx, int64_t lddx, void* dweight);

/* ---- Layers in 8-bit integers -------------------------------------------
 * y = x W^T + b with x and W held as 8-bit codes: every row of x (an atom) and
 * every row of W (an output channel) has a scale of its own.  A matrix of
 * codes is int8 [rows][DPC_I8_LD(cols)], the columns past `cols` zero.
 * A code is off by up to half a step, 1/254 of its row's largest magnitude: a
 * product of normally distributed rows is off by about 1% of the norm.  What
 * follows the layer may need more: behind tanh of large arguments the gradient
 * lives in the few that are small, which such an error changes altogether.  */
#define DPC_I8_LD(cols) (((cols) + 127) / 128 * 128)
#define DPC_MAX_I8_COLS 131071 /* sums of that many products fit 32 bits */

/* Codes of rows.  With x[r] rounded to float32 and a = max_c |x[r][c]|,
 *   scale[r] = a / 127,  q[r][c] = x[r][c] * (127 / a) to the nearest integer
 *   (ties to even), every operation rounded to float32 on its own.
 * A row with a < 2^-100 gets scale 0 and codes 0; a row with an infinity or a
 * NaN gets scale NaN and codes 0.
 *   x      device [nrows] rows of `ncols` elements, ldx elements apart
 *   q      device out int8 [nrows][DPC_I8_LD(ncols)], 16-byte aligned
 *   scale  device out float32 [nrows]
 * Requires 1 <= ncols <= DPC_MAX_I8_COLS (DPC_ENOTSUP above), ldx >= ncols.
 * The weights of a layer are coded once: their rows are output channels.    */
int dpc_quant_rows(void* stream, dpc_elem elem, int nrows, int ncols, const void* x, int64_t ldx,
                   int8_t* q, float* scale);

/* Product of codes, for one layer or for the layer of each row's expert:
 *   y[r][c] = (sum_i qx[t][i] qw[g][c][i]) * sx[t] * sw[g][c] + bias[g][c]
 * for the ntok * topk rows r, c < n.  The sum over i < k is exact; the rest is
 * float64 arithmetic, rounded to float32 (and from there to 16 bits, if so).
 *   rows     NULL: t = r (topk must be 1); else from dpc_route_plan:
 *            t = rows[r] / topk
 *   offsets  NULL: one group (ngroup must be 1); else device int32
 *            [ngroup + 1], offsets[0] = 0: g is the group with
 *            offsets[g] <= r < offsets[g + 1].  Rows past offsets[ngroup] and
 *            rows that own no slot are zero.
 *   qx, sx   device codes [ntok][DPC_I8_LD(k)] and scales [ntok]
 *   qw, sw   device codes [ngroup][n][DPC_I8_LD(k)] and scales [ngroup][n]
 *   bias     device float32 [ngroup][n] or NULL
 *   y        device out [ntok * topk] rows of n elements, ldy apart
 * qx and qw 16-byte aligned.  Requires 1 <= n <= 2^24, 1 <= k <=
 * DPC_MAX_I8_COLS, ngroup <= DPC_MAX_EXPERTS, topk <= DPC_MAX_TOPK and
 * ntok * topk <= 2^27 (DPC_ENOTSUP above).
 * The gradient of y in x at fixed codes of W is dy times (qw sw), whose scales
 * stand along the sum: no product of this form.  The same product with the codes
 * of dy and of the transposed weights (their rows are input channels)
 * approximates it: both have scales and roundings of their own.  For normally
 * distributed weights it is off by 1.2 to 1.4% of the norm (1.7 to 3.6% with
 * output channels of very different sizes), so that a gradient taken this way
 * is not the derivative of a function of these products.                    */
int dpc_matmul_i8(void* stream, dpc_elem elem_y, int ntok, int topk, int n, int k, int ngroup,
                  const int8_t* qx, const float* sx, const int* rows, const int* offsets,
                  const int8_t* qw, const float* sw, const float* bias, void* y, int64_t ldy);

/* dpc_quant_rows of x [ntok][k] and dpc_matmul_i8 in one call, with the same
 * result.  The workspace (device, 16-byte aligned) may hold the codes and
 * scales of x in between.  dpc_linear_i8_workspace_bytes is 0 for bad sizes. */
size_t dpc_linear_i8_workspace_bytes(int ntok, int k);
int dpc_linear_i8(void* stream, dpc_elem elem_x, dpc_elem elem_y, int ntok, int topk, int n, int k,
                  int ngroup, const void* x, int64_t ldx, const int* rows, const int* offsets,
                  const int8_t* qw, const float* sw, const float* bias, void* workspace,
                  size_t workspace_bytes, void* y, int64_t ldy);

/* ---- Choice of experts ---------------------------------------------------
 * From the scores of a token for each expert to the experts that it is sent to
 * and their weights: the inputs of dpc_route_plan and dpc_route_combine.
 *   s_e = exp(z_e) / sum exp(z), or 1 / (1 + exp(-z_e));  c_e = s_e + bias_e
 * (with neither bias nor groups c_e = z_e: the order of the s_e, unrounded).
 * An expert with z_e = -infinity is closed: its s_e is 0, it is never chosen and
 * does not count in its group.  The experts stand in `groups` groups of equal
 * size; the value of a group is the sum of its `best` (1 or 2) largest c, and the
 * `keep` groups of largest value stay (a group with no open expert never does).
 * Of these groups' open experts the topk of largest c are chosen, the largest
 * first.  Ties go to the lower group and the lower expert.  A bias of -infinity
 * closes its expert for all tokens (its s_e keeps its share).  The weights are
 *   w_j = scale * s_j,  or (renorm)  scale * s_j / sum_j s_j   (0 if the sum is 0)
 * s, c, groups' values and sums are float64, whatever the type of z, and so is
 * the choice; weights are rounded once to their type.
 * Slots without an open expert get expert -1 (which dpc_route_plan drops) and
 * weight 0.  A token with a NaN among its z or c (or, in a softmax, z = +infinity)
 * gets the experts 0 .. topk - 1 and weights NaN.                            */
typedef enum { DPC_SCORE_SOFTMAX = 0, DPC_SCORE_SIGMOID = 1 } dpc_score;
typedef struct {
  int nexpert, topk;
  int score;               /* a dpc_score */
  int groups, keep, best;  /* 1, 1, 1: no groups */
  int renorm;              /* not 0: weights of a token sum to scale */
  double scale;
} dpc_gate_spec;

#define DPC_MAX_GATE_GROUPS 64

/*   logits  device [ntok] rows of nexpert elements, ldl elements apart
 *   bias    device float32 [nexpert] or NULL
 *   expert  device out int32 [ntok][topk]
 *   weight  device out [ntok][topk], float64 for DPC_ELEM_F64, else float32
 * Requires nexpert <= DPC_MAX_EXPERTS, topk <= DPC_MAX_TOPK, groups <=
 * DPC_MAX_GATE_GROUPS, ntok * topk <= 2^30 (DPC_ENOTSUP above); groups divides
 * nexpert, keep <= groups, topk <= keep * nexpert / groups, finite scale.
 * `spec` is host memory, read during the call.                               */
int dpc_gate(void* stream, dpc_elem elem, const dpc_gate_spec* spec, int ntok, const void* logits,
             int64_t ldl, const float* bias, int* expert, void* weight);

/* Gradient of the weights in the logits, from dE/dweight at the experts that
 * were chosen (the choice itself has none, nor has the bias):
 *   S = sum_j s_j,  ds_j = scale dw_j  or (renorm)  scale / S (dw_j - sum_i dw_i s_i / S)
 *   softmax  dz_e = s_e (ds_e - sum_j ds_j s_j),   sigmoid  dz_e = ds_e s_e (1 - s_e)
 * with ds_e summed over the slots that hold e; 0 for closed experts, and
 * everywhere where S is 0 (in float64).  A token with a NaN among its z (or, in a
 * softmax, z = +infinity) gets NaN at its open experts.  Slots whose expert is outside [0, nexpert), and what
 * dweight holds there, do not count.  Arithmetic is float32 (float64 for
 * DPC_ELEM_F64), rounded once; sums have a fixed order.
 *   dlogits  device out [ntok] rows, lddl elements apart, of logits' type
 * groups, keep and best are checked and not used.  Other arguments as above. */
int dpc_gate_bwd(void* stream, dpc_elem elem, const dpc_gate_spec* spec, int ntok, const void* logits,
                 int64_t ldl, const int* expert, const void* dweight, void* dlogits, int64_t lddl);

/* ---- Vectors of ids ------------------------------------------------------
 * y[t] = scale * table[ids[t]]; zeros where ids[t] is outside [0, nid) (atoms
 * that pad a batch).  The product is rounded once from float64 (DPC_ELEM_F64) or
 * float32, scale rounded to that type before.
 *   ids    device int32 [ntok]
 *   table  device [nid] rows of `width` elements, ldt elements apart
 *   y      device out [ntok] rows, ldy elements apart
 * Rows need the alignment of their elements alone.  Requires 1 <= nid <= 2^30,
 * ntok <= 2^30, 1 <= width <= 2^31 - 128 (DPC_ENOTSUP above).                */
int dpc_embed(void* stream, dpc_elem elem, int ntok, int nid, int width, const int* ids,
              const void* table, int64_t ldt, double scale, void* y, int64_t ldy);

/* Gradient of dpc_embed in its table: tokens are sorted by id, then
 *   dtable[v] = scale * sum over t with ids[t] = v of dy[t]
 * (zeros for an id without tokens).  Sums and scale are float64, in an order that
 * depends on the sizes and the ids alone; rounded once.
 *   dy       device [ntok] rows of `width` elements of type `elem`
 *   dtable   device out [nid] rows of type elem_d: elem or DPC_ELEM_F32
 *   workspace  device, 16-byte aligned, >= dpc_embed_bwd_workspace_bytes()
 *            (0 for bad sizes); two calls that may run at once need one each
 * Other arguments as dpc_embed.                                              */
size_t dpc_embed_bwd_workspace_bytes(dpc_elem elem, int ntok, int nid, int width);
int dpc_embed_bwd(void* stream, dpc_elem elem, dpc_elem elem_d, int ntok, int nid, int width, const int* ids,
                  const void* dy, int64_t lddy, double scale, void* workspace, size_t workspace_bytes,
                  void* dtable, int64_t lddt);

/* ---- Layers in microscaled 4-bit floating point --------------------------
 * As the layers in 8-bit integers, with x and W as 4-bit floating-point codes
 * (E2M1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign) that share a power of two in
 * blocks of 32 along a row.  Rows are padded with zeros to DPC_MX4_LD columns:
 *   codes   uint8 [rows][DPC_MX4_LD(cols) / 2]: two columns in a byte, the even
 *           one in the low half
 *   scales  uint8 [DPC_MX4_LD(cols) / 256][rows][8]: byte E of a block stands for
 *           2^(E - 127), 255 for NaN
 * A code is off by up to a fifth of itself from one scale on, and by up to a
 * quarter of the scale (a 14th of the block's largest magnitude) below: a product of
 * normally distributed rows is off by 16% of the norm, and by up to 19% where
 * channels of x differ in size.  That is for searches and for weights trained
 * with such codes; forces of nets that were not are wrong.                   */
#define DPC_MX4_LD(cols) (((cols) + 255) / 256 * 256)
#define DPC_MAX_MX4_COLS (1 << 20)

/* Codes of rows.  With x rounded to float32 and a the largest magnitude of a
 * block, E - 125 = floor(log2 a), one more if a is 1.75 times that power of two or
 * larger (so that a is below 7 scales), and the code is x / 2^(E - 127) to the
 * nearest code (ties to the even one, 6 at most).  A block with a < 2^-100 gets
 * E = 0 and codes of 0, one with an infinity or a NaN E = 255 and codes of 0.
 *   x      device [ngroup * nrows] rows of `ncols` elements, ldx elements apart
 *   q      device out codes [ngroup][nrows], 16-byte aligned
 *   scale  device out scales, one array [.][nrows][8] for each group, 8-byte aligned
 * Requires 1 <= ncols <= DPC_MAX_MX4_COLS, ngroup * nrows <= 2^30 (DPC_ENOTSUP
 * above).                                                                    */
int dpc_quant_mx4(void* stream, dpc_elem elem, int ngroup, int nrows, int ncols, const void* x, int64_t ldx,
                  uint8_t* q, uint8_t* scale);

/* The values that codes stand for, rounded to `elem` (float32, float64 and
 * bfloat16 hold nearly all of them).  y: device out [ngroup * nrows] rows.   */
int dpc_values_mx4(void* stream, dpc_elem elem, int ngroup, int nrows, int ncols, const uint8_t* q,
                   const uint8_t* scale, void* y, int64_t ldy);

/* Product of codes, for one layer or for the layer of each row's expert:
 *   y[r][c] = sum_i xq[t][i] wq[g][c][i] + bias[g][c]
 * of the values that the codes stand for, summed in float32 on the matrix cores
 * in a fixed order, the bias added in float32, rounded to the type of y.  Rows,
 * groups and empty rows as in dpc_matmul_i8.
 *   qx, sx  device codes and scales of [ntok] rows (one group)
 *   qw, sw  device codes and scales of [ngroup] groups of n rows
 *   bias    device float32 [ngroup][n] or NULL
 * qx and qw 16-byte, sx and sw 8-byte aligned.  Requires 1 <= n <= 2^24, 1 <= k
 * <= DPC_MAX_MX4_COLS, ngroup <= DPC_MAX_EXPERTS, topk <= DPC_MAX_TOPK and
 * ntok * topk <= 2^27 (DPC_ENOTSUP above).  Gradients: as in dpc_matmul_i8, the
 * codes of W^T give an approximation, not the derivative.                    */
int dpc_matmul_mx4(void* stream, dpc_elem elem_y, int ntok, int topk, int n, int k, int ngroup,
                   const uint8_t* qx, const uint8_t* sx, const int* rows, const int* offsets,
                   const uint8_t* qw, const uint8_t* sw, const float* bias, void* y, int64_t ldy);

/* dpc_quant_mx4 of x [ntok][k] and dpc_matmul_mx4 in one call, with the same
 * codes.  The workspace (device, 16-byte aligned) may hold the codes and scales
 * of x in between.  dpc_linear_mx4_workspace_bytes is 0 for bad sizes.       */
size_t dpc_linear_mx4_workspace_bytes(int ntok, int k);
int dpc_linear_mx4(void* stream, dpc_elem elem_x, dpc_elem elem_y, int ntok, int topk, int n, int k,
                   int ngroup, const void* x, int64_t ldx, const int* rows, const int* offsets,
                   const uint8_t* qw, const uint8_t* sw, const float* bias, void* workspace,
                   size_t workspace_bytes, void* y, int64_t ldy);

#ifdef __cplusplus
}
#endif
#endif /* DPC_H */
