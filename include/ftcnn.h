/*
 * ftcnn.h — checksum-protected convolution on AMD MI355X (gfx950).
 *
 * Implements the algorithm-based fault tolerance of FT-CNN (Zhao et al.,
 * "FT-CNN: Algorithm-Based Fault Tolerance for Convolutional Neural
 * Networks", arXiv 2003.12203) for one convolution layer:
 *
 *   encode    input checksums Cd1, Cd2 of D and Cw1, Cw2 of W     (Sec. 3.2)
 *   conv_fwd  the layer itself, O = D (x) W                       (Sec. 2.1, eq. 1)
 *   checksum  output checksums Co1..Co7 as convolutions of        (Sec. 3.2)
 *   _conv     checksum blocks
 *   verify    CoC-D detection: So5 = sum_{n,m} O_nm against Co5    (Sec. 3.6, Sec. 4.3)
 *   correct   the correction chain CoC -> RC -> ClC -> FC          (Sec. 3.3-3.6, 4.1, 4.3)
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * - Every tensor pointer is a DEVICE pointer owned by the caller.  The
 *   library never allocates, frees or retains device memory; scratch comes
 *   from a caller-supplied workspace of ftcnn_workspace_bytes() bytes
 *   (256-byte aligned).
 * - Layouts are dense row-major: D [n][ch][h][w], W [m][ch/groups][r][s]
 *   (W [m][ch][r][s] when groups = 1), O [n][m][E][F] with
 *   E = floor((h + 2*pad - r)/stride) + 1 and
 *   F = floor((w + 2*pad - s)/stride) + 1.  D, W and O share the dtype of the
 *   descriptor (fp32, or bf16 as raw 16-bit patterns); accumulation is fp32 in
 *   the convolution and fp64 everywhere on the checksum side, except that a
 *   bf16 layer's convolution epilogue adds each run of 16 filters of a pixel in
 *   fp32 (every term exact; at most 15 roundings of 2^-24 a run) before fp64.
 * - Checksum arrays are float64: Cd1, Cd2 [ch][h][w]; Cw1, Cw2 [ch][r][s];
 *   Co5, Co6, Co7, So5, So6, So7, Q5 [E][F]; Co1, Co3 [m][E][F];
 *   Co2, Co4 [n][E][F].
 * - Block index weights: Cd2 = sum_n (n + wbase) D_n, Cw2 = sum_m (m + wbase) W_m,
 *   and the weighted summations use the same weights.  wbase = 0 is the
 *   paper's definition (Sec. 3.2).
 * - Calls taking a stream are asynchronous on it and never synchronize it.
 *   The shape and size queries are host-only.
 * - Return value: FTCNN_OK (0) or a negative FTCNN_E_* code; on error the
 *   stream receives no work and ftcnn_last_error() describes the failure.
 *   A detected soft error is NOT an error: it is reported in ftcnn_report.
 * - Functions are thread-safe for distinct streams and distinct buffers.
 *   Calls sharing a workspace or report must be ordered on one stream.
 */
#ifndef FTCNN_H
#define FTCNN_H

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
    FTCNN_OK = 0,
    FTCNN_E_ARG = -1,          /* null pointer or inconsistent argument          */
    FTCNN_E_SHAPE = -2,        /* non-positive or oversized dimension            */
    FTCNN_E_DTYPE = -3,        /* dtype not FTCNN_F32 / FTCNN_BF16               */
    FTCNN_E_WORKSPACE = -4,    /* workspace missing or misaligned                */
    FTCNN_E_HIP = -5,          /* kernel launch failed                           */
    FTCNN_E_UNSUPPORTED = -6   /* a combination that is not built, e.g. a grouped
                                  layer without a workspace, a pooling window
                                  other than 1/1, 2/2 and 3/2                     */
};

typedef enum { FTCNN_F32 = 0, FTCNN_BF16 = 1 } ftcnn_dtype;

/* One convolution layer (notation of Sec. 2.1, Table 1: N, Ch, H, M, R, U). */
typedef struct {
    int32_t n, ch, h, w;     /* D [n][ch][h][w]                                  */
    int32_t m, r, s;         /* W [m][ch/groups][r][s]                           */
    int32_t stride, pad;     /* U of eq. (1); zero padding on every side         */
    int32_t groups;          /* G >= 1 dividing ch and m (Sec. 5.2): filter m
                                sees channels [(m / (m_total/G)) * ch/G, + ch/G).
                                G > 1 needs the workspace in every call that
                                reads W (the convolution runs on the
                                block-diagonal expansion of W kept there):
                                ftcnn_conv_fwd and Co1/Co3 of
                                ftcnn_checksum_conv return FTCNN_E_UNSUPPORTED */
    int32_t dtype;           /* ftcnn_dtype of D, W and O                        */
    int32_t wbase;           /* block index weight offset, 0 or 1                */
} ftcnn_conv_desc;

/* Device pointers to the float64 checksum arrays of one layer (Sec. 3.2).
 * A call reads or writes only the members its description names; the others
 * may be NULL.  The struct itself lives in host memory. */
typedef struct {
    double *cd1, *cd2;              /* [ch][h][w]   input checksums of D   */
    double *cw1, *cw2;              /* [ch][r][s]   input checksums of W   */
    double *co5, *co6, *co7;        /* [E][F]       checksum of checksums  */
    double *so5, *so6, *so7, *q5;   /* [E][F]       summations of O, and sqrt(sum O^2) */
    double *co1, *co3;              /* [m][E][F]    row checksums          */
    double *co2, *co4;              /* [n][E][F]    column checksums       */
    /* Optional bias (Sec. 5.1): bias[m] (fp32, for either layer dtype) is added to every
     * element of O[n][m] by the calls that compute O with the checksums (ftcnn_conv_fwd_sums,
     * ftcnn_protected_conv); cb = {sum_m bias[m], sum_m (m + wbase) bias[m]}, from
     * ftcnn_encode(which = 2), once per layer.  The checksums Co1..Co7 stay those of the
     * convolution; every detection and correction call given a non-NULL bias subtracts the
     * bias share of Table 5 from each summation before comparing it (N bias[m] from So1[m],
     * (sum_n (n + wbase)) bias[m] from So3[m], cb[0] from So2[n], cb[1] from So4[n],
     * N cb[0] from So5, N cb[1] from So6, (sum_n (n + wbase)) cb[0] from So7), and a
     * recomputed element includes its bias.  NULL bias: no bias (cb unused). */
    const float *bias;              /* [m]                                  */
    double *cb;                     /* [2]                                  */
} ftcnn_checksums;

/* Correction schemes, as recorded per repaired element and per position. */
enum {
    FTCNN_SCHEME_NONE = 0,
    FTCNN_SCHEME_COC = 1,          /* checksum-of-checksum, Sec. 3.6          */
    FTCNN_SCHEME_RC = 2,           /* row checksum, Sec. 3.4                  */
    FTCNN_SCHEME_CLC = 3,          /* column checksum, Sec. 3.5               */
    FTCNN_SCHEME_FC = 4,           /* full checksum, Sec. 3.3 and Sec. 4.1.5  */
    FTCNN_SCHEME_CKSUM = 5,        /* the checksums were corrupt, Sec. 4.1.4  */
    FTCNN_SCHEME_UNRESOLVED = 6    /* left for recomputation, Sec. 4.1.1      */
};

enum {
    FTCNN_STATUS_CLEAN = 0,            /* nothing detected                        */
    FTCNN_STATUS_CORRECTED = 1,        /* every flagged position resolved         */
    FTCNN_STATUS_NEEDS_RECOMPUTE = 2,  /* some position unresolved: rerun the layer */
    FTCNN_STATUS_RECOMPUTED = 3,       /* set by a caller that reran and re-verified */
    FTCNN_STATUS_FAILED = 4            /* set by a caller whose rerun still mismatches */
};

typedef struct { int32_t n, m, x, y, scheme; } ftcnn_fix;

/* Detection and correction report, in device memory (updated with device
 * atomics).  ftcnn_verify() resets it; ftcnn_correct() fills in the repairs.
 * fixes[] is in no particular order; n_fixes counts every repair even past
 * cap_fixes. */
typedef struct {
    int32_t detected;          /* CoC-D verdict for the layer                     */
    int32_t n_flagged;         /* positions p with Co5 - So5 beyond tolerance     */
    int32_t status;            /* FTCNN_STATUS_*                                  */
    int32_t resolved_by[7];    /* positions per FTCNN_SCHEME_*                    */
    int32_t n_fixes;
    int32_t cap_fixes;
    int32_t reserved[2];       /* internal to the library (zeroed with the report)  */
    ftcnn_fix fixes[];
} ftcnn_report;

/* Tolerance and workflow policy.  A checksum difference d at one element is
 * bad when it is non-finite or |d| > kappa * (2^-24 sqrt(ch*r*s) + u_out) * Q,
 * Q being the root sum of squares of the weighted terms of the summation and
 * u_out = 0 (fp32) or 2^-8 (bf16).  A located index is legal when its ratio is
 * within eta of an integer inside the index range.  rc_on / clc_on enable the
 * RC and ClC stages per layer (Sec. 4.3). */
enum { FTCNN_REPAIR_CHECKSUM = 0, FTCNN_REPAIR_RECOMPUTE = 1 };
typedef struct {
    int32_t rc_on, clc_on;
    int32_t repair;            /* FTCNN_REPAIR_*: exclusive checksum sum, or eq. (1) again */
    int32_t reserved;
    double kappa, eta;         /* defaults 16 and 0.1                             */
} ftcnn_policy;

/* A fault planted for testing (the paper's source-level injection, Sec. 6.1)
 * at output element (n, m, x, y): kind 0 flips bit `bit` of the stored fp32 or
 * bf16 pattern, kind 1 adds `value`, kind 2 stores `value` (both rounded to
 * the dtype). */
typedef struct { int32_t n, m, x, y, kind, bit; double value; } ftcnn_fault;

/* ---- host-only queries -------------------------------------------------- */

/* E and F of eq. (1) with zero padding.  Returns FTCNN_E_SHAPE when either is < 1. */
int ftcnn_out_shape(const ftcnn_conv_desc *desc, int32_t *E, int32_t *F);

/* Bytes of workspace every call on this layer may use (0 on a bad descriptor). */
size_t ftcnn_workspace_bytes(const ftcnn_conv_desc *desc);

/* Bytes of an ftcnn_report holding cap_fixes repairs. */
size_t ftcnn_report_bytes(int32_t cap_fixes);

/* Description of the last error on the calling thread ("" if none). */
const char *ftcnn_last_error(void);

/* INSTRUMENTATION (host-only, no device work; not an operation of the paper): the
 * convolution kernel this layer's calls launch.  path 0: ftcnn_conv_fwd and
 * ftcnn_conv_fwd_bias without a workspace (D and W read as given); path 1: every call
 * that takes a workspace (ftcnn_conv_fwd_ws, ftcnn_conv_fwd_sums, ftcnn_protected_conv,
 * ...).  out[0] = filters (rows of W) per workgroup tile, out[1] = output pixels per tile,
 * out[2] = k per LDS chunk, out[3] = main loop (0 register-staged gather, 1 gather woven
 * between the matrix-core instructions, 2 two chunks in flight, 3 direct-to-LDS loads,
 * 4 the same with three stages, 5 and 6 like 3 and 4 from packed copies, 7 like 3 for
 * kernels above 32 rows or columns; an fp32 layer on 3 to 7 multiplies bf16 planes),
 * out[4] = 1 when the convolution reads copies of D and W, out[5] = 1 when its tiles
 * skip the channels of other groups (grouped layers).  Lets a test check that it covers
 * every kernel a set of layers runs. */
int ftcnn_conv_tile(const ftcnn_conv_desc *desc, int32_t path, int32_t out[6]);

/* INSTRUMENTATION (host query of the current device, no device work): *workgroups = the
 * stream-K workgroups of the convolution launched by the calls that take a workspace (path 1
 * of ftcnn_conv_tile), or 0 when it runs one workgroup per output tile.  Stream-K is a
 * schedule, not another operation: every workgroup takes an equal run of the layer's
 * (tile, chunk of K) pairs, and a tile whose chunks span several workgroups is summed by the
 * last of them to finish, in chunk order (so the protected convolution and its unprotected
 * twin store the same bits).  It is used for dense channels-last fp32 layers whose whole tiles
 * would leave workgroups idle (in the last round, or all along) for longer than sharing takes. */
int ftcnn_conv_stream_k(const ftcnn_conv_desc *desc, int32_t *workgroups);

/* ---- device work -------------------------------------------------------- */

/* Sec. 3.2 input checksums.  which = 0: X is D, c1 = Cd1 = sum_n D_n and
 * c2 = Cd2 = sum_n (n + wbase) D_n, each [ch][h][w].  which = 1: X is W,
 * c1 = Cw1, c2 = Cw2, each [ch][r][s] (computed once per layer, before the
 * application, Sec. 4.2).  which = 2: X is a bias (float [m]), c1 = sum_m bias[m]
 * and c2 = sum_m (m + wbase) bias[m], one double each (the precomputed bias sums
 * of Sec. 5.1).  float64 accumulation; deterministic. */
int ftcnn_encode(const ftcnn_conv_desc *desc, int32_t which, const void *X,
                 double *c1, double *c2, void *workspace, hipStream_t stream);

/* Weights in memory (Sec. 4.1.2): a soft error in W shows as a difference between Cw1
 * re-encoded from the current W and cw1 encoded before the application (ftcnn_encode,
 * which = 1); the remedy is to reload W.  The re-encode runs the same deterministic kernels,
 * so intact weights reproduce cw1 bit for bit and the comparison is exact.  *mismatches
 * (device int32) receives the number of columns (c, r, s) whose sums differ: 0 when W is
 * intact.  Uses the workspace. */
int ftcnn_check_weights(const ftcnn_conv_desc *desc, const void *W, const double *cw1, int32_t *mismatches,
                        void *workspace, hipStream_t stream);

/* Eq. (1) without bias, with zero padding: O[n][m][x][y] = sum_{k,i,j}
 * D[n][k][Ux+i-P][Uy+j-P] W[m][k][i][j].  Implicit GEMM on the matrix cores,
 * fp32 accumulation, O rounded to the layer dtype (nearest even). */
int ftcnn_conv_fwd(const ftcnn_conv_desc *desc, const void *D, const void *W, void *O,
                   hipStream_t stream);

/* Eq. (1) plus a bias (Sec. 5.1): O[n][m][x][y] = (eq. (1)) + bias[m], added to the fp32
 * accumulator before O is rounded to the layer dtype.  bias: device, fp32 [m].  With a
 * workspace (ftcnn_workspace_bytes) the convolution runs through the kernels of the
 * protected path (ftcnn_conv_fwd_ws), so O is
 * bitwise that of ftcnn_conv_fwd_sums with the same bias; with NULL, through those of
 * ftcnn_conv_fwd. */
int ftcnn_conv_fwd_bias(const ftcnn_conv_desc *desc, const void *D, const void *W, const float *bias,
                        void *O, void *workspace, hipStream_t stream);

/* Output checksums of Sec. 3.2, as convolutions of checksum blocks, float64:
 *   FTCNN_CO1 | FTCNN_CO3: Co1 = Cd1 (x) W, Co3 = Cd2 (x) W   (reads cd1/cd2, W)
 *   FTCNN_CO2 | FTCNN_CO4: Co2 = D (x) Cw1, Co4 = D (x) Cw2   (reads D, cw1/cw2)
 *   FTCNN_CO5..7:          Co5 = Cd1 (x) Cw1, Co6 = Cd1 (x) Cw2, Co7 = Cd2 (x) Cw1
 * CoC-D needs only Co5; the correction chain computes what else it needs at
 * the flagged positions by itself, so the full Co1..Co4 arrays are optional. */
enum { FTCNN_CO1 = 1u << 0, FTCNN_CO2 = 1u << 1, FTCNN_CO3 = 1u << 2, FTCNN_CO4 = 1u << 3,
       FTCNN_CO5 = 1u << 4, FTCNN_CO6 = 1u << 5, FTCNN_CO7 = 1u << 6 };
int ftcnn_checksum_conv(const ftcnn_conv_desc *desc, uint32_t which, const void *D,
                        const void *W, const ftcnn_checksums *ck, hipStream_t stream);

/* CoC-D detection (Sec. 3.6, Sec. 4.3).  Reads O and ck->co5; writes
 * ck->so5, so6, so7, q5 and a per-position flag map into the workspace;
 * resets *rep (cap_fixes recorded) and sets rep->detected and rep->n_flagged. */
int ftcnn_verify(const ftcnn_conv_desc *desc, const void *O, const ftcnn_checksums *ck,
                 const ftcnn_policy *policy, ftcnn_report *rep, int32_t cap_fixes,
                 void *workspace, hipStream_t stream);

/* Correction module (Sec. 4.3): two device-gated launches that do nothing
 * unless rep->detected.  Every flagged position runs CoC, then RC and ClC if
 * enabled, then FC (with the fallbacks of Sec. 4.1.5), each scheme undone
 * unless Co5..Co7 agree with the re-summed output afterwards.  Repairs O in
 * place.  Positions where a weighted checksum agrees while Co5 does not are
 * re-checked against checksums re-encoded from D and W (Sec. 4.1.4).  The first
 * launch hands the flagged positions over; the second computes the row and
 * column checksums Co1..Co4 and the per-filter and per-image summations at
 * them over the whole device, and its last workgroup takes every decision.
 * Reads D, W, ck->cd1/cd2/cw1/cw2/co5/co6/co7, ck->so5/so6/so7/q5 when set (as
 * ftcnn_verify leaves them) and the verify flag map in the workspace.  Leaves
 * status NEEDS_RECOMPUTE if any position is unresolved; the caller then reruns
 * ftcnn_conv_fwd and ftcnn_verify (Sec. 4.1.1). */
int ftcnn_correct(const ftcnn_conv_desc *desc, const void *D, const void *W, void *O,
                  const ftcnn_checksums *ck, const ftcnn_policy *policy, ftcnn_report *rep,
                  void *workspace, hipStream_t stream);

/* ftcnn_verify and ftcnn_correct in two launches: the final detection stage
 * hands every position it flags to the correction's second launch, which does
 * nothing when none was flagged, so a clean layer pays one empty launch for the
 * correction module.  Same inputs, outputs and report as the two calls in
 * sequence. */
int ftcnn_verify_correct(const ftcnn_conv_desc *desc, const void *D, const void *W, void *O,
                         const ftcnn_checksums *ck, const ftcnn_policy *policy, ftcnn_report *rep,
                         int32_t cap_fixes, void *workspace, hipStream_t stream);

/* Eq. (1) as ftcnn_conv_fwd, through the path the protected calls below use:
 * D and W are first copied into the workspace so that the convolution reads
 * 16-byte runs: channels-last (D as [n][h][w][ch], W as [m][r][s][ch]) on layers with ch
 * a multiple of 32, packed (taps of padded channels) on those of other counts that are
 * predicted to be faster so; the rest take ftcnn_conv_fwd's kernel.  K is then summed in (r, s, ch) order, so
 * O may differ from ftcnn_conv_fwd's in the last bits (both are eq. (1) with
 * fp32 accumulation).  Where it is predicted to be faster, fp32 copies hold every value as three
 * bf16 planes whose sum it is, six of whose nine products the matrix cores add up, the other
 * three being below an fp32 rounding of the product; outputs that this leaves non-finite, which
 * besides infinities and NaN are those of operands from 2e31 or sums from 1.2e24, are computed
 * again from D and W with fp32 products, at about a quarter of the speed.  O is bitwise that of
 * ftcnn_conv_fwd_sums.  Needs the workspace of ftcnn_workspace_bytes. */
int ftcnn_conv_fwd_ws(const ftcnn_conv_desc *desc, const void *D, const void *W, void *O,
                      void *workspace, hipStream_t stream);

/* Eq. (1) as ftcnn_conv_fwd_ws (same kernels, bitwise the same O), with the
 * CoC-D summations of Sec. 3.6 computed in the epilogue from the values as
 * stored: every workgroup tile writes, for each of its output pixels, the
 * partial So5, So6, So7 and sum of squares over its filters into the
 * workspace, so detection never re-reads O.  Also resets *rep (cap_fixes
 * recorded).  Follow it with ftcnn_verify_correct_sums on the same workspace
 * and report.
 * ck: may be NULL.  When ck->cd1 and ck->cd2 are set, Cd1 and Cd2 are encoded
 * from D as ftcnn_encode(which = 0) does (Sec. 3.2): by the launch that copies
 * D, or by extra workgroups beside the matrix-core tiles of layers without copies.
 * When ck->cw1 and ck->cw2 (the encoded W) are set as well, most layers
 * with copies also compute the products Co5, Co6, Co7 of Sec. 3.2
 * in extra workgroups of the convolution launch, as per-channel-range partials
 * in the workspace that ftcnn_verify_correct_sums(which = CO5|CO6|CO7) adds up.
 * Other members are not used.
 * faults / nf: TEST ONLY, NULL / 0 otherwise.  A HOST array of at most 64
 * faults planted in the output values before they are summed and stored, as
 * a fault of the convolution's own arithmetic would appear (Sec. 6.1).
 * Checks every fault as ftcnn_inject does. */
int ftcnn_conv_fwd_sums(const ftcnn_conv_desc *desc, const void *D, const void *W, void *O,
                        const ftcnn_checksums *ck, ftcnn_report *rep, int32_t cap_fixes,
                        const ftcnn_fault *faults, int32_t nf, void *workspace, hipStream_t stream);

/* ftcnn_conv_fwd_sums for a layer whose input checksums are already encoded:
 * ck->cd1 and ck->cd2 (required) hold Cd1, Cd2 of D as inputs, for instance from
 * ftcnn_relu_pool_encode of the layer before (Sec. 3.2), and are not written.  The
 * copies are then only copies, and no encode workgroups run;
 * everything else is as ftcnn_conv_fwd_sums (same O, same sums, Co5..Co7 partials when
 * ck->cw1 and ck->cw2 are set).  Follow it with ftcnn_verify_correct_sums. */
int ftcnn_conv_fwd_sums_given(const ftcnn_conv_desc *desc, const void *D, const void *W, void *O,
                              const ftcnn_checksums *ck, ftcnn_report *rep, int32_t cap_fixes,
                              const ftcnn_fault *faults, int32_t nf, void *workspace, hipStream_t stream);

/* ftcnn_verify_correct over the partial sums that ftcnn_conv_fwd_sums left in
 * the workspace (one launch; O is read only at flagged positions).  The
 * report must be the one ftcnn_conv_fwd_sums reset.  which = 0: Co5..Co7 are
 * read from ck (ftcnn_checksum_conv ran before); which = FTCNN_CO5 |
 * FTCNN_CO6 | FTCNN_CO7: the same launch produces them at every position
 * first, adding the partial products ftcnn_conv_fwd_sums computed (when it
 * did) or else evaluating them from ck->cd1, cd2, cw1, cw2, and stores them in
 * ck->co5, co6, co7.  Writes ck->so5, so6, so7, q5 and the flag map; same
 * decisions and repairs as ftcnn_verify_correct. */
int ftcnn_verify_correct_sums(const ftcnn_conv_desc *desc, const void *D, const void *W, void *O,
                              const ftcnn_checksums *ck, const ftcnn_policy *policy, ftcnn_report *rep,
                              uint32_t which, void *workspace, hipStream_t stream);

/* The whole path of one protected layer on one stream:
 * conv_fwd_sums (with the encode of Cd1, Cd2, and Co5..Co7 on most layers with
 * copies) -> verify_correct_sums (with Co5..Co7): three launches, four for
 * layers with copies, one more on grouped ones.  ck->cw1/cw2 must hold the encoded W (ftcnn_encode with
 * which = 1); ck->cd1, cd2, co5..co7, so5..so7 and q5 are written. */
int ftcnn_protected_conv(const ftcnn_conv_desc *desc, const void *D, const void *W, void *O,
                         const ftcnn_checksums *ck, const ftcnn_policy *policy,
                         ftcnn_report *rep, int32_t cap_fixes, void *workspace,
                         hipStream_t stream);

/* ftcnn_protected_conv for callers that cannot allocate device memory (code under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc): the same
 * launches with no workspace argument.  Scratch comes from a static device array of the
 * library, 128 MiB on each device, which that device holds from the first call there until
 * the process ends; nothing is allocated or freed by the call.  The call uses the plan of
 * ftcnn_protected_conv when that plan's workspace (ftcnn_workspace_bytes) fits the array, and
 * otherwise the first that does of: that plan without scratch for shared tiles, the one on
 * fp32 copies, the one without copies, whose convolution gathers from D as given
 * (the same results within the output tolerance; K summed in (ch, r, s) order); a layer that
 * needs more than 128 MiB even then is rejected with FTCNN_E_WORKSPACE before any launch.
 * The device is the stream's (the current device for the NULL stream).  Every call on one
 * device shares that device's array and leaves its contents behind; calls whose work overlaps
 * on one device (other streams, other threads) race on it and must be ordered by the caller.
 * Arguments, outputs and report as ftcnn_protected_conv. */
int ftcnn_protected_conv_noalloc(const ftcnn_conv_desc *desc, const void *D, const void *W, void *O,
                                 const ftcnn_checksums *ck, const ftcnn_policy *policy,
                                 ftcnn_report *rep, int32_t cap_fixes, hipStream_t stream);

/* INSTRUMENTATION (measurement, not an operation of the paper): the next call
 * on the calling thread that launches the convolution kernel (ftcnn_conv_fwd,
 * ftcnn_conv_fwd_ws, ftcnn_conv_fwd_sums, ftcnn_protected_conv) records
 * `before` on its stream immediately before that launch and `after`
 * immediately after it, so that their elapsed time is the kernel's alone (the
 * channels-last copy and the other launches of the call fall outside); the
 * hook is then cleared.  Either may be NULL.  The events must be created by
 * the caller (with timing enabled) on the device of that stream. */
int ftcnn_set_kernel_events(hipEvent_t before, hipEvent_t after);

/* Between two protected layers of a network (AlexNet, VGG-19 and Darknet-19 in
 * Sec. 6): Y = k x k / s max pooling (no padding) of relu(X), relu(v) = v > 0 ? v : +0
 * (NaN and both zeros give +0).  X [n][c][h][w] and Y [n][c][(h-k)/s+1][(w-k)/s+1]
 * are device tensors of the dtype (FTCNN_F32 or FTCNN_BF16); every output is an input
 * value or +0, so the result is exact.  (k, s) is (1, 1) (ReLU only; X == Y allowed),
 * (2, 2) or (3, 2) (X and Y must not overlap), else FTCNN_E_UNSUPPORTED.  The next
 * layer then encodes its Cd1, Cd2 from Y, the corrected output of this layer after
 * these operations. */
int ftcnn_relu_pool(int32_t dtype, int32_t n, int32_t c, int32_t h, int32_t w, int32_t k, int32_t s,
                    const void *X, void *Y, hipStream_t stream);

/* ftcnn_relu_pool, and with it the input checksums of the layer that reads Y
 * (Sec. 3.2): cd1[c][i][j] = sum_n Y[n][c][i][j] and cd2[c][i][j] = sum_n (n + wbase)
 * Y[n][c][i][j], float64 device arrays of c * ((h-k)/s+1) * ((w-k)/s+1) elements, the
 * images added in order.  Y is the corrected output of one layer after the operations
 * between layers, so the next layer's checksums come from the values it will read, in the
 * pass that writes them; pass them to that layer's ftcnn_conv_fwd_sums_given.  wbase is
 * 0 or 1 (the next layer's descriptor's). */
int ftcnn_relu_pool_encode(int32_t dtype, int32_t n, int32_t c, int32_t h, int32_t w, int32_t k, int32_t s,
                           int32_t wbase, const void *X, void *Y, double *cd1, double *cd2,
                           hipStream_t stream);

/* TEST ONLY: corrupt stored outputs, reproducing the paper's source-level
 * fault injection (Sec. 6.1).  faults is a HOST array of at most 64 entries
 * (ftcnn_fault above), applied in order.  Positions must be in range. */
int ftcnn_inject(const ftcnn_conv_desc *desc, void *O, const ftcnn_fault *faults, int32_t nf,
                 hipStream_t stream);

/* ---- serving an attention layer -------------------------------------------
 * The operators between the projections of an attention layer (layers of 1 x 1 maps with the
 * tokens as the batch), for the new tokens of a batch of sequences whose keys and values live in
 * a cache of fixed-size pages.  They are not checksum-protected.
 *
 * Strides are in elements; the innermost dimension (the `dim` values of a head) is always
 * contiguous.  dtype (FTCNN_F32 or FTCNN_BF16) is that of every tensor of the call but the
 * table, the weights (fp32, or the dtype) and the index arrays.  All arithmetic is fp32 or
 * wider, and results are rounded once (nearest even), except the softmax weights of bf16
 * attention (see there).  Index arrays are device arrays; what they say is not known to the host:
 * the kernels bring every index into range, as each call describes, and never leave the
 * tensors described. */

/* Which values of a head a rotation pairs: (i, i + rot/2), or (2i, 2i + 1), i < rot/2. */
enum { FTCNN_ROPE_HALF = 0, FTCNN_ROPE_INTERLEAVED = 1 };

/* How angles p * f_j, f_j = base^(-2j/rot), are scaled for longer contexts: not at all; every f_j
 * divided by factor; base multiplied by factor^(rot/(rot-2)), so that the slowest pair is slowed
 * by factor and the fastest kept; or by parts: with t = original * f_j / (2 pi) turns within the
 * `original` positions and keep = clamp((t - low) / (high - low), 0, 1), f_j is multiplied by
 * keep + (1 - keep) / factor. */
enum { FTCNN_ROPE_PLAIN = 0, FTCNN_ROPE_LINEAR = 1, FTCNN_ROPE_BASE = 2, FTCNN_ROPE_PARTS = 3 };
typedef struct {
    int32_t max_pos, rot;    /* positions, rotated values of a head (even, at most 256) */
    int32_t scaling;         /* FTCNN_ROPE_PLAIN ..                                     */
    int32_t original;        /* FTCNN_ROPE_PARTS                                        */
    double base, factor;     /* factor is not read by FTCNN_ROPE_PLAIN                  */
    double low, high;        /* FTCNN_ROPE_PARTS                                        */
    double amplitude;        /* cos and sin are multiplied by it                        */
} ftcnn_rope_scaling;

/* table[p][j] = (cos, sin) of position p < max_pos and pair j < rot/2, fp32
 * [max_pos][rot/2][2], evaluated in float64.  Made once, before the application. */
int ftcnn_rope_table(const ftcnn_rope_scaling *scaling, float *table, hipStream_t stream);

typedef struct {
    int32_t dtype, tokens;
    int32_t heads, kv_heads;         /* either may be 0: that tensor is not read          */
    int32_t dim;                     /* even, at most 256                                 */
    int32_t rot, layout, max_pos;    /* of the table                                      */
    int32_t weight_dtype;            /* FTCNN_F32 or dtype                                */
    float eps;
    int64_t q_stride[2], k_stride[2], q_out_stride[2], k_out_stride[2];   /* token, head  */
} ftcnn_rope_desc;

/* Per head of every token: x * rsqrt(mean(x^2) + eps) * weight (no norm where the weight is
 * NULL), then the rotation of its first rot values by the token's position: a pair (a, b) becomes
 * (a cos - b sin, b cos + a sin).  positions [tokens] and table go together; both NULL: no
 * rotation.  The rotated values of a token whose position is not in [0, max_pos) are NaN.
 * q_out may be q and k_out k (with the same strides); outputs that overlap inputs otherwise are
 * undefined.  One launch. */
int ftcnn_qk_norm_rope(const ftcnn_rope_desc *desc, const void *q, const void *k, const int32_t *positions,
                       const float *table, const void *q_weight, const void *k_weight, void *q_out, void *k_out,
                       hipStream_t stream);

typedef struct {
    int32_t dtype, tokens, kv_heads;
    int32_t dim;                     /* even, at most 256                                 */
    int32_t rot, layout, max_pos;
    int32_t weight_dtype;
    int32_t pages, page;             /* pages of the cache, rows of a page                */
    float eps;
    int32_t reserved;
    int64_t k_stride[2], v_stride[2];               /* token, head                        */
    int64_t k_cache_stride[3], v_cache_stride[3];   /* page, row, head                    */
} ftcnn_append_desc;

/* Keys, normed and rotated as ftcnn_qk_norm_rope does it, and values as they are, into the
 * cache: token t into row slots[t] % page of page slots[t] / page.  A token whose slot is not in
 * [0, pages * page) (padding: -1) is written nowhere.  Two tokens of one slot leave either's
 * values.  One launch. */
int ftcnn_kv_append(const ftcnn_append_desc *desc, const void *k, const void *v, const int32_t *positions,
                    const float *table, const void *k_weight, const int64_t *slots, void *k_cache, void *v_cache,
                    hipStream_t stream);

typedef struct {
    int32_t dtype, batch, tokens;
    int32_t heads, kv_heads;         /* query head h reads key head h / (heads / kv_heads) */
    int32_t dim;                     /* a multiple of 8, at most 256                      */
    int32_t pages, page;             /* pages of the cache, rows of a page (any number)   */
    int32_t list_len;                /* entries of a sequence's page list                 */
    int32_t causal, window;          /* window > 0 (causal only): the last window positions */
    int32_t max_q, max_kv;           /* the longest sequence's new and cached tokens; 0: not
                                        known.  They shape the launch: too small or too large
                                        costs time, and changes the order of the sums and,
                                        in bf16, which weights are rounded (see below)    */
    float scale;                     /* positive, below 2.3e38                            */
    int64_t q_stride[2], out_stride[2];             /* token, head                        */
    int64_t k_cache_stride[3], v_cache_stride[3];   /* page, row, head                    */
    int64_t list_stride;
} ftcnn_attention_desc;

/* Attention of every sequence's new tokens over its cached ones.  The new tokens of sequence b
 * are rows q_starts[b] .. q_starts[b + 1] - 1 of q and out [tokens][heads][dim] (q_starts
 * [batch + 1], not falling; NULL: row b alone); their keys and values are cached already, as the
 * last of its kv_lens[b] rows, so that the i-th of n sits at position kv_lens[b] - n + i and sees
 * positions up to its own (causal), of those the last `window`, or all (not causal).  Position j
 * lies in row j % page of page page_list[b][j / page].
 *   out = sum_j softmax_j(scale q . k_j) v_j,   lse = log sum_j exp(scale q . k_j)
 * with lse (fp32 [tokens][heads], NULL: not wanted) the natural logarithm.  A row that sees
 * nothing (an empty cache, or fewer cached tokens than new ones) is 0, its lse -infinity; so are
 * rows of no sequence, before q_starts[0] and from q_starts[batch] on (padding).
 * Scores, maxima, sums and outputs are held in fp32.  bf16 calls of more than 16 rows a key head
 * (max_q * heads / kv_heads) round the softmax weights, relative to a maximum, to bf16 for the
 * product with the values, not for their sum; others keep them in fp32.  Infinities and NaN of keys
 * and values that a row does not see do not reach it.
 * kv_lens are taken within [0, list_len * page], q_starts within [0, tokens], and a page number
 * outside [0, pages) as the nearest one inside.  Rows of q, out and the cache start on 16 bytes;
 * the cache's strides are 0 to 2^29.  out may be q.  The result does not depend on timing: calls
 * on the same arguments give the same bits.  One launch, or two where the cached tokens are split
 * over workgroups: then the workspace holds the parts. */
int ftcnn_paged_attention(const ftcnn_attention_desc *desc, const void *q, const void *k_cache, const void *v_cache,
                          const int32_t *page_list, const int32_t *kv_lens, const int32_t *q_starts, void *out,
                          float *lse, void *workspace, hipStream_t stream);

/* Bytes of 256-byte-aligned workspace that ftcnn_paged_attention takes for this descriptor: 0
 * where it needs none (NULL will do), and on a bad descriptor. */
size_t ftcnn_paged_attention_workspace_bytes(const ftcnn_attention_desc *desc);

/* ---- what differs from request to request ----------------------------------
 * Requests that one layer serves together may bring adapters of their own beside its projections, and
 * keep their caches within budgets of their own.  Conventions are those of the serving operators above:
 * strides in elements, innermost dimensions contiguous, fp32 arithmetic, results rounded once, and index
 * arrays on the device, brought into range by the kernels. */

typedef struct {
    int32_t dtype, tokens;
    int32_t ch, m;                   /* of the projection; multiples of 16 bytes          */
    int32_t adapters, rank;          /* rank: a multiple of 16 bytes, at most 128         */
    int64_t x_stride, y_stride, out_stride;      /* token                                 */
    int64_t a_stride[2], b_stride[2];            /* adapter, row                          */
} ftcnn_low_rank_desc;

/* out_t = y_t + scales[a] B_a (A_a x_t) with a = ids[t]: x [tokens][ch], the output y [tokens][m] of the
 * projection that all tokens share, A [adapters][rank][ch], B [adapters][m][rank].  ids [tokens] may come in
 * any order; a token whose id is not in [0, adapters) (none: -1) keeps y as it is.  scales (fp32
 * [adapters], NULL: 1).  ranks [adapters] (NULL: rank): adapter a has the first ranks[a] rows of A_a and
 * columns of B_a, taken within [0, rank]; what lies past them is not used, and may be anything where a rank is
 * padded to 16 bytes.  A_a x_t is held in fp32; bf16: for the second product as the sum of two bf16 values, within
 * 2^-17 of it (below 2^-117: within 2^-134).  Infinities and NaN of a token or adapter reach only the tokens that
 * have them.  An infinity in B comes out as itself or as NaN.
 * out may be y (with its strides); outputs that overlap inputs otherwise are undefined.  Rows start on 16
 * bytes.  The workspace holds the products A x and, of many tokens, which have the same adapter.  The result does
 * not depend on timing.  One launch for few tokens, two, or three where many are grouped. */
int ftcnn_low_rank_add(const ftcnn_low_rank_desc *desc, const void *y, const void *x, const void *a, const void *b,
                       const int32_t *ids, const float *scales, const int32_t *ranks, void *out, void *workspace,
                       hipStream_t stream);

/* Bytes of 256-byte-aligned workspace of the call; 0 where it needs none, and on a bad descriptor. */
size_t ftcnn_low_rank_workspace_bytes(const ftcnn_low_rank_desc *desc);

typedef struct {
    int32_t dtype, batch, tokens;    /* as in ftcnn_attention_desc, to scale              */
    int32_t heads, kv_heads, dim;
    int32_t pages, page, list_len;
    int32_t causal, window;
    int32_t max_q, max_kv;           /* shape the launch, as there                        */
    float scale;
    int64_t q_stride[2];             /* token, head                                       */
    int64_t k_cache_stride[3];       /* page, row, head                                   */
    int64_t mass_stride;             /* sequence; at least list_len * page                */
    int64_t list_stride;
} ftcnn_mass_desc;

/* The softmax weight that every cached key got from the new tokens, of all heads:
 *   mass[b][j] += sum over the rows i of sequence b that see position j of exp(scale q_i . k_j - lse_i)
 * for j < kv_lens[b], with the queries, cache, lists, lengths and masks of the ftcnn_paged_attention call
 * before, and the lse (fp32 [tokens][heads]) that it gave.  mass is fp32 [batch][list_len * page]; what lies
 * past kv_lens[b] is left as it was.  Infinities and NaN of keys and rows reach only each other.  Indices are
 * taken as there; rows of q and the cache start on 16 bytes.  The result does not depend on timing.  One
 * launch, or two where workgroups share a key's rows: then the workspace holds the parts. */
int ftcnn_attention_mass(const ftcnn_mass_desc *desc, const void *q, const void *k_cache, const int32_t *page_list,
                         const int32_t *kv_lens, const int32_t *q_starts, const float *lse, float *mass, void *workspace,
                         hipStream_t stream);

/* Bytes of 256-byte-aligned workspace of the call; 0 where it needs none, and on a bad descriptor. */
size_t ftcnn_attention_mass_workspace_bytes(const ftcnn_mass_desc *desc);

typedef struct {
    int32_t dtype, batch;
    int32_t kv_heads, dim;
    int32_t pages, page, list_len;
    int32_t first;                   /* rows at positions below it are kept               */
    int32_t max_kv;                  /* the longest sequence's rows (0: not known): shapes the launch */
    int32_t reserved;
    int64_t k_cache_stride[3], v_cache_stride[3];   /* page, row, head                    */
    int64_t list_stride;
    int64_t mass_stride, position_stride, mass_out_stride, position_out_stride;   /* sequence */
} ftcnn_evict_desc;

/* Takes rows out of the sequences' caches: of the n = kv_lens[b] rows of sequence b, k = min(keep[b], n) stay,
 * and the length becomes lens_out[b] = k.  Those stay that come first by: kept for its position or not, then
 * larger mass[b][j] (NaN below all), then lower place j.  A row is kept for its position where
 * positions[b][j] < first or positions[b][j] >= since[b] (since NULL: no such); positions NULL: a row's place is
 * its position.  The i-th place below k whose row goes takes the keys and values of all heads of the i-th row
 * that stays from place k on, so rows do not stay in the order of their positions: attention over them is the
 * same in any order, but not with a window, which goes by places.  mass_out and positions_out
 * [batch][list_len * page] move with the rows; from place k on they are 0 and -1.  They may be mass and
 * positions, and lens_out may be kv_lens.  Cache rows from place k on keep what they held.
 * A page that rows of two sequences lie in, or that a list has twice, holds undefined values after it.  keep and kv_lens are
 * taken as at least 0, kv_lens as at most list_len * page, page numbers as in ftcnn_paged_attention.  Rows of the
 * cache start on 16 bytes, at most 2^29 units of 16 bytes of all key heads; its strides are 0 to 2^29.  Two launches, or
 * six where sequences are long. */
int ftcnn_evict(const ftcnn_evict_desc *desc, void *k_cache, void *v_cache, const int32_t *page_list, const int32_t *kv_lens,
                const int32_t *keep, const float *mass, const int32_t *positions, const int32_t *since, int32_t *lens_out,
                float *mass_out, int32_t *positions_out, void *workspace, hipStream_t stream);

/* Bytes of 256-byte-aligned workspace of the call; 0 on a bad descriptor. */
size_t ftcnn_evict_workspace_bytes(const ftcnn_evict_desc *desc);

#ifdef __cplusplus
}
#endif
#endif /* FTCNN_H */
