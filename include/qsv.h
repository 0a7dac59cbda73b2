/* qsv — batched complex64 state-vector simulation of layered parameterised circuits on one
 * AMD MI355X (gfx950).  C ABI of libqsv.so.
 *
 * What the calls compute is fixed by the task statement (its "north star" paragraph and the five
 * workload configs); the source paper itself contains no circuit material, so the conventions
 * below are the stated readings that the CPU oracle pins with closed forms.
 *
 * Conventions
 *   - qubit q is bit q of the amplitude index k (qubit 0 = least-significant bit = stride 1).
 *   - state: DEVICE memory, complex64 [batch][2^n], interleaved (re, im) float32, sample-major.
 *   - RX(t) = [[c,-is],[-is,c]], RY(t) = [[c,-s],[s,c]], RZ(t) = diag(e^{-it/2}, e^{+it/2}),
 *     c = cos(t/2), s = sin(t/2).
 *   - one layer = [re-upload RX(w[l][q] * feats[b][q]) on q = 0..n-1, if reupload]
 *                 -> rotation slot 0 on q = 0..n-1 -> slot 1 ... -> entangler.
 *   - CNOT ring: CNOT(control q, target (q+1) mod n) for q = 0,1,...,n-1 in that order (none for
 *     n = 1).  CZ ladder: CZ(q, q+1) for q = 0..n-2.
 *   - parameters: float32 [P] shared by the whole batch, P = n_layers*(reupload+n_rot)*n, flat
 *     index p = (l*(reupload+n_rot) + slot)*n + q; slot 0 holds w when reupload = 1.
 *
 * Ownership and execution
 *   - The caller owns every device buffer (state, inputs, outputs, workspace); the context owns
 *     only host-side plans.  No call allocates or frees device memory.
 *   - All work is enqueued on the HIP stream given to qsv_create and is asynchronous with respect
 *     to the host; no call synchronises the stream (one exception, a measurement aid and no part of
 *     the path: qsv_probe_pass).  The pass plans of the circuits a context has run are kept in host
 *     memory until qsv_destroy and uploaded by asynchronous copies on the stream; when the plan
 *     region of the workspace is full it is refilled from its start, in stream order.
 *     Part of a call's kernels may run on a second
 *     stream that the context owns (default priority); it waits for the caller's stream at the
 *     start of that work and the caller's stream waits for it before the call's remaining work, so
 *     to the caller everything is ordered as if it ran on the one stream (also under stream
 *     capture, where the second stream joins the capture and leaves it within the call).  Host
 *     structs (qsv_circuit, qsv_measure_req) are read during the call and may be reused afterwards.
 *   - Pointers named *_dev are device pointers; everything else is host memory.
 *   - Argument errors are detected on the host before anything is launched and reported through
 *     the return code; qsv_last_error gives the text.  No exceptions, no abort.
 *   - One context per stream; a context is not thread-safe.
 */
#ifndef QSV_H
#define QSV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct qsv_ctx qsv_ctx;

typedef enum {
    QSV_OK = 0,
    QSV_ERR_INVALID_ARG = 1,
    QSV_ERR_UNSUPPORTED = 2,
    QSV_ERR_ZERO_NORM = 3,   /* reserved, never returned: calls are asynchronous, so a zero vector
                                is reported in band (norm 0 and an all-zero state from
                                qsv_amp_encode, -1 for every shot from QSV_M_SAMPLE) */
    QSV_ERR_WORKSPACE = 4,
    QSV_ERR_HIP = 5
} qsv_status;

typedef enum { QSV_RX = 1, QSV_RY = 2, QSV_RZ = 3 } qsv_axis;
typedef enum { QSV_ENT_NONE = 0, QSV_ENT_CNOT_RING = 1, QSV_ENT_CZ_LADDER = 2 } qsv_ent;

/* Layered circuit (task statement: "encoder/decoder variational layers", "data re-uploading
 * blocks"; workload configs 0-4 give the rotation lists and entanglers). */
typedef struct {
    int32_t n_layers;  /* >= 0 */
    int32_t reupload;  /* 1: every layer starts with RX(w[l][q] * feats[b][q]) on each qubit */
    int32_t n_rot;     /* 0..3 rotation slots per layer */
    int32_t rot[3];    /* qsv_axis of each slot, in application order */
    int32_t entangler; /* qsv_ent */
} qsv_circuit;

/* Number of parameters P of a circuit on n qubits; -1 on a bad descriptor. */
int64_t qsv_num_params(const qsv_circuit* c, int n_qubits);

/* Workspace size in bytes that is enough for every call below at (n_qubits, batch) with up to
 * 64 layers, a copy of the state for qsv_apply_layers with deferred CNOTs included (up to 28
 * qubits).  Returns 0 for n_qubits outside 1..30 or batch < 1.  A larger workspace lets
 * qsv_param_shift_grad run more circuits per launch. */
size_t qsv_workspace_bytes(int n_qubits, int batch);

/* Workspace size in bytes with which qsv_param_shift_grad can work layer by layer on circuit c:
 * qsv_workspace_bytes plus room for n_layers + 1 states per sample.  Returns 0 on bad arguments.
 * With less, qsv_param_shift_grad still works and runs every shifted circuit whole. */
size_t qsv_grad_workspace_bytes(int n_qubits, int batch, const qsv_circuit* c);

/* Create a context bound to (n_qubits, batch), a device ordinal, a HIP stream (hipStream_t cast
 * to void*, NULL = default stream), the caller's state buffer complex64 [batch][2^n] and the
 * caller's workspace (256-byte aligned device memory of at least qsv_workspace_bytes bytes).
 * batch must be in 1..2^24 with batch * 2^n_qubits <= 2^36.  Nothing is launched. */
qsv_status qsv_create(qsv_ctx** out, int n_qubits, int batch, int device, void* hip_stream,
                      void* state_dev, void* ws_dev, size_t ws_bytes);
void qsv_destroy(qsv_ctx* ctx);

/* Text of the last error on this context (or of the last failed qsv_create when ctx is NULL).
 * The string is owned by the library and stays valid until the next call on the context. */
const char* qsv_last_error(const qsv_ctx* ctx);

/* Amplitude encoding (task statement: "amplitude encoding of classical vectors"; every config):
 * state[b][k] = x[b][k] / ||x[b]||_2 for k < dim, 0 for dim <= k < 2^n, imaginary part 0.
 * x_dev: float32 [batch][dim], 1 <= dim <= 2^n.  norm_out_dev: float32 [batch] or NULL, receives
 * ||x[b]||_2.  A zero vector gives an all-zero state and norm 0 (no NaN). */
qsv_status qsv_amp_encode(qsv_ctx* ctx, const float* x_dev, int64_t dim, float* norm_out_dev);

/* Apply the layered circuit to every sample of the state, in place (task statement: "encoder/
 * decoder variational layers, data re-uploading blocks").  params_dev: float32 [P].  feats_dev:
 * float32 [batch][n], required when c->reupload = 1, ignored otherwise.  inverse = 1 applies the
 * exact inverse: layers last..first, inside a layer the entangler gates in reverse order, then
 * the rotation slots in reverse order with negated angles, then the re-upload RX negated.
 * Amplitudes are 0 or such that float32 holds their probability (modulus 2^-75 to 2^64): inside the
 * call they may be off by a common factor of up to 2^32, which the last gates take back. */
qsv_status qsv_apply_layers(qsv_ctx* ctx, const qsv_circuit* c, const float* params_dev,
                            const float* feats_dev, int inverse);

/* Measurement kinds (task statement: "measurement probabilities/expectations", "trash-qubit
 * probability", "fidelity with the input state", "seeded measurement samples"). */
typedef enum {
    QSV_M_PROBS = 1,        /* out float32 [batch][2^n]: p[k] = |a[k]|^2 */
    QSV_M_EXPZ_ALL = 2,     /* out float32 [batch][n]: <Z_q> = sum_k (1-2 bit_q(k)) p[k] */
    QSV_M_EXPZ_ONE = 3,     /* out float32 [batch]: <Z_qubit> */
    QSV_M_MARGINAL = 4,     /* out float32 [batch][2^m], m = popcount(mask) <= 20: probability of
                               each reading v of the mask qubits (lowest mask qubit = bit 0 of v) */
    QSV_M_PROJECT_ZERO = 5, /* out float32 [batch]: P0 = P(all mask qubits read 0); the state is
                               then projected onto that subspace (other amplitudes set to 0) and,
                               when renormalise = 1, divided by sqrt(P0); P0 = 0 leaves zeros */
    QSV_M_FIDELITY = 6,     /* out float32 [batch]: |<a_in|a>|^2 with a_in = x/||x||, x_dev float32
                               [batch][dim] zero-padded to 2^n */
    QSV_M_SAMPLE = 7        /* out int64 [batch][shots]: basis-state indices drawn by the integer
                               inverse-CDF rule below from the caller's uniforms */
} qsv_mkind;

/* Sampling rule (bit-exact by construction): with p32[k] = float32(|a[k]|^2) exactly as
 * QSV_M_PROBS writes it, w[k] = floor(double(p32[k]) * 2^60) as uint64, W[k] = w[0]+...+w[k],
 * r = floor(u * 2^53), t = floor(r * W[last] / 2^53) (128-bit product); the sample is the smallest
 * k with W[k] > t.  Shots keep the order of the uniforms.  W[last] = 0 writes -1 for every shot. */
typedef struct {
    int32_t kind;               /* qsv_mkind */
    int32_t qubit;              /* EXPZ_ONE */
    uint64_t mask;              /* MARGINAL, PROJECT_ZERO: non-empty subset of qubits 0..n-1 */
    int32_t renormalise;        /* PROJECT_ZERO */
    int32_t reserved;           /* must be 0 */
    const float* x_dev;         /* FIDELITY */
    int64_t dim;                /* FIDELITY: 1..2^n */
    const double* uniforms_dev; /* SAMPLE: float64 [batch][shots], values in [0,1) */
    int64_t shots;              /* SAMPLE: >= 0 */
    void* out_dev;              /* result, type and shape fixed by kind */
} qsv_measure_req;

qsv_status qsv_measure(qsv_ctx* ctx, const qsv_measure_req* req);

/* A whole small workload in ONE kernel launch (task statement: "batch-parallel launches across
 * samples"; workload configs 0 and 1, whose separate calls cost more in launches than in arithmetic):
 * qsv_amp_encode(x), qsv_apply_layers(c, inverse = 0), with decode = 1 then qsv_apply_layers(c,
 * inverse = 1) (encoder followed by its decoder), the final state written to the context's state
 * buffer, and one measurement of it, kind = QSV_M_PROBS (out_dev float32 [batch][2^n]) or
 * QSV_M_EXPZ_ALL (out_dev float32 [batch][n]).  Arguments as in those calls; norm_out_dev may be
 * NULL.  Same definitions and tolerances as the separate calls (the probabilities are the same
 * float32 function of the stored state; sums may differ in their last bits from the separate
 * calls', which add in another order).  A thread keeps 4, 8 or 16 amplitudes in registers and a
 * workgroup of at most 256 threads holds a sample, so this serves n_qubits <= 10, and circuits with
 * at most 512 matrices per workgroup: n_layers * n_qubits, times the samples that share a
 * wavefront when reupload = 1 (2^(8 - n_qubits) of them up to 8 qubits, one above).  Anything else
 * returns QSV_ERR_UNSUPPORTED before a launch, and the separate calls serve it.  Needs no
 * workspace.  It pays while the launches of the separate calls cost more than their arithmetic:
 * up to about 2^21 amplitudes in the whole batch (measured: 10 qubits x 1024 samples 35 against
 * 72 us); per gate it is about three times slower than the fused passes of qsv_apply_layers, so
 * larger batches are better served by the separate calls. */
qsv_status qsv_forward_small(qsv_ctx* ctx, const float* x_dev, int64_t dim, const qsv_circuit* c,
                             const float* params_dev, const float* feats_dev, int decode, int kind,
                             void* out_dev, float* norm_out_dev);

/* qsv_measure for callers that cannot allocate device memory and have no workspace to spare for it:
 * code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same request,
 * same kernels, same results bit for bit; only the kernels' partial results (block sums, cumulative
 * weights) go to a fixed array of 4 MiB inside the library's code object instead of the caller's
 * workspace.  The call allocates and frees nothing, on the device or through any library.  Every GPU
 * the library runs on holds one copy of the array until the process ends.  A request whose partial
 * results need more than 4 MiB (enough for all five workload configs; the need grows with
 * batch * 2^n_qubits / 4096) is rejected with QSV_ERR_WORKSPACE before anything is launched.  All
 * calls on one GPU share that GPU's array, whatever their context or stream: calls that overlap in
 * time on one GPU race, so keep them on one stream or order them with events.  Nothing in the array
 * needs to start at zero: every byte that is read has been written earlier in the same call. */
qsv_status qsv_measure_static(qsv_ctx* ctx, const qsv_measure_req* req);

/* Fidelity of an autoencoder with a true reset of its trash qubits (task statement, workload
 * config 3; the projection of QSV_M_PROJECT_ZERO is the post-selected stand-in for it).  The
 * context's state is taken as the encoder output.  For every outcome t of measuring the qubits of
 * mask (at most 10), the unnormalised conditional state with the trash qubits set to 0 is run
 * through circuit c in inverse mode (the decoder) and
 *   out[b] = sum_t | <x_b / ||x_b||  |  D (psi_t (x) |0>) > |^2        (float [batch]).
 * Works in the workspace, 2^m decoder runs per sample in chunks; the state is left as it was. */
qsv_status qsv_reset_fidelity(qsv_ctx* ctx, const qsv_circuit* c, const float* params_dev,
                              const float* feats_dev, uint64_t mask, const float* x_dev, int64_t dim,
                              float* out_dev);

/* Finite-shot estimate of <Z_q> for every qubit from basis-state samples as QSV_M_SAMPLE writes
 * them: samples_dev int64 [batch][shots]; out_dev float [batch][n_qubits] = mean over the shots of
 * (1 - 2 bit_q); entries < 0 (no valid outcome) are skipped, a row without valid shots gives 0. */
qsv_status qsv_shot_expz(qsv_ctx* ctx, const long long* samples_dev, int64_t shots, float* out_dev);

/* What a row of outcomes is given as: scores (natural logarithms of weights, up to a constant), probabilities (as
 * QSV_M_PROBS and QSV_M_MARGINAL write them, up to a factor), or the context's state, whose probabilities are taken as
 * QSV_M_PROBS would write them. */
typedef enum {
    QSV_S_F32 = 1,    /* scores, IEEE 32 bits */
    QSV_S_F16 = 2,    /* scores, IEEE 16 bits */
    QSV_S_BF16 = 3,   /* scores, the upper half of a float32 */
    QSV_S_PROBS = 4,  /* probabilities, float32 */
    QSV_S_STATE = 5   /* the context's state: scores_dev NULL, rows = batch, cols = 2^n, row_stride ignored */
} qsv_scores_kind;

/* Outcomes drawn from rows of scores, probabilities or amplitudes after temperature, min-p, top-k and top-p, from the
 * caller's uniforms.  v_k is the value of outcome k, m the highest one.  Masked outcomes (scores: -inf or NaN;
 * probabilities: NaN and all that are not positive) are never drawn; the type's lowest finite value is an ordinary score.
 * The order is v descending, the lowest index first among equals (-0 equals 0), and e_k = exp((v_k - m) / T) for scores,
 * (v_k / m)^(1 / T) for probabilities, 1 where v_k = m (which may be +inf).  Then, one after the other:
 *   temperature  T, finite, >= 0; T = 0 keeps the first outcome alone and ends the list;
 *   min_p        keeps e_k >= min_p, in 0..1 (0: all);
 *   top_k        keeps the first top_k of these (0: all);
 *   top_p        >= 0, with w_k = rint(e_k 2^S), S = min(51, 62 - ceil(log2 cols)), W the sum of w over these and
 *                H = ceil(rint(top_p 2^31) W / 2^31): keeps an outcome while the weights before it in the order sum to
 *                less than H, and the first one always (top_p >= 1: all).
 * The draw is QSV_M_SAMPLE's: W' the sum of w over what is left, r = floor(u 2^53), t = floor(r W' / 2^53), the smallest k
 * whose running sum in the order of the INDEX exceeds t.  e_k is taken in float64, so a result can differ from the
 * definition only where a value lies within about 2^-48 (probabilities at T != 1: 2^-45 / T) of a border; sums are of whole
 * numbers, so a call's results do not depend on how its work is split.  A row without an outcome, or with a parameter out of
 * its range (NaN too), gives -1 for every shot, logp -inf and kept 0; a uniform outside [0, 1) gives -1 and -inf for its shot. */
typedef struct {
    int32_t kind;                 /* qsv_scores_kind */
    int32_t reserved;             /* must be 0 */
    const void* scores_dev;       /* row r starts at element r * row_stride; aligned to its element */
    int64_t rows;                 /* 0..2^24; 0 is a no-op */
    int64_t cols;                 /* 1..2^30 */
    int64_t row_stride;           /* >= cols (any value for one row), in elements */
    const float* temperature_dev; /* [rows] or NULL (1) */
    const int32_t* top_k_dev;     /* [rows] or NULL (0) */
    const float* top_p_dev;       /* [rows] or NULL (1) */
    const float* min_p_dev;       /* [rows] or NULL (0) */
    const double* uniforms_dev;   /* float64 [rows][shots], values in [0, 1) */
    int64_t shots;                /* >= 0, rows * shots <= 2^32 */
    int64_t* out_dev;             /* int64 [rows][shots] */
    float* logp_dev;              /* float32 [rows][shots] or NULL: ln(w_k / W') of the outcome drawn */
    int32_t* kept_dev;            /* int32 [rows] or NULL: the number of outcomes left */
} qsv_sample_req;

/* Workspace size in bytes that qsv_sample needs for such rows, that of the plans included; 0 on bad arguments.  (Up to 32 shots
 * a row need none beside the plans' up to 262144 outcomes.) */
size_t qsv_sample_workspace_bytes(int64_t rows, int64_t cols);
qsv_status qsv_sample(qsv_ctx* ctx, const qsv_sample_req* req);

/* Expectation value of a Pauli string on the current state (task statement: "measurement
 * (... <Z> ...)", widened to X and Y): P = product over qubits of X (bit set in xmask), Y (ymask)
 * or Z (zmask), identity elsewhere; the masks must not overlap and name qubits < n_qubits.
 * out_dev: float [batch].  Computed directly as sum_k conj(a[k ^ f]) i^nY (-1)^popcount(k & s) a[k]
 * with f = xmask | ymask, s = ymask | zmask: one read pass, the state is not modified. */
qsv_status qsv_pauli_expect(qsv_ctx* ctx, uint64_t xmask, uint64_t ymask, uint64_t zmask, float* out_dev);

/* Parameter-shift gradient of f_b = <Z_obs> after encode + circuit (task statement: "parameter-
 * shift gradients over the batch"; config 2: "2 circuits per param per sample"):
 *   grad[b][p] = 1/2 [ f_b(angle_p + pi/2) - f_b(angle_p - pi/2) ]
 * (times feats[b][q] when p is a re-upload weight, whose angle is w*feat).  x_dev float32
 * [batch][dim]; loss_dev float32 [batch] receives the unshifted f_b; grad_dev float32 [batch][P];
 * mean_loss_dev [1] and mean_grad_dev [P] receive the batch means when not NULL.  Uses the
 * workspace for the shifted circuits' states; the context's state buffer is left untouched.
 * When the workspace has room for n_layers + 1 states per sample (qsv_grad_workspace_bytes), the
 * unshifted circuit's state before every layer is kept and a circuit that shifts a parameter of
 * layer l runs layers l..L-1 only, from that state: the same values with about half the gate
 * applications (option grad_layered = 0 switches this off).  From 10 qubits on, unless the batch is small, the two
 * shifted states of a parameter are then formed from one run instead of two, with the angle turned by
 * pi: R(t +- pi/2) = (R(t) +- R(t + pi)) / sqrt 2, so they are (unshifted +- turned) / sqrt 2, and both expectation values are
 * taken of them; larger batches start such runs behind the layer's rotations. */
qsv_status qsv_param_shift_grad(qsv_ctx* ctx, const qsv_circuit* c, const float* x_dev, int64_t dim,
                                const float* params_dev, const float* feats_dev, int32_t obs_qubit,
                                float* loss_dev, float* grad_dev, float* mean_loss_dev,
                                float* mean_grad_dev);

/* The same loss and gradient as qsv_param_shift_grad (same arguments, same outputs, equal up to
 * rounding), evaluated in reverse mode (task statement: "gradients over the batch"; listed there
 * as the cross-check of the shift rule).  Per sample one forward run gives psi and the loss; psi
 * and lambda = Z_obs psi are then taken back through the layers together, and at the start of
 * each layer the derivative with respect to an angle of slot s on qubit q is
 * 2 Re <lambda| W^dagger (-i/2 P_s) W |psi> on that qubit, W = the layer's earlier slots on it,
 * read off the 2x2 sums  M_q[a][b] = sum_rest conj(lambda[a, rest]) psi[b, rest].
 * Work: about 3 L layers and L n reductions per sample instead of 2 P circuits.  Uses the workspace (at
 * least three states per sample of a chunk; with room for the states between the passes of the circuit, which
 * qsv_grad_workspace_bytes nearly always has up to 20 qubits and beyond for few samples of few layers, the way back reads them
 * and takes the sums as it goes, in a third to two thirds of the time); the context's state buffer is left untouched. */
qsv_status qsv_adjoint_grad(qsv_ctx* ctx, const qsv_circuit* c, const float* x_dev, int64_t dim,
                            const float* params_dev, const float* feats_dev, int32_t obs_qubit,
                            float* loss_dev, float* grad_dev, float* mean_loss_dev,
                            float* mean_grad_dev);

/* Training losses built from the measured quantities (task statement: the autoencoder of workload
 * config 3 empties its trash qubits; the re-uploading model of config 1 regresses <Z_q>).
 *   QSV_LOSS_TRASH: loss_b = 1 - P0_b, P0 = probability that every qubit of mask reads 0.
 *   QSV_LOSS_MSE_Z: loss_b = 1/n sum_q (<Z_q>_b - targets[b][q])^2, targets_dev float [batch][n]. */
typedef enum { QSV_LOSS_TRASH = 1, QSV_LOSS_MSE_Z = 2 } qsv_loss_kind;
typedef struct {
    int32_t kind;             /* qsv_loss_kind */
    int32_t reserved;         /* 0 */
    uint64_t mask;            /* QSV_LOSS_TRASH: trash qubits, bit q = qubit q; at least one, all < n_qubits */
    const float* targets_dev; /* QSV_LOSS_MSE_Z: [batch][n_qubits]; else ignored */
} qsv_loss;

/* Per-sample loss [batch] and gradient [batch][P] of a training loss, and optionally their batch
 * means, evaluated in reverse mode as in qsv_adjoint_grad (lambda = O psi with O = -P0 projector,
 * or sum_q 2/n (<Z_q> - y) Z_q); the values are those of the shift rule.  Arguments as
 * qsv_param_shift_grad; loss is a host struct read during the call. */
qsv_status qsv_loss_grad(qsv_ctx* ctx, const qsv_circuit* c, const float* x_dev, int64_t dim,
                         const float* params_dev, const float* feats_dev, const qsv_loss* loss,
                         float* loss_dev, float* grad_dev, float* mean_loss_dev, float* mean_grad_dev);

/* A teacher known by its top logits: n_top entries for every row (or sample).  q_j = exp(t_j / T - norm), norm the
 * logarithm of the sum of exp(t_j / T) over the row's entries, or top_lse: the teacher's own logarithm of that sum over all
 * its outcomes, at the same T; Q = sum of q.  Entries with an index outside 0..cols-1 (padding) or a logit of -inf count
 * for nothing, and a row without any other has loss 0 and gradient 0; entries with the same index add up.  With one entry
 * a row (and its logit anything finite) the loss is the cross entropy of labels. */
typedef struct {
    int32_t n_top;               /* 1..1024 */
    int32_t reserved;            /* must be 0 */
    const int32_t* top_idx_dev;  /* [rows][n_top] */
    const float* top_logits_dev; /* [rows][n_top] */
    const float* top_lse_dev;    /* [rows] or NULL */
    double temperature;          /* T: 2^-100..2^100 */
} qsv_teacher;

/* Loss of rows of scores z of a student against a teacher's top logits, and its gradient:
 *   p = softmax(z / T),   loss = sum_j q_j (ln q_j - ln p_{i_j}),
 *   d loss / d z_k = g / T (Q p_k - sum over the entries j with i_j = k of q_j),   g = grad_loss (1 if NULL).
 * (No factor T^2 is put in: it can go into grad_loss.  g / T has to be in float32's range.)  Scores of -inf are masked: p = 0;
 * an entry with q > 0 there makes the loss +inf.  A NaN or +inf among a row's scores makes its loss and gradient NaN, unless the row has no entry.
 * stats: [rows][2], the row's highest score m and the sum of exp((z - m) / T); written when have_stats = 0, and read instead
 * of being worked out when have_stats = 1, which is the backward pass by itself (loss_dev must be NULL then).
 * The gradient has the type of the scores, rounded once, and may be written over them (the same address and row stride);
 * otherwise the two must not overlap.  Any of loss_dev, stats_dev and grad_dev may be NULL. */
typedef struct {
    int32_t kind;                /* QSV_S_F32, QSV_S_F16 or QSV_S_BF16 */
    int32_t have_stats;
    const void* scores_dev;      /* row r starts at element r * row_stride; aligned to its element */
    int64_t rows;                /* 0..2^24; 0 is a no-op */
    int64_t cols;                /* 1..2^30 */
    int64_t row_stride;          /* >= cols (any value for one row), in elements */
    float* loss_dev;             /* [rows] or NULL */
    float* stats_dev;            /* [rows][2] or NULL */
    const float* grad_loss_dev;  /* [rows] or NULL */
    void* grad_dev;              /* [rows] rows of cols, of the scores' type, or NULL */
    int64_t grad_stride;         /* >= cols (any value for one row), in elements */
} qsv_distill_req;

/* Workspace size in bytes that qsv_distill needs for such rows, that of the plans included; 0 on bad arguments.  (A call with
 * have_stats = 1 needs none beside the plans'.) */
size_t qsv_distill_workspace_bytes(int64_t rows, int64_t cols);
qsv_status qsv_distill(qsv_ctx* ctx, const qsv_distill_req* req, const qsv_teacher* teacher);

/* Per-sample loss [batch] and gradient [batch][P] of a circuit's own outcome distribution against a teacher's top logits
 * (outcomes 0..2^n-1; teacher arrays of batch rows), and optionally their batch means, in reverse mode as qsv_loss_grad:
 *   p_k = |a_k|^2 of the encoded sample's final state,   loss_b = sum_j q_j (ln q_j - ln p_{i_j}).
 * The teacher's temperature softens q alone.  An entry with q > 0 at an outcome of amplitude 0 makes the loss +inf; one at
 * an amplitude below 2^-126 adds nothing to the gradient.  Arguments as qsv_param_shift_grad; teacher is a host struct read
 * during the call.
 * qsv_distill_grad_workspace_bytes: the workspace with which this call works as qsv_loss_grad does with
 * qsv_grad_workspace_bytes, a state per sample more; with less it still works, layer by layer.  Returns 0 on bad arguments. */
size_t qsv_distill_grad_workspace_bytes(int n_qubits, int batch, const qsv_circuit* c);
qsv_status qsv_distill_grad(qsv_ctx* ctx, const qsv_circuit* c, const float* x_dev, int64_t dim,
                            const float* params_dev, const float* feats_dev, const qsv_teacher* teacher,
                            float* loss_dev, float* grad_dev, float* mean_loss_dev, float* mean_grad_dev);

/* Penalties for repeated outcomes, biases and masks on rows of scores (alone: probabilities and amplitudes have a norm to keep), before a
 * draw (qsv_sample) or a loss (qsv_distill):
 *   v = z
 *   s_k:  v = v > 0 ? v / R : v R           s_k: outcome k is among the row's earlier outcomes that count
 *   v -= F c_k + A [c_k > 0]                c_k: how often it is among those from prompt_len on
 *   v += b_k + sum over the entries j with i_j = k of e_j
 *   masked: v = -inf, whatever v is.
 * Earlier outcomes: the first prior_len entries of the row's prior, of which the first prompt_len (a prompt) count for R alone;
 * outcomes outside 0..cols-1 (padding) count for nothing.  Biases may be -inf; entries with an index outside 0..cols-1 count for
 * nothing, those with the same index add up in their order.  Bit k % 32 of word k / 32 of a mask allows outcome
 * k (bits behind cols are not looked at); a mask may leave a row without any.  A score of -inf stays -inf, NaN stays NaN.
 * A place with a history or an entry is worked out in float64 and rounded once to the scores' type (beyond its range: to infinity);
 * the others, a score plus a shared bias, are one sum in float32, rounded to that and to the type.
 * A row with a parameter out of its range (R not positive and finite, F or A not finite, not 0 <= prompt_len <= prior_len <= n_prior,
 * with n_prior = 0 too, a mask outside -1..n_masks-1) becomes NaN, which qsv_sample takes as a row without outcomes.
 * out may be the scores themselves (the same address and row stride): then only the places that change are written, and, without a
 * shared bias, read; otherwise the two must not overlap.  The other arrays must not overlap out. */
typedef struct {
    int32_t kind;                 /* QSV_S_F32, QSV_S_F16 or QSV_S_BF16 */
    int32_t n_entries;            /* 0..1023: a row's own biases */
    const void* scores_dev;       /* row r starts at element r * row_stride; aligned to its element */
    int64_t rows;                 /* 0..2^24; 0 is a no-op */
    int64_t cols;                 /* 1..2^30 */
    int64_t row_stride;           /* >= cols (any value for one row), in elements */
    void* out_dev;                /* of the scores' type */
    int64_t out_stride;           /* >= cols (any value for one row) */
    const int32_t* prior_dev;     /* row r starts at element r * prior_stride; may be NULL where n_prior = 0 */
    int64_t n_prior;              /* 0..2^20 */
    int64_t prior_stride;         /* >= n_prior (any value for one row) */
    const int32_t* prior_len_dev; /* [rows] or NULL (n_prior) */
    const int32_t* prompt_len_dev; /* [rows] or NULL (0) */
    const float* repetition_dev;  /* R: [rows] or NULL (1) */
    const float* frequency_dev;   /* F: [rows] or NULL (0) */
    const float* presence_dev;    /* A: [rows] or NULL (0) */
    const float* bias_dev;        /* b: [cols], the same for all rows, or NULL (0) */
    const int32_t* entry_idx_dev; /* i: [rows][n_entries] */
    const float* entry_bias_dev;  /* e: [rows][n_entries] */
    const uint32_t* masks_dev;    /* mask i starts at word i * mask_stride; NULL: all outcomes are allowed */
    int64_t n_masks;              /* 1..2^24 where masks_dev is given */
    int64_t mask_stride;          /* >= ceil(cols / 32) (any value for one mask) */
    const int32_t* mask_of_dev;   /* [rows]: the row's mask, -1: none; NULL: mask r for row r (n_masks = rows) or one for all (n_masks = 1) */
} qsv_adjust_req;

qsv_status qsv_adjust(qsv_ctx* ctx, const qsv_adjust_req* req);

/* The backward pass of qsv_adjust, G the gradient by its result and a_k 1 where the mask allows outcome k, 0 elsewhere:
 *   d / d z_k = a_k G_k f,  f = s_k ? (z_k > 0 ? 1 / R : R) : 1,
 *   d / d b_k = sum over the rows of a_k G_k,   d / d e_j = a_k G_k at k = i_j (0 for an index outside 0..cols-1).
 * A masked place gives 0 whatever G is there.  req is the forward call's: out_dev, out_stride, bias_dev and entry_bias_dev are not
 * looked at, and scores_dev may be NULL where it has no repetition_dev or no history, or where grad_dev is NULL.  G and grad have
 * the scores' type, rounded once.  grad may be G itself (the same address and row stride; then only the places that change are
 * written, and unless grad_bias_dev is asked for, read), and must not overlap the scores.  Sums over rows are in float64, in an order
 * that the sizes alone decide.  A row with a parameter out of its range gives NaN, in d / d b too.  Any of the results may be
 * NULL; but for grad over G they must not overlap each other or what is read.  Workspace: for grad_bias_dev alone, qsv_adjust_grad_workspace_bytes (that of the plans included; 0 on bad arguments). */
typedef struct {
    const void* grad_out_dev;     /* G: row r starts at element r * grad_out_stride */
    int64_t grad_out_stride;      /* >= cols (any value for one row) */
    void* grad_dev;               /* or NULL */
    int64_t grad_stride;          /* >= cols (any value for one row) */
    float* grad_bias_dev;         /* [cols] or NULL */
    float* grad_entry_dev;        /* [rows][n_entries] or NULL */
} qsv_adjust_grad_req;

size_t qsv_adjust_grad_workspace_bytes(int64_t rows, int64_t cols);
qsv_status qsv_adjust_grad(qsv_ctx* ctx, const qsv_adjust_req* req, const qsv_adjust_grad_req* grad);

/* Optimiser steps on the device, asynchronous on the context's stream; arithmetic in double, storage
 * float.  qsv_sgd_step: params -= lr * grad.  qsv_adam_step (Kingma and Ba, Algorithm 1): m, v are
 * the caller's moment buffers [count] (zero before the first step), t >= 1 the step count.
 * count = 0 is a no-op; bad arguments return QSV_ERR_INVALID_ARG. */
qsv_status qsv_sgd_step(qsv_ctx* ctx, float* params_dev, const float* grad_dev, int64_t count, double lr);
qsv_status qsv_adam_step(qsv_ctx* ctx, float* params_dev, const float* grad_dev, float* m_dev, float* v_dev,
                         int64_t count, int64_t t, double lr, double beta1, double beta2, double eps);

/* The norm of the gradients of many tensors together, and the gradients scaled to a highest norm:
 *   N = sqrt(sum over all values of g^2),  f = N > max_norm ? max_norm / N : 1,  out = f g.
 * Squares, their sum and the products are in float64; norm_dev (float32 [1] or NULL) receives N, and every value is rounded to float32
 * and to its tensor's type.  outs NULL: in place (nothing is written where f = 1); otherwise n tensors of the gradients' kinds and shapes.
 * max_norm = +inf: f = 1, so that with outs NULL the norm alone is worked out.  As arithmetic has it, a NaN among the gradients makes
 * N and, with a finite max_norm, all values NaN; an infinite one makes N infinite, finite values 0 and infinite ones NaN.
 * Results do not depend on anything but the list.  An out must be its own gradient (the same address and row stride) or overlap no
 * gradient, and outs must not overlap each other.  Columns of one buffer do not overlap: rows between each other's are told apart by where
 * they lie in the greatest common divisor of their row strides (a single row has the other's); rows that meet there are refused.  norm_dev
 * must lie in none of them.
 * The lists are host arrays of 2^38 values at most, read during the call.  No workspace beyond what qsv_workspace_bytes asks for. */
typedef struct {
    int32_t kind;        /* QSV_S_F32, QSV_S_F16 or QSV_S_BF16 */
    int32_t reserved;    /* must be 0 */
    void* data_dev;      /* row r starts at element r * row_stride; aligned to its element; may be NULL where it has no values */
    int64_t rows, cols;  /* >= 0 */
    int64_t row_stride;  /* >= cols (any value for one row), in elements, <= 2^38; (rows - 1) * row_stride <= 2^56 */
} qsv_tensor;

qsv_status qsv_clip_grads(qsv_ctx* ctx, const qsv_tensor* grads, const qsv_tensor* outs, int64_t n /* 0..4096 */, double max_norm /* >= 0 */,
                          float* norm_dev);

/* qsv_adam_step over many tensors at once, of the gradients times f of qsv_clip_grads (which are read, not written): the values
 * are those of qsv_adam_step on f g.  norm_dev receives N.  Where N, rounded to float32 as norm_dev has it, is not finite, nothing but
 * norm_dev is written: the step is left out.
 * max_norm = +inf: f = 1.  param, m and v of the tensors must not overlap each other or any gradient, and norm_dev must lie in none
 * of these. */
typedef struct {
    int32_t kind;          /* of the gradient: QSV_S_F32, QSV_S_F16 or QSV_S_BF16 */
    int32_t reserved;      /* must be 0 */
    float* param_dev;      /* [count] */
    const void* grad_dev;  /* [count] */
    float* m_dev;          /* [count] */
    float* v_dev;          /* [count] */
    int64_t count;         /* 0..2^38 */
} qsv_adam_tensor;

qsv_status qsv_adam_clipped(qsv_ctx* ctx, const qsv_adam_tensor* tensors, int64_t n /* 0..4096 */, int64_t t, double lr, double beta1,
                            double beta2, double eps, double max_norm, float* norm_dev);

/* Host-only introspection of the pass plan the library would run for a circuit (no GPU needed):
 * writes a text description (one line per pass, one token per operation) into buf and returns the
 * number of bytes needed (excluding the terminator), or -1 on a bad descriptor.  tile_log2 = 0
 * picks the library's default tile size.  Used by the host-logic tests. */
int64_t qsv_plan_describe(const qsv_circuit* c, int n_qubits, int batch, int inverse,
                          int tile_log2, char* buf, int64_t buf_bytes);

/* Measurement aid: one pass of the fused-pass kernel that only loads every tile (low_bits low index
 * bits plus a window starting at bit window_start, as the planner would choose), moves the
 * register run through LDS `transposes` times and stores the tile back unchanged.  It gives the
 * streaming ceiling of the pass kernel's access pattern, with no gate arithmetic.  The state is
 * left as it was.  Unlike every other call it synchronises the stream once (after uploading its
 * operation list) and must not be called while the stream is being captured. */
qsv_status qsv_probe_pass(qsv_ctx* ctx, int low_bits, int window_start, int transposes);

/* Testing/tuning knobs: tile_log2 in 10..14 (0 = default: 11, 12 or 13 by the number of qubits, of layers and
 * of amplitudes) forces the tile size of the fused pass kernel (14 exists with one LDS plane only);
 * defer_cnots = 1 / 0 lets qsv_apply_layers carry the CNOTs whose target qubit lies outside a pass's tile by the index the pass writes each amplitude to
 * (fewer passes over the state; such passes write a second buffer taken from the workspace), or keeps
 * every CNOT a register operation (-1, the default, defers whenever the circuit has a CNOT ring, more
 * qubits than the tile has index bits, at most 28 of them, and the workspace has room for a copy of
 * the state; the result is the same up to rounding order); load_store_priority = 1 (default) / 0 lets
 * the pass kernel's wavefronts raise their issue priority while they issue a tile's loads and stores (the
 * layer-by-layer reverse-mode sweep on two streams does so below 18 qubits only, the one in whole passes never);
 * small_apply = 1 (default) / 0 lets qsv_apply_layers run states of at most 10 qubits and 2^21 amplitudes in
 * all (10 qubits: 2^20) in one launch with the gates in registers and lane exchanges (the kernel of qsv_forward_small, started
 * from the state; measured 1.6 to 4 times faster there than the fused passes, whose launches cost more than
 * their arithmetic on such states), or always takes the fused passes; with it qsv_adjoint_grad and
 * qsv_loss_grad run circuits of at most 10 qubits and 512 unitaries (layers times qubits) in one launch too (10 qubits
 * without re-uploading: up to 2^20 amplitudes where the workspace has room for more),
 * unless tile_log2, naive, grad_layered = 0 or grad_chunk_rows is set or the workspace has no room for
 * its matrices and sums (1 KiB at most per sample and layer);
 * small_regs = 2, 3 or 4 fixes the amplitudes per thread of qsv_forward_small at 4, 8 or 16 (0, the
 * default, takes the most that still gives the chip about four wavefronts per SIMD); low_bits in 3..10
 * (0 = default) forces the planner's minimum number of low index bits per tile; lds_planes = 1 (default) moves real and imaginary parts through one LDS plane one
 * after the other, 2 through two planes at once; naive = 1 routes qsv_apply_layers through the
 * one-gate-per-launch kernels; grad_layered = 0 makes qsv_param_shift_grad run every shifted
 * circuit whole and the reverse-mode calls take psi back beside lambda, a layer at a time; nt_store = 1 / 0 forces nontemporal / ordinary tile stores in the fused pass (-1,
 * the default, for passes that touch 384 MiB or more); reverse_passes = 1 / 0 makes every other fused
 * pass take its tiles from the last to the first, so that it starts with what the pass before it
 * wrote last, or not (-1, the default, is 1; the result does not depend on it); split_streams = 1 / 0 sends the state rows through a sequence of fused passes as
 * two halves, the second on a stream of the library's own that forks from and rejoins the caller's
 * stream inside the call, or not (-1, the default, does so from 32 MiB of states; it takes at least two rows and more
 * qubits than the tile has index bits; the result does not depend on it);
 * probe_layout in 0..9 (-1 = the highest) sets the register run qsv_probe_pass loads
 * and stores the tile in; grad_chunk_rows in 1..32768 (0 = as many as fit) caps the circuits per
 * launch of qsv_param_shift_grad.  Unknown names and values out of range return
 * QSV_ERR_INVALID_ARG. */
qsv_status qsv_set_option(qsv_ctx* ctx, const char* name, int64_t value);

#ifdef __cplusplus
}
#endif
#endif /* QSV_H */
