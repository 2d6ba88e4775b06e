/*
 * rslx — single-GPU (gfx950) library for the data-parallel hot path of a GPU-only PPO
 * training loop: batched actor-critic inference (act), the GAE / returns reverse scan,
 * the multi-epoch minibatch PPO update, the DAgger-style behaviour-cloning update,
 * symmetry augmentation and the RND curiosity reward.
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 *  - Plain C ABI.  Every function returns an int32 status (RSLX_OK = 0); on failure nothing
 *    has been launched unless stated, and rslx_last_error() gives a thread-local message.
 *  - "device" pointers are HIP device memory owned by the caller.  The library never
 *    allocates, frees or keeps them.  Scratch memory comes from the caller's workspace
 *    (`ws`, `ws_bytes`), sized by the matching *_workspace_bytes() query; a workspace that is
 *    too small gives RSLX_ERR_WORKSPACE.  Where a call has a faster form that needs more memory
 *    (rslx_ppo_update and rslx_bc_update of small networks, rslx_act_recurrent, rslx_memory_step;
 *    and their _dc forms), the query asks for the larger size and a workspace that holds the
 *    general form is taken too: the call then runs in that form, whose results differ in their
 *    last bits.  Device pointers must be 16-byte aligned.
 *  - "host" pointers are ordinary host memory, read (or written) before the call returns.
 *  - All matrices are dense row-major fp32 unless said otherwise.
 *  - All work is enqueued on `stream` (a hipStream_t passed as void*; NULL = default stream).
 *    No entry point synchronises with the host; outputs are valid once the stream reaches
 *    the end of the enqueued work.  Calls that share a workspace must be stream-ordered.
 *  - Flat parameter layout of a network (struct rslx_mlp): for each linear layer l in order,
 *    W_l as [dims[l], dims[l+1]] row-major (y = x W + b), then b_l [dims[l+1]]; an actor's
 *    buffer ends with log_std[dims[n_layers]].  grads / adam_m / adam_v mirror this layout.
 *    Hidden layers use ELU with parameter elu_alpha; the last layer is linear.
 */
#ifndef RSLX_H
#define RSLX_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define RSLX_OK 0
#define RSLX_ERR_INVALID_ARG 1
#define RSLX_ERR_SHAPE 2
#define RSLX_ERR_WORKSPACE 3
#define RSLX_ERR_HIP 4
#define RSLX_ERR_UNSUPPORTED 5

#define RSLX_MAX_LAYERS 8
#define RSLX_MAX_ACTIONS 64

/* Columns of the per-minibatch statistics rows written by the update calls. */
#define RSLX_NSTATS 8
#define RSLX_STAT_SURROGATE 0
#define RSLX_STAT_VALUE_LOSS 1
#define RSLX_STAT_ENTROPY 2
#define RSLX_STAT_KL 3
#define RSLX_STAT_GRAD_NORM 4 /* before clipping */
#define RSLX_STAT_CLIP_FRAC 5
#define RSLX_STAT_MIRROR_LOSS 6
#define RSLX_STAT_RND_LOSS 7
/* rslx_bc_update uses column 0 for the MSE loss and column 4 for the gradient norm. */

/* rslx_act flags */
#define RSLX_ACT_DETERMINISTIC 1u /* actions := mu (no noise) */
#define RSLX_ACT_VALUES_ONLY 2u   /* only the critic runs; only `values` is written */

/* A multi-layer perceptron over caller-owned device buffers (paper Sec. 3, "Network"). */
typedef struct rslx_mlp {
  int32_t n_layers;                  /* number of linear layers, 1..RSLX_MAX_LAYERS */
  int32_t dims[RSLX_MAX_LAYERS + 1]; /* dims[0] = input width, dims[n_layers] = output width */
  float elu_alpha;                   /* ELU parameter of the hidden layers (workloads use 1) */
  int32_t has_log_std;               /* 1: params end with log_std[dims[n_layers]] (actor) */
  float* params;                     /* device, flat layout above */
  float* grads;                      /* device, same layout; NULL for frozen networks */
  float* adam_m;                     /* device, same layout; NULL for frozen networks */
  float* adam_v;                     /* device, same layout; NULL for frozen networks */
} rslx_mlp;

/* Rollout storage [T, N, .] flattened to B = T*N rows, flat row b = t*N + n (paper Sec. 3:
 * the Runner stores what act() and the environment return; all device, read-only). */
typedef struct rslx_rollout {
  int32_t T, N;            /* steps per rollout, parallel environments */
  int32_t Da, Dc, A;       /* actor obs width, critic obs width, action width */
  const float* obs_actor;  /* [B, Da] */
  const float* obs_critic; /* [B, Dc] (may alias obs_actor) */
  const float* actions;    /* [B, A] */
  const float* logp;       /* [B]  log-density of actions under the collecting policy */
  const float* values;     /* [B]  critic values at collection */
  const float* mu;         /* [B, A] collecting policy mean (KL statistic) */
  const float* sigma;      /* [B, A] collecting policy std  (KL statistic) */
  const float* advantages; /* [B]  (normalised) advantages from rslx_gae */
  const float* returns;    /* [B]  returns from rslx_gae */
} rslx_rollout;

/* Hyper-parameters of the PPO update (paper Sec. 2.1; Schulman et al. 2017). */
typedef struct rslx_ppo_cfg {
  float clip;          /* epsilon of the ratio clip and of the value clip */
  float value_coef;    /* c_v */
  float entropy_coef;  /* c_e */
  float max_grad_norm; /* global L2 clip; <= 0 or inf disables */
  float lr, beta1, beta2, adam_eps;
  int32_t epochs;      /* E */
  int32_t minibatches; /* M; B % M must be 0 */
  int32_t use_clipped_value_loss;
  uint64_t seed;        /* permutation stream */
  uint64_t call_index;  /* permutation stream: which update call */
  int32_t epoch_offset; /* permutation of epoch e uses e + epoch_offset (resume mid-update) */
} rslx_ppo_cfg;

/* Mirror maps (paper Sec. 2.2): mirror(x)[j] = sign[j] * x[perm[j]].  The host copies are
 * validated (each must be a signed permutation with mirror o mirror = id).  The device copies are
 * what the kernels read.  rslx_ppo_update accepts all six device pointers NULL: it then uploads
 * the validated host copies into its workspace itself (hipMemcpyAsync from the caller's host arrays
 * on the call's stream: not under stream capture, where device copies must be passed).  Where
 * device copies are passed they must hold the same values as the host copies; the library cannot
 * check that.  rslx_sym_augment has no workspace and needs the device copies. */
typedef struct rslx_sym {
  const int32_t* perm_obs_a_host; const float* sign_obs_a_host; /* [Da] */
  const int32_t* perm_obs_c_host; const float* sign_obs_c_host; /* [Dc] */
  const int32_t* perm_act_host;   const float* sign_act_host;   /* [A]  */
  const int32_t* perm_obs_a; const float* sign_obs_a;           /* device copies */
  const int32_t* perm_obs_c; const float* sign_obs_c;
  const int32_t* perm_act;   const float* sign_act;
  float mirror_loss_coef; /* c_sym; 0 keeps the augmentation and drops the loss term */
} rslx_sym;

/* RND predictor training inside the PPO update (paper Sec. 2.2). */
typedef struct rslx_rnd_train {
  const rslx_mlp* target;    /* frozen */
  rslx_mlp* predictor;       /* trained: params, grads, adam_m, adam_v required */
  const int32_t* subset_idx; /* device [n_subset] columns of obs_actor fed to both nets, or NULL = all */
  int32_t n_subset;          /* must equal target->dims[0]; Da when subset_idx is NULL */
  float lr;                  /* predictor's own Adam learning rate (betas/eps as in the PPO cfg) */
  int64_t* adam_step;        /* host, in-out: predictor's own step counter */
} rslx_rnd_train;

/* Hyper-parameters of the behaviour-cloning update (paper Sec. 2.1, DAgger-style BC). */
typedef struct rslx_bc_cfg {
  float lr, beta1, beta2, adam_eps;
  float max_grad_norm; /* <= 0 disables clipping */
  int32_t epochs, minibatches;
  uint64_t seed, call_index;
  int32_t epoch_offset;
} rslx_bc_cfg;

/* ---- housekeeping ------------------------------------------------------------------- */

/* Library version as major*10000 + minor*100 + patch. */
int32_t rslx_version(void);
/* Message of the last failure on the calling thread ("" if none).  Never NULL. */
const char* rslx_last_error(void);
/* RSLX_OK if the current HIP device is a gfx950 part, RSLX_ERR_UNSUPPORTED / RSLX_ERR_HIP otherwise. */
int32_t rslx_device_check(void);

/* ---- launch trace (measurement aid) ---------------------------------------------------------- */

/* While a trace is open, every kernel launch of the library is bracketed by a pair of HIP events on
 * its stream and tagged with its algorithmic work.  rslx_trace_begin clears any earlier trace and
 * keeps at most max_records launches.  A launch that runs two networks in different forms side by side leaves a record for
 * each of them, both with the launch's time.  rslx_trace_end stops recording, WAITS on the host for the
 * recorded events, and copies up to `cap` records (launch order) to `out` (host); *n_out receives the
 * number recorded.  Calling it with out == NULL only reports the count and keeps the records for a
 * second call.  Launches beyond max_records are counted, not recorded: rslx_trace_end then still
 * delivers the records it has and returns RSLX_ERR_WORKSPACE.  `kernel` names a launch site: "gemm_<fwd|dx|dw>_<BM>x<BN>" are the matrix-core
 * kernels (flops = 2 M N K summed over the grouped problems), the others are streaming kernels
 * (bytes = algorithmic HBM bytes).  Not thread-safe; tracing costs two event records per launch. */
typedef struct rslx_trace_record {
  char kernel[48];
  double flops;
  double bytes;
  float ms;
} rslx_trace_record;
int32_t rslx_trace_begin(int32_t max_records);
int32_t rslx_trace_end(rslx_trace_record* out, int32_t cap, int32_t* n_out);

/* ---- permutation of one epoch (first step of the update: minibatch order) -------------- */

/* Shuffled minibatch order (paper Sec. 2.1: multi-epoch minibatch updates; the generator is this
 * library's own):  mix64 = SplitMix64 output function,
 *   key_i = mix64(mix64(mix64(mix64(seed) ^ call_index) ^ epoch) ^ i),  i in [0, B)
 *   perm  = indices sorted ascending by (key_i, i).
 * perm_out: device int32 [B].  Result is bit-exact and independent of scheduling. */
size_t rslx_permutation_workspace_bytes(int32_t B);
int32_t rslx_permutation(uint64_t seed, uint64_t call_index, int32_t epoch, int32_t B,
                         int32_t* perm_out, void* ws, size_t ws_bytes, void* stream);

/* ---- act(): one rollout step (paper Sec. 2.1 / Sec. 3: Runner -> Algorithm.act) ------ */

/* mu = actor(obs_actor), V = critic(obs_critic); sigma = exp(log_std);
 * a = mu + sigma * eps;  logp = -1/2 sum ((a-mu)/sigma)^2 - sum log sigma - A/2 log(2 pi).
 * eps: device [N, A] standard-normal noise, or NULL to draw it from the counter generator
 *   h = mix64(mix64(mix64(seed ^ 0xAC7) ^ step) ^ (n*A + j)); u1 = ((h>>40)+1) 2^-24;
 *   u2 = ((h>>8) & 0xFFFFFF) 2^-24; eps = sqrt(-2 ln u1) cos(2 pi u2).
 * Outputs (device): actions [N,A], logp [N], values [N], mu [N,A], sigma [N,A]; typically
 * pointers into slot t of the rollout storage.  With RSLX_ACT_VALUES_ONLY only `values` is
 * written and actor / actor outputs may be NULL. */
size_t rslx_act_workspace_bytes(const rslx_mlp* actor, const rslx_mlp* critic, int32_t N);
int32_t rslx_act(const rslx_mlp* actor, const rslx_mlp* critic, const float* obs_actor,
                 const float* obs_critic, int32_t N, uint64_t seed, uint64_t step,
                 const float* eps_or_null, float* actions, float* logp, float* values, float* mu,
                 float* sigma, uint32_t flags, void* ws, size_t ws_bytes, void* stream);

/* ---- GAE / returns (paper Sec. 2.1; time-limit handling Sec. 3) ---------------------- */

/* With V_T = last_values and A_T = 0, for t = T-1..0:
 *   delta = r_t + gamma (1-d_t) V_{t+1} - V_t;  A_t = delta + gamma lam (1-d_t) A_{t+1};
 *   R_t = A_t + V_t.   If timeouts != NULL, r_t is first replaced by r_t + gamma V_t timeout_t.
 * If normalize_adv != 0, advantages are then replaced by (A - mean) / (std + 1e-8) with the
 * mean and the unbiased (n-1) std taken over all T*N entries; returns use the raw A.
 * rewards, values [T,N]; last_values [N]; dones, timeouts uint8 [T,N]; outputs [T,N]. All device.
 * advantages and returns may be the buffers rewards and values themselves (one each, in either order),
 * which are then overwritten; they must not overlap an input in any other way, nor each other. */
size_t rslx_gae_workspace_bytes(int32_t T, int32_t N);
int32_t rslx_gae(const float* rewards, const float* values, const float* last_values,
                 const uint8_t* dones, const uint8_t* timeouts_or_null, int32_t T, int32_t N,
                 float gamma, float lam, int32_t normalize_adv, float* advantages, float* returns,
                 void* ws, size_t ws_bytes, void* stream);

/* rslx_gae for callers that cannot allocate or hand over a workspace (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc).  Same arguments, layouts,
 * results (bit for bit) and error behaviour as rslx_gae, without ws / ws_bytes: the partial sums
 * of the advantage normalisation live in a 65 600-byte array inside the library's device image,
 * of which every GPU the library runs on holds its own copy until the process ends.  The call
 * allocates and frees nothing (with rslx_trace_begin active the trace still creates events).
 * Limit: N <= RSLX_GAE_NOALLOC_MAX_ENVS, else RSLX_ERR_SHAPE and nothing is launched (T is not
 * limited).  All calls on one GPU share that GPU's array: calls that overlap on one GPU (two
 * streams, two host threads) race on it and must be serialised by the caller; calls on one
 * stream, and replays of a graph that holds one, are ordered and need no clearing in between. */
#define RSLX_GAE_NOALLOC_MAX_ENVS (1 << 20)
int32_t rslx_gae_noalloc(const float* rewards, const float* values, const float* last_values,
                         const uint8_t* dones, const uint8_t* timeouts_or_null, int32_t T,
                         int32_t N, float gamma, float lam, int32_t normalize_adv,
                         float* advantages, float* returns, void* stream);

/* ---- fused gradient-clip + Adam over one flat buffer (last steps of the update) -------- */

/* s = min(1, max_grad_norm / (||g||_2 + 1e-6)) (1 when max_grad_norm <= 0), then Adam
 * (Kingma & Ba 2015) with g*s:  m,v moments in place, bias correction with step t = *adam_step+1,
 * theta -= lr * m_hat / (sqrt(v_hat) + eps).  *adam_step (host) is incremented.
 * params, grads, m, v: device [n].  grad_norm_out: device float[1] or NULL. */
size_t rslx_adam_workspace_bytes(int64_t n);
int32_t rslx_adam_step(float* params, const float* grads, float* m, float* v, int64_t n, float lr,
                       float beta1, float beta2, float eps, float max_grad_norm, int64_t* adam_step,
                       float* grad_norm_out, void* ws, size_t ws_bytes, void* stream);

/* ---- PPO update (paper Sec. 2.1, 2.2, 3) ---------------------------------------------- */

/* E epochs x M minibatches over the B = T*N rollout rows.  For every minibatch (rows
 * perm_e[m*mb : (m+1)*mb], mb = B/M): forward of actor and critic, Gaussian log-density and
 * entropy, ratio = exp(logp_new - logp_old),
 *   L_pi = mean max(-A ratio, -A clamp(ratio, 1-clip, 1+clip))
 *   L_V  = mean max((V-R)^2, (V_old + clamp(V-V_old, -clip, clip) - R)^2)   (or mean (R-V)^2)
 *   L    = L_pi + c_v L_V - c_e mean(entropy) [+ c_sym L_mirror]
 * backward, one global gradient norm over actor (with log_std) and critic, clip, Adam.
 * With `sym`: every minibatch is followed by its mirrored copy (2*mb rows; obs and actions
 * mirrored, advantages / returns / old values / old log-densities copied), means run over
 * 2*mb rows, and L_mirror = mean over mb rows and A dims of
 * (mu(mirror(o)) - stopgrad(mirror_a(mu(o))))^2.
 * With `rnd`: the predictor is trained on the same rows with its own Adam on
 * mean((pred(x) - target(x))^2), outside the PPO gradient norm.
 * In-out: actor/critic params, adam_m, adam_v (device), *adam_step (host, shared by both nets).
 * Out: grads hold the last minibatch's unclipped gradient; stats: device [E*M, RSLX_NSTATS].
 * Action widths up to RSLX_MAX_ACTIONS; the fused output-layer + loss launch covers A <= 32 with
 * last hidden widths of 32, 64 or a multiple of 4 from 68 to 256 (other widths than 128 and 256 up
 * to as many minibatch rows as it pays), everything else runs the same arithmetic unfused. */
size_t rslx_ppo_update_workspace_bytes(const rslx_mlp* actor, const rslx_mlp* critic,
                                       const rslx_rollout* ro, const rslx_ppo_cfg* cfg,
                                       const rslx_sym* sym_or_null, const rslx_rnd_train* rnd_or_null);
int32_t rslx_ppo_update(rslx_mlp* actor, rslx_mlp* critic, const rslx_rollout* ro,
                        const rslx_ppo_cfg* cfg, const rslx_sym* sym_or_null,
                        const rslx_rnd_train* rnd_or_null, int64_t* adam_step, float* stats,
                        void* ws, size_t ws_bytes, void* stream);

/* ---- replayable variants: call-to-call counters in device memory ----------------------- */

/* The iteration of paper Sec. 3 (T x act, advantage estimation, update) is a fixed sequence of
 * launches; a caller that records it once (HIP graph) and replays it needs every value that
 * changes between iterations to live in device memory.  rslx_dev_counters (device, 32 bytes)
 * holds them; the *_dc entry points read it in their kernels and advance it with a kernel of
 * their own, so host arguments are the same for every replay:
 *   act_step       noise stream position: rslx_act_dc draws with step = act_step, then act_step += 1
 *                  (not with RSLX_ACT_VALUES_ONLY, which draws nothing)
 *   call_index     permutation stream of rslx_ppo_update_dc (cfg->call_index is ignored), += 1 per call
 *   adam_step      optimiser steps of actor + critic so far, += epochs * minibatches per call
 *   rnd_adam_step  the same for the RND predictor (rnd->adam_step is ignored)
 * Everything else is as in rslx_act / rslx_ppo_update; the bias corrections 1 - beta^t are formed
 * in fp64 on the device.  The caller initialises the struct (e.g. zeros) and must not run two
 * calls that share it concurrently. */
typedef struct rslx_dev_counters {
  int64_t act_step;
  uint64_t call_index;
  int64_t adam_step;
  int64_t rnd_adam_step;
} rslx_dev_counters;

int32_t rslx_act_dc(const rslx_mlp* actor, const rslx_mlp* critic, const float* obs_actor,
                    const float* obs_critic, int32_t N, uint64_t seed, rslx_dev_counters* counters,
                    const float* eps_or_null, float* actions, float* logp, float* values, float* mu,
                    float* sigma, uint32_t flags, void* ws, size_t ws_bytes, void* stream);
int32_t rslx_ppo_update_dc(rslx_mlp* actor, rslx_mlp* critic, const rslx_rollout* ro,
                           const rslx_ppo_cfg* cfg, const rslx_sym* sym_or_null,
                           const rslx_rnd_train* rnd_or_null, rslx_dev_counters* counters,
                           float* stats, void* ws, size_t ws_bytes, void* stream);

/* ---- recurrent actor-critic (paper Sec. 3: hidden states managed across roll-outs, BPTT) ---- */

/* A recurrent memory in front of an MLP, one of two cells over one flat device buffer
 *   W_ih [in_dim, G*H] row-major, b_ih [G*H], W_hh [H, G*H] row-major, b_hh [G*H]      (H = hidden)
 * RSLX_CELL_GRU (G = 3, gate order r, z, n; Cho et al. 2014 with the reset gate on the hidden-side
 * candidate term, bias included), state per row: h [H]
 *   gi = x W_ih + b_ih,  gh = h W_hh + b_hh
 *   r = sigmoid(gi_r + gh_r), z = sigmoid(gi_z + gh_z), n = tanh(gi_n + r gh_n), h' = (1-z) n + z h
 * RSLX_CELL_LSTM (G = 4, gate order i, f, g, o; forget gate, no peepholes), state per row: [h | c] [2H]
 *   a = x W_ih + b_ih + h W_hh + b_hh
 *   i = sigmoid(a_i), f = sigmoid(a_f), g = tanh(a_g), o = sigmoid(a_o), c' = f c + i g, h' = o tanh(c')
 * "State" below always means the packed row of width S = H (GRU) or 2H (LSTM); the MLP reads h.
 * hidden must be a multiple of 4; buffers 16-byte aligned; grads/adam_* NULL for inference. */
#define RSLX_CELL_GRU 0
#define RSLX_CELL_LSTM 1
typedef struct rslx_memory {
  int32_t cell;
  int32_t in_dim, hidden;
  float* params;
  float* grads;
  float* adam_m;
  float* adam_v;
} rslx_memory;

/* One roll-out step of a recurrent actor-critic: each network is a memory whose new hidden state
 * feeds its MLP (mlp.dims[0] == memory.hidden).  For every environment n:
 *   sin = reset[n] ? 0 : s[n];   s[n] <- cell(obs[n], sin);   mu, V = MLPs(h of s[n]);  then as rslx_act.
 * reset_or_null (device uint8 [N]) carries the previous step's episode-end flags.  h_actor
 * [N, S_a] and h_critic [N, S_c] (device, packed states) are updated in place; when h0_actor_out / h0_critic_out
 * are not NULL they receive sin, the state the step started from - the roll-out's first step
 * stores it for rslx_ppo_update_recurrent.  With RSLX_ACT_VALUES_ONLY only the critic runs and
 * NO state is written (the bootstrap value of the observation that opens the next roll-out).
 * Everything else (noise, outputs, flags, errors) is as in rslx_act. */
size_t rslx_act_recurrent_workspace_bytes(const rslx_memory* mem_actor, const rslx_mlp* actor,
                                          const rslx_memory* mem_critic, const rslx_mlp* critic, int32_t N);
int32_t rslx_act_recurrent(const rslx_memory* mem_actor, const rslx_mlp* actor, const rslx_memory* mem_critic,
                           const rslx_mlp* critic, const float* obs_actor, const float* obs_critic,
                           int32_t N, float* h_actor, float* h_critic, const uint8_t* reset_or_null,
                           float* h0_actor_out, float* h0_critic_out, uint64_t seed, uint64_t step,
                           const float* eps_or_null, float* actions, float* logp, float* values,
                           float* mu, float* sigma, uint32_t flags, void* ws, size_t ws_bytes,
                           void* stream);

/* PPO update of a recurrent actor-critic with back-propagation through time.  Minibatches are
 * whole environment columns: per epoch the N environments are shuffled (the permutation stream of
 * rslx_ppo_update, over N instead of T*N) and minibatch m takes the m-th slice of N / minibatches
 * environments with all T steps, rows ordered step-major.  Each minibatch is re-run through both
 * memories from h0 (the packed states the roll-out's first step started from, [N, S]) with the state
 * zeroed after every step whose `dones` flag is set; the loss of rslx_ppo_update (means over the
 * T * N / minibatches samples) is back-propagated through the MLPs into the hidden states and
 * through time, truncated at the roll-out start and never across an episode end.  One gradient
 * norm over the four parameter sets, one Adam step counter.  ro->Da / ro->Dc are the memories' input
 * widths; both memories use the same cell.  dones: device uint8 [T, N].  N % minibatches != 0 is RSLX_ERR_SHAPE.  Symmetry and RND
 * are not available here.  grads of all four hold the last minibatch's gradient on return. */
size_t rslx_ppo_update_recurrent_workspace_bytes(const rslx_memory* mem_actor, const rslx_mlp* actor,
                                                 const rslx_memory* mem_critic, const rslx_mlp* critic,
                                                 const rslx_rollout* ro, const rslx_ppo_cfg* cfg);
int32_t rslx_ppo_update_recurrent(rslx_memory* mem_actor, rslx_mlp* actor, rslx_memory* mem_critic,
                                  rslx_mlp* critic, const rslx_rollout* ro, const uint8_t* dones,
                                  const float* h0_actor, const float* h0_critic, const rslx_ppo_cfg* cfg,
                                  int64_t* adam_step, float* stats, void* ws, size_t ws_bytes,
                                  void* stream);

/* Replayable variants (see rslx_dev_counters): the noise position / permutation stream / optimiser
 * step count come from device memory and are advanced by the calls' own kernels, so a recurrent
 * iteration can be recorded as a HIP graph like a feed-forward one. */
int32_t rslx_act_recurrent_dc(const rslx_memory* mem_actor, const rslx_mlp* actor, const rslx_memory* mem_critic,
                              const rslx_mlp* critic, const float* obs_actor, const float* obs_critic,
                              int32_t N, float* h_actor, float* h_critic, const uint8_t* reset_or_null,
                              float* h0_actor_out, float* h0_critic_out, uint64_t seed,
                              rslx_dev_counters* counters, const float* eps_or_null, float* actions,
                              float* logp, float* values, float* mu, float* sigma, uint32_t flags,
                              void* ws, size_t ws_bytes, void* stream);
int32_t rslx_ppo_update_recurrent_dc(rslx_memory* mem_actor, rslx_mlp* actor, rslx_memory* mem_critic,
                                     rslx_mlp* critic, const rslx_rollout* ro, const uint8_t* dones,
                                     const float* h0_actor, const float* h0_critic, const rslx_ppo_cfg* cfg,
                                     rslx_dev_counters* counters, float* stats, void* ws, size_t ws_bytes,
                                     void* stream);

/* One step of a single memory (the recurrent student of the distillation loop, paper Sec. 2.1 with
 * Sec. 3): sin = reset[n] ? 0 : s[n];  s[n] <- cell(obs[n], sin), in place on the packed state
 * s [N, S]; s0_out (optional, [N, S]) receives sin; h_dense_out (optional, [N, H]) receives the
 * new hidden state as a dense matrix (for a GRU the state itself is that matrix).  The student's
 * action and the expert's label then come from
 * rslx_bc_collect(student_mlp, teacher, hidden state, obs_teacher, ...). */
size_t rslx_memory_step_workspace_bytes(const rslx_memory* mem, int32_t N);
int32_t rslx_memory_step(const rslx_memory* mem, const float* obs, int32_t N, float* s,
                         const uint8_t* reset_or_null, float* s0_out, float* h_dense_out, void* ws,
                         size_t ws_bytes, void* stream);

/* Behaviour cloning of a recurrent student (memory + MLP, student->dims[0] == mem->hidden) on
 * a roll-out: obs_student [T, N, Ds], targets [T, N, A] (the expert's actions on the visited
 * states), dones uint8 [T, N], h0 [N, S] (the packed state the roll-out's first step started from); all
 * device.  Minibatches are whole environment columns as in rslx_ppo_update_recurrent (cfg's
 * permutation stream over N; N % minibatches != 0 is RSLX_ERR_SHAPE); per minibatch
 * L = mean over the T * N / minibatches rows and the A action dims of (student - target)^2,
 * back-propagated through the MLP and through time, optional clip, Adam (one step counter for
 * memory and MLP).  stats as in rslx_bc_update. */
size_t rslx_bc_update_recurrent_workspace_bytes(const rslx_memory* mem, const rslx_mlp* student, int32_t T,
                                                int32_t N, const rslx_bc_cfg* cfg);
int32_t rslx_bc_update_recurrent(rslx_memory* mem, rslx_mlp* student, const float* obs_student,
                                 const float* targets, const uint8_t* dones, const float* h0, int32_t T,
                                 int32_t N, const rslx_bc_cfg* cfg, int64_t* adam_step, float* stats,
                                 void* ws, size_t ws_bytes, void* stream);

/* ---- behaviour cloning update (paper Sec. 2.1) ---------------------------------------- */

/* targets = teacher(obs_teacher) (once; or the caller's precomputed `targets_or_null` [B, A]);
 * per minibatch L = mean over rows and action dims of (student(obs_student) - target)^2,
 * backward, optional clip, Adam.  obs_student [B, Ds], obs_teacher [B, Dt] device.
 * stats: device [E*M, RSLX_NSTATS] (column 0 loss, column 4 gradient norm, others 0). */
size_t rslx_bc_update_workspace_bytes(const rslx_mlp* student, const rslx_mlp* teacher, int32_t B,
                                      const rslx_bc_cfg* cfg);
int32_t rslx_bc_update(rslx_mlp* student, const rslx_mlp* teacher, const float* obs_student,
                       const float* obs_teacher, const float* targets_or_null, int32_t B,
                       const rslx_bc_cfg* cfg, int64_t* adam_step, float* stats, void* ws,
                       size_t ws_bytes, void* stream);

/* As rslx_bc_update with the permutation stream (counters->call_index, += 1) and the optimiser step
 * count (counters->adam_step, += epochs * minibatches) in device memory; cfg->call_index is ignored.
 * See rslx_dev_counters. */
int32_t rslx_bc_update_dc(rslx_mlp* student, const rslx_mlp* teacher, const float* obs_student,
                          const float* obs_teacher, const float* targets_or_null, int32_t B,
                          const rslx_bc_cfg* cfg, rslx_dev_counters* counters, float* stats, void* ws,
                          size_t ws_bytes, void* stream);

/* One collection step of the distillation loop (paper Sec. 2.1: the student is rolled out, the
 * expert relabels what it visits): actions = student(obs_student) (mean action, no noise) and
 * targets = teacher(obs_teacher) for the same N states, one launch for both networks.
 * obs_student [N, Ds], obs_teacher [N, Dt], actions [N, A], targets [N, A]; all device.  The
 * targets written over a rollout are what rslx_bc_update takes as `targets_or_null`.
 * RSLX_ERR_SHAPE if the two networks' output widths differ. */
size_t rslx_bc_collect_workspace_bytes(const rslx_mlp* student, const rslx_mlp* teacher, int32_t N);
int32_t rslx_bc_collect(const rslx_mlp* student, const rslx_mlp* teacher, const float* obs_student,
                        const float* obs_teacher, int32_t N, float* actions, float* targets, void* ws,
                        size_t ws_bytes, void* stream);

/* ---- symmetry augmentation (paper Sec. 2.2) -------------------------------------------- */

/* obs_out[0:B] = obs_in, obs_out[B:2B][:, j] = sign_obs_a[j] * obs_in[:, perm_obs_a[j]]; the same
 * for actions with perm_act / sign_act.  Uses the *_obs_a and *_act maps of `sym` (host copies
 * validated, device copies read by the kernel).  obs_in [B, D], act_in [B, A] (either may be
 * NULL to skip it), outputs [2B, D], [2B, A]; all device.  RSLX_ERR_INVALID_ARG if a map is not
 * an involutive signed permutation. */
int32_t rslx_sym_augment(const rslx_sym* sym, const float* obs_in, const float* act_in, int32_t B,
                         int32_t D, int32_t A, float* obs_out, float* act_out, void* stream);

/* ---- RND intrinsic reward (paper Sec. 2.2) --------------------------------------------- */

/* x = obs[:, subset]; r_raw_n = sum_k (predictor(x_n) - target(x_n))_k^2.  If update_stats,
 * running = {mean, var, count} (device float[3], population variance) is merged with the N new
 * values (Chan et al. pairwise update) before use.  r_int = r_raw / sqrt(var + 1e-8) is written
 * to r_int_out [N]; if rewards_inout != NULL, rewards_inout[n] += weight * r_int[n] (its own buffer). */
size_t rslx_rnd_workspace_bytes(const rslx_mlp* target, int32_t N);
int32_t rslx_rnd(const rslx_mlp* target, const rslx_mlp* predictor, const float* obs, int32_t N,
                 int32_t D, const int32_t* subset_idx_or_null, int32_t n_subset, float* running,
                 float weight, int32_t update_stats, float* r_int_out, float* rewards_inout_or_null,
                 void* ws, size_t ws_bytes, void* stream);

/* ---- linear attention with a decay for each head (a memory over whole sequences) ------------- */

/* Types of the activations of the operators from here on; parameters, states and statistics are fp32, and so is
 * arithmetic, with one exception: over whole sequences in 16 bits, outputs and gradients are made of states and weighted
 * scores with 16 significant bits (errors up to 2^-17 of a term in bf16, 2^-15 in fp16, beside the result's own rounding
 * of 2^-8 and 2^-11).  What is added to a state has fp32's. */
#define RSLX_F32 0
#define RSLX_BF16 1
#define RSLX_F16 2

/* A matrix [T, N, H, width] (steps, sequences or environments, heads): element (t, n, h, i) lies at
 * data + t*step + n*seq + h*head + i, strides in elements.  Inputs may have any strides, zero among
 * them (a row shared by heads or sequences; its gradient then comes per head, for the caller to add
 * up); rows of outputs must not overlap.  `data` is aligned to its type; where all of a call's matrices
 * start at multiples of 16 bytes, with widths and strides of whole 16 bytes, they are moved 16 bytes
 * at a time. */
typedef struct rslx_seq_view {
  void* data;
  int64_t step, seq, head;
} rslx_seq_view;

/* With l_h = exp(log_decay[h]), per sequence n and head h, state S [Dk, Dv]:
 *   S_t = l keep_{t-1} S_{t-1} + k_t v_t^T,   o_t = scale S_t^T q_t,   S_{-1} = s0 (0 if NULL), keep_{-1} = 1
 * keep_t = 0 where dones[t, n] is set: the state is zeroed after every step that ends an episode, as in
 * rslx_ppo_update_recurrent.  s_last = keep_{T-1} S_{T-1} is what the next call starts from: a sequence
 * in two calls gives what one call gives, up to rounding.  With lengths, sequence n has the first
 * lengths[n] steps only (values outside 0..T count as 0 or T): behind them outputs and gradients are
 * zero, inputs are not looked at, and s_last is the state behind the last step that exists (s0 if none does).
 * log_decay is at most 0 in earnest (-inf: no memory); it is a constant of the layer and has no gradient.
 * What is not finite stays where the recurrence above puts it: a step's values reach no earlier step
 * and no other episode. */
#define RSLX_ATTN_MAX_DIM 128
#define RSLX_ATTN_MAX_STEPS 2147483583 /* 2^31 - 65 */
typedef struct rslx_linear_attn {
  int32_t dtype;                 /* RSLX_F32, RSLX_BF16, RSLX_F16: q, k, v, o and their gradients */
  int32_t T, N, H;               /* T: 0..RSLX_ATTN_MAX_STEPS; N * H: 0..2^24 */
  int32_t Dk, Dv;                /* 1..RSLX_ATTN_MAX_DIM */
  float scale;
  const float* log_decay;        /* device [H] */
  const uint8_t* dones;          /* device [T, N] or NULL */
  const int32_t* lengths;        /* device [N] or NULL */
} rslx_linear_attn;

/* The whole sequence.  q, k: width Dk; v, o: width Dv; s0, s_last: device [N, H, Dk, Dv] or NULL (s_last may be
 * the buffer of s0).  Outputs must not overlap inputs or each other otherwise.  A few long sequences are walked in
 * pieces side by side, which takes workspace; otherwise ws may be NULL. */
size_t rslx_linear_attention_workspace_bytes(const rslx_linear_attn* a);
int32_t rslx_linear_attention(const rslx_linear_attn* a, const rslx_seq_view* q, const rslx_seq_view* k,
                              const rslx_seq_view* v, const float* s0_or_null, const rslx_seq_view* o,
                              float* s_last_or_null, void* ws, size_t ws_bytes, void* stream);

/* Gradients of a loss L through the call above, from those of its outputs, d_o and ds_last (NULL = 0):
 *   dS_t = scale q_t d_o_t^T + keep_t (t + 1 < T ? l dS_{t+1} : ds_last)
 *   dq_t = scale S_t d_o_t,   dk_t = dS_t v_t,   dv_t = dS_t^T k_t,   ds0 = l dS_0 (ds_last where there is no step)
 * Nothing is kept from the forward call: states are walked again.  No output (ds0 may be NULL) may
 * overlap an input or another output. */
size_t rslx_linear_attention_backward_workspace_bytes(const rslx_linear_attn* a);
int32_t rslx_linear_attention_backward(const rslx_linear_attn* a, const rslx_seq_view* q, const rslx_seq_view* k,
                                       const rslx_seq_view* v, const float* s0_or_null, const rslx_seq_view* d_o,
                                       const float* ds_last_or_null, const rslx_seq_view* dq, const rslx_seq_view* dk,
                                       const rslx_seq_view* dv, float* ds0_or_null, void* ws, size_t ws_bytes,
                                       void* stream);

/* One step of every environment, while acting (a->T = 1, dones and lengths NULL; the views' step is not used):
 *   s_out = (reset[n] ? 0 : l s_in) + k v^T,   o = scale s_out^T q
 * reset_or_null (device uint8 [N]) carries the previous step's episode-end flags, as in rslx_act_recurrent;
 * s_in (NULL = 0) and s_out may be one buffer; o may be q, k or v, each row in place of the same head's; nothing else
 * that is written may overlap what is read or written. */
int32_t rslx_linear_attention_step(const rslx_linear_attn* a, const rslx_seq_view* q, const rslx_seq_view* k,
                                   const rslx_seq_view* v, const uint8_t* reset_or_null, const float* s_in_or_null,
                                   float* s_out, const rslx_seq_view* o, void* stream);

/* ---- layer norm ------------------------------------------------------------------------ */

/* Per row:  m = mean x,  r = 1 / sqrt(mean (x - m)^2 + eps),  y = (x - m) r weight + bias.
 * x, y: [rows, cols] of `dtype`, rows ldx and ldy elements apart; y may be x with the same distance, and must not overlap
 * it otherwise (the columns beside x in one buffer do not).  weight, bias: device fp32 [cols], NULL = 1 and 0.
 * mean, rstd: device fp32 [rows] or NULL; the backward pass reads them. */
#define RSLX_NORM_MAX_COLS 16384
int32_t rslx_layer_norm(int32_t dtype, const void* x, int64_t ldx, int64_t rows, int32_t cols,
                        const float* weight_or_null, const float* bias_or_null, float eps, void* y, int64_t ldy,
                        float* mean_or_null, float* rstd_or_null, void* stream);

/* With g = dy weight and h = (x - mean) rstd:  dx = rstd (g - mean(g) - h mean(g h)) per row,
 * dweight = sum over rows of dy h, dbias = sum over rows of dy (device fp32 [cols]; zero where there are no rows).
 * Any of dx, dweight, dbias may be NULL; dx may be dy or x, with the same distance, and must not overlap them otherwise.
 * The sums are taken in a fixed order: the same inputs give the same bits.  Without dweight and dbias no workspace is
 * needed. */
size_t rslx_layer_norm_backward_workspace_bytes(int64_t rows, int32_t cols);
int32_t rslx_layer_norm_backward(int32_t dtype, const void* dy, int64_t lddy, const void* x, int64_t ldx,
                                 int64_t rows, int32_t cols, const float* weight_or_null, const float* mean,
                                 const float* rstd, void* dx_or_null, int64_t lddx, float* dweight_or_null,
                                 float* dbias_or_null, void* ws, size_t ws_bytes, void* stream);

/* ---- gated linear recurrence (a memory of one state per channel) ------------------------ */

/* Per sequence n and channel d, with f = sigmoid(g):
 *   h_t = f_t keep_{t-1} h_{t-1} + (1 - f_t) x_t,   h_{-1} = s0 (0 if NULL), keep_{-1} = 1
 * keep_t = 0 where dones[t, n] is set, s_last = keep_{T-1} h_{T-1}, and lengths: all as in linear attention above.  1 - f is
 * sigmoid(-g), so gates next to one keep their digits; g = +inf holds the state, g below -87 counts as -87 (f = 1.6e-38).
 * x, g and h (and their gradients) are matrices [T, N, D]: views whose `head` is not used, under the conditions above.
 * A step's values reach no earlier step and no other episode, whatever they are; an infinite state may be a NaN some
 * steps later, where the product of the gates between is zero in fp32. */
#define RSLX_REC_MAX_TILES 16777215 /* 2^24 - 1 */
typedef struct rslx_gated_rec {
  int32_t dtype;                 /* RSLX_F32, RSLX_BF16, RSLX_F16: x, g, h and their gradients; states are fp32 */
  int32_t T, N, D;               /* T: 0..RSLX_ATTN_MAX_STEPS; N: 0 or more; D: 1 or more; N ceil(D / 64), in whole calls times the pieces
                                    of 64 steps or more that long sequences are cut into: to RSLX_REC_MAX_TILES (cut ones
                                    have less than 2^28 channels N * D, D rounded up to four) */
  const uint8_t* dones;          /* device [T, N] or NULL */
  const int32_t* lengths;        /* device [N] or NULL */
} rslx_gated_rec;

/* The whole sequence.  s0, s_last: device [N, D] or NULL (s_last may be the buffer of s0).  Outputs must not overlap inputs
 * or each other otherwise. */
size_t rslx_gated_recurrence_workspace_bytes(const rslx_gated_rec* a);
int32_t rslx_gated_recurrence(const rslx_gated_rec* a, const rslx_seq_view* x, const rslx_seq_view* g, const float* s0_or_null,
                              const rslx_seq_view* h, float* s_last_or_null, void* ws, size_t ws_bytes, void* stream);

/* Gradients of a loss through the call above, from those of its outputs, dh and ds_last (NULL = 0):
 *   d_t = dh_t + keep_t (t + 1 < T ? f_{t+1} d_{t+1} : ds_last)
 *   dx_t = (1 - f_t) d_t,   dg_t = f_t (1 - f_t) d_t (keep_{t-1} h_{t-1} - x_t),   ds0 = f_0 d_0 (ds_last where there is no step)
 * Nothing is kept from the forward call: states are walked again, in fp32.  No output (ds0 may be NULL) may overlap an
 * input or another output. */
size_t rslx_gated_recurrence_backward_workspace_bytes(const rslx_gated_rec* a);
int32_t rslx_gated_recurrence_backward(const rslx_gated_rec* a, const rslx_seq_view* x, const rslx_seq_view* g,
                                       const float* s0_or_null, const rslx_seq_view* dh, const float* ds_last_or_null,
                                       const rslx_seq_view* dx, const rslx_seq_view* dg, float* ds0_or_null, void* ws,
                                       size_t ws_bytes, void* stream);

/* One step of every environment, while acting (a->T = 1, dones and lengths NULL; the views' step is not used):
 *   s_out = f (reset[n] ? 0 : s_in) + (1 - f) x,   h = s_out in its type
 * reset_or_null, s_in and s_out as in rslx_linear_attention_step; h may be x or g, each row in place of the same sequence's;
 * nothing else that is written may overlap what is read or written. */
int32_t rslx_gated_recurrence_step(const rslx_gated_rec* a, const rslx_seq_view* x, const rslx_seq_view* g,
                                   const uint8_t* reset_or_null, const float* s_in_or_null, float* s_out,
                                   const rslx_seq_view* h, void* stream);

/* ---- root-mean-square norm with the residual's addition --------------------------------- */

/* Per row:  z = x + residual (x alone where that is NULL),  r = 1 / sqrt(mean z^2 + eps),  y = z r weight.
 * x, residual, total, y: [rows, cols] of `dtype`, rows ldx, ldr, ldt and ldy elements apart.  total (or NULL) receives z, rounded
 * to the type: the stream that goes on behind the block, and what the backward pass reads; y is made of z before that
 * rounding.  weight: device fp32 [cols] or NULL = 1; rstd: device fp32 [rows] or NULL receives r.  total and y may each
 * be x or residual, with the same distance, and overlap nothing otherwise.
 * Squares are fp32: a row whose sum of squares passes 3e38 gives zeros (NaN where a value is not finite). */
int32_t rslx_rms_norm(int32_t dtype, const void* x, int64_t ldx, const void* residual_or_null, int64_t ldr, int64_t rows,
                      int32_t cols, const float* weight_or_null, float eps, void* total_or_null, int64_t ldt, void* y,
                      int64_t ldy, float* rstd_or_null, void* stream);

/* The same with y in a byte a value: e4m3 (4 bits of exponent, 3 of fraction, largest value 448; OCP's, without infinities),
 * y = scales[row] * y8, scales[row] = max |y| / 448 of the row (at least 2^-126: with eps > 0 a row of zeros has zeros).  y8 is rounded to nearest,
 * ties to even; it overlaps nothing.  A row that holds a NaN is NaN, its scale too. */
int32_t rslx_rms_norm_e4m3(int32_t dtype, const void* x, int64_t ldx, const void* residual_or_null, int64_t ldr, int64_t rows,
                           int32_t cols, const float* weight_or_null, float eps, void* total_or_null, int64_t ldt, void* y8,
                           int64_t ldy, float* scales, float* rstd_or_null, void* stream);

/* With h = total rstd and k = dy weight:  dx = dtotal + rstd (k - h mean(k h)) per row (dtotal, the gradient of the stream behind
 * the block: NULL = 0), dweight = sum over rows of dy h (device fp32 [cols]; zero where there are no rows).  dx is the gradient of x and
 * of residual.  Either of dx, dweight may be NULL; dx may be dy, total or dtotal, with the same distance, and must not overlap them otherwise.
 * Sums are taken in a fixed order.  Without dweight no workspace is needed. */
size_t rslx_rms_norm_backward_workspace_bytes(int64_t rows, int32_t cols);
int32_t rslx_rms_norm_backward(int32_t dtype, const void* dy, int64_t lddy, const void* total, int64_t ldt, int64_t rows,
                               int32_t cols, const float* weight_or_null, const float* rstd, const void* dtotal_or_null,
                               int64_t lddt, void* dx_or_null, int64_t lddx, float* dweight_or_null, void* ws,
                               size_t ws_bytes, void* stream);

/* ---- Muon: momentum whose update is made orthogonal ------------------------------------- */

/* For every matrix [rows, cols] (dense, row-major, fp32; a layer's weights inside a flat parameter buffer among them):
 *   m_out = momentum m_in + grad,   u = nesterov ? grad + momentum m_out : m_out
 *   X = u / |u|_F,   `steps` times  X <- a X + (b A + c A^2) X  with A = X X^T      (a, b, c = 3.4445, -4.7750, 2.0315)
 *   w_out = (1 - lr weight_decay) w_in - lr scale X
 * (Jordan et al. 2024: quintic Newton-Schulz steps, which bring every singular value near one).  Each product is fp32's in effect:
 * operands are held as pairs of fp16 values (22 significant bits), sums in fp32.  u = 0 leaves X = 0; a matrix whose u
 * holds a value that is not finite gets NaN, the others of the call nothing of it.  Tiles are chosen for
 * the call: a matrix's rounding may depend on the sizes of those beside it, the same call gives the same bits.
 * w_in NULL: 0; m_in NULL: 0; m_out NULL: not kept (w_in = m_in = m_out = NULL, lr = -1: X itself).  w_out may be w_in and m_out
 * may be m_in; nothing else that is written may overlap what is read or written.  Pointers are aligned to 4 bytes; the descriptions are host memory,
 * read before the call returns (a captured call keeps them, lr among them). */
#define RSLX_MUON_MAX_MATRICES 32
#define RSLX_MUON_MAX_DIM 65536
#define RSLX_MUON_MAX_STEPS 32
typedef struct rslx_muon_matrix {
  const float* w_in;
  float* w_out;
  const float* grad;
  const float* m_in;
  float* m_out;
  int32_t rows, cols;            /* 1..RSLX_MUON_MAX_DIM */
  float scale;
} rslx_muon_matrix;
typedef struct rslx_muon_cfg {
  float lr, momentum, weight_decay;
  int32_t nesterov, steps;       /* steps: 1..RSLX_MUON_MAX_STEPS */
} rslx_muon_cfg;
size_t rslx_muon_step_workspace_bytes(const rslx_muon_matrix* matrices, int32_t count, const rslx_muon_cfg* cfg);
int32_t rslx_muon_step(const rslx_muon_matrix* matrices, int32_t count, const rslx_muon_cfg* cfg, void* ws, size_t ws_bytes,
                       void* stream);

#ifdef __cplusplus
}
#endif
#endif /* RSLX_H */
