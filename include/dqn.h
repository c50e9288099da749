/*
 * libdqn: the minibatch training step of deep Q-learning (DQN / Double DQN /
 * dueling head / proportional prioritized replay) for one AMD MI355X (gfx950),
 * as described in arxiv 1804.05834 (Sections 2.2-2.5, Section 3, Table 1).
 *
 * C ABI.  Every function returns an int32 status (0 = ok, negative = error) and
 * never throws.  On error no output buffer has been written by that call and
 * dqn_last_error() describes the cause.
 *
 * Pointers: unless a parameter says "host", every data pointer is a HIP DEVICE
 * pointer, 256-byte aligned, owned by the caller for the lifetime of the
 * context.  `stream` is a hipStream_t passed as void* (NULL = the null stream).
 * Calls enqueue work on that stream and return without synchronising; scalar
 * results land in caller-supplied device memory.  A context must not be used
 * from two streams at once.
 *
 * Actions are 0-based int32 in [0, num_actions) (the paper's set {1..K},
 * Section 2.1).  States are uint8 [4][84][84] stacks of grey frames
 * (Section 3); the network sees x = uint8 / 255.
 *
 * Canonical parameter blob (what dqn_get_params / dqn_set_params exchange;
 * fp32, concatenated, row-major), following the layer list of Section 3:
 *   conv1.W[32][4][8][8] conv1.b[32]  conv2.W[64][32][4][4] conv2.b[64]
 *   conv3.W[64][64][3][3] conv3.b[64] fc1.W[512][3136] fc1.b[512]
 *     (fc1 input index = c*49 + h*7 + w)
 *   plain head  : out.W[K][512] out.b[K]
 *   dueling head: V.W[1][512] V.b[1] A.W[K][512] A.b[K]          (Eq.13)
 * The library keeps its parameter buffers in an internal (channel-last)
 * permutation of this blob; only get/set translate.  With precision 1 the
 * shadow buffer holds copies of both networks' weights that the library's own
 * calls keep up to date: a program that writes the parameter buffers itself (a
 * copy of all of a context's buffers, say) writes that one along with them.
 */
#ifndef DQN_H_
#define DQN_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
    DQN_OK = 0,
    DQN_ERR_INVALID_ARG = -1, /* NULL / misaligned pointer, size out of range      */
    DQN_ERR_OOM = -2,         /* host allocation failed                            */
    DQN_ERR_HIP = -3,         /* a HIP runtime call failed                         */
    DQN_ERR_STATE = -4,       /* e.g. sampling before any priority was stored      */
    DQN_ERR_UNSUPPORTED = -5  /* valid request this build does not implement       */
};

typedef struct dqn_ctx dqn_ctx;

/* All fields are explicit; there are no hidden defaults (Table 1 values in
 * brackets are what the paper's benchmark uses). */
typedef struct {
    int32_t num_actions;   /* K, 1..64                                              */
    int32_t dueling;       /* 0 plain output layer / 1 dueling head (Eq.13)         */
    int32_t double_q;      /* 0 target of Eq.8 / 1 Double-DQN target of Eq.9        */
    int32_t precision;     /* 0 fp32 / 1 bf16 compute with fp32 master + accumulate */
    int32_t loss_kind;     /* 0 = 0.5*td^2 (Eq.7) / 1 = Huber                       */
    float huber_delta;     /* Huber threshold [1]                                   */
    float gamma;           /* discount [0.99]                                       */
    float lr;              /* RMSProp step size                                     */
    float rms_decay;       /* RMSProp rho                                           */
    float rms_eps;         /* RMSProp epsilon (inside the square root)              */
    int32_t rms_centered;  /* 1 = subtract the squared running mean of g            */
    int32_t max_batch;     /* largest B of dqn_train_step, 1..1024                  */
    int32_t max_act_batch; /* largest E of dqn_act, 1..8192                         */
    int32_t per_stratified;/* 0 independent draws (Alg.2) / 1 one draw per stratum  */
    int64_t replay_capacity; /* N frames/transitions in the ring [1,000,000]; 0 = none */
    float per_alpha;       /* prioritisation exponent of Eq.10 [0.6]                */
    float per_eps;         /* the small constant of Eq.11                           */
    uint64_t seed;         /* online-network initialisation stream                  */
    uint64_t target_seed;  /* target-network initialisation stream                  */
} dqn_config;

/* Byte sizes of the caller-owned device buffers for a configuration.  A size
 * of 0 means the buffer is not used and its pointer may be NULL. */
typedef struct {
    size_t params;        /* ONE network's fp32 parameters (online, target: each)  */
    size_t opt_state;     /* RMSProp accumulators                                  */
    size_t shadow_bf16;   /* bf16 copies of both networks' weights (precision 1)   */
    size_t grads;         /* fp32 gradient of the last step                        */
    size_t replay_frames; /* uint8 [capacity][84][84]                              */
    size_t replay_meta;   /* action / reward / terminal flag per slot              */
    size_t tree;          /* sum-tree: float [2L] heap + 64 floats of state        */
    size_t workspace;     /* activations, partial sums, minibatch staging: nothing
                             in it has to survive between calls, except for
                             dqn_get_activations                                   */
    int64_t param_count;  /* number of fp32 parameters of one network              */
    int64_t tree_leaves;  /* L = capacity rounded up to a power of two             */
} dqn_sizes;

typedef struct {
    void *online, *target, *opt_state, *shadow_bf16, *grads;
    void *replay_frames, *replay_meta, *tree, *workspace;
} dqn_buffers;

/* An explicit minibatch (Alg.1 "sample random minibatch"): B transitions. */
typedef struct {
    const uint8_t *s;      /* [B][4][84][84]                                         */
    const uint8_t *s_next; /* [B][4][84][84]                                         */
    const int32_t *a;      /* [B]                                                    */
    const float *r;        /* [B]                                                    */
    const uint8_t *done;   /* [B] 1 = s_next is terminal                             */
    const float *w;        /* [B] importance weights, or NULL = all 1                */
} dqn_batch;

/* Optional per-step outputs; any member may be NULL. */
typedef struct {
    float *loss;          /* [1]    (1/B) sum_j w_j l(td_j)                          */
    float *q_s;           /* [B][K] Q(s_j, . ; theta)                                */
    float *q_next_online; /* [B][K] Q(s'_j, . ; theta)                               */
    float *q_next_target; /* [B][K] Q(s'_j, . ; theta^-)                             */
    float *y;             /* [B]    targets (Eq.8 / Eq.9, y = r for terminal s')     */
    float *td;            /* [B]    y_j - Q(s_j, a_j; theta)                         */
    int32_t *a_star;      /* [B]    the action the target bootstraps from            */
    int32_t *idx;         /* [B]    sampled replay slots (replay mode only)          */
    float *is_w;          /* [B]    importance weights used                          */
    float *td_abs_mean;   /* [1]    (1/B) sum_j |td_j| (rows with a finite error)    */
    float *q_max_mean;    /* [1]    (1/B) sum_j max_a Q(s_j, a; theta)               */
} dqn_step_out;

/* Sizes of every buffer dqn_init needs.  `cfg`, `out`: host pointers. */
int32_t dqn_query_sizes(const dqn_config *cfg, dqn_sizes *out);

/* Creates a context over caller-owned device buffers (sizes from
 * dqn_query_sizes), initialises the online and target parameters on the host
 * (Alg.1 "random weights": uniform in +-sqrt(6/fan_in) from the counter-based
 * draws of cfg->seed / cfg->target_seed, biases 0), zeroes the optimizer state
 * and empties the replay.  `out`, `cfg`, `bufs`: host pointers.  The context
 * owns only host-side bookkeeping; free it with dqn_destroy. */
int32_t dqn_init(dqn_ctx **out, const dqn_config *cfg, const dqn_buffers *bufs, void *stream);

/* Epsilon-greedy action selection for E observations (Alg.1, the two action
 * lines; Eq.3): with u = draw(draw_seed, 2e), if u < epsilon the action is
 * floor(draw(draw_seed, 2e+1) * K), else argmax_a Q(obs_e, a; theta) with the
 * lowest index winning ties.  obs: [E][4][84][84]; actions: [E];
 * q_opt: [E][K] or NULL.  1 <= E <= max_act_batch. */
int32_t dqn_act(dqn_ctx *ctx, const uint8_t *obs, int32_t E, float epsilon, uint64_t draw_seed,
                int32_t *actions, float *q_opt, void *stream);

/* One minibatch training step (Alg.1 target + gradient-step lines; Alg.2
 * inner loop and weight update; Eq.7-9, Eq.13; RMSProp of Table 1):
 * forward of the online net on s and s', of the target net on s', target y,
 * TD error, loss L = (1/B) sum w l(td), exact gradient, RMSProp update of the
 * online parameters.  `batch` (host pointer to a struct of device pointers)
 * selects the explicit mode.  batch == NULL selects the replay mode: B slots
 * are drawn as by per_sample(beta, draw_seed), their frame stacks gathered
 * from the ring, and after the update their priorities are set from |td| as by
 * per_update.  `out` (host pointer, may be NULL) names optional outputs.
 * 1 <= B <= max_batch.
 * A row whose action lies outside [0, num_actions) is not trained on: it enters
 * the loss and the gradient with weight 0, its td is reported as NaN, and in
 * replay mode its priority is left alone.  In replay mode, if the tree holds no
 * mass at all (every stored transition has priority zero: nothing can be drawn),
 * every importance weight is 0, the parameters do not move and no priority is
 * written. */
int32_t dqn_train_step(dqn_ctx *ctx, int32_t B, const dqn_batch *batch, float beta,
                       uint64_t draw_seed, const dqn_step_out *out, void *stream);

/* Proportional prioritized sampling (Eq.10, Eq.12; Alg.2 sampling and
 * weighting lines).  Draw j uses u_j = draw(draw_seed, j); independent mode
 * descends the sum-tree with mass fp32(u_j * total), stratified mode with
 * fp32((j + u_j) * fp32(total / B)).  idx[j] is the leaf reached (clamped to
 * the stored size); is_w[j] = (N * P(j))^-beta / max_j(...), N = stored
 * transitions.  A slot whose leaf is 0 has probability zero and is never
 * returned, also where the fp32 sums of the tree would let the textbook
 * descent overshoot into it: the walk turns left whenever the right child is 0.
 * Returns DQN_ERR_STATE if nothing is stored (the call cannot see on the host
 * whether every stored leaf is 0: then idx = 0 and is_w = 0 are written).
 * 1 <= B <= 1024. */
int32_t per_sample(dqn_ctx *ctx, int32_t B, float beta, uint64_t draw_seed, int32_t *idx,
                   float *is_w, void *stream);

/* Priority update (Eq.11; Alg.2 priority line): leaf[idx_j] = fp32((|td_j| +
 * per_eps)^alpha) for j = 0..n-1 with the last occurrence of a repeated index
 * winning, every ancestor recomputed as fp32(left + right), and the running
 * maximum priority raised to max_j(|td_j| + per_eps).  idx values must lie in
 * [0, stored size); out-of-range entries and entries whose td is not finite are
 * skipped (their leaves keep their values).  1 <= n <= 1024. */
int32_t per_update(dqn_ctx *ctx, const int32_t *idx, const float *td_abs, int32_t n, void *stream);

/* dqn_act for callers that cannot allocate device memory or pass a workspace of
 * their own sizing: code under HIP graph capture, tight serving loops, harnesses
 * that forbid hipMalloc.  Same arguments, same kernels and bit-identical results
 * as dqn_act, but the activations and partial sums go to a static device array
 * inside the library (4 MiB per GPU, held until the process ends) instead of
 * the context's workspace, so E is limited to DQN_ACT_STATIC_MAX; a larger E
 * is DQN_ERR_INVALID_ARG.  The call allocates nothing (no hipMalloc, no
 * hipFree, no events); the array's device address is looked up once per device,
 * at dqn_init or on the first call there.  Nothing in the array has to start
 * at zero: every word read has been written earlier in the same call.  All
 * calls on one GPU share the array: calls that overlap on one GPU (two
 * streams, two contexts, two threads) race and give undefined results. */
#define DQN_ACT_STATIC_MAX 32
int32_t dqn_act_static(dqn_ctx *ctx, const uint8_t *obs, int32_t E, float epsilon, uint64_t draw_seed,
                       int32_t *actions, float *q_opt, void *stream);

/* ---- auxiliary calls needed to drive and to check the five above ---- */

/* Bulk (re)build of the sum-tree from n raw priorities p_i > 0 for slots
 * 0..n-1 (leaf = fp32(p^alpha), slots >= n get 0) and sets the stored size to
 * n.  n <= replay_capacity. */
int32_t per_fill(dqn_ctx *ctx, const float *priorities, int64_t n, void *stream);

/* Stores n consecutive single frames and their transition data into ring slots
 * slot0 .. slot0+n-1 (mod capacity) (Alg.1 "store transition").  Transition i
 * is read back as s = frames (i-3..i), s' = frames (i-2..i+1), slots taken
 * modulo the capacity.  Priorities are not touched.  frames: [n][84][84]. */
int32_t dqn_replay_write(dqn_ctx *ctx, int64_t slot0, int64_t n, const uint8_t *frames,
                         const int32_t *a, const float *r, const uint8_t *done, void *stream);

/* Store path (Alg.1 "store transition"; Alg.2 "store transition with maximal
 * priority").  Appends n consecutive time steps of ONE environment stream at the
 * write cursor (slot = stream position mod capacity): frame x_t with the action
 * a_t taken on it, the reward r_t and the terminal flag done_t.  Transition i is
 * read back as s = frames (i-3..i), s' = frames (i-2..i+1), so a time step
 * completes the transition before it.  Each completed transition enters the
 * sum-tree with the maximal priority seen so far (1 before the first update),
 * leaf = fp32(max_p^alpha); a transition whose state stack would reach back
 * before the start of the stream or across an episode end (done at one of the
 * three slots before it) gets leaf 0 and is never sampled, and so do the last
 * written slot (its transition is not complete yet) and the three slots after
 * it, whose windows mix the newest frames with the oldest.
 * The stored count (N of Eq.12) becomes min(time steps stored, capacity).
 * frames: [n][84][84] device, 16-byte aligned; a, r, done: [n] device, not NULL.
 * 1 <= n <= min(1020, capacity - 8); the ring must have at least 16 slots.
 * per_fill sets the cursor to n mod capacity; dqn_replay_write does not move it. */
int32_t dqn_replay_store(dqn_ctx *ctx, int64_t n, const uint8_t *frames, const int32_t *a,
                         const float *r, const uint8_t *done, void *stream);

/* Store path for many environment streams (Alg.1 "store transition" with one
 * emulator per stream, as batched acting needs it).  The ring becomes E sub-rings
 * of C = capacity / E slots (integer division; stream e owns slots [eC, (e+1)C));
 * the first call on an empty context fixes E.  Every call appends ONE time step to
 * every stream, at local slot (calls so far) mod C: frame x_t of stream e with the
 * action taken on it, reward and terminal flag.  Each stream follows the rules of
 * dqn_replay_store within its own sub-ring: the transition before the new step
 * enters with the maximal priority unless its stack would reach before the
 * stream's start or across an episode end; the slot just written and the three
 * after it get leaf 0.  A transition's frames are read back modulo its sub-ring, so
 * no stack ever mixes two streams.  The stored count (N of Eq.12) is
 * E * min(calls, C).  frames: [E][84][84] device, 16-byte aligned; a, r, done: [E].
 * 1 <= E <= capacity / 16.  per_fill returns the context to one stream. */
int32_t dqn_replay_store_envs(dqn_ctx *ctx, int32_t E, const uint8_t *frames, const int32_t *a,
                              const float *r, const uint8_t *done, void *stream);

/* Host-side view of the store path: next slot, stored count, time steps so far.
 * Any pointer may be NULL. */
int32_t dqn_replay_state(const dqn_ctx *ctx, int64_t *cursor, int64_t *stored, int64_t *steps);

/* Frame preprocessing (Sec.3: raw palette frame -> grey-scale -> linearly
 * interpolated to 84 x 84), batched.  raw: [n][height][width] bytes (device);
 * grey_lut: 256 floats (device) mapping a byte to its grey level in 0..255, or
 * NULL when the bytes already are grey levels; frames: [n][84][84] (device).
 * Output pixel (i,j) samples the source at (i+1/2)*height/84 - 1/2,
 * (j+1/2)*width/84 - 1/2 (clamped), blends the four neighbours bilinearly in
 * fp32 and rounds to the nearest integer (ties to even).  Needs no context.
 * 1 <= n <= 65535. */
int32_t dqn_preprocess(const uint8_t *raw, int64_t n, int32_t height, int32_t width,
                       const float *grey_lut, uint8_t *frames, void *stream);

/* Schedules of Table 1 as functions of the environment step t = 1, 2, ... (host
 * only, no device work): a value "a -> b (1 -> T steps)" is a at t = 1, b at
 * t >= T, linear in between; train is set when t is past learning_start and
 * t = 0 mod update_period (Alg.2 "if t = 0 mod K"); sync_target when
 * t = 0 mod target_period (Alg.2 last line).  dqn_schedule_default fills in
 * Table 1: learning start 50,000, update period 4, target period 30,000,
 * epsilon 1.0 -> 0.1 over 5,000,000 steps, beta 0.4 -> 1.0 over 100,000,000. */
typedef struct {
    int64_t learning_start, update_period, target_period, eps_steps, beta_steps;
    float eps_start, eps_end, beta_start, beta_end;
} dqn_schedule;
typedef struct {
    float epsilon, beta;
    int32_t train, sync_target;
} dqn_schedule_point;
int32_t dqn_schedule_default(dqn_schedule *s);
int32_t dqn_schedule_at(const dqn_schedule *s, int64_t step, dqn_schedule_point *out);

/* Materialises the stacks of n slots: s, s_next [n][4][84][84], a, r, done [n]
 * (any output may be NULL).  1 <= n <= max_batch. */
int32_t dqn_replay_gather(dqn_ctx *ctx, const int32_t *idx, int32_t n, uint8_t *s, uint8_t *s_next,
                          int32_t *a, float *r, uint8_t *done, void *stream);

/* Diagnostics: the stored outputs (after ReLU) of layer 1-3 (the convolutions) or
 * 4 (the 512-unit hidden layer) of Section 3's network for the first n rows of
 * the online pass on s of the last dqn_train_step, as fp32 in canonical order:
 * dst [n][32][20][20], [n][64][9][9], [n][64][7][7] or [n][512].  These are
 * the numbers the backward pass takes its ReLU decisions on.  1 <= n <= max_batch. */
int32_t dqn_get_activations(dqn_ctx *ctx, int32_t layer, int32_t n, float *dst, void *stream);

/* Host-only self-check, no device work: searches, for a run of ns samples per
 * workgroup (1..32), every state that the waves of the fused conv1 to conv3
 * forward launch of the bf16 path can reach in any order of their steps, where
 * waves hand conv1's and conv2's output of a sample (Section 3, first and second
 * layer) to the next layer's waves through rings of images in LDS, by counts, using
 * the very functions the kernel's loops call.  A step is to begin or to end the
 * storing of a share of a sample or the reading of a sample.  Returns 0 if every
 * sample is complete before it is read, read exactly once, and never overwritten while
 * unread, and in no state but the last every wave waits; a positive code otherwise. */
int32_t dqn_selftest_fused_conv_schedule(int32_t ns);

/* theta^- <- theta (Alg.2 "copy weights into target network"). */
int32_t dqn_sync_target(dqn_ctx *ctx, void *stream);

/* which: 0 online, 1 target, 2 gradient of the last step, 3 RMSProp v,
 * 4 RMSProp m (centered only).  dst / src: device, canonical blob. */
int32_t dqn_get_params(dqn_ctx *ctx, int32_t which, float *dst, void *stream);
int32_t dqn_set_params(dqn_ctx *ctx, int32_t which, const float *src, void *stream);

/* Per-kernel timing: after dqn_profile_begin every kernel launched through
 * this context is bracketed by HIP events on its stream; dqn_profile_end
 * synchronises, disables timing, and copies up to `cap` records (name, launch
 * count, total milliseconds) to host arrays.  Returns the number of distinct
 * kernels seen (may exceed cap) or a negative status.  names: host array of
 * cap pointers to static strings. */
int32_t dqn_profile_begin(dqn_ctx *ctx);
int32_t dqn_profile_end(dqn_ctx *ctx, int32_t cap, const char **names, int64_t *counts,
                        double *total_ms);

/* Last error message of this context (host string, valid until the next call
 * on the context); for a NULL ctx, the last error of a failed dqn_init /
 * dqn_query_sizes on this thread. */
const char *dqn_last_error(const dqn_ctx *ctx);

int32_t dqn_destroy(dqn_ctx *ctx);

/* ---- operators of a recurrent Q-network ----
 *
 * What a network with a memory of its episode needs next to the calls above:
 * blocks of a normalised residual stream, projections and a gated linear
 * recurrence over time, trained over sequences with AdamW and stepped once per
 * environment step while acting.  None needs a context.  Errors are reported by
 * dqn_last_error(NULL).  Data pointers are device pointers aligned to their
 * elements (weaker than the 256 bytes above); strides count elements, rows are
 * contiguous.  A stride may be larger than the row, so that a tensor can be a
 * part of a wider one.  Inputs and outputs of a call must not overlap except
 * where it says so.  Structs of arguments are host pointers, read during the
 * call.  Nothing is allocated.  Every call can be recorded into a HIP graph but
 * dqn_adamw_init and dqn_muon_init, which wait for their stream; a recorded dqn_adamw_step repeats its
 * step number, rate and seed, and so its random bits, with every replay, a recorded dqn_muon_step
 * its rate.  A call's workspace is its own until it has run: graphs that may run at the same
 * time, or calls on several streams, take one each. */

/* dtype of activations and their gradients: fp32, or bf16 with sums, states and
 * statistics in fp32. */
enum { DQN_F32 = 0, DQN_BF16 = 1 };

/* Gated linear recurrence over time, per channel, with a_t = sigmoid(f_t):
 *   h_t = a_t k_t h_{t-1} + (1 - a_t) x_t,   t = 0 .. T-1,   h_{-1} = h0
 * k_t = 0 where reset_t != 0 (step t is the first of an episode: whatever the
 * state was, a NaN too, is forgotten; until then one that is not finite stays not
 * finite, infinite or NaN), else 1.  The state is fp32.  T = 1 is the
 * step of an acting agent; h_last may be h0 then, and for any T. */
typedef struct {
    int32_t dtype;                      /* DQN_F32 / DQN_BF16, of f, x, h           */
    int32_t B, C;                       /* sequences 0..65535, channels 0..2^24, the
                                           product of both at most 2^28             */
    int64_t T;                          /* steps, >= 0 (0: h_last = h0)             */
    const void *f, *x;                  /* [B][T][C]                                */
    int64_t f_bs, f_ts, x_bs, x_ts;     /* strides of a sequence and of a step; that
                                           of a step at most 2^24 (any with T = 1)  */
    const float *h0;                    /* [B][C], or NULL = zeros                  */
    const uint8_t *reset;               /* [B][T], or NULL = no episode starts      */
    int64_t reset_bs, reset_ts;
    void *h;                            /* [B][T][C]                                */
    int64_t h_bs, h_ts;
    float *h_last;                      /* [B][C], or NULL                          */
    float *carry;                       /* for dqn_scan_backward, or NULL: states at
                                           some of the steps, bytes from
                                           dqn_scan_sizes                           */
    void *workspace;                    /* bytes from dqn_scan_sizes, 16-byte aligned;
                                           free for other use after the call         */
} dqn_scan_args;

/* Gradients of the recurrence.  With l_t = dh_t + a_{t+1} k_{t+1} l_{t+1}
 * (h_last adds dlast to the last):
 *   dx_t = (1 - a_t) l_t,  df_t = a_t (1 - a_t) l_t (k_t h_{t-1} - x_t),  dh0 = a_0 k_0 l_0.
 * The states are computed again from `carry` as the forward call left it. */
typedef struct {
    int32_t dtype, B, C;
    int64_t T;
    const void *f, *x;
    int64_t f_bs, f_ts, x_bs, x_ts;
    const float *carry;
    const uint8_t *reset;
    int64_t reset_bs, reset_ts;
    const void *dh;                     /* [B][T][C]                                */
    int64_t dh_bs, dh_ts;
    const float *dlast;                 /* [B][C], or NULL = zeros                  */
    void *df, *dx;                      /* [B][T][C]                                */
    int64_t df_bs, df_ts, dx_bs, dx_ts;
    float *dh0;                         /* [B][C], or NULL                          */
    void *workspace;
} dqn_scan_grad_args;

/* Bytes of `carry` and of `workspace` (of either call) for these sizes. */
int32_t dqn_scan_sizes(int32_t dtype, int32_t B, int64_t T, int32_t C, size_t *carry, size_t *workspace);
int32_t dqn_scan_forward(const dqn_scan_args *args, void *stream);
int32_t dqn_scan_backward(const dqn_scan_grad_args *args, void *stream);

/* Gated delta rule: a memory of one matrix per head, S [Dk][Dv] in fp32, with
 * a_t = sigmoid(f_t) and beta_t = sigmoid(b_t):
 *   S_t = a_t (I - beta_t k_t k_t^T) S_{t-1} + beta_t k_t v_t^T,   o_t = scale S_t^T q_t
 * for t = 0 .. T-1, S_{-1} = s0.  The state is zero before a step whose reset flag is set
 * (whatever it was, a NaN too).  A step that holds a NaN or an infinity spoils the
 * outputs of its own episode from that step on (a q its own step's) and, in the backward call, the gradients
 * of its own episode, nothing else; a gate that is shut (f = -200, say) does not end that, 0 times a NaN
 * being one.  32 steps that hold such a number are formed one by one, far slower, and their other results
 * differ by rounding: padding is better finite.  Keys are taken as they are: the rule contracts the state for
 * beta_t |k_t|^2 <= 2, beyond that it grows.  A stride of a head or of any other
 * dimension of an input may be 0 (heads that share keys); the gradients are per head then as well.
 * T = 1 is the step of an acting agent; s_last may be s0 then, and for any T. */
#define DQN_DELTA_MAX 128
typedef struct {
    int32_t dtype;                      /* DQN_F32 / DQN_BF16, of q, k, v, f, b, o  */
    int32_t B, H;                       /* sequences and heads, each 0..65535, the
                                           product of both at most 2^20             */
    int32_t Dk, Dv;                     /* 1..DQN_DELTA_MAX; a Dk of 33..63 costs what
                                           64 costs, of 65..127 what 128 costs      */
    float scale;                        /* finite                                   */
    int64_t T;                          /* steps, >= 0 (0: s_last = s0);
                                           B H ceil(T / 32) at most 2^24            */
    const void *q, *k, *v;              /* [B][T][H][Dk], the same, [B][T][H][Dv]   */
    const void *f, *b;                  /* [B][T][H]                                */
    int64_t q_s[3], k_s[3], v_s[3], f_s[3], b_s[3];
                                        /* strides of a sequence, a step, a head;
                                           that of a step at most 2^24 (any with
                                           T = 1)                                   */
    const float *s0;                    /* [B][H][Dk][Dv], or NULL = zeros          */
    const uint8_t *reset;               /* [B][T], or NULL = no episode starts      */
    int64_t reset_bs, reset_ts;
    void *o;                            /* [B][T][H][Dv]                            */
    int64_t o_s[3];
    float *s_last;                      /* [B][H][Dk][Dv], or NULL                  */
    float *carry;                       /* for dqn_delta_backward, or NULL: states at
                                           some of the steps and what lies between
                                           them, bytes from dqn_delta_sizes, 16-byte
                                           aligned                                  */
    void *workspace;                    /* forward_workspace bytes from
                                           dqn_delta_sizes, 16-byte aligned; free for
                                           other use after the call                 */
} dqn_delta_args;

/* Gradients of the rule: of all five inputs and of s0, from the gradient of o and of s_last.
 * The states are computed again from `carry` as the forward call left it. */
typedef struct {
    int32_t dtype, B, H, Dk, Dv;
    float scale;
    int64_t T;
    const void *q, *k, *v, *f, *b;
    int64_t q_s[3], k_s[3], v_s[3], f_s[3], b_s[3];
    const float *carry;
    const uint8_t *reset;
    int64_t reset_bs, reset_ts;
    const void *dout;                   /* [B][T][H][Dv]                            */
    int64_t dout_s[3];
    const float *dlast;                 /* [B][H][Dk][Dv], or NULL = zeros          */
    void *dq, *dk, *dv, *df, *db;       /* as q, k, v, f, b                         */
    int64_t dq_s[3], dk_s[3], dv_s[3], df_s[3], db_s[3];
    float *ds0;                         /* [B][H][Dk][Dv], or NULL                  */
    void *workspace;                    /* backward_workspace bytes                 */
} dqn_delta_grad_args;

/* Bytes of `carry` and of either call's workspace for these sizes. */
int32_t dqn_delta_sizes(int32_t dtype, int32_t B, int64_t T, int32_t H, int32_t Dk, int32_t Dv, size_t *carry,
                        size_t *forward_workspace, size_t *backward_workspace);
int32_t dqn_delta_forward(const dqn_delta_args *args, void *stream);
int32_t dqn_delta_backward(const dqn_delta_grad_args *args, void *stream);

/* Root-mean-square norm with the residual's addition, per row of C elements:
 *   r = x + residual,  y = weight r rstd,  rstd = 1 / sqrt(mean(r^2) + eps)
 * y is taken of the fp32 sum, r is rounded once as it is stored.  Either y (in
 * dtype) or q and scale are written: 8-bit numbers (e4m3) with y ~ q scale and
 * scale = max(max |y|, 2^-117) / 448 (a row of zeros has scale 0), the rows
 * dqn_rows_product reads.  A row that holds a NaN or an infinity has a NaN as
 * scale. */
typedef struct {
    int32_t dtype, C;                   /* 1 <= C <= DQN_NORM_MAX                   */
    int64_t M;                          /* rows, >= 0                               */
    const void *x, *residual;           /* [M][C]; residual may be NULL             */
    int64_t x_rs, residual_rs;          /* strides of a row                         */
    const float *weight;                /* [C]                                      */
    float eps;                          /* >= 0                                     */
    void *r;                            /* [M][C], or NULL; may be x or residual    */
    int64_t r_rs;
    void *y;                            /* [M][C], or NULL                          */
    int64_t y_rs;
    uint8_t *q;                         /* [M][C], or NULL; q_rs a multiple of 16,
                                           q 16-byte aligned; the bytes from C to the
                                           next multiple of 16 are set to zero       */
    int64_t q_rs;
    float *scale;                       /* [M]                                      */
    float *rstd;                        /* [M], or NULL                             */
} dqn_norm_args;
#define DQN_NORM_MAX 16384

/* Gradients of the norm, from rstd and the same x and residual: with xh = (x + residual)
 * rstd, g = weight dy,
 *   dx = rstd (g - xh mean(g xh)) + dr   (of x and of the residual alike)
 *   dw = sum over rows of dy xh          (in a fixed order)
 * With fp32 the stored r may be given as x, without a residual. */
typedef struct {
    int32_t dtype, C;
    int64_t M;
    const void *dy, *x, *residual, *dr; /* [M][C]; residual and dr may be NULL      */
    int64_t dy_rs, x_rs, residual_rs, dr_rs;
    const float *weight, *rstd;
    void *dx;                           /* [M][C]; may be dr                        */
    int64_t dx_rs;
    float *dw;                          /* [C]; M = 0 gives zeros                   */
    void *workspace;                    /* bytes from dqn_norm_sizes, 16-byte aligned */
} dqn_norm_grad_args;

int32_t dqn_norm_sizes(int64_t M, int32_t C, size_t *workspace);
int32_t dqn_norm_forward(const dqn_norm_args *args, void *stream);
int32_t dqn_norm_backward(const dqn_norm_grad_args *args, void *stream);

/* Queries and keys per head: per head of D elements a root-mean-square norm, and the rotation by
 * position in the same pass,
 *   z = weight x rstd,  rstd = 1 / sqrt(mean(x^2) + eps),
 *   y_i = z_i cos t_i - z_{i+R/2} sin t_i,  y_{i+R/2} = z_{i+R/2} cos t_i + z_i sin t_i,  i < R/2,
 *   t_i = 2 pi position turns_i,  y_i = z_i for i >= R.
 * A weight of 1 / sqrt(D) makes keys of length one, as dqn_delta_forward wants them.  Angles are
 * exact for any position: what counts of position times turns_i is its fraction, kept to
 * 2^-32 of a full turn. */
#define DQN_HEADS_MAX 256
typedef struct {
    int32_t dtype, Hq, Hk;              /* heads of queries and of keys, 0..65535   */
    int32_t D, R;                       /* 1 <= D <= DQN_HEADS_MAX; R even, 0..D    */
    float eps;                          /* >= 0                                     */
    int64_t M;                          /* rows, 0..2^31-1                          */
    const void *q, *k;                  /* [M][Hq][D], [M][Hk][D]                   */
    int64_t q_rs, q_hs, k_rs, k_hs;     /* strides of a row and of a head           */
    const float *q_weight, *k_weight;   /* [D]                                      */
    const int32_t *position;            /* [M], not read if R = 0                   */
    const double *turns;                /* HOST array [R/2], read during the call:
                                           full turns per position, finite          */
    void *yq, *yk;                      /* [M][Hq][D], [M][Hk][D]; may be q, k      */
    int64_t yq_rs, yq_hs, yk_rs, yk_hs;
    float *rstd;                        /* [M][Hq + Hk], or NULL                    */
} dqn_heads_args;

/* Gradients, from rstd and the same inputs: with dy turned back, g = weight dy and xh = x rstd,
 *   dx = rstd (g - xh mean(g xh)),   dweight = sum over rows and heads of dy xh  (in a fixed order). */
typedef struct {
    int32_t dtype, Hq, Hk, D, R;
    int64_t M;
    const void *dyq, *dyk, *q, *k;
    int64_t dyq_rs, dyq_hs, dyk_rs, dyk_hs, q_rs, q_hs, k_rs, k_hs;
    const float *q_weight, *k_weight, *rstd;
    const int32_t *position;
    const double *turns;
    void *dq, *dk;                      /* may be dyq, dyk                          */
    int64_t dq_rs, dq_hs, dk_rs, dk_hs;
    float *dq_weight, *dk_weight;       /* [D]; M = 0 gives zeros                   */
    void *workspace;                    /* bytes from dqn_heads_sizes, 16-byte aligned */
} dqn_heads_grad_args;

int32_t dqn_heads_sizes(int64_t M, int32_t Hq, int32_t Hk, int32_t D, size_t *workspace);
int32_t dqn_heads_forward(const dqn_heads_args *args, void *stream);
int32_t dqn_heads_backward(const dqn_heads_grad_args *args, void *stream);

/* Rows [M][K] to 8 bits, 1 <= K <= DQN_NORM_MAX, as dqn_norm_forward writes them: scale = max(max |x|, 2^-117) / 448
 * per row, 0 for a row of zeros. */
int32_t dqn_rows_quantize(int32_t dtype, int64_t M, int32_t K, const void *x, int64_t x_rs, uint8_t *q,
                          int64_t q_rs, float *scale, void *stream);

/* Product of 8-bit rows with 8-bit weights, y[m][n] = a_scale[m] w_scale[n] sum_k a[m][k] w[n][k] + bias[n]:
 * e4m3 numbers, y fp32 or bf16.  Sums are fp32 where y is.  For y in bf16 the e4m3 matrix
 * instructions form them: of 128 products at a time, from a multiple of 128 on, each is kept to 16 bits below the
 * exponent of the largest, so such a part of the sum is off by up to 2^-9 of its largest product
 * (rounding a number to e4m3 puts its product off by up to 2^-4; over random numbers the sums are 1.5e-5
 * off in the 2-norm, where rounding y to bf16 is 2e-3).  Ask for fp32 where small differences of
 * large products count.  Row strides of a and w are multiples of 16 bytes and the rows 16-byte
 * aligned; what lies between K and the next multiple of 16 may be read but does not count. */
typedef struct {
    int32_t dtype, N, K;                /* of y; N >= 0, K >= 0                     */
    int64_t M;                          /* >= 0; ceil(M / 256) ceil(N / 256) <= 2^22 */
    const uint8_t *a, *w;               /* [M][K], [N][K]                           */
    int64_t a_rs, w_rs;
    const float *a_scale, *w_scale;     /* [M], [N]                                 */
    const float *bias;                  /* [N], or NULL                             */
    void *y;                            /* [M][N]                                   */
    int64_t y_rs;
} dqn_product_args;
int32_t dqn_rows_product(const dqn_product_args *args, void *stream);

/* AdamW over many tensors in one launch, decoupled weight decay:
 *   m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2
 *   p <- p (1 - lr decay) - lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps)
 * Parameters are fp32.  The moments of all tensors lie one behind the other, a
 * tensor beginning at a multiple of 256 elements (the places between hold the
 * caller's zeros).  bits = 32: fp32.  bits = 8: m as e4m3, v as e5m2, each with one fp32
 * scale per 256 elements, scale = largest / 448 and largest / 57344 (a largest that is
 * not zero counts as at least 2^-117 and 2^-110); the step is computed in fp32 and p
 * takes the moments before they are rounded.  They are rounded
 * up or down at random, in proportion, since one step changes v by about 0.1 %,
 * far less than half the distance of two 8-bit numbers, and rounding to the nearest
 * would keep v where it is for ever; a v that is not zero stays so.  The random bits of
 * element i of the buffer of moments come from the library's counter-based draws:
 * 32 bits of output i / 2 for `seed` (the lower half for even i), the lower 16 for
 * m, the upper 16 for v, so a step is a function of its arguments alone.  A gradient
 * that is not finite spoils its parameter as with 32 bits, and with 8 the moments of its 256
 * elements. */
typedef struct {
    float *param;                       /* [n]                                      */
    const void *grad;                   /* [n], in the optimizer's grad_dtype       */
    uint16_t *copy;                     /* [n] bf16 copy of the new param, or NULL  */
    int64_t n;                          /* >= 0                                     */
    float decay;
} dqn_adamw_tensor;

typedef struct {
    int64_t elements;                   /* of each buffer of moments                */
    size_t m, v, m_scale, v_scale;      /* bytes; the scales are 0 for 32 bits      */
    size_t plan;                        /* bytes of the device table of tensors     */
} dqn_adamw_bytes;

typedef struct {
    void *m, *v;                        /* 256-byte aligned, like the others; the   */
    float *m_scale, *v_scale;           /* caller sets them (zeros at the start)    */
    void *plan;
} dqn_adamw_buffers;

typedef struct dqn_adamw dqn_adamw;

/* `tensors`: host array of `count` descriptions, 1 <= count <= 65536; its device pointers must
 * stay valid.  The handle owns host-side bookkeeping only; the table is copied to `plan`
 * on `stream` during dqn_adamw_init, which waits for the copy. */
int32_t dqn_adamw_sizes(const dqn_adamw_tensor *tensors, int32_t count, int32_t bits, dqn_adamw_bytes *out);
int32_t dqn_adamw_init(dqn_adamw **out, const dqn_adamw_tensor *tensors, int32_t count, int32_t bits,
                       int32_t grad_dtype, const dqn_adamw_buffers *bufs, void *stream);
/* One step, number `step` >= 1.  `seed` is used with 8 bits and should differ from step to step. */
int32_t dqn_adamw_step(dqn_adamw *opt, double lr, double beta_m, double beta_v, double eps, int64_t step,
                       uint64_t seed, void *stream);
int32_t dqn_adamw_destroy(dqn_adamw *opt);

/* A step for matrices whose momentum is made orthogonal, for many of them at once:
 *   m <- mu m + g,   u = g + mu m (nesterov) or m,   X = u / (|u| + eps), |u| the root of all squares' sum
 *   `rounds` times:  A = X X^T,  X <- 3.4445 X + (-4.775 A + 2.0315 A^2) X   (of the transposed if rows > cols)
 *   p <- p (1 - lr decay) - lr sqrt(max(1, rows / cols)) X
 * Parameters and momentum are fp32.  Within the rounds numbers are kept to 16 bits (pairs of
 * bf16), sums are fp32; five rounds take singular values between 1e-2 and 1 of |u| to 0.7 .. 1.2.  A gradient that is not finite
 * spoils its own matrix alone.  Nothing but m is kept from step to step. */
typedef struct {
    float *param, *momentum;            /* [rows][cols]; the caller sets momentum (zeros at the start) */
    const void *grad;                   /* [rows][cols], in the optimizer's grad_dtype */
    uint16_t *copy;                     /* [rows][cols] bf16 copy of the new param, or NULL */
    int64_t rows, cols;                 /* 0..2^20, the smaller at most 65536       */
    float decay;                        /* finite, >= 0                             */
} dqn_muon_matrix;

typedef struct dqn_muon dqn_muon;

/* `matrices`: host array of `count` descriptions, 1 <= count <= 65536; its device pointers must stay valid, as must plan and
 * workspace (256-byte aligned, bytes from dqn_muon_sizes): a step uses both, so steps of one handle are not to overlap.
 * The handle owns host-side bookkeeping only; the table is copied to `plan` on `stream` during dqn_muon_init, which
 * waits for the copy and so cannot be recorded into a graph.  No param, momentum or copy may lie on another buffer (gradients may
 * lie on each other). */
int32_t dqn_muon_sizes(const dqn_muon_matrix *matrices, int32_t count, size_t *plan, size_t *workspace);
int32_t dqn_muon_init(dqn_muon **out, const dqn_muon_matrix *matrices, int32_t count, int32_t grad_dtype, void *plan,
                      void *workspace, void *stream);
/* One step; 0 <= momentum < 1, 1 <= rounds <= 100. */
int32_t dqn_muon_step(dqn_muon *opt, double lr, double momentum, int32_t nesterov, double eps, int32_t rounds, void *stream);
int32_t dqn_muon_destroy(dqn_muon *opt);

#ifdef __cplusplus
}
#endif
#endif /* DQN_H_ */
