/*
 * dgs.h -- C ABI of the DGS push / apply / pull loop on one GPU.
 *
 * DGS (dual-way gradient sparsification with sparsification-aware momentum,
 * arXiv 1910.10929) lets N asynchronous workers exchange sparse updates with a
 * parameter server in both directions.  This library keeps the N workers and the
 * server on ONE device and runs, per arrival ("event") of a worker k:
 *
 *   push   worker side, Algorithm 3:  t = m*u_k + eta*grad;  per layer keep the
 *          k_j entries of largest |t| (the packet g);  u_k <- t on the sent
 *          entries and t*(1/m) on the others (Eq. 11a, Eq. 12).
 *   apply  server side, Algorithm 2:  M <- M - decode(g)  (Eq. 1).  The model is
 *          stored as theta = theta_0 + M (Eq. 2) and every worker's model
 *          difference D_q = M - v_q (Eq. 3) moves with M.
 *   pull   server side, Algorithm 2 with secondary compression (Eq. 6a/6b):
 *          per layer keep the k_j entries of largest |D_k| (the packet G), clear
 *          them in D_k (v_k <- v_k + G), leave the rest as the server's residual;
 *          optionally the worker installs theta_k <- theta_k + G (Eq. 5).
 *
 * Conventions
 *   - All numbers are IEEE binary32; every arithmetic step is one rounded
 *     operation (no fused multiply-add, no flush-to-zero), so results do not
 *     depend on launch shapes.  Inputs must be finite.
 *   - "Largest |x|" compares the bit pattern of x with the sign bit cleared.
 *     Exactly k_j entries are kept per layer; among equal magnitudes the lowest
 *     index wins.  Packets list (index, value) pairs in ascending index order.
 *   - DEVICE pointers are marked DEVICE, everything else is host memory.
 *   - The caller owns all device memory (the arena); the library allocates no device
 *     memory.  Calls only enqueue work and return.  The work runs on streams of the
 *     library's own (an event's steps follow one another on one of them, and consecutive
 *     events take several in turn, so that they overlap; a dependency tracker keeps, per
 *     buffer, the order of the calls); it is ordered after
 *     everything the caller had enqueued on the stream given at dgs_init when the call
 *     was made.  Results (packets, state) are complete for that stream after dgs_flush,
 *     and for the host after any call that is documented to wait.  One host thread per
 *     context.
 *   - The library's streams are eight at most (two for a single worker); each is created when it
 *     is first needed, and a caller that calls dgs_flush after every event uses one.  The CUDA driver maps streams onto a fixed number of hardware queues, 8 unless the
 *     environment variable CUDA_DEVICE_MAX_CONNECTIONS says otherwise, and streams that
 *     share a queue run one after the other.  The variable is read when the process creates
 *     its CUDA context, so a process that wants the overlap must set it (to 12 or more; 32
 *     is the most) BEFORE its first CUDA call; the library cannot do it later.  Results do
 *     not depend on it, only speed does.  dgs_hardware_queues tells what the process has.
 *   - 16-bit packet values (DGS_PACKET_BF16 / DGS_PACKET_FP16; not part of the paper's algorithms, its
 *     closing section names the combination with other compression as the next step): the selection is
 *     made on the unrounded magnitudes; a packet carries q = the selected value rounded to the 16-bit
 *     format (nearest, ties to even), stored as the float32 number with that value, so that a transport
 *     may ship 16 bits per value.  A push leaves the worker's velocity as Eq. 12 says (a sent entry keeps
 *     t; sparsification-aware momentum has no residual that could take t - q); under DGS_RESIDUAL_MODE
 *     the residual keeps t - q.  A pull lowers D_k by q (Eq. 6b: v_k <- v_k + G with the G that was
 *     sent), so what rounding left behind stays with the server and goes out with a later pull.
 *   - Every function returns DGS_OK (0) or a negative dgs_error.  Nothing aborts,
 *     throws or waits without bound.
 */
#ifndef DGS_H_
#define DGS_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  DGS_OK = 0,
  DGS_EINVAL = -1,   /* null pointer, worker out of range, bad segment table, m not in (0,1], n >= 2^32, misaligned pointer */
  DGS_ENOMEM = -2,   /* arena too small */
  DGS_ECUDA = -3,    /* a CUDA runtime call or launch failed; see dgs_last_cuda_error */
  DGS_ETIMEOUT = -4, /* a bounded device-side wait gave up (reported by dgs_status) */
  DGS_ESTATE = -5,   /* context already freed or unusable after an earlier error */
  DGS_ELIMIT = -6    /* size beyond a fixed capacity: dgs_topk_encode_static, or (as device status) more nonzero
                        entries than a dgs_worker_pull_all packet can carry */
} dgs_error;

typedef struct dgs_ctx dgs_ctx; /* opaque, host side */

/* One layer j of the per-layer loops of Algorithm 3 / Algorithm 2: a contiguous
 * slice [offset, offset+len) of the flat parameter vector that is sparsified on
 * its own.  Segments must be listed in ascending order and tile [0, n) exactly.
 * 1 <= k_push <= len and 1 <= k_pull <= len. */
typedef struct {
  uint64_t offset;
  uint64_t len;
  uint32_t k_push; /* entries the worker sends per push from this layer   */
  uint32_t k_pull; /* entries the server sends per pull from this layer   */
} dgs_segment;

/* A sparse update in coordinate format (the paper's encode()): count pairs,
 * idx ascending.  Packets returned by the library point into the context's own
 * packet slots (DEVICE) and stay valid until the next call that produces a packet
 * of the same kind (push or pull). */
typedef struct {
  const uint32_t* idx; /* DEVICE u32[count], flat parameter index */
  const float* val;    /* DEVICE f32[count]                        */
  uint32_t count;      /* = sum of k_push (push) or k_pull (pull)  */
} dgs_packet;

/* A sparse update whose number of entries is only known on the device (the pull without
 * secondary compression sends however many entries the difference vector holds). */
typedef struct {
  const uint32_t* idx;   /* DEVICE u32[capacity], ascending; the first *count entries are valid */
  const float* val;      /* DEVICE f32[capacity]                                                */
  const uint32_t* count; /* DEVICE u32: entries written, <= capacity                            */
  uint32_t capacity;     /* = dgs_config.pull_all_capacity                                      */
} dgs_var_packet;

enum {
  DGS_KEEP_LOCAL_MODEL = 1u << 0, /* keep theta_k per worker and add every pulled G to it (Eq. 5) */
  DGS_RESIDUAL_MODE = 1u << 1,    /* worker rule of Algorithm 1 instead of Algorithm 3: v <- v + eta*grad,
                                     sent entries leave v, the rest stay (no momentum, no 1/m rescale) */
  DGS_HOST_IO = 1u << 2,          /* reserve staging buffers for dgs_event_host */
  DGS_NO_SPECULATION = 1u << 3,   /* always take the two-pass selection (histogram pass, then stream pass) */
  DGS_SINGLE_STREAM = 1u << 4,    /* enqueue every step on ONE internal stream: kernels run one after the other in
                                     call order (same results; for debugging and for timing a kernel on its own) */
  DGS_PACKET_BF16 = 1u << 6,      /* packets carry values rounded to bfloat16 (see "16-bit packet values" below)  */
  DGS_PACKET_FP16 = 1u << 7,      /* ... to IEEE binary16, saturating at 65504; not together with DGS_PACKET_BF16  */
  DGS_TEST_STALLED_BARRIER = 1u << 5 /* testing only: the barrier among the CTAs of the finalize kernels waits for one
                                     CTA that does not exist, with a limit of a few thousand polls.  Every wait then
                                     runs out: the kernels return early, packets and state are NOT valid, and
                                     dgs_status reports DGS_ETIMEOUT.  Shows that a wait that cannot end costs a
                                     status word, not the GPU. */
};

typedef struct {
  uint64_t n;                  /* number of parameters, 1 <= n < 2^32                                  */
  uint32_t num_workers;        /* N >= 1                                                               */
  float lr;                    /* eta, finite                                                          */
  float momentum;              /* m, 0 < m <= 1 (1/m is taken once, by IEEE division)                  */
  uint32_t num_segments;       /* S >= 1, S < 65536                                                    */
  const dgs_segment* segments; /* HOST array [S], copied                                               */
  const float* theta0;         /* DEVICE f32[n], initial model (Algorithm 3, first line), copied       */
  void* arena;                 /* DEVICE memory owned by the caller, 256-byte aligned                  */
  uint64_t arena_bytes;        /* >= what dgs_arena_bytes reports for this configuration               */
  void* stream;                /* cudaStream_t on which all work is enqueued (NULL = default stream)   */
  uint32_t flags;              /* DGS_* flags above                                                    */
  uint32_t pull_all_capacity;  /* most entries a dgs_worker_pull_all packet can carry (0: that call is not
                                  used and no packet slots are set aside for it); at most n              */
} dgs_config;

enum { DGS_THETA = 0, DGS_U = 1, DGS_D = 2, DGS_THETA_LOCAL = 3 };

/* Bytes of device memory a context for this configuration carves from the arena
 * (model, N velocities + spares, N differences, packet slots, the log of applied
 * packets, selection scratch).  No GPU work.  arena/arena_bytes/theta0/stream are ignored. */
int dgs_arena_bytes(const dgs_config* cfg, uint64_t* out_bytes);

/* Creates the context: u_k = 0 and D_k = 0 for every worker (Algorithm 3 and
 * Algorithm 2, initialisation), theta = theta0, theta_k = theta0 if kept.
 * Enqueues the clears and copies on cfg->stream.  The arena must stay alive and
 * untouched by others until dgs_free. */
int dgs_init(const dgs_config* cfg, dgs_ctx** out);

/* Worker push (Algorithm 3, velocity update through encode(); Eq. 11a, Eq. 12).
 * grad: DEVICE f32[n], 16-byte aligned, read only, must stay valid until the work of
 * this call has run (dgs_flush, then the stream reaching that point).  On return *out
 * describes the push packet slot (a few slots are used in turn). */
int dgs_worker_push(dgs_ctx* ctx, uint32_t worker, const float* grad, dgs_packet* out);

/* Server apply (Algorithm 2, "M <- M - decode(g)"; Eq. 1-3): theta[i] -= val and
 * D_q[i] -= val for every worker q, the sender included, for each (i, val) of the
 * packet.  pkt may be the library's own push packet or any DEVICE packet with
 * strictly ascending indices < n (the device status word becomes negative if it is not).
 * Also advances the server timestamp t.
 * The subtraction from D_q is deferred (unless the packet is longer than the library's own): the packet is
 * filed in a log and folded into D_q, in arrival order, before anything reads D_q
 * (that worker's next pull, dgs_state_ptr); every D_q[i] sees the same subtractions
 * in the same order, so the values are the same bit for bit. */
int dgs_server_apply(dgs_ctx* ctx, uint32_t worker, const dgs_packet* pkt);

/* Worker pull with secondary compression (Algorithm 2, per-layer top-k of
 * G = M - v_k; Eq. 6a, 6b): builds the pull packet from D_worker, clears the sent
 * entries there, adds them to theta_worker when DGS_KEEP_LOCAL_MODEL is set
 * (Eq. 5), and records prev(worker) = t. */
int dgs_worker_pull(dgs_ctx* ctx, uint32_t worker, dgs_packet* out);

/* Worker pull WITHOUT secondary compression (Algorithm 2 with the switch off, the paper's
 * normal case; Eq. 3, Eq. 4): the packet lists every entry of D_worker that is not zero (+0 and
 * -0 both count as zero), in ascending index order, and those entries are cleared, so that
 * v_worker = M afterwards; they are added to theta_worker when DGS_KEEP_LOCAL_MODEL is set
 * (Eq. 5); prev(worker) = t.  The number of entries is written to a device word of the packet
 * slot (no host synchronisation); *out is filled at once.  If D_worker holds more nonzero
 * entries than cfg.pull_all_capacity, the first `capacity` of them (lowest indices) are sent
 * and cleared, the others stay in D_worker for a later pull, and the device status word
 * becomes DGS_ELIMIT (see dgs_status).  Needs pull_all_capacity > 0, else DGS_EINVAL.  A few
 * packet slots are used in turn: a packet stays valid until the fourth later call. */
int dgs_worker_pull_all(dgs_ctx* ctx, uint32_t worker, dgs_var_packet* out);

/* One whole event for `worker`: push, apply of that packet, pull.  Either packet
 * pointer may be NULL. */
int dgs_event(dgs_ctx* ctx, uint32_t worker, const float* grad, dgs_packet* push_out, dgs_packet* pull_out);

/* Makes the stream given at dgs_init wait (on the device, not the host) for all work
 * enqueued by earlier calls: what that stream runs afterwards sees their packets and
 * state.  (No counterpart in the paper: it joins the library's own streams to the caller's.) */
int dgs_flush(dgs_ctx* ctx);

/* The same event with HOST buffers (needs DGS_HOST_IO): copies grad (HOST f32[n],
 * ideally pinned) to the device, runs the event, copies the pull packet back into
 * out_idx / out_val (HOST, sum(k_pull) entries each, may be NULL to skip) and
 * waits for that work and for what earlier calls had enqueued.  This is the end-to-end path: what a worker process
 * without its own device buffers would call. */
int dgs_event_host(dgs_ctx* ctx, uint32_t worker, const float* grad_host, uint32_t* out_idx, float* out_val);

/* Pointer to a state vector, DEVICE f32[n]: which = DGS_THETA (worker ignored),
 * DGS_U, DGS_D or DGS_THETA_LOCAL.  Waits for all work in flight (velocity buffers are
 * exchanged with a spare on the device, so their address is only known then).
 * The pointer is valid until the next push of that worker (DGS_U) or dgs_free. */
int dgs_state_ptr(dgs_ctx* ctx, int which, uint32_t worker, const float** out);

/* Overwrites a state vector from src (DEVICE f32[n]) on the stream: restores a
 * checkpoint, or loads a vector to be selected from with dgs_worker_pull.  The copy runs on the stream
 * given at dgs_init, after the work in flight on that vector; only DGS_U waits on the host.  src may be a state
 * vector of the context itself: the copy then comes after all work in flight. */
int dgs_state_load(dgs_ctx* ctx, int which, uint32_t worker, const float* src);

/* Waits for all work in flight and returns the sticky device status word in
 * *device_status (0 = clean; negative dgs_error values are stored by kernels that
 * detect an out-of-range index or give up a bounded wait). */
int dgs_status(dgs_ctx* ctx, int* device_status);

/* Waits for all work in flight and reports counters: out[0] selections served by the
 * single-pass (speculative) route, out[1] selections that took the two-pass
 * route from the start or started over because the carried bound admitted fewer
 * than k candidates, out[2] server timestamp t (packets applied), out[3] candidates
 * the finalize steps have examined in total (the k selected ones included). */
int dgs_stats(dgs_ctx* ctx, uint64_t out[4]);

/* Waits for all work in flight and reports how much of the difference vectors the pulls'
 * passes had to read: out[0] chunks (4096 elements, fewer where a CTA's share ends) that
 * the passes covered, out[1] those of them of which some part was actually read.  The
 * library keeps, per 512 elements of every D_q, an upper bound on the magnitudes in it; a
 * block that no filed packet has an entry in and whose bound is below the selection's lower
 * bound cannot hold a selected entry (Eq. 6a takes the largest magnitudes) and is not read.
 * The selection stays exact. */
int dgs_pull_read_stats(dgs_ctx* ctx, uint64_t out[2]);

/* prev(worker): the server timestamp at that worker's last pull, -1 before it. */
int dgs_prev(dgs_ctx* ctx, uint32_t worker, int64_t* out);

/* Number of kernels this context has launched so far (host-side count). */
int dgs_launch_count(dgs_ctx* ctx, uint64_t* out);

/* Kernels the library launches, as indices into the arrays of dgs_timing_read. */
enum {
  DGS_KERNEL_STREAM_PUSH = 0,   /* push, single-pass route: velocity update + candidate collection      */
  DGS_KERNEL_FINALIZE_PUSH = 1, /* push, single-pass route: exact k-th key, ordered packet, fix-ups      */
  DGS_KERNEL_TWO_PASS_PUSH = 2, /* push, two-pass route only: histogram of the whole input + bound pick  */
  DGS_KERNEL_SCATTER = 3,       /* apply: theta -= packet, packet filed in the log (or the eager scatter) */
  DGS_KERNEL_STREAM_PULL = 4,   /* pull: filed packets folded in and candidates collected in one pass    */
  DGS_KERNEL_FINALIZE_PULL = 5,
  DGS_KERNEL_TWO_PASS_PULL = 6,
  DGS_KERNEL_CATCH_UP = 7,      /* filed packets folded into a difference vector without a selection     */
  DGS_NUM_KERNELS = 8
};

/* Measurement aid (no counterpart in the paper).  While on, every kernel launch of
 * this context is bracketed by two CUDA events on the stream it runs on (at most
 * 65536 launches between two reads are recorded).  A selection from a short vector that is one
 * kernel otherwise runs as its two parts, DGS_KERNEL_STREAM_* and DGS_KERNEL_FINALIZE_*, while
 * timing is on: the results are the same, but the times are of kernels that an untimed run does
 * not launch. */
int dgs_timing_enable(dgs_ctx* ctx, int on);

/* Waits for all work in flight; ms[i] / count[i] receive the summed device time in
 * milliseconds and the number of recorded launches of kernel i since the last
 * read, and the accumulators restart from zero. */
int dgs_timing_read(dgs_ctx* ctx, double ms[DGS_NUM_KERNELS], uint64_t count[DGS_NUM_KERNELS]);

/* Measurement aid (no counterpart in the paper): the launches recorded since the last read as
 * a timeline instead of sums.  Waits for all work in flight.  For the first min(cap, recorded)
 * launches, in the order they were enqueued: start_ms / stop_ms (HOST f32[cap]) receive the
 * device times of the two events around the launch, in milliseconds after the first recorded
 * launch began; kernel[i] one of DGS_KERNEL_*; stream[i] the index of the library stream it
 * ran on.  *count receives how many entries were written.  The record restarts empty (the sums
 * of dgs_timing_read do not include these launches). */
int dgs_timing_trace(dgs_ctx* ctx, uint32_t cap, float* start_ms, float* stop_ms, int32_t* kernel, int32_t* stream,
                     uint32_t* count);

/* How many hardware queues a process should ask for (*needed: room for the streams of a context, the caller's and
 * a few more) and how many the process asked the driver for (*configured: CUDA_DEVICE_MAX_CONNECTIONS as the
 * process environment has it now, 8 if unset or unreadable).  configured < needed means that some of
 * the library's streams share a queue and their kernels do not overlap.  No GPU work; either
 * pointer may be NULL.  (No counterpart in the paper.) */
int dgs_hardware_queues(int* needed, int* configured);

/* The cudaError_t of the last failed runtime call of this context (0 if none). */
int dgs_last_cuda_error(dgs_ctx* ctx);

/* Frees the host-side context.  The arena stays the caller's.  Waits for all work in flight. */
int dgs_free(dgs_ctx* ctx);

/* Largest vector dgs_topk_encode_static accepts (elements). */
#define DGS_STATIC_MAX_N (1u << 20)

/* Top-k selection and coordinate-format encoding of one flat vector, for callers that
 * must not allocate.  (No counterpart in the paper: this is the selection + encode() step
 * of dgs_worker_pull offered on its own, for one layer, without a context.)
 *
 * Who needs it: code that runs where device allocation is off limits -- inside a region
 * whose memory plan is frozen (a pre-sized pool that must not grow, a real-time or
 * serving loop that may not call into the allocator), or a plug-in that is handed
 * buffers but no allocator.  Such a caller cannot give dgs_init an arena either.  Here
 * all scratch is shared memory of the one kernel that does the selection; the only global
 * memory is the status word, which is part of the library's device image.
 *
 *   x        DEVICE f32[n], read only
 *   n, k     1 <= k <= n <= DGS_STATIC_MAX_N; a larger n returns DGS_ELIMIT, other bad
 *            arguments DGS_EINVAL, and nothing is enqueued
 *   out_idx  DEVICE u32[k], out_val DEVICE f32[k]: the k entries of largest |x| (ties to
 *            the lowest index), ascending index, exactly as dgs_worker_pull would list them;
 *            they must not overlap x, which may be read again while they are written
 *   stream   cudaStream_t; the work is enqueued there and the call returns
 *
 * The function calls no cudaMalloc / cudaFree and no allocating library routine.  The
 * first call on each device (which must be current, as for every call) sizes the launches;
 * make that first call outside any stream capture.  Calls whose work overlaps on the GPU
 * (different streams, no ordering) share nothing but the status word. */
int dgs_topk_encode_static(const float* x, uint32_t n, uint32_t k, uint32_t* out_idx, float* out_val, void* stream);

/* Device-side outcome of the dgs_topk_encode_static calls enqueued on `stream` so far.  (No
 * counterpart in the paper.)  dgs_topk_encode_static only enqueues work, so it cannot report a
 * failure that happens on the device: an internal rank check that failed leaves
 * out_idx / out_val partly unwritten.  This call waits
 * for `stream` (host-side wait), then stores in *device_status the status word of the last
 * call's kernels: 0 = the packet is complete, negative = it is not.  Like the selection itself
 * it allocates nothing (one 4-byte copy from the fixed array). */
int dgs_topk_encode_static_status(void* stream, int* device_status);

/* ---- what a worker computes before its push ------------------------------------------------------------------
 *
 * (No counterparts in the paper, whose workers compute their gradients with a framework.)  The calls below take a
 * worker from its activations to the flat gradient vector that dgs_worker_push reads: activations held in 8 bits
 * between forward and backward pass, weight and bias gradients formed from them and written to the layers'
 * slices of that vector, and, for models with experts, the router whose selection says which rows belong to which
 * expert.  They need no context.  Common rules:
 *   - Nothing is allocated; outputs and workspaces are the caller's.  Work is enqueued on `stream` (a cudaStream_t of
 *     the current device; NULL = default stream) and the call returns.  All of them may be captured into a graph once a call of
 *     the kind has been made on the device outside a capture.
 *     Two calls whose work may overlap need workspaces of their own.
 *   - Results are the same bits for the same inputs, on every run.
 *   - Outputs must not overlap inputs unless a call says so; where the ranges do, it returns DGS_EINVAL.
 *   - Sizes of zero rows (tokens) are legal: outputs that do not depend on rows are still written.
 *   - A row index or a list that points outside its matrix is skipped on the device and reported by
 *     dgs_operator_status. */

enum { DGS_TYPE_F32 = 0, DGS_TYPE_BF16 = 1, DGS_TYPE_FP16 = 2 };

/* A matrix of the caller: element [r][c] is data[r * stride + c].  stride >= cols, or 0 for a matrix that is only read
 * and whose rows are all the same one.  data is aligned to the element.  rows < 2^31. */
typedef struct {
  void* data;      /* DEVICE */
  uint64_t rows;
  uint64_t stride; /* elements */
  uint32_t cols;
  uint32_t type;   /* DGS_TYPE_* */
} dgs_matrix;

enum { DGS_FORMAT_INT8 = 0, /* codes are int8, -127 .. 127            */
       DGS_FORMAT_E4M3 = 1 /* codes are e4m3 numbers, up to 448 */ };
enum { DGS_ACT_NONE = 0, DGS_ACT_RELU = 1, DGS_ACT_GELU = 2, DGS_ACT_GELU_TANH = 3, DGS_ACT_SILU = 4 };

/* A rows x cols matrix held in 8 bits: one byte a value and one exponent byte for each 32 values of a row.  The
 * buffer holds codes [rows][W], W = cols up to a multiple of 32, then scale bytes [rows][4 for each 128 columns begun]; a
 * value is code * 2^(byte - 127), 2^e the smallest power of two for which the block's largest magnitude is at most
 * 127 * 2^e (int8) or 448 * 2^e (e4m3), with e from -126 to 121 (int8) or -117 to 119 (e4m3).  Codes are rounded to
 * nearest, ties to even: an int8 value is off by at most 2^e / 2, which is 1/127 of the block's largest magnitude, an
 * e4m3 value by 2^-4 of itself (or 2^e / 1024 near zero).  A block that holds an infinity or a NaN gets byte 255 and reads as NaN.
 * Bytes behind the last column are zero. */
typedef struct {
  void* data;      /* DEVICE, 16-byte aligned, dgs_checkpoint_bytes long */
  uint64_t rows;   /* < 2^31 */
  uint32_t cols;   /* 1 .. 2^30 */
  uint32_t format; /* DGS_FORMAT_* */
} dgs_checkpoint;

int dgs_checkpoint_bytes(uint64_t rows, uint32_t cols, uint64_t* out_bytes);

/* Holds x (rows x cols) in ckpt and, unless y is NULL, writes y = act(x), of x's type, in the same pass.  y may be x
 * itself (in place).  act: DGS_ACT_*, DGS_ACT_NONE copies. */
int dgs_checkpoint_save(const dgs_checkpoint* ckpt, const dgs_matrix* x, int act, const dgs_matrix* y, void* stream);

/* Writes the values that ckpt holds to x (in f32 and bfloat16 exactly, in fp16 rounded). */
int dgs_checkpoint_load(const dgs_checkpoint* ckpt, const dgs_matrix* x, void* stream);

/* dx = dy * act'(h), h the values that ckpt holds; dx and dy are of one type, and may be the same matrix (in place).
 * relu'(0) = 0. */
int dgs_checkpoint_activation_grad(const dgs_checkpoint* ckpt, int act, const dgs_matrix* dy, const dgs_matrix* dx, void* stream);

enum { DGS_WEIGHT_IN_OUT = 1u << 0, /* dw is [inputs][outputs]; without it [outputs][inputs] */
       DGS_WEIGHT_ADD = 1u << 1     /* dw and db are added to; without it they are set      */ };

/* Which rows belong to which expert.  Row j of dy with offsets[e] <= j < offsets[e + 1] belongs to expert e and to
 * row rows[j] / rows_per of the checkpoint (to row j if rows is NULL).  Offsets ascend; where they do not, the gradients are
 * not specified.  A row of dy in a list that names no row of the checkpoint takes no part in dw or db and is reported. */
typedef struct {
  const uint32_t* offsets; /* DEVICE u32[experts + 1] */
  const uint32_t* rows;    /* DEVICE u32[rows of dy] or NULL */
  uint32_t experts;
  uint32_t rows_per;       /* >= 1 */
} dgs_row_lists;

/* The gradient of a layer y = x W (+ b) from dy and the checkpoint of x:
 *     dw[o][i] = sum over rows r of dy[r][o] * h[r][i],     db[o] = sum over r of dy[r][o]
 * dw: DEVICE f32, inputs * outputs elements (4-byte aligned: a layer's slice of the flat gradient); db: DEVICE f32[outputs]
 * or NULL.  inputs = ckpt->cols, outputs = dy->cols.  With lists, one such gradient per expert over the expert's rows,
 * dw [experts][...] and db [experts][outputs]; an expert without rows gets zeros.  Without lists (NULL) dy has the
 * checkpoint's rows.  Products are exact and are summed in f32 (f16 and f32 gradients are taken apart into bfloat16
 * numbers whose sum they are; of an f32 gradient below 2^-110 what lies under 2^-133, the last bit of a bfloat16 number, may be lost).  A row of dy that is in no list has no part in anything.  At most DGS_ROUTE_MAX_EXPERTS experts.
 * workspace: DEVICE, 16-byte aligned, at least what dgs_checkpoint_weight_grad_bytes says for these arguments (data pointers
 * included: their alignment counts).  It takes the checkpoint's values as bfloat16 numbers (2 bytes a value for each row of dy), dy as
 * bfloat16 numbers unless it is that with rows on 16 bytes (2 bytes a value, fp16 4, f32 6), and partial results where
 * rows are split.  Rows times parts of a value below 2^31, else DGS_ELIMIT. */
int dgs_checkpoint_weight_grad_bytes(const dgs_checkpoint* ckpt, const dgs_matrix* dy, const dgs_row_lists* lists, uint32_t flags,
                                     uint64_t* out_bytes);
int dgs_checkpoint_weight_grad(const dgs_checkpoint* ckpt, const dgs_matrix* dy, const dgs_row_lists* lists, float* dw, float* db,
                               uint32_t flags, void* workspace, uint64_t workspace_bytes, void* stream);

enum { DGS_SCORE_SOFTMAX = 0, DGS_SCORE_SIGMOID = 1 };
#define DGS_ROUTE_MAX_EXPERTS 1024u
#define DGS_ROUTE_MAX_K 32u
#define DGS_NO_EXPERT 0xffffffffu /* an empty slot */

/* How a router chooses.  Scores s are the softmax of a token's logits or their sigmoid; keys are s + bias.  Experts
 * lie in `groups` equal groups; a group's key is the sum of its group_best (1 or 2) largest keys, and the
 * groups_kept groups of largest key stay.  Of their experts the k of largest key are chosen; ties go to the lowest
 * index, for groups and experts.  Without bias and with group_best = 1 the logits themselves are the keys; otherwise keys
 * are compared as 64-bit arithmetic gives them.  A token's slots list its experts in ascending order, as
 * packets list indices.  Weights are scale * s, or scale * s / (sum of the chosen s) with renormalise.
 * A logit of -inf takes the expert away from the token (score 0): never chosen, and a token with fewer than k experts left
 * has DGS_NO_EXPERT and weight 0 in its last slots.  A token with a NaN or +inf among its logits has no experts and NaN weights. */
typedef struct {
  uint32_t k;            /* 1 .. min(DGS_ROUTE_MAX_K, experts in the kept groups) */
  uint32_t score;        /* DGS_SCORE_* */
  uint32_t groups;       /* divides the number of experts; 1: no groups */
  uint32_t groups_kept;  /* 1 .. groups */
  uint32_t group_best;   /* 1 or 2 */
  uint32_t renormalise;  /* 0 or 1 */
  float scale;           /* finite */
} dgs_router;

/* logits: tokens x experts, 1 .. DGS_ROUTE_MAX_EXPERTS experts, tokens * k < 2^31.  bias: DEVICE f32[experts], finite, or NULL.  Outputs:
 *   expert   DEVICE u32[tokens][k], weight DEVICE f32[tokens][k]
 *   offsets  DEVICE u32[experts + 1]: the list of expert e is order[offsets[e] .. offsets[e + 1])
 *   order    DEVICE u32[tokens * k]: slots t * k + j, ascending in each list; DGS_NO_EXPERT behind the last list
 *   place    DEVICE u32[tokens][k]: where in order a slot stands; DGS_NO_EXPERT for an empty one
 * offsets, order and place may be NULL, all three.  workspace: DEVICE, 16-byte aligned, dgs_route_experts_bytes long. */
int dgs_route_experts_bytes(const dgs_router* router, uint64_t tokens, uint32_t experts, uint64_t* out_bytes);
int dgs_route_experts(const dgs_router* router, const dgs_matrix* logits, const float* bias, uint32_t* expert, float* weight,
                      uint32_t* offsets, uint32_t* order, uint32_t* place, void* workspace, uint64_t workspace_bytes, void* stream);

/* The gradient of the weights taken back to the logits: dlogits (tokens x experts, of the logits' type) from the logits,
 * the experts chosen (DEVICE u32[tokens][k], as dgs_route_experts writes them; an index past the last expert is treated as an empty slot
 * and reported) and dweight (DEVICE f32[tokens][k]).  The choice itself has no gradient.  dlogits may be logits (in place). */
int dgs_route_experts_grad(const dgs_router* router, const dgs_matrix* logits, const uint32_t* expert, const float* dweight,
                           const dgs_matrix* dlogits, void* stream);

/* Waits for `stream` and stores in *device_status the lowest status that kernels of the calls above have left on the current device
 * since the last time it was read: 0, DGS_EINVAL (an index or list pointed outside its matrix) or DGS_ETIMEOUT (a bounded wait gave up).  The word is one
 * for the device and is read and cleared in one step: a report is returned once, to whichever caller reads it first. */
int dgs_operator_status(void* stream, int* device_status);

/* Static text for a dgs_error value. */
const char* dgs_error_string(int err);

#ifdef __cplusplus
}
#endif
#endif /* DGS_H_ */
