/* fusedinf.h -- C ABI of the fused multi-model CNN inference library (gfx950).
 *
 * The library implements the hot path of FusedInf (Section IV "System Design",
 * Algorithm 1): several independent CNN inference models are compiled into ONE
 * DAG -- the disjoint union of the members' layer graphs, no edge between members
 * -- which is then loaded, executed and swapped as a unit.  "Efficient memory
 * allocation" and "Fewer memory calls" (Section IV-B) become: one device
 * allocation per load, holding one contiguous weight arena for all members that
 * is filled by one pinned-host-to-device copy.  The inference loop of Algorithm 1
 * (every node evaluates phi(sum_j u_j x_j) on tensors of its own model) becomes
 * one launch schedule in which nodes of different members at the same depth run
 * as grouped kernels; members of different architecture, which rarely share a
 * kernel shape, form separate lanes of that schedule that run concurrently.
 * Properties C1 / C4 (Section III-A, Section IV-C) are kept: no operator is
 * merged across members, each member's output is bit-identical to the member run
 * alone, and no member reads another member's tensors.
 *
 * Conventions
 *  - Every call returns fi_status; on error out-parameters are untouched and
 *    fi_last_error() holds a thread-local message.  No exception crosses the ABI.
 *  - "host" / "device" is stated for every pointer.  Specs and host weight blobs
 *    are BORROWED: the caller keeps them alive until fi_destroy().
 *  - State machine:  BUILT --fi_load--> LOADED --fi_run*--> LOADED --fi_unload-->
 *    BUILT --fi_destroy--> gone.  Any other transition returns FI_ESTATE.
 *  - All members of one DAG share the weight dtype and the input shape.  fi_run
 *    feeds one shared input batch to every member; fi_run_inputs gives each
 *    member an input of its own (Algorithm 1's per-model inputs x^m).
 *  - Buffers: a run over `batch` images reads batch x fi_dag_info.input_image_bytes
 *    bytes from every input pointer it is given and writes batch x
 *    fi_member_info.output_row_bytes bytes to each member's output pointer.  The
 *    library cannot see how much memory stands behind a pointer: size the buffers
 *    from those two figures.
 *  - The planner may fold a node into its neighbours (a concatenation written in
 *    place by its producers, a per-channel affine or squeeze-excite scaling
 *    applied by the convolution that reads it, a concatenation that a shuffle
 *    interleaves): such a node has no launch and no tensor of its own, and every
 *    output keeps the bits of the unfolded schedule (fi_build_opts.copy_concats,
 *    fi_build_opts.separate_affine switch the folding off).
 */
#ifndef FUSEDINF_H
#define FUSEDINF_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct fi_dag fi_dag; /* opaque, owned by the library, one per fi_build_dag */

typedef enum {
  FI_OK = 0,
  FI_EINVAL = 1,        /* malformed spec / argument (cycle, dangling index, shape mismatch) */
  FI_EUNSUPPORTED = 2,  /* well-formed but outside what the kernels cover */
  FI_ESTATE = 3,        /* call not allowed in the handle's current state */
  FI_ENOMEM_HOST = 4,   /* host / pinned allocation failed */
  FI_ENOMEM_DEVICE = 5, /* device allocation failed; handle stays BUILT */
  FI_EBUDGET = 6,       /* DAG needs more device bytes than fi_build_opts.max_device_bytes */
  FI_EHIP = 7           /* a HIP runtime call failed */
} fi_status;

typedef enum { FI_F32 = 0, FI_BF16 = 1 } fi_dtype;
typedef enum { FI_CONV2D = 0, FI_DWCONV2D = 1, FI_MAXPOOL2D = 2, FI_GLOBAL_AVGPOOL = 3, FI_FC = 4, FI_SOFTMAX = 5, FI_CONCAT = 6, FI_AVGPOOL2D = 7, FI_MUL = 8, FI_SLICE = 9, FI_SHUFFLE = 10 } fi_op;
/* hard sigmoid h(v) = min(max(v + 3, 0), 6) / 6, hard swish v * h(v); sigmoid s(v) = 1 / (1 + exp(-v)), SiLU v * s(v) */
typedef enum { FI_ACT_NONE = 0, FI_ACT_RELU = 1, FI_ACT_RELU6 = 2, FI_ACT_HARDSWISH = 3, FI_ACT_HARDSIGMOID = 4,
               FI_ACT_SILU = 5, FI_ACT_SIGMOID = 6 } fi_act;

#define FI_INPUT (-1)       /* fi_layer_spec.input: the model's input tensor */
#define FI_NO_RESIDUAL (-2) /* fi_layer_spec.residual: nothing is added */
#define FI_MAX_GROUP 16     /* most problems one grouped launch carries */

/* One node u_i of a member's layer graph (Algorithm 1: node, its in-edge, its
 * activation phi_i).  Nodes are listed in topological order.
 *   conv2d / depthwise: y = act(conv(x, w) + b [+ residual]); cross-correlation,
 *     zero padding, floor output size.  Kernels are square (kh == kw) except that a
 *     dense conv2d may be rectangular (e.g. 1x7, 7x1); `pad` then applies only along the
 *     dimensions the kernel extends over (size > 1).  The residual
 *     is added BEFORE the activation.  Depthwise: cin == cout, one filter/channel.
 *     conv2d with groups = G > 1: output channel o sees only the input channels of
 *     its group o / (cout/G); canonical weights are then [cout][cin/G][kh][kw].  (Packed
 *     as block-diagonal dense rows: exact, at dense cost.)
 *   maxpool2d: max over in-range taps (padding acts as -inf); floor output size, or with
 *     ceil_mode the size rounded up (windows may hang over the far edge, the last one still
 *     starts inside the input or its leading padding).
 *   avgpool2d: in-range taps summed, divided by the window area kh*kw (zero padding counts),
 *     floor output size, one rounding on store.
 *   mul: `input` scaled per (image, channel) by the 1x1 tensor `residual` (the gate of a
 *     squeeze-and-excitation block); no activation.
 *   slice: channels [c_first, c_first + cout) of `input`.   shuffle: the channels, seen as a
 *     groups x (C/groups) matrix, transposed (output channel i*groups + g = input channel
 *     g*(C/groups) + i).  Both move values unchanged; no activation.
 *   concat: the channels of `input` followed by the channels of `residual` (here: the
 *     second source, same height and width); no activation.  cout = sum of both.
 *   global_avgpool: mean over H*W.   softmax: over the channel axis of a 1x1 tensor.
 *   fc: y = act(x W^T + b); cin = C*H*W of its input, flattened in (c,h,w) order.
 * w_off / b_off: byte offsets into the member's CANONICAL blob: weights
 * [cout][cin/groups][kh][kw] (fc: [cout][cin]) in the model dtype, bias [cout] fp32.
 * cin/cout of pooling, global_avgpool and softmax nodes are ignored (derived). */
typedef struct {
  int32_t op;       /* fi_op */
  int32_t input;    /* node index in this model, or FI_INPUT */
  int32_t residual; /* node index, or FI_NO_RESIDUAL */
  int32_t cin, cout, kh, kw, stride, pad;
  int32_t act;      /* fi_act */
  int32_t ceil_mode; /* maxpool2d only: 1 = output size rounds up */
  int32_t groups;    /* conv2d: channel groups (0 or 1 = dense), must divide cin and cout; shuffle: groups */
  int32_t c_first;   /* slice only: first channel taken */
  int32_t reserved;
  uint64_t w_off, b_off;
} fi_layer_spec;

/* One member model m.  `weights` (host) is either the canonical blob described
 * above (weights_packed == 0; the library converts it while building) or a blob
 * already in device layout written by fi_model_pack (weights_packed == 1; the
 * repository-time form that makes loading a pure copy).
 * act_dtype: storage precision of this member's intermediate tensors.  FI_BF16
 * (bf16 weights only) rounds every stored activation to bf16 once per node;
 * FI_F32 keeps activations in fp32 (mandatory for an FI_F32 model; for a bf16
 * model it buys fp32-grade accuracy at twice the activation traffic). */
typedef struct {
  const char* name;             /* host, borrowed, may be NULL */
  int32_t dtype;                /* fi_dtype of the weights */
  int32_t act_dtype;            /* fi_dtype of stored activations */
  int32_t in_c, in_h, in_w;     /* logical input [batch, in_c, in_h, in_w] */
  int32_t n_layers;
  const fi_layer_spec* layers;  /* host, borrowed */
  int32_t output_node;          /* node whose value is the member's prediction */
  int32_t weights_packed;       /* 0 canonical, 1 device layout (fi_model_pack) */
  const void* weights;          /* host, borrowed until fi_destroy */
  uint64_t weight_bytes;
} fi_model_spec;

typedef enum {
  FI_LOAD_ONE_COPY = 0,  /* gather members into one pinned image at build; fi_load = 1 H2D copy */
  FI_LOAD_PER_MODEL = 1, /* no host gather; fi_load copies each member's packed blob (+1 for the schedule) */
  FI_LOAD_AUTO = 2       /* gather only when it pays: members that are all in device layout are copied one by one
                          * straight out of the repository's blobs by the FIRST load of the handle (a set of models
                          * that is loaded once, as when the subset changes with every request, never pays a host
                          * gather); a handle that is loaded AGAIN gathers its image then, once, and from there on
                          * every load is one copy.  With a canonical member the image has to be written at build
                          * anyway and the mode is FI_LOAD_ONE_COPY. */
} fi_load_mode;

/* Allocator callbacks let the caller's memory pool (e.g. a tensor library's
 * caching allocator) back the library's memory.  NULL = hipMalloc / hipHostMalloc.
 * A callback returning NULL is reported as FI_ENOMEM_DEVICE / FI_ENOMEM_HOST. */
typedef struct {
  int32_t max_batch;         /* largest batch fi_run will be given (>= 1) */
  int32_t group_levels;      /* 1: same-depth nodes of different members share launches; 0: one launch per node */
  int32_t load_mode;         /* fi_load_mode */
  int32_t use_graph;         /* 1: fi_run replays the schedule as one HIP graph (needs a non-NULL stream) */
  int32_t serial_lanes;      /* 0: members of different architecture run concurrently on internal streams; 1: one stream */
  int32_t per_member_inputs; /* 1: every member reads an input of its own (fi_run_inputs); 0: one shared input */
  uint64_t max_device_bytes; /* 0 = unlimited; else fi_build_dag fails with FI_EBUDGET beyond it */
  void* (*dev_alloc)(size_t bytes, void* user);
  void (*dev_free)(void* ptr, void* user);
  void* (*pin_alloc)(size_t bytes, void* user);
  void (*pin_free)(void* ptr, void* user);
  void* user;
  uint64_t swap_headroom_bytes; /* extra device bytes fi_load allocates beyond the plan, for later fi_swap_model calls */
  int32_t copy_concats;      /* 0: producers whose only other readers allow it write straight into the concatenation's
                              * tensor and the concatenation needs no launch; 1: every concatenation copies its sources.
                              * The outputs are the same bits either way. */
  int32_t separate_affine;   /* 0: a per-channel affine node (1x1 depthwise, e.g. a DenseNet layer's normalisation + ReLU) or a
                              * squeeze-excite scaling (FI_MUL) read only by a 1x1 convolution is applied by that convolution
                              * while it loads its input and needs no launch; 1: it runs as a launch of its own.  The outputs
                              * are the same bits either way. */
  int32_t separate_chains;   /* 0: a dense convolution whose only reader is a 1x1 convolution (and that one's 1x1 reader, if it has
                              * one) runs with it in ONE launch per 128-pixel tile: the first output stays in registers, the second
                              * is written once and not read back (a ResNet bottleneck: 3x3 -> 1x1 expand -> the next block's 1x1
                              * reduce); 1: every convolution is a launch of its own.  The outputs are the same bits either way. */
  int32_t member_chunks;     /* 0 / 1: every level runs all members of a lane together.  c >= 2: the early, activation-heavy levels
                              * of a lane's members (up to the depth after which a member's live activations stay below two thirds
                              * of their peak) run for one chunk of ceil(members / c) members after the other, the deeper levels for
                              * all members together as ever: the chunks' early tensors share memory, so the activation arena shrinks,
                              * at the price of more, smaller launches.  The outputs are the same bits either way. */
  int32_t separate_stem;     /* 0: a 7x7 stride-2, 3x3 stride-1 or 3x3 stride-2 convolution over the model input with 64 output channels
                              * (the first layer of the ResNet-style families, of VGG, of SqueezeNet 1.1) runs from an input patch held on
                              * chip, and a 3x3 stride-2 max-pool (padding 0 or 1) that alone reads a stride-2 one runs in the same launch
                              * (the convolution's output is stored nowhere); a 3x3 stride-1 convolution of 64 to 64 channels on images wider than
                              * 91 pixels (VGG's second layer) and the 2x2 stride-2 max-pool that alone reads it are one launch in DAGs of one lane;
                              * 1: the general convolution kernels and pooling launches of their own.  The outputs are the same bits either way. */
  int32_t reserved0;
} fi_build_opts;

typedef struct {
  uint64_t arena_bytes;      /* weight arena: schedule tables + every member's packed weights */
  uint64_t act_bytes;        /* activation arena at max_batch (liveness-planned) */
  uint64_t workspace_bytes;  /* kernel scratch */
  uint64_t device_bytes;     /* the one allocation fi_load makes = sum of the three (aligned) */
  uint64_t macs_per_image;   /* multiply-accumulates of conv/depthwise/fc nodes, all members */
  int32_t n_models, n_nodes, n_levels, n_launches;
  int32_t n_device_allocs;   /* device allocations per fi_load (1) */
  int32_t n_h2d_copies;      /* host-to-device copies per fi_load (1 in FI_LOAD_ONE_COPY) */
  int32_t state;             /* 0 BUILT, 1 LOADED */
  int32_t n_lanes;           /* concurrent launch lanes (groups of members with identical architecture) */
  uint64_t device_capacity;  /* bytes of the loaded allocation (device_bytes at load + swap headroom); 0 when BUILT */
  uint64_t last_h2d_bytes;   /* bytes moved by the most recent fi_load or fi_swap_model */
  int32_t last_h2d_copies;   /* copies issued by the most recent fi_load or fi_swap_model */
  int32_t reserved;
  uint64_t input_image_bytes; /* one input image [in_h, in_w, in_c] in the weight dtype: a run over `batch` images reads
                               * batch x this many bytes from the input pointer it is given, so size the buffer from it */
} fi_dag_info;

typedef struct {
  uint64_t arena_off, packed_bytes; /* placement of the member's packed weights in the weight arena */
  int32_t lane;                     /* launch lane of the member */
  int32_t first_node, n_nodes;      /* its nodes are [first_node, first_node + n_nodes) */
  int32_t reserved;
  uint64_t output_row_bytes;        /* one image's output row (fp32): a run writes batch x this many bytes to the member's output pointer */
} fi_member_info;

/* Introspection of the compiled DAG (tests, reports). */
typedef struct {
  int32_t model, index;      /* member and node index inside the member */
  int32_t op, level, launch; /* depth level (1-based) and the launch that executes it */
  int32_t out_c, out_h, out_w, out_cp; /* logical shape and padded channel stride of the output */
  int32_t out_dtype;         /* fi_dtype of the stored output */
  int32_t is_output;         /* 1: written to the caller's output buffer, not the arena */
  int32_t first_level, last_level; /* live range of the output tensor in levels */
  uint64_t out_off, out_bytes;     /* placement in the activation arena (at max_batch) */
  uint64_t w_off, b_off;           /* placement in the weight arena */
  uint64_t macs;                   /* per image */
} fi_node_info;

typedef struct {
  int32_t level, kind, n_problems, first_node; /* kind: internal kernel family id */
  int32_t lane, tile;        /* launch lane (stream); tile: which of the kernels of that name it is, 0 where there is one (internal id, as kind) */
  uint64_t macs_per_image;   /* dense work of the launch */
  uint64_t bytes_per_image;  /* compulsory activation bytes (in + out + residual), per image */
  uint64_t weight_bytes;     /* weight + bias bytes read once per launch */
  char name[32];             /* name of the kernel, e.g. "conv_mfma_128x128" */
} fi_launch_info;

/* Section IV, "DNN model repository": the repository keeps every model ready to
 * be served, with its memory requirement.  Here: the size and the content of a
 * member's device-layout blob, computed at repository time on the host (no device
 * is touched).  model: host, borrowed for the call, canonical weights
 * (weights_packed == 0).  bytes: out, untouched on error.  FI_EINVAL for a null
 * argument or a malformed spec, FI_EUNSUPPORTED for an operator or size the
 * kernels do not cover. */
fi_status fi_model_packed_size(const fi_model_spec* model, uint64_t* bytes);
/* Same passage.  dst (host, caller-owned, ideally pinned) receives
 * fi_model_packed_size bytes: the exact image of the member's range in the weight
 * arena, so that a later load is a plain copy.  FI_EINVAL when dst_bytes is too
 * small or the blob is already packed; dst is then untouched. */
fi_status fi_model_pack(const fi_model_spec* model, void* dst, uint64_t dst_bytes);

/* Algorithm 1, DAG compilation: union the members' graphs, assign depth levels,
 * form grouped launches, lay out the weight arena and the activation arena.  Host
 * only: touches no device.  models: host array of n (1..) specs. */
fi_status fi_build_dag(const fi_model_spec* models, int32_t n, const fi_build_opts* opts, fi_dag** out);
fi_status fi_query(const fi_dag* dag, fi_dag_info* info);
fi_status fi_node(const fi_dag* dag, int32_t i, fi_node_info* info);     /* i in [0, n_nodes) */
/* i in [0, n_launches): the launch as planned.  Launches of many rows are issued to kernels of their own where the images that a pass brings
 * are enough (the outputs are the same bits); fi_launch_at names the kernel that a pass of `batch` images per member issues, 1 <= batch <= max_batch. */
fi_status fi_launch(const fi_dag* dag, int32_t i, fi_launch_info* info);
fi_status fi_launch_at(const fi_dag* dag, int32_t i, int32_t batch, fi_launch_info* info);
fi_status fi_member(const fi_dag* dag, int32_t m, fi_member_info* info); /* m in [0, n_models) */

/* The footprint fi_build_dag would report for these members (Section IV: the
 * repository knows every model's memory requirement, the manager sizes DAGs by
 * it), computed from the architectures alone: no pinned image is made and no
 * weight byte is read.  Same errors as fi_build_dag. */
fi_status fi_footprint(const fi_model_spec* models, int32_t n, const fi_build_opts* opts, fi_dag_info* info);

/* Section IV-B, "Efficient memory allocation" and "Fewer memory calls": the whole
 * DAG gets ONE device allocation (weight arena, activation arena and workspace
 * together, through fi_build_opts.dev_alloc when given) and, in FI_LOAD_ONE_COPY,
 * ONE pinned-to-device copy of fi_dag_info.arena_bytes bytes (in
 * FI_LOAD_PER_MODEL: the 256-byte header plus one copy per member).  The copy is
 * asynchronous on hip_stream (a hipStream_t, NULL = default stream); every later
 * pass, on whichever stream it is issued, is ordered after it by the library.
 * BUILT -> LOADED.  FI_ESTATE when already loaded, FI_ENOMEM_DEVICE when the
 * allocation fails, FI_EHIP when a copy cannot be issued (the handle stays BUILT
 * and the allocation is returned). */
fi_status fi_load(fi_dag* dag, void* hip_stream);

/* Algorithm 1, DAG inference: one pass of the launch schedule, asynchronous on
 * hip_stream.  d_input: device, [batch, in_h, in_w, in_c] (NHWC) in the DAG's
 * weight dtype (fp32, or bf16 bit patterns), read-only, shared by all members.
 * d_outputs: HOST array of n_models DEVICE pointers; member m receives its output
 * node's value as fp32 [batch, out_h, out_w, out_c] (unpadded NHWC), i.e.
 * [batch, classes_m] logits for a classifier, or probabilities if the output
 * node is a softmax.  1 <= batch <= max_batch.  Allocates nothing. */
fi_status fi_run(fi_dag* dag, const void* d_input, int32_t batch, void* const* d_outputs, void* hip_stream);

/* For callers that cannot allocate device memory or let the library do it (code being
 * recorded into a HIP graph, tight serving loops, harnesses that forbid hipMalloc): the
 * pass of fi_run, same arguments and same output bits, with the split-K partial sums
 * kept in a static device array of the library (FI_STATIC_SCRATCH_BYTES per GPU, held
 * until the process ends) instead of the workspace region of the loaded allocation.
 * Calls no hipMalloc / hipFree and no allocating library routine; always launches
 * eagerly (use_graph is ignored).  FI_EBUDGET when fi_dag_info.workspace_bytes exceeds
 * FI_STATIC_SCRATCH_BYTES (fi_run still serves such a DAG).  Every call on a GPU shares
 * that GPU's array: two calls that overlap in time on one GPU, from whichever handle,
 * stream or thread, race on it.  Nothing in the array needs clearing between calls. */
#define FI_STATIC_SCRATCH_BYTES (32u << 20)
fi_status fi_run_static(fi_dag* dag, const void* d_input, int32_t batch, void* const* d_outputs, void* hip_stream);

/* Algorithm 1 gives every member model m its own input x^m: the same pass with
 * d_inputs a HOST array of n_models DEVICE pointers, member m reading
 * d_inputs[m] ([batch, in_h, in_w, in_c] NHWC in the weight dtype, read-only; all
 * members share the input shape and the batch).  Needs a DAG built with
 * fi_build_opts.per_member_inputs = 1 (else FI_ESTATE); such a DAG stages one
 * channel-padded copy per member instead of one per activation dtype and channel
 * stride, and fi_run
 * on it feeds the one input to every member.  Always launches eagerly (use_graph
 * applies to fi_run). */
fi_status fi_run_inputs(fi_dag* dag, const void* const* d_inputs, int32_t batch, void* const* d_outputs, void* hip_stream);

/* The same pass when the members have gathered different numbers of requests
 * (Section IV: the manager aggregates, per model, the requests that arrived while
 * the device was busy): member m runs on batches[m] images (HOST array of n_models
 * entries, 0 <= batches[m] <= max_batch) read from d_inputs[m] and writes
 * [batches[m], classes_m] to d_outputs[m].  A member with batches[m] == 0 sits the
 * pass out: none of its kernels get a workgroup, its pointers may be NULL and its
 * output buffer is not touched.  An image's output bits do not depend on the batch
 * it travels in.  Needs per_member_inputs = 1 (else FI_ESTATE); launches eagerly. */
fi_status fi_run_batches(fi_dag* dag, const void* const* d_inputs, const int32_t* batches, void* const* d_outputs,
                         void* hip_stream);

/* One lane of that pass, on the caller's stream: only the launches of the members of `lane`
 * (fi_member_info.lane; lanes are 0 .. fi_dag_info.n_lanes - 1) run, for batches[m] images of each of
 * them; the entries of members of other lanes are ignored.  Lanes share no tensor and the call touches
 * no state of the handle, so calls for DIFFERENT lanes may be in flight at the same time, on different
 * streams and from different threads (two calls for one lane may not).  Needs per_member_inputs = 1. */
fi_status fi_run_lane(fi_dag* dag, int32_t lane, const void* const* d_inputs, const int32_t* batches,
                      void* const* d_outputs, void* hip_stream);

/* Same pass with every launch issued on hip_stream (lanes serialised) and a HIP
 * event between launches; ms[i] (host, n_launches floats) receives launch i's
 * elapsed milliseconds: the kernel's own time with the chip to itself.
 * Synchronises the stream. */
fi_status fi_profile(fi_dag* dag, const void* d_input, int32_t batch, void* const* d_outputs, void* hip_stream,
                     float* ms, int32_t n_ms);

/* Same pass issued exactly as fi_run issues it (Section 3: independent members
 * run side by side, here as concurrent lanes), with a HIP event after every
 * launch on the stream it went to.  Launch i occupies [begin_ms[i], end_ms[i]]
 * (host arrays, n >= n_launches floats each), in milliseconds since the pass
 * began: from the end of the previous launch on the same stream to its own
 * end.  Intervals of different lanes overlap.  Synchronises the stream. */
fi_status fi_timeline(fi_dag* dag, const void* d_input, int32_t batch, void* const* d_outputs, void* hip_stream,
                      float* begin_ms, float* end_ms, int32_t n);

/* Section V, "individual model swaps in a DAG" (Table IV): replaces member `slot`
 * by `model` without recompiling or reloading the rest.  The sub-graph of the
 * outgoing member is dropped, the newcomer's is compiled into the schedule, and
 * in a LOADED handle only the newcomer's packed weights travel to the device
 * (one copy, asynchronous on hip_stream) into the lowest free range of the weight
 * arena that holds them; every other member's weights stay where they are, and
 * their outputs keep their bits.  The handle may be BUILT (host work only) or
 * LOADED; no fi_run may be in flight on another stream.  `model` follows the rules
 * of fi_build_dag (borrowed; same weight dtype and input shape as the other
 * members; device layout required in FI_LOAD_PER_MODEL).  Fails, leaving the DAG
 * exactly as it was, with FI_EBUDGET when the new plan does not fit the loaded
 * allocation (fi_build_opts.swap_headroom_bytes reserves room at load) or
 * max_device_bytes, and with the fi_build_dag errors for a bad model. */
fi_status fi_swap_model(fi_dag* dag, int32_t slot, const fi_model_spec* model, void* hip_stream);

/* ---- manager-side scheduling (Section IV, "Manager"; Section V, consecutive swaps) ----
 * A set of models that does not fit the device at once is cut into batches that
 * each fit; every batch is compiled into its own DAG; the scheduler runs a fixed
 * number of iterations per DAG, swaps it out and takes the next, round robin. */

/* Batches in the caller's order, first fit: model m joins the current batch while
 * the batch's exact device footprint (fi_footprint) stays within budget_bytes.
 * group_of: host, n entries out (batch index of every model, non-decreasing);
 * n_groups: out.  FI_EBUDGET when a single model exceeds the budget. */
fi_status fi_partition(const fi_model_spec* models, int32_t n, const fi_build_opts* opts, uint64_t budget_bytes,
                       int32_t* group_of, int32_t* n_groups);

typedef struct {
  int32_t iterations;   /* fi_run passes per DAG before it is swapped out (>= 1) */
  int32_t rounds;       /* round-robin rounds over all batches (>= 1) */
  int32_t overlap_load; /* 1: the next batch is loaded on an internal copy stream while the current one
                           computes, so two batches are resident at a time; 0: unload, then load */
  int32_t reserved;
} fi_sched_opts;

typedef struct {
  double build_ms;            /* compiling every batch (host, once) */
  double total_ms;            /* all rounds: loads, runs, unloads */
  double run_ms;              /* time spent waiting for the runs of a batch (incl. a load still in flight) */
  double swap_ms;             /* time spent in unload (+ the next load when not overlapped) */
  uint64_t peak_device_bytes; /* largest resident footprint (two batches with overlap_load) */
  int32_t n_loads, n_runs, n_groups, reserved;
} fi_sched_stats;

/* Compiles one DAG per batch (group_of as produced by fi_partition; any grouping
 * with every batch non-empty is accepted), then for `rounds` rounds visits the
 * batches in order: load, `iterations` x fi_run on hip_stream with the shared
 * d_input (device, as for fi_run), unload.  d_outputs: HOST array of n DEVICE
 * pointers indexed like `models`; model m's buffer holds the output of its last
 * run on return.  A single batch stays resident for all rounds.  With
 * opts->max_device_bytes set, FI_EBUDGET if the resident peak would exceed it.
 * Synchronous: returns after the last unload.  stats may be NULL. */
fi_status fi_round_robin(const fi_model_spec* models, int32_t n, const fi_build_opts* opts, const int32_t* group_of,
                         int32_t n_groups, const fi_sched_opts* sched, const void* d_input, int32_t batch,
                         void* const* d_outputs, void* hip_stream, fi_sched_stats* stats);

/* ---- request aggregation (Section IV, "Manager": requests that arrive while the device
 * is busy are gathered per model into the next batch) ----
 * A server sits in front of a LOADED DAG built with per_member_inputs = 1.  Callers submit
 * single images for single members; every lane of the DAG has a worker thread (with a stream
 * of its own) that repeatedly takes up to max_batch waiting requests of each of its members,
 * runs ONE fi_run_lane pass and hands every request its output row.  The busier the device,
 * the larger the batches; a short model never waits for a long one.  While a server runs,
 * nothing else may use the DAG. */
typedef struct fi_server fi_server; /* opaque, owned by the library */

typedef struct {
  int32_t max_wait_us; /* when a request finds the server idle, wait this long for companions before
                          the pass starts (0 = start at once) */
  int32_t reserved;
} fi_server_opts;

typedef struct {
  uint64_t requests, passes;    /* requests served; lane passes (fi_run_lane) issued */
  uint64_t max_images_per_pass; /* most requests one lane pass carried (all members of the lane together) */
  double mean_images_per_pass;
  double mean_latency_ms, max_latency_ms; /* submit to output written, host clock */
  double busy_ms;               /* time with a pass in flight, summed over the lanes */
} fi_server_stats;

/* Allocates, through the DAG's allocator callbacks, one batch buffer of max_batch images and one of
 * max_batch output rows per member, and starts the worker on the current device.  opts may be NULL.
 * FI_ESTATE unless the DAG is LOADED and was built with per_member_inputs = 1. */
fi_status fi_server_start(fi_dag* dag, const fi_server_opts* opts, fi_server** out);
/* Queues one image for member `member`.  d_image: device, [in_h, in_w, in_c] in the weight dtype,
 * complete in memory before the call and untouched until fi_server_wait returns; d_output: device,
 * receives the member's output row (fp32, classes_m values).  Requests of one member are served in
 * order.  Thread-safe.  ticket: out, never 0. */
fi_status fi_server_submit(fi_server* srv, int32_t member, const void* d_image, void* d_output, uint64_t* ticket);
/* Blocks until the request's output is in d_output (the copy has completed).  Thread-safe.  Reports
 * the worker's error, if it met one, on this and every later call. */
fi_status fi_server_wait(fi_server* srv, uint64_t ticket);
fi_status fi_server_query(fi_server* srv, fi_server_stats* stats);
/* Section V, individual model swaps, under load: replaces member `slot` of the served DAG (fi_swap_model).
 * The requests already queued for the slot are served by the outgoing model first; then every lane
 * finishes its pass in flight, the swap re-plans the DAG (its lanes included) and new workers start.
 * Requests for the slot submitted while the call is in progress are refused with FI_ESTATE; requests
 * for the other members are accepted throughout and served before or after the swap.  Blocks until
 * the newcomer's weights are on the device.
 * `model` is borrowed as by fi_swap_model (until fi_destroy of the DAG).  Errors of fi_swap_model are
 * returned and leave the server as it was. */
fi_status fi_server_swap(fi_server* srv, int32_t slot, const fi_model_spec* model);
/* Serves what is queued, joins the worker, releases the buffers and the handle; the DAG stays LOADED. */
fi_status fi_server_stop(fi_server* srv);

/* Sections I and III (problem statement: models are swapped in and out of device
 * memory many times a day; C3, low overhead): the swap-out half.  Synchronises the
 * device, returns the one allocation (through fi_build_opts.dev_free when given);
 * the handle goes back to BUILT with its plan and pinned image intact, so the same
 * DAG can be loaded again without recompiling.  FI_ESTATE unless LOADED. */
fi_status fi_unload(fi_dag* dag);
/* Same passages: the end of a DAG's life.  Unloads if needed, frees the pinned image
 * and the plan; the specs and host blobs the handle borrowed are the caller's again.
 * NULL is allowed. */
void fi_destroy(fi_dag* dag);

/* ---- decoder operators ----
 * What a decoder member runs on every step, as operators of their own on the caller's device tensors: the norms of its
 * queries and keys with the position rotation (the step's keys and values go to their slots of a paged cache), attention
 * over whole prompts, attention of drafted trees (or single tokens) over that cache, and products with 4-bit weights.
 *
 * Common to all of them
 *  - Every call is asynchronous on hip_stream (a hipStream_t of the current device, NULL = default stream), allocates
 *    nothing, synchronises nothing and may be recorded into a HIP graph.  The argument struct is read during the call only.
 *  - dtype is FI_BF16 or FI_F32 and holds for every tensor of data; sums, softmax statistics and norms are fp32, and a
 *    result is rounded once, when it is stored.  Attention on bf16 also rounds the softmax weights that it multiplies the values
 *    with (to 8 bits; to 16 and more over a cache where max_nodes times the query heads of a key head is 32 at most).
 *  - All tensor pointers are device pointers.  Strides are in elements of the tensor's type; the last dimension (head_dim,
 *    inputs, outputs) is contiguous.  Inputs may have any strides >= 0; rows that start on 16-byte boundaries take the fast kernels.
 *    Outputs must not overlap themselves (every dimension, from the shortest stride on, strides over all that the ones before it
 *    reach) or an input, except that q_out may be q, k_out k and v_out v with equal strides.
 *  - What sits in device memory (offsets, lengths, page and slot numbers) cannot be checked by the call: the kernels clamp
 *    it to the sizes given here, so that nothing outside the tensors is read or written, and the rows concerned are unspecified.
 *  - FI_EINVAL for a null or misaligned pointer, a negative size or stride or sizes that contradict each other,
 *    FI_EUNSUPPORTED for well-formed sizes that the kernels do not cover, FI_EHIP when a launch fails.  Nothing is
 *    written then.  Sizes of zero (no tokens, no rows, no sequences) are no error: there is nothing to do.
 */
#define FI_MAX_AXES 4
#define FI_MAX_HEAD_DIM 256

/* y = rotate(x * w / sqrt(mean(x^2) + eps)) for every head of every token's q and k, in one launch; v is copied.
 * The first rot_dim values of a head are rotated in pairs: pair i is (i, i + rot_dim / 2), or (2i, 2i + 1) when
 * interleaved, and turns by the angle positions[token][axis of i] * inv_freq[i] (fp32): (a, b) -> (a cos - b sin,
 * b cos + a sin).  The pairs are dealt to the axes in order, sections[a] of them to axis a (time, height, width of an image or
 * video patch; one axis for text): the first n_axes sections add up to rot_dim / 2.  The values behind rot_dim are normed only. */
typedef struct {
  int32_t dtype;                 /* fi_dtype of q, k, v and of the outputs */
  int32_t tokens, q_heads, kv_heads, head_dim; /* head_dim in [1, FI_MAX_HEAD_DIM] */
  int32_t rot_dim;               /* even, in [0, head_dim] */
  int32_t interleaved;           /* 0 / 1 */
  int32_t n_axes;                /* in [1, FI_MAX_AXES] */
  int32_t sections[FI_MAX_AXES];
  float eps;                     /* >= 0 */
  int32_t page_size;             /* with slots: tokens per page (>= 1) */
  int64_t n_slots;               /* with slots: slots of the cache (pages x page_size); a token whose slot lies outside [0, n_slots)
                                  * leaves the cache as it is (padding), its q is still written */
  const void *q, *k, *v;         /* [tokens, heads, head_dim]; v may be NULL (then v_out is, too); k is not NULL where kv_heads > 0 */
  const float *q_weight, *k_weight; /* [head_dim], fp32; NULL = ones */
  const int32_t* positions;      /* [tokens, n_axes], contiguous */
  const float* inv_freq;         /* [rot_dim / 2], fp32 */
  const int64_t* slots;          /* [tokens]: where the token's k and v go, page * page_size + place in the page; no two tokens share a
                                  * slot.  NULL = k_out and v_out are [tokens, kv_heads, head_dim] */
  void *q_out, *k_out, *v_out;
  int64_t q_strides[2], k_strides[2], v_strides[2], q_out_strides[2]; /* token, head */
  int64_t k_out_strides[3], v_out_strides[3];                        /* page (unused without slots), token, head */
} fi_qk_norm_rope_args;
fi_status fi_qk_norm_rope(const fi_qk_norm_rope_args* args, void* hip_stream);

/* out = softmax(scale * q k^T) v over packed sequences: sequence b has the queries [cu_q[b], cu_q[b + 1]) and the keys
 * [cu_k[b], cu_k[b + 1]); query head h reads key head h / (q_heads / kv_heads).  causal: the sequence's last query sees every key and
 * each one before it a key less (with more keys than queries the first keys are a prefix that all see; with fewer, the first
 * queries see nothing).  A query that sees nothing yields zeros, and what a key or value holds that a query does not see, were it NaN,
 * has no influence on it. */
typedef struct {
  int32_t dtype;
  int32_t n_seqs, q_heads, kv_heads, head_dim; /* kv_heads divides q_heads; head_dim in [1, FI_MAX_HEAD_DIM] */
  int32_t causal;                /* 0 / 1 */
  float scale;                   /* finite, > 0 */
  int32_t reserved;
  int64_t q_tokens, k_tokens;    /* rows of q and out, of k and v; below 2^31 - 1024 */
  const void *q, *k, *v;         /* [tokens, heads, head_dim] */
  const int32_t *cu_q, *cu_k;    /* [n_seqs + 1], ascending from 0 to q_tokens / k_tokens */
  void* out;                     /* [q_tokens, q_heads, head_dim] */
  int64_t q_strides[2], k_strides[2], v_strides[2], out_strides[2]; /* token, head */
} fi_prompt_attention_args;
fi_status fi_prompt_attention(const fi_prompt_attention_args* args, void* hip_stream);

/* The same for trees of drafted tokens over a paged cache.  Sequence b has cached[b] committed tokens and the nodes
 * [cu_nodes[b], cu_nodes[b + 1]) of q, whose own keys and values are in the cache already, at the places cached[b] ... behind the
 * committed ones (fi_qk_norm_rope puts them there).  Place p of the sequence is row p % page_size of page
 * block_table[b][p / page_size].  A node sees every committed token, and node j of its own sequence where bit j % 64 of
 * mask[node][j / 64] is set (its ancestors and itself); without a mask, the nodes up to itself (a chain).  A tree of one node is
 * a decoding step.  Rows that see nothing and unseen NaNs: as above.
 * With long histories and few nodes the keys are shared out over workgroups, whose parts a second launch joins, always in
 * the same order; they are kept in `workspace` meanwhile, the caller's, of at least fi_tree_attention_workspace bytes (0: may be
 * NULL).  Calls that overlap in time need a workspace each. */
typedef struct {
  int32_t dtype;
  int32_t n_seqs, q_heads, kv_heads, head_dim;
  int32_t page_size, n_pages;    /* tokens per page, pages of the caches */
  int32_t table_columns;         /* pages that a row of block_table names; page_size * table_columns below 2^31 - 1024 */
  int32_t mask_words;            /* 64-bit words per node; a sequence has at most 64 * mask_words nodes (later ones are not seen).  0 without a mask */
  int32_t max_nodes;             /* most nodes of a sequence: later ones are neither computed nor seen */
  int32_t max_length;            /* most committed tokens and nodes of a sequence together; only guides how the work is shared out */
  float scale;                   /* finite, > 0 */
  int64_t nodes;                 /* rows of q and out, of all sequences; nodes * q_heads below 2^31 - 1024 */
  const void *q, *k_cache, *v_cache; /* [nodes, q_heads, head_dim], [n_pages, page_size, kv_heads, head_dim] */
  const int32_t* block_table;    /* [n_seqs, table_columns], rows table_stride apart */
  const int32_t* cached;         /* [n_seqs] */
  const int32_t* cu_nodes;       /* [n_seqs + 1], ascending from 0 to nodes */
  const uint64_t* mask;          /* [nodes, mask_words], contiguous, or NULL */
  void* out;                     /* [nodes, q_heads, head_dim] */
  void* workspace;               /* 16-byte aligned */
  uint64_t workspace_bytes;
  int64_t q_strides[2], out_strides[2]; /* token, head */
  int64_t k_strides[3], v_strides[3];   /* page, token, head */
  int64_t table_stride;
} fi_tree_attention_args;
/* Bytes of workspace that fi_tree_attention needs for these sizes (pointers and strides are not looked at). */
fi_status fi_tree_attention_workspace(const fi_tree_attention_args* args, uint64_t* bytes);
fi_status fi_tree_attention(const fi_tree_attention_args* args, void* hip_stream);

/* y[m][n] = sum over groups g of scales[n][g] * sum over k in g of (w[n][k] - zeros[n][g]) * x[m][k]: a few rows times a
 * matrix of 4-bit weights, read once per 1 to 32 rows, by the sizes.  w holds two weights in [0, 15] per byte, the even one in the low half;
 * a group is `group` consecutive inputs.  The weights enter the products exactly, scales are applied to fp32 sums; fp32 inputs may enter as
 * three bf16 terms, exactly from about 1e-33 on, below that to 2^-133.  A result that is no finite number that way is computed
 * again term by term, (q - zero) * scale * x in fp32: infinities, NaNs and inputs near the largest number give what the formula gives
 * (a row with them takes longer), and the other rows are not touched by it.
 * With more than a few rows the inputs are shared out over workgroups, whose sums a second launch adds, always in the same
 * order; they are kept in `workspace` meanwhile, the caller's, of at least fi_q4_matmul_workspace bytes (0: may be NULL).
 * Calls that overlap in time need a workspace each. */
typedef struct {
  int32_t dtype;                 /* of x and out */
  int32_t rows, inputs, outputs;
  int32_t group;                 /* 32, 64 or a multiple of 128; divides inputs */
  int32_t reserved;
  const void* x;                 /* [rows, inputs] */
  const uint8_t* w;              /* [outputs, inputs / 2] */
  const float* scales;           /* [outputs, inputs / group] */
  const uint8_t* zeros;          /* [outputs, inputs / group], values in [0, 15]; NULL = 8 */
  void* out;                     /* [rows, outputs] */
  void* workspace;               /* 16-byte aligned */
  uint64_t workspace_bytes;
  int64_t x_stride, w_stride, scales_stride, zeros_stride, out_stride; /* between rows */
} fi_q4_matmul_args;
/* Bytes of workspace that fi_q4_matmul needs for these sizes (pointers and strides are not looked at). */
fi_status fi_q4_matmul_workspace(const fi_q4_matmul_args* args, uint64_t* bytes);
fi_status fi_q4_matmul(const fi_q4_matmul_args* args, void* hip_stream);

/* ---- beams over a cache held in 4 bits ----
 * What a decoder member needs when several continuations of a request live at a time: a paged cache that takes a quarter of the memory, attention
 * over it, the selection of the continuations, and the bookkeeping of pages that they share.  All of it stays on the device, so that a whole step is one
 * graph: fi_beam_select's parents are fi_fork_pages' parents, whose slots are fi_fp4_cache_write's slots.
 * What is common to the decoder operators above holds for these too.
 *
 * The 4-bit cache: a head's values in blocks of FI_FP4_BLOCK, the last one maybe shorter.  A value is a code times the block's power of two.  Codes are
 * E2M1: 0 to 7 are 0, 0.5, 1, 1.5, 2, 3, 4, 6, plus 8 negative; two to a byte, the even value in the low half.  A block's scale is one byte b: 2^(b - 127), b in
 * [0, 252], or 255: every value of the block is NaN.  (253 and 254 count as 255 where a query does not see the key, and may give infinities where it does.)
 * codes are [n_pages, page_size, kv_heads, head_dim / 2] and scales [n_pages, page_size, kv_heads, blocks], with strides in bytes: the tokens of a head in
 * a page should lie together in memory (strides of a page kv_heads * page_size rows, of a head page_size rows, of a token one row).  Strides and starts of codes are
 * multiples of 4 bytes. */
#define FI_FP4_BLOCK 32

/* A step's keys and values into the cache.  A block's scale is the smallest power of two from 2^-125 to 2^125 whose six-fold no value of the block exceeds (what
 * exceeds 6 * 2^125 is cut to that), its codes are the nearest ones, on a border the even code; a block with a NaN or an infinity gets scale 255 and codes 0. */
typedef struct {
  int32_t dtype;                 /* of k, v, k_held and v_held */
  int32_t tokens, kv_heads, head_dim; /* head_dim: a multiple of 8, at most FI_MAX_HEAD_DIM */
  int32_t page_size;
  int32_t reserved;
  int64_t n_slots;               /* pages x page_size; a token whose slot lies outside [0, n_slots) leaves the cache as it is */
  const void *k, *v;             /* [tokens, kv_heads, head_dim]; v may be NULL (then v_codes, v_scales and v_held are, too) */
  const int64_t* slots;          /* [tokens]: page * page_size + place in the page; no two tokens share a slot */
  uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
  void *k_held, *v_held;         /* NULL, or [tokens, kv_heads, head_dim]: what the cache holds for the tokens, for attention over a prompt that is to
                                  * agree with later steps; written for tokens without a slot, too */
  int64_t k_strides[2], v_strides[2], k_held_strides[2], v_held_strides[2];                     /* token, head; elements */
  int64_t k_codes_strides[3], k_scales_strides[3], v_codes_strides[3], v_scales_strides[3];     /* page, token, head; bytes */
} fi_fp4_cache_write_args;
fi_status fi_fp4_cache_write(const fi_fp4_cache_write_args* args, void* hip_stream);

/* fi_tree_attention over such a cache; the values of the cache enter the products exactly.  Pages of 16 tokens, or a multiple, take the fast kernels; others two to three
 * times as long over long histories.  Queries enter exactly, too, up to the largest number of their type; scores before `scale`, their differences, and sums over the keys of 2^8 times their
 * values have to be in fp32's range.
 * Softmax weights are fp32 in their sum; before they multiply a value they are rounded to 24 bits for fp32, for bf16 to 16, or to 8 in heads of up to 128 where a key head has more than 32 rows
 * (the smaller of max_nodes and nodes, times the query heads that share it): relative errors of 1.65e-3, what rounding the result to bf16 makes, and 2.1e-3. */
typedef struct {
  int32_t dtype;                 /* of q and out */
  int32_t n_seqs, q_heads, kv_heads, head_dim;
  int32_t page_size, n_pages, table_columns, mask_words, max_nodes, max_length;
  float scale;
  int64_t nodes;
  const void* q;                 /* [nodes, q_heads, head_dim] */
  const uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
  const int32_t* block_table;    /* from here on as in fi_tree_attention_args */
  const int32_t* cached;
  const int32_t* cu_nodes;
  const uint64_t* mask;
  void* out;
  void* workspace;
  uint64_t workspace_bytes;
  int64_t q_strides[2], out_strides[2]; /* token, head; elements */
  int64_t k_codes_strides[3], k_scales_strides[3], v_codes_strides[3], v_scales_strides[3]; /* page, token, head; bytes */
  int64_t table_stride;
} fi_fp4_tree_attention_args;
fi_status fi_fp4_tree_attention_workspace(const fi_fp4_tree_attention_args* args, uint64_t* bytes);
fi_status fi_fp4_tree_attention(const fi_fp4_tree_attention_args* args, void* hip_stream);

/* The `keep` best continuations of every sequence over its beams and the vocabulary.  Row s * beams + b of logits is beam b of sequence s, whose score is
 * scores[s][b]; a continuation with token t scores scores[s][b] + logits[row][t] - log(sum over u of exp(logits[row][u])), and one that is NaN or minus infinity is none (so a
 * beam with score minus infinity has none, nor a row of logits with a NaN or plus infinity; minus infinity is a masked token).  Best first; of equal scores the lowest beam's first, of
 * one beam's the higher logit's, then the lower token's.  Where there are fewer than `keep`, the rest is token -1, parent -1, score minus infinity.
 * end >= 0: the token that ends a sequence.  A beam with ended[s][b] != 0 has one continuation, itself: token `end`, its score unchanged; its logits are not looked at. ended_out
 * tells for each continuation whether it has ended. */
#define FI_MAX_BEAMS 64
typedef struct {
  int32_t dtype;                 /* of logits */
  int32_t n_seqs, beams, keep, vocab; /* beams and keep in [1, FI_MAX_BEAMS]; beams * vocab below 2^31 - 1024 */
  int32_t end;                   /* below vocab; negative: none */
  int64_t logits_stride;         /* elements between rows */
  const void* logits;            /* [n_seqs * beams, vocab] */
  const float* scores;           /* [n_seqs, beams] */
  const uint8_t* ended;          /* [n_seqs, beams] or NULL (none has); only with end >= 0 */
  int32_t* tokens_out;           /* [n_seqs, keep] */
  int32_t* parents_out;          /* [n_seqs, keep]: rows of logits */
  float* scores_out;             /* [n_seqs, keep] */
  uint8_t* ended_out;            /* [n_seqs, keep], 0 / 1; NULL without end */
  void* workspace;               /* 16-byte aligned */
  uint64_t workspace_bytes;
} fi_beam_select_args;
fi_status fi_beam_select_workspace(const fi_beam_select_args* args, uint64_t* bytes);
fi_status fi_beam_select(const fi_beam_select_args* args, void* hip_stream);

/* One cache whose pages are copied: page p is the page_bytes bytes from base + p * page_stride (bytes) on. */
typedef struct {
  void* base;
  int64_t page_stride, page_bytes;
} fi_page_cache;

/* The rows of a block table after a selection.  Row r of block_table holds ceil(held[r] / page_size) pages for its lengths[r] committed tokens and those that room was
 * made for; refs[p] counts how often page p is held (by these rows or anyone else), 0: it is free.
 *  1. All rows let go of what they hold.  New row i continues row parents[i]: it shares the pages of that row's committed tokens.  A parent
 *     outside [0, rows) is none: the new row is empty, length 0, and holds nothing.
 *  2. With room > 0 every continuing row gets pages for `room` tokens behind the committed ones, the lowest free page first, in the order of the rows.  A row whose last
 *     page is partly filled and held more than once gets a copy of it in its place, whose page is the first that the row gets.  Rows are looked at in order: one that
 *     copies has given the old page up for those after it, so the last of those that share a page keeps it.  A row whose tokens do not fit the table's columns gets
 *     nothing and copies nothing.  Nor does one for which, counting what all rows before it need, pages are lacking, or one that would go on in a page of which such a row
 *     holds more (it would write over that row's tokens).
 * Written are the new rows (-1 behind the pages that a row holds), lengths, held (lengths + room for the rows that got it, else lengths), refs, and the slots of the
 * `room` tokens, page * page_size + place (-1 where there is no room: what writes to a cache leaves such tokens out).  A copy is of the whole page, in every one of
 * `caches`; nothing else in them changes.  Entries that are no pages are kept, count nowhere and are no slots. */
typedef struct {
  int32_t rows, new_rows;        /* of block_table, of what comes out; at most 2^16 each */
  int32_t columns, page_size, n_pages, room; /* page_size * columns and n_pages below 2^31 - 1024, room at most 2^16 */
  int32_t n_caches;              /* at most FI_MAX_PAGE_CACHES */
  int32_t reserved;
  int64_t table_stride, table_out_stride;
  const int32_t* block_table;    /* [rows, columns] */
  const int32_t* lengths;        /* [rows] */
  const int32_t* held;           /* [rows] or NULL (lengths) */
  const int32_t* refs;           /* [n_pages] */
  const int32_t* parents;        /* [new_rows], or NULL: row i continues row i */
  const fi_page_cache* caches;   /* [n_caches], host memory, read during the call only */
  int32_t *table_out, *lengths_out, *held_out, *refs_out; /* [new_rows, columns], [new_rows], [new_rows], [n_pages]; none of them may be an input */
  int64_t* slots_out;            /* [new_rows, room]; NULL with room 0 */
  void* workspace;               /* 16-byte aligned */
  uint64_t workspace_bytes;
} fi_fork_pages_args;
#define FI_MAX_PAGE_CACHES 128
fi_status fi_fork_pages_workspace(const fi_fork_pages_args* args, uint64_t* bytes);
fi_status fi_fork_pages(const fi_fork_pages_args* args, void* hip_stream);

/* Moves the pages in use (refs > 0), `live` of them, to the page numbers below `live`: those there stay, the ones above move into the free ones below,
 * in ascending order both.  A page is copied in every one of `caches`; what it leaves is not cleared.  Entries of block_table that are pages in use are renumbered, others are kept. */
typedef struct {
  int32_t rows, columns, n_pages, n_caches; /* rows at most 2^16, n_pages below 2^31 - 1024 */
  int64_t table_stride, table_out_stride;
  const int32_t* block_table;    /* [rows, columns] */
  const int32_t* refs;           /* [n_pages] */
  const fi_page_cache* caches;   /* [n_caches], host memory, read during the call only */
  int32_t *table_out, *refs_out; /* none of them may be an input */
  int32_t* moved_out;            /* [n_pages]: the new number of every page, -1 for a free one */
  int32_t* live_out;             /* [1] */
  void* workspace;               /* 16-byte aligned */
  uint64_t workspace_bytes;
} fi_compact_pages_args;
fi_status fi_compact_pages_workspace(const fi_compact_pages_args* args, uint64_t* bytes);
fi_status fi_compact_pages(const fi_compact_pages_args* args, void* hip_stream);

const char* fi_last_error(void); /* thread-local, valid until the next call on this thread */
const char* fi_version(void);

#ifdef __cplusplus
}
#endif
#endif /* FUSEDINF_H */
