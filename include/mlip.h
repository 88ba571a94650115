/*
 * libmlip -- graph-partitioned inference of a radial message-passing
 * interatomic potential on one AMD MI355X (gfx950).  C ABI, no C++ or torch
 * types.  Every pointer argument is marked HOST or DEVICE.
 *
 * The problem statement followed here is the paper's: the inputs are atom
 * positions, the periodic cell and chemical identities (Introduction,
 * E = phi(r_i, C_i); appendix "Parallelizing a Model": the distributed object
 * takes positions, periodic boundary conditions and cell lattice and builds
 * the graph partitions and their transfer metadata), the output is the energy
 * and the forces F = -dE/dr obtained by a reverse pass that runs through the
 * per-layer border-node transfers (Introduction, "graph-level partitioning";
 * Methods, "Graph-Parallel Message Passing").
 *
 * Conventions
 *   - every function returns 0 (MLIP_OK) or a negative mlip_status; no C++
 *     exception or abort crosses this boundary; on error no output argument is
 *     written and mlip_last_error() describes the failure (thread-local text);
 *   - a graph handle owns all device memory it obtains - from the caller's
 *     allocator if the handle was made by mlip_graph_create with one, from
 *     hipMalloc otherwise - until mlip_graph_destroy; inputs are borrowed for
 *     the duration of the call and never written; one handle must not be used
 *     from two threads at once (different handles may be);
 *   - all work is enqueued on the HIP stream given to mlip_build_graph
 *     (a hipStream_t passed as void*, NULL = default stream); outputs of
 *     mlip_forward are valid after that stream is synchronised;
 *   - atoms are numbered 0..N-1 in input order; edges are directed i <- j
 *     (i receives, j sends) and carry an integer image shift S so that the
 *     sender's image sits at r_j + S.C, C = rows of `cell`.
 */
#ifndef MLIP_H
#define MLIP_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    MLIP_OK = 0,
    MLIP_EINVAL = -1,      /* null pointer, N <= 0, r_cut <= 0, n_slabs outside [1,64], bad model dims, types or strides */
    MLIP_ECELL = -2,       /* singular cell, or cell/positions outside the supported image range */
    MLIP_ECOINCIDENT = -3, /* two atoms (or an atom and an image) at distance 0 */
    MLIP_ENOMEM = -4,      /* device allocation failed */
    MLIP_EHIP = -5,        /* HIP runtime error */
    MLIP_ESTATE = -6       /* call not valid for this handle (e.g. SLABS mode on a graph built with n_slabs = 1) */
} mlip_status;

enum { MLIP_MODE_WHOLE = 0, MLIP_MODE_SLABS = 1 };
/*
 * Filters: w_e = MLP(basis(d_e)) is a function of the edge length alone.  A model's filters are tabulated on the device
 * (piecewise polynomials made in fp64, kept and evaluated in fp32), checked there feature by feature against what the
 * evaluation of the MLP in fp32 rounds, and looked up per edge; weights whose filters the tables do not represent (they bend
 * too fast: large W1, or a cutoff short in the units of W1) take the MLP per edge.  Which of the two a call takes follows
 * from the weights and the cutoff alone.
 *
 * MLIP_PRECISION_FP32: everything from the basis on in fp32 (products as exact sums of three bf16 parts per operand on the
 *   bf16 matrix units, all terms down to 2^-24, accumulated in fp32).  An operand beyond the bf16 range (3.39e38; fp32 ends
 *   at 3.40e38) or infinite makes its row of the product NaN, as it does in the fp32 products of the other modes: a result
 *   that is not finite may be NaN where an fp32 multiplication would have given an infinity.
 * MLIP_PRECISION_BF16: the F x F products of the filter MLP (forward w = SiLU(t) W2, reverse sbar = wbar W2^T)
 *   take bf16 operands with fp32 accumulation (benchmark configuration 4: "edge MLPs in bf16 with fp32
 *   accumulation"), and in mlip_forward_bonds the F x F products of the bond MLPs as well; everything else stays
 *   fp32 (arrays, the K = 8 products, activations, sums).  Forces then agree with the fp64 result to about
 *   4e-3 max|F|.  Tables are made from W2 rounded to bf16 and from activations that are not rounded.
 * MLIP_PRECISION_FP32_SPLIT: the same products (the bond MLPs' included) with every operand split into two fp16 parts (hi + lo, 22
 *   significant bits) and taken as three fp16 MFMA products with fp32 accumulation.  The results meet the fp32
 *   mode's bounds (the dropped terms are of the size of fp32 accumulation rounding) in a fraction of the matrix
 *   time; the operands of those products - SiLU outputs and the products abar * g of the reverse pass - must
 *   stay below the fp16 range (65504), which holds for any physical input but is not checked: a value beyond it
 *   becomes infinite in the split and the energy and forces come out non-finite.  On tables the mode is the fp32 one.
 */
enum { MLIP_PRECISION_FP32 = 0, MLIP_PRECISION_BF16 = 1, MLIP_PRECISION_FP32_SPLIT = 2 };

typedef struct mlip_graph mlip_graph_t;

/*
 * Caller-supplied device allocator (appendix "Parallelizing a Model": the distributed object owns the graph
 * metadata while the features live in the framework's tensors - here the framework's allocator hands out every
 * device block the handle uses, graph arrays and feature workspace alike, so that the framework's memory
 * accounting sees them).
 *   alloc(bytes, ctx)  returns a DEVICE pointer aligned to at least 256 bytes, valid on the handle's stream, or
 *                      NULL when out of memory (the call in progress then fails with MLIP_ENOMEM);
 *   free(ptr, ctx)     takes a block back; the library synchronises the handle's stream first, so no enqueued
 *                      kernel still uses the block.
 * Both are called on the thread that calls into the library, only from mlip_build_graph, mlip_forward,
 * mlip_forward_bonds and mlip_graph_destroy.  Buffers are grow-only: a rebuilt handle asks for memory only when
 * a buffer must grow.
 */
typedef struct {
    void *(*alloc)(size_t bytes, void *ctx);
    void (*free)(void *ptr, void *ctx);
    void *ctx;
} mlip_alloc_t;

/*
 * Creates an empty handle that takes all its device memory from `alloc` (copied; NULL or a NULL alloc function:
 * hipMalloc / hipFree).  Pass the handle to mlip_build_graph, which fills it.  mlip_build_graph with *graph ==
 * NULL is the same as creating a handle without an allocator first.
 */
int mlip_graph_create(const mlip_alloc_t *alloc, mlip_graph_t **graph);

/*
 * Weights of the radial message-passing potential (benchmark configuration 0
 * defines it): species embedding; per layer l the filter MLP W1_l (K x F),
 * W2_l (F x F), the sender projection Wm_l (F x F) and the update Wo_l (F x F);
 * readout Wr1 (F x F), wr2 (F).  All fp32, row-major [fan_in][fan_out]
 * (y = x W), no biases.  DEVICE pointers, borrowed.
 * Supported: F in {32, 64}, K = 8, 0 <= L <= 8, 2 <= p <= 64, n_species >= 1.
 */
typedef struct {
    int32_t n_species, F, L, K, p, precision;
    const float *emb; /* [n_species][F] */
    const float *W1;  /* [L][K][F] */
    const float *W2;  /* [L][F][F] */
    const float *Wm;  /* [L][F][F] */
    const float *Wo;  /* [L][F][F] */
    const float *Wr1; /* [F][F] */
    const float *wr2; /* [F] */
} mlip_weights_t;

/*
 * One partition's node array and local graph (Alg. "Atom Subgraph Creation":
 * concatenated buckets plus a marker array of span starts).  All pointers are
 * DEVICE memory borrowed from the handle, valid until the next
 * mlip_build_graph on it or its destruction.
 *
 *   nodes[n_local]   local -> global atom id, laid out as
 *                    PURE | BORDER | FROM[0] | FROM[1] | ... | FROM[P-1]
 *                    (BORDER = owned atoms some other partition needs, stored
 *                    once; every span in ascending global id)
 *   markers[P+3]     HOST copy of the span starts: 0, |PURE|, |PURE|+|BORDER|
 *                    (= n_owned), then the cumulative FROM lengths
 *   row_ptr[n_local+1], senders[n_edges]
 *                    receiver-sorted CSR over local rows with local sender ids.
 *                    Rows [0, n_owned) are the owned atoms' complete rows (the
 *                    edges this partition computes: an edge belongs to the
 *                    partition of its receiving node, Distributing Atom Graphs);
 *                    rows [n_owned, n_local) list, for each ghost atom, only its
 *                    neighbours owned by this partition (used by the reverse
 *                    pass to form the ghost rows' gradients without atomics).
 *                    Order inside a row: ascending (global sender id, Sx, Sy, Sz).
 */
typedef struct {
    int64_t n_owned, n_pure, n_border, n_ghost, n_local;
    int64_t n_edges_owned; /* edges of rows [0, n_owned)  */
    int64_t n_edges;       /* edges of all local rows     */
    const int32_t *nodes;
    const int64_t *markers; /* HOST */
    const int64_t *row_ptr;
    const int32_t *senders;
    const int32_t *owned_sorted; /* the n_owned owned atoms, ascending global id */
} mlip_slab_info_t;

/*
 * Build the periodic radius graph and its slab partition
 * (neighbour-list construction, Graph-Parallel Message Passing; vertical-wall
 * partition and PURE/TO/FROM buckets, Distributing Atom Graphs, Algs.
 * "Atom Subgraph Creation" and "assign_to_partitions").
 *
 *   positions  DEVICE [n_atoms][3] fp64, Cartesian Angstrom, need not lie inside the cell
 *   cell       HOST   [3][3] fp64, rows are the lattice vectors; full periodic boundaries
 *   species    DEVICE [n_atoms] int32 in [0, n_species)
 *   r_cut      edge iff 0 < d <= r_cut with
 *                delta_k = (r_j,k - r_i,k) + ((Sx C[0][k] + Sy C[1][k]) + Sz C[2][k]),
 *                d^2 = (delta_x^2 + delta_y^2) + delta_z^2 in fp64 without FMA contraction
 *   n_slabs    P >= 1 equal-width slabs along the longest lattice vector (ties: lowest index);
 *              slab(i) = min(floor(f P), P-1), f = fractional coordinate wrapped into [0,1),
 *              computed as ((x n_x + y n_y) + z n_z) / V with n = a_{k+1} x a_{k+2}, V = a_k . n
 *   stream     hipStream_t as void*
 *   graph      in/out HOST: *graph == NULL creates a handle; a handle from an earlier call is
 *              rebuilt in place and reuses its device buffers (grow-only); on another stream than
 *              before, the call waits for what the handle has queued on the old one first
 *
 * Edges are stored sorted by (receiver, sender, Sx, Sy, Sz).  The call synchronises the stream where it needs sizes or
 * error flags on the host: for the edge count, and with slabs twice more (span starts; edge counts of the partitions).
 * Further waits: one where an atom has more neighbours than the search's staging rows hold (64 found by itself, 64 by its
 * partners), and then, as in every build with a skin or of more than 6.7 million atoms, one at the end of a whole graph;
 * one or two where a skin's candidate list is made or made anew.  The build's last kernels may still run when the call
 * returns.  Positions and species are copied into the handle.
 */
int mlip_build_graph(const double *positions, const double *cell, const int32_t *species,
                     int64_t n_atoms, double r_cut, int32_t n_slabs, void *stream,
                     mlip_graph_t **graph);

/*
 * Verlet skin for repeated builds on one handle (molecular dynamics: the paper's workload is long MD with the graph
 * and its partition rebuilt at every step - "Molecular Dynamics Simulation Stability", appendix "Graph
 * Partitioning").  With skin > 0 the handle keeps a candidate neighbour list for the cutoff r_cut + skin and the
 * positions it was built at.  A later mlip_build_graph with the same atom count, cell and r_cut first checks, on the
 * device, that no atom has moved further than skin / 2 from those positions; if so the neighbour list is the
 * candidates that pass the edge test at the new positions (no cell list, no search, no sort: same fp64 expression,
 * same order, so the graph is bit-identical to a fresh build), otherwise the candidate list is rebuilt first.
 * Positions must be continuous between builds (an atom folded back into the cell by a lattice vector counts as
 * moved).  Species may change freely.  skin = 0 (the default) searches at every build.  The partition is built
 * from the neighbour list either way.
 */
int mlip_graph_set_skin(mlip_graph_t *graph, double skin);
/* How often the candidate list was rebuilt and how often it was reused since the handle was made (HOST outputs). */
int mlip_graph_skin_stats(const mlip_graph_t *graph, int64_t *list_builds, int64_t *list_reuses);

/*
 * Energy and forces (Methods: per-layer border-node transfer forward, the same
 * transfers reversed for the gradients; appendix "Parallelizing a Model":
 * distribute / atom_transfer / aggregate).
 *
 *   mode          MLIP_MODE_WHOLE: one partition holding every atom;
 *                 MLIP_MODE_SLABS: the P slabs processed one after another, ghost rows
 *                 refreshed from their owners before every layer's edge step, ghost-row
 *                 gradients (features and positions) added back to the owners in the reverse pass
 *   energy        DEVICE [1] fp64, sum of the per-atom energies of owned atoms
 *   forces        DEVICE [n_atoms][3] fp32, F = -dE/dr, input atom order
 *   atom_energy   DEVICE [n_atoms] fp32 or NULL
 *
 * Forces are the energy's derivative to rounding: where the filters come from tables, values and slopes are tabulated apart,
 * each to some 5e-8 of the filter.
 *
 * Asynchronous on the graph's stream; does not modify the graph's topology (it uses
 * workspace owned by the handle, so two forwards on one handle must not overlap).
 *
 * The weights are re-laid-out for the matrix units and the filters tabulated (0.33 MB per layer and 32 features) on the
 * first call and kept in the handle: a later call whose mlip_weights_t (pointers, dimensions, precision) and graph cutoff
 * are identical reuses them.  After changing weight VALUES in place, or when another model's arrays have come to lie at the
 * same addresses, call mlip_graph_invalidate_weights.
 */
int mlip_forward(mlip_graph_t *graph, const mlip_weights_t *weights, int32_t mode,
                 double *energy, float *forces, float *atom_energy);

/*
 * mlip_forward for callers that cannot allocate device memory: code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc.  Same arguments, results and error codes as mlip_forward, but every
 * piece of workspace (node features and their gradients, kept filter values, per-edge accumulators, packed
 * weights, energy partial sums) is carved from one fixed device array inside the library of
 * mlip_static_scratch_bytes() = 64 MiB per GPU (beside it 5.2 MB for the filter tables), held until the process ends; the
 * call allocates and frees nothing and clears what must start at zero with fill kernels.  A graph and model whose workspace
 * (about n_local (4 + 2 L) F 4 + n_edges (36 + (L - 1) F 2) bytes summed over the partitions of the mode - the kept
 * filter values take one row per edge pair and layer, the lists of the pairs' edges are rebuilt in the array on
 * every call - plus the packed weights) exceeds the array are rejected with MLIP_EINVAL; with the event profiler enabled the call
 * returns MLIP_ESTATE.  All calls on one GPU, from any handle, share the array and find the previous call's
 * contents in it: calls that overlap on one GPU (two streams, two threads) race and must be serialised by the
 * caller.  Weights are packed and filters tabulated on every call (nothing is cached in the shared array).  The graph itself must
 * have been built before (mlip_build_graph allocates).
 */
int mlip_forward_static(mlip_graph_t *graph, const mlip_weights_t *weights, int32_t mode,
                        double *energy, float *forces, float *atom_energy);
size_t mlip_static_scratch_bytes(void);

/* Drops the handle's packed copies of the weights (two-body and bond part); the next forward call packs again. */
int mlip_graph_invalidate_weights(mlip_graph_t *graph);

/*
 * Three-body (bond graph) variant: benchmark configuration 4; the paper's counterpart is the bond graph built
 * over the atom graph, whose nodes are the atom-graph edges within a second, smaller cutoff (Methods,
 * "Distributing Bond Graphs").  Extra weights, all fp32 row-major [fan_in][fan_out], DEVICE, borrowed:
 *   We0 [K][F]        bond embedding  e0_b = bbond(d_b) We0 (Bessel basis and envelope at r_bond)
 *   Wt1 [2F + A][F]   first triplet layer, input [e0_b1, e0_b2, cos(n theta) n = 0..A-1]
 *   Wt2 [F][F]        second triplet layer, applied to sum_{b2 != b1} u_b2 SiLU(.)
 *   Wb  [L][F][F]     bond term of layer l's filter: w_e += e1_b Wb_l for a bonded edge
 * with e1_b = e0_b + u_b SiLU(m_b), u_b = u(d_b / r_bond).  A = 8.
 */
typedef struct {
    float r_bond;
    int32_t A;
    const float *We0, *Wt1, *Wt2, *Wb;
} mlip_bond_weights_t;

/*
 * Energy and forces of the three-body variant.  Arguments as mlip_forward, both modes.  The bond list of a
 * partition (edges of its owned rows with d <= r_bond, same fp64 predicate as the neighbour list; all bonds and
 * triplets of an owned centre are local to its partition) is built on the first call after a graph build or a
 * change of r_bond, which synchronises the stream once per partition.
 */
int mlip_forward_bonds(mlip_graph_t *graph, const mlip_weights_t *weights, const mlip_bond_weights_t *bond_weights,
                       int32_t mode, double *energy, float *forces, float *atom_energy);

/*
 * Bond list of the last mlip_forward_bonds, of the whole graph (p = -1, after a WHOLE call) or of partition p
 * (after a SLABS call).  Borrowed DEVICE pointers: bond_edge[n_bonds] = index of every bond's edge in that
 * graph's CSR, ascending; bond_ptr[rows + 1] = bonds of owned row i are bond_ptr[i] .. bond_ptr[i + 1];
 * n_bonds HOST.
 */
int mlip_graph_bonds(const mlip_graph_t *graph, int32_t p, const int32_t **bond_edge, const int64_t **bond_ptr,
                     int64_t *n_bonds);

/*
 * Upper / lower split of the edges of partition p's owned rows (p = -1: of the whole graph), the form in which the
 * reverse edge kernels that evaluate the filter MLP walk them.  The filter of the radial message-passing layer is a function of the edge length
 * alone (benchmark description: w_e = MLP(basis(d_e))), and the two edges of an edge / reverse-edge pair have the
 * same length, so its values are kept for one of them, the "upper" one: the edge whose reverse edge lies at a
 * larger index of the partition's edge list.  (An edge from a ghost sender is always upper: its reverse edge is in
 * a ghost row, behind all owned rows.)  All other edges of the owned rows are "lower".
 * Borrowed DEVICE pointers, valid until the next mlip_build_graph on the handle:
 *   u_row_ptr [n_owned + 1]   CSR of the upper edges over the owned rows, the edges in the order of the full list
 *   u_senders, u_eid, u_mirror [n_upper]   sender row, index of the edge and index of its reverse edge in the full list
 *   u_d [n_upper]             edge length
 *   l_row_ptr [n_owned + 1], l_senders [n_lower]   the same for the lower edges
 *   l_slot [n_lower]          index of the pair's upper edge in the upper-edge lists
 * Built on the handle's stream on first use after a graph build (by mlip_forward where its weights take the MLP, and where
 * the handle has yet to find out); n_upper and n_lower are HOST values.  Errors: MLIP_ESTATE without a graph, MLIP_EINVAL for a partition index out of range.
 */
typedef struct {
    int64_t n_upper, n_lower;
    const int64_t *u_row_ptr;
    const int32_t *u_senders, *u_eid, *u_mirror;
    const float *u_d;
    const int64_t *l_row_ptr;
    const int32_t *l_senders, *l_slot;
} mlip_pairs_t;
int mlip_graph_pairs(mlip_graph_t *graph, int32_t p, mlip_pairs_t *out);

void mlip_graph_destroy(mlip_graph_t *graph);

/*
 * N atoms, E directed edges, P slabs, all HOST outputs (any may be NULL): the sizes of the graph object the
 * paper's create_distributed returns (appendix "Parallelizing a Model in DistMLIP").
 */
int mlip_graph_sizes(const mlip_graph_t *graph, int64_t *n_atoms, int64_t *n_edges, int32_t *n_slabs);

/*
 * Whole-graph CSR, borrowed DEVICE pointers: row_ptr[N+1], senders[E], d[E] (fp32 edge lengths).  This is what the
 * paper's graph object exposes as src_nodes / dst_nodes (appendix "Parallelizing a Model in DistMLIP"): edge e of
 * row i has destination (receiver) i and source senders[e]; the neighbour list itself is the one of Methods,
 * "Graph-Parallel Message Passing".  The arrays are complete when the call returns (so are mlip_graph_mirror's): the
 * first call after a build waits for the build's last kernels if they may still run.
 */
int mlip_graph_csr(const mlip_graph_t *graph, const int64_t **row_ptr, const int32_t **senders,
                   const float **d);

/*
 * mirror[E] (DEVICE, borrowed): position of every edge's reverse edge, i.e. for e = (i <- j, S) the
 * index of (j <- i, -S).  The edge set of a radius graph is symmetric; the reverse pass uses this to
 * evaluate the distance derivative once per pair.
 */
int mlip_graph_mirror(const mlip_graph_t *graph, const int32_t **mirror);

/*
 * Image shifts of all edges written to a caller-owned DEVICE buffer [E][3] int32 (enqueued on the stream): the
 * periodic-boundary part of an edge (the distributed object is built from positions, periodic boundary
 * conditions and the cell lattice, appendix "Parallelizing a Model in DistMLIP"); the sender's image sits at
 * r_j + S.C.
 */
int mlip_graph_shifts(const mlip_graph_t *graph, int32_t *shifts);

/*
 * slab_of[N] (DEVICE, borrowed) and the axis the walls are perpendicular to (HOST): the vertical-wall partition
 * of Methods, "Distributing Atom Graphs" (walls along the longest cell dimension; appendix "Graph Partitioning").
 */
int mlip_graph_slab_of(const mlip_graph_t *graph, const int32_t **slab_of, int32_t *axis);

/* Partition p's node array and local graph. */
int mlip_graph_slab(const mlip_graph_t *graph, int32_t p, mlip_slab_info_t *info);

/*
 * FROM_p[q]: atoms partition p receives from partition q (ascending global ids), a span of p's
 * node array.  TO_q[p] is by construction the same array (Distributing Atom Graphs), so
 * mlip_graph_to(g, q, p, ...) returns the same pointer.  DEVICE, borrowed.
 */
int mlip_graph_from(const mlip_graph_t *graph, int32_t p, int32_t q, const int32_t **ids, int64_t *n);
int mlip_graph_to(const mlip_graph_t *graph, int32_t p, int32_t q, const int32_t **ids, int64_t *n);

/*
 * Per-kernel-group timing with HIP events on the graph's stream.  While enabled, every launch
 * group is bracketed by events; mlip_profile_read synchronises the stream and returns, for each of
 * the MLIP_PROF_COUNT groups, the accumulated milliseconds and launch count since the last reset.
 */
enum {
    MLIP_PROF_GRAPH = 0,   /* neighbour list, CSR, partition                 */
    MLIP_PROF_NODE = 1,    /* embedding, node projections/updates, readout    */
    MLIP_PROF_EDGE_FWD = 2,
    MLIP_PROF_EDGE_BWD = 3,
    MLIP_PROF_GHOST = 4,   /* ghost row copies and gradient add-backs         */
    MLIP_PROF_FORCE = 5,   /* force assembly and energy reduction            */
    MLIP_PROF_BOND = 6,    /* three-body variant: bond list, the kernels over bonds and the bonds' share of the rows' sums */
    MLIP_PROF_TRIPLET_FWD = 7,   /* three-body variant: the triplet sum           */
    MLIP_PROF_TRIPLET_BWD = 8,   /* three-body variant: its reverse               */
    MLIP_PROF_EDGE_FWD_LOWER = 9,  /* no launches: the forward edge step is one pass over the full edge list */
    MLIP_PROF_EDGE_BWD_LOWER = 10, /* reverse edge step, second pass (none on filter tables): the lower edges' share of the projected rows'
                                     gradients, from the kept filter values */
    MLIP_PROF_COUNT = 11
};
int mlip_profile_enable(mlip_graph_t *graph, int32_t on);
int mlip_profile_read(mlip_graph_t *graph, float *ms /*HOST [MLIP_PROF_COUNT]*/,
                      int64_t *launches /*HOST [MLIP_PROF_COUNT]*/, int32_t reset);

/* Plain device -> host copy of `bytes` bytes after synchronising the graph's stream. */
int mlip_copy_to_host(const mlip_graph_t *graph, void *dst_host, const void *src_device, size_t bytes);

/*
 * Per-species parameter tables, for programs that fit a potential's parameters (the paper's appendix demonstrates training on batches of
 * structures).  A potential keeps one row of parameters for each species (its embedding, reference energies and scales of the
 * atoms' energies) or for each pair of species; a step of a fit looks rows up, sums the atoms' gradients by species and bounds
 * the norm of all gradients before the update.
 *
 * These calls use no handle: they work on the caller's arrays, on the HIP stream given (hipStream_t as void*, NULL = default
 * stream), and take scratch memory from the caller, so they can be captured in a HIP graph and run on any stream or thread.  Results
 * are the same bits on every call with the same arguments.  Element pointers must be aligned to their elements; outputs must not
 * overlap inputs (a clipped tensor may be its own output) or each other.
 */
enum { MLIP_DTYPE_F32 = 0, MLIP_DTYPE_BF16 = 1, MLIP_DTYPE_F16 = 2 };

/*
 * Lookup: out[i][f] = scale * table[ids[i]][f], the product in fp32, rounded once to the output's type.
 *   table   DEVICE [n_rows][width] of table_dtype, element (r, f) at r * table_row_stride + f * table_col_stride (in elements, >= 0)
 *   ids     DEVICE [n] int32 (id_bits = 32) or int64 (id_bits = 64).  A negative id stands for a place that pads a batch: its row
 *           is zeros.  An id >= n_rows has no row in the table: its
 *           row here is NaN, so that it does not pass unnoticed.
 *   out     DEVICE [n][width] of out_dtype, element (i, f) at i * out_row_stride + f, out_row_stride >= width
 * n may be 0; 1 <= n_rows < 2^31, 1 <= width <= 2^20, n < 2^31.
 */
int mlip_embed(const void *table, int32_t table_dtype, int64_t n_rows, int64_t width, int64_t table_row_stride,
               int64_t table_col_stride, const void *ids, int32_t id_bits, int64_t n, float scale, void *out,
               int32_t out_dtype, int64_t out_row_stride, void *stream);

/*
 * Its gradient: out[r][f] = scale * sum over i with ids[i] == r of grad[i][f], rows that no id names are scale * 0; with
 * accumulate != 0 the old out[r][f] is added, in fp64.  Ids outside [0, n_rows) contribute nothing, whatever grad holds there.
 *   grad    DEVICE [n][width] of grad_dtype, element (i, f) at i * grad_row_stride + f * grad_col_stride (>= 0; 0 for a
 *           gradient that is the same for all atoms)
 *   out     DEVICE [n_rows][width] of out_dtype, element (r, f) at r * out_row_stride + f
 *   workspace   DEVICE scratch of at least mlip_embed_grad_workspace(n, n_rows, width) bytes, aligned to 16 bytes; its
 *           contents do not matter before and mean nothing after the call
 * Sums run in the order of the atoms, over fewer than MLIP_EMBED_GRAD_RUN atoms at a time in fp32 and over those parts in fp64 (rounded to
 * fp32 up to twice on the way: fewer than MLIP_EMBED_GRAD_RUN fp32 roundings in all); the result is rounded to fp32 and then to the output's type.
 * mlip_embed_grad_workspace returns 0 for sizes that the call refuses.
 */
enum { MLIP_EMBED_GRAD_RUN = 1024 };
size_t mlip_embed_grad_workspace(int64_t n, int64_t n_rows, int64_t width);
int mlip_embed_grad(const void *grad, int32_t grad_dtype, int64_t grad_row_stride, int64_t grad_col_stride, const void *ids,
                    int32_t id_bits, int64_t n, int64_t n_rows, int64_t width, float scale, int32_t accumulate, void *out,
                    int32_t out_dtype, int64_t out_row_stride, void *workspace, size_t workspace_bytes, void *stream);

/* One gradient tensor: n elements of type dtype, one after another.  dst: where the clipped tensor goes (may be src). */
typedef struct {
    const void *src; /* DEVICE */
    void *dst;       /* DEVICE; not used by mlip_grad_norm */
    int64_t n;
    int32_t dtype;
} mlip_tensor_t;

/*
 * Global norm of a list of tensors, sqrt(sum of all elements' squares), summed in fp64 and rounded to fp32 once.
 *   tensors   HOST [count], read before the call returns; count and any n may be 0 (norm 0)
 *   norm      DEVICE [1] fp32
 *   workspace DEVICE scratch of at least mlip_grad_workspace(count) bytes, aligned to 16 bytes
 */
size_t mlip_grad_workspace(int32_t count);
int mlip_grad_norm(const mlip_tensor_t *tensors, int32_t count, float *norm, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Norm as above, and dst = src * c for every element, with c = max_norm / norm where norm > max_norm and norm is finite, else
 * c = 1 (max_norm >= 0; finite: as an fp32 number).  A norm that is infinite or NaN leaves the values as they are: the caller sees it in `norm` and drops
 * the step.  c is rounded to fp32, products are fp32, rounded to the tensor's type.  A tensor that is its own output is not
 * written where c = 1.
 */
int mlip_clip_grads(const mlip_tensor_t *tensors, int32_t count, float max_norm, float *norm, void *workspace,
                    size_t workspace_bytes, void *stream);

/*
 * Networks on the nodes of a potential and their training (the models of the paper's Methods, "Graph-Parallel Message Passing", update their node features
 * by such networks): gated projections, the norms, gate and residual sum around a block, and orthogonal updates of weight matrices.
 * As the table calls they use no handle, run on the stream given and take scratch memory from the caller (aligned to 16 bytes, its contents do not matter
 * before and mean nothing after the call), so they can be captured in a HIP graph; calls that share scratch memory must not overlap in time.
 * Element pointers must be aligned to their elements; strides are in elements and not negative; outputs must not overlap inputs or each other except where said.
 * Results are the same bits on every call with the same arguments.  Sums, statistics and what lies between input and output are fp32 or more,
 * rounded to the output's type once, except where said.
 */

/*
 * Gated projections: h = phi(g, v) for every element of g = x Wg + bg, v = x Wv + bv, with phi =
 *   MLIP_GATE_SILU          silu(g) v              (silu(t) = t sigmoid(t))
 *   MLIP_GATE_GELU          g Phi(g) v             (Phi the normal distribution function)
 *   MLIP_GATE_SIGMOID       sigmoid(g) v
 *   MLIP_GATE_SILU_SIGMOID  sigmoid(g) silu(v)
 * All arrays are of type dtype; products are exact, sums fp32.  fp32 arrays: products of three bf16 parts each, all terms down to 2^-24; those that make
 * g and v where d <= 128, and of mlip_gated where n d f >= 5e8, of two fp16 parts (22 bits) of values brought by powers of two into their range row by row of x and column by column
 * of the weights, except in the rows and columns whose values differ too much in size for that, where they are products of fp32 values; what is left out or rounded is below 2^-20 of
 * the sum of the terms' sizes.  A value that is infinite, or beyond the bf16 range of 3.39e38, makes its row of x, or its column of the weights, NaN.
 *   x        DEVICE [n][d], any strides;  w_gate, w_value DEVICE [d][f], any strides (so that weights kept as [f][d] serve as well)
 *   b_gate, b_value   DEVICE [f], one element after another, or NULL
 *   out      DEVICE [n][f], element (i, k) at i * out_row_stride + k
 * 0 <= n < 2^31, 1 <= d, f <= 65536.  mlip_gated_workspace returns 0 for calls that are refused.  It asks for the weights once more (fp32: in parts) and, where they are laid out
 * first, for x, gradients also for 4 f values of 16 bits a row (fp32: 6 f) and for the weights' gradients in fp32 as many times as rows are split for them; of many rows, those of one chunk, 4 GB
 * (32,768 x 1024 -> 4096 bf16: 89 MB, its gradient 1255 MB; 1,000,188 x 64 -> 128 fp32: 0.1 MB and 2.3 GB).
 */
enum { MLIP_GATE_SILU = 0, MLIP_GATE_GELU = 1, MLIP_GATE_SIGMOID = 2, MLIP_GATE_SILU_SIGMOID = 3 };
typedef struct {
    int32_t dtype, act;
    int64_t n, d, f;
    const void *x;
    int64_t x_row_stride, x_col_stride;
    const void *w_gate;
    int64_t w_gate_row_stride, w_gate_col_stride;
    const void *w_value;
    int64_t w_value_row_stride, w_value_col_stride;
    const void *b_gate, *b_value;
} mlip_gated_t;
size_t mlip_gated_workspace(const mlip_gated_t *call, int32_t grad /* 0: of mlip_gated, 1: of mlip_gated_grad */);
int mlip_gated(const mlip_gated_t *call, void *out, int64_t out_row_stride, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Its gradient, from the gradient of out.  The products are computed again: nothing is kept from the forward call.  The gradients of g and v are rounded
 * before the products with x and the weights take them up, of 16-bit arrays to 16 bits with the range of fp32, of fp32 arrays not at all.
 *   grad     DEVICE [n][f], any strides
 *   x        DEVICE [n][d], element (i, k) at i * x_row_stride + k;  w_gate, w_value DEVICE [d][f], any strides that keep elements apart
 *   b_gate, b_value   DEVICE [f]
 * Every output may be NULL, and is then left out.
 */
typedef struct {
    const void *grad;
    int64_t grad_row_stride, grad_col_stride;
    void *x;
    int64_t x_row_stride;
    void *w_gate;
    int64_t w_gate_row_stride, w_gate_col_stride;
    void *w_value;
    int64_t w_value_row_stride, w_value_col_stride;
    void *b_gate, *b_value;
} mlip_gated_grad_t;
int mlip_gated_grad(const mlip_gated_t *call, const mlip_gated_grad_t *grad, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Residual sum of a block with its norms and gate:  y = x + factor * gate * scale * post(z),  norm = pre(y) (of y before it is rounded), where the norm
 * of a row t is  (t - m) / sqrt(mean of (t - m)^2 + eps) * w + b  with m the row's mean (MLIP_NORM_LAYER) or 0 (MLIP_NORM_RMS).
 *   x, z     DEVICE [n][width] of dtype, any strides;  z NULL: y = x, and pre(x) is all there is to compute (y NULL, no gate, scale or post)
 *   gate     DEVICE of dtype: one for each element [n][width], row [n] (column stride not used) or column [width] (row stride not used), by gate_kind
 *   scale, post_w, post_b, pre_w, pre_b   DEVICE [width] of param_dtype (fp32 or dtype), one element after another, or NULL (1, and 0 for a bias)
 *   post, pre   whether there is such a norm
 *   y, norm  DEVICE [n][width] of dtype, element (i, k) at i * row stride + k;  y may be NULL (only the norm is wanted), norm is NULL if pre is 0.
 *            y may be x itself or z itself, with the same strides.
 * 0 <= n < 2^31, 1 <= width <= 8192.
 */
enum { MLIP_NORM_RMS = 0, MLIP_NORM_LAYER = 1 };
enum { MLIP_RESIDUAL_GATE_NONE = 0, MLIP_RESIDUAL_GATE_FULL = 1, MLIP_RESIDUAL_GATE_ROW = 2, MLIP_RESIDUAL_GATE_COL = 3 };
typedef struct {
    int32_t dtype, param_dtype, kind, gate_kind, post, pre;
    int64_t n, width;
    float eps, factor;
    const void *x;
    int64_t x_row_stride, x_col_stride;
    const void *z;
    int64_t z_row_stride, z_col_stride;
    const void *gate;
    int64_t gate_row_stride, gate_col_stride;
    const void *scale, *post_w, *post_b, *pre_w, *pre_b;
} mlip_residual_t;
int mlip_residual(const mlip_residual_t *call, void *y, int64_t y_row_stride, void *norm, int64_t norm_row_stride, void *stream);

/*
 * Its gradient, from the gradients of y and of norm (either may be NULL: zeros; not both) and the inputs; y and the norms are computed again.
 *   y, norm   DEVICE [n][width] of dtype, any strides
 *   x, z, gate   outputs of dtype, element (i, k) at i * row stride + k; the gate's as the gate is: [n][width], [n] (i * row stride) or [width]
 *   scale, post_w, post_b, pre_w, pre_b   outputs [width] of param_dtype
 * Every output may be NULL; outputs of what the call does not have must be.  x may be y or norm itself, z the other one, with the same strides.
 * Sums over the rows: fp32, over fewer than n / 256 + 64 rows at a time, and those parts in fp32.
 */
typedef struct {
    const void *y;
    int64_t y_row_stride, y_col_stride;
    const void *norm;
    int64_t norm_row_stride, norm_col_stride;
    void *x;
    int64_t x_row_stride;
    void *z;
    int64_t z_row_stride;
    void *gate;
    int64_t gate_row_stride;
    void *scale, *post_w, *post_b, *pre_w, *pre_b;
} mlip_residual_grad_t;
size_t mlip_residual_grad_workspace(int64_t n, int64_t width);
int mlip_residual_grad(const mlip_residual_t *call, const mlip_residual_grad_t *grad, void *workspace, size_t workspace_bytes, void *stream);

/* A matrix of a list: element (i, k) at i * row stride + k * col stride of src, and of dst, where its result goes (dst may be src, with the same strides). */
typedef struct {
    const void *src; /* DEVICE */
    void *dst;       /* DEVICE */
    int64_t rows, cols, src_row_stride, src_col_stride, dst_row_stride, dst_col_stride;
    int32_t dtype;
} mlip_matrix_t;

/*
 * Orthogonalises the matrices of a list (gradients or their running means, before an optimiser's update): X_0 = G / max(|G|, eps) with |G| the root of the sum of
 * squares, then `steps` times X <- (a + b X X^T + c (X X^T)^2) X, of the transpose where a matrix has more rows than columns; dst = scale * X.
 * |G| is summed in fp64.  X and the products X X^T are held in two fp16 parts (22 bits), sums are fp32, for matrices of all types: results are as of fp32 arithmetic, rounded
 * to the type once.
 * Entries of X must stay below 2^11 / sqrt(columns) and those off the diagonals of the polynomials below 2^7, which coefficients hold that keep singular values
 * in [0, 1] below 1.3 (larger ones become infinite or NaN).
 * A matrix with values that are not finite gets none that is; one of zeros stays so.  The same matrix must not be in the list twice.
 *   matrices      HOST [count], read before the call returns; count, rows and cols may be 0;  rows, cols <= 2^20, the smaller one of them <= 32768, elements < 2^31
 *   coefficients  HOST [3] a, b, c
 */
size_t mlip_orthogonalise_workspace(const mlip_matrix_t *matrices, int32_t count);
int mlip_orthogonalise(const mlip_matrix_t *matrices, int32_t count, int32_t steps, const double *coefficients, double eps, float scale, void *workspace,
                       size_t workspace_bytes, void *stream);

const char *mlip_last_error(void);
const char *mlip_version(void);

#ifdef __cplusplus
}
#endif
#endif /* MLIP_H */
