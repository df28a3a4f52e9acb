/*
 * rheo.h -- C ABI of the RheoSampling hot path on AMD Instinct MI355X (gfx950).
 *
 * RheoSampling (arXiv 2609.21827) builds a speculative-decoding draft tree by
 * EAGLE's expand-then-rerank (Sec. 2.1) with one stochastic slot per candidate
 * pool: the top-m draft tokens, then one token Y sampled from the tail
 * distribution q~, then the highest-ranked remaining tokens (Sec. 3.2, "Hybrid
 * sampling mechanism"; App. C.1).  Y competes in expansion and pruning with
 * the proxy probability min{q(x_m), z} and is verified with its true
 * probability q~(Y) (Sec. 3.2, "Dual treatment").  The tree is pruned globally
 * to R nodes by path score with a fixed tie-break (App. C.1) and verified
 * layer by layer by RheoVerification (Algorithm 1; Thm. 1).
 *
 * One decoding step for B independent sequences is
 *     rheo_begin_step
 *     rheo_expand_level  x depth     (draft logits of the current frontier)
 *     rheo_prune
 *     rheo_verify                    (target logits of the pruned tree)
 * and the caller runs its draft / target model between the calls, using
 * rheo_frontier and rheo_pruned_view to learn which rows to compute.
 *
 * Conventions
 *   - All data pointers are device pointers (HBM) unless marked "host".
 *     The caller owns every logit and output buffer; the tree handle owns its
 *     own device state, sized at rheo_create.
 *   - Every call that takes a stream enqueues work on that HIP stream
 *     (hipStream_t, passed as void*; NULL = the default stream) and returns
 *     without synchronising.  A handle must not be used from two streams at
 *     once; calls on one handle must follow the step order above.
 *   - Return value: RHEO_OK or a negative error code; rheo_last_error()
 *     gives a message for the calling thread's last failure.  Arguments are
 *     validated on the host before anything is enqueued, so an error leaves
 *     the device state as it was.
 *   - Logit rows: dtype RHEO_F32 or RHEO_BF16, V contiguous elements per row,
 *     consecutive rows row_stride elements apart, base pointer 16-byte aligned
 *     and row_stride a multiple of 16 bytes.  A logit is finite or -inf (a
 *     masked token, the truncation of Sec. 3.2: probability 0).  NaN and
 *     +inf are not allowed and not checked.  Device error bit 9 (512)
 *     reports the cases where the method is undefined: a draft row whose
 *     x_{m+1} (the (m+1)-th token by construction weight, ties by id) has
 *     logit -inf, so q~_T has no reference; a target row with no finite
 *     logit (see rheo_verify).
 *   - Decisions are exact: each probability is an integer weight (a
 *     fixed-point softmax numerator evaluated by a fixed fp32 operation
 *     sequence), sums are exact 64-bit integers and every sampling or
 *     acceptance decision is an exact integer comparison, so results do not
 *     depend on launch shapes or reduction order.  Random draws are
 *     Philox4x64-10 (Salmon et al., SC'11) blocks keyed by rng_key with the
 *     counter (index, sequence, purpose, 0), purposes 1 = the sampled token
 *     of the node with uid index, 2 = acceptance test 32*level + j (j = 0 for
 *     the sampled child, else the candidate's slot), 3 = the final sample of
 *     a level.
 */
#ifndef RHEO_H
#define RHEO_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct rheo_tree rheo_tree;

enum {
    RHEO_OK = 0,
    RHEO_EINVAL = -1,   /* invalid argument or configuration             */
    RHEO_ENOMEM = -2,   /* device allocation failed                      */
    RHEO_EHIP = -3,     /* a HIP runtime call failed (message attached)  */
    RHEO_ESTATE = -4    /* call out of the step order                    */
};

enum { RHEO_F32 = 0, RHEO_BF16 = 1,
       RHEO_F16 = 2 };  /* rheo_cache_create and rheo_scorer_create alone */

enum { RHEO_METHOD_RHEO = 0, RHEO_METHOD_RRSW = 1, RHEO_METHOD_TOPK = 2 };

typedef struct rheo_config {
    int32_t batch;               /* B >= 1 independent sequences                      */
    int32_t vocab;               /* V, 2 <= V <= 262143                               */
    int32_t pool;                /* K slots per candidate pool, sampled slot included
                                    (Sec. 3.2); 1 <= K <= 15                           */
    int32_t leads;               /* m deterministic lead tokens, 0 <= m <= K-1          */
    int32_t depth;               /* D expansion levels, 1 <= D <= 15                   */
    int32_t n_expand;            /* parents expanded per level below the root,
                                    1..K (EAGLE expands K, Sec. 2.1); 0 means K         */
    int32_t support;             /* S: draft logits truncated to their top-S entries
                                    before the softmax (Sec. 3.2, sparse draft; the
                                    paper uses 128, App. B).  K <= S <= 1024.
                                    S <= 0 selects dense mode: the support is the whole
                                    vocabulary, and verification re-reads the draft
                                    rows (see rheo_expand_level)                        */
    int32_t construct_tempered;  /* 0: tree built on untempered q (Sec. 5.4);
                                    1: on the tempered q_T                              */
    int32_t dtype;               /* RHEO_F32 or RHEO_BF16                               */
    int32_t method;              /* RHEO_METHOD_RHEO: the pools of Sec. 3.2 verified by
                                    Algorithm 1 (the sampled child first);
                                    RHEO_METHOD_RRSW: the same pools verified leads
                                    first -- the leads under p, then the sampled child
                                    under what remains, then the fills under
                                    norm(max(0, r - q~)) (App. D.2);
                                    RHEO_METHOD_TOPK: pure top-K pools, no sampled
                                    slot (Sec. 2.1), sequential tests under p        */
    int32_t construct_full;      /* sparse mode: 0 builds the tree on q truncated to
                                    the support (Sec. 3.2); 1 on q over the whole
                                    vocabulary, the support then limiting only the
                                    sampled token's tail q~ and verification (the
                                    reading of Sec. 5.5 that truncation touches only
                                    the sampled token).  Costs one extra read of each
                                    draft row.  0 or 1; no effect in dense mode     */
    int64_t row_stride;          /* elements between consecutive logit rows (>= V)     */
    double eps_m0;               /* epsilon of the m = 0 proxy q(x_1) + eps (Sec. 3.2);
                                    0 selects 2^-40                                     */
} rheo_config;

/* Allocates a tree for cfg (host pointer, copied).  *out receives the handle.
 * Node capacity per sequence: 1 + K + (D-1) * n_expand * K.
 * Launch shapes, read from the environment here and never changing a
 * result: RHEO_EXPAND_ROW (0: levels on the chunked kernels, 1: on the
 * one-block-per-row kernels wherever the row fits them; dense fp32 levels are
 * always chunked), RHEO_ROW_MIN (fewest rows of a sparse level for the per-row
 * kernel, default 1),
 * RHEO_ROW_NARROW (1 or 0: the per-row kernel's 256-thread blocks always or
 * never; by default when a level has more rows than the device holds
 * 512-thread blocks at once), RHEO_EXPAND_VARIANT (chunk size of the
 * chunked kernels), RHEO_VERIFY_BLOCKS (blocks of all verification teams,
 * default 1024 and at most 32 a team with at least two chunks a wave; capped
 * by what the device holds at once).  RHEO_VERIFY_SPIN,
 * read at each rheo_verify, sets the polls of a team wait before it gives up
 * (see rheo_verify). */
int rheo_create(const rheo_config* cfg, rheo_tree** out);

/* rheo_create for callers that cannot allocate device memory (serving loops
 * and harnesses that forbid hipMalloc): the tree's whole device state lives
 * in a static array of the library, 44 MiB per device, which every device
 * that loads the library holds until the process ends.  No device memory is
 * allocated or freed.  A configuration whose state (64 bytes a node, the
 * tails, the selection and verification scratch) exceeds 32 MiB returns
 * RHEO_EINVAL before any device call (the five workload shapes of the
 * sparse and dense modes fit; supports of 512 and more at large batches do
 * not).  There is one static tree per device (the current device): every
 * call on a device re-initialises it and returns the same handle in *out, so
 * a static tree from an earlier call on that device becomes this one.
 * Calls on one device that overlap -- two threads creating, or work still
 * using the earlier static tree -- race.  The call synchronises the device
 * (not for use under graph capture); the handle's other calls behave as for
 * rheo_create, and rheo_destroy on it only synchronises. */
int rheo_create_static(const rheo_config* cfg, rheo_tree** out);

/* Frees the handle and its device memory (synchronises the device); for the
 * handle of rheo_create_static it frees nothing. */
int rheo_destroy(rheo_tree* tree);

/* Starts a new step: the next rheo_expand_level builds level 0 from the root. */
int rheo_begin_step(rheo_tree* tree);

/* Expands the current frontier by one level (Sec. 2.1 with the pools of
 * Sec. 3.2 / App. C.1).
 *   draft_logits  [B][P][row_stride] of cfg.dtype, P = 1 at level 0 (the
 *                 root) and n_expand afterwards; row (b, j) holds the draft
 *                 model's logits at frontier node j of sequence b.
 *   T             sampling temperature (> 0, finite): Y ~ q~_T.
 *   rng_key       key of the step's Philox draws.
 * T and rng_key are fixed for the whole step: the first call of a step sets
 * them, and a later rheo_expand_level or the step's rheo_verify with another
 * value returns RHEO_EINVAL (the stored tail weights and the draws of the
 * sampled slots depend on both).
 * Writes K children per frontier node (token, proxy, true probability,
 * path score) and, below the last level, selects the n_expand children with
 * the highest path scores as the next frontier.  With support S, the
 * truncated distribution is kept in the tree for verification, so the
 * draft buffer may be reused as soon as this call's work has run.  In dense
 * mode the tree borrows draft_logits: verification re-reads the rows of the
 * nodes it walks, so the buffer of every level must stay allocated and
 * unchanged until the step's rheo_verify has run on its stream. */
int rheo_expand_level(rheo_tree* tree, const void* draft_logits, float T,
                      uint64_t rng_key, void* stream);

/* The frontier chosen by the last rheo_expand_level, in rank order, copied
 * into caller buffers on `stream`:
 *   parent_index  [B][n_expand] int32: index of the node's parent in the
 *                 previous frontier (0 at level 1)
 *   token         [B][n_expand] int32: the node's token
 * (device pointers; either may be NULL).  Valid below the last level.
 * RHEO_ESTATE if no level below the last has been expanded in this step. */
int rheo_frontier(rheo_tree* tree, int32_t* parent_index, int32_t* token,
                  void* stream);

/* The same frontier without a copy: *parent_index and *token receive the
 * tree-owned device arrays ([B][n_expand] int32 each, layout as above).  The
 * pointers stay fixed for the life of the handle; their contents are those
 * of the last rheo_expand_level below the last level, once that call's
 * work has run on its stream, until the next such call.  Host-only: no
 * device work, no synchronisation. */
int rheo_frontier_view(const rheo_tree* tree, const int32_t** parent_index,
                       const int32_t** token);

/* Keeps the budget R best non-root nodes (1 <= R <= K + (D-1) n_expand K) by
 * path score, ties by depth (shallower first) then left-to-right sibling
 * order (App. C.1); the root does not count towards R. */
int rheo_prune(rheo_tree* tree, int32_t budget, void* stream);

/* The pruned tree in rank order, index 0 = root:
 *   parent  [B][R+1] int32 (pruned index of the parent, -1 for the root and
 *           where device error bit 1 reports a kept node's parent as pruned)
 *   token   [B][R+1] int32 (-1 for the root)
 * Row i of the target buffer given to rheo_verify must hold the target
 * model's logits at pruned node i. */
int rheo_pruned_view(rheo_tree* tree, int32_t* parent, int32_t* token,
                     void* stream);

/* What the target model needs to score the pruned tree in one forward
 * pass, all drafted paths at once (Sec. 1; Sec. 2.1), in pruned order.
 * Valid after rheo_prune.  Either pointer may be NULL.
 *   mask   [B][R+1][R+1] uint8: mask[b][i][j] = 1 iff pruned node j is on
 *          the path from the root to pruned node i (i included), else 0.
 *          Parents precede their children in pruned order, so the mask is
 *          lower triangular.
 *   depth  [B][R+1] int32: depth of each pruned node (root 0), its
 *          position after the prefix.
 * Buffers are the caller's, written completely. */
int rheo_tree_mask(rheo_tree* tree, uint8_t* mask, int32_t* depth, void* stream);

/* RheoVerification (Algorithm 1) applied layer by layer from the root
 * (Thm. 1), with p = softmax(target / T) over the whole vocabulary.
 *   target_logits [B][R+1][row_stride] of cfg.dtype (pruned-node order)
 *   accepted      [B][depth] int32: accepted draft tokens, -1 after the end
 *   accept_len    [B] int32: number of accepted draft tokens
 *   final_token   [B] int32: the token emitted after them (residual sample,
 *                 or a sample of p below an accepted leaf)
 * The output of a step is accepted[0..accept_len) followed by final_token.
 * T and rng_key must be the step's (see rheo_expand_level), else RHEO_EINVAL.
 * The kernel's blocks wait for each other (teams of blocks per sequence);
 * its grid never exceeds what the device holds at once, so on a device that
 * runs nothing else at the same time every wait completes.  Work running
 * concurrently on the same device can delay some blocks: a wait longer than
 * about a second then ends that sequence's walk with the failure result
 * accept_len[b] = final_token[b] = -1 and accepted[b][*] = -1, and sets
 * device error bit 7 (128).  Callers check accept_len >= 0; a failed
 * sequence's step is not Algorithm 1's and must be run again.  A walk that
 * reaches a node whose target row has no finite logit (p undefined) ends
 * with the same failure result and sets device error bit 9 (512). */
int rheo_verify(rheo_tree* tree, const void* target_logits, float T,
                uint64_t rng_key, int32_t* accepted, int32_t* accept_len,
                int32_t* final_token, void* stream);

/* Copies the unpruned tree of the current step (uid order, [B][N], N =
 * 1 + K + (D-1) n_expand K, uid 0 = root; children of a level are numbered
 * in frontier order, then slot order).  Any pointer may be NULL.
 *   kind: 0 lead, 1 sampled, 2 fill; qtrue: q~(Y) for the sampled slot,
 *   q(x) for the others; score: product of proxies from the root. */
int rheo_read_nodes(rheo_tree* tree, int32_t* token, int32_t* parent,
                    int32_t* depth, int32_t* slot, int32_t* kind,
                    double* proxy, double* qtrue, double* score, void* stream);

/* Synchronises the device and copies the tree's sticky device error flag to
 * *host_flag (0 = no error; bit 0: no sampled token found, bit 1: pruned
 * tree not ancestor-closed, bit 2: sampled child missing from its parent's
 * tail, bit 3: residual sample out of range, bit 4: corrupt frontier,
 * bit 5: corrupt verification walk, bit 6: invalid launch shape, bit 7:
 * verification team barrier timed out, bit 8: a support slot left empty by
 * the expand merge, bit 9: a draft row whose x_{m+1} is -inf or a target
 * row without a finite logit).
 * Diagnostic only. */
int rheo_device_error(rheo_tree* tree, int32_t* host_flag);

/* Nodes per sequence of the unpruned tree (root included). */
int32_t rheo_node_count(const rheo_tree* tree);

/* ---------------------------------------------------------------------------
 * The key/value cache around a drafted tree
 *
 * The target forward that scores a pruned tree attends from every pruned node
 * to the tokens before the tree (the prefix) and to the node's ancestors
 * (rheo_tree_mask).  Keys and values lie in pages:
 *   k_cache, v_cache  [layers][pages][page_size][kv_heads][head_dim]
 * of cfg.dtype, page_stride elements between pages and layer_stride between
 * layers.  A slot is page * page_size + place in the page.  Sequence b holds
 * held[b] pages, named in order by its row of the block table
 *   table             [B][table_width] int32
 * and entry e of the sequence lies in slot
 * table[b][e / page_size] * page_size + e % page_size.  lens[b] entries are
 * the prefix; the rows of one step (the pruned tree, root first, or any
 * other rows) are the entries lens[b] + i behind it.  One step is
 *     rheo_cache_plan        pages and slots for the rows of the step; its status
 *     per layer: rheo_cache_write, rheo_tree_attention (of the served)
 *     (rheo_verify)
 *     rheo_cache_commit_served   the accepted path moved together, lens advanced
 *     rheo_token_logprobs    (of what was emitted, where asked for)
 * The caller owns the pages, tables and lengths; the handle owns workspace
 * and an error flag.  The conventions above hold: device pointers,
 * work enqueued on `stream` (of the handle's device, whichever is current),
 * no synchronisation, nothing allocated after creation (so every call may be
 * captured into a graph), one handle on one stream at a time (two graphs that
 * share a handle must not run at once).  Strides are in elements; tensor
 * pointers and strides are multiples of 16 bytes unless noted.
 * Lengths, tables, slots and tokens are data that the host cannot check: a
 * value out of range sets a bit of the error flag (rheo_cache_error) and
 * never reads or writes outside the arrays as declared by the arguments.
 * A call takes up to B * n = 2^30 rows, rheo_cache_write up to 2^26 - 4.
 * n = 0 rows: rheo_cache_write and rheo_tree_attention do nothing.
 * A sequence that rheo_cache_plan could not serve (status not 0) has no place for
 * its rows: its row of the table still names pages behind those that it holds, and
 * they may be another sequence's by now.  rheo_cache_write leaves it out by its
 * slots of -1; rheo_tree_attention (`status` of its arguments) and the commit
 * (rheo_cache_commit_served) have to be given the plan's status, or a count of
 * 0 and an accept_len below 0, and rheo_token_logprobs the commit's path.  Then
 * nothing of it changes in the step, and its rows of q_out and out are left as they
 * were (of a new buffer: anything; rheo_verify wants logits that are no NaN).
 * ------------------------------------------------------------------------ */

typedef struct rheo_cache rheo_cache;

typedef struct rheo_cache_config {
    int32_t batch;               /* B, 1..4096 sequences                              */
    int32_t heads;               /* query heads, a multiple of kv_heads, <= 1024         */
    int32_t kv_heads;            /* key/value heads, >= 1                               */
    int32_t head_dim;            /* a multiple of 8, 8..256                             */
    int32_t page_size;           /* entries of a page: a power of two, 1..4096           */
    int32_t pages;               /* pages of the pool, >= 1                             */
    int32_t table_width;         /* pages a sequence may hold, >= 1; table_width *
                                    page_size <= 2^30                                 */
    int32_t layers;              /* layers one rheo_cache_commit moves, 1..1024          */
    int32_t dtype;               /* RHEO_BF16 or RHEO_F16                               */
    int64_t page_stride;         /* >= page_size * kv_heads * head_dim; 0: equal to it;
                                    pages * page_stride <= 2^48                       */
    int64_t layer_stride;        /* >= pages * page_stride; 0: equal to it               */
} rheo_cache_config;

/* Allocates the workspace (of the current device, which becomes the handle's):
 * some 70 MB, most of it partial results of rheo_tree_attention. */
int rheo_cache_create(const rheo_cache_config* cfg, rheo_cache** out);
/* Frees it (synchronises the device). */
int rheo_cache_destroy(rheo_cache* cache);

/* Synchronises the handle's device and reads its sticky error flag: bit 0:
 * lens, count, held, free_count or the free list out of range in
 * rheo_cache_plan, count in rheo_tree_attention; bit 1: a slot >= pages *
 * page_size; bit 2: a position outside the rotation table; bit 3: a page
 * outside the pool; bit 4: an accepted token that is no child, at a higher
 * index, of the node before it; bit 5: entries past the table's row. */
int rheo_cache_error(rheo_cache* cache, int32_t* host_flag);

/* Pages and slots for the next rows of every sequence.
 * Sequence b needs ceil((lens[b] + count[b]) / page_size) pages (count NULL:
 * n rows each).  Pages it holds beyond that go back to the free list, pages it
 * lacks come from it; so a call with n = 0 after a step returns what the
 * step no longer needs, and with lens[b] = 0 all of a finished sequence.
 *   lens, count  [B] int32 in; 0 <= count[b] <= n
 *   depth        [B][n] int32 in, or NULL: i for row i
 *   held         [B] int32 in/out
 *   table        [B][table_width] int32 in/out; places at and past held[b]
 *                are not read, and not written but by a page that comes
 *   free_list    [pages] int32 in/out, a stack, its top at free_count - 1
 *   free_count   [1] int32 in/out
 *   slots        [B][n] int64 out: of entry lens[b] + i, -1 for i >= count[b]
 *   positions    [B][n] int32 out: lens[b] + depth[b][i], -1 for i >= count[b]
 *   status       [B] int32 out: 0 served; 1 the free pages do not reach; 2 the
 *                sequence would not fit its row of the table (or bit 0 above).
 *                With 1 or 2 the sequence keeps what it has and its slots and
 *                positions are -1.
 * Order: returned pages are pushed first, the last page of the last sequence
 * before all others; then pages are popped for one sequence after another.
 * A sequence is served iff it lacks none, or the pages lacked by it and by
 * those before it (served or not) are there.  n = 0: slots, positions and
 * depth may be NULL. */
int rheo_cache_plan(rheo_cache* cache, int32_t n, const int32_t* lens, const int32_t* count,
                    const int32_t* depth, int32_t* held, int32_t* table, int32_t* free_list,
                    int32_t* free_count, int64_t* slots, int32_t* positions, int32_t* status,
                    void* stream);

typedef struct rheo_write_args {
    int32_t n;                   /* rows of a sequence; row (b, i) is row b * n + i       */
    int32_t rot_dim;             /* leading elements of a head that are rotated, even,
                                    0..head_dim                                       */
    int32_t max_position;        /* rows of `rotation`                                  */
    int32_t interleaved;         /* pairs (2j, 2j+1) instead of (j, j + rot_dim / 2)     */
    const void* q;               /* [B * n] rows of [heads][head_dim]; or NULL: keys and
                                    values alone                                      */
    const void* k;               /* [B * n] rows of [kv_heads][head_dim]                */
    const void* v;
    void* q_out;                 /* as q; may be q itself with q's stride               */
    int64_t q_stride, k_stride, v_stride, q_out_stride;   /* between rows               */
    const int64_t* slots;        /* [B * n]; a row of slot < 0 is left out whole         */
    const int32_t* positions;    /* [B * n] int32, or NULL with rot_dim 0               */
    const float* rotation;       /* [max_position][rot_dim]: cosines, then sines         */
    const void* q_weight;        /* [head_dim] of cfg.dtype, or NULL: no norm            */
    const void* k_weight;
    float eps;                   /* of the norms, >= 0                                  */
    void* k_cache;               /* one layer's pages                                  */
    void* v_cache;
} rheo_write_args;

/* Norm, rotation and store in one pass: each head of q and k is divided by the
 * root of its mean square plus eps and multiplied by its weight, its first
 * rot_dim elements are rotated by the row of `rotation` at the row's
 * position ((a, b) -> (a cos - b sin, b cos + a sin)); q goes to q_out, k
 * and v to the row's slot.  fp32 inside, one rounding at the end.  Slots of one
 * call are distinct (else which row stays is undefined); q, k and v do not
 * overlap the pages, and q_out, unless it is q, none of them. */
int rheo_cache_write(rheo_cache* cache, const rheo_write_args* args, void* stream);

typedef struct rheo_attention_args {
    int32_t n;                   /* query rows of a sequence; row (b, i) is row b * n + i */
    int32_t tail;                /* entries behind the prefix, >= n or with a mask any   */
    const void* q;               /* [B * n] rows of [heads][head_dim]                   */
    int64_t q_stride, out_stride;/* between rows                                        */
    const void* k_cache;         /* one layer's pages                                  */
    const void* v_cache;
    const int32_t* table;        /* [B][table_width]                                    */
    const int32_t* lens;         /* [B] entries of the prefix                            */
    const int32_t* count;        /* [B] or NULL: the first count[b] of the n rows are
                                    there and the first tail - (n - count[b]) entries
                                    behind the prefix                                 */
    const uint8_t* mask;         /* [B][n][tail], row i attends entry lens[b] + j iff
                                    not 0; NULL: iff j <= i + tail - n                  */
    float scale;                 /* 2^-100..2^100                                       */
    void* out;                   /* as q; overlaps neither q nor the pages               */
    float* lse;                  /* [B * n][heads] or NULL: log of the sum of
                                    exp(scale q.k) over what the row attends            */
    const int32_t* status;       /* [B] as rheo_cache_plan wrote it, or NULL: a sequence of
                                    status not 0 is left out, as with a count of 0      */
} rheo_attention_args;

/* Attention of the step's rows over the pages: softmax(scale q.k) v over the
 * whole prefix and the entries behind it that the mask names.  Query head h
 * reads key/value head h / (heads / kv_heads).  fp32 scores, sums and
 * accumulators; the probabilities enter the second product in cfg.dtype.  A row
 * that attends nothing gives 0 and lse -inf.  Rows i >= count[b] are left as
 * they were.  What a row does not attend has no effect on it, whatever it
 * holds; keys that it does attend are finite (else its output may be NaN). */
int rheo_tree_attention(rheo_cache* cache, const rheo_attention_args* args, void* stream);

/* Keeps the accepted path of a verified tree: with parent and token [B][n] as
 * rheo_pruned_view gives them (n = R + 1) and accepted [B][depth] and
 * accept_len [B] as rheo_verify does, the entries of the root and of the
 * accepted nodes are moved in every layer, keys and values, from lens[b] +
 * pruned index to lens[b] + 0, 1, 2, ...; the entries between are then free.
 *   path      [B][depth + 1] int32 out: pruned indices of the root and the
 *             accepted nodes, -1 past the end (what rheo_token_logprobs takes)
 *   new_lens  [B] int32 out: lens[b] + 1 + accept_len[b]; may be lens itself
 * A sequence with accept_len < 0 (a failed walk), or one that sets an error
 * bit, keeps its entries and length; its path is all -1. */
int rheo_cache_commit(rheo_cache* cache, int32_t n, int32_t depth, const int32_t* parent,
                      const int32_t* token, const int32_t* accepted, const int32_t* accept_len,
                      const int32_t* lens, const int32_t* table, void* k_cache, void* v_cache,
                      int32_t* path, int32_t* new_lens, void* stream);
/* The same for the sequences that rheo_cache_plan served: one of status [B] not 0
 * is treated as one of accept_len < 0, whatever its accept_len.  status NULL: as
 * rheo_cache_commit. */
int rheo_cache_commit_served(rheo_cache* cache, int32_t n, int32_t depth, const int32_t* parent,
                             const int32_t* token, const int32_t* accepted,
                             const int32_t* accept_len, const int32_t* lens, const int32_t* table,
                             const int32_t* status, void* k_cache, void* v_cache, int32_t* path,
                             int32_t* new_lens, void* stream);

/* ---------------------------------------------------------------------------
 * Log probabilities of given tokens
 * ------------------------------------------------------------------------ */

typedef struct rheo_scorer rheo_scorer;

/* A scorer of logit rows of `vocab` elements (2 <= vocab <= 2^24), row_stride
 * elements apart (conventions as for logit rows above; RHEO_F32, RHEO_BF16 or
 * RHEO_F16).  It owns a workspace of fixed size; creation synchronises the
 * device. */
int rheo_scorer_create(int32_t vocab, int32_t dtype, int64_t row_stride, rheo_scorer** out);
int rheo_scorer_destroy(rheo_scorer* scorer);

/* For the token of every entry (b, j), fewer than 2^24 in all, p = softmax(row / T):
 *   logits       [B][n][row_stride]
 *   path         [B][m] int32: the entry's row of the sequence's n, or NULL: row j
 *                (m <= n)
 *   token        [B][m] int32
 *   logprob      [B][m] float out: ln p of the token
 *   entropy      [B][m] float out: -sum p ln p
 *   rank         [B][m] int32 out: tokens that precede it by (logit descending,
 *                id ascending)
 *   top_token    [B][m][top] int32 out, top_logprob [B][m][top] float out: the
 *                first `top` tokens of that order, 0 <= top <= 32 and <= vocab
 * entropy, rank and, with top = 0, the last two may be NULL.  Entries whose
 * path lies outside [0, n) or whose token lies outside [0, vocab) are left as
 * they were.  -inf is a token of probability 0; a row without a finite logit
 * has no distribution: NaN. */
int rheo_token_logprobs(rheo_scorer* scorer, const void* logits, int32_t B, int32_t n,
                        const int32_t* path, const int32_t* token, int32_t m, int32_t top,
                        float T, float* logprob, float* entropy, int32_t* rank,
                        int32_t* top_token, float* top_logprob, void* stream);

/* Message of the calling thread's last failed call ("" if none). */
const char* rheo_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* RHEO_H */
