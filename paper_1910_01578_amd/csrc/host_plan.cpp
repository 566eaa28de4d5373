// Host-only argument checks, workspace planning and the graph validator.
#include "host_plan.h"

#include <float.h>
#include <limits.h>
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <algorithm>
#include <vector>

namespace gdp {

namespace {
thread_local char g_err[512] = "";
}

int fail(int code, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof(g_err), fmt, ap);
  va_end(ap);
  return code;
}

void clear_error() { g_err[0] = '\0'; }

size_t elem_size(int32_t dtype) { return dtype == GDP_BF16 ? 2 : 4; }

static bool supported_width(int h) { return h == 64 || h == 128 || h == 256; }

static bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

int check_graph(const gdp_graph* g) {
  if (!g) return fail(GDP_E_INVALID_ARG, "graph is NULL");
  if (g->n_graphs < 1) return fail(GDP_E_INVALID_ARG, "n_graphs = %d < 1", g->n_graphs);
  if (g->n_graphs > GDP_MAX_GRAPHS)
    return fail(GDP_E_UNSUPPORTED, "n_graphs = %d exceeds GDP_MAX_GRAPHS = %d", g->n_graphs, GDP_MAX_GRAPHS);
  if (!g->graph_ptr_h) return fail(GDP_E_INVALID_ARG, "graph_ptr_h is NULL");
  if (g->n_nodes < 1) return fail(GDP_E_INVALID_ARG, "n_nodes = %d < 1", g->n_nodes);
  if (g->graph_ptr_h[0] != 0) return fail(GDP_E_BAD_GRAPH, "graph_ptr_h[0] = %d, expected 0", g->graph_ptr_h[0]);
  for (int i = 0; i < g->n_graphs; ++i)
    if (g->graph_ptr_h[i + 1] <= g->graph_ptr_h[i])
      return fail(GDP_E_BAD_GRAPH, "graph %d is empty or graph_ptr_h decreases", i);
  if (g->graph_ptr_h[g->n_graphs] != g->n_nodes)
    return fail(GDP_E_BAD_GRAPH, "graph_ptr_h[G] = %d != n_nodes = %d", g->graph_ptr_h[g->n_graphs], g->n_nodes);
  if (g->n_edges < 0 || g->n_edges > INT32_MAX)
    return fail(GDP_E_INVALID_ARG, "n_edges = %lld out of range", (long long)g->n_edges);
  if (!g->row_ptr || !g->x) return fail(GDP_E_INVALID_ARG, "row_ptr or x is NULL");
  if (g->n_edges > 0 && !g->col_idx) return fail(GDP_E_INVALID_ARG, "col_idx is NULL");
  if (g->dtype != GDP_F32 && g->dtype != GDP_BF16) return fail(GDP_E_INVALID_ARG, "dtype = %d", g->dtype);
  if (g->feat_dim < 32 || g->feat_dim % 32 != 0)
    return fail(GDP_E_UNSUPPORTED, "feat_dim = %d must be a positive multiple of 32", g->feat_dim);
  if (g->flags & ~GDP_TOPO_IDS) return fail(GDP_E_INVALID_ARG, "unknown flags 0x%x", g->flags);
  return GDP_OK;
}

int check_gnn(const gdp_graph* g, const gdp_gnn* n) {
  if (!n) return fail(GDP_E_INVALID_ARG, "gnn is NULL");
  if (n->n_layers < 1) return fail(GDP_E_INVALID_ARG, "gnn.n_layers = %d < 1", n->n_layers);
  if (n->in_dim != g->feat_dim)
    return fail(GDP_E_INVALID_ARG, "gnn.in_dim = %d != feat_dim = %d", n->in_dim, g->feat_dim);
  if (!supported_width(n->hidden)) return fail(GDP_E_UNSUPPORTED, "gnn.hidden = %d not in {64,128,256}", n->hidden);
  if (n->fanout < 1 || n->fanout > GDP_MAX_FANOUT)
    return fail(GDP_E_UNSUPPORTED, "fanout = %d outside 1..%d", n->fanout, GDP_MAX_FANOUT);
  if (!n->layers) return fail(GDP_E_INVALID_ARG, "gnn.layers is NULL");
  for (int l = 0; l < n->n_layers; ++l) {
    const gdp_gnn_layer& L = n->layers[l];
    if (!L.w_pool || !L.b_pool || !L.w_self || !L.w_neigh || !L.b_upd)
      return fail(GDP_E_INVALID_ARG, "gnn layer %d has a NULL weight", l);
  }
  return GDP_OK;
}

int check_placer(const gdp_graph* g, const gdp_placer* p) {
  if (!p) return fail(GDP_E_INVALID_ARG, "placer is NULL");
  if (p->n_layers < 1) return fail(GDP_E_INVALID_ARG, "placer.n_layers = %d < 1", p->n_layers);
  if (!supported_width(p->d_model)) return fail(GDP_E_UNSUPPORTED, "d_model = %d not in {64,128,256}", p->d_model);
  if (p->attention != 0 && p->attention != 1)
    return fail(GDP_E_INVALID_ARG, "attention = %d must be 0 or 1", p->attention);
  if (p->attention) {
    if (p->n_heads < 1 || p->d_model % p->n_heads != 0)
      return fail(GDP_E_INVALID_ARG, "d_model = %d not divisible by n_heads = %d", p->d_model, p->n_heads);
    const int dh = p->d_model / p->n_heads;
    if (dh != 16 && dh != 32 && dh != 64) return fail(GDP_E_UNSUPPORTED, "head dim %d not in {16,32,64}", dh);
    if (p->seg_len < 1) return fail(GDP_E_INVALID_ARG, "seg_len = %d < 1", p->seg_len);
    if (p->mem_len < 0) return fail(GDP_E_INVALID_ARG, "mem_len = %d < 0", p->mem_len);
  } else if (p->n_layers > 16) {
    return fail(GDP_E_UNSUPPORTED, "n_layers = %d > 16 without attention", p->n_layers);
  }
  if (p->d_ff < 128 || p->d_ff % 128 != 0)
    return fail(GDP_E_UNSUPPORTED, "d_ff = %d must be a positive multiple of 128", p->d_ff);
  if (p->n_devices < 2 || p->n_devices > GDP_MAX_DEVICES)
    return fail(GDP_E_UNSUPPORTED, "n_devices = %d outside 2..%d", p->n_devices, GDP_MAX_DEVICES);
  if (p->film != 0 && p->film != 1) return fail(GDP_E_INVALID_ARG, "film = %d must be 0 or 1", p->film);
  if (!p->layers || !p->w_out || !p->b_out) return fail(GDP_E_INVALID_ARG, "placer weights are NULL");
  for (int l = 0; l < p->n_layers; ++l) {
    const gdp_placer_layer& L = p->layers[l];
    if (!L.w_1 || !L.b_1 || !L.w_2 || !L.b_2 || !L.ln2_g || !L.ln2_b ||
        (p->attention && (!L.w_qkv || !L.b_qkv || !L.w_o || !L.b_o || !L.ln1_g || !L.ln1_b)))
      return fail(GDP_E_INVALID_ARG, "placer layer %d has a NULL weight", l);
    if (p->film && (!L.film_wg || !L.film_bg || !L.film_wb || !L.film_bb))
      return fail(GDP_E_INVALID_ARG, "placer layer %d has a NULL FiLM weight", l);
    // The layer kernels stage these matrices and vectors by 16-byte loads.
    if (!aligned16(L.w_1) || !aligned16(L.b_1) || !aligned16(L.w_2) ||
        (p->attention && (!aligned16(L.w_qkv) || !aligned16(L.b_qkv) || !aligned16(L.w_o))))
      return fail(GDP_E_INVALID_ARG, "placer layer %d: w_qkv, b_qkv, w_o, w_1, b_1 and w_2 must be 16-byte aligned", l);
  }
  (void)g;
  return GDP_OK;
}

int check_sample(const gdp_graph* g, int32_t n_devices, int32_t k_samples) {
  (void)g;
  if (n_devices < 2 || n_devices > GDP_MAX_DEVICES)
    return fail(GDP_E_UNSUPPORTED, "n_devices = %d outside 2..%d", n_devices, GDP_MAX_DEVICES);
  if (k_samples < 1) return fail(GDP_E_INVALID_ARG, "k_samples = %d < 1", k_samples);
  if (k_samples > 65535) return fail(GDP_E_UNSUPPORTED, "k_samples = %d > 65535", k_samples);
  return GDP_OK;
}

void carve_init(Carve* c) {
  c->total = 0;
  c->n = 0;
}

size_t carve_add(Carve* c, size_t bytes) {
  const size_t off = c->total;
  c->total += (bytes + 255) & ~size_t(255);
  if (c->n < 24) c->off[c->n++] = off;
  return off;
}

int prefix_blocks_rows(const int32_t* gp, int G, int rows, int32_t* blk) {
  blk[0] = 0;
  for (int g = 0; g < G; ++g) blk[g + 1] = blk[g] + (gp[g + 1] - gp[g] + rows - 1) / rows;
  return blk[G];
}

int blocks_below(const int32_t* gp, int G, int rows, int R, int* started) {
  int n = 0, s = 0;
  for (int g = 0; g < G; ++g) {
    if (gp[g + 1] <= R) {
      n += (gp[g + 1] - gp[g] + rows - 1) / rows;
      s = n;
    } else {
      if (gp[g] < R) {
        n += (R - gp[g]) / rows;                // block b ends at gp[g] + (b + 1) rows <= R
        s = n + ((R - gp[g]) % rows != 0);      // a block starts below R and ends above it
      } else {
        s = n;
      }
      break;
    }
  }
  if (started) *started = s;
  return n;
}

int segment_len(const gdp_graph* g, const gdp_placer* p) {
  constexpr int kMost = 1 << 30;
  return g->n_nodes <= kMost && p->seg_len > kMost ? kMost : p->seg_len;
}

int prefix_blocks_attention(const int32_t* gp, int G, int seg_len, int bq, int32_t* blk) {
  const int qbs = (seg_len + bq - 1) / bq;
  blk[0] = 0;
  for (int g = 0; g < G; ++g) {
    const int n = gp[g + 1] - gp[g];
    const int nseg = (n + seg_len - 1) / seg_len;
    const int last = n - (nseg - 1) * seg_len;
    blk[g + 1] = blk[g] + (nseg - 1) * qbs + (last + bq - 1) / bq;
  }
  return blk[G];
}

int segment_split(const int32_t* gp, int G, int seg_len, int bq, int target, int* qblocks_below) {
  const int qbs = (seg_len + bq - 1) / bq;
  const int N = gp[G];
  int best = 0, best_q = 0;
  long best_dist = -1;
  int qb = 0;   // query blocks of the graphs before g
  for (int g = 0; g < G; ++g) {
    const int n = gp[g + 1] - gp[g];
    const int nseg = (n + seg_len - 1) / seg_len;
    for (int k = 0; k < nseg; ++k) {
      const int b = gp[g] + k * seg_len;
      if (b <= 0 || b >= N) continue;
      const long dist = b > target ? (long)b - target : (long)target - b;
      if (best_dist < 0 || dist < best_dist) {
        best = b;
        best_q = qb + k * qbs;
        best_dist = dist;
      }
    }
    if (nseg > 0) qb += (nseg - 1) * qbs + (n - (nseg - 1) * seg_len + bq - 1) / bq;
  }
  *qblocks_below = best_q;
  return best;
}

void plan_embed(const gdp_graph* g, const gdp_gnn* gnn, EmbedPlan* p) {
  const size_t N = (size_t)g->n_nodes, E = (size_t)g->n_edges, H = (size_t)gnn->hidden;
  const size_t es = elem_size(g->dtype);
  int32_t blk[GDP_MAX_GRAPHS + 1];
  p->pool_chunks = prefix_blocks_rows(g->graph_ptr_h, g->n_graphs, kPoolRows, blk);
  const size_t cap_a = 2 * E, cap_b = N * (size_t)gnn->fanout;
  p->s_cap = (int64_t)(cap_a < cap_b ? cap_a : cap_b);
  carve_init(&p->c);
  p->counters = carve_add(&p->c, (2 * N + 1) * 4);
  p->scan_tmp = carve_add(&p->c, 2 * ((N + 1023) / 1024) * 4);
  p->heavy = carve_add(&p->c, N * 4);
  p->in_ptr = carve_add(&p->c, (N + 1) * 4);
  p->in_idx = carve_add(&p->c, (E > 0 ? E : 1) * 4);
  p->s_ptr = carve_add(&p->c, (N + 1) * 4);
  p->s_idx = carve_add(&p->c, (p->s_cap > 0 ? (size_t)p->s_cap : 1) * 4);
  p->P = carve_add(&p->c, N * H * es);
  p->A = carve_add(&p->c, N * H * es);
  p->h0 = carve_add(&p->c, gnn->n_layers > 1 ? N * H * es : 0);
  p->h1 = carve_add(&p->c, gnn->n_layers > 2 ? N * H * es : 0);
  p->pool = carve_add(&p->c, (size_t)p->pool_chunks * H * 4);
}

void plan_place(const gdp_graph* g, const gdp_placer* pl, PlacePlan* p) {
  const size_t N = (size_t)g->n_nodes, d = (size_t)pl->d_model, es = elem_size(g->dtype);
  int32_t blk[GDP_MAX_GRAPHS + 1];
  carve_init(&p->c);
  p->film = carve_add(&p->c, (size_t)pl->n_layers * g->n_graphs * d * 2 * 4);
  p->y0 = carve_add(&p->c, N * d * 4);      // residual stream: fp32
  p->head_partial = carve_add(&p->c, ((N + kHeadBwdRows - 1) / kHeadBwdRows) * (size_t)pl->n_devices * (d + 1) * 4);
  p->split = p->split_qblocks = 0;
  if (!pl->attention) {                     // only the head's input, when the head runs on its own
    p->qblocks = 0;
    p->y1 = p->qkv = p->qkv2 = p->o = p->y0;
    return;
  }
  p->qblocks = prefix_blocks_attention(g->graph_ptr_h, g->n_graphs, segment_len(g, pl), kAttnQ, blk);
  p->y1 = carve_add(&p->c, N * d * 4);
  p->qkv = carve_add(&p->c, N * 3 * d * es);
  p->o = carve_add(&p->c, N * d * es);
  // Two parts only where part B still fills a round of its own (and a
  // layer is long enough that the overlap outweighs the extra launches).
  if (N >= (size_t)kSplitRows + kSplitRows / 4)
    p->split = segment_split(g->graph_ptr_h, g->n_graphs, segment_len(g, pl), kAttnQ, kSplitRows, &p->split_qblocks);
  p->qkv2 = p->split > 0 ? carve_add(&p->c, N * 3 * d * es) : p->qkv;
}

static int longest_graph(const gdp_graph* g) {
  int longest = 0;
  for (int i = 0; i < g->n_graphs; ++i) {
    const int n = g->graph_ptr_h[i + 1] - g->graph_ptr_h[i];
    if (n > longest) longest = n;
  }
  return longest;
}

bool eval_by_lanes(const gdp_graph* g, int32_t k_samples) {
  const int64_t waves = (int64_t)g->n_graphs * ((k_samples + 63) / 64);
  return waves >= 256 && longest_graph(g) <= (waves < 2048 ? waves : 2048) && g->n_edges <= 3 * (int64_t)g->n_nodes;
}

void plan_evaluate(const gdp_graph* g, int32_t n_devices, int32_t k, EvalPlan* p) {
  const size_t N = (size_t)g->n_nodes, E = (size_t)g->n_edges;
  int32_t blk[GDP_MAX_GRAPHS + 1];
  const int windows = prefix_blocks_rows(g->graph_ptr_h, g->n_graphs, kEvalWindowRows, blk);
  p->by_lanes = eval_by_lanes(g, k);
  p->far_stride = (N + 63) / 64 * 64;
  carve_init(&p->c);
  p->counters = carve_add(&p->c, (2 * N + 1) * 4);
  p->scan_tmp = carve_add(&p->c, 2 * ((N + 1023) / 1024) * 4);
  p->in_ptr = carve_add(&p->c, (N + 1) * 4);
  p->s_ptr = carve_add(&p->c, (N + 1) * 4);
  p->in_idx = carve_add(&p->c, (E > 0 ? E : 1) * 4);
  p->rec = carve_add(&p->c, (E > 0 ? E : 1) * 8);
  p->hdr = carve_add(&p->c, p->by_lanes ? 0 : N * 16);
  p->win = carve_add(&p->c, p->by_lanes ? 0 : (size_t)windows * 16);
  p->memsum = carve_add(&p->c, p->by_lanes ? (size_t)g->n_graphs * (size_t)k * (size_t)n_devices * 8 : 0);
  if (p->by_lanes) p->far = carve_add(&p->c, ((size_t)k + 63) / 64 * 64 * N * 4);
  else p->far = carve_add(&p->c, longest_graph(g) > kEvalMinRing ? (size_t)k * p->far_stride * 4 : 0);
}

int check_train(const gdp_graph* g, const gdp_gnn* gnn, const gdp_placer* p) {
  int r;
  if ((r = check_gnn(g, gnn)) != GDP_OK) return r;
  if ((r = check_placer(g, p)) != GDP_OK) return r;
  if (gnn->n_layers > kMaxTrainGnnLayers)
    return fail(GDP_E_UNSUPPORTED, "training supports at most %d GNN layers (got %d)", kMaxTrainGnnLayers, gnn->n_layers);
  if (p->n_layers > kMaxTrainPlacerLayers)
    return fail(GDP_E_UNSUPPORTED, "training supports at most %d placer layers (got %d)", kMaxTrainPlacerLayers,
                p->n_layers);
  if (p->d_model != gnn->hidden)
    return fail(GDP_E_INVALID_ARG, "d_model = %d != gnn.hidden = %d", p->d_model, gnn->hidden);
  return GDP_OK;
}

bool vec_stride(long stride) { return stride >= 0 && stride < (1L << 23); }

void plan_train(const gdp_graph* g, const gdp_gnn* gnn, const gdp_placer* pl, TrainPlan* t) {
  const size_t N = (size_t)g->n_nodes, E = (size_t)g->n_edges, H = (size_t)gnn->hidden, d = (size_t)pl->d_model;
  const size_t G = (size_t)g->n_graphs, dff = (size_t)pl->d_ff, F = (size_t)g->feat_dim;
  const size_t heads = pl->attention ? (size_t)pl->n_heads : 1;
  int32_t blk[GDP_MAX_GRAPHS + 1];
  t->chunks = prefix_blocks_rows(g->graph_ptr_h, g->n_graphs, kColSumRows, blk);
  const size_t cap_a = 2 * E, cap_b = N * (size_t)gnn->fanout;
  t->s_cap = (int64_t)(cap_a < cap_b ? cap_a : cap_b);
  Carve c;
  carve_init(&c);
  t->s_ptr = carve_add(&c, (N + 1) * 4);
  t->s_idx = carve_add(&c, (t->s_cap > 0 ? (size_t)t->s_cap : 1) * 4);
  t->in_ptr = carve_add(&c, (N + 1) * 4);
  t->in_idx = carve_add(&c, (E > 0 ? E : 1) * 4);
  t->x0 = carve_add(&c, G * H * 4);
  t->film = carve_add(&c, (size_t)pl->n_layers * 2 * G * d * 4);
  for (int l = 0; l < gnn->n_layers; ++l) {
    t->P[l] = carve_add(&c, N * H * 4);
    t->A[l] = carve_add(&c, N * H * 4);
    t->arg[l] = carve_add(&c, N * H * 4);
    t->h[l + 1] = carve_add(&c, N * H * 4);
  }
  t->h[0] = 0;
  t->X[0] = t->h[gnn->n_layers];
  for (int l = 0; l < pl->n_layers; ++l) {
    t->Y[l] = pl->film ? carve_add(&c, N * d * 4) : 0;   // without FiLM the layer reads X[l]
    t->QKV[l] = pl->attention ? carve_add(&c, N * 3 * d * 4) : 0;
    t->O[l] = pl->attention ? carve_add(&c, N * d * 4) : 0;
    t->lse_att[l] = pl->attention ? carve_add(&c, N * heads * 4) : 0;
    t->R1[l] = pl->attention ? carve_add(&c, N * d * 4) : 0;
    t->Z[l] = pl->attention ? carve_add(&c, N * d * 4) : 0;
    t->H1[l] = carve_add(&c, N * dff * 4);
    t->R2[l] = carve_add(&c, N * d * 4);
    t->X[l + 1] = carve_add(&c, N * d * 4);
  }
  t->store_total = c.total;

  const size_t wide = d > H ? d : H;
  const size_t fin = F > wide ? F : wide;
  carve_init(&c);
  t->counters = carve_add(&c, (2 * N + 1) * 4);
  t->scan_tmp = carve_add(&c, 2 * ((N + 1023) / 1024) * 4);
  t->heavy = carve_add(&c, N * 4);
  t->dX = carve_add(&c, N * d * 4);
  t->dY = carve_add(&c, N * d * 4);
  t->dR = carve_add(&c, N * d * 4);
  t->dZ = carve_add(&c, N * d * 4);
  t->dH = carve_add(&c, N * dff * 4);
  t->dqkv = carve_add(&c, N * 3 * d * 4);
  t->dkva = carve_add(&c, N * 2 * d * 4);
  t->Dq = carve_add(&c, N * heads * 4);
  t->head_partial = carve_add(&c, ((N + kHeadBwdRows - 1) / kHeadBwdRows) * (size_t)pl->n_devices * (d + 1) * 4);
  t->dfilm = carve_add(&c, (size_t)pl->n_layers * 2 * G * d * 4);
  t->dx0 = carve_add(&c, G * H * 4);
  t->dh = carve_add(&c, N * fin * 4);
  t->dA = carve_add(&c, N * H * 4);
  t->dP = carve_add(&c, N * H * 4);
  t->dU = carve_add(&c, N * H * 4);
  t->colpart = carve_add(&c, ((size_t)t->chunks + G) * 2 * wide * 4);
  const size_t big = (dff * d > 3 * d * d ? dff * d : 3 * d * d);
  // weight gradients: k = N split into pieces of at most 2,048 rows, more of them for small matrices
  const size_t few = (N + 255) / 256 < 8 ? (N + 255) / 256 : 8, splits = (N + 1023) / 1024;
  t->gemm_partial_floats = (splits > few ? splits : few) * ((big > H * fin ? big : H * fin) + dff + 3 * wide);
  t->gemm_partial = carve_add(&c, t->gemm_partial_floats * 4);
  t->ws_total = c.total;
}

void plan_sample(const gdp_graph* g, int32_t k, SamplePlan* p) {
  int32_t blk[GDP_MAX_GRAPHS + 1];
  p->chunks = prefix_blocks_rows(g->graph_ptr_h, g->n_graphs, kSampleRows, blk);
  carve_init(&p->c);
  p->partial = carve_add(&p->c, (size_t)k * p->chunks * 4);
  p->coef = carve_add(&p->c, (size_t)g->n_graphs * (k + 1) * 4);
}

// ---------------------------------------------------------------------------
// Layer operators.
// ---------------------------------------------------------------------------
int norm_backward_blocks(int64_t rows, int32_t width) {
  const int64_t most = std::max<int64_t>(256, (1 << 20) / width);
  return (int)std::min<int64_t>(std::min<int64_t>(1024, most), std::min<int64_t>(rows, (rows * width + 4095) / 4096));
}

static int check_dtype(int32_t dtype) {
  if (dtype != GDP_F32 && dtype != GDP_BF16) return fail(GDP_E_INVALID_ARG, "dtype = %d", dtype);
  return GDP_OK;
}

int check_norm(int64_t rows, int32_t width, int32_t dtype, float eps) {
  if (rows < 0) return fail(GDP_E_INVALID_ARG, "rows = %lld < 0", (long long)rows);
  if (rows > INT64_MAX / 65536) return fail(GDP_E_UNSUPPORTED, "rows = %lld", (long long)rows);
  if (width < 1) return fail(GDP_E_INVALID_ARG, "width = %d < 1", width);
  if (width > GDP_MAX_NORM_WIDTH)
    return fail(GDP_E_UNSUPPORTED, "width = %d exceeds GDP_MAX_NORM_WIDTH = %d", width, GDP_MAX_NORM_WIDTH);
  if (!(eps >= 0.f) || eps > FLT_MAX) return fail(GDP_E_INVALID_ARG, "eps = %g must be finite and >= 0", (double)eps);
  return check_dtype(dtype);
}

int check_ld(const char* name, int64_t ld, int64_t least) {
  if (ld < least) return fail(GDP_E_INVALID_ARG, "%s = %lld < %lld", name, (long long)ld, (long long)least);
  if (ld > (int64_t(1) << 40)) return fail(GDP_E_UNSUPPORTED, "%s = %lld", name, (long long)ld);
  return GDP_OK;
}

int check_fc(const gdp_fc_layer* f) {
  if (!f) return fail(GDP_E_INVALID_ARG, "fc layer is NULL");
  if (f->rows < 0) return fail(GDP_E_INVALID_ARG, "rows = %lld < 0", (long long)f->rows);
  if (f->in_dim < 1 || f->out_dim < 1)
    return fail(GDP_E_INVALID_ARG, "in_dim = %d and out_dim = %d must be at least 1", f->in_dim, f->out_dim);
  if (f->act != GDP_ACT_NONE && f->act != GDP_ACT_RELU) return fail(GDP_E_INVALID_ARG, "act = %d", f->act);
  if (f->rows > INT32_MAX) return fail(GDP_E_UNSUPPORTED, "rows = %lld exceeds %d", (long long)f->rows, INT32_MAX);
  // tiles of 64 x 64 at the least
  const int64_t m = f->rows / 64 + 1, k = f->in_dim / 64 + 1, n = f->out_dim / 64 + 1;
  if (m * std::max(k, n) > INT32_MAX / 64 || k * n > INT32_MAX / 64)
    return fail(GDP_E_UNSUPPORTED, "%lld rows of %d to %d are too many tiles", (long long)f->rows, f->in_dim, f->out_dim);
  return check_dtype(f->dtype);
}

void plan_fc_backward(const gdp_fc_layer* f, FcPlan* p) {
  carve_init(&p->c);
  const int64_t M = f->rows, K = f->in_dim, N = f->out_dim;
  const bool f32 = f->dtype == GDP_F32, relu = f->act == GDP_ACT_RELU;
  auto whole = [](int64_t n, int64_t v) { return (n + v - 1) / v * v; };
  p->ldp = p->ldx = p->ldw = 0;
  p->partial_floats = 0;
  p->splits = p->rows_per_split = 0;
  if (f32) {
    // ReLU's selection of dy, for both products; and they tell a matrix's order by which
    // stride is 1, so a column (row stride 1) is copied too
    if (relu || f->ld_dy == 1) p->ldp = whole(N, 4);
  } else {
    // bf16: rows of whole 16-byte vectors, which the direct loads need (12,001 rows of 515 to
    // 1,003: 73 us, 141 without); and ReLU's selection of dy (made where the products read
    // dy instead: 143 against 139 us at 52,000 rows of 256 to 1,024, 470 against 314 at
    // 16,384 of 2,048 to 2,048)
    if (relu || N % 8 != 0 || f->ld_dy % 8 != 0) p->ldp = whole(N, 8);
    if (K % 8 != 0 || f->ld_x % 8 != 0) p->ldx = whole(K, 8);
    if (K % 8 != 0) p->ldw = whole(K, 8);
  }
  p->dp = carve_add(&p->c, (size_t)(p->ldp * M) * elem_size(f->dtype));
  p->x = carve_add(&p->c, (size_t)(p->ldx * M) * 2);
  p->w = carve_add(&p->c, (size_t)(p->ldw * N) * 2);
  if (f32) {
    const int64_t pieces = std::min<int64_t>(64, std::max<int64_t>(1, M / 256));
    p->partial_floats = whole(N * (K + 1) * pieces, 64);
    p->partial = carve_add(&p->c, (size_t)(p->partial_floats + N * K) * 4);
  } else {
    // two work-groups per CU, each at least 256 rows of the sum
    const int64_t tiles = ((N + 127) / 128) * ((K + 127) / 128);
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>(512 / tiles, (M + 255) / 256));
    const int64_t per = std::max<int64_t>(64, whole((M + want - 1) / want, 64));
    p->rows_per_split = (int)std::min<int64_t>(per, INT32_MAX / 64 * 64);
    p->splits = (int)std::max<int64_t>(1, (M + p->rows_per_split - 1) / p->rows_per_split);
    p->partial = carve_add(&p->c, (size_t)p->splits * (size_t)(N * K + N) * 4);
  }
  if (p->c.total == 0) carve_add(&p->c, 256);
}

static int rel_queries(const gdp_rel_attn* a, int g) { return a->n_query_h ? a->n_query_h[g] : a->len_h[g]; }

int check_rel(const gdp_rel_attn* a, bool backward) {
  if (!a) return fail(GDP_E_INVALID_ARG, "attention is NULL");
  if (a->n_graphs < 1) return fail(GDP_E_INVALID_ARG, "n_graphs = %d < 1", a->n_graphs);
  if (a->n_graphs > GDP_MAX_GRAPHS)
    return fail(GDP_E_UNSUPPORTED, "n_graphs = %d exceeds GDP_MAX_GRAPHS = %d", a->n_graphs, GDP_MAX_GRAPHS);
  if (!a->key_start_h || !a->len_h) return fail(GDP_E_INVALID_ARG, "key_start_h or len_h is NULL");
  if (a->n_heads < 1 || a->n_kv_heads < 1 || a->n_heads % a->n_kv_heads != 0)
    return fail(GDP_E_INVALID_ARG, "n_heads = %d is not a positive multiple of n_kv_heads = %d", a->n_heads, a->n_kv_heads);
  if (a->head_dim != 16 && a->head_dim != 32 && a->head_dim != 64)
    return fail(GDP_E_UNSUPPORTED, "head_dim = %d not in {16,32,64}", a->head_dim);
  if (a->seg_len < 1) return fail(GDP_E_INVALID_ARG, "seg_len = %d < 1", a->seg_len);
  if (a->mem_len < 0) return fail(GDP_E_INVALID_ARG, "mem_len = %d < 0", a->mem_len);
  if (a->causal != 0 && a->causal != 1) return fail(GDP_E_INVALID_ARG, "causal = %d must be 0 or 1", a->causal);
  if (a->n_bounds < 0) return fail(GDP_E_INVALID_ARG, "n_bounds = %d < 0", a->n_bounds);
  if (a->n_bounds > GDP_MAX_REL_BOUNDS)
    return fail(GDP_E_UNSUPPORTED, "n_bounds = %d exceeds GDP_MAX_REL_BOUNDS = %d", a->n_bounds, GDP_MAX_REL_BOUNDS);
  if (a->n_bounds > 0 && !a->bounds_h) return fail(GDP_E_INVALID_ARG, "bounds_h is NULL");
  for (int i = 0; i < a->n_bounds; ++i)
    if (a->bounds_h[i] < 1 || (i > 0 && a->bounds_h[i] <= a->bounds_h[i - 1]))
      return fail(GDP_E_INVALID_ARG, "bounds_h[%d] = %d: the bounds must ascend from 1 on", i, a->bounds_h[i]);
  if (!(a->scale >= -FLT_MAX && a->scale <= FLT_MAX)) return fail(GDP_E_INVALID_ARG, "scale is not finite");
  int r = check_dtype(a->dtype);
  if (r != GDP_OK) return r;
  int64_t queries = 0, qblocks = 0, kblocks = 0;
  for (int g = 0; g < a->n_graphs; ++g) {
    const int len = a->len_h[g];
    if (len < 0 || a->key_start_h[g] < 0)
      return fail(GDP_E_INVALID_ARG, "graph %d: key_start_h = %d and len_h = %d must not be negative", g, a->key_start_h[g], len);
    if (len > GDP_MAX_REL_LEN) return fail(GDP_E_UNSUPPORTED, "len_h[%d] = %d exceeds GDP_MAX_REL_LEN", g, len);
    const int nq = rel_queries(a, g);
    if (nq < 0 || nq > len) return fail(GDP_E_INVALID_ARG, "n_query_h[%d] = %d outside 0..%d", g, nq, len);
    queries += nq;
    qblocks += (nq + 63) / 64;
    kblocks += (len + 63) / 64;
    if (backward)
      for (int h = 0; h < g; ++h)
        if (len > 0 && a->len_h[h] > 0 && a->key_start_h[g] < (int64_t)a->key_start_h[h] + a->len_h[h] &&
            a->key_start_h[h] < (int64_t)a->key_start_h[g] + len)
          return fail(GDP_E_INVALID_ARG, "the key rows of graphs %d and %d overlap", h, g);
  }
  if (queries > INT32_MAX || std::max(qblocks, kblocks) * a->n_heads > INT32_MAX / 64)
    return fail(GDP_E_UNSUPPORTED, "%lld queries of %d heads are too many", (long long)queries, a->n_heads);
  const int64_t wq = (int64_t)a->n_heads * a->head_dim, wk = (int64_t)a->n_kv_heads * a->head_dim;
  r = check_ld("ld_q", a->ld_q, wq);
  if (r == GDP_OK) r = check_ld("ld_k", a->ld_k, wk);
  if (r == GDP_OK) r = check_ld("ld_v", a->ld_v, wk);
  if (r == GDP_OK) r = check_ld("ld_o", a->ld_o, wq);
  if (r == GDP_OK && backward) r = check_ld("ld_do", a->ld_do, wq);
  if (r == GDP_OK && backward) r = check_ld("ld_dq", a->ld_dq, wq);
  if (r == GDP_OK && backward) r = check_ld("ld_dk", a->ld_dk, wk);
  if (r == GDP_OK && backward) r = check_ld("ld_dv", a->ld_dv, wk);
  return r;
}

void plan_rel(const gdp_rel_attn* a, bool backward, RelPlan* p) {
  carve_init(&p->c);
  int longest = 1;
  int64_t wide = 0;                                // blocks of 128 queries
  p->queries = 0;
  for (int g = 0; g < a->n_graphs; ++g) {
    longest = std::max(longest, a->len_h[g]);
    p->queries += rel_queries(a, g);
    wide += (rel_queries(a, g) + 127) / 128;
  }
  p->seg = std::min(a->seg_len, longest);
  p->mem = std::min(a->mem_len, longest);
  p->buckets = (a->n_bounds + 1) * (a->causal ? 1 : 2);
  // Two columns a wave halve the tile reads a product, where that leaves two work-groups
  // a CU and the registers hold them (not three planes of d_h = 64): 52,000 queries of 8 heads
  // of 32, 147 us with two and 192 with one, 29,000 of 8 of 16 51 and 63.  The backward keeps
  // one: with two, half as many waves fit (29,000 rows, d_h = 16: dK and dV 110 us with one and
  // 155 with two, dQ 92 and 147).
  const bool fits = a->dtype == GDP_BF16 || a->head_dim < 64;
  p->cols = fits && wide * a->n_heads >= 512 ? 2 : 1;
  // Few queries: about two work-groups a CU in all, each at least 4 tiles of 64 keys.
  int most = 0;
  int64_t groups = 0;
  for (int g = 0; g < a->n_graphs; ++g) {
    most = std::max(most, rel_queries(a, g));
    groups += ((int64_t)rel_queries(a, g) * (a->n_heads / a->n_kv_heads) + 15) / 16 * a->n_kv_heads;
  }
  p->parts = 0;
  const int64_t seen = std::min<int64_t>(longest, (int64_t)p->seg + p->mem + kRelFewQueries);
  if (!backward && most > 0 && most <= kRelFewQueries)
    p->parts = (int)std::max<int64_t>(1, std::min<int64_t>((512 + groups - 1) / groups, (seen + 255) / 256));
  p->key_blocks = 0;
  for (int g = 0; g < a->n_graphs; ++g) p->key_blocks += (a->len_h[g] + 63) / 64;
  p->d = carve_add(&p->c, backward ? (size_t)p->queries * a->n_heads * 4
                          : p->parts > 1 ? (size_t)p->queries * a->n_heads * p->parts * (a->head_dim + 4) * 4 : 256);
  p->table_partial = carve_add(&p->c, backward ? (size_t)p->key_blocks * a->n_heads * p->buckets * 4 : 0);
  if (p->c.total == 0) carve_add(&p->c, 256);
}

}  // namespace gdp

using namespace gdp;

extern "C" const char* gdp_last_error(void) { return g_err; }

extern "C" int gdp_abi_version(void) { return GDP_ABI_VERSION; }

extern "C" int gdp_validate_graph_host(const int32_t* graph_ptr, int32_t G, const int32_t* row_ptr,
                                       int32_t N, const int32_t* col_idx, int64_t E, uint32_t flags) {
  clear_error();
  if (!graph_ptr || !row_ptr || (E > 0 && !col_idx)) return fail(GDP_E_INVALID_ARG, "NULL array");
  if (G < 1 || N < 1 || E < 0 || E > INT32_MAX) return fail(GDP_E_INVALID_ARG, "bad sizes G=%d N=%d E=%lld", G, N, (long long)E);
  if (flags & ~GDP_TOPO_IDS) return fail(GDP_E_INVALID_ARG, "unknown flags 0x%x", flags);
  if (graph_ptr[0] != 0 || graph_ptr[G] != N) return fail(GDP_E_BAD_GRAPH, "graph_ptr must run from 0 to N");
  for (int g = 0; g < G; ++g)
    if (graph_ptr[g + 1] <= graph_ptr[g]) return fail(GDP_E_BAD_GRAPH, "graph %d is empty or graph_ptr decreases", g);
  if (row_ptr[0] != 0 || row_ptr[N] != E) return fail(GDP_E_BAD_GRAPH, "row_ptr must run from 0 to E");
  for (int v = 0; v < N; ++v)
    if (row_ptr[v + 1] < row_ptr[v]) return fail(GDP_E_BAD_GRAPH, "row_ptr decreases at node %d", v);
  std::vector<int32_t> indeg((size_t)N, 0);
  std::vector<int32_t> mark((size_t)N, -1);
  int g = 0;
  for (int u = 0; u < N; ++u) {
    while (u >= graph_ptr[g + 1]) ++g;
    for (int32_t e = row_ptr[u]; e < row_ptr[u + 1]; ++e) {
      const int32_t v = col_idx[e];
      if (v < 0 || v >= N) return fail(GDP_E_BAD_GRAPH, "edge %d: col_idx %d out of range", e, v);
      if (v == u) return fail(GDP_E_BAD_GRAPH, "self-loop at node %d", u);
      if (v < graph_ptr[g] || v >= graph_ptr[g + 1]) return fail(GDP_E_BAD_GRAPH, "edge %d -> %d crosses graphs", u, v);
      if ((flags & GDP_TOPO_IDS) && v < u) return fail(GDP_E_BAD_GRAPH, "edge %d -> %d breaks topological ids", u, v);
      if (mark[(size_t)v] == u) return fail(GDP_E_BAD_GRAPH, "duplicate edge %d -> %d", u, v);
      mark[(size_t)v] = u;
      ++indeg[(size_t)v];
    }
  }
  // Kahn's algorithm: every node must be removable.
  std::vector<int32_t> queue;
  queue.reserve((size_t)N);
  for (int v = 0; v < N; ++v)
    if (indeg[(size_t)v] == 0) queue.push_back(v);
  size_t head = 0;
  while (head < queue.size()) {
    const int32_t u = queue[head++];
    for (int32_t e = row_ptr[u]; e < row_ptr[u + 1]; ++e)
      if (--indeg[(size_t)col_idx[e]] == 0) queue.push_back(col_idx[e]);
  }
  if (queue.size() != (size_t)N) return fail(GDP_E_BAD_GRAPH, "graph has a cycle");
  return GDP_OK;
}
