// Host side of the packed-token calls: layer writes (gambit_kv_write_layer),
// prompt attention (gambit_prompt_attn) and draft-tree attention
// (gambit_tree_attn) - validation against the host mirror and the plans that
// their kernels read.
//
// A call's plan depends on what it lists and on the mirror alone, so the
// layers of a step, which list the same, share one: it is made and uploaded
// by the first call and kept until the mirror changes or a call of its kind
// (write, prompt, tree) lists something else.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <numeric>
#include <vector>

#include "../../include/gambit.h"
#include "pool.h"
#include "rows.h"

using namespace gambit::host;
using gambit::RowItem;
using gambit::WriteItem;

namespace {

// ---- calls -----------------------------------------------------------------
// The checks that every packed call shares.
gambit_status check_call(gambit_pool* p, int32_t layer, int32_t n, const int32_t* ids, const int32_t* counts,
                         hipStream_t s, int64_t* total) {
  if (p->step_next) return step_open(p);
  if (layer < 0 || layer >= p->dev.num_layers)
    return fail(p, GAMBIT_ERR_INVALID, "layer %d of %d", layer, p->dev.num_layers);
  gambit_status st = check_ids(p, n, ids, "trace");
  if (st) return st;
  if (n > 0 && !counts) return fail(p, GAMBIT_ERR_INVALID, "token counts are NULL");
  *total = 0;
  for (int i = 0; i < n; ++i) {
    if (counts[i] < 0) return fail(p, GAMBIT_ERR_INVALID, "negative token count");
    if (p->ghost[ids[i]]) return fail(p, GAMBIT_ERR_INVALID, "slot %d holds a ghost trace", ids[i]);
    *total += counts[i];
  }
  if (*total > p->L.max_packed)
    return fail(p, GAMBIT_ERR_UNSUPPORTED, "%lld tokens in one call, at most %d", (long long)*total, p->L.max_packed);
  // A plan is uploaded through buffers that the next call reuses, so a
  // replayed graph would read another call's.
  hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
  HIP_TRY(p, hipStreamIsCapturing(s, &cap), "capture status");
  if (cap != hipStreamCaptureStatusNone) return fail(p, GAMBIT_ERR_UNSUPPORTED, "the stream is being captured");
  int dev = 0;
  HIP_TRY(p, hipGetDevice(&dev), "device");
  if (dev != p->device)
    return fail(p, GAMBIT_ERR_INVALID, "device %d is current, the pool is on device %d", dev, p->device);
  return GAMBIT_OK;
}

bool aligned16(const void* x) { return reinterpret_cast<uintptr_t>(x) % 16 == 0; }

// What a call lists, as one list of ints to compare with its kind's next call's.
std::vector<int32_t> listing(int32_t n, const int32_t* ids, const int32_t* a, const int32_t* b, const int32_t* c,
                             size_t nc) {
  std::vector<int32_t> v;
  v.reserve(2 + 3 * (size_t)n + nc);
  v.push_back(n);
  v.insert(v.end(), ids, ids + n);
  v.insert(v.end(), a, a + n);
  if (b) v.insert(v.end(), b, b + n);
  v.push_back(c != nullptr);
  if (c) v.insert(v.end(), c, c + nc);
  return v;
}

// Fills one plan's pinned image piece by piece; the pieces' device addresses
// follow the image's layout.
struct Image {
  uint8_t *host, *dev;
  size_t cap, at = 0;
  bool fits = true;
  template <class T>
  const T* put(const T* src, size_t n) {
    const size_t o = at;
    at = align_up(at + n * sizeof(T));
    if (at > cap) {
      fits = false;
      return nullptr;
    }
    if (n) std::memcpy(host + o, src, n * sizeof(T));
    return reinterpret_cast<const T*>(dev + o);
  }
};

// ---- attention plan --------------------------------------------------------
// The listed tokens' rows are cut into tiles of up to kRowsTile rows of one
// trace, or, over blocks that several of the listed traces hold, of all of
// them.  A tile's positions are cut into chunks where there are too few tiles
// for the chip, or where one would run far longer than the others.
struct Listed {
  int trace, base, m;  // packed tokens base .. base + m - 1
  int ctx;             // positions every one of them sees
  int full;            // blocks that they all see whole
  int priv;            // first block that no other listed trace reads with it
};

struct Plan {
  std::vector<RowItem> items;
  std::vector<int32_t> list, off, nk, merge;
  int parts = 0;
};

// Positions of a chunk at least: below that a workgroup's start and its
// partial rows cost more than its keys.
constexpr int kLeastChunk = 256;
// Workgroups a call is cut into: as many as the chip runs at once.  More rounds
// share the chip more evenly but start more often and leave more partials: 64
// trees of eight nodes 156, 165, 177, 186 us with 1, 1.5, 2, 3 rounds; sixteen long
// trees 297, 319, 309, 318; insertions into 64 traces 284, 283, 288, 296.
// Choosing the rounds per call by the estimated length of the longest-first
// schedule moved these by -1 to +4%.  Where all of a call fits one round, its
// chunks are the shortest that one round holds (the sixteen trees 290 -> 276 us);
// where it does not, they are cut to about the even share, no shorter (at most that
// share: the 64 trees 130 -> 134, the insertions 252 -> 254).

struct Run {
  int j0, j1;                    // blocks
  int owner;                     // a listed trace that holds them
  std::vector<int32_t> members;  // listed traces, ascending
};

// The runs of blocks that several of the listed traces (those marked) read.
// Sharing only comes from forks, so along a trace the set of sharers can
// only shrink: equal counts on consecutive blocks mean equal sets.
void shared_runs(gambit_pool* p, std::vector<Listed>& L, const std::vector<char>& share, std::vector<Run>* runs,
                 std::vector<std::vector<int32_t>>* runs_of) {
  if (p->first.size() != p->refcount.size()) p->first.assign(p->refcount.size(), -1);
  std::vector<int32_t> touched, starts;
  for (size_t i = 0; i < L.size(); ++i) {
    if (!share[i]) continue;
    const auto& row = p->table[L[i].trace];
    for (int j = 0; j < L[i].full && p->refcount[row[j]] > 1; ++j)
      if (p->cnt[row[j]]++ == 0) touched.push_back(row[j]);
  }
  for (size_t i = 0; i < L.size(); ++i) {
    L[i].priv = 0;
    if (!share[i]) continue;
    const auto& row = p->table[L[i].trace];
    int j = 0;
    while (j < L[i].full && p->cnt[row[j]] > 1) {
      const int b = row[j], c = p->cnt[b];
      int j1 = j + 1;
      while (j1 < L[i].full && p->cnt[row[j1]] == c) ++j1;
      if (p->first[b] < 0) {
        p->first[b] = (int)runs->size();
        starts.push_back(b);
        runs->push_back(Run{j, j1, L[i].trace, {}});
      }
      (*runs)[p->first[b]].members.push_back((int)i);
      (*runs_of)[i].push_back(p->first[b]);
      j = j1;
    }
    L[i].priv = j;
  }
  for (int b : starts) p->first[b] = -1;
  for (int b : touched) p->cnt[b] = 0;
}

// The length of a chunk: about `target` positions, or `most` at most.
struct Cut {
  int64_t target;
  bool most;
  int chunks(int64_t tokens) const {
    return (int)std::max<int64_t>(1, (tokens + (most ? target - 1 : target / 2)) / target);
  }
};

bool try_plan(gambit_pool* p, const std::vector<Listed>& L, const std::vector<Run>& runs,
              const std::vector<std::vector<int32_t>>& runs_of, bool tree, Cut cut, Plan* out) {
  const int tile = gambit::kRowsTile / p->g;  // tokens of a tile
  *out = Plan{};
  int N = 0;
  for (const Listed& x : L) N += x.m;
  out->off.assign(N, 0);
  out->nk.assign(N, 0);
  // chunks of the shared runs, the same for all of a run's members
  std::vector<int> run_chunks(runs.size());
  for (size_t r = 0; r < runs.size(); ++r) run_chunks[r] = cut.chunks(16LL * (runs[r].j1 - runs[r].j0));
  std::vector<int> before(L.size(), 0);  // a trace's partials over its shared runs
  std::vector<std::vector<int32_t>> run_kidx(runs.size());
  for (size_t i = 0; i < L.size(); ++i)
    for (int r : runs_of[i]) {
      run_kidx[r].push_back(before[i]);
      before[i] += run_chunks[r];
    }
  int64_t parts = 0;
  auto chunked = [&](RowItem it, int j0, int end, int nch, int kidx) {  // positions [16 j0, end) in nch chunks
    const int tiles = cdiv(std::max(end - 16 * j0, 0), gambit::kKeyTile);
    for (int k = 0, at = 0; k < nch; ++k) {
      const int sz = tiles / nch + (k < tiles % nch ? 1 : 0);
      it.jb0 = j0 + 4 * at;
      it.end = k == nch - 1 ? end : std::min(end, 16 * j0 + gambit::kKeyTile * (at + sz));
      it.kidx = kidx < 0 ? -1 : kidx + k;
      RowItem one = it;
      if (k != nch - 1) one.draft = -1, one.ndraft = 0;
      out->items.push_back(one);
      at += sz;
    }
  };
  for (size_t i = 0; i < L.size(); ++i) {
    const Listed& x = L[i];
    for (int a = 0; a < x.m; a += tile) {
      const int ntok = std::min(tile, x.m - a);
      const int end = tree ? x.ctx : x.ctx + a + ntok;
      const int64_t tokens = std::max(0, end - 16 * x.priv);
      int nch = cut.chunks(tokens);
      nch = std::min(nch, std::max(1, cdiv((int)tokens, gambit::kKeyTile)));
      const int nk = before[i] + nch;
      for (int t = a; t < a + ntok; ++t) {
        out->nk[x.base + t] = nk;
        if (nk > 1) {
          out->off[x.base + t] = (int)std::min<int64_t>(parts, 1 << 30);
          out->merge.push_back(x.base + t);
          parts += nk;
        }
      }
      if (parts > p->L.max_parts) return false;
      RowItem it{};
      it.trace = x.trace;
      it.tok = x.base + a;
      it.ntok = ntok;
      it.pos0 = tree ? gambit::kNoLimit : x.ctx + a;
      it.draft = tree ? x.base : -1;
      it.ndraft = tree ? x.m : 0;
      it.once = x.m <= tile;
      chunked(it, x.priv, end, nch, nk > 1 ? before[i] : -1);
    }
  }
  for (size_t r = 0; r < runs.size(); ++r) {
    // tokens of the members, in tiles; members that reached the run over other
    // chunks (never: they share every block before it) would differ in kidx
    const Run& R = runs[r];
    std::vector<int32_t> toks;
    for (int i : R.members)
      for (int t = 0; t < L[i].m; ++t) toks.push_back(L[i].base + t);
    const int first = (int)out->list.size();
    out->list.insert(out->list.end(), toks.begin(), toks.end());
    for (int a = 0; a < (int)toks.size(); a += tile) {
      RowItem it{};
      it.trace = R.owner;
      it.tok = first + a;
      it.ntok = std::min(tile, (int)toks.size() - a);
      it.listed = 1;
      it.pos0 = gambit::kNoLimit;
      it.draft = -1;
      it.once = (int)toks.size() <= tile;
      chunked(it, R.j0, 16 * R.j1, run_chunks[r], run_kidx[r][0]);
    }
  }
  out->parts = (int)parts;
  return (int)out->items.size() <= p->L.max_items[tree] && (int)out->list.size() <= p->L.max_parts;
}

// Plans the call and uploads the plan: `anc` (trees) rides along.
gambit_status plan_rows(gambit_pool* p, std::vector<Listed> L, bool tree, const std::vector<uint64_t>& anc,
                        hipStream_t s) {
  const int tile = gambit::kRowsTile / p->g;
  // Traces of up to two tiles read shared blocks together, their rows packed
  // into common tiles; a longer prompt fills tiles of its own well enough, which
  // read the blocks once each either way.  64 traces in fours, 9 to 64 tokens of
  // four heads each: 270 us with one tile as the limit, 256 with two or four.
  std::vector<char> share(L.size());
  for (size_t i = 0; i < L.size(); ++i) share[i] = L[i].m > 0 && L[i].m <= 2 * tile;
  std::vector<Run> runs;
  std::vector<std::vector<int32_t>> runs_of(L.size());
  shared_runs(p, L, share, &runs, &runs_of);
  // f(row tiles, positions) of every range
  auto ranges = [&](auto&& f) {
    for (const Listed& x : L)
      for (int a = 0; a < x.m; a += tile)
        f(1, std::max(0, (tree ? x.ctx : x.ctx + std::min(x.m, a + tile)) - 16 * x.priv));
    for (const Run& R : runs) {
      int m = 0;
      for (int i : R.members) m += L[i].m;
      f(cdiv(m, tile), 16 * (R.j1 - R.j0));
    }
  };
  const int64_t round = 2 * p->n_cu, heads = p->d.num_kv_heads;
  auto groups = [&](Cut cut) {
    int64_t n = 0;
    ranges([&](int tiles, int tokens) { n += tiles * cut.chunks(tokens); });
    return n * heads;
  };
  int64_t work = 0;  // positions that the row tiles go over; a tile of drafts, or a masked one, with every trace's
  ranges([&](int tiles, int tokens) { work += (int64_t)tiles * tokens; });
  for (const Listed& x : L) work += (int64_t)gambit::kKeyTile * cdiv(x.m, tile);
  Plan plan;
  Cut cut{std::max<int64_t>(kLeastChunk, work * heads / round), groups(Cut{1LL << 40, true}) <= round};
  if (cut.most && groups(cut) > round) {
    int64_t lo = cut.target, hi = 1LL << 31;
    while (hi - lo > gambit::kKeyTile) {
      const int64_t mid = (lo + hi) / 2;
      (groups(Cut{mid, true}) <= round ? hi : lo) = mid;
    }
    cut.target = hi;
  }
  bool ok = try_plan(p, L, runs, runs_of, tree, cut, &plan);
  while (!ok && cut.target < (1LL << 31)) {
    cut.target *= 2;
    ok = try_plan(p, L, runs, runs_of, tree, cut, &plan);
  }
  if (!ok) {  // every trace by itself, in one piece: no partials
    for (Listed& x : L) x.priv = 0;
    runs.clear();
    for (auto& r : runs_of) r.clear();
    ok = try_plan(p, L, runs, runs_of, tree, Cut{1LL << 40, true}, &plan);
  }
  if (!ok) return fail(p, GAMBIT_ERR_UNSUPPORTED, "plan exceeds workspace bounds");
  for (RowItem& it : plan.items)
    for (int b = 0; b < 4 && it.end > 16 * it.jb0; ++b)
      it.first[b] = p->table[it.trace][std::min(it.jb0 + b, (it.end - 1) / 16)];
  // longest first, so that no long one starts late
  std::stable_sort(plan.items.begin(), plan.items.end(), [](const RowItem& a, const RowItem& b) {
    return a.end - 16 * a.jb0 > b.end - 16 * b.jb0;
  });
  const int kind = tree ? kTreePlan : kPromptPlan;
  KeptPlan<gambit::RowsLaunch>& slot = p->rows[kind];
  HIP_TRY(p, hipEventSynchronize(slot.ev), "plan fence");
  slot.key.valid = false;
  Image im{slot.image, p->ws + p->L.rows_plan[kind], p->L.rows_plan_bytes[kind]};
  gambit::RowsLaunch& A = slot.launch;
  A = gambit::RowsLaunch{};
  A.items = im.put(plan.items.data(), plan.items.size());
  A.n_items = (int)plan.items.size();
  A.anc = tree ? im.put(anc.data(), anc.size()) : nullptr;
  A.list = im.put(plan.list.data(), plan.list.size());
  A.off = im.put(plan.off.data(), plan.off.size());
  A.nk = im.put(plan.nk.data(), plan.nk.size());
  A.merge = im.put(plan.merge.data(), plan.merge.size());
  A.n_merge = (int)plan.merge.size();
  if (!im.fits) return fail(p, GAMBIT_ERR_UNSUPPORTED, "plan exceeds workspace bounds");
  HIP_TRY(p, hipMemcpyAsync(im.dev, im.host, im.at, hipMemcpyHostToDevice, s), "plan upload");
  HIP_TRY(p, hipEventRecord(slot.ev, s), "plan fence");
  return GAMBIT_OK;
}

// Launches a kept plan on one layer.
gambit_status launch_rows(gambit_pool* p, int kind, int32_t layer, const void* q, const void* k_new, const void* v_new, void* out,
                          int32_t out_dtype, float sm_scale, hipStream_t s) {
  gambit::RowsLaunch A = p->rows[kind].launch;
  A.q = static_cast<const uint16_t*>(q);
  A.k_new = static_cast<const uint16_t*>(k_new);
  A.v_new = static_cast<const uint16_t*>(v_new);
  A.out = out;
  A.out_f32 = out_dtype == GAMBIT_OUT_F32;
  // the sign of the scale goes to the queries, a scale of zero makes them zero
  A.c = sm_scale == 0.f ? 1.f : std::max(std::fabs(sm_scale) * 1.4426950408889634f, 0x1p-120f);
  A.q_and = sm_scale == 0.f ? 0u : 0xffffffffu;
  A.q_xor = sm_scale < 0.f ? 0x80008000u : 0u;
  A.gshift = __builtin_ctz(p->g);
  A.part_acc = ws_ptr<float>(p, p->L.part_acc);
  A.part_ml = ws_ptr<float2>(p, p->L.part_ml);
  HIP_TRY(p, gambit::launch_rows_attention(p->dev.layer(layer), A, s), "rows attention");
  return GAMBIT_OK;
}

gambit_status check_attention(gambit_pool* p, const void* q, const void* out, int32_t out_dtype, float sm_scale) {
  if (!q || !out) return fail(p, GAMBIT_ERR_INVALID, "NULL buffer");
  if (!aligned16(q) || !aligned16(out)) return fail(p, GAMBIT_ERR_INVALID, "a buffer is not 16-byte aligned");
  if (out_dtype != GAMBIT_OUT_BF16 && out_dtype != GAMBIT_OUT_F32)
    return fail(p, GAMBIT_ERR_INVALID, "bad output dtype");
  if (!std::isfinite(sm_scale)) return fail(p, GAMBIT_ERR_INVALID, "softmax scale is not finite");
  return GAMBIT_OK;
}

bool kept(const gambit_pool* p, const PackedKey& k, const std::vector<int32_t>& now) {
  return k.valid && k.epoch == p->epoch && k.listed == now;
}

void keep(gambit_pool* p, PackedKey* k, std::vector<int32_t>&& now) {
  k->listed = std::move(now);
  k->epoch = p->epoch;
  k->valid = true;
}

gambit_status prompt_attn(gambit_pool* p, int32_t layer, int32_t n, const int32_t* ids, const int32_t* ntok,
                          const void* q, void* out, int32_t out_dtype, float sm_scale, hipStream_t s) {
  int64_t total = 0;
  gambit_status st = check_call(p, layer, n, ids, ntok, s, &total);
  if (st) return st;
  for (int i = 0; i < n; ++i)
    if (ntok[i] > p->seq_len[ids[i]])
      return fail(p, GAMBIT_ERR_INVALID, "%d tokens of trace %d, which holds %d", ntok[i], ids[i], p->seq_len[ids[i]]);
  if (total == 0) return GAMBIT_OK;
  if ((st = check_attention(p, q, out, out_dtype, sm_scale))) return st;
  std::vector<int32_t> now = listing(n, ids, ntok, nullptr, nullptr, 0);
  if (!kept(p, p->rows[kPromptPlan].key, now)) {
    std::vector<Listed> L;
    for (int i = 0, base = 0; i < n; base += ntok[i++]) {
      const int ctx = p->seq_len[ids[i]] - ntok[i];
      L.push_back(Listed{ids[i], base, ntok[i], ctx, ctx / 16, 0});
    }
    if ((st = plan_rows(p, std::move(L), false, {}, s))) return st;
    keep(p, &p->rows[kPromptPlan].key, std::move(now));
  }
  return launch_rows(p, kPromptPlan, layer, q, nullptr, nullptr, out, out_dtype, sm_scale, s);
}

gambit_status tree_attn(gambit_pool* p, int32_t layer, int32_t n, const int32_t* ids, const int32_t* nodes,
                        const int32_t* parents, const void* q, const void* k_new, const void* v_new, void* out,
                        int32_t out_dtype, float sm_scale, hipStream_t s) {
  int64_t total = 0;
  gambit_status st = check_call(p, layer, n, ids, nodes, s, &total);
  if (st) return st;
  for (int i = 0; i < n; ++i)
    if (nodes[i] > gambit::kMaxNodes)
      return fail(p, GAMBIT_ERR_UNSUPPORTED, "a tree of %d nodes, at most %d", nodes[i], gambit::kMaxNodes);
  if (total == 0) return GAMBIT_OK;
  if (!parents) return fail(p, GAMBIT_ERR_INVALID, "parent list is NULL");
  for (int i = 0, base = 0; i < n; base += nodes[i++])
    for (int j = 0; j < nodes[i]; ++j)
      if (parents[base + j] < -1 || parents[base + j] >= j)
        return fail(p, GAMBIT_ERR_INVALID, "node %d of trace %d has parent %d", j, ids[i], parents[base + j]);
  if ((st = check_attention(p, q, out, out_dtype, sm_scale))) return st;
  if (!k_new || !v_new) return fail(p, GAMBIT_ERR_INVALID, "NULL buffer");
  if (!aligned16(k_new) || !aligned16(v_new)) return fail(p, GAMBIT_ERR_INVALID, "a buffer is not 16-byte aligned");
  std::vector<int32_t> now = listing(n, ids, nodes, nullptr, parents, (size_t)total);
  if (!kept(p, p->rows[kTreePlan].key, now)) {
    std::vector<Listed> L;
    std::vector<uint64_t> anc((size_t)total);
    for (int i = 0, base = 0; i < n; base += nodes[i++]) {
      const int len = p->seq_len[ids[i]];
      L.push_back(Listed{ids[i], base, nodes[i], len, len / 16, 0});
      for (int j = 0; j < nodes[i]; ++j) {
        const int up = parents[base + j];
        anc[base + j] = (up < 0 ? 0 : anc[base + up]) | 1ull << j;
      }
    }
    if ((st = plan_rows(p, std::move(L), true, anc, s))) return st;
    keep(p, &p->rows[kTreePlan].key, std::move(now));
  }
  return launch_rows(p, kTreePlan, layer, q, k_new, v_new, out, out_dtype, sm_scale, s);
}

gambit_status kv_write_layer(gambit_pool* p, int32_t layer, int32_t n, const int32_t* ids, const int32_t* pos0,
                             const int32_t* ntok, const int32_t* rows, int32_t n_rows, const void* k, const void* v,
                             hipStream_t s) {
  int64_t total = 0;
  gambit_status st = check_call(p, layer, n, ids, ntok, s, &total);
  if (st) return st;
  if (n > 0 && !pos0) return fail(p, GAMBIT_ERR_INVALID, "positions are NULL");
  for (int i = 0; i < n; ++i) {
    const int t = ids[i];
    if (pos0[i] < 0 || (int64_t)pos0[i] + ntok[i] > p->seq_len[t])
      return fail(p, GAMBIT_ERR_INVALID, "write of %d tokens at %d outside trace %d's %d positions", ntok[i], pos0[i], t,
                  p->seq_len[t]);
  }
  if (n_rows < 0 || (!rows && n_rows != total))
    return fail(p, GAMBIT_ERR_INVALID, "%d rows of K and V for %lld tokens", n_rows, (long long)total);
  if (total == 0) return GAMBIT_OK;
  if (rows)
    for (int64_t i = 0; i < total; ++i)
      if (rows[i] < 0 || rows[i] >= n_rows) return fail(p, GAMBIT_ERR_INVALID, "row %d of %d", rows[i], n_rows);
  if (!k || !v) return fail(p, GAMBIT_ERR_INVALID, "K or V is NULL");
  if (!aligned16(k) || !aligned16(v)) return fail(p, GAMBIT_ERR_INVALID, "a buffer is not 16-byte aligned");
  for (int i = 0; i < n; ++i)
    if (ntok[i] > 0)
      for (int j = pos0[i] / 16; j <= (pos0[i] + ntok[i] - 1) / 16; ++j)
        if (p->refcount[p->table[ids[i]][j]] != 1)
          return fail(p, GAMBIT_ERR_SHARED_WRITE, "block %d of trace %d is shared", j, ids[i]);
  std::vector<int32_t> now = listing(n, ids, ntok, pos0, rows, (size_t)total);
  if (!kept(p, p->write.key, now)) {
    std::vector<WriteItem> items;
    for (int i = 0, base = 0; i < n; base += ntok[i++]) {
      const int a = pos0[i], e = a + ntok[i];
      for (int j = a / 16; 16 * j < e && ntok[i] > 0; ++j) {
        const int r0 = std::max(a - 16 * j, 0), r1 = std::min(e - 16 * j, 16);
        const float floor = r0 ? 0.f : r1 == 16 ? 0x1p-20f : p->append_scale;
        items.push_back(WriteItem{p->table[ids[i]][j], base + 16 * j + r0 - a, (int16_t)r0, (int16_t)r1, floor});
      }
    }
    HIP_TRY(p, hipEventSynchronize(p->write.ev), "plan fence");
    p->write.key.valid = false;
    Image im{p->write.image, p->ws + p->L.write_plan, p->L.write_plan_bytes};
    gambit::WriteLaunch& W = p->write.launch;
    W = gambit::WriteLaunch{};
    W.items = im.put(items.data(), items.size());
    W.n_items = (int)items.size();
    W.rows = rows ? im.put(rows, (size_t)total) : nullptr;
    if (!im.fits) return fail(p, GAMBIT_ERR_UNSUPPORTED, "plan exceeds workspace bounds");
    HIP_TRY(p, hipMemcpyAsync(im.dev, im.host, im.at, hipMemcpyHostToDevice, s), "plan upload");
    HIP_TRY(p, hipEventRecord(p->write.ev, s), "plan fence");
    keep(p, &p->write.key, std::move(now));
  }
  gambit::WriteLaunch W = p->write.launch;
  W.k = static_cast<const uint16_t*>(k);
  W.v = static_cast<const uint16_t*>(v);
  HIP_TRY(p, gambit::launch_rows_write(p->dev.layer(layer), W, s), "layer write");
  return GAMBIT_OK;
}

// No exception leaves a C entry; one that ended a plan half made leaves the
// planners' per-block scratch as they expect it.
template <class F>
gambit_status guarded(gambit_pool* p, F&& f) {
  if (!p) return GAMBIT_ERR_INVALID;
  try {
    return f();
  } catch (...) {
    std::fill(p->cnt.begin(), p->cnt.end(), 0);
    std::fill(p->first.begin(), p->first.end(), -1);
    for (auto& x : p->rows) x.key.valid = false;
    p->write.key.valid = false;
    return fail(p, GAMBIT_ERR_DEVICE, "out of host memory");
  }
}

}  // namespace

extern "C" {

gambit_status gambit_kv_write_layer(gambit_pool* p, int32_t layer, int32_t n, const int32_t* ids, const int32_t* pos0,
                                    const int32_t* ntok, const int32_t* rows, int32_t n_rows, const void* k,
                                    const void* v, void* stream) {
  return guarded(p, [&] { return kv_write_layer(p, layer, n, ids, pos0, ntok, rows, n_rows, k, v, S(stream)); });
}

gambit_status gambit_prompt_attn(gambit_pool* p, int32_t layer, int32_t n, const int32_t* ids, const int32_t* ntok,
                                 const void* q, void* out, int32_t out_dtype, float sm_scale, void* stream) {
  return guarded(p, [&] { return prompt_attn(p, layer, n, ids, ntok, q, out, out_dtype, sm_scale, S(stream)); });
}

gambit_status gambit_tree_attn(gambit_pool* p, int32_t layer, int32_t n, const int32_t* ids, const int32_t* nodes,
                               const int32_t* parents, const void* q, const void* k_new, const void* v_new, void* out,
                               int32_t out_dtype, float sm_scale, void* stream) {
  return guarded(p, [&] {
    return tree_attn(p, layer, n, ids, nodes, parents, q, k_new, v_new, out, out_dtype, sm_scale, S(stream));
  });
}

}  // extern "C"
