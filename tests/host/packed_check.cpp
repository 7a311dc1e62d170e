// Host harness for the packed-token calls (built with g++ under sanitizers;
// see tests/test_packed_plan.py): the pool's host source and the packed
// calls' host source against the host-only HIP stand-in, with launch
// functions that do nothing.  What runs is the library's validation and the
// plans it stages into the caller's workspace.
//
// Protocol: one operation per input line, one JSON object per output line.
//   create NB HQ HKV T MAXB SPLITS FP8 LAYERS
//   alloc t n ...; fork p c ...; free t ...; decode t ...
//   prompt LAYER t n ...                  gambit_prompt_attn, then its plan
//   tree LAYER ntraces t m ... parents..  gambit_tree_attn, then its plan
//   write LAYER n_rows t pos0 n ... [rows r ...]   gambit_kv_write_layer, then its items
//   uploads                               copies to the device so far
#include <hip/hip_runtime.h>

enum hipStreamCaptureStatus { hipStreamCaptureStatusNone = 0, hipStreamCaptureStatusActive = 1 };
static bool g_capturing = false;
static int g_device = 0;
inline hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* s) {
  *s = g_capturing ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone;
  return hipSuccess;
}
#define hipGetDevice(d) (*(d) = g_device, hipSuccess)
static int g_uploads = 0;
inline hipError_t counted_copy(void* d, const void* s, size_t n, hipMemcpyKind k, hipStream_t q) {
  g_uploads += k == hipMemcpyHostToDevice;
  return hipMemcpyAsync(d, s, n, k, q);
}
#define hipMemcpyAsync counted_copy

#include "../../paper_2608_08020_amd/csrc/gambit_pool.cpp"
#include "../../paper_2608_08020_amd/csrc/rows_attn.cpp"

#include <iostream>
#include <sstream>

namespace gambit {
hipError_t launch_pool_init(const DevPool&, hipStream_t) { return hipSuccess; }
hipError_t launch_alloc(const DevPool&, const int32_t*, const int32_t*, int32_t, int32_t, float, bool, hipStream_t) {
  return hipSuccess;
}
hipError_t launch_write(const DevPool&, int32_t, int32_t, int32_t, const void*, const void*, const float*, hipStream_t) {
  return hipSuccess;
}
hipError_t launch_free(const DevPool&, const int32_t*, int32_t, int32_t, hipStream_t) { return hipSuccess; }
hipError_t launch_fork(const DevPool&, const int32_t*, int32_t, int32_t*, int32_t*, hipStream_t) { return hipSuccess; }
hipError_t launch_attention_units(const DevPool&, const AttnLaunch&, hipStream_t) { return hipSuccess; }
hipError_t launch_attention_merge(const DevPool&, const AttnLaunch&, hipStream_t) { return hipSuccess; }
hipError_t launch_probe_rank(const ProbeLaunch&, hipStream_t) { return hipSuccess; }
hipError_t launch_rank_topk(int32_t, const int32_t*, const float*, int32_t, int32_t*, hipStream_t) { return hipSuccess; }
hipError_t launch_score_update(const DevPool&, const ScoreLaunch&, hipStream_t) { return hipSuccess; }
hipError_t launch_evict_pick(const DevPool&, const int32_t*, int32_t, int32_t*, hipStream_t) { return hipSuccess; }
hipError_t launch_tournament(const DevPool&, int32_t, int32_t, int32_t, int32_t*, int32_t*, hipStream_t) {
  return hipSuccess;
}
hipError_t launch_mlp_score(const MlpLaunch&, hipStream_t) { return hipSuccess; }
hipError_t launch_record_scores(const DevPool&, const int32_t*, const float*, int32_t, hipStream_t) { return hipSuccess; }

static RowsLaunch g_rows;
static WriteLaunch g_write;
static int g_launched = 0;
hipError_t launch_rows_attention(const DevPool&, const RowsLaunch& L, hipStream_t) {
  g_rows = L;
  ++g_launched;
  return hipSuccess;
}
hipError_t launch_rows_write(const DevPool&, const WriteLaunch& L, hipStream_t) {
  g_write = L;
  ++g_launched;
  return hipSuccess;
}
}  // namespace gambit

namespace {

struct Buffers {
  std::vector<uint8_t> kc, vc;
  std::vector<int32_t> table, seq, ref;
  std::vector<float> scale;
  uint8_t* ws_raw = nullptr;
  ~Buffers() { std::free(ws_raw); }
};

template <class T>
void print_list(std::ostream& o, const char* name, const T* a, size_t n) {
  o << ",\"" << name << "\":[";
  for (size_t i = 0; i < n; ++i) o << (i ? "," : "") << a[i];
  o << "]";
}

void dump_rows(gambit_pool* p, int st, int total, int launched) {
  std::ostringstream o;
  o << "{\"status\":" << st << ",\"launched\":" << launched << ",\"error\":\"" << (st ? gambit_last_error(p) : "") << "\"";
  if (st == GAMBIT_OK && launched) {
    const gambit::RowsLaunch& A = gambit::g_rows;
    o << ",\"max_parts\":" << p->L.max_parts << ",\"items\":[";
    int listed = 0;
    for (int i = 0; i < A.n_items; ++i) {
      const RowItem& u = A.items[i];
      if (u.listed) listed = std::max(listed, u.tok + u.ntok);
      o << (i ? "," : "") << "[" << u.trace << "," << u.jb0 << "," << u.end << "," << u.tok << "," << u.ntok << ","
        << u.listed << "," << u.pos0 << "," << u.kidx << "," << u.draft << "," << u.ndraft << "]";
    }
    o << "]";
    std::vector<int32_t> first;
    for (int i = 0; i < A.n_items; ++i) first.insert(first.end(), A.items[i].first, A.items[i].first + 4);
    print_list(o, "first", first.data(), first.size());
    print_list(o, "list", A.list, listed);
    print_list(o, "off", A.off, total);
    print_list(o, "nk", A.nk, total);
    print_list(o, "merge", A.merge, A.n_merge);
    if (A.anc) print_list(o, "anc", A.anc, total);
  }
  o << "}";
  std::cout << o.str() << "\n";
}

void dump_write(gambit_pool* p, int st, int launched) {
  std::ostringstream o;
  o << "{\"status\":" << st << ",\"launched\":" << launched << ",\"error\":\"" << (st ? gambit_last_error(p) : "") << "\"";
  if (st == GAMBIT_OK && launched) {
    const gambit::WriteLaunch& W = gambit::g_write;
    o << ",\"items\":[";
    for (int i = 0; i < W.n_items; ++i) {
      const WriteItem& u = W.items[i];
      o << (i ? "," : "") << "[" << u.blk << "," << u.src << "," << u.r0 << "," << u.r1 << "," << u.floor << "]";
    }
    o << "]";
  }
  o << "}";
  std::cout << o.str() << "\n";
}

}  // namespace

int main() {
  Buffers B;
  gambit_pool* p = nullptr;
  std::string line;
  void* fake = reinterpret_cast<void*>(uintptr_t(1) << 20);  // never dereferenced
  while (std::getline(std::cin, line)) {
    std::istringstream in(line);
    std::string op, word;
    in >> op;
    std::vector<int32_t> a, rows;
    bool with_rows = false;
    while (in >> word) {
      if (word == "rows")
        with_rows = true;
      else
        (with_rows ? rows : a).push_back((int32_t)std::stol(word));
    }
    const int before = gambit::g_launched;
    if (op == "create") {
      gambit_pool_desc d{};
      d.num_blocks = a[0], d.block_size = 16, d.num_q_heads = a[1], d.num_kv_heads = a[2], d.head_dim = 128;
      d.max_traces = a[3], d.max_blocks_per_trace = a[4], d.max_splits = a[5];
      d.kv_dtype = a[6] ? GAMBIT_KV_FP8_E4M3 : GAMBIT_KV_BF16;
      d.num_layers = a[7];
      const size_t ws = gambit_workspace_size(&d);
      B.kc.resize(16), B.vc.resize(16);
      B.table.assign((size_t)a[3] * a[4], -1), B.seq.assign(a[3], 0), B.ref.assign(a[0], 0), B.scale.assign(2, 0.f);
      B.ws_raw = static_cast<uint8_t*>(std::malloc(ws + 256));
      const uintptr_t base = (reinterpret_cast<uintptr_t>(B.ws_raw) + 255) / 256 * 256;
      d.k_cache = B.kc.data(), d.v_cache = B.vc.data(), d.block_table = B.table.data(), d.seq_len = B.seq.data();
      d.refcount = B.ref.data(), d.kv_scale = a[6] ? B.scale.data() : nullptr;
      d.workspace = reinterpret_cast<void*>(base), d.workspace_bytes = ws;
      const int st = gambit_pool_create(&d, nullptr, &p);
      std::cout << "{\"status\":" << st << ",\"max_packed\":" << (p ? p->L.max_packed : 0) << "}\n";
    } else if (op == "uploads") {
      std::cout << "{\"status\":0,\"uploads\":" << g_uploads << "}\n";
    } else if (op == "capturing" || op == "device") {
      if (op == "device") g_device = a[0];
      if (op == "capturing") g_capturing = a[0] != 0;
      std::cout << "{\"status\":0}\n";
    } else if (op == "prompt") {
      std::vector<int32_t> t, n;
      long total = 0;
      for (size_t i = 1; i + 1 < a.size(); i += 2) t.push_back(a[i]), n.push_back(a[i + 1]), total += a[i + 1];
      const int st = gambit_prompt_attn(p, a[0], (int)t.size(), t.data(), n.data(), fake, fake, 0, 0.1f, nullptr);
      dump_rows(p, st, (int)total, gambit::g_launched - before);
    } else if (op == "tree") {
      std::vector<int32_t> t, n;
      long total = 0;
      size_t i = 2;
      for (int k = 0; k < a[1]; ++k, i += 2) t.push_back(a[i]), n.push_back(a[i + 1]), total += a[i + 1];
      const std::vector<int32_t> up(a.begin() + i, a.end());
      const int st = gambit_tree_attn(p, a[0], (int)t.size(), t.data(), n.data(), up.data(), fake, fake, fake, fake, 1,
                                      0.1f, nullptr);
      dump_rows(p, st, (int)total, gambit::g_launched - before);
    } else if (op == "write") {
      std::vector<int32_t> t, p0, n;
      for (size_t i = 2; i + 2 < a.size(); i += 3) t.push_back(a[i]), p0.push_back(a[i + 1]), n.push_back(a[i + 2]);
      const int st = gambit_kv_write_layer(p, a[0], (int)t.size(), t.data(), p0.data(), n.data(),
                                           with_rows ? rows.data() : nullptr, a[1], fake, fake, nullptr);
      dump_write(p, st, gambit::g_launched - before);
    } else {
      int st = -99;
      std::vector<int32_t> x, y;
      for (size_t i = 0; i + 1 < a.size(); i += 2) x.push_back(a[i]), y.push_back(a[i + 1]);
      if (op == "alloc") st = gambit_kv_alloc(p, (int)x.size(), x.data(), y.data(), nullptr);
      if (op == "fork") st = gambit_kv_fork(p, (int)x.size(), x.data(), y.data(), nullptr);
      if (op == "free") st = gambit_kv_free(p, (int)a.size(), a.data(), nullptr);
      if (op == "decode")
        st = gambit_decode_attn_layer(p, p->step_next, (int)a.size(), a.data(), fake, fake, fake, 0, fake, 0, 0.1f, nullptr);
      std::cout << "{\"status\":" << st << "}\n";
    }
    std::cout.flush();
  }
  if (p) gambit_pool_destroy(p);
  return 0;
}
