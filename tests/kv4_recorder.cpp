// The operators of long contexts on a compressed cache (rotary positions, 4-bit cache, attention over it, eviction) over the runtime of the launch recorder: their
// refusals and their launches on a machine without a GPU.
//
// usage: kv4_recorder <call> key=value ...   with null=, misalign= naming a pointer, same=a,b giving b the address of a
#include "gemm.h"
#include "kernels.h"
#define main launch_recorder_main
#define hipGetDevice recorder_hip_get_device
#include "launch_recorder.cpp"
#undef hipGetDevice
#undef main

static int g_device;
extern "C" hipError_t hipGetDevice(int *d) { *d = g_device; return hipSuccess; }

static std::map<std::string, char *> g_ptrs;
template <typename T>
static T *ptr(const char *name, size_t bytes) {
  const std::string same = g_opt.count("same") ? g_opt["same"] : "";
  char *p = (char *)fake(bytes + 16);
  const size_t comma = same.find(',');
  if (comma != std::string::npos && same.substr(comma + 1) == name) p = g_ptrs[same.substr(0, comma)] + num("offset", 0);
  if (g_opt.count("null") && g_opt["null"] == name) p = nullptr;
  if (g_opt.count("misalign") && g_opt["misalign"] == name) p += num("by", 2);
  g_ptrs[name] = p;
  return (T *)p;
}
static double real(const char *k, double dflt) { return g_opt.count(k) ? atof(g_opt[k].c_str()) : dflt; }

int main(int argc, char **argv) {
  const std::string call = argc > 1 ? argv[1] : "";
  for (int i = 2; i < argc; ++i) {
    const char *e = strchr(argv[i], '=');
    if (!e) return 2;
    g_opt[std::string(argv[i], e - argv[i])] = e + 1;
  }
  (void)stream_id(nullptr);
  const int32_t hkv = (int32_t)num("hkv", 4), group = (int32_t)num("group", 2), hd = (int32_t)num("hd", 64), n = (int32_t)num("n", 100);
  mace_model_t m = {256, hkv * group, hkv, hd, 704, 2048, 1e-6f, 1e4f, num("bf16", 1) ? MACE_BF16 : MACE_F32};
  mace_handle_t h;
  if (mace_create(&h, &m) != MACE_OK) return 3;
  g_device = (int)num("device", 0);
  const size_t rows = n > 0 ? (size_t)n : 0;
  const int32_t n_req = (int32_t)num("n_req", 3), max_rows = (int32_t)num("max_rows", 1), max_context = (int32_t)num("max_context", 1000);
  const size_t need = call == "attention" ? mace_kv4_attention_workspace_bytes(h, n_req, max_rows, max_context)
                      : call == "evict"   ? mace_kv4_evict_workspace_bytes(h, n_req, max_context)
                                          : 0;
  printf("{\"op\": \"need\", \"bytes\": %zu}\n", need);
  const size_t have = (size_t)num("work", (long long)need);
  if (g_opt.count("null") && g_opt["null"] == "handle") h = nullptr;

  mace_kv4_cache_t c = {};
  c.num_blocks = num("blocks", 300);
  c.block_size = (int32_t)num("block", 16);
  const size_t tokens = c.num_blocks > 0 && c.block_size > 0 ? (size_t)c.num_blocks * c.block_size * hkv : 0;
  c.k = ptr<void>("k", tokens * hd / 2);
  c.v = ptr<void>("v", tokens * hd / 2);
  c.k_scale = ptr<void>("k_scale", tokens * hd / 32);
  c.v_scale = ptr<void>("v_scale", tokens * hd / 32);
  c.weight = ptr<float>("weight", tokens * 4);
  c.position = ptr<int32_t>("position", tokens * 4);
  const mace_kv4_cache_t *cache = g_opt.count("null") && g_opt["null"] == "cache" ? nullptr : &c;
  const int64_t cols = (int64_t)hkv * hd, qcols = cols * group;
  const int32_t heads = (int32_t)num("heads", 1), tables = (int32_t)num("tables", 70);
  int rc = 1;
  if (call == "rotary") {
    const int32_t nh = (int32_t)num("n_heads", 6), rot = (int32_t)num("rot", hd);
    const int64_t ld_x = num("ld_x", (int64_t)nh * hd), ld_out = num("ld_out", (int64_t)nh * hd);
    void *x = ptr<void>("x", rows * ld_x * 4);
    int32_t *pos = ptr<int32_t>("positions", rows * 4);
    double *freq = ptr<double>("freq", 4096);
    rc = mace_rotary(h, x, ld_x, pos, freq, rot, (int)num("inter", 0), real("magnitude", 1), (int)num("inverse", 0), n, nh, ptr<void>("out", rows * ld_out * 4), ld_out, nullptr);
  } else if (call == "append") {
    const int64_t ld_k = num("ld_k", cols), ld_v = num("ld_v", cols);
    void *k = ptr<void>("k_new", rows * ld_k * 4), *v = ptr<void>("v_new", rows * ld_v * 4);
    int32_t *slots = ptr<int32_t>("slots", rows * 4 * hkv);
    rc = mace_kv4_append(h, cache, k, ld_k, v, ld_v, slots, heads, ptr<int32_t>("positions", rows * 4), n, nullptr);
  } else if (call == "gather") {
    int32_t *slots = ptr<int32_t>("slots", rows * 4 * hkv);
    void *k = ptr<void>("k_out", rows * cols * 4);
    rc = mace_kv4_gather(h, cache, slots, heads, n, k, ptr<void>("v_out", rows * cols * 4), nullptr);
  } else if (call == "attention") {
    const int32_t n_rows = (int32_t)num("n_rows", (long long)n_req * max_rows);
    const int64_t ld_q = num("ld_q", qcols), ld_out = num("ld_out", qcols);
    const size_t r = n_rows > 0 ? n_rows : 0, req = n_req > 0 ? n_req : 0;
    void *q = ptr<void>("q", r * ld_q * 4);
    int32_t *off = num("offsets", max_rows > 1) ? ptr<int32_t>("q_offsets", (req + 1) * 4) : nullptr;
    int32_t *bt = ptr<int32_t>("block_tables", req * tables * 4), *lens = ptr<int32_t>("lens", req * 4 * hkv);
    void *out = ptr<void>("out", r * ld_out * 4);
    float *lse = ptr<float>("lse", r * 4 * hkv * group);
    rc = mace_kv4_attention(h, cache, q, ld_q, off, n_req, n_rows, max_rows, bt, tables, lens, heads, max_context, (float)real("scale", 0.125), (int)num("add", 0), out, ld_out, lse,
                            ptr<void>("work", need), have, nullptr);
  } else if (call == "evict") {
    const size_t req = n_req > 0 ? n_req : 0;
    int32_t *bt = ptr<int32_t>("block_tables", req * tables * 4), *lens = ptr<int32_t>("lens", req * 4 * hkv), *seq = ptr<int32_t>("seq", req * 4);
    int32_t *budgets = ptr<int32_t>("budgets", req * 4 * hkv), *nl = ptr<int32_t>("new_lens", req * 4 * hkv);
    rc = mace_kv4_evict(h, cache, bt, n_req, tables, lens, heads, max_context, seq, budgets, (int)num("sink", 4), (int)num("recent", 10), nl, ptr<void>("work", need), have, nullptr);
  } else {
    return 2;
  }
  printf("{\"op\": \"return\", \"status\": %d, \"error\": \"%s\"}\n", rc, rc ? mace_last_error() : "");
  return 0;
}
