// The entry points at the two ends of a model (embedding rows, token log-probabilities and their gradients) over the runtime of the
// launch recorder: their refusals and their launches on a machine without a GPU.
//
// usage: token_ops_recorder <call> key=value ...   with null=, misalign= naming a pointer, same=a,b giving b the address of a
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

int main(int argc, char **argv) {
  const std::string call = argc > 1 ? argv[1] : "";
  for (int i = 2; i < argc; ++i) {
    const char *e = strchr(argv[i], '=');
    if (!e) return 2;
    g_opt[std::string(argv[i], e - argv[i])] = e + 1;
  }
  (void)stream_id(nullptr);
  const int32_t d = (int32_t)num("d", 256), V = (int32_t)num("V", 2048), n = (int32_t)num("n", 100), vocab = (int32_t)num("vocab", V);
  const int32_t dtype = (int32_t)num("dtype", MACE_F32), d_dtype = (int32_t)num("d_dtype", MACE_BF16), k = (int32_t)num("top_k", 0);
  const int64_t ld = num("ld", vocab), ld_d = num("ld_d", vocab);
  const float scale = g_opt.count("scale") ? (float)atof(g_opt["scale"].c_str()) : 1.f;
  mace_model_t m = {d, 4, 4, 64, 704, V, 1e-6f, 1e4f, num("bf16", 1) ? MACE_BF16 : MACE_F32};
  mace_handle_t h;
  if (mace_create(&h, &m) != MACE_OK) return 3;
  g_device = (int)num("device", 0);
  const size_t rows = n > 0 ? (size_t)n : 0, e = 4;
  const size_t need = call == "embed_grad" ? mace_embed_grad_workspace_bytes(h, n) : call == "logprobs" ? mace_token_logprobs_workspace_bytes(h, n, vocab, k) : 0;
  printf("{\"op\": \"need\", \"bytes\": %zu}\n", need);
  const size_t have = (size_t)num("work", (long long)need);
  if (g_opt.count("null") && g_opt["null"] == "handle") h = nullptr;
  int rc = 1;
  int32_t *ids = ptr<int32_t>("ids", rows * 4);
  if (call == "embed") {
    void *table = ptr<void>("table", (size_t)V * d * e);
    rc = mace_embed_tokens(h, table, ids, n, scale, ptr<void>("out", rows * d * e), nullptr);
  } else if (call == "embed_grad") {
    float *dx = ptr<float>("dx", rows * d * e), *dt = ptr<float>("d_table", (size_t)V * d * e);
    rc = mace_embed_tokens_grad(h, ids, n, dx, scale, dt, (int)num("accumulate", 0), ptr<void>("work", need), have, nullptr);
  } else if (call == "logprobs") {
    const bool top = num("top", k > 0);
    void *x = ptr<void>("logits", rows * ld * e);
    float *lp = ptr<float>("logp", rows * 4), *en = ptr<float>("entropy", rows * 4), *rs = ptr<float>("stats", rows * 8);
    if (num("no_outputs", 0)) lp = en = rs = nullptr;
    int32_t *ti = top ? ptr<int32_t>("top_ids", rows * 128) : nullptr;
    float *tl = top ? ptr<float>("top_logp", rows * 128) : nullptr;
    rc = mace_token_logprobs(h, x, dtype, n, vocab, ld, ids, k, lp, en, rs, ti, tl, ptr<void>("work", need), have, nullptr);
  } else if (call == "logprobs_grad") {
    void *x = ptr<void>("logits", rows * ld * e);
    float *rs = ptr<float>("stats", rows * 8), *en = ptr<float>("entropy", rows * 4), *dl = ptr<float>("d_logp", rows * 4), *de = ptr<float>("d_entropy", rows * 4);
    if (num("no_weights", 0)) dl = de = nullptr;
    rc = mace_token_logprobs_grad(h, x, dtype, n, vocab, ld, ids, rs, en, dl, de, ptr<void>("d_logits", rows * ld_d * e), d_dtype, ld_d, nullptr);
  } else {
    return 2;
  }
  printf("{\"op\": \"return\", \"status\": %d, \"error\": \"%s\"}\n", rc, rc ? mace_last_error() : "");
  return 0;
}
