// api.cu -- the extern "C" entry points of libsimsd.so (declared in
// include/simsd.h): argument checks on the host, then kernel launches on the
// caller's stream.  No call allocates memory or synchronises, except
// simsd_check_error.
#include <cuda.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdio>
#include <cstring>
#include <mutex>

#include "../../include/simsd.h"
#include "kernels.h"

namespace {

thread_local char g_last_error[256] = "";

// Planted wait expiry armed by simsd_debug_expire_next_wait for the next
// launch of one kernel on this thread (index: SIMSD_DEBUG_WAIT_*).
thread_local simsd::WaitFault g_armed[3];

simsd::WaitFault take_armed(int which) {
  const simsd::WaitFault f = g_armed[which];
  g_armed[which] = simsd::WaitFault{};
  return f;
}

int cuda_fail(cudaError_t e, const char* where) {
  std::snprintf(g_last_error, sizeof(g_last_error), "%s: %s", where, cudaGetErrorString(e));
  return SIMSD_ERR_CUDA;
}

int arg_fail(const char* what) {
  std::snprintf(g_last_error, sizeof(g_last_error), "invalid argument: %s", what);
  return SIMSD_ERR_INVALID_ARG;
}

int unsupported(const char* what) {
  std::snprintf(g_last_error, sizeof(g_last_error), "unsupported: %s", what);
  return SIMSD_ERR_UNSUPPORTED;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

struct DeviceInfo {
  int num_sms = 0;
  int major = 0, minor = 0;
};

// Per-device properties, queried once per device.
int device_info(DeviceInfo* out) {
  static std::mutex mu;
  static DeviceInfo cache[64];
  static bool have[64] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_fail(e, "cudaGetDevice");
  if (dev < 0 || dev >= 64) return unsupported("device ordinal >= 64");
  std::lock_guard<std::mutex> lk(mu);
  if (!have[dev]) {
    DeviceInfo d;
    if ((e = cudaDeviceGetAttribute(&d.num_sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess ||
        (e = cudaDeviceGetAttribute(&d.major, cudaDevAttrComputeCapabilityMajor, dev)) != cudaSuccess ||
        (e = cudaDeviceGetAttribute(&d.minor, cudaDevAttrComputeCapabilityMinor, dev)) != cudaSuccess)
      return cuda_fail(e, "cudaDeviceGetAttribute");
    cache[dev] = d;
    have[dev] = true;
  }
  *out = cache[dev];
  return SIMSD_OK;
}

int require_sm103(DeviceInfo* info) {
  int rc = device_info(info);
  if (rc != SIMSD_OK) return rc;
  if (info->major != 10 || info->minor != 3) return unsupported("this library is built for sm_103a only");
  return SIMSD_OK;
}

simsd::EncodeTiledFn encoder() {
  static simsd::EncodeTiledFn fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) ==
            cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<simsd::EncodeTiledFn>(p);
  });
  return fn;
}

cudaStream_t as_stream(void* s) { return static_cast<cudaStream_t>(s); }

// Shared body of the two attention entry points.  static_scratch: the
// split partials go to the library's static array instead of the caller's
// workspace.
int verify_attention_impl(int dtype, const void* q, const void* k_new, const void* v_new, const void* k_cache,
                          const void* v_cache, int num_pages, const int32_t* block_table, int max_pages,
                          int page_size, const int32_t* prefix_len, const int32_t* tau, const uint8_t* section,
                          const int32_t* rope_pos, float rope_theta, int Bt, int gamma, int Hq, int Hkv, int d,
                          float softmax_scale, void* out, void* workspace, size_t workspace_bytes,
                          bool static_scratch, const simsd::WaitFault& fault, int32_t* err_word, void* stream) {
  if (Bt < 0) return arg_fail("Bt < 0");
  if (gamma < 1 || gamma > 32) return arg_fail("gamma must be in [1, 32]");
  if (Hq <= 0 || Hkv <= 0 || Hq % Hkv != 0) return arg_fail("Hq must be a positive multiple of Hkv");
  if (num_pages < 0 || max_pages < 0) return arg_fail("negative page count");
  if (page_size < 8 || !((page_size % 64 == 0) || (64 % page_size == 0)))
    return unsupported("page_size must be a multiple of 64 or a divisor of 64 (>= 8)");
  if (rope_pos && (!(rope_theta > 0.f) || std::isinf(rope_theta)))
    return arg_fail("rope_theta must be positive and finite when rope_pos is given");
  if (!(softmax_scale >= 0.f) || std::isinf(softmax_scale)) return arg_fail("softmax_scale");
  if (Bt == 0) return SIMSD_OK;
  if (!q || !k_new || !v_new || !prefix_len || !tau || !section || !out) return arg_fail("null pointer");
  if (max_pages > 0 && (!block_table || !k_cache || !v_cache || num_pages == 0))
    return arg_fail("null cache or block table");
  if (!aligned16(q) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(out) ||
      (k_cache && !aligned16(k_cache)) || (v_cache && !aligned16(v_cache)))
    return arg_fail("tensor pointers must be 16-byte aligned");
  DeviceInfo info;
  int rc = require_sm103(&info);
  if (rc != SIMSD_OK) return rc;
  const float scale = softmax_scale > 0.f ? softmax_scale : 1.0f / std::sqrt(static_cast<float>(d));
  cudaStream_t s = as_stream(stream);
  if (dtype == SIMSD_F32) {
    // the fp32 path uses no scratch
    if (d != 64 && d != 128) return unsupported("fp32 path needs d in {64, 128}");
    simsd::AttnF32Args a{};
    a.q = static_cast<const float*>(q);
    a.k_new = static_cast<const float*>(k_new);
    a.v_new = static_cast<const float*>(v_new);
    a.k_cache = static_cast<const float*>(k_cache);
    a.v_cache = static_cast<const float*>(v_cache);
    a.block_table = block_table;
    a.prefix_len = prefix_len;
    a.tau = tau;
    a.section = section;
    a.rope_pos = rope_pos;
    if (rope_pos) a.rope = simsd::make_rope_table(rope_theta, d);
    a.out = static_cast<float*>(out);
    a.err_word = err_word;
    a.num_pages = num_pages;
    a.max_pages = max_pages;
    a.page_size = page_size;
    a.Bt = Bt;
    a.gamma = gamma;
    a.Hq = Hq;
    a.Hkv = Hkv;
    a.d = d;
    a.scale = scale;
    cudaError_t e = simsd::launch_attention_f32(a, s);
    return e == cudaSuccess ? SIMSD_OK : cuda_fail(e, "attention_f32 launch");
  }
  if (dtype != SIMSD_BF16) return unsupported("dtype");
  if (d != 128) return unsupported("bf16 path needs d = 128");
  if (static_cast<long long>(num_pages) * Hkv * page_size >= (1ll << 31))
    return unsupported("page pool too large for 32-bit TMA row coordinates");
  if (static_cast<long long>(Bt) * 2 * gamma * Hq >= (1ll << 31)) return unsupported("too many query rows");
  simsd::AttnTcPlan plan;
  if (!simsd::plan_attention_tc(Bt, gamma, Hq, Hkv, max_pages, page_size, info.num_sms, &plan, !static_scratch))
    return unsupported("query rows per KV head: need 2*gamma*Hq/Hkv <= 128 or 128 % (Hq/Hkv) == 0");
  if (static_scratch) {
    // (stream-K runs are not used here: their partials would outgrow the array)
    if (plan.ws_bytes > simsd::noalloc_scratch_capacity()) {
      std::snprintf(g_last_error, sizeof(g_last_error),
                    "unsupported: these sizes need %zu bytes of scratch, more than the %zu-byte static array; "
                    "use simsd_verify_attention with a caller workspace",
                    plan.ws_bytes, simsd::noalloc_scratch_capacity());
      return SIMSD_ERR_UNSUPPORTED;
    }
    workspace = nullptr;
    if (plan.ws_bytes > 0) {
      cudaError_t e = simsd::noalloc_scratch_pointer(&workspace);
      if (e != cudaSuccess) return cuda_fail(e, "cudaGetSymbolAddress of the static scratch");
    }
  } else if (plan.ws_bytes > 0 && (!workspace || workspace_bytes < plan.ws_bytes || !aligned16(workspace))) {
    return arg_fail("workspace smaller than simsd_verify_workspace_bytes()");
  }
  simsd::EncodeTiledFn enc = encoder();
  if (!enc) return cuda_fail(cudaErrorNotSupported, "cuTensorMapEncodeTiled entry point");
  simsd::AttnTcArgs a{};
  a.q = q;
  a.k_new = k_new;
  a.v_new = v_new;
  // a pool with no pages is still described by a valid (never read) map
  a.k_cache = k_cache ? k_cache : q;
  a.v_cache = v_cache ? v_cache : q;
  a.block_table = block_table;
  a.prefix_len = prefix_len;
  a.tau = tau;
  a.section = section;
  a.rope_pos = rope_pos;
  if (rope_pos) a.rope = simsd::make_rope_table(rope_theta, d);
  a.out = out;
  a.workspace = workspace;
  a.err_word = err_word;
  a.num_pages = num_pages > 0 ? num_pages : 1;
  a.max_pages = max_pages;
  a.page_size = page_size;
  a.Bt = Bt;
  a.gamma = gamma;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.scale = scale;
  a.fault = fault;
  if (num_pages == 0) {
    a.max_pages = 0;
    a.num_pages = 0;
  }
  cudaError_t e = simsd::launch_attention_tc(a, plan, enc, s);
  return e == cudaSuccess ? SIMSD_OK : cuda_fail(e, "attention_tc launch");
}

}  // namespace

namespace simsd {

RopeTable make_rope_table(double theta, int d) {
  RopeTable t{};
  for (int i = 0; i < d / 2 && i < 64; ++i) {
    const double f = std::pow(theta, -2.0 * i / d);
    const float hi = static_cast<float>(f);
    t.f[i] = make_float2(hi, static_cast<float>(f - static_cast<double>(hi)));
  }
  return t;
}

}  // namespace simsd

extern "C" {

int simsd_version(void) { return 1 * 10000 + 1 * 100 + 0; }

const char* simsd_last_error(void) { return g_last_error; }

int simsd_build_mask(const int32_t* step_map, const int32_t* prefix_len, int Bt, int gamma, int32_t* tau,
                     uint8_t* section, int32_t* rope_pos, uint64_t* mask_bits, int32_t* err_word, void* stream) {
  if (Bt < 0) return arg_fail("Bt < 0");
  if (gamma < 1 || gamma > 32) return arg_fail("gamma must be in [1, 32]");
  if (Bt == 0) return SIMSD_OK;
  if (!prefix_len || !tau || !section || !rope_pos) return arg_fail("null pointer");
  DeviceInfo info;
  int rc = require_sm103(&info);
  if (rc != SIMSD_OK) return rc;
  cudaError_t e = simsd::launch_build_mask(step_map, prefix_len, Bt, gamma, tau, section, rope_pos, mask_bits,
                                           err_word, as_stream(stream));
  return e == cudaSuccess ? SIMSD_OK : cuda_fail(e, "build_mask launch");
}

size_t simsd_verify_workspace_bytes(int dtype, int Bt, int gamma, int Hq, int Hkv, int d, int max_pages,
                                    int page_size) {
  if (dtype != SIMSD_BF16 || Bt <= 0 || gamma < 1 || gamma > 32 || Hkv <= 0 || Hq % Hkv != 0 || d != 128 ||
      max_pages < 0 || page_size <= 0)
    return 0;
  DeviceInfo info;
  if (device_info(&info) != SIMSD_OK) return 0;
  simsd::AttnTcPlan plan;
  if (!simsd::plan_attention_tc(Bt, gamma, Hq, Hkv, max_pages, page_size, info.num_sms, &plan)) return 0;
  return plan.ws_bytes;
}

int simsd_verify_attention(int dtype, const void* q, const void* k_new, const void* v_new, const void* k_cache,
                           const void* v_cache, int num_pages, const int32_t* block_table, int max_pages,
                           int page_size, const int32_t* prefix_len, const int32_t* tau, const uint8_t* section,
                           const int32_t* rope_pos, float rope_theta, int Bt, int gamma, int Hq, int Hkv, int d,
                           float softmax_scale, void* out, void* workspace, size_t workspace_bytes,
                           int32_t* err_word, void* stream) {
  // an armed wait expiry is consumed by this call whatever its outcome
  const simsd::WaitFault fault = take_armed(SIMSD_DEBUG_WAIT_ATTENTION);
  return verify_attention_impl(dtype, q, k_new, v_new, k_cache, v_cache, num_pages, block_table, max_pages,
                               page_size, prefix_len, tau, section, rope_pos, rope_theta, Bt, gamma, Hq, Hkv, d,
                               softmax_scale, out, workspace, workspace_bytes, false, fault, err_word, stream);
}

int simsd_verify_attention_noalloc(int dtype, const void* q, const void* k_new, const void* v_new,
                                   const void* k_cache, const void* v_cache, int num_pages,
                                   const int32_t* block_table, int max_pages, int page_size,
                                   const int32_t* prefix_len, const int32_t* tau, const uint8_t* section,
                                   const int32_t* rope_pos, float rope_theta, int Bt, int gamma, int Hq, int Hkv,
                                   int d, float softmax_scale, void* out, int32_t* err_word, void* stream) {
  return verify_attention_impl(dtype, q, k_new, v_new, k_cache, v_cache, num_pages, block_table, max_pages,
                               page_size, prefix_len, tau, section, rope_pos, rope_theta, Bt, gamma, Hq, Hkv, d,
                               softmax_scale, out, nullptr, 0, true, simsd::WaitFault{}, err_word, stream);
}

namespace {

// Greedy acceptance: the cluster kernel, or with a workspace (ws_ok) the
// split over many CTAs when the shape takes it.
int accept_impl(const float* logits, const int32_t* draft, int Bt, int gamma, int vocab, int32_t* accepted_len,
                int32_t* out_tokens, int32_t* row_argmax, bool ws_ok, void* workspace, size_t workspace_bytes,
                int32_t* err_word, void* stream) {
  // an armed wait expiry is consumed by this call whatever its outcome
  const simsd::WaitFault fault = take_armed(SIMSD_DEBUG_WAIT_ACCEPT);
  if (Bt < 0) return arg_fail("Bt < 0");
  if (gamma < 1 || gamma > 32) return arg_fail("gamma must be in [1, 32]");
  if (vocab < 1 || vocab > (1 << 28)) return arg_fail("vocab must be in [1, 2^28]");
  if (Bt == 0) return SIMSD_OK;
  if (!logits || !draft || !accepted_len || !out_tokens) return arg_fail("null pointer");
  DeviceInfo info;
  int rc = require_sm103(&info);
  if (rc != SIMSD_OK) return rc;
  const size_t need = ws_ok ? simsd::accept_workspace_bytes(Bt, gamma, vocab, info.num_sms) : 0;
  cudaError_t e;
  if (need > 0) {
    if (!workspace || workspace_bytes < need) return arg_fail("workspace smaller than simsd_accept_workspace_bytes()");
    if ((reinterpret_cast<uintptr_t>(workspace) & 7u) != 0) return arg_fail("workspace not 8-byte aligned");
    if (fault.extra) return unsupported("a planted wait expiry needs the cluster kernel (this path has no wait)");
    e = simsd::launch_accept_parts(logits, draft, Bt, gamma, vocab, accepted_len, out_tokens, row_argmax, workspace,
                                   err_word, info.num_sms, as_stream(stream));
  } else {
    e = simsd::launch_accept(logits, draft, Bt, gamma, vocab, accepted_len, out_tokens, row_argmax, err_word,
                             info.num_sms, as_stream(stream), fault);
    if (e == cudaErrorNotSupported && fault.extra)
      return unsupported("a planted wait expiry needs one CTA per sequence (a batch too large for clusters)");
  }
  return e == cudaSuccess ? SIMSD_OK : cuda_fail(e, "accept launch");
}

}  // namespace

int simsd_accept(const float* logits, const int32_t* draft, int Bt, int gamma, int vocab, int32_t* accepted_len,
                 int32_t* out_tokens, int32_t* row_argmax, int32_t* err_word, void* stream) {
  return accept_impl(logits, draft, Bt, gamma, vocab, accepted_len, out_tokens, row_argmax, false, nullptr, 0,
                     err_word, stream);
}

size_t simsd_accept_workspace_bytes(int Bt, int gamma, int vocab) {
  if (Bt <= 0 || gamma < 1 || gamma > 32 || vocab < 1 || vocab > (1 << 28)) return 0;
  DeviceInfo info;
  if (require_sm103(&info) != SIMSD_OK) return 0;
  return simsd::accept_workspace_bytes(Bt, gamma, vocab, info.num_sms);
}

int simsd_accept_ws(const float* logits, const int32_t* draft, int Bt, int gamma, int vocab, int32_t* accepted_len,
                    int32_t* out_tokens, int32_t* row_argmax, void* workspace, size_t workspace_bytes,
                    int32_t* err_word, void* stream) {
  return accept_impl(logits, draft, Bt, gamma, vocab, accepted_len, out_tokens, row_argmax, true, workspace,
                     workspace_bytes, err_word, stream);
}

namespace {

int accept_sampled_impl(const float* target_logits, const float* draft_logits, const int32_t* draft,
                        const float* u_accept, const float* u_sample, float temperature, int Bt, int gamma, int vocab,
                        int32_t* accepted_len, int32_t* out_tokens, bool ws_ok, void* workspace,
                        size_t workspace_bytes, int32_t* err_word, void* stream) {
  if (Bt < 0) return arg_fail("Bt < 0");
  if (gamma < 1 || gamma > 32) return arg_fail("gamma must be in [1, 32]");
  if (vocab < 1 || vocab > (1 << 24)) return arg_fail("vocab must be in [1, 2^24]");
  if (!(temperature > 0.f) || std::isinf(temperature)) return arg_fail("temperature must be positive and finite");
  if (Bt == 0) return SIMSD_OK;
  if (!target_logits || !draft_logits || !draft || !u_accept || !u_sample || !accepted_len || !out_tokens)
    return arg_fail("null pointer");
  DeviceInfo info;
  int rc = require_sm103(&info);
  if (rc != SIMSD_OK) return rc;
  const size_t need = ws_ok ? simsd::samp_workspace_bytes(Bt, gamma, vocab, info.num_sms) : 0;
  if (need > 0) {
    if (!workspace || workspace_bytes < need)
      return arg_fail("workspace smaller than simsd_accept_sampled_workspace_bytes()");
    if ((reinterpret_cast<uintptr_t>(workspace) & 7u) != 0) return arg_fail("workspace not 8-byte aligned");
  }
  cudaError_t e = simsd::launch_accept_sampled(target_logits, draft_logits, draft, u_accept, u_sample, temperature,
                                               Bt, gamma, vocab, accepted_len, out_tokens, err_word,
                                               as_stream(stream), need > 0 ? workspace : nullptr, info.num_sms);
  return e == cudaSuccess ? SIMSD_OK : cuda_fail(e, "accept_sampled launch");
}

}  // namespace

int simsd_accept_sampled(const float* target_logits, const float* draft_logits, const int32_t* draft,
                         const float* u_accept, const float* u_sample, float temperature, int Bt, int gamma,
                         int vocab, int32_t* accepted_len, int32_t* out_tokens, int32_t* err_word, void* stream) {
  return accept_sampled_impl(target_logits, draft_logits, draft, u_accept, u_sample, temperature, Bt, gamma, vocab,
                             accepted_len, out_tokens, false, nullptr, 0, err_word, stream);
}

size_t simsd_accept_sampled_workspace_bytes(int Bt, int gamma, int vocab) {
  if (Bt <= 0 || gamma < 1 || gamma > 32 || vocab < 1 || vocab > (1 << 24)) return 0;
  DeviceInfo info;
  if (require_sm103(&info) != SIMSD_OK) return 0;
  return simsd::samp_workspace_bytes(Bt, gamma, vocab, info.num_sms);
}

int simsd_plan_attention(int dtype, int Bt, int gamma, int Hq, int Hkv, int d, int max_pages, int page_size,
                         int num_sms, int32_t* plan, size_t* ws_bytes) {
  if (!plan || !ws_bytes || num_sms < 1) return arg_fail("null output or num_sms < 1");
  if (Bt < 0 || gamma < 1 || gamma > 32 || Hq <= 0 || Hkv <= 0 || Hq % Hkv != 0 || max_pages < 0 ||
      page_size <= 0)
    return arg_fail("sizes out of range");
  for (int i = 0; i < 5; ++i) plan[i] = 0;
  *ws_bytes = 0;
  if (dtype == SIMSD_F32) {
    if (d != 64 && d != 128) return unsupported("fp32 path needs d = 64 or 128");
    plan[0] = 2;
    plan[1] = 1;
    plan[3] = 2 * gamma * (Hq / Hkv);
    return SIMSD_OK;
  }
  if (dtype != SIMSD_BF16) return unsupported("dtype");
  if (d != 128) return unsupported("bf16 path needs d = 128");
  simsd::AttnTcPlan pl;
  if (!simsd::plan_attention_tc(Bt > 0 ? Bt : 1, gamma, Hq, Hkv, max_pages, page_size, num_sms, &pl))
    return unsupported("query rows per KV head: need 2*gamma*Hq/Hkv <= 128 or 128 % (Hq/Hkv) == 0");
  plan[0] = pl.kind;
  plan[1] = pl.nsplit;
  plan[2] = pl.streamk;
  plan[3] = pl.rows_blk;
  plan[4] = pl.fuse;
  *ws_bytes = Bt > 0 ? pl.ws_bytes : 0;
  return SIMSD_OK;
}

int simsd_plan_accept(int sampled, int Bt, int gamma, int vocab, int num_sms, int32_t* parts, size_t* ws_bytes) {
  if (!parts || !ws_bytes || num_sms < 1) return arg_fail("null output or num_sms < 1");
  if (Bt < 0 || gamma < 1 || gamma > 32 || vocab < 1 || vocab > (sampled ? (1 << 24) : (1 << 28)))
    return arg_fail("sizes out of range");
  *parts = 0;
  *ws_bytes = 0;
  if (Bt == 0) return SIMSD_OK;
  *parts = sampled ? simsd::samp_parts(Bt, gamma, vocab, num_sms) : simsd::accept_parts(Bt, gamma, vocab, num_sms);
  *ws_bytes = sampled ? simsd::samp_workspace_bytes(Bt, gamma, vocab, num_sms)
                      : simsd::accept_workspace_bytes(Bt, gamma, vocab, num_sms);
  return SIMSD_OK;
}

int simsd_accept_sampled_ws(const float* target_logits, const float* draft_logits, const int32_t* draft,
                            const float* u_accept, const float* u_sample, float temperature, int Bt, int gamma,
                            int vocab, int32_t* accepted_len, int32_t* out_tokens, void* workspace,
                            size_t workspace_bytes, int32_t* err_word, void* stream) {
  return accept_sampled_impl(target_logits, draft_logits, draft, u_accept, u_sample, temperature, Bt, gamma, vocab,
                             accepted_len, out_tokens, true, workspace, workspace_bytes, err_word, stream);
}

int simsd_kv_commit(int dtype, const void* k_new, const void* v_new, int L, const int32_t* tau,
                    const uint8_t* section, const int32_t* rope_pos, float rope_theta, const int32_t* accepted_len,
                    void* k_cache, void* v_cache, int num_pages, const int32_t* block_table, int max_pages,
                    int page_size, int32_t* prefix_len, int Bt, int gamma, int Hkv, int d, int32_t* err_word,
                    void* stream) {
  if (Bt < 0 || L < 0) return arg_fail("Bt < 0 or L < 0");
  if (gamma < 1 || gamma > 32) return arg_fail("gamma must be in [1, 32]");
  if (Hkv <= 0 || page_size <= 0 || num_pages < 0 || max_pages < 0) return arg_fail("sizes");
  if (dtype != SIMSD_F32 && dtype != SIMSD_BF16) return unsupported("dtype");
  const int eb = dtype == SIMSD_F32 ? 4 : 2;
  if (d <= 0 || (d * eb) % 16 != 0) return arg_fail("d * element size must be a multiple of 16 bytes");
  if (rope_pos && (!(rope_theta > 0.f) || std::isinf(rope_theta) || d > 128 || d % 2 != 0))
    return arg_fail("rope needs a positive finite rope_theta and an even d <= 128");
  if (Bt == 0) return SIMSD_OK;
  if (!tau || !section || !accepted_len || !prefix_len) return arg_fail("null pointer");
  if (L > 0 && (!k_new || !v_new || !k_cache || !v_cache || !block_table)) return arg_fail("null pointer");
  if ((k_new && !aligned16(k_new)) || (v_new && !aligned16(v_new)) || (k_cache && !aligned16(k_cache)) ||
      (v_cache && !aligned16(v_cache)))
    return arg_fail("tensor pointers must be 16-byte aligned");
  DeviceInfo info;
  int rc = require_sm103(&info);
  if (rc != SIMSD_OK) return rc;
  const simsd::RopeTable table = rope_pos ? simsd::make_rope_table(rope_theta, d) : simsd::RopeTable{};
  cudaError_t e = simsd::launch_kv_commit(eb, k_new, v_new, L, tau, section, accepted_len, k_cache, v_cache,
                                          num_pages, block_table, max_pages, page_size, prefix_len, Bt, gamma, Hkv,
                                          d, rope_pos, table, err_word, as_stream(stream));
  return e == cudaSuccess ? SIMSD_OK : cuda_fail(e, "kv_commit launch");
}

int simsd_rope_plan_init(simsd_rope_plan* plan, int layout, int rot_dim, double theta, int scaling, double factor,
                         int context, double beta_fast, double beta_slow) {
  if (!plan) return arg_fail("null plan");
  if (layout != SIMSD_ROPE_HALF && layout != SIMSD_ROPE_INTERLEAVED) return arg_fail("layout");
  if (rot_dim < 2 || rot_dim > 128 || rot_dim % 2 != 0) return arg_fail("rot_dim must be even, 2 .. 128");
  if (!(theta > 0.0) || std::isinf(theta)) return arg_fail("theta must be positive and finite");
  if (scaling < SIMSD_ROPE_UNSCALED || scaling > SIMSD_ROPE_YARN) return arg_fail("scaling");
  if (scaling != SIMSD_ROPE_UNSCALED && (!(factor >= 1.0) || std::isinf(factor)))
    return arg_fail("factor must be at least 1 and finite");
  if (scaling == SIMSD_ROPE_NTK && rot_dim == 2) return arg_fail("NTK scaling needs rot_dim > 2");
  if (scaling == SIMSD_ROPE_YARN &&
      (context <= 0 || !(beta_slow >= 0.0) || !(beta_fast > beta_slow) || std::isinf(beta_fast)))
    return arg_fail("YARN needs a positive context and beta_fast > beta_slow >= 0");
  const double kTwoPi = 6.283185307179586476925286766559;
  const double r = rot_dim;
  if (scaling == SIMSD_ROPE_NTK) theta *= std::pow(factor, r / (r - 2.0));
  std::memset(plan, 0, sizeof(*plan));
  plan->layout = layout;
  plan->rot_dim = rot_dim;
  plan->magnitude = scaling == SIMSD_ROPE_YARN ? static_cast<float>(0.1 * std::log(factor) + 1.0) : 1.0f;
  for (int i = 0; i < rot_dim / 2; ++i) {
    double f = std::pow(theta, -2.0 * i / r);
    if (scaling == SIMSD_ROPE_LINEAR) f /= factor;
    if (scaling == SIMSD_ROPE_YARN) {
      const double rho = context * f / kTwoPi;
      const double g = std::fmin(1.0, std::fmax(0.0, (rho - beta_slow) / (beta_fast - beta_slow)));
      f = (1.0 - g) * f / factor + g * f;
    }
    // whole turns of a position (theta < 1 only) do not change the angle
    double turns = f / kTwoPi;
    turns -= std::floor(turns);
    const double scaled = std::nearbyint(std::ldexp(turns, 64));
    plan->turn[i] = scaled >= 18446744073709551616.0 ? 0 : static_cast<uint64_t>(scaled);
  }
  return SIMSD_OK;
}

namespace {

int check_rope_plan(const simsd_rope_plan* plan, int d) {
  if (!plan) return arg_fail("null plan");
  if ((plan->layout != SIMSD_ROPE_HALF && plan->layout != SIMSD_ROPE_INTERLEAVED) || plan->rot_dim < 2 ||
      plan->rot_dim > 128 || plan->rot_dim % 2 != 0 || !(plan->magnitude > 0.f) || std::isinf(plan->magnitude) ||
      plan->reserved != 0)
    return arg_fail("plan not made by simsd_rope_plan_init");
  if (plan->rot_dim > d) return arg_fail("rot_dim larger than the head");
  return SIMSD_OK;
}

// a [T][H][d] array with dense heads and the given token stride
bool rows_ok(const void* p, int64_t stride, int H, int d, int eb) {
  return p && aligned16(p) && stride >= static_cast<int64_t>(H) * d && stride * eb % 16 == 0;
}

// token numbers, rounded up to a block of tokens, stay within 32 bits
constexpr int kMaxRopeTokens = 0x7fffff00;

bool page_size_ok(int P) { return P >= 8 && (P % 64 == 0 || 64 % P == 0); }

}  // namespace

int simsd_rope_rotate(int dtype, const simsd_rope_plan* plan, const int32_t* positions, const void* q,
                      int64_t q_stride, void* q_out, int64_t q_out_stride, int Hq, const void* k, int64_t k_stride,
                      void* k_out, int64_t k_out_stride, int Hkv, int T, int d, void* stream) {
  if (dtype != SIMSD_F32 && dtype != SIMSD_BF16) return unsupported("dtype");
  const int eb = dtype == SIMSD_F32 ? 4 : 2;
  if (T < 0 || Hq <= 0 || Hkv < 0 || d <= 0) return arg_fail("sizes");
  if ((d * eb) % 16 != 0) return arg_fail("d * element size must be a multiple of 16 bytes");
  int rc = check_rope_plan(plan, d);
  if (rc != SIMSD_OK) return rc;
  if (T > kMaxRopeTokens) return unsupported("too many tokens");
  if (T == 0) return SIMSD_OK;
  if (!positions) return arg_fail("null pointer");
  if (!rows_ok(q, q_stride, Hq, d, eb) || !rows_ok(q_out, q_out_stride, Hq, d, eb))
    return arg_fail("q / q_out: null, misaligned or overlapping rows");
  if (Hkv > 0 ? !rows_ok(k, k_stride, Hkv, d, eb) || !rows_ok(k_out, k_out_stride, Hkv, d, eb) : (k || k_out))
    return arg_fail("k / k_out: null, misaligned or overlapping rows, or Hkv = 0");
  DeviceInfo info;
  rc = require_sm103(&info);
  if (rc != SIMSD_OK) return rc;
  simsd::RopeArgs a{};
  a.plan = *plan;
  a.positions = positions;
  a.q = q;
  a.q_stride = q_stride;
  a.q_out = q_out;
  a.q_out_stride = q_out_stride;
  a.k = k;
  a.k_stride = k_stride;
  a.k_out = k_out;
  a.k_out_stride = k_out_stride;
  a.T = T;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.d = d;
  cudaError_t e = simsd::launch_rope(eb, a, info.num_sms, as_stream(stream));
  return e == cudaSuccess ? SIMSD_OK : cuda_fail(e, "rope_rotate launch");
}

int simsd_rope_append(int dtype, const simsd_rope_plan* plan, const void* q, int64_t q_stride, const void* k,
                      int64_t k_stride, const void* v, int64_t v_stride, const int32_t* token_start,
                      const int32_t* prefix_len, const int32_t* positions, int T, int Bt, int Hq, int Hkv, int d,
                      void* q_out, void* k_cache, void* v_cache, int num_pages, const int32_t* block_table,
                      int max_pages, int page_size, int32_t* err_word, void* stream) {
  if (dtype != SIMSD_F32 && dtype != SIMSD_BF16) return unsupported("dtype");
  const int eb = dtype == SIMSD_F32 ? 4 : 2;
  if (T < 0 || Bt < 0 || Hq <= 0 || Hkv <= 0 || d <= 0 || num_pages < 0 || max_pages < 0 || page_size <= 0)
    return arg_fail("sizes");
  if ((d * eb) % 16 != 0) return arg_fail("d * element size must be a multiple of 16 bytes");
  if (static_cast<long long>(max_pages) * page_size > 0x7fffff00ll) return unsupported("more than 2^31 rows a sequence");
  int rc = check_rope_plan(plan, d);
  if (rc != SIMSD_OK) return rc;
  if (T > kMaxRopeTokens) return unsupported("too many tokens");
  if (T == 0 || Bt == 0) return SIMSD_OK;
  if (!token_start || !prefix_len || !block_table || !k_cache || !v_cache) return arg_fail("null pointer");
  if (!rows_ok(q, q_stride, Hq, d, eb) || !rows_ok(k, k_stride, Hkv, d, eb) || !rows_ok(v, v_stride, Hkv, d, eb))
    return arg_fail("q / k / v: null, misaligned or overlapping rows");
  if (!q_out || !aligned16(q_out) || !aligned16(k_cache) || !aligned16(v_cache))
    return arg_fail("tensor pointers must be 16-byte aligned");
  DeviceInfo info;
  rc = require_sm103(&info);
  if (rc != SIMSD_OK) return rc;
  simsd::RopeArgs a{};
  a.plan = *plan;
  a.q = q;
  a.q_stride = q_stride;
  a.k = k;
  a.k_stride = k_stride;
  a.v = v;
  a.v_stride = v_stride;
  a.q_out = q_out;
  a.q_out_stride = static_cast<long long>(Hq) * d;
  a.k_cache = k_cache;
  a.v_cache = v_cache;
  a.token_start = token_start;
  a.prefix_len = prefix_len;
  a.positions = positions;
  a.block_table = block_table;
  a.err_word = err_word;
  a.T = T;
  a.Bt = Bt;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.d = d;
  a.num_pages = num_pages;
  a.max_pages = max_pages;
  a.page_size = page_size;
  cudaError_t e = simsd::launch_rope(eb, a, info.num_sms, as_stream(stream));
  return e == cudaSuccess ? SIMSD_OK : cuda_fail(e, "rope_append launch");
}

size_t simsd_chunk_workspace_bytes(int dtype, int T, int Bt, int Hq, int Hkv, int d, int max_pages, int page_size) {
  if ((dtype != SIMSD_BF16 && dtype != SIMSD_F32) || T <= 0 || Bt <= 0 || Hq <= 0 || Hkv <= 0 || Hq % Hkv != 0 ||
      (d != 64 && d != 128) || max_pages < 0 || page_size <= 0)
    return 0;
  DeviceInfo info;
  if (device_info(&info) != SIMSD_OK) return 0;
  if (dtype == SIMSD_F32)
    return simsd::chunk_f32_workspace_bytes(T, Bt, Hq, Hkv, d, static_cast<long long>(max_pages) * page_size,
                                            info.num_sms);
  return simsd::chunk_tc_workspace_bytes(T, Bt, d, info.num_sms);
}

int simsd_chunk_attention(int dtype, const void* q, int64_t q_stride, const int32_t* token_start,
                          const int32_t* prefix_len, const int32_t* key_start, const void* k_cache,
                          const void* v_cache, int num_pages, const int32_t* block_table, int max_pages,
                          int page_size, int T, int Bt, int Hq, int Hkv, int d, int mask_block, int window,
                          float softmax_scale, void* out, float* lse, void* workspace, size_t workspace_bytes,
                          int32_t* err_word, void* stream) {
  if (dtype != SIMSD_F32 && dtype != SIMSD_BF16) return unsupported("dtype");
  const int eb = dtype == SIMSD_F32 ? 4 : 2;
  if (T < 0 || Bt < 0) return arg_fail("T < 0 or Bt < 0");
  if (Hq <= 0 || Hkv <= 0 || Hq % Hkv != 0) return arg_fail("Hq must be a positive multiple of Hkv");
  if (num_pages < 0 || max_pages < 0 || mask_block < 0 || window < 0) return arg_fail("negative size");
  if (!page_size_ok(page_size)) return unsupported("page_size must be a multiple of 64 or a divisor of 64 (>= 8)");
  if (d != 64 && d != 128) return unsupported("d must be 64 or 128");
  if (!(softmax_scale >= 0.f) || std::isinf(softmax_scale)) return arg_fail("softmax_scale");
  if (static_cast<long long>(max_pages) * page_size > 0x7fffff00ll) return unsupported("more than 2^31 rows a sequence");
  if (static_cast<long long>(T) * Hq >= (1ll << 31)) return unsupported("too many query rows");
  if (T == 0 || Bt == 0) return SIMSD_OK;
  if (!token_start || !prefix_len || !block_table || !k_cache || !v_cache || !out) return arg_fail("null pointer");
  if (num_pages == 0 || max_pages == 0) return arg_fail("no pages");
  if (!rows_ok(q, q_stride, Hq, d, eb)) return arg_fail("q: null, misaligned or overlapping rows");
  if (!aligned16(k_cache) || !aligned16(v_cache) || !aligned16(out))
    return arg_fail("tensor pointers must be 16-byte aligned");
  DeviceInfo info;
  int rc = require_sm103(&info);
  if (rc != SIMSD_OK) return rc;
  simsd::ChunkArgs a{};
  a.q = q;
  a.q_stride = q_stride;
  a.token_start = token_start;
  a.prefix_len = prefix_len;
  a.key_start = key_start;
  a.k_cache = k_cache;
  a.v_cache = v_cache;
  a.block_table = block_table;
  a.out = out;
  a.lse = lse;
  a.err_word = err_word;
  a.T = T;
  a.Bt = Bt;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.d = d;
  a.num_pages = num_pages;
  a.max_pages = max_pages;
  a.page_size = page_size;
  a.mask_block = mask_block;
  a.window = window;
  a.scale = softmax_scale > 0.f ? softmax_scale : 1.0f / std::sqrt(static_cast<float>(d));
  const long long max_keys = static_cast<long long>(max_pages) * page_size;
  const size_t need = dtype == SIMSD_F32
                          ? simsd::chunk_f32_workspace_bytes(T, Bt, Hq, Hkv, d, max_keys, info.num_sms)
                          : simsd::chunk_tc_workspace_bytes(T, Bt, d, info.num_sms);
  if (need > 0 && (!workspace || workspace_bytes < need || !aligned16(workspace)))
    return arg_fail("workspace smaller than simsd_chunk_workspace_bytes()");
  a.workspace = workspace;
  if (dtype == SIMSD_F32) {
    cudaError_t e = simsd::launch_chunk_attention_f32(a, info.num_sms, as_stream(stream));
    return e == cudaSuccess ? SIMSD_OK : cuda_fail(e, "chunk_attention_f32 launch");
  }
  if (Hq / Hkv > 128) return unsupported("Hq / Hkv above 128");
  if (Bt > simsd::kChunkMaxSeqs) return unsupported("more than 16384 sequences");
  if (static_cast<long long>(num_pages) * Hkv * page_size >= (1ll << 31))
    return unsupported("page pool too large for 32-bit TMA row coordinates");
  // key tiles are counted in 32 bits (2^31 of them take some 20 s)
  if ((static_cast<long long>(T) * Hq / 128 + static_cast<long long>(Bt) * Hkv + 1) * (max_keys / 128 + 1) >= (1ll << 31))
    return unsupported("too many key tiles in one call");
  simsd::EncodeTiledFn enc = encoder();
  if (!enc) return cuda_fail(cudaErrorNotSupported, "cuTensorMapEncodeTiled entry point");
  cudaError_t e = simsd::launch_chunk_attention_tc(a, info.num_sms, enc, as_stream(stream));
  return e == cudaSuccess ? SIMSD_OK : cuda_fail(e, "chunk_attention_tc launch");
}

int simsd_sample(int dtype, const void* logits, int64_t row_stride, int R, int vocab, const float* u,
                 const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                 int32_t* token, int32_t* kept, float* log_prob, float* log_probs, int32_t* err_word, void* stream) {
  if (dtype != SIMSD_F32 && dtype != SIMSD_BF16) return unsupported("dtype");
  if (R < 0) return arg_fail("R < 0");
  if (vocab < 1 || vocab > (1 << 24)) return arg_fail("vocab must be in [1, 2^24]");
  if (row_stride < vocab) return arg_fail("row_stride smaller than the vocabulary");
  if (R == 0) return SIMSD_OK;
  if (!logits || !u || !token) return arg_fail("null pointer");
  if (!aligned16(logits) || (log_probs && !aligned16(log_probs)))
    return arg_fail("tensor pointers must be 16-byte aligned");
  DeviceInfo info;
  int rc = require_sm103(&info);
  if (rc != SIMSD_OK) return rc;
  simsd::SampleArgs a{};
  a.logits = logits;
  a.row_stride = row_stride;
  a.R = R;
  a.V = vocab;
  a.u = u;
  a.temperature = temperature;
  a.top_k = top_k;
  a.top_p = top_p;
  a.min_p = min_p;
  a.token = token;
  a.kept = kept;
  a.log_prob = log_prob;
  a.log_probs = log_probs;
  a.err_word = err_word;
  cudaError_t e = simsd::launch_sample(dtype == SIMSD_F32 ? 4 : 2, a, info.num_sms, as_stream(stream));
  return e == cudaSuccess ? SIMSD_OK : cuda_fail(e, "sample launch");
}

int simsd_debug_expire_next_wait(int which, unsigned int limit_us) {
  if (which != SIMSD_DEBUG_WAIT_ATTENTION && which != SIMSD_DEBUG_WAIT_ACCEPT) return arg_fail("which");
  if (limit_us < 10 || limit_us > 1000000) return arg_fail("limit_us must be in [10, 10^6]");
  g_armed[which].extra = 1;
  g_armed[which].wait_ns = 1000ull * limit_us;
  return SIMSD_OK;
}

int simsd_check_error(const int32_t* err_word, int32_t* host_word, void* stream) {
  if (!err_word) return arg_fail("null error word");
  int32_t w = 0;
  cudaError_t e = cudaMemcpyAsync(&w, err_word, sizeof(w), cudaMemcpyDeviceToHost, as_stream(stream));
  if (e == cudaSuccess) e = cudaStreamSynchronize(as_stream(stream));
  if (e != cudaSuccess) return cuda_fail(e, "check_error");
  if (host_word) *host_word = w;
  return w ? SIMSD_ERR_DEVICE : SIMSD_OK;
}

}  // extern "C"
