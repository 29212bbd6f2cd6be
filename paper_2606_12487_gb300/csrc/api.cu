// api.cu -- the C ABI of include/dptq.h: argument checks, the layer handle, the
// per-device scratch, and the launch sequence of each call.  No compute happens here: the
// kernels are in rotate_quant.cu and qgemm.cu (the linear layer), kv_policy.cu (KV4, the
// policy), norm_quant.cu, rotary.cu, kv8_*.cu and kv4_*.cu (the operators around the layer).
#include <cmath>
#include <cstdint>
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <atomic>
#include <map>
#include <mutex>
#include <set>
#include <utility>
#include <string>
#include <vector>

#include <cuda_runtime.h>
#include <nvtx3/nvToolsExt.h>

#include "../../include/dptq.h"
#include "dptq_device.cuh"
#include "dptq_internal.h"

using namespace dptq;

namespace {

thread_local std::string g_msg;

dptq_status fail(dptq_status st, const std::string& m) {
  g_msg = m;
  return st;
}
dptq_status cuda_fail(cudaError_t e, const char* where) {
  g_msg = std::string(where) + ": " + cudaGetErrorString(e);
  return e == cudaErrorMemoryAllocation ? DPTQ_ERR_OOM : DPTQ_ERR_CUDA;
}
#define DPTQ_CUDA(call, where)                      \
  do {                                              \
    cudaError_t e_ = (call);                        \
    if (e_ != cudaSuccess) return cuda_fail(e_, where); \
  } while (0)

bool is_pow2(int v) { return v > 0 && (v & (v - 1)) == 0; }

bool is_prime_int(int v) {
  if (v < 2) return false;
  for (int d = 2; d * d <= v; ++d)
    if (v % d == 0) return false;
  return true;
}

// A tail block of r elements is r = p 2^k: p = 1 for a power of two; otherwise p is the
// smallest Paley order (odd part of r times 2^m, m >= 2, with p - 1 prime) that divides r,
// and the tail's Hadamard matrix is H_p (x) H_(2^k) with H_p from Paley's first
// construction.  False when r is neither.
bool tail_factor(int r, int& p, int& k) {
  if (r <= 0) return false;
  if (is_pow2(r)) {
    p = 1;
    k = 0;
    while ((1 << k) < r) ++k;
    return true;
  }
  int tz = 0;
  while (((r >> tz) & 1) == 0) ++tz;
  const int odd = r >> tz;
  for (int m = 2; m <= tz; ++m) {
    if (is_prime_int((odd << m) - 1)) {
      p = odd << m;
      k = tz - m;
      return true;
    }
  }
  return false;
}

// Block layout of R along K: nfull blocks of B then a tail (or none) that is a power of
// two or a Paley order times a power of two.
bool hadamard_layout(int K, int B, int& nfull, int& tail, int& log2B) {
  if (!is_pow2(B) || K <= 0) return false;
  nfull = K / B;
  tail = K % B;
  int p, k;
  if (tail != 0 && !tail_factor(tail, p, k)) return false;
  log2B = 0;
  while ((1 << log2B) < B) ++log2B;
  return true;
}

// Elements per rotation pass: whole blocks, at least 4096 elements when K allows.
int rq_chunk(int K, int B) {
  int c = B;
  while (c < 4096 && c < K) c += B;
  return c < K ? c : K;
}

// Whether K's tail block is a power of two (or absent); the fused decode launch and the
// whole-row kernel handle only those.
bool pow2_tail(int K, int B) { return K % B == 0 || is_pow2(K % B); }

dptq_status check_shape(int K, int B, int& nfull, int& tail, int& log2B) {
  if (K % 32 != 0) return fail(DPTQ_ERR_UNSUPPORTED, "K must be a multiple of 32");
  if (B > 4096) return fail(DPTQ_ERR_UNSUPPORTED, "had_block above 4096 is not supported");
  if (!hadamard_layout(K, B, nfull, tail, log2B))
    return fail(DPTQ_ERR_UNSUPPORTED,
                "K must split into blocks of had_block (a power of two) plus a tail that is a power of two or a "
                "Paley order times a power of two");
  int p = 1, k = 0;
  if (tail != 0 && !is_pow2(tail)) {
    tail_factor(tail, p, k);
    if (p > 256) return fail(DPTQ_ERR_UNSUPPORTED, "the tail block's Paley order is above 256");
    // The tail must lie in the last 4096-element rotation pass.
    if (nfull * B < ((K - 1) / 4096) * 4096)
      return fail(DPTQ_ERR_UNSUPPORTED, "a non-power-of-two tail must lie in the last 4096 elements of K");
  }
  if (rotate_quant_smem(K, rq_chunk(K, B)) > kSmemPerBlock)
    return fail(DPTQ_ERR_UNSUPPORTED, "K and had_block exceed the shared memory of one CTA");
  return DPTQ_OK;
}

RQArgs make_rq(const void* x, int rows_in, int rows_out, int K, int KB, int B, int nfull, int tail, int log2B,
               int bits, float* scales, void* out) {
  RQArgs a{};
  a.x = static_cast<const __half*>(x);
  a.rows_in = rows_in;
  a.rows_out = rows_out;
  a.K = K;
  a.KB = KB;
  a.B = B;
  a.log2B = log2B;
  a.nfull = nfull;
  a.tail = tail;
  a.log2T = 0;
  a.tail_p = 1;
  a.tail_j = 0;
  int p = 1, k = 0;
  if (tail && tail_factor(tail, p, k)) {
    a.log2T = k;
    a.tail_p = p;
    if (p > 1) {   // y = S 2^-24 / sqrt(p 2^k) = S 2^-(24 + k/2) / sqrt(p 2^(k mod 2))
      const double t = 1.0 / std::sqrt((double)p * (double)(1 << (k & 1)));
      a.tail_j = k >> 1;
      a.t_hi = (float)t;
      a.t_lo = (float)(t - (double)a.t_hi);
    }
  }
  a.chunk = rq_chunk(K, B);
  const double r2 = 1.0 / std::sqrt(2.0);
  a.c_hi = (float)r2;
  a.c_lo = (float)(r2 - (double)a.c_hi);
  a.bits = bits;
  a.scales = scales;
  a.out = out;
  return a;
}

// Per-device scratch shared by the online calls: E4M3 activation planes, per-token
// scales, split-tile partial sums and their counters, and the device error word.
// Activation planes and scales grow on demand.  A buffer that growth supersedes is never
// freed: work enqueued earlier, or captured into a CUDA graph, may still read or write
// it, so it stays allocated (in `retired`) until the process exits.  Growth is geometric
// (at least doubling), so the retired buffers together hold less than the live ones.
struct Scratch {
  uint8_t* act = nullptr;
  size_t act_bytes = 0;
  float* sa = nullptr;
  size_t sa_count = 0;
  int32_t* ws = nullptr;
  // [SMs] split-tile arrivals, [2] fused-launch grid counters, then (128-byte aligned)
  // the row-maximum slots of the fused launch's row parts, [64][kRowMaxStride]
  uint32_t* counters = nullptr;
  size_t counter_words = 0;
  uint32_t* gsync = nullptr;
  uint32_t* pmax = nullptr;
  int* err = nullptr;                 // [2] device error words: waits that gave up; KV8 arrays out of range
  int num_sms = 0;
  float* kv8_ws = nullptr;            // partial attention results and their arrival counters,
  uint32_t* kv8_counters = nullptr;   // from the first attention call or dptq_kv8_reserve on
  std::vector<std::pair<void*, size_t>> retired;   // superseded act / sa buffers, still allocated
};
std::mutex g_mu;
std::map<int, Scratch> g_scratch;

bool capturing(cudaStream_t s) {
  cudaStreamCaptureStatus st = cudaStreamCaptureStatusNone;
  if (cudaStreamIsCapturing(s, &st) != cudaSuccess) return false;
  return st != cudaStreamCaptureStatusNone;
}

constexpr int kMaxNT = 256;
// Rows of up to 16384 elements take the fused launch (at most two CTAs of 8 warps a row,
// 1024 elements a warp).
constexpr int kFusedMaxKPad = 16384;
// Counter words: split-tile arrivals and grid counters, then the row-maximum slots, one
// 128-byte line per row (only the parts of one row poll a line).
size_t pmax_offset(int sms) { return ((size_t)sms + 2 + 31) & ~(size_t)31; }
size_t counter_words(int sms) { return pmax_offset(sms) + (size_t)64 * kRowMaxStride; }

// Every device allocation of the library goes through here.  Host-side fault injection
// for tests of the out-of-memory path: with DPTQ_FAULT_ALLOC=n (n >= 1) in the
// environment, the n-th allocation the library attempts in this process fails as
// cudaErrorMemoryAllocation without calling cudaMalloc.
cudaError_t dev_malloc(void** p, size_t bytes) {
  static const long long fail_at = [] {
    const char* v = std::getenv("DPTQ_FAULT_ALLOC");
    return v ? std::atoll(v) : 0LL;
  }();
  static long long n = 0;
  if (fail_at > 0 && ++n == fail_at) {
    *p = nullptr;
    return cudaErrorMemoryAllocation;
  }
  return cudaMalloc(p, bytes);
}

// Make sure the device's scratch holds `act_bytes` of activation planes and `sa_count`
// scales.  Growth allocates, so it is refused while `s` is being captured.
dptq_status ensure_scratch(int dev, size_t act_bytes, size_t sa_count, cudaStream_t s, Scratch** out) {
  std::lock_guard<std::mutex> lk(g_mu);
  Scratch& sc = g_scratch[dev];
  const bool grow_act = act_bytes > sc.act_bytes;
  const bool grow_sa = sa_count > sc.sa_count;
  const bool first = sc.err == nullptr;
  if ((grow_act || grow_sa || first) && capturing(s))
    return fail(DPTQ_ERR_UNSUPPORTED, "scratch must grow during stream capture: call dptq_reserve first");
  if (first) {
    int sms = 0;
    DPTQ_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev), "cudaDeviceGetAttribute");
    const size_t ws_bytes = (size_t)sms * kMaxNT * 128 * sizeof(int32_t);
    int32_t* ws = nullptr;
    uint32_t* counters = nullptr;
    int* err = nullptr;
    cudaError_t e = dev_malloc(reinterpret_cast<void**>(&ws), ws_bytes);
    if (e == cudaSuccess) e = dev_malloc(reinterpret_cast<void**>(&counters), sizeof(uint32_t) * counter_words(sms));
    if (e == cudaSuccess) e = dev_malloc(reinterpret_cast<void**>(&err), 2 * sizeof(int));
    if (e == cudaSuccess) e = cudaMemset(ws, 0, ws_bytes);
    if (e == cudaSuccess) e = cudaMemset(counters, 0, sizeof(uint32_t) * counter_words(sms));
    if (e == cudaSuccess) e = cudaMemset(err, 0, 2 * sizeof(int));
    if (e != cudaSuccess) {   // nothing has used these yet: release them and stay uninitialized
      if (ws) cudaFree(ws);
      if (counters) cudaFree(counters);
      if (err) cudaFree(err);
      return cuda_fail(e, "scratch allocation");
    }
    sc.counter_words = counter_words(sms);
    sc.pmax = counters + pmax_offset(sms);
    // DPTQ_MAX_GRID=n caps the CTAs of a GEMM launch (tuning experiments; default: the
    // device's SMs).
    if (const char* v = std::getenv("DPTQ_MAX_GRID")) {
      const int cap = std::atoi(v);
      if (cap > 0 && cap < sms) sms = cap;
    }
    sc.num_sms = sms;
    sc.ws = ws;
    sc.counters = counters;
    sc.gsync = counters + sms;
    sc.err = err;
  }
  if (grow_act) {
    const size_t bytes = std::max(act_bytes, 2 * sc.act_bytes);
    void* p = nullptr;
    DPTQ_CUDA(dev_malloc(&p, bytes), "cudaMalloc(act)");
    if (sc.act) sc.retired.emplace_back(sc.act, sc.act_bytes);
    sc.act = static_cast<uint8_t*>(p);
    sc.act_bytes = bytes;
  }
  if (grow_sa) {
    const size_t count = std::max(sa_count, 2 * sc.sa_count);
    void* p = nullptr;
    DPTQ_CUDA(dev_malloc(&p, sizeof(float) * count), "cudaMalloc(sa)");
    if (sc.sa) sc.retired.emplace_back(sc.sa, sizeof(float) * sc.sa_count);
    sc.sa = static_cast<float*>(p);
    sc.sa_count = count;
  }
  *out = &sc;
  return DPTQ_OK;
}

// The attention's part of the scratch, of a size that the device alone fixes.
dptq_status ensure_kv8_scratch(Scratch* sc, cudaStream_t s) {
  std::lock_guard<std::mutex> lk(g_mu);
  if (sc->kv8_ws) return DPTQ_OK;
  if (capturing(s)) return fail(DPTQ_ERR_UNSUPPORTED, "scratch must grow during stream capture: call dptq_kv8_reserve first");
  float* ws = nullptr;
  uint32_t* counters = nullptr;
  const size_t words = sizeof(uint32_t) * kv8_counter_words(sc->num_sms);
  cudaError_t e = dev_malloc(reinterpret_cast<void**>(&ws), kv8_ws_bytes(sc->num_sms));
  if (e == cudaSuccess) e = dev_malloc(reinterpret_cast<void**>(&counters), words);
  if (e == cudaSuccess) e = cudaMemset(counters, 0, words);
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  if (e != cudaSuccess) {
    if (ws) cudaFree(ws);
    if (counters) cudaFree(counters);
    return cuda_fail(e, "scratch allocation");
  }
  sc->kv8_ws = ws;
  sc->kv8_counters = counters;
  return DPTQ_OK;
}

dptq_status current_device(int* dev) {
  DPTQ_CUDA(cudaGetDevice(dev), "cudaGetDevice");
  return DPTQ_OK;
}

dptq_status check_handle(dptq_handle h, int* dev) {
  if (!h) return fail(DPTQ_ERR_INVALID_ARG, "null handle");
  dptq_status st = current_device(dev);
  if (st != DPTQ_OK) return st;
  if (*dev != h->device) return fail(DPTQ_ERR_INVALID_ARG, "handle belongs to another device than the current one");
  return DPTQ_OK;
}

// GEMM + epilogue from the E4M3 planes already in scratch.
dptq_status run_gemm(dptq_handle h, const GemmPlan& plan0, const uint8_t* act, const float* sa, void* out,
                     int32_t* acc, Scratch* sc, cudaStream_t s) {
  GemmPlan plan = plan0;
  GemmArgs& g = plan.args;
  g.wt = h->wt;
  g.act = act;
  g.sa = sa;
  g.sw = h->sw;
  g.out = static_cast<__half*>(out);
  g.out_vec = (reinterpret_cast<uintptr_t>(out) & 15u) == 0;
  g.acc_out = acc;
  g.ws = sc->ws;
  g.counters = sc->counters;
  g.gsync = sc->gsync;
  g.err = sc->err;
  g.wait_cycles = wait_cycles_setting();
  if (plan.fused) g.rq_shortfall = take_rows_shortfall();
  DPTQ_CUDA(launch_gemm(plan, s, true), "qgemm launch");
  return DPTQ_OK;
}

}  // namespace

namespace dptq {
bool pdl_allowed() {
  static const bool on = [] {
    const char* v = std::getenv("DPTQ_PDL");
    return !(v && v[0] == '0');
  }();
  return on;
}

// NVTX ranges named after the entry points, around every call that launches work, for
// timelines in NVIDIA's tools (DPTQ_NVTX=1; off by default, when a range costs one load).
bool nvtx_enabled() {
  static const bool on = [] {
    const char* v = std::getenv("DPTQ_NVTX");
    return v && v[0] == '1';
  }();
  return on;
}
struct NvtxRange {
  const bool on;
  explicit NvtxRange(const char* name) : on(nvtx_enabled()) {
    if (on) nvtxRangePushA(name);
  }
  ~NvtxRange() {
    if (on) nvtxRangePop();
  }
  NvtxRange(const NvtxRange&) = delete;
  NvtxRange& operator=(const NvtxRange&) = delete;
};

bool fused_allowed() {
  static const bool on = [] {
    const char* v = std::getenv("DPTQ_FUSED");
    return !(v && v[0] == '0');
  }();
  return on;
}

// Decode grids of one CTA per whole weight tile when the tiles fit the SMs (default), or,
// with DPTQ_DECODE_WHOLE_TILES=0, every SM with split tiles (tuning).
bool decode_whole_tiles() {
  static const bool on = [] {
    const char* v = std::getenv("DPTQ_DECODE_WHOLE_TILES");
    return !(v && v[0] == '0');
  }();
  return on;
}

// A8 prefill tiles: 192 tokens with the widened weights in tensor memory (default), or,
// with DPTQ_A8_TILE128=1, 128 tokens with the weights widened into shared memory.
bool a8_tile128() {
  static const bool on = [] {
    const char* v = std::getenv("DPTQ_A8_TILE128");
    return v && v[0] == '1';
  }();
  return on;
}

long long wait_cycles_setting() {
  static const long long v = [] {
    const char* e = std::getenv("DPTQ_WAIT_CYCLES");
    const long long c = e ? std::atoll(e) : 0LL;
    return c > 0 ? c : 2000000000LL;
  }();
  return v;
}

int take_rows_shortfall() {
  static std::atomic<int> left{[] {
    const char* e = std::getenv("DPTQ_TEST_ROWS_SHORTFALL");
    return e ? std::atoi(e) : 0;
  }()};
  return left.exchange(0);
}

// DPTQ_TEST_KV8_SHORTFALL=abc: the digits, one for each call of dptq_kv8_attention or dptq_kv4_attention.
int take_kv8_shortfall() {
  static const char* const v = std::getenv("DPTQ_TEST_KV8_SHORTFALL");
  if (v == nullptr) return 0;
  static std::atomic<size_t> calls{0};
  const size_t i = calls++;
  return i < std::strlen(v) ? v[i] - '0' : 0;
}

cudaError_t ensure_max_dyn_smem_impl(const void* fn) {
  // One entry per (kernel, device) whose ceiling is already raised.
  static std::mutex mu;
  static std::set<std::pair<const void*, int>> done;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  std::lock_guard<std::mutex> lk(mu);
  if (done.count({fn, dev})) return cudaSuccess;
  // The ceiling is the device's opt-in maximum per block less the kernel's static shared
  // memory.
  int optin = 0;
  e = cudaDeviceGetAttribute(&optin, cudaDevAttrMaxSharedMemoryPerBlockOptin, dev);
  if (e != cudaSuccess) return e;
  cudaFuncAttributes fa{};
  e = cudaFuncGetAttributes(&fa, fn);
  if (e != cudaSuccess) return e;
  e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, optin - (int)fa.sharedSizeBytes);
  if (e == cudaSuccess) done.insert({fn, dev});
  return e;
}

bool rows_kernel_allowed() {
  static const bool on = [] {
    const char* v = std::getenv("DPTQ_ROWS_KERNEL");
    return !(v && v[0] == '0');
  }();
  return on;
}

// Record the message returned by dptq_last_error_message for this thread.
void set_error_message(const std::string& m) { g_msg = m; }
}  // namespace dptq

extern "C" {

const char* dptq_status_str(dptq_status s) {
  switch (s) {
    case DPTQ_OK: return "ok";
    case DPTQ_ERR_INVALID_ARG: return "invalid argument";
    case DPTQ_ERR_UNSUPPORTED: return "unsupported shape";
    case DPTQ_ERR_CUDA: return "CUDA error";
    case DPTQ_ERR_OOM: return "out of device memory";
    case DPTQ_ERR_TIMEOUT: return "device wait timed out";
  }
  return "unknown status";
}

const char* dptq_last_error_message(void) { return g_msg.c_str(); }

namespace {
// Shared body of dptq_pack_weights and dptq_pack_weights_rh (signs_host null: plain).
dptq_status pack_weights_impl(const void* W_fp16, int N, int K, int had_block, const int8_t* signs_host,
                              int w_on_device, dptq_handle* out) {
  if (!W_fp16 || !out) return fail(DPTQ_ERR_INVALID_ARG, "null pointer");
  *out = nullptr;
  if (N <= 0 || K <= 0 || had_block <= 0) return fail(DPTQ_ERR_INVALID_ARG, "sizes must be positive");
  if (N % 16 != 0) return fail(DPTQ_ERR_UNSUPPORTED, "N must be a multiple of 16");
  int nfull, tail, log2B;
  dptq_status st = check_shape(K, had_block, nfull, tail, log2B);
  if (st != DPTQ_OK) return st;
  int dev;
  if ((st = current_device(&dev)) != DPTQ_OK) return st;

  dptq_linear* h = new dptq_linear{};
  h->device = dev;
  h->N = N;
  h->K = K;
  h->K_pad = round_up(K, kKPad);
  h->KB = h->K_pad / kKBlock;
  h->N_pad = round_up(N, 128);
  h->had_block = had_block;
  if (signs_host != nullptr) {
    for (int k = 0; k < K; ++k)
      if (signs_host[k] != 1 && signs_host[k] != -1) {
        delete h;
        return fail(DPTQ_ERR_INVALID_ARG, "signs must be +1 or -1");
      }
  }
  const size_t wt_bytes = (size_t)(h->N_pad / 128) * h->KB * kWTileBytes;
  void* tmp = nullptr;
  cudaError_t e = dev_malloc(reinterpret_cast<void**>(&h->wt), wt_bytes);
  if (e == cudaSuccess) e = dev_malloc(reinterpret_cast<void**>(&h->sw), sizeof(float) * h->N_pad);
  if (e == cudaSuccess && signs_host != nullptr) {
    e = dev_malloc(reinterpret_cast<void**>(&h->signs), (size_t)h->K_pad);
    if (e == cudaSuccess) e = cudaMemset(h->signs, 1, (size_t)h->K_pad);
    if (e == cudaSuccess) e = cudaMemcpy(h->signs, signs_host, (size_t)K, cudaMemcpyHostToDevice);
  }
  const void* src = W_fp16;
  if (e == cudaSuccess && !w_on_device) {
    e = dev_malloc(&tmp, (size_t)N * K * 2);
    if (e == cudaSuccess) e = cudaMemcpy(tmp, W_fp16, (size_t)N * K * 2, cudaMemcpyHostToDevice);
    src = tmp;
  }
  if (e == cudaSuccess) {
    RQArgs a = make_rq(src, N, h->N_pad, K, h->KB, had_block, nfull, tail, log2B, 4, h->sw, h->wt);
    a.signs = h->signs;
    e = launch_rotate_quant(kRQWeights, a, 0, false);
  }
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  if (tmp) cudaFree(tmp);
  if (e != cudaSuccess) {
    dptq_destroy(h);
    return cuda_fail(e, "dptq_pack_weights");
  }
  *out = h;
  return DPTQ_OK;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
}  // namespace

dptq_status dptq_pack_weights(const void* W_fp16, int N, int K, int had_block, int w_on_device, dptq_handle* out) {
  NvtxRange nvtx_range("dptq_pack_weights");
  return pack_weights_impl(W_fp16, N, K, had_block, nullptr, w_on_device, out);
}

dptq_status dptq_pack_weights_rh(const void* W_fp16, int N, int K, int had_block, const int8_t* signs_host,
                                 int w_on_device, dptq_handle* out) {
  NvtxRange nvtx_range("dptq_pack_weights_rh");
  if (!signs_host) return fail(DPTQ_ERR_INVALID_ARG, "null pointer");
  return pack_weights_impl(W_fp16, N, K, had_block, signs_host, w_on_device, out);
}

dptq_status dptq_rotate_quant_act_rh(const void* x_fp16, int M, int K, int had_block, int bits,
                                     const int8_t* signs_dev, void* codes, float* scales, void* stream) {
  NvtxRange nvtx_range("dptq_rotate_quant_act_rh");
  if (bits != 4 && bits != 8) return fail(DPTQ_ERR_INVALID_ARG, "bits must be 4 or 8");
  if (M < 0 || K <= 0 || had_block <= 0) return fail(DPTQ_ERR_INVALID_ARG, "bad sizes");
  if (M == 0) return DPTQ_OK;
  if (!x_fp16 || !codes || !scales) return fail(DPTQ_ERR_INVALID_ARG, "null pointer");
  if (signs_dev && !aligned16(signs_dev)) return fail(DPTQ_ERR_INVALID_ARG, "signs must be 16-byte aligned");
  int nfull, tail, log2B;
  dptq_status st = check_shape(K, had_block, nfull, tail, log2B);
  if (st != DPTQ_OK) return st;
  RQArgs a = make_rq(x_fp16, M, M, K, round_up(K, kKBlock) / kKBlock, had_block, nfull, tail, log2B, bits, scales,
                     codes);
  a.signs = signs_dev;
  DPTQ_CUDA(launch_rotate_quant(kRQPublic, a, static_cast<cudaStream_t>(stream), true), "rotate_quant launch");
  return DPTQ_OK;
}

dptq_status dptq_rotate_act_rh(const void* x_fp16, int M, int K, int had_block, const int8_t* signs_dev,
                               float* y_f32, void* stream) {
  NvtxRange nvtx_range("dptq_rotate_act_rh");
  if (M < 0 || K <= 0 || had_block <= 0) return fail(DPTQ_ERR_INVALID_ARG, "bad sizes");
  if (M == 0) return DPTQ_OK;
  if (!x_fp16 || !y_f32) return fail(DPTQ_ERR_INVALID_ARG, "null pointer");
  if (signs_dev && !aligned16(signs_dev)) return fail(DPTQ_ERR_INVALID_ARG, "signs must be 16-byte aligned");
  int nfull, tail, log2B;
  dptq_status st = check_shape(K, had_block, nfull, tail, log2B);
  if (st != DPTQ_OK) return st;
  RQArgs a = make_rq(x_fp16, M, M, K, round_up(K, kKBlock) / kKBlock, had_block, nfull, tail, log2B, 4, nullptr,
                     y_f32);
  a.signs = signs_dev;
  DPTQ_CUDA(launch_rotate_quant(kRQY, a, static_cast<cudaStream_t>(stream), true), "rotate launch");
  return DPTQ_OK;
}

dptq_status dptq_rotate_quant_act(const void* x_fp16, int M, int K, int had_block, int bits, void* codes,
                                  float* scales, void* stream) {
  NvtxRange nvtx_range("dptq_rotate_quant_act");
  if (bits != 4 && bits != 8) return fail(DPTQ_ERR_INVALID_ARG, "bits must be 4 or 8");
  if (M < 0 || K <= 0 || had_block <= 0) return fail(DPTQ_ERR_INVALID_ARG, "bad sizes");
  if (M == 0) return DPTQ_OK;
  if (!x_fp16 || !codes || !scales) return fail(DPTQ_ERR_INVALID_ARG, "null pointer");
  int nfull, tail, log2B;
  dptq_status st = check_shape(K, had_block, nfull, tail, log2B);
  if (st != DPTQ_OK) return st;
  RQArgs a = make_rq(x_fp16, M, M, K, round_up(K, kKBlock) / kKBlock, had_block, nfull, tail, log2B, bits, scales,
                     codes);
  DPTQ_CUDA(launch_rotate_quant(kRQPublic, a, static_cast<cudaStream_t>(stream), true), "rotate_quant launch");
  return DPTQ_OK;
}

dptq_status dptq_rotate_act(const void* x_fp16, int M, int K, int had_block, float* y_f32, void* stream) {
  NvtxRange nvtx_range("dptq_rotate_act");
  if (M < 0 || K <= 0 || had_block <= 0) return fail(DPTQ_ERR_INVALID_ARG, "bad sizes");
  if (M == 0) return DPTQ_OK;
  if (!x_fp16 || !y_f32) return fail(DPTQ_ERR_INVALID_ARG, "null pointer");
  int nfull, tail, log2B;
  dptq_status st = check_shape(K, had_block, nfull, tail, log2B);
  if (st != DPTQ_OK) return st;
  RQArgs a = make_rq(x_fp16, M, M, K, round_up(K, kKBlock) / kKBlock, had_block, nfull, tail, log2B, 4, nullptr,
                     y_f32);
  DPTQ_CUDA(launch_rotate_quant(kRQY, a, static_cast<cudaStream_t>(stream), true), "rotate launch");
  return DPTQ_OK;
}

}  // extern "C"

namespace {

// Shape checks and scratch sizing shared by the qlinear entry points.
dptq_status prepare_qlinear(dptq_handle h, int M, int bits, cudaStream_t s, int* dev, GemmPlan* plan,
                            Scratch** sc) {
  if (bits != 4 && bits != 8) return fail(DPTQ_ERR_INVALID_ARG, "bits must be 4 or 8");
  if (M < 0) return fail(DPTQ_ERR_INVALID_ARG, "M must be >= 0");
  dptq_status st = check_handle(h, dev);
  if (st != DPTQ_OK) return st;
  if (M == 0) return DPTQ_OK;
  if ((st = ensure_scratch(*dev, 0, 0, s, sc)) != DPTQ_OK) return st;
  if (!plan_launch(M, h->N, h->K_pad, bits, (*sc)->num_sms, *plan)) return fail(DPTQ_ERR_UNSUPPORTED, "no GEMM plan");
  const int planes = bits == 8 ? 2 : 1;
  return ensure_scratch(*dev, (size_t)planes * h->K_pad * plan->M_pad, plan->M_pad, s, sc);
}

dptq_status quantize_into_scratch(dptq_handle h, const void* x_fp16, int M, int bits, const GemmPlan& plan,
                                  Scratch* sc, cudaStream_t s) {
  int nfull, tail, log2B;
  dptq_status st = check_shape(h->K, h->had_block, nfull, tail, log2B);
  if (st != DPTQ_OK) return st;
  RQArgs a = make_rq(x_fp16, M, plan.M_pad, h->K, h->KB, h->had_block, nfull, tail, log2B, bits, sc->sa, sc->act);
  a.signs = h->signs;
  DPTQ_CUDA(launch_rotate_quant(kRQAct, a, s, true), "rotate_quant launch");
  return DPTQ_OK;
}

}  // namespace

extern "C" {

dptq_status dptq_qlinear(dptq_handle h, const void* x_fp16, int M, int bits, void* out_fp16, void* stream) {
  NvtxRange nvtx_range("dptq_qlinear");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int dev;
  GemmPlan plan;
  Scratch* sc = nullptr;
  dptq_status st = prepare_qlinear(h, M, bits, s, &dev, &plan, &sc);
  if (st != DPTQ_OK || M == 0) return st;
  if (!x_fp16 || !out_fp16) return fail(DPTQ_ERR_INVALID_ARG, "null pointer");
  // Small M: one launch that rotates and quantizes the rows and runs the GEMM, with a CTA (or
  // two) per row, or else as many rows side by side in a CTA as its warps hold.
  GemmPlan fp;
  int cpr = 0, wpc = 0, rpc = 1;
  bool one = fused_allowed() && plan.M_pad <= 64 && h->K_pad <= kFusedMaxKPad && pow2_tail(h->K, h->had_block) &&
             fused_rotation_split(h->K, h->had_block, h->K % h->had_block, cpr, wpc);
  int items = M * cpr;
  if (one && !plan_launch(M, h->N, h->K_pad, bits, sc->num_sms, fp, items)) {
    rpc = cpr == 1 ? 8 / wpc : 1;
    items = ceil_div(M, rpc);
    one = rpc > 1 && plan_launch(M, h->N, h->K_pad, bits, sc->num_sms, fp, items);
  }
  if (one && fp.M_pad == plan.M_pad) {
    int nfull, tail, log2B;
    if ((st = check_shape(h->K, h->had_block, nfull, tail, log2B)) != DPTQ_OK) return st;
    fp.args.rq = make_rq(x_fp16, M, fp.M_pad, h->K, h->KB, h->had_block, nfull, tail, log2B, bits, sc->sa, sc->act);
    fp.args.rq.signs = h->signs;
    fp.args.rq.pmax = sc->pmax;
    fp.args.rq_cpr = cpr;
    fp.args.rq_wpc = wpc;
    fp.args.rq_rpc = rpc;
    fp.args.rq_items = items;
    return run_gemm(h, fp, sc->act, sc->sa, out_fp16, nullptr, sc, s);
  }
  if ((st = quantize_into_scratch(h, x_fp16, M, bits, plan, sc, s)) != DPTQ_OK) return st;
  return run_gemm(h, plan, sc->act, sc->sa, out_fp16, nullptr, sc, s);
}

dptq_status dptq_qlinear_quantize(dptq_handle h, const void* x_fp16, int M, int bits, void* stream) {
  NvtxRange nvtx_range("dptq_qlinear_quantize");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int dev;
  GemmPlan plan;
  Scratch* sc = nullptr;
  dptq_status st = prepare_qlinear(h, M, bits, s, &dev, &plan, &sc);
  if (st != DPTQ_OK || M == 0) return st;
  if (!x_fp16) return fail(DPTQ_ERR_INVALID_ARG, "null pointer");
  return quantize_into_scratch(h, x_fp16, M, bits, plan, sc, s);
}

dptq_status dptq_qlinear_gemm(dptq_handle h, int M, int bits, void* out_fp16, void* stream) {
  NvtxRange nvtx_range("dptq_qlinear_gemm");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int dev;
  GemmPlan plan;
  Scratch* sc = nullptr;
  dptq_status st = prepare_qlinear(h, M, bits, s, &dev, &plan, &sc);
  if (st != DPTQ_OK || M == 0) return st;
  if (!out_fp16) return fail(DPTQ_ERR_INVALID_ARG, "null pointer");
  return run_gemm(h, plan, sc->act, sc->sa, out_fp16, nullptr, sc, s);
}

dptq_status dptq_qgemm_codes(dptq_handle h, const void* codes, const float* scales, int M, int bits, void* out_fp16,
                             int32_t* acc_i32, void* stream) {
  NvtxRange nvtx_range("dptq_qgemm_codes");
  if (bits != 4 && bits != 8) return fail(DPTQ_ERR_INVALID_ARG, "bits must be 4 or 8");
  if (M < 0) return fail(DPTQ_ERR_INVALID_ARG, "M must be >= 0");
  int dev;
  dptq_status st = check_handle(h, &dev);
  if (st != DPTQ_OK) return st;
  if (M == 0) return DPTQ_OK;
  if (!codes || !scales || !out_fp16) return fail(DPTQ_ERR_INVALID_ARG, "null pointer");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  Scratch* sc = nullptr;
  if ((st = ensure_scratch(dev, 0, 0, s, &sc)) != DPTQ_OK) return st;
  GemmPlan plan;
  if (!plan_launch(M, h->N, h->K_pad, bits, sc->num_sms, plan)) return fail(DPTQ_ERR_UNSUPPORTED, "no GEMM plan");
  const int planes = bits == 8 ? 2 : 1;
  if ((st = ensure_scratch(dev, (size_t)planes * h->K_pad * plan.M_pad, 0, s, &sc)) != DPTQ_OK) return st;
  CodesArgs c{};
  c.codes = static_cast<const uint8_t*>(codes);
  c.M = M;
  c.M_pad = plan.M_pad;
  c.K = h->K;
  c.KB = h->KB;
  c.bits = bits;
  c.act = sc->act;
  DPTQ_CUDA(launch_codes_to_act(c, s), "codes_to_act launch");
  return run_gemm(h, plan, sc->act, scales, out_fp16, acc_i32, sc, s);
}

dptq_status dptq_kv4_quantize(const void* kv_fp16, int rows, int cols, int group, void* codes, float* scales,
                              void* stream) {
  NvtxRange nvtx_range("dptq_kv4_quantize");
  if (rows < 0 || cols <= 0 || group <= 0) return fail(DPTQ_ERR_INVALID_ARG, "bad sizes");
  if (rows == 0) return DPTQ_OK;
  if (!kv_fp16 || !codes || !scales) return fail(DPTQ_ERR_INVALID_ARG, "null pointer");
  if (!aligned16(kv_fp16)) return fail(DPTQ_ERR_INVALID_ARG, "kv must be 16-byte aligned");
  if ((reinterpret_cast<uintptr_t>(codes) & 1u) != 0)   // (the narrowest stores are 16 bits wide)
    return fail(DPTQ_ERR_INVALID_ARG, "codes must be 2-byte aligned");
  if (group % 128 != 0 || group > 1024 || cols % group != 0)
    return fail(DPTQ_ERR_UNSUPPORTED, "group must be a multiple of 128 up to 1024 that divides cols");
  int dev;
  dptq_status st = current_device(&dev);
  if (st != DPTQ_OK) return st;
  int sms = 0;
  DPTQ_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev), "cudaDeviceGetAttribute");
  KvArgs a{static_cast<const __half*>(kv_fp16), rows, cols, group, static_cast<uint8_t*>(codes), scales};
  DPTQ_CUDA(launch_kv4(a, sms, static_cast<cudaStream_t>(stream)), "kv4 launch");
  return DPTQ_OK;
}

dptq_status dptq_sensitivity_policy(const float* x, const float* dx, int L, int T, int d, int bits, double eps,
                                    double tau_jr, double tau_snr, double* jr, double* snr, uint8_t* bits_out,
                                    void* stream) {
  NvtxRange nvtx_range("dptq_sensitivity_policy");
  if (bits != 4 && bits != 8) return fail(DPTQ_ERR_INVALID_ARG, "bits must be 4 or 8");
  if (L < 0 || T <= 0 || d <= 0 || !(eps >= 0.0)) return fail(DPTQ_ERR_INVALID_ARG, "bad sizes or eps");
  if (L == 0) return DPTQ_OK;
  if (!x || !dx || !jr || !snr || !bits_out) return fail(DPTQ_ERR_INVALID_ARG, "null pointer");
  if (!aligned16(x) || !aligned16(dx) || d % 4 != 0)
    return fail(DPTQ_ERR_INVALID_ARG, "x and dx must be 16-byte aligned and d a multiple of 4");
  int dev;
  dptq_status st = current_device(&dev);
  if (st != DPTQ_OK) return st;
  Scratch* sc = nullptr;
  st = ensure_scratch(dev, 0, 0, static_cast<cudaStream_t>(stream), &sc);
  if (st != DPTQ_OK) return st;
  PolicyArgs a{x, dx, L, T, d, bits, eps, tau_jr, tau_snr, jr, snr, bits_out, sc->err};
  DPTQ_CUDA(launch_policy(a, sc->num_sms, static_cast<cudaStream_t>(stream)), "policy launch");
  return DPTQ_OK;
}

namespace {
// The bounds of a batch; *none: nothing to do.
dptq_status check_batch_sizes(const dptq_kv8_batch* b) {
  if (b->seqs < 0 || b->tokens < 0 || b->max_tokens < 0 || b->max_len < 0 || b->table_stride < 0)
    return fail(DPTQ_ERR_INVALID_ARG, "bad batch sizes");
  return DPTQ_OK;
}
dptq_status check_batch_limits(const dptq_kv8_batch* b, bool* none) {
  if (b->seqs > 65535) return fail(DPTQ_ERR_UNSUPPORTED, "too many heads or sequences");
  if (b->max_tokens > 65535) return fail(DPTQ_ERR_UNSUPPORTED, "more than 65535 rows of a sequence in one call");
  if (b->max_len > 1 << 27) return fail(DPTQ_ERR_UNSUPPORTED, "sequences longer than 2^27 tokens");
  *none = b->seqs == 0 || b->tokens == 0 || b->max_tokens == 0;
  return DPTQ_OK;
}
// The kernels' view of a batch, and the device's scratch (its error words).
dptq_status take_batch(const dptq_kv8_batch* b, cudaStream_t s, Kv8Args* a, Scratch** sc) {
  int dev;
  dptq_status st = current_device(&dev);
  if (st != DPTQ_OK) return st;
  if ((st = ensure_scratch(dev, 0, 0, s, sc)) != DPTQ_OK) return st;
  *a = Kv8Args{};
  a->cu = b->cu_tokens;
  a->lens = b->seq_lens;
  a->table = b->block_table;
  a->seqs = b->seqs;
  a->table_stride = b->table_stride;
  a->tokens = b->tokens;
  a->max_tokens = std::min(b->max_tokens, b->tokens);
  a->max_len = b->max_len;
  a->err = (*sc)->err;
  a->bad = (*sc)->err + 1;
  return DPTQ_OK;
}

// The host's part of the checks of a call on a paged cache (Cache: dptq_kv8_cache or dptq_kv4_cache, whose
// scales are of `scale_bytes`); *none: nothing to do.
extern "C++" template <class Cache>
dptq_status check_paged(const Cache* c, const dptq_kv8_batch* b, unsigned scale_bytes, cudaStream_t s, Kv8Args* a,
                        bool* none, Scratch** sc) {
  *none = false;
  if (!c || !b) return fail(DPTQ_ERR_INVALID_ARG, "null pointer");
  if (c->num_blocks <= 0 || c->kv_heads <= 0 || c->block_tokens <= 0 || c->head_dim <= 0)
    return fail(DPTQ_ERR_INVALID_ARG, "bad cache sizes");
  dptq_status st = check_batch_sizes(b);
  if (st != DPTQ_OK) return st;
  if (c->head_dim != 64 && c->head_dim != 128) return fail(DPTQ_ERR_UNSUPPORTED, "head_dim must be 64 or 128");
  if (c->block_tokens < 16 || c->block_tokens > 128 || !is_pow2(c->block_tokens))
    return fail(DPTQ_ERR_UNSUPPORTED, "block_tokens must be 16, 32, 64 or 128");
  if (c->kv_heads > 1023) return fail(DPTQ_ERR_UNSUPPORTED, "too many heads or sequences");
  if ((st = check_batch_limits(b, none)) != DPTQ_OK || *none) return st;
  if (!c->k_codes || !c->v_codes || !c->k_scales || !c->v_scales || !b->cu_tokens || !b->seq_lens || !b->block_table)
    return fail(DPTQ_ERR_INVALID_ARG, "null pointer");
  if (!aligned16(c->k_codes) || !aligned16(c->v_codes))
    return fail(DPTQ_ERR_INVALID_ARG, "codes must be 16-byte aligned");
  const uintptr_t scales = reinterpret_cast<uintptr_t>(c->k_scales) | reinterpret_cast<uintptr_t>(c->v_scales);
  if ((scales & (scale_bytes - 1)) != 0 || !aligned4(b->cu_tokens) || !aligned4(b->seq_lens) || !aligned4(b->block_table))
    return fail(DPTQ_ERR_INVALID_ARG,
                "scales must be " + std::to_string(scale_bytes) + "-byte aligned, the batch's arrays 4-byte aligned");
  if (b->max_len > (long long)b->table_stride * c->block_tokens)
    return fail(DPTQ_ERR_INVALID_ARG, "max_len exceeds the block table");
  if ((st = take_batch(b, s, a, sc)) != DPTQ_OK) return st;
  a->num_blocks = c->num_blocks;
  a->kv_heads = c->kv_heads;
  a->head_dim = c->head_dim;
  a->log2_page = c->block_tokens == 16 ? 4 : c->block_tokens == 32 ? 5 : c->block_tokens == 64 ? 6 : 7;
  return DPTQ_OK;
}
dptq_status check_kv8(const dptq_kv8_cache* c, const dptq_kv8_batch* b, cudaStream_t s, Kv8Args* a, bool* none,
                      Scratch** sc) {
  const dptq_status st = check_paged(c, b, 4, s, a, none, sc);
  if (st != DPTQ_OK || *none) return st;
  a->codes[0] = c->k_codes;
  a->codes[1] = c->v_codes;
  a->scales[0] = c->k_scales;
  a->scales[1] = c->v_scales;
  return DPTQ_OK;
}
dptq_status check_kv4(const dptq_kv4_cache* c, const dptq_kv8_batch* b, cudaStream_t s, Kv4Args* a, bool* none,
                      Scratch** sc) {
  if (c && c->num_blocks > 0 && c->kv_heads > 0 && c->block_tokens > 0 &&
      (double)c->num_blocks * c->kv_heads * c->block_tokens > 4294967295.0)
    return fail(DPTQ_ERR_UNSUPPORTED, "a cache of 2^32 tokens and heads or more");
  // (16 scales of a page's tokens are read at a time)
  const dptq_status st = check_paged(c, b, 16, s, &a->c, none, sc);
  if (st != DPTQ_OK || *none) return st;
  a->codes[0] = c->k_codes;
  a->codes[1] = c->v_codes;
  a->scales[0] = c->k_scales;
  a->scales[1] = c->v_scales;
  return DPTQ_OK;
}

// Rows of `heads` heads: aligned, and no row reaching into the next.
dptq_status check_rows(const void* p, long long stride, long long heads, int D) {
  if (!p) return fail(DPTQ_ERR_INVALID_ARG, "null pointer");
  if (!aligned16(p) || stride % 8 != 0)
    return fail(DPTQ_ERR_INVALID_ARG, "rows must be 16-byte aligned: base pointers, and strides of multiples of 8");
  if (stride < heads * D) return fail(DPTQ_ERR_INVALID_ARG, "a row's stride is below its length");
  return DPTQ_OK;
}
}  // namespace

dptq_status dptq_kv8_append(const dptq_kv8_cache* cache, const dptq_kv8_batch* batch, const void* k_fp16,
                            const void* v_fp16, long long token_stride, void* stream) {
  NvtxRange nvtx_range("dptq_kv8_append");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  Kv8AppendArgs a{};
  Scratch* sc = nullptr;
  bool none;
  dptq_status st = check_kv8(cache, batch, s, &a.c, &none, &sc);
  if (st != DPTQ_OK || none) return st;
  if ((st = check_rows(k_fp16, token_stride, cache->kv_heads, cache->head_dim)) != DPTQ_OK) return st;
  if ((st = check_rows(v_fp16, token_stride, cache->kv_heads, cache->head_dim)) != DPTQ_OK) return st;
  a.rows[0] = static_cast<const __half*>(k_fp16);
  a.rows[1] = static_cast<const __half*>(v_fp16);
  a.stride = token_stride;
  DPTQ_CUDA(launch_kv8_append(a, s), "kv8_append launch");
  return DPTQ_OK;
}

namespace {
dptq_status check_attention(int q_heads, int kv_heads, float scale, int window, int sinks) {
  if (q_heads <= 0 || window < 0 || sinks < 0 || !std::isfinite(scale))
    return fail(DPTQ_ERR_INVALID_ARG, "bad q_heads, window, sinks or scale");
  if (kv_heads > 0) {
    if (q_heads % kv_heads != 0) return fail(DPTQ_ERR_INVALID_ARG, "q_heads must be a multiple of kv_heads");
    if (q_heads / kv_heads > 64) return fail(DPTQ_ERR_UNSUPPORTED, "more than 64 query heads for a KV head");
  }
  return DPTQ_OK;
}
// The rows, masks and scratch of an attention call.
extern "C++" template <class Args>
dptq_status fill_attention(Args& a, Scratch* sc, cudaStream_t s, const dptq_kv8_batch* batch, int kv_heads, int head_dim,
                           const void* q_fp16, long long q_stride, int q_heads, float scale, int window, int sinks,
                           void* out_fp16, long long out_stride) {
  dptq_status st;
  if ((st = check_rows(q_fp16, q_stride, q_heads, head_dim)) != DPTQ_OK) return st;
  if ((st = check_rows(out_fp16, out_stride, q_heads, head_dim)) != DPTQ_OK) return st;
  a.q = static_cast<const __half*>(q_fp16);
  a.out = static_cast<__half*>(out_fp16);
  a.q_stride = q_stride;
  a.out_stride = out_stride;
  a.q_heads = q_heads;
  a.group = q_heads / kv_heads;
  a.scale = scale;
  a.window = window < batch->max_len ? window : 0;   // (a window that holds every position)
  a.sinks = std::min(sinks, batch->max_len);
  if ((st = ensure_kv8_scratch(sc, s)) != DPTQ_OK) return st;
  a.ws = sc->kv8_ws;
  a.counters = sc->kv8_counters;
  a.wait_cycles = wait_cycles_setting();
  a.shortfall = take_kv8_shortfall();
  return DPTQ_OK;
}
}  // namespace

dptq_status dptq_kv8_attention(const dptq_kv8_cache* cache, const dptq_kv8_batch* batch, const void* q_fp16,
                               long long q_stride, int q_heads, float scale, int window, int sinks, void* out_fp16,
                               long long out_stride, void* stream) {
  NvtxRange nvtx_range("dptq_kv8_attention");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  dptq_status st = check_attention(q_heads, cache ? cache->kv_heads : 0, scale, window, sinks);
  if (st != DPTQ_OK) return st;
  Kv8AttendArgs a{};
  Scratch* sc = nullptr;
  bool none;
  st = check_kv8(cache, batch, s, &a.c, &none, &sc);
  if (st != DPTQ_OK || none) return st;
  if ((st = fill_attention(a, sc, s, batch, cache->kv_heads, cache->head_dim, q_fp16, q_stride, q_heads, scale, window,
                           sinks, out_fp16, out_stride)) != DPTQ_OK)
    return st;
  const bool decode = (long long)a.c.max_tokens * a.group <= kDecodeRows;
  DPTQ_CUDA(decode ? launch_kv8_decode(a, sc->num_sms, s) : launch_kv8_prefill(a, sc->num_sms, s), "kv8_attention launch");
  return DPTQ_OK;
}

namespace {
dptq_status kv4_rows(const char* what, const dptq_kv4_cache* cache, const dptq_kv8_batch* batch, const void* k,
                     const void* v, long long stride, void* stream,
                     cudaError_t (*launch)(const Kv4RowsArgs&, cudaStream_t)) {
  NvtxRange nvtx_range(what);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  Kv4RowsArgs a{};
  Scratch* sc = nullptr;
  bool none;
  dptq_status st = check_kv4(cache, batch, s, &a.k, &none, &sc);
  if (st != DPTQ_OK || none) return st;
  if ((st = check_rows(k, stride, cache->kv_heads, cache->head_dim)) != DPTQ_OK) return st;
  if ((st = check_rows(v, stride, cache->kv_heads, cache->head_dim)) != DPTQ_OK) return st;
  a.rows[0] = static_cast<__half*>(const_cast<void*>(k));
  a.rows[1] = static_cast<__half*>(const_cast<void*>(v));
  a.stride = stride;
  DPTQ_CUDA(launch(a, s), what);
  return DPTQ_OK;
}
}  // namespace

dptq_status dptq_kv4_append(const dptq_kv4_cache* cache, const dptq_kv8_batch* batch, const void* k_fp16,
                            const void* v_fp16, long long token_stride, void* stream) {
  return kv4_rows("dptq_kv4_append", cache, batch, k_fp16, v_fp16, token_stride, stream, launch_kv4_append);
}

dptq_status dptq_kv4_read(const dptq_kv4_cache* cache, const dptq_kv8_batch* batch, void* k_out, void* v_out,
                          long long token_stride, void* stream) {
  return kv4_rows("dptq_kv4_read", cache, batch, k_out, v_out, token_stride, stream, launch_kv4_read);
}

dptq_status dptq_kv4_attention(const dptq_kv4_cache* cache, const dptq_kv8_batch* batch, const void* q_fp16,
                               long long q_stride, int q_heads, float scale, int window, int sinks, void* out_fp16,
                               long long out_stride, void* stream) {
  NvtxRange nvtx_range("dptq_kv4_attention");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  dptq_status st = check_attention(q_heads, cache ? cache->kv_heads : 0, scale, window, sinks);
  if (st != DPTQ_OK) return st;
  Kv4AttendArgs a{};
  Scratch* sc = nullptr;
  bool none;
  st = check_kv4(cache, batch, s, &a.k, &none, &sc);
  if (st != DPTQ_OK || none) return st;
  if ((st = fill_attention(a, sc, s, batch, cache->kv_heads, cache->head_dim, q_fp16, q_stride, q_heads, scale, window,
                           sinks, out_fp16, out_stride)) != DPTQ_OK)
    return st;
  const bool decode = (long long)a.k.c.max_tokens * a.group <= kDecodeRows;
  DPTQ_CUDA(decode ? launch_kv4_decode(a, sc->num_sms, s) : launch_kv4_prefill(a, sc->num_sms, s), "kv4_attention launch");
  return DPTQ_OK;
}

dptq_status dptq_rotary_frequencies(int rot_dim, double base, int scaling, double factor, double trained_len, double low,
                                    double high, double* freq) {
  if (!freq) return fail(DPTQ_ERR_INVALID_ARG, "null pointer");
  if (rot_dim < 2 || rot_dim % 2 != 0) return fail(DPTQ_ERR_INVALID_ARG, "rot_dim must be even and at least 2");
  if (!(base > 1.0) || !std::isfinite(base)) return fail(DPTQ_ERR_INVALID_ARG, "base must be finite and above 1");
  if (scaling < DPTQ_ROTARY_NONE || scaling > DPTQ_ROTARY_RAMP) return fail(DPTQ_ERR_INVALID_ARG, "unknown scaling");
  if (scaling != DPTQ_ROTARY_NONE && (!(factor > 0.0) || !std::isfinite(factor)))
    return fail(DPTQ_ERR_INVALID_ARG, "factor must be finite and above 0");
  if (scaling == DPTQ_ROTARY_NTK) {
    if (rot_dim < 4) return fail(DPTQ_ERR_INVALID_ARG, "NTK scaling takes a rot_dim of at least 4");
    base *= std::pow(factor, rot_dim / (rot_dim - 2.0));
  }
  const bool by_turns = scaling == DPTQ_ROTARY_WAVELENGTH || scaling == DPTQ_ROTARY_RAMP;
  if (by_turns && !(trained_len > 0.0 && std::isfinite(trained_len) && low > 0.0 && low < high && std::isfinite(high)))
    return fail(DPTQ_ERR_INVALID_ARG, "trained_len must be above 0 and 0 < low < high");
  constexpr double kTwoPi = 6.283185307179586476925;
  double a = 0.0, b = 0.0;
  if (scaling == DPTQ_ROTARY_RAMP) {
    auto dim = [&](double turns) { return rot_dim * std::log(trained_len / (kTwoPi * turns)) / (2.0 * std::log(base)); };
    a = std::max(std::floor(dim(high)), 0.0);
    b = std::min(std::ceil(dim(low)), rot_dim - 1.0);
  }
  for (int i = 0; i < rot_dim / 2; ++i) {
    const double f = std::pow(base, -2.0 * i / rot_dim);
    double keep = 1.0;
    if (scaling == DPTQ_ROTARY_LINEAR) keep = 0.0;
    if (scaling == DPTQ_ROTARY_WAVELENGTH) keep = (trained_len * f / kTwoPi - low) / (high - low);
    if (scaling == DPTQ_ROTARY_RAMP) keep = 1.0 - (i - a) / std::max(b - a, 0.001);
    keep = std::min(std::max(keep, 0.0), 1.0);
    freq[i] = keep == 1.0 ? f : keep * f + (1.0 - keep) * f / factor;
  }
  return DPTQ_OK;
}

dptq_status dptq_rotary_turns(const double* freq, int n, uint64_t* turns) {
  if (n < 0 || (n > 0 && (!freq || !turns))) return fail(DPTQ_ERR_INVALID_ARG, "null pointer or negative size");
  for (int i = 0; i < n; ++i)
    if (!std::isfinite(freq[i])) return fail(DPTQ_ERR_INVALID_ARG, "a frequency is not finite");
  constexpr double kPerTurn = 0.159154943091895335769;   // 1 / 2 pi
  for (int i = 0; i < n; ++i) {
    const double t = std::fabs(freq[i]) * kPerTurn;
    const uint64_t u = static_cast<uint64_t>(std::rint(std::ldexp(t - std::floor(t), 64)));   // (at most 2^64 - 2^11)
    turns[i] = freq[i] < 0.0 ? ~u + 1u : u;
  }
  return DPTQ_OK;
}

dptq_status dptq_rotary(const dptq_kv8_batch* batch, const void* x_fp16, long long x_stride, int heads, int head_dim,
                        const uint64_t* turns, int rot_dim, int interleaved, float amplitude, void* out_fp16,
                        long long out_stride, void* stream) {
  NvtxRange nvtx_range("dptq_rotary");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (!batch) return fail(DPTQ_ERR_INVALID_ARG, "null pointer");
  dptq_status st = check_batch_sizes(batch);
  if (st != DPTQ_OK) return st;
  if (heads <= 0 || head_dim <= 0 || rot_dim < 2 || rot_dim > head_dim || rot_dim % 2 != 0)
    return fail(DPTQ_ERR_INVALID_ARG, "bad heads, head_dim or rot_dim");
  if (!std::isfinite(amplitude)) return fail(DPTQ_ERR_INVALID_ARG, "amplitude must be finite");
  if (head_dim % 8 != 0 || head_dim > 512) return fail(DPTQ_ERR_UNSUPPORTED, "head_dim must be a multiple of 8 up to 512");
  if (heads > 65535) return fail(DPTQ_ERR_UNSUPPORTED, "more than 65535 heads");
  bool none;
  if ((st = check_batch_limits(batch, &none)) != DPTQ_OK || none) return st;
  if (!batch->cu_tokens || !batch->seq_lens || !turns) return fail(DPTQ_ERR_INVALID_ARG, "null pointer");
  if (!aligned4(batch->cu_tokens) || !aligned4(batch->seq_lens) || (reinterpret_cast<uintptr_t>(turns) & 7u) != 0)
    return fail(DPTQ_ERR_INVALID_ARG, "the batch's arrays must be 4-byte aligned, turns 8-byte aligned");
  if ((st = check_rows(x_fp16, x_stride, heads, head_dim)) != DPTQ_OK) return st;
  if ((st = check_rows(out_fp16, out_stride, heads, head_dim)) != DPTQ_OK) return st;
  if (x_fp16 == out_fp16 && x_stride != out_stride && batch->tokens > 1)
    return fail(DPTQ_ERR_INVALID_ARG, "in place both strides are the same");
  RotaryArgs a{};
  Scratch* sc = nullptr;
  if ((st = take_batch(batch, s, &a.c, &sc)) != DPTQ_OK) return st;
  a.x = static_cast<const __half*>(x_fp16);
  a.out = static_cast<__half*>(out_fp16);
  a.turns = turns;
  a.x_stride = x_stride;
  a.out_stride = out_stride;
  a.heads = heads;
  a.head_dim = head_dim;
  a.rot = rot_dim;
  a.interleaved = interleaved != 0;
  a.amplitude = amplitude;
  DPTQ_CUDA(launch_rotary(a, sc->num_sms, s), "rotary launch");
  return DPTQ_OK;
}

dptq_status dptq_kv8_reserve(void) {
  NvtxRange nvtx_range("dptq_kv8_reserve");
  int dev;
  dptq_status st = current_device(&dev);
  if (st != DPTQ_OK) return st;
  Scratch* sc = nullptr;
  if ((st = ensure_scratch(dev, 0, 0, 0, &sc)) != DPTQ_OK) return st;
  return ensure_kv8_scratch(sc, 0);
}

dptq_status dptq_add_rmsnorm_quant(const void* x_fp16, const void* residual_fp16, const void* gamma_fp16, int M,
                                   int K, float eps, int bits, void* residual_out, void* codes, float* scales,
                                   void* stream) {
  NvtxRange nvtx_range("dptq_add_rmsnorm_quant");
  if (bits != 4 && bits != 8) return fail(DPTQ_ERR_INVALID_ARG, "bits must be 4 or 8");
  if (M < 0 || K <= 0 || !(eps >= 0.f)) return fail(DPTQ_ERR_INVALID_ARG, "bad sizes or eps");
  if (K % 32 != 0 || K > 49152) return fail(DPTQ_ERR_UNSUPPORTED, "K must be a multiple of 32 up to 49152");
  if (M == 0) return DPTQ_OK;
  if (!x_fp16 || !codes || !scales) return fail(DPTQ_ERR_INVALID_ARG, "null pointer");
  if ((residual_fp16 == nullptr) != (residual_out == nullptr))
    return fail(DPTQ_ERR_INVALID_ARG, "residual and residual_out go together");
  if (!aligned16(x_fp16) || !aligned16(residual_fp16) || !aligned16(gamma_fp16) || !aligned16(residual_out))
    return fail(DPTQ_ERR_INVALID_ARG, "x, residual, gamma and residual_out must be 16-byte aligned");
  if ((reinterpret_cast<uintptr_t>(codes) & (bits == 8 ? 7u : 3u)) != 0 || (reinterpret_cast<uintptr_t>(scales) & 3u) != 0)
    return fail(DPTQ_ERR_INVALID_ARG, "codes must be aligned to 8 codes, scales to 4 bytes");
  NormArgs a{static_cast<const __half*>(x_fp16), static_cast<const __half*>(residual_fp16),
             static_cast<const __half*>(gamma_fp16), static_cast<__half*>(residual_out),
             static_cast<uint8_t*>(codes), scales, M, K, bits, eps};
  DPTQ_CUDA(launch_norm_quant(a, static_cast<cudaStream_t>(stream)), "norm_quant launch");
  return DPTQ_OK;
}

namespace {
void write_plan(const GemmPlan& plan, int* info, int len) {
  const GemmArgs& g = plan.args;
  const long long sk = g.sk_iters;
  const int v[DPTQ_LAUNCH_PLAN_LEN] = {plan.nt, plan.kps, plan.M_pad, plan.grid, plan.smem_bytes, g.stages,
                                       g.conv_slots, plan.a_tmem ? 1 : 0, g.nbuf, g.segs, g.seg_iters,
                                       (int)g.tmem_cols, (int)g.a_col0, g.KI, g.n_wtiles, g.m_tiles, g.dp_tiles,
                                       sk > 0x7fffffffLL ? 0x7fffffff : (int)sk, g.rq_np, plan.fused ? 1 : 0,
                                       g.sk_ctas, g.cl, g.pair};
  for (int i = 0; i < len; ++i) info[i] = v[i];
}
dptq_status check_plan_args(int M, int N, int K, int bits, int num_sms, const int* info, int info_len, int want) {
  if (M < 1 || N < 1 || K < 1 || num_sms < 1) return fail(DPTQ_ERR_INVALID_ARG, "sizes must be >= 1");
  if (bits != 4 && bits != 8) return fail(DPTQ_ERR_INVALID_ARG, "bits must be 4 or 8");
  if (info == nullptr || info_len < want) return fail(DPTQ_ERR_INVALID_ARG, "info too short");
  return DPTQ_OK;
}
}  // namespace

dptq_status dptq_plan_info(int M, int N, int K, int bits, int num_sms, int fused, int* info, int info_len) {
  const dptq_status st = check_plan_args(M, N, K, bits, num_sms, info, info_len, DPTQ_PLAN_INFO_LEN);
  if (st != DPTQ_OK) return st;
  GemmPlan plan{};
  if (!plan_gemm(M, N, round_up(K, kKPad), bits, num_sms, plan, fused != 0))
    return fail(DPTQ_ERR_UNSUPPORTED, "no GEMM plan for this shape");
  write_plan(plan, info, DPTQ_PLAN_INFO_LEN);
  return DPTQ_OK;
}

dptq_status dptq_launch_plan(int M, int N, int K, int bits, int num_sms, int row_ctas, int* info, int info_len) {
  const dptq_status st = check_plan_args(M, N, K, bits, num_sms, info, info_len, DPTQ_LAUNCH_PLAN_LEN);
  if (st != DPTQ_OK) return st;
  if (row_ctas < 0) return fail(DPTQ_ERR_INVALID_ARG, "row_ctas must be >= 0");
  GemmPlan plan{};
  if (!plan_launch(M, N, round_up(K, kKPad), bits, num_sms, plan, row_ctas))
    return fail(DPTQ_ERR_UNSUPPORTED, "no GEMM plan for this shape");
  write_plan(plan, info, DPTQ_LAUNCH_PLAN_LEN);
  return DPTQ_OK;
}

dptq_status dptq_reserve(int max_M, int max_K, int max_N) {
  NvtxRange nvtx_range("dptq_reserve");
  if (max_M < 0 || max_K < 0 || max_N < 0) return fail(DPTQ_ERR_INVALID_ARG, "sizes must be >= 0");
  int dev;
  dptq_status st = current_device(&dev);
  if (st != DPTQ_OK) return st;
  (void)max_N;
  // Rows of the widest token tile and of the 192-token prefill tile.
  const int m_res = max_M > 0 ? max_M : 1;
  const size_t M_pad = (size_t)std::max(round_up(m_res, kMaxNT), round_up(m_res, 192));
  const size_t K_pad = (size_t)round_up(max_K > 0 ? max_K : 1, kKPad);   // as layers pad K
  Scratch* sc = nullptr;
  st = ensure_scratch(dev, 2 * K_pad * M_pad, M_pad, 0, &sc);
  if (st != DPTQ_OK) return st;
  DPTQ_CUDA(cudaDeviceSynchronize(), "cudaDeviceSynchronize");
  return DPTQ_OK;
}

dptq_status dptq_get_packed(dptq_handle h, void* wq_host, float* sw_host) {
  int dev;
  dptq_status st = check_handle(h, &dev);
  if (st != DPTQ_OK) return st;
  if (sw_host) DPTQ_CUDA(cudaMemcpy(sw_host, h->sw, sizeof(float) * h->N, cudaMemcpyDeviceToHost), "cudaMemcpy(sw)");
  if (!wq_host) return DPTQ_OK;
  const size_t wt_bytes = (size_t)(h->N_pad / 128) * h->KB * kWTileBytes;
  std::vector<uint8_t> t(wt_bytes);
  DPTQ_CUDA(cudaMemcpy(t.data(), h->wt, wt_bytes, cudaMemcpyDeviceToHost), "cudaMemcpy(wt)");
  uint8_t* dst = static_cast<uint8_t*>(wq_host);
  for (int n = 0; n < h->N; ++n) {
    for (int k = 0; k < h->K; k += 2) {
      int code[2];
      for (int d = 0; d < 2; ++d) {
        const int kk = k + d;
        const int e = kk & 15;  // position in the 16-weight chunk
        const size_t chunk = (((size_t)(n >> 7) * h->KB + (kk >> 7)) * kWTileBytes) + ((kk & 127) >> 5) * 2048 +
                             (n & 127) * 16 + (((kk & 127) >> 4) & 1) * 8;
        const int i = e & 3, high = (e & 7) >= 4;
        const uint8_t* word = t.data() + chunk + (e >> 3) * 4;
        const int mag = high ? (word[i] >> 4) & 7 : word[i] & 7;
        const int neg = high ? (word[(i + 1) & 3] >> 3) & 1 : word[i] >> 7;
        code[d] = neg ? -mag : mag;
      }
      dst[(size_t)n * (h->K / 2) + k / 2] = (uint8_t)((code[0] & 0xF) | ((code[1] & 0xF) << 4));
    }
  }
  return DPTQ_OK;
}

dptq_status dptq_get_shape(dptq_handle h, int* N, int* K, int* had_block) {
  if (!h) return fail(DPTQ_ERR_INVALID_ARG, "null handle");
  if (N) *N = h->N;
  if (K) *K = h->K;
  if (had_block) *had_block = h->had_block;
  return DPTQ_OK;
}

dptq_status dptq_last_device_error(dptq_handle h) {
  (void)h;
  int dev;
  dptq_status st = current_device(&dev);
  if (st != DPTQ_OK) return st;
  DPTQ_CUDA(cudaDeviceSynchronize(), "cudaDeviceSynchronize");
  int word = 0, bad = 0;
  {
    std::lock_guard<std::mutex> lk(g_mu);
    auto it = g_scratch.find(dev);
    if (it != g_scratch.end() && it->second.err != nullptr) {
      Scratch& sc = it->second;
      int words[2];
      DPTQ_CUDA(cudaMemcpy(words, sc.err, sizeof(words), cudaMemcpyDeviceToHost), "cudaMemcpy(err)");
      word = words[0];
      bad = words[1];
      if (word != 0) {
        // A wait gave up: clear the word, the split-tile sums and every counter (split-tile
        // arrivals, the fused launch's two grid counters and its row-maximum slots) the
        // aborted kernel may have left non-zero.
        DPTQ_CUDA(cudaMemset(sc.err, 0, sizeof(int)), "cudaMemset(err)");
        DPTQ_CUDA(cudaMemset(sc.ws, 0, (size_t)sc.num_sms * kMaxNT * 128 * sizeof(int32_t)), "cudaMemset(ws)");
        DPTQ_CUDA(cudaMemset(sc.counters, 0, sizeof(uint32_t) * sc.counter_words), "cudaMemset(counters)");
      }
    }
  }
  // The fixed scratch of dptq_qlinear_static keeps its own error word.
  int sword = 0;
  const cudaError_t e = static_scratch_check_reset(dev, &sword);
  if (e != cudaSuccess) return cuda_fail(e, "static scratch error word");
  if (word == 0) word = sword;
  if (word != 0) {   // (a bad array waits for the next question)
    char buf[64];
    snprintf(buf, sizeof(buf), "device wait timed out (code 0x%x)", word);
    return fail(DPTQ_ERR_TIMEOUT, buf);
  }
  if (bad == 0) return DPTQ_OK;
  {
    std::lock_guard<std::mutex> lk(g_mu);
    DPTQ_CUDA(cudaMemset(g_scratch[dev].err + 1, 0, sizeof(int)), "cudaMemset(err)");
  }
  return fail(DPTQ_ERR_INVALID_ARG, bad == kDevBadPage ? "a KV8 call met a page number outside the cache"
                                                       : "a KV8 call's sequence exceeded its declared tokens or length");
}

dptq_status dptq_scratch_buffers(void** ptrs, size_t* bytes, int* allocated, int max, int* count) {
  if (count == nullptr || max < 0 || (max > 0 && (ptrs == nullptr || bytes == nullptr || allocated == nullptr)))
    return fail(DPTQ_ERR_INVALID_ARG, "null pointer or negative max");
  int dev;
  dptq_status st = current_device(&dev);
  if (st != DPTQ_OK) return st;
  std::vector<std::pair<void*, size_t>> list;
  {
    std::lock_guard<std::mutex> lk(g_mu);
    auto it = g_scratch.find(dev);
    if (it != g_scratch.end()) {
      const Scratch& sc = it->second;
      if (sc.act) list.emplace_back(sc.act, sc.act_bytes);
      if (sc.sa) list.emplace_back(sc.sa, sizeof(float) * sc.sa_count);
      list.insert(list.end(), sc.retired.rbegin(), sc.retired.rend());
    }
  }
  *count = (int)list.size();
  for (int i = 0; i < (int)list.size() && i < max; ++i) {
    ptrs[i] = list[i].first;
    bytes[i] = list[i].second;
    cudaPointerAttributes at{};
    const cudaError_t e = cudaPointerGetAttributes(&at, list[i].first);
    allocated[i] = (e == cudaSuccess && at.type == cudaMemoryTypeDevice) ? 1 : 0;
    if (e != cudaSuccess) (void)cudaGetLastError();
  }
  return DPTQ_OK;
}

void dptq_destroy(dptq_handle h) {
  if (!h) return;
  if (h->wt) cudaFree(h->wt);
  if (h->sw) cudaFree(h->sw);
  if (h->signs) cudaFree(h->signs);
  delete h;
}

}  // extern "C"
