// Kernel-level entry points of the C ABI: each runs the kernels that
// fusion_run launches for one step of Algorithm 1 (Sec. III-B..E), on
// caller-supplied packed ragged buffers instead of the model's workspace, so
// that a step can be checked, or used, on its own.  Host arrays describe the
// ragged layout (per-sample offsets, merge counts); every argument is checked
// on the host before anything is enqueued.  The calls that need scratch
// (identity live and row maps, device copies of the offsets, keep flags)
// either take it from the caller (the _ws entries, asynchronous) or allocate
// it for the call and synchronise the stream before freeing it.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <initializer_list>
#include <mutex>
#include <string>
#include <utility>

#include "../../include/fusion.h"
#include "kernels.h"

using namespace fusion;

// Scratch of fusion_test_merge_noalloc: a static device array, one copy per
// GPU the library runs on, held until the process ends.  Host code never
// passes the array's name to a kernel (on the host it is a stand-in, not a
// device address): its address on the current device comes from
// hipGetSymbolAddress, looked up once per device.
constexpr size_t kNoAllocScratchBytes = (size_t)1 << 20;
static __device__ __align__(256) char scratch[kNoAllocScratchBytes];

namespace {

int bad(const std::string& m) { return api_fail(FUSION_E_INVALID_ARG, m.c_str()); }

int hip_fail(const char* what, hipError_t e) {
  return api_fail(FUSION_E_HIP, (std::string(what) + ": " + hipGetErrorString(e)).c_str());
}

#define HIP_TRY(expr)                               \
  do {                                              \
    hipError_t e_ = (expr);                         \
    if (e_ != hipSuccess) return hip_fail(#expr, e_); \
  } while (0)

constexpr int kMaxTokens = 640;  // tokens per sample, the adapt / attention limit

// Offsets of a packed ragged batch (host): cu[0] = 0, every sample holds
// 1 .. kMaxTokens rows.  Returns the row count and the largest sample.
int check_offsets(const int32_t* cu, int batch, int* M, int* T_ub) {
  if (!cu) return bad("offsets are null");
  if (batch < 1 || batch > 65536) return bad("batch must be in 1 .. 65536");
  if (cu[0] != 0) return bad("offsets must start at 0");
  int tmax = 0;
  for (int i = 0; i < batch; i++) {
    const long t = (long)cu[i + 1] - cu[i];
    if (t < 1 || t > kMaxTokens)
      return bad("sample " + std::to_string(i) + " has " + std::to_string(t) +
                 " rows (1 .. 640 allowed)");
    tmax = std::max(tmax, (int)t);
  }
  // row offsets into the fp32 rows are 32-bit in the adapt kernel
  if ((long)cu[batch] * 768 > (long)INT32_MAX) return bad("too many rows");
  *M = cu[batch];
  *T_ub = tmax;
  return FUSION_OK;
}

size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

// Scratch of one adaptive-step call, carved from one device buffer.
struct StepScratch {
  int* cu;          // [B + 1]
  int* live;        // [B] identity
  int* rmap;        // [M] identity
  float* size;      // [M] working copy (the merge adds sizes in place)
  int* keep;        // [M]
  int* newlen;      // [B]
  int* r;           // [B]
  LiveCounts* cnt;  // nlive = B, M
  float* sim_v;     // [M / 2] best matches of long samples
  int* sim_i;
};

// with_sim: also the best-match buffers that let long samples spread the
// merge similarity over several workgroups (results are identical without)
size_t step_scratch_bytes(int B, int M, bool with_sim = false) {
  return align256((size_t)(B + 1) * 4) + 3 * align256((size_t)B * 4) +
         3 * align256((size_t)M * 4) + align256(sizeof(LiveCounts)) +
         (with_sim ? 2 * align256((size_t)(M / 2 + 1) * 4) : 0);
}

StepScratch carve(char* p, int B, int M, bool with_sim = false) {
  StepScratch s;
  auto take = [&](size_t bytes) {
    char* q = p;
    p += align256(bytes);
    return q;
  };
  s.cu = (int*)take((size_t)(B + 1) * 4);
  s.live = (int*)take((size_t)B * 4);
  s.newlen = (int*)take((size_t)B * 4);
  s.r = (int*)take((size_t)B * 4);
  s.rmap = (int*)take((size_t)M * 4);
  s.size = (float*)take((size_t)M * 4);
  s.keep = (int*)take((size_t)M * 4);
  s.cnt = (LiveCounts*)take(sizeof(LiveCounts));
  s.sim_v = with_sim ? (float*)take((size_t)(M / 2 + 1) * 4) : nullptr;
  s.sim_i = with_sim ? (int*)take((size_t)(M / 2 + 1) * 4) : nullptr;
  return s;
}

// Per-call device scratch: allocated here, freed after the stream has
// drained (the kernels read it until then).
struct CallScratch {
  char* p = nullptr;
  hipStream_t s;
  explicit CallScratch(hipStream_t s_) : s(s_) {}
  hipError_t alloc(size_t bytes) { return hipMalloc((void**)&p, bytes); }
  ~CallScratch() {
    if (p) {
      hipStreamSynchronize(s);
      hipFree(p);
    }
  }
};

int check_ragged(const fusion_ragged* in, int* M, int* T_ub) {
  if (!in) return bad("ragged input is null");
  if (!in->x || !in->size || !in->origin) return bad("null row buffer");
  if (in->d < 32 || in->d > 768 || in->d % 32) return bad("width d must be a multiple of 32 in 32 .. 768");
  return check_offsets(in->cu, in->batch, M, T_ub);
}

int check_packed_out(const fusion_packed_out* o) {
  if (!o) return bad("packed output is null");
  if (!o->rows || !o->size || !o->origin || !o->cu || !o->live || !o->counts)
    return bad("null packed output buffer");
  return FUSION_OK;
}

// The caller's workspace of a _ws entry: large enough, 256-byte aligned, and
// not under graph capture (the offsets and counts are those of the call).
int check_ws(const void* ws, size_t bytes, size_t need, hipStream_t s) {
  if (!ws || (uintptr_t)ws % 256) return bad("workspace is null or not 256-byte aligned");
  if (bytes < need)
    return api_fail(FUSION_E_CAPACITY, ("the call needs " + std::to_string(need) +
                                        " bytes of workspace").c_str());
  hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
  HIP_TRY(hipStreamIsCapturing(s, &st));
  if (st != hipStreamCaptureStatusNone)
    return api_fail(FUSION_E_HIP, "not available while the stream is being captured");
  return FUSION_OK;
}

// Offsets (and merge counts) to the scratch, identity maps, counts; `size`:
// the working copy of the sizes.
StepInit step_init(const StepScratch& sc, int B, int M, const float* size, bool r) {
  StepInit a{};
  a.live = sc.live; a.rmap = sc.rmap; a.cnt = sc.cnt; a.cu = sc.cu;
  a.r = r ? sc.r : nullptr;
  a.size_in = size; a.size_out = sc.size;
  a.B = B; a.M = M;
  return a;
}

template <typename T>
int compact(const fusion_ragged* in, const StepScratch& sc, int T_ub,
            const float* ln_g, const float* ln_b, void* ln_out,
            const fusion_packed_out* o, bool fill, hipStream_t s) {
  CompactArgs c{};
  c.x = in->x; c.rmap = sc.rmap; c.size = sc.size; c.origin = in->origin;
  c.cu = sc.cu; c.live = sc.live; c.cnt = sc.cnt; c.keep = sc.keep; c.newlen = sc.newlen;
  c.rmap2 = o->rows; c.size2 = o->size; c.origin2 = o->origin; c.cu2 = o->cu;
  c.live2 = o->live; c.cnt2 = (LiveCounts*)o->counts;
  c.d = in->d; c.n0 = T_ub - 1; c.B = in->batch; c.b = 1; c.tr_ids = nullptr;
  c.nlive_ub = in->batch;
  c.ln_g = ln_g; c.ln_b = ln_b; c.ln_out = ln_out;
  c.fill_rows = fill ? in->cu[in->batch] : 0;
  HIP_TRY(launch_compact<T>(c, s));
  return FUSION_OK;
}

int merge_impl(const fusion_ragged* in, const int32_t* r, int id_stride, int32_t* merge_dst,
               const fusion_packed_out* out, hipStream_t s, char* mem, size_t mem_cap,
               int* M_out, bool with_sim, bool fill = false) {
  int M = 0, T_ub = 0;
  if (int rc = check_ragged(in, &M, &T_ub)) return rc;
  if (int rc = check_packed_out(out)) return rc;
  if (!r) return bad("merge counts are null");
  for (int i = 0; i < in->batch; i++) {
    const int N = in->cu[i + 1] - in->cu[i] - 1;
    if (r[i] < 0 || r[i] > N / 2)
      return bad("merge count of sample " + std::to_string(i) + " outside 0 .. floor(N/2)");
  }
  if (merge_dst && (id_stride < 1 || id_stride > (1 << 20))) return bad("id_stride out of range");
  *M_out = M;
  if (!mem) return FUSION_OK;  // sizing pass
  if (step_scratch_bytes(in->batch, M, with_sim) > mem_cap) return bad("scratch too small");
  StepScratch sc = carve(mem, in->batch, M, with_sim);
  StepInit st = step_init(sc, in->batch, M, in->size, true);
  if (fill && merge_dst) st.fill[0] = {merge_dst, (size_t)in->batch * id_stride, 0xFFFFFFFFu};
  HIP_TRY(launch_step_init(st, in->cu, r, s));
  AdaptArgs a{};
  a.x = in->x; a.rmap = sc.rmap; a.size = sc.size; a.origin = in->origin;
  a.cu = sc.cu; a.live = sc.live; a.cnt = sc.cnt;
  a.d = in->d; a.H = 1; a.n0 = merge_dst ? id_stride - 1 : T_ub - 1; a.C = 0; a.L = 1;
  a.B = in->batch; a.b = 1;
  a.isM = 1; a.isE = 0; a.isP = 0;
  a.r_fixed = sc.r; a.rho = 1.0; a.delta = 1.0f; a.tau_eff = 1.0;
  a.tmax = T_ub; a.keep = sc.keep; a.newlen = sc.newlen;
  a.tr_merge = merge_dst;
  a.sim_v = sc.sim_v; a.sim_i = sc.sim_i;
  a.nlive_ub = in->batch; a.T_ub = T_ub;
  HIP_TRY(launch_adapt(a, s));
  return compact<float>(in, sc, T_ub, nullptr, nullptr, nullptr, out, fill, s);
}

int check_attention(int precision, const void* qkv, const float* size, const int32_t* cu,
                    int batch, int heads, int d, int prop_attn, const void* out,
                    const float* cls_scores, int tmax, int* M, int* T_ub) {
  if (precision != 0 && precision != 1) return bad("precision must be 0 (fp32) or 1 (bf16)");
  if (!qkv || !size || !out) return bad("null buffer");
  if (heads < 1 || d < 1 || d % heads || d % 4 || d > 768) return bad("bad width or heads");
  if (prop_attn != 0 && prop_attn != 1) return bad("prop_attn must be 0 or 1");
  if (int rc = check_offsets(cu, batch, M, T_ub)) return rc;
  if (cls_scores && tmax < *T_ub) return bad("tmax below the longest sample");
  if (precision == 1 && d / heads != 64) return bad("the bf16 attention kernels need 64-wide heads");
  return FUSION_OK;
}

int attention_impl(int precision, const void* qkv, const float* size, const int32_t* cu, int batch,
                   int heads, int d, int prop_attn, void* out, float* cls_scores, int tmax, int M,
                   int T_ub, char* mem, bool fill, hipStream_t s) {
  const int dh = d / heads;
  StepScratch sc = carve(mem, batch, M);
  StepInit st = step_init(sc, batch, M, nullptr, false);
  if (fill && cls_scores)
    st.fill[0] = {cls_scores, (size_t)batch * heads * tmax, 0xBF800000u};  // -1.0f
  HIP_TRY(launch_step_init(st, cu, nullptr, s));
  AttnArgs a{};
  a.qkv = qkv; a.size = size; a.cu = sc.cu; a.live = sc.live; a.cnt = sc.cnt;
  a.H = heads; a.dh = dh; a.d = d; a.scale = (float)(1.0 / std::sqrt((double)dh));
  a.prop_attn = prop_attn; a.out = out; a.cls_scores = cls_scores; a.tmax = tmax;
  a.token_counts = nullptr; a.L = 1; a.b0 = 0; a.nlive_ub = batch; a.T_ub = T_ub;
  hipError_t err = precision == 1 ? launch_attention<bf16_t>(a, s) : launch_attention<float>(a, s);
  if (err != hipSuccess) return hip_fail("launch_attention", err);
  return FUSION_OK;
}

int check_topk(const fusion_ragged* in, const float* scores, int heads, int tmax,
               const float* prune_w, const float* prune_b, double keep_ratio,
               const float* exit_logits, int classes, float delta, const float* logits,
               const int32_t* exit_block, int precision, const float* ln_g, const float* ln_b,
               const void* ln_out, const fusion_packed_out* out, int* M, int* T_ub) {
  if (int rc = check_ragged(in, M, T_ub)) return rc;
  if (int rc = check_packed_out(out)) return rc;
  if (!scores && !(prune_w && prune_b)) return bad("give CLS-attention scores or a learned scorer");
  if (scores && (heads < 1 || heads > 64 || tmax < *T_ub)) return bad("bad score layout");
  if (!(keep_ratio >= 0.0 && keep_ratio <= 1.0)) return bad("keep ratio outside [0, 1]");
  if (exit_logits) {
    if (classes < 1 || !logits || !exit_block) return bad("exit check needs classes, logits and exit_block");
    if (!(delta >= 0.f && delta <= 1.f)) return bad("threshold outside [0, 1]");
  }
  if (precision != 0 && precision != 1) return bad("precision must be 0 (fp32) or 1 (bf16)");
  if (ln_out && (!ln_g || !ln_b)) return bad("LayerNorm output needs its gain and bias");
  return FUSION_OK;
}

int topk_impl(const fusion_ragged* in, const float* scores, int heads, int tmax,
              const float* prune_w, const float* prune_b, double keep_ratio,
              const float* exit_logits, int classes, float delta, float* logits,
              int32_t* exit_block, int precision, const float* ln_g, const float* ln_b,
              void* ln_out, const fusion_packed_out* out, int M, int T_ub, char* mem, bool fill,
              hipStream_t s) {
  StepScratch sc = carve(mem, in->batch, M);
  StepInit st = step_init(sc, in->batch, M, in->size, false);
  if (fill && exit_logits) {
    st.fill[0] = {logits, (size_t)in->batch * classes, 0xC0E00000u};  // -7.0f
    st.fill[1] = {exit_block, (size_t)in->batch, 0xFFFFFFFFu};
  }
  HIP_TRY(launch_step_init(st, in->cu, nullptr, s));
  AdaptArgs a{};
  a.x = in->x; a.rmap = sc.rmap; a.size = sc.size; a.origin = in->origin;
  a.cu = sc.cu; a.live = sc.live; a.cnt = sc.cnt;
  a.d = in->d; a.H = scores ? heads : 1; a.n0 = T_ub - 1; a.C = exit_logits ? classes : 0;
  a.L = 1; a.B = in->batch; a.b = 1;
  a.isM = 0; a.isE = exit_logits ? 1 : 0; a.isP = 1;
  a.prune_rule = scores ? FUSION_PRUNE_CLS_ATTN : FUSION_PRUNE_LEARNED;
  a.prune_w = prune_w; a.prune_b = prune_b;
  a.head_buf = exit_logits; a.delta = exit_logits ? delta : 1.0f;
  a.logits = logits; a.exit_block = exit_block;
  a.cls_scores = scores; a.tmax = tmax; a.tau_eff = keep_ratio;
  a.keep = sc.keep; a.newlen = sc.newlen;
  a.nlive_ub = in->batch; a.T_ub = T_ub;
  HIP_TRY(launch_adapt(a, s));
  if (precision == 1) return compact<bf16_t>(in, sc, T_ub, ln_g, ln_b, ln_out, out, fill, s);
  return compact<float>(in, sc, T_ub, ln_g, ln_b, ln_out, out, fill, s);
}

// Arguments shared by the calls on long sequences and token caches.
int check_heads(int precision, int heads, int kv_heads, int dh) {
  if (precision != 0 && precision != 1) return bad("precision must be 0 (fp32) or 1 (bf16)");
  if (kv_heads < 1 || heads < 1 || heads > 4096 || heads % kv_heads)
    return bad("heads must be a multiple of kv_heads, at most 4096");
  if (dh < 8 || dh > 128 || dh % 8) return bad("head width must be a multiple of 8 in 8 .. 128");
  return FUSION_OK;
}

int check_rows(const int32_t* cu, int batch) {
  if (!cu) return bad("offsets are null");
  if (batch < 1 || batch > 65536) return bad("batch must be in 1 .. 65536");
  if (cu[0] != 0) return bad("offsets must start at 0");
  for (int i = 0; i < batch; i++)
    if (cu[i + 1] < cu[i]) return bad("offsets must not decrease");
  if (cu[batch] > (1 << 30)) return bad("more than 2^30 rows");
  return FUSION_OK;
}

int check_strides(int precision, const int64_t* strides, int n) {
  for (int i = 0; i < n; i++)
    if (strides[i] < 0 || strides[i] % (precision == 1 ? 8 : 4))
      return bad("strides must be multiples of 16 bytes, not negative");
  return FUSION_OK;
}

int check_space(const void* ws, size_t bytes, size_t need) {
  if (!ws || (uintptr_t)ws % 256) return bad("workspace is null or not 256-byte aligned");
  if (bytes < need)
    return api_fail(FUSION_E_CAPACITY, ("the call needs " + std::to_string(need) +
                                        " bytes of workspace").c_str());
  return FUSION_OK;
}

// (sc: the scales of a cache in 4 bits, else null)
int check_cache(const fusion_cache* c, CacheArgs* a, const fusion_cache_scales* sc = nullptr) {
  if (!c) return bad("cache is null");
  if (int rc = check_heads(c->precision, c->kv_heads, c->kv_heads, c->dh)) return rc;
  if (c->batch < 1 || c->batch > 65536) return bad("batch must be in 1 .. 65536");
  if (c->pages < 1 || c->page_size < 1 || c->max_pages < 1)
    return bad("pages, page_size and max_pages must be positive");
  if ((int64_t)c->max_pages * c->page_size > (1 << 30)) return bad("capacity above 2^30 slots");
  if ((int64_t)c->batch * c->max_pages * c->page_size > (int64_t)1 << 34)
    return bad("more than 2^34 slots");
  if (!c->k || !c->v || !c->table || !c->len || !c->seen || !c->weight || !c->pos)
    return bad("null cache buffer");
  if (((uintptr_t)c->k | (uintptr_t)c->v) % 16) return bad("buffers must be 16-byte aligned");
  if (sc) {
    if (!sc->k || !sc->v) return bad("null scales");
    if (c->dh % 32) return bad("a cache in 4 bits needs a head width that is a multiple of 32");
    for (int i = 0; i < 3; i++) {
      if (c->k_strides[i] < 0 || c->k_strides[i] % 16 || c->v_strides[i] < 0 || c->v_strides[i] % 16)
        return bad("strides must be multiples of 16 bytes, not negative");
      if (sc->k_strides[i] < 0 || sc->v_strides[i] < 0) return bad("strides must not be negative");
    }
  } else {
    if (int rc = check_strides(c->precision, c->k_strides, 3)) return rc;
    if (int rc = check_strides(c->precision, c->v_strides, 3)) return rc;
  }
  *a = CacheArgs{c->k, c->v, c->k_strides[0], c->k_strides[1], c->k_strides[2],
                 c->v_strides[0], c->v_strides[1], c->v_strides[2], c->table, c->len, c->seen,
                 c->weight, c->pos, c->batch, c->pages, c->max_pages,
                 c->max_pages * c->page_size, c->kv_heads, c->dh,
                 fast_div((uint32_t)c->page_size), nullptr, nullptr, 0, 0, 0, 0, 0, 0};
  if (sc) {
    a->ks = sc->k; a->vs = sc->v;
    a->ks_page = sc->k_strides[0]; a->ks_row = sc->k_strides[1]; a->ks_head = sc->k_strides[2];
    a->vs_page = sc->v_strides[0]; a->vs_row = sc->v_strides[1]; a->vs_head = sc->v_strides[2];
  }
  return FUSION_OK;
}

// Memory of a tensor, from its first byte to the one past its last (0 to 0: none); rows
// of n elements at the strides of some dims.
struct Span {
  uintptr_t first, past;
};
Span span(const void* p, size_t bytes) { return p && bytes ? Span{(uintptr_t)p, (uintptr_t)p + bytes} : Span{0, 0}; }
Span span(const void* p, std::initializer_list<std::pair<int64_t, int64_t>> dims, int64_t n, size_t size) {
  if (!p) return {0, 0};
  unsigned __int128 last = n;
  for (auto [count, stride] : dims) {
    if (count < 1) return {0, 0};
    last += (unsigned __int128)(count - 1) * (uint64_t)stride;
  }
  const unsigned __int128 past = (uintptr_t)p + last * size;
  return {(uintptr_t)p, past > UINTPTR_MAX ? UINTPTR_MAX : (uintptr_t)past};
}
bool overlap(Span a, Span b) { return a.first < b.past && b.first < a.past; }

// A cache's tensors: those that an append writes, then the table.
constexpr int kCacheSpans = 9;
struct CacheSpans {
  Span s[kCacheSpans];
};
CacheSpans cache_spans(const fusion_cache* c, const CacheArgs& ca, const fusion_cache_scales* sc) {
  const size_t size = sc ? 1 : c->precision == 1 ? 2 : 4, batch = c->batch, slots = batch * ca.cap;
  auto pages = [&](const void* p, const int64_t* st, int64_t n, size_t bytes) {
    return span(p, {{c->pages, st[0]}, {c->page_size, st[1]}, {c->kv_heads, st[2]}}, n, bytes);
  };
  const int64_t held = sc ? c->dh / 2 : c->dh;
  const Span none{0, 0};
  return {{pages(c->k, c->k_strides, held, size), pages(c->v, c->v_strides, held, size),
           sc ? pages(sc->k, sc->k_strides, c->dh / 32, 1) : none,
           sc ? pages(sc->v, sc->v_strides, c->dh / 32, 1) : none, span(c->len, batch * 4),
           span(c->seen, batch * 4), span(c->weight, slots * 4), span(c->pos, slots * 4),
           span(c->table, batch * c->max_pages * 4)}};
}
// Outputs overlap neither each other nor the cache nor what else is read.
bool outputs_apart(std::initializer_list<Span> out, const CacheSpans& cache, std::initializer_list<Span> in) {
  bool shared = false;
  for (const Span& w : out) {
    for (const Span& x : out) shared |= &x != &w && overlap(w, x);
    for (const Span& x : in) shared |= overlap(w, x);
    for (const Span& x : cache.s) shared |= overlap(w, x);
  }
  return !shared;
}

// What an append of turned rows reads and writes lies apart.
int check_apart(const fusion_cache* c, const CacheArgs& ca, const fusion_cache_scales* sc,
                const fusion_rotary_rows* r, int rows) {
  const size_t size = c->precision == 1 ? 2 : 4;
  const CacheSpans cache = cache_spans(c, ca, sc);
  auto heads = [&](const void* p, const int64_t* st, int n) {
    return span(p, {{rows, st[0]}, {n, st[1]}}, c->dh, size);
  };
  const Span q = heads(r->q, r->q_strides, r->heads), k = heads(r->k, r->k_strides, c->kv_heads),
             v = heads(r->v, r->v_strides, c->kv_heads), freq = span(r->freq, (size_t)r->half * 4),
             drop = span(r->drop, (size_t)c->batch * 4);
  bool shared = !outputs_apart({span(r->q_out, (size_t)rows * r->heads * c->dh * size),
                                span(r->k_out, (size_t)rows * c->kv_heads * c->dh * size)},
                               cache, {q, k, v, freq, drop});
  // (a sequence's drop is read before its length and position are written)
  const bool own = r->drop == c->len || r->drop == c->seen;
  for (int i = 0; i < kCacheSpans - 1; i++) {
    const Span& w = cache.s[i];
    shared |= overlap(w, q) | overlap(w, k) | overlap(w, v) | overlap(w, freq) | (!own && overlap(w, drop));
  }
  return shared ? bad("rows, freq or drop overlap what the call writes of the cache, or an output overlaps one of them")
                : FUSION_OK;
}

// Queries, output and workspace of one new token per sequence.
int check_queries(const fusion_cache* c, const void* q, const int64_t* strides, const void* out) {
  if (!q || !strides || !out) return bad("null buffer");
  if (int rc = check_strides(c->precision, strides, 2)) return rc;
  if (((uintptr_t)q | (uintptr_t)out) % 16) return bad("buffers must be 16-byte aligned");
  return FUSION_OK;
}
PagedArgs paged_args(const fusion_cache* c, const CacheArgs& ca, const void* q, const int64_t* strides, int heads, int window,
                     int sinks, int accumulate, void* out, void* ws) {
  PagedArgs a{};
  a.q = q; a.q_row = strides[0]; a.q_head = strides[1]; a.out = out;
  a.H = heads; a.group = heads / c->kv_heads;
  a.window = window; a.sinks = sinks; a.accumulate = accumulate;
  a.scale = (float)(1.0 / std::sqrt((double)c->dh)); a.ws = ws;
  a.flat = ca.ks && window == 0 && c->page_size % 16 == 0 &&
           ((ca.k_page | ca.v_page | ca.ks_page | ca.vs_page) >> 32) == 0 &&
           ((ca.k_row | ca.v_row | ca.ks_row | ca.vs_row) >> 26) == 0;
  return a;
}
size_t paged_bytes(const fusion_cache* c, const CacheArgs& a, int heads, int accumulate) {
  if (a.ks)
    return c->precision == 1 ? paged4_workspace_bytes<bf16_t>(a, heads, accumulate)
                             : paged4_workspace_bytes<float>(a, heads, accumulate);
  return c->precision == 1 ? paged_workspace_bytes<bf16_t>(a, heads, accumulate)
                           : paged_workspace_bytes<float>(a, heads, accumulate);
}
int paged_attention(const fusion_cache* c, const fusion_cache_scales* sc, const void* q,
                    const int64_t* strides, int heads, int window, int sinks, int accumulate, void* out,
                    void* ws, size_t ws_bytes, void* stream) {
  CacheArgs ca;
  if (int rc = check_cache(c, &ca, sc)) return rc;
  if (int rc = check_heads(c->precision, heads, c->kv_heads, c->dh)) return rc;
  if (window < 0 || sinks < 0) return bad("window and sinks must not be negative");
  if (accumulate != 0 && accumulate != 1) return bad("accumulate must be 0 or 1");
  if (int rc = check_queries(c, q, strides, out)) return rc;
  if (int rc = check_space(ws, ws_bytes, paged_bytes(c, ca, heads, accumulate))) return rc;
  const PagedArgs a = paged_args(c, ca, q, strides, heads, window, sinks, accumulate, out, ws);
  hipStream_t s = (hipStream_t)stream;
  hipError_t err;
  if (sc)
    err = c->precision == 1 ? launch_paged4_attention<bf16_t>(ca, a, s) : launch_paged4_attention<float>(ca, a, s);
  else
    err = c->precision == 1 ? launch_paged_attention<bf16_t>(ca, a, s) : launch_paged_attention<float>(ca, a, s);
  return err == hipSuccess ? FUSION_OK : hip_fail("launch_paged_attention", err);
}
int cache_evict(const fusion_cache* c, const fusion_cache_scales* sc, int budget, int sinks, int recent,
                int32_t* src, void* ws, size_t ws_bytes, void* stream) {
  CacheArgs ca;
  if (int rc = check_cache(c, &ca, sc)) return rc;
  if (budget < 1 || budget > kNoWindow) return bad("budget must be in 1 .. 2^30");
  if (sinks < 0 || recent < 0 || (int64_t)sinks + recent > budget)
    return bad("sinks and recent must not be negative and fit the budget together");
  if (!src) return bad("null buffer");
  if (int rc = check_space(ws, ws_bytes, evict_workspace_bytes(ca, budget))) return rc;
  const EvictArgs a{budget, sinks, recent, src, ws};
  hipStream_t s = (hipStream_t)stream;
  hipError_t err = c->precision == 1 ? launch_cache_evict<bf16_t>(ca, a, s)
                                     : launch_cache_evict<float>(ca, a, s);
  return err == hipSuccess ? FUSION_OK : hip_fail("launch_cache_evict", err);
}

// Device address of `scratch` on the current device, looked up on the
// first call on each device (with that device current) and kept.
constexpr int kMaxDevices = 64;
std::mutex g_scratch_mu;
char* g_scratch_ptr[kMaxDevices] = {};

int noalloc_scratch(char** out) {
  int dev = 0;
  HIP_TRY(hipGetDevice(&dev));
  if (dev < 0 || dev >= kMaxDevices) return bad("device index beyond the scratch table");
  std::lock_guard<std::mutex> lock(g_scratch_mu);
  if (!g_scratch_ptr[dev]) {
    void* ptr = nullptr;
    HIP_TRY(hipGetSymbolAddress((void**)&ptr, HIP_SYMBOL(scratch)));
    if (!ptr) return api_fail(FUSION_E_HIP, "no device address for the static scratch");
    g_scratch_ptr[dev] = (char*)ptr;
  }
  *out = g_scratch_ptr[dev];
  return FUSION_OK;
}

}  // namespace

extern "C" {

FUSION_API int fusion_test_gemm(int precision, const void* A, int lda, const void* W, int N,
                                int K, int M, const float* bias, int epi, void* out, int ldo,
                                const int32_t* rows, void* stream) {
  if (precision != 0 && precision != 1) return bad("precision must be 0 (fp32) or 1 (bf16)");
  if (!A || !W || !bias || !out) return bad("null buffer");
  if (M < 1 || N < 4 || K < 1) return bad("M >= 1, N >= 4 and K >= 1 required");
  if (epi < FUSION_EPI_STORE || epi > FUSION_EPI_F32) return bad("unknown epilogue");
  if (lda < K || ldo < N) return bad("leading dimensions below K / N");
  if (rows && (epi == FUSION_EPI_STORE || epi == FUSION_EPI_GELU))
    return bad("a row map applies to the fp32 epilogues only");
  if (precision == 1) {
    if (K % 32 || lda % 8) return bad("bf16 GEMM needs K % 32 == 0 and lda % 8 == 0");
    if (N % 4 || ldo % 4) return bad("bf16 GEMM needs N and ldo multiples of 4");
    if ((epi == FUSION_EPI_STORE || epi == FUSION_EPI_GELU) && (N % 8 || ldo % 8))
      return bad("bf16 outputs need N and ldo multiples of 8");
  }
  const int mode = epi == FUSION_EPI_STORE ? EPI_STORE
                   : epi == FUSION_EPI_GELU ? EPI_GELU
                   : epi == FUSION_EPI_RESID ? EPI_RESID : EPI_F32;
  Epi e{mode, out, ldo, bias, rows, nullptr, 0};
  hipStream_t s = (hipStream_t)stream;
  hipError_t err =
      precision == 1
          ? launch_gemm<bf16_t>((const bf16_t*)A, lda, (const bf16_t*)W, N, K, nullptr, M, M, 0, e, s)
          : launch_gemm<float>((const float*)A, lda, (const float*)W, N, K, nullptr, M, M, 0, e, s);
  if (err != hipSuccess) return hip_fail("launch_gemm", err);
  return FUSION_OK;
}

FUSION_API size_t fusion_test_workspace_bytes(int batch, int rows) {
  if (batch < 1 || batch > 65536 || rows < 1) return 0;
  return step_scratch_bytes(batch, rows, true);
}

FUSION_API int fusion_test_attention(int precision, const void* qkv, const float* size,
                                     const int32_t* cu, int batch, int heads, int d,
                                     int prop_attn, void* out, float* cls_scores, int tmax,
                                     void* stream) {
  hipStream_t s = (hipStream_t)stream;
  int M = 0, T_ub = 0;
  if (int rc = check_attention(precision, qkv, size, cu, batch, heads, d, prop_attn, out,
                               cls_scores, tmax, &M, &T_ub))
    return rc;
  CallScratch mem(s);
  HIP_TRY(mem.alloc(step_scratch_bytes(batch, M)));
  return attention_impl(precision, qkv, size, cu, batch, heads, d, prop_attn, out, cls_scores,
                        tmax, M, T_ub, mem.p, false, s);
}

FUSION_API int fusion_test_attention_ws(int precision, const void* qkv, const float* size,
                                        const int32_t* cu, int batch, int heads, int d,
                                        int prop_attn, void* out, float* cls_scores, int tmax,
                                        void* ws, size_t ws_bytes, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  int M = 0, T_ub = 0;
  if (int rc = check_attention(precision, qkv, size, cu, batch, heads, d, prop_attn, out,
                               cls_scores, tmax, &M, &T_ub))
    return rc;
  if (int rc = check_ws(ws, ws_bytes, step_scratch_bytes(batch, M), s)) return rc;
  return attention_impl(precision, qkv, size, cu, batch, heads, d, prop_attn, out, cls_scores,
                        tmax, M, T_ub, (char*)ws, true, s);
}

FUSION_API int fusion_test_merge(const fusion_ragged* in, const int32_t* r, int id_stride,
                                 int32_t* merge_dst, const fusion_packed_out* out,
                                 void* stream) {
  hipStream_t s = (hipStream_t)stream;
  int M = 0;
  if (int rc = merge_impl(in, r, id_stride, merge_dst, out, s, nullptr, 0, &M, true)) return rc;
  CallScratch mem(s);
  const size_t need = step_scratch_bytes(in->batch, M, true);
  HIP_TRY(mem.alloc(need));
  return merge_impl(in, r, id_stride, merge_dst, out, s, mem.p, need, &M, true);
}

FUSION_API int fusion_test_merge_ws(const fusion_ragged* in, const int32_t* r, int id_stride,
                                    int32_t* merge_dst, const fusion_packed_out* out, void* ws,
                                    size_t ws_bytes, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  int M = 0;
  if (int rc = merge_impl(in, r, id_stride, merge_dst, out, s, nullptr, 0, &M, true)) return rc;
  if (int rc = check_ws(ws, ws_bytes, step_scratch_bytes(in->batch, M, true), s)) return rc;
  return merge_impl(in, r, id_stride, merge_dst, out, s, (char*)ws, ws_bytes, &M, true, true);
}

FUSION_API int fusion_test_merge_noalloc(const fusion_ragged* in, const int32_t* r,
                                         int id_stride, int32_t* merge_dst,
                                         const fusion_packed_out* out, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  int M = 0;
  if (int rc = merge_impl(in, r, id_stride, merge_dst, out, s, nullptr, 0, &M, false)) return rc;
  const size_t need = step_scratch_bytes(in->batch, M);
  if (need > kNoAllocScratchBytes)
    return api_fail(FUSION_E_CAPACITY,
                    ("the call needs " + std::to_string(need) + " bytes of scratch; the static " +
                     "array holds " + std::to_string(kNoAllocScratchBytes))
                        .c_str());
  char* mem = nullptr;
  if (int rc = noalloc_scratch(&mem)) return rc;
  // every scratch word the kernels read is written earlier in this call
  // (offsets, counts and sizes copied in, maps set by the init kernel, keep
  // flags and new lengths by the adapt kernel), so nothing is cleared
  return merge_impl(in, r, id_stride, merge_dst, out, s, mem, kNoAllocScratchBytes, &M, false);
}

FUSION_API int fusion_test_topk_compact(const fusion_ragged* in, const float* scores, int heads,
                                        int tmax, const float* prune_w, const float* prune_b,
                                        double keep_ratio, const float* exit_logits,
                                        int classes, float delta, float* logits,
                                        int32_t* exit_block, int precision, const float* ln_g,
                                        const float* ln_b, void* ln_out,
                                        const fusion_packed_out* out, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  int M = 0, T_ub = 0;
  if (int rc = check_topk(in, scores, heads, tmax, prune_w, prune_b, keep_ratio, exit_logits,
                          classes, delta, logits, exit_block, precision, ln_g, ln_b, ln_out, out,
                          &M, &T_ub))
    return rc;
  CallScratch mem(s);
  HIP_TRY(mem.alloc(step_scratch_bytes(in->batch, M)));
  return topk_impl(in, scores, heads, tmax, prune_w, prune_b, keep_ratio, exit_logits, classes,
                   delta, logits, exit_block, precision, ln_g, ln_b, ln_out, out, M, T_ub, mem.p,
                   false, s);
}

FUSION_API int fusion_test_topk_compact_ws(const fusion_ragged* in, const float* scores, int heads,
                                           int tmax, const float* prune_w, const float* prune_b,
                                           double keep_ratio, const float* exit_logits,
                                           int classes, float delta, float* logits,
                                           int32_t* exit_block, int precision, const float* ln_g,
                                           const float* ln_b, void* ln_out,
                                           const fusion_packed_out* out, void* ws,
                                           size_t ws_bytes, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  int M = 0, T_ub = 0;
  if (int rc = check_topk(in, scores, heads, tmax, prune_w, prune_b, keep_ratio, exit_logits,
                          classes, delta, logits, exit_block, precision, ln_g, ln_b, ln_out, out,
                          &M, &T_ub))
    return rc;
  if (int rc = check_ws(ws, ws_bytes, step_scratch_bytes(in->batch, M), s)) return rc;
  return topk_impl(in, scores, heads, tmax, prune_w, prune_b, keep_ratio, exit_logits, classes,
                   delta, logits, exit_block, precision, ln_g, ln_b, ln_out, out, M, T_ub, (char*)ws,
                   true, s);
}

FUSION_API int fusion_window_attention(int precision, const void* q, const void* k, const void* v,
                                       const int64_t* strides, const float* size,
                                       const int32_t* cu, int batch, int heads, int kv_heads,
                                       int dh, int window, int sinks, int causal, void* out,
                                       void* stream) {
  if (int rc = check_heads(precision, heads, kv_heads, dh)) return rc;
  if (int rc = check_rows(cu, batch)) return rc;
  if (window < 0 || sinks < 0) return bad("window and sinks must not be negative");
  if (causal != 0 && causal != 1) return bad("causal must be 0 or 1");
  if (cu[batch] == 0) return FUSION_OK;  // no rows
  if (!q || !k || !v || !strides || !out) return bad("null buffer");
  if (int rc = check_strides(precision, strides, 6)) return rc;
  if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)out) % 16)
    return bad("buffers must be 16-byte aligned");
  // (a tile's rows are addressed by 32-bit byte offsets from its first)
  if (strides[2] > (1 << 23) || strides[4] > (1 << 23))
    return bad("row strides of k and v must be at most 2^23");
  WindowArgs a{};
  a.q = q; a.k = k; a.v = v; a.size = size; a.out = out;
  a.q_row = strides[0]; a.q_head = strides[1]; a.k_row = strides[2]; a.k_head = strides[3];
  a.v_row = strides[4]; a.v_head = strides[5];
  a.H = heads; a.group = heads / kv_heads; a.dh = dh;
  a.window = window == 0 ? kNoWindow : std::min(window, kNoWindow);
  a.sinks = std::min(sinks, kNoWindow); a.causal = causal;
  a.scale = (float)(1.0 / std::sqrt((double)dh));
  hipStream_t s = (hipStream_t)stream;
  hipError_t err = precision == 1 ? launch_window_attention<bf16_t>(a, cu, batch, s)
                                  : launch_window_attention<float>(a, cu, batch, s);
  return err == hipSuccess ? FUSION_OK : hip_fail("launch_window_attention", err);
}

FUSION_API int fusion_cache_append(const fusion_cache* c, const void* k, const void* v,
                                   const int64_t* strides, const int32_t* cu, void* stream) {
  CacheArgs ca;
  if (int rc = check_cache(c, &ca)) return rc;
  if (cu) {
    if (int rc = check_rows(cu, c->batch)) return rc;
    if (cu[c->batch] == 0) return FUSION_OK;  // no rows
  }
  if (!k || !v || !strides) return bad("null buffer");
  if (int rc = check_strides(c->precision, strides, 4)) return rc;
  if (((uintptr_t)k | (uintptr_t)v) % 16) return bad("buffers must be 16-byte aligned");
  const AppendArgs a{k, v, strides[0], strides[1], strides[2], strides[3]};
  hipStream_t s = (hipStream_t)stream;
  hipError_t err = c->precision == 1 ? launch_cache_append<bf16_t>(ca, a, cu, s)
                                     : launch_cache_append<float>(ca, a, cu, s);
  return err == hipSuccess ? FUSION_OK : hip_fail("launch_cache_append", err);
}

FUSION_API size_t fusion_paged_attention_workspace_bytes(const fusion_cache* c, int heads,
                                                         int accumulate) {
  CacheArgs ca;
  if (check_cache(c, &ca) || check_heads(c->precision, heads, c->kv_heads, c->dh)) return 0;
  return paged_bytes(c, ca, heads, accumulate);
}

FUSION_API int fusion_paged_attention(const fusion_cache* c, const void* q, const int64_t* strides,
                                      int heads, int window, int sinks, int accumulate, void* out,
                                      void* ws, size_t ws_bytes, void* stream) {
  return paged_attention(c, nullptr, q, strides, heads, window, sinks, accumulate, out, ws, ws_bytes, stream);
}

FUSION_API size_t fusion_cache_evict_workspace_bytes(const fusion_cache* c, int budget) {
  CacheArgs ca;
  if (check_cache(c, &ca) || budget < 1) return 0;
  return evict_workspace_bytes(ca, budget);
}

FUSION_API int fusion_cache_evict(const fusion_cache* c, int budget, int sinks, int recent,
                                  int32_t* src, void* ws, size_t ws_bytes, void* stream) {
  return cache_evict(c, nullptr, budget, sinks, recent, src, ws, ws_bytes, stream);
}

FUSION_API size_t fusion_cache4_attention_workspace_bytes(const fusion_cache* c,
                                                          const fusion_cache_scales* sc, int heads,
                                                          int accumulate) {
  CacheArgs ca;
  if (!sc) { bad("null scales"); return 0; }
  if (check_cache(c, &ca, sc) || check_heads(c->precision, heads, c->kv_heads, c->dh)) return 0;
  return paged_bytes(c, ca, heads, accumulate);
}

FUSION_API int fusion_cache4_attention(const fusion_cache* c, const fusion_cache_scales* sc, const void* q,
                                       const int64_t* strides, int heads, int window, int sinks,
                                       int accumulate, void* out, void* ws, size_t ws_bytes,
                                       void* stream) {
  if (!sc) return bad("null scales");
  return paged_attention(c, sc, q, strides, heads, window, sinks, accumulate, out, ws, ws_bytes, stream);
}

FUSION_API size_t fusion_cache4_evict_workspace_bytes(const fusion_cache* c, const fusion_cache_scales* sc,
                                                      int budget) {
  CacheArgs ca;
  if (!sc) { bad("null scales"); return 0; }
  if (check_cache(c, &ca, sc) || budget < 1) return 0;
  return evict_workspace_bytes(ca, budget);
}

FUSION_API int fusion_cache4_evict(const fusion_cache* c, const fusion_cache_scales* sc, int budget, int sinks,
                                   int recent, int32_t* src, void* ws, size_t ws_bytes, void* stream) {
  if (!sc) return bad("null scales");
  return cache_evict(c, sc, budget, sinks, recent, src, ws, ws_bytes, stream);
}

FUSION_API int fusion_cache_append_rotary(const fusion_cache* c, const fusion_cache_scales* sc,
                                          const fusion_rotary_rows* r, const int32_t* cu, void* stream) {
  CacheArgs ca;
  if (int rc = check_cache(c, &ca, sc)) return rc;
  if (!r) return bad("rows are null");
  if (r->heads < 0 || r->heads > 4096) return bad("heads must be in 0 .. 4096");
  if (r->half < 0 || r->half % 4 || r->half > c->dh / 2)
    return bad("the frequencies must be a multiple of 4, for no more dims than a head has");
  if (r->half > 0 && !r->freq) return bad("null frequencies");
  if (r->interleaved != 0 && r->interleaved != 1) return bad("interleaved must be 0 or 1");
  if (cu) {
    if (int rc = check_rows(cu, c->batch)) return rc;
    if (cu[c->batch] == 0 && !r->drop) return FUSION_OK;  // no rows
  }
  if (!cu || cu[c->batch] > 0) {
    if (!r->k || !r->v || (r->heads > 0 && (!r->q || !r->q_out))) return bad("null buffer");
  }
  if (int rc = check_strides(c->precision, r->q_strides, 2)) return rc;
  if (int rc = check_strides(c->precision, r->k_strides, 2)) return rc;
  if (int rc = check_strides(c->precision, r->v_strides, 2)) return rc;
  if (((uintptr_t)r->q | (uintptr_t)r->k | (uintptr_t)r->v | (uintptr_t)r->q_out | (uintptr_t)r->k_out) % 16)
    return bad("buffers must be 16-byte aligned");
  if (int rc = check_apart(c, ca, sc, r, cu ? cu[c->batch] : c->batch)) return rc;
  const RotaryArgs a{r->q, r->k, r->v, r->q_strides[0], r->q_strides[1], r->k_strides[0], r->k_strides[1],
                     r->v_strides[0], r->v_strides[1], r->q_out, r->k_out, r->freq, r->drop,
                     r->heads, r->half, r->interleaved};
  hipStream_t s = (hipStream_t)stream;
  hipError_t err = c->precision == 1 ? launch_append_rotary<bf16_t>(ca, a, cu, s)
                                     : launch_append_rotary<float>(ca, a, cu, s);
  return err == hipSuccess ? FUSION_OK : hip_fail("launch_append_rotary", err);
}

FUSION_API int fusion_page_bounds(const fusion_cache* c, const fusion_cache_scales* sc, void* lo, void* hi,
                                  int newest, void* stream) {
  CacheArgs ca;
  if (int rc = check_cache(c, &ca, sc)) return rc;
  if (newest < 0) return bad("newest must not be negative");
  if (!lo || !hi) return bad("null buffer");
  if (((uintptr_t)lo | (uintptr_t)hi) % 16) return bad("buffers must be 16-byte aligned");
  const size_t bytes = (size_t)c->pages * c->kv_heads * c->dh * (c->precision == 1 ? 2 : 4);
  if (!outputs_apart({span(lo, bytes), span(hi, bytes)}, cache_spans(c, ca, sc), {}))
    return bad("bounds overlap each other or the cache");
  const BoundsArgs a{lo, hi, newest};
  hipStream_t s = (hipStream_t)stream;
  hipError_t err = c->precision == 1 ? launch_page_bounds<bf16_t>(ca, a, s)
                                     : launch_page_bounds<float>(ca, a, s);
  return err == hipSuccess ? FUSION_OK : hip_fail("launch_page_bounds", err);
}

FUSION_API size_t fusion_block_attention_workspace_bytes(const fusion_cache* c,
                                                         const fusion_cache_scales* sc, int heads,
                                                         int blocks) {
  CacheArgs ca;
  if (check_cache(c, &ca, sc) || check_heads(c->precision, heads, c->kv_heads, c->dh)) return 0;
  if (blocks < 1 || blocks > kNoWindow) { bad("blocks must be in 1 .. 2^30"); return 0; }
  return c->precision == 1 ? block_workspace_bytes<bf16_t>(ca, heads, blocks)
                           : block_workspace_bytes<float>(ca, heads, blocks);
}

FUSION_API int fusion_block_attention(const fusion_cache* c, const fusion_cache_scales* sc, const void* lo,
                                      const void* hi, const void* q, const int64_t* strides, int heads,
                                      int blocks, int first, int recent, void* out, int32_t* chosen,
                                      void* ws, size_t ws_bytes, void* stream) {
  CacheArgs ca;
  if (int rc = check_cache(c, &ca, sc)) return rc;
  if (int rc = check_heads(c->precision, heads, c->kv_heads, c->dh)) return rc;
  if (blocks < 1 || blocks > kNoWindow) return bad("blocks must be in 1 .. 2^30");
  if (first < 0 || recent < 1 || (int64_t)first + recent > blocks)
    return bad("recent must be at least 1, first not negative, and the blocks hold both");
  if (int rc = check_queries(c, q, strides, out)) return rc;
  if (!lo || !hi || !chosen) return bad("null buffer");
  if (((uintptr_t)lo | (uintptr_t)hi) % 16) return bad("buffers must be 16-byte aligned");
  const size_t need = c->precision == 1 ? block_workspace_bytes<bf16_t>(ca, heads, blocks)
                                        : block_workspace_bytes<float>(ca, heads, blocks);
  if (int rc = check_space(ws, ws_bytes, need)) return rc;
  const size_t size = c->precision == 1 ? 2 : 4, bytes = (size_t)c->pages * c->kv_heads * c->dh * size;
  if (!outputs_apart({span(out, (size_t)c->batch * heads * c->dh * size),
                      span(chosen, (size_t)c->batch * c->kv_heads * blocks * 4), span(ws, need)},
                     cache_spans(c, ca, sc),
                     {span(lo, bytes), span(hi, bytes),
                      span(q, {{c->batch, strides[0]}, {heads, strides[1]}}, c->dh, size)}))
    return bad("out, chosen or ws overlap each other or what the call reads");
  BlockArgs a{paged_args(c, ca, q, strides, heads, 0, 0, 0, out, ws), lo, hi, first, recent, chosen};
  a.p.blocks = blocks;
  hipStream_t s = (hipStream_t)stream;
  hipError_t err = c->precision == 1 ? launch_block_attention<bf16_t>(ca, a, s)
                                     : launch_block_attention<float>(ca, a, s);
  return err == hipSuccess ? FUSION_OK : hip_fail("launch_block_attention", err);
}

}  // extern "C"
