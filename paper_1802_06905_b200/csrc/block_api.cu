// Entry points of the feed-forward sub-block (include/cconv_block.h): checks of arguments, workspace
// layout, launches.  Nothing here allocates or synchronises (cconv_block_status synchronises).
#include <algorithm>
#include <cmath>
#include <cstring>
#include <numeric>
#include <string>
#include <vector>

#include "block.h"
#include "block_clip.h"
#include "block_ffn.h"
#include "block_fp8.h"
#include "block_gemm.h"
#include "block_int4.h"
#include "block_moe.h"
#include "block_norm.h"
#include "block_quant.h"
#include "host_setup.h"

namespace cconv {

int block_cuda_error(cudaError_t e, const char* where) {
  if (e == cudaSuccess) return CCONV_OK;
  set_last_cuda_error(std::string(where) + ": " + cudaGetErrorString(e));
  return CCONV_ECUDA;
}

int block_sm_count() {
  static int counts[64] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return block_cuda_error(e, "cudaGetDevice");
  if (dev < 0 || dev >= 64) return CCONV_EUNSUPPORTED;
  int n = __atomic_load_n(&counts[dev], __ATOMIC_RELAXED);
  if (n == 0) {
    int major = 0;
    e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev);
    if (e != cudaSuccess) return block_cuda_error(e, "cudaDeviceGetAttribute");
    if (major != 10) return CCONV_EUNSUPPORTED;
    __atomic_store_n(&counts[dev], n, __ATOMIC_RELAXED);
  }
  return n;
}

int64_t& block_launches() {
  static thread_local int64_t n = 0;
  return n;
}

namespace {

constexpr int64_t kMaxLength = (int64_t(1) << 31) - 1024;  // of one dimension: coordinates of tiles are 32 bits
constexpr int64_t kMaxStride = int64_t(1) << 40;

// The bytes of an operand: [lo, hi), and where they are rows at a pitch, `width` bytes of every `pitch`; its
// elements of `unit` bytes begin multiples of `step` bytes behind lo (0: it is one element).
struct Bytes {
  const char *lo = nullptr, *hi = nullptr;
  int64_t pitch = 0, width = 0, unit = 1, step = 1;
  // Whether b, which repeats every `period` bytes like this, lies beside these `mine` bytes of each period.
  bool beside(const Bytes& b, int64_t period, int64_t mine, int64_t its) const {
    const int64_t d = ((b.lo - lo) % period + period) % period;
    return d >= mine && d + its <= period;
  }
  bool meets(const Bytes& o) const {
    if (lo >= o.hi || o.lo >= hi) return false;
    if (pitch && pitch == o.pitch && beside(o, pitch, width, o.width)) return false;  // column slices of one array
    const int64_t each = std::gcd(step, o.step);
    return each == 0 || !beside(o, each, unit, o.unit);  // columns of one array in turn
  }
  bool operator==(const Bytes& o) const { return lo == o.lo && hi == o.hi && pitch == o.pitch && width == o.width && step == o.step; }
};

// The bytes of an operand of rows x cols > 0 elements; whether they can be an operand's (of a result: are distinct).
bool bytes_of(const cconv_matrix& m, int64_t rows, int64_t cols, int es, bool written, Bytes* out) {
  if (!m.data || (reinterpret_cast<uintptr_t>(m.data) & uintptr_t(es - 1)) || m.row_stride < 0 || m.col_stride < 0 ||
      m.row_stride > kMaxStride || m.col_stride > kMaxStride)
    return false;
  const double last = double(rows - 1) * double(m.row_stride) + double(cols - 1) * double(m.col_stride);
  if (last > 4.0e18 / es) return false;
  bool ok = true;
  if (written) {
    // distinct elements: one stride steps over the whole extent of the other
    const int64_t r = m.row_stride, c = m.col_stride;
    const bool rows_outer = (rows == 1 || r > (cols - 1) * c) && (cols == 1 || c > 0);
    const bool cols_outer = (cols == 1 || c > (rows - 1) * r) && (rows == 1 || r > 0);
    ok = rows_outer || cols_outer;
  }
  const char* lo = static_cast<const char*>(m.data);
  Bytes b{lo, lo + ((rows - 1) * m.row_stride + (cols - 1) * m.col_stride + 1) * es, 0, 0, es,
          std::gcd(rows > 1 ? m.row_stride * es : 0, cols > 1 ? m.col_stride * es : 0)};
  const int64_t wr = ((cols - 1) * m.col_stride + 1) * es, wc = ((rows - 1) * m.row_stride + 1) * es;
  if (rows > 1 && m.row_stride * es >= wr) b.pitch = m.row_stride * es, b.width = wr;
  else if (cols > 1 && m.col_stride * es >= wc) b.pitch = m.col_stride * es, b.width = wc;
  *out = b;
  return ok;
}

// Collects the byte ranges that a call reads and writes, and checks each operand on the way.
class Operands {
 public:
  bool ok = true;
  // An operand of rows x cols elements, or a vector; inputs may repeat rows and columns.  Its number, or -1 if it
  // has no element.
  int in(const cconv_matrix& m, int64_t rows, int64_t cols, int es) { return add(m, rows, cols, es, false); }
  int out(const cconv_matrix& m, int64_t rows, int64_t cols, int es) { return add(m, rows, cols, es, true); }
  int in(const void* v, int64_t n, int es) { return in(vec(v, n), 1, n, es); }
  int out(const void* v, int64_t n, int es) { return out(vec(v, n), 1, n, es); }
  // The result `out` may be written in the place of `in`, if they are one and the same matrix (numbers from above).
  void may_be_one(int in, int out) {
    in_ = in;
    out_ = out;
  }
  void workspace(void* p, uint64_t have, int64_t need) {
    if (need == 0) return;
    if (!p || (reinterpret_cast<uintptr_t>(p) & 255u) || have < uint64_t(need)) {
      ok = false;
      return;
    }
    push({static_cast<const char*>(p), static_cast<const char*>(p) + need}, true);
  }
  // Whether any result has an element.  A call without one launches nothing and needs no device.
  bool writes() const {
    for (int i = 0; i < n_; ++i)
      if (written_[i]) return true;
    return false;
  }
  // Runs the launches of a call with these operands, and then tells the stream's bookkeeping that it is under
  // way: its kernels wait for the work in front of them (which the bookkeeping may forget from now on), but let
  // the next be put in place, so that a convolution whose arrays meet these (their hulls, which may take in
  // more) has to wait for it too.  A call that failed before its first launch waits for nothing: no entry.
  template <typename F>
  int run(void* stream, int sms, F launches) const {
    const int64_t before = block_launches();
    const int rc = launches();
    if (block_launches() != before) note(stream, sms);
    return rc;
  }
  // No output meets another output or an input, but for the pair that may be one.
  bool distinct() const {
    for (int i = 0; i < n_; ++i)
      for (int j = 0; j < n_; ++j) {
        if (i == j || !written_[i] || (written_[j] && j < i)) continue;
        if (i == out_ && j == in_ && range_[i] == range_[j]) continue;
        if (range_[i].meets(range_[j])) return false;
      }
    return ok;
  }

 private:
  void note(void* stream, int sms) const {
    CallSpans c;
    for (int i = 0; i < n_; ++i) {
      Span& s = written_[i] ? c.out : c.image;
      if (!s.lo || range_[i].lo < s.lo) s.lo = range_[i].lo;
      if (!s.hi || range_[i].hi > s.hi) s.hi = range_[i].hi;
    }
    note_call(stream, c, Overlap::kInputsEarly, sms);
  }
  static cconv_matrix vec(const void* v, int64_t n) { return cconv_matrix{const_cast<void*>(v), n, 1}; }
  int push(Bytes b, bool written) {
    range_[n_] = b;
    written_[n_] = written;
    return n_++;
  }
  int add(const cconv_matrix& m, int64_t rows, int64_t cols, int es, bool written) {
    if (rows == 0 || cols == 0) return -1;  // nothing is touched
    Bytes b;
    if (!bytes_of(m, rows, cols, es, written, &b)) ok = false;
    if (!b.lo) return -1;
    return push(b, written);
  }
  Bytes range_[24];
  bool written_[24] = {};
  int n_ = 0, in_ = -1, out_ = -1;
};

bool length_ok(int64_t n) { return n >= 0 && n < kMaxLength; }

// Runs the body of an entry point; nothing is thrown through the C boundary.
template <typename F>
auto guarded(F f) noexcept -> decltype(f()) {
  try {
    return f();
  } catch (...) {  // host memory ran out: nothing else here throws
    return CCONV_ENOMEM;
  }
}

// ---- feed-forward --------------------------------------------------------------------------------
bool ffn_sizes_ok(const cconv_ffn_args& a) {
  return length_ok(a.T) && length_ok(a.D) && length_ok(a.F) &&
         (a.dtype == CCONV_TYPE_BF16 || a.dtype == CCONV_TYPE_FP16) && a.act >= CCONV_ACT_SILU &&
         a.act <= CCONV_ACT_RELU && double(a.T) * a.F < 1e15 && double(a.D) * a.F < 1e15 && double(a.T) * a.D < 1e15;
}

cudaError_t zero_rows(void* p, int64_t pitch, int64_t bytes, int64_t rows, cudaStream_t s) {
  const cudaError_t e = cudaMemset2DAsync(p, size_t(pitch), 0, size_t(bytes), size_t(rows), s);
  block_launches() += e == cudaSuccess;
  return e;
}
cudaError_t zero_out(const cconv_matrix& m, int64_t rows, int64_t cols, int es, cudaStream_t s) {
  if (rows == 0 || cols == 0) return cudaSuccess;
  if (m.col_stride == 1 || cols == 1) return zero_rows(m.data, (rows == 1 ? cols : m.row_stride) * es, cols * es, rows, s);
  if (m.row_stride == 1 || rows == 1) return zero_rows(m.data, (cols == 1 ? rows : m.col_stride) * es, rows * es, cols, s);
  for (int64_t r = 0; r < rows; ++r) {
    const cudaError_t e = zero_rows(static_cast<char*>(m.data) + r * m.row_stride * es, m.col_stride * es, es, cols, s);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

#define BLOCK_CUDA(call)                                              \
  do {                                                                \
    const cudaError_t e_ = (call);                                    \
    if (e_ != cudaSuccess) return block_cuda_error(e_, "feed-forward sub-block");     \
  } while (0)

bool ffn_empty(const cconv_ffn_args& a) { return a.T == 0 || a.D == 0 || a.F == 0; }
// Where a length is zero every result is empty or an empty sum.
int ffn_zeros(const cconv_ffn_args& a, bool backward, cudaStream_t s) {
  if (!backward) {
    BLOCK_CUDA(zero_out(a.out, a.T, a.D, 2, s));
    if (a.gate_pre.data) BLOCK_CUDA(zero_out(a.gate_pre, a.T, a.F, 2, s));
    if (a.up_pre.data) BLOCK_CUDA(zero_out(a.up_pre, a.T, a.F, 2, s));
    return CCONV_OK;
  }
  BLOCK_CUDA(zero_out(a.dx, a.T, a.D, 2, s));
  BLOCK_CUDA(zero_out(a.dw_gate, a.F, a.D, 2, s));
  BLOCK_CUDA(zero_out(a.dw_up, a.F, a.D, 2, s));
  BLOCK_CUDA(zero_out(a.dw_down, a.D, a.F, 2, s));
  return CCONV_OK;
}
int64_t ffn_bytes(const cconv_ffn_args* a, bool backward) {
  if (!a || !ffn_sizes_ok(*a)) return CCONV_EINVAL;
  const int sms = block_sm_count();
  if (sms < 0) return sms;
  return ffn_empty(*a) ? 0 : ffn_workspace(*a, backward, sms);
}

// ---- residual norm -------------------------------------------------------------------------------
bool norm_sizes_ok(const cconv_residual_norm_args& a) {
  return length_ok(a.T) && length_ok(a.D) && a.dtype >= CCONV_TYPE_BF16 && a.dtype <= CCONV_TYPE_FP32 &&
         a.rows_per_gate >= 0 && a.rows_per_gate <= kMaxStride && std::isfinite(a.scale) && std::isfinite(a.eps) &&
         a.eps > 0 && double(a.T) * a.D < 1e15;
}
bool unit(const cconv_matrix& m, int64_t cols) { return !m.data || cols <= 1 || m.col_stride == 1; }
int64_t gate_rows(const cconv_residual_norm_args& a) { return a.rows_per_gate ? cdiv64(a.T, a.rows_per_gate) : 1; }

NormParams norm_params(const cconv_residual_norm_args& a) {
  NormParams p{};
  p.T = a.T;
  p.D = int(a.D);
  p.scale = a.scale;
  p.eps = a.eps;
  p.rows_per_gate = a.rows_per_gate >= a.T ? 0 : a.rows_per_gate;
  p.resid = a.resid.data; p.resid_rs = a.resid.row_stride;
  p.block = a.block.data; p.block_rs = a.block.row_stride;
  p.gate = a.gate.data; p.gate_rs = a.gate.row_stride;
  p.w_post = a.w_post;
  p.w_pre = a.w_pre;
  p.resid_out = a.resid_out.data; p.resid_out_rs = a.resid_out.row_stride;
  p.norm_out = a.norm_out.data; p.norm_out_rs = a.norm_out.row_stride;
  p.dresid_out = a.dresid_out.data; p.dresid_out_rs = a.dresid_out.row_stride;
  p.dnorm_out = a.dnorm_out.data; p.dnorm_out_rs = a.dnorm_out.row_stride;
  p.dresid = a.dresid.data; p.dresid_rs = a.dresid.row_stride;
  p.dblock = a.dblock.data; p.dblock_rs = a.dblock.row_stride;
  p.dgate = a.dgate.data; p.dgate_rs = a.dgate.row_stride;
  p.dw_post = a.dw_post;
  p.dw_pre = a.dw_pre;
  return p;
}

// The row stride of a matrix of one row is never used; a made-up one must not look misaligned or overlapping.
cconv_matrix same_row(cconv_matrix m, int64_t rows, int64_t cols) {
  if (rows <= 1) m.row_stride = cols;
  if (cols <= 1) m.col_stride = 1;
  return m;
}

int64_t norm_workspace(const cconv_residual_norm_args& a, int sms) {
  if (a.T == 0 || a.D == 0) return 0;
  const int64_t nb = norm_backward_blocks(a.T, a.D, type_bytes(a.dtype), sms);
  return round_up64(nb * 5 * a.D * 4, 256);
}

// The forward call; with q and q_scale the second norm's result goes there in 8 bits.
int norm_forward(cconv_residual_norm_args a, const cconv_matrix* q, const cconv_matrix* q_scale, void* cuda_stream) {
  if (!norm_sizes_ok(a)) return CCONV_EINVAL;
  const int es = type_bytes(a.dtype);
  a.resid = same_row(a.resid, a.T, a.D);
  a.block = same_row(a.block, a.T, a.D);
  a.gate = same_row(a.gate, gate_rows(a), a.D);
  a.resid_out = same_row(a.resid_out, a.T, a.D);
  a.norm_out = same_row(a.norm_out, a.T, a.D);
  if (!unit(a.resid, a.D) || !unit(a.block, a.D) || !unit(a.gate, a.D) || !unit(a.resid_out, a.D) || !unit(a.norm_out, a.D))
    return CCONV_EINVAL;
  if (a.T && a.D && ((!a.block.data && (a.gate.data || a.w_post)) || (!a.norm_out.data && !q && a.w_pre))) return CCONV_EINVAL;
  Operands o;
  const int resid = o.in(a.resid, a.T, a.D, es);
  if (a.block.data) o.in(a.block, a.T, a.D, es);
  if (a.gate.data) o.in(a.gate, gate_rows(a), a.D, es);
  if (a.w_post) o.in(a.w_post, a.D, es);
  if (a.w_pre) o.in(a.w_pre, a.D, es);
  o.may_be_one(resid, o.out(a.resid_out, a.T, a.D, es));
  if (a.norm_out.data) o.out(a.norm_out, a.T, a.D, es);
  cconv_matrix values{}, scales{};
  if (q) {
    values = same_row(*q, a.T, a.D);
    scales = same_row(*q_scale, a.T, cdiv64(a.D, 128));
    if (!unit(values, a.D)) return CCONV_EINVAL;
    o.out(values, a.T, a.D, 1);
    o.out(scales, a.T, cdiv64(a.D, 128), 4);
  }
  if (!o.distinct()) return CCONV_EINVAL;
  if (!o.writes()) return CCONV_OK;
  const int sms = block_sm_count();
  if (sms < 0) return sms;
  NormParams p = norm_params(a);
  p.q = static_cast<uint8_t*>(values.data); p.q_rs = values.row_stride;
  p.q_scale = static_cast<float*>(scales.data); p.q_scale_rs = scales.row_stride; p.q_scale_cs = scales.col_stride;
  const int rc = block_status_word(&p.status);
  if (rc != CCONV_OK) return rc;
  p.limit_ns = block_wait_limit_ns();
  return o.run(cuda_stream, sms, [&] {
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    return block_cuda_error(q ? run_norm_quantize(p, a.dtype, sms, s) : run_norm_forward(p, a.dtype, sms, s),
                            "cconv_residual_norm_forward");
  });
}

bool fp8_sizes_ok(const cconv_fp8_product_args& a) {
  return length_ok(a.M) && length_ok(a.N) && length_ok(a.K) && a.dtype >= CCONV_TYPE_BF16 &&
         a.dtype <= CCONV_TYPE_FP32 && a.reserved == 0 && double(a.M) * a.N < 1e15 && double(a.M) * a.K < 1e15 &&
         double(a.N) * a.K < 1e15;
}

bool type_ok(int32_t t) { return t >= CCONV_TYPE_BF16 && t <= CCONV_TYPE_FP32; }

// ---- clipping ------------------------------------------------------------------------------------
constexpr int64_t kMostTensors = 1 << 20;

bool clip_sizes_ok(const cconv_clip_args& a, bool clips) {
  if (a.count < 0 || a.count > kMostTensors || (a.count && !a.grads) || a.reserved != 0 || a.norm_given < 0 || a.norm_given > 1)
    return false;
  if (clips && (!(a.max_norm >= 0) || !(a.eps >= 0) || !std::isfinite(a.eps) || !(a.max_norm + a.eps > 0))) return false;
  double all = 0;
  for (int64_t i = 0; i < a.count; ++i) {
    const cconv_tensor& g = a.grads[i];
    if (g.rows < 0 || g.cols < 0 || !type_ok(g.dtype) || g.reserved != 0) return false;
    all += double(g.rows) * double(g.cols);
    if (clips && a.outs) {
      const cconv_tensor& o = a.outs[i];
      if (o.rows != g.rows || o.cols != g.cols || o.dtype != g.dtype || o.reserved != 0) return false;
    }
  }
  return all < 1e15;
}

cconv_matrix matrix_of(const cconv_tensor& t) {
  return cconv_matrix{t.data, t.rows > 1 ? t.row_stride : t.cols, t.cols > 1 ? t.col_stride : 1};
}

// The operands of a call of any number of tensors: checked, told from one another in the order of their addresses,
// and noted in the stream's bookkeeping.
class Tensors {
 public:
  bool ok = true;
  explicit Tensors(size_t n) { all_.reserve(n); }
  void add(const cconv_matrix& m, int64_t rows, int64_t cols, int es, bool written, int64_t of) {
    if (rows == 0 || cols == 0) return;
    Entry e{{}, written, of};
    if (!bytes_of(m, rows, cols, es, written, &e.bytes)) ok = false;
    else all_.push_back(e);
  }
  // No result meets anything but its own gradient (`of` equal) lying in the very same place.
  bool distinct() {
    std::vector<std::pair<const char*, const Entry*>> order;
    order.reserve(all_.size());
    for (const Entry& e : all_) order.emplace_back(e.bytes.lo, &e);
    std::sort(order.begin(), order.end());
    std::vector<const Entry*> open;  // those that reach beyond the current one's start
    for (const auto& at : order) {
      const Entry& e = *at.second;
      size_t kept = 0;
      for (const Entry* o : open) {
        if (o->bytes.hi <= e.bytes.lo) continue;
        open[kept++] = o;
        if (!o->written && !e.written) continue;
        if (o->of == e.of && o->written != e.written && o->bytes == e.bytes) continue;
        if (o->bytes.meets(e.bytes)) return false;
      }
      open.resize(kept);
      open.push_back(&e);
    }
    return ok;
  }
  void note(void* stream, int sms) const {
    CallSpans c;
    for (const Entry& e : all_) {
      Span& s = e.written ? c.out : c.image;
      if (!s.lo || e.bytes.lo < s.lo) s.lo = e.bytes.lo;
      if (!s.hi || e.bytes.hi > s.hi) s.hi = e.bytes.hi;
    }
    note_call(stream, c, Overlap::kInputsEarly, sms);
  }

 private:
  struct Entry {
    Bytes bytes;
    bool written;
    int64_t of;  // the tensor's number
  };
  std::vector<Entry> all_;
};

int clip_call(const cconv_clip_args& a, bool clips, void* cuda_stream) {
  if (!clip_sizes_ok(a, clips)) return CCONV_EINVAL;
  const bool sums = !clips || !a.norm_given;
  bool any = false;
  Tensors o(size_t(a.count) * 2 + 2);
  for (int64_t i = 0; i < a.count; ++i) {
    const cconv_tensor& g = a.grads[i];
    const int es = type_bytes(g.dtype);
    any |= g.rows && g.cols;
    o.add(matrix_of(g), g.rows, g.cols, es, clips && !a.outs, i);
    if (clips && a.outs) o.add(matrix_of(a.outs[i]), g.rows, g.cols, es, true, i);
  }
  o.add(cconv_matrix{a.norm, 1, 1}, 1, 1, 4, sums, -1);
  if (!o.distinct()) return CCONV_EINVAL;
  if (!any && !sums) return CCONV_OK;
  const int sms = block_sm_count();
  if (sms < 0) return sms;
  const int64_t need = sums ? clip_workspace(a, sms) : 0;
  if (need) {
    if (!a.workspace || (reinterpret_cast<uintptr_t>(a.workspace) & 255u) || a.workspace_bytes < uint64_t(need)) return CCONV_EINVAL;
    o.add(cconv_matrix{a.workspace, need, 1}, 1, need, 1, true, -2);
  }
  if (!o.distinct()) return CCONV_EINVAL;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const int64_t before = block_launches();
  int n = 0, rc = sums && any ? run_square_sums(a, sms, &n, s) : CCONV_OK;
  if (rc == CCONV_OK) rc = clips && any ? run_clip(a, sms, n, s) : run_norm_of_sums(a, n, s);
  if (block_launches() != before) o.note(cuda_stream, sms);
  return rc;
}

// ---- mixture of experts --------------------------------------------------------------------------
bool moe_sizes_ok(const cconv_moe_args& a) {
  return a.T >= 0 && a.T <= (1 << 20) && a.D >= 0 && a.D <= (1 << 29) && a.F >= 0 && a.F <= (1 << 29) && a.E >= 0 && a.E <= kMostExperts &&
         (a.dtype == CCONV_TYPE_BF16 || a.dtype == CCONV_TYPE_FP16) && a.act >= CCONV_ACT_SILU && a.act <= CCONV_ACT_RELU &&
         a.top_k >= 1 && a.top_k <= kMostChosen && (a.normalize == 0 || a.normalize == 1) &&
         (!a.router.data || a.top_k <= a.E || a.T == 0) && double(a.D) * a.F < 1e12 && double(a.T) * a.D < 1e15 &&
         double(a.T) * a.F < 1e13;
}
bool moe_empty(const cconv_moe_args& a) { return a.T == 0 || a.D == 0 || a.F == 0 || a.E == 0; }
// Whether anything but zeros comes of the call: without hidden channels the router still chooses.
bool moe_runs(const cconv_moe_args& a) { return a.T && a.D && a.E && (a.F || a.router.data); }
// The matrices of all experts as one vector of their elements' hull; false if it is none.
bool experts_ok(const cconv_matrix& m, int64_t stride, int64_t rows, int64_t cols, int64_t experts, int64_t* n) {
  for (int64_t s : {m.row_stride, m.col_stride, stride})
    if (s < 0 || s > kMaxStride) return false;
  const double last = double(rows - 1) * m.row_stride + double(cols - 1) * m.col_stride + double(experts - 1) * stride;
  if (last > 2.0e18) return false;
  *n = (rows - 1) * m.row_stride + (cols - 1) * m.col_stride + (experts - 1) * stride + 1;
  return true;
}

bool group_ok(int32_t group) { return group == 32 || group == 64 || group == 128; }
bool int4_sizes_ok(const cconv_int4_product_args& a) {
  return length_ok(a.M) && length_ok(a.N) && length_ok(a.K) && (a.dtype == CCONV_TYPE_BF16 || a.dtype == CCONV_TYPE_FP16) &&
         type_ok(a.scale_dtype) && group_ok(a.group) && a.reserved == 0 && double(a.M) * a.N < 1e15 &&
         double(a.M) * a.K < 1e15 && double(a.N) * a.K < 1e15;
}
bool int4_empty(const cconv_int4_product_args& a) { return a.M == 0 || a.N == 0 || a.K == 0; }

bool fp8_empty(const cconv_fp8_product_args& a) { return a.M == 0 || a.N == 0 || a.K == 0; }

}  // namespace
}  // namespace cconv

using namespace cconv;

extern "C" {

int64_t cconv_ffn_forward_workspace(const cconv_ffn_args* args) {
  return guarded([&] { return ffn_bytes(args, false); });
}
int64_t cconv_ffn_backward_workspace(const cconv_ffn_args* args) {
  return guarded([&] { return ffn_bytes(args, true); });
}

int cconv_ffn_forward(const cconv_ffn_args* args, void* cuda_stream) {
  return guarded([&]() -> int {
    if (!args || !ffn_sizes_ok(*args)) return CCONV_EINVAL;
    const cconv_ffn_args& a = *args;
    if (!a.gate_pre.data != !a.up_pre.data && a.T && a.F) return CCONV_EINVAL;
    Operands o;
    o.in(a.x, a.T, a.D, 2);
    o.in(a.w_gate, a.F, a.D, 2);
    o.in(a.w_up, a.F, a.D, 2);
    o.in(a.w_down, a.D, a.F, 2);
    o.out(a.out, a.T, a.D, 2);
    if (a.gate_pre.data) {
      o.out(a.gate_pre, a.T, a.F, 2);
      o.out(a.up_pre, a.T, a.F, 2);
    }
    if (!o.distinct()) return CCONV_EINVAL;
    if (!o.writes()) return CCONV_OK;
    const int sms = block_sm_count();
    if (sms < 0) return sms;
    o.workspace(a.workspace, a.workspace_bytes, ffn_empty(a) ? 0 : ffn_workspace(a, false, sms));
    if (!o.distinct()) return CCONV_EINVAL;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    return o.run(cuda_stream, sms, [&] { return ffn_empty(a) ? ffn_zeros(a, false, s) : run_ffn(a, false, sms, s); });
  });
}

int cconv_ffn_backward(const cconv_ffn_args* args, void* cuda_stream) {
  return guarded([&]() -> int {
    if (!args || !ffn_sizes_ok(*args)) return CCONV_EINVAL;
    const cconv_ffn_args& a = *args;
    Operands o;
    o.in(a.dout, a.T, a.D, 2);
    o.in(a.x, a.T, a.D, 2);
    o.in(a.w_gate, a.F, a.D, 2);
    o.in(a.w_up, a.F, a.D, 2);
    o.in(a.w_down, a.D, a.F, 2);
    o.in(a.gate_pre, a.T, a.F, 2);
    o.in(a.up_pre, a.T, a.F, 2);
    o.out(a.dx, a.T, a.D, 2);
    o.out(a.dw_gate, a.F, a.D, 2);
    o.out(a.dw_up, a.F, a.D, 2);
    o.out(a.dw_down, a.D, a.F, 2);
    if (!o.distinct()) return CCONV_EINVAL;
    if (!o.writes()) return CCONV_OK;
    const int sms = block_sm_count();
    if (sms < 0) return sms;
    o.workspace(a.workspace, a.workspace_bytes, ffn_empty(a) ? 0 : ffn_workspace(a, true, sms));
    if (!o.distinct()) return CCONV_EINVAL;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    return o.run(cuda_stream, sms, [&] { return ffn_empty(a) ? ffn_zeros(a, true, s) : run_ffn(a, true, sms, s); });
  });
}

int64_t cconv_residual_norm_backward_workspace(const cconv_residual_norm_args* args) {
  return guarded([&]() -> int64_t {
    if (!args || !norm_sizes_ok(*args)) return CCONV_EINVAL;
    const int sms = block_sm_count();
    if (sms < 0) return sms;
    return norm_workspace(*args, sms);
  });
}

int cconv_residual_norm_forward(const cconv_residual_norm_args* args, void* cuda_stream) {
  return guarded([&]() -> int { return args ? norm_forward(*args, nullptr, nullptr, cuda_stream) : CCONV_EINVAL; });
}

int cconv_residual_norm_quantize(const cconv_residual_norm_quantize_args* args, void* cuda_stream) {
  return guarded([&]() -> int {
    return args ? norm_forward(args->norm, &args->q, &args->q_scale, cuda_stream) : CCONV_EINVAL;
  });
}

int cconv_residual_norm_backward(const cconv_residual_norm_args* args, void* cuda_stream) {
  return guarded([&]() -> int {
    if (!args || !norm_sizes_ok(*args)) return CCONV_EINVAL;
    cconv_residual_norm_args a = *args;
    const int es = type_bytes(a.dtype);
    a.block = same_row(a.block, a.T, a.D);
    a.gate = same_row(a.gate, gate_rows(a), a.D);
    a.resid_out = same_row(a.resid_out, a.T, a.D);
    a.dresid_out = same_row(a.dresid_out, a.T, a.D);
    a.dnorm_out = same_row(a.dnorm_out, a.T, a.D);
    a.dresid = same_row(a.dresid, a.T, a.D);
    a.dblock = same_row(a.dblock, a.T, a.D);
    a.dgate = same_row(a.dgate, gate_rows(a), a.D);
    for (const cconv_matrix* m : {&a.block, &a.gate, &a.resid_out, &a.dresid_out, &a.dnorm_out, &a.dresid, &a.dblock, &a.dgate})
      if (!unit(*m, a.D)) return CCONV_EINVAL;
    if (a.T && a.D) {
      if (!a.block.data && (a.gate.data || a.w_post)) return CCONV_EINVAL;
      if (!a.block.data != !a.dblock.data) return CCONV_EINVAL;
      if (!a.dnorm_out.data && !a.dresid_out.data) return CCONV_EINVAL;
    }
    if (a.D && (!a.gate.data != !a.dgate.data || !a.w_post != !a.dw_post)) return CCONV_EINVAL;
    // (without tokens dnorm_out may be given with no address, or absent: dw_pre is zeroed if it is there)
    if (a.D && a.dw_pre && !a.w_pre) return CCONV_EINVAL;
    if (a.T && a.D && (a.w_pre && a.dnorm_out.data) != (a.dw_pre != nullptr)) return CCONV_EINVAL;
    Operands o;
    if (a.block.data) o.in(a.block, a.T, a.D, es);
    if (a.gate.data) o.in(a.gate, gate_rows(a), a.D, es);
    if (a.w_post) o.in(a.w_post, a.D, es);
    if (a.w_pre) o.in(a.w_pre, a.D, es);
    if (a.dnorm_out.data) o.in(a.resid_out, a.T, a.D, es);
    const int direct = a.dresid_out.data ? o.in(a.dresid_out, a.T, a.D, es) : -1;
    if (a.dnorm_out.data) o.in(a.dnorm_out, a.T, a.D, es);
    o.may_be_one(direct, o.out(a.dresid, a.T, a.D, es));
    if (a.dblock.data) o.out(a.dblock, a.T, a.D, es);
    if (a.dgate.data) o.out(a.dgate, gate_rows(a), a.D, es);
    if (a.dw_post) o.out(a.dw_post, a.D, es);
    if (a.dw_pre) o.out(a.dw_pre, a.D, es);
    if (!o.distinct()) return CCONV_EINVAL;
    if (!o.writes()) return CCONV_OK;
    const int sms = block_sm_count();
    if (sms < 0) return sms;
    o.workspace(a.workspace, a.workspace_bytes, norm_workspace(a, sms));
    if (!o.distinct()) return CCONV_EINVAL;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    if (a.T == 0) {
      return o.run(cuda_stream, sms, [&]() -> int {
        if (a.dgate.data) BLOCK_CUDA(zero_out(a.dgate, gate_rows(a), a.D, es, s));
        if (a.dw_post) BLOCK_CUDA(zero_rows(a.dw_post, a.D * es, a.D * es, 1, s));
        if (a.dw_pre) BLOCK_CUDA(zero_rows(a.dw_pre, a.D * es, a.D * es, 1, s));
        return CCONV_OK;
      });
    }
    NormParams p = norm_params(a);
    p.nb = norm_backward_blocks(a.T, a.D, type_bytes(a.dtype), sms);
    p.part = static_cast<float*>(a.workspace);
    const int rc = block_status_word(&p.status);
    if (rc != CCONV_OK) return rc;
    p.limit_ns = block_wait_limit_ns();
    return o.run(cuda_stream, sms, [&] {
      return block_cuda_error(run_norm_backward(p, a.dtype, s), "cconv_residual_norm_backward");
    });
  });
}

int64_t cconv_fp8_product_workspace(const cconv_fp8_product_args* args) {
  return guarded([&]() -> int64_t {
    if (!args || !fp8_sizes_ok(*args)) return CCONV_EINVAL;
    const int sms = block_sm_count();
    if (sms < 0) return sms;
    return fp8_empty(*args) ? 0 : fp8_workspace(*args, sms);
  });
}

int cconv_fp8_product(const cconv_fp8_product_args* args, void* cuda_stream) {
  return guarded([&]() -> int {
    if (!args || !fp8_sizes_ok(*args)) return CCONV_EINVAL;
    const cconv_fp8_product_args& a = *args;
    const int es = type_bytes(a.dtype);
    Operands o;
    o.in(a.a, a.M, a.K, 1);
    o.in(a.b, a.N, a.K, 1);
    o.in(a.a_scale, a.M, cdiv64(a.K, 128), 4);
    o.in(a.b_scale, cdiv64(a.N, 128), cdiv64(a.K, 128), 4);
    o.out(a.c, a.M, a.N, es);
    if (!o.distinct()) return CCONV_EINVAL;
    if (!o.writes()) return CCONV_OK;
    const int sms = block_sm_count();
    if (sms < 0) return sms;
    o.workspace(a.workspace, a.workspace_bytes, fp8_empty(a) ? 0 : fp8_workspace(a, sms));
    if (!o.distinct()) return CCONV_EINVAL;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    return o.run(cuda_stream, sms, [&] {
      return fp8_empty(a) ? block_cuda_error(zero_out(a.c, a.M, a.N, es, s), "cconv_fp8_product") : run_fp8(a, sms, s);
    });
  });
}

int cconv_quantize_blocks(const cconv_quantize_args* args, void* cuda_stream) {
  return guarded([&]() -> int {
    if (!args) return CCONV_EINVAL;
    const cconv_quantize_args& a = *args;
    if (!length_ok(a.T) || !length_ok(a.D) || a.dtype < CCONV_TYPE_BF16 || a.dtype > CCONV_TYPE_FP32 ||
        (a.block_rows != 1 && a.block_rows != 128) || double(a.T) * a.D >= 1e15)
      return CCONV_EINVAL;
    Operands o;
    o.in(a.x, a.T, a.D, type_bytes(a.dtype));
    o.out(a.q, a.T, a.D, 1);
    o.out(a.scale, cdiv64(a.T, a.block_rows), cdiv64(a.D, 128), 4);
    if (!o.distinct()) return CCONV_EINVAL;
    if (!o.writes()) return CCONV_OK;
    const int sms = block_sm_count();
    if (sms < 0) return sms;
    QuantParams p{};
    p.T = a.T;
    p.D = a.D;
    p.x = a.x.data; p.x_rs = a.x.row_stride; p.x_cs = a.x.col_stride;
    p.q = static_cast<uint8_t*>(a.q.data); p.q_rs = a.q.row_stride; p.q_cs = a.q.col_stride;
    p.scale = static_cast<float*>(a.scale.data); p.scale_rs = a.scale.row_stride; p.scale_cs = a.scale.col_stride;
    return o.run(cuda_stream, sms, [&] {
      return block_cuda_error(run_quantize(p, a.dtype, a.block_rows, sms, static_cast<cudaStream_t>(cuda_stream)),
                              "cconv_quantize_blocks");
    });
  });
}

int64_t cconv_int4_product_workspace(const cconv_int4_product_args* args) {
  return guarded([&]() -> int64_t {
    if (!args || !int4_sizes_ok(*args)) return CCONV_EINVAL;
    const int sms = block_sm_count();
    if (sms < 0) return sms;
    return int4_empty(*args) ? 0 : int4_workspace(*args, sms);
  });
}

int cconv_int4_product(const cconv_int4_product_args* args, void* cuda_stream) {
  return guarded([&]() -> int {
    if (!args || !int4_sizes_ok(*args)) return CCONV_EINVAL;
    const cconv_int4_product_args& a = *args;
    const int64_t groups = cdiv64(a.K, a.group);
    Operands o;
    o.in(a.x, a.M, a.K, 2);
    o.in(a.q, a.N, cdiv64(a.K, 2), 1);
    o.in(a.scale, a.N, groups, type_bytes(a.scale_dtype));
    if (a.zero.data) o.in(a.zero, a.N, groups, 1);
    o.out(a.c, a.M, a.N, 2);
    if (!o.distinct()) return CCONV_EINVAL;
    if (!o.writes()) return CCONV_OK;
    const int sms = block_sm_count();
    if (sms < 0) return sms;
    o.workspace(a.workspace, a.workspace_bytes, int4_empty(a) ? 0 : int4_workspace(a, sms));
    if (!o.distinct()) return CCONV_EINVAL;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    return o.run(cuda_stream, sms, [&] {
      return int4_empty(a) ? block_cuda_error(zero_out(a.c, a.M, a.N, 2, s), "cconv_int4_product") : run_int4(a, sms, s);
    });
  });
}

int cconv_quantize_groups(const cconv_quantize_groups_args* args, void* cuda_stream) {
  return guarded([&]() -> int {
    if (!args) return CCONV_EINVAL;
    const cconv_quantize_groups_args& a = *args;
    if (!length_ok(a.N) || !length_ok(a.K) || !type_ok(a.dtype) || !type_ok(a.scale_dtype) || !group_ok(a.group) ||
        a.reserved != 0 || double(a.N) * a.K >= 1e15)
      return CCONV_EINVAL;
    const int64_t groups = cdiv64(a.K, a.group);
    Operands o;
    o.in(a.w, a.N, a.K, type_bytes(a.dtype));
    o.out(a.q, a.N, cdiv64(a.K, 2), 1);
    o.out(a.scale, a.N, groups, type_bytes(a.scale_dtype));
    if (a.zero.data) o.out(a.zero, a.N, groups, 1);
    if (!o.distinct()) return CCONV_EINVAL;
    if (!o.writes()) return CCONV_OK;
    const int sms = block_sm_count();
    if (sms < 0) return sms;
    return o.run(cuda_stream, sms, [&] {
      return block_cuda_error(run_quantize_groups(a, static_cast<cudaStream_t>(cuda_stream)), "cconv_quantize_groups");
    });
  });
}

int64_t cconv_moe_workspace(const cconv_moe_args* args) {
  return guarded([&]() -> int64_t {
    if (!args || !moe_sizes_ok(*args)) return CCONV_EINVAL;
    const int sms = block_sm_count();
    if (sms < 0) return sms;
    return moe_runs(*args) ? moe_workspace(*args, sms) : 0;
  });
}

int cconv_moe_forward(const cconv_moe_args* args, void* cuda_stream) {
  return guarded([&]() -> int {
    if (!args || !moe_sizes_ok(*args)) return CCONV_EINVAL;
    const cconv_moe_args& a = *args;
    const bool routes = a.router.data != nullptr;
    // (a router that must choose among no experts, or from no channels, has nothing to choose by)
    if (routes && a.T && (a.E == 0 || a.D == 0)) return CCONV_EINVAL;
    Operands o;
    o.in(a.x, a.T, a.D, 2);
    if (routes) o.in(a.router, a.E, a.D, 2);
    if (!moe_empty(a)) {
      int64_t n[3];
      if (!experts_ok(a.w_gate, a.gate_stride, a.F, a.D, a.E, &n[0]) || !experts_ok(a.w_up, a.up_stride, a.F, a.D, a.E, &n[1]) ||
          !experts_ok(a.w_down, a.down_stride, a.D, a.F, a.E, &n[2]))
        return CCONV_EINVAL;
      o.in(a.w_gate.data, n[0], 2);
      o.in(a.w_up.data, n[1], 2);
      o.in(a.w_down.data, n[2], 2);
    }
    if (routes) {
      o.out(a.ids, a.T, a.top_k, 4);
      o.out(a.weights, a.T, a.top_k, 4);
    } else {
      o.in(a.ids, a.T, a.top_k, 4);
      o.in(a.weights, a.T, a.top_k, 4);
    }
    o.out(a.out, a.T, a.D, 2);
    if (!o.distinct()) return CCONV_EINVAL;
    if (!o.writes()) return CCONV_OK;
    const int sms = block_sm_count();
    if (sms < 0) return sms;
    o.workspace(a.workspace, a.workspace_bytes, moe_runs(a) ? moe_workspace(a, sms) : 0);
    if (!o.distinct()) return CCONV_EINVAL;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    return o.run(cuda_stream, sms, [&]() -> int {
      if (moe_runs(a)) {
        const int rc = run_moe(a, sms, s);
        if (rc != CCONV_OK) return rc;
      }
      if (moe_empty(a)) BLOCK_CUDA(zero_out(a.out, a.T, a.D, 2, s));
      return CCONV_OK;
    });
  });
}

int64_t cconv_clip_workspace(const cconv_clip_args* args) {
  return guarded([&]() -> int64_t {
    if (!args || !clip_sizes_ok(*args, false)) return CCONV_EINVAL;
    const int sms = block_sm_count();
    if (sms < 0) return sms;
    return clip_workspace(*args, sms);
  });
}

int cconv_gradient_norm(const cconv_clip_args* args, void* cuda_stream) {
  return guarded([&]() -> int { return args ? clip_call(*args, false, cuda_stream) : CCONV_EINVAL; });
}

int cconv_clip_gradients(const cconv_clip_args* args, void* cuda_stream) {
  return guarded([&]() -> int { return args ? clip_call(*args, true, cuda_stream) : CCONV_EINVAL; });
}

int cconv_block_status(void* cuda_stream, int* detail_out) {
  return guarded([&]() -> int {
    if (detail_out) *detail_out = 0;
    const int sms = block_sm_count();
    if (sms < 0) return sms;
    int* word = nullptr;
    const int rc = block_status_word(&word);
    if (rc != CCONV_OK) return rc;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    int bits = 0;
    BLOCK_CUDA(cudaMemcpyAsync(&bits, word, sizeof bits, cudaMemcpyDeviceToHost, s));
    BLOCK_CUDA(cudaStreamSynchronize(s));
    if (bits == 0) return CCONV_OK;
    if (detail_out) *detail_out = bits;
    BLOCK_CUDA(cudaMemsetAsync(word, 0, sizeof bits, s));
    BLOCK_CUDA(cudaStreamSynchronize(s));
    return CCONV_EDEVICE_TIMEOUT;
  });
}

}  // extern "C"
