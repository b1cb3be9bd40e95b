// Entry points of the feed-forward sub-block (include/cconv_block.h): checks of arguments, workspace
// layout, launches.  Nothing here allocates or synchronises (cconv_block_status synchronises).
#include <cmath>
#include <cstring>
#include <numeric>
#include <string>

#include "block.h"
#include "block_ffn.h"
#include "block_fp8.h"
#include "block_gemm.h"
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
    if (!m.data || (reinterpret_cast<uintptr_t>(m.data) & uintptr_t(es - 1)) || m.row_stride < 0 || m.col_stride < 0 ||
        m.row_stride > kMaxStride || m.col_stride > kMaxStride) {
      ok = false;
      return -1;
    }
    const double last = double(rows - 1) * double(m.row_stride) + double(cols - 1) * double(m.col_stride);
    if (last > 4.0e18 / es) {
      ok = false;
      return -1;
    }
    if (written) {
      // distinct elements: one stride steps over the whole extent of the other
      const int64_t r = m.row_stride, c = m.col_stride;
      const bool rows_outer = (rows == 1 || r > (cols - 1) * c) && (cols == 1 || c > 0);
      const bool cols_outer = (cols == 1 || c > (rows - 1) * r) && (rows == 1 || r > 0);
      if (!rows_outer && !cols_outer) ok = false;
    }
    const char* lo = static_cast<const char*>(m.data);
    Bytes b{lo, lo + ((rows - 1) * m.row_stride + (cols - 1) * m.col_stride + 1) * es, 0, 0, es,
            std::gcd(rows > 1 ? m.row_stride * es : 0, cols > 1 ? m.col_stride * es : 0)};
    const int64_t wr = ((cols - 1) * m.col_stride + 1) * es, wc = ((rows - 1) * m.row_stride + 1) * es;
    if (rows > 1 && m.row_stride * es >= wr) b.pitch = m.row_stride * es, b.width = wr;
    else if (cols > 1 && m.col_stride * es >= wc) b.pitch = m.col_stride * es, b.width = wc;
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

bool fp8_sizes_ok(const cconv_fp8_product_args& a) {
  return length_ok(a.M) && length_ok(a.N) && length_ok(a.K) && a.dtype >= CCONV_TYPE_BF16 &&
         a.dtype <= CCONV_TYPE_FP32 && a.reserved == 0 && double(a.M) * a.N < 1e15 && double(a.M) * a.K < 1e15 &&
         double(a.N) * a.K < 1e15;
}

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
  return guarded([&]() -> int {
    if (!args || !norm_sizes_ok(*args)) return CCONV_EINVAL;
    cconv_residual_norm_args a = *args;
    const int es = type_bytes(a.dtype);
    a.resid = same_row(a.resid, a.T, a.D);
    a.block = same_row(a.block, a.T, a.D);
    a.gate = same_row(a.gate, gate_rows(a), a.D);
    a.resid_out = same_row(a.resid_out, a.T, a.D);
    a.norm_out = same_row(a.norm_out, a.T, a.D);
    if (!unit(a.resid, a.D) || !unit(a.block, a.D) || !unit(a.gate, a.D) || !unit(a.resid_out, a.D) || !unit(a.norm_out, a.D))
      return CCONV_EINVAL;
    if (a.T && a.D && ((!a.block.data && (a.gate.data || a.w_post)) || (!a.norm_out.data && a.w_pre))) return CCONV_EINVAL;
    Operands o;
    const int resid = o.in(a.resid, a.T, a.D, es);
    if (a.block.data) o.in(a.block, a.T, a.D, es);
    if (a.gate.data) o.in(a.gate, gate_rows(a), a.D, es);
    if (a.w_post) o.in(a.w_post, a.D, es);
    if (a.w_pre) o.in(a.w_pre, a.D, es);
    o.may_be_one(resid, o.out(a.resid_out, a.T, a.D, es));
    if (a.norm_out.data) o.out(a.norm_out, a.T, a.D, es);
    if (!o.distinct()) return CCONV_EINVAL;
    if (!o.writes()) return CCONV_OK;
    const int sms = block_sm_count();
    if (sms < 0) return sms;
    NormParams p = norm_params(a);
    const int rc = block_status_word(&p.status);
    if (rc != CCONV_OK) return rc;
    p.limit_ns = block_wait_limit_ns();
    return o.run(cuda_stream, sms, [&] {
      return block_cuda_error(run_norm_forward(p, a.dtype, sms, static_cast<cudaStream_t>(cuda_stream)),
                              "cconv_residual_norm_forward");
    });
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
