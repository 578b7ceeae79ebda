// C ABI of liboz2 (see include/oz2.h): argument checks, workspace bookkeeping, stage sequencing.
#include <mutex>
#include <new>

#include "../../include/oz2.h"
#include "oz2_bound.h"
#include "oz2_internal.h"
#include "oz2_kv4.h"
#include "oz2_route.h"
#include "oz2_w4.h"

namespace {

struct State {
  std::mutex mu;
  char* ws = nullptr;
  size_t ws_bytes = 0;
  int64_t kblock = 65536;
  int shift_mode = 0;
  int nonfinite_check = 1;
  int bit_split = 0;
  int product_format = OZ2_PRODUCT_RESIDUE_U8;
  int gemm_algorithm = OZ2_GEMM_AUTO;
  hipEvent_t ev[4] = {nullptr, nullptr, nullptr, nullptr};
  bool ev_on = false;
  Oz2Plan plan;
  int plan_N = 0;
  int64_t plan_k = -1;
  int plan_rc = 0;
};

// The context the calling thread works on: the process-wide default one, or, inside an oz2_context_* call, the
// caller's.  Every entry point below reaches its settings, workspace and plan cache through state().
thread_local State* tl_state = nullptr;
State& state() {
  static State s;
  return tl_state ? *tl_state : s;
}
struct UseContext {
  State* prev;
  explicit UseContext(oz2_context* ctx) : prev(tl_state) { tl_state = reinterpret_cast<State*>(ctx); }
  ~UseContext() { tl_state = prev; }
};

// cached plan for (N, k); caller holds the mutex
int get_plan(State& s, int N, int64_t k, const Oz2Plan** out) {
  if (s.plan_N != N || s.plan_k != k) {
    s.plan_rc = oz2_build_plan(N, k, &s.plan);
    s.plan_N = N;
    s.plan_k = k;
  }
  *out = &s.plan;
  return s.plan_rc;
}

// One-time device set-up of the GEMM kernels, made before any launch under a lock of its own: contexts have
// separate locks, so two of them may reach their first launch together.
std::mutex g_setup_mu;
bool g_setup_done = false;
bool ensure_setup() {
  std::lock_guard<std::mutex> lock(g_setup_mu);
  if (!g_setup_done)
    g_setup_done = oz2_gemm_setup() == hipSuccess && oz2_gemm_tiles_setup() == hipSuccess && oz2_stage1_setup() == hipSuccess &&
                   oz2_thin_setup() == hipSuccess;
  return g_setup_done;
}

bool n_ok(int N) { return N >= OZ2_MIN_N && N <= OZ2_MAX_N; }

// grid dimension limits of the kernels
bool dims_ok(int64_t m, int64_t n, int64_t k) {
  const int64_t lim = (int64_t)1 << 31;
  if (m >= lim - 512 || n >= lim - 512 || k >= lim - 512) return false;
  if ((k + 63) / 64 > 65535) return false;  // second grid dimension of the row-wise kernels
  if ((m + 511) / 512 > 65535) return false;
  return true;
}

// A workspace a call runs in: the registered one, or the library's own static buffer.
struct WsRef {
  char* p;
  size_t bytes;
};

int prepare(State& s, const WsRef& w, int64_t m, int64_t n, int64_t k, int N, const Oz2Plan** plan, Oz2Layout* lay) {
  int rc = get_plan(s, N, k, plan);
  if (rc == 2 && (s.shift_mode == OZ2_SHIFT_MAX || (*plan)->beta < 1)) return OZ2_ERR_BUDGET;
  if (rc == 2) rc = 0;
  if (rc != 0) return -10;
  // unequal budgets must leave at least one bit and at most 110 on each side
  if (s.bit_split != 0) {
    const Oz2Plan& p = **plan;
    int a, b;
    if (s.shift_mode == OZ2_SHIFT_MAX) { a = p.kappa - s.bit_split; b = p.kappa_sum - a; }
    else if (s.shift_mode == OZ2_SHIFT_CAUCHY_SCHWARZ) { a = p.beta - s.bit_split; b = p.budget2 - a; }
    else { a = p.budget2 / 2 - s.bit_split; b = p.budget2 / 2 + s.bit_split; }
    if (a < 1 || b < 1 || a > 110 || b > 110) return OZ2_ERR_BUDGET;
  }
  // the INT8 product of the 6-bit bounds must stay below 2^31
  if (s.shift_mode == OZ2_SHIFT_INT8_PRODUCT && (k + 63) / 64 * 64 >= ((int64_t)1 << 19)) return OZ2_ERR_BUDGET;
  oz2_make_layout(m, n, k, N, s.product_format == OZ2_PRODUCT_INT32 ? 4 : 1, lay);
  if (!w.p || w.bytes < lay->total) return OZ2_ERR_WORKSPACE;
  return ensure_setup() ? OZ2_OK : OZ2_ERR_HIP;
}

int prepare(State& s, int64_t m, int64_t n, int64_t k, int N, const Oz2Plan** plan, Oz2Layout* lay) {
  return prepare(s, WsRef{s.ws, s.ws_bytes}, m, n, k, N, plan, lay);
}

// The Strassen form pays when the matrix-core work it saves (an eighth of 2 m n k N) outweighs the extra plane
// traffic of its conversion and CRT passes (three quarters more bytes per plane) and the lower rate of products
// with a short inner dimension.  Measured on MI355X with 16 moduli, Strassen against classical form on one box, whole
// calls: -3 % at 8192^3 and at 6144 x 6144 x 16384, even at 8192 x 8192 x 10240 and x 12288 and at 10240^3, +1 % at
// 8192 x 8192 x 16384, +3 % at 12288 x 12288 x 10240, +4 % at 14336^3, +6 % at 16384^3.
bool strassen_pays(int64_t m, int64_t n, int64_t k) { return m >= 8192 && n >= 8192 && k >= 10240; }

// Does a general product of this shape use the Strassen form under the current settings?  It needs UINT8 residue
// planes and, in the INT8-product shift mode, a padded inner dimension below 2^19.  On a yes, *lay is its layout.
bool strassen_applies(const State& s, int64_t m, int64_t n, int64_t k, int N, Oz2Layout* lay) {
  if (s.gemm_algorithm == OZ2_GEMM_CLASSICAL || s.product_format != OZ2_PRODUCT_RESIDUE_U8) return false;
  if (s.gemm_algorithm == OZ2_GEMM_AUTO && !strassen_pays(m, n, k)) return false;
  oz2_make_layout_strassen(m, n, k, N, lay);
  if (s.shift_mode == OZ2_SHIFT_INT8_PRODUCT && lay->k_pad >= ((int64_t)1 << 19)) return false;
  return true;
}

// prepare() for the general product: *strassen tells which form the call takes.  The automatic choice falls back to
// the plain form when the workspace only suffices for that; a forced Strassen form reports the workspace as too small.
int prepare_general(State& s, const WsRef& w, int64_t m, int64_t n, int64_t k, int N, const Oz2Plan** plan, Oz2Layout* lay,
                    bool* strassen) {
  *strassen = false;
  Oz2Layout plain;
  const int rc = prepare(s, w, m, n, k, N, plan, &plain);
  if (rc != OZ2_OK && rc != OZ2_ERR_WORKSPACE) return rc;
  Oz2Layout sl;
  if (strassen_applies(s, m, n, k, N, &sl)) {
    if (w.p && w.bytes >= sl.total) {
      *lay = sl;
      *strassen = true;
      return ensure_setup() ? OZ2_OK : OZ2_ERR_HIP;
    }
    if (s.gemm_algorithm == OZ2_GEMM_STRASSEN) return OZ2_ERR_WORKSPACE;
  }
  *lay = plain;
  return rc;
}

}  // namespace

extern "C" {

int oz2_init(void) {
  State& s = state();
  std::lock_guard<std::mutex> lock(s.mu);
  if (!ensure_setup()) return OZ2_ERR_HIP;
  char* p;
  size_t bytes;
  return oz2_static_scratch(&p, &bytes) == hipSuccess ? OZ2_OK : OZ2_ERR_HIP;
}

int oz2_min_moduli(void) { return OZ2_MIN_N; }
int oz2_max_moduli(void) { return OZ2_MAX_N; }

int oz2_get_moduli(int num_moduli, int* moduli_out, int* kappa_out, int64_t k) {
  if (!n_ok(num_moduli)) return -1;
  if (k < 1) return -4;
  if (moduli_out) oz2_table_moduli(num_moduli, moduli_out);
  if (kappa_out) *kappa_out = oz2_table_kappa(num_moduli, k);
  return OZ2_OK;
}

int oz2_moduli_for_bits(int64_t k, int bits) {
  if (k < 1) return -1;
  if (bits < 1) return -2;
  for (int N = OZ2_MIN_N; N <= OZ2_MAX_N; ++N)
    if (oz2_table_kappa(N, k) >= bits) return N;
  return 0;
}

size_t oz2_workspace_bytes_for(int64_t m, int64_t n, int64_t k, int num_moduli, int product_format) {
  if (m < 0 || n < 0 || k < 0 || !n_ok(num_moduli) || !dims_ok(m, n, k)) return 0;
  if (product_format != OZ2_PRODUCT_INT32 && product_format != OZ2_PRODUCT_RESIDUE_U8) return 0;
  Oz2Layout lay;
  oz2_make_layout(m, n, k, num_moduli, product_format == OZ2_PRODUCT_INT32 ? 4 : 1, &lay);
  return lay.total;
}

size_t oz2_workspace_bytes(int64_t m, int64_t n, int64_t k, int num_moduli) {
  return oz2_workspace_bytes_for(m, n, k, num_moduli, OZ2_PRODUCT_INT32);
}

size_t oz2_workspace_bytes_strassen(int64_t m, int64_t n, int64_t k, int num_moduli) {
  if (m < 0 || n < 0 || k < 0 || !n_ok(num_moduli) || !dims_ok(m, n, k)) return 0;
  Oz2Layout lay;
  oz2_make_layout_strassen(m, n, k, num_moduli, &lay);
  return lay.total;
}

size_t oz2_workspace_bytes_preferred(int64_t m, int64_t n, int64_t k, int num_moduli) {
  if (m < 0 || n < 0 || k < 0 || !n_ok(num_moduli) || !dims_ok(m, n, k)) return 0;
  State& s = state();
  std::lock_guard<std::mutex> lock(s.mu);
  Oz2Layout lay;
  if (m > 0 && n > 0 && k > 0 && strassen_applies(s, m, n, k, num_moduli, &lay)) return lay.total;
  oz2_make_layout(m, n, k, num_moduli, s.product_format == OZ2_PRODUCT_INT32 ? 4 : 1, &lay);
  return lay.total;
}

int oz2_set_gemm_algorithm(int algorithm) {
  if (algorithm != OZ2_GEMM_AUTO && algorithm != OZ2_GEMM_CLASSICAL && algorithm != OZ2_GEMM_STRASSEN) return -1;
  State& s = state();
  std::lock_guard<std::mutex> lock(s.mu);
  s.gemm_algorithm = algorithm;
  return OZ2_OK;
}

int oz2_gemm_algorithm_for(int64_t m, int64_t n, int64_t k, int num_moduli) {
  if (m < 0) return -1;
  if (n < 0) return -2;
  if (k < 0) return -3;
  if (!n_ok(num_moduli)) return -4;
  if (!dims_ok(m, n, k)) return -1;
  State& s = state();
  std::lock_guard<std::mutex> lock(s.mu);
  Oz2Layout sl;
  if (m == 0 || n == 0 || k == 0 || !strassen_applies(s, m, n, k, num_moduli, &sl)) return OZ2_GEMM_CLASSICAL;
  if (s.gemm_algorithm == OZ2_GEMM_AUTO && !(s.ws && s.ws_bytes >= sl.total)) return OZ2_GEMM_CLASSICAL;
  return OZ2_GEMM_STRASSEN;
}

int oz2_set_workspace(void* dev_ptr, size_t bytes) {
  State& s = state();
  std::lock_guard<std::mutex> lock(s.mu);
  if ((!dev_ptr && bytes) || (reinterpret_cast<uintptr_t>(dev_ptr) & 255u)) return -1;
  s.ws = static_cast<char*>(dev_ptr);
  s.ws_bytes = dev_ptr ? bytes : 0;
  return OZ2_OK;
}

int oz2_workspace_layout(int64_t m, int64_t n, int64_t k, int num_moduli, size_t offsets[10], int64_t dims[3]) {
  if (m < 0) return -1;
  if (n < 0) return -2;
  if (k < 0) return -3;
  if (!n_ok(num_moduli)) return -4;
  if (!dims_ok(m, n, k)) return -1;
  if (!offsets) return -5;
  if (!dims) return -6;
  Oz2Layout lay;
  {
    State& s = state();
    std::lock_guard<std::mutex> lock(s.mu);
    oz2_make_layout(m, n, k, num_moduli, s.product_format == OZ2_PRODUCT_INT32 ? 4 : 1, &lay);
  }
  offsets[0] = lay.off_rowmax;
  offsets[1] = lay.off_colmax;
  offsets[2] = lay.off_sa;
  offsets[3] = lay.off_sb;
  offsets[4] = lay.off_a;
  offsets[5] = lay.off_b;
  offsets[6] = lay.off_c;
  offsets[7] = lay.off_rownorm;
  offsets[8] = lay.off_colnorm;
  offsets[9] = lay.off_flags;
  dims[0] = lay.m_pad;
  dims[1] = lay.n_pad;
  dims[2] = lay.k_pad;
  return OZ2_OK;
}

int oz2_set_stage_events(void* const events[4]) {
  State& s = state();
  std::lock_guard<std::mutex> lock(s.mu);
  s.ev_on = events != nullptr;
  for (int i = 0; i < 4; ++i) s.ev[i] = events ? static_cast<hipEvent_t>(events[i]) : nullptr;
  return OZ2_OK;
}

int oz2_set_shift_mode(int mode) {
  if (mode != OZ2_SHIFT_MAX && mode != OZ2_SHIFT_CAUCHY_SCHWARZ && mode != OZ2_SHIFT_INT8_PRODUCT) return -1;
  State& s = state();
  std::lock_guard<std::mutex> lock(s.mu);
  s.shift_mode = mode;
  return OZ2_OK;
}

int oz2_set_nonfinite_check(int on) {
  if (on != 0 && on != 1) return -1;
  State& s = state();
  std::lock_guard<std::mutex> lock(s.mu);
  s.nonfinite_check = on;
  return OZ2_OK;
}

int oz2_set_bit_split(int delta) {
  if (delta < -100 || delta > 100) return -1;
  State& s = state();
  std::lock_guard<std::mutex> lock(s.mu);
  s.bit_split = delta;
  return OZ2_OK;
}

int oz2_set_product_format(int format) {
  if (format != OZ2_PRODUCT_INT32 && format != OZ2_PRODUCT_RESIDUE_U8) return -1;
  State& s = state();
  std::lock_guard<std::mutex> lock(s.mu);
  s.product_format = format;
  return OZ2_OK;
}

int oz2_set_round_sync(int spins) {
  if (spins < 0 || spins > (1 << 20)) return -1;
  State& s = state();
  std::lock_guard<std::mutex> lock(s.mu);
  oz2_gemm_set_sync_spins(spins);
  return OZ2_OK;
}

int oz2_set_kblock(int64_t kblock) {
  if (kblock < OZ2_TILE_K || kblock > 65536 || kblock % OZ2_TILE_K) return -1;
  State& s = state();
  std::lock_guard<std::mutex> lock(s.mu);
  s.kblock = kblock;
  return OZ2_OK;
}

int oz2_stage1_convert(int64_t m, int64_t n, int64_t k, const double* A, int64_t lda, const double* B, int64_t ldb,
                       int num_moduli, void* stream) {
  if (m < 0) return -1;
  if (n < 0) return -2;
  if (k < 0) return -3;
  if (!dims_ok(m, n, k)) return -1;
  if (lda < (m > 1 ? m : 1)) return -5;
  if (ldb < (k > 1 ? k : 1)) return -7;
  if (!n_ok(num_moduli)) return -8;
  if (m == 0 || n == 0 || k == 0) return OZ2_OK;
  if (!A) return -4;
  if (!B) return -6;
  State& s = state();
  std::lock_guard<std::mutex> lock(s.mu);
  const Oz2Plan* plan;
  Oz2Layout lay;
  int rc = prepare(s, m, n, k, num_moduli, &plan, &lay);
  if (rc) return rc;
  hipError_t e = oz2_launch_stage1(0, 0, m, n, k, A, lda, B, ldb, 0, 0, *plan, s.shift_mode, s.bit_split, 0, lay, s.ws,
                                   static_cast<hipStream_t>(stream), 0, nullptr, nullptr);
  return e == hipSuccess ? OZ2_OK : OZ2_ERR_HIP;
}

int oz2_stage2_gemm(int64_t m, int64_t n, int64_t k, int num_moduli, void* stream) {
  if (m < 0) return -1;
  if (n < 0) return -2;
  if (k < 0) return -3;
  if (!dims_ok(m, n, k)) return -1;
  if (!n_ok(num_moduli)) return -4;
  if (m == 0 || n == 0 || k == 0) return OZ2_OK;
  State& s = state();
  std::lock_guard<std::mutex> lock(s.mu);
  const Oz2Plan* plan;
  Oz2Layout lay;
  int rc = prepare(s, m, n, k, num_moduli, &plan, &lay);
  if (rc) return rc;
  // the counters of the round synchronisation must be zero at launch; in oz2_dgemm stage 1 has cleared them
  hipError_t e = oz2_launch_clear_sync(lay, s.ws, static_cast<hipStream_t>(stream));
  if (e == hipSuccess)
    e = oz2_launch_products(*plan, lay, s.ws, m, n, s.kblock, s.product_format, 0, OZ2_KRANGE_ALL, 0, Oz2ScanFinish{nullptr, 0u, nullptr, 0},
                          static_cast<hipStream_t>(stream));
  return e == hipSuccess ? OZ2_OK : OZ2_ERR_HIP;
}

int oz2_stage3_crt(int64_t m, int64_t n, int64_t k, double* C, int64_t ldc, int num_moduli, void* stream) {
  if (m < 0) return -1;
  if (n < 0) return -2;
  if (k < 0) return -3;
  if (!dims_ok(m, n, k)) return -1;
  if (ldc < (m > 1 ? m : 1)) return -5;
  if (!n_ok(num_moduli)) return -6;
  if (m == 0 || n == 0) return OZ2_OK;
  if (!C) return -4;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (k == 0) return oz2_launch_scale_c(m, n, 0.0, C, ldc, 0, st) == hipSuccess ? OZ2_OK : OZ2_ERR_HIP;
  State& s = state();
  std::lock_guard<std::mutex> lock(s.mu);
  const Oz2Plan* plan;
  Oz2Layout lay;
  int rc = prepare(s, m, n, k, num_moduli, &plan, &lay);
  if (rc) return rc;
  hipError_t e = oz2_launch_stage3(m, n, 1.0, 0.0, C, ldc, *plan, lay, s.ws, s.product_format, 0, 0, st);
  return e == hipSuccess ? OZ2_OK : OZ2_ERR_HIP;
}

namespace {
int trans_code(char c) {
  switch (c) {
    case 'N': case 'n': return 0;
    case 'T': case 't': case 'C': case 'c': return 1;
    default: return -1;
  }
}
}  // namespace

namespace {
// Below 2^24 elements of C the blocks of the fallback ride in the launch of stage 3 (above, its registers cost more than the launch: 10
// moduli 4096 x 4096 x 300 164 us, apart 155): one launch less (whole calls, us: 2200 x 2200 x 500 103 -> 98, 3000 x 3000 x 1000 224 -> 220, 18
// moduli 3001 x 2777 x 3500 674 -> 667), and with its smaller tiles the fallback itself is the faster one (1024^3 612 -> 277, 4000^3 7770 -> 5430).
bool fallback_in_stage3(const State& s, int64_t m, int64_t n) {
  return s.nonfinite_check && s.product_format == OZ2_PRODUCT_RESIDUE_U8 && m * n < ((int64_t)1 << 24);
}

// The general product on the registered workspace (static_ws == false) or on the library's static buffer.
int dgemm_ex_impl(bool static_ws, char transa, char transb, int64_t m, int64_t n, int64_t k, double alpha, const double* A,
                  int64_t lda, const double* B, int64_t ldb, double beta, double* C, int64_t ldc, int num_moduli,
                  void* stream) {
  const int ta = trans_code(transa), tb = trans_code(transb);
  if (ta < 0) return -1;
  if (tb < 0) return -2;
  if (m < 0) return -3;
  if (n < 0) return -4;
  if (k < 0) return -5;
  if (!dims_ok(m, n, k)) return -3;
  const int64_t rows_a = ta ? k : m, rows_b = tb ? n : k;
  if (lda < (rows_a > 1 ? rows_a : 1)) return -8;
  if (ldb < (rows_b > 1 ? rows_b : 1)) return -10;
  if (ldc < (m > 1 ? m : 1)) return -13;
  if (!n_ok(num_moduli)) return -14;
  if (m == 0 || n == 0) return OZ2_OK;
  if (!C) return -12;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (k == 0 || alpha == 0.0) {
    if (beta == 1.0) return OZ2_OK;
    return oz2_launch_scale_c(m, n, beta, C, ldc, 0, st) == hipSuccess ? OZ2_OK : OZ2_ERR_HIP;
  }
  if (!A) return -7;
  if (!B) return -9;
  State& s = state();
  std::lock_guard<std::mutex> lock(s.mu);
  WsRef w{s.ws, s.ws_bytes};
  if (static_ws) {
    // the static buffer of the current device; its address is looked up once per device, nothing is allocated
    if (oz2_static_scratch(&w.p, &w.bytes) != hipSuccess) return OZ2_ERR_HIP;
  }
  const Oz2Plan* plan;
  Oz2Layout lay;
  bool strassen;
  int rc = prepare_general(s, w, m, n, k, num_moduli, &plan, &lay, &strassen);
  if (rc == OZ2_ERR_WORKSPACE && static_ws) return OZ2_ERR_STATIC_LIMIT;
  if (rc) return rc;
  char* const ws = w.p;
  auto mark = [&](int i) { return !s.ev_on || hipEventRecord(s.ev[i], st) == hipSuccess; };
  Oz2ScanFinish fin;
  const int thin =
      !strassen && s.product_format == OZ2_PRODUCT_RESIDUE_U8 ? oz2_thin_applies(m, n, *plan, lay, s.kblock, oz2_gemm_cus()) : 0;
  int two_level = 0;
  if (!mark(0)) return OZ2_ERR_HIP;
  if (oz2_launch_stage1(ta, tb, m, n, k, A, lda, B, ldb, 0, 0, *plan, s.shift_mode, s.bit_split, strassen ? 1 : 0, lay, ws,
                        st, thin, &two_level, &fin) != hipSuccess ||
      !mark(1))
    return OZ2_ERR_HIP;
  if (strassen) {
    if (oz2_launch_strassen_gemm(*plan, lay, ws, s.kblock, s.nonfinite_check, st) != hipSuccess || !mark(2))
      return OZ2_ERR_HIP;
    if (oz2_launch_strassen_crt(m, n, alpha, beta, C, ldc, *plan, lay, ws, s.nonfinite_check, st) != hipSuccess || !mark(3))
      return OZ2_ERR_HIP;
  } else {
    const hipError_t e =
        thin == 1 ? oz2_launch_thin_products(1, ta == 0, A, lda, m, n, k, two_level, *plan, lay, ws, s.nonfinite_check, st)
        : thin == 2 ? oz2_launch_thin_products(2, tb != 0, B, ldb, n, m, k, two_level, *plan, lay, ws, s.nonfinite_check, st)
                    : oz2_launch_products(*plan, lay, ws, m, n, s.kblock, s.product_format, 0, OZ2_KRANGE_ALL,
                                          s.nonfinite_check, fin, st);
    if (e != hipSuccess || !mark(2)) return OZ2_ERR_HIP;
    if (fallback_in_stage3(s, m, n)) {
      if (oz2_launch_stage3_or_fallback(ta, tb, m, n, k, alpha, A, lda, B, ldb, beta, C, ldc, *plan, lay, ws, st) !=
              hipSuccess ||
          !mark(3))
        return OZ2_ERR_HIP;
      return OZ2_OK;
    }
    if (oz2_launch_stage3(m, n, alpha, beta, C, ldc, *plan, lay, ws, s.product_format, s.nonfinite_check, 0, st) !=
            hipSuccess ||
        !mark(3))
      return OZ2_ERR_HIP;
  }
  if (s.nonfinite_check &&
      oz2_launch_fallback(reinterpret_cast<const unsigned long long*>(ws + lay.off_flags), ta, tb, m, n, k, alpha, A, lda,
                          B, ldb, beta, C, ldc, 0, 0, 0, st) != hipSuccess)
    return OZ2_ERR_HIP;
  return OZ2_OK;
}

// same argument numbering as oz2_dgemm's declaration: map the codes of the general form
int dgemm_code(int rc) {
  switch (rc) {
    case -3: return -1;
    case -4: return -2;
    case -5: return -3;
    case -7: return -4;
    case -8: return -5;
    case -9: return -6;
    case -10: return -7;
    case -12: return -8;
    case -13: return -9;
    case -14: return -10;
    default: return rc;
  }
}
}  // namespace

int oz2_dgemm_ex(char transa, char transb, int64_t m, int64_t n, int64_t k, double alpha, const double* A, int64_t lda,
                 const double* B, int64_t ldb, double beta, double* C, int64_t ldc, int num_moduli, void* stream) {
  return dgemm_ex_impl(false, transa, transb, m, n, k, alpha, A, lda, B, ldb, beta, C, ldc, num_moduli, stream);
}

int oz2_dsyrk(char uplo, char trans, int64_t n, int64_t k, double alpha, const double* A, int64_t lda, double beta,
              double* C, int64_t ldc, int num_moduli, void* stream) {
  const int tri = (uplo == 'L' || uplo == 'l') ? 1 : (uplo == 'U' || uplo == 'u') ? 2 : 0;
  const int ta = trans_code(trans);
  if (tri == 0) return -1;
  if (ta < 0) return -2;
  if (n < 0) return -3;
  if (k < 0) return -4;
  if (!dims_ok(n, n, k)) return -3;
  const int64_t rows_a = ta ? k : n;
  if (lda < (rows_a > 1 ? rows_a : 1)) return -7;
  if (ldc < (n > 1 ? n : 1)) return -10;
  if (!n_ok(num_moduli)) return -11;
  if (n == 0) return OZ2_OK;
  if (!C) return -9;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (k == 0 || alpha == 0.0) {
    if (beta == 1.0) return OZ2_OK;
    return oz2_launch_scale_c(n, n, beta, C, ldc, tri, st) == hipSuccess ? OZ2_OK : OZ2_ERR_HIP;
  }
  if (!A) return -6;
  State& s = state();
  std::lock_guard<std::mutex> lock(s.mu);
  const Oz2Plan* plan;
  Oz2Layout lay;
  int rc = prepare(s, n, n, k, num_moduli, &plan, &lay);
  if (rc) return rc;
  auto mark = [&](int i) { return !s.ev_on || hipEventRecord(s.ev[i], st) == hipSuccess; };
  Oz2ScanFinish fin;
  if (!mark(0)) return OZ2_ERR_HIP;
  // op(A) op(A)^T: the columns of the second operand are the rows of the first, so A is converted once and
  // its planes serve as both operands
  if (oz2_launch_stage1(ta, 0, n, n, k, A, lda, nullptr, 0, 0, 0, *plan, s.shift_mode, 0, 0, lay, s.ws, st, 0, nullptr, &fin) != hipSuccess ||
      !mark(1))
    return OZ2_ERR_HIP;
  if (oz2_launch_products(*plan, lay, s.ws, n, n, s.kblock, s.product_format, tri, OZ2_KRANGE_ALL, s.nonfinite_check, fin, st) != hipSuccess ||
      !mark(2))
    return OZ2_ERR_HIP;
  if (oz2_launch_stage3(n, n, alpha, beta, C, ldc, *plan, lay, s.ws, s.product_format, s.nonfinite_check, tri, st) !=
          hipSuccess ||
      !mark(3))
    return OZ2_ERR_HIP;
  // fallback: op(B) = op(A)^T is A read with the other orientation
  if (s.nonfinite_check &&
      oz2_launch_fallback(reinterpret_cast<const unsigned long long*>(s.ws + lay.off_flags), ta, !ta, n, n, k, alpha, A, lda,
                          A, lda, beta, C, ldc, tri, 0, 0, st) != hipSuccess)
    return OZ2_ERR_HIP;
  return OZ2_OK;
}

int oz2_dtrmm(char side, char uplo, char transa, char diag, int64_t m, int64_t n, double alpha, const double* A,
              int64_t lda, double* B, int64_t ldb, int num_moduli, void* stream) {
  const int left = (side == 'L' || side == 'l') ? 1 : (side == 'R' || side == 'r') ? 0 : -1;
  const int lower = (uplo == 'L' || uplo == 'l') ? 1 : (uplo == 'U' || uplo == 'u') ? 0 : -1;
  const int ta = trans_code(transa);
  const int unit = (diag == 'U' || diag == 'u') ? 1 : (diag == 'N' || diag == 'n') ? 0 : -1;
  if (left < 0) return -1;
  if (lower < 0) return -2;
  if (ta < 0) return -3;
  if (unit < 0) return -4;
  if (m < 0) return -5;
  if (n < 0) return -6;
  const int64_t ka = left ? m : n;  // order of A = inner dimension of the product
  if (!dims_ok(m, n, ka)) return -5;
  if (lda < (ka > 1 ? ka : 1)) return -9;
  if (ldb < (m > 1 ? m : 1)) return -11;
  if (!n_ok(num_moduli)) return -12;
  if (m == 0 || n == 0) return OZ2_OK;
  if (!B) return -10;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (alpha == 0.0) return oz2_launch_scale_c(m, n, 0.0, B, ldb, 0, st) == hipSuccess ? OZ2_OK : OZ2_ERR_HIP;
  if (!A) return -8;
  State& s = state();
  std::lock_guard<std::mutex> lock(s.mu);
  const Oz2Plan* plan;
  Oz2Layout lay;
  int rc = prepare(s, m, n, ka, num_moduli, &plan, &lay);
  if (rc) return rc;
  const int tri = (lower ? 1 : 2) | (unit ? 4 : 0);    // structure of the stored A
  const bool op_lower = (lower != 0) != (ta != 0);     // structure of op(A)
  // the product X * Y with X = op(A), Y = B (left) or X = B, Y = op(A) (right)
  const double* X = left ? A : B;
  const double* Y = left ? B : A;
  const int64_t ldx = left ? lda : ldb, ldy = left ? ldb : lda;
  const int tx = left ? ta : 0, ty = left ? 0 : ta;
  const int trix = left ? tri : 0, triy = left ? 0 : tri;
  const int krange = left ? (op_lower ? OZ2_KRANGE_UPTO_ROW : OZ2_KRANGE_FROM_ROW)
                          : (op_lower ? OZ2_KRANGE_FROM_COL : OZ2_KRANGE_UPTO_COL);
  auto mark = [&](int i) { return !s.ev_on || hipEventRecord(s.ev[i], st) == hipSuccess; };
  Oz2ScanFinish fin;
  if (!mark(0)) return OZ2_ERR_HIP;
  if (oz2_launch_stage1(tx, ty, m, n, ka, X, ldx, Y, ldy, trix, triy, *plan, s.shift_mode, 0, 0, lay, s.ws, st, 0, nullptr, &fin) != hipSuccess ||
      !mark(1))
    return OZ2_ERR_HIP;
  if (oz2_launch_products(*plan, lay, s.ws, m, n, s.kblock, s.product_format, 0, krange, s.nonfinite_check, fin, st) != hipSuccess || !mark(2))
    return OZ2_ERR_HIP;
  // B is overwritten: stage 1 has read all of it by now (stream order)
  if (oz2_launch_stage3(m, n, alpha, 0.0, B, ldb, *plan, lay, s.ws, s.product_format, s.nonfinite_check, 0, st) !=
          hipSuccess ||
      !mark(3))
    return OZ2_ERR_HIP;
  if (s.nonfinite_check) {
    // the FP64 fallback cannot work in place: it forms the product in the (then unused) product region of the
    // workspace and a second conditional kernel copies it over B
    const unsigned long long* flag = reinterpret_cast<const unsigned long long*>(s.ws + lay.off_flags);
    double* tmp = reinterpret_cast<double*>(s.ws + lay.off_c);
    if (oz2_launch_fallback(flag, tx, ty, m, n, ka, alpha, X, ldx, Y, ldy, 0.0, tmp, m, 0, trix, triy, st) != hipSuccess ||
        oz2_launch_copy_if(flag, m, n, tmp, B, ldb, st) != hipSuccess)
      return OZ2_ERR_HIP;
  }
  return OZ2_OK;
}

int oz2_dgemm(int64_t m, int64_t n, int64_t k, const double* A, int64_t lda, const double* B, int64_t ldb, double* C,
              int64_t ldc, int num_moduli, void* stream) {
  return dgemm_code(dgemm_ex_impl(false, 'N', 'N', m, n, k, 1.0, A, lda, B, ldb, 0.0, C, ldc, num_moduli, stream));
}

int oz2_dgemm_static(int64_t m, int64_t n, int64_t k, const double* A, int64_t lda, const double* B, int64_t ldb, double* C,
                     int64_t ldc, int num_moduli, void* stream) {
  return dgemm_code(dgemm_ex_impl(true, 'N', 'N', m, n, k, 1.0, A, lda, B, ldb, 0.0, C, ldc, num_moduli, stream));
}

int oz2_context_create(oz2_context** ctx) {
  if (!ctx) return -1;
  State* s = new (std::nothrow) State();
  if (!s) return OZ2_ERR_HIP;
  *ctx = reinterpret_cast<oz2_context*>(s);
  return OZ2_OK;
}

int oz2_context_destroy(oz2_context* ctx) {
  if (!ctx) return -1;
  delete reinterpret_cast<State*>(ctx);
  return OZ2_OK;
}

int oz2_context_set_workspace(oz2_context* ctx, void* dev_ptr, size_t bytes) {
  UseContext use(ctx);
  return oz2_set_workspace(dev_ptr, bytes);
}

int oz2_context_set(oz2_context* ctx, int option, int64_t value) {
  UseContext use(ctx);
  const bool fits = value >= INT32_MIN && value <= INT32_MAX;
  int rc;
  switch (option) {
    case OZ2_OPT_SHIFT_MODE: rc = fits ? oz2_set_shift_mode((int)value) : -1; break;
    case OZ2_OPT_PRODUCT_FORMAT: rc = fits ? oz2_set_product_format((int)value) : -1; break;
    case OZ2_OPT_GEMM_ALGORITHM: rc = fits ? oz2_set_gemm_algorithm((int)value) : -1; break;
    case OZ2_OPT_KBLOCK: rc = oz2_set_kblock(value); break;
    case OZ2_OPT_BIT_SPLIT: rc = fits ? oz2_set_bit_split((int)value) : -1; break;
    case OZ2_OPT_NONFINITE_CHECK: rc = fits ? oz2_set_nonfinite_check((int)value) : -1; break;
    default: return -2;
  }
  return rc == OZ2_OK ? OZ2_OK : -3;
}

int oz2_context_get(oz2_context* ctx, int option, int64_t* value) {
  if (!value) return -3;
  UseContext use(ctx);
  State& s = state();
  std::lock_guard<std::mutex> lock(s.mu);
  switch (option) {
    case OZ2_OPT_SHIFT_MODE: *value = s.shift_mode; break;
    case OZ2_OPT_PRODUCT_FORMAT: *value = s.product_format; break;
    case OZ2_OPT_GEMM_ALGORITHM: *value = s.gemm_algorithm; break;
    case OZ2_OPT_KBLOCK: *value = s.kblock; break;
    case OZ2_OPT_BIT_SPLIT: *value = s.bit_split; break;
    case OZ2_OPT_NONFINITE_CHECK: *value = s.nonfinite_check; break;
    default: return -2;
  }
  return OZ2_OK;
}

size_t oz2_context_workspace_bytes(oz2_context* ctx, int64_t m, int64_t n, int64_t k, int num_moduli) {
  UseContext use(ctx);
  return oz2_workspace_bytes_preferred(m, n, k, num_moduli);
}

int oz2_context_dgemm(oz2_context* ctx, char transa, char transb, int64_t m, int64_t n, int64_t k, double alpha,
                      const double* A, int64_t lda, const double* B, int64_t ldb, double beta, double* C, int64_t ldc,
                      int num_moduli, void* stream) {
  UseContext use(ctx);
  const int rc = oz2_dgemm_ex(transa, transb, m, n, k, alpha, A, lda, B, ldb, beta, C, ldc, num_moduli, stream);
  return rc < 0 ? rc - 1 : rc;  // argument codes count the context as the first argument
}

int oz2_context_dsyrk(oz2_context* ctx, char uplo, char trans, int64_t n, int64_t k, double alpha, const double* A,
                      int64_t lda, double beta, double* C, int64_t ldc, int num_moduli, void* stream) {
  UseContext use(ctx);
  const int rc = oz2_dsyrk(uplo, trans, n, k, alpha, A, lda, beta, C, ldc, num_moduli, stream);
  return rc < 0 ? rc - 1 : rc;
}

int oz2_context_dtrmm(oz2_context* ctx, char side, char uplo, char transa, char diag, int64_t m, int64_t n, double alpha,
                      const double* A, int64_t lda, double* B, int64_t ldb, int num_moduli, void* stream) {
  UseContext use(ctx);
  const int rc = oz2_dtrmm(side, uplo, transa, diag, m, n, alpha, A, lda, B, ldb, num_moduli, stream);
  return rc < 0 ? rc - 1 : rc;
}

int oz2_calibrate_mfma(int workgroups, int iters, int random_operands, int* sink, long long* clocks, void* stream) {
  if (workgroups < 1 || workgroups > 65536) return -1;
  if (iters < 1) return -2;
  if (!sink) return -4;
  if (!clocks) return -5;
  hipError_t e = oz2_launch_mfma_calibration(workgroups, iters, random_operands, sink, clocks,
                                             static_cast<hipStream_t>(stream));
  return e == hipSuccess ? OZ2_OK : OZ2_ERR_HIP;
}

namespace {
// What the two hooks below need of a call: the arguments checked, the plan and the layout.
int host_call(State& s, int call, int64_t m, int64_t n, int64_t k, int num_moduli, int compute_units, const Oz2Plan** plan, Oz2Layout* lay) {
  if (call < 0 || call > 2) return -1;
  if (m < 1) return -2;
  if (n < 1 || (call == 1 && n != m)) return -3;
  if (k < 1 || (call == 2 && k != m && k != n)) return -4;
  if (!dims_ok(m, n, k)) return -2;
  if (!n_ok(num_moduli)) return -5;
  if (compute_units < 1) return -6;
  if (get_plan(s, num_moduli, k, plan) < 0) return -5;
  oz2_make_layout(m, n, k, num_moduli, s.product_format == OZ2_PRODUCT_RESIDUE_U8 ? 1 : 4, lay);
  return OZ2_OK;
}
}  // namespace

int oz2_host_kernel_choice(int call, int64_t m, int64_t n, int64_t k, int num_moduli, int compute_units, int choice[3]) {
  State& s = state();
  std::lock_guard<std::mutex> lock(s.mu);
  const Oz2Plan* plan;
  Oz2Layout lay;
  if (const int rc = host_call(s, call, m, n, k, num_moduli, compute_units, &plan, &lay); rc != OZ2_OK) return rc;
  if (!choice) return -7;
  const int u8 = s.product_format == OZ2_PRODUCT_RESIDUE_U8;
  const int krange = call == 2 ? OZ2_KRANGE_UPTO_ROW : OZ2_KRANGE_ALL;  // (the rules treat the four ranges alike)
  choice[1] = u8 && call == 0 ? oz2_thin_applies(m, n, *plan, lay, s.kblock, compute_units) : 0;
  choice[0] = choice[1] ? 0 : oz2_one_pass_vectors(*plan, lay, 1, 0, m % 16 == 0, 0, call == 1, s.shift_mode, call == 0 ? s.bit_split : 0, compute_units);
  choice[2] = choice[1] ? 0 : oz2_products_tile(*plan, lay, m, n, s.kblock, u8, call == 1, krange, compute_units);
  return OZ2_OK;
}

int oz2_host_route(int call, char transa, char transb, int64_t m, int64_t n, int64_t k, int num_moduli, int compute_units, int route[4]) {
  const int ta = trans_code(transa), tb = trans_code(transb);
  if (ta < 0) return -2;
  if (tb < 0) return -3;
  State& s = state();
  std::lock_guard<std::mutex> lock(s.mu);
  const Oz2Plan* plan;
  Oz2Layout lay;
  const int rc = host_call(s, call, m, n, k, num_moduli, compute_units, &plan, &lay);
  if (rc != OZ2_OK) return rc == -1 ? -1 : rc - 2;
  if (!route) return -9;
  // dtrmm: A from the left where k is m, else from the right, where it is the second operand
  const bool right = call == 2 && k != m, symmetric = call == 1;
  const int strided_a = right ? 1 : !ta, strided_b = right ? ta : call == 0 ? tb : 0;
  const int lines_a = strided_a && m % 16 == 0, lines_b = strided_b && n % 16 == 0;
  const int u8 = s.product_format == OZ2_PRODUCT_RESIDUE_U8, split = call == 0 ? s.bit_split : 0;
  const int thin = u8 && call == 0 ? oz2_thin_applies(m, n, *plan, lay, s.kblock, compute_units) : 0;
  const bool both = !thin && oz2_one_pass_vectors(*plan, lay, strided_a, strided_b, lines_a, lines_b, symmetric, s.shift_mode, split, compute_units);
  const bool bounds = s.shift_mode == OZ2_SHIFT_INT8_PRODUCT;
  route[0] = both ? 3 : thin ? 0 : oz2_one_pass_operand(*plan, lay, strided_a, strided_b, lines_a, lines_b, call == 2, symmetric, s.shift_mode,
                                                             split, compute_units);
  route[1] = both && !bounds && oz2_planes_through_caches(num_moduli, lay, m, n, symmetric);
  route[2] = bounds ? oz2_bound_tile(lay, m, n, symmetric, compute_units) : 0;
  route[3] = call == 0 && fallback_in_stage3(s, m, n) ? 0 : oz2_crt_on_matrix_cores(*plan, m, n, u8, symmetric) ? 2 : 1;
  return OZ2_OK;
}

int oz2_host_crt_element(int num_moduli, const int32_t* cprod, double* x_out) {
  if (!n_ok(num_moduli)) return -1;
  if (!cprod) return -2;
  if (!x_out) return -3;
  Oz2Plan plan;
  if (oz2_build_plan(num_moduli, 1, &plan) < 0) return -1;  // the CRT tables do not depend on k
  *x_out = oz2_host_crt_impl(plan.crt, cprod);
  return OZ2_OK;
}

static int host_crt_element_digits(int num_moduli, int fewest, int most, const uint8_t* residues, double* x_out) {
  if (!n_ok(num_moduli) || num_moduli < fewest || num_moduli > most) return -1;
  if (!residues) return -2;
  if (!x_out) return -3;
  Oz2Plan plan;
  if (oz2_build_plan(num_moduli, 1, &plan) < 0 || !plan.digits.valid) return -1;
  for (int t = 0; t < num_moduli; ++t)
    if (residues[t] >= plan.moduli[t]) return -2;
  *x_out = oz2_host_crt_digits_impl(plan.crt, plan.digits, residues);
  return OZ2_OK;
}

int oz2_host_crt_element_digits(int num_moduli, const uint8_t* residues, double* x_out) {
  return host_crt_element_digits(num_moduli, OZ2_MIN_N, 16, residues, x_out);
}

int oz2_host_crt_element_wide_digits(int num_moduli, const uint8_t* residues, double* x_out) {
  return host_crt_element_digits(num_moduli, 17, OZ2_MFMA_N, residues, x_out);
}

int oz2_host_residues(int num_moduli, int kappa, double a, int shift, int8_t* res_out) {
  if (!n_ok(num_moduli)) return -1;
  if (kappa < 1 || kappa > 110) return -2;
  if (!res_out) return -5;
  Oz2Plan plan;
  if (oz2_build_plan(num_moduli, 1, &plan) < 0) return -1;
  plan.conv.two_level = kappa > 75;  // same rule as the launcher: |x| < 2^kappa
  return oz2_host_residues_impl(plan.conv, a, shift, res_out) ? OZ2_OK : -6;
}

typedef void (*Oz2HostResidues)(int p, int64_t count, const int32_t* products, uint8_t* out);
static int host_product_residues(int index, int64_t count, const int32_t* products, uint8_t* res_out, Oz2HostResidues impl) {
  if (index < 0 || index >= OZ2_MAX_N) return -1;
  if (count < 0) return -2;
  if (count == 0) return OZ2_OK;
  if (!products) return -3;
  if (!res_out) return -4;
  int moduli[OZ2_MAX_N];
  oz2_table_moduli(OZ2_MAX_N, moduli);
  impl(moduli[index], count, products, res_out);
  return OZ2_OK;
}

int oz2_host_product_residues(int index, int64_t count, const int32_t* products, uint8_t* res_out) {
  return host_product_residues(index, count, products, res_out, oz2_host_product_residues_impl);
}

int oz2_host_short_product_residues(int index, int64_t count, const int32_t* products, uint8_t* res_out) {
  return host_product_residues(index, count, products, res_out, oz2_host_short_product_residues_impl);
}

namespace {
bool type_ok(int type) { return type == OZ2_F32 || type == OZ2_BF16 || type == OZ2_F16; }

// A matrix (of a stack, if stacks are asked for) that the kernels can read: extents that they count in, rows that do not overlap.
bool w4_ok(const oz2_w4_matrix& w, bool stack) {
  if (w.n < 0 || w.k < 0 || w.n >= ((int64_t)1 << 31) - 65536 || w.k >= (int64_t)1 << 23) return false;
  if (w.group != 32 && w.group != 64 && (w.group < 128 || w.group % 128 != 0)) return false;
  if (!type_ok(w.scale_type)) return false;
  if (w.n == 0 || w.k == 0) return true;
  const int64_t bytes = (w.k + 1) / 2, groups = (w.k + w.group - 1) / w.group;
  if (!w.codes || !w.scales) return false;
  // one row has no next one, so its pitch says nothing
  if (w.n > 1 && (w.ld_codes < bytes || w.ld_scales < groups || (w.zeros && w.ld_zeros < groups))) return false;
  if (!stack) return true;
  if (w.count < 1) return false;
  const int64_t rows = w.n - 1;
  return w.count == 1 || (w.stride_codes >= rows * w.ld_codes + bytes && w.stride_scales >= rows * w.ld_scales + groups &&
                          (!w.zeros || w.stride_zeros >= rows * w.ld_zeros + groups));
}

int64_t size_of(int type) { return type == OZ2_F32 ? 4 : 2; }

// Whether any byte of `rows` rows of width_a bytes, pitch_a apart, belongs to as many of width_b, pitch_b apart; all four as checked.  Rows that lie
// between each other's do not meet.
bool rows_meet(const void* a, int64_t width_a, int64_t pitch_a, const void* b, int64_t width_b, int64_t pitch_b, int64_t rows) {
  if (rows == 1) pitch_a = pitch_b = 0;
  const int64_t start = (int64_t)((uintptr_t)b - (uintptr_t)a), far = (int64_t)1 << 46;  // (further apart no memory is; rows are below 2^16)
  if (pitch_a >= far || pitch_b >= far) return false;
  if (start >= (rows - 1) * pitch_a + width_a || start + (rows - 1) * pitch_b + width_b <= 0) return false;
  for (int64_t i = 0; i < rows; ++i) {
    const int64_t after = i * pitch_a - start - width_b, before = i * pitch_a + width_a - start;  // a row of b that meets row i begins between these
    const int64_t j = after < 0 ? 0 : pitch_b ? after / pitch_b + 1 : rows;
    if (j < rows && j * pitch_b < before) return true;
  }
  return false;
}

bool moe_ok(const oz2_moe_layer* m) {
  if (!m || !w4_ok(m->gate, true) || !w4_ok(m->up, true) || !w4_ok(m->down, true)) return false;
  const int64_t f = m->gate.n, d = m->gate.k, experts = m->gate.count;
  if (d < 1 || f < 1 || experts < 1 || experts > OZ2_MOE_MAX_EXPERTS) return false;
  if (m->up.n != f || m->up.k != d || m->up.count != experts) return false;
  if (m->up.group != m->gate.group || m->up.scale_type != m->gate.scale_type || !m->up.zeros != !m->gate.zeros) return false;
  if (m->down.n != d || m->down.k != f || m->down.count != experts) return false;
  if (!m->router || !type_ok(m->router_type) || (experts > 1 && m->ld_router < d)) return false;
  if (m->top_k < 1 || m->top_k > OZ2_MOE_MAX_TOP_K || m->top_k > experts) return false;
  if (m->score != OZ2_SCORE_SOFTMAX && m->score != OZ2_SCORE_SIGMOID) return false;
  return m->activation == OZ2_ACT_SILU || m->activation == OZ2_ACT_GELU;
}
}  // namespace

int oz2_w4_matvec(const oz2_w4_matrix* W, int64_t t, float alpha, int x_type, const void* X, int64_t ldx, float beta, const void* C,
                  int64_t ldc, int y_type, void* Y, int64_t ldy, void* stream) {
  if (!W) return -1;
  oz2_w4_matrix w = *W;
  if (alpha == 0.f) w.k = 0;
  if (!w4_ok(w, false)) return -1;
  if (t < 0 || t > 65535) return -2;
  if (!type_ok(x_type)) return -4;
  if (t > 1 && w.k > 0 && ldx < w.k) return -6;
  if (beta != 0.f && t > 1 && ldc < (w.n > 1 ? w.n : 1)) return -9;
  if (!type_ok(y_type)) return -10;
  if (t > 1 && ldy < (w.n > 1 ? w.n : 1)) return -12;
  if (w.n == 0 || t == 0) return OZ2_OK;
  if (w.k > 0 && !X) return -5;
  if (beta != 0.f && !C) return -8;
  if (!Y) return -11;
  const int64_t xs = size_of(x_type), ys = size_of(y_type);
  if (beta != 0.f && !(C == Y && (t == 1 || ldc == ldy)) && rows_meet(C, w.n * ys, ldc * ys, Y, w.n * ys, ldy * ys, t)) return -8;
  if (w.k > 0 && rows_meet(X, w.k * xs, ldx * xs, Y, w.n * ys, ldy * ys, t)) return -11;
  return oz2_launch_w4_matvec(w, t, alpha, x_type, X, ldx, beta, C, ldc, y_type, Y, ldy, static_cast<hipStream_t>(stream)) == hipSuccess
             ? OZ2_OK : OZ2_ERR_HIP;
}

size_t oz2_w4_moe_workspace_bytes(const oz2_moe_layer* layer, int64_t t) {
  if (!moe_ok(layer) || t < 0 || t > OZ2_MOE_MAX_TOKENS) return 0;
  return oz2_w4_moe_space(*layer, t ? t : 1);
}

int oz2_w4_moe(const oz2_moe_layer* layer, int64_t t, int x_type, const void* X, int64_t ldx, const uint8_t* active, int y_type, void* Y,
               int64_t ldy, int32_t* ids, float* weights, void* stream) {
  if (!moe_ok(layer)) return -1;
  if (t < 0 || t > OZ2_MOE_MAX_TOKENS) return -2;
  if (!type_ok(x_type)) return -3;
  if (t > 1 && ldx < layer->gate.k) return -5;
  if (!type_ok(y_type)) return -7;
  if (t > 1 && ldy < layer->gate.k) return -9;
  if (t == 0) return OZ2_OK;
  if (!X) return -4;
  if (!Y) return -8;
  // (a token's own x may become its y: it is read before the launch that writes y, and no later piece of the call has it)
  const int64_t d = layer->gate.k, xs = size_of(x_type), ys = size_of(y_type);
  if (!(X == Y && xs == ys && (t == 1 || ldx == ldy)) && rows_meet(X, d * xs, ldx * xs, Y, d * ys, ldy * ys, t)) return -8;
  State& s = state();
  std::lock_guard<std::mutex> lock(s.mu);
  if (!s.ws || s.ws_bytes < oz2_w4_moe_space(*layer, t)) return OZ2_ERR_WORKSPACE;
  return oz2_launch_w4_moe(*layer, t, x_type, X, ldx, active, y_type, Y, ldy, ids, weights, s.ws, static_cast<hipStream_t>(stream)) == hipSuccess
             ? OZ2_OK : OZ2_ERR_HIP;
}

int oz2_context_w4_moe(oz2_context* ctx, const oz2_moe_layer* layer, int64_t t, int x_type, const void* X, int64_t ldx,
                       const uint8_t* active, int y_type, void* Y, int64_t ldy, int32_t* ids, float* weights, void* stream) {
  UseContext use(ctx);
  const int rc = oz2_w4_moe(layer, t, x_type, X, ldx, active, y_type, Y, ldy, ids, weights, stream);
  return rc < 0 ? rc - 1 : rc;
}

namespace {
// Rows of width `width` at i step_a + j step_b (i < a, j < b) that do not overlap: the smaller step keeps rows apart, the larger one runs of them.
bool lattice_ok(int64_t width, int64_t a, int64_t step_a, int64_t b, int64_t step_b) {
  if ((a > 1 && step_a < width) || (b > 1 && step_b < width)) return false;
  typedef __int128 wide;
  if ((a > 1 ? (wide)(a - 1) * step_a : 0) + (b > 1 ? (wide)(b - 1) * step_b : 0) >= (wide)1 << 46) return false;  // (no memory is that large)
  if (a <= 1 || b <= 1) return true;
  return step_a < step_b ? step_b - width >= (a - 1) * step_a : step_a - width >= (b - 1) * step_b;
}
bool rows_ok(const oz2_rows* r, int64_t tokens, int64_t heads, int64_t dim) {
  return r && type_ok(r->type) && (tokens == 0 || (r->data && lattice_ok(dim, tokens, r->ld_token, heads, r->ld_head)));  // (strides of no tokens say nothing)
}
// Whether two tensors of heads have no byte in common, as far as that is easily seen: one lies behind the other, or what one has of a token (or, where these are
// further apart, of a head) lies between what the other has of two, like parts of one packed tensor.
bool rows_apart(const oz2_rows& a, int64_t heads_a, const oz2_rows& b, int64_t heads_b, int64_t tokens, int64_t dim) {
  const int64_t size_a = size_of(a.type), size_b = size_of(b.type);
  // (a stride of a single token or head says nothing)
  const int64_t tokens_a = tokens > 1 ? (tokens - 1) * a.ld_token * size_a : 0, tokens_b = tokens > 1 ? (tokens - 1) * b.ld_token * size_b : 0;
  const int64_t all_a = heads_a > 1 ? (heads_a - 1) * a.ld_head * size_a : 0, all_b = heads_b > 1 ? (heads_b - 1) * b.ld_head * size_b : 0;
  const uintptr_t pa = (uintptr_t)a.data, pb = (uintptr_t)b.data;
  if (pa >= pb + tokens_b + all_b + dim * size_b || pb >= pa + tokens_a + all_a + dim * size_a) return true;
  auto between = [&](int64_t step_a, int64_t step_b, int64_t inner_a, int64_t inner_b) {
    const int64_t step = step_a ? step_a : step_b, bytes_a = inner_a + dim * size_a, bytes_b = inner_b + dim * size_b;
    if (!step || (step_a && step_b && step_a != step_b) || step < bytes_a || step < bytes_b) return false;
    int64_t from = (int64_t)(pb - pa) % step;
    if (from < 0) from += step;
    return from >= bytes_a && from + bytes_b <= step;
  };
  return between(tokens > 1 ? a.ld_token * size_a : 0, tokens > 1 ? b.ld_token * size_b : 0, all_a, all_b) ||
         between(heads_a > 1 ? a.ld_head * size_a : 0, heads_b > 1 ? b.ld_head * size_b : 0, tokens_a, tokens_b);
}
bool same_rows(const oz2_rows& a, const oz2_rows& b) {
  return a.data == b.data && a.ld_token == b.ld_token && a.ld_head == b.ld_head && a.type == b.type;
}

constexpr int64_t kMostRows = (int64_t)1 << 23, kMostSequences = 65535;  // (grid extents; a grid has fewer than 2^32 threads)

bool cache_ok(const oz2_kv4_cache* c) {
  if (!c || c->pages < 1 || c->pages > INT32_MAX || c->heads < 1 || c->heads > 65535) return false;
  if (c->page_size < 16 || c->page_size % 16 || c->page_size > ((int64_t)1 << 24) || c->dim < 8 || c->dim % 8 || c->dim > OZ2_ATTENTION_MAX_DIM) return false;
  if (!c->k_codes || !c->v_codes || !c->k_scales || !c->v_scales) return false;
  if (((uintptr_t)c->k_codes | (uintptr_t)c->v_codes) % 4 || ((uintptr_t)c->k_scales | (uintptr_t)c->v_scales) % 16) return false;
  if ((c->pages > 1 && (c->codes_page % 4 || c->scales_page % 4)) || (c->heads > 1 && (c->codes_head % 4 || c->scales_head % 4))) return false;
  return lattice_ok(c->page_size * c->dim / 2, c->pages, c->codes_page, c->heads, c->codes_head) &&
         lattice_ok(c->page_size, c->pages, c->scales_page, c->heads, c->scales_head);
}
bool capacity_ok(const oz2_kv4_cache& c, int64_t sequences, int64_t max_pages) {
  return sequences >= 0 && sequences <= kMostSequences && sequences * c.heads <= ((int64_t)1 << 21) && max_pages >= 0 &&
         max_pages <= 65535 * (int64_t)4096 / c.page_size;  // (65535 chunks of 4096 places, a grid's extent)
}
// arrays of (sequence, head, place)
bool places_ok(const oz2_kv4_cache& c, const oz2_kv4_sequences& on, int64_t sequence, int64_t head) {
  const int64_t capacity = on.max_pages * c.page_size;
  return capacity == 0 || lattice_ok(capacity, on.sequences, sequence, c.heads, head);
}
bool sequences_ok(const oz2_kv4_cache& c, const oz2_kv4_sequences* on, bool fresh) {
  if (!on || !capacity_ok(c, on->sequences, on->max_pages)) return false;
  if (fresh && (on->tokens < 0 || on->tokens > ((int64_t)1 << 26) / c.heads)) return false;
  if (on->sequences == 0) return true;
  if (!on->lengths || (fresh && !on->cu) || (on->max_pages && !on->table) || (on->sequences > 1 && on->ld_table < on->max_pages)) return false;
  return (!on->positions || places_ok(c, *on, on->positions_sequence, on->positions_head)) &&
         (!on->weights || places_ok(c, *on, on->weights_sequence, on->weights_head));
}
bool apart(const void* p, int64_t bytes_p, const void* q, int64_t bytes_q) {
  return (uintptr_t)p + bytes_p <= (uintptr_t)q || (uintptr_t)q + bytes_q <= (uintptr_t)p;
}
// Arrays of (sequence, head, place) of 4 bytes, and whether two of them have no byte in common, as far as that is easily seen: one lies behind the other, or with the same
// strides what one has of a sequence or a head lies between what the other has of two.
struct Places { const void* data; int64_t sequence, head; };
int64_t places_bytes(const Places& a, int64_t sequences, int64_t heads, int64_t capacity) {
  return 4 * ((sequences > 1 ? (sequences - 1) * a.sequence : 0) + (heads > 1 ? (heads - 1) * a.head : 0) + capacity);
}
bool places_apart(const Places& a, const Places& b, int64_t sequences, int64_t heads, int64_t capacity) {
  const int64_t bytes = places_bytes(a, sequences, heads, capacity);
  if (apart(a.data, bytes, b.data, places_bytes(b, sequences, heads, capacity))) return true;
  if ((sequences > 1 && a.sequence != b.sequence) || (heads > 1 && a.head != b.head)) return false;
  // rows of `width` at `inner` steps, which repeat at `outer` ones (0: there is but one)
  const int64_t s = sequences > 1 ? 4 * a.sequence : 0, h = heads > 1 ? 4 * a.head : 0, inner = s && h ? (s < h ? s : h) : s + h, outer = s && h ? (s < h ? h : s) : 0;
  const int64_t width = 4 * capacity, by = (int64_t)((uintptr_t)b.data - (uintptr_t)a.data);
  auto between = [](int64_t by, int64_t step, int64_t width) {
    const int64_t from = (by % step + step) % step;
    return from >= width && from + width <= step;
  };
  if (!inner) return false;
  if (!outer) return between(by, inner, width);
  if (between(by, outer, bytes - (outer == s ? (sequences - 1) * s : (heads - 1) * h))) return true;
  const int64_t from = (by % outer + outer) % outer;
  return between(from, inner, width) && between(from - outer, inner, width);
}
// Whether what an eviction writes is in each case the array that it reads the same of, or apart from all others.
bool kept_ok(const oz2_kv4_cache& c, const oz2_kv4_sequences& on, const oz2_kv4_kept& to) {
  const int64_t n = on.sequences, capacity = on.max_pages * c.page_size;
  const Places read[2] = {{on.positions, on.positions_sequence, on.positions_head}, {on.weights, on.weights_sequence, on.weights_head}};
  const Places write[2] = {{to.positions, to.positions_sequence, to.positions_head}, {to.weights, to.weights_sequence, to.weights_head}};
  if (to.lengths != on.lengths && !apart(to.lengths, 4 * n, on.lengths, 4 * n)) return false;
  if (!capacity) return true;
  const int64_t ld = on.ld_table < ((int64_t)1 << 40) ? on.ld_table : (int64_t)1 << 40, table = 4 * ((n > 1 ? (n - 1) * ld : 0) + on.max_pages);  // (no memory is larger)
  if (!apart(to.lengths, 4 * n, on.table, table)) return false;
  for (int i = 0; i < 2; ++i) {
    const int64_t bytes = places_bytes(write[i], n, c.heads, capacity);
    if (!apart(write[i].data, bytes, to.lengths, 4 * n) || !apart(write[i].data, bytes, on.lengths, 4 * n) || !apart(write[i].data, bytes, on.table, table)) return false;
    if (to.lengths != on.lengths && !apart(to.lengths, 4 * n, read[i].data, places_bytes(read[i], n, c.heads, capacity))) return false;
    for (int j = 0; j < 2; ++j) {
      // (the same array with other strides would be read and written at once)
      const bool same = i == j && write[i].data == read[j].data && (n <= 1 || write[i].sequence == read[j].sequence) && (c.heads <= 1 || write[i].head == read[j].head);
      if (!same && !places_apart(write[i], read[j], n, c.heads, capacity)) return false;
    }
  }
  return places_apart(write[0], write[1], n, c.heads, capacity);
}
// (most: kernels take it times log2(e), on a cache times 2^69 too, and the power of two above that, or its reciprocal)
bool scale_ok(float scale, float most) { return scale > 0.f && scale <= most; }
}  // namespace

int oz2_attention(int64_t tokens, int64_t sequences, const int32_t* cu, int64_t heads, int64_t kv_heads, int64_t dim, float scale, int causal,
                  const oz2_rows* q, const oz2_rows* k, const oz2_rows* v, const oz2_rows* out, void* stream) {
  if (tokens < 0 || tokens > ((int64_t)1 << 28)) return -1;
  if (sequences < 0 || sequences > ((int64_t)1 << 20)) return -2;
  if (heads < 1 || heads > 65535 || tokens * heads > ((int64_t)1 << 28)) return -4;
  if (kv_heads < 1 || heads % kv_heads) return -5;
  if (sequences * kv_heads > ((int64_t)1 << 22)) return -2;
  if (dim < 1 || dim > OZ2_ATTENTION_MAX_DIM) return -6;
  if (!scale_ok(scale, 0x1p126f)) return -7;
  if (!rows_ok(q, tokens, heads, dim)) return -9;
  if (!rows_ok(k, tokens, kv_heads, dim) || k->type != q->type) return -10;
  if (!rows_ok(v, tokens, kv_heads, dim) || v->type != q->type) return -11;
  if (!rows_ok(out, tokens, heads, dim)) return -12;
  if (tokens == 0 || sequences == 0) return OZ2_OK;
  if (!cu) return -3;
  if (!rows_apart(*out, heads, *q, heads, tokens, dim) || !rows_apart(*out, heads, *k, kv_heads, tokens, dim) ||
      !rows_apart(*out, heads, *v, kv_heads, tokens, dim))
    return -12;
  return oz2_launch_attention(tokens, sequences, cu, heads, kv_heads, dim, scale, causal, *q, *k, *v, *out, static_cast<hipStream_t>(stream)) == hipSuccess
             ? OZ2_OK : OZ2_ERR_HIP;
}

int oz2_kv4_append(const oz2_kv4_cache* cache, const oz2_kv4_sequences* on, const int32_t* at, const oz2_rows* k, const oz2_rows* v, const oz2_rows* held_k,
                   const oz2_rows* held_v, void* stream) {
  if (!cache_ok(cache)) return -1;
  if (!sequences_ok(*cache, on, true)) return -2;
  if (at && !on->positions) return -3;
  const int64_t tokens = on->tokens, heads = cache->heads, dim = cache->dim;
  if (!rows_ok(k, tokens, heads, dim)) return -4;
  if (!rows_ok(v, tokens, heads, dim) || v->type != k->type) return -5;
  if (held_k && (!rows_ok(held_k, tokens, heads, dim) || held_k->type != k->type)) return -6;
  if (held_v && (!rows_ok(held_v, tokens, heads, dim) || held_v->type != k->type)) return -7;
  if (tokens == 0 || on->sequences == 0) return OZ2_OK;
  if (held_k && !((same_rows(*held_k, *k) || rows_apart(*held_k, heads, *k, heads, tokens, dim)) && rows_apart(*held_k, heads, *v, heads, tokens, dim))) return -6;
  if (held_v && !((same_rows(*held_v, *v) || rows_apart(*held_v, heads, *v, heads, tokens, dim)) && rows_apart(*held_v, heads, *k, heads, tokens, dim))) return -7;
  if (held_k && held_v && !rows_apart(*held_k, heads, *held_v, heads, tokens, dim)) return -7;
  return oz2_launch_kv4_append(*cache, *on, at, *k, *v, held_k, held_v, static_cast<hipStream_t>(stream)) == hipSuccess ? OZ2_OK : OZ2_ERR_HIP;
}

size_t oz2_kv4_attention_workspace_bytes(const oz2_kv4_cache* cache, int64_t sequences, int64_t max_pages, int64_t tokens, int64_t heads, int weights) {
  if (!cache_ok(cache) || !capacity_ok(*cache, sequences, max_pages) || tokens < 0 || heads < 1 || heads % cache->heads || tokens > kMostRows / heads) return 0;
  return oz2_kv4_attention_space(*cache, sequences, max_pages, tokens, heads, weights) + 256;
}

int oz2_kv4_attention(const oz2_kv4_cache* cache, const oz2_kv4_sequences* on, int64_t heads, float scale, const oz2_rows* q, const oz2_rows* out, void* stream) {
  if (!cache_ok(cache)) return -1;
  if (!sequences_ok(*cache, on, true)) return -2;
  const int64_t tokens = on->tokens;
  if (heads < 1 || heads % cache->heads || tokens > kMostRows / heads) return -3;
  if (!scale_ok(scale, 0x1p55f)) return -4;
  if (!rows_ok(q, tokens, heads, cache->dim)) return -5;
  if (!rows_ok(out, tokens, heads, cache->dim)) return -6;
  if (tokens == 0 || on->sequences == 0) return OZ2_OK;
  if (!rows_apart(*out, heads, *q, heads, tokens, cache->dim)) return -6;
  State& s = state();
  std::lock_guard<std::mutex> lock(s.mu);
  if (!s.ws || s.ws_bytes < oz2_kv4_attention_space(*cache, on->sequences, on->max_pages, tokens, heads, on->weights != nullptr)) return OZ2_ERR_WORKSPACE;
  return oz2_launch_kv4_attention(*cache, *on, heads, scale, *q, *out, s.ws, static_cast<hipStream_t>(stream)) == hipSuccess ? OZ2_OK : OZ2_ERR_HIP;
}

int oz2_context_kv4_attention(oz2_context* ctx, const oz2_kv4_cache* cache, const oz2_kv4_sequences* on, int64_t heads, float scale, const oz2_rows* q,
                              const oz2_rows* out, void* stream) {
  UseContext use(ctx);
  const int rc = oz2_kv4_attention(cache, on, heads, scale, q, out, stream);
  return rc < 0 ? rc - 1 : rc;
}

size_t oz2_kv4_evict_workspace_bytes(const oz2_kv4_cache* cache, int64_t sequences, int64_t max_pages, int64_t keep) {
  if (!cache_ok(cache) || !capacity_ok(*cache, sequences, max_pages) || keep < 0) return 0;
  return oz2_kv4_evict_space(*cache, sequences, max_pages, keep) + 256;
}

int oz2_kv4_evict(const oz2_kv4_cache* cache, const oz2_kv4_sequences* on, int64_t keep, int64_t recent, const oz2_kv4_kept* to, void* stream) {
  if (!cache_ok(cache)) return -1;
  if (!sequences_ok(*cache, on, false) || (on->sequences && (!on->positions || !on->weights))) return -2;
  if (keep < 0) return -3;
  if (recent < 0 || recent > keep) return -4;
  oz2_kv4_kept here = {const_cast<int32_t*>(on->lengths), on->positions, on->positions_sequence, on->positions_head, on->weights, on->weights_sequence, on->weights_head};
  if (to) {
    if (on->sequences && (!to->lengths || !to->positions || !to->weights)) return -5;
    if (on->sequences && (!places_ok(*cache, *on, to->positions_sequence, to->positions_head) || !places_ok(*cache, *on, to->weights_sequence, to->weights_head))) return -5;
    if (on->sequences && !kept_ok(*cache, *on, *to)) return -5;
    here = *to;
  }
  if (on->sequences == 0) return OZ2_OK;
  State& s = state();
  std::lock_guard<std::mutex> lock(s.mu);
  if (!s.ws || s.ws_bytes < oz2_kv4_evict_space(*cache, on->sequences, on->max_pages, keep)) return OZ2_ERR_WORKSPACE;
  return oz2_launch_kv4_evict(*cache, *on, keep, recent, here, s.ws, static_cast<hipStream_t>(stream)) == hipSuccess ? OZ2_OK : OZ2_ERR_HIP;
}

int oz2_context_kv4_evict(oz2_context* ctx, const oz2_kv4_cache* cache, const oz2_kv4_sequences* on, int64_t keep, int64_t recent, const oz2_kv4_kept* to,
                          void* stream) {
  UseContext use(ctx);
  const int rc = oz2_kv4_evict(cache, on, keep, recent, to, stream);
  return rc < 0 ? rc - 1 : rc;
}

const char* oz2_status_string(int status) {
  switch (status) {
    case OZ2_OK: return "success";
    case OZ2_ERR_WORKSPACE: return "workspace not registered or too small";
    case OZ2_ERR_BUDGET: return "bit budget: moduli product too small for this inner dimension, or a bit split or shift mode it cannot serve";
    case OZ2_ERR_HIP: return "HIP call failed";
    case OZ2_ERR_STATIC_LIMIT: return "problem needs more workspace than the library's static buffer holds (OZ2_STATIC_SCRATCH_BYTES)";
    default: return status < 0 ? "invalid argument" : "unknown status";
  }
}

}  // extern "C"
