// Host side of the checkpointed linear layer: argument checking, workspaces and launches.
// The C ABI is declared in include/efsparse.h, the kernels are in ef_linear.h.

#include "ef_host.h"
#include "ef_linear.h"

#include <algorithm>
#include <cmath>
#include <initializer_list>

using namespace efs;

namespace {

constexpr int64_t kMaxWidth = (int64_t)1 << 26;  // columns, and output features
constexpr int64_t kMaxRows = (int64_t)1 << 31;
constexpr int64_t kMaxThreads = ((int64_t)1 << 32) - 1;  // of a grid, along one dimension

bool dtype_ok(int t) { return t == EF_F32 || t == EF_BF16; }
bool fmt_ok(int f) { return f == EF_CKPT_INT8 || f == EF_CKPT_E4M3; }
bool act_ok(int a) { return a >= EF_ACT_NONE && a <= EF_ACT_SILU; }
int64_t bytes_of(int t) { return t == EF_F32 ? 4 : 2; }
int32_t groups(int64_t c) { return (int32_t)((c + kGroup - 1) / kGroup); }

// A matrix argument: aligned to its elements, rows at least as far apart as they are long.
bool mat_ok(const void* p, int64_t rows, int64_t cols, int64_t ld, int t) {
  return ld >= cols && ld < ((int64_t)1 << 40) && (rows == 0 || (p && aligned(p, (size_t)bytes_of(t))));
}

bool kept_ok(const uint8_t* codes, const uint8_t* scales, int64_t rows) {
  return rows == 0 || (codes && scales && aligned(codes, 16));
}

// The bytes of a matrix: from a to b, `width` of every `stride`.
struct Range {
  const char *a, *b;
  int64_t stride, width;
};
Range range(const void* p, int64_t rows, int64_t cols, int64_t ld, int64_t size) {
  const char* q = static_cast<const char*>(p);
  if (!q || !rows) return {nullptr, nullptr, 0, 0};
  return {q, q + ((rows - 1) * ld + cols) * size, ld * size, cols * size};
}
Range range_kept(const uint8_t* codes, int64_t rows, int64_t c) {
  const int64_t row = (int64_t)groups(c) * kGroup;
  return range(codes, rows, row, row, 1);
}
Range range_scales(const uint8_t* s, int64_t rows, int64_t c) { return range(s, rows, groups(c), groups(c), 1); }
bool meet(Range x, Range y) {
  if (!(x.a < y.b && y.a < x.b)) return false;
  if (x.stride != y.stride) return true;
  // rows equally far apart: side by side in the same rows (columns of one buffer) they do not meet
  const int64_t d = ((y.a - x.a) % x.stride + x.stride) % x.stride;
  return d < x.width || d + y.width > x.stride;
}
template <typename... R> bool meet_any(Range x, R... y) { return (meet(x, y) || ...); }

// Grid of the elementwise passes: lanes per row (as a power of two's exponent), and workgroups: columns along y, rows
// along x and, from 2^23 on, z.
struct Flat {
  dim3 grid;
  int txs;
};
int flat_of(int64_t n, int64_t c, Flat* f) {
  const int64_t lanes = (int64_t)groups(c) * 4;
  int txs = 2;
  while (txs < 8 && ((int64_t)1 << txs) < lanes) ++txs;
  const int64_t gx = (n + (256 >> txs) - 1) / (256 >> txs), gy = (lanes + ((int64_t)1 << txs) - 1) >> txs;
  const int64_t most = (int64_t)1 << 23, gz = (gx + most - 1) / most;
  if (gz > 65535 || gy > 65535) return EF_ERANGE;
  f->grid = dim3((unsigned)std::min(gx, most), (unsigned)gy, (unsigned)gz);
  f->txs = txs;
  return EF_OK;
}

// One product: sizes of C and of the sum, the operands and the epilogue.
struct Product {
  int64_t M, N, K;
  Mat A, B;
  Kept BK;
  Epi ep;
};

int check_sizes(int64_t n, int64_t i, int64_t o) {
  if (n < 0 || n >= kMaxRows || i < 1 || i > kMaxWidth || o < 1 || o > kMaxWidth) return EF_ERANGE;
  return EF_OK;
}

// bfloat16 matrices whose rows start on 16 bytes and hold whole 16-byte chunks
bool fast_mat(const Mat& m, int64_t cols) {
  return aligned(m.p, 16) && m.ld % 8 == 0 && cols % 8 == 0 && m.ld <= kFastLd;
}

template <int KIND>
bool fast_ok(const Product& p) {
  if (p.K == 0 || p.K > ((int64_t)1 << 30) || !fast_mat(p.A, KIND == K_WGRAD ? p.M : p.K)) return false;
  return KIND == K_WGRAD ? p.N <= kFastLd : fast_mat(p.B, KIND == K_FWD ? p.K : p.N);
}

// Few tokens: rows on 16 bytes, whole chunks of eight.
template <int DT>
bool few_ok(const Product& p) {
  const int64_t a = 16 / bytes_of(DT);
  return p.K % 8 == 0 && aligned(p.A.p, 16) && aligned(p.B.p, 16) && p.A.ld % a == 0 && p.B.ld % a == 0 &&
         std::max(p.A.ld, p.B.ld) <= kFastLd / 2;
}

// How a product is run: over `splits` parts of k, `per` steps each (the last may have fewer), whose sums are joined.
enum Form { kAny, kSmall, kLarge };  // k_linear_any, k_linear_bf16 of 128 x 128, of 256 x 256
struct Plan {
  Form form;
  int32_t splits, per;
};

constexpr int kCUs = 256;

// Microseconds that a form takes, fitted to what was measured: for each round of the workgroups that the CUs hold at
// one time, `few` to `full` for one step along k (from where half of them are at work, one a CU, to all of them:
// workgroups share a CU, and the chip its power) and `fixed` for the start and the epilogue; then the partial sums
// written, and the join: a launch, and the sums read.  For instance forward of normal values, n, i, o = 2048, 4096, 4096:
// 128 x 128 tiles 63 measured, 67 by this; 256 x 256 tiles 73 and 80, in two parts of k 76 and 93.  8192, 4096, 4096:
// 256 x 256 tiles 207 and 238 (values of activations: 236).  wgrad of 8192 tokens, 768 x 768, 128 x 128 tiles, in 4, 7, 8
// and 13 parts: 34, 27, 31 and 27 measured, 42, 33, 32 and 33 by this: the forms are told apart, the parts of k only
// nearly (8 are taken).
struct Cost {
  int tile, k, per_cu;
  double few, full, fixed;
};
Cost cost_of_form(int form, bool wgrad, bool f32) {
  if (form == kLarge) return {256, kBK, 1, 1.1, wgrad ? 1.8 : 1.7, wgrad ? 17.0 : 10.0};
  if (form == kSmall) return {128, kBK, 2, wgrad ? 0.9 : 0.45, wgrad ? 1.3 : 0.95, 6.0};
  if (f32) return {kAnyTile, kAnyK, 2, wgrad ? 1.4 : 2.2, wgrad ? 2.1 : 3.3, 5.0};
  return {kAnyTile, kAnyK, 2, wgrad ? 0.8 : 0.6, 1.1, 5.0};
}

double cost_of(const Cost& c, int64_t M, int64_t N, int64_t splits, int64_t per) {
  const double wgs = (double)((M + c.tile - 1) / c.tile) * (double)((N + c.tile - 1) / c.tile) * (double)splits;
  const double slots = (double)kCUs * c.per_cu, rounds = std::ceil(wgs / slots);
  const double busy = std::min(std::max(2.0 * wgs / slots - 1.0, 0.0), 1.0);
  double t = rounds * ((c.few + (c.full - c.few) * busy) * (double)per + c.fixed);
  if (splits > 1) t += 3.5 + (double)splits * (double)M * (double)N * (4.0 / 6e6 + 4.0 / 5e6);
  return t;
}

// The form and the number of splits that these costs are least for.  The choice goes by sizes, types and alignment
// alone: the same call always sums in the same order.
Plan plan_of(bool fast, bool wgrad, bool f32, int64_t M, int64_t N, int64_t K) {
  Plan best{kAny, 1, 1};
  double least = 0.0;
  for (int f = fast ? kSmall : kAny; f <= (fast ? kLarge : kAny); ++f) {
    const Cost c = cost_of_form(f, wgrad, f32);
    const int64_t steps = std::max<int64_t>((K + c.k - 1) / c.k, 1);
    const int64_t tiles = ((M + c.tile - 1) / c.tile) * ((N + c.tile - 1) / c.tile);
    for (int64_t s = 1; s <= 64 && s <= steps && (s == 1 || tiles * s <= 2 * kCUs * c.per_cu); ++s) {
      const int64_t per = (steps + s - 1) / s, splits = (steps + per - 1) / per;
      if (splits != s) continue;
      const double t = cost_of(c, M, N, splits, per);
      if (least == 0.0 || t < least) {
        least = t;
        best = {(Form)f, (int32_t)splits, (int32_t)per};
      }
    }
  }
  return best;
}

int32_t padded(int64_t N) { return groups(N) * kGroup; }

// The workspace of a product, whatever the alignment of its matrices turns out to be.
size_t product_bytes(bool wgrad, int dtype, int64_t M, int64_t N, int64_t K) {
  int32_t splits = M ? plan_of(false, wgrad, dtype == EF_F32, M, N, K).splits : 1;
  if (M && dtype == EF_BF16) splits = std::max(splits, plan_of(true, wgrad, false, M, N, K).splits);
  return splits == 1 ? 0 : align_up((size_t)splits * ((size_t)M * padded(N) + (size_t)M) * 4, kAlign);
}

// Names of the products' launches in the timing records, by kernel and kind.
constexpr const char* kLabel[4][3] = {
    {"k_linear_bf16<256> forward", "k_linear_bf16<256> dgrad", "k_linear_bf16<256> wgrad"},
    {"k_linear_bf16<128> forward", "k_linear_bf16<128> dgrad", "k_linear_bf16<128> wgrad"},
    {"k_linear_any forward", "k_linear_any dgrad", "k_linear_any wgrad"},
    {"k_linear_join forward", "k_linear_join dgrad", "k_linear_join wgrad"}};

template <int KIND, int DT, int DO>
int run_product(const Product& p, void* ws, size_t ws_bytes, hipStream_t st, std::initializer_list<Range> others) {
  const size_t need = product_bytes(KIND == K_WGRAD, DT, p.M, p.N, p.K);
  if (need) {
    if (!ws || !aligned(ws, kAlign)) return EF_EINVAL;
    if (ws_bytes < need) return EF_EWORKSPACE;
    const Range r = range(ws, 1, (int64_t)need, (int64_t)need, 1);
    for (const Range& x : others)
      if (meet(r, x)) return EF_EINVAL;
  }
  const bool fast = DT == EF_BF16 && fast_ok<KIND>(p);
  if constexpr (KIND == K_FWD) {
    if (p.M <= kFewTokens && few_ok<DT>(p)) {
      // (32 outputs a workgroup where a group of the checkpoint needs them, or where half the workgroups fill the CUs)
      const int ot = p.ep.k.codes || p.N >= 16 * 4 * kCUs ? 2 : 1;
      const dim3 grid((unsigned)((p.N + 16 * ot - 1) / (16 * ot))), blk(kFewWaves * 64);
#define EF_FEW(TT, OT) EF_LAUNCH_AS("k_linear_few forward", (k_linear_few<DT, TT, OT>), grid, blk, 0, st, (int32_t)p.M, (int32_t)p.N, (int32_t)p.K, p.A, p.B, p.ep)
      if (p.M <= 16 && ot == 1) EF_FEW(1, 1);
      else if (p.M <= 16) EF_FEW(1, 2);
      else if (ot == 1) EF_FEW(2, 1);
      else EF_FEW(2, 2);
#undef EF_FEW
      return launched();
    }
  }
  const Plan pl = plan_of(fast, KIND == K_WGRAD, DT == EF_F32, p.M, p.N, p.K);
  const int64_t tile = pl.form == kLarge ? 256 : 128, tiles = ((p.M + tile - 1) / tile) * ((p.N + tile - 1) / tile);
  if (tiles * pl.splits > kMaxThreads / (pl.form == kLarge ? 512 : 256)) return EF_ERANGE;
  Split sp{nullptr, nullptr, p.M * padded(p.N), padded(p.N), pl.per, pl.splits};
  if (pl.splits > 1) {
    sp.part = static_cast<float*>(ws);
    sp.part_db = sp.part + (int64_t)pl.splits * sp.plane;
  }
  const dim3 grid((unsigned)(tiles * pl.splits));
  const int32_t M = (int32_t)p.M, N = (int32_t)p.N, K = (int32_t)p.K;
#define EF_FORM(FMT)                                                                                                  \
  do {                                                                                                                \
    if (pl.form == kLarge)                                                                                            \
      EF_LAUNCH_AS(kLabel[0][KIND], (k_linear_bf16<KIND, DO, FMT, 256, 256, 2, 4>), grid, dim3(512), 0, st, M, N, K, p.A, p.B, p.BK, p.ep, sp); \
    else                                                                                                              \
      EF_LAUNCH_AS(kLabel[1][KIND], (k_linear_bf16<KIND, DO, FMT, 128, 128, 2, 2>), grid, dim3(256), 0, st, M, N, K, p.A, p.B, p.BK, p.ep, sp); \
  } while (0)
  if constexpr (DT == EF_BF16) {
    if (pl.form == kAny) {
      EF_LAUNCH_AS(kLabel[2][KIND], (k_linear_any<KIND, DT, DO>), grid, dim3(256), 0, st, M, N, K, p.A, p.B, p.BK, p.ep, sp);
    } else if constexpr (KIND == K_WGRAD) {
      if (p.BK.fmt == EF_CKPT_E4M3) EF_FORM(EF_CKPT_E4M3);
      else EF_FORM(EF_CKPT_INT8);
    } else {
      EF_FORM(EF_CKPT_INT8);  // (read no checkpoint along k)
    }
  } else {
    EF_LAUNCH_AS(kLabel[2][KIND], (k_linear_any<KIND, DT, DO>), grid, dim3(256), 0, st, M, N, K, p.A, p.B, p.BK, p.ep, sp);
  }
#undef EF_FORM
  EF_TRY(launched());
  if (pl.splits == 1) return EF_OK;
  const int64_t lanes = p.M * (sp.Np / 8) + (KIND == K_WGRAD && p.ep.db ? p.M : 0);
  EF_LAUNCH_AS(kLabel[3][KIND], (k_linear_join<KIND, DO>), dim3((unsigned)((lanes + 255) / 256)), dim3(256), 0, st, M, N, sp, p.ep);
  return launched();
}

}  // namespace

extern "C" {

int64_t ef_ckpt_row_bytes(int64_t c) { return c < 1 || c > kMaxWidth ? 0 : (int64_t)groups(c) * kGroup; }

int ef_ckpt_pack(int64_t n, int64_t c, const void* x, int64_t ldx, int dtype, int fmt, uint8_t* codes,
                 uint8_t* scales, void* stream) {
  EF_TRY(check_sizes(n, c, 1));
  if (!dtype_ok(dtype) || !fmt_ok(fmt) || !mat_ok(x, n, c, ldx, dtype) || !kept_ok(codes, scales, n)) return EF_EINVAL;
  const Range q = range_kept(codes, n, c), s = range_scales(scales, n, c);
  if (meet(q, s) || meet_any(range(x, n, c, ldx, bytes_of(dtype)), q, s)) return EF_EINVAL;
  if (n == 0) return EF_OK;
  Flat f;
  EF_TRY(flat_of(n, c, &f));
  const Kept k{codes, scales, groups(c), fmt};
  if (dtype == EF_F32) EF_LAUNCH(k_ckpt_pack<EF_F32>, f.grid, dim3(256), 0, S(stream), n, (int32_t)c, x, ldx, k, f.txs);
  else EF_LAUNCH(k_ckpt_pack<EF_BF16>, f.grid, dim3(256), 0, S(stream), n, (int32_t)c, x, ldx, k, f.txs);
  return launched();
}

int ef_ckpt_unpack(int64_t n, int64_t c, const uint8_t* codes, const uint8_t* scales, int fmt, void* y, int64_t ldy,
                   int dtype, void* stream) {
  EF_TRY(check_sizes(n, c, 1));
  if (!dtype_ok(dtype) || !fmt_ok(fmt) || !mat_ok(y, n, c, ldy, dtype) || !kept_ok(codes, scales, n)) return EF_EINVAL;
  if (meet_any(range(y, n, c, ldy, bytes_of(dtype)), range_kept(codes, n, c), range_scales(scales, n, c)))
    return EF_EINVAL;
  if (n == 0) return EF_OK;
  Flat f;
  EF_TRY(flat_of(n, c, &f));
  const Kept k{const_cast<uint8_t*>(codes), const_cast<uint8_t*>(scales), groups(c), fmt};
  if (dtype == EF_F32)
    EF_LAUNCH((k_ckpt_unpack<EF_F32, false>), f.grid, dim3(256), 0, S(stream), n, (int32_t)c, 0, k, nullptr, (int64_t)0, y, ldy, f.txs);
  else
    EF_LAUNCH((k_ckpt_unpack<EF_BF16, false>), f.grid, dim3(256), 0, S(stream), n, (int32_t)c, 0, k, nullptr, (int64_t)0, y, ldy, f.txs);
  return launched();
}

int ef_ckpt_act_backward(int64_t n, int64_t c, int act, const uint8_t* codes, const uint8_t* scales, int fmt,
                         const void* dy, int64_t lddy, void* dz, int64_t lddz, int dtype, void* stream) {
  EF_TRY(check_sizes(n, c, 1));
  if (!dtype_ok(dtype) || !fmt_ok(fmt) || !act_ok(act) || !mat_ok(dy, n, c, lddy, dtype) ||
      !mat_ok(dz, n, c, lddz, dtype) || !kept_ok(codes, scales, n))
    return EF_EINVAL;
  const Range out = range(dz, n, c, lddz, bytes_of(dtype));
  if (meet_any(out, range_kept(codes, n, c), range_scales(scales, n, c))) return EF_EINVAL;
  if (meet(out, range(dy, n, c, lddy, bytes_of(dtype))) && !(dz == dy && lddz == lddy)) return EF_EINVAL;
  if (n == 0) return EF_OK;
  Flat f;
  EF_TRY(flat_of(n, c, &f));
  const Kept k{const_cast<uint8_t*>(codes), const_cast<uint8_t*>(scales), groups(c), fmt};
  if (dtype == EF_F32)
    EF_LAUNCH((k_ckpt_unpack<EF_F32, true>), f.grid, dim3(256), 0, S(stream), n, (int32_t)c, act, k, dy, lddy, dz, lddz, f.txs);
  else
    EF_LAUNCH((k_ckpt_unpack<EF_BF16, true>), f.grid, dim3(256), 0, S(stream), n, (int32_t)c, act, k, dy, lddy, dz, lddz, f.txs);
  return launched();
}

size_t ef_linear_workspace_bytes(int op, int64_t n, int64_t i, int64_t o, int dtype) {
  if (check_sizes(n, i, o) != EF_OK || !dtype_ok(dtype) || op < EF_OP_FORWARD || op > EF_OP_WGRAD) return 0;
  const int64_t M = op == EF_OP_WGRAD ? o : n, N = op == EF_OP_FORWARD ? o : i, K = op == EF_OP_FORWARD ? i : op == EF_OP_DGRAD ? o : n;
  return product_bytes(op == EF_OP_WGRAD, dtype, M, N, K);
}

int ef_linear_forward(int64_t n, int64_t i, int64_t o, const void* x, int64_t ldx, const void* w, int64_t ldw,
                      const void* bias, int act, const void* res, int64_t ldr, void* y, int64_t ldy, int dtype,
                      uint8_t* codes, uint8_t* scales, int fmt, void* ws, size_t ws_bytes, void* stream) {
  EF_TRY(check_sizes(n, i, o));
  if (!dtype_ok(dtype) || !act_ok(act) || !mat_ok(x, n, i, ldx, dtype) || !mat_ok(w, o, i, ldw, dtype) ||
      !mat_ok(y, n, o, ldy, dtype) || (bias && !aligned(bias, (size_t)bytes_of(dtype))) ||
      (res && !mat_ok(res, n, o, ldr, dtype)) || !codes != !scales)
    return EF_EINVAL;
  if (codes && (!fmt_ok(fmt) || !kept_ok(codes, scales, n))) return EF_EINVAL;
  const int64_t b = bytes_of(dtype);
  const Range out = range(y, n, o, ldy, b), rx = range(x, n, i, ldx, b), rw = range(w, o, i, ldw, b),
              rb = range(bias, 1, o, o, b), rr = range(res, n, o, ldr, b),
              q = codes ? range_kept(codes, n, o) : Range{nullptr, nullptr, 0, 0},
              s = codes ? range_scales(scales, n, o) : Range{nullptr, nullptr, 0, 0};
  if (meet_any(out, rx, rw, rb, q, s) || meet_any(q, s, rx, rw, rb, rr) || meet_any(s, rx, rw, rb, rr)) return EF_EINVAL;
  if (meet(out, rr) && !(res == y && ldr == ldy)) return EF_EINVAL;
  if (n == 0) return EF_OK;
  Product p{n, o, i, {x, ldx}, {w, ldw}, {}, {y, ldy, bias, res, ldr, {codes, scales, groups(o), fmt}, act, 0, nullptr}};
  return dtype == EF_F32 ? run_product<K_FWD, EF_F32, EF_F32>(p, ws, ws_bytes, S(stream), {out, rx, rw, rb, rr, q, s})
                         : run_product<K_FWD, EF_BF16, EF_BF16>(p, ws, ws_bytes, S(stream), {out, rx, rw, rb, rr, q, s});
}

int ef_linear_dgrad(int64_t n, int64_t i, int64_t o, const void* dy, int64_t lddy, const void* w, int64_t ldw, int act,
                    const uint8_t* codes, const uint8_t* scales, int fmt, const void* res, int64_t ldr, void* dx,
                    int64_t lddx, int dtype, void* ws, size_t ws_bytes, void* stream) {
  EF_TRY(check_sizes(n, i, o));
  if (!dtype_ok(dtype) || !act_ok(act) || !mat_ok(dy, n, o, lddy, dtype) || !mat_ok(w, o, i, ldw, dtype) ||
      !mat_ok(dx, n, i, lddx, dtype) || (res && !mat_ok(res, n, i, ldr, dtype)))
    return EF_EINVAL;
  const bool kept = act != EF_ACT_NONE;
  if (kept && (!fmt_ok(fmt) || !kept_ok(codes, scales, n))) return EF_EINVAL;
  const int64_t b = bytes_of(dtype);
  const Range out = range(dx, n, i, lddx, b), rr = range(res, n, i, ldr, b), ry = range(dy, n, o, lddy, b),
              rw = range(w, o, i, ldw, b), q = kept ? range_kept(codes, n, i) : Range{nullptr, nullptr, 0, 0},
              s = kept ? range_scales(scales, n, i) : Range{nullptr, nullptr, 0, 0};
  if (meet_any(out, ry, rw, q, s)) return EF_EINVAL;
  if (meet(out, rr) && !(res == dx && ldr == lddx)) return EF_EINVAL;
  if (n == 0) return EF_OK;
  Product p{n, i, o, {dy, lddy}, {w, ldw}, {},
            {dx, lddx, nullptr, res, ldr, {const_cast<uint8_t*>(codes), const_cast<uint8_t*>(scales), groups(i), fmt}, act, 0, nullptr}};
  return dtype == EF_F32 ? run_product<K_DGRAD, EF_F32, EF_F32>(p, ws, ws_bytes, S(stream), {out, ry, rw, rr, q, s})
                         : run_product<K_DGRAD, EF_BF16, EF_BF16>(p, ws, ws_bytes, S(stream), {out, ry, rw, rr, q, s});
}

int ef_linear_wgrad(int64_t n, int64_t i, int64_t o, const void* dy, int64_t lddy, int dtype, const uint8_t* codes,
                    const uint8_t* scales, int fmt, void* dw, void* db, int g_dtype, int accumulate, void* ws,
                    size_t ws_bytes, void* stream) {
  EF_TRY(check_sizes(n, i, o));
  if (!dtype_ok(dtype) || !dtype_ok(g_dtype) || !fmt_ok(fmt) || !mat_ok(dy, n, o, lddy, dtype) ||
      !kept_ok(codes, scales, n) || !dw || !aligned(dw, (size_t)bytes_of(g_dtype)) ||
      (db && !aligned(db, (size_t)bytes_of(g_dtype))) || (accumulate && g_dtype != EF_F32))
    return EF_EINVAL;
  const int64_t b = bytes_of(g_dtype);
  const Range rw = range(dw, o, i, i, b), rb = range(db, 1, o, o, b), ry = range(dy, n, o, lddy, bytes_of(dtype)),
              q = range_kept(codes, n, i), s = range_scales(scales, n, i);
  if (meet_any(rw, rb, ry, q, s) || meet_any(rb, ry, q, s)) return EF_EINVAL;
  hipStream_t st = S(stream);
  Product p{o, i, n, {dy, lddy}, {}, {const_cast<uint8_t*>(codes), const_cast<uint8_t*>(scales), groups(i), fmt},
            {dw, i, nullptr, nullptr, 0, {}, EF_ACT_NONE, accumulate ? 1 : 0, db}};
  if (dtype == EF_F32)
    return g_dtype == EF_F32 ? run_product<K_WGRAD, EF_F32, EF_F32>(p, ws, ws_bytes, st, {rw, rb, ry, q, s})
                             : run_product<K_WGRAD, EF_F32, EF_BF16>(p, ws, ws_bytes, st, {rw, rb, ry, q, s});
  return g_dtype == EF_F32 ? run_product<K_WGRAD, EF_BF16, EF_F32>(p, ws, ws_bytes, st, {rw, rb, ry, q, s})
                           : run_product<K_WGRAD, EF_BF16, EF_BF16>(p, ws, ws_bytes, st, {rw, rb, ry, q, s});
}

}  // extern "C"
