// The gated projections of a feed-forward block, forward and backward, and the
// per-language weight gradient of a linear layer (include/bkmoo.h): argument
// checks, the choice of tiles, and the pass that turns dh into da and db.  The
// products are tile_gemm.cuh's.
#include "gate_few.cuh"
#include "tile_host.cuh"

namespace bkmoo {
namespace {

bool act_ok(int32_t act) { return act == BKMOO_SILU || act == BKMOO_GELU || act == BKMOO_GELU_TANH; }
int32_t up(int64_t n, int64_t by) { return (int32_t)((n + by - 1) / by); }

struct SlopeArgs {
  const __nv_bfloat16 *dh, *a, *b;
  __nv_bfloat16 *da, *db;
  int64_t ld_dh, ld_ab, ld_d;
  int64_t rows;
  int32_t cols, act;
};

__device__ __forceinline__ void slope8(const uint4& xh, const uint4& xa, const uint4& xb, int act,
                                       uint4* da, uint4* db) {
  const uint32_t h[4] = {xh.x, xh.y, xh.z, xh.w}, u[4] = {xa.x, xa.y, xa.z, xa.w},
                 v[4] = {xb.x, xb.y, xb.z, xb.w};
  uint32_t oa[4], ob[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    auto wide = [](uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); };
    float2 f, df;
    activation_slope2(act, wide(u[j]), &f, &df);
    const float2 g = wide(h[j]), x = __fmul2_rn(__fmul2_rn(g, wide(v[j])), df), y = __fmul2_rn(g, f);
    oa[j] = pack_bf16(x.x, x.y);
    ob[j] = pack_bf16(y.x, y.y);
  }
  *da = make_uint4(oa[0], oa[1], oa[2], oa[3]);
  *db = make_uint4(ob[0], ob[1], ob[2], ob[3]);
}
// da = dh b act'(a), db = dh act(a).  Bound by memory: 10 bytes an element, in
// vectors of 8 (one thread one vector; the last of a row element by element).
// The products behind it take bf16 operands, so da and db are rounded to bf16
// here, once, from fp32.  8192 x 8192 99 us, 6.8 TB/s
// (1216 CTAs that stay, of which 912 fit at a time, 109).  (Done inside the products'
// kernel instead, by the warps that wait for its first tiles, row by row ahead of
// them, it takes 140 us and slows the products beside it: 8192 rows 2048 -> 8192
// backward 751 us so, 724 in turn.)
__global__ void __launch_bounds__(256) gate_slope_kernel(const SlopeArgs p) {
  grid_wait();
  const int64_t per = (p.cols + 7) / 8, n = p.rows * per;
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n;
       i += (int64_t)gridDim.x * blockDim.x) {
    const int64_t row = n < (1ll << 32) ? (uint32_t)i / (uint32_t)per : i / per;
    const int col = (int)(i - row * per) * 8;
    const __nv_bfloat16 *dh = p.dh + row * p.ld_dh + col, *a = p.a + row * p.ld_ab + col,
                        *b = p.b + row * p.ld_ab + col;
    __nv_bfloat16 *da = p.da + row * p.ld_d + col, *db = p.db + row * p.ld_d + col;
    if (col + 8 <= p.cols) {
      // (not by the read-only path: the kernel may begin before the one that writes dh has ended)
      slope8(*reinterpret_cast<const uint4*>(dh), *reinterpret_cast<const uint4*>(a),
             *reinterpret_cast<const uint4*>(b), p.act, reinterpret_cast<uint4*>(da),
             reinterpret_cast<uint4*>(db));
    } else {
      for (int j = 0; col + j < p.cols; ++j) {
        float f, d;
        const float h = __bfloat162float(dh[j]);
        activation_slope(p.act, __bfloat162float(a[j]), &f, &d);
        da[j] = __float2bfloat16_rn(h * __bfloat162float(b[j]) * d);
        db[j] = __float2bfloat16_rn(h * f);
      }
    }
  }
}

// What does not depend on the tiles' shape of dW_k = dy_k^T x_k for one or two dy
// (mats), every language.  *any: there is something to write.
int weight_args(TileArgs<kWeight>& p, const void* const* dy, int64_t ld_dy, int mats, const void* x,
                int64_t ldx, int64_t M, int64_t N, int32_t K, const int64_t* rows,
                void* const* const* dw, int32_t dw_dtype, int32_t accumulate, bool* any) {
  const int elem = dw_dtype == BKMOO_F32 ? 4 : 2;
  *any = false;
  for (int k = 0; k < K; ++k) {
    const int64_t n = rows[k + 1] - rows[k], at = rows[k];
    p.nkt[k] = up(n, kTileK);
    int j = k;                                  // insertion by falling length
    while (j > 0 && p.nkt[p.order[j - 1]] < p.nkt[k]) p.order[j] = p.order[j - 1], --j;
    p.order[j] = k;
    for (int i = 0; i < mats; ++i) {
      p.out[i * kMaxK + k] = dw[i][k];
      p.vec[i * kMaxK + k] = store_width(dw[i][k], N, elem);
    }
    *any = *any || n > 0 || !accumulate;
    if (n == 0) continue;
    int r = tile_map(&p.b[k], static_cast<const __nv_bfloat16*>(x) + at * ldx, n, N, ldx, kTileK);
    for (int i = 0; i < mats && r == BKMOO_OK; ++i)
      r = tile_map(&p.a[i * kMaxK + k], static_cast<const __nv_bfloat16*>(dy[i]) + at * ld_dy, n, M,
                   ld_dy, kTileK);
    if (r != BKMOO_OK) return r;
  }
  p.rows = (int32_t)M;
  p.cols = (int32_t)N;
  p.mats = mats;
  p.n_lang = K;
  p.out_dtype = dw_dtype;
  p.accumulate = accumulate;
  return BKMOO_OK;
}
int weight_mode(const TileArgs<kWeight>& p) {
  bool whole = p.cols % 32 == 0;
  for (int k = 0; k < p.n_lang; ++k)
    for (int i = 0; i < p.mats; ++i) whole = whole && p.vec[i * kMaxK + k] >= 16;
  if (p.out_dtype == BKMOO_F32)
    return whole ? (p.accumulate ? kSumsAdded : kSums) : p.accumulate ? kSumsTurnedAdded : kSumsTurned;
  return !whole ? kTurned : p.accumulate ? kAdded : kPlain;
}
void weight_tiles(TileArgs<kWeight>& p, TileShape shape) {
  p.tiles_m = up(p.rows, kTileM * shape.cg);
  p.tiles_n = up(p.cols, shape.bn);
  p.tiles = p.tiles_m * p.tiles_n * p.mats * p.n_lang;
}

bool grads_ok(void* const* dw, int32_t K, int32_t dtype) {
  if (!dw) return false;
  for (int k = 0; k < K; ++k)
    if (!dw[k] || ((uintptr_t)dw[k] & (dtype == BKMOO_F32 ? 3u : 1u))) return false;
  return true;
}

}  // namespace
}  // namespace bkmoo

using namespace bkmoo;

extern "C" int bkmoo_gate_forward(const void* x, int64_t ldx, const void* w_gate, const void* w_up,
                                  int64_t ldw, int64_t T, int64_t D, int64_t F, int32_t act,
                                  void* h, int64_t ldh, void* a, void* b, int64_t ld_ab,
                                  void* stream) {
  if (!act_ok(act) || !operand_ok(w_gate, F, D, ldw) || !operand_ok(w_up, F, D, ldw) || T < 0 ||
      (a == nullptr) != (b == nullptr))
    return BKMOO_ERR_INVALID;
  if (T == 0) return BKMOO_OK;
  if (!operand_ok(x, T, D, ldx) || (!h && !a) || (h && !operand_ok(h, T, F, ldh)) ||
      (a && (!operand_ok(a, T, F, ld_ab) || !operand_ok(b, T, F, ld_ab))))
    return BKMOO_ERR_INVALID;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int sms = 0, r = tile_sms(&sms);
  if (r != BKMOO_OK) return r;
  if (few_rows(T, D, F)) {
    const FewArgs q = {static_cast<const __nv_bfloat16*>(x), static_cast<const __nv_bfloat16*>(w_gate),
                       static_cast<const __nv_bfloat16*>(w_up), static_cast<__nv_bfloat16*>(h),
                       static_cast<__nv_bfloat16*>(a), static_cast<__nv_bfloat16*>(b), ldx, ldw, ldh,
                       ld_ab, (int32_t)T, (int32_t)D, (int32_t)F, act};
    return launch_gate_few(q, sms, s) == cudaSuccess ? BKMOO_OK : BKMOO_ERR_CUDA;
  }
  const int32_t nkt = up(D, kTileK);
  const TileShape shape = tile_shape({T, F, true, &nkt, 1, 1}, nullptr, kPlain, sms, nullptr);
  TileArgs<kGate> p = {};
  r = tile_status_word(s, &p.status);
  if (r == BKMOO_OK) r = tile_map(&p.a, x, T, D, ldx, kTileM);
  if (r == BKMOO_OK) r = tile_map(&p.b[0], w_gate, F, D, ldw, shape.bn / 2);
  if (r == BKMOO_OK) r = tile_map(&p.b[1], w_up, F, D, ldw, shape.bn / 2);
  if (r != BKMOO_OK) return r;
  p.out[0] = {h, ldh, store_width(h, ldh, 2)};
  p.out[1] = {a, ld_ab, store_width(a, ld_ab, 2)};
  p.out[2] = {b, ld_ab, store_width(b, ld_ab, 2)};
  p.rows = (int32_t)T;
  p.cols = (int32_t)F;
  p.tiles_m = up(T, kTileM * shape.cg);
  p.tiles_n = up(F, shape.bn / 2);
  p.nkt = nkt;
  p.act = act;
  p.tiles = p.tiles_m * p.tiles_n;
  return tile_launch(tile_gate_fn(shape.cg, shape.bn), shape, &p, p.tiles, s);
}

extern "C" int bkmoo_gate_backward_workspace_size(int64_t T, int64_t F, size_t* bytes) {
  if (!bytes || T < 0 || F < 1) return BKMOO_ERR_INVALID;
  *bytes = 2 * align256((size_t)T * (size_t)((F + 7) / 8 * 8) * 2);
  return BKMOO_OK;
}

extern "C" int bkmoo_gate_backward(const void* dh, int64_t ld_dh, const void* a, const void* b,
                                   int64_t ld_ab, const void* x, int64_t ldx, const void* w_gate,
                                   const void* w_up, int64_t ldw, int64_t T, int64_t D, int64_t F,
                                   int32_t act, int32_t K, const int64_t* rows, void* dx,
                                   int64_t ld_dx, void* const* dw_gate, void* const* dw_up,
                                   int32_t dw_dtype, int32_t accumulate, void* ws, size_t ws_bytes,
                                   void* stream) {
  const bool weights = dw_gate || dw_up;
  if (!act_ok(act) || T < 0 || (dw_dtype != BKMOO_F32 && dw_dtype != BKMOO_BF16) ||
      !operand_ok(w_gate, F, D, ldw) || !operand_ok(w_up, F, D, ldw) || !size_ok(F, D) ||
      !languages_ok(rows, K, T) ||
      (!dx && !weights && T > 0) ||
      (weights && (!grads_ok(dw_gate, K, dw_dtype) || !grads_ok(dw_up, K, dw_dtype))))
    return BKMOO_ERR_INVALID;
  size_t need = 0;
  if (T > 0 && (!operand_ok(dh, T, F, ld_dh) || !operand_ok(a, T, F, ld_ab) ||
                !operand_ok(b, T, F, ld_ab) || !operand_ok(x, T, D, ldx) ||
                (dx && !operand_ok(dx, T, D, ld_dx)) || !ws || ((uintptr_t)ws & 255u) ||
                bkmoo_gate_backward_workspace_size(T, F, &need) != BKMOO_OK))
    return BKMOO_ERR_INVALID;
  if (ws_bytes < need) return BKMOO_ERR_WORKSPACE;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int32_t* status = nullptr;
  int sms = 0, r = tile_sms(&sms);
  if (r == BKMOO_OK) r = tile_status_word(s, &status);
  if (r != BKMOO_OK) return r;
  const int64_t ld = (F + 7) / 8 * 8;
  __nv_bfloat16* d[2] = {static_cast<__nv_bfloat16*>(ws), static_cast<__nv_bfloat16*>(ws) + need / 4};
  if (T > 0) {
    SlopeArgs q = {static_cast<const __nv_bfloat16*>(dh), static_cast<const __nv_bfloat16*>(a),
                   static_cast<const __nv_bfloat16*>(b), d[0], d[1], ld_dh, ld_ab, ld, T, (int32_t)F, act};
    const int64_t blocks = (T * (ld / 8) + 255) / 256, most = 1 << 30;
    void* list[] = {&q};
    if (launch_behind((const void*)gate_slope_kernel, dim3((unsigned)(blocks < most ? blocks : most)),
                      dim3(256), list, 0, s, true) != cudaSuccess)
      return BKMOO_ERR_CUDA;
  }
  // both products in one launch, or the one that is wanted
  TileArgs<kBoth> p = {};
  p.status = status;
  bool any = false;
  if (weights) {
    const void* dy[2] = {d[0], d[1]};
    void* const* dw[2] = {dw_gate, dw_up};
    r = weight_args(p.w, dy, ld, 2, x, ldx, F, D, K, rows, dw, dw_dtype, accumulate, &any);
    if (r != BKMOO_OK) return r;
  }
  const bool input = dx && T > 0;
  if (!input && !any) return BKMOO_OK;
  const int32_t nkt = 2 * up(F, kTileK);
  const TileSet in = {T, D, false, &nkt, 1, 1}, w = {F, D, false, p.w.nkt, K, 2};
  const int mode = any ? weight_mode(p.w) : kPlain;
  const TileShape shape = input ? tile_shape(in, any ? &w : nullptr, mode, sms, &p.head_start)
                                : tile_shape(w, nullptr, mode, sms, nullptr);
  if (any) weight_tiles(p.w, shape);
  if (input) {
    const void* m[2] = {w_gate, w_up};
    for (int i = 0; i < 2 && r == BKMOO_OK; ++i) {
      r = tile_map(&p.in.a[i], d[i], T, F, ld, kTileM);
      if (r == BKMOO_OK) r = tile_map(&p.in.b[i], m[i], F, D, ldw, kTileK);
    }
    if (r != BKMOO_OK) return r;
    p.in.out = {dx, ld_dx, store_width(dx, ld_dx, 2)};
    p.in.rows = (int32_t)T;
    p.in.cols = (int32_t)D;
    p.in.tiles_m = up(T, kTileM * shape.cg);
    p.in.tiles_n = up(D, shape.bn);
    p.in.nkt = nkt / 2;
    p.in.tiles = p.in.tiles_m * p.in.tiles_n;
  }
  return tile_launch(tile_both_fn(shape.cg, shape.bn, mode), shape, &p,
                     (int64_t)p.in.tiles + p.w.tiles, s);
}

extern "C" int bkmoo_language_wgrad(const void* dy, int64_t ld_dy, const void* x, int64_t ldx,
                                    int64_t T, int64_t M, int64_t N, int32_t K, const int64_t* rows,
                                    void* const* dw, int32_t dw_dtype, int32_t accumulate,
                                    void* stream) {
  if (T < 0 || !size_ok(M, N) || !languages_ok(rows, K, T) ||
      (dw_dtype != BKMOO_F32 && dw_dtype != BKMOO_BF16) || !grads_ok(dw, K, dw_dtype) ||
      (T > 0 && (!operand_ok(dy, T, M, ld_dy) || !operand_ok(x, T, N, ldx))))
    return BKMOO_ERR_INVALID;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int32_t* status = nullptr;
  int sms = 0, r = tile_sms(&sms);
  if (r == BKMOO_OK) r = tile_status_word(s, &status);
  if (r != BKMOO_OK) return r;
  TileArgs<kWeight> p = {};
  p.status = status;
  bool any = false;
  r = weight_args(p, &dy, ld_dy, 1, x, ldx, M, N, K, rows, &dw, dw_dtype, accumulate, &any);
  if (r != BKMOO_OK || !any) return r;
  const int mode = weight_mode(p);
  const TileShape shape = tile_shape({M, N, false, p.nkt, K, 1}, nullptr, mode, sms, nullptr);
  weight_tiles(p, shape);
  return tile_launch(tile_weight_fn(shape.cg, shape.bn, mode), shape, &p, p.tiles, s);
}

// (Nothing is read or written but the status word: no operand is copied, and the warps that
// write results wait for a sum that never comes.)
extern "C" int bkmoo_selftest_give_up(int32_t what, void* stream) {
  if (what < 0 || what > 2) return BKMOO_ERR_INVALID;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  TileArgs<kGate> p = {};
  const int r = tile_status_word(s, &p.status);
  if (r != BKMOO_OK) return r;
  if (what == 0) return launch_wait_runs_out(p.status, s);
  const TileShape shape = {what, 256};
  p.rows = kTileM * what;
  p.cols = 128;
  p.tiles = p.tiles_m = p.tiles_n = p.nkt = p.withhold = 1;
  return tile_launch(tile_gate_fn(shape.cg, shape.bn), shape, &p, 1, s);
}
