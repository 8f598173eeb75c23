// C entry points of the operators around the attention: argument checks and launches
// (csrc/norm.cu, csrc/rope.cu).  The forward and backward with rotary positions are in csrc/moga_api.cu.
#include <initializer_list>

#include "moga_internal.cuh"

using namespace moga;

namespace {

constexpr size_t kMaxRowBytes = 32768;   // of a normed row

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

struct Span {
  const void* p;
  size_t bytes;
};
bool overlaps(const Span& a, const Span& b) {
  if (a.p == nullptr || b.p == nullptr || a.bytes == 0 || b.bytes == 0) return false;
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return x < y + b.bytes && y < x + a.bytes;
}
// out is apart from every other tensor
bool apart(const Span& out, std::initializer_list<Span> others) {
  for (const Span& o : others)
    if (overlaps(out, o)) return false;
  return true;
}
// the outputs are apart from each other and from the inputs
bool outputs_apart(std::initializer_list<Span> out, std::initializer_list<Span> in) {
  for (const Span* a = out.begin(); a != out.end(); ++a) {
    if (!apart(*a, in)) return false;
    for (const Span* b = a + 1; b != out.end(); ++b)
      if (overlaps(*a, *b)) return false;
  }
  return true;
}
// out is the same tensor as `in` or apart from it
bool same_or_apart(const Span& out, std::initializer_list<Span> in) {
  for (const Span& i : in)
    if (out.p != i.p && overlaps(out, i)) return false;
  return true;
}

size_t token_bytes(const moga_shape& s) { return elem_size(s.dtype) * (size_t)s.B * s.N * s.C; }

bool check_norm(const moga_shape* s, const moga_norm* n, moga_status* st) {
  if (!check_shape(s, st)) return false;
  if (n == nullptr || !(n->eps > 0.f) || n->eps > 3.0e38f || (n->per_batch != 0 && n->per_batch != 1)) {
    *st = MOGA_ERR_INVALID_ARG;
    return false;
  }
  if ((size_t)s->C * elem_size(s->dtype) > kMaxRowBytes || (long long)s->B * s->N >= (1ll << 31)) {
    *st = MOGA_ERR_UNSUPPORTED;
    return false;
  }
  return true;
}
bool check_dropout(const moga_dropout* d) {
  return d != nullptr && d->p >= 0.0 && d->p < 1.0 && (reinterpret_cast<uintptr_t>(d->step) & 7u) == 0;
}
Span step_span(const moga_dropout* d) { return {d != nullptr ? d->step : nullptr, sizeof(uint64_t)}; }
size_t param_bytes(const moga_shape& s, const moga_norm& n) { return sizeof(float) * (size_t)s.C * (n.per_batch ? s.B : 1); }

// Extent of the [B, H, N, D] tensor of the shape's strides.
size_t head_bytes(const moga_shape& s) {
  const Strides d = qkv_strides(s);
  return elem_size(s.dtype) * (size_t)((long long)(s.B - 1) * d.b + (long long)(s.H - 1) * d.h + (long long)(s.N - 1) * d.n + s.D);
}
Span position_span(const moga_shape& s, const moga_rope_plan& rope, const int32_t* pos, int32_t pos_per_batch) {
  return {pos, sizeof(int32_t) * (size_t)(pos_per_batch ? s.B : 1) * s.N * rope.n_axes};
}
// The axes of the shape's strides, the longest stride first.
void descending_axes(const moga_shape& s, long long (&stride)[3], long long (&size)[3]) {
  const Strides d = qkv_strides(s);
  stride[0] = d.b, stride[1] = d.h, stride[2] = d.n;
  size[0] = s.B, size[1] = s.H, size[2] = s.N;
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 3; ++j)
      if (stride[j] > stride[i]) {
        const long long t = stride[i], u = size[i];
        stride[i] = stride[j], size[i] = size[j];
        stride[j] = t, size[j] = u;
      }
}
// Whether the contiguous tensor c shares bytes with a row of the [B, H, N, D] tensor at a (so it may lie in the gaps
// between rows, or behind the tokens of a padded batch item).  A row starts at a sum of i stride over the axes and meets c
// if that lies in (lo, hi).  Axis by axis: a multiple of the stride inside (lo, hi) is such a row, all other indexes 0; else
// only the last multiple at or below lo has rows that can reach it, as the axes inside a stride extend over less than it.
// Where they extend over more (rows that share bytes, which inputs may have) the whole extent counts.
bool touches(const moga_shape& s, const void* a, const Span& c) {
  if (!overlaps({a, head_bytes(s)}, c)) return false;
  const long long es = (long long)elem_size(s.dtype);
  long long stride[3], size[3], lo = (long long)(reinterpret_cast<uintptr_t>(c.p) - reinterpret_cast<uintptr_t>(a)) - s.D * es, hi = lo + s.D * es + (long long)c.bytes;
  descending_axes(s, stride, size);
  for (int i = 0; i < 3; ++i) {
    if (size[i] == 1 || stride[i] == 0) continue;
    long long inner = 0;
    for (int j = i + 1; j < 3; ++j) inner += (size[j] - 1) * stride[j];
    if (inner >= stride[i]) return true;
    const long long step = stride[i] * es, below = lo < 0 ? -1 : lo / step, next = below + 1;   // below: at or below lo
    if (next < size[i] && next * step < hi) return true;
    if (below < 0) return false;                  // lo < 0 and no row starts before hi
    const long long q = below < size[i] ? below : size[i] - 1;
    lo -= q * step, hi -= q * step;
  }
  return lo < 0 && hi > 0;
}
bool any_touches(const moga_shape& s, std::initializer_list<const void*> rows, std::initializer_list<Span> whole) {
  for (const void* a : rows)
    for (const Span& c : whole)
      if (touches(s, a, c)) return true;
  return false;
}
// Whether a row of the [B, H, N, D] tensor at a shares bytes with a row of the one at b, both with the shape's
// strides (whose own rows are apart): tensors may lie in one another's gaps, as Q, K and V do in the output of
// one projection.  With delta elements between them it asks for i_b, i_h, i_n with |delta - sum i stride| < D; the
// axes inside a stride reach less far than it, so each leaves two candidates.
bool rows_meet(const moga_shape& s, const void* a, const void* b) {
  if (a == nullptr || b == nullptr) return false;
  const long long bytes = (long long)(reinterpret_cast<uintptr_t>(b) - reinterpret_cast<uintptr_t>(a));
  const long long es = (long long)elem_size(s.dtype), delta = bytes >= 0 ? bytes / es : -(-bytes / es);
  long long stride[3], size[3];
  descending_axes(s, stride, size);
  for (int pick = 0; pick < 8; ++pick) {
    long long left = delta;
    bool inside = true;
    for (int i = 0; i < 3 && inside; ++i) {
      if (size[i] == 1) continue;
      const long long down = left / stride[i] - (left % stride[i] < 0 ? 1 : 0), q = down + (pick >> i & 1);
      inside = q > -size[i] && q < size[i];
      left -= q * stride[i];
    }
    if (inside && left > -s.D && left < s.D) return true;
  }
  return false;
}

moga_status zero_params(const moga_shape& s, const moga_norm& n, float* dW, float* dbias, cudaStream_t cs) {
  if (dW != nullptr) MOGA_CUDA_OK(cudaMemsetAsync(dW, 0, param_bytes(s, n), cs));
  if (dbias != nullptr) MOGA_CUDA_OK(cudaMemsetAsync(dbias, 0, param_bytes(s, n), cs));
  return MOGA_OK;
}

moga_status norm_forward(const moga_shape* s, const moga_norm* n, const moga_dropout* d, const void* X, const void* R,
                         const float* W, const float* bias, void* Hs, void* Y, float* mean, float* rstd, bool residual,
                         void* stream) {
  moga_status st;
  if (!check_norm(s, n, &st)) return st;
  if (d != nullptr && !check_dropout(d)) return MOGA_ERR_INVALID_ARG;
  if (s->N == 0) return MOGA_OK;
  if (!PTR_OK(X) || !PTR_OK(Y) || (residual && (!PTR_OK(R) || !PTR_OK(Hs))) || !aligned16(W) || !aligned16(bias) ||
      !aligned4(mean) || !aligned4(rstd))
    return MOGA_ERR_INVALID_ARG;
  const size_t t = token_bytes(*s), p = param_bytes(*s, *n), r = sizeof(float) * (size_t)s->B * s->N;
  const Span x{X, t}, res{R, t}, h{Hs, t}, y{Y, t}, w{W, p}, b{bias, p}, m{mean, r}, v{rstd, r}, step = step_span(d);
  if (!same_or_apart(y, {x, res}) || !same_or_apart(h, {x, res}) || !apart(y, {h, w, b, m, v}) || !apart(h, {w, b, m, v}) ||
      !apart(m, {x, res, w, b, v}) || !apart(v, {x, res, w, b}) || !apart(step, {h, y, m, v}))
    return MOGA_ERR_INVALID_ARG;
  return launch_norm(*s, *n, d, X, R, W, bias, Hs, Y, mean, rstd, static_cast<cudaStream_t>(stream));
}

moga_status norm_backward(const moga_shape* s, const moga_norm* n, const moga_dropout* d, const void* X, const float* W,
                          const float* mean, const float* rstd, const void* dY, const void* dH, void* dX, void* dR,
                          float* dW, float* dbias, bool residual, void* ws, size_t ws_bytes, void* stream) {
  moga_status st;
  if (!check_norm(s, n, &st)) return st;
  if (d != nullptr && !check_dropout(d)) return MOGA_ERR_INVALID_ARG;
  if (!aligned4(dW) || !aligned4(dbias)) return MOGA_ERR_INVALID_ARG;
  cudaStream_t cs = static_cast<cudaStream_t>(stream);
  if (s->N == 0) return zero_params(*s, *n, dW, dbias, cs);
  if (!PTR_OK(X) || !PTR_OK(dY) || !PTR_OK(dX) || mean == nullptr || rstd == nullptr || !aligned4(mean) ||
      !aligned4(rstd) || !aligned16(W) || !aligned16(dH) || (residual && !PTR_OK(dR)))
    return MOGA_ERR_INVALID_ARG;
  const size_t t = token_bytes(*s), p = param_bytes(*s, *n), r = sizeof(float) * (size_t)s->B * s->N;
  const size_t need = norm_backward_bytes(*s, *n);
  const Span x{X, t}, dy{dY, t}, dh{dH, t}, dx{dX, t}, dr{dR, t}, w{W, p}, gw{dW, p}, gb{dbias, p}, m{mean, r}, v{rstd, r},
      scratch{ws, need};
  if (!same_or_apart(dx, {x, dy, dh}) || !same_or_apart(dr, {x, dy, dh}) || !apart(dx, {dr, w, gw, gb, m, v, scratch}) ||
      !apart(dr, {w, gw, gb, m, v, scratch}) || !apart(gw, {x, dy, dh, w, gb, m, v, scratch}) ||
      !apart(gb, {x, dy, dh, w, m, v, scratch}) || !apart(scratch, {x, dy, dh, w, m, v}) ||
      !apart(step_span(d), {dx, dr, gw, gb, scratch}))
    return MOGA_ERR_INVALID_ARG;
  if (!check_ws(ws, ws_bytes, need, &st)) return st;
  return launch_norm_backward(*s, *n, d, X, W, mean, rstd, dY, dH, dX, dR, dW, dbias, static_cast<char*>(ws), cs);
}

}  // namespace

namespace moga {

bool check_rope(const moga_shape& s, const moga_rope_plan* rope, const int32_t* pos, int32_t pos_per_batch,
                moga_status* st) {
  *st = MOGA_ERR_INVALID_ARG;
  if (rope == nullptr || rope->n_axes < 1 || rope->n_axes > 3 || rope->pairs < 1 ||
      (rope->layout != MOGA_ROPE_INTERLEAVED && rope->layout != MOGA_ROPE_HALF) ||
      rope->axis_pairs[0] < 0 || rope->axis_pairs[1] < 0 || rope->axis_pairs[2] < 0 || !aligned4(pos) ||
      (pos_per_batch != 0 && pos_per_batch != 1) || (pos == nullptr && rope->n_axes > 1 && rope->grid_w < 1) ||
      (pos == nullptr && rope->n_axes > 2 && rope->grid_h < 1))
    return false;
  if (rope->pairs > 64 || 2 * rope->pairs > s.D) {
    *st = MOGA_ERR_UNSUPPORTED;
    return false;
  }
  *st = MOGA_OK;
  return true;
}

// Whether no two rows of the [B, H, N, D] tensor of the shape's strides share bytes (for outputs).
bool rows_apart(const moga_shape& s) {
  if (s.N == 0) return true;
  const Strides d = qkv_strides(s);
  long long stride[3] = {d.b, d.h, d.n}, size[3] = {s.B, s.H, s.N};
  for (int i = 0; i < 3; ++i)                     // ascending strides; axes of one element do not count
    for (int j = i + 1; j < 3; ++j)
      if (stride[j] < stride[i]) {
        const long long t = stride[i], u = size[i];
        stride[i] = stride[j], size[i] = size[j];
        stride[j] = t, size[j] = u;
      }
  long long reach = s.D;                          // elements that the axes so far extend over
  for (int i = 0; i < 3; ++i) {
    if (size[i] == 1) continue;
    if (stride[i] < reach) return false;
    reach += (size[i] - 1) * stride[i];
  }
  return true;
}

// The outputs of the rotating gather, its workspace among them, are apart from each other and from its inputs.
bool permute_rope_apart(const moga_shape& s, const moga_rope_plan& rope, const int32_t* pos, int32_t pos_per_batch,
                        const int32_t* gid, const void* Q, const void* K, const void* V, const int32_t* perm,
                        const int32_t* inv, const int32_t* offsets, const void* Qp, const void* Kp, const void* Vp,
                        const void* ws) {
  const size_t a = (size_t)s.B * s.N * s.k, u = elem_size(s.dtype) * a * s.H * s.D, ints = sizeof(int32_t) * a;
  const Span p{perm, ints}, i{inv, ints}, f{offsets, sizeof(int32_t) * (size_t)s.B * (s.M + 1)}, q{Qp, u}, k{Kp, u}, v{Vp, u},
      w{ws, ws_layout(s).scratch_end};
  return outputs_apart({p, i, f, q, k, v, w}, {{gid, ints}, position_span(s, rope, pos, pos_per_batch)}) &&
         !any_touches(s, {Q, K, V}, {p, i, f, q, k, v, w});
}

// The outputs of the forward with rotary positions, its workspace among them, are apart from each other and from its
// inputs; rows of O may lie between rows of Q, K and V.
bool forward_rope_apart(const moga_shape& s, const moga_rope_plan& rope, const int32_t* pos, int32_t pos_per_batch,
                        const void* X, const float* Wr, const float* bias, const void* Q, const void* K, const void* V,
                        const void* O, const int32_t* gid, const float* gate, const int32_t* perm, const int32_t* offsets,
                        const void* ws) {
  const size_t words = 4 * (size_t)s.B * s.N * s.k;
  const Span g{gid, words}, a{gate, words}, p{perm, words}, f{offsets, sizeof(int32_t) * (size_t)s.B * (s.M + 1)}, w{ws, ws_layout(s).total},
      x{X, token_bytes(s)}, wr{Wr, sizeof(float) * (size_t)s.C * s.M}, b{bias, sizeof(float) * (size_t)s.M},
      at = position_span(s, rope, pos, pos_per_batch);
  return outputs_apart({g, a, p, f, w}, {x, wr, b, at}) && !any_touches(s, {Q, K, V, O}, {g, a, p, f, w}) &&
         !any_touches(s, {O}, {x, wr, b, at}) && !rows_meet(s, O, Q) && !rows_meet(s, O, K) && !rows_meet(s, O, V);
}

// The same for the backward with rotary positions (ws_need: the bytes of its workspace); rows of dQ, dK, dV and dO may lie
// between one another.
bool backward_rope_apart(const moga_shape& s, const moga_rope_plan& rope, const int32_t* pos, int32_t pos_per_batch,
                         const void* Qp, const void* Kp, const void* Vp, const void* Op, const float* lse,
                         const float* gate, const int32_t* perm, const int32_t* inv, const int32_t* offsets,
                         const void* dO, const void* dQ, const void* dK, const void* dV, const float* dgate,
                         const void* ws, size_t ws_need) {
  const size_t a = (size_t)s.B * s.N * s.k, u = elem_size(s.dtype) * a * s.H * s.D;
  const std::initializer_list<Span> in = {{Qp, u}, {Kp, u}, {Vp, u}, {Op, u}, {lse, sizeof(float) * a * s.H}, {gate, 4 * a}, {perm, 4 * a},
                                          {inv, 4 * a}, {offsets, sizeof(int32_t) * (size_t)s.B * (s.M + 1)},
                                          position_span(s, rope, pos, pos_per_batch)};
  const Span g{dgate, 4 * a}, w{ws, ws_need};
  const void* out[3] = {dQ, dK, dV};
  if (!outputs_apart({g, w}, in) || any_touches(s, {dO, dQ, dK, dV}, {g, w}) || any_touches(s, {dQ, dK, dV}, in)) return false;
  for (int j = 0; j < 3; ++j)
    if (rows_meet(s, out[j], dO) || rows_meet(s, out[j], out[(j + 1) % 3])) return false;
  return true;
}

}  // namespace moga

extern "C" {

moga_status moga_layernorm(const moga_shape* s, const moga_norm* n, const void* X, const float* W, const float* bias,
                           void* Y, float* mean, float* rstd, void* stream) {
  return norm_forward(s, n, nullptr, X, nullptr, W, bias, nullptr, Y, mean, rstd, false, stream);
}

size_t moga_layernorm_backward_workspace_bytes(const moga_shape* s, const moga_norm* n) {
  moga_status st;
  return check_norm(s, n, &st) ? norm_backward_bytes(*s, *n) : 0;
}

moga_status moga_layernorm_backward(const moga_shape* s, const moga_norm* n, const void* X, const float* W,
                                    const float* mean, const float* rstd, const void* dY, void* dX, float* dW,
                                    float* dbias, void* ws, size_t ws_bytes, void* stream) {
  return norm_backward(s, n, nullptr, X, W, mean, rstd, dY, nullptr, dX, nullptr, dW, dbias, false, ws, ws_bytes, stream);
}

moga_status moga_dropout_add(const moga_shape* s, const moga_dropout* d, const void* X, const void* R, void* Y,
                             void* stream) {
  moga_status st;
  if (!check_shape(s, &st)) return st;
  if (!check_dropout(d)) return MOGA_ERR_INVALID_ARG;
  if (s->N == 0) return MOGA_OK;
  const size_t t = token_bytes(*s);
  if (!PTR_OK(X) || !PTR_OK(Y) || !aligned16(R) || !same_or_apart({Y, t}, {{X, t}, {R, t}}) || overlaps({Y, t}, step_span(d)))
    return MOGA_ERR_INVALID_ARG;
  return launch_dropout(*s, *d, X, R, Y, static_cast<cudaStream_t>(stream));
}

moga_status moga_residual_norm(const moga_shape* s, const moga_norm* n, const moga_dropout* d, const void* X,
                               const void* R, const float* W, const float* bias, void* Hs, void* Y, float* mean,
                               float* rstd, void* stream) {
  return norm_forward(s, n, d, X, R, W, bias, Hs, Y, mean, rstd, true, stream);
}

moga_status moga_residual_norm_backward(const moga_shape* s, const moga_norm* n, const moga_dropout* d,
                                        const void* Hs, const float* W, const float* mean, const float* rstd,
                                        const void* dY, const void* dH, void* dX, void* dR, float* dW, float* dbias,
                                        void* ws, size_t ws_bytes, void* stream) {
  return norm_backward(s, n, d, Hs, W, mean, rstd, dY, dH, dX, dR, dW, dbias, true, ws, ws_bytes, stream);
}

moga_status moga_rope_build(const moga_rope_config* c, moga_rope_plan* out) {
  if (c == nullptr || out == nullptr) return MOGA_ERR_INVALID_ARG;
  return rope_build(*c, out);
}

moga_status moga_rope(const moga_shape* s, const moga_rope_plan* rope, const int32_t* pos, int32_t pos_per_batch,
                      const void* Q, const void* K, void* Qo, void* Ko, int32_t transpose, void* stream) {
  moga_status st;
  if (!check_shape(s, &st) || !check_rope(*s, rope, pos, pos_per_batch, &st)) return st;
  if (s->N == 0) return MOGA_OK;
  if (!PTR_OK(Q) || !PTR_OK(Qo) || (K == nullptr) != (Ko == nullptr) || !aligned16(K) || !aligned16(Ko) || !rows_apart(*s))
    return MOGA_ERR_INVALID_ARG;
  const Span p = position_span(*s, *rope, pos, pos_per_batch);
  if ((Qo != Q && rows_meet(*s, Qo, Q)) || (Ko != K && rows_meet(*s, Ko, K)) || rows_meet(*s, Qo, K) || rows_meet(*s, Qo, Ko) ||
      rows_meet(*s, Ko, Q) || any_touches(*s, {Qo, Ko}, {p}))
    return MOGA_ERR_INVALID_ARG;
  return launch_rope(*s, *rope, pos, pos_per_batch, Q, K, Qo, Ko, transpose != 0, static_cast<cudaStream_t>(stream));
}

moga_status moga_permute_rope_backward(const moga_shape* s, const moga_rope_plan* rope, const int32_t* pos,
                                       int32_t pos_per_batch, const void* dQp, const void* dKp, const void* dVp,
                                       const int32_t* inv, void* dQ, void* dK, void* dV, void* stream) {
  moga_status st;
  if (!check_shape(s, &st) || !check_rope(*s, rope, pos, pos_per_batch, &st)) return st;
  if (s->N == 0) return MOGA_OK;
  if (!PTR_OK(dQp) || !PTR_OK(dKp) || !PTR_OK(dVp) || !PTR_OK(inv) || !PTR_OK(dQ) || !PTR_OK(dK) || !PTR_OK(dV) ||
      !rows_apart(*s))
    return MOGA_ERR_INVALID_ARG;
  const size_t T = (size_t)s->N * s->k, u = elem_size(s->dtype) * (size_t)s->B * s->H * T * s->D;
  if (any_touches(*s, {dQ, dK, dV}, {{dQp, u}, {dKp, u}, {dVp, u}, {inv, sizeof(int32_t) * (size_t)s->B * T}, position_span(*s, *rope, pos, pos_per_batch)}) ||
      rows_meet(*s, dQ, dK) || rows_meet(*s, dK, dV) || rows_meet(*s, dV, dQ))
    return MOGA_ERR_INVALID_ARG;
  return launch_rope_ungather(*s, *rope, pos, pos_per_batch, dQp, dKp, dVp, inv, dQ, dK, dV,
                              static_cast<cudaStream_t>(stream));
}

}  // extern "C"
