// The torch calls of the package: rotary.burst_rotary and burst_norm_rotary with their gradients, paged's calls, RingWalk's usual calls, and
// the differentiable call behind autograd.burst_attention: attention of a query slice against key/value
// chunks as one torch autograd node, in C++.  Argument marshalling and buffers only; every arithmetic
// step is a call into libburst.so (paper Alg. 1 forward, Alg. 2 backward).
// Why native: in Python the two halves of a call ran on two threads (autograd's backward thread is another
// one) and cost 200 us of host time at any size, several times the GPU time of a short sequence.
#include <torch/extension.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPGraphsC10Utils.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/functions/utils.h>

#include <cmath>
#include <mutex>
#include <optional>
#include <string>
#include <vector>

#include "../../include/burst.h"

namespace {

using torch::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

void check(int status, const char* where) {
  TORCH_CHECK(status == BURST_OK, where, ": ", burst_strerror(status), " (status ", status, ")");
}

// Whether the library can read a [B, H, rows, d] tensor where it lies: last dimension contiguous, the
// other strides and the base address multiples of 16 bytes, rows not overlapping.
bool addressable(const Tensor& t) {
  if (t.dim() != 4 || (t.size(3) != 1 && t.stride(3) != 1)) return false;
  if (reinterpret_cast<uintptr_t>(t.data_ptr()) % 16 != 0) return false;
  const int64_t unit = 16 / (int64_t)t.element_size();
  for (int i = 0; i < 3; i++)
    if (t.size(i) != 1 && (t.stride(i) <= 0 || t.stride(i) % unit != 0)) return false;
  return t.size(2) == 1 || t.stride(2) >= t.size(3);
}

// Strides for the parameter block; all zero for a contiguous tensor.  Dimensions of size 1 (whose stride
// addresses nothing) get the row length.
void set_strides(int64_t (&out)[3], const Tensor& t) {
  const bool dense = t.is_contiguous();
  for (int i = 0; i < 3; i++) out[i] = dense ? 0 : t.size(i) > 1 ? t.stride(i) : t.size(3);
}

// K and V of a chunk as they are if one set of strides addresses both, else contiguous copies.
void pair_in_place(Tensor& k, Tensor& v) {
  bool same = addressable(k) && addressable(v) && k.is_contiguous() == v.is_contiguous() && k.sizes() == v.sizes();
  for (int j = 0; j < 3 && same; j++) same = k.size(j) == 1 || k.stride(j) == v.stride(j);
  if (!same) { k = k.contiguous(); v = v.contiguous(); }
}

// t if it lies in memory like q, else a copy that does.
Tensor lying_like(const Tensor& t, const Tensor& q) {
  return t.strides() == q.strides() ? t : torch::empty_strided(q.sizes(), q.strides(), q.options()).copy_(t);
}

struct Call {                        // what forward and backward have in common
  burst_params p{};
  std::vector<burst_chunk> chunks;
};

// mask_of: for each chunk the place of its block flags in `masks`, -1 = none (empty: no chunk has any).
Call describe(const Tensor& q, const variable_list& ks, const variable_list& vs, const variable_list& masks,
              const std::vector<int64_t>& mask_of, double scale, bool causal, int64_t q_off, int64_t window, int64_t block) {
  Call c;
  burst_params& p = c.p;
  p.B = (int32_t)q.size(0); p.H = (int32_t)q.size(1); p.Nq = (int32_t)q.size(2); p.d = (int32_t)q.size(3);
  p.dtype = q.scalar_type() == torch::kBFloat16 ? BURST_BF16 : BURST_F32;
  p.causal = causal; p.scale = (float)scale; p.q_off = q_off; p.window = window; p.block = (int32_t)block;
  p.kv_heads = ks[0].size(1) != q.size(1) ? (int32_t)ks[0].size(1) : 0;
  set_strides(p.q_strides, q);
  int64_t at = 0;
  c.chunks.resize(ks.size());
  for (size_t i = 0; i < ks.size(); i++) {
    burst_chunk& k = c.chunks[i];
    k = burst_chunk{};
    k.K = ks[i].data_ptr(); k.V = vs[i].data_ptr();
    k.Nc = (int32_t)ks[i].size(2);
    k.k_off = at;
    at += ks[i].size(2);
    set_strides(k.kv_strides, ks[i]);
    if (!mask_of.empty() && mask_of[i] >= 0) {
      const Tensor& m = masks[mask_of[i]];
      const int64_t rows = (q.size(2) + block - 1) / block, cols = (ks[i].size(2) + block - 1) / block;
      const bool one = m.dim() == 2 && m.size(0) == rows && m.size(1) == cols;
      const bool each = m.dim() == 4 && m.size(0) == q.size(0) && m.size(1) == q.size(1) && m.size(2) == rows && m.size(3) == cols;
      TORCH_CHECK_VALUE(m.scalar_type() == torch::kByte && m.is_cuda() && m.is_contiguous(),
                        "block_mask: contiguous uint8 device tensor expected");
      TORCH_CHECK_VALUE(one || each, "block_mask: shape must be [ceil(Nq/block), ceil(Nc/block)], alone or after [B, H]");
      k.block_mask = m.data_ptr<uint8_t>();
      k.block_mask_stride = each ? rows * cols : 0;
    }
  }
  return c;
}

Tensor scratch(const Call& c, int flags, const Tensor& like) {
  const size_t need = burst_walk_workspace_bytes(c.chunks.data(), (int)c.chunks.size(), &c.p, flags);
  return need ? torch::empty({(int64_t)need}, like.options().dtype(torch::kByte)) : Tensor();
}
void* ptr(const Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
size_t bytes(const Tensor& t) { return t.defined() ? (size_t)t.nbytes() : 0; }
void* stream_of(const Tensor& t) { return (void*)c10::hip::getCurrentHIPStream(t.device().index()).stream(); }

// Gradients of a captured pass go to nodes of their own streams.  A leaf whose node was made by an earlier graph on the default stream, and lives because
// that graph does, has the engine make that stream wait for the captured one, which no capture allows and the process may not survive.  (On the
// device's guard.)
void refuse_outside_of_capture(const torch::autograd::Node& node, const char* what) {
  if (c10::hip::currentStreamCaptureStatusMayInitCtx() == c10::hip::CaptureStatus::None) return;
  for (size_t i = 0; i < node.num_outputs(); i++) {
    const auto& to = node.next_edge(i).function;
    if (to == nullptr || !node.task_should_compute_output(i)) continue;
    const auto stream = to->stream();
    TORCH_CHECK(!stream.has_value() || stream->id() != c10::hip::getDefaultHIPStream(stream->device_index()).id(), what,
                ": a captured backward pass whose gradients go to a graph that was made on the default stream and still lives (let it go before the capture, or "
                "make its tensors' graph in it)");
  }
}

class Attention : public torch::autograd::Function<Attention> {
 public:
  // kvm: the keys of n chunks, then their values, then the block flags of those that have some (mask_of)
  static variable_list forward(AutogradContext* ctx, const Tensor& q_in, at::TensorList kvm, int64_t n_chunks,
                               const std::vector<int64_t>& mask_of, double scale, bool causal, int64_t q_off, int64_t window,
                               int64_t block) {
    const c10::DeviceGuard on(q_in.device());     // the library launches on the current device
    const size_t n = (size_t)n_chunks;
    const Tensor q = addressable(q_in) ? q_in : q_in.contiguous();
    variable_list ks(kvm.begin(), kvm.begin() + n), vs(kvm.begin() + n, kvm.begin() + 2 * n), masks(kvm.begin() + 2 * n, kvm.end());
    for (size_t i = 0; i < n; i++) pair_in_place(ks[i], vs[i]);
    const Call c = describe(q, ks, vs, masks, mask_of, scale, causal, q_off, window, block);
    Tensor O = torch::empty_strided(q.sizes(), q.strides(), q.options());   // O lies in memory like Q
    Tensor lse = torch::empty({q.size(0), q.size(1), q.size(2)}, q.options().dtype(torch::kFloat));
    const Tensor ws = scratch(c, BURST_WALK_NO_STATE | BURST_WALK_FORWARD, q);
    check(burst_walk_fwd(q.data_ptr(), c.chunks.data(), (int)n, nullptr, nullptr, nullptr, O.data_ptr(), lse.data_ptr<float>(),
                         ptr(ws), bytes(ws), &c.p, stream_of(q)), "burst_walk_fwd");
    variable_list saved = {q, O, lse};
    for (auto* l : {&ks, &vs, &masks}) saved.insert(saved.end(), l->begin(), l->end());
    ctx->save_for_backward(saved);
    ctx->saved_data["n"] = (int64_t)n;
    ctx->saved_data["mask_of"] = mask_of;
    ctx->saved_data["scale"] = scale;
    ctx->saved_data["causal"] = causal;
    ctx->saved_data["q_off"] = q_off;
    ctx->saved_data["window"] = window;
    ctx->saved_data["block"] = block;
    ctx->mark_non_differentiable({lse});
    ctx->set_materialize_grads(false);            // (no zeros for the gradient of lse)
    return {O, lse};
  }

  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    const variable_list s = ctx->get_saved_variables();
    const size_t n = (size_t)ctx->saved_data["n"].toInt();
    variable_list out(1 + (s.size() - 3) + 7);    // q, kvm, and seven arguments that are no tensors
    if (!grads[0].defined()) return out;
    const c10::DeviceGuard on(s[0].device());
    if (const auto node = torch::autograd::get_current_node()) refuse_outside_of_capture(*node, "burst_attention");
    // Hooks on saved tensors may have returned each of them in another layout than it was saved in.
    const Tensor q = addressable(s[0]) ? s[0] : s[0].contiguous(), O = lying_like(s[1], q), lse = s[2].contiguous();
    variable_list ks(s.begin() + 3, s.begin() + 3 + n), vs(s.begin() + 3 + n, s.begin() + 3 + 2 * n), masks(s.begin() + 3 + 2 * n, s.end());
    for (size_t i = 0; i < n; i++) pair_in_place(ks[i], vs[i]);
    Call c = describe(q, ks, vs, masks, ctx->saved_data["mask_of"].toIntVector(), ctx->saved_data["scale"].toDouble(),
                      ctx->saved_data["causal"].toBool(), ctx->saved_data["q_off"].toInt(), ctx->saved_data["window"].toInt(),
                      ctx->saved_data["block"].toInt());
    const Tensor g = lying_like(grads[0].to(q.scalar_type()), q);
    Tensor D = torch::empty(lse.sizes(), lse.options()), dQ = torch::empty(q.sizes(), q.options());
    out[0] = dQ;
    for (size_t i = 0; i < n; i++) {
      out[1 + i] = torch::empty(ks[i].sizes(), ks[i].options());
      out[1 + n + i] = torch::empty(vs[i].sizes(), vs[i].options());
      c.chunks[i].dK = out[1 + i].data_ptr();
      c.chunks[i].dV = out[1 + n + i].data_ptr();
    }
    const Tensor ws = scratch(c, BURST_WALK_HALF_GRADS, q);
    check(burst_walk_bwd(q.data_ptr(), c.chunks.data(), (int)n, O.data_ptr(), g.data_ptr(), lse.data_ptr<float>(),
                         D.data_ptr<float>(), dQ.data_ptr(), 0, 0, 1, ptr(ws), bytes(ws), &c.p, stream_of(q)), "burst_walk_bwd");
    return out;
  }
};

std::vector<Tensor> attention(const Tensor& q, const std::vector<Tensor>& ks, const std::vector<Tensor>& vs,
                              const std::vector<std::optional<Tensor>>& masks, double scale, bool causal, int64_t q_off,
                              int64_t window, int64_t block) {
  TORCH_CHECK_VALUE(!ks.empty() && ks.size() == vs.size(), "one key and one value tensor per chunk, at least one chunk, expected");
  TORCH_CHECK_VALUE(masks.empty() || masks.size() == ks.size(), "one block mask per chunk expected");
  TORCH_CHECK_VALUE(q.dim() == 4 && (q.scalar_type() == torch::kBFloat16 || q.scalar_type() == torch::kFloat),
                    "q: [B, H, Nq, d] of bfloat16 or float32 expected");
  variable_list kvm(ks);
  kvm.insert(kvm.end(), vs.begin(), vs.end());
  for (size_t i = 0; i < ks.size(); i++)
    TORCH_CHECK_VALUE(ks[i].dim() == 4 && ks[i].sizes() == vs[i].sizes(), "the keys and values of a chunk: the same sizes expected");
  for (const Tensor& t : kvm) {
    TORCH_CHECK_VALUE(t.dim() == 4 && t.scalar_type() == q.scalar_type() && t.size(0) == q.size(0) && t.size(1) == ks[0].size(1) &&
                      t.size(3) == q.size(3), "keys and values: [B, Hkv, Nc, d] of the type of q expected");
    TORCH_CHECK_VALUE(t.is_cuda() && t.device() == q.device(), "tensors on one device expected");
  }
  std::vector<int64_t> mask_of;
  for (const auto& m : masks) {
    mask_of.push_back(m.has_value() ? (int64_t)(kvm.size() - 2 * ks.size()) : -1);
    if (m.has_value()) kvm.push_back(*m);
  }
  return Attention::apply(q, at::TensorList(kvm), (int64_t)ks.size(), mask_of, scale, causal, q_off, window, block);
}

// harness.RingWalk's two calls for tensors as they usually are: chunks that lie densely, of the walk's type and sizes and without
// block flags, state and statistics as the walk made them, a workspace that suffices, no capture.  kOther where something
// is not so, with nothing enqueued: the caller's own marshalling then sees to it, and to its errors.  (A pass over four chunks of 256
// rows spent more time in the interpreter than on the GPU: see RingWalk.)
constexpr int kOther = 1;
bool plain_f32(const Tensor& t, const Tensor& q) { return t.is_cuda() && t.device() == q.device() && t.scalar_type() == torch::kFloat && t.is_contiguous(); }
bool like_q(const Tensor& t, const Tensor& q) {
  return t.is_cuda() && t.device() == q.device() && t.scalar_type() == q.scalar_type() && t.sizes() == q.sizes() && t.strides() == q.strides();
}
bool usual(Call& c, const Tensor& q, const std::vector<Tensor>& ks, const std::vector<Tensor>& vs, const std::vector<int64_t>& k_offs, double scale,
           bool causal, int64_t q_off, int64_t window, int64_t kv_heads) {
  if (ks.empty() || vs.size() != ks.size() || k_offs.size() != ks.size() || q.dim() != 4 || !q.is_cuda() || q.numel() == 0) return false;
  if (q.scalar_type() != torch::kBFloat16 && q.scalar_type() != torch::kFloat) return false;
  // (not every stride of a view can go into the parameter block: all of them 0, as of an expanded row, means dense there)
  if (!(q.is_contiguous() || addressable(q)) || q.device().index() != c10::hip::current_device()) return false;
  if (c10::hip::currentStreamCaptureStatusMayInitCtx() != c10::hip::CaptureStatus::None) return false;
  const int64_t heads = kv_heads != 0 ? kv_heads : q.size(1);
  for (size_t i = 0; i < ks.size(); i++) {
    const Tensor &k = ks[i], &v = vs[i];
    if (!k.is_cuda() || !v.is_cuda() || k.device() != q.device() || v.device() != q.device() || k.scalar_type() != q.scalar_type() ||
        v.scalar_type() != q.scalar_type() || k.dim() != 4 || k.sizes() != v.sizes() || !k.is_contiguous() || !v.is_contiguous()) return false;
    if (k.size(0) != q.size(0) || k.size(1) != heads || k.size(3) != q.size(3) || k.size(2) > 0x7fffffff) return false;
  }
  c = describe(q, ks, vs, {}, {}, scale, causal, q_off, window, 0);
  c.p.kv_heads = (int32_t)kv_heads;
  for (size_t i = 0; i < ks.size(); i++) c.chunks[i].k_off = k_offs[i];
  return true;
}
// The walk's workspace, if the call needs one: false where it is too small or belongs to another stream.
bool suffices(const Call& c, int flags, const std::optional<Tensor>& ws, uint64_t ws_stream, void* stream, void*& at, size_t& bytes) {
  const size_t need = burst_walk_workspace_bytes(c.chunks.data(), (int)c.chunks.size(), &c.p, flags);
  at = nullptr; bytes = 0;
  if (need == 0) return true;
  if (!ws.has_value() || (size_t)ws->nbytes() < need || ws_stream != (uint64_t)stream) return false;
  at = ws->data_ptr(); bytes = (size_t)ws->nbytes();
  return true;
}

int walk_forward(const Tensor& q, const std::vector<Tensor>& ks, const std::vector<Tensor>& vs, const std::vector<int64_t>& k_offs, double scale,
                 bool causal, int64_t q_off, int64_t window, int64_t kv_heads, const Tensor& O_acc, const Tensor& m, const Tensor& l,
                 const Tensor& O, const Tensor& lse, const std::optional<Tensor>& ws, uint64_t ws_stream) {
  Call c;
  if (!usual(c, q, ks, vs, k_offs, scale, causal, q_off, window, kv_heads) || !like_q(O, q)) return kOther;
  for (const Tensor* t : {&O_acc, &m, &l, &lse}) if (!plain_f32(*t, q)) return kOther;
  void *at, *const stream = stream_of(q);
  size_t bytes;
  if (!suffices(c, BURST_WALK_FORWARD, ws, ws_stream, stream, at, bytes)) return kOther;
  return burst_walk_fwd(q.data_ptr(), c.chunks.data(), (int)ks.size(), O_acc.data_ptr<float>(), m.data_ptr<float>(), l.data_ptr<float>(),
                        O.data_ptr(), lse.data_ptr<float>(), at, bytes, &c.p, stream);
}

// dQ, dK, dV: new tensors, fp32.
std::tuple<int, Tensor, std::vector<Tensor>, std::vector<Tensor>> walk_backward(
    const Tensor& q, const std::vector<Tensor>& ks, const std::vector<Tensor>& vs, const std::vector<int64_t>& k_offs, double scale, bool causal,
    int64_t q_off, int64_t window, int64_t kv_heads, const Tensor& O, const Tensor& dO, const Tensor& lse, const Tensor& D,
    const std::optional<Tensor>& ws, uint64_t ws_stream) {
  Call c;
  Tensor dQ;
  std::vector<Tensor> dK, dV;
  void *at, *stream = nullptr;
  size_t bytes;
  if (!usual(c, q, ks, vs, k_offs, scale, causal, q_off, window, kv_heads) || !like_q(O, q) || !like_q(dO, q) || !plain_f32(lse, q) || !plain_f32(D, q) ||
      !suffices(c, 0, ws, ws_stream, stream = stream_of(q), at, bytes)) return {kOther, dQ, dK, dV};
  const auto f32 = q.options().dtype(torch::kFloat);
  try {
    dQ = torch::empty(q.sizes(), f32);
    for (size_t i = 0; i < ks.size(); i++) {
      dK.push_back(torch::empty(ks[i].sizes(), f32));
      dV.push_back(torch::empty(vs[i].sizes(), f32));
      c.chunks[i].dK = dK[i].data_ptr();
      c.chunks[i].dV = dV[i].data_ptr();
    }
  } catch (const c10::OutOfMemoryError&) {         // (raised again, as torch's own, by the caller's allocations)
    return {kOther, Tensor(), {}, {}};
  }
  const int st = burst_walk_bwd(q.data_ptr(), c.chunks.data(), (int)ks.size(), O.data_ptr(), dO.data_ptr(), lse.data_ptr<float>(), D.data_ptr<float>(),
                                dQ.data_ptr(), 0, 0, 0, at, bytes, &c.p, stream);
  return {st, dQ, dK, dV};
}

void fits_int(const Tensor& t) {
  for (const int64_t n : t.sizes()) TORCH_CHECK_VALUE(n <= 0x7fffffff, "sizes below 2^31 expected");
}
// These calls have no rule for tangents: results of a dual tensor would have none, which says that their derivatives are 0.
void refuse_tangent(const Tensor& t) {
  TORCH_CHECK_NOT_IMPLEMENTED(!t._fw_grad(0).defined(), "forward-mode derivatives are not implemented for this call: a tensor without a tangent expected");
}
// A caller's tensor that a call has written: graphs that saved it are told so.  (Inference tensors have no version; nothing can save them.)
void written(const Tensor& t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
// ---- rotary.burst_rotary: several tensors rotated by one call, and their gradients brought back by another.
bool rows_in_place(const Tensor& t) {              // strides that burst_rotate takes: all zero would mean dense ones
  if (t.size(3) != 1 && t.stride(3) != 1) return false;
  for (int i = 0; i < 3; i++) if (t.size(i) > 1 && t.stride(i) != 0) return true;
  return t.is_contiguous();
}
void check_turns(const Tensor& turns, int64_t d, const Tensor& like) {
  TORCH_CHECK_VALUE(turns.scalar_type() == torch::kDouble && turns.dim() == 1 && turns.is_contiguous() && turns.device() == like.device(),
                    "turns: contiguous float64 tensor [pairs] on the tensors' device expected");
  refuse_tangent(turns);
  TORCH_CHECK_VALUE(!turns.requires_grad(), "turns: a tensor that needs no gradient expected");
  TORCH_CHECK_VALUE(turns.numel() >= 1 && 2 * turns.numel() <= d, "turns: between one pair and all of the head's columns expected");
}
// The positions of x's rows as they are where their rows are contiguous, else a copy.
Tensor positions_for(const Tensor& p, const Tensor& x) {
  TORCH_CHECK_VALUE(p.scalar_type() == torch::kLong && p.device() == x.device() && (p.dim() == 1 || (p.dim() == 2 && p.size(0) == x.size(0))) &&
                    p.size(-1) == x.size(2), "positions: int64 [rows] or [B, rows] on the tensors' device expected");
  return p.size(-1) <= 1 || p.stride(-1) == 1 ? p : p.contiguous();
}
variable_list rotate_all(const variable_list& xs, const Tensor& turns, const variable_list& positions, const std::vector<int64_t>& position_of,
                         const std::vector<int64_t>& offsets, bool interleaved, double amplitude, bool inverse) {
  const Tensor& like = xs[0];
  const c10::DeviceGuard on(like.device());
  variable_list from, out;
  std::vector<burst_rows> items(xs.size());
  for (size_t i = 0; i < xs.size(); i++) {
    from.push_back(rows_in_place(xs[i]) ? xs[i] : xs[i].contiguous());
    const Tensor& x = from[i];
    out.push_back(torch::empty_like(x));           // lies in memory like x, without its gaps
    if (out[i].stride(3) != 1) out[i] = torch::empty(x.sizes(), x.options());   // (x has rows or heads one element apart: windows of a sequence)
    burst_rows& c = items[i];
    c = burst_rows{};
    c.x = x.data_ptr(); c.y = out[i].data_ptr();
    c.B = (int32_t)x.size(0); c.heads = (int32_t)x.size(1); c.rows = (int32_t)x.size(2);
    set_strides(c.x_strides, x);
    set_strides(c.y_strides, out[i]);
    c.offset = offsets[i];
    if (position_of[i] >= 0) {
      const Tensor& p = positions[position_of[i]];
      c.positions = p.data_ptr<int64_t>();
      c.positions_stride = p.dim() == 2 && p.size(0) > 1 ? p.stride(0) : 0;
    }
  }
  burst_rotary r{};
  r.turns = turns.data_ptr<double>(); r.dims = (int32_t)(2 * turns.numel()); r.interleaved = interleaved; r.amplitude = (float)amplitude; r.inverse = inverse;
  check(burst_rotate(items.data(), (int)items.size(), &r, (int)like.size(3), like.scalar_type() == torch::kBFloat16 ? BURST_BF16 : BURST_F32,
                     stream_of(like)), "burst_rotate");
  return out;
}
// What the rotation of some tensors is; position_of: for each tensor the place of its positions, -1 = none.
struct Turning {
  std::vector<int64_t> position_of, offsets;
  bool interleaved;
  double amplitude;
  bool inverse;
};
variable_list rotate_differentiably(const variable_list& xs, const Tensor& turns, const variable_list& positions, const Turning& how);
// (A node of its own instead of a torch::autograd::Function, whose saved values go through a dictionary: host us of a call on two tensors with
// its gradients 73 so, 69 here, of which two views with theirs take 54.)
struct RotateBackward : public torch::autograd::Node {
  torch::autograd::SavedVariable turns;
  std::vector<torch::autograd::SavedVariable> positions;
  Turning how;
  at::ScalarType type;
  variable_list apply(variable_list&& grads) override {
    const std::lock_guard<std::mutex> lock(mutex_);   // (threads that go back through one graph: another one's release_variables)
    variable_list out(grads.size()), some, where;
    Turning back{{}, {}, how.interleaved, how.amplitude, !how.inverse};
    std::vector<size_t> to;
    for (size_t i = 0; i < grads.size(); i++) {
      if (!grads[i].defined() || !task_should_compute_output(i)) continue;
      to.push_back(i);
      some.push_back(grads[i].scalar_type() == type ? grads[i] : grads[i].to(type));
      // (the engine gives gradients of the outputs' sizes; a caller of the node itself, what it likes)
      TORCH_CHECK_VALUE(some.back().dim() == 4 && some.back().size(3) == some[0].size(3) && some.back().device() == some[0].device(),
                        "gradients: [B, heads, rows, d] tensors of one d and device expected");
      back.position_of.push_back(how.position_of[i] >= 0 ? (int64_t)where.size() : -1);
      if (how.position_of[i] >= 0) where.push_back(positions_for(positions[how.position_of[i]].unpack(), some.back()));
      back.offsets.push_back(how.offsets[i]);
    }
    if (some.empty()) return out;
    const c10::DeviceGuard on(some[0].device());
    refuse_outside_of_capture(*this, "burst_rotary");
    const Tensor t = turns.unpack().contiguous();  // (hooks on saved tensors may return them in another layout than they were saved in)
    check_turns(t, some[0].size(3), some[0]);
    const variable_list g = rotate_differentiably(some, t, where, back);   // (create_graph: a rotation again)
    for (size_t k = 0; k < to.size(); k++) out[to[k]] = g[k];
    return out;
  }
  void release_variables() override {
    const std::lock_guard<std::mutex> lock(mutex_);
    turns.reset_data();
    for (auto& p : positions) p.reset_data();
  }
  std::string name() const override { return "BurstRotaryBackward"; }
};
variable_list rotate_differentiably(const variable_list& xs, const Tensor& turns, const variable_list& positions, const Turning& how) {
  for (const Tensor& x : xs) refuse_tangent(x);
  std::shared_ptr<RotateBackward> node;
  std::vector<size_t> wanted;                      // the tensors that need a gradient: the others, frozen keys say, are no part of the graph
  if (at::GradMode::is_enabled())
    for (size_t i = 0; i < xs.size(); i++)
      if (xs[i].requires_grad()) wanted.push_back(i);
  if (!wanted.empty()) {
    node = std::shared_ptr<RotateBackward>(new RotateBackward(), torch::autograd::deleteNode);
    node->how = Turning{{}, {}, how.interleaved, how.amplitude, how.inverse};
    for (const size_t i : wanted) {
      node->add_next_edge(torch::autograd::impl::gradient_edge(xs[i]));
      node->how.position_of.push_back(how.position_of[i] >= 0 ? (int64_t)node->positions.size() : -1);
      if (how.position_of[i] >= 0) node->positions.emplace_back(positions[how.position_of[i]], false);
      node->how.offsets.push_back(how.offsets[i]);
    }
    node->turns = torch::autograd::SavedVariable(turns, false);
    node->type = xs[0].scalar_type();
  }
  variable_list out;
  {
    const at::NoGradGuard no_grad;
    out = rotate_all(xs, turns, positions, how.position_of, how.offsets, how.interleaved, how.amplitude, how.inverse);
  }
  for (const size_t i : wanted) torch::autograd::set_history(out[i], node);
  return out;
}
std::vector<Tensor> rotate(const std::vector<Tensor>& xs, const Tensor& turns, const std::vector<int64_t>& offsets,
                           const std::vector<std::optional<Tensor>>& positions, bool interleaved, double amplitude) {
  TORCH_CHECK_VALUE(!xs.empty() && offsets.size() == xs.size() && positions.size() == xs.size(), "one offset and one entry of positions per tensor expected");
  for (const Tensor& x : xs)
    TORCH_CHECK_VALUE(x.dim() == 4 && x.is_cuda() && x.device() == xs[0].device() && x.scalar_type() == xs[0].scalar_type() && x.size(3) == xs[0].size(3) &&
                      (x.scalar_type() == torch::kBFloat16 || x.scalar_type() == torch::kFloat),
                      "[B, heads, rows, d] tensors of bfloat16 or float32, of one type, d and device, expected");
  for (const Tensor& x : xs) fits_int(x);
  check_turns(turns, xs[0].size(3), xs[0]);
  Turning how{{}, offsets, interleaved, amplitude, false};
  variable_list at;
  for (size_t i = 0; i < xs.size(); i++) {
    const auto& p = positions[i];
    how.position_of.push_back(p.has_value() ? (int64_t)at.size() : -1);
    if (!p.has_value()) continue;
    at.push_back(positions_for(*p, xs[i]));
  }
  return rotate_differentiably(xs, turns, at, how);
}

// ---- rotary.burst_norm_rotary: tensors normalised, weighted and rotated by one call, and all gradients by another.
struct Norming {
  std::vector<int64_t> weight_of, position_of, offsets;   // for each tensor: the place of its weight and of its positions, -1 = none
  bool rotated, interleaved;
  double amplitude, eps;
};
struct NormCall {                                  // what both of its calls take, and the tensors that it points into
  std::vector<burst_norm_rows> items;
  std::vector<burst_norm_weight> weights;
  variable_list holds;
  burst_rotary r{};
  const burst_rotary* rotary = nullptr;
  int d = 0, dtype = 0;
};
void set_rows(burst_rows& c, const Tensor& x, const Tensor& y, const Tensor* positions, int64_t offset) {
  c.x = x.data_ptr();
  set_strides(c.x_strides, x);
  c.B = (int32_t)x.size(0); c.heads = (int32_t)x.size(1); c.rows = (int32_t)x.size(2);
  if (y.defined()) {
    c.y = y.data_ptr();
    set_strides(c.y_strides, y);
  }
  c.offset = offset;
  if (positions != nullptr) {
    c.positions = positions->data_ptr<int64_t>();
    c.positions_stride = positions->dim() == 2 && positions->size(0) > 1 ? positions->stride(0) : 0;
  }
}
Tensor result_like(const Tensor& x) {              // lies in memory like x, without its gaps
  Tensor y = torch::empty_like(x);
  return y.stride(3) == 1 ? y : torch::empty(x.sizes(), x.options());   // (x has rows or heads one element apart: windows of a sequence)
}
void set_norm(NormCall& c, const Tensor& like, const variable_list& weights, const Tensor& turns, const Norming& how) {
  c.d = (int)like.size(3);
  c.dtype = like.scalar_type() == torch::kBFloat16 ? BURST_BF16 : BURST_F32;
  for (const Tensor& w : weights) {
    burst_norm_weight b{};
    b.w = w.data_ptr();
    b.f32 = w.scalar_type() == torch::kFloat;
    c.weights.push_back(b);
  }
  if (how.rotated) {
    c.r.turns = turns.data_ptr<double>(); c.r.dims = (int32_t)(2 * turns.numel()); c.r.interleaved = how.interleaved; c.r.amplitude = (float)how.amplitude;
    c.rotary = &c.r;
  }
}
void check_weight(const Tensor& w, const Tensor& like) {
  TORCH_CHECK_VALUE(w.dim() == 1 && w.size(0) == like.size(3) && w.device() == like.device() && (w.scalar_type() == like.scalar_type() || w.scalar_type() == torch::kFloat),
                    "weights: [d] on the tensors' device, of their type or float32, expected");
  refuse_tangent(w);
}
struct NormRotaryBackward : public torch::autograd::Node {
  std::vector<torch::autograd::SavedVariable> xs, weights, positions;
  torch::autograd::SavedVariable turns;
  Norming how;
  at::ScalarType type;
  variable_list apply(variable_list&& grads) override {
    const std::lock_guard<std::mutex> lock(mutex_);   // (threads that go back through one graph: another one's release_variables)
    const size_t n = xs.size();
    variable_list out(n + weights.size()), x(n), g(n), at(positions.size()), w;
    const Tensor* like = nullptr;
    for (size_t i = 0; i < n; i++) {
      if (!grads[i].defined()) continue;
      const int64_t k = how.weight_of[i];
      if (!task_should_compute_output(i) && !(k >= 0 && task_should_compute_output(n + k))) continue;
      x[i] = xs[i].unpack();
      g[i] = grads[i].scalar_type() == type ? grads[i] : grads[i].to(type);
      // (the engine gives gradients of the outputs' sizes; a caller of the node itself, what it likes.  So do hooks on saved tensors.)
      TORCH_CHECK_VALUE(x[i].dim() == 4 && x[i].scalar_type() == type && g[i].sizes() == x[i].sizes() && g[i].device() == x[i].device(),
                        "gradients and saved tensors: of the sizes and device of the call's tensors expected");
      if (like == nullptr) like = &x[i];
      TORCH_CHECK_VALUE(x[i].device() == like->device() && x[i].size(3) == like->size(3), "gradients and saved tensors: of one d and device expected");
    }
    if (like == nullptr) return out;
    const c10::DeviceGuard on(like->device());
    refuse_outside_of_capture(*this, "burst_norm_rotary");
    Tensor t;
    variable_list given(x);                        // (as they are part of a graph)
    given.insert(given.end(), g.begin(), g.end());
    {
      const at::NoGradGuard no_grad;
      for (auto& s : weights) {
        w.push_back(s.unpack().contiguous());
        check_weight(w.back(), *like);
        given.push_back(w.back());
      }
      if (how.rotated) {
        t = turns.unpack().contiguous();
        check_turns(t, like->size(3), *like);
      }
      NormCall c;
      set_norm(c, *like, w, t, how);
      std::vector<bool> fed(weights.size(), false);
      for (size_t i = 0; i < n; i++) {
        if (!g[i].defined()) continue;
        const Tensor from = rows_in_place(x[i]) ? x[i].detach() : x[i].contiguous(), grad = rows_in_place(g[i]) ? g[i].detach() : g[i].contiguous();
        Tensor p;
        if (how.position_of[i] >= 0) p = positions_for(positions[how.position_of[i]].unpack(), from);
        if (task_should_compute_output(i)) out[i] = result_like(from);
        burst_norm_rows b{};
        set_rows(b.rows, grad, out[i], p.defined() ? &p : nullptr, how.offsets[i]);
        b.from = from.data_ptr();
        set_strides(b.from_strides, from);
        b.weight = (int32_t)how.weight_of[i];
        if (b.weight >= 0) fed[b.weight] = true;
        c.items.push_back(b);
        c.holds.insert(c.holds.end(), {from, grad, p});
      }
      for (size_t k = 0; k < weights.size(); k++) {
        if (!fed[k] || !task_should_compute_output(n + k)) continue;
        out[n + k] = torch::empty(w[k].sizes(), w[k].options());
        c.weights[k].dw = out[n + k].data_ptr();
      }
      const size_t need = burst_norm_workspace_bytes(c.items.data(), (int)c.items.size(), c.weights.data(), (int)c.weights.size(), (float)how.eps, c.rotary, c.d, c.dtype);
      const Tensor ws = need ? torch::empty({(int64_t)need}, like->options().dtype(torch::kByte)) : Tensor();
      check(burst_norm_rotate_bwd(c.items.data(), (int)c.items.size(), c.weights.data(), (int)c.weights.size(), (float)how.eps, c.rotary, c.d, c.dtype, ptr(ws),
                                  bytes(ws), stream_of(*like)), "burst_norm_rotate_bwd");
    }
    if (at::GradMode::is_enabled()) {              // (create_graph: these gradients are right, theirs are not implemented)
      variable_list some;
      for (const Tensor& v : given) if (v.defined()) some.push_back(v);
      const auto end = std::make_shared<torch::autograd::Error>("burst_norm_rotary: gradients of its gradients are not implemented",
                                                                torch::autograd::collect_next_edges(some));
      for (Tensor& v : out) if (v.defined()) torch::autograd::set_history(v, end);
    }
    return out;
  }
  void release_variables() override {
    const std::lock_guard<std::mutex> lock(mutex_);
    turns.reset_data();
    for (auto* l : {&xs, &weights, &positions})
      for (auto& v : *l) v.reset_data();
  }
  std::string name() const override { return "BurstNormRotaryBackward"; }
};
std::vector<Tensor> norm_rotate(const std::vector<Tensor>& xs, const std::vector<Tensor>& weights_in, const std::vector<int64_t>& weight_of,
                                const std::optional<Tensor>& turns, double eps, const std::vector<int64_t>& offsets,
                                const std::vector<std::optional<Tensor>>& positions, bool interleaved, double amplitude) {
  TORCH_CHECK_VALUE(!xs.empty() && offsets.size() == xs.size() && positions.size() == xs.size() && weight_of.size() == xs.size(),
                    "one offset and one entry of weights and of positions per tensor expected");
  for (const Tensor& x : xs) {
    TORCH_CHECK_VALUE(x.dim() == 4 && x.is_cuda() && x.device() == xs[0].device() && x.scalar_type() == xs[0].scalar_type() && x.size(3) == xs[0].size(3) &&
                      (x.scalar_type() == torch::kBFloat16 || x.scalar_type() == torch::kFloat),
                      "[B, heads, rows, d] tensors of bfloat16 or float32, of one type, d and device, expected");
    fits_int(x);
    refuse_tangent(x);
  }
  TORCH_CHECK_VALUE(xs[0].size(3) >= 2, "at least two columns expected");
  TORCH_CHECK_VALUE(eps > 0 && std::isnormal((float)eps), "eps: positive, in fp32 2^-126 at least, expected");
  variable_list weights;
  for (const Tensor& w : weights_in) {
    check_weight(w, xs[0]);
    weights.push_back(w.is_contiguous() ? w : w.contiguous());   // (a copy that is part of the graph)
  }
  if (turns.has_value()) check_turns(*turns, xs[0].size(3), xs[0]);
  Norming how{weight_of, {}, offsets, turns.has_value(), interleaved, amplitude, eps};
  variable_list at;
  for (size_t i = 0; i < xs.size(); i++) {
    TORCH_CHECK_VALUE(weight_of[i] >= -1 && weight_of[i] < (int64_t)weights.size(), "weights: a place among them expected");
    const auto& p = positions[i];
    how.position_of.push_back(p.has_value() ? (int64_t)at.size() : -1);
    if (p.has_value()) at.push_back(positions_for(*p, xs[i]));
  }
  std::shared_ptr<NormRotaryBackward> node;
  std::vector<size_t> wanted;                      // the tensors that are part of a graph
  if (at::GradMode::is_enabled())
    for (size_t i = 0; i < xs.size(); i++)
      if (xs[i].requires_grad() || (weight_of[i] >= 0 && weights[weight_of[i]].requires_grad())) wanted.push_back(i);
  if (!wanted.empty()) {
    node = std::shared_ptr<NormRotaryBackward>(new NormRotaryBackward(), torch::autograd::deleteNode);
    node->how = Norming{{}, {}, {}, how.rotated, interleaved, amplitude, eps};
    for (const size_t i : wanted) {
      node->add_next_edge(torch::autograd::impl::gradient_edge(xs[i]));
      node->xs.emplace_back(xs[i], false);
      node->how.weight_of.push_back(how.weight_of[i]);
      node->how.position_of.push_back(how.position_of[i] >= 0 ? (int64_t)node->positions.size() : -1);
      if (how.position_of[i] >= 0) node->positions.emplace_back(at[how.position_of[i]], false);
      node->how.offsets.push_back(offsets[i]);
    }
    for (const Tensor& w : weights) {
      node->add_next_edge(torch::autograd::impl::gradient_edge(w));
      node->weights.emplace_back(w, false);
    }
    if (turns.has_value()) node->turns = torch::autograd::SavedVariable(*turns, false);
    node->type = xs[0].scalar_type();
  }
  variable_list out;
  {
    const at::NoGradGuard no_grad;
    const c10::DeviceGuard on(xs[0].device());
    NormCall c;
    set_norm(c, xs[0], weights, turns.has_value() ? *turns : Tensor(), how);
    for (size_t i = 0; i < xs.size(); i++) {
      const Tensor x = rows_in_place(xs[i]) ? xs[i] : xs[i].contiguous();
      out.push_back(result_like(x));
      burst_norm_rows b{};
      set_rows(b.rows, x, out[i], how.position_of[i] >= 0 ? &at[how.position_of[i]] : nullptr, offsets[i]);
      b.weight = (int32_t)weight_of[i];
      c.items.push_back(b);
      c.holds.push_back(x);
    }
    check(burst_norm_rotate(c.items.data(), (int)c.items.size(), c.weights.data(), (int)c.weights.size(), (float)eps, c.rotary, c.d, c.dtype,
                            stream_of(xs[0])), "burst_norm_rotate");
  }
  for (const size_t i : wanted) torch::autograd::set_history(out[i], node);
  return out;
}

// ---- paged: new tokens [rows, heads, d], pages [pages, kv_heads, page, d]
void check_tokens(const Tensor& t, const Tensor& k_pages, const char* what) {
  TORCH_CHECK_VALUE(t.dim() == 3 && t.device() == k_pages.device() && t.scalar_type() == k_pages.scalar_type() && t.size(2) == k_pages.size(3), what,
                    ": [rows, heads, d] of the type, device and d of the pages expected");
  fits_int(t);
  refuse_tangent(t);
  TORCH_CHECK_VALUE(!(at::GradMode::is_enabled() && t.requires_grad()), what, ": the paged calls have no gradient (call them under torch.no_grad)");
}
// A token tensor as it is where its strides can be handed on (unit: elements that they have to be multiples of), else a copy.
bool tokens_in_place(const Tensor& t, int64_t unit) {
  if (t.size(2) != 1 && t.stride(2) != 1) return false;
  if (reinterpret_cast<uintptr_t>(t.data_ptr()) % (unit * t.element_size()) != 0) return false;
  for (int i = 0; i < 2; i++)
    if (t.size(i) > 1 && (t.stride(i) <= 0 || t.stride(i) % unit != 0)) return false;
  return true;
}
void set_token_strides(int64_t (&out)[2], const Tensor& t) {
  out[0] = t.size(0) > 1 ? t.stride(0) : t.size(1) * t.size(2);
  out[1] = t.size(1) > 1 ? t.stride(1) : t.size(2);
}
// Whether the rows of a matrix can be handed on: contiguous, one behind the other (of an empty one they may have any strides).
bool rows_lie(const Tensor& t) { return t.numel() == 0 || ((t.size(1) <= 1 || t.stride(1) == 1) && (t.size(0) <= 1 || t.stride(0) >= t.size(1))); }
burst_paged_params describe_paged(const Tensor& k_pages, const Tensor& v_pages, const Tensor& table, const Tensor& lengths, const Tensor& starts) {
  TORCH_CHECK_VALUE(k_pages.dim() == 4 && k_pages.is_cuda() && (k_pages.scalar_type() == torch::kBFloat16 || k_pages.scalar_type() == torch::kFloat),
                    "k_pages: device tensor [pages, kv_heads, page, d] of bfloat16 or float32 expected");
  fits_int(k_pages);
  fits_int(table);
  refuse_tangent(k_pages);
  refuse_tangent(v_pages);
  TORCH_CHECK_VALUE(v_pages.scalar_type() == k_pages.scalar_type() && v_pages.device() == k_pages.device() && v_pages.sizes() == k_pages.sizes() &&
                    v_pages.strides() == k_pages.strides(), "v_pages: like k_pages in type, sizes and strides expected");
  TORCH_CHECK_VALUE(k_pages.size(3) == 1 || k_pages.stride(3) == 1, "pages: a contiguous last dimension expected");
  for (int i = 0; i < 3; i++)                      // (an expanded dimension has no place for more than one row, and strides of zero mean dense ones)
    TORCH_CHECK_VALUE(k_pages.size(i) <= 1 || k_pages.stride(i) >= k_pages.size(3), "pages: rows that lie in memory one after the other expected");
  for (const Tensor* t : {&table, &lengths, &starts})
    TORCH_CHECK_VALUE(t->scalar_type() == torch::kInt && t->device() == k_pages.device(), "table, lengths, starts: int32 tensors on the pages' device expected");
  TORCH_CHECK_VALUE(lengths.dim() == 1 && starts.dim() == 1 && starts.size(0) == lengths.size(0) + 1 && table.dim() == 2 && table.size(0) == lengths.size(0),
                    "table [sequences, width], lengths [sequences], starts [sequences + 1] expected");
  TORCH_CHECK_VALUE(lengths.is_contiguous() && starts.is_contiguous() && rows_lie(table), "lengths, starts and the table's rows: contiguous expected");
  burst_paged_params p{};
  p.sequences = (int32_t)lengths.size(0); p.kv_heads = (int32_t)k_pages.size(1); p.d = (int32_t)k_pages.size(3);
  p.dtype = k_pages.scalar_type() == torch::kBFloat16 ? BURST_BF16 : BURST_F32;
  p.pages = (int32_t)k_pages.size(0); p.page = (int32_t)k_pages.size(2); p.width = (int32_t)table.size(1);
  p.starts = starts.data_ptr<int>(); p.lengths = lengths.data_ptr<int>(); p.table = table.data_ptr<int>();
  p.table_stride = table.size(0) > 1 ? table.stride(0) : 0;
  for (int i = 0; i < 3; i++) p.page_strides[i] = k_pages.size(i) > 1 ? k_pages.stride(i) : i == 2 ? k_pages.size(3) : k_pages.size(2) * k_pages.size(3);
  p.scale = 1.f;
  return p;
}

std::optional<Tensor> cache_append(const Tensor& k_in, const Tensor& v_in, const Tensor& k_pages, const Tensor& v_pages, const Tensor& table,
                                   const Tensor& lengths, const Tensor& starts, const std::optional<Tensor>& q_in, const std::optional<Tensor>& turns,
                                   bool interleaved, double amplitude, const std::optional<Tensor>& offsets, const std::optional<Tensor>& q_norm,
                                   const std::optional<Tensor>& k_norm, double eps, const std::optional<Tensor>& slots, const std::optional<Tensor>& positions) {
  burst_paged_params p = describe_paged(k_pages, v_pages, table, lengths, starts);
  check_tokens(k_in, k_pages, "k");
  check_tokens(v_in, k_pages, "v");
  TORCH_CHECK_VALUE(k_in.size(1) == k_pages.size(1) && v_in.sizes() == k_in.sizes(), "k, v: [rows, kv_heads, d] expected");
  TORCH_CHECK_VALUE(!(at::GradMode::is_enabled() && (k_pages.requires_grad() || v_pages.requires_grad())), "pages that require a gradient are not written");
  if (turns.has_value()) check_turns(*turns, k_pages.size(3), k_pages);
  if (offsets.has_value())
    TORCH_CHECK_VALUE(offsets->scalar_type() == torch::kLong && offsets->device() == k_pages.device() && offsets->is_contiguous() &&
                      offsets->sizes() == lengths.sizes(), "offsets: contiguous int64 [sequences] on the pages' device expected");
  burst_store how{};
  bool told = false;                               // more than burst_cache_append can be told
  Tensor norms[2];
  for (int i = 0; i < 2; i++) {
    const auto& w = i ? k_norm : q_norm;
    if (!w.has_value()) continue;
    TORCH_CHECK_VALUE(w->dim() == 1 && w->size(0) == k_pages.size(3) && w->device() == k_pages.device() &&
                      (w->scalar_type() == k_pages.scalar_type() || w->scalar_type() == torch::kFloat),
                      "q_norm, k_norm: [d] on the pages' device, of their type or float32, expected");
    refuse_tangent(*w);
    TORCH_CHECK_VALUE(!(at::GradMode::is_enabled() && w->requires_grad()), "q_norm, k_norm: the paged calls have no gradient (call them under torch.no_grad)");
    TORCH_CHECK_VALUE(eps > 0 && std::isnormal((float)eps), "eps: positive, in fp32 2^-126 at least, expected");
    norms[i] = w->contiguous();
    (i ? how.k_weight : how.q_weight) = norms[i].data_ptr();
    (i ? how.k_weight_f32 : how.q_weight_f32) = w->scalar_type() == torch::kFloat;
    told = true;
  }
  how.eps = (float)eps;
  for (int i = 0; i < 2; i++) {
    const auto& at = i ? positions : slots;
    if (!at.has_value()) continue;
    TORCH_CHECK_VALUE(at->scalar_type() == torch::kLong && at->device() == k_pages.device() && at->is_contiguous() && at->dim() == 1 && at->size(0) == k_in.size(0),
                      "slots, positions: contiguous int64 [rows] on the pages' device expected");
    (i ? how.positions : how.slots) = at->data_ptr<int64_t>();
    told = true;
  }
  TORCH_CHECK_VALUE(!(positions.has_value() && offsets.has_value()), "positions say where the tokens are: no offsets expected");
  TORCH_CHECK_VALUE(!q_norm.has_value() || q_in.has_value(), "q_norm without q: there is nothing to do with it");
  how.offsets = offsets.has_value() ? offsets->data_ptr<int64_t>() : nullptr;
  const c10::DeviceGuard on(k_pages.device());
  Tensor k = k_in, v = v_in, q, out;
  if (!(tokens_in_place(k, 1) && tokens_in_place(v, 1)) || (k.size(0) > 1 && k.stride(0) != v.stride(0)) || (k.size(1) > 1 && k.stride(1) != v.stride(1))) {
    k = k.contiguous();
    v = v.contiguous();
  }
  p.rows = (int32_t)k.size(0);
  p.H = p.kv_heads;
  set_token_strides(p.kv_strides, k);
  if (q_in.has_value()) {
    TORCH_CHECK_VALUE(turns.has_value() || q_norm.has_value(), "q without turns: there is nothing to do to it");
    check_tokens(*q_in, k_pages, "q");
    TORCH_CHECK_VALUE(q_in->size(0) == k.size(0) && q_in->size(1) >= 1 && q_in->size(1) % k_pages.size(1) == 0, "q: [rows, H, d] with H a multiple of kv_heads expected");
    q = tokens_in_place(*q_in, 1) ? *q_in : q_in->contiguous();
    out = torch::empty(q.sizes(), q.options());
    p.H = (int32_t)q.size(1);
    set_token_strides(p.q_strides, q);
  }
  burst_rotary r{};
  if (turns.has_value()) {
    r.turns = turns->data_ptr<double>(); r.dims = (int32_t)(2 * turns->numel()); r.interleaved = interleaved; r.amplitude = (float)amplitude;
  }
  if (told)
    check(burst_cache_store(k.data_ptr(), v.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), ptr(q), ptr(out), &how, turns.has_value() ? &r : nullptr, &p,
                            stream_of(k_pages)), "burst_cache_store");
  else
    check(burst_cache_append(k.data_ptr(), v.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), ptr(q), ptr(out),
                             how.offsets, turns.has_value() ? &r : nullptr, &p, stream_of(k_pages)),
          "burst_cache_append");
  written(k_pages);
  written(v_pages);
  if (!q_in.has_value()) return std::nullopt;
  return out;
}

std::tuple<Tensor, Tensor> paged_attention(const Tensor& q_in, const Tensor& k_pages, const Tensor& v_pages, const Tensor& table, const Tensor& lengths,
                                           const Tensor& starts, double scale, bool causal, int64_t window, int64_t max_new,
                                           const std::optional<Tensor>& o_out, const std::optional<Tensor>& lse_out, bool full_p,
                                           const std::optional<Tensor>& tree) {
  burst_paged_params p = describe_paged(k_pages, v_pages, table, lengths, starts);
  check_tokens(q_in, k_pages, "q");
  TORCH_CHECK_VALUE(!(at::GradMode::is_enabled() && (k_pages.requires_grad() || v_pages.requires_grad())),
                    "pages that require a gradient: the paged calls have no gradient (call them under torch.no_grad)");
  TORCH_CHECK_VALUE(max_new >= 0 && max_new <= 0x7fffffff && window >= 0, "max_new, window: not negative expected");
  if (tree.has_value()) {
    TORCH_CHECK_VALUE(tree->scalar_type() == torch::kLong && tree->device() == k_pages.device() && tree->dim() == 2 && tree->size(0) == q_in.size(0) &&
                      tree->size(1) >= 1 && tree->size(1) <= 1 << 20 && rows_lie(*tree), "tree: int64 [rows, words] on the pages' device, its rows contiguous, expected");
    TORCH_CHECK_VALUE(causal, "tree: masks of a causal call expected");
  }
  const c10::DeviceGuard on(k_pages.device());
  const int64_t unit = 16 / (int64_t)q_in.element_size();
  const Tensor q = tokens_in_place(q_in, unit) ? q_in : q_in.contiguous();
  Tensor O, lse;
  if (o_out.has_value()) {
    O = *o_out;
    refuse_tangent(O);
    TORCH_CHECK_VALUE(O.device() == q.device() && O.sizes() == q.sizes() && (O.scalar_type() == q.scalar_type() || O.scalar_type() == torch::kFloat) &&
                      tokens_in_place(O, 16 / (int64_t)O.element_size()) && (p.dtype == BURST_F32 || O.scalar_type() == torch::kFloat || tokens_in_place(O, 8)),
                      "out: like q in sizes, of its type or float32, on 16-byte boundaries expected");
    TORCH_CHECK_VALUE(!O.requires_grad(), "out: a tensor that needs no gradient expected");
  } else {
    O = torch::empty(q.sizes(), q.options());
  }
  if (lse_out.has_value()) {
    lse = *lse_out;
    refuse_tangent(lse);
    TORCH_CHECK_VALUE(lse.device() == q.device() && lse.scalar_type() == torch::kFloat && lse.is_contiguous() && lse.dim() == 2 && lse.size(0) == q.size(0) &&
                      lse.size(1) == q.size(1), "lse: contiguous float32 [rows, H] expected");
    TORCH_CHECK_VALUE(!lse.requires_grad(), "lse: a tensor that needs no gradient expected");
  } else {
    lse = torch::empty({q.size(0), q.size(1)}, q.options().dtype(torch::kFloat));
  }
  p.rows = (int32_t)q.size(0); p.H = (int32_t)q.size(1);
  // No more rows than sequences, and nothing said about them: single tokens, as a step of serving has.  (us a call as if nothing were known / so:
  // 64 sequences of 16 to 16384 keys, 32 heads over 8, 147 / 128; 256 of 16 to 300 59 / 37; 32 over 2000, 32 heads, 201 / 190; 16 over 4096, fp32,
  // 177 / 110; 1 over 32768 36.3 / 36.4.)
  if (max_new == 0 && q.size(0) <= lengths.size(0)) max_new = 1;
  p.scale = (float)scale; p.causal = causal; p.window = window; p.max_new = (int32_t)max_new;
  p.out_f32 = O.scalar_type() == torch::kFloat;
  p.full_p = full_p;
  set_token_strides(p.q_strides, q);
  set_token_strides(p.o_strides, O);
  const size_t need = burst_paged_workspace_bytes(&p);
  const Tensor ws = need ? torch::empty({(int64_t)need}, q.options().dtype(torch::kByte)) : Tensor();
  if (tree.has_value())
    check(burst_paged_tree_fwd(q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), O.data_ptr(), lse.data_ptr<float>(), tree->data_ptr<int64_t>(),
                               (int)tree->size(1), tree->size(0) > 1 ? tree->stride(0) : 0, ptr(ws), bytes(ws), &p, stream_of(q)), "burst_paged_tree_fwd");
  else
    check(burst_paged_fwd(q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), O.data_ptr(), lse.data_ptr<float>(), ptr(ws), bytes(ws), &p, stream_of(q)),
          "burst_paged_fwd");
  if (o_out.has_value()) written(O);
  if (lse_out.has_value()) written(lse);
  return {O, lse};
}

std::tuple<Tensor, Tensor, Tensor, Tensor, std::optional<Tensor>> cache_plan(const Tensor& added, const Tensor& lengths, const Tensor& table, const Tensor& free_pages,
                                                                             const Tensor& free_count, int64_t page, int64_t rows,
                                                                             const std::optional<Tensor>& parents, int64_t words, int64_t window) {
  TORCH_CHECK_VALUE(table.is_cuda(), "table: device tensor expected");
  for (const Tensor* t : {&added, &lengths, &table, &free_pages, &free_count})
    TORCH_CHECK_VALUE(t->scalar_type() == torch::kInt && t->device() == table.device(), "new, lengths, table, free, count: int32 tensors on one device expected");
  TORCH_CHECK_VALUE(added.dim() == 1 && lengths.sizes() == added.sizes() && table.dim() == 2 && table.size(0) == added.size(0) && free_pages.dim() == 1 &&
                    free_count.numel() == 1, "new, lengths [sequences], table [sequences, width], free [pages], count [1] expected");
  TORCH_CHECK_VALUE(added.is_contiguous() && lengths.is_contiguous() && free_pages.is_contiguous() && rows_lie(table), "new, lengths, free and the table's rows: contiguous expected");
  fits_int(table);
  fits_int(free_pages);
  TORCH_CHECK_VALUE(added.size(0) <= 4096 && rows >= 0 && rows < 1 << 20, "at most 4096 sequences and 2^20 - 1 rows expected");
  TORCH_CHECK_VALUE(page >= 16 && page < 1 << 30, "page: a power of two from 16 on expected");
  // (tensors that are written must not be read as another: the same memory twice)
  for (const Tensor* t : {&added, &lengths, &free_count}) TORCH_CHECK_VALUE(t->numel() == 0 || (t->data_ptr() != table.data_ptr() && t->data_ptr() != free_pages.data_ptr()),
                                                                            "the table and the stack: memory of their own expected");
  TORCH_CHECK_VALUE(table.numel() == 0 || table.data_ptr() != free_pages.data_ptr(), "the table and the stack: memory of their own expected");
  if (parents.has_value()) {
    TORCH_CHECK_VALUE(parents->scalar_type() == torch::kInt && parents->device() == table.device() && parents->dim() == 2 && parents->size(0) == added.size(0) && rows_lie(*parents),
                      "parents: int32 [sequences, most] on the table's device, its rows contiguous, expected");
    fits_int(*parents);
    TORCH_CHECK_VALUE(parents->numel() == 0 || (parents->data_ptr() != table.data_ptr() && parents->data_ptr() != free_pages.data_ptr()),
                      "the table and the stack: memory of their own expected");
    TORCH_CHECK_VALUE(words >= 1 && words <= 1 << 20, "words: at least one expected");
    TORCH_CHECK_VALUE(window >= 0, "window: not negative expected");
  }
  const c10::DeviceGuard on(table.device());
  const auto i32 = table.options(), i64 = i32.dtype(torch::kLong);
  Tensor starts = torch::empty({added.size(0) + 1}, i32), totals = torch::empty({added.size(0)}, i32), slots = torch::empty({rows}, i64), positions = torch::empty({rows}, i64);
  std::optional<Tensor> tree;
  burst_plan p{};
  p.sequences = (int32_t)added.size(0); p.rows = (int32_t)rows; p.pages = (int32_t)free_pages.size(0); p.page = (int32_t)page; p.width = (int32_t)table.size(1);
  p.added = added.data_ptr<int>(); p.lengths = lengths.data_ptr<int>(); p.table = table.data_ptr<int>(); p.free_pages = free_pages.data_ptr<int>();
  p.free_count = free_count.data_ptr<int>();
  p.table_stride = table.size(0) > 1 ? table.stride(0) : 0;
  p.starts = starts.data_ptr<int>(); p.totals = totals.data_ptr<int>(); p.slots = slots.data_ptr<int64_t>(); p.positions = positions.data_ptr<int64_t>();
  if (parents.has_value()) {
    tree = torch::empty({rows, words}, i64);
    p.words = (int32_t)words; p.window = (int32_t)std::min<int64_t>(window, 0x7fffffff); p.most = (int32_t)parents->size(1); p.tree = tree->data_ptr<int64_t>();
    p.parents_stride = parents->size(0) > 1 ? parents->stride(0) : 0;
    static const int none = -1;                    // (not read: no columns, or no sequences)
    p.parents = parents->numel() > 0 ? parents->data_ptr<int>() : &none;
  }
  check(burst_cache_plan(&p, stream_of(table)), "burst_cache_plan");
  for (const Tensor* t : {&table, &free_pages, &free_count}) written(*t);
  return {starts, totals, slots, positions, tree};
}

Tensor cache_keep(const std::vector<Tensor>& k_pages, const std::vector<Tensor>& v_pages, const Tensor& table, const Tensor& lengths, const Tensor& starts,
                  const Tensor& kept, const Tensor& counts) {
  TORCH_CHECK_VALUE(!k_pages.empty() && k_pages.size() == v_pages.size(), "as many v_pages as k_pages, one at least, expected");
  burst_paged_params p = describe_paged(k_pages[0], v_pages[0], table, lengths, starts);
  std::vector<void*> pools;
  for (size_t i = 0; i < k_pages.size(); i++)
    for (const Tensor* t : {&k_pages[i], &v_pages[i]}) {
      TORCH_CHECK_VALUE(t->scalar_type() == k_pages[0].scalar_type() && t->device() == k_pages[0].device() && t->sizes() == k_pages[0].sizes() &&
                        t->strides() == k_pages[0].strides(), "all layers' pages: like the first one's in type, sizes and strides expected");
      refuse_tangent(*t);
      TORCH_CHECK_VALUE(!(at::GradMode::is_enabled() && t->requires_grad()), "pages that require a gradient are not written");
      for (void* other : pools) TORCH_CHECK_VALUE(t->numel() == 0 || other != t->data_ptr(), "pages: every layer's keys and values once expected");
      pools.push_back(t->data_ptr());
    }
  for (const Tensor* t : {&kept, &counts})
    TORCH_CHECK_VALUE(t->scalar_type() == torch::kInt && t->device() == table.device(), "kept, counts: int32 tensors on the pages' device expected");
  TORCH_CHECK_VALUE(kept.dim() == 2 && kept.size(0) == lengths.size(0) && counts.sizes() == lengths.sizes() && counts.is_contiguous() && rows_lie(kept),
                    "kept [sequences, most], its rows contiguous, counts [sequences] expected");
  fits_int(kept);
  const c10::DeviceGuard on(table.device());
  p.rows = (1 << 30) - 1;                          // (there are no token tensors)
  p.H = p.kv_heads;
  Tensor out = torch::empty(lengths.sizes(), lengths.options());
  check(burst_cache_keep(pools.data(), (int)pools.size(), kept.data_ptr<int>(), kept.size(0) > 1 ? kept.stride(0) : 0, (int)kept.size(1), counts.data_ptr<int>(),
                         out.data_ptr<int>(), &p, stream_of(table)), "burst_cache_keep");
  for (const auto* l : {&k_pages, &v_pages})
    for (const Tensor& t : *l) written(t);
  return out;
}

}  // namespace

PYBIND11_MODULE(TORCH_EXTENSION_NAME, m) {
  m.def("attention", &attention, pybind11::call_guard<pybind11::gil_scoped_release>());
  m.def("norm_rotate", &norm_rotate, pybind11::call_guard<pybind11::gil_scoped_release>());
  m.def("rotate", &rotate, pybind11::call_guard<pybind11::gil_scoped_release>());
  m.def("cache_append", &cache_append, pybind11::call_guard<pybind11::gil_scoped_release>());
  m.def("cache_plan", &cache_plan, pybind11::call_guard<pybind11::gil_scoped_release>());
  m.def("cache_keep", &cache_keep, pybind11::call_guard<pybind11::gil_scoped_release>());
  m.def("paged_attention", &paged_attention, pybind11::call_guard<pybind11::gil_scoped_release>());
  m.def("walk_forward", &walk_forward, pybind11::call_guard<pybind11::gil_scoped_release>());
  m.def("walk_backward", &walk_backward, pybind11::call_guard<pybind11::gil_scoped_release>());
}
