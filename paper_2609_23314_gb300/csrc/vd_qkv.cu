// vd_qkv.cu -- vd_qkv_norm_rope (include/vd.h): from the projection rows of new
// tokens to the queries and to the new rows of one layer, in one pass (vd_qkv.cuh).
//
// Bound by DRAM for prompts (16384 tokens of 48 heads of 128 values 69.4 us, 86 % of the copy
// peak; 82.5 without the early load of the next head), by launch and latency for single
// tokens (4.2 us in a graph).
#include <cuda_runtime.h>

#include <cstdint>

#include "vd_host.cuh"
#include "vd_qkv.cuh"

namespace vd {

namespace {

struct NewRowsArgs {
  const int32_t* pos_first_new;
  uint16_t *k_new, *v_new;
  int layer, n_layer;
};

struct NewRows {  // rows of [n_seq][n_layer][n_kv_head][B][head_dim]
  const QkvArgs& a;
  const NewRowsArgs& n;
  size_t* new_row;  // a token's row of the new rows' first head

  __device__ void place(int t, int tok) const {
    new_row[t] = ((size_t)(tok / a.B) * n.n_layer + n.layer) * a.n_kv * a.B + tok % a.B;
  }
  __device__ long long position(int tok) const {
    return (long long)n.pos_first_new[tok / a.B] + tok % a.B;
  }
  static constexpr bool kRows = true;
  __device__ uint16_t* row(int t, int kh, bool key) const {
    return (key ? n.k_new : n.v_new) + (new_row[t] + (size_t)kh * a.B) * a.d;
  }
};

// Up to 3 tokens an SM take the kernel with registers for the norm weights, whose CTAs all run at once
// then (us in a graph, 32 + 16 heads: 456 tokens 6.4 / 7.5 without, 608 9.5 / 7.5)
constexpr int kFewCtas = 3;

template <bool INTERLEAVED, bool FEW>
__global__ void __launch_bounds__(kThreads) qkv_norm_rope_kernel(QkvArgs a, NewRowsArgs n) {
  extern __shared__ __align__(16) float table[];
  __shared__ size_t new_row[kMaxTokens];
  norm_rope_tokens<INTERLEAVED, FEW>(a, table, NewRows{a, n, new_row});
}

}  // namespace

}  // namespace vd

extern "C" vd_status vd_qkv_norm_rope(const void* qkv, int32_t n_seq, int32_t B, int32_t n_q_head,
                                      int32_t n_kv_head, int32_t head_dim, const void* q_weight,
                                      const void* k_weight, float eps, const float* inv_freq,
                                      int32_t rotary_dim, int32_t interleaved,
                                      const int32_t* pos_first_new, void* q_out, void* k_new,
                                      void* v_new, int32_t layer, int32_t n_layer,
                                      vd_stream_t stream) {
  using namespace vd;
  if (!k_new || !v_new || n_layer < 1 || layer < 0 || layer >= n_layer ||
      (rotary_dim > 0 && !pos_first_new))
    return VD_ERR_INVALID_ARG;
  vd_status r = validate_qkv(qkv, n_seq, B, n_q_head, n_kv_head, head_dim, q_weight, k_weight, eps,
                             inv_freq, rotary_dim, q_out, k_new, v_new);
  if (r != VD_OK) return r;
  DeviceInfo dev;
  r = device_info(&dev);
  if (r != VD_OK) return r;
  const QkvArgs a = qkv_args(qkv, n_seq, B, n_q_head, n_kv_head, head_dim, q_weight, k_weight, eps,
                             inv_freq, rotary_dim, q_out, dev.sms);
  const NewRowsArgs n = {pos_first_new, static_cast<uint16_t*>(k_new),
                         static_cast<uint16_t*>(v_new), layer, n_layer};
  return launch_clusters(qkv_grid(a), kThreads, 1, qkv_smem(a),
                         reinterpret_cast<cudaStream_t>(stream),
                         a.tokens <= kFewCtas * dev.sms
                             ? (interleaved ? qkv_norm_rope_kernel<true, true>
                                            : qkv_norm_rope_kernel<false, true>)
                             : (interleaved ? qkv_norm_rope_kernel<true, false>
                                            : qkv_norm_rope_kernel<false, false>),
                         a, n);
}
