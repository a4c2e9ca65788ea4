// vd_q4_attend.cu -- host side of vd_q4_attend (include/vd.h): argument checks, the
// choice of tile and cluster, the launch.
#include <cuda_runtime.h>

#include <climits>
#include <mutex>

#include "vd_host.cuh"
#include "vd_q4_attend.cuh"
#include "vd_q4_tile.cuh"

namespace vd {

namespace {

struct Kernel {
  void (*kern)(AttendArgs);
  int smem, rows, threads;
};

template <int M, int NT>
constexpr Kernel stream() {
  return {q4_attend_kernel<M, NT>, AttendShape<M, NT>::kTotal, AttendShape<M, NT>::kRows, kThreads};
}

template <int M>
constexpr Kernel block() {
  return {q4_tile_kernel<M>, TileShape<M>::kTotal, kTileRows, kTileThreads};
}

// [head_dim / 32 - 1][kind]: the streaming kernel with tiles of 8 and 16 rows (16 only where
// their sums fit the registers), the block kernel
constexpr int kKinds = 3;
const Kernel kKernel[8][kKinds] = {
    {stream<1, 1>(), stream<1, 2>(), block<1>()}, {stream<2, 1>(), stream<2, 2>(), block<2>()},
    {stream<3, 1>(), stream<3, 2>(), block<3>()}, {stream<4, 1>(), stream<4, 2>(), block<4>()},
    {stream<5, 1>(), stream<5, 1>(), block<5>()}, {stream<6, 1>(), stream<6, 1>(), block<6>()},
    {stream<7, 1>(), stream<7, 1>(), block<7>()}, {stream<8, 1>(), stream<8, 1>(), block<8>()}};

// CTAs of each kernel that run at once on the device, in clusters of 1, 2, 4, 8, 16
// (0: such a cluster does not fit); asked for once per device and head dim.
struct Slots {
  bool ready;
  int at[kKinds][5];
};
std::mutex g_slots_mu;
Slots g_slots[64][8];

vd_status slots_of(const DeviceInfo& dev, int m, const Slots** out) {
  std::lock_guard<std::mutex> lk(g_slots_mu);
  Slots& s = g_slots[dev.id][m];
  if (!s.ready) {
    for (int t = 0; t < kKinds; ++t) {
      const Kernel& k = kKernel[m][t];
      if (cudaFuncSetAttribute(k.kern, cudaFuncAttributeMaxDynamicSharedMemorySize, k.smem) !=
              cudaSuccess ||
          cudaFuncSetAttribute(k.kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) !=
              cudaSuccess) {
        cudaGetLastError();
        return VD_ERR_CUDA;
      }
      for (int e = 0; e < 5; ++e) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(16 * dev.sms);
        cfg.blockDim = dim3(k.threads);
        cfg.dynamicSmemBytes = k.smem;
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = 1u << e;
        attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        int n = 0;
        if (cudaOccupancyMaxActiveClusters(&n, k.kern, &cfg) != cudaSuccess) {
          cudaGetLastError();
          n = 0;
        }
        s.at[t][e] = n << e;
      }
      if (s.at[t][0] < 1) return VD_ERR_CUDA;
    }
    s.ready = true;
  }
  *out = &s;
  return VD_OK;
}

// 0, 1: the streaming kernel with tiles of 8 or 16 query rows, 2: the block kernel.  By the
// capacity, which the host knows, not by the lengths: a short cache in a large buffer takes the
// plan of a full one.  us at 8 KV heads a sequence, head_dim 128, 8-row tiles / 16-row tiles / block,
// full caches:
//   up to 16 rows always stream (8 sequences of 4000 tokens, 16 rows, 22.4 / 18.7 / 30.5;
//   head_dim 256 36.6 / - / 52.5), more only in one wave (head_dim 256, 8 sequences, 500
//   tokens, 24 rows 19.9 / - / 16.7) and up to 32 rows (8 sequences of 4000 tokens 36.3 / 30.8 /
//   31.2) or with little work (one sequence, 500 tokens, 128 rows 8.3 / 8.5 / 13.1; capacity
//   4096, 64 rows 14.1 / 12.8 / 15.5, 128 rows 21.5 / 18.7 / 17.5);
//   8-row tiles, which read the cache once for each, with little work (one sequence, capacity
//   4096, 32 rows 10.6 / 12.5 / 14.8, 64 rows 14.1 / 12.8 / 15.5; 32000, 16 rows 36.7 / 31.6 /
//   49.1).
// Both cuts go by the work alone, and between their measured sides the best kernel also depends
// on the rows: for one sequence 8-row tiles stay ahead for 32 rows (capacity 4104 10.7, 8192
// 14.7, 16384 22.3; the rule takes 16-row tiles at 12.5, 18.8, 31.4), and 16-row tiles for 64
// (4104 12.8, 8192 19.0; the rule takes the block kernel at 15.4, 20.3).
int choose_kernel(int m, long long rows, long long units, long long capacity, const Slots& slots) {
  const long long tiles8 = (rows + 7) / 8;
  const int kind =
      rows <= 8 || units * tiles8 * capacity <= (1 << 17) ? 0 : 1;
  const long long ctas = units * ((rows + kKernel[m][kind].rows - 1) / kKernel[m][kind].rows);
  if (rows <= 16) return kind;
  if (ctas <= slots.at[kind][0] && (rows <= 32 || units * rows * capacity <= (1 << 21)))
    return kind;
  return 2;
}

bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

}  // namespace

}  // namespace vd

extern "C" vd_status vd_q4_attend(const vd_q4_cache* c, int32_t layer, const void* q,
                                  int32_t n_q_head, const void* k_new, const void* v_new,
                                  int32_t B, float scale, void* out, float* lse_out,
                                  vd_stream_t stream) {
  using namespace vd;
  vd_status r = validate_q4(c);
  if (r != VD_OK) return r;
  if (!q || !out || (k_new == nullptr) != (v_new == nullptr)) return VD_ERR_INVALID_ARG;
  if (layer < 0 || layer >= c->n_layer || B < 1 || n_q_head < 1 || n_q_head % c->n_kv_head != 0)
    return VD_ERR_INVALID_ARG;
  if (!(scale > 0.f) || scale > 3.4e38f) return VD_ERR_INVALID_ARG;
  if (misaligned(q) || misaligned(out) || misaligned(k_new) || misaligned(v_new))
    return VD_ERR_ALIGNMENT;
  const int group = n_q_head / c->n_kv_head;
  const long long rows = (long long)B * group;
  const long long units = (long long)c->n_seq * c->n_kv_head;
  if (rows > (1 << 24) || units * rows > INT_MAX / 16) return VD_ERR_UNSUPPORTED;
  DeviceInfo dev;
  r = device_info(&dev);
  if (r != VD_OK) return r;
  const int m = c->head_dim / 32 - 1;
  const Slots* slots = nullptr;
  r = slots_of(dev, m, &slots);
  if (r != VD_OK) return r;

  const int want = env_int("VD_Q4_KERNEL", -1);
  const int kind = want >= 0 && want < kKinds ? want : choose_kernel(m, rows, units, c->capacity, *slots);
  const Kernel& k = kKernel[m][kind];
  AttendArgs a;
  const size_t unit0 = (size_t)layer * c->n_kv_head * c->capacity;
  const size_t new0 = (size_t)layer * c->n_kv_head * B;
  a.k = static_cast<const uint8_t*>(c->k) + unit0 * (c->head_dim / 2);
  a.v = static_cast<const uint8_t*>(c->v) + unit0 * (c->head_dim / 2);
  a.ks = static_cast<const uint8_t*>(c->k_scale) + unit0 * (c->head_dim / 16);
  a.vs = static_cast<const uint8_t*>(c->v_scale) + unit0 * (c->head_dim / 16);
  a.q = static_cast<const uint16_t*>(q);
  a.k_new = k_new ? static_cast<const uint16_t*>(k_new) + new0 * c->head_dim : nullptr;
  a.v_new = v_new ? static_cast<const uint16_t*>(v_new) + new0 * c->head_dim : nullptr;
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse_out;
  a.len = c->len;
  a.status = dev.status;
  a.seq_rows = (size_t)c->n_layer * c->n_kv_head * c->capacity;
  a.seq_new_rows = (size_t)c->n_layer * c->n_kv_head * B;
  a.heads = c->n_kv_head;
  a.group = group;
  a.B = B;
  a.cap = c->capacity;
  a.rows = (int)rows;
  a.tiles = (int)((rows + k.rows - 1) / k.rows);
  a.scale = scale;
  a.wait_limit = wait_limit();
  const long long base = units * a.tiles;
  // The largest cluster that runs in one wave and leaves each CTA enough tokens (by the
  // capacity, as above) to pay for the join; two streaming CTAs run on an SM, and clusters of
  // 16, which do not fill the GPU's groups of SMs, have to gain more.  us, C = 4, 8, 16, one
  // token: one sequence, 8 KV heads of 500 tokens 5.1, 5.5, 7.1; 5 sequences, 3 heads, 2500
  // tokens 7.7, 7.3, 12.5; one sequence, 8 heads, 4096 tokens 9.6, 7.6, 8.2, 32000 tokens 43.5,
  // 24.7, 21.8 (8 is taken below a capacity of 32768); two sequences, 131000 tokens 162, 127, 107.
  int e = 0;
  const int least[5] = {0, 128, 128, kind == 2 ? 128 : 512, kind == 2 ? 128 : 2048};
  while (e < 4 && slots->at[kind][e + 1] > 0 &&
         (base << (e + 1)) <= slots->at[kind][kind < 2 && e == 3 ? 0 : e + 1] &&
         c->capacity >= least[e + 1] << (e + 1))
    ++e;
  const int want_cluster = env_int("VD_Q4_CLUSTER", 0);
  for (int i = 0; i < 5; ++i)
    if (want_cluster == 1 << i && slots->at[kind][i] > 0) e = i;
  a.cluster = 1 << e;
  if (base << e > INT_MAX) return VD_ERR_UNSUPPORTED;
  return launch_clusters((unsigned)(base << e), (unsigned)k.threads, (unsigned)a.cluster, k.smem,
                         reinterpret_cast<cudaStream_t>(stream), k.kern, a);
}
