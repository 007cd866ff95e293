// Runs the host code of dropout, the norm, the cross-entropy over many classes
// and the model with dropout (api_head.hip, rows.hip, linear_loss.hip, over
// api.hip) in a build with AddressSanitizer and UndefinedBehaviorSanitizer: the
// checks of arguments, the plan's arithmetic on extents up to the largest, and
// every launch's.  Launches end here, in stand-ins of the runtime's entry points,
// which check that their extents are ones that a launch takes.  Device pointers are
// fake addresses that the host code never dereferences.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <random>

#include "gmb.h"

#define CHECK(c)                                                                                      \
  do {                                                                                                \
    if (!(c)) {                                                                                       \
      std::fprintf(stderr, "check failed at line %d: %s (%s)\n", __LINE__, #c, gmb_last_error());     \
      std::exit(1);                                                                                   \
    }                                                                                                 \
  } while (0)

namespace {
dim3 g_grid, g_block;
size_t g_shared;
hipStream_t g_stream;
long long g_launches;
}  // namespace

extern "C" hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t shared, hipStream_t stream) {
  g_grid = grid;
  g_block = block;
  g_shared = shared;
  g_stream = stream;
  return hipSuccess;
}
extern "C" hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* shared, hipStream_t* stream) {
  *grid = g_grid;
  *block = g_block;
  *shared = g_shared;
  *stream = g_stream;
  return hipSuccess;
}
extern "C" hipError_t hipLaunchKernel(const void*, dim3 grid, dim3 block, void** args, size_t, hipStream_t) {
  const uint64_t threads = static_cast<uint64_t>(block.x) * block.y * block.z;
  CHECK(threads >= 1 && threads <= 1024 && args);
  CHECK(grid.x >= 1 && grid.y >= 1 && grid.z >= 1 && grid.y <= 65535 && grid.z <= 65535);
  CHECK(static_cast<uint64_t>(grid.x) * block.x < (uint64_t{1} << 31));
  ++g_launches;
  return hipSuccess;
}
extern "C" hipError_t hipGetLastError() { return hipSuccess; }

static char* fake(uint64_t k) { return reinterpret_cast<char*>((k + 1) << 52); }

// One loss at these extents, in both types and layouts, with some of its gradients.
static long long loss(int64_t rows, int32_t d, int32_t classes) {
  const long long before = g_launches;
  for (int bf16 = 0; bf16 < 2; ++bf16)
    for (int layout = 0; layout < 4; ++layout)
      for (int want = 0; want < 8; ++want) {
        const int turned = layout & 1, far = layout >> 1;
        const int64_t near = turned ? classes : d;
        gmb_linear_head h{};
        h.x = fake(0);
        h.x_stride = far ? d + (int64_t{1} << 20) : d;
        h.w = fake(1) + (far ? 2 << bf16 : 0);
        (turned ? h.w_col_stride : h.w_row_stride) = near + (far ? 3 : 0);
        (turned ? h.w_row_stride : h.w_col_stride) = 1;
        h.bias = want & 1 ? reinterpret_cast<const float*>(fake(2)) : nullptr;
        h.labels = reinterpret_cast<const int32_t*>(fake(3));
        h.rows = rows;
        h.d = d;
        h.classes = classes;
        h.dtype = bf16 ? GMB_BF16 : GMB_F32;
        gmb_linear_grads g{want & 1 ? fake(4) : nullptr, want & 2 ? fake(5) : nullptr,
                           want & 4 ? reinterpret_cast<float*>(fake(6)) : nullptr, turned, 0};
        float* out = reinterpret_cast<float*>(fake(7));
        const size_t need = gmb_linear_loss_workspace_bytes(&h, &g);
        if (need == 0) {            // more than a launch takes: said, and nothing launched
          const long long now = g_launches;
          if (rows > 0) CHECK(gmb_linear_loss(&h, &g, out, fake(8), ~size_t{0}, nullptr) == GMB_EINVAL && g_launches == now);
          continue;
        }
        CHECK(need < size_t{1} << 46);
        CHECK(gmb_linear_loss(&h, &g, out, fake(8), need, nullptr) == GMB_OK);
        if (rows > 0 && need > 256) CHECK(gmb_linear_loss(&h, &g, out, fake(8), need - 1, nullptr) == GMB_ENOSPC);
      }
  return g_launches - before;
}

static void rows(int64_t n, int32_t dim) {
  const uint32_t step = 0;
  const gmb_dropout d{123, 0.5f, 7, &step};
  const int32_t* ids = reinterpret_cast<const int32_t*>(fake(1));
  float* w = reinterpret_cast<float*>(fake(2));
  for (int dtype : {GMB_F32, GMB_BF16}) {
    const gmb_rows x{fake(3), dim + 3}, y{fake(4), dim}, r{fake(5), dim}, o{fake(6), dim};
    CHECK(gmb_dropout_rows(&x, &y, &d, ids, nullptr, n, dim, dtype, &o, nullptr) == GMB_OK);
    for (int32_t format : {int32_t{0}, int32_t{GMB_MXFP4}, int32_t{GMB_MXFP8}}) {
      const gmb_rows to{fake(7), format ? int64_t{1} << 20 : dim};
      CHECK(gmb_rms_norm(&x, &y, &d, ids, ids, n, dim, dtype, w, 1e-6f, &r, format, &to, nullptr) == GMB_OK);
    }
    const size_t need = gmb_rms_norm_workspace_bytes(n, dim);
    CHECK(need > 0 && need <= size_t{1} << 30);
    CHECK(gmb_rms_norm_backward(&y, &r, &x, &d, ids, nullptr, n, dim, dtype, w, 1e-6f, &o, nullptr, w, fake(8), need,
                                nullptr) == GMB_OK);
  }
}

// A model of these layers over blocks of made-up capacities, forward and back.
static void model(int32_t L, int32_t dtype, float p) {
  gmb_blocks b{};
  gmb_sage_weights w{};
  gmb_sage_grads g{};
  b.num_layers = w.num_layers = g.num_layers = L;
  b.num_seeds = 100;
  w.dtype = dtype;
  int64_t cap = 100;
  for (int l = L - 1; l >= 0; --l) {
    gmb_block& k = b.blk[l];
    k.indptr = k.indices = k.nbr = k.src_ids = k.sizes = reinterpret_cast<int32_t*>(fake(1));
    k.cap_dst = cap;
    k.fanout = 5;
    k.cap_nnz = 5 * cap;
    k.cap_src = cap = 6 * cap;
    k.layer = l;
    w.w_self[l] = w.w_neigh[l] = fake(2);
    w.bias[l] = g.d_bias[l] = reinterpret_cast<float*>(fake(3));
    g.d_self[l] = g.d_neigh[l] = reinterpret_cast<float*>(fake(4));
  }
  for (int l = 0; l <= L; ++l) w.dims[l] = 16 * (l + 1);
  const gmb_dropout d{5, p, 2, nullptr};
  float* out = reinterpret_cast<float*>(fake(5));
  const size_t fw = gmb_forward_workspace_bytes(&b, &w), bw = gmb_backward_workspace_bytes(&b, &w);
  CHECK(fw > 0 && bw > 0);
  CHECK(gmb_sage_forward_dropout(&b, fake(6), nullptr, 0, &w, &d, out, fake(7), fw, nullptr, nullptr) == GMB_OK);
  CHECK(gmb_sage_forward_dropout(&b, fake(6), fake(8), 10000, &w, &d, out, fake(7), fw, nullptr, nullptr) == GMB_OK);
  CHECK(gmb_sage_backward_from(&b, fake(6), &w, out, &d, fake(7), fw, &g, fake(9), bw, nullptr, 0, 0.f, nullptr) == GMB_OK);
}

int main() {
  for (int32_t L : {1, 2, 3, GMB_MAX_LAYERS})
    for (int32_t dtype : {int32_t{GMB_F32}, int32_t{GMB_BF16}})
      for (float p : {0.f, 0.5f, 1.f}) model(L, dtype, p);
  for (int64_t n : {int64_t{0}, int64_t{1}, int64_t{2}, int64_t{45000}, int64_t{0x7FFFFFFF}})
    for (int32_t dim : {1, 7, 8, 100, 128, 256, 1270, 2049, 4096, 8192, 16392, 32769, 65536}) rows(n, dim);
  const int64_t some_rows[] = {0, 1, 15, 16, 17, 256, 257, 1000, 4096, 4097, 33024, 100000, 393217, (1 << 22) - 1, 1 << 22};
  const int32_t some_d[] = {1, 3, 64, 65, 256, 1024, 1025, 65536};
  const int32_t some_classes[] = {1, 2, 16, 47, 64, 65, 256, 257, 5003, 100000, 2449029, (1 << 27) - 1, 1 << 27};
  for (int64_t n : some_rows)
    for (int32_t d : some_d)
      for (int32_t c : some_classes) {
        // (many pieces are many launches: the largest products of rows and classes are only planned)
        if (n * c <= int64_t{1} << 36) loss(n, d, c);
        gmb_linear_head h{fake(0), d, fake(1), d, 1, nullptr, reinterpret_cast<const int32_t*>(fake(3)), n, d, c, GMB_BF16, 0};
        gmb_linear_grads g{fake(4), fake(5), reinterpret_cast<float*>(fake(6)), 0, 0};
        for (int dtype : {GMB_F32, GMB_BF16}) {
          h.dtype = dtype;
          const size_t need = gmb_linear_loss_workspace_bytes(&h, &g);
          CHECK(need < size_t{1} << 46);
        }
      }
  std::mt19937_64 rng(1);
  auto any = [&](int bits) { return static_cast<int64_t>(rng() & ((uint64_t{1} << (1 + rng() % bits)) - 1)); };
  for (int k = 0; k < 400; ++k) loss(any(15), static_cast<int32_t>(1 + any(11)), static_cast<int32_t>(1 + any(18)));
  std::printf("ok: %lld launches\n", g_launches);
  return 0;
}
