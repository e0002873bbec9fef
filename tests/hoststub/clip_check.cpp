// An iteration whose update fails, after one that measured the gradient's norm, on the real executor (graph.cpp, plan.cpp, engine.hip built for the
// host against the stand-in runtime beside this file).  usage: clip_check <spec.bin>, as executor_check.cpp.
// TEST INFRASTRUCTURE.
#include <cstdio>
#include <vector>

#include "../../include/accudnn.h"
#include "../../paper_1901_06773_amd/csrc/kernels.h"
#include "stub_runtime.h"

static int calls = 0, failing = -1;
static hipError_t update(float*, const float*, float, float, size_t, void*, float*, void*, size_t, hipStream_t) {
  return calls++ == failing ? hipErrorInvalidValue : hipSuccess;
}

int main(int argc, char** argv) {
  FILE* f = argc > 1 ? fopen(argv[1], "rb") : nullptr;
  int32_t hdr[4];
  if (!f || fread(hdr, 4, 4, f) != 4) return 2;
  std::vector<acc_layer> layers(hdr[0]);
  if (fread(layers.data(), sizeof(acc_layer), layers.size(), f) != layers.size()) return 2;
  fclose(f);
  const size_t budget = (size_t)1 << 30, arena = (size_t)1 << 30;
  void *pool = (void*)(uintptr_t)0x500000000000ull, *host = (void*)(uintptr_t)0x600000000000ull;      // nobody reads them
  stub_set_regions(pool, budget, host, arena);
  hipStream_t st[4];
  for (int i = 0; i < 4; ++i) st[i] = stub_make_stream(i);
  acc_resources res{pool, budget, host, arena, st[0], st[1], st[2], st[3]};
  acc_ctx* c = nullptr;
  if (acc_create(layers.data(), (int)layers.size(), hdr[1], hdr[2], hdr[3], ACC_F32, &res, &c) != ACC_OK) return 2;
  acc_plan_summary s;
  if (acc_plan_swaps(c, 2, budget, ACC_PLAN_NONE, &s) != ACC_OK) return 2;
  std::vector<int32_t> labels(2, 1), wrong(2, -1);
  const float* images = (const float*)(uintptr_t)0x700000000000ull;
  auto step = [&](const std::vector<int32_t>& l) { float loss; stub_new_epoch(); return acc_train_step(c, images, ACC_LOC_HOST, l.data(), 0.1f, &loss); };
  float norm = 0.f;
  printf("before any iteration: %d\n", acc_get_grad_norm(c, &norm));
  acc::set_clipped_update(c, update, 1.f);
  printf("measured: %d", step(labels));
  printf(" %d\n", acc_get_grad_norm(c, &norm));
  printf("refused: %d", step(wrong));
  printf(" %d\n", acc_get_grad_norm(c, &norm));
  failing = calls;
  const int rc = step(labels);
  printf("failed: %d %d\n", rc != ACC_OK, acc_get_grad_norm(c, &norm));
  printf("again: %d", step(labels));
  printf(" %d\n", acc_get_grad_norm(c, &norm));
  acc_destroy(c);
  for (int i = 0; i < 4; ++i) stub_free_stream(st[i]);
  return 0;
}
