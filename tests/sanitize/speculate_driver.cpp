// Drives the host side of the speculative-decoding entry points without a GPU: the kernel launchers are stand-ins that
// read what they are given.  Built with -fsanitize=address,undefined.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>

#include "treekv_internal.h"

#define CHECK(cond) do { if (!(cond)) { fprintf(stderr, "%s:%d: CHECK failed: %s\n", __FILE__, __LINE__, #cond); exit(1); } } while (0)

static int launches = 0;
namespace tkv {
size_t tree_scratch_bytes(const Params& p, int n) { return p.U < 8 ? (size_t)p.U * n * 256 : 0; }
int launch_tree_attend(const Params&, const Tree&, float*, float*, void*, hipStream_t) { ++launches; return TREEKV_OK; }
int launch_tree_colsums(const Params&, const Tree&, int32_t*, hipStream_t) { ++launches; return TREEKV_OK; }
int launch_tree_replay(const Params&, const Tree&, int32_t*, int32_t*, int32_t*, hipStream_t) { ++launches; return TREEKV_OK; }
int launch_fork(const Params& to, const Params& from, const int32_t* src, const int32_t* dst, int count, hipStream_t) {
  for (int i = 0; i < count; ++i) CHECK(dst[i] >= 0 && dst[i] < to.B && src[i] >= -1 && src[i] < from.B);
  ++launches;
  return TREEKV_OK;
}
int launch_qkv(const treekv_qkv_args&, hipStream_t) { ++launches; return TREEKV_OK; }
}  // namespace tkv

static treekv_ctx* context(int batch, uintptr_t at) {
  treekv_config c;
  memset(&c, 0, sizeof(c));
  c.budget = 64; c.q_heads = 4; c.kv_heads = 2; c.head_dim = 128; c.batch = batch; c.dtype = TREEKV_BF16; c.n_sink = 2; c.n_recent = 20;
  treekv_ctx* h = nullptr;
  CHECK(treekv_init_ex(&h, &c) == TREEKV_OK);
  CHECK(treekv_bind_workspace(h, (void*)at, (size_t)1 << 40) == TREEKV_OK);
  return h;
}

int main() {
  treekv_ctx *a = context(3, 0x100000), *b = context(70, 0x10000000);
  void* ok = (void*)0x1000;
  int32_t* ints = (int32_t*)ok;
  float* f = (float*)ok;
  const size_t need = treekv_tree_scratch_bytes(a, 256);
  CHECK(need > 0 && treekv_tree_scratch_bytes(b, 256) == 0);
  CHECK(treekv_tree_attend(a, ok, ok, ok, ints, 256, f, nullptr, ok, need, nullptr) == TREEKV_OK);
  CHECK(treekv_tree_attend(a, ok, ok, ok, ints, 256, f, f, ok, need - 1, nullptr) == TREEKV_EINVAL);
  CHECK(treekv_tree_attend(b, ok, ok, ok, ints, 1, f, f, nullptr, 0, nullptr) == TREEKV_OK);
  CHECK(treekv_tree_commit(a, ok, ok, ok, ints, f, 9, ints, ints, 9, ints, nullptr, nullptr, nullptr, nullptr) == TREEKV_OK);
  CHECK(launches == 4);
  // pairs on the heap, so that a read behind their end shows
  std::vector<int32_t> src(70, 0), dst(70);
  for (int i = 0; i < 70; ++i) dst[i] = i;
  CHECK(treekv_fork(b, a, src.data(), dst.data(), 70, nullptr) == TREEKV_OK);
  dst[69] = 0;
  CHECK(treekv_fork(b, a, src.data(), dst.data(), 70, nullptr) == TREEKV_EINVAL);
  dst[69] = 70;
  CHECK(treekv_fork(b, a, src.data(), dst.data(), 70, nullptr) == TREEKV_EINVAL);
  dst[69] = 69;
  CHECK(treekv_fork(b, b, src.data(), dst.data(), 70, nullptr) == TREEKV_OK);         // 0 goes to itself, and to the others
  src[0] = 1;
  CHECK(treekv_fork(b, b, src.data(), dst.data(), 70, nullptr) == TREEKV_EINVAL);     // 0 is written, and read for the others
  CHECK(treekv_fork(b, b, src.data() + 1, dst.data() + 1, 69, nullptr) == TREEKV_OK);
  CHECK(launches == 7);
  treekv_qkv_args q;
  memset(&q, 0, sizeof(q));
  q.q = (void*)0x10000; q.q_out = (void*)0x10000; q.tokens = 2147483647; q.q_heads = 65536; q.head_dim = 128; q.dtype = TREEKV_F32;
  q.q_stride = (int64_t)65536 * 128;
  CHECK(treekv_qkv_prepare(&q, nullptr) == TREEKV_OK);
  q.q_stride = INT64_MAX;
  CHECK(treekv_qkv_prepare(&q, nullptr) == TREEKV_EINVAL);
  q.tokens = 1;                                            // one token has no next one
  CHECK(treekv_qkv_prepare(&q, nullptr) == TREEKV_OK);
  CHECK(launches == 9);
  treekv_destroy(a);
  treekv_destroy(b);
  puts("speculate paths clean");
  return 0;
}
