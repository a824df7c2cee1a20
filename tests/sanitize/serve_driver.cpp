// Drives the host side of the paged cache's entry points and of treekv_tree_verify without a GPU: the kernel launchers are
// stand-ins.  Built with -fsanitize=address,undefined.
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "treekv_internal.h"

#define CHECK(cond) do { if (!(cond)) { fprintf(stderr, "%s:%d: CHECK failed: %s\n", __FILE__, __LINE__, #cond); exit(1); } } while (0)

static int launches = 0;
namespace tkv {
void fresh() {}
hipError_t take_hip_error() { return hipSuccess; }
int launch_paged_append(const treekv_paged_cache&, const void*, const void*, int64_t, int64_t, const int32_t*, int, const int32_t*, int32_t*, hipStream_t) { ++launches; return TREEKV_OK; }
size_t paged_attend_scratch_bytes(const treekv_paged_cache&, int tokens, int, int weigh) { return weigh ? (size_t)tokens * 256 : 0; }
int launch_paged_attend(const treekv_paged_cache&, const void*, int64_t, const int32_t*, int, int, void*, float*, int, void*, int32_t*, hipStream_t) { ++launches; return TREEKV_OK; }
size_t paged_evict_scratch_bytes(const treekv_paged_cache& c) { return (size_t)c.batch * c.kv_heads * c.table_width * c.page_size * 4; }
int launch_paged_evict(const treekv_paged_cache&, int, int, int, int32_t*, void*, int32_t*, hipStream_t) { ++launches; return TREEKV_OK; }
size_t verify_scratch_bytes(int batch, int, int) { return (size_t)batch * 256; }
int launch_verify(const treekv_verify_args&, hipStream_t) { ++launches; return TREEKV_OK; }
}  // namespace tkv

int main() {
  const uintptr_t T = (uintptr_t)1 << 40;
  treekv_paged_cache c;
  memset(&c, 0, sizeof(c));
  c.k = (void*)T; c.v = (void*)(2 * T); c.table = (int32_t*)(3 * T); c.lens = (int32_t*)(4 * T);
  c.weights = (float*)(5 * T); c.positions = (int32_t*)(6 * T);
  c.pages = 100; c.page_size = 256; c.table_width = 1 << 14; c.batch = 16; c.q_heads = 65536; c.kv_heads = 8; c.head_dim = 128; c.dtype = TREEKV_F32;
  void *a = (void*)(7 * T), *b = (void*)(8 * T), *o = (void*)(9 * T), *w = (void*)(10 * T);
  int32_t* ints = (int32_t*)(11 * T);
  CHECK(treekv_paged_append(&c, a, b, 1024, 1024, ints, 1 << 20, ints + (1 << 22), nullptr, nullptr) == TREEKV_OK);
  CHECK(treekv_paged_append(&c, a, b, INT64_MAX, 1024, ints, 2, ints + 64, nullptr, nullptr) == TREEKV_EINVAL);
  CHECK(treekv_paged_append(&c, a, b, INT64_MAX, INT64_MIN, ints, 1, ints + 64, nullptr, nullptr) == TREEKV_OK);     // one token has no next one
  CHECK(treekv_paged_attend(&c, a, 65536 * 128, ints, 4096, 1, o, nullptr, 0, nullptr, 0, nullptr, nullptr) == TREEKV_OK);
  CHECK(treekv_paged_attend(&c, a, 65536 * 128, ints, 2147483647, 2147483647, o, nullptr, 0, nullptr, 0, nullptr, nullptr) == TREEKV_EUNSUPPORTED);
  CHECK(treekv_paged_attend(&c, a, 65536 * 128, ints, 4, 4, o, nullptr, 1, w, 1024, nullptr, nullptr) == TREEKV_OK);
  CHECK(treekv_paged_attend(&c, a, 65536 * 128, ints, 4, 4, o, nullptr, 1, w, 1023, nullptr, nullptr) == TREEKV_EINVAL);
  const size_t need = treekv_paged_evict_scratch_bytes(&c);
  CHECK(need == (size_t)1 << 31);
  CHECK(treekv_paged_evict(&c, 2147483647, 2147483646, 1, nullptr, w, need, nullptr, nullptr) == TREEKV_OK);
  CHECK(treekv_paged_evict(&c, 2147483647, 2147483647, 2147483647, c.lens, w, need, nullptr, nullptr) == TREEKV_EINVAL);
  CHECK(launches == 5);
  treekv_verify_args v;
  memset(&v, 0, sizeof(v));
  v.target = (void*)(64 * T); v.tokens = ints; v.parents = ints; v.uniforms = (float*)ints; v.path = (int32_t*)a; v.path_len = (int32_t*)b;
  v.next_token = (int32_t*)o; v.scratch = w; v.scratch_bytes = (size_t)1 << 40; v.batch = 2147483647; v.n = 256; v.vocab = 1 << 24; v.dtype = TREEKV_F32;
  CHECK(treekv_tree_verify(&v, nullptr) == TREEKV_EUNSUPPORTED);
  v.batch = 1 << 20;
  CHECK(treekv_tree_verify(&v, nullptr) == TREEKV_OK);
  v.scratch_bytes = ((size_t)256 << 20) - 1;
  CHECK(treekv_tree_verify(&v, nullptr) == TREEKV_EINVAL);
  CHECK(launches == 6);
  puts("serve paths clean");
  return 0;
}
