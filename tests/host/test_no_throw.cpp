// The C entry points of the dense attention and the layer norm when memory for a
// message runs out: operator new (the library's too) fails once `failing` is set.
#include <dlfcn.h>

#include <cstdio>
#include <cstdlib>
#include <new>

#include "mita.h"

static bool failing = false;
void *operator new(size_t n) {
  if (failing) throw std::bad_alloc();
  void *p = malloc(n ? n : 1);
  if (!p) throw std::bad_alloc();
  return p;
}
void operator delete(void *p) noexcept { free(p); }
void operator delete(void *p, size_t) noexcept { free(p); }

int main(int argc, char **argv) {
  void *lib = argc > 1 ? dlopen(argv[1], RTLD_NOW) : nullptr;
  if (!lib) return printf("cannot load: %s\n", dlerror()), 1;
  const auto dense_size = (size_t(*)(const mita_dense_cfg_t *, int))dlsym(lib, "mita_dense_workspace_size");
  const auto dense_check = (int (*)(const mita_dense_cfg_t *))dlsym(lib, "mita_dense_check");
  const auto norm_size = (size_t(*)(const mita_norm_cfg_t *))dlsym(lib, "mita_norm_workspace_size");
  const auto norm_check = (int (*)(const mita_norm_cfg_t *))dlsym(lib, "mita_norm_check");
  if (!dense_size || !dense_check || !norm_size || !norm_check) return 1;
  mita_dense_cfg_t d{};
  d.B = d.H = d.H_kv = 1, d.N = d.N_k = 1 << 30, d.d = 64, d.left = d.right = -1;
  mita_norm_cfg_t n{};
  n.n[0] = n.n[1] = n.n[2] = 1, n.C = 1 << 30, n.eps = 1e-5f;
  failing = true;
  const bool ok = dense_size(&d, MITA_WS_FORWARD) == 0 && norm_size(&n) == 0 && dense_check(&d) != MITA_OK &&
                  norm_check(&n) != MITA_OK;
  failing = false;
  printf(ok ? "no throw ok\n" : "wrong answers\n");
  return ok ? 0 : 1;
}
