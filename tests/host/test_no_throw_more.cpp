// The C entry points of the RMS norm, the rotary positions and the attention over
// shared prefixes when memory for a message runs out: operator new (the library's too)
// fails once `failing` is set.
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

template <typename F> F find(void *lib, const char *name) { return (F)dlsym(lib, name); }

int main(int argc, char **argv) {
  void *lib = argc > 1 ? dlopen(argv[1], RTLD_NOW) : nullptr;
  if (!lib) return printf("cannot load: %s\n", dlerror()), 1;
  const auto rms_check = find<decltype(&mita_rms_check)>(lib, "mita_rms_check");
  const auto rms_size = find<decltype(&mita_rms_workspace_size)>(lib, "mita_rms_workspace_size");
  const auto rms_forward = find<decltype(&mita_rms_forward)>(lib, "mita_rms_forward");
  const auto rms_backward = find<decltype(&mita_rms_backward)>(lib, "mita_rms_backward");
  const auto rope_check = find<decltype(&mita_rope_check)>(lib, "mita_rope_check");
  const auto rope_forward = find<decltype(&mita_rope_forward)>(lib, "mita_rope_forward");
  const auto rope_backward = find<decltype(&mita_rope_backward)>(lib, "mita_rope_backward");
  const auto prefix_check = find<decltype(&mita_prefix_check)>(lib, "mita_prefix_check");
  const auto prefix_size = find<decltype(&mita_prefix_workspace_size)>(lib, "mita_prefix_workspace_size");
  const auto prefix_forward = find<decltype(&mita_prefix_forward)>(lib, "mita_prefix_forward");
  if (!rms_check || !rms_size || !rms_forward || !rms_backward || !rope_check || !rope_forward || !rope_backward ||
      !prefix_check || !prefix_size || !prefix_forward)
    return 1;
  mita_rms_cfg_t r{};
  r.n[0] = r.n[1] = r.n[2] = 1, r.C = 64, r.eps = 1e-5f, r.ytype = 7;
  mita_rope_cfg_t o{};
  o.B = o.H = o.H_kv = o.N = 1, o.d = o.rot = 64, o.base = 0.5;
  mita_prefix_cfg_t p{};
  p.B = p.Bp = p.H = p.H_kv = p.N = 1, p.P = 1 << 30, p.d = 64, p.left = p.right = -1;
  void *const q = (void *)0x10000000;
  failing = true;
  bool ok = rms_check(&r) != MITA_OK && rms_size(&r) == 0 && rope_check(&o) != MITA_OK && prefix_check(&p) != MITA_OK &&
            prefix_size(&p) == 0;
  ok = ok && rms_forward(&r, q, 0, 0, 0, q, 0, 0, 0) != MITA_OK && rms_backward(&r, q, 0, 0, q, 0, q, 0, 0, 0, 0) != MITA_OK;
  ok = ok && rope_forward(&o, q, 0, 0, q, 0, 0) != MITA_OK && rope_backward(&o, q, 0, 0, q, 0, 0) != MITA_OK;
  ok = ok && prefix_forward(&p, q, q, q, q, q, 0, 0, 0, q, 0, 0, 0, 0) != MITA_OK;
  r.ytype = MITA_F32, o.base = 1e4, p.P = 64;  // and of refused pointers
  ok = ok && rms_forward(&r, 0, 0, 0, 0, q, 0, 0, 0) != MITA_OK && rope_forward(&o, 0, 0, 0, q, 0, 0) != MITA_OK &&
       prefix_forward(&p, 0, q, q, q, q, 0, 0, 0, q, 0, 0, 0, 0) != MITA_OK;
  failing = false;
  printf(ok ? "no throw ok\n" : "wrong answers\n");
  return ok ? 0 : 1;
}
