// Loaded in front of the C++ runtime (LD_PRELOAD): the n-th allocation after fail_new(n) throws, once.
#include <cstdlib>
#include <new>

static int left;

extern "C" void fail_new(int n) { left = n; }

void* operator new(std::size_t n) {
  if (left && --left == 0) throw std::bad_alloc();
  if (void* p = std::malloc(n ? n : 1)) return p;
  throw std::bad_alloc();
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, std::size_t) noexcept { std::free(p); }
