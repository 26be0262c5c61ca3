// Host-side harness for tests/test_window_tiles_host.py: the row tiles of every windowed kernel, by the sizes that the
// library's header gives them, with the checks of window_harness.cpp.  Nothing runs on a GPU.
#define main lists_main
#include "window_harness.cpp"
#undef main

int main() {
  std::mt19937 rng(11);
  for (int i = 0; i < 20000; ++i)
    if (!check_tiles<kMfmaRows>(rng) || !check_tiles<kWideRows>(rng) || !check_tiles<kF32Rows>(rng) ||
        !check_tiles<2 * kF32Rows>(rng)) {
      printf("tiles %d\n", i);
      return 0;
    }
  printf("ok\n");
  return 0;
}
