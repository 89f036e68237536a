// Appends whose length arrays overlap, on a machine without a GPU: which are
// refused, and which tell the kernel to wait for the other work-groups' reads.
// The stand-in runtime and the checks are paged_driver.cpp's.
#define main paged_driver_main
#include "paged_driver.cpp"
#undef main

int main() {
  alignas(16) static char mem[256];
  static int32_t ints[32];
  bifattn_paged_dims_t d = dims();
  bifattn_paged_plan_t P;
  CHECK(bifattn_paged_plan_create(&d, &P) == BIFATTN_OK);
  bifattn_pages_t pg{};
  pg.K = pg.V = mem;
  auto append = [&](const int32_t* lens, const int32_t* counts, int32_t* lens_out) {
    bifattn_new_rows_t r{};
    r.samples = 3, r.n = 5, r.k = r.v = mem, r.counts = counts;
    g_launches = 0;
    const bifattn_status_t st = bifattn_paged_append(P, &pg, ints + 30, &r, lens, lens_out, nullptr);
    CHECK((st == BIFATTN_OK) == (g_launches == 8));
    return st;
  };
  int32_t *a = ints, *b = ints + 4, *c = ints + 8;
  CHECK(append(a, nullptr, b) == BIFATTN_OK && !g_append.in_place);
  CHECK(append(a, b, c) == BIFATTN_OK && !g_append.in_place);
  CHECK(append(a, a, c) == BIFATTN_OK && !g_append.in_place);
  CHECK(append(a, c, a + 3) == BIFATTN_OK && !g_append.in_place);  // side by side
  CHECK(append(a, nullptr, a) == BIFATTN_OK && g_append.in_place);
  CHECK(append(a, b, a) == BIFATTN_OK && g_append.in_place);
  CHECK(append(a, b, b) == BIFATTN_OK && g_append.in_place);  // the counts are replaced by the lengths
  CHECK(append(a, a, a) == BIFATTN_OK && g_append.in_place);
  for (int off : {-2, -1, 1, 2}) {  // one sample's new length is another's input
    CHECK(append(c, nullptr, c + off) == BIFATTN_EINVAL);
    CHECK(append(a, c, c + off) == BIFATTN_EINVAL);
    CHECK(append(c, c + off, c) == BIFATTN_EINVAL);
  }
  CHECK(bifattn_paged_plan_destroy(P) == BIFATTN_OK);
  std::printf("all checks passed\n");
  return 0;
}
