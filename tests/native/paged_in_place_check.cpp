// In place means the same rows: an output that begins where the queries do, with another
// stride, would be written over rows that other workgroups still read, and is refused.
// Prints the number of calls checked.
#define main refusals_main
#include "paged_refusals_check.cpp"
#undef main

int main() {
  const auto SHAPE = CRF_ERR_SHAPE;
  for (Entry e : {&Call::append, &Call::attend}) {
    expect("in place", e, CRF_OK, 1, [](Call &) {});
    expect("wider rows", e, CRF_OK, 1, [](Call &c) { c.q_ld = c.o_ld = 512; });
    expect("in place, output wider", e, SHAPE, 0, [](Call &c) { c.o_ld = 512; });
    expect("in place, queries wider", e, SHAPE, 0, [](Call &c) { c.q_ld = 512; });
    expect("one row", e, CRF_OK, 1, [](Call &c) { c.q_ld = 512, c.batch.n_rows = 1; });
    expect("elsewhere", e, CRF_OK, 1, [](Call &c) { c.q_ld = 512, c.q_out = c.out = c.at + (1 << 20); });
  }
  if (g_wrong) return 1;
  printf("ok %d\n", g_checked);
  return 0;
}
