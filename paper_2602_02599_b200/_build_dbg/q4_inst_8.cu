// generated by build.py: instantiations of the tensor-core scan over a 4-bit cache, part 8
#include "rap_attn_q4_kernel.cuh"
namespace {
template <int K, int V, int C> rap_q4_entry entry() {
  return rap_q4_entry{K, V, C, Q4Cfg<K, V, C>::SMEM, Q4Cfg<K, V, C>::NW * 32, (const void*)attn_q4_kernel<K, V, C>};
}
}  // namespace
const rap_q4_entry* rap_q4_table_8(int* n) {
  static const rap_q4_entry table[] = {
    entry<5, 3, 1>(),
    entry<9, 3, 1>(),
    entry<13, 3, 1>(),
    entry<17, 3, 1>(),
    entry<5, 3, 2>(),
    entry<9, 3, 2>(),
    entry<13, 3, 2>(),
    entry<17, 3, 2>(),
  };
  *n = (int)(sizeof(table) / sizeof(table[0]));
  return table;
}
