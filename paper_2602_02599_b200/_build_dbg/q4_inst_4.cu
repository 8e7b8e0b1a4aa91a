// generated by build.py: instantiations of the tensor-core scan over a 4-bit cache, part 4
#include "rap_attn_q4_kernel.cuh"
namespace {
template <int K, int V, int C> rap_q4_entry entry() {
  return rap_q4_entry{K, V, C, Q4Cfg<K, V, C>::SMEM, Q4Cfg<K, V, C>::NW * 32, (const void*)attn_q4_kernel<K, V, C>};
}
}  // namespace
const rap_q4_entry* rap_q4_table_4(int* n) {
  static const rap_q4_entry table[] = {
    entry<3, 11, 1>(),
    entry<7, 11, 1>(),
    entry<11, 11, 1>(),
    entry<15, 11, 1>(),
    entry<3, 11, 2>(),
    entry<7, 11, 2>(),
    entry<11, 11, 2>(),
    entry<15, 11, 2>(),
  };
  *n = (int)(sizeof(table) / sizeof(table[0]));
  return table;
}
