// generated by build.py: lookup over the instantiation tables
#include "rap_internal.h"
const rap_q4_entry* rap_q4_table_0(int* n);
const rap_q4_entry* rap_q4_table_1(int* n);
const rap_q4_entry* rap_q4_table_2(int* n);
const rap_q4_entry* rap_q4_table_3(int* n);
const rap_q4_entry* rap_q4_table_4(int* n);
const rap_q4_entry* rap_q4_table_5(int* n);
const rap_q4_entry* rap_q4_table_6(int* n);
const rap_q4_entry* rap_q4_table_7(int* n);
const rap_q4_entry* rap_q4_table_8(int* n);
const rap_q4_entry* rap_q4_table_9(int* n);
const rap_q4_entry* rap_q4_table_10(int* n);
const rap_q4_entry* rap_q4_table_11(int* n);
const rap_q4_entry* rap_q4_table_12(int* n);
const rap_q4_entry* rap_q4_table_13(int* n);
const rap_q4_entry* rap_q4_table_14(int* n);
const rap_q4_entry* rap_q4_table_15(int* n);
const rap_q4_entry* rap_q4_find(int k_words, int v_words, int heads_per_lane) {
  typedef const rap_q4_entry* (*table_fn)(int*);
  static const table_fn parts[] = {rap_q4_table_0, rap_q4_table_1, rap_q4_table_2, rap_q4_table_3, rap_q4_table_4, rap_q4_table_5, rap_q4_table_6, rap_q4_table_7, rap_q4_table_8, rap_q4_table_9, rap_q4_table_10, rap_q4_table_11, rap_q4_table_12, rap_q4_table_13, rap_q4_table_14, rap_q4_table_15};
  for (table_fn f : parts) {
    int n = 0;
    const rap_q4_entry* t = f(&n);
    for (int i = 0; i < n; ++i)
      if (t[i].k_words == k_words && t[i].v_words == v_words && t[i].heads_per_lane == heads_per_lane) return &t[i];
  }
  return nullptr;
}
const rap_scan_entry* rap_q8_table_0(int* n);
const rap_scan_entry* rap_q8_table_1(int* n);
const rap_scan_entry* rap_q8_table_2(int* n);
const rap_scan_entry* rap_q8_table_3(int* n);
const rap_scan_entry* rap_q8_find(int G, int WK, int DV) {
  typedef const rap_scan_entry* (*table_fn)(int*);
  static const table_fn parts[] = {rap_q8_table_0, rap_q8_table_1, rap_q8_table_2, rap_q8_table_3};
  for (table_fn f : parts) {
    int n = 0;
    const rap_scan_entry* t = f(&n);
    for (int i = 0; i < n; ++i)
      if (t[i].G == G && t[i].WK == WK && t[i].DV == DV) return &t[i];
  }
  return nullptr;
}
const rap_scan_entry* rap_mma_table_0(int* n);
const rap_scan_entry* rap_mma_table_1(int* n);
const rap_scan_entry* rap_mma_table_2(int* n);
const rap_scan_entry* rap_mma_table_3(int* n);
const rap_scan_entry* rap_mma_table_4(int* n);
const rap_scan_entry* rap_mma_table_5(int* n);
const rap_scan_entry* rap_mma_table_6(int* n);
const rap_scan_entry* rap_mma_table_7(int* n);
const rap_scan_entry* rap_mma_find(int G, int WK, int DV) {
  typedef const rap_scan_entry* (*table_fn)(int*);
  static const table_fn parts[] = {rap_mma_table_0, rap_mma_table_1, rap_mma_table_2, rap_mma_table_3, rap_mma_table_4, rap_mma_table_5, rap_mma_table_6, rap_mma_table_7};
  for (table_fn f : parts) {
    int n = 0;
    const rap_scan_entry* t = f(&n);
    for (int i = 0; i < n; ++i)
      if (t[i].G == G && t[i].WK == WK && t[i].DV == DV) return &t[i];
  }
  return nullptr;
}
const rap_scan_entry* rap_scan_table_0(int* n);
const rap_scan_entry* rap_scan_table_1(int* n);
const rap_scan_entry* rap_scan_table_2(int* n);
const rap_scan_entry* rap_scan_table_3(int* n);
const rap_scan_entry* rap_scan_table_4(int* n);
const rap_scan_entry* rap_scan_table_5(int* n);
const rap_scan_entry* rap_scan_table_6(int* n);
const rap_scan_entry* rap_scan_table_7(int* n);
const rap_scan_entry* rap_scan_find(int G, int WK, int DV) {
  typedef const rap_scan_entry* (*table_fn)(int*);
  static const table_fn parts[] = {rap_scan_table_0, rap_scan_table_1, rap_scan_table_2, rap_scan_table_3, rap_scan_table_4, rap_scan_table_5, rap_scan_table_6, rap_scan_table_7};
  for (table_fn f : parts) {
    int n = 0;
    const rap_scan_entry* t = f(&n);
    for (int i = 0; i < n; ++i)
      if (t[i].G == G && t[i].WK == WK && t[i].DV == DV) return &t[i];
  }
  return nullptr;
}
