// C interface of the record layout and of the cut of 4-bit batches for the CPU tests.
#include "../../paper_2605_27740_amd/csrc/quant_plan.hpp"

extern "C" int tile_bytes(int S, int D) { return unique::QuantTile{S, D}.bytes(); }
extern "C" int tile_part(int S, int D, int part) {
  const unique::QuantTile t = {S, D};
  return part == 0 ? t.k_codes() : (part == 1 ? t.v_codes() : (part == 2 ? t.k_scales() : t.v_scales()));
}
extern "C" int v_at(int S, int D, int tok, int unit) { return unique::QuantTile{S, D}.v_at(tok, unit); }
extern "C" int balances(int batch, int kv_heads, int max_pages, int page_bytes) {
  return unique::QuantBatch{batch, kv_heads, max_pages, page_bytes, true}.balances();
}
// Chunks of a launch at most, workgroups at a time, and the cut of a batch of these lengths in pages: chunks per row.
extern "C" void cut(int batch, int kv_heads, int max_pages, int page_bytes, int three, const int* pages, int* out, int* chunks) {
  const unique::QuantBatch b = {batch, kv_heads, max_pages, page_bytes, three != 0};
  const int rows = b.rows(), max_chunks = b.max_chunks();
  int total = 0;
  for (int i = 0; i < batch; ++i) total += pages[i] * kv_heads;
  const int slots = unique::dense_slots(total, max_chunks, b.round());
  const bool room = unique::dense_has_room(rows, slots, max_chunks);
  bool even = true;
  for (int i = 1; i < batch; ++i) even = even && pages[i] == pages[0];
  const uint32_t rate = unique::dense_rate(total, rows, slots, [&](uint32_t r) {
    int sum = 0;
    for (int i = 0; i < batch; ++i) sum += unique::dense_row_weight(pages[i], r, room) * kv_heads;
    return sum;
  });
  for (int i = 0; i < batch; ++i) chunks[i] = even ? unique::dense_even_chunks(pages[i], rows, slots) : unique::dense_row_chunks(pages[i], rate);
  out[0] = max_chunks;
  out[1] = slots;
}
extern "C" void list_plan(int batch, int kv_heads, int len, int max_pages, int S, int D, int* out) {
  const unique::SplitPlan p = unique::plan_splits(batch, kv_heads, len, max_pages, S * D * 2, false);
  out[0] = p.pages_per_split; out[1] = p.num_splits; out[2] = p.rotate;
  out[3] = unique::most_splits(batch * kv_heads, len).num_splits;
}
