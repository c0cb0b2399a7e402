// C interface of the record layout and of the cut of 4-bit batches for the CPU tests.
#include "../../paper_2605_27740_amd/csrc/quant_plan.hpp"

extern "C" int tile_bytes(int S, int D) { return unique::QuantTile{S, D}.bytes(); }
extern "C" int tile_part(int S, int D, int part) {
  const unique::QuantTile t = {S, D};
  return part == 0 ? t.k_codes() : (part == 1 ? t.v_codes() : (part == 2 ? t.k_scales() : t.v_scales()));
}
extern "C" int v_at(int S, int D, int tok, int unit) { return unique::QuantTile{S, D}.v_at(tok, unit); }
extern "C" int balances(int batch, int kv_heads, int max_pages, int page_bytes) {
  return unique::dense_balances(batch, kv_heads, max_pages, page_bytes, unique::kQuantLeastBytes);
}
// Slots of the partial results, chunks of a launch at most, and the cut of a batch of these lengths in pages: chunks per row.
extern "C" void cut(int batch, int kv_heads, int max_pages, const int* pages, long long* out, int* chunks) {
  const int rows = batch * kv_heads;
  const unique::DenseRound round = unique::quant_round(rows, max_pages);
  const int max_chunks = unique::dense_max_chunks(rows, max_pages, round);
  int total = 0;
  for (int b = 0; b < batch; ++b) total += pages[b] * kv_heads;
  const int slots = unique::dense_slots(total, max_chunks, round);
  const bool room = unique::dense_has_room(rows, slots, max_chunks);
  bool even = true;
  for (int b = 1; b < batch; ++b) even = even && pages[b] == pages[0];
  const uint32_t rate = unique::dense_rate(total, rows, slots, [&](uint32_t r) {
    int sum = 0;
    for (int b = 0; b < batch; ++b) sum += unique::dense_row_weight(pages[b], r, room) * kv_heads;
    return sum;
  });
  for (int b = 0; b < batch; ++b) chunks[b] = even ? unique::dense_even_chunks(pages[b], rows, slots) : unique::dense_row_chunks(pages[b], rate);
  out[0] = (long long)rows * unique::most_splits(rows, max_pages).num_splits;
  out[1] = max_chunks;
  out[2] = slots;
}
extern "C" void list_plan(int batch, int kv_heads, int len, int max_pages, int S, int D, int* out) {
  const unique::SplitPlan p = unique::plan_splits(batch, kv_heads, len, max_pages, S * D * 2, false);
  out[0] = p.pages_per_split; out[1] = p.num_splits; out[2] = p.rotate;
  out[3] = unique::most_splits(batch * kv_heads, len).num_splits;
}
