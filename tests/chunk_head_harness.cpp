// Host harness for the header of a chunk plan (put_chunk_head in chunk.hpp): reads "items parts rows max_rows
// max_items key written" lines from stdin and prints each header's six words.
#include <cstdio>

#include "chunk.hpp"

int main() {
  long long items, parts, rows;
  int max_rows, max_items, written;
  unsigned long long key;
  while (std::scanf("%lld %lld %lld %d %d %llu %d", &items, &parts, &rows, &max_rows, &max_items, &key, &written) == 7) {
    alignas(16) int32_t head[bdlm::kChunkHead] = {};
    bdlm::ChunkPlanArgs a{};
    a.plan = head;
    a.rows = max_rows;
    a.max_items = max_items;
    a.key = key;
    bdlm::put_chunk_head(a, items, parts, rows, written != 0);
    for (int i = 0; i < 6; ++i) std::printf("%d ", head[i]);
    std::printf("\n");
  }
  return 0;
}
