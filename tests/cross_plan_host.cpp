// What cross_plan.h chooses, as a program for the CPU tests: one line of hints in, one line out.
#include <cstdio>

#include "cross_plan.h"

int main() {
  long rows, streams, total_q, max_q, max_kv;
  int batch, columns, head_dim, can_cut;
  while (scanf("%ld %d %ld %d %ld %ld %ld %d %d", &rows, &batch, &streams, &columns, &total_q, &max_q, &max_kv, &head_dim, &can_cut) == 9) {
    const sp::CrossShape s = sp::cross_shape(rows, batch, streams, columns, total_q, max_q, max_kv, head_dim, can_cut != 0);
    const sp::CrossResident r = sp::cross_resident(rows, streams, columns, max_q, max_kv, head_dim);
    const sp::CrossTiles t = sp::cross_tiles(batch, (int)(streams / batch), 32 / columns, max_q, max_kv, head_dim, can_cut != 0);
    printf("%d %d %d %d %d %d %d %d %d %d %d\n", s.halves, s.ranked, s.pieces, r.blocks, r.waves, r.rounds, sp::cross_resident_for_few(streams, max_kv, head_dim), s.solo,
           t.tiles, t.splits, t.chunk);
  }
}
