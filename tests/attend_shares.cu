// Prints the key tiles of one key head of a sequence, as the attention kernel
// counts them, for each line "rows_per_item start count group causal" of the
// standard input.
#include <cstdio>

#include "sjd_kv_device.cuh"

int main() {
  int rows, start, count, group, causal;
  while (std::scanf("%d %d %d %d %d", &rows, &start, &count, &group, &causal) == 5) {
    sjd_kv_ops::AttendParams p{};
    p.c.group = group;
    const sjd_kv_ops::Divisor d = sjd_kv_ops::divisor(group);
    p.c.group_mul = d.mul, p.c.group_shift = d.shift;
    p.mask_kind = causal ? SJD_MASK_CAUSAL : SJD_MASK_ALL;
    const int2 span = make_int2(start, count);
    std::printf("%lld\n", static_cast<long long>(rows == 256 ? sjd_kv_ops::tiles_of<2>(p, span) : sjd_kv_ops::tiles_of<1>(p, span)));
  }
}
