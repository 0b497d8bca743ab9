// Prints how the adapters' kernels divide the work of each query line (the library's own choices, host only).
#include "../paper_2609_33977_amd/csrc/gm_lora.h"

#include <cstdio>
#include <cstring>

int main() {
  char op[32];
  long T, n, d_in, r, parts;
  while (std::scanf("%31s %ld %ld %ld %ld %ld", op, &T, &n, &d_in, &r, &parts) == 6) {
    int w[gm::kLoraMaxParts], in[1] = {int(d_in)};
    if (parts < 1 || parts > gm::kLoraMaxParts) return 1;
    long blocks = (d_in + gm::kLoraGradCols - 1) / gm::kLoraGradCols;
    for (long p = 0; p < parts; ++p) {
      if (std::scanf("%d", &w[p]) != 1) return 1;
      blocks += (w[p] + gm::kLoraGradCols - 1) / gm::kLoraGradCols;
    }
    const long tiles = long(gm::lora_plan_layout(T, n).max_tiles);
    const int R = int(parts * r);
    if (!std::strcmp(op, "length")) {  // tokens of a gradient tile
      std::printf("%d\n", gm::kLoraGradTokens << gm::lora_grad_len(T, blocks));
    } else if (!std::strcmp(op, "fwd")) {  // columns of a block, and of its weights in LDS
      std::printf("%d/%d\n", gm::lora_up_span(w, int(parts), T, tiles, int(r), false),
                  gm::lora_up_cols(gm::lora_up_rank_tiles(int(r))));
    } else if (!std::strcmp(op, "dx")) {
      std::printf("%d/%d\n", gm::lora_up_span(in, 1, T, tiles, R, true), gm::lora_up_cols(gm::lora_up_rank_tiles(R)));
    } else {
      return 1;
    }
  }
  return 0;
}
