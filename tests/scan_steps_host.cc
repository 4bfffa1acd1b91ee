// Byte offsets of a scan's steps (csrc/dgc_steps.h), compared in 64 bits with where the rows are: a lane's own steps lie in
// their rows, and whatever else it asks for behind the buffer's end, at every accepted stride.
#include "dgc_steps.h"

#include <cstdio>
#include <vector>

using dgc::StepOffsets;

namespace {

struct Shape {
  int element, vec, groups, steps;
};

long checked = 0;

bool check(const Shape& shape, uint64_t stride_elements, uint64_t column) {
  const uint64_t stride = stride_elements * shape.element, wide = (uint64_t)shape.element * shape.vec;
  for (int rows = 0; rows <= shape.groups * shape.steps; ++rows) {
    const uint64_t end = (uint64_t)rows * stride;
    if (StepOffsets::buffer_bytes(rows, (uint32_t)stride) != end || end > 0x7fffffffu) return false;
    for (int group = 0; group < shape.groups; ++group) {
      const int left = rows - group * shape.steps, mine = left < 0 ? 0 : left > shape.steps ? shape.steps : left;
      for (int steps : {0, mine}) {  // none of a lane whose channels are not there
        const StepOffsets at(steps, group * shape.steps, (uint32_t)(column * shape.element), (uint32_t)stride);
        for (int i = 0; i < shape.steps; ++i, ++checked) {
          const uint64_t got = at.at(i);
          if (i < steps ? got != (uint64_t)(group * shape.steps + i) * stride + column * shape.element || got + wide > end : got < end) {
            std::printf("element %d x %d, %d groups of %d, stride %llu, %d rows: group %d with %d steps, step %d at %llu of %llu\n", shape.element,
                        shape.vec, shape.groups, shape.steps, (unsigned long long)stride_elements, rows, group, steps, i,
                        (unsigned long long)got, (unsigned long long)end);
            return false;
          }
        }
      }
    }
  }
  return true;
}

}  // namespace

int main() {
  const std::vector<Shape> shapes = {{2, 4, 2, 8}, {2, 2, 1, 16}, {2, 1, 1, 16}, {4, 2, 2, 8}, {4, 1, 1, 16}};
  const uint64_t most = (uint64_t)dgc::kWidthLimit - 1;
  std::vector<uint64_t> strides = {1, 2, 3, 64, 1500, 4473924, 4473925, 4500001, 8947848, 8947849, 9586980, 9586981, most - 3, most};
  for (uint64_t s = 4001; s < most; s += 99991) strides.push_back(s);
  for (const Shape& shape : shapes)
    for (uint64_t stride : strides) {
      stride = stride / shape.vec * shape.vec;
      if (stride == 0) continue;
      for (uint64_t column : {(uint64_t)0, stride / 2 / shape.vec * shape.vec, stride - shape.vec})
        if (!check(shape, stride, column)) return 1;
    }
  std::printf("ok %ld offsets\n", checked);
  return 0;
}
