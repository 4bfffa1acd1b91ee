// Where the sequences and steps of a scan lie in its arrays: plain arithmetic, for the host too.
#ifndef DGC_STEPS_H_
#define DGC_STEPS_H_

#include <stdint.h>

namespace dgc {

constexpr int64_t kWidthLimit = (int64_t)1 << 24;  // channels and row strides of a scan: offsets inside a tile take 32 bits
constexpr int kWaveRows = 16;                      // a wavefront's at most, and so a lane's

// Rows [begin, begin + length) of a sequence whose offsets are `lo` and `hi`, cut to the arrays and to max_length whatever
// these are.
struct SequenceRows {
  int64_t begin, length;
  constexpr SequenceRows(int64_t lo, int64_t hi, int64_t rows, int64_t max_length) : begin(inside(lo, rows)), length(inside(hi, rows) - begin) {
    length = length < 0 ? 0 : length > max_length ? max_length : length;
  }
  static constexpr int64_t inside(int64_t row, int64_t rows) { return row < 0 ? 0 : row > rows ? rows : row; }
};

// Byte offsets of a lane's steps in the buffer of its wavefront's rows, which holds rows * stride bytes.  A lane asks for
// all the steps of its shape, also for those that it does not have: these have to lie behind the buffer's end, where nothing
// is read or stored, however wide the rows are.
struct StepOffsets {
  uint32_t first, stride;
  // `steps` of the lane's are there, the first one is row `row` of the buffer, `column` bytes in
  constexpr StepOffsets(int steps, int row, uint32_t column, uint32_t stride_)
      : first(steps > 0 ? (uint32_t)row * stride_ + column : kNowhere), stride(stride_) {}
  constexpr uint32_t at(int step) const { return first + (uint32_t)step * stride; }
  static constexpr uint32_t buffer_bytes(int rows, uint32_t stride) { return (uint32_t)rows * stride; }

  // For a lane without steps: not before the largest buffer's end, and its last step does not pass 32 bits.
  static constexpr uint32_t kNowhere = 0x80000000u;
};
static_assert(kWaveRows * kWidthLimit * 4 <= StepOffsets::kNowhere, "a lane without steps starts behind every buffer");
static_assert(StepOffsets::kNowhere + (kWaveRows - 1) * kWidthLimit * 4 < (int64_t)1 << 32, "and its steps stay there");

}  // namespace dgc
#endif  // DGC_STEPS_H_
