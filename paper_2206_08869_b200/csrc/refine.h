// The refinement of a level's prior parameters that a codec applies (include/iodf.h: iodf_codec_set_refinement).
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "../../include/iodf.h"

namespace iodf {

struct Refinement {
  iodf_refinement parts{};
  uint64_t channels = 0, pixels = 0;      // of the level's factored-out block
  void *mem = nullptr, *n = nullptr, *u = nullptr, *b = nullptr;
  size_t ldn = 0, ldu = 0, ldb = 0;
  int32_t* start = nullptr;               // first row of each image
  int8_t* h = nullptr;                    // the projections' workspace: theirs serves the calls of their owner
  int* row_slot = nullptr;
  uint32_t* status = nullptr;             // the codec's words for this level: [0] a bounded wait gave up, [1] bad adapter slots
};

// A status. `out` must be empty; nothing is left in it after an error. status: two words of the device, zero.
int refinement_create(const iodf_refinement& parts, int device, uint64_t channels, uint64_t pixels, uint32_t max_batch, uint32_t* status,
                      Refinement* out);
void refinement_free(Refinement* r);
// mu: the level's first mean of image 0; image_stride: values from one image to the next.
int refinement_run(const Refinement& r, int32_t* mu, uint64_t image_stride, int batch, void* stream);

}  // namespace iodf
