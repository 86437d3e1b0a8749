// What the products keep on a device.
#pragma once

#include <mutex>

#include "as_fp8.h"

constexpr int MAX_PARTS = 8;                 // CTAs that may share a tile

struct as_fp8_context_s {
  int device = -1, sms = 0;
  int clusters[MAX_PARTS + 1] = {};          // of so many CTAs that the device holds at once
  uint32_t* status = nullptr;
  std::mutex reading;                        // of the word behind the status word, where a read leaves what it took
};
