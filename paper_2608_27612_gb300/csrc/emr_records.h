// The records of device-side waits that gave up, one of each translation unit that waits. Host only.
#pragma once

#include <stdint.h>

#include "../../include/emr.h"

namespace emr {

// Reads the first record that holds a number, and sets that one back. first, second: each reads a record into its argument and sets
// it back. What stands behind a number is not read, so that the next call tells of it.
template <typename First, typename Second>
emr_status first_record(First first, Second second, int32_t* code) {
  int32_t got = 0;
  emr_status ok = first(&got);
  if (ok == EMR_OK && got == 0) ok = second(&got);
  if (ok == EMR_OK) *code = got;
  return ok;
}

}  // namespace emr
