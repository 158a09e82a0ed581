// errors.hpp -- what the entry points without a handle report.
#pragma once

namespace moe {

// Keeps `msg` for moe_stage_last_error(NULL) and returns `code`.  Throws nothing: without the memory
// for a message there is none.
int record_error(int code, const char* what, const char* msg) noexcept;

}  // namespace moe
