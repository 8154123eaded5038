// The text of a failing call that has no context (flover_last_error(NULL)), for the files of the C ABI.
#pragma once
#include <string>

namespace flk {
int fail_call(int code, const std::string& msg);     // records msg for the calling thread, returns code
}
