// The text of the last failure of a call without a context (first_last_error(NULL)), of this host thread.
#pragma once
#include <string>

namespace first {
extern thread_local std::string g_create_error;
}
