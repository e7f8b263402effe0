// The decoder's host side with a way for the library's other files to set
// lb_last_error's message, which is lb_api.cpp's own: one translation unit.
#include "lb_api.cpp"

namespace lb {
lb_status set_last_error(lb_status st, const std::string& msg) { return fail(st, msg); }
}  // namespace lb
