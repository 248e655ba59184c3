// Body of a C entry that may run out of host memory while it puts a message
// together: no exception leaves it.
#pragma once

#include <string>

#include "../../include/sangam_attn.h"

namespace sangam {

void set_error(const std::string& msg);

template <typename Body>
sangam_status entry(Body&& body) noexcept {
    try {
        return body();
    } catch (...) {
        try {
            set_error("no host memory");  // (as short as a string that takes none)
        } catch (...) {
        }
        return SANGAM_ERR_MEMORY;
    }
}

}  // namespace sangam
