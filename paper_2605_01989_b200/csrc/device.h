// The device this library is built for.
#pragma once

namespace dblp {

constexpr unsigned kSms = 148;                // streaming multiprocessors

}  // namespace dblp
