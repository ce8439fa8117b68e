// Which pages a compaction moves where (host only).
#pragma once
#include <cstdint>
#include <vector>

namespace bs {
// named[i]: whether page i is live.  Every live page from the number of live pages on moves to the smallest hole below it, both in
// ascending order: src -> dst, and to[i] for every page.  Returns the number of live pages.
int32_t plan_compaction(const std::vector<char> &named, std::vector<int32_t> &to, std::vector<int32_t> &src, std::vector<int32_t> &dst);
}  // namespace bs
