// Host checks shared by the calls on a paged cache.
#pragma once

#include <cstdint>
#include <string>
#include <vector>

#include "../../include/t2vattn.h"
#include "t2v_host.h"

namespace t2v {

// Checks all that the struct says, pointers included (not against other tensors).
int check_pages(const t2v_pages* cache);

// Bytes from the first element of k's (v's) pages to behind the last.
int64_t pages_bytes(const t2v_pages& c, const int64_t (&strides)[3]);

// That n words at an input's address do not overlap any output.
int check_words_apart(const int32_t* words, int64_t n, const char* name, const std::vector<Range>& outputs);

// cu_seqlens' address, and that neither it nor the lengths nor the table overlap an output.
int check_tables_apart(const t2v_pages& c, const int32_t* cu_seqlens, const std::vector<Range>& outputs);

}  // namespace t2v
