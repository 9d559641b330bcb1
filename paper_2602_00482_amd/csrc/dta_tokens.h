// Token tables of a tree (dta_tokens_t): host build and what the kernels of the vocabulary ends read.
// Not part of the public interface.
#pragma once

#include <cstddef>
#include <cstdint>
#include <mutex>
#include <vector>

#include "dta.h"

namespace dta {

// Rows of d_x that one block of the embedding gradient sums: an id with more tokens than this is summed in parts,
// side by side, so that the most frequent token of a batch (several per cent of it) is not one block's work.
constexpr int kPartTokens = 64;
// The row list is padded to whole tiles of rows by repeating its last entry.
constexpr int kRowPad = 256;

// Tokens order[begin, end) have id `id`.  slot < 0: all of them, the sum is the gradient's row;
// otherwise the sum is partial sum `slot`.
struct EmbedPart {
  int32_t id, begin, end, slot;
};
// The row of id `id` is the sum of partial sums [first, first + n).
struct EmbedMerge {
  int32_t id, first, n, pad;
};

// The tables on a device, pointers into one block.
struct TokenTables {
  const int32_t* id;          // [T]
  const int32_t* slot;        // [T]  place of a row in `row`, -1: before no scored token
  const int32_t* before;      // [T]  row before the token if it is scored, -1 otherwise
  const int32_t* row;         // [R padded to kRowPad]
  const int32_t* edge_ptr;    // [R padded + 1]  scored tokens after row r: edges [edge_ptr[r], edge_ptr[r+1])
  const int32_t* only;        // [R padded]  the id of the one scored token after row r; -1: none (padding), -2: several
  const int32_t* edge_token;  // [N]  by row, within a row by id
  const int32_t* edge_id;     // [N]
  const int32_t* order;       // [T]  tokens by id
  const EmbedPart* part;
  const EmbedMerge* merge;
  const uint32_t* present;    // [ceil(V / 32)]  bit v % 32 of word v / 32: id v occurs
};

}  // namespace dta

struct dta_tokens {
  int64_t n_tokens = 0, n_distinct = 0;
  int32_t vocab = 0;
  std::vector<int32_t> before;   // [T] row before each token
  std::vector<int32_t> rows;     // [R]
  int64_t n_scored = 0;
  int32_t n_parts = 0, n_merges = 0, n_slots = 0;
  // the device tables as one block of int32, and where each begins (256-byte steps)
  std::vector<int32_t> table;
  struct Begin {
    size_t id, slot, before, row, edge_ptr, only, edge_token, edge_id, order, part, merge, present;
  } at{};
  struct Copy {
    int device;
    void* block;
    size_t cap;
  };
  std::vector<Copy> copies;   // one per device the tables were used on
  // per stream that was used an event (hipEvent_t) that completes after the latest call on it
  struct Use {
    void* stream;
    uint64_t thread;   // where the handle means another stream in every thread, the number of this one; 0 elsewhere
    int device;
    void* event;
  };
  std::vector<Use> uses;
  std::mutex mu;

  int64_t n_rows() const { return (int64_t)rows.size(); }
  int64_t rows_padded() const { return (n_rows() + dta::kRowPad - 1) / dta::kRowPad * dta::kRowPad; }
};

namespace dta {

int validate_vocab_params(const dta_vocab_params_t* p);

}  // namespace dta
