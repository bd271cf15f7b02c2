// Host helpers of the C-ABI layer, shared by its source files.
#pragma once

#include "common.h"
#include "errors.h"

namespace parrot {

// The checks of a problem's own fields (and their combinations) that every entry
// point makes, without the bound on group members that row counts replace.
parrot_status check_problem_fields(const parrot_problem* p);
// Compute units of the current device (cached; no device sync).
int device_cus();
// PARROT_OK, or an error that names the pointer: NULL, or not `align`-byte aligned.
struct PtrCheck { const void* ptr; const char* name; size_t align; };
template <size_t N>
parrot_status check_pointers(const PtrCheck (&list)[N]) {
  for (const PtrCheck& c : list) {
    if (!c.ptr) return set_error(PARROT_ERR_INVALID_ARGUMENT, "%s is NULL", c.name);
    if (reinterpret_cast<uintptr_t>(c.ptr) % c.align)
      return set_error(PARROT_ERR_INVALID_ARGUMENT, "%s is not %zu-byte aligned", c.name, c.align);
  }
  return PARROT_OK;
}
// The device-side content check behind the validate entry points.  `rows` NULL: a
// decode call; `tree` not NULL: a tree call (offsets may end below the row count), whose
// drafted rows' parents `tree->parents` (may be NULL) are checked too.
struct ValidateTree { const int32_t* parents; };
parrot_status validate_inputs(const parrot_problem* p, const int32_t* prefix_block_tables,
                              const int32_t* prefix_lens, const int32_t* prefix_parents,
                              const int32_t* suffix_block_tables, const int32_t* suffix_lens,
                              const int32_t* group_ids, int32_t* scratch, void* stream,
                              const parrot_prefill_rows* rows, const int32_t* query_offsets,
                              const ValidateTree* tree);

// Fills of new rows: the checks of their counts, those of the other arguments but for the
// cache with the kernels' arguments and how partners come, and the split of their heads.
struct FillArgs;
parrot_status check_fill(const parrot_problem* p, const parrot_fill_rows* rows);
parrot_status fill_args(const parrot_problem* p, const parrot_fill_rows* rows, const parrot_rotary* rotary, const void* q,
                        const void* k, const void* v, const void* q_norm, const void* k_norm, const int32_t* positions,
                        const int32_t* query_offsets, const int32_t* suffix_block_tables, const int32_t* suffix_lens,
                        void* q_out, FillArgs* out, int* partner);
void fill_slabs(FillArgs* a, long step, long items);

}  // namespace parrot
