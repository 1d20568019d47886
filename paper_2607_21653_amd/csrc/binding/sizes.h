// Whether a call takes these numbers: what the entries of the same names check before all else, for calls.cpp,
// which makes a call's outputs and asks first. 0, or the entry's error with its words (molt_last_error).
#pragma once

extern "C" {
int molt_plan_blocks_takes(int B, int n, int max_blocks, int num_blocks);
int molt_key_bounds_read_takes(int M, int n_kv_heads, int head_dim, int num_blocks);
int molt_select_blocks_takes(int B, int k, int n_q_heads, int n_kv_heads, int head_dim, int max_blocks, int num_blocks,
                             int n_select, int n_first, int n_last);
int molt_paged_attention_blocks_takes(int B, int k, int n_q_heads, int n_kv_heads, int head_dim, int max_blocks,
                                      int num_blocks, int n_list);
}
