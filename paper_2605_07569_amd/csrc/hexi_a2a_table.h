// Slot table of the head redistribution: one slot per (rank, head of that rank's list), in send-buffer order.
#pragma once
#include "hexi_attn.h"

struct A2ATable {
    int n_slots;
    unsigned short head[HEXI_A2A_MAX_SLOTS];        // head index in x
    unsigned short n_j[HEXI_A2A_MAX_SLOTS];         // heads of the slot's rank
    unsigned short local[HEXI_A2A_MAX_SLOTS];       // index of the head within its rank's list
    unsigned short heads_before[HEXI_A2A_MAX_SLOTS];   // heads of all earlier ranks
};

inline void hexi_build_a2a_table(int n_ranks, const int* heads_per_rank, const int* head_list, A2ATable* tb)
{
    int slot = 0, before = 0;
    for (int j = 0; j < n_ranks; ++j) {
        for (int i = 0; i < heads_per_rank[j]; ++i, ++slot) {
            tb->head[slot] = (unsigned short)head_list[slot];
            tb->n_j[slot] = (unsigned short)heads_per_rank[j];
            tb->local[slot] = (unsigned short)i;
            tb->heads_before[slot] = (unsigned short)before;
        }
        before += heads_per_rank[j];
    }
    tb->n_slots = slot;
}
