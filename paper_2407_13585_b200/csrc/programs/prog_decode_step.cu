// Generated by `python -m paper_2407_13585_b200.instantiate workloads:decode_step:5,4,2,16,64,4,10,7,100,12`.
// Every cluster of every legal clustering of the programs named above, and every node alone.
#include "device/launch.cuh"

namespace acc {

constexpr CProgram make_decode_step() {
  CProgram p{23, (1ull << 16) | (1ull << 18) | (1ull << 19) | (1ull << 20) | (1ull << 21) | (1ull << 22), {}};
  p.nodes[0] = pnode(ACC_INPUT, ACC_I32, 1, 0, 0, 0);
  p.nodes[1] = pnode(ACC_INPUT, ACC_I32, 1, 0, 0, 0);
  p.nodes[2] = pnode(ACC_INPUT, ACC_I32, 2, 0, 0, 0);
  p.nodes[3] = pnode(ACC_INPUT, ACC_F32, 2, 0, 0, 0);
  p.nodes[4] = pnode(ACC_INPUT, ACC_F32, 2, 0, 0, 0);
  p.nodes[5] = pnode(ACC_INPUT, ACC_F32, 2, 0, 0, 0);
  p.nodes[6] = pnode(ACC_INPUT, ACC_F32, 2, 0, 0, 0);
  p.nodes[7] = pnode(ACC_INPUT, ACC_F32, 2, 0, 0, 0);
  p.nodes[8] = pnode(ACC_INPUT, ACC_F32, 2, 0, 0, 0);
  p.nodes[9] = pnode(ACC_INPUT, ACC_I32, 2, 0, 0, 0);
  p.nodes[10] = pnode(ACC_INPUT, ACC_F32, 2, 0, 0, 0);
  p.nodes[11] = pnode(ACC_INPUT, ACC_I32, 2, 0, 0, 0);
  p.nodes[12] = pnode(ACC_INPUT, ACC_F32, 2, 0, 0, 0);
  p.nodes[13] = pnode(ACC_INPUT, ACC_U32, 2, 0, 0, 0);
  p.nodes[14] = pnode(ACC_MAP, ACC_I32, 1, ACC_FN_ADD_CONST, 0, 1, 0);  // lens
  p.nodes[15] = pnode(ACC_GENERATE, ACC_I32, 1, ACC_FN_IOTA, 0, 0);  // off
  p.nodes[16] = pnode(ACC_BLOCK_TABLE, ACC_I32, 2, 0, 0, 4, 14, 1, 0, 2);  // table
  p.nodes[17] = pnode(ACC_SLOT_MAP, ACC_I32, 1, 0, 0, 3, 16, 14, 15);  // new_slots
  p.nodes[18] = pnode(ACC_PUT_ROWS, ACC_F32, 2, 0, 0, 3, 6, 17, 4);  // new_keys
  p.nodes[19] = pnode(ACC_PUT_ROWS, ACC_F32, 2, 0, 0, 3, 7, 17, 5);  // new_values
  p.nodes[20] = pnode(ACC_PAGED_ATTENTION, ACC_F32, 2, 0, 0, 5, 3, 18, 19, 16, 14);  // out
  p.nodes[21] = pnode(ACC_PENALIZE, ACC_F32, 2, 0, 0, 6, 8, 9, 10, 11, 12, 13);  // penalized
  p.nodes[22] = pnode(ACC_FOLD, ACC_F32, 1, ACC_FN_MAX, 0, 1, 21);  // best
  return p;
}
inline constexpr CProgram k_decode_step = make_decode_step();
ACC_CLUSTER(k_decode_step, 0x4000, decode_step__lens)
ACC_CLUSTER(k_decode_step, 0x8000, decode_step__off)
ACC_CLUSTER(k_decode_step, 0x400000, decode_step__best)

}  // namespace acc
