// Draft-tree attention on tcgen05, head size 64.
#include "tree_instances.cuh"

template int instinfer::api::launch_tree<64, false>(const TreeRows &, const TreeLaunch &);
template int instinfer::api::launch_tree<64, true>(const TreeRows &, const TreeLaunch &);
