// Draft-tree attention on tcgen05, head size 128.
#include "tree_instances.cuh"

template int instinfer::api::launch_tree<128, false>(const TreeRows &, const TreeLaunch &);
template int instinfer::api::launch_tree<128, true>(const TreeRows &, const TreeLaunch &);
