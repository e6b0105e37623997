// Draft-tree attention on tcgen05, head size 256.
#include "tree_instances.cuh"

template int instinfer::api::launch_tree<256, false>(const TreeRows &, const TreeLaunch &);
template int instinfer::api::launch_tree<256, true>(const TreeRows &, const TreeLaunch &);
