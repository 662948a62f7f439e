#!/bin/bash
# Collect the rocprofv3 summaries of the operators around the attention, from
# 100 pairs through the Qwen3-8B-shaped layer with 8-bit products (12,900
# tokens; the bf16 layer runs beside it for comparison):
#   quant_layer_qwen3_8b_kernel_stats.txt   time of every kernel
#   k_product_qwen3_8b_pmc.txt              shader counters of the products
# Raw output stays under $out, the summaries are written to $sum.
# usage: bash paper_2609_03311_amd/profile_operators.sh
set -o pipefail
R=$(cd "$(dirname "$0")/.." && pwd)
out=$R/gpurun_out/prof_operators
sum=$R/gpurun_out/summaries
mkdir -p "$out" "$sum"
me="bash paper_2609_03311_amd/profile_operators.sh"
run="-m paper_2609_03311_amd.quant_layer --config qwen3_8b --pairs 100 --steps 3"
pm() { python3 -c "import sys; sys.path.insert(0, '$R'); from paper_2609_03311_amd import profiling as p; print(p.PMC_PASSES[$1])"; }
export TMPDIR=/tmp PYTHONPATH=$R
cd /tmp

step() {  # name, rocprofv3 options...
  local name=$1
  shift
  echo "== $name" && timeout -k 10 -s KILL 200 rocprofv3 "$@" -d "$out/$name" \
    -o run --output-format csv -- python3 $run > "$out/$name.log" 2>&1
  local rc=$?
  tail -1 "$out/$name.log" | cut -c1-160
  return $rc
}

step stats --kernel-trace --stats &&
  step pmc_a --pmc $(pm 0) &&
  step pmc_b --pmc $(pm 1) || exit $?

P="python3 -m paper_2609_03311_amd.profiling"
cd "$R" &&
  $P stats "$out/stats" --sources operators \
    --command "$me (rocprofv3 --kernel-trace --stats -- python3 $run)" \
    > "$sum/quant_layer_qwen3_8b_kernel_stats.txt" &&
  $P pmc "$out/pmc_a" "$out/pmc_b" --sources operators --kernel "k_product<" \
    --command "$me (rocprofv3 --pmc <PMC_PASSES[0]>, then <PMC_PASSES[1]> -- python3 $run)" \
    > "$sum/k_product_qwen3_8b_pmc.txt"
