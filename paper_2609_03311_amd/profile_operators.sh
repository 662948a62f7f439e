#!/bin/bash
# Collect the rocprofv3 summaries of the operators around the attention, from
# 100 pairs through the Qwen3-8B-shaped layer with 8-bit products (12,900
# tokens; the bf16 layer runs beside it for comparison):
#   quant_layer_qwen3_8b_kernel_stats.txt   time of every kernel
#   k_product_qwen3_8b_pmc.txt              shader counters of the products
# and from one pair (129 tokens) through it:
#   k_product_one_pair_pmc.txt              shader and L2 counters of the products
# Raw output stays under $out, the summaries are written to $sum.
# usage: bash paper_2609_03311_amd/profile_operators.sh
set -o pipefail
R=$(cd "$(dirname "$0")/.." && pwd)
out=$R/gpurun_out/prof_operators
sum=$R/gpurun_out/summaries
mkdir -p "$out" "$sum"
me="bash paper_2609_03311_amd/profile_operators.sh"
layer="-m paper_2609_03311_amd.quant_layer --config qwen3_8b --steps 3 --pairs"
run="$layer 100" run1="$layer 1"
pm() { python3 -c "import sys; sys.path.insert(0, '$R'); from paper_2609_03311_amd import profiling as p; print(p.PMC_PASSES[$1])"; }
export TMPDIR=/tmp PYTHONPATH=$R
cd /tmp

step() {  # name, what to run, rocprofv3 options...
  local name=$1 what=$2
  shift 2
  echo "== $name" && timeout -k 10 -s KILL 200 rocprofv3 "$@" -d "$out/$name" \
    -o run --output-format csv -- python3 $what > "$out/$name.log" 2>&1
  local rc=$?
  tail -1 "$out/$name.log" | cut -c1-160
  return $rc
}

step stats "$run" --kernel-trace --stats &&
  step pmc_a "$run" --pmc $(pm 0) &&
  step pmc_b "$run" --pmc $(pm 1) &&
  step one_a "$run1" --pmc $(pm 0) &&
  step one_b "$run1" --pmc $(pm 1) &&
  step one_c "$run1" --pmc $(pm 2) || exit $?

P="python3 -m paper_2609_03311_amd.profiling"
cd "$R" &&
  $P stats "$out/stats" --sources operators \
    --command "$me (rocprofv3 --kernel-trace --stats -- python3 $run)" \
    > "$sum/quant_layer_qwen3_8b_kernel_stats.txt" &&
  $P pmc "$out/pmc_a" "$out/pmc_b" --sources operators --kernel "k_product<" \
    --command "$me (rocprofv3 --pmc <PMC_PASSES[0]>, then <PMC_PASSES[1]> -- python3 $run)" \
    > "$sum/k_product_qwen3_8b_pmc.txt" &&
  $P pmc "$out/one_a" "$out/one_b" "$out/one_c" --sources operators --kernel "k_product<" \
    --command "$me (rocprofv3 --pmc <PMC_PASSES[0]>, [1], [2] -- python3 $run1)" \
    > "$sum/k_product_one_pair_pmc.txt"
