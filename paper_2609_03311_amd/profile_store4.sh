#!/bin/bash
# Collect the rocprofv3 summaries of the kernels of a 4-bit store, from the
# Qwen3-8B-shaped layer that fills it and runs pairs over it:
#   store4_qwen3_8b_kernel_stats.txt   time of every kernel, 1,600 pairs of 129
#                                      tokens
#   store4_tokens_qwen3_8b_kernel_stats.txt   the same, 4,000 pairs of one token
#   k_rows_fp4_qwen3_8b_pmc.txt        shader counters of the many tokens'
#   k_token_fp4_qwen3_8b_pmc.txt       kernels, and of the single tokens'
# Raw output stays under $out, the summaries are written to $sum.
# usage: bash paper_2609_03311_amd/profile_store4.sh
set -o pipefail
R=$(cd "$(dirname "$0")/.." && pwd)
out=$R/gpurun_out/prof_store4
sum=$R/gpurun_out/summaries
mkdir -p "$out" "$sum"
me="bash paper_2609_03311_amd/profile_store4.sh"
layer="-m paper_2609_03311_amd.quant_layer --config qwen3_8b --store fp4 --steps 3"
many="$layer --pairs 1600" one="$layer --pairs 4000 --tokens 1"
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

step many "$many" --kernel-trace --stats &&
  step one "$one" --kernel-trace --stats &&
  step many_a "$many" --pmc $(pm 0) &&
  step many_b "$many" --pmc $(pm 1) &&
  step one_a "$one" --pmc $(pm 0) &&
  step one_b "$one" --pmc $(pm 1) || exit $?

P="python3 -m paper_2609_03311_amd.profiling"
cd "$R" &&
  $P stats "$out/many" --sources store4 \
    --command "$me (rocprofv3 --kernel-trace --stats -- python3 $many)" \
    > "$sum/store4_qwen3_8b_kernel_stats.txt" &&
  $P stats "$out/one" --sources store4 \
    --command "$me (rocprofv3 --kernel-trace --stats -- python3 $one)" \
    > "$sum/store4_tokens_qwen3_8b_kernel_stats.txt" &&
  $P pmc "$out/many_a" "$out/many_b" --sources store4 \
    --kernel "k_rows_fp4<|k_own_keys<|k_put_states<" \
    --command "$me (rocprofv3 --pmc <PMC_PASSES[0]>, then <PMC_PASSES[1]> -- python3 $many)" \
    > "$sum/k_rows_fp4_qwen3_8b_pmc.txt" &&
  $P pmc "$out/one_a" "$out/one_b" --sources store4 --kernel "k_token_fp4<" \
    --command "$me (rocprofv3 --pmc <PMC_PASSES[0]>, then <PMC_PASSES[1]> -- python3 $one)" \
    > "$sum/k_token_fp4_qwen3_8b_pmc.txt"
