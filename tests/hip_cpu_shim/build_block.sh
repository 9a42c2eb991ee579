#!/bin/bash
# usage: build_block.sh <source dir with the .hip/.cpp files> <output dir> [extra compiler flags]
# Translates the HIP sources of a trained block, compiles them with their driver for the host under ASan + UBSan.
set -e
here=$(cd "$(dirname "$0")" && pwd)
src=$1; out=$2; shift 2
mkdir -p "$out"
for f in block.hip few.hip ffn.hip join.hip product.hip; do
  python3 "$here/translate_block.py" "$src/$f" "$out/${f%.hip}_hip.cpp" $f
done
for f in common.hpp element.hpp product.hpp; do python3 "$here/translate_block.py" "$src/$f" "$out/$f" $f; done     # found first by the translated sources
CXX=${SHIM_CXX:-/opt/rocm/lib/llvm/bin/clang++}
FLAGS="-std=c++20 -gline-tables-only -fno-omit-frame-pointer -fsanitize=address,undefined -fno-sanitize-recover=undefined -pthread -I $here -I $out -I $here/../../include -I $src -Wno-unknown-attributes -Wno-pass-failed -Wno-psabi"
pids=""
for f in block few ffn join; do $CXX $FLAGS -O0 -include "$here/block_lanes.hpp" "$@" -c "$out/${f}_hip.cpp" -o "$out/${f}_hip.o" & pids="$pids $!"; done
for i in 0 1 2; do $CXX $FLAGS -O0 -DCCDC_PRODUCT_PART=$i -include "$here/block_lanes.hpp" "$@" -c "$out/product_hip.cpp" -o "$out/product_hip_$i.o" & pids="$pids $!"; done
for f in "$src/block.cpp" "$here/block_runtime.cpp" "$here/block_driver.cpp"; do $CXX $FLAGS -O2 "$@" -c "$f" -o "$out/$(basename "$f").o" & pids="$pids $!"; done
for p in $pids; do wait $p; done
$CXX $FLAGS "$out"/*.o -o "$out/block_driver"
echo "$out/block_driver"
