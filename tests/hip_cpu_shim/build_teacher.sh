#!/bin/bash
# usage: build_teacher.sh <source dir with the .hip/.cpp files> <output dir> [extra compiler flags]
# As build_block.sh, for the kernels that learn from a teacher.
set -e
here=$(cd "$(dirname "$0")" && pwd)
src=$1; out=$2; shift 2
mkdir -p "$out"
names="block eight few8 product8 top distill"
for f in $names; do python3 "$here/translate_block.py" "$src/$f.hip" "$out/${f}_hip.cpp" $f.hip; done
for f in common.hpp element.hpp eight.hpp vocabulary.hpp; do python3 "$here/translate_block.py" "$src/$f" "$out/$f" $f; done     # found first by the translated sources
CXX=${SHIM_CXX:-/opt/rocm/lib/llvm/bin/clang++}
FLAGS="-std=c++20 -gline-tables-only -fno-omit-frame-pointer -fsanitize=address,undefined -fno-sanitize-recover=undefined -pthread -I $here -I $out -I $here/../../include -I $src -Wno-unknown-attributes -Wno-pass-failed -Wno-psabi"
pids=""
for f in $names; do $CXX $FLAGS -O0 -include "$here/teacher_lanes.hpp" "$@" -c "$out/${f}_hip.cpp" -o "$out/${f}_hip.o" & pids="$pids $!"; done
for f in "$src/block.cpp" "$here/block_runtime.cpp" "$here/teacher_driver.cpp"; do $CXX $FLAGS -O2 "$@" -c "$f" -o "$out/$(basename "$f").o" & pids="$pids $!"; done
for p in $pids; do wait $p; done
$CXX $FLAGS "$out"/*.o -o "$out/teacher_driver"
echo "$out/teacher_driver"
