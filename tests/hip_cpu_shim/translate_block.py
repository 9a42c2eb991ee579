"""Rewrite the HIP sources of a trained block so that a host C++ compiler accepts them (test infrastructure only).

As translate.py, which does the launches, and what these kernels use besides:

  __shared__ T name[A][B]...       a reference to an array of that type, so that every index is checked against its own bound;
                                  a kernel may have several
  address_space(...)              none
  the kernel's arguments          as the kernel has them, in place of the segment that they are in
  asm                             barriers, counts of copies that are waited for and copies to LDS become calls of the
                                  runtime (block_runtime.cpp); what only hides a value from the compiler goes
  what a wavefront hands itself through LDS, whose accesses are in the program's order there: the lanes wait for one another
  the rules that choose a tile    ask `shim::force` first, so that small shapes reach the kernels of every tile

A construct that is not found stops the translation: the sources have changed, and this has to follow."""
import re
import sys

import translate


def _shared(m):
    align, kind, name, dims = m.group(1) or "16", m.group(2), m.group(3), m.group(4)
    return f"auto &{name} = *static_cast<{kind} (*){dims}>(shim::block_shared(sizeof({kind}{dims}), {align}));"


_COPIES = [
    (r"#define CCDC_LDS .*", "#define CCDC_LDS", 1),
    (r"const uint32_t lds_at = \(uint32_t\)\(uintptr_t\)lds;", "const uint32_t lds_at = 0; shim::lds = memory;", 1),
    (r'asm volatile\("s_mov_b32 m0, %0[^;]*?dwordx4 %1, %2"[^;]*?"s"\(base\) : "memory"\);', "shim::copy_to_lds(to, (const char *)base + offset);", 1),
    (r'asm volatile\("s_mov_b32 m0, %0[^;]*?dword %1, %2"[^;]*?"s"\(base\) : "memory"\);', "shim::copy_words_to_lds(to, (const char *)base + offset);", 1),
    (r'asm volatile\("s_barrier" ::: "memory"\);', "shim::barrier_wait();", 1),
    (r'asm volatile\("s_waitcnt vmcnt\(%0\) lgkmcnt\(0\)" ::"n"\((.*?)\) : "memory"\);', r"shim::wait_copies(\1);", 4),
    (r'asm volatile\("s_waitcnt vmcnt\(0\) lgkmcnt\(0\)" ::: "memory"\);', "shim::wait_copies(0);", 2),
    (r'asm volatile\("s_waitcnt lgkmcnt\(0\)" ::: "memory"\);', "", 1),
]

# file: (pattern, replacement, how often at least)
RULES = {
    "vocabulary.hpp": [(r'asm volatile\("" : "\+v"\([\w\[\]]+\)\);', ";", 2)],
    "distill.hip": [(r"extern __shared__ __attribute__\(\(aligned\(16\)\)\) uint32_t mask\[\];", "uint32_t *mask = reinterpret_cast<uint32_t *>(shim::dyn_smem);", 1)],
    "eight.hip": [(r"return few_rows8\(b, a\) \?", "return shim::force < 0 && few_rows8(b, a) ?", 1)],
    "product8.hip": _COPIES + [
        (r"(?=\n#pragma unroll\n        for \(int q = 0; q < 4; q\+\+\) \{\n            const uint32_t row = q \* 8)", "\n        shim::wave_in_step();", 1),
        (r"if \(largest <= least\)", "if (shim::force >= 0 ? shim::force == 1 : largest <= least)", 1),
        (r"if \(small == least\)", "if (shim::force >= 0 ? shim::force == 2 : small == least)", 1),
        (r"if \(tall == least\)", "if (shim::force >= 0 ? shim::force == 3 : tall == least)", 1),
        (r"if \(one == least\)", "if (shim::force >= 0 ? shim::force == 4 : one == least)", 1),
    ],
    "element.hpp": [(r'asm volatile\("" : "\+[vs]"\(v\)\);', "", 2)],
    "join.hip": [(r"\(const __attribute__\(\(address_space\(4\)\)\) JoinArgs \*\)__builtin_amdgcn_kernarg_segment_ptr\(\)", "&a", 1)],
    "product.hip": [
        (r"#define CCDC_LDS .*", "#define CCDC_LDS", 1),
        (r"const uint32_t lds_at = \(uint32_t\)\(uintptr_t\)lds;", "const uint32_t lds_at = 0; shim::lds = memory;", 1),
        (r'asm volatile\("s_mov_b32 m0, %0[^;]*?"s"\(base\) : "memory"\);', "shim::copy_to_lds(to, (const char *)base + offset);", 1),
        (r'asm volatile\("s_mov_b32 m0, %0[^;]*?"v"\(from\) : "memory"\);', "shim::copy_to_lds(to, from);", 1),
        (r'asm volatile\("s_barrier" ::: "memory"\);', "shim::barrier_wait();", 1),
        (r'asm volatile\("s_waitcnt vmcnt\(%0\) lgkmcnt\(0\)" ::"n"\((.*?)\) : "memory"\);', r"shim::wait_copies(\1);", 4),
        (r'asm volatile\("s_waitcnt vmcnt\(0\) lgkmcnt\(0\)" ::: "memory"\);', "shim::wait_copies(0);", 2),
        (r'asm volatile\("s_waitcnt lgkmcnt\(0\)" ::: "memory"\);', "", 1),
        (r"// numbers 8 pack \.\.\. 8 pack \+ 7 of a row", "shim::wave_in_step();", 1),
        (r"return rounds\(256, 256\) \* time <= rounds\(128, 512\);", "return shim::force >= 0 ? shim::force == 1 : rounds(256, 256) * time <= rounds(128, 512);", 1),
        (r"rounds\(256\) \* 1\.6 <= rounds\(128\)", "(shim::force >= 0 ? shim::force == 1 : rounds(256) * 1.6 <= rounds(128))", 1),
        (r"if \(small > 256\)", "if (shim::force >= 0 ? shim::force == 2 : small > 256)", 1),
    ],
}


def translate_block(text, name):
    for pattern, new, least in RULES.get(name, []):
        text, count = re.subn(pattern, new, text, flags=re.S if "[^;]" in pattern else 0)
        if count < least:
            raise SystemExit(f"{name}: {pattern!r} found {count} times, not {least}")
    text = re.sub(r"__shared__\s+(?:__attribute__\(\(aligned\((\d+)\)\)\)\s+)?([\w ]+?)\s+(\w+)((?:\[[^\]]+\])+);", _shared, text)
    text = re.sub(r"__shared__\s+(\w+)\s+(\w+);", r"auto &\2 = *static_cast<\1 *>(shim::block_shared(sizeof(\1), 16));", text)
    text = translate.translate(text)
    code = re.sub(r"#ifdef __HIP_DEVICE_COMPILE__.*?#(else|endif)", "", re.sub(r"//.*", "", text), flags=re.S)
    for left in ("__shared__", "<<<", "asm volatile", "address_space"):
        if left in code:
            raise SystemExit(f"{name}: {left} is left")
    return text


if __name__ == "__main__":
    src, dst, name = sys.argv[1:4]
    with open(src) as fh:
        made = translate_block(fh.read(), name)
    with open(dst, "w") as fh:
        fh.write(made)
