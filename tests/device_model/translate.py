"""Turns the library's CUDA sources into one C++ file that runs on the host (model.hpp)."""
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
CSRC = os.path.join(ROOT, "paper_1905_10988_b200", "csrc")


def _read(name):
    with open(os.path.join(CSRC, name)) as f:
        return f.read()


def _functions(text):
    """(begin, end, name, body) of the function definitions outside other functions."""
    for m in re.finditer(r"^(?:template <[^\n]*>\s*)?(?:__[a-z_]+__ |inline |static )+[^;{}()]*?"
                         r"\b(\w+)\(", text, re.M):
        at = text.index("(", m.end() - 1)
        depth = 0
        while True:
            depth += {"(": 1, ")": -1}.get(text[at], 0)
            at += 1
            if depth == 0:
                break
        rest = re.match(r"\s*(?:const)?\s*\{", text[at:])
        if not rest:
            continue
        end = at + rest.end()
        depth = 1
        while depth:
            depth += {"{": 1, "}": -1}.get(text[end], 0)
            end += 1
        yield m.start(), end, m.group(1), text[m.start():end]


def _without(text, names=(), instructions=False):
    """`text` without the functions called `names`, and, instructions, those that hold assembly"""
    cut = [(b, e) for b, e, name, body in _functions(text)
           if name in names or (instructions and re.search(r"\basm\b", body))]
    for b, e in reversed(cut):
        text = text[:b] + text[e:]
    return text


def _shared(text):
    """__shared__ declarations -> references into the running block's memory"""
    text = re.sub(r"extern __shared__ (\w+) (\w+)\[\];",
                  r"\1* \2 = reinterpret_cast<\1*>(model::dynamic_memory());", text)
    count = [0]

    def one(m):
        out = []
        depth, item, items = 0, "", []
        for ch in m.group(2) + ",":
            depth += {"[": 1, "]": -1, "(": 1, ")": -1, "{": 1, "}": -1}.get(ch, 0)
            if ch == "," and depth == 0:
                items.append(item.strip())
                item = ""
            else:
                item += ch
        for it in items:
            name, dims = re.match(r"(\w+)(.*)", it, re.S).groups()
            count[0] += 1
            out.append("typedef %s %s_shared%s; %s_shared& %s = *reinterpret_cast<%s_shared*>("
                       "model::static_memory(%d, sizeof(%s_shared)));"
                       % (m.group(1), name, dims, name, name, name, count[0], name))
        return " ".join(out)

    return re.sub(r"__shared__ (?:__align__\(16\) )?(\w+)\s+([^;]+);", one, text)


MODEL_PAIRS = """
typedef unsigned long long f32x2;
static inline f32x2 pair_of(float lo, float hi) {
    return (f32x2)__float_as_uint(hi) << 32 | __float_as_uint(lo);
}
static inline void of_pair(f32x2 v, float& lo, float& hi) {
    lo = __uint_as_float((uint32_t)v);
    hi = __uint_as_float((uint32_t)(v >> 32));
}
template <typename F> static inline f32x2 model_pairwise(f32x2 a, f32x2 b, f32x2 c, F f) {
    float a0, a1, b0, b1, c0, c1;
    of_pair(a, a0, a1); of_pair(b, b0, b1); of_pair(c, c0, c1);
    return pair_of(f(a0, b0, c0), f(a1, b1, c1));
}
static inline f32x2 add2(f32x2 a, f32x2 b) {
    return model_pairwise(a, b, 0, [](float x, float y, float) { return x + y; });
}
static inline f32x2 mul2(f32x2 a, f32x2 b) {
    return model_pairwise(a, b, 0, [](float x, float y, float) { return x * y; });
}
static inline f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
    return model_pairwise(a, b, c, [](float x, float y, float z) { return fmaf(x, y, z); });
}
static inline float max3_abs(float a, float b, float c) {
    if (isnan(a) || isnan(b) || isnan(c)) return NAN;
    return fmaxf(fabsf(a), fmaxf(fabsf(b), fabsf(c)));
}
static inline Bytes32 ld_bytes32(const void* p, bool wide) {
    if ((uintptr_t)p % (wide ? 32 : 16)) model::fail("load that is not aligned");
    return *static_cast<const Bytes32*>(p);
}
static inline void st_bytes32(void* p, const Bytes32& r, bool wide) {
    if ((uintptr_t)p % (wide ? 32 : 16)) model::fail("store that is not aligned");
    *static_cast<Bytes32*>(p) = r;
}
"""


def _clean(text):
    text = re.sub(r'#include[^\n]*\n', "", text).replace("#pragma once", "")
    text = re.sub(r'asm\("sub\.rn\.bf16x2.*?\);', "v = model::sub_bf16x2(a, b);", text, flags=re.S)
    text = re.sub(r'asm volatile\("bar\.sync (\d+), %0;" ::"r"\((.*?)\) : "memory"\);',
                  r"model::named_barrier(\1, \2);", text)
    text = re.sub(r'asm volatile\("bar\.sync %0, %1;" ::"r"\((.*?)\), "r"\((.*?)\) : "memory"\);',
                  r"model::named_barrier(\1, \2);", text)
    text = text.replace('asm volatile("");', "")
    text = re.sub(r"(\w+)<<<(.*?)>>>\(", r"model::chevrons(\1, \2)(", text, flags=re.S)
    text = re.sub(r"__launch_bounds__\(.*?\)\n(?=\w+\(|__)", "", text)
    text = re.sub(r"__launch_bounds__\((?:[^()]|\([^()]*\))*\)", "", text)
    text = re.sub(r"__cluster_dims__\([^)]*\)", "", text)
    text = text.replace("__grid_constant__", "")
    assert not re.search(r"\basm\b", text), re.search(r".*\basm\b.*", text).group(0)
    return _shared(text)


def translate(sources, constants=None, change=None):
    """The text of the C++ file: the sources of csrc with their entry points.  constants: other values
    of integer constants, by name.  change: a function of (file, text), for a test that wants to see
    another text fail."""
    change = change or (lambda name, text: text)
    common = _without(change("common.cuh", _read("common.cuh")), ["launch_overlapping"], True)
    common = re.sub(r"#ifdef NC_BOUNDS.*?#else", "#if 1", common, flags=re.S)
    core = _without(change("tensor_core.cuh", _read("tensor_core.cuh")),
                    ["smem_u32", "mma_operand", "mma_shape", "make_tensor_map"], True)
    act8 = change("act8_common.cuh", _read("act8_common.cuh"))
    act8 = re.sub(r"typedef unsigned long long f32x2;", MODEL_PAIRS, act8)
    keep = {"act8_pair_bf16"}
    cut = [(b, e) for b, e, name, body in _functions(act8)
           if re.search(r"\basm\b", body) and name not in keep]
    for b, e in reversed(cut):
        act8 = act8[:b] + act8[e:]
    parts = [common, _read("philox.cuh"), act8, core]
    # the vector accesses stand before their use
    head = act8.index("struct Bytes32")
    end = act8.index("};", head) + 2
    stub = act8[:end] + """
static inline Bytes32 ld_bytes32(const void* p, bool wide);
static inline void st_bytes32(void* p, const Bytes32& r, bool wide);
""" + act8[end:]
    parts[2] = stub
    for name in sources:
        parts.append(change(name, _read(name)))
    text = "\n".join(_clean(p) for p in parts)
    for name, value in (constants or {}).items():
        text, n = re.subn(r"(constexpr \w+ %s = )\d+;" % name, r"\g<1>%d;" % value, text)
        assert n == 1, name
    return '#include "model.hpp"\n' + text
