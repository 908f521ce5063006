"""The product of large tiles keeps its accumulators in accumulation registers and multiplies in inline assembly, for which the
compiler counts no wait states, and the kernel that walks over tiles waits for loads by how many memory operations it
started since.  What the sources rely on, checked on the assembly of all such kernels (no GPU needed)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2508_18182_amd import build as B

FENCE = ("s_nop", "15")


@pytest.fixture(scope="module")
def text(tmp_path_factory):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not shutil.which(hipcc):
        pytest.skip("no hipcc")
    asm = tmp_path_factory.mktemp("asm") / "k.s"
    subprocess.run([hipcc, *B.HIPCC_FLAGS, "-I", os.path.join(B.ROOT, "include"), "-I", B.CSRC, "-S", "--offload-device-only",
                    os.path.join(B.CSRC, "block8_kernels.hip"), "-o", str(asm)], check=True, capture_output=True)
    return asm.read_text()


def bodies(text, shape):
    """{name: assembly} of the product kernels whose template arguments begin with `shape`."""
    return dict(re.findall(r"^(_Z\S*product_tile_kernelI%s\S*):.*?\n(.*?)^\.Lfunc_end" % shape, text, re.M | re.S))


PINNED = "Li8ELi8ELb0E"                # 256 x 256, products by the 8-bit instruction
WALKING, STANDING = PINNED + "Lb1E", PINNED + "Lb0E"


def registers(word, kind):
    m = re.fullmatch(r"%s\[(\d+):(\d+)\]" % kind, word) or re.fullmatch(r"%s(\d+)" % kind, word)
    return set(range(int(m[1]), int(m[m.lastindex]) + 1)) if m else set()


def graph(body):
    """(blocks, followers): label -> [(inline, words)] in the order of the text, label -> labels that may come next."""
    inside, blocks, label = False, {"": []}, ""
    for line in body.splitlines():
        if "#ASMSTART" in line or "#ASMEND" in line:
            inside = "#ASMSTART" in line
            continue
        code = line.split(";")[0].replace(",", " ").split()
        if code and code[0].endswith(":"):
            label = code[0][:-1]
            blocks[label] = []
        elif code and not code[0].startswith("."):
            blocks[label].append((inside, code))
            if code[0].startswith("s_cbranch"):
                label += "'"
                blocks[label] = []
    names = list(blocks)
    follows = {n: [c[1] for _, c in blocks[n] if c[0].startswith(("s_branch", "s_cbranch"))] for n in names}
    for n, after in zip(names, names[1:]):
        if not blocks[n] or blocks[n][-1][1][0] not in ("s_branch", "s_endpgm"):
            follows[n].append(after)
    return blocks, follows


def walk(body, step, join):
    """Runs step(state, inline, words) -> state over every path, states joined where paths meet; a state of None: not reached."""
    blocks, follows = graph(body)
    entering, todo = {n: None for n in blocks}, [next(iter(blocks))]
    entering[todo[0]] = {}
    while todo:
        n = todo.pop()
        state = dict(entering[n])
        for inline, code in blocks[n]:
            state = step(state, inline, code)
        for m in follows[n]:
            both = dict(state) if entering[m] is None else join(entering[m], state)
            if both != entering[m]:
                entering[m] = both
                todo.append(m)


def operands_too_fresh(body, least=2):
    """Inline MFMAs that read a vector register which a vector instruction wrote fewer than `least` wait states before."""
    found = set()

    def step(age, inline, code):                       # register -> wait states since it was written
        if code[0].startswith("v_mfma"):
            if inline:
                for w in code[2:]:
                    if any(age.get(r, least) < least for r in registers(w, "v")):
                        found.add(" ".join(code))
            written = set()
        else:
            written = registers(code[1], "v") if code[0].startswith("v_") and len(code) > 1 else set()
        states = int(code[1]) + 1 if code[0] == "s_nop" else 1
        age = {r: n + states for r, n in age.items() if n + states < least}
        age.update({r: 0 for r in written})
        return age

    walk(body, step, lambda x, y: {r: min(x.get(r, least), y.get(r, least)) for r in x.keys() | y.keys()})
    return found


def accumulators_unfenced(body):
    """What touches an accumulation register: reads of one that an MFMA wrote, or MFMAs on one that was written otherwise, with no
    fence in between; and anything but writes from outside the assembly.  (violations, MFMAs, reads)"""
    found, seen = set(), {"mfma": set(), "read": set()}

    def step(state, inline, code):                     # register -> "m": by an MFMA, "w": otherwise, since the last fence
        line = " ".join(code)
        touched = [registers(w, "a") for w in code[1:]]
        if inline and tuple(code[:2]) == FENCE:
            return {}
        if not any(touched):
            return state
        if inline and code[0].startswith("v_mfma"):
            seen["mfma"].add(line)
            if any(state.get(r) == "w" for t in touched for r in t):
                found.add(line)
            state.update({r: "m" for r in touched[0]})
        elif inline and code[0].startswith("v_accvgpr_read"):
            seen["read"].add(line)
            if any(state.get(r) for t in touched for r in t):
                found.add(line)
        elif not inline and code[0] in ("v_accvgpr_write_b32", "v_accvgpr_mov_b32") and touched[0]:
            if any(state.get(r) == "m" for t in touched for r in t):
                found.add(line)
            state.update({r: "w" for r in touched[0]})
        else:
            found.add(line)
        return state

    walk(body, step, lambda x, y: {r: "".join(sorted(set(x.get(r, "") + y.get(r, "")))) for r in x.keys() | y.keys()})
    return found, len(seen["mfma"]), len(seen["read"])


def test_nothing_is_spilled(text):
    every = bodies(text, "")
    assert len(every) >= 9
    for name, body in every.items():
        kd = re.search(r"\.amdhsa_kernel %s\n(.*?)\.end_amdhsa_kernel" % re.escape(name), text, re.S)[1]
        assert re.search(r"\.amdhsa_private_segment_fixed_size 0\n", kd) and "scratch_" not in body, name


def test_operands_are_not_fresh_from_the_vector_unit(text):
    made = bodies(text, PINNED)
    assert len(made) == 4                              # two types, walking and not
    for name, body in made.items():
        assert not operands_too_fresh(body), name
        # the check sees an exponent, and a value, that is written just before one
        at = [m.start() for m in re.finditer(r"\t;+#ASMSTART\n\tv_mfma_scale", body)][40]
        mfma = re.match(r".*\n\tv_mfma_scale\S+ \S+ v\[(\d+):\d+\], v\[\d+:\d+\], \S+ v(\d+),", body[at:])
        for r in (mfma[1], mfma[2]):
            planted = body[:at] + f"\tv_mov_b32_e32 v{r}, 0\n\ts_nop 0\n" + body[at:]
            assert len(operands_too_fresh(planted)) == 1
            assert not operands_too_fresh(planted.replace(f"v{r}, 0\n\ts_nop 0\n", f"v{r}, 0\n\ts_nop 1\n"))


def test_fences_stand_between_the_accumulators_and_others(text):
    for name, body in bodies(text, PINNED).items():
        found, mfmas, reads = accumulators_unfenced(body)
        assert not found, f"{name}: {sorted(found)[:5]}"
        assert mfmas >= 128 and reads >= 256
        fence = re.compile(r"\ts_nop 15\n\ts_nop 15\n")
        last = [m for m in fence.finditer(body)][-1]
        assert accumulators_unfenced(body[:last.start()] + "\ts_nop 7\n" + body[last.end():])[0]       # one of them weakened
        at = [m.start() for m in re.finditer(r"\t;+#ASMSTART\n\tv_mfma_scale", body)][70]
        assert accumulators_unfenced(body[:at] + "\tv_accvgpr_read_b32 v0, a3\n" + body[at:])[0]       # a copy of the compiler's


def test_no_one_else_touches_them_in_the_walking_kernel(text):
    made = bodies(text, WALKING)
    assert len(made) == 2
    for name, body in made.items():
        blocks, _ = graph(body)
        others = [" ".join(c) for b in blocks.values() for inline, c in b if not inline and any(registers(w, "a") for w in c[1:])]
        assert not others, f"{name}: {others[:5]}"
        kd = re.search(r"\.amdhsa_kernel %s\n(.*?)\.end_amdhsa_kernel" % re.escape(name), text, re.S)[1]
        free, offset = (int(re.search(r"\.amdhsa_%s (\d+)" % f, kd)[1]) for f in ("next_free_vgpr", "accum_offset"))
        assert free - offset == 256


def memory_operations(block):
    return [(inline, c) for inline, c in block if re.match(r"(global|buffer|flat|scratch)_", c[0])]


FIRST, SECOND, STORES = 13, 4, 32       # direct loads of a block's two parts, stores of a tile: per wave


@pytest.mark.parametrize("shape", [WALKING, STANDING])
def test_waits_count_the_loads_that_are_there(text, shape):
    """In the loop, parts of 13 and 4 loads alternate between the meetings of the waves, nothing else counts, and every meeting
    waits until a part of each kind is under way at most."""
    for name, body in bodies(text, shape).items():
        blocks, follows = graph(body)
        loops = [n for n in blocks if n in follows[n] and sum(c[0].startswith("v_mfma") for _, c in blocks[n]) >= 128]
        assert len(loops) == 1, name
        parts, waits = [0], []
        for inline, c in blocks[loops[0]]:
            if c[0] == "s_barrier":
                parts.append(0)
            elif re.match(r"(global|buffer|flat|scratch)_", c[0]):
                assert inline and c[0].startswith("global_load_lds_dword"), f"{name}: {' '.join(c)}"
                parts[-1] += 1
            elif c[0] == "s_waitcnt" and "vmcnt" in c[1]:
                assert inline
                waits.append(c[1])
        assert len(parts) == 5 and waits == [f"vmcnt({FIRST + SECOND})"] * 4
        assert [parts[0] + parts[4], *parts[1:4]] in ([FIRST, SECOND] * 2, [SECOND, FIRST] * 2), (name, parts)


def test_waits_behind_a_tile_count_its_stores(text):
    """A tile's way out that the walking kernel leaves under way is 32 stores and nothing else that counts; the waits that allow for
    them are those without plus 32."""
    for name, body in bodies(text, WALKING).items():
        blocks, _ = graph(body)
        out = [b for b in blocks.values() if len(memory_operations(b)) == STORES and sum(c[0].startswith("v_accvgpr_read") for _, c in b) == 256]
        assert len(out) == 1, name
        assert all(not inline and c[0] == "global_store_dwordx4" for inline, c in memory_operations(out[0]))
        waits = {c[1] for b in blocks.values() for inline, c in b if inline and c[0] == "s_waitcnt" and "vmcnt" in c[1]}
        plain = {FIRST + 2 * SECOND, FIRST + SECOND}
        # (and STORES itself, before a wave ends: its loads have to be in, its stores may be under way)
        assert waits == {f"vmcnt({n})" for n in plain | {n + STORES for n in plain} | {0, STORES}}, (name, waits)
