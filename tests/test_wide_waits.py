"""Waits for memory among the matrix instructions of wide layers' products: those written in assembler are counted, and the compiler adds none of its own, alone or in one
instruction with a wait for LDS (it would wait for the fetches of the next slabs with it)."""
from test_wide_assembly import assembly, kernels  # noqa: F401


def compilers_waits(lines):
    """Waits for loads and stores in blocks of at least four matrix instructions that no assembler text holds, and how many texts anywhere hold one."""
    own, by_hand_waits, block, by_hand, products = [], 0, [], False, 0
    for line in lines + [".LBB"]:
        if line.startswith(".LBB"):
            if products >= 4:
                own += [x for x, hand in block if not hand]
            by_hand_waits += sum(hand for _, hand in block)
            block, products = [], 0
        line = line.strip()
        if line.startswith(";;#ASM"):
            by_hand = line == ";;#ASMSTART"
        line = line.split(";")[0].strip()
        products += line.startswith("v_mfma")
        if line.startswith("s_waitcnt") and "vmcnt" in line:
            block.append((line, by_hand))
    return own, by_hand_waits


def test_planted_waits_are_seen():
    product = ["v_mfma_f32_32x32x16_bf16 a[0:15], v[0:3], v[4:7], a[0:15]"] * 4
    for wait in ("s_waitcnt vmcnt(0)", "s_waitcnt vmcnt(0) lgkmcnt(0)", "s_waitcnt vmcnt(3) lgkmcnt(1)"):
        assert compilers_waits([".LBB0_1:"] + product + ["\t" + wait] + product) == ([wait], 0)
        assert compilers_waits([".LBB0_1:"] + product + ["\t;;#ASMSTART", "\t" + wait, "\ts_barrier", "\t;;#ASMEND"] + product) == ([], 1)
    assert compilers_waits([".LBB0_1:"] + product + ["s_waitcnt lgkmcnt(0)"] + product) == ([], 0)
    assert compilers_waits([".LBB0_1:", "s_waitcnt vmcnt(0)", ".LBB0_2:"] + product) == ([], 0)


def test_products(assembly):  # noqa: F811
    seen = 0
    for name, lines in kernels(assembly):
        own, by_hand = compilers_waits(lines)
        assert not own, (name, own)
        assert by_hand >= 1, name
        seen += 1
    assert seen >= 6


def test_every_exchange_is_marked(assembly):  # noqa: F811
    """Lanes of a wavefront exchange results through LDS: the compiler is told so at each exchange, before the reads and before the next writes, and keeps the order that LDS
    then keeps as well (a lane's own addresses alone would let it move the one past the other)."""
    seen = 0
    for name, lines in kernels(assembly):
        marks = sum("wave barrier" in x for x in lines)
        assert marks >= 4 and marks % 2 == 0, (name, marks)
        seen += 1
    assert seen >= 6
