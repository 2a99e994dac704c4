"""The generated K loops of the 8-bit products, stepped on the CPU: which slice every load fetches, where it lands, what the fragments hold when the matrix
instructions use them, and that no load overwrites what a wave may still read (no GPU needed).

The model is one wave of a workgroup whose others run the same text: between two barriers they may be anywhere, so a load and a read of one interval meet in any order."""
import os
import re

import pytest

INC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2510_15620_amd", "csrc", "gemm_q8_kloop.inc")
# rows, columns, waves along both, stages of A and of W: as gemm_q8.hip launches them
TILES = {"256": (256, 256, 2, 2, 2, 3), "224": (224, 256, 2, 2, 2, 3), "192": (192, 256, 2, 2, 2, 3), "160": (160, 256, 2, 2, 3, 3), "128": (128, 256, 2, 2, 3, 3),
         "128x128_2": (128, 128, 2, 2, 2, 2), "128x128_5": (128, 128, 2, 2, 5, 5), "128x64_3": (128, 64, 4, 1, 3, 3), "128x64_6": (128, 64, 4, 1, 6, 6),
         "64x64_5": (64, 64, 2, 2, 5, 5), "32x64_4": (32, 64, 1, 1, 4, 4), "64x32_7": (64, 32, 2, 1, 7, 7), "32x32_9": (32, 32, 2, 2, 9, 9)}


def texts():
    """The instructions of each loop, (name, operands)."""
    out = {}
    for name, body in re.findall(r'#define PRISM_KLOOP_Q8_(\w+) \\\n((?:  ".*" \\\n)+)  ""', open(INC).read()):
        lines = [l.strip() for q in re.findall(r'"(.*)" \\\n', body) for l in q.split("\\n") if l.strip()]
        out[name] = [(l.split(None, 1)[0], [x.strip() for x in l.split(None, 1)[1].split(",")] if " " in l else []) for l in lines]
    return out


TEXTS = texts()


def test_every_tile_has_a_loop():
    assert set(TEXTS) == set(TILES)


class Wave:
    def __init__(self, name, nk, first):
        self.bm, self.bn, wm, wn, sa, sb = TILES[name]
        self.tm, self.tn, nw = self.bm // wm // 16, self.bn // wn // 16, wm * wn
        self.count = {"A": self.bm // 8 // nw, "B": self.bn // 8 // nw}                   # loads of a wave and slice
        self.stage = {"A": self.bm * 128, "B": self.bn * 128}
        self.nk, self.first, self.lds_b = nk, first, sa * self.bm * 128
        # bases beside a multiple of 4 GiB, so that steps to both sides carry
        self.origin = {"A": (5 << 32) - 200, "B": (9 << 32) - nk * 128 + 72}
        self.s = {}
        self.given = {"%[nk]": nk, "%[wr]": nk - first, "%[bk]": (128 - nk * 128) & 0xffffffff, "%[la]": 0, "%[lb]": self.lds_b}
        self.v, self.frag, self.scc, self.m0 = {}, {}, 0, None
        self.landing, self.reading = [], []                       # loads, reads that are under way, in order
        self.landed = {(op, st): [None] * self.count[op] for op, n in (("A", sa), ("B", sb)) for st in range(n)}
        self.seen = {k: list(x) for k, x in self.landed.items()}   # by every wave: landed before the last barrier
        self.loads_here, self.reads_here = set(), set()            # of this interval between barriers
        self.products = {}

    def value(self, x):
        if x in self.given:
            return self.given[x]
        return self.s[x] if x[0] == "s" else int(x, 0) & 0xffffffff

    def load(self, ops):
        off, base = ops
        op, j = off[3].upper(), int(off[4:-1].rstrip("]"))
        at, imm = base.split(" offset:")
        imm = int(imm, 0)
        lo = int(at[2:at.index(":")])
        address = self.s[f"s{lo + 1}"] << 32 | self.s[f"s{lo}"]
        back = address - self.origin[op]
        assert back % 128 == 0 and 0 <= back < self.nk * 128, "a slice outside the row"
        assert imm == j % 4 * 1024, "the lane's offset comes without it"
        to = self.m0 + imm - (self.lds_b if op == "B" else 0)
        st, rest = divmod(to, self.stage[op])
        assert rest == j * 1024 and (op, st) in self.landed, "a load beside its rows"
        slice_ = back // 128
        self.landing.append((op, st, j, slice_))
        if self.seen[op, st][j] != slice_:
            self.seen[op, st][j] = None
        self.loads_here.add((op, st, slice_))

    def read(self, ops):
        dst, rest = ops
        reg, offset = rest.split(" offset:")
        which, k, add = self.v[reg]
        op = "A" if which == "aa" else "B"
        st, at = divmod(add + int(offset, 0), self.stage[op])
        half = max(self.tn // 2, 1)
        block, odd = divmod(at, 2048)
        assert odd == 0 and (op, st) in self.landed and block < (self.tm if op == "A" else half)
        held = set(self.seen[op, st])
        assert len(held) == 1 and None not in held, f"a read of a stage that has not landed: {op} {st} {self.seen[op, st]}"
        slice_ = held.pop()
        self.frag[dst] = None
        self.reading.append((dst, (op, slice_, k, block + (half if which == "ab2" else 0)), (op, st, slice_)))
        self.reads_here.add((op, st, slice_))

    def barrier(self):
        for op, st, slice_ in self.loads_here:
            for o, s, x in self.reads_here:
                assert (o, s) != (op, st) or x == slice_, "a load over a stage that may still be read"
        self.loads_here, self.reads_here = set(), {r[2] for r in self.reading}
        flying = {(op, st, j): x for op, st, j, x in self.landing}
        for k, rows in self.landed.items():
            self.seen[k] = [x if flying.get((*k, j), x) == x else None for j, x in enumerate(rows)]

    def multiply(self, ops):
        r = int(ops[0][2:].split(":")[0]) // 4
        i, j = divmod(r, self.tn)
        b, a = self.frag[ops[1]], self.frag[ops[2]]
        assert a and b, "a fragment that has not arrived"
        assert ops[0] == ops[3] and a == ("A", a[1], a[2], i) and b == ("B", a[1], a[2], j), (a, b, i, j)
        self.products[a[1], a[2], i, j] = self.products.get((a[1], a[2], i, j), 0) + 1

    def wait(self, args):
        for x in args:
            for kind, n in re.findall(r"(vmcnt|lgkmcnt)\((\d+)\)", x):
                if kind == "vmcnt":
                    while len(self.landing) > int(n):
                        op, st, j, slice_ = self.landing.pop(0)
                        self.landed[op, st][j] = slice_
                else:
                    while len(self.reading) > int(n):
                        dst, holds, _ = self.reading.pop(0)
                        self.frag[dst] = holds

    def run(self, text):
        at = {op[:-1]: n for n, (op, _) in enumerate(text) if op.endswith(":")}
        bases = {"%[pa]": self.origin["A"] + self.first * 128, "%[pb]": self.origin["B"] + self.first * 128}
        pc = 0
        while pc < len(text):
            op, a = text[pc]
            pc += 1
            if op.startswith("s_cbranch"):
                if self.scc == (op == "s_cbranch_scc1"):
                    pc = at[a[0]]
            elif op == "s_mov_b64":
                lo = int(a[0][2:a[0].index(":")])
                self.s[f"s{lo}"], self.s[f"s{lo + 1}"] = bases[a[1]] & 0xffffffff, bases[a[1]] >> 32
            elif op == "s_mov_b32":
                self.s[a[0]] = self.value(a[1])
            elif op in ("s_add_u32", "s_addc_u32"):
                x = self.value(a[1]) + self.value(a[2]) + (self.scc if op == "s_addc_u32" else 0)
                self.scc = x >> 32
                if a[0] == "m0":
                    self.m0 = x
                else:
                    self.s[a[0]] = x & 0xffffffff
            elif op == "s_sub_u32":
                x = self.value(a[1]) - self.value(a[2])
                self.scc, self.s[a[0]] = int(x < 0), x & 0xffffffff
            elif op == "s_cselect_b32":
                self.s[a[0]] = self.value(a[1] if self.scc else a[2])
            elif op == "s_ashr_i32":
                x = self.value(a[1])
                self.s[a[0]] = ((x - (x >> 31 << 32)) >> int(a[2])) & 0xffffffff
                self.scc = int(self.s[a[0]] != 0)
            elif op.startswith("s_cmp_"):
                x, y = self.value(a[0]), self.value(a[1])
                self.scc = int({"s_cmp_eq_u32": x == y, "s_cmp_lt_u32": x < y, "s_cmp_ge_u32": x >= y, "s_cmp_gt_u32": x > y}[op])
            elif op == "v_xor_b32":
                assert a[1] in ("0", "64") and a[2][2:-1] in ("aa", "ab", "ab2")
                self.v[a[0]] = (a[2][2:-1], int(a[1]) // 64, 0)
            elif op == "v_add_u32":
                which, k, add = self.v[a[2]]
                self.v[a[0]] = (which, k, add + int(a[1]))
            elif op == "global_load_lds_dwordx4":
                self.load(a)
            elif op == "ds_read_b128":
                self.read(a)
            elif op.startswith("v_mfma_i32_16x16x64_i8"):
                self.multiply(a)
            elif op == "s_waitcnt":
                self.wait(a)
            elif op == "s_barrier":
                self.barrier()
            else:
                assert op in ("s_nop", "v_accvgpr_write_b32") or op.endswith(":"), op
        self.barrier()


@pytest.mark.parametrize("name", TILES)
def test_a_loop_that_begins_anywhere(name):
    """Rows of 1 to 33 slices, the loop beginning at each of them (of the longest at some): every slice is multiplied once, no load leaves the rows, nothing is read before it has landed or
    while it may be overwritten, and nothing is under way at the end."""
    for nk in (1, 2, 3, 4, 5, 6, 7, 8, 11, 33):
        for first in range(nk) if nk < 9 else (0, 1, 5, nk - 2, nk - 1):
            w = Wave(name, nk, first)
            w.run(TEXTS[name])
            assert not w.landing and not w.reading
            assert w.products == {(s, k, i, j): 1 for s in range(nk) for k in range(2) for i in range(w.tm) for j in range(w.tn)}, (nk, first)


def test_the_model_notices_mistakes():
    """Loops with one instruction changed: a missing wait, a barrier's counter too high, a step that does not come round."""
    def changed(name, old, new, nth=0):
        text, n = [], -1
        for op, a in TEXTS[name]:
            n += (op, a) == old
            text.append(new if (op, a) == old and n == nth else (op, a))
        assert n >= nth
        return text
    nop = ("s_nop", ["0"])
    wait = next(x for x in TEXTS["256"] if x[0] == "s_waitcnt" and "vmcnt(8)" in x[1][0])
    for name, old, new, nth in (("256", wait, ("s_waitcnt", ["lgkmcnt(0)"]), 1), ("256", ("s_barrier", []), nop, 1), ("64x64_5", ("s_barrier", []), nop, 2),
                                ("192", ("s_cselect_b32", ["s27", "%[bk]", "128"]), ("s_cselect_b32", ["s27", "128", "128"]), 4),
                                ("32x32_9", ("s_cselect_b32", ["s25", "%[bk]", "128"]), ("s_cselect_b32", ["s25", "128", "128"]), 3)):
        with pytest.raises(AssertionError):
            for first in range(11):
                w = Wave(name, 11, first)
                w.run(changed(name, old, new, nth))
                assert w.products == {(s, k, i, j): 1 for s in range(11) for k in range(2) for i in range(w.tm) for j in range(w.tn)}
