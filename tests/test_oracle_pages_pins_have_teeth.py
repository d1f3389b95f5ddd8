"""Do the pins of the cache in pages bite? As test_oracle_pins_have_teeth: one plausible mistake at a time in a copy of the oracle's
source, and a pin has to fail. CPU only."""
import os
import types

import pytest

from test_oracle_pins_have_teeth import ROOT, _first_failure

SRC = open(os.path.join(ROOT, "oracle", "pages_oracle.py")).read()

MUTANTS = [
    ("scale: the largest value reaches 6, not 7", "top > 7 * math.ldexp", "top > 6 * math.ldexp"),
    ("scale of rows: the largest value reaches 6, not 7", "math.frexp(top / 7)", "math.frexp(top / 6)"),
    ("scale: a power of two too large where 7 is met", "k = e - 1 if m == 0.5 else e", "k = e"),
    ("scale: no lower limit", "min(max(k + 127, 2), 252)", "min(k + 127, 252)"),
    ("code: ties to the smaller magnitude", "if i % 2 == 0))", "if True))"),
    ("code of rows: ties to the smaller magnitude", "& (first % 2 == 1), first + 1, first)", "& (first % 2 == 2), first + 1, first)"),
    ("code: the sign is lost", "+ 8 * np.signbit(y)", "+ 0 * np.signbit(y)"),
    ("pack: the even channel in the high half", "return codes[:, ::2] | codes[:, 1::2] << 4, es", "return codes[:, 1::2] | codes[:, ::2] << 4, es"),
    ("a block that is not finite stands for numbers", "np.where(e == 255, math.nan,", "np.where(e == 256, math.nan,"),
    ("append: shared pages are written", "copies = more > 0 and n % P != 0 and", "copies = False and"),
    ("append: a shared page is not copied", "if len(k) and n % P and self.table[g, n // P] in shared:", "if False:"),
    ("append: the copy misses its last row", "for r in range(n % P):", "for r in range(n % P - 1):"),
    ("append: an item in want does not count for the next", "asked += sum(needs)", "asked = sum(needs)"),
    ("append: a sequence named twice is served twice", "or x in seqs[:i]", ""),
    ("append: a table row takes one page more", "> self.max_pages for", "> self.max_pages + 1 for"),
    ("search: not behind the page taken last", "self.search = (pages[-1] + 1) % self.n_pages", "self.search = pages[-1]"),
    ("fork: old owners are not counted off", "self.refs[table[g, j]] -= 1", "pass"),
    ("fork: rows that go are those of the head before the fork", "int(lengths[parent * H + h]) - max", "int(lengths[g]) - max"),
    ("keep: pages stay whatever is kept of them", "== list(range(same * P, (same + 1) * P)):", "!= []:"),
    ("keep: more rows than there are", "if b >= n:", "if b > n + 100:"),
    ("keep: old pages are not given back", "back += [int(p) for p in old[same:pages_of(n, P)]]", "pass"),
    ("read: rows begin at 0", "for r in range(f, f + n):", "for r in range(0, n):"),
    ("attend: the last row is missing", "reshape(len(pages) * P, (b - a) // P)[:n]", "reshape(len(pages) * P, (b - a) // P)[:n - 1]"),
    ("attend: query heads interleaved", "for j in range(h * G, (h + 1) * G):", "for j in range(h, q.shape[1], self.H):"),
    ("attend: log-sum-exp without the maximum", "lse[x, j] = m + math.log", "lse[x, j] = math.log"),
]


@pytest.mark.parametrize("name,old,new", MUTANTS, ids=[m[0] for m in MUTANTS])
def test_planted_mistake_is_caught(name, old, new):
    assert SRC.count(old) == 1, (name, SRC.count(old))
    mutant = types.ModuleType("pages_oracle_mutant")
    exec(compile(SRC.replace(old, new), "pages_oracle_mutant.py", "exec"), mutant.__dict__)
    assert _first_failure("test_oracle_pages", mutant), f"no pin notices: {name}"


def test_the_unmodified_copy_passes_every_pin():
    clean = types.ModuleType("pages_oracle_copy")
    exec(compile(SRC, "pages_oracle_copy.py", "exec"), clean.__dict__)
    assert _first_failure("test_oracle_pages", clean) is None
