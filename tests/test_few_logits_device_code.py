"""Host-only: the kernels of topk.hip and distill.hip hold what the kernels of flce.hip hold (the tests of those look at that source
alone): no spilled register and no scratch memory, the numbered accumulation registers used by the loop's assembly alone, the wait
states around it."""
import functools
import re
import subprocess
import tempfile

import pytest

import device_asm as A
import test_accumulation_registers as R
import test_wait_states as S
from paper_2511_17599_amd import build as BLD

SOURCES = [s for s in BLD.SOURCES if s != BLD.SRC]


@functools.lru_cache(None)
def compiled(src):
    with tempfile.TemporaryDirectory() as tmp:
        out = f"{tmp}/out.s"
        flags = [f for f in BLD.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
        res = subprocess.run([BLD.hipcc_path(), *flags, "-Rpass-analysis=kernel-resource-usage", "-S", "--offload-device-only", src,
                              "-o", out], capture_output=True, text=True)
        assert res.returncode == 0, res.stderr[-2000:]
        with open(out) as f:
            return A.parse(f.read()), res.stderr


def test_every_source_is_looked_at():
    assert len(SOURCES) == 2 and all(s.endswith(".hip") for s in SOURCES)


@pytest.mark.parametrize("src", SOURCES)
def test_no_spills(src):
    kernels, remarks = compiled(src)
    seen = 0
    for block in re.split(r"remark: [^\n]*Function Name: ", remarks)[1:]:
        name = block.split()[0]
        for pat in (r"VGPRs Spill: (\d+)", r"SGPRs Spill: (\d+)", r"ScratchSize \[bytes/lane\]: (\d+)"):
            assert int(re.search(pat, block).group(1)) == 0, (name, pat)
        seen += 1
        if "FastLoop" in name and ("logit_tiles" in name or "recompute" in name):
            assert int(re.search(r"AGPRs: (\d+)", block).group(1)) == 256, name
    assert seen == len(kernels) >= 20


@pytest.mark.parametrize("src", SOURCES)
def test_registers_of_the_loop(src):
    kernels, _ = compiled(src)
    loops = {n: k for n, k in kernels.items() if R.numbered(k)}
    # two edges, two hidden-size forms: the forward's tiles with and without the copy of H, in topk.hip with floors for whole K steps, in
    # distill.hip the two recompute steps too
    assert len(loops) == (10 if src.endswith("topk.hip") else 16)
    for n, k in loops.items():
        assert not list(R.misuse(k))[:3], n
    for n, k in kernels.items():
        assert not list(R.stray_m0(k))[:3], n


@pytest.mark.parametrize("src", SOURCES)
def test_wait_states(src):
    kernels, _ = compiled(src)
    requests = sum(x.in_asm and x.op.startswith("buffer_") for insts, _ in kernels.values() for x in insts)
    assert requests > 300
    for n, k in kernels.items():
        bad = list(S.too_early(k)) + list(S.early_operands(k)) + list(S.early_sums(k))
        assert not bad, (n, bad[:2])
