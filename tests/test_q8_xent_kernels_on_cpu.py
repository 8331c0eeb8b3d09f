"""Which kernels the loss takes at the sizes of xent_sizes.py, asked of its launchers compiled
for the host: each that is compiled for it runs there, so that the GPU tests compare it
and none is kept that no call reaches."""
import re
import subprocess

import pytest

import on_cpu
import xent_on_cpu
import xent_sizes

pytestmark = pytest.mark.skipif(not on_cpu.available(), reason="needs ROCm's clang")


def kernels_of(exe):
    """{address: name} of the kernels in the program."""
    r = subprocess.run(["nm", "-C", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    out = {}
    for line in r.stdout.splitlines():
        address, kind, name = line.split(" ", 2) if line[:1] != " " else ("", "", "")
        name = name.replace("(anonymous namespace)::", "")
        m = re.match(r"(?:void )?cpdp::q8::([a-z0-9_]+_kernel)(<[^()]*>)?\([^{]*\)$", name)
        if kind in ("t", "T", "w", "W") and m and not m[1].startswith("launch"):
            out[address.lstrip("0")] = m[1] + (m[2] or "")
    return out


def calls():
    for s in xent_sizes.SMALL + xent_sizes.MIDDLE + xent_sizes.LARGE:
        yield ("xent", *s)
        for t in xent_sizes.TYPES:
            yield ("xent_bwd", *s, *t)
    # (those that test_gpu_q8_xent.py makes with one gradient)
    for s in xent_sizes.ONE:
        for t in xent_sizes.ALONE:
            yield ("xent_bwd", *s, *t)


def test_every_kernel_is_reached(tmp_path):
    """All of the loss' own kernels, and those that make its products, which its unit has."""
    exe = xent_on_cpu.compile_calls(str(tmp_path))
    names = kernels_of(exe)
    own = subprocess.run(["nm", "-C", str(tmp_path / "q8_xent.hip.o")], capture_output=True,
                         text=True).stdout.replace("(anonymous namespace)::", "")
    wanted = {n for n in names.values() if n.startswith("xent_")}
    products = {m[1] for m in re.finditer(r"cpdp::q8::((?:gemm|join)_kernel<[^()]*>)\(", own)}
    assert len(wanted) > 30 and len(products) >= 8
    taken = set()
    some = list(calls())
    for call, (status, kernels) in zip(
            some, on_cpu.run(exe, "note", [" ".join(map(str, c)) for c in some])):
        assert status == 0, call
        for k in kernels:
            # (other units have products of the same name: up to 64 tokens it is theirs)
            if names[k].startswith("xent_") or call[1] > 64:
                taken.add(names[k])
    left = sorted((wanted | products) - taken)
    assert not left, "\n".join(left)
