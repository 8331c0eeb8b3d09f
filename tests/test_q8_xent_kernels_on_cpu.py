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


def test_launches_fit_a_grid(tmp_path):
    """At the ends of the sizes, as far as a card holds them: no launch of 2^32 work items."""
    exe = xent_on_cpu.compile_calls(str(tmp_path))
    some = ["xent 2097088 2 1", "xent 2097088 131072 8", "xent 70 2000000000 8",
            "xent 64 2000000000 16", "xent 1 2147483639 16", "xent 17 2000000 131071",
            "xent_bwd 2097088 131072 8 0 0", "xent_bwd 2097088 200000 8 1 1",
            "xent_bwd 65 2000000 64 0 0", "xent_bwd 1 1000000000 16 0 0",
            "xent_bwd 16 100000000 2000 0 0", "xent_bwd 64 100000000 1024 1 0",
            "xent_bwd 70 90000000 8 0 1", "xent_bwd 1000000 1 16384 0 0"]
    r = subprocess.run([exe, "note"], input="\n".join(some) + "\n", capture_output=True,
                       text=True, timeout=300)
    lines = r.stdout.splitlines()
    assert r.returncode == 0 and len(lines) == len(some)
    for call, line in zip(some, lines):
        assert line.split()[0] == "0" and "too large" not in line, (call, line[:80])
