"""What a Q8Mlp keeps and what its layers share, counted on the CPU."""
import pytest
import torch

from paper_2607_21224_amd.layer import Q8Mlp


def storages(*objects):
    """{address: bytes} of all tensors that belong to the objects."""
    found = {}

    def add(v):
        if isinstance(v, torch.Tensor):
            s = v.untyped_storage()
            found[s.data_ptr()] = s.nbytes()
        elif isinstance(v, (list, tuple)):
            for x in v:
                add(x)

    for o in objects:
        for v in vars(o).values():
            add(v)
    return found


@pytest.mark.parametrize("kind", ["gelu", "swiglu"])
@pytest.mark.parametrize("act_dt,e", [("bf16", 2), ("f32", 4)])
def test_layers_that_share_a_scratch(kind, act_dt, e):
    D, F, T = 384, 1536, 1024
    mlp = Q8Mlp(D, F, kind, act_dt=act_dt)
    scratch = mlp.scratch(T, device="cpu")
    layers = [mlp.saved(T, device="cpu", scratch=scratch) for _ in range(3)]
    nz = 2 if kind == "swiglu" else 1
    # a layer's own: n, z and a in a byte each, scales, rstd, h, y and dx, 8-bit weights
    own = T * (D + nz * F + F + 4 * (3 + nz) + 3 * e * D) + (nz + 1) * F * D + 4 * (nz * F + D)
    shared = T * e * (nz * F + F + D) + mlp.workspace_bytes(T)
    assert sum(storages(scratch).values()) == shared
    assert sum(storages(*layers).values()) == 3 * own + shared
    # without one, each has its own
    alone = [mlp.saved(T, device="cpu") for _ in range(2)]
    assert sum(storages(*alone).values()) == 2 * (own + shared)


def test_bytes_a_token_as_the_module_gives_them():
    T = 1024
    mlp = Q8Mlp(384, 1536)
    s, sc = mlp.saved(T, device="cpu"), mlp.scratch(T, device="cpu")
    per = lambda *ts: sum(t.untyped_storage().nbytes() for t in ts) // T  # noqa: E731
    assert per(s.n, s.cg, s.a) == 3456 and per(s.n_scale, s.g_scale, s.a_scale, s.rstd) == 16
    assert per(s.h) == per(s.y) == per(s.dx) == 768
    assert per(sc.z_all, sc.da, sc.dn) == 6912


def test_a_scratch_of_another_layer():
    mlp = Q8Mlp(64, 128)
    for other, T in ((Q8Mlp(64, 136), 5), (Q8Mlp(64, 128, "swiglu"), 5),
                     (Q8Mlp(64, 128, act_dt="f32"), 5), (mlp, 6)):
        with pytest.raises(ValueError, match="scratch"):
            mlp.saved(5, device="cpu", scratch=other.scratch(T, device="cpu"))
