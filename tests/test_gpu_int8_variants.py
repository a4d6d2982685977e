"""GPU parity of every kernel and launch that the 8-bit products choose among, each by name: few-row variants, tiles with and
without a split reduction, and the last rows in a launch of their own behind each kind of tiles. The bounds are
test_gpu_int8's, checked on every element."""
import pytest

from test_gpu_int8 import call, check, make

# tokens, features, outputs, activation, workspace (None: as much as the call can use), launches
CASES = [
    (23, 256, 5504, False, None, ["rows 32 x 2 of 16"]),
    (18, 256, 11008, False, None, ["rows 32 x 4 of 16"]),
    (28, 512, 2138, False, 0, ["rows 32 x 1 of 16"]),
    (16, 6016, 8034, False, None, ["rows 16 x 2 of 16"]),
    (84, 2560, 8402, False, None, ["rows 64 x 6 of 16"]),
    (67, 2816, 4436, True, None, ["rows 64 x 6 of 16"]),
    (132, 256, 11008, False, None, ["tiles 64"]),
    (12269, 640, 287, True, None, ["tiles 256+64"]),
    (3209, 5504, 58, False, None, ["tiles 128+64 split"]),
    (512, 11008, 3998, False, None, ["tiles 128 split"]),
    (262, 14208, 7605, False, None, ["tiles 256+64 split"]),
    (2080, 11008, 2048, False, None, ["mid", "rows 32 x 1 of 8"]),
    (1187, 11008, 3546, False, None, ["mid", "rows 64 x 1 of 16"]),
    (715, 8064, 5504, False, None, ["tiles 64", "rows 16 x 1 of 16"]),
    (2052, 5504, 2048, False, None, ["tiles 64", "rows 16 x 1 of 8"]),
    (1394, 4864, 11008, False, None, ["tiles 256+64", "rows 64 x 4 of 16"]),
    (1577, 5504, 10720, False, None, ["tiles 256", "rows 64 x 4 of 16"]),
    (668, 4864, 11008, False, None, ["tiles 128", "rows 32 x 4 of 16"]),
    (1028, 2048, 7480, False, None, ["tiles 128", "rows 16 x 1 of 16"]),
    (1006, 2048, 7266, False, 0, ["tiles 128+64", "rows 64 x 2 of 16"]),
    (1219, 20096, 2048, False, None, ["tiles 128+64 split", "rows 16 x 1 of 8"]),
    (583, 5504, 11008, True, None, ["tiles 256+64", "rows 16 x 2 of 16"]),
    (776, 5504, 10212, True, None, ["tiles 256", "rows 16 x 2 of 16"]),
    (776, 2048, 5219, True, None, ["tiles 128", "rows 16 x 4 of 16"]),
    (472, 5504, 6724, True, None, ["tiles 128+64", "rows 32 x 4 of 16"]),
    (2081, 1792, 2048, True, None, ["tiles 128", "rows 64 x 2 of 8"]),
    (429, 12288, 9760, True, None, ["tiles 128", "rows 64 x 6 of 16"]),
    (967, 25472, 2048, True, None, ["tiles 128+64 split", "rows 16 x 2 of 8"]),
    (1036, 9472, 2048, True, None, ["tiles 64", "rows 16 x 2 of 8"]),
    (132, 10496, 4048, True, 0, ["rows 64 x 4 of 16", "rows 16 x 2 of 16"]),
]


def name(c):
    if c["kernel"] == "rows":
        return f"rows {c['rows']} x {c['weight_tiles']} of {c['weight_rows']}"
    if c["kernel"] != "tiles":
        return c["kernel"]
    main = [str(c["rows"])] if c["main_tiles"] else []
    return "tiles " + "+".join(main + ["64"] * (c["small_tiles"] > 0)) + " split" * (c["splits"] > 1)


def launches(ppas, T, H, N, act, nbytes):
    return [name(c) for c in ppas.gateup_i8_choice(T, H, 2 * N if act else N, act, workspace_bytes=nbytes)]


@pytest.mark.parametrize("T,H,N,act,nbytes,want", CASES)
def test_choice_on_256_compute_units(T, H, N, act, nbytes, want):
    ppas = pytest.importorskip("paper_2608_15171_amd.ppas", reason="libppas.so not built")
    assert launches(ppas, T, H, N, act, nbytes) == want


def test_choice_elsewhere_and_refusals():
    ppas = pytest.importorskip("paper_2608_15171_amd.ppas", reason="libppas.so not built")
    for args in ((5, 100, 7), (5, 128, 7), (5, 192, 7)):        # no whole stages, or a single one
        assert launches(ppas, *args, False, None) == ["general"]
    assert ppas.gateup_i8_choice(5, 256, 7, aligned=False)[0]["kernel"] == "general"
    for bad in ((0, 256, 8, False), (4, 256, 7, True), (-1, 256, 8, False), (4, 0, 8, False)):
        with pytest.raises(ppas.PPASError) as e:
            ppas.gateup_i8_choice(*bad)
        assert e.value.status == ppas.PPAS_EINVAL
    with pytest.raises(ppas.PPASError) as e:
        ppas.gateup_i8_choice(4, 131072, 8)
    assert e.value.status == ppas.PPAS_ERANGE


@pytest.fixture(scope="module")
def lib():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2608_15171_amd import ppas, step
    return ppas, step, torch


@pytest.mark.gpu
@pytest.mark.parametrize("T,H,N,act,nbytes,want", CASES)
def test_every_element(lib, T, H, N, act, nbytes, want):
    print(f"i8 T={T} H={H} N={N} act={act} {want}", flush=True)
    a = make(lib, T, H, 2 * N if act else N, 41)
    check(lib, *a, call(lib, *a, act, True if nbytes is None else nbytes), act, " then ".join(want))


@pytest.mark.gpu
@pytest.mark.parametrize("T,H,N,act,nbytes,want", [c for c in CASES if len(c[5]) == 2][::4])
def test_last_rows_are_those_of_one_launch(lib, T, H, N, act, nbytes, want):
    """The rows of the second launch, alone and without splits."""
    torch = lib[2]
    x, sx, w, sw = make(lib, T, H, 2 * N if act else N, 42)
    whole = call(lib, x, sx, w, sw, act, True if nbytes is None else nbytes)
    n = T % 64
    alone = call(lib, x[-n:], sx[-n:], w, sw, act, 0)
    assert torch.equal(whole[-n:].view(torch.int16), alone.view(torch.int16))
