"""Sequence operators on the GPU at the sizes where a call is cut in another
way: workgroups that go through many series or tiles, rows whose tiles meet
through memory (more than one published state among them), one large tile,
chunks of wide and of odd groups.  Against the 64-bit oracle, within its bounds."""
import pytest

from test_gpu_sequence import check_norm, check_rec, env  # noqa: F401

pytestmark = pytest.mark.gpu


# n, L, C: rows are n times blocks of 64 channels (16 bits) or 32 (fp32)
@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("n,L,C,dtype", [
    (1, 9000, 66, "bfloat16"), (2, 8500, 33, "float32"),    # tiles that meet, three published states
    (2, 4224, 70, "float16"),                               # 33 tiles: the last one starts from a state
    (1, 20001, 3, "bfloat16"), (1, 33000, 1, "float16"),    # few channels: tiles of many runs
    (130, 300, 260, "bfloat16"), (130, 600, 140, "float32"),   # loops over three tiles, and five
    (70, 1100, 256, "float32"),                             # long fp32 rows, split though they are many
    (100, 1030, 384, "float16"),                            # 600 rows: a badly filled last round
    (130, 250, 260, "float16"),                             # gated backward: split in two; else one tile or two
    (3, 250, 64, "bfloat16"), (3, 500, 30, "float32"),      # one tile of 16 wavefronts
    (600, 150, 64, "bfloat16"), (600, 140, 31, "float32"),  # one tile of 10 and of 5
    (2000, 3, 40, "bfloat16")])
def test_recurrence_cuts(env, n, L, C, dtype, gate):  # noqa: F811
    check_rec(*env, n, L, C, dtype, gate)


@pytest.mark.parametrize("n,L,C,dtype", [(6, 8500, 66, "bfloat16"), (140, 600, 130, "float32"),
                                         (40, 1030, 70, "float16")])
def test_recurrence_cuts_ragged(env, n, L, C, dtype):  # noqa: F811
    check_rec(*env, n, L, C, dtype, True, with_lengths=True, packed=True)


@pytest.mark.parametrize("n,L,C,G", [
    (2, 3000, 2000, 1), (2, 700, 2042, 1), (2, 300, 4100, 2),   # chunks of the widest slabs, and of parts
    (20, 34, 5512, 106),                                         # held, columns in two groups
    (2, 1982, 1159, 19),                                         # chunks of odd groups
    (3, 5000, 24, 3), (2, 9000, 5, 5),                           # many chunks, of narrow rows too
    (3000, 1, 200, 2), (5000, 3, 64, 4), (900, 2, 1000, 1),      # many series in turn
    (1300, 40, 256, 16), (600, 100, 66, 2), (1100, 5, 7, 7)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_group_norm_cuts(env, n, L, C, G, dtype):  # noqa: F811
    check_norm(*env, n, L, C, G, dtype, "gelu", False)


@pytest.mark.parametrize("act", ["relu", "silu"])
@pytest.mark.parametrize("n,L,C,G", [(900, 20, 48, 6), (5, 2500, 99, 3), (40, 900, 64, 2)])
def test_group_norm_cuts_ragged(env, n, L, C, G, act):  # noqa: F811
    check_norm(*env, n, L, C, G, "float16", act, True)


# The slab's columns do not divide the workgroup (3 in 64 threads: 21 rows and a
# thread left over), and the series end with a whole pass over the rows: the
# threads left over have no step of their own to load.
@pytest.mark.parametrize("n,L,C,G", [
    (3, 21, 24, 3), (3, 84, 24, 3), (40, 85, 24, 3), (2, 340, 24, 3),   # held, by 64 and by 256 threads
    (3, 28, 66, 2), (3, 112, 66, 2),                                    # columns in two groups
    (2, 1360, 24, 3), (2, 5440, 24, 3), (2, 4480, 66, 2)])              # held by more threads, chunks
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_group_norm_whole_passes_with_threads_left_over(env, n, L, C, G, dtype):  # noqa: F811
    check_norm(*env, n, L, C, G, dtype, "silu", False)


@pytest.mark.parametrize("n,L,C,G", [(2, 20000, 33, 3), (3, 6000, 99, 3), (1, 9000, 331, 1)])
def test_chunks_in_place(env, n, L, C, G):  # noqa: F811
    """Columns that share channels with their neighbours, over the inputs."""
    torch, seq = env
    x, dy = (torch.randn(n, L, C, device="cuda").to(torch.bfloat16) for _ in range(2))
    y, mean, rstd = seq.group_norm(x, G, activation="silu")
    dx = seq.group_norm_backward(dy, x, G, mean, rstd, activation="silu")[0]
    a = x.clone()
    assert torch.equal(seq.group_norm(a, G, activation="silu", out=a)[0], y)
    for k in range(2):
        a = [x.clone(), dy.clone()]
        assert torch.equal(seq.group_norm_backward(a[1], a[0], G, mean, rstd, activation="silu", out=a[k])[0], dx)


@pytest.mark.parametrize("dtype", ["float32", "float16"])
def test_group_norm_many_long_series(env, dtype):  # noqa: F811
    """More than 1,024 slabs of more steps than 512 threads hold: the largest
    workgroup of the backward pass, several series in turn."""
    check_norm(*env, 1100, 530, 32 if dtype == "float32" else 64, 2, dtype, "silu", False)


def test_largest_workgroup_in_a_graph(env):  # noqa: F811
    """Its shared memory is asked for at the launch, also while capturing."""
    torch, seq = env
    x, dy = (torch.randn(1100, 530, 64, device="cuda").half() for _ in range(2))
    _, mean, rstd = seq.group_norm(x, 2)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = seq.group_norm_backward(dy, x, 2, mean, rstd, activation="silu")
    for _ in range(3):
        dy.normal_()
        want = seq.group_norm_backward(dy, x, 2, mean, rstd, activation="silu")
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
