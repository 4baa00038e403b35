"""A cache in 4 bits takes only a ring, table and lengths of its own sizes, shared or its own: the kernels would read and
write beyond smaller ones."""
import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def dar():
    from paper_2606_18587_gb300 import dar
    try:
        dar.load_library()
    except RuntimeError:
        from paper_2606_18587_gb300 import build
        build.build()
    return dar


def test_shares(dar):
    c = dar.DarCache(3, 2, 16, 8, 4, 20, dtype=torch.float32, device="cpu")
    for c4 in (dar.DarCacheQ4.beside(c), dar.DarCacheQ4(3, 2, 16, 8, 4, dtype=torch.float32, share=c),
               dar.DarCacheQ4.beside(c, num_pages=5)):
        assert c4.win_k is c.win_k and c4.block_table is c.block_table and c4.seq_lens is c.seq_lens
        assert c4.pool.device == c.win_k.device


@pytest.mark.parametrize("kw", [dict(B=4), dict(Hkv=3), dict(w=9), dict(max_pages_per_seq=5), dict(max_pages_per_seq=3),
                                dict(dtype=torch.bfloat16), dict(block_table=torch.zeros((3, 4), dtype=torch.int32))])
def test_refuses_other_sizes(dar, kw):
    c = dar.DarCache(3, 2, 16, 8, 4, dtype=torch.float32, device="cpu")
    args = dict(B=3, Hkv=2, d_down=16, w=8, max_pages_per_seq=4, dtype=torch.float32, share=c, device="cpu")
    dar.DarCacheQ4(**args)
    with pytest.raises(ValueError):
        dar.DarCacheQ4(**{**args, **kw})


def test_refuses_a_short_block_table(dar):
    """Every sequence has max_pages_per_seq entries, which kernels read."""
    for shape in ((3, 3), (2, 4), (0,)):
        with pytest.raises(ValueError):
            dar.DarCacheQ4(3, 2, 16, 8, 4, block_table=torch.zeros(shape, dtype=torch.int32), device="cpu")
    dar.DarCacheQ4(3, 2, 16, 8, 4, block_table=torch.zeros((3, 4), dtype=torch.int32), device="cpu")
    dar.DarCacheQ4(3, 2, 16, 8, 0, block_table=torch.zeros((3, 0), dtype=torch.int32), num_pages=1, device="cpu")
    dar.DarCacheQ4(0, 2, 16, 8, 4, device="cpu")
