"""How the attention calls are split over workgroups, as their workspace sizes show it (no GPU)."""
import random

import pytest

from paper_2609_24433_amd import fq


def parts(bytes_, seqs, new, Hq, D):
    """Parts of the tokens: partial results are fp32, D + 2 values a row and part."""
    each = seqs * new * Hq * (D + 2) * 4
    assert bytes_ % each == 0
    return max(1, bytes_ // each)


def cached(seqs, new, kv, Hq, Hk, D):
    return parts(fq.cache_attention_workspace_bytes(seqs * new, Hq, Hk, D, seqs, new, kv), seqs, new, Hq, D)


def cross(B, Sq, Sk, Hq, Hk, D):
    return parts(fq.cross_attention_workspace_bytes(B, Sq, Sk, Hq, Hk, D), B, Sq, Hq, D)


@pytest.mark.parametrize("count", [cached, cross])
@pytest.mark.parametrize("D", [64, 128, 144, 160, 256])
def test_tiles_split_tokens_to_fill_the_card_once(D, count):
    """One workgroup of 128 rows a compute unit where its LDS is all that fits (heads above 128), two below; of 256 rows one;
    256 compute units.  No part shorter than 128 tokens."""
    r = random.Random(D)
    for _ in range(300):
        Hk = r.choice([1, 2, 4, 8])
        Hq = Hk * r.choice([1, 2, 4, 8])
        seqs, new, kv = r.randint(1, 8), r.randint(200, 5000), r.randint(3000, 20000)
        rows = new * (Hq // Hk)
        if seqs * Hk * -(-rows // 16) * -(-kv // 64) <= 1024:
            continue  # streamed
        tile = 256 if 64 < D <= 128 and rows > 128 else 128
        groups, n = seqs * Hk * -(-rows // tile), count(seqs, new, kv, Hq, Hk, D)
        room = 256 if tile == 256 or D > 128 else 512
        assert n == 1 or (groups * n <= room and (n - 1) * 128 < kv), (seqs, new, kv, Hq, Hk)


@pytest.mark.parametrize("want,got", [
    (2, cached(1, 4096, 8190, 8, 2, 128)), (1, cached(1, 4096, 8190, 32, 8, 128)),  # a prompt chunk on 128 and on 512 row tiles
    (1, cached(1, 4096, 4096, 8, 1, 256)), (4, cached(1, 816, 816, 8, 1, 256)),  # head 256: 256 and 51 row tiles
    (14, cached(1, 1, 877, 8, 1, 256)), (14, cached(1, 50, 866, 8, 1, 256)), (32, cached(64, 1, 8192, 32, 8, 128)),
    (13, cross(1, 50, 816, 16, 16, 64)), (1, cross(4, 1031, 4099, 16, 8, 128)),
])
def test_parts_of_the_measured_sizes(want, got):
    assert got == want
