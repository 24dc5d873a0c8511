"""The attention's workspace is sized by the parts that can be, not by the requests (no GPU)."""
from paper_2603_05232_amd import binding


def test_room_for_parts_follows_the_chip():
    size = binding.kv_attention_workspace_bytes
    part = 8 * 16 * (8 + 4 * 128)                                  # eight heads of keys, sixteen columns: maximum and sum, values
    for B in (1, 2, 64, 1000, 4096):
        n = size(B, 32, 8, 128)
        # a request that is divided takes more than a workgroup's share of the blocks, so that there are at most twice as many parts as workgroups
        assert 8 * B + (64 + min(B, 64) + 2) * part <= n + 16 and n <= 8 * B + 16 + 140 * part, B
    assert size(4096, 32, 8, 128) < 10 << 20 and size(4096, 1024, 8, 256) < 250 << 20
